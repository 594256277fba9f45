"""Eviction from the paged cache: which tokens stay, and what the new pages hold."""
import pytest
import torch

import paper_2504_18547_b200 as vt
import paged_util as pu

pytestmark = pytest.mark.gpu

BF16, F16, I8 = torch.bfloat16, torch.float16, torch.int8


def plain_kept(w, length, budget, sinks, recent):
    """Indices kept of `length` weights."""
    if length <= budget:
        return list(range(length))
    free = range(sinks, length - recent)
    best = sorted(free, key=lambda i: (-float(w[i]), i))[:budget - sinks - recent]
    return sorted(list(range(sinks)) + best + list(range(length - recent, length)))


def run(seed, dim, places, ctype, heads, lengths, budget, sinks, recent, weigh=None, layout="hpd"):
    g = torch.Generator().manual_seed(seed)
    need, per = sum(-(-n // places) for n in lengths), -(-budget // places)
    pages = need + per * len(lengths) + 1
    cache = pu.random_cache(g, pages, heads, places, dim, ctype, layout=layout)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table, at = torch.full((len(lengths), max(-(-max(lengths) // places), 1)), -1, dtype=torch.int32), 0
    for b, n in enumerate(lengths):
        table[b, :-(-n // places)] = order[at:at + -(-n // places)]
        at += -(-n // places)
    new_table = order[at:at + per * len(lengths)].view(len(lengths), per)
    weights = (weigh or (lambda s: torch.rand(s, generator=g)))((pages, heads, places))
    gpu, w = pu.to_gpu(cache), weights.cuda()
    batch = vt.CacheBatch(table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), None, 0, max(max(lengths), 1))
    kept, counts = vt.vitint_cache_evict(gpu, batch, w, budget, new_table.cuda(), sinks=sinks, recent=recent)
    assert vt.vitint_device_status() == 0
    assert counts.tolist() == [min(n, budget) for n in lengths]
    want = {n: getattr(cache, n).clone() for n in ("k", "v", "k_steps", "v_steps") if getattr(cache, n) is not None} | {"weights": weights.clone()}
    for b, n in enumerate(lengths):
        for h in range(heads):
            j = torch.arange(n)
            mine = weights[table[b, j // places].long(), h, j % places]
            keep = plain_kept(mine, n, budget, sinks, recent)
            assert kept[b, h].tolist() == keep + [-1] * (budget - len(keep)), (b, h)
            to, src = torch.arange(len(keep)), torch.tensor(keep, dtype=torch.long)
            for name, x in want.items():
                old = getattr(cache, name) if name != "weights" else weights
                x[new_table[b, to // places].long(), h, to % places] = old[table[b, src // places].long(), h, src % places]
    for name, x in want.items():
        assert torch.equal((w if name == "weights" else getattr(gpu, name)).cpu(), x), name


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("ctype", [BF16, F16, I8])
@pytest.mark.parametrize("places", [16, 128])
def test_batches(places, ctype, dim):
    run(1, dim, places, ctype, 3, [100, 1, 0, 333, 57, 58], 57, 4, 20)


@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (50, 25, 25), (50, 50, 0), (50, 0, 49), (499, 0, 0), (500, 3, 3), (600, 0, 0)])
def test_budgets(budget, sinks, recent):
    run(2, 64, 16, BF16, 2, [500, 499], budget, sinks, recent)


def test_long():
    run(3, 64, 64, I8, 1, [70001], 9000, 4, 1000)
    run(4, 64, 32, BF16, 2, [5000, 20000], 1111, 0, 0, layout="phd")


def test_equal_weights_go_to_the_lowest_index():
    run(5, 64, 16, BF16, 2, [1000, 4097], 300, 2, 10, weigh=lambda s: torch.zeros(s))
    g = torch.Generator().manual_seed(9)
    run(6, 64, 16, BF16, 2, [1000, 4097], 300, 2, 10, weigh=lambda s: torch.randint(0, 3, s, generator=g).float())
    run(7, 64, 16, BF16, 1, [400], 200, 0, 0, weigh=lambda s: torch.where(torch.rand(s, generator=g) < 0.5, 0.0, -0.0))


def test_weights_of_any_size():
    g = torch.Generator().manual_seed(10)
    run(8, 64, 16, BF16, 2, [2000], 700, 0, 0, weigh=lambda s: torch.randn(s, generator=g) * 10.0 ** torch.randint(-30, 30, s, generator=g))
    run(9, 64, 16, BF16, 2, [2000], 700, 0, 0, weigh=lambda s: 1.0 + torch.randint(0, 50, s, generator=g) * 2.0 ** -23)
    def infinite(s):
        w = torch.rand(s, generator=g)
        w[w > 0.9] = float("inf")
        return w
    run(10, 64, 16, BF16, 1, [900], 30, 0, 0, weigh=infinite)


def test_bad_pages_are_reported():
    g = torch.Generator().manual_seed(11)
    cache = pu.to_gpu(pu.random_cache(g, 20, 2, 16, 64, BF16))
    w = torch.rand((20, 2, 16), generator=g).cuda()
    table = torch.arange(10, dtype=torch.int32)[None].cuda()
    table[0, 4] = 1 << 20
    new = torch.tensor([[12, -3]], dtype=torch.int32).cuda()
    batch = vt.CacheBatch(table, torch.tensor([160], dtype=torch.int32).cuda(), None, 0, 160)
    before = cache.k[:12].clone()
    vt.vitint_cache_evict(cache, batch, w, 32, new)
    assert vt.vitint_device_status() == -1 and torch.equal(cache.k[:12], before)


def test_parts_that_shared_memory_does_not_hold():
    """More than 40,960 tokens a block: 75 sequence-heads have a block each, and what it does not hold is read anew in every pass."""
    g = torch.Generator().manual_seed(12)
    run(12, 64, 128, I8, 15, [45000, 41500, 7, 0, 300], 300, 4, 100, weigh=lambda s: torch.randint(0, 400, s, generator=g).float())
    run(13, 64, 128, I8, 15, [100, 41111, 40960, 40961, 1], 35000, 0, 0)


@pytest.mark.parametrize("heads,lengths", [(1, [8191]), (1, [8192]), (1, [16383]), (1, [20000]), (9, [8200]), (18, [9001]), (37, [6000]), (74, [4097])])
def test_clusters_of_every_size(heads, lengths):
    g = torch.Generator().manual_seed(13)
    run(14, 64, 64, I8, heads, lengths, 1500, 3, 200, weigh=lambda s: torch.randint(0, 5000, s, generator=g) / 64)

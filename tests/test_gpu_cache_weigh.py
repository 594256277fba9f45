"""Attention weights accumulated over the paged cache against their definition in 64 bits."""
import math

import pytest
import torch

import paper_2504_18547_b200 as vt
import paged_util as pu

pytestmark = pytest.mark.gpu

BF16, F16, I8 = torch.bfloat16, torch.float16, torch.int8


def weights64(q, lse, cache, table, lengths, starts, scale, causal, window, before):
    """(weights, tolerance, places of the batch's tokens).  The tolerance of an fp32 evaluation: a score is off by (d + 4) 2^-24 scale sum |q||k|
    (products and their sum) and 2^-23 (|s| + |lse|) (scale, logarithm's base, the subtraction), its exponential relatively by that and
    2^-21, a sum of N positive terms relatively by N 2^-24, the last addition by half a step."""
    pages, heads, places, d = cache.k.shape
    group = q.shape[1] // heads
    out, tol = before.double().clone(), torch.zeros(before.shape, dtype=torch.float64)
    mine = torch.zeros(before.shape, dtype=torch.bool)
    for b, length in enumerate(lengths):
        if not length:
            continue
        first, new = int(starts[b]), int(starts[b + 1]) - int(starts[b])
        see = pu.visible(length, new, causal, window)
        j = torch.arange(length)
        page = table[b, j // places].long()
        for h in range(heads):
            k = pu.gathered(cache, table[b], length, h, "k")
            total, off = torch.zeros(length, dtype=torch.float64), torch.zeros(length, dtype=torch.float64)
            for x in range(h * group, (h + 1) * group):
                qq, z = q[first:first + new, x].double(), lse[first:first + new, x].double()[:, None]
                s = (qq @ k.T) * scale
                ds = (d + 4) * 2.0 ** -24 * (qq.abs() @ k.abs().T) * scale + 2.0 ** -23 * (s.abs() + z.abs())
                p = torch.where(see & (z > -math.inf), torch.exp(s - z), torch.zeros_like(s))
                total += p.sum(0)
                off += (p * (ds.masked_fill(p == 0, 0) + 2.0 ** -21 + new * group * 2.0 ** -24)).sum(0)
            out[page, h, j % places] += total
            tol[page, h, j % places] = off + 2.0 ** -23 * out[page, h, j % places]
            mine[page, h, j % places] = True
    return out, tol, mine


def run_case(seed, dim, places, qtype, ctype, heads, group, seqs, causal=True, window=0, same=False, none=False, layout="hpd"):
    g = torch.Generator().manual_seed(seed)
    lengths, news = [n for n, _ in seqs], [m for _, m in seqs]
    pages = sum(-(-n // places) for n in lengths) + 2
    cache = pu.random_cache(g, pages, heads, places, dim, ctype, layout=layout)
    table = pu.random_table(g, lengths, places, pages)
    pu.spoil_unused(cache, table, lengths)
    starts = torch.tensor([0] + news).cumsum(0).to(torch.int32)
    tokens, scale = int(starts[-1]), 1.0 / math.sqrt(dim)
    q = (torch.randn(tokens + 2, heads * group, dim, generator=g) * 1.5).to(qtype)
    lse = pu.attention64(q, cache, table, lengths, starts, scale, causal, window)[1].float()
    lse[tokens:] = float("nan")                                                       # rows of no sequence
    q[tokens:] = float("nan")
    before = torch.rand((pages, heads, places), generator=g)
    batch = vt.CacheBatch(table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts.cuda(), max(max(news), 1), max(max(lengths), 1))
    win = None if none else before.cuda()
    out = win if same else torch.full(before.shape, -5.0).cuda()
    vt.vitint_cache_weigh(q.cuda(), lse.cuda(), pu.to_gpu(cache), batch, scale, win, out, causal=causal, window=window)
    assert vt.vitint_device_status() == 0
    want, tol, mine = weights64(q, lse, cache, table, lengths, starts, scale, causal, window, before * 0 if none else before)
    got = out.double().cpu()
    assert bool((got[~mine] == (before.double() if same else torch.full_like(got, -5.0))[~mine]).all())
    off = (got - want).abs()
    assert bool((off[mine] <= tol[mine]).all()), (float((off - tol)[mine].max()), float(off[mine].max()))


@pytest.mark.parametrize("ctype,qtype", [(BF16, BF16), (F16, F16), (I8, BF16), (I8, F16)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("places", [16, 32, 64, 128])
def test_single_tokens(dim, places, ctype, qtype):
    run_case(1, dim, places, qtype, ctype, 2, 4, [(1, 1), (15, 1), (129, 1), (300, 1), (127, 1), (128, 1)])


@pytest.mark.parametrize("ctype", [BF16, I8])
@pytest.mark.parametrize("group,new", [(1, 130), (1, 300), (2, 65), (3, 50), (4, 33), (7, 100), (8, 17), (12, 40), (16, 8), (40, 7), (128, 3)])
def test_chunks(group, new, ctype):
    run_case(2, 128, 16, BF16, ctype, 2, group, [(new + 257, new), (new, new), (129, 1)])


@pytest.mark.parametrize("ctype", [F16, I8])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 17), (True, 128), (True, 200)])
def test_masks(causal, window, ctype):
    run_case(3, 64, 32, F16, ctype, 2, 3, [(700, 150), (64, 1), (130, 99), (150, 150)], causal, window)


def test_rows_without_keys_and_sequences_without_queries():
    run_case(4, 64, 16, BF16, BF16, 2, 2, [(0, 2), (3, 5), (200, 0), (0, 0), (33, 2)])


def test_split_runs_and_the_same_array():
    run_case(5, 128, 64, BF16, I8, 1, 8, [(5000, 1500)], same=True)
    run_case(6, 64, 16, BF16, BF16, 2, 2, [(9000, 3), (50, 1)], none=True, layout="phd")


def test_same_bits_every_time_and_replay():
    g = torch.Generator().manual_seed(7)
    cache = pu.to_gpu(pu.random_cache(g, 30, 2, 64, 128, BF16))
    lengths = [1500, 300]
    table = pu.random_table(g, lengths, 64, 30).cuda()
    batch = vt.CacheBatch(table, torch.tensor(lengths, dtype=torch.int32).cuda(), torch.tensor([0, 700, 701], dtype=torch.int32).cuda(), 700, 1500)
    q, lse = torch.randn(701, 8, 128, generator=g).to(BF16).cuda(), torch.rand(701, 8, generator=g).add(7).cuda()
    w = torch.zeros(30, 2, 64, device="cuda")
    first = vt.vitint_cache_weigh(q, lse, cache, batch, 0.09, None, w).clone()
    work = torch.empty(vt.vitint_cache_weigh_workspace_bytes(cache, batch), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        vt.vitint_cache_weigh(q, lse, cache, batch, 0.09, None, w, workspace=work)
    for _ in range(4):
        w.zero_(), work.fill_(0x77)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(w, first)


@pytest.mark.parametrize("bad", [18, 22, 27, 31])
@pytest.mark.parametrize("new", [3, 40])
def test_queries_that_are_not_numbers_show(new, bad):
    """A query row of NaN makes the weights of all tokens that it sees NaN, whichever column of the product it is; other heads' are as they were."""
    g = torch.Generator().manual_seed(8)
    cache = pu.random_cache(g, 20, 2, 16, 64, BF16)
    table, lengths = pu.random_table(g, [300], 16, 20), [300]
    starts, row = torch.tensor([0, new], dtype=torch.int32), bad % new
    q = torch.randn(new, 2, 64, generator=g).to(BF16)
    lse = pu.attention64(q, cache, table, lengths, starts, 0.1, True, 0)[1].float()
    q[row, 1] = float("nan")
    batch = vt.CacheBatch(table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts.cuda(), new, 300)
    w = vt.vitint_cache_weigh(q.cuda(), lse.cuda(), pu.to_gpu(cache), batch, 0.1, None, torch.zeros(20, 2, 16, device="cuda")).cpu()
    j = torch.arange(300)
    mine = w[table[0, j // 16].long(), :, j % 16]
    seen = 300 - new + row + 1
    assert bool(mine[:seen, 1].isnan().all()) and not bool(mine[seen:, 1].isnan().any()) and not bool(mine[:, 0].isnan().any())


@pytest.mark.parametrize("new", [1, 120])
def test_weights_too_small_for_their_type_are_zero(new):
    """Tokens 200 nats below the rows' sums: their weight is below 2^-149, and 0 in every column of the product."""
    g = torch.Generator().manual_seed(9)
    cache = vt.PagedCache(torch.zeros(20, 1, 16, 64, dtype=BF16), torch.zeros(20, 1, 16, 64, dtype=BF16))
    cache.k[:10, ..., 0] = -1.0
    q = torch.zeros(new, 1, 64, dtype=BF16)
    q[..., 0] = 200.0
    batch = vt.CacheBatch(torch.arange(20, dtype=torch.int32)[None].cuda(), torch.tensor([320], dtype=torch.int32).cuda(),
                          torch.tensor([0, new], dtype=torch.int32).cuda(), new, 320)
    gpu = pu.to_gpu(cache)
    _, lse = vt.vitint_paged_attention(q.cuda(), gpu, batch, 1.0, want_lse=True)
    w = vt.vitint_cache_weigh(q.cuda(), lse, gpu, batch, 1.0, None, torch.full((20, 1, 16), 7.0, device="cuda"))
    assert not bool(w[:10].any()) and bool((w[10:, 0, 0] > 0).all())

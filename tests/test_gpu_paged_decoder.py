"""The paged cache's operators together, as a decoder layer uses them next to the integerized linears: a prompt, its weights, eviction, and further
tokens.  Every stage is checked against its definition in 64 bits on what the stage in front gave."""
import math

import pytest
import torch

import paged_util as pu
import paper_2504_18547_b200 as vt

pytestmark = pytest.mark.gpu

DIM, HQ, HK, D, PLACES, PAGES = 256, 4, 2, 64, 16, 64


class Layer:
    def __init__(self, g):
        n = (HQ + 2 * HK) * D
        w = torch.randn(n, DIM, generator=g) * 0.05
        steps = w.abs().amax(1) / 127
        self.w = vt.vitint_quantize(w.cuda(), 0.0, 8, True, row_steps=steps.cuda())
        self.w_step = steps.cuda()
        self.gain = [torch.ones(D, device="cuda") + 0.1 * torch.randn(D, generator=g).cuda() for _ in range(2)]
        self.freq = 10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)

    def queries(self, x, positions, cache, slots, weights):
        """Integer projection to fp32 rows, then the head norms, rotation and store."""
        codes = vt.vitint_quantize(x, 0.03, 8, True)
        rows = vt.vitint_linear(codes, 0.03, self.w, self.w_step, None, vt.Epilogue(mode=vt.EPI_DEQUANT_F32))
        q, k, v = rows.split((HQ * D, HK * D, HK * D), 1)
        return vt.vitint_qk_norm_rotate(q, k, v, D, q_gain=self.gain[0], k_gain=self.gain[1], positions=positions, frequencies=self.freq, cache=cache, slots=slots,
                                        weights=weights, out_dtype=torch.bfloat16)[0]


def host(cache):
    cpu = lambda t: None if t is None else t.cpu()
    return vt.PagedCache(cpu(cache.k), cpu(cache.v), cpu(cache.k_steps), cpu(cache.v_steps))


def slots_of(table, rows):
    return torch.tensor([int(table[b, j // PLACES]) * PLACES + j % PLACES for b, j in rows])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_prompt_eviction_and_further_tokens(dtype):
    g = torch.Generator().manual_seed(1)
    layer, scale = Layer(g), 1.0 / math.sqrt(D)
    cache = vt.PagedCache.empty(PAGES, HK, PLACES, D, dtype)
    weights = torch.full((PAGES, HK, PLACES), float("nan"), device="cuda")
    order = torch.randperm(PAGES, generator=g).to(torch.int32)
    lengths, table = [150, 61], torch.full((2, 12), -1, dtype=torch.int32)
    table[0, :10], table[1, :4] = order[:10], order[10:14]
    new_table = order[20:26].view(2, 3)                                            # 40 kept tokens, and the pages that follow

    def step(table, lengths, news, positions):
        """One call of the layer: stores the new tokens, attends, adds up their weights.  Checks all of it."""
        rows = [(b, lengths[b] - news[b] + i) for b in range(2) for i in range(news[b])]
        x = torch.randn(len(rows), DIM, generator=g).cuda()
        q = layer.queries(x, torch.tensor(positions, dtype=torch.int32).cuda(), cache, slots_of(table, rows).cuda(), weights)
        starts = torch.tensor([0, news[0], news[0] + news[1]], dtype=torch.int32)
        batch = vt.CacheBatch(table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts.cuda(), max(news), table.shape[1] * PLACES)
        out, lse = vt.vitint_paged_attention(q, cache, batch, scale, want_lse=True)
        before = weights.cpu()
        vt.vitint_cache_weigh(q, lse, cache, batch, scale, weights, weights)
        assert vt.vitint_device_status() == 0
        at = host(cache)
        pu.check_attention(out, lse, pu.attention64(q.cpu(), at, table, lengths, starts, scale, True, 0))
        for b in range(2):                                                         # all weight that a row gives is given away: a row's sum is 1
            j = torch.arange(lengths[b])
            page = table[b, j // PLACES].long()
            gained = (weights.cpu()[page, :, j % PLACES] - before[page, :, j % PLACES]).double().sum(0)
            want = news[b] * (HQ // HK)
            assert bool(((gained - want).abs() <= 1e-5 * want + 1e-4).all()), gained
        return batch, out

    step(table, lengths, [150, 61], [*range(150), *range(61)])
    batch, _ = step(table, [151, 62], [1, 1], [150, 61])
    kept, counts = vt.vitint_cache_evict(cache, batch, weights, 40, new_table.cuda(), sinks=2, recent=8)
    assert counts.tolist() == [40, 40] and vt.vitint_device_status() == 0
    for b, n in enumerate((151, 62)):
        for h in range(HK):
            j = torch.arange(n)
            old = weights.cpu()[table[b, j // PLACES].long(), h, j % PLACES]
            free = sorted(range(2, n - 8), key=lambda i: (-float(old[i]), i))[:30]
            assert kept[b, h].tolist() == sorted([0, 1] + free + list(range(n - 8, n)))
            to = torch.arange(40)
            assert torch.equal(weights.cpu()[new_table[b, to // PLACES].long(), h, to % PLACES], old[kept[b, h].cpu().long()])
    # three more tokens, one and two, over what is left; positions go on as if nothing had been taken out
    step(new_table, [41, 42], [1, 2], [151, 62, 63])
    step(new_table, [42, 43], [1, 1], [152, 64])


def test_two_streams_side_by_side():
    """Two calls at once, each with its own workspace, queries and outputs, over one cache: the same bits as one after the other."""
    g = torch.Generator().manual_seed(2)
    cache = vt.PagedCache.empty(PAGES, HK, PLACES, D)
    cache.k.copy_(torch.randn(cache.k.shape, generator=g)), cache.v.copy_(torch.randn(cache.v.shape, generator=g))
    table = torch.randperm(PAGES, generator=g).to(torch.int32).view(2, -1).cuda()
    calls = []
    for lengths, news in (([500, 200], [1, 1]), ([430, 512], [100, 37])):
        starts = torch.tensor([0, news[0], sum(news)], dtype=torch.int32).cuda()
        batch = vt.CacheBatch(table, torch.tensor(lengths, dtype=torch.int32).cuda(), starts, max(news), 512)
        q = torch.randn(sum(news), HQ, D, generator=g).to(torch.bfloat16).cuda()
        work = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (vt.vitint_paged_attention_workspace_bytes(HQ, cache, batch),
                                                                            vt.vitint_cache_weigh_workspace_bytes(cache, batch))]
        calls.append((q, batch, work, torch.empty_like(q), torch.empty(q.shape[:2], device="cuda"), torch.zeros(PAGES, HK, PLACES, device="cuda")))

    def call(q, batch, work, out, lse, weights):
        vt.vitint_paged_attention(q, cache, batch, 0.125, out=out, lse=lse, workspace=work[0])
        vt.vitint_cache_weigh(q, lse, cache, batch, 0.125, None, weights, workspace=work[1])

    want = []
    for c in calls:
        call(*c)
        want.append([t.clone() for t in c[3:]])
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                for t in c[3:5]:
                    t.zero_()
                call(*c)
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert all(torch.equal(a, b) for a, b in zip(c[3:], w))
    assert vt.vitint_device_status() == 0

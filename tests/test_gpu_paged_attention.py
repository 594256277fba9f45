"""Attention over the paged cache against its definition in 64 bits."""
import math

import pytest
import torch

import paper_2504_18547_b200 as vt
import paged_util as pu
from gpu_util import GUARD_BYTES, check_guards, guarded_tensor

pytestmark = pytest.mark.gpu

BF16, F16, I8 = torch.bfloat16, torch.float16, torch.int8


def run_case(seed, dim, places, qtype, ctype, kv_heads, group, seqs, causal=True, window=0, q_size=1.5, layout="hpd", spare=2, max_length=None):
    """seqs: (cached tokens, new tokens) of each sequence."""
    g = torch.Generator().manual_seed(seed)
    lengths, news = [n for n, _ in seqs], [m for _, m in seqs]
    pages = sum(-(-n // places) for n in lengths) + spare
    cache = pu.random_cache(g, pages, kv_heads, places, dim, ctype, layout=layout)
    table = pu.random_table(g, lengths, places, pages)
    pu.spoil_unused(cache, table, lengths)
    starts = torch.tensor([0] + news).cumsum(0).to(torch.int32)
    tokens, heads = int(starts[-1]), kv_heads * group
    q = (torch.randn(tokens + 3, heads, dim, generator=g) * q_size).to(qtype)       # three rows that belong to no sequence
    scale = 1.0 / math.sqrt(dim)
    batch = vt.CacheBatch(table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts.cuda(), max(max(news), 1),
                          max_length or max(max(lengths), 1))
    out = guarded_tensor(q.shape, qtype)
    lse = guarded_tensor(q.shape[:2], torch.float32)
    out.fill_(7.0)
    lse.fill_(7.0)
    vt.vitint_paged_attention(q.cuda(), pu.to_gpu(cache), batch, scale, causal=causal, window=window, out=out, lse=lse)
    assert vt.vitint_device_status() == 0
    check_guards()
    assert bool((out[tokens:] == 7.0).all()) and bool((lse[tokens:] == 7.0).all())
    pu.check_attention(out, lse, pu.attention64(q, cache, table, lengths, starts, scale, causal, window))


# few rows a head of the cache: one token or a few, every group size that fits sixteen rows
@pytest.mark.parametrize("ctype,qtype", [(BF16, BF16), (F16, F16), (I8, BF16), (I8, F16)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("places", [16, 32, 64, 128])
def test_single_tokens(dim, places, ctype, qtype):
    run_case(1, dim, places, qtype, ctype, 2, 4, [(1, 1), (15, 1), (16, 1), (17, 1), (129, 1), (300, 1), (63, 1)])


@pytest.mark.parametrize("ctype", [BF16, I8])
@pytest.mark.parametrize("group,new", [(1, 1), (1, 16), (2, 7), (3, 5), (5, 3), (6, 2), (7, 2), (8, 2), (12, 1), (16, 1)])
def test_groups_and_drafts(group, new, ctype):
    run_case(2, 64, 16, BF16, ctype, 3, group, [(97, new), (new, new), (211, 1)])


def test_long_rows_are_split():
    run_case(3, 128, 64, BF16, BF16, 2, 4, [(20001, 1), (3, 1), (7777, 1)])
    run_case(4, 64, 16, F16, F16, 1, 1, [(30000, 2)])
    run_case(5, 128, 32, F16, I8, 1, 8, [(16385, 2)])


@pytest.mark.parametrize("ctype", [F16, I8])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 17), (True, 64), (True, 65), (True, 4000)])
def test_masks(causal, window, ctype):
    run_case(6, 64, 16, F16, ctype, 2, 3, [(200, 5), (64, 1), (130, 3), (5, 5)], causal, window)


@pytest.mark.parametrize("ctype", [BF16, I8])
def test_rows_without_keys(ctype):
    """Sequences that are empty, shorter than their new tokens, or bring none."""
    run_case(7, 128, 16, BF16, ctype, 2, 2, [(0, 2), (3, 5), (40, 0), (0, 0), (33, 2)])
    run_case(8, 64, 32, BF16, ctype, 1, 2, [(0, 1)])


def test_peaked_rows():
    """Scores of hundreds: almost all weight on one key, and a maximum that keeps growing."""
    run_case(9, 128, 16, BF16, BF16, 2, 4, [(700, 1), (333, 3)], q_size=60.0)
    run_case(10, 128, 16, F16, I8, 2, 4, [(700, 1), (333, 3)], q_size=60.0)


@pytest.mark.parametrize("ctype", [BF16, I8])
def test_small_steps_and_layouts(ctype):
    run_case(11, 128, 32, BF16, ctype, 4, 2, [(100, 2), (37, 1)], layout="phd")


def test_tiny_value_steps_in_fp16():
    """Steps far below fp16's range: the products are taken relative to the largest."""
    g = torch.Generator().manual_seed(12)
    cache = pu.random_cache(g, 20, 1, 16, 128, I8)
    cache.v_steps.mul_(1e-4)
    cache.v_steps[3:6].mul_(300.0)
    table = pu.random_table(g, [300], 16, 20)
    q = torch.randn(1, 4, 128, generator=g).to(F16)
    starts = torch.tensor([0, 1], dtype=torch.int32)
    batch = vt.CacheBatch(table.cuda(), torch.tensor([300], dtype=torch.int32).cuda(), starts.cuda(), 1, 300)
    out, lse = vt.vitint_paged_attention(q.cuda(), pu.to_gpu(cache), batch, 0.08, want_lse=True)
    want = list(pu.attention64(q, cache, table, [300], starts, 0.08, True, 0))
    want[2] += 2.0 ** -25                                  # outputs of 1e-3 and less: fp16's own subnormal step
    pu.check_attention(out, lse, want)


def _small(g, seqs=((90, 1), (200, 1)), dim=128, places=16, kv_heads=2, group=4, dtype=BF16, extra_pages=2, max_queries=None):
    lengths, news = [n for n, _ in seqs], [m for _, m in seqs]
    pages = sum(-(-n // places) for n in lengths) + extra_pages
    cache = pu.random_cache(g, pages, kv_heads, places, dim, dtype)
    table = pu.random_table(g, lengths, places, pages)
    starts = torch.tensor([0] + news).cumsum(0).to(torch.int32)
    q = torch.randn(int(starts[-1]), kv_heads * group, dim, generator=g).to(BF16)
    batch = vt.CacheBatch(table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts.cuda(), max_queries or max(news), max(lengths))
    return cache, table, lengths, starts, q, batch


@pytest.mark.parametrize("seqs", [((90, 1), (200, 1)), ((90, 30), (200, 77))])
def test_strided_queries_and_outputs(seqs):
    g = torch.Generator().manual_seed(20)
    cache, table, lengths, starts, q, batch = _small(g, seqs)
    fused = torch.zeros(q.shape[0], 3, 8 + 5, 128, dtype=BF16, device="cuda")        # queries inside wider rows
    fused[:, 1, 2:10] = q.cuda()
    wide = torch.full((q.shape[0], 20, 256), 3.0, dtype=BF16, device="cuda")
    lse = torch.empty(q.shape[:2], device="cuda")
    vt.vitint_paged_attention(fused[:, 1, 2:10], pu.to_gpu(cache), batch, 0.09, out=wide[:, 1:17:2, 128:], lse=lse)
    pu.check_attention(wide[:, 1:17:2, 128:], lse, pu.attention64(q, cache, table, lengths, starts, 0.09, True, 0))
    wide[:, 1:17:2, 128:] = 3.0
    assert bool((wide == 3.0).all())


@pytest.mark.parametrize("seqs", [((90, 1), (200, 1)), ((90, 30), (200, 77))])
def test_recorded_call_replayed_with_other_lengths_on_another_stream(seqs):
    g = torch.Generator().manual_seed(21)
    cache, table, lengths, starts, q, batch = _small(g, seqs)
    gpu, qd = pu.to_gpu(cache), q.cuda()
    out, lse = torch.empty_like(qd), torch.empty(q.shape[:2], device="cuda")
    workspace = torch.empty(vt.vitint_paged_attention_workspace_bytes(q.shape[1], gpu, batch), dtype=torch.uint8, device="cuda")
    call = lambda: vt.vitint_paged_attention(qd, gpu, batch, 0.09, out=out, lse=lse, workspace=workspace)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        for other in (lengths, [seqs[0][1], 131], [64, 199]):
            batch.lengths.copy_(torch.tensor(other, dtype=torch.int32))
            workspace.fill_(0x5A)
            out.fill_(0)
            graph.replay()
            stream.synchronize()
            pu.check_attention(out, lse, pu.attention64(q, cache, table, other, starts, 0.09, True, 0))
    assert vt.vitint_device_status() == 0


@pytest.mark.parametrize("seqs", [((9000, 1), (200, 1)), ((900, 30), (2000, 77))])
def test_same_bits_every_time(seqs):
    g = torch.Generator().manual_seed(22)
    cache, *_, q, batch = _small(g, seqs)
    gpu, qd = pu.to_gpu(cache), q.cuda()
    first = [t.clone() for t in vt.vitint_paged_attention(qd, gpu, batch, 0.09, want_lse=True)]
    for _ in range(5):
        again = vt.vitint_paged_attention(qd, gpu, batch, 0.09, want_lse=True)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("new", [1, 40])
def test_bad_pages_and_lengths_are_reported(new):
    """A page index outside the cache reads as zeros; lengths and ranges beyond the declared bounds are cut.  Nothing else is touched."""
    g = torch.Generator().manual_seed(23)
    cache, table, lengths, starts, q, batch = _small(g, ((200, new), (90, new)))
    gpu, qd = pu.to_gpu(cache), q.cuda()
    good = vt.vitint_paged_attention(qd, gpu, batch, 0.09).clone()
    assert vt.vitint_device_status() == 0
    bad = batch.page_table.clone()
    bad[1, 2], bad[1, 3] = -5, 1 << 30
    out = vt.vitint_paged_attention(qd, gpu, vt.CacheBatch(bad, batch.lengths, batch.query_starts, batch.max_queries, batch.max_length), 0.09)
    assert vt.vitint_device_status() == -1 and vt.vitint_device_status() == 0
    assert torch.equal(out[:new], good[:new])
    long = torch.tensor([1 << 29, 90], dtype=torch.int32).cuda()
    out = vt.vitint_paged_attention(qd, gpu, vt.CacheBatch(batch.page_table, long, batch.query_starts, batch.max_queries, batch.max_length), 0.09)
    assert vt.vitint_device_status() == -1
    assert torch.equal(out, good)                                                   # 2^29 counts as 200, the longest declared
    ranges = torch.tensor([0, new, 100000], dtype=torch.int32).cuda()
    out = vt.vitint_paged_attention(qd, gpu, vt.CacheBatch(batch.page_table, batch.lengths, ranges, batch.max_queries, batch.max_length), 0.09)
    assert vt.vitint_device_status() == -1
    assert torch.equal(out, good)
    short = torch.tensor([0, -7, 2 * new], dtype=torch.int32).cuda()
    vt.vitint_paged_attention(qd, gpu, vt.CacheBatch(batch.page_table, batch.lengths, short, batch.max_queries, batch.max_length), 0.09)
    assert vt.vitint_device_status() == -1


@pytest.mark.parametrize("new", [1, 40])
def test_offsets_beyond_32_bits(new):
    """Pages that lie more than 2^32 bytes (2^31 elements) into the cache."""
    g = torch.Generator().manual_seed(24)
    places, dim, heads, pages = 128, 128, 2, (1 << 31) // (128 * 128 * 2) + 40
    small = pu.random_cache(g, 8, heads, places, dim, BF16)
    k, v = (torch.empty((pages, heads, places, dim), dtype=BF16, device="cuda") for _ in range(2))
    at = torch.tensor([pages - 1, pages - 9, 0, 65536, pages - 3, pages - 4, 1, 2])
    k[at.cuda()], v[at.cuda()] = small.k.cuda(), small.v.cuda()
    order = torch.tensor([[0, 1, 2, 3, 4, 5, 6, 7]])
    lengths, starts = [1000], torch.tensor([0, new], dtype=torch.int32)
    q = torch.randn(new, 4, dim, generator=g).to(BF16)
    batch = vt.CacheBatch(at[None].to(torch.int32).cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts.cuda(), new, 1000)
    out, lse = vt.vitint_paged_attention(q.cuda(), vt.PagedCache(k, v), batch, 0.09, want_lse=True)
    pu.check_attention(out, lse, pu.attention64(q, small, order, lengths, starts, 0.09, True, 0))


# ---- more rows than one warp-level product: the tensor-core kernel ----------------------------------------------------------------

@pytest.mark.parametrize("ctype,qtype", [(BF16, BF16), (F16, F16), (I8, BF16), (I8, F16)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("places", [16, 32, 64, 128])
def test_chunks(dim, places, ctype, qtype):
    run_case(31, dim, places, qtype, ctype, 2, 4, [(1, 1), (100, 17), (128, 128), (129, 64), (300, 65), (400, 1)])


@pytest.mark.parametrize("ctype", [BF16, I8])
@pytest.mark.parametrize("group,new", [(1, 17), (1, 300), (2, 129), (3, 43), (4, 33), (5, 51), (7, 37), (8, 3), (12, 21), (24, 1), (40, 7), (128, 2)])
def test_chunk_groups(group, new, ctype):
    run_case(32, 128, 16, BF16, ctype, 2, group, [(new + 150, new), (new, new), (77, 1)])


@pytest.mark.parametrize("ctype", [F16, I8])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 17), (True, 64), (True, 128), (True, 129), (True, 500)])
def test_chunk_masks(causal, window, ctype):
    run_case(33, 64, 32, F16, ctype, 2, 3, [(900, 200), (64, 1), (130, 99), (150, 150)], causal, window)


@pytest.mark.parametrize("ctype", [BF16, I8])
def test_chunk_rows_without_keys(ctype):
    run_case(34, 128, 16, BF16, ctype, 2, 2, [(0, 40), (30, 150), (40, 0), (0, 0), (33, 20)])
    run_case(35, 64, 32, BF16, ctype, 1, 2, [(0, 40)])


def test_chunk_items_are_split():
    run_case(36, 128, 64, BF16, BF16, 1, 4, [(9000, 40), (3, 1), (777, 300)])
    run_case(37, 64, 16, F16, I8, 2, 2, [(5000, 130)])
    run_case(38, 128, 32, F16, F16, 1, 8, [(20000, 20)], window=3000)


def test_chunk_peaked_rows():
    """Maxima that keep growing: the outputs follow several times."""
    run_case(39, 128, 16, BF16, BF16, 1, 4, [(1700, 100)], q_size=60.0)
    run_case(40, 64, 16, F16, I8, 1, 4, [(1700, 100)], q_size=40.0)


@pytest.mark.parametrize("ctype", [BF16, I8])
def test_chunk_layouts(ctype):
    run_case(41, 128, 32, BF16, ctype, 4, 2, [(100, 40), (337, 100)], layout="phd")


def test_chunk_tiny_value_steps_in_fp16():
    g = torch.Generator().manual_seed(42)
    cache = pu.random_cache(g, 70, 1, 16, 128, I8)
    cache.v_steps.mul_(1e-4)
    cache.v_steps[3:6].mul_(300.0)
    table = pu.random_table(g, [1000], 16, 70)
    q = torch.randn(40, 4, 128, generator=g).to(F16)
    starts = torch.tensor([0, 40], dtype=torch.int32)
    batch = vt.CacheBatch(table.cuda(), torch.tensor([1000], dtype=torch.int32).cuda(), starts.cuda(), 40, 1000)
    out, lse = vt.vitint_paged_attention(q.cuda(), pu.to_gpu(cache), batch, 0.08, want_lse=True)
    want = list(pu.attention64(q, cache, table, [1000], starts, 0.08, True, 0))
    want[2] += 2.0 ** -25
    pu.check_attention(out, lse, want)


@pytest.mark.parametrize("new", [1, 23])
def test_many_sequences(new):
    """More sequences than lanes of a warp, some without new tokens: the plan walks them in blocks of 32."""
    seqs = [((37 * i) % 150 + new, new if i % 7 else 0) for i in range(101)]
    run_case(50, 64, 16, BF16, BF16, 2, 2, seqs)


def test_queries_over_themselves():
    """The output may be the queries' memory: an item's queries are read before its rows are written."""
    g = torch.Generator().manual_seed(51)
    for seqs in (((90, 1), (5000, 1)), ((90, 30), (2000, 77))):
        cache, table, lengths, starts, q, batch = _small(g, seqs)
        gpu, qd = pu.to_gpu(cache), q.cuda()
        want = vt.vitint_paged_attention(qd, gpu, batch, 0.09).clone()
        assert torch.equal(vt.vitint_paged_attention(qd, gpu, batch, 0.09, out=qd), want)


# ---- data that the mask hides or the page table does not name ---------------------------------------------------------------------

def _alternating(g, ctype, new, dim=128, places=16, group=1, count=400):
    """Sequences of 41 tokens, whose last page ends in NaN, and between them ones of 60 whose third page is none of the cache's (the reference has a
    page of zeros there): what a CTA had in shared memory before is NaN where the missing page's tokens lie."""
    lengths = [41, 60] * (count // 2)
    pages = sum(-(-n // places) for n in lengths) + 1
    cache = pu.random_cache(g, pages, 2, places, dim, ctype)
    table = pu.random_table(g, lengths, places, pages - 1)
    pu.spoil_unused(cache, table, lengths)
    with_zeros = vt.PagedCache(*(None if t is None else t.clone() for t in (cache.k, cache.v, cache.k_steps, cache.v_steps)))
    for t in (with_zeros.k, with_zeros.v, with_zeros.k_steps, with_zeros.v_steps):
        if t is not None:
            t[pages - 1] = 0
    bad, want = table.clone(), table.clone()
    bad[1::2, 2] = torch.where(torch.arange(count // 2) % 2 == 0, -1, 1 << 30).to(torch.int32)
    want[1::2, 2] = pages - 1
    starts = (torch.arange(count + 1) * new).to(torch.int32)
    q = torch.randn(count * new, 2 * group, dim, generator=g).to(F16 if ctype == F16 else BF16)
    batch = vt.CacheBatch(bad.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts.cuda(), new, 64)
    return cache, with_zeros, want, lengths, starts, q, batch


@pytest.mark.parametrize("window", [0, 10])
@pytest.mark.parametrize("ctype", [BF16, F16, I8])
@pytest.mark.parametrize("new", [1, 17])
def test_missing_pages_are_zeros(new, ctype, window):
    """Keys, values and steps of a page that is not there count as zeros, whatever shared memory held; behind a window they do not count."""
    g = torch.Generator().manual_seed(60)
    cache, with_zeros, table, lengths, starts, q, batch = _alternating(g, ctype, new, count=2400 if new == 1 else 400)      # several items a CTA
    out, lse = vt.vitint_paged_attention(q.cuda(), pu.to_gpu(cache), batch, 0.09, window=window, want_lse=True)
    assert vt.vitint_device_status() == -1
    pu.check_attention(out, lse, pu.attention64(q, with_zeros, table, lengths, starts, 0.09, True, window))


@pytest.mark.parametrize("new", [1, 3, 40])
def test_steps_of_hidden_tokens_do_not_count(new):
    """Tokens in front of the window with steps 2^30 times as large: the others are taken relative to the largest step that some row sees."""
    g = torch.Generator().manual_seed(61)
    cache = pu.random_cache(g, 12, 2, 16, 128, I8)
    table = pu.random_table(g, [120], 16, 12)
    hidden = torch.arange(120 - new - 9)                                           # in front of the first new token's ten
    seen_only = vt.PagedCache(cache.k, cache.v, cache.k_steps, cache.v_steps.clone())
    cache.v_steps[table[0, hidden // 16].long(), :, hidden % 16] *= 2.0 ** 30
    seen_only.v_steps[table[0, hidden // 16].long(), :, hidden % 16] = 0
    q = torch.randn(new, 4, 128, generator=g).to(BF16)
    starts = torch.tensor([0, new], dtype=torch.int32)
    batch = vt.CacheBatch(table.cuda(), torch.tensor([120], dtype=torch.int32).cuda(), starts.cuda(), new, 120)
    out, lse = vt.vitint_paged_attention(q.cuda(), pu.to_gpu(cache), batch, 0.09, window=10, want_lse=True)
    pu.check_attention(out, lse, pu.attention64(q, seen_only, table, [120], starts, 0.09, True, 10))


@pytest.mark.parametrize("qtype,ctype", [(F16, F16), (F16, I8), (BF16, I8)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group,new,length", [(4, 1, 131073), (4, 1, 200), (4, 4, 9000), (4, 40, 9000), (1, 20, 300)])
def test_a_tail_far_below_the_maximum_counts(group, new, length, dim, qtype, ctype):
    """Every sixteenth token has the value 0 and, 17.5 nats below it, all others have 512: the output is 512 times the others' share of the sum.

    A probability is off by half a step of the operand's type, 2^-11 relative, or where it is below fp16's normal range by half of 2^-24 over the
    offset that it is taken with (2^5 at least), 2^-30 of the maximum; the output's rounding and the score's error (of size 17.5: products of d
    channels and three roundings, (d + 8) 2^-24 17.5) come on top, and 2^-18 for ex2 and the sums."""
    places = 128
    pages = -(-length // places)
    shape = (pages, 1, places, dim)
    k, v = torch.zeros(shape), torch.full(shape, 512.0)
    k[..., 0] = -1.0
    k[:, 0, ::16, 0], v[:, 0, ::16] = 0.0, 0.0                                      # scores: 0, and -17.5 for all others
    if ctype == I8:
        cache = vt.PagedCache((k * 4).to(I8), (v / 256).to(I8), torch.full(shape[:3], 0.25), torch.full(shape[:3], 256.0))
    else:
        cache = vt.PagedCache(k.to(ctype), v.to(ctype))
    q = torch.zeros(new, group, dim, dtype=qtype)
    q[..., 0] = 17.5
    batch = vt.CacheBatch(torch.arange(pages, dtype=torch.int32)[None].cuda(), torch.tensor([length], dtype=torch.int32).cuda(),
                          torch.tensor([0, new], dtype=torch.int32).cuda(), new, length)
    out, lse = vt.vitint_paged_attention(q.cuda(), pu.to_gpu(cache), batch, 1.0, causal=False, want_lse=True)
    top = -(-length // 16)
    others = (length - top) * math.exp(-17.5)
    want, half = 512 * others / (top + others), pu.EPS[qtype] / 2
    relative = half + 2.0 ** -11 + 2 * (dim + 8) * 2.0 ** -24 * 17.5 + 2.0 ** -18
    absolute = 512 * (length - top) / top * 2.0 ** -30 + (2.0 ** -25 if qtype == F16 else 0.0)       # (fp16 outputs' own subnormal step)
    off = (out.double() - want).abs().max()
    assert float(off) <= relative * want + absolute, (float(off), want)
    z = math.log(top + others)
    assert float((lse.double() - z).abs().max()) <= 2.0 ** -18 + 2.0 ** -22 * z


def test_any_bound_of_the_new_tokens():
    """max_queries may be as large as its type holds: no sequence has more new tokens than there are rows."""
    g = torch.Generator().manual_seed(62)
    cache, table, lengths, starts, q, batch = _small(g, ((90, 30), (200, 77)))
    gpu, qd = pu.to_gpu(cache), q.cuda()
    want, lse = vt.vitint_paged_attention(qd, gpu, batch, 0.09, want_lse=True)
    loose = vt.CacheBatch(batch.page_table, batch.lengths, batch.query_starts, 2 ** 31 - 1, batch.max_length)
    assert torch.equal(vt.vitint_paged_attention(qd, gpu, loose, 0.09), want)
    places = (cache.k.shape[0], cache.k.shape[1], cache.k.shape[2])
    first = vt.vitint_cache_weigh(qd, lse, gpu, batch, 0.09, None, torch.zeros(places, device="cuda"))
    assert torch.equal(vt.vitint_cache_weigh(qd, lse, gpu, loose, 0.09, None, torch.zeros(places, device="cuda")), first)
    assert vt.vitint_device_status() == 0


def test_the_status_keeps_what_it_has_not_reported():
    """A wait that gave up and a page index outside the cache, both before the status is asked for: two answers, one after the other."""
    g = torch.Generator().manual_seed(63)
    cache, table, lengths, starts, q, batch = _small(g)
    batch.page_table[0, 0] = -1
    vt.vitint_paged_attention(q.cuda(), pu.to_gpu(cache), batch, 0.09)
    vt.vitint_selftest_wait_timeout(1000000)
    assert sorted(vt.vitint_device_status() for _ in range(3)) == [-7, -1, 0]
    assert vt.vitint_device_status() == 0


def test_strides_that_nothing_steps_by():
    """One query row, one head, one page: what their strides are does not matter, and keys' and values' need not agree there."""
    g = torch.Generator().manual_seed(64)
    d, places = 64, 16
    cache = pu.random_cache(g, 1, 1, places, d, BF16)
    table, lengths = torch.zeros(1, 1, dtype=torch.int32), [13]
    loose = lambda t, page, head: torch.empty(8192, dtype=t.dtype, device="cuda").as_strided(t.shape, (page, head, d, 1)).copy_(t)
    one_page = vt.PagedCache(loose(cache.k, 1031, 1), loose(cache.v, 17, 1025))
    for new, heads in ((1, 1), (1, 3), (5, 1), (13, 2), (3, 1)):
        q = torch.randn(new, heads, d, generator=g).to(BF16)
        strides = (2 * d * heads + 8 if new > 1 else 77, d if heads > 1 else 3, 1)
        qd, out = (torch.zeros(8192, dtype=BF16, device="cuda").as_strided(q.shape, strides) for _ in range(2))
        qd.copy_(q)
        starts = torch.tensor([0, new], dtype=torch.int32)
        batch = vt.CacheBatch(table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts.cuda(), new, 13)
        _, lse = vt.vitint_paged_attention(qd, one_page, batch, 0.09, out=out, want_lse=True)
        pu.check_attention(out, lse, pu.attention64(q, cache, table, lengths, starts, 0.09, True, 0))
    assert vt.vitint_device_status() == 0


@pytest.mark.parametrize("qtype,ctype", [(BF16, BF16), (F16, F16), (BF16, I8)])
@pytest.mark.parametrize("new", [1, 20])
def test_logarithms_of_equal_scores(new, qtype, ctype):
    """Scores of zero: the logarithm of the number of keys, off by a unit in the last place of log2 and the roundings of two products (2^-22 of it),
    and nothing that depends on what probabilities are taken relative to."""
    lengths = [2, 3, 5, 7, 13, 50, 100, 1000, 9000]
    table, pages = torch.zeros(len(lengths), 141, dtype=torch.int32), 1                  # (all sequences in one page of zeros)
    shape = (pages, 1, 64, 64)
    steps = [torch.ones(shape[:3])] * 2 if ctype == I8 else []
    cache = pu.to_gpu(vt.PagedCache(torch.zeros(shape, dtype=ctype), torch.zeros(shape, dtype=ctype), *steps))
    starts = (torch.arange(len(lengths) + 1) * new).to(torch.int32)
    batch = vt.CacheBatch(table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), starts.cuda(), new, 9000)
    _, lse = vt.vitint_paged_attention(torch.ones(len(lengths) * new, 1, 64, dtype=qtype, device="cuda"), cache, batch, 1.0, causal=False, want_lse=True)
    want = torch.tensor(lengths, dtype=torch.float64).log().repeat_interleave(new)
    off = (lse[:, 0].double().cpu() - want).abs()
    assert bool((off <= 2.0 ** -22 * want).all()), off / want

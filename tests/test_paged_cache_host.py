"""The paged cache's entry points reject bad arguments on the host, before anything is launched (no GPU is needed)."""
import pytest
import torch

OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 0, -1, -2, -3, -5
FAKE = 0x7000_0000_0000          # never dereferenced: every call below fails validation first
F32, BF16, F16, I8 = range(4)


@pytest.fixture(scope="module")
def B():
    from paper_2504_18547_b200.build import build_library
    build_library()
    import paper_2504_18547_b200.binding as b
    b.lib()
    return b


def cache(B, **change):
    f = dict(k=FAKE, v=FAKE, k_steps=0, v_steps=0, pages=10, page_stride=2 * 16 * 128, head_stride=16 * 128, token_stride=128, kv_heads=2, page_tokens=16,
             head_dim=128, type=BF16) | change
    return B._PACK_CACHE(*f.values())


def batch(B, **change):
    f = dict(table=FAKE, stride=8, lengths=FAKE, starts=FAKE, sequences=3, max_queries=1, max_length=100) | change
    return B._PACK_BATCH(*f.values())


def attention(B, c=None, b=None, **change):
    f = dict(q=FAKE, q_type=BF16, tokens=3, q_heads=8, q_token=1024, q_head=128, cache=c or cache(B), batch=b or batch(B), scale=0.1, causal=1, window=0,
             out=FAKE, out_token=1024, out_head=128, lse=None, workspace=None, size=0, stream=None) | change
    return B.lib().vitint_paged_attention(*f.values())


CACHE_FAULTS = [(dict(k=0), INVALID), (dict(v=0), INVALID), (dict(pages=0), INVALID), (dict(kv_heads=0), INVALID), (dict(type=F32), INVALID), (dict(type=9), INVALID),
                (dict(type=I8), INVALID), (dict(k_steps=FAKE, v_steps=FAKE), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED),
                (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=256), UNSUPPORTED), (dict(k=FAKE + 8), ALIGNMENT), (dict(v=FAKE + 2), ALIGNMENT),
                (dict(token_stride=132), ALIGNMENT), (dict(head_stride=100), ALIGNMENT), (dict(page_stride=0), INVALID), (dict(token_stride=64), INVALID),
                (dict(pages=1 << 31), UNSUPPORTED), (dict(type=I8, k_steps=FAKE + 4, v_steps=FAKE), ALIGNMENT), (dict(type=I8, k_steps=FAKE), INVALID)]
BATCH_FAULTS = [(dict(table=0), INVALID), (dict(lengths=0), INVALID), (dict(starts=0), INVALID), (dict(sequences=0), INVALID), (dict(max_queries=0), INVALID),
                (dict(max_length=0), INVALID), (dict(max_length=129), INVALID), (dict(stride=0), INVALID), (dict(sequences=70000), UNSUPPORTED),
                (dict(max_length=1 << 30, stride=1 << 30), UNSUPPORTED), (dict(lengths=FAKE + 2), ALIGNMENT), (dict(table=FAKE + 1), ALIGNMENT)]


@pytest.mark.parametrize("change,status", CACHE_FAULTS)
def test_cache_faults(B, change, status):
    c = cache(B, **change)
    assert attention(B, c=c) == status
    assert B.lib().vitint_cache_weigh(FAKE, BF16, 3, 8, 1024, 128, FAKE, c, batch(B), 0.1, 1, 0, None, FAKE, FAKE, 1 << 30, None) == status
    assert B.lib().vitint_cache_evict(c, batch(B), FAKE, 16, 0, 0, FAKE, 1, FAKE, FAKE + 4096, None) == status
    assert B.lib().vitint_paged_attention_workspace_bytes(8, c, batch(B)) == 0 == B.lib().vitint_cache_weigh_workspace_bytes(c, batch(B))


@pytest.mark.parametrize("change,status", BATCH_FAULTS)
def test_batch_faults(B, change, status):
    b = batch(B, **change)
    assert attention(B, b=b) == status
    assert B.lib().vitint_cache_weigh(FAKE, BF16, 3, 8, 1024, 128, FAKE, cache(B), b, 0.1, 1, 0, None, FAKE, FAKE, 1 << 30, None) == status
    if "starts" not in change and "max_queries" not in change:
        assert B.lib().vitint_cache_evict(cache(B), b, FAKE, 16, 0, 0, FAKE, 1, FAKE, FAKE + 4096, None) == status


@pytest.mark.parametrize("change,status", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(tokens=0), INVALID), (dict(q_heads=0), INVALID), (dict(q_heads=7), INVALID), (dict(q_type=F32), INVALID),
    (dict(q_type=F16), INVALID), (dict(q_heads=2 * 129), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(causal=2), INVALID), (dict(window=-1), INVALID), (dict(causal=0, window=4), INVALID), (dict(q=FAKE + 8), ALIGNMENT),
    (dict(q_token=1028), ALIGNMENT), (dict(q_head=130), ALIGNMENT), (dict(q_head=64), INVALID), (dict(q_token=0), INVALID), (dict(out=FAKE + 4), ALIGNMENT),
    (dict(out_token=1001), ALIGNMENT), (dict(out_head=64), INVALID), (dict(out_token=-1024), INVALID), (dict(), WORKSPACE), (dict(workspace=FAKE), WORKSPACE),
    (dict(workspace=FAKE + 16, size=1 << 30), WORKSPACE), (dict(tokens=1 << 25), UNSUPPORTED), (dict(lse=FAKE + 2), ALIGNMENT)])
def test_attention_faults(B, change, status):
    assert attention(B, **change) == status


def test_weigh_faults(B):
    f = lambda lse=FAKE, out=FAKE, work=FAKE, size=1 << 30: B.lib().vitint_cache_weigh(FAKE, BF16, 3, 8, 1024, 128, lse, cache(B), batch(B), 0.1, 1, 0, None, out,
                                                                                        work, size, None)
    assert f(lse=None) == INVALID and f(out=None) == INVALID and f(work=None) == WORKSPACE and f(work=FAKE + 8) == WORKSPACE and f(size=8) == WORKSPACE


@pytest.mark.parametrize("change,status", [
    (dict(weights=None), INVALID), (dict(kept=None), INVALID), (dict(counts=None), INVALID), (dict(table=None), INVALID), (dict(budget=0), INVALID), (dict(budget=-4), INVALID),
    (dict(sinks=-1), INVALID), (dict(recent=-1), INVALID), (dict(sinks=9, recent=8), INVALID), (dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), INVALID), (dict(stride=0), INVALID),
    (dict(budget=17), INVALID), (dict(counts=FAKE), INVALID), (dict(table=FAKE), INVALID), (dict(kept=FAKE + 2), ALIGNMENT), (dict(weights=FAKE + 1), ALIGNMENT)])
def test_evict_faults(B, change, status):
    f = dict(cache=cache(B), batch=batch(B), weights=FAKE, budget=16, sinks=0, recent=0, table=FAKE + 64, stride=1, kept=FAKE, counts=FAKE + 4096, stream=None) | change
    assert B.lib().vitint_cache_evict(*f.values()) == status


def rotate(B, c=None, **change):
    f = dict(q=FAKE, k=FAKE, v=FAKE, tokens=4, q_stride=2048, k_stride=2048, v_stride=2048, q_heads=8, kv_heads=2, head_dim=128, in_type=BF16, norm=1, eps=1e-6,
             q_gain=FAKE, k_gain=FAKE, q_offset=0, k_offset=0, positions=FAKE, frequencies=FAKE, rotary=128, pairs=0, q_out=FAKE, k_out=0, q_out_stride=2048,
             k_out_stride=0, out_type=BF16, reserved=0, slots=FAKE, weights=0) | change
    return B.lib().vitint_qk_norm_rotate(B._PACK_ROTATE(*f.values()), None if c == 0 else c or cache(B), None)


@pytest.mark.parametrize("change,status", [
    (dict(k=0), INVALID), (dict(q=0), INVALID), (dict(q_out=0), INVALID), (dict(tokens=0), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=3), INVALID), (dict(q_heads=-1), INVALID),
    (dict(in_type=I8), INVALID), (dict(out_type=F32), INVALID), (dict(out_type=F16), INVALID), (dict(norm=3), INVALID), (dict(norm=-1), INVALID), (dict(pairs=2), INVALID),
    (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=64), INVALID), (dict(rotary=130), INVALID), (dict(rotary=-2), INVALID), (dict(rotary=24), UNSUPPORTED), (dict(positions=0), INVALID),
    (dict(frequencies=0), INVALID), (dict(k_gain=0), INVALID), (dict(q_gain=0), INVALID), (dict(norm=0), INVALID), (dict(k_offset=FAKE), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(v=0), INVALID), (dict(slots=0), INVALID), (dict(q=FAKE + 8), ALIGNMENT), (dict(k=FAKE + 4), ALIGNMENT), (dict(q_stride=1025), ALIGNMENT),
    (dict(k_stride=200), INVALID), (dict(q_out_stride=512), INVALID), (dict(q_gain=FAKE + 4), ALIGNMENT), (dict(k_out=FAKE, k_out_stride=256, in_type=F32), INVALID),
    (dict(q_out_stride=1024), INVALID), (dict(tokens=1 << 25), UNSUPPORTED), (dict(slots=FAKE + 4), ALIGNMENT), (dict(frequencies=FAKE + 4), ALIGNMENT),
    (dict(positions=FAKE + 2), ALIGNMENT)])
def test_rotate_faults(B, change, status):
    if "k_out" in change:
        change = change | dict(k=FAKE)
    assert rotate(B, **change) == status


def test_rotate_without_a_cache(B):
    assert rotate(B, c=0) == INVALID                                                    # v and slots need one
    assert rotate(B, c=0, v=0, slots=0) == INVALID                                      # keys would go nowhere
    assert rotate(B, c=0, v=0, slots=0, k_out=FAKE + 16, k_out_stride=256, weights=FAKE) == INVALID


def test_the_binding_checks_its_tensors(B, monkeypatch):
    monkeypatch.setattr(B, "_cuda_device", lambda: -1)                                  # the CPU, where nothing is launched
    monkeypatch.setattr(B, "_stream", lambda: 0)
    c = lambda **k: B.PagedCache(**(dict(k=torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), v=torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)) | k))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    b = lambda **k: B.CacheBatch(**(dict(page_table=i32(2, 4), lengths=i32(2), query_starts=i32(3), max_queries=1, max_length=64) | k))
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    steps = torch.zeros(4, 2, 16)
    bad = [
        (q, c(v=torch.zeros(4, 2, 16, 64)), b()), (q, c(v=torch.zeros(4, 2, 32, 64, dtype=torch.bfloat16)), b()), (q, c(k_steps=steps, v_steps=steps), b()),
        (q, c(k=torch.zeros(4, 2, 16, 64), v=torch.zeros(4, 2, 16, 64)), b()), (q, c(k=torch.zeros(4, 2, 16, 64, dtype=torch.int8), v=torch.zeros(4, 2, 16, 64, dtype=torch.int8)), b()),
        (q[..., :32], c(), b()), (q[0], c(), b()), (q.transpose(1, 2).contiguous().transpose(1, 2), c(), b()), (q, c(), b(page_table=i32(3, 4))),
        (q, c(), b(page_table=i32(2, 4).long())), (q, c(), b(lengths=i32(2).float())), (q, c(), b(query_starts=i32(2))), (q, c(), b(query_starts=None)), (q, c(), b(max_length=65)),
        (q, c(), b(max_length=0)), (q, c(), b(max_queries=-1)), (q, c(), b(page_table=i32(2, 8)[:, ::2])), (q.float(), c(), b()), (q.half(), c(), b()),
        (q, c(k=torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16).transpose(1, 2), v=torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)), b()),
    ]
    for args in bad:
        with pytest.raises(B.VitintError):
            B.vitint_paged_attention(*args, 0.1)
    with pytest.raises(B.VitintError):
        B.vitint_paged_attention(q, c(), b(), 0.1, out=q.float())
    with pytest.raises(B.VitintError):
        B.vitint_paged_attention(q, c(), b(), 0.1, lse=torch.zeros(2, 3))
    with pytest.raises(B.VitintError):
        B.vitint_cache_weigh(q, torch.zeros(2, 4), c(), b(), 0.1, None, torch.zeros(4, 2, 17))
    with pytest.raises(B.VitintError):
        B.vitint_cache_evict(c(), b(), steps, 40, i32(2, 2))
    with pytest.raises(B.VitintError):
        B.vitint_cache_evict(c(), b(), steps, 0, i32(2, 2))
    rows = torch.zeros(3, 128, dtype=torch.bfloat16)
    for change in (dict(v=None), dict(slots=None), dict(slots=i32(3)), dict(norm="batch"), dict(frequencies=torch.zeros(32)), dict(positions=None), dict(q=rows[:2]), dict(q=rows.float()),
                   dict(q_out=torch.zeros(3, 2, 64)), dict(weights=torch.zeros(5)), dict(k_gain=torch.zeros(63))):
        f = dict(q=rows, k=rows, v=rows, head_dim=64, q_gain=torch.zeros(64), k_gain=torch.zeros(64), positions=i32(3), frequencies=torch.zeros(32, dtype=torch.float64), cache=c(),
                 slots=torch.zeros(3, dtype=torch.int64)) | change
        with pytest.raises(B.VitintError):
            B.vitint_qk_norm_rotate(**f)


@pytest.mark.parametrize("change", [
    dict(sequences=18705, max_length=57404 * 64, stride=1 << 20),                       # 2 heads x 57,404 tiles of 64: 2^31 - 8 tiles
    dict(sequences=65535, max_length=1 << 24, stride=1 << 20),
    dict(sequences=65535, max_length=1 << 24, stride=1 << 20, max_queries=2 ** 31 - 1)])
def test_more_tiles_than_the_plan_counts(B, change):
    """The plan rounds up to the CTAs' stretches in 32 bits: calls that come near 2^31 tiles are refused before anything else is done with them."""
    work = dict(workspace=FAKE, size=1 << 40)
    assert attention(B, b=batch(B, **change), tokens=(1 << 24) - 1, **work) == UNSUPPORTED
    weigh = lambda **c: B.lib().vitint_cache_weigh(FAKE, BF16, (1 << 24) - 1, 8, 1024, 128, FAKE, cache(B), batch(B, **c), 0.1, 1, 0, None, FAKE, FAKE, 1 << 40, None)
    if change["sequences"] == 65535:
        assert weigh(**change) == UNSUPPORTED
    assert weigh(**change | dict(max_length=14351 * 256, max_queries=4 * 32)) == UNSUPPORTED            # 4 runs of queries: the same number


def test_the_binding_refuses_what_its_types_do_not_hold(B, monkeypatch):
    """Counts beyond 32 bits (which would be cut to something else), and tensors of other orders: the library's error, not a wrong call or another error."""
    monkeypatch.setattr(B, "_cuda_device", lambda: -1)                                  # the CPU: every call below is refused before the library is entered
    monkeypatch.setattr(B, "_stream", lambda: 0)
    text = B.lib().vitint_status_string

    class Closed:
        def __getattr__(self, name):
            return text if name == "vitint_status_string" else pytest.fail(f"{name} was entered")

    monkeypatch.setattr(B, "lib", Closed)
    c = B.PagedCache(torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16))
    flat = B.PagedCache(torch.zeros(4, 32, 64, dtype=torch.bfloat16), torch.zeros(4, 32, 64, dtype=torch.bfloat16))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    b = B.CacheBatch(i32(2, 4), i32(2), i32(3), 1, 64)
    q, weights, lse, rows = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 16), torch.zeros(2, 4), torch.zeros(3, 128, dtype=torch.bfloat16)
    for window in (1 << 31, (1 << 32) + 5, -1, -(1 << 32)):
        with pytest.raises(B.VitintError):
            B.vitint_paged_attention(q, c, b, 0.1, window=window)
        with pytest.raises(B.VitintError):
            B.vitint_cache_weigh(q, lse, c, b, 0.1, None, weights, window=window)
    for change in (dict(sinks=1 << 32), dict(recent=(1 << 32) + 1), dict(sinks=-1), dict(recent=-(1 << 32))):
        with pytest.raises(B.VitintError):
            B.vitint_cache_evict(c, b, weights, 4, i32(2, 2), **change)
    for call in (lambda: B.vitint_paged_attention(q, flat, b, 0.1), lambda: B.vitint_cache_weigh(q, lse, flat, b, 0.1, None, weights),
                 lambda: B.vitint_cache_evict(flat, b, weights, 4, i32(2, 2)), lambda: B.vitint_qk_norm_rotate(rows, rows[0], rows, 64, norm="none"),
                 lambda: B.vitint_qk_norm_rotate(rows[0], rows, None, 64, norm="none"), lambda: B.vitint_qk_norm_rotate(rows, rows, None, 0, norm="none"),
                 lambda: B.vitint_qk_norm_rotate(rows, rows, None, -64, norm="none"), lambda: B.vitint_qk_norm_rotate(rows, rows, None, 1 << 40, norm="none")):
        with pytest.raises(B.VitintError):
            call()

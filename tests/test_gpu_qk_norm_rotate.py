"""Head norms, rotation and the store in the cache against their definition in 64 bits."""
import pytest
import torch

import paper_2504_18547_b200 as vt

pytestmark = pytest.mark.gpu

BF16, F16, F32, I8 = torch.bfloat16, torch.float16, torch.float32, torch.int8
EPS = {BF16: 2.0 ** -7, F16: 2.0 ** -10}


def definition(x, norm, eps, gain, offset, positions, frequencies, pairs):
    """x [tokens, heads, d] in 64 bits; and the tolerance of an fp32 evaluation: every one of about d + 30 roundings (sums of d squares, the
    norm, two products and a sum) is 2^-24 of the operands' size, and the angle's fp32 turn is off by 2^-24 of a turn, 2 pi 2^-24 rad."""
    y = x.double()
    d = y.shape[2]
    size = y.abs()
    if norm == "rms":
        r = 1 / torch.sqrt(y.square().mean(2, keepdim=True) + eps)
        y, size = y * r * gain, size * r * gain.abs()
    elif norm == "layer":
        c = y - y.mean(2, keepdim=True)
        r = 1 / torch.sqrt(c.square().mean(2, keepdim=True) + eps)
        size = (size + y.abs().mean(2, keepdim=True)) * r * gain.abs() + offset.abs()
        y = c * r * gain + offset
    n = len(frequencies)
    if n:
        a = positions.double()[:, None] * frequencies
        cos, sin = a.cos()[:, None], a.sin()[:, None]
        one, two = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if pairs else (slice(0, n), slice(n, 2 * n))
        z, s = y.clone(), size.clone()
        z[..., one], z[..., two] = y[..., one] * cos - y[..., two] * sin, y[..., two] * cos + y[..., one] * sin
        s[..., one] = s[..., two] = size[..., one] + size[..., two]
        y, size = z, s
    return y, size * (d + 60) * 2.0 ** -24


def run(seed, tokens, dim, hq, hk, norm, pairs, rotary, itype, otype, codes, places=16, far=1000, weights=True, k_out=True):
    g = torch.Generator().manual_seed(seed)
    rows = (torch.randn(tokens, (hq + 2 * hk) * dim + 16, generator=g) * 2 + 0.3).to(itype)
    q, k, v = (rows[:, a * dim:b * dim] for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    gain, offset = [torch.randn(dim, generator=g) for _ in range(2)], [torch.randn(dim, generator=g) for _ in range(2)]
    positions = torch.randint(0, far, (tokens,), generator=g, dtype=torch.int32)
    positions[0] = far
    freq = 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))
    pages = tokens // places + 2
    cache = vt.PagedCache.empty(pages, hk, places, dim, I8 if codes else otype)
    cache.k.fill_(5), cache.v.fill_(5)
    if codes:
        cache.k_steps.fill_(9), cache.v_steps.fill_(9)
    w = torch.full((pages, hk, places), 3.0, device="cuda")
    slots = torch.randperm(pages * places, generator=g)[:tokens]
    if tokens > 3:
        slots[1], slots[2] = -1, pages * places                                       # neither is stored
    on = lambda t: t.cuda()
    rd = rows.cuda()
    qd, kd, vd = (rd[:, a * dim:b * dim] for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk)))
    ko = torch.empty(tokens, hk, dim, dtype=otype, device="cuda") if k_out else None
    q_out, k_got = vt.vitint_qk_norm_rotate(
        qd, kd, vd, dim, norm=norm, eps=1e-5, q_gain=on(gain[0]) if norm != "none" else None, k_gain=on(gain[1]) if norm != "none" else None,
        q_offset=on(offset[0]) if norm == "layer" else None, k_offset=on(offset[1]) if norm == "layer" else None, positions=on(positions),
        frequencies=on(freq), pairs=pairs, out_dtype=otype, k_out=ko, cache=cache, slots=on(slots), weights=w if weights else None)
    assert vt.vitint_device_status() == 0
    want = []
    for i, (x, heads) in enumerate(((q, hq), (k, hk))):
        want.append(definition(x.reshape(tokens, heads, dim), norm, 1e-5, gain[i].double(), offset[i].double(), positions, freq, pairs))
    want.append((v.reshape(tokens, hk, dim).double(), torch.zeros(tokens, hk, dim, dtype=torch.float64)))
    half = EPS[otype] / 2
    least = 2.0 ** -25 if otype == F16 else 0.0

    def near(got, y, tol):
        off = (got.double().cpu() - y).abs()
        assert bool((off <= half * (y.abs() + tol) + tol + least).all()), float((off - half * y.abs() - tol).max())

    near(q_out, *want[0])
    if k_out:
        near(k_got, *want[1])
    stored = (slots >= 0) & (slots < pages * places)
    at = slots[stored]
    touched = torch.zeros(pages, places, dtype=torch.bool)
    touched[at // places, at % places] = True
    for name, (y, tol) in (("k", want[1]), ("v", want[2])):
        x = getattr(cache, name).cpu()
        assert bool((x.permute(0, 2, 1, 3)[~touched] == 5).all())
        x, y, tol = x[at // places, :, at % places], y[stored], tol[stored]
        if not codes:
            near(x, y, tol)
            continue
        steps = getattr(cache, name + "_steps").cpu()
        assert bool((steps.permute(0, 2, 1)[~touched] == 9).all())
        steps = steps[at // places, :, at % places].double()
        top, slack = y.abs().amax(2), tol.amax(2)
        assert bool(((steps * 127 - top).abs() <= slack + top * 2.0 ** -22).all())
        # a code is the nearest level: the value is at most half a step away, and the roundings of value and quotient
        value = x.double() * steps[..., None]
        assert bool(((value - y).abs() <= steps[..., None] * 0.5 + 2 * tol + 4 * slack[..., None] + 2.0 ** -20 * top[..., None]).all())
        assert int(x.abs().amax()) <= 127
    if weights:
        assert bool((w.cpu().permute(0, 2, 1)[touched] == 0).all()) and bool((w.cpu().permute(0, 2, 1)[~touched] == 3).all())
    else:
        assert bool((w == 3).all())


@pytest.mark.parametrize("itype,otype,codes", [(BF16, BF16, False), (F16, F16, False), (F32, BF16, False), (F32, F16, True), (BF16, BF16, True),
                                               (F16, BF16, False), (BF16, F16, True)])
@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("dim", [64, 128])
def test_types_and_norms(dim, norm, itype, otype, codes):
    run(1, 37, dim, 6, 2, norm, False, dim, itype, otype, codes)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dim,rotary", [(64, 0), (64, 16), (64, 32), (64, 48), (128, 16), (128, 96), (128, 112), (128, 128)])
def test_rotary_dimensions(dim, rotary, pairs):
    run(2, 9, dim, 3, 1, "rms", pairs, rotary, BF16, BF16, False)


@pytest.mark.parametrize("tokens", [1, 2, 63, 1000])
@pytest.mark.parametrize("hq,hk", [(1, 1), (12, 12), (32, 8), (7, 1)])
def test_tokens_and_heads(tokens, hq, hk):
    run(3, tokens, 128, hq, hk, "rms", False, 128, BF16, BF16, True, places=64, weights=tokens != 2, k_out=tokens != 63)


def test_far_positions():
    """At position 10^9 the angle's fp64 product keeps 10^9 2^-53 rad; an fp32 one would be off by whole turns."""
    run(4, 50, 128, 4, 2, "rms", False, 128, F32, BF16, False, far=1000000000)


def test_in_place_without_a_cache():
    g = torch.Generator().manual_seed(5)
    x = torch.randn(21, 5 * 64, generator=g).to(BF16)
    positions, freq = torch.arange(21, dtype=torch.int32), 100.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    one = torch.ones(64)
    y, tol = definition(x.view(21, 5, 64), "rms", 1e-6, one.double(), None, positions, freq, False)
    d = x.cuda()
    q, k = d[:, :192], d[:, 192:]
    q3 = q.view(21, 3, 64) if q.is_contiguous() else q.unflatten(1, (3, 64))
    vt.vitint_qk_norm_rotate(q, k, None, 64, q_gain=one.cuda(), k_gain=one.cuda(), positions=positions.cuda(), frequencies=freq.cuda(),
                             q_out=q3, k_out=k.unflatten(1, (2, 64)))
    off = (d.view(21, 5, 64).double().cpu() - y).abs()
    assert bool((off <= EPS[BF16] / 2 * (y.abs() + tol) + tol).all())


def test_rows_of_zeros():
    """RMS of zeros with eps 0 would be 0/0; with eps they stay zeros, and their step is 0."""
    z = torch.zeros(4, 128, device="cuda")
    cache = vt.PagedCache.empty(1, 1, 16, 128, I8)
    one = torch.ones(128, device="cuda")
    q, _ = vt.vitint_qk_norm_rotate(z, z, z, 128, q_gain=one, k_gain=one, cache=cache, slots=torch.arange(4, device="cuda"), out_dtype=BF16)
    assert not bool(q.any()) and not bool(cache.k[0, 0, :4].any()) and not bool(cache.k_steps[0, 0, :4].any()) and not bool(cache.v_steps[0, 0, :4].any())


def test_other_stream_and_replay():
    g = torch.Generator().manual_seed(6)
    x = torch.randn(8, 3 * 128, generator=g, ).to(BF16).cuda()
    cache = vt.PagedCache.empty(2, 1, 16, 128)
    one, slots = torch.ones(128, device="cuda"), torch.arange(8, device="cuda")
    positions, freq = torch.arange(8, dtype=torch.int32, device="cuda"), torch.ones(64, dtype=torch.float64, device="cuda") / 7
    call = lambda q_out=None: vt.vitint_qk_norm_rotate(x[:, :128], x[:, 128:256], x[:, 256:], 128, q_gain=one, k_gain=one, positions=positions,
                                                       frequencies=freq, cache=cache, slots=slots, q_out=q_out)[0]
    want, want_k = call().clone(), cache.k.clone()
    q_out = torch.empty_like(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(q_out)
    slots.add_(8)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(q_out, want) and torch.equal(cache.k[0, 0, 8:], want_k[0, 0, :8])


def test_one_token_of_rows_of_any_width():
    """A single row's stride is nothing that is stepped by: here 388 elements, no multiple of 16 bytes, and other outputs' likewise."""
    g = torch.Generator().manual_seed(7)
    rows = torch.randn(3, 388, generator=g).to(BF16).cuda()
    row = rows[2:3]                                                                    # (1552 bytes in: aligned)
    outs = [torch.zeros(1, 260, dtype=BF16, device="cuda").as_strided((1, n, 128), (131, 128, 1)) for n in (1, 1)]
    one = torch.ones(128, device="cuda")
    make = lambda: vt.PagedCache.empty(1, 1, 16, 128)
    given, plain = make(), make()
    for cache in (given, plain):
        cache.k.zero_(), cache.v.zero_()
    slot = torch.tensor([5], device="cuda")
    q, k = vt.vitint_qk_norm_rotate(row[:, :128], row[:, 128:256], row[:, 256:384], 128, q_gain=one, k_gain=one, q_out=outs[0], k_out=outs[1], cache=given, slots=slot)
    parts = [row[:, i:i + 128].contiguous() for i in (0, 128, 256)]
    q2, _ = vt.vitint_qk_norm_rotate(*parts, 128, q_gain=one, k_gain=one, cache=plain, slots=slot)
    assert torch.equal(q, q2) and torch.equal(k[0, 0], plain.k[0, 0, 5]) and torch.equal(given.k, plain.k) and torch.equal(given.v, plain.v)


@pytest.mark.parametrize("codes", [False, True])
def test_a_cache_with_places_outside_heads(codes):
    g = torch.Generator().manual_seed(8)
    x = torch.randn(30, 4 * 64, generator=g).to(BF16).cuda()
    plain = vt.PagedCache.empty(3, 2, 16, 64, I8 if codes else BF16)
    views = [torch.empty(3, 16, 2, 64, dtype=plain.k.dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    turned = vt.PagedCache(*views, *(None if s is None else torch.empty_like(s) for s in (plain.k_steps, plain.v_steps)))
    slots, one = torch.randperm(48, generator=g)[:30].cuda(), torch.ones(64, device="cuda")
    for c in (plain, turned):
        for t in (c.k, c.v, c.k_steps, c.v_steps):
            if t is not None:
                t.fill_(3)
        vt.vitint_qk_norm_rotate(None, x[:, :128], x[:, 128:], 64, k_gain=one, cache=c, slots=slots, out_dtype=BF16)
    for name in ("k", "v") + (("k_steps", "v_steps") if codes else ()):
        assert torch.equal(getattr(plain, name), getattr(turned, name)), name
    assert not bool((plain.k == 3).all())


def test_keys_alone_and_a_layer_norm_without_an_offset():
    g = torch.Generator().manual_seed(9)
    x, gain = torch.randn(33, 3 * 128, generator=g) + 0.5, torch.randn(128, generator=g)
    positions, freq = torch.arange(33, dtype=torch.int32), 50.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)
    y, tol = definition(x.view(33, 3, 128), "layer", 1e-6, gain.double(), torch.zeros(128, dtype=torch.float64), positions, freq, True)
    _, k = vt.vitint_qk_norm_rotate(None, x.cuda(), None, 128, norm="layer", k_gain=gain.cuda(), positions=positions.cuda(), frequencies=freq.cuda(), pairs=True,
                                    out_dtype=F16)
    off = (k.double().cpu() - y).abs()
    assert bool((off <= EPS[F16] / 2 * (y.abs() + tol) + tol + 2.0 ** -25).all())

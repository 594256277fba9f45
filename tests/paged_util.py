"""Helpers for the tests of the paged cache: random caches and batches, and the operators' definitions in 64 bits (loops, on the CPU)."""
from __future__ import annotations

import math

import torch

import paper_2504_18547_b200 as vt

EPS = {torch.bfloat16: 2.0 ** -7, torch.float16: 2.0 ** -10}


def random_cache(g, pages, heads, places, dim, dtype, junk=None, layout="hpd", k_size=1.0, v_size=0.5):
    """A cache of N(0, k_size) keys and N(0, v_size) values.  junk: every place is first filled with this (NaN for 16-bit values; codes get
    -128 and their steps the junk), to be overwritten by `fill`.  layout "phd": places outside heads (strided views)."""
    shape = (pages, heads, places, dim) if layout == "hpd" else (pages, places, heads, dim)
    def make(size):
        if dtype == torch.int8:
            x = torch.randint(-127, 128, shape, generator=g, dtype=torch.int8)
        else:
            x = (torch.randn(shape, generator=g) * size).to(dtype)
        return x if layout == "hpd" else x.transpose(1, 2)
    k, v = make(k_size), make(v_size)
    steps = [None, None]
    if dtype == torch.int8:
        steps = [(torch.rand((pages, heads, places), generator=g) + 0.5) * s / 64 for s in (k_size, v_size)]
    return vt.PagedCache(k, v, *steps)


def to_gpu(cache):
    def move(t):
        if t is None:
            return None
        if t.is_contiguous():
            return t.cuda()
        return t.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    return vt.PagedCache(move(cache.k), move(cache.v), move(cache.k_steps), move(cache.v_steps))


def random_table(g, lengths, places, pages):
    """Pages in no order, -1 behind each sequence's last."""
    need = [-(-n // places) for n in lengths]
    assert sum(need) <= pages
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lengths), max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table


def spoil_unused(cache, table, lengths, junk=float("nan")):
    """Whatever lies behind the sequences' lengths: NaN."""
    places = cache.k.shape[2]
    used = torch.zeros(cache.k.shape[0], places, dtype=torch.bool)
    for b, n in enumerate(lengths):
        for j in range(n):
            used[int(table[b, j // places]), j % places] = True
    for x, steps in ((cache.k, cache.k_steps), (cache.v, cache.v_steps)):
        if steps is not None:
            steps.permute(0, 2, 1)[~used] = junk
        else:
            x.permute(0, 2, 1, 3)[~used] = junk


def gathered(cache, table_row, length, head, which):
    """[length, dim] in 64 bits."""
    places = cache.k.shape[2]
    x, steps = (cache.k, cache.k_steps) if which == "k" else (cache.v, cache.v_steps)
    j = torch.arange(length)
    page = table_row[j // places].long()
    out = x[page, head, j % places].double()
    return out if steps is None else out * steps[page, head, j % places].double()[:, None]


def visible(length, new, causal, window):
    pos = torch.arange(new)[:, None] + (length - new)
    j = torch.arange(length)[None, :]
    see = torch.ones(new, length, dtype=torch.bool)
    if causal:
        see &= j <= pos
        if window:
            see &= j > pos - window
    return see


def attention64(q, cache, table, lengths, starts, scale, causal, window):
    """(out, lse, tolerance of out, tolerance of lse, rows that belong to a sequence) in 64 bits.

    A kernel that keeps scores, maxima and sums in fp32, rounds each probability (times a step) to the type T or more finely before the second
    contraction and the output once is off by at most
      eps/2 |o|                          the output's rounding (eps/2 is half a step of T),
      eps/2 sum p |v|                    the probabilities' rounding (normal ones),
      2^-25 L max|v|                     fp16 and codes: probabilities (times steps) below fp16's normal range, relative to a
                                         maximum of 1 or more (times the power of two of the largest step),
      (2 ds + 2^-19) sum p |v|           ds: error of a score, (d + 4) 2^-24 scale sum |q||k| for d products and their sum, the step and
                                         the scale, and 2^-24 |s| each for the maximum's subtraction; the sum of exponentials has it
                                         too; 2^-19 covers ex2's 2^-22, the sums' and rescalings' roundings.
    """
    t, heads, d = q.shape
    group = heads // cache.k.shape[1]
    out, lse = torch.zeros(t, heads, d, dtype=torch.float64), torch.full((t, heads), -math.inf, dtype=torch.float64)
    tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    mine = torch.zeros(t, dtype=torch.bool)
    half = EPS[q.dtype] / 2
    for b, length in enumerate(lengths):
        first, new = int(starts[b]), int(starts[b + 1]) - int(starts[b])
        mine[first:first + new] = True
        if length == 0 or new == 0:
            continue
        see = visible(length, new, causal, window)
        for h in range(heads):
            k, v = (gathered(cache, table[b], length, h // group, x) for x in "kv")
            x = q[first:first + new, h].double()
            s = (x @ k.T) * scale
            ds = (d + 4) * 2.0 ** -24 * ((x.abs() @ k.abs().T) * scale).masked_fill(~see, 0).amax(1) + 2.0 ** -22 * s.masked_fill(~see, 0).abs().amax(1)
            s = s.masked_fill(~see, -math.inf)
            z = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(z == -math.inf, torch.zeros_like(z), z)[:, None])
            o = p @ v
            out[first:first + new, h], lse[first:first + new, h] = o, z
            pv = p @ v.abs()
            tol[first:first + new, h] = half * o.abs() + (half * 1.01 + 2 * ds[:, None] + 2.0 ** -19) * pv
            if q.dtype == torch.float16 or cache.k.dtype == torch.int8:
                tol[first:first + new, h] += 2.0 ** -25 * length * v.abs().max()
            lse_tol[first:first + new, h] = ds + 2.0 ** -19 + 2.0 ** -22 * z.abs().masked_fill(z == -math.inf, 0)
    return out, lse, tol, lse_tol, mine


def check_attention(got, lse, want):
    out64, lse64, tol, lse_tol, mine = want
    got, lse = got.double().cpu(), lse.double().cpu()
    off = (got - out64).abs()
    assert bool((off[mine] <= tol[mine]).all()), f"off by {float((off - tol)[mine].max())} more than allowed; largest {float(off[mine].max())}"
    empty = lse64 == -math.inf
    assert bool((lse[mine & empty.all(1)] == -math.inf).all())
    rows = mine[:, None] & ~empty
    assert bool(((lse - lse64).abs()[rows] <= lse_tol[rows]).all()), float(((lse - lse64).abs() - lse_tol)[rows].max())

"""The work that a decoder's paged cache brings, as cases that can be timed and compared.

Four operators that are used together by a program that generates token by token next to the integerized linears:

  rotate     the norm of every query and key head, the rotation by the token's position, and the store of keys and values in the cache
  attention  queries of a chunk of new tokens (one token included) over all that the cache holds for their sequence
  weigh      the attention weight that every cached token received from those queries, added to what it had
  evict      the tokens of largest accumulated weight kept, and moved together into fewer pages

The cache holds 16-bit values, or signed 8-bit codes with a step for each token and head (applied behind the contraction, as in the
linears).  Sizes are generic ones of such programs, or the head counts and dimensions of the repository's configurations (12 heads of
64 channels).  Sequences of a batch have the lengths that `_lengths` spreads below the case's largest, so `work` can count them.
Forward only, as the library is.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one sequence, one token, heads of the repository's ViT-Base: what an interactive user waits for
        {"name": "decode_one", "op": "attention", "seqs": 1, "new": 1, "len": 777, "ragged": False, "q_heads": 12, "kv_heads": 12,
         "dim": 64, "page": 16, "type": "bf16", "codes": False, "causal": True, "window": 0},
        # a serving batch in full swing: one token each, contexts from a few tokens to 8192, grouped heads
        {"name": "decode_batch", "op": "attention", "seqs": 48, "new": 1, "len": 8192, "ragged": True, "q_heads": 32, "kv_heads": 8,
         "dim": 128, "page": 16, "type": "bf16", "codes": False, "causal": True, "window": 0},
        # the same with an 8-bit cache and larger pages
        {"name": "decode_codes", "op": "attention", "seqs": 64, "new": 1, "len": 6001, "ragged": True, "q_heads": 32, "kv_heads": 8,
         "dim": 128, "page": 64, "type": "bf16", "codes": True, "causal": True, "window": 0},
        # two long documents and a few drafted tokens each: all the parallelism lies along the keys
        {"name": "draft_long", "op": "attention", "seqs": 2, "new": 3, "len": 131072, "ragged": False, "q_heads": 16, "kv_heads": 4,
         "dim": 128, "page": 32, "type": "f16", "codes": False, "causal": True, "window": 0},
        # prompts of odd lengths behind shared prefixes, with a sliding window, in one call
        {"name": "chunk_ragged", "op": "attention", "seqs": 7, "new": 701, "len": 2999, "ragged": True, "q_heads": 12, "kv_heads": 4,
         "dim": 64, "page": 16, "type": "f16", "codes": False, "causal": True, "window": 1021},
        # a chunk of a long prompt over what is cached of it: the largest call
        {"name": "chunk_long", "op": "attention", "seqs": 1, "new": 2048, "len": 18432, "ragged": False, "q_heads": 32, "kv_heads": 8,
         "dim": 128, "page": 64, "type": "bf16", "codes": False, "causal": True, "window": 0},
        # the tokens of one decoding step, out of a fused projection into a 16-bit cache
        {"name": "rotate_step", "op": "rotate", "tokens": 64, "q_heads": 32, "kv_heads": 8, "dim": 128, "rotary": 128, "pairs": False,
         "norm": "rms", "input": "bf16", "type": "bf16", "codes": False, "page": 16, "position": 8191},
        # a prompt out of a projection that dequantizes to fp32, into an 8-bit cache, at far positions
        {"name": "rotate_prompt", "op": "rotate", "tokens": 8190, "q_heads": 24, "kv_heads": 8, "dim": 128, "rotary": 96, "pairs": True,
         "norm": "layer", "input": "f32", "type": "bf16", "codes": True, "page": 32, "position": 1000000},
        # the weights that one decoding step gives a batch's tokens
        {"name": "weigh_step", "op": "weigh", "seqs": 32, "new": 1, "len": 4096, "ragged": True, "q_heads": 32, "kv_heads": 8,
         "dim": 128, "page": 16, "type": "bf16", "codes": False, "causal": True, "window": 0},
        # the weights that a prompt's last chunk gives all of it, before the prompt is thinned out
        {"name": "weigh_chunk", "op": "weigh", "seqs": 1, "new": 1023, "len": 12287, "ragged": False, "q_heads": 32, "kv_heads": 8,
         "dim": 128, "page": 64, "type": "bf16", "codes": True, "causal": True, "window": 0},
        # a batch brought down to its budget after a step
        {"name": "evict_batch", "op": "evict", "seqs": 16, "len": 4097, "ragged": True, "kv_heads": 8, "dim": 128, "page": 16,
         "type": "bf16", "codes": False, "budget": 1024, "sinks": 4, "recent": 256},
        # one long document thinned to a quarter
        {"name": "evict_long", "op": "evict", "seqs": 1, "len": 65536, "ragged": False, "kv_heads": 8, "dim": 128, "page": 64,
         "type": "bf16", "codes": True, "budget": 16384, "sinks": 4, "recent": 2000},
    ]


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "rotate", "weigh", "evict"])
    dim, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 7, 8])
    case = {"op": op, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "page": page, "type": rng.choice(["bf16", "f16"]),
            "codes": rng.random() < 0.4}
    if op == "rotate":
        case |= {"tokens": min(_spread(rng, 1, 8192), 330000000 // ((q_heads + 2 * kv_heads) * dim) // 8 + 1),
                 "rotary": rng.choice([0, 32, dim // 2, dim, dim]), "pairs": rng.random() < 0.5,
                 "norm": rng.choice(["rms", "rms", "layer", "none"]), "input": rng.choice(["bf16", "f16", "f32"]),
                 "position": _spread(rng, 1, 1000000)}
        return case
    if op == "evict":
        length = _spread(rng, 16, 65536)
        seqs = min(_spread(rng, 1, 32), max(1, 65536 // length))
        budget = max(1, int(length * rng.uniform(0.1, 1.1)))
        recent = int(budget * rng.uniform(0, 0.6))
        del case["q_heads"]
        return case | {"seqs": seqs, "len": length, "ragged": rng.random() < 0.5, "budget": budget,
                       "sinks": min(rng.choice([0, 1, 4]), budget - recent), "recent": recent}
    new = 1 if rng.random() < 0.4 else _spread(rng, 2, 1500)
    length = new + _spread(rng, 1, 60000)
    # at most the largest listed case's query and key pairs, and its cache
    pairs = (300000000 if op == "weigh" else 1100000000)
    length = max(new, min(length, pairs // (q_heads * new), 500000000 // (kv_heads * dim)))
    room = min(pairs // (q_heads * new * length), 250000000 // (kv_heads * dim * length))
    seqs = max(1, min(_spread(rng, 1, 64), room))
    causal = rng.random() < 0.85
    window = _spread(rng, 1, length) if causal and rng.random() < 0.25 else 0
    return case | {"seqs": seqs, "new": new, "len": length, "ragged": rng.random() < 0.6, "causal": causal, "window": window}


def _lengths(case):
    """(cached tokens, new tokens) of each sequence; the first has the most of both."""
    out = []
    for i in range(case["seqs"]):
        length, new = case["len"], case.get("new", 1)
        if case["ragged"] and i:
            new = max(1, int(new * ((0.618034 * i + 0.3) % 1.0)))
            length = max(new, int(length * ((0.754878 * i + 0.2) % 1.0) ** 1.5))
        out.append((length, new))
    return out


def _batch(case, generator):
    """Lengths, query starts and page table of the sequences, pages in no order; and how many pages the cache has."""
    lens, page = _lengths(case), case["page"]
    need = [-(-n // page) for n, _ in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=generator, device="cuda", dtype=torch.int32)
    starts = torch.tensor([0] + need, device="cuda").cumsum(0)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device="cuda")
    at = torch.arange(max(need), device="cuda")[None, :]
    inside = at < torch.tensor(need, device="cuda")[:, None]
    table[inside] = order[(starts[:-1, None] + at)[inside]]
    first = [0]
    for _, n in lens:
        first.append(first[-1] + n)
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor([n for _, n in lens], device="cuda"))
    st = {"lengths": torch.tensor([n for n, _ in lens], dtype=torch.int32, device="cuda"),
          "query_starts": torch.tensor(first, dtype=torch.int32, device="cuda"), "table": table, "tokens": first[-1],
          "max_queries": max(n for _, n in lens), "max_length": max(n for n, _ in lens),
          "row_seq": seq, "row_at": torch.arange(first[-1], device="cuda") - torch.tensor(first, device="cuda")[seq]}
    return st, pages


def _cache(case, pages, generator):
    """Keys and values for every place of every page: N(0, 1) keys (they come out of a norm), N(0, 1/4) values."""
    shape = (pages, case["kv_heads"], case["page"], case["dim"])
    st = {}
    for name, size in (("k", 1.0), ("v", 0.5)):
        if case["codes"]:
            st[name] = torch.randn(shape, generator=generator, device="cuda", dtype=torch.float16).mul_(38.0).round_().clamp_(-127, 127).to(torch.int8)
            st[name + "_steps"] = torch.rand(shape[:3], generator=generator, device="cuda").add_(0.6).mul_(size / 38.0)
        else:
            st[name] = torch.randn(shape, generator=generator, device="cuda", dtype=_TYPES[case["type"]]).mul_(size)
            st[name + "_steps"] = None
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    d, ty = case["dim"], _TYPES[case["type"]]
    st = {"case": case}
    if case["op"] == "rotate":
        t, hq, hk, page = case["tokens"], case["q_heads"], case["kv_heads"], case["page"]
        st["qkv"] = torch.randn((t, (hq + 2 * hk) * d), generator=g, device="cuda").mul_(1.7).add_(0.1).to(_TYPES[case["input"]])
        # a program's positions: runs of following tokens that start anywhere up to the farthest
        run = torch.arange(t, device="cuda") // 97
        start = torch.randint(0, max(1, case["position"] - 96), (int(run[-1]) + 1,), generator=g, device="cuda")
        st["positions"] = (start[run] + torch.arange(t, device="cuda") % 97).to(torch.int32)
        pages = -(-t // page) + 1
        st["slots"] = torch.randperm(pages * page, generator=g, device="cuda")[:t]
        st["slots"][t // 2] = -1                                                   # a padded token: not stored
        st["frequencies"] = 10000.0 ** (-torch.arange(0, case["rotary"], 2, device="cuda", dtype=torch.float64) / max(1, case["rotary"]))
        for name in ("q", "k"):
            st[name + "_gain"] = torch.randn(d, generator=g, device="cuda").mul_(0.1).add_(1.0)
            st[name + "_offset"] = torch.randn(d, generator=g, device="cuda").mul_(0.1)
        shape = (pages, hk, page, d)
        for name in ("k", "v"):
            st[name] = torch.zeros(shape, device="cuda", dtype=torch.int8 if case["codes"] else ty)
            st[name + "_steps"] = torch.zeros(shape[:3], device="cuda") if case["codes"] else None
        st["q_out"] = torch.zeros((t, hq, d), device="cuda", dtype=ty)
        return st
    if case["op"] == "evict":
        more, pages = _batch(case, g)
        st |= more
        per = -(-case["budget"] // case["page"])                                    # pages that the kept tokens go to
        st |= _cache(case, pages + per * case["seqs"], g)
        st["new_table"] = (pages + torch.randperm(per * case["seqs"], generator=g, device="cuda", dtype=torch.int32)).view(case["seqs"], per)
        # accumulated weights: a few tokens have most, many have next to none, some are equal
        shape = st["k"].shape[:3]
        st["weights"] = torch.rand(shape, generator=g, device="cuda").pow_(6).mul_(40.0).mul_(64.0).round_().div_(64.0)
        return st
    more, pages = _batch(case, g)
    st |= more
    st |= _cache(case, pages, g)
    st["q"] = torch.randn((st["tokens"], case["q_heads"], d), generator=g, device="cuda").mul_(1.5).to(ty)
    st["scale"] = 1.0 / math.sqrt(d)
    if case["op"] == "weigh":
        st["lse"] = _plain_attention(st)[1]                                         # the attention call in front returned it
        st["weights"] = torch.rand(st["k"].shape[:3], generator=g, device="cuda")
        st["weights_out"] = torch.zeros_like(st["weights"])
    return st


# ---- plain forms ------------------------------------------------------------------------------------------------------------

def _gathered(st, name):
    """[seqs, kv_heads, places, dim] of what the page table names, in fp32 (steps applied)."""
    pages = st["table"].clamp(min=0).long()
    x = st[name][pages].float()
    if st[name + "_steps"] is not None:
        x = x * st[name + "_steps"][pages][..., None]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :st["max_length"]]


def _scores(st):
    """Scores [seqs, kv_heads, queries x group, keys] in fp32 with -inf where the mask hides the key."""
    case = st["case"]
    b, n, hk = case["seqs"], st["max_queries"], case["kv_heads"]
    group = case["q_heads"] // hk
    k = _gathered(st, "k")
    q = torch.zeros((b, n, case["q_heads"], case["dim"]), device="cuda")
    q[st["row_seq"], st["row_at"]] = st["q"].float()
    q = q.view(b, n, hk, group, case["dim"]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    s = (q @ k.transpose(2, 3)).mul_(st["scale"])
    key, length = torch.arange(k.shape[2], device="cuda"), st["lengths"].long()[:, None, None]
    news = (st["query_starts"][1:] - st["query_starts"][:-1]).long()[:, None, None]
    at = length - news + torch.arange(n, device="cuda")[None, :, None]
    seen = (key < length).expand(b, n, -1)
    if case["causal"]:
        seen = seen & (key <= at)
    if case["window"]:
        seen = seen & (key > at - case["window"])
    return s.view(b, hk, n, group, -1).masked_fill_(~seen[:, None, :, None, :], -math.inf).view_as(s)


def _rows(st, x):
    """[seqs, kv_heads, queries x group, ...] as [tokens, q_heads, ...]."""
    case = st["case"]
    n, hk = st["max_queries"], case["kv_heads"]
    x = x.view(case["seqs"], hk, n, case["q_heads"] // hk, *x.shape[3:]).transpose(1, 2).flatten(2, 3)
    return x[st["row_seq"], st["row_at"]]


def _plain_attention(st):
    s = _scores(st)
    top = s.amax(3, keepdim=True)
    p = s.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = p.sum(3, keepdim=True)
    o = (p @ _gathered(st, "v")) / total.clamp(min=1e-30)
    return _rows(st, o).to(st["q"].dtype), _rows(st, (total.log() + top).squeeze(3))


def _plain_weigh(st):
    case = st["case"]
    b, n, hk, group = case["seqs"], st["max_queries"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    lse = torch.full((b, n, case["q_heads"]), math.inf, device="cuda")
    lse[st["row_seq"], st["row_at"]] = st["lse"]
    lse = lse.view(b, n, hk, group).transpose(1, 2).flatten(2, 3)
    w = _scores(st).sub_(lse[..., None]).exp_().sum(2)                              # [seqs, kv_heads, keys]
    key = torch.arange(w.shape[2], device="cuda")
    seq, at = (key[None, :] < st["lengths"][:, None]).nonzero(as_tuple=True)
    page = st["table"][seq, at // case["page"]].long()
    out = st["weights_out"].clone()
    out[page, :, at % case["page"]] = st["weights"][page, :, at % case["page"]] + w[seq, :, at]
    return out


def _plain_rotate(st):
    case = st["case"]
    t, d, hq, hk, r = case["tokens"], case["dim"], case["q_heads"], case["kv_heads"], case["rotary"]
    x = st["qkv"].float().view(t, hq + 2 * hk, d)
    heads, v = x[:, :hq + hk], x[:, hq + hk:]
    gain = torch.cat((st["q_gain"].expand(hq, d), st["k_gain"].expand(hk, d)))
    if case["norm"] == "rms":
        heads = heads * (heads.square().mean(2, keepdim=True) + 1e-6).rsqrt() * gain
    elif case["norm"] == "layer":
        heads = heads - heads.mean(2, keepdim=True)
        heads = heads * (heads.square().mean(2, keepdim=True) + 1e-6).rsqrt() * gain
        heads = heads + torch.cat((st["q_offset"].expand(hq, d), st["k_offset"].expand(hk, d)))
    if r:
        angle = st["positions"].double()[:, None] * st["frequencies"]
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        if case["pairs"]:
            a, b = heads[..., 0:r:2], heads[..., 1:r:2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), 3).flatten(2)
        else:
            a, b = heads[..., :r // 2], heads[..., r // 2:r]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), 2)
        heads = torch.cat((turned, heads[..., r:]), 2)
    kept = st["slots"] >= 0
    slot = st["slots"][kept]
    page, at = slot // case["page"], slot % case["page"]
    out = {"q": heads[:, :hq].to(_TYPES[case["type"]])}
    for name, y in (("k", heads[kept, hq:]), ("v", v[kept])):
        if case["codes"]:
            step = y.abs().amax(2, keepdim=True) / 127.0
            code = torch.where(step > 0, torch.round(y / step.clamp(min=1e-38)), torch.zeros_like(y)).clamp(-127, 127)
            y = code * step
        cache = torch.zeros_like(st[name], dtype=_TYPES[case["type"]])
        cache[page, :, at] = y.to(cache.dtype)
        out[name] = cache
    return out


def _plain_evict(st):
    case = st["case"]
    b, hk, page = case["seqs"], case["kv_heads"], case["page"]
    pages = st["table"].clamp(min=0).long()
    w = st["weights"][pages].transpose(1, 2).flatten(2)                              # [seqs, kv_heads, places]
    at, length = torch.arange(w.shape[2], device="cuda"), st["lengths"].long()[:, None, None]
    always = (at < case["sinks"]) | (at >= length - case["recent"])
    w = w.masked_fill(always, math.inf).masked_fill(at >= length, -math.inf)
    counts = st["lengths"].clamp(max=case["budget"])
    order = w.sort(dim=2, descending=True, stable=True).indices[:, :, :case["budget"]]
    rank = torch.arange(order.shape[2], device="cuda")
    kept = order.masked_fill(rank >= counts[:, None, None], 1 << 40).sort(2).values
    out = torch.full((b, hk, case["budget"]), -1, dtype=torch.int32, device="cuda")
    out[:, :, :kept.shape[2]] = kept.masked_fill(kept >= 1 << 40, -1).to(torch.int32)
    seq, head, to = (out >= 0).nonzero(as_tuple=True)
    source = out[seq, head, to].long()
    moved = {}
    for name in ("k", "v", "k_steps", "v_steps", "weights"):
        if st[name] is None:
            continue
        x = st[name].clone()
        x[st["new_table"][seq, to // page].long(), head, to % page] = st[name][st["table"][seq, source // page].long(), head, source % page]
        moved[name] = x
    return moved | {"kept": out, "counts": counts}


# ---- the framework's own ------------------------------------------------------------------------------------------------------

def _own(st):
    import paper_2504_18547_b200 as vt

    case = st["case"]
    cache = vt.PagedCache(st["k"], st["v"], st["k_steps"], st["v_steps"])
    if case["op"] == "rotate":
        d, hq, hk = case["dim"], case["q_heads"], case["kv_heads"]
        layer = case["norm"] == "layer"
        q, k, v = st["qkv"].split((hq * d, hk * d, hk * d), 1)
        vt.vitint_qk_norm_rotate(
            q, k, v, d, norm=case["norm"], eps=1e-6, q_gain=None if case["norm"] == "none" else st["q_gain"],
            k_gain=None if case["norm"] == "none" else st["k_gain"], q_offset=st["q_offset"] if layer else None,
            k_offset=st["k_offset"] if layer else None, positions=st["positions"], frequencies=st["frequencies"], pairs=case["pairs"],
            q_out=st["q_out"], cache=cache, slots=st["slots"])
        out = {"q": st["q_out"], "k": st["k"], "v": st["v"]}
        if case["codes"]:                                                            # codes are returned as the values they stand for
            for name in ("k", "v"):
                out[name] = torch.mul(st[name], st[name + "_steps"][..., None], out=torch.empty_like(st[name], dtype=st["q_out"].dtype))
        return out
    batch = vt.CacheBatch(st["table"], st["lengths"], st.get("query_starts"), st["max_queries"], st["max_length"])
    if case["op"] == "evict":
        kept, counts = vt.vitint_cache_evict(cache, batch, st["weights"], case["budget"], st["new_table"], sinks=case["sinks"],
                                             recent=case["recent"])
        moved = {n: st[n] for n in ("k", "v", "k_steps", "v_steps", "weights") if st[n] is not None}
        return moved | {"kept": kept, "counts": counts}
    if case["op"] == "weigh":
        return vt.vitint_cache_weigh(st["q"], st["lse"], cache, batch, st["scale"], st["weights"], st["weights_out"],
                                     causal=case["causal"], window=case["window"])
    return vt.vitint_paged_attention(st["q"], cache, batch, st["scale"], causal=case["causal"], window=case["window"], want_lse=True)


def run(state):
    if own:
        return _own(state)
    return {"rotate": _plain_rotate, "evict": _plain_evict, "weigh": _plain_weigh, "attention": _plain_attention}[state["case"]["op"]](state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------------

def _visible(case, length, new):
    """Truth values [new, length]: what each new token sees of its sequence."""
    i = torch.arange(new, device="cuda")[:, None] + (length - new)
    j = torch.arange(length, device="cuda")[None, :]
    seen = torch.ones((new, length), dtype=torch.bool, device="cuda")
    if case["causal"]:
        seen &= j <= i
        if case["window"]:
            seen &= j > i - case["window"]
    return seen


def _exact_sequences(st):
    """For each sequence and cached head: its index, head, first row, keys, values and scores in 64 bits."""
    case = st["case"]
    group, first = case["q_heads"] // case["kv_heads"], 0
    for b, (length, new) in enumerate(_lengths(case)):
        seen = _visible(case, length, new)
        pages = st["table"][b, :-(-length // case["page"])].long()
        for h in range(case["kv_heads"]):
            kv = []
            for name in ("k", "v"):
                x = st[name][pages, h].double()
                if st[name + "_steps"] is not None:
                    x = x * st[name + "_steps"][pages, h].double().unsqueeze(-1)
                kv.append(x.reshape(-1, case["dim"])[:length])
            q = st["q"][first:first + new, h * group:(h + 1) * group].double()
            s = torch.einsum("ngd,ld->gnl", q, kv[0]) * st["scale"]
            s[:, ~seen] = -math.inf
            yield b, h, first, kv[1], s
        first += new


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attention":
        group = case["q_heads"] // case["kv_heads"]
        o = torch.zeros((st["tokens"], case["q_heads"], case["dim"]), dtype=torch.float64, device="cuda")
        lse = torch.zeros((st["tokens"], case["q_heads"]), dtype=torch.float64, device="cuda")
        for _, h, first, v, s in _exact_sequences(st):
            n = s.shape[1]
            z = torch.logsumexp(s, 2)
            lse[first:first + n, h * group:(h + 1) * group] = z.T
            p = torch.exp(s - torch.where(z == -math.inf, torch.zeros_like(z), z)[:, :, None])
            o[first:first + n, h * group:(h + 1) * group] = (p @ v).transpose(0, 1)
        return o, lse
    if case["op"] == "weigh":
        out = st["weights_out"].double()
        group = case["q_heads"] // case["kv_heads"]
        for b, h, first, _, s in _exact_sequences(st):
            n, length = s.shape[1:]
            z = st["lse"][first:first + n, h * group:(h + 1) * group].double().T
            w = torch.exp(s - z[:, :, None]).sum((0, 1))
            j = torch.arange(length, device="cuda")
            page = st["table"][b, j // case["page"]].long()
            out[page, h, j % case["page"]] = st["weights"][page, h, j % case["page"]].double() + w
        return out
    if case["op"] == "evict":
        return None                                                                  # nothing is computed: values are moved
    t, d, hq, hk, r = case["tokens"], case["dim"], case["q_heads"], case["kv_heads"], case["rotary"]
    x = st["qkv"].double().reshape(t, -1, d)
    parts = {"q": x[:, :hq], "k": x[:, hq:hq + hk], "v": x[:, hq + hk:]}
    for name in ("q", "k"):
        y = parts[name]
        if case["norm"] == "layer":
            y = torch.nn.functional.layer_norm(y, (d,), st[name + "_gain"].double(), st[name + "_offset"].double(), 1e-6)
        elif case["norm"] == "rms":
            y = y / torch.sqrt((y * y).sum(2, keepdim=True) / d + 1e-6) * st[name + "_gain"].double()
        if r:
            turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(st["positions"].double(), st["frequencies"]))
            front = y[..., :r].reshape(t, -1, r // 2, 2) if case["pairs"] else y[..., :r].reshape(t, -1, 2, r // 2).transpose(2, 3)
            z = torch.view_as_real(torch.view_as_complex(front.contiguous()) * turn[:, None])
            y = torch.cat(((z if case["pairs"] else z.transpose(2, 3)).reshape(t, -1, r), y[..., r:]), 2)
        parts[name] = y
    out = {"q": parts["q"]}
    for name in ("k", "v"):
        y = parts[name]
        if case["codes"]:
            step = y.abs().amax(2, keepdim=True) / 127.0
            y = torch.round(y / torch.where(step == 0, torch.ones_like(step), step)) * step
        flat = torch.zeros((st[name].shape[0] * case["page"], hk, d), dtype=torch.float64, device="cuda")
        stored = torch.nonzero(st["slots"] >= 0).squeeze(1)
        flat[st["slots"][stored]] = y[stored]
        out[name] = flat.view(-1, case["page"], hk, d).transpose(1, 2)
    return out


def work(case):
    hk, d = case["kv_heads"], case["dim"]
    stored = (d + 4) if case["codes"] else 2 * d                                     # bytes of one head's key (or value) of a token
    if case["op"] == "rotate":
        t, hq = case["tokens"], case["q_heads"]
        size = 4 if case["input"] == "f32" else 2
        return {"bytes": t * ((hq + 2 * hk) * d * size + hq * d * 2 + 2 * hk * stored + 12), "flops": t * (hq + hk) * d * 8}
    if case["op"] == "evict":
        total = sum(n for n, _ in _lengths(case))
        kept = sum(min(n, case["budget"]) for n, _ in _lengths(case))
        return {"bytes": hk * (4 * total + kept * (4 * stored + 12)), "flops": hk * total}
    hq, pairs, touched, rows = case["q_heads"], 0, 0, 0
    for length, new in _lengths(case):
        rows += new
        if not case["causal"]:
            pairs, touched = pairs + new * length, touched + length
            continue
        w = min(case["window"] or length, length)
        before = length - new                                                        # query i sees min(before + i + 1, w) keys
        short = max(0, min(new, w - before - 1))
        pairs += short * before + short * (short + 1) // 2 + (new - short) * w
        touched += min(length, w + new - 1)
    if case["op"] == "weigh":
        return {"bytes": touched * hk * (stored + 8) + rows * hq * (2 * d + 4), "flops": 2.0 * d * hq * pairs}
    return {"bytes": 2 * touched * hk * stored + rows * hq * (4 * d + 4), "flops": 4.0 * d * hq * pairs}

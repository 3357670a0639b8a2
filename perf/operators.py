"""Operators of the paged key-value cache: what is timed, on which inputs, and what their results have to be.

  append   lsa_kv_append    new keys and values (and the queries that go with them) of a batch of sequences are rotated to
                            their positions and the keys and values written to the rows of a paged cache; one token each
                            (a decode step) or runs of several (chunks of prompts)
  attend   lsa_paged_attn   attention of one new token per sequence over its whole paged cache (or sink and window)

The latent cache (one row of 576 dims per token, the value is its first 512 dims, 64 query heads) is that of the decode
configuration in configs.py, as are the 16 heads of 128 dims over one key-value head; grouped heads (32 over 8 and the
like) are the generic shapes of models with separate keys and values.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _append(name, batch, new_lo, new_hi, ctx_lo, ctx_hi, heads, kv_heads, d_qk, latent=False, dtype="bf16", e4m3=False, page=64,
            d_rope=0, interleaved=False):
    return {"name": name, "op": "append", "batch": batch, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "heads": heads, "kv_heads": kv_heads, "d_qk": d_qk, "latent": latent, "dtype": dtype, "e4m3": e4m3, "page": page,
            "d_rope": d_rope or d_qk, "interleaved": interleaved}


def _attend(name, batch, ctx_lo, ctx_hi, heads, kv_heads, d_qk, latent=False, dtype="bf16", e4m3=False, page=64, sink=0, window=0):
    return {"name": name, "op": "attend", "batch": batch, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi, "heads": heads, "kv_heads": kv_heads,
            "d_qk": d_qk, "latent": latent, "dtype": dtype, "e4m3": e4m3, "page": page, "sink": sink, "window": window}


def listed():
    return [
        # one user's decode step on the latent cache: 64 query heads and one latent row; a launch's latency
        _append("append_latent_1_seq", 1, 1, 1, 2000, 2000, 64, 1, 576, latent=True, d_rope=64, interleaved=True),
        # a serving batch's decode step on the latent cache
        _append("append_latent_64_seq", 64, 1, 1, 1000, 8000, 64, 1, 576, latent=True, d_rope=64, interleaved=True),
        # chunks of eight prompts of very different lengths, one of them a single token, grouped heads, rotation by halves
        _append("append_prompts_32_over_8", 8, 1, 6001, 0, 900, 32, 8, 128, page=16),
        # the same work into a cache of 8-bit codes with a scale per row and head; half of the dims rotated
        _append("append_prompts_e4m3", 5, 700, 4099, 100, 5000, 64, 8, 128, dtype="bf16", e4m3=True, d_rope=64, interleaved=True),
        # one user at a short context: latency
        _attend("attend_latent_1_short", 1, 777, 777, 64, 1, 576, latent=True),
        # one user at half a million tokens: the length has to be split over the whole GPU
        _attend("attend_latent_1_long", 1, 524288, 524288, 64, 1, 576, latent=True),
        # the serving batch of the decode configuration, contexts between 16K and 128K: the largest case
        _attend("attend_latent_64_seq", 64, 16384, 131072, 64, 1, 576, latent=True),
        # a large batch of chats, a few tokens to some thousands, small pages
        _attend("attend_32_over_8_chats", 128, 1, 7001, 32, 8, 128, page=16),
        # 16 heads over one key-value head of 128 dims, long documents, fp16
        _attend("attend_16_over_1_long", 12, 30011, 131072, 16, 1, 128, dtype="fp16"),
        # the 8-bit cache, 64 heads over 8
        _attend("attend_e4m3_64_over_8", 32, 500, 32768, 64, 8, 128, e4m3=True),
        # sink and sliding window of streaming layers: what is attended does not grow with the context
        _attend("attend_window_16_over_4", 40, 3, 60001, 16, 4, 64, page=32, sink=4, window=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    latent = rng.random() < 0.4
    e4m3 = not latent and rng.random() < 0.4
    if latent:
        shape = (rng.choice([16, 24, 64, 64]), 1, 576)
        page = rng.choice([64, 64, 128, 256])
    else:
        kv_heads = rng.choice([1, 2, 4, 6, 8])
        shape = (kv_heads * rng.choice([1, 2, 4, 5, 8, 16]), kv_heads, rng.choice([64, 128, 128]))
        page = rng.choice([16, 32, 64, 128])
    more = dict(latent=latent, dtype=rng.choice(["bf16", "bf16", "fp16"]), e4m3=e4m3, page=page)
    if rng.random() < 0.4:
        if rng.random() < 0.5:
            batch, new = _log(rng, 1, 256), (1, 1)
        else:
            batch = _log(rng, 1, 24)
            most = _log(rng, 2, 12000 // batch + 2)
            new = (rng.randrange(0, 3), most)
        ctx = _log(rng, 1, 6000)
        d_rope = 64 if latent else rng.choice([64, shape[2]])
        case = _append("", batch, *new, rng.randrange(0, ctx), ctx, *shape, d_rope=d_rope, interleaved=rng.random() < 0.5, **more)
    else:
        batch = _log(rng, 1, 160)
        per_token = shape[1] * shape[2]           # elements of a key row
        top = min(262144, 1_200_000_000 // (batch * per_token))
        hi = _log(rng, 2, top)
        window = _log(rng, 16, 8192) if rng.random() < 0.25 else 0
        case = _attend("", batch, rng.randrange(0, max(1, hi // 2)), hi, *shape, sink=rng.choice([0, 4, 20]) if window else 0, window=window, **more)
    del case["name"]
    return case


def _ragged(count, lo, hi):
    """`count` numbers from lo to hi, more of them small than large: the same for every seed, so that the work is."""
    if count == 1:
        return [hi]
    return [lo + (hi - lo) * i * i // ((count - 1) * (count - 1)) for i in range(count)]


def _lengths(case):
    """(tokens cached before the call, new tokens) of each sequence, before they are shuffled."""
    ctx = _ragged(case["batch"], case["ctx_lo"], case["ctx_hi"])
    if case["op"] == "attend":
        return ctx, [0] * case["batch"]
    new = _ragged(case["batch"], case["new_lo"], case["new_hi"])
    return ctx, new[::-1]


def _d_v(case):
    return 512 if case["latent"] else case["d_qk"]


def _attended(case, n):
    """Cache rows that the one query of a sequence of n tokens reads."""
    if not case["window"] or n <= case["sink"] + case["window"]:
        return n
    return case["sink"] + case["window"]


def work(case):
    ctx, new = _lengths(case)
    H, G, d, dv = case["heads"], case["kv_heads"], case["d_qk"], _d_v(case)
    kv = G * d + (0 if case["latent"] else G * dv)                # elements of a token's cache row(s)
    scales = 0 if not case["e4m3"] else 4 * G * (1 if case["latent"] else 2)
    row = kv * (1 if case["e4m3"] else 2) + scales
    if case["op"] == "append":
        n = sum(new)
        spans = sum(-(-(c + k) // case["page"]) - c // case["page"] for c, k in zip(ctx, new) if k)   # pages written to
        return {"bytes": n * (2 * kv + row + 4 * H * d) + 4 * n * case["d_rope"] + 4 * spans + 8 * case["batch"],
                "flops": 3 * n * case["d_rope"] * (H + G)}
    n = sum(_attended(case, c) for c in ctx)
    pages = sum(-(-_attended(case, c) // case["page"]) for c in ctx)
    return {"bytes": n * row + 4 * pages + case["batch"] * (2 * H * (d + dv) + 4 * H + 4), "flops": 2 * n * H * (d + dv)}


def _quantised(x, heads):
    """Rows of values as e4m3 codes and one scale per row and head."""
    y = x.float().unflatten(-1, (heads, -1))
    top = y.abs().amax(-1)
    scale = torch.where(top > 0, top / 448, torch.ones_like(top))
    return (y / scale[..., None]).to(torch.float8_e4m3fn).flatten(1), scale


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(dev).manual_seed(int(seed) * 1_000_003 + 17)
    host = torch.Generator().manual_seed(int(seed) * 1_000_003 + 29)
    dtype = _DTYPES[case["dtype"]]
    B, H, G, d, dv, page = case["batch"], case["heads"], case["kv_heads"], case["d_qk"], _d_v(case), case["page"]
    order = torch.randperm(B, generator=host)
    ctx, new = (torch.tensor(x, dtype=torch.int64)[order] for x in _lengths(case))
    # Pages are handed out at random to the sequences; the rest of the table is empty.
    n_of = (ctx + new + page - 1) // page
    width = max(1, int(n_of.max()))
    n_pages = int(n_of.sum()) + 3
    table = torch.full((B, width), -1, dtype=torch.int32)
    table[torch.arange(width)[None, :] < n_of[:, None]] = torch.randperm(n_pages, generator=host)[: int(n_of.sum())].to(torch.int32)

    def normal(*shape, scale=1.0):
        x = torch.randn(*shape, generator=gen, device=dev, dtype=dtype)
        return x if scale == 1.0 else x * scale

    def pool(width):
        x = normal(n_pages * page, width)
        return _quantised(x, G) if case["e4m3"] else (x, None)

    s = {"case": case, "n_pages": n_pages, "longest": int((ctx + new).max()), "ctx_len": ctx.to(dev, torch.int32), "page_table": table.to(dev)}
    s["k_pool"], s["k_scale"] = pool(G * d)
    s["v_pool"], s["v_scale"] = (None, None) if case["latent"] else pool(G * dv)
    if case["op"] == "attend":
        # scores of a few units: the weights are neither uniform nor one-hot
        s["q"] = normal(B, H, d, scale=2.5)
        s["out"] = torch.empty(B, H, dv, dtype=dtype, device=dev)
        s["lse"] = torch.empty(B, H, dtype=torch.float32, device=dev)
        return s
    n_tok = int(new.sum())
    s["n_tok"] = n_tok
    start = torch.zeros(B + 1, dtype=torch.int32)
    start[1:] = torch.cumsum(new, 0)
    s["tok_start"] = None if case["new_lo"] == case["new_hi"] == 1 else start.to(dev)
    if case["latent"]:
        s["q"], s["k_new"], s["v_new"] = normal(n_tok, H, d), normal(n_tok, 1, d), None
    else:   # the three parts of one projection's output
        qkv = normal(n_tok, H + 2 * G, d)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    half = torch.arange(case["d_rope"] // 2, device=dev, dtype=torch.float64)
    angle = torch.arange(s["longest"], device=dev, dtype=torch.float64)[:, None] * 10000.0 ** (-2 * half / case["d_rope"])
    s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    s["q_out"] = torch.empty(n_tok, H, d, dtype=dtype, device=dev)
    s["ctx_len_out"] = torch.empty(B, dtype=torch.int32, device=dev)
    return s


_contexts: dict = {}


def _context(s):
    """The library's handle, which a program keeps per stream for the shapes that it serves (its calls go to the stream it was made for)."""
    device = s["q"].get_device()
    stream = torch._C._cuda_getCurrentRawStream(device)   # (a number: torch.cuda.current_stream makes an object, 2 us a call)
    ctx = _contexts.get((s.get("kv_bytes"), device, stream))
    return ctx if ctx is not None else _new_context(s, device, stream)


def _new_context(s, device, stream):
    from paper_2608_01662_b200 import binding

    c = s["case"]
    kv = binding.make_kv_params(n_heads=c["heads"], n_kv_heads=c["kv_heads"], d_qk=c["d_qk"], d_v=_d_v(c), latent=c["latent"], dtype=c["dtype"],
                                e4m3=c["e4m3"], kv_page=c["page"], d_rope=c.get("d_rope", 0),
                                rope_at=c["d_qk"] - 64 if c["latent"] and c["op"] == "append" else 0,
                                rope_interleaved=c.get("interleaved", False), sink=c.get("sink", 0), window=c.get("window", 0),
                                sm_scale=c["d_qk"] ** -0.5)
    s["kv_bytes"] = bytes(kv)
    key = (s["kv_bytes"], device, stream)
    if key not in _contexts:
        _contexts[key] = binding.Context(None, 0, 0, device=s["q"].device, kv=kv)   # (on the current stream)
    return _contexts[key]


def run(state):
    s = state
    if own:
        ctx = _context(s)
        if s["case"]["op"] == "append":
            ctx.kv_append(s["k_new"], s["v_new"], s["k_pool"], s["v_pool"], s["page_table"], s["ctx_len"], s["ctx_len_out"],
                          tok_start=s["tok_start"], q=s["q"], q_out=s["q_out"], cos_sin=s["cos_sin"], k_scale=s["k_scale"], v_scale=s["v_scale"])
            return _appended(s, s["q_out"], s["ctx_len_out"])
        ctx.paged_attn(s["q"], s["k_pool"], s["v_pool"], s["page_table"], s["ctx_len"], s["out"], s["lse"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return {"out": s["out"], "lse": s["lse"]}
    return _append_plain(s) if s["case"]["op"] == "append" else _attend_plain(s)


def _appended(s, q_out, ctx_len_out):
    got = {"q": q_out, "k_pool": s["k_pool"], "ctx_len": ctx_len_out}
    if s["v_pool"] is not None:
        got["v_pool"] = s["v_pool"]
    if s["k_scale"] is not None:
        got["k_scale"], got["v_scale"] = s["k_scale"], s["v_scale"]
    return got


def _rotated(x, cos, sin, at, interleaved):
    """x [token, head, dim] in 32 bits with the dims from `at` on, as many as the angles are pairs, rotated."""
    n = cos.shape[-1]
    part = x[..., at:at + 2 * n]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :n], part[..., n:])
    c, s = cos[:, None, :], sin[:, None, :]
    u, v = a * c - b * s, b * c + a * s
    turned = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([x[..., :at], turned, x[..., at + 2 * n:]], -1)


def _append_plain(s):
    c = s["case"]
    G, page, n_tok = c["kv_heads"], c["page"], s["n_tok"]
    dev, dtype = s["q"].device, s["q"].dtype
    tok = torch.arange(n_tok, device=dev)
    if s["tok_start"] is None:
        seq, added = tok, torch.ones_like(s["ctx_len"])
        pos = s["ctx_len"].long()
    else:
        added = s["tok_start"][1:] - s["tok_start"][:-1]
        seq = torch.repeat_interleave(torch.arange(c["batch"], device=dev), added.long(), output_size=n_tok)
        pos = s["ctx_len"].long()[seq] + tok - s["tok_start"].long()[seq]
    rows = s["page_table"][seq, pos // page].long() * page + pos % page
    cos, sin = s["cos_sin"][pos].chunk(2, -1)
    at = c["d_qk"] - c["d_rope"] if c["latent"] else 0
    q = _rotated(s["q"].float(), cos, sin, at, c["interleaved"]).to(dtype)
    k = _rotated(s["k_new"].float(), cos, sin, at, c["interleaved"])
    if c["e4m3"]:
        (k_codes, s["k_scale"][rows]), (v_codes, s["v_scale"][rows]) = _quantised(k.flatten(1), G), _quantised(s["v_new"].flatten(1), G)
        s["k_pool"].view(torch.uint8)[rows], s["v_pool"].view(torch.uint8)[rows] = k_codes.view(torch.uint8), v_codes.view(torch.uint8)
    else:
        s["k_pool"][rows] = k.flatten(1).to(dtype)
        if s["v_new"] is not None:
            s["v_pool"][rows] = s["v_new"].flatten(1)
    return _appended(s, q, s["ctx_len"] + added)


def _seen(s):
    """The positions that a sequence's query sees, in a table as wide as the longest list of them, and which entries are one."""
    c, n = s["case"], s["ctx_len"].long()[:, None]
    width = s["longest"]
    if c["window"]:
        width = min(width, c["sink"] + c["window"])
    i = torch.arange(width, device=n.device)[None, :]
    if not c["window"]:
        return i.expand(c["batch"], width), i < n
    cut = n > c["sink"] + c["window"]
    return torch.where(cut & (i >= c["sink"]), i + n - c["window"] - c["sink"], i), i < n


def _attend_plain(s):
    c = s["case"]
    B, H, G, d, dv = c["batch"], c["heads"], c["kv_heads"], c["d_qk"], _d_v(c)
    pos, seen = _seen(s)
    rows = s["page_table"].long().gather(1, (pos // c["page"]).clamp(max=s["page_table"].shape[1] - 1)).clamp(min=0) * c["page"] + pos % c["page"]

    def cached(pool, scale, width):   # [sequence, head, position, dim]
        x = pool.view(torch.uint8)[rows].view(torch.float8_e4m3fn) if c["e4m3"] else pool[rows]
        x = x.float().unflatten(-1, (G, width))
        return (x * scale[rows][..., None] if c["e4m3"] else x).transpose(1, 2)

    k = cached(s["k_pool"], s["k_scale"], d)
    score = s["q"].float().view(B, G, H // G, d) @ k.transpose(-1, -2) * d ** -0.5
    v = k[..., :dv] if c["latent"] else cached(s["v_pool"], s["v_scale"], dv)
    score = score.masked_fill(~seen[:, None, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return {"out": out.reshape(B, H, dv).to(s["q"].dtype), "lse": (top + torch.log(total)).reshape(B, H)}


def exact(case, seed):
    """The operators' definitions in 64 bits, one sequence after another."""
    s = prepare(case, seed)
    B, H, G, d, dv, page = case["batch"], case["heads"], case["kv_heads"], case["d_qk"], _d_v(case), case["page"]
    table, ctx = s["page_table"].cpu().long(), s["ctx_len"].cpu().tolist()
    dev = s["q"].device

    def rows_of(b, first, last):
        pos = torch.arange(first, last)
        return (table[b, pos // page] * page + pos % page).to(dev)

    if case["op"] == "attend":
        out = torch.zeros(B, H, dv, dtype=torch.float64, device=dev)
        lse = torch.full((B, H), -math.inf, dtype=torch.float64, device=dev)

        def values(pool, scale, rows, g, width):
            x = pool.view(torch.uint8)[rows].view(torch.float8_e4m3fn) if case["e4m3"] else pool[rows]
            x = x[:, g * width:(g + 1) * width].double()
            return x * scale[rows, g].double()[:, None] if case["e4m3"] else x

        for b in range(B):
            n = ctx[b]
            if n == 0:
                continue
            if case["window"] and n > case["sink"] + case["window"]:
                rows = torch.cat([rows_of(b, 0, case["sink"]), rows_of(b, n - case["window"], n)])
            else:
                rows = rows_of(b, 0, n)
            for g in range(G):
                heads = slice(g * (H // G), (g + 1) * (H // G))
                k = values(s["k_pool"], s["k_scale"], rows, g, d)
                z = s["q"][b, heads].double() @ k.T / math.sqrt(d)
                lse[b, heads] = torch.logsumexp(z, -1)
                v = k[:, :dv] if case["latent"] else values(s["v_pool"], s["v_scale"], rows, g, dv)
                out[b, heads] = torch.softmax(z, -1) @ v
        return {"out": out, "lse": lse}

    # append: each sequence's angles as complex numbers
    starts = list(range(B + 1)) if s["tok_start"] is None else s["tok_start"].cpu().tolist()
    n_rot, at = case["d_rope"] // 2, d - case["d_rope"] if case["latent"] else 0

    def turned(x, pos):
        table = s["cos_sin"][pos].double()
        turn = torch.complex(table[:, :n_rot], table[:, n_rot:])[:, None, :]
        y = x.double().clone()
        part = y[..., at:at + 2 * n_rot].unflatten(-1, (n_rot, 2) if case["interleaved"] else (2, n_rot))
        part = part if case["interleaved"] else part.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
        y[..., at:at + 2 * n_rot] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        return y

    got = {"q": torch.empty(s["n_tok"], H, d, dtype=torch.float64, device=dev), "ctx_len": s["ctx_len"].clone()}
    if case["e4m3"]:   # codes are roundings of quotients of roundings: only the scales have a value here
        got |= {"k_pool": None, "v_pool": None, "k_scale": s["k_scale"].double(), "v_scale": s["v_scale"].double()}
    else:
        got |= {"k_pool": s["k_pool"].double()} | ({} if case["latent"] else {"v_pool": s["v_pool"].double()})
    for b in range(B):
        t0, t1 = starts[b], starts[b + 1]
        got["ctx_len"][b] += t1 - t0
        if t1 == t0:
            continue
        pos = torch.arange(ctx[b], ctx[b] + t1 - t0, device=dev)
        rows = rows_of(b, ctx[b], ctx[b] + t1 - t0)
        got["q"][t0:t1] = turned(s["q"][t0:t1], pos)
        k = turned(s["k_new"][t0:t1], pos)
        v = None if case["latent"] else s["v_new"][t0:t1].double()
        for name, x in (("k", k), ("v", v)):
            if x is None:
                continue
            if case["e4m3"]:
                top = x.abs().amax(-1)
                got[name + "_scale"][rows] = torch.where(top > 0, top / 448, torch.ones_like(top))
            else:
                got[name + "_pool"][rows] = x.flatten(1)
    return got

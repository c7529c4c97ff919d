"""Rotary positions and the KV cache in 8 bits: listed calls, a generator of more of the same kinds, and their plain forms.

Every case is one call that one layer of a serving loop makes: q and k get their positions, new K and V rows are
quantised into the cache's pages (with or without the rotation in the same launch), slots of the cache are read back,
and a prefill batch, a cross-attention batch or a decode step attends over the cache.  Head counts and lengths are those
of the library's named workloads: 28 / 4 and 32 / 8 heads of 128 in bf16, 4 / 1 heads of 64 in fp32, images of some
hundred to some thousand tokens, videos of 16384, text of up to 2048.

`own` false: the formulas in elementary torch operations, in 32 bits (angles in 64).  `own` true: the library's calls.

A case is a dict of plain values:
  op         "rope"      emm_rope of q and k
             "write"     emm_kv_scatter_fp8, or emm_rope_kv_scatter_fp8 where "rotary" > 0
             "read"      emm_kv_gather_fp8 of whole contexts
             "chunk"     emm_prefill_attn_fp8 (a prefill batch)
             "cross"     emm_cross_attn_fp8
             "decode"    emm_decode_attn_fp8
  dtype, heads, kv_heads, head_dim, page    shapes ("page": tokens per page)
  reqs       requests in the batch; each has cached_lo .. cached_hi cached tokens and new_lo .. new_hi new ones
  lengths    seed of the lengths (they belong to the case, the tensors' values to prepare's seed)
  rotary     rotated channels of a head (0: no rotation); layout "half" or "interleaved"
  axes       0: a token's position is its place in its request; 1 or 3: positions are given, that many per token
  stretch    positions' frequencies are divided by this (long contexts), inverse: the rotation the other way round
  fused      the rows of q, k and v lie in one projection's output, [T][heads + 2 kv_heads][head_dim]
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
E4M3_MAX = 448.0
LEAST_EXPONENT = -117
ROPE_BASE = 1000000.0


def _case(name, op, **kw):
    case = {"name": name, "op": op, "dtype": "bf16", "heads": 28, "kv_heads": 4, "head_dim": 128, "page": 16, "reqs": 1,
            "cached_lo": 0, "cached_hi": 0, "new_lo": 1, "new_hi": 1, "lengths": 0, "rotary": 0, "layout": "half", "axes": 0,
            "stretch": 1.0, "inverse": False, "fused": False}
    assert set(kw) <= set(case), kw
    case.update(kw)
    return case


def listed():
    return [
        # positions of a short fp32 prompt behind a small cached prefix, half of each head rotated: the smallest call
        _case("rope_small_prompt", "rope", dtype="f32", heads=4, kv_heads=1, head_dim=64, cached_lo=256, cached_hi=256, new_lo=64,
              new_hi=64, rotary=32, layout="interleaved"),
        # two long prompts behind cached videos, time / height / width positions, straight from the projection's rows
        _case("rope_video_prompts", "rope", reqs=2, cached_lo=16384, cached_hi=16384, new_lo=2048, new_hi=2048, rotary=128, axes=3, fused=True),
        # a decode step of 64 requests: rotate q and k, quantise k and v into the cache
        _case("write_step", "write", reqs=64, cached_lo=500, cached_hi=8191, rotary=128, axes=3, lengths=11),
        # the K and V rows of an ordinary prefill batch into the cache
        _case("write_prompts", "write", heads=32, kv_heads=8, reqs=32, cached_lo=0, cached_hi=4096, new_lo=256, new_hi=2400, lengths=12),
        # the cache of one chat about an image read back, and that of two videos
        _case("read_chat", "read", cached_lo=1500, cached_hi=1500),
        _case("read_videos", "read", reqs=2, cached_lo=16384, cached_hi=18432, lengths=13),
        # eight questions about images in the cache
        _case("chunk_image_batch", "chunk", reqs=8, cached_lo=1056, cached_hi=1056, new_lo=128, new_hi=512, lengths=14),
        # two long prompts behind cached videos: the largest call
        _case("chunk_video_prompts", "chunk", reqs=2, cached_lo=16384, cached_hi=16384, new_lo=2048, new_hi=2048),
        # one short question about a video seen before
        _case("chunk_question", "chunk", cached_lo=16384, cached_hi=16384, new_lo=36, new_hi=36),
        # decode steps: one chat, a ragged batch, a long uniform one
        _case("decode_one_chat", "decode", cached_lo=1500, cached_hi=1500),
        _case("decode_ragged", "decode", heads=32, kv_heads=8, reqs=32, cached_lo=300, cached_hi=4600, lengths=15),
        _case("decode_long_batch", "decode", reqs=64, cached_lo=8191, cached_hi=8191),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


#: the most that a drawn case may ask for: what the largest listed ones do, scores that the plain form can hold, caches that are quickly made
MOST_FLOPS, MOST_BYTES, MOST_SCORES, MOST_SLOTS = 1.03e12, 5.5e8, 2.2e9, 550000


def draw(rng):
    while True:
        case = _draw_once(rng)
        w = work(case)
        cached, new = _lengths(case)
        scores = case["reqs"] * case["heads"] * max(new) * (max(cached) + max(new)) if case["op"] in ("chunk", "cross", "decode") else 0
        slots = case["reqs"] * max(cached) if case["op"] != "rope" else 0
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and scores <= MOST_SCORES and slots <= MOST_SLOTS:
            return case


def _draw_once(rng):
    op = rng.choice(["rope", "rope", "write", "write", "read", "chunk", "chunk", "question", "cross", "decode", "decode", "decode"])
    heads, kv_heads = rng.choice([(28, 4), (32, 8), (16, 2)])
    kw = {"heads": heads, "kv_heads": kv_heads, "page": rng.choice([16, 16, 32, 64]), "lengths": rng.randrange(1 << 20)}
    if op in ("rope", "write"):
        if rng.random() < 0.25:
            kw.update(dtype="f32", heads=rng.choice([4, 8]), kv_heads=rng.choice([1, 2]), head_dim=rng.choice([64, 128]))
        cached, new = _log_int(rng, 1, 100000), _log_int(rng, 1, 4096)
        kw.update(reqs=_log_int(rng, 1, 64), cached_lo=cached // 2, cached_hi=cached, new_lo=max(1, new // 4), new_hi=new, fused=rng.random() < 0.5)
        if op == "rope" or rng.random() < 0.6:
            whole = kw.get("head_dim", 128)
            kw.update(rotary=rng.choice([whole, whole, whole // 2, whole // 4]), layout=rng.choice(["half", "half", "interleaved"]), axes=rng.choice([0, 1, 3]),
                      stretch=rng.choice([1.0, 1.0, 4.0]), inverse=op == "rope" and rng.random() < 0.25)
    elif op == "read":
        cached = _log_int(rng, 64, 32768)
        kw.update(reqs=_log_int(rng, 1, 16), cached_lo=cached // 2, cached_hi=cached, dtype=rng.choice(["bf16", "bf16", "f32"]))
    elif op == "chunk":
        cached, new = _log_int(rng, 256, 16384), _log_int(rng, 64, 2048)
        kw.update(reqs=_log_int(rng, 1, 16), cached_lo=cached // 2, cached_hi=cached, new_lo=max(1, new // 4), new_hi=new)
    elif op == "question":
        op, cached = "chunk", _log_int(rng, 1024, 32768)
        kw.update(reqs=_log_int(rng, 1, 32), cached_lo=cached // 2, cached_hi=cached, new_lo=2, new_hi=rng.randint(4, 64))
    elif op == "cross":
        image = rng.randint(576, 6516)
        kw.update(reqs=rng.randint(1, 8), cached_lo=image // 4, cached_hi=image, new_lo=1, new_hi=_log_int(rng, 8, 512))
    else:
        ctx = _log_int(rng, 100, 32768)
        kw.update(reqs=_log_int(rng, 1, 64), cached_lo=int(ctx * rng.choice([0.1, 0.5, 1.0])), cached_hi=ctx)
    case = _case("", op, **kw)
    del case["name"]
    return case


def _lengths(case):
    """Cached and new tokens of every request."""
    rng = random.Random(case["lengths"])
    n = case["reqs"]
    return ([rng.randint(case["cached_lo"], case["cached_hi"]) for _ in range(n)], [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(n)])


def _context(case, cached, new):
    """Slots that a request's pages hold: of the operators that attend or write causally the new tokens' too."""
    return cached if case["op"] in ("read", "cross") else cached + new


def work(case):
    cached, new = _lengths(case)
    d, heads, kv_heads = case["head_dim"], case["heads"], case["kv_heads"]
    elt = 4 if case["dtype"] == "f32" else 2
    tokens, row = sum(new), 2 * kv_heads * (d + 1)                            # row: a slot's K and V codes and scale bytes
    if case["op"] == "rope":
        return {"bytes": 2 * tokens * (heads + kv_heads) * d * elt, "flops": 3 * tokens * (heads + kv_heads) * case["rotary"]}
    if case["op"] == "write":
        rotated = 2 * heads * d * elt if case["rotary"] else 0
        return {"bytes": tokens * (2 * kv_heads * d * elt + row + rotated), "flops": 4 * tokens * kv_heads * d}
    if case["op"] == "read":
        return {"bytes": sum(cached) * (row + 2 * kv_heads * d * elt), "flops": 2 * sum(cached) * kv_heads * d}
    causal = case["op"] != "cross"
    pairs = sum(m * c + (m * (m + 1) // 2 if causal else 0) for c, m in zip(cached, new))
    slots = sum(_context(case, c, m) for c, m in zip(cached, new))
    return {"bytes": slots * row + 2 * tokens * heads * d * elt + 4 * tokens * heads, "flops": 4 * d * heads * pairs}


def _sections(case):
    """How many of the frequencies each axis of the positions has: a quarter for time, the rest in equal parts for height and width."""
    n = case["rotary"] // 2
    return [n // 4, (n - n // 4) // 2, n - n // 4 - (n - n // 4) // 2] if case["axes"] == 3 else [n]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    heads, kv_heads, d, page, reqs = case["heads"], case["kv_heads"], case["head_dim"], case["page"], case["reqs"]
    cached, new = _lengths(case)
    first, count = (cached, new) if case["op"] != "read" else ([0] * reqs, cached)
    tokens = sum(count)
    pages = [-(-_context(case, c, m) // page) for c, m in zip(cached, new)]
    num_pages, width = sum(pages) + 8, max(1, max(pages))

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=DEVICE)

    order = torch.randperm(num_pages, generator=gen, device=DEVICE).to(torch.int32)
    starts = [sum(pages[:r]) for r in range(reqs)]
    place = torch.arange(width, device=DEVICE)[None, :]
    table = torch.where(place < ints(pages)[:, None], order[(ints(starts)[:, None] + place).clamp(max=num_pages - 1)], -1).to(torch.int32)
    s = {"case": case, "page_table": table, "prefix_lens": ints(first), "new_lens": ints(count),
         "cu_new_lens": ints([sum(count[:r]) for r in range(reqs + 1)]), "tokens": tokens, "longest_new": max(count),
         "longest": max(_context(case, c, m) for c, m in zip(cached, new)), "num_pages": num_pages}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=dt)

    if case["op"] in ("rope", "write"):
        # a projection's rows; some channels of K are larger than the others, as they are in earnest
        rows = normal(tokens, heads + 2 * kv_heads, d)
        rows[:, heads : heads + kv_heads] *= torch.where(torch.rand(kv_heads, d, generator=gen, device=DEVICE) < 0.03, 8.0, 1.0).to(dt)
        q, k, v = rows[:, :heads], rows[:, heads : heads + kv_heads], rows[:, heads + kv_heads :]
        s.update(q=q, k=k, v=v) if case["fused"] else s.update(q=q.contiguous(), k=k.contiguous(), v=v.contiguous())
        s["stride"] = (heads + 2 * kv_heads) * d if case["fused"] else 0
        s["q_out"] = torch.empty((tokens, heads, d), device=DEVICE, dtype=dt)
        s["k_out"] = torch.empty((tokens, kv_heads, d), device=DEVICE, dtype=dt)
        if case["rotary"]:
            i = torch.arange(case["rotary"] // 2, device=DEVICE, dtype=torch.float64)
            s["inv_freq"] = ROPE_BASE ** (-2.0 * i / case["rotary"]) / case["stretch"]
            s["factor"] = 0.1 * math.log(case["stretch"]) + 1.0
            s["positions"] = None
            if case["axes"]:
                # text goes on behind the cached tokens; of an image or video the axes differ
                s["positions"] = torch.randint(0, max(cached) + max(new), (case["axes"], tokens), generator=gen, device=DEVICE, dtype=torch.int32)
    if case["op"] != "rope":
        # codes as a quantiser leaves them (rows that fill the format's range), values of about one
        pool = (num_pages, kv_heads, page, d)
        for name in ("k", "v"):
            s[name + "_cache"] = (torch.randn(pool, generator=gen, device=DEVICE) * 120).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
            s[name + "_scale"] = torch.randint(119, 122, pool[:3], generator=gen, device=DEVICE, dtype=torch.uint8)
    if case["op"] == "read":
        s["k_out"], s["v_out"] = (torch.empty((tokens, kv_heads, d), device=DEVICE, dtype=dt) for _ in range(2))
    if case["op"] in ("chunk", "cross", "decode"):
        s["q"] = normal(tokens, heads, d)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((tokens, heads), device=DEVICE, dtype=torch.float32)
    if own:
        # the descriptors and the workspace that a serving loop keeps
        from paper_2507_10069_amd import binding as B
        s["batch"] = B.make_batch(num_reqs=reqs, num_q_heads=heads, num_kv_heads=kv_heads, head_dim=d, page_size=page, num_pages=num_pages,
                                  max_pages_per_req=width, total_new_tokens=tokens, max_new_len=s["longest_new"], dtype=case["dtype"],
                                  softmax_scale=1.0 / math.sqrt(d), page_table=table, prefix_lens=s["prefix_lens"], new_lens=s["new_lens"],
                                  cu_new_lens=s["cu_new_lens"])
        if case["op"] != "rope":
            s["cache"] = B.make_fp8_cache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        if case["rotary"]:
            s["rope"] = B.make_rope(s["inv_freq"], rotary_dim=case["rotary"], layout=case["layout"], factor=s["factor"], inverse=case["inverse"],
                                    positions=s["positions"], sections=_sections(case))
        if case["op"] in ("chunk", "cross", "decode"):
            n = B.emm_attn_fp8_workspace_size(s["batch"])
            s["workspace"] = torch.empty(n, device=DEVICE, dtype=torch.uint8) if n else None
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2507_10069_amd import binding as B
    op = s["case"]["op"]
    if op == "rope":
        B.emm_rope(s["batch"], s["rope"], s["q"], s["k"], s["q_out"], s["k_out"], token_stride=s["stride"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "write":
        if s["case"]["rotary"]:
            B.emm_rope_kv_scatter_fp8(s["batch"], s["rope"], s["q"], s["k"], s["v"], s["q_out"], s["cache"], token_stride=s["stride"])
        else:
            B.emm_kv_scatter_fp8(s["batch"], s["k"], s["v"], s["cache"], token_stride=s["stride"])
        return _written(s)
    if op == "read":
        B.emm_kv_gather_fp8(s["batch"], s["cache"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    call = {"chunk": B.emm_prefill_attn_fp8, "cross": B.emm_cross_attn_fp8, "decode": B.emm_decode_attn_fp8}[op]
    call(s["batch"], s["q"], s["cache"], s["out"], s["lse"], s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def _written(s):
    """The cache after a write: code values, and scales as the bytes that they are (whole numbers)."""
    out = {"k": s["k_cache"], "v": s["v_cache"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    return dict(out, q=s["q_out"]) if s["case"]["rotary"] else out


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _tokens(s):
    """The request of every packed token, and its place in the request."""
    reqs = s["case"]["reqs"]
    req = torch.repeat_interleave(torch.arange(reqs, device=DEVICE), s["new_lens"].long(), output_size=s["tokens"])
    return req, torch.arange(s["tokens"], device=DEVICE) - s["cu_new_lens"].long()[req]


def _slots(s):
    """Page and place in the page of every packed token's slot."""
    req, j = _tokens(s)
    at = s["prefix_lens"].long()[req] + j
    page = s["case"]["page"]
    return s["page_table"].long()[req, at // page], at % page


def _power(e):
    """2^e for whole numbers -126 .. 127, by the bits of the format."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _cos_sin(s):
    case = s["case"]
    if s["positions"] is None:
        req, j = _tokens(s)
        at = (s["prefix_lens"].long()[req] + j)[:, None]
    else:
        axis = torch.repeat_interleave(torch.arange(len(_sections(case)), device=DEVICE), torch.tensor(_sections(case), device=DEVICE),
                                       output_size=case["rotary"] // 2)
        at = s["positions"].t()[:, axis]
    angle = at.double() * s["inv_freq"]
    sign = -1.0 if case["inverse"] else 1.0
    return (torch.cos(angle) * s["factor"]).float()[:, None, :], (torch.sin(angle) * (s["factor"] * sign)).float()[:, None, :]


def _rotated(case, x, cos, sin):
    n, x = case["rotary"], x.float()
    a, b = (x[..., : n // 2], x[..., n // 2 : n]) if case["layout"] == "half" else (x[..., 0:n:2], x[..., 1:n:2])
    p, q = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([p, q], dim=-1) if case["layout"] == "half" else torch.stack([p, q], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., n:]], dim=-1)


def _quantised(x):
    """Codes and scale bytes of rows along the last axis."""
    x = x.float()
    finite = torch.isfinite(x)
    most = torch.where(finite, x.abs(), 0.0).amax(dim=-1)
    part, e = torch.frexp(most)                                              # most = part * 2^e, 448 = 0.875 * 2^9
    e = torch.where(most > 0, e - 9 + (part > 0.875), LEAST_EXPONENT).clamp(min=LEAST_EXPONENT)
    y = torch.where(finite, x * _power(-e)[..., None], math.nan)
    return y.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _values(s, which, pages, places):
    """Cached values of slots, in 32 bits: the slots' axes, then KV heads, channels."""
    codes = s[which + "_cache"].view(torch.uint8)[pages, :, places].view(torch.float8_e4m3fn).float()
    return codes * _power(s[which + "_scale"][pages, :, places].to(torch.int32) - 127)[..., None]


def _run_plain(s):
    case = s["case"]
    op, dt = case["op"], torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    if op in ("rope", "write") and case["rotary"]:
        cos, sin = _cos_sin(s)
        q, k = _rotated(case, s["q"], cos, sin).to(dt), _rotated(case, s["k"], cos, sin).to(dt)
        if op == "rope":
            return {"q": q, "k": k}
    if op == "write":
        pages, places = _slots(s)
        if not case["rotary"]:
            k = s["k"]
        s["k_cache"].view(torch.uint8)[pages, :, places], s["k_scale"][pages, :, places] = _quantised(k)
        s["v_cache"].view(torch.uint8)[pages, :, places], s["v_scale"][pages, :, places] = _quantised(s["v"])
        return dict(_written(s), q=q) if case["rotary"] else _written(s)
    if op == "read":
        pages, places = _slots(s)
        return {"k": _values(s, "k", pages, places).to(dt), "v": _values(s, "v", pages, places).to(dt)}
    # attention: contexts and queries padded to the longest, scores of all of them
    reqs, heads, kv_heads, d, page = case["reqs"], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    g, n, length = heads // kv_heads, s["longest_new"], s["longest"]
    req, j = _tokens(s)
    at = torch.arange(length, device=DEVICE)
    pages = s["page_table"].long()[:, at // page].clamp(min=0)
    places = (at % page)[None, :].expand(reqs, length)
    held = s["prefix_lens"].long() + (0 if op == "cross" else s["new_lens"].long())
    q = torch.zeros((reqs, n, heads, d), device=DEVICE)
    q[req, j] = s["q"].float()
    q = q.view(reqs, n, kv_heads, g, d).permute(0, 2, 1, 3, 4).reshape(reqs, kv_heads, n * g, d)
    k = _values(s, "k", pages, places).permute(0, 2, 3, 1).contiguous()
    scores = torch.matmul(q, k) * (1.0 / math.sqrt(d))
    del k
    last = s["prefix_lens"].long()[:, None] + (torch.arange(n, device=DEVICE)[None, :] if op != "cross" else -1)
    last = last.expand(reqs, n).repeat_interleave(g, dim=1)
    scores.masked_fill_((at[None, None, :] > last[:, :, None])[:, None], -math.inf)
    most = scores.amax(dim=-1, keepdim=True)
    most = torch.where(torch.isinf(most), 0.0, most)
    weights = scores.sub_(most).exp_()
    total = weights.sum(dim=-1, keepdim=True)
    v = torch.where((at[None, :] < held[:, None])[:, :, None, None], _values(s, "v", pages, places), 0.0).permute(0, 2, 1, 3).contiguous()
    out = torch.matmul(weights, v) / torch.where(total > 0, total, 1.0)
    lse = (most + torch.log(total))[..., 0]
    out = out.view(reqs, kv_heads, n, g, d).permute(0, 2, 1, 3, 4).reshape(reqs, n, heads, d)[req, j]
    lse = lse.view(reqs, kv_heads, n, g).permute(0, 2, 1, 3).reshape(reqs, n, heads)[req, j]
    return {"out": out.to(dt), "lse": lse}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _to_e4m3(y):
    """Nearest value with four significant bits (ties to even), at least 2^-9 apart."""
    _, e = torch.frexp(y)                                                    # |y| in [2^(e-1), 2^e)
    step = torch.exp2((e.double() - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    op, dt = case["op"], torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    reqs, heads, kv_heads, d, page = case["reqs"], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    host = {k: s[k].tolist() for k in ("prefix_lens", "new_lens", "cu_new_lens", "page_table")}

    def turned(x):
        n = case["rotary"]
        if s["positions"] is None:
            at = torch.cat([torch.arange(c, c + m, device=DEVICE) for c, m in zip(host["prefix_lens"], host["new_lens"])]).double()[:, None].expand(-1, n // 2)
        else:
            parts, lo = [], 0
            for axis, width in enumerate(_sections(case)):
                parts.append(s["positions"][axis].double()[:, None].expand(-1, width))
                lo += width
            at = torch.cat(parts, dim=1)
        angle = at * s["inv_freq"] * (-1 if case["inverse"] else 1)
        turn = torch.polar(torch.full_like(angle, s["factor"]), angle)[:, None, :]
        x = x.double().clone()
        pair = (slice(0, n // 2), slice(n // 2, n)) if case["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
        z = torch.complex(x[..., pair[0]].contiguous(), x[..., pair[1]].contiguous()) * turn
        x[..., pair[0]], x[..., pair[1]] = z.real, z.imag
        return x

    def slots(r):
        at = torch.arange(host["prefix_lens"][r], host["prefix_lens"][r] + host["new_lens"][r], device=DEVICE)
        return torch.tensor(host["page_table"][r], device=DEVICE)[at // page], at % page

    if op == "rope":
        return {"q": turned(s["q"]), "k": turned(s["k"])}
    if op == "write":
        rows = {"k": turned(s["k"]).to(dt).double() if case["rotary"] else s["k"].double(), "v": s["v"].double()}
        out = {}
        for name, x in rows.items():
            part, e = torch.frexp(x.abs().amax(dim=-1) / E4M3_MAX)
            e = torch.where(part > 0.5, e, e - 1).clamp(min=LEAST_EXPONENT)
            y = _to_e4m3(x / torch.exp2(e.double())[..., None])
            values, scales = s[name + "_cache"].double(), s[name + "_scale"].long()
            for r in range(reqs):
                pages, places = slots(r)
                lo, hi = host["cu_new_lens"][r], host["cu_new_lens"][r + 1]
                values[pages, :, places] = y[lo:hi]
                scales[pages, :, places] = e[lo:hi].long() + 127
            out[name], out[name + "_scale"] = values, scales.to(torch.uint8)
        if case["rotary"]:
            out["q"] = turned(s["q"])
        return out

    def held(name, r, n):
        """The first n slots of request r in 64 bits, [n][kv_heads][d]."""
        ids = torch.tensor(host["page_table"][r][: -(-n // page)], device=DEVICE)
        x = s[name + "_cache"].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * torch.exp2(s[name + "_scale"][ids].double() - 127)[..., None]
        return x.transpose(1, 2).reshape(-1, kv_heads, d)[:n]

    if op == "read":
        return {name: torch.cat([held(name, r, host["new_lens"][r]) for r in range(reqs)]) for name in ("k", "v")}
    g = heads // kv_heads
    out = torch.zeros((s["tokens"], heads, d), device=DEVICE, dtype=torch.float64)
    lse = torch.full((s["tokens"], heads), -math.inf, device=DEVICE, dtype=torch.float64)
    for r in range(reqs):
        c, m, at = host["prefix_lens"][r], host["new_lens"][r], host["cu_new_lens"][r]
        ctx = _context(case, c, m)
        if ctx == 0:
            continue
        k_all, v_all = held("k", r, ctx), held("v", r, ctx)
        for h in range(kv_heads):
            k, v = k_all[:, h].t().contiguous(), v_all[:, h].contiguous()
            step = max(1, (1 << 27) // (ctx * g))                            # at most a gigabyte of scores at a time
            for t0 in range(0, m, step):
                t1 = min(m, t0 + step)
                sc = (s["q"][at + t0 : at + t1, h * g : (h + 1) * g].double().reshape(-1, d) @ k) / math.sqrt(d)
                if op != "cross":
                    last = (c + torch.arange(t0, t1, device=DEVICE)).repeat_interleave(g)
                    sc.masked_fill_(torch.arange(ctx, device=DEVICE)[None, :] > last[:, None], -math.inf)
                top = torch.logsumexp(sc, dim=1)
                lse[at + t0 : at + t1, h * g : (h + 1) * g] = top.reshape(-1, g)
                out[at + t0 : at + t1, h * g : (h + 1) * g] = (torch.exp(sc - top[:, None]) @ v).reshape(-1, g, d)
    return {"out": out, "lse": lse}

"""What a decoder layer's step needs around and in place of full attention: listed calls, a generator of more of the same kinds, and
their plain forms.

Every case is one call that a serving loop makes of a model whose layers look back a fixed distance: the step's page tables, packed
offsets, positions and slots made on the device from the requests' lengths; q and k normalised head by head and rotated, with or without
the write of K and V into the cache; attention over the last `window` tokens and the first `sinks`, of a prefill batch and of a decode
step.  Head counts and lengths are those of the library's named workloads: 28 / 4 and 32 / 8 heads of 128 in bf16, 4 / 1 heads of 64 in
fp32, images of some hundred to some thousand tokens, videos of 16384, text of up to 2048; windows of 128 to 4096 tokens.

`own` false: the formulas in elementary torch operations, in 32 bits (angles in 64).  `own` true: the library's calls.

A case is a dict of plain values:
  op         "pages"     emm_page_step: a step's tables, offsets, positions and slots
             "norm"      emm_norm_rope of q and k
             "write"     emm_norm_rope_kv_scatter: the same, with k's and v's way into the cache
             "chunk"     emm_prefill_attn_window (a prefill batch)
             "decode"    emm_decode_attn_window
  dtype, heads, kv_heads, head_dim, page    shapes ("page": tokens per page)
  reqs       requests in the batch; each has cached_lo .. cached_hi cached tokens and new_lo .. new_hi new ones
  lengths    seed of the lengths (they belong to the case, the tensors' values to prepare's seed)
  window     tokens that a query sees, itself among them (pages: how far the next queries look back; 0: all of it, no page is given back)
  sinks      tokens at the start that stay visible
  spare      pages: free pages that the pool has for every one that the step takes (under 1: some requests get none)
  rotary     rotated channels of a head (0: norms alone); layout "half" or "interleaved"
  axes       0: a token's position is its place in its request; 1 or 3: positions are given, that many per token
  slots      write: the tokens' slots are given
  fused      the rows of q, k and v lie in one projection's output, [T][heads + 2 kv_heads][head_dim]
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
ROPE_BASE = 1000000.0
EPS = 1e-6


def _case(name, op, **kw):
    case = {"name": name, "op": op, "dtype": "bf16", "heads": 28, "kv_heads": 4, "head_dim": 128, "page": 16, "reqs": 1,
            "cached_lo": 0, "cached_hi": 0, "new_lo": 1, "new_hi": 1, "lengths": 0, "window": 0, "sinks": 0, "spare": 2.0,
            "rotary": 0, "layout": "half", "axes": 0, "slots": False, "fused": False}
    assert set(kw) <= set(case), kw
    case.update(kw)
    return case


def listed():
    return [
        # the tables of a decode step: 64 requests, one token each, most of them behind their window
        _case("pages_step", "pages", reqs=64, cached_lo=500, cached_hi=8191, window=4096, sinks=4, lengths=21),
        # the tables of a large prefill batch: pages for some thousand tokens of each request at once
        _case("pages_prompts", "pages", reqs=48, cached_lo=0, cached_hi=4096, new_lo=64, new_hi=1300, lengths=22),
        # heads of a short fp32 prompt, half of each rotated: the smallest call of its kind
        _case("norm_small_prompt", "norm", dtype="f32", heads=4, kv_heads=1, head_dim=64, cached_lo=256, cached_hi=256, new_lo=64,
              new_hi=64, rotary=32, layout="interleaved"),
        # two long prompts behind cached videos, time / height / width positions, straight from the projection's rows
        _case("norm_video_prompts", "norm", reqs=2, cached_lo=16384, cached_hi=16384, new_lo=2048, new_hi=2048, rotary=128, axes=3, fused=True),
        # a decode step of 64 requests: norm, rotation and write, slots and positions from the step's tables
        _case("write_step", "write", reqs=64, cached_lo=500, cached_hi=8191, rotary=128, axes=1, slots=True, lengths=23),
        # the rows of an ordinary prefill batch on their way into the cache
        _case("write_prompts", "write", heads=32, kv_heads=8, reqs=32, cached_lo=0, cached_hi=4096, new_lo=256, new_hi=2400, rotary=128,
              fused=True, lengths=24),
        # a short fp32 prompt with a short window: the smallest attention
        _case("window_small_prompt", "chunk", dtype="f32", heads=4, kv_heads=1, head_dim=64, cached_lo=256, cached_hi=256, new_lo=64,
              new_hi=64, window=128, sinks=4),
        # eight questions about images in the cache
        _case("window_image_batch", "chunk", reqs=8, cached_lo=1056, cached_hi=1056, new_lo=128, new_hi=512, window=1024, sinks=4, lengths=25),
        # two long prompts behind cached videos: the largest call
        _case("window_video_prompts", "chunk", reqs=2, cached_lo=16384, cached_hi=16384, new_lo=2048, new_hi=2048, window=4096, sinks=4),
        # one short question about a video seen before
        _case("window_question", "chunk", cached_lo=16384, cached_hi=16384, new_lo=36, new_hi=36, window=2048, sinks=64),
        # decode steps: one chat, and a long batch
        _case("window_one_chat", "decode", cached_lo=1500, cached_hi=1500, window=1024, sinks=4),
        _case("window_long_batch", "decode", reqs=64, cached_lo=8191, cached_hi=8191, window=4096, sinks=4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


#: the most that a drawn case may ask for: what the largest listed ones do, scores that the plain form can hold, caches that are quickly made
MOST_FLOPS, MOST_BYTES, MOST_SCORES, MOST_SLOTS = 2.4e11, 6e8, 1.2e9, 550000


def draw(rng):
    while True:
        case = _draw_once(rng)
        w = work(case)
        cached, new = _lengths(case)
        spans = [_span(case, c, n) for c, n in zip(cached, new)]
        scores = case["reqs"] * case["heads"] * max(new) * max(spans) if case["op"] in ("chunk", "decode") else 0
        slots = sum(spans) if case["op"] in ("write", "chunk", "decode") else 0
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES and scores <= MOST_SCORES and slots <= MOST_SLOTS:
            return case


def _draw_once(rng):
    op = rng.choice(["pages", "pages", "norm", "write", "write", "chunk", "chunk", "question", "decode", "decode"])
    heads, kv_heads = rng.choice([(28, 4), (32, 8), (16, 2), (8, 8)])
    kw = {"heads": heads, "kv_heads": kv_heads, "page": rng.choice([16, 16, 32, 64]), "lengths": rng.randrange(1 << 20)}
    if op == "pages":
        cached, new = _log_int(rng, 16, 30000), rng.choice([1, 1, _log_int(rng, 2, 1500)])
        kw.update(reqs=_log_int(rng, 1, 256), cached_lo=cached // 8, cached_hi=cached, new_lo=0 if rng.random() < 0.3 else max(1, new // 4), new_hi=new,
                  window=rng.choice([0, _log_int(rng, 64, 8192)]), sinks=rng.choice([0, 4, 100]), spare=rng.choice([2.0, 2.0, 1.0, 0.6]))
    elif op in ("norm", "write"):
        if rng.random() < 0.3:
            kw.update(dtype="f32", heads=rng.choice([4, 8]), kv_heads=rng.choice([1, 2]), head_dim=rng.choice([64, 128]))
        cached, new = _log_int(rng, 1, 60000), _log_int(rng, 1, 4096)
        whole = kw.get("head_dim", 128)
        kw.update(reqs=_log_int(rng, 1, 64), cached_lo=cached // 2, cached_hi=cached, new_lo=max(1, new // 4), new_hi=new, fused=rng.random() < 0.5,
                  rotary=rng.choice([0, whole, whole, whole // 2, whole // 4]), layout=rng.choice(["half", "half", "interleaved"]))
        if kw["rotary"]:
            kw.update(axes=rng.choice([0, 1, 3]))
        if op == "write":
            kw.update(slots=rng.random() < 0.5)
    else:
        if op != "decode" and rng.random() < 0.25:
            kw.update(dtype="f32", heads=rng.choice([4, 8]), kv_heads=rng.choice([1, 2]), head_dim=rng.choice([64, 128]))
        kw.update(window=rng.choice([_log_int(rng, 64, 4096), 512, 1024, 2048]), sinks=rng.choice([0, 1, 4, 16, 100]))
        if op == "chunk":
            cached, new = _log_int(rng, 16, 16384), _log_int(rng, 64, 2048)
            kw.update(reqs=_log_int(rng, 1, 16), cached_lo=cached // 2, cached_hi=cached, new_lo=max(1, new // 4), new_hi=new)
        elif op == "question":
            op, cached = "chunk", _log_int(rng, 512, 32768)
            kw.update(reqs=_log_int(rng, 1, 32), cached_lo=cached // 2, cached_hi=cached, new_lo=2, new_hi=rng.randint(4, 64))
        else:
            ctx = _log_int(rng, 100, 32768)
            kw.update(reqs=_log_int(rng, 1, 128), cached_lo=int(ctx * rng.choice([0.1, 0.5, 1.0])), cached_hi=ctx)
    case = _case("", op, **kw)
    del case["name"]
    return case


def _lengths(case):
    """Cached and new tokens of every request."""
    rng = random.Random(case["lengths"])
    n = case["reqs"]
    return ([rng.randint(case["cached_lo"], case["cached_hi"]) for _ in range(n)], [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(n)])


def _low(case, cached):
    """The first slot behind the sinks that any of the new tokens sees."""
    return max(cached - case["window"] + 1, 0) if case["window"] else 0


def _span(case, cached, new):
    """Slots of a request that its new tokens see."""
    low = _low(case, cached)
    return cached + new - low + min(case["sinks"] if case["window"] else 0, low)


def _dead(case, cached):
    """Entries of a request's table that no token from slot `cached` on sees: from the first to behind the last."""
    kept = -(-case["sinks"] // case["page"])
    return (kept, max(kept, _low(case, cached) // case["page"])) if case["window"] else (kept, kept)


def work(case):
    cached, new = _lengths(case)
    d, heads, kv_heads, page = case["head_dim"], case["heads"], case["kv_heads"], case["page"]
    elt = 4 if case["dtype"] == "f32" else 2
    tokens = sum(new)
    if case["op"] == "pages":
        # lengths in and out, offsets, a slot and a position for every token, and the ids of pages taken and given back, read and written
        taken = sum(-(-(c + m) // page) - -(-c // page) for c, m in zip(cached, new))
        back = sum(hi - lo for lo, hi in (_dead(case, c) for c in cached))
        return {"bytes": 12 * tokens + 32 * case["reqs"] + 8 * taken + 8 * back, "flops": 4 * tokens}
    if case["op"] in ("norm", "write"):
        rows = heads + kv_heads + (kv_heads if case["op"] == "write" else 0)
        return {"bytes": 2 * tokens * rows * d * elt, "flops": tokens * (heads + kv_heads) * (4 * d + 3 * case["rotary"])}
    w, s = case["window"], case["sinks"]
    pairs = 0
    for c, m in zip(cached, new):
        # a token at slot p sees min(p + 1, w) slots of its window and min(s, max(0, p + 1 - w)) sinks before it
        full = max(0, min(m, w - 1 - c))                                     # tokens that see all before them
        pairs += full * (c + 1) + full * (full - 1) // 2 + (m - full) * w
        first = c + full + 1 - w                                             # slots behind the window of the first of the others, one more for each
        n, short = m - full, max(0, min(m - full, s - max(first, 0)))
        pairs += short * max(first, 0) + short * (short - 1) // 2 + (n - short) * s
    slots = sum(_span(case, c, m) for c, m in zip(cached, new))
    return {"bytes": 2 * slots * kv_heads * d * elt + 2 * tokens * heads * d * elt + 4 * tokens * heads, "flops": 4 * d * heads * pairs}


def _sections(case):
    """How many of the frequencies each axis of the positions has: a quarter for time, the rest in equal parts for height and width."""
    n = case["rotary"] // 2
    return [n // 4, (n - n // 4) // 2, n - n // 4 - (n - n // 4) // 2] if case["axes"] == 3 else [n]


def prepare(case, seed):
    return _prepare_pages(case, seed) if case["op"] == "pages" else _prepare_rows(case, seed)


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    return gen


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _prepare_pages(case, seed):
    """Tables as a loop's earlier steps left them: pages of the cached tokens, those behind the window given back up to some steps ago."""
    gen = _generator(seed)
    page, reqs = case["page"], case["reqs"]
    cached, new = _lengths(case)
    rng = random.Random(seed)
    held_from = []
    for c in cached:
        lo, hi = _dead(case, c)
        held_from.append(rng.randint(max(lo, hi - 3), hi) if c else lo)
    entries = [-(-c // page) for c in cached]
    needed = sum(-(-(c + m) // page) - n for c, m, n in zip(cached, new, entries))
    free = int(needed * case["spare"]) + (2 if case["spare"] >= 1 else 0)
    width = max(1, max(-(-(c + m) // page) for c, m in zip(cached, new)))
    num_pages = sum(entries) + free
    order = torch.randperm(max(num_pages, 1), generator=gen, device=DEVICE).to(torch.int32)
    starts = [sum(entries[:r]) for r in range(reqs)]
    place = torch.arange(width, device=DEVICE)[None, :]
    at = (_ints(starts)[:, None] + place).clamp(max=order.numel() - 1)
    table = torch.where(place < _ints(entries)[:, None], order[at], -1).to(torch.int32).contiguous()
    free_pages = torch.full((max(num_pages, 1),), -1, dtype=torch.int32, device=DEVICE)
    free_pages[:free] = order[sum(entries):]
    s = {"case": case, "num_pages": max(num_pages, 1), "width": width, "tokens": max(sum(new), 1), "page_table": table, "free_pages": free_pages,
         "lens": _ints(cached), "add_lens": _ints(new), "held_from": _ints(held_from), "free_count": _ints([free])}
    for name, n, dt in (("prefix_lens", reqs, torch.int32), ("new_lens", reqs, torch.int32), ("cu_new_lens", reqs + 1, torch.int32),
                        ("lens_out", reqs, torch.int32), ("held_out", reqs, torch.int32), ("free_count_out", 1, torch.int32),
                        ("slots", s["tokens"], torch.int64), ("positions", s["tokens"], torch.int32), ("refused", 1, torch.int32)):
        s[name] = torch.zeros(n, dtype=dt, device=DEVICE)
    if own:
        from paper_2507_10069_amd import binding as B
        s["step"] = B.make_page_step(num_reqs=reqs, page_size=page, num_pages=s["num_pages"], max_pages_per_req=width, max_tokens=s["tokens"],
                                     window=case["window"], sinks=case["sinks"], page_table=table, free_pages=free_pages, lens=s["lens"],
                                     add_lens=s["add_lens"], held_from=s["held_from"], free_count=s["free_count"], prefix_lens=s["prefix_lens"],
                                     new_lens=s["new_lens"], cu_new_lens=s["cu_new_lens"], lens_out=s["lens_out"], held_out=s["held_out"],
                                     free_count_out=s["free_count_out"], slots=s["slots"], positions=s["positions"], refused=s["refused"])
    return s


def _prepare_rows(case, seed):
    gen = _generator(seed)
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    heads, kv_heads, d, page, reqs = case["heads"], case["kv_heads"], case["head_dim"], case["page"], case["reqs"]
    cached, new = _lengths(case)
    tokens = sum(new)
    # what a request's table still holds: the sinks' pages, and those from the first that its new tokens see on
    attends = case["op"] in ("chunk", "decode")
    dead = [_dead(case, c) if attends else (0, 0) for c in cached]
    if case["op"] == "write":
        dead = [(0, c // page) for c in cached]                              # (pages before the first that is written are not looked at)
    entries = [-(-(c + m) // page) for c, m in zip(cached, new)]
    held = [n - (hi - lo) for n, (lo, hi) in zip(entries, dead)]
    num_pages, width = sum(held) + 8, max(1, max(entries))
    order = torch.randperm(num_pages, generator=gen, device=DEVICE).to(torch.int32)
    starts = _ints([sum(held[:r]) for r in range(reqs)])[:, None]
    place = torch.arange(width, device=DEVICE)[None, :]
    lo, hi = _ints([x[0] for x in dead])[:, None], _ints([x[1] for x in dead])[:, None]
    nth = torch.where(place < lo, place, place - (hi - lo))
    live = (place < _ints(entries)[:, None]) & ((place < lo) | (place >= hi))
    table = torch.where(live, order[(starts + nth).clamp(0, num_pages - 1)], -1).to(torch.int32).contiguous()
    s = {"case": case, "page_table": table, "prefix_lens": _ints(cached), "new_lens": _ints(new),
         "cu_new_lens": _ints([sum(new[:r]) for r in range(reqs + 1)]), "tokens": tokens, "longest_new": max(new), "num_pages": num_pages,
         "longest_span": max(_span(case, c, m) for c, m in zip(cached, new))}

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=dt)

    pool = (num_pages, kv_heads, page, d)
    if case["op"] in ("norm", "write"):
        # a projection's rows; some channels of K are larger than the others, as they are in earnest
        rows = normal(tokens, heads + 2 * kv_heads, d)
        rows[:, heads : heads + kv_heads] *= torch.where(torch.rand(kv_heads, d, generator=gen, device=DEVICE) < 0.03, 8.0, 1.0).to(dt)
        q, k, v = rows[:, :heads], rows[:, heads : heads + kv_heads], rows[:, heads + kv_heads :]
        s.update(q=q, k=k, v=v) if case["fused"] else s.update(q=q.contiguous(), k=k.contiguous(), v=v.contiguous())
        s["stride"] = (heads + 2 * kv_heads) * d if case["fused"] else 0
        s["q_out"] = torch.empty((tokens, heads, d), device=DEVICE, dtype=dt)
        s["q_weight"], s["k_weight"] = (1.0 + 0.2 * torch.randn(d, generator=gen, device=DEVICE) for _ in range(2))
        s["positions"] = s["slots"] = None
        if case["rotary"]:
            i = torch.arange(case["rotary"] // 2, device=DEVICE, dtype=torch.float64)
            s["inv_freq"] = ROPE_BASE ** (-2.0 * i / case["rotary"])
            if case["axes"]:
                # text goes on behind the cached tokens; of an image or video the axes differ
                s["positions"] = torch.randint(0, max(cached) + max(new), (case["axes"], tokens), generator=gen, device=DEVICE, dtype=torch.int32)
        if case["op"] == "norm":
            s["k_out"] = torch.empty((tokens, kv_heads, d), device=DEVICE, dtype=dt)
        else:
            s["k_cache"], s["v_cache"] = normal(*pool), normal(*pool)
            if case["slots"]:
                pages, places = _slots(s)
                s["slots"] = pages * page + places
    else:
        s["k_cache"], s["v_cache"] = normal(*pool), normal(*pool)
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
        if case["op"] in ("norm", "write"):
            s["norm"] = B.make_qk_norm(s["q_weight"], s["k_weight"], eps=EPS)
            s["rope"] = B.make_rope(s["inv_freq"], rotary_dim=case["rotary"], layout=case["layout"], positions=s["positions"],
                                    sections=_sections(case)) if case["rotary"] else None
        else:
            n = B.emm_attn_window_workspace_size(s["batch"], case["window"], case["sinks"])
            s["workspace"] = torch.empty(n, device=DEVICE, dtype=torch.uint8) if n else None
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    return _plain_pages(s) if op == "pages" else _plain_rows(s) if op in ("norm", "write") else _plain_window(s)


PAGES_OUT = ("page_table", "free_pages", "prefix_lens", "new_lens", "cu_new_lens", "lens_out", "held_out", "free_count_out", "slots", "positions",
             "refused")


def _run_own(s, op):
    from paper_2507_10069_amd import binding as B
    if op == "pages":
        B.emm_page_step(s["step"])
        return {k: s[k] for k in PAGES_OUT}
    if op == "norm":
        B.emm_norm_rope(s["batch"], s["norm"], s["rope"], s["q"], s["k"], s["q_out"], s["k_out"], token_stride=s["stride"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "write":
        B.emm_norm_rope_kv_scatter(s["batch"], s["norm"], s["rope"], s["q"], s["k"], s["v"], s["q_out"], s["k_cache"], s["v_cache"],
                                   token_stride=s["stride"], slots=s["slots"])
        return {"q": s["q_out"], "k": s["k_cache"], "v": s["v_cache"]}
    call = B.emm_prefill_attn_window if op == "chunk" else B.emm_decode_attn_window
    call(s["batch"], s["case"]["window"], s["case"]["sinks"], s["q"], s["k_cache"], s["v_cache"], s["out"], s["lse"], s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _plain_pages(s):
    case = s["case"]
    page, width, reqs = case["page"], s["width"], case["reqs"]
    lens, add, count = s["lens"].long(), s["add_lens"].long(), s["free_count"].long()
    # pages that no later token sees, by request and then by place, lie on top of those that were free
    kept = -(-case["sinks"] // page)
    start = s["held_from"].long().clamp(min=kept)
    held = torch.maximum(start, (lens - case["window"] + 1).clamp(min=0) // page) if case["window"] else start
    back = held - start
    back_end = torch.cumsum(back, 0)
    returned = back_end[-1:]
    entry = torch.arange(width, device=DEVICE)[None, :]
    at = torch.arange(s["num_pages"], device=DEVICE)
    nth = at - count                                                         # the nth page given back lies there
    of = torch.searchsorted(back_end, nth.clamp(min=0), right=True).clamp(max=reqs - 1)
    place = (start[of] + nth - (back_end - back)[of]).clamp(0, width - 1)
    given = s["page_table"].long()[of, place]
    stack = torch.where(nth < 0, s["free_pages"].long(), given)              # (of which count + returned are free)
    # requests take their pages from the top in turn; one that finds too few gets none
    fits = lens + add <= width * page
    have, want = -(-lens // page), -(-(lens + add) // page)
    need = torch.where(fits, want - have, 0)
    need_end = torch.cumsum(need, 0)
    free = count + returned
    served = fits & ((need == 0) | (need_end <= free))
    new = torch.where(served, add, 0)
    taken = torch.where(served, need_end, 0).amax()
    nth = entry - have[:, None]
    takes = served[:, None] & (nth >= 0) & (entry < want[:, None])
    top = (free - 1 - (need_end - need)[:, None] - nth).clamp(0, s["num_pages"] - 1)
    s["page_table"].copy_(torch.where(takes, stack[top], s["page_table"].long()))
    left = free - taken
    s["free_pages"].copy_(torch.where((at >= count) & (at < left), stack, s["free_pages"].long()))
    # packed offsets, and where every token is
    cu = torch.cumsum(new, 0)
    t = torch.arange(s["slots"].numel(), device=DEVICE)
    r = torch.searchsorted(cu, t, right=True).clamp(max=reqs - 1)
    position = lens[r] + t - (cu - new)[r]
    slot = s["page_table"].long()[r, (position // page).clamp(0, width - 1)] * page + position % page
    some = t < cu[-1]
    s["prefix_lens"].copy_(lens)
    s["new_lens"].copy_(new)
    s["cu_new_lens"].copy_(torch.cat([torch.zeros_like(cu[:1]), cu]))
    s["lens_out"].copy_(lens + new)
    s["held_out"].copy_(held)
    s["free_count_out"].copy_(left)
    s["slots"].copy_(torch.where(some, slot, -1))
    s["positions"].copy_(torch.where(some, position, 0))
    s["refused"].copy_((~served & (add > 0)).sum().reshape(1))
    return {k: s[k] for k in PAGES_OUT}


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


def _plain_rows(s):
    case = s["case"]
    dt, n = s["q"].dtype, case["rotary"]

    def normed(x, weight):
        x = x.float()
        return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * weight

    q, k = normed(s["q"], s["q_weight"]), normed(s["k"], s["k_weight"])
    if n:
        if s["positions"] is None:
            req, j = _tokens(s)
            at = (s["prefix_lens"].long()[req] + j)[:, None]
        else:
            axis = torch.repeat_interleave(torch.arange(len(_sections(case)), device=DEVICE), torch.tensor(_sections(case), device=DEVICE),
                                           output_size=n // 2)
            at = s["positions"].t()[:, axis]
        angle = at.double() * s["inv_freq"]
        cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]

        def rotated(x):
            half = case["layout"] == "half"
            a, b = (x[..., : n // 2], x[..., n // 2 : n]) if half else (x[..., 0:n:2], x[..., 1:n:2])
            p, q = a * cos - b * sin, b * cos + a * sin
            return torch.cat([torch.cat([p, q], dim=-1) if half else torch.stack([p, q], dim=-1).flatten(-2), x[..., n:]], dim=-1)

        q, k = rotated(q), rotated(k)
    q, k = q.to(dt), k.to(dt)
    if case["op"] == "norm":
        return {"q": q, "k": k}
    if s["slots"] is None:
        pages, places = _slots(s)
    else:
        pages, places = s["slots"] // case["page"], s["slots"] % case["page"]
    s["k_cache"][pages, :, places] = k
    s["v_cache"][pages, :, places] = s["v"]
    return {"q": q, "k": s["k_cache"], "v": s["v_cache"]}


def _plain_window(s):
    """Slots that some new token of a request sees, padded to the most of them, and scores of all of these."""
    case = s["case"]
    reqs, heads, kv_heads, d, page = case["reqs"], case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    w, sinks = case["window"], case["sinks"]
    g, n, span = heads // kv_heads, s["longest_new"], s["longest_span"]
    req, j = _tokens(s)
    cached = s["prefix_lens"].long()[:, None]
    low = (cached - w + 1).clamp(min=0)
    first = low.clamp(max=sinks)                                             # sinks before what the window holds
    nth = torch.arange(span, device=DEVICE)[None, :]
    at = torch.where(nth < first, nth, nth - first + low)                    # [reqs][span]
    pages = s["page_table"].long().gather(1, (at // page).clamp(max=s["page_table"].shape[1] - 1)).clamp(min=0)
    places = at % page
    held = at < cached + s["new_lens"].long()[:, None]
    q = torch.zeros((reqs, n, heads, d), device=DEVICE)
    q[req, j] = s["q"].float()
    q = q.view(reqs, n, kv_heads, g, d).permute(0, 2, 1, 3, 4).reshape(reqs, kv_heads, n * g, d)
    k = s["k_cache"][pages, :, places].float().permute(0, 2, 3, 1).contiguous()
    scores = torch.matmul(q, k) * (1.0 / math.sqrt(d))
    del k
    own_at = (cached + torch.arange(n, device=DEVICE)[None, :])[:, :, None]
    seen = (at[:, None, :] <= own_at) & ((at[:, None, :] > own_at - w) | (at[:, None, :] < sinks))
    scores.view(reqs, kv_heads, n, g, span).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    most = scores.amax(dim=-1, keepdim=True)
    weights = scores.sub_(most).exp_()
    total = weights.sum(dim=-1, keepdim=True)
    v = torch.where(held[:, :, None, None], s["v_cache"][pages, :, places].float(), 0.0).permute(0, 2, 1, 3).contiguous()
    out = torch.matmul(weights, v) / total
    lse = (most + torch.log(total))[..., 0]
    out = out.view(reqs, kv_heads, n, g, d).permute(0, 2, 1, 3, 4).reshape(reqs, n, heads, d)[req, j]
    lse = lse.view(reqs, kv_heads, n, g).permute(0, 2, 1, 3).reshape(reqs, n, heads)[req, j]
    return {"out": out.to(s["q"].dtype), "lse": lse}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"pages": _exact_pages, "norm": _exact_rows, "write": _exact_rows}.get(case["op"], _exact_window)(case, s)


def _exact_pages(case, s):
    """The step as a loop over the requests, with the free pages as a list."""
    page, width = case["page"], s["width"]
    table, lens, add, held = (s[k].tolist() for k in ("page_table", "lens", "add_lens", "held_from"))
    count = s["free_count"].tolist()[0]
    buffer = s["free_pages"].tolist()
    free = buffer[:count]
    for r, c in enumerate(lens):
        held[r] = max(held[r], -(-case["sinks"] // page))
        if case["window"]:
            while (held[r] + 1) * page <= c - case["window"] + 1:            # the next token sees nothing of that page
                free.append(table[r][held[r]])
                held[r] += 1
    new, refused, enough = [], 0, True
    for r, (c, m) in enumerate(zip(lens, add)):
        have, want = -(-c // page), -(-(c + m) // page)
        ok = c + m <= width * page
        if ok and want > have:
            enough = enough and want - have <= len(free)
            ok = enough
            if ok:
                for e in range(have, want):
                    table[r][e] = free.pop()
        new.append(m if ok else 0)
        refused += 0 if ok or m == 0 else 1
    buffer[count : max(count, len(free))] = free[count:]
    cu, slots, positions = [0], [], []
    for r, (c, m) in enumerate(zip(lens, new)):
        cu.append(cu[-1] + m)
        positions += range(c, c + m)
        slots += [table[r][p // page] * page + p % page for p in range(c, c + m)]
    behind = s["slots"].numel() - len(slots)
    out = {"page_table": table, "free_pages": buffer, "prefix_lens": lens, "new_lens": new, "cu_new_lens": cu,
           "lens_out": [c + m for c, m in zip(lens, new)], "held_out": held, "free_count_out": [len(free)], "slots": slots + [-1] * behind,
           "positions": positions + [0] * behind, "refused": [refused]}
    return {k: torch.tensor(v, dtype=s[k].dtype, device=DEVICE) for k, v in out.items()}


def _exact_rows(case, s):
    host = {k: s[k].tolist() for k in ("prefix_lens", "new_lens", "cu_new_lens", "page_table")}
    n, d = case["rotary"], case["head_dim"]
    dt = s["q"].dtype
    turn = None
    if n:
        if s["positions"] is None:
            at = torch.cat([torch.arange(c, c + m, device=DEVICE) for c, m in zip(host["prefix_lens"], host["new_lens"])]).double()[:, None].expand(-1, n // 2)
        else:
            at = torch.cat([s["positions"][a].double()[:, None].expand(-1, width) for a, width in enumerate(_sections(case))], dim=1)
        angle = at * s["inv_freq"]
        turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]

    def row(x, weight):
        x = x.double()
        x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / d + EPS) * weight.double()
        if n:
            pair = (slice(0, n // 2), slice(n // 2, n)) if case["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
            z = torch.complex(x[..., pair[0]].contiguous(), x[..., pair[1]].contiguous()) * turn
            x[..., pair[0]], x[..., pair[1]] = z.real, z.imag
        return x

    out = {"q": row(s["q"], s["q_weight"]), "k": row(s["k"], s["k_weight"])}
    if case["op"] == "norm":
        return out
    page = case["page"]
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].to(dt).double()
    for r, (c, m) in enumerate(zip(host["prefix_lens"], host["new_lens"])):
        at = torch.arange(c, c + m, device=DEVICE)
        pages, lo = torch.tensor(host["page_table"][r], device=DEVICE)[at // page], host["cu_new_lens"][r]
        k_cache[pages, :, at % page] = out["k"][lo : lo + m]
        v_cache[pages, :, at % page] = s["v"][lo : lo + m].double()
    return {"q": out["q"], "k": k_cache, "v": v_cache}


def _exact_window(case, s):
    host = {k: s[k].tolist() for k in ("prefix_lens", "new_lens", "cu_new_lens", "page_table")}
    heads, kv_heads, d, page, w = case["heads"], case["kv_heads"], case["head_dim"], case["page"], case["window"]
    g = heads // kv_heads
    out = torch.zeros((s["tokens"], heads, d), device=DEVICE, dtype=torch.float64)
    lse = torch.full((s["tokens"], heads), -math.inf, device=DEVICE, dtype=torch.float64)
    for r in range(case["reqs"]):
        c, m, row0 = host["prefix_lens"][r], host["new_lens"][r], host["cu_new_lens"][r]
        ids = torch.tensor(host["page_table"][r], device=DEVICE)
        step = max(1, (1 << 27) // ((w + m + case["sinks"]) * g))            # at most a gigabyte of scores at a time
        for t0 in range(0, m, step):
            t1 = min(m, t0 + step)
            token = torch.arange(c + t0, c + t1, device=DEVICE)
            low = max(0, c + t0 - w + 1)
            at = torch.cat([torch.arange(0, min(case["sinks"], low), device=DEVICE), torch.arange(low, c + t1, device=DEVICE)])
            hidden = (at[None, :] > token[:, None]) | ((token[:, None] - at[None, :] >= w) & (at[None, :] >= case["sinks"]))
            hidden = hidden.repeat_interleave(g, dim=0)
            k_all, v_all = (s[name][ids[at // page], :, at % page].double() for name in ("k_cache", "v_cache"))
            for h in range(kv_heads):
                sc = (s["q"][row0 + t0 : row0 + t1, h * g : (h + 1) * g].double().reshape(-1, d) @ k_all[:, h].t().contiguous()) / math.sqrt(d)
                sc.masked_fill_(hidden, -math.inf)
                top = torch.logsumexp(sc, dim=1)
                lse[row0 + t0 : row0 + t1, h * g : (h + 1) * g] = top.reshape(-1, g)
                out[row0 + t0 : row0 + t1, h * g : (h + 1) * g] = (torch.exp(sc - top[:, None]) @ v_all[:, h].contiguous()).reshape(-1, g, d)
    return {"out": out, "lse": lse}

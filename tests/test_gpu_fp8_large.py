"""The calls of the 8-bit cache and of rotary positions at the ends of what they take: contexts as long as a row of the page
table may be, batches whose rows, slots or requests make the kernels go their ways for large calls.  References and
tolerances are those of test_gpu_fp8_cache.py unless a test says otherwise."""
import math

import numpy as np
import pytest
import torch

from oracle import fp8_model as F
from paper_2507_10069_amd import binding as B
from test_gpu_fp8_cache import DEV, Batch, _check_rotated, _dev, _f64, _torch_dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [20, 7], ids=["chunk kernel", "few rows"])
def test_the_longest_context(heads):
    """2^30 slots, the most that a row of the page table may hold, in two pages: every key counts, the last ones too.  Queries of
    zeros make all weights 1 and every sum exact in 32 bits: V is 1, and 2 in the last 1/128, so that out is 129 / 128 (exact in bf16)
    and lse 30 ln 2 (2^-22 of itself: one logarithm, one product)."""
    print("case longest context", heads, flush=True)
    slots, page = 1 << 30, 256
    table = torch.zeros((1, slots // page), dtype=torch.int32, device=DEV)
    table[0, slots // page // 128 * 127:] = 1
    lens = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([slots - 1], [1], [0, 1])]
    batch = B.make_batch(num_reqs=1, num_q_heads=heads, num_kv_heads=1, head_dim=128, page_size=page, num_pages=2, max_pages_per_req=slots // page,
                         total_new_tokens=1, max_new_len=1, dtype="bf16", softmax_scale=1.0, page_table=table, prefix_lens=lens[0], new_lens=lens[1],
                         cu_new_lens=lens[2])
    k = torch.full((2, 1, page, 128), 0x31, dtype=torch.uint8, device=DEV)
    v = torch.full((2, 1, page, 128), 0x38, dtype=torch.uint8, device=DEV)                 # the code of 1
    k_scale = torch.full((2, 1, page), 127, dtype=torch.uint8, device=DEV)
    v_scale = torch.tensor([127, 128], dtype=torch.uint8, device=DEV)[:, None, None].expand(2, 1, page).contiguous()
    q, out = torch.zeros((1, heads, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((1, heads, 128), dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((1, heads), device=DEV)
    workspace = torch.empty(B.emm_attn_fp8_workspace_size(batch), dtype=torch.uint8, device=DEV)
    B.emm_decode_attn_fp8(batch, q, B.make_fp8_cache(k, v, k_scale, v_scale), out, lse, workspace)
    torch.cuda.synchronize()
    assert (out == 129 / 128).all(), out.float().unique()
    assert ((lse.double() - 30 * math.log(2)).abs() <= 2.0 ** -22 * 30 * math.log(2)).all(), lse.unique()


# ---- rows of large calls: several passes of one wave over a token's rows, two slots of one wave, many requests ------------

WAVES_AT_ONCE = 4096                                         # rows are spread over a wave for each pass up to so many waves


def _passes(rows, d):
    return -(-rows * (d // 16) // 64)


def _in_small_calls(b, size):
    """(batch of one request, its packed rows) for at most `size` new tokens of a request at a time."""
    for r in range(len(b.new)):
        for j in range(0, int(b.new[r]), size):
            n = min(size, int(b.new[r]) - j)
            lens = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([int(b.prefix[r]) + j], [n], [0, n])]
            yield B.make_batch(num_reqs=1, num_q_heads=b.heads, num_kv_heads=b.kv_heads, head_dim=b.d, page_size=b.page, num_pages=b.num_pages,
                               max_pages_per_req=b.table.shape[1], total_new_tokens=n, max_new_len=n, dtype=b.dtype, softmax_scale=1.0,
                               page_table=b.dev["table"][r:r + 1].contiguous(), prefix_lens=lens[0], new_lens=lens[1],
                               cu_new_lens=lens[2]), slice(int(b.cu[r]) + j, int(b.cu[r]) + j + n)


@pytest.mark.parametrize("dtype,d,heads,kv_heads,rot,layout,axes,strided", [
    ("bf16", 128, 28, 4, 128, "half", 3, True), ("bf16", 128, 28, 4, 128, "half", 0, False), ("bf16", 128, 32, 8, 64, "interleaved", 0, True),
    ("f32", 64, 60, 5, 64, "half", 1, False)])
def test_rotation_and_write_of_a_long_prompt(dtype, d, heads, kv_heads, rot, layout, axes, strided):
    """A wave does all passes over a token's K, V and q rows: the reference's values, and the bits of the same rows in calls so small
    that a wave does one."""
    print("case long rotation and write", dtype, d, heads, kv_heads, rot, layout, axes, strided, flush=True)
    b = Batch([16, 0, 700, 5, 3], [701, 0, 530, 33, 1], heads=heads, kv_heads=kv_heads, d=d, dtype=dtype, seed=rot + axes)
    dt, small = _torch_dtype(dtype), 64
    assert b.T * _passes(heads + kv_heads, d) > WAVES_AT_ONCE >= small * _passes(heads + 2 * kv_heads, d)
    rows = _dev(b.rng.standard_normal((b.T, heads + 2 * kv_heads, d)).astype(np.float32), dt)
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv_heads], rows[:, heads + kv_heads:]
    stride = (heads + 2 * kv_heads) * d if strided else 0
    if not strided:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    at = np.concatenate([np.arange(p, p + n) for p, n in zip(b.prefix, b.new)])
    sections = [rot // 4, rot // 8, rot // 2 - rot // 4 - rot // 8] if axes == 3 else [rot // 2]
    pos = b.rng.integers(0, 100000, (axes, b.T)).astype(np.int32) if axes else at[None]
    inv, factor = B.emm_rope_inv_freq_host(rot, 1e6, "yarn", 2.0, 32768)

    def rope_of(part):
        given = _dev(pos[:, part]) if axes else None
        return B.make_rope(_dev(inv), rotary_dim=rot, layout=layout, factor=factor, positions=given, sections=sections if axes else None)
    q_out, k_out, fused = torch.full((b.T, heads, d), 9.0, dtype=dt, device=DEV), torch.full((b.T, kv_heads, d), 9.0, dtype=dt, device=DEV), {}
    fused_q = torch.full_like(q_out, 9.0)
    every = rope_of(slice(None))
    B.emm_rope(b.batch, every, q, k, q_out, k_out, token_stride=stride)
    B.emm_rope_kv_scatter_fp8(b.batch, every, q, k, v, fused_q, b.to_device(), token_stride=stride)
    fused = {n: t.clone() for n, t in b.pools.items()}
    assert torch.equal(fused_q, q_out)
    per_freq = np.concatenate([np.repeat(pos[a][:, None], w, 1) for a, w in enumerate(sections)], 1)
    for x, got in ((q, q_out), (k, k_out)):
        _check_rotated(_f64(got), _f64(x), F.rotate(_f64(x), per_freq, inv, rot, layout, factor), per_freq, rot, layout, factor, dtype)
    if not strided:                                          # in place, alone and with the write
        x, y, z = q.clone(), k.clone(), q.clone()
        B.emm_rope(b.batch, every, x, y, x, y)
        B.emm_rope_kv_scatter_fp8(b.batch, every, z, k, v, z, b.to_device())
        assert torch.equal(x, q_out) and torch.equal(y, k_out) and torch.equal(z, q_out)
        assert all(torch.equal(fused[n], t) for n, t in b.pools.items())
    cache, small_q = b.to_device(), torch.full_like(q_out, 9.0)
    for batch, part in _in_small_calls(b, small):
        B.emm_rope_kv_scatter_fp8(batch, rope_of(part), q[part], k[part], v[part], small_q[part], cache, token_stride=stride)
    assert torch.equal(small_q, q_out)
    assert all(torch.equal(fused[n], t) for n, t in b.pools.items())
    for r in range(len(b.new)):
        lo, hi = b.cu[r], b.cu[r + 1]
        b.fill("k", r, int(b.prefix[r]), _f64(k_out)[lo:hi]), b.fill("v", r, int(b.prefix[r]), _f64(v)[lo:hi])
    b.check_pools()


@pytest.mark.parametrize("dtype,d,kv_heads", [("bf16", 128, 8), ("f32", 64, 9)])
def test_write_of_many_rows(dtype, d, kv_heads):
    print("case many rows", dtype, d, kv_heads, flush=True)
    b = Batch([9, 0, 31], [2001, 0, 2300], heads=kv_heads, kv_heads=kv_heads, d=d, dtype=dtype, seed=d, extra_rows=3)
    assert _passes(2 * kv_heads, d) > 1 and b.T * _passes(2 * kv_heads, d) > WAVES_AT_ONCE
    k, v = (_dev((b.rng.standard_normal((b.rows, kv_heads, d)) * np.exp2(b.rng.integers(-9, 9, (b.rows, kv_heads, 1)))).astype(np.float32), _torch_dtype(dtype))
            for _ in range(2))
    B.emm_kv_scatter_fp8(b.batch, k, v, b.to_device())
    for r in range(3):
        lo, hi = b.cu[r], b.cu[r + 1]
        b.fill("k", r, int(b.prefix[r]), _f64(k)[lo:hi]), b.fill("v", r, int(b.prefix[r]), _f64(v)[lo:hi])
    b.check_pools()


@pytest.mark.parametrize("requests", [65, 130, 200])
def test_many_requests(requests):
    """A token's request is looked for among more than 64: empty ones in a row, at the head, at the end."""
    print("case many requests", requests, flush=True)
    rng = np.random.default_rng(requests)
    new = rng.integers(0, 4, requests)
    new[:3] = new[60:68] = new[-2:] = 0
    new[5], new[64] = 90, 0
    b = Batch(rng.integers(0, 50, requests), new, heads=4, kv_heads=2, seed=requests, extra_rows=7)
    rows = [_dev(b.rng.standard_normal((b.rows, 2, 128)).astype(np.float32), torch.bfloat16) for _ in range(2)]
    inv, _ = B.emm_rope_inv_freq_host(128, 1e4)
    turned = torch.full_like(rows[0], 5.0)
    B.emm_rope(b.batch, B.make_rope(_dev(inv), rotary_dim=128), None, rows[0], None, turned)
    at = np.concatenate([np.arange(p, p + n) for p, n in zip(b.prefix, b.new)])
    per_freq, x = np.repeat(at[:, None], 64, 1), _f64(rows[0])[: b.T]
    _check_rotated(_f64(turned)[: b.T], x, F.rotate(x, per_freq, inv, 128, "half"), per_freq, 128, "half", 1.0, "bf16")
    assert (turned[b.T:] == 5).all()
    cache = b.to_device()
    B.emm_kv_scatter_fp8(b.batch, *rows, cache)
    for r in range(requests):
        for n, x in zip("kv", rows):
            b.fill(n, r, int(b.prefix[r]), _f64(x)[b.cu[r]:b.cu[r + 1]])
    b.check_pools()
    back = [torch.full_like(x, 3.0) for x in rows]
    B.emm_kv_gather_fp8(b.batch, cache, *back)
    pages, places = b.new_slots()
    for n, x in zip("kv", back):
        assert np.array_equal(_f64(x)[: b.T], F.values_of(b.codes[n][pages, :, places], b.scales[n][pages, :, places])) and (x[b.T:] == 3).all()


@pytest.mark.parametrize("dtype,d,kv_heads,new", [("bf16", 128, 8, [7001, 0, 9403, 1, 2]), ("f32", 128, 8, [1, 9000, 1001, 3]), ("bf16", 64, 16, [16383, 0, 0, 2])])
def test_reading_back_more_than_the_caches_hold(dtype, d, kv_heads, new):
    """From 96 MiB on a wave has two slots: of two requests, of none, and one alone at the end."""
    print("case large read", dtype, d, kv_heads, flush=True)
    b = Batch([0] * len(new), new, heads=kv_heads, kv_heads=kv_heads, d=d, dtype=dtype, seed=d, extra_rows=4)
    assert 2 * b.rows * kv_heads * (d + 1 + d * (2 if dtype == "bf16" else 4)) >= 96 << 20 and b.rows % 2 == 1
    codes = {n: b.rng.integers(0, 256, b.codes[n].shape, dtype=np.uint8) for n in "kv"}
    b.codes = {n: np.where((x & 0x7F) == 0x7F, 0x12, x).astype(np.uint8) for n, x in codes.items()}
    b.scales = {n: b.rng.integers(10, 247, b.scales[n].shape).astype(np.uint8) for n in "kv"}
    gone = (int(b.cu[0]) + 16, int(b.cu[0]) + 32) if new[0] > 32 else (int(b.cu[1]) + 16, int(b.cu[1]) + 32)
    b.table[0 if new[0] > 32 else 1, 1] = b.num_pages         # a page that there is not
    b.dev["table"].copy_(torch.from_numpy(b.table))
    back = [torch.full((b.rows, kv_heads, d), 3.0, dtype=_torch_dtype(dtype), device=DEV) for _ in range(2)]
    B.emm_kv_gather_fp8(b.batch, b.to_device(), *back)
    pages, places = (torch.from_numpy(x).to(DEV) for x in b.new_slots())
    for (c, sc), got in zip((("k", "ks"), ("v", "vs")), back):
        at = pages.clamp(max=b.num_pages - 1)
        want = b.pools[c][at, :, places].view(torch.float8_e4m3fn).double() * torch.exp2(b.pools[sc][at, :, places].double() - 127)[..., None]
        want[gone[0]:gone[1]] = 3
        assert torch.equal(got[: b.T].double(), want) and (got[b.T:] == 3).all()


# ---- attention dealt as a line ------------------------------------------------------------------------------------------

LINE_BYTES = {16: 2 * 512 * 16 * 130 * 4, 32: 2 * 512 * 32 * 130 * 4}        # of the workspace: two records for each of 512 workgroups
STREAMED_TILES = 12000                                       # 32-key tiles of a call from which on private pages go past the caches


def _over_few_pages(prefix, new, seed, shared=(), pool=400, **kw):
    """Long contexts over a pool of few pages, each held many times; requests in `shared` begin with the same pages, nine tenths of the longest."""
    b = Batch([16 * (pool // len(prefix) - 1)] * len(prefix), new, seed=seed, **kw)
    b.prefix[:] = prefix
    width = -(-int((b.prefix + b.new).max()) // b.page)
    # no two requests have the same page in the same place, but for those that share
    b.table = np.argsort(b.rng.random((b.num_pages, width)), axis=0)[: len(prefix)].astype(np.int32)
    for group in shared:
        b.table[group, : width * 9 // 10] = b.table[group[0], : width * 9 // 10]
    codes = {n: torch.from_numpy(b.rng.standard_normal(b.codes[n].shape).astype(np.float32) * 120).clamp(-448, 448) for n in "kv"}
    b.codes = {n: x.to(torch.float8_e4m3fn).view(torch.uint8).numpy() for n, x in codes.items()}
    b.scales = {n: b.rng.integers(118, 122, b.codes[n].shape[:3]).astype(np.uint8) for n in "kv"}
    b.valid = {n: np.ones(b.codes[n].shape[:3], bool) for n in "kv"}
    b.dev["table"], b.batch.max_pages_per_req = _dev(b.table), width
    b.batch.page_table = b.dev["table"].data_ptr()
    b.dev["prefix"].copy_(torch.from_numpy(b.prefix))
    b.to_device()
    return b


LINES = {
    # requests that share most of their pages, and others of other lengths beside them: from one part of a pair to the next a
    # workgroup goes from loads through the caches to loads past them and back
    "shared and private pages": (16, dict(prefix=[3000 + 37 * i for i in range(64)], new=[1] * 64, shared=[list(range(0, 20)), [25, 40, 41]])),
    "shared and private pages, 28 rows": (32, dict(prefix=[1800 + 23 * (i % 7) for i in range(70)], new=[4, 3, 4, 0, 1] * 14, shared=[list(range(9)), [30, 68]])),
    "all private, 28 rows": (32, dict(prefix=[1700] * 70, new=[4] * 70)),
    # parts of more than 128 tiles: a wave asks for page ids again
    "long parts": (16, dict(prefix=[150000, 149990, 120001, 150000, 3], new=[1] * 5)),
    "long parts, 28 rows": (32, dict(prefix=[150000, 149990, 120001, 150000, 3], new=[4, 4, 4, 3, 1])),
}


def _ways_of_workgroups(b, tiles):
    """For each of 512 workgroups, part by part: does another request hold the page that the part begins with?  The line is cut evenly; a part
    ends with its workgroup's share or with its (request, KV head) pair."""
    share, x, ways, own = -(-tiles // 512), 0, [[] for _ in range(512)], -(-(b.prefix + b.new) // 32)
    for r in range(len(b.new)):
        for _ in range(b.kv_heads if b.new[r] else 0):
            t = 0
            while t < own[r]:
                column = b.table[:, 2 * t]
                ways[x // share].append(int((column == b.table[r, 2 * t]).sum() > 1))
                step = min(int(own[r]) - t, share - x % share)
                x, t = x + step, t + step
    assert x == tiles
    return ways


@pytest.mark.parametrize("name", list(LINES))
def test_line_of_tiles(name):
    print("case line", name, flush=True)
    rows, kw = LINES[name]
    b = _over_few_pages(seed=len(name), **kw)
    tiles = int((-(-(b.prefix + b.new) // 32) * (b.new > 0)).sum()) * b.kv_heads
    assert B.emm_attn_fp8_workspace_size(b.batch) == LINE_BYTES[rows] and tiles >= STREAMED_TILES      # it goes the way that it is here for
    assert ("long" in name) == (-(-tiles // 512) > 128)
    if "shared" in name:                                     # some go from one way of loading to the other, and some back
        changes = [(u, v) for w in _ways_of_workgroups(b, tiles) for u, v in zip(w, w[1:])]
        assert (0, 1) in changes and (1, 0) in changes
    q = b.queries()
    out, lse = b.attend(q)
    tokens = sorted(set(b.rng.choice(b.T, min(b.T, 24), replace=False).tolist()) | {0, b.T - 1})
    b.compare(q, out, lse, tokens)
    again, lse_again = b.attend(q)
    assert torch.equal(out, again) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("wider", [0, 40, 300, 1200])
@pytest.mark.parametrize("causal", [True, False])
def test_few_rows_under_tables_of_any_width(wider, causal):
    """A pair's workgroups share its own tiles, not the table's: contexts on both sides of every least part, next to nothing, under tables up to
    the widest that is dealt so."""
    print("case table width", wider, causal, flush=True)
    b = Batch([511, 512, 2047, 2048, 0, 33, 1500], [1, 1, 1, 1, 1, 0, 1], heads=21, kv_heads=3, seed=wider, wider=wider, causal=causal).fill_contexts()
    b.to_device()
    n = B.emm_attn_fp8_workspace_size(b.batch)
    parts, rest = divmod(n, 7 * 3 * 16 * 130 * 4)
    assert rest == 0 and 2 <= parts <= 512 // 21              # a record for each of a pair's workgroups: not the line's
    q, guarded = b.queries(), torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    out, lse = b.attend(q, workspace=guarded[:n])
    b.compare(q, out, lse)
    assert (guarded[n:] == 0xA5).all()
    guarded[:n] = 0xFF                                       # (records of NaN, as far as nobody writes them)
    again, lse_again = b.attend(q, workspace=guarded[:n])
    assert torch.equal(out, again) and torch.equal(lse, lse_again)

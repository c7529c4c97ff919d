"""Rotary positions and the 8-bit cache on the GPU against references in 64 bits (oracle/fp8_model.py for the format and
the rotation, oracle.c over the dequantised pools for the attention).

Tolerances.  Quantising, scales, reading back and moves are exact: bytes are compared.  A rotation: half a step of the
dtype (2^-8 of the value in bf16, 2^-24 in fp32) and the 32-bit arithmetic before it: cosine and sine are at most 5e-7 off
(angle in turns rounded to 2^-25 turns = 1.9e-7 rad, sincospi 2 ulp), the products and their sum 3 * 2^-24: 1e-6 (|a| + |b|).
Attention: softmax weights and the result are rounded to bf16, at most 2^-8 relative each: 2^-8 (sum of p |v| + |out|); a
score is off by at most e = 130 * 2^-24 * scale * |q| |k| (128 sums in 32 bits of exact products), which changes the
weights by 2 e relative, and lse by e, 2^-24 per key summed and 2^-22 of itself."""
import numpy as np
import pytest
import torch

import oracle
from oracle import fp8_model as F
from paper_2507_10069_amd import binding as B
from paper_2507_10069_amd import workloads as W

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _f64(t):
    return t.detach().double().cpu().numpy()


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    return t if dtype is None else t.to(dtype)


def _torch_dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


class Batch:
    """Lengths, a shuffled page table with unused entries of -1, and 8-bit pools full of bytes that mean nothing."""

    def __init__(self, prefix, new, *, heads=28, kv_heads=4, d=128, page=16, dtype="bf16", causal=True, seed=0, spare=3, extra_rows=0, wider=0):
        rng = np.random.default_rng(seed)
        self.rng, self.heads, self.kv_heads, self.d, self.page, self.dtype, self.causal = rng, heads, kv_heads, d, page, dtype, causal
        self.prefix, self.new = np.array(prefix, np.int32), np.array(new, np.int32)
        self.cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.T = int(self.cu[-1])
        ctx = self.prefix + (self.new if causal else 0)
        pages = -(-ctx // page)
        self.num_pages = int(pages.sum()) + spare
        order = rng.permutation(self.num_pages).astype(np.int32)
        self.table = np.full((len(prefix), max(1, int(pages.max())) + wider), -1, np.int32)
        at = 0
        for r, n in enumerate(pages):
            self.table[r, :n] = order[at:at + n]
            at += n
        shape = (self.num_pages, kv_heads, page, d)
        # unused slots: codes of NaN and scale bytes of NaN among other bytes
        self.codes = {n: rng.choice(np.array([0x7F, 0xFF, 0x7E, 0x31], np.uint8), shape) for n in "kv"}
        self.scales = {n: rng.choice(np.array([0xFF, 0, 200, 130], np.uint8), shape[:3]) for n in "kv"}
        self.valid = {n: np.zeros(shape[:3], bool) for n in "kv"}            # slots that hold a row
        self.dev = {n: _dev(getattr(self, n)) for n in ("table", "prefix", "new", "cu")}
        self.rows = self.T + extra_rows
        self.batch = B.make_batch(num_reqs=len(prefix), num_q_heads=heads, num_kv_heads=kv_heads, head_dim=d, page_size=page, num_pages=self.num_pages,
                                  max_pages_per_req=self.table.shape[1], total_new_tokens=self.rows, max_new_len=int(self.new.max()), dtype=dtype,
                                  softmax_scale=1.0 / np.sqrt(d), page_table=self.dev["table"], prefix_lens=self.dev["prefix"], new_lens=self.dev["new"],
                                  cu_new_lens=self.dev["cu"])

    def slots(self, r, first, count):
        at = np.arange(first, first + count)
        return self.table[r, at // self.page], at % self.page

    def new_slots(self):
        """Page and place of every packed token."""
        parts = [self.slots(r, int(p), int(n)) for r, (p, n) in enumerate(zip(self.prefix, self.new))]
        return np.concatenate([a for a, _ in parts]).astype(np.int64), np.concatenate([c for _, c in parts])

    def fill(self, name, r, first, x):
        """Quantises x [n][kv_heads][d] into the host pools."""
        pages, places = self.slots(r, first, len(x))
        self.codes[name][pages, :, places], self.scales[name][pages, :, places] = F.quantise(x)
        self.valid[name][pages, :, places] = True

    def fill_contexts(self, k_scale=1.0):
        for r, (p, n) in enumerate(zip(self.prefix, self.new)):
            c = int(p + (n if self.causal else 0))
            self.fill("k", r, 0, self.rng.standard_normal((c, self.kv_heads, self.d)) * k_scale)
            self.fill("v", r, 0, self.rng.standard_normal((c, self.kv_heads, self.d)))
        return self

    def to_device(self):
        self.pools = {n: _dev(a) for n, a in (("k", self.codes["k"]), ("v", self.codes["v"]), ("ks", self.scales["k"]), ("vs", self.scales["v"]))}
        self.cache = B.make_fp8_cache(self.pools["k"], self.pools["v"], self.pools["ks"], self.pools["vs"])
        return self.cache

    def check_pools(self):
        """The device pools have the bytes of the host's (a NaN code's sign is free)."""
        for n, dev in (("k", "k"), ("v", "v")):
            got, want = self.pools[dev].cpu().numpy(), self.codes[n]
            same = (got == want) | (((got & 0x7F) == 0x7F) & ((want & 0x7F) == 0x7F))
            assert same.all(), (n, np.argwhere(~same)[:3], got[~same][:3], want[~same][:3])
            assert np.array_equal(self.pools[dev + "s"].cpu().numpy(), self.scales[n]), n

    def bits(self, name, absolute=False):
        """The dequantised pool as bf16 bits (exact), slots without meaning at zero."""
        with np.errstate(over="ignore", invalid="ignore"):
            x = F.values_of(self.codes[name], self.scales[name]).astype(np.float32)
        x = np.where(self.valid[name][..., None], x, 0).astype(np.float32)
        return W.to_bf16_bits(np.abs(x) if absolute else x)

    def reference(self, q_bits, tokens=None):
        """out, lse, and sum of p |v| in 64 bits."""
        kind = "causal" if self.causal else "cross"
        args = (kind, self.table, self.prefix, self.new, self.cu, q_bits, self.bits("k"))
        out, lse = oracle.attention(*args, self.bits("v"), self.batch.softmax_scale, tokens)
        size, _ = oracle.attention(*args, self.bits("v", True), self.batch.softmax_scale, tokens)
        return out, lse, size

    def attend(self, q, out=None, lse=None, workspace=None, stream=None):
        out = torch.full((self.rows, self.heads, self.d), 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
        lse = torch.full((self.rows, self.heads), 7.0, dtype=torch.float32, device=DEV) if lse is None else lse
        if workspace is None:
            n = B.emm_attn_fp8_workspace_size(self.batch)
            workspace = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
        call = B.emm_cross_attn_fp8 if not self.causal else B.emm_decode_attn_fp8 if self.new.max() <= 1 else B.emm_prefill_attn_fp8
        call(self.batch, q, self.cache, out, lse, workspace, stream)
        return out, lse

    def queries(self, scale=1.0):
        return _dev(self.rng.standard_normal((self.rows, self.heads, self.d)).astype(np.float32) * scale, torch.bfloat16)

    def compare(self, q, out, lse, tokens=None, rows=slice(None)):
        q_bits = B.DeviceWorkload.to_numpy_bits(q)[: self.T]
        want, want_lse, size = self.reference(q_bits, tokens)
        got, got_lse = _f64(out)[: self.T], _f64(lse)[: self.T]
        if tokens is not None:
            got, got_lse = got[tokens], got_lse[tokens]
        q_len = np.linalg.norm(_f64(q)[: self.T], axis=-1).max(initial=0)
        k_len = np.linalg.norm(W.bf16_bits_to_f32(self.bits("k")).astype(np.float64), axis=-1).max()
        e = 130 * 2.0 ** -24 * self.batch.softmax_scale * q_len * k_len
        keys = int((self.prefix + self.new).max())
        bound = (2.0 ** -8 + 2 * e + keys * 2.0 ** -24) * size + 2.0 ** -8 * np.abs(want) + 1e-30
        off = np.abs(got - want)
        assert np.isfinite(got).all() and (off <= bound).all(), (float(off.max()), np.argwhere(off > bound)[:4], float((off / bound).max()))
        none = np.isneginf(want_lse)
        assert (got[none] == 0).all() and np.isneginf(got_lse[none]).all()
        lse_off, lse_bound = np.abs(got_lse[~none] - want_lse[~none]), e + keys * 2.0 ** -24 + 2.0 ** -22 * np.abs(want_lse[~none]) + 2.0 ** -22
        assert (lse_off <= lse_bound).all(), (float(lse_off.max()), float(lse_bound.min()))
        return float((off / bound).max()), float(lse_off.max()) if lse_off.size else 0.0


# ---- rotary positions -----------------------------------------------------------------------------------------------

def _positions(b, axes, rng):
    """Device positions (or None) and every frequency's own position [T][n] as the reference wants them."""
    if axes == 0:
        at = np.concatenate([np.arange(p, p + n) for p, n in zip(b.prefix, b.new)])
        return None, at
    pos = rng.integers(0, 2 ** 20, (axes, b.rows)).astype(np.int32)
    pos[:, 0] = [2 ** 31 - 1, 0, -5, 17][:axes]
    return _dev(pos), pos


def _check_rotated(got, x, want, per_freq, rot, layout, factor, dtype):
    a = np.abs(x[..., :rot])
    pair = np.roll(a, rot // 2, axis=-1) if layout == "half" else a.reshape(a.shape[:-1] + (rot // 2, 2))[..., ::-1].reshape(a.shape)
    bound = np.zeros(x.shape)
    bound[..., :rot] = 1e-6 * abs(factor) * (a + pair) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want[..., :rot])
    off = np.abs(got - want)
    assert (off <= bound + 1e-38).all(), (float(off.max()), np.argwhere(off > bound)[:3])


ROPE_CASES = [("bf16", 128, 128, "half", 0), ("bf16", 128, 128, "interleaved", 1), ("bf16", 128, 32, "half", 3), ("bf16", 128, 48, "interleaved", 4),
              ("bf16", 64, 64, "half", 3), ("bf16", 64, 16, "interleaved", 0), ("f32", 64, 64, "half", 2), ("f32", 64, 32, "interleaved", 0),
              ("f32", 128, 128, "half", 1), ("f32", 128, 112, "interleaved", 3)]


@pytest.mark.parametrize("dtype,d,rot,layout,axes", ROPE_CASES)
@pytest.mark.parametrize("strided", [False, True])
def test_rope(dtype, d, rot, layout, axes, strided):
    print("case rope", dtype, d, rot, layout, axes, strided, flush=True)
    b = Batch([0, 100000, 31, 5, 0], [3, 1, 0, 17, 1], heads=6, kv_heads=2, d=d, dtype=dtype, seed=d + rot + axes, wider=70000 // 16)
    dt, (H, K) = _torch_dtype(dtype), (6, 2)
    pos, ref_pos = _positions(b, axes, b.rng)
    sections = {0: [], 1: [rot // 2], 2: [3, rot // 2 - 3], 3: [rot // 4, 0, rot // 2 - rot // 4], 4: [1, 2, 3, rot // 2 - 6]}[axes]
    if axes == 0:
        per_freq = np.repeat(ref_pos[:, None], rot // 2, 1)
    else:
        per_freq = np.concatenate([np.repeat(ref_pos[a][:, None], w, 1) for a, w in enumerate(sections)], 1)
    inv, _ = B.emm_rope_inv_freq_host(rot, 1e6)
    rows = _dev(b.rng.standard_normal((b.T, H + 2 * K, d)).astype(np.float32), dt)
    q, k = rows[:, :H], rows[:, H:H + K]
    stride = (H + 2 * K) * d if strided else 0
    if not strided:
        q, k = q.contiguous(), k.contiguous()
    for factor, inverse in ((1.0, False), (1.25, True)):
        rope = B.make_rope(_dev(inv), rotary_dim=rot, layout=layout, factor=factor, inverse=inverse, positions=pos, sections=sections or None)
        q_out, k_out = torch.full((b.T, H, d), 9.0, dtype=dt, device=DEV), torch.full((b.T, K, d), 9.0, dtype=dt, device=DEV)
        before = rows.clone()
        B.emm_rope(b.batch, rope, q, k, q_out, k_out, token_stride=stride)
        assert torch.equal(rows, before)
        for x, got in ((q, q_out), (k, k_out)):
            want = F.rotate(_f64(x), per_freq, inv, rot, layout, factor, inverse)
            _check_rotated(_f64(got), _f64(x), want, per_freq, rot, layout, factor, dtype)
        # one of the two alone, and in place: the same bits
        alone = torch.empty_like(k_out)
        B.emm_rope(b.batch, rope, None, k, None, alone, token_stride=stride)
        assert torch.equal(alone, k_out)
        if not strided:
            x = q.clone()
            B.emm_rope(b.batch, rope, x, None, x, None)
            assert torch.equal(x, q_out)


def test_rope_is_its_own_gradient_and_undone_by_inverse():
    """The inverse is the transpose: <R x, y> = <x, R^T y>, and a difference quotient of x -> <R x, y>."""
    b = Batch([7], [40], heads=2, kv_heads=1, d=64, dtype="f32", seed=3)
    inv, _ = B.emm_rope_inv_freq_host(64, 1e4)
    x, y = (_dev(b.rng.standard_normal((40, 2, 64)).astype(np.float32)) for _ in range(2))

    def turn(t, inverse, factor=1.5):
        out = torch.empty_like(t)
        B.emm_rope(b.batch, B.make_rope(_dev(inv), rotary_dim=64, factor=factor, inverse=inverse), t, None, out, None)
        return out
    grad = _f64(turn(y, True))
    # a rotated pair is off by 1e-6 * 1.5 (|a| + |b|) + 2^-24 of itself: |x| |y| bounds the sums
    tol = 4e-6 * float(torch.linalg.norm(x.double()) * torch.linalg.norm(y.double()))
    assert abs((_f64(turn(x, False)) * _f64(y)).sum() - (_f64(x) * grad).sum()) <= tol
    step = torch.zeros_like(x)
    step[11, 1, 5] = 1.0                                     # linear: a step of 1 is as good as a small one
    diff = ((_f64(turn(x + step, False)) - _f64(turn(x, False))) * _f64(y)).sum()
    assert abs(diff - grad[11, 1, 5]) <= 2e-5 * 8            # |x|, |y| here are below 8 by a wide margin
    back = _f64(turn(turn(x, False, 1.0), True, 1.0))
    assert np.abs(back - _f64(x)).max() <= 1e-5 * 8


def test_rope_leaves_rows_of_no_request():
    b = Batch([3, 9], [4, 2], heads=4, kv_heads=2, seed=5, extra_rows=5)
    inv, _ = B.emm_rope_inv_freq_host(128, 1e4)
    rope = B.make_rope(_dev(inv), rotary_dim=128)
    q = b.queries()[:, :4].contiguous()
    out = torch.full_like(q, 5.0)
    B.emm_rope(b.batch, rope, q, None, out, None)
    assert (out[b.T:] == 5).all() and not (out[: b.T] == 5).any(dim=-1).all()


# ---- the cache: written and read back -------------------------------------------------------------------------------

def _hard_rows(rng, n, kv_heads, d):
    """Rows of all sizes, with ties, zeros, infinities and NaN among them."""
    x = rng.standard_normal((n, kv_heads, d)) * np.exp2(rng.integers(-20, 20, (n, kv_heads, 1)))
    x[rng.random(x.shape) < 0.02] *= 64
    for i, f in enumerate([lambda r: 0 * r, lambda r: np.where(np.arange(d) % 5 == 0, np.inf, r), lambda r: np.where(np.arange(d) % 7 == 0, np.nan, r),
                           lambda r: np.full(d, np.nan), lambda r: np.full(d, 448.0), lambda r: np.full(d, 3.3e38), lambda r: r * 1e-36, lambda r: np.full(d, 1e-40),
                           lambda r: (np.arange(d) - d / 2) * 2.0 ** -4, lambda r: np.where(np.arange(d) == 3, 1.75, np.arange(d) / 256.0)]):
        if i < n:
            x[i, i % kv_heads] = f(x[i, i % kv_heads])
    return x


CACHE_CASES = [([0, 15, 16, 200], [1, 1, 1, 1], 16), ([0, 0, 0], [40, 0, 7], 16), ([7, 1000], [129, 300], 64), ([31, 250, 0], [1, 30, 520], 256), ([5], [1], 32)]


@pytest.mark.parametrize("dtype,d,kv_heads", [("bf16", 128, 4), ("bf16", 64, 3), ("f32", 128, 8), ("f32", 64, 1)])
@pytest.mark.parametrize("prefix,new,page", CACHE_CASES)
@pytest.mark.parametrize("strided", [False, True])
def test_scatter_and_gather(dtype, d, kv_heads, prefix, new, page, strided):
    print("case scatter", dtype, d, kv_heads, prefix, new, page, strided, flush=True)
    b = Batch(prefix, new, heads=kv_heads, kv_heads=kv_heads, d=d, page=page, dtype=dtype, seed=page + d)
    cache, dt = b.to_device(), _torch_dtype(dtype)
    rows = torch.stack([_dev(_hard_rows(b.rng, b.T, kv_heads, d).astype(np.float32), dt) for _ in range(2)], dim=1)      # [T][k, v][heads][d]
    k, v = (rows[:, 0], rows[:, 1]) if strided else (rows[:, 0].contiguous(), rows[:, 1].contiguous())
    B.emm_kv_scatter_fp8(b.batch, k, v, cache, token_stride=2 * kv_heads * d if strided else 0)
    for r in range(len(prefix)):
        lo, hi = b.cu[r], b.cu[r + 1]
        b.fill("k", r, int(b.prefix[r]), _f64(k)[lo:hi])
        b.fill("v", r, int(b.prefix[r]), _f64(v)[lo:hi])
    b.check_pools()
    k_back, v_back = torch.full((b.T, kv_heads, d), 3.0, dtype=dt, device=DEV), torch.full((b.T, kv_heads, d), 3.0, dtype=dt, device=DEV)
    B.emm_kv_gather_fp8(b.batch, cache, k_back, v_back)
    pages, places = b.new_slots()
    for name, back, x in (("k", k_back, k), ("v", v_back, v)):
        want = F.values_of(b.codes[name][pages, :, places], b.scales[name][pages, :, places])
        assert np.array_equal(_f64(back), want, equal_nan=True)
        x = _f64(x)
        x = np.where(np.isfinite(x), np.clip(x, -448 * 2.0 ** 119, 448 * 2.0 ** 119), x)     # what is above is held as that
        finite = np.isfinite(x)
        most = np.where(finite, np.abs(x), 0).max(axis=-1, keepdims=True)
        # half a step: 2^-4 of a value, or half of the least step, 2^-10 of 2^e with 2^e < most / 224 (or the least exponent)
        bound = np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * np.maximum(most / 224, 2.0 ** -117))
        assert (np.abs(_f64(back) - x)[finite] <= np.broadcast_to(bound, x.shape)[finite]).all()
        assert np.isnan(_f64(back)[~finite]).all()


@pytest.mark.parametrize("dtype,layout,axes,strided,heads", [("bf16", "half", 3, True, 28), ("bf16", "interleaved", 0, False, 28), ("f32", "half", 1, True, 4),
                                                              ("bf16", "half", 0, False, 4)])
def test_rope_scatter_has_the_bits_of_the_two_calls(dtype, layout, axes, strided, heads):
    print("case rope + scatter", dtype, layout, axes, strided, heads, flush=True)
    K, d, dt = 4, 128, _torch_dtype(dtype)
    b = Batch([0, 1000, 33, 4], [70, 1, 0, 5], heads=heads, kv_heads=K, d=d, dtype=dtype, seed=heads + axes)
    rows = _dev(b.rng.standard_normal((b.T, heads + 2 * K, d)).astype(np.float32), dt)
    q, k, v = rows[:, :heads], rows[:, heads:heads + K], rows[:, heads + K:]
    stride = (heads + 2 * K) * d if strided else 0
    if not strided:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    pos, _ = _positions(b, axes, b.rng)
    inv, factor = B.emm_rope_inv_freq_host(96, 1e6, "yarn", 4.0, 32768)
    rope = B.make_rope(_dev(inv), rotary_dim=96, layout=layout, factor=factor, positions=pos, sections=[8, 20, 20] if axes == 3 else None)
    cache = b.to_device()
    q_out = torch.empty((b.T, heads, d), dtype=dt, device=DEV)
    B.emm_rope_kv_scatter_fp8(b.batch, rope, q, k, v, q_out, cache, token_stride=stride)
    fused = {n: t.clone() for n, t in b.pools.items()}
    cache = b.to_device()
    q_two, k_two = torch.empty_like(q_out), torch.empty((b.T, K, d), dtype=dt, device=DEV)
    B.emm_rope(b.batch, rope, q, k, q_two, k_two, token_stride=stride)
    B.emm_kv_scatter_fp8(b.batch, k_two, v.contiguous(), cache)
    assert torch.equal(q_out, q_two)
    for n, t in b.pools.items():
        assert torch.equal(fused[n], t), n
    for r in range(4):                                       # and those of the reference, of the rotated rows
        b.fill("k", r, int(b.prefix[r]), _f64(k_two)[b.cu[r]:b.cu[r + 1]])
        b.fill("v", r, int(b.prefix[r]), _f64(v)[b.cu[r]:b.cu[r + 1]])
    b.check_pools()
    if not strided:
        x = q.clone()
        B.emm_rope_kv_scatter_fp8(b.batch, rope, x, k, v, x, b.to_device())
        assert torch.equal(x, q_out)


def test_scatter_and_gather_skip_what_has_no_slot():
    """Entries of the table outside the pool, slots outside the table, rows of no request: nothing is written."""
    b = Batch([10, 0, 60], [8, 3, 8], kv_heads=2, heads=2, seed=8, extra_rows=4)
    b.table[1, 0] = b.num_pages + 7
    b.prefix[2] = b.table.shape[1] * 16 - 3                  # its last five tokens lie behind the table
    b.table[2, -1] = b.table[2, 3]
    b.dev["table"].copy_(_dev(b.table))
    b.dev["prefix"].copy_(_dev(b.prefix))
    cache = b.to_device()
    k = _dev(b.rng.standard_normal((b.rows, 2, 128)).astype(np.float32), torch.bfloat16)
    B.emm_kv_scatter_fp8(b.batch, k, k, cache)
    b.fill("k", 0, 10, _f64(k)[:8]), b.fill("v", 0, 10, _f64(k)[:8])
    b.fill("k", 2, int(b.prefix[2]), _f64(k)[11:14]), b.fill("v", 2, int(b.prefix[2]), _f64(k)[11:14])
    b.check_pools()
    out = torch.full_like(k, 3.0)
    B.emm_kv_gather_fp8(b.batch, cache, out, out.clone())
    assert (out[8:11] == 3).all() and (out[14:] == 3).all() and not (out[:8] == 3).all()


def test_pages_migrate_as_they_are():
    """Codes and scales of a request's pages to another pool by the migration calls; attention over them has the same bits."""
    b = Batch([90], [5], seed=9).fill_contexts()
    b.to_device()
    q = b.queries()
    want, _ = b.attend(q)
    n, ids = 6, b.dev["table"][0, :6].contiguous()
    other = torch.tensor([4, 1, 7, 0, 6, 2], dtype=torch.int32, device=DEV)
    moved = {}
    for a, c, page_bytes in (("k", "v", 4 * 16 * 128), ("ks", "vs", 4 * 16)):
        staging = torch.empty(n * 2 * page_bytes, dtype=torch.uint8, device=DEV)
        moved[a], moved[c] = (torch.zeros((8,) + b.pools[x].shape[1:], dtype=torch.uint8, device=DEV) for x in (a, c))
        B.emm_kv_pages_pack(b.pools[a], b.pools[c], b.num_pages, page_bytes, ids, n, staging)
        B.emm_kv_pages_unpack(staging, other, n, moved[a], moved[c], 8, page_bytes)
    b.dev["table"][0, :6] = other
    b.batch.num_pages = 8
    b.cache = B.make_fp8_cache(moved["k"], moved["v"], moved["ks"], moved["vs"])
    got, _ = b.attend(q)
    assert torch.equal(got, want)


# ---- attention ------------------------------------------------------------------------------------------------------

ATTENTION_CASES = {
    "decode_ragged": dict(prefix=[0, 1, 15, 16, 31, 33, 500, 1500], new=[1] * 8),
    "decode_gaps": dict(prefix=[40, 7, 300, 0], new=[1, 0, 1, 0]),
    "decode_mha": dict(prefix=[100, 64], new=[1, 1], heads=8, kv_heads=8, page=64),
    "decode_16_heads_a_group": dict(prefix=[257, 30], new=[1, 1], heads=16, kv_heads=1, page=32),
    "decode_20_heads_a_group": dict(prefix=[127, 1023], new=[1, 1], heads=40, kv_heads=2),
    "decode_many": dict(prefix=list(range(3, 300, 3)), new=[1] * 99, heads=8, kv_heads=2),
    "decode_long": dict(prefix=[20000, 3, 9000], new=[1, 1, 1]),
    "decode_wide_table": dict(prefix=[900, 77], new=[1, 1], wider=4000),
    "decode_wider_table": dict(prefix=[900, 77, 0, 2500, 31], new=[1, 1, 1, 1, 0], wider=12000),
    "decode_wider_table_cross": dict(prefix=[900, 77, 0, 2500, 31], new=[1, 1, 1, 1, 0], wider=12000, causal=False),
    "decode_whole_pairs": dict(prefix=[511, 0, 31, 32, 255, 500], new=[1, 1, 1, 1, 0, 1]),
    "decode_20_heads_a_group_more": dict(prefix=[127, 1023, 0, 31, 32, 5, 64, 700, 96, 2], new=[1] * 10, heads=40, kv_heads=2),
    "few_rows_of_many": dict(prefix=[1000, 0, 63, 31, 200], new=[2, 3, 4, 1, 4]),
    "few_rows_of_many_cross": dict(prefix=[1000, 0, 63, 31, 200], new=[2, 3, 4, 0, 4], causal=False),
    "few_rows": dict(prefix=[1000, 0, 63], new=[2, 3, 5]),
    "few_rows_one_head": dict(prefix=[95, 96, 97], new=[33, 1, 64], heads=2, kv_heads=2),
    "prompts": dict(prefix=[0, 17, 100, 0], new=[33, 1, 64, 100]),
    "prompts_pages_of_256": dict(prefix=[0, 300], new=[257, 90], page=256, heads=8, kv_heads=2),
    "prompt_alone": dict(prefix=[0], new=[700], heads=8, kv_heads=2),
    "prompt_and_decode": dict(prefix=[2000, 300, 0, 5000], new=[1, 300, 0, 1], heads=32, kv_heads=8),
    "question": dict(prefix=[16384], new=[36]),
    "questions": dict(prefix=[3000, 4100, 2047], new=[9, 40, 2]),
    "many_short": dict(prefix=[(37 * i) % 90 for i in range(70)], new=[1 + (i * 7) % 12 for i in range(70)], heads=8, kv_heads=2),
    "units_cut_in_two": dict(prefix=[700] * 5, new=[180] * 5),
    "decode_600_requests": dict(prefix=[640 + i % 64 for i in range(600)], new=[1] * 600, heads=8, kv_heads=1),
    "cross": dict(prefix=[0, 5, 1000, 64], new=[3, 300, 17, 1], causal=False),
    "cross_one_token_each": dict(prefix=[700, 0, 33], new=[1, 1, 1], causal=False),
    "cross_nothing": dict(prefix=[0, 0], new=[5, 1], causal=False),
}


@pytest.mark.parametrize("name", list(ATTENTION_CASES))
def test_attention(name):
    print("case attention", name, flush=True)
    kw = ATTENTION_CASES[name]
    b = Batch(seed=len(name), **kw).fill_contexts()
    b.to_device()
    q = b.queries()
    out, lse = b.attend(q)
    print("   of the bound, lse:", b.compare(q, out, lse), flush=True)
    again, lse_again = b.attend(q)
    assert torch.equal(out, again) and torch.equal(lse, lse_again)           # every run the same bits
    no_lse = torch.empty_like(out)
    n = B.emm_attn_fp8_workspace_size(b.batch)
    call = B.emm_prefill_attn_fp8 if b.causal else B.emm_cross_attn_fp8
    call(b.batch, q, b.cache, no_lse, None, torch.empty(n, dtype=torch.uint8, device=DEV) if n else None)
    assert torch.equal(out, no_lse)


@pytest.mark.parametrize("prefix,new,reqs", [(16384, 2048, 2), (8191, 1, 64)])
def test_attention_of_large_batches_on_sampled_tokens(prefix, new, reqs):
    print("case large", prefix, new, reqs, flush=True)
    b = Batch([prefix] * reqs, [new] * reqs, seed=1)
    codes = (torch.randn((b.num_pages, 4, 16, 128), device=DEV, generator=torch.Generator(DEV).manual_seed(1)) * 120).clamp(-448, 448).to(torch.float8_e4m3fn)
    b.codes = {"k": codes.view(torch.uint8).cpu().numpy(), "v": codes.flip(0).contiguous().view(torch.uint8).cpu().numpy()}
    b.scales = {n: b.rng.integers(118, 122, b.codes["k"].shape[:3]).astype(np.uint8) for n in "kv"}
    b.valid = {n: np.ones(b.codes[n].shape[:3], bool) for n in "kv"}
    b.to_device()
    q = b.queries()
    out, lse = b.attend(q)
    tokens = sorted({0, 1, new - 1, new, b.T - 1} & set(range(b.T)) | set(b.rng.integers(0, b.T, 12).tolist()))
    print("   of the bound, lse:", b.compare(q, out, lse, tokens), flush=True)


LAST_ROUNDS = {
    "cut behind whole ones": ([600 + 40 * i for i in range(16)], [180] * 16),                # 320 units of 256 rows
    "three quarters of a round": ([4200] * 8, [200] * 8),                                    # 192
    "of many lengths": ([100, 6000, 0, 9000, 4500, 300, 5000], [300, 200, 256, 37, 220, 250, 300]),     # 188
    "more behind whole ones": ([4300, 4100, 5000] * 4, [340, 256, 300] * 4),                # 416
}


@pytest.mark.parametrize("name", list(LAST_ROUNDS))
def test_units_behind_the_last_whole_round(name):
    """What fills less than half of the chip is cut along the keys, more is not."""
    print("case last round", name, flush=True)
    b = Batch(*LAST_ROUNDS[name], seed=23).fill_contexts()
    b.to_device()
    q = b.queries()
    out, lse = b.attend(q)
    firsts = [int(x) for c in b.cu[:-1] for x in (c, c + 20)]
    b.compare(q, out, lse, sorted(set(b.rng.choice(b.T, 40, replace=False).tolist() + firsts + [b.T - 1])))
    again, lse_again = b.attend(q)
    assert torch.equal(out, again) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("prefix,new", [([3300] * 32, [1] * 32), ([3000, 2000, 3001], [1, 1, 1]), ([2048] * 3, [50] * 3)])
def test_pages_in_several_places(prefix, new):
    """Requests whose contexts begin with the same pages, and a context that holds a page twice."""
    b = Batch(prefix, new, seed=24).fill_contexts()
    for r in range(1, len(prefix)):
        b.table[r, :100] = b.table[r // 2, :100]
    b.table[0, 20:25] = b.table[0, 7]
    b.table[-1, 101] = b.table[-1, 100]
    b.dev["table"].copy_(torch.from_numpy(b.table))
    b.to_device()
    q = b.queries()
    b.compare(q, *b.attend(q), sorted(set(b.rng.integers(0, b.T, 20).tolist()) | {0, b.T - 1}))


@pytest.mark.parametrize("prefix,new", [([900, 3, 40], [1, 1, 1]), ([700, 0, 33], [60, 300, 2])])
def test_pools_of_more_than_4_gib(prefix, new):
    """Pages whose codes lie below and beyond 2^31 and 2^32 bytes: writing, reading back and attention have the bits of a small pool's."""
    b = Batch(prefix, new, seed=25, spare=4).fill_contexts()
    cache, q = b.to_device(), b.queries()
    rows = [_dev(b.rng.standard_normal((b.T, 4, 128)).astype(np.float32), torch.bfloat16) for _ in range(2)]

    def run(batch, cache):
        B.emm_kv_scatter_fp8(batch, *rows, cache)
        read = [torch.empty_like(x) for x in rows]
        B.emm_kv_gather_fp8(batch, cache, *read)
        b.batch, b.cache = batch, cache
        return (*read, *b.attend(q))
    far_pages = 530000                                       # of 8 KiB: 4.04 GiB of codes for K, and for V
    at = torch.linspace(0, far_pages - 1, b.num_pages).round().long().to(DEV)
    far = {n: torch.empty((far_pages,) + x.shape[1:], dtype=torch.uint8, device=DEV) for n, x in b.pools.items()}
    for n, x in far.items():
        x[at] = b.pools[n]
    want = run(b.batch, cache)
    table = b.dev["table"].long()
    b.dev["table"].copy_(torch.where(table >= 0, at[table.clamp(min=0)], table))
    b.batch.num_pages = far_pages
    got = run(b.batch, B.make_fp8_cache(far["k"], far["v"], far["ks"], far["vs"]))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    for n, x in far.items():
        assert torch.equal(x[at], b.pools[n]), n


@pytest.mark.parametrize("new", [[1, 1], [40, 300]])
def test_scores_that_jump(new):
    """Keys far above everything before them, in the middle and at the end of a context: the running reference has to follow."""
    b = Batch([3000, 1111], new, seed=12).fill_contexts()
    for r, at in ((0, 64), (0, 1500), (0, 2999), (1, 1000), (1, 1110)):
        b.fill("k", r, at, b.rng.standard_normal((1, 4, 128)) * (20 if at != 1500 else 60))
    b.to_device()
    q = b.queries(4.0)
    out, lse = b.attend(q)
    print("   of the bound, lse:", b.compare(q, out, lse), flush=True)


def test_values_of_many_sizes():
    """V rows whose scales differ by many powers of two: they meet the weights as exact factors."""
    b = Batch([400, 90], [1, 60], seed=13).fill_contexts()
    for r, c in ((0, 401), (1, 150)):
        b.fill("v", r, 0, b.rng.standard_normal((c, 4, 128)) * np.exp2(b.rng.integers(-30, 31, (c, 4, 1)).astype(np.float64)))
    b.to_device()
    q = b.queries()
    b.compare(q, *b.attend(q))


@pytest.mark.parametrize("prefix,new,heads", [([50], [4], 4), ([50], [200], 28), ([2000], [90], 28), ([300], [3], 28)])
@pytest.mark.parametrize("bad", ["v", "k"])
def test_what_is_not_a_number_reaches_only_rows_that_see_it(prefix, new, heads, bad):
    b = Batch(prefix, new, heads=heads, seed=14).fill_contexts()
    at = new[0] // 2                                         # a token in the middle of the new ones
    pages, places = b.slots(0, prefix[0] + at, 1)
    b.codes[bad][pages[0], 1, places[0], 5:9] = [0x7F, 0xFF, 0x7F, 0x7F]
    b.to_device()
    q = b.queries()
    out, lse = b.attend(q)
    got = _f64(out)
    G = heads // 4
    hit = np.zeros(got.shape, bool)
    if bad == "v":
        hit[at:, G:2 * G, 5:9] = True
    else:
        hit[at:, G:2 * G] = True
    assert np.array_equal(np.isnan(got), hit)
    b.codes[bad][pages[0], 1, places[0], 5:9] = 0            # the others as if it were a zero
    want, want_lse, size = b.reference(B.DeviceWorkload.to_numpy_bits(q))
    clean = np.zeros(hit.shape, bool)
    clean[:at] = True
    clean[:, :G] = clean[:, 2 * G:] = True
    if bad == "v":
        clean |= ~hit
    assert (np.abs(got - want)[clean] <= (2.0 ** -7 * (size + np.abs(want)) + 1e-4)[clean]).all()
    assert not np.isnan(_f64(lse)[:at]).any() and np.isnan(_f64(lse)[at:, G]).all() == (bad == "k")


@pytest.mark.parametrize("bad", ["v", "k"])
def test_what_is_not_a_number_among_few_rows_of_many(bad):
    """Several new tokens in one pass of two accumulators: those before the slot, and the other requests, keep their bits."""
    b = Batch([300, 40, 500, 31, 64], [4, 4, 2, 1, 4], seed=26).fill_contexts()
    b.to_device()
    q = b.queries()
    clean, clean_lse = b.attend(q)
    page, place = b.slots(1, 42, 1)                          # token 2 of request 1, rows 6 and 7
    b.pools[bad][int(page[0]), 2, int(place[0]), 9] = 0x7F
    got, lse = b.attend(q)
    hit = torch.zeros_like(clean, dtype=torch.bool)
    hit[6:8, 14:21, 9:10] = True
    if bad == "k":
        hit[6:8, 14:21] = True
    assert torch.equal(torch.isnan(got), hit) and torch.equal(got[~hit.any(-1)], clean[~hit.any(-1)])
    assert torch.equal(torch.isnan(lse), hit.all(-1)) and torch.equal(lse[~hit.any(-1)], clean_lse[~hit.any(-1)])


def test_a_row_of_q_that_is_not_a_number_stays_alone():
    b = Batch([300, 40], [1, 1], seed=15).fill_contexts()
    b.to_device()
    q = b.queries()
    clean, _ = b.attend(q)
    q[0, 3, 17], q[1, 9, 0] = float("nan"), float("inf")
    got, _ = b.attend(q)
    assert torch.isnan(got[0, 3]).all() and torch.isnan(got[1, 9]).all()
    got[0, 3], got[1, 9] = clean[0, 3], clean[1, 9]
    assert torch.equal(got, clean)


def test_rows_behind_the_batch_and_bytes_behind_the_workspace_stay():
    for prefix, new in (([900, 30], [1, 1]), ([5000], [36]), ([600, 100], [300, 20])):
        b = Batch(prefix, new, seed=16, extra_rows=6).fill_contexts()
        b.to_device()
        q = b.queries()
        n = B.emm_attn_fp8_workspace_size(b.batch)
        guarded = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
        out, lse = b.attend(q, workspace=guarded[:n] if n else None)
        assert (guarded[n:] == 0xA5).all() and (out[b.T:] == 7).all() and (lse[b.T:] == 7).all()
        b.compare(q, out, lse)


def test_a_batch_padded_for_capture():
    """max_new_len and the token count say what there could be; the lengths say what there is."""
    for new, most in (([3, 1, 0, 0], 64), ([1, 1, 0, 0], 16), ([40, 2, 0, 0], 64)):
        b = Batch([900, 30, 0, 0], new, seed=22, extra_rows=64, wider=70).fill_contexts()
        b.batch.max_new_len = most
        b.to_device()
        q = b.queries()
        out, lse = torch.full((b.rows, 28, 128), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((b.rows, 28), 7.0, device=DEV)
        ws = torch.empty(max(16, B.emm_attn_fp8_workspace_size(b.batch)), dtype=torch.uint8, device=DEV)
        B.emm_prefill_attn_fp8(b.batch, q, b.cache, out, lse, ws)
        assert (out[b.T:] == 7).all() and (lse[b.T:] == 7).all()
        b.compare(q, out, lse)


def _two_streams_case():
    a, c = Batch([4000, 50, 700], [1, 1, 1], seed=17).fill_contexts(), Batch([2500], [40], seed=18).fill_contexts()
    a.to_device(), c.to_device()
    return a, c


def test_calls_on_two_streams_at_once():
    a, c = _two_streams_case()
    qa, qc = a.queries(), c.queries()
    want = [a.attend(qa)[0].clone(), c.attend(qc)[0].clone()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    bufs = [[torch.empty_like(want[i]) for _ in range(8)] for i in range(2)]
    spaces = [torch.empty(max(16, B.emm_attn_fp8_workspace_size(x.batch)), dtype=torch.uint8, device=DEV) for x in (a, c)]
    lses = [torch.empty(w.shape[:2], device=DEV) for w in want]
    torch.cuda.synchronize()
    for k in range(8):
        for i, (x, q) in enumerate(((a, qa), (c, qc))):
            x.attend(q, out=bufs[i][k], lse=lses[i], workspace=spaces[i], stream=streams[i])
            got[i].append(bufs[i][k])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_a_step_captured_and_replayed():
    """Rotation, write and attention of a decode step and of a question in a graph; eager work between the replays."""
    for prefix, new in (([700, 50, 3000], [1, 1, 1]), ([2500], [30])):
        b = Batch(prefix, new, seed=19).fill_contexts()
        cache = b.to_device()
        inv, _ = B.emm_rope_inv_freq_host(128, 1e6)
        rope = B.make_rope(_dev(inv), rotary_dim=128)
        rows = _dev(b.rng.standard_normal((b.T, 36, 128)).astype(np.float32), torch.bfloat16)
        q_out, out = torch.empty((b.T, 28, 128), dtype=torch.bfloat16, device=DEV), torch.empty((b.T, 28, 128), dtype=torch.bfloat16, device=DEV)
        lse = torch.empty((b.T, 28), device=DEV)
        ws = torch.empty(max(16, B.emm_attn_fp8_workspace_size(b.batch)), dtype=torch.uint8, device=DEV)

        def step():
            B.emm_rope_kv_scatter_fp8(b.batch, rope, rows[:, :28], rows[:, 28:32], rows[:, 32:], q_out, cache, token_stride=36 * 128)
            b.attend(q_out, out=out, lse=lse, workspace=ws)
        step()
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for i in range(4):
            rows.copy_(_dev(b.rng.standard_normal(rows.shape).astype(np.float32), torch.bfloat16))
            out.zero_(), lse.zero_(), ws.fill_(0x55)
            graph.replay()
            torch.cuda.synchronize()
            replayed, replayed_lse = out.clone(), lse.clone()
            out.zero_(), lse.zero_()
            step()
            torch.cuda.synchronize()
            assert torch.equal(replayed, out) and torch.equal(replayed_lse, lse), i


@pytest.mark.parametrize("wider", [0, 12000])
def test_a_captured_step_follows_the_lengths(wider):
    """A decode step and a chunk are captured once; lengths, pages and padding change between the replays."""
    for most, heads, new_of in ((1, 28, lambda rng: [1, 1, 0, 1]), (40, 28, lambda rng: rng.integers(0, 41, 4).tolist())):
        rng = np.random.default_rng(27)
        b = Batch([3000] * 4, [most] * 4, heads=heads, seed=27, wider=wider).fill_contexts()
        b.to_device()
        q, out, lse = b.queries(), torch.empty((b.rows, heads, 128), dtype=torch.bfloat16, device=DEV), torch.empty((b.rows, heads), device=DEV)
        ws = torch.empty(max(16, B.emm_attn_fp8_workspace_size(b.batch)), dtype=torch.uint8, device=DEV)

        def step():
            b.attend(q, out=out, lse=lse, workspace=ws)
        step()
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for i in range(4):
            b.prefix[:] = [[0, 17, 2999, 512], [1, 511, 64, 3000], [700, 31, 32, 33], [1500, 1500, 0, 0]][i]
            b.new[:] = new_of(rng)
            b.cu[:] = np.concatenate([[0], np.cumsum(b.new)])
            b.table[:] = b.table[rng.permutation(4)]
            for n, x in (("prefix", b.prefix), ("new", b.new), ("cu", b.cu), ("table", b.table)):
                b.dev[n].copy_(torch.from_numpy(x))
            b.T = int(b.cu[-1])
            out.fill_(7), lse.fill_(7), ws.fill_(0xA5)
            graph.replay()
            torch.cuda.synchronize()
            assert (out[b.T:] == 7).all() and (lse[b.T:] == 7).all()
            b.compare(q, out, lse, sorted(set(rng.integers(0, b.T, 12).tolist())))
            replayed = out.clone()
            out.fill_(7)
            step()
            torch.cuda.synchronize()
            assert torch.equal(out, replayed), i


# ---- together, as they would be used --------------------------------------------------------------------------------

def test_serving_loop_over_the_prefix_cache():
    """Two requests that share an image's pages, a prompt each and some decode steps: prefix cache -> rotation and quantising
    write -> attention, against dense attention in 64 bits over the rows that the cache stands for."""
    from paper_2507_10069_amd import prefix_cache as PC
    H, K, D, PS, MAXP, NP = 28, 4, 128, 16, 40, 64
    rng = np.random.default_rng(21)
    inv, factor = B.emm_rope_inv_freq_host(D, 1e6, "yarn", 2.0, 4096)
    weights = {n: rng.standard_normal((199, h, D)).astype(np.float32) for n, h in (("q", H), ("k", K), ("v", K))}
    pools = [torch.zeros((NP, K, PS, D), dtype=torch.uint8, device=DEV) for _ in range(2)] + [torch.zeros((NP, K, PS), dtype=torch.uint8, device=DEV) for _ in range(2)]
    fp8 = B.make_fp8_cache(*pools)
    cache = PC.emm_prefix_cache_create(NP, PS)
    image = PC.emm_mm_token_ids(PC.emm_mm_content_hash(b"an image"), 200).tolist()
    live, dense = [], {}

    def dense_rows(rid, tokens, first, name):
        return torch.from_numpy(weights[name][np.asarray(tokens[first:]) % 199]).to(torch.bfloat16)

    def run(reqs):
        new = np.array([len(t) - p for _, t, _, p in reqs], np.int32)
        cu, prefix = np.concatenate([[0], np.cumsum(new)]).astype(np.int32), np.array([p for *_, p in reqs], np.int32)
        table = np.stack([row for _, _, row, _ in reqs]).astype(np.int32)
        dev = [_dev(x) for x in (table, prefix, new, cu)]
        batch = B.make_batch(num_reqs=len(reqs), num_q_heads=H, num_kv_heads=K, head_dim=D, page_size=PS, num_pages=NP, max_pages_per_req=MAXP,
                             total_new_tokens=int(cu[-1]), max_new_len=int(new.max()), dtype="bf16", softmax_scale=D ** -0.5, page_table=dev[0],
                             prefix_lens=dev[1], new_lens=dev[2], cu_new_lens=dev[3])
        rows = torch.cat([torch.cat([dense_rows(rid, t, p, n) for rid, t, _, p in reqs]) for n in ("q", "k", "v")], dim=1).to(DEV)
        rope = B.make_rope(_dev(inv), rotary_dim=D, factor=factor)
        q, out = (torch.empty((int(cu[-1]), H, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        B.emm_rope_kv_scatter_fp8(batch, rope, rows[:, :H], rows[:, H:H + K], rows[:, H + K:], q, fp8, token_stride=(H + 2 * K) * D)
        n = B.emm_attn_fp8_workspace_size(batch)
        B.emm_prefill_attn_fp8(batch, q, fp8, out, None, torch.empty(n, dtype=torch.uint8, device=DEV) if n else None)
        torch.cuda.synchronize()
        for i, (rid, t, _, p) in enumerate(reqs):
            # the whole sequence, from its tokens alone
            at = np.repeat(np.arange(len(t))[:, None], D // 2, 1)
            kr = torch.from_numpy(F.rotate(_f64(dense_rows(rid, t, 0, "k")), at, inv, D, "half", factor)).to(torch.bfloat16)
            k, v = F.values_of(*F.quantise(_f64(kr))), F.values_of(*F.quantise(_f64(dense_rows(rid, t, 0, "v"))))
            qr = F.rotate(_f64(dense_rows(rid, t, p, "q")), at[p:], inv, D, "half", factor)
            for h in range(H):
                s = qr[:, h] @ k[:, h // 7].T * D ** -0.5
                s[np.arange(len(t))[None] > np.arange(p, len(t))[:, None]] = -np.inf
                w = np.exp(s - s.max(1, keepdims=True))
                w /= w.sum(1, keepdims=True)
                want, size = w @ v[:, h // 7], w @ np.abs(v[:, h // 7])
                # q and K are rounded to bf16 after the rotation (2^-8 each): scores of |q| |k| scale / sqrt(128) rms, at most 2^-7 of the
                # largest |q| |k| scale off in all and 2^-7 / sqrt(128) * 6 beyond doubt; one code of K may fall the other way beside a border (2^-3 of it)
                e = 6 * (2.0 ** -7 + 2.0 ** -3 / 16) / np.sqrt(D) * np.linalg.norm(qr[:, h], axis=1).max() * np.linalg.norm(k[:, h // 7], axis=1).max() * D ** -0.5
                assert (np.abs(_f64(out)[cu[i]:cu[i + 1], h] - want) <= (2.0 ** -7 + 2 * e) * size + 2.0 ** -8 * np.abs(want)).all(), (rid, h)
    for text in (list(range(1000, 1030)), list(range(2000, 2075))):
        tokens = list(range(1, 50)) + image + text
        row, prefix_len, rid = PC.emm_prefix_cache_begin(cache, tokens, MAXP)
        live.append([rid, tokens, row, prefix_len])
        run([live[-1]])
        PC.emm_prefix_cache_commit(cache, rid, len(tokens))
    assert live[1][3] >= 240                                 # the second found the image's pages
    for step in range(4):
        for req in live:
            req[3] = len(req[1])
            req[1].append(3000 + step)
            req[2] = PC.emm_prefix_cache_append(cache, req[0], [3000 + step], MAXP)
        run(live)
    PC.emm_prefix_cache_destroy(cache)

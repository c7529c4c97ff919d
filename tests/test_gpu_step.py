"""Page steps, and norms with rotation and cache write, on the GPU against oracle/step_model.py.

Page steps are whole numbers: equal.  Tolerances of rows: the result is rounded, half a step (2^-8 of the value in bf16, 2^-24 in fp32).
Before that, in 32 bits: the mean of squares is d / 16 + 5 roundings of sums of positive terms and d exact-to-2^-24 squares, at most 2^-20 of
itself, half of that in the root, whose instruction is 2^-23 off; two products, 2^-23; so 2^-19 of the value generously.  The rotation: cosine and
sine are at most 5e-7 off, products and their sum 3 * 2^-24: 1e-6 (|a| + |b|) of a pair."""
import numpy as np
import pytest
import torch

from oracle import step_model as M
from paper_2507_10069_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _f64(t):
    return t.detach().double().cpu().numpy()


def _ints(a, dtype=torch.int32):
    return torch.tensor(np.ascontiguousarray(a), dtype=dtype, device=DEV)


# ---- page steps -----------------------------------------------------------------------------------------------------

NAMES = ("page_table", "free_pages", "prefix_lens", "new_lens", "cu_new_lens", "lens_out", "held_out", "free_count_out", "slots", "positions", "refused")


class Step:
    """Tables of requests with `lens` tokens, entries behind the window's start given back up to `late` entries ago."""

    def __init__(self, lens, add, *, page=16, window=0, sinks=0, free=None, width=None, max_tokens=None, late=2, held=None, in_place=False, seed=0):
        rng = np.random.default_rng(seed)
        self.page, self.window, self.sinks, self.in_place = page, window, sinks, in_place
        self.lens, self.add = list(lens), list(add)
        n = len(lens)
        entries = [-(-c // page) for c in lens]
        need = sum(-(-(c + max(m, 0)) // page) - e for c, m, e in zip(lens, add, entries))
        self.count = need + 3 if free is None else free
        self.width = width or max([1] + [-(-(c + max(m, 0)) // page) for c, m in zip(lens, add)])
        self.num_pages = max(1, sum(entries) + self.count)
        order = rng.permutation(self.num_pages)
        self.table = np.full((n, self.width), -1, np.int64)
        at = 0
        for r, e in enumerate(entries):
            self.table[r, :e] = order[at:at + e]
            at += e
        self.free = np.full(self.num_pages, -5)
        self.free[:self.count] = order[at:at + self.count]
        if held is None:
            held = []
            for c in lens:
                lo = -(-sinks // page)
                hi = max(lo, max(0, c - window + 1) // page) if window else lo
                held.append(max(0, hi - int(rng.integers(late + 1))))
        self.held = list(held)
        self.max_tokens = sum(max(m, 0) for m in add) if max_tokens is None else max_tokens
        i = {"page_table": self.table, "free_pages": self.free, "lens": self.lens, "add_lens": self.add, "held_from": self.held, "free_count": [self.count]}
        self.dev = {k: _ints(v) for k, v in i.items()}
        for name, size in (("prefix_lens", n), ("new_lens", n), ("cu_new_lens", n + 1), ("lens_out", n), ("held_out", n), ("free_count_out", 1),
                           ("positions", self.max_tokens), ("refused", 1)):
            self.dev[name] = torch.full((size,), -9, dtype=torch.int32, device=DEV)
        self.dev["slots"] = torch.full((self.max_tokens,), -9, dtype=torch.int64, device=DEV)
        if in_place:
            for out, src in (("lens_out", "lens"), ("held_out", "held_from"), ("free_count_out", "free_count")):
                self.dev[out] = self.dev[src]
        self.step = B.make_page_step(num_reqs=n, page_size=page, num_pages=self.num_pages, max_pages_per_req=self.width, max_tokens=self.max_tokens,
                                     window=window, sinks=sinks, **self.dev)

    def want(self):
        return M.page_step(self.table, self.free, self.count, self.lens, self.add, self.held, self.page, self.window, self.sinks, self.max_tokens)

    def check(self, want):
        for name in NAMES:
            got = self.dev[name].cpu().numpy()
            assert np.array_equal(got, np.asarray(want[name], got.dtype).reshape(got.shape)), (name, np.argwhere(got != np.asarray(want[name]).reshape(got.shape))[:4])

    def run_and_check(self):
        want = self.want()
        B.emm_page_step(self.step)
        self.check(want)
        if not self.in_place:                                                # the step can be done again
            B.emm_page_step(self.step)
            self.check(want)
        return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (40, 4), (100, 33), (500, 0), (2 ** 31 - 1, 5), (7, 2 ** 31 - 1)])
def test_steps(window, sinks, page, in_place):
    Step([0, 1, 15, 16, 17, 500, 31, 255, 256, 1000], [1, 15, 1, 1, 0, 70, -3, 1, 1, 300], page=page, window=window, sinks=sinks, in_place=in_place,
         seed=page).run_and_check()


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 256, 257, 1024, 1025, 4096])
@pytest.mark.parametrize("in_place", [False, True])
def test_decode_steps_of_many_requests(n, in_place):
    rng = np.random.default_rng(n)
    Step(rng.integers(0, 300, n).tolist(), rng.integers(0, 2, n).tolist(), window=100, sinks=4, in_place=in_place, seed=n).run_and_check()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,most", [(3, 3000), (64, 700), (300, 40), (1100, 12)])
def test_prompts_take_pages_from_many_workgroups(n, most, in_place):
    rng = np.random.default_rng(n + 1)
    step = Step(rng.integers(0, 2000, n).tolist(), rng.integers(0, most, n).tolist(), window=300, sinks=20, in_place=in_place, late=9, seed=n)
    assert step.max_tokens > 4096
    step.run_and_check()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("free", [0, 1, 5, 6, 7, 40])
def test_requests_that_find_too_few_pages_are_refused(free, in_place):
    want = Step([16, 5, 32, 90, 0, 16, 7], [1, 3, 80, 1, 16, 0, 20], free=free, in_place=in_place, max_tokens=130).run_and_check()
    assert (want["refused"][0] > 0) == (free < 10)
    # pages that are given back in the same step serve as well
    Step([16, 500, 32, 300], [20, 1, 80, 1], free=free, window=60, sinks=4, late=8, in_place=in_place, max_tokens=120).run_and_check()


def test_requests_that_do_not_fit_their_row_are_refused():
    want = Step([60, 10, 64, 64], [5, 3, 1, 0], width=4, free=9, max_tokens=16).run_and_check()
    assert want["refused"] == [2] and want["new_lens"] == [0, 3, 0, 0]


def test_shared_leading_pages_are_never_given_back():
    want = Step([400, 400], [1, 1], window=50, sinks=4, held=[20, 3]).run_and_check()
    assert want["held_out"] == [21, 21]


def test_outputs_that_are_not_wanted_and_batches_without_requests():
    step = Step([5, 20], [3, 40])
    s = B.make_page_step(num_reqs=2, page_size=16, num_pages=step.num_pages, max_pages_per_req=step.width, max_tokens=43,
                         **{k: v for k, v in step.dev.items() if k not in ("slots", "positions", "refused")})
    want = step.want()
    B.emm_page_step(s)
    for k in ("slots", "positions", "refused"):
        assert (step.dev[k] == -9).all()
        want[k] = step.dev[k].cpu().numpy()
    step.check(want)
    empty = Step([], [], free=4, max_tokens=7)
    B.emm_page_step(empty.step)
    for name, value in (("cu_new_lens", 0), ("free_count_out", 4), ("slots", -1), ("positions", 0), ("refused", 0)):
        assert (empty.dev[name] == value).all(), name


def test_inconsistent_arrays_stay_inside_the_buffers():
    """Lengths, counts and first entries that mean nothing: guard bands around every output stay as they were."""
    rng = np.random.default_rng(4)
    big = 2 ** 31 - 1
    for lens, add, held, count in (([big, -7, 50, 200], [big, 5, -big, 9], [0, 0, 0, 0], 3), ([40, 200, 60, 1], [1, 1, 1, 1], [-big, big, 5, 0], big),
                                   ([100, 200, 60, 1], [9, 1, 1, 1], [0, 0, 0, 0], -4)):
        step = Step([10, 20, 30, 40], [1, 1, 1, 1], window=20, width=13, max_tokens=6)
        step.dev["lens"].copy_(_ints(lens))
        step.dev["add_lens"].copy_(_ints(add))
        step.dev["held_from"].copy_(_ints(held))
        step.dev["free_count"].fill_(count)
        outs = [n for n in NAMES]
        guarded = {}
        for n in outs:
            t = step.dev[n]
            g = torch.full((t.numel() + 64,), -77, dtype=t.dtype, device=DEV)
            g[32:-32] = t.flatten()
            guarded[n] = g
        arrays = {n: guarded[n][32:-32] if n in guarded else t for n, t in step.dev.items()}
        B.emm_page_step(B.make_page_step(num_reqs=4, page_size=16, num_pages=step.num_pages, max_pages_per_req=13, max_tokens=6, window=20, sinks=0, **arrays))
        for n, g in guarded.items():
            assert (g[:32] == -77).all() and (g[-32:] == -77).all(), n
    del rng


# ---- norms, rotation, write -----------------------------------------------------------------------------------------

class Rows:
    def __init__(self, prefix, new, *, heads=28, kv_heads=4, d=128, page=16, dtype="bf16", seed=0, extra_rows=0, fused=False, magnitude=1.0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.heads, self.kv_heads, self.d, self.page, self.dtype, self.dt = heads, kv_heads, d, page, dtype, DTYPES[dtype]
        self.prefix, self.new = np.array(prefix, np.int32), np.array(new, np.int32)
        self.cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.T, self.rows = int(self.cu[-1]), int(self.cu[-1]) + extra_rows
        entries = -(-(self.prefix + self.new) // page)
        self.num_pages = int(entries.sum()) + 4
        order = rng.permutation(self.num_pages)
        self.table = np.full((len(prefix), max(1, int(entries.max(initial=1)))), -1, np.int32)
        at = 0
        for r, n in enumerate(entries):
            self.table[r, :n] = order[at:at + n]
            at += n
        x = (torch.randn((self.rows, heads + 2 * kv_heads, d), generator=gen) * magnitude).to(self.dt)
        self.x = x.to(DEV)
        self.stride = (heads + 2 * kv_heads) * d if fused else 0
        parts = self.x[:, :heads], self.x[:, heads:heads + kv_heads], self.x[:, heads + kv_heads:]
        self.q, self.k, self.v = parts if fused else [p.contiguous() for p in parts]
        self.weights = [(1 + 0.3 * torch.randn(d, generator=gen)).to(DEV) for _ in range(2)]
        self.dev = {n: _ints(getattr(self, n)) for n in ("table", "prefix", "new", "cu")}
        self.batch = B.make_batch(num_reqs=len(prefix), num_q_heads=heads, num_kv_heads=kv_heads, head_dim=d, page_size=page, num_pages=self.num_pages,
                                  max_pages_per_req=self.table.shape[1], total_new_tokens=self.rows, max_new_len=max(1, int(self.new.max(initial=0))), dtype=dtype,
                                  softmax_scale=0.1, page_table=self.dev["table"], prefix_lens=self.dev["prefix"], new_lens=self.dev["new"], cu_new_lens=self.dev["cu"])
        self.pool_shape = (self.num_pages, kv_heads, page, d)

    def places(self):
        """Slot of every packed token, -1: none."""
        out = np.full(self.rows, -1, np.int64)
        for r, (c, m) in enumerate(zip(self.prefix, self.new)):
            at = np.arange(c, c + m)
            out[self.cu[r]:self.cu[r] + m] = self.table[r, at // self.page].astype(np.int64) * self.page + at % self.page
        return out

    def positions(self):
        out = np.zeros(self.rows, np.int64)
        for r, (c, m) in enumerate(zip(self.prefix, self.new)):
            out[self.cu[r]:self.cu[r] + m] = np.arange(c, c + m)
        return out

    def descriptors(self, norm, rotary, layout, axes, eps, inverse=False, seed=1):
        self.eps, self.normed, self.rotary, self.interleaved = eps, norm, rotary, layout == "interleaved"
        self.norm = B.make_qk_norm(*self.weights, eps=eps) if norm else None
        self.angle, self.rope = None, None
        if rotary:
            inv = 1e6 ** (-2.0 * np.arange(rotary // 2) / rotary)
            given, sections = None, None
            at = np.repeat(self.positions()[:, None], rotary // 2, axis=1)
            if axes:
                sections = [rotary // 2] if axes == 1 else [rotary // 8, rotary // 8, rotary // 4]
                pos = np.random.default_rng(seed).integers(0, 100000, (axes, self.rows))
                at = np.concatenate([np.repeat(pos[a][:, None], n, axis=1) for a, n in enumerate(sections)], axis=1)
                given = _ints(pos)
            self.angle = at * inv * (-1 if inverse else 1)
            self.rope = B.make_rope(torch.from_numpy(inv).to(DEV), rotary_dim=rotary, layout=layout, positions=given, sections=sections, inverse=inverse)

    def exact(self, t, which):
        return M.norm_rope(_f64(t), _f64(self.weights[which]) if self.normed else None, self.eps, self.angle, self.rotary, self.interleaved)

    def tolerance(self, want):
        # of a pair, whose rotated values have its length
        pair = np.abs(want)
        if self.rotary:
            a = (slice(0, self.rotary, 2), slice(1, self.rotary, 2)) if self.interleaved else (slice(0, self.rotary // 2), slice(self.rotary // 2, self.rotary))
            length = np.hypot(want[..., a[0]], want[..., a[1]])
            pair[..., a[0]] = pair[..., a[1]] = 1.5 * length                 # |a| + |b| before the rotation, at most sqrt(2) times as long
        return HALF_STEP[self.dtype] * (1 + 2.0 ** -10) * np.abs(want) + (2.0 ** -19 + 1e-6) * pair + 1e-38

    def near(self, got, want):
        assert np.array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want)
        tol = self.tolerance(want)
        worst = np.where(ok, np.abs(np.where(ok, got, 0) - np.where(ok, want, 0)) / np.where(ok, tol, 1), 0)
        assert worst.max(initial=0) <= 1, worst.max()


SHAPES = [dict(heads=28, kv_heads=4, d=128, dtype="bf16"), dict(heads=8, kv_heads=8, d=64, dtype="bf16"), dict(heads=4, kv_heads=1, d=64, dtype="f32"),
          dict(heads=9, kv_heads=3, d=128, dtype="f32"), dict(heads=33, kv_heads=1, d=128, dtype="bf16")]
FORMS = [(True, 0, "half", 0), (True, 128, "half", 0), (True, 32, "interleaved", 3), (True, 64, "half", 1), (False, 64, "interleaved", 0), (False, 128, "half", 3)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("norm,rotary,layout,axes", FORMS)
@pytest.mark.parametrize("fused", [False, True])
def test_norm_rope(shape, norm, rotary, layout, axes, fused):
    rows = Rows([0, 5, 1000, 70000], [1, 40, 0, 7], extra_rows=2, fused=fused, seed=rotary + axes, **shape)
    rotary = min(rotary, rows.d)
    rows.descriptors(norm, rotary, layout, axes, 1e-6)
    q_out = torch.full((rows.rows, rows.heads, rows.d), 7.0, dtype=rows.dt, device=DEV)
    k_out = torch.full((rows.rows, rows.kv_heads, rows.d), 7.0, dtype=rows.dt, device=DEV)
    B.emm_norm_rope(rows.batch, rows.norm, rows.rope, rows.q, rows.k, q_out, k_out, token_stride=rows.stride)
    done = rows.T if rotary and not axes else rows.rows                      # rows of no request: done unless their positions come from the batch
    for got, x, which in ((q_out, rows.q, 0), (k_out, rows.k, 1)):
        rows.near(_f64(got)[:done], rows.exact(x, which)[:done])
        assert (got[done:] == 7).all()
    # each alone, and in place, has the same bits
    only_k = torch.empty_like(k_out).fill_(7.0)
    B.emm_norm_rope(rows.batch, rows.norm, rows.rope, None, rows.k, None, only_k, token_stride=rows.stride)
    assert torch.equal(only_k, k_out)
    if not fused:
        q = rows.q.clone()
        B.emm_norm_rope(rows.batch, rows.norm, rows.rope, q, None, q, None)
        assert torch.equal(q[:done], q_out[:done])


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("norm,rotary,layout,axes", FORMS)
@pytest.mark.parametrize("given", [False, True])
def test_norm_rope_and_write(shape, norm, rotary, layout, axes, given):
    rows = Rows([0, 5, 100, 700], [1, 40, 0, 7], extra_rows=2, fused=given, page=32, seed=rotary + axes, **shape)
    rotary = min(rotary, rows.d)
    rows.descriptors(norm, rotary, layout, axes, 1e-5)
    gen = torch.Generator().manual_seed(3)
    pools = [torch.randn(rows.pool_shape, generator=gen).to(rows.dt).to(DEV) for _ in range(2)]
    before = [p.clone() for p in pools]
    q_out = torch.full((rows.rows, rows.heads, rows.d), 7.0, dtype=rows.dt, device=DEV)
    places = rows.places()
    if given:
        places[3] = -1                                                       # a token that is not written
        places[rows.T:] = [rows.num_pages * rows.page, 2 ** 62]              # and some that name no slot
    rows.v[2, 0, :4] = torch.tensor([float("nan"), float("inf"), -0.0, 1e-40], device=DEV).to(rows.dt)
    slots = _ints(places, torch.int64) if given else None
    B.emm_norm_rope_kv_scatter(rows.batch, rows.norm, rows.rope, rows.q, rows.k, rows.v, q_out, *pools, token_stride=rows.stride, slots=slots)
    q_alone, k_alone = torch.full_like(q_out, 7.0), torch.full((rows.rows, rows.kv_heads, rows.d), 7.0, dtype=rows.dt, device=DEV)
    B.emm_norm_rope(rows.batch, rows.norm, rows.rope, rows.q, rows.k, q_alone, k_alone, token_stride=rows.stride)
    assert torch.equal(q_out, q_alone)
    written = np.flatnonzero((places >= 0) & (places < rows.num_pages * rows.page))
    assert len(written) == rows.T - int(given)
    page, place = places[written] // rows.page, places[written] % rows.page
    for pool, old, x in ((pools[0], before[0], k_alone), (pools[1], before[1], rows.v)):
        old[page, :, place] = x[written]
        assert torch.equal(pool.view(torch.uint8), old.view(torch.uint8))


@pytest.mark.parametrize("norm,rotary,layout,axes", FORMS)
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_rope_and_quantising_write(norm, rotary, layout, axes, given, dtype):
    rows = Rows([0, 5, 100], [1, 40, 7], seed=rotary, dtype=dtype, extra_rows=1)
    rows.descriptors(norm, rotary, layout, axes, 1e-6)

    def pools():
        return [torch.full(s, 9, dtype=torch.uint8, device=DEV) for s in (rows.pool_shape, rows.pool_shape, rows.pool_shape[:3], rows.pool_shape[:3])]
    got, want = pools(), pools()
    q_out, q_alone = torch.full_like(rows.q, 7.0), torch.full_like(rows.q, 7.0)
    k_alone = torch.full_like(rows.k, 7.0)
    slots = _ints(rows.places(), torch.int64) if given else None
    B.emm_norm_rope_kv_scatter_fp8(rows.batch, rows.norm, rows.rope, rows.q, rows.k, rows.v, q_out, B.make_fp8_cache(*got), slots=slots)
    B.emm_norm_rope(rows.batch, rows.norm, rows.rope, rows.q, rows.k, q_alone, k_alone)
    B.emm_kv_scatter_fp8(rows.batch, k_alone, rows.v, B.make_fp8_cache(*want))
    assert torch.equal(q_out, q_alone)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("magnitude,eps", [(1e-25, 1e-6), (1e-12, 1e-20), (1e18, 1e-6), (1e30, 1e-6), (3e37, 1e-30), (1.0, 1e30), (0.0, 1.2e-38)])
def test_rows_of_any_magnitude(magnitude, eps, dtype):
    rows = Rows([3], [9], dtype=dtype, magnitude=magnitude, seed=5)
    rows.descriptors(True, 0, "half", 0, eps)
    q_out, k_out = torch.empty_like(rows.q), torch.empty_like(rows.k)
    B.emm_norm_rope(rows.batch, rows.norm, None, rows.q, rows.k, q_out, k_out)
    rows.near(_f64(q_out), rows.exact(rows.q, 0))
    rows.near(_f64(k_out), rows.exact(rows.k, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("magnitude,eps", [(1e18, 3.4e38), (3e18, 3.38e38), (1.0, 3.4e38), (1e30, 3.4e38)])
def test_eps_near_the_end_of_the_range(magnitude, eps, d, dtype):
    """The mean of squares and eps are each below 2^128, their sum is not."""
    rows = Rows([3], [9], dtype=dtype, d=d, magnitude=magnitude, seed=6)
    rows.descriptors(True, 0, "half", 0, eps)
    q_out, k_out = torch.empty_like(rows.q), torch.empty_like(rows.k)
    B.emm_norm_rope(rows.batch, rows.norm, None, rows.q, rows.k, q_out, k_out)
    rows.near(_f64(q_out), rows.exact(rows.q, 0))
    rows.near(_f64(k_out), rows.exact(rows.k, 1))


def test_a_row_with_nan_leaves_the_others():
    rows = Rows([3], [9])
    rows.descriptors(True, 128, "half", 0, 1e-6)
    out, clean = torch.empty_like(rows.q), torch.empty_like(rows.q)
    B.emm_norm_rope(rows.batch, rows.norm, rows.rope, rows.q, None, clean, None)
    rows.q[4, 7, 3], rows.q[5, 1, 0] = float("nan"), float("inf")
    B.emm_norm_rope(rows.batch, rows.norm, rows.rope, rows.q, None, out, None)
    same = torch.ones(9, 28, dtype=torch.bool, device=DEV)
    same[4, 7] = same[5, 1] = False
    assert torch.equal(out[same], clean[same]) and out[4, 7].isnan().all()


def test_many_tokens_and_no_requests():
    rows = Rows([7, 0], [3000, 1300], heads=32, kv_heads=8, seed=2, fused=True)
    rows.descriptors(True, 128, "half", 3, 1e-6)
    q_out, k_out = torch.empty((rows.rows, 32, 128), dtype=rows.dt, device=DEV), torch.empty((rows.rows, 8, 128), dtype=rows.dt, device=DEV)
    B.emm_norm_rope(rows.batch, rows.norm, rows.rope, rows.q, rows.k, q_out, k_out, token_stride=rows.stride)
    rows.near(_f64(q_out), rows.exact(rows.q, 0))
    rows.near(_f64(k_out), rows.exact(rows.k, 1))
    # without requests q alone is done, and k and v go where slots say
    bare = B.make_batch(num_reqs=0, num_q_heads=32, num_kv_heads=8, head_dim=128, page_size=16, num_pages=rows.num_pages, max_pages_per_req=0,
                        total_new_tokens=rows.rows, max_new_len=1, dtype="bf16", softmax_scale=0.1)
    again = torch.empty_like(q_out)
    pools = [torch.zeros(rows.pool_shape, dtype=rows.dt, device=DEV) for _ in range(2)]
    B.emm_norm_rope_kv_scatter(bare, rows.norm, rows.rope, rows.q, rows.k, rows.v, again, *pools, token_stride=rows.stride)
    assert torch.equal(again, q_out) and not pools[0].any()
    B.emm_norm_rope_kv_scatter(bare, rows.norm, rows.rope, rows.q, rows.k, rows.v, again, *pools, token_stride=rows.stride, slots=_ints(rows.places(), torch.int64))
    places = rows.places()
    assert torch.equal(pools[0][places // 16, :, places % 16], k_out) and torch.equal(pools[1][places // 16, :, places % 16], rows.v)

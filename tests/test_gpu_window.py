"""Attention with a window and sinks on the GPU against oracle/step_model.py in 64 bits.

Tolerances.  bf16: weights are rounded to bf16, at most 2^-8 of themselves, for the numerator: 2^-8 (sum of p |v|); the result is rounded:
2^-8 |out|.  A score is off by at most e = (d + 2) 2^-24 scale |q| |k| (sums of exact products in 32 bits), and
its exponential by 2^-20 (its argument, below 2^6 in powers of two, is rounded in 32 bits: 2^-19 ln 2; 1 unit in the last place): a
weight changes by e + 2^-19, in numerator and denominator.  Sums over n keys in 32 bits: n 2^-24 of sum of p |v|.  lse: e + 2^-19,
n 2^-24, 2^-22 of itself.  fp32: the same without the 2^-8, and 2^-22 |out| for the division and the result."""
import numpy as np
import pytest
import torch

from oracle import step_model as M
from paper_2507_10069_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HUGE = 2 ** 31 - 1


def _f64(t):
    return t.detach().double().cpu().numpy()


class Case:
    """A batch whose tables hold only pages that some new token sees; other entries name a page of NaN, of infinities, or none."""

    def __init__(self, prefix, new, window, sinks, *, heads=28, kv_heads=4, d=128, page=16, dtype="bf16", seed=0, extra_rows=0, wider=0, magnitude=1.0):
        rng = np.random.default_rng(seed)
        self.rng, self.window, self.sinks, self.page, self.heads, self.kv_heads, self.d, self.dtype = rng, window, sinks, page, heads, kv_heads, d, dtype
        self.prefix, self.new = np.array(prefix, np.int32), np.array(new, np.int32)
        self.cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.rows = int(self.cu[-1]) + extra_rows
        entries = [-(-(int(c) + int(m)) // page) for c, m in zip(prefix, new)]
        first = [max(0, int(c) - window + 1) // page for c in prefix]
        live = [[e for e in range(n) if m > 0 and (e >= f or e * page < sinks)] for n, f, m in zip(entries, first, new)]
        self.num_pages = sum(map(len, live)) + 3
        order = rng.permutation(self.num_pages)
        odd = order[-3:]                                                     # pages of no request: NaN, infinities, and one not named
        self.table = np.full((len(prefix), max(1, max(entries, default=1)) + wider), -1, np.int32)
        for r, n in enumerate(entries):
            self.table[r, :n] = rng.choice([odd[0], odd[1], -1, 2 ** 30], n)
        at = 0
        for r, es in enumerate(live):
            self.table[r, es] = order[at:at + len(es)]
            at += len(es)
        shape = (self.num_pages, kv_heads, page, d)
        dt = DTYPES[dtype]
        gen = torch.Generator().manual_seed(seed)
        self.k = (torch.randn(shape, generator=gen) * magnitude).to(dt)
        self.v = torch.randn(shape, generator=gen).to(dt)
        # slots that hold no token, and those that nobody sees, hold what breaks a sum
        held = torch.zeros(shape[0], page, dtype=torch.bool)
        for r, (c, m) in enumerate(zip(prefix, new)):
            if m > 0:
                low = max(0, int(c) - window + 1)
                slots = np.concatenate([np.arange(min(sinks, low)), np.arange(low, int(c) + int(m))]).astype(np.int64)
                held[self.table[r, slots // page], slots % page] = True
        poison = torch.tensor([float("nan"), float("inf"), -float("inf")])[torch.randint(0, 3, shape, generator=gen)].to(dt)
        hidden = ~held[:, None, :, None].expand(shape)
        self.k, self.v = torch.where(hidden, poison, self.k), torch.where(hidden, poison, self.v)
        self.q = torch.randn((self.rows, heads, d), generator=gen).to(dt)
        self.scale = 1.0 / np.sqrt(d)

    def slot(self, r, s):
        return int(self.table[r, s // self.page]), s % self.page

    def to_device(self):
        self.dev = {n: torch.from_numpy(np.ascontiguousarray(getattr(self, n))).to(DEV) for n in ("table", "prefix", "new", "cu")}
        self.dq, self.dk, self.dv = (t.to(DEV) for t in (self.q, self.k, self.v))
        self.batch = B.make_batch(num_reqs=len(self.prefix), num_q_heads=self.heads, num_kv_heads=self.kv_heads, head_dim=self.d, page_size=self.page,
                                  num_pages=self.num_pages, max_pages_per_req=self.table.shape[1], total_new_tokens=self.rows,
                                  max_new_len=max(1, int(self.new.max(initial=0))), dtype=self.dtype, softmax_scale=self.scale, page_table=self.dev["table"],
                                  prefix_lens=self.dev["prefix"], new_lens=self.dev["new"], cu_new_lens=self.dev["cu"])
        n = B.emm_attn_window_workspace_size(self.batch, self.window, self.sinks)
        # NaN in the workspace: what it held means nothing
        self.workspace = torch.full((max(n, 16) // 4,), float("nan"), device=DEV).view(torch.uint8) if n else None
        return self

    def run(self, decode=False, lse=True, stream=None):
        out = torch.full((self.rows, self.heads, self.d), 7.0, dtype=DTYPES[self.dtype], device=DEV)
        sums = torch.full((self.rows, self.heads), 7.0, device=DEV)
        call = B.emm_decode_attn_window if decode else B.emm_prefill_attn_window
        call(self.batch, self.window, self.sinks, self.dq, self.dk, self.dv, out, sums if lse else None, self.workspace, stream)
        return out, sums

    def check(self, out, lse):
        q, k, v = _f64(self.q), _f64(self.k), _f64(self.v)
        want, want_lse, size = M.window_attention(self.table, self.prefix, self.new, self.cu, q, k, v, self.page, self.window, self.sinks, self.scale, self.rows)
        got, got_lse = _f64(out), _f64(lse)
        T = int(self.cu[-1])
        assert (got[T:] == 7).all() and (got_lse[T:] == 7).all()             # rows of no request
        got, got_lse, want, want_lse, size, q = got[:T], got_lse[:T], want[:T], want_lse[:T], size[:T], q[:T]
        if T == 0:
            return
        with np.errstate(invalid="ignore"):
            longest = np.sqrt(np.nanmax(np.where(np.isfinite(k), k, 0).__pow__(2).sum(-1)))
        keys = min(int((self.prefix + self.new).max()), self.window + self.sinks)
        e = ((self.d + 2) * 2.0 ** -24 * self.scale * np.linalg.norm(q, axis=-1) * longest)      # [T][H]
        weight = (e + 2.0 ** -19 + keys * 2.0 ** -24)
        bf16 = self.dtype == "bf16"
        tol = 2.0 ** -8 * bf16 * size + weight[..., None] * (size + np.abs(want)) + (2.0 ** -8 if bf16 else 2.0 ** -22) * np.abs(want) + 1e-30
        finite = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want)), "infinities and NaN elsewhere"
        assert np.array_equal(np.sign(got[np.isinf(want)]), np.sign(want[np.isinf(want)]))
        worst = np.where(finite, np.abs(np.where(finite, got, 0) - np.where(finite, want, 0)) / tol, 0)
        assert worst.max() <= 1, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))
        tol = weight + 2.0 ** -22 * np.abs(want_lse)
        ok = np.isfinite(want_lse)
        assert (np.abs(got_lse - want_lse)[ok] <= tol[ok]).all(), (np.abs(got_lse - want_lse)[ok] / tol[ok]).max()

    def run_and_check(self, decode=False):
        self.to_device()
        out, lse = self.run(decode)
        self.check(out, lse)
        again, lse2 = self.run(decode)
        assert torch.equal(out.view(torch.uint8), again.view(torch.uint8)) and torch.equal(lse.view(torch.uint8), lse2.view(torch.uint8))
        return out, lse


EDGES = [(1, 0), (1, 1), (2, 3), (15, 0), (16, 4), (17, 16), (63, 17), (64, 0), (65, 100), (100, 4), (129, 1), (1000, 5), (HUGE, 0), (HUGE, HUGE), (5, HUGE)]
PREFIX = [0, 1, 15, 16, 17, 63, 200, 0, 500, 31, 2]
NEW = [1, 5, 0, 37, 1, 20, 3, 64, 2, 0, 1]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", EDGES)
def test_windows_and_sinks(window, sinks, dtype):
    Case(PREFIX, NEW, window, sinks, heads=8 if dtype == "f32" else 28, kv_heads=2 if dtype == "f32" else 4, d=64 if dtype == "f32" else 128,
         dtype=dtype, seed=window % 1000 + sinks % 7, extra_rows=3, wider=2).run_and_check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", EDGES)
def test_decode_steps(window, sinks, dtype):
    Case([0, 1, 15, 16, 17, 63, 64, 1000, 127, 300, 5], [1, 1, 1, 1, 0, 1, 1, 1, 1, 1, 1], window, sinks, heads=28 if dtype == "bf16" else 8,
         kv_heads=4 if dtype == "bf16" else 1, dtype=dtype, seed=window % 997, extra_rows=2).run_and_check(decode=True)


@pytest.mark.parametrize("heads,kv_heads", [(8, 8), (16, 1), (33, 1), (40, 1), (6, 2), (1, 1)])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_head_layouts_and_pages(heads, kv_heads, page):
    Case([300, 40, 0, 777], [1, 30, 129, 2], 100, 20, heads=heads, kv_heads=kv_heads, page=page, seed=page + heads).run_and_check()
    Case([300, 40, 0, 777], [1, 1, 1, 1], 100, 20, heads=heads, kv_heads=kv_heads, page=page, seed=page + heads).run_and_check(decode=True)


@pytest.mark.parametrize("window,sinks,page", [(1, 0, 16), (40, 4, 16), (128, 0, 64), (500, 130, 32), (1000, 16, 256), (HUGE, 0, 16)])
@pytest.mark.parametrize("heads,kv_heads", [(28, 4), (32, 8), (16, 16)])
def test_large_prompts(window, sinks, page, heads, kv_heads):
    """Row tiles of 128 rows whose waves share their keys; the last ones of an XCD are cut where they are few."""
    Case([700, 0, 33], [400, 900, 801], window, sinks, heads=heads, kv_heads=kv_heads, page=page, seed=heads + window % 13, extra_rows=5).run_and_check()


@pytest.mark.parametrize("new,window", [([1180, 1180, 1180], 300), ([2400, 5, 77], 200), ([40] * 70, 500), ([1200] * 2 + [0] * 200, 700)])
def test_cut_tails_and_many_requests(new, window):
    """65 to 96 row tiles on an XCD, of which the last are cut into many parts or few; requests beyond those that a wave sees at a time."""
    rng = np.random.default_rng(len(new))
    Case(rng.integers(0, 900, len(new)).tolist(), new, window, 7, seed=len(new)).run_and_check()


@pytest.mark.parametrize("prefix,new,window,heads,kv_heads", [([3000], [300], 2100, 28, 4), ([2500, 40, 9000], [290, 30, 77], 2048, 28, 4),
                                                              ([2600, 2600], [128, 128], HUGE, 32, 8), ([4000], [1100], 2500, 28, 4), ([2500] * 66, [20] * 66, 2400, 8, 2)])
def test_long_windows_cut_into_parts(prefix, new, window, heads, kv_heads):
    """Row tiles of 256 rows, the last of which are cut along their keys: none, all, or those behind full rounds."""
    case = Case(prefix, new, window, 20, heads=heads, kv_heads=kv_heads, seed=len(prefix)).to_device()
    assert case.workspace is not None
    case.run_and_check()


def test_one_context_is_cut_into_parts():
    case = Case([5000], [1], 4096, 64, seed=5).to_device()
    assert case.workspace is not None
    case.run_and_check(decode=True)
    case = Case([5000], [33], 2048, 4, seed=6).to_device()
    assert case.workspace is not None
    case.run_and_check()


@pytest.mark.parametrize("prefix,new,heads,kv_heads", [([90], [40], 28, 4), ([200, 33], [1, 1], 28, 4), ([900, 100], [1200, 300], 28, 4), ([10], [3], 8, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan_reach_the_rows_that_see_them_alone(prefix, new, heads, kv_heads, dtype):
    """In V at slots that only some rows see, and NaN in K at slots that leave some rows' windows."""
    case = Case(prefix, new, 50, 6, heads=heads, kv_heads=kv_heads, dtype=dtype, seed=9)
    rng = np.random.default_rng(1)
    for r, (c, m) in enumerate(zip(prefix, new)):
        if m == 1:
            continue
        for s in (c - 30, c - 1, c + m // 2, c + m - 1):
            page, place = case.slot(r, max(s, 0))
            h, ch = rng.integers(kv_heads), rng.integers(128, size=3)
            case.v[page, h, place, ch] = torch.tensor([float("nan"), float("inf"), -float("inf")]).to(case.v.dtype)
        page, place = case.slot(r, c + 1)
        case.k[page, 0, place, 5] = float("nan")
    case.to_device()
    out, lse = case.run()
    case.check(out, lse)
    assert not np.isfinite(_f64(out)).all() or max(new) == 1


def test_hundreds_of_requests_with_some_tokens():
    rng = np.random.default_rng(8)
    new = rng.integers(0, 60, 700).tolist()
    new[3] = 300
    Case(rng.integers(0, 200, 700).tolist(), new, 64, 3, heads=8, kv_heads=2, seed=8, extra_rows=9).run_and_check()


@pytest.mark.parametrize("idle", [14, 600, 5000])
def test_a_few_tokens_among_many_requests(idle):
    new = [0] * (idle // 2) + [9] + [0] * (idle - idle // 2) + [3]
    prefix = [40] * (idle // 2) + [3000] + [0] * (idle - idle // 2) + [700]
    case = Case(prefix, new, 2048, 4, kv_heads=1).to_device()
    case.check(*case.run())


def test_scores_that_differ_by_far():
    """Scores of hundreds: the reference has to be raised on the way, and what came before vanishes."""
    for seed in range(3):
        case = Case([3000, 100], [40, 700], 1500, 4, seed=seed, magnitude=40.0)
        case.run_and_check()
        Case([3000, 100], [1, 1], 1500, 4, seed=seed, magnitude=40.0).run_and_check(decode=True)


def test_lse_is_optional():
    case = Case([300, 5], [20, 1], 64, 4).to_device()
    a, _ = case.run()
    b, untouched = case.run(lse=False)
    assert torch.equal(a, b) and (untouched == 7).all()


def test_a_full_window_is_the_full_attention():
    case = Case([1000, 17], [60, 128], 4096, 0, seed=3).to_device()
    out, _ = case.run()
    full = torch.empty_like(out)
    n = B.emm_prefill_attn_workspace_size(case.batch)
    B.emm_prefill_attn(case.batch, case.dq, case.dk, case.dv, full, None, torch.empty(max(n, 16), dtype=torch.uint8, device=DEV))
    assert (out.float() - full.float()).abs().max() <= 2.0 ** -6


def test_batches_without_tokens():
    case = Case([5, 6], [0, 0], 4, 0, extra_rows=4).to_device()
    out, lse = case.run()
    assert (out == 7).all() and (lse == 7).all()


# prefix, new, window, heads, KV heads, dtype, are keys cut over workgroups, whose records a second kernel adds up?
CUT_AND_UNCUT = [([5000], [1], 4096, 28, 4, "bf16", True),                       # decode shape
                 ([500] * 10, [1] * 10, 400, 28, 28, "bf16", False),
                 ([200, 60], [1, 1], 50, 28, 4, "bf16", False),
                 ([5000], [33], 2048, 28, 4, "bf16", True),                      # keys shape
                 ([300], [9], 60, 28, 4, "bf16", False),
                 ([2000], [250], 1024, 28, 4, "bf16", True),                     # rows shape, four waves
                 ([1000] * 5, [200] * 5, 900, 28, 4, "bf16", False),             # (in halves)
                 ([1000] * 8, [200] * 8, 900, 28, 4, "bf16", False),             # (whole)
                 ([3000], [300], 2100, 28, 4, "bf16", True),                     # eight waves
                 ([900, 70], [1, 1], 60, 8, 2, "f32", False),
                 ([2000], [33], 1000, 8, 2, "f32", False)]


def _of_odd_values(prefix, new, window, heads, kv_heads, dtype, cut, far):
    """far: the scores of the older 5/8 of a window are 522 powers of two below the others, so that its parts have a weight of 0."""
    case = Case(prefix, new, window, 20, heads=heads, kv_heads=kv_heads, dtype=dtype, seed=len(prefix) + window)
    case.q[:, :, 0] = 8
    places = []
    for c, m, r in zip(prefix, new, range(len(prefix))):
        for s in range(c - window + 1, c + m):
            page, place = case.slot(r, s)
            case.k[page, :, place, 0] = -512 if far and s < c - 3 * window // 8 else 0
        # slots that all of the request's rows see, and some
        assert m == 1 or m < window // 4 + window // 8
        places.append((case.slot(r, c - window + 3 * window // 8), case.slot(r, c - window + 1 + m // 2)))
    return case, places


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("prefix,new,window,heads,kv_heads,dtype,cut", CUT_AND_UNCUT)
def test_infinities_and_nan_reach_the_rows_that_see_them_however_a_call_is_cut(prefix, new, window, heads, kv_heads, dtype, cut, far):
    """In V.  A channel is then infinite or NaN (which of them is left open: a weight that is 0 in 32 bits, times an infinity, is NaN)."""
    case, places = _of_odd_values(prefix, new, window, heads, kv_heads, dtype, cut, far)
    odd = torch.tensor([float("nan"), float("inf"), -float("inf")]).to(case.v.dtype)
    for (page, place), (page2, place2) in places:
        case.v[page, 0, place, [3, 40, 77]] = odd
        case.v[page2, kv_heads - 1, place2, [9, 50, 127]] = odd
    case.to_device()
    assert (case.workspace is not None) == cut
    out, lse = case.run(decode=max(new) == 1)
    want, _, _ = M.window_attention(case.table, case.prefix, case.new, case.cu, _f64(case.q), _f64(case.k), _f64(case.v), case.page, window, 20, case.scale, case.rows)
    want = torch.from_numpy(want).to(DEV)
    odd = ~want.isfinite()
    assert odd.any(dim=2).any(dim=1).all() and not odd.all(dim=2).any()
    assert torch.equal(odd, ~out.isfinite())
    case.check(torch.where(odd, want, out.double()), lse)                    # the others' values


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("prefix,new,window,heads,kv_heads,dtype,cut", CUT_AND_UNCUT)
def test_nan_in_k_reaches_the_rows_that_see_it_however_a_call_is_cut(prefix, new, window, heads, kv_heads, dtype, cut, far):
    """Their scores are NaN: so are the rows, and lse."""
    case, places = _of_odd_values(prefix, new, window, heads, kv_heads, dtype, cut, far)
    for (page, place), (page2, place2) in places:
        case.k[page, 0, place, 5] = float("nan")
        case.k[page2, 0, place2, 6] = float("nan")
    case.to_device()
    out, lse = case.run(decode=max(new) == 1)
    want, want_lse, _ = M.window_attention(case.table, case.prefix, case.new, case.cu, _f64(case.q), _f64(case.k), _f64(case.v), case.page, window, 20, case.scale, case.rows)
    assert np.isnan(want).any() and not np.isnan(want).all()
    assert np.array_equal(np.isnan(want_lse), np.isnan(_f64(lse)))
    case.check(out, lse)

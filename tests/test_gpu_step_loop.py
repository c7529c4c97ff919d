"""Page steps, norms with rotation and write, and attention with a window as a serving loop runs them: a prompt and then decode steps of several
requests, from a pool that is too small for whole contexts, the decode step captured once and replayed.  Each step against oracle/step_model.py in
64 bits over the whole history, rounded where the cache rounds.  Besides: two captured graphs with one workspace, other streams, pools beyond
32-bit offsets.

Tolerances.  Of attention those of test_gpu_window.py, of rows those of test_gpu_step.py; here K and q themselves are results, so that what their
rounding may move (half a step, 2^-8, of each of q and k) goes into the scores: 2 * 2^-8 * sum |q_i k_i| * scale where a value lies next to a
border.  That bound is far too wide to tell a mistake, so the oracle takes the rows that the device wrote, which are compared with its own first."""
import numpy as np
import pytest
import torch

from oracle import step_model as M
from paper_2507_10069_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _f64(t):
    return t.detach().double().cpu().numpy()


def _i32(a):
    return torch.tensor(np.ascontiguousarray(a), dtype=torch.int32, device=DEV)


def _bits(t):
    return t.contiguous().view(torch.uint8)


class Loop:
    def __init__(self, reqs, *, window, sinks, pages, width, heads=8, kv_heads=2, d=128, page=16, dtype="bf16", seed=0):
        self.n, self.window, self.sinks, self.pages, self.width, self.page = reqs, window, sinks, pages, width, page
        self.heads, self.kv_heads, self.d, self.dtype = heads, kv_heads, d, dtype
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.gen = torch.Generator().manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        z = lambda n, v=0, dt=torch.int32: torch.full((n,), v, dtype=dt, device=DEV)
        self.table, self.free = torch.full((reqs, width), -1, dtype=torch.int32, device=DEV), _i32(self.rng.permutation(pages))
        self.lens, self.held, self.count = z(reqs), z(reqs), z(1, pages)
        self.prefix, self.new, self.cu, self.add, self.refused = z(reqs), z(reqs), z(reqs + 1), z(reqs), z(1)
        shape = (pages, kv_heads, page, d)
        nan = float("nan")
        self.k_pool, self.v_pool = (torch.full(shape, nan, dtype=self.dt, device=DEV) for _ in range(2))
        self.weights = [(1 + 0.2 * torch.randn(d, generator=self.gen)).to(DEV) for _ in range(2)]
        self.norm = B.make_qk_norm(*self.weights, eps=1e-6)
        self.inv = 1e4 ** (-2.0 * np.arange(d // 2) / d)
        self.inv_dev = torch.from_numpy(self.inv).to(DEV)
        self.history = [[np.zeros((0, kv_heads, d)) for _ in range(2)] for _ in range(reqs)]             # K and V rows of every token so far

    def descriptors(self, tokens, longest):
        """What a step of at most `tokens` tokens works with; each kind of step keeps its own."""
        s = {"tokens": tokens, "slots": torch.zeros(tokens, dtype=torch.int64, device=DEV), "positions": torch.zeros(tokens, dtype=torch.int32, device=DEV)}
        s["rows"] = torch.zeros((tokens, self.heads + 2 * self.kv_heads, self.d), dtype=self.dt, device=DEV)
        s["q"], s["out"] = (torch.zeros((tokens, self.heads, self.d), dtype=self.dt, device=DEV) for _ in range(2))
        s["lse"] = torch.zeros((tokens, self.heads), device=DEV)
        s["step"] = B.make_page_step(num_reqs=self.n, page_size=self.page, num_pages=self.pages, max_pages_per_req=self.width, max_tokens=tokens,
                                     window=self.window, sinks=self.sinks, page_table=self.table, free_pages=self.free, lens=self.lens, add_lens=self.add,
                                     held_from=self.held, free_count=self.count, prefix_lens=self.prefix, new_lens=self.new, cu_new_lens=self.cu,
                                     lens_out=self.lens, held_out=self.held, free_count_out=self.count, slots=s["slots"], positions=s["positions"],
                                     refused=self.refused)
        s["batch"] = B.make_batch(num_reqs=self.n, num_q_heads=self.heads, num_kv_heads=self.kv_heads, head_dim=self.d, page_size=self.page, num_pages=self.pages,
                                  max_pages_per_req=self.width, total_new_tokens=tokens, max_new_len=longest, dtype=self.dtype, softmax_scale=self.d ** -0.5,
                                  page_table=self.table, prefix_lens=self.prefix, new_lens=self.new, cu_new_lens=self.cu)
        s["rope"] = B.make_rope(self.inv_dev, rotary_dim=self.d, positions=s["positions"])
        n = B.emm_attn_window_workspace_size(s["batch"], self.window, self.sinks)
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
        s["longest"] = longest
        return s

    def calls(self, s):
        B.emm_page_step(s["step"])
        rows, h, kv = s["rows"], self.heads, self.kv_heads
        B.emm_norm_rope_kv_scatter(s["batch"], self.norm, s["rope"], rows[:, :h], rows[:, h:h + kv], rows[:, h + kv:], s["q"], self.k_pool, self.v_pool,
                                   token_stride=rows.stride(0), slots=s["slots"])
        call = B.emm_decode_attn_window if s["longest"] == 1 else B.emm_prefill_attn_window
        call(s["batch"], self.window, self.sinks, s["q"], self.k_pool, self.v_pool, s["out"], s["lse"], s["workspace"])

    def feed(self, s, add):
        """The step's inputs: tokens of every request and a projection's rows."""
        self.before = [x.cpu().numpy().copy() for x in (self.table, self.free, self.count, self.lens, self.held)]
        self.add.copy_(_i32(add))
        s["rows"].copy_(torch.randn(s["rows"].shape, generator=self.gen).to(self.dt))
        self.added = [int(x) for x in add]

    def check(self, s):
        table, free, count, lens, held = self.before
        want = M.page_step(table, free, int(count[0]), lens, self.added, held, self.page, self.window, self.sinks, s["tokens"])
        for name, t in (("page_table", self.table), ("free_pages", self.free), ("prefix_lens", self.prefix), ("new_lens", self.new), ("cu_new_lens", self.cu),
                        ("lens_out", self.lens), ("held_out", self.held), ("free_count_out", self.count), ("slots", s["slots"]), ("positions", s["positions"]),
                        ("refused", self.refused)):
            got = t.cpu().numpy()
            assert np.array_equal(got, np.asarray(want[name], got.dtype).reshape(got.shape)), name
        T = want["cu_new_lens"][-1]
        rows = _f64(s["rows"])[:T]
        h, kv = self.heads, self.kv_heads
        angle = want["positions"][:T, None] * self.inv
        q, k = (M.norm_rope(x, _f64(w), 1e-6, angle, self.d, False) for x, w in ((rows[:, :h], self.weights[0]), (rows[:, h:h + kv], self.weights[1])))
        half = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
        slots = want["slots"][:T]
        got_k, got_v = (_f64(p[torch.from_numpy(slots // self.page).to(DEV), :, torch.from_numpy(slots % self.page).to(DEV)]) for p in (self.k_pool, self.v_pool))
        for got, x in ((_f64(s["q"])[:T], q), (got_k, k)):
            length = np.hypot(x[..., :self.d // 2], x[..., self.d // 2:])
            assert (np.abs(got - x) <= 1.01 * half * np.abs(x) + 4.5e-6 * np.concatenate([length, length], axis=-1) + 1e-38).all()
        assert np.array_equal(got_v, rows[:, h + kv:])
        for r, m in enumerate(want["new_lens"]):
            at = slice(want["cu_new_lens"][r], want["cu_new_lens"][r] + m)
            for which, x in ((0, got_k), (1, got_v)):
                self.history[r][which] = np.concatenate([self.history[r][which], x[at]])
        # attention over the whole history, each request in a table of its own
        longest = max(len(x[0]) for x in self.history)
        width = -(-max(longest, 1) // self.page)
        pools = [np.zeros((self.n * width, kv, self.page, self.d)) for _ in range(2)]
        for r in range(self.n):
            for which in range(2):
                x = self.history[r][which]
                i = np.arange(len(x))
                pools[which][r * width + i // self.page, :, i % self.page] = x
        own = np.arange(self.n * width).reshape(self.n, width)
        out, lse, size = M.window_attention(own, want["prefix_lens"], want["new_lens"], want["cu_new_lens"], _f64(s["q"]), pools[0], pools[1], self.page, self.window,
                                            self.sinks, self.d ** -0.5, s["tokens"])
        if T:
            e = (self.d + 2) * 2.0 ** -24 * self.d ** -0.5 * np.linalg.norm(_f64(s["q"])[:T], axis=-1) * np.sqrt((pools[0] ** 2).sum(-1).max())
            weight = e + 2.0 ** -19 + (self.window + self.sinks) * 2.0 ** -24
            bf16 = self.dtype == "bf16"
            tol = 2.0 ** -8 * bf16 * size[:T] + weight[..., None] * (size[:T] + np.abs(out[:T])) + (2.0 ** -8 if bf16 else 2.0 ** -22) * np.abs(out[:T]) + 1e-30
            assert (np.abs(_f64(s["out"])[:T] - out[:T]) <= tol).all()
            assert (np.abs(_f64(s["lse"])[:T] - lse[:T]) <= weight + 2.0 ** -22 * np.abs(lse[:T])).all()
        return want


@pytest.mark.parametrize("dtype,heads,kv_heads", [("bf16", 28, 4), ("bf16", 8, 8), ("f32", 4, 1)])
def test_prompt_and_captured_decode_steps(dtype, heads, kv_heads):
    """5 requests whose contexts pass 200 tokens in a pool that holds 58 pages of 16: with a window of 60 they live on 6 pages each."""
    loop = Loop(5, window=60, sinks=5, pages=58, width=24, heads=heads, kv_heads=kv_heads, dtype=dtype, d=128 if dtype == "bf16" else 64, seed=heads)
    prompt = loop.descriptors(420, 160)
    loop.feed(prompt, [130, 1, 77, 0, 150])
    loop.calls(prompt)
    loop.check(prompt)
    decode = loop.descriptors(5, 1)
    loop.feed(decode, [1, 1, 1, 1, 1])
    loop.calls(decode)                                       # once before the capture
    loop.check(decode)
    torch.cuda.synchronize()
    kept = [x.clone() for x in (loop.table, loop.free, loop.count, loop.lens, loop.held)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.calls(decode)
    for x, was in zip((loop.table, loop.free, loop.count, loop.lens, loop.held), kept):
        assert torch.equal(x, was)                           # a capture runs nothing
    taken = set()
    for step in range(150):
        loop.feed(decode, loop.rng.integers(0, 4, 5).clip(0, 1) if step % 7 else [0] * 5)
        graph.replay()
        if step % 10 < 3:
            want = loop.check(decode)
            assert want["refused"] == [0]
        else:
            loop.history_of(decode)
        taken.add(int(loop.count[0]))
    assert int(loop.lens.max()) > 200 and min(taken) > 20    # pages came back


def _history_of(self, s):
    """A step that is not compared: its rows still are part of the contexts."""
    T = int(self.cu[-1])
    slots = s["slots"][:T]
    k, v = (_f64(p[slots // self.page, :, slots % self.page]) for p in (self.k_pool, self.v_pool))
    cu = self.cu.cpu().numpy()
    for r in range(self.n):
        for which, x in ((0, k), (1, v)):
            self.history[r][which] = np.concatenate([self.history[r][which], x[cu[r]:cu[r + 1]]])


Loop.history_of = _history_of


def test_a_pool_that_runs_out_refuses_and_goes_on():
    loop = Loop(3, window=0x7fffffff, sinks=0, pages=6, width=8, seed=3)
    s = loop.descriptors(60, 40)
    refused = 0
    for add in ([30, 20, 0], [10, 10, 10], [0, 40, 16], [2, 0, 1], [0, 0, 33]):
        loop.feed(s, add)
        loop.calls(s)
        refused += loop.check(s)["refused"][0]
    assert refused == 3


def _attention(seed, reqs=3, context=3000, window=2500, new=1, heads=28, kv_heads=4, pages=None, high=False):
    """A decode or prefill batch that is cut into parts; with `high` its pages lie at the end of a large pool."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    width = -(-(context + new) // 16)
    used = reqs * width
    pages = pages or used
    k, v = (torch.empty((pages, kv_heads, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ids = torch.randperm(used, generator=gen, device=DEV).int() + (pages - used if high else 0)
    k[ids.long()] = torch.randn((used, kv_heads, 16, 128), generator=gen, device=DEV, dtype=torch.bfloat16)
    v[ids.long()] = torch.randn((used, kv_heads, 16, 128), generator=gen, device=DEV, dtype=torch.bfloat16)
    table = ids.view(reqs, width)
    s = {"k": k, "v": v, "table": table, "q": torch.randn((reqs * new, heads, 128), generator=gen, device=DEV, dtype=torch.bfloat16), "window": window}
    s["lens"] = [torch.full((reqs,), context, dtype=torch.int32, device=DEV), torch.full((reqs,), new, dtype=torch.int32, device=DEV),
                 torch.arange(reqs + 1, dtype=torch.int32, device=DEV) * new]
    s["batch"] = B.make_batch(num_reqs=reqs, num_q_heads=heads, num_kv_heads=kv_heads, head_dim=128, page_size=16, num_pages=pages, max_pages_per_req=width,
                              total_new_tokens=reqs * new, max_new_len=new, dtype="bf16", softmax_scale=128 ** -0.5, page_table=table, prefix_lens=s["lens"][0],
                              new_lens=s["lens"][1], cu_new_lens=s["lens"][2])
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((reqs * new, heads), device=DEV)
    s["bytes"] = B.emm_attn_window_workspace_size(s["batch"], window, 4)
    return s


def _run(s, workspace, stream=None):
    B.emm_prefill_attn_window(s["batch"], s["window"], 4, s["q"], s["k"], s["v"], s["out"], s["lse"], workspace, stream)


@pytest.mark.parametrize("new", [1, 9, 120])
def test_two_graphs_share_a_workspace(new):
    a, b = _attention(1, new=new), _attention(2, new=new, reqs=2, context=4000)
    assert a["bytes"] > 0 and b["bytes"] > 0
    workspace = torch.empty(max(a["bytes"], b["bytes"]), dtype=torch.uint8, device=DEV)
    want = []
    for s in (a, b):
        _run(s, workspace)
        want.append((s["out"].clone(), s["lse"].clone()))
    graphs = []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            _run(s, workspace)
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0, 0):
        s = (a, b)[i]
        s["out"].fill_(9.0)
        workspace.fill_(0xFF)                                # NaN: nothing of an earlier replay is used
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(_bits(s["out"]), _bits(want[i][0])) and torch.equal(_bits(s["lse"]), _bits(want[i][1]))


def test_two_streams_at_once():
    a, b = _attention(3, new=1), _attention(4, new=120, reqs=2)
    spaces = [torch.empty(s["bytes"], dtype=torch.uint8, device=DEV) for s in (a, b)]
    want = []
    for s, w in zip((a, b), spaces):
        _run(s, w)
        want.append(s["out"].clone())
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, w, st in zip((a, b), spaces, streams):
            _run(s, w, st)
    torch.cuda.synchronize()
    for s, x in zip((a, b), want):
        assert torch.equal(_bits(s["out"]), _bits(x))


@pytest.mark.parametrize("new", [1, 9, 120, 1500])
def test_pools_beyond_32_bit_offsets(new):
    """Pages whose bytes lie beyond 2^32, and their elements beyond 2^31: the same values in a small pool have the same bits."""
    pages = 300000                                           # 16 KB each: 4.9 GB
    near, far = _attention(5, reqs=2, new=new), _attention(5, reqs=2, new=new, pages=pages, high=True)
    assert far["k"].numel() > 2 ** 31
    for s in (near, far):
        _run(s, torch.empty(max(s["bytes"], 16), dtype=torch.uint8, device=DEV))
    assert torch.equal(_bits(near["out"]), _bits(far["out"])) and torch.equal(_bits(near["lse"]), _bits(far["lse"]))


@pytest.mark.parametrize("given", [False, True])
def test_writes_beyond_32_bit_offsets(given):
    pages, T = 300000, 20
    k_pool, v_pool = (torch.zeros((pages, 4, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.tensor([[pages - 1, pages - 7]], dtype=torch.int32, device=DEV)
    lens = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([3], [T], [0, T])]
    batch = B.make_batch(num_reqs=1, num_q_heads=8, num_kv_heads=4, head_dim=128, page_size=16, num_pages=pages, max_pages_per_req=2, total_new_tokens=T, max_new_len=T,
                         dtype="bf16", softmax_scale=0.1, page_table=table, prefix_lens=lens[0], new_lens=lens[1], cu_new_lens=lens[2])
    q, k, v = (torch.randn((T, h, 128), device=DEV).bfloat16() for h in (8, 4, 4))
    w = torch.ones(128, device=DEV)
    at = torch.arange(3, 3 + T, device=DEV)
    slots = table[0].long()[at // 16] * 16 + at % 16
    q_out, k_alone = torch.empty_like(q), torch.empty_like(k)
    norm = B.make_qk_norm(w, w, eps=1e-6)
    B.emm_norm_rope_kv_scatter(batch, norm, None, q, k, v, q_out, k_pool, v_pool, slots=slots if given else None)
    B.emm_norm_rope(batch, norm, None, None, k, None, k_alone)
    assert torch.equal(k_pool[slots // 16, :, slots % 16], k_alone) and torch.equal(v_pool[slots // 16, :, slots % 16], v)
    assert int((v_pool != 0).any(dim=-1).sum()) == 4 * T     # nothing else was written

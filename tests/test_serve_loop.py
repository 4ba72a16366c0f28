"""The operators around a verification together, as a serving loop uses them, eagerly and as one captured graph; and the
attention in every form of its kernel, at its limits, and with what is no finite number."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import serveref  # noqa: E402
from tests.test_serve_ops import BF, HF, Attn, Shape, binding, handle, tree  # noqa: E402,F401


class Loop:
    """A loop of B trajectories with random queries, keys, values and logits in place of a model; what has to come out is kept
    on the CPU as plain lists: the cached rows of every trajectory in order, the tokens that were generated."""

    def __init__(self, binding, dtype, logits, V=96, N=9, L=2, H=4, G=2, d=64, page=8, P=60, width=12):
        self.rng, self.gen = np.random.default_rng(7), torch.Generator().manual_seed(7)
        self.B, self.V, self.N, self.L, self.H, self.G, self.d, self.page = 4, V, N, L, H, G, d, page
        self.parent = tree(N)
        self.h = handle(binding, self.B, self.parent, V, binding.STAND_F32 if logits == torch.float32 else binding.STAND_BF16)
        self.dtype, self.logits_dtype, self.W = dtype, logits, self.h.W
        i32, B = dict(dtype=torch.int32, device="cuda"), self.B
        pool = torch.randn((2, L, P, page, G, d), generator=self.gen).to(dtype).cuda()
        self.cache, self.pool = binding.PagedCache(pool[0], pool[1]), pool
        self.pages = binding.Pages.new(B, P, page, width)
        self.tok, self.next = torch.full((B, N), -1, **i32), torch.full((B, N), -1, **i32)
        self.count, self.out_len = torch.zeros((B, V), **i32), torch.zeros(B, **i32)
        self.out_tok, self.out_node = torch.zeros((B, self.W), **i32), torch.zeros((B, self.W), **i32)
        self.slots, self.missing = torch.zeros((B, self.W), dtype=torch.int64, device="cuda"), torch.zeros(B, **i32)
        self.room = torch.full((B,), self.W, **i32)
        self.qkv = torch.zeros((L, B, N, H + 2 * G, d), dtype=dtype, device="cuda")
        self.out = torch.zeros((L, B, N, H, d), dtype=dtype, device="cuda")
        self.x, self.shaped = (torch.zeros((B, N, V), dtype=logits, device="cuda") for _ in range(2))
        self.penalty = torch.tensor([[1.3, 0.2, 0.1], [1.0, 0.0, 0.0], [0.8, 0.0, 0.3], [1.1, -0.1, 0.0]], device="cuda")
        self.bias_id, self.bias = torch.tensor([[3, 5, -1]] * B, **i32), torch.tensor([[2.0, -np.inf, 1.0]] * B, device="cuda")
        self.allow = torch.full((B, N, (V + 31) // 32), -1, **i32)
        # prompts: tokens into contexts and counts, their rows but the last into the cache
        lens = [11, 1, 24, 8]
        prompt = self.rng.integers(0, V, (B, max(lens))).astype(np.int32)
        for b, n in enumerate(lens):
            self.h.set_context(b, prompt[b, :n].tolist())
        self.h.count_tokens(self.count, torch.from_numpy(prompt).cuda(), torch.tensor(lens, **i32), prompt=True)
        n = torch.tensor(lens, **i32) - 1
        slots = torch.zeros((B, max(lens)), dtype=torch.int64, device="cuda")
        assert not self.h.cache_pages(self.pages, None, n, slots).any()
        rows = torch.randn((2, L, B, max(lens), G, d), generator=self.gen).to(dtype)
        self.h.cache_commit(self.cache, rows[0].cuda(), rows[1].cuda(), slots, None, n)
        self.out_len.copy_(n)
        self.rows = [[rows[:, :, b, j] for j in range(lens[b] - 1)] for b in range(B)]       # of [2, L, G, d]
        self.made = np.zeros((B, V), np.int64)
        for b, m in enumerate(lens):
            self.made[b, prompt[b, :m]] |= 1 << 30
        self.h.draft(7, self.tok)

    def iteration(self):
        h, H, G = self.h, self.H, self.G
        q, k, v = self.qkv[..., :H, :], self.qkv[..., H:H + G, :], self.qkv[..., H + G:, :]
        h.cache_pages(self.pages, self.out_len, self.room, self.slots, self.missing)
        for l in range(self.L):
            h.tree_attention(self.cache, l, self.pages.length, self.pages.table, self.tok, q[l], k[l], v[l], out=self.out[l])
        h.shape_logits(self.x, self.shaped, self.tok, self.count, self.penalty, self.bias_id, self.bias, self.allow)
        h.step(7, self.shaped, self.out_tok, self.out_node, self.out_len, self.next)
        h.cache_commit(self.cache, k, v, self.slots, self.out_node, self.out_len)
        h.count_tokens(self.count, self.out_tok, self.out_len)

    def step(self, run, leaves=None):
        """One iteration by `run` on new random rows and logits, everything compared."""
        B, N, V, page = self.B, self.N, self.V, self.page
        qkv = torch.randn(self.qkv.shape, generator=self.gen).to(self.dtype)
        x = torch.randn((B, N, V), generator=self.gen) * 2
        x[:, :, :4] += 3.0                               # few tokens, so that the table learns and drafts are accepted
        x = x.to(self.logits_dtype)
        allow = self.rng.integers(0, 2 ** 32, self.allow.shape, dtype=np.uint64) | 15
        allow[0, 3:] = 0
        self.qkv.copy_(qkv)
        self.x.copy_(x)
        self.allow.copy_(torch.from_numpy(allow.astype(np.uint32).view(np.int32)))
        self.room.fill_(self.W)
        if leaves is not None:
            self.room[leaves] = -1
            self.rows[leaves] = []
        tok = self.tok.clone()
        run()
        torch.cuda.synchronize()
        lens = [len(r) for r in self.rows]
        assert self.pages.length.tolist() == lens and self.missing.tolist() == [0] * B
        # attention over the rows as they were committed, in a cache of one long page for each trajectory
        most = max(lens) + 1
        flat = torch.zeros((2, self.L, B, most, self.G, self.d), dtype=self.dtype)
        for b, r in enumerate(self.rows):
            for j, row in enumerate(r):
                flat[:, :, b, j] = row
        H, G = self.H, self.G
        for l in range(self.L):
            want, tol = serveref.attention(self.parent, lens, torch.arange(B)[:, None], tok.cpu(), qkv[l, :, :, :H], qkv[l, :, :, H:H + G],
                                           qkv[l, :, :, H + G:], flat[0, l], flat[1, l], self.d ** -0.5)
            assert bool(((self.out[l].cpu().double() - want).abs() <= tol).all()), "layer %d" % l
        want, tol = serveref.shape(self.parent, x, tok.cpu(), torch.from_numpy(self.made.astype(np.int32)), self.penalty.cpu(), self.bias_id.cpu(),
                                   self.bias.cpu(), self.allow.cpu())
        got = self.shaped.cpu().double()
        assert bool((((got - want).abs() <= tol) | (got == want)).all())
        # what was accepted: tokens into the counts, rows into the cache
        out_tok, out_node, out_len = self.out_tok.cpu().numpy(), self.out_node.cpu().numpy(), self.out_len.cpu().numpy()
        for b in range(B):
            assert 1 <= out_len[b] <= self.W
            for j in range(out_len[b]):
                u, t = out_node[b, j], out_tok[b, j]
                assert np.isfinite(float(got[b, u, t]))          # no token that a mask or a bias forbids
                self.made[b, t] += 1
                if b != leaves:
                    self.rows[b].append(torch.stack([qkv[:, b, u, H:H + G], qkv[:, b, u, H + G:]]))
        assert np.array_equal(self.count.cpu().numpy(), self.made)
        slots = self.slots.cpu().numpy()
        if leaves is not None:
            assert (slots[leaves] == -1).all()
        pool = self.pool.cpu()
        for b, r in enumerate(self.rows):
            for j in range(out_len[b] if b != leaves else 0):
                at = slots[b, j]
                assert torch.equal(pool[:, :, at // page, at % page], r[lens[b] + j])
        self.tok.copy_(self.next)
        return int(out_len.sum())


@pytest.mark.parametrize("dtype,logits", [(BF, BF), (HF, torch.float32)])
@pytest.mark.parametrize("captured", [False, True], ids=["eager", "graph"])
def test_a_serving_loop(binding, dtype, logits, captured):
    t = Loop(binding, dtype, logits)
    emitted = t.step(t.iteration)
    run = t.iteration
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):                    # (records, runs nothing)
            t.iteration()
        run = graph.replay
    for i in range(7):
        emitted += t.step(run, leaves=2 if i == 3 else None)
    assert emitted >= 8 * t.B


def test_two_captured_loops_at_once(binding):
    """Two graphs, each with its own buffers and workspaces, replayed on two streams without waiting for each other."""
    ts = [Attn(binding, 70 + i, [900, 40 * i], 16, 8, 2, 128, 16, BF) for i in range(2)]
    sh = [Shape(binding, 72 + i, 2, 16, 1500, BF, 5, True) for i in range(2)]
    graphs = []
    for t, s in zip(ts, sh):
        a, b = t.on_gpu(), s.args()
        a["out"], b["out"] = torch.empty(a["q"].shape, dtype=BF, device="cuda"), torch.empty_like(b["logits"])
        t.h.tree_attention(**a)
        s.h.shape_logits(**b)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(3):
                t.h.tree_attention(**a)
                s.h.shape_logits(**b)
        graphs.append((g, torch.cuda.Stream(), a, b))
    for rep in range(3):
        for g, stream, a, b in graphs:
            a["out"].fill_(9.0)
            b["out"].fill_(9.0)
        torch.cuda.synchronize()
        for g, stream, a, b in graphs:
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        for t, s, (_, _, a, b) in zip(ts, sh, graphs):
            t.check(a["out"])
            s.check(b["out"])


# ---- every form of the attention kernel ---------------------------------------------------------------------------------

FORMS = [(1, 1, 1), (16, 2, 1), (32, 2, 1), (33, 1, 1), (64, 1, 1), (64, 2, 1), (33, 7, 1), (130, 4, 2), (64, 8, 2),   # N, heads, kv heads
         (130, 3, 1), (130, 4, 1)]                  # a full tile and a small one, a full one and most of one


@pytest.mark.parametrize("d,dtype", [(64, BF), (64, HF), (128, BF), (128, HF)])
@pytest.mark.parametrize("N,H,G", FORMS)
def test_forms(binding, N, H, G, d, dtype):
    """Long and short caches side by side: whole units in the fast loop, ends inside a tile, shares of several items."""
    Attn(binding, 80 + N + H, [1500, 577, 0, 40], N, H, G, d, 16, dtype, 0.8 if N > 1 else 1.0).check()


@pytest.mark.parametrize("d,dtype", [(64, HF), (128, BF)])
@pytest.mark.parametrize("N,H,G", FORMS)
def test_forms_with_values_that_are_not_finite(binding, N, H, G, d, dtype):
    """NaN and infinities behind the lengths change nothing; an infinite cached value reaches its element, and nothing else."""
    t = Attn(binding, 90 + N + H, [700, 130, 0, 40], N, H, G, d, 16, dtype, 0.8 if N > 1 else 1.0)
    used = torch.zeros((t.pages, t.page), dtype=torch.bool)
    for b, n in enumerate(t.lens):
        for p in range(n):
            used[t.table[b, p // t.page], p % t.page] = True
    t.kp[0][~used], t.vp[0][~used] = float("nan"), float("-inf")
    t.check()
    at = (t.table[0, 300 // 16], 300 % 16)
    clean, tol = t.want()
    t.vp[0][at][0, 5] = float("inf")
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    drafted = torch.from_numpy(t.tok[0]) >= 0
    per = H // G
    assert not bool(torch.isfinite(got[0, drafted][:, :per, 5]).any())
    got[0, :, :per, 5] = clean[0, :, :per, 5]
    assert bool(((got - clean).abs() <= tol).all())
    leaf = max(u for u in range(N) if t.tok[1, u] >= 0)      # nobody sees it but itself
    t.v[1, leaf, 0, 7], t.v[1, leaf, G - 1, 9] = float("-inf"), float("nan")
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    assert not bool(torch.isfinite(got[1, leaf, :per, 7]).any()) and bool(torch.isnan(got[1, leaf, (G - 1) * per:, 9]).all())
    got[0, :, :per, 5], got[1, leaf, :per, 7], got[1, leaf, (G - 1) * per:, 9] = (
        clean[0, :, :per, 5], clean[1, leaf, :per, 7], clean[1, leaf, (G - 1) * per:, 9])
    assert bool(((got - clean).abs() <= tol).all())


def test_attention_of_nothing_drafted(binding):
    t = Attn(binding, 95, [300, 5], 16, 8, 2, 128, 16, BF)
    t.tok[:] = -1
    a = t.on_gpu()
    a["out"] = torch.full(a["q"].shape, float("nan"), dtype=BF, device="cuda")
    assert bool((t.h.tree_attention(**a) == 0).all())


def test_attention_of_shared_pages_and_broadcast_queries(binding):
    """Trajectories with the same pages; one query, key and value for all of them."""
    t = Attn(binding, 96, [200, 200, 200], 9, 4, 2, 64, 16, BF, 1.0)
    t.table[1:] = t.table[0]
    t.lens = [200, 150, 7]
    t.q, t.k, t.v = (x[:1].expand(3, *x.shape[1:]) for x in (t.q, t.k, t.v))
    a = t.on_gpu()
    for n in ("q", "k", "v"):
        a[n] = a[n][:1].expand(3, *a[n].shape[1:])
    t.check(t.h.tree_attention(**dict(a, out=torch.empty((3, 9, 4, 64), dtype=BF, device="cuda"))))


def test_attention_of_as_many_trajectories_as_it_takes(binding):
    lens = [int(x) for x in np.random.default_rng(3).integers(0, 40, 4096)]
    Attn(binding, 97, lens, 1, 2, 1, 64, 16, BF, 1.0).check()
    t = Attn(binding, 98, lens + [3], 1, 2, 1, 64, 16, BF, 1.0)
    with pytest.raises(binding.StandError):
        t.h.tree_attention(**t.on_gpu())


def test_attention_workspaces_that_are_too_small_are_refused(binding):
    t = Attn(binding, 99, [40], 9, 4, 2, 64, 16, BF)
    a = t.on_gpu()
    need = t.h._lib.stand_tree_attention_work(t.h.h, a["cache"].ref, 4)
    assert need > 0 and t.h._lib.stand_tree_attention_work(t.h.h, a["cache"].ref, 3) == 0
    t.h._work_bytes = {k: need - 1 for k in [(4, 2, 64, a["cache"].desc.dtype)]}
    with pytest.raises(binding.StandError):
        t.h.tree_attention(**a)


# ---- more of the others -------------------------------------------------------------------------------------------------

def test_pages_of_many_trajectories(binding):
    """Several trajectories to a thread and to a workgroup."""
    B, page, width, P, W = 20011, 16, 3, 50000, 5
    rng = np.random.default_rng(11)
    h = handle(binding, B, tree(2))
    p = binding.Pages.new(B, P, page, width)
    state = dict(table=p.table.cpu().tolist(), ring=p.ring.cpu().tolist(), length=[0] * B, held=[0] * B, mark=[0, P])
    for rep in range(3):
        add, room = rng.integers(0, 9, B).tolist(), np.where(rng.random(B) < 0.1, -1, rng.integers(0, 40, B)).tolist()
        want = serveref.pages(page, state["table"], state["ring"], state["length"], state["held"], state["mark"], add, room, W, 2)
        slots = torch.empty((B, W), dtype=torch.int64, device="cuda")
        i32 = dict(dtype=torch.int32, device="cuda")
        missing = h.cache_pages(p, torch.tensor(add, **i32), torch.tensor(room, **i32), slots)
        got = dict(length=p.length, held=p.held, mark=p.mark, table=p.table, ring=p.ring, missing=missing, slots=slots)
        for k, x in got.items():
            assert x.cpu().tolist() == want[k], k
        state = {k: want[k] for k in state}


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_shape_of_logits_that_are_not_finite(binding, dtype):
    """Infinite logits of repeated tokens stay infinite, NaN stays NaN, overflow rounds to infinity."""
    t = Shape(binding, 61, 1, 2, 64, dtype, 0, None, True, False, share=1.0)
    t.count = torch.full((1, 64), 1, dtype=torch.int32)
    t.penalty = torch.tensor([[0.5, 0.25, 0.5]])
    t.x[:, :, 0], t.x[:, :, 1], t.x[:, :, 2], t.x[:, :, 3] = float("inf"), float("-inf"), float("nan"), 3e38
    got = t.h.shape_logits(out=None, **t.args()).cpu()
    assert bool(torch.isposinf(got[:, :, 0]).all()) and bool(torch.isneginf(got[:, :, 1]).all())
    assert bool(torch.isnan(got[:, :, 2]).all()) and bool(torch.isposinf(got[:, :, 3]).all())
    assert bool(torch.isfinite(got[:, :, 4:]).all())

"""A cache in 4 bits and the way into it: heads normed and rotated, rows into the cache and out of it, attention over it, against
plain implementations in 64 bits; alone, together as a serving loop uses them, captured, and at their limits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_04708_amd import synth  # noqa: E402
from tests import serveref, serveref4, test_serve_ops  # noqa: E402
from tests.test_serve_ops import BF, HF, Attn, binding, drafts, handle, tree  # noqa: E402,F401

I32 = dict(dtype=torch.int32, device="cuda")
for _n, _deep, _fan in ((70, 8, [8, 4, 2, 1]), (300, 12, [8, 4, 2, 1]), (1024, 31, [8, 4, 2, 1])):
    test_serve_ops.TREES.setdefault(_n, synth.make_tree(_n, _deep, _fan).tolist())


def norm_weights(gen, d, dtype, norm):
    return [(1 + 0.3 * torch.randn(d, generator=gen)).to(dtype) if n else None for n in norm]


def cuda(t):
    return None if t is None else t.cuda()


def layout_of(x, layout):
    """x [layers, pages, page, heads, e] on the GPU in that order of memory."""
    return x.cuda() if layout == "nhd" else x.transpose(2, 3).contiguous().cuda().transpose(2, 3)


# ---- rotation -------------------------------------------------------------------------------------------------------------

class Rotate:
    def __init__(self, binding, seed, lens, N, H, G, d, dtype, dims, pairs="halves", norm=(True, True), share=0.7, fused=True, positions=None, eps=1e-6):
        rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        B = len(lens)
        self.lens, self.parent, self.pairs, self.eps, self.dtype = lens, tree(N), pairs, eps, dtype
        self.depth = torch.from_numpy(serveref.depths(self.parent))
        self.tok = drafts(rng, B, self.parent, share)
        self.turns = serveref4.turns(positions or max(lens) + int(self.depth.max()) + 1, dims) if dims else None
        self.w = norm_weights(gen, d, dtype, norm)
        qk = torch.randn((B, N, H + G, d), generator=gen).to(dtype)
        self.q, self.k = (qk[:, :, :H], qk[:, :, H:]) if fused else (qk[:, :, :H].contiguous(), qk[:, :, H:].contiguous())
        self.h, self.binding, self.fused = handle(binding, B, self.parent), binding, fused

    def args(self):
        q, k = self.q, self.k
        if self.fused:
            qk = torch.cat([q, k], 2).cuda()
            q, k = qk[:, :, :q.shape[2]], qk[:, :, q.shape[2]:]
        else:
            q, k = q.cuda(), k.cuda()
        return dict(rotation=self.binding.Rotation(cuda(self.turns), self.pairs, *(cuda(w) for w in self.w), self.eps), length=torch.tensor(self.lens, **I32),
                    draft_tok=torch.from_numpy(self.tok).cuda(), q=q, k=k)

    def check(self, got, left):
        pos = torch.tensor(self.lens)[:, None].long() + self.depth
        drafted = torch.from_numpy(self.tok) >= 0
        for x, w, y, l in zip((self.q, self.k), self.w, got, left):
            want = serveref4.turned(x, pos, self.turns, self.pairs, w, self.eps)
            tol = serveref4.turned_error(want, self.dtype)
            y = y.cpu()
            ok = ((y.double() - want).abs() <= tol) | (torch.isnan(want) & torch.isnan(y))
            assert bool(ok[drafted].all()), (y[drafted][~ok[drafted]][:3], want[drafted][~ok[drafted]][:3])
            assert torch.equal(y[~drafted], l[~drafted])


@pytest.mark.parametrize("case", [
    # lengths, N, query heads, kv heads, d, type, rotated elements, pairs, norms, share of drafted nodes, fused
    ([0], 1, 1, 1, 64, BF, 64, "halves", (False, False), 1.0, True),
    ([5], 1, 3, 1, 128, HF, 128, "neighbours", (True, True), 1.0, False),
    ([37], 16, 14, 2, 64, HF, 64, "halves", (True, False), 0.8, True),
    ([1000, 0, 33], 9, 28, 4, 128, BF, 128, "halves", (True, True), 0.7, True),
    ([4, 90, 2, 7], 33, 5, 5, 64, BF, 48, "halves", (False, True), 0.6, False),
    ([4, 90], 130, 16, 8, 128, HF, 48, "neighbours", (True, True), 0.6, True),
    ([70000, 3], 64, 7, 1, 128, BF, 64, "halves", (True, True), 1.0, True),
    ([12, 1], 32, 2, 1, 64, HF, 16, "neighbours", (False, False), 0.97, True),
    ([12, 1], 9, 2, 1, 128, BF, 0, "halves", (True, True), 0.9, True),
    ([9] * 70, 2, 2, 1, 128, BF, 112, "halves", (True, True), 0.9, True),
    ([3], 1024, 3, 1, 64, BF, 32, "halves", (True, True), 0.98, False),
    ([7, 900] * 8, 300, 40, 20, 128, HF, 128, "halves", (True, False), 0.7, True),    # more rows than the L2 keeps
], ids=lambda c: "B%d-N%d-%dx%d-d%d-%s%d" % (len(c[0]), c[1], c[2], c[3], c[4], c[7][0], c[6]))
def test_rotate(binding, case):
    lens, N, H, G, d, dtype, dims, pairs, norm, share, fused = case
    t = Rotate(binding, N + H + d, lens, N, H, G, d, dtype, dims, pairs, norm, share, fused)
    a = t.args()
    out = [torch.full((len(lens), N, x, d), 7.0, dtype=dtype, device="cuda") for x in (H, G)]
    got = t.h.tree_rotate(**a, q_out=out[0], k_out=out[1])
    assert got[0] is out[0] and got[1] is out[1]
    t.check(out, [x.fill_(7.0) for x in (torch.empty(o.shape, dtype=dtype) for o in out)])
    assert torch.equal(a["q"].cpu(), t.q) and torch.equal(a["k"].cpu(), t.k)
    t.check(t.h.tree_rotate(**a), (t.q, t.k))                # in place
    b = t.args()
    t.h.tree_rotate(**dict(b, q=b["q"].clone()), q_out=out[0], k_out=b["k"])
    assert torch.equal(b["k"], a["k"])


def test_rotate_keys_alone_and_positions_outside(binding):
    t = Rotate(binding, 3, [5, 40, 0], 9, 4, 2, 64, BF, 32, norm=(True, True), share=1.0, positions=42)
    t.lens = [5, 40, -1]                                     # of the second one's nodes those below depth 1 are outside, the third one's root
    a = t.args()
    q, k = t.h.tree_rotate(**a)
    t.check((q, k), (t.q, t.k))
    assert bool(torch.isnan(k[2, 0, :, :32]).all()) and bool(torch.isfinite(k[2, 0, :, 32:]).all()) and bool(torch.isfinite(k[2, 1]).all())
    b = t.args()
    none, only = t.h.tree_rotate(b["rotation"], b["length"], b["draft_tok"], None, b["k"])
    assert none is None and torch.equal(torch.nan_to_num(only), torch.nan_to_num(k)) and torch.equal(b["q"].cpu(), t.q)


@pytest.mark.parametrize("dtype,size", [(BF, 1e38), (BF, 1e-38), (HF, 6e4), (HF, 1e-7)])
def test_rotate_of_large_and_small_rows(binding, dtype, size):
    """Squares that no fp32 number holds; rows of zeros, infinities and NaN."""
    t = Rotate(binding, 5, [5, 40], 16, 4, 2, 128, dtype, 128, eps=0.0, share=1.0)
    for x in (t.q, t.k):
        x.copy_((x.double() / x.double().abs().amax() * size).to(dtype))
    t.check(t.h.tree_rotate(**t.args()), (t.q, t.k))
    t.eps = 1e-6
    t.q[0, 0, 0] = 0
    t.q[0, 1, 0, 5], t.q[0, 2, 0, 5] = float("inf"), float("nan")
    q, k = t.h.tree_rotate(**t.args())
    assert bool((q[0, 0, 0] == 0).all()) and bool(torch.isnan(q[0, 1, 0, 5])) and bool(torch.isnan(q[0, 2, 0]).all())
    t.q[0, 1:3, 0] = q[0, 1:3, 0] = 0
    t.check((q, k), (t.q, t.k))


# ---- rows into the cache and out of it --------------------------------------------------------------------------------------

class Cached:
    """A pool of either kind with random contents, kept on the CPU beside it."""

    def __init__(self, binding, gen, L, pages, page, G, d, dtype, bits, layout):
        self.dtype, self.bits, self.layout, self.binding = dtype, bits, layout, binding
        x = [torch.randn((L, pages, page, G, d), generator=gen).to(dtype) for _ in range(2)]
        if bits == 4:
            (k, ks), (v, vs) = (serveref4.pack(y, dtype) for y in x)
            self.want = [k, v, ks, vs]
        else:
            self.want = x
        self.gpu = [layout_of(y, layout) for y in self.want]
        self.cache = binding.PagedCache(*self.gpu, dtype=dtype) if bits == 4 else binding.PagedCache(*self.gpu)

    def put(self, l, at, place, k, v):
        """Rows [G, d], in 64 bits, where they have to be."""
        if self.bits == 4:
            for i, x in enumerate((k, v)):
                self.want[i][l, at, place], self.want[i + 2][l, at, place] = serveref4.pack(x.float(), self.dtype)
        else:
            self.want[0][l, at, place], self.want[1][l, at, place] = k.to(self.dtype), v.to(self.dtype)

    def values(self, i):
        return serveref4.unpack(self.want[i], self.want[i + 2], self.dtype) if self.bits == 4 else self.want[i]

    def check(self, near=False):
        """near: the keys were rounded from 64 bits by way of fp32 there and here, off by a step at the most."""
        for i, (x, y) in enumerate(zip(self.gpu, self.want)):
            x = x.cpu()
            if near and i == 0 and self.bits == 16:
                assert bool(((x.double() - y.double()).abs() <= 2 * serveref4.turned_error(y.double(), self.dtype)).all())
            else:
                assert torch.equal(x, y), (i, (x != y).nonzero()[:4], x[x != y][:4], y[x != y][:4])


APPENDS = [
    # layers, layer, rows, counts, starts, H, G, d, page, type, bits, layout, rotated, pairs, norms, queries
    (1, 0, 1, [1], [0], 1, 1, 64, 16, BF, 4, "nhd", 64, "halves", (False, False), True),
    (2, 1, 1, None, [0, 7, 900], 8, 2, 128, 16, HF, 16, "hnd", 128, "halves", (True, True), True),
    (1, 0, 40, [40, 0, 13], [0, 5, 300], 28, 4, 128, 64, BF, 4, "nhd", 128, "halves", (True, True), True),
    (3, 2, 33, [99, 7, -1], [3, 0, 60], 3, 3, 64, 8, HF, 4, "hnd", 48, "halves", (True, False), True),
    (1, 0, 17, [17, 16], [0, 1], 5, 5, 64, 1, BF, 16, "nhd", 32, "neighbours", (False, True), True),
    (1, 0, 70, [70, 66], None, 4, 1, 128, 32, HF, 4, "nhd", 128, "neighbours", (True, True), False),
    (2, 0, 130, [130], [2000], 4, 2, 128, 4096, BF, 4, "hnd", 16, "neighbours", (True, True), True),
    (1, 0, 600, [599, 1], [0, 17], 2, 1, 64, 16, HF, 16, "nhd", 64, "halves", (True, True), True),
    (1, 0, 24, [24, 3], [1, 2], 2, 2, 128, 16, BF, 4, "nhd", 0, "halves", (False, True), False),
]


def slots_of(rng, B, W, pages, page):
    """Distinct slots, a few of them none or past the end."""
    s = rng.permutation(pages * page)[: B * W].reshape(B, W).astype(np.int64)
    s[rng.random((B, W)) < 0.1] = -1
    if W > 3:
        s[0, 2], s[-1, 1] = pages * page, 2 ** 40
    return s


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "L%d-R%d-%dx%d-d%d-%dbit-%s%d" % (c[0], c[2], c[5], c[6], c[7], c[10], c[13][0], c[12]))
def test_append(binding, case):
    L, layer, R, counts, starts, H, G, d, page, dtype, bits, layout, dims, pairs, norm, queries = case
    seed = R + H + d + bits
    rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    B = len(counts or starts)
    W = R + 3 * (seed % 2)
    pages = -(-B * W // page) + 2
    c = Cached(binding, gen, L, pages, page, G, d, dtype, bits, layout)
    slots = slots_of(rng, B, W, pages, page)
    turns = serveref4.turns(max(starts or [0]) + R, dims) if dims else None
    w = norm_weights(gen, d, dtype, norm)
    qkv = torch.randn((B, R, H + 2 * G, d), generator=gen).to(dtype)
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + G], qkv[:, :, H + G:]
    pos = torch.tensor(starts or [0] * B)[:, None].long() + torch.arange(R)
    yk = serveref4.turned(k, pos, turns, pairs, w[1], 1e-6)
    yq = serveref4.turned(q, pos, turns, pairs, w[0], 1e-6)
    dev = qkv.cuda()
    rot = binding.Rotation(cuda(turns), pairs, *(cuda(x) for x in w), 1e-6)
    k_out = torch.full((B, R, G, d), 3.0, dtype=dtype, device="cuda")
    q_out = torch.full((B, R, H, d), 3.0, dtype=dtype, device="cuda")
    h = handle(binding, B, tree(1))
    h.cache_append(c.cache, layer, dev[:, :, H:H + G], dev[:, :, H + G:], torch.from_numpy(slots).cuda(), None if starts is None else torch.tensor(starts, **I32),
                   None if counts is None else torch.tensor(counts, **I32), rot, *((dev[:, :, :H], q_out) if queries else (None, None)), k_out)
    n = [min(max(x, 0), R) for x in counts] if counts else [R] * B
    for b in range(B):
        for j in range(n[b]):
            s = int(slots[b, j])
            if 0 <= s < pages * page:
                c.put(layer, s // page, s % page, yk[b, j], v[b, j].double())
    c.check(near=True)
    rows = torch.arange(R)[None] < torch.tensor(n)[:, None]
    for y, got in ((yk, k_out.cpu()),) + (((yq, q_out.cpu()),) if queries else ()):
        assert bool(((got.double() - y).abs() <= serveref4.turned_error(y, dtype))[rows].all()) and bool((got[~rows] == 3.0).all())
    assert torch.equal(dev.cpu(), qkv)


def test_append_as_it_stands_is_a_commit(binding):
    """Without a rotation the rows are copied or quantized as a commit does it."""
    gen = torch.Generator().manual_seed(1)
    for bits, dtype, d in ((16, BF, 64), (4, BF, 128), (4, HF, 64)):
        k, v = (torch.randn((2, 9, 3, d), generator=gen).to(dtype).cuda() for _ in range(2))
        slots = torch.randperm(48, generator=gen)[:18].reshape(2, 9).cuda()
        pair = [Cached(binding, torch.Generator().manual_seed(2), 1, 3, 16, 3, d, dtype, bits, "nhd") for _ in range(2)]
        h = handle(binding, 2, tree(1))
        h.cache_append(pair[0].cache, 0, k, v, slots)
        h.cache_commit(pair[1].cache, k[None], v[None], slots)
        for x, y in zip(pair[0].gpu, pair[1].gpu):
            assert torch.equal(x, y)


def test_append_in_place_and_rotated_rows_of_a_tree(binding):
    """A chain's nodes rotated as a tree's and appended as rows are the same bits; rotated rows committed are the appended ones."""
    gen, N, B, H, G, d = torch.Generator().manual_seed(4), 32, 3, 6, 2, 128
    for dtype in (BF, HF):
        parent = np.arange(-1, N - 1, dtype=np.int32)
        h = handle(binding, B, parent)
        q, k, v = (torch.randn((B, N, x, d), generator=gen).to(dtype).cuda() for x in (H, G, G))
        rot = binding.Rotation(serveref4.turns(600, 128).cuda(), "halves", *(cuda(w) for w in norm_weights(gen, d, dtype, (True, True))))
        length, tok = torch.tensor([0, 500, 33], **I32), torch.zeros((B, N), **I32)
        q1, k1 = h.tree_rotate(rot, length, tok, q, k, torch.empty_like(q), torch.empty_like(k))
        pool = torch.zeros((2, 1, 8, 16, G, d), dtype=dtype, device="cuda")
        slots = torch.randperm(128, generator=gen)[:B * N].reshape(B, N).cuda()
        q2, k2 = q.clone(), k.clone()
        h.cache_append(binding.PagedCache(pool[0], pool[1]), 0, k2, v, slots, length, None, rot, q2, None, k2)
        assert torch.equal(q1, q2) and torch.equal(k1, k2)
        assert torch.equal(pool[0].reshape(128, G, d)[slots], k1) and torch.equal(pool[1].reshape(128, G, d)[slots], v)


@pytest.mark.parametrize("L,B,R,G,d,page,W,dtype,layout,how", [
    (1, 1, 1, 1, 64, 16, 1, BF, "nhd", "all"),
    (3, 2, 9, 2, 128, 16, 5, BF, "nhd", "path"),
    (2, 5, 16, 3, 64, 8, 9, HF, "hnd", "path"),
    (2, 2, 70, 8, 128, 1, 70, HF, "nhd", "all"),
    (1, 3, 300, 1, 64, 64, 300, BF, "hnd", "count"),
])
def test_commit_into_four_bits(binding, L, B, R, G, d, page, W, dtype, layout, how):
    rng, gen = np.random.default_rng(L + B + R), torch.Generator().manual_seed(L + B + R)
    pages = -(-B * W // page) + 3
    c = Cached(binding, gen, L, pages, page, G, d, dtype, 4, layout)
    kv = torch.randn((L, B, R, 2, G, d), generator=gen)
    kv = (kv * torch.exp2(torch.randint(-14, 12, (L, B, R, 2, G, 1), generator=gen).float())).to(dtype)
    slots = rng.permutation(pages * page)[: B * W].reshape(B, W).astype(np.int64)
    if how != "all":
        slots[rng.random((B, W)) < 0.1] = -1
        slots[0, 0] = pages * page
    row = rng.integers(-1, R + 1, (B, W)).astype(np.int32) if how == "path" else None
    count = rng.integers(0, W + 2, B).astype(np.int32) if how != "all" else None
    dev = kv.cuda()
    handle(binding, B, tree(1)).cache_commit(c.cache, dev[:, :, :, 0], dev[:, :, :, 1], torch.from_numpy(slots).cuda(), None if row is None else torch.from_numpy(row).cuda(),
                                             None if count is None else torch.from_numpy(count).cuda())
    for b in range(B):
        for j in range(W if count is None else min(W, int(count[b]))):
            s, r = int(slots[b, j]), j if row is None else int(row[b, j])
            if 0 <= s < pages * page and 0 <= r < R:
                for l in range(L):
                    c.put(l, s // page, s % page, kv[l, b, r, 0].double(), kv[l, b, r, 1].double())
    c.check()


@pytest.mark.parametrize("dtype", [BF, HF])
def test_every_value_into_four_bits(binding, dtype):
    """All finite numbers of the type beside others of their size, borders of scales and elements, and blocks with what is no finite number."""
    lo = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(dtype)
    lo = lo[torch.isfinite(lo)]
    lo = torch.cat([lo, torch.zeros(-len(lo) % 4096, dtype=dtype)])
    x = lo[torch.argsort(lo.double().abs(), stable=True)].reshape(-1, 64, 64).transpose(1, 2).reshape(-1, 64)   # blocks of neighbours in size, and of many sizes
    x = torch.cat([x, lo.reshape(-1, 64), lo.reshape(64, -1).t().reshape(-1, 64)])
    n = x.shape[0]
    c = Cached(binding, torch.Generator().manual_seed(3), 1, n // 16, 16, 1, 64, dtype, 4, "nhd")
    h = handle(binding, 1, tree(1))
    k, v = x.reshape(1, 1, n, 1, 64), x.flip(0).reshape(1, 1, n, 1, 64)
    h.cache_commit(c.cache, k.cuda(), v.cuda(), torch.arange(n, device="cuda")[None])
    for i, y in enumerate((k, v)):
        p, s = serveref4.pack(y.reshape(1, n // 16, 16, 1, 64), dtype)
        c.want[i], c.want[i + 2] = p, s
        # a zero's sign may be lost nowhere, and nothing passes the type's range
        assert bool(torch.isfinite(serveref4.unpack(p, s, dtype)).all())
    c.check()
    bad = torch.ones((1, 1, 16, 1, 64), dtype=dtype)
    bad[0, 0, 0, 0, 3], bad[0, 0, 1, 0, 40], bad[0, 0, 2, 0, 63] = float("inf"), float("nan"), -float("inf")
    h.cache_commit(c.cache, bad.cuda(), bad.cuda(), torch.arange(16, device="cuda")[None])
    s = c.gpu[2][0, 0, :, 0].cpu()
    want = torch.full((16, 2), serveref4.scale_of(1.0, dtype), dtype=torch.uint8)
    want[0, 0] = want[1, 1] = want[2, 1] = 255
    assert torch.equal(s, want)
    out = [torch.zeros((1, 1, 16, 1, 64), dtype=dtype, device="cuda") for _ in range(2)]
    h.cache_read(c.cache, torch.zeros((1, 1), **I32), *out)
    nan = torch.isnan(out[0][0, 0, :, 0].cpu()).reshape(16, 2, 32)
    assert torch.equal(nan.all(2), want == 255) and torch.equal(nan.any(2), want == 255)


@pytest.mark.parametrize("L,first,layers,G,d,page,dtype,bits,layout,counts,starts,R", [
    (1, 0, 1, 1, 64, 16, BF, 4, "nhd", [1], None, 1),
    (3, 1, 2, 2, 128, 16, HF, 4, "hnd", [40, 0, 99], [0, 3, 17], 40),
    (2, 0, 2, 3, 64, 8, BF, 16, "nhd", [7, -1], [5, 0], 7),
    (1, 0, 1, 8, 128, 64, BF, 4, "nhd", None, [0, 100], 90),
    (2, 1, 1, 4, 128, 1, HF, 16, "hnd", [33, 20], None, 33),
    (1, 0, 1, 2, 64, 32, HF, 4, "nhd", [64, 64, 64], [-3, 90, 2 ** 31 - 5], 64),
])
def test_read(binding, L, first, layers, G, d, page, dtype, bits, layout, counts, starts, R):
    seed = L + G + d + R
    rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    B, pages = len(counts or starts), 12
    c = Cached(binding, gen, L, pages, page, G, d, dtype, bits, layout)
    if bits == 4:                                            # blocks that are NaN too
        for i in (2, 3):
            c.want[i][torch.rand(c.want[i].shape, generator=gen) < 0.05] = 255
            c.gpu[i].copy_(c.want[i])
    width = 5
    table = rng.integers(0, pages, (B, width)).astype(np.int32)
    table[0, width - 1], table[-1, 1] = -1, pages            # pages outside the cache
    kv = torch.full((layers, B, R, 2, G, d), 3.0, dtype=dtype)
    dev = kv.cuda()
    handle(binding, B, tree(1)).cache_read(c.cache, torch.from_numpy(table).cuda(), dev[:, :, :, 0], dev[:, :, :, 1], None if counts is None else torch.tensor(counts, **I32),
                                           None if starts is None else torch.tensor(starts, **I32), first)
    for b in range(B):
        for j in range(R if counts is None else min(max(counts[b], 0), R)):
            t = (starts[b] if starts else 0) + j
            p = int(table[b, t // page]) if 0 <= t < width * page else -1
            for i in range(2):
                kv[:, b, j, i] = c.values(i)[first:first + layers, p, t % page] if 0 <= p < pages else 0.0
    got = dev.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(kv)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(kv))


# ---- attention --------------------------------------------------------------------------------------------------------------

class Attn4(Attn):
    """The same calls over the cache in 4 bits; the plain implementation has the numbers that it stands for."""

    def __init__(self, *a, **kw):
        super().__init__(*a, **kw)
        self.hold()

    def hold(self):
        """The pools as they are now into 4 bits and back."""
        dtype = self.q.dtype
        self.four = [serveref4.pack(x.contiguous(), dtype) for x in (self.kp, self.vp)]
        self.kp, self.vp = (serveref4.unpack(p, s, dtype) for p, s in self.four)

    def on_gpu(self, device="cuda:0"):
        layout, self.layout = self.layout, "nhd"
        a = super().on_gpu(device)
        self.layout = layout
        (k, ks), (v, vs) = self.four
        if layout == "nhd":
            k, v, ks, vs = (x.to(device) for x in (k, v, ks, vs))
        else:
            k, v, ks, vs = (x.transpose(2, 3).contiguous().to(device).transpose(2, 3) for x in (k, v, ks, vs))
        a["cache"] = self.binding.PagedCache(k, v, ks, vs, self.q.dtype)
        return a


@pytest.mark.parametrize("case", [
    # lengths, N, query heads, kv heads, d, page, type, share of drafted nodes, layout, fused
    ([0], 1, 1, 1, 64, 16, BF, 1.0, "nhd", False),
    ([1], 1, 4, 1, 128, 16, HF, 1.0, "nhd", False),
    ([0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 400], 1, 8, 2, 128, 8, BF, 1.0, "hnd", True),
    ([15, 16, 17, 0, 255, 256, 257], 1, 28, 4, 64, 16, HF, 1.0, "nhd", False),
    ([37], 16, 14, 2, 64, 16, HF, 0.8, "nhd", False),
    ([0, 5], 2, 6, 3, 128, 32, BF, 1.0, "nhd", True),
    ([100, 3, 64], 9, 3, 1, 128, 64, BF, 0.7, "hnd", False),
    ([70, 0, 500], 9, 28, 4, 64, 8, HF, 0.6, "nhd", True),
    ([129, 1000], 16, 28, 4, 128, 16, BF, 0.9, "nhd", True),
    ([1, 320, 64, 77], 16, 16, 8, 64, 128, BF, 0.5, "hnd", False),
    ([200, 63], 33, 8, 2, 128, 16, HF, 0.8, "nhd", False),
    ([200, 63, 0, 129], 33, 2, 2, 64, 16, BF, 0.8, "nhd", False),
    ([300, 0, 1], 64, 7, 1, 128, 64, BF, 0.75, "nhd", True),
    ([90, 444], 64, 8, 2, 64, 1, HF, 1.0, "nhd", False),
    ([65, 0], 130, 4, 2, 64, 16, BF, 0.5, "hnd", True),
    ([65, 10], 130, 16, 2, 128, 16, HF, 1.0, "nhd", False),
    ([50, 0, 700], 32, 5, 1, 128, 4096, BF, 0.97, "nhd", False),
], ids=lambda c: "len%s-N%d-%dx%d-d%d-p%d-%s" % (c[0][-1], c[1], c[2], c[3], c[4], c[5], "f16" if c[6] is HF else "bf16"))
def test_attention(binding, case):
    lens, N, H, G, d, page, dtype, share, layout, fused = case
    Attn4(binding, 1 + sum(lens) + N, lens, N, H, G, d, page, dtype, share, layout, fused).check()


@pytest.mark.parametrize("N,H,G,d,dtype,lens", [
    (1, 8, 2, 128, BF, [9000]),
    (1, 4, 1, 64, HF, [20000, 3]),
    (16, 7, 1, 128, HF, [6000, 0, 17]),
    (33, 8, 1, 64, BF, [3001]),
    (33, 2, 1, 128, BF, [5003, 64]),                         # the form of up to 64 rows
    (33, 1, 1, 64, HF, [5003, 1]),
])
def test_attention_of_long_caches(binding, N, H, G, d, dtype, lens):
    Attn4(binding, 7 + N, lens, N, H, G, d, 16, dtype, 0.6).check()


def test_attention_of_one_layer_of_many(binding):
    Attn4(binding, 3, [70, 33], 9, 4, 2, 64, 16, BF, layers=3, layer=2, layout="hnd").check()
    Attn4(binding, 4, [70, 33], 9, 4, 2, 128, 16, HF, layers=3, layer=1).check()


@pytest.mark.parametrize("spread", [0.0, 40.0])
def test_attention_of_flat_and_of_steep_scores(binding, spread):
    Attn4(binding, 5, [700, 30], 16, 4, 2, 128, 16, BF, spread=spread).check()
    Attn4(binding, 6, [700, 30], 16, 4, 2, 64, 16, HF, spread=spread / 4).check()


@pytest.mark.parametrize("d,dtype,size", [(64, BF, 2.0 ** 100), (128, BF, 2.0 ** -100), (64, HF, 2.0 ** 11), (128, HF, 2.0 ** -17)])
def test_attention_of_large_and_small_scales(binding, d, dtype, size):
    """Scales at both ends of what they may be, and blocks of one head of very different ones."""
    t = Attn4(binding, 9, [300, 31], 16, 4, 2, d, 16, dtype)
    t.kp[..., 32:] *= 2.0 ** -6
    t.vp *= size
    t.vp[..., :32] *= 2.0 ** 3
    t.v *= size
    t.hold()
    t.check()


@pytest.mark.parametrize("N,d,dtype", [(16, 128, BF), (64, 64, HF), (1, 128, HF), (33, 64, BF)])
def test_attention_never_uses_what_is_masked(binding, N, d, dtype):
    """NaN in undrafted nodes, behind the lengths and in pages of nobody; a block of NaN in a cached value and in a cached key."""
    t = Attn4(binding, 11, [33, 70, 0, 128], N, 8 if N != 33 else 2, 2, d, 16, dtype, 0.6 if N > 1 else 1.0)
    used = torch.zeros((t.pages, t.page), dtype=torch.bool)
    for b, n in enumerate(t.lens):
        for p in range(n):
            used[t.table[b, p // t.page], p % t.page] = True
    for _, s in t.four:
        s[0][~used] = 255
    gone = torch.from_numpy(t.tok) < 0
    for x in (t.q, t.k, t.v):
        x[gone] = float("nan")
    t.check()
    want, tol = t.want()
    per = t.q.shape[2] // 2
    t.four[1][1][0, t.table[1, 3], 2, 0, 1] = 255            # token 50 of the second one, head 0: values 32 .. 63
    t.four[0][1][0, t.table[3, 7], 15, 1, 0] = 255           # the last token of the fourth one, head 1: the key
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    there = torch.from_numpy(t.tok) >= 0
    assert bool(torch.isnan(got[1, :, :per, 32:64][there[1]]).all()) and bool(torch.isnan(got[3, :, per:][there[3]]).all())
    clean = torch.ones(got.shape, dtype=torch.bool)
    clean[1, :, :per, 32:64] = False
    clean[3, :, per:] = False
    assert bool(((got - want).abs() <= tol)[clean].all())


def test_attention_pages_outside_the_cache_and_odd_lengths_are_not_read(binding):
    t = Attn4(binding, 12, [64, 64], 9, 4, 2, 64, 16, BF, 1.0)
    a = t.on_gpu()
    a["length"] = torch.tensor([10 ** 9, -5], **I32)
    a["table"] = torch.tensor(t.table.clip(0, t.pages - 1), **I32)
    got = t.h.tree_attention(**a)
    t.table, t.lens = t.table.clip(0, t.pages - 1), [t.width * t.page, 0]
    t.check(got)
    a["table"] = torch.where(torch.arange(t.width, device="cuda") % 2 == 0, a["table"], torch.tensor(2 ** 31 - 1, **I32))
    got = t.h.tree_attention(**a)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(got).all())


def test_attention_on_another_stream_and_twice_at_once(binding):
    ts = [Attn4(binding, 20 + i, [300 + 100 * i, 9], 16, 8, 2, 128, 16, BF) for i in range(2)]
    args = [t.on_gpu() for t in ts]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ts]
    got = [[], []]
    for rep in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(ts[i].h.tree_attention(**args[i]))
    torch.cuda.synchronize()
    for t, many in zip(ts, got):
        for g in many:
            t.check(g)


def test_attention_gives_the_same_bits_again(binding):
    for N, H, lens in ((16, 8, [5000, 40]), (1, 8, [7000, 0, 300])):
        t = Attn4(binding, 31, lens, N, H, 2, 128, 16, BF)
        a = t.on_gpu()
        one = t.h.tree_attention(**a)
        for _ in range(3):
            assert torch.equal(one, t.h.tree_attention(**a))


@pytest.mark.parametrize("B,N,H,G,d,dtype", [(40, 70, 1, 1, 64, HF), (260, 9, 3, 1, 128, HF), (70, 33, 1, 1, 128, BF), (100, 1, 4, 4, 64, BF)])
def test_attention_of_many_trees(binding, B, N, H, G, d, dtype):
    lens = [int(x) for x in np.random.default_rng(B + N).integers(0, 150, B)]
    Attn4(binding, 250 + B + N, lens, N, H, G, d, 16, dtype, 0.5).check()


@pytest.mark.parametrize("N,H,G,d,dtype,share", [(300, 3, 3, 128, HF, 1.0), (1024, 1, 1, 128, BF, 1.0), (1024, 2, 2, 64, BF, 0.6)])
def test_attention_of_large_trees(binding, N, H, G, d, dtype, share):
    Attn4(binding, 260 + N + H, [170, 0], N, H, G, d, 16, dtype, share).check()


@pytest.mark.parametrize("d,dtype,N", [(64, BF, 9), (128, HF, 9), (64, HF, 64), (128, BF, 64)])
def test_scales_in_another_order_than_their_blocks(binding, d, dtype, N):
    """Blocks as [page, place, head], scales as [page, head, place] with room between pages: one's place is not the other's."""
    t = Attn4(binding, 280 + N + d, [300, 0, 77], N, 4, 2, d, 16, dtype, 0.8)
    a = t.on_gpu()
    c = a["cache"]

    def moved(s):
        layers, pages, page, G, n = s.shape
        room = torch.full((layers, pages + 1, G + 1, page, n), 255, dtype=torch.uint8, device="cuda")
        room[:, :pages, :G] = s.transpose(2, 3)
        return room[:, :pages, :G].transpose(2, 3)

    other = binding.PagedCache(c.k, c.v, moved(c.k_scale), moved(c.v_scale), dtype)
    out = t.h.tree_attention(**dict(a, cache=other))
    t.check(out)
    drafted = torch.from_numpy(t.tok).cuda() >= 0
    assert torch.equal(out[drafted], t.h.tree_attention(**a)[drafted])


@pytest.mark.parametrize("d,dtype,N", [(64, BF, 1), (128, HF, 16), (128, BF, 64)])
def test_places_far_into_a_cache(binding, d, dtype, N):
    """Pages 9 GiB apart, their scales nearly 2: places past 2^32 bytes and 2^31 heads' scales, for rows that come and rows that are read."""
    t = Attn4(binding, 270 + N, [64, 33], N, 4, 2, d, 16, dtype, 1.0)
    page, G = 16, 2
    t.pages = 5
    t.kp, t.vp = t.kp[:, :5].contiguous(), t.vp[:, :5].contiguous()
    t.hold()
    t.table[0, :4], t.table[1, :3] = [4, 1, 0, 3], [4, 2, 3]
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("needs 50 GiB of device memory")

    def spread(e, apart):
        flat = torch.empty(4 * apart + 2 * page * G * e, dtype=torch.uint8, device="cuda")
        return [flat.as_strided((1, 5, page, G, e), (128, apart, G * e, e, 1), i * page * G * e) for i in range(2)]

    k, v = spread(d // 2, 9 << 30)
    ks, vs = spread(d // 32, (2 << 30) - 4096)
    cache = binding.PagedCache(k, v, ks, vs, dtype)
    slots = torch.arange(5 * page, dtype=torch.int64, device="cuda").flip(0).contiguous()[None]
    rows = [x.cuda().reshape(1, 1, 5 * page, G, d) for x in (t.kp, t.vp)]
    one = handle(binding, 1, tree(1))
    one.cache_commit(cache, rows[0], rows[1], slots, slots.int())
    for got, (p, s) in zip(((k, ks), (v, vs)), t.four):
        assert torch.equal(serveref4.unpack(got[0].cpu(), got[1].cpu(), dtype), serveref4.unpack(p, s, dtype))
    t.check(t.h.tree_attention(**dict(t.on_gpu(), cache=cache)))
    back = [torch.empty((1, 1, 4 * page, G, d), dtype=dtype, device="cuda") for _ in range(2)]
    one.cache_read(cache, torch.tensor([[4, 1, 0, 3]], **I32), *back)
    for got, x in zip(back, (t.kp, t.vp)):
        assert torch.equal(got.cpu()[0, 0], x[0][[4, 1, 0, 3]].reshape(4 * page, G, d))
    one.cache_append(cache, 0, rows[0][0], rows[1][0], slots)
    one.cache_read(cache, torch.tensor([[0, 2, 4]], **I32), *(x[:, :, :48] for x in back))
    for got, x in zip(back, (t.kp, t.vp)):
        assert torch.equal(got.cpu()[0, 0, :48], x.reshape(80, G, d).flip(0)[list(range(16)) + list(range(32, 48)) + list(range(64, 80))])


# ---- refusals, devices, together ----------------------------------------------------------------------------------------------

def test_refusals(binding):
    t = Rotate(binding, 8, [5, 4], 9, 4, 2, 64, BF, 64)
    a = t.args()
    c = Cached(binding, torch.Generator().manual_seed(1), 2, 4, 16, 2, 64, BF, 4, "nhd")
    v, slots = a["k"].clone(), torch.zeros((2, 9), dtype=torch.int64, device="cuda")
    q0, k0 = a["q"].clone(), a["k"].clone()
    bad = (binding.StandError, AssertionError, TypeError)

    def rotate(**kw):
        with pytest.raises(bad):
            t.h.tree_rotate(**dict(a, **kw))

    def append(cache=c.cache, layer=0, k=a["k"], v=v, s=slots, **kw):
        with pytest.raises(bad):
            t.h.cache_append(cache, layer, k, v, s, **kw)

    short = binding.Rotation(serveref4.turns(9, 24).cuda())
    wide = binding.Rotation(serveref4.turns(9, 80).cuda())
    half = binding.Rotation(None, "halves", torch.ones(64, dtype=HF, device="cuda"))
    for r in (short, wide, half, binding.Rotation(None, "halves", torch.ones(128, dtype=BF, device="cuda")), binding.Rotation(a["rotation"].turns, eps=-1.0, q_norm=torch.ones(64, dtype=BF, device="cuda"))):
        rotate(rotation=r)
        append(rotation=r)
    rotate(k=a["k"].half())
    rotate(k=a["k"][:, :5])
    rotate(length=a["length"].long())
    rotate(draft_tok=a["draft_tok"][:, :5].contiguous())
    rotate(q=a["q"][:, :, :, :32])
    rotate(q_out=torch.empty((2, 9, 5, 64), dtype=BF, device="cuda"))
    rotate(q_out=torch.empty((2, 9, 4, 64), dtype=HF, device="cuda"))
    rotate(k=a["k"][:, :, :1].expand(2, 9, 2, 64))           # in place, but one head for both
    rotate(q_out=torch.empty((2, 1, 4, 64), dtype=BF, device="cuda").expand(2, 9, 4, 64))
    append(k_out=torch.empty((1, 9, 2, 64), dtype=BF, device="cuda").expand(2, 9, 2, 64))
    append(layer=2)
    append(layer=-1)
    append(k=a["k"].half())
    append(k=a["k"][:, :, :1])
    append(v=v.half())
    append(s=slots[:, :5].contiguous())
    append(s=slots.int())
    append(count=torch.zeros(2, dtype=torch.int64, device="cuda"))
    append(start=torch.zeros(3, **I32))
    out = [torch.zeros((2, 2, 9, 2, 64), dtype=BF, device="cuda") for _ in range(2)]
    table = torch.zeros((2, 3), **I32)
    for kw in (dict(layer=1), dict(layer=-1), dict(k=out[0].half()), dict(v=out[0][:, :, :5]), dict(table=table.long()), dict(table=table[:1]), dict(count=torch.zeros(3, **I32)),
               dict(k=torch.zeros((3, 2, 9, 2, 64), dtype=BF, device="cuda"), v=torch.zeros((3, 2, 9, 2, 64), dtype=BF, device="cuda"))):
        with pytest.raises(bad):
            t.h.cache_read(**dict(dict(cache=c.cache, table=table, k=out[0], v=out[1]), **kw))
    p = c.gpu
    for wrong in ((p[0], p[1], p[2]), (p[0], p[1], p[2], p[3]), (p[0], p[1], p[2][..., :1], p[3][..., :1], BF), (p[0], p[1], p[2], p[3], torch.float32), (p[0].int(), p[1].int(), p[2], p[3], BF)):
        with pytest.raises(bad):
            binding.PagedCache(*wrong)
    odd = torch.zeros((2, 4, 16, 2, 40), dtype=torch.uint8, device="cuda")[..., :32]      # heads 40 bytes apart
    with pytest.raises(bad):
        t.h.cache_append(binding.PagedCache(odd, odd, p[2], p[3], BF), 0, a["k"], v, slots)
    torch.cuda.synchronize()
    c.check()
    assert torch.equal(a["q"], q0) and torch.equal(a["k"], k0) and all(bool((o == 0).all()) for o in out)


@pytest.mark.parametrize("dtype,d,norm", [(BF, 128, True), (HF, 64, False)])
def test_together_eagerly_and_as_a_graph(binding, dtype, d, norm):
    """Prompts are appended, then trees are rotated, attended and committed, step by step; lengths, pages and accepted nodes are on the
    GPU alone.  A dense cache on the CPU is kept beside it.  The captured step is replayed between eager ones."""
    gen, rng = torch.Generator().manual_seed(d), np.random.default_rng(d)
    B, H, G, N, L, page, P, width = 3, 4, 2, 9, 2, 8, 60, 16
    parent = tree(N)
    h = handle(binding, B, parent)
    depth = torch.from_numpy(serveref.depths(parent))
    W = h.W
    cache = binding.PagedCache.new4(L, P, page, G, d, dtype)
    pages = binding.Pages.new(B, P, page, width)
    turns, w = serveref4.turns(200, d), norm_weights(gen, d, dtype, (norm, norm))
    rot = binding.Rotation(turns.cuda(), "halves", *(cuda(x) for x in w))
    # the prompts
    lens = [11, 1, 24]
    n, R = torch.tensor(lens, **I32), max(lens)
    slots = torch.zeros((B, R), dtype=torch.int64, device="cuda")
    assert not h.cache_pages(pages, None, n, slots).any()
    kept = [[[], []] for _ in range(L)]                      # [layer][k | v]: dense, in 4 bits and back
    for l in range(L):
        qkv = torch.randn((B, R, H + 2 * G, d), generator=gen).to(dtype)
        dev = qkv.cuda()
        h.cache_append(cache, l, dev[:, :, H:H + G], dev[:, :, H + G:], slots, pages.length, n, rot, dev[:, :, :H])
        yk = serveref4.turned(qkv[:, :, H:H + G], torch.arange(R).expand(B, R), turns, "halves", w[1], 1e-6).float()
        for i, x in enumerate((yk, qkv[:, :, H + G:])):
            x = serveref4.unpack(*serveref4.pack(x, dtype), dtype)
            kept[l][i] = [[x[b, j] for j in range(lens[b])] for b in range(B)]
    out_len, out_node = n.clone(), torch.zeros((B, W), **I32)
    tok = torch.full((B, N), -1, **I32)
    qkv = torch.zeros((L, B, N, H + 2 * G, d), dtype=dtype, device="cuda")
    out = torch.zeros((L, B, N, H, d), dtype=dtype, device="cuda")
    tslots, back = torch.zeros((B, W), dtype=torch.int64, device="cuda"), torch.zeros((2, L, B, 60, G, d), dtype=dtype, device="cuda")
    node, count = torch.zeros((B, W), **I32), torch.zeros(B, **I32)

    def step():
        h.cache_pages(pages, out_len, None, tslots)
        for l in range(L):
            q, k, v = qkv[l, :, :, :H], qkv[l, :, :, H:H + G], qkv[l, :, :, H + G:]
            h.tree_rotate(rot, pages.length, tok, q, k)
            h.tree_attention(cache, l, pages.length, pages.table, tok, q, k, v, out=out[l])
        h.cache_commit(cache, qkv[..., H:H + G, :], qkv[..., H + G:, :], tslots, node, count)
        out_len.copy_(count)
        h.cache_read(cache, pages.table, back[0], back[1], pages.length)

    def one(run):
        x = torch.randn(qkv.shape, generator=gen).to(dtype)
        t = drafts(rng, B, parent, 0.8)
        t[:, 0] = 3
        leaf = [max(u for u in range(N) if t[b, u] >= 0) for b in range(B)]
        path = [serveref.path(parent, u)[::-1] for u in leaf]
        node.copy_(torch.tensor([p + [-1] * (W - len(p)) for p in path]))
        count.copy_(torch.tensor([len(p) for p in path]))
        qkv.copy_(x)
        tok.copy_(torch.from_numpy(t))
        run()
        torch.cuda.synchronize()
        now = [len(r) for r in kept[0][0]]
        assert pages.length.tolist() == now
        most = max(now) + 1
        drafted = torch.from_numpy(t) >= 0
        pos = torch.tensor(now)[:, None] + depth
        for l in range(L):
            q, k = (serveref4.turned(y, pos, turns, "halves", u, 1e-6) for y, u in ((x[l, :, :, :H], w[0]), (x[l, :, :, H:H + G], w[1])))
            gq, gk = qkv[l, :, :, :H].cpu(), qkv[l, :, :, H:H + G].cpu()
            assert bool(((gq.double() - q).abs() <= serveref4.turned_error(q, dtype))[drafted].all())
            assert bool(((gk.double() - k).abs() <= serveref4.turned_error(k, dtype))[drafted].all())
            flat = torch.zeros((2, B, most, G, d), dtype=dtype)
            for i in range(2):
                for b in range(B):
                    for j, r in enumerate(kept[l][i][b]):
                        flat[i, b, j] = r
                    assert torch.equal(back[i, l, b, :now[b]].cpu(), flat[i, b, :now[b]])
            want, tol = serveref.attention(parent, now, torch.arange(B)[:, None], tok.cpu(), gq, gk, x[l, :, :, H + G:], flat[0], flat[1], d ** -0.5)
            assert bool(((out[l].cpu().double() - want).abs() <= tol).all())
            for b in range(B):
                for u in path[b]:
                    for i, y in enumerate((gk[b, u], x[l, b, u, H + G:])):
                        kept[l][i][b].append(serveref4.unpack(*serveref4.pack(y, dtype), dtype))

    one(step)
    one(step)
    torch.cuda.synchronize()
    state = [y.clone() for y in (pages.table, pages.ring, pages.length, pages.held, pages.mark, out_len, cache.k, cache.v, cache.k_scale, cache.v_scale)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.synchronize()
    for y, s in zip((pages.table, pages.ring, pages.length, pages.held, pages.mark, out_len, cache.k, cache.v, cache.k_scale, cache.v_scale), state):
        assert torch.equal(y, s)                             # (capturing runs nothing)
    one(g.replay)
    one(step)
    one(g.replay)
    one(g.replay)

"""The operators around a verification at the ends of what their documentation allows: wide tables, extreme scores, places far
into a cache, large trees and many of them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2506_04708_amd import synth  # noqa: E402
from tests import test_serve_ops  # noqa: E402
from tests.serveref import depths as serveref_depths  # noqa: E402
from tests.test_serve_ops import BF, HF, Attn, binding, drafts, handle, tree  # noqa: E402,F401

for _n, _deep, _fan in ((20, 5, [4, 2, 2, 1]), (70, 8, [8, 4, 2, 1]), (300, 12, [8, 4, 2, 1]), (1024, 31, [8, 4, 2, 1])):
    test_serve_ops.TREES.setdefault(_n, synth.make_tree(_n, _deep, _fan).tolist())


@pytest.mark.parametrize("G,d,width", [(64, 128, 2 ** 21 + 5), (8, 128, 2 ** 21 + 5), (64, 128, 2 ** 24 + 5)])
def test_commit_of_wide_tables(binding, G, d, width):
    """Every slot of the table is a good one; only what the counts leave is copied, from the first position to the last."""
    L, B, R, pages, page = 1, 2, 4, 5, 8
    pool = [torch.randn((L, pages, page, G, d)).to(BF).cuda() for _ in range(2)]
    k, v = (torch.randn((L, B, R, G, d)).to(BF).cuda() for _ in range(2))
    slots = torch.full((B, width), 3, dtype=torch.int64, device="cuda")
    row = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    h = handle(binding, B, tree(1))
    cache = binding.PagedCache(*pool)
    for counts, at in (([0, -1], []), ([-2 ** 31, 0], []), ([2, width], [(0, 0, 2, 9), (0, 1, 0, 39), (1, 0, 3, 17), (1, width - 1, 1, 30), (1, width // 2, 0, 1)]),
                       ([1, width - 1], [(0, 0, 1, 4), (1, width - 2, 2, 12)]), ([2 ** 31 - 1, 0], [(0, width - 1, 3, 0)])):
        want = [x.clone() for x in pool]
        row.fill_(-1)
        if not at:
            row.fill_(0)                                  # all of them good rows as well
        for b, j, r, s in at:
            row[b, j], slots[b, j] = r, s
            want[0][:, s // page, s % page], want[1][:, s // page, s % page] = k[:, b, r], v[:, b, r]
        if at:                                            # behind the counts: rows that may not be copied
            for b in range(B):
                row[b, max(0, min(counts[b], width)):] = 0
        h.cache_commit(cache, k, v, slots, row, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert torch.equal(pool[0], want[0]) and torch.equal(pool[1], want[1]), counts
        for b, j, r, s in at:
            slots[b, j] = 3


def hard_attention(t):
    """(outputs, truth values [B, N, H]) of rows whose largest score is so far above the others that its value alone is the
    output: by more than twice what sums in fp32 may be off, and by 40 more, below which no weight changes a rounding."""
    B, N, H, d = t.q.shape
    per = H // t.k.shape[2]
    out, sure = torch.zeros((B, N, H, d), dtype=t.q.dtype), torch.zeros((B, N, H), dtype=torch.bool)
    for b, n in enumerate(t.lens):
        pos = torch.arange(n)
        at = torch.from_numpy(t.table[b]).long()[pos // t.page]
        for u in range(N):
            if t.tok[b, u] < 0:
                continue
            own, v = [], u
            while v >= 0:
                own.append(v)
                v = int(t.parent[v])
            for i in range(H):
                g = i // per
                K = torch.cat([t.kp[t.layer][at, pos % t.page, g], t.k[b, own, g]]).double()
                V = torch.cat([t.vp[t.layer][at, pos % t.page, g], t.v[b, own, g]])
                q = t.q[b, u, i].double()
                s = K @ q * t.scale
                off = (K.abs() @ q.abs()) * t.scale * (d + 8) * 2.0 ** -24
                top = int(s.argmax())
                rest = torch.cat([s[:top] + off[:top], s[top + 1:] + off[top + 1:]])
                out[b, u, i] = V[top]
                sure[b, u, i] = len(rest) == 0 or bool(s[top] - off[top] > rest.max() + 40)
    return out, sure


def far(t, sign, size):
    """Every product of a query and a key gets this sign and about this size; some queries are as they were."""
    root = (size / t.q.shape[3]) ** 0.5
    for x, s in ((t.q, sign), (t.k, 1.0), (t.kp, 1.0)):
        y = torch.where(x == 0, torch.ones_like(x), x.abs()).double().clamp(0.5, 1.0 if size > 1e38 else 4.0)
        x.copy_((y * root * s).to(x.dtype))
    return t


@pytest.mark.parametrize("N,H,G,lens", [(1, 4, 1, [300, 0, 3, 5000]), (16, 4, 1, [300, 0, 1]), (16, 14, 1, [700, 33, 0]), (33, 1, 1, [2000, 1])])
@pytest.mark.parametrize("d,dtype,sign,size,scale", [
    (128, BF, -1.0, 1.5e38, 1.0),      # scores are finite, and less than -1e38
    (64, BF, -1.0, 2.0e38, 1.6),       # ... also where their product with log2(e) is not
    (64, BF, 1.0, 2.0e38, 1.6),
    (128, BF, 1.0, 1e12, 1.0),         # far above what a difference of rounded products would keep inside the range
    (64, HF, -1.0, 1.6e9, 1.0),
    (128, HF, 1.0, 1.6e9, 1.0),
])
def test_attention_of_far_scores(binding, N, H, G, lens, d, dtype, sign, size, scale):
    """Scores of any size that fp32 holds: the row is that of its largest one, not NaN."""
    t = far(Attn(binding, 200 + N + H, lens, N, H, G, d, 16, dtype, 0.8 if N > 1 else 1.0), sign, size)
    t.scale = scale
    want, sure = hard_attention(t)
    drafted = torch.from_numpy(t.tok) >= 0
    assert int(sure.sum()) * 4 > int(drafted.sum()) * H
    got = t.h.tree_attention(**t.on_gpu()).cpu()
    assert bool(torch.isfinite(got).all())
    assert torch.equal(got[sure], want[sure])
    assert bool((got[~drafted] == 0).all())


def test_attention_of_far_scores_beside_ordinary_ones(binding):
    """Rows of one wave with scores of 1e9 and rows with scores of 1: the ordinary rows keep their errors."""
    for N, H, G, d, dtype in ((16, 4, 2, 128, BF), (33, 7, 1, 64, HF), (16, 2, 1, 64, HF)):
        t = Attn(binding, 230 + N, [900, 77, 0], N, H, G, d, 16, dtype, 1.0)
        t.q[:, ::3] *= 2.0 ** 13                          # (eight times 2^13 and more is infinite in fp16: such queries have no value)
        loud = t.q[:, ::3].clone()
        known = torch.isfinite(t.q).all(dim=3)
        got = t.h.tree_attention(**t.on_gpu()).cpu()
        want, sure = hard_attention(t)
        sure &= known
        assert bool(torch.isfinite(got[known]).all()) and bool(sure[:, ::3].any()) and torch.equal(got[sure], want[sure])
        t.q[:, ::3] = 0
        want, tol = t.want()
        keep = torch.arange(N) % 3 != 0
        assert bool(((got.double() - want).abs() <= tol)[:, keep].all())
        t.q[:, ::3] = loud


@pytest.mark.parametrize("N,H,G", [(1, 4, 1), (16, 4, 1), (16, 14, 1)])
def test_attention_of_extreme_scales(binding, N, H, G):
    """From the smallest number, which leaves the mean of the values, to the largest that is accepted, which leaves one of them."""
    for d, dtype in ((64, HF), (128, BF)):
        t = Attn(binding, 245 + N + H, [300, 0, 2000], N, H, G, d, 16, dtype, 0.8 if N > 1 else 1.0)
        for t.scale in (2.0 ** -149, 1e-40, 2.0 ** -126, 1e-20):
            t.check()
        t.scale = 2.0 ** 127
        want, sure = hard_attention(t)
        got = t.h.tree_attention(**t.on_gpu()).cpu()
        assert bool(sure.any()) and bool(torch.isfinite(got).all()) and torch.equal(got[sure], want[sure])


@pytest.mark.parametrize("N,H,G,lens", [(1, 4, 1, [5000, 0]), (16, 3, 1, [1500, 40, 3]), (16, 14, 1, [3000, 1])])
@pytest.mark.parametrize("d,dtype,e", [(128, BF, 20), (128, BF, 22), (64, BF, 23), (64, BF, 60), (64, HF, 21), (128, HF, 22), (64, HF, 23), (128, HF, 30)])
def test_attention_of_equal_scores_of_any_size(binding, N, H, G, lens, d, dtype, e):
    """Keys that are all the same leave the mean of the values, below the size from which maxima are taken off and above it, also
    where a row is joined from several parts; rows of both kinds and of both signs in one wave."""
    t = Attn(binding, 248 + N + H, lens, N, H, G, d, 16, dtype, 0.8 if N > 1 else 1.0)
    t.scale = 1.0
    for x in (t.k, t.kp):
        x.fill_(2.0 ** (e // 2 - 3))
    t.q.fill_(2.0 ** (e - e // 2 + 3) / d)                 # scores of 2^e exactly, some of -2^e, 3 * 2^e and 1
    t.q[:, ::3] *= -1
    t.q[:, 1::4] *= 3
    t.q[:, 2::5] *= 2.0 ** -e if dtype is BF else 2.0 ** -10
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    half = 2.0 ** -8 if dtype is BF else 2.0 ** -11
    for b, n in enumerate(lens):
        pos = torch.arange(n)
        V = t.vp[0][torch.from_numpy(t.table[b]).long()[pos // 16], pos % 16].double()
        for u in range(N):
            if t.tok[b, u] < 0:
                continue
            own, v = [], u
            while v >= 0:
                own.append(v)
                v = int(t.parent[v])
            for i in range(H):
                all_v = torch.cat([V[:, i // (H // G)], t.v[b, own, i // (H // G)].double()])
                mean = all_v.mean(0)
                # equal weights: sums of so many terms in fp32, parts joined, one quotient and the rounding of the result
                tol = all_v.abs().mean(0) * (len(all_v) + 64) * 2.0 ** -24 * 2 + mean.abs() * half + (2.0 ** -25 if dtype is HF else 0)
                assert bool(((got[b, u, i] - mean).abs() <= tol).all()), (b, u, i)


@pytest.mark.parametrize("size", [2 ** 15, 2 ** 20, 2 ** 21 + 2 ** 20, -(2 ** 21) - 2 ** 20, 2907264, 2907272, -2907264, -2907272, 2 ** 22 + 2 ** 21])
@pytest.mark.parametrize("N,H,G,n", [(1, 1, 1, 700), (16, 1, 1, 700), (1, 4, 1, 9000), (16, 3, 1, 700), (16, 14, 1, 700), (16, 14, 1, 9000)])
def test_attention_raises_its_maximum_exactly(binding, N, H, G, n, size):
    """Many keys of one score and then one of six more, exact numbers both: what the sums so far are scaled by is as exact as a
    weight, whatever the size of the scores (2^22 / log2(e) lies between two of them)."""
    for d, dtype in ((64, BF), (128, HF)):
        t = Attn(binding, 285 + N + H, [n], N, H, G, d, 16, dtype, 1.0)
        t.scale = 1.0
        sign, whole, rest = (1 if size > 0 else -1), abs(size) >> 9, abs(size) & 511
        parts = [whole >> 9, whole & 511]                  # |size| = 512 * (512 * parts[0] + parts[1]) + rest
        for x in (t.q, t.k, t.kp, t.v, t.vp):
            x.zero_()
        t.q[..., 0], t.q[..., 1], t.q[..., 2], t.q[..., 3], t.q[..., 4] = 512.0, 512.0, 1.0, 2.0, 1.0
        for x in (t.k, t.kp):
            for e, (y, by) in enumerate(((parts[0], 512), (parts[1], 1))):
                x[..., e] = sign * float(y) * by           # (whole numbers of at most eight bits, times powers of two: exact in both types)
            x[..., 2], x[..., 3] = sign * float(rest & 255), sign * float(rest >> 8) * 128.0
        assert float(t.kp[0, 0, 0, 0, :5].double() @ t.q[0, 0, 0, :5].double()) == size
        t.vp[..., :] = 1.0
        t.v[..., :] = 1.0
        last = (t.table[0, (n - 1) // 16], (n - 1) % 16)
        t.kp[0][last][:, 4] = 6.0
        t.vp[0][last] = 0.0
        deep = serveref_depths(t.parent)
        got = t.h.tree_attention(**t.on_gpu()).cpu().double()
        many = torch.tensor(n - 1 + deep + 1.0)[None, :, None, None]      # keys of the one score: the cache's and the path's
        want = many / (many + np.exp(6.0))
        # a weight of either kind is off by half a step, the exponent by a rounding of the difference and c's own (six of 2^-24)
        half = 2.0 ** -8 if dtype is BF else 2.0 ** -11
        tol = want * (1 - want) * 2 * half + want * (half + (n + 64) * 2.0 ** -23)
        assert bool(((got - want).abs() <= tol).all()), (float(got.min()), float(got.max()), float(want.min()), float(want.max()))


@pytest.mark.parametrize("N,H,G", [(1, 4, 1), (16, 4, 1), (16, 14, 1)])
def test_attention_scores_that_are_minus_infinity_count_for_nothing(binding, N, H, G):
    """Keys of minus infinity leave a row to the others; a row that has no other is NaN, as is one with an infinite score."""
    t = Attn(binding, 240 + N + H, [200, 40, 0], N, H, G, 64, 16, BF, 1.0)
    t.q.copy_(t.q.abs() + 0.25)
    want, tol = t.want()
    used = [(t.table[0, p // 16], p % 16) for p in range(0, 200)]
    for a, p in used[:150]:                               # whole stages and parts of one
        t.kp[0][a, p] = float("-inf")
    want, tol = (x.clone() for x in (want, tol))
    s = t.lens
    t.lens = [50, 40, 0]
    table, t.table = t.table, t.table.copy()
    keep = used[150:]
    K = torch.stack([t.kp[0][a, p] for a, p in keep])
    V = torch.stack([t.vp[0][a, p] for a, p in keep])
    kp, vp = t.kp, t.vp
    t.kp, t.vp = t.kp.clone(), t.vp.clone()
    for i in range(50):
        t.kp[0][t.table[0, i // 16], i % 16], t.vp[0][t.table[0, i // 16], i % 16] = K[i], V[i]
    want, tol = t.want()
    t.kp, t.vp, t.table, t.lens = kp, vp, table, s
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    assert bool(((got - want).abs() <= tol).all())
    t.k[1, 0] = float("inf")                              # the root's key: every row of that trajectory sees it
    t.k[2] = float("-inf")                                # nothing but the tree, and nothing of it counts
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    assert bool(((got - want).abs() <= tol)[0].all()) and bool(torch.isnan(got[1:]).all())


def test_attention_workspaces_of_refused_calls_have_no_size(binding):
    """0 bytes say that the call would be refused: a caller can ask before it has any queries."""
    h, many = handle(binding, 2, tree(9)), handle(binding, 4097, tree(1))
    x = torch.zeros((1, 4, 16, 2, 64), dtype=BF, device="cuda")
    cache = binding.PagedCache(x, x)
    size = h._lib.stand_tree_attention_work
    assert size(h.h, cache.ref, 4) > 0 and size(h.h, cache.ref, 65534) > 0
    assert size(h.h, cache.ref, 65536) == 0 and size(h.h, cache.ref, 3) == 0 and size(h.h, cache.ref, 0) == 0 and size(None, cache.ref, 4) == 0
    assert size(many.h, cache.ref, 4) == 0 and size(h.h, None, 4) == 0
    cache.desc.page_stride, cache.desc.pages = 2 ** 40, 2 ** 20
    assert size(h.h, cache.ref, 4) == 0


@pytest.mark.parametrize("B,N,H,G,d,dtype", [
    (20, 70, 1, 1, 64, BF), (20, 70, 2, 1, 128, HF),     # drafted nodes counted eight trajectories at a time
    (40, 70, 1, 1, 64, HF), (100, 70, 1, 1, 128, BF),    # ... and sixteen, more of them than a wave has lanes
    (90, 20, 1, 1, 64, BF), (260, 9, 3, 1, 128, HF),     # several trajectories in a wave, in many turns
    (70, 33, 1, 1, 128, BF), (70, 33, 1, 1, 64, HF),     # the form of up to 64 rows
])
def test_attention_of_many_trees(binding, B, N, H, G, d, dtype):
    lens = [int(x) for x in np.random.default_rng(B + N).integers(0, 50, B)]
    Attn(binding, 250 + B + N, lens, N, H, G, d, 16, dtype, 0.5).check()


@pytest.mark.parametrize("N,H,G,d,dtype,share", [
    (300, 2, 1, 64, BF, 0.7), (300, 3, 3, 128, HF, 1.0), (1024, 1, 1, 128, BF, 1.0), (1024, 2, 1, 64, HF, 0.9), (1024, 2, 2, 64, BF, 0.6),
])
def test_attention_of_large_trees(binding, N, H, G, d, dtype, share):
    """The longest lists of nodes, with NaN in the nodes that were not drafted and values that are not finite in leaves."""
    t = Attn(binding, 260 + N + H, [70, 0], N, H, G, d, 16, dtype, share)
    if share < 1:
        t.tok[1] = t.tok[0]                                # (the last one has nothing drafted)
    gone = torch.from_numpy(t.tok) < 0
    for x in (t.q, t.k, t.v):
        x[gone] = float("nan")
    t.check()
    want, tol = t.want()
    drafted = np.nonzero(t.tok[0] >= 0)[0]
    inner = set(t.parent[drafted].tolist())
    leaves = [int(u) for u in drafted if int(u) not in inner]
    per = H // G
    some = [leaves[0], leaves[len(leaves) // 2], leaves[-1]]
    for i, u in enumerate(some):
        t.v[0, u, G - 1, 5 + i] = float("-inf") if i % 2 else float("nan")
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    for i, u in enumerate(some):
        assert not bool(torch.isfinite(got[0, u, (G - 1) * per:, 5 + i]).any())
        got[0, u, (G - 1) * per:, 5 + i] = want[0, u, (G - 1) * per:, 5 + i]
    assert bool(((got - want).abs() <= tol).all())


@pytest.mark.parametrize("d,dtype,N", [(64, BF, 1), (128, HF, 16), (128, BF, 64)])
def test_places_far_into_a_cache(binding, d, dtype, N):
    """Pages 9 GiB apart: places past 2^32 bytes and past 2^31 chunks of 16 bytes, for rows that come and rows that are read."""
    apart, page, G = (9 << 30) // 2, 16, 2
    t = Attn(binding, 270 + N, [64, 33], N, 4, G, d, page, dtype, 1.0)
    t.pages = 5
    t.kp, t.vp = t.kp[:, :5].contiguous(), t.vp[:, :5].contiguous()
    t.table[0, :4], t.table[1, :3] = [4, 1, 0, 3], [4, 2, 3]  # (shared pages: both read the same)
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 36 GiB of device memory")
    flat = torch.empty(4 * apart + 2 * page * G * d, dtype=dtype, device="cuda")
    shape, strides = (1, 5, page, G, d), (8, apart, G * d, d, 1)
    k, v = (flat.as_strided(shape, strides, i * page * G * d) for i in range(2))
    cache = binding.PagedCache(k, v)
    slots = torch.arange(5 * page, dtype=torch.int64, device="cuda").flip(0).contiguous()[None]
    rows = [x.cuda().reshape(1, 1, 5 * page, G, d) for x in (t.kp, t.vp)]
    one = handle(binding, 1, tree(1))
    one.cache_commit(cache, rows[0], rows[1], slots, slots.int())
    assert torch.equal(k.cpu(), t.kp) and torch.equal(v.cpu(), t.vp)
    t.check(t.h.tree_attention(**dict(t.on_gpu(), cache=cache)))


def test_attention_of_many_small_weights(binding):
    """fp16 weights far below the largest are as coarse as the documentation says, and not coarser."""
    t = Attn(binding, 280, [30000, 5], 1, 4, 1, 64, 16, HF, 1.0)
    for x in (t.q, t.k, t.kp):
        x.zero_()
    t.q[..., 0] = 8.0
    t.kp[..., 0] = -1.85 - torch.rand(t.kp.shape[:-1], generator=torch.Generator().manual_seed(1)) * 0.1
    t.scale = 1.0
    t.check()


@pytest.mark.parametrize("rho", [2.0 ** -126, 1e-30, 1e30, 3.4e38, float("inf")])
def test_repetition_penalties_of_any_size(binding, rho):
    """Quotients and products by what a penalty may be: 1 / rho is then subnormal, zero or nearly infinite."""
    t = test_serve_ops.Shape(binding, 290, 1, 2, 64, torch.float32, 0, None, True, False, share=1.0)
    t.count = torch.full((1, 64), 1, dtype=torch.int32)
    t.penalty = torch.tensor([[rho, 0.0, 0.0]])
    t.x[0, 0] = torch.cat([torch.linspace(-3, -0.1, 31), torch.linspace(0.1, 3, 33)])
    t.x[0, 1] = torch.cat([10.0 ** torch.linspace(-37, 38, 40), -10.0 ** torch.linspace(-37, 38, 24)])
    got = t.h.shape_logits(out=None, **t.args()).cpu()
    r = t.penalty[0, 0].double()
    x = t.x.double()
    exact = torch.where(x > 0, x / r, x * r)
    want = exact.float()
    # half a step, of a subnormal number 2^-150; past the largest number infinity
    off = (got.double() - want.double()).abs()
    same = (got == want) | (off <= want.double().abs() * 2.0 ** -23) | (off <= 2.0 ** -149)
    assert bool(same.all()), (got[~same], want[~same])

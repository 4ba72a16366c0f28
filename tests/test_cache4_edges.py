"""The attention over a cache of 4 bits, and rows into and out of such a cache, at the ends of what their documentation allows: values of
the tree that are no finite numbers, scores of every size, workspaces, captured calls, wide tables.  Every case runs in both forms of the
attention: waves by themselves (up to 64 rows that share a key/value head) and teams of waves."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests import serveref, serveref4, test_serve_edges  # noqa: E402
from tests.test_cache4 import Attn4, Cached  # noqa: E402
from tests.test_serve_ops import BF, HF, binding, drafts, handle, tree  # noqa: E402,F401

I32 = dict(dtype=torch.int32, device="cuda")


def sees(parent):
    """[node, other]: the other one is the node or an ancestor of it."""
    N = len(parent)
    out = torch.zeros((N, N), dtype=torch.bool)
    for u in range(N):
        out[u, serveref.path(parent, u)] = True
    return out


# ---- the tree's values ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("N,H,G,lens,share", [
    (9, 4, 2, [70, 0], 1.0),                                 # waves by themselves
    (16, 8, 2, [3000, 33, 0], 0.8),                          # ... two tiles of an item, and items cut into shares
    (64, 2, 2, [40, 700], 1.0),                              # ... that see more than 32 nodes
    (16, 14, 2, [700, 0, 33], 0.8),                          # teams
    (64, 8, 2, [5000, 31], 0.9),                             # ... with items cut into shares
    (300, 4, 2, [64, 0], 0.9),                               # ... that see more than 32 nodes
    (1024, 2, 2, [170], 0.95),
])
@pytest.mark.parametrize("d,dtype", [(64, BF), (64, HF), (128, BF), (128, HF)])
def test_values_of_the_tree_that_are_no_finite_numbers(binding, N, H, G, lens, share, d, dtype):
    """They reach their element of the rows that see their node, whatever its weight, and nothing else; likewise a key that is NaN."""
    t = Attn4(binding, 400 + N + H + d, lens, N, H, G, d, 16, dtype, share)
    want, tol = t.want()
    see, per = sees(t.parent), H // G
    wild = torch.zeros(want.shape, dtype=torch.bool)
    drafted = np.nonzero(t.tok[0] >= 0)[0]
    inner = set(t.parent[drafted].tolist())
    leaves = [int(u) for u in drafted if int(u) not in inner]
    some = [leaves[0], leaves[len(leaves) // 2], leaves[-1]] + [int(u) for u in sorted(inner) if u > 0][-2:]
    for i, u in enumerate(some):                             # elements of all blocks and of both halves of a lane's
        for g, e in ((0, (5 + 17 * i) % d), (G - 1, d - 1 - 9 * i)):
            t.v[0, u, g, e] = (float("inf"), float("nan"), float("-inf"))[(i + g) % 3]
            wild[0, see[:, u], g * per:(g + 1) * per, e] = True
    def compare():
        got = t.h.tree_attention(**t.on_gpu()).cpu().double()
        there = (torch.from_numpy(t.tok) >= 0)[..., None, None].expand(want.shape)
        assert bool((got[~there] == 0).all())
        assert not bool(torch.isfinite(got[wild & there]).any())
        assert bool(((got - want).abs() <= tol)[~wild].all()), (((got - want).abs() > tol) & ~wild).nonzero()[:4]
        return got
    got = compare()
    for i, u in enumerate(some[:1]):                         # of the leaf alone the element is what stands there
        x = float(t.v[0, u, 0, (5 + 17 * i) % d])
        y = got[0, u, :per, (5 + 17 * i) % d]
        assert bool((torch.isnan(y) if x != x else y == x).all())
    t.k[0, leaves[-1], G - 1] = float("nan")
    wild[0, leaves[-1], (G - 1) * per:] = True
    compare()
    t.v[0, 0, 0, 2] = float("-inf")                          # the root's: every row of that head sees it
    wild[0, :, :per, 2] = True
    compare()


@pytest.mark.parametrize("N,H,G", [(16, 4, 1), (16, 14, 1), (64, 4, 1)])
def test_nothing_drafted(binding, N, H, G):
    t = Attn4(binding, 410, [300, 5], N, H, G, 128, 16, BF)
    t.tok[:] = -1
    a = t.on_gpu()
    a["out"] = torch.full(a["q"].shape, float("nan"), dtype=BF, device="cuda")
    assert bool((t.h.tree_attention(**a) == 0).all())


@pytest.mark.parametrize("N,H", [(9, 4), (64, 6)])
def test_shared_pages_and_broadcast_queries(binding, N, H):
    t = Attn4(binding, 411, [200, 200, 200], N, H, 2, 64, 16, BF, 1.0)
    t.table[1:] = t.table[0]
    t.lens = [200, 150, 7]
    t.q, t.k, t.v = (x[:1].expand(3, *x.shape[1:]) for x in (t.q, t.k, t.v))
    a = t.on_gpu()
    for n in ("q", "k", "v"):
        a[n] = a[n][:1].expand(3, *a[n].shape[1:])
    t.check(t.h.tree_attention(**a))


# ---- scores of every size -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("N,H,G,lens", [(1, 4, 1, [300, 0, 3, 5000]), (16, 4, 1, [300, 0, 1]), (16, 14, 1, [700, 33, 0]), (33, 1, 1, [2000, 1]), (64, 4, 1, [3000, 2, 65])])
@pytest.mark.parametrize("d,dtype,sign,size,scale", [
    (128, BF, -1.0, 1.3e38, 1.0), (64, BF, -1.0, 1.8e38, 1.6), (64, BF, 1.0, 1.8e38, 1.6), (128, BF, 1.0, 1e12, 1.0), (64, HF, -1.0, 1.6e9, 1.0), (128, HF, 1.0, 1.6e9, 1.0),
])
def test_far_scores(binding, N, H, G, lens, d, dtype, sign, size, scale):
    """Scores of any size that fp32 holds: the row is that of its largest one, not NaN."""
    t = test_serve_edges.far(Attn4(binding, 420 + N + H, lens, N, H, G, d, 16, dtype, 0.8 if N > 1 else 1.0), sign, size)
    t.hold()
    t.scale = scale
    # (what a sum of products may reach on its way stays a number of fp32)
    assert float(t.q.double().abs().amax() * max(t.kp.double().abs().amax(), t.k.double().abs().amax()) * d) < 2.0 ** 128
    want, sure = test_serve_edges.hard_attention(t)
    drafted = torch.from_numpy(t.tok) >= 0
    assert bool(sure[drafted].any())
    got = t.h.tree_attention(**t.on_gpu()).cpu()
    assert bool(torch.isfinite(got).all())
    assert torch.equal(got[sure], want[sure])
    assert bool((got[~drafted] == 0).all())


@pytest.mark.parametrize("N,H,G,d,dtype", [(16, 4, 2, 128, BF), (33, 7, 1, 64, HF), (16, 2, 1, 64, HF), (64, 6, 2, 128, HF), (64, 6, 2, 64, BF)])
def test_far_scores_beside_ordinary_ones(binding, N, H, G, d, dtype):
    """Rows of one wave with scores of thousands and rows with scores of 1: the ordinary rows keep their errors."""
    t = Attn4(binding, 430 + N, [900, 77, 0], N, H, G, d, 16, dtype, 1.0)
    t.q[:, ::3] *= 2.0 ** (13 if dtype is HF else 26)
    known = torch.isfinite(t.q).all(dim=3)
    got = t.h.tree_attention(**t.on_gpu()).cpu()
    want, sure = test_serve_edges.hard_attention(t)
    sure &= known
    assert bool(torch.isfinite(got[known]).all()) and bool(sure[:, ::3].any()) and torch.equal(got[sure], want[sure])
    t.q[:, ::3] = 0
    want, tol = t.want()
    keep = torch.arange(N) % 3 != 0
    assert bool(((got.double() - want).abs() <= tol)[:, keep].all())


@pytest.mark.parametrize("N,H,G", [(1, 4, 1), (16, 4, 1), (16, 14, 1)])
@pytest.mark.parametrize("d,dtype", [(64, HF), (64, BF), (128, HF), (128, BF)])
def test_extreme_scales(binding, N, H, G, d, dtype):
    """From the smallest number, which leaves the mean of the values, to the largest that is accepted, which leaves one of them."""
    t = Attn4(binding, 445 + N + H, [300, 0, 2000], N, H, G, d, 16, dtype, 0.8 if N > 1 else 1.0)
    for t.scale in (2.0 ** -149, 1e-40, 2.0 ** -126, 1e-20):
        t.check()
    t.scale = 2.0 ** 127
    want, sure = test_serve_edges.hard_attention(t)
    got = t.h.tree_attention(**t.on_gpu()).cpu()
    assert bool(sure.any()) and bool(torch.isfinite(got).all()) and torch.equal(got[sure], want[sure])


@pytest.mark.parametrize("N,H,G,lens", [(1, 4, 1, [5000, 0]), (16, 3, 1, [1500, 40, 3]), (16, 14, 1, [3000, 1])])
@pytest.mark.parametrize("d,dtype,e", [(128, BF, 20), (128, BF, 22), (64, BF, 23), (64, BF, 60), (64, HF, 21), (128, HF, 22), (64, HF, 23), (128, HF, 30)])
def test_equal_scores_of_any_size(binding, N, H, G, lens, d, dtype, e):
    """Keys that are all the same leave the mean of the values, below the size from which maxima are taken off and above it, also
    where a row is joined from several parts; rows of both kinds and of both signs in one wave."""
    t = Attn4(binding, 448 + N + H, lens, N, H, G, d, 16, dtype, 0.8 if N > 1 else 1.0)
    t.scale = 1.0
    for x in (t.k, t.kp):
        x.fill_(2.0 ** (e // 2 - 3))
    t.hold()
    assert bool((t.kp == 2.0 ** (e // 2 - 3)).all())          # (a power of two is held as it is)
    t.q.fill_(2.0 ** (e - e // 2 + 3) / d)
    t.q[:, ::3] *= -1
    t.q[:, 1::4] *= 3
    t.q[:, 2::5] *= 2.0 ** -e if dtype is BF else 2.0 ** -10
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    half = serveref.EPS[dtype]
    for b, n in enumerate(lens):
        pos = torch.arange(n)
        V = t.vp[0][torch.from_numpy(t.table[b]).long()[pos // 16], pos % 16].double()
        for u in range(N):
            if t.tok[b, u] < 0:
                continue
            own = serveref.path(t.parent, u)
            for i in range(H):
                all_v = torch.cat([V[:, i // (H // G)], t.v[b, own, i // (H // G)].double()])
                mean = all_v.mean(0)
                # equal weights: sums of so many terms in fp32, parts joined, one quotient and the rounding of the result
                tol = all_v.abs().mean(0) * (len(all_v) + 64) * 2.0 ** -24 * 2 + mean.abs() * half + (2.0 ** -25 if dtype is HF else 0)
                assert bool(((got[b, u, i] - mean).abs() <= tol).all()), (b, u, i)


@pytest.mark.parametrize("size", [2 ** 15, 2 ** 20, 2 ** 21 + 2 ** 20, -(2 ** 21) - 2 ** 20, 2907264, 2907272, -2907264, -2907272, 2 ** 22 + 2 ** 21])
@pytest.mark.parametrize("N,H,G,n", [(1, 1, 1, 700), (16, 1, 1, 700), (1, 4, 1, 9000), (16, 3, 1, 700), (16, 14, 1, 700), (16, 14, 1, 9000)])
@pytest.mark.parametrize("d,dtype", [(64, BF), (128, HF)])
def test_the_maximum_is_raised_exactly(binding, N, H, G, n, size, d, dtype):
    """Many keys of one score and then one of six more, exact numbers both: what the sums so far are scaled by is as exact as a
    weight, whatever the size of the scores (2^22 / log2(e) lies between two of them).  A score is the sum of a whole number's bits: bit e
    is the product of 2^e and 1 in a key's first block, of 2^(e - 8) and 2^8 in its second, numbers that 4 bits hold."""
    t = Attn4(binding, 485 + N + H, [n], N, H, G, d, 16, dtype, 1.0)
    t.scale = 1.0
    for x in (t.q, t.k, t.kp, t.v, t.vp):
        x.zero_()
    for e in range(24):
        at, by = (e, 1.0) if e < 12 else (32 + e - 12, 2.0 ** 8)
        t.q[..., at] = 2.0 ** e / by
        if abs(size) >> e & 1:
            for x in (t.k, t.kp):
                x[..., at] = by if size > 0 else -by
    t.q[..., 12] = 1.0
    t.v[..., :] = 1.0
    t.vp[..., :] = 1.0
    last = (t.table[0, (n - 1) // 16], (n - 1) % 16)
    t.kp[0][last][:, 12] = 6.0
    t.vp[0][last] = 0.0
    asked = t.kp.clone(), t.vp.clone()
    t.hold()
    assert torch.equal(t.kp, asked[0]) and torch.equal(t.vp, asked[1])
    some = (t.table[0, 0], 0)
    assert float(t.kp[0][some][0].double() @ t.q[0, 0, 0].double()) == size and float(t.kp[0][last][0].double() @ t.q[0, 0, 0].double()) == size + 6
    deep = serveref.depths(t.parent)
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    many = torch.tensor(n - 1 + deep + 1.0)[None, :, None, None]          # keys of the one score: the cache's and the path's
    want = many / (many + np.exp(6.0))
    # a weight of either kind is off by half a step, the exponent by a rounding of the difference and c's own (six of 2^-24)
    half = serveref.EPS[dtype]
    tol = want * (1 - want) * 2 * half + want * (half + (n + 64) * 2.0 ** -23)
    assert bool(((got - want).abs() <= tol).all()), (float(got.min()), float(got.max()), float(want.min()), float(want.max()))


def over(q, K, V, scale, dtype):
    """(output, largest error allowed) of one row [d] over keys and values [n, d]: as serveref.attention has them."""
    t = serveref.attention(np.array([-1], np.int32), [len(K) - 1], torch.arange(1)[:, None], torch.zeros((1, 1)), q[None, None, None], K[-1:][None, :, None],
                           V[-1:][None, :, None], K[None, :, None], V[None, :, None], scale)
    return t[0][0, 0, 0], t[1][0, 0, 0]


@pytest.mark.parametrize("N,H,G,lens", [(1, 4, 1, [200, 40, 0, 96]), (16, 4, 1, [200, 40, 0, 96]), (16, 14, 1, [200, 40, 0, 96]), (16, 14, 1, [5000, 40, 0, 96]), (1, 4, 1, [5000, 40, 0, 96])])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_are_minus_infinity_count_for_nothing(binding, N, H, G, lens, d):
    """Products below what fp32 holds leave a row to its other keys, whether they are cached or the tree's; a row that has no other is NaN, as is
    one with an infinite score."""
    t = Attn4(binding, 440 + N + H, lens, N, H, G, d, 16, BF, 1.0)
    t.q[..., 0] = 2.0 ** 64
    for x in (t.k, t.kp):
        x[..., 0] = 0.0
    out = torch.zeros((len(lens), max(lens)), dtype=torch.bool)            # cached keys that count for nothing
    out[0, :150] = True                                                    # whole units and parts of one
    out[0, 170:180] = True
    out[3] = True                                                          # all of them: what is left is the tree
    for b in (0, 3):
        for p in range(lens[b]):
            if out[b, p]:
                t.kp[0][t.table[b, p // 16], p % 16, :, 0] = -2.0 ** 80    # (the rest of its block becomes zero)
    t.hold()
    tree_counts = [True, False, True, True]                                # the second one's tree does not: its rows have the cache alone
    t.k[1, ..., 0] = -2.0 ** 80
    got = t.h.tree_attention(**t.on_gpu()).cpu().double()
    per = H // G
    for b, n in enumerate(lens):
        pos = torch.arange(n)[~out[b, :n]]
        at = torch.from_numpy(t.table[b]).long()[pos // 16]
        for u in range(N):
            own = serveref.path(t.parent, u) if tree_counts[b] else []
            for i in range(H):
                K, V = (torch.cat([pool[0][at, pos % 16, i // per], new[b, own, i // per]]) for pool, new in ((t.kp, t.k), (t.vp, t.v)))
                want, tol = over(t.q[b, u, i], K, V, t.scale, BF)
                assert bool(((got[b, u, i] - want).abs() <= tol).all()), (b, u, i)
    t.k[3, ..., 0] = -2.0 ** 80                                            # nothing is left of the fourth one
    t.k[2, 0, ..., 0] = 2.0 ** 80                                          # every row of the third one sees its root
    again = t.h.tree_attention(**t.on_gpu()).cpu().double()
    assert torch.equal(again[:2], got[:2]) and bool(torch.isnan(again[2:]).all())


def test_many_small_weights(binding):
    """fp16 weights far below the largest are as coarse as the documentation says, and not coarser."""
    for N, H in ((1, 4), (16, 6)):
        t = Attn4(binding, 480, [30000 if N == 1 else 6000, 5], N, H, 1, 64, 16, HF, 1.0)
        for x in (t.q, t.k, t.kp):
            x.zero_()
        t.q[..., 0] = 8.0
        t.kp[..., 0] = -1.0 - 0.5 * (torch.rand(t.kp.shape[:-1], generator=torch.Generator().manual_seed(1)) < 0.9).to(HF)
        t.hold()
        t.scale = 1.0
        t.check()


# ---- workspaces, graphs ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("N,H", [(9, 4), (64, 6)])
@pytest.mark.parametrize("d,dtype", [(64, BF), (128, HF)])
def test_workspaces(binding, N, H, d, dtype):
    """One byte less than asked for is refused, and a refused call leaves its output; nothing is written behind the workspace."""
    t = Attn4(binding, 499, [4000, 33], N, H, 2, d, 16, dtype)
    a = t.on_gpu()
    need = t.h._lib.stand_tree_attention_work(t.h.h, a["cache"].ref, H)
    assert need > 0 and need % 16 == 0 and t.h._lib.stand_tree_attention_work(t.h.h, a["cache"].ref, H + 1) == 0
    key = (H, 2, d, a["cache"].desc.dtype)
    out = torch.full(a["q"].shape, 5.0, dtype=dtype, device="cuda")
    t.h._work_bytes = {key: need - 1}
    with pytest.raises(binding.StandError):
        t.h.tree_attention(**dict(a, out=out))
    torch.cuda.synchronize()
    assert bool((out == 5.0).all())
    t.h._work_bytes = {}
    t.check(t.h.tree_attention(**a))
    # a workspace inside a larger piece of memory, full of what is no number
    room = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    pack = binding._TREE_ROWS.pack(a["q"].data_ptr(), a["k"].data_ptr(), a["v"].data_ptr(), out.data_ptr(), H, a["scale"], *a["q"].stride()[:3], *a["k"].stride()[:3],
                                   *a["v"].stride()[:3], *out.stride()[:3])
    rc = t.h._lib.stand_tree_attention(t.h.h, a["cache"].ref, 0, a["length"].data_ptr(), a["table"].data_ptr(), a["table"].shape[1], a["draft_tok"].data_ptr(), pack,
                                       room.data_ptr() + 2048, need, torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    t.check(out)
    assert bool((room[:2048] == 255).all()) and bool((room[2048 + need:] == 255).all())


def test_workspaces_of_refused_calls_have_no_size(binding):
    many = handle(binding, 4097, tree(1))
    h = handle(binding, 2, tree(9))
    cache = binding.PagedCache.new4(1, 4, 16, 2, 64)
    size = h._lib.stand_tree_attention_work
    assert size(h.h, cache.ref, 4) > 0 and size(h.h, cache.ref, 65534) > 0
    assert size(h.h, cache.ref, 65536) == 0 and size(h.h, cache.ref, 3) == 0 and size(h.h, cache.ref, 0) == 0 and size(None, cache.ref, 4) == 0
    assert size(many.h, cache.ref, 4) == 0
    cache.whole.scale_page_stride, cache.desc.pages = 2 ** 40, 2 ** 20
    assert size(h.h, cache.ref, 4) == 0


@pytest.mark.parametrize("N,H,d,dtype", [(16, 8, 128, BF), (1, 4, 64, HF), (64, 8, 64, BF), (64, 6, 128, HF)])
def test_captured_calls_follow_what_changes_on_the_device(binding, N, H, d, dtype):
    """Two graphs of one handle, lengths, drafts and tables changed between their replays, eager calls in between."""
    lens = [1500, 77, 3]
    t = Attn4(binding, 500 + N, lens, N, H, 2, d, 16, dtype)
    a = t.on_gpu()
    a["out"] = torch.empty(a["q"].shape, dtype=dtype, device="cuda")
    b = dict(a, out=torch.empty_like(a["out"]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        t.h.tree_attention(**a)
    side.synchronize()
    graphs = []
    for x in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            t.h.tree_attention(**x)
        graphs.append(g)
    rng = np.random.default_rng(1)
    whole = t.table.copy()
    for rep in range(4):
        t.lens = [int(rng.integers(0, n + 1)) for n in lens]
        t.tok = drafts(rng, 3, t.parent, 0.6 if N > 1 else 1.0)
        used = max(1, -(-lens[0] // 16))
        t.table[0, :used] = rng.permutation(whole[0, :used])
        a["length"].copy_(torch.tensor(t.lens))
        a["draft_tok"].copy_(torch.from_numpy(t.tok))
        a["table"].copy_(torch.from_numpy(t.table))
        for x in (a, b):
            x["out"].fill_(9.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        t.check(a["out"])
        eager = t.h.tree_attention(**dict(a, out=None))
        torch.cuda.synchronize()
        assert torch.equal(eager, a["out"]) and torch.equal(eager, b["out"])


# ---- wide tables --------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("G,d,dtype,width", [(64, 128, BF, 2 ** 21 + 5), (8, 64, HF, 2 ** 21 + 5), (64, 128, HF, 2 ** 24 + 5)])
def test_commit_of_wide_tables_into_four_bits(binding, G, d, dtype, width):
    """Every slot of the table is a good one; only what the counts leave goes in, from the first position to the last."""
    B, R, pages, page = 2, 4, 5, 8
    c = Cached(binding, torch.Generator().manual_seed(6), 1, pages, page, G, d, dtype, 4, "nhd")
    gen = torch.Generator().manual_seed(7)
    k, v = (torch.randn((1, B, R, G, d), generator=gen).to(dtype) for _ in range(2))
    slots = torch.full((B, width), 3, dtype=torch.int64, device="cuda")
    row = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    h = handle(binding, B, tree(1))
    dev = k.cuda(), v.cuda()
    for counts, at in (([0, -1], []), ([-2 ** 31, 0], []), ([2, width], [(0, 0, 2, 9), (0, 1, 0, 39), (1, 0, 3, 17), (1, width - 1, 1, 30), (1, width // 2, 0, 1)]),
                       ([1, width - 1], [(0, 0, 1, 4), (1, width - 2, 2, 12)]), ([2 ** 31 - 1, 0], [(0, width - 1, 3, 0)])):
        row.fill_(-1 if at else 0)
        for b, j, r, s in at:
            row[b, j], slots[b, j] = r, s
            c.put(0, s // page, s % page, k[0, b, r].double(), v[0, b, r].double())
        if at:                                               # behind the counts: rows that may not go in
            for b in range(B):
                row[b, max(0, min(counts[b], width)):] = 0
        h.cache_commit(c.cache, *dev, slots, row, torch.tensor(counts, **I32))
        c.check()
        for b, j, r, s in at:
            slots[b, j] = 3


@pytest.mark.parametrize("bits,G,d,dtype,R", [(4, 64, 128, BF, 2 ** 20 + 5), (16, 8, 64, HF, 2 ** 21 + 5), (4, 3, 64, HF, 2 ** 22 + 1)])
def test_append_of_many_rows(binding, bits, G, d, dtype, R):
    """A row for all positions, slots of a few of them; the first, the last one and those around the counts."""
    B, pages, page = 2, 5, 8
    gen = torch.Generator().manual_seed(8)
    c = Cached(binding, gen, 1, pages, page, G, d, dtype, bits, "nhd")
    k, v = (torch.randn((B, 1, G, d), generator=gen).to(dtype) for _ in range(2))
    slots = torch.full((B, R), -1, dtype=torch.int64, device="cuda")
    h = handle(binding, B, tree(1))
    dims = 32
    table = serveref4.turns(R + 10, dims)
    rot = binding.Rotation(table.cuda(), "neighbours")
    dev = [x.cuda().expand(B, R, G, d) for x in (k, v)]
    start = [10, 0]
    for counts, at in (([0, -5], []), ([2, R], [(0, 0, 3), (0, 1, 39), (1, 0, 17), (1, R - 1, 30), (1, R // 2, 1)]), ([R - 1, 1], [(0, R - 2, 7), (1, 0, 8)]), (None, [(0, R - 1, 2), (1, R - 1, 5)])):
        slots.fill_(-1)
        for b, j, s in at:
            slots[b, j] = s
            y = serveref4.turned(k[b, 0], torch.tensor(start[b] + j), table, "neighbours", None, 0.0)
            c.put(0, s // page, s % page, y, v[b, 0].double())
        if counts:
            for b in range(B):
                n = max(0, counts[b])
                if n < R:
                    slots[b, n], slots[b, R - 1] = 4, 6      # behind the counts: these may not go in
        h.cache_append(c.cache, 0, *dev, slots, torch.tensor(start, **I32), None if counts is None else torch.tensor(counts, **I32), rot)
        c.check(near=True)


# ---- rows that no 4 bits hold -------------------------------------------------------------------------------------------------------

def held(c, i):
    """The numbers that the cache's keys (0) or values (1) stand for."""
    return serveref4.unpack(c.gpu[i].cpu(), c.gpu[i + 2].cpu(), c.dtype)


@pytest.mark.parametrize("dtype,d,pairs,dims,norm", [(BF, 64, "halves", 64, True), (HF, 64, "neighbours", 32, False), (BF, 128, "neighbours", 128, False), (HF, 128, "halves", 96, True)])
def test_appended_rows_that_are_no_finite_numbers(binding, dtype, d, pairs, dims, norm):
    """A block with an infinity or a NaN, whether it was in the row, came of its turn or of a position without one, is NaN as a whole; the
    others are as they would be without it.  Keys past what a scale reaches are held as its largest number."""
    gen = torch.Generator().manual_seed(d + dims)
    B, R, G, pages, page, positions = 3, 12, 2, 4, 16, 40
    k, v = (torch.randn((B, R, G, d), generator=gen).to(dtype) for _ in range(2))
    inf, nan, top = float("inf"), float("nan"), torch.finfo(dtype).max
    k[0, 0, 0, 3], k[0, 1, 1, d - 1], k[0, 2, 0, 17] = inf, nan, -inf
    v[0, 0, 1, 40], v[0, 1, 0, 0], v[0, 2, 1, 63] = nan, -inf, inf
    k[0, 3], v[0, 3] = 0.0, -0.0
    k[0, 4, 0], v[0, 4, 0] = top, -top
    k[0, 5, 0, 5], v[0, 5, 0, 5] = top, top
    smallest = 2.0 ** -133 if dtype is BF else 2.0 ** -24
    k[0, 6, 0], v[0, 6, 0] = smallest, smallest
    table = serveref4.turns(positions, dims)
    w = (1 + 0.3 * torch.randn(d, generator=gen)).to(dtype) if norm else None
    start = [5, positions - 6, -4]                           # the second one's last rows and the third one's first have no position
    slots = torch.randperm(pages * page, generator=gen)[:B * R].reshape(B, R)
    c = Cached(binding, gen, 1, pages, page, G, d, dtype, 4, "nhd")
    before = [held(c, i) for i in range(2)]
    h = handle(binding, B, tree(1))
    rot = binding.Rotation(table.cuda(), pairs, None, None if w is None else w.cuda(), 0.0 if not norm else 1e-6)
    h.cache_append(c.cache, 0, k.cuda(), v.cuda(), slots.cuda(), torch.tensor(start, **I32), None, rot)
    pos = torch.tensor(start)[:, None].long() + torch.arange(R)
    want = [serveref4.turned(k, pos, table, pairs, w, 1e-6).float(), v.float()]
    for i in range(2):
        x = before[i].clone()
        flat = x.reshape(pages * page, G, d)
        flat[slots] = serveref4.unpack(*serveref4.pack(want[i], dtype), dtype)
        got = held(c, i)
        assert torch.equal(torch.isnan(got), torch.isnan(x)), (torch.isnan(got) != torch.isnan(x)).nonzero()[:4]
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(x))
        assert not bool(torch.isinf(got).any())
    nans = torch.isnan(held(c, 0).reshape(-1, G, d)[slots])
    assert bool(nans[1, 6:, :, :dims // 32 * 32].all()) and bool(nans[2, :4, :, :dims // 32 * 32].all())


# ---- many trajectories, long texts ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("N,H,G,d,dtype,most", [(1, 2, 1, 64, BF, 40), (2, 40, 1, 64, HF, 40), (1, 1, 1, 128, HF, 40)])
def test_as_many_trajectories_as_it_takes(binding, N, H, G, d, dtype, most):
    lens = [int(x) for x in np.random.default_rng(3).integers(0, most, 4096)]
    Attn4(binding, 97, lens, N, H, G, d, 16, dtype, 1.0).check()


def test_more_trajectories_are_refused(binding):
    t = Attn4(binding, 98, [3] * 4097, 1, 2, 1, 64, 16, BF, 1.0)
    with pytest.raises(binding.StandError):
        t.h.tree_attention(**t.on_gpu())


@pytest.mark.parametrize("N,H,d,dtype,page", [(1, 4, 64, BF, 16), (9, 8, 64, HF, 8), (9, 4, 128, BF, 64), (9, 10, 128, BF, 4096)])
def test_long_texts(binding, N, H, d, dtype, page):
    """Two hundred thousand tokens, many times the same pages: a table may name a page as often as it likes."""
    t = Attn4(binding, 600 + N + d, [16 * page, 33], N, H, 1, d, page, dtype, 1.0)
    n = 200003
    t.width = -(-n // page)
    t.table = np.random.default_rng(5).integers(0, t.pages, (2, t.width)).astype(np.int32)
    t.lens = [n, 33]
    t.check()


@pytest.mark.parametrize("N,H", [(9, 4), (64, 6)])
def test_graphs_on_two_streams(binding, N, H):
    """Two graphs, each with its own buffers and workspaces, replayed on two streams without waiting for each other, rotations and appends
    in them; eager calls in between."""
    d, dtype, B = 128, BF, 2
    ts = [Attn4(binding, 700 + i, [900, 70], N, H, 2, d, 16, dtype, 0.9) for i in range(2)]
    turns = serveref4.turns(1000, d)
    rot = binding.Rotation(turns.cuda())
    sides, graphs, all_args, q_in = [torch.cuda.Stream() for _ in ts], [], [], []
    for t, s in zip(ts, sides):
        a = t.on_gpu()
        x = [a["q"].clone(), a["k"].clone()]
        a["out"] = torch.empty_like(a["q"])

        def call(a=a, x=x, t=t):
            t.h.tree_rotate(rot, a["length"], a["draft_tok"], x[0], x[1], a["q"], a["k"])
            t.h.tree_attention(**a)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            call()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
        graphs.append(g)
        all_args.append(a)
        q_in.append(x)
    torch.cuda.synchronize()
    for rep in range(5):
        for a in all_args:
            a["out"].fill_(3.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, sides):
            with torch.cuda.stream(s):
                g.replay()
                g.replay()
        torch.cuda.synchronize()
        for t, a in zip(ts, all_args):
            if rep == 0:                                     # what the attention saw: the rotated rows as they are
                t.q, t.k = a["q"].cpu(), a["k"].cpu()
            t.check(a["out"])
            eager = t.h.tree_attention(**dict(a, out=None))
            torch.cuda.synchronize()
            assert torch.equal(eager, a["out"])

"""A cache in four bits and the way into it, as cases that can be timed and compared.

What a target model's layer does with its queries, keys and values around the attention of a drafted tree, and the same
attention over a cache that holds 4 bits an element (blocks of 32 elements of a head with a power of two for scale), so that
four times as many cached tokens fit and a decoded token reads a quarter of the bytes:

  rotate   queries and keys of the drafted nodes: a norm for each head, and the rotation by the nodes' positions
  append   keys and values of prompts and single tokens into the paged cache (16 bits or 4), normed and rotated on the way
  commit   the accepted path's keys and values of all layers, or prompts as they stand, into a cache of 4 bits
  attn     attention of the drafted nodes over a paged cache of 4 bits and over their own ancestors in the tree

Where the cache has 4 bits, `append` and `commit` are followed by a read of the tokens as rows of 16 bits (what a prompt's
next chunk attends to), so that what was written comes back as the values it stands for.

`own` selects what `run` calls: the plain forms below (elementary torch operations), or the framework's operators.  A tree is
the breadth-first `parent` list of the framework; node 0 is the last committed token.
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---- cases ------------------------------------------------------------------------------------------------------------

def _rotate(name, B, N, D, fan, drafted, lo, hi, Hq, Hkv, d, dims, pairs, norm, dtype="bf16", fused=False):
    return dict(name=name, op="rotate", B=B, N=N, D=D, fan=fan, drafted=drafted, lo=lo, hi=hi, Hq=Hq, Hkv=Hkv, d=d, dims=dims, pairs=pairs,
                norm=norm, dtype=dtype, fused=fused)


def _append(name, B, R, rlo, lo, hi, Hq, Hkv, d, page, dims, pairs, norm, bits, dtype="bf16", layout="nhd", fused=True):
    return dict(name=name, op="append", B=B, R=R, rlo=rlo, lo=lo, hi=hi, Hq=Hq, Hkv=Hkv, d=d, page=page, dims=dims, pairs=pairs, norm=norm,
                bits=bits, dtype=dtype, layout=layout, fused=fused)


def _commit(name, layers, B, R, W, rlo, lo, hi, Hkv, d, page, dtype="bf16", layout="nhd", path=True):
    return dict(name=name, op="commit", layers=layers, B=B, R=R, W=W, rlo=rlo, lo=lo, hi=hi, Hkv=Hkv, d=d, page=page, dtype=dtype, layout=layout,
                path=path)


def _attn(name, B, N, D, fan, drafted, lo, hi, Hq, Hkv, d, page, dtype="bf16", layout="nhd", fused=False):
    return dict(name=name, op="attn", B=B, N=N, D=D, fan=fan, drafted=drafted, lo=lo, hi=hi, Hq=Hq, Hkv=Hkv, d=d, page=page,
                dtype=dtype, layout=layout, fused=fused)


def listed():
    return [
        # one short request on a small model: no norms, a launch and its round trips
        _rotate("rotate_short", 1, 16, 4, "4-2-1-1", 0.8, 37, 37, 14, 2, 64, 64, "halves", False, "bf16", True),
        # tree search over 128 beams, large trees far into their texts: norms, half of a head rotated
        _rotate("rotate_beams", 128, 128, 10, "8-4-2-1", 0.6, 200, 30000, 16, 8, 128, 64, "neighbours", True, "f16", True),
        # the first tokens after 64 prompts, or single tokens that are not drafted: one row of each
        _append("append_decode", 64, 1, 1, 0, 16000, 32, 8, 128, 32, 128, "halves", True, 16, "bf16", "hnd"),
        # prompts of up to 2100 tokens, queries along with them
        _append("append_prompt", 4, 2100, 900, 0, 0, 32, 8, 128, 16, 128, "halves", False, 16, "f16", "nhd"),
        # a chunk of long prompts into 4 bits; the context so far comes back as rows for the chunk's attention
        _append("append_chunk4", 4, 1024, 500, 0, 6000, 28, 4, 128, 64, 128, "halves", True, 4, "bf16", "nhd"),
        # the accepted paths of a step: one to nine tokens of each trajectory, 28 layers
        _commit("commit_step4", 28, 32, 64, 9, 1, 1000, 9000, 4, 128, 64),
        # prompts go into the cache as they stand, and out of it again (a request that makes room and comes back)
        _commit("commit_prompt4", 16, 4, 2100, 2100, 900, 0, 0, 8, 128, 16, "f16", "hnd", False),
        # one short request on a small model: nothing but launches and dependent round trips
        _attn("attn4_short", 1, 16, 4, "4-2-1-1", 0.8, 37, 37, 14, 2, 64, 16, "f16"),
        # one user with a long reasoning trace, a tree of 32 nodes: few heads, a long axis
        _attn("attn4_single", 1, 32, 6, "4-2-2-1", 0.8, 60001, 60001, 28, 4, 128, 16, "bf16", "nhd", True),
        # best-of-32 in the middle of its run, trajectories of very different lengths
        _attn("attn4_best32", 32, 64, 8, "8-4-2-1", 0.75, 1000, 9000, 28, 4, 128, 64),
        # single tokens (a tree of one node) of 64 requests, from an empty cache to long ones: the cache is read once
        _attn("attn4_decode", 64, 1, 0, "1", 1.0, 0, 32000, 32, 8, 128, 32, "bf16", "hnd"),
        # tree search over 128 beams, large trees, short caches, 64 wide heads
        _attn("attn4_beams", 128, 128, 10, "8-4-2-1", 0.6, 200, 3000, 16, 8, 64, 16, "f16", "nhd", True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _full(D, fan):
    """Nodes of the tree of depth D that has all the children its fan-outs allow."""
    f = [int(x) for x in fan.split("-")]
    total = level = 1
    for dep in range(D):
        level *= f[min(dep, len(f) - 1)]
        total += level
    return total


def _draw_tree(rng, most):
    if rng.random() < 0.25:
        return 1, 0, "1"
    fan = rng.choice(["4-2-1-1", "4-2-2-1", "6-3-2-1", "8-4-2-1"])
    D = rng.randint(2, 12)
    return min(max(_log_uniform(rng, 8, most), int(fan[0]) + D + 1), _full(D, fan)), D, fan


def _draw_heads(rng):
    Hkv = rng.choice([1, 2, 3, 4, 8])
    return Hkv * rng.choice([1, 2, 3, 4, 5, 7, 8]), Hkv, rng.choice([64, 128])


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "commit", "append", "append", "rotate"])
    dtype, layout, page = rng.choice(["bf16", "f16"]), rng.choice(["nhd", "hnd"]), rng.choice([8, 16, 32, 64, 128])
    Hq, Hkv, d = _draw_heads(rng)
    dims, pairs, norm = rng.choice([d, d, d // 2, 48]), rng.choice(["halves", "neighbours"]), rng.random() < 0.5
    top = {c["name"]: work(c)["bytes"] for c in listed()}
    if op == "attn":
        N, D, fan = _draw_tree(rng, 300)
        hi = _log_uniform(rng, 1, 60000)
        c = _attn("", _log_uniform(rng, 1, 128), N, D, fan, rng.choice([0.3, 0.6, 0.8, 1.0]), rng.choice([0, hi // 9, hi]), hi, Hq, Hkv, d, page,
                  dtype, layout, rng.random() < 0.5)
        while work(c)["flops"] > 6.5e10 or work(c)["bytes"] > top["attn4_decode"] or c["B"] * c["hi"] * Hkv * d > 64 * 32000 * 8 * 128:
            c["B"] = c["B"] // 2
            if c["B"] == 0:
                c["B"], c["hi"] = 1, max(1, c["hi"] // 2)
                c["lo"] = min(c["lo"], c["hi"])
    elif op == "commit":
        path = rng.random() < 0.6
        N, D, _ = _draw_tree(rng, 160)
        W = D + 1 if path else _log_uniform(rng, 1, 3000)
        hi = _log_uniform(rng, 1, 20000 if path else 1000)
        c = _commit("", _log_uniform(rng, 1, 48), _log_uniform(rng, 1, 128 if path else 8), N if path else W, W, rng.choice([0, 1, W]), 0, hi,
                    Hkv, d, page, dtype, layout, path)
        while work(c)["bytes"] > top["commit_prompt4"] or c["layers"] * c["B"] * (c["hi"] + W + page) * Hkv * d > 64 * 32000 * 8 * 128:
            c["layers"], c["B"] = max(1, c["layers"] // 2), max(1, c["B"] // 2)
    elif op == "append":
        R = 1 if rng.random() < 0.25 else _log_uniform(rng, 2, 3000)
        hi = _log_uniform(rng, 1, 40000)
        c = _append("", _log_uniform(rng, 1, 128 if R < 30 else 8), R, rng.choice([0, R // 3, R]), 0, hi, Hq, Hkv, d, page, dims, pairs, norm,
                    rng.choice([16, 4]), dtype, layout, rng.random() < 0.7)
        while work(c)["bytes"] > min(top["append_prompt"], top["append_chunk4"]) or c["B"] * (hi + R + page) * Hkv * d > 16 * 32000 * 8 * 128:
            if c["B"] > 1:
                c["B"] //= 2
            else:
                hi = c["hi"] = max(1, c["hi"] // 2)
                R = c["R"] = max(1, c["R"] // 2)
                c["rlo"] = min(c["rlo"], c["R"])
    else:
        N, D, fan = _draw_tree(rng, 300)
        hi = _log_uniform(rng, 1, 60000)
        c = _rotate("", _log_uniform(rng, 1, 128), N, D, fan, rng.choice([0.3, 0.6, 1.0]), rng.choice([0, hi]), hi, Hq, Hkv, d, dims, pairs, norm,
                    dtype, rng.random() < 0.5)
        while work(c)["bytes"] > top["rotate_beams"]:
            c["B"] = max(1, c["B"] // 2)
    del c["name"]
    return c


# ---- trees, lengths, pages ----------------------------------------------------------------------------------------------

def _tree(N, D, fan):
    """A breadth-first tree of N nodes and depth D: fan-outs by depth, cut where the nodes run out; the first node of
    every level above the last has a child.  N is at most _full(D, fan)."""
    f = [int(x) for x in fan.split("-")]
    parent, level = [-1], [0]
    for dep in range(D):
        left = N - len(parent) - (D - dep - 1)       # one node is kept for every level below
        nxt = []
        for u in level:
            for _ in range(f[min(dep, len(f) - 1)]):
                if left > 0:
                    nxt.append(len(parent))
                    parent.append(u)
                    left -= 1
        level = nxt
    return np.array(parent, np.int32)


def _ancestors(parent):
    """[N, N] truth values: column v is on the path from the root to row u, u included."""
    N = len(parent)
    a = np.zeros((N, N), bool)
    for u in range(N):
        if u:
            a[u] = a[parent[u]]
        a[u, u] = True
    return a


def _depth(parent):
    d = np.zeros(len(parent), np.int64)
    for u in range(1, len(parent)):
        d[u] = d[parent[u]] + 1
    return d


def _kept(case):
    """Drafted nodes of each trajectory: from that share of the tree down to a third of it."""
    N, B = case["N"], case["B"]
    return [max(1, int(round(N * case["drafted"] * (1.0 - 0.6 * ((b * 0.618034) % 1.0))))) for b in range(B)]


def _drafted(case, parent, rs):
    """[B, N]: the root and a random set of nodes that is closed under parents, of the sizes of _kept."""
    B, N = case["B"], case["N"]
    key = rs.random_sample((B, N))
    key[:, 0] = -1.0
    for u in range(1, N):
        key[:, u] = np.maximum(key[:, u], key[:, parent[u]] + 1e-9)
    rank = np.argsort(np.argsort(key, axis=1, kind="stable"), axis=1)
    return rank < np.array(_kept(case))[:, None]


def _spread(lo, hi, B, rs=None):
    """A number between lo and hi for each trajectory, the same set for every seed, in an order of the seed's."""
    n = np.array([lo + int(round((hi - lo) * ((0.5 + b * 0.754878) % 1.0))) for b in range(B)], np.int64)
    if B > 1:
        n[0], n[1] = lo, hi
    return n if rs is None else n[rs.permutation(B)]


def _table(tokens, page, rs):
    """(table, pages) for so many tokens of each trajectory on pages from anywhere; behind them a row holds what was there before."""
    per = -(-tokens // page)
    width, pages = int(max(1, per.max() + 1)), int(per.sum()) + 3
    order = rs.permutation(pages)
    table = rs.randint(0, pages, (len(tokens), width))
    at = 0
    for b in range(len(tokens)):
        table[b, :per[b]] = order[at:at + per[b]]
        at += per[b]
    return table, pages


# ---- four bits ----------------------------------------------------------------------------------------------------------
# A block is 32 neighbouring elements of a head.  Its scale is a power of two, 2^(s - 127) with s in a byte: that of the largest
# magnitude, rounded to two significant bits, divided by four (so that it comes to lie at 4 or 6, or below 7 and is held as 6).
# An element is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times the scale (ties to the even code), with a sign.

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# smallest and largest scale: products are numbers of the rows' type, without loss
_LOW, _HIGH = {"bf16": 127 - 125, "f16": 127 - 23}, {"bf16": 127 + 125, "f16": 127 + 13}


def _power(s):
    """2^(s - 127), fp32."""
    return (s.to(torch.int32) << 23).view(torch.float32)


def _codes(x, dtype):
    """fp32 [..., d] -> (codes 0 .. 15 [..., d], scales [..., d / 32]), both bytes."""
    y = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    s = torch.clamp(((y.abs().amax(dim=-1).view(torch.int32) + 0x200000) >> 23) - 2, min=_LOW[dtype], max=_HIGH[dtype])
    a = y.abs() * _power(254 - s[..., None])
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.clamp(torch.round(a / step) * step, max=6.0)
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4))
    code = code.to(torch.uint8) + 8 * (y < 0).to(torch.uint8)
    return code.reshape(x.shape), s.to(torch.uint8)


def _packed(x, dtype):
    """fp32 [..., d] -> (bytes of two elements, the first one in the low half [..., d / 2], scales [..., d / 32])."""
    code, s = _codes(x, dtype)
    return code[..., 0::2] | (code[..., 1::2] << 4), s


def _unpacked(p, s):
    """The values of packed codes and scales, fp32."""
    code = torch.stack([p & 15, p >> 4], dim=-1).reshape(*s.shape, 32).long()
    g = torch.tensor(_GRID + tuple(-v for v in _GRID), dtype=torch.float32, device=p.device)[code]
    return (g * _power(s[..., None])).reshape(*p.shape[:-1], 2 * p.shape[-1])


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _handle(B, parent):
    from paper_2506_04708_amd import binding
    fan = int(np.bincount(parent[1:]).max()) if len(parent) > 1 else 1
    return binding.Stand(64, B, 1, 2, min(32, max(fan, 8)), parent, 0.6, 64, 8, 1, binding.STAND_BF16)


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _laid(x, layout):
    """[layers, pages, page, heads, ...] of that order in memory."""
    return x if layout == "nhd" else x.transpose(2, 3).contiguous().transpose(2, 3)


def _pool16(case, layers, pages, gen):
    out = []
    for _ in range(2):
        x = torch.empty((layers, pages, case["page"], case["Hkv"], case["d"]), dtype=_DT[case["dtype"]], device="cuda")
        for l in range(layers):
            x[l].normal_(generator=gen)
        out.append(_laid(x, case["layout"]))
    return out


def _pool4(case, layers, pages, gen):
    """What normal keys and values become in 4 bits: keys, values and their scales."""
    page, Hkv, d = case["page"], case["Hkv"], case["d"]
    out = []
    for _ in range(2):
        p = torch.empty((layers, pages, page, Hkv, d // 2), dtype=torch.uint8, device="cuda")
        s = torch.empty((layers, pages, page, Hkv, d // 32), dtype=torch.uint8, device="cuda")
        some = max(1, (1 << 26) // (page * Hkv * d))
        for l in range(layers):
            for a in range(0, pages, some):
                x = torch.empty((min(some, pages - a), page, Hkv, d), device="cuda").normal_(generator=gen)
                p[l, a:a + some], s[l, a:a + some] = _packed(x, case["dtype"])
        out.append((_laid(p, case["layout"]), _laid(s, case["layout"])))
    (kp, ks), (vp, vs) = out
    return kp, vp, ks, vs


def _qkv(case, B, R, gen):
    """Queries, keys and values as projections leave them: slices of one tensor, or three."""
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    dt = dict(dtype=_DT[case["dtype"]], device="cuda")
    if case["fused"]:
        x = torch.empty((B, R, Hq + 2 * Hkv, d), **dt).normal_(generator=gen)
        return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    return tuple(torch.empty((B, R, h, d), **dt).normal_(generator=gen) for h in (Hq, Hkv, Hkv))


def _turns(case, most, gen):
    """cos and sin of the positions 0 .. most - 1 (angles in 64 bits), [cos | sin] of half of `dims`, and the norms' weights."""
    half = case["dims"] // 2
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    angle = torch.arange(most, dtype=torch.float64, device="cuda")[:, None] * freq
    table = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    q = k = None
    if case["norm"]:
        q, k = ((1.0 + 0.2 * torch.empty(case["d"], device="cuda").normal_(generator=gen)).to(_DT[case["dtype"]]) for _ in range(2))
    return dict(turns=table, q_norm=q, k_norm=k, eps=1e-6)


def _rotation(st):
    from paper_2506_04708_amd import binding
    return binding.Rotation(st["turns"], st["case"]["pairs"], st["q_norm"], st["k_norm"], st["eps"])


def _cache(st):
    from paper_2506_04708_amd import binding
    if "ks" in st:
        return binding.PagedCache(st["kp"], st["vp"], st["ks"], st["vs"], dtype=_DT[st["case"]["dtype"]])
    return binding.PagedCache(st["kp"], st["vp"])


def prepare(case, seed):
    seed = int(seed) & 0x7FFFFFFF
    rs, gen = np.random.RandomState(seed), torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case)
    {"rotate": _prepare_rotate, "append": _prepare_append, "commit": _prepare_commit, "attn": _prepare_attn}[case["op"]](st, case, rs, gen)
    return st


def _prepare_tree(st, case, rs):
    parent = _tree(case["N"], case["D"], case["fan"])
    drafted = _drafted(case, parent, rs)
    n = _spread(case["lo"], case["hi"], case["B"], rs)
    st.update(parent=parent, drafted=drafted, lens=n, length=_i32(n), tok=_i32(np.where(drafted, rs.randint(0, 64, drafted.shape), -1)))
    if own:
        st["h"] = _handle(case["B"], parent)


def _prepare_rotate(st, case, rs, gen):
    _prepare_tree(st, case, rs)
    B, N = st["tok"].shape
    st["q"], st["k"], _ = _qkv(case, B, N, gen)
    st.update(_turns(case, case["hi"] + case["D"] + 1, gen))
    # rows of nodes that are not drafted are left as they were
    st["q_out"], st["k_out"] = torch.zeros_like(st["q"].contiguous()), torch.zeros_like(st["k"].contiguous())
    st["depth"] = torch.from_numpy(_depth(st["parent"])).cuda()
    if own:
        st["rotation"] = _rotation(st)


def _prepare_append(st, case, rs, gen):
    B, R, page = case["B"], case["R"], case["page"]
    first, count = _spread(case["lo"], case["hi"], B, rs), _spread(case["rlo"], R, B, rs)
    table, pages = _table(first + count, page, rs)
    pos = first[:, None] + np.arange(R)
    slots = np.take_along_axis(table, np.minimum(pos // page, table.shape[1] - 1), axis=1) * page + pos % page
    slots = np.where(np.arange(R) < count[:, None], slots, -1)
    st["q"], st["k"], st["v"] = _qkv(case, B, R, gen)
    st.update(_turns(case, case["hi"] + R, gen))
    # rows behind a trajectory's last one are left as they were
    st["q_out"] = torch.zeros(st["q"].shape, dtype=st["q"].dtype, device="cuda")
    st.update(slots=torch.from_numpy(slots).cuda(), start=_i32(first), count=_i32(count), table=_i32(table), pos=torch.from_numpy(pos).cuda(),
              first=first, counts=count)
    if case["bits"] == 4:
        st["kp"], st["vp"], st["ks"], st["vs"] = _pool4(case, 1, pages, gen)
        st["back"] = torch.zeros((2, 1, B, case["hi"] + R, case["Hkv"], case["d"]), dtype=_DT[case["dtype"]], device="cuda")
        st["total"] = _i32(first + count)
    else:
        st["kp"], st["vp"] = _pool16(case, 1, pages, gen)
    if own:
        st["h"] = _handle(B, np.arange(-1, 0, dtype=np.int32))
        st["rotation"], st["cache"] = _rotation(st), _cache(st)
    else:
        st["which"] = [torch.from_numpy(x).cuda() for x in np.nonzero(np.arange(R)[None] < count[:, None])]


def _prepare_commit(st, case, rs, gen):
    layers, B, R, W, Hkv, d, page = (case[k] for k in ("layers", "B", "R", "W", "Hkv", "d", "page"))
    first, count = _spread(case["lo"], case["hi"], B, rs), _spread(case["rlo"], W, B, rs)
    table, pages = _table(first + count, page, rs)
    pos = first[:, None] + np.arange(W)
    slots = np.take_along_axis(table, np.minimum(pos // page, table.shape[1] - 1), axis=1) * page + pos % page
    slots = np.where(np.arange(W) < count[:, None], slots, -1)
    st["kp"], st["vp"], st["ks"], st["vs"] = _pool4(case, layers, pages, gen)
    # what the layers' projections left behind, keys and values of a row beside each other
    kv = torch.empty((layers, B, R, 2, Hkv, d), dtype=_DT[case["dtype"]], device="cuda")
    for l in range(layers):
        kv[l].normal_(generator=gen)
    row = np.full((B, W), -1, np.int32)
    for b in range(B):                               # increasing nodes, the root first
        n = int(count[b])
        if n:
            row[b, :n] = np.concatenate([[0], 1 + np.sort(rs.choice(R - 1, n - 1, replace=False))]) if n > 1 else 0
    st.update(k=kv[:, :, :, 0], v=kv[:, :, :, 1], slots=torch.from_numpy(slots).cuda(), row=_i32(row) if case["path"] else None, count=_i32(count),
              start=_i32(first), table=_i32(table), first=first, counts=count,
              back=torch.zeros((2, layers, B, W, Hkv, d), dtype=_DT[case["dtype"]], device="cuda"))
    if own:
        st["h"] = _handle(B, np.arange(-1, min(W, 32) - 1, dtype=np.int32))
        st["cache"] = _cache(st)
    else:
        st["which"] = [torch.from_numpy(x).cuda() for x in np.nonzero(np.arange(W)[None] < count[:, None])]


def _prepare_attn(st, case, rs, gen):
    _prepare_tree(st, case, rs)
    B, N = st["tok"].shape
    table, pages = _table(st["lens"], case["page"], rs)
    st["kp"], st["vp"], st["ks"], st["vs"] = _pool4(case, 1, pages, gen)
    st["q"], st["k"], st["v"] = _qkv(case, B, N, gen)
    st["q"].mul_(2.0)                                # queries that meet some keys far better than others: scores of a deviation of two
    st.update(table=_i32(table), scale=case["d"] ** -0.5, out=torch.empty((B, N, case["Hq"], case["d"]), dtype=_DT[case["dtype"]], device="cuda"))
    if own:
        st["cache"] = _cache(st)
    else:
        st["anc"] = torch.from_numpy(_ancestors(st["parent"])).cuda()


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(st):
    return {"rotate": _run_rotate, "append": _run_append, "commit": _run_commit, "attn": _run_attn}[st["case"]["op"]](st)


def _turned(x, pos, weight, st, pairs):
    """Rows x [..., heads, d] at positions pos [...]: normed, then rotated, in 64 bits (what is held in 4 is decided next to borders)."""
    x, turns = x.double(), st["turns"]
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + st["eps"]) * weight.double()
    half = turns.shape[1] // 2
    cs = turns[pos].double()[..., None, :]
    cos, sin = cs[..., :half], cs[..., half:]
    y = x.clone()
    if pairs == "halves":
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, b * cos + a * sin
    return y.float()


def _run_rotate(st):
    if own:
        st["h"].tree_rotate(st["rotation"], st["length"], st["tok"], st["q"], st["k"], st["q_out"], st["k_out"])
        return st["q_out"], st["k_out"]
    drafted = (st["tok"] >= 0)[:, :, None, None]
    pos = st["length"].long()[:, None] + st["depth"]
    for x, w, out in ((st["q"], st["q_norm"], st["q_out"]), (st["k"], st["k_norm"], st["k_out"])):
        out.copy_(torch.where(drafted, _turned(x, pos, w, st, st["case"]["pairs"]), out))
    return st["q_out"], st["k_out"]


def _read_plain(st, first, count):
    """The tokens first .. first + count - 1 of each trajectory, from all layers, into st["back"] [2, layers, B, rows, heads, d]."""
    case, back = st["case"], st["back"]
    page, rows = case["page"], back.shape[3]
    j = torch.arange(rows, device="cuda")[None]
    pos = (first[:, None] if first is not None else 0) + j
    at = torch.gather(st["table"].long(), 1, torch.clamp(pos // page, max=st["table"].shape[1] - 1).expand(case["B"], rows))
    there = (j < count[:, None])[:, :, None, None]
    for i, (p, s) in enumerate(((st["kp"], st["ks"]), (st["vp"], st["vs"]))):
        place = (pos % page).expand(case["B"], rows)
        back[i].copy_(torch.where(there, _unpacked(p[:, at, place], s[:, at, place]), back[i]))
    return back


def _run_append(st):
    case = st["case"]
    if own:
        st["h"].cache_append(st["cache"], 0, st["k"], st["v"], st["slots"], st["start"], st["count"], st["rotation"], st["q"], st["q_out"])
        if case["bits"] == 16:
            return st["q_out"], st["kp"], st["vp"]
        st["h"].cache_read(st["cache"], st["table"], st["back"][0], st["back"][1], st["total"])
        return st["q_out"], st["back"]
    b, j = st["which"]
    pos, at = st["pos"][b, j], st["slots"][b, j]
    page = case["page"]
    st["q_out"][b, j] = _turned(st["q"][b, j], pos, st["q_norm"], st, case["pairs"]).to(st["q"].dtype)
    k, v = _turned(st["k"][b, j], pos, st["k_norm"], st, case["pairs"]), st["v"][b, j]
    if case["bits"] == 16:
        st["kp"][0, at // page, at % page] = k.to(st["k"].dtype)
        st["vp"][0, at // page, at % page] = v
        return st["q_out"], st["kp"], st["vp"]
    for x, p, s in ((k, st["kp"], st["ks"]), (v.float(), st["vp"], st["vs"])):
        p[0, at // page, at % page], s[0, at // page, at % page] = _packed(x, case["dtype"])
    return st["q_out"], _read_plain(st, None, st["total"].long())


def _run_commit(st):
    case = st["case"]
    if own:
        st["h"].cache_commit(st["cache"], st["k"], st["v"], st["slots"], st["row"], st["count"])
        st["h"].cache_read(st["cache"], st["table"], st["back"][0], st["back"][1], st["count"], st["start"])
        return st["back"]
    page = case["page"]
    b, j = st["which"]
    at = st["slots"][b, j]
    row = st["row"][b, j].long() if st["row"] is not None else j
    for x, p, s in ((st["k"], st["kp"], st["ks"]), (st["v"], st["vp"], st["vs"])):
        p[:, at // page, at % page], s[:, at // page, at % page] = _packed(x[:, b, row].float(), case["dtype"])
    return _read_plain(st, st["start"].long(), st["count"].long())


def _run_attn(st):
    if own:
        return st["h"].tree_attention(st["cache"], 0, st["length"], st["table"], st["tok"], st["q"], st["k"], st["v"], st["scale"], st["out"])
    # all trajectories at once, as long as the longest: what lies behind a length is masked
    case = st["case"]
    Hq, Hkv, d, page = case["Hq"], case["Hkv"], case["d"], case["page"]
    B, N = st["tok"].shape
    G, most = Hq // Hkv, case["hi"]
    ids = st["table"][:, : -(-most // page)].long()

    def rows(p, s, new):                             # [B, Hkv, most + N, d]
        old = _unpacked(p[0][ids], s[0][ids]).reshape(B, -1, Hkv, d)[:, :most]
        return torch.cat([old, new.float()], dim=1).transpose(1, 2)

    see = torch.cat([(torch.arange(most, device="cuda") < st["length"][:, None])[:, None].expand(B, N, most),
                     st["anc"].expand(B, N, N)], dim=2) & (st["tok"] >= 0)[:, :, None]
    see = see.repeat_interleave(G, dim=1)[:, None]   # [B, 1, N G, most + N]
    q = st["q"].float().reshape(B, N, Hkv, G, d).transpose(1, 2).reshape(B, Hkv, N * G, d)
    s = torch.matmul(q, rows(st["kp"], st["ks"], st["k"]).transpose(2, 3).contiguous()) * st["scale"]
    s = torch.where(see, s, -math.inf)
    m = s.amax(dim=3, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
    t = p.sum(dim=3, keepdim=True)
    o = torch.matmul(p, rows(st["vp"], st["vs"], st["v"])) / torch.where(t > 0, t, 1.0)
    st["out"].copy_(o.reshape(B, Hkv, N, G, d).transpose(1, 2).reshape(B, N, Hq, d))
    return st["out"]


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    B, Hkv, d = case["B"], case["Hkv"], case["d"]
    four = d / 2 + d / 32                            # bytes of a head's row in 4 bits
    if case["op"] == "rotate":
        rows, heads = float(sum(_kept(case))), case["Hq"] + Hkv
        return {"bytes": rows * heads * d * 4.0 + (case["D"] + B) * 4.0 * case["dims"], "flops": rows * heads * (3.0 * case["dims"] + (3.0 * d if case["norm"] else 0.0))}
    if case["op"] == "append":
        count, first = _spread(case["rlo"], case["R"], B), _spread(case["lo"], case["hi"], B)
        n = float(max(1, count.sum()))
        turned = n * (case["Hq"] + Hkv) * (3.0 * case["dims"] + (3.0 * d if case["norm"] else 0.0))
        held = 2.0 * d if case["bits"] == 16 else four
        bytes_ = n * (case["Hq"] * 4.0 * d + 2 * Hkv * (2.0 * d + held)) + 4.0 * case["dims"] * min(n, case["hi"] + case["R"])
        if case["bits"] == 4:
            bytes_ += 2.0 * Hkv * (four + 2.0 * d) * float((first + count).sum())
        return {"bytes": bytes_, "flops": turned}
    if case["op"] == "commit":
        n = float(max(1, _spread(case["rlo"], case["W"], B).sum()))
        return {"bytes": n * case["layers"] * Hkv * 2 * 2 * (2.0 * d + four), "flops": 0.0}
    Hq = case["Hq"]
    n, kept = _spread(case["lo"], case["hi"], B), np.array(_kept(case))
    pairs = float((n * kept).sum() + kept.sum() * (1 + case["D"] / 2))
    rows = float(kept.sum())
    return {"bytes": 2.0 * Hkv * four * n.sum() + 4.0 * (Hkv + Hq) * d * rows, "flops": 4.0 * d * Hq * pairs}


# ---- the operators in 64 bits, from their definitions -------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"rotate": _exact_rotate, "append": _exact_append, "commit": _exact_commit, "attn": _exact_attn}[case["op"]](case, st)


def _complex_turn(case, st, x, pos, weight):
    """Pairs as complex numbers, times e^(i angle)."""
    x = x.double()
    if weight is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + st["eps"]).sqrt() * weight.double()
    half = case["dims"] // 2
    e = torch.complex(st["turns"][pos, :half].double(), st["turns"][pos, half:].double()).unsqueeze(-2)
    if case["pairs"] == "halves":
        z = torch.complex(x[..., :half], x[..., half:2 * half]) * e
        return torch.cat([z.real, z.imag, x[..., 2 * half:]], dim=-1)
    z = torch.view_as_complex(x[..., :2 * half].reshape(*x.shape[:-1], half, 2)) * e
    return torch.cat([torch.view_as_real(z).flatten(-2), x[..., 2 * half:]], dim=-1)


def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest4(x, dtype):
    """Each element's nearest value in its block, found among all of them."""
    y = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = y.abs().amax(dim=-1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    e = e + (top * _two_to(-e) >= 1.75).double() - 2
    unit = _two_to(torch.where(top > 0, e, -1e9).clamp(_LOW[dtype] - 127, _HIGH[dtype] - 127))
    best, off = torch.zeros_like(y), y.abs() / unit
    for code in (1, 2, 3, 4, 5, 6, 7):
        here = (y.abs() / unit - _GRID[code]).abs()
        better = (here < off) if code % 2 else (here <= off)      # ties go to the even code
        best, off = torch.where(better, _GRID[code], best), torch.where(better, here, off)
    return (torch.sign(y) * best * unit).reshape(x.shape)


def _exact_rotate(case, st):
    out = []
    for x, w in ((st["q"], st["q_norm"]), (st["k"], st["k_norm"])):
        y = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        for b in range(case["B"]):
            nodes = torch.from_numpy(np.nonzero(st["drafted"][b])[0]).cuda()
            y[b, nodes] = _complex_turn(case, st, x[b, nodes], int(st["lens"][b]) + st["depth"][nodes], w)
        out.append(y)
    return tuple(out)


def _tokens_of(st, pool, l, b, a, z):
    """Rows a .. z - 1 of trajectory b in layer l of a pool of any kind."""
    page = st["case"]["page"]
    pos = torch.arange(a, z, device="cuda")
    return pool[l, st["table"][b].long()[pos // page], pos % page]


def _value4(p, s):
    """Values of packed codes, by their bits: sign, two of exponent, one of fraction."""
    x = torch.empty((*p.shape[:-1], p.shape[-1] * 2), dtype=torch.float64, device=p.device)
    for i in (0, 1):
        c = (p.long() >> (4 * i)) & 15
        e, f = (c >> 1) & 3, (c & 1).double()
        mag = torch.where(e == 0, f / 2, (1 + f / 2) * _two_to(e - 1))
        x[..., i::2] = torch.where(c >= 8, -mag, mag)
    return x * _two_to(s.long() - 127).repeat_interleave(32, dim=-1)


def _exact_append(case, st):
    Hkv, d = case["Hkv"], case["d"]
    q_out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    if case["bits"] == 16:
        kp, vp = st["kp"].double(), st["vp"].double()
    else:
        back = torch.zeros(st["back"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        first, n = int(st["first"][b]), int(st["counts"][b])
        pos = first + torch.arange(n, device="cuda")
        q_out[b, :n] = _complex_turn(case, st, st["q"][b, :n], pos, st["q_norm"])
        k, v = _complex_turn(case, st, st["k"][b, :n], pos, st["k_norm"]), st["v"][b, :n].double()
        if case["bits"] == 16:
            at, place = st["table"][b].long()[pos // case["page"]], pos % case["page"]
            kp[0, at, place], vp[0, at, place] = k, v
            continue
        for i, (new, p, s) in enumerate(((k, st["kp"], st["ks"]), (v, st["vp"], st["vs"]))):
            back[i, 0, b, :first] = _value4(_tokens_of(st, p, 0, b, 0, first), _tokens_of(st, s, 0, b, 0, first))
            back[i, 0, b, first:first + n] = _nearest4(new, case["dtype"])
    return (q_out, kp, vp) if case["bits"] == 16 else (q_out, back)


def _exact_commit(case, st):
    back = torch.zeros(st["back"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["B"]):
        n = int(st["counts"][b])
        rows = st["row"][b, :n].long() if st["row"] is not None else torch.arange(n, device="cuda")
        for i, x in enumerate((st["k"], st["v"])):
            if n:
                back[i, :, b, :n] = _nearest4(x[:, b, rows], case["dtype"])
    return back


def _exact_attn(case, st):
    """Node by node along its own path: softmax over the cached tokens and the path's tokens, no mask."""
    parent = st["parent"]
    G, Hkv = case["Hq"] // case["Hkv"], case["Hkv"]
    B, N = st["tok"].shape
    deep = int(_depth(parent).max()) + 1
    path = np.full((N, deep), -1, np.int64)
    for u in range(N):
        at, v = 0, u
        while v >= 0:
            path[u, at] = v
            at, v = at + 1, int(parent[v])
    path = torch.from_numpy(path).cuda()
    out = torch.zeros((B, N, case["Hq"], case["d"]), dtype=torch.float64, device="cuda")
    for b in range(B):
        nodes = torch.from_numpy(np.nonzero(st["drafted"][b])[0]).cuda()
        n = int(st["lens"][b])
        along = path[nodes]                          # [n, deep]
        K, V = (_value4(_tokens_of(st, p, 0, b, 0, n), _tokens_of(st, s, 0, b, 0, n)) for p, s in ((st["kp"], st["ks"]), (st["vp"], st["vs"])))
        for h in range(Hkv):
            Kt, Vt = st["k"][b, :, h].double()[along.clamp(min=0)], st["v"][b, :, h].double()[along.clamp(min=0)]
            Kh, Vh = K[:, h].contiguous(), V[:, h].contiguous()
            for g in range(G):
                q = st["q"][b, nodes, h * G + g].double() * st["scale"]
                a = q @ Kh.t()
                t = (q[:, None, :] * Kt).sum(dim=2).masked_fill(along < 0, -math.inf)
                top = t.amax(dim=1) if n == 0 else torch.maximum(a.amax(dim=1), t.amax(dim=1))
                a, t = torch.exp(a - top[:, None]), torch.exp(t - top[:, None])
                o = a @ Vh + (t[:, :, None] * Vt).sum(dim=1)
                out[b, nodes, h * G + g] = o / (a.sum(dim=1) + t.sum(dim=1))[:, None]
    return out

"""The operators around a verification of drafted trees, as cases that can be timed and compared.

Between two target model passes a server that drafts trees does four things beside the speculation step itself, all on
data that only the GPU knows (how many tokens were accepted, which nodes were drafted), so that the host never waits:

  attn    attention of the drafted tree's nodes over a paged key/value cache and over their own ancestors in the tree
  commit  the accepted path's keys and values of all layers go to their slots in the paged cache
  pages   lengths move on, pages are taken from and given back to a ring of free ones, block tables and slot maps follow
  shape   repetition, presence and frequency penalties, biases and grammar masks on the logits of every node

`own` selects what `run` calls: the plain forms below (elementary torch operations in 32 bits), or the framework's
operators.  A tree is the breadth-first `parent` list of the framework; node 0 is the last committed token.
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---- cases ------------------------------------------------------------------------------------------------------------

def _attn(name, B, N, D, fan, drafted, lo, hi, Hq, Hkv, d, page, dtype="bf16", layout="nhd", fused=False):
    return dict(name=name, op="attn", B=B, N=N, D=D, fan=fan, drafted=drafted, lo=lo, hi=hi, Hq=Hq, Hkv=Hkv, d=d, page=page,
                dtype=dtype, layout=layout, fused=fused)


def _commit(name, layers, B, R, W, lo, hi, Hkv, d, page, pool, dtype="bf16", layout="nhd", path=True):
    return dict(name=name, op="commit", layers=layers, B=B, R=R, W=W, lo=lo, hi=hi, Hkv=Hkv, d=d, page=page, pool=pool,
                dtype=dtype, layout=layout, path=path)


def _pages(name, B, page, width, lo, hi, add, room, leave, W, spare):
    return dict(name=name, op="pages", B=B, page=page, width=width, lo=lo, hi=hi, add=add, room=room, leave=leave, W=W, spare=spare)


def _shape(name, B, N, D, fan, drafted, V, dtype="bf16", bias=0, mask=True, prompt=0):
    return dict(name=name, op="shape", B=B, N=N, D=D, fan=fan, drafted=drafted, V=V, dtype=dtype, bias=bias, mask=mask, prompt=prompt)


def listed():
    return [
        # one short request on a small model: nothing but launches and dependent round trips
        _attn("attn_short", 1, 16, 4, "4-2-1-1", 0.8, 37, 37, 14, 2, 64, 16, "f16"),
        # one user with a long reasoning trace, a tree of 32 nodes: few heads, a long axis
        _attn("attn_single", 1, 32, 6, "4-2-2-1", 0.8, 30001, 30001, 28, 4, 128, 16, "bf16", "nhd", True),
        # best-of-32 in the middle of its run, trajectories of very different lengths
        _attn("attn_best32", 32, 64, 8, "8-4-2-1", 0.75, 1000, 9000, 28, 4, 128, 64),
        # single tokens (a tree of one node) of 64 requests, from an empty cache to long ones: the cache is read once
        _attn("attn_decode", 64, 1, 0, "1", 1.0, 0, 16000, 32, 8, 128, 32, "bf16", "hnd"),
        # tree search over 128 beams, large trees, short caches, 64 wide heads
        _attn("attn_beams", 128, 128, 10, "8-4-2-1", 0.6, 200, 3000, 16, 8, 64, 16, "f16", "nhd", True),
        # the accepted paths of a step: one to nine tokens of each trajectory, 28 layers
        _commit("commit_step", 28, 32, 64, 9, 1, 9, 4, 128, 64, 8192),
        # prompts go into the cache, in the order they stand
        _commit("commit_prompt", 16, 4, 2100, 2100, 900, 2100, 8, 128, 16, 12000, "f16", "hnd", False),
        # a step of best-of-32: few tokens more each, a few pages taken
        _pages("pages_step", 32, 16, 1024, 100, 12000, 9, 9, 0.03, 9, 2000),
        # 512 requests, a fifth of them leave or come with prompts of up to 4000 tokens
        _pages("pages_admit", 512, 16, 600, 0, 5000, 0, 4000, 0.2, 4000, 90000),
        # one request on a small model, fp32 logits, no grammar
        _shape("shape_tiny", 1, 16, 4, "4-2-1-1", 0.8, 32000, "f32", 3, False),
        # best-of-32 under a grammar
        _shape("shape_best32", 32, 64, 8, "8-4-2-1", 0.75, 152064, "bf16", 16),
        # the first logits of 64 requests: their prompts are counted, rows of an odd vocabulary are shaped
        _shape("shape_first", 64, 1, 0, "1", 1.0, 50257, "bf16", 300, True, 4000),
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


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "commit", "pages", "shape"])
    if op == "attn":
        N, D, fan = _draw_tree(rng, 300)
        B = _log_uniform(rng, 1, 128)
        Hkv = rng.choice([1, 2, 3, 4, 8])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 5, 7, 8])
        d = rng.choice([64, 128])
        hi = _log_uniform(rng, 1, 40000)
        lo = rng.choice([0, hi // 9, hi])
        c = _attn("", B, N, D, fan, rng.choice([0.3, 0.6, 0.8, 1.0]), lo, hi, Hq, Hkv, d, rng.choice([8, 16, 32, 64, 128]),
                  rng.choice(["bf16", "f16"]), rng.choice(["nhd", "hnd"]), rng.random() < 0.5)
        while work(c)["flops"] > 6.5e10 or work(c)["bytes"] > 1.3e9:
            c["B"] = c["B"] // 2
            if c["B"] == 0:
                c["B"], c["hi"] = 1, max(1, c["hi"] // 2)
                c["lo"] = min(c["lo"], c["hi"])
    elif op == "commit":
        path = rng.random() < 0.6
        N, D, _ = _draw_tree(rng, 160)
        W = D + 1 if path else _log_uniform(rng, 1, 3000)
        B = _log_uniform(rng, 1, 128 if path else 8)
        Hkv, d, layers = rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 128]), _log_uniform(rng, 1, 48)
        R = N if path else W
        while layers * B * R * Hkv * d > 16 * 4 * 2100 * 8 * 128:
            layers, B = max(1, layers // 2), max(1, B // 2)
        c = _commit("", layers, B, R, W, rng.choice([0, 1, W]), W, Hkv, d, rng.choice([8, 16, 64]), B * W + _log_uniform(rng, 200, 4000),
                    rng.choice(["bf16", "f16"]), rng.choice(["nhd", "hnd"]), path)
    elif op == "pages":
        page = rng.choice([8, 16, 64, 128])
        hi = _log_uniform(rng, 20, 20000)
        step = rng.random() < 0.5
        W = rng.randint(2, 13) if step else _log_uniform(rng, 10, 4000)
        B = _log_uniform(rng, 1, 512)
        width = -(-(hi + W + 32) // page)
        while B * width > 512 * 600 or B * W > 512 * 4000:
            B //= 2
        c = _pages("", max(1, B), page, width - (width // 8 if rng.random() < 0.2 else 0), 0, hi, W if step else 0, W, rng.choice([0.0, 0.05, 0.3]), W,
                   rng.choice([0, 10, B * -(-W // page) + B]))
    else:
        N, D, fan = _draw_tree(rng, 160)
        V = _log_uniform(rng, 1000, 200000)
        if rng.random() < 0.4:
            V -= V % 64
        B = _log_uniform(rng, 1, 128)
        while B * N * V > 32 * 64 * 152064:
            B = max(1, B // 2)
            N = N if B > 1 else max(D + 1, min(N, 64))
        c = _shape("", B, N, D, fan, rng.choice([0.3, 0.7, 1.0]), V, rng.choice(["bf16", "bf16", "f32"]), rng.choice([0, 0, 5, 300]),
                   rng.random() < 0.6, rng.choice([0, 0, _log_uniform(rng, 1, 8000)]))
        if c["dtype"] == "f32" and B * N * V > 16 * 64 * 152064:
            c["dtype"] = "bf16"
    del c["name"]
    return c


# ---- trees and lengths ------------------------------------------------------------------------------------------------

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


def _lengths(case, rs=None):
    """A length between lo and hi for each trajectory, the same set for every seed, in an order of the seed's."""
    lo, hi, B = case["lo"], case["hi"], case["B"]
    n = np.array([lo + int(round((hi - lo) * ((0.5 + b * 0.754878) % 1.0))) for b in range(B)], np.int64)
    if B > 1:
        n[0], n[1] = lo, hi
    return n if rs is None else n[rs.permutation(B)]


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _handle(case, parent, V=64, dtype="bf16"):
    from paper_2506_04708_amd import binding
    fan = int(np.bincount(parent[1:]).max()) if len(parent) > 1 else 1
    return binding.Stand(V, case["B"], 1, 2, min(32, max(fan, 8)), parent, 0.6, 64, 8, 1,
                         binding.STAND_F32 if dtype == "f32" else binding.STAND_BF16)


def _pool(case, layers, pages, gen):
    """Keys and values of a paged cache, indexed [layer, page, slot, head, element] whatever the order in memory."""
    Hkv, d, page = case["Hkv"], case["d"], case["page"]
    shape = (layers, pages, page, Hkv, d) if case["layout"] == "nhd" else (layers, pages, Hkv, page, d)
    out = []
    for _ in range(2):
        x = torch.empty(shape, dtype=_DT[case["dtype"]], device="cuda")
        for l in range(layers):
            x[l].normal_(generator=gen)
        out.append(x if case["layout"] == "nhd" else x.transpose(2, 3))
    return out


def prepare(case, seed):
    seed = int(seed)
    rs = np.random.RandomState(seed & 0x7FFFFFFF)
    gen = torch.Generator(device="cuda").manual_seed(seed & 0x7FFFFFFF)
    st = dict(case=case)
    {"attn": _prepare_attn, "commit": _prepare_commit, "pages": _prepare_pages, "shape": _prepare_shape}[case["op"]](st, case, rs, gen)
    return st


def _prepare_attn(st, case, rs, gen):
    B, N, Hq, Hkv, d, page = (case[k] for k in ("B", "N", "Hq", "Hkv", "d", "page"))
    parent = _tree(N, case["D"], case["fan"])
    N = len(parent)
    n = _lengths(case, rs)
    per = -(-n // page)
    width = int(max(1, per.max() + 1))
    pages = int(per.sum()) + 3
    order = rs.permutation(pages)
    table = rs.randint(0, pages, (B, width))         # past its pages a row of the table holds what was there before
    at = 0
    for b in range(B):
        table[b, :per[b]] = order[at:at + per[b]]
        at += per[b]
    kp, vp = _pool(case, 1, pages, gen)
    dt = _DT[case["dtype"]]
    # queries that meet some keys far better than others: scores of a deviation of two
    if case["fused"]:
        qkv = torch.empty((B, N, Hq + 2 * Hkv, d), dtype=dt, device="cuda").normal_(generator=gen)
        qkv[:, :, :Hq].mul_(2.0)
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    else:
        q = torch.empty((B, N, Hq, d), dtype=dt, device="cuda").normal_(generator=gen).mul_(2.0)
        k = torch.empty((B, N, Hkv, d), dtype=dt, device="cuda").normal_(generator=gen)
        v = torch.empty((B, N, Hkv, d), dtype=dt, device="cuda").normal_(generator=gen)
    drafted = _drafted(case, parent, rs)
    tok = np.where(drafted, rs.randint(0, 64, drafted.shape), -1).astype(np.int32)
    i32 = dict(dtype=torch.int32, device="cuda")
    st.update(parent=parent, lens=n, drafted=drafted, kp=kp, vp=vp, q=q, k=k, v=v, scale=d ** -0.5,
              tok=torch.tensor(tok, **i32), length=torch.tensor(n, **i32), table=torch.tensor(table, **i32),
              out=torch.empty((B, N, Hq, d), dtype=dt, device="cuda"))
    if own:
        from paper_2506_04708_amd import binding
        st["h"] = _handle(case, parent)
        st["cache"] = binding.PagedCache(kp, vp)
    else:
        st["anc"] = torch.from_numpy(_ancestors(parent)).cuda()


def _prepare_commit(st, case, rs, gen):
    layers, B, R, W, Hkv, d, page = (case[k] for k in ("layers", "B", "R", "W", "Hkv", "d", "page"))
    pages = -(-max(case["pool"], B * W) // page)
    kp, vp = _pool(case, layers, pages, gen)
    dt = _DT[case["dtype"]]
    # what the layers' projections left behind, keys and values of a row beside each other
    kv = torch.empty((layers, B, R, 2, Hkv, d), dtype=dt, device="cuda")
    for l in range(layers):
        kv[l].normal_(generator=gen)
    n = _lengths(case, rs)
    # consecutive positions of a trajectory, on pages from anywhere: distinct slots
    slots = np.full((B, W), -1, np.int64)
    order = rs.permutation(pages)
    at = 0
    for b in range(B):
        first = rs.randint(0, page)
        pos = first + np.arange(W)
        need = int(pos[-1] // page) + 1
        if at + need > pages:
            first, pos, need = 0, np.arange(W), -(-W // page)
        if at + need > pages:
            n[b] = 0
            continue
        slots[b] = order[at + pos // page] * page + pos % page
        at += need
    row = np.full((B, W), -1, np.int32)
    for b in range(B):                               # increasing nodes, the root first
        if n[b]:
            row[b, :n[b]] = np.concatenate([[0], 1 + np.sort(rs.choice(R - 1, n[b] - 1, replace=False))]) if n[b] > 1 else 0
    st.update(kp=kp, vp=vp, k=kv[:, :, :, 0], v=kv[:, :, :, 1], lens=n, slots=torch.from_numpy(slots).cuda(),
              row=torch.from_numpy(row).cuda() if case["path"] else None, count=torch.tensor(n, dtype=torch.int32, device="cuda"))
    if own:
        from paper_2506_04708_amd import binding
        st["h"] = _handle(case, np.arange(-1, min(W, 32) - 1, dtype=np.int32))
        st["cache"] = binding.PagedCache(kp, vp)
    else:
        st["which"] = [torch.from_numpy(x).cuda() for x in np.nonzero(np.arange(W)[None] < n[:, None])]


def _prepare_pages(st, case, rs, gen):
    B, page, width, W = case["B"], case["page"], case["width"], case["W"]
    n = np.minimum(_lengths(case, rs), width * page - 1)
    room = np.full(B, case["room"], np.int64)
    if case["add"]:                                  # a step: room for a whole path was there, part of it was taken
        add = rs.randint(1, case["add"] + 1, B)
        held = np.minimum(-(-(n + case["add"]) // page), width)
    else:                                            # requests that come, most of them with nothing yet, others that wait
        add = np.zeros(B, np.int64)
        come = rs.random_sample(B) < 0.6
        n = np.where(come, 0, n)
        held = np.where(come, 0, -(-n // page))
        room = np.where(come, rs.randint(1, case["room"] + 1, B), rs.randint(0, 2 * page, B))
    room = np.where(rs.random_sample(B) < case["leave"], -1, room)      # these leave
    total = B * width + case["spare"] + 1            # pages that are neither held nor free belong to others
    order = rs.permutation(total)
    table = np.full((B, width), -1, np.int64)
    at = 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    taken = int(rs.randint(0, 10 ** 6))
    ring = np.full(total, -1, np.int64)
    free = order[at:at + case["spare"] + 1]
    ring[(taken + np.arange(len(free))) % total] = free
    i32 = dict(dtype=torch.int32, device="cuda")
    mark = torch.tensor([taken, taken + len(free)], dtype=torch.int64, device="cuda")
    st.update(table=torch.tensor(table, **i32), ring=torch.tensor(ring, **i32), length=torch.tensor(n, **i32),
              held=torch.tensor(held, **i32), mark=mark, add=torch.tensor(add, **i32), room=torch.tensor(room, **i32),
              slots=torch.empty((B, W), dtype=torch.int64, device="cuda"), missing=torch.empty(B, **i32))
    if own:
        from paper_2506_04708_amd import binding
        st["h"] = _handle(case, np.arange(-1, min(W, 32) - 1, dtype=np.int32))
        now = binding.Pages(page, st["table"], st["ring"], st["length"], st["held"], st["mark"])
        st["now"], st["then"] = now, now.beside()


def _prepare_shape(st, case, rs, gen):
    B, V = case["B"], case["V"]
    parent = _tree(case["N"], case["D"], case["fan"])
    N = len(parent)
    dt = _DT[case["dtype"]]
    drafted = _drafted(case, parent, rs)

    def words(*shape):                               # token ids as texts have them: few common ones, many rare ones
        return np.minimum((V ** rs.random_sample(shape)).astype(np.int64) - 1 + rs.randint(0, 3, shape), V - 1).clip(0)

    tok = np.where(drafted, words(B, N), -1)
    x = torch.empty((B, N, V), dtype=dt, device="cuda")
    for b in range(B):
        x[b].normal_(generator=gen).mul_(3.0)
    # tokens generated so far, and the prompts' tokens
    count = torch.zeros((B, V), dtype=torch.int32, device="cuda")
    said = torch.from_numpy(words(B, 700)).cuda()
    count.scatter_add_(1, said, torch.ones_like(said, dtype=torch.int32))
    st["prompt"] = None
    if case["prompt"]:
        st["prompt"] = torch.from_numpy(words(B, case["prompt"]).astype(np.int32)).cuda()
        st["prompt_len"] = torch.tensor(rs.randint(0, case["prompt"] + 1, B), dtype=torch.int32, device="cuda")
    penalty = np.stack([rs.choice([1.0, 1.1, 1.3, 0.9], B), rs.choice([0.0, 0.5, -0.2], B), rs.choice([0.0, 0.3], B)], axis=1).astype(np.float32)
    st["bias_id"] = st["bias"] = st["allow"] = None
    if case["bias"]:
        ids = words(B, case["bias"])
        ids[:, case["bias"] - case["bias"] // 3:] = np.where(rs.random_sample((B, case["bias"] // 3)) < 0.7, -1, ids[:, : case["bias"] // 3])
        val = np.where(rs.random_sample(ids.shape) < 0.3, -np.inf, rs.standard_normal(ids.shape) * 4.0)
        st["bias_id"] = torch.from_numpy(ids.astype(np.int32)).cuda()
        st["bias"] = torch.from_numpy(val.astype(np.float32)).cuda()
    if case["mask"]:
        # a free text position, a closed set of a few tokens, half of the vocabulary, a node that the grammar does not reach
        nw = -(-V // 32)
        rnd = torch.randint(-2 ** 31, 2 ** 31, (B, N, nw), generator=gen, device="cuda", dtype=torch.int64)
        more = torch.randint(-2 ** 31, 2 ** 31, (B, N, nw), generator=gen, device="cuda", dtype=torch.int64)
        kind = torch.from_numpy(rs.choice([0, 0, 1, 1, 2, 3], (B, N, 1))).cuda()
        few = rnd & more & (torch.rand((B, N, nw), generator=gen, device="cuda") < 20.0 / nw).long() * -1
        w = torch.where(kind == 0, rnd | more | (rnd << 3), torch.where(kind == 1, few, torch.where(kind == 2, rnd, torch.zeros_like(rnd))))
        w = ((w + 2 ** 31) & (2 ** 32 - 1)) - 2 ** 31
        st["allow"] = w.to(torch.int32)
    st.update(parent=parent, drafted=drafted, x=x, count=count, penalty=torch.from_numpy(penalty).cuda(),
              tok=torch.from_numpy(tok.astype(np.int32)).cuda(), out=torch.empty_like(x))
    if own:
        st["h"] = _handle(case, parent, V, case["dtype"])
    else:
        st["anc"] = torch.from_numpy(_ancestors(parent)).cuda()


# ---- one pass ---------------------------------------------------------------------------------------------------------

def run(st):
    return {"attn": _run_attn, "commit": _run_commit, "pages": _run_pages, "shape": _run_shape}[st["case"]["op"]](st)


def _run_attn(st):
    if own:
        return st["h"].tree_attention(st["cache"], 0, st["length"], st["table"], st["tok"], st["q"], st["k"], st["v"], st["scale"], st["out"])
    # all trajectories at once, as long as the longest: what lies behind a length is masked
    case = st["case"]
    Hq, Hkv, d, page = case["Hq"], case["Hkv"], case["d"], case["page"]
    B, N = st["tok"].shape
    G, most = Hq // Hkv, case["hi"]
    ids = st["table"][:, : -(-most // page)].long()

    def rows(pool, new):                             # [B, Hkv, most + N, d]
        return torch.cat([pool[0][ids].reshape(B, -1, Hkv, d)[:, :most].float(), new.float()], dim=1).transpose(1, 2)

    see = torch.cat([(torch.arange(most, device="cuda") < st["length"][:, None])[:, None].expand(B, N, most),
                     st["anc"].expand(B, N, N)], dim=2) & (st["tok"] >= 0)[:, :, None]
    see = see.repeat_interleave(G, dim=1)[:, None]   # [B, 1, N G, most + N]
    q = st["q"].float().reshape(B, N, Hkv, G, d).transpose(1, 2).reshape(B, Hkv, N * G, d)
    s = torch.matmul(q, rows(st["kp"], st["k"]).transpose(2, 3).contiguous()) * st["scale"]
    s = torch.where(see, s, -math.inf)
    m = s.amax(dim=3, keepdim=True)
    p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
    t = p.sum(dim=3, keepdim=True)
    o = torch.matmul(p, rows(st["vp"], st["v"])) / torch.where(t > 0, t, 1.0)
    st["out"].copy_(o.reshape(B, Hkv, N, G, d).transpose(1, 2).reshape(B, N, Hq, d))
    return st["out"]


def _run_commit(st):
    if own:
        st["h"].cache_commit(st["cache"], st["k"], st["v"], st["slots"], st["row"], st["count"])
        return st["kp"], st["vp"]
    page = st["case"]["page"]
    b, j = st["which"]
    at = st["slots"][b, j]
    row = st["row"][b, j].long() if st["row"] is not None else j
    st["kp"][:, at // page, at % page] = st["k"][:, b, row]
    st["vp"][:, at // page, at % page] = st["v"][:, b, row]
    return st["kp"], st["vp"]


def _run_pages(st):
    if own:
        st["h"].cache_pages(st["now"], st["add"], st["room"], st["slots"], st["missing"], st["then"])
        t = st["then"]
        return t.length, t.held, t.mark, st["table"], st["ring"], st["slots"], st["missing"]
    case = st["case"]
    page, width, W = case["page"], case["width"], case["W"]
    table, ring = st["table"], st["ring"]
    P = ring.numel()
    room, held = st["room"].long(), st["held"].long()
    stays = room >= 0
    new = torch.where(stays, torch.minimum(torch.clamp(st["length"].long() + st["add"], min=0), held * page), 0)
    need = torch.where(stays, (new + room + page - 1) // page, 0)
    want = torch.clamp(need - held, min=0)
    asks = torch.where(need <= width, want, 0)
    give = torch.clamp(held - need, min=0)
    before, given_before = torch.cumsum(asks, 0) - asks, torch.cumsum(give, 0) - give
    ok = (want == 0) | ((need <= width) & (before + asks <= st["mark"][1] - st["mark"][0]))
    now = torch.where(ok, need, held)
    i = torch.arange(width, device="cuda")[None]
    back = (i >= need[:, None]) & (i < held[:, None])
    to = torch.where(back, (st["mark"][1] + given_before[:, None] + i - need[:, None]) % P, P)
    more = torch.cat([ring, ring[:1]])
    more[to.reshape(-1)] = table.reshape(-1)
    fresh = ok[:, None] & (i >= held[:, None]) & (i < need[:, None])
    table.copy_(torch.where(fresh, ring[(st["mark"][0] + before[:, None] + i - held[:, None]) % P], table))
    ring.copy_(more[:P])
    j = torch.arange(W, device="cuda")[None]
    pos = new[:, None] + j
    slots = torch.gather(table, 1, torch.clamp(pos // page, max=width - 1)).long() * page + pos % page
    slots = torch.where((j < room[:, None]) & (pos // page < now[:, None]), slots, -1)
    mark = torch.stack([st["mark"][0] + torch.where(ok, asks, 0).sum(), st["mark"][1] + give.sum()])
    return new.int(), now.int(), mark, table, ring, slots, torch.where(ok, 0, want).int()


def _run_shape(st):
    if own:
        if st["prompt"] is not None:
            st["h"].count_tokens(st["count"], st["prompt"], st["prompt_len"], prompt=True)
        out = st["h"].shape_logits(st["x"], st["out"], st["tok"], st["count"], st["penalty"], st["bias_id"], st["bias"], st["allow"])
        return out, st["count"]
    B, N, V = st["x"].shape
    flag = 1 << 30
    if st["prompt"] is not None:
        here = torch.zeros((B, V + 1), dtype=torch.bool, device="cuda")
        j = torch.arange(st["prompt"].shape[1], device="cuda")[None]
        here.scatter_(1, torch.where(j < st["prompt_len"][:, None], st["prompt"].long(), V), True)
        st["count"].copy_(torch.where(here[:, :V], st["count"] | flag, st["count"]))
    rho, present, often = (st["penalty"][:, i, None, None] for i in range(3))
    x, drafted = st["x"].float(), (st["tok"] >= 0)[:, :, None]
    on_path = (st["anc"] & (torch.arange(N, device="cuda") > 0)).float()
    c = (st["count"] & (flag - 1)).float()[:, None].repeat(1, N, 1)
    c.scatter_add_(2, st["tok"].long().clamp(min=0)[:, None].expand(B, N, N), on_path.expand(B, N, N).contiguous())
    seen = (c > 0) | ((st["count"] & flag) != 0)[:, None]
    y = torch.where(seen, torch.where(x > 0, x / rho, x * rho), x) - often * c - torch.where(c > 0, present, 0.0)
    if st["bias_id"] is not None:                    # of several entries with one id the last one counts
        ids, M = st["bias_id"].long(), st["bias_id"].shape[1]
        last = torch.full((B, V + 1), -1, dtype=torch.int64, device="cuda")
        last.scatter_reduce_(1, torch.where(ids >= 0, ids, V), torch.arange(M, device="cuda").expand(B, M).contiguous(), "amax")
        last = last[:, :V]
        y = y + torch.where(last >= 0, torch.gather(st["bias"], 1, last.clamp(min=0)), 0.0)[:, None]
    if st["allow"] is not None:                      # a row that allows nothing stays as it is
        bits = (st["allow"][:, :, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        bits = bits.reshape(B, N, -1)[:, :, :V] > 0
        y = torch.where(bits | ~bits.any(dim=2, keepdim=True), y, -math.inf)
    st["out"].copy_(torch.where(drafted, y, x))
    return st["out"], st["count"]


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    B = case["B"]
    if case["op"] == "attn":
        Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
        n, kept = _lengths(case), np.array(_kept(case))
        pairs = float((n * kept).sum() + kept.sum() * (1 + case["D"] / 2))
        rows = float(kept.sum())
        return {"bytes": 2.0 * (2 * Hkv * d * (n.sum() + rows) + 2 * Hq * d * rows), "flops": 4.0 * d * Hq * pairs}
    if case["op"] == "commit":
        return {"bytes": 2.0 * 2 * 2 * case["layers"] * case["Hkv"] * case["d"] * max(1, int(_lengths(case).sum())), "flops": 0.0}
    if case["op"] == "pages":
        return {"bytes": B * (32.0 + 8 * case["W"] * (1.0 if case["add"] else 0.35)), "flops": 0.0}
    rows, V = float(B * case["N"]), case["V"]
    e = 4 if case["dtype"] == "f32" else 2
    return {"bytes": rows * V * (2 * e + (0.125 if case["mask"] else 0.0)) + 4.0 * B * V + 4.0 * B * case["prompt"] / 2, "flops": 4.0 * rows * V}


# ---- the operators in 64 bits, from their definitions -----------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "attn":
        return _exact_attn(case, st)
    if case["op"] == "shape":
        return _exact_shape(case, st), None
    return None                                      # copies and whole numbers


def _exact_attn(case, st):
    """Node by node along its own path: softmax over the cached tokens and the path's tokens, no mask."""
    parent, page, d = st["parent"], case["page"], case["d"]
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
    out = torch.zeros((B, N, case["Hq"], d), dtype=torch.float64, device="cuda")
    for b in range(B):
        nodes = torch.from_numpy(np.nonzero(st["drafted"][b])[0]).cuda()
        pos = torch.arange(int(st["lens"][b]), device="cuda")
        where = st["table"][b].long()[pos // page]
        along = path[nodes]                          # [n, deep]
        for h in range(Hkv):
            K, V = st["kp"][0, where, pos % page, h].double(), st["vp"][0, where, pos % page, h].double()
            Kt, Vt = st["k"][b, :, h].double()[along.clamp(min=0)], st["v"][b, :, h].double()[along.clamp(min=0)]
            for g in range(G):
                q = st["q"][b, nodes, h * G + g].double() * st["scale"]
                a = q @ K.t()
                t = (q[:, None, :] * Kt).sum(dim=2).masked_fill(along < 0, -math.inf)
                top = t.amax(dim=1) if a.shape[1] == 0 else torch.maximum(a.amax(dim=1), t.amax(dim=1))
                a, t = torch.exp(a - top[:, None]), torch.exp(t - top[:, None])
                o = a @ V + (t[:, :, None] * Vt).sum(dim=1)
                out[b, nodes, h * G + g] = o / (a.sum(dim=1) + t.sum(dim=1))[:, None]
    return out


def _exact_shape(case, st):
    """Row by row: the counts of the row's own path, then every rule in its order."""
    x, parent = st["x"], st["parent"]
    B, N, V = x.shape
    tok = st["tok"].cpu().numpy()
    out = x.double()
    bit = torch.arange(V, device="cuda")
    for b in range(B):
        made = (st["count"][b] & 0x3FFFFFFF).double()
        known = (st["count"][b] >> 30) & 1
        if st["prompt"] is not None:
            known = known.clone()
            known[st["prompt"][b, : int(st["prompt_len"][b])].long()] = 1
        rho, present, often = (float(p) for p in st["penalty"][b].cpu())
        shift = torch.zeros(V, dtype=torch.float64, device="cuda")
        if st["bias_id"] is not None:
            ids, val = st["bias_id"][b].cpu().numpy(), st["bias"][b].cpu().numpy()
            last = {int(i): float(v) for i, v in zip(ids, val) if i >= 0}
            if last:
                shift[torch.tensor(list(last), device="cuda")] = torch.tensor(list(last.values()), dtype=torch.float64, device="cuda")
        for u in range(N):
            if tok[b, u] < 0:
                continue
            c, v = made.clone(), u
            while v > 0:
                c[int(tok[b, v])] += 1
                v = int(parent[v])
            y = out[b, u].clone()
            seen = (c > 0) | (known > 0)
            y[seen] = torch.where(y[seen] > 0, y[seen] / rho, y[seen] * rho)
            y = y - often * c - present * (c > 0) + shift
            if st["allow"] is not None:
                ok = ((st["allow"][b, u].long()[bit // 32] >> (bit % 32)) & 1) != 0
                if bool(ok.any()):
                    y = y.masked_fill(~ok, -math.inf)
            out[b, u] = y
    return out

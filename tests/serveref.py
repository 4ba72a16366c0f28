"""Plain implementations, in 64 bits on the CPU, of the operators around a verification, and the errors they allow: every
bound counts the roundings that the library's documentation names."""
import math

import numpy as np
import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}   # half a step, relative to the value


def depths(parent):
    d = [0] * len(parent)
    for u in range(1, len(parent)):
        d[u] = d[parent[u]] + 1
    return np.array(d)


def path(parent, u):
    """Nodes from u up to the root."""
    out = []
    while u >= 0:
        out.append(u)
        u = int(parent[u])
    return out


def attention(parent, length, table, tok, q, k, v, kp, vp, scale):
    """(values, largest errors allowed) of stand_tree_attention: kp, vp [pages, page, heads, d] of one layer."""
    B, N, H, d = q.shape
    G, page = k.shape[2], kp.shape[1]
    per = H // G
    half = EPS[q.dtype]
    out, tol = torch.zeros((B, N, H, d), dtype=torch.float64), torch.zeros((B, N, H, d), dtype=torch.float64)
    for b in range(B):
        n = min(max(int(length[b]), 0), table.shape[1] * page)
        pos = torch.arange(n)
        at = table[b].long()[pos // page]
        K, V = kp[at, pos % page].double(), vp[at, pos % page].double()          # [n, G, d]
        for u in range(N):
            if int(tok[b, u]) < 0:
                continue
            own = path(parent, u)
            for g in range(G):
                KK, VV = torch.cat([K[:, g], k[b, own, g].double()]), torch.cat([V[:, g], v[b, own, g].double()])
                qq = q[b, u, g * per:(g + 1) * per].double()
                s = qq @ KK.t() * scale
                p = torch.softmax(s, dim=1)
                o = p @ VV
                # d products summed in fp32, one more rounding of the scaled score; exp2 and the sums: a few roundings more
                ds = ((qq.abs() @ KK.abs().t()) * scale * (d + 4) + s.abs() * 4 + 16) * 2.0 ** -24
                mean = p @ VV.abs()
                weight = p @ VV.abs() * half + o.abs() * half                   # weights rounded, summed as rounded
                score = (p * ds) @ VV.abs() + o.abs() * (p * ds).sum(1, keepdim=True)
                if q.dtype == torch.float16:                                    # weights below 2^-20 of the largest are subnormal
                    weight = weight + 2.0 ** -31 * VV.abs().sum(0)[None] / torch.exp(s - s.amax(1, keepdim=True)).sum(1, keepdim=True) * 2
                sums = mean * (len(KK) + 64) * 2.0 ** -24
                t = (weight + 2 * score + sums) * (1 + 4 * half) + o.abs() * half
                out[b, u, g * per:(g + 1) * per] = o
                tol[b, u, g * per:(g + 1) * per] = t + (2.0 ** -25 if q.dtype == torch.float16 else 0.0)
    return out, tol


def shape(parent, x, tok, count, penalty, bias_id, bias, allow):
    """(values, largest errors allowed) of stand_shape_logits."""
    B, N, V = x.shape
    half = EPS[x.dtype]
    out, tol = x.double().clone(), torch.zeros((B, N, V), dtype=torch.float64)
    for b in range(B):
        rho, present, often = (float(t) for t in penalty[b]) if penalty is not None else (1.0, 0.0, 0.0)
        shift = torch.zeros(V, dtype=torch.float64)
        if bias_id is not None:
            for i, t in zip(bias_id[b].tolist(), bias[b].tolist()):
                if 0 <= i < V:
                    shift[i] = t
        for u in range(N):
            if int(tok[b, u]) < 0:
                continue
            made = (count[b].long() & 0x3FFFFFFF).double() if count is not None else torch.zeros(V, dtype=torch.float64)
            known = ((count[b] >> 30) & 1 > 0) if count is not None else torch.zeros(V, dtype=torch.bool)
            for w in path(parent, u):
                if w:
                    made[int(tok[b, w])] += 1
            y = out[b, u].clone()
            seen = (made > 0) | known
            y = torch.where(seen, torch.where(y > 0, y / rho, y * rho), y)
            mag = y.abs()
            y = y - often * made
            mag = mag + (often * made).abs()
            y = torch.where(made > 0, y - present, y)
            mag = mag + abs(present)
            y = y + shift
            fin = torch.where(torch.isinf(shift), torch.zeros_like(shift), shift.abs())
            mag = mag + fin
            if allow is not None:
                w = allow[b, u].long()
                ok = (w[torch.arange(V) // 32] >> (torch.arange(V) % 32)) & 1 > 0
                if bool(ok.any()):
                    y = torch.where(ok, y, -math.inf)
            out[b, u] = y
            # five roundings to binary32 of numbers no larger than `mag`, one to the type of the logits
            tol[b, u] = torch.where(torch.isinf(y), 0.0, mag * 5 * 2.0 ** -24 + y.abs() * half * (1 if x.dtype != torch.float32 else 0))
    return out, tol


def pages(page, table, ring, length, held, mark, add, room, slot_width, path_room):
    """Everything that stand_cache_pages writes, as lists of whole numbers."""
    table, ring = [list(r) for r in table], list(ring)
    B, width, P = len(table), len(table[0]), len(ring)
    front = list(ring)
    taken, given = mark
    avail, asked, back, granted = given - taken, 0, 0, 0
    out = dict(length=[], held=[], missing=[], slots=[])
    for b in range(B):
        r = path_room if room is None else room[b]
        n = 0 if r < 0 else min(max(length[b] + (0 if add is None else add[b]), 0), held[b] * page)
        need = 0 if r < 0 else -(-(n + r) // page)
        now, missing = held[b], 0
        if need < held[b]:
            for i in range(need, held[b]):
                ring[(given + back) % P] = table[b][i]
                back += 1
            now = need
        elif need > width:
            missing = need - held[b]
        elif need > held[b]:
            ask = need - held[b]
            if asked + ask <= avail:
                for i in range(ask):
                    table[b][held[b] + i] = front[(taken + asked + i) % P]
                now, granted = need, granted + ask
            else:
                missing = ask
            asked += ask
        out["length"].append(n)
        out["held"].append(now)
        out["missing"].append(missing)
        out["slots"].append([table[b][(n + j) // page] * page + (n + j) % page if j < r and (n + j) // page < now else -1
                             for j in range(slot_width)])
    return dict(out, table=table, ring=ring, mark=[taken + granted, given + back])

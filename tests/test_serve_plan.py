"""The host side of the operators around a verification, without a GPU: every unit of the attention's work is in one share
and every part of a cut item is joined once; bad lengths and pages are replaced; bad calls are refused before a launch."""
import ctypes as C
import random
import re
import os

import pytest

from tests import serveplan

EINVAL, ELIMIT, BF16, F32, F16 = -1, -5, 0, 1, 2


def trajectories(rng, kind):
    """(lengths, drafted nodes, nodes of the tree, query heads of a kv head, kv heads, most cached tokens)"""
    B = rng.choice([1, 2, 7, 40])
    N = rng.choice([1, 3, 32, 130, 1024]) if kind != "short" else rng.choice([1, 2])
    per, heads = rng.choice([1, 4, 7]), rng.choice([1, 2, 8])
    most = 1 << 14
    lens = [rng.choice([0, 1, 5, 63, 64, 65, rng.randrange(most), most, most + 9, -3]) if kind != "short" else rng.randrange(3) for _ in range(B)]
    return lens, [rng.choice([0, 1, N, rng.randrange(N + 1)]) for _ in range(B)], N, per, heads, most


@pytest.mark.parametrize("kind", ["short", "any"])
@pytest.mark.parametrize("tile,keys,start,heavy,light", [(32, 128, 2, 1, 1), (64, 64, 4, 1, 1), (256, 64, 4, 3, 2), (256, 64, 4, 2, 1), (128, 64, 8, 1, 1)])
def test_shares_cover_every_unit_once(kind, tile, keys, start, heavy, light):
    """The kernel's walk over its shares, unit by unit, and what the join does with the parts."""
    L, rng = serveplan.lib(), random.Random(tile + start + heavy)
    for rep in range(60):
        lens, drafted, N, per, heads, most = trajectories(rng, kind)
        launched = rng.choice([8, 256, 512, 1024])
        items, total = [], 0                                   # (first place, units, weight) of every item
        for n, t in zip(lens, drafted):
            u = L.units(n, most, N, keys)
            assert u == -(-min(max(n, 0), most) // keys) + -(-N // keys) and u >= 1
            tiles = [min(tile, t * per - r) for r in range(0, t * per, tile)]
            weights = [L.weight(r, tile, heavy, light) for r in tiles]
            assert weights == [heavy if r > tile // 2 else light for r in tiles] and L.head(t * per, tile, heavy, light) == sum(weights)
            assert heavy in weights[:-1] or len(weights) < 2
            for _ in range(heads):
                for w in weights:
                    items.append((total, u, w))
                    total += w * (u + start)
        W = L.groups(total, launched, start, heavy)
        assert 0 <= W <= launched and (W > 0) == (total > 0)
        if not total:
            continue
        done, records = {}, {}
        starts = [L.begin(w, total, W) for w in range(W + 1)]
        assert starts[0] == 0 and starts[-1] == total
        at = 0
        for w in range(W):
            place, end = starts[w], starts[w + 1]
            assert end - place >= heavy * (start + 1) or W == 1
            assert L.owner(place, total, W) == w and L.owner(end - 1, total, W) == w
            while at + 1 < len(items) and items[at + 1][0] <= place:
                at += 1
            for k in range(at, len(items)):
                s, u, weight = items[k]
                u0, u1 = L.before(place - s, weight, start, u), L.before(end - s, weight, start, u)
                if s >= end or u1 == 0:
                    break
                assert 0 <= u0 < u1 <= u
                if w not in records:
                    records[w] = (k, L.first(s, total, W, start, weight), L.owner(s + weight * (u + start) - 1, total, W), u0 > 0)
                done.setdefault(k, []).append((u0, u1, w))
                if u1 < u:
                    break
                place = s + weight * (u + start)
                if place >= end:
                    break
            assert w in records                                # (every share leaves its record)
        assert len(done) == len(items)
        for k, (s, u, weight) in enumerate(items):
            parts = done[k]
            assert [p[0] for p in parts] == [0] + [p[1] for p in parts[:-1]] and parts[-1][1] == u
            if len(parts) > 1:                                 # joined by the second share's record, from all of the shares
                ws = [p[2] for p in parts]
                assert ws == list(range(ws[0], ws[-1] + 1))
                for w in ws[1:]:
                    assert records[w] == (k, ws[0], ws[-1], True)
        for w, (k, a, b, cut) in records.items():
            if not cut:                                        # nothing to join by this one
                assert done[k][0][2] == w


def test_bad_pages_and_lengths_are_replaced():
    L = serveplan.lib()
    for pages in (1, 2, 1000, 2 ** 31 - 1):
        for p in (-2 ** 31, -1, 0, 1, pages - 1, pages if pages < 2 ** 31 - 1 else 0, 2 ** 31 - 1):
            assert 0 <= L.page(p, pages) < pages
            assert L.page(p, pages) == p or not 0 <= p < pages
    for most in (1, 16, 1 << 30):
        for n in (-2 ** 31, -1, 0, 1, most - 1, most, most + 1, 2 ** 31 - 1):
            assert L.length(n, most) == min(max(n, 0), most)


def cache(**kw):
    d = dict(d_k=1 << 20, d_v=1 << 21, dtype=BF16, layers=2, pages=64, page_size=16, kv_heads=2, head_dim=64,
             layer_stride=64 * 16 * 128, page_stride=16 * 128, slot_stride=128, head_stride=64)
    d.update(kw)
    return serveplan.Cache(**d)


BAD_CACHE = [dict(d_k=0), dict(d_v=0), dict(d_k=8), dict(d_v=24), dict(dtype=F32), dict(dtype=3), dict(layers=0), dict(pages=0), dict(page_size=0),
             dict(page_size=12), dict(page_size=8192), dict(page_size=-16), dict(kv_heads=0), dict(kv_heads=4097), dict(head_dim=0), dict(head_dim=96),
             dict(head_dim=256), dict(layer_stride=-8), dict(page_stride=4), dict(slot_stride=129), dict(head_stride=1 << 48)]


def test_refusals_of_the_attention():
    L = serveplan.lib()

    def call(B=3, c=None, layer=1, length=64, table=64, width=9, tok=64, work=256, no_rows=False, **kw):
        r = dict(d_q=4096, d_k=4096, d_v=4096, d_out=8192, q_heads=4, scale=0.125)
        strides = {k: kw.pop(k, [4096, 256, 64]) for k in ("q_stride", "k_stride", "v_stride", "out_stride")}
        r.update(kw)
        rows = serveplan.TreeRows(**r)
        for k, v in strides.items():
            getattr(rows, k)[:] = v
        return L.attention(B, C.byref(c or cache()), layer, length, table, width, tok, None if no_rows else C.byref(rows), work)

    assert call() == 0 and call(layer=0, B=4096) == 0 and call(c=cache(dtype=F16, head_dim=128)) == 0
    assert call(q_stride=[0, 0, 0]) == 0                       # one row for all: fine to read
    for kw in BAD_CACHE:
        assert call(c=cache(**kw)) == EINVAL, kw
    for kw in (dict(layer=-1), dict(layer=2), dict(length=0), dict(table=0), dict(width=0), dict(width=-1), dict(tok=0), dict(work=0), dict(work=8),
               dict(no_rows=True), dict(d_q=0), dict(d_k=0), dict(d_v=0), dict(d_out=0), dict(d_q=8), dict(d_k=8), dict(d_v=8), dict(d_out=8), dict(q_heads=0),
               dict(q_heads=3), dict(q_heads=-2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(width=(1 << 30) // 16 + 1), dict(q_stride=[4096, 256, 60]), dict(k_stride=[-8, 256, 64]), dict(v_stride=[1, 256, 64]),
               dict(out_stride=[4096, 1 << 48, 64])):
        assert call(**kw) == EINVAL, kw
    assert call(B=4097) == ELIMIT and call(q_heads=65536) == ELIMIT
    # a layer's places are counted in 16-byte chunks, in 32 bits: 64 GiB
    wide = dict(pages=2 ** 15 + 1, page_size=16)
    assert call(c=cache(page_stride=2 ** 20, **wide)) == ELIMIT and call(c=cache(page_stride=2 ** 20 - 128, **wide)) == 0
    assert call(c=cache(pages=2 ** 31 - 1, page_stride=(1 << 48) - 8)) == ELIMIT
    assert call(c=cache(page_size=4096, slot_stride=(1 << 48) - 8)) == ELIMIT


def test_refusals_of_the_cache():
    L = serveplan.lib()

    def commit(B=3, c=None, slots=64, width=5, **kw):
        r = dict(d_k=4096, d_v=4096, rows=9, layer_stride=4096, batch_stride=2048, row_stride=128, head_stride=64)
        r.update(kw)
        return L.commit(B, C.byref(c or cache()), C.byref(serveplan.CacheRows(**r)), slots, width)

    assert commit() == 0 and commit(B=65535, width=1 << 30) == 0
    for kw in BAD_CACHE:
        assert commit(c=cache(**kw)) == EINVAL, kw
    for kw in (dict(slots=0), dict(width=0), dict(width=(1 << 30) + 1), dict(d_k=0), dict(d_v=0), dict(d_k=8), dict(rows=0), dict(layer_stride=3),
               dict(batch_stride=-8), dict(row_stride=1 << 48), dict(head_stride=4)):
        assert commit(**kw) == EINVAL, kw
    assert commit(B=65536) == ELIMIT and commit(c=cache(layers=65536)) == ELIMIT

    def pages(B=3, slots=64, width=5, missing=64, out=None, **kw):
        d = dict(d_table=64, d_ring=128, d_length=192, d_held=256, d_mark=320, width=9, pages=64, page_size=16)
        d.update(kw)
        o = dict(d)
        o.update(out or {})
        return L.cache_pages(B, C.byref(serveplan.Pages(**d)), slots, width, missing, C.byref(serveplan.Pages(**o)))

    assert pages() == 0 and pages(slots=0, width=0) == 0 and pages(B=65535, out=dict(d_length=512, d_held=768, d_mark=1024)) == 0
    for kw in (dict(d_table=0), dict(d_ring=0), dict(d_length=0), dict(d_held=0), dict(d_mark=0), dict(missing=0), dict(slots=0), dict(width=-1),
               dict(width=(1 << 30) + 1), dict(page_size=12), dict(page_size=0), dict(pages=0), dict(page_size=8192)):
        assert pages(**kw) == EINVAL, kw
    for out in (dict(d_table=512), dict(d_ring=512), dict(width=8), dict(pages=63), dict(page_size=32), dict(d_length=0), dict(d_held=0), dict(d_mark=0)):
        assert pages(out=out) == EINVAL, out
    assert pages(B=65536) == ELIMIT


def test_refusals_of_logits_and_counts():
    L = serveplan.lib()

    def shape(B=3, dtype=BF16, x=64, out=64, tok=64, ids=64, bias=64, width=5):
        return L.shape(B, dtype, x, out, tok, ids, bias, width)

    assert shape() == 0 and shape(ids=0, bias=0, width=0) == 0 and shape(x=66, out=2) == 0
    for kw in (dict(x=0), dict(out=0), dict(tok=0), dict(ids=0), dict(bias=0), dict(width=-1), dict(width=(1 << 30) + 1), dict(x=65), dict(out=67),
               dict(dtype=F32, x=66), dict(dtype=F32, out=70)):
        assert shape(**kw) == EINVAL, kw
    assert shape(B=65536) == ELIMIT
    assert L.count(3, 64, 64, 9) == 0 and L.count(3, 0, 64, 9) == EINVAL and L.count(3, 64, 0, 9) == EINVAL
    assert L.count(3, 64, 64, 0) == EINVAL and L.count(3, 64, 64, (1 << 30) + 1) == EINVAL and L.count(65536, 64, 64, 9) == ELIMIT


def test_the_binding_packs_the_same_structures():
    binding = pytest.importorskip("paper_2506_04708_amd.binding")
    assert binding._TREE_ROWS.size == C.sizeof(serveplan.TreeRows) and binding._CACHE_ROWS.size == C.sizeof(serveplan.CacheRows)
    assert C.sizeof(binding.CacheDesc) == C.sizeof(serveplan.Cache) and C.sizeof(binding.PagesDesc) == C.sizeof(serveplan.Pages)
    x = serveplan.TreeRows.from_buffer_copy(binding._TREE_ROWS.pack(1, 2, 3, 4, 5, 0.5, *range(10, 22)))
    assert (x.d_q, x.d_k, x.d_v, x.d_out, x.q_heads, x.scale) == (1, 2, 3, 4, 5, 0.5)
    assert list(x.q_stride) + list(x.k_stride) + list(x.v_stride) + list(x.out_stride) == list(range(10, 22))
    y = serveplan.CacheRows.from_buffer_copy(binding._CACHE_ROWS.pack(1, 2, 3, 4, 5, 6, 7))
    assert (y.d_k, y.d_v, y.rows, y.layer_stride, y.batch_stride, y.row_stride, y.head_stride) == (1, 2, 3, 4, 5, 6, 7)


def test_constants_agree_with_the_header():
    text = open(os.path.join(serveplan.ROOT, "include", "stand.h")).read()
    got = {m.group(1): m.group(2) for m in re.finditer(r"#define (STAND_\w+) \(?(-?\d+)", text)}
    assert int(got["STAND_EINVAL"]) == EINVAL and int(got["STAND_ELIMIT"]) == ELIMIT and int(got["STAND_F16"]) == F16
    assert int(got["STAND_BF16"]) == BF16 and int(got["STAND_F32"]) == F32

"""A cache in 4 bits, norms and rotations of heads: what the calls accept, and the scales of blocks, without a GPU."""
import ctypes as C
import math
import struct

import numpy as np
import pytest
import torch

from tests import servehost, serveref4

I, U, L, P = C.c_int, C.c_uint32, C.c_int64, C.c_void_p
BF, HF, MX, EINVAL, ELIMIT = 0, 2, 4, -1, -5


class Cache(C.Structure):
    """stand_cache4, the stand_cache that it begins with spelled out."""
    _fields_ = [("d_k", P), ("d_v", P), ("dtype", C.c_int32), ("layers", C.c_int32), ("pages", C.c_int32), ("page_size", C.c_int32),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("layer_stride", L), ("page_stride", L), ("slot_stride", L), ("head_stride", L),
                ("d_k_scale", P), ("d_v_scale", P), ("scale_layer_stride", L), ("scale_page_stride", L), ("scale_slot_stride", L),
                ("scale_head_stride", L)]


class Rotation(C.Structure):
    _fields_ = [("d_turns", P), ("positions", C.c_int32), ("dims", C.c_int32), ("neighbours", C.c_int32), ("eps", C.c_float), ("d_q_norm", P),
                ("d_k_norm", P)]


class Rows(C.Structure):
    _fields_ = [("d_q", P), ("d_k", P), ("d_v", P), ("d_q_out", P), ("d_k_out", P), ("dtype", C.c_int32), ("rows", C.c_int32), ("q_heads", C.c_int32),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("q_stride", L * 3), ("k_stride", L * 3), ("v_stride", L * 3),
                ("q_out_stride", L * 3), ("k_out_stride", L * 3)]


class Out(C.Structure):
    _fields_ = [("d_k", P), ("d_v", P), ("rows", C.c_int32), ("layer_stride", L), ("batch_stride", L), ("row_stride", L), ("head_stride", L)]


@pytest.fixture(scope="module")
def lib():
    return servehost.build("""
#include "serve_checks.hpp"
#include "mx4.hpp"
using namespace stand;
extern "C" {
int scale(uint32_t top, int f16) { return mx4_scale(top, f16 != 0); }
int sized(int64_t B, const stand_cache *c, int q_heads) { return check_attention_size(B, c, q_heads); }
int commit(const stand_cache *c)
{
    stand_cache_rows r{(void *)4096, (void *)4096, 9, 4096, 2048, 128, 64};
    return check_cache_commit(3, c, &r, (const int64_t *)64, 5);
}
int rotate(int64_t B, int N, const stand_rotation *r, const void *len, const void *tok, const stand_turned_rows *rows)
{ return check_tree_rotate(B, N, r, (const int32_t *)len, (const int32_t *)tok, rows); }
int append(int64_t B, const stand_cache *c, int layer, const stand_rotation *r, const stand_turned_rows *rows, const void *slots, int width)
{ return check_cache_append(B, c, layer, r, rows, (const int64_t *)slots, width); }
int rd(int64_t B, const stand_cache *c, int first, int layers, const void *table, int width, const stand_cache_rows_out *rows)
{ return check_cache_read(B, c, first, layers, (const int32_t *)table, width, rows); }
int sizes(int i) { const int s[] = {sizeof(stand_cache4), sizeof(stand_rotation), sizeof(stand_turned_rows), sizeof(stand_cache_rows_out)}; return s[i]; }
int64_t groups(int64_t rows, int64_t heads, int d) { return turn_groups(rows, heads, d); }
}""", dict(scale=([U, I], I), sized=([L, P, I], I), commit=([P], I), rotate=([L, I, P, P, P, P], I), append=([L, P, I, P, P, P, I], I),
           rd=([L, P, I, I, P, I, P], I), sizes=([I], I), groups=([L, L, I], L)))


def test_structures_are_as_the_binding_packs_them(lib):
    from paper_2506_04708_amd import binding
    assert [lib.sizes(i) for i in range(4)] == [C.sizeof(Cache), C.sizeof(Rotation), C.sizeof(Rows), C.sizeof(Out)]
    assert C.sizeof(binding.Cache4Desc) == lib.sizes(0) and C.sizeof(binding.RotationDesc) == lib.sizes(1)
    assert binding._TURNED_ROWS.size == lib.sizes(2) and binding._CACHE_ROWS.size == lib.sizes(3)
    assert binding.STAND_MXFP4 == MX


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scales_of_blocks(lib, dtype):
    """Every magnitude of 16 bits, and fp32 ones beside the places where the scale changes."""
    f16 = dtype is torch.float16
    x = np.arange(32768, dtype=np.uint16)
    mags = torch.from_numpy(x.view(np.int16).copy()).view(dtype).double().tolist()
    mags += [m * (1 + e) for m in (1.75, 1.0, 3.5, 7.0, 2.0 ** -120 * 1.75, 2.0 ** 120 * 1.75) for e in (-2.0 ** -24, -2.0 ** -23, 2.0 ** -23)]
    for m in mags:
        bits = struct.unpack("I", struct.pack("f", m))[0]
        assert lib.scale(bits, int(f16)) == serveref4.scale_of(struct.unpack("f", struct.pack("I", bits))[0], dtype), m
    lo, hi = serveref4.LIMITS[dtype]
    for s in (lo, hi):                                       # every product is a number of the type
        v = torch.from_numpy(serveref4.GRID * 2.0 ** (s - 127))
        assert torch.equal(v.to(dtype).double(), v) and bool(torch.isfinite(v.to(dtype)).all())


def test_a_blocks_largest_element_is_off_by_half_a_step(lib):
    rng = np.random.default_rng(1)
    for dtype in (torch.bfloat16, torch.float16):
        x = torch.from_numpy(rng.standard_normal((2000, 64)) * np.exp2(rng.integers(-8, 8, (2000, 1)))).to(dtype)
        p, s = serveref4.pack(x, dtype)
        got = serveref4.unpack(p, s, dtype).double()
        unit = torch.from_numpy(np.ldexp(1.0, s.numpy().astype(int) - 127)).repeat_interleave(32, 1)
        a = x.double().abs() / unit
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        assert bool(((got - x.double()).abs() <= step / 2 * unit).all()) and float(a.max()) < 7 and bool((a.reshape(-1, 32).amax(1) >= 3.5).all())


def cache(**kw):
    d = dict(d_k=1 << 20, d_v=1 << 21, dtype=MX + BF, layers=2, pages=64, page_size=16, kv_heads=2, head_dim=64, layer_stride=64 * 16 * 128,
             page_stride=16 * 128, slot_stride=128, head_stride=64, d_k_scale=1 << 22, d_v_scale=1 << 23, scale_layer_stride=64 * 16 * 4,
             scale_page_stride=16 * 4, scale_slot_stride=4, scale_head_stride=2)
    d.update(kw)
    return Cache(**d)


BAD4 = [dict(d_k_scale=0), dict(d_v_scale=0), dict(d_k_scale=4097), dict(d_v_scale=4097), dict(d_k_scale=4098, head_dim=128),
        dict(layer_stride=8), dict(page_stride=16), dict(slot_stride=72), dict(head_stride=40), dict(head_stride=-32), dict(scale_layer_stride=1),
        dict(scale_page_stride=-2), dict(scale_slot_stride=3), dict(scale_head_stride=1), dict(scale_head_stride=2, head_dim=128),
        dict(scale_slot_stride=1 << 48), dict(dtype=5), dict(dtype=7), dict(dtype=8), dict(dtype=MX + 1), dict(d_k=8), dict(pages=0), dict(head_dim=96)]


def test_caches_of_four_bits(lib):
    for kw in (dict(), dict(dtype=MX + HF), dict(head_dim=128, scale_head_stride=4), dict(d_k_scale=4098), dict(scale_layer_stride=0)):
        assert lib.commit(C.byref(cache(**kw))) == 0 and lib.sized(3, C.byref(cache(**kw)), 4) == 0, kw
    for kw in BAD4:
        c = cache(**kw)
        assert lib.commit(C.byref(c)) == EINVAL and lib.sized(3, C.byref(c), 4) == EINVAL, kw
    # of 16 bits the members behind the strides do not matter
    assert lib.commit(C.byref(cache(dtype=BF, d_k_scale=0, d_v_scale=1, scale_head_stride=-7, head_stride=8))) == 0
    # 2^32 chunks of 16 bytes, 2^32 heads' scales
    wide = dict(pages=2 ** 15 + 1, page_size=16)
    assert lib.sized(3, C.byref(cache(page_stride=2 ** 22, **wide)), 4) == ELIMIT
    assert lib.sized(3, C.byref(cache(page_stride=2 ** 22 - 512, **wide)), 4) == 0
    assert lib.sized(3, C.byref(cache(scale_page_stride=2 ** 18, **wide)), 4) == ELIMIT
    assert lib.sized(3, C.byref(cache(scale_page_stride=2 ** 18 - 32, **wide)), 4) == 0


def rotation(**kw):
    d = dict(d_turns=4096, positions=100, dims=64, neighbours=0, eps=1e-6, d_q_norm=0, d_k_norm=8192)
    d.update(kw)
    return Rotation(**d)


def rows(**kw):
    strides = {k: kw.pop(k, [4096, 256, 64]) for k in ("q_stride", "k_stride", "v_stride", "q_out_stride", "k_out_stride")}
    d = dict(d_q=4096, d_k=8192, d_v=16384, d_q_out=32768, d_k_out=65536, dtype=BF, rows=9, q_heads=6, kv_heads=2, head_dim=64)
    d.update(kw)
    r = Rows(**d)
    for k, v in strides.items():
        getattr(r, k)[:] = v
    return r


BAD_ROTATION = [dict(d_turns=0), dict(d_turns=4100), dict(positions=0), dict(positions=-1), dict(dims=-16), dict(dims=8), dict(dims=24), dict(dims=80), dict(d_q_norm=8),
                dict(d_k_norm=8200), dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf)]
BAD_ROWS = [dict(d_k=0), dict(d_k=8), dict(d_q=8), dict(d_q_out=0), dict(d_q_out=8), dict(dtype=1), dict(dtype=MX), dict(dtype=3), dict(head_dim=96), dict(head_dim=0),
            dict(kv_heads=0), dict(kv_heads=4097), dict(q_heads=0), dict(q_heads=-1), dict(rows=0), dict(rows=-3), dict(d_k_out=8), dict(q_stride=[4096, 256, 60]),
            dict(k_stride=[-8, 256, 64]), dict(k_stride=[1 << 48, 256, 64]), dict(q_out_stride=[4096, 4, 64]), dict(k_out_stride=[4, 256, 64]),
            dict(d_q_out=4096, q_out_stride=[4096, 256, 128]), dict(d_k_out=8192, k_out_stride=[2048, 256, 64])]


def test_refusals_of_the_rotation(lib):
    def call(B=3, N=9, r=None, length=64, tok=64, no_rows=False, no_rotation=False, **kw):
        return lib.rotate(B, N, None if no_rotation else C.byref(r or rotation()), length, tok, None if no_rows else C.byref(rows(**kw)))

    assert call() == 0 and call(d_q=0, d_q_out=0, q_heads=0) == 0 and call(B=65535) == 0 and call(d_v=0) == 0
    assert call(d_q_out=4096, d_k_out=8192) == 0             # in place
    for r in (dict(dims=0, d_turns=0, positions=0), dict(dims=16), dict(neighbours=1), dict(d_k_norm=0, eps=math.nan), dict(eps=0.0)):
        assert call(r=rotation(**r)) == 0, r
    for r in BAD_ROTATION:
        assert call(r=rotation(**r)) == EINVAL, r
    # outputs that repeat a place
    for out in ("q_out_stride", "k_out_stride"):
        for i in range(3):
            zero = [0 if i == j else s for j, s in enumerate((4096, 256, 64))]
            assert call(**{out: zero}) == EINVAL and call(d_q_out=4096, d_k_out=8192, **{out: zero, out.replace("_out", ""): zero}) == EINVAL
            assert call(**{out.replace("_out", ""): zero}) == 0
    assert call(B=1, q_out_stride=[0, 256, 64]) == 0 and call(N=1, rows=1, k_out_stride=[4096, 0, 64]) == 0 and call(kv_heads=1, k_out_stride=[4096, 256, 0]) == 0
    for kw in BAD_ROWS + [dict(d_k_out=0), dict(length=0), dict(tok=0), dict(N=8), dict(no_rows=True), dict(no_rotation=True)]:
        assert call(**kw) == EINVAL, kw
    assert call(B=65536) == ELIMIT and call(q_heads=65536) == ELIMIT


def test_refusals_of_the_append(lib):
    def call(B=3, c=None, layer=1, r=None, slots=64, width=9, no_rows=False, no_rotation=False, **kw):
        return lib.append(B, C.byref(c or cache(dtype=BF)), layer, None if no_rotation else C.byref(r or rotation()), None if no_rows else C.byref(rows(**kw)),
                          slots, width)

    assert call() == 0 and call(no_rotation=True) == 0 and call(d_k_out=0) == 0 and call(d_q=0, d_q_out=0) == 0 and call(width=1 << 30) == 0
    assert call(c=cache()) == 0 and call(c=cache(dtype=MX + HF), dtype=HF) == 0
    for r in BAD_ROTATION:
        assert call(r=rotation(**r)) == EINVAL, r
    for kw in BAD4:
        assert call(c=cache(**kw)) == EINVAL, kw
    for kw in BAD_ROWS + [dict(d_v=0), dict(d_v=8), dict(v_stride=[1, 256, 64]), dict(layer=-1), dict(layer=2), dict(slots=0), dict(width=8), dict(width=(1 << 30) + 1),
                          dict(no_rows=True), dict(dtype=HF), dict(kv_heads=3), dict(head_dim=128), dict(c=cache(dtype=HF)), dict(c=cache(dtype=MX + HF))]:
        assert call(**kw) == EINVAL, kw
    assert call(B=65536) == ELIMIT and call(q_heads=65536) == ELIMIT
    # workgroups of a launch's dimension, 64 heads of 64 each
    assert call(rows=1 << 29, width=1 << 29, d_q=0, d_q_out=0, d_k_out=0) == ELIMIT
    assert call(rows=1 << 28, width=1 << 28, d_q=0, d_q_out=0, d_k_out=0) == ELIMIT and call(rows=(1 << 28) - 64, width=1 << 28, d_q=0, d_q_out=0) == 0
    assert lib.groups(1, 1, 64) == 1 and lib.groups(9, 64, 64) == 9 and lib.groups(9, 33, 128) == 10 and lib.groups(1 << 30, 65535, 128) == (1 << 30) * 65535 // 32


def test_refusals_of_the_read(lib):
    def call(B=3, c=None, first=0, layers=2, table=64, width=9, no_rows=False, **kw):
        d = dict(d_k=4096, d_v=8192, rows=7, layer_stride=4096, batch_stride=2048, row_stride=128, head_stride=64)
        d.update(kw)
        return lib.rd(B, C.byref(c or cache()), first, layers, table, width, None if no_rows else C.byref(Out(**d)))

    assert call() == 0 and call(first=1, layers=1) == 0 and call(c=cache(dtype=HF)) == 0 and call(B=65535, rows=1 << 30) == 0
    for kw in BAD4:
        assert call(c=cache(**kw)) == EINVAL, kw
    for kw in (dict(first=-1), dict(first=1), dict(first=2, layers=1), dict(layers=0), dict(layers=3), dict(layers=2 ** 31 - 1, first=1), dict(table=0), dict(width=0), dict(width=(1 << 26) + 1),
               dict(no_rows=True), dict(d_k=0), dict(d_v=0), dict(d_k=8), dict(d_v=8), dict(rows=0), dict(rows=(1 << 30) + 1), dict(layer_stride=4), dict(batch_stride=-8),
               dict(row_stride=1 << 48), dict(head_stride=12),
               dict(layer_stride=0), dict(batch_stride=0), dict(row_stride=0), dict(head_stride=0)):
        assert call(**kw) == EINVAL, kw
    assert call(B=65536) == ELIMIT and call(c=cache(layers=65536), layers=65536) == ELIMIT

"""The host side of the operators around a verification (csrc/attn_plan.hpp, csrc/serve_checks.hpp, plain host code), compiled
with the host compiler: how the attention's work is cut, and what the calls refuse."""
import ctypes as C
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
_SRC = """
#include "serve_checks.hpp"
using namespace stand;
extern "C" {
int64_t units(int64_t len, int64_t most, int nodes, int keys) { return item_units(len, most, nodes, keys); }
int64_t head(int rows, int tile, int heavy, int light) { return head_weight(rows, tile, heavy, light); }
int weight(int rows, int tile, int heavy, int light) { return tile_weight(rows, tile, heavy, light); }
int64_t before(int64_t place, int weight, int start, int64_t units) { return units_before(place, weight, start, units); }
int64_t groups(int64_t total, int launched, int start, int heavy) { return attn_groups(total, launched, start, heavy); }
int64_t begin(int64_t w, int64_t total, int64_t W) { return group_start(w, total, W); }
int64_t owner(int64_t unit, int64_t total, int64_t W) { return group_of(unit, total, W); }
int64_t first(int64_t item, int64_t total, int64_t W, int start, int weight) { return first_group(item, total, W, start, weight); }
int page(int p, int pages) { return clamp_page(p, pages); }
int64_t length(int64_t len, int64_t most) { return clamp_length(len, most); }
int attention(int64_t B, const stand_cache *c, int layer, const int32_t *len, const int32_t *table, int width, const int32_t *tok,
              const stand_tree_rows *rows, void *work) { return check_tree_attention(B, c, layer, len, table, width, tok, rows, work); }
int commit(int64_t B, const stand_cache *c, const stand_cache_rows *rows, const int64_t *slots, int width) { return check_cache_commit(B, c, rows, slots, width); }
int cache_pages(int64_t B, const stand_pages *p, const int64_t *slots, int width, const int32_t *missing, const stand_pages *out)
{ return check_cache_pages(B, p, slots, width, missing, out); }
int shape(int64_t B, int dtype, const void *x, const void *out, const int32_t *tok, const int32_t *id, const float *bias, int width)
{ return check_shape_logits(B, dtype, x, out, tok, id, bias, width); }
int count(int64_t B, const int32_t *c, const int32_t *tok, int width) { return check_count_tokens(B, c, tok, width); }
}
"""
_lib = None


class Cache(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("dtype", C.c_int32), ("layers", C.c_int32), ("pages", C.c_int32),
                ("page_size", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("layer_stride", C.c_int64),
                ("page_stride", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64)]


class TreeRows(C.Structure):
    _fields_ = [("d_q", C.c_void_p), ("d_k", C.c_void_p), ("d_v", C.c_void_p), ("d_out", C.c_void_p), ("q_heads", C.c_int32),
                ("scale", C.c_float), ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3),
                ("out_stride", C.c_int64 * 3)]


class CacheRows(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("rows", C.c_int32), ("layer_stride", C.c_int64), ("batch_stride", C.c_int64),
                ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class Pages(C.Structure):
    _fields_ = [("d_table", C.c_void_p), ("d_ring", C.c_void_p), ("d_length", C.c_void_p), ("d_held", C.c_void_p), ("d_mark", C.c_void_p),
                ("width", C.c_int32), ("pages", C.c_int32), ("page_size", C.c_int32)]


def lib():
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            src, so = os.path.join(d, "serve.cpp"), os.path.join(d, "serve.so")
            open(src, "w").write(_SRC)
            subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I",
                            os.path.join(ROOT, "paper_2506_04708_amd", "csrc"), "-o", so, src], check=True)
            _lib = C.CDLL(so)
        i, l, p = C.c_int, C.c_int64, C.c_void_p
        for name, args, res in (("units", [l, l, i, i], l), ("head", [i, i, i, i], l), ("weight", [i, i, i, i], i),
                                ("before", [l, i, i, l], l), ("groups", [l, i, i, i], l),
                                ("begin", [l, l, l], l), ("owner", [l, l, l], l), ("first", [l, l, l, i, i], l), ("page", [i, i], i),
                                ("length", [l, l], l), ("attention", [l, p, i, p, p, i, p, p, p], i), ("commit", [l, p, p, p, i], i),
                                ("cache_pages", [l, p, p, i, p, p], i), ("shape", [l, i, p, p, p, p, p, i], i), ("count", [l, p, p, i], i)):
            f = getattr(_lib, name)
            f.argtypes, f.restype = args, res
    return _lib

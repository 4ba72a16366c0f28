"""Thin ctypes binding of libstand.so (see include/stand.h): argument marshalling only.

Device buffers are torch tensors (PyTorch-ROCm is used for memory and streams, nothing else);
every step of the path runs in the HIP kernels of the library.  There is no CPU fallback: if
the library has not been built, importing this module raises.
"""
import ctypes as C
import os
import struct

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libstand.so")

STAND_BF16, STAND_F32, STAND_F16, STAND_MXFP4 = 0, 1, 2, 4
DRAFT_GUMBEL_TOPK, DRAFT_MULTINOMIAL, DRAFT_DETERMINISTIC = 0, 1, 2
MERGE_MEAN, MERGE_REPLACE = 0, 1
STEP_AUTO, STEP_SERIAL, STEP_FUSED = 0, 1, 2
MAX_ORDER = 8

EXPORTED = [
    "stand_create", "stand_destroy", "stand_depth", "stand_set_context", "stand_reorder", "stand_update",
    "stand_draft", "stand_verify", "stand_step", "stand_row_results", "stand_table_export", "stand_table_import",
    "stand_get_context", "stand_get_stats", "stand_strerror", "stand_last_hip_error",
    "stand_profile_begin", "stand_profile_end", "stand_copy_bytes", "stand_read_rows", "stand_set_filter_margin",
    "stand_tree_initial", "stand_tree_select", "stand_get_node_counts", "stand_reset_node_counts",
    "stand_tree_packing", "stand_verify_static", "stand_static_scratch_need",
    "stand_set_step_plan", "stand_set_wait_limit", "stand_step_timeline", "stand_step_is_one_launch",
    "stand_get_record_slots",
    "stand_tree_attention", "stand_tree_attention_work", "stand_cache_commit", "stand_cache_pages", "stand_shape_logits",
    "stand_shape_logits_work",    "stand_count_tokens",
    "stand_tree_rotate", "stand_cache_append", "stand_cache_read",
]


class Config(C.Structure):
    _fields_ = [
        ("vocab", C.c_int32), ("max_batch", C.c_int32), ("order_min", C.c_int32), ("order_max", C.c_int32),
        ("topk", C.c_int32), ("tree_nodes", C.c_int32), ("tree_parent", C.POINTER(C.c_int32)),
        ("temperature", C.c_float), ("table_capacity", C.c_uint64), ("max_probe", C.c_int32),
        ("seed", C.c_uint64), ("logits_dtype", C.c_int32), ("update_mode", C.c_int32), ("device", C.c_int32),
        ("draft_mode", C.c_int32), ("merge_policy", C.c_int32),
    ]


class Stats(C.Structure):
    _fields_ = [
        ("hits", C.c_uint64 * (MAX_ORDER + 1)), ("misses", C.c_uint64),
        ("inserts", C.c_uint64), ("merges", C.c_uint64), ("drops", C.c_uint64),
        ("near_threshold", C.c_uint64), ("tokens_emitted", C.c_uint64), ("accept_tests", C.c_uint64),
        ("filter_mismatch", C.c_uint64), ("wait_expired", C.c_uint64), ("late_paths", C.c_uint64),
    ]


class CacheDesc(C.Structure):
    _fields_ = [
        ("d_k", C.c_void_p), ("d_v", C.c_void_p), ("dtype", C.c_int32), ("layers", C.c_int32), ("pages", C.c_int32),
        ("page_size", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("layer_stride", C.c_int64),
        ("page_stride", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64),
    ]


class Cache4Desc(C.Structure):
    _fields_ = [
        ("cache", CacheDesc), ("d_k_scale", C.c_void_p), ("d_v_scale", C.c_void_p), ("scale_layer_stride", C.c_int64),
        ("scale_page_stride", C.c_int64), ("scale_slot_stride", C.c_int64), ("scale_head_stride", C.c_int64),
    ]


class RotationDesc(C.Structure):
    _fields_ = [
        ("d_turns", C.c_void_p), ("positions", C.c_int32), ("dims", C.c_int32), ("neighbours", C.c_int32), ("eps", C.c_float),
        ("d_q_norm", C.c_void_p), ("d_k_norm", C.c_void_p),
    ]


# stand_tree_rows, stand_cache_rows (and stand_cache_rows_out) and stand_turned_rows, filled in anew by every call (a ctypes structure
# takes three times as long)
_TREE_ROWS = struct.Struct("@4Pif12q")
_CACHE_ROWS = struct.Struct("@2Pi4x4q")
_TURNED_ROWS = struct.Struct("@5P5i4x15q")


class PagesDesc(C.Structure):
    _fields_ = [
        ("d_table", C.c_void_p), ("d_ring", C.c_void_p), ("d_length", C.c_void_p), ("d_held", C.c_void_p),
        ("d_mark", C.c_void_p), ("width", C.c_int32), ("pages", C.c_int32), ("page_size", C.c_int32),
    ]


def load_library():
    if not os.path.exists(LIB_PATH):
        raise ImportError("libstand.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                          "(or python -m paper_2506_04708_amd.build) first; there is no fallback path")
    lib = C.CDLL(LIB_PATH)
    vp, i32p = C.c_void_p, C.c_void_p
    lib.stand_create.argtypes = [C.POINTER(Config), C.POINTER(vp)]
    lib.stand_destroy.argtypes = [vp]
    lib.stand_depth.argtypes = [vp]
    lib.stand_set_context.argtypes = [vp, C.c_int32, i32p, C.c_int32, vp]
    lib.stand_reorder.argtypes = [vp, i32p, vp]
    lib.stand_update.argtypes = [vp, C.c_uint64, vp, i32p, i32p, i32p, vp]
    lib.stand_draft.argtypes = [vp, C.c_uint64, i32p, vp]
    lib.stand_verify.argtypes = [vp, C.c_uint64, vp, i32p, i32p, i32p, vp]
    lib.stand_verify_static.argtypes = [vp, C.c_uint64, vp, i32p, i32p, i32p, vp]
    lib.stand_static_scratch_need.argtypes = [vp]
    lib.stand_static_scratch_need.restype = C.c_uint64
    lib.stand_set_step_plan.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_uint32]
    lib.stand_set_wait_limit.argtypes = [vp, C.c_uint64]
    lib.stand_step_is_one_launch.argtypes = [vp]
    lib.stand_step_timeline.argtypes = [vp, C.c_int32, vp, C.POINTER(C.c_uint64)]
    lib.stand_step.argtypes = [vp, C.c_uint64, vp, i32p, i32p, i32p, i32p, i32p, vp]
    lib.stand_row_results.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.stand_table_export.argtypes = [vp, vp, C.POINTER(C.c_uint64)]
    lib.stand_table_import.argtypes = [vp, vp, C.c_uint64]
    lib.stand_get_context.argtypes = [vp, C.c_int32, i32p, C.c_int32, C.POINTER(C.c_int64), vp]
    lib.stand_get_stats.argtypes = [vp, C.POINTER(Stats)]
    lib.stand_set_filter_margin.argtypes = [vp, C.c_float]
    lib.stand_profile_begin.argtypes = [vp, C.c_int32]
    lib.stand_profile_end.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int32)]
    lib.stand_copy_bytes.argtypes = [vp, vp, C.c_uint64, vp]
    lib.stand_read_rows.argtypes = [vp, C.c_uint64, C.c_uint64, vp, vp]
    lib.stand_tree_initial.argtypes = [C.c_int32, i32p, C.c_int32, C.POINTER(C.c_int32)]
    lib.stand_tree_select.argtypes = [i32p, vp, C.c_int32, C.c_int32, i32p, i32p]
    lib.stand_get_node_counts.argtypes = [vp, vp]
    lib.stand_get_record_slots.argtypes = [vp, vp]
    lib.stand_tree_packing.argtypes = [vp, vp, vp, vp]
    lib.stand_reset_node_counts.argtypes = [vp]
    lib.stand_tree_attention.argtypes = [vp, vp, C.c_int32, vp, vp, C.c_int32, vp, vp, vp, C.c_uint64, vp]
    lib.stand_tree_attention_work.argtypes = [vp, vp, C.c_int32]
    lib.stand_tree_attention_work.restype = C.c_uint64
    lib.stand_cache_commit.argtypes = [vp, vp, vp, vp, C.c_int32, vp, vp, vp]
    lib.stand_cache_pages.argtypes = [vp, vp, vp, vp, vp, C.c_int32, vp, vp, vp]
    lib.stand_shape_logits.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, C.c_int32, vp, vp, C.c_uint64, vp]
    lib.stand_shape_logits_work.argtypes = [vp]
    lib.stand_shape_logits_work.restype = C.c_uint64
    lib.stand_count_tokens.argtypes = [vp, vp, vp, vp, C.c_int32, C.c_int32, vp]
    lib.stand_tree_rotate.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.stand_cache_append.argtypes = [vp, vp, C.c_int32, vp, vp, vp, vp, C.c_int32, vp, vp]
    lib.stand_cache_read.argtypes = [vp, vp, C.c_int32, C.c_int32, vp, C.c_int32, vp, vp, vp, vp]
    lib.stand_strerror.restype = C.c_char_p
    lib.stand_strerror.argtypes = [C.c_int]
    lib.stand_last_hip_error.argtypes = [vp]
    return lib


_lib = None


def copy_bytes(dst, src, nbytes, stream=None):
    """Plain device copy (measurement aid): dst, src are torch tensors on the GPU."""
    rc = lib().stand_copy_bytes(dst.data_ptr(), src.data_ptr(), nbytes, stream)
    if rc:
        raise RuntimeError("stand_copy_bytes: %s" % lib().stand_strerror(rc).decode())


def read_rows(src, row_bytes, rows, sink, stream=None):
    """Bare read of `rows` rows in the row pass's launch shape (measurement aid); sink: int32 tensor of 4 * rows."""
    rc = lib().stand_read_rows(src.data_ptr(), row_bytes, rows, sink.data_ptr(), stream)
    if rc:
        raise RuntimeError("stand_read_rows: %s" % lib().stand_strerror(rc).decode())


def tree_initial(levels=20):
    """parent[] of the initial tree of the tree optimisation (host only)."""
    n = C.c_int32(0)
    rc = lib().stand_tree_initial(levels, None, 0, C.byref(n))
    if rc:
        raise RuntimeError("stand_tree_initial: %s" % lib().stand_strerror(rc).decode())
    out = np.zeros(n.value, np.int32)
    rc = lib().stand_tree_initial(levels, out.ctypes.data, n.value, C.byref(n))
    if rc:
        raise RuntimeError("stand_tree_initial: %s" % lib().stand_strerror(rc).decode())
    return out


def tree_select(parent, counts, n_keep):
    """(new parent[], old ids) of the n_keep most often accepted nodes, re-packed (host only)."""
    parent = np.ascontiguousarray(parent, np.int32)
    counts = np.ascontiguousarray(counts, np.uint64)
    out = np.zeros(n_keep, np.int32)
    old = np.zeros(n_keep, np.int32)
    rc = lib().stand_tree_select(parent.ctypes.data, counts.ctypes.data, parent.shape[0], n_keep, out.ctypes.data,
                                 old.ctypes.data)
    if rc:
        raise RuntimeError("stand_tree_select: %s" % lib().stand_strerror(rc).decode())
    return out, old


def lib():
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


class StandError(RuntimeError):
    pass


def _check(rc, handle=None):
    if rc:
        msg = lib().stand_strerror(rc).decode()
        if handle is not None and rc == -3:
            msg += " [hip error %d]" % lib().stand_last_hip_error(handle)
        raise StandError("libstand: %s (%d)" % (msg, rc))


def _dptr(t, dtype=None):
    # (a plain integer: the functions' argtypes make the pointer)
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous()
    if dtype is not None:
        assert t.dtype is dtype, (t.dtype, dtype)
    return t.data_ptr()


def _stream_ptr():
    return torch.cuda.current_stream().cuda_stream


# The same for calls that have just been given tensors of the GPU (torch's runtime is up): without the stream object, which
# costs more than the rest of such a call's arguments together.
try:
    _raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice

    def _stream_ptr_up():
        return _raw_stream(_device())
except AttributeError:   # (a torch without them)
    _stream_ptr_up = _stream_ptr


def _stream_of(device):
    return torch.cuda.current_stream(device).cuda_stream


try:
    _stream_of = _raw_stream
except NameError:
    pass


_HALF = {torch.bfloat16: STAND_BF16, torch.float16: STAND_F16}


class PagedCache:
    """Keys and values of a paged cache: tensors indexed [layer, page, place, head, element], any strides but for the last.  In 4 bits: bytes
    of two elements [.., d / 2] with their blocks' scales [.., d / 32], also bytes, and the type of the rows given with the cache."""

    def __init__(self, k, v, k_scale=None, v_scale=None, dtype=None):
        assert k.dim() == 5 and k.shape == v.shape and k.stride() == v.stride() and k.dtype == v.dtype and k.device == v.device
        assert k.is_cuda and k.stride(4) == 1 and (k_scale is None) == (v_scale is None) == (dtype is None)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.index, (self.layers, self.pages, self.page_size, self.heads, self.dim) = k.get_device(), k.shape
        if k_scale is None:
            assert k.dtype in _HALF
            self.dtype = k.dtype
            self.desc = CacheDesc(k.data_ptr(), v.data_ptr(), _HALF[k.dtype], *k.shape, *k.stride()[:4])
        else:
            assert k.dtype is k_scale.dtype is v_scale.dtype is torch.uint8 and dtype in _HALF
            self.dtype, self.dim = dtype, 2 * self.dim
            assert k_scale.shape == v_scale.shape == (*k.shape[:4], self.dim // 32) and k_scale.stride() == v_scale.stride() and k_scale.stride(4) == 1
            assert k_scale.device == v_scale.device == k.device
            desc = CacheDesc(k.data_ptr(), v.data_ptr(), STAND_MXFP4 + _HALF[dtype], *k.shape[:4], self.dim, *(2 * s for s in k.stride()[:4]))
            self.whole = Cache4Desc(desc, k_scale.data_ptr(), v_scale.data_ptr(), *k_scale.stride()[:4])
            self.desc = self.whole.cache    # (its first member, in place)
        self.ref = C.addressof(self.desc)

    @classmethod
    def new4(cls, layers, pages, page_size, heads, dim, dtype=torch.bfloat16, device="cuda"):
        """An empty cache of 4 bits, to be given rows of `dtype`."""
        k, v = (torch.zeros((layers, pages, page_size, heads, dim // 2), dtype=torch.uint8, device=device) for _ in range(2))
        ks, vs = (torch.full((layers, pages, page_size, heads, dim // 32), 127, dtype=torch.uint8, device=device) for _ in range(2))
        return cls(k, v, ks, vs, dtype)


class Rotation:
    """Rotation of heads by positions, and norms of heads before it (stand_rotation): turns [positions, dims] fp32, cosines of the dims / 2
    pairs, then their sines (None: no rotation); pairs "halves" (dims / 2 apart) or "neighbours"; weights [d] of the rows' type or None."""

    def __init__(self, turns=None, pairs="halves", q_norm=None, k_norm=None, eps=1e-6):
        assert pairs in ("halves", "neighbours") and (turns is None or (turns.dim() == 2 and turns.dtype is torch.float32 and turns.is_contiguous()))
        some = [t for t in (turns, q_norm, k_norm) if t is not None]
        norms = [t for t in (q_norm, k_norm) if t is not None]
        assert all(t.is_cuda and t.device == some[0].device for t in some)
        assert all(t.dim() == 1 and t.is_contiguous() and t.dtype is norms[0].dtype and t.shape == norms[0].shape for t in norms)
        self.turns, self.q_norm, self.k_norm = turns, q_norm, k_norm
        self.index = some[0].get_device() if some else None
        self.dtype, self.dim = (norms[0].dtype, norms[0].shape[0]) if norms else (None, None)
        positions, dims = (0, 0) if turns is None else turns.shape
        self.desc = RotationDesc(None if turns is None else turns.data_ptr(), positions, dims, int(pairs == "neighbours"), eps,
                                 *(None if t is None else t.data_ptr() for t in (q_norm, k_norm)))
        self.ref = C.addressof(self.desc)

    def fits(self, dtype, dim, index):
        return self.index in (None, index) and (self.dtype is None or (self.dtype is dtype and self.dim == dim))


class Pages:
    """Block tables, lengths and the ring of free pages of a cache (stand_pages)."""

    def __init__(self, page_size, table, ring, length, held, mark):
        assert table.dim() == 2 and length.shape == held.shape == table.shape[:1] and mark.shape == (2,) and ring.dim() == 1
        assert all(t.device == table.device for t in (ring, length, held, mark))
        self.page_size, self.table, self.ring, self.length, self.held, self.mark = page_size, table, ring, length, held, mark
        self.desc = PagesDesc(*[_dptr(t, torch.int32) for t in (table, ring, length, held)], _dptr(mark, torch.int64),
                              table.shape[1], ring.shape[0], page_size)
        self.ref, self.index = C.addressof(self.desc), table.get_device()

    @classmethod
    def new(cls, batch, pages, page_size, width, device="cuda"):
        """Nothing in the cache, all pages free."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(page_size, torch.full((batch, width), -1, **i32), torch.arange(pages, **i32), torch.zeros(batch, **i32),
                   torch.zeros(batch, **i32), torch.tensor([0, pages], dtype=torch.int64, device=device))

    def beside(self):
        """Other lengths, held counts and marks beside the same table and ring."""
        return Pages(self.page_size, self.table, self.ring, *(torch.empty_like(t) for t in (self.length, self.held, self.mark)))


class Stand:
    """One n-gram table shared by B trajectories on one GPU; methods carry the C ABI's names."""

    def __init__(self, vocab, max_batch, order_min, order_max, topk, tree_parent, temperature, table_capacity,
                 max_probe, seed, logits_dtype, device=0, draft_mode=0, update_mode=0, merge_policy=0):
        par = np.ascontiguousarray(tree_parent, dtype=np.int32)
        cfg = Config(vocab, max_batch, order_min, order_max, topk, par.shape[0],
                     par.ctypes.data_as(C.POINTER(C.c_int32)), temperature, table_capacity, max_probe, seed,
                     logits_dtype, update_mode, device, draft_mode, merge_policy)
        self.h = C.c_void_p()
        _check(lib().stand_create(C.byref(cfg), C.byref(self.h)))
        self.B, self.N, self.K, self.V = max_batch, par.shape[0], topk, vocab
        self._lib, self._logits = lib(), max_batch * par.shape[0] * vocab
        self.D = lib().stand_depth(self.h)
        self.W = self.D + 1
        self.logits_dtype = logits_dtype
        self.device = torch.device("cuda", device)
        self._index = device
        self._work_bytes = {}   # of an attention, by its heads and type

    def close(self):
        if getattr(self, "h", None):
            lib().stand_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _logits_ptr(self, logits):
        assert logits.is_cuda and logits.is_contiguous() and logits.numel() == self._logits
        if self.logits_dtype == STAND_BF16:
            assert logits.dtype in (torch.bfloat16, torch.uint16, torch.int16)
        else:
            assert logits.dtype == torch.float32
        return logits.data_ptr()

    def new_outputs(self):
        i32 = dict(dtype=torch.int32, device=self.device)
        return (torch.empty((self.B, self.W), **i32), torch.empty((self.B, self.W), **i32),
                torch.empty((self.B,), **i32), torch.empty((self.B, self.N), **i32))

    def set_context(self, b, tokens):
        t = np.ascontiguousarray(tokens, dtype=np.int32)
        _check(lib().stand_set_context(self.h, b, t.ctypes.data_as(C.c_void_p), t.shape[0], _stream_ptr()), self.h)

    def reorder(self, src_of):
        s = np.ascontiguousarray(src_of, dtype=np.int32)
        assert s.shape[0] == self.B
        _check(lib().stand_reorder(self.h, s.ctypes.data_as(C.c_void_p), _stream_ptr()), self.h)

    def update(self, step, logits, commit_tok, commit_row, commit_len):
        assert commit_tok.shape == (self.B, self.W) and commit_row.shape == (self.B, self.W) and commit_len.shape == (self.B,)
        _check(self._lib.stand_update(self.h, step, self._logits_ptr(logits), _dptr(commit_tok, torch.int32),
                                  _dptr(commit_row, torch.int32), _dptr(commit_len, torch.int32), _stream_ptr_up()), self.h)

    def draft(self, step, draft_tok):
        assert draft_tok.shape == (self.B, self.N)
        _check(self._lib.stand_draft(self.h, step, _dptr(draft_tok, torch.int32), _stream_ptr_up()), self.h)

    def verify(self, step, logits, out_tok, out_node, out_len):
        _check(self._lib.stand_verify(self.h, step, self._logits_ptr(logits), _dptr(out_tok, torch.int32),
                                  _dptr(out_node, torch.int32), _dptr(out_len, torch.int32), _stream_ptr_up()), self.h)

    def verify_static(self, step, logits, out_tok, out_node, out_len):
        _check(self._lib.stand_verify_static(self.h, step, self._logits_ptr(logits), _dptr(out_tok, torch.int32),
                                         _dptr(out_node, torch.int32), _dptr(out_len, torch.int32), _stream_ptr_up()), self.h)

    def static_scratch_need(self):
        return int(lib().stand_static_scratch_need(self.h))

    def step(self, step, logits, out_tok, out_node, out_len, next_draft_tok, force_tok=None):
        _check(self._lib.stand_step(self.h, step, self._logits_ptr(logits), _dptr(out_tok, torch.int32),
                                _dptr(out_node, torch.int32), _dptr(out_len, torch.int32),
                                _dptr(next_draft_tok, torch.int32), _dptr(force_tok, torch.int32), _stream_ptr_up()), self.h)

    def row_results(self):
        rows = self.B * self.N
        m = torch.empty(rows, dtype=torch.float32, device=self.device)
        s = torch.empty(rows, dtype=torch.float32, device=self.device)
        idx = torch.empty((rows, self.K), dtype=torch.int32, device=self.device)
        p = torch.empty((rows, self.K), dtype=torch.float32, device=self.device)
        _check(self._lib.stand_row_results(self.h, _dptr(m), _dptr(s), _dptr(idx), _dptr(p), _stream_ptr_up()), self.h)
        return m, s, idx, p

    def table_export(self):
        n = C.c_uint64(0)
        _check(lib().stand_table_export(self.h, None, C.byref(n)), self.h)
        buf = np.zeros(max(int(n.value), 1), np.uint8)
        n2 = C.c_uint64(buf.shape[0])
        _check(lib().stand_table_export(self.h, buf.ctypes.data_as(C.c_void_p), C.byref(n2)), self.h)
        return buf[: int(n2.value)]

    def table_import(self, buf):
        b = np.ascontiguousarray(buf, dtype=np.uint8)
        _check(lib().stand_table_import(self.h, b.ctypes.data_as(C.c_void_p), b.shape[0]), self.h)

    def get_context(self, b, n):
        out = np.zeros(max(n, 1), np.int32)
        ln = C.c_int64(0)
        _check(lib().stand_get_context(self.h, b, out.ctypes.data_as(C.c_void_p), n, C.byref(ln), _stream_ptr()), self.h)
        return out[:n], int(ln.value)

    def set_step_plan(self, mode=0, upper_depth=2, tail_groups=0, shuffle=0, rows_first=0):
        _check(lib().stand_set_step_plan(self.h, mode, upper_depth, tail_groups, rows_first, shuffle), self.h)

    def step_is_one_launch(self):
        return lib().stand_step_is_one_launch(self.h) == 1

    def set_wait_limit(self, microseconds):
        _check(lib().stand_set_wait_limit(self.h, microseconds), self.h)

    def step_timeline(self, enable=True, read=False):
        """Switches the recording of the one-launch step's clock readings on or off; with read=True returns
        (row_start, row_end, per-trajectory stamps [B, 8]) of the last such step in microseconds from row_start."""
        rate = C.c_uint64(0)
        buf = np.zeros(2 + 8 * self.B, np.uint64) if read else None
        _check(lib().stand_step_timeline(self.h, int(enable), buf.ctypes.data if read else None, C.byref(rate)), self.h)
        if not read:
            return None
        us = (buf.astype(np.int64) - np.int64(buf[0])) * (1e6 / rate.value)
        return float(us[0]), float(us[1]), us[2:].reshape(self.B, 8)

    def set_filter_margin(self, margin):
        _check(lib().stand_set_filter_margin(self.h, margin), self.h)

    def profile_begin(self, max_launches):
        _check(lib().stand_profile_begin(self.h, max_launches), self.h)

    def profile_end(self):
        ms = C.c_double(0)
        n = C.c_int32(0)
        _check(lib().stand_profile_end(self.h, C.byref(ms), C.byref(n)), self.h)
        return ms.value, n.value

    def stats(self):
        s = Stats()
        _check(lib().stand_get_stats(self.h, C.byref(s)), self.h)
        return s

    def tree_packing(self):
        """(mask [B, N, N] uint8, positions [B, N] int64) of the pending drafts, on the GPU."""
        mask = torch.empty((self.B, self.N, self.N), dtype=torch.uint8, device=self.device)
        pos = torch.empty((self.B, self.N), dtype=torch.int64, device=self.device)
        _check(self._lib.stand_tree_packing(self.h, _dptr(mask), _dptr(pos), _stream_ptr_up()), self.h)
        return mask, pos

    def _arg(self, t, dtype):
        """Pointer of a contiguous tensor on the handle's device (None: none)."""
        if t is None:
            return None
        assert t.dtype is dtype and t.get_device() == self._index and t.is_contiguous(), (t.dtype, dtype, t.device)
        return t.data_ptr()

    def _stream(self):
        # the caller's stream on the handle's device, whichever device is the current one
        return _stream_of(self._index)

    def tree_attention(self, cache, layer, length, table, draft_tok, q, k, v, scale=None, out=None):
        """Attention of the drafted nodes over the cache's first length[b] tokens and their own ancestors: q [B, N, heads, d],
        k, v [B, N, kv heads, d] (slices of a fused projection are fine) -> out, like q."""
        B, N, H, d = shape = q.shape
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=q.device)
        assert B == self.B and N == self.N and d == cache.dim and k.shape == v.shape == (B, N, cache.heads, d) and out.shape == shape
        assert cache.dtype is q.dtype and cache.dtype is k.dtype and cache.dtype is v.dtype and cache.dtype is out.dtype
        (q0, q1, q2, q3), (k0, k1, k2, k3), (v0, v1, v2, v3), (o0, o1, o2, o3) = q.stride(), k.stride(), v.stride(), out.stride()
        assert q3 == k3 == v3 == o3 == 1
        rows, width = table.shape
        assert rows == B and length.shape == (B,) and draft_tok.shape == (B, N)
        assert self._index == cache.index == q.get_device() == k.get_device() == v.get_device() == out.get_device()
        desc = _TREE_ROWS.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), H, d ** -0.5 if scale is None else scale,
                               q0, q1, q2, k0, k1, k2, v0, v1, v2, o0, o1, o2)
        key = (H, cache.heads, d, cache.desc.dtype)
        need = self._work_bytes.get(key)
        if not need:
            need = self._work_bytes[key] = self._lib.stand_tree_attention_work(self.h, cache.ref, H)
        # (torch's allocator hands this memory on in the order of the stream, and keeps a captured graph's apart)
        work = torch.empty(max(need, 16), dtype=torch.uint8, device=self.device)
        _check(self._lib.stand_tree_attention(self.h, cache.ref, layer, self._arg(length, torch.int32), self._arg(table, torch.int32), width,
                                              self._arg(draft_tok, torch.int32), desc, work.data_ptr(), need, self._stream()), self.h)
        return out

    def cache_commit(self, cache, k, v, slots, row=None, count=None):
        """Rows k, v [layers, B, rows, kv heads, d] into the cache: row[b][j] (None: j) to slots[b][j], j < count[b] (None: all)."""
        layers, B, rows, heads, d = k.shape
        stride = k.stride()
        assert k.shape == v.shape and stride == v.stride() and stride[4] == 1 and cache.dtype is k.dtype and cache.dtype is v.dtype
        assert layers == cache.layers and B == self.B and heads == cache.heads and d == cache.dim
        assert slots.dim() == 2 and slots.shape[0] == B and (row is None or row.shape == slots.shape) and (count is None or count.shape == (B,))
        assert self._index == cache.index == k.get_device() == v.get_device()
        desc = _CACHE_ROWS.pack(k.data_ptr(), v.data_ptr(), rows, *stride[:4])
        _check(self._lib.stand_cache_commit(self.h, cache.ref, desc, self._arg(slots, torch.int64), slots.shape[1],
                                            self._arg(row, torch.int32), self._arg(count, torch.int32), self._stream()), self.h)

    def _turned(self, dtype, shape, q, k, v, q_out, k_out):
        """stand_turned_rows of k, whose shape is [B, rows, kv heads, d], and what goes with it."""
        B, rows, heads, d = shape
        index, of_q, zero = self._index, 0, (0, 0, 0)
        k0, k1, k2, k3 = k.stride()
        assert dtype in _HALF and B == self.B and k.get_device() == index and k.dtype is dtype and k3 == 1
        qs = vs = qos = kos = zero
        pq = pv = pqo = pko = 0
        if q is None:
            assert q_out is None
        else:
            q_shape = q.shape
            q_batch, q_rows, of_q, q_dim = q_shape
            *qs, q3 = q.stride()
            pq = q.data_ptr()
            assert q_batch == B and q_rows == rows and q_dim == d and q3 == 1 and q.dtype is dtype and q.get_device() == index
            if q_out is q:
                qos, pqo = qs, pq
            else:
                *qos, q3 = q_out.stride()
                pqo = q_out.data_ptr()
                assert q_out.shape == q_shape and q3 == 1 and q_out.dtype is dtype and q_out.get_device() == index
        if v is not None:
            *vs, v3 = v.stride()
            pv = v.data_ptr()
            assert v.shape == shape and v3 == 1 and v.dtype is dtype and v.get_device() == index
        pk = k.data_ptr()
        if k_out is k:
            kos, pko = (k0, k1, k2), pk
        elif k_out is not None:
            *kos, k3 = k_out.stride()
            pko = k_out.data_ptr()
            assert k_out.shape == shape and k3 == 1 and k_out.dtype is dtype and k_out.get_device() == index
        return _TURNED_ROWS.pack(pq, pk, pv, pqo, pko, _HALF[dtype], rows, of_q, heads, d, *qs, k0, k1, k2, *vs, *qos, *kos)

    def tree_rotate(self, rotation, length, draft_tok, q, k, q_out=None, k_out=None):
        """Queries q [B, N, heads, d] and keys k [B, N, kv heads, d] of the drafted nodes normed and rotated by their positions; an
        output that is None is the input."""
        B, N, _, d = shape = k.shape
        dtype = k.dtype
        assert N == self.N and length.shape == (B,) and draft_tok.shape == (B, N) and rotation.fits(dtype, d, self._index)
        q_out, k_out = q if q_out is None else q_out, k if k_out is None else k_out
        desc = self._turned(dtype, shape, q, k, None, q_out, k_out)
        _check(self._lib.stand_tree_rotate(self.h, rotation.ref, self._arg(length, torch.int32), self._arg(draft_tok, torch.int32), desc,
                                           self._stream()), self.h)
        return q_out, k_out

    def cache_append(self, cache, layer, k, v, slots, start=None, count=None, rotation=None, q=None, q_out=None, k_out=None):
        """Rows k, v [B, rows, kv heads, d] into one layer of the cache: row j < count[b] (None: all) at position start[b] + j, to slot
        slots[b][j], its key normed and rotated; queries q [B, rows, heads, d] along with them into q_out (None: in place)."""
        B, rows, heads, d = shape = k.shape
        assert slots.dim() == 2
        of_slots, width = slots.shape
        assert of_slots == B and width >= rows and heads == cache.heads and d == cache.dim and self._index == cache.index
        assert (start is None or start.shape == (B,)) and (count is None or count.shape == (B,))
        assert rotation is None or rotation.fits(cache.dtype, d, self._index)
        q_out = q if q_out is None else q_out
        desc = self._turned(cache.dtype, shape, q, k, v, q_out, k_out)
        _check(self._lib.stand_cache_append(self.h, cache.ref, layer, None if rotation is None else rotation.ref, desc, self._arg(start, torch.int32),
                                            self._arg(slots, torch.int64), width, self._arg(count, torch.int32), self._stream()), self.h)
        return q_out

    def cache_read(self, cache, table, k, v, count=None, start=None, layer=0):
        """Tokens start[b] + j (None: j), j < count[b] (None: all rows), of the layers from `layer` on into rows k, v
        [layers, B, rows, kv heads, d]."""
        layers, B, rows, heads, d = k.shape
        stride = k.stride()
        assert k.shape == v.shape and stride == v.stride() and stride[4] == 1 and cache.dtype is k.dtype and cache.dtype is v.dtype
        assert B == self.B and heads == cache.heads and d == cache.dim and table.dim() == 2 and table.shape[0] == B
        assert (count is None or count.shape == (B,)) and (start is None or start.shape == (B,))
        assert self._index == cache.index == k.get_device() == v.get_device()
        desc = _CACHE_ROWS.pack(k.data_ptr(), v.data_ptr(), rows, *stride[:4])
        _check(self._lib.stand_cache_read(self.h, cache.ref, layer, layers, self._arg(table, torch.int32), table.shape[1], self._arg(start, torch.int32),
                                          self._arg(count, torch.int32), desc, self._stream()), self.h)
        return k, v

    def cache_pages(self, pages, add=None, room=None, slots=None, missing=None, out=None):
        """Moves lengths on by add, takes and gives back pages for room more tokens (None: a whole path); slots [B, any] and
        missing [B] are written.  out: Pages that receives the new state (None: in place)."""
        if missing is None:
            missing = torch.empty(self.B, dtype=torch.int32, device=self.device)
        out = pages if out is None else out
        assert pages.table.shape[0] == self.B and missing.shape == (self.B,) and (slots is None or (slots.dim() == 2 and slots.shape[0] == self.B))
        assert (add is None or add.shape == (self.B,)) and (room is None or room.shape == (self.B,))
        assert self._index == pages.index == out.index
        _check(self._lib.stand_cache_pages(self.h, pages.ref, self._arg(add, torch.int32), self._arg(room, torch.int32), self._arg(slots, torch.int64),
                                           0 if slots is None else slots.shape[1], self._arg(missing, torch.int32), out.ref, self._stream()), self.h)
        return missing

    def shape_logits(self, logits, out, draft_tok, count=None, penalty=None, bias_id=None, bias=None, allow=None):
        """Penalties [B, 3] (repetition, presence, frequency), biases [B, M] and a grammar's bits [B, N, (V + 31) // 32] (int32) on
        the logits of a drafted tree; out may be logits (None: it is)."""
        out = logits if out is None else out
        M = 0 if bias_id is None else bias_id.shape[1]
        assert draft_tok.shape == (self.B, self.N) and (count is None or count.shape == (self.B, self.V))
        assert penalty is None or penalty.shape == (self.B, 3)
        assert (bias_id is None) == (bias is None) and (bias is None or bias.shape == bias_id.shape == (self.B, M))
        assert allow is None or allow.shape == (self.B, self.N, (self.V + 31) // 32)
        assert self._index == logits.get_device() == out.get_device()
        work = None if allow is None else torch.empty(self.B * self.N, dtype=torch.uint8, device=self.device)
        _check(self._lib.stand_shape_logits(self.h, self._logits_ptr(logits), self._logits_ptr(out), self._arg(draft_tok, torch.int32),
                                            self._arg(count, torch.int32), self._arg(penalty, torch.float32), self._arg(bias_id, torch.int32),
                                            self._arg(bias, torch.float32), M, self._arg(allow, torch.int32),
                                            None if work is None else work.data_ptr(), self.B * self.N, self._stream()), self.h)
        return out

    def count_tokens(self, count, tok, length=None, prompt=False):
        """Tokens tok [B, any] (the first length[b] of them) into count [B, V]: generated ones, or the prompt's."""
        assert count.shape == (self.B, self.V) and tok.dim() == 2 and tok.shape[0] == self.B and (length is None or length.shape == (self.B,))
        _check(self._lib.stand_count_tokens(self.h, self._arg(count, torch.int32), self._arg(tok, torch.int32), self._arg(length, torch.int32),
                                            tok.shape[1], int(prompt), self._stream()), self.h)

    def record_slots(self, rows_per_trajectory, orders):
        """Slot of every merge record of the last update, [B, R, orders] (-1: no such record, or dropped)."""
        out = np.zeros(self.B * rows_per_trajectory * orders, np.int64)
        _check(lib().stand_get_record_slots(self.h, out.ctypes.data), self.h)
        return out.reshape(self.B, rows_per_trajectory, orders)

    def node_counts(self):
        out = np.zeros(self.N, np.uint64)
        _check(lib().stand_get_node_counts(self.h, out.ctypes.data), self.h)
        return out

    def reset_node_counts(self):
        _check(lib().stand_reset_node_counts(self.h), self.h)

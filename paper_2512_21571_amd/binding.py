"""ctypes binding of include/nnc.h.  Argument marshalling only: every step of the
forward pass runs in the library's HIP kernels.  PyTorch supplies device memory
(through the allocator hooks) and the stream; there is no CPU or PyTorch fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
import threading

import numpy as np

from . import _build

OK, E_ARG, E_CONFIG, E_BLOB, E_NOMEM, E_KV_FULL, E_DEVICE, E_STATE = range(8)
F32, BF16, F16 = 0, 1, 2
W8 = 3   # blob dtype only (weight-only 8 bits); computes in BF16
I8, E4M3 = 4, 5   # paged KV cache only
OPT_GRAPH, OPT_PREFILL_EXACT, OPT_PERSISTENT, OPT_STAGE_TRACE, OPT_PREFILL_TILE, OPT_SPIN_LIMIT = 0, 1, 2, 3, 4, 5
OPT_PREFILL_ATTN = 6
OPT_FUSE_QK = 7
OPT_TAIL_OVERLAP = 8
OPT_PREFILL_BLOCK = 9
OPT_PLANNER = 10
OPT_FUSE_NORM = 11
OPT_DECODE_PIECES = 12
OPT_PREFILL_KSLICES = 13
OPT_TAG_LIMIT = 14

# every symbol include/nnc.h declares
EXPORTS = [
    "nnc_model_create", "nnc_model_destroy", "nnc_prefill", "nnc_decode_step", "nnc_decode_step_static",
    "nnc_decode_greedy",
    "nnc_kv_reset", "nnc_synchronize", "nnc_slot_len", "nnc_prefill_hidden", "nnc_decode_step_hidden", "nnc_kv_read",
    "nnc_set_option", "nnc_profile_begin", "nnc_profile_end", "nnc_stage_trace", "nnc_blob_bytes",
    "nnc_last_error", "nnc_plan_prefill_gemm_query", "nnc_plan_skinny_gemm_query",
    "nnc_page_append", "nnc_page_read", "nnc_page_attention_workspace", "nnc_page_attention", "nnc_page_reorder",
    "nnc_beam_select_workspace", "nnc_beam_select", "nnc_pages_store", "nnc_decode_step_paged", "nnc_decode_beam",
    "nnc_page_attention_shared_workspace", "nnc_page_attention_shared", "nnc_page_attention_picked_workspace", "nnc_page_attention_picked",
    "nnc_page_bound", "nnc_page_pick_workspace", "nnc_page_pick", "nnc_draft_verify_workspace", "nnc_draft_verify", "nnc_decode_step_drafts",
]


class NncConfig(ctypes.Structure):
    _fields_ = [("struct_bytes", ctypes.c_uint32)] + [(n, ctypes.c_uint32) for n in (
        "hidden", "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "vocab")] + [
        ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float)] + [(n, ctypes.c_uint32) for n in (
            "has_embed_and_head", "tied_lm_head", "blob_dtype", "compute_dtype", "max_batch", "max_seq")]


ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p)
FREE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p)


class NncDevice(ctypes.Structure):
    _fields_ = [("alloc", ALLOC_FN), ("free", FREE_FN), ("ctx", ctypes.c_void_p), ("stream", ctypes.c_void_p)]


class NncKernelStat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("launches", ctypes.c_uint64), ("total_ms", ctypes.c_double),
                ("bytes", ctypes.c_double), ("flops", ctypes.c_double)]


class NncGemmPlan(ctypes.Structure):
    _fields_ = [("tile_rows", ctypes.c_uint32), ("tile_cols", ctypes.c_uint32), ("tile_code", ctypes.c_int32),
                ("k_slices", ctypes.c_uint32), ("workgroups", ctypes.c_uint32), ("t_comp_us", ctypes.c_double),
                ("t_mem_us", ctypes.c_double), ("t_us", ctypes.c_double), ("candidates", ctypes.c_uint32),
                ("rejected_by_capacity", ctypes.c_uint32)]


class NncPages(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint32) for n in ("struct_bytes", "dtype", "n_layers", "n_pages", "page_tokens", "n_kv_heads", "head_dim")] + [
        (n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]


class NncPageTable(ctypes.Structure):
    _fields_ = [("entries", ctypes.c_void_p), ("n_seqs", ctypes.c_uint32), ("max_pages", ctypes.c_uint32)]


class NncPageRows(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_uint32)] + [
        (n, ctypes.c_int64) for n in ("k_row_stride", "k_head_stride", "v_row_stride", "v_head_stride")] + [
        ("n", ctypes.c_uint32), ("seq", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("seq0", ctypes.c_int32), ("pos0", ctypes.c_int32)]


class NncPageQuery(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("out", ctypes.c_void_p), ("dtype", ctypes.c_uint32), ("n_q_heads", ctypes.c_uint32)] + [
        (n, ctypes.c_int64) for n in ("q_row_stride", "q_head_stride", "out_row_stride", "out_head_stride")] + [
        ("lens", ctypes.c_void_p), ("max_len", ctypes.c_uint32), ("window", ctypes.c_uint32), ("scale", ctypes.c_float)]


class NncPageShare(ctypes.Structure):
    _fields_ = [("width", ctypes.c_uint32), ("prefix", ctypes.c_void_p), ("max_own", ctypes.c_uint32)]


class NncPageBounds(ctypes.Structure):
    _fields_ = [("lo", ctypes.c_void_p), ("hi", ctypes.c_void_p)]


class NncPick(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("dtype", ctypes.c_uint32), ("n_q_heads", ctypes.c_uint32), ("q_row_stride", ctypes.c_int64),
                ("q_head_stride", ctypes.c_int64), ("lens", ctypes.c_void_p)] + [(n, ctypes.c_uint32) for n in ("max_len", "keep", "first", "last")] + [
        ("tables_out", ctypes.c_void_p), ("lens_out", ctypes.c_void_p)]


class NncDrafts(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("draft_logits", ctypes.c_void_p), ("dtype", ctypes.c_uint32), ("row_stride", ctypes.c_int64),
                ("draft_row_stride", ctypes.c_int64)] + [(n, ctypes.c_uint32) for n in ("n", "k", "vocab")] + [
        (n, ctypes.c_void_p) for n in ("drafts", "counts", "uniforms", "temperatures")] + [("temperature", ctypes.c_float)] + [
        (n, ctypes.c_void_p) for n in ("tokens_out", "accepted_out")]


class NncBeam(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("dtype", ctypes.c_uint32), ("row_stride", ctypes.c_int64), ("n_groups", ctypes.c_uint32),
                ("width", ctypes.c_uint32), ("vocab", ctypes.c_uint32), ("scores", ctypes.c_void_p), ("finished", ctypes.c_void_p),
                ("eos", ctypes.c_int32), ("tokens_out", ctypes.c_void_p), ("parents_out", ctypes.c_void_p),
                ("scores_out", ctypes.c_void_p), ("finished_out", ctypes.c_void_p)]


class NncBeamRun(ctypes.Structure):
    _fields_ = [("tables", ctypes.c_void_p), ("max_pages", ctypes.c_uint32), ("n_groups", ctypes.c_uint32), ("width", ctypes.c_uint32),
                ("lens", ctypes.c_void_p), ("max_len", ctypes.c_uint32), ("first_logits", ctypes.c_void_p), ("tokens", ctypes.c_void_p),
                ("eos", ctypes.c_int32), ("n_steps", ctypes.c_uint32), ("tokens_out", ctypes.c_void_p), ("parents_out", ctypes.c_void_p),
                ("scores", ctypes.c_void_p), ("finished", ctypes.c_void_p)]


class NncError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"nnc status {status}: {message}")
        self.status = status


_lib = None
_torch = None   # set with _lib: an import statement in a call that takes 8 us is one of 0.3


def lib():
    """Load libnnc.so (building it first only if no built library exists)."""
    global _lib, _torch
    if _lib is None:
        # PyTorch ships its own HIP runtime (soname libamdhip64.so.7).  Import it first so
        # that libnnc.so binds to that already-loaded runtime: two HIP runtimes in one
        # process cannot both own the device.
        import torch
        _torch = torch
        if not os.path.exists(_build.LIB_PATH):
            _build.build(True)
        L = ctypes.CDLL(_build.LIB_PATH)   # raises OSError if the library cannot be loaded
        vp, u32, i32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_int32
        P = ctypes.POINTER
        sig = {
            "nnc_model_create": (i32, [P(NncConfig), vp, ctypes.c_size_t, P(NncDevice), P(vp)]),
            "nnc_model_destroy": (None, [vp]),
            "nnc_prefill": (i32, [vp, u32, vp, u32, vp, vp]),
            "nnc_decode_step": (i32, [vp, vp, vp, u32, vp, vp]),
            "nnc_decode_step_static": (i32, [vp, vp, vp, u32, vp, vp]),
            "nnc_decode_greedy": (i32, [vp, vp, vp, u32, u32, vp, vp]),
            "nnc_kv_reset": (i32, [vp, i32]),
            "nnc_synchronize": (i32, [vp]),
            "nnc_slot_len": (i32, [vp, u32, P(u32)]),
            "nnc_prefill_hidden": (i32, [vp, u32, vp, u32, vp]),
            "nnc_decode_step_hidden": (i32, [vp, vp, vp, u32, vp]),
            "nnc_kv_read": (i32, [vp, u32, u32, u32, u32, u32, vp]),
            "nnc_set_option": (i32, [vp, i32, i32]),
            "nnc_profile_begin": (i32, [vp]),
            "nnc_profile_end": (i32, [vp, P(NncKernelStat), u32, P(u32)]),
            "nnc_stage_trace": (i32, [vp, vp, u32, P(u32), P(u32)]),
            "nnc_blob_bytes": (ctypes.c_uint64, [P(NncConfig)]),
            "nnc_last_error": (ctypes.c_char_p, []),
            "nnc_plan_prefill_gemm_query": (i32, [u32, u32, u32, u32, u32, u32, u32, P(NncGemmPlan)]),
            "nnc_plan_skinny_gemm_query": (i32, [u32, u32, u32, u32, u32, u32, u32, P(NncGemmPlan)]),
            "nnc_page_append": (i32, [P(NncPages), u32, P(NncPageTable), P(NncPageRows), vp]),
            "nnc_page_read": (i32, [P(NncPages), u32, P(NncPageTable), P(NncPageRows), vp]),
            "nnc_page_attention_workspace": (i32, [P(NncPages), P(NncPageTable), P(NncPageQuery), P(ctypes.c_size_t)]),
            "nnc_page_attention": (i32, [P(NncPages), u32, P(NncPageTable), P(NncPageQuery), vp, ctypes.c_size_t, vp]),
            "nnc_page_attention_shared_workspace": (i32, [P(NncPages), P(NncPageTable), P(NncPageQuery), P(NncPageShare), P(ctypes.c_size_t)]),
            "nnc_page_attention_shared": (i32, [P(NncPages), u32, P(NncPageTable), P(NncPageQuery), P(NncPageShare), vp, ctypes.c_size_t, vp]),
            "nnc_page_attention_picked_workspace": (i32, [P(NncPages), P(NncPageTable), P(NncPageQuery), P(ctypes.c_size_t)]),
            "nnc_page_attention_picked": (i32, [P(NncPages), u32, P(NncPageTable), P(NncPageQuery), vp, ctypes.c_size_t, vp]),
            "nnc_page_bound": (i32, [P(NncPages), u32, P(NncPageBounds), P(NncPageTable), vp, vp, i32, u32, vp]),
            "nnc_page_pick_workspace": (i32, [P(NncPages), P(NncPageTable), P(NncPick), P(ctypes.c_size_t)]),
            "nnc_page_pick": (i32, [P(NncPages), u32, P(NncPageBounds), P(NncPageTable), P(NncPick), vp, ctypes.c_size_t, vp]),
            "nnc_draft_verify_workspace": (i32, [P(NncDrafts), P(ctypes.c_size_t)]),
            "nnc_draft_verify": (i32, [P(NncDrafts), vp, ctypes.c_size_t, vp]),
            "nnc_decode_step_drafts": (i32, [vp, P(NncPages), P(NncPageTable), vp, u32, u32, vp, vp, vp, vp]),
            "nnc_page_reorder": (i32, [P(NncPages), P(NncPageTable), vp, vp, vp, u32, vp]),
            "nnc_beam_select_workspace": (i32, [P(NncBeam), P(ctypes.c_size_t)]),
            "nnc_beam_select": (i32, [P(NncBeam), vp, ctypes.c_size_t, vp]),
            "nnc_pages_store": (i32, [vp, P(NncPages), P(NncPageTable), u32, u32, u32, u32]),
            "nnc_decode_step_paged": (i32, [vp, P(NncPages), P(NncPageTable), vp, u32, vp, vp, vp]),
            "nnc_decode_beam": (i32, [vp, P(NncPages), P(NncBeamRun)]),
        }
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def last_error() -> str:
    return lib().nnc_last_error().decode()


def _check(st: int):
    if st != OK:
        raise NncError(st, last_error())


def make_config(shape, max_batch: int, max_seq: int, compute_dtype: int | None = None) -> NncConfig:
    """shape: any object with the field names of nnc_config (hidden, n_layers, ...) and `dtype`."""
    return NncConfig(ctypes.sizeof(NncConfig), shape.hidden, shape.n_layers, shape.n_q_heads,
                     shape.n_kv_heads, shape.head_dim, shape.ffn, shape.vocab, shape.rms_eps,
                     shape.rope_theta, int(shape.has_embed_and_head), int(shape.tied_lm_head),
                     shape.dtype, (BF16 if shape.dtype == W8 else shape.dtype) if compute_dtype is None else compute_dtype,
                     max_batch, max_seq)


def blob_bytes(cfg: NncConfig) -> int:
    return int(lib().nnc_blob_bytes(ctypes.byref(cfg)))


def plan_prefill_gemm(rows, k, n_tokens, pieces, epilogue, max_k_slices=1, n_cus=256) -> NncGemmPlan:
    out = NncGemmPlan()
    _check(lib().nnc_plan_prefill_gemm_query(rows, k, n_tokens, pieces, epilogue, max_k_slices, n_cus, ctypes.byref(out)))
    return out


def plan_skinny_gemm(rows, k, n_seq, pieces, epilogue, max_k_slices=1, n_cus=256) -> NncGemmPlan:
    out = NncGemmPlan()
    _check(lib().nnc_plan_skinny_gemm_query(rows, k, n_seq, pieces, epilogue, max_k_slices, n_cus, ctypes.byref(out)))
    return out


def _i32(a):
    return np.ascontiguousarray(a, dtype=np.int32)


def _u32(a):
    return np.ascontiguousarray(a, dtype=np.uint32)


# ---- paged KV cache and beam selection -------------------------------------------------------

def _bad(message: str):
    raise NncError(E_ARG, message)


_ROW_TYPES: dict = {}


def _count(least, **numbers):
    """Whole numbers least .. 2^31 - 1.  (ctypes would drop the upper bits of others: 2^32 + 5 would become 5.)"""
    for name, n in numbers.items():
        if not least <= n <= 0x7fffffff:
            _bad(f"{name} {n}: {least} .. 2^31 - 1 expected")


def _dtype_of(t):
    if not _ROW_TYPES:
        _ROW_TYPES.update({_torch.float32: F32, _torch.bfloat16: BF16, _torch.float16: F16})
    code = _ROW_TYPES.get(t.dtype)
    return _bad(f"{t.dtype} is not one of float32, bfloat16, float16") if code is None else code


def _on(device, dtype, shape, **tensors):
    """Tensors of one device, type and shape, contiguous (None is skipped)."""
    for name, t in tensors.items():
        if t is not None and (t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous()):
            _bad(f"{name}: contiguous {dtype} {list(shape)} on {device} expected, not {t.dtype} {list(t.shape)} on {t.device}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _enqueue(device, f, *args):
    """f(*args, stream) on the caller's current stream of a device, which is made current for the call if it is not.  (Device and
    stream as torch's own launchers get them: a device guard and a Stream object cost 3.4 us.)"""
    i, c = device.index, _torch._C
    if c._cuda_getDevice() == i:
        st = f(*args, c._cuda_getCurrentRawStream(i))
    else:
        with _torch.cuda.device(i):
            st = f(*args, c._cuda_getCurrentRawStream(i))
    if st != OK:
        raise NncError(st, last_error())


class Pages:
    """A paged KV cache: the tensors of a pool and the operators on it.

    k, v: [layers, pages, kv heads, positions of a page, head_dim] of float32, bfloat16, float16, int8 or float8_e4m3fn;
    k_scale, v_scale: float32 [layers, pages, kv heads, positions of a page] for the last two.  The tensors are kept, not
    copied.  A table is an int32 tensor [sequences, pages of a sequence].  Calls run on the caller's current stream of the
    pool's device; outputs and workspaces are allocated for that stream."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        lib()
        self.torch = torch = _torch
        code = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16, torch.int8: I8, torch.float8_e4m3fn: E4M3}.get(k.dtype)
        if code is None or k.dim() != 5:
            _bad(f"k: a pool of five dimensions in float32, bfloat16, float16, int8 or float8_e4m3fn expected, not {k.dtype} {list(k.shape)}")
        if k.device.type != "cuda":
            _bad("k: device memory expected")
        _on(k.device, k.dtype, k.shape, k=k, v=v)
        _on(k.device, torch.float32, k.shape[:-1], k_scale=k_scale, v_scale=v_scale)
        if (code in (I8, E4M3)) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
            _bad("k_scale and v_scale go with int8 and float8_e4m3fn, and only with those")
        self.k, self.v, self.k_scale, self.v_scale, self.dtype, self.device = k, v, k_scale, v_scale, code, k.device
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_tokens, self.head_dim = k.shape
        self.desc = NncPages(ctypes.sizeof(NncPages), code, self.n_layers, self.n_pages, self.page_tokens, self.n_kv_heads, self.head_dim,
                             k.data_ptr(), v.data_ptr(), _ptr(k_scale), _ptr(v_scale))
        self._desc, self._i32 = ctypes.byref(self.desc), torch.int32

    @classmethod
    def empty(cls, n_layers: int, n_pages: int, page_tokens: int, n_kv_heads: int, head_dim: int, dtype, device: str = "cuda:0"):
        """A pool of its own memory; dtype: a torch type of those above."""
        import torch
        shape = (n_layers, n_pages, n_kv_heads, page_tokens, head_dim)
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        scales = [torch.empty(shape[:-1], dtype=torch.float32, device=device) if dtype in (torch.int8, torch.float8_e4m3fn) else None for _ in range(2)]
        return cls(k, v, *scales)

    def _table(self, tables, name="tables"):
        if tables.dtype != self._i32 or tables.dim() != 2 or tables.device != self.device or not tables.is_contiguous():
            _bad(f"{name}: contiguous int32 [sequences, pages] on {self.device} expected, not {tables.dtype} {list(tables.shape)} on {tables.device}")
        n, m = tables.shape
        return NncPageTable(tables.data_ptr() or None, n, m)

    def _tables_of_heads(self, tables):
        if (tables.dtype != self._i32 or tables.dim() != 3 or tables.shape[1] != self.n_kv_heads or tables.device != self.device
                or not tables.is_contiguous()):
            _bad(f"tables: contiguous int32 [sequences, {self.n_kv_heads}, pages] on {self.device} expected, not {tables.dtype} {list(tables.shape)} on {tables.device}")
        n, heads, m = tables.shape
        return NncPageTable(tables.data_ptr() or None, n * heads, m)

    def _index(self, x, n, name):
        """seq or pos of n rows: (pointer, 0) of a tensor, (None, value) of a number."""
        if not isinstance(x, self.torch.Tensor):
            if not -0x80000000 <= x <= 0x7fffffff or int(x) != x:   # (ctypes would drop the upper bits, int what is behind the point)
                _bad(f"{name}: {x} is no whole number of 32 bits")
            return None, int(x)
        if x.dtype != self._i32 or x.shape != (n,) or x.device != self.device or not x.is_contiguous():
            _bad(f"{name}: contiguous int32 [{n}] on {self.device} expected, not {x.dtype} {list(x.shape)} on {x.device}")
        return x.data_ptr(), 0

    def _heads(self, x, n, what):
        """(row stride, head stride) of a tensor [n, heads, head_dim] whose elements of a head lie next to each other."""
        if x.dim() != 3 or x.shape[0] != n or x.shape[2] != self.head_dim or x.device != self.device:
            _bad(f"{what}: [{n}, heads, {self.head_dim}] on {self.device} expected, not {list(x.shape)} on {x.device}")
        row, head, one = x.stride()
        if one != 1 and n:
            _bad(f"{what}: the elements of a head must lie next to each other")
        return row, head

    def _rows(self, k, v, seq, pos):
        some = v if k is None else k
        if some is None:
            _bad("rows: k and v are both None")
        shape = some.shape
        n = shape[0] if len(shape) == 3 else 0
        if len(shape) != 3 or shape[1] != self.n_kv_heads:
            _bad(f"rows: [rows, {self.n_kv_heads}, {self.head_dim}] expected, not {list(shape)}")
        row, head = self._heads(some, n, "rows")
        v_row, v_head = row, head
        if v is not None and v is not some:
            if v.shape != shape or v.dtype != some.dtype:
                _bad(f"rows: k and v of one type and shape expected, not {k.dtype} {list(shape)} and {v.dtype} {list(v.shape)}")
            v_row, v_head = self._heads(v, n, "rows")
        sp, s0 = self._index(seq, n, "seq")
        pp, p0 = self._index(pos, n, "pos")
        return NncPageRows(_ptr(k), _ptr(v), _dtype_of(some), row, head, v_row, v_head, n, sp, pp, s0, p0)

    def append(self, layer: int, k, v, tables, seq, pos):
        """Write rows [n, kv heads, head_dim] (any strides between rows and heads) as positions `pos` of sequences `seq`: int32
        tensors [n], or one number: the sequence of all rows, the position of the first.  Negative positions are padding."""
        if k is None or v is None:
            _bad("rows: k or v is None")
        rows, table = self._rows(k, v, seq, pos), self._table(tables)
        _enqueue(self.device, lib().nnc_page_append, self._desc, self._layer(layer), ctypes.byref(table), ctypes.byref(rows))

    def read(self, layer: int, tables, seq, pos, dtype=None, n: int | None = None, k=None, v=None):
        """Rows (k, v) [n, kv heads, head_dim] of the named positions, in `dtype` (float32).  n: with two numbers for seq and
        pos, how many.  k, v: tensors to write into instead of new ones (one of them: only that is read)."""
        if k is None and v is None:
            if n is None:
                n = next((x.shape[0] for x in (seq, pos) if isinstance(x, self.torch.Tensor)), None)
                if n is None:
                    _bad("read: n is missing")
            k = self.torch.empty((n, self.n_kv_heads, self.head_dim), dtype=dtype or self.torch.float32, device=self.device)
            v = self.torch.empty_like(k)
        rows, table = self._rows(k, v, seq, pos), self._table(tables)
        _enqueue(self.device, lib().nnc_page_read, self._desc, self._layer(layer), ctypes.byref(table), ctypes.byref(rows))
        return k, v

    def _layer(self, layer):
        if not 0 <= layer < self.n_layers:
            _bad(f"layer {layer} of {self.n_layers}")
        return layer

    def _workspace(self, workspace, size, *args):
        """(tensor to keep, pointer, bytes) of a call's workspace: what the caller passes, or a new one of size(*args) bytes."""
        if workspace is None:
            n = ctypes.c_size_t()
            _check(size(*args, ctypes.byref(n)))
            t = self.torch.empty(n.value, dtype=self.torch.uint8, device=self.device) if n.value else None
            return t, _ptr(t), n.value
        if workspace.device != self.device or not workspace.is_contiguous():
            _bad("workspace: contiguous memory of the pool's device expected")
        return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()

    def _query(self, q, n, lens, max_len, scale, window, out, heads=False):
        if not (0 <= max_len <= 0x7fffffff and 0 <= window <= 0x7fffffff):
            _bad(f"max_len {max_len}, window {window}: 0 .. 2^31 - 1 expected")
        row, head = self._heads(q, n, "q")
        o_row = o_head = 0
        if out is not None:
            o_row, o_head = self._heads(out, n, "out")
            if out.shape != q.shape or out.dtype != q.dtype:
                _bad("out: type and shape of q expected")
        of = (n, self.n_kv_heads) if heads else (n,)
        if lens.dtype != self._i32 or lens.shape != of or lens.device != self.device or not lens.is_contiguous():
            _bad(f"lens: contiguous int32 {list(of)} on {self.device} expected, not {lens.dtype} {list(lens.shape)} on {lens.device}")
        return NncPageQuery(q.data_ptr(), _ptr(out), _dtype_of(q), q.shape[1], row, head, o_row, o_head, lens.data_ptr(), max_len, window,
                            self.head_dim ** -0.5 if scale is None else scale)

    def _attention_bytes(self, table, query):
        n = ctypes.c_size_t()
        _check(lib().nnc_page_attention_workspace(self._desc, ctypes.byref(table), ctypes.byref(query), ctypes.byref(n)))
        return n.value

    def attention_workspace(self, q, tables, lens, max_len: int = 0, window: int = 0) -> int:
        """Bytes of workspace of the same call of `attention`."""
        heads = tables.dim() == 3
        table = self._tables_of_heads(tables) if heads else self._table(tables)
        query = self._query(q, q.shape[0] if heads else table.n_seqs, lens, max_len, None, window, None, heads)
        if heads:
            n = ctypes.c_size_t()
            _check(lib().nnc_page_attention_picked_workspace(self._desc, ctypes.byref(table), ctypes.byref(query), ctypes.byref(n)))
            return n.value
        return self._attention_bytes(table, query)

    def attention(self, layer: int, q, tables, lens, max_len: int = 0, scale: float | None = None, window: int = 0, out=None, workspace=None):
        """One query row per sequence, q [sequences, query heads, head_dim], against the first lens[i] (int32) cached positions
        of each; max_len: an upper bound of lens (0: what the table holds); scale: 1 / sqrt(head_dim) unless given; window: only
        that many last positions (0: all).  tables [sequences, kv heads, pages] with lens [sequences, kv heads], as `pick` leaves
        them: every kv head has its own (then without a window).  workspace: a tensor of attention_workspace bytes instead of a new one."""
        if out is None:
            out = self.torch.empty_like(q, memory_format=self.torch.contiguous_format)
        if tables.dim() == 3:
            return self._attention_picked(layer, q, tables, lens, max_len, scale, window, out, workspace)
        table = self._table(tables)
        query = self._query(q, table.n_seqs, lens, max_len, scale, window, out)
        if workspace is None:
            size = self._attention_bytes(table, query)
            workspace = self.torch.empty(size, dtype=self.torch.uint8, device=self.device) if size else None
        elif workspace.device != self.device or not workspace.is_contiguous():
            _bad("workspace: contiguous memory of the pool's device expected")
        else:
            size = workspace.numel() * workspace.element_size()
        _enqueue(self.device, lib().nnc_page_attention, self._desc, self._layer(layer), ctypes.byref(table), ctypes.byref(query), _ptr(workspace), size)
        return out

    def _attention_picked(self, layer, q, tables, lens, max_len, scale, window, out, workspace):
        L, table = lib(), self._tables_of_heads(tables)
        query = self._query(q, tables.shape[0], lens, max_len, scale, window, out, True)
        kept, at, size = self._workspace(workspace, L.nnc_page_attention_picked_workspace, self._desc, ctypes.byref(table), ctypes.byref(query))
        _enqueue(self.device, L.nnc_page_attention_picked, self._desc, self._layer(layer), ctypes.byref(table), ctypes.byref(query), at, size)
        return out

    def _share(self, q, tables, lens, prefix, max_len, max_own, scale, out):
        """(table, query, share) of a call of attention_shared."""
        if q.dim() != 4 or lens.shape != q.shape[:2] or q.shape[3] != self.head_dim:
            _bad(f"q [groups, width, heads, {self.head_dim}] and lens [groups, width] expected, not {list(q.shape)} and {list(lens.shape)}")
        shape, i32, device = q.shape, self._i32, self.device
        groups, width, heads, _ = shape
        n = groups * width
        row, head = self._apart(q, "q")
        o_row = o_head = 0
        if out is not None:
            if out.shape != shape or out.dtype != q.dtype:
                _bad("out: type and shape of q expected")
            o_row, o_head = self._apart(out, "out")
        if not 0 <= max_len <= 0x7fffffff or not (max_own is None or 0 <= max_own <= 0x7fffffff):
            _bad(f"max_len {max_len}, max_own {max_own}: 0 .. 2^31 - 1 expected")
        *of, pages = tables.shape
        if math.prod(of) != (groups if prefix is None else n) or not 1 <= len(of) <= (1 if prefix is None else 2):
            _bad(f"tables: a row for each of {groups} groups expected, not {list(tables.shape)}" if prefix is None else
                 f"tables: a row for each of {groups} x {width} sequences expected, not {list(tables.shape)}")
        if tables.dtype != i32 or tables.device != device or not tables.is_contiguous():
            _bad(f"tables: contiguous int32 on {device} expected, not {tables.dtype} {list(tables.shape)} on {tables.device}")
        if prefix is not None and (prefix.dtype != i32 or prefix.shape != (groups,) or prefix.device != device or not prefix.is_contiguous()):
            _bad(f"prefix: contiguous int32 [{groups}] on {device} expected, not {prefix.dtype} {list(prefix.shape)} on {prefix.device}")
        if lens.dtype != i32 or lens.device != device or not lens.is_contiguous():
            _bad(f"lens: contiguous int32 [{groups}, {width}] on {device} expected, not {lens.dtype} {list(lens.shape)} on {lens.device}")
        query = NncPageQuery(q.data_ptr(), _ptr(out), _dtype_of(q), heads, row, head, o_row, o_head, lens.data_ptr(), max_len, 0,
                             self.head_dim ** -0.5 if scale is None else scale)
        if max_own is None:
            max_own = max_len or pages * self.page_tokens
        return NncPageTable(tables.data_ptr() or None, math.prod(of), pages), query, NncPageShare(width, _ptr(prefix), max_own)

    def _apart(self, x, name):
        """(row stride, head stride) of a tensor [groups, width, heads, head_dim] whose rows are all one distance apart."""
        (groups, width, _, _), (between, row, head, one) = x.shape, x.stride()
        if width == 1:
            row = between   # (one row a group: no rows are `row` apart)
        if x.device != self.device or ((one != 1 or (groups > 1 and between != width * row)) and x.numel()):
            _bad(f"{name}: on {self.device}, the elements of a head next to each other and one distance between all rows expected")
        return row, head

    def attention_shared_workspace(self, q, tables, lens, prefix=None, max_len: int = 0, max_own: int | None = None) -> int:
        """Bytes of workspace of the same call of `attention_shared`."""
        if q.numel() == 0:
            return 0
        table, query, share = self._share(q, tables, lens, prefix, max_len, max_own, None, None)
        n = ctypes.c_size_t()
        _check(lib().nnc_page_attention_shared_workspace(self._desc, ctypes.byref(table), ctypes.byref(query), ctypes.byref(share), ctypes.byref(n)))
        return n.value

    def attention_shared(self, layer: int, q, tables, lens, prefix=None, max_len: int = 0, max_own: int | None = None, scale: float | None = None,
                         out=None, workspace=None):
        """Query rows q [groups, width, query heads, head_dim] against the first lens[g, w] (int32) cached positions of each, what the
        rows of a group share being read once for all of them.  With prefix (int32 [groups]): a batch behind one prompt, or beams;
        tables [groups, width, pages] or [groups * width, pages], the positions below prefix[g] are read through the group's first row.  Without:
        new tokens of one sequence, tables [groups, pages].  max_len: an upper bound of lens (0: what the table holds); max_own: one of
        what a row has behind its prefix (None: max_len's; 0: nothing).  workspace: a tensor of attention_shared_workspace bytes instead of a new one."""
        L = lib()
        if out is None:
            out = self.torch.empty_like(q, memory_format=self.torch.contiguous_format)
        table, query, share = self._share(q, tables, lens, prefix, max_len, max_own, scale, out)
        layer = self._layer(layer)
        if not (table.n_seqs and share.width):
            return out
        kept, at, size = self._workspace(workspace, L.nnc_page_attention_shared_workspace, self._desc, ctypes.byref(table), ctypes.byref(query), ctypes.byref(share))
        _enqueue(self.device, L.nnc_page_attention_shared, self._desc, layer, ctypes.byref(table), ctypes.byref(query), ctypes.byref(share), at, size)
        return out

    def empty_bounds(self):
        """Two tensors (lo, hi) for the bounds of all pages: [layers, pages, kv heads, head_dim] of the pool's type, bfloat16 for 8 bits."""
        dtype = self.torch.bfloat16 if self.dtype in (I8, E4M3) else self.k.dtype
        return tuple(self.torch.empty((self.n_layers, self.n_pages, self.n_kv_heads, self.head_dim), dtype=dtype, device=self.device) for _ in range(2))

    def _bounds(self, bounds):
        lo, hi = bounds
        dtype = self.torch.bfloat16 if self.dtype in (I8, E4M3) else self.k.dtype
        _on(self.device, dtype, (self.n_layers, self.n_pages, self.n_kv_heads, self.head_dim), lo=lo, hi=hi)
        return NncPageBounds(lo.data_ptr(), hi.data_ptr())

    def bound(self, layer: int, bounds, tables, lens, since=0, max_new: int = 0):
        """Bring the bounds (lo, hi) of the pages up to date that hold positions since[i] .. lens[i] - 1 of every sequence: the smallest and
        the largest key of each, dimension by dimension.  since: an int32 tensor [sequences] or one number; max_new: no sequence has more
        such positions (0: what the table holds)."""
        table = self._table(tables)
        _count(0, max_new=max_new)
        at, first = self._index(since, table.n_seqs, "since")
        _on(self.device, self._i32, (table.n_seqs,), lens=lens)
        b = self._bounds(bounds)
        _enqueue(self.device, lib().nnc_page_bound, self._desc, self._layer(layer), ctypes.byref(b), ctypes.byref(table), lens.data_ptr(), at, first, max_new)

    def pick(self, layer: int, bounds, q, tables, lens, keep: int, first: int = 1, last: int = 1, max_len: int = 0, workspace=None):
        """The `keep` pages of every sequence and kv head that the query rows q [sequences, query heads, head_dim] may score highest on, by
        the bounds (lo, hi) of their keys; the first and last ones of a sequence in any case.  Returns tables [sequences, kv heads, keep] and lens
        [sequences, kv heads], int32, as `attention` takes them.  max_len: an upper bound of lens (0: what the table holds)."""
        L, table = lib(), self._table(tables)
        _count(0, max_len=max_len, first=first)
        _count(1, keep=keep, last=last)
        row, head = self._heads(q, table.n_seqs, "q")
        _on(self.device, self._i32, (table.n_seqs,), lens=lens)
        b = self._bounds(bounds)
        picked = self.torch.empty((table.n_seqs, self.n_kv_heads, keep), dtype=self._i32, device=self.device)
        seen = self.torch.empty((table.n_seqs, self.n_kv_heads), dtype=self._i32, device=self.device)
        pick = NncPick(q.data_ptr(), _dtype_of(q), q.shape[1], row, head, lens.data_ptr(), max_len, keep, first, last, picked.data_ptr(), seen.data_ptr())
        layer = self._layer(layer)
        kept, at, size = self._workspace(workspace, L.nnc_page_pick_workspace, self._desc, ctypes.byref(table), ctypes.byref(pick))
        _enqueue(self.device, L.nnc_page_pick, self._desc, layer, ctypes.byref(b), ctypes.byref(table), ctypes.byref(pick), at, size)
        return picked, seen

    def reorder(self, before, after, lens, parents):
        """Beams take over the cache of their parents: tables before and after [groups * width, pages] (may be one tensor), lens
        [groups * width], parents [groups, width], all int32."""
        if parents.dim() != 2:
            _bad("parents: [groups, width] expected")
        table = self._table(before, "before")
        _on(self.device, self._i32, before.shape, after=after)
        _on(self.device, self._i32, (table.n_seqs,), lens=lens)
        _on(self.device, self._i32, parents.shape, parents=parents)
        if parents.numel() != table.n_seqs:
            _bad(f"parents: {table.n_seqs} beams expected, not {list(parents.shape)}")
        _enqueue(self.device, lib().nnc_page_reorder, self._desc, ctypes.byref(table), after.data_ptr(), lens.data_ptr(), parents.data_ptr(),
                 parents.shape[1])


def beam_select(logits, scores, finished=None, eos: int = -1, workspace=None):
    """The best continuations of every group of beams (nnc_beam_select): logits [groups, width, vocab] (float32, bfloat16,
    float16), scores [groups, width] float32, finished [groups, width] bool or None, eos: the token that ends a beam (-1: none).
    Returns tokens, parents (int32), scores, finished, each [groups, width], best first."""
    L, torch = lib(), _torch
    if logits.dim() != 3 or logits.device.type != "cuda":
        _bad("logits: [groups, width, vocab] in device memory expected")
    (g, w, v), (between, row, one), device = logits.shape, logits.stride(), logits.device
    if w == 1:
        row = between   # (one beam a group: no rows are `row` apart)
    if g and w and ((one != 1 and v > 1) or (g > 1 and between != w * row)):
        _bad("logits: rows of adjacent elements, one distance between all rows, expected")
    if finished is not None and finished.dtype != torch.bool:
        _bad("finished: bool expected")
    if not -1 <= eos < v:
        _bad(f"eos: {eos} is no token of {v}, nor -1")
    _on(device, torch.float32, (g, w), scores=scores)
    _on(device, torch.bool, (g, w), finished=finished)
    tokens = torch.empty((g, w), dtype=torch.int32, device=device)
    parents, out, ended = torch.empty_like(tokens), torch.empty_like(scores), torch.empty_like(scores, dtype=torch.bool)
    beam = NncBeam(logits.data_ptr(), _dtype_of(logits), row, g, w, v, scores.data_ptr(), _ptr(finished), eos, tokens.data_ptr(),
                   parents.data_ptr(), out.data_ptr(), ended.data_ptr())
    if workspace is None:
        n = ctypes.c_size_t()
        _check(L.nnc_beam_select_workspace(ctypes.byref(beam), ctypes.byref(n)))
        size = n.value
        workspace = torch.empty(size, dtype=torch.uint8, device=device)
    elif workspace.device != device or not workspace.is_contiguous():
        _bad("workspace: contiguous memory of the logits' device expected")
    else:
        size = workspace.numel() * workspace.element_size()
    _enqueue(device, L.nnc_beam_select, ctypes.byref(beam), workspace.data_ptr(), size)
    return tokens, parents, out, ended


def _rows_apart(x, rows, name):
    """Elements between the rows of a tensor [n, rows, vocab] whose rows are adjacent elements, all one distance apart."""
    between, row, one = x.stride()
    if x.shape[1] == 1:
        row = between
    if x.numel() and ((one != 1 and x.shape[2] > 1) or (x.shape[0] > 1 and between != rows * row)):
        _bad(f"{name}: rows of adjacent elements, one distance between all rows, expected")
    return row


def draft_verify(logits, drafts, uniforms, draft_logits=None, counts=None, temperature=1.0, workspace=None):
    """Which drafted tokens are kept and the token behind them (nnc_draft_verify): logits [n, k + 1, vocab] of the target (float32,
    bfloat16, float16), drafts int32 [n, k], uniforms float32 [n, k + 1] of [0, 1), draft_logits [n, k, vocab] of the logits' type or None (drafts
    that were not drawn), counts int32 [n] (0 .. k drafts each) or None, temperature: a number or float32 [n]; 0: greedy.  A token is forbidden by -infinity
    (a finite mask leaves it next to nothing, which a random number of exactly 0 may pick).
    Returns tokens int32 [n, k + 1] (the kept drafts, one token more, then -1) and how many were kept, int32 [n]."""
    L, torch = lib(), _torch
    if logits.dim() != 3 or logits.device.type != "cuda":
        _bad("logits: [n, k + 1, vocab] in device memory expected")
    (n, rows, v), device = logits.shape, logits.device
    if rows < 1:
        _bad("logits: a row for every draft and one behind them expected")
    row = _rows_apart(logits, rows, "logits")
    draft_row = 0
    if draft_logits is not None:
        if draft_logits.dtype != logits.dtype or draft_logits.shape != (n, rows - 1, v) or draft_logits.device != device:
            _bad(f"draft_logits: {logits.dtype} {[n, rows - 1, v]} on {device} expected, not {draft_logits.dtype} {list(draft_logits.shape)} on {draft_logits.device}")
        draft_row = _rows_apart(draft_logits, rows - 1, "draft_logits")
    _on(device, torch.int32, (n, rows - 1), drafts=drafts)
    _on(device, torch.int32, (n,), counts=counts)
    _on(device, torch.float32, (n, rows), uniforms=uniforms)
    heat = temperature if isinstance(temperature, torch.Tensor) else None
    _on(device, torch.float32, (n,), temperature=heat)
    tokens = torch.empty((n, rows), dtype=torch.int32, device=device)
    accepted = torch.empty((n,), dtype=torch.int32, device=device)
    d = NncDrafts(logits.data_ptr(), _ptr(draft_logits), _dtype_of(logits), row, draft_row, n, rows - 1, v, drafts.data_ptr(), _ptr(counts),
                  uniforms.data_ptr(), _ptr(heat), 1.0 if heat is not None else temperature, tokens.data_ptr(), accepted.data_ptr())
    if workspace is None:
        size = ctypes.c_size_t()
        _check(L.nnc_draft_verify_workspace(ctypes.byref(d), ctypes.byref(size)))
        size = size.value
        workspace = torch.empty(size, dtype=torch.uint8, device=device)
    elif workspace.device != device or not workspace.is_contiguous():
        _bad("workspace: contiguous memory of the logits' device expected")
    else:
        size = workspace.numel() * workspace.element_size()
    _enqueue(device, L.nnc_draft_verify, ctypes.byref(d), workspace.data_ptr(), size)
    return tokens, accepted


class Model:
    """A model on cuda:0.  Device memory comes from torch's allocator, work runs on a
    torch stream of default priority (`stream`), which waits for the caller's current stream; outputs are
    tensors of the caller's current stream, which waits for the model's before anything it runs later.
    Calls on one model, from whatever threads, must not overlap inside the library."""

    def __init__(self, shape, blob: np.ndarray, max_batch: int, max_seq: int,
                 compute_dtype: int | None = None, device: str = "cuda:0"):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("nnc needs an MI355X: torch.cuda.is_available() is False")
        self.torch = torch
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.stream = torch.cuda.Stream(device=self.device)
        self._local = threading.local()  # the hand-over of a thread's call: its stream and two events
        self.cfg = make_config(shape, max_batch, max_seq, compute_dtype)
        self._held = {}

        def _alloc(nbytes, _ctx):
            try:
                t = torch.empty(int(nbytes), dtype=torch.uint8, device=self.device)
            except Exception:
                return None
            self._held[t.data_ptr()] = t
            return t.data_ptr()

        def _free(p, _ctx):
            self._held.pop(p, None)

        self._alloc_cb, self._free_cb = ALLOC_FN(_alloc), FREE_FN(_free)
        self._dev = NncDevice(self._alloc_cb, self._free_cb, None, self.stream.cuda_stream)
        blob = np.ascontiguousarray(blob)
        h = ctypes.c_void_p()
        _check(lib().nnc_model_create(ctypes.byref(self.cfg), blob.ctypes.data, blob.nbytes,
                                      ctypes.byref(self._dev), ctypes.byref(h)))
        self.h = h
        self.V, self.H = self.cfg.vocab, self.cfg.hidden

    # -- lifetime -----------------------------------------------------------------
    def close(self):
        if getattr(self, "h", None):
            lib().nnc_model_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _empty(self, shape, dtype):
        # a tensor of the caller's current stream: the model's stream waits for that stream before it
        # writes (_before), and that stream waits for the model's before anything it runs later (_after)
        return self.torch.empty(shape, dtype=dtype, device=self.device)

    def synchronize(self):
        """Wait for the model's stream; raises NncError if a resident decode launch gave up."""
        _check(lib().nnc_synchronize(self.h))

    def _before(self):
        # inputs may have been produced on the caller's current stream (two events kept per thread for the
        # hand-over: recording one again does not disturb a wait that was already enqueued)
        here = self._local
        if not hasattr(here, "ev_in"):
            here.ev_in, here.ev_out = self.torch.cuda.Event(), self.torch.cuda.Event()
        here.caller = self.torch.cuda.current_stream(self.device)
        here.ev_in.record(here.caller)
        self.stream.wait_event(here.ev_in)

    def _after(self):
        # outputs are consumed on the caller's current stream
        here = self._local
        here.ev_out.record(self.stream)
        here.caller.wait_event(here.ev_out)

    # -- forward pass ---------------------------------------------------------------
    def prefill(self, slot: int, tokens, want_logits: bool = True):
        t = _i32(tokens)
        logits = self._empty((self.V,), self.torch.float32) if want_logits else None
        nxt = self._empty((1,), self.torch.int32)
        self._before()
        try:
            _check(lib().nnc_prefill(self.h, slot, t.ctypes.data, t.size,
                                     logits.data_ptr() if want_logits else None, nxt.data_ptr()))
        finally:
            self._after()
        return logits, nxt

    def decode_step(self, slots, tokens, want_logits: bool = True):
        s, t = _u32(slots), _i32(tokens)
        b = s.size
        logits = self._empty((b, self.V), self.torch.float32) if want_logits else None
        nxt = self._empty((b,), self.torch.int32)
        self._before()
        try:
            _check(lib().nnc_decode_step(self.h, s.ctypes.data, t.ctypes.data, b,
                                         logits.data_ptr() if want_logits else None, nxt.data_ptr()))
        finally:
            self._after()
        return logits, nxt

    def decode_step_static(self, slots, tokens, logits=None, nxt=None):
        """nnc_decode_step_static: the caller passes the output tensors (nothing is allocated,
        here or in the library); either may be None."""
        s, t = _u32(slots), _i32(tokens)
        self._before()
        try:
            _check(lib().nnc_decode_step_static(self.h, s.ctypes.data, t.ctypes.data, s.size,
                                                logits.data_ptr() if logits is not None else None,
                                                nxt.data_ptr() if nxt is not None else None))
        finally:
            self._after()
        return logits, nxt

    def decode_greedy(self, slots, first_tokens, n_steps: int, want_logits: bool = False):
        s, t = _u32(slots), _i32(first_tokens)
        b = s.size
        toks = self._empty((n_steps, b), self.torch.int32)
        logits = self._empty((n_steps, b, self.V), self.torch.float32) if want_logits else None
        self._before()
        try:
            _check(lib().nnc_decode_greedy(self.h, s.ctypes.data, t.ctypes.data, b, n_steps, toks.data_ptr(),
                                           logits.data_ptr() if want_logits else None))
        finally:
            self._after()
        return toks, logits

    def prefill_hidden(self, slot: int, x):
        """x: [n, hidden] float32 torch tensor on the device (or array-like, copied)."""
        x = self._as_dev(x)
        y = self._empty(tuple(x.shape), self.torch.float32)
        self._before()
        try:
            _check(lib().nnc_prefill_hidden(self.h, slot, x.data_ptr(), x.shape[0], y.data_ptr()))
        finally:
            self._after()
        return y

    def decode_step_hidden(self, slots, x):
        s = _u32(slots)
        x = self._as_dev(x)
        y = self._empty(tuple(x.shape), self.torch.float32)
        self._before()
        try:
            _check(lib().nnc_decode_step_hidden(self.h, s.ctypes.data, x.data_ptr(), s.size, y.data_ptr()))
        finally:
            self._after()
        return y

    def _as_dev(self, x):
        torch = self.torch
        if not isinstance(x, torch.Tensor):
            x = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
        # (a conversion runs on the caller's stream, which _before waits for)
        x = x.to(self.device, dtype=torch.float32, non_blocking=False).contiguous()
        if x.dim() == 1:
            x = x[None]
        return x

    # -- pages --------------------------------------------------------------------------
    def _paged(self, pages: Pages, tables):
        if pages.device != self.stream.device:
            _bad(f"pages on {pages.device}, the model is on {self.stream.device}")
        return pages._table(tables)

    def pages_store(self, pages: Pages, tables, seq: int, slot: int, pos0: int = 0, n: int | None = None):
        """Positions pos0 .. pos0 + n - 1 (to the slot's end) of a slot's cache to the same positions of a sequence in pages."""
        n = self.slot_len(slot) - pos0 if n is None else n
        table = self._paged(pages, tables)
        if min(seq, slot, pos0, n) < 0 or max(seq, slot, pos0, n) > 0x7fffffff:
            _bad(f"sequence {seq}, slot {slot}, positions {pos0} .. + {n}")
        self._before()
        try:
            _check(lib().nnc_pages_store(self.h, ctypes.byref(pages.desc), ctypes.byref(table), seq, slot, pos0, n))
        finally:
            self._after()

    def decode_step_paged(self, pages: Pages, tables, lens, tokens, max_len: int = 0, want_logits: bool = True):
        """nnc_decode_step_paged: lens and tokens are int32 tensors [sequences]; lens grow by one."""
        _count(0, max_len=max_len)
        table = self._paged(pages, tables)
        b = tables.shape[0]
        _on(pages.device, self.torch.int32, (b,), lens=lens, tokens=tokens)
        logits = self._empty((b, self.V), self.torch.float32) if want_logits else None
        nxt = self._empty((b,), self.torch.int32)
        self._before()
        try:
            _check(lib().nnc_decode_step_paged(self.h, ctypes.byref(pages.desc), ctypes.byref(table), lens.data_ptr(), max_len, tokens.data_ptr(),
                                               _ptr(logits), nxt.data_ptr()))
        finally:
            self._after()
        return logits, nxt

    def decode_step_drafts(self, pages: Pages, tables, lens, tokens, counts=None, max_len: int = 0, want_next: bool = False):
        """nnc_decode_step_drafts: tokens int32 [sequences, k + 1], the newest token of each and k drafts behind it, become positions
        lens[i] .. lens[i] + k (lens stay as they are); counts int32 [sequences]: drafts of each (None: k).  Returns logits
        [sequences, k + 1, vocab], as draft_verify takes them, and the greedy tokens [sequences, k + 1] or None."""
        _count(0, max_len=max_len)
        table = self._paged(pages, tables)
        b = tables.shape[0]
        if tokens.dim() != 2 or tokens.shape[0] != b or tokens.shape[1] < 1:
            _bad(f"tokens: int32 [{b}, drafts + 1] expected, not {list(tokens.shape)}")
        k = tokens.shape[1] - 1
        if b * (k + 1) > 21:
            _bad(f"{b} sequences of {k} + 1 tokens (21 in all at most)")
        _on(pages.device, self.torch.int32, (b,), lens=lens, counts=counts)
        _on(pages.device, self.torch.int32, tokens.shape, tokens=tokens)
        logits = self._empty((b, k + 1, self.V), self.torch.float32)
        nxt = self._empty((b, k + 1), self.torch.int32) if want_next else None
        self._before()
        try:
            _check(lib().nnc_decode_step_drafts(self.h, ctypes.byref(pages.desc), ctypes.byref(table), lens.data_ptr(), max_len, k, tokens.data_ptr(),
                                                _ptr(counts), logits.data_ptr(), _ptr(nxt)))
        finally:
            self._after()
        return logits, nxt

    def decode_beam(self, pages: Pages, tables, lens, n_steps: int, first_logits=None, tokens=None, scores=None, finished=None, width: int | None = None,
                    eos: int = -1, max_len: int = 0):
        """nnc_decode_beam.  Begin: first_logits [groups, vocab] and width.  Go on: tokens, scores, finished [groups, width] of the
        call before; beams that have ended stay so whatever eos is now.  Returns tokens and parents [n_steps, groups, width], scores and finished [groups, width]."""
        _count(0, max_len=max_len)
        _count(1, n_steps=n_steps)
        torch, beams = self.torch, tables.shape[0]
        table = self._paged(pages, tables)
        if not -1 <= eos < self.V:
            _bad(f"eos: {eos} is no token of {self.V}, nor -1")
        if first_logits is not None:
            groups = first_logits.shape[0]
            if width is None or groups * width != beams:
                _bad(f"{beams} sequences are not {groups} groups of {width} beams")
            _on(pages.device, torch.float32, (groups, self.V), first_logits=first_logits)
            scores, finished = self._empty((groups, width), torch.float32), self._empty((groups, width), torch.bool)
        else:
            if tokens is None or scores is None or finished is None or scores.dim() != 2 or scores.numel() != beams:
                _bad("first_logits, or tokens, scores and finished [groups, width] expected")
            groups, width = scores.shape
            _on(pages.device, torch.int32, scores.shape, tokens=tokens)
            _on(pages.device, torch.float32, scores.shape, scores=scores)
            _on(pages.device, torch.bool, scores.shape, finished=finished)
            scores, finished = scores.clone(), finished.clone()
        _on(pages.device, torch.int32, (beams,), lens=lens)
        out, parents = (self._empty((n_steps, groups, width), torch.int32) for _ in range(2))
        run = NncBeamRun(tables.data_ptr(), table.max_pages, groups, width, lens.data_ptr(), max_len, _ptr(first_logits), _ptr(tokens), eos, n_steps,
                         out.data_ptr(), parents.data_ptr(), scores.data_ptr(), finished.data_ptr())
        self._before()
        try:
            _check(lib().nnc_decode_beam(self.h, ctypes.byref(pages.desc), ctypes.byref(run)))
        finally:
            self._after()
        return out, parents, scores, finished

    # -- state ------------------------------------------------------------------------
    def kv_reset(self, slot: int = -1):
        _check(lib().nnc_kv_reset(self.h, slot))

    def slot_len(self, slot: int) -> int:
        n = ctypes.c_uint32()
        _check(lib().nnc_slot_len(self.h, slot, ctypes.byref(n)))
        return n.value

    def kv_read(self, layer: int, slot: int, which: int, pos0: int, n: int):
        dkv = self.cfg.n_kv_heads * self.cfg.head_dim
        out = self._empty((n, dkv), self.torch.float32)
        self._before()
        try:
            _check(lib().nnc_kv_read(self.h, layer, slot, which, pos0, n, out.data_ptr()))
        finally:
            self._after()
        return out

    def set_option(self, opt: int, value: int):
        _check(lib().nnc_set_option(self.h, opt, value))

    def stage_trace(self):
        """[workgroups, points] uint64 wall-clock ticks (10 ns) of the traced decode step."""
        cap = 1024 * (8 * self.cfg.n_layers + 3)
        buf = np.zeros(cap, dtype=np.uint64)
        nwg, npts = ctypes.c_uint32(), ctypes.c_uint32()
        _check(lib().nnc_stage_trace(self.h, buf.ctypes.data, cap, ctypes.byref(nwg), ctypes.byref(npts)))
        return buf[: nwg.value * npts.value].reshape(nwg.value, npts.value)

    # -- per-kernel event timing ---------------------------------------------------------
    def profile_begin(self):
        _check(lib().nnc_profile_begin(self.h))

    def profile_end(self):
        cap = 32
        arr = (NncKernelStat * cap)()
        n = ctypes.c_uint32()
        _check(lib().nnc_profile_end(self.h, arr, cap, ctypes.byref(n)))
        return [dict(name=arr[i].name.decode(), launches=int(arr[i].launches), total_ms=arr[i].total_ms,
                     bytes=arr[i].bytes, flops=arr[i].flops) for i in range(n.value)]

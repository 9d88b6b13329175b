"""Python binding of the ADSA HIP library: same names as include/adsa.h, marshalling only.

Every function takes torch tensors (device memory) or raw integers for pointers, packs the
host parameter struct and calls the C entry point.  No step of the decode path runs here.  The calls of a decode step
go through a small CPython module (csrc/native_binding.c), the others through ctypes.
The library must be built (paper_2506_18226_amd/build.py) -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import importlib.machinery
import importlib.util
import os
from typing import Optional

import numpy as np

from . import build as _build

F32, BF16 = 0, 1
SCORE_ATTN_MASS, SCORE_VCOS, SCORE_EXT_LARGEST, SCORE_EXT_SMALLEST, SCORE_VCOS_FUSED = 0, 1, 2, 3, 4
FLAG_NO_COMPACT, FLAG_NO_ACCUMULATE, FLAG_PLAN_APPEND, FLAG_APPEND, FLAG_ADVANCE, FLAG_NEW_F32, FLAG_SPLIT_P = 1, 2, 4, 8, 16, 32, 64
SEQ_CACHE_FULL, SEQ_BAD_STATE, SEQ_SEL_OVERFLOW = 1, 2, 4
MAX_CAP = 8192
EVICT_ROW_END, EVICT_WHEN_FULL, EVICT_REUSE_SLOT = 0, 1, 2
MAX_AXES = 3
PAIRINGS = {"halves": 0, "neighbours": 1}
MASK_CAUSAL, MASK_PREFIX = 0, 1

ERRORS = {0: "ADSA_OK", -1: "ADSA_ERR_NULL", -2: "ADSA_ERR_SHAPE", -3: "ADSA_ERR_DTYPE", -4: "ADSA_ERR_ALIGN",
          -5: "ADSA_ERR_CAPACITY", -6: "ADSA_ERR_WORKSPACE", -7: "ADSA_ERR_LAUNCH", -8: "ADSA_ERR_UNSUPPORTED",
          -9: "ADSA_ERR_STATIC_SCRATCH"}
ERR_WORKSPACE = -6
STATIC_SCRATCH_BYTES = 4 << 20

EXPORTS = ["adsa_workspace_bytes", "adsa_workspace_init", "adsa_select", "adsa_attend", "adsa_compact", "adsa_step",
           "adsa_step_static", "adsa_rotate", "adsa_append", "adsa_prefill", "adsa_prefill_workspace_bytes", "adsa_attend_shared",
           "adsa_shared_workspace_bytes",
           "adsa_profile_enable", "adsa_profile_read", "adsa_strerror", "adsa_version"]


class AdsaParams(C.Structure):
    """Mirror of `adsa_params` (host struct)."""
    _fields_ = [
        ("n_seq", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
        ("grid_h", C.c_int32), ("grid_w", C.c_int32),
        ("win_rows_back", C.c_int32), ("win_col_radius", C.c_int32),
        ("sel_groups", C.c_int32), ("dtype", C.c_int32), ("score_mode", C.c_int32),
        ("cap", C.c_int32), ("sel_cap", C.c_int32),
        ("kv_slot_stride", C.c_int64), ("kv_head_stride", C.c_int64),
        ("softmax_scale", C.c_float), ("win_recent_m", C.c_int32), ("evict_policy", C.c_int32),
        ("q_per_kv", C.c_int32),
    ]


class _HostStruct(C.Structure):
    """A host struct of device pointers: it keeps the tensors they belong to alive, and what their shapes say for the checks of the calls
    (nothing where a field was filled with a raw pointer)."""
    sizes = ()                     # (name, elements along the first axis); see _check_sizes
    width = None                   # elements along the second axis of what has one

    def _hold(self, *tensors, sizes=(), width=None):
        self.held, self.sizes, self.width = tensors, tuple((name, n) for name, n in sizes if n is not None), width
        return self


class AdsaRope(_HostStruct):
    """Mirror of `adsa_rope` (host struct)."""
    _fields_ = [("freq", C.c_void_p), ("n_axes", C.c_int32), ("pairing", C.c_int32), ("text", C.c_int32 * MAX_AXES),
                ("origin", C.c_int32 * MAX_AXES), ("row", C.c_int32 * MAX_AXES), ("col", C.c_int32 * MAX_AXES)]


class AdsaTokens(_HostStruct):
    """Mirror of `adsa_tokens` (host struct)."""
    _fields_ = [("n_tokens", C.c_int32), ("max_len", C.c_int32), ("begin", C.c_void_p), ("slot0", C.c_void_p), ("pos0", C.c_void_p),
                ("coords", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64), ("v_stride", C.c_int64)]


class AdsaMods(_HostStruct):
    """Mirror of `adsa_mods` (host struct)."""
    _fields_ = [("softcap", C.c_float), ("mask", C.c_int32), ("slopes", C.c_void_p), ("doc", C.c_void_p), ("doc_stride", C.c_int64)]


class AdsaShared(_HostStruct):
    """Mirror of `adsa_shared` (host struct)."""
    rows = None                    # (heads, head_dim, dtype) of the prompts' caches
    _fields_ = [("n_groups", C.c_int32), ("max_prompt", C.c_int32), ("max_members", C.c_int32), ("reserved", C.c_int32),
                ("prompts", C.c_void_p), ("members", C.c_void_p), ("kv_slot_stride", C.c_int64), ("kv_head_stride", C.c_int64)]


# Mirror of `adsa_seq` (device struct array), 96 bytes per entry.
SEQ_DTYPE = np.dtype([
    ("k", np.uint64), ("v", np.uint64), ("pos", np.uint64), ("score", np.uint64),
    ("n_res", np.int32), ("step", np.int32), ("grid_origin", np.int32), ("n_keep_prefix", np.int32),
    ("budget", np.int32), ("budget_num", np.int32), ("budget_den", np.int32), ("status", np.int32),
    ("compacted", np.int32), ("pending_slot", np.int32), ("hole", np.int32), ("reserved", np.int32),
    ("vcos_u", np.uint64), ("reserved2", np.int64),
])
assert SEQ_DTYPE.itemsize == 96


class AdsaError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {ERRORS.get(code, code)} ({strerror(code)})")


_lib = None


def library_path() -> str:
    return _build.LIB_PATH


def load_library() -> C.CDLL:
    """dlopen the built HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise FileNotFoundError(f"{path} is missing: run `python -m paper_2506_18226_amd.build` "
                                    "(or __graft_entry__.build()) first; there is no fallback path")
        # torch ships its own HIP runtime: bring it in first so that this library binds to the SAME
        # runtime instance that owns the tensors' memory and streams (two runtimes in one process
        # do not see each other's allocations)
        import torch  # noqa: F401
        lib = C.CDLL(path)
        vp, i32p, f32p = C.c_void_p, C.c_void_p, C.c_void_p
        pp = C.POINTER(AdsaParams)
        lib.adsa_workspace_bytes.restype = C.c_size_t
        lib.adsa_workspace_bytes.argtypes = [pp]
        lib.adsa_workspace_init.restype = C.c_int
        lib.adsa_workspace_init.argtypes = [pp, vp, C.c_size_t, vp]
        lib.adsa_select.restype = C.c_int
        lib.adsa_select.argtypes = [pp, vp, i32p, i32p, C.c_uint32, vp, C.c_size_t, vp]
        lib.adsa_attend.restype = C.c_int
        lib.adsa_attend.argtypes = [pp, vp, vp, vp, vp, i32p, i32p, vp, f32p, C.c_uint32, vp, C.c_size_t, vp]
        lib.adsa_compact.restype = C.c_int
        lib.adsa_compact.argtypes = [pp, vp, i32p, C.c_uint32, vp, C.c_size_t, vp]
        lib.adsa_step.restype = C.c_int
        lib.adsa_step.argtypes = [pp, vp, vp, vp, vp, vp, f32p, i32p, i32p, i32p, C.c_uint32, vp, C.c_size_t, vp]
        lib.adsa_step_static.restype = C.c_int
        lib.adsa_step_static.argtypes = [pp, vp, vp, vp, vp, vp, f32p, i32p, i32p, i32p, C.c_uint32, vp]
        rp, tp, mp, sp = C.POINTER(AdsaRope), C.POINTER(AdsaTokens), C.POINTER(AdsaMods), C.POINTER(AdsaShared)
        lib.adsa_rotate.restype = C.c_int
        lib.adsa_rotate.argtypes = [pp, rp, vp, i32p, vp, vp, C.c_int64, C.c_int64, vp, vp, C.c_uint32, vp]
        lib.adsa_append.restype = C.c_int
        lib.adsa_append.argtypes = [pp, tp, rp, vp, vp, vp, vp, vp, C.c_uint32, vp]
        lib.adsa_prefill.restype = C.c_int
        lib.adsa_prefill.argtypes = [pp, tp, mp, vp, vp, vp, f32p, C.c_uint32, vp, C.c_size_t, vp]
        lib.adsa_prefill_workspace_bytes.restype = C.c_size_t
        lib.adsa_prefill_workspace_bytes.argtypes = [pp, tp]
        lib.adsa_attend_shared.restype = C.c_int
        lib.adsa_attend_shared.argtypes = [pp, sp, mp, vp, vp, vp, vp, i32p, i32p, vp, f32p, C.c_uint32, vp, C.c_size_t, vp]
        lib.adsa_shared_workspace_bytes.restype = C.c_size_t
        lib.adsa_shared_workspace_bytes.argtypes = [pp, sp]
        lib.adsa_profile_enable.restype = C.c_int
        lib.adsa_profile_enable.argtypes = [C.c_int]
        lib.adsa_profile_read.restype = C.c_int
        lib.adsa_profile_read.argtypes = [C.POINTER(C.c_int64), C.POINTER(C.c_double)]
        lib.adsa_strerror.restype = C.c_char_p
        lib.adsa_strerror.argtypes = [C.c_int]
        lib.adsa_version.restype = C.c_int
        lib.adsa_version.argtypes = []
        _lib = lib
    return _lib


_call = _call_static = _call_prompt = None       # the CPython module's functions
_entry = {}                       # C entry point -> its address


def _load_native():
    global _call, _call_static, _call_prompt
    lib, path = load_library(), _build.NATIVE_PATH
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: run `python -m paper_2506_18226_amd.build` (or __graft_entry__.build()) first; "
                                "there is no fallback path")
    loader = importlib.machinery.ExtensionFileLoader("_adsa_native", path)
    module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_adsa_native", loader))
    loader.exec_module(module)
    for name in ("adsa_select", "adsa_attend", "adsa_compact", "adsa_step", "adsa_step_static", "adsa_rotate", "adsa_append", "adsa_prefill",
                 "adsa_attend_shared"):
        _entry[name] = C.cast(getattr(lib, name), C.c_void_p).value
    module.set_params_type(AdsaParams)
    _call_static, _call_prompt = module.call_static, module.call_prompt
    _call = module.call


def _enqueue(name: str, params, flags, workspace, stream, *pointers) -> None:
    """One C call; seqs is the first of the pointers."""
    if _call is None:
        _load_native()
    rc = _call(_entry[name], params, flags, _current_stream() if stream is None else _stream(stream), workspace, *pointers)
    if rc != 0:
        raise AdsaError(rc, name)


def _ptr(x) -> Optional[int]:
    """Device pointer of a torch tensor, the integer itself, one of these with a byte offset, or None."""
    if isinstance(x, tuple):
        return _ptr(x[0]) + x[1]
    return x if x is None or isinstance(x, int) else x.data_ptr()


def _nbytes(x) -> int:
    return 0 if x is None else x.numel() * x.element_size()


_raw_stream = None


def _current_stream() -> int:
    """Handle of the current device's current stream.  torch.cuda.current_stream() wraps it in a Stream object, which takes
    2.7 us, as much as a kernel launch; the handle alone 0.2 us.  The first call goes through torch's own way, which also
    initialises the device; so does every call where torch does not have the two functions (they are not documented)."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        handle = torch.cuda.current_stream().cuda_stream
        raw, device = (getattr(torch._C, name, None) for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        if raw is None or device is None:
            return handle
        _raw_stream = raw, device
        return handle
    return _raw_stream[0](_raw_stream[1]())


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(rc: int, where: str) -> None:
    if rc != 0:
        raise AdsaError(rc, where)


def make_params(*, n_seq, n_heads, head_dim, grid_h, grid_w, win_rows_back, win_col_radius, dtype,
                score_mode, cap, sel_cap=None, sel_groups=1, layout="head_major", kv_slot_stride=None,
                kv_head_stride=None, softmax_scale=0.0, win_recent_m=0, evict_policy=0, q_per_kv=0) -> AdsaParams:
    """Fill `adsa_params`.  layout "head_major" = [head][slot][D] (a head's rows are contiguous: the
    fast path), "slot_major" = [slot][head][D]; explicit strides override it."""
    if kv_head_stride is None:
        kv_head_stride = cap * head_dim if layout == "head_major" else head_dim
    if kv_slot_stride is None:
        kv_slot_stride = head_dim if layout == "head_major" else n_heads * head_dim
    return AdsaParams(n_seq, n_heads, head_dim, grid_h, grid_w, win_rows_back, win_col_radius, sel_groups,
                      dtype, score_mode, cap, cap if sel_cap is None else sel_cap,
                      kv_slot_stride, kv_head_stride, softmax_scale, win_recent_m, evict_policy, q_per_kv)


def score_rows(params: AdsaParams) -> int:
    """Rows of adsa_seq.score: one per head for ATTN_MASS, two per head for VCOS_FUSED, else one.  (With per-head
    attended sets, sel_groups == n_heads, every record describes one head.)"""
    heads = 1 if params.sel_groups == params.n_heads else params.n_heads
    if params.score_mode == SCORE_VCOS_FUSED:
        return 2 * heads
    return heads if params.score_mode == SCORE_ATTN_MASS else 1


def query_heads(params: AdsaParams) -> int:
    """Heads of q / out / lse: n_heads cache heads times q_per_kv query heads each."""
    return params.n_heads * max(params.q_per_kv, 1)


def strerror(code: int) -> str:
    return load_library().adsa_strerror(code).decode()


def adsa_version() -> int:
    return load_library().adsa_version()


def adsa_workspace_bytes(params: AdsaParams) -> int:
    return int(load_library().adsa_workspace_bytes(C.byref(params)))


def adsa_workspace_init(params, workspace, stream=None) -> None:
    _check(load_library().adsa_workspace_init(C.byref(params), _ptr(workspace), _nbytes(workspace),
                                              _stream(stream)), "adsa_workspace_init")


def adsa_select(params, seqs, sel_idx, sel_cnt, workspace=None, flags=0, stream=None) -> None:
    _enqueue("adsa_select", params, flags, workspace, stream, seqs, sel_idx, sel_cnt)


def adsa_attend(params, seqs, q, sel_idx, sel_cnt, out, lse, workspace, flags=0, k_new=None, v_new=None,
                stream=None) -> None:
    _enqueue("adsa_attend", params, flags, workspace, stream, seqs, q, k_new, v_new, sel_idx, sel_cnt, out, lse)


def adsa_compact(params, seqs, keep_map, workspace, flags=0, stream=None) -> None:
    _enqueue("adsa_compact", params, flags, workspace, stream, seqs, keep_map)


def adsa_step(params, seqs, q, k_new, v_new, out, lse, sel_idx, sel_cnt, keep_map, workspace,
              flags=0, stream=None) -> None:
    _enqueue("adsa_step", params, flags, workspace, stream, seqs, q, k_new, v_new, out, lse, sel_idx, sel_cnt, keep_map)


def adsa_step_static(params, seqs, q, k_new, v_new, out, lse, sel_idx, sel_cnt, keep_map, flags=0, stream=None) -> None:
    """adsa_step on the library's built-in scratch array: no workspace argument, no allocation."""
    if _call_static is None:
        _load_native()
    rc = _call_static(_entry["adsa_step_static"], params, flags, _current_stream() if stream is None else _stream(stream),
                      seqs, q, k_new, v_new, out, lse, sel_idx, sel_cnt, keep_map)
    if rc != 0:
        raise AdsaError(rc, "adsa_step_static")


def _axes(name, values, n):
    values = tuple(int(x) for x in values)
    if len(values) != n:
        raise ValueError(f"{name}: one number for each of {n} axes expected")
    return (C.c_int32 * MAX_AXES)(*values)


def _expect(name, x, dtype, *shape):
    """A device tensor that the C side reads as dtype without gaps (raw integers go through unchecked)."""
    if x is None or isinstance(x, int):
        return
    if str(x.dtype) != f"torch.{dtype}" or not x.is_contiguous() or (shape and tuple(x.shape) != shape):
        raise ValueError(f"{name}: a contiguous {dtype} tensor{' of shape ' + str(shape) if shape else ''} expected")


def _length(x):
    """Elements of a tensor along its first axis; None of a raw pointer, whose shape nobody knows."""
    return None if x is None or isinstance(x, int) else x.shape[0] if x.dim() else 1


def _check_sizes(struct, **least) -> None:
    """What a call reads of a host struct's tensors has to be there."""
    if struct is not None:
        for name, n in struct.sizes:
            if n < least.get(name, 0):
                raise ValueError(f"{name}: {least[name]} expected along the first axis, {n} there")


def _check_rope(params, rope, coords_width) -> None:
    if rope is None:
        return
    if rope.width not in (None, params.head_dim // 2):
        raise ValueError(f"freq: [axes][{params.head_dim // 2}] expected, {rope.width} there")
    if coords_width not in (None, rope.n_axes):
        raise ValueError(f"coords: one number for each of {rope.n_axes} axes expected, {coords_width} there")


def make_rope(freq, *, pairing="halves", text, origin, row, col) -> AdsaRope:
    """Fill `adsa_rope`.  freq: fp64 device tensor [axes][head_dim / 2], radians by which one unit of each axis turns each pair; the other
    arguments hold one integer per axis (see include/adsa.h for the rule from position to coordinates)."""
    _expect("freq", freq, "float64")
    if freq.dim() != 2 or not 1 <= freq.shape[0] <= MAX_AXES:
        raise ValueError(f"freq: [1..{MAX_AXES}][head_dim / 2] expected")
    n = freq.shape[0]
    return AdsaRope(_ptr(freq), n, PAIRINGS[pairing], _axes("text", text, n), _axes("origin", origin, n), _axes("row", row, n),
                    _axes("col", col, n))._hold(freq, width=freq.shape[1])


def make_tokens(begin, slot0, n_tokens, max_len, *, pos0=None, coords=None, q_stride=0, k_stride=0, v_stride=0) -> AdsaTokens:
    """Fill `adsa_tokens`: int32 device tensors begin [n_seq + 1], slot0 and pos0 [n_seq], coords [n_tokens][axes]."""
    for name, x in (("begin", begin), ("slot0", slot0), ("pos0", pos0), ("coords", coords)):
        _expect(name, x, "int32")
    if _length(coords) is not None and (coords.dim() != 2 or coords.shape[0] < n_tokens):
        raise ValueError(f"coords: [{n_tokens}][axes] expected")
    return AdsaTokens(n_tokens, max_len, _ptr(begin), _ptr(slot0), _ptr(pos0), _ptr(coords), q_stride, k_stride, v_stride)._hold(
        begin, slot0, pos0, coords, sizes=(("begin", _length(begin)), ("slot0", _length(slot0)), ("pos0", _length(pos0))),
        width=None if _length(coords) is None else coords.shape[1])


def make_mods(*, softcap=0.0, mask=MASK_CAUSAL, slopes=None, doc=None) -> AdsaMods:
    """Fill `adsa_mods`: slopes float32 [query heads], doc int32 [n_seq][>= cap], both on the device."""
    _expect("slopes", slopes, "float32")
    _expect("doc", doc, "int32")
    stride = 0 if doc is None else doc.shape[-1]
    return AdsaMods(softcap, mask, _ptr(slopes), _ptr(doc), stride)._hold(
        slopes, doc, sizes=(("slopes", _length(slopes)), ("doc", None if doc is None else doc.numel() // max(stride, 1))))


def make_shared(prompt_params, prompts, members, *, max_members) -> AdsaShared:
    """Fill `adsa_shared`: the records `prompts` (one per group; a tensor, or one and a byte offset) of caches made for prompt_params, and int32
    members [n_groups + 1]."""
    _expect("members", members, "int32")
    p = prompt_params
    records, skipped = prompts if isinstance(prompts, tuple) else (prompts, 0)
    there = None if records is None or isinstance(records, int) else (_nbytes(records) - skipped) // SEQ_DTYPE.itemsize
    shared = AdsaShared(p.n_seq, p.cap, max_members, 0, _ptr(prompts), _ptr(members), p.kv_slot_stride, p.kv_head_stride)._hold(
        prompts, members, sizes=(("members", _length(members)), ("prompts", there)))
    _check_sizes(shared, members=p.n_seq + 1, prompts=p.n_seq)
    shared.rows = p.n_heads, p.head_dim, p.dtype
    return shared


def _host(x):
    return None if x is None else C.byref(x)


_PROMPT_CALLS = {"adsa_rotate": 0, "adsa_append": 1, "adsa_prefill": 2, "adsa_attend_shared": 3}


def _struct(x, kind, name):
    if x is not None and type(x) is not kind:
        raise TypeError(f"{name}: {kind.__name__} expected")
    return x


def _prompt_call(name, params, second, third, flags, stream, workspace, *rest) -> None:
    if _call_prompt is None:
        _load_native()
    rc = _call_prompt(_PROMPT_CALLS[name], _entry[name], params, second, third, flags, _current_stream() if stream is None else _stream(stream),
                      workspace, *rest)
    if rc != 0:
        raise AdsaError(rc, name)


def adsa_rotate(params, rope, seqs, q, k, q_out, k_out, coords=None, flags=0, stream=None, q_stride=0, k_stride=0) -> None:
    _struct(rope, AdsaRope, "rope")
    width = None
    if not (coords is None or isinstance(coords, (int, tuple))):
        _expect("coords", coords, "int32")
        if coords.dim() != 2 or coords.shape[0] < params.n_seq:
            raise ValueError(f"coords: [{params.n_seq}][axes] expected")
        width = coords.shape[1]
    _check_rope(params, rope, width)
    _prompt_call("adsa_rotate", params, rope, None, flags, stream, None, seqs, coords, q, k, q_out, k_out, q_stride, k_stride)


def _tokens(params, tokens):
    _struct(tokens, AdsaTokens, "tokens")
    _check_sizes(tokens, begin=params.n_seq + 1, slot0=params.n_seq, pos0=params.n_seq)
    return tokens


def _mods(params, mods, docs):
    _struct(mods, AdsaMods, "mods")
    if mods is not None:
        _check_sizes(mods, slopes=query_heads(params), doc=docs)
    return mods


def adsa_append(params, tokens, rope, seqs, q, k, v, q_out, flags=0, stream=None) -> None:
    _struct(rope, AdsaRope, "rope")
    _tokens(params, tokens)
    _check_rope(params, rope, None if tokens is None else tokens.width)
    _prompt_call("adsa_append", params, tokens, rope, flags, stream, None, seqs, q, k, v, q_out)


def adsa_prefill_workspace_bytes(params, tokens) -> int:
    return int(load_library().adsa_prefill_workspace_bytes(_host(params), _host(tokens)))


def adsa_prefill(params, tokens, mods, seqs, q, out, lse, workspace, flags=0, stream=None) -> None:
    _prompt_call("adsa_prefill", params, _tokens(params, tokens), _mods(params, mods, params.n_seq), flags, stream, workspace, seqs, q, out, lse)


def adsa_shared_workspace_bytes(params, shared) -> int:
    return int(load_library().adsa_shared_workspace_bytes(_host(params), _host(shared)))


def adsa_attend_shared(params, shared, mods, seqs, q, k_new, v_new, sel_idx, sel_cnt, out, lse, workspace, flags=0, stream=None) -> None:
    _struct(shared, AdsaShared, "shared")
    if shared is not None and shared.rows not in (None, (params.n_heads, params.head_dim, params.dtype)):
        raise ValueError(f"shared: prompts of (heads, head_dim, dtype) {shared.rows}, sequences of {(params.n_heads, params.head_dim, params.dtype)}")
    _prompt_call("adsa_attend_shared", params, shared, _mods(params, mods, 0), flags, stream, workspace, seqs, q,
                 k_new, v_new, sel_idx, sel_cnt, out, lse)


def adsa_profile_enable(on: bool) -> None:
    _check(load_library().adsa_profile_enable(1 if on else 0), "adsa_profile_enable")


def adsa_profile_read():
    """(number of bracketed attention launches, their summed duration in ms)."""
    n, ms = C.c_int64(0), C.c_double(0.0)
    _check(load_library().adsa_profile_read(C.byref(n), C.byref(ms)), "adsa_profile_read")
    return n.value, ms.value

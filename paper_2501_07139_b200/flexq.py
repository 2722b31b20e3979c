"""ctypes binding of libflexq.so: argument marshalling only.

Every method has the name of the C function it calls.  torch is used for device memory
and streams; all computation happens inside the library's CUDA kernels.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from array import array
from operator import attrgetter
from typing import List, Optional, Sequence

import torch

FQ_FMT_PACKED = 0
FQ_FMT_PLANES = 1
FQ_MAX_BATCH = 8
FQ_DT_F16 = 0
FQ_DT_BF16 = 1
FQ_DT_F32 = 2
FQ_MAX_TOP = 128
FQ_MAX_VOCAB = 393216
_I8, _F32, _I32, _I64, _IDS = (torch.int8,), (torch.float32,), (torch.int32,), (torch.int64,), (torch.int32, torch.int64)
_dtype_of = attrgetter("dtype")
_HALF = (torch.float16, torch.bfloat16)
_TYPES = {torch.float16: FQ_DT_F16, torch.bfloat16: FQ_DT_BF16, torch.float32: FQ_DT_F32}

_HERE = os.path.dirname(os.path.abspath(__file__))
# FLEXQ_LIBRARY selects the file: unset = libflexq.so, "checked" = libflexq_checked.so (the bounds-checked build,
# `python -m paper_2501_07139_b200.build --checked`), anything else = a path.
_LIB_PATH = {None: os.path.join(_HERE, "libflexq.so"), "": os.path.join(_HERE, "libflexq.so"),
             "checked": os.path.join(_HERE, "libflexq_checked.so")}.get(os.environ.get("FLEXQ_LIBRARY"),
                                                                        os.environ.get("FLEXQ_LIBRARY"))
_lib = None

EXPORTS = [
    "fq_create", "fq_destroy", "fq_store_bytes", "fq_quantize_layer", "fq_pack_layer",
    "fq_set_config", "fq_gemv", "fq_gemv_batched", "fq_gemv_stack", "fq_gemm", "fq_export_layer",
    "fq_export_meta", "fq_storage_bytes", "fq_active_bits", "fq_status", "fq_strerror", "fq_gemv_static", "fq_transition", "fq_save", "fq_load", "fq_search_chain", "fq_prune_chain", "fq_sqdiff",
    "fq_set_wait_limit_ns", "fq_code_bytes", "fq_meta_bytes", "fq_stream_read", "fq_gemm_two_pass", "fq_gemm_plan",
    "fq_host_variant", "fq_transition_swap", "fq_quantize_rows", "fq_gemm_i8", "fq_linear_i8", "fq_token_logprobs", "fq_distill_topk",
    "fq_distill_topk_grad", "fq_cache_step", "fq_cache_move", "fq_rotary_table", "fq_rotary", "fq_rotary_cache", "fq_tree_attention_scratch",
    "fq_tree_attention",
]


class TransitionReport(C.Structure):
    _fields_ = [("bytes_freed", C.c_uint64), ("bytes_loaded", C.c_uint64), ("footprint_from", C.c_uint64),
                ("footprint_to", C.c_uint64), ("layers_changed", C.c_int), ("one_way", C.c_int)]


class SwapReport(C.Structure):
    _fields_ = [("bytes_loaded", C.c_uint64), ("bytes_freed", C.c_uint64), ("peak_extra_bytes", C.c_uint64),
                ("resident_bytes", C.c_uint64), ("footprint_from", C.c_uint64), ("footprint_to", C.c_uint64),
                ("layers_changed", C.c_int), ("one_way", C.c_int)]


class GemmPlan(C.Structure):
    _fields_ = [("two_pass", C.c_int), ("shared", C.c_int), ("blocks", C.c_int), ("tile_tokens", C.c_int), ("tiles", C.c_longlong)]


# The structures that the calls between the linear layers take, packed as C lays them out: an address, then strides, then counts.
_HEADS, _CACHE = "qqqi4x", "qqqqqiii4x"
_STEP_ARGS = struct.Struct("qqqqqqqqqqqqiiiiii")
_MOVE_ARGS = struct.Struct("q" + _CACHE + "qqqqqqqqiiiiii")
_ROTARY_ARGS = struct.Struct(4 * _HEADS + "qqiiiiiiiif4x")
_ROTARY_CACHE_ARGS = struct.Struct(4 * _HEADS + _CACHE + "qqqiiiiiif4x")
_ATTENTION_ARGS = struct.Struct(2 * _HEADS + _CACHE + "qqqqqqqqiiiiiiif")
_NO_HEADS = (0, 0, 0, 0)


class FlexQError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {fq_strerror(code)} ({code})")


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Loads libflexq.so (once).  Raises if it is missing: build it with
    `python -m paper_2501_07139_b200.build` or `__graft_entry__.build()`."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(f"{_LIB_PATH} not built; run `python -m paper_2501_07139_b200.build`")
    L = C.CDLL(_LIB_PATH)
    vp, i, u64 = C.c_void_p, C.c_int, C.c_uint64
    L.fq_create.argtypes = [C.POINTER(vp), i, i]
    L.fq_destroy.argtypes = [vp]
    L.fq_store_bytes.argtypes = [i, i, i, i]
    L.fq_store_bytes.restype = C.c_size_t
    L.fq_quantize_layer.argtypes = [vp, i, i, i, i, vp, vp, vp, vp]
    L.fq_pack_layer.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, vp]
    L.fq_set_config.argtypes = [vp, vp, i, C.POINTER(u64), vp]
    L.fq_transition.argtypes = [vp, vp, i, i, C.POINTER(TransitionReport), vp]
    L.fq_host_variant.argtypes = [vp, i, i, i, i, vp]
    L.fq_transition_swap.argtypes = [vp, vp, i, i, C.POINTER(SwapReport), vp]
    L.fq_save.argtypes = [vp, C.c_char_p, C.POINTER(u64)]
    L.fq_load.argtypes = [vp, C.c_char_p]
    L.fq_search_chain.argtypes = [vp, vp, vp, i, i, i, i, vp, C.POINTER(i), C.POINTER(C.c_double)]
    L.fq_prune_chain.argtypes = [vp, i, i, i, vp, C.c_double, vp, vp, C.POINTER(u64), C.POINTER(u64)]
    L.fq_sqdiff.argtypes = [vp, vp, C.c_size_t, vp, vp]
    L.fq_gemv.argtypes = [vp, i, vp, vp, vp]
    L.fq_gemv_batched.argtypes = [vp, i, vp, i, vp, vp]
    L.fq_gemv_static.argtypes = [vp, i, vp, vp, vp]
    L.fq_gemv_stack.argtypes = [vp, i, vp, vp, vp, vp, i, vp]
    L.fq_gemm.argtypes = [vp, i, vp, i, i, vp, i, vp]
    L.fq_gemm_two_pass.argtypes = [vp, i, vp, i, i, vp, i, vp]
    L.fq_gemm_plan.argtypes = [vp, i, i, C.POINTER(GemmPlan)]
    L.fq_export_layer.argtypes = [vp, i, i, vp, vp]
    L.fq_export_meta.argtypes = [vp, i, i, vp, vp, vp]
    L.fq_storage_bytes.argtypes = [vp]
    L.fq_storage_bytes.restype = u64
    L.fq_active_bits.argtypes = [vp, i]
    L.fq_status.argtypes = [vp]
    L.fq_set_wait_limit_ns.argtypes = [vp, u64]
    L.fq_stream_read.argtypes = [vp, vp, C.c_size_t, vp]
    L.fq_code_bytes.argtypes = [i, i, i]
    L.fq_code_bytes.restype = C.c_size_t
    L.fq_meta_bytes.argtypes = [i, i, i]
    L.fq_meta_bytes.restype = C.c_size_t
    ll, fl = C.c_longlong, C.c_float
    L.fq_quantize_rows.argtypes = [vp, vp, i, i, i, ll, vp, ll, vp, vp]
    L.fq_gemm_i8.argtypes = [vp, vp, vp, i, ll, vp, vp, i, i, ll, vp, i, ll, vp]
    L.fq_linear_i8.argtypes = [vp, vp, i, i, ll, vp, vp, i, i, ll, vp, ll, vp, vp, i, ll, vp]
    L.fq_token_logprobs.argtypes = [vp, vp, i, i, i, ll, vp, i, fl, vp, vp, i, vp, vp, vp]
    L.fq_distill_topk.argtypes = [vp, vp, i, i, i, ll, vp, i, vp, i, fl, vp, vp, vp, vp, ll, vp]
    L.fq_distill_topk_grad.argtypes = [vp, vp, i, i, i, ll, vp, i, vp, i, fl, vp, vp, vp, ll, vp]
    db = C.c_double
    for name in ("fq_cache_step", "fq_cache_move", "fq_rotary", "fq_rotary_cache", "fq_tree_attention"):
        getattr(L, name).argtypes = [vp, vp, vp]
    L.fq_rotary_table.argtypes = [i, db, db, i, db, db, vp]
    L.fq_tree_attention_scratch.argtypes = [vp, i, i, i, i, i, i]
    L.fq_tree_attention_scratch.restype = C.c_size_t
    L.fq_strerror.argtypes = [i]
    L.fq_strerror.restype = C.c_char_p
    for name in EXPORTS:
        fn = getattr(L, name)
        if fn.restype is C.c_int or fn.restype is None:
            fn.restype = C.c_int
    _lib = L
    return L


def fq_strerror(code: int) -> str:
    return lib().fq_strerror(int(code)).decode()


def fq_store_bytes(n_out: int, k_in: int, bits: int, fmt: int) -> int:
    return int(lib().fq_store_bytes(n_out, k_in, bits, fmt))


def fq_code_bytes(n_out: int, k_in: int, bits: int) -> int:
    return int(lib().fq_code_bytes(n_out, k_in, bits))


def fq_meta_bytes(n_out: int, k_in: int, group: int = 128) -> int:
    return int(lib().fq_meta_bytes(n_out, k_in, group))


# torch's own short way to the stream's handle, where there is one: without building a Stream object, a call is a few microseconds in all
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    if _raw_stream and _device and torch.cuda.is_initialized():
        return _raw_stream(_device())
    return torch.cuda.current_stream().cuda_stream


def _stream_on(device: torch.device) -> int:
    """The stream that is current on `device`, which need not be the current device."""
    if _raw_stream and torch.cuda.is_initialized():
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _check(rc: int, where: str) -> int:
    if rc != 0:
        raise FlexQError(rc, where)
    return rc


def fq_search_chain(cost, sens, foot, stems: int, branches: int):
    """Algorithm 1 on host tables [module][level]; returns (chain as a list of level lists, curve cost)."""
    import numpy as np
    c = np.ascontiguousarray(cost, np.float64)
    s_ = np.ascontiguousarray(sens, np.float64)
    f = np.ascontiguousarray(foot, np.uint64)
    m, lv = c.shape
    chain = np.zeros((m * (lv - 1) + 1, m), np.uint8)
    n_states, curve = C.c_int(0), C.c_double(0.0)
    _check(lib().fq_search_chain(c.ctypes.data, s_.ctypes.data, f.ctypes.data, m, lv, stems, branches, chain.ctypes.data,
                                 C.byref(n_states), C.byref(curve)), "fq_search_chain")
    return chain[:n_states.value].tolist(), float(curve.value)


def fq_prune_chain(chain, n_levels: int, foot, fraction: float):
    """Sec. III-C; returns (pruned chain, set of dropped (module, level), storage before, storage after)."""
    import numpy as np
    ch = np.ascontiguousarray(chain, np.uint8)
    f = np.ascontiguousarray(foot, np.uint64)
    n_states, m = ch.shape
    out = np.zeros_like(ch)
    dropped = np.zeros((m, n_levels), np.uint8)
    before, after = C.c_uint64(0), C.c_uint64(0)
    _check(lib().fq_prune_chain(ch.ctypes.data, n_states, m, n_levels, f.ctypes.data, float(fraction), out.ctypes.data,
                                dropped.ctypes.data, C.byref(before), C.byref(after)), "fq_prune_chain")
    return out.tolist(), {(int(a), int(b)) for a, b in zip(*np.nonzero(dropped))}, int(before.value), int(after.value)


def fq_sqdiff(a: torch.Tensor, b: torch.Tensor) -> torch.Tensor:
    """Device tensor [sum (a-b)^2, sum b^2] (float64) over two bf16 tensors of the same size."""
    assert a.dtype == torch.bfloat16 and b.dtype == torch.bfloat16 and a.is_contiguous() and b.is_contiguous()
    assert a.numel() == b.numel()
    out = torch.empty(2, dtype=torch.float64, device=a.device)
    _check(lib().fq_sqdiff(a.data_ptr(), b.data_ptr(), a.numel(), out.data_ptr(), _stream()), "fq_sqdiff")
    return out


def fq_quantize_layer(w: torch.Tensor, bits: int, group: int = 128):
    """W float32 [N][K] on the GPU -> (codes uint8 [N][K], scales fp16 [N][K/128], zeros fp16 [N][K/128])."""
    assert w.is_cuda and w.dtype == torch.float32 and w.is_contiguous()
    n, k = w.shape
    codes = torch.empty((n, k), dtype=torch.uint8, device=w.device)
    scales = torch.empty((n, k // group), dtype=torch.float16, device=w.device)
    zeros = torch.empty((n, k // group), dtype=torch.float16, device=w.device)
    with torch.cuda.device(w.device):
        _check(lib().fq_quantize_layer(w.data_ptr(), n, k, bits, group, codes.data_ptr(), scales.data_ptr(),
                                       zeros.data_ptr(), _stream()), "fq_quantize_layer")
    return codes, scales, zeros


def fq_rotary_table(rot_dim: int, base: float = 10000.0, factor: float = 1.0, context: int = 0, low: float = 1.0, high: float = 32.0,
                    device="cuda") -> torch.Tensor:
    """Angles for fq_rotary and fq_rotary_cache, int64 [rot_dim / 2] on `device`: pair i turns by base^(-2i / rot_dim) radians a position.  For contexts `factor`
    times as long as the trained one, of `context` tokens: pairs that turn `high` times in it and more stay, those that turn `low` times and
    less are slowed by `factor`, between them both are mixed; with context 0 all are slowed."""
    turns = torch.empty(max(rot_dim // 2, 1), dtype=torch.int64)
    _check(lib().fq_rotary_table(rot_dim, base, factor, context, low, high, turns.data_ptr()), "fq_rotary_table")
    return turns.to(device)


class FlexQ:
    """One library context.  Keeps the retained device buffers (the stored variants) alive."""

    def __init__(self, n_layers: int, device: int = 0):
        self._h = C.c_void_p()
        self.device = torch.device("cuda", device)
        self._index = device
        _check(lib().fq_create(C.byref(self._h), device, n_layers), "fq_create")
        self.n_layers = n_layers
        self._keep = {}          # (layer, bits) -> stored variant retained by the context
        self._stack_keep = None
        self._scratch = {}       # sizes of an attention call -> bytes of scratch

    # -- lifetime -----------------------------------------------------------------
    def fq_destroy(self):
        if self._h:
            lib().fq_destroy(self._h)
            self._h = C.c_void_p()
            self._keep.clear()

    def __del__(self):
        try:
            self.fq_destroy()
        except Exception:
            pass

    # -- packing --------------------------------------------------------------------
    def fq_pack_layer(self, layer: int, codes: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor,
                      bits: int, fmt: int = FQ_FMT_PACKED, group: int = 128):
        assert codes.is_cuda and codes.dtype == torch.uint8 and codes.is_contiguous()
        assert scales.dtype == torch.float16 and zeros.dtype == torch.float16
        n, k = codes.shape
        sb = fq_store_bytes(n, k, bits, fmt)
        if sb == 0 or group != 128:
            # let the library name the problem
            _check(lib().fq_pack_layer(self._h, layer, n, k, bits, group, fmt, codes.data_ptr(), scales.data_ptr(),
                                       zeros.data_ptr(), codes.data_ptr(), _stream()), "fq_pack_layer")
        store = torch.empty(sb, dtype=torch.uint8, device=self.device)
        _check(lib().fq_pack_layer(self._h, layer, n, k, bits, group, fmt, codes.data_ptr(),
                                   scales.contiguous().data_ptr(), zeros.contiguous().data_ptr(),
                                   store.data_ptr(), _stream()), "fq_pack_layer")
        self._keep[(layer, bits)] = store
        return store

    # -- configuration -------------------------------------------------------------------
    def fq_set_config(self, bits: Sequence[int]) -> int:
        arr = (C.c_uint8 * len(bits))(*[int(b) for b in bits])
        fp = C.c_uint64(0)
        _check(lib().fq_set_config(self._h, arr, len(bits), C.byref(fp), _stream()), "fq_set_config")
        return int(fp.value)

    def fq_transition(self, bits: Sequence[int], require_one_way: bool = True) -> dict:
        arr = (C.c_uint8 * len(bits))(*[int(b) for b in bits])
        rep = TransitionReport()
        _check(lib().fq_transition(self._h, arr, len(bits), 1 if require_one_way else 0, C.byref(rep), _stream()),
               "fq_transition")
        return {"bytes_freed": int(rep.bytes_freed), "bytes_loaded": int(rep.bytes_loaded),
                "layers_changed": int(rep.layers_changed), "one_way": bool(rep.one_way),
                "footprint_from": int(rep.footprint_from), "footprint_to": int(rep.footprint_to)}

    def fq_host_variant(self, layer: int, n_out: int, k_in: int, bits: int, store_host: torch.Tensor) -> None:
        """Registers a PACKED variant whose stored bytes lie in the (page-locked) host tensor `store_host`."""
        if store_host.device.type != "cpu" or not store_host.is_contiguous():
            raise ValueError("store_host must be a contiguous host tensor")
        if store_host.numel() * store_host.element_size() < fq_store_bytes(n_out, k_in, bits, FQ_FMT_PACKED):
            raise ValueError("store_host is smaller than fq_store_bytes")
        self._keep[("host", layer, bits)] = store_host       # the library reads it at every swap-in
        _check(lib().fq_host_variant(self._h, layer, n_out, k_in, bits, store_host.data_ptr()), "fq_host_variant")

    def fq_transition_swap(self, bits: Sequence[int], require_one_way: bool = True) -> dict:
        arr = (C.c_uint8 * len(bits))(*[int(b) for b in bits])
        rep = SwapReport()
        _check(lib().fq_transition_swap(self._h, arr, len(bits), 1 if require_one_way else 0, C.byref(rep), _stream()),
               "fq_transition_swap")
        return {k: int(getattr(rep, k)) for k, _ in SwapReport._fields_}

    def fq_save(self, path: str) -> int:
        """Writes every stored variant to `path`; returns the bytes written."""
        n = C.c_uint64(0)
        _check(lib().fq_save(self._h, os.fsencode(path), C.byref(n)), "fq_save")
        return int(n.value)

    def fq_load(self, path: str):
        """Registers the layers of a file written by fq_save (the library allocates their device buffers)."""
        _check(lib().fq_load(self._h, os.fsencode(path)), "fq_load")

    def fq_storage_bytes(self) -> int:
        return int(lib().fq_storage_bytes(self._h))

    def fq_active_bits(self, layer: int) -> int:
        rc = lib().fq_active_bits(self._h, layer)
        if rc < 0:
            raise FlexQError(rc, "fq_active_bits")
        return rc

    def fq_status(self) -> int:
        return int(lib().fq_status(self._h))

    def fq_stream_read(self, buf: torch.Tensor):
        """One read-only pass over a device buffer (measurement support)."""
        _check(lib().fq_stream_read(self._h, buf.data_ptr(), buf.numel() * buf.element_size(), _stream()), "fq_stream_read")

    def fq_set_wait_limit_ns(self, ns: int):
        """Limit of every device-side wait of the decode kernels (0 restores the default of 2 s)."""
        _check(lib().fq_set_wait_limit_ns(self._h, int(ns)), "fq_set_wait_limit_ns")

    # -- decode --------------------------------------------------------------------------
    def fq_gemv(self, layer: int, x: torch.Tensor, y: torch.Tensor):
        _check(lib().fq_gemv(self._h, layer, x.data_ptr(), y.data_ptr(), _stream()), "fq_gemv")
        return y

    def fq_gemv_static(self, layer: int, x: torch.Tensor, y: torch.Tensor):
        """fq_gemv without any device allocation: split-K scratch lives in a fixed array inside the
        library (see include/flexq.h).  Raises FlexQError(-9) when the layer does not fit."""
        _check(lib().fq_gemv_static(self._h, layer, x.data_ptr(), y.data_ptr(), _stream()), "fq_gemv_static")
        return y

    def fq_gemv_batched(self, layer: int, x: torch.Tensor, y: torch.Tensor):
        _check(lib().fq_gemv_batched(self._h, layer, x.data_ptr(), x.shape[0], y.data_ptr(), _stream()),
               "fq_gemv_batched")
        return y

    def fq_gemv_stack(self, layers: Sequence[int], xs: Sequence[torch.Tensor], ys: Sequence[torch.Tensor],
                      phases: Optional[Sequence[int]] = None, batch: int = 1):
        n = len(layers)
        la = (C.c_int * n)(*[int(v) for v in layers])
        xa = (C.c_void_p * n)(*[t.data_ptr() for t in xs])
        ya = (C.c_void_p * n)(*[t.data_ptr() for t in ys])
        pa = (C.c_int * n)(*[int(v) for v in phases]) if phases is not None else None
        self._stack_keep = (la, xa, ya, pa)
        _check(lib().fq_gemv_stack(self._h, n, la, xa, ya, pa, batch, _stream()), "fq_gemv_stack")

    def stack_args(self, layers, xs, ys, phases=None):
        """Pre-marshalled argument arrays for repeated fq_gemv_stack_raw calls."""
        n = len(layers)
        la = (C.c_int * n)(*[int(v) for v in layers])
        xa = (C.c_void_p * n)(*[t.data_ptr() for t in xs])
        ya = (C.c_void_p * n)(*[t.data_ptr() for t in ys])
        pa = (C.c_int * n)(*[int(v) for v in phases]) if phases is not None else None
        return (n, la, xa, ya, pa)

    def fq_gemv_stack_raw(self, args, batch: int = 1):
        n, la, xa, ya, pa = args
        _check(lib().fq_gemv_stack(self._h, n, la, xa, ya, pa, batch, _stream()), "fq_gemv_stack")

    # -- prefill --------------------------------------------------------------------------
    def fq_gemm(self, layer: int, X: torch.Tensor, Y: torch.Tensor):
        assert X.dtype == torch.bfloat16 and Y.dtype == torch.bfloat16
        _check(lib().fq_gemm(self._h, layer, X.data_ptr(), X.shape[0], X.stride(0), Y.data_ptr(), Y.stride(0),
                             _stream()), "fq_gemm")
        return Y

    def fq_gemm_two_pass(self, layer: int, X: torch.Tensor, Y: torch.Tensor):
        """The comparison point of fq_gemm: dequantise to a bf16 workspace, then a plain tcgen05 GEMM."""
        assert X.dtype == torch.bfloat16 and Y.dtype == torch.bfloat16
        _check(lib().fq_gemm_two_pass(self._h, layer, X.data_ptr(), X.shape[0], X.stride(0), Y.data_ptr(), Y.stride(0),
                                      _stream()), "fq_gemm_two_pass")
        return Y

    # -- export (tests / reporting) ----------------------------------------------------------
    def fq_gemm_plan(self, layer: int, tokens: int) -> dict:
        """How `fq_gemm` runs that many tokens through a layer."""
        r = GemmPlan()
        _check(lib().fq_gemm_plan(self._h, layer, tokens, C.byref(r)), "fq_gemm_plan")
        return {f: getattr(r, f) for f, _ in GemmPlan._fields_}

    def fq_export_layer(self, layer: int, bits: int, n_out: int, k_in: int) -> torch.Tensor:
        out = torch.empty(n_out * k_in * bits // 32, dtype=torch.int32, device=self.device)
        _check(lib().fq_export_layer(self._h, layer, bits, out.data_ptr(), _stream()), "fq_export_layer")
        return out

    def fq_export_meta(self, layer: int, bits: int, n_out: int, k_in: int):
        s = torch.empty((n_out, k_in // 128), dtype=torch.float16, device=self.device)
        z = torch.empty((n_out, k_in // 128), dtype=torch.float16, device=self.device)
        _check(lib().fq_export_meta(self._h, layer, bits, s.data_ptr(), z.data_ptr(), _stream()), "fq_export_meta")
        return s, z

    # -- 8-bit layers ------------------------------------------------------------------------
    def _matrix(self, t: torch.Tensor, name: str, types) -> tuple:
        """(rows, columns, elements from one row to the next; of one row, any that the library takes)"""
        shape, st = t.shape, t.stride()
        if len(shape) != 2 or t.dtype not in types or t.get_device() != self._index or (st[1] != 1 and shape[1] > 1):
            raise ValueError(f"{name}: a matrix of {', '.join(str(d) for d in types)} on {self.device} with dense rows is needed, not "
                             f"{t.dtype} {tuple(shape)} with strides {st} on {t.device}")
        rows, cols = shape
        return rows, cols, st[0] if rows > 1 else -(-cols // 16) * 16

    def _dense(self, t: torch.Tensor, name: str, types, shape: tuple) -> torch.Tensor:
        if t.shape != shape or t.dtype not in types or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError(f"{name}: dense {shape} values of {', '.join(str(d) for d in types)} on {self.device} are needed, not "
                             f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")
        return t

    def _codes_and_scales(self, codes, scales, rows, cols):
        """Given or new ones: codes, their pitch, scales.  New codes get a row pitch that fq_gemm_i8 takes (a multiple of 16)."""
        if codes is None:
            pitch = -(-cols // 16) * 16
            codes = torch.empty((rows, pitch), dtype=torch.int8, device=self.device)
            if pitch != cols:
                codes = codes[:, :cols]
        else:
            r, c, pitch = self._matrix(codes, "codes", _I8)
            if r != rows or c != cols:
                raise ValueError(f"codes: {rows} x {cols} are needed, not {r} x {c}")
        if scales is None:
            scales = torch.empty(rows, dtype=torch.float32, device=self.device)
        else:
            self._dense(scales, "scales", _F32, (rows,))
        return codes, pitch, scales

    def fq_quantize_rows(self, x: torch.Tensor, codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None):
        """Rows of x (tokens, or the channels of a weight matrix) -> (int8 codes, fp32 scale per row).  New codes get a row pitch
        that fq_gemm_i8 takes (a multiple of 16)."""
        rows, cols, ldx = self._matrix(x, "x", _TYPES)
        codes, ldc, scales = self._codes_and_scales(codes, scales, rows, cols)
        _check(lib().fq_quantize_rows(self._h, x.data_ptr(), _TYPES[x.dtype], rows, cols, ldx, codes.data_ptr(), ldc, scales.data_ptr(),
                                      _stream_on(self.device)), "fq_quantize_rows")
        return codes, scales

    def _weights(self, w_codes, w_scales, y, m, k):
        n, kw, ldw = self._matrix(w_codes, "w_codes", _I8)
        self._dense(w_scales, "w_scales", _F32, (n,))
        my, ny, ldy = self._matrix(y, "y", _TYPES)
        if kw != k or my != m or ny != n:
            raise ValueError(f"shapes do not fit: {m} rows of {k}, weights {n} x {kw}, outputs {my} x {ny}")
        return n, ldw, ldy

    def fq_gemm_i8(self, x_codes: torch.Tensor, x_scales: torch.Tensor, w_codes: torch.Tensor, w_scales: torch.Tensor, y: torch.Tensor):
        """y[m][n] = x_scales[m] * w_scales[n] * sum_k x_codes[m][k] * w_codes[n][k]; y fp16, bf16 or fp32."""
        m, k, ldx = self._matrix(x_codes, "x_codes", _I8)
        self._dense(x_scales, "x_scales", _F32, (m,))
        n, ldw, ldy = self._weights(w_codes, w_scales, y, m, k)
        _check(lib().fq_gemm_i8(self._h, x_codes.data_ptr(), x_scales.data_ptr(), m, ldx, w_codes.data_ptr(), w_scales.data_ptr(), n, k, ldw,
                                y.data_ptr(), _TYPES[y.dtype], ldy, _stream_on(self.device)), "fq_gemm_i8")
        return y

    def fq_linear_i8(self, x: torch.Tensor, w_codes: torch.Tensor, w_scales: torch.Tensor, y: torch.Tensor,
                     codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None):
        """fq_quantize_rows of x, then fq_gemm_i8, in one call.  `codes` and `scales` are scratch; new where they are not given."""
        m, k, ldx = self._matrix(x, "x", _TYPES)
        n, ldw, ldy = self._weights(w_codes, w_scales, y, m, k)
        codes, ldc, scales = self._codes_and_scales(codes, scales, m, k)
        _check(lib().fq_linear_i8(self._h, x.data_ptr(), _TYPES[x.dtype], m, ldx, w_codes.data_ptr(), w_scales.data_ptr(), n, k, ldw,
                                  codes.data_ptr(), ldc, scales.data_ptr(), y.data_ptr(), _TYPES[y.dtype], ldy, _stream_on(self.device)),
               "fq_linear_i8")
        return y

    # -- what a model answers ------------------------------------------------------------------
    def fq_token_logprobs(self, logits: torch.Tensor, tokens: torch.Tensor, n_top: int = 0, temperature: float = 1.0, out=None):
        """Rows of logits and one token each -> (log probability fp32 [rows], entropy fp32 [rows], ids int32 [rows][n_top] of the most
        likely tokens, their log probabilities fp32 [rows][n_top]).  `out`: the four tensors to write to; new ones are parts of one
        allocation, which lives as long as any of them."""
        rows, vocab, ld = self._matrix(logits, "logits", _TYPES)
        self._dense(tokens, "tokens", _IDS, (rows,))
        if n_top < 0:
            raise ValueError("n_top is negative")
        if out is None:                                  # one allocation for all four
            all4 = torch.empty(rows * (2 + 2 * n_top), dtype=torch.float32, device=self.device)
            logprob, entropy = all4.as_strided((rows,), (1,), 0), all4.as_strided((rows,), (1,), rows)
            tops = all4.as_strided((rows, n_top), (n_top, 1), 2 * rows)
            ids = all4.view(torch.int32).as_strided((rows, n_top), (n_top, 1), (2 + n_top) * rows)
        else:
            logprob, entropy, ids, tops = out
            self._dense(logprob, "logprob", _F32, (rows,))
            self._dense(entropy, "entropy", _F32, (rows,))
            self._dense(ids, "ids", _I32, (rows, n_top))
            self._dense(tops, "tops", _F32, (rows, n_top))
        _check(lib().fq_token_logprobs(self._h, logits.data_ptr(), _TYPES[logits.dtype], rows, vocab, ld, tokens.data_ptr(),
                                       tokens.element_size(), temperature, logprob.data_ptr(), entropy.data_ptr(), n_top, ids.data_ptr(),
                                       tops.data_ptr(), _stream_on(self.device)), "fq_token_logprobs")
        return logprob, entropy, ids, tops

    def _slots(self, logits, ids, teacher, grad_loss, grad):
        rows, vocab, ld = self._matrix(logits, "logits", _TYPES)
        n_top = ids.shape[1] if ids.dim() == 2 else 0
        self._dense(ids, "ids", _IDS, (rows, n_top))
        self._dense(teacher, "teacher", _F32, (rows, n_top))
        if grad_loss is not None:
            self._dense(grad_loss, "grad_loss", _F32, (rows,))
            if grad is None:
                grad = torch.empty((rows, vocab), dtype=logits.dtype, device=self.device)
        elif grad is not None:
            raise ValueError("grad without grad_loss")
        ldg = 0
        if grad is not None:
            r, c, ldg = self._matrix(grad, "grad", (logits.dtype,))
            if r != rows or c != vocab:
                raise ValueError(f"grad: {rows} x {vocab} are needed, not {r} x {c}")
        return rows, vocab, ld, n_top, grad, ldg

    def fq_distill_topk(self, logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, temperature: float = 1.0,
                        grad_loss: Optional[torch.Tensor] = None, grad: Optional[torch.Tensor] = None):
        """KL of every row's distribution from its teacher's top logits -> (loss fp32 [rows], lse fp32 [rows][2], gradient or None).
        ids int32 / int64 [rows][n] and teacher fp32 [rows][n] are the teacher's tokens and logits, or log probabilities (an empty slot: a negative
        id, or a logit of -inf).  With `grad_loss` (fp32 [rows], upstream) the gradient with respect to the logits comes from the same call, into
        `grad` if that is given (it may be `logits`); without, fq_distill_topk_grad gives it later from `lse`."""
        rows, vocab, ld, n_top, grad, ldg = self._slots(logits, ids, teacher, grad_loss, grad)
        both = torch.empty(3 * rows, dtype=torch.float32, device=self.device)
        lse, loss = both.as_strided((rows, 2), (2, 1), 0), both.as_strided((rows,), (1,), 2 * rows)
        _check(lib().fq_distill_topk(self._h, logits.data_ptr(), _TYPES[logits.dtype], rows, vocab, ld, ids.data_ptr(), ids.element_size(),
                                     teacher.data_ptr(), n_top, temperature, None if grad_loss is None else grad_loss.data_ptr(),
                                     loss.data_ptr(), lse.data_ptr(), None if grad is None else grad.data_ptr(), ldg,
                                     _stream_on(self.device)), "fq_distill_topk")
        return loss, lse, grad

    def fq_distill_topk_grad(self, logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, lse: torch.Tensor, grad_loss: torch.Tensor,
                             temperature: float = 1.0, grad: Optional[torch.Tensor] = None):
        """The gradient of fq_distill_topk's losses, weighted with `grad_loss`, from the `lse` that it returned."""
        rows, vocab, ld, n_top, grad, ldg = self._slots(logits, ids, teacher, grad_loss, grad)
        self._dense(lse, "lse", _F32, (rows, 2))
        _check(lib().fq_distill_topk_grad(self._h, logits.data_ptr(), _TYPES[logits.dtype], rows, vocab, ld, ids.data_ptr(), ids.element_size(),
                                          teacher.data_ptr(), n_top, temperature, grad_loss.data_ptr(), lse.data_ptr(), grad.data_ptr(), ldg,
                                          _stream_on(self.device)), "fq_distill_topk_grad")
        return grad

    # -- between the linear layers of a block -----------------------------------------------------
    def _heads(self, t: torch.Tensor, name: str, types, tokens: Optional[int] = None, dim: Optional[int] = None) -> tuple:
        shape, st = t.shape, t.stride()
        if len(shape) == 3:
            n, heads, d = shape
            if t.dtype in types and t.get_device() == self._index and (st[2] == 1 or d < 2) and (tokens is None or (n == tokens and d == dim)):
                return t.data_ptr(), st[0], st[1], heads
        wanted = "[tokens][heads][values]" if tokens is None else f"[{tokens}][heads][{dim}]"
        raise ValueError(f"{name}: {wanted} of {', '.join(str(d) for d in types)} on {self.device} with dense values are needed, not "
                         f"{t.dtype} {tuple(shape)} with strides {st} on {t.device}")

    def _cache(self, k: torch.Tensor, v: torch.Tensor, types, dim: Optional[int] = None) -> tuple:
        shape, st, dt = k.shape, k.stride(), k.dtype
        if len(shape) == 4 and dt in types and k.get_device() == self._index and (st[3] == 1 or shape[3] < 2) and (
                k is v or (v.shape == shape and v.stride() == st and v.dtype is dt and v.get_device() == self._index)):
            blocks, block, heads, d = shape
            if dim is not None and d != dim:
                raise ValueError(f"caches: heads of {dim} are needed, not of {d}")
            return k.data_ptr(), v.data_ptr(), st[0], st[1], st[2], blocks, block, heads
        raise ValueError(f"caches: two of [blocks][block size][heads][values], {', '.join(str(d) for d in types)} on {self.device} with dense values and the "
                         f"same strides are needed, not {dt} {tuple(shape)} {st} on {k.device} and {v.dtype} {tuple(v.shape)} {v.stride()} on {v.device}")

    def _table(self, table: torch.Tensor, n_seqs: int):
        rows, cols, ld = self._matrix(table, "table", _I32)
        if rows != n_seqs:
            raise ValueError(f"table: a row for each of {n_seqs} sequences is needed, not {rows}")
        return cols, max(ld, cols)

    def fq_cache_step(self, lens: torch.Tensor, keep: torch.Tensor, new: torch.Tensor, table: torch.Tensor, free: torch.Tensor, count: torch.Tensor,
                      block_size: int, tokens: int, parents: Optional[torch.Tensor] = None, words: int = 1):
        """One step of a batch's paged caches: every sequence is cut back to its first keep[b] tokens, then grows by new[b].  lens [n] and table [n][blocks]
        (int32), the free list `free` and how many it holds, count [1], are updated in place.  `tokens`: rows of the batch (at least the new tokens).
        -> (starts int32 [n + 1], slots int64 [tokens], positions int32 [tokens], bits int64 [tokens][words] of drafted trees given by `parents`
        int32 [tokens], or None).  What does not fit is recorded for fq_status and changes nothing."""
        n = lens.shape[0] if lens.dim() == 1 else 0
        for t, name in ((lens, "lens"), (keep, "keep"), (new, "new")):
            self._dense(t, name, _I32, (n,))
        blocks, ld = self._table(table, n)
        self._dense(free, "free", _I32, (free.numel(),))
        self._dense(count, "count", _I32, (1,))
        if parents is not None:
            self._dense(parents, "parents", _I32, (tokens,))
        width = words if parents is not None else 0
        if tokens < 1 or width < 0:
            raise ValueError("tokens and words have to be positive")
        # one allocation: slots, bits, positions, starts
        wide = tokens * (1 + width)
        all4 = torch.empty(wide + (tokens + n + 2) // 2, dtype=torch.int64, device=self.device)
        narrow = all4.view(torch.int32)
        slots, positions, starts = all4.as_strided((tokens,), (1,), 0), narrow.as_strided((tokens,), (1,), 2 * wide), narrow.as_strided((n + 1,), (1,), 2 * wide + tokens)
        mask = all4.as_strided((tokens, width), (width, 1), tokens) if width else None
        at = all4.data_ptr()
        args = _STEP_ARGS.pack(lens.data_ptr(), keep.data_ptr(), new.data_ptr(), table.data_ptr(), ld, free.data_ptr(), count.data_ptr(),
                               0 if parents is None else parents.data_ptr(), at + 8 * wide + 4 * tokens, at, at + 8 * wide, at + 8 * tokens if width else 0, n,
                               blocks, block_size, free.numel(), tokens, width)
        _check(lib().fq_cache_step(self._h, args, _stream_on(self.device)), "fq_cache_step")
        return starts, slots, positions, mask

    def fq_cache_move(self, caches: Sequence[torch.Tensor], table: torch.Tensor, starts: torch.Tensor, lens: torch.Tensor, kept: torch.Tensor,
                      n_kept: torch.Tensor):
        """Moves the accepted branch of every sequence's new tokens together, in all `caches` (keys and values of all layers, [blocks][block size][heads][values] each, of
        one shape and type, none twice): new token kept[b][i] goes to the i-th cell behind what was cached before, i < n_kept[b].  kept int32 [n][most], rising.
        -> keep int32 [n], what fq_cache_step is to keep."""
        caches = list(caches)
        if not caches:
            raise ValueError("caches: none given")
        layout, count = self._cache(caches[0], caches[0], _TYPES), len(caches)
        shape, st, dt = caches[0].shape, caches[0].stride(), caches[0].dtype
        # (a tensor's properties for all of them at once: there are two caches a layer)
        alike = all(map(torch.Tensor.is_contiguous, caches)) if caches[0].is_contiguous() else list(map(torch.Tensor.stride, caches)).count(st) == count
        if not alike or list(map(torch.Tensor.size, caches)).count(shape) != count or \
                list(map(_dtype_of, caches)).count(dt) != count or list(map(torch.Tensor.get_device, caches)).count(self._index) != count:
            raise ValueError(f"caches: {dt} {tuple(shape)} with strides {st} on {self.device} are needed for all")
        pointers = array("Q", map(torch.Tensor.data_ptr, caches))
        n = lens.shape[0] if lens.dim() == 1 else 0
        self._dense(lens, "lens", _I32, (n,))
        self._dense(n_kept, "n_kept", _I32, (n,))
        self._dense(starts, "starts", _I32, (n + 1,))
        blocks, ld = self._table(table, n)
        rows, most, ld_kept = self._matrix(kept, "kept", _I32)
        if rows != n:
            raise ValueError(f"kept: a row for each of {n} sequences is needed, not {rows}")
        keep = torch.empty(n, dtype=torch.int32, device=self.device)
        args = _MOVE_ARGS.pack(pointers.buffer_info()[0], *layout, table.data_ptr(), ld, starts.data_ptr(), lens.data_ptr(), kept.data_ptr(), max(ld_kept, most),
                               n_kept.data_ptr(), keep.data_ptr(), count, _TYPES[dt], shape[3], n, blocks, most)
        _check(lib().fq_cache_move(self._h, args, _stream_on(self.device)), "fq_cache_move")
        return keep

    def _positions(self, positions, turns, tokens):
        self._dense(positions, "positions", _IDS, (tokens,))
        self._dense(turns, "turns", _I64, (turns.numel(),))
        return 2 * turns.numel()

    def fq_rotary(self, q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, turns: torch.Tensor, q_out: Optional[torch.Tensor] = None,
                  k_out: Optional[torch.Tensor] = None, interleaved: bool = False, inverse: bool = False, magnitude: float = 1.0):
        """Rotary positions of q and k, [tokens][heads][values] (any strides, values dense): the first 2 * len(turns) values of every head are turned in pairs by the
        angles of fq_rotary_table, values i and i + len(turns), or `interleaved` 2i and 2i + 1.  `inverse` turns back, which is the gradient.  Into q_out and
        k_out, which may be q and k; new ones where they are not given.  k may be None.  -> (q_out, k_out)"""
        tokens, _, dim = q.shape if q.dim() == 3 else (0, 0, 0)
        same = (q.dtype,)
        hq, hk, hk_out = self._heads(q, "q", _TYPES), _NO_HEADS, _NO_HEADS
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
        elif q_out.shape != q.shape:
            raise ValueError(f"q_out: {tuple(q.shape)} is needed, not {tuple(q_out.shape)}")
        hq_out = self._heads(q_out, "q_out", same)
        if k is not None:
            hk = self._heads(k, "k", same, tokens, dim)
            if k_out is None:
                k_out = torch.empty(k.shape, dtype=k.dtype, device=self.device)
            elif k_out.shape != k.shape:
                raise ValueError(f"k_out: {tuple(k.shape)} is needed, not {tuple(k_out.shape)}")
            hk_out = self._heads(k_out, "k_out", same)
        elif k_out is not None:
            raise ValueError("k_out without k")
        rot = self._positions(positions, turns, tokens)
        args = _ROTARY_ARGS.pack(*hq, *hk, *hq_out, *hk_out, positions.data_ptr(), turns.data_ptr(), 1 if k is None else 2, _TYPES[q.dtype], tokens, dim, rot,
                                 positions.element_size(), 1 if interleaved else 0, 1 if inverse else 0, magnitude)
        _check(lib().fq_rotary(self._h, args, _stream_on(self.device)), "fq_rotary")
        return q_out, k_out

    def fq_rotary_cache(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor, turns: torch.Tensor,
                        k_cache: torch.Tensor, v_cache: torch.Tensor, q_out: Optional[torch.Tensor] = None, interleaved: bool = False, magnitude: float = 1.0):
        """fq_rotary in a serving step: q goes to q_out (new if it is not given; may be q), k is turned and stored with v in the layer's caches
        [blocks][block size][heads][values], at slots int64 [tokens] (negative: not stored).  -> q_out"""
        tokens, _, dim = q.shape if q.dim() == 3 else (0, 0, 0)
        same = (q.dtype,)
        hq, hk, hv = self._heads(q, "q", _TYPES), self._heads(k, "k", same, tokens, dim), self._heads(v, "v", same, tokens, dim)
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
        elif q_out.shape != q.shape:
            raise ValueError(f"q_out: {tuple(q.shape)} is needed, not {tuple(q_out.shape)}")
        ho = self._heads(q_out, "q_out", same)
        cache = self._cache(k_cache, v_cache, same, dim)
        rot = self._positions(positions, turns, tokens)
        self._dense(slots, "slots", _I64, (tokens,))
        args = _ROTARY_CACHE_ARGS.pack(*hq, *ho, *hk, *hv, *cache, positions.data_ptr(), slots.data_ptr(), turns.data_ptr(), _TYPES[q.dtype], tokens, dim, rot,
                                       positions.element_size(), 1 if interleaved else 0, magnitude)
        _check(lib().fq_rotary_cache(self._h, args, _stream_on(self.device)), "fq_rotary_cache")
        return q_out

    def fq_tree_attention(self, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, starts: torch.Tensor,
                          mask: Optional[torch.Tensor] = None, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                          lse: Optional[torch.Tensor] = None, new: Optional[int] = None):
        """Attention of every sequence's new tokens over its paged cache, whose last cells they are: q [tokens][heads][values], rows starts[b] .. starts[b + 1] of
        sequence b, caches [blocks][block size][key heads][values], table int32 [n][blocks], lens int32 [n] (the new tokens counted).  A token sees what was cached
        before and, of the new tokens, those of its bits in `mask` int64 [tokens][words] (from fq_cache_step), or those up to itself.  `scale`:
        values^-1/2 if not given.  `new`: how many new tokens a sequence has, about (tokens / n if not given); rows are dealt for that many, so that many single
        tokens and a long prompt are faster in a call each.  Log-sum-exps go to `lse` fp32 [tokens][heads] if it is given.  10 to 39 MB of scratch are taken from
        torch's allocator for the call.  -> out, new if not given (not q); rows behind the last new token are left as they are."""
        tokens, heads, dim = q.shape if q.dim() == 3 else (0, 0, 0)
        hq = self._heads(q, "q", _HALF)
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
        elif out.shape != q.shape:
            raise ValueError(f"out: {tuple(q.shape)} is needed, not {tuple(out.shape)}")
        ho = self._heads(out, "out", (q.dtype,))
        cache = self._cache(k_cache, v_cache, (q.dtype,), dim)
        n = lens.shape[0] if lens.dim() == 1 else 0
        self._dense(lens, "lens", _I32, (n,))
        self._dense(starts, "starts", _I32, (n + 1,))
        blocks, ld = self._table(table, n)
        words = 0
        if mask is not None:
            words = mask.shape[1] if mask.dim() == 2 else 0
            self._dense(mask, "mask", _I64, (tokens, words))
        if lse is not None:
            self._dense(lse, "lse", _F32, (tokens, heads))
        if new is None:
            new = -(-tokens // max(n, 1))
        sizes = (n, tokens, heads, cache[7], dim, new)
        size = self._scratch.get(sizes)
        if size is None:
            if len(self._scratch) >= 1024:
                self._scratch.clear()
            size = self._scratch[sizes] = lib().fq_tree_attention_scratch(self._h, *sizes)
        scratch = torch.empty(max(size, 16), dtype=torch.uint8, device=self.device)
        args = _ATTENTION_ARGS.pack(*hq, *ho, *cache, starts.data_ptr(), lens.data_ptr(), table.data_ptr(), ld, 0 if mask is None else mask.data_ptr(),
                                    0 if lse is None else lse.data_ptr(), scratch.data_ptr(), size, _TYPES[q.dtype], dim, tokens, n, blocks, words, new,
                                    dim ** -0.5 if scale is None else scale)
        _check(lib().fq_tree_attention(self._h, args, _stream_on(self.device)), "fq_tree_attention")
        return out

"""Thin ctypes binding of libqadc.so: argument marshalling only.

Every function here has the name of the C entry point it forwards to (see
``include/qadc.h``).  PyTorch supplies device memory (``tensor.data_ptr()``) and
the stream; no step of the search path runs in Python or in PyTorch ops.  There
is no CPU fallback: if the library is missing or a call fails, an exception is
raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Sequence, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqadc.so")
_lib = None

PQ_OK, PQ_EINVAL, PQ_ENOMEM, PQ_EHIP = 0, -1, -2, -3
QPARAMS_BYTES = 24

EXPORTS = [
    "pq_index_create", "pq_index_destroy", "pq_code_size", "pq_table_len", "pq_workspace_bytes",
    "ivf_workspace_bytes", "ivf_sorted_workspace_bytes", "pq_compute_tables", "pq_quantize_tables", "pq_adc_scan_topk",
    "ivf_adc_scan_topk", "pq_search_workspace_bytes", "pq_search_topk",
    "pq_adc_scan_candidates", "pq_adc_rescan_candidates", "pq_select_topk", "pq_copy_bytes", "pq_last_error",
    "ivf_coarse_workspace_bytes", "ivf_coarse_search", "pq_encode", "pq_adc_scan_topk_static",
    "pq_set_option", "pq_get_option", "ivf_adc_scan_topk_tightening", "pq_lds_read_probe",
    "ivf_coarse_form", "pq_search_form", "pq_scan_form",
]
# include/qadc_vec.h: the operators on the vectors themselves
VEC_EXPORTS = [
    "vec_lookup", "vec_lookup_grad_workspace_bytes", "vec_lookup_grad", "vec_norm", "vec_norm_grad_workspace_bytes",
    "vec_norm_grad", "vec_quantize_blocks", "vec_matmul_blocks_workspace_bytes", "vec_matmul_blocks",
    "vec_dropout", "vec_adapter_workspace_bytes", "vec_adapter", "vec_adapter_grad_workspace_bytes", "vec_adapter_grad",
]
PQ_KEY_BOUND_UNKNOWN = 0xFFFFFFFF
(PQ_OPT_SCAN_BLOCKS, PQ_OPT_PILOT_CODES, PQ_OPT_PILOT_CODES_SINGLE, PQ_OPT_PILOT_BLOCKS, PQ_OPT_IVF_THREADS,
 PQ_OPT_SHARED_PASSES, PQ_OPT_COARSE_FILTER, PQ_OPT_IVF_SHARED_LISTS) = range(8)
PQ_SCAN_LOOKUP, PQ_SCAN_MATRIX = range(2)
PQ_COARSE_MATRIX, PQ_COARSE_FILTER, PQ_COARSE_HALF, PQ_COARSE_DIRECT = range(4)


class QadcError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libqadc error {code}: {msg}")
        self.code = code


def load() -> ctypes.CDLL:
    """Load libqadc.so, building it first only if it was never built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        from . import build as _build
        _build.build()
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    lib.pq_index_create.argtypes = [ctypes.POINTER(vp), i32, i32, vp, vp, vp, i32]
    lib.pq_index_create.restype = i32
    lib.pq_index_destroy.argtypes = [vp]
    lib.pq_index_destroy.restype = None
    lib.pq_code_size.argtypes = [vp]
    lib.pq_code_size.restype = sz
    lib.pq_table_len.argtypes = [vp]
    lib.pq_table_len.restype = sz
    lib.pq_workspace_bytes.argtypes = [vp, i32, i64, i32]
    lib.pq_workspace_bytes.restype = sz
    lib.ivf_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.ivf_workspace_bytes.restype = sz
    lib.ivf_sorted_workspace_bytes.argtypes = [vp, i32, i32, i32, i32]
    lib.ivf_sorted_workspace_bytes.restype = sz
    lib.pq_compute_tables.argtypes = [vp, vp, i32, vp, vp]
    lib.pq_compute_tables.restype = i32
    lib.pq_quantize_tables.argtypes = [vp, vp, i32, vp, i64, i32, i32, vp, vp, vp]
    lib.pq_quantize_tables.restype = i32
    lib.pq_adc_scan_topk.argtypes = [vp, vp, vp, i32, vp, i64, i32, vp, vp, vp, vp, sz, vp]
    lib.pq_adc_scan_topk.restype = i32
    lib.pq_adc_scan_topk_static.argtypes = [vp, vp, vp, i32, vp, i64, i32, vp, vp, vp, vp]
    lib.pq_adc_scan_topk_static.restype = i32
    lib.ivf_adc_scan_topk.argtypes = [vp, vp, i32, vp, vp, vp, vp, i32, vp, i32, i32, i32, vp, vp,
                                      vp, sz, vp]
    lib.ivf_adc_scan_topk.restype = i32
    lib.ivf_adc_scan_topk_tightening.argtypes = lib.ivf_adc_scan_topk.argtypes
    lib.ivf_adc_scan_topk_tightening.restype = i32
    lib.pq_lds_read_probe.argtypes = [i32, i32, vp, vp]
    lib.pq_lds_read_probe.restype = i32
    lib.pq_search_workspace_bytes.argtypes = [vp, i32, i64, i32]
    lib.pq_search_workspace_bytes.restype = sz
    lib.pq_search_topk.argtypes = [vp, vp, i32, vp, i64, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.pq_search_topk.restype = i32
    lib.pq_adc_scan_candidates.argtypes = [vp, vp, vp, i32, vp, i64, i32, vp, sz, vp]
    lib.pq_adc_scan_candidates.restype = i32
    lib.pq_adc_rescan_candidates.argtypes = [vp, vp, vp, i32, vp, i64, i32, vp, sz, vp]
    lib.pq_adc_rescan_candidates.restype = i32
    lib.pq_select_topk.argtypes = [vp, vp, vp, i32, vp, i64, i32, vp, vp, vp, vp, sz, vp]
    lib.pq_select_topk.restype = i32
    lib.pq_copy_bytes.argtypes = [vp, vp, sz, vp]
    lib.pq_copy_bytes.restype = i32
    lib.pq_set_option.argtypes = [i32, i64]
    lib.pq_set_option.restype = i32
    lib.pq_get_option.argtypes = [i32]
    lib.pq_get_option.restype = i64
    lib.pq_last_error.argtypes = []
    lib.pq_last_error.restype = ctypes.c_char_p
    lib.pq_encode.argtypes = [vp, vp, i64, vp, vp, vp, vp]
    lib.pq_encode.restype = i32
    lib.ivf_coarse_workspace_bytes.argtypes = [i32, i32]
    lib.ivf_coarse_workspace_bytes.restype = sz
    lib.ivf_coarse_search.argtypes = [vp, i32, vp, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.ivf_coarse_search.restype = i32
    lib.pq_search_form.argtypes = [vp, i32, i64, i32]
    lib.pq_search_form.restype = i32
    lib.pq_scan_form.argtypes = lib.pq_search_form.argtypes
    lib.pq_scan_form.restype = i32
    lib.ivf_coarse_form.argtypes = [i32, i32, i32, i32, sz]
    lib.ivf_coarse_form.restype = i32
    f32 = ctypes.c_float
    lib.vec_lookup.argtypes = [vp, i64, i32, i64, i32, vp, i32, i64, f32, vp, i64, i32, vp]
    lib.vec_lookup_grad_workspace_bytes.argtypes = [i64, i64, i32]
    lib.vec_lookup_grad.argtypes = [vp, i64, i32, i64, i32, vp, i32, f32, i32, vp, i64, i64, i32, vp, sz, vp]
    lib.vec_norm.argtypes = [vp, i64, vp, i64, i32, vp, i32, i64, i32, f32, vp, i64, vp, i64, vp, i64, i32, vp, i64, i32, vp]
    lib.vec_norm_grad_workspace_bytes.argtypes = [i64, i32]
    lib.vec_norm_grad.argtypes = [vp, i64, vp, i64, vp, i64, i32, vp, i32, i64, i32, f32, vp, i64, vp, vp, sz, vp]
    lib.vec_quantize_blocks.argtypes = [vp, i64, i32, i64, i64, i32, vp, i64, i32, vp, i64, i32, vp]
    lib.vec_matmul_blocks_workspace_bytes.argtypes = [i64, i64, i64]
    lib.vec_matmul_blocks.argtypes = [vp, i64, i32, vp, i64, vp, i64, i32, vp, i64, i32, i64, i64, i64, vp, i64, i32, vp, sz, vp]
    f64, u32 = ctypes.c_double, ctypes.c_uint32
    lib.vec_dropout.argtypes = [vp, i64, vp, i64, i32, i64, i64, f64, vp, u32, vp, i64, vp]
    lib.vec_adapter_workspace_bytes.argtypes = lib.vec_adapter_grad_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i32]
    factors = [vp, i64, i64, vp, i64, i64, i32, i32, i32, vp, vp, i32, i64, i32, i32]
    lib.vec_adapter.argtypes = [vp, i64, *factors, vp, i64, vp, i64, i32, f64, vp, u32, vp, vp, sz, vp]
    lib.vec_adapter_grad.argtypes = [vp, i64, vp, i64, vp, *factors, vp, i64, vp, i64, f64, vp, u32, i32, vp, i64, i64, vp, i64, i64, i32, vp, sz, vp]
    for name in VEC_EXPORTS:
        getattr(lib, name).restype = sz if name.endswith("_bytes") else i32
    _lib = lib
    return lib


def _check(rc: int) -> None:
    if rc != PQ_OK:
        raise QadcError(rc, load().pq_last_error().decode("utf-8", "replace"))


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous(), "libqadc needs contiguous tensors"
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


def _dev(t: torch.Tensor, dtype) -> None:
    assert t.is_cuda and t.dtype == dtype, (t.device, t.dtype, dtype)


class PqIndex:
    """Owner of a ``pq_index_t*`` (pq_index_create / pq_index_destroy)."""

    def __init__(self, d: int, nbits: Sequence[int], dsub: Sequence[int], codebooks: torch.Tensor,
                 acc_bits: int):
        lib = load()
        _dev(codebooks, torch.float32)
        self.codebooks = codebooks.contiguous()  # the handle keeps this pointer
        nb = (ctypes.c_int32 * len(nbits))(*nbits)
        ds = (ctypes.c_int32 * len(dsub))(*dsub)
        h = ctypes.c_void_p()
        with torch.cuda.device(codebooks.device):
            _check(lib.pq_index_create(ctypes.byref(h), d, len(nbits), ctypes.cast(nb, ctypes.c_void_p),
                                       ctypes.cast(ds, ctypes.c_void_p), self.codebooks.data_ptr(),
                                       acc_bits))
        self.handle = h
        self.d, self.m, self.acc_bits = d, len(nbits), acc_bits
        self.nbits, self.dsub = list(nbits), list(dsub)
        self.code_size = int(lib.pq_code_size(h))
        self.table_len = int(lib.pq_table_len(h))
        self.q_max = (1 << acc_bits) - 1
        self.qdtype = torch.uint8 if acc_bits == 8 else torch.uint16
        self.device = codebooks.device

    def close(self) -> None:
        if getattr(self, "handle", None):
            load().pq_index_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def pq_workspace_bytes(idx: PqIndex, nq: int, n: int, R: int) -> int:
    return int(load().pq_workspace_bytes(idx.handle, nq, n, R))


def ivf_workspace_bytes(idx: PqIndex, nq: int, nprobe: int, R: int) -> int:
    return int(load().ivf_workspace_bytes(idx.handle, nq, nprobe, R))


def ivf_sorted_workspace_bytes(idx: PqIndex, nq: int, nprobe: int, R: int, K: int) -> int:
    return int(load().ivf_sorted_workspace_bytes(idx.handle, nq, nprobe, R, K))


def pq_compute_tables(idx: PqIndex, queries: torch.Tensor, tables: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    _dev(queries, torch.float32)
    nq = queries.shape[0]
    if tables is None:
        tables = torch.empty((nq, idx.table_len), dtype=torch.float32, device=queries.device)
    _check(load().pq_compute_tables(idx.handle, _ptr(queries), nq, _ptr(tables), _stream(stream)))
    return tables


def pq_quantize_tables(idx: PqIndex, tables: torch.Tensor, codes: torch.Tensor, t: int, R: int,
                       qtables: Optional[torch.Tensor] = None,
                       qparams: Optional[torch.Tensor] = None, stream=None
                       ) -> Tuple[torch.Tensor, torch.Tensor]:
    """qparams is a [nq, 24] uint8 tensor holding pq_qparams_t records."""
    _dev(tables, torch.float32)
    _dev(codes, torch.uint8)
    nq = tables.shape[0]
    if qtables is None:
        qtables = torch.empty((nq, idx.table_len), dtype=idx.qdtype, device=tables.device)
    if qparams is None:
        qparams = torch.empty((nq, QPARAMS_BYTES), dtype=torch.uint8, device=tables.device)
    _check(load().pq_quantize_tables(idx.handle, _ptr(tables), nq, _ptr(codes), codes.shape[0], t, R,
                                     _ptr(qtables), _ptr(qparams), _stream(stream)))
    return qtables, qparams


def pq_adc_scan_topk(idx: PqIndex, qtables: torch.Tensor, qparams: torch.Tensor,
                     codes: torch.Tensor, R: int, workspace: Optional[torch.Tensor] = None,
                     out=None, stream=None):
    _dev(codes, torch.uint8)
    nq, n = qtables.shape[0], codes.shape[0]
    dev = codes.device
    if workspace is None:
        workspace = torch.empty(pq_workspace_bytes(idx, nq, n, R), dtype=torch.uint8, device=dev)
    if out is None:
        out = (torch.empty((nq, R), dtype=torch.int32, device=dev),
               torch.empty((nq, R), dtype=torch.uint16, device=dev),
               torch.empty((nq, R), dtype=torch.float32, device=dev))
    ids, keys, dist = out
    _check(load().pq_adc_scan_topk(idx.handle, _ptr(qtables), _ptr(qparams), nq, _ptr(codes), n, R,
                                   _ptr(ids), _ptr(keys), _ptr(dist), _ptr(workspace),
                                   workspace.numel(), _stream(stream)))
    return ids, keys, dist


def pq_adc_scan_topk_static(idx: PqIndex, qtables: torch.Tensor, qparams: torch.Tensor,
                            codes: torch.Tensor, R: int, out, stream=None):
    """The caller passes inputs and outputs; the library's own scratch array is the workspace."""
    _dev(codes, torch.uint8)
    ids, keys, dist = out
    _check(load().pq_adc_scan_topk_static(idx.handle, _ptr(qtables), _ptr(qparams), qtables.shape[0],
                                          _ptr(codes), codes.shape[0], R, _ptr(ids), _ptr(keys),
                                          _ptr(dist), _stream(stream)))
    return ids, keys, dist


def pq_search_workspace_bytes(idx: PqIndex, nq: int, n: int, R: int) -> int:
    return int(load().pq_search_workspace_bytes(idx.handle, nq, n, R))


def pq_search_form(idx: PqIndex, nq: int, n: int, R: int) -> int:
    """PQ_SCAN_*: the form that pq_search_topk takes for such a call."""
    form = load().pq_search_form(idx.handle, nq, n, R)
    if form < 0:
        _check(form)
    return form


def pq_scan_form(idx: PqIndex, nq: int, n: int, R: int) -> int:
    """PQ_SCAN_*: the form that pq_adc_scan_topk takes for such a call."""
    form = load().pq_scan_form(idx.handle, nq, n, R)
    if form < 0:
        _check(form)
    return form


def pq_search_topk(idx: PqIndex, queries: torch.Tensor, codes: torch.Tensor, t: int, R: int,
                   workspace: Optional[torch.Tensor] = None, out=None, stream=None):
    _dev(queries, torch.float32)
    _dev(codes, torch.uint8)
    nq, n = queries.shape[0], codes.shape[0]
    dev = codes.device
    if workspace is None:
        workspace = torch.empty(pq_search_workspace_bytes(idx, nq, n, R), dtype=torch.uint8,
                                device=dev)
    if out is None:
        out = (torch.empty((nq, R), dtype=torch.int32, device=dev),
               torch.empty((nq, R), dtype=torch.uint16, device=dev),
               torch.empty((nq, R), dtype=torch.float32, device=dev))
    ids, keys, dist = out
    _check(load().pq_search_topk(idx.handle, _ptr(queries), nq, _ptr(codes), n, t, R, _ptr(ids),
                                 _ptr(keys), _ptr(dist), _ptr(workspace), workspace.numel(),
                                 _stream(stream)))
    return ids, keys, dist


def ivf_adc_scan_topk(idx: PqIndex, coarse: torch.Tensor, list_offsets: torch.Tensor,
                      list_codes: torch.Tensor, list_ids: torch.Tensor, queries: torch.Tensor,
                      probe_ids: torch.Tensor, t: int, R: int,
                      workspace: Optional[torch.Tensor] = None, out=None, stream=None):
    _dev(coarse, torch.float32)
    _dev(list_offsets, torch.int64)
    _dev(list_codes, torch.uint8)
    _dev(list_ids, torch.int32)
    _dev(queries, torch.float32)
    _dev(probe_ids, torch.int32)
    nq, nprobe = probe_ids.shape
    dev = queries.device
    if workspace is None:
        workspace = torch.empty(ivf_sorted_workspace_bytes(idx, nq, nprobe, R, coarse.shape[0]),
                                dtype=torch.uint8, device=dev)
    if out is None:
        out = (torch.empty((nq, R), dtype=torch.int32, device=dev),
               torch.empty((nq, R), dtype=torch.float32, device=dev))
    ids, dist = out
    _check(load().ivf_adc_scan_topk(idx.handle, _ptr(coarse), coarse.shape[0], _ptr(list_offsets),
                                    _ptr(list_codes), _ptr(list_ids), _ptr(queries), nq,
                                    _ptr(probe_ids), nprobe, t, R, _ptr(ids), _ptr(dist),
                                    _ptr(workspace), workspace.numel(), _stream(stream)))
    return ids, dist


def ivf_adc_scan_topk_tightening(idx: PqIndex, coarse: torch.Tensor, list_offsets: torch.Tensor,
                                 list_codes: torch.Tensor, list_ids: torch.Tensor, queries: torch.Tensor,
                                 probe_ids: torch.Tensor, t: int, R: int,
                                 workspace: Optional[torch.Tensor] = None, out=None, stream=None):
    _dev(coarse, torch.float32)
    _dev(list_offsets, torch.int64)
    _dev(list_codes, torch.uint8)
    _dev(list_ids, torch.int32)
    _dev(queries, torch.float32)
    _dev(probe_ids, torch.int32)
    nq, nprobe = probe_ids.shape
    dev = queries.device
    if workspace is None:
        workspace = torch.empty(ivf_workspace_bytes(idx, nq, nprobe, R), dtype=torch.uint8, device=dev)
    if out is None:
        out = (torch.empty((nq, R), dtype=torch.int32, device=dev),
               torch.empty((nq, R), dtype=torch.float32, device=dev))
    ids, dist = out
    _check(load().ivf_adc_scan_topk_tightening(idx.handle, _ptr(coarse), coarse.shape[0], _ptr(list_offsets),
                                               _ptr(list_codes), _ptr(list_ids), _ptr(queries), nq,
                                               _ptr(probe_ids), nprobe, t, R, _ptr(ids), _ptr(dist),
                                               _ptr(workspace), workspace.numel(), _stream(stream)))
    return ids, dist


def pq_adc_scan_candidates(idx: PqIndex, qtables: torch.Tensor, qparams: torch.Tensor,
                           codes: torch.Tensor, R: int, workspace: torch.Tensor, stream=None) -> None:
    _dev(codes, torch.uint8)
    _check(load().pq_adc_scan_candidates(idx.handle, _ptr(qtables), _ptr(qparams), qtables.shape[0],
                                         _ptr(codes), codes.shape[0], R, _ptr(workspace),
                                         workspace.numel(), _stream(stream)))


def pq_adc_rescan_candidates(idx: PqIndex, qtables: torch.Tensor, qparams: torch.Tensor,
                             codes: torch.Tensor, R: int, workspace: torch.Tensor, stream=None) -> None:
    _dev(codes, torch.uint8)
    _check(load().pq_adc_rescan_candidates(idx.handle, _ptr(qtables), _ptr(qparams),
                                           qtables.shape[0], _ptr(codes), codes.shape[0], R,
                                           _ptr(workspace), workspace.numel(), _stream(stream)))


def pq_select_topk(idx: PqIndex, qtables: torch.Tensor, qparams: torch.Tensor, codes: torch.Tensor,
                   R: int, workspace: torch.Tensor, out=None, stream=None):
    _dev(codes, torch.uint8)
    nq, dev = qtables.shape[0], codes.device
    if out is None:
        out = (torch.empty((nq, R), dtype=torch.int32, device=dev),
               torch.empty((nq, R), dtype=torch.uint16, device=dev),
               torch.empty((nq, R), dtype=torch.float32, device=dev))
    ids, keys, dist = out
    _check(load().pq_select_topk(idx.handle, _ptr(qtables), _ptr(qparams), nq, _ptr(codes),
                                 codes.shape[0], R, _ptr(ids), _ptr(keys), _ptr(dist),
                                 _ptr(workspace), workspace.numel(), _stream(stream)))
    return ids, keys, dist


def pq_copy_bytes(dst: torch.Tensor, src: torch.Tensor, stream=None) -> None:
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == nbytes
    _check(load().pq_copy_bytes(_ptr(dst), _ptr(src), nbytes, _stream(stream)))


PQ_LDS_UNIFORM, PQ_LDS_LINEAR, PQ_LDS_RANDOM_2K, PQ_LDS_RANDOM_128 = range(4)
PQ_LDS_PROBE_BLOCKS = 2048


def pq_lds_read_probe(pattern: int, iters: int, sink: torch.Tensor, stream=None) -> int:
    """Launches the probe; returns the number of 8-byte lane reads it performs."""
    _dev(sink, torch.int32)
    _check(load().pq_lds_read_probe(pattern, iters, _ptr(sink), _stream(stream)))
    return PQ_LDS_PROBE_BLOCKS * 256 * 8 * iters


def pq_set_option(option: int, value: int) -> None:
    _check(load().pq_set_option(option, value))


def pq_get_option(option: int) -> int:
    return int(load().pq_get_option(option))


def unpack_qparams(qparams: torch.Tensor):
    """[nq,24] uint8 -> dict of numpy arrays (d_min, delta, d_max, key_bound)."""
    import numpy as np
    raw = qparams.detach().cpu().numpy()
    rec = np.dtype([("d_min", "<f8"), ("delta", "<f8"), ("d_max", "<f4"), ("key_bound", "<u4")])
    return raw.view(rec).reshape(-1)


def ivf_coarse_workspace_bytes(nq: int, K: int) -> int:
    return int(load().ivf_coarse_workspace_bytes(nq, K))


def ivf_coarse_form(nq: int, K: int, d: int, nprobe: int, workspace_bytes: Optional[int] = None) -> int:
    """PQ_COARSE_*: the form such a call takes (with the workspace that ivf_coarse_workspace_bytes names)."""
    if workspace_bytes is None:
        workspace_bytes = ivf_coarse_workspace_bytes(nq, K)
    form = load().ivf_coarse_form(nq, K, d, nprobe, workspace_bytes)
    if form < 0:
        _check(form)
    return form


def ivf_coarse_search(queries: torch.Tensor, centroids: torch.Tensor, nprobe: int,
                      workspace: Optional[torch.Tensor] = None, out=None, want_scores: bool = True,
                      stream=None):
    """Returns (probe_ids [nq, nprobe] int32, probe_scores [nq, nprobe] float32 or None)."""
    _dev(queries, torch.float32)
    _dev(centroids, torch.float32)
    nq, d = queries.shape
    K = centroids.shape[0]
    assert centroids.shape[1] == d
    dev = queries.device
    if workspace is None:
        workspace = torch.empty(ivf_coarse_workspace_bytes(nq, K), dtype=torch.uint8, device=dev)
    if out is None:
        out = (torch.empty((nq, nprobe), dtype=torch.int32, device=dev),
               torch.empty((nq, nprobe), dtype=torch.float32, device=dev) if want_scores else None)
    ids, sc = out
    _check(load().ivf_coarse_search(_ptr(queries), nq, _ptr(centroids), K, d, nprobe, _ptr(ids),
                                    _ptr(sc) if sc is not None else None, _ptr(workspace),
                                    workspace.numel(), _stream(stream)))
    return ids, sc


def pq_encode(idx: PqIndex, vectors: torch.Tensor, shift_rows: Optional[torch.Tensor] = None,
              shift_ids: Optional[torch.Tensor] = None, codes: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """Packed codes [n, code_size] uint8 of vectors [n, d] (minus shift_rows[shift_ids], if given)."""
    _dev(vectors, torch.float32)
    if shift_rows is not None:
        _dev(shift_rows, torch.float32)
        _dev(shift_ids, torch.int32)
    n = vectors.shape[0]
    if codes is None:
        codes = torch.empty((n, idx.code_size), dtype=torch.uint8, device=vectors.device)
    _check(load().pq_encode(idx.handle, _ptr(vectors), n, _ptr(shift_rows), _ptr(shift_ids),
                            _ptr(codes), _stream(stream)))
    return codes


# ------------------------------------------- operators on the vectors (qadc_vec.h) --
# Matrices are two-dimensional, their last stride 1; rows may lie any distance apart.  Outputs that are not given, and workspaces,
# are allocated for the stream that the call runs on.  Nothing is recorded for autograd: results require no gradient whatever the inputs do, and the
# gradients are calls of their own (vec_lookup_grad, vec_norm_grad, and vec_matmul_blocks of transposed blocks).
VEC_F32, VEC_BF16, VEC_F16, VEC_E4M3, VEC_E5M2, VEC_E8M0 = range(6)
VEC_BLOCK = 128
_VEC_TYPE = {torch.float32: VEC_F32, torch.bfloat16: VEC_BF16, torch.float16: VEC_F16, torch.float8_e4m3fn: VEC_E4M3,
             torch.float8_e5m2: VEC_E5M2, torch.float8_e8m0fnu: VEC_E8M0}


def _refuse(name: str, msg: str):
    raise QadcError(PQ_EINVAL, f"{name}: {msg}")


@functools.lru_cache(maxsize=1024)
def _vec_bytes(name: str, *sizes) -> int:
    """A workspace's bytes, which sizes alone decide."""
    return getattr(load(), name)(*sizes)


class _Call:
    """The device and the stream of a call, for its checks, allocations and launch.  (A call of a few microseconds on the GPU waits
    for what is done here, so messages are only put together for a refusal, and outputs made here are not looked over.)"""
    __slots__ = ("name", "device", "index", "stream", "raw")

    def __init__(self, name: str, first: torch.Tensor, stream):
        if not first.is_cuda:
            _refuse(name, f"tensors of the GPU, got {first.device}")
        self.name, self.index, self.stream = name, first.get_device(), None
        if stream is not None and stream.device.index != self.index:
            _refuse(name, f"a stream of {stream.device} for tensors of {first.device}")
        self.raw = torch._C._cuda_getCurrentRawStream(self.index)
        self.device = first.device
        if (stream is not None and stream.cuda_stream != self.raw) or torch._C._cuda_getDevice() != self.index:
            self.stream = stream if stream is not None else torch.cuda.current_stream(self.index)  # (entered around allocations and the launch)
            self.raw = self.stream.cuda_stream

    def empty(self, dtype, *shape) -> torch.Tensor:
        if self.stream is not None:
            with torch.cuda.stream(self.stream):
                return torch.empty(*shape, dtype=dtype, device=self.device)
        return torch.empty(*shape, dtype=dtype, device=self.device)

    def rows(self, what: str, t: torch.Tensor, n: int, d: int, dtype):
        """Address of a matrix [n, d] and the distance of its rows, checked."""
        shape, stride = t.shape, t.stride()
        if len(shape) == 2 and shape[0] == n and shape[1] == d and t.dtype == dtype and t.get_device() == self.index:
            ld = stride[0] if n > 1 else (d or 1)
            if ld >= d and (stride[1] == 1 or d <= 1):
                return t.data_ptr(), ld or 1
            _refuse(self.name, f"{what}'s rows of {d} are {ld} apart, the values of a row {stride[1]}")
        if t.get_device() != self.index:
            _refuse(self.name, f"{what} is on {t.device}, not {self.device}")
        if t.dtype != dtype:
            _refuse(self.name, f"{what} is {t.dtype}, not {dtype}")
        _refuse(self.name, f"{what} of shape {tuple(shape)}, not {(n, d)}")

    def first_rows(self, what: str, t: torch.Tensor):
        shape = t.shape
        if len(shape) != 2:
            _refuse(self.name, f"{what} of shape {tuple(shape)}, not a matrix")
        n, d = shape
        if t.is_contiguous():
            return n, d, t.data_ptr(), d or 1
        return (n, d, *self.rows(what, t, n, d, t.dtype))

    def columns(self, d: int) -> None:
        """(ctypes would pass the low 32 bits of a C int)"""
        if d > 0x7FFFFFFF:
            _refuse(self.name, f"d={d}")

    def vector(self, what: str, t: torch.Tensor, n: Optional[int] = None, dtype=None) -> int:
        if t.get_device() != self.index or (dtype is not None and t.dtype != dtype) or not t.is_contiguous() or (
                n is not None and (t.dim() != 1 or t.numel() != n)):
            _refuse(self.name, f"{what}: {t.dtype} of shape {tuple(t.shape)}, strides {t.stride()}, on {t.device}")
        return t.data_ptr()

    def workspace(self, t: Optional[torch.Tensor], nbytes: int):
        """Address, bytes, and the tensor, to be kept until the launch."""
        if t is None:
            if nbytes == 0:
                return None, 0, None
            t = self.empty(torch.uint8, nbytes)
            return t.data_ptr(), nbytes, t
        return self.vector("workspace", t), t.numel() * t.element_size(), t

    def matrices(self, what: str, t: torch.Tensor, count: int, n: int, d: int, dtype):
        """Address of [count, n, d], the distances of its rows and of its matrices, checked."""
        if t.shape != (count, n, d) or t.dtype != dtype or t.get_device() != self.index:
            _refuse(self.name, f"{what}: {t.dtype} of shape {tuple(t.shape)} on {t.device}, not {dtype} of {(count, n, d)} on {self.device}")
        if t.is_contiguous():
            return t.data_ptr(), d, n * d
        stride = t.stride()
        ld = stride[1] if n > 1 else d
        if ld < d or (stride[2] != 1 and d > 1):
            _refuse(self.name, f"{what}'s rows of {d} are {ld} apart, the values of a row {stride[2]}")
        return t.data_ptr(), ld, stride[0] if count > 1 else 0

    def mask(self, p: float, state: Optional[torch.Tensor], layer: int):
        """Dropout's arguments: the rate, the address of seed and step, the layer."""
        if not 0 <= layer <= 0xFFFFFFFF:
            _refuse(self.name, f"layer={layer}")
        if p == 0 or state is None:
            return p, None, layer
        if state.numel() != 2 or (state.dtype != torch.int64 and state.dtype != torch.uint64):
            _refuse(self.name, f"state of {state.dtype}, shape {tuple(state.shape)}: seed and step, int64")
        return p, self.vector("state", state), layer

    def type(self, what: str, dtype) -> int:
        t = _VEC_TYPE.get(dtype)
        if t is None:
            _refuse(self.name, f"{what}: no operator takes {dtype}")
        return t

    def ids(self, t: torch.Tensor):
        size = 8 if t.dtype == torch.int64 else 4
        if size == 4 and t.dtype != torch.int32:
            _refuse(self.name, f"ids are int32 or int64, got {t.dtype}")
        if t.get_device() != self.index or not t.is_contiguous():
            self.vector("ids", t)  # (refuses)
        return t.data_ptr(), size

    def out_type(self, out: Optional[torch.Tensor], dtype, default):
        """The type of a result that may be given, named, or left to the default."""
        if out is None:
            return dtype or default
        if dtype is not None and out.dtype != dtype:
            _refuse(self.name, f"out is {out.dtype}, not {dtype}")
        return out.dtype

    def launch(self, fn, *args) -> None:
        if self.stream is None:
            rc = fn(*args, self.raw)
        else:
            with torch.cuda.device(self.index):
                rc = fn(*args, self.raw)
        if rc != PQ_OK:
            _check(rc)


def vec_lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, dtype: Optional[torch.dtype] = None,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """scale * table[ids] as [*ids.shape, d]; zeros where an id is outside the table (a search pads with -1)."""
    call = _Call("vec_lookup", table, stream)
    rows, d, ptr, ld = call.first_rows("table", table)
    call.columns(d)
    idp, id_bytes = call.ids(ids)
    n = ids.numel()
    to = call.out_type(out, dtype, table.dtype)
    if out is None:
        out = call.empty(to, *ids.shape, d)
        optr, old = out.data_ptr(), d
    else:
        optr, old = call.rows("out", out, n, d, to)
    call.launch((_lib or load()).vec_lookup, ptr, rows, d, ld, call.type("table", table.dtype), idp, id_bytes, n, scale, optr, old,
                call.type("out", to))
    return out


def vec_lookup_grad_workspace_bytes(n: int, rows: int, d: int) -> int:
    return int(load().vec_lookup_grad_workspace_bytes(n, rows, d))


def vec_lookup_grad(grad: torch.Tensor, ids: torch.Tensor, rows: int, scale: float = 1.0, dtype: Optional[torch.dtype] = None,
                    out: Optional[torch.Tensor] = None, accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """Gradient [rows, d] of vec_lookup's table from the gradient [n, d] (or [*ids.shape, d]) of its result; with `accumulate` it
    is added to `out`."""
    call = _Call("vec_lookup_grad", grad, stream)
    if grad.dim() != 2:
        if not grad.is_contiguous() or grad.dim() == 0:
            _refuse(call.name, "grad of other than two dimensions is contiguous")
        grad = grad.view(-1, grad.shape[-1])
    n, d = ids.numel(), grad.shape[1]
    call.columns(d)
    ptr, ld = call.rows("grad", grad, n, d, grad.dtype)
    idp, id_bytes = call.ids(ids)
    if accumulate and out is None:
        _refuse(call.name, "accumulate needs an out to add to")
    to = call.out_type(out, dtype, grad.dtype)
    if out is None:
        out = call.empty(to, rows, d)
        optr, old = out.data_ptr(), d
    else:
        optr, old = call.rows("out", out, rows, d, to)
    lib = _lib or load()
    wptr, wbytes, keep = call.workspace(workspace, _vec_bytes("vec_lookup_grad_workspace_bytes", n, rows, d))
    call.launch(lib.vec_lookup_grad, ptr, n, d, ld, call.type("grad", grad.dtype), idp, id_bytes, scale, int(accumulate), optr, rows,
                old, call.type("out", to), wptr, wbytes)
    return out


def _blocks_out(call: _Call, n: int, d: int, quant, scale_dtype, out):
    """8-bit values and scales with their addresses and distances: those given, or new ones whose rows start at multiples of 16 bytes."""
    if scale_dtype != torch.float8_e8m0fnu and scale_dtype != torch.float32:
        _refuse(call.name, f"scales of {scale_dtype}")
    if quant != torch.float8_e4m3fn and quant != torch.float8_e5m2:
        _refuse(call.name, f"8-bit values of {quant}")
    nb = -(-d // VEC_BLOCK)
    if out is not None:
        q, scales = out
        return (q, scales, *call.rows("q", q, n, d, quant), *call.rows("scales", scales, n, nb, scale_dtype))
    ld = -(-d // 16) * 16
    q, scales = call.empty(quant, n, ld), call.empty(scale_dtype, n, nb)
    return (q if ld == d else q[:, :d]), scales, q.data_ptr(), ld or 1, scales.data_ptr(), nb or 1


def vec_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
             want_y: bool = True, quant: Optional[torch.dtype] = None, scale_dtype: Optional[torch.dtype] = torch.float8_e8m0fnu,
             out=None, stream=None):
    """Root-mean-square norm of x + residual.  Returns (y, h, q, scales): y where wanted, h = x + residual where there is one,
    8-bit values and scales of y where `quant` names their type; else None.  `out`: the same four, to be written (h may be x or
    residual)."""
    call = _Call("vec_norm", x, stream)
    n, d, xp, ldx = call.first_rows("x", x)
    call.columns(d)
    t = x.dtype
    rp = hp = yp = qp = sp = None
    ldr = ldh = ldy = ldq = lds = 0
    if residual is not None:
        rp, ldr = call.rows("residual", residual, n, d, t)
    wp = call.vector("weight", weight, d)
    y = h = q = scales = None
    if out is None:
        if want_y:
            y = call.empty(t, n, d)
            yp, ldy = y.data_ptr(), d
        if residual is not None:
            h = call.empty(t, n, d)
            hp, ldh = h.data_ptr(), d
        if quant is not None:
            q, scales, qp, ldq, sp, lds = _blocks_out(call, n, d, quant, scale_dtype, None)
    else:
        y, h, q, scales = out
        if y is not None:
            yp, ldy = call.rows("y", y, n, d, t)
        if h is not None:
            hp, ldh = call.rows("h", h, n, d, t)
        if q is not None:
            quant, scale_dtype = q.dtype, scales.dtype
            q, scales, qp, ldq, sp, lds = _blocks_out(call, n, d, quant, scale_dtype, (q, scales))
    call.launch((_lib or load()).vec_norm, xp, ldx, rp, ldr, call.type("x", t), wp, call.type("weight", weight.dtype), n, d, eps, hp, ldh,
                yp, ldy, qp, ldq, _VEC_TYPE.get(quant, VEC_E4M3), sp, lds, _VEC_TYPE.get(scale_dtype, VEC_E8M0))
    return y, h, q, scales


def vec_norm_grad_workspace_bytes(n: int, d: int) -> int:
    return int(load().vec_norm_grad_workspace_bytes(n, d))


def vec_norm_grad(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, dh: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  out=None, workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, dweight) of vec_norm: h is its second result (x without a residual), dh the gradient that reaches h past the norm.
    `out`: the same two, to be written (dx may be dy or dh; dweight is float32)."""
    call = _Call("vec_norm_grad", dy, stream)
    n, d, yp, ldy = call.first_rows("dy", dy)
    call.columns(d)
    t = dy.dtype
    hp, ldh = call.rows("h", h, n, d, t)
    ep, lde = call.rows("dh", dh, n, d, t) if dh is not None else (None, 0)
    wp = call.vector("weight", weight, d)
    if out is None:
        dx, dweight = call.empty(t, n, d), call.empty(torch.float32, d)
        xp, ldx, dwp = dx.data_ptr(), d, dweight.data_ptr()
    else:
        dx, dweight = out
        xp, ldx = call.rows("dx", dx, n, d, t)
        dwp = call.vector("dweight", dweight, d, torch.float32)
    lib = _lib or load()
    wsp, wbytes, keep = call.workspace(workspace, _vec_bytes("vec_norm_grad_workspace_bytes", n, d))
    call.launch(lib.vec_norm_grad, yp, ldy, hp, ldh, ep, lde, call.type("dy", t), wp, call.type("weight", weight.dtype), n, d, eps, xp, ldx,
                dwp, wsp, wbytes)
    return dx, dweight


def vec_quantize_blocks(x: torch.Tensor, dtype: torch.dtype = torch.float8_e4m3fn, scale_dtype: torch.dtype = torch.float8_e8m0fnu,
                        transposed: bool = False, out=None, stream=None):
    """(q, scales): x in 8 bits with a scale for each 128 values of a row, or, transposed, of a column (q is then x's transpose)."""
    call = _Call("vec_quantize_blocks", x, stream)
    n, d, xp, ldx = call.first_rows("x", x)
    q, scales, qp, ldq, sp, lds = _blocks_out(call, d if transposed else n, n if transposed else d, dtype, scale_dtype, out)
    call.launch((_lib or load()).vec_quantize_blocks, xp, ldx, call.type("x", x.dtype), n, d, int(transposed), qp, ldq, _VEC_TYPE[dtype], sp,
                lds, _VEC_TYPE[scale_dtype])
    return q, scales


def vec_matmul_blocks_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(load().vec_matmul_blocks_workspace_bytes(m, n, k))


def vec_matmul_blocks(a: torch.Tensor, a_scales: torch.Tensor, b: torch.Tensor, b_scales: torch.Tensor,
                      dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """a b^T of 8-bit matrices [m, k] and [n, k] with their scales [m or n, ceil(k / 128)]; bfloat16 unless `dtype` or `out` says else."""
    call = _Call("vec_matmul_blocks", a, stream)
    m, k, ap, lda = call.first_rows("a", a)
    n, nb, st = b.shape[0], -(-k // VEC_BLOCK), a_scales.dtype
    bp, ldb = call.rows("b", b, n, k, b.dtype)
    asp, ldas = call.rows("a_scales", a_scales, m, nb, st)
    bsp, ldbs = call.rows("b_scales", b_scales, n, nb, st)
    to = call.out_type(out, dtype, torch.bfloat16)
    if out is None:
        out = call.empty(to, m, n)
        cp, ldc = out.data_ptr(), n or 1
    else:
        cp, ldc = call.rows("out", out, m, n, to)
    lib = _lib or load()
    wptr, wbytes, keep = call.workspace(workspace, _vec_bytes("vec_matmul_blocks_workspace_bytes", m, n, k))
    call.launch(lib.vec_matmul_blocks, ap, lda, call.type("a", a.dtype), asp, ldas, bp, ldb, call.type("b", b.dtype), bsp, ldbs,
                call.type("scales", st), m, n, k, cp, ldc, call.type("out", to), wptr, wbytes)
    return out


def vec_dropout(x: torch.Tensor, p: float, state: Optional[torch.Tensor] = None, layer: int = 0, residual: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """residual + x / (1 - p) where kept.  state: int64 [seed, step] on the GPU, from which, with `layer`, the mask is made; the gradient
    of x is the same call on the result's gradient, without a residual.  `out` may be x or residual."""
    call = _Call("vec_dropout", x, stream)
    n, d, xp, ldx = call.first_rows("x", x)
    rp, ldr = call.rows("residual", residual, n, d, x.dtype) if residual is not None else (None, 0)
    p, sp, layer = call.mask(p, state, layer)
    if out is None:
        out = call.empty(x.dtype, n, d)
        yp, ldy = out.data_ptr(), d
    else:
        yp, ldy = call.rows("out", out, n, d, x.dtype)
    call.launch((_lib or load()).vec_dropout, xp, ldx, rp, ldr, call.type("x", x.dtype), n, d, p, sp, layer, yp, ldy)
    return out


def _adapters(call: _Call, x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, ids: torch.Tensor, scales: Optional[torch.Tensor]):
    """What both calls of the adapters take: rows, columns, ranks, adapters; x's address and distance; and the C arguments from a to dout."""
    n, din, xp, ldx = call.first_rows("x", x)
    if a.dim() != 3 or b.dim() != 3:
        _refuse(call.name, f"a and b of shapes {tuple(a.shape)} and {tuple(b.shape)}, not [adapters, rank, columns]")
    count, rank, _ = a.shape
    dout = b.shape[2]
    if max(din, dout, rank, count) > 0x7FFFFFFF:
        _refuse(call.name, f"din={din}, dout={dout}, rank={rank}, adapters={count}")
    ap, lda, sta = call.matrices("a", a, count, rank, din, x.dtype)
    bp, ldb, stb = call.matrices("b", b, count, rank, dout, x.dtype)
    idp, id_bytes = call.ids(ids)
    if ids.numel() != n:
        _refuse(call.name, f"{ids.numel()} ids for {n} rows")
    sp = call.vector("scales", scales, count, torch.float32) if scales is not None else None
    t = call.type("x", x.dtype)
    return n, din, dout, rank, count, t, xp, ldx, (ap, lda, sta, bp, ldb, stb, t, count, rank, sp, idp, id_bytes, n, din, dout)


def vec_adapter_workspace_bytes(n: int, din: int, dout: int, rank: int, adapters: int, dtype: torch.dtype) -> int:
    return int(load().vec_adapter_workspace_bytes(n, din, dout, rank, adapters, _VEC_TYPE[dtype]))


def vec_adapter(x: torch.Tensor, a: torch.Tensor, b: torch.Tensor, ids: torch.Tensor, scales: Optional[torch.Tensor] = None,
                base: Optional[torch.Tensor] = None, p: float = 0.0, state: Optional[torch.Tensor] = None, layer: int = 0,
                dtype: Optional[torch.dtype] = None, want_t: bool = False, out=None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Low-rank adapters of many requests: y = base + t b[e] with t = scales[e] * dropout(x) a[e]^T and e the row's id, y = base where
    that is outside.  a [adapters, rank, din], b [adapters, rank, dout]; p, state and layer as in vec_dropout.  Returns (y, t), t (float32,
    for the gradient) where wanted, else None.  `out`: the same two, to be written (y may be base, not x; its type x's or float32)."""
    call = _Call("vec_adapter", x, stream)
    n, din, dout, rank, count, tx, xp, ldx, args = _adapters(call, x, a, b, ids, scales)
    p, statep, layer = call.mask(p, state, layer)
    if out is None:
        to = dtype or (base.dtype if base is not None else x.dtype)
        y = call.empty(to, n, dout)
        yp, ldy = y.data_ptr(), dout
        t = call.empty(torch.float32, n, rank) if want_t else None
        tp = t.data_ptr() if want_t else None
    else:
        y, t = out
        to = call.out_type(y, dtype, None)
        yp, ldy = call.rows("y", y, n, dout, to)
        tp = None
        if t is not None:
            tp, ldt = call.rows("t", t, n, rank, torch.float32)
            if ldt != rank:
                _refuse(call.name, f"t's rows of {rank} are {ldt} apart")
    bp, ldb = call.rows("base", base, n, dout, to) if base is not None else (None, 0)
    lib = _lib or load()
    wptr, wbytes, keep = call.workspace(workspace, _vec_bytes("vec_adapter_workspace_bytes", n, din, dout, rank, count, tx))
    call.launch(lib.vec_adapter, xp, ldx, *args, bp, ldb, yp, ldy, call.type("y", to), p, statep, layer, tp, wptr, wbytes)
    return y, t


def vec_adapter_grad_workspace_bytes(n: int, din: int, dout: int, rank: int, adapters: int, dtype: torch.dtype) -> int:
    return int(load().vec_adapter_grad_workspace_bytes(n, din, dout, rank, adapters, _VEC_TYPE[dtype]))


def vec_adapter_grad(dy: torch.Tensor, x: torch.Tensor, t: torch.Tensor, a: torch.Tensor, b: torch.Tensor, ids: torch.Tensor,
                     scales: Optional[torch.Tensor] = None, dx_base: Optional[torch.Tensor] = None, p: float = 0.0,
                     state: Optional[torch.Tensor] = None, layer: int = 0, dtype: Optional[torch.dtype] = None, want_dx: bool = True,
                     accumulate: bool = False, out=None, workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, da, db) of vec_adapter: t is its second result, dx_base the gradient that reaches x past the adapters; da and db are float32
    unless `dtype` says x's type, and zeros for adapters without a row.  `out`: the same three, to be written (dx may be None or dx_base); with
    `accumulate` the sums are added to its da and db."""
    call = _Call("vec_adapter_grad", x, stream)
    n, din, dout, rank, count, tx, xp, ldx, args = _adapters(call, x, a, b, ids, scales)
    dyp, lddy = call.rows("dy", dy, n, dout, x.dtype)
    tp, ldt = call.rows("t", t, n, rank, torch.float32)
    if ldt != rank and n > 1:
        _refuse(call.name, f"t's rows of {rank} are {ldt} apart")
    p, statep, layer = call.mask(p, state, layer)
    if accumulate and out is None:
        _refuse(call.name, "accumulate needs an out to add to")
    if out is None:
        to = dtype or torch.float32
        dx = call.empty(x.dtype, n, din) if want_dx else None
        da, db = call.empty(to, count, rank, din), call.empty(to, count, rank, dout)
    else:
        dx, da, db = out
        to = call.out_type(da, dtype, None)
    dxp, lddx = call.rows("dx", dx, n, din, x.dtype) if dx is not None else (None, 0)
    ep, lde = call.rows("dx_base", dx_base, n, din, x.dtype) if dx_base is not None else (None, 0)
    dap, ldda, stda = call.matrices("da", da, count, rank, din, to)
    dbp, lddb, stdb = call.matrices("db", db, count, rank, dout, to)
    lib = _lib or load()
    wptr, wbytes, keep = call.workspace(workspace, _vec_bytes("vec_adapter_grad_workspace_bytes", n, din, dout, rank, count, tx))
    call.launch(lib.vec_adapter_grad, dyp, lddy, xp, ldx, tp, *args, ep, lde, dxp, lddx, p, statep, layer, int(accumulate), dap, ldda, stda, dbp, lddb, stdb,
                call.type("da", to), wptr, wbytes)
    return dx, da, db

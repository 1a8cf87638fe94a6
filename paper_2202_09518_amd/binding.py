"""Thin ctypes binding of libnmfmu.so: argument marshalling only.

Every function has the name and argument order of its C entry point in
``include/nmfmu.h``; tensors are torch tensors whose ``data_ptr()`` is handed
over.  Nothing is computed here and there is no fallback: if the HIP library
has not been built, importing the symbols raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnmfmu.so")

EXPORTS = [
    "nmf_status_string", "nmf_last_error",
    "nmf_mu_dense", "nmf_mu_dense_noalloc", "nmf_mu_dense_profile", "nmf_residual_dense", "nmf_mu_dense_tol", "nmf_mu_dense_monitor", "nmf_mu_csr", "nmf_mu_csr_monitor", "nmf_mu_csr_tol", "nmf_mu_ooc", "nmf_mu_ooc_monitor", "nmf_mu_ooc_hostw", "nmf_mu_csr_ooc", "nmf_mu_dense_batched",
    "nmf_mu_workspace_bytes", "nmf_mu_set_workspace", "nmf_mu_release",
    "nmf_csr_partition", "nmf_split_planes", "nmf_csr_to_csc", "nmf_gram_w", "nmf_wta_dense", "nmf_h_update", "nmf_aht_w_update_dense",
    "nmf_grouped_product", "nmf_grouped_gradient", "nmf_lowrank_product", "nmf_lowrank_gradient", "nmf_ragged_work_bytes",
    "nmf_rms_norm", "nmf_rms_norm_gradient", "nmf_round_blocks", "nmf_grouped_product8", "nmf_route", "nmf_route_gradient",
    "nmf_spread_rows", "nmf_collect_rows", "nmf_collect_gradient", "nmf_routed_work_bytes",
]

NMF_OK, NMF_EINVAL, NMF_ENOMEM, NMF_EHIP, NMF_EUNSUPPORTED = range(5)
NMF_MU_MAX_K = 64
NMF_MU_MAX_K_SLICED = 1024
NMF_LOWRANK_MAX_K = 256
NMF_F32, NMF_BF16, NMF_F16, NMF_E4M3 = range(4)
NMF_NORM_MAX_M, NMF_ROUTE_MAX_GROUPS, NMF_ROUTE_MAX_K = 32768, 1024, 16
NMF_ODD_X, NMF_ODD_B, NMF_ODD_FACTORS, NMF_ONE_B, NMF_B_M_X_N, NMF_B_N_X_M = 16, 32, 64, 128, 256, 512
_FAR = 1 << 22                          # leading dimensions of codes from here on are odd ones too

_lib = None


class NmfError(RuntimeError):
    def __init__(self, status: int, name: str, detail: str):
        super().__init__(f"{name}: {detail}" if detail else name)
        self.status = status


def lib() -> ctypes.CDLL:
    """Load libnmfmu.so (built by ``paper_2202_09518_amd.build``); no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it first (python -m paper_2202_09518_amd.build); "
            "there is no CPU or PyTorch fallback")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32, f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
    L.nmf_status_string.restype = ctypes.c_char_p
    L.nmf_status_string.argtypes = [ctypes.c_int]
    L.nmf_last_error.restype = ctypes.c_char_p
    L.nmf_mu_dense.argtypes = [vp, i64, i64, i32, vp, vp, i32, f32, vp]
    L.nmf_mu_dense_noalloc.argtypes = [vp, i64, i64, i32, vp, vp, i32, f32, vp]
    L.nmf_mu_dense_profile.argtypes = [vp, i64, i64, i32, vp, vp, i32, f32, vp, vp]
    L.nmf_residual_dense.argtypes = [vp, i64, i64, i32, vp, vp, vp, vp]
    L.nmf_mu_dense_tol.argtypes = [vp, i64, i64, i32, vp, vp, i32, f32, ctypes.c_double, i32, vp, vp, vp]
    L.nmf_mu_csr.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp, vp, i32, f32, vp]
    L.nmf_mu_csr_monitor.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp, vp, i32, f32, vp, vp]
    L.nmf_mu_csr_tol.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp, vp, i32, f32, ctypes.c_double, i32, vp, vp, vp]
    L.nmf_mu_ooc.argtypes = [vp, i64, i64, i32, vp, vp, i32, f32, i64, i64, vp]
    L.nmf_mu_ooc_monitor.argtypes = [vp, i64, i64, i32, vp, vp, i32, f32, i64, i64, vp, vp]
    L.nmf_mu_dense_monitor.argtypes = [vp, i64, i64, i32, vp, vp, i32, f32, vp, vp]
    L.nmf_mu_csr_ooc.argtypes = [vp, vp, vp, i64, i64, i64, i32, vp, vp, i32, f32, i64, i64, vp]
    L.nmf_mu_ooc_hostw.argtypes = [vp, vp, i64, i64, i32, vp, i32, f32, i64, i32, vp, vp]
    L.nmf_mu_dense_batched.argtypes = [i32, vp, i64, i64, vp, vp, vp, i32, f32, vp]
    L.nmf_mu_workspace_bytes.restype = ctypes.c_size_t
    L.nmf_mu_workspace_bytes.argtypes = [ctypes.c_int, i64, i64, i64, i32, i64]
    L.nmf_mu_set_workspace.argtypes = [vp, ctypes.c_size_t]
    L.nmf_mu_release.argtypes = []
    L.nmf_csr_partition.argtypes = [vp, i64, i32, vp, vp]
    L.nmf_split_planes.argtypes = [vp, i64, i32, vp, vp]
    L.nmf_csr_to_csc.argtypes = [vp, vp, vp, i64, i64, i64, vp, vp, vp, vp]
    L.nmf_gram_w.argtypes = [vp, i64, i32, vp, vp]
    L.nmf_wta_dense.argtypes = [vp, i64, i64, i32, vp, vp, vp]
    L.nmf_h_update.argtypes = [vp, vp, vp, i32, i64, f32, vp, vp]
    L.nmf_aht_w_update_dense.argtypes = [vp, i64, i64, i32, vp, vp, vp, f32, vp]
    L.nmf_grouped_product.argtypes = [i32, vp, i64, vp, i32, i64, vp, i64, i64, i32, i64, i64, vp, i64, vp, ctypes.c_size_t, vp]
    L.nmf_grouped_gradient.argtypes = [i32, vp, i64, vp, i64, vp, i32, i64, i64, i64, vp, i64, i64, vp, ctypes.c_size_t, vp]
    L.nmf_lowrank_product.argtypes = [i32, vp, i64, i64, vp, i64, i32, i64, i64, vp, vp, i32, vp, vp, vp, i32, i32, i64, vp, vp, vp, i64, vp,
                                      ctypes.c_size_t, vp]
    L.nmf_lowrank_gradient.argtypes = [i32, vp, i64, vp, i64, i64, i64, i64, vp, vp, i32, vp, i32, i32, i64, vp, vp, vp, vp, vp,
                                       ctypes.c_size_t, vp]
    L.nmf_ragged_work_bytes.restype = ctypes.c_size_t
    L.nmf_ragged_work_bytes.argtypes = [ctypes.c_int, i32, i64, i64, i64, i32, i32, i32, i64]
    size = ctypes.c_size_t
    L.nmf_rms_norm.argtypes = [i32, vp, i64, vp, i64, vp, i64, i64, f32, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp]
    L.nmf_rms_norm_gradient.argtypes = [i32, vp, i64, vp, vp, vp, i64, vp, i64, i64, i64, vp, i64, vp, vp, size, vp]
    L.nmf_round_blocks.argtypes = [i32, vp, i64, i64, i32, i64, i64, i32, vp, i64, i64, vp, i64, i64, vp]
    L.nmf_grouped_product8.argtypes = [i32, vp, i64, vp, i64, vp, i32, i64, vp, i64, i64, vp, i64, i64, i32, i64, i64, vp, i64, vp, size, vp]
    L.nmf_route.argtypes = [i32, vp, i64, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, size, vp]
    L.nmf_route_gradient.argtypes = [i32, vp, i64, i64, i32, i32, i32, vp, vp, vp, vp, vp, i64, vp]
    L.nmf_spread_rows.argtypes = [i32, vp, i64, i64, i32, vp, i64, vp, i64, i64, vp, i64, vp, i64, vp]
    L.nmf_collect_rows.argtypes = [i32, vp, i64, i64, i64, i32, vp, vp, i64, vp, i64, vp]
    L.nmf_collect_gradient.argtypes = [i32, vp, i64, i64, i32, vp, vp, i64, vp, i64, i64, vp, i64, vp, vp]
    L.nmf_routed_work_bytes.restype = size
    L.nmf_routed_work_bytes.argtypes = [ctypes.c_int, i64, i64, i64, i32]
    for name in EXPORTS:
        fn = getattr(L, name)
        if fn.restype is ctypes.c_int and name not in ("nmf_status_string", "nmf_last_error"):
            fn.restype = ctypes.c_int
    _lib = L
    return L


def _check(status: int) -> None:
    if status != NMF_OK:
        L = lib()
        raise NmfError(status, L.nmf_status_string(status).decode(), L.nmf_last_error().decode())


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _dev(t: torch.Tensor, dtype, what: str) -> int:
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError(f"{what}: need a contiguous {dtype} device tensor")
    return t.data_ptr()


def nmf_status_string(status: int) -> str:
    return lib().nmf_status_string(int(status)).decode()


def nmf_last_error() -> str:
    return lib().nmf_last_error().decode()


def nmf_mu_dense(A, m, n, k, W, H, iters, eps, stream=None) -> None:
    _check(lib().nmf_mu_dense(_dev(A, torch.float32, "A"), m, n, k, _dev(W, torch.float32, "W"),
                              _dev(H, torch.float32, "H"), iters, eps, _stream(stream)))


def nmf_mu_dense_noalloc(A, m, n, k, W, H, iters, eps, stream=None) -> None:
    _check(lib().nmf_mu_dense_noalloc(_dev(A, torch.float32, "A"), m, n, k, _dev(W, torch.float32, "W"),
                                      _dev(H, torch.float32, "H"), iters, eps, _stream(stream)))


def nmf_mu_dense_profile(A, m, n, k, W, H, iters, eps, stream=None):
    """Returns [six average kernel times in ms (launch order of one iteration), mirrored flag,
    ms per launch of the pass over A and of the pass over A^T launched back to back]."""
    ms = (ctypes.c_float * 9)()
    _check(lib().nmf_mu_dense_profile(_dev(A, torch.float32, "A"), m, n, k, _dev(W, torch.float32, "W"),
                                      _dev(H, torch.float32, "H"), iters, eps, _stream(stream), ms))
    return list(ms)


def nmf_residual_dense(A, m, n, k, W, H, stream=None) -> float:
    """||A - W H||_F (blocking)."""
    out = ctypes.c_double()
    _check(lib().nmf_residual_dense(_dev(A, torch.float32, "A"), m, n, k, _dev(W, torch.float32, "W"),
                                    _dev(H, torch.float32, "H"), ctypes.byref(out), _stream(stream)))
    return out.value


def nmf_mu_dense_tol(A, m, n, k, W, H, max_iters, eps, tol, check_every, stream=None):
    """Returns (iterations applied, ||A - W H||_F of the returned factors); blocking."""
    done = ctypes.c_int32()
    res = ctypes.c_double()
    _check(lib().nmf_mu_dense_tol(_dev(A, torch.float32, "A"), m, n, k, _dev(W, torch.float32, "W"),
                                  _dev(H, torch.float32, "H"), max_iters, eps, tol, check_every,
                                  ctypes.byref(done), ctypes.byref(res), _stream(stream)))
    return done.value, res.value


def nmf_mu_csr(rowptr, colidx, vals, m, n, nnz, k, W, H, iters, eps, stream=None) -> None:
    _check(lib().nmf_mu_csr(_dev(rowptr, torch.int64, "rowptr"), _dev(colidx, torch.int32, "colidx"),
                            _dev(vals, torch.float32, "vals"), m, n, nnz, k,
                            _dev(W, torch.float32, "W"), _dev(H, torch.float32, "H"),
                            iters, eps, _stream(stream)))


def nmf_mu_ooc_monitor(A_host, m, n, k, W, H, iters, eps, batch_rows, device_budget_bytes, stream=None):
    """nmf_mu_ooc that also returns the objective after each iteration (list of floats, blocking)."""
    if A_host.is_cuda or A_host.dtype != torch.float32 or not A_host.is_contiguous():
        raise ValueError("A_host: need a contiguous float32 host tensor (pinned for overlap)")
    out = (ctypes.c_double * max(iters, 1))()
    _check(lib().nmf_mu_ooc_monitor(A_host.data_ptr(), m, n, k, _dev(W, torch.float32, "W"),
                                    _dev(H, torch.float32, "H"), iters, eps, batch_rows,
                                    device_budget_bytes, out, _stream(stream)))
    return list(out)[:iters]


def nmf_mu_csr_monitor(rowptr, colidx, vals, m, n, nnz, k, W, H, iters, eps, stream=None):
    """Runs `iters` iterations on a CSR matrix; returns the objective after each (list of floats, blocking)."""
    out = (ctypes.c_double * max(iters, 1))()
    _check(lib().nmf_mu_csr_monitor(_dev(rowptr, torch.int64, "rowptr"), _dev(colidx, torch.int32, "colidx"),
                                    _dev(vals, torch.float32, "vals"), m, n, nnz, k,
                                    _dev(W, torch.float32, "W"), _dev(H, torch.float32, "H"),
                                    iters, eps, out, _stream(stream)))
    return list(out)[:iters]


def nmf_mu_csr_tol(rowptr, colidx, vals, m, n, nnz, k, W, H, max_iters, eps, tol, check_every=1, stream=None):
    """Algorithm 1's loop on a CSR matrix; returns (iterations applied, final objective).  Blocking."""
    done = ctypes.c_int32(0)
    res = ctypes.c_double(0.0)
    _check(lib().nmf_mu_csr_tol(_dev(rowptr, torch.int64, "rowptr"), _dev(colidx, torch.int32, "colidx"),
                                _dev(vals, torch.float32, "vals"), m, n, nnz, k,
                                _dev(W, torch.float32, "W"), _dev(H, torch.float32, "H"),
                                max_iters, eps, tol, check_every, ctypes.byref(done), ctypes.byref(res),
                                _stream(stream)))
    return done.value, res.value


def nmf_mu_ooc(A_host, m, n, k, W, H, iters, eps, batch_rows, device_budget_bytes, stream=None) -> None:
    if A_host.is_cuda or A_host.dtype != torch.float32 or not A_host.is_contiguous():
        raise ValueError("A_host: need a contiguous float32 host tensor (pinned for overlap)")
    _check(lib().nmf_mu_ooc(A_host.data_ptr(), m, n, k, _dev(W, torch.float32, "W"),
                            _dev(H, torch.float32, "H"), iters, eps, batch_rows,
                            device_budget_bytes, _stream(stream)))


def nmf_mu_ooc_hostw(A_host, W_host, m, n, k, H, iters, eps, batch_rows, slots, stream=None) -> int:
    """W_host is updated in place (valid after the stream is synchronised).  Returns the
    device bytes the call used (workspace + staging)."""
    for t, what in ((A_host, "A_host"), (W_host, "W_host")):
        if t.is_cuda or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError(f"{what}: need a contiguous float32 host tensor (pinned for overlap)")
    used = ctypes.c_size_t(0)
    _check(lib().nmf_mu_ooc_hostw(A_host.data_ptr(), W_host.data_ptr(), m, n, k, _dev(H, torch.float32, "H"),
                                  iters, eps, batch_rows, slots, _stream(stream), ctypes.byref(used)))
    return int(used.value)


def nmf_mu_dense_monitor(A, m, n, k, W, H, iters, eps, stream=None):
    """Runs `iters` iterations; returns the objective after each (list of floats, blocking)."""
    out = (ctypes.c_double * max(iters, 1))()
    _check(lib().nmf_mu_dense_monitor(_dev(A, torch.float32, "A"), m, n, k, _dev(W, torch.float32, "W"),
                                      _dev(H, torch.float32, "H"), iters, eps, out, _stream(stream)))
    return list(out)[:iters]


def nmf_mu_csr_ooc(rowptr, colidx, vals, m, n, nnz, k, W, H, iters, eps, batch_nnz, device_budget_bytes,
                   stream=None) -> None:
    """rowptr (int64), colidx (int32), vals (float32): contiguous HOST tensors (pinned for overlap)."""
    for t, dt, what in ((rowptr, torch.int64, "rowptr"), (colidx, torch.int32, "colidx"), (vals, torch.float32, "vals")):
        if t.is_cuda or t.dtype != dt or not t.is_contiguous():
            raise ValueError(f"{what}: need a contiguous {dt} host tensor")
    _check(lib().nmf_mu_csr_ooc(rowptr.data_ptr(), colidx.data_ptr(), vals.data_ptr(), m, n, nnz, k,
                                _dev(W, torch.float32, "W"), _dev(H, torch.float32, "H"), iters, eps,
                                batch_nnz, device_budget_bytes, _stream(stream)))


def nmf_mu_dense_batched(n_runs, A, m, n, k, W, H, iters, eps, stream=None) -> None:
    """A, W, H: sequences of device tensors (A entries may repeat); k: sequence of ranks."""
    PtrArr = ctypes.c_void_p * n_runs
    a = PtrArr(*[_dev(t, torch.float32, "A[r]") for t in A])
    w = PtrArr(*[_dev(t, torch.float32, "W[r]") for t in W])
    h = PtrArr(*[_dev(t, torch.float32, "H[r]") for t in H])
    ks = (ctypes.c_int32 * n_runs)(*[int(x) for x in k])
    _check(lib().nmf_mu_dense_batched(n_runs, a, m, n, ks, w, h, iters, eps, _stream(stream)))


def nmf_mu_workspace_bytes(kind, m, n, nnz, k, batch_rows) -> int:
    return int(lib().nmf_mu_workspace_bytes(kind, m, n, nnz, k, batch_rows))


def nmf_mu_set_workspace(buf, nbytes=None) -> None:
    if buf is None:
        _check(lib().nmf_mu_set_workspace(None, 0))
    else:
        _check(lib().nmf_mu_set_workspace(buf.data_ptr(), buf.numel() * buf.element_size() if nbytes is None else nbytes))


def nmf_mu_release() -> None:
    _check(lib().nmf_mu_release())


def nmf_csr_partition(rowptr, m, nparts, part, stream=None) -> None:
    _check(lib().nmf_csr_partition(_dev(rowptr, torch.int64, "rowptr"), m, nparts,
                                   _dev(part, torch.int64, "part"), _stream(stream)))


def nmf_split_planes(X, rows, k, planes, stream=None) -> None:
    """planes: int16 device tensor of ceil(rows / 8) * 24 * KP elements (bf16 bit patterns),
    KP = 32 for k <= 32, else 64."""
    _check(lib().nmf_split_planes(_dev(X, torch.float32, "X"), rows, k, _dev(planes, torch.int16, "planes"),
                                  _stream(stream)))


def nmf_csr_to_csc(rowptr, colidx, vals, m, n, nnz, colptr, rowidx, cvals, stream=None) -> None:
    _check(lib().nmf_csr_to_csc(_dev(rowptr, torch.int64, "rowptr"), _dev(colidx, torch.int32, "colidx"),
                                _dev(vals, torch.float32, "vals"), m, n, nnz,
                                _dev(colptr, torch.int64, "colptr"), _dev(rowidx, torch.int32, "rowidx"),
                                _dev(cvals, torch.float32, "cvals"), _stream(stream)))


def nmf_gram_w(W, m, k, G, stream=None) -> None:
    _check(lib().nmf_gram_w(_dev(W, torch.float32, "W"), m, k, _dev(G, torch.float32, "G"), _stream(stream)))


def nmf_wta_dense(A, m, n, k, W, P, stream=None) -> None:
    _check(lib().nmf_wta_dense(_dev(A, torch.float32, "A"), m, n, k, _dev(W, torch.float32, "W"),
                               _dev(P, torch.float32, "P"), _stream(stream)))


def nmf_h_update(H, P, G, k, n, eps, GH=None, stream=None) -> None:
    _check(lib().nmf_h_update(_dev(H, torch.float32, "H"), _dev(P, torch.float32, "P"),
                              _dev(G, torch.float32, "G"), k, n, eps,
                              None if GH is None else _dev(GH, torch.float32, "GH"), _stream(stream)))


def nmf_aht_w_update_dense(A, m, n, k, H, GH, W, eps, stream=None) -> None:
    _check(lib().nmf_aht_w_update_dense(_dev(A, torch.float32, "A"), m, n, k,
                                        _dev(H, torch.float32, "H"), _dev(GH, torch.float32, "GH"),
                                        _dev(W, torch.float32, "W"), eps, _stream(stream)))


# ---- products over ragged ranges of rows (include/nmfmu_ragged.h) ------------------
# Types and leading dimensions are the tensors'; the scratch is torch's unless `work` (a uint8 device tensor) is given.  All
# tensors lie on X's device, and the call runs there, whichever device is current.  `odd` tells the size query which operands lie off
# 16-byte borders by their pointer, leading dimension or stride, and whether one matrix serves all groups.

_TYPES = {torch.float32: NMF_F32, torch.bfloat16: NMF_BF16, torch.float16: NMF_F16}


def _type(t: torch.Tensor, what: str) -> int:
    typ = _TYPES.get(t.dtype)
    if typ is None or not t.is_cuda:
        raise ValueError(f"{what}: need a float32, bfloat16 or float16 device tensor")
    return typ


def _rows_of(t, dtype, device, rows, cols, what):
    """(pointer, leading dimension) of a rows x cols matrix whose rows are contiguous."""
    if t.dtype is dtype and t.get_device() == device and t.shape == (rows, cols):
        ld, step = t.stride()
        if step == 1 or cols <= 1:
            if ld >= cols:
                return t.data_ptr(), ld
            if rows <= 1:
                return t.data_ptr(), cols
    raise ValueError(f"{what}: need a {rows} x {cols} {dtype} tensor on device {device} with contiguous rows that do not overlap")


def _stack_of(t, dtype, device, count, rows, cols, what):
    """(pointer, leading dimension, stride) of `count` such matrices."""
    if t.dtype is dtype and t.get_device() == device and t.shape == (count, rows, cols):
        stride, ld, step = t.stride()
        if step == 1 or cols <= 1:
            if rows <= 1 and ld < cols:
                ld = cols
            if ld >= cols:
                return t.data_ptr(), ld, stride if count > 1 else max((rows - 1) * ld + cols, stride)
    raise ValueError(f"{what}: need a {count} x {rows} x {cols} {dtype} tensor on device {device} with contiguous rows that do not overlap")


def _list(t, dtype, device, count, what):
    if t.dtype is dtype and t.get_device() == device and t.numel() == count and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{what}: need a contiguous {dtype} tensor of {count} entries on device {device}")


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)      # 3 us less a call
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)      # the tensors have opened the device


def _stream_at(device, stream) -> int:
    """The stream of a call: the current one of its device if none is given."""
    if stream is None:
        return _raw_stream(device)
    if isinstance(stream, torch.cuda.Stream) and stream.device_index != device:
        raise ValueError(f"stream: need one of device {device}")
    return _stream(stream)


def _call_on(device, call, *args) -> None:
    """A call with its device current: a launch goes to the current one."""
    with torch.cuda.device(device):
        call(*args)


@functools.lru_cache(maxsize=1024)
def _need(kind, typ, rows, m, n, parts, runs, kmax, ktotal) -> int:
    return int(lib().nmf_ragged_work_bytes(kind, typ, rows, m, n, parts, runs, kmax, ktotal))


def _work(kind, typ, rows, m, n, parts, runs, kmax, ktotal, work, device, stream):
    """(pointer, bytes, tensor to keep) of the scratch of a call."""
    return _scratch(0 if work is not None else _need(kind, typ, rows, m, n, parts, runs, kmax, ktotal), work, device, stream)


def _scratch(need, work, device, stream):
    if work is not None:
        if not (work.get_device() == device and work.dtype == torch.uint8 and work.is_contiguous()):
            raise ValueError(f"work: need a contiguous uint8 tensor on device {device}")
        return work.data_ptr(), work.numel(), work
    if need == 0:
        return None, 0, None
    if stream is None:
        buf = torch.empty(need, dtype=torch.uint8, device=device)
    else:                                   # memory that is free in the order of the call's stream
        with torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream), device=device)):
            buf = torch.empty(need, dtype=torch.uint8, device=device)
    return buf.data_ptr(), need, buf


def nmf_ragged_work_bytes(kind, type, rows, m, n, parts, runs=0, kmax=0, ktotal=0) -> int:
    return int(lib().nmf_ragged_work_bytes(kind, type, rows, m, n, parts, runs, kmax, ktotal))


def nmf_grouped_product(X, offsets, groups, rows, B, transposed, m, n, Y, work=None, stream=None) -> None:
    """Y_g = X_g B_g; B: groups x m x n, or groups x n x m if transposed."""
    typ, dt, d = _type(X, "X"), X.dtype, X.get_device()
    if d != _current_device():
        return _call_on(d, nmf_grouped_product, X, offsets, groups, rows, B, transposed, m, n, Y, work, stream)
    x, ldx = _rows_of(X, dt, d, rows, m, "X")
    b, ldb, stride_b = _stack_of(B, dt, d, groups, *((n, m) if transposed else (m, n)), "B")
    y, ldy = _rows_of(Y, dt, d, rows, n, "Y")
    e = 4 if typ == NMF_F32 else 2
    odd = (NMF_ODD_X if (x | ldx * e) & 15 else 0) | (NMF_ODD_B if (b | (ldb | (stride_b if groups > 1 else 0)) * e) & 15 else 0)
    if stride_b == 0:
        odd |= NMF_ONE_B
    w, nbytes, _keep = _work(odd, typ, rows, m, n, groups, 0, 0, 0, work, d, stream)
    _check(lib().nmf_grouped_product(typ, x, ldx, _list(offsets, torch.int64, d, groups + 1, "offsets"), groups, rows, b, ldb, stride_b,
                                     int(bool(transposed)), m, n, y, ldy, w, nbytes, _stream_at(d, stream)))


def nmf_grouped_gradient(X, dY, offsets, groups, rows, m, n, G, work=None, stream=None) -> None:
    """G_g = X_g^T dY_g (groups x m x n)."""
    typ, dt, d = _type(X, "X"), X.dtype, X.get_device()
    if d != _current_device():
        return _call_on(d, nmf_grouped_gradient, X, dY, offsets, groups, rows, m, n, G, work, stream)
    x, ldx = _rows_of(X, dt, d, rows, m, "X")
    dy, ldy = _rows_of(dY, dt, d, rows, n, "dY")
    g, ldg, stride_g = _stack_of(G, dt, d, groups, m, n, "G")
    e = 4 if typ == NMF_F32 else 2
    odd = (NMF_ODD_X if (x | ldx * e) & 15 else 0) | (NMF_ODD_B if (dy | ldy * e) & 15 else 0)
    w, nbytes, _keep = _work(1 | odd, typ, rows, m, n, groups, 0, 0, 0, work, d, stream)
    _check(lib().nmf_grouped_gradient(typ, x, ldx, dy, ldy, _list(offsets, torch.int64, d, groups + 1, "offsets"), groups, rows, m, n,
                                      g, ldg, stride_g, w, nbytes, _stream_at(d, stream)))


def nmf_lowrank_product(X, rows, A, transposed, m, n, offsets, run, segments, Wt, H, koff, runs, kmax, scale, U, Y,
                        work=None, stream=None) -> None:
    """Y = X A + scale_r (X W_r) H_r; Wt: ktotal x m, H: ktotal x n, contiguous; U: rows x kmax float32, written."""
    typ, dt, d = _type(X, "X"), X.dtype, X.get_device()
    if d != _current_device():
        return _call_on(d, nmf_lowrank_product, X, rows, A, transposed, m, n, offsets, run, segments, Wt, H, koff, runs, kmax, scale, U, Y, work, stream)
    ktotal = Wt.shape[0]
    x, ldx = _rows_of(X, dt, d, rows, m, "X")
    a, lda = _rows_of(A, dt, d, *((n, m) if transposed else (m, n)), "A")
    y, ldy = _rows_of(Y, dt, d, rows, n, "Y")
    down, up = _list(Wt, dt, d, ktotal * m, "Wt"), _list(H, dt, d, ktotal * n, "H")
    e = 4 if typ == NMF_F32 else 2
    odd = (NMF_ODD_X if (x | ldx * e) & 15 else 0) | (NMF_ODD_B if (a | lda * e) & 15 else 0) | (NMF_ODD_FACTORS if (down | up) & 15 and segments else 0)
    w, nbytes, _keep = _work(2 | odd, typ, rows, m, n, segments, runs, kmax, ktotal, work, d, stream)
    _check(lib().nmf_lowrank_product(
        typ, x, ldx, rows, a, lda, int(bool(transposed)), m, n, _list(offsets, torch.int64, d, segments + 1, "offsets"),
        _list(run, torch.int32, d, segments, "run"), segments, down, up,
        _list(koff, torch.int32, d, runs + 1, "koff"), runs, kmax, ktotal,
        None if scale is None else _list(scale, torch.float32, d, runs, "scale"), _list(U, torch.float32, d, rows * kmax, "U"), y, ldy,
        w, nbytes, _stream_at(d, stream)))


def nmf_lowrank_gradient(X, dY, rows, m, n, offsets, run, segments, koff, runs, kmax, U, V, dWt, dH, work=None, stream=None) -> None:
    """dW_r = X^T V and dH_r = U^T dY over the rows of each run; dWt: ktotal x m, dH: ktotal x n, contiguous."""
    typ, dt, d = _type(X, "X"), X.dtype, X.get_device()
    if d != _current_device():
        return _call_on(d, nmf_lowrank_gradient, X, dY, rows, m, n, offsets, run, segments, koff, runs, kmax, U, V, dWt, dH, work, stream)
    ktotal = dWt.shape[0]
    x, ldx = _rows_of(X, dt, d, rows, m, "X")
    dy, ldy = _rows_of(dY, dt, d, rows, n, "dY")
    w, nbytes, _keep = _work(3, typ, rows, m, n, segments, runs, kmax, ktotal, work, d, stream)
    _check(lib().nmf_lowrank_gradient(
        typ, x, ldx, dy, ldy, rows, m, n, _list(offsets, torch.int64, d, segments + 1, "offsets"), _list(run, torch.int32, d, segments, "run"),
        segments, _list(koff, torch.int32, d, runs + 1, "koff"), runs, kmax, ktotal, _list(U, torch.float32, d, rows * kmax, "U"),
        _list(V, torch.float32, d, rows * kmax, "V"), _list(dWt, dt, d, ktotal * m, "dWt"), _list(dH, dt, d, ktotal * n, "dH"),
        w, nbytes, _stream_at(d, stream)))


# ---- the rows' way to the products and back (include/nmfmu_routed.h) ----------------
# As above: types and leading dimensions are the tensors', all of which lie on the first one's device.  Codes are float8_e4m3fn
# (or uint8, the same bytes).

_CODES = (torch.float8_e4m3fn, torch.uint8)


def _codes(t, what):
    if t.dtype not in _CODES or not t.is_cuda:
        raise ValueError(f"{what}: need a float8_e4m3fn or uint8 device tensor")
    return t.dtype


@functools.lru_cache(maxsize=1024)
def _need_routed(kind, rows, m, n, parts) -> int:
    return int(lib().nmf_routed_work_bytes(kind, rows, m, n, parts))


def nmf_routed_work_bytes(kind, rows, m, n=0, parts=0) -> int:
    return int(lib().nmf_routed_work_bytes(kind, rows, m, n, parts))


def nmf_rms_norm(X, rows, m, eps, weight=None, R=None, H=None, Y=None, Y8=None, scale=None, rstd=None, stream=None) -> None:
    """H = X + R, Y = H weight / sqrt(mean H^2 + eps), in X's type (Y) and in 8 bits (Y8, scale); rstd: rows float32."""
    typ, dt, d = _type(X, "X"), X.dtype, X.get_device()
    if d != _current_device():
        return _call_on(d, nmf_rms_norm, X, rows, m, eps, weight, R, H, Y, Y8, scale, rstd, stream)
    x, ldx = _rows_of(X, dt, d, rows, m, "X")
    r, ldr = (None, 0) if R is None else _rows_of(R, dt, d, rows, m, "R")
    h, ldh = (None, 0) if H is None else _rows_of(H, dt, d, rows, m, "H")
    y, ldy = (None, 0) if Y is None else _rows_of(Y, dt, d, rows, m, "Y")
    y8, ldy8 = (None, 0) if Y8 is None else _rows_of(Y8, _codes(Y8, "Y8"), d, rows, m, "Y8")
    s, lds = (None, 0) if scale is None else _rows_of(scale, torch.float32, d, rows, (m + 127) // 128, "scale")
    _check((_lib or lib()).nmf_rms_norm(typ, x, ldx, r, ldr, None if weight is None else _list(weight, dt, d, m, "weight"), rows, m, eps, h, ldh, y, ldy, y8, ldy8, s, lds,
                              None if rstd is None else _list(rstd, torch.float32, d, rows, "rstd"), _stream_at(d, stream)))


def nmf_rms_norm_gradient(H, rstd, dY, rows, m, dX, weight=None, dH=None, dweight=None, work=None, stream=None) -> None:
    """dX from dY (and dH, what reaches H on other ways), and the weight's gradient."""
    typ, dt, d = _type(H, "H"), H.dtype, H.get_device()
    if d != _current_device():
        return _call_on(d, nmf_rms_norm_gradient, H, rstd, dY, rows, m, dX, weight, dH, dweight, work, stream)
    h, ldh = _rows_of(H, dt, d, rows, m, "H")
    dy, ldy = _rows_of(dY, dt, d, rows, m, "dY")
    dh, lddh = (None, 0) if dH is None else _rows_of(dH, dt, d, rows, m, "dH")
    dx, ldx = _rows_of(dX, dt, d, rows, m, "dX")
    w, nbytes, _keep = _scratch(0 if dweight is None else _need_routed(1, rows, m, 0, 0), work, d, stream)
    _check((_lib or lib()).nmf_rms_norm_gradient(typ, h, ldh, _list(rstd, torch.float32, d, rows, "rstd"), None if weight is None else _list(weight, dt, d, m, "weight"), dy, ldy,
                                       dh, lddh, rows, m, dx, ldx, None if dweight is None else _list(dweight, dt, d, m, "dweight"), w, nbytes, _stream_at(d, stream)))


def nmf_round_blocks(X, rows, m, block, X8, scale, stream=None) -> None:
    """Codes and scales of blocks of block x 128 (1 or 128) of a matrix (rows x m) or of a stack of them (count x rows x m)."""
    typ, dt, d = _type(X, "X"), X.dtype, X.get_device()
    if d != _current_device():
        return _call_on(d, nmf_round_blocks, X, rows, m, block, X8, scale, stream)
    lines, M = (rows + block - 1) // max(block, 1), (m + 127) // 128
    codes = _codes(X8, "X8")
    if X.dim() == 3:
        count = X.shape[0]
        x, ldx, stride = _stack_of(X, dt, d, count, rows, m, "X")
        x8, ldx8, stride8 = _stack_of(X8, codes, d, count, rows, m, "X8")
        s, lds, stride_s = _stack_of(scale, torch.float32, d, count, lines, M, "scale")
    else:
        count, stride, stride8, stride_s = 1, 0, 0, 0
        x, ldx = _rows_of(X, dt, d, rows, m, "X")
        x8, ldx8 = _rows_of(X8, codes, d, rows, m, "X8")
        s, lds = _rows_of(scale, torch.float32, d, lines, M, "scale")
    _check((_lib or lib()).nmf_round_blocks(typ, x, ldx, stride, count, rows, m, block, x8, ldx8, stride8, s, lds, stride_s, _stream_at(d, stream)))


def nmf_grouped_product8(X8, xscale, offsets, groups, rows, B8, bscale, transposed, m, n, Y, work=None, stream=None) -> None:
    """Y_g = X_g B_g from codes and scales; B8: groups x m x n, or groups x n x m if transposed; the result has Y's type."""
    typ, codes, d = _type(Y, "Y"), _codes(X8, "X8"), X8.get_device()
    if d != _current_device():
        return _call_on(d, nmf_grouped_product8, X8, xscale, offsets, groups, rows, B8, bscale, transposed, m, n, Y, work, stream)
    M, N = (m + 127) // 128, (n + 127) // 128
    x, ldx = _rows_of(X8, codes, d, rows, m, "X8")
    xs, ldxs = _rows_of(xscale, torch.float32, d, rows, M, "xscale")
    b, ldb, stride_b = _stack_of(B8, _codes(B8, "B8"), d, groups, *((n, m) if transposed else (m, n)), "B8")
    bs, ldbs, stride_bs = _stack_of(bscale, torch.float32, d, groups, *((N, M) if transposed else (M, N)), "bscale")
    y, ldy = _rows_of(Y, Y.dtype, d, rows, n, "Y")
    odd = NMF_B_N_X_M if transposed else NMF_B_M_X_N
    if (x | ldx) & 15 or ldx >= _FAR:
        odd |= NMF_ODD_X
    if (b | ldb | (stride_b if groups > 1 else 0)) & 15 or ldb >= _FAR:
        odd |= NMF_ODD_B
    if stride_b == 0:
        odd |= NMF_ONE_B
    w, nbytes, _keep = _scratch(_need_routed(2 | odd, rows, m, n, groups) if work is None else 0, work, d, stream)
    _check((_lib or lib()).nmf_grouped_product8(typ, x, ldx, xs, ldxs, _list(offsets, torch.int64, d, groups + 1, "offsets"), groups, rows, b, ldb, stride_b,
                                      bs, ldbs, stride_bs, int(bool(transposed)), m, n, y, ldy, w, nbytes, _stream_at(d, stream)))


def nmf_route(logits, rows, groups, k, normalise, choice, gate, offsets, place, balance, work=None, stream=None) -> None:
    """k groups of each row, gates, the groups' offsets, places of the sorted rows, and how unequal the groups are."""
    typ, d = _type(logits, "logits"), logits.get_device()
    if d != _current_device():
        return _call_on(d, nmf_route, logits, rows, groups, k, normalise, choice, gate, offsets, place, balance, work, stream)
    l, ldl = _rows_of(logits, logits.dtype, d, rows, groups, "logits")
    w, nbytes, _keep = _scratch(_need_routed(0, rows, groups, 0, 0), work, d, stream)
    _check((_lib or lib()).nmf_route(typ, l, ldl, rows, groups, k, int(bool(normalise)), _list(choice, torch.int32, d, rows * k, "choice"),
                           _list(gate, torch.float32, d, rows * k, "gate"), _list(offsets, torch.int64, d, groups + 1, "offsets"),
                           _list(place, torch.int32, d, rows * k, "place"), _list(balance, torch.float32, d, 1, "balance"), w, nbytes,
                           _stream_at(d, stream)))


def nmf_route_gradient(logits, rows, groups, k, normalise, choice, offsets, dgate, dbalance, dlogits, stream=None) -> None:
    """Gradient of the logits from those of the gates and of balance, either of which may be None."""
    typ, d = _type(logits, "logits"), logits.get_device()
    if d != _current_device():
        return _call_on(d, nmf_route_gradient, logits, rows, groups, k, normalise, choice, offsets, dgate, dbalance, dlogits, stream)
    l, ldl = _rows_of(logits, logits.dtype, d, rows, groups, "logits")
    dl, lddl = _rows_of(dlogits, logits.dtype, d, rows, groups, "dlogits")
    _check((_lib or lib()).nmf_route_gradient(typ, l, ldl, rows, groups, k, int(bool(normalise)), _list(choice, torch.int32, d, rows * k, "choice"),
                                    _list(offsets, torch.int64, d, groups + 1, "offsets"), None if dgate is None else _list(dgate, torch.float32, d, rows * k, "dgate"),
                                    None if dbalance is None else _list(dbalance, torch.float32, d, 1, "dbalance"), dl, lddl, _stream_at(d, stream)))


def nmf_spread_rows(X, rows, k, place, m, Y, scale=None, Yscale=None, stream=None) -> None:
    """Each row of X to its k places among Y's rows; codes take their scales along (scale to Yscale)."""
    dt, d = X.dtype, X.get_device()
    if dt in _CODES:
        _codes(X, "X")
    typ = NMF_E4M3 if dt in _CODES else _type(X, "X")
    if d != _current_device():
        return _call_on(d, nmf_spread_rows, X, rows, k, place, m, Y, scale, Yscale, stream)
    x, ldx = _rows_of(X, dt, d, rows, m, "X")
    count = Y.shape[0]
    y, ldy = _rows_of(Y, dt, d, count, m, "Y")
    xs, ldxs = (None, 0) if scale is None else _rows_of(scale, torch.float32, d, rows, (m + 127) // 128, "scale")
    ys, ldys = (None, 0) if Yscale is None else _rows_of(Yscale, torch.float32, d, count, (m + 127) // 128, "Yscale")
    _check((_lib or lib()).nmf_spread_rows(typ, x, ldx, rows, k, _list(place, torch.int32, d, rows * k, "place"), m, y, ldy, count, xs, ldxs, ys, ldys,
                                 _stream_at(d, stream)))


def nmf_collect_rows(X, rows, k, place, gate, m, Y, stream=None) -> None:
    """Y[r] = sum over a row's choices of gate X[place]; gate None: 1."""
    typ, dt, d = _type(X, "X"), X.dtype, X.get_device()
    if d != _current_device():
        return _call_on(d, nmf_collect_rows, X, rows, k, place, gate, m, Y, stream)
    x, ldx = _rows_of(X, dt, d, X.shape[0], m, "X")
    y, ldy = _rows_of(Y, dt, d, rows, m, "Y")
    _check((_lib or lib()).nmf_collect_rows(typ, x, ldx, X.shape[0], rows, k, _list(place, torch.int32, d, rows * k, "place"),
                                  None if gate is None else _list(gate, torch.float32, d, rows * k, "gate"), m, y, ldy, _stream_at(d, stream)))


def nmf_collect_gradient(dY, rows, k, place, gate, m, dX, X=None, dgate=None, stream=None) -> None:
    """dX[place] = gate dY[r], and with X and dgate the gates' gradients <dY[r], X[place]>."""
    typ, dt, d = _type(dY, "dY"), dY.dtype, dY.get_device()
    if d != _current_device():
        return _call_on(d, nmf_collect_gradient, dY, rows, k, place, gate, m, dX, X, dgate, stream)
    dy, ldy = _rows_of(dY, dt, d, rows, m, "dY")
    count = dX.shape[0]
    dx, lddx = _rows_of(dX, dt, d, count, m, "dX")
    x, ldx = (None, 0) if X is None else _rows_of(X, dt, d, count, m, "X")
    _check((_lib or lib()).nmf_collect_gradient(typ, dy, ldy, rows, k, _list(place, torch.int32, d, rows * k, "place"),
                                      None if gate is None else _list(gate, torch.float32, d, rows * k, "gate"), m, dx, lddx, count, x, ldx,
                                      None if dgate is None else _list(dgate, torch.float32, d, rows * k, "dgate"), _stream_at(d, stream)))

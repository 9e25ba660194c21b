"""Python binding of the LQ C ABI (include/lq.h): argument marshalling only.

torch supplies device memory and the current stream; every step of the path runs in the HIP
library.  There is no fallback: if the library is missing, importing this module fails.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import weakref

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblq_hip.so")

V_DTYPES = {"fp32": 0, "bf16": 1, "fp16": 2}
T_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


class LqError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = _lib.lq_status_string(status).decode()
        if status == -7:
            msg += f" (hipError {_lib.lq_last_hip_error()})"
        super().__init__(f"{where}: {msg}")


class Config(C.Structure):
    """lq_config: (bits b0, block B0, scale_block B1, scale_bits b1, v_dtype b2)."""
    _fields_ = [("bits", C.c_int32), ("block", C.c_int32), ("scale_block", C.c_int32),
                ("scale_bits", C.c_int32), ("v_dtype", C.c_int32)]

    def __repr__(self):
        return f"Config({self.bits},{self.block},{self.scale_block},{self.scale_bits},{self.v_dtype})"


def config(bits, block, scale_block, scale_bits=8, v_dtype="fp32") -> Config:
    return Config(bits, block, scale_block, scale_bits, V_DTYPES[v_dtype] if isinstance(v_dtype, str) else v_dtype)


class SvdParams(C.Structure):
    """lq_svd_params; zero fields select the library defaults."""
    _fields_ = [("first_width", C.c_int32), ("first_tol", C.c_float), ("first_check", C.c_int32),
                ("first_max", C.c_int32), ("warm_width", C.c_int32), ("warm_power", C.c_int32),
                ("warm_power_2", C.c_int32), ("max_batch", C.c_int32), ("gemm_mode", C.c_int32),
                ("streams", C.c_int32), ("init_quantized", C.c_int32), ("warm_power_coarse", C.c_int32),
                ("warm_power_fine", C.c_int32)]


class Fp8Matrix(C.Structure):
    """lq_fp8_matrix."""
    _fields_ = [("codes", C.c_void_p), ("ld", C.c_int64), ("scale", C.c_void_p), ("scale_row", C.c_int64),
                ("scale_block", C.c_int64), ("tiles", C.c_int32)]


class Gradient(C.Structure):
    """lq_gradient."""
    _fields_ = [("g", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32)]


class AdamWTensor(C.Structure):
    """lq_adamw_tensor."""
    _fields_ = [(name, C.c_void_p) for name in ("p", "g", "m", "v", "m_scale", "v_scale", "copy")] + [
        ("n", C.c_int64), ("p_dtype", C.c_int32), ("g_dtype", C.c_int32)]


class AdamWParams(C.Structure):
    """lq_adamw_params."""
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("step", C.c_int64), ("lr_device", C.c_void_p), ("step_device", C.c_void_p), ("seed", C.c_uint64)]


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2311_12023_amd.build`")
_lib = C.CDLL(LIB_PATH)

_vp, _i64, _int, _sz = C.c_void_p, C.c_int64, C.c_int, C.c_size_t
_lib.lq_status_string.restype = C.c_char_p
_lib.lq_status_string.argtypes = [_int]
_lib.lq_last_hip_error.restype = _int
_lib.lq_nf_codebook.argtypes = [_int, _vp]
_lib.lq_codes_bytes.restype = _sz
_lib.lq_codes_bytes.argtypes = [_i64, _int]
_lib.lq_storage_bits.restype = C.c_double
_lib.lq_storage_bits.argtypes = [_i64, Config]
_lib.lq_nf_quantize.argtypes = [_vp, _i64, Config, _vp, _vp, _vp, _vp]
_lib.lq_nf_dequantize.argtypes = [_vp, _vp, _vp, _i64, Config, _vp, _vp]
_lib.lq_pack_scale_indices.argtypes = [_vp, _i64, _int, _vp, _vp]
_lib.lq_unpack_scale_indices.argtypes = [_vp, _i64, _int, _vp, _vp]
_PP = C.POINTER(SvdParams)
_lib.lq_factorize_workspace_bytes.restype = _sz
_lib.lq_factorize_workspace_bytes.argtypes = [_i64, _i64, _int, _PP]
_lib.lq_factorize.argtypes = [_vp, _i64, _i64, _int, _vp, _vp, C.c_uint64, _PP, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.lq_decompose_workspace_bytes.restype = _sz
_lib.lq_decompose_workspace_bytes.argtypes = [_i64, _i64, _int, _PP]
_lib.lq_decompose.argtypes = [_vp, _i64, _i64, _int, Config, _int, _int, _vp, _vp, C.c_uint64, _PP,
                              _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.lq_error_table_workspace_bytes.restype = _sz
_lib.lq_error_table_workspace_bytes.argtypes = [_i64, _i64, _int, _int, _PP]
_lib.lq_error_table.argtypes = [_vp, _i64, _i64, _int, _vp, _int, _int, _int, _vp, _vp, C.c_uint64, _PP,
                                _vp, _vp, _vp, _vp, _sz, _vp]
_lib.lq_assign_configs.argtypes = [_vp, _vp, _int, _int, C.c_double, _i64, _vp, _vp, _vp, _vp]
_lib.lq_fisher_row_col_workspace_bytes.restype = _sz
_lib.lq_fisher_row_col_workspace_bytes.argtypes = [_i64, _i64]
_lib.lq_fisher_row_col.argtypes = [_vp, _i64, _i64, _vp, _vp, _vp, _sz, _vp]
_lib.lq_matmul_workspace_bytes.restype = _sz
_lib.lq_matmul_workspace_bytes.argtypes = [_i64, _i64, _i64, _int]
_lib.lq_matmul_workspace_bytes_precision.restype = _sz
_lib.lq_matmul_workspace_bytes_precision.argtypes = [_i64, _i64, _i64, _int, _int]
_lib.lq_matmul.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, Config, _vp, _vp, _int, _int, _vp, _vp, _sz, _vp]
_lib.lq_matmul_few_rows_static_scratch_bytes.restype = _sz
_lib.lq_matmul_few_rows_static.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, Config, _vp, _vp, _int, _vp, _vp]
_lib.lq_dropout.argtypes = [_vp, _i64, _int, C.c_double, C.c_uint64, C.c_uint64, _vp, _vp]
_lib.lq_cross_entropy_workspace_bytes.restype = _sz
_lib.lq_cross_entropy_workspace_bytes.argtypes = [_i64, _i64, _i64, _int, _int, _int]
_lib.lq_cross_entropy.argtypes = [_vp, _i64, _vp, _i64, _vp, _i64, _i64, _i64, _int, _int, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.lq_adapter_workspace_bytes.restype = _sz
_lib.lq_adapter_workspace_bytes.argtypes = [_i64, _i64, _i64, _int, _int, _int]
_lib.lq_adapter_forward.argtypes = [_vp, _i64, _i64, _i64, _vp, _vp, _vp, Config, _vp, _vp, _int, _int, C.c_double, C.c_uint64,
                                    C.c_uint64, _vp, _vp, _vp, _sz, _vp]
_lib.lq_adapter_backward.argtypes = [_vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, Config, _vp, _vp, _int, _int, _vp, C.c_double,
                                     C.c_uint64, C.c_uint64, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.lq_fp8_quantize.argtypes = [_vp, _i64, _i64, _i64, _int, _int, _vp, _i64, _vp, _vp, _i64, _vp, _vp]
for _name, _args in (("matmul", [_i64] * 3), ("forward", [_i64] * 3), ("backward", [_i64] * 3 + [_int] * 2)):
    getattr(_lib, f"lq_fp8_{_name}_workspace_bytes").restype = _sz
    getattr(_lib, f"lq_fp8_{_name}_workspace_bytes").argtypes = _args
_MP = C.POINTER(Fp8Matrix)
_lib.lq_fp8_matmul.argtypes = [_MP, _MP, _i64, _i64, _i64, _vp, _i64, _vp, _sz, _vp]
_lib.lq_fp8_forward.argtypes = [_vp, _i64, _int, _MP, _i64, _i64, _i64, _vp, _vp, _sz, _vp]
_lib.lq_fp8_backward.argtypes = [_vp, _i64, _int, _vp, _i64, _int, _MP, _i64, _i64, _i64, _vp, _vp, _vp, _sz, _vp]
_lib.lq_grad_norm_workspace_bytes.restype = _sz
_lib.lq_grad_norm_workspace_bytes.argtypes = [_vp, _i64]
_lib.lq_grad_norm.argtypes = [_vp, _i64, C.c_double, _vp, _vp, _sz, _vp]
_lib.lq_adamw.argtypes = [_vp, _i64, _int, C.POINTER(AdamWParams), _vp, _vp]

_lib.lq_profile_enable.argtypes = [_int]
_lib.lq_profile_class_name.restype = C.c_char_p
_lib.lq_profile_class_name.argtypes = [_int]
_lib.lq_profile_read.argtypes = [_int, _vp, _vp, _vp]


def _check(status, where):
    if status != 0:
        raise LqError(status, where)


def _dev(t, dtype, name):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name}: need a contiguous {dtype} tensor on the GPU")
    return t.data_ptr()


def _stream():
    # the handle of torch.cuda.current_stream() without the Stream object around it (0.2 instead of 2.7 us, a quarter of what
    # a small call takes on the host)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _pp(p):
    return None if p is None else C.byref(p)


def nf_codebook(bits: int) -> np.ndarray:
    out = np.zeros(1 << max(bits, 0) if 0 < bits <= 8 else 1, np.float32)
    _check(_lib.lq_nf_codebook(bits, out.ctypes.data), "lq_nf_codebook")
    return out


def codes_bytes(n: int, bits: int) -> int:
    return _lib.lq_codes_bytes(n, bits)


def storage_bits(n: int, cfg: Config) -> float:
    return _lib.lq_storage_bits(n, cfg)


def nf_quantize(x: torch.Tensor, cfg: Config, out=None):
    """Quantize(x, c): -> (codes_packed uint8, scale_idx uint8, v fp32), all on x's device; `out`: such a triple of the
    right sizes to write into instead of new tensors."""
    n = x.numel()
    nb = n // max(cfg.block, 1)
    ng = (nb + max(cfg.scale_block, 1) - 1) // max(cfg.scale_block, 1)
    if out is not None:
        codes, sidx, v = out
        if codes.numel() < codes_bytes(n, cfg.bits) or sidx.numel() < nb or v.numel() < ng:
            raise ValueError("nf_quantize: output buffers too small")
        _dev(codes, torch.uint8, "codes"), _dev(sidx, torch.uint8, "scale_idx"), _dev(v, torch.float32, "v")
    else:
        codes = torch.empty(max(codes_bytes(n, cfg.bits), 1), dtype=torch.uint8, device=x.device)
        sidx = torch.empty(max(nb, 1), dtype=torch.uint8, device=x.device)
        v = torch.empty(max(ng, 1), dtype=torch.float32, device=x.device)
    _check(_lib.lq_nf_quantize(_dev(x, torch.float32, "x"), n, cfg, codes.data_ptr(), sidx.data_ptr(), v.data_ptr(),
                               _stream()), "lq_nf_quantize")
    return codes, sidx, v


def nf_dequantize(codes: torch.Tensor, scale_idx: torch.Tensor, v: torch.Tensor, n: int, cfg: Config,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device=codes.device)
    _check(_lib.lq_nf_dequantize(_dev(codes, torch.uint8, "codes"), _dev(scale_idx, torch.uint8, "scale_idx"),
                                 _dev(v, torch.float32, "v"), n, cfg, _dev(out, torch.float32, "out"), _stream()),
           "lq_nf_dequantize")
    return out


def pack_scale_indices(scale_idx: torch.Tensor, scale_bits: int) -> torch.Tensor:
    """One-byte scale indices -> bit stream of scale_bits bits each."""
    out = torch.empty(max(codes_bytes(scale_idx.numel(), scale_bits), 1), dtype=torch.uint8, device=scale_idx.device)
    _check(_lib.lq_pack_scale_indices(_dev(scale_idx, torch.uint8, "scale_idx"), scale_idx.numel(), scale_bits,
                                      out.data_ptr(), _stream()), "lq_pack_scale_indices")
    return out


def unpack_scale_indices(packed: torch.Tensor, count: int, scale_bits: int) -> torch.Tensor:
    out = torch.empty(max(count, 1), dtype=torch.uint8, device=packed.device)
    _check(_lib.lq_unpack_scale_indices(_dev(packed, torch.uint8, "packed"), count, scale_bits, out.data_ptr(),
                                        _stream()), "lq_unpack_scale_indices")
    return out


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(nbytes + 256, dtype=torch.uint8, device=device)


def _aligned_ptr(ws: torch.Tensor) -> int:
    p = ws.data_ptr()
    return (p + 255) & ~255


def _bytes_left(ws: torch.Tensor) -> int:
    """Bytes of a workspace from its first aligned one on; none where it ends before that."""
    if not ws.is_cuda:
        raise TypeError("workspace: need a tensor on the GPU")
    return max(0, ws.numel() - (_aligned_ptr(ws) - ws.data_ptr()))


def factorize(a: torch.Tensor, rank: int, row_w=None, col_w=None, seed: int = 0, params: SvdParams | None = None,
              workspace: torch.Tensor | None = None):
    """Factorize(A, F, r): -> (L1 d x r, L2 r x k, sigma numpy float64[r])."""
    d, k = a.shape
    need = _lib.lq_factorize_workspace_bytes(d, k, rank, _pp(params))
    ws = workspace if workspace is not None else _workspace(need, a.device)
    l1 = torch.empty((d, rank), dtype=torch.float32, device=a.device)
    l2 = torch.empty((rank, k), dtype=torch.float32, device=a.device)
    sigma = np.zeros(max(rank, 1))
    _check(_lib.lq_factorize(_dev(a, torch.float32, "a"), d, k, rank, _dev(row_w, torch.float32, "row_w"),
                             _dev(col_w, torch.float32, "col_w"), seed, _pp(params), l1.data_ptr(), l2.data_ptr(),
                             sigma.ctypes.data, _aligned_ptr(ws), _bytes_left(ws),
                             _stream()), "lq_factorize")
    return l1, l2, sigma


def decompose(w: torch.Tensor, rank: int, cfg: Config, iters: int, early_stop: bool = False, row_w=None, col_w=None,
              seed: int = 0, params: SvdParams | None = None, want_dense: bool = False,
              workspace: torch.Tensor | None = None):
    """LQ(W, F, c, r): -> dict(L1, L2, codes, scale_idx, v, Q, err, trace, iters_done, sigma)."""
    d, k = w.shape
    n = d * k
    nb = n // max(cfg.block, 1)
    ng = (nb + max(cfg.scale_block, 1) - 1) // max(cfg.scale_block, 1)
    need = _lib.lq_decompose_workspace_bytes(d, k, rank, _pp(params))
    ws = workspace if workspace is not None else _workspace(need, w.device)
    dev = w.device
    out = dict(L1=torch.empty((d, max(rank, 1)), dtype=torch.float32, device=dev),
               L2=torch.empty((max(rank, 1), k), dtype=torch.float32, device=dev),
               codes=torch.empty(max(codes_bytes(n, cfg.bits), 1), dtype=torch.uint8, device=dev),
               scale_idx=torch.empty(max(nb, 1), dtype=torch.uint8, device=dev),
               v=torch.empty(max(ng, 1), dtype=torch.float32, device=dev),
               Q=torch.empty((d, k), dtype=torch.float32, device=dev) if want_dense else None)
    err = C.c_double(float("nan"))
    done = C.c_int32(0)
    trace = np.full(max(iters, 1), np.nan)
    sigma = np.zeros(max(rank, 1))
    _check(_lib.lq_decompose(_dev(w, torch.float32, "w"), d, k, rank, cfg, iters, int(early_stop),
                             _dev(row_w, torch.float32, "row_w"), _dev(col_w, torch.float32, "col_w"), seed,
                             _pp(params), out["L1"].data_ptr(), out["L2"].data_ptr(), out["codes"].data_ptr(),
                             out["scale_idx"].data_ptr(), out["v"].data_ptr(),
                             None if out["Q"] is None else out["Q"].data_ptr(), C.addressof(err), trace.ctypes.data,
                             C.addressof(done), sigma.ctypes.data, _aligned_ptr(ws), _bytes_left(ws), _stream()), "lq_decompose")
    out.update(err=err.value, trace=trace, iters_done=done.value, sigma=sigma)
    return out


def error_table_workspace(d: int, k: int, rank: int, n_cfgs: int, params: SvdParams | None = None, device="cuda"):
    return _workspace(_lib.lq_error_table_workspace_bytes(d, k, rank, n_cfgs, _pp(params)), device)


def error_table(w: torch.Tensor, rank: int, cfgs, iters: int, early_stop: bool = False, row_w=None, col_w=None,
                seed: int = 0, params: SvdParams | None = None, workspace: torch.Tensor | None = None,
                want_trace: bool = False):
    """Algorithm 3 inner loops for one matrix: -> (err_sq, storage_bits[, trace]) numpy float64."""
    d, k = w.shape
    arr = (Config * max(len(cfgs), 1))(*cfgs)
    ws = workspace if workspace is not None else error_table_workspace(d, k, rank, len(cfgs), params, w.device)
    e = np.zeros(max(len(cfgs), 1))
    s = np.zeros(max(len(cfgs), 1))
    tr = np.full((max(len(cfgs), 1), max(iters, 1)), np.nan) if want_trace else None
    _check(_lib.lq_error_table(_dev(w, torch.float32, "w"), d, k, rank, C.addressof(arr), len(cfgs), iters,
                               int(early_stop), _dev(row_w, torch.float32, "row_w"),
                               _dev(col_w, torch.float32, "col_w"), seed, _pp(params), e.ctypes.data, s.ctypes.data,
                               None if tr is None else tr.ctypes.data, _aligned_ptr(ws), _bytes_left(ws), _stream()), "lq_error_table")
    return (e, s, tr) if want_trace else (e, s)


def fisher_row_col(f: torch.Tensor):
    """RowAverage / ColAverage of sqrt(F) (Algorithm 4) as Fisher-scale vectors for row_w / col_w."""
    d, k = f.shape
    ws = _workspace(_lib.lq_fisher_row_col_workspace_bytes(d, k), f.device)
    row_w = torch.empty(d, dtype=torch.float32, device=f.device)
    col_w = torch.empty(k, dtype=torch.float32, device=f.device)
    _check(_lib.lq_fisher_row_col(_dev(f, torch.float32, "f"), d, k, row_w.data_ptr(), col_w.data_ptr(),
                                  _aligned_ptr(ws), _bytes_left(ws), _stream()),
           "lq_fisher_row_col")
    return row_w, col_w


def release_streams() -> None:
    """Destroys the idle HIP streams the library keeps for lq_error_table's interleaved sub-batches."""
    _check(_lib.lq_release_streams(), "lq_release_streams")


def profile_enable(on: bool) -> None:
    _check(_lib.lq_profile_enable(1 if on else 0), "lq_profile_enable")


def profile_reset() -> None:
    _check(_lib.lq_profile_reset(), "lq_profile_reset")


def profile_read() -> dict:
    """-> {kernel class name: (total_ms, launches, algorithmic work)} for classes that were launched."""
    out = {}
    for cls in range(_lib.lq_profile_num_classes()):
        ms, n, wk = C.c_double(0), C.c_int64(0), C.c_double(0)
        _check(_lib.lq_profile_read(cls, C.addressof(ms), C.addressof(n), C.addressof(wk)), "lq_profile_read")
        if n.value:
            out[_lib.lq_profile_class_name(cls).decode()] = (ms.value, n.value, wk.value)
    return out


def matmul_workspace(m: int, d: int, k: int, rank: int, device="cuda") -> torch.Tensor:
    return _workspace(_lib.lq_matmul_workspace_bytes(m, d, k, rank), device)


def matmul(x: torch.Tensor, codes: torch.Tensor, scale_idx: torch.Tensor, v: torch.Tensor, cfg: Config, k: int,
           l1: torch.Tensor | None = None, l2: torch.Tensor | None = None, precision: int = 0,
           out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Y = X (Q + L1 L2) with Q (d x k) in quantized form, dequantized inside the GEMM."""
    m, d = x.shape
    rank = 0 if l1 is None else l1.shape[1]
    if out is None:
        out = torch.empty((m, k), dtype=torch.float32, device=x.device)
    ws = workspace
    if ws is None:
        ws = _workspace(_lib.lq_matmul_workspace_bytes_precision(m, d, k, rank, precision), x.device)
    _check(_lib.lq_matmul(_dev(x, torch.float32, "x"), m, d, k, _dev(codes, torch.uint8, "codes"),
                          _dev(scale_idx, torch.uint8, "scale_idx"), _dev(v, torch.float32, "v"), cfg,
                          _dev(l1, torch.float32, "l1"), _dev(l2, torch.float32, "l2"), rank, precision,
                          _dev(out, torch.float32, "out"), _aligned_ptr(ws), _bytes_left(ws), _stream()), "lq_matmul")
    return out


def matmul_few_rows_static(x: torch.Tensor, codes: torch.Tensor, scale_idx: torch.Tensor, v: torch.Tensor, cfg: Config,
                           k: int, l1: torch.Tensor | None = None, l2: torch.Tensor | None = None,
                           out: torch.Tensor | None = None) -> torch.Tensor:
    """Y = X (Q + L1 L2) for at most 8 rows of X through the entry point that allocates nothing: its partial sums live
    in the library's fixed device array (lq_matmul_few_rows_static).  `out`: m x k fp32 tensor to write into."""
    m, d = x.shape
    rank = 0 if l1 is None else l1.shape[1]
    if out is None:
        out = torch.empty((m, k), dtype=torch.float32, device=x.device)
    _check(_lib.lq_matmul_few_rows_static(_dev(x, torch.float32, "x"), m, d, k, _dev(codes, torch.uint8, "codes"),
                                          _dev(scale_idx, torch.uint8, "scale_idx"), _dev(v, torch.float32, "v"), cfg,
                                          _dev(l1, torch.float32, "l1"), _dev(l2, torch.float32, "l2"), rank,
                                          _dev(out, torch.float32, "out"), _stream()), "lq_matmul_few_rows_static")
    return out


def _type_code(dtype, name: str) -> int:
    if dtype not in T_DTYPES:
        raise TypeError(f"{name}: need torch.float32 or torch.bfloat16")
    return T_DTYPES[dtype]


def _dtype(t: torch.Tensor, name: str) -> int:
    if not (isinstance(t, torch.Tensor) and t.dtype in T_DTYPES):
        raise TypeError(f"{name}: need a tensor of torch.float32 or torch.bfloat16")
    return T_DTYPES[t.dtype]


def _rows(t, dtype, name):
    """Pointer and row stride of a matrix whose rows are contiguous."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.dim() == 2 and
            (t.stride(1) == 1 or t.shape[1] == 1) and (t.shape[0] == 1 or t.stride(0) >= t.shape[1])):
        raise TypeError(f"{name}: need a {dtype} matrix with contiguous rows on the GPU")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _space(ws):
    """Aligned start and bytes of a caller's workspace: the kernels write there, so it has to be one piece of the GPU's memory."""
    if not (isinstance(ws, torch.Tensor) and ws.is_cuda and ws.dtype == torch.uint8 and ws.is_contiguous()):
        raise TypeError("workspace: need a contiguous torch.uint8 tensor on the GPU")
    return _aligned_ptr(ws), _bytes_left(ws)


def _shaped(t, shape, name):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, need {tuple(shape)}")


def _stored(codes, scale_idx, v, cfg, n):
    """The quantized component's buffers have to hold n weights: the kernels read them by the configuration's sizes."""
    if (codes.numel() < codes_bytes(n, cfg.bits) or scale_idx.numel() * max(cfg.block, 1) < n or
            v.numel() * max(cfg.block, 1) * max(cfg.scale_block, 1) < n):
        raise ValueError("codes, scale_idx or v too small for the matrix")


def dropout(x: torch.Tensor, p: float, seed: int, offset: int = 0, out: torch.Tensor | None = None) -> torch.Tensor:
    """y = kept ? x / (1 - p) : 0 with the mask of (seed, offset, element); the gradient is the same call on dy.
    `out`: tensor like x to write into, x itself among them."""
    code = _dtype(x, "x")
    if out is None:
        out = torch.empty_like(x)
    _shaped(out, x.shape, "out")
    _check(_lib.lq_dropout(_dev(x, x.dtype, "x"), x.numel(), code, p, seed, offset, _dev(out, x.dtype, "out"), _stream()),
           "lq_dropout")
    return out


def cross_entropy_workspace(n: int, d: int, vocab: int, dtype=torch.float32, want_dx: bool = True, want_dw: bool = False,
                            device="cuda") -> torch.Tensor:
    return _workspace(_lib.lq_cross_entropy_workspace_bytes(n, d, vocab, _type_code(dtype, "dtype"), int(want_dx), int(want_dw)), device)


def cross_entropy(x: torch.Tensor, w: torch.Tensor, targets: torch.Tensor, mean: bool = True, want_dx: bool = True,
                  want_dw: bool = False, workspace: torch.Tensor | None = None):
    """Softmax cross entropy of the logits X W^T, which are never stored, against `targets` (rows with a target outside the
    vocabulary do not count): -> dict(loss, row_loss, lse, dx, dw), the gradients being those of `loss`, None if not wanted.
    Up to 128 rows, asking for dw may change the other outputs' last bits."""
    code = _dtype(x, "x")
    (xp, ldx), (wp, ldw) = _rows(x, x.dtype, "x"), _rows(w, x.dtype, "w")
    n, d = x.shape
    vocab = w.shape[0]
    _shaped(w, (vocab, d), "w")
    _shaped(targets, (n,), "targets")
    ws = workspace if workspace is not None else cross_entropy_workspace(n, d, vocab, x.dtype, want_dx, want_dw, x.device)
    out = dict(loss=torch.empty((), dtype=torch.float32, device=x.device),
               row_loss=torch.empty(n, dtype=torch.float32, device=x.device),
               lse=torch.empty(n, dtype=torch.float32, device=x.device),
               dx=torch.empty((n, d), dtype=x.dtype, device=x.device) if want_dx else None,
               dw=torch.empty((vocab, d), dtype=x.dtype, device=x.device) if want_dw else None)
    ptr = {name: None if t is None else t.data_ptr() for name, t in out.items()}
    _check(_lib.lq_cross_entropy(xp, ldx, wp, ldw, _dev(targets, torch.int64, "targets"), n, d, vocab, code, int(mean), ptr["loss"],
                                 ptr["row_loss"], ptr["lse"], ptr["dx"], ptr["dw"], *_space(ws), _stream()), "lq_cross_entropy")
    return out


def adapter_workspace(m: int, d: int, k: int, rank: int, dtype=torch.float32, backward: bool = False, device="cuda") -> torch.Tensor:
    return _workspace(_lib.lq_adapter_workspace_bytes(m, d, k, rank, _type_code(dtype, "dtype"), int(backward)), device)


def adapter_forward(x: torch.Tensor, codes: torch.Tensor, scale_idx: torch.Tensor, v: torch.Tensor, cfg: Config,
                    l1: torch.Tensor, l2: torch.Tensor, p: float = 0.0, seed: int = 0, offset: int = 0,
                    workspace: torch.Tensor | None = None):
    """T = drop(X) L1, Y = X Q + T L2: -> (Y, T); T is what adapter_backward takes.  Without a need for T or dropout, few rows of a
    large layer go faster through matmul, which decodes no copy of Q."""
    code = _dtype(x, "x")
    m, d = x.shape
    rank, k = l2.shape
    _shaped(l1, (d, rank), "l1")
    _stored(codes, scale_idx, v, cfg, d * k)
    ws = workspace if workspace is not None else adapter_workspace(m, d, k, rank, x.dtype, False, x.device)
    y = torch.empty((m, k), dtype=x.dtype, device=x.device)
    t = torch.empty((m, rank), dtype=torch.float32, device=x.device)
    _check(_lib.lq_adapter_forward(_dev(x, x.dtype, "x"), m, d, k, _dev(codes, torch.uint8, "codes"),
                                   _dev(scale_idx, torch.uint8, "scale_idx"), _dev(v, torch.float32, "v"), cfg,
                                   _dev(l1, torch.float32, "l1"), _dev(l2, torch.float32, "l2"), rank, code, p, seed, offset,
                                   y.data_ptr(), t.data_ptr(), *_space(ws), _stream()), "lq_adapter_forward")
    return y, t


def adapter_backward(dy: torch.Tensor, x: torch.Tensor, codes: torch.Tensor, scale_idx: torch.Tensor, v: torch.Tensor, cfg: Config,
                     l1: torch.Tensor, l2: torch.Tensor, t: torch.Tensor, p: float = 0.0, seed: int = 0, offset: int = 0,
                     want_dx: bool = True, workspace: torch.Tensor | None = None):
    """Gradients of adapter_forward with the same p, seed and offset: -> (dX or None, dL1, dL2)."""
    code = _dtype(x, "x")
    m, d = x.shape
    rank, k = l2.shape
    _shaped(dy, (m, k), "dy")
    _shaped(l1, (d, rank), "l1")
    _shaped(t, (m, rank), "t")
    _stored(codes, scale_idx, v, cfg, d * k)
    ws = workspace if workspace is not None else adapter_workspace(m, d, k, rank, x.dtype, True, x.device)
    dx = torch.empty((m, d), dtype=x.dtype, device=x.device) if want_dx else None
    dl1, dl2 = torch.empty_like(l1), torch.empty_like(l2)
    _check(_lib.lq_adapter_backward(_dev(dy, x.dtype, "dy"), _dev(x, x.dtype, "x"), m, d, k, _dev(codes, torch.uint8, "codes"),
                                    _dev(scale_idx, torch.uint8, "scale_idx"), _dev(v, torch.float32, "v"), cfg,
                                    _dev(l1, torch.float32, "l1"), _dev(l2, torch.float32, "l2"), rank, code,
                                    _dev(t, torch.float32, "t"), p, seed, offset, None if dx is None else dx.data_ptr(),
                                    dl1.data_ptr(), dl2.data_ptr(), *_space(ws), _stream()), "lq_adapter_backward")
    return dx, dl1, dl2


FP8 = torch.float8_e4m3fn


def _blocks(n: int) -> int:
    return -(-n // 128)


def _codes_like(rows: int, cols: int, device) -> torch.Tensor:
    """rows x cols codes whose rows begin on 16-byte addresses; long rows on lines of 128 bytes, a block each."""
    unit = 128 if cols >= 1024 else 16
    return torch.empty((rows, -(-cols // unit) * unit), dtype=FP8, device=device)[:, :cols]


def _scales_like(rows: int, cols: int, tiles: bool, device) -> torch.Tensor:
    """Scales of rows x cols codes: of tiles row-major, of rows with the rows next to one another."""
    if tiles:
        return torch.empty((_blocks(rows), _blocks(cols)), dtype=torch.float32, device=device)
    return torch.empty_strided((rows, _blocks(cols)), (1, rows), dtype=torch.float32, device=device)


def fp8_quantize(x: torch.Tensor, tiles: bool = False, both: bool = False):
    """Codes (torch.float8_e4m3fn) and fp32 scales of a matrix in blocks of 128 along its rows (scale: rows x blocks), or in tiles of
    128 x 128 (scale: blocks x blocks): -> (codes, scale), or with both=True those of its transpose as well, from the same pass:
    (codes, scale, codes_t, scale_t)."""
    code = _dtype(x, "x")
    xp, ldx = _rows(x, x.dtype, "x")
    m, d = x.shape
    _here(x)
    q = _codes_like(m, d, x.device)
    scale = _scales_like(m, d, tiles, x.device)
    qt = _codes_like(d, m, x.device) if both else None
    scale_t = _scales_like(d, m, False, x.device) if both and not tiles else None
    _check(_lib.lq_fp8_quantize(xp, m, d, ldx, code, int(tiles), q.data_ptr(), q.stride(0), scale.data_ptr(),
                                qt.data_ptr() if both else None, qt.stride(0) if both else 0,
                                None if scale_t is None else scale_t.data_ptr(), _stream()), "lq_fp8_quantize")
    return (q, scale, qt, scale.t() if tiles else scale_t) if both else (q, scale)


def _here(*tensors):
    """The calls launch on the current device's stream: operands elsewhere are refused."""
    current = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != current:
            raise ValueError(f"tensor on {t.device}, the current device is cuda:{current}")


def _fp8_matrix(codes, scale, name):
    """lq_fp8_matrix of codes and scales; the scales' shape says whether they are of rows or of tiles."""
    if not (isinstance(codes, torch.Tensor) and codes.is_cuda and codes.dtype == FP8 and codes.dim() == 2):
        raise TypeError(f"{name}: need a {FP8} matrix on the GPU")
    if not (isinstance(scale, torch.Tensor) and scale.is_cuda and scale.dtype == torch.float32 and scale.dim() == 2):
        raise TypeError(f"{name}: need a torch.float32 matrix of scales on the GPU")
    _here(codes, scale)
    rows, cols = codes.shape
    ld = codes.stride(0) if rows > 1 else -(-cols // 16) * 16
    if (codes.stride(1) != 1 and cols > 1) or ld % 16 or ld < cols or codes.data_ptr() % 16:
        raise ValueError(f"{name}: rows have to begin on 16-byte addresses and be contiguous (as fp8_quantize lays them out)")
    if tuple(scale.shape) not in ((rows, _blocks(cols)), (_blocks(rows), _blocks(cols))):
        raise ValueError(f"{name}: scales of shape {tuple(scale.shape)} for {rows} x {cols} codes")
    return Fp8Matrix(codes.data_ptr(), ld, scale.data_ptr(), scale.stride(0), scale.stride(1), int(scale.shape[0] != rows))


def fp8_matmul(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor, out: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Y = A B^T (bf16) of two matrices in 8 bits, A m x k and B n x k, each with scales of rows or of tiles (fp8_quantize)."""
    am, bm = _fp8_matrix(a, a_scale, "a"), _fp8_matrix(b, b_scale, "b")
    (m, k), n = a.shape, b.shape[0]
    _shaped(b, (n, k), "b")
    if out is None:
        out = torch.empty((m, n), dtype=torch.bfloat16, device=a.device)
    _shaped(out, (m, n), "out")
    yp, ldy = _rows(out, torch.bfloat16, "out")
    _here(out, workspace)
    ws = workspace if workspace is not None else _workspace(_lib.lq_fp8_matmul_workspace_bytes(m, n, k), a.device)
    _check(_lib.lq_fp8_matmul(C.byref(am), C.byref(bm), m, n, k, yp, ldy, *_space(ws), _stream()), "lq_fp8_matmul")
    torch.autograd.graph.increment_version(out)              # for graphs that have saved what lay there
    return out


def fp8_workspace(m: int, n: int, k: int, backward: bool = False, want_dx: bool = True, want_dw: bool = True, device="cuda") -> torch.Tensor:
    """Workspace of fp8_forward, or of fp8_backward, for m rows through a layer of k inputs and n outputs."""
    return _workspace(_lib.lq_fp8_backward_workspace_bytes(m, n, k, int(want_dx), int(want_dw)) if backward else
                      _lib.lq_fp8_forward_workspace_bytes(m, n, k), device)


def fp8_forward(x: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Y = X W^T (bf16) with X (m x k, fp32 or bf16) quantized along its rows inside the call and W (n x k) in 8 bits."""
    code = _dtype(x, "x")
    xp, ldx = _rows(x, x.dtype, "x")
    wm = _fp8_matrix(w, w_scale, "w")
    _here(x, workspace)
    (m, k), n = x.shape, w.shape[0]
    _shaped(w, (n, k), "w")
    ws = workspace if workspace is not None else fp8_workspace(m, n, k, device=x.device)
    y = torch.empty((m, n), dtype=torch.bfloat16, device=x.device)
    _check(_lib.lq_fp8_forward(xp, ldx, code, C.byref(wm), m, n, k, y.data_ptr(), *_space(ws), _stream()), "lq_fp8_forward")
    return y


def fp8_backward(dy: torch.Tensor, x: torch.Tensor | None, wt: torch.Tensor | None = None, wt_scale: torch.Tensor | None = None,
                 want_dx: bool = True, want_dw: bool = True, workspace: torch.Tensor | None = None):
    """Gradients of fp8_forward, bf16: -> (dX = dY W or None, dW = dY^T X or None).  wt, wt_scale: W^T (k x n) in 8 bits, as
    fp8_quantize(w, tiles=True, both=True) gives it, for dX; x for dW."""
    code = _dtype(dy, "dy")
    yp, ldy = _rows(dy, dy.dtype, "dy")
    m, n = dy.shape
    _here(dy, x if want_dw else None, workspace)
    if not (want_dx or want_dw):
        raise ValueError("fp8_backward: neither gradient is wanted")
    if (want_dx and wt is None) or (want_dw and x is None):
        raise ValueError("fp8_backward: dX needs wt, dW needs x")
    xp, ldx, xcode, wm = None, 0, 0, None
    if want_dx:
        wm = _fp8_matrix(wt, wt_scale, "wt")
        k = wt.shape[0]
        _shaped(wt, (k, n), "wt")
    if want_dw:
        xcode = _dtype(x, "x")
        xp, ldx = _rows(x, x.dtype, "x")
        k = wt.shape[0] if want_dx else x.shape[1]
        _shaped(x, (m, k), "x")
    ws = workspace if workspace is not None else fp8_workspace(m, n, k, True, want_dx, want_dw, dy.device)
    dx = torch.empty((m, k), dtype=torch.bfloat16, device=dy.device) if want_dx else None
    dw = torch.empty((n, k), dtype=torch.bfloat16, device=dy.device) if want_dw else None
    _check(_lib.lq_fp8_backward(yp, ldy, code, xp, ldx, xcode, None if wm is None else C.byref(wm), m, n, k,
                                None if dx is None else dx.data_ptr(), None if dw is None else dw.data_ptr(), *_space(ws), _stream()),
           "lq_fp8_backward")
    return dx, dw


def _gradients(grads):
    """Addresses, sizes and types of gradients, checked: there may be hundreds, so the checks are made where they are cheap and told
    apart only where one fails."""
    places, sizes, types = [], [], []
    for g in grads[:1]:
        _dtype(g, "grads"), _dev(g, g.dtype, "grads")
    current = torch._C._cuda_getDevice() if grads else 0
    for g in grads:
        code = T_DTYPES.get(g.dtype) if isinstance(g, torch.Tensor) else None
        if code is None or g.get_device() != current or not g.is_contiguous():
            _dtype(g, "grads"), _dev(g, g.dtype, "grads"), _here(g)
        places.append(g.data_ptr())
        sizes.append(g.numel())
        types.append(code)
    return places, sizes, types


def grad_norm(grads, max_norm: float = float("inf"), workspace: torch.Tensor | None = None):
    """2-norm of all gradients together and the factor that brings it to max_norm at most (NaN where the norm is not finite, which makes
    AdamW.step change nothing): -> (norm, coef), fp32 of no dimensions on the GPU."""
    grads = list(grads)
    places, sizes, types = _gradients(grads)
    total = sum(sizes)
    table = struct.pack("QqQ" * len(grads), *[x for entry in zip(places, sizes, types) for x in entry])      # lq_gradient[]
    device = grads[0].device if grads else "cuda"
    if workspace is None:                        # behind the results, in one piece with them: 8 bytes for every 2048 values at most
        need = (total // 2048 + len(grads) + 32) * 8
        out = torch.empty(64 + need // 4, dtype=torch.float32, device=device)
        space = (out.data_ptr() + 256, need)
    else:
        _here(workspace)
        out, space = torch.empty(2, dtype=torch.float32, device=device), _space(workspace)
    _check(_lib.lq_grad_norm(table, len(grads), max_norm, out.data_ptr(), *space, _stream()), "lq_grad_norm")
    return out[0], out[1]


def _one(t, dtype, name):
    """Address of a tensor of one element on the current device."""
    place = _dev(t, dtype, name)
    if t.numel() != 1:
        raise ValueError(f"{name}: need one element")
    _here(t)
    return place


class AdamW:
    """AdamW over many tensors in one call, with states in 32 bits or in 8 (lq_adamw).

    params: contiguous GPU tensors of fp32 or bf16, updated in place.  copies: bf16 tensors (or None) that take each fp32 parameter's
    rounded value in the same pass.  States start at zero and lie in `buffers` ("m", "v", with bits=8 also "m_scale", "v_scale"), tensor
    after tensor, each from a multiple of 256 on.  `t` counts the steps taken: an int, or with device_step=True an int64 tensor of one
    element on the GPU, so that a captured step counts on when it is replayed.  seed: of the rounding of 8-bit states.  buffers, t and seed
    are what a checkpoint needs: copied into, or replaced by others of their type and size on the GPU, which the next step takes up.  A
    captured step goes on with the tensors it was captured with, which have to live as long: copy into those.  The order of params belongs to
    the rounding of 8-bit states."""

    def __init__(self, params, bits: int = 32, copies=None, seed: int = 0, device_step: bool = False):
        if bits not in (8, 32):
            raise ValueError("bits: need 8 or 32")
        self.params, self.bits, self.seed = list(params), bits, seed
        if not self.params:
            raise ValueError("params: none given")
        self.copies = list(copies) if copies is not None else [None] * len(self.params)
        if len(self.copies) != len(self.params):
            raise ValueError("copies: need one for each parameter")
        device = self.params[0].device
        starts, total = [], 0
        for p in self.params:
            starts.append(total)
            total += -(-p.numel() // 256) * 256
        self._sizes = [p.numel() for p in self.params]
        self._table, self._params = (AdamWTensor * len(self.params))(), AdamWParams()
        self._columns = np.frombuffer(self._table, dtype=np.dtype(AdamWTensor))
        self._held = self.params + [c for c in self.copies if c is not None]
        self._describe()
        self._starts, state = np.array(starts, dtype=np.uint64), FP8 if bits == 8 else torch.float32
        self._states = {name: (state, total, 1 if bits == 8 else 4) for name in ("m", "v")}        # type, size, bytes for a value of p
        if bits == 8:
            self._states.update({name: (torch.float32, total // 256, 1 / 64) for name in ("m_scale", "v_scale")})
        self.buffers = {name: torch.zeros(n, dtype=dtype, device=device) for name, (dtype, n, _) in self._states.items()}
        self._used = [("m", lambda: None, 0, 0)]             # nothing yet: the first step looks
        self.t = torch.zeros((), dtype=torch.int64, device=device) if device_step else 0

    def _describe(self):
        """Parameters and copies into the table, checked."""
        self._places = None                                  # none known, should one be refused
        for entry, p, c, n in zip(self._table, self.params, self.copies, self._sizes):
            _dtype(p, "params")
            entry.p, entry.n, entry.p_dtype = _dev(p, p.dtype, "params"), n, T_DTYPES[p.dtype]
            if p.device != self.params[0].device:
                raise ValueError("params: on different devices")
            if p.numel() != n:
                raise ValueError("params: another size than at first")
            if c is not None:
                _shaped(c, p.shape, "copies")
            entry.copy = _dev(c, torch.bfloat16, "copies")
        self._places = [x.data_ptr() for x in self._held]

    def _find_states(self):
        """The states' addresses into the table, checked: others may lie in `buffers` than at the last step."""
        used = []
        for name, (dtype, n, _) in self._states.items():
            buffer = self.buffers.get(name)
            if buffer is None:
                raise TypeError(f"buffers: no {name}")
            place = _dev(buffer, dtype, name)
            if buffer.numel() != n:
                raise ValueError(f"buffers: {name} has {buffer.numel()} elements, needs {n}")
            _here(buffer)
            used.append((name, weakref.ref(buffer), place, n))
        for name, _, place, _ in used:
            self._columns[name] = place + (self._starts * self._states[name][2]).astype(np.uint64)
        self._used = used

    def step(self, grads, lr, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, coef: torch.Tensor | None = None) -> None:
        """One step.  grads: one for each parameter, fp32 or bf16, of its size.  lr: a number, or an fp32 tensor of one element on the GPU.
        coef: such a tensor that multiplies every gradient (grad_norm's); where it is not finite, nothing but `t` changes."""
        grads = list(grads)
        places, sizes, types = _gradients(grads)
        if sizes != self._sizes:
            raise ValueError("grads: need one for each parameter, of its size")
        _here(self.params[0])
        now = [x.data_ptr() for x in self._held]
        if now != self._places:                              # parameters that have moved
            self._describe()
        buffers = self.buffers
        for name, ref, place, n in self._used:               # the same tensors, where they were: not others at their address
            buffer = buffers.get(name)
            if buffer is None or buffer is not ref() or buffer.data_ptr() != place or buffer.numel() != n:
                self._find_states()
                break
        if len(grads) > 16:
            self._columns["g"], self._columns["g_dtype"] = places, types
        else:
            for entry, place, code in zip(self._table, places, types):
                entry.g, entry.g_dtype = place, code
        on_device = isinstance(self.t, torch.Tensor)
        if not on_device and torch._C._cuda_isCurrentStreamCapturing():
            raise RuntimeError("a captured step needs device_step=True: a replay would repeat this step's number")
        h = self._params
        (h.beta1, h.beta2), h.eps, h.weight_decay, h.seed = betas, eps, weight_decay, self.seed
        h.lr_device = h.step_device = None                   # the last step's
        if isinstance(lr, torch.Tensor):
            h.lr_device = _one(lr, torch.float32, "lr")
        else:
            h.lr = lr
        scale = None if coef is None else _one(coef, torch.float32, "coef")
        if on_device:
            h.step_device = _one(self.t, torch.int64, "t")
            self.t += 1
        else:
            h.step = self.t + 1
        status = _lib.lq_adamw(C.addressof(self._table), len(grads), self.bits, C.byref(h), scale, _stream())
        if status != 0 and on_device:
            self.t -= 1                                      # a refused step does not count
        _check(status, "lq_adamw")
        if not on_device:
            self.t += 1
        # a graph that has saved old values has to say so, and it saves what requires no gradient too
        torch.autograd.graph.increment_version(self._held)


def assign_configs(err: np.ndarray, storage: np.ndarray, budget_bits: float, node_limit: int = 0):
    """ILPSolve: -> (choice int32[n_matrices], total_err, total_storage, lower_bound).  Host only."""
    err = np.ascontiguousarray(err, np.float64)
    storage = np.ascontiguousarray(storage, np.float64)
    n, c = err.shape
    assert storage.shape == (n, c)
    choice = np.zeros(n, np.int32)
    te, ts, lb = C.c_double(0), C.c_double(0), C.c_double(0)
    _check(_lib.lq_assign_configs(err.ctypes.data, storage.ctypes.data, n, c, float(budget_bits), node_limit,
                                  choice.ctypes.data, C.addressof(te), C.addressof(ts), C.addressof(lb)),
           "lq_assign_configs")
    return choice, te.value, ts.value, lb.value


def lq_lora_decompose(matrices, rank: int, cfgs, bits_per_weight: float, iters: int, fishers=None, seed: int = 0,
                      params: SvdParams | None = None):
    """Algorithm 1 without the finetuning: error tables of all matrices (GetConfig, Algorithm 3), the assignment under
    the budget bits_per_weight * (total number of weights), then the decomposition of every matrix with its chosen
    configuration.  matrices: list of fp32 GPU tensors; fishers: None or a list of (row_w, col_w) pairs.
    -> (choice, list of lq.decompose results, err table, storage table)."""
    n = len(matrices)
    err = np.zeros((n, len(cfgs)))
    sto = np.zeros((n, len(cfgs)))
    for i, w in enumerate(matrices):
        rw, cw = fishers[i] if fishers is not None else (None, None)
        err[i], sto[i] = error_table(w, rank, cfgs, iters, row_w=rw, col_w=cw, seed=seed, params=params)
    budget = bits_per_weight * sum(w.numel() for w in matrices)
    choice, _, _, _ = assign_configs(err, sto, budget)
    outs = []
    for i, w in enumerate(matrices):
        rw, cw = fishers[i] if fishers is not None else (None, None)
        outs.append(decompose(w, rank, cfgs[choice[i]], iters, row_w=rw, col_w=cw, seed=seed, params=params))
    return choice, outs, err, sto

"""Thin ctypes binding over the C ABI of include/rtn.h.

Argument marshalling only (plain calls of the linear layer: in the native module): every step
of the path runs in the HIP kernels of the shared library.  PyTorch supplies device memory and
the current stream, nothing else.  There is no fallback: if the library cannot be loaded, importing this module raises.
"""
from __future__ import annotations

import collections
import ctypes as C
import os
import sysconfig
import warnings

import torch

from . import build as _build

RTN_SCALE_QMAX, RTN_SCALE_EQ2 = 0, 1
RTN_POLICY_FIRST, RTN_POLICY_LAST, RTN_POLICY_MIDDLE = 0, 1, 2
POLICY = {"first": RTN_POLICY_FIRST, "last": RTN_POLICY_LAST, "middle": RTN_POLICY_MIDDLE}


class RtnError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: rtn_status {status} ({_lib.rtn_status_str(status).decode()})")


class rtn_linear_cfg(C.Structure):
    _fields_ = [("path", C.c_int), ("prefetch", C.c_int), ("waves_n", C.c_int),
                ("waves_k", C.c_int), ("split_k", C.c_int), ("m_rows16", C.c_int), ("n_tiles16", C.c_int)]


class rtn_module(C.Structure):
    _fields_ = [("dev_A", C.c_void_p), ("M", C.c_int64), ("dev_qweight", C.c_void_p),
                ("dev_scales", C.c_void_p), ("N", C.c_int64), ("K", C.c_int64),
                ("bits", C.c_int), ("group_size", C.c_int), ("dev_C", C.c_void_p)]


class rtn_kv_cache(C.Structure):
    _fields_ = [("dev_k", C.c_void_p), ("dev_v", C.c_void_p), ("pages", C.c_int64), ("page_size", C.c_int), ("kv_heads", C.c_int),
                ("head_dim", C.c_int), ("dtype", C.c_int), ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("token_stride", C.c_int64)]


def _load() -> C.CDLL:
    path = _build.LIB_PATH
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built: run `python paper_2505_15909_amd/build.py` (or __graft_entry__.build()) first")
    lib = C.CDLL(path)
    vp, i64, ci, sz = C.c_void_p, C.c_int64, C.c_int, C.c_size_t
    lib.rtn_status_str.restype = C.c_char_p
    lib.rtn_status_str.argtypes = [ci]
    lib.rtn_layout_version.restype = ci
    lib.rtn_qweight_nbytes.restype = sz
    lib.rtn_qweight_nbytes.argtypes = [i64, i64, ci]
    lib.rtn_scales_nbytes.restype = sz
    lib.rtn_scales_nbytes.argtypes = [i64, i64, ci]
    lib.rtn_workspace_nbytes.restype = sz
    lib.rtn_workspace_nbytes.argtypes = [i64, i64, i64, ci, ci]
    lib.rtn_quantize.restype = ci
    lib.rtn_quantize.argtypes = [vp, i64, i64, ci, ci, ci, vp, vp, vp]
    lib.rtn_linear.restype = ci
    lib.rtn_linear.argtypes = [vp, i64, vp, vp, i64, i64, ci, ci, vp, vp, sz, vp]
    lib.rtn_linear_ex.restype = ci
    lib.rtn_linear_ex.argtypes = [vp, i64, vp, vp, i64, i64, ci, ci, vp, vp, sz, vp, C.POINTER(rtn_linear_cfg)]
    lib.rtn_linear_query.restype = ci
    lib.rtn_linear_query.argtypes = [i64, i64, i64, ci, ci, C.POINTER(rtn_linear_cfg)]
    lib.rtn_unpack.restype = ci
    lib.rtn_unpack.argtypes = [vp, i64, i64, ci, vp, vp]
    lib.rtn_dequantize.restype = ci
    lib.rtn_dequantize.argtypes = [vp, vp, i64, i64, ci, ci, vp, vp]
    lib.rtn_quantize_host_staging_nbytes.restype = sz
    lib.rtn_quantize_host_staging_nbytes.argtypes = [i64, i64]
    lib.rtn_quantize_from_host.restype = ci
    lib.rtn_quantize_from_host.argtypes = [vp, i64, i64, ci, ci, ci, vp, vp, vp, sz, i64, vp, vp]
    lib.rtn_gemm_fp16.restype = ci
    lib.rtn_gemm_fp16.argtypes = [vp, i64, vp, i64, i64, vp, vp, sz, vp]
    lib.rtn_dense_weight_nbytes.restype = sz
    lib.rtn_dense_weight_nbytes.argtypes = [i64, i64]
    lib.rtn_linear_dense.restype = ci
    lib.rtn_linear_dense.argtypes = [vp, i64, vp, vp, i64, i64, ci, ci, vp, vp, sz, vp, sz, vp]
    lib.rtn_layer_forward.restype = ci
    lib.rtn_layer_forward.argtypes = [C.POINTER(rtn_module), ci, vp, sz, vp]
    lib.rtn_quantize_asym.restype = ci
    lib.rtn_quantize_asym.argtypes = [vp, i64, i64, ci, ci, vp, vp, vp, vp]
    lib.rtn_dequantize_asym.restype = ci
    lib.rtn_dequantize_asym.argtypes = [vp, vp, vp, i64, i64, ci, ci, vp, vp]
    lib.rtn_linear_asym.restype = ci
    lib.rtn_linear_asym.argtypes = [vp, i64, vp, vp, vp, i64, i64, ci, ci, vp, vp, sz, vp]
    lib.rtn_grouped_forward.restype = ci
    lib.rtn_grouped_forward.argtypes = [C.POINTER(rtn_module), ci, vp, sz, vp]
    lib.rtn_problem_status.restype = ci
    lib.rtn_problem_status.argtypes = [i64, i64, ci, ci]
    lib.rtn_linear_validate.restype = ci
    lib.rtn_linear_validate.argtypes = [i64, i64, i64, ci, ci, sz, C.POINTER(rtn_linear_cfg)]
    lib.rtn_linear_noalloc.restype = ci
    lib.rtn_linear_noalloc.argtypes = [vp, i64, vp, vp, i64, i64, ci, ci, vp, vp]
    lib.rtn_bench_read_stream.restype = ci
    lib.rtn_bench_read_stream.argtypes = [vp, sz, ci, vp, vp]
    lib.rtn_plan_bits.restype = ci
    lib.rtn_plan_bits.argtypes = [ci, ci, ci, ci, ci, C.c_uint]
    lib.rtn_plan_effective_bits.restype = C.c_double
    lib.rtn_plan_effective_bits.argtypes = [ci, C.POINTER(i64), ci, ci, C.c_uint]
    lib.rtn_cache_plan.restype = ci
    lib.rtn_cache_plan.argtypes = [vp, vp, ci, ci, vp, i64, ci, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, vp]
    lib.rtn_rope_cache.restype = ci
    lib.rtn_rope_cache.argtypes = [vp, i64, i64, ci, vp, ci, i64, ci, vp, vp, vp, vp, C.c_float, C.POINTER(rtn_kv_cache), vp, vp]
    lib.rtn_paged_attention_workspace_nbytes.restype = sz
    lib.rtn_paged_attention_workspace_nbytes.argtypes = [i64, ci, ci, C.POINTER(rtn_kv_cache), ci]
    lib.rtn_paged_attention.restype = ci
    lib.rtn_paged_attention.argtypes = [vp, i64, i64, ci, C.POINTER(rtn_kv_cache), vp, i64, ci, vp, vp, ci, ci, C.c_float, C.c_float, ci,
                                        vp, vp, sz, vp]
    return lib


_lib = _load()


def _load_native():
    """The small calls in native code (csrc/rtn_native.cpp), or None where they were not built; without them a linear call takes 5.3 us of host time
    instead of 3.1.  They read PyTorch's own objects, so a module compiled for another PyTorch or Python is left alone."""
    if not os.path.exists(os.path.join(os.path.dirname(__file__), "_native.so")):
        return None
    here = f"torch {torch.__version__}, Python {sysconfig.get_python_version()}"
    try:
        from . import _native as module
        built_for = module.built_for
    except (ImportError, AttributeError) as e:
        built_for = f"something else: {e}"
    if built_for != here:
        warnings.warn(f"the binding's native calls were compiled for {built_for}, this is {here}: build the library again", RuntimeWarning)
        return None
    module.bind(*(C.cast(f, C.c_void_p).value for f in (_lib.rtn_linear, _lib.rtn_linear_asym, _lib.rtn_cache_plan, _lib.rtn_rope_cache,
                                                        _lib.rtn_paged_attention)))
    return module


_native = _load_native()
EXPORTS = ["rtn_status_str", "rtn_layout_version", "rtn_qweight_nbytes", "rtn_scales_nbytes",
           "rtn_workspace_nbytes", "rtn_quantize", "rtn_quantize_host_staging_nbytes", "rtn_quantize_from_host", "rtn_linear", "rtn_linear_ex", "rtn_linear_query",
           "rtn_problem_status", "rtn_linear_validate", "rtn_linear_noalloc", "rtn_unpack", "rtn_dequantize", "rtn_gemm_fp16", "rtn_dense_weight_nbytes", "rtn_linear_dense",
           "rtn_quantize_asym", "rtn_dequantize_asym", "rtn_linear_asym",
           "rtn_layer_forward", "rtn_grouped_forward", "rtn_bench_read_stream", "rtn_plan_bits", "rtn_plan_effective_bits",
           "rtn_cache_plan", "rtn_rope_cache", "rtn_paged_attention_workspace_nbytes", "rtn_paged_attention"]


def _check(status: int, what: str):
    if status != 0:
        raise RtnError(status, what)


# The current stream's handle without the Stream object that torch.cuda.current_stream() makes: 0.2 us instead of 2 of the
# 8 us that a small call took on the host.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    if _raw_stream is None or _device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dev_fp16(t: torch.Tensor, name: str):
    if not (t.is_cuda and t.dtype is torch.float16 and t.is_contiguous() and t.dim() == 2):
        raise ValueError(f"{name} must be a contiguous fp16 CUDA matrix")


def _dev_workspace(t: torch.Tensor, device: torch.device, name: str = "workspace"):
    """One piece of memory on the GPU that the call runs on: kernels write anywhere in its bytes."""
    if not (t.is_cuda and t.is_contiguous() and t.device == device):
        raise ValueError(f"{name} must be a contiguous CUDA tensor on the call's device")


def rtn_layout_version() -> int:
    return _lib.rtn_layout_version()


def rtn_qweight_nbytes(N, K, bits):
    return _lib.rtn_qweight_nbytes(N, K, bits)


def rtn_scales_nbytes(N, K, group_size):
    return _lib.rtn_scales_nbytes(N, K, group_size)


def rtn_workspace_nbytes(M, N, K, bits, group_size):
    return _lib.rtn_workspace_nbytes(M, N, K, bits, group_size)


def rtn_quantize(W: torch.Tensor, bits: int, group_size: int, flags: int = RTN_SCALE_QMAX, out=None):
    """W fp16 [N, K] on the GPU -> (qweight uint8 [N*K*bits/8], scales fp16 [N, K/g])."""
    _dev_fp16(W, "W")
    N, K = W.shape
    g = K if group_size <= 0 else group_size
    if out is None:
        nb = _lib.rtn_qweight_nbytes(N, K, bits)
        ns = _lib.rtn_scales_nbytes(N, K, g)
        if nb == 0 or ns == 0:
            _check(_lib.rtn_problem_status(N, K, bits, group_size) or 4, "rtn_quantize")
        qweight = torch.empty(nb, dtype=torch.uint8, device=W.device)
        scales = torch.empty((N, K // g), dtype=torch.float16, device=W.device)
    else:
        qweight, scales = out
    _check(_lib.rtn_quantize(W.data_ptr(), N, K, bits, group_size, flags, qweight.data_ptr(),
                             scales.data_ptr(), _stream()), "rtn_quantize")
    return qweight, scales


def make_cfg(cfg):
    if cfg is None:
        return None
    if isinstance(cfg, rtn_linear_cfg):
        return cfg
    return rtn_linear_cfg(**cfg)


def rtn_linear(A: torch.Tensor, qweight: torch.Tensor, scales: torch.Tensor, bits: int, group_size: int,
               out: torch.Tensor = None, workspace: torch.Tensor = None, cfg=None) -> torch.Tensor:
    """A fp16 [M, K], packed qweight, scales fp16 [N, K/g] -> C fp16 [M, N]."""
    if _native is not None and out is not None and workspace is not None and cfg is None:
        st = _native.linear(A, qweight, scales, bits, group_size, out, workspace)
        if st is not None:                                # (None: not for native code, see there)
            _check(st, "rtn_linear")
            return out
    _dev_fp16(A, "A")
    M, K = A.shape
    N = scales.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=A.device)
    if workspace is None:
        workspace = torch.empty(max(256, _lib.rtn_workspace_nbytes(M, N, K, bits, group_size)),
                                dtype=torch.uint8, device=A.device)
    _dev_workspace(workspace, A.device)
    c = make_cfg(cfg)
    st = _lib.rtn_linear_ex(A.data_ptr(), M, qweight.data_ptr(), scales.data_ptr(), N, K, bits, group_size,
                            out.data_ptr(), workspace.data_ptr(), workspace.nbytes,
                            _stream(), C.byref(c) if c is not None else None)
    _check(st, "rtn_linear")
    return out


def rtn_linear_query(M, N, K, bits, group_size) -> dict:
    c = rtn_linear_cfg()
    _check(_lib.rtn_linear_query(M, N, K, bits, group_size, C.byref(c)), "rtn_linear_query")
    return {k: getattr(c, k) for k, _ in rtn_linear_cfg._fields_}


def rtn_problem_status(N, K, bits, group_size) -> int:
    return _lib.rtn_problem_status(N, K, bits, group_size)


def rtn_linear_validate(M, N, K, bits, group_size, workspace_nbytes, cfg=None) -> int:
    """Host only: the status rtn_linear_ex would return for this problem and configuration (0 = it would launch)."""
    c = make_cfg(cfg)
    return _lib.rtn_linear_validate(M, N, K, bits, group_size, workspace_nbytes, None if c is None else C.byref(c))


def rtn_linear_noalloc(A: torch.Tensor, qweight: torch.Tensor, scales: torch.Tensor, bits: int, group_size: int,
                       out: torch.Tensor) -> torch.Tensor:
    """rtn_linear without a workspace argument: split-K partials go to the library's fixed device array."""
    _dev_fp16(A, "A")
    M, K = A.shape
    N = scales.shape[0]
    _check(_lib.rtn_linear_noalloc(A.data_ptr(), M, qweight.data_ptr(), scales.data_ptr(), N, K, bits, group_size,
                                   out.data_ptr(), _stream()), "rtn_linear_noalloc")
    return out


def rtn_bench_read_stream(buf: torch.Tensor, nbytes: int, kib_per_wavefront: int, sink: torch.Tensor):
    """Measurement hook: streams the first nbytes of buf once with a plain read kernel."""
    if buf.numel() * buf.element_size() < nbytes or sink.numel() * sink.element_size() < 4:
        raise ValueError(f"rtn_bench_read_stream: buffer of {buf.numel() * buf.element_size()} bytes, asked to read {nbytes}")
    _check(_lib.rtn_bench_read_stream(buf.data_ptr(), nbytes, kib_per_wavefront, sink.data_ptr(), _stream()),
           "rtn_bench_read_stream")


def rtn_unpack(qweight: torch.Tensor, N: int, K: int, bits: int) -> torch.Tensor:
    codes = torch.empty((N, K), dtype=torch.int8, device=qweight.device)
    _check(_lib.rtn_unpack(qweight.data_ptr(), N, K, bits, codes.data_ptr(), _stream()), "rtn_unpack")
    return codes


def rtn_dequantize(qweight: torch.Tensor, scales: torch.Tensor, K: int, bits: int, group_size: int,
                   out: torch.Tensor = None) -> torch.Tensor:
    N = scales.shape[0]
    W = out if out is not None else torch.empty((N, K), dtype=torch.float16, device=qweight.device)
    _check(_lib.rtn_dequantize(qweight.data_ptr(), scales.data_ptr(), N, K, bits, group_size, W.data_ptr(),
                               _stream()), "rtn_dequantize")
    return W


def rtn_quantize_from_host(W_host: torch.Tensor, bits: int, group_size: int, rows_per_shard: int, copy_stream,
                           flags: int = RTN_SCALE_QMAX, staging: torch.Tensor = None, out=None, device="cuda:0"):
    """W_host: fp16 [N, K] in (pinned) host memory -> (qweight, scales) on the GPU, quantised shard by shard with the
    host-to-device copies on `copy_stream` (a torch.cuda.Stream other than the current one) overlapping the kernels."""
    if W_host.is_cuda or W_host.dtype != torch.float16 or not W_host.is_contiguous() or W_host.dim() != 2:
        raise ValueError("W_host must be a contiguous fp16 host matrix")
    N, K = W_host.shape
    g = K if group_size <= 0 else group_size
    need = _lib.rtn_quantize_host_staging_nbytes(K, rows_per_shard)
    if staging is None:
        staging = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    if out is None:
        nb = _lib.rtn_qweight_nbytes(N, K, bits)
        ns = _lib.rtn_scales_nbytes(N, K, g)
        qweight = torch.empty(max(nb, 16), dtype=torch.uint8, device=device)[:nb]
        scales = torch.empty((N, max(K // max(g, 1), 1)), dtype=torch.float16, device=device) if ns else torch.empty((N, 1), dtype=torch.float16, device=device)
    else:
        qweight, scales = out
    _check(_lib.rtn_quantize_from_host(W_host.data_ptr(), N, K, bits, group_size, flags, qweight.data_ptr(),
                                       scales.data_ptr(), staging.data_ptr(), staging.numel(), rows_per_shard,
                                       _stream(), copy_stream.cuda_stream), "rtn_quantize_from_host")
    return qweight, scales


def rtn_gemm_fp16(A: torch.Tensor, W: torch.Tensor, out: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
    """Dense A fp16 [M, K] times W fp16 [N, K] transposed -> C fp16 [M, N]."""
    _dev_fp16(A, "A")
    _dev_fp16(W, "W")
    M, K = A.shape
    N = W.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=A.device)
    if workspace is not None:
        _dev_workspace(workspace, A.device)
    wp, wn = (workspace.data_ptr(), workspace.nbytes) if workspace is not None else (None, 0)
    _check(_lib.rtn_gemm_fp16(A.data_ptr(), M, W.data_ptr(), N, K, out.data_ptr(), wp, wn, _stream()), "rtn_gemm_fp16")
    return out


def rtn_linear_dense(A: torch.Tensor, qweight: torch.Tensor, scales: torch.Tensor, bits: int, group_size: int,
                     w_tmp: torch.Tensor, out: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
    """The dequantise-then-GEMM path: w_tmp is a caller-owned buffer of rtn_dense_weight_nbytes(N, K) bytes."""
    _dev_fp16(A, "A")
    M, K = A.shape
    N = scales.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=A.device)
    _dev_workspace(w_tmp, A.device, "w_tmp")
    if workspace is not None:
        _dev_workspace(workspace, A.device)
    wp, wn = (workspace.data_ptr(), workspace.nbytes) if workspace is not None else (None, 0)
    _check(_lib.rtn_linear_dense(A.data_ptr(), M, qweight.data_ptr(), scales.data_ptr(), N, K, bits, group_size,
                                 out.data_ptr(), w_tmp.data_ptr(), w_tmp.numel() * w_tmp.element_size(), wp, wn,
                                 _stream()), "rtn_linear_dense")
    return out


def rtn_dense_weight_nbytes(N: int, K: int) -> int:
    return _lib.rtn_dense_weight_nbytes(N, K)


class LayerPlan:
    """A prepared rtn_layer_forward call: the module descriptor array is built once."""

    def __init__(self, modules, workspace: torch.Tensor = None):
        """modules: list of dicts {A, qweight, scales, bits, group_size, C}."""
        self.n = len(modules)
        self.arr = (rtn_module * self.n)()
        self.keep = modules
        need = 256
        for i, m in enumerate(modules):
            M, K = m["A"].shape
            N = m["scales"].shape[0]
            self.arr[i] = rtn_module(m["A"].data_ptr(), M, m["qweight"].data_ptr(), m["scales"].data_ptr(),
                                     N, K, m["bits"], m["group_size"], m["C"].data_ptr())
            need = max(need, _lib.rtn_workspace_nbytes(M, N, K, m["bits"], m["group_size"]))
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=modules[0]["A"].device)
        if modules:
            _dev_workspace(workspace, modules[0]["A"].device)
        self.workspace = workspace

    def run(self):
        _check(_lib.rtn_layer_forward(self.arr, self.n, self.workspace.data_ptr(), self.workspace.numel(),
                                      _stream()), "rtn_layer_forward")

    def run_grouped(self):
        """The modules as independent problems (rtn_grouped_forward): no C may be another module's A."""
        _check(_lib.rtn_grouped_forward(self.arr, self.n, self.workspace.data_ptr(), self.workspace.numel(),
                                        _stream()), "rtn_grouped_forward")


def rtn_layer_forward(modules, workspace: torch.Tensor = None):
    LayerPlan(modules, workspace).run()


def rtn_quantize_asym(W: torch.Tensor, bits: int, group_size: int):
    """W fp16 [N, K] on the GPU -> (qweight uint8, scales fp16 [N, K/g], zeros fp16 [N, K/g]); weight = S (q + Z)."""
    _dev_fp16(W, "W")
    N, K = W.shape
    G = 1 if group_size <= 0 else K // max(group_size, 1)
    nq = _lib.rtn_qweight_nbytes(N, K, bits)
    if nq == 0:
        raise ValueError("unsupported shape or bits")
    q = torch.empty(nq, dtype=torch.uint8, device=W.device)
    s = torch.empty((N, max(G, 1)), dtype=torch.float16, device=W.device)
    z = torch.empty((N, max(G, 1)), dtype=torch.float16, device=W.device)
    _check(_lib.rtn_quantize_asym(W.data_ptr(), N, K, bits, group_size, q.data_ptr(), s.data_ptr(), z.data_ptr(),
                                  _stream()), "rtn_quantize_asym")
    return q, s, z


def rtn_dequantize_asym(qweight, scales, zeros, N, K, bits, group_size, out=None):
    if out is None:
        out = torch.empty((N, K), dtype=torch.float16, device=qweight.device)
    _check(_lib.rtn_dequantize_asym(qweight.data_ptr(), scales.data_ptr(), zeros.data_ptr(), N, K, bits, group_size,
                                    out.data_ptr(), _stream()), "rtn_dequantize_asym")
    return out


def rtn_linear_asym(A, qweight, scales, zeros, bits, group_size, out=None, workspace=None):
    if _native is not None and out is not None and workspace is not None:
        st = _native.linear_asym(A, qweight, scales, zeros, bits, group_size, out, workspace)
        if st is not None:
            _check(st, "rtn_linear_asym")
            return out
    _dev_fp16(A, "A")
    M, K = A.shape
    N = scales.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float16, device=A.device)
    if workspace is None:
        workspace = torch.empty(max(256, _lib.rtn_workspace_nbytes(M, N, K, bits, group_size)), dtype=torch.uint8,
                                device=A.device)
    _dev_workspace(workspace, A.device)
    _check(_lib.rtn_linear_asym(A.data_ptr(), M, qweight.data_ptr(), scales.data_ptr(), zeros.data_ptr(), N, K, bits,
                                group_size, out.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream()),
           "rtn_linear_asym")
    return out


def rtn_grouped_forward(modules, workspace: torch.Tensor = None):
    LayerPlan(modules, workspace).run_grouped()


def rtn_plan_bits(layer, n_layers, module_id, policy, X, modules=(1, 2, 3, 4)) -> int:
    mask = 0
    for m in modules:
        mask |= 1 << (m - 1)
    pol = POLICY[policy] if isinstance(policy, str) else policy
    return _lib.rtn_plan_bits(layer, n_layers, module_id, pol, X, mask)


def rtn_plan_effective_bits(n_layers, module_params, policy, X, modules=(1, 2, 3, 4)) -> float:
    mask = 0
    for m in modules:
        mask |= 1 << (m - 1)
    pol = POLICY[policy] if isinstance(policy, str) else policy
    arr = (C.c_int64 * 4)(*[int(v) for v in module_params])
    return _lib.rtn_plan_effective_bits(n_layers, arr, pol, X, mask)


# ---- The paged KV cache: what a step of token generation does between the QKV projection and the attention output projection -----------

RTN_TYPE_F16, RTN_TYPE_BF16 = 0, 1
_TYPES = {torch.float16: RTN_TYPE_F16, torch.bfloat16: RTN_TYPE_BF16}


class PagedCache:
    """The K and V pools of one layer, [pages, kv_heads, page_size, head_dim] in fp16 or bf16: contiguous, or any view of that shape whose last
    dimension is (pools stored [pages, page_size, kv_heads, head_dim] are passed as .transpose(1, 2))."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        if not (k.is_cuda and v.is_cuda and k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype and k.dtype in _TYPES and k.device == v.device):
            raise ValueError("k and v must be CUDA tensors [pages, kv_heads, page_size, head_dim] of one type, fp16 or bf16")
        if k.stride() != v.stride() or k.stride(3) != 1:
            raise ValueError("k and v must have the same strides, with head_dim contiguous")
        self.k, self.v = k, v
        self.pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.dtype, self.device = k.dtype, k.device
        self.desc = rtn_kv_cache(k.data_ptr(), v.data_ptr(), self.pages, self.page_size, self.kv_heads, self.head_dim, _TYPES[k.dtype],
                                 k.stride(0), k.stride(1), k.stride(2))
        self._ref, self._address = C.byref(self.desc), C.addressof(self.desc)


class CachePlan(collections.namedtuple("CachePlan", "seq_lens query_start positions slots free_count status")):
    """What rtn_cache_plan gives, int32 on the GPU: seq_lens [requests], query_start [requests + 1], positions and slots [max_tokens],
    free_count [1], status [1]."""
    __slots__ = ()

    @classmethod
    def empty(cls, requests: int, max_tokens: int, device="cuda:0"):
        return cls(*(torch.empty(n, dtype=torch.int32, device=device) for n in (requests, requests + 1, max_tokens, max_tokens, 1, 1)))


def _dev_int32(t: torch.Tensor, name: str, n: int = None):
    if not (t.is_cuda and t.dtype is torch.int32 and t.dim() == 1 and t.is_contiguous() and (n is None or t.shape[0] == n)):
        raise ValueError(f"{name} must be a contiguous int32 CUDA vector" + ("" if n is None else f" of {n}"))


def _dev_table(t: torch.Tensor):
    if not (t.is_cuda and t.dtype is torch.int32 and t.dim() == 2 and t.stride(1) == 1):
        raise ValueError("block_table must be an int32 CUDA matrix with contiguous rows")


def _c_int(n: int) -> int:
    """Of a bound that may be any width: what C's int has of it.  (ctypes takes the lower 32 bits.)"""
    return max(-1, min(n, 2 ** 31 - 1))


def _row_stride(t: torch.Tensor) -> int:
    """Elements from row to row; a single row may have any stride."""
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t[0].numel() if t.shape[0] else 0)


def rtn_cache_plan(step: torch.Tensor, cached_lens: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor, free_count: torch.Tensor,
                   page_size: int, max_tokens: int, out: CachePlan = None) -> CachePlan:
    """A step's block tables, slots and positions: request b appends step[b] tokens to its cached_lens[b] (or ends, step[b] < 0), with pages
    off the stack free_pages[:free_count].  block_table [requests, blocks] and free_pages are updated.  out.seq_lens may be cached_lens and
    out.free_count free_count, for a loop of replays.  out.status says what did not fit (0: nothing), and then nothing has changed."""
    if _native is not None and out is not None:
        st = _native.cache_plan(step, cached_lens, block_table, free_pages, free_count, page_size, max_tokens, out)
        if st is not None:
            _check(st, "rtn_cache_plan")
            return out
    _dev_int32(step, "step")
    B = step.shape[0]
    _dev_int32(cached_lens, "cached_lens", B)
    _dev_int32(free_pages, "free_pages")
    _dev_int32(free_count, "free_count", 1)
    _dev_table(block_table)
    if block_table.shape[0] != B:
        raise ValueError(f"block_table must have a row for each of the {B} requests")
    if _c_int(page_size) != page_size:
        raise ValueError("page_size must be 16, 32, 64, 128 or 256")
    if out is None:
        out = CachePlan.empty(B, max_tokens, step.device)
    for t, name, n in zip(out, CachePlan._fields, (B, B + 1, max_tokens, max_tokens, 1, 1)):
        _dev_int32(t, "out." + name, n)
    _check(_lib.rtn_cache_plan(step.data_ptr(), cached_lens.data_ptr(), B, page_size, block_table.data_ptr(), _row_stride(block_table), block_table.shape[1],
                               free_pages.data_ptr(), free_pages.shape[0], free_count.data_ptr(), out.seq_lens.data_ptr(), out.query_start.data_ptr(),
                               out.positions.data_ptr(), out.slots.data_ptr(), max_tokens, out.free_count.data_ptr(), out.status.data_ptr(), _stream()),
           "rtn_cache_plan")
    return out


def rtn_rope_cache(qkv: torch.Tensor, q_heads: int, rope: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor, cache: PagedCache,
                   q_norm: torch.Tensor = None, k_norm: torch.Tensor = None, eps: float = 1e-6, interleaved: bool = False,
                   out: torch.Tensor = None) -> torch.Tensor:
    """qkv [tokens, (q_heads + 2 kv_heads) * head_dim], the QKV projection's output -> queries [tokens, q_heads, head_dim], normed (where weights
    are given) and rotated; keys, the same way, and values go to the cache's slots.  rope fp32 [positions, rotary_dim]: cosines, then sines."""
    if _native is not None and out is not None:
        st = _native.rope_cache(qkv, q_heads, rope, positions, slots, cache._address, q_norm, k_norm, eps, interleaved, out)
        if st is not None:
            _check(st, "rtn_rope_cache")
            return out
    D, Hk, T = cache.head_dim, cache.kv_heads, qkv.shape[0]
    if not (qkv.is_cuda and qkv.dtype is cache.dtype and qkv.dim() == 2 and qkv.shape[1] == (q_heads + 2 * Hk) * D and qkv.stride(1) == 1):
        raise ValueError(f"qkv must be a CUDA matrix of the cache's type with {(q_heads + 2 * Hk) * D} contiguous columns")
    if not (rope.is_cuda and rope.dtype is torch.float32 and rope.dim() == 2 and rope.is_contiguous()):
        raise ValueError("rope must be a contiguous fp32 CUDA matrix [positions, rotary_dim]")
    _dev_int32(positions, "positions", T)
    _dev_int32(slots, "slots", T)
    for w, name in ((q_norm, "q_norm"), (k_norm, "k_norm")):
        if w is not None and not (w.is_cuda and w.dtype is cache.dtype and w.shape == (D,) and w.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous CUDA vector of {D} of the cache's type")
    if out is None:
        out = torch.empty((T, q_heads, D), dtype=cache.dtype, device=qkv.device)
    elif not (out.is_cuda and out.dtype is cache.dtype and out.shape == (T, q_heads, D) and out.is_contiguous()):
        raise ValueError("out must be a contiguous CUDA tensor [tokens, q_heads, head_dim] of the cache's type")
    _check(_lib.rtn_rope_cache(qkv.data_ptr(), T, _row_stride(qkv), q_heads, rope.data_ptr(), rope.shape[1], rope.shape[0], int(interleaved),
                               positions.data_ptr(), slots.data_ptr(), _ptr(q_norm), _ptr(k_norm), eps, cache._ref, out.data_ptr(), _stream()),
           "rtn_rope_cache")
    return out


def rtn_paged_attention_workspace_nbytes(tokens: int, requests: int, q_heads: int, cache: PagedCache, max_new: int) -> int:
    return _lib.rtn_paged_attention_workspace_nbytes(tokens, requests, q_heads, cache._ref, _c_int(max_new))


def rtn_paged_attention(q: torch.Tensor, cache: PagedCache, block_table: torch.Tensor, seq_lens: torch.Tensor, query_start: torch.Tensor, max_new: int,
                        scale: float = None, softcap: float = 0.0, window: int = 0, out: torch.Tensor = None,
                        workspace: torch.Tensor = None) -> torch.Tensor:
    """q [tokens, q_heads, head_dim], request b's new tokens being rows query_start[b] .. query_start[b + 1] - 1 and the last of its seq_lens[b]
    tokens in the cache -> attention output of the same shape.  max_new: a bound on the new tokens of one request."""
    if _native is not None and out is not None and workspace is not None:
        st = _native.paged_attention(q, cache._address, block_table, seq_lens, query_start, max_new, scale, softcap, window, out, workspace)
        if st is not None:
            _check(st, "rtn_paged_attention")
            return out
    max_new, window = _c_int(max_new), _c_int(window)
    T, Hq, D = q.shape
    if not (q.is_cuda and q.dtype is cache.dtype and D == cache.head_dim and q.stride(2) == 1 and (q.stride(1) == D or Hq == 1)):
        raise ValueError("q must be a CUDA tensor [tokens, q_heads, head_dim] of the cache's type, contiguous within a token")
    _dev_int32(seq_lens, "seq_lens")
    B = seq_lens.shape[0]
    _dev_int32(query_start, "query_start", B + 1)
    _dev_table(block_table)
    if block_table.shape[0] != B:
        raise ValueError(f"block_table must have a row for each of the {B} requests")
    if out is None:
        out = torch.empty((T, Hq, D), dtype=q.dtype, device=q.device)
    elif not (out.is_cuda and out.dtype is q.dtype and out.shape == (T, Hq, D) and out.is_contiguous()):
        raise ValueError("out must be a contiguous CUDA tensor of q's shape and type")
    if workspace is None:
        need = _lib.rtn_paged_attention_workspace_nbytes(T, B, Hq, cache._ref, max_new)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    _dev_workspace(workspace, q.device)
    _check(_lib.rtn_paged_attention(q.data_ptr(), T, _row_stride(q), Hq, cache._ref, block_table.data_ptr(), _row_stride(block_table), block_table.shape[1],
                                    seq_lens.data_ptr(), query_start.data_ptr(), B, max_new, D ** -0.5 if scale is None else scale, softcap, window,
                                    out.data_ptr(), workspace.data_ptr(), workspace.nbytes, _stream()), "rtn_paged_attention")
    return out

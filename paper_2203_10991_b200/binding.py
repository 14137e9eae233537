"""Python binding of the C ABI in include/mvue.h, mvue_train.h and mvue_layer.h: argument marshalling only.

Tensors are torch CUDA tensors used purely as device memory; every function passes
raw pointers, sizes and the current CUDA stream to the library.  There is no
fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
from pathlib import Path

import torch

_LIB_PATH = Path(__file__).resolve().parent / "libmvue_b200.so"
_lib = None

MVUE_F32, MVUE_BF16 = 0, 1
MVUE_LAYOUT_CANONICAL = 0
MVUE_LAYOUT_TC = 1
MVUE_JOINT_TABLE, MVUE_JOINT_SYSTEMATIC, MVUE_JOINT_APPROX = 0, 1, 2
MVUE_OPT_NONE, MVUE_OPT_STOCHASTIC_ROUNDING, MVUE_OPT_EPS16 = 0, 1, 2
MVUE_OPT_NESTEROV = 16            # of mvue_muon_step
MVUE_MUON_SCALES = {"rms": 0, "shape": 1}
MVUE_ERR_WORKSPACE = -7
MVUE_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}

EXPORTS = ("mvue_version", "mvue_status_string", "mvue_last_cuda_error", "mvue_packed_sizes",
           "mvue_prune", "mvue_prune_joint", "mvue_prune_opts", "mvue_prune_4of8", "mvue_unpack", "mvue_sparse_update_gemm", "mvue_sparse_backward_gemm",
           "mvue_sparse_backward_gemm_pruned",
           "mvue_gemm_workspace_bytes", "mvue_sparse_update_gemm_noalloc", "mvue_fused_update_gemm", "mvue_fused_update_gemm_joint",
           "mvue_probe_sparse_mma", "mvue_selftest_wait_timeout",
           "mvue_adamw_step", "mvue_embedding", "mvue_embedding_grad", "mvue_embedding_grad_workspace_bytes",
           "mvue_group_norm_act", "mvue_group_norm_act_backward", "mvue_group_norm_workspace_bytes",
           "mvue_selftest_group_norm_timeout",
           "mvue_layer_norm", "mvue_layer_norm_backward", "mvue_layer_norm_workspace_bytes",
           "mvue_quantize_e4m3", "mvue_scaled_forward_gemm", "mvue_scaled_backward_gemm",
           "mvue_orthogonalize", "mvue_orthogonalize_workspace_bytes", "mvue_muon_step", "mvue_muon_workspace_bytes")


class AdamWTensor(ctypes.Structure):
    """mvue_adamw_tensor"""
    _fields_ = [(name, ctypes.c_void_p) for name in ("param", "master", "grad", "exp_avg", "exp_avg_sq", "exp_avg_scale",
                                                     "exp_avg_sq_scale")] + \
               [("numel", ctypes.c_int64), ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32)]


class AdamWConfig(ctypes.Structure):
    """mvue_adamw_config"""
    _fields_ = [(name, ctypes.c_double) for name in ("lr", "beta1", "beta2", "eps", "weight_decay")] + \
               [("step", ctypes.c_int64), ("grad_scale", ctypes.c_double), ("dev_grad_scale", ctypes.c_void_p),
                ("seed", ctypes.c_uint64), ("state_bits", ctypes.c_int32), ("options", ctypes.c_uint32)]


class MuonTensor(ctypes.Structure):
    """mvue_muon_tensor"""
    _fields_ = [(name, ctypes.c_void_p) for name in ("param", "master", "grad", "momentum")] + \
               [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32)]


class MuonConfig(ctypes.Structure):
    """mvue_muon_config"""
    _fields_ = [(name, ctypes.c_double) for name in ("lr", "momentum", "weight_decay", "grad_scale")] + \
               [("dev_grad_scale", ctypes.c_void_p), ("seed", ctypes.c_uint64), ("ns_steps", ctypes.c_int32),
                ("scale_rule", ctypes.c_int32), ("options", ctypes.c_uint32)]


class MvueError(RuntimeError):
    def __init__(self, status: int, what: str):
        L = lib()
        msg = L.mvue_status_string(status).decode()
        cuda = L.mvue_last_cuda_error().decode()
        super().__init__(f"{what}: {msg} [{status}]" + (f" -- {cuda}" if status == -9 and cuda else ""))
        self.status = status


def lib() -> ctypes.CDLL:
    """Load libmvue_b200.so (built by `python -m paper_2203_10991_b200.build`)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "`python -m paper_2203_10991_b200.build` (there is no CPU fallback)")
        L = ctypes.CDLL(str(_LIB_PATH))
        i64, u64, vp, ci = ctypes.c_int64, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_int
        szp = ctypes.POINTER(ctypes.c_size_t)
        L.mvue_version.restype = ci
        L.mvue_status_string.argtypes = [ci]
        L.mvue_status_string.restype = ctypes.c_char_p
        L.mvue_last_cuda_error.restype = ctypes.c_char_p
        L.mvue_packed_sizes.argtypes = [i64, i64, ci, ci, ci, ci, szp, szp]
        L.mvue_prune.argtypes = [vp, ci, i64, i64, i64, ci, ci, ci, u64, i64, i64, vp, vp, ci, vp]
        L.mvue_prune_joint.argtypes = [vp, ci, i64, i64, i64, ci, ci, ci, u64, i64, i64, vp, vp, ci, ci, vp]
        L.mvue_prune_opts.argtypes = [vp, ci, i64, i64, i64, ci, ci, ci, u64, i64, i64, vp, vp, ci, ci, ctypes.c_uint, vp]
        L.mvue_prune_4of8.argtypes = [vp, ci, i64, i64, i64, ci, u64, i64, i64, vp, vp, vp]
        L.mvue_unpack.argtypes = [vp, vp, ci, i64, i64, vp, vp]
        L.mvue_sparse_update_gemm.argtypes = [vp, vp, ci, i64, i64, vp, i64, i64, vp, ci, i64, ci, vp,
                                              ctypes.c_size_t, vp, vp]
        L.mvue_sparse_backward_gemm.argtypes = [vp, vp, ci, i64, i64, vp, i64, i64, vp, vp, ci, i64, vp,
                                                ctypes.c_size_t, vp, vp]
        L.mvue_sparse_backward_gemm_pruned.argtypes = [vp, vp, ci, i64, i64, vp, i64, i64, vp, vp, i64, u64, ci,
                                                       ctypes.c_uint, vp, vp, vp, ctypes.c_size_t, vp, vp]
        L.mvue_gemm_workspace_bytes.argtypes = [ci, i64, i64, i64, szp]
        L.mvue_fused_update_gemm.argtypes = [vp, ci, i64, i64, i64, ci, ci, u64, vp, i64, i64, vp, ci, i64, ci, vp,
                                             ctypes.c_size_t, vp, vp]
        L.mvue_fused_update_gemm_joint.argtypes = [vp, ci, i64, i64, i64, ci, ci, ci, u64, vp, i64, i64, vp, ci, i64, ci, vp,
                                                   ctypes.c_size_t, vp, vp]
        L.mvue_sparse_update_gemm_noalloc.argtypes = [vp, vp, ci, i64, i64, vp, i64, i64, vp, ci, i64, ci, vp, vp]
        L.mvue_probe_sparse_mma.argtypes = [ci, ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_double), vp, vp]
        L.mvue_selftest_wait_timeout.argtypes = [ci, vp, vp]
        cf, csz = ctypes.c_float, ctypes.c_size_t
        L.mvue_embedding.argtypes = [vp, ci, i64, vp, ci, i64, i64, i64, cf, vp, ci, i64, vp, vp]
        L.mvue_embedding_grad.argtypes = [vp, ci, i64, vp, ci, i64, i64, cf, i64, vp, ci, i64, i64, ci, vp, csz, vp, vp]
        L.mvue_embedding_grad_workspace_bytes.argtypes = [i64, i64, szp]
        L.mvue_group_norm_act.argtypes = [vp, ci, i64, i64, i64, i64, ci, vp, vp, ci, cf, ci, vp, i64, vp, vp, vp, csz, vp, vp]
        L.mvue_group_norm_act_backward.argtypes = [vp, i64, vp, i64, ci, i64, i64, i64, ci, vp, vp, vp, vp, ci, ci, vp, i64, vp, vp,
                                                   vp, csz, vp, vp]
        L.mvue_group_norm_workspace_bytes.argtypes = [i64, i64, i64, ci, szp]
        L.mvue_selftest_group_norm_timeout.argtypes = [ci, vp, vp, ci, i64, i64, i64, ci, vp, vp, vp, vp, csz, vp, vp]
        L.mvue_layer_norm.argtypes = [vp, ci, i64, i64, i64, vp, vp, ci, cf, vp, i64, vp, vp, vp]
        L.mvue_layer_norm_backward.argtypes = [vp, i64, vp, i64, ci, i64, i64, vp, vp, vp, ci, vp, i64, vp, vp, vp, csz, vp]
        L.mvue_layer_norm_workspace_bytes.argtypes = [i64, i64, szp]
        L.mvue_quantize_e4m3.argtypes = [vp, ci, i64, i64, i64, ci, ctypes.c_uint, u64, vp, i64, vp, vp]
        L.mvue_orthogonalize.argtypes = [vp, ci, i64, i64, i64, i64, i64, ci, vp, ci, i64, i64, vp, csz, vp, vp]
        L.mvue_orthogonalize_workspace_bytes.argtypes = [i64, i64, i64, szp]
        L.mvue_muon_step.argtypes = [ctypes.POINTER(MuonTensor), i64, ctypes.POINTER(MuonConfig), vp, csz, vp, vp]
        L.mvue_muon_workspace_bytes.argtypes = [ctypes.POINTER(MuonTensor), i64, szp]
        for product in (L.mvue_scaled_forward_gemm, L.mvue_scaled_backward_gemm):
            product.argtypes = [vp, vp, i64, i64, i64, vp, vp, i64, i64, vp, ci, i64, vp, vp]
        L.mvue_adamw_step.argtypes = [ctypes.POINTER(AdamWTensor), i64, ctypes.POINTER(AdamWConfig), vp]
        _lib = L
    return _lib


def _check(status: int, what: str):
    if status != 0:
        raise MvueError(status, what)


def _stream_ptr() -> int:
    # the current stream's handle without a Stream object around it (0.5 us instead of 5 us)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


_DTYPE_CODES = {torch.float32: MVUE_F32, torch.bfloat16: MVUE_BF16}


def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}")
    return code


def mvue_packed_sizes(rows: int, cols: int, n: int, m: int, axis: int, layout: int = MVUE_LAYOUT_CANONICAL):
    vb, mb = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().mvue_packed_sizes(rows, cols, n, m, axis, layout, ctypes.byref(vb), ctypes.byref(mb)),
           "mvue_packed_sizes")
    return vb.value, mb.value


def mvue_prune(g: torch.Tensor, n: int, m: int, axis: int, seed: int, *, k_total: int | None = None,
               k_offset: int = 0, values: torch.Tensor | None = None, meta: torch.Tensor | None = None,
               layout: int = MVUE_LAYOUT_CANONICAL, joint: int | None = None, options: int = MVUE_OPT_NONE):
    """MVUE n:m prune + pack of a 2-D CUDA tensor g (fp32 or bf16, unit column stride).

    joint: None calls mvue_prune (App. A.2 pair table); an mvue_joint value calls mvue_prune_joint.
    options: non-zero calls mvue_prune_opts (MVUE_OPT_STOCHASTIC_ROUNDING: unbiased bf16 storage of the survivors).
    Returns (values bf16 [Mrows, K/2], meta uint8 [Mrows, K/8]).
    """
    assert g.is_cuda and g.dim() == 2 and g.stride(1) == 1
    rows, cols = g.shape
    mrows, k = (rows, cols) if axis == 1 else (cols, rows)
    if values is None or meta is None:
        _, meta_bytes = mvue_packed_sizes(rows, cols, n, m, axis, layout)   # validates before allocating
        values = torch.empty((mrows, k // 2), dtype=torch.bfloat16, device=g.device)
        meta = torch.empty((meta_bytes // (k // 8), k // 8), dtype=torch.uint8, device=g.device)
    if options:
        _check(lib().mvue_prune_opts(g.data_ptr(), _dtype_code(g), rows, cols, g.stride(0), n, m, axis,
                                     seed & (2**64 - 1), k if k_total is None else k_total, k_offset,
                                     values.data_ptr(), meta.data_ptr(), layout,
                                     MVUE_JOINT_TABLE if joint is None else int(joint), int(options), _stream_ptr()),
               "mvue_prune_opts")
    elif joint is None:
        _check(lib().mvue_prune(g.data_ptr(), _dtype_code(g), rows, cols, g.stride(0), n, m, axis,
                                seed & (2**64 - 1), k if k_total is None else k_total, k_offset,
                                values.data_ptr(), meta.data_ptr(), layout, _stream_ptr()), "mvue_prune")
    else:
        _check(lib().mvue_prune_joint(g.data_ptr(), _dtype_code(g), rows, cols, g.stride(0), n, m, axis,
                                      seed & (2**64 - 1), k if k_total is None else k_total, k_offset,
                                      values.data_ptr(), meta.data_ptr(), layout, int(joint), _stream_ptr()),
               "mvue_prune_joint")
    return values, meta


def mvue_prune_4of8(g: torch.Tensor, axis: int, seed: int, *, k_total: int | None = None, k_offset: int = 0):
    """Approx-4:8 prune (prune only) of a 2-D CUDA tensor: (values bf16 [Mrows, K/2], mask uint8 [Mrows, K/8])."""
    assert g.is_cuda and g.dim() == 2 and g.stride(1) == 1
    rows, cols = g.shape
    mrows, k = (rows, cols) if axis == 1 else (cols, rows)
    values = torch.empty((mrows, k // 2), dtype=torch.bfloat16, device=g.device)
    mask = torch.empty((mrows, k // 8), dtype=torch.uint8, device=g.device)
    _check(lib().mvue_prune_4of8(g.data_ptr(), _dtype_code(g), rows, cols, g.stride(0), axis, seed & (2**64 - 1),
                                 k if k_total is None else k_total, k_offset, values.data_ptr(), mask.data_ptr(),
                                 _stream_ptr()), "mvue_prune_4of8")
    return values, mask


def mvue_unpack(values: torch.Tensor, meta: torch.Tensor, layout: int = MVUE_LAYOUT_CANONICAL) -> torch.Tensor:
    mrows, kh = values.shape
    dense = torch.empty((mrows, 2 * kh), dtype=torch.bfloat16, device=values.device)
    _check(lib().mvue_unpack(values.data_ptr(), meta.data_ptr(), layout, mrows, 2 * kh, dense.data_ptr(),
                             _stream_ptr()), "mvue_unpack")
    return dense


def mvue_gemm_workspace_bytes(which: int, M: int, N: int, K: int) -> int:
    b = ctypes.c_size_t()
    _check(lib().mvue_gemm_workspace_bytes(which, M, N, K, ctypes.byref(b)), "mvue_gemm_workspace_bytes")
    return b.value


def _workspace(which, M, N, K, device, workspace):
    need = mvue_gemm_workspace_bytes(which, M, N, K)
    if need == 0:
        return None, 0
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, workspace.numel() * workspace.element_size()


def mvue_sparse_update_gemm(values: torch.Tensor, meta: torch.Tensor, h: torch.Tensor, *,
                            out: torch.Tensor | None = None, out_dtype=torch.float32, accumulate: bool = False,
                            workspace: torch.Tensor | None = None, dev_status: torch.Tensor | None = None,
                            layout: int = MVUE_LAYOUT_TC) -> torch.Tensor:
    """dW[out, in] (+)= theta(g)^T . h with the packed operand of mvue_prune(g, axis=0, layout=MVUE_LAYOUT_TC)."""
    n_out, half_t = values.shape
    T, n_in = h.shape
    assert h.dtype == torch.bfloat16 and h.stride(1) == 1 and 2 * half_t == T
    if out is None:
        out = torch.empty((n_out, n_in), dtype=out_dtype, device=h.device)
    ws, ws_bytes = _workspace(0, n_out, n_in, T, h.device, workspace)
    _check(lib().mvue_sparse_update_gemm(values.data_ptr(), meta.data_ptr(), layout, n_out, T, h.data_ptr(), n_in,
                                         h.stride(0), out.data_ptr(), _dtype_code(out), out.stride(0),
                                         int(accumulate), None if ws is None else ws.data_ptr(), ws_bytes,
                                         None if dev_status is None else dev_status.data_ptr(), _stream_ptr()),
           "mvue_sparse_update_gemm")
    return out


def mvue_sparse_backward_gemm(values: torch.Tensor, meta: torch.Tensor, W: torch.Tensor, *,
                              act_grad: torch.Tensor | None = None, out: torch.Tensor | None = None,
                              out_dtype=torch.bfloat16, workspace: torch.Tensor | None = None,
                              dev_status: torch.Tensor | None = None,
                              layout: int = MVUE_LAYOUT_TC) -> torch.Tensor:
    """dh[T, in] = (theta(g) . W) (* act_grad) with the packed operand of mvue_prune(g, axis=1, layout=MVUE_LAYOUT_TC)."""
    T, half_o = values.shape
    n_out, n_in = W.shape
    assert W.dtype == torch.bfloat16 and W.stride(1) == 1 and 2 * half_o == n_out
    if out is None:
        out = torch.empty((T, n_in), dtype=out_dtype, device=W.device)
    if act_grad is not None:
        assert act_grad.dtype == torch.bfloat16 and act_grad.shape == out.shape and act_grad.stride(0) == out.stride(0)
    ws, ws_bytes = _workspace(1, T, n_in, n_out, W.device, workspace)
    _check(lib().mvue_sparse_backward_gemm(values.data_ptr(), meta.data_ptr(), layout, T, n_out, W.data_ptr(), n_in,
                                           W.stride(0), None if act_grad is None else act_grad.data_ptr(),
                                           out.data_ptr(), _dtype_code(out), out.stride(0),
                                           None if ws is None else ws.data_ptr(), ws_bytes,
                                           None if dev_status is None else dev_status.data_ptr(), _stream_ptr()),
           "mvue_sparse_backward_gemm")
    return out


def mvue_sparse_backward_gemm_pruned(values: torch.Tensor, meta: torch.Tensor, W: torch.Tensor, act_grad: torch.Tensor,
                                     next_seed: int, *, next_joint: int = MVUE_JOINT_TABLE, next_options: int = MVUE_OPT_NONE,
                                     workspace: torch.Tensor | None = None, dev_status: torch.Tensor | None = None,
                                     layout: int = MVUE_LAYOUT_TC):
    """dh = (theta(g) . W) * act_grad (bf16) and, from the same launch, dh pruned 2:4 along its columns in tensor-core
    order (what mvue_prune(dh, 2, 4, axis=1, next_seed, layout=MVUE_LAYOUT_TC, joint=next_joint,
    options=next_options) gives).
    Returns (dh, next_values, next_meta)."""
    T, half_o = values.shape
    n_out, n_in = W.shape
    assert W.dtype == torch.bfloat16 and W.stride(1) == 1 and 2 * half_o == n_out
    out = torch.empty((T, n_in), dtype=torch.bfloat16, device=W.device)
    assert act_grad.dtype == torch.bfloat16 and act_grad.shape == out.shape and act_grad.stride(0) == out.stride(0)
    _, meta_bytes = mvue_packed_sizes(T, n_in, 2, 4, 1, MVUE_LAYOUT_TC)
    next_values = torch.empty((T, n_in // 2), dtype=torch.bfloat16, device=W.device)
    next_meta = torch.empty((meta_bytes // (n_in // 8), n_in // 8), dtype=torch.uint8, device=W.device)
    ws, ws_bytes = _workspace(1, T, n_in, n_out, W.device, workspace)
    _check(lib().mvue_sparse_backward_gemm_pruned(values.data_ptr(), meta.data_ptr(), layout, T, n_out, W.data_ptr(), n_in,
                                                  W.stride(0), act_grad.data_ptr(), out.data_ptr(), out.stride(0),
                                                  next_seed & (2**64 - 1), int(next_joint), int(next_options), next_values.data_ptr(),
                                                  next_meta.data_ptr(), None if ws is None else ws.data_ptr(), ws_bytes,
                                                  None if dev_status is None else dev_status.data_ptr(), _stream_ptr()),
           "mvue_sparse_backward_gemm_pruned")
    return out, next_values, next_meta


def mvue_sparse_update_gemm_noalloc(values: torch.Tensor, meta: torch.Tensor, h: torch.Tensor, out: torch.Tensor, *,
                                    accumulate: bool = False, dev_status: torch.Tensor | None = None,
                                    layout: int = MVUE_LAYOUT_TC) -> torch.Tensor:
    """The update product for callers that may not allocate: the caller passes every buffer, including
    `out`, and the split-K scratch is the fixed array inside the library (8 MiB per GPU).  Nothing is
    allocated here either.  Raises MvueError(-7) when the problem needs more scratch than that."""
    n_out, half_t = values.shape
    T, n_in = h.shape
    _check(lib().mvue_sparse_update_gemm_noalloc(values.data_ptr(), meta.data_ptr(), layout, n_out, T, h.data_ptr(),
                                                 n_in, h.stride(0), out.data_ptr(), _dtype_code(out), out.stride(0),
                                                 int(accumulate),
                                                 None if dev_status is None else dev_status.data_ptr(),
                                                 _stream_ptr()), "mvue_sparse_update_gemm_noalloc")
    return out


def mvue_fused_update_gemm(g: torch.Tensor, h: torch.Tensor, n: int, m: int, seed: int, *,
                           out: torch.Tensor | None = None, out_dtype=torch.float32, accumulate: bool = False,
                           workspace: torch.Tensor | None = None,
                           dev_status: torch.Tensor | None = None, joint: int = MVUE_JOINT_TABLE) -> torch.Tensor:
    """dW[out, in] (+)= theta(g)^T . h in one kernel: g bf16 [T, out] is pruned along the tokens on the fly
    (joint: the 2:4 law, MVUE_JOINT_TABLE or MVUE_JOINT_SYSTEMATIC)."""
    T, n_out = g.shape
    T2, n_in = h.shape
    assert T == T2 and g.stride(1) == 1 and h.stride(1) == 1
    if out is None:
        out = torch.empty((n_out, n_in), dtype=out_dtype, device=h.device)
    ws, ws_bytes = _workspace(2, n_out, n_in, T, h.device, workspace)
    _check(lib().mvue_fused_update_gemm_joint(g.data_ptr(), _dtype_code(g), T, n_out, g.stride(0), n, m, int(joint),
                                              seed & (2**64 - 1),
                                        h.data_ptr(), n_in, h.stride(0), out.data_ptr(), _dtype_code(out),
                                        out.stride(0), int(accumulate), None if ws is None else ws.data_ptr(), ws_bytes,
                                        None if dev_status is None else dev_status.data_ptr(), _stream_ptr()),
           "mvue_fused_update_gemm")
    return out


def mvue_probe_sparse_mma(iters: int, dev_status: torch.Tensor | None = None):
    """One launch of the sparse tensor-core issue-rate probe on the current stream.
    Returns (pairs, dense-equivalent flops of the launch); time it with CUDA events."""
    pairs, flops = ctypes.c_int(), ctypes.c_double()
    _check(lib().mvue_probe_sparse_mma(iters, ctypes.byref(pairs), ctypes.byref(flops),
                                       None if dev_status is None else dev_status.data_ptr(), _stream_ptr()),
           "mvue_probe_sparse_mma")
    return pairs.value, flops.value


def mvue_selftest_wait_timeout(polls: int, dev_status: torch.Tensor) -> None:
    """One launch whose only wait nobody answers: it expires after `polls` polls and the blocks leave through the
    ordinary exit, writing MVUE_ERR_DEVICE_TIMEOUT (-10) to dev_status (int32 CUDA tensor)."""
    _check(lib().mvue_selftest_wait_timeout(polls, dev_status.data_ptr(), _stream_ptr()), "mvue_selftest_wait_timeout")


def mvue_adamw_step(tensors: ctypes.Array, count: int, config: AdamWConfig) -> None:
    """One AdamW step over `count` entries of a ctypes array of AdamWTensor (optim.AdamWPlan fills and keeps one)."""
    _check(lib().mvue_adamw_step(tensors, count, config, _stream_ptr()), "mvue_adamw_step")


def _operands(first: torch.Tensor, *others: torch.Tensor | None, workspace: torch.Tensor | None = None,
              dev_status: torch.Tensor | None = None) -> None:
    """Raises unless all tensors are on one CUDA device and that is the current one, whose stream the call goes to: the
    library reads every address on the device."""
    device = first.get_device()                              # -1 on the CPU
    if device < 0:
        raise ValueError("wants CUDA tensors")
    for t in (*others, workspace, dev_status):
        if t is not None and t.get_device() != device:
            raise ValueError("the operands are on different devices")
    if device != torch.cuda.current_device():
        raise ValueError(f"the operands are on device {device}, the current device is {torch.cuda.current_device()}")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("the workspace is contiguous")
    if dev_status is not None and (dev_status.dtype is not torch.int32 or dev_status.numel() == 0):
        raise ValueError("dev_status is an int32 tensor")


def _id_list(ids: torch.Tensor) -> tuple[torch.Tensor, int]:
    if ids.dtype is torch.int64:
        return ids.contiguous(), 64
    if ids.dtype is torch.int32:
        return ids.contiguous(), 32
    raise TypeError(f"unsupported id dtype {ids.dtype}")


def mvue_embedding(ids: torch.Tensor, W: torch.Tensor, *, scale: float = 1.0, out: torch.Tensor | None = None, out_dtype=None,
                   dev_status: torch.Tensor | None = None) -> torch.Tensor:
    """scale * W[ids]: ids int32 or int64 of any shape, W [vocab, cols] fp32 or bf16 (unit column stride).  Ids outside the
    vocabulary give rows of zeros and write MVUE_ERR_INDEX (-13) to dev_status (int32 CUDA tensor).  Returns
    [*ids.shape, cols] of out_dtype (W's own unless given); out: [tokens, cols] with unit column stride instead."""
    _operands(ids, W, out, dev_status=dev_status)
    flat, id_bits = _id_list(ids)
    assert W.dim() == 2 and W.stride(1) == 1
    vocab, cols = W.shape
    tokens = flat.numel()
    if out is None:
        out = W.new_empty((*ids.shape, cols), dtype=out_dtype)
        ldout = cols
    else:
        assert out.shape == (tokens, cols) and out.stride(1) == 1
        ldout = out.stride(0) if tokens > 1 else cols
    _check(lib().mvue_embedding(flat.data_ptr(), id_bits, tokens, W.data_ptr(), _dtype_code(W), vocab, cols,
                                W.stride(0) if vocab > 1 else cols, scale, out.data_ptr(), _dtype_code(out), ldout,
                                None if dev_status is None else dev_status.data_ptr(), _stream_ptr()), "mvue_embedding")
    return out


def mvue_embedding_grad_workspace_bytes(tokens: int, cols: int) -> int:
    b = ctypes.c_size_t()
    _check(lib().mvue_embedding_grad_workspace_bytes(tokens, cols, ctypes.byref(b)), "mvue_embedding_grad_workspace_bytes")
    return b.value


def mvue_embedding_grad(ids: torch.Tensor, dy: torch.Tensor, vocab: int, *, scale: float = 1.0, padding_idx: int = -1,
                        out: torch.Tensor | None = None, out_dtype=torch.float32, accumulate: bool = False,
                        workspace: torch.Tensor | None = None, dev_status: torch.Tensor | None = None) -> torch.Tensor:
    """dW[v] (+)= scale * sum of dy[t] over ids[t] = v: dy [*ids.shape, cols] fp32 or bf16, or [tokens, cols] with a row
    stride.  Rows that no token names are zero (accumulate: out, fp32, is added to).  Returns dW [vocab, cols]."""
    _operands(ids, dy, out, workspace=workspace, dev_status=dev_status)
    flat, id_bits = _id_list(ids)
    cols = dy.shape[-1]
    tokens = flat.numel()
    if dy.dim() != 2:
        dy = dy.reshape(tokens, cols)
    assert dy.shape[0] == tokens and dy.stride(1) == 1
    if out is None:
        if accumulate:
            raise ValueError("accumulate adds to a given out")
        out = dy.new_empty((vocab, cols), dtype=out_dtype)
    assert out.shape == (vocab, cols) and out.stride(1) == 1
    need = mvue_embedding_grad_workspace_bytes(tokens, cols)
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = dy.new_empty(need, dtype=torch.uint8)
    _check(lib().mvue_embedding_grad(flat.data_ptr(), id_bits, tokens, dy.data_ptr(), _dtype_code(dy), cols,
                                     dy.stride(0) if tokens > 1 else cols, scale, padding_idx, out.data_ptr(), _dtype_code(out), vocab,
                                     out.stride(0) if vocab > 1 else cols, int(accumulate), workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(),
                                     None if dev_status is None else dev_status.data_ptr(), _stream_ptr()), "mvue_embedding_grad")
    return out


def _ptr(t: torch.Tensor | None):
    return None if t is None else t.data_ptr()


def _positions(t: torch.Tensor):
    """(n, s, c, ld) of a channels-last tensor [n, ..., c] whose positions lie one row stride apart."""
    if t.dim() >= 2 and t.numel() and t.is_contiguous():
        n, c = t.shape[0], t.shape[-1]
        return n, t.numel() // (n * c), c, c
    if t.dim() < 2 or t.stride(-1) != 1 and t.shape[-1] != 1:
        raise ValueError("wants [n, ..., channels] with unit channel stride")
    c = t.shape[-1]
    rows = t.numel() // c if c else 0
    s = rows // t.shape[0] if t.shape[0] else 1
    for d in t.shape[1:-1]:
        if t.shape[0] == 0:
            s *= d
    ld, step = None, None
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):       # innermost position first
        if size != 1:
            if ld is None:
                ld = stride
            elif stride != step:
                raise ValueError("positions are not one row stride apart")
            step = stride * size
    return t.shape[0], s, c, c if ld is None or t.numel() == 0 else ld


def _affine(weight, bias, c: int) -> int:
    for t in (weight, bias):
        if t is not None and (t.dim() != 1 or t.numel() != c or not t.is_contiguous()):
            raise ValueError("weight and bias are contiguous CUDA tensors of one element per channel")
    if weight is not None and bias is not None and weight.dtype is not bias.dtype:
        raise TypeError("weight and bias have one dtype")
    return MVUE_F32 if weight is None and bias is None else _dtype_code(bias if weight is None else weight)


def mvue_group_norm_workspace_bytes(n: int, s: int, c: int, groups: int) -> int:
    b = ctypes.c_size_t()
    _check(lib().mvue_group_norm_workspace_bytes(n, s, c, groups, ctypes.byref(b)), "mvue_group_norm_workspace_bytes")
    return b.value


def mvue_group_norm_act(x: torch.Tensor, groups: int, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, *,
                        eps: float = 1e-5, act: str = "none", out: torch.Tensor | None = None,
                        workspace: torch.Tensor | None = None, dev_status: torch.Tensor | None = None):
    """act(group_norm(x) * weight + bias) on a channels-last CUDA tensor x [n, ..., c], fp32 or bf16 (act: none, relu, silu,
    gelu).  Returns (y, mean, rstd); mean and rstd [n, groups] fp32 are what the backward pass takes."""
    _operands(x, weight, bias, out, workspace=workspace, dev_status=dev_status)
    n, s, c, ldx = _positions(x)
    code = _affine(weight, bias, c)
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
        ldy = c
    else:
        assert out.shape == x.shape and out.dtype == x.dtype
        ldy = _positions(out)[3]
    mean, rstd = x.new_empty((n, groups), dtype=torch.float32), x.new_empty((n, groups), dtype=torch.float32)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    while True:
        status = lib().mvue_group_norm_act(x.data_ptr(), _dtype_code(x), n, s, c, ldx, groups, _ptr(weight), _ptr(bias), code, eps,
                                           MVUE_ACTS[act], out.data_ptr(), ldy, mean.data_ptr(), rstd.data_ptr(), _ptr(workspace),
                                           ws_bytes, _ptr(dev_status), _stream_ptr())
        need = 0 if status != MVUE_ERR_WORKSPACE else mvue_group_norm_workspace_bytes(n, s, c, groups)
        if need <= ws_bytes:
            break
        workspace, ws_bytes = x.new_empty(need, dtype=torch.uint8), need       # only maps that no cluster holds need it
    _check(status, "mvue_group_norm_act")
    return out, mean, rstd


def mvue_group_norm_act_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, groups: int,
                                 weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, *, act: str = "none",
                                 out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                                 dev_status: torch.Tensor | None = None):
    """Backward pass of mvue_group_norm_act.  Returns (dx, dweight, dbias); the last two [c] fp32."""
    _operands(x, dy, mean, rstd, weight, bias, out, workspace=workspace, dev_status=dev_status)
    n, s, c, ldx = _positions(x)
    assert dy.shape == x.shape and dy.dtype is x.dtype
    for t in (mean, rstd):
        assert t.dim() == 2 and t.shape[1] == groups and t.numel() == n * groups and t.dtype is torch.float32 and t.is_contiguous()
    code = _affine(weight, bias, c)
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
        lddx = c
    else:
        assert out.shape == x.shape and out.dtype == x.dtype
        lddx = _positions(out)[3]
    dweight, dbias = x.new_empty(c, dtype=torch.float32), x.new_empty(c, dtype=torch.float32)
    need = mvue_group_norm_workspace_bytes(n, s, c, groups)
    if workspace is None or workspace.numel() * workspace.element_size() < need:
        workspace = x.new_empty(need, dtype=torch.uint8)
    _check(lib().mvue_group_norm_act_backward(dy.data_ptr(), _positions(dy)[3], x.data_ptr(), ldx, _dtype_code(x), n, s, c, groups,
                                              mean.data_ptr(), rstd.data_ptr(), _ptr(weight), _ptr(bias), code, MVUE_ACTS[act],
                                              out.data_ptr(), lddx, dweight.data_ptr(), dbias.data_ptr(), workspace.data_ptr(),
                                              workspace.numel() * workspace.element_size(), _ptr(dev_status), _stream_ptr()),
           "mvue_group_norm_act_backward")
    return out, dweight, dbias


def mvue_selftest_group_norm_timeout(polls: int, x: torch.Tensor, groups: int, mean: torch.Tensor, rstd: torch.Tensor, out: torch.Tensor,
                                     dev_status: torch.Tensor, dy: torch.Tensor | None = None) -> None:
    """A forward launch (or, with dy, a backward one) on contiguous x [n, s, c] whose blocks send one another nothing, so that
    their bounded waits run out: MVUE_ERR_DEVICE_TIMEOUT in dev_status, NaN in the outputs."""
    _operands(x, dy, mean, rstd, out, dev_status=dev_status)
    n, s, c = x.shape
    assert all(t is None or (t.shape == x.shape and t.dtype is x.dtype and t.is_contiguous()) for t in (x, dy, out))
    assert all(t.shape == (n, groups) and t.dtype is torch.float32 and t.is_contiguous() for t in (mean, rstd))
    workspace = x.new_empty(mvue_group_norm_workspace_bytes(n, s, c, groups), dtype=torch.uint8)
    _check(lib().mvue_selftest_group_norm_timeout(polls, x.data_ptr(), _ptr(dy), _dtype_code(x), n, s, c, groups, mean.data_ptr(),
                                                  rstd.data_ptr(), out.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                                  dev_status.data_ptr(), _stream_ptr()), "mvue_selftest_group_norm_timeout")


def _rows(t: torch.Tensor):
    """(rows, cols, ld) of a tensor [..., cols] whose rows lie one stride apart."""
    if t.dim() == 0:
        raise ValueError("wants [..., columns]")
    cols = t.shape[-1]
    if t.is_contiguous():
        return (t.numel() // cols if cols else 0), cols, cols
    if t.dim() == 1:
        t = t[None]
    n, s, cols, ld = _positions(t)
    return n * s, cols, ld


def mvue_layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, *, eps: float = 1e-5,
                    out: torch.Tensor | None = None):
    """layer_norm(x) * weight + bias over the last dimension of a CUDA tensor x [..., cols], fp32 or bf16, whose rows lie one stride
    apart.  Returns (y, mean, rstd); mean and rstd [...] fp32 are what the backward pass takes.  out may be x."""
    _operands(x, weight, bias, out)
    rows, cols, ldx = _rows(x)
    code = _affine(weight, bias, cols)
    if out is None:
        out = torch.empty_like(x) if ldx == cols else torch.empty_like(x, memory_format=torch.contiguous_format)
        ldy = cols
    else:
        assert out.shape == x.shape and out.dtype == x.dtype
        ldy = _rows(out)[2]
    mean = x.new_empty(rows, dtype=torch.float32) if x.dim() == 2 else x.new_empty(x.shape[:-1], dtype=torch.float32)
    rstd = torch.empty_like(mean)
    _check(lib().mvue_layer_norm(x.data_ptr(), _dtype_code(x), rows, cols, ldx, _ptr(weight), _ptr(bias), code, eps, out.data_ptr(), ldy,
                                 mean.data_ptr(), rstd.data_ptr(), _stream_ptr()), "mvue_layer_norm")
    return out, mean, rstd


@functools.lru_cache(maxsize=1024)
def _layer_norm_workspace(rows: int, cols: int, device: int) -> int:
    return mvue_layer_norm_workspace_bytes(rows, cols)


def mvue_layer_norm_workspace_bytes(rows: int, cols: int) -> int:
    b = ctypes.c_size_t()
    _check(lib().mvue_layer_norm_workspace_bytes(rows, cols, ctypes.byref(b)), "mvue_layer_norm_workspace_bytes")
    return b.value


def mvue_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: torch.Tensor | None = None, *,
                             out: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """Backward pass of mvue_layer_norm.  Returns (dx, dweight, dbias); the last two [cols] fp32.  out may be dy or x."""
    _operands(x, dy, mean, rstd, weight, out, workspace=workspace)
    rows, cols, ldx = _rows(x)
    assert dy.shape == x.shape and dy.dtype is x.dtype
    for t in (mean, rstd):
        assert t.numel() == rows and t.dtype is torch.float32 and t.is_contiguous()
    code = _affine(weight, None, cols)
    if out is None:
        out = torch.empty_like(x) if ldx == cols else torch.empty_like(x, memory_format=torch.contiguous_format)
        lddx = cols
    else:
        assert out.shape == x.shape and out.dtype == x.dtype
        lddx = _rows(out)[2]
    dweight = x.new_empty(cols, dtype=torch.float32)
    dbias = torch.empty_like(dweight)
    need = _layer_norm_workspace(rows, cols, x.get_device())
    size = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if size < need:
        workspace, size = x.new_empty(need, dtype=torch.uint8), need
    _check(lib().mvue_layer_norm_backward(dy.data_ptr(), cols if dy.is_contiguous() else _rows(dy)[2], x.data_ptr(), ldx, _dtype_code(x),
                                          rows, cols, mean.data_ptr(), rstd.data_ptr(), _ptr(weight), code, out.data_ptr(), lddx,
                                          dweight.data_ptr(), dbias.data_ptr(), _ptr(workspace), size, _stream_ptr()),
           "mvue_layer_norm_backward")
    return out, dweight, dbias


SCALE_BLOCK = 128                 # elements along the reduction axis that share a scale (MVUE_SCALE_BLOCK)


def mvue_quantize_e4m3(x: torch.Tensor, block_rows: int = 1, *, seed: int | None = None, codes: torch.Tensor | None = None,
                       scales: torch.Tensor | None = None):
    """e4m3 codes of a matrix x [rows, cols] (fp32 or bf16, unit column stride) with one power-of-two scale for each block of
    block_rows x 128 elements (block_rows: 1 for activations and gradients, 128 for weights).  seed: None rounds to the nearest code, ties
    to even; a number rounds at random without bias, keyed by it (another one each step).
    Returns (codes float8_e4m3fn [rows, cols], its rows 16-byte aligned; scales uint8: the exponent byte e of a scale 2^(e - 127),
    [ceil(cols / 128), rows] for block_rows = 1, [ceil(rows / 128), ceil(cols / 128)] for 128)."""
    _operands(x, codes, scales)
    if x.dim() != 2 or (x.stride(1) != 1 and x.shape[1] != 1):
        raise ValueError("wants a matrix with unit column stride")
    rows, cols = x.shape
    blocks = -(-cols // SCALE_BLOCK)
    shape = (blocks, rows) if block_rows == 1 else (-(-rows // SCALE_BLOCK), blocks)
    if codes is None:
        pitch = -(-cols // 16) * 16
        codes = x.new_empty(rows, pitch, dtype=torch.float8_e4m3fn)       # (sizes one by one: 1.2 us, as a tuple 1.7 us)
        if pitch != cols:
            codes = codes[:, :cols]
    elif codes.shape != x.shape:
        raise ValueError("codes have the shape of x")
    else:
        pitch = _code_pitch(codes)
    if scales is None:
        scales = x.new_empty(*shape, dtype=torch.uint8)
    else:
        _scale_bytes(scales, shape)
    _check(lib().mvue_quantize_e4m3(x.data_ptr(), _dtype_code(x), rows, cols, x.stride(0) if rows > 1 else cols, block_rows,
                                    MVUE_OPT_NONE if seed is None else MVUE_OPT_STOCHASTIC_ROUNDING, (seed or 0) & (2**64 - 1),
                                    codes.data_ptr(), pitch, scales.data_ptr(), _stream_ptr()), "mvue_quantize_e4m3")
    return codes, scales


_CODE_DTYPES = (torch.float8_e4m3fn, torch.uint8)


def _code_pitch(codes: torch.Tensor) -> int:
    """Bytes from row to row of a matrix of e4m3 codes."""
    if codes.dim() == 2 and codes.dtype in _CODE_DTYPES:
        (rows, cols), (pitch, step) = codes.shape, codes.stride()
        if step == 1 or cols == 1:
            return pitch if rows > 1 else -(-cols // 16) * 16
    raise ValueError("codes are a float8_e4m3fn matrix with unit column stride")


def _scale_bytes(scales: torch.Tensor, shape: tuple[int, int]) -> None:
    if scales.dtype is not torch.uint8 or scales.shape != shape or not scales.is_contiguous():
        raise ValueError(f"wants contiguous uint8 scales {list(shape)}")


def _scaled_gemm(name, forward, a, a_scales, W, W_scales, out, out_dtype, dev_status):
    _operands(a, a_scales, W, W_scales, out, dev_status=dev_status)
    lda, ldw = _code_pitch(a), _code_pitch(W)
    rows, k = a.shape
    outs, ins = W.shape
    n = outs if forward else ins
    if k != (ins if forward else outs):
        raise ValueError("the operands differ along the reduction axis")
    _scale_bytes(a_scales, (-(-k // SCALE_BLOCK), rows))
    _scale_bytes(W_scales, (-(-outs // SCALE_BLOCK), -(-ins // SCALE_BLOCK)))
    if out is None:
        out = a.new_empty(rows, n, dtype=out_dtype)
        ldc = n
    else:
        assert out.shape == (rows, n) and (out.stride(1) == 1 or n == 1)
        ldc = out.stride(0) if rows > 1 else n
    status = getattr(lib(), name)(a.data_ptr(), a_scales.data_ptr(), rows, k, lda, W.data_ptr(), W_scales.data_ptr(), n, ldw, out.data_ptr(),
                                  _dtype_code(out), ldc, None if dev_status is None else dev_status.data_ptr(), _stream_ptr())
    if status != 0:
        _check(status, name)
    return out


def mvue_scaled_forward_gemm(x: torch.Tensor, x_scales: torch.Tensor, W: torch.Tensor, W_scales: torch.Tensor, *,
                             out: torch.Tensor | None = None, out_dtype=torch.bfloat16, dev_status: torch.Tensor | None = None) -> torch.Tensor:
    """x . W^T from e4m3 codes: x [tokens, in] with scales [ceil(in / 128), tokens], W [out, in] with scales
    [ceil(out / 128), ceil(in / 128)] (what mvue_quantize_e4m3 returns for block_rows = 1 and 128).  bf16 or fp32 out."""
    return _scaled_gemm("mvue_scaled_forward_gemm", True, x, x_scales, W, W_scales, out, out_dtype, dev_status)


def mvue_scaled_backward_gemm(g: torch.Tensor, g_scales: torch.Tensor, W: torch.Tensor, W_scales: torch.Tensor, *,
                              out: torch.Tensor | None = None, out_dtype=torch.bfloat16, dev_status: torch.Tensor | None = None) -> torch.Tensor:
    """g . W from e4m3 codes: g [tokens, out] with scales [ceil(out / 128), tokens]; W and its scales as in the forward product."""
    return _scaled_gemm("mvue_scaled_backward_gemm", False, g, g_scales, W, W_scales, out, out_dtype, dev_status)


def _matrices(t: torch.Tensor):
    """(batch, rows, cols, ld, stride) of a tensor [..., rows, cols] whose matrices lie one stride apart."""
    if t.dim() < 2 or (t.stride(-1) != 1 and t.shape[-1] != 1):
        raise ValueError("wants [..., rows, columns] with unit column stride")
    rows, cols = t.shape[-2:]
    ld = t.stride(-2) if rows > 1 else cols
    batch, stride, step = 1, rows * ld, None
    for size, s in zip(reversed(t.shape[:-2]), reversed(t.stride()[:-2])):                # innermost matrix first
        if size != 1 and t.numel():
            if step is None:
                stride = s
            elif s != step:
                raise ValueError("matrices are not one stride apart")
            step = s * size
        batch *= size
    return batch, rows, cols, ld, stride


def mvue_orthogonalize_workspace_bytes(batch: int, rows: int, cols: int) -> int:
    b = ctypes.c_size_t()
    _check(lib().mvue_orthogonalize_workspace_bytes(batch, rows, cols, ctypes.byref(b)), "mvue_orthogonalize_workspace_bytes")
    return b.value


def mvue_orthogonalize(x: torch.Tensor, *, steps: int = 5, out: torch.Tensor | None = None, out_dtype=None,
                       workspace: torch.Tensor | None = None, dev_status: torch.Tensor | None = None) -> torch.Tensor:
    """Each matrix of x [..., rows, cols] (fp32 or bf16) with its singular values brought towards one by `steps` Newton-Schulz steps, its
    singular vectors kept.  Returns a tensor of out_dtype (x's own unless given); out may be x.  From 1024 columns (or rows) on, how many matrices
    a call has decides in what order a matrix's sums are added: alone and among others it may differ by roundings."""
    _operands(x, out, workspace=workspace, dev_status=dev_status)
    batch, rows, cols, ldx, stride = _matrices(x)
    if out is None:
        out = torch.empty_like(x, dtype=out_dtype, memory_format=torch.contiguous_format)
    assert out.shape == x.shape
    _, _, _, ldo, out_stride = _matrices(out)
    need = mvue_orthogonalize_workspace_bytes(batch, rows, cols)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = x.new_empty(need, dtype=torch.uint8)
    _check(lib().mvue_orthogonalize(x.data_ptr(), _dtype_code(x), batch, rows, cols, ldx, stride, steps, out.data_ptr(), _dtype_code(out), ldo,
                                    out_stride, _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                    _ptr(dev_status), _stream_ptr()), "mvue_orthogonalize")
    return out


def mvue_muon_workspace_bytes(tensors: ctypes.Array, count: int) -> int:
    b = ctypes.c_size_t()
    _check(lib().mvue_muon_workspace_bytes(tensors, count, ctypes.byref(b)), "mvue_muon_workspace_bytes")
    return b.value


def mvue_muon_step(tensors: ctypes.Array, count: int, config: MuonConfig, workspace: torch.Tensor | None,
                   dev_status: torch.Tensor | None = None) -> None:
    """One Muon step over `count` entries of a ctypes array of MuonTensor (optim.MuonPlan fills and keeps one)."""
    _check(lib().mvue_muon_step(tensors, count, config, _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                _ptr(dev_status), _stream_ptr()), "mvue_muon_step")

"""Python binding of the C ABI in include/mvue.h: argument marshalling only.

Tensors are torch CUDA tensors used purely as device memory; every function passes
raw pointers, sizes and the current CUDA stream to the library.  There is no
fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import torch

_LIB_PATH = Path(__file__).resolve().parent / "libmvue_b200.so"
_lib = None

MVUE_F32, MVUE_BF16 = 0, 1
MVUE_LAYOUT_CANONICAL = 0
MVUE_LAYOUT_TC = 1
MVUE_JOINT_TABLE, MVUE_JOINT_SYSTEMATIC, MVUE_JOINT_APPROX = 0, 1, 2
MVUE_OPT_NONE, MVUE_OPT_STOCHASTIC_ROUNDING, MVUE_OPT_EPS16 = 0, 1, 2
MVUE_ERR_WORKSPACE = -7
MVUE_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}

EXPORTS = ("mvue_version", "mvue_status_string", "mvue_last_cuda_error", "mvue_packed_sizes",
           "mvue_prune", "mvue_prune_joint", "mvue_prune_opts", "mvue_prune_4of8", "mvue_unpack", "mvue_sparse_update_gemm", "mvue_sparse_backward_gemm",
           "mvue_sparse_backward_gemm_pruned",
           "mvue_gemm_workspace_bytes", "mvue_sparse_update_gemm_noalloc", "mvue_fused_update_gemm", "mvue_fused_update_gemm_joint",
           "mvue_probe_sparse_mma", "mvue_selftest_wait_timeout",
           "mvue_adamw_step", "mvue_embedding", "mvue_embedding_grad", "mvue_embedding_grad_workspace_bytes",
           "mvue_group_norm_act", "mvue_group_norm_act_backward", "mvue_group_norm_workspace_bytes",
           "mvue_selftest_group_norm_timeout")


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

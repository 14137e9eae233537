"""Optimisers over the tensors of a model.  AdamW: one library call (one launch for up to 320 tensors) per step.

    plan = AdamWPlan.zeros(params, state_bits=8)            # or AdamWPlan(params, exp_avgs, exp_avg_sqs, ...)
    plan.step(grads, step=t, lr=1e-3)                       # grads: as mvue_sparse_update_gemm left them

Muon, for the weights that are matrices: one library call per step.

    plan = MuonPlan.zeros(weights)                          # or MuonPlan(weights, momentums, ...)
    plan.step(grads, lr=1e-3)
"""
from __future__ import annotations

import torch

from . import binding

BLOCK = 256                       # elements that share one scale of the 8-bit states (MVUE_ADAMW_BLOCK)


def _same_layout(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether element i in memory of one is element i in memory of the other (all dense)."""
    if a.numel() != b.numel():
        return False
    if a.is_contiguous() and b.is_contiguous():
        return True
    # the stride of a dimension of size one says nothing
    return a.shape == b.shape and all(n == 1 or s == t for n, s, t in zip(a.shape, a.stride(), b.stride()))


def _dense(t: torch.Tensor) -> bool:
    """Whether the tensor covers its memory without gaps or overlaps, in any order of its dimensions."""
    if t.numel() == 0:
        return True
    want = 1
    for size, stride in sorted(((n, s) for n, s in zip(t.shape, t.stride()) if n != 1), key=lambda d: d[1]):
        if stride != want:
            return False
        want *= size
    return True


def _addresses(tensors) -> list[int]:
    return list(map(torch.Tensor.data_ptr, tensors))


class AdamWPlan:
    """The tensors of an optimiser, marshalled once.  The step updates them in place, in the memory that they had when the plan
    was made: the plan keeps that memory (do not resize it), and once a param's memory has been exchanged (p.data = ..., a
    move to another device) the model wants a new plan.  step() with gradients raises then; without, it goes on with the old memory.

    params:     list of CUDA tensors, fp32 or bf16, dense (any dimension order).
    exp_avgs, exp_avg_sqs: 32-bit states: fp32 tensors; 8-bit states: torch.float8_e4m3fn tensors (of m and of sqrt(v)) with
                exp_avg_scales, exp_avg_sq_scales: fp32 tensors of ceil(numel / 256) elements.
    masters:    optional list of fp32 copies for bf16 params (None entries allowed).
    grads:      optional list of gradient buffers (fp32 or bf16) that every step reads; otherwise step() takes them.
    """

    def __init__(self, params, exp_avgs, exp_avg_sqs, *, masters=None, exp_avg_scales=None, exp_avg_sq_scales=None, grads=None):
        n = len(params)
        self.state_bits = 8 if exp_avg_scales is not None else 32
        state = torch.float8_e4m3fn if self.state_bits == 8 else torch.float32
        if (exp_avg_scales is None) != (exp_avg_sq_scales is None):
            raise ValueError("8-bit states have both lists of scales, 32-bit states none")
        masters = [None] * n if masters is None else masters
        scales = (exp_avg_scales, exp_avg_sq_scales) if self.state_bits == 8 else ([None] * n, [None] * n)
        if any(len(x) != n for x in (exp_avgs, exp_avg_sqs, masters, *scales)):
            raise ValueError("the lists differ in length")
        self._array = (binding.AdamWTensor * n)()
        self._device = params[0].device if n else None
        for e, p, w, m, v, ms, vs in zip(self._array, params, masters, exp_avgs, exp_avg_sqs, *scales):
            if not p.is_cuda or p.device != self._device or not _dense(p):
                raise ValueError("params are dense CUDA tensors of one device")
            e.param_dtype, e.numel, e.param = binding._dtype_code(p), p.numel(), p.data_ptr()
            for t, dtype, field in ((w, torch.float32, "master"), (m, state, "exp_avg"), (v, state, "exp_avg_sq")):
                if t is None and field == "master":
                    continue
                if t.dtype != dtype or t.device != p.device or not _same_layout(t, p):
                    raise ValueError(f"{field}: wants {dtype}, the param's device, size and strides")
                setattr(e, field, t.data_ptr())
            if w is not None and p.dtype != torch.bfloat16:
                raise ValueError("a float copy belongs to a bf16 param")
            for t, field in ((ms, "exp_avg_scale"), (vs, "exp_avg_sq_scale")):
                if t is None:
                    continue
                if t.dtype != torch.float32 or t.device != p.device or not t.is_contiguous() or t.numel() != -(-p.numel() // BLOCK):
                    raise ValueError(f"{field}: wants ceil(numel / {BLOCK}) fp32 elements on the param's device")
                setattr(e, field, t.data_ptr())
        self.params, self.exp_avgs, self.exp_avg_sqs, self.masters = list(params), list(exp_avgs), list(exp_avg_sqs), list(masters)
        self.exp_avg_scales, self.exp_avg_sq_scales = (list(scales[0]), list(scales[1]))
        # tensors of the plan's own over the same memory, which outlives an exchange of a tensor's data thereby
        self._memory = [t.detach() for ts in (params, masters, exp_avgs, exp_avg_sqs, *scales) for t in ts if t is not None]
        self._addresses = _addresses(self.params)
        self._config = binding.AdamWConfig(state_bits=self.state_bits)
        self._grads = self._grad_addresses = None
        if grads is not None:
            self._point(grads)
            self._memory += [g.detach() for g in grads]
            self._grad_addresses = None

    @classmethod
    def zeros(cls, params, *, state_bits: int = 32, master: bool = False, grads=None) -> "AdamWPlan":
        """A plan with fresh (zero) states, and float copies of the bf16 params if asked for."""
        if state_bits not in (8, 32):
            raise ValueError("states have 8 or 32 bits")
        dtype = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        m, v = ([torch.empty_like(p, dtype=torch.uint8 if state_bits == 8 else dtype).zero_().view(dtype) for p in params] for _ in range(2))
        scales = {}
        if state_bits == 8:
            scales = {k: [torch.zeros(-(-p.numel() // BLOCK), device=p.device) for p in params]
                      for k in ("exp_avg_scales", "exp_avg_sq_scales")}
        masters = [p.float() if p.dtype == torch.bfloat16 else None for p in params] if master else None
        return cls(params, m, v, masters=masters, grads=grads, **scales)

    def _point(self, grads) -> None:
        if len(grads) != len(self._array):
            raise ValueError("one gradient for each param")
        if _addresses(self.params) != self._addresses:
            raise ValueError("a param's memory has been exchanged since the plan was made: make a new plan")
        found = []
        for p, g in zip(self.params, grads):
            if g.device != self._device or not _same_layout(g, p):
                raise ValueError("a gradient has its param's device, size and strides")
            found.append((binding._dtype_code(g), g.data_ptr()))
        for e, (code, ptr) in zip(self._array, found):                       # nothing was refused
            e.grad_dtype, e.grad = code, ptr
        self._grads, self._grad_addresses = list(grads), [ptr for _, ptr in found]

    def step(self, grads=None, *, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
             weight_decay: float = 0.01, grad_scale: float = 1.0, dev_grad_scale: torch.Tensor | None = None, seed: int | None = None,
             stochastic_rounding: bool = False) -> None:
        """One step (step >= 1 counts them) on the current stream of the params' device.  grads: this step's gradients (they stay the plan's
        until others are given); None reads the buffers the plan has.  seed keys what is rounded at random (8-bit states; bf16
        params without a float copy when stochastic_rounding): None takes the step's number; a seed of one's own has to be another
        one each step, since the same random numbers every time are a fixed threshold for each element, which averages and
        params do not cross."""
        if grads is not None:
            self._point(grads)
        elif self._grads is None and len(self._array):
            raise ValueError("no gradients")
        elif self._grad_addresses is not None and _addresses(self._grads) != self._grad_addresses:
            raise ValueError("a gradient's memory has been exchanged since it was given")
        if dev_grad_scale is not None and (dev_grad_scale.dtype != torch.float32 or dev_grad_scale.device != self._device
                                           or dev_grad_scale.numel() != 1):
            raise ValueError("dev_grad_scale is one fp32 element on the params' device")
        c = self._config
        c.lr, c.beta1, c.beta2, c.eps, c.weight_decay, c.step, c.grad_scale = lr, beta1, beta2, eps, weight_decay, step, grad_scale
        c.dev_grad_scale = None if dev_grad_scale is None else dev_grad_scale.data_ptr()
        c.seed = (step if seed is None else seed) & (2**64 - 1)
        c.options = binding.MVUE_OPT_STOCHASTIC_ROUNDING if stochastic_rounding else binding.MVUE_OPT_NONE
        if self._device is None or self._device.index == torch.cuda.current_device():
            binding.mvue_adamw_step(self._array, len(self._array), c)
        else:
            with torch.cuda.device(self._device):
                binding.mvue_adamw_step(self._array, len(self._array), c)


class MuonPlan:
    """The matrices of a Muon optimiser, marshalled once, and the workspace of its steps.  As AdamWPlan, the plan keeps the memory that
    its tensors had when it was made, and a param whose memory has been exchanged is refused with the next gradients.

    params:     list of 2-D CUDA tensors, fp32 or bf16, contiguous.
    momentums:  fp32 tensors of the same shapes.
    masters:    optional list of fp32 copies for bf16 params (None entries allowed).
    grads:      optional list of gradient buffers (fp32 or bf16) that every step reads; otherwise step() takes them.
    """

    def __init__(self, params, momentums, *, masters=None, grads=None):
        n = len(params)
        masters = [None] * n if masters is None else masters
        if len(momentums) != n or len(masters) != n:
            raise ValueError("the lists differ in length")
        self._array = (binding.MuonTensor * n)()
        self._device = params[0].device if n else None
        for e, p, w, m in zip(self._array, params, masters, momentums):
            if not p.is_cuda or p.device != self._device or p.dim() != 2 or not p.is_contiguous():
                raise ValueError("params are contiguous matrices on one CUDA device")
            e.param_dtype, e.rows, e.cols, e.param = binding._dtype_code(p), p.shape[0], p.shape[1], p.data_ptr()
            for t, field in ((w, "master"), (m, "momentum")):
                if t is None and field == "master":
                    continue
                if t.dtype != torch.float32 or t.device != p.device or t.shape != p.shape or not t.is_contiguous():
                    raise ValueError(f"{field}: wants a contiguous fp32 tensor of the param's shape on its device")
                setattr(e, field, t.data_ptr())
            if w is not None and p.dtype != torch.bfloat16:
                raise ValueError("a float copy belongs to a bf16 param")
        self.params, self.momentums, self.masters = list(params), list(momentums), list(masters)
        self._memory = [t.detach() for ts in (params, masters, momentums) for t in ts if t is not None]
        self._addresses = _addresses(self.params)
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in self._memory if t.numel())
        if any(end > start for (_, end), (start, _) in zip(spans, spans[1:])):
            raise ValueError("two of the plan's tensors share memory")
        self._config = binding.MuonConfig()
        need = binding.mvue_muon_workspace_bytes(self._array, n)
        self._workspace = torch.empty(need, dtype=torch.uint8, device=self._device) if need else None
        self._stream = torch.cuda.current_stream(self._device) if need else None        # the workspace's own
        self._grads = self._grad_addresses = None
        if grads is not None:
            self._point(grads)
            self._memory += [g.detach() for g in grads]
            self._grad_addresses = None

    @classmethod
    def zeros(cls, params, *, master: bool = False, grads=None) -> "MuonPlan":
        """A plan with fresh (zero) momentum, and float copies of the bf16 params if asked for."""
        momentums = [torch.zeros_like(p, dtype=torch.float32) for p in params]
        masters = [p.float() if p.dtype == torch.bfloat16 else None for p in params] if master else None
        return cls(params, momentums, masters=masters, grads=grads)

    def _point(self, grads) -> None:
        if len(grads) != len(self._array):
            raise ValueError("one gradient for each param")
        if _addresses(self.params) != self._addresses:
            raise ValueError("a param's memory has been exchanged since the plan was made: make a new plan")
        found = []
        for p, g in zip(self.params, grads):
            if g.device != self._device or g.shape != p.shape or not g.is_contiguous():
                raise ValueError("a gradient is contiguous and has its param's device and shape")
            found.append((binding._dtype_code(g), g.data_ptr()))
        for e, (code, ptr) in zip(self._array, found):                       # nothing was refused
            e.grad_dtype, e.grad = code, ptr
        self._grads, self._grad_addresses = list(grads), [ptr for _, ptr in found]

    def step(self, grads=None, *, lr: float, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.01, ns_steps: int = 5,
             scale: str = "rms", grad_scale: float = 1.0, dev_grad_scale: torch.Tensor | None = None, stochastic_rounding: bool = False,
             seed: int | None = None, dev_status: torch.Tensor | None = None) -> None:
        """One step on the current stream of the params' device.  grads: this step's gradients (they stay the plan's until others are
        given); None reads the buffers the plan has.  scale: "rms" multiplies the orthogonal update by 0.2 sqrt(max(rows, cols)), which makes
        it as large as AdamW's; "shape" by sqrt(max(1, rows / cols)).  stochastic_rounding (bf16 params without a float copy)
        wants a seed, another one each step.  Steps of one plan share its workspace: they run in the order of one stream, and a graph
        that has captured one needs the plan alive."""
        if grads is not None:
            self._point(grads)
        elif self._grads is None and len(self._array):
            raise ValueError("no gradients")
        elif self._grad_addresses is not None and _addresses(self._grads) != self._grad_addresses:
            raise ValueError("a gradient's memory has been exchanged since it was given")
        if dev_grad_scale is not None and (dev_grad_scale.dtype != torch.float32 or dev_grad_scale.device != self._device
                                           or dev_grad_scale.numel() != 1):
            raise ValueError("dev_grad_scale is one fp32 element on the params' device")
        if dev_status is not None and (dev_status.dtype is not torch.int32 or dev_status.device != self._device or dev_status.numel() == 0):
            raise ValueError("dev_status is an int32 tensor on the params' device")
        if stochastic_rounding and seed is None:
            raise ValueError("stochastic rounding wants a seed, another one each step")
        if scale not in binding.MVUE_MUON_SCALES:
            raise ValueError(f"scale is one of {', '.join(binding.MVUE_MUON_SCALES)}")
        if self._workspace is not None and not torch.cuda.is_current_stream_capturing():
            stream = torch.cuda.current_stream(self._device)
            if stream != self._stream:
                self._workspace.record_stream(stream)        # it outlives the plan until this step is done
        c = self._config
        c.lr, c.momentum, c.weight_decay, c.grad_scale = lr, momentum, weight_decay, grad_scale
        c.dev_grad_scale = None if dev_grad_scale is None else dev_grad_scale.data_ptr()
        c.seed = (seed or 0) & (2**64 - 1)
        c.ns_steps, c.scale_rule = ns_steps, binding.MVUE_MUON_SCALES[scale]
        c.options = (binding.MVUE_OPT_NESTEROV if nesterov else 0) | (binding.MVUE_OPT_STOCHASTIC_ROUNDING if stochastic_rounding else 0)
        if self._device is None or self._device.index == torch.cuda.current_device():
            binding.mvue_muon_step(self._array, len(self._array), c, self._workspace, dev_status)
        else:
            with torch.cuda.device(self._device):
                binding.mvue_muon_step(self._array, len(self._array), c, self._workspace, dev_status)

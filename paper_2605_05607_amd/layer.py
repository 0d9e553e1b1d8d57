"""Device-buffer bookkeeping around the C ABI: allocates the caller-owned arrays once and forwards every step
to the library.  No arithmetic happens here."""
from __future__ import annotations

import math

import numpy as np

from . import binding as B


def to_device(a: np.ndarray, device="cuda"):
    """Host array -> device tensor.  uint16 arrays are bf16 bit patterns and become torch.bfloat16."""
    import torch
    a = np.ascontiguousarray(a)
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(a).to(device)


def from_device_bf16_bits(t) -> np.ndarray:
    import torch
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


class MoELayer:
    """All device state of one layer: routing outputs, dispatch tables, packed weights, workspaces, y."""

    def __init__(self, cfg, device="cuda", unfused: bool = False):
        import torch
        self.cfg = cfg
        self.device = device
        self.shape = B.shape_of(cfg)
        s = self.shape
        self.elt_dtype = torch.bfloat16 if cfg.dtype == B.MOE_BF16 else torch.float32
        n = max(1, s.T * s.k)
        self.topk_idx = torch.empty(n, dtype=torch.int32, device=device)
        self.topk_w = torch.empty(n, dtype=torch.float32, device=device)
        self.tables = B.DispatchTables(s, device)
        self.dispatch_ws = torch.empty(max(1, B.moe_dispatch_workspace_bytes(s)), dtype=torch.uint8, device=device)
        nbytes = B.moe_unfused_workspace_bytes(s) if unfused else B.moe_forward_workspace_bytes(s)
        self.forward_ws = torch.empty(max(1, nbytes), dtype=torch.uint8, device=device)
        self.y = torch.empty((max(1, s.T), s.d), dtype=self.elt_dtype, device=device)
        self.packed_gate_up = None
        self.packed_down = None
        self.fp8_gate_up = None
        self.fp8_down = None
        self.optimizer = None

    def load_weights(self, W_gate: np.ndarray, W_up: np.ndarray, W_down: np.ndarray) -> None:
        import torch
        s = self.shape
        self.packed_gate_up = torch.empty(B.moe_packed_weight_bytes(s, 0), dtype=torch.uint8, device=self.device)
        self.packed_down = torch.empty(B.moe_packed_weight_bytes(s, 1), dtype=torch.uint8, device=self.device)
        self.optimizer = None  # (it has weights of its own, and would bring those back)
        g, u, d = (to_device(a, self.device) for a in (W_gate, W_up, W_down))
        B.moe_pack_weights(s, g, u, d, self.packed_gate_up, self.packed_down)
        torch.cuda.synchronize()
        del g, u, d

    def load_weights_fp8(self, W_gate: np.ndarray, W_up: np.ndarray, W_down: np.ndarray, h_scale: np.ndarray) -> None:
        """Quantise and pack the weights for the FP8 form of the GEMMs; h_scale [E_loc] is the static scale of h."""
        import torch
        s = self.shape
        self.fp8_gate_up = torch.empty(B.moe_fp8_packed_weight_bytes(s, 0), dtype=torch.uint8, device=self.device)
        self.fp8_down = torch.empty(B.moe_fp8_packed_weight_bytes(s, 1), dtype=torch.uint8, device=self.device)
        self.fp8_ws = torch.empty(max(1, B.moe_fp8_forward_workspace_bytes(s)), dtype=torch.uint8, device=self.device)
        self.h_scale = to_device(np.ascontiguousarray(h_scale, dtype=np.float32), self.device)
        g, u, d = (to_device(a, self.device) for a in (W_gate, W_up, W_down))
        B.moe_fp8_pack_weights(s, g, u, d, self.fp8_gate_up, self.fp8_down)
        torch.cuda.synchronize()
        del g, u, d

    def forward_fp8(self, x, events=None) -> None:
        B.moe_fp8_fused_forward(self.shape, x, self.topk_idx, self.topk_w, self.tables, self.fp8_gate_up,
                                self.fp8_down, self.h_scale, self.y, self.fp8_ws, events)

    def forward_fp8_codes(self, codes, scales, events=None) -> None:
        """The FP8 forward on token rows that are codes already (``norm`` writes them)."""
        B.moe_fp8_fused_forward_codes(self.shape, codes, scales, self.topk_idx, self.topk_w, self.tables, self.fp8_gate_up,
                                      self.fp8_down, self.h_scale, self.y, self.fp8_ws, events)

    def enable_norm(self, weight, eps: float = 1e-6) -> None:
        """Buffers of the norm in front of the layer: the sum of the residual stream, the layer's input and its codes."""
        import torch
        s, dev = self.shape, self.device
        self.norm_weight = weight if isinstance(weight, torch.Tensor) else to_device(weight, dev)
        if self.norm_weight.dtype != self.elt_dtype or self.norm_weight.numel() != s.d:
            raise ValueError("the norm's weight has d values in the layer's element type")
        if self.norm_weight.device != self.y.device or not self.norm_weight.is_contiguous():
            raise ValueError("the norm's weight is contiguous, on the layer's device")
        self.norm_eps = eps
        self.norm_sum, self.x = (torch.empty((max(1, s.T), s.d), dtype=self.elt_dtype, device=dev) for _ in range(2))
        self.x_codes = torch.empty((max(1, s.T), s.d), dtype=torch.uint8, device=dev)
        self.x_scales, self.rstd = (torch.empty(max(1, s.T), dtype=torch.float32, device=dev) for _ in range(2))
        self.norm_ws = torch.empty(max(1, B.moe_rmsnorm_backward_workspace_bytes(s.T, s.d)), dtype=torch.uint8, device=dev)
        self.d_norm_weight = torch.empty(s.d, dtype=torch.float32, device=dev)

    def norm(self, h, residual=None, codes: bool = False) -> None:
        """x (and, for forward_fp8_codes, its codes) from the output h of what comes before the layer; with a residual the new
        one is left in ``norm_sum``.  norm_backward reads that (without a residual h) again."""
        B.moe_rmsnorm(self.shape.T, self.shape.d, self.shape.dtype, h, residual, self.norm_weight, self.norm_eps,
                      None if residual is None else self.norm_sum, self.x, self.x_codes if codes else None,
                      self.x_scales if codes else None, self.rstd)
        self._normed = h if residual is None else self.norm_sum

    def norm_backward(self, dx, dsum, dh) -> None:
        """dh from the gradient dx of the layer's input and dsum of the residual stream (or None); d_norm_weight."""
        B.moe_rmsnorm_backward(self.shape.T, self.shape.d, self.shape.dtype, self._normed, self.norm_weight, self.rstd, dx,
                               dsum, dh, self.d_norm_weight, self.norm_ws)

    def enable_training(self, W_gate: np.ndarray, W_up: np.ndarray, W_down: np.ndarray, wgrad: bool = True) -> None:
        """Buffers of the training path: transposed weight packs, the kept activations, gradients, workspace."""
        import torch
        s = self.shape
        dev = self.device
        self.optimizer = None  # (it has the present weights, and reads the present gradients)
        self.packed_down_t = torch.empty(B.moe_backward_packed_weight_bytes(s, 0), dtype=torch.uint8, device=dev)
        self.packed_gate_up_t = torch.empty(B.moe_backward_packed_weight_bytes(s, 1), dtype=torch.uint8, device=dev)
        g, u, d = (to_device(a, dev) for a in (W_gate, W_up, W_down))
        B.moe_pack_weights_backward(s, g, u, d, self.packed_down_t, self.packed_gate_up_t)
        torch.cuda.synchronize()
        del g, u, d
        self.kept = torch.empty(max(1, B.moe_train_kept_bytes(s)), dtype=torch.uint8, device=dev)
        self.backward_ws = torch.empty(max(1, B.moe_backward_workspace_bytes(s)), dtype=torch.uint8, device=dev)
        self.dx = torch.empty((max(1, s.T), s.d), dtype=torch.bfloat16, device=dev)
        self.d_topk_w = torch.empty(max(1, s.T * s.k), dtype=torch.float32, device=dev)
        El = self.cfg.E_loc
        if wgrad:
            self.dW_gate = torch.empty((El, s.d, s.f), dtype=torch.bfloat16, device=dev)
            self.dW_up = torch.empty((El, s.d, s.f), dtype=torch.bfloat16, device=dev)
            self.dW_down = torch.empty((El, s.f, s.d), dtype=torch.bfloat16, device=dev)
        else:
            self.dW_gate = self.dW_up = self.dW_down = None

    def enable_optimizer(self, W_gate: np.ndarray, W_up: np.ndarray, W_down: np.ndarray, lr: float, **kw) -> None:
        """An AdamW step on the three expert weights, after load_weights and enable_training with weight gradients: fp32 parameters,
        bf16 copies of them and the optimizer (`kw` as for AdamW).  Either of the two called again ends it."""
        import torch
        if getattr(self, "dW_gate", None) is None or self.packed_gate_up is None:
            raise ValueError("load_weights and enable_training with weight gradients come first")
        self.weights = [to_device(a, self.device) for a in (W_gate, W_up, W_down)]
        self.masters = [w.to(torch.float32) for w in self.weights]
        self.optimizer = AdamW(self.masters, [self.dW_gate, self.dW_up, self.dW_down], lr, copies=self.weights, **kw)

    def optimizer_step(self, **kw) -> None:
        """The step with the gradients of the last `backward`, and the new weights packed for the next forward and backward, in every
        form that the layer holds (FP8 too after load_weights_fp8; h_scale stays as it is).  A captured step packs the forms that
        were there when it was captured."""
        if self.optimizer is None:
            raise ValueError("enable_optimizer comes first, and again after load_weights or enable_training")
        self.optimizer.step(**kw)
        B.moe_pack_weights(self.shape, *self.weights, self.packed_gate_up, self.packed_down)
        B.moe_pack_weights_backward(self.shape, *self.weights, self.packed_down_t, self.packed_gate_up_t)
        if self.fp8_gate_up is not None:
            B.moe_fp8_pack_weights(self.shape, *self.weights, self.fp8_gate_up, self.fp8_down)

    def forward_train(self, x) -> None:
        B.moe_fused_forward_train(self.shape, x, self.topk_idx, self.topk_w, self.tables, self.packed_gate_up,
                                  self.packed_down, self.y, self.kept, self.forward_ws)

    def backward(self, x, dy) -> None:
        B.moe_fused_backward(self.shape, x, dy, self.topk_idx, self.topk_w, self.tables, self.packed_down_t,
                             self.packed_gate_up_t, self.kept, self.dx, self.d_topk_w, self.dW_gate, self.dW_up,
                             self.dW_down, self.backward_ws)

    def backward_copies(self, x, dy) -> None:
        """The same with the weight gradients from transposed copies of the operands."""
        B.moe_fused_backward_copies(self.shape, x, dy, self.topk_idx, self.topk_w, self.tables, self.packed_down_t,
                                    self.packed_gate_up_t, self.kept, self.dx, self.d_topk_w, self.dW_gate, self.dW_up,
                                    self.dW_down, self.backward_ws)

    def route(self, logits) -> None:
        B.moe_route_topk(self.shape, logits, self.topk_idx, self.topk_w)

    def build_dispatch(self) -> None:
        B.moe_build_dispatch(self.shape, self.topk_idx, self.tables, self.dispatch_ws)

    def forward(self, x) -> None:
        B.moe_fused_forward(self.shape, x, self.topk_idx, self.topk_w, self.tables, self.packed_gate_up,
                            self.packed_down, self.y, self.forward_ws)

    def forward_two_launch(self, x, events=None) -> None:
        B.moe_fused_forward_two_launch(self.shape, x, self.topk_idx, self.topk_w, self.tables, self.packed_gate_up,
                                       self.packed_down, self.y, self.forward_ws, events)

    def forward_one_launch(self, x, events=None) -> None:
        B.moe_fused_forward_one_launch(self.shape, x, self.topk_idx, self.topk_w, self.tables, self.packed_gate_up,
                                       self.packed_down, self.y, self.forward_ws, events)

    def forward_resident(self, x, events=None) -> None:
        """GEMM-1, GEMM-2 and Combine in one launch."""
        B.moe_fused_forward_resident(self.shape, x, self.topk_idx, self.topk_w, self.tables, self.packed_gate_up,
                                     self.packed_down, self.y, self.forward_ws, events)

    def forward_unfused(self, x) -> None:
        B.moe_unfused_forward(self.shape, x, self.topk_idx, self.topk_w, self.tables, self.packed_gate_up,
                              self.packed_down, self.y, self.forward_ws)

    def step(self, logits, x) -> None:
        """One pass of the whole hot path."""
        B.moe_step(self.shape, logits, x, self.topk_idx, self.topk_w, self.tables, self.dispatch_ws, self.packed_gate_up,
                   self.packed_down, self.y, self.forward_ws)

    def y_host(self) -> np.ndarray:
        """y as float64 on the host (bf16 values widened exactly)."""
        import torch
        return self.y[: self.shape.T].to(torch.float64).cpu().numpy()


class AdamW:
    """One optimizer over a list of fp32 device tensors: holds both states and forwards every step to moe_adamw_step.

    grads: a tensor for each parameter, fp32 or bf16, read by every step.  copies: None, or a bf16 tensor (or None) for each
    parameter that receives its rounded value.  All arrays stay where they are in memory.  bits: 32 or 8, the states' width (8:
    E4M3 codes of m and of sqrt(v), a scale per 256 values).  weight_decay: one number, or one for each parameter.  states:
    [(m, v, m_scale, v_scale)] to go on from, zeros without; steps: steps taken so far, without skipped ones, as ``steps`` tells
    them.  device_scalars: lr, grad_scale and the number of the call live in device memory (``scalars``), so that a captured
    ``step`` advances with every replay; change lr and grad_scale there.  (Captured without, every replay is the same step.)
    """

    def __init__(self, params, grads, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, copies=None, bits=32, seed=0,
                 states=None, steps=0, device_scalars=False):
        import torch
        n = len(params)
        copies = [None] * n if copies is None else list(copies)
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        if bits not in (8, 32):
            raise ValueError("bits is 32 or 8")
        if not len(grads) == len(copies) == len(decay) == n or (states is not None and len(states) != n):
            raise ValueError("a gradient, copy, decay and state for each parameter")
        state = torch.float32 if bits == 32 else torch.uint8
        if states is None:
            states = []
            for p in params:
                m, v = (torch.zeros(p.numel(), dtype=state, device=p.device) for _ in range(2))
                scale = (torch.ones(-(-p.numel() // B.MOE_ADAMW_BLOCK), dtype=torch.float32, device=p.device)
                         for _ in range(2)) if bits == 8 else (None, None)
                states.append((m, v, *scale))
        for p, g, c, (m, v, ms, vs) in zip(params, grads, copies, states):
            blocks = -(-p.numel() // B.MOE_ADAMW_BLOCK)
            held = [(p, torch.float32, p.numel()), (g, g.dtype, p.numel()), (m, state, p.numel()), (v, state, p.numel())]
            held += [(c, torch.bfloat16, p.numel())] if c is not None else []
            held += [(ms, torch.float32, blocks), (vs, torch.float32, blocks)] if bits == 8 else []
            if g.dtype not in (torch.float32, torch.bfloat16):
                raise ValueError("gradients are fp32 or bf16")
            for t, dtype, size in held:
                if t is None or t.dtype != dtype or t.numel() != size or not t.is_contiguous() or t.device != params[0].device:
                    raise ValueError("contiguous tensors of the parameter's size on one device: fp32 parameters, bf16 copies")
        held = [(t, True) for t in (*params, *copies, *(t for s in states for t in s[: 4 if bits == 8 else 2]))]
        held = [(t, w) for t, w in held + [(g, False) for g in grads] if t is not None and t.numel()]
        end = end_written = 0  # of the arrays that begin before this one
        for at, size, w in sorted((t.data_ptr(), t.numel() * t.element_size(), w) for t, w in held):
            if at < (end if w else end_written):
                raise ValueError("an array that a step writes overlaps another one")
            end = max(end, at + size)
            end_written = max(end_written, at + size) if w else end_written
        self.params, self.grads, self.copies, self.states = list(params), list(grads), copies, states
        self._steps = steps
        self.config = B.moe_adamw_config(beta1, beta2, eps, bits, B.moe_adamw_device(lr, 1.0, 0, seed))
        self._list = (B.moe_adamw_tensor * max(1, n))(*[
            B.moe_adamw_tensor(*(B._ptr(t) for t in (p, c, g, *s)), p.numel(), d,
                               B.MOE_BF16 if g.dtype == torch.bfloat16 else B.MOE_F32)
            for p, g, c, s, d in zip(params, grads, copies, states, decay)])
        self.scalars = None
        if device_scalars and n:  # a moe_adamw_device: lr and grad_scale as floats, the call's number, the seed; the skipped calls
            words = np.array([lr, 1.0], dtype=np.float32).view(np.int32).tolist() + [steps, int(np.uint32(seed).view(np.int32)), 0]
            self._device = torch.tensor(words, dtype=torch.int32, device=params[0].device)
            self.scalars, self._count, self._skipped = self._device[:4], self._device[2:3], self._device[4:]
            self._scale = self._device.view(torch.float32)[1:2]

    @property
    def steps(self) -> int:
        """Steps taken, without skipped ones.  With device scalars those of the device: waits for it."""
        if self.scalars is None:
            return self._steps
        words = self._device.tolist()
        return words[2] - words[4]

    @steps.setter
    def steps(self, taken: int) -> None:
        self._steps = taken
        if self.scalars is not None:
            self._count.fill_(taken)
            self._skipped.zero_()

    def step(self, lr=None, grad_scale=1.0) -> None:
        """One step with the gradients as they are.  lr: a new rate from now on.  grad_scale: multiplies the gradients; one that is
        not finite skips the step, which then does not count in the averages' corrections.  With device scalars both are set there."""
        if self.scalars is not None:
            if lr is not None or grad_scale != 1.0:
                raise ValueError("lr and grad_scale are in `scalars`")
        import torch
        if self.params and self.params[0].device.index != torch.cuda.current_device():
            with torch.cuda.device(self.params[0].device):
                return self.step(lr, grad_scale)
        if self.scalars is not None:
            self._count += 1
            self._skipped += (self._scale - self._scale).ne(0)  # (0 where it is finite, else NaN)
        now = self.config.now
        held, now.lr = now.lr, now.lr if lr is None else lr
        now.grad_scale = grad_scale
        now.step = self._steps + 1
        try:
            B.moe_adamw_step(self.config, self._list, len(self.params), self.scalars)
        except B.MoeError:
            now.lr = held
            raise
        if self.scalars is None and math.isfinite(now.grad_scale):
            self._steps += 1

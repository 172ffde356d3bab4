"""Driver of the elastic training schedule over the C ABI (Section 3.1 of the paper):
periods that open with a window of all-tensor steps, an importance evaluation at the end of
the window, a re-selection by the host selector, then masked steps.

Control flow and marshalling only: every tensor operation is a library call
(et_forward_stack, et_loss_mse_grad or a given loss, et_backward_elastic with the fused importance / SGD
epilogues or et_update_clipped, et_select_dp); torch is used for device buffers, snapshots (plain copies) and events.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as et


class ElasticLoop:
    """loss: None for the mean-squared error against `target`, else a callable (y, dY, loss_out, stream) that enqueues
    calls which write dL/dy into dY and the loss into loss_out[0]; loss_out is a device float[4], what the token losses
    (et_loss_policy_grad, et_loss_preference_grad) take as loss_dev.  `target` is then not used.  max_norm: clip the selected gradients by their global norm before each update (et_update_clipped, with the
    optimiser the stack is set to); the gradients then take buffers of their own.  x of a stack with an embedding: int32 ids.
    dropout_seed: seed of the stack's dropout layers; step i of the loop, counted over all calls of `run`, drops what {dropout_seed, i} says, in its
    forward and its backward pass, and behind `run` nothing is dropped (evaluation).  None: the stack keeps the seed it has, and every
    step the same elements."""

    def __init__(self, stack, W, b, x, target, lr, period, window, rho, t_dw, t_dy, t_fwd=0.0, Tq=1000,
                 variant=et.ET_COST_STRICT, stream=None, master=False, loss=None, max_norm=None,
                 dropout_seed=None):
        self.stack, self.W, self.b, self.x, self.target = stack, W, b, x, target
        self.lr, self.period, self.window, self.rho = float(lr), int(period), int(window), float(rho)
        self.t_dw, self.t_dy, self.t_fwd, self.Tq, self.variant = t_dw, t_dy, float(t_fwd), int(Tq), variant
        self.stream = stream
        self.L = stack.L
        dev = x.device
        self.y = torch.empty((stack.M, stack.out_width), dtype=W[-1].dtype if W[-1].numel() else x.dtype, device=dev)
        self.dY = torch.empty_like(self.y)
        self.params = [t for pair in zip(W, b) for t in pair]
        # master=True: fp32 master copies of bf16 parameters; updates and snapshots then live in fp32
        self.master = None
        if master:
            self.W32 = [t.float() for t in W]
            self.b32 = [t.float() for t in b]
            et.et_stack_bind_master(stack, self.W32, self.b32)
            self.master = [t for pair in zip(self.W32, self.b32) for t in pair]
        self.snap = [torch.empty_like(p) for p in (self.master or self.params)]
        self.imp = torch.zeros(2 * self.L, dtype=torch.float32, device=dev)
        # layers without tensors (attention core, patch gather) hold empty slots that cannot be selected
        self.all_mask = np.array([1 if p.numel() > 0 else 0 for p in self.params], dtype=np.uint8)
        self.mask = self.all_mask.copy()
        self.loss, self.max_norm = loss, max_norm
        self.dropout_seed, self.dropout_step, self.seeds = dropout_seed, 0, None
        if dropout_seed is not None:
            et.et_stack_set_dropout_seed(stack, None)      # refused here where the stack has no dropout layer
        self.grads = None
        if max_norm is not None:
            self.grads = [torch.empty(p.shape, dtype=torch.float32, device=dev) if m else None
                          for p, m in zip(self.params, self.all_mask)]

    def run(self, steps, elastic=True, time_steps=False):
        """Runs `steps` training steps.  elastic=False trains every tensor at every step (full
        backprop, no evaluation).  Returns losses, the mask used at each step, the importances
        of each evaluation and, with time_steps, the mean device time per step in ms.
        Everything is enqueued on the loop's stream (None: the default stream), behind the current stream's work and before what
        follows there."""
        if not self.x.is_cuda:
            return self._run(steps, elastic, time_steps)
        dev = self.x.device
        st = self.stream
        if st is None:
            st = torch.cuda.default_stream(dev)
        elif isinstance(st, int):
            st = torch.cuda.ExternalStream(st, dev) if st else torch.cuda.default_stream(dev)
        current = torch.cuda.current_stream(dev)
        st.wait_stream(current)
        with torch.cuda.stream(st):
            out = self._run(steps, elastic, time_steps)
        current.wait_stream(st)
        return out

    def _run(self, steps, elastic, time_steps):
        losses = torch.zeros((steps, 4), dtype=torch.float32, device=self.x.device)    # a row a step: the token losses report four numbers
        masks, evaluations, dp_ms = [], [], []
        e0 = e1 = None
        if time_steps:
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
        flags = et.ET_FLAG_FUSE_SGD if self.max_norm is None else 0
        if self.dropout_seed is not None:
            # a row {seed, step} for each step, kept until the next call: work in flight reads it
            seed = self.dropout_seed % 2 ** 64
            rows = [[seed - 2 ** 64 if seed >= 2 ** 63 else seed, self.dropout_step + i] for i in range(steps)]
            self.seeds = torch.tensor(rows, dtype=torch.int64, device=self.x.device)
            self.dropout_step += steps
        for step in range(steps):
            phase = step % self.period
            if self.dropout_seed is not None:
                et.et_stack_set_dropout_seed(self.stack, self.seeds[step])
            if elastic and phase == 0:
                self.mask = self.all_mask.copy()
                for s_, p_ in zip(self.snap, self.master or self.params):
                    s_.copy_(p_)
            et.et_forward_stack(self.stack, self.x, self.y, stream=self.stream)
            if self.loss is None:
                et.et_loss_mse_grad(self.stack, self.y, self.target, self.dY, losses[step], stream=self.stream)
            else:
                self.loss(self.y, self.dY, losses[step], self.stream)
            mask = self.mask.copy()
            masks.append(mask)
            if elastic and phase == self.window - 1:
                et.et_backward_elastic(self.stack, self.dY, self.mask, self.grads, self.snap, self.imp,
                                       flags | et.ET_FLAG_DELTA_IS_SNAPSHOT, self.lr, None, stream=self.stream)
                S = self.imp.cpu().numpy().astype(np.float64)          # synchronises
                S = np.nan_to_num(S, nan=0.0, posinf=0.0, neginf=0.0)  # a diverged run must not stop the selector
                evaluations.append(S)
                import time
                t0 = time.perf_counter()
                self.mask, _, _ = et.et_select_dp(-S * self.all_mask, self.t_dw, self.t_dy, self.t_fwd, self.rho, self.Tq,
                                                  self.variant)
                self.mask = self.mask & self.all_mask
                dp_ms.append(1e3 * (time.perf_counter() - t0))
            else:
                et.et_backward_elastic(self.stack, self.dY, self.mask, self.grads, None, None, flags, self.lr, None,
                                       stream=self.stream)
            if self.max_norm is not None:
                et.et_update_clipped(self.stack, mask, self.grads, self.lr, self.max_norm, stream=self.stream)
        if self.dropout_seed is not None:
            et.et_stack_set_dropout_seed(self.stack, None)
        out = dict(masks=masks, importances=evaluations, dp_ms=dp_ms)
        if time_steps:
            e1.record()
            torch.cuda.synchronize()
            out["ms_per_step"] = e0.elapsed_time(e1) / steps
        out["losses"] = losses[:, 0].cpu().numpy().astype(np.float64)
        return out


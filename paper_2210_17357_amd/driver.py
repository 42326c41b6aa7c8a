"""Periodic run of the algorithm around the per-step compressor (section "Implementation" and
"Parameter ranges" of the paper's experimental setup): gradients are accumulated between runs;
every `period` steps, once `warmup` steps have passed, the error table is built on the
accumulated gradients (no error feedback), the budget is the uniform default's error, the DP picks
the per-layer parameters, and the communication engine uses them until the next run.

This class only sequences calls of the C ABI (accumulate, profile_solve, payload_layout,
compress); it does no arithmetic on gradients itself.

AdamW is the other end of a step: the workers' payloads are turned back and summed, their sum's norm is
taken, and the parameters are updated, again as calls of the C ABI alone.
"""
from __future__ import annotations

import numpy as np

from . import binding as B


class PeriodicRun:
    def __init__(self, handle: "B.Handle", layers, cands, default: int, n_bins: int, period: int,
                 warmup: int = 0, bucket: int = 128):
        if period < 1 or warmup < 0:
            raise ValueError("period >= 1 and warmup >= 0")
        self.h, self.layers, self.cands = handle, layers, cands
        self.default, self.n_bins, self.period, self.warmup, self.bucket = default, n_bins, period, warmup, bucket
        self.choice = np.full(len(layers), default, np.int32)       # uniform default until the first run
        self.offsets = B.payload_layout(layers, cands, self.choice, bucket)
        self.step_count = 0
        self.in_window = 0
        self.acc = None
        self.last = None            # (errors, sizes, e_max, status) of the latest run

    def payload_bytes(self) -> int:
        """Upper bound of the payload buffer over every possible choice."""
        return int(B.sizes(self.layers, self.cands, self.bucket).max(axis=1).sum()) + 16 * (len(self.layers) + 1)

    def step(self, d_grads, d_ef, d_payload, d_q=None, d_q0=None):
        """One training step: accumulate, re-run the algorithm when a window ends, compress.
        Returns (choice, offsets) the payload was written with; compression is off (returns
        None) during the warm-up steps."""
        import torch
        if self.acc is None:
            self.acc = torch.empty_like(d_grads)
        self.h.accumulate(self.acc, d_grads, reset=self.in_window == 0)
        self.in_window += 1
        self.step_count += 1
        if self.step_count >= self.warmup and self.in_window >= self.period:
            st, errors, sizes, e_max, choice, _, _ = self.h.profile_solve(
                self.acc, None, self.layers, self.cands, self.default, self.n_bins, d_q0)
            if st == B.OK:
                self.choice = choice
                self.offsets = B.payload_layout(self.layers, self.cands, choice, self.bucket)
            self.last = (errors, sizes, e_max, st)
            self.in_window = 0
        if self.step_count <= self.warmup:
            return None
        self.h.compress(d_grads, d_ef, self.layers, self.cands, self.choice, d_payload, self.offsets, d_q)
        return self.choice, self.offsets


class AdamW:
    """Parameters' update behind the exchange: moments (fp32, or 8 bits with `coded`), step count and norms of the
    layers of one flat parameter buffer.  `layers` are all the tensors to be stepped, also those that travel
    uncompressed.  With `guard` (always with clipping) a step whose gradients are not finite, or too large for their squares
    or for clipping's factor in fp32, is left out.
    Nothing waits for the GPU in `step`; it may be captured into a HIP graph.  The state is made and read out on torch's
    current stream: a caller whose steps run on another one orders the two."""

    def __init__(self, layers, d_params, settings: "B.AdamW", lr_scale=None, decay_scale=None, coded: bool = False,
                 d_copy=None, guard: bool = False):
        import torch
        self.plan = B.Optim(layers, lr_scale, decay_scale)
        self.settings, self.d_params, self.d_copy, self.coded = settings, d_params, d_copy, coded
        kind = torch.uint8 if coded else torch.float32
        self.d_m, self.d_v = (torch.zeros(d_params.numel(), dtype=kind, device=d_params.device) for _ in range(2))
        self.d_exps = torch.zeros(2 * self.plan.blocks, dtype=torch.uint8, device=d_params.device) if coded else None
        self.d_step = torch.zeros(1, dtype=torch.int64, device=d_params.device)
        self.d_sumsq = None
        if guard or settings.max_norm > 0:
            self.d_sumsq = torch.zeros(len(layers) + 1, dtype=torch.float64, device=d_params.device)

    def step(self, d_grads, d_lr=None, stream=None):
        """Norms, where they are wanted, and the update."""
        if self.d_sumsq is not None:
            self.plan.norms(d_grads, self.d_sumsq, stream=stream)
        if self.coded:
            self.plan.adamw_coded(self.settings, d_grads, self.d_params, self.d_m, self.d_v, self.d_exps, self.d_step,
                                  d_copy=self.d_copy, d_sumsq=self.d_sumsq, d_lr=d_lr, stream=stream)
        else:
            self.plan.adamw(self.settings, d_grads, self.d_params, self.d_m, self.d_v, self.d_step, d_copy=self.d_copy,
                            d_sumsq=self.d_sumsq, d_lr=d_lr, stream=stream)

    def receive(self, handle: "B.Handle", d_payloads, offsets, layers, cands, choice, d_grads, d_lr=None, stream=None):
        """The sum of the workers' payloads into d_grads, then a step on it (settings.grad_scale = 1 / workers makes
        it the mean).  Layers that travel uncompressed hold their summed gradients in d_grads already.  The sum is fp32 whatever
        gradients `step` takes."""
        import torch
        payloads = list(d_payloads)
        if not payloads:
            raise ValueError("no payloads")
        # the receiver's kernels go by the tables alone: what they would write or read past an end is refused in front of them
        if d_grads.dtype is not torch.float32:
            raise ValueError("the payloads' sum is fp32, not %s" % d_grads.dtype)
        need, size = max(self.plan.extent, B.table_extent(layers)), int(offsets[len(layers)])
        if d_grads.numel() < need:
            raise ValueError("the tensor has %d elements, %d are needed" % (d_grads.numel(), need))
        for payload in payloads:
            if payload.numel() * payload.element_size() < size:
                raise ValueError("a payload is shorter than its layout (%d bytes)" % size)
        for w, payload in enumerate(payloads):
            handle.decompress(payload, offsets, layers, cands, choice, d_grads, accumulate=w > 0, stream=stream)
        self.step(d_grads, d_lr=d_lr, stream=stream)

    def moments(self):
        """The moments as new fp32 tensors (elements outside the layers: zero)."""
        if not self.coded:
            return self.d_m.clone(), self.d_v.clone()
        import torch
        out = [torch.zeros(self.d_m.numel(), dtype=torch.float32, device=self.d_m.device) for _ in range(2)]
        self.plan.decode(self.d_m, self.d_v, self.d_exps, *out)
        return tuple(out)

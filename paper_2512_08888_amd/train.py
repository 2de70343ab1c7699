"""The optimiser's side of a training step: the norm and clip factor of all gradients, and AdamW over all parameters,
through the C-ABI library (include/unettrain.h).  This module only owns the device buffers (torch tensors as plain
memory) and the order of the calls; no arithmetic of the method happens here.

    python -m paper_2512_08888_amd.train [--steps 60] [--dtype bf16] [--state mx8] [--graph]

trains a small stack with group norms (paper_2512_08888_amd/unet.py) on one synthetic batch and prints its loss.
"""
from __future__ import annotations

import math

from . import binding as rc


class _Control:
    """The control block as device tensors: `step`, `nonfinite` and `skipped` (int32), `lr`, `coef` and `norm` (fp32)."""

    def __init__(self, device):
        import torch

        self.control = torch.zeros(16, dtype=torch.int32, device=device)
        f = self.control.view(torch.float32)
        self.step_count, self.nonfinite, self.skipped = self.control[0], self.control[4], self.control[5]
        self.lr, self.coef, self.norm = f[1], f[2], f[3]


class GradNorm(_Control):
    """Norm of every gradient (`norms`), of all together (`norm`) and the factor that clips it (`coef`), on the device."""

    def __init__(self, grads):
        import torch

        self.list = rc.TrainList(grads)
        dev = self.list.tensors[1][0].device
        super().__init__(dev)
        rc.train_control_init(self.control)
        self.norms = torch.zeros(self.list.count, device=dev)
        self.ws = torch.empty(self.list.workspace_bytes, dtype=torch.uint8, device=dev)

    def compute(self, max_norm=math.inf):
        rc.train_grad_norm(self.list, max_norm, self.norms, self.control, self.ws)


class AdamW(_Control):
    """AdamW over fp32 parameters whose gradients (fp32 or bf16) lie in fixed buffers.

    state "f32" keeps m and v in 32 bits; "mx8" keeps m and sqrt(v) in e4m3 with a power-of-two scale for each block of
    32 elements (2.06 bytes an element instead of 8).  copies: bf16 tensors that every step refreshes from the
    parameters.  weight_decay: one number, or one for each tensor.  The step number, the learning rate, the clip factor
    and the skip of a step with a non-finite gradient live on the device, so that step() can be recorded into a HIP
    graph: write a schedule's rate with `lr.fill_()`."""

    def __init__(self, params, grads, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, state="f32", copies=None,
                 seed=0):
        import torch

        if state not in rc.STATES:
            raise ValueError(f"state must be one of {sorted(rc.STATES)}")
        self.list = rc.TrainList(grads, params, copies, weight_decay)
        dev = self.list.tensors[1][0].device
        super().__init__(dev)
        self.kind = state
        self.options = rc.TrainAdamW(betas[0], betas[1], eps, rc.STATES[state], seed & 0xFFFFFFFF, 0)
        n = self.list.elements
        # one allocation of zeros: m, v, and in 8 bits their scales
        if state == "mx8":
            self.m, self.v = (torch.zeros(n, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn) for _ in range(2))
            self.m_scale, self.v_scale = (torch.zeros(n // 32, dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu)
                                          for _ in range(2))
        else:
            self.m, self.v = (torch.zeros(n, dtype=torch.float32, device=dev) for _ in range(2))
            self.m_scale = self.v_scale = None
        self.norms = torch.zeros(self.list.count, device=dev)
        self.ws = torch.empty(self.list.workspace_bytes, dtype=torch.uint8, device=dev)
        rc.train_control_init(self.control, 0, lr)

    def clip(self, max_norm):
        """Measures the gradients; the next step, and no other, multiplies them with `coef`, or is skipped where
        `nonfinite` is set.  (A factor written into `coef` by hand serves every step until another is written.)"""
        rc.train_grad_norm(self.list, max_norm, self.norms, self.control, self.ws)

    def step(self):
        rc.train_adamw_step(self.list, self.options, self.m, self.v, self.m_scale, self.v_scale, self.control)

    def state(self):
        """The states' own buffers: m and v (32 bits), or m, sqrt(v) (named v) and their scales (8 bits)."""
        s = {"m": self.m, "v": self.v}
        return s if self.kind == "f32" else {**s, "m_scale": self.m_scale, "v_scale": self.v_scale}

    def load_state(self, step, **state):
        """Continues from a saved step number and state(), taken from a list of the same sizes in the same order.  A state
        that does not fit is refused as a whole."""
        import torch

        mine, step = self.state(), int(step)
        if not 0 <= step < 2**31 - 1:
            raise ValueError(f"load_state: a step number is from 0 to 2^31 - 2, got {step}")
        if set(state) != set(mine):
            raise ValueError(f"load_state: expected {sorted(mine)}, got {sorted(state)}")
        for name, t in state.items():
            if t.dtype != mine[name].dtype or t.numel() != mine[name].numel():
                raise ValueError(f"load_state: {name} must be {mine[name].dtype} with {mine[name].numel()} elements")
        for name, t in state.items():
            mine[name].view(torch.uint8).copy_(t.reshape(-1).view(torch.uint8))
        self.step_count.fill_(step)


def main(argv=None):
    """A stack of two levels learns to tell the quadrants of its images apart (labels by pixel position and brightness):
    group norm, clipping and AdamW as a training program uses them.  Returns the losses."""
    import argparse

    import numpy as np
    import torch

    from . import unet

    ap = argparse.ArgumentParser(description=main.__doc__)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--state", choices=sorted(rc.STATES), default="f32")
    ap.add_argument("--lr", type=float, default=3e-3)
    ap.add_argument("--graph", action="store_true", help="record the step into a HIP graph and replay it")
    a = ap.parse_args(argv)
    cfg = unet.UNetConfig("train", 2, 3, 64, 64, (16, 32, 64), 4, R=4, norm_groups=8, seed=11)
    net = unet.UNet(cfg, unet.make_params(cfg), dtype=a.dtype)
    images, _ = unet.make_batch(cfg)
    labels = (images.mean(1) > 0.5).astype(np.int32) + 2 * (np.arange(cfg.W) >= cfg.W // 2).astype(np.int32)
    net.load_batch(images, labels)
    opt = net.optimizer(lr=a.lr, weight_decay=0.01, state=a.state)
    if a.graph:
        net.capture(opt, max_norm=1.0)
    losses = []
    for k in range(a.steps):
        loss = net.replay() if a.graph else net.train_step(opt, max_norm=1.0)
        if k % 10 == 0 or k == a.steps - 1:
            losses.append(float(loss.cpu()[0]))
            print(f"step {k:4d}  loss {losses[-1]:.4f}  gradient norm {opt.norm.item():.4f}  clipped by {opt.coef.item():.3f}", flush=True)
    torch.cuda.synchronize()
    return losses


if __name__ == "__main__":
    main()

"""The optimiser's side of a training step: the norm and clip factor of all gradients, AdamW over all parameters, and Muon
over matrices (with AdamW for the rest), through the C-ABI library (include/unettrain.h).  This module only owns the
device buffers (torch tensors as plain memory) and the order of the calls; no arithmetic of the methods happens here, but for the
draw of labels (sampled()) that the command's policy loss starts from.

    python -m paper_2512_08888_amd.train [--steps 60] [--dtype bf16] [--state mx8] [--method muon] [--loss policy] [--graph]

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


def _load(optimizer, step, state):
    """Copies a saved state into an optimizer's own buffers, or refuses all of it."""
    import torch

    mine, step = optimizer.state(), int(step)
    if not 0 <= step < 2**31 - 1:
        raise ValueError(f"load_state: a step number is from 0 to 2^31 - 2, got {step}")
    if set(state) != set(mine):
        raise ValueError(f"load_state: expected {sorted(mine)}, got {sorted(state)}")
    for name, t in state.items():
        if t.dtype != mine[name].dtype or t.numel() != mine[name].numel():
            raise ValueError(f"load_state: {name} must be {mine[name].dtype} with {mine[name].numel()} elements")
    for name, t in state.items():
        mine[name].view(torch.uint8).copy_(t.reshape(-1).view(torch.uint8))
    optimizer.step_count.fill_(step)


class AdamW(_Control):
    """AdamW over fp32 parameters whose gradients (fp32 or bf16) lie in fixed buffers.

    state "f32" keeps m and v in 32 bits; "mx8" keeps m and sqrt(v) in e4m3 with a power-of-two scale for each block of
    32 elements (2.06 bytes an element instead of 8).  copies: bf16 tensors that every step refreshes from the
    parameters.  weight_decay: one number, or one for each tensor.  The step number, the learning rate, the clip factor
    and the skip of a step with a non-finite gradient live on the device, so that step() can be recorded into a HIP
    graph: write a schedule's rate with `lr.fill_()`."""

    call = "train_adamw_step"            # what step() issues

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
        _load(self, step, state)


class Muon(_Control):
    """Muon over fp32 matrices [rows, cols], or stacks of them [count, rows, cols], whose gradients (fp32 or bf16) lie in
    fixed buffers: the momentum's direction, orthogonalised, times lr and a scale.  Momentum and parameters are fp32; the products
    that orthogonalise multiply fp16 values and add in fp32 (2e-4 to 8e-4 of the result's norm, up to 6e-3 for momenta of
    few singular values).

    scale "rms": 0.2 sqrt(max(rows, cols)), with which an update's elements are as large as AdamW's, so that one learning
    rate and weight decay serve both; "spectral": sqrt(max(1, rows / cols)); or a number.  rest: an AdamW of the network's other
    tensors, whose step follows in step() under this one's control block (its own lr, clip factor and step number are not
    used).  Step number, learning rate, clip factor and the skip of a step live on the device as AdamW's do."""

    call = "train_muon_step"             # what step() issues (and train_adamw_step for the rest)

    def __init__(self, params, grads, lr=1e-3, momentum=0.95, nesterov=True, weight_decay=0.0, steps=5, scale="rms", eps=1e-12,
                 copies=None, rest=None):
        import torch

        params, grads = list(params), list(grads)
        if scale == "rms":
            factors = [0.2 * math.sqrt(max(p.shape[-2:])) for p in params]
        elif scale == "spectral":
            factors = [math.sqrt(max(1.0, p.shape[-2] / p.shape[-1])) for p in params]
        elif isinstance(scale, (int, float)):
            factors = float(scale)
        else:
            raise ValueError(f"Muon: scale must be 'rms', 'spectral' or a number, got {scale!r}")
        self.matrices = rc.TrainMatrices(grads, params, factors, copies, weight_decay)
        dev = self.matrices.tensors[1][0].device
        super().__init__(dev)
        self.rest = rest
        self.options = rc.TrainMuon(momentum, eps, int(bool(nesterov)), steps, int(rest is not None), 0)
        self.m = torch.zeros(self.matrices.elements, device=dev)
        self.work = torch.empty(self.matrices.workspace_bytes, dtype=torch.uint8, device=dev)
        # the norm is that of all gradients, the rest's among them
        self.list = rc.TrainList(grads + (rest.list.tensors[1] if rest is not None else []))
        self.norms = torch.zeros(self.list.count, device=dev)
        self.ws = torch.empty(self.list.workspace_bytes, dtype=torch.uint8, device=dev)
        rc.train_control_init(self.control, 0, lr)

    def clip(self, max_norm):
        """As AdamW.clip, over the matrices' gradients and the rest's."""
        rc.train_grad_norm(self.list, max_norm, self.norms, self.control, self.ws)

    def step(self):
        rc.train_muon_step(self.matrices, self.options, self.m, self.control, self.work)
        if self.rest is not None:
            r = self.rest
            rc.train_adamw_step(r.list, r.options, r.m, r.v, r.m_scale, r.v_scale, self.control)

    def state(self):
        """The momentum's own buffer; with a rest, its states as rest_m and so on."""
        more = {} if self.rest is None else {"rest_" + k: t for k, t in self.rest.state().items()}
        return {"m": self.m, **more}

    def load_state(self, step, **state):
        """Continues from a saved step number and state().  A state that does not fit is refused as a whole."""
        _load(self, step, state)


def sampled(logits, uniform):
    """A label for each pixel of logits [N, K, H, W], drawn by its class probabilities with uniform numbers [N, H, W] from 0 to below 1.
    No class without a probability is drawn."""
    p = logits.float().softmax(1).cumsum(1)
    at = uniform.unsqueeze(1) * p[:, -1:]
    # the classes before the one in whose share `at` lies (a product that rounds up to the whole lies in the last share that is not empty)
    return ((at >= p) & (p < p[:, -1:])).sum(1).int()


def main(argv=None):
    """A stack of two levels learns to tell the quadrants of its images apart (labels by pixel position and brightness):
    group norm, clipping and AdamW or Muon as a training program uses them.  With --loss policy the stack samples its labels
    itself and is told only which of them were right.  Returns the losses."""
    import argparse

    import numpy as np
    import torch

    from . import unet

    ap = argparse.ArgumentParser(description=main.__doc__)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--state", choices=sorted(rc.STATES), default="f32")
    ap.add_argument("--method", choices=("adamw", "muon"), default="adamw")
    ap.add_argument("--loss", choices=("ce", "policy"), default="ce")
    ap.add_argument("--lr", type=float, default=3e-3)
    ap.add_argument("--graph", action="store_true", help="record the step into a HIP graph and replay it")
    a = ap.parse_args(argv)
    cfg = unet.UNetConfig("train", 2, 3, 64, 64, (16, 32, 64), 4, R=4, norm_groups=8, seed=11)
    net = unet.UNet(cfg, unet.make_params(cfg), dtype=a.dtype)
    images, _ = unet.make_batch(cfg)
    labels = (images.mean(1) > 0.5).astype(np.int32) + 2 * (np.arange(cfg.W) >= cfg.W // 2).astype(np.int32)
    net.load_batch(images, labels)
    opt = net.optimizer(lr=a.lr, weight_decay=0.01, state=a.state, method=a.method)
    right = net.labels.clone()
    draws = torch.Generator(device=net.dev).manual_seed(cfg.seed)

    def roll_out():
        """Samples labels and puts the loss of what they earned in place; the share of right ones."""
        taken = sampled(net.forward_logits(), torch.rand(right.shape, generator=draws, device=net.dev))
        earned = (taken == right).float()
        old = net.label_logp(taken)
        net.load_policy(taken, earned - earned.mean(), logp_old=old, entropy=0.01)
        return earned.mean()

    if a.loss == "policy":
        roll_out()
    if a.graph:
        net.capture(opt, max_norm=1.0)
    losses = []
    for k in range(a.steps):
        earned = roll_out() if a.loss == "policy" else None
        loss = net.replay() if a.graph else net.train_step(opt, max_norm=1.0)
        if k % 10 == 0 or k == a.steps - 1:
            losses.append(float(loss.cpu()[0]))
            more = "" if earned is None else f"  right {earned.item():.3f}"
            print(f"step {k:4d}  loss {losses[-1]:.4f}  gradient norm {opt.norm.item():.4f}  clipped by {opt.coef.item():.3f}{more}", flush=True)
    torch.cuda.synchronize()
    return losses


if __name__ == "__main__":
    main()

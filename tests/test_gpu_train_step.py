"""The stack with group norms and its training step (paper_2512_08888_amd/unet.py): every new call against the 64-bit oracle
on the tensors that the step itself produced, whole steps against the same calls one by one, graph replays, and a run of the
command that trains."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import rotconv_oracle as orc
from oracle import train_oracle as to
from paper_2512_08888_amd import train
from paper_2512_08888_amd import unet as un
from parity_util import RTOL, assert_close, layer_bwd_bf16, layer_fwd_bf16

pytestmark = pytest.mark.gpu
BF_RTOL = 1e-2
CFG = un.UNetConfig("norm", 2, 3, 24, 16, (8, 16), 4, R=4, norm_groups=4, seed=31)
R8 = un.UNetConfig("norm8", 1, 3, 16, 24, (8, 16), 3, R=8, mode="bilinear", norm_groups=8, seed=32)


def make(cfg, dtype="f32"):
    params = un.make_params(cfg)
    rng = np.random.default_rng(cfg.seed)
    for n in params:
        if n.endswith((".gamma", ".beta")):
            params[n] = (params[n] + 0.2 * rng.standard_normal(params[n].shape)).astype(np.float32)
    net = un.UNet(cfg, params, dtype=dtype)
    images, labels = un.make_batch(cfg)
    net.load_batch(images, labels)
    return net, params


def host(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cfg", [CFG, R8], ids=lambda c: c.name)
def test_layers_of_a_step(cfg, dtype):
    net, _ = make(cfg, dtype)
    net.step()
    torch.cuda.synchronize()
    fwd, bwd = (orc.layer_fwd, orc.layer_bwd) if dtype == "f32" else (layer_fwd_bf16, layer_bwd_bf16)
    for i, sp in enumerate(net.specs):
        name, a = sp["name"], net.act[sp["name"]]
        w, ga, be = (host(net.params[name + k]) for k in ("", ".gamma", ".beta"))
        rtol = RTOL if dtype == "f32" else BF_RTOL
        _, pooled, _, _ = fwd(host(a["x"]), w, sp["R"], None, sp["mode"], 1, 1, sp["pool_group"])
        assert_close(host(a["pre"]), pooled, f"{name} pooled", rtol=rtol)
        flat = lambda t: host(t).reshape(t.shape[0], t.shape[1], -1)  # noqa: E731
        y, mean, rstd = to.groupnorm_fwd(flat(a["pre"]), ga, be, cfg.norm_groups, cfg.norm_eps, "relu")
        assert_close(flat(a["y"]), y, f"{name} norm", rtol=rtol)
        assert_close(host(a["mean"]), mean, f"{name} mean")
        assert_close(host(a["rstd"]), rstd, f"{name} rstd")
        f32 = lambda t: flat(t).astype(np.float32)  # noqa: E731
        dx, dga, dbe = to.groupnorm_bwd(f32(a["pre"]), f32(a["g"]), ga.astype(np.float32), be.astype(np.float32),
                                        host(a["mean"]).astype(np.float32), host(a["rstd"]).astype(np.float32),
                                        cfg.norm_groups, "relu")
        assert_close(flat(a["gpre"]), dx, f"{name} norm gradient", rtol=rtol)
        assert_close(host(net.grads[name + ".gamma"]), dga, f"{name} gamma")
        assert_close(host(net.grads[name + ".beta"]), dbe, f"{name} beta")
        _, dw = bwd(host(a["x"]), w, host(a["gpre"]), host(a["idx"]).astype(np.uint8), sp["R"], None, sp["mode"], 1, 1,
                    sp["pool_group"])
        assert_close(host(net.grads[name]), dw, f"{name} dW",
                     rtol=BF_RTOL if net.plans[name].kernel_name(2).endswith("_lut") else RTOL)


@pytest.mark.parametrize("dtype,state", [("f32", "f32"), ("bf16", "f32"), ("bf16", "mx8")])
def test_train_step_updates_every_parameter(dtype, state):
    net, params = make(CFG, dtype)
    opt = net.optimizer(lr=1e-2, weight_decay=0.1, state=state, seed=3)
    net.load_params(params)                     # masters keep what was loaded, not its bf16 rounding
    before = {n: host(t) for n, t in net.masters.items()}
    assert all(np.array_equal(before[n], params[n].astype(np.float64)) for n in params)
    net.train_step(opt, max_norm=0.5)
    torch.cuda.synchronize()
    grads = {n: host(t) for n, t in net.grads.items()}
    _, norm, coef = to.grad_norm(list(grads.values()), 0.5)
    assert abs(opt.norm.item() - norm) <= 1e-6 * norm and abs(opt.coef.item() - coef) <= 1e-6 * coef
    lr = opt.lr.item()
    for n, t in net.masters.items():
        wd = 0.0 if n.endswith((".gamma", ".beta")) else float(np.float32(0.1))
        z = np.zeros_like(grads[n])
        ref, _, _ = to.adamw(before[n], grads[n], z, z, 1, lr, 0.9, 0.999, 1e-8, wd, coef)
        # a first step moves every element by lr but for eps: 2^-20 of that, and the parameter's own rounding
        assert np.all(np.abs(host(t) - ref) <= 2.0 ** -20 * lr + 2.0 ** -22 * np.abs(ref)), n
        if net.params[n] is not t:
            assert torch.equal(net.params[n], t.bfloat16())


@pytest.mark.parametrize("dtype,state", [("f32", "f32"), ("bf16", "mx8")])
def test_training_replays_from_a_graph(dtype, state):
    """Replays of a recorded training step against eager ones: same losses, parameters and states, bit for bit."""
    nets = [make(CFG, dtype)[0] for _ in range(2)]
    opts = [n.optimizer(lr=3e-3, weight_decay=0.01, state=state, seed=8) for n in nets]
    nets[1].capture(opts[1], max_norm=1.0)
    for k in range(4):
        for o in opts:
            o.lr.fill_(3e-3 / (1 + k))
        a = nets[0].train_step(opts[0], max_norm=1.0)
        torch.cuda.synchronize()
        b = nets[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(a, b), k
        assert opts[0].step_count.item() == opts[1].step_count.item() == k + 1
        same = lambda p, q: torch.equal(p.view(torch.uint8), q.view(torch.uint8))  # noqa: E731
        assert all(same(nets[0].params[n], nets[1].params[n]) and same(nets[0].masters[n], nets[1].masters[n]) for n in nets[0].params)
        assert all(same(p, q) for p, q in zip(opts[0].state().values(), opts[1].state().values()))


def test_a_step_without_norms_is_what_it_was():
    """norm_groups = 0 leaves the stack's parameters, calls and results as they are."""
    plain = dataclasses.replace(CFG, norm_groups=0)
    assert not any("." in n for n in un.param_shapes(plain))
    a, b = un.make_params(plain), un.make_params(CFG)
    assert all(np.array_equal(a[n], b[n]) for n in a) and set(b) - set(a) == {n for n in b if "." in n}


@pytest.mark.parametrize("args", [["--dtype", "f32"], ["--dtype", "bf16", "--state", "mx8", "--graph"]])
def test_the_command_learns(args):
    losses = train.main(["--steps", "41", *args])
    assert losses[-1] < 0.6 * losses[0]


@pytest.mark.parametrize("bad", [None, float("nan"), float("inf")])
def test_a_step_without_clipping_behind_a_clipped_or_skipped_one(bad):
    """train_step(opt) takes the gradients as they are, whatever the step before did to its own."""
    nets = [make(CFG)[0] for _ in range(2)]
    a, b = (n.optimizer(lr=1e-2) for n in nets)
    if bad is None:
        nets[0].train_step(a, max_norm=1e-3)
        b.coef.copy_(a.coef)
        nets[1].train_step(b)
        b.coef.fill_(1.0)
    else:
        keep = nets[0].images.clone()
        nets[0].images[0, 0, 3, 3] = bad
        nets[0].train_step(a, max_norm=1.0)
        assert a.skipped.item() == 1 and a.step_count.item() == 0
        nets[0].images.copy_(keep)
    for _ in range(2):
        nets[0].train_step(a)
        nets[1].train_step(b)
    torch.cuda.synchronize()
    assert all(torch.equal(nets[0].params[n], nets[1].params[n]) for n in nets[0].params)
    assert all(bool(torch.isfinite(t).all()) for t in nets[0].params.values())


STD = un.UNetConfig("norm_std", 2, 3, 16, 24, (8, 16), 3, R=8, mode="bilinear", block="rot_std", norm_groups=4, seed=33)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layers_of_a_step_with_standard_convolutions(dtype):
    """Norms behind rotation convolutions and behind the standard convolutions of the other kind of block."""
    test_layers_of_a_step(STD, dtype)


def test_an_optimizer_that_only_the_graph_needs():
    """Replays of a step recorded with an optimizer that nobody else holds, with memory allocated and freed in between."""
    import gc

    nets = [make(CFG)[0] for _ in range(2)]
    opt = nets[0].optimizer(lr=3e-3)
    nets[1].capture(nets[1].optimizer(lr=3e-3), max_norm=1.0)
    gc.collect()
    for k in range(3):
        junk = [torch.full((n,), float("nan"), device="cuda") for n in (16, 4096, 100_000, 1 << 22)]
        a = nets[0].train_step(opt, max_norm=1.0)
        torch.cuda.synchronize()
        b = nets[1].replay()
        torch.cuda.synchronize()
        del junk
        assert torch.equal(a, b) and all(torch.equal(nets[0].params[n], nets[1].params[n]) for n in nets[0].params), k

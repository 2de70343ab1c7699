"""The stack tuned by rewards (paper_2512_08888_amd/unet.py): log-probabilities of sampled labels, the policy loss in the cross-
entropy's place, clipping, Muon over the filters and AdamW over the rest, one behind the other as a training program uses
them; also recorded in a HIP graph, and by the command that trains."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import train_oracle as to
from paper_2512_08888_amd import train
from paper_2512_08888_amd import unet as un

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
CFG = un.UNetConfig("policy", 2, 3, 16, 16, (8, 16), 4, R=4, norm_groups=4, seed=41)
STEER = un.UNetConfig("policy2", 1, 3, 16, 16, (8, 16), 3, R=8, mode="steerable", norm_groups=8, seed=42)


def make(cfg, dtype="f32"):
    net = un.UNet(cfg, un.make_params(cfg), dtype=dtype)
    net.load_batch(*un.make_batch(cfg))
    return net


def host(t):
    return t.detach().double().cpu().numpy()


def roll(net, seed, per="pixel", ref=True, weight=True):
    """Sampled labels with what a roll-out keeps of them; every 17th pixel without a label."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    taken = train.sampled(net.forward_logits(), rand(net.labels.shape))
    taken.view(-1)[::17] = -1
    old = net.label_logp(taken)
    kw = dict(labels=taken, advantage=rand(net.labels.shape) - 0.5 if per == "pixel" else rand(net.cfg.N) - 0.5, logp_old=old - 0.3 + 0.6 * rand(old.shape))
    if ref:
        kw["logp_ref"] = old + 0.2 * rand(old.shape)
    if weight:
        kw["weight"] = (rand(old.shape) > 0.2).float() / old.numel()
    return kw


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cfg,per", [(CFG, "pixel"), (CFG, "image"), (STEER, "pixel")])
def test_policy_step_and_gradient(cfg, per, dtype):
    net = make(cfg, dtype)
    kw = roll(net, 3, per)
    rows = lambda t: host(t).reshape(t.shape[0], t.shape[1], -1).transpose(0, 2, 1).reshape(-1, t.shape[1])  # noqa: E731
    z = rows(net.act["head"]["y"])
    labels = kw["labels"].cpu().numpy().reshape(-1)
    r = to.logp_rows(z, labels)
    # a handful of classes: logarithm, maximum and difference are rounded a few times each
    assert np.abs(host(net.label_logp(kw["labels"])).reshape(-1) - r["logp"]).max() <= 64 * U * (1 + np.abs(z).max())
    net.load_policy(**kw, kl=0.1, entropy=0.02)
    net.step()
    A = host(kw["advantage"]).reshape(-1)
    A = np.repeat(A, labels.size // A.size) if A.size != labels.size else A
    low, high = float(np.float32(1) - np.float32(0.2)), float(np.float32(1) + np.float32(0.2))
    f = lambda k: host(kw[k]).reshape(-1)  # noqa: E731
    out, dz, _, live, G, ratio, r = to.policy(z, labels, A, f("logp_old"), f("logp_ref"), f("weight"), low, high, float(np.float32(0.1)),
                                              float(np.float32(0.02)))
    edge = np.minimum(np.abs(ratio - low), np.abs(ratio - high)) < 1e-4             # pixels that 32 bits may put on either side
    err = 256 * U * (1 + np.abs(z).max()) * f("weight") * (1 + np.abs(A) * ratio)
    got = rows(net.act["head"]["g"])
    bar = err[:, None] + (2.0 ** -8 * np.abs(dz) if dtype == "bf16" else 0)
    assert (np.abs(got - dz) <= bar)[~edge].all() and (got[~live] == 0).all()
    assert np.abs(host(net.parts)[:3] - out[:3]).max() <= err.sum() + (f("weight") * edge).sum() + 4 * U
    net.load_batch(*un.make_batch(cfg))                                              # back to the cross-entropy
    assert net.policy is None
    net.step()
    assert torch.isfinite(net.loss).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cfg", [CFG, STEER], ids=lambda c: c.name)
def test_muon_step_of_the_network(cfg, dtype):
    net = make(cfg, dtype)
    opt = net.optimizer(method="muon", lr=0.02, weight_decay=0.1, momentum=0.9, nesterov=False, steps=4, scale=1.0, betas=(0.8, 0.9))
    filters = [n for n in net.params if not n.endswith((".gamma", ".beta")) and n not in ("head", "enc0a")]
    others = [n for n in net.params if n not in filters]
    lr, wd = float(np.float32(0.02)), float(np.float32(0.1))
    before = {n: host(net.masters[n]) for n in net.params}
    net.load_policy(**roll(net, 5))
    net.train_step(opt, max_norm=0.5)
    norm = np.sqrt(sum((host(net.grads[n]) ** 2).sum() for n in net.params))
    assert abs(opt.norm.item() - norm) <= 1e-6 * norm
    coef = float(opt.coef.item())
    assert opt.step_count.item() == 1
    for n in filters:
        shape = before[n].shape
        mats = (lambda a: a.reshape(shape[0], shape[1], -1)) if len(shape) == 5 else (lambda a: a.reshape(1, shape[0], -1))
        for p0, g, p1 in zip(mats(before[n]), mats(host(net.grads[n])), mats(host(net.masters[n]))):
            want, _, o = to.muon(p0, g, np.zeros_like(g), lr, 0.9, False, wd, 1.0, coef, 4)
            rough = np.linalg.norm(to.newton_schulz_fp16(coef * g, 4) - o)
            bar = lr * (3 * rough + 5.0 ** 4 * 2.0 ** -21 * np.linalg.norm(o)) + 4 * U * np.linalg.norm(p0)
            assert np.linalg.norm(p1 - want) <= bar, n
    for n in others:
        decay = 0.0 if n.endswith((".gamma", ".beta")) else wd
        p, g = before[n], host(net.grads[n])
        want, _, _ = to.adamw(p, g, 0 * p, 0 * p, 1, lr, 0.8, 0.9, float(np.float32(1e-8)), decay, coef)
        # the first step's quotient is 1 beside eps: rounded a few times, and beta in fp32
        assert (np.abs(host(net.masters[n]) - want) <= 64 * U * (np.abs(p) + lr)).all(), n
    if dtype == "bf16":
        for n in net.params:
            assert n.endswith((".gamma", ".beta")) or torch.equal(net.params[n], net.masters[n].to(torch.bfloat16))


def test_recorded_steps_are_the_eager_ones():
    nets = [make(CFG), make(CFG)]
    opts = [n.optimizer(method="muon", lr=0.01, weight_decay=0.05) for n in nets]
    kw = roll(nets[0], 7)
    for n in nets:
        n.load_policy(**kw, kl=0.1)
    nets[0].capture(opts[0], max_norm=0.3)
    nets[1].step()
    for k in range(4):
        kw = roll(nets[1], 8 + k)
        for n, o in zip(nets, opts):
            n.load_policy(**kw, kl=0.1)
            o.lr.fill_(0.01 / (k + 1))
        nets[0].replay()
        torch.cuda.synchronize()
        nets[1].train_step(opts[1], max_norm=0.3)
        torch.cuda.synchronize()
        assert torch.equal(nets[0].parts, nets[1].parts)
        for n in nets[0].params:
            assert torch.equal(nets[0].params[n], nets[1].params[n]), (k, n)
    assert opts[0].step_count.item() == opts[1].step_count.item() == 4


def test_a_step_with_a_bad_gradient_changes_nothing():
    net = make(CFG)
    opt = net.optimizer(method="muon", lr=0.01)
    kw = roll(net, 9, weight=False)
    kw["advantage"][0, 0, 1] = float("nan")
    net.load_policy(**kw)
    before = {n: t.clone() for n, t in net.params.items()}
    net.train_step(opt, max_norm=1.0)
    assert all(torch.equal(before[n], t) for n, t in net.params.items())
    assert opt.skipped.item() == 1 and opt.step_count.item() == 0


def test_refusals():
    net = make(dataclasses.replace(CFG, N=1))
    kw = roll(net, 11)
    with pytest.raises(ValueError):
        net.load_policy(kw["labels"], kw["advantage"][0, :3])
    with pytest.raises(ValueError):
        net.load_policy(kw["labels"][:, :2], kw["advantage"])
    with pytest.raises(ValueError):
        net.optimizer(method="other")


@pytest.mark.parametrize("args", [["--method", "muon"], ["--loss", "policy"], ["--method", "muon", "--loss", "policy", "--graph", "--dtype", "bf16"]])
def test_command(args):
    losses = train.main(["--steps", "3", *args])
    assert len(losses) == 2 and np.isfinite(losses).all()

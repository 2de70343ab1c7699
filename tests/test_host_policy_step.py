"""CPU checks of the loss in place and the recorded one (paper_2512_08888_amd/unet.py), by a network without kernels whose recording is
replaced, and of the draw of labels (paper_2512_08888_amd/train.py)."""
import contextlib
import types

import numpy as np
import pytest
import torch

from paper_2512_08888_amd import train, unet

SHAPE, PIXELS = (2, 4, 4), 32


def network():
    net = unet.UNet.__new__(unet.UNet)
    graph = type("Graph", (), {"replays": 0, "replay": lambda self: setattr(self, "replays", self.replays + 1)})
    cuda = types.SimpleNamespace(synchronize=lambda: None, CUDAGraph=graph, graph=lambda g: contextlib.nullcontext())
    names = ("is_tensor", "from_numpy", "empty", "float32", "int32")
    net.torch = types.SimpleNamespace(cuda=cuda, **{n: getattr(torch, n) for n in names})
    net.cfg, net.dev, net.trace, net._policy = types.SimpleNamespace(N=2, H=4, W=4), "cpu", None, {}
    net.images, net.labels, net.loss = torch.zeros(2, 3, 4, 4), torch.full(SHAPE, 3, dtype=torch.int32), torch.zeros(1)
    net.step, net.train_step = lambda: None, lambda optimizer, max_norm: None
    return net


def given(**more):
    return dict(dict(labels=np.ones(SHAPE, np.int32), advantage=np.ones(SHAPE, np.float32), logp_old=torch.zeros(SHAPE)), **more)


def batch(net):
    net.load_batch(np.zeros((2, 3, 4, 4)), np.zeros(SHAPE, np.int32))


def test_a_recorded_cross_entropy_is_not_replayed_for_the_policy_loss():
    net = network()
    batch(net)
    graph = net.capture()
    net.replay()
    net.load_policy(**given())
    with pytest.raises(RuntimeError, match="another loss"):
        net.replay()
    assert graph.replays == 1
    batch(net)
    net.replay()
    assert graph.replays == 2
    net.load_policy(**given())
    net.capture().replay()
    net.replay()


OTHERS = [dict(advantage=np.ones(2, np.float32)), dict(logp_old=None), dict(logp_ref=torch.zeros(SHAPE)), dict(weight=np.ones(SHAPE)),
          dict(clip=(0.2, 0.3)), dict(clip=(0.1, 0.2)), dict(kl=0.1), dict(entropy=0.1)]


@pytest.mark.parametrize("other", OTHERS, ids=lambda o: next(iter(o)))
def test_a_recorded_policy_loss_is_not_replayed_for_another(other):
    net = network()
    net.load_policy(**given())
    graph = net.capture()
    net.load_policy(**given(advantage=np.zeros(SHAPE), logp_old=np.ones(SHAPE), clip=[np.float32(0.2), 0.2], kl=0, entropy=0))      # other values alone
    net.replay()
    for put in (lambda: net.load_policy(**given(**other)), lambda: batch(net)):
        put()
        with pytest.raises(RuntimeError, match="another loss"):
            net.replay()
    net.load_policy(**given())
    net.replay()
    assert graph.replays == 2


def test_a_recording_that_fails_leaves_the_loss_of_the_one_before():
    net = network()
    net.load_policy(**given())
    graph = net.capture()
    batch(net)

    def broken():
        raise RuntimeError("not recorded")

    net.step = broken
    with pytest.raises(RuntimeError, match="not recorded"):
        net.capture()
    with pytest.raises(RuntimeError, match="another loss"):
        net.replay()
    net.load_policy(**given())
    net.replay()
    assert graph.replays == 1


class Broken:
    """Neither a tensor nor an array of numbers."""


REFUSED = [dict(labels=np.ones(31, np.int32)), dict(labels=None), dict(advantage=np.zeros(5)), dict(advantage=None), dict(logp_old=torch.zeros(1)),
           dict(logp_ref=np.zeros((2, 4, 5))), dict(weight=torch.zeros(33)), dict(weight=Broken()), dict(clip=0.2), dict(clip=(0.2,)), dict(clip=("low", 0.2)), dict(kl=None)]


@pytest.mark.parametrize("bad", REFUSED, ids=lambda o: next(iter(o)))
def test_a_refused_call_leaves_the_loss_in_place(bad):
    """Every earlier argument differs from what is in place, and none of it may arrive."""
    net = network()
    net.load_policy(**given(logp_ref=torch.full(SHAPE, -1.0), weight=np.ones(SHAPE)), kl=0.1)
    graph, policy, buffers = net.capture(), net.policy, {k: v.clone() for k, v in net._policy.items()}
    labels = net.labels.clone()
    other = dict(labels=np.zeros(SHAPE, np.int32), advantage=np.full(SHAPE, 5.0), logp_old=torch.full(SHAPE, 6.0), logp_ref=torch.full(SHAPE, 7.0),
                 weight=np.full(SHAPE, 8.0), kl=0.1)
    with pytest.raises((ValueError, TypeError)):
        net.load_policy(**{**other, **bad})
    assert net.policy is policy and torch.equal(net.labels, labels)
    assert all(torch.equal(net._policy[k], v) for k, v in buffers.items())
    net.replay()
    net.load_policy(**other)
    net.replay()
    assert graph.replays == 2 and (net.labels == 0).all() and (net.policy["advantage"] == 5).all() and (net.policy["weight"] == 8).all()


def test_sampled_labels_have_a_probability():
    """Classes of -infinity at the start, in the middle and at the end; the smallest and the largest uniform numbers."""
    inf = float("inf")
    logits = torch.tensor([[-inf, 0.0, 1.0, 2.0], [0.0, -inf, -inf, 1.0], [1.0, 2.0, 0.5, -inf], [-inf, -200.0, 0.0, -inf], [-inf, -inf, 3.0, -inf]])
    uniform = torch.tensor([0.0, 2.0 ** -24, 0.2, 0.25, 0.5, 0.75, 1 - 2.0 ** -24])
    maps = logits.t().reshape(1, 4, 5, 1).expand(1, 4, 5, 7).contiguous()
    got = train.sampled(maps, uniform.expand(1, 5, 7).contiguous())
    assert got.shape == (1, 5, 7) and got.dtype == torch.int32
    p = logits.softmax(1)
    assert (p.gather(1, got[0].long()) > 0).all()
    # shares in 64 bits, but for numbers within rounding of a border
    ends = logits.double().softmax(1).cumsum(1)
    for r in range(5):
        for k, u in enumerate(uniform.double()):
            if (ends[r] - u).abs().min() > 1e-6:
                assert got[0, r, k].item() == (u > ends[r]).sum().item()

"""CPU checks of the label log-probabilities, the policy loss and Muon: refusals before a device is touched, the oracle's gradients
against differences, the oracle's roundings."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import train_oracle as to
from paper_2512_08888_amd import binding as rc
from paper_2512_08888_amd import train

NAN, INF = float("nan"), float("inf")
WS = 1 << 20


def fwd(z=16, labels=16, logp=16, ent=None, stat=None, N=2, K=4, P=4, layout=0, ws=WS, size=WS, bf16=False):
    f = rc.lib().train_logp_fwd_bf16 if bf16 else rc.lib().train_logp_fwd
    return f(z, labels, logp, ent, stat, N, K, P, layout, ws, size, None)


def bwd(z=16, labels=16, stat=16, ent=None, dlogp=16, dent=None, dz=16, N=2, K=4, P=4, layout=0, bf16=False):
    f = rc.lib().train_logp_bwd_bf16 if bf16 else rc.lib().train_logp_bwd
    return f(z, labels, stat, ent, dlogp, dent, dz, N, K, P, layout, None)


def loss(z=16, labels=16, adv=16, old=None, ref=None, w=None, out=16, dz=None, logp=None, N=2, K=4, P=4, layout=0, ws=WS, size=WS, bf16=False,
         options=True, **kw):
    o = rc.TrainPolicy(0.2, 0.2, 0.0, 0.0, 0, 0)
    for k, v in kw.items():
        setattr(o, k, v)
    f = rc.lib().train_policy_loss_bf16 if bf16 else rc.lib().train_policy_loss
    return f(z, labels, adv, old, ref, w, out, dz, logp, N, K, P, layout, ctypes.byref(o) if options else None, ws, size, None)


SHAPES = [dict(N=0), dict(N=-1), dict(K=0), dict(K=-3), dict(P=0), dict(K=(1 << 24) + 1), dict(P=1 << 31), dict(N=1 << 16, P=1 << 15), dict(P=1 << 63)]


@pytest.mark.parametrize("bf16", (False, True))
def test_outputs_in_each_others_place_are_refused(bf16):
    """2 images of 4 classes, 4 pixels: 32 logits, 8 rows (nothing is read or written: a call is refused, or there is no device)."""
    z, labels, adv, logp, stat, ent, out, dz = (1 << 20 | k << 10 for k in range(8))
    ws, size = 1 << 30, 1 << 22
    ok = lambda code: code != rc.ERR_UNSUPPORTED
    if not torch.cuda.is_available():                      # (addresses of nothing: no launch may get them)
        assert ok(fwd(z, labels, logp, ent, stat, ws=ws, size=size, bf16=bf16))
        assert ok(bwd(z, labels, stat, ent, adv, adv, dz, bf16=bf16)) and ok(bwd(z, labels, stat, None, adv, None, z, bf16=bf16))
        assert ok(loss(z, labels, adv, logp, logp, adv, out, dz, ent, ws=ws, size=size, bf16=bf16))
        assert ok(loss(z, labels, adv, out=out, dz=z, ws=ws, size=size, bf16=bf16))
    end = 32 * (2 if bf16 else 4)
    bad = [lambda: fwd(z, labels, z + end - 4, ws=ws, size=size, bf16=bf16), lambda: fwd(z, labels, logp, logp + 28, ws=ws, size=size, bf16=bf16),
           lambda: fwd(z, labels, logp, None, labels - 60, ws=ws, size=size, bf16=bf16), lambda: fwd(z, labels, ws, ws=ws, size=size, bf16=bf16),
           lambda: bwd(z, labels, stat, None, adv, None, z + 4, bf16=bf16), lambda: bwd(z, labels, stat, None, adv, None, labels, bf16=bf16),
           lambda: bwd(z, labels, stat, ent, adv, adv, ent, bf16=bf16),
           lambda: loss(z, labels, adv, logp, out=out, logp=logp, ws=ws, size=size, bf16=bf16),
           lambda: loss(z, labels, adv, out=out, dz=z - 4, ws=ws, size=size, bf16=bf16),
           lambda: loss(z, labels, adv, out=z, dz=z, ws=ws, size=size, bf16=bf16),
           lambda: loss(z, labels, adv, out=out, dz=dz, logp=out - 28, ws=ws, size=size, bf16=bf16)]
    assert [call() for call in bad] == [rc.ERR_UNSUPPORTED] * len(bad)


@pytest.mark.parametrize("bf16", [False, True])
def test_loss_refusals(bf16):
    for f in (fwd, bwd, loss):
        assert f(z=None, bf16=bf16) == rc.ERR_NULL and f(labels=None, bf16=bf16) == rc.ERR_NULL
        for kw in SHAPES:
            assert f(bf16=bf16, **kw) == rc.ERR_SHAPE, kw
        for kw in (dict(layout=2), dict(layout=-1), dict(z=17), dict(labels=18)):
            assert f(bf16=bf16, **kw) == rc.ERR_UNSUPPORTED, kw
    for f in (fwd, loss):
        for kw in (dict(ws=None), dict(size=8), dict(ws=WS + 4)):
            assert f(bf16=bf16, **kw) == rc.ERR_WORKSPACE, kw
    assert fwd(logp=None, bf16=bf16) == rc.ERR_NULL and fwd(logp=18, bf16=bf16) == rc.ERR_UNSUPPORTED
    for name in ("stat", "dlogp", "dz"):
        assert bwd(bf16=bf16, **{name: None}) == rc.ERR_NULL, name
    assert bwd(dent=16, bf16=bf16) == rc.ERR_NULL                              # the entropy's gradient without the entropy
    for name in ("adv", "out"):
        assert loss(bf16=bf16, **{name: None}) == rc.ERR_NULL, name
    assert loss(options=False, bf16=bf16) == rc.ERR_NULL and loss(kl=0.1, bf16=bf16) == rc.ERR_NULL
    for kw in (dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=NAN), dict(clip_high=-0.1), dict(clip_high=INF), dict(kl=-1.0, ref=16),
               dict(kl=NAN, ref=16), dict(entropy=-1.0), dict(entropy=INF), dict(per_image=2), dict(reserved=1), dict(out=18), dict(w=18)):
        assert loss(bf16=bf16, **kw) == rc.ERR_UNSUPPORTED, kw


def test_loss_workspace():
    assert rc.train_logp_workspace_bytes(4, 6, 512 * 512) > 0
    for N, K, P in ((0, 4, 4), (1, 0, 4), (1, 4, 0), (1, 1 << 25, 1)):
        assert rc.train_logp_workspace_bytes(N, K, P) == 0
    with pytest.raises(rc.RotconvError):
        rc.train_logp_workspace_bytes(2**32 + 2, 4, 4)


def matrices(rows, grad_dtype=0, count=None):
    arr = (rc.TrainMatrix * max(1, len(rows)))(*[rc.TrainMatrix(*r) for r in rows])
    h = ctypes.c_void_p()
    return rc.lib().train_matrices_create(arr, len(rows) if count is None else count, grad_dtype, ctypes.byref(h))


def test_matrices_refusals():
    L = rc.lib()
    good = (16, 32, None, 1, 5, 7, 0.0, 1.0, 0)
    assert L.train_matrices_create(None, 1, 0, ctypes.byref(ctypes.c_void_p())) == rc.ERR_NULL
    assert L.train_matrices_create((rc.TrainMatrix * 1)(rc.TrainMatrix(*good)), 1, 0, None) == rc.ERR_NULL
    assert matrices([good], count=0) == rc.ERR_SHAPE and matrices([good], count=-1) == rc.ERR_SHAPE
    assert matrices([good], grad_dtype=2) == rc.ERR_UNSUPPORTED
    for k in (0, 1):
        assert matrices([good[:k] + (None,) + good[k + 1:]]) == rc.ERR_NULL
    for extents in ((0, 5, 7), (1, 0, 7), (1, 5, 0), (-1, 5, 7), (1, -5, 7), (1, 32769, 32769), (1, 1, (1 << 24) + 1), (1 << 20, 1 << 15, 1 << 15),
                    (65536, 1, 1), (60000, 32768, 32768)):
        assert matrices([(16, 32, None, *extents, 0.0, 1.0, 0)]) == rc.ERR_SHAPE, extents
    for bad in ((16, 32, None, 1, 5, 7, -0.1, 1.0, 0), (16, 32, None, 1, 5, 7, NAN, 1.0, 0), (16, 32, None, 1, 5, 7, 0.0, INF, 0),
                (16, 32, None, 1, 5, 7, 0.0, NAN, 0), (16, 32, None, 1, 5, 7, 0.0, 1.0, 1), (18, 32, None, 1, 5, 7, 0.0, 1.0, 0),
                (16, 34, None, 1, 5, 7, 0.0, 1.0, 0), (16, 32, 33, 1, 5, 7, 0.0, 1.0, 0)):
        assert matrices([bad]) == rc.ERR_UNSUPPORTED, bad
    # what a step writes, named twice: the same matrix, one inside a stack, a copy over another's parameters
    for pair in ((good, good), ((4096, 32, None, 3, 4, 4, 0.0, 1.0, 0), (4096 + 64, 32, None, 1, 4, 4, 0.0, 1.0, 0)),
                 ((4096, 32, None, 1, 4, 4, 0.0, 1.0, 0), (8192, 32, 4096 + 32, 1, 4, 4, 0.0, 1.0, 0))):
        assert matrices(list(pair)) == rc.ERR_UNSUPPORTED, pair
    assert L.train_matrices_destroy(None) == rc.OK
    assert L.train_matrices_elements(None) == 0 and L.train_matrices_workspace_bytes(None) == 0
    o = rc.TrainMuon(0.9, 1e-12, 1, 5, 0, 0)
    assert L.train_muon_step(None, ctypes.byref(o), 64, 64, 64, 64, None) == rc.ERR_NULL


def test_binding_refusals():
    import torch

    z, one = torch.zeros(2, 6, 3, 5), torch.zeros(30)
    labels = torch.zeros(30, dtype=torch.int32)
    for call in (lambda: rc.train_logp_fwd(z, labels, one), lambda: rc.train_logp_bwd(z, labels, one, one, torch.zeros_like(z)),
                 lambda: rc.train_policy_loss(z, labels, one, one[:4]), lambda: rc.train_logp_fwd(z.transpose(2, 3), labels, one),
                 lambda: rc.TrainMatrices([torch.zeros(3, 4)], [torch.zeros(3, 4)], 1.0),
                 lambda: rc.TrainMatrices([torch.zeros(3)], [torch.zeros(3)], 1.0),
                 lambda: rc.TrainMatrices([torch.zeros(3, 4)], [torch.zeros(3, 4)], [1.0, 2.0]),
                 lambda: train.Muon([torch.zeros(3, 4)], [torch.zeros(3, 4)], scale="other")):
        with pytest.raises(ValueError):
            call()
    for g, p, c in ((torch.zeros(3, 4), torch.zeros(4, 3), None), (torch.zeros(3, 4), torch.zeros(3, 4).double(), None),
                    (torch.zeros(3, 4), torch.zeros(3, 4), torch.zeros(3, 4)), (torch.zeros(3, 4).half(), torch.zeros(3, 4), None)):
        with pytest.raises(TypeError):
            rc.TrainMatrices([g], [p], 1.0, None if c is None else [c])


class Elsewhere:
    """What the bindings ask of a tensor, for one on a device that is not the current one."""

    def __init__(self, t, device):
        self.t, self.device_number, self.is_cuda = t, device, True
        self.shape, self.dtype = t.shape, t.dtype

    def get_device(self):
        return self.device_number

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_binding_refuses_other_devices(monkeypatch):
    import torch

    monkeypatch.setattr(rc, "_device", lambda: 0)
    z, labels, one = torch.zeros(4, 6), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    here = lambda t: Elsewhere(t, 0)  # noqa: E731
    with pytest.raises(ValueError, match="current device"):
        rc.train_logp_fwd(Elsewhere(z, 1), Elsewhere(labels, 1), Elsewhere(one, 1))
    with pytest.raises(ValueError, match="labels"):
        rc.train_logp_fwd(here(z), Elsewhere(labels, 1), here(one), ws=here(torch.zeros(1 << 19, dtype=torch.uint8)))
    with pytest.raises(ValueError, match="logp"):
        rc.train_logp_fwd(here(z), here(labels), Elsewhere(one, 1), ws=here(torch.zeros(1 << 19, dtype=torch.uint8)))
    with pytest.raises(ValueError, match="dlogits"):
        rc.train_policy_loss(here(z), here(labels), here(one), here(one), Elsewhere(z, 1))
    with pytest.raises(ValueError, match="workspace"):
        rc.train_policy_loss(here(z), here(labels), here(one), here(one), ws=Elsewhere(torch.zeros(1 << 19, dtype=torch.uint8), 1))


def differences(f, x, h=1e-6):
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        y = x.copy()
        y[i] += h
        hi = f(y)
        y[i] -= 2 * h
        out[i] = (hi - f(y)) / (2 * h)
    return out


@pytest.mark.parametrize("kl,entropy", [(0.0, 0.0), (0.3, 0.2)])
def test_oracle_policy_gradient_against_differences(kl, entropy):
    rng = np.random.default_rng(1)
    z = rng.standard_normal((7, 5))
    labels = np.array([0, 4, 2, -1, 3, 5, 1])
    A, w = rng.standard_normal(7), np.abs(rng.standard_normal(7))
    w[2] = 0
    lp = to.logp_rows(z, labels)["logp"]
    old, ref = lp + 0.3 * rng.standard_normal(7), lp + 0.3 * rng.standard_normal(7)
    args = (labels, A, old, ref, w, 0.8, 1.25, kl, entropy)
    got = to.policy(z, *args)[1]
    # a difference's error: about 1e-16 / 1e-6, and h^2 times a third derivative of order one
    assert np.abs(got - differences(lambda x: to.policy(x, *args)[0][0], z)).max() <= 1e-8


def test_oracle_logp_gradient_against_differences():
    rng = np.random.default_rng(2)
    z, labels = rng.standard_normal((4, 6)), np.array([5, 0, 2, 2])
    c1, c2 = rng.standard_normal(4), rng.standard_normal(4)

    def f(x):
        r = to.logp_rows(x, labels)
        return (c1 * r["logp"] + c2 * r["entropy"]).sum()

    got = to.logp_gradient(to.logp_rows(z, labels), labels, c1, c2)
    assert np.abs(got - differences(f, z)).max() <= 1e-8


@pytest.mark.parametrize("rows,cols", [(20, 60), (60, 20), (30, 30), (1, 9), (9, 1)])
def test_oracle_orthogonalises(rows, cols):
    u = np.random.default_rng(3).standard_normal((rows, cols))
    o = to.newton_schulz(u)
    left, s, right = np.linalg.svd(u, full_matrices=False)
    x = s / np.sqrt((s ** 2).sum())
    for _ in range(5):
        x = to.NS[0] * x + to.NS[1] * x ** 3 + to.NS[2] * x ** 5
    assert np.abs(o - (left * x) @ right).max() <= 1e-10              # the polynomial of the singular values
    # three parts in a thousand at most of fp16's roundings, as the kernels' notes say
    assert np.linalg.norm(to.newton_schulz_fp16(u) - o) <= 3e-3 * np.linalg.norm(o)


def test_the_polynomial_stays_where_fp16_holds_it():
    x = np.linspace(0, 1.21, 200001)
    p = to.NS[0] * x + to.NS[1] * x ** 3 + to.NS[2] * x ** 5
    assert p.min() >= 0 and p.max() <= 1.21
    s = x ** 2
    b = to.NS[1] * s + to.NS[2] * s * s
    assert b.min() >= -2.82 and b.max() <= 0
    assert 1.21 * 2 ** 15 < 65504 and 1.21 ** 2 * 2 ** 15 < 65504 and 2.82 * 2 ** 14 < 65504

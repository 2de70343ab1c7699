"""CPU checks of the training operators: the library exports what include/unettrain.h declares and refuses bad arguments
before it touches a device; the 64-bit oracle's gradients agree with differences; the hash is uniform."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import train_oracle as to
from paper_2512_08888_amd import binding as rc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INF = float("inf")
NAN = float("nan")


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "unettrain.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(train_[a-z_0-9]+)\s*\(", text)))
    assert sorted(rc.TRAIN_EXPORTS) == names
    for n in names:
        assert hasattr(rc.lib(), n), n


def fwd(x=16, y=32, mean=None, rstd=None, N=1, C=4, P=4, G=2, eps=1e-5, act=0, layout=0, ws=1 << 20, ws_bytes=1 << 20, bf16=False):
    f = rc.lib().train_groupnorm_fwd_bf16 if bf16 else rc.lib().train_groupnorm_fwd
    return f(x, None, None, y, mean, rstd, N, C, P, G, eps, act, layout, ws, ws_bytes, None)


def bwd(x=16, dy=16, mean=16, rstd=16, dx=16, N=1, C=4, P=4, G=2, act=0, layout=0, ws=1 << 20, ws_bytes=1 << 20, bf16=False):
    f = rc.lib().train_groupnorm_bwd_bf16 if bf16 else rc.lib().train_groupnorm_bwd
    return f(x, dy, None, None, mean, rstd, dx, None, None, N, C, P, G, act, layout, ws, ws_bytes, None)


SHAPES = [dict(N=0), dict(N=-1), dict(C=0), dict(P=0), dict(G=0), dict(G=3), dict(G=8), dict(P=1 << 41), dict(N=1 << 30, C=1 << 10, G=1)]


@pytest.mark.parametrize("bf16", [False, True])
def test_groupnorm_refusals(bf16):
    for f in (fwd, bwd):
        assert f(x=None, bf16=bf16) == rc.ERR_NULL
        for kw in SHAPES:
            assert f(bf16=bf16, **kw) == rc.ERR_SHAPE, kw
        for kw in (dict(act=3), dict(act=-1), dict(layout=2), dict(layout=-1), dict(x=17)):
            assert f(bf16=bf16, **kw) == rc.ERR_UNSUPPORTED, kw
        for kw in (dict(ws=None), dict(ws_bytes=8), dict(ws=(1 << 20) + 4)):
            assert f(bf16=bf16, **kw) == rc.ERR_WORKSPACE, kw
    assert fwd(y=None, bf16=bf16) == rc.ERR_NULL
    assert fwd(eps=-1.0, bf16=bf16) == rc.ERR_UNSUPPORTED and fwd(eps=NAN, bf16=bf16) == rc.ERR_UNSUPPORTED
    for name in ("dy", "mean", "rstd", "dx"):
        assert bwd(bf16=bf16, **{name: None}) == rc.ERR_NULL, name


def test_groupnorm_workspace():
    assert rc.train_groupnorm_workspace_bytes(4, 64, 512 * 512, 32) > 0
    for N, C, P, G in ((0, 4, 4, 2), (1, 4, 4, 3), (1, 4, 0, 2)):
        assert rc.train_groupnorm_workspace_bytes(N, C, P, G) == 0


def make_list(rows, grad_dtype=0, count=None):
    arr = (rc.TrainTensor * max(1, len(rows)))(*[rc.TrainTensor(*r) for r in rows])
    h = ctypes.c_void_p()
    return rc.lib().train_list_create(arr, len(rows) if count is None else count, grad_dtype, ctypes.byref(h))


def test_list_refusals():
    good = (16, 32, None, 5, 0.0, 0)
    assert rc.lib().train_list_create(None, 1, 0, ctypes.byref(ctypes.c_void_p())) == rc.ERR_NULL
    assert rc.lib().train_list_create((rc.TrainTensor * 1)(rc.TrainTensor(*good)), 1, 0, None) == rc.ERR_NULL
    assert make_list([good], count=0) == rc.ERR_SHAPE and make_list([good], count=-1) == rc.ERR_SHAPE
    assert make_list([good], grad_dtype=2) == rc.ERR_UNSUPPORTED
    assert make_list([good, (16, None, None, 5, 0.0, 0)]) == rc.ERR_NULL
    assert make_list([good, (None, 32, None, 5, 0.0, 0)]) == rc.ERR_NULL          # some with a parameter, some without
    assert make_list([(None, 32, 64, 5, 0.0, 0)]) == rc.ERR_NULL                  # a copy of no parameter
    assert make_list([good, (16, 32, None, 0, 0.0, 0)]) == rc.ERR_SHAPE
    assert make_list([(16, 32, None, 1 << 41, 0.0, 0)]) == rc.ERR_SHAPE
    for bad in ((16, 32, None, 5, -0.1, 0), (16, 32, None, 5, NAN, 0), (16, 32, None, 5, 0.0, 1), (18, 32, None, 5, 0.0, 0),
                (16, 34, None, 5, 0.0, 0), (16, 32, 65, 5, 0.0, 0)):
        assert make_list([bad]) == rc.ERR_UNSUPPORTED, bad
    assert rc.lib().train_list_destroy(None) == rc.OK
    assert rc.lib().train_list_elements(None) == 0 and rc.lib().train_list_workspace_bytes(None) == 0


def test_calls_on_lists_refuse_null():
    L, o = rc.lib(), rc.TrainAdamW(0.9, 0.999, 1e-8, 0, 0, 0)
    assert L.train_control_init(None, 0, 0.1, None) == rc.ERR_NULL
    assert L.train_control_init(64, -1, 0.1, None) == rc.ERR_SHAPE
    assert L.train_control_init(66, 0, 0.1, None) == rc.ERR_UNSUPPORTED
    assert L.train_grad_norm(None, 1.0, None, 64, 64, 64, None) == rc.ERR_NULL
    assert L.train_adamw_step(None, ctypes.byref(o), 64, 64, None, None, 64, None) == rc.ERR_NULL


def test_binding_refusals():
    import torch

    x = torch.zeros(2, 6, 3, 5)
    last = x.contiguous(memory_format=torch.channels_last)
    v, s = torch.ones(6), torch.zeros(2, 3)
    for args in ((x, last), (x, x[:, :, :, :4]), (x.transpose(2, 3), x.transpose(2, 3)), (x, x[:1])):
        with pytest.raises(ValueError):
            rc.train_groupnorm_fwd(args[0], v, v, args[1], s, s, 3)
    for kw in (dict(gamma=torch.ones(5)), dict(beta=v.double()), dict(mean=torch.zeros(2, 2)), dict(act="tanh")):
        a = dict(gamma=v, beta=v, mean=s, act="none")
        a.update(kw)
        with pytest.raises(ValueError):
            rc.train_groupnorm_fwd(x, a["gamma"], a["beta"], torch.zeros_like(x), a["mean"], s, 3, act=a["act"])
    with pytest.raises(TypeError):
        rc.TrainList([torch.zeros(3), torch.zeros(3, dtype=torch.bfloat16)])
    with pytest.raises(TypeError):
        rc.TrainList([torch.zeros(3)], [torch.zeros(4)])
    with pytest.raises(TypeError):
        rc.TrainList([torch.zeros(3)], [torch.zeros(3)], [torch.zeros(3)])
    with pytest.raises(ValueError):
        rc.TrainList([torch.zeros(3)], [torch.zeros(3)], weight_decay=[0.1, 0.1])
    with pytest.raises(ValueError):
        rc.TrainList([torch.zeros(4, 4).t()])


def test_binding_refuses_host_memory():
    import torch

    x, v, s = torch.zeros(2, 6, 3, 5), torch.ones(6), torch.zeros(2, 3)
    with pytest.raises(ValueError, match="GPU"):
        rc.train_groupnorm_fwd(x, v, v, torch.zeros_like(x), s, s, 3)
    with pytest.raises(ValueError, match="GPU"):
        rc.train_groupnorm_bwd(x, x, v, v, s, s, torch.zeros_like(x), v, v, 3)
    with pytest.raises(ValueError, match="GPU"):
        rc.TrainList([torch.zeros(3)], [torch.zeros(3)])
    with pytest.raises(ValueError, match="GPU"):
        rc.train_control_init(torch.zeros(16, dtype=torch.int32))


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("shape,groups", [((2, 6, 5), 3), ((1, 4, 1), 1), ((3, 4, 7), 4)])
def test_oracle_gradients_against_differences(act, shape, groups):
    rng = np.random.default_rng(1)
    N, C, P = shape
    x, w = rng.standard_normal(shape) + 0.5, rng.standard_normal(shape)
    ga, be = 1 + 0.2 * rng.standard_normal(C), 0.3 * rng.standard_normal(C)

    def loss(x, ga, be):
        return (w * to.groupnorm_fwd(x, ga, be, groups, 1e-3, act)[0]).sum()

    mean, rstd = to.groupnorm_stats(x, groups, 1e-3)
    dx, dga, dbe = to.groupnorm_bwd(x, w, ga, be, mean, rstd, groups, act)
    h = 1e-5
    for grad, k in ((dx, 0), (dga, 1), (dbe, 2)):
        args = [x, ga, be]
        for i in np.ndindex(grad.shape):
            lo, hi = [a.copy() for a in args], [a.copy() for a in args]
            lo[k][i] -= h
            hi[k][i] += h
            # central differences: h^2 times a third derivative (below 1e4 here: rstd <= 32 cubed times weights), 1e-16 / h rounding
            assert abs((loss(*hi) - loss(*lo)) / (2 * h) - grad[i]) < 1e-5 * (1 + abs(grad[i]))


def test_e4m3_values_and_exponents():
    import torch

    codes = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(to.e4m3(codes), ref, equal_nan=True)
    x = np.zeros((6, 32))
    x[0, 3], x[1, 5], x[2, 7], x[3, 9], x[4, 1] = 448.0, -448.0001, 224.0, 1e-45, 3.4e38
    assert to.block_exponents(x).tolist() == [0, 1, -1, -127, 120, -127]


def test_random_bits_are_uniform():
    """Sixteen bits of 2^18 consecutive positions in two steps: mean, correlation of neighbours and of the two steps within
    five standard deviations, every 64th of the range filled evenly (chi-square, 63 degrees of freedom, below 150)."""
    n = 1 << 18
    a, b = to.random16(np.arange(n), 1, 7), to.random16(np.arange(n), 2, 7)
    for u in (a, b):
        assert abs(u.mean() - 0.5) < 5 * np.sqrt(1 / 12 / n)
        for lag in (1, 2, 32):
            assert abs(np.corrcoef(u[:-lag], u[lag:])[0, 1]) < 5 / np.sqrt(n)
        hist = np.bincount((u * 64).astype(int), minlength=64)
        assert ((hist - n / 64) ** 2 / (n / 64)).sum() < 150
    assert abs(np.corrcoef(a, b)[0, 1]) < 5 / np.sqrt(n)


def test_lists_of_more_tensors_than_a_launch_has_workgroups_are_refused():
    """2^24 tensors of one element: refused before anything is copied to a device."""
    row = np.zeros(1, dtype=[("param", "u8"), ("grad", "u8"), ("copy", "u8"), ("n", "u8"), ("weight_decay", "f4"), ("reserved", "i4")])
    assert row.itemsize == ctypes.sizeof(rc.TrainTensor)
    row["grad"], row["n"] = 64, 1
    rows = np.broadcast_to(row, 1 << 24).copy()
    h = ctypes.c_void_p()
    at = ctypes.cast(rows.ctypes.data, ctypes.POINTER(rc.TrainTensor))
    assert rc.lib().train_list_create(at, rows.size, 0, ctypes.byref(h)) == rc.ERR_SHAPE and not h


def test_numbers_that_no_c_int_holds_are_refused():
    for call in (lambda: rc.train_groupnorm_workspace_bytes((1 << 32) + 1, 4, 4, 2), lambda: rc.train_groupnorm_workspace_bytes(1, 4, 4, (1 << 32) + 2),
                 lambda: rc.train_control_init(None, 1 << 32)):
        with pytest.raises(rc.RotconvError) as e:
            call()
        assert e.value.status == rc.ERR_SHAPE


def test_a_step_number_without_a_successor_is_refused():
    assert rc.lib().train_control_init(64, 2**31 - 1, 0.1, None) == rc.ERR_SHAPE

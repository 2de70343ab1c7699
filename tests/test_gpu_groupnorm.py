"""Group normalisation with an activation (include/unettrain.h) against the 64-bit oracle.

Bars.  u = 2^-24.  A statistic is a sum of at most K = 256 terms one after the other at the sizes here, joined in pairs
or in 64 bits: relative to the sums of magnitudes, the mean is off by (K + 4) u and the variance by 4 (K + 4) u, whence
rstd by 2 (K + 4) u and xh by (K + 4) u (2 |xh| + (mean |x - x0| + |mean|) rstd).  A gradient's two means are sums of
products: (K + 8) u of the sums of magnitudes.  Forming z, the activation (an exponential within 16 |z| u) and the result
adds fewer than 64 + 16 |z| units of u each.  A bf16 result adds one rounding, 2^-8 of its magnitude at the most.
"""
import numpy as np
import pytest
import torch

from oracle import train_oracle as to
from paper_2512_08888_amd import binding as rc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
K = 256 + 4
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dtype).cuda()


class Guarded:
    """A map between two stretches of a known pattern, at `shift` elements past an aligned address."""

    def __init__(self, shape, dtype, layout, shift=0):
        N, C, H, W = shape
        n = N * C * H * W
        self.flat = torch.full((n + 128 + shift,), 77.0, dtype=dtype, device="cuda")
        body = self.flat[64 + shift:64 + shift + n]
        body.fill_(float("nan"))
        self.map = body.view(N, C, H, W) if layout == "nchw" else body.view(N, H, W, C).permute(0, 3, 1, 2)
        self.lo, self.hi = self.flat[:64 + shift], self.flat[64 + shift + n:]

    def put(self, t):
        self.map.copy_(t)
        return self

    def intact(self):
        return bool((self.lo == 77).all()) and bool((self.hi == 77).all())


class Case:
    def __init__(self, N, C, H, W, G, act="none", layout="nchw", dtype="f32", affine=True, shift=0, offset=0.7, seed=0):
        rng = np.random.default_rng(seed + N * 1000 + C * 10 + H)
        self.N, self.C, self.H, self.W, self.G, self.act, self.dtype = N, C, H, W, G, act, dtype
        self.shape = (N, C, H, W)
        self.layout, self.shift = layout, shift
        self.x = self.round(rng.standard_normal(self.shape) * (0.5 + rng.random((1, C, 1, 1))) + offset)
        self.dy = self.round(rng.standard_normal(self.shape))
        self.gamma = (1 + 0.3 * rng.standard_normal(C)).astype(np.float32) if affine else None
        self.beta = (0.3 * rng.standard_normal(C)).astype(np.float32) if affine else None

    def round(self, a):
        return torch.from_numpy(a.astype(np.float32)).to(DT[self.dtype]).float().numpy()

    def map(self, a=None):
        m = Guarded(self.shape, DT[self.dtype], self.layout, self.shift)
        return m if a is None else m.put(dev(a, DT[self.dtype]))

    def vec(self, a):
        return None if a is None else dev(a)

    def affine64(self):
        one, zero = np.ones(self.C), np.zeros(self.C)
        return (one if self.gamma is None else self.gamma), (zero if self.beta is None else self.beta)

    def ws(self):
        n = rc.train_groupnorm_workspace_bytes(self.N, self.C, self.H * self.W, self.G)
        buf = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        return buf, buf[:n]

    def forward(self, stats=True, eps=1e-5):
        x, y = self.map(self.x), self.map()
        mean, rstd = (torch.full((self.N, self.G), float("nan"), device="cuda") for _ in range(2))
        buf, ws = self.ws()
        rc.train_groupnorm_fwd(x.map, self.vec(self.gamma), self.vec(self.beta), y.map, mean if stats else None,
                               rstd if stats else None, self.G, eps=eps, act=self.act, ws=ws)
        torch.cuda.synchronize()
        assert y.intact() and x.intact() and bool((buf[ws.numel():] == 0xA5).all())
        return y.map.float().cpu().numpy(), mean.cpu().numpy(), rstd.cpu().numpy()

    def backward(self, mean, rstd, inplace=False, vectors=True):
        x, dy = self.map(self.x), self.map(self.dy)
        dx = dy if inplace else self.map()
        dga, dbe = (torch.full((self.C,), float("nan"), device="cuda") for _ in range(2))
        buf, ws = self.ws()
        rc.train_groupnorm_bwd(x.map, dy.map, self.vec(self.gamma), self.vec(self.beta), dev(mean), dev(rstd), dx.map,
                               dga if vectors else None, dbe if vectors else None, self.G, act=self.act, ws=ws)
        torch.cuda.synchronize()
        assert dx.intact() and dy.intact() and x.intact() and bool((buf[ws.numel():] == 0xA5).all())
        return dx.map.float().cpu().numpy(), dga.cpu().numpy(), dbe.cpu().numpy()

    def flat(self, a):
        return a.reshape(self.N, self.C, -1)

    def spread(self, t):           # [N, G] -> [N, C, 1]
        return np.repeat(np.asarray(t, np.float64), self.C // self.G, axis=1)[..., None]

    def check_forward(self, eps=1e-5):
        y, mean, rstd = self.forward(eps=eps)
        ga, be = self.affine64()
        x = self.flat(self.x).astype(np.float64)
        ry, rmean, rrstd = to.groupnorm_fwd(x, ga, be, self.G, eps, self.act)
        g = x.reshape(self.N, self.G, -1)
        dev0 = np.abs(g - g[..., :1]).mean(2) + np.abs(g - g.mean(2, keepdims=True)).mean(2) * 2
        e_mean = K * U * (dev0 + np.abs(rmean))
        assert np.all(np.abs(mean - rmean) <= e_mean)
        # a variance near nothing: its error is that of the mean, squared, and of the deviations' own rounding
        assert np.all(np.abs(rstd - rrstd) <= rrstd * (2 * K * U + 0.5 * rrstd ** 2 * (e_mean ** 2 + 4 * K * U * dev0 ** 2)))
        xh = (x - self.spread(rmean)) * self.spread(rrstd)
        z = xh * ga[None, :, None] + be[None, :, None]
        e_xh = K * U * (2 * np.abs(xh)) + self.spread(e_mean * rrstd) + 4 * U * (np.abs(x) + np.abs(self.spread(rmean))) * self.spread(rrstd) \
            + np.abs(xh) * self.spread(0.5 * rrstd ** 2 * (e_mean ** 2 + 4 * K * U * dev0 ** 2))
        bar = 1.2 * (np.abs(ga)[None, :, None] * e_xh) + U * (64 + 16 * np.abs(z)) * (np.abs(z) + np.abs(be)[None, :, None]) + 1e-30
        if self.dtype == "bf16":
            bar = bar + 2.0 ** -8 * np.abs(ry)
        assert np.all(np.abs(self.flat(y) - ry) <= bar)
        return mean, rstd

    def check_backward(self, mean, rstd, **kw):
        dx, dga, dbe = self.backward(mean, rstd, **kw)
        ga, be = self.affine64()
        x, dy = self.flat(self.x), self.flat(self.dy)
        rdx, rdga, rdbe = to.groupnorm_bwd(x, dy, ga, be, mean, rstd, self.G, self.act)
        x64, dy64 = x.astype(np.float64), np.abs(dy.astype(np.float64))
        r = self.spread(rstd)
        xh = np.abs((x64 - self.spread(mean)) * r)
        z = xh * np.abs(ga)[None, :, None] + np.abs(be)[None, :, None]
        # |xh| carries the cancellation of x - mean; silu's derivative is at most 1.1, its slope at most 0.5
        e_xh = 2 * U * xh + U * np.abs(x64) * r
        dz = 1.1 * dy64
        e_dz = dy64 * (U * (64 + 16 * z) + (0.5 * np.abs(ga)[None, :, None] * e_xh + 2 * U * z if self.act == "silu" else 0))
        t, e_t = dz * np.abs(ga)[None, :, None], (e_dz + U * dz) * np.abs(ga)[None, :, None]
        mean_of = lambda a: self.spread(a.reshape(self.N, self.G, -1).mean(2))  # noqa: E731
        c1, c2 = mean_of(t), mean_of(t * xh)
        e_c1, e_c2 = (K + 4) * U * c1 + mean_of(e_t), (K + 4) * U * c2 + mean_of(e_t * xh + t * e_xh)
        bar = r * (e_t + e_c1 + xh * e_c2 + e_xh * c2 + 8 * U * (t + c1 + xh * c2)) + 1e-30
        if self.dtype == "bf16":
            bar = bar + 2.0 ** -8 * np.abs(rdx)
        assert np.all(np.abs(self.flat(dx) - rdx) <= bar)
        if kw.get("vectors", True):
            sum_of = lambda a: a.sum((0, 2))  # noqa: E731
            assert np.all(np.abs(dbe - rdbe) <= (K + 4) * U * sum_of(dz) + sum_of(e_dz) + 1e-30)
            assert np.all(np.abs(dga - rdga) <= (K + 4) * U * sum_of(dz * xh) + sum_of(e_dz * xh + dz * e_xh) + 1e-30)


# (N, C, H, W, G): one pixel, one element a group, one channel a group (instance norm), one group (layer norm), odd
# everything, vectors that end inside a row, more channels than threads, groups as large as a workgroup holds and larger
SHAPES = [
    (1, 1, 1, 1, 1), (2, 4, 1, 1, 2), (3, 4, 1, 1, 4), (1, 32, 1, 1, 1), (5, 6, 2, 3, 6), (2, 10, 7, 9, 5), (1, 7, 5, 5, 1),
    (3, 12, 13, 11, 4), (2, 24, 16, 16, 6), (4, 64, 16, 16, 8), (1, 3, 101, 75, 3), (2, 60, 33, 37, 12), (1, 600, 3, 5, 100),
    (1, 1030, 2, 2, 10), (2, 32, 64, 64, 4), (1, 16, 96, 80, 2), (2, 8, 128, 128, 2), (1, 4, 200, 333, 1), (1, 2, 512, 512, 1),
    (70, 8, 4, 4, 2), (1, 512, 20, 20, 1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_against_the_oracle(act, layout, dtype):
    for shape in SHAPES:
        c = Case(*shape, act=act, layout=layout, dtype=dtype)
        print(shape, flush=True)
        mean, rstd = c.check_forward()
        c.check_backward(mean, rstd)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_addresses_off_the_vector_grid(layout, dtype):
    """Maps that start one to three elements past an aligned address, of sizes that would otherwise take vectors."""
    for shift in (1, 2, 3, 4):
        for shape in ((2, 16, 8, 8, 4), (1, 8, 64, 64, 1), (2, 64, 32, 40, 8)):
            c = Case(*shape, act="relu", layout=layout, dtype=dtype, shift=shift)
            mean, rstd = c.check_forward()
            c.check_backward(mean, rstd)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
def test_optional_arguments(layout):
    for shape in ((2, 12, 9, 7, 4), (1, 8, 96, 96, 2)):
        c = Case(*shape, act="silu", layout=layout, affine=False)
        y0, mean, rstd = c.forward()
        c.check_forward()
        y1, m1, r1 = c.forward(stats=False)
        assert np.array_equal(y0, y1) and np.isnan(m1).all() and np.isnan(r1).all()
        a, b = c.backward(mean, rstd), c.backward(mean, rstd, vectors=False)
        c.check_backward(mean, rstd)
        assert np.array_equal(a[0], b[0]) and np.isnan(b[1]).all() and np.isnan(b[2]).all()


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_in_place(layout, dtype):
    for shape in ((2, 16, 8, 8, 4), (1, 6, 31, 29, 2), (1, 16, 160, 160, 2), (3, 40, 40, 41, 5)):
        c = Case(*shape, act="relu", layout=layout, dtype=dtype)
        _, mean, rstd = c.forward()
        assert np.array_equal(c.backward(mean, rstd)[0], c.backward(mean, rstd, inplace=True)[0])
        c.check_backward(mean, rstd, inplace=True)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("shape", [(2, 8, 16, 16, 2), (1, 4, 128, 128, 1), (2, 30, 33, 31, 5)])
def test_maps_far_from_zero(layout, shape):
    """A mean a few thousand times the spread: the variance is that of the deviations, not a difference of two squares."""
    c = Case(*shape, act="none", layout=layout, offset=4096.0)
    mean, rstd = c.check_forward()
    c.check_backward(mean, rstd)


def test_constant_groups():
    for shape in ((2, 4, 8, 8, 2), (1, 2, 128, 128, 1)):
        c = Case(*shape, act="none")
        c.x[:] = 3.25
        y, mean, rstd = c.forward()
        assert np.array_equal(mean, np.full_like(mean, 3.25))
        assert np.allclose(rstd, 1 / np.sqrt(1e-5), rtol=4 * U, atol=0)
        assert np.array_equal(y, np.broadcast_to(c.beta[None, :, None, None], y.shape))


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_value_that_is_not_finite_stays_in_its_group(bad, act, layout):
    for shape in ((2, 12, 9, 7, 4), (2, 4, 96, 90, 2)):
        c, ref = Case(*shape, act=act, layout=layout), Case(*shape, act=act, layout=layout)
        N, C, H, W, G = shape
        cg = C // G
        c.x[1, cg, H // 2, W // 2] = bad              # image 1, group 1
        y, mean, rstd = c.forward()
        ry, rmean, rrstd = ref.forward()
        inside = np.zeros((N, C), bool)
        inside[1, cg:2 * cg] = True
        assert np.isnan(y[inside]).all() and np.isnan(rstd[1, 1])
        assert np.array_equal(y[~inside], ry[~inside])
        keep = np.ones((N, G), bool)
        keep[1, 1] = False
        assert np.array_equal(mean[keep], rmean[keep]) and np.array_equal(rstd[keep], rrstd[keep])
        dx, dga, dbe = c.backward(mean, rstd)
        rdx, _, _ = ref.backward(rmean, rrstd)
        assert np.isnan(dx[inside]).all() and np.array_equal(dx[~inside], rdx[~inside])
        outside = [k for k in range(C) if not cg <= k < 2 * cg]
        assert np.isfinite(dga[outside]).all() and np.isnan(dga[cg:2 * cg]).all()


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_on_every_run_and_stream(layout, dtype):
    for shape in ((4, 64, 32, 32, 8), (2, 16, 200, 120, 2)):
        c = Case(*shape, act="silu", layout=layout, dtype=dtype)
        a, g = c.forward(), None
        g = c.backward(a[1], a[2])
        side = torch.cuda.Stream()
        for k in range(3):
            torch.cuda.synchronize()
            with torch.cuda.stream(side if k else torch.cuda.current_stream()):
                b = c.forward()
                h = c.backward(b[1], b[2])
            assert all(np.array_equal(p, q) for p, q in zip(a + g, b + h))


def test_gradient_against_differences():
    """The library's dx along a direction d against differences of its own forward pass: L(x + h d) - L(x - h d) over 2 h.
    With h = 2^-6 the difference is off by h^2 / 6 times a third derivative of L along d (measured on the oracle in 64 bits,
    where h is shrunk until the difference stands), and by the forward's rounding, 2^-18 of the sum of magnitudes, over h."""
    for layout in ("nchw", "nhwc"):
        c = Case(2, 12, 15, 17, 3, act="silu", layout=layout)
        rng = np.random.default_rng(5)
        d = rng.standard_normal(c.shape).astype(np.float32)
        w = c.dy.astype(np.float64)
        _, mean, rstd = c.forward()
        slope = (c.backward(mean, rstd)[0].astype(np.float64) * d).sum()
        x0, h = c.x.copy(), 2.0 ** -6
        loss, exact = [], []
        for s in (-1, 1):
            c.x = (x0 + s * h * d).astype(np.float32)
            loss.append((c.forward()[0].astype(np.float64) * w).sum())
        for s in (-h, h, -h / 64, h / 64):
            exact.append((to.groupnorm_fwd(c.flat(x0 + s * d.astype(np.float64)), *c.affine64(), 3, 1e-5, "silu")[0] * c.flat(w)).sum())
        curve = abs((exact[1] - exact[0]) / (2 * h) - (exact[3] - exact[2]) / (2 * h / 64))
        rounding = 2.0 ** -18 * np.abs(w).sum() / h
        assert abs((loss[1] - loss[0]) / (2 * h) - slope) <= 1.01 * curve + rounding + 2.0 ** -12 * abs(slope)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
def test_offsets_beyond_32_bits(layout):
    """A bf16 map of more than 2^32 elements: the first and the last image against the oracle's formula in 64 bits (torch on
    the device).  The images repeat one pattern, shifted and scaled for each image."""
    N, C, H, W, G = 5, 8, 12288, 8800, 2
    assert N * C * H * W > 1 << 32
    order = torch.channels_last if layout == "nhwc" else torch.contiguous_format
    x = torch.empty((N, C, H, W), dtype=torch.bfloat16, device="cuda", memory_format=order)
    y = torch.empty((N, C, H, W), dtype=torch.bfloat16, device="cuda", memory_format=order)
    base = torch.linspace(-1, 1, H * W, device="cuda").view(H, W)
    for n in range(N):
        for k in range(C):
            x[n, k].copy_(base * (1 + 0.1 * k) + 0.25 * n)
    mean, rstd = (torch.empty(N, G, device="cuda") for _ in range(2))
    rc.train_groupnorm_fwd(x, None, None, y, mean, rstd, G, act="relu")
    for n in (0, N - 1):
        for g in range(G):
            v = x[n, 4 * g:4 * g + 4].double()
            mu, sd = v.mean(), (v.var(unbiased=False) + 1e-5).sqrt()
            assert abs(mean[n, g].item() - mu.item()) < 1e-5 and abs(rstd[n, g].item() * sd.item() - 1) < 1e-4
            ref = ((v - mu) / sd).clamp(min=0)
            assert float((y[n, 4 * g:4 * g + 4].double() - ref).abs().max()) <= 2.0 ** -8 * 2.5 + 1e-3
            del v, ref
    # dy = 1 without an activation: dx is 0 but for rounding, dbeta the number of pixels
    dx, dy = y, x.clone(memory_format=torch.preserve_format).fill_(1)
    dga, dbe = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    rc.train_groupnorm_bwd(x, dy, None, None, mean, rstd, dx, dga, dbe, G)
    assert float(dx[0].float().abs().max()) < 1e-3 and float(dx[N - 1].float().abs().max()) < 1e-3
    assert torch.allclose(dbe, torch.full_like(dbe, float(N * H * W)), rtol=1e-4)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_workgroups_that_do_not_wait(layout, dtype):
    """With no time to wait for one another, workgroups that share a group sum its other parts themselves: the same bits."""
    for shape in ((2, 8, 128, 128, 2), (1, 4, 200, 333, 1), (3, 60, 101, 75, 12), (1, 32, 64, 63, 32)):
        c = Case(*shape, act="silu", layout=layout, dtype=dtype)
        a = c.forward()
        g = c.backward(a[1], a[2])
        before = rc.train_diag_groupnorm_wait(0)
        try:
            b = c.forward()
            h = c.backward(a[1], a[2])
            i = c.backward(a[1], a[2], inplace=True)
        finally:
            assert rc.train_diag_groupnorm_wait(before) == 0
        assert all(np.array_equal(p, q) for p, q in zip(a + g + g, b + h + i)), shape


def test_pieces_that_divide_a_channel_but_for_its_end():
    """A channel's whole vectors divide evenly over its pieces and a few pixels are left."""
    for P, dtype in ((8 * 2520 + 3, "f32"), (20480 + 1, "f32"), (4 * 8 * 512 + 3, "f32"), (16 * 1031 + 7, "bf16"), (8 * 512 * 2 + 5, "bf16"),
                     (8 * 4096 + 7, "bf16"), (16 * 4096 + 1, "bf16")):
        c = Case(2, 3, 1, P, 1, act="relu", dtype=dtype)
        mean, rstd = c.check_forward()
        c.check_backward(mean, rstd)


# Maps of more than 8 MiB, whose workgroups exchange their groups' sums within the launch: odd numbers of pixels, a channel
# in several pieces, several channels to a workgroup's part, vectors across groups, channels that fill no vector
SHARED = {"nchw": [(4, 64, 133, 131, 4), (9, 24, 141, 143, 1)], "nhwc": [(4, 64, 133, 131, 4), (5, 56, 131, 127, 14), (10, 33, 120, 123, 3)]}
# Groups of more parts than wait for one another, or of more sums than a workgroup collects; groups wider than a run of
# channels, and runs that are not of whole groups
THREE = {"nchw": [(1, 6, 1201, 1200, 1), (1, 12, 1201, 1200, 1), (1, 65700, 1, 7, 1), (1, 33000, 8, 8, 1)],
         "nhwc": [(2, 521, 5, 7, 521), (1, 2060, 3, 3, 2), (1, 2064, 4, 3, 2), (2, 2056, 3, 7, 2), (1, 64, 130, 130, 64), (2, 33, 190, 199, 11)]}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("which", ["shared", "three"])
def test_large_groups_against_the_oracle(which, layout, dtype):
    for k, shape in enumerate((SHARED if which == "shared" else THREE)[layout]):
        c = Case(*shape, act=("silu", "relu", "none")[k % 3], layout=layout, dtype=dtype, shift=k % 2)
        print(shape, flush=True)
        mean, rstd = c.check_forward()
        c.check_backward(mean, rstd)


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_groups_have_the_same_bits_however_they_wait(layout, dtype):
    """With no time to wait, every part is left to the launch behind; also in place, and without what may be left out."""
    for shape in SHARED[layout] + THREE[layout]:
        c = Case(*shape, act="silu", layout=layout, dtype=dtype)
        print(shape, flush=True)
        a = c.forward()
        g = c.backward(a[1], a[2])
        before = rc.train_diag_groupnorm_wait(0)
        try:
            b, n = c.forward(), c.forward(stats=False)
            h, i = c.backward(a[1], a[2]), c.backward(a[1], a[2], inplace=True)
            v = c.backward(a[1], a[2], vectors=False)
        finally:
            assert rc.train_diag_groupnorm_wait(before) == 0
        j = c.backward(a[1], a[2], inplace=True)
        assert all(np.array_equal(p, q) for p, q in zip(a + g + g + g, b + h + i + j)), shape
        assert np.array_equal(n[0], a[0]) and np.array_equal(v[0], g[0])


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
def test_large_groups_far_from_zero(layout):
    for shape in (SHARED[layout][0], THREE[layout][-2 if layout == "nhwc" else 0]):
        c = Case(*shape, act="none", layout=layout, offset=4096.0)
        mean, rstd = c.check_forward()
        c.check_backward(mean, rstd)


def test_more_groups_than_a_launch_has_workgroups_for():
    """20 million groups of one element, in runs of channels that hold no whole number of vectors: x - mean is 0."""
    N, C = 300, 65521
    x = torch.randn(N, C, 1, 1, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(N, C, device="cuda"), torch.empty(N, C, device="cuda")
    rc.train_groupnorm_fwd(x, None, None, y, mean, rstd, C)
    assert torch.equal(mean, x[:, :, 0, 0]) and bool((y == 0).all())
    assert float((rstd * (1e-5 ** 0.5) - 1).abs().max()) <= 4 * U
    dy, dga, dbe = torch.randn_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    dx = torch.empty_like(x)
    rc.train_groupnorm_bwd(x, dy, None, None, mean, rstd, dx, dga, dbe, C)
    assert bool((dx == 0).all()) and bool((dga == 0).all())
    assert bool(((dbe.double() - dy[:, :, 0, 0].double().sum(0)).abs() <= 2 * U * dy.double().abs().sum((0, 2, 3))).all())


# Maps whose first pixel (a corner, the edge of a padding) is far from the others, which are noise or all alike; one workgroup a
# group, two launches, groups shared by workgroups that wait for one another, three launches
OUTLIERS = [(1, 1, 64, 64, 1), (2, 8, 64, 64, 2), (3, 12, 13, 11, 4), (2, 10, 7, 9, 5), (1, 1030, 2, 2, 10), (4, 64, 128, 128, 32),
            (1, 2, 512, 512, 1), (2, 60, 101, 75, 12), (4, 64, 133, 131, 4), (1, 6, 1201, 1200, 1), (1, 64, 130, 130, 64), (1, 8, 1024, 1024, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("rest,far", [(0.0, 7.3), (0.0, -300.0), (0.1, 5.0), (1.0, 1000.0), (1e-3, 1e4)])
@pytest.mark.parametrize("where", ["channels", "one", "strip", "sparse"])
def test_values_far_from_the_others(where, rest, far, layout, dtype):
    """The bars here do not grow with the distance of the first element.  Statistics are sums of deviations from a point at most a
    deviation from the mean (see the bars above): the mean is off by K u (mean |x - mean| + |mean|), the variance by 8 K u of
    itself, rstd by half of that."""
    for shape in OUTLIERS:
        N, C, H, W, G = shape
        rng = np.random.default_rng(C + H)
        c = Case(*shape, layout=layout, dtype=dtype, affine=False)
        x = rest * rng.standard_normal((N, C, H * W)) + (0.25 if far < 0 else 0.0)
        if where == "channels":
            x[:, :, 0] = far
        elif where == "one":
            x[:, 0, 0] = far
        elif where == "strip":
            x[:, :, : H * W // 32] = far
        else:
            x[rng.random(x.shape) < 1 / 5000] = far
            x[:, :: max(1, C // G), 0] = far
        c.x = c.round(x.reshape(N, C, H, W))
        y, mean, rstd = c.forward()
        x = c.flat(c.x).astype(np.float64)
        ry, rmean, rrstd = to.groupnorm_fwd(x, np.ones(C), np.zeros(C), G, 1e-5, "none")
        g = x.reshape(N, G, -1)
        e_mean = K * U * (np.abs(g - rmean[..., None]).mean(2) + np.abs(rmean))
        print(shape, flush=True)
        assert np.all(np.abs(mean - rmean) <= e_mean), shape
        assert np.all(np.abs(rstd - rrstd) <= rrstd * 4 * K * U), shape
        bar = c.spread(e_mean * rrstd) + np.abs(ry) * (4 * K * U + 64 * U) + 4 * U * (np.abs(x) + np.abs(c.spread(rmean))) * c.spread(rrstd) + 1e-30
        if dtype == "bf16":
            bar = bar + 2.0 ** -8 * np.abs(ry)
        assert np.all(np.abs(c.flat(y) - ry) <= bar), shape


@pytest.mark.parametrize("layout", ["nchw", "nhwc"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sums_over_the_images_pass_a_nan_on(dtype, act, layout):
    """A group whose results are NaN makes its channels' gradients NaN, the shift's too (where there is an activation: without
    one it is the sum of dy alone), and no others: a ReLU does not take its elements for dead ones.  One workgroup a group, groups shared by several, three launches."""
    for shape in ((2, 12, 9, 7, 4), (2, 4, 96, 90, 2), (2, 64, 133, 131, 4), (1, 6, 1201, 1200, 2), (2, 521, 5, 7, 521)):
        N, C, H, W, G = shape
        cg = C // G
        for bad in (float("nan"), float("inf")):
            c, ref = Case(*shape, act=act, layout=layout, dtype=dtype), Case(*shape, act=act, layout=layout, dtype=dtype)
            c.x[N - 1, cg, H // 2, W // 2] = bad
            _, mean, rstd = c.forward()
            _, rmean, rrstd = ref.forward()
            _, dga, dbe = c.backward(mean, rstd)
            _, rdga, rdbe = ref.backward(rmean, rrstd)
            inside = np.arange(C) // cg == 1
            assert np.isnan(dga[inside]).all(), shape
            assert np.array_equal(dbe[inside], rdbe[inside]) if act == "none" else np.isnan(dbe[inside]).all(), shape
            assert np.array_equal(dga[~inside], rdga[~inside]) and np.array_equal(dbe[~inside], rdbe[~inside]), shape


def test_a_shift_or_scale_that_is_nan():
    """The channel's own gradients are NaN, and its group's maps."""
    for layout in ("nchw", "nhwc"):
        for which in ("gamma", "beta"):
            c = Case(2, 12, 9, 7, 4, act="relu", layout=layout)
            _, mean, rstd = c.forward()
            getattr(c, which)[4] = np.nan
            dx, dga, dbe = c.backward(mean, rstd)
            group = np.arange(12) // 3 == 1
            assert np.isnan(dx[:, group]).all() and np.isfinite(dx[:, ~group]).all()
            assert np.isnan(dbe[4]) and np.isfinite(np.delete(dbe, 4)).all() and np.isfinite(np.delete(dga, 4)).all()


def test_extents_beyond_32_bits_are_refused():
    """2^32 + 2 groups are not two, and a map of 2^32 + 4 images is not one of four."""
    x = torch.randn(2, 4, 3, 3, device="cuda")
    y, keep = torch.zeros_like(x), torch.zeros_like(x)
    for groups in ((1 << 32) + 2, -(1 << 32) + 2):
        with pytest.raises(rc.RotconvError) as e:
            rc.train_groupnorm_fwd(x, None, None, y, None, None, groups)
        assert e.value.status == rc.ERR_SHAPE
    x = torch.ones((1 << 32) + 4, 1, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(x)
    with pytest.raises(rc.RotconvError) as e:
        rc.train_groupnorm_fwd(x, None, None, out, None, None, 1)
    assert e.value.status == rc.ERR_SHAPE and torch.equal(y, keep) and not bool(out[:4].any())
    del x, out
    torch.cuda.empty_cache()

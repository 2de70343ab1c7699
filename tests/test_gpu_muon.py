"""Muon's step over many matrices (include/unettrain.h) against the 64-bit oracle.

Bars.  u = 2^-24.  Momentum and decay are a few operations, each rounded once: 4 u of the magnitudes that meet in a sum.  The
orthogonalised matrix is compared in the Frobenius norm with two errors added: three times the one that the same
roundings to fp16 make in the oracle (they are of another draw here, since fp32 sums round too), and what is left for
arithmetic in 22 bits and more: |x p'(x) / p(x)| is below 5 on [0, 1.21], so that a relative error of 2^-22 an iteration
grows to less than (5 + 5^2 + .. + 5^steps) 2^-22 < 5^steps 2^-21.
"""
import numpy as np
import pytest
import torch
from scipy.linalg import hadamard

from oracle import train_oracle as to
from paper_2512_08888_amd import binding as rc
from paper_2512_08888_amd import train

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# (count, rows, cols)
SMALL = [(1, 64, 576), (2, 16, 144), (1, 6, 64), (1, 1, 1), (1, 1, 70), (1, 70, 1), (3, 5, 3), (1, 64, 27), (1, 33, 65), (2, 65, 33)]
# a workgroup keeps a matrix (16, 32 and 64 blocks of 32 x 32), or launches of products serve all of them
LISTS = {"block": [(1, 20, 500), (1, 500, 20), (2, 30, 40)], "two": [(1, 64, 512), (1, 480, 50), (1, 33, 64)],
         "least": SMALL + [(1, 64, 1024), (1, 1024, 64), (1, 1000, 63), (1, 40, 1001)],
         "all": SMALL + [(1, 130, 129), (1, 128, 256), (1, 200, 300), (1, 65, 64), (1, 64, 1025)]}


class Net:
    """Parameters, gradients and copies of the given stacks inside guarded buffers, `shift` elements past aligned addresses."""

    def __init__(self, stacks, grad=torch.float32, copy=False, shift=0, seed=0):
        self.rng, self.stacks = np.random.default_rng(seed), stacks
        sizes = [c * r * k for c, r, k in stacks]
        total = sum(-(-n // 64) * 64 + 64 for n in sizes) + 64 + shift
        bufs = [torch.full((total,), 77.0, dtype=d, device="cuda") for d in (torch.float32, grad, torch.bfloat16)]
        mask = torch.ones(total, dtype=torch.bool, device="cuda")
        parts, at = [[], [], []], 64 + shift
        for n, shape in zip(sizes, stacks):
            for b, p in zip(bufs, parts):
                p.append(b[at:at + n].view(shape))
            mask[at:at + n] = False
            at += -(-n // 64) * 64 + 64
        self.bufs, self.mask = bufs, mask
        self.params, self.grads, copies = parts
        self.copies = copies if copy else None
        for p in self.params:
            p.copy_(torch.from_numpy(0.05 * self.rng.standard_normal(p.shape)))
        self.new_grads()

    def new_grads(self, scale=1e-2):
        for g in self.grads:
            rows = np.exp(0.4 * self.rng.standard_normal((*g.shape[:2], 1)))
            g.copy_(torch.from_numpy(scale * rows * self.rng.standard_normal(g.shape)))

    def read(self, tensors):
        return [t.float().cpu().numpy().astype(np.float64) for t in tensors]

    def intact(self):
        torch.cuda.synchronize()
        return all(bool((b[self.mask] == 77).all()) for b in self.bufs)


def cut(flat, stacks):
    flat, out, at = flat.cpu().numpy().astype(np.float64), [], 0
    for c, r, k in stacks:
        out.append(flat[at:at + c * r * k].reshape(c, r, k))
        assert (flat[at + c * r * k:at + -(-c * r * k // 32) * 32] == 0).all()
        at += -(-c * r * k // 32) * 32
    assert at == flat.size
    return out


def check_step(net, before, momentum, after, m, lr, mu, nesterov, wd, scales, coef, steps):
    for s, (p0, g, m0, p1, m1) in enumerate(zip(before, net.read(net.grads), momentum, after, m)):
        for i in range(len(p0)):
            want, mw, o = to.muon(p0[i], g[i], m0[i], lr, mu, nesterov, wd, scales[s], coef, steps)
            assert (np.abs(m1[i] - mw) <= 4 * U * (mu * np.abs(m0[i]) + np.abs(coef * g[i]))).all()
            u = coef * g[i] + mu * mw if nesterov else mw
            rough = np.linalg.norm(to.newton_schulz_fp16(u, steps) - o)
            bar = 3 * rough + 5.0 ** steps * 2.0 ** -21 * np.linalg.norm(o)
            off = np.linalg.norm(p1[i] - want)
            assert off <= lr * scales[s] * bar + 4 * U * (np.linalg.norm(p0[i]) + np.linalg.norm(want)), (net.stacks[s], off)


def rms(stacks):
    return [float(np.float32(0.2 * max(r, k) ** 0.5)) for _, r, k in stacks]


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift,nesterov,steps", [(0, True, 5), (1, False, 5), (3, True, 1), (0, False, 2)])
@pytest.mark.parametrize("stacks", LISTS)
def test_steps(grad, shift, nesterov, steps, stacks):
    stacks = LISTS[stacks]
    net = Net(stacks, grad, copy=True, shift=shift, seed=1)
    lr, mu, wd = (float(np.float32(v)) for v in (0.05, 0.9, 0.1))
    opt = train.Muon(net.params, net.grads, lr=lr, momentum=mu, nesterov=nesterov, weight_decay=wd, steps=steps, copies=net.copies)
    opt.work.fill_(0xff)                                        # whatever the workspace held: fp16 NaN here
    for k in range(3):
        net.new_grads()
        coef = float(np.float32(0.7)) if k == 1 else 1.0
        opt.coef.fill_(coef)
        before, m0 = net.read(net.params), cut(opt.m, stacks)
        opt.step()
        check_step(net, before, m0, net.read(net.params), cut(opt.m, stacks), lr, mu, nesterov, wd, rms(stacks), coef, steps)
        for p, c in zip(net.params, net.copies):
            assert torch.equal(c, p.to(torch.bfloat16))
        assert net.intact() and opt.step_count.item() == k + 1


@pytest.mark.parametrize("rows,cols", [(256, 2304), (1024, 300), (512, 512), (384, 4608)])
def test_larger_matrices(rows, cols):
    net = Net([(1, rows, cols)], seed=2)
    opt = train.Muon(net.params, net.grads, lr=0.02, scale=1.0)
    before = net.read(net.params)
    opt.step()
    lr, mu = (float(np.float32(v)) for v in (0.02, 0.95))
    check_step(net, before, [np.zeros((1, rows, cols))], net.read(net.params), cut(opt.m, net.stacks), lr, mu, True, 0.0, [1.0], 1.0, 5)


@pytest.mark.parametrize("rank,noise", [(4, 0.1), (1, 0.0), (30, 1e-4)])
def test_gradients_of_low_rank(rank, noise):
    rng = np.random.default_rng(3)
    net = Net([(1, 96, 160)], seed=3)
    g = rng.standard_normal((96, rank)) @ rng.standard_normal((rank, 160)) + noise * rng.standard_normal((96, 160))
    net.grads[0].copy_(torch.from_numpy(g[None]))
    net.params[0].zero_()
    opt = train.Muon(net.params, net.grads, lr=1.0, nesterov=False, scale=1.0)
    opt.step()
    o = to.newton_schulz(net.read(net.grads)[0][0])
    rough = np.linalg.norm(to.newton_schulz_fp16(net.read(net.grads)[0][0]) - o)
    assert np.linalg.norm(-net.read(net.params)[0][0] - o) <= 3 * rough + 5.0 ** 5 * 2.0 ** -21 * np.linalg.norm(o)


def test_singular_values():
    net = Net([(1, 100, 400)], seed=4)
    net.params[0].zero_()
    train.Muon(net.params, net.grads, lr=1.0, scale=1.0).step()
    s = np.linalg.svd(net.read(net.params)[0][0], compute_uv=False)
    # p maps [0.02, 1] into [0.68, 1.21] in five steps; a random matrix's singular values start above that
    assert s.min() > 0.65 and s.max() < 1.22


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e15, 1e30])
def test_gradients_of_any_size(size):
    """X = u / (|u| + eps): the same matrix whatever the gradient's size, and a smaller one as eps meets it."""
    net = Net([(2, 40, 72)], seed=5)
    net.new_grads(size)
    net.params[0].zero_()
    opt = train.Muon(net.params, net.grads, lr=1.0, nesterov=False, scale=1.0, eps=float(np.float32(1e-12)))
    opt.step()
    for i in range(2):
        u = net.read(net.grads)[0][i]
        o = to.newton_schulz(u, eps=float(np.float32(1e-12)))
        rough = np.linalg.norm(to.newton_schulz_fp16(u, eps=float(np.float32(1e-12))) - o)
        # below eps X keeps fp16's absolute step of 2^-25, times 2^-15, in every element
        tiny = 3.4445 ** 5 * 2.0 ** -50 * 54
        assert np.linalg.norm(-net.read(net.params)[0][i] - o) <= 3 * rough + 5.0 ** 5 * 2.0 ** -21 * np.linalg.norm(o) + tiny


def test_zero_gradients_decay_only():
    net = Net([(1, 20, 30), (1, 30, 8)], seed=6)
    for g in net.grads:
        g.zero_()
    before = net.read(net.params)
    opt = train.Muon(net.params, net.grads, lr=0.1, weight_decay=0.5)
    opt.step()
    for a, b in zip(before, net.read(net.params)):
        assert (np.abs(b - a * 0.95) <= 4 * U * np.abs(a)).all()
    assert (opt.m == 0).all()


@pytest.mark.parametrize("stacks", [[(3, 20, 50), (1, 60, 30)], [(3, 20, 50), (1, 60, 30), (1, 140, 200)]])
def test_nan_stays_in_its_matrix_and_a_bad_norm_skips_the_step(stacks):
    net = Net(stacks, seed=7)
    net.grads[0][1, 3, 4] = float("nan")
    opt = train.Muon(net.params, net.grads, lr=0.1)
    before = [p.clone() for p in net.params]
    opt.clip(1.0)
    opt.step()
    assert all(torch.equal(a, b) for a, b in zip(before, net.params)) and (opt.m == 0).all()
    assert opt.skipped.item() == 1 and opt.step_count.item() == 0 and opt.nonfinite.item() == 0
    opt.step()
    ok = [torch.isfinite(net.params[0][0]), torch.isfinite(net.params[0][2]), torch.isfinite(net.params[1])]
    assert all(t.all() for t in ok) and torch.isnan(net.params[0][1]).all() and opt.step_count.item() == 1


@pytest.mark.parametrize("stacks", [[(1, 24, 40), (2, 10, 7)], [(1, 24, 40), (1, 200, 65)]])
def test_the_rest_shares_the_control_block(stacks):
    """Clipping over all gradients, Muon for the matrices and AdamW for the rest, as each alone with that factor."""
    def build():
        net, other = Net(stacks, seed=8), Net([(1, 1, 50), (1, 1, 9)], seed=9)
        return net, other, [p.view(-1) for p in other.params], [g.view(-1) for g in other.grads]

    net, other, ps, gs = build()
    rest = train.AdamW(ps, gs, weight_decay=0.01)
    opt = train.Muon(net.params, net.grads, lr=0.01, weight_decay=0.1, rest=rest)
    net2, other2, ps2, gs2 = build()
    alone, adamw = train.Muon(net2.params, net2.grads, lr=0.01, weight_decay=0.1), train.AdamW(ps2, gs2, lr=0.01, weight_decay=0.01)
    for k in range(3):
        for n in (net, other, net2, other2):
            n.new_grads(1.0)
        opt.clip(0.5)
        coef = opt.coef.item()
        assert coef < 1
        opt.step()
        alone.coef.fill_(coef)
        adamw.coef.fill_(coef)
        alone.step()
        adamw.step()
        for a, b in zip(net.params + ps + [opt.m, rest.m, rest.v], net2.params + ps2 + [alone.m, adamw.m, adamw.v]):
            assert torch.equal(a, b)
        assert opt.step_count.item() == k + 1
    # a clip factor serves one step
    opt.step()
    alone.coef.fill_(1.0)
    alone.step()
    assert torch.equal(net.params[0], net2.params[0])
    gs[0][3] = float("inf")                                     # in the rest alone: nothing moves
    before = [t.clone() for t in net.params + ps + [opt.m, rest.m]]
    opt.clip(0.5)
    opt.step()
    assert all(torch.equal(a, b) for a, b in zip(before, net.params + ps + [opt.m, rest.m])) and opt.skipped.item() == 1
    saved = {k: t.clone() for k, t in opt.state().items()}
    assert sorted(saved) == ["m", "rest_m", "rest_v"]
    opt.load_state(7, **saved)
    assert opt.step_count.item() == 7
    with pytest.raises(ValueError):
        opt.load_state(7, m=saved["m"])


def test_same_bits_every_time():
    results = []
    for _ in range(2):
        net = Net([(1, 300, 700), (2, 64, 64), (1, 700, 130)], seed=10)
        opt = train.Muon(net.params, net.grads, lr=0.1)
        for _ in range(2):
            opt.step()
        results.append([p.clone() for p in net.params])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_a_matrix_alone_and_among_others():
    stacks = [(1, 40, 90), (1, 200, 130), (2, 33, 33)]
    net, one = Net(stacks, seed=11), []
    for s in range(3):
        single = Net([stacks[s]], seed=12)
        single.params[0].copy_(net.params[s])
        single.grads[0].copy_(net.grads[s])
        train.Muon(single.params, single.grads, lr=0.1).step()
        one.append(single.params[0])
    train.Muon(net.params, net.grads, lr=0.1).step()
    lengths = [float((a - b).norm() / b.norm()) for a, b in zip(net.params, one)]
    # how a product is shared among workgroups may go by what else there is: 22 bits' rounding, as above
    assert max(lengths) <= 5.0 ** 5 * 2.0 ** -21


@pytest.mark.parametrize("stacks", [[(1, 64, 200), (1, 150, 40)], [(1, 64, 200), (1, 150, 2000), (1, 300, 70)]])
def test_graph_and_streams(stacks):
    net, twin = Net(stacks, seed=13), Net(stacks, seed=13)
    opt, eager = train.Muon(net.params, net.grads, lr=0.1), train.Muon(twin.params, twin.grads, lr=0.1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        opt.clip(1.0)
        opt.step()
    side.synchronize()
    eager.clip(1.0)
    eager.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.clip(1.0)
        opt.step()
    for k in range(4):
        for a, b in zip(net.grads, twin.grads):
            a.copy_(torch.randn(a.shape, generator=torch.Generator().manual_seed(k)).cuda())
            b.copy_(a)
        if k == 2:
            net.grads[0][0, 0, 0] = twin.grads[0][0, 0, 0] = float("nan")
        opt.lr.fill_(0.1 / (k + 1))
        eager.lr.fill_(0.1 / (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        eager.clip(1.0)
        eager.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(net.params + [opt.m], twin.params + [eager.m]))
    assert opt.step_count.item() == eager.step_count.item() == 4 and opt.skipped.item() == 1


def test_refusals():
    net = Net([(1, 8, 12)], seed=14)
    opt = train.Muon(net.params, net.grads)
    lib, o = rc.lib(), opt.options
    import ctypes

    def step(momentum=opt.m.data_ptr(), control=opt.control.data_ptr(), ws=opt.work.data_ptr(), size=opt.work.nbytes, **kw):
        q = rc.TrainMuon(o.momentum, o.eps, o.nesterov, o.steps, o.keep, 0)
        for k, v in kw.items():
            setattr(q, k, v)
        return lib.train_muon_step(opt.matrices.handle, ctypes.byref(q), momentum, control, ws, size, None)

    assert step(momentum=None) == rc.ERR_NULL and step(control=None) == rc.ERR_NULL
    assert step(ws=None) == rc.ERR_WORKSPACE and step(size=opt.work.nbytes - 1) == rc.ERR_WORKSPACE
    assert step(ws=opt.work.data_ptr() + 8) == rc.ERR_WORKSPACE and step(momentum=opt.m.data_ptr() + 4) == rc.ERR_UNSUPPORTED
    for kw in (dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=float("nan")), dict(eps=0.0), dict(eps=1e-40), dict(nesterov=2),
               dict(steps=0), dict(steps=17), dict(keep=2), dict(reserved=1)):
        name, v = next(iter(kw.items()))
        if name == "momentum":
            q = rc.TrainMuon(v, o.eps, 1, 5, 0, 0)
            assert lib.train_muon_step(opt.matrices.handle, ctypes.byref(q), opt.m.data_ptr(), opt.control.data_ptr(), opt.work.data_ptr(),
                                       opt.work.nbytes, None) == rc.ERR_UNSUPPORTED
        else:
            assert step(**kw) == rc.ERR_UNSUPPORTED, kw
    with pytest.raises(ValueError):
        rc.train_muon_step(opt.matrices, o, opt.m[:5], opt.control, opt.work)
    with pytest.raises(ValueError):
        train.Muon(net.params, net.grads, scale="other")


def test_deep_products_and_a_small_matrix_among_them():
    """1600 rows: X's products go by tiles of 256 columns, a matrix of fewer columns than that among them."""
    stacks = [(1, 1600, 1801), (1, 40, 300), (1, 130, 129)]
    net = Net(stacks, seed=5)
    opt = train.Muon(net.params, net.grads, lr=0.02, scale=1.0)
    opt.work.fill_(0xff)
    net.new_grads()
    before, m0 = net.read(net.params), cut(opt.m, stacks)
    opt.step()
    check_step(net, before, m0, net.read(net.params), cut(opt.m, stacks), float(np.float32(0.02)), float(np.float32(0.95)), True, 0.0, [1.0] * 3, 1.0, 5)
    assert net.intact()


def moved_by(p, o, rough, steps):
    """Whether parameters that were 0 moved by the oracle's o (lr and scale 1), within the bars above."""
    return np.linalg.norm(-p - o) <= 3 * rough + 5.0 ** steps * 2.0 ** -21 * np.linalg.norm(o)


LEAST_EPS = float(np.finfo(np.float32).tiny)


@pytest.mark.parametrize("stacks", [[(1, 20, 30), (1, 30, 8)], [(1, 20, 30), (1, 70, 90), (1, 300, 90)]])
@pytest.mark.parametrize("eps", [LEAST_EPS, 1e-36, 9e-35])
def test_zero_gradients_beside_the_smallest_eps(stacks, eps):
    """0 / eps is 0, also where fp32 holds no 2^15 / eps: decay alone."""
    net = Net(stacks, copy=True, seed=6)
    for g in net.grads:
        g.zero_()
    before = net.read(net.params)
    opt = train.Muon(net.params, net.grads, lr=0.1, weight_decay=0.5, eps=eps, copies=net.copies)
    opt.work.fill_(0xff)
    opt.step()
    for a, b in zip(before, net.read(net.params)):
        assert (np.abs(b - a * 0.95) <= 4 * U * np.abs(a)).all()
    assert (opt.m == 0).all() and all(torch.equal(c, p.to(torch.bfloat16)) for c, p in zip(net.copies, net.params))


@pytest.mark.parametrize("shape", [(2, 40, 72), (1, 90, 200), (1, 200, 90)])
@pytest.mark.parametrize("size", [1e-36, 1e-34, 1e37])
def test_gradients_at_the_ends_of_fp32(shape, size):
    net = Net([shape], seed=5)
    net.new_grads(size)
    net.params[0].zero_()
    opt = train.Muon(net.params, net.grads, lr=1.0, nesterov=False, scale=1.0, eps=LEAST_EPS)
    opt.step()
    for u, p in zip(net.read(net.grads)[0], net.read(net.params)[0]):
        o = to.newton_schulz(u, eps=LEAST_EPS)
        assert moved_by(p, o, np.linalg.norm(to.newton_schulz_fp16(u, eps=LEAST_EPS) - o), 5)


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 64, 1024), (1, 128, 2048), (1, 2048, 128)])
def test_norms_whose_reciprocal_is_no_normal_number(shape, grad):
    """Orthogonal rows of elements 1.9 2^127 and their negatives: X's are 2^-8 or 2^-9, which fp16 holds, and so is all that its products add
    up, so that nothing but the norm's reciprocal and the last sums are rounded."""
    net = Net([shape], grad, seed=5)
    signs = hadamard(max(shape))[:shape[1], :shape[2]]
    net.grads[0].copy_(torch.from_numpy(signs * (1.8984375 * 2.0 ** 127))[None])
    net.params[0].zero_()
    opt = train.Muon(net.params, net.grads, lr=1.0, nesterov=False, scale=1.0, steps=1)
    opt.step()
    u = net.read(net.grads)[0][0]
    o = to.newton_schulz(u, 1)
    rough = np.linalg.norm(to.newton_schulz_fp16(u, 1) - o)
    assert rough <= 1e-9 * np.linalg.norm(o) and moved_by(net.read(net.params)[0][0], o, rough, 1)


@pytest.mark.parametrize("shift", [4, 8, 12])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
def test_rows_of_whole_vectors_between_borders(grad, shift):
    """Gradients 4 and 12 elements past a border of 16 bytes, rows of a multiple of eight elements."""
    stacks = [(1, 128, 256), (1, 200, 64), (2, 65, 72), (1, 16, 8)]
    net = Net(stacks, grad, copy=True, shift=shift, seed=15)
    lr, mu = (float(np.float32(v)) for v in (0.05, 0.9))
    opt = train.Muon(net.params, net.grads, lr=lr, momentum=mu, scale=1.0, copies=net.copies)
    opt.work.fill_(0xff)
    for _ in range(2):
        net.new_grads()
        before, m0 = net.read(net.params), cut(opt.m, stacks)
        opt.step()
        check_step(net, before, m0, net.read(net.params), cut(opt.m, stacks), lr, mu, True, 0.0, [1.0] * len(stacks), 1.0, 5)
        assert net.intact()


def test_many_products_of_middling_matrices():
    """90 matrices of 300 x 300: A^2 goes by tiles of 128 from 512 of them on (here 540)."""
    stacks = [(90, 300, 300)]
    net = Net(stacks, seed=16)
    opt = train.Muon(net.params, net.grads, lr=0.02, scale=1.0)
    opt.work.fill_(0xff)
    before, m0 = net.read(net.params), cut(opt.m, stacks)
    opt.step()
    check_step(net, before, m0, net.read(net.params), cut(opt.m, stacks), float(np.float32(0.02)), float(np.float32(0.95)), True, 0.0, [1.0], 1.0, 5)
    assert net.intact()

"""The gradient norm and AdamW over many tensors (include/unettrain.h) against the 64-bit oracle.

Bars.  u = 2^-24.  Norms are summed in 64 bits and rounded once: 2 u.  m, v and the parameter are a few operations, each
rounded once: 4 u of the magnitudes that meet in a sum, and the update 64 u of what it would be if the two terms of m did
not cancel (their rounding stays where they do).  A state in 8 bits starts from the
library's own codes before the step (read back), so the same bars hold up to its rounding, which is checked as the rule
that it is: m is the nearest e4m3 value; s one of the two around it, the upper where the sixteen random bits say so.  A
value within 2^-16 of a step from the point where the rule turns may take either.
"""
import math

import numpy as np
import pytest
import torch

from oracle import train_oracle as to
from paper_2512_08888_amd import binding as rc
from paper_2512_08888_amd import train

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [1, 31, 32, 33, 64, 1000, 1023, 1024, 1025, 4096, 16384, 16385, 70001, 3, 262144]
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8)


def flat_of(parts):
    """The states' layout: every tensor from a multiple of 32 on, zeros between."""
    out = []
    for a in parts:
        out += [a, np.zeros(-a.size % 32, a.dtype)]
    return np.concatenate(out)


class Net:
    """Parameters, gradients and copies of the given sizes inside guarded buffers, `shift` elements past aligned addresses."""

    def __init__(self, sizes, grad=torch.float32, copy=False, shift=0, seed=0):
        self.rng = np.random.default_rng(seed)
        self.sizes, self.grad_dtype = sizes, grad
        gap = 64 + shift
        total = sum(-(-n // 64) * 64 + 64 for n in sizes) + 2 * gap + 64 * len(sizes)
        self.p_buf = torch.full((total,), 77.0, device="cuda")
        self.g_buf = torch.full((total,), 77.0, dtype=grad, device="cuda")
        self.c_buf = torch.full((total,), 77.0, dtype=torch.bfloat16, device="cuda")
        self.params, self.grads, self.copies, self.holes = [], [], [], []
        at = gap
        mask = torch.ones(total, dtype=torch.bool, device="cuda")
        for n in sizes:
            self.params.append(self.p_buf[at:at + n])
            self.grads.append(self.g_buf[at:at + n])
            self.copies.append(self.c_buf[at:at + n])
            mask[at:at + n] = False
            at += -(-n // 64) * 64 + 64
        self.mask = mask
        for p in self.params:
            p.copy_(torch.from_numpy((0.05 * self.rng.standard_normal(p.numel())).astype(np.float32)))
        self.copies = self.copies if copy else None
        self.new_grads()

    def new_grads(self, scale=1e-2):
        for g in self.grads:
            spread = np.exp(1.5 * self.rng.standard_normal(g.numel()))
            g.copy_(torch.from_numpy((scale * spread * self.rng.standard_normal(g.numel())).astype(np.float32)))

    def read(self, tensors):
        return [t.float().cpu().numpy().astype(np.float64) for t in tensors]

    def intact(self):
        torch.cuda.synchronize()
        return all(bool((b[self.mask] == 77).all()) for b in (self.p_buf, self.g_buf, self.c_buf))


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 1])
def test_grad_norm(grad, shift):
    for sizes in (SIZES, [1], [5], [40000], [7] * 300, [3_000_000, 2]):
        net = Net(sizes, grad, shift=shift)
        n = train.GradNorm(net.grads)
        ref = to.grad_norm(net.read(net.grads), 1.0)
        for limit in (math.inf, ref[1] * 2, ref[1] * 0.5):
            n.compute(limit)
            norms, norm, coef = to.grad_norm(net.read(net.grads), limit)
            assert np.all(np.abs(n.norms.cpu().numpy() - norms) <= 2 * U * norms)
            assert abs(n.norm.item() - norm) <= 2 * U * norm and abs(n.coef.item() - coef) <= 4 * U * coef
            assert n.nonfinite.item() == 0 and n.control[6:8].tolist() == [0, 0]
        assert net.intact()


def test_grad_norm_of_extremes():
    net = Net([1000, 5, 40000])
    n = train.GradNorm(net.grads)
    for g in net.grads:
        g.zero_()
    n.compute(1.0)
    assert n.norm.item() == 0 and n.coef.item() == 1 and n.nonfinite.item() == 0
    for scale in (1e30, 1e-30):          # squares beyond fp32 at both ends
        for g in net.grads:
            g.fill_(scale)
        n.compute(1.0)
        ref = scale * math.sqrt(41005)
        assert abs(n.norm.item() / ref - 1) < 1e-6 and abs(n.coef.item() - min(1.0, 1 / ref)) <= 1e-6 * min(1.0, 1 / ref)
        assert n.nonfinite.item() == 0
    for bad in (math.inf, -math.inf, math.nan):
        net.grads[2][39999] = bad
        n.compute(1.0)
        assert n.nonfinite.item() == 1
        net.grads[2][39999] = 0.0
    n.compute(1.0)
    assert n.nonfinite.item() == 0


def check_param(after, ref, before, g, m, v, t, wd, lr):
    """after: the parameters; ref: the oracle's; the others: what went into the step."""
    move = to.adamw(np.zeros_like(before), np.abs(g), np.abs(m), v, t, lr, 0.9, 0.99, 1e-8, 0.0)[0]
    bar = 4 * U * (np.abs(before) * (1 + lr * wd) + np.abs(ref)) + 64 * U * np.abs(move)
    assert np.all(np.abs(after - ref) <= bar)


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("copy", [False, True])
@pytest.mark.parametrize("shift", [0, 1, 2])
def test_adamw_states_in_32_bits(grad, copy, shift):
    net = Net(SIZES, grad, copy, shift)
    decay = [0.1 * (k % 3) for k in range(len(SIZES))]
    opt = train.AdamW(net.params, net.grads, weight_decay=decay, copies=net.copies, **HYPER)
    m = [np.zeros(n) for n in SIZES]
    v = [np.zeros(n) for n in SIZES]
    for t in range(1, 5):
        coef = 1.0 if t % 2 else 0.375
        opt.coef.fill_(coef)
        lr = HYPER["lr"] / t
        opt.lr.fill_(lr)
        lr = opt.lr.item()
        before, g = net.read(net.params), net.read(net.grads)
        opt.step()
        after = net.read(net.params)
        fm, fv = opt.m.cpu().numpy().astype(np.float64), opt.v.cpu().numpy().astype(np.float64)
        rm, rv = [], []
        for k in range(len(SIZES)):
            p, mk, vk = to.adamw(before[k], g[k], m[k], v[k], t, lr, 0.9, 0.99, 1e-8, decay[k], coef)
            check_param(after[k], p, before[k], g[k] * coef, m[k], v[k], t, decay[k], lr)
            rm.append(mk)
            rv.append(vk)
        rm, rv = flat_of(rm), flat_of(rv)
        size = flat_of([np.abs(a) + np.abs(0.1 * b) for a, b in zip(m, g)])
        assert fm.size == rm.size and np.all(np.abs(fm - rm) <= 4 * U * size + 1e-44)
        assert np.all(np.abs(fv - rv) <= 6 * U * rv + 1e-44)
        if copy:
            assert all(torch.equal(c, p.bfloat16()) for c, p in zip(net.copies, net.params))
        assert opt.step_count.item() == t and opt.skipped.item() == 0 and opt.control[6:8].tolist() == [0, 0]
        at = 0
        for k, n in enumerate(SIZES):        # continue from the library's own states
            m[k], v[k] = fm[at:at + n], fv[at:at + n]
            at += -(-n // 32) * 32
        net.new_grads()
    assert net.intact()


def decode(codes, scales):
    c, e = codes.view(torch.uint8).cpu().numpy(), scales.view(torch.uint8).cpu().numpy()
    assert np.all(e != 255)
    return (to.e4m3(c).reshape(-1, 32) * 2.0 ** (e.astype(np.float64) - 127)[:, None]).ravel(), c, e.astype(np.int64) - 127


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("copy,shift", [(False, 0), (True, 1), (True, 0)])
def test_adamw_states_in_8_bits(grad, copy, shift):
    seed = 0xFFFF1234
    net = Net(SIZES, grad, copy, shift)
    opt = train.AdamW(net.params, net.grads, weight_decay=0.1, copies=net.copies, state="mx8", seed=seed, **HYPER)
    assert opt.m.numel() == opt.list.elements and opt.m_scale.numel() == opt.list.elements // 32
    lr = opt.lr.item()
    for t in range(1, 6):
        m0, s0 = decode(opt.m, opt.m_scale)[0], decode(opt.v, opt.v_scale)[0]
        before, g = net.read(net.params), net.read(net.grads)
        opt.step()
        after = net.read(net.params)
        fb, fg = flat_of(before), flat_of(g)
        p, m, v = to.adamw(fb, fg, m0, s0 ** 2, t, lr, 0.9, 0.99, 1e-8, 0.1)
        check_param(flat_of(after), p, fb, fg, m0, s0 ** 2, t, 0.1, lr)
        s = np.sqrt(v)
        real = flat_of([np.ones(n) for n in SIZES]) > 0
        fm, cm, em = decode(opt.m, opt.m_scale)
        fs, cs, es = decode(opt.v, opt.v_scale)
        for exact, e in ((m, em), (s, es)):
            want = to.block_exponents(exact)
            top = np.abs(exact).reshape(-1, 32).max(1)
            edge = np.abs(top / (448 * 2.0 ** np.minimum(e, want)) - 1) < 16 * U       # within rounding of the turn
            assert np.all((e == want) | edge)
        # m: nearest
        unit = np.repeat(2.0 ** em, 32)
        q = m / unit
        step = to.grid_step(q)
        err = np.abs(fm / unit - q) / step
        size = np.repeat(np.abs(m0).reshape(-1, 32).max(1) + 0.1 * np.abs(fg).reshape(-1, 32).max(1), 32)
        assert np.all(err <= 0.5 + 2.0 ** -16 + 8 * U * size / unit / step)
        # s: down or up by the random bits, never to 0
        unit = np.repeat(2.0 ** es, 32)
        q = s / unit
        step = to.grid_step(q)
        u = to.random16(np.arange(q.size), t, seed)
        want = np.where(q > 0, np.maximum(np.floor(q / step + u), 1), 0) * step
        frac = q / step + u
        turn = np.abs(frac - np.round(frac)) < 2.0 ** -15
        got = fs / unit
        assert np.all((got == want) | turn)
        assert np.all(np.abs(got - q) <= np.maximum(step, 2.0 ** -9) * (1 + 2.0 ** -15))
        assert np.all(got[(q > 0) & real] > 0) and np.all(cm[~real] & 127 == 0) and np.all(cs[~real] == 0)
        if copy:
            assert all(torch.equal(c, p.bfloat16()) for c, p in zip(net.copies, net.params))
        assert opt.step_count.item() == t
        net.new_grads()
    assert net.intact()


def test_states_in_8_bits_move_by_changes_below_a_step():
    """v decays by 0.1 % a step where no gradient comes: far below the distance of two codes.  Over 400 steps sqrt(v) has to
    fall to 0.8186 on average (over 2^16 elements of one size, with one in each block held large so that the scale stays);
    each step rounds by at most one code (an eighth) with mean zero, so an element's relative deviation stays below
    sqrt(400 * 0.0005 * 0.125) = 0.16 and the average's below 0.16 / 2^8 * 5 = 0.0031."""
    n = 1 << 16
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    opt = train.AdamW([p], [g], lr=0.0, betas=(0.9, 0.999), state="mx8", seed=5)
    g.fill_(1.0)
    g[::32] = 4.0
    opt.step()
    first = decode(opt.v, opt.v_scale)[0].reshape(-1, 32)[:, 1:].mean()
    g.zero_()
    big = 4.0 * math.sqrt(0.001)
    for _ in range(400):
        g[::32] = big
        opt.step()
    last = decode(opt.v, opt.v_scale)[0].reshape(-1, 32)[:, 1:].mean()
    assert abs(last / first - 0.999 ** 200) < 0.0031 + 0.0031


@pytest.mark.parametrize("state", ["f32", "mx8"])
def test_zero_gradients_and_zero_states_move_nothing(state):
    net = Net([100, 2000])
    for g in net.grads:
        g.zero_()
    opt = train.AdamW(net.params, net.grads, state=state, **HYPER)
    before = [p.clone() for p in net.params]
    for _ in range(3):
        opt.step()
    assert all(torch.equal(a, b) for a, b in zip(before, net.params))
    assert not opt.m.view(torch.uint8).any() and not opt.v.view(torch.uint8).any()


@pytest.mark.parametrize("state", ["f32", "mx8"])
def test_a_step_with_a_gradient_that_is_not_finite_is_skipped(state):
    net = Net([100, 40000, 33])
    opt = train.AdamW(net.params, net.grads, state=state, **HYPER)
    opt.clip(1.0)
    opt.step()
    keep = [t.clone() for t in (*net.params, *opt.state().values())]
    good = net.grads[1][777].clone()
    for bad in (math.nan, math.inf):
        net.grads[1][777] = bad
        opt.clip(1.0)
        opt.step()
    same = lambda: all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(keep, (*net.params, *opt.state().values())))  # noqa: E731
    assert same() and opt.step_count.item() == 1 and opt.skipped.item() == 2 and opt.nonfinite.item() == 0
    net.grads[1][777] = good
    opt.clip(1.0)
    opt.step()
    assert not same() and opt.step_count.item() == 2 and opt.skipped.item() == 2


def test_a_block_with_a_nan_is_marked():
    """Without a clip in front of it a NaN reaches the states: its block reads back as NaN, the others do not."""
    net = Net([320])
    opt = train.AdamW(net.params, net.grads, state="mx8", **HYPER)
    net.grads[0][70] = math.nan
    opt.step()
    for s in (opt.m_scale, opt.v_scale):
        assert (s.view(torch.uint8).cpu().numpy() == 255).tolist() == [k == 2 for k in range(10)]
    p = net.params[0].cpu().numpy()
    assert np.isnan(p[70]) and np.isfinite(np.delete(p, 70)).all()
    opt.step()
    assert np.isnan(net.params[0].cpu().numpy()[64:96]).all() and np.isfinite(net.params[0].cpu().numpy()[:64]).all()


@pytest.mark.parametrize("state", ["f32", "mx8"])
def test_clip_and_step_recorded_in_a_graph(state):
    """Replays of one recorded clip and step against the same calls one by one, with eager work in between."""
    nets = [Net(SIZES, copy=True, seed=3) for _ in range(2)]
    opts = [train.AdamW(n.params, n.grads, copies=n.copies, weight_decay=0.05, state=state, seed=9, **HYPER) for n in nets]
    opts[1].clip(0.5)           # warm up on gradients that the comparison does not use
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        opts[1].clip(0.5)
        opts[1].step()
    for k in range(5):
        for n in nets:
            n.new_grads()
        for o in opts:
            o.lr.fill_(1e-3 / (k + 1))
        torch.cuda.synchronize()
        opts[0].clip(0.5)
        opts[0].step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((nets[0].p_buf, nets[0].c_buf, *opts[0].state().values(), opts[0].control, opts[0].norms),
                        (nets[1].p_buf, nets[1].c_buf, *opts[1].state().values(), opts[1].control, opts[1].norms)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), k
        assert opts[1].step_count.item() == k + 1


def test_saved_states_continue():
    nets = [Net([500, 33], seed=4) for _ in range(2)]
    a = train.AdamW(nets[0].params, nets[0].grads, state="mx8", seed=1, **HYPER)
    b = train.AdamW(nets[1].params, nets[1].grads, state="mx8", seed=1, **HYPER)
    a.step()
    for p, q in zip(nets[0].params, nets[1].params):
        q.copy_(p)
    b.load_state(a.step_count.item(), **a.state())
    a.step()
    b.step()
    assert torch.equal(nets[0].p_buf, nets[1].p_buf) and torch.equal(a.v.view(torch.uint8), b.v.view(torch.uint8))
    for bad in (dict(m=a.m), dict(m=a.m, v=a.v, m_scale=a.m_scale, v_scale=a.v_scale[:-1]), dict(a.state(), m=a.m.float())):
        with pytest.raises(ValueError):
            b.load_state(1, **bad)


def test_refusals_on_the_device():
    net = Net([100])
    opt = train.AdamW(net.params, net.grads)
    norm = train.GradNorm(net.grads)
    L, none = rc.lib(), None

    def code(f, *args, **kw):
        with pytest.raises(rc.RotconvError) as e:
            f(*args, **kw)
        return e.value.status

    for limit in (0.0, -1.0, math.nan):
        assert code(opt.clip, limit) == rc.ERR_UNSUPPORTED
    assert code(rc.train_grad_norm, opt.list, 1.0, none, opt.control, none) == rc.ERR_WORKSPACE
    assert code(rc.train_grad_norm, opt.list, 1.0, none, opt.control, opt.ws[:4]) == rc.ERR_WORKSPACE
    assert code(rc.train_grad_norm, opt.list, 1.0, none, none, opt.ws) == rc.ERR_NULL
    step = lambda o=opt.options, l=opt.list, m=opt.m, v=opt.v, ms=none, vs=none: code(rc.train_adamw_step, l, o, m, v, ms, vs, opt.control)  # noqa: E731
    assert step(l=norm.list) == rc.ERR_UNSUPPORTED                 # a list without parameters
    assert step(m=none) == rc.ERR_NULL and step(ms=opt.ws) == rc.ERR_NULL
    O = rc.TrainAdamW
    for bad in (O(1.0, 0.9, 1e-8, 0, 0, 0), O(-0.1, 0.9, 1e-8, 0, 0, 0), O(0.9, 1.0, 1e-8, 0, 0, 0), O(0.9, 0.9, 0.0, 0, 0, 0),
                O(0.9, 0.9, math.nan, 0, 0, 0), O(0.9, 0.9, 1e-8, 2, 0, 0), O(0.9, 0.9, 1e-8, 0, 0, 1)):
        assert step(o=bad) == rc.ERR_UNSUPPORTED
    assert step(o=O(0.9, 0.9, 1e-8, 1, 0, 0)) == rc.ERR_NULL       # 8 bits without scales
    assert step(m=opt.m[1:]) == rc.ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert opt.step_count.item() == 0


@pytest.mark.parametrize("state", ["f32", "mx8"])
def test_buffers_that_are_too_small_or_elsewhere(state):
    net = Net([100, 7])
    opt = train.AdamW(net.params, net.grads, state=state)
    n = opt.list.elements
    assert n == 160

    def step(**kw):
        a = dict(m=opt.m, v=opt.v, m_scale=opt.m_scale, v_scale=opt.v_scale, control=opt.control)
        a.update(kw)
        rc.train_adamw_step(opt.list, opt.options, *a.values())

    bad = [dict(m=opt.m[:n - 4]), dict(v=opt.v[:n - 4]), dict(m=opt.m.cpu()), dict(control=opt.control[:8])]
    if state == "mx8":
        bad += [dict(m_scale=opt.m_scale[:4]), dict(v_scale=opt.v_scale[1:])]
    for kw in bad:
        with pytest.raises(ValueError):
            step(**kw)
    for norms, control in ((opt.norms[:1], opt.control), (opt.norms, opt.control[:15]), (opt.norms.cpu(), opt.control)):
        with pytest.raises(ValueError):
            rc.train_grad_norm(opt.list, 1.0, norms, control, opt.ws)
    with pytest.raises(ValueError):
        rc.train_control_init(opt.control[:15])
    with pytest.raises(ValueError):
        rc.TrainList([net.grads[0], net.grads[1].cpu()])
    with pytest.raises(rc.RotconvError):                               # an eps whose reciprocal is not finite
        rc.train_adamw_step(opt.list, rc.TrainAdamW(0.9, 0.999, 1e-40, rc.STATES[state], 0, 0), opt.m, opt.v, opt.m_scale, opt.v_scale, opt.control)
    torch.cuda.synchronize()
    assert opt.step_count.item() == 0


def test_offsets_beyond_32_bits():
    """One tensor of more than 2^32 elements, states in 8 bits: its first and last elements against the formula."""
    n = (1 << 32) + 100
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[:5] = 0.5
    g[-5:] = -0.25
    p[-5:] = 1.0
    opt = train.AdamW([p], [g], state="mx8", weight_decay=0.1, **HYPER)
    opt.clip(math.inf)
    opt.step()
    assert abs(opt.norm.item() - math.sqrt(5 * 0.25 + 5 * 0.0625)) < 1e-6
    lr = opt.lr.item()
    for at, x0, grad in ((slice(0, 5), 0.0, 0.5), (slice(n - 5, n), 1.0, -0.25)):
        ref, m, v = to.adamw(np.full(5, x0), np.full(5, grad), np.zeros(5), np.zeros(5), 1, lr, 0.9, 0.99, 1e-8, 0.1)
        assert np.allclose(p[at].cpu().numpy(), ref, rtol=1e-6, atol=1e-9)
        blk = at.start // 32
        unit = 2.0 ** (int(opt.m_scale.view(torch.uint8)[blk]) - 127)
        assert np.all(np.abs(opt.m[at].float().cpu().numpy() * unit - m) <= np.abs(m) / 16)
    assert int(opt.m[5:64].view(torch.uint8).any()) == 0 and float(p[5:n - 5].abs().max()) == 0


# sqrt(v) far from 1: its square is below or above what fp32 holds, sqrt(v) itself is not.
@pytest.mark.parametrize("eps", [2.0 ** -126, 1e-8])
@pytest.mark.parametrize("size", [1e-24, 1e-22, 3e-21, 1e-20, 1e-18, 1e-14, 1e-11, 1.0, 1e9, 1e12, 1e18, 1e21, 1e24, 1e30, 1e37])
def test_8_bit_states_far_from_one(size, eps):
    """Codes and scales of sqrt(v) are those of 64 bits wherever fp32 holds sqrt(v) as a normal number, no finite gradient marks its
    block, no positive sqrt(v) becomes 0, and the parameters move by the formula.  Blocks of one size, of sizes up to 2^20 apart,
    and with a few elements at 0."""
    n, seed, lr = 4096, 17, 1e-3
    rng = np.random.default_rng(3)
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    opt = train.AdamW([p], [g], lr=lr, betas=(0.9, 0.999), eps=eps, state="mx8", seed=seed)
    lr, eps = opt.lr.item(), float(np.float32(eps))
    for t in range(1, 5):
        spread = np.where(np.arange(n) < n // 2, 1.0, 2.0 ** -rng.integers(0, 21, n))
        g.copy_(torch.from_numpy((size * spread * (0.5 + rng.random(n)) * rng.choice([-1.0, 1.0], n)).astype(np.float32)))
        g[5::97] = 0.0
        g64 = g.double().cpu().numpy()
        m0, s0 = decode(opt.m, opt.m_scale)[0], decode(opt.v, opt.v_scale)[0]
        before = p.double().cpu().numpy()
        opt.step()
        ref, m, v = to.adamw(before, g64, m0, s0 ** 2, t, lr, 0.9, 0.999, eps, 0.0)
        s = np.sqrt(v)
        fs, cs, es = decode(opt.v, opt.v_scale)
        assert np.array_equal(es, to.block_exponents(s)) and np.all(cs[s > 0] > 0) and np.all(cs[s == 0] == 0)
        unit = np.repeat(2.0 ** es, 32)
        q = s / unit
        step = to.grid_step(q)
        at = q / step + to.random16(np.arange(n), t, seed)
        want = np.where(q > 0, np.maximum(np.floor(at), 1), 0) * step * unit
        assert np.all((fs == want) | (np.abs(at - np.round(at)) < 2.0 ** -44))
        # the update is lr times a quotient of at most sqrt(1 / (1 - beta2)): 64 u of it with m's terms as magnitudes
        move = to.adamw(np.zeros(n), np.abs(g64), np.abs(m0), s0 ** 2, t, lr, 0.9, 0.999, eps, 0.0)[0]
        assert np.all(np.abs(p.double().cpu().numpy() - ref) <= 4 * U * (np.abs(before) + np.abs(ref)) + 64 * U * np.abs(move))


def test_8_bit_states_at_the_ends_of_the_range():
    """The smallest gradient and the largest: no code of 0 beside a positive sqrt(v), and nothing that is not finite."""
    for size in (2.0 ** -149, 2.0 ** -126, 3.3e38):
        p, g = torch.zeros(64, device="cuda"), torch.full((64,), size, device="cuda")
        opt = train.AdamW([p], [g], lr=1e-3, betas=(0.9, 0.999), eps=2.0 ** -126, state="mx8")
        for _ in range(3):
            opt.step()
            fs, cs, _ = decode(opt.v, opt.v_scale)
            assert np.all(cs > 0) and bool(torch.isfinite(p).all()) and np.isfinite(decode(opt.m, opt.m_scale)[0]).all()


def test_elements_that_vanish_beside_their_block():
    """A positive sqrt(v) 2^-200 times its block's largest: the smallest code."""
    g = torch.full((32,), 2.0 ** -100, device="cuda")
    g[3], g[4] = 2.0 ** 100, 0.0
    opt = train.AdamW([torch.zeros(32, device="cuda")], [g], lr=1e-3, betas=(0.9, 0.999), state="mx8")
    opt.step()
    cs = decode(opt.v, opt.v_scale)[1]
    assert cs[4] == 0 and cs[3] > 1 and np.all(np.delete(cs, [3, 4]) == 1)


@pytest.mark.parametrize("state", ["f32", "mx8"])
def test_a_clip_factor_serves_one_step(state):
    """Steps without a clip behind a clipped one, or behind a skipped one, take their gradients as they are; a factor that the
    caller writes stays until another is written.  A second optimizer that never clips takes the same steps."""
    nets = [Net([100, 2000, 33], seed=5) for _ in range(2)]
    a, b = (train.AdamW(n.params, n.grads, state=state, seed=2, **HYPER) for n in nets)
    same = lambda: torch.equal(nets[0].p_buf, nets[1].p_buf) and all(  # noqa: E731
        torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(a.state().values(), b.state().values()))
    a.clip(0.01)
    coef = a.coef.item()
    assert coef < 0.1
    b.coef.fill_(coef)
    a.step()
    b.step()
    assert same() and a.coef.item() == coef          # still there to be read
    b.coef.fill_(1.0)
    for _ in range(2):
        a.step()
        b.step()
        assert same()
    for bad in (math.nan, math.inf):
        good = nets[0].grads[1][7].clone()
        nets[0].grads[1][7] = bad
        a.clip(0.01)
        a.step()
        nets[0].grads[1][7] = good
        assert a.skipped.item() == (1 if math.isnan(bad) else 2) and same()
        a.step()
        b.step()
        assert same() and a.step_count.item() == b.step_count.item()
    a.clip(math.inf)                                 # measured, not clipped: nothing to take back
    a.step()
    b.step()
    for o in (a, b):
        o.coef.fill_(0.25)
    for _ in range(2):
        a.step()
        b.step()
    assert same() and a.coef.item() == 0.25


def test_a_clip_factor_serves_one_replay():
    """The same where the step alone is recorded and the clip comes from outside, now and then."""
    nets = [Net([100, 2000, 33], seed=5) for _ in range(2)]
    a, b = (train.AdamW(n.params, n.grads, **HYPER) for n in nets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for k in range(6):
        if k % 3 == 1:
            a.clip(0.01)
        b.coef.fill_(a.coef.item() if k % 3 == 1 else 1.0)
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        assert torch.equal(nets[0].p_buf, nets[1].p_buf) and torch.equal(a.v, b.v), k


def test_saved_states_in_32_bits_continue():
    nets = [Net([500, 33], seed=4) for _ in range(2)]
    a, b = (train.AdamW(n.params, n.grads, **HYPER) for n in nets)
    a.step()
    for p, q in zip(nets[0].params, nets[1].params):
        q.copy_(p)
    b.load_state(a.step_count.item(), **{k: t.cpu() for k, t in a.state().items()})
    a.step()
    b.step()
    assert torch.equal(nets[0].p_buf, nets[1].p_buf) and torch.equal(a.m, b.m) and torch.equal(a.v, b.v)


def test_more_elements_than_a_launch_has_threads_for():
    """2^34 elements and two small tensors, states in 8 bits (140 GB): a step of more than 2^24 workgroups.  Both ends, the middle and
    the small tensors against the formula; the step counts once, a skipped one too."""
    n = (1 << 34) + 77
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    small = [torch.zeros(5, device="cuda") for _ in range(2)]
    grads = [torch.full((5,), 0.5, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    opt = train.AdamW([small[0], p, small[1]], [grads[0], g, grads[1]], state="mx8", **HYPER)
    spots = [0, (1 << 33) + 5, (1 << 34) - 2048, n - 5]
    for at in spots:
        g[at:at + 5] = 0.5
    opt.clip(math.inf)
    assert abs(opt.norm.item() - math.sqrt(0.25 * 5 * 6)) < 1e-6
    opt.step()
    lr = opt.lr.item()
    ref, _, _ = to.adamw(np.zeros(5), np.full(5, 0.5), np.zeros(5), np.zeros(5), 1, lr, 0.9, 0.99, 1e-8, 0.0)
    for t in (*small, *(p[at:at + 5] for at in spots)):
        assert np.allclose(t.cpu().numpy(), ref, rtol=1e-6, atol=0)
    assert opt.step_count.item() == 1 and opt.skipped.item() == 0
    g[n - 1] = math.inf
    opt.clip(1.0)
    opt.step()
    assert opt.step_count.item() == 1 and opt.skipped.item() == 1 and np.allclose(small[1].cpu().numpy(), ref, rtol=1e-6, atol=0)
    del p, g, small, grads, opt, t
    torch.cuda.empty_cache()


@pytest.mark.parametrize("state", ["f32", "mx8"])
def test_a_state_that_is_refused_changes_nothing(state):
    net = Net([100, 2000])
    opt = train.AdamW(net.params, net.grads, state=state, **HYPER)
    opt.step()
    opt.step()
    good = {k: t.clone() for k, t in opt.state().items()}
    other = {k: torch.zeros_like(t.view(torch.uint8)).view(t.dtype) for k, t in good.items()}
    last = list(other)[-1]
    for step, s in ((7, {**other, last: other[last][:-1]}), (-1, other), (1 << 31, other), (7, {**other, "more": other[last]})):
        with pytest.raises(ValueError):
            opt.load_state(step, **s)
        assert all(torch.equal(good[k].view(torch.uint8), t.view(torch.uint8)) for k, t in opt.state().items())
        assert opt.step_count.item() == 2

"""Log-probabilities of labels (forward, backward) and the clipped policy loss (include/unettrain.h) against the 64-bit oracle.

Bars, from the order of the operations.  u = 2^-24.  y = z - t and the product in front of exp2 are rounded once each, the
exponential to 2 u: an e_j is off by (3 |y_j| + 4) u.  A row's sums add at most `adds` terms one after the other.  With
S1 = sum p |y| and S2 = sum p y^2:
    s: (3 S1 + 4 + adds) u relative; l: that and 2 u l; h / s: (3 S2 + (9 + 2 adds + 3 S1) S1) u
    p_j: (3 |y_j| + 4) u and s's error, relative
Results add the roundings of their own last operations; a bf16 gradient is rounded once more, by 2^-8 at most.
"""
import numpy as np
import pytest
import torch

from oracle import train_oracle as to
from paper_2512_08888_amd import binding as rc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}
LAYOUTS = ["nchw", "nhwc", "rows"]
# N, K, H, W: few classes, more than a vector, one class, single rows, strips that end inside a vector, many classes
SHAPES = [(2, 6, 8, 12), (1, 1, 1, 1), (3, 2, 5, 7), (2, 9, 6, 6), (1, 16, 16, 9), (2, 17, 4, 8), (1, 64, 3, 5), (2, 65, 7, 3), (3, 300, 5, 4),
          (1, 513, 3, 3), (1, 1025, 1, 2)]
ROWS = [(1, 5), (7, 513), (3, 1020), (2, 1021), (5, 2040), (3, 2049), (2, 4092), (3, 8184), (2, 8185), (2, 16380), (3, 20011), (2, 32768),
        (1, 65528), (2, 65536), (1, 65537), (1, 131072), (2, 131065), (1, 150001)]


def adds(K):
    return 24 + min(K, 160)


def to_rows(t, layout, K):
    t = t.detach().float().cpu().numpy().astype(np.float64)
    return t if layout == "rows" else np.moveaxis(t, 1, -1).reshape(-1, K)


class Case:
    def __init__(self, N, K, H, W, layout, dtype, seed=0, ignored=True):
        rng = np.random.default_rng(seed)
        self.N, self.K, self.P, self.layout, self.dtype = N, K, H * W, layout, dtype
        self.rows = N * H * W
        z = torch.from_numpy(rng.standard_normal((N, K, H, W)).astype(np.float32) * 3 + 1).to(dtype)
        if layout == "rows":
            z = z.permute(0, 2, 3, 1).reshape(-1, K).contiguous()
            self.N, self.P = self.rows, 1
        z = z.cuda()
        self.z = z.contiguous(memory_format=torch.channels_last) if layout == "nhwc" else z.contiguous()
        self.labels = torch.from_numpy(rng.integers(0, K, self.rows).astype(np.int32))
        if ignored and self.rows > 3:
            self.labels[1], self.labels[self.rows - 1] = -1, K
        self.labels = self.labels.cuda()
        self.rng = rng

    def values(self, scale=1.0, per=None):
        return torch.from_numpy((scale * self.rng.standard_normal(per or self.rows)).astype(np.float32)).cuda()

    def read(self, t):
        return to_rows(t, self.layout, self.K)

    def reference(self):
        return to.logp_rows(self.read(self.z), self.labels.cpu().numpy())


def bars(r, K):
    a = adds(K)
    s = (3 * r["s1"] + 4 + a) * U
    l = s + 2 * U * np.abs(r["l"])
    ratio = (3 * r["s2"] + (9 + 2 * a + 3 * r["s1"]) * r["s1"]) * U
    with np.errstate(invalid="ignore"):
        logp = l + 2 * U * np.abs(r["za"] - r["t"]) + U * np.abs(r["logp"])
    return dict(s=s, l=l, logp=logp, ent=l + ratio + 2 * U * (np.abs(r["l"]) + r["s1"]))


def cases(shapes=SHAPES):
    for N, K, H, W in shapes:
        for layout in LAYOUTS:
            yield N, K, H, W, layout
    for N, K in ROWS:
        yield N, K, 1, 1, "rows"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,K,H,W,layout", list(cases()))
def test_forward(N, K, H, W, layout, dtype):
    c = Case(N, K, H, W, layout, dtype, seed=K)
    logp, ent = (torch.full((c.rows,), 7.0, device="cuda") for _ in range(2))
    stat = torch.full((c.rows, 2), 7.0, device="cuda")
    rc.train_logp_fwd(c.z, c.labels, logp, entropy=ent, stat=stat)
    only = torch.full((c.rows,), 7.0, device="cuda")
    rc.train_logp_fwd(c.z, c.labels, only)
    r = c.reference()
    b = bars(r, K)
    got = [t.cpu().numpy().astype(np.float64) for t in (logp, ent, stat)]
    assert (np.abs(got[0] - r["logp"]) <= b["logp"]).all()
    assert (np.abs(got[1] - r["entropy"]) <= b["ent"]).all()
    assert (got[2][:, 0] == np.where(r["has"], r["t"], 0)).all()
    assert (np.abs(got[2][:, 1] - np.where(r["live"], r["l"], 0)) <= b["l"]).all()
    assert (got[0][~r["has"]] == 0).all() and (got[1][~r["has"]] == 0).all()
    assert torch.equal(only, logp)


def gradient_bar(r, K, c1, c2, e1, dtype, dz):
    """Bar of dz for coefficients c1 (off by e1) and c2, both exact in 64 bits."""
    b = bars(r, K)
    y = np.where(r["y"] == -np.inf, 0.0, r["y"])
    rel = (3 * np.abs(y) + 8) * U + (b["s"] + b["l"])[:, None]
    base = np.abs(c1) + np.abs(c2) * (np.abs(r["entropy"]) + np.abs(r["l"]))
    ebase = e1 + np.abs(c2) * (b["ent"] + b["l"]) + 4 * U * base
    inner = base[:, None] + np.abs(c2)[:, None] * np.abs(y)
    bar = r["p"] * (rel * inner + ebase[:, None] + 4 * U * inner) + 2 * U * np.abs(dz)
    own = np.zeros_like(bar)
    np.put_along_axis(own, np.where(r["has"], r["label"], 0)[:, None], (e1 + 2 * U * np.abs(c1))[:, None], 1)
    return (bar + own) * (1 + BF[dtype]) + BF[dtype] * np.abs(dz) + 1e-37


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("N,K,H,W,layout", list(cases(SHAPES[::2])))
def test_backward(N, K, H, W, layout, entropy, dtype):
    c = Case(N, K, H, W, layout, dtype, seed=K + 1)
    r = c.reference()
    r["label"] = c.labels.cpu().numpy()
    logp, ent = (torch.empty(c.rows, device="cuda") for _ in range(2))
    stat = torch.empty(c.rows, 2, device="cuda")
    rc.train_logp_fwd(c.z, c.labels, logp, entropy=ent, stat=stat)
    d1, d2 = c.values(), c.values(0.3)
    if c.rows > 4:
        d1[3] = d2[3] = 0.0
    dz = torch.full_like(c.z, 7.0)
    kw = dict(entropy=ent, dentropy=d2) if entropy else {}
    rc.train_logp_bwd(c.z, c.labels, stat, d1, dz, **kw)
    c1 = d1.cpu().numpy().astype(np.float64) * r["live"]
    c2 = (d2.cpu().numpy().astype(np.float64) if entropy else np.zeros(c.rows)) * r["live"]
    ref = to.logp_gradient(r, r["label"], c1, c2)
    got = c.read(dz)
    assert (np.abs(got - ref) <= gradient_bar(r, K, c1, c2, np.zeros(c.rows), dtype, ref)).all()
    assert (got[~r["live"]] == 0).all() and (c.rows <= 4 or (got[3] == 0).all())
    same = c.z.clone(memory_format=torch.preserve_format)       # in place
    rc.train_logp_bwd(same, c.labels, stat, d1, same, **kw)
    assert torch.equal(same, dz)


def policy_inputs(c, ref=True, per="pixel", weight=True):
    r = c.reference()
    d = 0.2 * c.rng.standard_normal(c.rows)
    for end in (np.log(0.8), np.log(1.25)):                      # no decision within 32 bits' errors
        d = np.where(np.abs(d - end) < 2e-3, d + 5e-3, d)
    f = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731
    a = c.values(1.0, c.rows if per == "pixel" else c.N)
    if c.rows > 6 and per == "pixel":
        a[5] = 0.0
    w = np.abs(c.rng.standard_normal(c.rows)) / c.rows
    if c.rows > 2:
        w[0] = 0.0
    return dict(advantage=a, logp_old=f(r["logp"] - d), logp_ref=f(r["logp"] + 0.4 * c.rng.standard_normal(c.rows)) if ref else None,
                weight=f(w) if weight else None)


def policy_reference(c, a, kl, entropy):
    n = lambda t: None if t is None else t.cpu().numpy().astype(np.float64)  # noqa: E731
    A = n(a["advantage"])
    A = np.repeat(A, c.P) if A.size != c.rows else A
    w = n(a["weight"]) if a["weight"] is not None else np.full(c.rows, float(np.float32(1.0 / c.rows)))
    labels = c.labels.cpu().numpy()
    low, high = float(np.float32(1) - np.float32(0.2)), float(np.float32(1) + np.float32(0.25))
    kl, entropy = float(np.float32(kl)), float(np.float32(entropy))
    out, dz, logp, live, G, ratio, r = to.policy(c.read(c.z), labels, A, n(a["logp_old"]), n(a["logp_ref"]), w, low, high, kl, entropy)
    r["label"] = labels
    return out, dz, logp, live, G, ratio, r, A, w, n(a["logp_old"]), n(a["logp_ref"]), kl, entropy


def check_policy(c, a, kl, entropy, out, dz, logp):
    want, dwant, lwant, live, G, ratio, r, A, w, old, ref, kl, entropy = policy_reference(c, a, kl, entropy)
    b = bars(r, c.K)
    lp = b["logp"] * live
    x = np.exp(np.where(live, ref - r["logp"], 0.0)) if ref is not None and kl else np.zeros(c.rows)
    q = np.abs(np.where(live, ref - r["logp"], 0.0)) if ref is not None and kl else np.zeros(c.rows)
    dist = 2 * U * (np.abs(r["logp"]) + q)                        # of logp - old, ref - logp as they are formed
    er = ratio * np.abs(A) * (lp + dist + 6 * U)
    eG = er + kl * ((x + 1) * (lp + dist + 4 * U))
    assert (np.abs(logp.cpu().numpy() - lwant) <= lp).all()
    eloss = er * 1.3 + kl * ((x + 1) * (lp + dist) + 6 * U * (x + q)) + entropy * b["ent"] + 6 * U * (np.abs(A) * 1.3 * ratio + kl * (x + q) + entropy * r["entropy"])
    ed = (x + 1) * (lp + dist) + 6 * U * (x + q)
    got = out.cpu().numpy().astype(np.float64)
    for k, e in ((0, eloss), (1, ed), (2, b["ent"]), (3, np.zeros(c.rows))):
        assert abs(got[k] - want[k]) <= (w * e)[live].sum() + 2 * U * abs(want[k]) + 1e-37, k
    c1, c2 = np.where(live, w * G, 0.0), np.where(live, -entropy * w, 0.0)
    d = c.read(dz)
    assert (np.abs(d - dwant) <= gradient_bar(r, c.K, c1, c2, w * eG + 3 * U * np.abs(c1), c.dtype, dwant)).all()
    assert (d[~live] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kl,entropy,weight,per", [(0.05, 0.01, True, "pixel"), (0.0, 0.0, False, "image"), (0.5, 0.0, True, "pixel")])
@pytest.mark.parametrize("N,K,H,W,layout", list(cases(SHAPES[::2])))
def test_policy(N, K, H, W, layout, kl, entropy, weight, per, dtype):
    c = Case(N, K, H, W, layout, dtype, seed=K + 2)
    a = policy_inputs(c, kl > 0, per, weight)
    out, logp, dz = torch.full((4,), 7.0, device="cuda"), torch.full((c.rows,), 7.0, device="cuda"), torch.full_like(c.z, 7.0)
    kw = dict(logp_old=a["logp_old"], logp_ref=a["logp_ref"], weight=a["weight"], clip=(0.2, 0.25), kl=kl, entropy=entropy)
    rc.train_policy_loss(c.z, c.labels, a["advantage"], out, dz, logp=logp, **kw)
    check_policy(c, a, kl, entropy, out, dz, logp)
    again = torch.empty(4, device="cuda")
    rc.train_policy_loss(c.z, c.labels, a["advantage"], again, None, **kw)          # the loss alone
    assert torch.equal(again, out)
    same = c.z.clone(memory_format=torch.preserve_format)                            # in place
    rc.train_policy_loss(same, c.labels, a["advantage"], again, same, **kw)
    assert torch.equal(same, dz) and torch.equal(again, out)


SPECIAL = [("nchw", 6), ("nchw", 40), ("nhwc", 6), ("nhwc", 40), ("rows", 300), ("rows", 1500), ("rows", 9000), ("rows", 140000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout,K", SPECIAL)
def test_classes_that_cannot_be_taken(layout, K, dtype):
    """-infinity and the type's lowest value in most classes; a row with no class left; rows left out that hold NaN."""
    c = Case(2, K, 3, 4 if K < 10000 else 1, layout, dtype, seed=K + 3, ignored=False)
    rows = np.arange(c.rows)
    z = c.read(c.z).astype(np.float32)
    z[0, 1:] = -np.inf
    z[0, 0] = 2.0
    z[1, ::2] = torch.finfo(dtype).min
    z[2] = -np.inf
    z[3, :] = np.nan
    z[4, 1:] = np.nan
    labels = c.labels.cpu().numpy().copy()
    labels[0], labels[1], labels[3] = 0, 1, -1
    c.labels = torch.from_numpy(labels).cuda()
    back = torch.from_numpy(z) if layout == "rows" else torch.from_numpy(np.moveaxis(z.reshape(2, *c.z.shape[2:], K), -1, 1).copy())
    c.z.copy_(back.to(dtype))
    logp, ent, stat = torch.empty(c.rows, device="cuda"), torch.empty(c.rows, device="cuda"), torch.empty(c.rows, 2, device="cuda")
    rc.train_logp_fwd(c.z, c.labels, logp, entropy=ent, stat=stat)
    r = c.reference()
    r["label"] = labels
    good = rows[r["live"] & (rows != 4)]
    b = bars(r, K)
    assert (np.abs(logp.cpu().numpy() - r["logp"])[good] <= b["logp"][good]).all()
    lp, en = logp.cpu().numpy(), ent.cpu().numpy()
    assert lp[0] == 0 and en[0] == 0 and lp[2] == 0 and en[2] == 0 and lp[3] == 0 and np.isnan(lp[4]) and np.isnan(en[4])
    assert stat[2, 0].item() == -np.inf and abs(en[1] - r["entropy"][1]) <= b["ent"][1]
    d1, d2 = c.values(), c.values(0.3)
    dz = torch.full_like(c.z, 7.0)
    rc.train_logp_bwd(c.z, c.labels, stat, d1, dz, entropy=ent, dentropy=d2)
    got = c.read(dz)
    assert (got[2] == 0).all() and (got[3] == 0).all() and np.isnan(got[4]).all() and (got[0] == 0).all()
    live = [0, 1] + list(range(5, c.rows))
    sub = {k: v[live] for k, v in r.items()}
    c1, c2 = d1.cpu().numpy().astype(np.float64)[live], d2.cpu().numpy().astype(np.float64)[live]
    ref = to.logp_gradient(sub, sub["label"], c1, c2)
    assert (np.abs(got[live] - ref) <= gradient_bar(sub, K, c1, c2, np.zeros(len(live)), dtype, ref)).all()
    # the loss with those rows left out by their weight
    w = np.ones(c.rows, np.float32) / c.rows
    w[4] = 0
    a = dict(advantage=c.values(), logp_old=torch.from_numpy(np.where(np.isfinite(r["logp"]), r["logp"], 0).astype(np.float32) - 0.1).cuda(),
             logp_ref=None, weight=torch.from_numpy(w).cuda())
    out = torch.empty(4, device="cuda")
    rc.train_policy_loss(c.z, c.labels, a["advantage"], out, dz, logp_old=a["logp_old"], weight=a["weight"], clip=(0.2, 0.25), entropy=0.01,
                         logp=logp)
    assert torch.isfinite(out).all() and torch.isfinite(dz).all()
    got = c.read(dz)
    assert (got[2] == 0).all() and (got[3] == 0).all() and (got[4] == 0).all()
    # a class that cannot be taken, taken all the same: its log-probability is -infinity, its ratio 0
    c.labels[0] = 1
    rc.train_policy_loss(c.z, c.labels, a["advantage"].abs(), out, dz, logp_old=a["logp_old"], weight=a["weight"], logp=logp)
    assert logp[0].item() == -np.inf and torch.isfinite(out).all() and (c.read(dz)[0] == 0).all()


def test_infinite_ratios_and_advantages_of_zero():
    z = torch.tensor([[0.0, 1.0, -1.0]] * 4, device="cuda")
    labels = torch.tensor([0, 1, 2, 0], dtype=torch.int32, device="cuda")
    old = torch.tensor([-1e4, -1e4, -1e4, 0.0], device="cuda")
    out, dz = torch.empty(4, device="cuda"), torch.empty_like(z)
    rc.train_policy_loss(z, labels, torch.tensor([1.0, 0.0, 0.0, 0.0], device="cuda"), out, dz, logp_old=old)
    assert abs(out[0].item() + 1.2 / 4) <= 1e-6 and abs(out[3].item() - 0.25) <= 1e-7 and (dz == 0).all()
    rc.train_policy_loss(z, labels, torch.tensor([-1.0, 0.0, 0.0, 0.0], device="cuda"), out, dz, logp_old=old)
    assert out[0].item() == np.inf


@pytest.mark.parametrize("layout,K", [("nchw", 5), ("nhwc", 20), ("rows", 700)])
def test_gradient_against_differences(layout, K):
    """The loss of perturbed logits, from the library itself, in the direction of a random vector."""
    c = Case(2, K, 3, 3, layout, torch.float32, seed=5)
    a = policy_inputs(c)
    kw = dict(logp_old=a["logp_old"], logp_ref=a["logp_ref"], weight=a["weight"], clip=(0.2, 0.25), kl=0.3, entropy=0.1)
    v = torch.randn(c.z.shape, generator=torch.Generator().manual_seed(3)).cuda()
    v = v.contiguous(memory_format=torch.channels_last) if layout == "nhwc" else v
    out, dz = torch.empty(4, device="cuda"), torch.empty_like(c.z)
    rc.train_policy_loss(c.z, c.labels, a["advantage"], out, dz, **kw)
    ends, h = [], 2e-4          # no ratio crosses a border: they stay 2e-3 away, and v_label - sum p v is below 8
    for s in (h, -h):
        rc.train_policy_loss(c.z + s * v, c.labels, a["advantage"], out, None, **kw)
        ends.append(out[0].item())
    want = (dz.double() * v.double()).sum().item()
    # the losses are of order 1 and off by about 40 u each; the third derivative's part is below h^2 times 30
    assert abs((ends[0] - ends[1]) / (2 * h) - want) <= 40 * U / h + 30 * h * h + 1e-6


def test_unaligned_tensors_and_neighbours_untouched():
    for dtype in (torch.float32, torch.bfloat16):
        for K, T in ((5, 9), (63, 4), (600, 3), (1001, 3), (9001, 2), (140001, 1)):
            n = T * K
            for shift, dshift in ((1, 1), (3, 2), (0, 1)):
                buf = torch.full((n + 16,), 7.0, dtype=dtype, device="cuda")
                z = buf[shift:shift + n].view(T, K)
                c = Case(T, K, 1, 1, "rows", dtype, seed=K)
                z.copy_(c.z)
                dbuf = torch.full((n + 16,), 7.0, dtype=dtype, device="cuda")
                dz, want = dbuf[dshift:dshift + n].view(T, K), torch.empty_like(c.z)
                out, ref = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
                a = c.values()
                rc.train_policy_loss(z, c.labels, a, out, dz, entropy=0.1)
                rc.train_policy_loss(c.z, c.labels, a, ref, want, entropy=0.1)
                # the order in which a row's sums are formed goes by its place: same values within their bars
                assert torch.allclose(dz.float(), want.float(), rtol=2.0 ** -7 if dtype == torch.bfloat16 else 1e-4, atol=1e-7)
                assert torch.allclose(out, ref, rtol=1e-4, atol=1e-6)
                assert (dbuf[:dshift] == 7).all() and (dbuf[dshift + n:] == 7).all()
                assert (buf[:shift] == 7).all() and (buf[shift + n:] == 7).all()


def test_more_rows_than_workgroups():
    for shape, layout in (((9000, 6), "rows"), ((70000, 40), "rows"), ((5000, 600), "rows"), ((4200, 9000), "rows")):
        T, K = shape
        c = Case(T, K, 1, 1, layout, torch.bfloat16, seed=2)
        a = c.values()
        out, dz, logp = torch.empty(4, device="cuda"), torch.empty_like(c.z), torch.empty(T, device="cuda")
        rc.train_policy_loss(c.z, c.labels, a, out, dz, logp=logp, entropy=0.01)
        z = c.z.float()
        lp = torch.log_softmax(z, 1)
        ok = (c.labels >= 0) & (c.labels < K)
        want = torch.where(ok, lp.gather(1, c.labels.long().clamp(0, K - 1)[:, None])[:, 0], 0.0)
        assert (logp - want).abs().max().item() <= 1e-4
        ent = -(lp.exp() * lp).sum(1)
        loss = torch.where(ok, -a.double() - 0.01 * ent.double(), 0.0).sum() / T
        assert abs(out[0].item() - loss.item()) <= 1e-5 * max(1.0, abs(loss.item()))


@pytest.mark.parametrize("layout,K", [("nchw", 6), ("nchw", 30), ("nhwc", 6), ("rows", 5000)])
def test_graph_and_streams(layout, K):
    c = Case(2, K, 8, 8, layout, torch.float32, seed=9)
    a = policy_inputs(c)
    ws = torch.empty(rc.train_logp_workspace_bytes(c.N, K, c.P), dtype=torch.uint8, device="cuda")
    out, dz, logp = torch.empty(4, device="cuda"), torch.empty_like(c.z), torch.empty(c.rows, device="cuda")
    kw = dict(logp_old=a["logp_old"], logp_ref=a["logp_ref"], weight=a["weight"], kl=0.1, entropy=0.1, ws=ws)

    def call():
        rc.train_policy_loss(c.z, c.labels, a["advantage"], out, dz, logp=logp, **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call()
    eager = [t.clone() for t in (out, dz, logp)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for t in (out, dz, logp):
            t.zero_()
        call()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(eager, (out, dz, logp)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        c.z.copy_(torch.randn(c.z.shape, generator=torch.Generator().manual_seed(k)).cuda())
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, dz, logp)]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, (out, dz, logp)))


def test_label_rows_of_a_map_and_of_tokens_agree():
    c = Case(2, 40, 5, 8, "nchw", torch.float32, seed=4)
    rows = c.z.permute(0, 2, 3, 1).reshape(-1, 40).contiguous()
    one, two = torch.empty(c.rows, device="cuda"), torch.empty(c.rows, device="cuda")
    rc.train_logp_fwd(c.z, c.labels, one)
    rc.train_logp_fwd(rows, c.labels, two)
    r = c.reference()
    assert (np.abs(one.cpu().numpy() - two.cpu().numpy()) <= 2 * bars(r, 40)["logp"]).all()


@pytest.mark.parametrize("rows,K,dtype", [(1500, 15000, torch.float32), (1204, 20001, torch.float32), (2200, 16384, torch.float32),
                                          (4400, 16384, torch.bfloat16), (4000, 20011, torch.bfloat16)])
def test_large_logits_give_what_their_parts_do(rows, K, dtype):
    """86 to 152 MiB, which pass the caches by, and 400 rows at a time, which do not: rows know nothing of each other."""
    gen = torch.Generator(device="cuda").manual_seed(K)
    f = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    z = (f(rows, K) * 3).to(dtype)
    labels = torch.randint(0, K, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    labels[7] = -1
    adv, weight, d1, d2, old = f(rows), f(rows).abs(), f(rows), f(rows), f(rows) - 9.0
    empty = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731

    def run(i, j):
        n = j - i
        logp, ent, stat, lp, out = empty(n), empty(n), empty(n, 2), empty(n), empty(4)
        dz, dp = torch.empty_like(z[i:j]), torch.empty_like(z[i:j])
        rc.train_logp_fwd(z[i:j], labels[i:j], logp, entropy=ent, stat=stat)
        rc.train_logp_bwd(z[i:j], labels[i:j], stat, d1[i:j], dz, entropy=ent, dentropy=d2[i:j])
        rc.train_policy_loss(z[i:j], labels[i:j], adv[i:j], out, dp, logp_old=old[i:j], weight=weight[i:j], logp=lp, entropy=0.01)
        return logp, ent, stat, lp, dz, dp

    whole = run(0, rows)
    for i in range(0, rows, 400):
        j = min(i + 400, rows)
        for k, (a, b) in enumerate(zip(whole, run(i, j))):
            assert torch.equal(a[i:j], b), (k, i)


@pytest.mark.parametrize("N,K,P,layout", [(33000, 65536, 1, "rows"), (2, 16, 8192 * 8192, "nchw"), (2, 16, 8192 * 8192, "nhwc"),
                                          (2, 1100, 1024 * 1024, "nchw")])
def test_offsets_past_32_bits(N, K, P, layout):
    """More than 2^31 logits: the last rows (the last image) by themselves give the same bits."""
    gen = torch.Generator(device="cuda").manual_seed(K)
    side = int(P ** 0.5)
    shape = (N, K) if P == 1 else (N, K, side, side) if layout == "nchw" else (N, side, side, K)
    z = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    z = z.permute(0, 3, 1, 2) if layout == "nhwc" else z
    labels = torch.randint(0, K, (N, P), generator=gen, device="cuda", dtype=torch.int32)
    adv, weight = (torch.rand(N, P, generator=gen, device="cuda") for _ in range(2))
    first = N - 200 if P == 1 else 1
    parts = []
    for part in (slice(0, N), slice(first, N)):
        x, at, w = z[part], labels[part], weight[part]
        logp, lp, out = torch.empty_like(w), torch.empty_like(w), torch.empty(4, device="cuda")
        stat = torch.empty(*w.shape, 2, device="cuda")
        dz, dp = torch.empty_like(x), torch.empty_like(x)
        rc.train_logp_fwd(x, at, logp, stat=stat)
        rc.train_logp_bwd(x, at, stat, w, dz)
        rc.train_policy_loss(x, at, adv[part], out, dp, weight=w, logp=lp, entropy=0.01)
        parts.append((logp, lp, stat, dz, dp))
    for a, b in zip(*parts):
        assert torch.equal(a[first:], b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout,K", SPECIAL + [("nchw", 1), ("nhwc", 1), ("rows", 1)])
def test_rows_of_nan_that_have_a_label(layout, K, dtype):
    """NaN everywhere, or beside classes that cannot be taken: log-probability, entropy and gradient are NaN, and a row of -infinity
    alone is left out as it is elsewhere."""
    c = Case(2, K, 3, 4 if K < 10000 else 1, layout, dtype, seed=K + 4, ignored=False)
    z = c.read(c.z).astype(np.float32)
    z[1] = np.nan
    z[2] = -np.inf
    z[3], z[3, K // 2] = -np.inf, np.nan
    z[4], z[4, 0] = -np.inf, np.nan
    labels = c.labels.cpu().numpy().copy()
    labels[4] = 0                                                # a label that is the NaN itself
    labels[3] = K - 1
    c.labels = torch.from_numpy(labels).cuda()
    c.z.copy_((torch.from_numpy(z) if layout == "rows" else torch.from_numpy(np.moveaxis(z.reshape(2, *c.z.shape[2:], K), -1, 1).copy())).to(dtype))
    logp, ent, stat = torch.empty(c.rows, device="cuda"), torch.empty(c.rows, device="cuda"), torch.empty(c.rows, 2, device="cuda")
    rc.train_logp_fwd(c.z, c.labels, logp, entropy=ent, stat=stat)
    nan, rest = [1, 3, 4], [0, 5]
    assert all(torch.isnan(t[nan]).all() for t in (logp, ent, stat[:, 1])) and all(torch.isfinite(t[rest]).all() for t in (logp, ent, stat))
    assert logp[2].item() == 0 and ent[2].item() == 0 and stat[2].tolist() == [-np.inf, 0.0]
    d1, d2 = c.values(), c.values(0.3)
    for kw in ({}, dict(entropy=ent, dentropy=d2)):
        for dz in (torch.full_like(c.z, 7.0), c.z.clone(memory_format=torch.preserve_format)):
            rc.train_logp_bwd(dz if (dz != 7.0).any() else c.z, c.labels, stat, d1, dz, **kw)
            got = c.read(dz)
            assert np.isnan(got[nan]).all() and np.isfinite(got[rest]).all() and (got[2] == 0).all()
    out, dz = torch.empty(4, device="cuda"), torch.full_like(c.z, 7.0)
    rc.train_policy_loss(c.z, c.labels, d1, out, dz, logp=logp, entropy=0.1)
    got = c.read(dz)
    assert np.isnan(got[nan]).all() and np.isfinite(got[rest]).all() and (got[2] == 0).all() and np.isnan(out[0].item())

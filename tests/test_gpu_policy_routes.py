"""Log-probabilities and the policy loss (include/unettrain.h) against the 64-bit oracle where other kernels serve them than for the sizes
of test_gpu_policy.py, whose bars hold here too: more than 128 rows of more than 8192 vectors, which one workgroup takes each, in registers or
read twice, and maps of 2^18 pixels and more, whose lanes take four pixels.

Where a row's sums move to a larger maximum on the way, they are multiplied: with the difference D of a row's largest logit and its smallest,
no thread's sums move by more than D together, (3 D + 5 moves) u more for the bars of test_gpu_policy.py.
"""
import numpy as np
import pytest
import torch

import test_gpu_policy as tp
from paper_2512_08888_amd import binding as rc

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
# rows, classes, type, whether a row is read twice, with a running maximum
ROWS = [(130, 50001, F32, False), (130, 65536, F32, False), (129, 70001, F32, True), (130, 70004, F32, True),
        (130, 100003, BF16, False), (130, 131072, BF16, False), (130, 131080, BF16, True), (129, 150001, BF16, True)]
MAPS = [3, 6, 8, 11, 16, 21, 70]


def check(c, monkeypatch, adds, per):
    """Forward, backward and loss of a case against the oracle; in place; rows of NaN among the others."""
    monkeypatch.setattr(tp, "adds", lambda K: adds)
    r = c.reference()
    r["label"] = c.labels.cpu().numpy()
    b = tp.bars(r, c.K)
    logp, ent = (torch.full((c.rows,), 7.0, device="cuda") for _ in range(2))
    stat = torch.full((c.rows, 2), 7.0, device="cuda")
    rc.train_logp_fwd(c.z, c.labels, logp, entropy=ent, stat=stat)
    got = [t.cpu().numpy().astype(np.float64) for t in (logp, ent, stat)]
    assert (np.abs(got[0] - r["logp"]) <= b["logp"]).all()
    assert (np.abs(got[1] - r["entropy"]) <= b["ent"]).all()
    assert (got[2][:, 0] == np.where(r["has"], r["t"], 0)).all()
    assert (np.abs(got[2][:, 1] - np.where(r["live"], r["l"], 0)) <= b["l"]).all()
    only = torch.full((c.rows,), 7.0, device="cuda")
    rc.train_logp_fwd(c.z, c.labels, only)
    assert torch.equal(only, logp)
    d1, d2 = c.values(), c.values(0.3)
    for kw in (dict(entropy=ent, dentropy=d2), {}):
        dz = torch.full_like(c.z, 7.0)
        rc.train_logp_bwd(c.z, c.labels, stat, d1, dz, **kw)
        c1 = d1.cpu().numpy().astype(np.float64) * r["live"]
        c2 = d2.cpu().numpy().astype(np.float64) * r["live"] * bool(kw)
        want = tp.to.logp_gradient(r, r["label"], c1, c2)
        d = c.read(dz)
        assert (np.abs(d - want) <= tp.gradient_bar(r, c.K, c1, c2, np.zeros(c.rows), c.dtype, want)).all() and (d[~r["live"]] == 0).all()
        same = c.z.clone(memory_format=torch.preserve_format)
        rc.train_logp_bwd(same, c.labels, stat, d1, same, **kw)
        assert torch.equal(same, dz)
    del r, d, want
    losses = []
    for kl, entropy, weight in ((0.05, 0.01, True), (0.0, 0.0, False)):
        a = tp.policy_inputs(c, kl > 0, per, weight)
        kw = dict(logp_old=a["logp_old"], logp_ref=a["logp_ref"], weight=a["weight"], clip=(0.2, 0.25), kl=kl, entropy=entropy)
        out, dz = torch.full((4,), 7.0, device="cuda"), torch.full_like(c.z, 7.0)
        rc.train_policy_loss(c.z, c.labels, a["advantage"], out, dz, logp=logp, **kw)
        tp.check_policy(c, a, kl, entropy, out, dz, logp)
        same, again = c.z.clone(memory_format=torch.preserve_format), torch.empty(4, device="cuda")
        rc.train_policy_loss(same, c.labels, a["advantage"], again, same, **kw)
        assert torch.equal(same, dz) and torch.equal(again, out)
        losses.append((a["advantage"], kw, dz))
    return stat, ent, d1, d2, losses


def nan_rows(c, rows, found):
    """The same calls with NaN in some rows' logits: their results are NaN, and nobody else's change."""
    stat, ent, d1, d2, losses = found
    before = torch.empty_like(c.z)
    rc.train_logp_bwd(c.z, c.labels, stat, d1, before, entropy=ent, dentropy=d2)
    flat = lambda t: t if c.layout == "rows" else t.permute(0, 2, 3, 1).reshape(-1, c.K)  # noqa: E731
    z, mask = c.z.clone(memory_format=torch.preserve_format), torch.zeros(c.rows, dtype=torch.bool, device="cuda")
    for row in rows:
        mask[row] = True
        at = (row,) if c.layout == "rows" else (row // c.P, slice(None), row % c.P // c.z.shape[3], row % c.P % c.z.shape[3])
        z[at] = float("nan") if row % 2 else float("-inf")
        z[at][c.K // 2] = float("nan")
    live = (c.labels >= 0) & (c.labels < c.K)
    assert live[mask].all()
    rc.train_logp_fwd(z, c.labels, torch.empty(c.rows, device="cuda"), entropy=ent, stat=stat)
    dz = torch.full_like(z, 7.0)
    rc.train_logp_bwd(z, c.labels, stat, d1, dz, entropy=ent, dentropy=d2)
    assert torch.isnan(flat(dz)[mask]).all() and torch.equal(flat(dz)[~mask], flat(before)[~mask])
    advantage, kw, want = losses[1]
    out = torch.empty(4, device="cuda")
    rc.train_policy_loss(z, c.labels, advantage, out, dz, **kw)
    assert torch.isnan(flat(dz)[mask]).all() and torch.equal(flat(dz)[~mask], flat(want)[~mask]) and torch.isnan(out[0])


@pytest.mark.parametrize("rows,K,dtype,twice", ROWS)
def test_many_long_rows(rows, K, dtype, twice, monkeypatch):
    c = tp.Case(rows, K, 1, 1, "rows", dtype, seed=K + 5)
    z = c.read(c.z)
    # 1024 threads: a vector each at a time; a tree over lanes and waves
    moves = -(-K // (1024 * (4 if dtype is F32 else 8))) + 1
    own = moves * (4 if dtype is F32 else 8)
    found = check(c, monkeypatch, own + 12 + (3 * (z.max(1) - z.min(1)).max() + 5 * (moves + 1) if twice else 0), "pixel")
    nan_rows(c, [4, 7, rows - 2], found)
    if K % 2:                            # gradients that lie elsewhere in their lines
        stat, ent, d1, d2, losses = found
        advantage, kw, want = losses[0]
        buf = torch.full((rows * K + 16,), 7.0, dtype=dtype, device="cuda")
        dz = buf[1:1 + rows * K].view(rows, K)
        rc.train_policy_loss(c.z, c.labels, advantage, torch.empty(4, device="cuda"), dz, **kw)
        assert torch.equal(dz, want) and buf[0] == 7 and (buf[1 + rows * K:] == 7).all()


@pytest.mark.parametrize("per", ["pixel", "image"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K", MAPS)
def test_large_maps(K, dtype, per, monkeypatch):
    """2 x K x 512 x 256, the smallest whose lanes take four pixels; in strips beyond sixteen classes."""
    c = tp.Case(2, K, 512, 256, "nchw", dtype, seed=K + 6)
    z = c.read(c.z)
    found = check(c, monkeypatch, K + 12 + (3 * (z.max(1) - z.min(1)).max() + 5 * (K // 8 + 5) if K > 16 else 0), per)
    nan_rows(c, [4, 7, 1026, 131072 + 70, c.rows - 2], found)

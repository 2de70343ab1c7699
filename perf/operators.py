"""Workloads of the training operators: group norm with an activation, the gradient norm over many tensors, and the
AdamW step over many tensors, as a training program of the UNet-shaped stack issues them.

Kinds of cases:

  gn_fwd   train_groupnorm_fwd: normalised and activated map, mean and reciprocal deviation of every group
  gn_bwd   train_groupnorm_bwd: gradients of the map, the scale and the shift
  norm     the norm of every parameter's gradient, of all together, and the factor that clips it
  adamw    one AdamW step over all parameters; states in 32 bits, or in 8 bits ("mx8": e4m3 elements, a power-of-two
           scale for each block of 32), with or without a bf16 copy of the parameters

Parameter tensors lie in one buffer, each from a multiple of 32 elements on, so that the plain forms can work on the
whole buffer at once; the library is handed the tensors one by one.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BLOCK = 32                      # elements that share a scale; tensors start on multiples of it
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


# ---- cases ----------------------------------------------------------------------------------------
def _gn(kind, N, C, H, W, G, act, layout, dtype):
    return dict(kind=kind, N=N, C=C, H=H, W=W, G=G, act=act, layout=layout, dtype=dtype)


def _opt(kind, tensors, grad, state="f32", copy=False, **more):
    return dict(kind=kind, tensors=tensors, grad=grad, state=state, copy=copy, **more)


def listed():
    return [
        # one small image's deep map while serving: launches and latency count
        dict(_gn("gn_fwd", 1, 64, 16, 16, 8, "relu", "nchw", "f32"), name="fwd_tile_f32"),
        # the second encoder level of the benchmark's stack, mixed precision
        dict(_gn("gn_fwd", 4, 128, 256, 256, 32, "relu", "nchw", "bf16"), name="fwd_level1_bf16"),
        # the first level at full resolution in 32 bits: the largest map of the stack, larger than the caches
        dict(_gn("gn_fwd", 4, 64, 512, 512, 32, "relu", "nchw", "f32"), name="fwd_full_f32"),
        # a cropped image held channels last: odd rows, a channel count that fills no vector evenly
        dict(_gn("gn_fwd", 3, 60, 101, 75, 12, "silu", "nhwc", "bf16"), name="fwd_ragged_last_bf16"),
        # backward of the level above the bottleneck: deep channels, small map
        dict(_gn("gn_bwd", 4, 512, 32, 32, 32, "relu", "nchw", "f32"), name="bwd_deep_f32"),
        # backward of a middle level, channels last
        dict(_gn("gn_bwd", 4, 256, 128, 128, 32, "silu", "nhwc", "f32"), name="bwd_level2_last_f32"),
        # backward at full resolution, mixed precision: the largest map again
        dict(_gn("gn_bwd", 4, 64, 512, 512, 32, "relu", "nchw", "bf16"), name="bwd_full_bf16"),
        # clipping before the step: every gradient of the benchmark's stack
        dict(_opt("norm", "unet", "f32"), name="norm_unet_f32"),
        # the same of a small network of odd tensors
        dict(_opt("norm", "drawn", "bf16", count=19, most=20011, pick=7), name="norm_small_bf16"),
        # the step over the benchmark's stack, states in 32 bits, bf16 copies for the next forward
        dict(_opt("adamw", "unet", "f32", copy=True), name="adamw_unet_f32"),
        # the same with states in 8 bits
        dict(_opt("adamw", "unet", "f32", state="mx8"), name="adamw_unet_mx8"),
        # the step over a small network of odd tensors: one launch's latency
        dict(_opt("adamw", "drawn", "bf16", state="mx8", copy=True, count=19, most=20011, pick=3), name="adamw_small_mx8"),
    ]


_MAP = 4 * 64 * 512 * 512        # elements of the largest listed map
_PARAMS = 31_000_000             # at most the elements of the benchmark's stack


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["gn_fwd", "gn_bwd", "gn_fwd", "gn_bwd", "norm", "adamw", "adamw"])
    if kind in ("norm", "adamw"):
        c = _opt(kind, "drawn", rng.choice(["f32", "bf16"]), count=_log(rng, 1, 160), most=_log(rng, 100, 4_000_000),
                 pick=rng.randrange(1 << 20))
        if kind == "adamw":
            c.update(state=rng.choice(["f32", "mx8"]), copy=rng.choice([False, True]))
        return c
    while True:
        G, cg = rng.choice([1, 2, 4, 8, 12, 16, 32]), _log(rng, 1, 64)
        N, H, W = _log(rng, 1, 16), _log(rng, 4, 512), _log(rng, 4, 512)
        if G * cg <= 1024 and cg * H * W >= 64 and N * G * cg * H * W <= _MAP // (1 if kind == "gn_fwd" else 2):
            break
    return _gn(kind, N, G * cg, H, W, G, rng.choice(["none", "relu", "silu"]), rng.choice(["nchw", "nhwc"]),
               rng.choice(["f32", "bf16"]))


def _sizes(case):
    """Elements of every parameter, and whether it decays (tensors of one axis, the norms' scales and shifts, do not)."""
    if case["tensors"] == "unet":
        w, out = (64, 128, 256, 512, 1024), []
        blocks = list(zip((3,) + w[:-1], w)) + [(2 * a, a) for a in reversed(w[:-1])]
        for a, b in blocks:
            out += [(9 * a * b, True), (b, False), (b, False), (9 * b * b, True), (b, False), (b, False)]
        return out + [(4 * a * b, True) for a, b in zip(w[1:], w[:-1])] + [(6 * w[0], True)]
    s, out, total = (case["pick"] * 2654435761 + 12345) % 2**32, [], 0
    for _ in range(case["count"]):
        s = (s * 1664525 + 1013904223) % 2**32
        n = max(1, int(case["most"] ** ((s >> 8) / 2**24)))
        if total + n > _PARAMS:
            break
        total += n
        out.append((n, n > 1000))
    return out


def _starts(sizes):
    at, out = 0, []
    for n, _ in sizes:
        out.append(at)
        at += -(-n // _BLOCK) * _BLOCK
    return out, at


def work(case):
    if case["kind"] in ("gn_fwd", "gn_bwd"):
        n, e = case["N"] * case["C"] * case["H"] * case["W"], 2 if case["dtype"] == "bf16" else 4
        if case["kind"] == "gn_fwd":
            return {"bytes": 2 * n * e + 8 * case["C"] + 8 * case["N"] * case["G"], "flops": 10 * n}
        return {"bytes": 3 * n * e + 16 * case["C"] + 8 * case["N"] * case["G"], "flops": 20 * n}
    n, g = sum(k for k, _ in _sizes(case)), 2 if case["grad"] == "bf16" else 4
    if case["kind"] == "norm":
        return {"bytes": n * g, "flops": 2 * n}
    states = 16 if case["state"] == "f32" else 4 + 4 / _BLOCK
    return {"bytes": n * (8 + g + states + (2 if case["copy"] else 0)), "flops": (14 if case["state"] == "f32" else 40) * n}


# ---- inputs ---------------------------------------------------------------------------------------
def _rand(seed, k, *shape):
    gen = torch.Generator(device="cuda").manual_seed(1000 * seed + k)
    return torch.randn(*shape, generator=gen, device="cuda")


def _gn_inputs(case, seed):
    """The map (pooled responses: a mean and a spread of its own for every channel), scale near one, shift near zero."""
    N, C, H, W, G = (case[k] for k in ("N", "C", "H", "W", "G"))
    order = torch.channels_last if case["layout"] == "nhwc" else torch.contiguous_format
    per = (1, C, 1, 1)
    x = _rand(seed, 1, N, C, H, W) * (1 + 0.2 * _rand(seed, 2, *per)) + 0.7 + 0.3 * _rand(seed, 3, *per)
    s = dict(case=case, x=x.to(_DT[case["dtype"]]).contiguous(memory_format=order),
             gamma=1 + 0.1 * _rand(seed, 4, C), beta=0.1 * _rand(seed, 5, C))
    del x
    if case["kind"] == "gn_bwd":
        dy = _rand(seed, 6, N, C, H, W)
        s["dy"] = dy.to(_DT[case["dtype"]]).contiguous(memory_format=order)
        # what the forward kept
        x = s["x"].float().unflatten(1, (G, C // G))
        s["mean"] = x.mean((2, 3, 4))
        s["rstd"] = 1 / torch.sqrt((x - s["mean"][:, :, None, None, None]).square().mean((2, 3, 4)) + 1e-5)
    return s


_HYPER = dict(lr=3e-4, b1=0.9, b2=0.999, eps=1e-8, wd=0.05, seed=77)


def _code_m(m):
    """m in blocks of 32 -> e4m3 elements, e8m0 scales (to nearest)."""
    b = m.view(-1, _BLOCK)
    inv, scale = _scale(b.abs().amax(1))
    return (b * inv[:, None]).to(_E4M3).view(-1), scale


def _scale(top):
    """Smallest power of two 2^e with top <= 448 * 2^e, e within -127..127: its reciprocal, and itself as e8m0."""
    bits = top.view(torch.int32)
    e = ((bits >> 23) - 135 + ((bits & 0x7fffff) > 0x600000).int()).clamp(-127, 127)
    return torch.ldexp(torch.ones_like(top), -e), (e + 127).to(torch.uint8).view(_E8M0)


def _opt_inputs(case, seed):
    sizes = _sizes(case)
    starts, total = _starts(sizes)
    real = torch.zeros(total, device="cuda")
    decay = torch.zeros(total, device="cuda")
    for at, (n, d) in zip(starts, sizes):
        real[at:at + n] = 1
        decay[at:at + n] = _HYPER["wd"] if d else 0.0
    # gradients whose size changes from place to place, as layers' do
    spread = torch.exp(1.5 * _rand(seed, 11, total // _BLOCK)).repeat_interleave(_BLOCK)
    cut = lambda flat: [flat[at:at + n] for at, (n, _) in zip(starts, sizes)]  # noqa: E731
    g = (1e-3 * _rand(seed, 12, total) * spread * real).to(_DT[case["grad"]])
    s = dict(case=case, g=g, grads=cut(g), max_norm=1.0)
    if case["kind"] == "adamw":
        s["p"] = 0.05 * _rand(seed, 13, total) * real
        m = 3e-4 * _rand(seed, 14, total) * spread * real
        v = (1e-3 * spread * real) ** 2 * (0.5 + _rand(seed, 15, total).square())
        if case["state"] == "mx8":
            s["m"], s["m_scale"] = _code_m(m)
            s["v"], s["v_scale"] = _code_m(torch.sqrt(v))
        else:
            s["m"], s["v"] = m, v
        s["copy"] = s["p"].to(torch.bfloat16) if case["copy"] else None
        s["coef"] = torch.full((1,), 0.75, device="cuda") * (1 + 0.1 * torch.rand(1, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
        s["step"], s["decay"], s["params"] = 400, decay, cut(s["p"])
        s["copies"] = cut(s["copy"]) if case["copy"] else None
        s["wds"] = [_HYPER["wd"] if d else 0.0 for _, d in sizes]
        s["position"] = torch.arange(total, device="cuda")
    return s


def prepare(case, seed):
    if case["kind"] in ("gn_fwd", "gn_bwd"):
        s = _gn_inputs(case, seed)
        if own:
            from paper_2512_08888_amd import binding as rc

            N, C, H, W, G = (case[k] for k in ("N", "C", "H", "W", "G"))
            s["rc"] = rc
            s["ws"] = torch.empty(rc.train_groupnorm_workspace_bytes(N, C, H * W, G), dtype=torch.uint8, device="cuda")
            s["y" if case["kind"] == "gn_fwd" else "dx"] = torch.empty_like(s["x"])
            if case["kind"] == "gn_fwd":
                s["mean"], s["rstd"] = (torch.empty(N, G, device="cuda") for _ in range(2))
            else:
                s["dgamma"], s["dbeta"] = (torch.empty(C, device="cuda") for _ in range(2))
        return s
    s = _opt_inputs(case, seed)
    if own:
        from paper_2512_08888_amd import train

        if case["kind"] == "norm":
            s["norm"] = train.GradNorm(s["grads"])
        else:
            h = _HYPER
            s["opt"] = train.AdamW(s["params"], s["grads"], lr=h["lr"], betas=(h["b1"], h["b2"]), eps=h["eps"],
                                   weight_decay=s["wds"], state=case["state"], copies=s["copies"], seed=h["seed"])
            s["opt"].load_state(s["step"], **{k: s[k] for k in ("m", "v", "m_scale", "v_scale") if k in s})
            s["opt"].coef.copy_(s["coef"][0])
    return s


# ---- one pass -------------------------------------------------------------------------------------
def _grouped(t, G):
    return t.float().unflatten(1, (G, t.shape[1] // G))


def _per_channel(t, G):
    return t.view(G, -1, 1, 1)


def _plain_gn_fwd(s):
    c, G = s["case"], s["case"]["G"]
    x = _grouped(s["x"], G)
    mean = x.mean((2, 3, 4), keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean((2, 3, 4), keepdim=True) + 1e-5)
    z = (x - mean) * rstd * _per_channel(s["gamma"], G) + _per_channel(s["beta"], G)
    if c["act"] == "relu":
        z = z.clamp(min=0)
    elif c["act"] == "silu":
        z = z * (1 / (1 + torch.exp(-z)))
    return {"y": z.flatten(1, 2).to(s["x"].dtype), "mean": mean.flatten(1), "rstd": rstd.flatten(1)}


def _plain_gn_bwd(s):
    c, G = s["case"], s["case"]["G"]
    x, dy, gamma = _grouped(s["x"], G), _grouped(s["dy"], G), _per_channel(s["gamma"], G)
    mean, rstd = (s[k][:, :, None, None, None] for k in ("mean", "rstd"))
    xh = (x - mean) * rstd
    z = xh * gamma + _per_channel(s["beta"], G)
    if c["act"] == "relu":
        dy = torch.where(z > 0, dy, 0.0)
    elif c["act"] == "silu":
        sig = 1 / (1 + torch.exp(-z))
        dy = dy * (sig * (1 + z * (1 - sig)))
    dgamma, dbeta = (dy * xh).sum((0, 3, 4)).flatten(), dy.sum((0, 3, 4)).flatten()
    t = dy * gamma
    c1, c2 = t.mean((2, 3, 4), keepdim=True), (t * xh).mean((2, 3, 4), keepdim=True)
    dx = rstd * (t - c1 - xh * c2)
    return {"dx": dx.flatten(1, 2).to(s["x"].dtype), "dgamma": dgamma, "dbeta": dbeta}


def _plain_norm(s):
    squares = torch.stack([g.float().square().sum() for g in s["grads"]])
    total = torch.sqrt(squares.sum())
    return {"norms": torch.sqrt(squares), "norm": total, "coef": torch.clamp(s["max_norm"] / total, max=1.0)}


def _mix(x, key):
    """32 well-mixed bits of each counter x (int64 holding 32-bit values)."""
    low = 0xffffffff
    x = (x + key) & low
    x = ((x ^ (x >> 16)) * 0x9E3779B9) & low
    x = ((x ^ (x >> 15)) * 0x6A09E667) & low
    return x ^ (x >> 16)


def _code_s(q, u):
    """0 <= q <= 448 to e4m3: up with the probability of the part cut off (u: uniform in [0, 1)), never a positive q to 0."""
    step = (((q.view(torch.int32) >> 23).clamp(min=121) - 3) << 23).view(torch.float32)
    n = torch.floor(q / step + u)
    return torch.where(q > 0, n.clamp(min=1), 0.0) * step


def _plain_adamw(s):
    c, h = s["case"], _HYPER
    s["step"] += 1
    t, b1, b2 = s["step"], h["b1"], h["b2"]
    g = s["g"].float() * s["coef"]
    if c["state"] == "mx8":
        m = (s["m"].float().view(-1, _BLOCK) * s["m_scale"].float()[:, None]).view(-1)
        v = (s["v"].float().view(-1, _BLOCK) * s["v_scale"].float()[:, None]).view(-1).square()
    else:
        m, v = s["m"], s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    root = torch.sqrt(v)
    update = m / (root * (1 / math.sqrt(1 - b2 ** t)) + h["eps"])
    p = s["p"]
    p = p - p * (s["decay"] * h["lr"]) - update * (h["lr"] / (1 - b1 ** t))
    if c["state"] == "mx8":
        s["m"], s["m_scale"] = _code_m(m)
        bits = _mix((s["position"] >> 1) & 0xffffffff, (h["seed"] + t * 0x9E3779B9) & 0xffffffff)
        u = torch.where(s["position"] & 1 == 0, bits & 0xffff, bits >> 16).float() * 2.0 ** -16
        inv, s["v_scale"] = _scale(root.view(-1, _BLOCK).amax(1))
        s["v"] = _code_s((root.view(-1, _BLOCK) * inv[:, None]).view(-1), u).to(_E4M3)
    else:
        s["m"], s["v"] = m, v
    s["p"] = p
    if c["copy"]:
        s["copy"] = p.to(torch.bfloat16)
    return _opt_outputs(s)


def _opt_outputs(s):
    return {k: s[k] for k in ("p", "copy", "m", "v", "m_scale", "v_scale") if s.get(k) is not None}


_PLAIN = dict(gn_fwd=_plain_gn_fwd, gn_bwd=_plain_gn_bwd, norm=_plain_norm, adamw=_plain_adamw)


def run(state):
    s = state
    c = s["case"]
    if not own:
        return _PLAIN[c["kind"]](s)
    if c["kind"] == "gn_fwd":
        s["rc"].train_groupnorm_fwd(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], c["G"], eps=1e-5, act=c["act"], ws=s["ws"])
        return {k: s[k] for k in ("y", "mean", "rstd")}
    if c["kind"] == "gn_bwd":
        s["rc"].train_groupnorm_bwd(s["x"], s["dy"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"],
                                    c["G"], act=c["act"], ws=s["ws"])
        return {k: s[k] for k in ("dx", "dgamma", "dbeta")}
    if c["kind"] == "norm":
        n = s["norm"]
        n.compute(s["max_norm"])
        return {"norms": n.norms, "norm": n.norm, "coef": n.coef}
    o = s["opt"]
    o.step()
    return {"p": s["p"], "copy": s["copy"], **o.state()}


# ---- the definition in 64 bits --------------------------------------------------------------------
def _exact_gn(c, s):
    N, C, H, W, G = (c[k] for k in ("N", "C", "H", "W", "G"))
    x = s["x"].contiguous().double().view(N, G, -1)
    per = lambda t: t.double().view(1, C, 1)  # noqa: E731
    if c["kind"] == "gn_fwd":
        var, mean = torch.var_mean(x, 2, unbiased=False, keepdim=True)
        rstd = (var + 1e-5) ** -0.5
    else:
        mean, rstd = s["mean"].double()[..., None], s["rstd"].double()[..., None]
    xh = ((x - mean) * rstd).view(N, C, H * W)
    z = xh * per(s["gamma"]) + per(s["beta"])
    if c["kind"] == "gn_fwd":
        y = {"none": lambda: z, "relu": lambda: torch.relu(z), "silu": lambda: z * torch.sigmoid(z)}[c["act"]]()
        return {"y": y.view(N, C, H, W), "mean": mean[..., 0], "rstd": rstd[..., 0]}
    dz = s["dy"].contiguous().double().view(N, C, H * W)
    if c["act"] == "relu":
        dz = dz * (z > 0)
    elif c["act"] == "silu":
        dz = dz * torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    out = {"dgamma": (dz * xh).sum(2).sum(0), "dbeta": dz.sum(2).sum(0)}
    t, xg = (dz * per(s["gamma"])).view(N, G, -1), xh.view(N, G, -1)
    dx = rstd * (t - t.mean(2, keepdim=True) - xg * (t * xg).mean(2, keepdim=True))
    return {"dx": dx.view(N, C, H, W), **out}


def _exact_codes(x, up=None):
    """x in blocks of 32 as e4m3 multiples of a power of two: (elements, scales), in 64 bits.  up: uniforms of the
    stochastic rounding; without them to nearest, ties to even."""
    x = x.view(-1, _BLOCK)
    top = x.abs().amax(1, keepdim=True)
    e = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)), -127.0).clamp(-127, 127)
    q = x * 2.0 ** -e
    grid = 2.0 ** (torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    n = torch.round(q / grid) if up is None else torch.where(q > 0, torch.floor(q / grid + up.view(-1, _BLOCK)).clamp(min=1), 0.0)
    return (n * grid).view(-1), (2.0 ** e).view(-1)


def _exact_adamw(c, s):
    h, t = _HYPER, s["step"] + 1
    g = s["g"].double() * s["coef"].double()
    m, v = s["m"].double(), s["v"].double()
    if c["state"] == "mx8":
        m = m * s["m_scale"].double().repeat_interleave(_BLOCK)
        v = (v * s["v_scale"].double().repeat_interleave(_BLOCK)) ** 2
    m = h["b1"] * m + (1 - h["b1"]) * g
    v = h["b2"] * v + (1 - h["b2"]) * g ** 2
    p = s["p"].double()
    p = p * (1 - h["lr"] * s["decay"].double()) - h["lr"] * (m / (1 - h["b1"] ** t)) / (torch.sqrt(v / (1 - h["b2"] ** t)) + h["eps"])
    out = {"p": p}
    if c["copy"]:
        out["copy"] = p
    if c["state"] == "f32":
        return {**out, "m": m, "v": v}
    k = torch.arange(p.numel(), device=p.device)
    bits = _mix((k // 2) % 2**32, (h["seed"] + t * 0x9E3779B9) % 2**32)
    out["m"], out["m_scale"] = _exact_codes(m)
    out["v"], out["v_scale"] = _exact_codes(torch.sqrt(v), ((bits // 65536 ** (k % 2)) % 65536).double() / 65536)
    return out


def exact(case, seed):
    if case["kind"] in ("gn_fwd", "gn_bwd"):
        return _exact_gn(case, _gn_inputs(case, seed))
    s = _opt_inputs(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(case, s)
    norms = torch.stack([g.double().norm() for g in s["grads"]])
    return {"norms": norms, "norm": norms.norm(), "coef": torch.clamp(s["max_norm"] / norms.norm(), max=1.0)}

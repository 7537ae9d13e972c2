"""The operators of a diffusion transformer's block, as cases whose time can be measured.

    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program holds before the call (on the GPU)
    run(state)          one pass through one operator, and its outputs
    work(case)          the bytes and operations the pass cannot do without
    exact(case, seed)   run's outputs in 64 bits

Layer norm ahead of a projection, rotary positions with several axes on queries and keys, and projections with bias,
activation and residual; forward as in serving, backward as in training what stands around them.  `own` false: elementary
torch operations; true: this package's kernels.
"""
import math

import torch

own = False

BF16, F32 = torch.bfloat16, torch.float32
TYPES = {"bf16": BF16, "f32": F32}
EPS = 1e-5


def listed():
    return [
        # one time-step or text embedding normalised on its own: latency of a call and of one row
        _case("ln_token", "ln_fwd", M=1, C=1280, x="f32", y="bf16", affine=True, stats=False),
        # the guidance pair's 64 x 64 latent, fp32 residual stream to the bf16 rows of a projection, statistics kept for training
        _case("ln_pair_64x64", "ln_fwd", M=8192, C=1280, x="f32", y="bf16", affine=True, stats=True),
        # the same layer's backward pass: gradient of the bf16 rows in, gradient of the fp32 stream out, with the weights' gradients
        _case("ln_bwd_pair_64x64", "ln_bwd", M=8192, C=1280, x="f32", y="bf16", affine=True),
        # rows of a length that no vector width divides, bf16 throughout, a row count off every tile
        _case("ln_bwd_odd", "ln_bwd", M=2777, C=1155, x="bf16", y="bf16", affine=True),
        # one new token's query and key: latency
        _case("rope_token", "rope_fwd", Bn=1, T=1, Hq=20, Hk=20, D=64, axes="16,16", layout="axis_halves", whole=False, theta=10000.0, x="bf16"),
        # the guidance pair's 64 x 64 latent, height and width, queries and keys out of the rows of one packed projection
        _case("rope_pair_64x64", "rope_fwd", Bn=2, T=4096, Hq=20, Hk=20, D=64, axes="16,16", layout="axis_halves", whole=False, theta=10000.0, x="bf16"),
        # backward through a clip of 13 frames of 26 x 38 latents: time, height, width, fewer key heads than query heads, fp32
        _case("rope_bwd_video", "rope_bwd", Bn=1, T=12844, Hq=24, Hk=8, D=128, axes="16,24,24", layout="interleaved", whole=False, theta=10000.0, x="f32"),
        # one row through the feed-forward's first projection: the time that the weights take to come in
        _case("linear_token", "linear_fwd", M=1, K=1280, N=5120, act="gelu", y="bf16", residual=False, z=False),
        # the feed-forward's first projection of the pair's 64 x 64 latent, as in training: the pre-activation is kept
        _case("linear_pair_64x64", "linear_fwd", M=8192, K=1280, N=5120, act="gelu_tanh", y="bf16", residual=False, z=True),
        # its second projection at 52 x 38, one sample: an uneven number of rows into the fp32 residual stream
        _case("linear_out_52x38", "linear_fwd", M=1976, K=5120, N=1280, act="none", y="f32", residual=True, z=False),
        # the first projection's backward pass for the pair
        _case("linear_bwd_pair_64x64", "linear_bwd", M=8192, K=1280, N=5120, act="gelu_tanh", y="bf16"),
        # a small projection's, on ragged sizes: the reduction over the rows is what little there is to split
        _case("linear_bwd_odd", "linear_bwd", M=1003, K=648, N=317, act="silu", y="bf16"),
    ]


def _case(name, kind, **kw):
    return dict({"name": name, "kind": kind}, **kw)


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["ln_fwd", "ln_bwd", "rope_fwd", "rope_bwd", "linear_fwd", "linear_bwd"])
    if kind.startswith("ln"):
        C = _log(rng, 64, 4096)
        step = rng.choice([1, 2, 4, 8, 64])
        C = C // step * step
        c = {"kind": kind, "M": _log(rng, 1, min(32768, 10485760 // C)), "C": C, "x": rng.choice(["f32", "bf16"]), "y": rng.choice(["bf16", "bf16", "f32"]),
             "affine": rng.random() < 0.8}
        if kind == "ln_fwd":
            c["stats"] = rng.random() < 0.5
        return c
    if kind.startswith("rope"):
        D = rng.choice([32, 40, 64, 72, 80, 88, 96, 128, 256])
        n = rng.choice([1, 2, 2, 3, 3])
        pairs = D // 2 if rng.random() < 0.8 else D // 4
        cut = [pairs * i // n // 4 * 4 for i in range(1, n)]
        if rng.random() < 0.3 or 0 in cut or len(set(cut)) < n - 1:
            cut = sorted(rng.sample(range(1, pairs), n - 1))
        axes = [b - a for a, b in zip([0] + cut, cut + [pairs])]
        Hq = rng.randint(1, 24)
        Hk = rng.choice([0, 1, Hq, max(1, Hq // 4)])
        Bn = rng.choice([1, 2, 2, 3])
        T = _log(rng, 1, min(16384, max(1, 52000000 // (Bn * (Hq + Hk) * D))))
        return {"kind": kind, "Bn": Bn, "T": T, "Hq": Hq, "Hk": Hk, "D": D, "axes": ",".join(str(a) for a in axes),
                "layout": rng.choice(["interleaved", "halves", "axis_halves"]), "whole": rng.random() < 0.3, "theta": rng.choice([100.0, 10000.0, 1000000.0]),
                "x": rng.choice(["bf16", "bf16", "f32"])}
    K = 8 * _log(rng, 8, 640)
    N = _log(rng, 8, 5120)
    if rng.random() < 0.7:
        N = max(8, N // 8 * 8)
    M = _log(rng, 1, min(8192, max(1, 8192 * 1280 * 5120 // (K * N))))
    act = rng.choice(["none", "gelu", "gelu_tanh", "silu", "relu"])
    c = {"kind": kind, "M": M, "K": K, "N": N, "act": act, "y": rng.choice(["bf16", "bf16", "f32"])}
    if kind == "linear_fwd":
        c["residual"] = rng.random() < 0.5
        c["z"] = act != "none" and rng.random() < 0.5
    return c


# ---- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _rows(g, M, C, dtype):
    """A residual stream: rows of different scales and offsets, a few channels far from the others."""
    x = torch.randn(M, C, generator=g, device="cuda")
    x = x * torch.exp(0.5 * torch.randn(M, 1, generator=g, device="cuda")) + 0.5 * torch.randn(M, 1, generator=g, device="cuda")
    return (x + torch.where(torch.rand(C, generator=g, device="cuda") < 0.01, 20.0, 0.0)).to(dtype)


def _positions(g, Bn, T, axes):
    """A grid of frames, rows and columns, in token order, each sample's grid moved a little (a crop of a larger image)."""
    n = len(axes)
    t = torch.arange(T, device="cuda", dtype=torch.float32)
    side = max(1, int(math.ceil(T ** (1.0 / n))))
    pos = torch.stack([torch.div(t, float(side ** (n - 1 - i)), rounding_mode="floor") % side for i in range(n)], dim=-1)
    if n == 1:
        pos = t[:, None]
    return pos[None] + torch.randint(0, 64, (Bn, 1, n), generator=g, device="cuda").float()


def prepare(case, seed):
    g = _gen(seed)
    k = case["kind"]
    s = dict(case)
    if k.startswith("ln"):
        M, C = case["M"], case["C"]
        s["in"] = _rows(g, M, C, TYPES[case["x"]])
        s["gamma"] = (1 + 0.2 * _randn(g, C)).to(BF16) if case["affine"] else None
        s["beta"] = _randn(g, C, dtype=BF16, scale=0.2) if case["affine"] else None
        if k == "ln_bwd":
            # what the forward pass keeps
            x = s["in"].double()
            s["mean"] = x.mean(1).float()
            s["rstd"] = torch.rsqrt(x.var(1, unbiased=False) + EPS).float()
            s["dy"] = _randn(g, M, C, dtype=TYPES[case["y"]])
    elif k.startswith("rope"):
        Bn, T, Hq, Hk, D = (case[n] for n in ("Bn", "T", "Hq", "Hk", "D"))
        axes = [int(a) for a in case["axes"].split(",")]
        # forward: the rows of one packed projection (queries, keys, values); backward: gradients as attention leaves them
        s["packed"] = _randn(g, Bn, T, (Hq + 2 * Hk) * D, dtype=TYPES[case["x"]])
        s["pos"] = _positions(g, Bn, T, axes)
        q, kk = s["packed"][..., :Hq * D].unflatten(-1, (Hq, D)), s["packed"][..., Hq * D:(Hq + Hk) * D].unflatten(-1, (Hk, D)) if Hk else None
        if k == "rope_bwd":
            q, kk = q.contiguous(), kk.contiguous() if Hk else None
            s["packed"] = None
        s["q"], s["k"], s["pairs"] = q, kk, axes
    else:
        M, K, N = case["M"], case["K"], case["N"]
        s["in"] = _randn(g, M, K, dtype=BF16)
        s["W"] = _randn(g, N, K, dtype=BF16, scale=1.0 / math.sqrt(K))
        s["bias"] = _randn(g, N, dtype=BF16, scale=0.5)
        if k == "linear_fwd":
            s["res"] = _randn(g, M, N, dtype=TYPES[case["y"]]) if case["residual"] else None
        else:
            s["zin"] = None if case["act"] == "none" else (s["in"].float() @ s["W"].float().T + s["bias"].float()).to(BF16)
            s["dy"] = _randn(g, M, N, dtype=TYPES[case["y"]])
    return s


# ---- the plain forms
def _ln_fwd(s):
    x = s["in"].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    y = d * rstd
    if s["gamma"] is not None:
        y = y * s["gamma"].float() + s["beta"].float()
    y = y.to(TYPES[s["y"]])
    return (y, mean[:, 0], rstd[:, 0]) if s["stats"] else (y,)


def _ln_bwd(s):
    x, dy, rstd = s["in"].float(), s["dy"].float(), s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    g = dy if s["gamma"] is None else dy * s["gamma"].float()
    dx = (rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))).to(TYPES[s["x"]])
    return (dx,) if s["gamma"] is None else (dx, (dy * xh).sum(0), dy.sum(0))


def _pairing(s, dev):
    """First and second element of every pair, its axis, and its angle per unit of position."""
    axes, total = s["pairs"], sum(s["pairs"])
    i = torch.cat([torch.arange(n, device=dev) for n in axes])
    n = torch.cat([torch.full((a,), a, device=dev) for a in axes])
    ax = torch.cat([torch.full((a,), j, device=dev) for j, a in enumerate(axes)])
    p = torch.arange(total, device=dev)
    if s["layout"] == "interleaved":
        lo, hi = 2 * p, 2 * p + 1
    elif s["layout"] == "halves":
        lo, hi = p, p + total
    else:
        lo = p + (p - i)          # each axis' section begins at twice its first pair
        hi = lo + n
    e = p.double() / total if s["whole"] else i.double() / n
    return lo, hi, ax, s["theta"] ** (-e)


def _rope(s, sign):
    lo, hi, ax, w = _pairing(s, s["q"].device)
    a = s["pos"].double()[..., ax] * w
    c, sn = torch.cos(a).float()[:, :, None], (sign * torch.sin(a)).float()[:, :, None]

    def turn(x):
        f = x.float()
        a, b = f[..., lo], f[..., hi]
        y = f.clone()
        y[..., lo] = a * c - b * sn
        y[..., hi] = a * sn + b * c
        return y.to(x.dtype)
    return (turn(s["q"]),) if s["k"] is None else (turn(s["q"]), turn(s["k"]))


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return torch.clamp(z, min=0) if act == "relu" else z


def _slope(z, act):
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        e = 1 / (1 + torch.exp(-z))
        return e * (1 + z * (1 - e))
    return (z > 0).to(z.dtype)


def _linear_fwd(s):
    z = s["in"].float() @ s["W"].float().T + s["bias"].float()
    y = _act(z, s["act"])
    if s["res"] is not None:
        y = y + s["res"].float()
    y = y.to(TYPES[s["y"]])
    return (y, z.to(BF16)) if s["z"] else (y,)


def _linear_bwd(s):
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _slope(s["zin"].float(), s["act"])
    return (dz @ s["W"].float()).to(BF16), (dz.T @ s["in"].float()).to(BF16), dz.sum(0)


def run(s):
    k = s["kind"]
    if own:
        from paper_2407_02031_amd import binding as B
        if k == "ln_fwd":
            out = B.layernorm_fwd(s["in"], s["gamma"], s["beta"], EPS, out_dtype=TYPES[s["y"]], stats=s["stats"])
            return out if s["stats"] else (out,)
        if k == "ln_bwd":
            return tuple(t for t in B.layernorm_bwd(s["dy"], s["in"], s["mean"], s["rstd"], s["gamma"], weight_grads=s["affine"]) if t is not None)
        if k.startswith("rope"):
            if "rope" not in s:
                s["rope"] = B.Rope(s["D"], s["pairs"], s["theta"], {"interleaved": B.SD_ROPE_INTERLEAVED, "halves": B.SD_ROPE_HALVES, "axis_halves": B.SD_ROPE_AXIS_HALVES}[s["layout"]], whole=s["whole"])
            return tuple(t for t in (B.rope_fwd if k == "rope_fwd" else B.rope_bwd)(s["rope"], s["pos"], s["q"], s["k"]) if t is not None)
        act = {"none": B.SD_ACT_NONE, "gelu": B.SD_ACT_GELU, "gelu_tanh": B.SD_ACT_GELU_TANH, "silu": B.SD_ACT_SILU, "relu": B.SD_ACT_RELU}[s["act"]]
        if k == "linear_fwd":
            out = B.linear_fwd(s["in"], s["W"], s["bias"], act, residual=s["res"], out_dtype=TYPES[s["y"]], save_z=s["z"])
            return out if s["z"] else (out,)
        return B.linear_bwd(s["dy"], s["in"], s["W"], s["zin"], act)
    if k == "ln_fwd":
        return _ln_fwd(s)
    if k == "ln_bwd":
        return _ln_bwd(s)
    if k.startswith("rope"):
        return _rope(s, 1.0 if k == "rope_fwd" else -1.0)
    return _linear_fwd(s) if k == "linear_fwd" else _linear_bwd(s)


def work(case):
    k = case["kind"]
    size = {"bf16": 2, "f32": 4}
    if k.startswith("ln"):
        M, C = case["M"], case["C"]
        if k == "ln_fwd":
            return {"bytes": M * C * (size[case["x"]] + size[case["y"]]) + 4 * C * case["affine"] + 8 * M * case["stats"], "flops": 8 * M * C}
        return {"bytes": M * C * (2 * size[case["x"]] + size[case["y"]]) + 8 * M + 10 * C * case["affine"], "flops": 14 * M * C}
    if k.startswith("rope"):
        rows, n = case["Bn"] * case["T"], len(case["axes"].split(","))
        return {"bytes": 2 * rows * (case["Hq"] + case["Hk"]) * case["D"] * size[case["x"]] + 4 * rows * n, "flops": 3 * rows * (case["Hq"] + case["Hk"]) * case["D"]}
    M, K, N = case["M"], case["K"], case["N"]
    y = size[case["y"]]
    if k == "linear_fwd":
        return {"bytes": 2 * (M * K + N * K + N) + M * N * (y * (1 + case["residual"]) + 2 * case["z"]), "flops": 2 * M * N * K}
    return {"bytes": 4 * (M * K + N * K) + 4 * N + M * N * (y + 2 * (case["act"] != "none")), "flops": 4 * M * N * K}


# ---- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    k = case["kind"]
    if k == "ln_fwd":
        x = s["in"].double()
        m = x.sum(1) / x.shape[1]
        v = ((x - m[:, None]) ** 2).sum(1) / x.shape[1]
        r = (v + EPS) ** -0.5
        y = (x - m[:, None]) * r[:, None]
        if s["gamma"] is not None:
            y = s["beta"].double() + y * s["gamma"].double()
        return (y, m, r) if case["stats"] else (y,)
    if k == "ln_bwd":
        x, dy, m, r = s["in"].double(), s["dy"].double(), s["mean"].double()[:, None], s["rstd"].double()[:, None]
        n = (x - m) * r
        g = dy * s["gamma"].double() if s["gamma"] is not None else dy
        C = x.shape[1]
        dx = r * (g - (g.sum(1, keepdim=True) + n * (g * n).sum(1, keepdim=True)) / C)
        return (dx,) if s["gamma"] is None else (dx, (dy * n).sum(0), dy.sum(0))
    if k.startswith("rope"):
        outs, D, total = [], case["D"], sum(s["pairs"])
        # a complex number per pair, turned by its angle
        first, at, where = 0, 0, []
        for j, n in enumerate(s["pairs"]):
            for i in range(n):
                p = first + i
                lo, hi = {"interleaved": (2 * p, 2 * p + 1), "halves": (p, p + total), "axis_halves": (at + i, at + n + i)}[case["layout"]]
                where.append((lo, hi, j, case["theta"] ** -(p / total if case["whole"] else i / n)))
            first, at = first + n, at + 2 * n
        lo, hi, ax = (torch.tensor([w[c] for w in where], device="cuda") for c in range(3))
        w = torch.tensor([w[3] for w in where], dtype=torch.float64, device="cuda")
        ang = s["pos"].double().index_select(-1, ax) * w
        rot = torch.polar(torch.ones_like(ang), ang if k == "rope_fwd" else -ang)[:, :, None]
        for x in (s["q"], s["k"]):
            if x is not None:
                y = x.double()
                z = torch.complex(y.index_select(-1, lo), y.index_select(-1, hi)) * rot
                outs.append(y.clone().index_copy_(-1, lo, z.real.contiguous()).index_copy_(-1, hi, z.imag.contiguous()))
        return tuple(outs)
    x, W = s["in"].double(), s["W"].double()
    if k == "linear_fwd":
        z = x @ W.T + s["bias"].double()
        y = _exact_act(z, case["act"])
        if s["res"] is not None:
            y = y + s["res"].double()
        return (y, z) if case["z"] else (y,)
    dz = s["dy"].double()
    if case["act"] != "none":
        with torch.enable_grad():
            z = s["zin"].double().requires_grad_(True)
            dz = torch.autograd.grad(_exact_act(z, case["act"]), z, dz)[0]
    return dz @ W, dz.T.contiguous() @ x, dz.sum(0)


def _exact_act(z, act):
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    if act == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z * (z > 0) if act == "relu" else z

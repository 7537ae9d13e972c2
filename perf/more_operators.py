"""The feed-forward of a transformer block in 8 bits and in training, as cases whose time can be measured.

    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program holds before the call (on the GPU)
    run(state)          one pass through one operator, and its outputs
    work(case)          the bytes and operations the pass cannot do without
    exact(case, seed)   run's outputs in 64 bits

Root-mean-square norm with the residual's addition, rows in 8 bits (e4m3, a power of two as the scale of each block of 128), products of such rows, and the gated
feed-forward projection y = (x Wv^T + bv) act(x Wg^T + bg): in 8 bits as in serving, in bf16 with its backward pass as in training.  `own` false: elementary torch operations; true:
this package's kernels.
"""
import math

import torch

own = False

BF16, F32, E4M3, E8M0 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.float8_e8m0fnu
TYPES = {"bf16": BF16, "f32": F32, "fp8": E4M3}
EPS = 1e-6
BLOCK = 128


def listed():
    return [
        # one token's row: the branch's bf16 result onto the fp32 stream, normalised, in 8 bits for the next projection; latency
        _case("rms8_token", "rms_fwd", M=1, C=1280, x="bf16", res="f32", y="fp8", affine=True, stats=False),
        # the same for the guidance pair's 64 x 64 latent
        _case("rms8_pair_64x64", "rms_fwd", M=8192, C=1280, x="bf16", res="f32", y="fp8", affine=True, stats=False),
        # its backward pass in training: the norm's gradient joined with the stream's own, and the weight's gradient
        _case("rms_bwd_pair_64x64", "rms_bwd", M=8192, C=1280, x="f32", y="bf16", dres=True, affine=True),
        # two short rows on their own, a pooled embedding's: latency
        _case("quant_rows", "quant", M=2, C=640, x="bf16"),
        # a gated projection's weights, as when an adapter has been merged and the serving copy is made again
        _case("quant_weight", "quant", M=10240, C=1280, x="bf16"),
        # one token through the feed-forward's second projection, onto the stream: the time that the weights take to come in
        _case("linear8_token", "linear8", M=1, K=5120, N=1280, act="none", y="f32", residual=True),
        # the same projection at 52 x 38, one sample: an uneven number of rows
        _case("linear8_out_52x38", "linear8", M=1976, K=5120, N=1280, act="none", y="f32", residual=True),
        # one token through the gated projection
        _case("gated8_token", "gated8", M=1, K=1280, N=5120, act="silu", y="fp8"),
        # the pair's gated projection in serving: 8 bits in, 8 bits out
        _case("gated8_pair_64x64", "gated8", M=8192, K=1280, N=5120, act="silu", y="fp8"),
        # the same projection in training, its pre-activations kept
        _case("gated_pair_64x64", "gated_fwd", M=8192, K=1280, N=5120, act="silu", y="bf16", z=True),
        # its backward pass
        _case("gated_bwd_pair_64x64", "gated_bwd", M=8192, K=1280, N=5120, act="silu", y="bf16"),
        # a small projection's, on ragged sizes
        _case("gated_bwd_odd", "gated_bwd", M=1003, K=648, N=317, act="gelu_tanh", y="bf16"),
    ]


def _case(name, kind, **kw):
    return dict({"name": name, "kind": kind}, **kw)


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rms_fwd", "rms_bwd", "quant", "linear8", "linear8", "gated8", "gated8", "gated_fwd", "gated_bwd"])
    if kind in ("rms_fwd", "rms_bwd"):
        y = rng.choice(["fp8", "fp8", "bf16", "f32"] if kind == "rms_fwd" else ["bf16", "bf16", "f32"])
        C = _log(rng, 64, 4096)
        step = rng.choice([16, 32, 128] if y == "fp8" else [1, 2, 4, 8, 64])
        C = C // step * step or step
        c = {"kind": kind, "M": _log(rng, 1, min(32768, 10485760 // C)), "C": C, "x": rng.choice(["bf16", "bf16", "f32"]), "y": y, "affine": rng.random() < 0.8}
        if kind == "rms_fwd":
            c["res"] = rng.choice(["none", "f32", "f32", "bf16"] if c["x"] == "bf16" else ["none", "f32"])
            c["stats"] = rng.random() < 0.5
        else:
            c["dres"] = rng.random() < 0.6
        return c
    if kind == "quant":
        C = 16 * _log(rng, 4, 320)
        return {"kind": kind, "M": _log(rng, 1, min(16384, 13107200 // C)), "C": C, "x": rng.choice(["bf16", "bf16", "f32"])}
    act = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu", "none"])
    if kind in ("linear8", "gated8"):
        K = 16 * _log(rng, 4, 320)
        N = _log(rng, 16, 5120)
        if kind == "gated8" or rng.random() < 0.7:
            N = N // 16 * 16
        c = {"kind": kind, "M": _log(rng, 1, min(8192, max(1, 8192 * 1280 * 5120 // (K * N)))), "K": K, "N": N, "act": act}
        if kind == "linear8":
            c["act"] = rng.choice(["none", "none", act])
            c["residual"] = rng.random() < 0.5
            c["y"] = rng.choice(["bf16", "bf16", "f32"])
        else:
            c["y"] = rng.choice(["fp8", "fp8", "bf16", "f32"])
        return c
    K = 8 * _log(rng, 8, 640)
    N = _log(rng, 8, 5120)
    if rng.random() < 0.7:
        N = N // 8 * 8
    c = {"kind": kind, "M": _log(rng, 1, min(8192, max(1, 8192 * 1280 * 5120 // (K * N)))), "K": K, "N": N, "act": act, "y": rng.choice(["bf16", "bf16", "f32"])}
    if kind == "gated_fwd":
        c["z"] = rng.random() < 0.6
    return c


# ---- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _rows(g, M, C, dtype=F32):
    """Rows of different scales, a few channels far from the others."""
    x = torch.randn(M, C, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(M, 1, generator=g, device="cuda"))
    return (x + torch.where(torch.rand(C, generator=g, device="cuda") < 0.01, 20.0, 0.0)).to(dtype)


def _scales_buffer(blocks, rows, device):
    """Scales lie block by block, the rows of each padded to a multiple of 4."""
    return torch.ones(blocks, (rows + 3) // 4 * 4, device=device).to(E8M0)[:, :rows]


def _quantize(x):
    """x [M, K] in fp32 -> e4m3 [M, K] and scales [blocks, M]."""
    M, K = x.shape
    nb = (K + BLOCK - 1) // BLOCK
    p = torch.zeros(M, nb * BLOCK, device=x.device)
    p[:, :K] = x
    p = p.view(M, nb, BLOCK)
    m, e = torch.frexp(p.abs().amax(2))               # amax = m 2^e, 0.5 <= m < 1
    e = torch.where(m > 0.875, e - 8, e - 9)          # 448 = 0.875 * 2^9
    e = torch.where(m == 0, -126, e).clamp(min=-126)
    q = (p * ((127 - e) << 23).view(F32)[..., None]).view(M, nb * BLOCK)[:, :K].to(E4M3)      # by 2^-e, from its bits
    s = _scales_buffer(nb, M, x.device)
    s.view(torch.uint8).copy_((e + 127).to(torch.uint8).T)
    return q, s


def _values(q, s):
    """What e4m3 rows and their scales stand for, in fp32."""
    return q.float() * s.T.float().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def prepare(case, seed):
    g = _gen(seed)
    k = case["kind"]
    s = dict(case)
    if k in ("rms_fwd", "rms_bwd", "quant"):
        M, C = case["M"], case["C"]
        if k == "quant":
            s["in"] = _rows(g, M, C, TYPES[case["x"]])
            return s
        s["gamma"] = (1 + 0.2 * _randn(g, C)).to(BF16) if case["affine"] else None
        if k == "rms_fwd":
            # a branch's result, and the stream it goes onto
            s["in"] = _rows(g, M, C, TYPES[case["x"]]) if case["res"] == "none" else _randn(g, M, C, dtype=TYPES[case["x"]], scale=0.7)
            s["r"] = None if case["res"] == "none" else _rows(g, M, C, TYPES[case["res"]])
        else:
            # what the forward pass keeps
            s["in"] = _rows(g, M, C, TYPES[case["x"]])
            s["rstd"] = torch.rsqrt((s["in"].double() ** 2).mean(1) + EPS).float()
            s["dy"] = _randn(g, M, C, dtype=TYPES[case["y"]])
            s["dr"] = _randn(g, M, C, dtype=TYPES[case["x"]], scale=0.5) if case["dres"] else None
        return s
    M, K, N = case["M"], case["K"], case["N"]
    rows = N if k == "linear8" else 2 * N
    x, W = _randn(g, M, K), _randn(g, rows, K, scale=1.0 / math.sqrt(K))
    s["bias"] = _randn(g, rows, dtype=BF16, scale=0.5)
    if k in ("linear8", "gated8"):
        s["x8"], s["W8"] = _quantize(x), _quantize(W)
        if k == "linear8":
            s["res"] = _randn(g, M, N, dtype=TYPES[case["y"]]) if case["residual"] else None
        return s
    s["in"], s["W"] = x.to(BF16), W.to(BF16)
    if k == "gated_bwd":
        s["zin"] = (s["in"].float() @ s["W"].float().T + s["bias"].float()).to(BF16)
        s["dy"] = _randn(g, M, N, dtype=TYPES[case["y"]])
    return s


# ---- the plain forms
def _rms_fwd(s):
    h = s["in"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    rstd = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    y = h * rstd
    if s["gamma"] is not None:
        y = y * s["gamma"].float()
    out = _quantize(y) if s["y"] == "fp8" else (y.to(TYPES[s["y"]]),)
    if s["r"] is not None:
        out += (h.to(s["r"].dtype),)
    return out + (rstd[:, 0],) if s["stats"] else out


def _rms_bwd(s):
    n, dy, rstd = s["in"].float() * s["rstd"][:, None], s["dy"].float(), s["rstd"][:, None]
    g = dy if s["gamma"] is None else dy * s["gamma"].float()
    dx = rstd * (g - n * (g * n).mean(1, keepdim=True))
    if s["dr"] is not None:
        dx = dx + s["dr"].float()
    dx = dx.to(TYPES[s["x"]])
    return (dx,) if s["gamma"] is None else (dx, (dy * n).sum(0))


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
    return (z > 0).to(z.dtype) if act == "relu" else torch.ones_like(z)


def _linear8(s):
    y = _act(_values(*s["x8"]) @ _values(*s["W8"]).T + s["bias"].float(), s["act"])
    if s["res"] is not None:
        y = y + s["res"].float()
    return (y.to(TYPES[s["y"]]),)


def _gate(z, s):
    N = s["N"]
    return z[:, :N] * _act(z[:, N:], s["act"])


def _gated8(s):
    y = _gate(_values(*s["x8"]) @ _values(*s["W8"]).T + s["bias"].float(), s)
    return _quantize(y) if s["y"] == "fp8" else (y.to(TYPES[s["y"]]),)


def _gated_fwd(s):
    z = s["in"].float() @ s["W"].float().T + s["bias"].float()
    y = _gate(z, s).to(TYPES[s["y"]])
    return (y, z.to(BF16)) if s["z"] else (y,)


def _gated_bwd(s):
    N, dy, z = s["N"], s["dy"].float(), s["zin"].float()
    v, g = z[:, :N], z[:, N:]
    dz = torch.cat([dy * _act(g, s["act"]), dy * v * _slope(g, s["act"])], 1)
    return (dz @ s["W"].float()).to(BF16), (dz.T @ s["in"].float()).to(BF16), dz.sum(0)


def run(s):
    k = s["kind"]
    if own:
        from paper_2407_02031_amd import binding as B
        if k == "rms_fwd":
            out = B.rmsnorm_fwd(s["in"], s["gamma"], EPS, residual=s["r"], out_dtype=TYPES[s["y"]], stats=s["stats"])
            out = out if isinstance(out, tuple) and not isinstance(out, B.Fp8Rows) else (out,)
            return tuple(out[0]) + out[1:] if s["y"] == "fp8" else out
        if k == "rms_bwd":
            return tuple(t for t in B.rmsnorm_bwd(s["dy"], s["in"], s["rstd"], s["gamma"], dres=s["dr"], weight_grad=s["affine"]) if t is not None)
        if k == "quant":
            return tuple(B.quantize_fp8(s["in"]))
        act = {"none": B.SD_ACT_NONE, "gelu": B.SD_ACT_GELU, "gelu_tanh": B.SD_ACT_GELU_TANH, "silu": B.SD_ACT_SILU, "relu": B.SD_ACT_RELU}[s["act"]]
        if k == "linear8":
            return (B.linear_fp8_fwd(B.Fp8Rows(*s["x8"]), B.Fp8Rows(*s["W8"]), s["bias"], act, residual=s["res"], out_dtype=TYPES[s["y"]]),)
        if k == "gated8":
            out = B.gated_linear_fp8_fwd(B.Fp8Rows(*s["x8"]), B.Fp8Rows(*s["W8"]), s["bias"], act, out_dtype=TYPES[s["y"]])
            return tuple(out) if s["y"] == "fp8" else (out,)
        if k == "gated_fwd":
            out = B.gated_linear_fwd(s["in"], s["W"], s["bias"], act, out_dtype=TYPES[s["y"]], save_z=s["z"])
            return out if s["z"] else (out,)
        return B.gated_linear_bwd(s["dy"], s["in"], s["W"], s["zin"], act)
    if k == "quant":
        return _quantize(s["in"].float())
    return {"rms_fwd": _rms_fwd, "rms_bwd": _rms_bwd, "linear8": _linear8, "gated8": _gated8, "gated_fwd": _gated_fwd, "gated_bwd": _gated_bwd}[k](s)


def work(case):
    k = case["kind"]
    size = {"bf16": 2, "f32": 4, "fp8": 1, "none": 0}
    if k in ("rms_fwd", "rms_bwd", "quant"):
        M, C = case["M"], case["C"]
        scales = M * ((C + BLOCK - 1) // BLOCK)
        if k == "quant":
            return {"bytes": M * C * (size[case["x"]] + 1) + scales, "flops": 2 * M * C}
        if k == "rms_fwd":
            return {"bytes": M * C * (size[case["x"]] + 2 * size[case["res"]] + size[case["y"]]) + scales * (case["y"] == "fp8") + 2 * C * case["affine"] + 4 * M * case["stats"], "flops": 5 * M * C}
        return {"bytes": M * C * (size[case["x"]] * (2 + case["dres"]) + size[case["y"]]) + 4 * M + 6 * C * case["affine"], "flops": 9 * M * C}
    M, K, N = case["M"], case["K"], case["N"]
    y = size[case["y"]]
    if k in ("linear8", "gated8"):
        rows, blocks = N if k == "linear8" else 2 * N, (K + BLOCK - 1) // BLOCK
        b = (M + rows) * (K + blocks) + 2 * rows + M * N * y
        b += M * N * y * case["residual"] if k == "linear8" else M * ((N + BLOCK - 1) // BLOCK) * (case["y"] == "fp8")
        return {"bytes": b, "flops": 2 * M * rows * K}
    if k == "gated_fwd":
        return {"bytes": 2 * (M * K + 2 * N * K + 2 * N) + M * N * (y + 4 * case["z"]), "flops": 4 * M * N * K}
    return {"bytes": 4 * (M * K + 2 * N * K) + 8 * N + M * N * (y + 4), "flops": 8 * M * N * K}


# ---- the definitions in 64 bits
def _exact_rows8(y):
    """e4m3 values and scales of rows in 64 bits."""
    def power(e):          # 2^e (a power function may be off by a digit)
        return ((e + 1023).long() << 52).view(torch.float64)
    q, sc = torch.empty(y.shape, device=y.device), torch.empty((y.shape[1] + BLOCK - 1) // BLOCK, y.shape[0], device=y.device)
    for b, part in enumerate(torch.split(y, BLOCK, 1)):
        top = part.abs().amax(1)
        near = torch.floor(torch.log2(top.clamp(min=2.0 ** -130) / 448))      # (a logarithm may round across a whole number)
        e = torch.where(top <= 448 * power(near - 1), near - 1, torch.where(top <= 448 * power(near), near, near + 1)).clamp(min=-126)
        v = part / power(e)[:, None]
        lead = torch.frexp(v).exponent.clamp(min=-5)
        step = power(lead - 4)         # three digits behind the leading one, down to 2^-9
        q[:, b * BLOCK:b * BLOCK + part.shape[1]] = torch.round(v / step) * step
        sc[b] = power(e)
    return q, sc


def _exact_act(z, act):
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    if act == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z * (z > 0) if act == "relu" else z


def _exact_values(q, sc):
    v = q.double()
    for b in range(sc.shape[0]):
        v[:, b * BLOCK:(b + 1) * BLOCK] *= sc[b].double()[:, None]
    return v


def exact(case, seed):
    s = prepare(case, seed)
    k = case["kind"]
    if k == "quant":
        return _exact_rows8(s["in"].double())
    if k == "rms_fwd":
        h = s["in"].double() + (0 if s["r"] is None else s["r"].double())
        r = (h.square().sum(1) / h.shape[1] + EPS) ** -0.5
        y = h * r[:, None] * (1 if s["gamma"] is None else s["gamma"].double())
        out = _exact_rows8(y) if case["y"] == "fp8" else (y,)
        return out + ((h,) if s["r"] is not None else ()) + ((r,) if case["stats"] else ())
    if k == "rms_bwd":
        h, dy, r = s["in"].double(), s["dy"].double(), s["rstd"].double()[:, None]
        g = dy * s["gamma"].double() if s["gamma"] is not None else dy
        dx = g * r - h * (r ** 3 * (g * h).sum(1, keepdim=True) / h.shape[1])
        if s["dr"] is not None:
            dx = dx + s["dr"].double()
        return (dx,) if s["gamma"] is None else (dx, (dy * h * r).sum(0))
    N = case["N"]
    if k in ("linear8", "gated8"):
        z = torch.addmm(s["bias"].double(), _exact_values(*s["x8"]), _exact_values(*s["W8"]).T)
        if k == "linear8":
            y = _exact_act(z, case["act"])
            return (y if s["res"] is None else y + s["res"].double(),)
        y = z[:, :N] * _exact_act(z[:, N:], case["act"])
        return _exact_rows8(y) if case["y"] == "fp8" else (y,)
    x, W = s["in"].double(), s["W"].double()
    if k == "gated_fwd":
        z = torch.addmm(s["bias"].double(), x, W.T)
        y = z[:, :N] * _exact_act(z[:, N:], case["act"])
        return (y, z) if case["z"] else (y,)
    with torch.enable_grad():
        z = s["zin"].double().requires_grad_(True)
        dz = torch.autograd.grad(z[:, :N] * _exact_act(z[:, N:], case["act"]), z, s["dy"].double())[0]
    return dz @ W, dz.T.contiguous() @ x, dz.sum(0)

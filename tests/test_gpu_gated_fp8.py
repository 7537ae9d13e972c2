"""Root-mean-square norm, rows in 8 bits and the gated feed-forward, against their formulas in 64 bits on an MI355X.

Tolerances are bounds: a rounding to the output's type is off by half a step, eps / 2 relative to the value (e4m3: 2^-4, and 2^-10 of the scale below its
normal range); an fp32 operation by U = 2^-24, one that truncates by 2 U; a sum of n terms added up in steps of depth d by d of those times the sum of their absolute values."""
import math

import pytest

from test_gpu_operators import act64, gen, lin_inputs, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_02031_amd import binding
    return binding


def randn(g, *shape, scale=1.0, dtype=None):
    import torch
    x = torch.randn(*shape, generator=g, device="cuda") * scale
    return x if dtype is None else x.to(dtype)


# ---- rows in 8 bits ----------------------------------------------------------------------------------------------------------
def power(e):
    """2^e in 64 bits, from whole numbers"""
    import torch
    return ((e.long() + 1023) << 52).view(torch.float64)


def blocks_of(x):
    """x [M, K] as [M, blocks, 128], zeros behind K"""
    import torch
    M, K = x.shape
    nb = (K + 127) // 128
    return torch.nn.functional.pad(x, (0, nb * 128 - K)).view(M, nb, 128)


def least_scale(amax):
    """e of the least 2^e >= amax / 448, at least -126"""
    import torch
    m, e = torch.frexp(amax)                 # m in [0.5, 1): 448 = 0.875 * 2^9
    return torch.where(amax == 0, -126, e - 9 + (m > 0.875).int()).clamp(min=-126)


def quantized(x):
    """q's values and e of the scales, of x in 64 bits"""
    import torch
    p = blocks_of(x.double())
    fin = torch.where(p.isfinite(), p, 0)
    e = least_scale(fin.abs().amax(2))
    v = fin / power(e)[..., None]
    step = power(torch.frexp(v).exponent.clamp(min=-5) - 4)
    q = torch.where(p.isfinite(), torch.round(v / step) * step, math.nan)
    return q.flatten(1)[:, :x.shape[1]], e


def values(r):
    """What rows in 8 bits stand for"""
    s = r.scales.double().T.repeat_interleave(128, 1)[:, :r.q.shape[1]]
    return r.q.double() * s


def same_rows(got, x):
    import torch
    q, e = quantized(x)
    assert torch.equal(got.scales.double().T, power(e))
    g = got.q.double()
    assert torch.equal(g.isnan(), q.isnan()) and torch.equal(g.nan_to_num(), q.nan_to_num())


@pytest.mark.parametrize("K", [16, 48, 128, 144, 512, 528, 1280, 5120])
@pytest.mark.parametrize("M", [1, 2, 5, 16, 33, 1000])
@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
def test_quantize(B, M, K, dt):
    import torch
    g = gen(M + K)
    x = randn(g, M, K) * torch.exp(2 * randn(g, M, 1))
    x = x.to(getattr(torch, dt))
    got = B.quantize_fp8(x)
    assert got.q.shape == (M, K) and got.scales.shape == ((K + 127) // 128, M)
    same_rows(got, x)


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
def test_quantize_many(B, dt):
    """Blocks in groups of four a wavefront, the last group short; the last workgroup's rows too"""
    import torch
    g = gen(3)
    x = randn(g, 5005, 1936).to(getattr(torch, dt))
    same_rows(B.quantize_fp8(x), x)


def test_quantize_borders(B):
    """Largest elements at and beside 448 2^e, ties, subnormals of e4m3, zeros, the largest and smallest numbers, NaN and infinities."""
    import torch
    x = torch.zeros(24, 256, device="cuda")
    for i, top in enumerate((448.0, 448.0 * (1 + 2.0 ** -23), 447.9, 1.75 * 2.0 ** -40, 1.7500001 * 2.0 ** 60, 3.4028234e38, 2.0 ** -126, 2.0 ** -149, 1.75 * 2.0 ** -118, 1.7500001 * 2.0 ** -118, 2.0 ** -117)):
        x[i, :128] = torch.linspace(-1, 1, 128, device="cuda") * top
        x[i, 5] = top
    x[11] = torch.arange(256, device="cuda") / 16.0                               # ties
    x[12] = torch.arange(256, device="cuda") * 2.0 ** -11 + 2.0 ** -12            # below the normal range of a block that holds 448
    x[12, 0] = x[12, 128] = 448
    x[13, 7], x[14, 200], x[15, 0] = math.inf, -math.inf, math.nan
    x[13:16] += torch.linspace(-3, 5, 256, device="cuda")
    x[16] = math.nan
    x[17, :128] = math.inf
    same_rows(B.quantize_fp8(x), x)
    same_rows(B.quantize_fp8(x.bfloat16()), x.bfloat16())


def test_quantize_into_rows_of_a_larger_result(B):
    """Scales of other rows, and what lies between the last row and the next block, stay as they were."""
    import torch
    g = gen(4)
    q = torch.full((40, 272), 3, dtype=torch.uint8, device="cuda")
    s = torch.full((3, 44), 7, dtype=torch.uint8, device="cuda")
    x = randn(g, 18, 272)
    out = B.Fp8Rows(q[16:34].view(torch.float8_e4m3fn), s[:, 16:34].view(torch.float8_e8m0fnu))
    B.quantize_fp8(x, out=out)
    same_rows(out, x)
    assert (q[:16] == 3).all() and (q[34:] == 3).all() and (s[:, :16] == 7).all() and (s[:, 34:] == 7).all()


# ---- root-mean-square norm ---------------------------------------------------------------------------------------------------
LENGTHS = [4, 5, 63, 64, 65, 128, 129, 255, 257, 320, 321, 511, 513, 768, 769, 1280, 1283, 2048, 2049, 4095, 4096, 5000, 8192, 8193, 16384]
TYPES = [("bfloat16", None), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float32", None), ("float32", "float32")]


def within_fp8(got, y, slack):
    """Rows in 8 bits of something that lies within `slack` of y"""
    import torch
    s = got.scales.double().T
    p, sl = blocks_of(y).abs(), blocks_of(slack)
    lo, hi = least_scale((p - sl).clamp(min=0).amax(2)), least_scale((p + sl).amax(2))
    assert (power(lo) <= s).all() and (s <= power(hi)).all()
    full = s.repeat_interleave(128, 1)[:, :y.shape[1]]
    off = (values(got) - y).abs()
    assert (off <= torch.maximum(2.0 ** -4 * (y.abs() + slack), 2.0 ** -10 * full) + slack).all()


def check_rms_fwd(B, x, r, gamma, yt, eps=1e-6):
    import torch
    fp8 = yt == torch.float8_e4m3fn
    out = B.rmsnorm_fwd(x, gamma, eps, residual=r, out_dtype=yt, stats=True)
    y, rstd = out[0], out[-1]
    h = x.double() + (r.double() if r is not None else 0)
    rs = (h.square().mean(-1, keepdim=True) + eps).rsqrt()
    ref = h * rs * (gamma.double() if gamma is not None else 1)
    # the sum of squares: h off by U of itself, squares in at most 40 steps, so 42 U, half of that in rstd and six operations; then h, rstd and gamma
    slack = 32 * U * ref.abs() + (U * (x.double().abs() + h.abs()) * rs if r is not None else 0)
    if fp8:
        within_fp8(y, ref, slack)
    else:
        within(y, ref, slack)
    within(rstd, rs[..., 0], 28 * U * rs[..., 0])
    if r is not None:
        within(out[1], h, U * h.abs())
    again = B.rmsnorm_fwd(x, gamma, eps, residual=r, out_dtype=yt)
    again = again[0] if r is not None else again
    for a, b in zip(again, y) if fp8 else ((again, y),):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    return out


def rms_inputs(M, C, xt, rt, seed):
    import torch
    g = gen(seed)
    x = randn(g, M, C, scale=1.5, dtype=getattr(torch, xt))
    return x, None if rt is None else randn(g, M, C, scale=2.0, dtype=getattr(torch, rt)), (1 + randn(g, C, scale=0.3)).bfloat16(), g


@pytest.mark.parametrize("C", LENGTHS)
@pytest.mark.parametrize("xt,rt", TYPES)
def test_rmsnorm_fwd(B, C, xt, rt):
    import torch
    for yt in (torch.bfloat16, torch.float32) + ((torch.float8_e4m3fn,) if C % 16 == 0 else ()):
        for M in (1, 7):
            x, r, ga, _ = rms_inputs(M, C, xt, rt, C + M)
            check_rms_fwd(B, x, r, ga, yt)
        check_rms_fwd(B, x, r, None, yt)


@pytest.mark.parametrize("C", [16, 48, 112, 144, 272, 304, 496, 528, 784, 1296, 2032, 2064, 4112, 8176, 8208, 16368])
def test_rmsnorm_blocks_that_end_early(B, C):
    import torch
    for xt, rt in TYPES:
        x, r, ga, _ = rms_inputs(5, C, xt, rt, C)
        check_rms_fwd(B, x, r, ga, torch.float8_e4m3fn)


@pytest.mark.parametrize("M,C", [(40003, 64), (33001, 63), (33001, 128), (20001, 320), (20001, 512), (8195, 768), (4101, 515), (8195, 1280), (8195, 1283), (5003, 2048), (2051, 4096), (1030, 4095),
                                 (2051, 8192), (1030, 16384)])
def test_rmsnorm_fwd_rows_in_turn(B, M, C):
    """More rows than a launch has places for (1024 workgroups of 16, 4 or 1 rows): two rounds and more, the last not full."""
    import torch
    for xt, rt in (TYPES[1], TYPES[3]):
        x, r, ga, _ = rms_inputs(M, C, xt, rt, C)
        check_rms_fwd(B, x, r, ga, torch.bfloat16)
        if C % 16 == 0:
            check_rms_fwd(B, x, r, ga, torch.float8_e4m3fn)


@pytest.mark.parametrize("C", [320, 1155, 3000])
def test_rmsnorm_hard_rows(B, C):
    """Zeros, one element far from the rest, large and tiny rows; infinities and NaN stay in their rows."""
    import torch
    x, r, ga, g = rms_inputs(12, C, "float32", "float32", 1)
    x[0], r[0] = 0, 0
    x[1, 0], x[2, C - 1] = 3e4, -3e4
    x[3] *= 1e15
    x[4] *= 1e-12
    r[4] *= 1e-12
    for yt in (torch.bfloat16, torch.float32):
        check_rms_fwd(B, x, r, ga, yt)
    x[5, 3], x[6, 5], r[7, C - 1] = math.inf, math.nan, -math.inf
    y, h = B.rmsnorm_fwd(x, ga, residual=r, out_dtype=torch.float32)
    clean, _ = B.rmsnorm_fwd(x[8:].contiguous(), ga, residual=r[8:].contiguous(), out_dtype=torch.float32)
    assert torch.equal(y[8:], clean) and torch.isfinite(y[:5]).all()
    # an infinite sum of squares: rstd 0, so that the infinity is NaN and the others are 0
    for i, c in ((5, 3), (7, C - 1)):
        assert y[i, c].isnan() and (y[i, :c] == 0).all() and (y[i, c + 1:] == 0).all()
    assert y[6].isnan().all()


def test_rmsnorm_in_place_and_empty(B):
    import torch
    for C in (1280, 4095, 5001):       # (of the latter two, threads of other wavefronts share elements)
        x, r, ga, _ = rms_inputs(300, C, "bfloat16", "float32", C)
        y, h = B.rmsnorm_fwd(x, ga, residual=r)
        r2, x2 = r.clone(), x.clone()
        out = B.rmsnorm_fwd(x2, ga, residual=r2, out=x2, h_out=r2)
        assert out[0] is x2 and out[1] is r2 and torch.equal(x2, y) and torch.equal(r2, h)
        dy, dres = torch.randn_like(h), torch.randn_like(h)
        rstd = B.rmsnorm_fwd(x, ga, residual=r, stats=True)[2]
        want = B.rmsnorm_bwd(dy, h, rstd, ga, dres=dres)
        for i in range(3):
            a = [dy.clone(), h.clone(), dres.clone()]
            got = B.rmsnorm_bwd(a[0], a[1], rstd, ga, dres=a[2], out=a[i])
            assert torch.equal(got[0], want[0])
            assert torch.allclose(got[1], want[1], rtol=0, atol=float(2 * 400 * U * (dy * h * rstd[:, None]).abs().sum(0).max()))
    e = torch.empty(0, 64, device="cuda")
    assert B.rmsnorm_fwd(e).shape == (0, 64) and B.rmsnorm_fwd(e, out_dtype=torch.float8_e4m3fn).scales.shape == (1, 0)
    dh, dg = B.rmsnorm_bwd(e, e, torch.empty(0, device="cuda"))
    assert dh.shape == (0, 64) and not dg.any() and dg.shape == (64,)
    x = randn(gen(1), 2, 3, 64)
    assert torch.equal(B.rmsnorm_fwd(x), B.rmsnorm_fwd(x.view(6, 64)).view(2, 3, 64))


def check_rms_bwd(B, h, dy, dres, gamma, rstd):
    import torch
    M, C = h.shape
    dh, dg = B.rmsnorm_bwd(dy, h, rstd, gamma, dres=dres)
    x, d, r = h.double(), dy.double(), rstd.double()[:, None]
    n = x * r
    g = d * (gamma.double() if gamma is not None else 1)
    c = (g * n).mean(1, keepdim=True)
    ref = r * (g - n * c) + (dres.double() if dres is not None else 0)
    # the mean of products: four operations each, 40 steps
    slack = r * (8 * U * (g.abs() + (n * c).abs()) + 46 * U * n.abs() * (g * n).abs().mean(1, keepdim=True)) + 2 * U * ref.abs()
    within(dh, ref, slack)
    # sums over rows: of a workgroup's, of its wavefronts', of workgroups
    within(dg, (d * n).sum(0), (min(M, 64 + M / 64) + 40) * U * (d * n).abs().sum(0))
    again = B.rmsnorm_bwd(dy, h, rstd, gamma, dres=dres)
    assert torch.equal(again[0], dh) and torch.equal(again[1], dg)
    alone = B.rmsnorm_bwd(dy, h, rstd, gamma, dres=dres, weight_grad=False)
    assert alone[1] is None and torch.equal(alone[0], dh)


@pytest.mark.parametrize("C", LENGTHS)
@pytest.mark.parametrize("ht,yt", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("float32", "float32"), ("bfloat16", "float32")])
def test_rmsnorm_bwd(B, C, ht, yt):
    import torch
    for M in (1, 7, 130):
        h, _, ga, g = rms_inputs(M, C, ht, None, C + M)
        dy = randn(g, M, C, dtype=getattr(torch, yt))
        dres = randn(g, M, C, dtype=h.dtype)
        rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
        check_rms_bwd(B, h, dy, dres, ga, rstd)
    check_rms_bwd(B, h, dy, None, ga, rstd)
    check_rms_bwd(B, h, dy, None, None, rstd)


@pytest.mark.parametrize("M,C", [(40003, 64), (33001, 63), (40003, 128), (9001, 256), (9001, 768), (8201, 515), (5003, 1280), (4101, 1283), (5003, 2048), (1100, 4096), (1031, 5000), (2051, 8192), (600, 16384)])
def test_rmsnorm_bwd_rows_in_turn(B, M, C):
    import torch
    for ht, yt in (("float32", "bfloat16"), ("bfloat16", "bfloat16")):
        h, _, ga, g = rms_inputs(M, C, ht, None, C)
        dy, dres = randn(g, M, C, dtype=getattr(torch, yt)), randn(g, M, C, dtype=h.dtype)
        rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
        check_rms_bwd(B, h, dy, dres, ga, rstd)


def test_rmsnorm_gradients_against_differences(B):
    import torch
    M, C, eps = 3, 20, 1e-6
    x, r, ga, g = rms_inputs(M, C, "float32", "float32", 9)
    dy = randn(g, M, C)
    _, h, rstd = B.rmsnorm_fwd(x, ga, eps, residual=r, out_dtype=torch.float32, stats=True)
    dh, dg = B.rmsnorm_bwd(dy, h, rstd, ga)

    def loss(x, r, ga):
        h = x + r
        return (h * (h.square().mean(1, keepdim=True) + eps).rsqrt() * ga * dy.double()).sum()
    args = [t.double() for t in (x, r, ga)]
    for i, got in ((0, dh), (1, dh), (2, dg)):
        for j in range(0, args[i].numel(), 7):
            d = []
            for s in (1e-5, -1e-5):
                a = [t.clone() for t in args]
                a[i].view(-1)[j] += s
                d.append(loss(*a))
            # central differences in 64 bits: third derivatives times 1e-10, roundings 2^-53 / 1e-5; the kernel's own error as above
            assert abs(float((d[0] - d[1]) / 2e-5) - float(got.view(-1)[j])) < 1e-5 * (1 + abs(float(got.view(-1)[j])))


def test_rmsnorm_offsets_past_32_bits(B):
    """Rows whose elements, and bytes, lie beyond 2^31 and 2^32"""
    import torch
    C = 16384
    M = 2 ** 32 // (2 * C) + 5
    x = torch.empty(M, C, dtype=torch.bfloat16, device="cuda")
    for i in range(0, M, 8192):
        x[i:i + 8192].normal_()
    y = B.rmsnorm_fwd(x)
    q = B.rmsnorm_fwd(x, out_dtype=torch.float8_e4m3fn)
    q2 = B.quantize_fp8(x)
    for rows in (slice(0, 3), slice(65530, 65540), slice(M - 6, M)):
        part = x[rows].contiguous()
        assert torch.equal(y[rows], B.rmsnorm_fwd(part))
        for got, want in ((q, B.rmsnorm_fwd(part, out_dtype=torch.float8_e4m3fn)), (q2, B.quantize_fp8(part))):
            assert torch.equal(got.q[rows].view(torch.uint8), want.q.view(torch.uint8)) and torch.equal(got.scales[:, rows].contiguous().view(torch.uint8), want.scales.contiguous().view(torch.uint8))


# ---- gated linear layer in bf16 ----------------------------------------------------------------------------------------------
def gated_ref(z, ez, act, extra=0.0):
    """y = v act(g) of z = [v, g] off by ez, and its bound"""
    N = z.shape[1] // 2
    v, g, ev, eg = z[:, :N], z[:, N:], ez[:, :N], ez[:, N:]
    a = act64(g, act)
    # slopes are below 1.13, the activations' own error below 4e-7 (1 + |g|)
    ea = 1.13 * eg + 4e-7 * (1 + g.abs()) * (act > 0)
    return v * a, a.abs() * ev + (v.abs() + ev) * ea + 2 * U * (v * a).abs()


def check_gated_fwd(B, x, W, bias, act, yt, save_z=True):
    import torch
    out = B.gated_linear_fwd(x, W, bias, act, out_dtype=yt, save_z=save_z)
    y, zk = out if save_z else (out, None)
    K = x.shape[1]
    xd, wd = x.double(), W.double()
    b = bias.double() if bias is not None else torch.zeros(W.shape[0], dtype=torch.float64, device="cuda")
    z = xd @ wd.T + b
    ez = (K + 8) * U * (xd.abs() @ wd.abs().T + b.abs())
    within(y, *gated_ref(z, ez, act))
    if save_z:
        within(zk, z, ez)
    return y


SIZES = [(1, 8, 8), (1, 2560, 64), (2, 1, 64), (3, 31, 72), (16, 130, 640), (17, 64, 200), (64, 64, 64), (65, 65, 136), (129, 317, 648), (200, 256, 320), (300, 515, 1024), (530, 36, 72), (700, 333, 128)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("yt", ["bfloat16", "float32"])
def test_gated_fwd(B, M, N, K, yt):
    import torch
    yt = getattr(torch, yt)
    x, W, bias, _ = lin_inputs(M, 2 * N, K, M + N + K)
    for act in range(5):
        y = check_gated_fwd(B, x, W, bias, act, yt)
        assert torch.equal(check_gated_fwd(B, x, W, bias, act, yt, save_z=False), y)
    check_gated_fwd(B, x, W, None, 3, yt)
    assert torch.equal(B.gated_linear_fwd(x, W, bias, 3, out_dtype=yt), B.gated_linear_fwd(x, W, bias, 3, out=torch.empty(M, N, dtype=yt, device="cuda")))


@pytest.mark.parametrize("M,N,K", [(4133, 320, 320), (2048, 1288, 648), (1976, 1280, 1280), (700, 2560, 640), (1030, 5120, 264), (9000, 161, 128), (5003, 2580, 64), (8192, 640, 8)])
def test_gated_fwd_large(B, M, N, K):
    import torch
    x, W, bias, _ = lin_inputs(M, 2 * N, K, M + N)
    check_gated_fwd(B, x, W, bias, 3, torch.bfloat16)
    check_gated_fwd(B, x, W, bias, 1, torch.float32, save_z=False)


def check_gated_bwd(B, dy, x, W, z, act, dwt):
    import torch
    M, K = x.shape
    N2 = W.shape[0]
    N = N2 // 2
    got = B.gated_linear_bwd(dy, x, W, z, act, dw_dtype=dwt)
    zz = z.double().requires_grad_(True)
    dz = torch.autograd.grad(zz[:, :N] * act64(zz[:, N:], act), zz, dy.double())[0]
    # dv = dy act(g), dg = dy v act'(g): the activation's own error and its slope's, dz rounded to bf16; sums of 2 N, or M, products
    d, v, g = dy.double().abs(), z.double()[:, :N].abs(), z.double()[:, N:].abs()
    own = torch.cat([4e-7 * (1 + g) * d, 1e-6 * d * v], 1) * (act > 0) + 3 * U * dz.abs()
    ez = 2.0 ** -8 * (dz.abs() + own) + own
    wd, xd = W.double(), x.double()
    rx, rw = dz @ wd, dz.T.contiguous() @ xd
    within(got[0], rx, ez @ wd.abs() + (N2 + 8) * U * (dz.abs() @ wd.abs()))
    within(got[1], rw, ez.T.contiguous() @ xd.abs() + (M + 8) * U * (dz.abs().T.contiguous() @ xd.abs()))
    for a, ref in ((got[0], rx), (got[1], rw)):
        if ref.norm() > 0 and min(M, N) > 30:
            assert float((a.double() - ref).norm() / ref.norm()) <= math.hypot(2.0 ** -8, torch.finfo(a.dtype).eps / 2) + 1e-5
    within(got[2], dz.sum(0), own.sum(0) + (M / 64 + 40) * U * dz.abs().sum(0))
    again = B.gated_linear_bwd(dy, x, W, z, act, dw_dtype=dwt)
    assert all(torch.equal(a, b) for a, b in zip(again, got))
    for i in range(3):
        part = B.gated_linear_bwd(dy, x, W, z, act, grads=[j == i for j in range(3)], dw_dtype=dwt)
        assert all((p is None) if j != i else torch.equal(p, got[i]) for j, p in enumerate(part))


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("yt", ["bfloat16", "float32"])
def test_gated_bwd(B, M, N, K, yt):
    import torch
    x, W, _, g = lin_inputs(M, 2 * N, K, M + N + K)
    dy = randn(g, M, N, dtype=getattr(torch, yt))
    z = randn(g, M, 2 * N, scale=1.5).bfloat16()
    for act in range(5):
        check_gated_bwd(B, dy, x, W, z, act, torch.float32 if act % 2 else torch.bfloat16)


@pytest.mark.parametrize("M,N,K", [(4133, 320, 320), (2048, 644, 648), (8192, 160, 1280), (5000, 32, 64), (60, 2560, 1280), (1, 2048, 2048), (3000, 645, 328)])
def test_gated_bwd_large(B, M, N, K):
    import torch
    x, W, _, g = lin_inputs(M, 2 * N, K, M + N)
    z = randn(g, M, 2 * N, scale=1.5).bfloat16()
    check_gated_bwd(B, randn(g, M, N).bfloat16(), x, W, z, 3, torch.bfloat16)
    check_gated_bwd(B, randn(g, M, N), x, W, z, 2, torch.float32)


@pytest.mark.parametrize("M,N,K", [(8200, 2064, 16), (8400, 2001, 24)])
def test_gated_results_past_the_caches(B, M, N, K):
    """z of more than 2^25 elements"""
    import torch
    x, W, bias, g = lin_inputs(M, 2 * N, K, M + N)
    check_gated_fwd(B, x, W, bias, 3, torch.bfloat16)
    _, z = B.gated_linear_fwd(x, W, bias, 3, save_z=True)
    dy = randn(g, M, N).bfloat16()
    check_gated_bwd(B, dy, x, W, z, 3, torch.bfloat16)
    check_gated_bwd(B, dy.float(), x, W, z, 1, torch.float32)


def test_gated_fp8_past_the_caches(B):
    """y in 8 bits of more than 2^23 elements"""
    import torch
    g = gen(31)
    x, W = rows8(B, g, 8200, 144), rows8(B, g, 2 * 1040, 144, 0.1)
    check_gated8(B, x, W, randn(g, 2 * 1040, scale=0.5).bfloat16(), 3, torch.float8_e4m3fn)


def test_gated_gradients_against_differences(B):
    import torch
    M, N, K = 3, 9, 16
    x, W, bias, g = lin_inputs(M, 2 * N, K, 1)
    dy = randn(g, M, N)
    for act in range(1, 4):
        _, z = B.gated_linear_fwd(x, W, bias, act, save_z=True)
        db = B.gated_linear_bwd(dy[:1].contiguous(), x[:1].contiguous(), W, z[:1].contiguous(), act)[2]       # of one row: dz itself

        def loss(z):
            return (z[:, :N] * act64(z[:, N:], act) * dy[:1].double()).sum()
        for j in range(2 * N):
            d = []
            for s in (1e-5, -1e-5):
                zz = z[:1].double().clone()
                zz[0, j] += s
                d.append(float(loss(zz)))
            # third derivatives times 1e-10, roundings in 64 bits over 1e-5; the slopes' own error
            assert abs((d[0] - d[1]) / 2e-5 - float(db[j])) < 1e-5 * (1 + abs(float(db[j])))


def test_gated_edges(B):
    import torch
    x, W, bias, g = lin_inputs(6, 48, 16, 1)
    e = torch.empty(0, 16, dtype=torch.bfloat16, device="cuda")
    assert B.gated_linear_fwd(e, W, bias).shape == (0, 24)
    dx, dW, db = B.gated_linear_bwd(torch.empty(0, 24, dtype=torch.bfloat16, device="cuda"), e, W, torch.empty(0, 48, dtype=torch.bfloat16, device="cuda"))
    assert dx.shape == (0, 16) and not dW.any() and not db.any()
    dx, dW, db = B.gated_linear_bwd(torch.empty(6, 0, dtype=torch.bfloat16, device="cuda"), x, W[:0], torch.empty(6, 0, dtype=torch.bfloat16, device="cuda"))
    assert not dx.any() and dW.shape == (0, 16) and db.shape == (0,)
    # NaN and infinities stay in their rows and columns
    x[2, 3] = math.nan
    y = B.gated_linear_fwd(x, W, bias, 1)
    assert y[2].isnan().all() and torch.isfinite(y[[0, 1, 3, 4, 5]].float()).all()


# ---- products of rows in 8 bits ----------------------------------------------------------------------------------------------
def rows8(B, g, M, K, scale=1.0, spread=1.0):
    import torch
    return B.quantize_fp8(randn(g, M, K, scale=scale) * torch.exp(spread * randn(g, M, 1)) * torch.exp(spread * randn(g, 1, (K + 127) // 128)).repeat_interleave(128, 1)[:, :K])


def product(x, W, bias, fp32):
    """z and its bound.  Products are exact.  In bf16 (y in fp32, and few rows, for which this bound is the looser one too) every one of K + 8 additions may be off by 2 U of the sum of magnitudes.  The scaled MFMA adds
    eight products at a time and drops what is below 2^-13 of the largest one's power of two: seven of them lose less than 2^-13 of it each."""
    xd, wd = values(x), values(W)
    z, mag = xd @ wd.T, xd.abs() @ wd.abs().T
    if bias is not None:
        z, mag = z + bias.double(), mag + bias.double().abs()
    M, K = x.q.shape
    e = (K + 8) * 2 * U * mag
    if not fp32:
        xa, wa = xd.abs().float(), wd.abs().float()
        top = sum((xa[:, None, k:k + 8] * wa[None, :, k:k + 8]).amax(2).double() for k in range(0, K, 8)) if M * wd.shape[0] <= 1 << 20 else mag
        e = e + 7 * 2.0 ** -13 * top
    return z, e


def check_linear8(B, x, W, bias, act, res, yt):
    import torch
    y = B.linear_fp8_fwd(x, W, bias, act, residual=res, out_dtype=yt)
    z, ez = product(x, W, bias, yt == torch.float32)
    ref = act64(z, act) + (res.double() if res is not None else 0)
    within(y, ref, 1.13 * ez + 4e-7 * (1 + z.abs()) * (act > 0) + 2 * U * ref.abs())
    # all together: independent roundings, of y and of products (2^-13 of the largest of eight, in a sum of eight)
    assert float((y.double() - ref).norm() / ref.norm().clamp(min=1e-30)) <= (torch.finfo(yt).eps / 2) + (0 if yt == torch.float32 else 2.0 ** -13) + (x.q.shape[1] + 8) * 2 * U
    return y


def check_gated8(B, x, W, bias, act, yt):
    import torch
    y = B.gated_linear_fp8_fwd(x, W, bias, act, out_dtype=yt)
    z, ez = product(x, W, bias, yt == torch.float32)
    ref, slack = gated_ref(z, ez, act)
    if yt == torch.float8_e4m3fn:
        within_fp8(y, ref, slack)
    else:
        within(y, ref, slack)
    return y


SIZES8 = [(1, 16, 16), (1, 5120, 64), (2, 1, 64), (3, 31, 80), (16, 130, 640), (17, 64, 208), (64, 64, 64), (65, 65, 144), (129, 317, 656), (200, 256, 320), (300, 515, 1024), (530, 36, 80), (700, 333, 128), (1000, 640, 1936)]


@pytest.mark.parametrize("M,N,K", SIZES8)
@pytest.mark.parametrize("yt", ["bfloat16", "float32"])
def test_linear_fp8(B, M, N, K, yt):
    import torch
    yt, g = getattr(torch, yt), gen(M + N + K)
    x, W = rows8(B, g, M, K), rows8(B, g, N, K, 1.3 / math.sqrt(K), 0.3)
    bias, res = randn(g, N, scale=0.5).bfloat16(), randn(g, M, N, dtype=yt)
    for act in range(5):
        check_linear8(B, x, W, bias, act, res, yt)
        y = check_linear8(B, x, W, bias, act, None, yt)
    assert torch.equal(B.linear_fp8_fwd(x, W, bias, 4, out_dtype=yt), y)
    check_linear8(B, x, W, None, 0, res, yt)
    ref = B.linear_fp8_fwd(x, W, bias, 3, residual=res, out_dtype=yt)
    assert torch.equal(B.linear_fp8_fwd(x, W, bias, 3, residual=res, out=res), ref)


@pytest.mark.parametrize("M,N,K", [(4133, 640, 320), (2048, 1280, 656), (8192, 640, 1280), (1976, 1280, 5120), (700, 5120, 640), (1030, 2560, 2064), (9000, 321, 128), (5003, 1292, 64)])
def test_linear_fp8_large(B, M, N, K):
    import torch
    g = gen(M + N)
    x, W = rows8(B, g, M, K), rows8(B, g, N, K, 1.3 / math.sqrt(K), 0.3)
    bias = randn(g, N, scale=0.5).bfloat16()
    check_linear8(B, x, W, bias, 0, randn(g, M, N), torch.float32)
    check_linear8(B, x, W, bias, 1, None, torch.bfloat16)


@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (1, 5120, 1280), (2, 144, 64), (16, 320, 640), (17, 64, 208), (65, 128, 144), (129, 336, 656), (300, 528, 1024), (513, 48, 80), (530, 112, 272), (700, 336, 128), (2100, 640, 1296), (1976, 1280, 320)])
def test_gated_fp8(B, M, N, K):
    import torch
    g = gen(M + N + K)
    x, W = rows8(B, g, M, K), rows8(B, g, 2 * N, K, 1.3 / math.sqrt(K), 0.3)
    bias = randn(g, 2 * N, scale=0.5).bfloat16()
    for yt in (torch.float8_e4m3fn, torch.bfloat16, torch.float32):
        for act in range(5):
            y = check_gated8(B, x, W, bias, act, yt)
        check_gated8(B, x, W, None, 3, yt)
        again = B.gated_linear_fp8_fwd(x, W, bias, 4, out_dtype=yt)
        for a, b in zip(again, y) if isinstance(y, tuple) else ((again, y),):
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_scales_of_blocks(B):
    """Every block of either operand has a scale of its own: far apart, so that a wrong one would show"""
    import torch
    g = gen(5)
    for M, N, K in ((3, 48, 1296), (70, 144, 1296), (600, 272, 1296)):
        x, W = rows8(B, g, M, K, 1.0, 3.0), rows8(B, g, N, K, 1.0, 3.0)
        check_linear8(B, x, W, None, 0, None, torch.float32)
        check_gated8(B, x, rows8(B, g, 2 * N, K, 1.0, 3.0), None, 0, torch.float32)


def test_rows_of_larger_matrices(B):
    """Operands and results that are some rows of others: scales of theirs further apart; the others' stay as they were"""
    import torch
    g = gen(6)
    M, N, K = 100, 48, 272
    big, W = rows8(B, g, 180, K), rows8(B, g, 2 * N, K, 0.1)
    x = B.Fp8Rows(big.q[16:16 + M], big.scales[:, 16:16 + M])
    alone = B.Fp8Rows(x.q.clone(), x.scales.contiguous())
    assert torch.equal(B.linear_fp8_fwd(x, W), B.linear_fp8_fwd(alone, W))
    for rows in (M, 13):
        q, s = torch.full((160, N), 3, dtype=torch.uint8, device="cuda"), torch.full((1, 160), 7, dtype=torch.uint8, device="cuda")
        out = B.Fp8Rows(q[32:32 + rows].view(torch.float8_e4m3fn), s[:, 32:32 + rows].view(torch.float8_e8m0fnu))
        xr = B.Fp8Rows(x.q[:rows], x.scales[:, :rows])
        B.gated_linear_fp8_fwd(xr, W, out=out)
        want = B.gated_linear_fp8_fwd(B.Fp8Rows(alone.q[:rows], alone.scales[:, :rows]), W, out_dtype=torch.float8_e4m3fn)
        assert torch.equal(out.q.view(torch.uint8), want.q.view(torch.uint8)) and torch.equal(out.scales.view(torch.uint8), want.scales.contiguous().view(torch.uint8))
        assert (q[:32] == 3).all() and (q[32 + rows:] == 3).all() and (s[:, :32] == 7).all() and (s[:, 32 + rows:] == 7).all()


def test_fp8_special_values(B):
    """A NaN stays in its row (of x) or column (of W); the largest values do not overflow; empty sizes"""
    import torch
    g = gen(7)
    for M in (5, 600):
        x, W = randn(g, M, 256), randn(g, 48, 256)
        x[2, 130], W[7, 3] = math.nan, math.inf
        x8, W8 = B.quantize_fp8(x), B.quantize_fp8(W)
        bad = ~torch.isfinite(B.linear_fp8_fwd(x8, W8).float())
        want = torch.zeros_like(bad)
        want[2] = True
        want[:, 7] = True
        assert torch.equal(bad, want)
        top = B.quantize_fp8(torch.full((M, 256), 448.0, device="cuda"))
        y = B.linear_fp8_fwd(top, B.quantize_fp8(torch.full((16, 256), -448.0, device="cuda")), out_dtype=torch.float32)
        assert (y == -256 * 448.0 ** 2).all()
    e = B.Fp8Rows(x8.q[:0], x8.scales[:, :0])
    assert B.linear_fp8_fwd(e, W8).shape == (0, 48) and B.gated_linear_fp8_fwd(e, B.Fp8Rows(W8.q[:32], W8.scales[:, :32]), out_dtype=torch.float8_e4m3fn).q.shape == (0, 16)
    assert B.linear_fp8_fwd(x8, B.Fp8Rows(W8.q[:0], W8.scales[:, :0])).shape == (600, 0)


LIN8_KERNELS = [("bfloat16", *c) for c in [
    (1, 1, 768, "few rows 8 bits 16x16"), (4579, 1, 768, "few rows 8 bits 32x16"), (11378, 129, 128, "gemm cols 8 bits 128x128/4 waves/2 stages"),
    (3684, 4459, 768, "gemm cols 8 bits 128x128/4 waves/2 stages"), (8807, 197, 16, "gemm cols 8 bits 128x128/4 waves/2 stages guard"),
    (11547, 291, 128, "gemm cols 8 bits 128x192/8 waves/3 stages"), (8380, 424, 768, "gemm cols 8 bits 128x192/8 waves/3 stages"),
    (11162, 289, 864, "gemm cols 8 bits 128x192/8 waves/3 stages guard"), (1310, 5559, 768, "gemm cols 8 bits 128x256/8 waves/3 stages"),
    (1325, 5606, 16, "gemm cols 8 bits 128x256/8 waves/3 stages guard"), (10937, 412, 768, "gemm cols 8 bits 256x128/8 waves/3 stages"),
    (8465, 603, 816, "gemm cols 8 bits 256x128/8 waves/3 stages guard"), (9654, 792, 128, "gemm cols 8 bits 256x256/8 waves/2 stages"),
    (3914, 2073, 768, "gemm cols 8 bits 256x256/8 waves/2 stages"), (10005, 781, 800, "gemm cols 8 bits 256x256/8 waves/2 stages guard"),
    (10530, 69, 384, "gemm cols 8 bits 64x128/4 waves/3 stages"), (8735, 73, 768, "gemm cols 8 bits 64x128/4 waves/3 stages"),
    (8200, 72, 944, "gemm cols 8 bits 64x128/4 waves/3 stages guard"), (1, 4216, 768, "gemm cols 8 bits 64x64/4 waves/4 stages"),
    (3, 4463, 784, "gemm cols 8 bits 64x64/4 waves/4 stages guard"), (6877, 263, 256, "gemm cols 8 bits 96x128/4 waves/3 stages"),
    (11111, 141, 768, "gemm cols 8 bits 96x128/4 waves/3 stages"), (8807, 197, 784, "gemm cols 8 bits 96x128/4 waves/3 stages guard")]] + [("float32", *c) for c in [
    (4281, 1, 768, "few rows 8 bits 32x16"), (1, 4228, 784, "few rows 8 bits 32x32"), (8397, 1, 16, "few rows 8 bits 64x32"),
    (6254, 419, 768, "gemm cols 8 bits wide 64x64/8 waves/4 stages"), (6639, 263, 16, "gemm cols 8 bits wide 96x128/8 waves/3 stages guard"),
    (777, 5036, 768, "gemm cols 8 bits wide 128x192/8 waves/3 stages"), (8203, 456, 880, "gemm cols 8 bits wide 128x192/8 waves/3 stages guard"),
    (8239, 67, 896, "gemm cols 8 bits wide 64x128/8 waves/3 stages"), (9071, 78, 16, "gemm cols 8 bits wide 64x128/8 waves/3 stages guard"),
    (71, 4864, 768, "gemm cols 8 bits wide 64x64/8 waves/4 stages"), (66, 4143, 816, "gemm cols 8 bits wide 64x64/8 waves/4 stages guard"),
    (1239, 4937, 128, "gemm cols 8 bits wide 128x256/8 waves/3 stages"), (8465, 603, 816, "gemm cols 8 bits wide 128x256/8 waves/3 stages guard"), (11391, 154, 768, "gemm cols 8 bits wide 96x128/8 waves/3 stages"),
    (11271, 153, 784, "gemm cols 8 bits wide 96x128/8 waves/3 stages guard")]]


@pytest.mark.parametrize("yt,M,N,K,kernel", LIN8_KERNELS)
def test_linear_fp8_every_kernel(B, yt, M, N, K, kernel):
    """Each kernel with and without bias and residual; the choice does not depend on them."""
    import torch
    yt, g = getattr(torch, yt), gen(M + K)
    x, W = rows8(B, g, M, K), rows8(B, g, N, K, 1.3 / math.sqrt(K), 0.3)
    bias, res = randn(g, N, scale=0.5).bfloat16(), randn(g, M, N, dtype=yt)
    with B.dry_run() as names:
        B.linear_fp8_fwd(x, W, bias, 1, residual=res, out_dtype=yt)
        B.linear_fp8_fwd(x, W, out_dtype=yt)
    assert names == [kernel] * 2
    check_linear8(B, x, W, bias, 3, res, yt)
    check_linear8(B, x, W, None, 0, None, yt)


GATED8_KERNELS = [("bfloat16", *c) for c in [
    (1, 16, 768, "few rows 8 bits gated 16x16"), (17, 2096, 768, "few rows 8 bits gated 32x16"), (149, 5616, 128, "gemm cols 8 bits gated 128x128/4 waves/2 stages"), (4934, 800, 1280, "gemm cols 8 bits gated 128x128/4 waves/2 stages"),
    (808, 4640, 912, "gemm cols 8 bits gated 128x128/4 waves/2 stages guard"), (525, 5600, 768, "gemm cols 8 bits gated 128x256/8 waves/3 stages"), (10904, 144, 16, "gemm cols 8 bits gated 128x256/8 waves/3 stages guard"),
    (555, 5504, 928, "gemm cols 8 bits gated 128x256/8 waves/3 stages guard"), (11125, 144, 768, "gemm cols 8 bits gated 256x128/8 waves/3 stages"), (10904, 144, 800, "gemm cols 8 bits gated 256x128/8 waves/3 stages guard"),
    (10892, 336, 768, "gemm cols 8 bits gated 256x256/8 waves/2 stages"), (6700, 592, 784, "gemm cols 8 bits gated 256x256/8 waves/2 stages guard"), (65, 4416, 768, "gemm cols 8 bits gated 64x128/4 waves/3 stages"),
    (69, 4544, 832, "gemm cols 8 bits gated 64x128/4 waves/3 stages guard"), (1, 4144, 768, "gemm cols 8 bits gated 64x64/2 waves/4 stages"), (1, 4256, 848, "gemm cols 8 bits gated 64x64/2 waves/4 stages guard")]] + [("float32", *c) for c in [
    (17, 2224, 784, "few rows 8 bits gated 32x16"), (1, 4288, 768, "few rows 8 bits gated 32x32"), (130, 5600, 896, "gemm cols 8 bits wide gated 128x128/8 waves/3 stages"),
    (145, 5632, 784, "gemm cols 8 bits wide gated 128x128/8 waves/3 stages guard"), (412, 4800, 768, "gemm cols 8 bits wide gated 128x128/4 waves/2 stages"),
    (583, 3328, 848, "gemm cols 8 bits wide gated 128x128/4 waves/2 stages guard"), (70, 4336, 768, "gemm cols 8 bits wide gated 64x128/4 waves/3 stages"), (67, 4480, 848, "gemm cols 8 bits wide gated 64x128/4 waves/3 stages guard"),
    (8255, 16, 768, "gemm cols 8 bits wide gated 64x64/4 waves/4 stages"), (8909, 16, 784, "gemm cols 8 bits wide gated 64x64/4 waves/4 stages guard")]] + [("float8_e4m3fn", *c) for c in [
    (1, 16, 1936, "few rows 8 bits gated 16x16; quantize"), (9309, 144, 768, "gemm cols 8 bits gated to 8 bits 128x256/8 waves/3 stages"), (9045, 144, 880, "gemm cols 8 bits gated to 8 bits 128x256/8 waves/3 stages guard"),
    (6662, 544, 768, "gemm cols 8 bits gated to 8 bits 256x256/8 waves/2 stages"), (11037, 272, 784, "gemm cols 8 bits gated to 8 bits 256x256/8 waves/2 stages guard"), (1, 16, 768, "gemm cols 8 bits wide gated to 8 bits 32x256/4 waves/3 stages"),
    (3, 144, 784, "gemm cols 8 bits wide gated to 8 bits 32x256/4 waves/3 stages guard"), (64, 1296, 640, "gemm cols 8 bits wide gated to 8 bits 32x256/4 waves/3 stages"),
    (64, 32896, 128, "gemm cols 8 bits gated to 8 bits 64x256/4 waves/3 stages"), (65, 144, 768, "gemm cols 8 bits gated to 8 bits 64x256/4 waves/3 stages"), (70, 144, 784, "gemm cols 8 bits gated to 8 bits 64x256/4 waves/3 stages guard")]]


@pytest.mark.parametrize("yt,M,N,K,kernel", GATED8_KERNELS)
def test_gated_fp8_every_kernel(B, yt, M, N, K, kernel):
    import torch
    yt, g = getattr(torch, yt), gen(M + K)
    x, W = rows8(B, g, M, K), rows8(B, g, 2 * N, K, 1.3 / math.sqrt(K), 0.3)
    bias = randn(g, 2 * N, scale=0.5).bfloat16()
    with B.dry_run() as names:
        B.gated_linear_fp8_fwd(x, W, bias, 1, out_dtype=yt)
        B.gated_linear_fp8_fwd(x, W, None, 0, out_dtype=yt)
    assert "; ".join(names) == "; ".join([kernel] * 2)
    check_gated8(B, x, W, bias, 3, yt)
    check_gated8(B, x, W, None, 2, yt)


@pytest.mark.parametrize("M,N,K", [(300, 1296, 5120), (130, 640, 4112)])
def test_gated_fp8_in_two_launches(B, M, N, K):
    """Tiles whose columns are not whole blocks of y: y in fp32 into the workspace, which is all that is asked for"""
    import torch
    g = gen(M)
    x, W = rows8(B, g, M, K), rows8(B, g, 2 * N, K, 1.3 / math.sqrt(K), 0.3)
    need = B.lib().sd_gated_linear_fp8_workspace_bytes(M, N, K)
    assert need == M * N * 4
    with B.dry_run() as names:
        B.gated_linear_fp8_fwd(x, W, out_dtype=torch.float8_e4m3fn)
    assert len(names) == 2 and names[1] == "quantize"
    y = check_gated8(B, x, W, None, 3, torch.float8_e4m3fn)
    ws = torch.full((need + 256,), 77, dtype=torch.uint8, device="cuda")
    mine = B.gated_linear_fp8_fwd(x, W, out_dtype=torch.float8_e4m3fn, ws=ws)
    assert torch.equal(mine.q.view(torch.uint8), y.q.view(torch.uint8)) and (ws[need:] == 77).all()


@pytest.mark.parametrize("M,N,K", [(1, 5120, 128), (1, 16, 16), (5, 144, 80), (33, 1296, 112), (64, 640, 48)])
def test_gated_fp8_of_few_rows_keeps_all_of_a_sum(B, M, N, K):
    """Up to 64 rows are multiplied widened: of products of 8 beside one of 2^14 the scaled MFMA drops up to 2 each, and what fp32 may lose of a sum is (K + 8) 2^-23 2^15, 0.5 at most"""
    import torch
    g = gen(M + N)
    a, w = randn(g, M, K, scale=2.8), randn(g, 2 * N, K, scale=2.8)
    a[:, 0], a[:, 8], w[:, 0], w[:, 8] = 128.0, -128.0, 128.0, 128.0
    x, W = B.quantize_fp8(a), B.quantize_fp8(w)
    with B.dry_run() as names:
        B.gated_linear_fp8_fwd(x, W, None, 0, out_dtype=torch.float8_e4m3fn)
    assert "wide" in names[0]
    y = B.gated_linear_fp8_fwd(x, W, None, 0, out_dtype=torch.float8_e4m3fn)
    ref, slack = gated_ref(*product(x, W, None, True), 0)
    within_fp8(y, ref, slack)


def test_scales_at_their_ends(B):
    """The least, the largest and the NaN scale byte, as a caller's own rows may have them, mean the same in every kernel"""
    import torch
    g = gen(11)
    K, N = 256, 48
    W = rows8(B, g, N, K, 1.0, 0.0)
    for M in (3, 600):
        for yt in (torch.bfloat16, torch.float32):
            x = rows8(B, g, M, K, 1.0, 0.0)
            s = x.scales.contiguous().view(torch.uint8).clone()
            s[0, 1], s[1, 2] = 255, 0                     # NaN; 2^-127
            s = torch.nn.functional.pad(s, (0, -M % 4)).view(torch.float8_e8m0fnu)[:, :M]
            mine = B.Fp8Rows(x.q, s)
            y, clean = B.linear_fp8_fwd(mine, W, out_dtype=yt), B.linear_fp8_fwd(x, W, out_dtype=yt)
            assert y[1].isnan().all()
            keep = [i for i in range(M) if i not in (1, 2)]
            assert torch.equal(y[keep], clean[keep])
            # row 2 is its first block's product alone: the second's, below 2^-127 * 448^2 * 128, is nothing beside it
            first = values(x)[2:3, :128] @ values(W)[:, :128].T
            assert torch.allclose(y[2:3].double(), first, rtol=2.0 ** -7, atol=1e-2 * float(first.abs().max()))
        big = B.quantize_fp8(torch.full((M, K), 2.0 ** 100, device="cuda"))
        tiny = B.quantize_fp8(torch.full((16, K), 2.0 ** -100, device="cuda"))
        for yt in (torch.bfloat16, torch.float32):
            assert (B.linear_fp8_fwd(big, tiny, out_dtype=yt) == 256).all()


def test_fp8_offsets_past_32_bits(B):
    """Rows of x, of W and of y beyond 2^32 bytes"""
    import torch
    K = 4096
    M = 2 ** 32 // K + 70
    x = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    for i in range(0, M, 65536):
        x[i:i + 65536].normal_()
    x8 = B.quantize_fp8(x)
    del x
    few = lambda a, rows: B.Fp8Rows(a.q[rows], torch.nn.functional.pad(a.scales[:, rows].view(torch.uint8), (0, -len(range(*rows.indices(a.q.shape[0]))) % 4)).view(torch.float8_e8m0fnu)[:, :len(range(*rows.indices(a.q.shape[0])))])
    last = slice(M - 70, M)
    W = rows8(B, gen(1), 32, K, 1 / 64, 0.0)
    y = B.linear_fp8_fwd(x8, W)
    z, ez = product(few(x8, last), W, None, False)
    within(y[last], z, ez)
    # as weights: value and gate far apart
    xs = rows8(B, gen(2), 20, K, 1 / 64, 0.0)
    N = M // 32 * 16
    Wg = B.Fp8Rows(x8.q[:2 * N], x8.scales[:, :2 * N])
    for yt in (torch.float8_e4m3fn, torch.bfloat16):
        y = B.gated_linear_fp8_fwd(xs, Wg, None, 0, out_dtype=yt)
        y = values(y) if yt == torch.float8_e4m3fn else y.double()
        cols = slice(N - 128, N)
        v, g = (product(xs, few(x8, slice(s + N - 128, s + N)), None, False)[0] for s in (0, N))
        assert float((y[:, cols] - v * g).norm() / (v * g).norm()) < 2.0 ** -4
    del y, Wg, x8
    # a y of more than 2^32 bytes, in bf16 and its z
    M, N = 40000, 54016
    x, W, bias, g = lin_inputs(M, 2 * N, 64, 5)
    y, z = B.gated_linear_fwd(x, W, bias, save_z=True)
    assert y.numel() * 2 > 2 ** 32
    rows = slice(M - 40, M)
    check = B.gated_linear_fwd(x[rows].contiguous(), W, bias, save_z=True)
    zr = x[rows].double() @ W.double().T + bias.double()
    within(z[rows], zr, 72 * U * (x[rows].double().abs() @ W.double().abs().T + bias.double().abs()))
    assert float((y[rows].double() - check[0].double()).norm() / check[0].double().norm()) < 2.0 ** -8


GATED_KERNELS = [(1, 1, 384, "few rows gated 16x16"), (4249, 1, 8, "few rows gated 32x16"), (3, 4271, 392, "few rows gated 32x32"), (8507, 74, 64, "gemm cols gated 64x64/4 waves/4 stages"), (5481, 162, 384, "gemm cols gated 128x128/8 waves/3 stages"),
                 (141, 5711, 464, "gemm cols gated 128x128/8 waves/3 stages guard"), (524, 5757, 384, "gemm cols gated 128x256/8 waves/3 stages"), (2420, 1606, 400, "gemm cols gated 128x256/8 waves/3 stages guard"),
                 (5466, 350, 384, "gemm cols gated 256x128/8 waves/3 stages"), (11124, 129, 408, "gemm cols gated 256x128/8 waves/3 stages guard"), (10947, 334, 64, "gemm cols gated 256x256/8 waves/2 stages"),
                 (10947, 334, 384, "gemm cols gated 256x256/8 waves/2 stages"), (770, 5075, 392, "gemm cols gated 256x256/8 waves/2 stages guard"), (8523, 34, 384, "gemm cols gated 64x128/4 waves/3 stages"),
                 (9192, 37, 392, "gemm cols gated 64x128/4 waves/3 stages guard"), (8277, 1, 384, "gemm cols gated 64x64/4 waves/4 stages"), (8417, 3, 464, "gemm cols gated 64x64/4 waves/4 stages guard")]


@pytest.mark.parametrize("M,N,K,kernel", GATED_KERNELS)
def test_gated_fwd_every_kernel(B, M, N, K, kernel):
    import torch
    x, W, bias, _ = lin_inputs(M, 2 * N, K, M + K)
    for yt in (torch.bfloat16, torch.float32):
        with B.dry_run() as names:
            B.gated_linear_fwd(x, W, bias, out_dtype=yt, save_z=True)
            B.gated_linear_fwd(x, W, None, 0, out_dtype=yt)
        assert names == [kernel] * 2
        check_gated_fwd(B, x, W, bias, 3, yt)
        check_gated_fwd(B, x, W, None, 2, yt, save_z=False)


# ---- together ----------------------------------------------------------------------------------------------------------------
class FeedForward:
    """h + down(v act(g)), [v, g] = up(norm(h)), of a branch's result that comes onto the stream first"""

    def __init__(self, B, C, F, seed):
        import torch
        g = gen(seed)
        self.B, self.F = B, F
        self.ga = (1 + randn(g, C, scale=0.1)).bfloat16()
        self.wu, self.bu = randn(g, 2 * F, C, scale=1 / math.sqrt(C)).bfloat16(), randn(g, 2 * F, scale=0.1).bfloat16()
        self.wd, self.bd = randn(g, C, F, scale=1 / math.sqrt(F)).bfloat16(), randn(g, C, scale=0.1).bfloat16()
        if C % 16 == 0 and F % 16 == 0:
            self.wu8, self.wd8 = B.quantize_fp8(self.wu), B.quantize_fp8(self.wd)

    def serve(self, x, h):
        import torch
        B = self.B
        n, h = B.rmsnorm_fwd(x, self.ga, residual=h, out_dtype=torch.float8_e4m3fn)
        f = B.gated_linear_fp8_fwd(n, self.wu8, self.bu, out_dtype=torch.float8_e4m3fn)
        return B.linear_fp8_fwd(f, self.wd8, self.bd, residual=h, out_dtype=torch.float32)

    def train(self, x, h, dy):
        """The result, and gradients of x (and h), the norm's weight, both projections' weights and biases"""
        import torch
        B = self.B
        n, s, rstd = B.rmsnorm_fwd(x, self.ga, residual=h, stats=True)
        f, z = B.gated_linear_fwd(n, self.wu, self.bu, save_z=True)
        y = B.linear_fwd(f, self.wd, self.bd, residual=s, out_dtype=torch.float32)
        df, dwd, dbd = B.linear_bwd(dy, f, self.wd)
        dn, dwu, dbu = B.gated_linear_bwd(df, n, self.wu, z)
        dh, dga = B.rmsnorm_bwd(dn, s, rstd, self.ga, dres=dy)
        return y, dh, dga, dwu, dbu, dwd, dbd

    def plain(self, x, h, dy):
        import torch
        with torch.enable_grad():
            P = [t.double().requires_grad_(True) for t in (x, self.ga, self.wu, self.bu, self.wd, self.bd)]
            s = P[0] + h.double()
            n = s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt() * P[1]
            z = n @ P[2].T + P[3]
            y = s + (z[:, :self.F] * act64(z[:, self.F:], 3)) @ P[4].T + P[5]
            return (y.detach(), *torch.autograd.grad(y, P, dy.double()))


@pytest.mark.parametrize("M,C,F", [(1, 128, 320), (77, 144, 336), (640, 320, 1280), (333, 136, 520)])
def test_feed_forward(B, M, C, F):
    import torch
    ff = FeedForward(B, C, F, M)
    g = gen(M + 1)
    x, h, dy = randn(g, M, C).bfloat16(), randn(g, M, C, scale=2.0), randn(g, M, C)
    want = ff.plain(x, h, dy)
    # up to seven roundings to bf16 on the way to each gradient, 2^-8 each, independent
    for got, ref in zip(ff.train(x, h, dy), want):
        assert float((got.double() - ref).norm() / ref.norm()) <= math.sqrt(7) * 2.0 ** -8
    if C % 16 == 0 and F % 16 == 0:
        # of the branch: n, W and their products' gate and value, f and W: roundings to 8 bits, 2^-4 at most and independent, twice in each of value and gate (whose
        # slope times its argument is up to 1.2 times the activation where that is not small), then f's and the last W's
        branch = want[0] - (x.double() + h.double())
        got = ff.serve(x, h).double() - (x.double() + h.double())
        assert float((got - branch).norm() / branch.norm()) <= math.sqrt(2 + 2 * 1.44 + 2) * 2.0 ** -4


def test_feed_forward_captured_and_replayed(B):
    """Two graphs with workspaces of their own, replayed in turn with eager work between, inputs changed in place"""
    import torch
    C, F = 320, 640
    ff = FeedForward(B, C, F, 3)
    g = gen(8)
    for M in (3, 600):
        data = [(randn(g, M, C).bfloat16(), randn(g, M, C), randn(g, M, C)) for _ in range(2)]
        step = lambda x, h, dy: (ff.serve(x, h), *ff.train(x, h, dy))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for d in data:
                step(*d)
        torch.cuda.current_stream().wait_stream(s)
        graphs, outs = [], []
        for d in data:
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr):
                outs.append(step(*d))
            graphs.append(gr)
        for rep in range(4):
            for d in data:
                for t in d:
                    t.normal_()
            for gr in graphs:
                gr.replay()
            for d, o in zip(data, outs):
                assert all(torch.equal(a, b) for a, b in zip(o, step(*d)))
            torch.cuda.synchronize()


def test_feed_forward_on_two_streams(B):
    import torch
    ff = FeedForward(B, 320, 640, 4)
    g = gen(9)
    jobs = [(randn(g, M, 320).bfloat16(), randn(g, M, 320), randn(g, M, 320)) for M in (2000, 9)]
    work = lambda x, h, dy: (ff.serve(x, h), *ff.train(x, h, dy))
    want = [work(*j) for j in jobs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in jobs], [[], []]
    for rep in range(5):
        for s, j, o in zip(streams, jobs, got):
            with torch.cuda.stream(s):
                o.append(work(*j))
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        for r in o:
            assert all(torch.equal(a, b) for a, b in zip(r, w))


def test_the_same_operand_twice(B):
    """x and W, x and the residual, dy, h and dres one tensor"""
    import torch
    g = gen(21)
    for M in (9, 200, 700):
        x = rows8(B, g, M, 320, 0.1)
        check_linear8(B, x, x, None, 0, None, torch.float32)
        check_linear8(B, x, x, None, 3, None, torch.bfloat16)
    x = rows8(B, g, 64, 320, 0.1)
    for yt in (torch.float32, torch.bfloat16, torch.float8_e4m3fn):
        check_gated8(B, x, x, None, 3, yt)
    x = randn(g, 64, 64, scale=0.3).bfloat16()
    assert torch.equal(B.gated_linear_fwd(x, x.clone(), None, 3), B.gated_linear_fwd(x, x, None, 3))
    for a in (randn(g, 7, 515), randn(g, 2000, 1280)):
        y, h, rstd = B.rmsnorm_fwd(a, None, residual=a, stats=True)
        assert torch.equal(h, 2 * a)
        y2, _, _ = B.rmsnorm_fwd(a, None, residual=a.clone(), stats=True)
        assert torch.equal(y, y2)
        one, two = B.rmsnorm_bwd(a, a, rstd, None, dres=a), B.rmsnorm_bwd(a.clone(), a, rstd, None, dres=a.clone())
        assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


def test_two_launches_captured_with_one_workspace(B):
    """Two graphs that share a workspace, replayed one behind the other"""
    import torch
    M, N, K = 130, 640, 4112
    g = gen(22)
    need = B.lib().sd_gated_linear_fp8_workspace_bytes(M, N, K)
    assert need
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    src = [randn(g, M, K) for _ in range(2)]
    W = rows8(B, g, 2 * N, K, 1.3 / math.sqrt(K), 0.3)
    step = lambda a: B.gated_linear_fp8_fwd(B.quantize_fp8(a), W, out_dtype=torch.float8_e4m3fn, ws=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for a in src:
            step(a)
    torch.cuda.current_stream().wait_stream(s)
    graphs, outs = [], []
    for a in src:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(step(a))
        graphs.append(gr)
    for rep in range(4):
        for a in src:
            a.normal_()
        for gr in graphs:
            gr.replay()
        for a, o in zip(src, outs):
            w = step(a)
            assert torch.equal(o.q.view(torch.uint8), w.q.view(torch.uint8)) and torch.equal(o.scales.view(torch.uint8).contiguous(), w.scales.view(torch.uint8).contiguous())
        torch.cuda.synchronize()


@pytest.mark.parametrize("M,N,K", [(1, 10240, 5120), (16, 10240, 5120), (33, 5120, 5120), (64, 5120, 4096), (64, 1296, 5120), (7, 5120, 5120), (1, 16, 5120)])
def test_gated_fp8_of_few_rows_in_two_launches_keeps_all_of_a_sum(B, M, N, K):
    """The bytes are those of y in fp32, which is summed whole.  (Two products of 2^14 cancel, with smaller ones beside them of which the scaled MFMA would drop up to 2 each.)"""
    import torch
    g = gen(M + N)
    a, w = randn(g, M, K, scale=2.8), randn(g, 2 * N, K, scale=2.8)
    a[:, 0], a[:, 8], w[:, 0], w[:, 8] = 128.0, -128.0, 128.0, 128.0
    a[:, 128:] = 0                                # sums of 128 products: fp32 loses 136 2^-23 2^15, 0.6, at most
    x, W = B.quantize_fp8(a), B.quantize_fp8(w)
    with B.dry_run() as names:
        y = B.gated_linear_fp8_fwd(x, W, None, 0, out_dtype=torch.float8_e4m3fn)
    assert names[1] == "quantize" and ("wide" in names[0] or "few rows" in names[0])
    y = B.gated_linear_fp8_fwd(x, W, None, 0, out_dtype=torch.float8_e4m3fn)
    whole = B.quantize_fp8(B.gated_linear_fp8_fwd(x, W, None, 0, out_dtype=torch.float32))
    assert torch.equal(y.q.view(torch.uint8), whole.q.view(torch.uint8)) and torch.equal(y.scales.contiguous().view(torch.uint8), whole.scales.contiguous().view(torch.uint8))
    first = lambda r: B.Fp8Rows(r.q[:, :128], r.scales[:1])
    ref, slack = gated_ref(*product(first(x), first(W), None, True), 0)
    within_fp8(y, ref, slack)


def drops_low_bits(B, g, M, N, K):
    """Rows whose sums of products hold two of 2^14 that cancel, and beside them, in the same eights, smaller ones, of which the scaled MFMA drops up to 2 each"""
    a, w = randn(g, M, K, scale=2.8), randn(g, N, K, scale=2.8)
    a[:, 0], a[:, 8], w[:, 0], w[:, 8] = 128.0, -128.0, 128.0, 128.0
    return B.quantize_fp8(a), B.quantize_fp8(w)


@pytest.mark.parametrize("M,N,K", [(65, 65, 64), (300, 515, 80), (700, 333, 128), (2100, 640, 64), (8200, 1040, 80)])
def test_linear_fp8_whole_sums(B, M, N, K):
    import torch
    g = gen(M + N)
    x, W = drops_low_bits(B, g, M, N, K)
    bias, res = randn(g, N, scale=0.5).bfloat16(), randn(g, M, N, dtype=torch.bfloat16)
    z, ez = product(x, W, bias, True)
    y = B.linear_fp8_fwd(x, W, bias, residual=res, whole_sums=True)
    within(y, z + res.double(), ez + 2 * U * (z + res.double()).abs())
    assert torch.equal(y, B.linear_fp8_fwd(x, W, bias, residual=res, whole_sums=True))
    # y in fp32 is summed whole whether it is asked for or not
    assert torch.equal(B.linear_fp8_fwd(x, W, bias, 3, out_dtype=torch.float32, whole_sums=True), B.linear_fp8_fwd(x, W, bias, 3, out_dtype=torch.float32))


WHOLE_KERNELS = [(65, 144, 64, "gemm cols 8 bits wide gated to 8 bits 32x256/4 waves/3 stages guard"), (300, 1296, 128, "gemm cols 8 bits wide gated to 8 bits 32x256/4 waves/3 stages"),
                 (1500, 2560, 128, "gemm cols 8 bits wide gated to 8 bits 128x256/8 waves/3 stages"), (8200, 1040, 80, "gemm cols 8 bits wide gated to 8 bits 128x256/8 waves/3 stages guard"),
                 (500, 2064, 128, "gemm cols 8 bits wide gated to 8 bits 64x256/8 waves/3 stages"), (500, 2064, 112, "gemm cols 8 bits wide gated to 8 bits 64x256/8 waves/3 stages guard"), (64, 32896, 128, "gemm cols 8 bits wide gated to 8 bits 64x256/8 waves/3 stages")]


@pytest.mark.parametrize("M,N,K,kernel", WHOLE_KERNELS)
def test_gated_fp8_whole_sums(B, M, N, K, kernel):
    import torch
    g = gen(M + N)
    x, W = drops_low_bits(B, g, M, 2 * N, K)
    bias = randn(g, 2 * N, scale=0.5).bfloat16()
    for act in (0, 4):
        ref, slack = gated_ref(*product(x, W, bias, True), act)
        with B.dry_run() as names:
            B.gated_linear_fp8_fwd(x, W, bias, act, out_dtype=torch.float8_e4m3fn, whole_sums=True)
        assert names == [kernel]
        within_fp8(B.gated_linear_fp8_fwd(x, W, bias, act, out_dtype=torch.float8_e4m3fn, whole_sums=True), ref, slack)
        within(B.gated_linear_fp8_fwd(x, W, bias, act, whole_sums=True), ref, slack)
        within(B.gated_linear_fp8_fwd(x, W, bias, act, out_dtype=torch.float32, whole_sums=True), ref, slack)


@pytest.mark.parametrize("M,N,K", [(130, 640, 4112), (300, 1296, 5120)])
def test_gated_fp8_whole_sums_in_two_launches(B, M, N, K):
    import torch
    g = gen(M)
    x, W = rows8(B, g, M, K), rows8(B, g, 2 * N, K, 1.3 / math.sqrt(K), 0.3)
    y = B.gated_linear_fp8_fwd(x, W, None, 3, out_dtype=torch.float8_e4m3fn, whole_sums=True)
    want = B.quantize_fp8(B.gated_linear_fp8_fwd(x, W, None, 3, out_dtype=torch.float32))
    assert torch.equal(y.q.view(torch.uint8), want.q.view(torch.uint8)) and torch.equal(y.scales.contiguous().view(torch.uint8), want.scales.contiguous().view(torch.uint8))


@pytest.mark.parametrize("M,N,K", [(1500, 2560, 1296), (500, 2064, 272), (300, 1296, 640)])
def test_gated_fp8_whole_sums_of_usual_rows(B, M, N, K):
    """Steps, stages and scales of the kernels that only whole sums take"""
    import torch
    g = gen(K)
    x, W = rows8(B, g, M, K), rows8(B, g, 2 * N, K, 1.3 / math.sqrt(K), 0.3)
    bias = randn(g, 2 * N, scale=0.5).bfloat16()
    for act in (1, 3):
        ref, slack = gated_ref(*product(x, W, bias, True), act)
        within_fp8(B.gated_linear_fp8_fwd(x, W, bias, act, out_dtype=torch.float8_e4m3fn, whole_sums=True), ref, slack)


# ---- scales, NaN and the largest values in every kernel ------------------------------------------------------------------------
def with_rows(r, bytes_, q=None):
    """Rows in 8 bits with other scale bytes (and values)"""
    import torch
    M = r.q.shape[0]
    return B_rows(r.q if q is None else q, torch.nn.functional.pad(bytes_.to(torch.uint8), (0, -M % 4)).view(torch.float8_e8m0fnu)[:, :M])


def B_rows(q, s):
    from paper_2407_02031_amd import binding
    return binding.Fp8Rows(q, s)


def bytes_of(r):
    import torch
    return r.scales.contiguous().view(torch.uint8).int()


def spoiled(r, at):
    """A NaN among the scales of row at[0], and one among the values of row at[1]; +-448 everywhere in row at[2].  The rows that are NaN for it."""
    import torch
    s, q, bad = bytes_of(r), r.q.view(torch.uint8).clone(), torch.zeros(r.q.shape[0], dtype=torch.bool, device="cuda")
    K = q.shape[1]
    if len(at) > 0:
        s[-1, at[0]], bad[at[0]] = 255, True
    if len(at) > 1:
        q[at[1], K // 2], bad[at[1]] = 0x7f, True
    if len(at) > 2:
        q[at[2]] = 0x7e + 128 * (torch.arange(K, device="cuda") % 3 == 0).to(torch.uint8)
    return with_rows(r, s, q.view(torch.float8_e4m3fn)), bad


def at_the_end(r, at, high, shift):
    """Rows `at` with scale byte 254 and values +-1, or byte 0 and their values; the others' scales by 2^shift"""
    import torch
    s, q = (bytes_of(r) + shift).clamp(1, 250), r.q.view(torch.uint8).clone()
    for i in at:
        s[:, i] = 254 if high else 0
        if high:
            q[i] = 0x38 + (q[i] & 128)
    return with_rows(r, s, q.view(torch.float8_e4m3fn))


def check_ends(B, M, N, K, yt, gated, **kw):
    import torch
    g = gen(M + N + K + 1)
    x, W = rows8(B, g, M, K, 1.0, 2.0), rows8(B, g, 2 * N if gated else N, K, 1.3 / math.sqrt(K), 2.0)
    R = W.q.shape[0]
    some = lambda n: [i for i in sorted({n // 3, n // 2 + 1, n - 1, n // 5}) if 0 < i < n][:3]      # (row 0 is left alone)

    def check(x, W, bx, bw, lost=None):
        if gated:
            y = B.gated_linear_fp8_fwd(x, W, None, 0, out_dtype=yt, **kw)
            bw = bw[:N] | bw[N:]
        else:
            y = B.linear_fp8_fwd(x, W, out_dtype=yt, **kw)
        bad = bx[:, None] | bw[None, :]
        clean = lambda r: B_rows(torch.where(r.q.double().isnan(), 0.0, r.q.float()).to(torch.float8_e4m3fn), torch.where(r.scales.double().isnan(), 1.0, r.scales.float()).to(torch.float8_e8m0fnu))
        z, ez = product(clean(x), clean(W), None, yt == torch.float32 or kw.get("whole_sums", False))
        if lost is not None:
            ez = ez + lost
        ref, slack = gated_ref(z, ez, 0) if gated else (z, ez)
        over = ref.abs() + slack >= 2.0 ** 127        # (a product of value and gate near 2^128 and beyond: infinite, or its neighbour)
        assert int(over.sum()) <= 1e-4 * over.numel()
        if yt == torch.float8_e4m3fn:
            bad = bad | over
            assert torch.equal(y.q.double().isnan() | over, bad)
            ref, slack = torch.where(bad, 0.0, ref), torch.where(bad, 0.0, slack)
            within_fp8(B_rows(torch.where(bad, 0.0, y.q.float()).to(torch.float8_e4m3fn), y.scales), ref, slack)
        else:
            assert torch.equal(y.isnan(), bad)
            bad = bad | over
            within(torch.where(bad, 0.0, y), torch.where(bad, 0.0, ref), torch.where(bad, 0.0, slack))
    nx, nw = torch.zeros(M, dtype=torch.bool, device="cuda"), torch.zeros(R, dtype=torch.bool, device="cuda")
    check(*(p for a in zip(spoiled(x, some(M)), spoiled(W, some(R))) for p in a))
    for mine, other, first in ((x, W, True), (W, x, False)):
        at = some(mine.q.shape[0])
        for high, up, down in ((True, 50, -80), (False, -60, 100)):
            a, b = at_the_end(mine, at, high, up), at_the_end(other, [], False, down)
            # elements below 2^-126, of which bf16 holds multiples of 2^-133: off by 2^-134 at most
            lost = 2.0 ** -134 * values(b).abs().sum(1)
            if first:
                check(a, b, nx, nw, lost[None, :])
            else:
                check(b, a, nx, nw, lost[:, None])


@pytest.mark.parametrize("yt,M,N,K,kernel", LIN8_KERNELS + [("bfloat16", 700, 700, 256, "gemm cols 8 bits 64x64/4 waves/4 stages"), ("bfloat16", 2100, 640, 272, "gemm cols 8 bits 64x128/4 waves/3 stages guard")])
def test_linear_fp8_ends_in_every_kernel(B, yt, M, N, K, kernel):
    """NaN scales and values stay in their rows and columns; +-448 throughout; scale bytes 254 and 0; scales far apart in both operands"""
    import torch
    with B.dry_run() as names:
        B.linear_fp8_fwd(*(B.Fp8Rows(torch.empty(n, K, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((K + 127) // 128, (n + 3) // 4 * 4, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)[:, :n]) for n in (M, N)),
                         out_dtype=getattr(torch, yt))
    assert names == [kernel]
    check_ends(B, M, N, K, getattr(torch, yt), False)


@pytest.mark.parametrize("yt,M,N,K", [k[:4] for k in GATED8_KERNELS] + [("float8_e4m3fn", 130, 640, 4112)])
def test_gated_fp8_ends_in_every_kernel(B, yt, M, N, K):
    import torch
    check_ends(B, M, N, K, getattr(torch, yt), True)


@pytest.mark.parametrize("M,N,K", [k[:3] for k in WHOLE_KERNELS] + [(700, 336, 640)])
def test_whole_sums_ends_in_every_kernel(B, M, N, K):
    import torch
    check_ends(B, M, N, K, torch.float8_e4m3fn, True, whole_sums=True)
    check_ends(B, M, N, K, torch.bfloat16, True, whole_sums=True)
    check_ends(B, M, N, K, torch.bfloat16, False, whole_sums=True)


@pytest.mark.parametrize("M,N,kernel", [(256, 32, "few rows 8 bits 16x16"), (2100, 640, "gemm cols 8 bits wide 64x128/8 waves/3 stages")])
def test_widened_elements_are_those_of_bf16(B, M, N, kernel):
    """One element a product, of every scale byte up to 246: exact from 2^-126 on, the nearest multiple of 2^-133 below"""
    import torch
    K = 128
    q = torch.tensor([1, 2, 3, 7, 8, 9, 15, 16, 31, 48, 55, 56, 63, 64, 88, 112, 126, 0x81, 0x87, 0xb8, 0xfe], dtype=torch.uint8, device="cuda")[torch.arange(K, device="cuda") % 21].expand(M, K).contiguous()
    s = (torch.arange(M, device="cuda") % 247)[None]
    x = with_rows(B_rows(q.view(torch.float8_e4m3fn), None), s)
    w = torch.zeros(N, K, dtype=torch.uint8, device="cuda")
    w[torch.arange(N), torch.arange(N) % K] = 0x38
    held = (q.view(torch.float8_e4m3fn).double() * power(s[0] - 127)[:, None]).bfloat16().double()[:, torch.arange(N) % K]
    for t in (127 - 100, 127, 127 + 100):
        W = with_rows(B_rows(w.view(torch.float8_e4m3fn), None), torch.full((1, N), t, device="cuda"))
        with B.dry_run() as names:
            B.linear_fp8_fwd(x, W, out_dtype=torch.float32)
        assert names == [kernel]
        want = (held * 2.0 ** (t - 127)).float()
        y = B.linear_fp8_fwd(x, W, out_dtype=torch.float32)
        keep = (want.abs() >= 2.0 ** -126) & want.isfinite() | (want == 0)          # (results of less are the matrix core's to round)
        assert torch.equal(y[keep], want[keep]) and bool((y[~want.isfinite()].isinf()).all())


# ---- NaN and infinities on the way into 8 bits -----------------------------------------------------------------------------------
def same_but_nan(got, clean, bad):
    """Rows in 8 bits that are NaN in columns `bad` and, scales included, those of `clean` elsewhere"""
    import torch
    assert torch.equal(got.scales.contiguous().view(torch.uint8), clean.scales.contiguous().view(torch.uint8))
    assert got.q[:, bad].double().isnan().all()
    assert torch.equal(got.q[:, ~bad].contiguous().view(torch.uint8), clean.q[:, ~bad].contiguous().view(torch.uint8)) and not clean.q.double().isnan().any()


@pytest.mark.parametrize("M,N,K,whole,kernel", [
    (5, 528, 256, False, "wide gated to 8 bits 32x256"), (100, 528, 256, False, "gated to 8 bits 64x256"), (9309, 528, 144, False, "gated to 8 bits 256x256"), (4200, 528, 256, False, "gated to 8 bits 128x256"), (8200, 1040, 144, False, "gated to 8 bits 256x256"),
    (300, 528, 144, True, "wide gated to 8 bits 32x256"), (1900, 528, 144, True, "wide gated to 8 bits 64x256"), (3800, 528, 256, True, "wide gated to 8 bits 128x256"), (130, 528, 4112, False, "quantize"), (5, 528, 5120, False, "quantize")])
def test_gated_fp8_bias_that_is_not_finite(B, M, N, K, whole, kernel):
    """Columns whose bias, the value's or the gate's, is NaN or infinite, in either half of a block, some of a block and all of it: NaN, and the others' bytes and scales are those of a call where these columns are zero"""
    import torch
    g = gen(M)
    columns = [0, 5, 62, 64, 101, 127] + [128 + 17] + [256 + 70] + list(range(384, 512)) + [N - 1, N - 16]
    bad = torch.zeros(N, dtype=torch.bool, device="cuda")
    bad[columns] = True
    w = randn(g, 2 * N, K, scale=1.3 / math.sqrt(K))
    w[:N][bad] = 0
    x, W, bias = B.quantize_fp8(randn(g, M, K)), B.quantize_fp8(w), randn(g, 2 * N, scale=0.5).bfloat16()
    bias[:N][bad] = 0
    run = lambda b, act: B.gated_linear_fp8_fwd(x, W, b, act, out_dtype=torch.float8_e4m3fn, whole_sums=whole)
    with B.dry_run() as names:
        run(bias, 0)
    assert kernel in names[-1]
    for act in (0, 3, 1):
        clean = run(bias, act)
        for values_of, gate_of in (((math.inf,), ()), ((-math.inf,), ()), ((math.nan,), ()), ((), (math.nan,)), ((), (math.inf,)), ((math.nan, math.inf, -math.inf), (math.nan, math.inf))):
            b = bias.clone()
            for i, c in enumerate(columns):
                if values_of and (i % 2 == 0 or not gate_of):
                    b[c] = values_of[i % len(values_of)]
                else:
                    b[N + c] = gate_of[i % len(gate_of)]
            same_but_nan(run(b, act), clean, bad)


@pytest.mark.parametrize("C", [16, 64, 128, 320, 512, 768, 1280, 2048, 4096, 8192, 16384])
def test_rmsnorm_to_8_bits_of_what_is_not_finite(B, C):
    """A weight that is NaN or infinite: its column is NaN, and the others' bytes and scales are those of a weight of zero there; a row that holds a NaN is NaN, with the least scale"""
    import torch
    for xt, rt in (("bfloat16", "float32"), ("float32", None)):
        for M in (1, 37):
            x, r, ga, g = rms_inputs(M, C, xt, rt, C + M)
            columns = sorted({0, 3, min(C - 1, 70), C // 2 + 1, C - 1} | (set(range(128, 256)) if C > 256 else set()))
            bad = torch.zeros(C, dtype=torch.bool, device="cuda")
            bad[columns] = True
            run = lambda w, x=x: (lambda o: o[0] if r is not None else o)(B.rmsnorm_fwd(x, w, residual=r, out_dtype=torch.float8_e4m3fn))
            zero = ga.clone()
            zero[bad] = 0
            clean = run(zero)
            for what in ((math.inf,), (math.nan,), (-math.inf, math.nan, math.inf)):
                w = zero.clone()
                for i, c in enumerate(columns):
                    w[c] = what[i % len(what)]
                same_but_nan(run(w), clean, bad)
            spoiled_x = x.clone()
            spoiled_x[M // 2, C // 3] = math.nan
            got, whole = run(ga, spoiled_x), run(ga)
            rows = torch.arange(M, device="cuda") != M // 2
            assert got.q[M // 2].double().isnan().all() and (got.scales.contiguous().view(torch.uint8)[:, M // 2] == 1).all()
            assert torch.equal(got.q.view(torch.uint8)[rows], whole.q.view(torch.uint8)[rows])


@pytest.mark.parametrize("M,N,K", [(1003, 317, 648), (2048, 640, 320), (600, 2560, 1280)])
@pytest.mark.parametrize("act", [1, 2, 3])
def test_gated_bwd_loses_the_rounding_of_dz_alone(B, M, N, K, act):
    """Against products of dz as bf16 holds it: what is left is the results' own rounding, sums in fp32, and dz that fp32 rounds to the other side of a tie (1e-6 of it off, steps of 2^-8 apart: one in a thousand, 2^-8 each)"""
    import torch
    x, W, _, g = lin_inputs(M, 2 * N, K, M + N)
    dy, z = randn(g, M, N).bfloat16(), randn(g, M, 2 * N, scale=1.5).bfloat16()
    zz = z.double().requires_grad_(True)
    dz = torch.autograd.grad(zz[:, :N] * act64(zz[:, N:], act), zz, dy.double())[0]
    held = dz.bfloat16().double()
    off = lambda a, ref: float((a.double() - ref).norm() / ref.norm())
    dx, dW, _ = B.gated_linear_bwd(dy, x, W, z, act, dw_dtype=torch.float32)
    rx, rw = held @ W.double(), held.T.contiguous() @ x.double()
    assert off(dW, rw) <= math.sqrt(1e-3) * 2.0 ** -8 and off(dx, rx) <= off(rx.bfloat16(), rx) + math.sqrt(1e-3) * 2.0 ** -8
    # ... and dz's rounding, uniform in steps of 2^-8 to 2^-7 of it, is what it costs
    assert 1e-3 < off(rw, dz.T.contiguous() @ x.double()) < 2.0 ** -9


@pytest.mark.parametrize("M,N,K,kernel", [k[1:] for k in LIN8_KERNELS if k[0] == "float32"] + [(1000, 500, 144, "few rows 8 bits 64x32")])
def test_linear_fp8_whole_sums_every_kernel(B, M, N, K, kernel):
    """In bf16, with bias and residual, from the kernels that y in fp32 has"""
    import torch
    g = gen(M + K)
    x, W = rows8(B, g, M, K), rows8(B, g, N, K, 1.3 / math.sqrt(K), 0.3)
    bias, res = randn(g, N, scale=0.5).bfloat16(), randn(g, M, N).bfloat16()
    with B.dry_run() as names:
        B.linear_fp8_fwd(x, W, bias, 1, residual=res, whole_sums=True)
    assert names == [kernel]
    z, ez = product(x, W, bias, True)
    for r in (res, None):
        ref = act64(z, 3) + (r.double() if r is not None else 0)
        within(B.linear_fp8_fwd(x, W, bias, 3, residual=r, whole_sums=True), ref, 1.13 * ez + 4e-7 * (1 + z.abs()) + 2 * U * ref.abs())


@pytest.mark.parametrize("M,N,K,kernel", [k[1:] for k in GATED8_KERNELS if k[0] == "float32"])
def test_gated_fp8_whole_sums_every_kernel(B, M, N, K, kernel):
    import torch
    g = gen(M + K)
    x, W = rows8(B, g, M, K), rows8(B, g, 2 * N, K, 1.3 / math.sqrt(K), 0.3)
    bias = randn(g, 2 * N, scale=0.5).bfloat16()
    with B.dry_run() as names:
        B.gated_linear_fp8_fwd(x, W, bias, 3, whole_sums=True)
    assert names == [kernel]
    within(B.gated_linear_fp8_fwd(x, W, bias, 3, whole_sums=True), *gated_ref(*product(x, W, bias, True), 3))

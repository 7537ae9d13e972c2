"""Layer norm, rotary positions and the linear layer, forward and backward, against their formulas in 64 bits on an MI355X.

Tolerances are bounds: a rounding to the output's type is off by half a step, eps / 2 relative to the value; an fp32 operation by
U = 2^-24; a sum of n terms added up in steps of depth d by d U times the sum of their absolute values."""
import math

import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2407_02031_amd import binding
    return binding


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def within(got, ref, slack, half=True):
    """got (bf16 or fp32) lies within its type's rounding of ref, and `slack` more"""
    import torch
    step = torch.finfo(got.dtype).eps / 2 if half else 0.0
    off = (got.double() - ref).abs()
    # what is rounded is ref + up to slack
    bad = ~(off <= step * (ref.abs() + slack) + slack)
    assert not bad.any(), (int(bad.sum()), bad.numel(), float((off / (step * ref.abs() + slack + 1e-300)).max()))


# ---- layer norm ------------------------------------------------------------------------------------------------------------
def ln_inputs(M, C, xt, seed, offset=0.5):
    import torch
    g = gen(seed)
    x = torch.randn(M, C, generator=g, device="cuda") * 1.5 + offset
    return x.to(xt), (1 + 0.3 * torch.randn(C, generator=g, device="cuda")).bfloat16(), (0.3 * torch.randn(C, generator=g, device="cuda")).bfloat16(), g


def check_ln_fwd(B, x, gamma, beta, yt, eps=1e-5):
    import torch
    y, mean, rstd = B.layernorm_fwd(x, gamma, beta, eps, out_dtype=yt, stats=True)
    d = x.double()
    m = d.mean(-1, keepdim=True)
    r = ((d - m).square().mean(-1, keepdim=True) + eps).rsqrt()
    n = (d - m) * r
    ga, be = (gamma.double() if gamma is not None else torch.ones_like(n[0])), (beta.double() if beta is not None else torch.zeros_like(n[0]))
    # sums in at most 40 steps (chunks of a thread, lanes, wavefronts): the mean is off by 40 U of the deviations' mean, the variance by 80 U of itself, n by
    # half of that and its own four operations
    within(y, n * ga + be, 64 * U * ((n.abs() + 1) * ga.abs() + be.abs()))
    within(mean, m[..., 0], 41 * U * ((d - m).abs().mean(-1)) + U * m[..., 0].abs())
    within(rstd, r[..., 0], 48 * U * r[..., 0])
    again = B.layernorm_fwd(x, gamma, beta, eps, out_dtype=yt)
    assert torch.equal(again.view(torch.uint8), y.view(torch.uint8))
    return y, mean, rstd


LENGTHS = [4, 5, 63, 255, 256, 257, 768, 1001, 1280, 1283, 2048, 2049, 4095, 4096, 5000, 8191, 8192, 8193, 16384]


@pytest.mark.parametrize("C", LENGTHS)
@pytest.mark.parametrize("xt,yt", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("float32", "float32"), ("bfloat16", "float32")])
def test_layernorm_fwd(B, C, xt, yt):
    import torch
    for M in (1, 7):
        x, ga, be, _ = ln_inputs(M, C, getattr(torch, xt), C + M)
        check_ln_fwd(B, x, ga, be, getattr(torch, yt))
    check_ln_fwd(B, x, None, None, getattr(torch, yt))
    check_ln_fwd(B, x, ga, None, getattr(torch, yt))
    check_ln_fwd(B, x, None, be, getattr(torch, yt))


@pytest.mark.parametrize("C", [320, 1155, 3000])
def test_layernorm_fwd_hard_rows(B, C):
    """A large offset; one element far from the rest, the first or another; constant rows; zeros; infinities and NaN stay in their rows."""
    import torch
    x, ga, be, g = ln_inputs(12, C, torch.float32, 5)
    x[0] += 4096.0
    x[1, 0] = 30000.0
    x[2, C // 2] = -1e6
    x[3] = 3.25
    x[4] = 0.0
    x[5] *= 1e-4
    x[6] *= 1e15
    check_ln_fwd(B, x[:7].contiguous(), ga, be, torch.float32)
    x[7, 3], x[8, C - 1], x[9, 0] = math.nan, math.inf, -math.inf
    y = B.layernorm_fwd(x, ga, be, out_dtype=torch.bfloat16)
    assert torch.isnan(y[7:10].float()).all() and torch.isfinite(y[10:].float()).all() and torch.isfinite(y[:7].float()).all()


def check_ln_bwd(B, x, dy, gamma, mean, rstd):
    import torch
    dx, dg, db = B.layernorm_bwd(dy, x, mean, rstd, gamma)
    M, C = x.shape
    r = rstd.double()[:, None]
    n = (x.double() - mean.double()[:, None]) * r
    g = dy.double() * (gamma.double() if gamma is not None else 1.0)
    c1, c2 = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
    ref = r * (g - c1 - n * c2)
    # n: three operations on x, whose own size may exceed the difference's
    en = 4 * U * (n.abs() + r * x.double().abs())
    slack = r * (64 * U * (g.abs() + g.abs().mean(1, keepdim=True) + n.abs() * (g * n).abs().mean(1, keepdim=True))
                 + en * c2.abs() + n.abs() * (g.abs() * en).mean(1, keepdim=True))
    within(dx, ref, slack)
    depth = M / 256 + 64          # rows of a thread, wavefronts of a workgroup, workgroups
    within(dg, (dy.double() * n).sum(0), depth * U * (dy.double() * n).abs().sum(0) + (dy.double().abs() * en).sum(0))
    within(db, dy.double().sum(0), depth * U * dy.double().abs().sum(0))
    dx2, dg2, db2 = B.layernorm_bwd(dy, x, mean, rstd, gamma)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2) and torch.equal(db, db2)
    only, a, b = B.layernorm_bwd(dy, x, mean, rstd, gamma, weight_grads=False)
    assert torch.equal(only, dx) and a is None and b is None
    return dx, dg, db


@pytest.mark.parametrize("C", LENGTHS)
@pytest.mark.parametrize("xt,yt", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("float32", "float32"), ("bfloat16", "float32")])
def test_layernorm_bwd(B, C, xt, yt):
    import torch
    for M in (1, 6, 2061 if C < 2100 else 517):
        x, ga, be, g = ln_inputs(M, C, getattr(torch, xt), C + M)
        dy = torch.randn(M, C, generator=g, device="cuda").to(getattr(torch, yt))
        _, mean, rstd = B.layernorm_fwd(x, ga, be, stats=True)
        check_ln_bwd(B, x, dy, ga, mean, rstd)
    check_ln_bwd(B, x, dy, None, mean, rstd)


def test_layernorm_gradients_against_differences(B):
    """<dx, v> against the central difference of <y, dy> along v, y in 64 bits: the formula itself."""
    import torch
    x, ga, be, g = ln_inputs(9, 77, torch.float32, 3)
    dy, v = (torch.randn(9, 77, generator=g, device="cuda") for _ in range(2))
    _, mean, rstd = B.layernorm_fwd(x, ga, be, stats=True, out_dtype=torch.float32)
    dx, dg, db = B.layernorm_bwd(dy, x, mean, rstd, ga)

    def f(a, gm, bt):
        m = a.mean(1, keepdim=True)
        return (((a - m) * ((a - m).square().mean(1, keepdim=True) + 1e-5).rsqrt() * gm + bt) * dy.double()).sum()
    X, G, T, h = x.double(), ga.double(), be.double(), 1e-5
    w = torch.randn(77, generator=g, device="cuda").double()
    for num, ana in (((f(X + h * v.double(), G, T) - f(X - h * v.double(), G, T)) / (2 * h), (dx.double() * v.double()).sum()),
                     ((f(X, G + h * w, T) - f(X, G - h * w, T)) / (2 * h), (dg.double() * w).sum()),
                     ((f(X, G, T + h * w) - f(X, G, T - h * w)) / (2 * h), (db.double() * w).sum())):
        # differences: h^2 of third derivatives and 1e-16 / h of the sum, below 1e-8; fp32 results: 1e-6 of terms of order 1, 693 of them
        assert abs(float(num - ana)) < 1e-4 * (1 + abs(float(num)))


def test_layernorm_offsets_past_32_bits(B):
    import torch
    M, C = 530000, 4100
    x = torch.empty(M, C, dtype=torch.bfloat16, device="cuda")
    x.copy_(torch.randn(1, C, generator=gen(1), device="cuda").expand(M, C))
    x[-3:] *= 2
    x[-1, 0] = 50
    y, mean, rstd = B.layernorm_fwd(x, stats=True)
    d = x[-3:].double()
    m = d.mean(1, keepdim=True)
    n = (d - m) * ((d - m).square().mean(1, keepdim=True) + 1e-5).rsqrt()
    within(y[-3:], n, 64 * U * (n.abs() + 1))
    assert torch.equal(y[0], y[M // 2]) and torch.equal(y[0], y[M - 4])
    dx, dg, db = B.layernorm_bwd(y, x, mean, rstd, out=y)      # in the gradient's place
    tail = x[-3:].clone()
    dx2, _, _ = B.layernorm_bwd(B.layernorm_fwd(tail), tail, mean[-3:].clone(), rstd[-3:].clone())
    assert torch.equal(dx[-3:], dx2)


def test_layernorm_in_place_and_empty(B):
    import torch
    x, ga, be, g = ln_inputs(37, 1283, torch.bfloat16, 9)
    ref, mean, rstd = B.layernorm_fwd(x, ga, be, stats=True)
    dy = torch.randn(37, 1283, generator=g, device="cuda").bfloat16()
    dref, _, _ = B.layernorm_bwd(dy, x, mean, rstd, ga)
    a, b = x.clone(), x.clone()
    assert torch.equal(B.layernorm_fwd(a, ga, be, out=a), ref)
    assert torch.equal(B.layernorm_bwd(dy, b, mean, rstd, ga, out=b)[0], dref)
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = B.layernorm_fwd(e, stats=True)
    dx, dg, db = B.layernorm_bwd(e, e, mean, rstd)
    assert y.shape == (0, 64) and not dg.any() and not db.any() and dg.shape == (64,)


# ---- rotary positions ------------------------------------------------------------------------------------------------------
def rope_ref(x, pos, pairs, theta, layout, whole, sign):
    """By the definition, pair by pair, in 64 bits; and a bound of what fp32 cosines and products are off by"""
    import torch
    y, bound = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    R, first, p0 = sum(pairs), 0, 0
    for a, n in enumerate(pairs):
        for i in range(n):
            p = p0 + i
            lo, hi = ((2 * p, 2 * p + 1), (p, p + R), (2 * p0 + i, 2 * p0 + n + i))[layout]
            ang = pos[..., a].double() * theta ** -(p / R if whole else i / n)
            c, s = torch.cos(ang)[:, :, None], sign * torch.sin(ang)[:, :, None]
            u, v = x[..., lo].double(), x[..., hi].double()
            y[..., lo], y[..., hi] = u * c - v * s, u * s + v * c
            # the turn's fraction rounded (pi U of angle), cosine and sine (2 U each), two products and a sum
            bound[..., lo] = bound[..., hi] = 8 * U * (u.abs() + v.abs())
        p0 += n
    return y, bound


def rope_case(B, Bn, T, Hq, Hk, D, pairs, layout, whole=False, theta=1e4, dt="bfloat16", packed=True, shared=False, far=1.0, seed=0):
    import torch
    g = gen(seed)
    dt = getattr(torch, dt)
    buf = torch.randn(Bn, T, (Hq + 2 * Hk) * D, generator=g, device="cuda").to(dt)
    q, k = buf[..., :Hq * D].unflatten(-1, (Hq, D)), buf[..., Hq * D:(Hq + Hk) * D].unflatten(-1, (Hk, D)) if Hk else None
    if not packed:
        q, k = q.contiguous(), k.contiguous() if Hk else None
    pos = (torch.rand(1 if shared else Bn, T, len(pairs), generator=g, device="cuda") * 100 * far).round_(decimals=1)
    rope = B.Rope(D, pairs, theta, layout, whole)
    before = buf.clone()
    for fn, sign in ((B.rope_fwd, 1.0), (B.rope_bwd, -1.0)):
        yq, yk = fn(rope, pos, q, k)
        for x, y in ((q, yq), (k, yk)):
            if x is None:
                assert y is None
                continue
            assert y.is_contiguous() and y.shape == x.shape and y.dtype == x.dtype
            ref, bound = rope_ref(x, pos.expand(Bn, T, -1), pairs, theta, layout, whole, sign)
            within(y, ref, bound)
            R = sum(pairs)
            assert torch.equal(y[..., 2 * R:], x[..., 2 * R:])
    assert torch.equal(buf, before)
    # in place, in the packed rows: the same bits, and nothing else touched
    if packed:
        yq, yk = B.rope_fwd(rope, pos, q, k)
        B.rope_fwd(rope, pos, q, k, q_out=q, k_out=k)
        assert torch.equal(q, yq) and (k is None or torch.equal(k, yk))
        assert torch.equal(buf[..., (Hq + Hk) * D:], before[..., (Hq + Hk) * D:])


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("layout", [0, 1, 2])
@pytest.mark.parametrize("Bn,T,Hq,Hk,D,pairs", [
    (1, 1, 1, 0, 8, (4,)), (1, 1, 20, 20, 64, (16, 16)), (2, 33, 3, 1, 64, (16, 16)), (3, 5, 2, 2, 128, (16, 24, 24)), (2, 70, 5, 5, 72, (12, 12, 12)),
    (1, 9, 24, 8, 128, (13, 30, 21)), (2, 17, 1, 1, 256, (128,)), (1, 130, 7, 7, 40, (3, 7, 4, 5)), (2, 3, 4, 2, 96, (8, 8)), (1, 4, 3, 3, 88, (11, 10)),
    (2, 1, 256, 256, 16, (4, 4)), (1, 50, 1, 0, 24, (1, 2, 3))])
def test_rope(B, Bn, T, Hq, Hk, D, pairs, layout, dt):
    rope_case(B, Bn, T, Hq, Hk, D, pairs, layout, dt=dt, seed=D + T)


@pytest.mark.parametrize("layout", [0, 1, 2])
def test_rope_variants(B, layout):
    rope_case(B, 2, 40, 4, 2, 128, (16, 24, 24), layout, whole=True, theta=1e6, dt="float32")
    rope_case(B, 2, 40, 4, 2, 64, (16, 16), layout, shared=True, packed=False)
    rope_case(B, 2, 40, 4, 4, 64, (32,), layout, far=1e5, dt="float32")         # positions of ten million
    rope_case(B, 3, 700, 2, 1, 64, (8, 12, 12), layout, packed=False, theta=100.0)


def test_rope_special_values_and_gradient(B):
    """Infinities and NaN reach their pair alone; the unturned rest is copied bit by bit; the backward pass is the transpose."""
    import torch
    g = gen(4)
    q = torch.randn(1, 6, 2, 64, generator=g, device="cuda")
    pos = torch.rand(6, 1, generator=g, device="cuda") * 50
    r = B.Rope(64, [16], layout=B.SD_ROPE_HALVES)
    q[0, 1, 0, 3], q[0, 2, 1, 40], q[0, 3, 0, 50], q[0, 4, 1, 33] = math.nan, math.inf, math.nan, -0.0
    y, _ = B.rope_fwd(r, pos, q)
    bad = torch.isnan(y) | torch.isinf(y)
    want = torch.zeros_like(bad)
    want[0, 1, 0, 3] = want[0, 1, 0, 19] = want[0, 2, 1, 40] = want[0, 3, 0, 50] = True
    assert torch.equal(bad, want) and torch.equal(y[..., 32:].view(torch.int32), q[..., 32:].view(torch.int32))
    u, v = (torch.randn(2, 50, 3, 64, generator=g, device="cuda") for _ in range(2))
    p = torch.rand(2, 50, 2, generator=g, device="cuda") * 1000
    r = B.Rope(64, [20, 12], layout=B.SD_ROPE_AXIS_HALVES)
    a = (B.rope_fwd(r, p, u)[0].double() * v.double()).sum()
    b = (u.double() * B.rope_bwd(r, p, v)[0].double()).sum()
    # each product is off by at most 9 U of |u| |v| over its pair
    assert abs(float(a - b)) <= 40 * U * float((u.double().abs() * v.double().abs()).sum()) * 2


def test_rope_rows_far_apart(B):
    import torch
    D, ld, T = 64, 9 << 20, 260
    buf = torch.zeros(T * ld, dtype=torch.bfloat16, device="cuda")
    q = torch.as_strided(buf, (1, T, 2, D), (T * ld, ld, D, 1))
    q.copy_(torch.randn(1, T, 2, D, generator=gen(2), device="cuda"))
    pos = torch.arange(T, device="cuda", dtype=torch.float32)[:, None]
    r = B.Rope(D, [32])
    y, _ = B.rope_fwd(r, pos, q)
    y2, _ = B.rope_fwd(r, pos, q.contiguous())
    assert torch.equal(y, y2) and (T - 1) * ld > 2 ** 31
    B.rope_fwd(r, pos, q, q_out=q)
    assert torch.equal(q, y)


# ---- linear layer ----------------------------------------------------------------------------------------------------------
def act64(z, act):
    import torch
    if act == 1:
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if act == 2:
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if act == 3 else z.clamp(min=0) if act == 4 else z


def lin_inputs(M, N, K, seed):
    import torch
    g = gen(seed)
    return torch.randn(M, K, generator=g, device="cuda").bfloat16(), (torch.randn(N, K, generator=g, device="cuda") * 1.3 / math.sqrt(K)).bfloat16(), \
        (0.5 * torch.randn(N, generator=g, device="cuda")).bfloat16(), g


def check_lin_fwd(B, x, W, bias, act, res, yt, save_z):
    import torch
    out = B.linear_fwd(x, W, bias, act, residual=res, out_dtype=yt, save_z=save_z)
    y, zk = out if save_z else (out, None)
    K = x.shape[1]
    xd, wd = x.double(), W.double()
    z = xd @ wd.T + (bias.double() if bias is not None else 0)
    # every one of K products may be rounded into the sum; the activations' slopes are below 1.13, their own error below 4e-7 (1 + |z|)
    ez = (K + 8) * U * (xd.abs() @ wd.abs().T + (bias.double().abs() if bias is not None else 0))
    ref = act64(z, act) + (res.double() if res is not None else 0)
    within(y, ref, 1.13 * ez + 4e-7 * (1 + z.abs()) * (act > 0) + 2 * U * ref.abs())
    if save_z:
        within(zk, z, ez)
    return y


SIZES = [(1, 8, 8), (1, 5120, 64), (2, 1, 64), (3, 31, 72), (16, 130, 640), (17, 64, 200), (64, 64, 64), (65, 65, 136), (129, 317, 648), (200, 256, 320), (300, 515, 1024), (1000, 36, 72)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("yt", ["bfloat16", "float32"])
def test_linear_fwd(B, M, N, K, yt):
    import torch
    yt = getattr(torch, yt)
    x, W, bias, g = lin_inputs(M, N, K, M + N + K)
    res = torch.randn(M, N, generator=g, device="cuda").to(yt)
    for act in range(5):
        check_lin_fwd(B, x, W, bias, act, res, yt, True)
        check_lin_fwd(B, x, W, bias, act, None, yt, False)
    check_lin_fwd(B, x, W, None, 1, res, yt, False)
    check_lin_fwd(B, x, W, None, 0, res, yt, False)
    # the residual's place
    ref = B.linear_fwd(x, W, bias, 3, residual=res, out_dtype=yt)
    assert torch.equal(B.linear_fwd(x, W, bias, 3, residual=res, out=res), ref)


@pytest.mark.parametrize("M,N,K", [(4133, 640, 320), (2048, 1280, 648), (8192, 640, 1280), (1976, 1280, 1280), (700, 5120, 640), (4096, 5120, 2056), (9000, 321, 128), (5003, 5160, 64)])
def test_linear_fwd_large(B, M, N, K):
    import torch
    x, W, bias, g = lin_inputs(M, N, K, M)
    res = torch.randn(M, N, generator=g, device="cuda")
    check_lin_fwd(B, x, W, bias, 2, None, torch.bfloat16, True)
    check_lin_fwd(B, x, W, bias, 1, res, torch.float32, False)
    check_lin_fwd(B, x, W, bias, 0, res, torch.float32, False)


@pytest.mark.parametrize("M,N,K,kernel", [
    (16, 333, 648, "linear rows 16x16"), (31, 130, 1000, "linear rows 32x16"), (77, 1493, 200, "linear rows 32x32"), (500, 999, 72, "linear rows 64x32"), (9031, 8, 16, "linear rows 64x32"),
    (22, 64, 320, "thin 32x32/0"), (33, 4288, 320, "thin 32x64/0"), (97, 4736, 1088, "thin 64x64/0"), (17, 76, 192, "gemm16 64x80/0"), (681, 2752, 64, "gemm16 64x160/0"), (5028, 832, 128, "gemm16 128x160/0"),
    (588, 899, 64, "gemm act 64x128/4 waves/3 stages"), (588, 899, 72, "gemm act 64x128/4 waves/3 stages guard"), (9235, 796, 64, "gemm act 128x128/4 waves/2 stages"),
    (9235, 792, 24, "gemm act 128x128/4 waves/2 stages guard"), (6555, 1283, 128, "gemm act 128x160/4 waves/2 stages"), (2770, 2986, 8, "gemm act 128x160/4 waves/2 stages guard"),
    (6940, 1088, 192, "gemm act 256x128/8 waves/3 stages"), (11162, 593, 24, "gemm act 256x128/8 waves/3 stages guard"), (8281, 453, 256, "gemm act 128x256/8 waves/3 stages"), (8434, 401, 72, "gemm act 128x256/8 waves/3 stages guard")])
def test_linear_fwd_every_kernel(B, M, N, K, kernel):
    """Each kernel with and without z and residual, results of both types; the choice does not depend on them."""
    import torch
    x, W, bias, g = lin_inputs(M, N, K, M + K)
    for yt in (torch.bfloat16, torch.float32):
        res = torch.randn(M, N, generator=g, device="cuda").to(yt)
        with B.dry_run() as names:
            B.linear_fwd(x, W, bias, 1, residual=res, out_dtype=yt, save_z=True)
            B.linear_fwd(x, W, None, 0, out_dtype=yt)
        assert names == [kernel] * 2
        check_lin_fwd(B, x, W, bias, 3, res, yt, True)
        check_lin_fwd(B, x, W, None, 1, None, yt, True)
        check_lin_fwd(B, x, W, bias, 0, res, yt, False)


def check_lin_bwd(B, dy, x, W, z, act, dwt):
    import torch
    M, K = x.shape
    N = W.shape[0]
    dx, dW, db = B.linear_bwd(dy, x, W, z, act, dw_dtype=dwt)
    zz = z.double().requires_grad_(True) if act else None
    dz = dy.double()
    if act:
        dz = torch.autograd.grad(act64(zz, act), zz, dz)[0]
    # slopes: below 1.13, their own error below 1e-6; dz rounded to bf16; sums of N, or M, products
    ez = 2.0 ** -8 * dz.abs() + 1.01 * (1e-6 if act else U) * dy.double().abs()
    plain = act == 0 and dy.dtype == torch.bfloat16
    if plain:
        ez = torch.zeros_like(dz)
    wd, xd = W.double(), x.double()
    rx, rw = dz @ wd, dz.T @ xd
    within(dx, rx, ez @ wd.abs() + (N + 8) * U * (dz.abs() @ wd.abs()))
    within(dW, rw, ez.T @ xd.abs() + (M + 8) * U * (dz.abs().T @ xd.abs()))
    # roundings are independent of each other: together they are no more than half a step of the whole, the output's another
    for got, ref in ((dx, rx), (dW, rw)):
        own = torch.finfo(got.dtype).eps / 2
        if ref.norm() > 0 and min(M, N) > 30:
            assert float((got.double() - ref).norm() / ref.norm()) <= math.hypot(2.0 ** -8 * (not plain), own) + 1e-5
    within(db, dz.sum(0), (1e-6 if act else 0) * dy.double().abs().sum(0) + (M / 64 + 40) * U * dz.abs().sum(0))
    again = B.linear_bwd(dy, x, W, z, act, dw_dtype=dwt)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dW, db)))
    for i in range(3):
        part = B.linear_bwd(dy, x, W, z, act, grads=[j == i for j in range(3)], dw_dtype=dwt)
        assert all((p is None) if j != i else torch.equal(p, (dx, dW, db)[i]) for j, p in enumerate(part))


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("yt", ["bfloat16", "float32"])
def test_linear_bwd(B, M, N, K, yt):
    import torch
    x, W, bias, g = lin_inputs(M, N, K, M + N + K)
    dy = torch.randn(M, N, generator=g, device="cuda").to(getattr(torch, yt))
    z = (1.5 * torch.randn(M, N, generator=g, device="cuda")).bfloat16()
    for act in range(5):
        check_lin_bwd(B, dy, x, W, z if act else None, act, torch.bfloat16 if act % 2 else torch.float32)


@pytest.mark.parametrize("M,N,K", [(4133, 640, 320), (2048, 1288, 648), (8192, 320, 1280), (5000, 64, 64), (60, 5120, 1280), (1, 4096, 2048)])
def test_linear_bwd_large(B, M, N, K):
    import torch
    x, W, bias, g = lin_inputs(M, N, K, M)
    dy = torch.randn(M, N, generator=g, device="cuda").bfloat16()
    z = (1.5 * torch.randn(M, N, generator=g, device="cuda")).bfloat16()
    check_lin_bwd(B, dy, x, W, z, 2, torch.bfloat16)
    check_lin_bwd(B, dy, x, W, None, 0, torch.float32)


@pytest.mark.parametrize("M,N,K,launches", [
    (300, 64, 64, "gemm bwd 64x128/4 waves/3 stages guard, 1 of dW, 1 of dx"), (64, 1408, 640, "gemm bwd 64x128/4 waves/3 stages, 1 of dW, 4 of dx"),
    (2, 4680, 520, "gemm bwd 64x128/4 waves/3 stages guard, 1 of dW, 8 of dx"), (17000, 260, 136, "gemm bwd 64x128/4 waves/3 stages guard, 8 of dW, 1 of dx"),
    (4096, 1280, 264, "gemm bwd 64x128/4 waves/3 stages, 4 of dW, 1 of dx"), (5760, 768, 832, "gemm bwd 256x128/8 waves/3 stages, 4 of dW, 1 of dx"),
    (9000, 2300, 200, "gemm bwd 256x128/8 waves/3 stages guard, 6 of dW, 2 of dx"), (8192, 5120, 1280, "gemm bwd 256x128/8 waves/3 stages, 1 of dW, 5 of dx")])
def test_linear_bwd_every_cut(B, M, N, K, launches):
    import torch
    x, W, bias, g = lin_inputs(M, N, K, M)
    z = (1.5 * torch.randn(M, N, generator=g, device="cuda")).bfloat16()
    for yt, act, dwt in ((torch.bfloat16, 3, torch.bfloat16), (torch.float32, 2, torch.float32)):
        dy = torch.randn(M, N, generator=g, device="cuda").to(yt)
        with B.dry_run(True) as names:
            B.linear_bwd(dy, x, W, z, act, dw_dtype=dwt)
        assert names[1] == launches
        check_lin_bwd(B, dy, x, W, z, act, dwt)


def test_linear_more_columns_than_a_grid_has_rows(B):
    import torch
    M, N, K = 2, 1100000, 8
    x, W, bias, g = lin_inputs(M, N, K, 3)
    check_lin_fwd(B, x, W, bias, 2, None, torch.bfloat16, True)
    dy = torch.randn(M, N, generator=g, device="cuda").bfloat16()
    dx, dW, db = B.linear_bwd(dy, x, W)
    dz = dy.double()
    rx = dz @ W.double()
    within(dx, rx, (N + 8) * U * (dz.abs() @ W.double().abs()))
    within(dW, dz.T @ x.double(), (M + 8) * U * (dz.abs().T @ x.double().abs()))
    within(db, dz.sum(0), 4 * U * dz.abs().sum(0))


def test_linear_offsets_past_32_bits(B):
    """Rows of x and y behind 2^31 elements: the same bits as at the start."""
    import torch
    M, N, K = 600064, 4096, 4096
    x, W, bias, g = lin_inputs(64, N, K, 3)
    big = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    big.view(M // 64, 64, K).copy_(x.expand(M // 64, 64, K))
    y, z = B.linear_fwd(big, W, bias, 3, save_z=True)
    for t in (y, z):
        t = t.view(M // 64, 64, N)
        assert torch.equal(t[0], t[-1]) and torch.equal(t[0], t[M // 128])
    check = B.linear_fwd(big[:128].clone(), W, bias, 3)
    assert float((check.float() - y[:128].float()).abs().max()) <= 2.0 ** -7 * float(y[:128].float().abs().max())
    del y
    dx, dW, db = B.linear_bwd(z, big, W)
    t = dx.view(M // 64, 64, K)
    assert torch.equal(t[0], t[M // 128])
    rw = z[:64].double().T @ x.double() * (M // 64)
    # a thread's rows, its share of the row blocks, and the joins: fewer than 1300 additions in a row; the products' sums in fewer than M / 32, and one rounding
    within(db, z[:64].double().sum(0) * (M // 64), 1300 * U * z[:64].double().abs().sum(0) * (M // 64))
    within(dW, rw, M / 32 * U * (z[:64].double().abs().T @ x.double().abs() * (M // 64)))


def test_linear_gradients_against_differences(B):
    """Central differences of <act(x W^T + b), dy> in 64 bits along random directions."""
    import torch
    M, N, K = 40, 24, 32
    x, W, bias, g = lin_inputs(M, N, K, 8)
    dy = torch.randn(M, N, generator=g, device="cuda")
    vx, vw, vb = (torch.randn(*s, generator=g, device="cuda").double() for s in ((M, K), (N, K), (N,)))
    for act in (1, 2, 3):
        _, z = B.linear_fwd(x, W, bias, act, save_z=True)
        dx, dW, db = B.linear_bwd(dy, x, W, z, act, dw_dtype=torch.float32)
        f = lambda a, w, b: (act64(a @ w.T + b, act) * dy.double()).sum()
        X, Wd, bd, h = x.double(), W.double(), bias.double(), 1e-5
        for num, ana, size in (((f(X + h * vx, Wd, bd) - f(X - h * vx, Wd, bd)) / (2 * h), (dx.double() * vx).sum(), (dx.double() * vx).norm()),
                               ((f(X, Wd + h * vw, bd) - f(X, Wd - h * vw, bd)) / (2 * h), (dW.double() * vw).sum(), (dW.double() * vw).norm()),
                               ((f(X, Wd, bd + h * vb) - f(X, Wd, bd - h * vb)) / (2 * h), (db.double() * vb).sum(), (db.double() * vb).norm())):
            # z kept in bf16 moves the slope by up to 0.8 x 2^-8 |z| of dy, dz and dx are rounded: together below 2^-6 of each term, of independent signs, six of
            # their standard deviations
            assert abs(float(num - ana)) <= 6 * 2.0 ** -6 * float(size) + 1e-6


def test_linear_edges(B):
    import torch
    x, W, bias, g = lin_inputs(6, 24, 16, 1)
    e = torch.empty(0, 16, dtype=torch.bfloat16, device="cuda")
    assert B.linear_fwd(e, W, bias, 1).shape == (0, 24)
    dx, dW, db = B.linear_bwd(torch.empty(0, 24, dtype=torch.bfloat16, device="cuda"), e, W)
    assert dx.shape == (0, 16) and not dW.any() and not db.any()
    dx, dW, db = B.linear_bwd(torch.empty(6, 0, dtype=torch.bfloat16, device="cuda"), x, W[:0])
    assert not dx.any() and dW.shape == (0, 16) and db.shape == (0,)
    # large arguments: no overflow on the way to 0, 1 or z; NaN and infinities stay in their rows and columns
    z = torch.tensor([-3e38, -1e30, -200.0, -30.0, 0.0, 30.0, 200.0, 1e30], device="cuda").bfloat16()
    eye = torch.zeros(8, 8, dtype=torch.bfloat16, device="cuda")
    eye.fill_diagonal_(1)
    for act in range(5):
        y = B.linear_fwd(torch.diag(z.float()).bfloat16(), eye, None, act, out_dtype=torch.float32).diagonal()
        want = act64(z.double(), act)
        assert torch.isfinite(y).all() and torch.allclose(y.double(), want, rtol=1e-5, atol=1e-6), act
    x[2, 3], W[5, 1] = math.nan, math.inf
    y = B.linear_fwd(x, W, bias, 3)
    bad = ~torch.isfinite(y.float())
    want = torch.zeros_like(bad)
    want[2] = True
    # x[i, 1] of either sign against the infinity: silu(-inf) is 0 x inf
    want[:, 5] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("act", [1, 2, 3, 4])
def test_slopes_far_out(B, act):
    """dbias of one row is act'(z) itself: 0 or 1 far out, with no overflow on the way, and NaN where z is NaN."""
    import torch
    z = torch.tensor([-3e38, -1e30, -1e20, -3e18, -200.0, -30.0, -1.0, 0.0, 1.0, 30.0, 200.0, 3e18, 1e20, 1e30, 3e38, math.nan], device="cuda").bfloat16()[None]
    x, W = torch.zeros(1, 8, dtype=torch.bfloat16, device="cuda"), torch.zeros(16, 8, dtype=torch.bfloat16, device="cuda")
    db = B.linear_bwd(torch.ones_like(z), x, W, z, act, grads=(False, False, True))[2]
    d = z[0, 4:11].double().requires_grad_()
    # (the clamp in act64 has slope 1 at 0, relu by convention 0)
    (d.relu() if act == 4 else act64(d, act)).sum().backward()
    want = torch.cat([torch.zeros(4), d.grad.cpu(), torch.ones(4)]).cuda()
    # erf's polynomial is off by 1.5e-7, the exponential and the reciprocal by 4 U each, products of |z| <= 200 by less
    assert torch.allclose(db[:15].double(), want.double(), rtol=0, atol=2e-6) and torch.isnan(db[15])


# ---- together --------------------------------------------------------------------------------------------------------------
class Block:
    """A diffusion transformer's block out of the public calls: layer norm, packed projection, rotary positions, attention, projection into the fp32
    stream, layer norm, feed-forward with GELU into the stream."""

    def __init__(self, B, C, heads, pairs, seed):
        import torch
        g = gen(seed)
        w = lambda n, k: (torch.randn(n, k, generator=g, device="cuda") / math.sqrt(k)).bfloat16()
        v = lambda n, s, o=0.0: (o + s * torch.randn(n, generator=g, device="cuda")).bfloat16()
        self.B, self.C, self.heads = B, C, heads
        self.g1, self.b1, self.g2, self.b2 = v(C, 0.1, 1.0), v(C, 0.1), v(C, 0.1, 1.0), v(C, 0.1)
        self.wq, self.bq, self.wo, self.bo, self.w1, self.c1, self.w2, self.c2 = w(3 * C, C), v(3 * C, 0.1), w(C, C), v(C, 0.1), w(4 * C, C), v(4 * C, 0.1), w(C, 4 * C), v(C, 0.1)
        self.rope = B.Rope(C // heads, pairs, layout=B.SD_ROPE_AXIS_HALVES)

    def __call__(self, h, pos):
        B, C, H = self.B, self.C, self.heads
        Bn, T, _ = h.shape
        n = B.layernorm_fwd(h, self.g1, self.b1)
        qkv = B.linear_fwd(n.view(-1, C), self.wq, self.bq).view(Bn, T, 3, H, C // H)
        q, k = B.rope_fwd(self.rope, pos, qkv[:, :, 0], qkv[:, :, 1])
        vt = qkv[:, :, 2].reshape(Bn, T, C).permute(2, 0, 1)
        Tp = (T + 7) // 8 * 8
        import torch
        vt = torch.nn.functional.pad(vt, (0, Tp - T)).reshape(C, Bn * Tp).contiguous()
        a = B.attention_fwd(q.reshape(Bn, T, C), k.reshape(Bn, T, C), vt, H)
        h = B.linear_fwd(a.view(-1, C), self.wo, self.bo, residual=h.view(-1, C), out_dtype=h.dtype)
        n = B.layernorm_fwd(h, self.g2, self.b2)
        f = B.linear_fwd(n, self.w1, self.c1, B.SD_ACT_GELU_TANH)
        return B.linear_fwd(f, self.w2, self.c2, residual=h, out_dtype=h.dtype).view(Bn, T, C)

    def plain(self, h, pos):
        import torch
        C, H = self.C, self.heads
        Bn, T, _ = h.shape
        d = lambda t: t.double()

        def ln(x, g, b):
            m = x.mean(-1, keepdim=True)
            return (x - m) * ((x - m).square().mean(-1, keepdim=True) + 1e-5).rsqrt() * d(g) + d(b)
        x = d(h)
        qkv = (ln(x, self.g1, self.b1) @ d(self.wq).T + d(self.bq)).view(Bn, T, 3, H, C // H)
        q, k = (rope_ref(qkv[:, :, i], pos.expand(Bn, -1, -1), self.rope.axis_pairs, 1e4, 2, False, 1.0)[0].transpose(1, 2) for i in (0, 1))
        p = torch.softmax(q.contiguous() @ k.transpose(-1, -2).contiguous() / 8, -1) @ qkv[:, :, 2].transpose(1, 2).contiguous()
        x = x + p.transpose(1, 2).reshape(Bn, T, C) @ d(self.wo).T + d(self.bo)
        return x + act64(ln(x, self.g2, self.b2) @ d(self.w1).T + d(self.c1), 2) @ d(self.w2).T + d(self.c2)


@pytest.mark.parametrize("Bn,T", [(2, 77), (1, 1), (2, 256)])
def test_block_of_a_diffusion_transformer(B, Bn, T):
    import torch
    C, H = 320, 5
    blk = Block(B, C, H, (16, 16), 3)
    h = torch.randn(Bn, T, C, generator=gen(7), device="cuda")
    side = max(1, int(math.isqrt(T)))
    pos = torch.stack([torch.arange(T, device="cuda") // side, torch.arange(T, device="cuda") % side], -1).float()[None]
    y = blk(h, pos)
    ref = blk.plain(h, pos)
    # what is added to the stream passes through eight roundings to bf16, each at most 2^-8 of its own rms in rms, and sums of independent terms keep that ratio
    assert float((y.double() - ref).norm() / (ref - h.double()).norm()) <= math.sqrt(8) * 2.0 ** -8


def test_block_captured_and_replayed(B):
    """Three replays with new inputs in between, on a stream of its own, against the eager results; two graphs that replay in turn."""
    import torch
    C, H, Bn, T = 320, 5, 2, 77
    blk = Block(B, C, H, (16, 16), 3)
    pos = torch.rand(1, T, 2, generator=gen(1), device="cuda") * 30
    h = [torch.randn(Bn, T, C, generator=gen(i), device="cuda") for i in range(2)]
    dy = [torch.randn(Bn * T, C, generator=gen(9 + i), device="cuda").bfloat16() for i in range(2)]

    def step(hh, d):
        y = blk(hh, pos)
        x = hh.view(-1, C)
        n, mean, rstd = B.layernorm_fwd(x, blk.g2, blk.b2, stats=True)
        f, z = B.linear_fwd(n, blk.w1, blk.c1, B.SD_ACT_GELU_TANH, save_z=True)
        df, dw2, dc2 = B.linear_bwd(d, f, blk.w2)
        dn, dw1, dc1 = B.linear_bwd(df, n, blk.w1, z, B.SD_ACT_GELU_TANH)
        return (y, dw2, dc2, dw1, dc1, *B.layernorm_bwd(dn, x, mean, rstd, blk.g2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for i in range(2):
            step(h[i], dy[i])
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(step(h[i], dy[i]))
        graphs.append(gr)
    for rep in range(3):
        for i in range(2):
            h[i].normal_(generator=gen(100 * rep + i))
            dy[i].normal_(generator=gen(50 * rep + i))
        for gr in graphs:
            gr.replay()
        for i in range(2):
            for a, b in zip(outs[i], step(h[i], dy[i])):
                assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_feed_forward_gradients_as_they_would_be_used(B):
    """Layer norm, projection, GELU, projection, residual: the chain of backward calls against autograd in 64 bits."""
    import torch
    M, C, F = 333, 136, 520
    x, ga, be, g = ln_inputs(M, C, torch.float32, 2)
    _, w1, c1, _ = lin_inputs(1, F, C, 3)
    _, w2, c2, _ = lin_inputs(1, C, F, 4)
    dy = torch.randn(M, C, generator=g, device="cuda")
    n, mean, rstd = B.layernorm_fwd(x, ga, be, stats=True)
    f, z = B.linear_fwd(n, w1, c1, B.SD_ACT_GELU, save_z=True)
    B.linear_fwd(f, w2, c2, residual=x, out_dtype=torch.float32)
    df, dw2, dc2 = B.linear_bwd(dy, f, w2)
    dn, dw1, dc1 = B.linear_bwd(df, n, w1, z, B.SD_ACT_GELU)
    dx, dg, db = B.layernorm_bwd(dn, x, mean, rstd, ga)
    dx = dx + dy
    with torch.enable_grad():
        P = [t.double().requires_grad_(True) for t in (x, ga, be, w1, c1, w2, c2)]
        m = P[0].mean(1, keepdim=True)
        nn = (P[0] - m) * ((P[0] - m).square().mean(1, keepdim=True) + 1e-5).rsqrt() * P[1] + P[2]
        y = P[0] + act64(nn @ P[3].T + P[4], 1) @ P[5].T + P[6]
        ref = torch.autograd.grad(y, P, dy.double())
    # up to seven roundings to bf16 on the way to each gradient, 2^-8 each, independent
    for got, want in zip((dx, dg, db, dw1, dc1, dw2, dc2), ref):
        assert float((got.double() - want).norm() / want.norm()) <= math.sqrt(7) * 2.0 ** -8


def test_two_streams_at_once(B):
    """Calls on two streams, a workspace each, give what each gives alone."""
    import torch
    M, N, K = 3000, 640, 320
    jobs = []
    for i in range(2):
        x, W, bias, g = lin_inputs(M, N, K, 20 + i)
        dy = torch.randn(M, N, generator=g, device="cuda").bfloat16()
        h = torch.randn(M, K, generator=g, device="cuda")
        q, pos = torch.randn(1, M, 5, 64, generator=g, device="cuda").bfloat16(), torch.rand(M, 2, generator=g, device="cuda") * 64
        jobs.append((x, W, bias, dy, h, q, pos))
    rope = B.Rope(64, [16, 16])

    def work(x, W, bias, dy, h, q, pos):
        y, z = B.linear_fwd(x, W, bias, 2, save_z=True)
        n, mean, rstd = B.layernorm_fwd(h, stats=True)
        return (y, *B.linear_bwd(dy, x, W, z, 2), n, *B.layernorm_bwd(n, h, mean, rstd), B.rope_fwd(rope, pos, q)[0])
    want = [work(*j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[], []]
    for rep in range(5):
        for s, j, o in zip(streams, jobs, got):
            with torch.cuda.stream(s):
                o.append(work(*j))
    torch.cuda.synchronize()
    for o, w in zip(got, want):
        for r in o:
            assert all(torch.equal(a, b) for a, b in zip(r, w))


# ---- every shape and loop of the row kernels -------------------------------------------------------------------------------
# both sides of every length at which a kernel ends, and lengths inside that four elements do not divide
BORDERS = [64, 65, 66, 100, 127, 128, 129, 254, 258, 319, 320, 321, 333, 511, 512, 513, 767, 769, 1279, 1281, 2047, 4094, 4097, 8190]
TYPES = [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("float32", "float32"), ("bfloat16", "float32")]


@pytest.mark.parametrize("C", BORDERS)
def test_layernorm_borders(B, C):
    for xt, yt in TYPES:
        test_layernorm_fwd(B, C, xt, yt)
        test_layernorm_bwd(B, C, xt, yt)


@pytest.mark.parametrize("M,C", [(40003, 64), (33001, 63), (33001, 128), (40003, 100), (20001, 320), (33001, 319), (20001, 512), (16385, 333), (8195, 768), (4101, 515), (8195, 1280), (4097, 1155),
                                 (8195, 1283), (5003, 2048), (2051, 4096), (1030, 4095), (2051, 8192), (1030, 5001), (1030, 8193), (2051, 10001), (1030, 16384)])
def test_layernorm_fwd_rows_in_turn(B, M, C):
    """More rows than a launch has places for (1024 workgroups of 16, 4 or 1 rows): two rounds and more, of which the last is not full."""
    import torch
    for xt, yt in (TYPES[0], TYPES[1]) if C != 1280 else TYPES:
        x, ga, be, _ = ln_inputs(M, C, getattr(torch, xt), C + M)
        check_ln_fwd(B, x, ga, be, getattr(torch, yt))


@pytest.mark.parametrize("M,C", [(40003, 64), (33001, 63), (40003, 128), (33001, 101), (9001, 256), (8201, 131), (9001, 768), (8201, 515), (5003, 1280), (4101, 1283), (5003, 2048), (1100, 4096), (1031, 5000),
                                 (2051, 8192), (1100, 8193), (600, 16384)])
def test_layernorm_bwd_rows_in_turn(B, M, C):
    """The same backwards, with gradients of the weights (256 or 512 workgroups) and without (512 or 1024)."""
    import torch
    for xt, yt in (TYPES[0], TYPES[1]) if C != 1280 else TYPES:
        x, ga, be, g = ln_inputs(M, C, getattr(torch, xt), C + M)
        dy = torch.randn(M, C, generator=g, device="cuda").to(getattr(torch, yt))
        _, mean, rstd = B.layernorm_fwd(x, ga, be, stats=True)
        check_ln_bwd(B, x, dy, ga, mean, rstd)


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("layout", [0, 1, 2])
@pytest.mark.parametrize("Bn,T,Hq,Hk,D,pairs", [(4500, 1, 1, 0, 64, (16, 8)), (5003, 3, 1, 1, 24, (3, 4)), (1, 33001, 1, 0, 8, (4,)), (1, 40009, 1, 0, 8, (1, 2)), (1, 5003, 2, 1, 40, (3, 7)), (3, 701, 2, 2, 128, (16, 24)),
                                                (700, 7, 3, 1, 64, (13, 18))])
def test_rope_tokens_of_a_workgroup(B, Bn, T, Hq, Hk, D, pairs, layout, dt):
    """Several tokens a workgroup, from 2 to 32, of one sample or of many; one unit a token; heads with a rest that is not turned; single elements."""
    rope_case(B, Bn, T, Hq, Hk, D, pairs, layout, dt=dt, seed=D + T)


@pytest.mark.parametrize("M,N,K", [(129, 317, 648), (300, 512, 1024), (2100, 320, 136), (4133, 645, 320)])
def test_linear_bwd_rounds_dz_once_and_nothing_else(B, M, N, K):
    """Where dz needs no rounding the products have none but their sums'; where it does, theirs is the product of the rounded dz."""
    import torch
    x, W, bias, g = lin_inputs(M, N, K, M + N)
    xd, wd = x.double(), W.double()
    dy = torch.randn(M, N, generator=g, device="cuda").bfloat16()
    z = (1.5 * torch.randn(M, N, generator=g, device="cuda")).bfloat16()
    # relu's slope is 0 or 1; fp32 gradients that bf16 holds
    for d, act, dz in ((dy, 4, torch.where(z > 0, dy, 0).double()), (dy.float(), 4, torch.where(z > 0, dy, 0).double()), (dy.float(), 0, dy.double()), (dy, 0, dy.double())):
        dx, dW, db = B.linear_bwd(d, x, W, z if act else None, act, dw_dtype=torch.float32)
        within(dx, dz @ wd, (N + 8) * U * (dz.abs() @ wd.abs()))
        within(dW, dz.T @ xd, (M + 8) * U * (dz.abs().T @ xd.abs()))
        within(db, dz.sum(0), (M / 64 + 40) * U * dz.abs().sum(0))
        # every addition is off by U of the sum so far, whose norm over all elements is no more than the whole's
        assert float((dW.double() - dz.T @ xd).norm() / (dz.T @ xd).norm()) <= (M + 8) * U
    for d, act in ((torch.randn(M, N, generator=g, device="cuda"), 0), (dy, 1), (dy, 2), (dy.float(), 3)):
        zz = z.double().requires_grad_(True)
        dz = torch.autograd.grad(act64(zz, act), zz, d.double())[0] if act else d.double()
        r = dz.bfloat16().double()
        dW = B.linear_bwd(d, x, W, z if act else None, act, dw_dtype=torch.float32)[1].double()
        # fp32's error e <= (1e-6 or U) |dy| takes dz over a tie, and so one step (2^-7 |dz| at most) the other way, with probability 2 e / step: the mean square of that is
        # below 2 e 2^-7 |dz|.  x is independent of it, so that the product's error has the same ratio to the product; twice that.  The sums as above.
        flips = math.sqrt(float((2 * (1e-6 if act else U) * 2.0 ** -7 * d.double().abs() * dz.abs()).sum())) / float(dz.norm())
        off = float((dW - r.T @ xd).norm() / (dz.T @ xd).norm())
        assert off <= 2 * flips + (M + 8) * U < 2.0 ** -10, (act, off, flips)

"""Layer norm, rotary positions and the linear layer with its gradients: what the calls refuse, and what they would launch, without a GPU."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2407_02031_amd", "libswiftdiff.so")
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3
PX, PY, PZ, PW, PA, PB, PC = (i << 12 for i in range(1, 8))      # aligned addresses that nothing reads


@pytest.fixture(scope="module")
def B():
    if not os.path.exists(LIB):
        from paper_2407_02031_amd import build
        build.build(verbose=False)
    from paper_2407_02031_amd import binding
    return binding


def ln_fwd(L, x=PX, xt=0, g=PA, b=PB, y=PY, yt=0, mean=None, rstd=None, M=4, Cc=64):
    return L.sd_layernorm_fwd(x, xt, g, b, 1e-5, y, yt, mean, rstd, M, Cc, None)


def test_layernorm_refusals(B):
    L = B.lib()
    assert ln_fwd(L, x=None) == EINVAL and ln_fwd(L, y=None) == EINVAL
    assert ln_fwd(L, x=PX + 8) == EINVAL and ln_fwd(L, g=PA + 2) == EINVAL and b"aligned" in L.sd_last_error()
    assert ln_fwd(L, xt=2) == EINVAL and ln_fwd(L, yt=-1) == EINVAL
    assert ln_fwd(L, M=-1) == EINVAL and ln_fwd(L, Cc=0) == EINVAL
    assert ln_fwd(L, Cc=3) == EUNSUPPORTED and ln_fwd(L, Cc=16385) == EUNSUPPORTED
    assert ln_fwd(L, x=None, y=None, M=0) == 0
    bwd = lambda dy=PY, yt=0, x=PX, xt=0, mean=PA, rstd=PB, g=None, dx=PZ, dg=PC, db=PW, M=4, Cc=64, ws=1 << 20, n=1 << 20: L.sd_layernorm_bwd(
        dy, yt, x, xt, mean, rstd, g, dx, dg, db, M, Cc, ws, n, None)
    for k in ("dy", "x", "mean", "rstd", "dx"):
        assert bwd(**{k: None}) == EINVAL, k
    assert bwd(ws=None) == EWORKSPACE and bwd(n=16) == EWORKSPACE and bwd(ws=(1 << 20) + 16) == EWORKSPACE
    assert bwd(Cc=2) == EUNSUPPORTED and bwd(xt=7) == EINVAL and bwd(dg=PC + 4) == EINVAL
    assert L.sd_layernorm_bwd(None, 0, None, 0, None, None, None, None, None, None, 0, 64, None, 0, None) == 0


def rope(B, **kw):
    d = dict(D=64, pairs=(16, 16), layout=0, theta=1e4, n=None, pos=PA, stride=0, q=PX, ldq=640, hq=10, yq=PY, ldyq=640, k=PZ, ldk=640, hk=10, yk=PW, ldyk=640, t=0, Bn=2, T=5, bwd=False)
    d.update(kw)
    r = B.sd_rope(d["D"], len(d["pairs"]) if d["n"] is None else d["n"], (C.c_int32 * 4)(*d["pairs"][:4]), d["layout"], 0, d["theta"])
    fn = B.lib().sd_rope_bwd if d["bwd"] else B.lib().sd_rope_fwd
    return fn(C.byref(r), d["pos"], d["stride"], d["q"], d["ldq"], d["hq"], d["yq"], d["ldyq"], d["k"], d["ldk"], d["hk"], d["yk"], d["ldyk"], d["t"], d["Bn"], d["T"], None)


@pytest.mark.parametrize("bwd", [False, True])
def test_rope_refusals(B, bwd):
    f = lambda **kw: rope(B, bwd=bwd, **kw)
    assert f(D=63) == EUNSUPPORTED and f(D=264) == EUNSUPPORTED and f(D=0) == EUNSUPPORTED
    assert f(n=0) == EINVAL and f(n=5) == EINVAL and f(pairs=(16, 17)) == EINVAL and f(pairs=(0, 16)) == EINVAL and f(pairs=(2 ** 31 - 1, 2 ** 31 - 1)) == EINVAL
    assert f(layout=3) == EINVAL and f(theta=0.0) == EINVAL and f(theta=float("nan")) == EINVAL and f(t=3) == EINVAL
    assert f(q=None) == EINVAL and f(yk=None) == EINVAL and f(pos=None) == EINVAL and f(pos=PA + 2) == EINVAL
    assert f(q=PX + 8) == EINVAL and f(ldq=632) == EINVAL and f(ldyk=644) == EINVAL and f(stride=9) == EINVAL
    assert f(hq=-1) == EINVAL and f(hk=257) == EINVAL and f(Bn=-1) == EINVAL and f(T=-1) == EINVAL
    assert f(Bn=65536, T=65536) == EUNSUPPORTED
    assert f(T=0, q=None, pos=None) == 0 and f(Bn=0) == 0 and f(hq=0, hk=0, q=None) == 0


def test_rope_access_width(B):
    """16 bytes where every axis and the rest of the head end at such a border."""
    from paper_2407_02031_amd import binding
    for kw, name in ((dict(), "rope neighbours 8"), (dict(layout=2), "rope halves 8"), (dict(layout=2, pairs=(12, 20)), "rope halves 4"), (dict(layout=1, pairs=(13, 19)), "rope halves 8"),
                     (dict(layout=1, pairs=(13, 18)), "rope halves 1"), (dict(pairs=(13, 18)), "rope neighbours 2"), (dict(pairs=(13, 18), t=1), "rope neighbours 2"), (dict(layout=2, t=1), "rope halves 4"),
                     (dict(layout=1, pairs=(8, 8)), "rope halves 8"), (dict(layout=1, pairs=(4, 8)), "rope halves 4")):
        with binding.dry_run() as names:
            assert rope(B, **kw) == 0
        assert names == [name], kw


def lin_fwd(L, x=PX, W=PW, bias=PB, act=1, res=None, y=PY, yt=0, z=None, M=4, N=8, K=64):
    return L.sd_linear_fwd(x, W, bias, act, res, y, yt, z, M, N, K, None)


def test_linear_refusals(B):
    L = B.lib()
    assert lin_fwd(L, x=None) == EINVAL and lin_fwd(L, W=None) == EINVAL and lin_fwd(L, y=None) == EINVAL
    assert lin_fwd(L, y=PY + 4) == EINVAL and lin_fwd(L, z=PZ + 2) == EINVAL
    assert lin_fwd(L, K=12) == EUNSUPPORTED and lin_fwd(L, K=0) == EUNSUPPORTED and lin_fwd(L, K=1 << 22) == EUNSUPPORTED
    assert lin_fwd(L, act=5) == EINVAL and lin_fwd(L, act=-1) == EINVAL and lin_fwd(L, yt=2) == EINVAL and lin_fwd(L, M=-1) == EINVAL
    assert lin_fwd(L, x=None, M=0) == 0 and lin_fwd(L, W=None, N=0) == 0
    bwd = lambda dy=PY, yt=0, x=PX, W=PW, z=PZ, act=1, dx=PA, dW=PB, wt=0, db=PC, M=4, N=8, K=64, ws=1 << 20, n=1 << 20: L.sd_linear_bwd(
        dy, yt, x, W, z, act, dx, dW, wt, db, M, N, K, ws, n, None)
    assert bwd(dy=None) == EINVAL and bwd(x=None) == EINVAL and bwd(W=None) == EINVAL and bwd(z=None) == EINVAL
    assert bwd(K=4) == EUNSUPPORTED and bwd(wt=2) == EINVAL and bwd(act=9) == EINVAL and bwd(dx=PA + 8) == EINVAL
    assert bwd(ws=None) == EWORKSPACE and bwd(n=64) == EWORKSPACE and bwd(ws=(1 << 20) + 64) == EWORKSPACE
    assert L.sd_linear_bwd(PY, 0, None, None, None, 0, None, None, 0, None, 4, 8, 64, None, 0, None) == 0     # nothing asked for
    assert L.sd_linear_bwd_workspace_bytes(0, 8, 8) == 256 and L.sd_linear_bwd_workspace_bytes(100, 13, 8) >= 100 * 16 * 2 + 2 * 13 * 4


def test_results_in_an_inputs_place(B):
    """What may be in place is, within one type; anything else would be read after it is overwritten."""
    L = B.lib()
    with B.dry_run():
        assert ln_fwd(L, y=PX) == 0 and ln_fwd(L, y=PX, xt=1) == EINVAL
        bwd = lambda dx, xt=0: L.sd_layernorm_bwd(PY, 0, PX, xt, PA, PB, None, dx, None, None, 4, 64, None, 0, None)
        assert bwd(PX) == 0 and bwd(PY) == 0 and bwd(PX, 1) == 0 and bwd(PY, 1) == EINVAL
        assert rope(B, yq=PX, yk=PZ) == 0 and rope(B, k=PX) == 0 and rope(B, yk=PX, yq=PX, k=None, hk=0) == 0
        assert rope(B, yq=PZ) == EINVAL and rope(B, yk=PX) == EINVAL and rope(B, yk=PY) == EINVAL
        assert lin_fwd(L, res=PY) == 0 and lin_fwd(L, z=PZ, res=PY) == 0
        for kw in (dict(y=PX), dict(y=PW), dict(z=PX), dict(z=PW), dict(z=PY), dict(z=PZ, res=PZ)):
            assert lin_fwd(L, **kw) == EINVAL, kw
        lin = lambda dx=PA, dW=PB, db=PC: L.sd_linear_bwd(PY, 0, PX, PW, PZ, 1, dx, dW, 0, db, 4, 8, 64, 1 << 20, 1 << 20, None)
        assert lin() == 0
        for at in (PX, PY, PZ, PW):
            assert lin(dx=at) == EINVAL and lin(dW=at) == EINVAL and lin(db=at) == EINVAL


def test_sizes_beyond_a_launch(B):
    """No launch has 2^32 threads or more, no query of a workspace runs over, and no size loses its upper bits on the way to the C call."""
    L, top = B.lib(), 2 ** 31 - 1
    with B.dry_run():
        assert lin_fwd(L, M=1 << 28) == EUNSUPPORTED and lin_fwd(L, M=(1 << 28) - 1) == 0 and lin_fwd(L, N=1 << 22) == EUNSUPPORTED
        # 256 + 256 heads of eight pairs of single elements and more: a token for a workgroup
        many = dict(D=16, pairs=(7,), layout=1, hq=256, hk=256, ldq=4096, ldk=4096, ldyq=4096, ldyk=4096, Bn=1)
        assert rope(B, T=(1 << 24) - 1, **many) == 0 and rope(B, T=1 << 24, **many) == EUNSUPPORTED
        assert rope(B, T=top, Bn=1, hq=1, hk=1) == EUNSUPPORTED and rope(B, T=1 << 28, Bn=1, hq=1, hk=1) == 0
    assert L.sd_linear_bwd_workspace_bytes(top, top, top) == 256 and L.sd_linear_bwd_workspace_bytes((1 << 28) - 1, 8, 8) > 1 << 32
    assert L.sd_layernorm_bwd_workspace_bytes(top, 16384) > 0
    B._sizes(0, top)
    with pytest.raises(ValueError, match="2\\^31"):
        B._sizes(4, top + 1)


def test_linear_bwd_launches(B):
    """Which launches a choice of gradients takes: nothing sums the parts of a product that is not wanted."""
    L = B.lib()

    def names(dx, dW, db, act=0, M=1, N=5120, K=64):
        with B.dry_run() as n:
            assert L.sd_linear_bwd(PY, 0, PX, PW, PZ, act, PA if dx else None, PB if dW else None, 0, PC if db else None, M, N, K, 1 << 20, 1 << 40, None) == 0
        return n
    gemm, guarded = ("gemm bwd 64x128/4 waves/3 stages" + g for g in ("", " guard"))
    # one row: dx in parts, dW whole, dbias of one row block
    assert names(1, 0, 0) == [gemm, "part sums"] and names(0, 1, 0) == [guarded] and names(0, 0, 1) == ["dz sums only"]
    assert names(1, 1, 1) == ["dz sums only", guarded, "part sums"] and names(0, 1, 0, act=1) == ["dz no sums", guarded]
    # many rows of few columns: dW in parts, dx whole, dbias of many row blocks
    assert names(1, 0, 0, M=8192, N=64) == [gemm] and names(0, 1, 0, M=8192, N=64) == [gemm, "part sums"] and names(0, 0, 1, M=8192, N=64) == ["dz sums only", "part sums"]
    # large ones: dW whole, the last tiles of dx in parts; all of dW in parts
    gemm = "gemm bwd 256x128/8 waves/3 stages"
    assert names(1, 0, 0, M=8192, K=1280) == [gemm, "part sums"] and names(0, 1, 0, M=8192, K=1280) == [gemm]
    assert names(0, 1, 0, M=16384, N=1280, K=1280) == [gemm, "part sums"] and names(1, 0, 0, M=16384, N=1280, K=1280) == [gemm]


def test_binding_refuses_what_the_c_call_cannot_see(B):
    import torch
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="not on a GPU"):
        B.layernorm_fwd(x)
    with pytest.raises(ValueError, match="axes"):
        B.Rope(64, [])
    with pytest.raises(ValueError, match="shape"):
        B._expect("x", x, (4, 65), (torch.float32,), -1)
    with pytest.raises(TypeError, match="bfloat16"):
        B._expect("x", x, (4, 64), (torch.bfloat16,), -1)
    with pytest.raises(ValueError, match="others"):
        B._expect("x", x, (4, 64), (torch.float32,), 0)
    with pytest.raises(ValueError, match="contiguous"):
        B._expect("x", x.T, (64, 4), (torch.float32,), -1)
    q = torch.zeros(2, 5, 3, 8)
    assert B._token_rows("q", q, 8) == 24 and B._token_rows("q", q[:, :, :2], 8) == 24
    assert B._token_rows("q", q[:1, :1], 8) == 24 and B._token_rows("q", torch.zeros(2, 1, 3, 8), 8) == 24
    for bad in (q.transpose(1, 2), q[:, :4], q[:, ::2][:, :2], q[..., ::2]):
        with pytest.raises(ValueError):
            B._token_rows("q", bad, bad.shape[-1])


@pytest.mark.parametrize("bwd", [False, True])
def test_rope_in_place_keeps_its_distance(B, bwd):
    """A result in its own argument's place has the argument's distance between tokens, or tokens are overwritten that others have still to read."""
    f = lambda **kw: rope(B, bwd=bwd, **kw)
    with B.dry_run():
        # out of packed rows into dense ones at the same address, and the other way
        assert f(yq=PX, ldq=1920) == EINVAL and f(yq=PX, ldyq=1920) == EINVAL and b"place" in B.lib().sd_last_error()
        assert f(yk=PZ, ldk=1920) == EINVAL and f(yk=PZ, ldyk=1920) == EINVAL
        assert f(Bn=2, T=1, yq=PX, ldq=1920) == EINVAL and f(Bn=1, T=2, yk=PZ, ldk=1920) == EINVAL
        # at one distance; with one token, which has none; without heads
        assert f(yq=PX, ldq=1920, ldyq=1920, yk=PZ, ldk=1280, ldyk=1280) == 0
        assert f(Bn=1, T=1, yq=PX, ldq=1920, yk=PZ, ldk=1920) == 0
        assert f(hk=0, yk=PZ, ldk=1920) == 0 and f(hq=0, yq=PX, ldq=1920) == 0


def kernel_shapes(name):
    """(threads a row, chunks, whole chunks) of every instance of a layer norm kernel in the built library"""
    import re
    text = open(LIB, "rb").read()
    # their mangled names: types, then three integers
    return {tuple(map(int, m)) for m in re.findall(rb"_ZN2sd\d+" + name + rb"I[^E]*?Li(\d+)ELi(\d+)ELi(\d+)E", text)}


def test_layernorm_kernels_are_all_launched(B):
    """Each direction is built for the row lengths that it takes, and for no others."""
    short, long = {(16, 1, 0), (16, 2, 1)}, {(64, 3, 1), (64, 5, 3), (64, 8, 5), (256, 4, 2), (256, 8, 4), (1024, 4, 2)}
    assert kernel_shapes(b"ln_fwd_kernel") == short | {(16, 5, 2), (16, 8, 5)} | long
    assert kernel_shapes(b"ln_bwd_kernel") == kernel_shapes(b"ln_bwd_few_kernel") == short | {(64, 1, 0)} | long


class GemmProblem(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("p0", "q0", "p1", "q1", "bias", "res", "y")] + [(n, C.c_int64) for n in ("ldp0", "ldq0", "ldp1", "ldq1", "ldr", "ldy")] +
                [(n, C.c_int32) for n in ("Mp", "N", "K0", "K1", "geglu_F", "y_f32", "res_f32", "bias_on_rows")] + [("alpha", C.c_float)] +
                [(n, C.c_int32) for n in ("tile_begin", "tiles_m", "tiles_n")] + [(n, C.c_void_p) for n in ("signal_or_z", "wait")] +
                [(n, C.c_int32) for n in ("wait_need", "wait_cols")] + [("t_scale", C.c_float), ("readers", C.c_int32), ("nonce", C.c_uint64)])


class GemmGroup(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n", "total_tiles", "n_lead", "zero_n")] + [("zero_ptr", C.c_void_p), ("first_tile", C.c_int32 * 16), ("p", GemmProblem * 16)]


def test_linear_layers_and_projections_keep_apart(B):
    """A linear layer keeps z where a projection keeps its signal: neither is launched as the other, whatever a launcher has written into the group."""
    L = B.lib()
    assert C.sizeof(GemmProblem) == 192

    def launch(name, *problems):
        g = GemmGroup(n=len(problems))
        for i, kw in enumerate(problems):
            for k, v in dict(dict(p0=PX, q0=PW, y=PY, ldp0=640, ldq0=640, ldy=320, Mp=256, N=320, K0=640, alpha=1.0), **kw).items():
                setattr(g.p[i], k, v)
        with B.dry_run() as names:
            rc = getattr(L, name)(C.byref(g), None)
        return rc, names
    group, g16 = "_ZN2sd17launch_gemm_groupERNS_9GemmGroupEP12ihipStream_t", "_ZN2sd13launch_gemm16ERNS_9GemmGroupEP12ihipStream_t"
    gelu = dict(geglu_F=-2, signal_or_z=PZ)
    assert launch(g16, gelu)[0] == 0 and launch(g16, {})[0] == 0 and launch(group, {})[0] == 0
    assert launch(group, gelu)[0] == EINVAL and b"linear layer" in L.sd_last_error()
    adapter = dict(p1=PA, q1=PB, ldp1=16, ldq1=16, K1=16)
    assert launch(g16, adapter)[0] == 0 and launch(g16, dict(gelu, **adapter))[0] == EINVAL and launch(g16, gelu, adapter)[0] == EINVAL
    # a projection that the general launcher has been through: readers and tiles written, still no activation
    assert launch(g16, dict(readers=3, tiles_m=2, tiles_n=3)) == launch(g16, {})


def test_sums_over_nothing_beyond_a_launch(B):
    """Gradients without a row to sum over are cleared by as many threads as a launch has, or refused."""
    L = B.lib()
    zeros = lambda M, N, K, **kw: L.sd_linear_bwd(None, 0, None, None, None, 0, kw.get("dx"), kw.get("dW"), 0, None, M, N, K, None, 0, None)
    with B.dry_run() as names:
        assert zeros((1 << 24) - 1, 0, 1024, dx=PA) == 0 and zeros(1 << 24, 0, 1024, dx=PA) == EUNSUPPORTED
        assert zeros(0, (1 << 22) - 1, 4096, dW=PA) == 0 and zeros(0, (1 << 22) - 1, 4104, dW=PA) == EUNSUPPORTED
    assert names == ["part sums"] * 2


def test_z_past_the_caches(B):
    """A z above 24 Mi elements, and only from tiles that store whole lines of it."""
    L = B.lib()

    def name(M, N, K, z=PZ):
        with B.dry_run(True) as n:
            assert lin_fwd(L, M=M, N=N, K=K, z=z) == 0
        return n[0]
    past = ", z past the caches"
    assert name(8192, 5120, 1280) == "gemm act 128x256/8 waves/3 stages" + past and name(49152, 640, 2560) == "gemm act 256x128/8 waves/3 stages" + past
    assert name(8192, 5120, 1280, None) == "gemm act 128x256/8 waves/3 stages" and past not in name(4096, 3840, 1280)
    for M, N, K in ((42496, 960, 320), (42496, 960, 1280), (88576, 320, 320), (88576, 320, 1280)):
        assert M * N > 24 << 20 and name(M, N, K) == "gemm act 128x160/4 waves/2 stages"

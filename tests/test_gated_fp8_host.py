"""Root-mean-square norm, rows in 8 bits and the gated feed-forward: what the calls refuse, and what they would launch, without a GPU."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2407_02031_amd", "libswiftdiff.so")
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3
PX, PY, PZ, PW, PA, PB, PC, PD, PE = (i << 12 for i in range(1, 10))      # aligned addresses that nothing reads


@pytest.fixture(scope="module")
def B():
    if not os.path.exists(LIB):
        from paper_2407_02031_amd import build
        build.build(verbose=False)
    from paper_2407_02031_amd import binding
    return binding


def quant(L, x=PX, xt=0, q=PY, s=PA, ld=8, M=6, K=144):
    return L.sd_quantize_fp8(x, xt, q, s, ld, M, K, None)


def test_quantize_refusals(B):
    L = B.lib()
    for k in ("x", "q", "s"):
        assert quant(L, **{k: None}) == EINVAL, k
    assert quant(L, x=PX + 8) == EINVAL and quant(L, q=PY + 4) == EINVAL and quant(L, s=PA + 4) == EINVAL
    assert quant(L, xt=2) == EINVAL and quant(L, M=-1) == EINVAL and quant(L, M=1 << 27, ld=1 << 27) == EUNSUPPORTED
    assert quant(L, ld=4) == EINVAL and quant(L, ld=9) == EINVAL and quant(L, ld=-8) == EINVAL
    for K in (0, -16, 8, 136, 1 << 22):
        assert quant(L, K=K) == EUNSUPPORTED, K
    assert quant(L, q=PX) == EINVAL and quant(L, s=PX) == EINVAL and quant(L, s=PY) == EINVAL
    assert quant(L, x=None, q=None, s=None, M=0) == 0
    with B.dry_run() as names:
        assert quant(L) == 0 and quant(L, ld=1 << 40) == 0 and quant(L, M=(1 << 27) - 1, ld=1 << 27) == 0
    assert names == ["quantize"] * 3


def rms(L, x=PX, xt=0, r=PB, rt=1, g=PC, y=PY, yt=0, s=None, ld=0, h=PD, rstd=PE, M=4, Cc=64):
    return L.sd_rmsnorm_fwd(x, xt, r, rt, g, 1e-6, y, yt, s, ld, h, rstd, M, Cc, None)


def test_rmsnorm_refusals(B):
    L = B.lib()
    assert rms(L, x=None) == EINVAL and rms(L, y=None) == EINVAL and rms(L, M=-1) == EINVAL and rms(L, Cc=0) == EINVAL
    assert rms(L, xt=2) == EINVAL and rms(L, rt=2) == EINVAL and rms(L, yt=3) == EINVAL and rms(L, r=None) == EINVAL       # h without a residual
    assert rms(L, Cc=3) == EUNSUPPORTED and rms(L, Cc=16385) == EUNSUPPORTED and rms(L, xt=1, rt=0) == EUNSUPPORTED
    for k, p in (("x", PX), ("r", PB), ("g", PC), ("y", PY), ("h", PD), ("rstd", PE)):
        assert rms(L, **{k: p + 4}) == EINVAL, k
    assert rms(L, yt=2) == EINVAL and rms(L, yt=2, s=PA, ld=2) == EINVAL and rms(L, yt=2, s=PA, ld=6, M=5) == EINVAL and rms(L, yt=2, s=PA, ld=4, Cc=72) == EUNSUPPORTED
    assert rms(L, x=None, y=None, M=0) == 0
    with B.dry_run() as names:
        assert rms(L) == 0 and rms(L, yt=2, s=PA, ld=4) == 0 and rms(L, r=None, h=None) == 0 and rms(L, h=None) == 0 and rms(L, xt=1, r=None, h=None, g=None, rstd=None) == 0
        # in place: within one type
        assert rms(L, y=PX) == 0 and rms(L, y=PX, yt=1) == EINVAL and rms(L, y=PB, yt=1) == 0 and rms(L, y=PB) == EINVAL
        assert rms(L, h=PB) == 0 and rms(L, h=PX) == EINVAL and rms(L, h=PX, rt=0) == 0 and rms(L, h=PY) == EINVAL and rms(L, y=PX, yt=2, s=PA, ld=4) == EINVAL
    assert names[:5] == ["rmsnorm fwd", "rmsnorm fwd 8 bits"] + ["rmsnorm fwd"] * 3
    bwd = lambda dy=PY, yt=0, h=PX, ht=1, rstd=PA, g=PC, dr=None, dh=PZ, dg=PW, M=4, Cc=64, ws=1 << 20, n=1 << 20: L.sd_rmsnorm_bwd(dy, yt, h, ht, rstd, g, dr, dh, dg, M, Cc, ws, n, None)
    for k in ("dy", "h", "rstd", "dh"):
        assert bwd(**{k: None}) == EINVAL, k
    assert bwd(ws=None) == EWORKSPACE and bwd(n=16) == EWORKSPACE and bwd(ws=(1 << 20) + 16) == EWORKSPACE
    assert bwd(Cc=2) == EUNSUPPORTED and bwd(ht=2) == EINVAL and bwd(yt=2) == EINVAL and bwd(dr=PB + 8) == EINVAL and bwd(dg=PW + 4) == EINVAL
    assert L.sd_rmsnorm_bwd(None, 0, None, 0, None, None, None, None, None, 0, 64, None, 0, None) == 0
    with B.dry_run() as names:
        assert bwd() == 0 and bwd(dh=PX) == 0 and bwd(dh=PY) == EINVAL and bwd(dh=PY, yt=1) == 0 and bwd(dr=PB, dh=PB) == 0 and bwd(dg=None, ws=None, n=0) == 0 and bwd(M=5000) == 0
    # (a row that is overwritten in its place, a column has still to read)
    assert names == ["rmsnorm bwd few", "rmsnorm bwd", "sum partials", "rmsnorm bwd", "sum partials", "rmsnorm bwd few", "rmsnorm bwd", "rmsnorm bwd", "sum partials"]
    assert L.sd_rmsnorm_bwd_workspace_bytes(0, 64) == 256 and L.sd_rmsnorm_bwd_workspace_bytes(2 ** 31 - 1, 16384) > 0


def test_rmsnorm_results_in_other_places(B):
    L = B.lib()
    with B.dry_run():
        eight = dict(yt=2, s=PA, ld=4)
        assert rms(L, **eight) == 0
        for p in (PX, PB, PC, PY, PD, PE):
            assert rms(L, **{**eight, "s": p}) == EINVAL, p
        for p in (PX, PB, PC, PY, PD):
            assert rms(L, rstd=p) == EINVAL, p
        assert rms(L, y=PC) == EINVAL and rms(L, h=PC) == EINVAL
        bwd = lambda dh=PZ, dg=PW: L.sd_rmsnorm_bwd(PY, 1, PX, 1, PA, PC, PB, dh, dg, 4, 64, 1 << 20, 1 << 20, None)
        assert bwd() == 0 and bwd(dg=None) == 0
        for p in (PA, PC, PW):
            assert bwd(dh=p) == EINVAL, p
        for p in (PY, PX, PB, PA, PC, PZ):
            assert bwd(dg=p) == EINVAL, p


def gated(L, x=PX, W=PW, b=PB, act=3, y=PY, yt=0, z=PZ, M=4, N=8, K=64):
    return L.sd_gated_linear_fwd(x, W, b, act, y, yt, z, M, N, K, None)


def test_gated_refusals(B):
    L, top = B.lib(), 2 ** 31 - 1
    for k in ("x", "W", "y"):
        assert gated(L, **{k: None}) == EINVAL, k
    for k, p in (("x", PX), ("W", PW), ("b", PB), ("y", PY), ("z", PZ)):
        assert gated(L, **{k: p + 8}) == EINVAL, k
    assert gated(L, K=12) == EUNSUPPORTED and gated(L, K=0) == EUNSUPPORTED and gated(L, K=1 << 22) == EUNSUPPORTED and gated(L, N=1 << 21) == EUNSUPPORTED and gated(L, M=1 << 27) == EUNSUPPORTED
    assert gated(L, act=5) == EINVAL and gated(L, act=-1) == EINVAL and gated(L, yt=2) == EINVAL and gated(L, M=-1) == EINVAL and gated(L, N=-1) == EINVAL
    for kw in (dict(y=PX), dict(y=PW), dict(y=PB), dict(y=PZ), dict(z=PX), dict(z=PW), dict(z=PB)):
        assert gated(L, **kw) == EINVAL, kw
    assert gated(L, x=None, M=0) == 0 and gated(L, W=None, N=0) == 0
    with B.dry_run():
        assert gated(L) == 0 and gated(L, z=None, b=None) == 0
        # threads of a launch stay below 2^32
        assert gated(L, M=(1 << 27) - 64, N=1) == 0 and gated(L, M=(1 << 27) - 1, N=1) == 0 and gated(L, M=1 << 26, N=128) == EUNSUPPORTED and gated(L, M=65536, N=65536) == 0 and gated(L, M=1 << 16, N=1 << 17) == EUNSUPPORTED
    bwd = lambda dy=PY, yt=0, x=PX, W=PW, z=PZ, act=1, dx=PA, dW=PB, wt=0, db=PC, M=4, N=8, K=64, ws=1 << 20, n=1 << 30: L.sd_gated_linear_bwd(dy, yt, x, W, z, act, dx, dW, wt, db, M, N, K, ws, n, None)
    assert bwd(dy=None) == EINVAL and bwd(x=None) == EINVAL and bwd(W=None) == EINVAL and bwd(z=None) == EINVAL and bwd(z=None, act=0) == EINVAL
    assert bwd(K=4) == EUNSUPPORTED and bwd(wt=2) == EINVAL and bwd(act=9) == EINVAL and bwd(dx=PA + 8) == EINVAL and bwd(N=1 << 21) == EUNSUPPORTED and bwd(N=top) == EUNSUPPORTED and bwd(N=-1) == EINVAL
    assert bwd(ws=None) == EWORKSPACE and bwd(n=64) == EWORKSPACE and bwd(ws=(1 << 20) + 64) == EWORKSPACE
    for at in (PX, PY, PZ, PW):
        assert bwd(dx=at) == EINVAL and bwd(dW=at) == EINVAL and bwd(db=at) == EINVAL
    assert L.sd_gated_linear_bwd(PY, 0, None, None, PZ, 0, None, None, 0, None, 4, 8, 64, None, 0, None) == 0        # nothing asked for
    assert L.sd_gated_linear_bwd_workspace_bytes(0, 8, 8) == 256 and L.sd_gated_linear_bwd_workspace_bytes(top, top, top) == 256
    assert L.sd_gated_linear_bwd_workspace_bytes(100, 13, 8) >= 100 * 32 * 2 + 4 * 13 * 4
    zeros = lambda M, N, K, **kw: L.sd_gated_linear_bwd(None, 0, None, None, None, 0, kw.get("dx"), kw.get("dW"), 0, kw.get("db"), M, N, K, None, 0, None)
    with B.dry_run() as names:
        assert bwd() == 0 and bwd(x=None, dW=None) == 0 and bwd(W=None, dx=None) == 0 and bwd(dx=None, dW=None, x=None, W=None) == 0
        assert zeros(0, 8, 64, dW=PA, db=PB) == 0 and zeros(3, 0, 64, dx=PA) == 0 and zeros(0, (1 << 21) - 1, 4104, dW=PA) == EUNSUPPORTED
    assert names[0] == "gated dz" and names.count("gated dz") == 3 and names.count("gated dz sums only") == 1


def lin8(L, x=PX, xs=PA, xl=8, W=PW, wsc=PB, wl=12, b=PC, act=0, r=None, y=PY, yt=0, M=6, N=11, K=64):
    return L.sd_linear_fp8_fwd(x, xs, xl, W, wsc, wl, b, act, r, y, yt, M, N, K, None)


def gat8(L, x=PX, xs=PA, xl=8, W=PW, wsc=PB, wl=64, b=PC, act=3, y=PY, yt=2, ys=PD, yl=8, M=6, N=32, K=64, ws=None, n=0):
    return L.sd_gated_linear_fp8_fwd(x, xs, xl, W, wsc, wl, b, act, y, yt, ys, yl, M, N, K, ws, n, None)


def test_linear_fp8_refusals(B):
    L = B.lib()
    for f in (lin8, gat8):
        for k in ("x", "xs", "W", "wsc", "y"):
            assert f(L, **{k: None}) == EINVAL, k
        for k, p in (("x", PX), ("xs", PA), ("W", PW), ("wsc", PB), ("b", PC), ("y", PY)):
            assert f(L, **{k: p + 8}) == EINVAL, k
        assert f(L, xl=4) == EINVAL and f(L, xl=7) == EINVAL and f(L, wl=8) == EINVAL and f(L, wl=66) == EINVAL and f(L, xl=-8) == EINVAL
        for K in (0, 8, 24, 1 << 22):
            assert f(L, K=K) == EUNSUPPORTED, K
        assert f(L, act=5) == EINVAL and f(L, yt=3) == EINVAL and f(L, M=-1) == EINVAL and f(L, N=-16) == EINVAL
        assert f(L, M=1 << 27, xl=1 << 27) == EUNSUPPORTED and f(L, N=1 << 22, wl=1 << 23) == EUNSUPPORTED
        for at in (PX, PA, PW, PB, PC):
            assert f(L, y=at) == EINVAL
        assert f(L, x=None, M=0) == 0 and f(L, W=None, N=0) == 0
    assert lin8(L, yt=2) == EINVAL and lin8(L, r=PD + 4) == EINVAL
    assert gat8(L, ys=None) == EINVAL and gat8(L, ys=PD + 4) == EINVAL and gat8(L, yl=4) == EINVAL and gat8(L, yl=10) == EINVAL and gat8(L, ys=PY) == EINVAL
    assert gat8(L, N=24) == EUNSUPPORTED and gat8(L, N=24, yt=0) == EUNSUPPORTED and gat8(L, N=1 << 21, wl=1 << 23) == EUNSUPPORTED
    for at in (PX, PA, PW, PB, PC):
        assert gat8(L, ys=at) == EINVAL
    big = 1 << 30
    with B.dry_run():
        assert lin8(L) == 0 and lin8(L, r=PY) == 0 and lin8(L, r=PD, yt=1, b=None) == 0 and gat8(L) == 0 and gat8(L, yt=0, ys=None, yl=0) == 0 and gat8(L, yt=1, b=None) == 0
        assert lin8(L, M=1 << 20, xl=big, N=1 << 14, wl=big) == EUNSUPPORTED and lin8(L, M=1 << 20, xl=big, N=8192, wl=big) == 0
        assert gat8(L, M=1 << 20, xl=big, yl=big, N=8192, wl=big) == EUNSUPPORTED and gat8(L, M=1 << 20, xl=big, yl=big, N=4096, wl=big) == 0
        # by way of fp32 where the query asks for room
        need = L.sd_gated_linear_fp8_workspace_bytes(6, 32, 5120)
        assert need == 6 * 32 * 4 and L.sd_gated_linear_fp8_workspace_bytes(6, 32, 64) == 0
        assert gat8(L, K=5120) == EWORKSPACE and gat8(L, K=5120, ws=PE, n=need - 1) == EWORKSPACE and gat8(L, K=5120, ws=PE + 16, n=big) == EWORKSPACE and gat8(L, K=5120, ws=PE, n=need) == 0
        assert gat8(L, K=5120, yt=0, ys=None, yl=0) == 0
    top = 2 ** 31 - 1
    assert L.sd_gated_linear_fp8_workspace_bytes(top, top, top) == 0 and L.sd_gated_linear_fp8_workspace_bytes(-1, 16, 16) == 0 and L.sd_gated_linear_fp8_workspace_bytes(4, 16, 0) == 0


def test_workspaces_are_large_enough_for_what_is_launched(B):
    """Whatever the sizes, two launches where the query asks for room, and one where it does not"""
    import random
    L, rng = B.lib(), random.Random(3)
    for _ in range(400):
        M, N, K = int(2 ** rng.uniform(0, 14)), 16 * int(2 ** rng.uniform(0, 9)), 16 * int(2 ** rng.uniform(0, 9))
        need = L.sd_gated_linear_fp8_workspace_bytes(M, N, K)
        with B.dry_run() as names:
            assert gat8(L, M=M, N=N, K=K, xl=1 << 20, yl=1 << 20, wl=1 << 20, ws=PE if need else None, n=need) == 0
        assert len(names) == (2 if need else 1) and (names[-1] == "quantize") == bool(need) and need in (0, (M * N * 4 + 255) // 256 * 256)


def test_every_access_of_a_tile_is_inside(B):
    """The tiles' loads, by the arithmetic of the kernels: rows, chunks and scale words of every lane, wavefront and step stay inside the operands"""
    def spread(b, i, B_):
        return b // B_ * 16 * B_ + B_ * i + b % B_
    shapes = [(256, 256, 4, 2), (256, 256, 2, 4), (128, 256, 2, 4), (128, 256, 4, 2), (256, 128, 4, 2), (128, 192, 4, 2), (96, 128, 1, 4), (128, 128, 2, 2), (64, 128, 2, 2), (64, 128, 2, 4), (64, 64, 2, 2), (64, 64, 2, 1), (64, 256, 2, 2), (32, 256, 1, 2)]
    for BM, BN, WGM, WGN in shapes:
        for gated_, bq in ((False, 2), (True, 2), (True, 4)):
            NW, WM, WN = WGM * WGN, BM // WGM, BN // WGN
            NV = WN // 16 // 2 if gated_ else WN // 16
            if NV % bq or (bq == 4 and BN != 256):
                continue
            bp, bn_out, wn_out = 4 if WM // 16 % 4 == 0 else 2, BN // 2 if gated_ else BN, WN // 2 if gated_ else WN
            rows, cols = [], []
            for j in range((BM + BN) // 8 // NW):
                for wave in range(NW):
                    first = (j * NW + wave) * 8
                    for row in range(first, first + 8):
                        if j < BM // 8 // NW:
                            rows.append(first // WM * WM + spread(first % WM // 16, row % 16, bp))
                        else:
                            w, b = (first - BM) // WN, (first - BM) % WN // 16
                            gate = gated_ and b >= NV
                            cols.append((gate, w * wn_out + spread(b - NV if gate else b, row % 16, bq)))
            # every row of the tile once, value and gate
            assert sorted(rows) == list(range(BM))
            assert sorted(cols) == sorted((g, c) for g in ((False, True) if gated_ else (False,)) for c in range(bn_out))
            # scale words: of rows there are, for any number of them
            for M, N in ((1, 16), (5, 16), (BM + 3, bn_out + 16), (4 * BM - 1, 16)):
                for m0 in range(0, M, BM):
                    for a in range((BM + BN + 255) // 256 * 64):
                        jj = a * 4 - BM
                        at = min(m0 + (a * 4 if jj < 0 else 0), (M - 1) & ~3)
                        assert at % 4 == 0 and 0 <= at <= M - 1
                total = 2 * N if gated_ else N
                for n0 in range(0, N, bn_out):
                    for jj in range(0, BN, 4):
                        at = min(n0 + (N + jj - bn_out if gated_ and jj >= bn_out else jj), (total - 1) & ~3)
                        assert at % 4 == 0 and 0 <= at <= total - 1


def test_halved_steps(B):
    """Tiles whose wavefronts take half of each step: every row is loaded, also where some are dealt twice, and the halves' sums meet inside the stages"""
    for BM, BN, WGM, WGN, stages in ((96, 128, 1, 4, 3), (64, 128, 2, 2, 3), (64, 64, 2, 2, 4), (128, 128, 2, 2, 3), (64, 64, 2, 1, 4), (32, 256, 1, 2, 3)):
        group, total = WGM * WGN, (BM + BN) // 8
        waves = 2 * group
        dealt = [min(j * waves + w, total - 1) for j in range(-(-total // waves)) for w in range(waves)]
        assert sorted(set(dealt)) == list(range(total))
        blocks = (BM // WGM // 16) * (BN // WGN // 16)
        at = lambda wave, write: {(wave % group * blocks + ((1 - wave // group if write else wave // group) * blocks // 2 + i)) * 64 + lane for i in range(blocks // 2) for lane in range(64)}
        written = [at(w, True) for w in range(waves)]
        assert sum(map(len, written)) == len(set().union(*written)) and max(map(max, written)) < stages * (BM + BN) * 8
        for w in range(waves):
            assert at(w, False) == written[(w + group) % waves]       # what the other half wrote


def test_binding_refuses_what_the_c_call_cannot_see(B):
    import torch
    q, s = torch.zeros(6, 144, dtype=torch.float8_e4m3fn), torch.zeros(2, 8, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    ok = B._expect_fp8("x", B.Fp8Rows(q, s[:, :6]), 6, 144, -1)
    assert ok == (q.data_ptr(), s.data_ptr(), 8)
    for rows, what in ((B.Fp8Rows(q, s), "shape"), (B.Fp8Rows(q[:, :128], s[:, :6]), "shape"), (B.Fp8Rows(q, s[:1, :6]), "shape"), (B.Fp8Rows(q, torch.zeros(2, 6, dtype=torch.uint8).view(torch.float8_e8m0fnu)), "strides"),
                       (B.Fp8Rows(q, torch.zeros(8, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu).T[:, :6]), "strides"), (B.Fp8Rows(q, torch.zeros(14, dtype=torch.uint8).view(torch.float8_e8m0fnu).as_strided((2, 6), (8, 1))), "ends")):
        with pytest.raises(ValueError, match=what):
            B._expect_fp8("x", rows, 6, 144, -1)
    for rows in (B.Fp8Rows(q.view(torch.uint8), s[:, :6]), B.Fp8Rows(q, s[:, :6].view(torch.uint8)), B.Fp8Rows(q.float(), s[:, :6])):
        with pytest.raises(TypeError):
            B._expect_fp8("x", rows, 6, 144, -1)
    # one row: its scales a column, whose stride does not matter; one block
    one = torch.zeros(2, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    assert B._expect_fp8("x", B.Fp8Rows(q[:1], one[:, :1]), 1, 144, -1)[2] == 4
    assert B._expect_fp8("x", B.Fp8Rows(torch.zeros(8, 128, dtype=torch.float8_e4m3fn), s[:1]), 8, 128, -1)[2] == 8
    with pytest.raises(ValueError, match="not on a GPU"):
        B.quantize_fp8(torch.zeros(4, 64))


def shapes_of(name, pattern):
    import re
    text = open(LIB, "rb").read()
    return {m if isinstance(m, bytes) else tuple(map(int, m)) for m in re.findall(rb"_ZN2sd\d+" + name + pattern, text)}


def test_rmsnorm_kernels_are_all_launched(B):
    short, long = {(16, 1, 0), (16, 2, 1)}, {(64, 3, 1), (64, 5, 3), (64, 8, 5), (256, 4, 2), (256, 8, 4), (1024, 4, 2)}
    p = rb"I[^E]*?Li(\d+)ELi(\d+)ELi(\d+)E"
    assert shapes_of(b"rms_fwd_kernel", rb"I.{1,60}?Li(\d+)ELi(\d+)ELi(\d+)E") == short | {(16, 5, 2), (16, 8, 5)} | long
    assert shapes_of(b"rms_bwd_kernel", p) == shapes_of(b"rms_bwd_few_kernel", p) == short | {(64, 1, 0)} | long


@pytest.mark.parametrize("M,N,K,first", [(12, 3632, 1760, "few rows 8 bits gated 16x16"), (29, 1328, 1904, "few rows 8 bits gated 16x16"), (17, 2240, 2352, "few rows 8 bits gated 32x16"), (125, 992, 2576, "few rows 8 bits gated 32x16"),
                                         (2, 5680, 2592, "few rows 8 bits gated 32x32"), (242, 976, 3088, "few rows 8 bits gated 32x32"), (53, 15760, 2272, "gemm cols 8 bits wide gated 64x128"), (3, 15552, 4144, "gemm cols 8 bits wide gated 64x128"),
                                         (47, 7232, 3008, "gemm cols 8 bits wide gated 64x64"), (1, 5120, 1280, None), (1, 20000, 1280, None), (64, 1296, 640, None), (1, 5120, 128, None)])
def test_one_launch_or_two_by_what_is_launched(B, M, N, K, first):
    """Sizes of which two launches take 40 to 95 % of one's time go by way of fp32, and those of which one takes no longer do not"""
    L, ld = B.lib(), 1 << 20
    need = L.sd_gated_linear_fp8_workspace_bytes(M, N, K)
    assert bool(need) == (first is not None)
    with B.dry_run() as names:
        assert gat8(L, M=M, N=N, K=K, xl=ld, yl=ld, wl=ld, ws=PE if need else None, n=need) == 0
    assert (names[0].startswith(first) and names[1] == "quantize") if first else (len(names) == 1 and "to 8 bits 32x256" in names[0])


def test_whole_sums_are_widened(B):
    """SD_WHOLE_SUMS beside any activation: widened operands at every size and type of y, in the workspace that the query asks for"""
    import random
    L, rng, ld = B.lib(), random.Random(5), 1 << 20
    for f, yt in ((lin8, 0), (lin8, 1), (gat8, 0), (gat8, 1), (gat8, 2)):
        assert f(L, act=B.SD_WHOLE_SUMS + 5) == EINVAL and f(L, act=2 * B.SD_WHOLE_SUMS) == EINVAL and f(L, act=B.SD_WHOLE_SUMS - 1) == EINVAL and f(L, act=-1) == EINVAL
        for i in range(200):
            M, N, K = int(2 ** rng.uniform(0, 14)), 16 * int(2 ** rng.uniform(0, 8)), 16 * int(2 ** rng.uniform(0, 9))
            kw = dict(yl=ld, ys=PD, ws=PE, n=L.sd_gated_linear_fp8_workspace_bytes(M, N, K)) if f is gat8 else {}
            with B.dry_run() as names:
                assert f(L, M=M, N=N, K=K, xl=ld, wl=ld, yt=yt, act=B.SD_WHOLE_SUMS + i % 5, **kw) == 0
            assert "wide" in names[0] or "few rows" in names[0]
            assert names[1:] == (["quantize"] if kw.get("n") and yt == 2 else [])


def test_the_current_device_is_asked_for_by_its_public_name(B, monkeypatch):
    import torch

    class OnTheFirst:
        device = "cuda:0"
        get_device = staticmethod(lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert B._on(OnTheFirst) == 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="the current device is 1"):
        B._on(OnTheFirst)

"""Host logic of the 16-bit products and layer norm, without a GPU: exported symbols, refusals (all
decided before a device is touched), and the work decomposition."""
import os
import re

import pytest

import paper_2003_00532_b200 as dg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F16, BF16 = dg.HGEMM_TYPE_F16, dg.HGEMM_TYPE_BF16


@pytest.fixture(scope="module")
def lib():
    from paper_2003_00532_b200 import build as _build
    _build.build()
    return dg.load_library()


@pytest.mark.parametrize("header,names", [("hgemm.h", {"hgemm_epilogue", "hgemm_epilogue_bwd", "hgemm_gated", "hgemm_gated_bwd", "hgemm_plan",
                                                       "hgemm_last_device_status", "hgemm_set_test_drop_loads"}),
                                          ("layernorm.h", {"layernorm_fwd", "layernorm_bwd"})])
def test_declared_symbols_are_exported(lib, header, names):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    found = set(re.findall(r"DGEMM_API\s+[\w\s\*]+?\b((?:hgemm|layernorm)_\w+)\s*\(", text))
    assert names <= found
    for n in found:
        assert hasattr(lib, n), n


def test_headers_are_plain_c():
    import subprocess
    src = '#include "layernorm.h"\nint main(void){return HGEMM_TYPE_F32 + HGEMM_ACT_NONE;}\n'
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-x", "c", "-", "-fsyntax-only"],
                   input=src.encode(), check=True)


def test_constants_match_binding():
    text = open(os.path.join(ROOT, "include", "hgemm.h")).read()
    for name, val in re.findall(r"(HGEMM_(?:TYPE|ACT)_\w+)\s*=\s*(\d+)", text):
        if name != "HGEMM_ACT_COUNT":
            assert getattr(dg, name) == int(val), name


# addresses that no buffer has: a refused call must not get as far as using them
P = [0x10000000 * (i + 1) for i in range(10)]


def _epilogue(lib, type=BF16, ta=0, tb=0, M=4, N=6, K=8, A=P[0], lda=8, B=P[1], ldb=6, bias=None, act=0, R=None, ldr=6, D=P[2], ldd=6, Z=None, ldz=6):
    return lib.hgemm_epilogue(type, ta, tb, M, N, K, A, lda, B, ldb, bias, act, R, ldr, D, ldd, Z, ldz, None)


@pytest.mark.parametrize("change,code", [
    (dict(type=0), -9), (dict(type=3), -9), (dict(act=5), -9), (dict(act=-1), -9), (dict(ta=2), -1), (dict(tb=-1), -1),
    (dict(M=-1), -1), (dict(N=2 ** 31), -1), (dict(K=-5), -1), (dict(lda=7), -2), (dict(ldb=5), -2), (dict(ldd=5), -2),
    (dict(ta=1, lda=3), -2), (dict(tb=1, ldb=7), -2), (dict(R=P[3], ldr=5), -2), (dict(Z=P[3], ldz=1), -2),
    (dict(A=None), -3), (dict(B=None), -3), (dict(D=None), -3), (dict(A=P[0] + 1), -4), (dict(bias=P[4] + 1), -4), (dict(Z=P[3] + 1), -4),
    (dict(D=P[0]), -5), (dict(D=P[1] + 8), -5), (dict(Z=P[2]), -5), (dict(Z=P[0]), -5), (dict(bias=P[2] + 2), -5),
    (dict(R=P[2], ldr=7), -5),          # the residual may be D, but not a shifted or wider view of it
    (dict(R=P[2] + 2), -5), (dict(R=P[2], Z=P[2] + 4), -5)])
def test_epilogue_refusals(lib, change, code):
    assert _epilogue(lib, **change) == code


def test_empty_calls_inspect_nothing(lib):
    assert _epilogue(lib, M=0, A=None, D=None, lda=0) == 0
    assert _epilogue(lib, N=0, B=None) == 0
    assert lib.hgemm_gated(BF16, 0, 0, 5, 5, *([None, 0] * 3), 0, *([None, 0] * 3), None) == 0
    assert lib.layernorm_fwd(0, 0, 5, None, 0, None, None, 1e-5, None, 0, None, None, None) == 0
    assert lib.layernorm_bwd(0, 4, 0, None, 0, None, None, None, None, 0, None, 0, None, None, None) == 0


def test_gradient_refusals(lib):
    def bwd(A=P[0], Z=P[2], dD=P[3], dA=P[4], ldda=8, dB=P[5], db=P[6], act=4, lddd=6):
        return lib.hgemm_epilogue_bwd(BF16, 0, 0, 4, 6, 8, A, 8, P[1], 6, act, Z, 6, dD, lddd, dA, ldda, dB, 6, db, None)
    assert bwd(act=7) == -9 and bwd(dD=None) == -3 and bwd(Z=None) == -3 and bwd(A=None) == -3 and bwd(ldda=7) == -2
    assert bwd(lddd=5) == -2 and bwd(db=P[6] + 2) == -4 and bwd(dA=P[3]) == -5 and bwd(dB=P[4]) == -5 and bwd(db=P[5]) == -5

    def gated(U=P[4], dX=P[6], dWg=P[7], dWu=P[8], X=P[0], act=4):
        return lib.hgemm_gated_bwd(F16, 1, 4, 6, 8, X, 8, P[1], 8, P[2], 8, act, P[3], 6, U, 6, P[5], 6, dX, 8, dWg, 8, dWu, 8, None)
    assert gated(act=-2) == -9 and gated(U=None) == -3 and gated(X=None) == -3 and gated(dX=P[0]) == -5 and gated(dWu=P[7]) == -5
    assert gated(dX=P[6] + 1) == -4


def test_gated_refusals(lib):
    def call(type=F16, G=P[4], U=P[5], H=P[3], ldh=6, Wu=P[2]):
        return lib.hgemm_gated(type, 0, 4, 6, 8, P[0], 8, P[1], 6, Wu, 6, 4, H, ldh, G, 6, U, 6, None)
    assert call(type=0) == -9 and call(G=None) == -3 and call(U=None) == -3 and call(H=None) == -3 and call(ldh=5) == -2
    assert call(H=P[4]) == -5 and call(U=P[0]) == -5 and call(Wu=P[2] + 1) == -4


def test_layernorm_refusals(lib):
    def fwd(type=0, X=P[0], ldx=8, Y=P[1], mean=None, gamma=None, eps=1e-5, rows=4, cols=8):
        return lib.layernorm_fwd(type, rows, cols, X, ldx, gamma, None, eps, Y, 8, mean, None, None)
    assert fwd(type=3) == -9 and fwd(eps=-1.0) == -9 and fwd(eps=float("inf")) == -9 and fwd(rows=-1) == -1 and fwd(cols=2 ** 31) == -1
    assert fwd(ldx=7) == -2 and fwd(X=None) == -3 and fwd(X=P[0] + 2) == -4 and fwd(mean=P[3] + 2) == -4 and fwd(gamma=P[3] + 1) == -4
    assert fwd(Y=P[0]) == -5 and fwd(mean=P[1]) == -5 and fwd(gamma=P[1] + 16) == -5

    def bwd(mean=P[2], dX=P[5], dgamma=P[6], dbeta=P[7], type=2, dY=P[4]):
        return lib.layernorm_bwd(type, 4, 8, P[0], 8, P[1], mean, P[3], dY, 8, dX, 8, dgamma, dbeta, None)
    assert bwd(type=-1) == -9 and bwd(mean=None) == -3 and bwd(dY=None) == -3 and bwd(dX=P[4]) == -5 and bwd(dbeta=P[6]) == -5
    assert bwd(dgamma=P[6] + 2) == -4


def test_plan_arguments(lib):
    for bad in ((0, 4, 4), (4, -1, 4), (4, 4, 0), (2 ** 31, 4, 4)):
        with pytest.raises(dg.DgemmError):
            dg.hgemm_plan(*bad)
    assert lib.hgemm_plan(4, 4, 4, 0, 0, None) == -3
    with pytest.raises(dg.DgemmError):
        dg.hgemm_set_test_drop_loads(-1)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("sms", [0, 148, 20, 2])
def test_plan_covers_every_tile_and_k_block_once(sms, gated):
    import random
    rng = random.Random(sms + gated)
    shapes = [(1, 1, 1), (1, 4096, 4096), (8192, 4096, 8192), (16, 128, 100000), (1000, 1537, 777), (2088, 2088, 2088), (4097, 31, 4099)]
    shapes += [tuple(int(2 ** rng.uniform(0, 13)) for _ in range(3)) for _ in range(200)]
    for M, N, K in shapes:
        p = dg.hgemm_plan(M, N, K, gated=gated, sm_count=sms)
        assert p["kblocks"] == -(-K // 64)
        tiles = -(-M // p["tile_rows"]) * -(-N // p["tile_cols"])
        limit = (sms or 148) // p["ctas_per_tile"]
        # whole rounds take one tile per cluster each; what is left over is less than a round
        assert p["rounds"] * limit + p["rest"] == tiles and 0 <= p["rest"] < limit
        if p["span"] == 0:
            assert p["clusters"] == (limit if p["rounds"] else p["rest"])
        else:
            # equal spans that cover all k-blocks left over, each shorter than a tile, none empty
            # (end to end, or every tile cut alike into parts of its own)
            assert 0 < p["span"] < p["kblocks"]
            used = {-(-p["rest"] * p["kblocks"] // p["span"]), p["rest"] * -(-p["kblocks"] // p["span"])}
            assert min(used) <= limit and p["clusters"] in ({limit} if p["rounds"] else used)

"""RMS norm, rows in 8 bits, dropout and the products of 8-bit operands without a GPU: exported symbols, headers, refusals (all decided
before a device is touched), and the generator of dropout's mask against its published words."""
import os
import re

import pytest

import paper_2003_00532_b200 as dg
import rows_reference as rr

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, F16, BF16 = dg.HGEMM_TYPE_F32, dg.HGEMM_TYPE_F16, dg.HGEMM_TYPE_BF16
P = [0x10000000 * (i + 1) for i in range(10)]   # addresses that no buffer has


@pytest.fixture(scope="module")
def lib():
    from paper_2003_00532_b200 import build as _build
    _build.build()
    return dg.load_library()


@pytest.mark.parametrize("header,names", [
    ("rmsnorm.h", {"rmsnorm_fwd", "rmsnorm_fwd_e4m3", "quantize_rows_e4m3", "rmsnorm_bwd"}),
    ("dropout.h", {"dropout_fwd", "dropout_bwd"}), ("qgemm.h", {"qgemm_epilogue", "qgemm_gated"})])
def test_declared_symbols_are_exported_and_bound(lib, header, names):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    found = set(re.findall(r"DGEMM_API\s+[\w\s\*]+?\b(\w+)\s*\(", text))
    assert names == found
    from paper_2003_00532_b200 import binding
    for n in found:
        assert hasattr(lib, n) and n in binding.MARSHALLED and callable(getattr(dg, n))


def test_headers_are_plain_c():
    import subprocess
    src = '#include "dropout.h"\n#include "qgemm.h"\n#include "rmsnorm.h"\nint main(void){return HGEMM_TYPE_F32;}\n'
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-x", "c", "-", "-fsyntax-only"],
                   input=src.encode(), check=True)


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))])
def test_the_generator_gives_its_published_words(counter, key, want):
    assert tuple(rr.philox(counter, key)) == want


def test_words_of_a_matrix():
    w = rr.words(3, 10, 0x299f31d0a4093822, 0x0370734413198a2e, "cpu", first_row=5, first_col=8)
    for i in range(3):
        for j in range(10):
            assert int(w[i, j]) == rr.philox((2 + j // 4, 5 + i, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0))[j % 4]


def _fwd(lib, type=BF16, rows=4, cols=6, X=P[0], ldx=6, R=None, ldr=6, gamma=None, eps=1e-5, S=None, lds=6, Y=P[1], ldy=6, rstd=None):
    return lib.rmsnorm_fwd(type, rows, cols, X, ldx, R, ldr, gamma, eps, S, lds, Y, ldy, rstd, None)


@pytest.mark.parametrize("change,code", [
    (dict(type=3), -9), (dict(type=-1), -9), (dict(eps=-1.0), -9), (dict(eps=float("nan")), -9), (dict(eps=float("inf")), -9),
    (dict(rows=-1), -1), (dict(cols=2 ** 31), -1), (dict(ldx=5), -2), (dict(ldy=5), -2), (dict(R=P[2], ldr=5), -2), (dict(S=P[2], lds=1), -2),
    (dict(X=None), -3), (dict(Y=None), -3), (dict(X=P[0] + 1), -4), (dict(Y=P[1] + 1), -4), (dict(gamma=P[4] + 1), -4), (dict(rstd=P[4] + 2), -4),
    (dict(type=F32, X=P[0] + 2), -4), (dict(R=P[2] + 1), -4),
    (dict(Y=P[0]), -5), (dict(R=P[2], Y=P[2]), -5), (dict(S=P[1]), -5), (dict(rstd=P[1] + 8), -5), (dict(rstd=P[0] + 4), -5),
    (dict(S=P[0], lds=7), -5), (dict(S=P[0] + 2), -5), (dict(R=P[2], S=P[2] + 12), -5), (dict(gamma=P[1] + 4), -5),
    (dict(R=P[0], S=P[2], gamma=P[2] + 2), -5), (dict(rows=0, X=None), 0), (dict(cols=0, Y=None), 0)])
def test_refusals_of_the_norm(lib, change, code):
    assert _fwd(lib, **change) == code


def test_the_sum_may_take_an_operands_place(lib):
    # not refused: these get as far as the device, which is not there (or, with one, would be used)
    if __import__("torch").cuda.is_available():
        pytest.skip("the addresses are no buffers")
    for change in (dict(S=P[0]), dict(R=P[2], S=P[2]), dict(R=P[2], S=P[0]), dict(R=P[0], S=P[0])):
        assert _fwd(lib, **change) == -6


@pytest.mark.parametrize("change,code", [
    (dict(type=3), -9), (dict(eps=-1.0), -9), (dict(ldq=5), -2), (dict(Q=None), -3), (dict(scale=None), -3), (dict(scale=P[2] + 1), -4),
    (dict(Q=P[0] + 47), -5), (dict(Q=P[2]), -5), (dict(scale=P[0]), -5), (dict(S=P[1]), -5), (dict(rstd=P[2]), -5), (dict(rows=0), 0)])
def test_refusals_of_the_norm_to_8_bits(lib, change, code):
    a = dict(type=BF16, rows=4, cols=6, X=P[0], ldx=6, R=None, ldr=6, gamma=None, eps=1e-5, S=None, lds=6, Q=P[1], ldq=6, scale=P[2], rstd=None)
    a.update(change)
    assert lib.rmsnorm_fwd_e4m3(*a.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(type=3), -9), (dict(rows=-1), -1), (dict(ldx=5), -2), (dict(ldq=5), -2), (dict(X=None), -3), (dict(Q=None), -3), (dict(scale=None), -3),
    (dict(X=P[0] + 1), -4), (dict(scale=P[2] + 2), -4), (dict(Q=P[0]), -5), (dict(scale=P[1] + 16), -5), (dict(cols=0), 0)])
def test_refusals_of_rows_to_8_bits(lib, change, code):
    a = dict(type=F16, rows=4, cols=6, X=P[0], ldx=6, Q=P[1], ldq=6, scale=P[2])
    a.update(change)
    assert lib.quantize_rows_e4m3(*a.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(type=7), -9), (dict(cols=-1), -1), (dict(rows=2 ** 31), -1), (dict(lds=5), -2), (dict(lddy=5), -2), (dict(dS=P[5], ldds=5), -2), (dict(lddx=5), -2),
    (dict(S=None), -3), (dict(dY=None), -3), (dict(rstd=None), -3), (dict(dX=P[3] + 1), -4), (dict(dgamma=P[4] + 2), -4), (dict(rstd=P[1] + 2), -4),
    (dict(dX=P[0]), -5), (dict(dX=P[2]), -5), (dict(dS=P[3], ldds=7), -5), (dict(dS=P[3] + 2), -5), (dict(dgamma=P[3] + 8), -5), (dict(dgamma=P[1]), -5),
    (dict(dS=P[3], dgamma=P[3] + 8), -5), (dict(gamma=P[3] + 4), -5), (dict(cols=0), 0)])
def test_refusals_of_the_norms_gradients(lib, change, code):
    a = dict(type=BF16, rows=4, cols=6, S=P[0], lds=6, gamma=None, rstd=P[1], dY=P[2], lddy=6, dS=None, ldds=6, dX=P[3], lddx=6, dgamma=P[4])
    a.update(change)
    assert lib.rmsnorm_bwd(*a.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(type=3), -9), (dict(p=-0.1), -9), (dict(p=1.5), -9), (dict(p=float("nan")), -9), (dict(rows=-1), -1), (dict(ldx=5), -2), (dict(ldy=5), -2),
    (dict(R=P[3], ldr=2), -2), (dict(X=None), -3), (dict(Y=None), -3), (dict(X=P[0] + 1), -4), (dict(step=P[4] + 4), -4), (dict(Y=P[0] + 2), -5),
    (dict(Y=P[0], ldy=7), -5), (dict(R=P[1] + 2), -5), (dict(R=P[1], ldr=8), -5), (dict(step=P[1]), -5), (dict(rows=0, X=None), 0)])
def test_refusals_of_dropout(lib, change, code):
    a = dict(type=BF16, rows=4, cols=6, X=P[0], ldx=6, R=None, ldr=6, p=0.5, seed=2 ** 64 - 1, offset=3, step=None, Y=P[1], ldy=6)
    a.update(change)
    assert lib.dropout_fwd(*a.values(), None) == code
    if "R" not in change:
        del a["R"], a["ldr"]
        assert lib.dropout_bwd(*a.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(type=F32), -9), (dict(act=5), -9), (dict(M=-1), -1), (dict(K=2 ** 31), -1), (dict(lda=7), -2), (dict(ldb=7), -2), (dict(ldd=5), -2),
    (dict(R=P[5], ldr=5), -2), (dict(Z=P[5], ldz=5), -2), (dict(A=None), -3), (dict(B=None), -3), (dict(D=None), -3), (dict(D=P[4] + 1), -4),
    (dict(sa=P[2] + 2), -4), (dict(sb=P[3] + 1), -4), (dict(bias=P[6] + 1), -4), (dict(D=P[0] + 30), -5), (dict(D=P[1]), -5), (dict(sa=P[4]), -5),
    (dict(sb=P[4] + 4), -5), (dict(Z=P[4]), -5), (dict(R=P[4], ldr=7), -5), (dict(bias=P[4]), -5), (dict(M=0, A=None), 0), (dict(N=0, B=None), 0)])
def test_refusals_of_the_product(lib, change, code):
    a = dict(type=BF16, M=4, N=6, K=8, A=P[0], lda=8, sa=P[2], B=P[1], ldb=8, sb=P[3], bias=None, act=0, R=None, ldr=6, D=P[4], ldd=6, Z=None, ldz=6)
    a.update(change)
    assert lib.qgemm_epilogue(*a.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(type=0), -9), (dict(act=-1), -9), (dict(F=-1), -1), (dict(ldx=7), -2), (dict(ldwu=7), -2), (dict(ldh=5), -2), (dict(X=None), -3), (dict(Wu=None), -3),
    (dict(G=P[7]), -3), (dict(U=P[7]), -3), (dict(sg=P[8] + 2), -4), (dict(H=P[3] + 1), -4), (dict(H=P[0]), -5), (dict(G=P[7], U=P[7]), -5), (dict(su=P[3]), -5),
    (dict(M=0), 0)])
def test_refusals_of_the_gated_projections(lib, change, code):
    a = dict(type=F16, M=4, F=6, K=8, X=P[0], ldx=8, sx=None, Wg=P[1], ldwg=8, sg=None, Wu=P[2], ldwu=8, su=None, act=4, H=P[3], ldh=6, G=None, ldg=6,
             U=None, ldu=6)
    a.update(change)
    assert lib.qgemm_gated(*a.values(), None) == code


def test_arguments_of_the_python_names():
    import torch
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises((ValueError, RuntimeError)):
        dg.rmsnorm_fwd(x, None, x)               # host tensors
    with pytest.raises(TypeError):
        dg.rmsnorm_fwd(x, None)
    with pytest.raises(TypeError):
        dg.dropout_fwd(x, x, 0.1)
    with pytest.raises(TypeError):
        dg.qgemm_epilogue(x, x, x, scale=None)
    with pytest.raises(TypeError):
        dg.quantize_rows_e4m3(x, x, x, x, x, x, x)

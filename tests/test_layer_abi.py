"""CPU-only: the layer operators refuse bad arguments before they touch a device, and empty problems need none."""
import pytest


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import build
    build.build_library()
    from paper_2506_11728_b200 import binding
    return binding


P = 4096     # an aligned non-NULL address; never dereferenced on these paths


def test_rows(mg):
    bad = mg.ERR_INVALID_ARG
    for fn in (lambda t, M, N, X, ldx, Q, ldq, s: mg.mipgemm_quantize_rows(t, M, N, X, ldx, Q, ldq, s, 0, check=False),
               lambda t, M, N, X, ldx, Q, ldq, s: mg.mipgemm_dequantize_rows(t, M, N, Q, ldq, s, X, ldx, 0, check=False)):
        assert fn(3, 4, 8, P, 8, P, 8, P) == bad
        assert fn(-1, 4, 8, P, 8, P, 8, P) == bad
        assert fn(0, -1, 8, P, 8, P, 8, P) == bad
        assert fn(0, 4, 8, P, 7, P, 8, P) == bad
        assert fn(0, 4, 8, P, 8, P, 7, P) == bad
        assert fn(0, 4, 8, 0, 8, P, 8, P) == bad
        assert fn(0, 4, 8, P, 8, 0, 8, P) == bad
        assert fn(0, 4, 8, P, 8, P, 8, 0) == bad
        assert fn(0, 4, 8, P + 2, 8, P, 8, P) == bad       # float32 matrix on a 2-byte boundary
        assert fn(2, 4, 8, P + 1, 8, P, 8, P) == bad
        assert fn(0, 4, 8, P, 8, P, 8, P + 2) == bad
        assert fn(0, 0, 8, 0, 8, 0, 8, 0) == mg.OK


def linear(mg, t=0, act=0, M=4, N=8, K=16, A=P, lda=16, B=P, ldb=16, bs=P, bias=0, R=0, ldr=0, C=P, ldc=8, a_s=P, u8=False):
    fn = mg.mipgemm_u8s8_linear if u8 else mg.mipgemm_s8s8_linear
    return fn(t, act, M, N, K, A, lda, a_s, B, ldb, bs, bias, R, ldr, C, ldc, 0, check=False)


@pytest.mark.parametrize("wrong", [dict(t=3), dict(t=-1), dict(act=5), dict(act=-1), dict(M=-1), dict(N=-1), dict(K=-1), dict(lda=15),
                                   dict(ldb=15), dict(ldc=7), dict(A=0), dict(B=0), dict(C=0), dict(C=P + 2), dict(t=1, C=P + 1),
                                   dict(R=P, ldr=7), dict(R=P + 2, ldr=8), dict(bias=P + 1), dict(a_s=P + 2), dict(bs=P + 3)])
def test_linear_refuses(mg, wrong):
    assert linear(mg, **wrong) == mg.ERR_INVALID_ARG
    assert linear(mg, u8=True, **wrong) == mg.ERR_INVALID_ARG


def test_linear_limits(mg):
    assert linear(mg, K=131072, lda=131072, ldb=131072) == mg.ERR_K_TOO_LARGE
    assert linear(mg, K=65794, lda=65794, ldb=65794, u8=True) == mg.ERR_K_TOO_LARGE
    assert linear(mg, M=0, A=0, C=0) == mg.OK
    assert linear(mg, N=0, ldc=0, B=0, C=0) == mg.OK
    assert mg.mipgemm_last_path() & mg.PATH_MASK == mg.PATH_TRIVIAL


def gated(mg, t=0, act=4, M=4, F=8, K=16, X=P, ldx=16, xs=P, G=P, ldg=16, gs=P, U=P, ldu=16, us=P, H=P, ldh=8):
    return mg.mipgemm_s8s8_gated(t, act, M, F, K, X, ldx, xs, G, ldg, gs, U, ldu, us, H, ldh, 0, check=False)


@pytest.mark.parametrize("wrong", [dict(t=3), dict(act=5), dict(M=-1), dict(F=-1), dict(K=-1), dict(ldx=15), dict(ldg=15), dict(ldu=15),
                                   dict(ldh=7), dict(X=0), dict(G=0), dict(U=0), dict(H=0), dict(H=P + 2), dict(xs=P + 1), dict(gs=P + 1),
                                   dict(us=P + 2)])
def test_gated_refuses(mg, wrong):
    assert gated(mg, **wrong) == mg.ERR_INVALID_ARG


def test_gated_limits(mg):
    assert gated(mg, K=131072, ldx=131072, ldg=131072, ldu=131072) == mg.ERR_K_TOO_LARGE
    assert gated(mg, M=0, H=0) == mg.OK and gated(mg, F=0, ldh=0, H=0) == mg.OK


def grad(mg, t=0, act=4, M=4, F=8, K=16, X=P, ldx=16, xs=P, G=P, ldg=16, gs=P, U=P, ldu=16, us=P, dH=P, lddh=8, dG=P, lddg=8, dU=P, lddu=8):
    return mg.mipgemm_s8s8_gated_grad(t, act, M, F, K, X, ldx, xs, G, ldg, gs, U, ldu, us, dH, lddh, dG, lddg, dU, lddu, 0, check=False)


@pytest.mark.parametrize("wrong", [dict(t=3), dict(act=5), dict(M=-1), dict(K=-1), dict(ldx=15), dict(ldg=15), dict(ldu=15), dict(X=0), dict(G=0),
                                   dict(U=0), dict(dH=0), dict(dG=0), dict(dU=0), dict(lddh=7), dict(lddg=7), dict(lddu=7), dict(dH=P + 2),
                                   dict(dG=P + 2), dict(dU=P + 1), dict(us=P + 2)])
def test_gated_grad_refuses(mg, wrong):
    assert grad(mg, **wrong) == mg.ERR_INVALID_ARG


def test_gated_grad_limits(mg):
    assert grad(mg, K=131072, ldx=131072, ldg=131072, ldu=131072) == mg.ERR_K_TOO_LARGE
    assert grad(mg, M=0) == mg.OK


def product(mg, t=0, order=0, M=4, N=8, K=16, A=P, lda=16, B=P, ldb=8, s=P, C=P, ldc=8):
    return mg.mipgemm_bf16s8_product(t, order, M, N, K, A, lda, B, ldb, s, C, ldc, 0, 0, check=False)


@pytest.mark.parametrize("wrong", [dict(t=1), dict(t=3), dict(order=2), dict(M=-1), dict(N=-1), dict(K=-1), dict(lda=15), dict(order=1, lda=3),
                                   dict(ldb=7), dict(ldc=7), dict(A=0), dict(B=0), dict(C=0), dict(A=P + 1), dict(C=P + 2), dict(t=2, C=P + 1),
                                   dict(s=P + 2)])
def test_product_refuses(mg, wrong):
    assert product(mg, **wrong) == mg.ERR_INVALID_ARG


def test_product_limits(mg):
    assert product(mg, M=0) == mg.OK and product(mg, N=0, ldb=0, ldc=0) == mg.OK

"""CPU-only: the operators in 8-bit floating point and the step between two blocks refuse bad arguments before they touch a
device, and empty problems need none.  And the definitions that their GPU tests compare with, against others' outputs."""
import numpy as np
import pytest

import float8_util as f


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import build
    build.build_library()
    from paper_2506_11728_b200 import binding
    return binding


P = 4096     # an aligned non-NULL address; never dereferenced on these paths


def quantize(mg, t=0, f=0, M=200, N=300, X=P, ldx=300, Qr=P, ldqr=300, rs=P, ldrs=200, Qc=P, ldqc=300, cs=P, ldcs=300):
    return mg.mipgemm_f8_quantize(t, f, M, N, X, ldx, Qr, ldqr, rs, ldrs, Qc, ldqc, cs, ldcs, 0, check=False)


@pytest.mark.parametrize("wrong", [dict(t=3), dict(t=-1), dict(f=2), dict(f=-1), dict(M=-1), dict(N=-1), dict(ldx=299), dict(X=0), dict(X=P + 2),
                                   dict(ldqr=299), dict(ldqc=299), dict(ldrs=199), dict(ldcs=299), dict(Qr=0), dict(rs=0), dict(Qc=0), dict(cs=0),
                                   dict(rs=P + 2), dict(cs=P + 1), dict(Qr=0, rs=0, Qc=0, cs=0), dict(t=2, X=P + 1)])
def test_quantize_refuses(mg, wrong):
    assert quantize(mg, **wrong) == mg.ERR_INVALID_ARG


def squares(mg, t=0, f=0, M=200, N=300, X=P, ldx=300, Q=P, ldq=300, s=P, lds=3):
    return mg.mipgemm_f8_quantize_squares(t, f, M, N, X, ldx, Q, ldq, s, lds, 0, check=False)


@pytest.mark.parametrize("wrong", [dict(t=3), dict(f=2), dict(M=-1), dict(ldx=299), dict(X=0), dict(ldq=299), dict(lds=2), dict(Q=0), dict(s=0),
                                   dict(Q=0, s=0), dict(s=P + 2)])
def test_squares_refuse(mg, wrong):
    assert squares(mg, **wrong) == mg.ERR_INVALID_ARG


def dequantize(mg, t=0, f=0, b=0, M=200, N=300, Q=P, ldq=300, s=P, lds=200, X=P, ldx=300):
    return mg.mipgemm_f8_dequantize(t, f, b, M, N, Q, ldq, s, lds, X, ldx, 0, check=False)


@pytest.mark.parametrize("wrong", [dict(t=3), dict(f=2), dict(b=3), dict(b=-1), dict(M=-1), dict(N=-1), dict(ldq=299), dict(ldx=299), dict(lds=199),
                                   dict(b=1, lds=299), dict(b=2, lds=2), dict(Q=0), dict(s=0), dict(X=0), dict(s=P + 2), dict(X=P + 2)])
def test_dequantize_refuses(mg, wrong):
    assert dequantize(mg, **wrong) == mg.ERR_INVALID_ARG


def product(mg, t=0, fa=0, fb=0, ao=0, bo=0, bb=2, M=200, N=300, K=400, A=P, lda=400, sa=P, ldas=200, B=P, ldb=400, sb=P, ldbs=4, bias=0, R=0,
            ldr=300, C=P, ldc=300):
    return mg.mipgemm_f8f8_product(t, fa, fb, ao, bo, bb, M, N, K, A, lda, sa, ldas, B, ldb, sb, ldbs, bias, R, ldr, C, ldc, 0, check=False)


@pytest.mark.parametrize("wrong", [dict(t=3), dict(fa=2), dict(fb=-1), dict(ao=2), dict(bo=2), dict(bb=1), dict(bb=3), dict(bo=1, bb=0), dict(M=-1),
                                   dict(N=-1), dict(K=-1), dict(lda=399), dict(ao=1, lda=199), dict(ldb=399), dict(bo=1, ldb=299), dict(ldc=299),
                                   dict(R=P, ldr=299), dict(R=P, C=P, ldr=301), dict(ldas=199), dict(ldbs=3), dict(bo=1, ldb=300, ldbs=2),
                                   dict(bb=0, ldbs=299), dict(A=0), dict(B=0), dict(C=0), dict(C=P + 2), dict(t=2, C=P + 1), dict(R=P + 2),
                                   dict(sa=P + 1), dict(sb=P + 2), dict(bias=P + 3)])
def test_product_refuses(mg, wrong):
    assert product(mg, **wrong) == mg.ERR_INVALID_ARG


ROOM = dict(X=P, ldx=64, Z=P, ldz=64, Y=P, ldy=64, H=P, ldh=64)


def norm_step(mg, t=0, post=1, pre=1, M=20, N=64, eps=1e-5, **more):
    return mg.mipgemm_norm_step(t, post, pre, M, N, eps, **dict(ROOM, **more), stream=0, check=False)


STEP_WRONG = [dict(t=3), dict(post=3), dict(pre=-1), dict(M=-1), dict(N=-1), dict(N=32769, ldx=40000, ldz=40000, ldy=40000, ldh=40000), dict(eps=-1.0),
              dict(eps=float("nan")), dict(drop=-0.1), dict(drop=1.0), dict(drop=0.999999), dict(drop=float("nan")), dict(ldx=63), dict(ldz=63),
              dict(ldy=63), dict(ldh=63), dict(X=P + 2), dict(Z=P + 1), dict(H=P + 2), dict(gate=P, ldgate=63), dict(gate=P, ldgate=64, gate_rows=0),
              dict(gate=P + 2, ldgate=64), dict(counter=P + 4), dict(post_weight=P + 2), dict(pre_weight=P + 1), dict(post=2, post_bias=P + 2),
              dict(post_bias=P), dict(pre_bias=P), dict(post=0, post_weight=P), dict(pre=0, H=None, pre_weight=P), dict(pre=0), dict(stats=P + 2),
              dict(Z=None), dict(Z=None, post=0, drop=0.5), dict(Z=None, post=0, gate=P, ldgate=64), dict(X=None, Z=None, post=0),
              dict(Y=None, H=None), dict(codes=4), dict(codes=-1), dict(codes=1, Q=None, ldq=64, q_scale=P), dict(codes=1, Q=P, ldq=63, q_scale=P),
              dict(codes=1, Q=P, ldq=64, q_scale=None), dict(codes=2, Q=P, ldq=64, q_scale=P, ldqs=19), dict(codes=2, Q=P, ldq=64, q_scale=P + 2, ldqs=20),
              dict(pre=0, H=None, codes=1, Q=P, ldq=64, q_scale=P), dict(Y=2 * P, X=2 * P, ldx=65)]


@pytest.mark.parametrize("wrong", STEP_WRONG)
def test_norm_step_refuses(mg, wrong):
    assert norm_step(mg, **wrong) == mg.ERR_INVALID_ARG


GRAD_ROOM = dict(dY=P, lddy=64, dH=P, lddh=64, Y=P, ldy=64, Z=P, ldz=64, stats=P, dX=2 * P, lddx=64, dZ=3 * P, lddz=64)


def norm_step_grad(mg, t=0, post=1, pre=1, M=20, N=64, **more):
    return mg.mipgemm_norm_step_grad(t, post, pre, M, N, **dict(GRAD_ROOM, **more), stream=0, check=False)


GRAD_WRONG = [dict(t=3), dict(post=3), dict(pre=3), dict(M=-1), dict(N=-1), dict(N=40000, lddy=40000, lddh=40000, ldy=40000, ldz=40000, lddx=40000, lddz=40000),
              dict(drop=1.0), dict(drop=-1.0), dict(lddy=63), dict(lddh=63), dict(ldy=63), dict(ldz=63), dict(lddx=63), dict(lddz=63), dict(dY=P + 2),
              dict(Z=P + 1), dict(dX=P + 2), dict(stats=None), dict(stats=P + 2), dict(dH=None), dict(Y=None), dict(Z=None), dict(pre=0), dict(pre=0, dH=None, dY=None),
              dict(dgate=P, lddgate=64), dict(gate=P, ldgate=64, dgate=P, lddgate=63), dict(gate=P, ldgate=64, gate_rows=0), dict(counter=P + 2),
              dict(dpost_bias=P), dict(dpre_bias=P), dict(post=0, dpost_weight=P), dict(post=0, post_weight=P), dict(pre=0, dH=None, dpre_weight=P),
              dict(dpre_weight=P + 2), dict(dX=None, dZ=None), dict(dX=P, lddx=65)]


@pytest.mark.parametrize("wrong", GRAD_WRONG)
def test_norm_step_grad_refuses(mg, wrong):
    assert norm_step_grad(mg, **wrong) == mg.ERR_INVALID_ARG


def test_empty_problems(mg):
    assert quantize(mg, M=0, ldrs=0) == mg.OK and quantize(mg, N=0) == mg.OK
    assert squares(mg, M=0) == mg.OK and dequantize(mg, N=0) == mg.OK
    assert product(mg, M=0, A=0, C=0) == mg.OK and product(mg, N=0) == mg.OK
    assert mg.mipgemm_last_path() & mg.PATH_MASK == mg.PATH_TRIVIAL
    assert norm_step(mg, M=0) == mg.OK and norm_step(mg, N=0) == mg.OK
    assert norm_step_grad(mg, M=0) == mg.OK and norm_step_grad(mg, N=0) == mg.OK


# ------------------------------------------------------------------------------------------------ the tests' own definitions
@pytest.mark.parametrize("fmt", f.FORMATS)
def test_nearest_agrees_with_the_casts(fmt):
    import torch
    rng = np.random.default_rng(5)
    v = np.concatenate([(rng.standard_normal(4000) * 2.0 ** rng.integers(-20, 14, 4000)), [0.0, 2.0 ** -9, 3 * 2.0 ** -10, 2.0 ** -10, 2.0 ** -17, 17, 18, 19, 440]])
    v = np.clip(v.astype(np.float32), -f.LARGEST[fmt], f.LARGEST[fmt])
    want = torch.from_numpy(v).to(f.f8_type(fmt)).double().numpy()
    assert np.array_equal(f.nearest(v, fmt), want)


def test_philox_known_answers():
    """The generator's published known answers for ten rounds (counter, key -> words)."""
    low = 0xFFFFFFFF
    assert f.philox([0, 0, 0, 0], [0, 0]) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert f.philox([low] * 4, [low] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert f.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_step_gradient_formulas_against_differences():
    rng = np.random.default_rng(6)
    m, n, e = 6, 10, 1e-6
    for post, pre in (("layer", "rms"), ("rms", "layer"), ("none", "layer"), ("rms", "none")):
        c = dict(x=rng.standard_normal((m, n)), z=rng.standard_normal((m, n)), post=post, pre=pre, eps=1e-3, x_scale=0.7, gate_rows=4,
                 gate=rng.standard_normal((2, n)), mask=f.kept(m, n, 0.3, 77, 5), post_w=rng.standard_normal(n) if post != "none" else None,
                 post_b=rng.standard_normal(n) if post == "layer" else None, pre_w=rng.standard_normal(n) if pre != "none" else None,
                 pre_b=rng.standard_normal(n) if pre == "layer" else None)
        dy, dh = rng.standard_normal((m, n)), rng.standard_normal((m, n)) if pre != "none" else None
        y, h, stats = f.step(c)
        got = f.step_grad(c, y, stats, dy, dh)

        def loss(c):
            y, h, _ = f.step(c)
            return (dy * y).sum() + (0 if dh is None else (dh * h).sum())
        for name, grad in (("x", "dx"), ("z", "dz"), ("gate", "dgate"), ("post_w", "dpost_w"), ("post_b", "dpost_b"), ("pre_w", "dpre_w"), ("pre_b", "dpre_b")):
            if c[name] is None:
                continue
            for at in [tuple(rng.integers(0, s) for s in c[name].shape) for _ in range(4)]:
                up, down = c[name].copy(), c[name].copy()
                up[at] += e
                down[at] -= e
                d = (loss(dict(c, **{name: up})) - loss(dict(c, **{name: down}))) / (2 * e)
                assert abs(d - got[grad][at]) < 1e-6 * (1 + abs(d)), (post, pre, name)


def test_the_pair_kernel_allocates_behind_its_cluster_barrier():
    """Read from the source, as for the other pair kernels: the allocation follows the barrier that shows both CTAs running."""
    import os
    import re
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_11728_b200", "csrc", "float8_product_kernel.cu")
    text = re.sub(r"//[^\n]*", "", open(path).read())
    found = re.findall(r"if \(kPair\) \{\s*__syncwarp\(\);\s*cluster_arrive\(\);\s*cluster_wait\(\);\s*\}\s*if \(warp == 1\) \{\s*tmem_alloc<kCtas>", text)
    assert len(found) == 1 and len(re.findall(r"tmem_alloc<", text)) == 1

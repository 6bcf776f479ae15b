"""CPU-only: what the step's backward pass refuses before it touches a device, beyond its first tests."""
import pytest

P = 4096     # an aligned non-NULL address; never dereferenced on these paths
ROOM = dict(dY=P, lddy=64, dH=P, lddh=64, Y=P, ldy=64, Z=P, ldz=64, stats=P, dX=2 * P, lddx=64, dZ=3 * P, lddz=64)


@pytest.fixture(scope="module")
def mg():
    from paper_2506_11728_b200 import build
    build.build_library()
    from paper_2506_11728_b200 import binding
    return binding


@pytest.mark.parametrize("post,pre", [(1, 1), (0, 1), (0, 0)])
@pytest.mark.parametrize("shared", [P, 2 * P])
def test_both_gradients_in_one_matrix(mg, post, pre, shared):
    """In a matrix of their own, or in that of an input: one of them would be lost."""
    room = dict(ROOM, dX=shared, dZ=shared)
    if not pre:
        room.update(dH=None)
    for M in (20, 0):
        assert mg.mipgemm_norm_step_grad(0, post, pre, M, 64, **room, stream=0, check=False) == mg.ERR_INVALID_ARG

"""Buffers that a call of the linear attention layer's operators may not use twice: refused before anything is enqueued, no GPU is needed."""
import ctypes

import pytest

FAKE = 0x1000            # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    from paper_2606_08804_b200 import binding, build
    build.build()
    return binding.load()


@pytest.mark.parametrize("T,dk,dv,dtype", [(1, 128, 128, 0), (64, 128, 64, 1), (4000, 64, 64, 0), (4000, 128, 128, 1)])
def test_a_gradient_of_the_state_where_the_state_is(lib, T, dk, dv, dtype):
    """Walks of one launch, in any order: one reads h0 and dhT, another writes dh0."""
    from paper_2606_08804_b200.binding import QdLinearShape
    shape = ctypes.byref(QdLinearShape(2, T, 13, dk, dv, dtype))
    for h0, dhT, dh0 in ((9, None, 9), (9, 10, 9), (None, 10, 10), (9, 10, 10)):
        at = [None if n is None else n * FAKE for n in (h0, dhT, dh0)]
        assert lib.qdelta_linear_bwd(shape, FAKE, 2 * FAKE, 3 * FAKE, FAKE, at[0], 4 * FAKE, at[1], 5 * FAKE, 6 * FAKE, 7 * FAKE, at[2], 1.0, 8 * FAKE,
                                     1 << 40, 0, None) == 1, (h0, dhT, dh0)

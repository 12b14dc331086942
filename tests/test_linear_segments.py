"""Into how many segments a linear attention call cuts its sequences, seen from the workspace that it asks for: no GPU is needed."""
import ctypes

import pytest

SMS, STATUS = 148, 256


@pytest.fixture(scope="module")
def lib():
    from paper_2606_08804_b200 import binding, build
    build.build()
    return binding.load()


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("B,T,H,dk,dv,dtype", [(1, 32768, 16, 128, 128, 1), (1, 32768, 16, 64, 128, 1), (1, 32768, 4, 128, 64, 1), (2, 16384, 5, 64, 64, 1),
                                               (1, 16384, 2, 64, 128, 0), (1, 32768, 1, 128, 128, 0), (1, 8192, 3, 128, 64, 0), (3, 20000, 2, 64, 64, 0)])
def test_no_sm_has_much_more_than_its_part(lib, B, T, H, dk, dv, dtype, backward):
    """The chunks that one SM after another takes, over all launches of a long call (segments' sums: half a walk's work), against the least of
    all cuts, with two chunks a walk for its start."""
    from paper_2606_08804_b200.binding import QdLinearShape
    bytes_ = lib.qdelta_linear_workspace_bytes(ctypes.byref(QdLinearShape(B, T, H, dk, dv, dtype)), backward)
    segments = max(1, (bytes_ - STATUS) // ((2 if backward else 1) * B * H * dk * dv * 4))
    chunks = -(-T // (128 if dtype else 64))
    ctas = lambda dc: B * H * (1 if dtype else dc // 32)  # noqa: E731
    launches = [ctas(dv)] if not backward else [3 * ctas(dv)] if dk == dv else [2 * ctas(dk), ctas(dv)]

    def longest(n):
        length = -(-chunks // n) + 2
        sums = -(-(2 if backward else 1) * ctas(dv) * (n - 1) // SMS) * length / 2
        return sum(-(-c * n // SMS) for c in launches) * length + sums
    cuts = [n for n in range(1, 33) if -(-chunks // -(-chunks // n)) == n]
    assert segments in cuts and longest(segments) <= 1.1 * min(map(longest, cuts)), (segments, longest(segments), min((longest(n), n) for n in cuts))

"""The 64-bit forms of the linear attention layer's operators: two forms of the same sums, and gradients against differences."""
import math

import pytest
import torch

import layer_forms as lf
import linear_forms as f

N = lambda *s, seed=0: torch.randn(*s, dtype=torch.float64, generator=torch.Generator().manual_seed(seed + sum(s)))  # noqa: E731


@pytest.mark.parametrize("T,state", [(1, True), (2, False), (17, True)])
def test_attention_is_its_recurrence(T, state):
    q, k, v, g = N(2, T, 3, 5), N(2, T, 3, 5, seed=1), N(2, T, 3, 4), torch.tensor([-0.1, 0.0, -math.inf], dtype=torch.float64)
    h0 = N(2, 3, 5, 4) if state else None
    for a, b in zip(f.linear(q, k, v, g, h0, 0.7), f.linear_recurrence(q, k, v, g, h0, 0.7)):
        assert (a - b).abs().max() < 1e-12


def _differences(fn, ins, ups):
    leaves = [t.clone().requires_grad_() for t in ins]
    outs = fn(*leaves)
    g = lf.grads(outs, ups, leaves)
    way = [N(*t.shape, seed=50 + i) for i, t in enumerate(ins)]
    at = lambda e: sum(float((o * u).sum()) for o, u in zip(fn(*[t + e * w for t, w in zip(ins, way)]), ups))  # noqa: E731
    want = (at(1e-5) - at(-1e-5)) / 2e-5
    assert abs(sum(float((a * b).sum()) for a, b in zip(g, way)) - want) < 1e-6 * (1 + abs(want))


def test_gradients_against_differences():
    g = torch.tensor([-0.3, -0.01], dtype=torch.float64)
    _differences(lambda q, k, v, h: f.linear(q, k, v, g, h, 0.5), [N(1, 9, 2, 3), N(1, 9, 2, 3, seed=1), N(1, 9, 2, 4), N(1, 2, 3, 4)], [N(1, 9, 2, 4, seed=2), N(1, 2, 3, 4, seed=3)])
    for rms in (False, True):
        for silu in (False, True):
            _differences(lambda *a: (f.gated_norm(*a, rms=rms, silu=silu),), [N(5, 7), N(5, 7, seed=1), N(7), N(7, seed=1)], [N(5, 7, seed=2)])
        _differences(lambda *a: f.add_norm(*a, rms=rms), [N(5, 7), N(5, 7, seed=1), N(7), N(7, seed=1), N(7, seed=4)], [N(5, 7, seed=2), N(5, 7, seed=3)])
    ang = f.angles([1 << 61, 12345678901234567], [0, 1, 5, 1 << 40])[None]
    for il in (False, True):
        _differences(lambda x: (f.rotary(x, ang, il, 0.8),), [N(1, 4, 2, 6)], [N(1, 4, 2, 6, seed=1)])


def test_turns_of_a_position():
    from paper_2606_08804_b200 import binding as qd
    whole = lambda t: [int(x) % (1 << 64) / 2.0 ** 64 * 2 * math.pi for x in t]  # noqa: E731
    for pairs, base in ((1, 10000.0), (32, 10000.0), (64, 5e5)):
        got = whole(qd.rotary_turns(pairs, base, device="cpu"))
        assert all(abs(a - base ** (-j / pairs)) <= 1e-15 * base ** (-j / pairs) + 2.0 ** -61 for j, a in enumerate(got))      # a unit is 2 pi 2^-64
        assert all(abs(a - b / 8) <= 1e-15 for a, b in zip(whole(qd.rotary_turns(pairs, base, 8.0, device="cpu")), got))
    plain, blend = whole(qd.rotary_turns(64, device="cpu")), whole(qd.rotary_turns(64, factor=4.0, original=4096, device="cpu"))
    n = [4096 * a / (2 * math.pi) for a in plain]
    for a, b, t in zip(plain, blend, n):
        kept = min(1.0, max(0.0, (t - 1) / 31))
        assert abs(b - a * (kept + (1 - kept) / 4)) <= 1e-15 + 1e-15 * a
    assert blend[0] == plain[0] and abs(blend[-1] - plain[-1] / 4) < 1e-15
    for bad in (dict(pairs=0), dict(pairs=2, base=0.0), dict(pairs=2, factor=0.0), dict(pairs=2, original=0), dict(pairs=2, original=8, low=2.0, high=2.0)):
        with pytest.raises(qd.QdeltaError):
            qd.rotary_turns(**bad, device="cpu")

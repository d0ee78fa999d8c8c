"""What pins the oracle of hybrid linear attention: closed forms, differences, and invariants of the definition (CPU)."""
import numpy as np
import pytest

from hla_testlib import Sample
from oracle import hla_oracle as O


def sample(full=True, **kw):
    return Sample([3, 0, 5], [2, 1, 0], 4, 2, 8, full, **kw)


def weighted_sum(s, out, last, dout, dlast):
    there = ~np.isnan(out)
    return (out[there] * dout[there]).sum() + (last * dlast).sum()


@pytest.mark.parametrize("full", (True, False))
@pytest.mark.parametrize("state", (True, False))
def test_backward_against_differences(full, state):
    s = sample(full, state=state, seed=3)
    rng = np.random.RandomState(1)
    dlast = rng.randn(3, 4, 8, 8)
    args = dict(q=s.q, k=s.k, v=s.v, state=s.state if state else np.zeros((3, 4, 8, 8)))

    def loss(q, k, v, state):
        out, last = O.forward(q, k, v, s.log_decay, *s.ints(), s.scale, full, state=state)
        return weighted_sum(s, out, last, s.dout, dlast)

    dq, dk, dv, dstate = O.backward(s.dout, s.q, s.k, s.v, s.log_decay, *s.ints(), s.scale, full, state=s.state, dlast=dlast)
    for name, grad in (("q", dq), ("k", dk), ("v", dv), ("state", dstate)):
        for _ in range(12):
            at = tuple(rng.randint(n) for n in grad.shape)
            up, down = dict(args), dict(args)
            up[name], down[name] = args[name].astype(np.float64).copy(), args[name].astype(np.float64).copy()
            up[name][at] += 0.5
            down[name][at] -= 0.5   # (the loss is linear in each argument alone: differences are exact)
            assert abs(loss(**up) - loss(**down) - grad[at]) < 1e-9, (name, at)


def test_no_decay_is_a_sum_over_all_pairs():
    s = sample(log_decay=[0.0] * 4)
    out, last = O.forward(s.q, s.k, s.v, s.log_decay, *s.ints(), s.scale, True)
    k, v, q = s.k[:3, 1], s.v[:3, 1], s.q[:3, 3]
    assert np.allclose(out[2, 3], s.scale * (q[2] @ k.T) @ v)
    assert np.allclose(last[0, 3], k.T @ v)


@pytest.mark.parametrize("log_decay", (-np.inf, -1e30))
def test_decay_to_nothing_leaves_the_own_key(log_decay):
    s = sample(log_decay=[log_decay] * 4, state=True)
    out, last = O.forward(s.q, s.k, s.v, s.log_decay, *s.ints(), s.scale, True, state=s.state)
    for row in range(5):
        assert np.allclose(out[row, 2], s.scale * (s.q[row, 2] @ s.k[row, 1]) * s.v[row, 1])
    assert np.allclose(last[1], s.state[1])   # no history: the state as it was


def test_above_zero_and_nan_are_no_decay():
    s = sample()
    a, b = (O.forward(s.q, s.k, s.v, g, *s.ints(), s.scale, True)[0] for g in ([0.0] * 4, [0.5, np.nan, np.inf, 0.0]))
    assert np.array_equal(a, b)


def test_pieces_follow_from_each_other():
    s = Sample([9], [2], 2, 1, 8, True, state=True)
    out, last = O.forward(s.q, s.k, s.v, s.log_decay, *s.ints(), s.scale, True, state=s.state)
    cut = 4
    a, mid = O.forward(s.q[:cut], s.k[:cut], s.v[:cut], s.log_decay, [0, cut], [0, cut], [cut], [0], s.scale, True, state=s.state)
    b, end = O.forward(s.q[cut:], s.k[cut:], s.v[cut:], s.log_decay, [0, 7], [0, 7], [5], [2], s.scale, True, state=mid)
    assert np.allclose(np.concatenate((a, b)), out) and np.allclose(end, last)


def test_candidates_do_not_see_each_other():
    s = sample()
    out, last = O.forward(s.q, s.k, s.v, s.log_decay, *s.ints(), s.scale, True)
    k, v = s.k.copy(), s.v.copy()
    k[4], v[4] = 7.0, -3.0   # the second candidate of the first user
    other, last2 = O.forward(s.q, k, v, s.log_decay, *s.ints(), s.scale, True)
    same = np.arange(len(out)) != 4
    assert np.array_equal(out[same], other[same]) and np.array_equal(last, last2) and not np.allclose(out[4], other[4])

"""Hybrid linear attention on the GPU against its float64 oracle: forward, backward, states, at the lengths and heads where it can go wrong."""
import numpy as np
import pytest
import torch

from hla_testlib import Sample, check, host, run
from hta_testlib import say
from oracle import hla_oracle as O
from paper_2602_11235_amd import hla, hta

pytestmark = pytest.mark.gpu

HEADS = ((4, 2, 32), (4, 4, 64), (8, 2, 64), (6, 2, 64), (16, 2, 128), (3, 1, 128), (1, 1, 32), (8, 1, 32))
LENGTHS = (([0, 1, 63, 64], [0, 3, 1, 0]), ([65, 127, 128, 129], [64, 0, 65, 2]), ([200, 0], [1, 130]))


@pytest.mark.parametrize("full", (True, False))
@pytest.mark.parametrize("lengths", range(len(LENGTHS)))
@pytest.mark.parametrize("heads", HEADS)
def test_forward_and_backward(heads, lengths, full):
    say(f"  hla {heads} {LENGTHS[lengths]} full={full}")
    s = Sample(*LENGTHS[lengths], *heads, full, seed=lengths, state=(lengths + full) % 2 == 0)
    check(run(s), s)


def test_many_users_of_unlike_lengths():
    rng = np.random.RandomState(0)
    s = Sample(rng.randint(0, 150, 70), rng.randint(0, 40, 70), 4, 1, 32, True, seed=5, state=True)
    check(run(s), s)


@pytest.mark.parametrize("full", (True, False))
def test_a_long_history(full):
    s = Sample([2000], [5], 2, 1, 64, full, seed=6, state=True)
    check(run(s), s)


@pytest.mark.parametrize("log_decay", ([0.0, 0.5, float("nan"), -1e-4], [-np.inf, -1e30, -80.0, -3.0]))
def test_decays_at_the_ends_of_their_range(log_decay):
    s = Sample([150, 3], [4, 70], 4, 2, 64, True, seed=7, state=True, log_decay=log_decay)
    check(run(s), s)


@pytest.mark.parametrize("scale", (1e-3, 1.0, 300.0))
def test_scales(scale):
    s = Sample([100], [10], 4, 2, 32, True, seed=8, state=True, scale=scale)
    check(run(s), s)


def test_without_states_the_states_are_zero():
    s = Sample([130, 7], [3, 1], 4, 2, 64, True, seed=9)
    none = run(s)
    z = Sample([130, 7], [3, 1], 4, 2, 64, True, seed=9)
    z.state, z.dlast = np.zeros((2, 4, 64, 64), np.float32), np.zeros((2, 4, 64, 64), np.float32)
    zero = run(z)
    for name in ("out", "last", "dq"):
        assert torch.equal(none[name], zero[name])
    # backwards the state is kept to 24 bits where it is returned, to 16 otherwise (2^-16 of its size, what check() allows for a state): the gradients
    # are formed from its value in bf16, which may be the next one
    assert none["dstate"] is None
    check(none, s)
    check(zero, z)


def test_rows_of_no_user_and_other_buffers_stay():
    s = Sample([70, 64], [3, 0], 4, 2, 64, True, seed=10, state=True, pad=5)
    b = s.batch()
    b.prepare_backward()
    for t in (b.out, b.dq, b.dk, b.dv):
        t.fill_(7.0)
    got = run(s, b)
    for name, n in (("out", s.n_q), ("dq", s.n_q), ("dk", s.n_kv), ("dv", s.n_kv)):
        assert (got[name][n:] == 7.0).all(), name
    check({k: (v[: s.n_q] if k in ("out", "dq") else v[: s.n_kv] if k in ("dk", "dv") else v) for k, v in got.items()}, _cut(s))


def _cut(s):
    for name in ("q", "dout"):
        setattr(s, name, getattr(s, name)[: s.n_q])
    for name in ("k", "v"):
        setattr(s, name, getattr(s, name)[: s.n_kv])
    return s


def test_tokens_behind_a_users_own_are_not_touched():
    """hist_len + n_targets may be less than the offsets' rows; the rest belongs to nobody."""
    s = Sample([70, 20], [3, 9], 4, 2, 32, True, seed=11)
    b = s.batch(want_state=False)
    b.ints[3].copy_(torch.tensor([1, 9], dtype=torch.int32))
    b.out.fill_(5.0)
    out, _ = b.forward()
    assert (out[71:73] == 5.0).all()
    want, _ = O.forward(s.q, s.k, s.v, s.log_decay, *s.ints(), s.scale, True)
    keep = np.r_[0:71, 73:102]
    assert np.linalg.norm(host(out)[keep] - want[keep]) <= 2.0 ** -8 * np.linalg.norm(want[keep])


@pytest.mark.parametrize("value", (float("nan"), float("inf")))
def test_what_a_row_may_not_see_does_not_reach_it(value):
    """A value that is not finite in one token's v (or k, q, dout) reaches the rows that see it and no other."""
    for name in ("v", "k"):
        s = Sample([150, 80], [3, 2], 4, 2, 64, True, seed=12)
        at = 100
        getattr(s, name)[at, 1, 5] = value
        with np.errstate(invalid="ignore"):
            want, _ = O.forward(s.q, s.k, s.v, s.log_decay, *s.ints(), s.scale, True)
        out = host(s.batch().forward()[0])
        assert (np.isfinite(out) == np.isfinite(want)).all(), name
        clean = np.isfinite(want).all((1, 2))
        assert clean[:at].all() and clean[153:].all()
        assert np.linalg.norm(out[clean] - want[clean]) <= 2.0 ** -8 * np.linalg.norm(want[clean]), name
    s = Sample([150, 80], [3, 2], 4, 2, 64, True, seed=12)
    s.v[151, 0, 3] = value  # a candidate
    out = host(s.batch().forward()[0])
    bad = ~np.isfinite(out)
    assert bad[151, :2, 3].all() and bad.sum() == 2
    s = Sample([150, 80], [3, 2], 4, 2, 64, True, seed=12)
    s.dout[40, 3, 7] = value  # backwards it reaches the tokens in front of it and its own dq
    got = run(s)
    dk, dv, dq = host(got["dk"]), host(got["dv"]), host(got["dq"])
    assert np.isfinite(dv[41:]).all() and np.isfinite(dk[41:]).all() and not np.isfinite(dv[:41, 1, 7]).any()
    assert np.isfinite(np.delete(dq, 40, 0)).all()
    assert np.isfinite(dv[:, 0]).all() and np.isfinite(dk[:, 0]).all()


def test_histories_in_pieces_with_states_in_place():
    s = Sample([190], [6], 4, 2, 64, True, seed=13, state=True)
    whole = run(s)
    g = s.gpu
    state = g["state"].clone()
    cut = 77
    one = lambda *x: [torch.tensor(v, dtype=torch.int32, device="cuda") for v in x]
    outs = []
    for a, b, L, T in ((0, cut, cut, 0), (cut, 196, 190 - cut, 6)):
        p = hla.DecayBatch(g["q"][a:b], g["k"][a:b], g["v"][a:b], g["log_decay"], *one([0, b - a], [0, b - a], [L], [T]), L, T, s.scale, hta.LAYER_FULL,
                           state=state, want_state=True)
        p.final_state = state
        outs.append(p.forward()[0])
    check(dict(whole, out=torch.cat(outs), last=state), s)


def test_results_are_the_same_bits_in_every_run():
    s = Sample([150, 300, 20], [30, 1, 0], 8, 2, 64, True, seed=14, state=True)
    first = {k: v.clone() for k, v in run(s).items()}
    for _ in range(3):
        again = run(s)
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_another_stream_and_two_calls_at_once():
    a, b = Sample([150], [30], 8, 2, 64, True, seed=15), Sample([99, 70], [3, 4], 4, 4, 32, False, seed=16)
    ba, bb = a.batch(), b.batch()
    ba.prepare_backward()
    bb.prepare_backward()
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    ra, rb = run(a, ba, streams[0]), run(b, bb, streams[1])
    torch.cuda.synchronize()
    check(ra, a)
    check(rb, b)


def test_a_captured_step_replays():
    s = Sample([150, 300, 0], [30, 1, 4], 16, 2, 128, True, seed=17, state=True)
    b = s.batch()
    run(s, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(s, b)
    for turn in range(3):
        s.gpu["q"].mul_(-1.5)  # (replays read what the inputs hold by then)
        eager = {k: v.clone() for k, v in run(s, b).items()}
        for t in got.values():
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], eager[k]) for k in got), turn


def test_no_tokens_and_no_queries():
    s = Sample([0, 0], [0, 0], 4, 2, 32, True, seed=18, state=True)
    got = run(s)
    assert torch.equal(got["last"], s.gpu["state"]) and torch.equal(got["dstate"], s.gpu["dlast"])
    s = Sample([70, 5], [0, 0], 4, 2, 32, False, seed=19, state=True)  # histories without candidates: states only
    check(run(s), s, ("last", "dk", "dv", "dstate"))

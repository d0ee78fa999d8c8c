"""Hybrid linear attention where calls are planned otherwise: long histories of few users in pieces, many users of unlike lengths in another order, groups of
heads that are spread over workgroups; and the order of calls that a process makes."""
import numpy as np
import pytest
import torch

from hla_testlib import FULL, TARGET, Sample, check, host, run
from hta_testlib import say
from paper_2602_11235_amd import hla, hta

pytestmark = pytest.mark.gpu


def workspace(s, is_bwd):
    top = lambda a: int(a.max(initial=0))
    return hla.mtfm_hla_workspace_bytes(FULL if s.full else TARGET, hta.BF16, is_bwd, len(s.hist), len(s.q), len(s.k), top(s.hist), top(s.tgt), s.Hq, s.Hkv, s.d)


@pytest.mark.parametrize("full", (True, False))
@pytest.mark.parametrize("heads", ((2, 1, 32), (4, 2, 64), (2, 2, 128), (6, 1, 32)))
def test_histories_in_pieces(heads, full):
    """A few users whose histories are cut, one that has none, one that fills a piece exactly; candidates in more than one piece."""
    say(f"  hla pieces {heads} full={full}")
    s = Sample([2100, 0, 256, 513], [3, 5, 300, 0], *heads, full, seed=1, state=True)
    assert workspace(s, False) > 0 and workspace(s, True) > 0
    check(run(s), s)


@pytest.mark.parametrize("full", (True, False))
def test_pieces_with_states_in_place(full):
    s = Sample([1500, 700], [10, 2], 4, 2, 64, full, seed=2, state=True)
    assert workspace(s, True) > 0
    b = s.batch()
    state = s.gpu["state"].clone()
    b.state = b.final_state = state
    out = b.forward()[0].clone()
    last = state.clone()
    b.state, b.final_state = s.gpu["state"], None
    b.prepare_backward()
    dlast = s.gpu["dlast"].clone()
    b.dstate = dlast
    dq, dk, dv, dstate = b.backward(s.gpu["dout"], dstate=dlast)
    assert dstate is dlast
    check(dict(out=out, last=last, dq=dq, dk=dk, dv=dv, dstate=dstate), s)


def test_pieces_without_states_and_captured():
    s = Sample([1300, 40], [70, 1], 4, 1, 64, True, seed=3)
    b = s.batch()
    check(run(s, b), s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(s, b)
    for turn in range(3):
        s.gpu["k"].mul_(-0.5)
        eager = {k: v.clone() for k, v in run(s, b).items() if v is not None}
        for t in eager:
            got[t].fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], eager[k]) for k in eager), turn


@pytest.mark.parametrize("full", (True, False))
def test_many_users_in_an_order_of_their_own(full):
    """More users' heads than places and lengths far apart: the users are taken by decreasing work.  Every user is as in a call of its own."""
    rng = np.random.RandomState(4)
    n = 300
    hist = rng.randint(0, 60, n)
    hist[[7, 150, 299]] = 290, 600, 444
    s = Sample(hist, rng.randint(0, 9, n), 4, 2, 32, full, seed=4, state=True)
    assert workspace(s, False) > 0
    got = run(s)
    for u in (0, 7, 42, 150, 299):
        one = Sample([s.hist[u]], [s.tgt[u]], 4, 2, 32, full, seed=0, state=True)
        q, kv = slice(s.q_off[u], s.q_off[u + 1]), slice(s.kv_off[u], s.kv_off[u + 1])
        one.q, one.dout, one.k, one.v = s.q[q], s.dout[q], s.k[kv], s.v[kv]
        one.state, one.dlast = s.state[u:u + 1], s.dlast[u:u + 1]
        part = {k: got[k][q] for k in ("out", "dq")} | {k: got[k][kv] for k in ("dk", "dv")} | {k: got[k][u:u + 1] for k in ("last", "dstate")}
        check(part, one, context=f"user {u}")
    assert all(np.isfinite(host(t)).all() for t in got.values())


@pytest.mark.parametrize("heads", ((16, 1, 64), (16, 1, 128), (12, 1, 32), (7, 1, 64), (8, 4, 128)))
@pytest.mark.parametrize("full", (True, False))
def test_groups_of_many_heads(heads, full):
    s = Sample([70, 33], [4, 66], *heads, full, seed=5, state=True)
    check(run(s), s)


def test_lengths_beyond_the_rows_and_the_bounds():
    """hist_len and n_targets that reach beyond a user's rows, or beyond the bounds that the call was given, are cut to what is there."""
    s = Sample([90, 50], [3, 7], 4, 2, 32, True, seed=6)
    b = s.batch(want_state=False)
    want = b.forward()[0].clone()
    b.ints[3][1] = 1000000   # (the last user: more candidates than rows)
    assert torch.equal(b.forward()[0], want)
    b.ints[2][1] = 70        # more history than rows, within the bound of 90: all 57 rows are history
    out = host(b.forward()[0])
    assert np.isfinite(out).all() and np.array_equal(out[:93], host(want)[:93])
    b.ints[2].fill_(-5)
    b.ints[3].fill_(-5)
    b.out.fill_(3.0)
    assert (b.forward()[0] == 3.0).all()


def test_two_batches_take_turns_on_one_stream():
    a, b = Sample([1200], [2], 4, 2, 64, True, seed=7, state=True), Sample([80, 900], [5, 1], 2, 1, 32, False, seed=8)
    ba, bb = a.batch(), b.batch()
    first = run(a, ba), run(b, bb)
    first = [{k: None if v is None else v.clone() for k, v in r.items()} for r in first]
    again = run(a, ba), run(b, bb)
    for x, y in zip(first, again):
        assert all(x[k] is None or torch.equal(x[k], y[k]) for k in x)
    check(again[0], a)
    check(again[1], b)


def test_a_batch_of_another_device_than_the_current_one_is_refused(monkeypatch):
    s = Sample([20], [2], 4, 2, 32, True, seed=1)
    b = s.batch()
    monkeypatch.setattr(hta, "_device_index", lambda: 1)   # (the refusal stands in front of any launch)
    b.out.fill_(3.0)
    with pytest.raises(ValueError, match="current GPU"):
        b.forward()
    with pytest.raises(ValueError, match="current GPU"):
        b.backward(s.gpu["dout"])
    assert (b.out == 3.0).all()


@pytest.mark.parametrize("value", (float("nan"), float("inf")))
@pytest.mark.parametrize("heads", ((4, 2, 32), (4, 4, 64), (4, 2, 64), (8, 2, 64), (4, 2, 128)))
def test_what_a_row_may_not_see_does_not_reach_it_for_any_heads(heads, value):
    """Chunks of either length, at either end of one: rows in front of a token (behind it, backwards) do not see that it is not finite."""
    r = heads[0] // heads[1]
    for at in (31, 32, 64, 95, 130):
        s = Sample([150, 80], [3, 2], *heads, True, seed=at)
        s.v[at, 1, 5] = value
        out = host(s.batch().forward()[0])
        assert np.isfinite(out[:at]).all() and np.isfinite(out[:, :r]).all() and np.isfinite(out[153:]).all()
        assert not np.isfinite(out[at:150, r:2 * r, 5]).all(0).any()
        s = Sample([150, 80], [3, 2], *heads, True, seed=at)
        s.dout[at, r, 7] = value
        got = run(s)
        for name in ("dk", "dv"):
            g = host(got[name])
            assert np.isfinite(g[at + 1:]).all() and np.isfinite(np.delete(g, 1, 1)).all(), name
        assert not np.isfinite(host(got["dv"])[:at + 1, 1, 7]).all()
        assert np.isfinite(np.delete(host(got["dq"]), at, 0)).all()

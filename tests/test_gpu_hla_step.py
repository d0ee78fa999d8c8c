"""Single tokens of hybrid linear attention on the GPU: the pool of states, slots, padding, and what a history's forward pass gives."""
import numpy as np
import pytest
import torch

from hla_testlib import U, Sample, host
from hta_testlib import say
from paper_2602_11235_amd import hla

pytestmark = pytest.mark.gpu

HEADS = ((4, 2, 32), (8, 2, 64), (4, 4, 64), (16, 2, 128), (3, 1, 128))


def tokens(n, heads, n_slots, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    Hq, Hkv, d = heads
    rand = lambda *shape: torch.randn(shape, device="cuda", generator=gen)
    q, k, v = (rand(n, h, d).to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    decay = -torch.rand(Hq, device="cuda", generator=gen)
    return q, k, v, rand(n_slots, Hq, d, d), decay


def oracle(q, k, v, pool, slots, decay, scale):
    """Row by row in float64: (out, pool, sums of magnitudes of out and pool)."""
    r = q.shape[1] // k.shape[1]
    q, k, v = host(q), np.repeat(host(k), r, 1), np.repeat(host(v), r, 1)
    S, l = host(pool), np.exp(host(decay))[:, None, None]
    out, size, mags = np.zeros(q.shape), np.zeros(q.shape), np.abs(S)
    for i, s in enumerate(slots):
        if 0 <= s < len(S):
            S[s] = l * S[s] + k[i][:, :, None] * v[i][:, None, :]
            mags[s] = l * mags[s] + np.abs(k[i][:, :, None] * v[i][:, None, :])
            out[i] = scale * np.einsum("hi,hij->hj", q[i], S[s])
            size[i] = scale * np.einsum("hi,hij->hj", np.abs(q[i]), mags[s])
    return out, S, size, mags


def check(out, pool, want, d):
    w_out, w_pool, size, mags = want
    # float32: two roundings per product, d sums; the exponential and its argument within 2^-21
    assert (np.abs(host(pool) - w_pool) <= 2.0 ** -20 * mags).all()
    assert (np.abs(host(out) - w_out) <= U * np.abs(w_out) + (2.0 ** -20 + d * 2.0 ** -24) * size).all()


@pytest.mark.parametrize("n", (1, 2, 7, 65))
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("in_place", (True, False))
def test_step(heads, n, in_place):
    say(f"  hla step {heads} n={n} in_place={in_place}")
    q, k, v, pool, decay = tokens(n, heads, n + 3, n)
    slots = torch.randperm(n + 3, device="cuda")[:n].to(torch.int32)
    want = oracle(q, k, v, pool, slots.tolist(), decay, 0.3)
    new = pool.clone() if in_place else torch.full_like(pool, 7.0)
    before = pool.clone()
    out = hla.mtfm_hla_step(q, k, v, new if in_place else pool, slots, decay, 0.3, new_state=None if in_place else new)
    named = torch.zeros(n + 3, dtype=torch.bool, device="cuda").index_fill_(0, slots.long(), True)
    assert torch.equal(new[~named], before[~named] if in_place else torch.full_like(before[~named], 7.0))
    if not in_place:
        assert torch.equal(pool, before)
        new[~named] = before[~named]
    check(out, new, want, heads[2])


def test_without_slots_row_i_is_state_i():
    q, k, v, pool, decay = tokens(5, (4, 2, 32), 8)
    want = oracle(q, k, v, pool, range(5), decay, 0.2)
    check(hla.mtfm_hla_step(q, k, v, pool, None, decay, 0.2), pool, want, 32)


@pytest.mark.parametrize("in_place", (True, False))
def test_rows_of_one_slot_are_tokens_in_order(in_place):
    n = 600  # (more than a workgroup looks at in one go)
    q, k, v, pool, decay = tokens(n, (2, 1, 32), 5, 3)
    slots = [(i * 7) % 4 if i % 100 < 3 else 4 if i % 50 == 4 else -1 for i in range(n)]
    want = oracle(q, k, v, pool, slots, decay, 0.2)
    new = pool if in_place else pool.clone()
    out = hla.mtfm_hla_step(q, k, v, pool, torch.tensor(slots, dtype=torch.int32, device="cuda"), decay, 0.2, new_state=None if in_place else new)
    w_out, w_pool, size, mags = want
    many = 24  # tokens of a slot at most: roundings add up
    assert (np.abs(host(new) - w_pool) <= many * 2.0 ** -20 * mags).all()
    assert (np.abs(host(out) - w_out) <= U * np.abs(w_out) + many * 2.0 ** -20 * size).all()


def test_padding_gives_zero_and_touches_nothing():
    q, k, v, pool, decay = tokens(4, (4, 2, 64), 3)
    before = pool.clone()
    out = torch.full_like(q, 9.0)
    hla.mtfm_hla_step(q, k, v, pool, torch.tensor([-1, 3, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda"), decay, 0.2, out=out)
    assert (out == 0).all() and torch.equal(pool, before)


def test_steps_continue_a_history():
    """A history's forward pass, then single tokens: what one pass over all of them gives."""
    L, more = 70, 5
    s = Sample([L + more, 30 + more], [0, 0], 8, 2, 64, True, seed=2, state=True)
    whole, _ = s.batch().forward()
    g = s.gpu
    first = Sample([L, 30], [0, 0], 8, 2, 64, True, seed=2)
    rows = np.r_[0:L, L + more:L + more + 30]
    for n in ("q", "k", "v"):
        setattr(first, n, getattr(s, n)[rows])
    first.state, first.dlast = s.state, s.dlast
    b = first.batch()
    pool = b.forward()[1]
    for i in range(more):
        at = torch.tensor([L + i, L + more + 30 + i], device="cuda")
        out = hla.mtfm_hla_step(g["q"][at], g["k"][at], g["v"][at], pool, None, g["log_decay"], s.scale)
        a, w = host(out), host(whole[at])
        # both are within three roundings (together U of the norm, see check()) of the same values, the step's one of them
        assert np.linalg.norm(a - w) <= 2 * U * np.linalg.norm(w)
    want, size = s.oracle()["last"], s.oracle(sizes=True)["last"]
    assert (np.abs(host(pool) - want) <= (2.0 ** -15 + 200 * 2.0 ** -24) * size).all()


def test_a_captured_step_replays():
    q, k, v, pool, decay = tokens(9, (8, 2, 64), 9)
    slots = torch.randperm(9, device="cuda").to(torch.int32)
    new, out = torch.empty_like(pool), torch.empty_like(q)
    step = lambda: hla.mtfm_hla_step(q, k, v, pool, slots, decay, 0.2, new_state=new, out=out)
    step()
    eager = out.clone(), new.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        out.fill_(float("nan"))
        new.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(new, eager[1])
        step()

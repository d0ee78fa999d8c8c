"""Rows, states and shares whose elements lie past 2^31: every offset is held in 64 bits."""
import numpy as np
import pytest
import torch

import test_gpu_hla_step as steps
import test_gpu_rms as norms
from hla_testlib import Sample, check, run
from hta_testlib import say
from paper_2602_11235_amd import hla, rms

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads, full", (((2, 2, 128), True), ((8, 1, 128), False), ((4, 4, 32), True)))
def test_tokens(heads, full):
    """The users' rows stand behind 2^31 elements that belong to nobody (eight heads of 128 to one: in front of them shares of their gradients too)."""
    Hq, Hkv, d = heads
    say(f"  hla far {heads} full={full}")
    s = Sample([70, 0, 33], [4, 3, 0], *heads, full, seed=9, state=True)
    far = 2 ** 31 // (Hkv * d) + 11
    s.kv_off = s.kv_off + np.int32(far)
    if full:
        s.q_off = s.kv_off
    g = s.on_gpu()
    for n in ("k", "v") + (("q", "dout") if full else ()):
        t = torch.empty((far + g[n].shape[0], *g[n].shape[1:]), dtype=torch.bfloat16, device="cuda")
        t[far:] = g[n]
        g[n] = t
    b = hla.DecayBatch(g["q"], g["k"], g["v"], g["log_decay"], *g["ints"], 70, 4, s.scale, 0 if full else 1, state=g["state"], want_state=True)
    got = run(s, b)
    got = {n: t[far:] if n in ("dk", "dv") or (full and n in ("out", "dq")) else t for n, t in got.items()}
    s.kv_off = s.kv_off - np.int32(far)
    if full:
        s.q_off = s.kv_off
    check(got, s)


@pytest.mark.parametrize("in_place", (True, False))
def test_slots(in_place):
    heads, n_slots = (16, 2, 128), 2 ** 31 // (16 * 128 * 128) + 4
    say(f"  hla step far in_place={in_place}")
    q, k, v, near, decay = steps.tokens(3, heads, 3, 5)
    slots = [n_slots - 1, n_slots - 3, n_slots - 2]
    want = steps.oracle(q, k, v, near, [2, 0, 1], decay, 0.3)
    pool = torch.empty((n_slots, 16, 128, 128), device="cuda")
    pool[-3:] = near
    new = pool if in_place else torch.empty_like(pool)
    out = hla.mtfm_hla_step(q, k, v, pool, torch.tensor(slots, dtype=torch.int32, device="cuda"), decay, 0.3, new_state=new)
    steps.check(out, new[-3:], want, 128)


def test_normalized_rows():
    d, n = 1024, 2 ** 21 + 9
    say("  rms far")
    x, r, dy = (torch.zeros((n, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    x[-9:], r[-9:], dy[-9:] = norms.rows(9, d, torch.bfloat16), norms.rows(9, d, torch.bfloat16, 2), norms.rows(9, d, torch.bfloat16, 3)
    w = norms.weights(d)
    y, h, rstd = rms.mtfm_rms_fwd(x, w, norms.EPS, residual=r)
    norms.check_forward(x[-9:], r[-9:], w, y[-9:], h[-9:], rstd[-9:])
    dx, dw = rms.mtfm_rms_bwd(dy, h, w, rstd, dh=r)
    norms.check_backward(dy[-9:], h[-9:], w, r[-9:], dx[-9:], dw)   # (all other rows add nothing)

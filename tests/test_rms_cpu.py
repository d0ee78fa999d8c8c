"""The root-mean-square normalization without a GPU: pins of its oracle, exported symbols, refusals in front of any launch."""
import os
import re

import numpy as np
import pytest
import torch

from oracle import rms_oracle as R
from paper_2602_11235_amd import hta, rms

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000


def test_oracle_backward_against_differences():
    rng = np.random.RandomState(0)
    h, dy, dh, w = rng.randn(3, 7), rng.randn(3, 7), rng.randn(3, 7), rng.randn(7)
    loss = lambda h, w: (R.forward(h, w, 1e-3)[0] * dy).sum() + (h * dh).sum()
    dx, dw, _, _ = R.backward(dy, h, w, 1e-3, dh)
    e = 1e-5
    for i in range(3):
        for c in range(7):
            up, down = h.copy(), h.copy()
            up[i, c] += e
            down[i, c] -= e
            assert abs((loss(up, w) - loss(down, w)) / (2 * e) - dx[i, c]) < 1e-8
    for c in range(7):
        up, down = w.copy(), w.copy()
        up[c] += e
        down[c] -= e
        assert abs((loss(h, up) - loss(h, down)) / (2 * e) - dw[c]) < 1e-8


def test_oracle_against_torch():
    h, w = torch.randn(5, 33, dtype=torch.float64), torch.randn(33, dtype=torch.float64)
    want = torch.nn.functional.rms_norm(h, (33,), w, 1e-5)
    assert np.allclose(R.forward(h.numpy(), w.numpy(), 1e-5)[0], want.numpy())


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "mtfm_rms.h")).read()
    names = sorted(set(re.findall(r"MTFM_HTA_API[^;(]*?\b(mtfm_rms_\w+)\s*\(", text)))
    assert set(names) == set(rms.EXPORTS)
    lib = rms.load_library()
    for n in names:
        assert getattr(lib, n) is not None


def forward(q8=False, **kw):
    a = dict(x=FAKE, ldx=512, r=None, ldr=0, w=FAKE, h=None, y=FAKE, s=FAKE, n=10, d=512, eps=1e-5, dtype=hta.BF16, kind=0)
    a.update(kw)
    lib = rms.load_library()
    head = (a["x"], a["ldx"], a["r"], a["ldr"], a["w"], a["h"], a["y"], a["s"], a["n"], a["d"], a["eps"], a["dtype"])
    return lib.mtfm_rms_fwd_q8(*head, a["kind"], None) if q8 else lib.mtfm_rms_fwd(*head, None)


@pytest.mark.parametrize("q8", (False, True))
@pytest.mark.parametrize("kw, status", [
    (dict(d=0), hta.ERR_INVALID_ARG), (dict(d=8193, ldx=8193), hta.ERR_UNSUPPORTED), (dict(n=-1), hta.ERR_INVALID_ARG), (dict(dtype=3), hta.ERR_INVALID_ARG),
    (dict(eps=-1.0), hta.ERR_INVALID_ARG), (dict(eps=float("nan")), hta.ERR_INVALID_ARG), (dict(x=None), hta.ERR_INVALID_ARG),
    (dict(x=FAKE + 1), hta.ERR_INVALID_ARG), (dict(ldx=511), hta.ERR_INVALID_ARG), (dict(ldx=1 << 60), hta.ERR_INVALID_ARG), (dict(r=FAKE, ldr=512), hta.ERR_INVALID_ARG),
    (dict(h=FAKE), hta.ERR_INVALID_ARG), (dict(r=FAKE, h=FAKE, ldr=3), hta.ERR_INVALID_ARG), (dict(w=FAKE + 2), hta.ERR_INVALID_ARG), (dict(y=None), hta.ERR_INVALID_ARG)])
def test_forward_refuses(kw, status, q8):
    assert forward(q8, **kw) == status and hta.mtfm_hta_last_error()


def test_forward_in_8_bits_refuses():
    assert forward(True, kind=2) == hta.ERR_INVALID_ARG
    assert forward(True, s=None) == hta.ERR_INVALID_ARG


def backward(**kw):
    a = dict(dy=FAKE, h=FAKE, ld=512, w=FAKE, rstd=FAKE, dh=None, ldh=0, dx=FAKE, dw=FAKE, n=10, d=512, dtype=hta.BF16, ws=FAKE,
             ws_bytes=rms.mtfm_rms_bwd_workspace_bytes(512))
    a.update(kw)
    return rms.load_library().mtfm_rms_bwd(a["dy"], a["ld"], a["h"], 512, a["w"], a["rstd"], a["dh"], a["ldh"], a["dx"], a["dw"], a["n"], a["d"], a["dtype"],
                                           a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw, status", [
    (dict(d=0), hta.ERR_INVALID_ARG), (dict(n=-1), hta.ERR_INVALID_ARG), (dict(dy=None), hta.ERR_INVALID_ARG), (dict(dw=None), hta.ERR_INVALID_ARG),
    (dict(ld=100), hta.ERR_INVALID_ARG), (dict(dh=FAKE, ldh=4), hta.ERR_INVALID_ARG), (dict(h=FAKE + 1), hta.ERR_INVALID_ARG), (dict(ws=None), hta.ERR_WORKSPACE),
    (dict(ws_bytes=100), hta.ERR_WORKSPACE), (dict(ws=FAKE + 16), hta.ERR_WORKSPACE)])
def test_backward_refuses(kw, status):
    assert backward(**kw) == status and hta.mtfm_hta_last_error()


def test_empty_forward_and_workspace():
    assert forward(n=0, x=None, y=None, w=None) == hta.OK
    assert rms.mtfm_rms_bwd_workspace_bytes(512) == 512 * 512 * 4
    assert rms.mtfm_rms_bwd_workspace_bytes(7) == 512 * 8 * 4
    assert rms.mtfm_rms_bwd_workspace_bytes(0) == rms.mtfm_rms_bwd_workspace_bytes(8193) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    x, w = torch.zeros(4, 16), torch.zeros(16)
    bad = [lambda: rms.mtfm_rms_fwd(x[0], w, 1e-5), lambda: rms.mtfm_rms_fwd(x, w[:8], 1e-5), lambda: rms.mtfm_rms_fwd(x, w.double(), 1e-5),
           lambda: rms.mtfm_rms_fwd(x.t(), w[:4], 1e-5), lambda: rms.mtfm_rms_fwd(x, w, 1e-5, residual=x[:2]),
           lambda: rms.mtfm_rms_fwd(x, w, 1e-5, residual=x.bfloat16()), lambda: rms.mtfm_rms_fwd(x, w, 1e-5, h=x),
           lambda: rms.mtfm_rms_fwd(x, w, 1e-5, y=x[:, :8]), lambda: rms.mtfm_rms_fwd(x, w, 1e-5, rstd=w),
           lambda: rms.mtfm_rms_fwd_q8(x, w, 1e-5, q=torch.zeros(4, 16)), lambda: rms.mtfm_rms_fwd_q8(x, w, 1e-5, scale=w),
           lambda: rms.mtfm_rms_bwd(x[:2], x, w, torch.zeros(4)), lambda: rms.mtfm_rms_bwd(x, x, w, torch.zeros(3)),
           lambda: rms.mtfm_rms_bwd(x, x, w, torch.zeros(4), dh=x.bfloat16()), lambda: rms.mtfm_rms_bwd(x, x, w, torch.zeros(4), out=(x[:1], None))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: rms.mtfm_rms_fwd(x.double(), w, 1e-5), lambda: rms.mtfm_rms_fwd_q8(x, w, 1e-5, kind=torch.uint8)):
        with pytest.raises(TypeError):
            f()
    for f in (lambda: rms.mtfm_rms_fwd(x, w, 1e-5), lambda: rms.mtfm_rms_fwd_q8(x, w, 1e-5), lambda: rms.mtfm_rms_bwd(x, x, w, torch.zeros(4))):
        with pytest.raises(ValueError, match="current GPU"):
            f()

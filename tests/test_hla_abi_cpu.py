"""Host-side checks of hybrid linear attention that need no GPU: exported symbols, refusals in front of any launch."""
import os
import re

import pytest
import torch

from paper_2602_11235_amd import hla, hta

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000  # a 16-byte aligned non-null address: refused calls never dereference it


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "mtfm_hla.h")).read()
    names = sorted(set(re.findall(r"MTFM_HTA_API[^;(]*?\b(mtfm_hla_\w+)\s*\(", text)))
    assert set(names) == set(hla.EXPORTS)
    lib = hla.load_library()
    for n in names:
        assert getattr(lib, n) is not None


def call(back=False, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, decay=FAKE, state=None, out=FAKE, last=None, ints=FAKE, batch=2, total_q=10, total_kv=10, max_hist=4, max_targets=1,
             Hq=8, Hkv=2, d=64, scale=0.125, dtype=hta.BF16, layer=hta.LAYER_FULL, ws=None, ws_bytes=0)
    a.update(kw)
    lib = hla.load_library()
    tail = (*[a["ints"]] * 4, a["batch"], a["total_q"], a["total_kv"], a["max_hist"], a["max_targets"], a["Hq"], a["Hkv"], a["d"], a["scale"], a["dtype"],
            a["layer"], a["ws"], a["ws_bytes"], None)
    if back:
        return lib.mtfm_hla_bwd(FAKE, a["q"], a["k"], a["v"], a["decay"], a["state"], a["last"], a["out"], FAKE, FAKE, None, *tail)
    return lib.mtfm_hla_fwd(a["q"], a["k"], a["v"], a["decay"], a["state"], a["out"], a["last"], *tail)


BAD = [(dict(Hkv=3), hta.ERR_INVALID_ARG), (dict(Hq=0), hta.ERR_INVALID_ARG), (dict(d=0), hta.ERR_INVALID_ARG), (dict(d=48), hta.ERR_UNSUPPORTED),
       (dict(d=256), hta.ERR_UNSUPPORTED), (dict(dtype=hta.FP32), hta.ERR_UNSUPPORTED), (dict(dtype=7), hta.ERR_INVALID_ARG),
       (dict(layer=2), hta.ERR_INVALID_ARG), (dict(batch=-1), hta.ERR_INVALID_ARG), (dict(total_kv=-1), hta.ERR_INVALID_ARG),
       (dict(max_hist=-1), hta.ERR_INVALID_ARG), (dict(total_q=1 << 31), hta.ERR_UNSUPPORTED), (dict(batch=1 << 30), hta.ERR_UNSUPPORTED),
       (dict(scale=0.0), hta.ERR_INVALID_ARG), (dict(scale=float("nan")), hta.ERR_INVALID_ARG), (dict(scale=float("inf")), hta.ERR_INVALID_ARG),
       (dict(q=None), hta.ERR_INVALID_ARG), (dict(q=FAKE + 8), hta.ERR_INVALID_ARG), (dict(k=None), hta.ERR_INVALID_ARG),
       (dict(decay=None), hta.ERR_INVALID_ARG), (dict(decay=FAKE + 2), hta.ERR_INVALID_ARG), (dict(ints=None), hta.ERR_INVALID_ARG),
       (dict(ints=FAKE + 1), hta.ERR_INVALID_ARG), (dict(state=FAKE + 4), hta.ERR_INVALID_ARG), (dict(last=FAKE + 4), hta.ERR_INVALID_ARG)]


@pytest.mark.parametrize("back", (False, True))
@pytest.mark.parametrize("kw, status", BAD)
def test_bad_arguments_are_refused_without_launching(kw, status, back):
    assert call(back, **kw) == status and hta.mtfm_hta_last_error()


def test_empty_batch_is_ok_without_a_device():
    for back in (False, True):
        assert call(back, batch=0, q=None, k=None, v=None, out=None, decay=None, ints=None) == hta.OK


def test_workspace_is_asked_for():
    sizes = (hta.LAYER_FULL, hta.BF16, True, 2, 10, 10, 4, 1)
    need = hla.mtfm_hla_workspace_bytes(*sizes, 16, 1, 128)   # sixteen heads of a group do not fit a workgroup
    assert need > 0 and need % 256 == 0
    kw = dict(Hq=16, Hkv=1, d=128)
    assert call(True, **kw) == hta.ERR_WORKSPACE and str(need) in hta.mtfm_hta_last_error()
    assert call(True, ws=FAKE, ws_bytes=need - 1, **kw) == hta.ERR_WORKSPACE
    assert call(True, ws=FAKE + 16, ws_bytes=need, **kw) == hta.ERR_WORKSPACE
    with pytest.raises(hta.HtaError):
        hla.mtfm_hla_workspace_bytes(*sizes, 3, 2, 64)


def step(**kw):
    a = dict(q=FAKE, decay=FAKE, state=FAKE, new=FAKE, slots=FAKE, out=FAKE, rows=4, n_slots=8, Hq=8, Hkv=2, d=64, scale=0.125, dtype=hta.BF16)
    a.update(kw)
    return hla.load_library().mtfm_hla_step(a["q"], FAKE, FAKE, a["decay"], a["state"], a["new"], a["slots"], a["out"], a["rows"], a["n_slots"], a["Hq"],
                                            a["Hkv"], a["d"], a["scale"], a["dtype"], None)


@pytest.mark.parametrize("kw, status", [
    (dict(q=None), hta.ERR_INVALID_ARG), (dict(state=None), hta.ERR_INVALID_ARG), (dict(new=None), hta.ERR_INVALID_ARG), (dict(out=FAKE + 4), hta.ERR_INVALID_ARG),
    (dict(slots=FAKE + 2), hta.ERR_INVALID_ARG), (dict(rows=-1), hta.ERR_INVALID_ARG), (dict(n_slots=-1), hta.ERR_INVALID_ARG), (dict(Hkv=3), hta.ERR_INVALID_ARG),
    (dict(d=16), hta.ERR_UNSUPPORTED), (dict(dtype=hta.FP32), hta.ERR_UNSUPPORTED), (dict(scale=-1.0), hta.ERR_INVALID_ARG),
    (dict(slots=None, n_slots=3), hta.ERR_INVALID_ARG), (dict(rows=1 << 30), hta.ERR_UNSUPPORTED)])
def test_bad_step_arguments_are_refused(kw, status):
    assert step(**kw) == status and hta.mtfm_hta_last_error()


def test_empty_step_is_ok_without_a_device():
    assert step(rows=0, q=None, state=None, new=None, out=None, decay=None, slots=None) == hta.OK


def tensors(Hq=4, Hkv=2, d=32, n=6):
    bf = dict(dtype=torch.bfloat16)
    ints = [torch.tensor(x, dtype=torch.int32) for x in ([0, n], [0, n], [n], [0])]
    return torch.zeros(n, Hq, d, **bf), torch.zeros(n, Hkv, d, **bf), torch.zeros(n, Hkv, d, **bf), torch.zeros(Hq), ints


def test_binding_refuses_tensors_that_do_not_fit():
    q, k, v, decay, ints = tensors()
    make = lambda q=q, k=k, v=v, decay=decay, ints=ints, **kw: hla.DecayBatch(q, k, v, decay, *ints, 6, 0, 0.1, hta.LAYER_FULL, **kw)
    bad = [dict(q=q.float()), dict(k=k[:, :, :16]), dict(v=v[:3]), dict(k=k.transpose(0, 1)), dict(decay=decay[:2]), dict(decay=decay.double()),
           dict(ints=[i.long() for i in ints]), dict(ints=ints[:3] + [torch.zeros(2, dtype=torch.int32)]), dict(state=torch.zeros(1, 4, 32, 31)),
           dict(state=torch.zeros(1, 4, 32, 32, dtype=torch.bfloat16)), dict(q=q[:, 0])]
    for kw in bad:
        with pytest.raises(ValueError):
            make(**kw)
    with pytest.raises(ValueError, match="current GPU"):
        make()


def test_binding_refuses_steps_that_do_not_fit():
    q, k, v, decay, _ = tensors()
    state, slots = torch.zeros(8, 4, 32, 32), torch.zeros(6, dtype=torch.int32)
    make = lambda q=q, k=k, v=v, state=state, slots=slots, decay=decay, **kw: hla.mtfm_hla_step(q, k, v, state, slots, decay, 0.1, **kw)
    bad = [dict(k=k[:5], v=v[:5]), dict(state=state[:, :2]), dict(state=state[0]), dict(slots=slots.long()), dict(slots=slots[:2]), dict(new_state=state[:4]),
           dict(out=q.float()), dict(decay=decay[:1]), dict(q=q.float())]
    for kw in bad:
        with pytest.raises(ValueError):
            make(**kw)
    with pytest.raises(ValueError, match="current GPU"):
        make()


@pytest.mark.parametrize("back", (False, True))
@pytest.mark.parametrize("kw", [dict(batch=1 << 24, Hq=1, Hkv=1), dict(batch=1 << 20, Hq=16, Hkv=1), dict(batch=1 << 20, Hq=8, Hkv=8, d=128),
                                dict(total_kv=(1 << 30) + 1), dict(total_q=(1 << 30) + 1)])
def test_more_than_a_launch_takes_is_refused(kw, back):
    assert call(back, **kw) == hta.ERR_UNSUPPORTED


def test_more_steps_than_a_launch_takes_are_refused():
    assert step(rows=1 << 21, n_slots=1 << 21) == hta.ERR_UNSUPPORTED


@pytest.mark.parametrize("total", (10, 5000, 1 << 30))
@pytest.mark.parametrize("heads", ((4, 2, 64), (16, 1, 128), (1, 1, 32)))
def test_bounds_beyond_the_rows_ask_for_no_more_workspace(total, heads):
    for back in (False, True):
        need = [hla.mtfm_hla_workspace_bytes(layer, hta.BF16, back, 2, total, total, most, most, *heads)
                for layer in (hta.LAYER_FULL, hta.LAYER_TARGET) for most in (total, (1 << 31) - 1)]
        assert need[0] == need[1] and need[2] == need[3]
        assert max(need) <= 40 * total * heads[0] * heads[2] + (1 << 20)  # (shares of 8 bytes to an element, and states of pieces of a few hundred rows)

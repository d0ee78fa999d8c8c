"""Shared by the tests of hybrid linear attention: samples, calls and what two correct results may differ by."""
import numpy as np
import torch

from oracle import hla_oracle as O
from paper_2602_11235_amd import hla, hta

FULL, TARGET = hta.LAYER_FULL, hta.LAYER_TARGET
U = 2.0 ** -8  # half a step of bf16, relative


class Sample:
    """A jagged batch of bf16-representable values, as NumPy arrays in float64 (`pad`: rows behind the last user)."""

    def __init__(self, hist, tgt, Hq, Hkv, d, full, seed=0, state=False, pad=0, log_decay=None, scale=None):
        rng = np.random.RandomState(seed)
        bf = lambda *shape: torch.from_numpy(rng.randn(*shape)).to(torch.bfloat16).double().numpy()
        self.hist, self.tgt = np.array(hist, np.int32), np.array(tgt, np.int32)
        self.full, self.Hq, self.Hkv, self.d = full, Hq, Hkv, d
        off = lambda n: np.concatenate(([0], np.cumsum(n))).astype(np.int32)
        self.kv_off = off(self.hist + self.tgt)
        self.q_off = self.kv_off if full else off(self.tgt)
        self.n_q, self.n_kv = int(self.q_off[-1]), int(self.kv_off[-1])
        self.q, self.dout = bf(self.n_q + pad, Hq, d), bf(self.n_q + pad, Hq, d)
        self.k, self.v = bf(self.n_kv + pad, Hkv, d), bf(self.n_kv + pad, Hkv, d)
        # decays from "forgets at once" to "never"
        self.log_decay = (np.linspace(-2.0, 0.0, Hq) ** 3 if log_decay is None else np.array(log_decay)).astype(np.float32)
        self.scale = float(np.float32(d ** -0.5 if scale is None else scale))
        shape = (len(hist), Hq, d, d)
        self.state = rng.randn(*shape).astype(np.float32) if state else None
        self.dlast = rng.randn(*shape).astype(np.float32) if state else None

    def ints(self):
        return self.q_off, self.kv_off, self.hist, self.tgt

    def on_gpu(self):
        dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(t)
        self.gpu = {n: dev(getattr(self, n), torch.bfloat16) for n in ("q", "k", "v", "dout")}
        self.gpu |= {n: None if getattr(self, n) is None else dev(getattr(self, n), torch.float32) for n in ("state", "dlast", "log_decay")}
        self.gpu["ints"] = tuple(dev(a, torch.int32) for a in self.ints())
        return self.gpu

    def batch(self, want_state=True):
        g = self.on_gpu()
        top = lambda a: int(a.max()) if len(a) else 0
        return hla.DecayBatch(g["q"], g["k"], g["v"], g["log_decay"], *g["ints"], top(self.hist), top(self.tgt), self.scale,
                              FULL if self.full else TARGET, state=g["state"], want_state=want_state)

    def oracle(self, sizes=False):
        """The results in float64; with `sizes`, of the inputs' magnitudes (sums without cancellation)."""
        f = np.abs if sizes else (lambda a: a)
        s = lambda a: None if a is None else f(a)
        rest = (self.log_decay, *self.ints(), self.scale, self.full)
        out, last = O.forward(f(self.q), f(self.k), f(self.v), *rest, state=s(self.state))
        grads = O.backward(f(self.dout), f(self.q), f(self.k), f(self.v), *rest, state=s(self.state), dlast=s(self.dlast))
        return dict(zip(("out", "last", "dq", "dk", "dv", "dstate"), (out, last, *grads)))


def run(sample, batch=None, stream=None):
    b = batch or sample.batch()
    g = sample.gpu
    out, last = b.forward(stream=stream)
    dq, dk, dv, dstate = b.backward(g["dout"], dstate=g["dlast"], stream=stream)
    return dict(out=out, last=last, dq=dq, dk=dk, dv=dv, dstate=dstate)


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def check(got, sample, names=("out", "last", "dq", "dk", "dv", "dstate"), context=""):
    """Elementwise: a result row is a sum of terms each of which is rounded to bf16 once (a weight between two products, or a state),
    then rounded itself: U of itself and U of the sum of the magnitudes; float32 sums add less than a hundredth of that.  As a whole: the three
    roundings (weights, states, results) are independent and uniform, U / sqrt(3) of the norm each, together U.  (The norm counts where the
    values are many: 4096.)  States are float32 sums of terms kept to 2^-16."""
    want, size = sample.oracle(), sample.oracle(sizes=True)
    steps = int(sample.hist.max(initial=0)) + 64
    for name in names:
        if got[name] is None:
            continue
        x, y, m = host(got[name]), want[name], size[name]
        there = ~np.isnan(y)
        x, y, m = x[there], y[there], m[there]
        assert np.isfinite(x).all(), f"{context} {name}: not finite"
        if name in ("last", "dstate"):
            bound = (2.0 ** -15 + steps * 2.0 ** -24) * m
        else:
            bound = U * np.abs(y) + 1.01 * U * m
        off = np.abs(x - y)
        assert (off <= bound + 1e-30).all(), f"{context} {name}: {off.max():.3e} off, {np.max(off / (bound + 1e-30)):.2f} of the bound"
        if y.size >= 4096 and name not in ("last", "dstate"):
            rel = np.linalg.norm(x - y) / np.linalg.norm(y)
            assert rel <= U, f"{context} {name}: {rel:.2e} of the norm off"

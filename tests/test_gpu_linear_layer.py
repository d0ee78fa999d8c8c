"""The new operators as a layer uses them: normalization with the residual, projections (the caller's), linear attention, normalization per head --
trained in one call, and served from states in pieces and single tokens, with the same results."""
import numpy as np
import pytest
import torch

from paper_2602_11235_amd import hla, hta, rms

pytestmark = pytest.mark.gpu

Hq, Hkv, d, D = 4, 2, 64, 256
EPS = 1e-5


class Layer:
    def __init__(self, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, device="cuda", generator=gen)
        self.w_in, self.w_out = 1 + 0.1 * rand(D), 1 + 0.1 * rand(d)
        self.proj = (rand(D, (Hq + 2 * Hkv) * d) / D ** 0.5).bfloat16()
        self.log_decay = -torch.exp2(-torch.arange(1.0, Hq + 1, device="cuda"))

    def tokens(self, x, residual):
        y, h, rstd = rms.mtfm_rms_fwd(x, self.w_in, EPS, residual=residual)
        qkv = y @ self.proj
        q, k, v = (t.unflatten(1, (-1, d)).contiguous() for t in qkv.split((Hq * d, Hkv * d, Hkv * d), 1))
        return q, k, v, h, rstd

    def behind(self, out):
        return rms.mtfm_rms_fwd(out.reshape(-1, d), self.w_out, EPS)[0].view(len(out), Hq * d)


def inputs(n, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((n, D), device="cuda", generator=gen).bfloat16() for _ in range(2))


def ints(*lists):
    return [torch.tensor(x, dtype=torch.int32, device="cuda") for x in lists]


def batch(layer, q, k, v, L, T, state=None, kind=hta.LAYER_FULL):
    n = L + T
    nq = n if kind == hta.LAYER_FULL else T
    return hla.DecayBatch(q, k, v, layer.log_decay, *ints([0, nq], [0, n], [L], [T]), L, T, d ** -0.5, kind, state=state, want_state=True)


def test_serving_from_states_gives_what_one_pass_gives():
    layer = Layer()
    L, T, piece, singles = 150, 20, 90, 7
    x, r = inputs(L + T, 1)
    q, k, v, _, _ = layer.tokens(x, r)
    whole, last = batch(layer, q, k, v, L, T).forward()
    want = layer.behind(whole)
    got = []
    # a first piece, single tokens, the rest, then the candidates against the state that is there
    q1, k1, v1, _, _ = layer.tokens(x[:piece], r[:piece])
    out, pool = batch(layer, q1, k1, v1, piece, 0).forward()
    got.append(layer.behind(out))
    for i in range(piece, piece + singles):
        q1, k1, v1, _, _ = layer.tokens(x[i:i + 1], r[i:i + 1])
        got.append(layer.behind(hla.mtfm_hla_step(q1, k1, v1, pool, None, layer.log_decay, d ** -0.5)))
    a = piece + singles
    q1, k1, v1, _, _ = layer.tokens(x[a:L], r[a:L])
    out, pool = batch(layer, q1, k1, v1, L - a, 0, state=pool).forward()
    got.append(layer.behind(out))
    q1, k1, v1, _, _ = layer.tokens(x[L:], r[L:])
    out, same = batch(layer, q1, k1, v1, 0, T, state=pool, kind=hta.LAYER_TARGET).forward()
    got.append(layer.behind(out))
    assert torch.equal(same, pool)
    assert (pool - last).norm() <= 2.0 ** -14 * last.norm()
    got, want = torch.cat(got).float(), want.float()
    # either side: three roundings in the attention (together a half step of the norm), one in the norm behind it; the library's product may round
    # other shapes otherwise (one more, which q, k and v each carry)
    assert (got - want).norm() <= 8 * 2.0 ** -8 * want.norm()


def test_training_gradients_against_differences():
    """The loss sum(y c) of norm -> projections -> linear attention -> norm per head, along a direction in the inputs: the gradient that the backward
    calls give against a central difference of a float64 pass over the same formulas, and against that pass's own gradient."""
    layer = Layer(3)
    L, T = 100, 9
    n = L + T
    x, r = inputs(n, 5)
    gen = torch.Generator(device="cuda").manual_seed(9)
    c = torch.randn((n, Hq * d), device="cuda", generator=gen).bfloat16()
    # the calls
    q, k, v, h, rstd = layer.tokens(x, r)
    b = batch(layer, q, k, v, L, T)
    out, _ = b.forward()
    y2, o2, rstd2 = rms.mtfm_rms_fwd(out.reshape(-1, d), layer.w_out, EPS)
    dout, dw_out = rms.mtfm_rms_bwd(c.view(-1, d), o2, layer.w_out, rstd2)
    dq, dk, dv, _ = b.backward(dout.view(n, Hq, d))
    dqkv = torch.cat([t.flatten(1) for t in (dq, dk, dv)], 1)
    dy = dqkv @ layer.proj.t().contiguous()
    dx, dw_in = rms.mtfm_rms_bwd(dy, h, layer.w_in, rstd)

    def loss(h, w_in, w_out):
        y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * w_in
        q, k, v = (t.unflatten(1, (-1, d)).transpose(0, 1) for t in (y @ layer.proj.double().cpu()).split((Hq * d, Hkv * d, Hkv * d), 1))
        k, v = k.repeat_interleave(Hq // Hkv, 0), v.repeat_interleave(Hq // Hkv, 0)
        at = torch.arange(n).clamp(max=L)
        j = torch.arange(n)
        seen = (j[None] < L) & (j[None] <= j[:, None]) | (j[None] == j[:, None])
        m = torch.where(seen, torch.exp(layer.log_decay.double().cpu()[:, None, None] * (at[:, None] - at[None]).clamp(min=0)), 0.0)
        o = d ** -0.5 * ((q @ k.transpose(1, 2)) * m) @ v
        z = o * torch.rsqrt((o * o).mean(2, keepdim=True) + EPS) * w_out
        return (z.transpose(0, 1).reshape(n, -1) * c.double().cpu()).sum()

    leaves = [t.double().cpu().requires_grad_() for t in (h, layer.w_in, layer.w_out)]
    loss(*leaves).backward()
    for name, got, leaf in (("dx", dx, leaves[0]), ("dw_in", dw_in, leaves[1]), ("dw_out", dw_out, leaves[2])):
        want = leaf.grad
        # some dozen roundings of half a step lie between (y, q, k, v, three in the attention, the norm, and as many backwards): as independent, 4 half steps
        assert (got.double().cpu() - want).norm() <= 4 * 2.0 ** -8 * want.norm(), name
        direction = torch.randn(leaf.shape, dtype=torch.float64, generator=torch.Generator().manual_seed(1))
        e = 1e-5
        args = [t.detach() for t in leaves]
        i = [t is leaf for t in leaves].index(True)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + e * direction, args[i] - e * direction
        slope = (loss(*up) - loss(*down)) / (2 * e)
        assert abs(slope - (want * direction).sum()) <= 1e-6 * want.norm() * direction.norm(), name

"""Linear attention with decay where a result's terms cancel to a thousandth: what a state, or a
product of a query and a key under the decay, keeps beyond the first 16 bits shows then, in bf16
results too.

Terms come in pairs, x and -x (1 + d) with d below 2^-11, each of some 1 to 2; 32 or 64 pairs are a
result of 2e-3 (root mean square).  Tolerances: what terms of 24 bits and fp32 sums leave.  A term
is off by 4 roundings of 2^-24 (a product, a decay's exponential) and a sum of 128 of them in three
parts takes 384 additions at partial sums below 4, which add up at random: (8 sqrt(128) + 4
sqrt(384)) 2^-24 = 1e-5 of a term, held in the norm over all results, and half a step of bf16,
2^-8 of a result.  (Terms of 16 bits are off by 2^-18 at random: 128 of them by 4e-5 of one, 2e-2 of
a result, where half a step and 1e-5 are 8e-3.)"""

import pytest
import torch

import paper_2606_06034_amd as G

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
D, T = 128, 64


class Inputs:
    def __init__(self, dt, seed):
        self.r, self.dt = torch.Generator("cuda").manual_seed(seed), DT[dt]

    def uniform(self, *s):  # 1 .. 2
        return 1 + torch.rand(*s, generator=self.r, device="cuda")

    def signs(self, *s):
        return torch.randint(0, 2, s, generator=self.r, device="cuda") * 2.0 - 1

    def zeros(self, *s):
        return torch.zeros(*s, device="cuda")

    def pairs(self, *s):
        """[..., 2 n] of x, -x (1 + d)"""
        x = self.uniform(*s[:-1], s[-1] // 2)
        d = (self.uniform(*x.shape) - 1) * 2.0 ** -11
        return torch.stack([x, -x * (1 + d)], -1).flatten(-2)


def held(got, ref, term, what):
    off = (got.double() - ref).norm()
    lim = 1e-5 * term * ref.numel() ** 0.5
    if got.dtype == torch.bfloat16:
        lim = lim + 2.0 ** -8 * ref.norm()
    print(what, (off / lim).item(), flush=True)
    assert off <= lim, (what, (off / lim).item())


def twice(t, dim):
    return t.repeat_interleave(2, dim)


def groups(t, Hk):
    """Sum over the value heads of a key head."""
    return t.unflatten(2, (Hk, -1)).sum(3)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,Hv", [(2, 2), (2, 4), (1, 3)])
def test_states(Hk, Hv, dt):
    m = Inputs(dt, Hv)
    g = m.zeros(1, T, Hv)
    q0 = m.zeros(1, T, Hk, D).to(m.dt)
    v = twice(m.signs(1, T, Hv, D // 2), 3).to(m.dt)
    dO = twice(m.signs(1, T, Hv, D // 2), 3).to(m.dt)
    key = twice(m.signs(1, T, Hk, D // 2), 3).to(m.dt)
    rep = lambda t: t.repeat_interleave(Hv // Hk, 2).double()  # noqa: E731
    rows = m.pairs(1, Hv, D, D).transpose(2, 3).contiguous()  # [dk, dv], pairs of rows
    cols = m.pairs(1, Hv, D, D)
    O, _ = G.gdn_linear_forward(key, q0, v, g, S0=rows, scale=1.0)
    held(O, torch.einsum("bthk,bhkv->bthv", rep(key), rows.double()), 1, "O")
    for want_dg in (True, False):
        kw = dict(scale=1.0, want_dg=want_dg)
        dQ, dK, _, _, _ = G.gdn_linear_backward(q0, q0, v, g, dO, S0=cols, dS_final=cols, **kw)
        held(dQ, groups(torch.einsum("bthv,bhkv->bthk", dO.double(), cols.double()), Hk), 1,
             ("dQ", want_dg))
        held(dK, groups(torch.einsum("bthv,bhkv->bthk", v.double(), cols.double()), Hk), 1,
             ("dK", want_dg))
        dV = G.gdn_linear_backward(q0, key, v, g, m.zeros(1, T, Hv, D).to(m.dt), dS_final=rows,
                                   **kw)[2]
        held(dV, torch.einsum("bthk,bhkv->bthv", rep(key), rows.double()), 1, ("dV", want_dg))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,Hv", [(2, 2), (2, 4), (1, 3)])
def test_products_under_the_decay(Hk, Hv, dt):
    m = Inputs(dt, 10 + Hv)
    r = Hv // Hk
    g = -(m.uniform(1, T, Hv) - 1) * 2.0 ** -11
    g[:, 0::2] = 0  # within a pair alone (the pairs' terms stay of one size)
    rep = lambda t: t.repeat_interleave(r, 2).double()  # noqa: E731
    H = g.double().cumsum(1).transpose(1, 2)
    decay = (H[..., :, None] - H[..., None, :]).exp().tril()  # [1, Hv, T, T]
    scale = 1 / (2.25 * D)
    one = lambda *s: m.uniform(*s).to(m.dt)  # noqa: E731
    half = lambda h: one(1, T // 2, h, D).repeat_interleave(2, 1)  # noqa: E731

    def alternating(h):
        t = m.signs(1, T // 2, h, D).repeat_interleave(2, 1)
        t[:, 1::2] *= -1
        return t.to(m.dt)

    def product(x, y, z, back=False):
        p = scale * torch.einsum("bihd,bjhd->bhij", x, y) * decay
        return torch.einsum("bhij,bihd->bjhd" if back else "bhij,bjhd->bihd", p, z)

    # a pair's terms are of one product, so that they differ by the decay alone
    q, k, v = one(1, T, Hk, D), half(Hk), alternating(Hv)
    O, _ = G.gdn_linear_forward(q, k, v, g, scale=scale)
    odd = slice(1, None, 2)  # (tokens that end a pair)
    held(O[:, odd], product(rep(q), rep(k), v.double())[:, odd], 1, "O")
    for want_dg in (True, False):
        kw = dict(scale=scale, want_dg=want_dg)
        dO, v, k = one(1, T, Hv, D), half(Hv), alternating(Hk)
        dQ = G.gdn_linear_backward(q, k, v, g, dO, **kw)[0]
        ref = groups(product(dO.double(), v.double(), rep(k)), Hk)
        held(dQ[:, odd], ref[:, odd], r, ("dQ", want_dg))
        even = slice(0, None, 2)  # (tokens that begin one)
        dO, v, x = half(Hv), one(1, T, Hv, D), alternating(Hk)
        dK = G.gdn_linear_backward(x, k, v, g, dO, **kw)[1]
        ref = groups(product(dO.double(), v.double(), rep(x), True), Hk)
        held(dK[:, even], ref[:, even], r, ("dK", want_dg))
        x, k, dO = half(Hk), one(1, T, Hk, D), alternating(Hv)
        dV = G.gdn_linear_backward(x, k, v, g, dO, **kw)[2]
        held(dV[:, even], product(rep(x), rep(k), dO.double(), True)[:, even], 1, ("dV", want_dg))

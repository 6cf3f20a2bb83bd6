"""Group norm, channels last, and its gradients on the GPU against the fp64 oracle.

Tolerances.  Sums of fp32 terms taken in at most 200 serial steps and a tree are off by at most
220 * 2^-24 of the sum of magnitudes: 1.3e-5.  Values are products of a few such factors, taken
relative to the group's largest magnitude: 4e-5 of it in fp32; bf16 outputs add 2^-8 of the
entry.  dw and db sum over n and positions: 4e-5 of the sum of magnitudes."""

import numpy as np
import pytest
import torch

import paper_2606_06034_amd as G
from oracle import linear

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(N, S, C, groups, dt, wdt, bias, gate, seed):
    rng = np.random.default_rng(seed)

    def dev(a, t):
        return torch.from_numpy(a.astype(np.float32)).cuda().to(DT[t])

    D = C // groups
    x = rng.normal(size=(N, S, groups, D)) * np.exp(rng.normal(size=(N, 1, groups, 1)))
    x = (x + rng.normal(size=(N, 1, groups, 1))).reshape(N, S, C)
    return (dev(x, dt), dev(1 + 0.3 * rng.normal(size=C), wdt),
            dev(0.2 * rng.normal(size=C), wdt) if bias else None,
            dev(2 * rng.normal(size=(N, S, C)), dt) if gate else None,
            dev(rng.normal(size=(N, S, C)), dt))


def f64(*t):
    return [None if v is None else v.double().cpu().numpy() for v in t]


def near(got, ref, size, bf, what):
    got, ref = got.double().cpu().numpy(), np.asarray(ref)
    lim = 4e-5 * size + (np.abs(ref) * 2.0 ** -8 if bf else 0.0)
    assert got.shape == ref.shape and np.isfinite(got).all(), what
    assert (np.abs(got - ref) <= lim).all(), (what, (np.abs(got - ref) / (lim + 1e-30)).max())


SHAPES = [  # N, S, C, groups
    (1, 1, 8, 1), (5, 1, 12, 3), (7, 1, 64, 8), (130, 1, 96, 32), (33, 1, 512, 4),
    (9, 1, 4096, 32), (3, 1, 1025, 5), (2, 1, 8190, 3), (300, 1, 16, 16), (2, 1, 16384, 1),
    (2, 1, 65536, 1), (3, 7, 24, 3), (2, 49, 40, 4), (4, 100, 96, 8), (2, 1000, 33, 3),
    (1, 5000, 64, 2), (2, 4096, 32, 2), (1, 30011, 6, 2), (1, 20000, 10, 1), (2, 9, 9216, 2),
    (1, 3, 30000, 3), (2, 700, 2560, 1)]


def sizes(x, groups, stat):
    """A statistic [N, groups] at every value of x"""
    return np.repeat(stat, x.shape[2] // groups, 1)[:, None, :]


def most(x, groups):
    N, S, C = x.shape
    return np.abs(x).reshape(N, S, groups, -1).max((1, 3))


@pytest.mark.parametrize("dt,wdt", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"),
                                    ("f32", "bf16")])
@pytest.mark.parametrize("N,S,C,groups", SHAPES)
def test_forward_and_backward(N, S, C, groups, dt, wdt):
    for i, (act, bias, gate) in enumerate([(None, False, True), ("silu", True, False),
                                           ("silu", True, True), (None, True, False)]):
        x, w, b, z, dy = make(N, S, C, groups, dt, wdt, bias, gate, N * 7 + S + i)
        eps, bf = 1e-3, dt == "bf16"
        print(N, S, C, groups, dt, act, bias, gate, flush=True)
        y, mean, rstd = G.gdn_group_norm_forward(x, groups, w, bias=b, gate=z, act=act, eps=eps)
        xr, wr, br, zr, dyr = f64(x, w, b, z, dy)
        yr, mr, rr = linear.group_norm(xr, groups, wr, br, zr, act is not None, eps)
        # x - mean carries the rounding of the mean: the group's size times rstd
        size = (most(xr, groups) * rr)[:, None]
        big = sizes(xr, groups, most(xr, groups) * rr + 1) * (1 + np.abs(wr).max())
        f = 1 if z is None else 1 + np.abs(zr)
        near(y, yr, (big + (0 if b is None else 1)) * f, bf, "y")
        near(mean, mr, most(xr, groups), False, "mean")
        assert np.allclose(rstd.cpu().numpy(), rr, rtol=4e-5 * (1 + size.max()))
        dx, dw, db, dz = G.gdn_group_norm_backward(dy, x, groups, w, mean, rstd, bias=b, gate=z,
                                                   act=act)
        dxr, dwr, dbr, dzr = linear.group_norm_grad(dyr, xr, groups, wr, br, zr, act is not None,
                                                    eps)
        xh = linear.group_norm(xr, groups, eps=eps)[0]
        one = 2 if act else 1  # |silu'| is below 1.1, its slope below 0.5
        d = np.abs(dyr * f) * one
        g = most(d, groups) * rr * (1 + most(xh, groups)) ** 2 * (1 + size[:, 0])
        near(dx, dxr, sizes(xr, groups, g) * (1 + np.abs(wr).max()) ** 2, bf, "dx")
        s = (d * (1 + np.abs(xh)) * sizes(xr, groups, 1 + size[:, 0])).sum((0, 1))
        near(dw, dwr, s * (1 + np.abs(wr).max()), False, "dw")
        if b is not None:
            near(db, dbr, s * (1 + np.abs(wr).max()), False, "db")
        if z is not None:
            near(dz, dzr, np.abs(dyr) * (1 + np.abs(zr)) * big * 2, bf, "dz")


def test_more_dimensions_and_no_weight():
    x, _, _, z, dy = make(2, 12, 20, 5, "f32", "f32", False, True, 1)
    x4, z4, dy4 = (t.reshape(2, 3, 4, 20) for t in (x, z, dy))
    y, mean, rstd = G.gdn_group_norm_forward(x, 5, gate=z)
    y4, m4, r4 = G.gdn_group_norm_forward(x4, 5, gate=z4)
    assert torch.equal(y4.reshape(y.shape), y) and torch.equal(m4, mean) and torch.equal(r4, rstd)
    xr, zr, dyr = f64(x, z, dy)
    near(y, linear.group_norm(xr, 5, z=zr)[0], 30, False, "y")
    dx, dw, db, dz = G.gdn_group_norm_backward(dy4, x4, 5, None, mean, rstd, gate=z4, want_dw=False)
    assert dw is None and db is None and dx.shape == x4.shape and dz.shape == z4.shape
    near(dx.reshape(x.shape), linear.group_norm_grad(dyr, xr, 5, z=zr)[0], 300, False, "dx")
    y, mean, rstd = G.gdn_group_norm_forward(x[:, 0].contiguous(), 5)  # [N, C]
    assert mean.shape == (2, 5)
    near(y[:, None], linear.group_norm(xr[:, :1], 5)[0], 30, False, "y")
    y, mean, rstd = G.gdn_group_norm_forward(x, 5, want_stats=False)
    assert mean is None and rstd is None


def test_without_rows():
    e = torch.empty(0, 3, 8, device="cuda")
    y, mean, rstd = G.gdn_group_norm_forward(e, 2, act="silu")
    w = torch.ones(8, device="cuda")
    dx, dw, db, _ = G.gdn_group_norm_backward(e, e, 2, w, mean, rstd, want_db=True)
    assert y.shape == dx.shape == e.shape and (dw == 0).all() and (db == 0).all()


def test_means_far_from_zero():
    """Values of 1000 +- 1: the squares are taken about the mean.  x itself is rounded to 2^-24
    of 1000, which the oracle sees, and its mean once more: 6e-5 of the deviations."""
    for N, S, C, g in ((40, 1, 256, 2), (2, 3000, 64, 4), (2, 20000, 64, 4)):
        x = (1000 + torch.randn(N, S, C, generator=torch.Generator().manual_seed(3))).cuda()
        y, mean, rstd = G.gdn_group_norm_forward(x, g)
        yr, mr, rr = linear.group_norm(x.double().cpu().numpy(), g)
        assert np.allclose(rstd.cpu().numpy(), rr, rtol=4e-5)
        assert np.abs(y.cpu().numpy() - yr).max() < 4e-4


def test_a_group_s_nan_stays_in_it():
    for N, S, C, g in ((50, 1, 128, 4), (4, 60, 64, 4), (3, 20000, 32, 2)):
        x, w, b, _, dy = make(N, S, C, g, "bf16", "f32", True, False, 3)
        y0, m0, r0 = G.gdn_group_norm_forward(x, g, w, bias=b, act="silu")
        d0 = G.gdn_group_norm_backward(dy, x, g, w, m0, r0, bias=b, act="silu")[0]
        x[1, S // 2, C // g] = float("nan")  # in the second group
        y, m, r = G.gdn_group_norm_forward(x, g, w, bias=b, act="silu")
        dx = G.gdn_group_norm_backward(dy, x, g, w, m, r, bias=b, act="silu")[0]
        keep = torch.ones(N, S, C, dtype=torch.bool, device="cuda")
        keep[1, :, C // g:2 * (C // g)] = False
        for t, t0 in ((y, y0), (dx, d0)):
            assert torch.isnan(t[~keep]).all() and torch.equal(t[keep], t0[keep])


def test_the_same_every_time_on_another_stream_and_in_a_graph():
    for N, S, C, g in ((5000, 1, 384, 3), (3, 333, 96, 4), (2, 20000, 32, 2)):
        x, w, b, z, dy = make(N, S, C, g, "bf16", "f32", True, True, 4)

        def call(**kw):
            y, mean, rstd = G.gdn_group_norm_forward(x, g, w, bias=b, gate=z, act="silu", **kw)
            if kw:
                torch.cuda.current_stream().wait_stream(kw["stream"])
                kw["stream"].wait_stream(torch.cuda.current_stream())
            return (y, mean, rstd) + G.gdn_group_norm_backward(dy, x, g, w, mean, rstd, bias=b,
                                                               gate=z, act="silu", **kw)

        want = call()
        for _ in range(3):
            assert all(torch.equal(p, q) for p, q in zip(call(), want))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = call(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for i in range(4):
            x.normal_()
            eager = call()
            for t in got:
                t.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, eager)), i

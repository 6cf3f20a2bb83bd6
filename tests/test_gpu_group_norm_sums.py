"""Gradients of group norm, channels last, whose sums have something to show: dy has a mean and a
part along the normalised values, so that the groups' means that dx leaves out of it, and dw and
db, are as large as dx's other terms.

The reference is the formula in 64 bits in elementary torch operations.  Tolerances, in the norm
of a whole result.  dx, dz: products of some ten factors that are off by 2^-24 each, and of the
normalised values, which carry the rounding of a mean of twice the deviation: 30 of 2^-24, 2e-6,
of terms that are up to three times the result: 1e-5 with room for the hardware's exponential and
reciprocal (1e-7 of each); bf16 outputs add half a step, 2^-8.  dw, db: sums in fp32 of at most
300 serial steps, 300 * 2^-24 = 1.8e-5 of the sum of magnitudes, and what their terms are off by,
1e-5: 4e-5."""

import pytest
import torch

import paper_2606_06034_amd as G

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def reference(x, w, b, z, dy, groups, act, eps, means=(1, 1)):
    """(dx, dw, db, dz, sums of magnitudes of dw, of db) in 64 bits; means: of dh and of dh h, as
    they are taken out of dx"""
    N, S, C = x.shape
    x, w, b, z, dy = (None if t is None else t.double() for t in (x, w, b, z, dy))
    g = lambda t: t.view(N, S, groups, C // groups)  # noqa: E731
    mean = lambda t: g(t).mean((1, 3), keepdim=True)  # noqa: E731
    h = g(x) - mean(x)
    h = (h * (h.square().mean((1, 3), keepdim=True) + eps).rsqrt()).view(N, S, C)
    rstd = ((g(x) - mean(x)).square().mean((1, 3), keepdim=True) + eps).rsqrt()
    n = h if w is None else h * w
    n = n if b is None else n + b
    y, dn, dz = n, dy, None
    if act:
        s = torch.sigmoid(n)
        y = n * s
    if z is not None:
        t = torch.sigmoid(z)
        dz = dy * y * t * (1 + z * (1 - t))
        dn = dn * z * t
    if act:
        dn = dn * s * (1 + n * (1 - s))
    dh = dn if w is None else dn * w
    dx = g(dh) - means[0] * mean(dh) - means[1] * g(h) * mean(dh * h)
    dx = (rstd * dx).view(N, S, C)
    return (dx, (dn * h).sum((0, 1)), dn.sum((0, 1)), dz, (dn * h).abs().sum((0, 1)),
            dn.abs().sum((0, 1)))


def make(N, S, C, groups, dt, wdt, bias, gate, seed, device="cuda"):
    r = torch.Generator(device).manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=r, device=device)  # noqa: E731
    size, mean = normal(N, 1, groups, 1).exp(), 2 * torch.rand(N, 1, groups, 1, generator=r,
                                                              device=device) - 1
    h = normal(N, S, groups, C // groups)
    x = ((h + 2 * mean) * size).view(N, S, C).to(DT[dt])
    dy = (normal(N, S, C) + 1 + h.view(N, S, C)).to(DT[dt])
    return (x, (1 + 0.3 * normal(C)).to(DT[wdt]), (0.2 * normal(C)).to(DT[wdt]) if bias else None,
            (2 * normal(N, S, C)).to(DT[dt]) if gate else None, dy)


def in_norm(got, ref, c, what, size=None):
    lim = c * (ref if size is None else size).norm()
    off = (got.double() - ref).norm()
    assert off <= lim, (what, (off / lim).item())


def check(N, S, C, groups, dt, wdt, act, bias, gate):
    print(N, S, C, groups, dt, wdt, act, bias, gate, flush=True)
    x, w, b, z, dy = make(N, S, C, groups, dt, wdt, bias, gate, N + S + C)
    _, mean, rstd = G.gdn_group_norm_forward(x, groups, w, bias=b, gate=z, act=act, eps=1e-3)
    dx, dw, db, dz = G.gdn_group_norm_backward(dy, x, groups, w, mean, rstd, bias=b, gate=z,
                                               act=act, want_db=True)
    ref = reference(x, w, b, z, dy, groups, act, 1e-3)
    c = 1e-5 + (2.0 ** -8 if dt == "bf16" else 0)
    in_norm(dx, ref[0], c, "dx")
    in_norm(dw, ref[1], 4e-5, "dw", ref[4])
    in_norm(db, ref[2], 4e-5, "db", ref[5])
    if gate:
        in_norm(dz, ref[3], c, "dz")


MANY = [  # N, S, C, groups: maps of few positions, and rows of long groups
    (65536, 4, 64, 8), (30011, 2, 33, 3), (5000, 9, 40, 4), (4096, 1, 16384, 1), (2500, 1, 9000, 3),
    (2049, 3, 5120, 2)]


@pytest.mark.parametrize("dt,wdt,act,bias,gate", [("bf16", "bf16", None, False, True),
                                                  ("f32", "f32", "silu", True, False),
                                                  ("bf16", "f32", "silu", True, True)])
@pytest.mark.parametrize("N,S,C,groups", MANY)
def test_many_rows(N, S, C, groups, dt, wdt, act, bias, gate):
    check(N, S, C, groups, dt, wdt, act, bias, gate)


SHAPES = [  # groups of 32 values and more: in registers, in parts of positions, in column blocks
    (33, 1, 512, 4), (9, 1, 4096, 32), (3, 1, 1025, 5), (2, 1, 8190, 3), (700, 1, 2048, 16),
    (2, 1, 16384, 1), (2, 1, 65536, 1), (3, 7, 24, 3), (2, 49, 40, 4), (4, 100, 96, 8),
    (2, 1000, 33, 3), (1, 5000, 64, 2), (2, 4096, 32, 2), (1, 30011, 6, 2), (1, 20000, 10, 1),
    (2, 9, 9216, 2), (1, 3, 30000, 3), (2, 700, 2560, 1), (3, 3001, 328, 8), (60, 300, 640, 32)]


@pytest.mark.parametrize("dt,wdt", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"),
                                    ("f32", "bf16")])
@pytest.mark.parametrize("N,S,C,groups", SHAPES)
def test_means_and_sums(N, S, C, groups, dt, wdt):
    for act, bias, gate in ((None, False, True), ("silu", True, False), ("silu", True, True),
                            (None, True, False)):
        check(N, S, C, groups, dt, wdt, act, bias, gate)

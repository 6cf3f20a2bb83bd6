"""Linear attention and group norm on tensors past 2^32 bytes against 64 bits: what lies behind is
held to the norm of its own result, so that zeros, or another row's results, are far outside.

Tolerances, in norm: 1e-5 of the result for fp32 (2^-24 times the square root of 400 roundings
that add up at random, of sums that cancel to a tenth) and half a step of bf16, 2^-8, more where a
result is in bf16; the results of 500 tokens out of a long sequence may besides lack what is left
of those before them, e^-40."""

import pytest
import torch

import paper_2606_06034_amd as G
from oracle import linear
from test_gpu_group_norm_sums import in_norm as near
from test_gpu_linear_large import LAST, LONG, packed  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
STEP, FEW = 2.0 ** -8, 1e-5


def f64(t):
    return t.double().cpu().numpy()


def test_linear_attention_behind_2_to_the_32_bytes(packed):  # noqa: F811
    x, cu = packed
    names = ("Q", "K", "V", "g")
    O, S = G.gdn_linear_forward(*(x[k] for k in names), cu_seqlens=cu)
    got = G.gdn_linear_backward(*(x[k] for k in names), x["dO"], cu_seqlens=cu)
    torch.cuda.synchronize()
    for what, first, n, skip in (("last sequence", LONG, LAST, 0), ("end of the long one",
                                                                    LONG - 700, 700, 200)):
        print(what, flush=True)
        a = [f64(x[k][0, first:first + n]) for k in names]
        dO = f64(x["dO"][0, first:first + n])
        scale = 128 ** -0.5
        rO, rS = linear.linear(*a, scale=scale)
        ref = linear.linear_grad(*a, dO, scale=scale)
        rows = slice(first + skip, first + n)
        for t, r, c, name in [(O, rO, STEP, "O")] + list(zip(got[:4], ref[:4], (STEP,) * 3 + (0,),
                                                            ("dQ", "dK", "dV", "dg"))):
            near(t[0, rows], torch.from_numpy(r[skip:]).cuda(), FEW + c, (what, name))
        near(S[1 if first == LONG else 0], torch.from_numpy(rS).cuda(), FEW, (what, "S"))


def pieces(rows, n=50_000):
    return ((i, min(i + n, rows)) for i in range(0, rows, n))


def test_gradients_of_a_large_map():
    """A map of 750000 positions: 1500 serial steps and a tree, 1e-4 of the sums' magnitudes."""
    torch.manual_seed(3)
    N, S, C, groups = 3, 750_000, 1024, 32
    x = torch.randn(N, S, C, dtype=torch.bfloat16, device="cuda")
    dy = torch.randn(N, S, C, dtype=torch.bfloat16, device="cuda").add_(x).add_(1)
    assert x.numel() * 2 > 1 << 32
    w = 1 + 0.1 * torch.randn(C, device="cuda")
    y, mean, rstd = G.gdn_group_norm_forward(x, groups, w, act="silu")
    del y
    dx, dw, db, _ = G.gdn_group_norm_backward(dy, x, groups, w, mean, rstd, act="silu",
                                              want_db=True)
    torch.cuda.synchronize()
    each = lambda t: t.double().repeat_interleave(C // groups)  # noqa: E731

    def dn_h(n, i, j):
        h = (x[n, i:j].double() - each(mean[n])) * each(rstd[n])
        t = h * w
        s = torch.sigmoid(t)
        return dy[n, i:j].double() * s * (1 + t * (1 - s)), h

    sums, size = (torch.zeros(2, C, dtype=torch.float64, device="cuda") for _ in range(2))
    for n in range(N):
        own = torch.zeros_like(sums)
        for i, j in pieces(S):
            dn, h = dn_h(n, i, j)
            own += torch.stack([(dn * h).sum(0), dn.sum(0)])
            size += torch.stack([(dn * h).abs().sum(0), dn.abs().sum(0)])
        sums += own
    near(dw, sums[0], 1e-4, "dw", size[0])
    near(db, sums[1], 1e-4, "db", size[1])
    m = (own * w).view(2, groups, -1).sum(2) / (S * C // groups)  # of the last map
    for i, j in ((0, 1000), (S - 1000, S)):
        dn, h = dn_h(N - 1, i, j)
        ref = (dn * w - each(m[1]) - h * each(m[0])) * each(rstd[N - 1])
        near(dx[N - 1, i:j], ref, FEW + STEP, ("dx", i))


def test_gradients_of_many_rows():
    torch.manual_seed(4)
    N, C, groups = 2_250_000, 1024, 32
    x = torch.randn(N, C, dtype=torch.bfloat16, device="cuda")
    dy = torch.randn(N, C, dtype=torch.bfloat16, device="cuda").add_(x).add_(1)
    assert x.numel() * 2 > 1 << 32
    w = 1 + 0.1 * torch.randn(C, device="cuda")
    y, mean, rstd = G.gdn_group_norm_forward(x, groups, w, gate=dy)
    del y
    dx, dw, _, dz = G.gdn_group_norm_backward(dy, x, groups, w, mean, rstd, gate=dy)
    torch.cuda.synchronize()
    sums, size = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(2))
    each = lambda t: t.double().repeat_interleave(C // groups, 1)  # noqa: E731
    for i, j in pieces(N):
        z = dy[i:j].double()
        h = (x[i:j].double() - each(mean[i:j])) * each(rstd[i:j])
        s = torch.sigmoid(z)
        dn = z * z * s
        sums += (dn * h).sum(0)
        size += (dn * h).abs().sum(0)
    # (2250000 rows in 1024 parts of several at a time: below 2200 serial steps of the parts' sums)
    near(dw, sums, 2200 * 2.0 ** -24, "dw", size)
    g = lambda t: t.view(j - i, groups, -1).mean(2)  # noqa: E731  (of the last piece)
    dh = dn * w
    near(dx[i:j], (dh - each(g(dh)) - h * each(g(dh * h))) * each(rstd[i:j]), FEW + STEP, "dx")
    near(dz[i:j], z * h * w * s * (1 + z * (1 - s)), FEW + STEP, "dz")

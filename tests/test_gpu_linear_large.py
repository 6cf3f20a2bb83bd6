"""Linear attention and group norm on tensors past 2^32 bytes: what lies behind is what the same
rows give by themselves.

Tolerances.  Both sides round the same formulas at other cuts of a sequence: each is off by 1e-4
of the terms' magnitudes (below 64 here: unit keys, decays of e^-0.2 a token, so a reach of 30
tokens, values below 6) and half a step of bf16, 2^-8 of the entry."""

import pytest
import torch

import paper_2606_06034_amd as G

pytestmark = pytest.mark.gpu
LONG, LAST = 2_200_000, 333


def same(a, b, size):
    lim = 2 * (1e-4 * size + 2.0 ** -8 * b.float().abs())
    assert ((a.float() - b.float()).abs() <= lim).all()


@pytest.fixture(scope="module")
def packed():
    torch.manual_seed(1)
    n, Hk, Hv, d = LONG + LAST, 1, 8, 128
    unit = lambda: torch.nn.functional.normalize(  # noqa: E731
        torch.randn(1, n, Hk, d, device="cuda"), dim=-1).bfloat16()
    x = dict(Q=unit(), K=unit(), V=torch.randn(1, n, Hv, d, dtype=torch.bfloat16, device="cuda"),
             g=torch.full((1, n, Hv), -0.2, device="cuda"))
    x["dO"] = x["V"].flip(1)
    assert x["V"].numel() * 2 > 1 << 32
    yield x, torch.tensor([0, LONG, n], dtype=torch.int32, device="cuda")
    x.clear()


def test_the_last_sequence_of_a_large_pack(packed):
    x, cu = packed
    tail = {k: v[:, LONG:].contiguous() for k, v in x.items()}
    a, b = ([t[k] for k in ("Q", "K", "V", "g")] for t in (x, tail))
    print("forward", flush=True)
    O, S = G.gdn_linear_forward(*a, cu_seqlens=cu)
    want, Sw = G.gdn_linear_forward(*b)
    same(O[:, LONG:], want, 64)
    same(S[1], Sw[0], 64)
    # 500 tokens of the long one, from where nothing before them is left (e^-40 of it)
    mid = {k: v[:, LONG - 700:LONG].contiguous() for k, v in x.items()}
    c = [mid[k] for k in ("Q", "K", "V", "g")]
    want, Sw = G.gdn_linear_forward(*c)
    same(O[:, LONG - 500:LONG], want[:, 200:], 64)
    same(S[0], Sw[0], 64)
    del O, S
    print("backward", flush=True)
    got = G.gdn_linear_backward(*a, x["dO"], cu_seqlens=cu)
    for p, q in zip(got[:4], G.gdn_linear_backward(*b, tail["dO"])[:4]):
        same(p[:, LONG:], q, 64 * 8)  # (8 value heads to a key head)
    want = G.gdn_linear_backward(*c, mid["dO"])
    for p, q in zip(got[:4], want[:4]):
        same(p[:, LONG - 500:LONG], q[:, 200:], 64 * 8)
    del got
    print("recurrent", flush=True)
    O, S = G.gdn_linear_recurrent(a[0][:, LONG:], a[1][:, LONG:], a[2][:, LONG:], a[3][:, LONG:])
    same(O, G.gdn_linear_forward(*b)[0], 64)


def test_the_last_state_of_a_large_pool():
    n, Hv, d = 4200, 16, 128
    pool = torch.zeros(n, Hv, d, d, device="cuda")
    assert pool.numel() * 4 > 1 << 32
    pool[-1].normal_()
    last = pool[-1:].clone()
    q, k = (torch.randn(2, 1, 4, d, device="cuda").bfloat16() for _ in range(2))
    v = torch.randn(2, 1, Hv, d, device="cuda").bfloat16()
    g = torch.full((Hv,), -0.1, device="cuda")
    slots = torch.tensor([n - 1, 0], dtype=torch.int32, device="cuda")
    O, _ = G.gdn_linear_recurrent(q, k, v, g, S0=pool, S_final=pool, slots=slots)
    want, S = G.gdn_linear_recurrent(q[:1], k[:1], v[:1], g, S0=last)
    assert torch.equal(O[:1], want) and torch.equal(pool[-1:], S)
    assert (pool[1:-1].amax() == 0) and (pool[0] != 0).any()


def test_large_maps():
    torch.manual_seed(2)
    N, S, C, groups = 3, 750_000, 1024, 32
    x = torch.randn(N, S, C, dtype=torch.bfloat16, device="cuda")
    assert x.numel() * 2 > 1 << 32
    w = 1 + 0.1 * torch.randn(C, device="cuda")
    y, mean, rstd = G.gdn_group_norm_forward(x, groups, w, act="silu")
    # statistics of the last map, in 64 bits a piece at a time
    s = torch.zeros(2, groups, dtype=torch.float64, device="cuda")
    for t in x[-1].split(50_000):
        t = t.double().view(-1, groups, C // groups)
        s += torch.stack([t.sum((0, 2)), t.square().sum((0, 2))])
    n = S * C // groups
    m = s[0] / n
    r = (s[1] / n - m * m + 1e-5).rsqrt()
    assert (mean[-1] - m).abs().max() < 1e-5 and (rstd[-1] - r).abs().max() < 1e-4
    t = x[-1, -1000:].double().view(-1, groups, C // groups)
    t = ((t - m[:, None]) * r[:, None]).view(-1, C) * w
    same(y[-1, -1000:], t * torch.sigmoid(t), 10)
    del y
    rows = x.view(-1, C)  # as rows of heads
    y, mean, rstd = G.gdn_group_norm_forward(rows, groups, w, gate=rows)
    want = G.gdn_group_norm_forward(rows[-100:], groups, w, gate=rows[-100:])[0]
    assert torch.equal(y[-100:], want)
    dx, dw, _, dz = G.gdn_group_norm_backward(y, rows, groups, w, mean, rstd, gate=rows)
    want = G.gdn_group_norm_backward(y[-100:], rows[-100:], groups, w, mean[-100:], rstd[-100:],
                                     gate=rows[-100:])
    assert torch.equal(dx[-100:], want[0]) and torch.equal(dz[-100:], want[3])

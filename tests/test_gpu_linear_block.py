"""Linear attention and group norm as a layer has them: the heads' outputs, normalised head by
head and gated.  Its training step, its serving (a prompt at once, then token by token out of a
pool of states, in a graph), and what is left alone behind the last sequence.

Tolerances.  An output o of linear attention is off by e <= c size + 2^-8 |o| (test_gpu_linear.py;
the second in bf16 alone).  A head's norm takes an error of norm E = |e| to one of at most rstd E
of the normalised values (the derivative of x -> (x - mean) rstd is rstd times a projection, to
first order, with twice that for the rest), to which the norm adds its own (test_gpu_group_norm.py:
4e-5 of the largest magnitude, and half a step).  Gradients in fp32, from the first operand to the
last: each operator is off by 4e-5 of the magnitudes that it sums, which is 1e-3 of the norm of a
gradient of random operands at most (sums of n terms of random sign are smaller than their
magnitudes by sqrt n, n below 300: 17; three such steps)."""

import numpy as np
import pytest
import torch

import paper_2606_06034_amd as G
from oracle import linear
from test_gpu_linear import f64, make

pytestmark = pytest.mark.gpu
EPS = 1e-5


def layer(x, w, z, cu=None, **kw):
    """(y, O, mean, rstd, S): rows of Hv heads of dv."""
    O, S = G.gdn_linear_forward(x["Q"], x["K"], x["V"], x["g"], S0=x["S0"], cu_seqlens=cu, **kw)
    Hv, dv = O.shape[-2:]
    rows = O.view(-1, Hv * dv)
    return G.gdn_group_norm_forward(rows, Hv, w, gate=z, eps=EPS) + (rows, S)


def layer_grad(x, w, z, dy, mean, rstd, rows, cu=None):
    """(dQ, dK, dV, dg, dS0, dw, dz)"""
    Hv = x["V"].shape[2]
    dO, dw, _, dz = G.gdn_group_norm_backward(dy, rows, Hv, w, mean, rstd, gate=z)
    return G.gdn_linear_backward(x["Q"], x["K"], x["V"], x["g"], dO.view_as(x["V"]), S0=x["S0"],
                                 dS_final=x["dS"], want_dS0=x["S0"] is not None,
                                 cu_seqlens=cu) + (dw, dz)


def exact(x, w, z, lens, scale):
    """(y, O, its sizes) in 64 bits"""
    at, O, size = 0, [], []
    for s, n in enumerate(lens):
        a = [f64(x[k]) for k in ("Q", "K", "V", "g")]
        a = [v if v.ndim == 1 else v.reshape((-1,) + v.shape[2:])[at:at + n] for v in a]
        S0 = None if x["S0"] is None else f64(x["S0"])[s]
        O.append(linear.linear(*a, S0, scale)[0])
        size.append(linear.linear_sizes(*a, S0=S0, scale=scale)[0])
        at += n
    O, size = np.concatenate(O), np.concatenate(size)
    Hv = O.shape[1]
    y, mean, rstd = linear.group_norm(O.reshape(at, 1, -1), Hv, f64(w), None, f64(z)[:, None],
                                      eps=EPS)
    return y[:, 0], O, size, mean, rstd


def operands(lens, Hk, Hv, dt, per_token, packed, seed, state=True):
    x = make(lens, Hk, Hv, 64, 128, dt, per_token, state, seed, packed)
    n = sum(lens)
    w = (1 + 0.3 * torch.randn(Hv * 128, device="cuda")).to(x["V"].dtype)
    z, dy = (torch.randn(n, Hv * 128, device="cuda").to(x["V"].dtype) for _ in range(2))
    return x, w, z, dy


def close(y, ref, O, size, mean, rstd, w, z, bf):
    c = 1e-4 if bf else 3e-5
    e = c * size + (2.0 ** -8 * np.abs(O) if bf else 0)
    E = 2 * np.linalg.norm(e, axis=2) * rstd  # [rows, heads]
    most = np.abs(O - mean[:, :, None]).max(2) * rstd + np.abs(O).max(2) * rstd + 1
    f = np.abs(f64(w)) * np.abs(f64(z)) + 1e-30
    heads = lambda a: np.repeat(a, O.shape[2], 1)  # noqa: E731
    lim = heads(E + 4e-5 * most) * (f + 4e-5) + (2.0 ** -8 * np.abs(ref) if bf else 0)
    assert (np.abs(f64(y) - ref) <= lim).all(), (np.abs(f64(y) - ref) / lim).max()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("lens,packed,per_token", [([200, 200], False, False),
                                                   ([3, 0, 150, 1], True, True)])
def test_rows_of_heads(lens, packed, per_token, dt):
    x, w, z, _ = operands(lens, 2, 4, dt, per_token, packed, 3)
    y, mean, rstd, rows, S = layer(x, w, z, x["cu"])
    ref, O, size, m, r = exact(x, w, z, lens, 64 ** -0.5)
    close(y, ref, O, size, m, r, w, z, dt == "bf16")


def test_gradients_are_those_of_the_formulas_and_the_differences():
    """fp32, from the layer's first operand to its last."""
    lens, scale = [70], 64 ** -0.5
    x, w, z, dy = operands(lens, 1, 2, "f32", True, False, 5)
    x["dS"] = None
    y, mean, rstd, rows, S = layer(x, w, z)
    got = layer_grad(x, w, z, dy, mean, rstd, rows)
    a = [f64(x[k])[0] for k in ("Q", "K", "V", "g")] + [f64(x["S0"])[0]]
    wn, zn, dyn = f64(w), f64(z), f64(dy)
    O = linear.linear(*a, scale)[0]
    dO, dw, _, dz = linear.group_norm_grad(dyn[:, None], O.reshape(70, 1, -1), 2, wn, None,
                                           zn[:, None], eps=EPS)
    ref = linear.linear_grad(*a[:4], dO.reshape(O.shape), a[4], None, scale) + (dw, dz[:, 0])
    for p, r, name in zip(got, ref, ("dQ", "dK", "dV", "dg", "dS0", "dw", "dz")):
        p = f64(p).reshape(r.shape)
        assert np.linalg.norm(p - r) <= 1e-3 * np.linalg.norm(r), name

    def loss(v):
        O = linear.linear(*v[:4], v[4], scale)[0].reshape(70, 1, -1)
        return (linear.group_norm(O, 2, v[5], None, v[6][:, None], eps=EPS)[0][:, 0] * dyn).sum()

    rng = np.random.default_rng(0)
    at = a + [wn, zn]
    for i, p in enumerate(got):  # along a random direction: third differences are h^2 of it
        d = rng.normal(size=at[i].shape)
        h = 1e-4
        up, down = ([v + s * d if j == i else v for j, v in enumerate(at)] for s in (h, -h))
        want, mine = (loss(up) - loss(down)) / (2 * h), (f64(p).reshape(d.shape) * d).sum()
        assert abs(mine - want) <= 1e-3 * np.linalg.norm(f64(p)) * np.sqrt(np.log(d.size + 2)) * 3


def test_a_training_step_in_a_graph():
    """Replayed with new values, bit for bit the eager step's."""
    lens = [130, 1, 400]
    x, w, z, dy = operands(lens, 2, 4, "bf16", True, True, 6)

    def step():
        y, mean, rstd, rows, S = layer(x, w, z, x["cu"])
        return (y, S) + layer_grad(x, w, z, dy, mean, rstd, rows, x["cu"])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        for t in (x["V"], x["S0"], z, dy):
            t.normal_()
        eager = step()
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, eager)), i


def test_a_prompt_then_tokens_one_by_one():
    """Prompts packed, their states put into a pool, then one token of each a step in a graph:
    the rows of the whole sequences at once."""
    Hk, Hv, more, lens = 2, 4, 5, [37, 1, 129]
    x, w, z, _ = operands([n + more for n in lens], Hk, Hv, "bf16", True, True, 8, state=False)
    whole = [n + more for n in lens]
    starts = np.cumsum([0] + whole)
    prompt = np.concatenate([np.arange(s, s + n) for s, n in zip(starts, lens)])
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    p = {k: x[k][:, prompt].contiguous() for k in ("Q", "K", "V", "g")}
    p["S0"] = None
    _, _, _, rows, S = layer(p, w, z[prompt].contiguous(), cu)
    pool = torch.full((7,) + tuple(S.shape[1:]), float("nan"), device="cuda")
    slots = torch.tensor([4, 0, 6, -1], dtype=torch.int32, device="cuda")  # the last: padded
    pool[slots[:3].long()] = S
    one = {k: torch.zeros((4, 1) + tuple(x[k].shape[2:]), dtype=x[k].dtype, device="cuda")
           for k in ("Q", "K", "V", "g")}
    zt = torch.zeros(4, Hv * 128, dtype=z.dtype, device="cuda")

    def step():
        O, _ = G.gdn_linear_recurrent(one["Q"], one["K"], one["V"], one["g"], S0=pool,
                                      S_final=pool, slots=slots)
        return G.gdn_group_norm_forward(O.view(4, -1), Hv, w, gate=zt, eps=EPS, want_stats=False)[0]

    keep = pool.clone()
    step()  # (its launches are known before the capture)
    pool.copy_(keep)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    got = []
    for t in range(more):
        at = [s + n + t for s, n in zip(starts, lens)]
        for k in one:
            one[k][:3, 0] = x[k][0, at]
        zt[:3] = z[at]
        graph.replay()
        torch.cuda.synchronize()
        assert (y[3] == 0).all()  # (a padded row's zeros, normalised)
        got.append(y[:3].clone())
    ref, O, size, m, r = exact(x, w, z, whole, 64 ** -0.5)
    at = np.concatenate([[s + n + t for s, n in zip(starts, lens)] for t in range(more)])
    close(torch.cat(got), ref[at], O[at], size[at], m[at], r[at], w, z[at], True)
    left = [i for i in range(7) if i not in (4, 0, 6)]
    assert torch.isnan(pool[left]).all()


def test_rows_behind_the_last_sequence_are_left_alone():
    x, w, z, dy = operands([300], 2, 4, "bf16", True, True, 9)
    x["cu"] = torch.tensor([0, 100, 170], dtype=torch.int32, device="cuda")
    S0 = torch.randn(2, 4, 64, 128, device="cuda")
    a = [x[k] for k in ("Q", "K", "V", "g")]
    O = torch.full_like(x["V"], 7.0)
    out = [torch.full_like(x[k], 7.0) for k in ("K", "K", "V", "g")] + [torch.empty_like(S0)]
    G.gdn_linear_forward(*a, S0=S0, O=O, cu_seqlens=x["cu"])
    G.gdn_linear_backward(*a, x["dO"], S0=S0, want_dS0=True, out=out, cu_seqlens=x["cu"])
    R = torch.full_like(x["V"], 7.0)
    G.gdn_linear_recurrent(*a, S0=S0, O=R, cu_seqlens=x["cu"])
    for t in [O, R] + out[:4]:
        assert (t[:, 170:] == 7).all() and (t[:, :170] != 7).any()

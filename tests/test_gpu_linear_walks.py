"""Linear attention with decay where a workgroup walks over several chunks of a segment, and a
sequence has several such segments, against the fp64 oracle: many sequences at a time, of which a
few are compared (the segments are as long as the calls are large).

Tolerances: those of test_gpu_linear.py, whose decays these have.  The largest error of an entry is
held to 1e-4 (fp32 and three-term results 3e-5) of the magnitudes that it sums, and half a step of
bf16; the norm of the errors, which add up at random, to 1e-5 of the result's (2^-24 times the
square root of 400 roundings, of sums that cancel to a tenth) and half a step."""

import numpy as np
import pytest
import torch

import paper_2606_06034_amd as G
from oracle import linear
from test_gpu_linear import DT, f64, in_norm, make, near

pytestmark = pytest.mark.gpu


def tokens_a_segment(nseq, T, Hk, Hv, dk, dv, packed, dt):
    """(forward, backward): at least, from the workspaces, which hold the states [dk, dv] and the
    decay of each segment and head."""
    a = (nseq, T, Hk, Hv, dk, dv, packed, DT[dt])
    tok, state = T if packed else nseq * T, Hv * dk * dv
    fwd = G.gdn_linear_forward_workspace(*a) // 4 // (state + Hv)
    rest = 2 * Hv * tok + (2 * tok * Hk * dk if Hv > Hk else 0)
    bwd = (G.gdn_linear_backward_workspace(*a) // 4 - rest) // (2 * state)
    out = []
    for slots in (fwd, bwd):
        slots -= nseq if packed else 0  # (a packed sequence may end within one)
        out.append(tok // slots if slots > 0 else T)
    return out


def compare(lens, Hk, Hv, dk, dv, dt, packed, chosen, least):
    print(len(lens), max(lens), Hk, Hv, dk, dv, dt, packed, flush=True)
    x = make(lens, Hk, Hv, dk, dv, dt, True, True, sum(lens) + Hv, packed)
    bf, scale, a = dt == "bf16", 0.3, [x[k] for k in ("Q", "K", "V", "g")]
    sizes = (len(lens), sum(lens) if packed else lens[0], Hk, Hv, dk, dv, packed, dt)
    assert min(tokens_a_segment(*sizes)) >= least, tokens_a_segment(*sizes)
    O, S = G.gdn_linear_forward(*a, S0=x["S0"], scale=scale, cu_seqlens=x["cu"])
    got = G.gdn_linear_backward(*a, x["dO"], S0=x["S0"], dS_final=x["dS"], scale=scale,
                                want_dS0=True, cu_seqlens=x["cu"])
    less = G.gdn_linear_backward(*a, x["dO"], S0=x["S0"], dS_final=x["dS"], scale=scale,
                                 want_dg=False, cu_seqlens=x["cu"])
    torch.cuda.synchronize()
    assert all(torch.isfinite(t.float()).all() for t in (O, S, *got))
    at = np.concatenate([[0], np.cumsum(lens)])
    c, step = (1e-4, 2.0 ** -8) if bf else (3e-5, 0.0)

    def rows(t, s):
        return f64(t.flatten(0, 1)[at[s]:at[s + 1]])

    def held(t, ref, size, what):
        near(t, ref, size, c, bf, what)
        in_norm(t, ref, 1e-5 + step, what)

    for s in chosen:
        n = [rows(t, s) for t in a]
        S0, dS = f64(x["S0"])[s], f64(x["dS"])[s]
        ref, size = linear.linear(*n, S0, scale), linear.linear_sizes(*n, S0=S0, scale=scale)
        held(rows(O, s), ref[0], size[0], "O")
        near(f64(S)[s], ref[1], size[1], 3e-5, False, "S")
        in_norm(f64(S)[s], ref[1], 2e-6, "S")
        dO = rows(x["dO"], s)
        ref = linear.linear_grad(*n, dO, S0, dS, scale)
        size = linear.linear_sizes(*n, dO, S0, dS, scale)
        for i, what in enumerate(("dQ", "dK", "dV")):
            held(rows(got[i], s), ref[i], size[i], what)
            held(rows(less[i], s), ref[i], size[i], what + " without dg")
        near(rows(got[3], s), ref[3], size[3], 3e-5, False, "dg")
        in_norm(rows(got[3], s), ref[3], 1e-5, "dg")
        near(f64(got[4])[s], ref[4], size[4], 3e-5, False, "dS0")
        in_norm(f64(got[4])[s], ref[4], 2e-6, "dS0")
    return x, got


EQUAL = [  # sequences, tokens, key and value heads, dk, dv: groups of 1, 2, 3, 4 and 8
    (32, 400, 4, 4, 64, 64), (32, 400, 4, 8, 64, 64), (32, 400, 4, 12, 64, 64),
    (32, 400, 4, 16, 64, 64), (32, 500, 2, 16, 64, 64), (32, 400, 4, 4, 128, 128),
    (32, 400, 2, 8, 64, 128), (32, 400, 2, 8, 128, 64)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("B,T,Hk,Hv,dk,dv", EQUAL)
def test_walks_of_several_chunks(B, T, Hk, Hv, dk, dv, dt):
    compare([T] * B, Hk, Hv, dk, dv, dt, False, (0, B - 1), 100)


PACKED = [1300, 0, 700, 64, 65, 1, 129, 2, 513, 800, 640, 63, 576, 300, 1100, 17, 450, 512, 130,
          3, 0, 200, 90, 250, 1024, 900, 333, 705, 511, 602]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,Hv", [(8, 8), (4, 8), (4, 12), (4, 16)])
def test_packed_walks_of_several_chunks(Hk, Hv, dt):
    compare(PACKED, Hk, Hv, 64, 64, dt, True, (2, 8, 17, 29), 100)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("Hk,Hv", [(4, 4), (4, 16), (4, 12)])
def test_a_head_s_decay_over_several_chunks(Hk, Hv, dt):
    """A decay of each head, given as such and as every token's: its gradient is the sum of the
    tokens', of which there are 12800 a head in 7 or more partial sums (fp32 within a chunk's 64 and
    a workgroup's, 64 bits over these): 100 roundings of 2^-24 of the magnitudes."""
    x = make([400] * 32, Hk, Hv, 64, 64, dt, False, True, 3, False)
    a = [x[k] for k in ("Q", "K", "V")]
    kw = dict(S0=x["S0"], dS_final=x["dS"], want_dS0=True)
    one = G.gdn_linear_backward(*a, x["g"], x["dO"], **kw)
    each = G.gdn_linear_backward(*a, x["g"].expand(32, 400, Hv).contiguous(), x["dO"], **kw)
    assert (f64(one[3]) != 0).all()
    near(f64(one[3]), f64(each[3]).sum((0, 1)), np.abs(f64(each[3])).sum((0, 1)), 100 * 2.0 ** -24,
         False, "dg")
    for p, q in zip(one[:3] + one[4:], each[:3] + each[4:]):
        # the decays' sums are products in one and sums in the other: 2^-24 of each factor
        in_norm(f64(p), f64(q), 1e-6 + (2.0 ** -8 if p.dtype == torch.bfloat16 else 0.0), "others")

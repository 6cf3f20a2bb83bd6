"""Linear attention with decay on the GPU against the fp64 oracle: the chunked form, its gradients
and the recurrent form.

Tolerances.  A result is a sum whose terms' magnitudes add up to `size` (the oracle's
linear_sizes).  Its roundings: a state takes at most 2 more a chunk and 64 in it, of at most
8 chunks within the reach of the decays tested here or of 400 tokens; an output 128 terms of
the state, 64 of the chunk, and some factors: below 400 roundings of 2^-24 one after the other,
2.4e-5 of size; decays and bf16 terms (two of a state or of q . k, 2^-16 of each) are 4 of
2^-16 at most: together 1e-4 of size with bf16 inputs, 3e-5 with fp32.  bf16 outputs add half a
step, 2^-8 of the entry.  fp32 results of bf16 inputs (states, dg, dS0) are formed of three
terms: 3e-5.  (That is the worst case; a norm of the errors, which add up at random, is held to
2e-6 of the result's beside it: 2^-24 times the square root of 400, with some room, for what is
not a difference, and to 1e-5 for dg.)"""

import numpy as np
import pytest
import torch

import paper_2606_06034_amd as G
from oracle import linear

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, t=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda().to(t)


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def make(lens, Hk, Hv, dk, dv, dt, per_token, state, seed, packed):
    """Device tensors of sequences of the given lengths, equal ones or packed."""
    rng = np.random.default_rng(seed)
    n = sum(lens)

    def unit(*s):
        z = rng.normal(size=s)
        return z / np.linalg.norm(z, axis=-1, keepdims=True)

    lead = (1, n) if packed else (len(lens), lens[0])
    x = dict(Q=unit(n, Hk, dk), K=unit(n, Hk, dk), V=rng.normal(size=(n, Hv, dv)),
             dO=rng.normal(size=(n, Hv, dv)))
    x = {k: dev(v.reshape(lead + v.shape[1:]), DT[dt]) for k, v in x.items()}
    if per_token:  # slow and fast heads
        z = rng.normal(size=(n, Hv)) + np.where(np.arange(Hv) % 2, -4, 3)
        x["g"] = dev(-np.log1p(np.exp(z)).reshape(lead + (Hv,)))
    else:
        x["g"] = dev(-np.exp2(-6 * np.arange(1, Hv + 1) / Hv))
    s = (len(lens), Hv, dk, dv)
    x["S0"], x["dS"] = (dev(rng.normal(size=s)) if state else None for _ in range(2))
    x["cu"] = dev(np.concatenate([[0], np.cumsum(lens)]), torch.int32) if packed else None
    return x


def sequences(x, lens):
    """numpy arguments of the oracle, sequence by sequence"""
    at = 0
    for s, n in enumerate(lens):
        def take(k):
            t = f64(x[k])
            return t if t.ndim == 1 else t.reshape((-1,) + t.shape[2:])[at:at + n]
        yield s, slice(at, at + n), [take(k) for k in ("Q", "K", "V", "g")], take("dO")
        at += n


def flat(t):
    return f64(t).reshape((-1,) + tuple(t.shape[2:]))


def near(got, ref, size, c, bf, what):
    assert got.shape == ref.shape and np.isfinite(got).all(), what
    lim = c * size + (np.abs(ref) * 2.0 ** -8 if bf else 0.0) + 1e-37
    worst = (np.abs(got - ref) / lim).max() if got.size else 0.0
    assert worst <= 1, (what, worst)


def in_norm(got, ref, c, what):
    n = np.linalg.norm(ref)
    assert np.linalg.norm(got - ref) <= c * n + 1e-30, (what, np.linalg.norm(got - ref) / n)


CASES = [  # lens, Hk, Hv, dk, dv, per token, states, packed
    ([1], 1, 1, 64, 64, False, False, False),
    ([2, 2, 2], 2, 2, 128, 128, True, True, False),
    ([15], 1, 3, 128, 64, True, False, False),
    ([64, 64], 2, 4, 64, 128, False, True, False),
    ([65], 1, 1, 128, 128, True, True, False),
    ([100, 100, 100], 1, 2, 64, 64, True, False, False),
    ([255], 1, 2, 128, 128, False, True, False),
    ([400], 1, 1, 128, 128, True, True, False),          # two segments, the last one short
    ([300], 2, 6, 64, 64, False, False, False),          # three value heads to a key head
    ([1, 1, 1], 1, 2, 64, 64, True, True, True),
    ([3, 0, 64, 1, 130, 0, 63], 1, 2, 64, 128, True, True, True),
    ([0, 350, 17, 40], 1, 2, 128, 128, True, True, True),  # segments, with one inside a sequence
    ([70, 290], 2, 2, 64, 64, False, False, True),
]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[0])) + f"_{c[2]}x{c[3]}")
def test_forward_recurrent_and_backward(case, dt):
    lens, Hk, Hv, dk, dv, per_token, state, packed = case
    x = make(lens, Hk, Hv, dk, dv, dt, per_token, state, len(lens) * 131 + sum(lens), packed)
    bf = dt == "bf16"
    c, scale = 1e-4 if bf else 3e-5, 0.3
    print(case, dt, flush=True)
    O, S = G.gdn_linear_forward(x["Q"], x["K"], x["V"], x["g"], S0=x["S0"], scale=scale,
                                cu_seqlens=x["cu"])
    Or, Sr = G.gdn_linear_recurrent(x["Q"], x["K"], x["V"], x["g"], S0=x["S0"], scale=scale,
                                    cu_seqlens=x["cu"])
    dQ, dK, dV, dg, d0 = G.gdn_linear_backward(x["Q"], x["K"], x["V"], x["g"], x["dO"], S0=x["S0"],
                                               dS_final=x["dS"], scale=scale, want_dS0=True,
                                               cu_seqlens=x["cu"])
    torch.cuda.synchronize()
    assert dg.shape == x["g"].shape
    total, total_size, refs = 0.0, 0.0, []
    for s, rows, a, dO in sequences(x, lens):
        S0, dS = (None if x[k] is None else f64(x[k])[s] for k in ("S0", "dS"))
        if rows.start == rows.stop:
            for got, want in ((S, S0), (Sr, S0), (d0, dS)):
                want = np.zeros((Hv, dk, dv)) if want is None else want
                assert np.array_equal(f64(got)[s], want)
            continue
        ref, size = linear.linear(*a, S0, scale), linear.linear_sizes(*a, S0=S0, scale=scale)
        for o, st, k in ((O, S, "chunked"), (Or, Sr, "recurrent")):
            near(flat(o)[rows], ref[0], size[0], c, bf, k + " O")
            near(f64(st)[s], ref[1], size[1], 3e-5, False, k + " S")
            in_norm(f64(st)[s], ref[1], 2e-6, k + " S")
        ref = linear.linear_grad(*a, dO, S0, dS, scale)
        size = linear.linear_sizes(*a, dO, S0, dS, scale)
        near(flat(dQ)[rows], ref[0], size[0], c, bf, "dQ")
        near(flat(dK)[rows], ref[1], size[1], c, bf, "dK")
        near(flat(dV)[rows], ref[2], size[2], c, bf, "dV")
        near(f64(d0)[s], ref[4], size[4], 3e-5, False, "dS0")
        in_norm(f64(d0)[s], ref[4], 2e-6, "dS0")
        if per_token:
            near(flat(dg)[rows], ref[3], size[3], 3e-5, False, "dg")
            refs.append((flat(dg)[rows], ref[3]))
        else:
            total, total_size = total + ref[3], total_size + size[3].sum(0)
    if per_token:
        in_norm(*(np.concatenate([r[i] for r in refs]) for i in (0, 1)), 1e-5, "dg")
    else:
        near(f64(dg), total, total_size, 3e-5, False, "dg")
        in_norm(f64(dg), total, 1e-5, "dg")


def test_a_long_sequence_in_many_segments():
    """8 heads of 4096 tokens, against the recurrent form on the GPU (fp32 throughout): both
    within 1e-4 of size, taken as the forward pass of the magnitudes."""
    for dt, per_token in (("bf16", True), ("f32", False)):
        x = make([4096], 2, 8, 128, 128, dt, per_token, True, 5, False)
        a = [x[k] for k in ("Q", "K", "V", "g")]
        O, S = G.gdn_linear_forward(*a, S0=x["S0"])
        Or, Sr = G.gdn_linear_recurrent(*a, S0=x["S0"])
        size, ssize = G.gdn_linear_recurrent(*(t.abs() for t in a[:3]), x["g"], S0=x["S0"].abs())
        bf = dt == "bf16"
        near(f64(O), f64(Or), f64(size), 2e-4, False, "O") if not bf else \
            near(f64(O), f64(Or), 1.01 * f64(size), 2e-4 + 2.0 ** -7, False, "O")
        near(f64(S), f64(Sr), f64(ssize), 6e-5, False, "S")


def test_states_in_place_and_without():
    x = make([90, 90], 2, 2, 64, 64, "bf16", True, True, 7, False)
    a = [x[k] for k in ("Q", "K", "V", "g")]
    O, S = G.gdn_linear_forward(*a, S0=x["S0"])
    S0 = x["S0"].clone()
    O2, S2 = G.gdn_linear_forward(*a, S0=S0, S_final=S0)
    assert S2 is S0 and torch.equal(O, O2) and torch.equal(S, S0)
    O3, none = G.gdn_linear_forward(*a, S0=x["S0"], want_state=False)
    assert none is None and torch.equal(O, O3)
    # a prompt in two calls, the state handed on; then in segments
    for n, dt, tol in ((40, "f32", 3e-5), (300, "f32", 3e-5)):
        x = make([512], 1, 2, 64, 64, dt, True, True, 8, False)
        a = [x[k] for k in ("Q", "K", "V", "g")]
        O, S = G.gdn_linear_forward(*a, S0=x["S0"])
        st = x["S0"].clone()
        o1, _ = G.gdn_linear_forward(*(t[:, :n].contiguous() for t in a), S0=st, S_final=st)
        o2, _ = G.gdn_linear_forward(*(t[:, n:].contiguous() for t in a), S0=st, S_final=st)
        size, ss = G.gdn_linear_recurrent(*(t.abs() for t in a[:3]), x["g"], S0=x["S0"].abs())
        near(f64(torch.cat([o1, o2], 1)), f64(O), f64(size), 2 * tol, False, "O")
        near(f64(st), f64(S), f64(ss), 2 * tol, False, "S")


def test_without_tokens():
    x = make([4, 4], 1, 2, 64, 128, "bf16", True, True, 9, False)
    e = [x[k][:, :0].contiguous() for k in ("Q", "K", "V", "g", "dO")]
    O, S = G.gdn_linear_forward(*e[:4], S0=x["S0"])
    assert O.shape == (2, 0, 2, 128) and torch.equal(S, x["S0"])
    _, S = G.gdn_linear_forward(*e[:4])
    assert (S == 0).all()
    dQ, dK, dV, dg, d0 = G.gdn_linear_backward(*e, dS_final=x["dS"], want_dS0=True)
    assert dQ.shape == (2, 0, 1, 64) and dg.shape == (2, 0, 2) and torch.equal(d0, x["dS"])
    head = torch.full((2,), -0.5, device="cuda")
    dg = G.gdn_linear_backward(*e[:3], head, e[4])[3]
    assert dg.shape == (2,) and (dg == 0).all()
    none = [t[:0] for t in e[:3]]  # no sequences
    assert (G.gdn_linear_backward(*none, head, e[4][:0])[3] == 0).all()
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")  # packed, all of them empty
    e = [t[:1] for t in e]
    for g in (e[3], head):
        O, S = G.gdn_linear_forward(*e[:3], g, S0=x["S0"], cu_seqlens=cu)
        assert torch.equal(S, x["S0"])
        got = G.gdn_linear_backward(*e[:3], g, e[4], dS_final=x["dS"], want_dS0=True, cu_seqlens=cu)
        assert torch.equal(got[4], x["dS"]) and (got[3] == 0).all()


@pytest.mark.parametrize("per_token", [True, False])
def test_offsets_out_of_range(per_token):
    """A sequence with a bad offset is empty and leaves the others alone; tokens of no
    sequence are left as they were."""
    lens = [40, 70, 30, 100]
    x = make(lens, 1, 2, 64, 64, "bf16", per_token, True, 11, True)
    a = [x[k] for k in ("Q", "K", "V", "g")]
    n = sum(lens)
    good = torch.tensor([0, 40, 110, 140, 240], dtype=torch.int32, device="cuda")
    want = G.gdn_linear_forward(*a, S0=x["S0"], cu_seqlens=good)
    back = G.gdn_linear_backward(*a, x["dO"], S0=x["S0"], dS_final=x["dS"], want_dS0=True,
                                 cu_seqlens=good)
    rec = G.gdn_linear_recurrent(*a, S0=x["S0"], cu_seqlens=good)
    for offsets, whole in (([0, 40, n + 1, 140, 240], [0, 3]), ([0, 40, -5, 140, 240], [0, 3]),
                           ([-1, 40, 110, 140, 240], [1, 2, 3]),
                           ([0, 40, 110, 140, 2 ** 31 - 1], [0, 1, 2])):
        bad = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        O = torch.full_like(x["V"], 7.0)
        _, S = G.gdn_linear_forward(*a, S0=x["S0"], cu_seqlens=bad, O=O)
        Or = torch.full_like(x["V"], 7.0)
        _, Sr = G.gdn_linear_recurrent(*a, S0=x["S0"], cu_seqlens=bad, O=Or)
        out = [torch.full_like(t, 7.0) for t in back[:3]] + [torch.full_like(back[3], 7.0), None]
        got = G.gdn_linear_backward(*a, x["dO"], S0=x["S0"], dS_final=x["dS"], want_dS0=True,
                                    cu_seqlens=bad, out=out)
        rows = torch.zeros(n, dtype=torch.bool, device="cuda")
        for s in range(4):
            if s in whole:
                rows[good[s]:good[s + 1]] = True
                assert torch.equal(S[s], want[1][s]) and torch.equal(Sr[s], rec[1][s])
                assert torch.equal(got[4][s], back[4][s])
            else:
                assert torch.equal(S[s], x["S0"][s]) and torch.equal(Sr[s], x["S0"][s])
                assert torch.equal(got[4][s], x["dS"][s])
        pairs = [(O, want[0]), (Or, rec[0])] + list(zip(got[:3], back[:3]))
        if per_token:
            pairs.append((got[3], back[3]))
        for t, w in pairs:
            assert torch.equal(t[0, rows], w[0, rows]) and (t[0, ~rows] == 7).all()


def test_forgetting_all():
    """A log-decay of -inf starts the state again, in whole and for the gradients."""
    n, cut = 150, 77
    x = make([n], 1, 2, 64, 64, "f32", True, True, 12, False)
    x["g"][:, cut] = -float("inf")
    a = [x[k] for k in ("Q", "K", "V", "g")]
    O, S = G.gdn_linear_forward(*a, S0=x["S0"])
    back = G.gdn_linear_backward(*a, x["dO"], S0=x["S0"], want_dS0=True)
    rest = [t[:, cut:].clone() for t in a]
    Or, Sr = G.gdn_linear_forward(*rest)
    head = [t[:, :cut].contiguous() for t in a]
    Oh, _ = G.gdn_linear_forward(*head, S0=x["S0"])
    bh = G.gdn_linear_backward(*head, x["dO"][:, :cut].contiguous(), S0=x["S0"], want_dS0=True)
    br = G.gdn_linear_backward(*rest, x["dO"][:, cut:].clone())
    size = G.gdn_linear_recurrent(*(t.abs() for t in a[:3]), x["g"], S0=x["S0"].abs())[0]
    near(f64(O), f64(torch.cat([Oh, Or], 1)), f64(size), 6e-5, False, "O")
    near(f64(S), f64(Sr), f64(Sr.abs().amax()), 6e-5, False, "S")
    for i in range(4):
        ref = torch.cat([bh[i], br[i]], 1)
        near(f64(back[i]), f64(ref), f64(ref.abs().amax()) * n, 6e-5, False, i)
    near(f64(back[4]), f64(bh[4]), f64(bh[4].abs().amax()) * n, 6e-5, False, "dS0")
    o, s = G.gdn_linear_recurrent(*a, S0=x["S0"])
    near(f64(o), f64(O), f64(size), 6e-5, False, "recurrent")


def test_a_nan_reaches_no_other_sequence_and_no_other_head():
    lens = [100, 30, 200]
    x = make(lens, 2, 4, 64, 64, "bf16", True, True, 13, True)
    names = ("Q", "K", "V", "g", "dO")
    call = lambda y: (*G.gdn_linear_forward(*(y[k] for k in names[:4]), S0=y["S0"],  # noqa: E731
                                            cu_seqlens=y["cu"]),
                      *G.gdn_linear_backward(*(y[k] for k in names), S0=y["S0"], dS_final=y["dS"],
                                             want_dS0=True, cu_seqlens=y["cu"]))
    want = call(x)
    for k in names:
        y = dict(x)
        y[k] = x[k].clone()
        y[k][0, 110, 0] = float("nan")  # the second sequence, the first head
        got = call(y)
        own = slice(100, 130)
        reached = False
        for i, (t, w) in enumerate(zip(got, want)):
            if i in (1, 6):  # states
                keep = torch.ones(t.shape[:2], dtype=torch.bool, device="cuda")
                keep[1, :2] = False
            else:
                keep = torch.ones(t.shape[1:3], dtype=torch.bool, device="cuda")
                keep[own, :1 if i in (2, 3) else 2] = False
                t, w = t[0], w[0]
            assert torch.equal(t[keep], w[keep]), (k, i)
            reached |= not torch.isfinite(t.float()).all()
        assert reached, k


def test_pools_of_states():
    nseq, n = 5, 9
    x = make([3] * nseq, 2, 4, 128, 64, "bf16", True, False, 14, False)
    a = [x[k] for k in ("Q", "K", "V", "g")]
    pool = torch.randn(n, 4, 128, 64, device="cuda")
    slots = torch.tensor([7, -1, 0, n, 4], dtype=torch.int32, device="cuda")
    own = slots.clamp(0, n - 1).long()
    Or, Sr = G.gdn_linear_recurrent(*a, S0=pool[own].contiguous())
    before = pool.clone()
    O, S = G.gdn_linear_recurrent(*a, S0=pool, S_final=pool, slots=slots)
    assert S is pool
    for s in range(nseq):
        if s in (1, 3):  # padded
            assert (O[s] == 0).all()
        else:
            assert torch.equal(O[s], Or[s]) and torch.equal(pool[own[s]], Sr[s])
    rest = [i for i in range(n) if i not in (7, 0, 4)]
    assert torch.equal(pool[rest], before[rest])


def test_the_same_every_time_on_another_stream_and_in_a_graph():
    for packed, lens, per_token in ((False, [600], True), (True, [100, 1, 500], False)):
        x = make(lens, 2, 4, 128, 128, "bf16", per_token, True, 15, packed)
        a = [x[k] for k in ("Q", "K", "V", "g")]

        def call(**kw):
            f = G.gdn_linear_forward(*a, S0=x["S0"], cu_seqlens=x["cu"], **kw)
            b = G.gdn_linear_backward(*a, x["dO"], S0=x["S0"], dS_final=x["dS"], want_dS0=True,
                                      cu_seqlens=x["cu"], **kw)
            r = G.gdn_linear_recurrent(*a, S0=x["S0"], cu_seqlens=x["cu"], **kw)
            return f + b + r

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
            x["V"].normal_()
            x["S0"].normal_()
            eager = call()
            for t in got:
                t.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, eager)), i


def test_two_graphs_with_one_workspace():
    """Calls that a stream runs one after the other may share a workspace."""
    x = make([700], 1, 2, 64, 64, "bf16", True, True, 16, False)
    y = make([700], 1, 2, 64, 64, "bf16", True, True, 17, False)
    ws = torch.empty(G.gdn_linear_backward_workspace(1, 700, 1, 2, 64, 64), dtype=torch.uint8,
                     device="cuda")
    call = lambda t, **kw: G.gdn_linear_backward(  # noqa: E731
        *(t[k] for k in ("Q", "K", "V", "g", "dO")), S0=t["S0"], want_dS0=True, **kw)
    want = [call(x), call(y)]
    torch.cuda.synchronize()
    graphs, got = [], []
    for t in (x, y):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(call(t, workspace=ws))
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for i in (0, 1) for p, q in zip(got[i], want[i]))


def test_some_gradients_alone():
    x = make([200], 1, 3, 64, 64, "bf16", True, True, 18, False)
    a = [x[k] for k in ("Q", "K", "V", "g", "dO")]
    want = G.gdn_linear_backward(*a, S0=x["S0"], want_dS0=True)
    dQ, dK, dV, dg, d0 = G.gdn_linear_backward(*a, S0=x["S0"], want_dg=False)
    assert dg is None and d0 is None
    for p, q in zip((dQ, dK, dV), want):
        assert np.allclose(f64(p), f64(q), rtol=2.0 ** -7, atol=1e-4 * float(q.abs().max()))
    # the head's decay as a tensor of the tokens': the gradients' sum
    head = torch.tensor([-0.1, -0.7, -0.01], device="cuda")
    one = G.gdn_linear_backward(*a[:3], head, a[4], S0=x["S0"])
    each = G.gdn_linear_backward(*a[:3], head.expand(1, 200, 3).contiguous(), a[4], S0=x["S0"])
    for p, q in zip(one[:3], each[:3]):
        assert np.allclose(f64(p), f64(q), rtol=2.0 ** -7, atol=1e-4 * float(q.abs().max()))
    assert np.allclose(f64(one[3]), f64(each[3]).sum((0, 1)), rtol=1e-4,
                       atol=1e-5 * float(each[3].abs().sum()))


def test_the_decay_of_one_token():
    """Its gradient is e^g <S0, dS> where dO is 0: a sum of dk dv products that cancel to a
    hundredth, taken in 64 bits; e^g, its product and the results' sums are 8 roundings at most."""
    x = make([1, 1], 4, 32, 128, 128, "bf16", True, True, 19, False)
    x["dO"].zero_()
    for odd in (False, True):  # groups of eight, and of one
        a = [x[k] for k in ("Q", "K", "V", "g", "dO")]
        S0, dS = x["S0"], x["dS"]
        if odd:
            a[0], a[1] = (t.repeat_interleave(8, 2).contiguous() for t in a[:2])
        dg = G.gdn_linear_backward(*a, S0=S0, dS_final=dS)[3]
        ref = np.exp(f64(x["g"])) * (f64(S0) * f64(dS)).sum((2, 3))[:, None]
        assert (np.abs(f64(dg) - ref) <= 8 * 2.0 ** -24 * np.abs(ref)).all()

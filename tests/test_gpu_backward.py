"""The chunk-wise backward pass on the GPU against the fp64 oracle (reverse
accumulation token by token).

Tolerances.  Everything is formed in fp32 from products of at most 128 terms
and two recurrences that do not amplify (unit keys, beta in (0, 1)): a chunk
adds a few hundred roundings of 2^-24 at the size of the largest entry, at
random signs some tens of them, 2e-5 of the array's largest entry (of 1 where
that is smaller: dbeta and dg are sums of terms of that size that may cancel).
bf16 outputs add their own rounding, 2^-8 of the entry."""

import numpy as np
import pytest
import torch

import paper_2606_06034_amd as G
from oracle import layer

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("dQ", "dK", "dV", "dbeta", "dg", "dS0")


def make(lens, Hk, Hv, dk, dv, C, dt, seed, S0=True, dS=True, slow=True):
    rng = np.random.default_rng(seed)
    n = sum(lens)

    def dev(a, t=torch.float32):
        return torch.from_numpy(np.ascontiguousarray(a).astype(np.float32)).cuda().to(t)

    def unit(*s):
        z = rng.normal(size=s)
        return z / np.linalg.norm(z, axis=-1, keepdims=True)

    inc = rng.normal(size=(n, Hv)) + 1
    if slow:
        inc[:, ::2] -= 5  # heads that forget slowly
    inc = -np.log1p(np.exp(inc))
    g, t = np.zeros((n, Hv)), 0
    for m in lens:
        for a in range(0, m, C):
            e = min(a + C, m)
            g[t + a:t + e] = np.cumsum(inc[t + a:t + e], 0)
        t += m
    return dict(Q=dev(unit(n, Hk, dk), DT[dt]), K=dev(unit(n, Hk, dk), DT[dt]),
                V=dev(rng.normal(size=(n, Hv, dv)), DT[dt]),
                beta=dev(1 / (1 + np.exp(-rng.normal(size=(n, Hv))))), g=dev(g),
                dO=dev(rng.normal(size=(n, Hv, dv)), DT[dt]),
                S0=dev(rng.normal(size=(len(lens), Hv, dk, dv))) if S0 else None,
                dS=dev(rng.normal(size=(len(lens), Hv, dk, dv))) if dS else None)


def oracle(x, lens, C, scale):
    f = {k: None if v is None else v.double().cpu().numpy() for k, v in x.items()}
    parts, t = [], 0
    for s, m in enumerate(lens):
        w = slice(t, t + m)
        d = layer.token_decay(f["g"][w], C)
        dq, dk, dv, db, dl, ds = layer.recurrent_grad(
            f["Q"][w], f["K"][w], f["V"][w], f["beta"][w], d, f["dO"][w],
            None if f["S0"] is None else f["S0"][s], None if f["dS"] is None else f["dS"][s],
            scale)
        dg = dl.copy()  # token t's decay is g_t - g_{t-1} inside a chunk
        inside = np.arange(1, m)[np.arange(1, m) % C != 0] if m else np.arange(0)
        dg[inside - 1] -= dl[inside]
        parts.append((dq, dk, dv, db, dg, ds[None]))
        t += m
    return [np.concatenate(p) for p in zip(*parts)]


def compare(got, ref, dt):
    for name, a, r in zip(NAMES, got, ref):
        if a is None:
            continue
        a = a.double().cpu().numpy().reshape(r.shape)
        lim = 2e-5 * max(1.0, np.abs(r).max() if r.size else 0)
        if dt == "bf16" and name in ("dQ", "dK", "dV"):
            lim = lim + np.abs(r) * 2.0 ** -8
        assert np.isfinite(a).all(), name
        assert (np.abs(a - r) <= lim).all(), (name, np.abs(a - r).max())


def run(x, lens, C, scale, packed, want_dS0=True):
    lead = (1, -1) if packed else (len(lens), lens[0])
    y = {k: None if v is None else (v if k in ("S0", "dS") else
                                    v.reshape(lead + tuple(v.shape[1:])) if v.numel() or not packed
                                    else v[None]) for k, v in x.items()}
    args = [y[k] for k in ("Q", "K", "V", "beta", "g", "dO")]
    kw = dict(S0=x["S0"], dS_final=x["dS"], scale=scale, want_dS0=want_dS0)
    if packed:
        return G.gdn_chunk_backward_varlen(
            *args, G.gdn_varlen_tables(np.concatenate([[0], np.cumsum(lens)]), C), C, **kw)
    return G.gdn_chunk_backward(*args, C, **kw)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv,C", [
    (1, 1, 1, 1, 128, 128, 64), (2, 64, 1, 2, 128, 128, 64), (1, 65, 2, 2, 64, 64, 64),
    (1, 200, 1, 3, 64, 128, 64), (2, 127, 2, 4, 128, 64, 32), (1, 150, 1, 2, 128, 128, 16),
    (3, 17, 1, 1, 64, 64, 16), (1, 320, 1, 1, 128, 128, 64)])
def test_equal_lengths(dt, B, L, Hk, Hv, dk, dv, C):
    x = make([L] * B, Hk, Hv, dk, dv, C, dt, L + dk)
    compare(run(x, [L] * B, C, 0.3, False), oracle(x, [L] * B, C, 0.3), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("C", [64, 32, 16])
def test_packed(dt, C):
    lens = [5, 0, 64, 1, 130, 63, 0, 33]
    x = make(lens, 2, 4, 128, 64, C, dt, C)
    compare(run(x, lens, C, 64 ** -0.5, True), oracle(x, lens, C, 64 ** -0.5), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv,packed", [
    (3, 130, 11, 22, 128, 128, False), (5, 97, 9, 27, 64, 64, False),
    (2, 200, 17, 34, 64, 128, False), (140, 80, 3, 6, 128, 64, True)])
def test_many_slices(dt, B, L, Hk, Hv, dk, dv, packed):
    """Past 512 slices of 16 value columns (packed sequences: past six times
    that many) the walks run another way: sampled sequences and heads."""
    lens = [1 + s * (L - 1) // (B - 1) for s in range(B)] if packed else [L] * B
    assert B * Hv * dv // 16 > (3072 if packed else 512)
    x = make(lens, Hk, Hv, dk, dv, 64, dt, dv)
    got = run(x, lens, 64, 0.3, packed)
    r = Hv // Hk
    for s, hk in [(0, 0), (B - 1, Hk - 1), (B // 2, Hk // 2)]:
        t = sum(lens[:s])
        w, hv = slice(t, t + lens[s]), slice(hk * r, (hk + 1) * r)
        sub = {k: (v[s:s + 1, hv] if k in ("S0", "dS") else
                   v[w, hk:hk + 1] if k in ("Q", "K") else v[w, hv]) for k, v in x.items()}
        flat = [a.reshape((-1,) + tuple(a.shape[2:])) for a in got[:5]]
        part = [a[w, hk:hk + 1] if i < 2 else a[w, hv] for i, a in enumerate(flat)]
        compare(part + [got[5][s:s + 1, hv]], oracle(sub, [lens[s]], 64, 0.3), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv,C,packed", [
    (3, 450, 12, 24, 128, 128, 64, False), (2, 321, 22, 22, 64, 64, 16, False),
    (9, 129, 10, 30, 128, 64, 32, False), (1, 1100, 15, 15, 64, 128, 64, False),
    (90, 80, 3, 6, 128, 128, 64, True)])
def test_many_tiles(dt, B, L, Hk, Hv, dk, dv, C, packed):
    """Past 256 chunks by key heads the per-chunk gradients run another way: sampled
    sequences and key heads, among them the last."""
    lens = [1 + s * (L - 1) // (B - 1) for s in range(B)] if packed else [L] * B
    assert sum((m + 63) // 64 for m in lens) * Hk > 256
    x = make(lens, Hk, Hv, dk, dv, C, dt, L + dv)
    got = run(x, lens, C, 0.3, packed)
    r = Hv // Hk
    for s, hk in {(0, 0), (B - 1, Hk - 1), (B // 2, Hk // 2)}:
        t = sum(lens[:s])
        w, hv = slice(t, t + lens[s]), slice(hk * r, (hk + 1) * r)
        sub = {k: (v[s:s + 1, hv] if k in ("S0", "dS") else
                   v[w, hk:hk + 1] if k in ("Q", "K") else v[w, hv]) for k, v in x.items()}
        flat = [a.reshape((-1,) + tuple(a.shape[2:])) for a in got[:5]]
        part = [a[w, hk:hk + 1] if i < 2 else a[w, hv] for i, a in enumerate(flat)]
        compare(part + [got[5][s:s + 1, hv]], oracle(sub, [lens[s]], C, 0.3), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv,Hk,Hv", [(128, 128, 3, 9), (64, 128, 8, 8), (128, 64, 5, 20)])
def test_long_and_short_packed(dt, dk, dv, Hk, Hv):
    """Long and short packed sequences are walked in different ways by one launch."""
    lens = [5, 700, 0, 64, 321, 1, 130, 65]
    longest = sum(lens) * Hv * (dv // 16) // 30000
    assert 1 <= longest < 11
    x = make(lens, Hk, Hv, dk, dv, 64, dt, dk + dv)
    compare(run(x, lens, 64, 0.2, True), oracle(x, lens, 64, 0.2), dt)


def test_packed_is_each_sequence_alone_bit_for_bit():
    lens = [70, 3, 129]
    x = make(lens, 1, 2, 64, 64, 64, "bf16", 1)
    both = run(x, lens, 64, 0.5, True)
    t = 0
    for s, m in enumerate(lens):
        one = {k: (v[s:s + 1] if k in ("S0", "dS") else v[t:t + m]).clone()  # (aligned)
               for k, v in x.items()}
        for name, a, b in zip(NAMES, both, run(one, [m], 64, 0.5, False)):
            a = a[s:s + 1] if name == "dS0" else a[:, t:t + m]
            assert torch.equal(a, b), (name, s)
        t += m


def test_optional_states():
    for S0, dS in [(False, False), (True, False), (False, True)]:
        x = make([90], 1, 2, 64, 64, 64, "f32", 2, S0=S0, dS=dS)
        got = run(x, [90], 64, 0.5, False, want_dS0=S0)
        assert (got[5] is None) == (not S0)
        compare(got, oracle(x, [90], 64, 0.5), "f32")


def test_no_tokens_hands_the_state_s_gradient_through():
    x = make([0, 0], 1, 2, 64, 64, 64, "f32", 3)
    assert torch.equal(run(x, [0, 0], 64, 1.0, False)[5], x["dS"])
    assert torch.equal(run(x, [0, 0], 64, 1.0, True)[5], x["dS"])
    x["dS"] = None
    assert (run(x, [0, 0], 64, 1.0, False)[5] == 0).all()


def test_offsets_out_of_range_are_empty_sequences():
    x = make([60, 40], 1, 1, 64, 64, 64, "f32", 4)
    lens, T = [60, 40], 100
    y = [x[k][None] for k in ("Q", "K", "V", "beta", "g", "dO")]
    cu = torch.tensor([0, 60, 500], dtype=torch.int32, device="cuda")
    out = [torch.full_like(t, 7.0) for t in (y[0], y[1], y[2], y[3], y[4])] + [None]
    got = G.gdn_chunk_backward_varlen(*y, (cu, None, 0), 64, S0=x["S0"], dS_final=x["dS"],
                                      want_dS0=True, out=out)
    assert torch.equal(got[5][1], x["dS"][1])
    for a in got[:5]:
        assert (a[:, 60:] == 7).all() and torch.isfinite(a).all()
    ref = oracle(x, lens, 64, 64 ** -0.5)
    compare([a[:, :60] for a in got[:5]] + [got[5][:1]],
            [r[:60] for r in ref[:5]] + [ref[5][:1]], "f32")


def test_beta_zero_and_one_and_the_fastest_forgetting():
    x = make([100], 1, 2, 64, 64, 64, "f32", 5)
    x["beta"][10:20] = 0
    x["beta"][30:40] = 1
    inc = torch.from_numpy(layer.token_decay(x["g"].double().cpu().numpy(), 64)).cuda()
    inc[50] = -200.0  # e^-200 is 0 in fp32: the state is gone
    g = inc.clone()
    g[:64], g[64:] = inc[:64].cumsum(0), inc[64:].cumsum(0)
    x["g"] = g.float()
    # the sums past -200 round to 2^-17 there, and so does the decay they differ by
    got, ref = run(x, [100], 64, 0.5, False), oracle(x, [100], 64, 0.5)
    compare(got, ref, "f32")


def test_a_nan_stays_in_its_head_and_sequence():
    x = make([64, 64], 2, 4, 64, 64, 64, "bf16", 6)
    clean = run(x, [64, 64], 64, 0.5, False)
    x["V"][70, 1, 3] = float("nan")  # sequence 1, value head 1 (key head 0)
    got = run(x, [64, 64], 64, 0.5, False)
    for name, a, b in zip(NAMES, got, clean):
        hit = torch.isnan(a)
        assert torch.equal(a[0], b[0]), name
        if name in ("dV", "dbeta", "dg"):
            assert torch.equal(a[1][:, 2:], b[1][:, 2:]) and torch.equal(a[1][:, 0], b[1][:, 0])
        elif name in ("dQ", "dK"):
            assert torch.equal(a[1][:, 1], b[1][:, 1])
        if name in ("dQ", "dK", "dbeta"):
            assert hit.any(), name


def test_the_gradient_is_the_forward_s_difference():
    """Along a random direction, by central differences of the fp32 recurrent
    form: a step h of 1e-2 leaves h^2 f'''/6 and 2^-24 |loss| / h, both below
    1e-3 of the slope's size here (|loss| ~ 50, slope ~ 50)."""
    lens, C = [80], 16
    x = make(lens, 1, 2, 64, 64, C, "f32", 7)
    got = run(x, lens, C, 0.5, False)
    gen = torch.Generator(device="cuda").manual_seed(1)
    keys = ("Q", "K", "V", "beta", "g", "S0")
    for k, grad in zip(keys, got):
        d = torch.randn(x[k].shape, generator=gen, device="cuda")
        d /= d.norm()
        slope = (grad.reshape(d.shape).double() * d).sum().item()
        loss = []
        for h in (1e-2, -1e-2):
            y = {n: x[n] + (h * d if n == k else 0) for n in keys}
            inc = y["g"].clone()
            inside = torch.arange(80, device="cuda") % C != 0
            inc[inside] -= y["g"][torch.nonzero(inside)[:, 0] - 1]
            O, S = G.gdn_recurrent_forward(y["Q"][None], y["K"][None], y["V"][None],
                                           y["beta"][None], inc[None], S0=y["S0"], scale=0.5)
            loss.append((O[0].double() * x["dO"]).sum().item() +
                        (S.double() * x["dS"]).sum().item())
        assert abs((loss[0] - loss[1]) / 2e-2 - slope) < 1e-2 * max(1.0, abs(slope)), k


def test_on_another_stream_in_a_graph_and_the_same_every_time():
    x = make([200, 7], 1, 2, 128, 128, 64, "bf16", 8)
    ref = run(x, [200, 7], 64, 0.5, True)
    y = [x[k][None] for k in ("Q", "K", "V", "beta", "g", "dO")]
    tables = G.gdn_varlen_tables([0, 200, 207], 64)
    out = [torch.zeros_like(a) for a in ref]
    ws = torch.empty(G.gdn_chunk_backward_workspace(2, 207, 2, 128, 128, True),
                     dtype=torch.uint8, device="cuda")

    def call():
        G.gdn_chunk_backward_varlen(*y, tables, 64, S0=x["S0"], dS_final=x["dS"], scale=0.5,
                                    want_dS0=True, out=out, workspace=ws)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        call()
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        for a in out:
            a.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref)), i


def check_heads(x, lens, C, got, dt, picks):
    """Sequences s and key heads hk of `picks` with their value heads, against the oracle."""
    r = x["V"].shape[1] // x["K"].shape[1]
    for s, hk in picks:
        t = sum(lens[:s])
        w, hv = slice(t, t + lens[s]), slice(hk * r, (hk + 1) * r)
        sub = {k: (v[s:s + 1, hv] if k in ("S0", "dS") else
                   v[w, hk:hk + 1] if k in ("Q", "K") else v[w, hv]) for k, v in x.items()}
        flat = [a.reshape((-1,) + tuple(a.shape[2:])) for a in got[:5]]
        part = [a[w, hk:hk + 1] if i < 2 else a[w, hv] for i, a in enumerate(flat)]
        compare(part + [got[5][s:s + 1, hv]], oracle(sub, [lens[s]], C, 0.3), dt)


@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv", [
    (4, 130, 4, 8, 128, 128), (3, 130, 11, 11, 128, 128), (16, 65, 4, 4, 64, 64),
    (5, 65, 13, 13, 64, 64), (8, 65, 4, 4, 128, 128), (16, 65, 8, 8, 64, 64),
    (1, 65, 129, 129, 64, 64)])
def test_either_side_of_the_launch_rules(B, L, Hk, Hv, dk, dv):
    """Equal lengths in bf16: up to 256 slices of 16 value columns are walked by teams, more
    by lone waves; up to 256 chunks by key heads have their gradients from workgroups of
    eight waves, more from ones of four.  Both sides of both, as near as whole heads come."""
    slices, tiles = B * Hv * dv // 16, B * ((L + 63) // 64) * Hk
    assert slices in (256, 260, 264, 512, 516) and tiles in (48, 64, 99, 128, 130, 256, 258)
    x = make([L] * B, Hk, Hv, dk, dv, 64, "bf16", B + Hv)
    got = run(x, [L] * B, 64, 0.3, False)
    check_heads(x, [L] * B, 64, got, "bf16", [(0, 0), (B - 1, Hk - 1), (B // 2, Hk // 2)])


@pytest.mark.parametrize("dk,dv,Hv", [(128, 128, 12), (64, 64, 24), (128, 64, 24)])
def test_packed_sequences_at_the_length_that_parts_the_walks(dk, dv, Hv):
    """In bf16, sequences of more than tokens * slices a sequence / 30000 chunks are walked by
    teams and the others by lone waves: exactly that many, one more, and their neighbours."""
    lens = [192, 193, 129, 256, 1, 229]
    assert sum(lens) * Hv * (dv // 16) // 30000 == 3
    assert sorted((m + 63) // 64 for m in lens) == [1, 3, 3, 4, 4, 4]
    x = make(lens, Hv // 3, Hv, dk, dv, 64, "bf16", dk + Hv)
    got = run(x, lens, 64, 0.3, True)
    check_heads(x, lens, 64, got, "bf16", [(s, s % (Hv // 3)) for s in range(len(lens))])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cu,valid", [
    ([0, 200, 9999, 300, 400], (0, 3)), ([0, 200, -1, 300, 400], (0, 3)),
    ([0, 200, 401, 300, 400], (0, 3)), ([-5, 200, 300, 400], (1, 2)),
    ([0, -7, 2 ** 31 - 1, -(2 ** 31), 200, 300, 400], (4, 5))])
def test_a_bad_offset_leaves_the_other_sequences(dt, cu, valid):
    """Wherever in the table it is.  What is not formed keeps the 7 it had, and what would be
    read without having been formed is NaN."""
    x = make([200, 100, 100], 2, 4, 64, 128, 64, dt, 9, S0=False, dS=False)
    n = len(cu) - 1
    gen = torch.Generator(device="cuda").manual_seed(2)
    x["S0"], x["dS"] = torch.randn(2, n, 4, 64, 128, generator=gen, device="cuda")
    y = [x[k][None] for k in ("Q", "K", "V", "beta", "g", "dO")]
    out = [torch.full_like(t, 7.0) for t in y[:5]] + [None]
    ws = torch.full((G.gdn_chunk_backward_workspace(n, 400, 4, 64, 128, True),), 255,
                    dtype=torch.uint8, device="cuda")
    offsets = torch.tensor(cu, dtype=torch.int32, device="cuda")
    got = G.gdn_chunk_backward_varlen(*y, (offsets, None, 0), 64, S0=x["S0"], dS_final=x["dS"],
                                      scale=0.3, want_dS0=True, out=out, workspace=ws)
    rest = torch.ones(400, dtype=torch.bool)
    for s in valid:
        w = slice(cu[s], cu[s + 1])
        rest[w] = False
        sub = {k: v[s:s + 1] if k in ("S0", "dS") else v[w] for k, v in x.items()}
        compare([a[:, w] for a in got[:5]] + [got[5][s:s + 1]],
                oracle(sub, [cu[s + 1] - cu[s]], 64, 0.3), dt)
    for a in got[:5]:
        assert (a[0][rest] == 7).all()
    for s in set(range(n)) - set(valid):
        assert torch.equal(got[5][s], x["dS"][s])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("name,value", [
    ("V", float("inf")), ("dO", -float("inf")), ("S0", float("inf")), ("dS", float("inf")),
    ("S0", float(np.finfo(np.float32).max)), ("Q", float("inf")), ("beta", float("nan"))])
def test_what_is_not_finite_stays_in_its_heads(dt, name, value):
    x = make([130, 130], 2, 4, 64, 64, 64, dt, 10)
    clean = run(x, [130, 130], 64, 0.5, False)
    if name in ("S0", "dS"):
        x[name][1, 1, 5, 7] = value  # sequence 1, value head 1 (key head 0)
    elif name == "beta":
        x[name][140, 1] = value
    else:
        x[name][140, 0 if name == "Q" else 1, 7] = value
    got = run(x, [130, 130], 64, 0.5, False)
    kept = (2, 3) if name == "Q" else (0, 2, 3)  # value heads that do not have it
    for n, a, b in zip(NAMES, got, clean):
        assert torch.equal(a[0], b[0]), n
        if n in ("dQ", "dK"):
            assert torch.equal(a[1][:, 1], b[1][:, 1]), n
        else:
            heads = a[1].movedim(-3, 0) if n == "dS0" else a[1].movedim(1, 0)
            was = b[1].movedim(-3, 0) if n == "dS0" else b[1].movedim(1, 0)
            assert all(torch.equal(heads[h], was[h]) for h in kept), n
    if value != np.finfo(np.float32).max:
        assert not all(torch.isfinite(a).all() for a in got)

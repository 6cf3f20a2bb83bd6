"""The C ABI of gdnlayer.h on the CPU: every declared symbol is exported and
bound, and bad arguments are refused before anything reaches the GPU (no call
here passes validation with work to do)."""

import ctypes
import os
import re

import pytest
import torch

import paper_2606_06034_amd as G

HDR = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                   "gdnlayer.h")
OK, NULL, SHAPE, PARAM, DTYPE, ALIGN, ALIAS, UNSUP, WS = 0, -1, -2, -3, -4, -5, -6, -8, -9
P = [k << 40 for k in range(1, 20)]  # aligned addresses far apart
L = G.lib


def test_exports_every_declared_symbol():
    names = sorted(set(re.findall(r"^int (gdn_\w+)\s*\(", open(HDR).read(), re.M)))
    assert names == sorted(G.layer_abi_symbols())
    for n in names:
        assert hasattr(L, n), n


def call(f, args, **change):
    a = dict(args, **change)
    return f(*a.values())


REC = dict(Q=P[0], K=P[1], V=P[2], beta=P[3], g=P[4], S0=P[5], O=P[6], S_final=P[7], slots=None,
           n_states=4, cu=None, nseq=4, T=2, Hk=2, Hv=4, dk=128, dv=64, scale=1.0, dtype=1,
           stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(nseq=-1), SHAPE), (dict(T=-1), SHAPE), (dict(n_states=-1), SHAPE),
    (dict(Hk=3), SHAPE), (dict(Hk=0), SHAPE), (dict(Hk=-2), SHAPE), (dict(dk=96), SHAPE),
    (dict(dv=32), SHAPE), (dict(n_states=3), SHAPE), (dict(nseq=1 << 30, n_states=1 << 30), SHAPE),
    (dict(dtype=2), DTYPE), (dict(Q=None), NULL), (dict(K=None), NULL), (dict(V=None), NULL),
    (dict(beta=None), NULL), (dict(g=None), NULL), (dict(O=None), NULL),
    (dict(Q=P[0] + 8), ALIGN), (dict(S0=P[5] + 4), ALIGN), (dict(slots=P[8] + 4), ALIGN),
    (dict(cu=P[8] + 4), ALIGN), (dict(O=P[0]), ALIAS), (dict(S_final=P[5] + 16), ALIAS),
    (dict(S_final=P[6]), ALIAS), (dict(O=P[5]), ALIAS),
    (dict(nseq=0), OK), (dict(Hk=0, Hv=0), OK),
])
def test_recurrent_refusals(change, code):
    assert call(L.gdn_recurrent_forward, REC, **change) == code


NF = dict(x=P[0], w=P[1], b=P[2], z=P[3], y=P[4], mean=P[5], rstd=P[6], rows=8, D=100, eps=1e-6,
          kind=0, dtype=1, wdt=0, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(D=0), SHAPE),
    (dict(D=65537), SHAPE), (dict(kind=2), PARAM), (dict(eps=-1.0), PARAM),
    (dict(eps=float("nan")), PARAM), (dict(dtype=2), DTYPE), (dict(wdt=2), DTYPE),
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(x=P[0] + 4), ALIGN),
    (dict(rstd=P[6] + 8), ALIGN), (dict(y=P[0]), ALIAS), (dict(mean=P[6]), ALIAS),
    (dict(rows=0), OK),
])
def test_norm_forward_refusals(change, code):
    assert call(L.gdn_norm_forward, NF, **change) == code


NB = dict(dy=P[0], x=P[1], w=P[2], b=P[3], z=P[4], mean=P[5], rstd=P[6], dx=P[7], dw=P[8],
          db=P[9], dz=P[10], ws=P[11], wsb=1 << 30, rows=8, D=100, kind=0, dtype=1, wdt=0,
          stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), SHAPE), (dict(D=0), SHAPE), (dict(kind=-1), PARAM), (dict(dtype=7), DTYPE),
    (dict(wdt=-1), DTYPE), (dict(dy=None), NULL), (dict(x=None), NULL), (dict(mean=None), NULL),
    (dict(rstd=None), NULL), (dict(dx=None), NULL), (dict(dz=None), NULL), (dict(ws=None), NULL),
    (dict(wsb=8 * 100 * 8 - 1), WS), (dict(dw=P[8] + 4), ALIGN), (dict(dx=P[0]), ALIAS),
    (dict(db=P[8]), ALIAS), (dict(dz=P[4]), ALIAS), (dict(ws=P[1]), ALIAS),
])
def test_norm_backward_refusals(change, code):
    assert call(L.gdn_norm_backward, NB, **change) == code


def test_norm_backward_workspace():
    n = ctypes.c_int64()
    assert L.gdn_norm_backward_workspace(10, 33, ctypes.byref(n)) == OK
    assert n.value == 10 * 33 * 8  # a row of sums a workgroup, dw and db
    assert L.gdn_norm_backward_workspace(10, 33, None) == NULL
    assert L.gdn_norm_backward_workspace(-1, 33, ctypes.byref(n)) == SHAPE
    assert G.gdn_norm_backward_workspace(0, 33) == 0


BWD = dict(Q=P[0], K=P[1], V=P[2], beta=P[3], g=P[4], dO=P[5], S0=P[6], dSf=P[7], dQ=P[8], dK=P[9],
           dV=P[10], dbeta=P[11], dg=P[12], dS0=P[13], ws=P[14], wsb=1 << 39, B=2, L=100, Hk=2,
           Hv=4, dk=128, dv=64, C=64, scale=1.0, dtype=1, stream=None)
BWD_BAD = [
    (dict(L=-1), SHAPE), (dict(Hk=3), SHAPE), (dict(Hk=0), SHAPE), (dict(dk=32), SHAPE),
    (dict(dv=256), SHAPE), (dict(C=48), SHAPE), (dict(C=0), SHAPE), (dict(C=128), UNSUP),
    (dict(dtype=2), DTYPE), (dict(Q=None), NULL), (dict(K=None), NULL), (dict(V=None), NULL),
    (dict(beta=None), NULL), (dict(g=None), NULL), (dict(dO=None), NULL), (dict(dQ=None), NULL),
    (dict(dK=None), NULL), (dict(dV=None), NULL), (dict(dbeta=None), NULL), (dict(dg=None), NULL),
    (dict(ws=None), NULL), (dict(wsb=1000), WS), (dict(dO=P[5] + 2), ALIGN),
    (dict(dS0=P[13] + 4), ALIGN), (dict(dQ=P[0]), ALIAS), (dict(dK=P[8]), ALIAS),
    (dict(dS0=P[7]), ALIAS), (dict(ws=P[2]), ALIAS), (dict(Hk=0, Hv=0), OK)]


@pytest.mark.parametrize("change,code", BWD_BAD + [
    (dict(B=-1), SHAPE), (dict(B=1 << 20, L=1 << 20), SHAPE), (dict(B=0), OK)])
def test_backward_refusals(change, code):
    assert call(L.gdn_chunk_backward, BWD, **change) == code


@pytest.mark.parametrize("change,code", BWD_BAD + [
    (dict(nseq=-1), SHAPE), (dict(nseq=0), OK), (dict(cu=None), NULL), (dict(cu=P[15] + 4), ALIGN),
    (dict(dg=P[15]), ALIAS)])
def test_packed_backward_refusals(change, code):
    a = {}
    for k, v in BWD.items():
        if k == "B":
            a.update(cu=P[15], nseq=3)
        else:
            a[k] = v
    assert call(L.gdn_chunk_backward_varlen, a, **change) == code


def packed_args(**change):
    a = {}
    for k, v in BWD.items():
        if k == "B":
            a.update(cu=P[15], nseq=3)
        else:
            a[k] = v
    return dict(a, **change)


@pytest.mark.parametrize("dv,most", [(64, 838856), (128, 419424)])
def test_packed_backward_s_largest_launch(dv, most):
    """Both kinds of walk, both ways, are workgroups of one launch of 512 work items each:
    2 heads (dv / 16 + dv / 64) of them, heads rounded up to eights, have to fit 2^32 - 1.
    What fits gets as far as the missing workspace, here."""
    args = packed_args(nseq=most // 8, Hk=8, Hv=8, dk=64, dv=dv, ws=None)
    assert call(L.gdn_chunk_backward_varlen, args) == NULL
    args.update(nseq=most // 8 + 1)
    assert call(L.gdn_chunk_backward_varlen, args) == SHAPE
    # fp32 and equal lengths launch fewer
    assert call(L.gdn_chunk_backward_varlen, args, dtype=0) == NULL
    assert call(L.gdn_chunk_backward, dict(BWD, B=most // 8 + 1, L=1, Hk=8, Hv=8, dk=64, dv=dv,
                                           ws=None)) == NULL


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype,d,most", [(0, 128, 131072), (0, 64, 262144), (1, 128, 262144)])
def test_backward_s_widest_rows(packed, dtype, d, most):
    """A chunk's rows are reached by 32-bit byte offsets from its first: the rows of all heads
    of the tokens of a chunk hold 2^32 bytes at most, of Q and K and of V."""
    f = L.gdn_chunk_backward_varlen if packed else L.gdn_chunk_backward
    base = packed_args(nseq=1) if packed else dict(BWD, B=1)
    for wide in ("keys", "values"):
        def code(heads, tokens):  # NULL: as far as the missing workspace
            dims = dict(dk=d, dv=64, Hk=heads) if wide == "keys" else dict(dk=64, dv=d, Hk=1)
            return call(f, dict(base, **dims, Hv=heads, L=tokens, dtype=dtype, ws=None))

        assert (code(most, 64), code(most, 1000)) == (NULL, NULL)
        assert (code(most + 1, 64), code(most + 1, 1000)) == (SHAPE, SHAPE)
        assert code(most + 1, 63) == NULL  # the rows that there are


def test_backward_workspace():
    tile = 4 * (6 * 768 + 5 * 64 + 2 * 64 * 128 + 2 * 128 * 128)
    assert G.gdn_chunk_backward_workspace(2, 100, 3, 128, 128) == 2 * 2 * 3 * tile
    assert G.gdn_chunk_backward_workspace(5, 100, 3, 128, 128, packed=True) == (1 + 5) * 3 * tile
    assert G.gdn_chunk_backward_workspace(2, 0, 3, 128, 128) == 0
    assert L.gdn_chunk_backward_workspace(2, 100, 3, 128, 128, 0, None) == NULL
    with pytest.raises(G.GdnError):
        G.gdn_chunk_backward_workspace(2, 100, 3, 96, 128)


def test_backward_workspace_of_the_longest_lengths():
    n = ctypes.c_int64(7)
    for L_, Hv, packed, code in [(2 ** 31 - 1, 1, 0, SHAPE), (2 ** 31 - 1, 1, 1, SHAPE),
                                 (2 ** 31 - 1, 0, 0, OK), (2 ** 29 - 64, 1, 0, OK)]:
        assert L.gdn_chunk_backward_workspace(1, L_, Hv, 64, 64, packed, ctypes.byref(n)) == code
    assert n.value == (2 ** 23 - 1) * 4 * (6 * 768 + 5 * 64 + 2 * 64 * 64 + 2 * 64 * 64)


def test_binding_refuses_before_the_library():
    k, v = torch.zeros(2, 1, 2, 64), torch.zeros(2, 1, 4, 64)
    b = torch.zeros(2, 1, 4)
    with pytest.raises(ValueError, match="device tensor"):
        G.gdn_recurrent_forward(k, k, v, b, b)
    with pytest.raises(ValueError, match="multiple of the key heads"):
        G.gdn_recurrent_forward(k, k, torch.zeros(2, 1, 3, 64), b, b)
    with pytest.raises(ValueError, match="B = 1"):
        G.gdn_recurrent_forward(k, k, v, b, b, cu_seqlens=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="S_final"):
        G.gdn_recurrent_forward(k, k, v, b, b, slots=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError, match="dtype"):
        G.gdn_recurrent_forward(k, k.half(), v, b, b)
    with pytest.raises(ValueError, match="B = 1"):
        G.gdn_chunk_backward_varlen(k, k, v, b, b, v, (None, None, 0), 64)
    with pytest.raises(ValueError, match="device tensor"):
        G.gdn_chunk_backward(k, k, v, b, b, v, 64)
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="kind"):
        G.gdn_norm_forward(x, kind="batch")
    with pytest.raises(ValueError, match="device tensor"):
        G.gdn_norm_forward(x)
    with pytest.raises(TypeError, match="weight"):
        G.gdn_norm_forward(x, torch.zeros(8, dtype=torch.float64))
    with pytest.raises(ValueError, match="mean"):
        G.gdn_norm_backward(x, x, None, torch.zeros(4), kind="layer")

"""The C ABI of gdnlinear.h on the CPU: every declared symbol is exported and bound, and bad
arguments are refused before anything reaches the GPU (no call here passes validation with
work to do)."""

import ctypes
import os
import re

import pytest
import torch

import paper_2606_06034_amd as G

HDR = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                   "gdnlinear.h")
OK, NULL, SHAPE, PARAM, DTYPE, ALIGN, ALIAS, WS = 0, -1, -2, -3, -4, -5, -6, -9
P = [k << 40 for k in range(1, 20)]  # aligned addresses far apart
L = G.lib


def test_exports_every_declared_symbol():
    names = sorted(set(re.findall(r"^int (gdn_\w+)\s*\(", open(HDR).read(), re.M)))
    assert names == sorted(G.linear_abi_symbols())
    for n in names:
        assert hasattr(L, n), n


def call(f, args, **change):
    a = dict(args, **change)
    return f(*a.values())


REC = dict(Q=P[0], K=P[1], V=P[2], g=P[3], per_token=1, S0=P[5], O=P[6], S_final=P[7], slots=None,
           n_states=4, cu=None, nseq=4, T=2, Hk=2, Hv=4, dk=128, dv=64, scale=1.0, dtype=1,
           stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(nseq=-1), SHAPE), (dict(T=-1), SHAPE), (dict(n_states=-1), SHAPE),
    (dict(Hk=3), SHAPE), (dict(Hk=0), SHAPE), (dict(Hk=-2), SHAPE), (dict(dk=96), SHAPE),
    (dict(dv=32), SHAPE), (dict(n_states=3), SHAPE), (dict(nseq=1 << 30, n_states=1 << 30), SHAPE),
    (dict(dtype=2), DTYPE), (dict(Q=None), NULL), (dict(K=None), NULL), (dict(V=None), NULL),
    (dict(g=None), NULL), (dict(O=None), NULL), (dict(Q=P[0] + 8), ALIGN),
    (dict(S0=P[5] + 4), ALIGN), (dict(slots=P[8] + 4), ALIGN), (dict(cu=P[8] + 4), ALIGN),
    (dict(O=P[0]), ALIAS), (dict(S_final=P[5] + 16), ALIAS), (dict(S_final=P[6]), ALIAS),
    (dict(O=P[3], per_token=0), ALIAS), (dict(nseq=0), OK), (dict(Hk=0, Hv=0), OK),
])
def test_recurrent_refusals(change, code):
    assert call(L.gdn_linear_recurrent, REC, **change) == code


# 2 sequences of 5000 tokens: cut into segments, a workspace is needed
FWD = dict(Q=P[0], K=P[1], V=P[2], g=P[3], per_token=1, S0=P[5], O=P[6], S_final=P[7], ws=P[8],
           wsb=1 << 39, cu=None, nseq=2, T=5000, Hk=2, Hv=4, dk=128, dv=64, scale=1.0, dtype=1,
           stream=None)
SIZES = [
    (dict(nseq=-1), SHAPE), (dict(T=-1), SHAPE), (dict(Hk=3), SHAPE), (dict(Hk=0), SHAPE),
    (dict(dk=96), SHAPE), (dict(dv=256), SHAPE), (dict(dtype=2), DTYPE),
    (dict(nseq=1 << 30), SHAPE), (dict(Hk=1 << 24, Hv=1 << 24), SHAPE),
    # the rows of a chunk's tokens, all heads: 64 * 2^18 * 128 * 2 bytes are 4 GiB
    (dict(Hk=(1 << 18) + 1, Hv=(1 << 18) + 1, nseq=1, T=64), SHAPE),
    (dict(Hk=0, Hv=0), OK)]


@pytest.mark.parametrize("change,code", SIZES + [
    (dict(Q=None), NULL), (dict(K=None), NULL), (dict(V=None), NULL), (dict(g=None), NULL),
    (dict(O=None), NULL), (dict(ws=None), NULL), (dict(wsb=1000), WS), (dict(O=P[6] + 2), ALIGN),
    (dict(S0=P[5] + 4), ALIGN), (dict(cu=P[9] + 4), ALIGN), (dict(O=P[2]), ALIAS),
    (dict(S_final=P[5] + 16), ALIAS), (dict(S_final=P[8]), ALIAS), (dict(ws=P[1]), ALIAS),
    (dict(O=P[9], cu=P[9]), ALIAS), (dict(nseq=0), OK)])
def test_forward_refusals(change, code):
    assert call(L.gdn_linear_forward, FWD, **change) == code


BWD = dict(Q=P[0], K=P[1], V=P[2], g=P[3], per_token=1, dO=P[5], S0=P[6], dSf=P[7], dQ=P[8],
           dK=P[9], dV=P[10], dg=P[11], dS0=P[12], ws=P[13], wsb=1 << 39, cu=None, nseq=2, T=5000,
           Hk=2, Hv=4, dk=128, dv=64, scale=1.0, dtype=1, stream=None)


@pytest.mark.parametrize("change,code", SIZES + [
    (dict(Q=None), NULL), (dict(K=None), NULL), (dict(V=None), NULL), (dict(g=None), NULL),
    (dict(dO=None), NULL), (dict(dQ=None), NULL), (dict(dK=None), NULL), (dict(dV=None), NULL),
    (dict(ws=None), NULL), (dict(wsb=1000), WS), (dict(dO=P[5] + 2), ALIGN),
    (dict(dS0=P[12] + 4), ALIGN), (dict(cu=P[14] + 4), ALIGN), (dict(dQ=P[0]), ALIAS),
    (dict(dK=P[8]), ALIAS), (dict(dS0=P[7]), ALIAS), (dict(dS0=P[6]), ALIAS),
    (dict(dg=P[3]), ALIAS), (dict(ws=P[2]), ALIAS), (dict(nseq=0), OK),
    (dict(nseq=0, per_token=0, dg=None), OK),
    # sums over a group's heads are fp32: 32 * 2^18 * 128 * 4 bytes are 4 GiB
    (dict(Hk=(1 << 18) + 1, Hv=(1 << 19) + 2, dv=64, nseq=1, T=32), SHAPE),
    (dict(Hk=1 << 18, Hv=1 << 19, dv=64, nseq=1, T=32, Q=None), NULL)])
def test_backward_refusals(change, code):
    assert call(L.gdn_linear_backward, BWD, **change) == code


def test_workspaces():
    # many short sequences are a segment each: no workspace; the gradient of g takes some
    assert G.gdn_linear_forward_workspace(300, 256, 4, 4, 128, 128) == 0
    assert G.gdn_linear_forward_workspace(1, 64, 4, 4, 128, 128) == 0
    assert G.gdn_linear_forward_workspace(1, 0, 4, 4, 128, 128) == 0
    assert G.gdn_linear_backward_workspace(1, 0, 4, 4, 128, 128) >= 0
    assert 0 < G.gdn_linear_backward_workspace(300, 256, 4, 4, 64, 64) < 300 * 256 * 4 * 16
    n = 8192 * 16 * 128  # a long sequence: fewer states than tokens' values
    assert 0 < G.gdn_linear_forward_workspace(1, 8192, 16, 16, 128, 128) < 4 * n
    assert G.gdn_linear_forward_workspace(1, 8192, 16, 16, 128, 128, dtype=torch.float32) > 0
    assert L.gdn_linear_forward_workspace(1, 8192, 16, 16, 128, 128, 0, 1, None) == NULL
    assert L.gdn_linear_backward_workspace(1, 8192, 16, 16, 128, 128, 0, 1, None) == NULL
    n = ctypes.c_int64()
    # lengths near 2^31 are cut into segments in 64 bits
    for f in (L.gdn_linear_forward_workspace, L.gdn_linear_backward_workspace):
        for packed in (0, 1):
            assert f(1, 2 ** 31 - 1, 1, 1, 64, 64, packed, 1, ctypes.byref(n)) == OK
            assert n.value > 0
        assert f(2 ** 31 - 1, 2 ** 31 - 1, 1, 1, 64, 64, 0, 1, ctypes.byref(n)) == SHAPE
        assert f(1, 100, 1, 1, 64, 64, 0, 2, ctypes.byref(n)) == DTYPE
        assert f(1, 100, 3, 4, 64, 64, 0, 1, ctypes.byref(n)) == SHAPE
    # launches of 512 work items for each segment and head: 2^32 of them at most, in the backward
    # pass two workgroups a segment and head
    for f, most in ((L.gdn_linear_forward_workspace, 1 << 23), (L.gdn_linear_backward_workspace,
                                                                 1 << 22)):
        assert f(most // 4 - 8, 1, 2, 4, 64, 64, 0, 1, ctypes.byref(n)) == SHAPE
        assert f(most // 5 - 8, 1, 2, 4, 64, 64, 0, 1, ctypes.byref(n)) == OK
    with pytest.raises(G.GdnError):
        G.gdn_linear_backward_workspace(2, 100, 3, 3, 96, 128)


GN = dict(x=P[0], w=P[1], b=P[2], z=P[3], y=P[4], mean=P[5], rstd=P[6], ws=P[7], wsb=1 << 30, N=8,
          S=100, C=96, G=8, eps=1e-6, act=1, dtype=1, wdt=0, stream=None)
GROUP = [
    (dict(N=-1), SHAPE), (dict(N=1 << 31), SHAPE), (dict(S=0), SHAPE), (dict(S=(1 << 30) + 1), SHAPE),
    (dict(N=1 << 20, S=1 << 20, C=512), SHAPE), (dict(C=0), SHAPE), (dict(C=65544), SHAPE), (dict(G=0), SHAPE), (dict(G=7), SHAPE),
    (dict(G=-8), SHAPE), (dict(act=2), PARAM), (dict(act=-1), PARAM), (dict(dtype=2), DTYPE),
    (dict(wdt=2), DTYPE)]


@pytest.mark.parametrize("change,code", GROUP + [
    (dict(eps=-1.0), PARAM), (dict(eps=float("nan")), PARAM), (dict(x=None), NULL),
    (dict(y=None), NULL), (dict(x=P[0] + 4), ALIGN), (dict(rstd=P[6] + 8), ALIGN),
    (dict(y=P[0]), ALIAS), (dict(mean=P[6]), ALIAS), (dict(y=P[3]), ALIAS),
    # groups of 100000 positions and more are read twice
    (dict(S=100000, ws=None), NULL), (dict(S=100000, wsb=4), WS),
    (dict(S=100000, N=1 << 26), SHAPE), (dict(S=100000, ws=P[0]), ALIAS), (dict(N=0), OK),
])
def test_group_norm_forward_refusals(change, code):
    assert call(L.gdn_group_norm_forward, GN, **change) == code


GB = dict(dy=P[0], x=P[1], w=P[2], b=P[3], z=P[4], mean=P[5], rstd=P[6], dx=P[7], dw=P[8],
          db=P[9], dz=P[10], ws=P[11], wsb=1 << 30, N=8, S=100, C=96, G=8, act=1, dtype=1, wdt=0,
          stream=None)


@pytest.mark.parametrize("change,code", GROUP + [
    (dict(dy=None), NULL), (dict(x=None), NULL), (dict(mean=None), NULL), (dict(rstd=None), NULL),
    (dict(dx=None), NULL), (dict(dz=None), NULL), (dict(ws=None), NULL), (dict(wsb=4), WS),
    (dict(S=1, wsb=4), WS), (dict(N=1 << 26), SHAPE), (dict(dw=P[8] + 4), ALIGN),
    (dict(dx=P[0]), ALIAS), (dict(db=P[8]), ALIAS), (dict(dz=P[4]), ALIAS), (dict(ws=P[1]), ALIAS),
    (dict(N=0, dw=None, db=None), OK),
])
def test_group_norm_backward_refusals(change, code):
    assert call(L.gdn_group_norm_backward, GB, **change) == code


def test_group_norm_workspaces():
    n = ctypes.c_int64()
    assert G.gdn_group_norm_forward_workspace(8192, 1, 4096, 32) == 0
    assert G.gdn_group_norm_forward_workspace(4, 65536, 512, 32) > 0
    assert G.gdn_group_norm_backward_workspace(4, 1, 512, 32) > 0
    assert G.gdn_group_norm_backward_workspace(4, 64, 512, 32) > 0
    assert L.gdn_group_norm_forward_workspace(4, 64, 512, 32, 1, None) == NULL
    assert L.gdn_group_norm_backward_workspace(4, 64, 512, 32, 1, None) == NULL
    assert L.gdn_group_norm_backward_workspace(4, 64, 512, 33, 1, ctypes.byref(n)) == SHAPE
    assert L.gdn_group_norm_forward_workspace(4, 64, 512, 32, 3, ctypes.byref(n)) == DTYPE


def test_binding_refuses_before_the_library():
    k, v = torch.zeros(2, 1, 2, 64), torch.zeros(2, 1, 4, 64)
    g = torch.zeros(4)
    cu = torch.zeros(3, dtype=torch.int32)
    for f in (G.gdn_linear_forward, G.gdn_linear_recurrent):
        with pytest.raises(ValueError, match="device tensor"):
            f(k, k, v, g)
        with pytest.raises(ValueError, match="multiple of the key heads"):
            f(k, k, torch.zeros(2, 1, 3, 64), g)
        with pytest.raises(ValueError, match="B = 1"):
            f(k, k, v, g, cu_seqlens=cu)
        with pytest.raises(ValueError, match="nseq"):
            f(k[:1], k[:1], v[:1], g, cu_seqlens=cu[:0])
        with pytest.raises(TypeError, match="dtype"):
            f(k, k.half(), v, g)
    with pytest.raises(ValueError, match="S_final"):
        G.gdn_linear_recurrent(k, k, v, g, slots=cu[:2])
    with pytest.raises(ValueError, match="device tensor"):
        G.gdn_linear_backward(k, k, v, g, v)
    with pytest.raises(ValueError, match="B = 1"):
        G.gdn_linear_backward(k, k, v, g, v, cu_seqlens=cu)
    x = torch.zeros(4, 3, 8)
    with pytest.raises(ValueError, match="act"):
        G.gdn_group_norm_forward(x, 2, act="gelu")
    with pytest.raises(ValueError, match="groups"):
        G.gdn_group_norm_forward(x, 3)
    with pytest.raises(ValueError, match="groups"):
        G.gdn_group_norm_backward(x, x, 0, None, g, g)
    with pytest.raises(ValueError, match="dimension"):
        G.gdn_group_norm_forward(x[0, 0], 2)
    with pytest.raises(ValueError, match="device tensor"):
        G.gdn_group_norm_forward(x, 2)
    with pytest.raises(TypeError, match="weight"):
        G.gdn_group_norm_forward(x, 2, torch.zeros(8, dtype=torch.float64))

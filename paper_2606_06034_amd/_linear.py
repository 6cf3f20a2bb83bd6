"""ctypes marshalling for the operators of include/gdnlinear.h (same library
and manner as _layer.py): linear attention with a decay for each head, and
group norm, channels last."""

from __future__ import annotations

import ctypes
from typing import Optional

import torch

from ._binding import _FDT, _check, _fdtype, _on_stream, lib
from . import _layer
from ._layer import _groups, _params, _stream

_c_int, _c_i64, _c_f, _vp = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p

_SIGS = {
    "gdn_linear_forward": [_vp] * 4 + [_c_int] + [_vp] * 4 + [_c_i64, _vp] + [_c_int] * 6 +
                          [_c_f, _c_int, _vp],
    "gdn_linear_forward_workspace": [_c_int] * 8 + [ctypes.POINTER(_c_i64)],
    "gdn_linear_backward": [_vp] * 4 + [_c_int] + [_vp] * 9 + [_c_i64, _vp] + [_c_int] * 6 +
                           [_c_f, _c_int, _vp],
    "gdn_linear_backward_workspace": [_c_int] * 8 + [ctypes.POINTER(_c_i64)],
    "gdn_linear_recurrent": [_vp] * 4 + [_c_int] + [_vp] * 4 + [_c_int, _vp] + [_c_int] * 6 +
                            [_c_f, _c_int, _vp],
    "gdn_group_norm_forward": [_vp] * 8 + [_c_i64, _c_i64] + [_c_int] * 3 + [_c_f] +
                              [_c_int] * 3 + [_vp],
    "gdn_group_norm_forward_workspace": [_c_i64] + [_c_int] * 4 + [ctypes.POINTER(_c_i64)],
    "gdn_group_norm_backward": [_vp] * 12 + [_c_i64, _c_i64] + [_c_int] * 6 + [_vp],
    "gdn_group_norm_backward_workspace": [_c_i64] + [_c_int] * 4 + [ctypes.POINTER(_c_i64)],
}

for _name, _args in _SIGS.items():
    _fn = getattr(lib, _name)
    _fn.argtypes, _fn.restype = _args, _c_int


GDN_ACT_NONE, GDN_ACT_SILU = 0, 1


def linear_abi_symbols():
    return list(_SIGS)


_F32, _I32 = torch.float32, torch.int32
_device = _layer._device or torch.cuda.current_device


def _dev(t: torch.Tensor, name: str, dtype=None, numel: Optional[int] = None) -> int:
    """Address of a tensor of the current device, where the launches go."""
    try:
        if (t.is_cuda and t.get_device() == _device() and t.is_contiguous() and
                (dtype is None or t.dtype is dtype) and (numel is None or t.numel() == numel)):
            return t.data_ptr()
    except AttributeError:  # not a tensor
        pass
    _layer._dev(t, name, dtype, numel)
    raise ValueError(f"{name} is on {t.device}, not on the current device (cuda:{_device()}): "
                     f"call under torch.cuda.device(), or name a stream of {t.device}")


def _opt(t: Optional[torch.Tensor], name: str, dtype=None, numel: Optional[int] = None):
    return None if t is None else _dev(t, name, dtype, numel)


def _affine(weight, bias, C):
    """Pointers of weight and bias and their dtype (one dtype for both)."""
    p = _params(weight, bias, C)
    for t, name in ((weight, "weight"), (bias, "bias")):
        _opt(t, name)
    return p


def _sizes(K, V, cu):
    """(sequences, tokens of each or of all, tokens, Hk, Hv, dk, dv)"""
    B, T, Hk, dk = K.shape
    Hv, dv = V.shape[-2:]
    _groups(Hk, Hv)
    if cu is None:
        return B, T, B * T, Hk, Hv, dk, dv
    if B != 1:
        raise ValueError("packed sequences use B = 1")
    if cu.numel() < 1:
        raise ValueError("cu_seqlens must hold nseq + 1 offsets")
    return cu.numel() - 1, T, T, Hk, Hv, dk, dv


def _workspace(fn, args, device):
    n = _c_i64()
    _check(fn, getattr(lib, fn)(*args, ctypes.byref(n)))
    return n.value if device is None else torch.empty(max(n.value, 16), dtype=torch.uint8,
                                                      device=device)


def gdn_linear_forward_workspace(nseq: int, T: int, Hk: int, Hv: int, dk: int, dv: int,
                                 packed: bool = False,
                                 dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of workspace gdn_linear_forward needs for nseq sequences of T tokens, or with
    packed for nseq sequences of T tokens in all."""
    return _workspace("gdn_linear_forward_workspace",
                      (nseq, T, Hk, Hv, dk, dv, int(packed), _FDT[dtype]), None)


def gdn_linear_forward(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, g: torch.Tensor,
                       S0: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                       want_state: bool = True, O: Optional[torch.Tensor] = None,
                       S_final: Optional[torch.Tensor] = None,
                       cu_seqlens: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None):
    """Linear attention with decay over whole sequences: (O, S_final or None).  Q, K [B, T, Hk,
    dk], V [B, T, Hv, dv]; g, fp32: the log-decay of each token [B, T, Hv] or of each head [Hv].
    With cu_seqlens (nseq + 1 int32 offsets on the device) packed tokens, [1, T, ...].  S0,
    S_final [nseq, Hv, dk, dv] fp32, which may be one tensor.  The workspace (a byte tensor of
    gdn_linear_forward_workspace() bytes) is allocated when not given."""
    if stream is not None and (workspace is None or O is None or want_state and S_final is None):
        return _on_stream(stream, gdn_linear_forward, locals())
    nseq, T, tok, Hk, Hv, dk, dv = _sizes(K, V, cu_seqlens)
    dt, per_token = _fdtype(K, "K"), g.dim() != 1
    scale = dk ** -0.5 if scale is None else float(scale)
    O = torch.empty_like(V) if O is None else O
    if want_state and S_final is None:
        S_final = torch.empty((nseq, Hv, dk, dv), dtype=_F32, device=K.device)
    if workspace is None:
        workspace = _workspace("gdn_linear_forward_workspace",
                               (nseq, T, Hk, Hv, dk, dv, int(cu_seqlens is not None), dt),
                               K.device)
    states = nseq * Hv * dk * dv
    _check("gdn_linear_forward", lib.gdn_linear_forward(
        _dev(Q, "Q", K.dtype, tok * Hk * dk), _dev(K, "K"), _dev(V, "V", K.dtype, tok * Hv * dv),
        _dev(g, "g", _F32, tok * Hv if per_token else Hv), int(per_token),
        _opt(S0, "S0", _F32, states), _dev(O, "O", K.dtype, tok * Hv * dv),
        _opt(S_final, "S_final", _F32, states), _dev(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _opt(cu_seqlens, "cu_seqlens", _I32), nseq,
        T, Hk, Hv, dk, dv, scale, dt, _stream(stream)))
    return O, S_final


def gdn_linear_backward_workspace(nseq: int, T: int, Hk: int, Hv: int, dk: int, dv: int,
                                  packed: bool = False,
                                  dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of workspace gdn_linear_backward needs, wanting every gradient."""
    return _workspace("gdn_linear_backward_workspace",
                      (nseq, T, Hk, Hv, dk, dv, int(packed), _FDT[dtype]), None)


def gdn_linear_backward(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, g: torch.Tensor,
                        dO: torch.Tensor, S0: Optional[torch.Tensor] = None,
                        dS_final: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                        want_dg: bool = True, want_dS0: bool = False, out=None,
                        cu_seqlens: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradients of gdn_linear_forward: (dQ, dK, dV, dg or None, dS0 or None) from dO and, where
    given, the gradient of the final states; dg has g's shape, fp32.  out: the five outputs
    (None where one is to be allocated).  The workspace (a byte tensor of
    gdn_linear_backward_workspace() bytes) is allocated when not given."""
    if stream is not None and (workspace is None or out is None or any(t is None for t in out)):
        return _on_stream(stream, gdn_linear_backward, locals())
    nseq, T, tok, Hk, Hv, dk, dv = _sizes(K, V, cu_seqlens)
    dt, per_token = _fdtype(K, "K"), g.dim() != 1
    scale = dk ** -0.5 if scale is None else float(scale)
    dQ, dK, dV, dg, dS0 = out if out is not None else (None,) * 5
    dQ = torch.empty_like(K) if dQ is None else dQ
    dK = torch.empty_like(K) if dK is None else dK
    dV = torch.empty_like(V) if dV is None else dV
    if not want_dg:
        dg = None
    elif dg is None:
        dg = torch.empty_like(g)
    if not want_dS0:
        dS0 = None
    elif dS0 is None:
        dS0 = torch.empty((nseq, Hv, dk, dv), dtype=_F32, device=K.device)
    if workspace is None:
        workspace = _workspace("gdn_linear_backward_workspace",
                               (nseq, T, Hk, Hv, dk, dv, int(cu_seqlens is not None), dt),
                               K.device)
    states, gates = nseq * Hv * dk * dv, tok * Hv if per_token else Hv
    _check("gdn_linear_backward", lib.gdn_linear_backward(
        _dev(Q, "Q", K.dtype, tok * Hk * dk), _dev(K, "K"), _dev(V, "V", K.dtype, tok * Hv * dv),
        _dev(g, "g", _F32, gates), int(per_token), _dev(dO, "dO", K.dtype, tok * Hv * dv),
        _opt(S0, "S0", _F32, states), _opt(dS_final, "dS_final", _F32, states),
        _dev(dQ, "dQ", K.dtype, tok * Hk * dk), _dev(dK, "dK", K.dtype, tok * Hk * dk),
        _dev(dV, "dV", K.dtype, tok * Hv * dv), _opt(dg, "dg", _F32, gates),
        _opt(dS0, "dS0", _F32, states), _dev(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _opt(cu_seqlens, "cu_seqlens", _I32), nseq,
        T, Hk, Hv, dk, dv, scale, dt, _stream(stream)))
    return dQ, dK, dV, dg, dS0


def gdn_linear_recurrent(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, g: torch.Tensor,
                         S0: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                         want_state: bool = True, O: Optional[torch.Tensor] = None,
                         S_final: Optional[torch.Tensor] = None,
                         slots: Optional[torch.Tensor] = None,
                         cu_seqlens: Optional[torch.Tensor] = None, stream=None):
    """The same token by token, for decoding: (O, S_final or None).  S0, S_final [nseq, Hv, dk,
    dv] fp32, which may be one tensor (updated in place); with slots (int32 [nseq] on the
    device) they are pools [n_states, Hv, dk, dv], sequence s reads and writes state slots[s],
    an index outside the pool marks a padded sequence (O zeros), and S_final has to be given
    (S0 itself, for a pool updated in place)."""
    if stream is not None and (O is None or want_state and S_final is None):
        return _on_stream(stream, gdn_linear_recurrent, locals())
    nseq, T, tok, Hk, Hv, dk, dv = _sizes(K, V, cu_seqlens)
    dt, per_token = _fdtype(K, "K"), g.dim() != 1
    scale = dk ** -0.5 if scale is None else float(scale)
    O = torch.empty_like(V) if O is None else O
    if slots is None:
        n = nseq
    else:
        pool = S0 if S0 is not None else S_final
        n = pool.shape[0] if pool is not None else 0
        if want_state and S_final is None:
            raise ValueError("slots: S_final (the pool to write) has to be given")
    if want_state and S_final is None:
        S_final = torch.empty((nseq, Hv, dk, dv), dtype=_F32, device=K.device)
    states = n * Hv * dk * dv
    _check("gdn_linear_recurrent", lib.gdn_linear_recurrent(
        _dev(Q, "Q", K.dtype, tok * Hk * dk), _dev(K, "K"), _dev(V, "V", K.dtype, tok * Hv * dv),
        _dev(g, "g", _F32, tok * Hv if per_token else Hv), int(per_token),
        _opt(S0, "S0", _F32, states), _dev(O, "O", K.dtype, tok * Hv * dv),
        _opt(S_final, "S_final", _F32, states), _opt(slots, "slots", _I32, nseq), n,
        _opt(cu_seqlens, "cu_seqlens", _I32), nseq, T, Hk, Hv, dk, dv, scale, dt,
        _stream(stream)))
    return O, S_final


_ACTS = {None: GDN_ACT_NONE, "silu": GDN_ACT_SILU}


def _group_sizes(x, groups, act):
    """(N, S, C, dtype, act) of x [N, ..., C]."""
    if act not in _ACTS:
        raise ValueError("act must be None or 'silu'")
    if x.dim() < 2:
        raise ValueError("x must have a first and a last (channel) dimension")
    N, C = x.shape[0], x.shape[-1]
    if groups < 1 or C % groups:
        raise ValueError(f"the channels ({C}) must be a multiple of the groups ({groups})")
    S = 1
    for n in x.shape[1:-1]:
        S *= n
    return N, S, C, _fdtype(x, "x"), _ACTS[act]


def gdn_group_norm_forward_workspace(N: int, S: int, C: int, groups: int,
                                     dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of workspace gdn_group_norm_forward needs for x [N, S, C]."""
    return _workspace("gdn_group_norm_forward_workspace", (N, S, C, groups, _FDT[dtype]), None)


def gdn_group_norm_forward(x: torch.Tensor, groups: int, weight: Optional[torch.Tensor] = None,
                           bias: Optional[torch.Tensor] = None,
                           gate: Optional[torch.Tensor] = None, act: Optional[str] = None,
                           eps: float = 1e-5, y: Optional[torch.Tensor] = None,
                           want_stats: bool = True, workspace: Optional[torch.Tensor] = None,
                           stream=None):
    """(y, mean, rstd): group norm of x [N, ..., C], channels last, each of the groups of
    neighbouring channels over its channels and the dimensions between, times weight, plus bias
    ([C]), act (None or "silu") of it, times silu(gate).  mean and rstd, fp32 [N, groups], are
    what gdn_group_norm_backward takes (None with want_stats=False).  The workspace (a byte
    tensor of gdn_group_norm_forward_workspace() bytes) is allocated when not given."""
    if stream is not None:
        return _on_stream(stream, gdn_group_norm_forward, locals())
    N, S, C, dt, a = _group_sizes(x, groups, act)
    y = torch.empty_like(x) if y is None else y
    mean = rstd = None
    if want_stats:
        rstd = x.new_empty((N, groups), dtype=torch.float32)
        mean = torch.empty_like(rstd)
    wp, bp, wdt = _affine(weight, bias, C)
    if workspace is None:
        n = _workspace("gdn_group_norm_forward_workspace", (N, S, C, groups, dt), None)
        workspace = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None
    _check("gdn_group_norm_forward", lib.gdn_group_norm_forward(
        _dev(x, "x"), wp, bp, _opt(gate, "gate", x.dtype, x.numel()),
        _dev(y, "y", x.dtype, x.numel()), None if mean is None else mean.data_ptr(),
        None if rstd is None else rstd.data_ptr(), _opt(workspace, "workspace"),
        0 if workspace is None else workspace.numel() * workspace.element_size(), N, S, C, groups,
        eps, a, dt, wdt, _stream(stream)))
    return y, mean, rstd


def gdn_group_norm_backward_workspace(N: int, S: int, C: int, groups: int,
                                      dtype: torch.dtype = torch.bfloat16) -> int:
    """Bytes of workspace gdn_group_norm_backward needs for x [N, S, C]."""
    return _workspace("gdn_group_norm_backward_workspace", (N, S, C, groups, _FDT[dtype]), None)


def gdn_group_norm_backward(dy: torch.Tensor, x: torch.Tensor, groups: int,
                            weight: Optional[torch.Tensor], mean: torch.Tensor,
                            rstd: torch.Tensor, bias: Optional[torch.Tensor] = None,
                            gate: Optional[torch.Tensor] = None, act: Optional[str] = None,
                            want_dw: bool = True, want_db: Optional[bool] = None,
                            dx: Optional[torch.Tensor] = None, dz: Optional[torch.Tensor] = None,
                            workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, dw, db, dz) from dy and what gdn_group_norm_forward took and returned; dw and db fp32
    [C] (db None without a bias unless want_db), dz None without a gate.  The workspace (a byte
    tensor of gdn_group_norm_backward_workspace() bytes) is allocated when not given."""
    if stream is not None:
        return _on_stream(stream, gdn_group_norm_backward, locals())
    N, S, C, dt, a = _group_sizes(x, groups, act)
    n, f32 = x.numel(), torch.float32
    dx = torch.empty_like(x) if dx is None else dx
    if gate is None:
        dz = None
    elif dz is None:
        dz = torch.empty_like(gate)
    want_db = bias is not None if want_db is None else want_db
    dw = torch.empty(C, dtype=f32, device=x.device) if want_dw else None
    db = torch.empty(C, dtype=f32, device=x.device) if want_db else None
    if workspace is None:
        workspace = _workspace("gdn_group_norm_backward_workspace", (N, S, C, groups, dt),
                               x.device)
    wp, bp, wdt = _affine(weight, bias, C)
    _check("gdn_group_norm_backward", lib.gdn_group_norm_backward(
        _dev(dy, "dy", x.dtype, n), _dev(x, "x"), wp, bp, _opt(gate, "gate", x.dtype, n),
        _dev(mean, "mean", f32, N * groups), _dev(rstd, "rstd", f32, N * groups),
        _dev(dx, "dx", x.dtype, n), None if dw is None else dw.data_ptr(),
        None if db is None else db.data_ptr(), _opt(dz, "dz", x.dtype, n),
        _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(), N, S, C,
        groups, a, dt, wdt, _stream(stream)))
    return dx, dw, db, dz

"""ctypes marshalling for the operators of include/gdnlayer.h (same library
and manner as _binding.py): the recurrent gated delta rule, the chunk-wise
backward pass and the norms of the layer."""

from __future__ import annotations

import ctypes
from typing import Optional

import torch

from ._binding import (_FDT, _check, _dev as _dev_checked, _fdtype, _on_stream,
                       _stream as _stream_of, lib)

GDN_NORM_LAYER, GDN_NORM_RMS = 0, 1

_c_int, _c_i64, _c_f, _vp = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p

_SIGS = {
    "gdn_recurrent_forward": [_vp] * 9 + [_c_int, _vp] + [_c_int] * 6 + [_c_f, _c_int, _vp],
    "gdn_chunk_backward": [_vp] * 15 + [_c_i64] + [_c_int] * 7 + [_c_f, _c_int, _vp],
    "gdn_chunk_backward_varlen": [_vp] * 15 + [_c_i64, _vp] + [_c_int] * 7 + [_c_f, _c_int, _vp],
    "gdn_chunk_backward_workspace": [_c_int] * 6 + [ctypes.POINTER(_c_i64)],
    "gdn_norm_forward": [_vp] * 7 + [_c_i64, _c_int, _c_f] + [_c_int] * 3 + [_vp],
    "gdn_norm_backward": [_vp] * 12 + [_c_i64, _c_i64] + [_c_int] * 4 + [_vp],
    "gdn_norm_backward_workspace": [_c_i64, _c_int, ctypes.POINTER(_c_i64)],
}

for _name, _args in _SIGS.items():
    _fn = getattr(lib, _name)
    _fn.argtypes, _fn.restype = _args, _c_int


def layer_abi_symbols():
    return list(_SIGS)


# The smallest calls are bound by what happens here: the checks pass in one
# expression (and are made again one by one, for the message, where it fails), and
# the current stream is asked for without a Stream object (0.1 us, not 2.7).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _dev(t: torch.Tensor, name: str, dtype=None, numel: Optional[int] = None) -> int:
    try:
        if (t.is_cuda and t.is_contiguous() and (dtype is None or t.dtype is dtype) and
                (numel is None or t.numel() == numel)):
            return t.data_ptr()
    except AttributeError:  # not a tensor
        pass
    return _dev_checked(t, name, dtype, numel)


def _stream(stream) -> int:
    if stream is None and _raw_stream is not None and _device is not None:
        return _raw_stream(_device())
    return _stream_of(stream)


def _opt(t: Optional[torch.Tensor], name: str, dtype=None, numel: Optional[int] = None):
    return None if t is None else _dev(t, name, dtype, numel)


def _groups(Hk: int, Hv: int):
    if (Hk and Hv % Hk) or (Hv and not Hk):
        raise ValueError(f"the value heads ({Hv}) must be a multiple of the key heads ({Hk})")


def gdn_recurrent_forward(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, beta: torch.Tensor,
                          g: torch.Tensor, S0: Optional[torch.Tensor] = None,
                          scale: Optional[float] = None, want_state: bool = True,
                          O: Optional[torch.Tensor] = None,
                          S_final: Optional[torch.Tensor] = None,
                          slots: Optional[torch.Tensor] = None,
                          cu_seqlens: Optional[torch.Tensor] = None, stream=None):
    """The gated delta rule token by token: (O, S_final or None).  Q, K [nseq, T, Hk, dk],
    V [nseq, T, Hv, dv], beta and the per-token log-decay g [nseq, T, Hv] fp32; with
    cu_seqlens (nseq + 1 int32 offsets on the device) packed tokens, [1, T, ...].  S0,
    S_final [nseq, Hv, dk, dv] fp32, which may be one tensor (updated in place); with slots
    (int32 [nseq] on the device) they are pools [n_states, Hv, dk, dv], sequence s reads and
    writes state slots[s], an index outside the pool marks a padded sequence (O zeros), and
    S_final has to be given (S0 itself, for a pool updated in place)."""
    if stream is not None and (O is None or want_state and S_final is None):
        return _on_stream(stream, gdn_recurrent_forward, locals())
    B, T, Hk, dk = K.shape
    Hv, dv = V.shape[-2:]
    _groups(Hk, Hv)
    dt = _fdtype(K, "K")
    if cu_seqlens is not None and B != 1:
        raise ValueError("packed sequences use B = 1")
    nseq = B if cu_seqlens is None else cu_seqlens.numel() - 1
    if nseq < 0:
        raise ValueError("cu_seqlens must hold nseq + 1 offsets")
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
        S_final = torch.empty((nseq, Hv, dk, dv), dtype=torch.float32, device=K.device)
    tok, states = B * T, n * Hv * dk * dv
    _check("gdn_recurrent_forward", lib.gdn_recurrent_forward(
        _dev(Q, "Q", K.dtype, tok * Hk * dk), _dev(K, "K"), _dev(V, "V", K.dtype, tok * Hv * dv),
        _dev(beta, "beta", torch.float32, tok * Hv), _dev(g, "g", torch.float32, tok * Hv),
        _opt(S0, "S0", torch.float32, states), _dev(O, "O", K.dtype, tok * Hv * dv),
        _opt(S_final, "S_final", torch.float32, states), _opt(slots, "slots", torch.int32, nseq),
        n, _opt(cu_seqlens, "cu_seqlens", torch.int32), nseq, T, Hk, Hv, dk, dv, scale, dt,
        _stream(stream)))
    return O, S_final


def gdn_chunk_backward_workspace(nseq: int, L: int, Hv: int, dk: int, dv: int,
                                 packed: bool = False) -> int:
    """Bytes of workspace gdn_chunk_backward needs for nseq sequences of L tokens, or with
    packed gdn_chunk_backward_varlen for nseq sequences of L tokens in all."""
    n = _c_i64()
    _check("gdn_chunk_backward_workspace", lib.gdn_chunk_backward_workspace(
        nseq, L, Hv, dk, dv, int(packed), ctypes.byref(n)))
    return n.value


def _backward(fn, Q, K, V, beta, g, dO, C, cu, S0, dS_final, scale, want_dS0, out, workspace,
              stream):
    B, L, Hk, dk = K.shape
    Hv, dv = V.shape[-2:]
    _groups(Hk, Hv)
    dt = _fdtype(K, "K")
    nseq = B if cu is None else cu.numel() - 1
    if nseq < 0:
        raise ValueError("cu_seqlens must hold nseq + 1 offsets")
    scale = dk ** -0.5 if scale is None else float(scale)
    tok, states = B * L, nseq * Hv * dk * dv
    dQ, dK, dV, dbeta, dg, dS0 = out if out is not None else (None,) * 6
    dQ = torch.empty_like(K) if dQ is None else dQ
    dK = torch.empty_like(K) if dK is None else dK
    dV = torch.empty_like(V) if dV is None else dV
    dbeta = torch.empty_like(beta) if dbeta is None else dbeta
    dg = torch.empty_like(g) if dg is None else dg
    if want_dS0 and dS0 is None:
        dS0 = torch.empty((nseq, Hv, dk, dv), dtype=torch.float32, device=K.device)
    if workspace is None:
        need = gdn_chunk_backward_workspace(nseq, L, Hv, dk, dv, cu is not None)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=K.device)
    f32 = torch.float32
    args = [_dev(Q, "Q", K.dtype, tok * Hk * dk), _dev(K, "K"), _dev(V, "V", K.dtype, tok * Hv * dv),
            _dev(beta, "beta", f32, tok * Hv), _dev(g, "g", f32, tok * Hv),
            _dev(dO, "dO", K.dtype, tok * Hv * dv), _opt(S0, "S0", f32, states),
            _opt(dS_final, "dS_final", f32, states), _dev(dQ, "dQ", K.dtype, tok * Hk * dk),
            _dev(dK, "dK", K.dtype, tok * Hk * dk), _dev(dV, "dV", K.dtype, tok * Hv * dv),
            _dev(dbeta, "dbeta", f32, tok * Hv), _dev(dg, "dg", f32, tok * Hv),
            _opt(dS0, "dS0", f32, states), _dev(workspace, "workspace"),
            workspace.numel() * workspace.element_size()]
    if cu is not None:
        args.append(_dev(cu, "cu_seqlens", torch.int32))
    _check(fn, getattr(lib, fn)(*args, nseq, L, Hk, Hv, dk, dv, C, scale, dt, _stream(stream)))
    return dQ, dK, dV, dbeta, dg, dS0


def gdn_chunk_backward(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, beta: torch.Tensor,
                       g: torch.Tensor, dO: torch.Tensor, C: int,
                       S0: Optional[torch.Tensor] = None,
                       dS_final: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                       want_dS0: bool = False, out=None,
                       workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradients of gdn_chunk_forward(..., inverse="exact"): (dQ, dK, dV, dbeta, dg, dS0 or
    None) from dO and, where given, the gradient of its final state.  Q, K [B, L, Hk, dk], V,
    dO [B, L, Hv, dv], beta, g [B, L, Hv]; L need not be a multiple of C.  out: the six outputs
    (None where one is to be allocated).  The workspace (a byte tensor of
    gdn_chunk_backward_workspace() bytes) is allocated when not given."""
    if stream is not None and (workspace is None or out is None or any(t is None for t in out)):
        return _on_stream(stream, gdn_chunk_backward, locals())
    return _backward("gdn_chunk_backward", Q, K, V, beta, g, dO, C, None, S0, dS_final, scale,
                     want_dS0, out, workspace, stream)


def gdn_chunk_backward_varlen(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                              beta: torch.Tensor, g: torch.Tensor, dO: torch.Tensor, tables,
                              C: int, S0: Optional[torch.Tensor] = None,
                              dS_final: Optional[torch.Tensor] = None,
                              scale: Optional[float] = None, want_dS0: bool = False, out=None,
                              workspace: Optional[torch.Tensor] = None, stream=None):
    """The same over packed sequences (B = 1): tables = gdn_varlen_tables(cu_seqlens, C), of
    which the token offsets are read; S0, dS_final, dS0 [nseq, Hv, dk, dv]."""
    if stream is not None and (workspace is None or out is None or any(t is None for t in out)):
        return _on_stream(stream, gdn_chunk_backward_varlen, locals())
    if K.shape[0] != 1:
        raise ValueError("packed sequences use B = 1")
    return _backward("gdn_chunk_backward_varlen", Q, K, V, beta, g, dO, C, tables[0], S0,
                     dS_final, scale, want_dS0, out, workspace, stream)


_KINDS = {"layer": GDN_NORM_LAYER, "rms": GDN_NORM_RMS}


def _kind(kind: str) -> int:
    if kind not in _KINDS:
        raise ValueError(f"kind must be one of {sorted(_KINDS)}")
    return _KINDS[kind]


def _params(weight, bias, D):
    """Pointers of weight and bias and their dtype (one dtype for both)."""
    p = weight if weight is not None else bias
    dt = torch.float32 if p is None else p.dtype
    if dt not in _FDT:
        raise TypeError(f"weight: dtype {dt} not supported (float32 or bfloat16)")
    return _opt(weight, "weight", dt, D), _opt(bias, "bias", dt, D), _FDT[dt]


def gdn_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None,
                     bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                     kind: str = "rms", eps: float = 1e-6, y: Optional[torch.Tensor] = None,
                     want_stats: bool = True, stream=None):
    """(y, mean, rstd): the norm of x over its last dimension ("layer" or "rms"), times weight,
    plus bias, times silu(gate).  mean (None for "rms") and rstd, fp32 [x.shape[:-1]], are what
    gdn_norm_backward takes (None with want_stats=False)."""
    if stream is not None and (y is None or want_stats):
        return _on_stream(stream, gdn_norm_forward, locals())
    k, D = _kind(kind), x.shape[-1]
    dt = _fdtype(x, "x")
    rows = x.numel() // D if D else 0
    y = torch.empty_like(x) if y is None else y
    mean = rstd = None
    if want_stats:
        rstd = x.new_empty(x.shape[:-1], dtype=torch.float32)
        mean = torch.empty_like(rstd) if k == GDN_NORM_LAYER else None
    wp, bp, wdt = _params(weight, bias, D)
    _check("gdn_norm_forward", lib.gdn_norm_forward(
        _dev(x, "x"), wp, bp, _opt(gate, "gate", x.dtype, x.numel()),
        _dev(y, "y", x.dtype, x.numel()), None if mean is None else mean.data_ptr(),
        None if rstd is None else rstd.data_ptr(), rows, D, eps, k, dt, wdt, _stream(stream)))
    return y, mean, rstd


def gdn_norm_backward_workspace(rows: int, D: int) -> int:
    """Bytes of workspace gdn_norm_backward needs for these sizes."""
    n = _c_i64()
    _check("gdn_norm_backward_workspace",
           lib.gdn_norm_backward_workspace(rows, D, ctypes.byref(n)))
    return n.value


def gdn_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor],
                      rstd: torch.Tensor, mean: Optional[torch.Tensor] = None,
                      bias: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                      kind: str = "rms", want_dw: bool = True, want_db: Optional[bool] = None,
                      dx: Optional[torch.Tensor] = None, dz: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, dw, db, dz) from dy and what gdn_norm_forward took and returned; dw and db fp32 [D]
    (db None without a bias unless want_db), dz None without a gate.  The workspace (a byte
    tensor of gdn_norm_backward_workspace() bytes) is allocated when not given."""
    if stream is not None:
        return _on_stream(stream, gdn_norm_backward, locals())
    k, D = _kind(kind), x.shape[-1]
    dt = _fdtype(x, "x")
    n, rows = x.numel(), x.numel() // D if D else 0
    dx = torch.empty_like(x) if dx is None else dx
    if gate is not None and dz is None:
        dz = torch.empty_like(gate)
    want_db = bias is not None if want_db is None else want_db
    dw = torch.empty(D, dtype=torch.float32, device=x.device) if want_dw else None
    db = torch.empty(D, dtype=torch.float32, device=x.device) if want_db else None
    need = gdn_norm_backward_workspace(rows, D)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    if k == GDN_NORM_LAYER and mean is None:
        raise ValueError('mean must be given for kind "layer"')
    wp, bp, wdt = _params(weight, bias, D)
    _check("gdn_norm_backward", lib.gdn_norm_backward(
        _dev(dy, "dy", x.dtype, n), _dev(x, "x"), wp, bp, _opt(gate, "gate", x.dtype, n),
        _opt(mean, "mean", torch.float32, rows), _dev(rstd, "rstd", torch.float32, rows),
        _dev(dx, "dx", x.dtype, n), None if dw is None else dw.data_ptr(),
        None if db is None else db.data_ptr(), _opt(dz, "dz", x.dtype, n),
        _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(), rows, D, k,
        dt, wdt, _stream(stream)))
    return dx, dw, db, dz

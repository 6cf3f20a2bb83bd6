"""Linear attention with a decay for each head, and group norm, channels last, in fp64 numpy,
with their gradients.

Arrays are [tokens, heads, ...] of one sequence.  The recurrence is
    S_t = e^{g_t} S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,
its gradients by reverse accumulation token by token.
"""

from __future__ import annotations

import numpy as np

__all__ = ["linear", "linear_grad", "linear_sizes", "group_norm", "group_norm_grad"]


def _f64(*xs):
    return tuple(None if x is None else np.asarray(x, np.float64) for x in xs)


def _decay(g, T, Hv):
    """[T, Hv] of the log-decays of the tokens or of the heads."""
    g = np.asarray(g, np.float64)
    return np.broadcast_to(g, (T, Hv))


def linear(Q, K, V, g, S0=None, scale=1.0):
    """(O [T, Hv, dv], S [Hv, dk, dv]); Q, K [T, Hk, dk], value head h reading key head
    h // (Hv // Hk); g [T, Hv] or [Hv]."""
    Q, K, V, S0 = _f64(Q, K, V, S0)
    T, Hv, dv = V.shape
    r = Hv // K.shape[1]
    g = _decay(g, T, Hv)
    S = np.zeros((Hv, K.shape[2], dv)) if S0 is None else S0.copy()
    O = np.zeros((T, Hv, dv))
    for t in range(T):
        q, k = np.repeat(Q[t], r, 0), np.repeat(K[t], r, 0)
        S = np.exp(g[t])[:, None, None] * S + k[:, :, None] * V[t][:, None, :]
        O[t] = scale * np.einsum("hk,hkv->hv", q, S)
    return O, S


def linear_grad(Q, K, V, g, dO, S0=None, dS=None, scale=1.0):
    """(dQ, dK, dV, dg, dS0) of sum(O dO) + sum(S dS); dg [T, Hv], or [Hv] for g [Hv]."""
    Q, K, V, dO, S0, dS = _f64(Q, K, V, dO, S0, dS)
    T, Hv, dv = V.shape
    Hk, dk = K.shape[1:]
    r, a = Hv // Hk, np.exp(_decay(g, T, Hv))
    S = [np.zeros((Hv, dk, dv)) if S0 is None else S0]
    for t in range(T):
        k = np.repeat(K[t], r, 0)
        S.append(a[t][:, None, None] * S[-1] + k[:, :, None] * V[t][:, None, :])
    G = np.zeros((Hv, dk, dv)) if dS is None else dS.copy()
    dQ, dK, dV, dg = np.zeros((T, Hv, dk)), np.zeros((T, Hv, dk)), np.zeros_like(V), np.zeros((T, Hv))
    for t in reversed(range(T)):
        q, k = np.repeat(Q[t], r, 0), np.repeat(K[t], r, 0)
        dQ[t] = scale * np.einsum("hkv,hv->hk", S[t + 1], dO[t])
        G = G + scale * q[:, :, None] * dO[t][:, None, :]
        dK[t] = np.einsum("hkv,hv->hk", G, V[t])
        dV[t] = np.einsum("hkv,hk->hv", G, k)
        G = a[t][:, None, None] * G
        dg[t] = np.sum(G * S[t], (1, 2))
    dQ, dK = (x.reshape(T, Hk, r, dk).sum(2) for x in (dQ, dK))
    return dQ, dK, dV, dg if np.ndim(g) == 2 else dg.sum(0), G


def linear_sizes(Q, K, V, g, dO=None, S0=None, dS=None, scale=1.0):
    """Sums of the magnitudes that results add up, which their roundings are relative to:
    (O, S) or, with dO, (dQ, dK, dV, dg, dS0).  dQ, dK and dV are the recurrence over other
    operands (the last two in reversed time, where a token's decay passes to the next row); dg
    is taken as the sum over the tokens after it of q . dQ + k . dK, and <S, dS>."""
    Q, K, V, dO, S0, dS = (None if x is None else np.abs(x) for x in _f64(Q, K, V, dO, S0, dS))
    T, Hv = V.shape[:2]
    r, g = Hv // K.shape[1], _decay(g, T, Hv)
    O, S = linear(Q, K, V, g, S0, scale)
    if dO is None:
        return O, S
    q, k = np.repeat(Q, r, 1), np.repeat(K, r, 1)
    tr = lambda x: None if x is None else x.transpose(0, 2, 1)  # noqa: E731
    dQ, _ = linear(dO, V, k, g, tr(S0), scale)
    back = np.concatenate([np.zeros((1, Hv)), g[::-1][:-1]])
    dK, dS0 = linear(V[::-1], scale * dO[::-1], q[::-1], back, tr(dS))
    dV, _ = linear(k[::-1], scale * q[::-1], dO[::-1], back, dS)
    dK, dV = dK[::-1], dV[::-1]
    each = np.einsum("thk,thk->th", q, dQ) + np.einsum("thk,thk->th", k, dK)
    dg = np.cumsum(each[::-1], 0)[::-1] + (0 if dS is None else np.sum(S * dS, (1, 2)))
    group = lambda x: x.reshape(T, -1, r, x.shape[-1]).sum(2)  # noqa: E731
    return group(dQ), group(dK), dV, dg, np.exp(g[0])[:, None, None] * tr(dS0)


def _silu(z):
    s = 1.0 / (1.0 + np.exp(-z))
    return z * s, s * (1.0 + z * (1.0 - s))


def _spread(stat, x, groups):
    """A statistic of each (n, group) at every value of x [N, S, C]."""
    return np.repeat(stat, x.shape[2] // groups, 1)[:, None, :]


def _mean(x, groups):
    N, S, C = x.shape
    return x.reshape(N, S, groups, C // groups).mean((1, 3))


def group_norm(x, groups, w=None, b=None, z=None, act=False, eps=1e-5):
    """(y, mean, rstd) of x [N, S, C], channels last."""
    x, w, b, z = _f64(x, w, b, z)
    mean = _mean(x, groups)
    c = x - _spread(mean, x, groups)
    rstd = 1.0 / np.sqrt(_mean(c * c, groups) + eps)
    n = c * _spread(rstd, x, groups)
    n = n if w is None else n * w
    n = n if b is None else n + b
    y = _silu(n)[0] if act else n
    return (y if z is None else y * _silu(z)[0]), mean, rstd


def group_norm_grad(dy, x, groups, w=None, b=None, z=None, act=False, eps=1e-5):
    """(dx, dw, db, dz) of sum(y dy)."""
    dy, x, w, b, z = _f64(dy, x, w, b, z)
    _, mean, rstd = group_norm(x, groups, eps=eps)
    h = (x - _spread(mean, x, groups)) * _spread(rstd, x, groups)
    w = np.ones(x.shape[2]) if w is None else w
    n = h * w + (0.0 if b is None else b)
    y, dyn = _silu(n) if act else (n, 1.0)
    dz, dn = None, dy
    if z is not None:
        f, df = _silu(z)
        dz, dn = dy * y * df, dy * f
    dn = dn * dyn
    dh = dn * w
    dx = dh - _spread(_mean(dh, groups), x, groups)
    dx = (dx - h * _spread(_mean(dh * h, groups), x, groups)) * _spread(rstd, x, groups)
    return dx, (dn * h).sum((0, 1)), dn.sum((0, 1)), dz

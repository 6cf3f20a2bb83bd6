"""The layer's training and serving operators in fp64 numpy: the token
recurrence, its gradients by reverse accumulation token by token, and the
norms with their gradients.

Arrays are [tokens, heads, ...] of one sequence; the recurrence is written
with the matrices of its definition,
    S_t = a_t (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T,
    o_t = scale S_t^T q_t.
"""

from __future__ import annotations

import numpy as np

__all__ = ["recurrent", "recurrent_grad", "norm", "norm_grad", "token_decay"]


def _f64(*xs):
    return tuple(None if x is None else np.asarray(x, np.float64) for x in xs)


def token_decay(g, C):
    """Per-token log-decay from g, its cumulative sum within chunks of C."""
    g = np.asarray(g, np.float64)
    out = g.copy()
    inside = np.arange(1, len(g))[np.arange(1, len(g)) % C != 0]
    out[inside] -= g[inside - 1]
    return out


def recurrent(Q, K, V, beta, logdecay, S0=None, scale=1.0):
    """(O [T, Hv, dv], S [Hv, dk, dv]) of one sequence; Q, K [T, Hk, dk] with
    value head h reading key head h // (Hv // Hk)."""
    Q, K, V, beta, logdecay, S0 = _f64(Q, K, V, beta, logdecay, S0)
    T, Hk, dk = K.shape
    Hv, dv = V.shape[1:]
    S = np.zeros((Hv, dk, dv)) if S0 is None else S0.copy()
    O = np.zeros((T, Hv, dv))
    for h in range(Hv):
        hk = h // (Hv // Hk)
        for t in range(T):
            k, q = K[t, hk], Q[t, hk]
            M = np.exp(logdecay[t, h]) * (np.eye(dk) - beta[t, h] * np.outer(k, k))
            S[h] = M @ S[h] + beta[t, h] * np.outer(k, V[t, h])
            O[t, h] = scale * S[h].T @ q
    return O, S


def recurrent_grad(Q, K, V, beta, logdecay, dO, S0=None, dS=None, scale=1.0):
    """(dQ, dK, dV, dbeta, d logdecay, dS0) of sum(O dO) + sum(S dS)."""
    Q, K, V, beta, logdecay, dO, S0, dS = _f64(Q, K, V, beta, logdecay, dO, S0, dS)
    T, Hk, dk = K.shape
    Hv, dv = V.shape[1:]
    dQ, dK, dV = np.zeros_like(Q), np.zeros_like(K), np.zeros_like(V)
    db, dl = np.zeros_like(beta), np.zeros_like(logdecay)
    dS0 = np.zeros((Hv, dk, dv))
    for h in range(Hv):
        hk = h // (Hv // Hk)
        S = [np.zeros((dk, dv)) if S0 is None else S0[h]]
        for t in range(T):
            k, a, b = K[t, hk], np.exp(logdecay[t, h]), beta[t, h]
            S.append(a * (S[-1] - b * np.outer(k, k @ S[-1])) + b * np.outer(k, V[t, h]))
        G = np.zeros((dk, dv)) if dS is None else dS[h].copy()
        for t in reversed(range(T)):
            k, q, v, b = K[t, hk], Q[t, hk], V[t, h], beta[t, h]
            a, do = np.exp(logdecay[t, h]), scale * dO[t, h]
            M = a * S[t]  # the decayed state
            e = v - M.T @ k
            dQ[t, hk] += S[t + 1] @ do
            G = G + np.outer(q, do)
            Gk = G.T @ k
            dV[t, h] = b * Gk
            db[t, h] = Gk @ e
            dK[t, hk] += b * (G @ e) - b * (M @ Gk)
            dM = G - b * np.outer(k, Gk)
            dl[t, h] = np.sum(dM * M)
            G = a * dM
        dS0[h] = G
    return dQ, dK, dV, db, dl, dS0


def _silu(z):
    s = 1.0 / (1.0 + np.exp(-z))
    return z * s, s * (1.0 + z * (1.0 - s))


def norm(x, w=None, b=None, z=None, layer=False, eps=1e-6):
    """(y, mean, rstd) of rows x [rows, D]."""
    x, w, b, z = _f64(x, w, b, z)
    mean = x.mean(1) if layer else np.zeros(len(x))
    c = x - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).mean(1) + eps)
    y = c * rstd[:, None]
    y = y if w is None else y * w
    y = y if b is None else y + b
    return (y if z is None else y * _silu(z)[0]), mean, rstd


def norm_grad(dy, x, w=None, b=None, z=None, layer=False, eps=1e-6):
    """(dx, dw, db, dz) of sum(y dy); the Jacobian of a row's xh is
    rstd (I - xh xh^T / D [- 1 1^T / D])."""
    dy, x, w, b, z = _f64(dy, x, w, b, z)
    D = x.shape[1]
    xh, _, rstd = norm(x, layer=layer, eps=eps)
    w = np.ones(D) if w is None else w
    n = xh * w + (0.0 if b is None else b)
    dz, dn = None, dy
    if z is not None:
        f, df = _silu(z)
        dz, dn = dy * n * df, dy * f
    dh = dn * w
    dx = dh - xh * (dh * xh).sum(1, keepdims=True) / D
    if layer:
        dx = dx - dh.sum(1, keepdims=True) / D
    return dx * rstd[:, None], (dn * xh).sum(0), dn.sum(0), dz

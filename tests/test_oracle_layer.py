"""The fp64 oracle of the layer's operators, checked against the existing
forward oracle and against central differences (CPU)."""

import numpy as np
import pytest

from oracle import layer


def _seq(rng, T, Hk, Hv, dk, dv):
    unit = lambda *s: (lambda z: z / np.linalg.norm(z, axis=-1, keepdims=True))(rng.normal(size=s))
    return (unit(T, Hk, dk), unit(T, Hk, dk), rng.normal(size=(T, Hv, dv)),
            1 / (1 + np.exp(-rng.normal(size=(T, Hv)))),
            -np.log1p(np.exp(rng.normal(size=(T, Hv)) - 1)), rng.normal(size=(Hv, dk, dv)))


def test_recurrent_is_the_forward_oracle_s_recurrence():
    from oracle import gdn_forward as gf

    rng = np.random.default_rng(1)
    T, C, Hk, Hv = 32, 16, 2, 4
    Q, K, V, beta, l, S0 = _seq(rng, T, Hk, Hv, 8, 6)
    O, S = layer.recurrent(Q, K, V, beta, l, S0, scale=0.3)
    g = np.concatenate([np.cumsum(l[:C], 0), np.cumsum(l[C:], 0)])
    assert np.allclose(layer.token_decay(g, C), l, atol=1e-14)
    wide = lambda x: np.repeat(x, Hv // Hk, 1)[None]
    Of, Sf = gf.gdn_recurrent(wide(Q), wide(K), V[None], beta[None], g[None], C, S0[None],
                              scale=0.3)
    assert np.allclose(O, Of[0], atol=1e-12) and np.allclose(S, Sf[0], atol=1e-12)


@pytest.mark.parametrize("Hk,Hv", [(1, 1), (1, 2)])
def test_recurrent_grad_is_the_difference_quotient(Hk, Hv):
    rng = np.random.default_rng(2)
    T, dk, dv = 5, 4, 3
    x = list(_seq(rng, T, Hk, Hv, dk, dv))
    dO, dS = rng.normal(size=(T, Hv, dv)), rng.normal(size=(Hv, dk, dv))

    def loss(xs):
        O, S = layer.recurrent(*xs[:5], xs[5], scale=0.7)
        return np.sum(O * dO) + np.sum(S * dS)

    got = layer.recurrent_grad(*x[:5], dO, x[5], dS, scale=0.7)
    for i, grad in enumerate(got):
        for at in np.ndindex(*x[i].shape):
            xs = [v.copy() for v in x]
            xs[i][at] += 1e-5
            up = loss(xs)
            xs[i][at] -= 2e-5
            # central differences: error h^2 f'''/6 + eps |f| / h ~ 1e-9
            assert abs((up - loss(xs)) / 2e-5 - grad[at]) < 1e-7, (i, at)


@pytest.mark.parametrize("ln", [False, True])
@pytest.mark.parametrize("gate", [False, True])
def test_norm_grad_is_the_difference_quotient(ln, gate):
    rng = np.random.default_rng(3)
    x, w, b = rng.normal(size=(3, 5)), rng.normal(size=5), rng.normal(size=5)
    z = rng.normal(size=(3, 5)) if gate else None
    dy = rng.normal(size=(3, 5))
    got = layer.norm_grad(dy, x, w, b, z, ln, 1e-3)
    arrays = [x, w, b] + ([z] if gate else [])
    for i, a in enumerate(arrays):
        for at in np.ndindex(*a.shape):
            vals = []
            for h in (1e-5, -1e-5):
                xs = [v.copy() for v in arrays]
                xs[i][at] += h
                vals.append(np.sum(layer.norm(*xs[:3], xs[3] if gate else None, ln, 1e-3)[0] * dy))
            assert abs((vals[0] - vals[1]) / 2e-5 - got[i][at]) < 1e-7

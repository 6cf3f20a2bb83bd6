"""The fp64 oracle of linear attention with decay and of group norm, checked against the
definition over pairs of tokens and against central differences (CPU)."""

import numpy as np
import pytest

from oracle import layer, linear


def _seq(rng, T, Hk, Hv, dk, dv, per_token=True):
    g = -np.log1p(np.exp(rng.normal(size=(T, Hv) if per_token else Hv)))
    return [rng.normal(size=(T, Hk, dk)), rng.normal(size=(T, Hk, dk)), rng.normal(size=(T, Hv, dv)),
            g, rng.normal(size=(Hv, dk, dv))]


def test_linear_is_the_sum_over_pairs():
    rng = np.random.default_rng(1)
    Q, K, V, g, S0 = _seq(rng, 9, 1, 2, 4, 3)
    O, S = linear.linear(Q, K, V, g, S0, scale=0.3)
    G = np.cumsum(g, 0)
    for h in range(2):
        P = np.tril((Q[:, 0] @ K[:, 0].T) * np.exp(G[:, None, h] - G[None, :, h]))
        o = 0.3 * (P @ V[:, h] + np.exp(G[:, h])[:, None] * (Q[:, 0] @ S0[h]))
        assert np.allclose(O[:, h], o, atol=1e-12)
        w = np.exp(G[-1, h] - G[:, h])[:, None]
        assert np.allclose(S[h], np.exp(G[-1, h]) * S0[h] + (w * K[:, 0]).T @ V[:, h], atol=1e-12)


def test_linear_is_the_delta_rule_without_its_correction():
    # keys that are orthogonal to each other meet no state: the correction is zero
    rng = np.random.default_rng(2)
    Q, _, V, g, _ = _seq(rng, 4, 2, 2, 4, 3)
    K = np.stack([np.eye(4), np.eye(4)[::-1]], 1)
    O, S = linear.linear(Q, K, V, g)
    Or, Sr = layer.recurrent(Q, K, V, np.ones((4, 2)), g)
    assert np.allclose(O, Or, atol=1e-13) and np.allclose(S, Sr, atol=1e-13)


@pytest.mark.parametrize("Hk,Hv,per_token", [(1, 1, True), (1, 2, True), (1, 2, False)])
def test_linear_grad_is_the_difference_quotient(Hk, Hv, per_token):
    rng = np.random.default_rng(3)
    x = _seq(rng, 5, Hk, Hv, 4, 3, per_token)
    dO, dS = rng.normal(size=(5, Hv, 3)), rng.normal(size=(Hv, 4, 3))

    def loss(xs):
        O, S = linear.linear(*xs, scale=0.7)
        return np.sum(O * dO) + np.sum(S * dS)

    got = linear.linear_grad(*x[:4], dO, x[4], dS, scale=0.7)
    for i, grad in enumerate(got):
        for at in np.ndindex(*x[i].shape):
            xs = [v.copy() for v in x]
            xs[i][at] += 1e-5
            up = loss(xs)
            xs[i][at] -= 2e-5
            # central differences: error h^2 f'''/6 + eps |f| / h ~ 1e-9
            assert abs((up - loss(xs)) / 2e-5 - grad[at]) < 1e-7, (i, at)


def test_sizes_are_the_results_of_positive_operands():
    # of operands that are all positive nothing cancels: sizes and results are the same
    rng = np.random.default_rng(4)
    Q, K, V, g, S0 = _seq(rng, 7, 1, 3, 4, 2)
    Q, K, V, S0 = (np.abs(x) for x in (Q, K, V, S0))
    dO, dS = rng.random((7, 3, 2)), rng.random((3, 4, 2))
    got = linear.linear_grad(Q, K, V, g, dO, S0, dS, scale=0.7)
    size = linear.linear_sizes(Q, K, V, g, dO, S0, dS, scale=0.7)
    for i in (0, 1, 2, 4):
        assert np.allclose(got[i], size[i], atol=1e-12), i
    assert (size[3] >= np.abs(got[3]) - 1e-12).all()


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("gate", [False, True])
def test_group_norm_grad_is_the_difference_quotient(act, gate):
    rng = np.random.default_rng(5)
    x, w, b = rng.normal(size=(2, 3, 6)), rng.normal(size=6), rng.normal(size=6)
    z, dy = rng.normal(size=(2, 3, 6)) if gate else None, rng.normal(size=(2, 3, 6))
    got = linear.group_norm_grad(dy, x, 2, w, b, z, act, 1e-3)
    arrays = [x, w, b] + ([z] if gate else [])
    for i, a in enumerate(arrays):
        for at in np.ndindex(*a.shape):
            vals = []
            for h in (1e-5, -1e-5):
                xs = [v.copy() for v in arrays]
                xs[i][at] += h
                y = linear.group_norm(xs[0], 2, xs[1], xs[2], xs[3] if gate else None, act, 1e-3)[0]
                vals.append(np.sum(y * dy))
            assert abs((vals[0] - vals[1]) / 2e-5 - got[i][at]) < 1e-7


def test_one_group_a_row_is_layer_norm():
    rng = np.random.default_rng(6)
    x, w, b = rng.normal(size=(4, 1, 10)), rng.normal(size=10), rng.normal(size=10)
    y, mean, rstd = linear.group_norm(x, 1, w, b, eps=1e-3)
    yl, ml, rl = layer.norm(x[:, 0], w, b, layer=True, eps=1e-3)
    assert np.allclose(y[:, 0], yl, atol=1e-13) and np.allclose(mean[:, 0], ml, atol=1e-13)
    assert np.allclose(rstd[:, 0], rl, atol=1e-13)

"""What the GPU tests of group norm's gradients can see, on the CPU: their reference is the oracle's
formula, and with a mean of dx's left in it is far outside of what they allow."""

import numpy as np
import pytest

from oracle import linear
from test_gpu_group_norm_sums import MANY, SHAPES, make, reference

CASES = [(min(N, 300), S, C, g) for N, S, C, g in SHAPES + MANY if min(N, 300) * S * C <= 1 << 21]


@pytest.mark.parametrize("act,bias,gate", [(None, False, True), ("silu", True, False),
                                           ("silu", True, True), (None, True, False)])
@pytest.mark.parametrize("N,S,C,groups", CASES)
def test_reference(N, S, C, groups, act, bias, gate):
    x, w, b, z, dy = make(N, S, C, groups, "f32", "f32", bias, gate, N + S + C, "cpu")
    got = reference(x, w, b, z, dy, groups, act, 1e-3)
    n = [None if t is None else t.double().numpy() for t in (dy, x, w, b, z)]
    want = linear.group_norm_grad(n[0], n[1], groups, *n[2:], act is not None, 1e-3)
    for p, q in zip(got[:4], want):
        assert (p is None and q is None) or np.allclose(p.numpy(), q, rtol=1e-9, atol=1e-9)
    # bf16 results are held to 1e-5 and half a step
    for means in ((0, 1), (1, 0), (1.05, 1), (1, 1.05)):
        off = (reference(x, w, b, z, dy, groups, act, 1e-3, means)[0] - got[0]).norm()
        few = 5 if max(means) == 1 else 1
        assert off > few * (1e-5 + 2.0 ** -8) * got[0].norm(), means

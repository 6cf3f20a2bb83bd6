"""The example model: it learns to repeat what it has seen, and serving it token by token from
the prompt's states gives the logits of the whole sequence."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "gated_delta_block.py")


def load():
    spec = importlib.util.spec_from_file_location("gated_delta_block", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


# Served and whole logits differ by the order of the sums alone in fp32 (some tens of roundings
# of 2^-24 a layer, grown by the norms: 1e-4 leaves a hundredfold); in bf16 by roundings of
# activations to 2^-9 that fall differently, a dozen a layer in two layers.
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-4), (torch.bfloat16, 5e-2)])
def test_learns_and_serves(dtype, tol):
    first, last, diff = load().run(60, dtype, log=lambda *_: None)
    assert first > 3.0  # about log(32) at the start
    assert last < 0.1
    assert diff <= tol

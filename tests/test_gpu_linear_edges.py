"""Linear attention and group norm at the edges of what their entry points take, on the GPU."""

import pytest
import torch

import paper_2606_06034_amd as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 64, 512])
def test_packed_tokens_of_no_sequence(T, dt):
    """The gradient of a head's decay is 0 and nothing else is written, whatever lies behind the
    one offset (here the end of a sequence that is none)."""
    torch.manual_seed(T)
    q, k = (torch.randn(1, T, 2, 64, device="cuda").to(dt) for _ in range(2))
    v, dO = (torch.randn(1, T, 4, 64, device="cuda").to(dt) for _ in range(2))
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")[:1]
    for g in (torch.full((4,), -0.1, device="cuda"), torch.full((1, T, 4), -0.1, device="cuda")):
        print(T, dt, g.dim(), flush=True)
        out = [torch.full_like(t, 7.0) for t in (q, k, v, g)]
        got = G.gdn_linear_backward(q, k, v, g, dO, out=out + [None], want_dS0=True, cu_seqlens=cu)
        torch.cuda.synchronize()
        assert got[4].shape == (0, 4, 64, 64)
        assert all((t == 7).all() for t in got[:3])
        assert (got[3] == (0 if g.dim() == 1 else 7)).all()
        O = torch.full_like(v, 7.0)
        for f in (G.gdn_linear_forward, G.gdn_linear_recurrent):
            _, S = f(q, k, v, g, cu_seqlens=cu, O=O)
            assert S.shape == (0, 4, 64, 64) and (O == 7).all()


def test_group_norm_without_a_gate_has_no_gradient_of_one():
    x = torch.randn(5, 3, 16, device="cuda")
    w = torch.ones(16, device="cuda")
    _, mean, rstd = G.gdn_group_norm_forward(x, 2, w)
    dz = torch.full_like(x, 7.0)
    got = G.gdn_group_norm_backward(x, x, 2, w, mean, rstd, dz=dz)
    assert got[3] is None and (dz == 7).all()
    got = G.gdn_group_norm_backward(x, x, 2, w, mean, rstd, gate=x, dz=dz)
    assert got[3] is dz and not (dz == 7).any()


def test_group_norm_gradient_of_rows_alone():
    """Without dw and db, and without a workspace, dx is what it is with them."""
    x, dy, z = (torch.randn(300, 64, device="cuda") for _ in range(3))
    w = torch.rand(64, device="cuda")
    _, mean, rstd = G.gdn_group_norm_forward(x, 4, w, gate=z)
    want = G.gdn_group_norm_backward(dy, x, 4, w, mean, rstd, gate=z)
    dx, dz = torch.empty_like(x), torch.empty_like(x)
    code = G.lib.gdn_group_norm_backward(
        dy.data_ptr(), x.data_ptr(), w.data_ptr(), None, z.data_ptr(), mean.data_ptr(),
        rstd.data_ptr(), dx.data_ptr(), None, None, dz.data_ptr(), None, 0, 300, 1, 64, 4, 0, 0, 0,
        torch.cuda.current_stream().cuda_stream)
    assert code == 0 and torch.equal(dx, want[0]) and torch.equal(dz, want[3])

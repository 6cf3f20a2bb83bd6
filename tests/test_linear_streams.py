"""Calls of linear attention and group norm that name a stream, or a device: as the layer's
(test_streams.py)."""

import pytest
import torch

import paper_2606_06034_amd as G
import test_streams
from paper_2606_06034_amd import _linear
from test_streams import Stream


@pytest.fixture
def played(monkeypatch):
    """test_streams' streams without a GPU, for these operators too."""
    lib, log, marked = test_streams.played.__wrapped__(monkeypatch) if hasattr(
        test_streams.played, "__wrapped__") else test_streams.played.__pytest_wrapped__.obj(
            monkeypatch)
    monkeypatch.setattr(_linear, "lib", lib)
    monkeypatch.setattr(_linear, "_dev", lambda t, *a: t.data_ptr())
    monkeypatch.setattr(_linear, "_params", lambda w, b, C: (w.data_ptr(), None, 0))
    return lib, log, marked


def operands(dev="cpu", dt=torch.float32, T=600, H=2, d=64):
    gen = torch.Generator().manual_seed(T)

    def r(*s):
        return torch.randn(*s, generator=gen).to(dev)

    x = {k: r(1, T, H, d).to(dt) for k in ("Q", "K", "V", "dO")}
    return dict(x, g=-torch.rand(1, T, H, generator=gen).to(dev), w=r(H * d).to(dt),
                z=r(1, T, H * d).to(dt))


def calls(x):
    seq = [x[k] for k in ("Q", "K", "V", "g")]
    T, dev = x["V"].shape[1], x["V"].device
    cu = torch.tensor([0, 100, T], dtype=torch.int32, device=dev)
    row, map_ = x["V"].flatten(2)[0], x["V"].flatten(2)
    stat = torch.ones(T, 2, device=dev)
    return {
        "forward": lambda s: G.gdn_linear_forward(*seq, stream=s),
        "forward_packed": lambda s: G.gdn_linear_forward(*seq, cu_seqlens=cu, stream=s),
        "backward": lambda s: G.gdn_linear_backward(*seq, x["dO"], want_dS0=True, stream=s),
        "backward_packed": lambda s: G.gdn_linear_backward(*seq, x["dO"], cu_seqlens=cu, stream=s),
        "recurrent": lambda s: G.gdn_linear_recurrent(*seq, stream=s),
        "norm": lambda s: G.gdn_group_norm_forward(row, 2, x["w"], gate=x["z"][0], stream=s),
        "norm_map": lambda s: G.gdn_group_norm_forward(map_, 2, x["w"], act="silu", stream=s),
        "norm_backward": lambda s: G.gdn_group_norm_backward(row, row, 2, x["w"], stat, stat,
                                                             gate=x["z"][0], stream=s),
        "norm_map_backward": lambda s: G.gdn_group_norm_backward(
            map_, map_, 2, x["w"], stat[:1], stat[:1], act="silu", stream=s),
    }


ALL = sorted(calls(operands()))


@pytest.mark.parametrize("name", ALL)
def test_a_call_allocates_on_the_stream_it_names(played, name):
    lib, log, marked = played
    call = calls(operands())[name]
    log.clear()
    out = [t for t in call(Stream(2)) if t is not None]
    assert lib.launched == [2]
    assert log and all(s == 2 for _, s in log), log
    # the results are used on the caller's stream: not handed out before its work ends
    assert {t.data_ptr() for t in out} == {p for p, s in marked if s == 1}


@pytest.mark.parametrize("name", ALL)
def test_a_call_without_a_stream_stays_on_the_current_one(played, name):
    lib, log, marked = played
    call = calls(operands())[name]
    log.clear()
    call(None)
    assert lib.launched == [1] and log and all(s == 1 for _, s in log) and not marked


def test_a_call_that_allocates_nothing_changes_no_stream(played, monkeypatch):
    lib, log, marked = played
    x = operands()
    seq = [x[k] for k in ("Q", "K", "V", "g")]
    O, S = torch.zeros_like(x["V"]), torch.zeros(1, 2, 64, 64)
    out = [torch.zeros_like(t) for t in seq] + [S]
    ws = torch.zeros(G.gdn_linear_backward_workspace(1, 600, 2, 2, 64, 64), dtype=torch.uint8)
    monkeypatch.setattr(torch.cuda, "set_stream", None)
    log.clear()
    G.gdn_linear_recurrent(*seq, S0=S, S_final=S, O=O, stream=Stream(2))
    G.gdn_linear_forward(*seq, O=O, S_final=S, workspace=ws, stream=Stream(2))
    G.gdn_linear_backward(*seq, x["dO"], want_dS0=True, out=out, workspace=ws, stream=Stream(2))
    assert lib.launched == [2] * 3 and not log and not marked


class OnDevice1:
    """What the checks ask a contiguous tensor of the second device."""
    is_cuda, dtype, device = True, torch.float32, "cuda:1"

    def is_contiguous(self):
        return True

    def get_device(self):
        return 1

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return 4


def test_another_device_than_the_current_one_is_refused(monkeypatch):
    monkeypatch.setattr(_linear, "_device", lambda: 0)
    with pytest.raises(ValueError, match="x is on cuda:1, not on the current device"):
        _linear._dev(OnDevice1(), "x", torch.float32, 4)
    with pytest.raises(ValueError, match="bias is on cuda:1"):
        _linear._affine(None, OnDevice1(), 4)
    monkeypatch.setattr(_linear, "_device", lambda: 1)
    assert _linear._dev(OnDevice1(), "x", torch.float32, 4) == 1 << 20


@pytest.mark.gpu
def test_a_refused_device_launches_nothing(monkeypatch):
    x = operands("cuda", T=3)
    monkeypatch.setattr(_linear, "_device", lambda: 7)
    for call in calls(operands("cuda", T=128)).values():
        with pytest.raises(ValueError, match="not on the current device"):
            call(None)
    O = torch.full_like(x["V"], 3.0)
    with pytest.raises(ValueError, match="not on the current device"):
        G.gdn_linear_recurrent(*(x[k] for k in ("Q", "K", "V", "g")), O=O)
    torch.cuda.synchronize()
    assert (O == 3).all()


@pytest.mark.gpu
@pytest.mark.parametrize("name", ALL)
def test_results_on_a_named_stream(name):
    """Bit for bit those of the current stream, three times, while the caller goes on."""
    call = calls(operands("cuda", torch.bfloat16))[name]
    want = [t for t in call(None) if t is not None]
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        got = [t for t in call(side) if t is not None]
        busy = torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.current_stream().wait_stream(side)
        got = [t.clone() for t in got]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and (busy == 255).all()

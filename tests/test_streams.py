"""Calls that name a stream.

What a call allocates by itself has to belong to the stream that its kernels run
on: a workspace of another stream's memory is handed out again as soon as the
call returns and drops it, while the kernels still use it.  On the CPU the calls
run up to the library with the streams played by a stack; on the GPU the memory
of a dropped workspace is looked for in what the caller's stream gets next."""

import pytest
import torch

import paper_2606_06034_amd as G
from paper_2606_06034_amd import _binding, _layer


class Library:
    """The library's own sizes of workspaces and defaults; its launches note the stream."""

    def __init__(self, now):
        self.now, self.launched = now, []

    def __getattr__(self, name):
        if name.endswith("_workspace") or name == "gdn_default_order":
            return getattr(G.lib, name)

        def launch(*args):
            self.launched.append(args[-1])
            return 0

        return launch


class Stream:
    device_index, device = 0, "cuda:0"

    def __init__(self, number):
        self.cuda_stream = number


@pytest.fixture
def played(monkeypatch):
    """Streams without a GPU: every allocation and launch with the stream it was made on."""
    now, log = [Stream(1)], []

    def noting(make):
        def f(*a, **k):
            t = make(*a, **k)
            log.append((t.data_ptr(), now[-1].cuda_stream))
            return t

        return f

    lib = Library(lambda: now[-1])
    marked = []
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, noting(getattr(torch, name)))
    new_empty = torch.Tensor.new_empty
    monkeypatch.setattr(torch.Tensor, "new_empty", noting(new_empty))
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: marked.append((t.data_ptr(), s.cuda_stream)))
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "set_stream", now.append)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: now[-1])
    monkeypatch.setattr(_layer, "_raw_stream", None)
    for m in (_binding, _layer):
        monkeypatch.setattr(m, "lib", lib)
        monkeypatch.setattr(m, "_dev", lambda t, *a: t.data_ptr())
    return lib, log, marked


def operands(dev="cpu", dt=torch.float32, B=1, L=128, H=2, d=64):
    gen = torch.Generator().manual_seed(L)

    def r(*s):
        return torch.randn(*s, generator=gen)

    x = dict(Q=r(B, L, H, d) * d ** -0.5, K=torch.nn.functional.normalize(r(B, L, H, d), dim=-1),
             V=r(B, L, H, d), dO=r(B, L, H, d), beta=torch.sigmoid(r(B, L, H)),
             g=-0.01 * torch.arange(L).remainder(64).add(1).float().expand(B, H, L).mT.contiguous())
    return {k: (v.to(dt) if k in ("Q", "K", "V", "dO") else v).to(dev) for k, v in x.items()}


def layer_calls(x):
    """name -> call(stream) of the layer's training and serving operators."""
    seq = [x[k] for k in ("Q", "K", "V", "beta", "g")]
    row = x["V"].flatten(0, 2)
    w = torch.ones(row.shape[1], device=row.device)
    rstd = torch.ones(len(row), device=row.device)
    cu = (torch.tensor([0, 100, 128], dtype=torch.int32, device=row.device), None, 0)
    return {
        "recurrent": lambda s: G.gdn_recurrent_forward(*seq, stream=s),
        "backward": lambda s: G.gdn_chunk_backward(*seq, x["dO"], 64, want_dS0=True, stream=s),
        "backward_varlen": lambda s: G.gdn_chunk_backward_varlen(*seq, x["dO"], cu, 64,
                                                                 want_dS0=True, stream=s),
        "norm": lambda s: G.gdn_norm_forward(row, w, gate=row, stream=s),
        "norm_backward": lambda s: G.gdn_norm_backward(row, row, w, rstd, gate=row, stream=s),
    }


def chunk_calls(x):
    """The same of the chunk-wise forward and the inverses."""
    seq = [x[k] for k in ("Q", "K", "V", "beta", "g")]
    K, V, beta, g = seq[1:]
    dev = K.device
    A = 0.1 * torch.tril(torch.ones(3, 64, 64, device=dev), -1)
    codes = torch.zeros(3, 64, 64, dtype=torch.int8, device=dev)
    e = torch.zeros(3, dtype=torch.int32, device=dev)
    packed = G.gdn_varlen_tables([0, 100, 128], 64, device=dev)
    T = torch.zeros(K.shape[0], K.shape[2], 2, 64, 64, dtype=K.dtype, device=dev)
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device=dev)
    return {
        "forward": lambda s: G.gdn_chunk_forward(*seq, 64, stream=s),
        "forward_varlen": lambda s: G.gdn_chunk_forward_varlen(*seq, packed, 64, stream=s),
        "forward_state": lambda s: G.gdn_chunk_forward_state(
            seq[0], g, 64, G.gdn_chunk_forward_prepare(*seq, 64, ws, stream=s), V.shape[-1],
            stream=s),
        "build_A": lambda s: (G.gdn_build_A(K, beta, g, 64, stream=s),),
        "neumann": lambda s: (G.gdn_chunk_inverse_neumann(A, 3, 8, stream=s),),
        "fwdsub": lambda s: (G.gdn_chunk_inverse_fwdsub(A, stream=s),),
        "blockwise": lambda s: (G.gdn_chunk_inverse_blockwise(A, stream=s),),
        "wy_apply": lambda s: G.gdn_wy_apply(T, K, V, beta, 64, stream=s),
        "wy_fused": lambda s: G.gdn_chunk_wy_fused(K, V, beta, g, 64, 3, 8, stream=s),
        "wy_fused_blockwise": lambda s: G.gdn_chunk_wy_fused_blockwise(K, V, beta, g, 64, stream=s),
        "wy_fused_varlen": lambda s: G.gdn_chunk_wy_fused_varlen(K, V, beta, g, packed, 64,
                                                                 stream=s),
        "quantize_i8": lambda s: G.gdn_quantize_tiles_i8(A, stream=s),
        "inverse_i8": lambda s: G.gdn_chunk_inverse_neumann_i8(codes, e, 3, 8, stream=s),
        "fused_i8": lambda s: G.gdn_chunk_inverse_neumann_i8_fused(K, beta, g, 64, 3, 8, stream=s),
        "fwdsub_i8": lambda s: G.gdn_chunk_inverse_fwdsub_i8(codes, e, stream=s),
        "quantize_i16": lambda s: G.gdn_quantize_tiles_i16(A, stream=s),
        "inverse_i16": lambda s: G.gdn_chunk_inverse_neumann_i16(codes.short(), e, 3, 8, stream=s),
        "fused_i16": lambda s: G.gdn_chunk_inverse_neumann_i16_fused(K, beta, g, 64, 3, 8,
                                                                     stream=s),
        "fwdsub_i16": lambda s: G.gdn_chunk_inverse_fwdsub_i16(codes.short(), e, stream=s),
    }


def calls(x):
    return {**layer_calls(x), **chunk_calls(x)}


LAYER = sorted(layer_calls(operands()))
ALL = sorted(calls(operands()))


@pytest.mark.parametrize("name", ALL)
def test_a_call_allocates_on_the_stream_it_names(played, name):
    lib, log, marked = played
    call = calls(operands())[name]
    log.clear()
    out = [t for t in call(Stream(2)) if t is not None]
    assert set(lib.launched) == {2}
    assert log and all(s == 2 for _, s in log), log
    # the results are used on the caller's stream: not handed out before its work ends
    assert {t.data_ptr() for t in out} == {p for p, s in marked if s == 1}


@pytest.mark.parametrize("name", ALL)
def test_a_call_without_a_stream_stays_on_the_current_one(played, name):
    lib, log, marked = played
    call = calls(operands())[name]
    log.clear()
    call(None)
    assert set(lib.launched) == {1} and log and all(s == 1 for _, s in log) and not marked


@pytest.mark.gpu
@pytest.mark.parametrize("name", LAYER + ["forward", "forward_varlen"])
def test_results_on_a_named_stream(name):
    """Bit for bit those of the current stream; the memory of a dropped workspace is not
    what the caller's stream gets next."""
    x = operands("cuda", torch.bfloat16, 2, 128, 4, 128) if "varlen" not in name else \
        operands("cuda", torch.bfloat16, 1, 128, 4, 128)
    call = calls(x)[name]
    want = [t for t in call(None) if t is not None]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()  # (want's own workspace goes back)
    side, got, taken = torch.cuda.Stream(), [], []
    empty = torch.empty

    def noting(*a, **k):
        t = empty(*a, **k)
        taken.append((t.data_ptr(), t.numel() * t.element_size()))
        return t

    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        torch.empty = noting
        try:
            out = [t for t in call(side) if t is not None]
        finally:
            torch.empty = empty
        # at once on the caller's stream, while the call may still run
        mine = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _, n in taken]
        at = {p for p, _ in taken}
        assert not at & {t.data_ptr() for t in mine}
        torch.cuda.current_stream().wait_stream(side)
        got.append([t.clone() for t in out])
        del out, mine
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


@pytest.mark.gpu
def test_a_stream_from_outside_torch():
    """Any object with the handle of a stream is taken."""
    x = operands("cuda", torch.float32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    class Foreign:
        cuda_stream = side.cuda_stream

    call = layer_calls(x)["backward"]
    got = call(Foreign())
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, call(None)))


def test_a_call_that_allocates_nothing_changes_no_stream(played, monkeypatch):
    lib, log, marked = played
    x = operands()
    seq = [x[k] for k in ("Q", "K", "V", "beta", "g")]
    O, S = torch.zeros_like(x["V"]), torch.zeros(1, 2, 64, 64)
    out = [torch.zeros_like(t) for t in seq] + [S]
    ws = torch.zeros(G.gdn_chunk_backward_workspace(1, 128, 2, 64, 64), dtype=torch.uint8)
    monkeypatch.setattr(torch.cuda, "set_stream", None)
    log.clear()
    G.gdn_recurrent_forward(*seq, S0=S, S_final=S, O=O, stream=Stream(2))
    G.gdn_chunk_backward(*seq, x["dO"], 64, want_dS0=True, out=out, workspace=ws, stream=Stream(2))
    G.gdn_norm_forward(x["V"], y=O, want_stats=False, stream=Stream(2))
    G.gdn_chunk_forward(*seq, 64, O=O, S_final=S, workspace=ws, stream=Stream(2))
    assert lib.launched == [2] * 4 and not log and not marked

"""A small language model of gated delta rule blocks, trained and then run token by token.

    python examples/gated_delta_block.py [--steps 60] [--dtype bf16]

Each block is RMS norm -> q, k, v, gates -> gated delta rule -> norm with SiLU gate -> output
projection, on a residual.  Training runs the layer over whole sequences (gdn_chunk_forward with
the exact inverse, its gradients from gdn_chunk_backward; gdn_norm_forward, gdn_norm_backward).
Serving runs the prompt the same way, keeps its final states, and goes on with
gdn_recurrent_forward, which updates them in place.  The data are random tokens that repeat with
a fixed period, so that every period but the first can be predicted from the state.
"""

import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_06034_amd as G  # noqa: E402

C = 64  # tokens a chunk


class Norm(torch.autograd.Function):
    """RMS norm over the last dimension, times weight, times silu(gate)."""

    @staticmethod
    def forward(ctx, x, weight, gate):
        y, _, rstd = G.gdn_norm_forward(x, weight, gate=gate)
        ctx.save_for_backward(x, weight, gate, rstd)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, gate, rstd = ctx.saved_tensors
        dx, dw, _, dz = G.gdn_norm_backward(dy.contiguous(), x, weight, rstd, gate=gate)
        return dx, dw, dz


class DeltaRule(torch.autograd.Function):
    """O of the gated delta rule over whole sequences from a state of zeros; q and k may have
    fewer heads than v.  g: the log-decay summed up inside each chunk of C tokens."""

    @staticmethod
    def forward(ctx, q, k, v, beta, g):
        ctx.save_for_backward(q, k, v, beta, g)
        return prefill(q, k, v, beta, g, want_state=False)[0]

    @staticmethod
    def backward(ctx, dO):
        q, k, v, beta, g = ctx.saved_tensors
        return G.gdn_chunk_backward(q, k, v, beta, g, dO.contiguous(), C)[:5]


def prefill(q, k, v, beta, g, want_state=True):
    r = v.shape[2] // k.shape[2]
    q, k = (x.repeat_interleave(r, 2) for x in (q, k))  # the forward has a key head a value head
    return G.gdn_chunk_forward(q, k, v, beta, g, C, inverse="exact", want_state=want_state)


class Block(torch.nn.Module):
    def __init__(self, width, key_heads, value_heads, dim):
        super().__init__()
        self.shape = key_heads, value_heads, dim
        n = (2 * key_heads + 2 * value_heads) * dim + 2 * value_heads
        self.norm = torch.nn.Parameter(torch.ones(width))
        self.head_norm = torch.nn.Parameter(torch.ones(dim))
        self.w_in = torch.nn.Parameter(torch.randn(n, width) * width ** -0.5)
        self.w_out = torch.nn.Parameter(torch.randn(width, value_heads * dim) * 0.1 * width ** -0.5)

    def operands(self, x):
        """q, k, v, the gate z, beta and the log-decay of each token."""
        Hk, Hv, D = self.shape
        h = F.linear(Norm.apply(x, self.norm, None), self.w_in.to(x.dtype))
        q, k, v, z, b, a = h.split([Hk * D, Hk * D, Hv * D, Hv * D, Hv, Hv], -1)
        heads = lambda t, H: t.unflatten(-1, (H, D)).contiguous()
        unit = lambda t: F.normalize(heads(t, Hk).float(), dim=-1).to(x.dtype)
        return (unit(q), unit(k), heads(v, Hv), heads(z, Hv), torch.sigmoid(b.float()).contiguous(),
                F.logsigmoid(a.float() + 6.0).contiguous())

    def result(self, x, o, z):
        o = Norm.apply(o, self.head_norm, z)
        return x + F.linear(o.flatten(-2), self.w_out.to(x.dtype))

    @staticmethod
    def chunk_sums(a):
        return a.unflatten(1, (-1, C)).cumsum(2).flatten(1, 2)

    def forward(self, x):  # training
        q, k, v, z, beta, a = self.operands(x)
        return self.result(x, DeltaRule.apply(q, k, v, beta, self.chunk_sums(a)), z)

    def start(self, x):  # serving: the prompt; its final state
        q, k, v, z, beta, a = self.operands(x)
        o, state = prefill(q, k, v, beta, self.chunk_sums(a).contiguous())
        return self.result(x, o, z), state

    def step(self, x, state):  # serving: the next tokens; the state is updated in place
        q, k, v, z, beta, a = self.operands(x)
        o, _ = G.gdn_recurrent_forward(q, k, v, beta, a, S0=state, S_final=state)
        return self.result(x, o, z)


class Model(torch.nn.Module):
    def __init__(self, vocab=32, width=256, layers=2, key_heads=2, value_heads=4, dim=64,
                 dtype=torch.bfloat16):
        super().__init__()
        self.dtype = dtype
        self.emb = torch.nn.Parameter(torch.randn(2, vocab, width // 2))
        self.blocks = torch.nn.ModuleList(
            Block(width, key_heads, value_heads, dim) for _ in range(layers))
        self.norm = torch.nn.Parameter(torch.ones(width))
        self.head = torch.nn.Parameter(torch.randn(vocab, width) * width ** -0.5)

    def embed(self, tokens, before=None):
        """A token and the one before it (of the first: token 0), so that a state can hold what
        follows a token."""
        before = torch.zeros_like(tokens[:, :1]) if before is None else before
        pair = torch.cat([before, tokens], 1)
        return torch.cat([F.embedding(pair[:, 1:], self.emb[0]),
                          F.embedding(pair[:, :-1], self.emb[1])], -1).to(self.dtype)

    def logits(self, x):
        return F.linear(Norm.apply(x, self.norm, None).float(), self.head)

    def forward(self, tokens):
        x = self.embed(tokens)
        for b in self.blocks:
            x = b(x)
        return self.logits(x)

    @torch.no_grad()
    def generate(self, prompt, given):
        """The logits of a prompt (a multiple of C tokens), then of the tokens `given` one by
        one, each from the states that the ones before it left."""
        x, states = self.embed(prompt), []
        for b in self.blocks:
            x, s = b.start(x)
            states.append(s)
        out = [self.logits(x)]
        for t in range(given.shape[1]):
            x = self.embed(given[:, t:t + 1], given[:, t - 1:t] if t else prompt[:, -1:])
            for b, s in zip(self.blocks, states):
                x = b.step(x, s)
            out.append(self.logits(x))
        return torch.cat(out, 1)


def batch(n, period, vocab, gen):
    """2 C tokens: different random ones, repeated."""
    t = torch.rand(n, vocab, generator=gen).argsort(1)[:, :period]
    return t.repeat(1, 2 * C // period).cuda()


def run(steps=60, dtype=torch.bfloat16, n=64, period=16, vocab=32, lr=3e-3, log=print):
    """(first loss, last loss, largest difference of the served logits relative to the largest
    logit); the losses are those after the first period."""
    torch.manual_seed(0)
    gen = torch.Generator().manual_seed(1)
    model = Model(vocab=vocab, dtype=dtype).cuda()
    opt = torch.optim.AdamW(model.parameters(), lr=lr, weight_decay=0.0)
    losses = []
    for i in range(steps):
        t = batch(n, period, vocab, gen)
        logits = model(t)
        loss = F.cross_entropy(logits[:, period:-1].flatten(0, 1), t[:, period + 1:].flatten())
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        if i % 20 == 0 or i == steps - 1:
            log(f"step {i:4d}  loss {losses[-1].item():.4f}")
    with torch.no_grad():
        t = batch(n, period, vocab, gen)
        whole = model(t)
        served = model.generate(t[:, :C], t[:, C:])
        diff = ((whole - served).abs().max() / whole.abs().max()).item()
    log(f"served token by token: logits within {diff:.2e} of the whole sequence's")
    return losses[0].item(), losses[-1].item(), diff


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = p.parse_args()
    run(a.steps, {"bf16": torch.bfloat16, "f32": torch.float32}[a.dtype])

"""A small language model whose blocks remember in matrices: the gated delta rule behind a short convolution, dropout in training; trained for some
steps, then served token by token.

    python examples/delta_block.py [--steps 400]

A block is  n -> projection -> (q, k, v, z) and the gates;  (q, k, v) -> causal depthwise convolution -> gated delta rule, two heads of values to a head
of keys -> dropout -> norm, gate, residual and the next block's norm.  The projections, the embedding and the loss are torch's; everything else is a call of
``binding`` and ``block``.  Serving keeps the convolution's ring and the heads' states of every sequence in a pool; the program checks the logits of
both ways against each other.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from gated_block import EPS, FirstNorm, Norms, batch      # noqa: E402
from paper_2604_25422_amd import binding, block           # noqa: E402


class Mixer(torch.autograd.Function):
    """(q, k, v side by side [B, channels, L], taps [channels, K], g and beta [B, H, L]) -> the rule's output on their convolution."""

    @staticmethod
    def forward(ctx, x, taps, g, beta, keys, key_heads):
        x = x.contiguous()                                      # (the convolution takes dense tensors)
        u = binding.dwconv_fwd(x, taps, taps.shape[1] - 1)
        q, k, v = u.split((keys, keys, u.shape[1] - 2 * keys), 1)
        o, _, states = block.delta_fwd(q, k, v, g, beta, key_heads=key_heads)
        ctx.save_for_backward(x, u, taps, g, beta, states)
        ctx.keys, ctx.key_heads = keys, key_heads
        return o

    @staticmethod
    def backward(ctx, do):
        x, u, taps, g, beta, states = ctx.saved_tensors
        parts = (ctx.keys, ctx.keys, u.shape[1] - 2 * ctx.keys)
        du = torch.empty_like(u)
        _, _, _, dg, dbeta, _ = block.delta_bwd(do.contiguous(), *u.split(parts, 1), g, beta, states, key_heads=ctx.key_heads, out=tuple(du.split(parts, 1)))
        dx, dtaps = binding.dwconv_bwd(du, x, taps, taps.shape[1] - 1)
        return dx, dtaps, dg, dbeta, None, None


class Dropout(torch.autograd.Function):
    """The mask is formed again from rng in the backward pass: rng must not be counted up in between."""

    @staticmethod
    def forward(ctx, x, p, rng, layer):
        ctx.p, ctx.rng, ctx.layer = p, rng, layer
        return block.dropout_fwd(x, p, rng, layer)

    @staticmethod
    def backward(ctx, dout):
        return block.dropout_bwd(dout.contiguous(), ctx.p, ctx.rng, ctx.layer), None, None, None


class Model:
    def __init__(self, vocabulary, heads, key_heads, D, K, blocks, seed, p=0.1):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, std):
            return (torch.randn(*shape, generator=g) * std).cuda().requires_grad_()
        self.H, self.Hk, self.C, self.keys, self.K, self.p = heads, key_heads, heads * D, key_heads * D, K, p
        self.mixed = 2 * self.keys + self.C                     # channels of q, k, v
        self.scale = 1 / math.sqrt(2 * blocks)
        self.rng = torch.tensor([seed, 0], device="cuda")
        self.embedding = normal(vocabulary, self.C, std=1.0)
        self.norms = [torch.ones(self.C, device="cuda", requires_grad=True) for _ in range(blocks + 1)]
        self.blocks = [{"projection": normal(self.mixed + 2 * heads + self.C, self.C, std=1 / math.sqrt(self.C)), "taps": normal(self.mixed, K, std=1 / math.sqrt(K)),
                        "decay": torch.full((heads, 1), -3.0, device="cuda", requires_grad=True), "w": torch.ones(self.C, device="cuda", requires_grad=True)}
                       for _ in range(blocks)]
        self.head = normal(vocabulary, self.C, std=1 / math.sqrt(self.C))

    def parameters(self):
        return [self.embedding, *self.norms, self.head] + [p for b in self.blocks for p in b.values()]

    def gates(self, b, projected):
        """Log decays and strengths from their rows of the projection."""
        a, s = projected[:, self.mixed:self.mixed + self.H], projected[:, self.mixed + self.H:self.mixed + 2 * self.H]
        decay = b["decay"] if projected.dim() == 3 else b["decay"][:, 0]
        return -torch.nn.functional.softplus(a + decay), torch.sigmoid(s)

    def logits(self, tokens, train=False):
        """tokens [B, L] -> logits [B, vocabulary, L]."""
        x = self.embedding[tokens].transpose(1, 2).contiguous()
        n = FirstNorm.apply(x, self.norms[0])
        for i, (b, w_next) in enumerate(zip(self.blocks, self.norms[1:])):
            projected = torch.matmul(b["projection"], n)
            y = Mixer.apply(projected[:, :self.mixed], b["taps"], *self.gates(b, projected), self.keys, self.Hk)
            if train:
                y = Dropout.apply(y, self.p, self.rng, i)
            x, n = Norms.apply(y, projected, x, b["w"], w_next, self.scale)
        return torch.matmul(self.head, n)

    # ---- serving ----

    def new_pool(self, sequences):
        """The ring and the states of every block for so many sequences."""
        return [{"ring": torch.zeros(sequences, self.mixed, self.K, device="cuda"),
                 "s": torch.zeros(sequences, self.H, self.keys // self.Hk, self.C // self.H, device="cuda")} for _ in self.blocks]

    @torch.no_grad()
    def read(self, prompts, lengths, pool, slots):
        """Prompts [B, L], the first lengths[b] positions of each: fills the pool's rows slots[b], returns the logits behind the last position."""
        x = self.embedding[prompts].transpose(1, 2).contiguous()
        _, n, _ = block.norm_fwd(None, None, x, None, self.norms[0], EPS, save=False)
        for b, w_next, p in zip(self.blocks, self.norms[1:], pool):
            projected = torch.matmul(b["projection"], n)
            u = projected[:, :self.mixed].contiguous()
            block.conv_ring(u, p["ring"], lengths, slots)
            q, k, v = binding.dwconv_fwd(u, b["taps"], self.K - 1).split((self.keys, self.keys, self.C), 1)
            y, s, _ = block.delta_fwd(q, k, v, *self.gates(b, projected), lengths=lengths, key_heads=self.Hk, save=False)
            p["s"][slots.long()] = s
            x, n, _ = block.norm_fwd(y, projected[:, -self.C:], x, b["w"], w_next, EPS, self.scale, save=False)
        return n[torch.arange(len(lengths), device="cuda"), :, lengths.long() - 1] @ self.head.t()

    @torch.no_grad()
    def step(self, token, pos, pool, slots):
        """One token of every sequence of the batch -> logits [B, vocabulary]."""
        x = self.embedding[token][..., None]
        _, n, _ = block.norm_fwd(None, None, x, None, self.norms[0], EPS, save=False)
        for b, w_next, p in zip(self.blocks, self.norms[1:], pool):
            projected = n[..., 0] @ b["projection"].t()
            u = block.conv_step(projected[:, :self.mixed], b["taps"], p["ring"], pos, slots)
            y = block.delta_step(*u.split((self.keys, self.keys, self.C), 1), *self.gates(b, projected), p["s"], slots, self.Hk)
            x, n, _ = block.norm_fwd(y[..., None], projected[:, -self.C:, None], x, b["w"], w_next, EPS, self.scale, save=False)
        return n[..., 0] @ self.head.t()


def train(model, steps, vocabulary, B, L, lr=0.2, momentum=0.9, max_norm=1.0):
    params = model.parameters()
    velocity = [torch.zeros_like(p) for p in params]
    losses = []
    for k in range(steps):
        tokens = batch(vocabulary, B, L, seed=k)
        loss = torch.nn.functional.cross_entropy(model.logits(tokens[:, :-1], train=True), tokens[:, 1:])
        grads = list(torch.autograd.grad(loss, params))
        model.rng[1] += 1                                       # another mask for the next step
        block.clip_grad_norm(grads, max_norm)
        with torch.no_grad():
            for p, v, g in zip(params, velocity, grads):
                v.mul_(momentum).add_(g)
                p.add_(v, alpha=-lr)
        losses.append(loss.item())
    return losses


@torch.no_grad()
def serve(model, vocabulary, B, L, more):
    """Reads prompts of different lengths, goes on for `more` tokens of their own sequences; the largest difference of a logit to those of
    the whole sequences at once, and their largest size."""
    tokens = batch(vocabulary, B, L + more, seed=12345)
    whole = model.logits(tokens[:, :-1])
    lengths = (torch.arange(B, device="cuda") % (L // 2) + L // 2).int()
    slots = torch.randperm(B + 3, generator=torch.Generator().manual_seed(1))[:B].int().cuda()
    pool, rows = model.new_pool(B + 3), torch.arange(B, device="cuda")
    got = model.read(tokens[:, :L].contiguous(), lengths, pool, slots)
    off = float((got - whole[rows, :, lengths.long() - 1]).abs().max())
    pos = lengths.clone()
    for _ in range(more):
        got = model.step(tokens[rows, pos.long()], pos, pool, slots)
        off = max(off, float((got - whole[rows, :, pos.long()]).abs().max()))
        pos += 1
    return off, float(whole.abs().max())


def main(steps=400, vocabulary=32, heads=4, key_heads=2, D=16, K=4, blocks=2, B=32, L=96, report=print):
    model = Model(vocabulary, heads, key_heads, D, K, blocks, seed=0)
    losses = train(model, steps, vocabulary, B, L)
    off, size = serve(model, vocabulary, B, L, more=24)
    report(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps (a guess: {math.log(vocabulary):.3f}); "
           f"served token by token: logits up to {size:.1f}, off by at most {off:.1e}")
    return losses, off, size


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=400)
    main(ap.parse_args().steps)

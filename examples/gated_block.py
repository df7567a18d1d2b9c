"""A small language model of gated sequence blocks on the operators of this library: trained for some steps, then served token by token.

    python examples/gated_block.py [--steps 200]

A block is  n -> projection -> (u, r, i, z);  u -> causal depthwise convolution -> gated scan -> norm, gate, residual and the next
block's norm.  The projections, the embedding and the loss are torch's; the convolution, the scan, the norms and the clipping of the
gradients are calls of ``binding`` and ``block``, wired to autograd by the three functions below.  Serving reads a batch of prompts of
different lengths as the training pass does, keeps the convolution's ring and the scan's state of every sequence in a pool, and goes on one token at a
time; the program checks the logits of both ways against each other.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_25422_amd import binding, block      # noqa: E402

EPS = 1e-6


class Mixer(torch.autograd.Function):
    """(projected [B, 4C, L], taps [C, K], lam [C]) -> scan of the convolution; the channel slices go in and out as they are."""

    @staticmethod
    def forward(ctx, projected, taps, lam):
        C, K = taps.shape
        u, r, i, _ = projected.split(C, 1)
        u = u.contiguous()                                      # (the convolution takes dense tensors)
        v = binding.dwconv_fwd(u, taps, K - 1)
        y, _, states = block.scan_fwd(v, r, i, lam)
        ctx.save_for_backward(projected, u, v, taps, lam, states)
        return y

    @staticmethod
    def backward(ctx, dy):
        projected, u, v, taps, lam, states = ctx.saved_tensors
        C, K = taps.shape
        _, r, i, _ = projected.split(C, 1)
        grad = torch.zeros_like(projected)                      # (z's part comes from the norm)
        du, dr, di, _ = grad.split(C, 1)
        dv = torch.empty_like(v)
        _, _, _, dlam, _ = block.scan_bwd(dy.contiguous(), v, r, i, lam, states, out=(dv, dr, di))
        dx, dtaps = binding.dwconv_bwd(dv, u, taps, K - 1)
        du.copy_(dx)
        return grad, dtaps, dlam


class Norms(torch.autograd.Function):
    """(y, projected, res, w, w_next, scale) -> out, n: the norm behind a block, its gate (the last slice) and residual, the next norm."""

    @staticmethod
    def forward(ctx, y, projected, res, w, w_next, scale):
        z = projected[:, -res.shape[1]:]
        out, n, stats = block.norm_fwd(y, z, res, w, w_next, EPS, scale)
        ctx.save_for_backward(y, projected, res, w, w_next, stats)
        ctx.scale = scale
        return out, n

    @staticmethod
    def backward(ctx, dout, dn):
        y, projected, res, w, w_next, stats = ctx.saved_tensors
        C = res.shape[1]
        grad = torch.zeros_like(projected)
        dy, dres = torch.empty_like(y), torch.empty_like(res)
        _, _, _, dw, dw_next = block.norm_bwd(dout.contiguous(), dn.contiguous(), y, projected[:, -C:], res, w, w_next, stats, ctx.scale,
                                              out=(dy, grad[:, -C:], dres))
        return dy, grad, dres, dw, dw_next, None


class FirstNorm(torch.autograd.Function):
    """The norm in front of the first block."""

    @staticmethod
    def forward(ctx, res, w):
        _, n, stats = block.norm_fwd(None, None, res, None, w, EPS)
        ctx.save_for_backward(res, w, stats)
        return n

    @staticmethod
    def backward(ctx, dn):
        res, w, stats = ctx.saved_tensors
        _, _, dres, _, dw = block.norm_bwd(None, dn.contiguous(), None, None, res, None, w, stats)
        return dres, dw


class Model:
    def __init__(self, vocabulary, C, K, blocks, seed):
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, std):
            return (torch.randn(*shape, generator=g) * std).cuda().requires_grad_()
        self.C, self.K, self.scale = C, K, 1 / math.sqrt(2 * blocks)
        self.embedding = normal(vocabulary, C, std=1.0)
        self.norms = [torch.ones(C, device="cuda", requires_grad=True) for _ in range(blocks + 1)]
        self.blocks = [{"projection": normal(4 * C, C, std=1 / math.sqrt(C)), "taps": normal(C, K, std=1 / math.sqrt(K)),
                        "lam": torch.full((C,), -5.0, device="cuda", requires_grad=True), "w": torch.ones(C, device="cuda", requires_grad=True)}
                       for _ in range(blocks)]
        self.head = normal(vocabulary, C, std=1 / math.sqrt(C))

    def parameters(self):
        return [self.embedding, *self.norms, self.head] + [p for b in self.blocks for p in b.values()]

    def logits(self, tokens):
        """tokens [B, L] -> logits [B, vocabulary, L]."""
        x = self.embedding[tokens].transpose(1, 2).contiguous()
        n = FirstNorm.apply(x, self.norms[0])
        for b, w_next in zip(self.blocks, self.norms[1:]):
            projected = torch.matmul(b["projection"], n)
            y = Mixer.apply(projected, b["taps"], b["lam"])
            x, n = Norms.apply(y, projected, x, b["w"], w_next, self.scale)
        return torch.matmul(self.head, n)

    # ---- serving ----

    def new_pool(self, sequences):
        """The ring and the state of every block for so many sequences."""
        return [{"ring": torch.zeros(sequences, self.C, self.K, device="cuda"), "h": torch.zeros(sequences, self.C, device="cuda")} for _ in self.blocks]

    @torch.no_grad()
    def read(self, prompts, lengths, pool, slots):
        """Prompts [B, L], the first lengths[b] positions of each: fills the pool's rows slots[b], returns the logits behind the last position."""
        x = self.embedding[prompts].transpose(1, 2).contiguous()
        _, n, _ = block.norm_fwd(None, None, x, None, self.norms[0], EPS, save=False)
        for b, w_next, p in zip(self.blocks, self.norms[1:], pool):
            projected = torch.matmul(b["projection"], n)
            u, r, i, z = projected.split(self.C, 1)
            u = u.contiguous()
            block.conv_ring(u, p["ring"], lengths, slots)
            y, h, _ = block.scan_fwd(binding.dwconv_fwd(u, b["taps"], self.K - 1), r, i, b["lam"], lengths=lengths, save=False)
            p["h"][slots.long()] = h
            x, n, _ = block.norm_fwd(y, z, x, b["w"], w_next, EPS, self.scale, save=False)
        last = n[torch.arange(len(lengths), device="cuda"), :, lengths.long() - 1]
        return last @ self.head.t()

    @torch.no_grad()
    def step(self, token, pos, pool, slots):
        """One token of every sequence of the batch -> logits [B, vocabulary]."""
        C = self.C
        x = self.embedding[token][..., None]
        _, n, _ = block.norm_fwd(None, None, x, None, self.norms[0], EPS, save=False)
        for b, w_next, p in zip(self.blocks, self.norms[1:], pool):
            projected = n[..., 0] @ b["projection"].t()
            u, r, i, z = projected.split(C, 1)
            y = block.scan_step(block.conv_step(u, b["taps"], p["ring"], pos, slots), r, i, b["lam"], p["h"], slots)
            x, n, _ = block.norm_fwd(y[..., None], z[..., None], x, b["w"], w_next, EPS, self.scale, save=False)
        return n[..., 0] @ self.head.t()


def batch(vocabulary, B, L, seed):
    """Sequences that repeat themselves: each token is the one seven positions before, of a random first seven."""
    g = torch.Generator().manual_seed(seed)
    first = torch.randint(vocabulary, (B, 7), generator=g)
    return first.repeat(1, L // 7 + 2)[:, :L + 1].cuda()


def train(model, steps, vocabulary, B, L, lr=1.0, momentum=0.9, max_norm=1.0):
    params = model.parameters()
    velocity = [torch.zeros_like(p) for p in params]
    losses = []
    for k in range(steps):
        tokens = batch(vocabulary, B, L, seed=k)
        loss = torch.nn.functional.cross_entropy(model.logits(tokens[:, :-1]), tokens[:, 1:])
        grads = list(torch.autograd.grad(loss, params))
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
    pool = model.new_pool(B + 3)
    rows = torch.arange(B, device="cuda")
    got = model.read(tokens[:, :L].contiguous(), lengths, pool, slots)
    off = float((got - whole[rows, :, lengths.long() - 1]).abs().max())
    pos = lengths.clone()
    for _ in range(more):
        got = model.step(tokens[rows, pos.long()], pos, pool, slots)
        off = max(off, float((got - whole[rows, :, pos.long()]).abs().max()))
        pos += 1
    return off, float(whole.abs().max())


def main(steps=200, vocabulary=32, C=64, K=8, blocks=2, B=32, L=96, report=print):
    model = Model(vocabulary, C, K, blocks, seed=0)
    losses = train(model, steps, vocabulary, B, L)
    off, size = serve(model, vocabulary, B, L, more=24)
    report(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps (a guess: {math.log(vocabulary):.3f}); "
           f"served token by token: logits up to {size:.1f}, off by at most {off:.1e}")
    return losses, off, size


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    main(ap.parse_args().steps)

"""Sums of the gated delta rule whose terms nearly take each other away, on the GPU against whole formulas in 64 bits: what is left shows the bits that
the terms were formed with, where a sum of the terms' own size hides them behind the rounding of its output.

u = 2^-24 is one rounding of 32 bits relative to the value.  Operands as three bf16 limbs are exact, their products to 2^-24; operands of two limbs
would be off by up to 2^-17."""
import pytest
import torch

from paper_2604_25422_amd import block

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def rand(*shape, seed, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def uniform(*shape, seed, lo, hi):
    return (lo + (hi - lo) * torch.rand(*shape, generator=torch.Generator().manual_seed(seed))).cuda()


def within(got, want, bound):
    off = (got.double() - want).abs() - bound - HALF_STEP[got.dtype] * (want.abs() + bound)
    at = int(off.argmax())
    over, *rest = (float(x.reshape(-1)[at]) for x in (off, got, want, bound))
    assert over <= 0, (at, *rest)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("DK", [2, 40, 128])
def test_outputs_of_a_state_that_cancel(DK, dtype):
    """o = S^T q of two rows of S that are each other's opposite but for 2^-12."""
    B, H, DV, L = 2, 2, 96, 130
    s0 = rand(B, H, DK, DV, seed=1)
    s0[:, :, 0] = uniform(B, H, DV, seed=2, lo=1, hi=2)
    s0[:, :, DK - 1] = -s0[:, :, 0] * (1 + 2.0 ** -12 * uniform(B, H, DV, seed=3, lo=-1, hi=1))
    q = torch.zeros(B, H, DK, L, device="cuda", dtype=dtype)
    q[:, :, 0] = q[:, :, DK - 1] = 1
    q, zero = q.view(B, -1, L), torch.zeros(B, H, L, device="cuda")
    o, s_last, _ = block.delta_fwd(q, rand(B, H * DK, L, seed=4, dtype=dtype), rand(B, H * DV, L, seed=5, dtype=dtype), zero, zero, s0, scale=1.0, eps=0.0)
    assert torch.equal(s_last, s0)                      # (no decay, nothing written)
    two = s0.double()[:, :, [0, DK - 1]]
    want = two.sum(2)[..., None].expand(B, H, DV, L).reshape(B, H * DV, L)
    size = two.abs().sum(2)[..., None].expand(B, H, DV, L).reshape(B, H * DV, L)
    # exact products: at most six additions of each of the two, and the factors exp(0) and scale, both 1
    within(o, want, 16 * U * size)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("DK", [2, 40, 128])
@pytest.mark.parametrize("what", ["w", "P"])
def test_outputs_of_a_chunk_that_cancel(what, DK, dtype):
    """o of two positions' values that are each other's opposite but for 2^-12 of their strengths ("w"), or of the decay between them ("P")."""
    B, H, DV, L = 3, 4, 32, 64
    k, v = torch.zeros(B, H, DK, L, device="cuda", dtype=dtype), torch.zeros(B, H, DV, L, device="cuda", dtype=dtype)
    k[:, :, 0, 0] = k[:, :, DK - 1, 1] = 1              # (orthogonal: the second does not correct the first)
    v[:, :, :, 0] = uniform(B, H, DV, seed=1, lo=1, hi=2).to(dtype)
    v[:, :, :, 1] = -v[:, :, :, 0]
    q = torch.zeros_like(k)
    q[:, :, 0] = q[:, :, DK - 1] = 1
    g, beta, near = torch.zeros(B, H, L, device="cuda"), torch.ones(B, H, L, device="cuda"), 2.0 ** -12 * uniform(B, H, seed=2, lo=-1, hi=0)
    if what == "w":
        beta[:, :, 0] = uniform(B, H, seed=3, lo=0.5, hi=1)
        beta[:, :, 1] = beta[:, :, 0] * (1 + near)
    else:
        g[:, :, 2:] = -0.2 * rand(B, H, L - 2, seed=4).abs()
        g[:, :, 1] = near
    o, _, _ = block.delta_fwd(*(x.view(B, -1, L) for x in (q, k, v)), g, beta, scale=1.0, eps=0.0, save=False)
    G = g.double().cumsum(-1)
    at = [torch.where(torch.arange(L, device="cuda") >= j, torch.exp(torch.clamp(G - G[..., j:j + 1], max=0.0)), 0.0) * beta[..., j:j + 1].double() for j in (0, 1)]
    term = [at[j][:, :, None] * v[:, :, :, j:j + 1].double() for j in (0, 1)]
    want, size = (term[0] + term[1]).view(B, -1, L), (term[0].abs() + term[1].abs()).view(B, -1, L)
    # the exponential 4, its two factors, the product with beta and w's own sum, the sum of the two in as many additions as before
    within(o, want, 32 * U * size)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("DK", [2, 40, 128])
@pytest.mark.parametrize("L", [1, 130])
@pytest.mark.parametrize("each", [1, 3])
def test_gradients_along_a_key_that_cancel(each, L, DK, dtype):
    """A query that points where its own key does: o does not change when either becomes longer, so that of dq and dk, which lie along them, only
    eps / |x|^2 is left.  One position of every chunk has keys and values."""
    B, Hk, scale, eps, at = 4, 3, 0.75, 1e-6, 0 if L == 1 else 37
    H, t = each * Hk, torch.arange(L, device="cuda")
    on = (t % 64 == at).to(dtype)
    k = rand(B, Hk, DK, L, seed=1, dtype=dtype)
    k[:, :, 2:] = 0                                     # (two channels of a key: few terms to a sum, wherever the second lies)
    if DK > 2:
        k[:, :, DK - 1], k[:, :, 1] = k[:, :, 1], 0
    k = k * on
    q = -2 * k
    v, do = (rand(B, H, 1, L, seed=s, dtype=dtype) * on for s in (2, 3))
    beta, inf = uniform(B, H, L, seed=4, lo=0.5, hi=1), torch.full((B, H, L), -float("inf"), device="cuda")
    flat = [x.view(B, -1, L) for x in (q, k, v)]
    # (every position forgets what lies in front of it: each is a rule of its own)
    _, _, states = block.delta_fwd(*flat, inf, beta, key_heads=Hk, scale=scale, eps=eps)
    dq, dk, *_ = block.delta_bwd(do.view(B, -1, L), *flat, inf, beta, states, key_heads=Hk, scale=scale, eps=eps)
    x = k.double()
    square = x.square().sum(2, keepdim=True)
    ik, iq = 1 / torch.sqrt(square + eps), 1 / torch.sqrt(4 * square + eps)
    unit_k, unit_q = x * ik, -2 * x * iq
    pair = scale * (do.double() * v.double() * beta.double()[:, :, None]).view(B, Hk, each, 1, L)
    for got, other, own, i in ((dq, unit_k, unit_q, iq), (dk, unit_q, unit_k, ik)):
        one = pair.sum(2) * (other - own * (own * other).sum(2, keepdim=True)) * i
        size = pair.abs().sum(2) * (other.abs() + own.abs() * (own * other).abs().sum(2, keepdim=True)) * i
        # lengths 6 and twice, the pair's product and its factors 8, P in the sums along a key 12, the sums of two channels and of heads 8
        within(got, one.view(B, -1, L), 40 * U * size.view(B, -1, L))

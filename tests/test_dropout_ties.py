"""Dropout where the upper sixteen of an element's 32 bits are the limit's own, so that the lower sixteen decide: one element of 65536, whole tensors of
millions of them against the generator in whole numbers."""
import numpy as np
import pytest
import torch

import _delta_ref as ref

SEED, STEP, LAYER = 12345 + (7 << 40), 99, 3


def halves(seed, step, layer, B, n):
    """The upper and the lower sixteen bits of elements 0 .. n - 1 of B entries, [B, n] each (ref.bits, all at once)."""
    m = np.arange(-(-n // 8), dtype=np.uint64)
    low = np.uint64(0xFFFFFFFF)
    out = []
    for half in (0, 1):
        c = [np.broadcast_to(m & low, (B, m.size)), np.broadcast_to(np.arange(B, dtype=np.uint64)[:, None], (B, m.size)), np.uint64(step & 0xFFFFFFFF),
             np.broadcast_to(np.uint64(layer << 8 | half) | m >> np.uint64(32) << np.uint64(1), (B, m.size))]
        k = [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF]
        for _ in range(10):
            a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [b >> np.uint64(32) ^ c[1] ^ np.uint64(k[0]), b & low, a >> np.uint64(32) ^ c[3] ^ np.uint64(k[1]), a & low]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        words = np.stack(c, -1)
        out.append(np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(B, -1)[:, :n].astype(np.int64))
    return out


def test_halves_are_the_generator_s():
    hi, lo = halves(SEED, STEP, LAYER, 3, 100)
    for b in range(3):
        for j in range(100):
            assert int(hi[b, j]) << 16 | int(lo[b, j]) == ref.bits(SEED, STEP, LAYER, b, j)


def kept(limit, B, n):
    """Decisions and, of those that the lower half takes, how many there are of each kind: dropped or kept, in an even or an odd half-word."""
    hi, lo = halves(SEED, STEP, LAYER, B, n)
    keep = (hi << 16 | lo) >= limit
    tie, odd = hi == limit >> 16, np.broadcast_to(np.arange(n) & 1, (B, n)).astype(bool)
    return keep, [int((tie & (keep == k) & (odd == o)).sum()) for k in (False, True) for o in (False, True)]


# rates that 32-bit floats hold exactly, as limits of 2^32: an ordinary one, one below 2^-16 (whose upper half is zero), one close to 1, and one whose
# lower half is odd (a rate of 24 bits from 2^-8 down)
LIMITS = [0x4CCC8000, 0x00008000, 0xFFFE8000, 0x00A97F43]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("limit", LIMITS)
@pytest.mark.parametrize("tied,B,C,L", [(False, 3, 7, 100003), (False, 1 << 14, 3, 50), (True, 3, 700001, 2), (True, 1 << 14, 130, 3)])
def test_the_lower_half_decides(tied, B, C, L, limit, dtype):
    from paper_2604_25422_amd import block
    p, n = limit / 2 ** 32, C if tied else C * L
    assert float(torch.tensor(p, dtype=torch.float32)) * 2 ** 32 == limit
    want, kinds = kept(limit, B, n)
    assert min(kinds) >= 1, kinds
    y = block.dropout_fwd(torch.ones(B, C, L, dtype=dtype, device="cuda"), p, torch.tensor([SEED, STEP], device="cuda"), LAYER, tied=tied) != 0
    want = torch.from_numpy(want).view(B, C, -1).expand(B, C, L)
    assert torch.equal(y.cpu(), want)


def test_a_wrong_lower_half_would_show():
    """What the GPU test can see: the decisions by the upper half alone, or by the other block's half-words, are others of these elements."""
    for limit in LIMITS:
        for tied, B, n in ((False, 3, 700021), (False, 1 << 14, 150), (True, 3, 700001), (True, 1 << 14, 130)):
            hi, lo = halves(SEED, STEP, LAYER, B, n)
            keep = (hi << 16 | lo) >= limit
            swapped = (hi << 16 | lo.reshape(B, -1)[:, np.minimum(np.arange(n) ^ 1, n - 1)]) >= limit
            for other in (hi >= limit >> 16, hi > limit >> 16, swapped, (hi << 16 | hi) >= limit):
                assert (other != keep).any()


def test_a_factor_beyond_32_bits_is_refused():
    from paper_2604_25422_amd import _build, block
    if _build.is_stale():
        _build.build()
    P = 0x1000          # any aligned, never-dereferenced address

    def status(p, scale):
        return block.lib().dwconv_dropout(block.Seq(P, 1 << 20), block.Seq(None, 0), block.Seq(P, 1 << 20), P, 0, 2, 3, 10, p, scale, 0, 0, None)
    top = float(np.finfo(np.float32).max)
    for p, scale in ((0.5, top), (0.5, -top), (0.999, 1e36), (1 - 2.0 ** -24, 2.0 ** 104), (0.0, float("inf")), (0.0, float("nan"))):
        assert status(p, scale) == 9, (p, scale)

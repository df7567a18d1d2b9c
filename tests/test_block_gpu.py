"""The block operators on the GPU against their definitions in 64 bits (tests/_block_ref.py, which also derives the bounds), at the
lengths, layouts and masks where the kernels change form or could go wrong."""
import math

import pytest
import torch

import _block_ref as ref
from paper_2604_25422_amd import binding, block

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
RATE = 8.0


def rand(*shape, seed, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def strided(t, kind):
    """The same values as a slice of the channels of a wider tensor ("slice"), or off its granule ("odd")."""
    B, C = t.shape[:2]
    if kind == "slice":
        wide = torch.full((B, 2 * C + 3, *t.shape[2:]), float("nan"), dtype=t.dtype, device="cuda")
        v = wide[:, C + 1:2 * C + 1]
        v.copy_(t)
        return v
    if kind == "odd":
        flat = torch.full((t.numel() + 3,), float("nan"), dtype=t.dtype, device="cuda")
        v = flat[1:1 + t.numel()].view(t.shape)
        v.copy_(t)
        return v
    return t


def scan_inputs(B, C, L, dtype, seed, decay=-5.0):
    x, r, i, dy = (rand(B, C, L, seed=seed + k, dtype=dtype) for k in range(4))
    return x, r, i, dy, rand(C, seed=seed + 5) + decay


def check_scan(x, r, i, dy, lam, h0=None, dh=None, lengths=None, rate=RATE, workspace=False):
    dtype = x.dtype
    want, err = ref.scan(x, r, i, lam, h0, lengths, rate, dy, dh)
    y, h_last, states = block.scan_fwd(x, r, i, lam, h0, lengths, rate=rate)
    got = dict(zip(("dx", "dr", "di", "dlam", "dh0"), block.scan_bwd(dy, x, r, i, lam, states, dh, lengths, rate=rate)))
    got.update(y=y, h_last=h_last)
    for k, v in got.items():
        assert v.dtype == (dtype if k in ("y", "dx", "dr", "di") else F32)
        ref.check(v, want[k], err[k], v.dtype, k)
    if lengths is not None:
        for b, n in enumerate(lengths.cpu().clamp(0, x.shape[2]).tolist()):
            for k in ("y", "dx", "dr", "di"):
                assert (got[k][b, :, n:] == 0).all(), k
    return got


# (short rows in groups of 1 to 32 lanes, whole and not; one chunk and several, off the granule; more waves than chunks)
LENGTHS = (1, 2, 7, 8, 9, 16, 31, 48, 64, 65, 100, 129, 255, 256, 257, 300, 511, 512, 513, 1024, 1025, 2500)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L", LENGTHS)
def test_scan_lengths(L, dtype):
    x, r, i, dy, lam = scan_inputs(3, 5, L, dtype, 100 + L)
    check_scan(x, r, i, dy, lam, rand(3, 5, seed=1), rand(3, 5, seed=2))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,C,L", [(1, 1, 9000), (1, 3, 40001), (2, 1, 70000), (300, 1, 17), (1, 300, 5), (7, 129, 260), (513, 9, 600), (1, 1, 1),
                                   (70, 64, 1030), (33, 64, 2100),
                                   # (one to sixteen waves a row, one group of them and several; segments of one and of several groups)
                                   (9, 256, 700), (5, 260, 1100), (5, 130, 2100), (3, 100, 4200), (2, 70, 9000), (1, 129, 17000), (1, 64, 34000), (1, 127, 33500),
                                   # (a channel's batch in one workgroup, and just not)
                                   (8, 3, 257), (8, 70, 1024), (9, 70, 1024), (1, 7, 1000), (8, 33, 200), (9, 33, 200), (200, 3, 4), (256, 2, 8), (257, 2, 8), (32, 40, 60)])
def test_scan_shapes(B, C, L, dtype):
    x, r, i, dy, lam = scan_inputs(B, C, L, dtype, 7)
    check_scan(x, r, i, dy, lam, rand(B, C, seed=1), rand(B, C, seed=2))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L", [1, 2, 3, 4, 5, 6, 7, 8, 9, 15, 255, 257, 263, 511])
def test_scan_short_rows_of_many_lengths(L, dtype):
    """Rows that a lane has whole, and rows that end inside a lane's eight, in more workgroups than a run of them has."""
    B, C = 13, 131
    x, r, i, dy, lam = scan_inputs(B, C, L, dtype, 61)
    h0, dh = rand(B, C, seed=1), rand(B, C, seed=2)
    lengths = torch.tensor([0, 1, L, L // 2, -4, L + 9, max(1, L - 1), L, 2, 3, L - 2, L, 5], dtype=torch.int32).cuda()
    for n in (None, lengths):
        want, err = ref.scan(x, r, i, lam, h0, n, RATE, dy, dh)
        y, h_last, states = block.scan_fwd(x, r, i, lam, h0, n)
        got = dict(zip(("dx", "dr", "di", "dlam", "dh0"), block.scan_bwd(dy, x, r, i, lam, states, dh, n)), y=y, h_last=h_last)
        for k, v in got.items():
            ref.check(v, want[k], err[k], v.dtype, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,C,L", [(4000, 40, 5), (4000, 7, 100), (5000, 3, 300), (66000, 1, 257)])
def test_scan_sums_of_many_rows(B, C, L, dtype):
    """dlam over more rows than one launch adds up: in runs, of few and of many."""
    x, r, i, dy, lam = scan_inputs(B, C, L, dtype, 63)
    check_scan(x, r, i, dy, lam, rand(B, C, seed=1), rand(B, C, seed=2))


@pytest.mark.parametrize("B,C,L", [(1 << 21, 1, 1), (1 << 21, 32, 1), (1 << 18, 32, 8), (1 << 18, 1, 300), (100000, 2, 300), (60000, 1, 257), (11000, 32, 257)])
def test_scan_sums_of_many_rows_in_short_chains(B, C, L):
    """The same row B times over (stride 0): its terms round alike, so a chain of additions shows its length.  No term passes 400 of them."""
    x, r, i, dy, lam = scan_inputs(1, C, L, F32, 64)
    _, _, states = block.scan_fwd(x, r, i, lam)
    one = block.scan_bwd(dy, x, r, i, lam, states)[3].double()
    x, r, i, dy = (t.expand(B, C, L) for t in (x, r, i, dy))
    _, _, states = block.scan_fwd(x, r, i, lam)
    dlam = block.scan_bwd(dy, x, r, i, lam, states)[3].double()
    assert ((dlam - B * one).abs() <= 400 * 2.0 ** -24 * B * one.abs()).all(), float((dlam / (B * one) - 1).abs().max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,C,L", [(1, 100, 33300), (3, 45, 33300), (1, 100, 17000)])
def test_scan_of_rows_that_one_type_or_pass_cuts(B, C, L, dtype):
    """Few long rows, cut into segments by one type or direction and whole in the other, in a workspace of the size that is asked for."""
    x, r, i, dy, lam = scan_inputs(B, C, L, dtype, 66)
    h0, dh = rand(B, C, seed=1), rand(B, C, seed=2)
    space = [torch.full((block.scan_workspace_bytes(B, C, L, k),), 255, dtype=torch.uint8, device="cuda") for k in (False, True)]
    want, err = ref.scan(x, r, i, lam, h0, None, RATE, dy, dh)
    y, h_last, states = block.scan_fwd(x, r, i, lam, h0, workspace=space[0])
    got = dict(zip(("dx", "dr", "di", "dlam", "dh0"), block.scan_bwd(dy, x, r, i, lam, states, dh, workspace=space[1])), y=y, h_last=h_last)
    for k, v in got.items():
        ref.check(v, want[k], err[k], v.dtype, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L", [5, 100, 700, 5000, 33000])
def test_scan_masked_rows(L, dtype):
    """Sequences of no position, one, all, and lengths outside [0, L]; what lies behind an end is not read."""
    x, r, i, dy, lam = scan_inputs(7, 3, L, dtype, 31)
    lengths = torch.tensor([0, 1, L, L // 2, -4, L + 9, max(1, L - 1)], dtype=torch.int32)
    for b, n in enumerate(lengths.clamp(0, L).tolist()):
        for t, bad in ((x, float("nan")), (r, float("inf")), (i, -float("inf")), (dy, float("nan"))):
            t[b, :, n:] = bad
    clean = [torch.nan_to_num(t, nan=0.0, posinf=0.0, neginf=0.0) for t in (x, r, i, dy)]
    h0, dh, lengths = rand(7, 3, seed=1), rand(7, 3, seed=2), lengths.cuda()
    want, err = ref.scan(*clean[:3], lam, h0, lengths, RATE, clean[3], dh)
    y, h_last, states = block.scan_fwd(x, r, i, lam, h0, lengths)
    got = dict(zip(("dx", "dr", "di", "dlam", "dh0"), block.scan_bwd(dy, x, r, i, lam, states, dh, lengths)), y=y, h_last=h_last)
    for k, v in got.items():
        ref.check(v, want[k], err[k], v.dtype, k)
    assert torch.equal(h_last[0], h0[0]) and torch.equal(got["dh0"][0], dh[0]) and torch.equal(h_last[4], h0[4])
    assert (y[0] == 0).all() and (got["dx"][4] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L", [6, 77, 600, 9001])
@pytest.mark.parametrize("kind", ["slice", "odd"])
def test_scan_layouts(L, kind, dtype):
    x, r, i, dy, lam = scan_inputs(3, 4, L, dtype, 41)
    h0, dh = rand(3, 4, seed=1), rand(3, 4, seed=2)
    y, h_last, states = block.scan_fwd(x, r, i, lam, h0)
    want = (y, *block.scan_bwd(dy, x, r, i, lam, states, dh))
    xs, rs, is_, dys = (strided(t, kind) for t in (x, r, i, dy))
    outs = [strided(torch.zeros_like(x), kind) for _ in range(4)]
    y2, h2, s2 = block.scan_fwd(xs, rs, is_, lam, h0, out=outs[0])
    got = (y2, *block.scan_bwd(dys, xs, rs, is_, lam, s2, dh, out=outs[1:]))
    assert y2 is outs[0] and got[1] is outs[1] and torch.equal(h_last, h2) and torch.equal(states, s2)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    if kind == "slice":                                  # (nothing was written beside the slices)
        for t in outs:
            wide = t._base
            assert wide[:, :5].isnan().all() and wide[:, 9:].isnan().all()


def test_scan_of_a_broadcast_input():
    """One gate for the whole batch (stride 0): the gradient is that of every entry, the caller sums."""
    x, r, i, dy, lam = scan_inputs(4, 3, 700, F32, 51)
    r1 = r[:1].expand(4, 3, 700)
    got = block.scan_fwd(x, r1, i, lam)
    full = block.scan_fwd(x, r1.contiguous(), i, lam)
    assert torch.equal(got[0], full[0])
    a, b = block.scan_bwd(dy, x, r1, i, lam, got[2]), block.scan_bwd(dy, x, r1.contiguous(), i, lam, full[2])
    assert all(torch.equal(s, t) for s, t in zip(a, b)) and a[1].shape == (4, 3, 700)


@pytest.mark.parametrize("L", [40, 700, 20000])
def test_scan_of_extreme_gates(L):
    """Decays of exactly 0 and 1, gates that are shut or open as far as fp32 goes: everything finite and right."""
    lam = torch.tensor([-120.0, -80.0, -20.0, -5.0, 0.0, 3.0, 30.0, 1e4, 3e38], device="cuda")
    C = lam.numel()
    x, r, i, dy, _ = scan_inputs(2, C, L, F32, 61)
    for t, seed in ((r, 1), (i, 2)):
        pick = torch.randint(0, 8, t.shape, generator=torch.Generator().manual_seed(seed)).cuda()
        for k, v in enumerate((-200.0, -60.0, -30.0, 30.0, 90.0, 200.0)):
            t[pick == k] = v
    want, err = ref.scan(x, r, i, lam, None, None, RATE, dy, None)
    y, h_last, states = block.scan_fwd(x, r, i, lam)
    got = dict(zip(("dx", "dr", "di", "dlam", "dh0"), block.scan_bwd(dy, x, r, i, lam, states)), y=y, h_last=h_last)
    # a logit v puts |v| roundings of the exponential's argument on top of the 40 of an ordinary gate: up to 200 here, and what
    # lies below 2^-60 of the largest value may be flushed where a product on the way to it falls below the smallest normal number
    for k, v in got.items():
        ref.check(v, want[k], 6 * err[k], F32, k, floor=2.0 ** -60 * float(want[k].abs().max()))


@pytest.mark.parametrize("L", [1, 5, 30, 700, 40000])
def test_scan_of_infinite_decay_parameters(L):
    """lam of minus infinity: no decay and no input, the state goes through; of plus infinity: the state is the input of the position."""
    inf = float("inf")
    x, r, i, dy, lam = scan_inputs(2, 4, L, F32, 67)
    lam[1], lam[3] = -inf, inf
    h0, dh = rand(2, 4, seed=1), rand(2, 4, seed=2)
    y, h, states = block.scan_fwd(x, r, i, lam, h0)
    dx, dr, di, dlam, dh0 = block.scan_bwd(dy, x, r, i, lam, states, dh)
    assert (y[:, 1] == h0[:, 1, None]).all() and torch.equal(h[:, 1], h0[:, 1])
    for t in (dx, dr, di):
        assert (t[:, 1] == 0).all()
    want, err = ref.scan(x[:, :3], r[:, :3], i[:, :3], lam[:3], h0[:, :3], None, RATE, dy[:, :3], dh[:, :3])
    for k, v in dict(y=y, h_last=h, dx=dx, dr=dr, di=di, dh0=dh0).items():
        ref.check(v[:, :3], want[k], err[k], F32, k)
    ref.check(dlam[:3], want["dlam"], err["dlam"], F32, "dlam")
    # (q is infinite: a is 0 and sqrt(1 - a^2) 1)
    xi = x[:, 3].double().cpu() * torch.sigmoid(i[:, 3].double().cpu())
    ref.check(y[:, 3], xi, 40 * ref.U * xi.abs(), F32, "y")
    assert (dr[:, 3] == 0).all() and dlam[3] == 0 and (dh0[:, 3] == 0).all()
    g = dy[:, 3].double().cpu()
    g[:, -1] += dh[:, 3].double().cpu()
    ref.check(dx[:, 3], g * torch.sigmoid(i[:, 3].double().cpu()), 40 * ref.U * g.abs(), F32, "dx")
    ref.check(di[:, 3], g * xi * torch.sigmoid(-i[:, 3].double().cpu()), 40 * ref.U * (g * xi).abs(), F32, "di")
    tok = [t[..., 0].contiguous() for t in (x, r, i)]
    pool = h0.clone()
    y1 = block.scan_step(*tok, lam, pool)
    assert torch.equal(y1[:, 1], h0[:, 1]) and torch.equal(pool[:, 1], h0[:, 1]) and torch.isfinite(y1).all()


@pytest.mark.parametrize("L", [1, 30, 700, 9000])
@pytest.mark.parametrize("logit", [-200.0, -80.0, -60.0])
def test_scan_of_large_inputs_behind_shut_gates(logit, L):
    """x beyond 2^64 where the decay's gate is shut: 1 / sqrt(1 - a^2) times it does not fit fp32, the gradients do."""
    x, r, i, dy, lam = scan_inputs(2, 3, L, F32, 65)
    at = L // 2
    x[:, 1, at], r[:, 1, at] = torch.tensor([4e27, -3e30], device="cuda"), logit
    h0, dh = rand(2, 3, seed=1), rand(2, 3, seed=2)
    want, err = ref.scan(x, r, i, lam, h0, None, RATE, dy, dh)
    y, h_last, states = block.scan_fwd(x, r, i, lam, h0)
    got = dict(zip(("dx", "dr", "di", "dlam", "dh0"), block.scan_bwd(dy, x, r, i, lam, states, dh)), y=y, h_last=h_last)
    # (a logit v puts |v| roundings of the exponential's argument on top of the 40 of an ordinary gate)
    for k, v in got.items():
        c = (slice(1, 2),) if k == "dlam" else (slice(None), slice(1, 2))
        o = ([0, 2],) if k == "dlam" else (slice(None), [0, 2])
        ref.check(v[o], want[k][o], err[k][o], F32, k)
        assert torch.isfinite(v[c]).all(), k
        if logit > -87:                         # (beyond, the open part of the gate is below the smallest fp32 number: 0)
            ref.check(v[c], want[k][c], 6 * err[k][c], F32, k, floor=max(1e-30, 2.0 ** -60 * float(want[k][c].abs().max())))


@pytest.mark.parametrize("wide", ["r", "i"])
def test_scan_of_wide_logits_is_exact(wide):
    """fp32 gates as exact at logits of -75 to 60 as at small ones, in rows of one position, where nothing else adds up.  A gate, and 1 minus it:
    exponential and reciprocal within a unit (U), five roundings (U / 2).  q: 5 U of exp(lam) and its logarithm on top; sqrt(1 - a^2) and
    its reciprocal have half of that and 2 U of their own.  So y and dx stay below 16 U of themselves, di below 22 U, dr below 32 U."""
    B, C = 512, 96
    x, r, i, dy, lam = scan_inputs(B, C, 1, F32, 85)
    span = torch.linspace(-75, 60, B * C)[torch.randperm(B * C, generator=torch.Generator().manual_seed(3))].view(B, C, 1).cuda()
    r, i = (span, i) if wide == "r" else (r, span)
    want, _ = ref.scan(x, r, i, lam, None, None, RATE, dy)
    y, h, states = block.scan_fwd(x, r, i, lam)
    dx, dr, di, _, _ = block.scan_bwd(dy, x, r, i, lam, states)
    pool = torch.zeros(B, C, device="cuda")
    step = block.scan_step(x[..., 0], r[..., 0], i[..., 0], lam, pool)[..., None]
    for k, v, units in (("y", y, 16), ("y", step, 16), ("dx", dx, 16), ("di", di, 22), ("dr", dr, 32)):
        ref.check(v, want[k], units * ref.U * want[k].abs(), F32, k, floor=0.0)


@pytest.mark.parametrize("C,L", [(64, 1), (64, 3), (64, 40), (5000, 2)])
def test_norm_of_wide_logits_is_exact(C, L):
    """silu(z) alone (y and w are 1, res 0), whose gate is within 5 U: with the product, the norm of y and the last sum below 9 U."""
    B = 8
    z = torch.linspace(-75, 60, B * C * L)[torch.randperm(B * C * L, generator=torch.Generator().manual_seed(3))].view(B, C, L).cuda()
    one, w = torch.ones_like(z), torch.ones(C, device="cuda")
    out, _, stats = block.norm_fwd(one, z, torch.zeros_like(z), w, w, eps=1e-30)
    want = z.double().cpu() * torch.sigmoid(z.double().cpu())
    ref.check(out, want, 9 * ref.U * want.abs(), F32, "out", floor=0.0)
    # (dw of one entry and position is dout silu(z): dn is 0)
    dout = rand(1, C, 1, seed=4)
    part = z[:1, :, :1].contiguous()
    _, _, s1 = block.norm_fwd(one[:1, :, :1].contiguous(), part, torch.zeros_like(part), w, w, eps=1e-30)
    dw = block.norm_bwd(dout, torch.zeros_like(dout), one[:1, :, :1].contiguous(), part, torch.zeros_like(part), w, w, s1)[3]
    want = dout[0, :, 0].double().cpu() * want[0, :, 0]
    ref.check(dw, want, 12 * ref.U * want.abs(), F32, "dw", floor=0.0)


@pytest.mark.parametrize("L", [30, 700, 9000])
def test_scan_keeps_bad_values_in_their_row(L):
    x, r, i, dy, lam = scan_inputs(2, 3, L, F32, 71)
    clean = block.scan_fwd(x, r, i, lam)
    at = L // 2
    for t, bad in ((x, float("inf")), (r, float("nan")), (i, float("nan")), (x, float("nan"))):
        kept = t[0, 1, at].item()
        t[0, 1, at] = bad
        y, h_last, states = block.scan_fwd(x, r, i, lam)
        assert not torch.isfinite(y[0, 1, at]) and not torch.isfinite(y[0, 1, at:]).any() and not torch.isfinite(h_last[0, 1])
        assert torch.equal(y[0, 1, :at], clean[0][0, 1, :at])
        others = [(b, c) for b in range(2) for c in range(3) if (b, c) != (0, 1)]
        g = block.scan_bwd(dy, x, r, i, lam, states)
        for b, c in others:
            assert torch.equal(y[b, c], clean[0][b, c]) and all(torch.isfinite(t2[b, c]).all() for t2 in (*g[:3], g[4]))
        assert torch.isfinite(g[3][[0, 2]]).all() and not torch.isfinite(g[3][1])
        t[0, 1, at] = kept


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L", [1, 3, 5, 9, 100, 300, 700, 5000, 40000])
def test_scan_keeps_bad_values_in_front_of_the_end(L, dtype):
    """Behind a sequence's end outputs and gradients are 0 also where the state that reaches it is no number, and a bad state in front of a
    sequence of no position is in no gradient but its own."""
    B, C = 4, 3
    x, r, i, dy, lam = scan_inputs(B, C, L, dtype, 75)
    n = [(L + 1) // 2, L // 3, 0, L]
    lengths = torch.tensor(n, dtype=torch.int32, device="cuda")
    h0, dh = rand(B, C, seed=1), rand(B, C, seed=2)
    want = block.scan_fwd(x, r, i, lam, h0, lengths)
    clean = block.scan_bwd(dy, x, r, i, lam, want[2], dh, lengths)
    x[0, 1, n[0] // 2] = float("nan")
    if n[1]:
        x[1, 1, n[1] - 1] = float("inf")
    h0[2, 0], h0[2, 2] = float("nan"), -float("inf")
    y, h, states = block.scan_fwd(x, r, i, lam, h0, lengths)
    dx, dr, di, dlam, dh0 = block.scan_bwd(dy, x, r, i, lam, states, dh, lengths)
    for b in range(B):
        for t in (y, dx, dr, di):
            assert (t[b, :, n[b]:] == 0).all(), b
    assert torch.equal(dlam[[0, 2]], clean[3][[0, 2]]) and dlam[1].isnan()
    assert torch.equal(dh0[2], dh[2])
    for a, c in zip((dx, dr, di), clean):
        assert torch.equal(a[:, [0, 2]], c[:, [0, 2]]) and torch.equal(a[2:], c[2:])


def test_scan_against_differences():
    """The kernels' own forward pass, moved along a direction: 32-bit roundings of a sum of 10^4 terms of order 1 against steps of
    2^-5 give about 1e-4 of the sum's size, the third derivative 2^-10 of it."""
    B, C, L = 2, 4, 1500
    x, r, i, dy, lam = scan_inputs(B, C, L, F32, 81)
    h0, dh = rand(B, C, seed=1), rand(B, C, seed=2)
    args = {"x": x, "r": r, "i": i, "lam": lam, "h0": h0}

    def loss(a):
        y, h, _ = block.scan_fwd(a["x"], a["r"], a["i"], a["lam"], a["h0"], save=False)
        return float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())
    _, _, states = block.scan_fwd(x, r, i, lam, h0)
    grads = dict(zip(("x", "r", "i", "lam", "h0"), block.scan_bwd(dy, x, r, i, lam, states, dh)))
    for name, t in args.items():
        d = rand(*t.shape, seed=20)
        e = 2.0 ** -5
        num = (loss({**args, name: t + e * d}) - loss({**args, name: t - e * d})) / (2 * e)
        size = float((grads[name].double() * d.double()).abs().sum())
        assert abs(num - float((grads[name].double() * d.double()).sum())) <= 2.0 ** -9 * size, name


@pytest.mark.parametrize("B,C,L", [(3, 5, 300), (2, 2, 70), (1, 1, 50000)])
def test_scan_repeats_and_streams(B, C, L):
    """The same bits again, on another stream than the default one, and with workspaces the caller keeps."""
    x, r, i, dy, lam = scan_inputs(B, C, L, BF16, 91)
    first = block.scan_fwd(x, r, i, lam)
    grads = block.scan_bwd(dy, x, r, i, lam, first[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        wf = torch.empty(max(16, block.scan_workspace_bytes(B, C, L, False)), dtype=torch.uint8, device="cuda")
        wb = torch.full((block.scan_workspace_bytes(B, C, L, True),), 255, dtype=torch.uint8, device="cuda")
        again = block.scan_fwd(x, r, i, lam, workspace=wf)
        grads2 = block.scan_bwd(dy, x, r, i, lam, again[2], workspace=wb)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*first, *grads), (*again, *grads2)))


def test_scan_above_32_bits():
    """More than 2^31 elements and 4 GiB a tensor: the last rows are those of a call of their own."""
    B, C, L = 5, 512, 860000
    assert B * C * L > 2 ** 31
    x, r, i = (torch.randn(B, C, L, device="cuda", dtype=BF16) for _ in range(3))
    lam = rand(C, seed=3) - 5
    y, h, states = block.scan_fwd(x, r, i, lam)
    y1, h1, s1 = block.scan_fwd(x[-1:], r[-1:], i[-1:], lam)
    # (another number of rows may be cut into other spans: bounds, not bits; a state's own size is about 1)
    assert (h[-1] - h1[0]).abs().max() < 1e-4 and (y[-1].float() - y1[0].float()).abs().max() < 2.0 ** -5
    assert (states[-1] - s1[0]).abs().max() < 1e-4
    del y, y1
    dx, dr, di, dlam, dh0 = block.scan_bwd(x, x, r, i, lam, states)
    e = block.scan_bwd(x[-1:], x[-1:], r[-1:], i[-1:], lam, s1)
    for a, b in ((dx, e[0]), (dr, e[1]), (di, e[2]), (dh0, e[4])):
        assert torch.isfinite(a[-1].float()).all() and (a[-1].float() - b[0].float()).abs().max() < 2.0 ** -4 * (1 + b.float().abs().max())


def test_scan_step_is_the_scan():
    B, C, L, pool = 5, 70, 20, 9
    for dtype in (F32, BF16):
        x, r, i, _, lam = scan_inputs(B, C, L, dtype, 101)
        h0 = rand(B, C, seed=1)
        want, err = ref.scan(x, r, i, lam, h0)
        slots = torch.tensor([7, 0, -1, 3, 9], dtype=torch.int32, device="cuda")        # (two empty places, one of them outside)
        h = rand(pool, C, seed=4)
        used = [0, 1, 3]
        h[slots[used].long()] = h0[used]
        rest = h.clone()
        own = h0.clone()
        for t in range(L):
            wide = torch.stack([x[..., t], r[..., t], i[..., t]], 1)                    # (channel slices of one tensor)
            y = block.scan_step(wide[:, 0], wide[:, 1], wide[:, 2], lam, h, slots)
            y2 = block.scan_step(x[..., t].contiguous(), r[..., t].contiguous(), i[..., t].contiguous(), lam, own)
            assert torch.equal(y[used], y2[used]) and (y[[2, 4]] == 0).all()
            ref.check(y2, want["y"][..., t], err["y"][..., t], dtype, "y")
        ref.check(own, want["h_last"], err["h_last"], F32, "h")
        assert torch.equal(h[slots[used].long()], own[used])
        left = [1, 2, 4, 5, 6, 8]
        assert torch.equal(h[left], rest[left])


# ---- norms ----

NORM_SHAPES = [(2, 1, 1), (3, 5, 1), (2, 768, 1), (2, 5000, 1), (70, 33, 1), (3, 254, 1), (3, 257, 1), (2, 1023, 1), (2, 1030, 1), (2, 2047, 1), (3, 7, 2), (2, 33, 3), (2, 64, 7), (2, 100, 8), (3, 129, 9), (2, 256, 33),
               (1, 768, 100), (2, 700, 65), (1, 1100, 40), (1, 2300, 17), (1, 4200, 35), (1, 9000, 20), (40, 3, 100), (5, 32, 257),
               # (every number of rounds of channels, in workgroups of each size, and tiles that share a workgroup)
               (2, 20, 70), (2, 60, 64), (2, 130, 40), (1, 200, 66), (1, 390, 34), (1, 500, 31), (1, 650, 64), (1, 1500, 33), (1, 3300, 16), (17000, 3, 9)]


def norm_inputs(B, C, L, dtype, seed=200):
    y, z, res, dout, dn = (rand(B, C, L, seed=seed + k, dtype=dtype) for k in range(5))
    return y, z, res, dout, dn, 1 + 0.2 * rand(C, seed=seed + 6), 1 + 0.2 * rand(C, seed=seed + 7)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,C,L", NORM_SHAPES)
def test_norm(B, C, L, dtype):
    y, z, res, dout, dn, w, wn = norm_inputs(B, C, L, dtype)
    for case in ("block", "no block", "no dout"):
        d = None if case == "no dout" else dout
        a = (None, None, res, None, wn) if case == "no block" else (y, z, res, w, wn)
        want, err = ref.norm(*a, eps=1e-5, scale=0.5, dout=d, dn=dn)
        out, n, stats = block.norm_fwd(*a, eps=1e-5, scale=0.5)
        got = dict(zip(("dy", "dz", "dres", "dw", "dw_next"), block.norm_bwd(d, dn, *a, stats, scale=0.5)), out=out, n=n)
        got = {k: v for k, v in got.items() if v is not None}
        assert got.keys() == want.keys()
        for k, v in got.items():
            assert v.dtype == (F32 if k in ("dw", "dw_next") else dtype)
            ref.check(v, want[k], err[k], v.dtype, (case, k))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C,L", [(c, n) for c in (1, 64, 65, 150, 200, 300, 384, 385, 500, 640, 700, 768, 769) for n in (2, 3, 5, 7, 9)]
                         + [(c, n) for c in (31, 64, 65, 96, 128, 129, 192, 193, 300, 330) for n in (12, 17, 35)] + [(16, 64), (17, 70), (32, 33), (33, 130)])
def test_norm_of_short_rows(C, L, dtype):
    """Tiles of a wave and of two, of less than a pack and of one, the last workgroup with fewer tiles than it has room for."""
    y, z, res, dout, dn, w, wn = norm_inputs(5, C, L, dtype)
    for d, a in ((dout, (y, z, res, w, wn)), (None, (None, None, res, None, wn))):
        want, err = ref.norm(*a, eps=1e-5, scale=0.5, dout=d, dn=dn)
        out, n, stats = block.norm_fwd(*a, eps=1e-5, scale=0.5)
        got = dict(zip(("dy", "dz", "dres", "dw", "dw_next"), block.norm_bwd(d, dn, *a, stats, scale=0.5)), out=out, n=n)
        for k, v in got.items():
            if v is not None:
                ref.check(v, want[k], err[k], v.dtype, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [1, 63, 64, 65, 127, 128, 129, 200])
@pytest.mark.parametrize("L", [1, 2])
@pytest.mark.parametrize("B", [1023, 1024, 1500])
def test_norm_of_one_or_two_positions_of_many_entries(B, C, L, dtype):
    """On both sides of 1024 entries and of 128 channels, where tiles of a wave take over from other kernels; the last workgroup with fewer tiles than
    it has room for (1023, 1500) and not."""
    y, z, res, dout, dn, w, wn = norm_inputs(B, C, L, dtype)
    for d, a in ((dout, (y, z, res, w, wn)), (None, (None, None, res, None, wn))):
        want, err = ref.norm(*a, eps=1e-5, scale=0.5, dout=d, dn=dn)
        out, n, stats = block.norm_fwd(*a, eps=1e-5, scale=0.5)
        got = dict(zip(("dy", "dz", "dres", "dw", "dw_next"), block.norm_bwd(d, dn, *a, stats, scale=0.5)), out=out, n=n)
        for k, v in got.items():
            if v is not None:
                ref.check(v, want[k], err[k], v.dtype, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,C,L", [(70000, 3, 9), (300000, 2, 3)])
def test_norm_of_very_many_tiles(B, C, L, dtype):
    """Sums over more tiles than the first of their two launches has few runs for."""
    y, z, res, dout, dn, w, wn = norm_inputs(B, C, L, dtype)
    want, err = ref.norm(y, z, res, w, wn, eps=1e-5, scale=0.5, dout=dout, dn=dn)
    out, n, stats = block.norm_fwd(y, z, res, w, wn, eps=1e-5, scale=0.5)
    got = dict(zip(("dy", "dz", "dres", "dw", "dw_next"), block.norm_bwd(dout, dn, y, z, res, w, wn, stats, scale=0.5)), out=out, n=n)
    for k, v in got.items():
        ref.check(v, want[k], err[k], v.dtype, k)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C,L", [(12, 1), (11, 1), (12, 5), (12, 70), (700, 30), (5000, 21)])
@pytest.mark.parametrize("kind", ["slice", "odd"])
def test_norm_layouts(C, L, kind, dtype):
    y, z, res, dout, dn, w, wn = norm_inputs(3, C, L, dtype)
    out, n, stats = block.norm_fwd(y, z, res, w, wn)
    want = (out, n, *block.norm_bwd(dout, dn, y, z, res, w, wn, stats))
    ys, zs, rs, ds, ns = (strided(t, kind) for t in (y, z, res, dout, dn))
    o = [strided(torch.zeros_like(res), kind) for _ in range(5)]
    out, n, stats2 = block.norm_fwd(ys, zs, rs, w, wn, out=o[0], out_n=o[1])
    got = (out, n, *block.norm_bwd(ds, ns, ys, zs, rs, w, wn, stats2, out=o[2:]))
    assert torch.equal(stats, stats2) and all(torch.equal(a, b) for a, b in zip(want, got))
    if kind == "slice":
        for t in o:
            wide = t._base
            assert wide[:, :C + 1].isnan().all() and wide[:, 2 * C + 1:].isnan().all()


@pytest.mark.parametrize("C,L", [(20, 1), (20, 6), (20, 40), (5000, 20)])
def test_norm_keeps_bad_values_at_their_position(C, L):
    y, z, res, dout, dn, w, wn = norm_inputs(2, C, L, F32)
    clean = block.norm_fwd(y, z, res, w, wn)
    at = L // 2
    y[1, 3, at], z[0, 2, at] = float("nan"), float("inf")
    out, n, stats = block.norm_fwd(y, z, res, w, wn)
    keep = torch.ones(L, dtype=torch.bool)
    keep[at] = False
    for a, b in ((out, clean[0]), (n, clean[1])):
        assert torch.equal(a[..., keep], b[..., keep])
    assert out[1, :, at].isnan().all() and n[0, :, at].isnan().any()
    g = block.norm_bwd(dout, dn, y, z, res, w, wn, stats)
    assert all(torch.isfinite(t[..., keep]).all() for t in g[:3])


def test_norm_of_zeros_and_of_large_and_small_values():
    y, z, res, dout, dn, w, wn = norm_inputs(2, 48, 24, F32)
    y[0], res[1, :, 3] = 0.0, 0.0
    y[1, :, 5] *= 1e15
    y[1, :, 6] *= 1e-15
    z[1, :, 7], z[1, :, 8] = -200.0, 200.0
    want, err = ref.norm(y, z, res, w, wn, dout=dout, dn=dn)
    out, n, stats = block.norm_fwd(y, z, res, w, wn)
    got = dict(zip(("dy", "dz", "dres", "dw", "dw_next"), block.norm_bwd(dout, dn, y, z, res, w, wn, stats)), out=out, n=n)
    for k, v in got.items():
        # (a logit of 200 puts as many roundings on the exponential's argument; the products of shut gates may be flushed)
        ref.check(v, want[k], 6 * err[k], F32, k, floor=1e-30)


def test_norm_above_32_bits():
    B, C, L = 3, 768, 950000
    assert B * C * L > 2 ** 31
    y, z, res = (torch.randn(B, C, L, device="cuda", dtype=BF16) for _ in range(3))
    w, wn = rand(C, seed=1), rand(C, seed=2)
    out, n, stats = block.norm_fwd(y, z, res, w, wn)
    tail = slice(L - 64, L)
    args = [t[-1:, :, tail].contiguous() for t in (y, z, res)]
    o1, n1, s1 = block.norm_fwd(*args, w, wn)
    assert torch.equal(out[-1:, :, tail], o1) and torch.equal(n[-1:, :, tail], n1) and torch.equal(stats[-1:, :, tail], s1)
    dy, dz, dres, dw, dwn = block.norm_bwd(out, n, y, z, res, w, wn, stats)
    e = block.norm_bwd(o1, n1, *args, w, wn, s1)
    for a, b in ((dy, e[0]), (dz, e[1]), (dres, e[2])):
        assert torch.equal(a[-1:, :, tail], b)


# ---- clipping ----

@pytest.mark.parametrize("C,L", [(1, 4), (2, 9)])
def test_norm_of_more_tiles_than_a_grid_has(C, L):
    B = (1 << 22) + 5
    y, z, res, dout, dn = (torch.randn(B, C, L, device="cuda") for _ in range(5))
    w, wn = rand(C, seed=1), rand(C, seed=2)
    out, n, stats = block.norm_fwd(y, z, res, w, wn)
    dy, dz, dres, dw, dwn = block.norm_bwd(dout, dn, y, z, res, w, wn, stats)
    for at in (slice(0, 40), slice(B // 2, B // 2 + 40), slice(B - 40, B)):
        want, err = ref.norm(*(t[at] for t in (y, z, res)), w, wn, dout=dout[at], dn=dn[at])
        for k, v in dict(out=out, n=n, dy=dy, dz=dz, dres=dres).items():
            ref.check(v[at], want[k], err[k], F32, k)
    # (a workgroup adds up to 4200 tiles one by one, the rest in a tree; a term has fewer than 40 roundings)
    y, z, res, dout, dn = (t.double() for t in (y, z, res, dout, dn))
    wd, wnd = w.double()[:, None], wn.double()[:, None]
    yh, silu = y * (y.square().mean(1, keepdim=True) + 1e-6).rsqrt(), z * torch.sigmoid(z)
    o = res + silu * yh * wd
    r2 = (o.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    d = dout + r2 * (dn * wnd - o * r2 * (dn * wnd * o * r2).mean(1, keepdim=True))
    for got, term in ((dwn, dn * o * r2), (dw, d * silu * yh)):
        assert ((got.double() - term.sum((0, 2))).abs() <= 4300 * 2.0 ** -24 * term.abs().sum((0, 2))).all()


def clip_ref(grads, max_norm):
    norm = math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))
    return norm, min(1.0, max_norm / (norm + 1e-6))


@pytest.mark.parametrize("sizes", [[1], [0, 5, 0], [8191, 8192, 8193, 3], [100, 7] * 30, [33] * 250, [5_000_000, 17]])
@pytest.mark.parametrize("target", [0.3, 7.0])
def test_clip(sizes, target):
    total = sum(sizes)
    grads = [(rand(n, seed=k) * (target / math.sqrt(total))).to(BF16 if k % 3 == 1 else F32) for k, n in enumerate(sizes)]
    grads = [strided(g.view(1, -1), "odd").view(-1) if k % 4 == 2 and g.numel() else g for k, g in enumerate(grads)]
    norm, f = clip_ref(grads, 1.0)
    before = [g.clone() for g in grads]
    outs = [torch.full_like(g, float("nan")) for g in grads]
    got = block.clip_grad_norm(grads, 1.0, out=outs)
    assert got.dtype == F32 and got.dim() == 0 and abs(float(got) - norm) <= ref.U * norm
    for g, b, o in zip(grads, before, outs):
        assert torch.equal(g, b)                        # (inputs are not written)
        # the factor and the product are rounded once each
        ref.check(o, b.double().cpu() * f, b.double().abs().cpu() * f * 2 * ref.U, o.dtype, "out")
    assert torch.equal(block.clip_grad_norm(grads, 1.0), got)
    for g, b, o in zip(grads, before, outs):
        assert torch.equal(g, o)
        if target < 1:
            assert torch.equal(g, b)                    # (nothing to clip: not a bit changes)


def test_clip_of_large_small_and_bad_values():
    a, b = torch.full((1000,), 1e30, device="cuda"), torch.full((3,), 1e-30, device="cuda")
    n = block.clip_grad_norm([a, b], 1.0)
    assert abs(float(n) - 1e30 * math.sqrt(1000)) < 1e-6 * 1e32 and torch.allclose(a, torch.full_like(a, 1 / math.sqrt(1000)), rtol=1e-6)
    assert abs(float(block.clip_grad_norm([b], 1.0)) - 0) < 1e-30         # (below 1: unchanged)
    s = torch.full((4,), 1e-30, device="cuda")
    assert abs(float(block.clip_grad_norm([s], 1.0)) / 2e-30 - 1) < 1e-6 and (s == torch.tensor(1e-30)).all()
    g, h = torch.ones(10, device="cuda"), torch.ones(10, device="cuda", dtype=BF16)
    h[3] = float("inf")
    n = block.clip_grad_norm([g, h], 1.0)
    assert torch.isinf(n) and (g == 0).all() and h[3].isnan() and (h[:3] == 0).all()
    g, h = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    h[3] = float("nan")
    assert block.clip_grad_norm([g, h], 1.0).isnan() and g.isnan().all()
    z = torch.zeros(20, device="cuda")
    assert float(block.clip_grad_norm([z], 1.0)) == 0 and (z == 0).all()


def test_clip_layouts_and_refusals():
    base = rand(6, 10, seed=1)
    t = base.t()
    norm, f = clip_ref([t], 0.1)
    want = t.double().cpu() * f
    block.clip_grad_norm([t], 0.1)
    assert torch.allclose(t.double().cpu(), want, rtol=1e-6)
    x = rand(6, 10, seed=1)
    for bad in (lambda: block.clip_grad_norm([x[:, ::2]], 1.0), lambda: block.clip_grad_norm([x], 1.0, out=[x.t().contiguous().t()]),
                lambda: block.clip_grad_norm([x], 1.0, out=[]), lambda: block.clip_grad_norm([x, x.cpu()], 1.0), lambda: block.clip_grad_norm([x], 1.0, out=[x.bfloat16()])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        block.clip_grad_norm([x.half()], 1.0)
    for m in (0.0, -1.0, float("nan")):
        with pytest.raises(binding.DwconvError):
            block.clip_grad_norm([x], m)


# ---- the convolution, one token ----

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 8, 31, 32, 64, 100, 300])
def test_conv_step_is_the_convolution(K, dtype):
    """A prompt through dwconv_fwd and conv_ring, then token by token, against the whole sequence: K products of rounded values, a
    sum of K terms."""
    B, C, L, n, pool = 4, 37, 2 * K + 9, K + 3, 7
    x, w = rand(B, C, L, seed=K, dtype=dtype), (rand(C, K, seed=K + 1) / math.sqrt(K)).to(dtype)
    pad = torch.nn.functional.pad(x.double().cpu(), (K - 1, 0))
    win = pad.unfold(2, K, 1)
    want, size = (win * w.double().cpu()[:, None, :]).sum(-1), (win * w.double().cpu()[:, None, :]).abs().sum(-1)
    lengths = torch.tensor([n, 0, 1, n - 1], dtype=torch.int32, device="cuda")
    slots = torch.tensor([5, 2, -1, 0], dtype=torch.int32, device="cuda")
    ring = rand(pool, C, K, seed=9, dtype=dtype)
    other = ring.clone()
    block.conv_ring(x[:, :, :n].contiguous(), ring, lengths, slots)
    pos = lengths.clone()
    for _ in range(K + 3):
        t = pos.long()
        tok = x[torch.arange(B, device="cuda"), :, t]
        y = block.conv_step(tok, w, ring, pos, slots)
        assert (y[2] == 0).all()
        for b in (0, 1, 3):
            ref.check(y[b], want[b, :, int(t[b])], size[b, :, int(t[b])] * (K + 2) * ref.U / 2, dtype, ("y", b, int(t[b])))
        pos += 1
    assert torch.equal(ring[[1, 3, 4, 6]], other[[1, 3, 4, 6]])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,C,K", [(700, 300, 11), (3, 5000, 200), (2000, 260, 33), (5, 3, 2500), (70000, 2, 3), (1, 1, 1), (2, 33, 2045)])
def test_conv_step_of_any_batch(B, C, K, dtype):
    """One and several sequences of a workgroup in flight, rings longer than a workgroup's lanes and than LDS, places left empty."""
    x, w, ring = rand(B, C, seed=1, dtype=dtype), (rand(C, K, seed=2) / math.sqrt(K)).to(dtype), rand(B + 1, C, K, seed=3, dtype=dtype)
    pos = torch.randint(0, 2 ** 31 - 1, (B,), generator=torch.Generator().manual_seed(4)).int().cuda()
    slots = torch.randperm(B, generator=torch.Generator().manual_seed(5)).int().cuda() + 1
    slots[::7] = -1
    before = ring.clone()
    y = block.conv_step(x, w, ring, pos, slots)
    used = (slots >= 0).nonzero()[:, 0]
    at, p = slots[used].long(), (pos[used] % K).long()
    full = before[at].double()
    full.scatter_(2, p[:, None, None].expand(-1, C, 1), x[used].double()[..., None])
    order = (p[:, None] + 1 + torch.arange(K, device="cuda")) % K
    terms = torch.gather(full, 2, order[:, None, :].expand(-1, C, -1)) * w.double()
    # (a sum of K rounded products in any order)
    ref.check(y[used], terms.sum(-1).cpu(), terms.abs().sum(-1).cpu() * (K + 2) * ref.U / 2, dtype, "y")
    assert (y[slots < 0] == 0).all()
    want = before.clone()
    want[at] = full.to(dtype)
    assert torch.equal(ring, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("K", [1, 2, 3, 5, 7, 8, 9, 24, 31, 32, 33, 63, 100, 260, 300, 2500])
def test_conv_step_with_an_infinite_tap(K, dtype):
    """It meets one input of the ring and nothing else, wherever the position puts it."""
    B, C = min(K + 2, 200), 5
    x, ring = torch.ones(B, C, device="cuda", dtype=dtype), torch.ones(B, C, K, device="cuda", dtype=dtype)
    pos = torch.arange(B, device="cuda", dtype=torch.int32) + max(0, K - B // 2)
    for j in sorted({0, 1 % K, K // 2, max(0, K - 2), K - 1}):
        w = torch.full((C, K), 0.5, device="cuda", dtype=dtype)
        w[0, j], w[1, j], w[2, j] = float("inf"), -float("inf"), float("nan")
        y = block.conv_step(x, w, ring, pos)
        assert (y[:, 0] == float("inf")).all() and (y[:, 1] == -float("inf")).all() and y[:, 2].isnan().all(), j
        assert (y[:, 3:] == torch.tensor(K * 0.5, dtype=dtype)).all(), j


def test_conv_step_at_any_position():
    """Positions up to the largest int32, and no slots: the place in the ring is the position's remainder."""
    B, C, K = 3, 20, 7
    x, w, ring = rand(B, C, seed=1), rand(C, K, seed=2), rand(B, C, K, seed=3)
    pos = torch.tensor([2 ** 31 - 1, 6, 2 ** 31 - 8], dtype=torch.int32, device="cuda")
    r = ring.clone()
    y = block.conv_step(x, w, r, pos)
    for b, p in enumerate(pos.tolist()):
        full = ring[b].double().cpu()
        full[:, p % K] = x[b].double().cpu()
        want = (torch.roll(full, K - 1 - p % K, 1) * w.double().cpu())
        ref.check(y[b], want.sum(1), want.abs().sum(1) * (K + 2) * ref.U / 2, F32, "y")
        assert torch.equal(r[b].double().cpu(), full)


# ---- as many entries as a batch may have ----

def _most(value, dtype):
    """One value for 2^31 - 1 entries of one channel."""
    return torch.tensor([[value]], dtype=dtype, device="cuda").expand(2 ** 31 - 1, 1)


def test_steps_of_the_largest_batch():
    """Nearly all places empty: the last ones are what they are in a small batch, the others 0."""
    B, used = 2 ** 31 - 1, [5, 0, -1, 2, 6]
    n = len(used)
    slots = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    slots[-n:] = torch.tensor(used, dtype=torch.int32, device="cuda")
    few = slots[-n:].clone()
    x, r, i = (_most(v, BF16) for v in (0.75, -0.5, 1.25))
    lam, pool = torch.tensor([-5.0], device="cuda"), rand(7, 1, seed=1)
    h, h2 = pool.clone(), pool.clone()
    y = block.scan_step(x, r, i, lam, h, slots)
    y2 = block.scan_step(x[:n], r[:n], i[:n], lam, h2, few)
    assert torch.equal(y[-n:], y2) and torch.equal(h, h2) and y2.count_nonzero() == 4 and not y[:-n].any()
    del y
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    pos[-n:] = 11
    for K in (3, 2500):
        w, pool = rand(1, K, seed=2, dtype=BF16), rand(7, 1, K, seed=3, dtype=BF16)
        ring, ring2 = pool.clone(), pool.clone()
        y = block.conv_step(x, w, ring, pos, slots)
        y2 = block.conv_step(x[:n], w, ring2, pos[-n:], few)
        assert torch.equal(y[-n:], y2) and torch.equal(ring, ring2) and y2.count_nonzero() == 4 and not y[:-n].any()
        del y
    ring, ring2 = pool.clone(), pool.clone()
    block.conv_ring(x[..., None], ring, pos, slots)
    block.conv_ring(x[:n, :, None], ring2, pos[-n:], few)
    assert torch.equal(ring, ring2) and not torch.equal(ring, pool)


def test_norm_of_the_largest_batch():
    res, one = _most(-3.0, BF16)[..., None], torch.ones(1, device="cuda")
    _, n, _ = block.norm_fwd(None, None, res, None, one, save=False)
    assert bool((n == -1).all())


# ---- together ----

def test_a_token_in_a_graph():
    """Convolution, recurrence and norm of one token, recorded and replayed as the sequence goes on."""
    B, C, K, T = 6, 48, 9, 5
    w, lam, wn1, wn2 = rand(C, K, seed=1) / 3, rand(C, seed=2) - 5, 1 + 0.1 * rand(C, seed=3), 1 + 0.1 * rand(C, seed=4)
    tokens, gates = rand(T, B, C, seed=5), rand(T, B, 3 * C, seed=6)

    def step(x, g, ring, h, pos):
        u = block.conv_step(x, w, ring, pos)
        y = block.scan_step(u, g[:, :C], g[:, C:2 * C], lam, h)
        return block.norm_fwd(y[..., None], g[:, 2 * C:, None], x[..., None], wn1, wn2, save=False)
    new = lambda: (torch.zeros(B, C, K, device="cuda"), torch.zeros(B, C, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda"))   # noqa: E731
    ring, h, pos = new()
    want = []
    for t in range(T):
        want.append([v.clone() for v in step(tokens[t], gates[t], ring, h, pos)[:2]])
        pos += 1
    ring, h, pos = new()
    x, g = tokens[0].clone(), gates[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, g, *new())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, n, _ = step(x, g, ring, h, pos)
        pos += 1
    ring.zero_(), h.zero_(), pos.zero_()
    for t in range(T):
        x.copy_(tokens[t]), g.copy_(gates[t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[t][0]) and torch.equal(n, want[t][1]), t


def test_refusals():
    x, r, i, dy, lam = scan_inputs(2, 3, 20, F32, 1)
    y, h, states = block.scan_fwd(x, r, i, lam)
    c = torch.ones(3, device="cuda")
    value, kind = (
        lambda: block.scan_fwd(x, r[:, :2], i, lam), lambda: block.scan_fwd(x.transpose(1, 2), r, i, lam), lambda: block.scan_fwd(x[0], r, i, lam),
        lambda: block.scan_fwd(x[..., ::2], r[..., ::2], i[..., ::2], lam), lambda: block.scan_fwd(x, r, i, lam[:2]), lambda: block.scan_fwd(x, r, i, lam, h0=h[:1]),
        lambda: block.scan_fwd(x, r, i, lam, out=torch.empty(1, 3, 20, device="cuda").expand(2, 3, 20)), lambda: block.scan_fwd(x, r.cpu(), i, lam),
        lambda: block.scan_bwd(dy, x, r, i, lam, states[:, :, :0]), lambda: block.scan_bwd(dy, x, r, i, lam, states, out=(x, x)),
        lambda: block.norm_fwd(x, None, r, c, c), lambda: block.norm_fwd(None, None, r, None, c, out=x), lambda: block.norm_bwd(None, dy, x, r, i, c, c, torch.ones(2, 2, 19, device="cuda")),
        lambda: block.conv_step(x[..., 0], c[:, None], torch.zeros(2, 3, 1, device="cuda"), None), lambda: block.conv_ring(x, torch.zeros(2, 4, 5, device="cuda")),
    ), (
        lambda: block.scan_fwd(x, r.bfloat16(), i, lam), lambda: block.scan_fwd(x, r, i, lam.double()), lambda: block.scan_fwd(x.half(), r.half(), i.half(), lam),
        lambda: block.scan_fwd(x, r, i, lam, lengths=torch.ones(2, device="cuda", dtype=torch.int64)), lambda: block.norm_fwd(x, r, i, c.bfloat16(), c),
        lambda: block.scan_step(h, h, h, lam, h.bfloat16()),
    )
    for call in value:
        with pytest.raises(ValueError):
            call()
    for call in kind:
        with pytest.raises(TypeError):
            call()
    for call in (lambda: block.scan_fwd(x, r, i, lam, rate=0.0), lambda: block.norm_fwd(x, r, i, c, c, eps=0.0), lambda: block.norm_fwd(x, r, i, c, c, scale=float("inf")),
                 lambda: block.scan_step(x[:, :, 0].contiguous(), r[:, :, 0].contiguous(), i[:, :, 0].contiguous(), lam, h[:1].contiguous()),
                 lambda: block.scan_bwd(dy, x, r, i, lam, states, workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(binding.DwconvError):
            call()


# ---- the native form of the calls ----

def _calls():
    x, r, i, dy, lam = scan_inputs(2, 6, 70, BF16, 301)
    h0, dh = rand(2, 6, seed=1), rand(2, 6, seed=2)
    lengths, slots = torch.tensor([70, 9], dtype=torch.int32, device="cuda"), torch.tensor([1, -1], dtype=torch.int32, device="cuda")
    states = block.scan_fwd(x, r, i, lam, h0, lengths)[2]
    y, z, res, dout, dn, w, wn = norm_inputs(2, 6, 70, F32)
    stats, stats0 = block.norm_fwd(y, z, res, w, wn)[2], block.norm_fwd(None, None, res, None, wn)[2]
    tok, h, ring = x[..., 0].contiguous(), rand(3, 6, seed=3), rand(3, 6, 5, seed=4, dtype=BF16)
    taps, pos = rand(6, 5, seed=5, dtype=BF16), torch.tensor([3, 9], dtype=torch.int32, device="cuda")
    outs = lambda t, n: [torch.full_like(t, float("nan")) for _ in range(n)]        # noqa: E731
    space = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    return {
        "scan_fwd": lambda: block.scan_fwd(x, r, i, lam, h0, lengths), "scan_fwd bare": lambda: block.scan_fwd(x, r, i, lam, save=False),
        "scan_fwd out": lambda: block.scan_fwd(x, r, i, lam, out=outs(x, 1)[0], workspace=space),
        "scan_bwd": lambda: block.scan_bwd(dy, x, r, i, lam, states, dh, lengths),
        "scan_bwd out": lambda: block.scan_bwd(dy, x, r, i, lam, states, out=outs(x, 3), workspace=space),
        "scan_step": lambda: (block.scan_step(tok, tok, tok, lam, g := h.clone(), slots), g), "scan_step out": lambda: (block.scan_step(tok, tok, tok, lam, h.clone(), out=outs(tok, 1)[0]),),
        "norm_fwd": lambda: block.norm_fwd(y, z, res, w, wn, scale=0.5), "norm_fwd bare": lambda: block.norm_fwd(None, None, res, None, wn, save=False),
        "norm_fwd out": lambda: block.norm_fwd(y, z, res, w, wn, out=outs(y, 1)[0], out_n=outs(y, 1)[0]),
        "norm_bwd": lambda: block.norm_bwd(dout, dn, y, z, res, w, wn, stats), "norm_bwd bare": lambda: block.norm_bwd(None, dn, None, None, res, None, wn, stats0),
        "norm_bwd out": lambda: block.norm_bwd(dout, dn, y, z, res, w, wn, stats, out=outs(y, 3), workspace=space),
        "conv_step": lambda: (block.conv_step(tok, taps, g := ring.clone(), pos, slots), g),
        "clip": lambda: (block.clip_grad_norm(g := [y.clone(), x.clone()], 1.0), *g), "clip out": lambda: (block.clip_grad_norm((y, x), 1.0, out=(g := outs(y, 1) + outs(x, 1))), *g),
    }


def test_native_calls_give_the_same(monkeypatch):
    from paper_2604_25422_amd import _fastcall
    block.lib()
    assert block._fast is _fastcall
    for name, call in _calls().items():
        fast = call()
        with monkeypatch.context() as m:
            m.setattr(block, "_fast", block._Declines)
            general = call()
        assert len(fast) == len(general), name
        for a, b in zip(fast, general):
            assert (a is None) == (b is None), name
            if a is not None:
                assert a.dtype == b.dtype and a.shape == b.shape and not a.requires_grad and torch.equal(a, b), name


def test_native_calls_take_what_they_should(monkeypatch):
    """They are the ones that run: none of the calls above is left to the general form."""
    block.lib()
    monkeypatch.setattr(block, "_check", None)
    for name, call in _calls().items():
        call()


@pytest.mark.parametrize("native", [True, False])
def test_clip_for_the_norm_alone(native, monkeypatch):
    """The largest finite limit scales nothing; an infinite one is refused, by both forms of the calls."""
    block.lib()
    if not native:
        monkeypatch.setattr(block, "_fast", block._Declines)
    grads = [rand(3000, seed=1) * 1e6, rand(70, seed=2, dtype=BF16)]
    before, outs = [g.clone() for g in grads], [torch.full_like(g, float("nan")) for g in grads]
    norm, f = clip_ref(grads, torch.finfo(F32).max)
    assert f == 1
    for out in (outs, None):
        got = block.clip_grad_norm(grads, torch.finfo(F32).max, out=out)
        assert abs(float(got) - norm) <= ref.U * norm
        assert all(torch.equal(a, b) for a, b in zip(grads if out is None else out, before))
    with pytest.raises(binding.DwconvError):
        block.clip_grad_norm(grads, float("inf"))


@pytest.mark.parametrize("native", [True, False])
def test_an_empty_workspace_is_too_small(native, monkeypatch):
    """Refused by both forms of the calls, and taken where none is needed."""
    block.lib()
    if not native:
        monkeypatch.setattr(block, "_fast", block._Declines)
    x, r, i, dy, lam = scan_inputs(2, 3, 20, F32, 1)
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    y, h, states = block.scan_fwd(x, r, i, lam, workspace=none)
    assert torch.equal(y, block.scan_fwd(x, r, i, lam)[0])
    c = torch.ones(3, device="cuda")
    stats = block.norm_fwd(x, r, i, c, c)[2]
    long = [torch.zeros(1, 1, 1 << 16, device="cuda") for _ in range(3)]
    assert block.scan_workspace_bytes(1, 1, 1 << 16, False) > 0
    for call in (lambda: block.scan_fwd(*long, lam[:1], workspace=none), lambda: block.scan_bwd(dy, x, r, i, lam, states, workspace=none),
                 lambda: block.norm_bwd(None, dy, x, r, i, c, c, stats, workspace=none), lambda: block.clip_grad_norm([x], 1.0, workspace=none)):
        with pytest.raises(binding.DwconvError) as e:
            call()
        assert e.value.status == 5


@pytest.mark.parametrize("given", [False, True])
def test_native_clipping_holds_what_it_works_on(given):
    """Lists that lose their tensors while the call runs, as another thread's clear() does where the interpreter's lock is away: the tensors live on
    until the call is through.  (The query of the current device is Python that the call runs; it empties the lists here.)"""
    import ctypes

    lib = block.lib()
    fast = binding._fast
    assert fast is not binding._Declines
    values = [rand(n, seed=n) for n in (5000, 17, 300)]
    norm, f = clip_ref(values, 1.0)
    grads, outs = [v.clone() for v in values], [torch.empty_like(v) for v in values]
    kept = torch.empty(sum(v.numel() for v in values), device="cuda")
    if not given:                               # (in place: views of one tensor, which shows what has been written)
        grads = list(kept.split([v.numel() for v in values]))
        for g, v in zip(grads, values):
            g.copy_(v)
    else:
        outs = list(kept.split([v.numel() for v in values]))

    def current_device():
        grads.clear(), outs.clear()
        [torch.zeros(n, device="cuda") for n in (5000, 17, 300)]
        return binding._current_device()
    addresses = [ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in ("dwconv_fwd", "dwconv_bwd_input", "dwconv_bwd_weight", "dwconv_bwd")]
    fast.setup(*addresses, current_device, binding._raw_stream, binding._check)
    try:
        got = fast.clip_grad_norm(grads, 1.0, outs if given else None, None)
    finally:
        fast.setup(*addresses, binding._current_device, binding._raw_stream, binding._check)
    assert grads == [] and got is not None and abs(float(got) - norm) <= ref.U * norm
    want = torch.cat(values).double().cpu() * f
    ref.check(kept, want, want.abs() * 2 * ref.U, F32, "out")


def test_the_example_learns_and_serves():
    """Convolution, scan, norms and clipping in one model: its loss falls, and what it says token by token is what it says of the whole
    sequence.  (Logits of a model of this width pass some thousand 32-bit operations in another order: 2^-14 of the largest.)"""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block.py")
    spec = importlib.util.spec_from_file_location("gated_block", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, off, size = example.main(steps=60)
    assert losses[0] > 2.5 and losses[-1] < 0.5 * losses[0]
    assert off <= 2.0 ** -14 * size


def test_the_example_s_gradients():
    """A whole model's gradient along a direction against the difference of its loss."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_block.py")
    spec = importlib.util.spec_from_file_location("gated_block", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    model = example.Model(32, 48, 8, 2, seed=3)
    tokens = example.batch(32, 8, 70, seed=1)

    def loss():
        return torch.nn.functional.cross_entropy(model.logits(tokens[:, :-1]).double(), tokens[:, 1:])
    params = model.parameters()
    grads = torch.autograd.grad(loss(), params)
    for p, g in zip(params, grads):
        d = rand(*p.shape, seed=7) * 1e-2 * (1 + p.detach().abs().mean())
        with torch.no_grad():
            p += d
            up = float(loss())
            p -= 2 * d
            down = float(loss())
            p += d
        want = 2 * float((g.double() * d.double()).sum())
        # roundings of a 32-bit forward pass in a mean of 560 losses (1e-6 of about 4), and the third derivative: a steps's square of 1e-4
        assert abs(up - down - want) <= 2e-2 * abs(want) + 2e-5, tuple(p.shape)

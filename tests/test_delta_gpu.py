"""The gated delta rule and dropout on the GPU against their definitions in 64 bits and whole numbers (tests/_delta_ref.py, which also
derives the bounds), at the lengths, heads, layouts and masks where the kernels change form or could go wrong."""
import math

import pytest
import torch

import _delta_ref as ref
from paper_2604_25422_amd import binding, block

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def rand(*shape, seed, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def strided(t, kind):
    """The same values as a slice of the channels of a wider tensor ("slice"), or off its granule ("odd")."""
    B, C = t.shape[:2]
    if kind == "slice":
        wide = torch.full((B, 2 * C + 3, *t.shape[2:]), float("nan"), dtype=t.dtype, device="cuda")
        v = wide[:, C + 1:2 * C + 1]
    else:
        v = torch.full((t.numel() + 3,), float("nan"), dtype=t.dtype, device="cuda")[1:1 + t.numel()].view(t.shape)
    v.copy_(t)
    return v


def inputs(B, H, Hk, DK, DV, L, dtype, seed=1, rate=0.2):
    q, k = (rand(B, Hk * DK, L, seed=seed + i, dtype=dtype) for i in range(2))
    v, do = (rand(B, H * DV, L, seed=seed + 2 + i, dtype=dtype) for i in range(2))
    g, beta = -rate * rand(B, H, L, seed=seed + 4).abs(), torch.sigmoid(rand(B, H, L, seed=seed + 5))
    s0, ds = (rand(B, H, DK, DV, seed=seed + 6 + i) / math.sqrt(DK) for i in range(2))
    return q, k, v, g, beta, s0, do, ds


NAMES = ("dq", "dk", "dv", "dg", "dbeta", "ds0")


def check_rule(q, k, v, g, beta, s0, do, ds, lengths=None, key_heads=None, **more):
    want = ref.rule(q, k, v, g, beta, s0, lengths, key_heads, do=do, ds_last=ds, **more)
    o, s_last, states = block.delta_fwd(q, k, v, g, beta, s0, lengths, key_heads, **more)
    got = dict(zip(NAMES, block.delta_bwd(do, q, k, v, g, beta, states, ds, lengths, key_heads, **more)))
    got.update(o=o, s_last=s_last)
    for name, x in got.items():
        assert x.dtype == (q.dtype if name in ("o", "dq", "dk", "dv") else F32)
        ref.check(x, want[name], name)
    if lengths is not None:
        for b, n in enumerate(lengths.cpu().clamp(0, g.shape[2]).tolist()):
            for name in ("o", "dq", "dk", "dv", "dg", "dbeta"):
                assert (got[name][b, :, n:] == 0).all(), name
    return got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("L", [1, 2, 5, 7, 8, 9, 16, 17, 63, 64, 65, 100, 127, 128, 129, 200, 330])
def test_lengths(L, dtype):
    check_rule(*inputs(2, 2, 2, 24, 40, L, dtype, seed=L))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("DK,DV", [(1, 1), (1, 20), (16, 16), (17, 3), (31, 33), (32, 64), (33, 128), (64, 64), (64, 96), (65, 17), (100, 128), (128, 128),
                                   (128, 1), (96, 130), (128, 300), (5, 1000)])
def test_widths(DK, DV, dtype):
    check_rule(*inputs(2, 2, 2, DK, DV, 140, dtype, seed=DK + DV))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,H,Hk,DK,DV,L", [(1, 1, 1, 3, 65536, 70), (1, 1500, 500, 2, 3, 9), (2, 40, 40, 128, 2, 5)])
def test_widest(B, H, Hk, DK, DV, L, dtype):
    check_rule(*inputs(B, H, Hk, DK, DV, L, dtype, seed=DV), key_heads=Hk)


@pytest.mark.parametrize("size", [2.0 ** -90, 2.0 ** 100])
def test_sizes(size):
    """Values and states far from 1, fp32: every limb of theirs is still a normal number."""
    q, k, v, g, beta, s0, do, ds = inputs(2, 2, 1, 40, 24, 150, F32, seed=31)
    check_rule(q, k, v * size, g, beta, s0 * size, do, ds, key_heads=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,H,Hk,DK,DV", [(1, 4, 1, 32, 20), (2, 6, 3, 64, 48), (3, 8, 2, 128, 64), (1, 12, 12, 16, 16), (5, 1, 1, 40, 128), (2, 3, 1, 100, 70)])
def test_shared_keys(B, H, Hk, DK, DV, dtype):
    check_rule(*inputs(B, H, Hk, DK, DV, 150, dtype, seed=H + DK), key_heads=Hk)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("DK,DV,L", [(32, 32, 90), (64, 40, 200), (128, 128, 70), (20, 130, 193)])
def test_padded_batches(DK, DV, L, dtype):
    """Lengths of 0, 1, whole chunks, beyond the ends; what lies behind them is not looked at."""
    ends = [0, 1, 64, 65, L - 1, L, L + 7, -3]
    lengths = torch.tensor(ends, dtype=torch.int32, device="cuda")
    a = list(inputs(len(ends), 2, 1, DK, DV, L, dtype, seed=L))
    for i, bad in ((0, float("nan")), (1, float("inf")), (2, float("nan")), (3, float("inf")), (4, float("nan")), (6, -float("inf"))):
        a[i] = a[i].clone()
        for b, n in enumerate(ends):
            a[i][b, :, max(n, 0):] = bad
    got = check_rule(*a, lengths=lengths, key_heads=1)
    for b in (0, 7):
        assert torch.equal(got["s_last"][b], a[5][b]) and torch.equal(got["ds0"][b], a[7][b])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["slice", "odd"])
@pytest.mark.parametrize("L", [3, 70, 128])
def test_layouts(kind, L, dtype):
    q, k, v, g, beta, s0, do, ds = inputs(3, 4, 2, 20, 24, L, dtype, seed=L)
    want = block.delta_fwd(q, k, v, g, beta, s0, key_heads=2)
    grads = block.delta_bwd(do, q, k, v, g, beta, want[2], ds, key_heads=2)
    s = [strided(t, kind) for t in (q, k, v, g, beta, do)]
    o = strided(torch.empty_like(v), kind)
    got = block.delta_fwd(*s[:5], s0, key_heads=2, out=o)
    assert got[0] is o
    outs = tuple(strided(torch.empty_like(t), kind) for t in (q, k, v))
    got_grads = block.delta_bwd(s[5], *s[:5], got[2], ds, key_heads=2, out=outs)
    for a, b in zip((*want, *grads), (*got, *got_grads)):
        assert torch.equal(a, b)


def test_broadcast_inputs():
    """One sequence of keys and decays seen by the whole batch, and its gradients by entry."""
    q, k, v, g, beta, s0, do, ds = inputs(3, 2, 2, 16, 32, 100, F32)
    k1, g1 = k[:1].expand(3, -1, -1), g[:1].expand(3, -1, -1)
    a, b = check_rule(q, k1, v, g1, beta, s0, do, ds), check_rule(q, k1.contiguous(), v, g1.contiguous(), beta, s0, do, ds)
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("decay", [0.0, -1e-4, -3.0, -50.0, -90.0, -200.0, -float("inf")])
def test_decays(decay, dtype):
    """None at all, weak, so strong that nothing is left of a state, and all of them in one sequence."""
    q, k, v, g, beta, s0, do, ds = inputs(2, 2, 2, 32, 32, 150, dtype)
    check_rule(q, k, v, torch.full_like(g, decay), beta, s0, do, ds)
    g[:, 0, 5::7] = decay
    got = check_rule(q, k, v, g, beta, s0, do, ds)
    if decay < -104:
        assert (got["dg"][:, 0, 5::7] == 0).all()


def test_sequences_apart():
    """A decay of minus infinity at the start of every document of a packed row is a fresh start."""
    q, k, v, g, beta, s0, do, ds = inputs(1, 2, 2, 32, 48, 300, F32)
    starts = [0, 70, 71, 128, 250, 300]
    for t in starts[:-1]:
        g[:, :, t] = -float("inf")
    o, s_last, _ = block.delta_fwd(q, k, v, g, beta, s0)
    for a, b in zip(starts, starts[1:]):
        cut = [x[..., a:b].contiguous() for x in (q, k, v, g, beta)]
        alone, last, _ = block.delta_fwd(*cut, torch.zeros_like(s0))
        want = ref.rule(*cut)
        ref.check(o[..., a:b].contiguous(), want["o"], "o")
        ref.check(alone, want["o"], "o alone")
    ref.check(s_last, want["s_last"], "s_last")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("beta", [0.0, 1.0, 2.0])
def test_strengths(beta, dtype):
    q, k, v, g, b, s0, do, ds = inputs(2, 2, 1, 64, 32, 130, dtype)
    check_rule(q, k, v, g, torch.full_like(b, beta), s0, do, ds, key_heads=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_same_key_over_and_over(dtype):
    """beta = 1 writes what was there over: the state holds the last value alone."""
    q, k, v, g, beta, s0, do, ds = inputs(1, 1, 1, 32, 32, 128, dtype)
    k = k[..., :1].expand(-1, -1, 128).contiguous()
    check_rule(q, k, v, torch.zeros_like(g), torch.ones_like(beta), s0, do, ds)
    check_rule(q, k, v, g, beta, s0, do, ds)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_keys_of_no_length(dtype):
    q, k, v, g, beta, s0, do, ds = inputs(2, 2, 2, 32, 16, 100, dtype)
    k[:, :, 3::5], q[:, :, 4::5] = 0, 0
    check_rule(q, k, v, g, beta, s0, do, ds)
    check_rule(q, k / 4, v, g, beta, s0, do, ds, eps=0.0)
    check_rule(q * 1e-4, k * 1e-4, v, g, beta, s0, do, ds, eps=1e-6)


@pytest.mark.parametrize("scale", [0.0, -1.0, 3.5])
def test_scales(scale):
    check_rule(*inputs(1, 2, 2, 32, 16, 100, F32), scale=scale)
    q, k, *rest = inputs(1, 2, 2, 32, 16, 100, BF16)
    check_rule(q, k / 8, *rest, scale=scale, eps=0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H,Hk", [(2, 2), (4, 2)])
@pytest.mark.parametrize("scale", [1e-25, 1e25])
def test_scales_whose_squares_are_out_of_range(scale, H, Hk, dtype):
    check_rule(*inputs(2, H, Hk, 32, 32, 100, dtype, seed=21), key_heads=Hk, scale=scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,H,DK,DV,L", [(1, 1, 64, 64, 4200), (1, 2, 128, 128, 2100), (700, 1, 16, 16, 66), (40, 9, 32, 24, 70)])
def test_long_and_many(B, H, DK, DV, L, dtype):
    check_rule(*inputs(B, H, H, DK, DV, L, dtype, rate=0.05))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,H,Hk,DK,DV,L", [(2, 1, 1, 128, 40, 64 * 70 + 3), (3, 2, 1, 17, 130, 64 * 66), (1, 1, 1, 64, 64, 64 * 160 + 1)])
def test_many_segments(B, H, Hk, DK, DV, L, dtype):
    """Rows cut into so many segments that their spans are joined first; sequences that end in the first segments, in the last and between."""
    lengths = torch.tensor([L, 300, L - 70][:B], dtype=torch.int32, device="cuda")
    check_rule(*inputs(B, H, Hk, DK, DV, L, dtype, seed=L, rate=0.01), lengths=lengths, key_heads=Hk)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("DK", [20, 50, 100])
@pytest.mark.parametrize("B", [1024, 1030])
def test_as_many_chunks_as_run_at_once_and_more(B, DK, dtype):
    check_rule(*inputs(B, 1, 1, DK, 5, 9, dtype, seed=DK))


def test_without_what_may_be_left_out():
    q, k, v, g, beta, s0, do, ds = inputs(2, 2, 2, 24, 40, 100, F32)
    got = check_rule(q, k, v, g, beta, None, do, None)
    zero = check_rule(q, k, v, g, beta, torch.zeros_like(s0), do, torch.zeros_like(ds))
    assert all(torch.equal(got[n], zero[n]) for n in got)
    o, s_last, states = block.delta_fwd(q, k, v, g, beta, s0, save=False)
    full = block.delta_fwd(q, k, v, g, beta, s0)
    assert states is None and torch.equal(o, full[0]) and torch.equal(s_last, full[1])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("which", [0, 1, 2, 3, 4])
def test_bad_values_stay_in_their_head(which, bad):
    """... and behind the chunk that they are in."""
    a = list(inputs(2, 4, 2, 16, 24, 200, F32))
    good = check_rule(*a, key_heads=2)
    a[which] = a[which].clone()
    a[which][0, 0, 130] = bad
    o, s_last, states = block.delta_fwd(*a[:6], key_heads=2)
    grads = dict(zip(NAMES, block.delta_bwd(a[6], *a[:5], states, a[7], key_heads=2)))
    ov, gv = o.view(2, 4, 24, 200), good["o"].view(2, 4, 24, 200)
    heads = slice(0, 2) if which < 2 else slice(0, 1)           # those that share the key, or one
    rest = slice(heads.stop, 4)
    assert torch.equal(ov[1], gv[1]) and torch.equal(ov[0, rest], gv[0, rest]) and torch.equal(ov[0, heads, :, :128], gv[0, heads, :, :128])
    assert torch.equal(s_last[1], good["s_last"][1]) and torch.equal(s_last[0, rest], good["s_last"][0, rest])
    for name in NAMES:
        assert torch.equal(grads[name][1], good[name][1]), name
    for name in ("dg", "dbeta", "ds0"):
        assert torch.equal(grads[name][0, rest], good[name][0, rest]), name


@pytest.mark.parametrize("B,H,Hk,DK,DV,L", [(3, 4, 2, 24, 40, 300), (1, 2, 2, 128, 128, 700), (64, 2, 1, 32, 32, 65)])
def test_repeats_and_streams(B, H, Hk, DK, DV, L):
    """The same bits on another stream, after other work, with a workspace of the caller's that holds anything."""
    q, k, v, g, beta, s0, do, ds = inputs(B, H, Hk, DK, DV, L, BF16)
    run = lambda ws=None: (*(f := block.delta_fwd(q, k, v, g, beta, s0, key_heads=Hk, workspace=ws)), *block.delta_bwd(do, q, k, v, g, beta, f[2], ds, key_heads=Hk, workspace=ws))  # noqa: E731
    first = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ws = torch.full((block.delta_workspace_bytes(B, H, Hk, DK, DV, L, True) // 4,), float("nan"), device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = run(ws)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_a_step_of_training_in_a_graph():
    """Forward and backward recorded and replayed on other inputs, eager work of the same tensors between."""
    B, H, DK, DV, L = 2, 2, 32, 48, 130
    sets = [inputs(B, H, H, DK, DV, L, F32, seed=s) for s in (1, 50, 90)]
    rng = torch.tensor([7, 0], device="cuda")

    def step(q, k, v, g, beta, s0, do, ds):
        o, s_last, states = block.delta_fwd(q, k, v, g, beta, s0)
        y = block.dropout_fwd(o, 0.3, rng, 2, v)
        dy = block.dropout_bwd(do, 0.3, rng, 2)
        return (y, s_last, *block.delta_bwd(dy, q, k, v, g, beta, states, ds))
    held = [t.clone() for t in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*held)
    for n, s in enumerate((*sets, sets[1])):
        rng[1] = n
        want = [t.clone() for t in step(*s)]
        torch.cuda.synchronize()
        for h, t in zip(held, s):
            h.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), n


def test_rows_above_32_bits():
    """Batch entries that lie more than 2^31 elements apart."""
    B, H, DK, DV, L, far = 2, 1, 16, 32, 70, (1 << 31) + 4099
    q, k, v, g, beta, s0, do, ds = inputs(B, H, H, DK, DV, L, BF16)
    room = torch.zeros(far + DV * L, dtype=BF16, device="cuda")
    put = lambda t: (s := room.as_strided(t.shape, (far, L, 1)), s.copy_(t))[0]      # noqa: E731
    want = block.delta_fwd(q, k, v, g, beta, s0)
    grads = block.delta_bwd(do, q, k, v, g, beta, want[2], ds)
    got = block.delta_fwd(q, k, put(v), g, beta, s0)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    got = block.delta_bwd(put(do), q, k, v, g, beta, want[2], ds)
    assert all(torch.equal(a, b) for a, b in zip(grads, got))
    o = room.as_strided(v.shape, (far, L, 1))
    block.delta_fwd(q, k, v, g, beta, s0, out=o)
    assert torch.equal(o, want[0])


def test_states_above_32_bits():
    """More than 2^31 values of states, of which the last heads are looked at."""
    B, H, DK, DV, L = 1, 2100, 128, 128, 65 * 64 - 3
    assert B * H * 65 * DK * DV > 1 << 31
    q, k = (rand(1, 128, L, seed=i, dtype=BF16) for i in (1, 2))
    v = rand(1, 128, L, seed=3, dtype=BF16).repeat(1, H, 1)
    do = rand(1, 128, L, seed=4, dtype=BF16).repeat(1, H, 1)
    g, beta = -0.1 * rand(1, 1, L, seed=5).abs().expand(1, H, L), torch.sigmoid(rand(1, 1, L, seed=6)).expand(1, H, L)
    g, beta = g.contiguous(), beta.contiguous()
    o, s_last, states = block.delta_fwd(q, k, v, g, beta, key_heads=1)
    # (all heads are the same: the last as the first, which is checked; a call of one head may take another way and round differently)
    assert torch.equal(o[:, -128:], o[:, :128]) and torch.equal(s_last[:, -1], s_last[:, 0]) and torch.equal(states[:, -1], states[:, 0])
    want = ref.rule(q, k, v[:, :128], g[:, :1], beta[:, :1], do=do[:, :128])
    ref.check(o[:, :128], want["o"], "o"), ref.check(s_last[:, :1], want["s_last"], "s_last")
    grads = dict(zip(NAMES, block.delta_bwd(do, q, k, v, g, beta, states, key_heads=1)))
    for name, n in (("dv", 128), ("dg", 1), ("dbeta", 1), ("ds0", 1)):
        assert torch.equal(grads[name][:, -n:], grads[name][:, :n]), name
        ref.check(grads[name][:, :n], want[name], name)


def test_against_differences():
    """The gradients against differences of the forward pass itself."""
    q, k, v, g, beta, s0, do, ds = inputs(1, 2, 1, 16, 16, 80, F32)
    args = dict(q=q, k=k, v=v, g=g, beta=beta, s0=s0)

    def loss(a):
        o, s, _ = block.delta_fwd(**a, key_heads=1)
        return float((o.double() * do.double()).sum() + (s.double() * ds.double()).sum())
    _, _, states = block.delta_fwd(**args, key_heads=1)
    grads = dict(zip(NAMES, block.delta_bwd(do, q, k, v, g, beta, states, ds, key_heads=1)))
    want = ref.rule(**args, key_heads=1, do=do, ds_last=ds)
    for name, t in args.items():
        d, h = rand(*t.shape, seed=33), 2.0 ** -7
        num = (loss({**args, name: t + h * d}) - loss({**args, name: t - h * d})) / (2 * h)
        exact = float((want["d" + name][0] * d.double().cpu()).sum())
        # a central difference in 64 bits says how far this step is off; the forward pass's own bound over h the rest
        to = lambda s: {n: x.double().cpu() + (s * h * d.double().cpu() if n == name else 0) for n, x in args.items()}     # noqa: E731
        vals = []
        for s in (1, -1):
            r = ref.rule(**to(s), key_heads=1)
            vals.append(float((r["o"][0] * do.double().cpu()).sum() + (r["s_last"][0] * ds.double().cpu()).sum()))
            bound = float((r["o"][1] * do.double().cpu().abs()).sum() + (r["s_last"][1] * ds.double().cpu().abs()).sum())
        step = abs((vals[0] - vals[1]) / (2 * h) - exact)
        # (t + h d is rounded to 32 bits: 2^-24 of every input, by its gradient)
        moved = float((want["d" + name][0].abs() * (t.double().cpu().abs() + h * d.double().cpu().abs())).sum()) * 2.0 ** -24
        assert abs(num - float((grads["d" + name].double() * d.double()).sum())) <= step + (bound + moved) / h + float((want["d" + name][1] * d.double().cpu().abs()).sum()) + 1e-9, name


# ---- one token ----

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,H,Hk,DK,DV", [(1, 1, 1, 1, 1), (3, 2, 1, 16, 16), (2, 4, 4, 64, 64), (5, 4, 2, 100, 96), (2, 2, 2, 128, 128), (2, 1, 1, 17, 3),
                                          (1, 2, 1, 128, 300), (600, 1, 1, 33, 40), (1, 1, 1, 128, 5), (300, 2, 2, 8, 130)])
def test_a_token_is_the_rule(B, H, Hk, DK, DV, dtype):
    """Six tokens, one after the other, in rows of a pool in any order with places left empty; the others stay as they are."""
    T, pool = 6, B + 5
    q, k, v, g, beta, _, _, _ = inputs(B, H, Hk, DK, DV, T, dtype, seed=DK + DV)
    s = rand(pool, H, DK, DV, seed=3)
    slots = torch.randperm(pool, generator=torch.Generator().manual_seed(B))[:B].int().cuda()
    slots[2::3] = torch.tensor([-1, pool, -7, 1 << 30], dtype=torch.int32, device="cuda").repeat(B)[:slots[2::3].numel()]
    used = (slots >= 0) & (slots < pool)
    before = s.clone()
    at = slots[used].long()
    want = ref.rule(q, k, v, g, beta, torch.where(used[:, None, None, None], before[slots.clamp(0, pool - 1).long()], 0.0), key_heads=Hk)
    # (token by token the state is rounded at every one: six more roundings of its size and of what is written than the reference counts)
    more = 8 * 2.0 ** -24 * float(before.abs().max() * (T + 2) + v.float().abs().max() * T) * 2
    for t in range(T):
        o = block.delta_step(*(x[..., t].contiguous() for x in (q, k, v, g, beta)), s, slots, Hk)
        assert o.dtype == dtype and (o[~used] == 0).all()
        x, e = (w[..., t][used.cpu()] for w in want["o"])
        ref.check(o[used], (x, e + more * math.sqrt(DK) * DK ** -0.5), ("o", t))
    x, e = (w[used.cpu()] for w in want["s_last"])
    ref.check(s[at], (x, e + more), "s")
    rest = torch.ones(pool, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(s[rest], before[rest])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,H,Hk,DK,DV", [(280, 2, 1, 20, 64), (280, 2, 1, 20, 65), (140, 4, 2, 64, 96), (260, 2, 2, 30, 97), (130, 4, 4, 9, 129), (90, 4, 4, 40, 190)])
def test_tokens_of_many_heads(B, H, Hk, DK, DV, dtype):
    """So many that the columns of a head go to as few workgroups as they fit."""
    test_a_token_is_the_rule(B, H, Hk, DK, DV, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_layouts(dtype):
    q, k, v, g, beta, _, _, _ = inputs(4, 4, 2, 20, 24, 1, dtype)
    flat = [x[..., 0].contiguous() for x in (q, k, v, g, beta)]
    s = rand(4, 4, 20, 24, seed=9)
    want_s = s.clone()
    want = block.delta_step(*flat, want_s, key_heads=2)
    for kind in ("slice", "odd"):
        got_s, o = strided(s, "odd") if kind == "odd" else s.clone(), strided(torch.empty_like(flat[2]), kind)
        assert block.delta_step(*(strided(x, kind) for x in flat), got_s, key_heads=2, out=o) is o
        assert torch.equal(o, want) and torch.equal(got_s, want_s)


def test_token_gates():
    """A decay of minus infinity forgets the state (that holds anything finite), a strength of 0 writes nothing."""
    q, k, v, g, beta, _, _, _ = inputs(2, 2, 2, 32, 32, 1, F32)
    q, k, v, g, beta = (x[..., 0].contiguous() for x in (q, k, v, g, beta))
    s = rand(2, 2, 32, 32, seed=1)
    a, b = s.clone(), torch.zeros_like(s)
    inf = torch.full_like(g, -float("inf"))
    assert torch.equal(block.delta_step(q, k, v, inf, beta, a), block.delta_step(q, k, v, g, beta, b)) and torch.equal(a, b)
    c = s.clone()
    block.delta_step(q, k, v, torch.zeros_like(g), torch.zeros_like(beta), c)
    assert torch.equal(c, s)


def test_token_pools_above_32_bits():
    pool, H, DK, DV = 2100, 64, 128, 128
    assert pool * H * DK * DV > 1 << 31
    s = torch.zeros(pool, H, DK, DV, device="cuda")
    q, k, v, g, beta, s0, _, _ = inputs(2, H, H, DK, DV, 1, F32)
    a = [x[..., 0].contiguous() for x in (q, k, v, g, beta)]
    slots = torch.tensor([2099, 5], dtype=torch.int32, device="cuda")
    s[2099], s[5] = s0[0], s0[1]
    o = block.delta_step(*a, s, slots)
    want = s0.clone()
    assert torch.equal(o, block.delta_step(*a, want)) and torch.equal(s[2099], want[0]) and torch.equal(s[5], want[1]) and not s[6:2099].any()


# ---- dropout ----

def check_dropout(x, p, seed, step, layer, res=None, scale=1.0, tied=False, out=None, res_kept=None):
    B, C, L = x.shape
    rng = torch.tensor([seed, step], device="cuda")
    want_kept = ref.keeps(seed & (1 << 64) - 1, step, layer, B, C if tied else C * L, p).view(B, C, -1).expand(B, C, L)
    y = block.dropout_fwd(x, p, rng, layer, res, scale, tied, out)
    f = scale / (1 - float(torch.tensor(p, dtype=torch.float32)))
    r = torch.zeros(B, C, L, dtype=torch.float64) if res is None else (res if res_kept is None else res_kept).double().cpu()
    want = torch.where(want_kept, x.double().cpu() * f, 0.0) + r
    # the factor's rounding, the product and sum in one, and the rounding to the storage type
    bound = 2.0 ** -24 * ((want - r).abs() * 1.01 + want.abs()) + want.abs() * (1 + 2.0 ** -20) * ref.ROUND[x.dtype] + 1e-40
    assert ((y.double().cpu() - want).abs() <= bound).all()
    assert torch.equal((y == 0).cpu() | want_kept, torch.ones(B, C, L, dtype=torch.bool)) or res is not None
    dx = block.dropout_bwd(x, p, rng, layer, scale, tied)
    plain = block.dropout_fwd(x, p, rng, layer, None, scale, tied)
    assert torch.equal(dx, plain)
    return y


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("B,C,L", [(1, 1, 1), (3, 5, 7), (2, 3, 8), (2, 4, 100), (1, 2, 2600), (50, 3, 1), (7, 9, 3), (1, 300, 2), (2, 17, 129), (300, 2, 5)])
def test_dropout(B, C, L, tied, dtype):
    x, res = rand(B, C, L, seed=1, dtype=dtype), rand(B, C, L, seed=2, dtype=dtype)
    x[x == 0] = 1
    check_dropout(x, 0.3, 12345 + (7 << 40), 99, 3, tied=tied)
    check_dropout(x, 0.5, -1, (1 << 40) + 5, (1 << 24) - 1, res, 0.5, tied)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -32, 0.01, 0.25, 2.0 ** -16, 0.999, 1 - 2.0 ** -24])
def test_dropout_rates(p):
    x = rand(2, 40, 50, seed=3)
    x[x == 0] = 1
    y = check_dropout(x, p, 5, 6, 0)
    if p == 0:
        assert torch.equal(x, y)


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("kind", ["slice", "odd"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dropout_layouts(kind, dtype, tied):
    x, res = rand(3, 6, 45, seed=1, dtype=dtype), rand(3, 6, 45, seed=2, dtype=dtype)
    rng = torch.tensor([3, 4], device="cuda")
    want = block.dropout_fwd(x, 0.4, rng, 1, res, 0.7, tied)
    out = strided(torch.empty_like(x), kind)
    got = block.dropout_fwd(strided(x, kind), 0.4, rng, 1, strided(res, kind), 0.7, tied, out)
    assert got is out and torch.equal(got, want)
    # in place, on either
    a, b = x.clone(), res.clone()
    assert torch.equal(block.dropout_fwd(a, 0.4, rng, 1, res, 0.7, tied, a), want) and torch.equal(block.dropout_fwd(x, 0.4, rng, 1, b, 0.7, tied, b), want)
    # a residual that the batch shares
    one = res[:1].expand_as(res)
    assert torch.equal(block.dropout_fwd(x, 0.4, rng, 1, one, 0.7, tied), block.dropout_fwd(x, 0.4, rng, 1, one.contiguous(), 0.7, tied))


def test_dropped_values_do_not_enter():
    x = rand(2, 30, 40, seed=1)
    rng = torch.tensor([3, 4], device="cuda")
    kept = block.dropout_fwd(torch.ones_like(x), 0.5, rng) != 0
    bad = torch.where(kept, x, torch.tensor([float("nan"), float("inf")], device="cuda").repeat(20))
    res = rand(2, 30, 40, seed=2)
    assert torch.equal(block.dropout_fwd(bad, 0.5, rng, 0, res), block.dropout_fwd(x, 0.5, rng, 0, res))
    assert torch.isfinite(block.dropout_bwd(bad, 0.5, rng)).all()
    x[0, 0, 0] = float("nan")
    rng2 = torch.tensor([0, 0], device="cuda")
    y = block.dropout_fwd(x, 0.0, rng2)
    assert torch.isnan(y[0, 0, 0]) and int(torch.isnan(y).sum()) == 1


def test_dropout_is_as_often_as_said_and_its_own():
    """Shares of the dropped within five standard deviations, over steps, layers, entries and seeds that do not agree with each other."""
    x = torch.ones(4, 64, 1000, device="cuda")
    masks = []
    for seed, step, layer in ((1, 0, 0), (2, 0, 0), (1, 1, 0), (1, 0, 1), (1 << 32, 0, 0), (1, 0, 2)):
        m = block.dropout_fwd(x, 0.2, torch.tensor([seed, step], device="cuda"), layer) == 0
        for b in range(4):
            n = m[b].numel()
            assert abs(float(m[b].double().mean()) - 0.2) < 5 * math.sqrt(0.16 / n)
            masks.append(m[b])
    for i in range(len(masks)):
        for j in range(i):
            both = float((masks[i] & masks[j]).double().mean())
            assert abs(both - 0.04) < 6 * math.sqrt(0.04 * 0.96 / masks[i].numel()), (i, j)


def test_dropout_of_more_than_2_to_the_35():
    """An entry so long that a block's number has more than 32 bits: its end, in place."""
    n = (1 << 35) + 4096 + 5
    C, L = 1 << 6, n // (1 << 6) + 1
    x = torch.ones(1, C, L, dtype=BF16, device="cuda")
    seed, step = 77, 3
    block.dropout_fwd(x, 0.5, torch.tensor([seed, step], device="cuda"), 9, out=x)
    flat = x.view(-1)
    for j in [*range(0, 40), *range((1 << 35) - 9, (1 << 35) + 40), *range(C * L - 20, C * L)]:
        assert float(flat[j]) == (2.0 if ref.bits(seed, step, 9, 0, j) >= 1 << 31 else 0.0), j


@pytest.mark.parametrize("B,C,L", [(70000, 1, 3), (66000, 3, 400), (1 << 21, 1, 1)])
def test_dropout_of_many_entries(B, C, L):
    x = torch.ones(B, C, L, device="cuda")
    y = block.dropout_fwd(x, 0.5, torch.tensor([4, 5], device="cuda"), 6)
    for b in (0, 1, 255, 65534, 65535, 65536, B - 1):
        for j in {0, 1, C * L // 2, C * L - 1} & set(range(C * L)):
            assert float(y[b].view(-1)[j]) == (2.0 if ref.bits(4, 5, 6, b, j) >= 1 << 31 else 0.0), (b, j)


def test_refusals():
    q, k, v, g, beta, s0, do, ds = inputs(2, 2, 1, 8, 12, 20, F32)
    o, s, states = block.delta_fwd(q, k, v, g, beta, key_heads=1)
    rng = torch.tensor([1, 2], device="cuda")
    tok = [t[..., 0].contiguous() for t in (q, k, v, g, beta)]
    value, kind, status = (
        lambda: block.delta_fwd(q, k[:, :4], v, g, beta, key_heads=1), lambda: block.delta_fwd(q, k, v.transpose(1, 2), g, beta, key_heads=1),
        lambda: block.delta_fwd(q[..., ::2], k[..., ::2], v[..., ::2], g[..., ::2], beta[..., ::2], key_heads=1), lambda: block.delta_fwd(q, k, v, g, beta[:, :1], key_heads=1),
        lambda: block.delta_fwd(q, k, v, g, beta, s0[:1], key_heads=1), lambda: block.delta_fwd(q, k, v, g, beta, s0.transpose(2, 3), key_heads=1), lambda: block.delta_fwd(q, k.cpu(), v, g, beta, key_heads=1),
        lambda: block.delta_fwd(q, k, v, g, beta, key_heads=1, out=v[:1].expand_as(v)), lambda: block.delta_fwd(q, k, v, g, beta, lengths=torch.ones(3, device="cuda", dtype=torch.int32), key_heads=1),
        lambda: block.delta_bwd(do, q, k, v, g, beta, states[:, :, :0], key_heads=1), lambda: block.delta_bwd(do, q, k, v, g, beta, states, key_heads=1, out=(q, k)),
        lambda: block.delta_bwd(do[:, :8], q, k, v, g, beta, states, key_heads=1), lambda: block.delta_step(*tok, s[0], key_heads=1), lambda: block.delta_step(*tok, s[:, :1], key_heads=1),
        lambda: block.dropout_fwd(v[0], 0.1, rng), lambda: block.dropout_fwd(v, 0.1, rng[:1]), lambda: block.dropout_fwd(v, 0.1, rng, res=v[:, :3]), lambda: block.dropout_fwd(v, 0.1, rng, out=v[:1].expand_as(v)),
    ), (
        lambda: block.delta_fwd(q, k.bfloat16(), v, g, beta, key_heads=1), lambda: block.delta_fwd(q.bfloat16(), k.bfloat16(), v.bfloat16(), g.bfloat16(), beta, key_heads=1),
        lambda: block.delta_fwd(q.half(), k.half(), v.half(), g, beta, key_heads=1), lambda: block.delta_fwd(q, k, v, g, beta, s0.bfloat16(), key_heads=1),
        lambda: block.delta_fwd(q, k, v, g, beta, lengths=torch.ones(2, device="cuda", dtype=torch.int64), key_heads=1), lambda: block.delta_step(*tok, s.double(), key_heads=1),
        lambda: block.dropout_fwd(v.half(), 0.1, rng), lambda: block.dropout_fwd(v, 0.1, rng.int()), lambda: block.dropout_fwd(v, 0.1, rng, res=v.bfloat16()),
    ), (
        lambda: block.delta_fwd(q, k, v, g, beta, key_heads=1, eps=-1.0), lambda: block.delta_fwd(q, k, v, g, beta, key_heads=1, scale=float("nan")), lambda: block.delta_fwd(q, k, v, g, beta, key_heads=1, workspace=torch.empty(4, device="cuda")),
        lambda: block.delta_step(*tok, s[:1].contiguous(), key_heads=1), lambda: block.delta_bwd(do, q, k, v, g, beta, states, key_heads=1, workspace=torch.empty(4, device="cuda")),
        lambda: block.delta_fwd(*(torch.zeros(1, 129, 4, device="cuda") for _ in range(3)), g[:1, :1, :4], beta[:1, :1, :4]),
        lambda: block.dropout_fwd(v, 1.0, rng), lambda: block.dropout_fwd(v, -0.1, rng), lambda: block.dropout_fwd(v, 0.1, rng, layer=-1), lambda: block.dropout_fwd(v, 0.1, rng, layer=1 << 24),
        lambda: block.dropout_fwd(v, 0.1, rng, scale=float("inf")),
    )
    for calls, error in ((value, ValueError), (kind, TypeError), (status, binding.DwconvError)):
        for n, call in enumerate(calls):
            with pytest.raises(error):
                call()
                pytest.fail(f"{error} {n}")


# ---- runs of them together, and the native form of the calls ----

def test_a_block_trained_and_served():
    """Convolution, delta rule, norm with gate and residual and dropout as a block has them: gradients of the whole against autograd in 64 bits through
    the definitions, and the same sequence token by token (without dropout) against the prompt pass."""
    B, H, D, L, K = 2, 2, 16, 100, 4
    C = H * D
    x, z, w = rand(B, 3 * C, L, seed=1), rand(B, C, L, seed=2), rand(3 * C, K, seed=3) / 2
    g, beta = -0.2 * rand(B, H, L, seed=4).abs(), torch.sigmoid(rand(B, H, L, seed=5))
    res, wn, wn2, dn = rand(B, C, L, seed=6), 1 + 0.1 * rand(C, seed=7), 1 + 0.1 * rand(C, seed=8), rand(B, C, L, seed=9)
    rng, p = torch.tensor([5, 1], device="cuda"), 0.2

    def forward(drop):
        u = binding.dwconv_fwd(x, w, K - 1)
        q, k, v = u.split(C, 1)
        o, s_last, states = block.delta_fwd(q, k, v, g, beta)
        y = block.dropout_fwd(o, p, rng, 3) if drop else o
        out, n, stats = block.norm_fwd(y, z, res, wn, wn2)
        return u, o, s_last, states, y, out, n, stats
    u, o, s_last, states, y, out, n, stats = forward(True)
    dy, dz, dres, dwn, dwn2 = block.norm_bwd(None, dn, y, z, res, wn, wn2, stats)
    do = block.dropout_bwd(dy, p, rng, 3)
    q, k, v = u.split(C, 1)
    du = torch.empty_like(u)
    _, _, _, dg, dbeta, _ = block.delta_bwd(do, q, k, v, g, beta, states, out=tuple(du.split(C, 1)))
    dx, dw = binding.dwconv_bwd(du, x, w, K - 1)

    a = [t.double().cpu().requires_grad_() for t in (x, w, g, beta, z, res, wn, wn2)]
    ux = torch.nn.functional.conv1d(torch.nn.functional.pad(a[0], (K - 1, 0)), a[1][:, None], groups=3 * C)
    oo, _ = ref.one_by_one(*ux.split(C, 1), a[2], a[3])
    kept = ref.keeps(5, 1, 3, B, C * L, p).view(B, C, L)
    yy = torch.where(kept, oo / (1 - p), 0.0)
    hat = yy / torch.sqrt(yy.square().mean(1, keepdim=True) + 1e-6)
    ow = a[5] + torch.nn.functional.silu(a[4]) * hat * a[6][:, None]
    nn = ow / torch.sqrt(ow.square().mean(1, keepdim=True) + 1e-6) * a[7][:, None]
    want = torch.autograd.grad((nn * dn.double().cpu()).sum(), a)
    # every stage keeps 32 bits: a few hundred roundings of 2^-24 of the largest value that a sum of these sizes has
    for name, got, exact in (("n", n, nn.detach()), *zip(("dx", "dw", "dg", "dbeta", "dz", "dres", "dw1", "dw2"), (dx, dw, dg, dbeta, dz, dres, dwn, dwn2), want)):
        assert float((got.double().cpu() - exact).abs().max()) <= 400 * 2.0 ** -24 * float(exact.abs().max()) * math.sqrt(exact.shape[-1]), name

    u, o, s_last, _, _, _, n, _ = forward(False)
    pool, ring, pos = torch.zeros(B, H, D, D, device="cuda"), torch.zeros(B, 3 * C, K, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    for t in range(L):
        q, k, v = block.conv_step(x[..., t].contiguous(), w, ring, pos).split(C, 1)
        y = block.delta_step(q, k, v, g[..., t].contiguous(), beta[..., t].contiguous(), pool)
        _, one, _ = block.norm_fwd(y[..., None], z[..., t:t + 1].contiguous(), res[..., t:t + 1].contiguous(), wn, wn2, save=False)
        pos += 1
        assert float((one[..., 0] - n[..., t]).abs().max()) <= 400 * 2.0 ** -24 * float(n.abs().max()) * math.sqrt(L), t
    assert float((pool - s_last).abs().max()) <= 400 * 2.0 ** -24 * float(s_last.abs().max()) * math.sqrt(L)


def _calls():
    q, k, v, g, beta, s0, do, ds = inputs(2, 4, 2, 8, 12, 70, BF16, seed=40)
    lengths, slots = torch.tensor([70, 9], dtype=torch.int32, device="cuda"), torch.tensor([1, -1], dtype=torch.int32, device="cuda")
    states = block.delta_fwd(q, k, v, g, beta, s0, lengths, 2)[2]
    tok, s = [t[..., 0].contiguous() for t in (q, k, v, g, beta)], rand(3, 4, 8, 12, seed=3)
    x, res, rng = rand(2, 5, 30, seed=4), rand(2, 5, 30, seed=5), torch.tensor([3, 9], device="cuda")
    new = lambda *t: tuple(torch.full_like(a, float("nan")) for a in t)        # noqa: E731
    space = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    wide = torch.cat([q, k, v], 1)
    return {
        # (states behind a sequence's end are not written)
        "fwd": lambda: block.delta_fwd(q, k, v, g, beta, s0, lengths, 2)[:2], "fwd full": lambda: block.delta_fwd(q, k, v, g, beta, s0, None, 2), "fwd bare": lambda: block.delta_fwd(q, k, v, g, beta, key_heads=2, save=False)[:2],
        "fwd out": lambda: block.delta_fwd(*wide.split((16, 16, 48), 1), g, beta, key_heads=2, scale=0.5, eps=0.0, out=new(v)[0], workspace=space),
        "bwd": lambda: block.delta_bwd(do, q, k, v, g, beta, states, ds, lengths, 2), "bwd out": lambda: block.delta_bwd(do, q, k, v, g, beta, states, None, lengths, 2, out=new(q, k, v), workspace=space),
        "step": lambda: (block.delta_step(*tok, a := s.clone(), slots, 2), a), "step out": lambda: (block.delta_step(*tok, a := s.clone(), key_heads=2, scale=2.0, out=new(tok[2])[0]), a),
        "drop": lambda: (block.dropout_fwd(x, 0.3, rng), block.dropout_bwd(x, 0.3, rng, 5, 0.5, True)), "drop res": lambda: (block.dropout_fwd(x, 0.3, rng, 2, res, 0.5, False, new(x)[0]),),
    }


def test_native_calls_give_the_same(monkeypatch):
    native = {name: call() for name, call in _calls().items()}
    monkeypatch.setattr(block, "_fast", block._Declines)
    for name, call in _calls().items():
        for a, b in zip(native[name], call()):
            assert (a is None and b is None) or torch.equal(a, b), name


def test_native_calls_take_what_they_should(monkeypatch):
    """Plain calls do not come back to Python."""
    block.lib()
    if block._fast is block._Declines:
        pytest.skip("without the native calls")

    def no(*args):
        raise AssertionError("declined")
    calls = _calls()
    monkeypatch.setattr(block, "_seq", no)
    for name, call in calls.items():
        call()


@pytest.mark.parametrize("native", [True, False])
def test_an_empty_workspace_is_too_small(native, monkeypatch):
    q, k, v, g, beta, s0, do, ds = inputs(2, 2, 2, 8, 12, 70, F32)
    states = block.delta_fwd(q, k, v, g, beta)[2]
    if not native:
        monkeypatch.setattr(block, "_fast", block._Declines)
    empty = torch.empty(0, dtype=torch.uint8, device="cuda")
    for call in (lambda: block.delta_fwd(q, k, v, g, beta, workspace=empty), lambda: block.delta_bwd(do, q, k, v, g, beta, states, workspace=empty)):
        with pytest.raises(binding.DwconvError):
            call()


def _example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "delta_block.py")
    spec = importlib.util.spec_from_file_location("delta_block", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


def test_the_example_runs_and_serves():
    """What it says token by token is what it says of the whole sequence.  (Logits of a model of this width pass some thousand 32-bit operations in
    another order: 2^-14 of the largest.)"""
    losses, off, size = _example().main(steps=5)
    assert all(math.isfinite(x) for x in losses)
    assert off <= 2.0 ** -14 * size


def test_the_example_s_gradients():
    """A whole model's gradient along a direction against the difference of its loss, the same mask in both."""
    example = _example()
    model = example.Model(32, 4, 2, 12, 4, 2, seed=3, p=0.2)
    tokens = example.batch(32, 8, 70, seed=1)

    def loss():
        return torch.nn.functional.cross_entropy(model.logits(tokens[:, :-1], train=True).double(), tokens[:, 1:])
    params = model.parameters()
    grads = torch.autograd.grad(loss(), params)
    for p, g in zip(params, grads):
        d = rand(*p.shape, seed=7) * 1e-2 * (1 + p.detach().abs().mean())

        def over(step):
            with torch.no_grad():
                p.add_(d, alpha=step)
                up = float(loss())
                p.add_(d, alpha=-2 * step)
                down = float(loss())
                p.add_(d, alpha=step)
            return up - down
        want = 2 * float((g.double() * d.double()).sum())
        # A difference over a step h is 2 h f' + h^3 f3 / 3 + O(h^5), f3 the third derivative: 8 of those over h / 2 less one over h is 6 h f' without it
        # (a direction of thousands of elements is about as long as the parameter's own rows are, where h^2 f3 is some hundredths of f').  Roundings
        # of a 32-bit forward pass in a mean of 560 losses: 1e-6 of about 4, in 8 + 1 differences of two, over 3.
        assert abs((8 * over(0.5) - over(1.0)) / 3 - want) <= 2e-2 * abs(want) + 6e-5, tuple(p.shape)

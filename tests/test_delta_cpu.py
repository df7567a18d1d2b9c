"""CPU checks of the gated delta rule and of dropout: the ABI and its refusals, what the binding turns away, and the references that the GPU
tests compare with, against the definition, autograd and differences."""
import pytest
import torch

import _delta_ref as ref

P = 0x1000          # any non-NULL, aligned, never-dereferenced address


@pytest.fixture(scope="module")
def lib():
    from paper_2604_25422_amd import _build, block
    if _build.is_stale():
        _build.build()
    return block.lib()


def S(p=P, stride=1 << 20):
    from paper_2604_25422_amd import block
    return block.Seq(p, stride)


DIMS = dict(B=2, H=4, Hk=2, DK=8, DV=16, L=100)
BAD_DIMS = [dict(B=0), dict(H=0), dict(Hk=0), dict(Hk=3), dict(DK=0), dict(DK=129), dict(DV=0), dict(DV=65537), dict(L=0), dict(L=(1 << 30) + 1),
            dict(B=1 << 20, H=1 << 12), dict(H=(1 << 20) + 1, Hk=1), dict(H=1 << 20, Hk=1, DV=64), dict(B=1 << 15, H=1 << 10, Hk=1, L=1 << 13)]


def fwd(lib, k=None, v=None, ws=P, n=1 << 40, scale=1.0, eps=1e-6, dtype=0, **dims):
    a = dict(q=S(), k=S(), v=S(), g=S(), beta=S(), s0=None, lengths=None, o=S(), s_last=P, states=P)
    if k:
        a[k] = v
    return lib.dwconv_delta_fwd(*a.values(), ws, n, *{**DIMS, **dims}.values(), scale, eps, dtype, None)


def test_forward_refusals(lib):
    for k in ("q", "k", "v", "o"):
        assert fwd(lib, k, S(None)) == 1 and fwd(lib, k, S(P + 2)) == 6 and fwd(lib, k, S(P + 1), dtype=1) == 6
        assert fwd(lib, k, S(P, -1)) == 9 and fwd(lib, k, S(P, (1 << 40) + 1)) == 9
    for k in ("g", "beta"):             # (fp32 in calls of either type)
        assert fwd(lib, k, S(None)) == 1 and fwd(lib, k, S(P + 2), dtype=1) == 6 and fwd(lib, k, S(P, -1)) == 9
    for k in ("s0", "lengths", "s_last", "states"):
        assert fwd(lib, k, P + 2) == 6
    assert fwd(lib, "o", S(P, 4 * 16 * 100 - 1)) == 9
    for bad in BAD_DIMS:
        assert fwd(lib, **bad) == 2, bad
    assert fwd(lib, dtype=2) == 4 and fwd(lib, dtype=-1) == 4
    for x in (float("nan"), float("inf")):
        assert fwd(lib, scale=x) == 9 and fwd(lib, eps=x) == 9
    assert fwd(lib, eps=-1e-6) == 9
    need = lib.dwconv_delta_workspace_bytes(2, 4, 2, 8, 16, 100, 0)
    assert fwd(lib, ws=None) == 5 and fwd(lib, n=need - 1) == 5 and fwd(lib, ws=P + 8) == 5


def test_backward_refusals(lib):
    need = lib.dwconv_delta_workspace_bytes(2, 4, 2, 8, 16, 100, 1)
    # the states' gradients behind two chunks of every head, those of 64 positions' u, and what each of the heads that share a key adds to its gradients
    assert need == lib.dwconv_delta_workspace_bytes(2, 4, 2, 8, 16, 100, 0) + 2 * 4 * 2 * 16 * (8 + 64) * 4 + 2 * 4 * 2 * 8 * 100 * 4
    assert lib.dwconv_delta_workspace_bytes(2, 4, 4, 8, 16, 100, 1) == need - 2 * 4 * 2 * 8 * 100 * 4

    def f(k=None, v=None, ws=P, n=1 << 40, scale=1.0, eps=1e-6, dtype=0, **dims):
        a = dict(do=S(), q=S(), k=S(), v=S(), g=S(), beta=S(), states=P, ds_last=None, lengths=None, dq=S(), dk=S(), dv=S(), dg=P, dbeta=P, ds0=P)
        if k:
            a[k] = v
        return lib.dwconv_delta_bwd(*a.values(), ws, n, *{**DIMS, **dims}.values(), scale, eps, dtype, None)
    for k in ("do", "q", "k", "v", "dq", "dk", "dv"):
        assert f(k, S(None)) == 1 and f(k, S(P + 2)) == 6 and f(k, S(P, -1)) == 9
    for k in ("states", "dg", "dbeta"):
        assert f(k, None) == 1 and f(k, P + 2) == 6
    for k in ("ds_last", "lengths", "ds0"):
        assert f(k, P + 2) == 6
    assert f("dq", S(P, 2 * 8 * 100 - 1)) == 9 and f("dk", S(P, 2 * 8 * 100 - 1)) == 9 and f("dv", S(P, 4 * 16 * 100 - 1)) == 9
    for bad in BAD_DIMS:
        assert f(**bad) == 2, bad
    assert f(dtype=3) == 4 and f(scale=float("nan")) == 9 and f(eps=-1.0) == 9
    assert f(ws=None) == 5 and f(n=need - 1) == 5 and f(ws=P + 8) == 5


def test_states_and_workspaces(lib):
    assert [lib.dwconv_delta_states(L) for L in (0, -1, 1, 64, 65, 1 << 30, (1 << 30) + 1)] == [0, 0, 1, 1, 2, 1 << 24, 0]
    for bad in ((0, 1, 1, 1, 1, 1), (1, 0, 1, 1, 1, 1), (1, 2, 0, 1, 1, 1), (1, 3, 2, 1, 1, 1), (1, 1, 1, 0, 1, 1), (1, 1, 1, 129, 1, 1), (1, 1, 1, 1, 0, 1), (1, 1, 1, 1, 1, 0)):
        assert lib.dwconv_delta_workspace_bytes(*bad, 0) == 0 and lib.dwconv_delta_workspace_bytes(*bad, 1) == 0
    a, b = (lib.dwconv_delta_workspace_bytes(1, 1, 1, 1, 1, 64, x) for x in (0, 1))
    assert a > 0 and a % 16 == 0 and b == a + 16 + 64 * 4 and lib.dwconv_delta_workspace_bytes(3, 5, 5, 1, 1, 65, 0) == 30 * a
    # (rows of fewer than eight positions are copied to where they have room for that)
    assert lib.dwconv_delta_workspace_bytes(1, 1, 1, 1, 1, 7, 0) > a == lib.dwconv_delta_workspace_bytes(1, 1, 1, 1, 1, 8, 0)


def test_step_refusals(lib):
    def f(k=None, v=None, pool=4, scale=1.0, eps=1e-6, dtype=0, **dims):
        a = dict(q=S(), k=S(), v=S(), g=S(), beta=S(), s=P, slots=None)
        o, d = S(), {**DIMS, **dims}
        d.pop("L")
        if k == "o":
            o = v
        elif k:
            a[k] = v
        return lib.dwconv_delta_step(*a.values(), pool, o, *d.values(), scale, eps, dtype, None)
    for k in ("q", "k", "v", "g", "beta", "o"):
        assert f(k, S(None)) == 1 and f(k, S(P + 2)) == 6 and f(k, S(P, -1)) == 9
    assert f("s", None) == 1 and f("s", P + 2) == 6 and f("slots", P + 2) == 6 and f("o", S(P, 63)) == 9
    assert f(pool=1) == 2 and f("slots", P, pool=0) == 2 and f(dtype=2) == 4 and f(scale=float("inf")) == 9 and f(eps=float("nan")) == 9
    for bad in BAD_DIMS:
        if "L" not in bad:
            assert f(pool=1 << 30, **bad) == 2, bad
    assert f(B=1 << 20, H=1024, Hk=1, DK=1, DV=128, pool=1 << 20) == 2      # more workgroups than a grid has


def test_dropout_refusals(lib):
    def f(x=None, res=None, out=None, rng=P, layer=0, B=2, C=3, L=10, p=0.1, scale=1.0, tied=0, dtype=0):
        return lib.dwconv_dropout(x or S(), res or S(None, 0), out or S(), rng, layer, B, C, L, p, scale, tied, dtype, None)
    assert f(x=S(None)) == 1 and f(out=S(None)) == 1 and f(rng=None) == 1
    assert f(x=S(P + 2)) == 6 and f(res=S(P + 2)) == 6 and f(out=S(P + 1), dtype=1) == 6 and f(rng=P + 4) == 6
    assert f(x=S(P, -1)) == 9 and f(out=S(P, 29)) == 9 and f(B=0) == 2 and f(C=0) == 2 and f(L=0) == 2 and f(dtype=2) == 4
    for p in (-0.1, 1.0, 1.5, float("nan")):
        assert f(p=p) == 9
    assert f(scale=float("inf")) == 9 and f(scale=float("nan")) == 9 and f(layer=-1) == 9 and f(layer=1 << 24) == 9


def test_binding_refuses_what_it_cannot_take():
    from paper_2604_25422_amd import block
    q, v, g, s = torch.zeros(2, 4, 8), torch.zeros(2, 6, 8), torch.zeros(2, 2, 8), torch.zeros(2, 2, 2, 3)
    rng = torch.zeros(2, dtype=torch.int64)
    for call in (lambda: block.delta_fwd(q, q, v, g, g), lambda: block.delta_bwd(v, q, q, v, g, g, torch.zeros(2, 2, 1, 2, 3)),
                 lambda: block.delta_step(q[..., 0], q[..., 0], v[..., 0], g[..., 0], g[..., 0], s), lambda: block.dropout_fwd(q, 0.1, rng),
                 lambda: block.dropout_bwd(q, 0.1, rng)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    for call in (lambda: block.delta_fwd(q, q, v, g, g, key_heads=3), lambda: block.delta_fwd(q, q, v, g, g, key_heads=0), lambda: block.delta_fwd(q[:, :3], q, v, g, g),
                 lambda: block.delta_fwd(q, q, v[:, :5], g, g), lambda: block.delta_fwd(q[0], q, v, g, g), lambda: block.delta_fwd(q, q, v, g[:, :0], g),
                 lambda: block.delta_fwd(q[:, :0], q, v, g, g), lambda: block.delta_bwd(v, q, q, v, g, g, s, out=(q, q)), lambda: block.delta_step(q, q, v, g, g, s)):
        with pytest.raises(ValueError):
            call()


# ---- the references ----

def seeded(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("eps", [1e-6, 0.0])
@pytest.mark.parametrize("H,Hk,lengths", [(2, 2, None), (4, 2, [150, 0, 70])])
def test_reference_against_the_definition_and_autograd(H, Hk, lengths, eps):
    B, DK, DV, L = 3, 5, 7, 150
    q, k, v, do = (seeded(B, n, L, seed=i) for i, n in enumerate((Hk * DK, Hk * DK, H * DV, H * DV)))
    if not eps:
        k = k / 3
    g, beta = -0.3 * seeded(B, H, L, seed=5).abs(), torch.sigmoid(seeded(B, H, L, seed=6))
    s0, ds = seeded(B, H, DK, DV, seed=7), seeded(B, H, DK, DV, seed=8)
    ends = None if lengths is None else torch.tensor(lengths)
    args = [t.requires_grad_() for t in (q, k, v, g, beta, s0)]
    o, s = ref.one_by_one(*args, ends, Hk, eps=eps)
    grads = torch.autograd.grad((o * do).sum() + (s * ds).sum(), args)
    got = ref.rule(*(t.detach() for t in args), ends, Hk, eps=eps, do=do, ds_last=ds)
    for name, want in zip(("o", "s_last", "dq", "dk", "dv", "dg", "dbeta", "ds0"), (o, s, *grads)):
        x, e = got[name]
        # both in 64 bits: 2^-29 of what 32 bits may be off, and the roundings of a few thousand operations
        assert ((x - want).abs() <= e * 2.0 ** -29 * 64 + 1e-11 * (1 + want.abs().max())).all(), name
        assert (e <= 1e-2 * (1 + want.abs().max())).all(), (name, "a bound that says nothing")


def test_reference_against_differences():
    B, H, DK, DV, L = 2, 2, 3, 4, 70
    q, k, v, do = (seeded(B, n, L, seed=i) for i, n in enumerate((H * DK, H * DK, H * DV, H * DV)))
    args = {"q": q, "k": k, "v": v, "g": -0.2 * seeded(B, H, L, seed=5).abs() - 0.01, "beta": torch.sigmoid(seeded(B, H, L, seed=6)),
            "s0": seeded(B, H, DK, DV, seed=7)}
    ds = seeded(B, H, DK, DV, seed=8)

    def loss(a):
        r = ref.rule(**a)
        return float((r["o"][0] * do).sum() + (r["s_last"][0] * ds).sum())
    got = ref.rule(**args, do=do, ds_last=ds)
    for name, t in args.items():
        d, h = seeded(*t.shape, seed=20), 1e-5
        num = (loss({**args, name: t + h * d}) - loss({**args, name: t - h * d})) / (2 * h)
        # central differences: the third derivative of a function of order 100 times h^2, and the roundings of 64 bits over h
        assert abs(num - float((got["d" + name][0] * d).sum())) < 1e-6 * (1 + abs(num)), name


def test_generator_against_known_answers():
    """Those that the generator's authors publish."""
    assert ref.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert ref.philox((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert ref.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_native_calls_decline_what_is_not_a_device_tensor(lib):
    from paper_2604_25422_amd import _fastcall, block
    assert block._fast is _fastcall
    x, g, n = torch.zeros(2, 4, 8), torch.zeros(2, 2, 8), None
    for call in (lambda: _fastcall.delta_fwd(x, x, x, g, g, n, n, n, n, 1e-6, True, n, n), lambda: _fastcall.delta_fwd(x), lambda: _fastcall.delta_fwd(*[n] * 13),
                 lambda: _fastcall.delta_bwd(x, x, x, x, g, g, x, n, n, n, n, 1e-6, n, n, n, n), lambda: _fastcall.delta_bwd(*[n] * 16),
                 lambda: _fastcall.delta_step(x, x, x, g, g, x, n, n, n, 1e-6, n), lambda: _fastcall.delta_step(*[n] * 11),
                 lambda: _fastcall.dropout(x, 0.1, x, 0, n, 1.0, False, n), lambda: _fastcall.dropout(*[n] * 8)):
        assert call() is None


def test_few_heads_are_cut_into_segments(lib):
    """By what the workspace has room for beside a record a chunk: few heads with many chunks are, many heads are not."""
    record = lib.dwconv_delta_workspace_bytes(1, 1, 1, 16, 16, 64, 0)
    for heads, L, cut in ((1, 64, False), (1, 65, False), (2, 1024, True), (4, 65537, True), (32, 4096, True), (768, 1024, False), (4096, 256, False)):
        more = lib.dwconv_delta_workspace_bytes(1, heads, heads, 128, 128, L, 0) - record * heads * -(-L // 64)
        assert (more > 0) == cut and (not cut or more >= 4 * heads * 2 * 128 * 384), (heads, L)

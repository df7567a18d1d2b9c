"""CPU checks of the block operators: the ABI and its refusals (validation comes before any HIP call), what the binding turns away,
and the references that the GPU tests compare with, against differences."""
import os
import re

import pytest
import torch

import _block_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


def test_every_declared_symbol_is_exported(lib):
    from paper_2604_25422_amd import block
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dwconv_block.h")).read(), flags=re.S)
    syms = set(re.findall(r"\b(dwconv_[a-z_0-9]+)\s*\(", text))
    assert syms == set(block.SYMBOLS)
    assert all(hasattr(lib, s) for s in syms)
    assert lib.dwconv_status_string(9) != lib.dwconv_status_string(99)


def scan_fwd(lib, x=None, r=None, i=None, lam=P, h0=None, lengths=None, y=None, h_last=P, states=P, ws=P, nbytes=1 << 30, B=2, C=3, L=100,
             rate=8.0, dtype=0):
    return lib.dwconv_scan_fwd(x or S(), r or S(), i or S(), lam, h0, lengths, y or S(), h_last, states, ws, nbytes, B, C, L, rate, dtype, None)


def test_scan_refusals(lib):
    f = scan_fwd
    for k in ("x", "r", "i", "y"):
        assert f(lib, **{k: S(None)}) == 1
        assert f(lib, **{k: S(P + 2)}) == 6 and f(lib, dtype=1, **{k: S(P + 1)}) == 6
        assert f(lib, **{k: S(P, -1)}) == 9 and f(lib, **{k: S(P, (1 << 40) + 1)}) == 9
    assert f(lib, lam=None) == 1 and f(lib, lam=P + 2) == 6 and f(lib, h0=P + 1) == 6 and f(lib, lengths=P + 2) == 6
    assert f(lib, states=P + 2) == 6 and f(lib, h_last=P + 3) == 6
    assert f(lib, y=S(P, 299)) == 9                      # batch entries of an output overlap (C L = 300)
    for bad in (dict(B=0), dict(C=0), dict(L=0), dict(C=(1 << 25) + 1), dict(L=(1 << 30) + 1), dict(B=1 << 20, C=1 << 12), dict(B=1 << 10, C=1 << 11, L=1 << 20)):
        assert f(lib, **bad) == 2, bad
    assert f(lib, dtype=2) == 4 and f(lib, dtype=-1) == 4
    for rate in (0.0, -1.0, float("inf"), float("nan")):
        assert f(lib, rate=rate) == 9
    # few long rows: segments, whose spans need a workspace
    need = lib.dwconv_scan_workspace_bytes(1, 1, 1 << 20, 0)
    assert need > 0 and need % 16 == 0
    for ws, n in ((None, need), (P, need - 1), (P + 8, need)):
        assert f(lib, B=1, C=1, L=1 << 20, ws=ws, nbytes=n) == 5


def test_scan_backward_refusals(lib):
    need = lib.dwconv_scan_workspace_bytes(2, 3, 100, 1)
    assert need >= 4 * 2 * 3

    def f(k=None, v=None, B=2, C=3, L=100, rate=8.0, dtype=0, ws=P, n=need):
        a = dict(dy=S(), x=S(), r=S(), i=S(), lam=P, states=P, dh=None, lengths=None, dx=S(), dr=S(), di=S(), dlam=P, dh0=None)
        if k:
            a[k] = v
        return lib.dwconv_scan_bwd(*a.values(), ws, n, B, C, L, rate, dtype, None)
    for k in ("dy", "x", "r", "i", "dx", "dr", "di"):
        assert f(k, S(None)) == 1 and f(k, S(P + 2)) == 6 and f(k, S(P, -5)) == 9
    for k in ("lam", "states", "dlam"):
        assert f(k, None) == 1 and f(k, P + 2) == 6
    for k in ("dh", "lengths", "dh0"):
        assert f(k, P + 2) == 6
    for k in ("dx", "dr", "di"):
        assert f(k, S(P, 10)) == 9
    assert f(L=0) == 2 and f(dtype=7) == 4 and f(rate=0.0) == 9
    assert f(ws=None) == 5 and f(n=need - 1) == 5 and f(ws=P + 4) == 5


def test_states_and_workspaces(lib):
    assert [lib.dwconv_scan_states(L) for L in (0, -1, 1, 512, 513, 1 << 30, (1 << 30) + 1)] == [0, 0, 1, 1, 2, 1 << 21, 0]
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0)):
        assert lib.dwconv_scan_workspace_bytes(*bad, 1) == 0 and lib.dwconv_norm_workspace_bytes(*bad, 0) == 0
    assert lib.dwconv_norm_workspace_bytes(1, 1, 1, 2) == 0 and lib.dwconv_norm_workspace_bytes(2, 700, 1, 1) >= 2 * 4 * 700
    assert lib.dwconv_clip_workspace_bytes() % 16 == 0


def test_step_refusals(lib):
    def f(k=None, v=None, pool=4, B=2, C=3, rate=8.0, dtype=0):
        a = dict(x=S(), r=S(), i=S(), lam=P, h=P, slots=None)
        y = S()
        if k == "y":
            y = v
        elif k:
            a[k] = v
        return lib.dwconv_scan_step(*a.values(), pool, y, B, C, rate, dtype, None)
    for k in ("x", "r", "i", "y"):
        assert f(k, S(None)) == 1 and f(k, S(P + 2)) == 6 and f(k, S(P, -1)) == 9
    assert f("lam", None) == 1 and f("h", None) == 1 and f("h", P + 2) == 6 and f("slots", P + 2) == 6
    assert f(pool=1) == 2 and f("slots", P, pool=0) == 2 and f(B=0) == 2 and f(dtype=3) == 4 and f(rate=-1.0) == 9

    def g(x=None, w=P, ring=P, pos=P, slots=None, pool=4, y=None, B=2, C=3, K=5, dtype=0):
        return lib.dwconv_conv_step(x or S(), w, ring, pos, slots, pool, y or S(), B, C, K, dtype, None)
    assert g(x=S(None)) == 1 and g(w=None) == 1 and g(ring=None) == 1 and g(pos=None) == 1 and g(y=S(None)) == 1
    assert g(K=0) == 2 and g(pool=1) == 2 and g(C=0) == 2 and g(dtype=2) == 4 and g(w=P + 2) == 6 and g(ring=P + 1) == 6 and g(pos=P + 2) == 6
    assert g(x=S(P, -1)) == 9 and g(y=S(P, 2)) == 9

    def r(x=None, ring=P, lengths=None, slots=None, pool=4, B=2, C=3, L=10, K=5, dtype=0):
        return lib.dwconv_conv_ring(x or S(), ring, lengths, slots, pool, B, C, L, K, dtype, None)
    assert r(x=S(None)) == 1 and r(ring=None) == 1 and r(L=0) == 2 and r(K=0) == 2 and r(pool=1) == 2 and r(dtype=5) == 4 and r(ring=P + 2) == 6


def test_norm_refusals(lib):
    def f(k=None, v=None, B=2, C=3, L=10, eps=1e-6, scale=1.0, dtype=0):
        a = dict(y=S(), z=S(), res=S(), w=P, wn=P, out=S(), n=S(), stats=P)
        if k:
            a[k] = v
        return lib.dwconv_norm_fwd(*a.values(), B, C, L, eps, scale, dtype, None)
    for k in ("y", "z", "res", "out", "n"):
        assert f(k, S(None)) == 1 and f(k, S(P + 2)) == 6 and f(k, S(P, -1)) == 9
    assert f("w", None) == 1 and f("wn", None) == 1 and f("w", P + 2) == 6 and f("stats", P + 1) == 6 and f("n", S(P, 29)) == 9
    assert f(L=0) == 2 and f(dtype=2) == 4
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert f(eps=eps) == 9
    assert f(scale=float("inf")) == 9 and f(scale=float("nan")) == 9
    need = lib.dwconv_norm_workspace_bytes(2, 3, 10, 0)

    def g(k=None, v=None, ws=P, n=need, L=10, scale=1.0, dtype=0):
        a = dict(dout=S(), dn=S(), y=S(), z=S(), res=S(), w=P, wn=P, stats=P, dy=S(), dz=S(), dres=S(), dw=P, dwn=P)
        if k:
            a[k] = v
        return lib.dwconv_norm_bwd(*a.values(), ws, n, 2, 3, L, scale, dtype, None)
    for k in ("dn", "y", "z", "res", "dy", "dz", "dres"):
        assert g(k, S(None)) == 1 and g(k, S(P + 2)) == 6 and g(k, S(P, -1)) == 9
    for k in ("w", "wn", "stats", "dw", "dwn"):
        assert g(k, None) == 1 and g(k, P + 2) == 6
    assert g("dout", S(P + 2)) == 6 and g(L=0) == 2 and g(dtype=2) == 4 and g(scale=float("nan")) == 9
    assert g(ws=None) == 5 and g(n=need - 1) == 5 and g(ws=P + 8) == 5


def test_clip_refusals(lib):
    import ctypes
    V, I, Q = ctypes.c_void_p * 2, ctypes.c_int * 2, ctypes.c_longlong * 2
    n = lib.dwconv_clip_workspace_bytes()

    def f(i=(P, P), o=(P, P), sizes=(5, 6), dt=(0, 1), count=2, max_norm=1.0, norm=P, ws=P, nb=n):
        return lib.dwconv_clip_grad_norm(V(*i), V(*o), Q(*sizes), I(*dt), count, max_norm, norm, ws, nb, None)
    assert lib.dwconv_clip_grad_norm(None, V(P, P), Q(1, 1), I(0, 0), 2, 1.0, P, P, n, None) == 1
    assert f(i=(P, None)) == 1 and f(o=(None, P)) == 1 and f(norm=None) == 1
    assert f(count=0) == 2 and f(sizes=(5, -1)) == 2 and f(dt=(0, 2)) == 4 and f(i=(P + 2, P)) == 6 and f(o=(P, P + 1)) == 6 and f(norm=P + 2) == 6
    for m in (0.0, -1.0, float("inf"), float("nan")):
        assert f(max_norm=m) == 9
    assert f(ws=None) == 5 and f(nb=n - 1) == 5 and f(ws=P + 8) == 5


def test_binding_refuses_what_it_cannot_take():
    from paper_2604_25422_amd import block
    x, c = torch.zeros(2, 3, 8), torch.zeros(3)
    for call in (lambda: block.scan_fwd(x, x, x, c), lambda: block.scan_bwd(x, x, x, x, c, torch.zeros(2, 3, 1)),
                 lambda: block.scan_step(x[..., 0], x[..., 0], x[..., 0], c, torch.zeros(2, 3)), lambda: block.norm_fwd(x, x, x, c, c),
                 lambda: block.norm_bwd(None, x, x, x, x, c, c, torch.zeros(2, 2, 8)), lambda: block.clip_grad_norm([x], 1.0),
                 lambda: block.conv_step(x[..., 0], torch.zeros(3, 4), torch.zeros(2, 3, 4), torch.zeros(2, dtype=torch.int32)),
                 lambda: block.conv_ring(x, torch.zeros(2, 3, 4))):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    with pytest.raises(ValueError, match="nothing to clip"):
        block.clip_grad_norm([], 1.0)


def _seeded(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def test_reference_of_the_scan_against_differences():
    B, C, L = 2, 3, 11
    x, r, i, dy = (_seeded(B, C, L, seed=k) for k in range(4))
    lam, h0, dh = _seeded(C, seed=5) - 3, _seeded(B, C, seed=6), _seeded(B, C, seed=7)
    lengths = torch.tensor([11, 4])
    args = {"x": x, "r": r, "i": i, "lam": lam, "h0": h0}

    def loss(a):
        o, _ = ref.scan(**a, lengths=lengths)
        return float((o["y"] * dy).sum() + (o["h_last"] * dh).sum())
    out, _ = ref.scan(**args, lengths=lengths, dy=dy, dh_last=dh)
    for name, t in args.items():
        d = _seeded(*t.shape, seed=20)
        eps = 1e-5
        num = (loss({**args, name: t + eps * d}) - loss({**args, name: t - eps * d})) / (2 * eps)
        # central differences: the third derivative of a function of order 10 and the roundings of 64 bits over eps
        assert abs(num - float((out["d" + name] * d).sum())) < 1e-7 * (1 + abs(num)), name


def test_reference_of_the_norm_against_differences():
    B, C, L = 2, 5, 3
    y, z, res, dout, dn = (_seeded(B, C, L, seed=k) for k in range(5))
    w, wn = 1 + 0.3 * _seeded(C, seed=8), 1 + 0.3 * _seeded(C, seed=9)
    args = {"y": y, "z": z, "res": res, "w": w, "w_next": wn}

    def loss(a):
        o, _ = ref.norm(**a, eps=1e-3, scale=0.7)
        return float((o["out"] * dout).sum() + (o["n"] * dn).sum())
    out, _ = ref.norm(**args, eps=1e-3, scale=0.7, dout=dout, dn=dn)
    for name, t in args.items():
        d = _seeded(*t.shape, seed=20)
        eps = 1e-5
        num = (loss({**args, name: t + eps * d}) - loss({**args, name: t - eps * d})) / (2 * eps)
        assert abs(num - float((out["d" + name] * d).sum())) < 1e-7 * (1 + abs(num)), name


def test_native_calls_decline_what_is_not_a_device_tensor(lib):
    from paper_2604_25422_amd import _fastcall, block
    assert block._fast is _fastcall
    x, c = torch.zeros(2, 3, 8), torch.zeros(3)
    for call in (lambda: _fastcall.scan_fwd(x, x, x, c, None, None, 8.0, True, None, None), lambda: _fastcall.scan_fwd(x), lambda: _fastcall.scan_step(x, x, x, c, x, None, 8.0, None),
                 lambda: _fastcall.scan_bwd(x, x, x, x, c, x, None, None, 8.0, None, None, None, None), lambda: _fastcall.norm_fwd(x, x, x, c, c, 1e-6, 1.0, True, None, None),
                 lambda: _fastcall.norm_fwd(None, x, x, c, c, 1e-6, 1.0, True, None, None), lambda: _fastcall.norm_bwd(x, x, x, x, x, c, c, x, 1.0, None, None, None, None),
                 lambda: _fastcall.clip_grad_norm([x], 1.0, None, None), lambda: _fastcall.clip_grad_norm([], 1.0, None, None), lambda: _fastcall.clip_grad_norm([None], 1.0, [x], None),
                 lambda: _fastcall.conv_step(x, x, x, None, None, None), lambda: _fastcall.conv_step(None, None, None, None, None, None)):
        assert call() is None


def test_norm_workspace_of_many_tiles_is_bounded(lib):
    # (a row of sums for every tile only while a grid has all tiles)
    for B, L in ((1 << 30, 5), (1 << 22, 4), (1 << 22, 64)):
        assert 0 < lib.dwconv_norm_workspace_bytes(B, 1, L, 0) <= 1100 * 2 * 4
    assert lib.dwconv_norm_workspace_bytes((1 << 22) - 1, 1, 4, 0) >= 2 * 4 * ((1 << 22) - 1)


def test_few_long_rows_are_cut_where_that_takes_less(lib):
    """By what the workspace has room for: the spans of segments, 8 bytes each.  (Of 65537 positions cut rows take less up to some 115
    rows forward and 175 backward in bf16, fewer in fp32, whose workspace is the same.)"""
    whole = lambda rows: 4 * rows                               # noqa: E731  (a sum a row towards dlam)
    for rows in (1, 64, 104):
        assert lib.dwconv_scan_workspace_bytes(1, rows, 65537, 0) >= 8 * rows * 32
    for rows in (120, 127, 128, 300):
        assert lib.dwconv_scan_workspace_bytes(1, rows, 65537, 0) == 0
    for rows in (1, 64, 128, 144, 160):
        assert lib.dwconv_scan_workspace_bytes(1, rows, 65537, 1) >= 8 * rows * 32
    for rows in (192, 256, 320):
        assert lib.dwconv_scan_workspace_bytes(1, rows, 65537, 1) == whole(rows)
    for rows, L in ((112, 20000), (128, 20000), (1, 16384), (1, 512)):
        assert lib.dwconv_scan_workspace_bytes(1, rows, L, 1) == (whole(rows) + 15) // 16 * 16

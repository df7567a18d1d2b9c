"""The operators around the depthwise convolution in a sequence block, for torch device tensors: thin binding of the C ABI in
``include/dwconv_block.h`` (argument marshalling only, as ``binding`` is for the convolution itself).

``scan_fwd`` / ``scan_bwd`` / ``scan_step``: a gated linear recurrence along t.  ``delta_fwd`` / ``delta_bwd`` / ``delta_step``: the gated
delta rule, whose state is a matrix for every head.  ``norm_fwd`` / ``norm_bwd``: the norms before and after a block with its gate and residual.
``dropout_fwd`` / ``dropout_bwd``: dropout from a counter-based generator.  ``clip_grad_norm``: the global gradient norm and clipping.  ``conv_step`` /
``conv_ring``: the causal convolution for one token.

Sequences are [B, C, L] tensors whose positions are next to each other and whose channels lie L elements apart; the batch stride is
free, so slices of the channels of a wider tensor (``projected.chunk(3, dim=1)``) go in as they are, and out into.  Everything is
enqueued on the current stream and nothing synchronises; a missing library raises, there is no other path.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .binding import _DTYPE_CODES, _check, _dtype_code, _on_current_device, _stream

SYMBOLS = (
    "dwconv_scan_fwd", "dwconv_scan_bwd", "dwconv_scan_states", "dwconv_scan_workspace_bytes", "dwconv_scan_step",
    "dwconv_norm_fwd", "dwconv_norm_bwd", "dwconv_norm_workspace_bytes",
    "dwconv_clip_grad_norm", "dwconv_clip_workspace_bytes", "dwconv_conv_step", "dwconv_conv_ring",
    "dwconv_delta_fwd", "dwconv_delta_bwd", "dwconv_delta_states", "dwconv_delta_workspace_bytes", "dwconv_delta_step", "dwconv_dropout",
)


class Seq(ctypes.Structure):
    """struct dwconv_seq / dwconv_seq_out."""
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_longlong)]


_NONE = Seq(None, 0)
_lib = None


class _Declines:
    """In the place of the native calls until the library is loaded, and where they cannot be (see ``binding``)."""
    scan_fwd = scan_bwd = scan_step = norm_fwd = norm_bwd = clip_grad_norm = conv_step = staticmethod(lambda *args: None)
    delta_fwd = delta_bwd = delta_step = dropout = scan_fwd


_fast = _Declines
_FAST_ADDRESSES = ("dwconv_scan_fwd", "dwconv_scan_bwd", "dwconv_scan_states", "dwconv_scan_workspace_bytes", "dwconv_scan_step", "dwconv_norm_fwd",
                   "dwconv_norm_bwd", "dwconv_norm_workspace_bytes", "dwconv_clip_grad_norm", "dwconv_clip_workspace_bytes", "dwconv_conv_step")
_FAST_DELTA_ADDRESSES = ("dwconv_delta_fwd", "dwconv_delta_bwd", "dwconv_delta_states", "dwconv_delta_workspace_bytes", "dwconv_delta_step", "dwconv_dropout")


def lib():
    """The shared library, with the signatures of the block operators."""
    global _lib, _fast
    if _lib is None:
        l = binding.lib()
        vp, i, f, sz, s = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, Seq
        for name, args, res in (
                ("dwconv_scan_fwd", [s, s, s, vp, vp, vp, s, vp, vp, vp, sz, i, i, i, f, i, vp], i),
                ("dwconv_scan_bwd", [s, s, s, s, vp, vp, vp, vp, s, s, s, vp, vp, vp, sz, i, i, i, f, i, vp], i),
                ("dwconv_scan_states", [i], i),
                ("dwconv_scan_workspace_bytes", [i, i, i, i], sz),
                ("dwconv_scan_step", [s, s, s, vp, vp, vp, i, s, i, i, f, i, vp], i),
                ("dwconv_norm_fwd", [s, s, s, vp, vp, s, s, vp, i, i, i, f, f, i, vp], i),
                ("dwconv_norm_bwd", [s, s, s, s, s, vp, vp, vp, s, s, s, vp, vp, vp, sz, i, i, i, f, i, vp], i),
                ("dwconv_norm_workspace_bytes", [i, i, i, i], sz),
                ("dwconv_clip_grad_norm", [vp, vp, vp, vp, i, f, vp, vp, sz, vp], i),
                ("dwconv_clip_workspace_bytes", [], sz),
                ("dwconv_conv_step", [s, vp, vp, vp, vp, i, s, i, i, i, i, vp], i),
                ("dwconv_conv_ring", [s, vp, vp, vp, i, i, i, i, i, i, vp], i),
                ("dwconv_delta_fwd", [s, s, s, s, s, vp, vp, s, vp, vp, vp, sz, i, i, i, i, i, i, f, f, i, vp], i),
                ("dwconv_delta_bwd", [s, s, s, s, s, s, vp, vp, vp, s, s, s, vp, vp, vp, vp, sz, i, i, i, i, i, i, f, f, i, vp], i),
                ("dwconv_delta_states", [i], i),
                ("dwconv_delta_workspace_bytes", [i, i, i, i, i, i, i], sz),
                ("dwconv_delta_step", [s, s, s, s, s, vp, vp, i, s, i, i, i, i, i, f, f, i, vp], i),
                ("dwconv_dropout", [s, s, s, vp, i, i, i, i, f, f, i, i, vp], i)):
            fn = getattr(l, name)
            fn.argtypes, fn.restype = args, res
        if binding._fast is not binding._Declines:
            binding._fast.setup_block(*(ctypes.cast(getattr(l, n), vp).value for n in _FAST_ADDRESSES))
            binding._fast.setup_delta(*(ctypes.cast(getattr(l, n), vp).value for n in _FAST_DELTA_ADDRESSES))
            _fast = binding._fast
        _lib = l
    return _lib


# ---- what a tensor has to be ----

def _seq(t: torch.Tensor, name: str, shape, dtype, written: bool = False) -> Seq:
    """A [B, C, L] (or [B, C]) tensor with free batch stride."""
    _on_current_device(t, name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, is {list(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, is {t.dtype}")
    B, C, L = shape if len(shape) == 3 else (*shape, 1)
    st = t.stride() if len(shape) == 3 else (*t.stride(), 1)
    if (L > 1 and st[2] != 1) or (C > 1 and st[1] != L):
        raise ValueError(f"{name} must have its positions next to each other and its channels {L} elements apart (strides {tuple(t.stride())})")
    if written and B > 1 and st[0] < C * L:
        raise ValueError(f"{name} is written: its batch entries must not overlap")
    return Seq(t.data_ptr(), st[0] if B > 1 else C * L)


def _f32(t, name: str, shape, optional: bool = False):
    if t is None and optional:
        return None
    return _plain(t, name, shape, torch.float32)


def _plain(t, name: str, shape, dtype):
    _on_current_device(t, name)
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, is {t.dtype}")
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of shape {list(shape)}")
    return t.data_ptr()


def _index(t, name: str, B: int):
    return None if t is None else _plain(t, name, (B,), torch.int32)


def _shape3(x, name: str):
    if x.dim() != 3:
        raise ValueError(f"{name} must be a [B, C, L] tensor")
    return tuple(x.shape)


def _shape2(x, name: str):
    if x.dim() != 2:
        raise ValueError(f"{name} must be a [B, C] tensor")
    return tuple(x.shape)


def _out(t, name: str, shape, like):
    if t is None:
        t = torch.empty(shape, dtype=like.dtype, device=like.device)
    return t, _seq(t, name, shape, like.dtype, written=True)


def _workspace(t, need: int, like):
    if t is None:
        if need == 0:
            return None, 0, None
        t = torch.empty(need, dtype=torch.uint8, device=like.device)
    _on_current_device(t, "workspace")
    if not t.is_contiguous():
        raise ValueError("workspace must be a contiguous GPU tensor")
    return t.data_ptr(), t.numel() * t.element_size(), t


# ---- gated scan ----

def scan_states(L: int) -> int:
    """States of a row that ``scan_fwd`` keeps for ``scan_bwd``: one for every 512 positions."""
    return int(lib().dwconv_scan_states(int(L)))


def scan_workspace_bytes(B: int, C: int, L: int, backward: bool) -> int:
    return int(lib().dwconv_scan_workspace_bytes(B, C, L, int(backward)))


def scan_fwd(x, r, i, lam, h0=None, lengths=None, rate: float = 8.0, save: bool = True, out=None, workspace=None):
    """h[t] = a[t] h[t-1] + sqrt(1 - a[t]^2) sigmoid(i[t]) x[t] with a = exp(-rate softplus(lam) sigmoid(r)), along t of [B, C, L]
    tensors x, r, i of one type; lam [C], h0 [B, C] (None: zeros) fp32, lengths [B] int32 (None: L; y is 0 behind a sequence's end).
    Returns (y, h_last, states): y like x, h_last [B, C] fp32, states what ``scan_bwd`` takes (None without ``save``)."""
    done = _fast.scan_fwd(x, r, i, lam, h0, lengths, rate, save, out, workspace)
    if done is not None:
        return done
    shape = B, C, L = _shape3(x, "x")
    code = _dtype_code(x)
    xs, rs, is_ = _seq(x, "x", shape, x.dtype), _seq(r, "r", shape, x.dtype), _seq(i, "i", shape, x.dtype)
    lamp, h0p, lp = _f32(lam, "lam", (C,)), _f32(h0, "h0", (B, C), True), _index(lengths, "lengths", B)
    y, ys = _out(out, "out", shape, x)
    h_last = torch.empty((B, C), dtype=torch.float32, device=x.device)
    states = torch.empty((B, C, scan_states(L)), dtype=torch.float32, device=x.device) if save else None
    ws, nbytes, keep = _workspace(workspace, scan_workspace_bytes(B, C, L, False), x)
    _check(lib().dwconv_scan_fwd(xs, rs, is_, lamp, h0p, lp, ys, h_last.data_ptr(), states.data_ptr() if save else None, ws, nbytes,
                                 B, C, L, float(rate), code, _stream()))
    return y, h_last, states


def scan_bwd(dy, x, r, i, lam, states, dh_last=None, lengths=None, rate: float = 8.0, out=None, workspace=None):
    """Gradients of ``scan_fwd`` from dy [B, C, L] and dh_last [B, C] fp32 (None: zeros): returns (dx, dr, di, dlam, dh0), the
    first three like x (or into the three tensors of ``out``), dlam [C] and dh0 [B, C] fp32."""
    given = out if out is not None else (None,) * 3
    if len(given) != 3:
        raise ValueError("out must be three tensors (dx, dr, di)")
    done = _fast.scan_bwd(dy, x, r, i, lam, states, dh_last, lengths, rate, *given, workspace)
    if done is not None:
        return done
    shape = B, C, L = _shape3(x, "x")
    code = _dtype_code(x)
    ins = [_seq(t, n, shape, x.dtype) for t, n in ((dy, "dy"), (x, "x"), (r, "r"), (i, "i"))]
    lamp, lp = _f32(lam, "lam", (C,)), _index(lengths, "lengths", B)
    sp, dhp = _f32(states, "states", (B, C, scan_states(L))), _f32(dh_last, "dh_last", (B, C), True)
    outs = [_out(t, n, shape, x) for t, n in zip(given, ("dx", "dr", "di"))]
    dlam = torch.empty((C,), dtype=torch.float32, device=x.device)
    dh0 = torch.empty((B, C), dtype=torch.float32, device=x.device)
    ws, nbytes, keep = _workspace(workspace, scan_workspace_bytes(B, C, L, True), x)
    _check(lib().dwconv_scan_bwd(*ins, lamp, sp, dhp, lp, *(s for _, s in outs), dlam.data_ptr(), dh0.data_ptr(), ws, nbytes,
                                 B, C, L, float(rate), code, _stream()))
    return outs[0][0], outs[1][0], outs[2][0], dlam, dh0


def scan_step(x, r, i, lam, h, slots=None, rate: float = 8.0, out=None):
    """One token of the gated scan for a batch: x, r, i [B, C]; h [pool, C] fp32 is updated in place, place b of the batch in row
    slots[b] (int32; outside [0, pool): an empty place, y is 0 there) or, without slots, in row b.  Returns y like x."""
    done = _fast.scan_step(x, r, i, lam, h, slots, rate, out)
    if done is not None:
        return done
    shape = B, C = _shape2(x, "x")
    code = _dtype_code(x)
    ins = [_seq(t, n, shape, x.dtype) for t, n in ((x, "x"), (r, "r"), (i, "i"))]
    lamp, sp = _f32(lam, "lam", (C,)), _index(slots, "slots", B)
    hp = _f32(h, "h", (_shape2(h, "h")[0], C))
    y, ys = _out(out, "out", shape, x)
    _check(lib().dwconv_scan_step(*ins, lamp, hp, sp, h.shape[0], ys, B, C, float(rate), code, _stream()))
    return y


# ---- gated delta rule ----

def delta_states(L: int) -> int:
    """States of a head that ``delta_fwd`` keeps for ``delta_bwd``: one for every 64 positions."""
    return int(lib().dwconv_delta_states(int(L)))


def delta_workspace_bytes(B: int, H: int, key_heads: int, DK: int, DV: int, L: int, backward: bool) -> int:
    return int(lib().dwconv_delta_workspace_bytes(B, H, key_heads, DK, DV, L, int(backward)))


def _heads(q, v, g, key_heads, dims: int):
    """(B, H, Hk, DK, DV) of a call: heads of values from the gate's channels, of keys as given."""
    for t, name in ((q, "q"), (v, "v"), (g, "g")):
        if t.dim() != dims:
            raise ValueError(f"{name} must be a {'[B, channels, L]' if dims == 3 else '[B, channels]'} tensor")
    B, H = int(g.shape[0]), int(g.shape[1])
    Hk = H if key_heads is None else int(key_heads)
    if H < 1 or Hk < 1 or H % Hk:
        raise ValueError(f"{H} heads of values do not share {Hk} heads of keys evenly")
    if q.shape[1] % Hk or v.shape[1] % H or q.shape[1] < Hk:
        raise ValueError(f"q has {q.shape[1]} channels for {Hk} heads, v {v.shape[1]} for {H}")
    return B, H, Hk, int(q.shape[1]) // Hk, int(v.shape[1]) // H


def delta_fwd(q, k, v, g, beta, s0=None, lengths=None, key_heads=None, scale=None, eps: float = 1e-6, save: bool = True, out=None, workspace=None):
    """The gated delta rule along t: with a state S [DK, DV] of every head, S <- exp(g) S, u = v - S^T k, S <- S + beta k u^T, o = scale S^T q.
    q, k [B, key_heads * DK, L] and v [B, H * DV, L] of one type, g (log decays) and beta [B, H, L] fp32; H a multiple of key_heads (None: H),
    neighbouring heads of values share one of keys.  scale None: DK^-1/2.  eps: q and k are brought to unit length, x / sqrt(|x|^2 + eps); 0: taken as
    they are.  s0 [B, H, DK, DV] fp32 (None: zeros), lengths [B] int32 (None: L; o is 0 behind a sequence's end).
    Returns (o, s_last, states): o like v, s_last [B, H, DK, DV] fp32, states what ``delta_bwd`` takes (None without ``save``)."""
    done = _fast.delta_fwd(q, k, v, g, beta, s0, lengths, key_heads, scale, eps, save, out, workspace)
    if done is not None:
        return done
    B, H, Hk, DK, DV = _heads(q, v, g, key_heads, 3)
    scale = DK ** -0.5 if scale is None else scale
    L, code, keys, values = int(q.shape[2]), _dtype_code(q), (B, Hk * DK, q.shape[2]), (B, H * DV, q.shape[2])
    ins = [_seq(q, "q", keys, q.dtype), _seq(k, "k", keys, q.dtype), _seq(v, "v", values, q.dtype),
           _seq(g, "g", (B, H, L), torch.float32), _seq(beta, "beta", (B, H, L), torch.float32)]
    sp, lp = _f32(s0, "s0", (B, H, DK, DV), True), _index(lengths, "lengths", B)
    o, os_ = _out(out, "out", values, q)
    s_last = torch.empty((B, H, DK, DV), dtype=torch.float32, device=q.device)
    states = torch.empty((B, H, delta_states(L), DK, DV), dtype=torch.float32, device=q.device) if save else None
    ws, nbytes, keep = _workspace(workspace, delta_workspace_bytes(B, H, Hk, DK, DV, L, False), q)
    _check(lib().dwconv_delta_fwd(*ins, sp, lp, os_, s_last.data_ptr(), states.data_ptr() if save else None, ws, nbytes, B, H, Hk, DK, DV, L,
                                  float(scale), float(eps), code, _stream()))
    return o, s_last, states


def delta_bwd(do, q, k, v, g, beta, states, ds_last=None, lengths=None, key_heads=None, scale=None, eps: float = 1e-6, out=None, workspace=None):
    """Gradients of ``delta_fwd`` from do like v and ds_last [B, H, DK, DV] fp32 (None: zeros): returns (dq, dk, dv, dg, dbeta, ds0), the first
    three like q, k, v (or into the three tensors of ``out``; those of a shared head of keys are summed over its heads), dg and dbeta [B, H, L] and
    ds0 [B, H, DK, DV] fp32."""
    given = out if out is not None else (None,) * 3
    if len(given) != 3:
        raise ValueError("out must be three tensors (dq, dk, dv)")
    done = _fast.delta_bwd(do, q, k, v, g, beta, states, ds_last, lengths, key_heads, scale, eps, *given, workspace)
    if done is not None:
        return done
    B, H, Hk, DK, DV = _heads(q, v, g, key_heads, 3)
    scale = DK ** -0.5 if scale is None else scale
    L, code, keys, values = int(q.shape[2]), _dtype_code(q), (B, Hk * DK, q.shape[2]), (B, H * DV, q.shape[2])
    ins = [_seq(do, "do", values, q.dtype), _seq(q, "q", keys, q.dtype), _seq(k, "k", keys, q.dtype), _seq(v, "v", values, q.dtype),
           _seq(g, "g", (B, H, L), torch.float32), _seq(beta, "beta", (B, H, L), torch.float32)]
    sp = _f32(states, "states", (B, H, delta_states(L), DK, DV))
    dsp, lp = _f32(ds_last, "ds_last", (B, H, DK, DV), True), _index(lengths, "lengths", B)
    outs = [_out(t, n, shape, q) for t, n, shape in zip(given, ("dq", "dk", "dv"), (keys, keys, values))]
    dg, dbeta = (torch.empty((B, H, L), dtype=torch.float32, device=q.device) for _ in range(2))
    ds0 = torch.empty((B, H, DK, DV), dtype=torch.float32, device=q.device)
    ws, nbytes, keep = _workspace(workspace, delta_workspace_bytes(B, H, Hk, DK, DV, L, True), q)
    _check(lib().dwconv_delta_bwd(*ins, sp, dsp, lp, *(s for _, s in outs), dg.data_ptr(), dbeta.data_ptr(), ds0.data_ptr(), ws, nbytes, B, H, Hk, DK, DV,
                                  L, float(scale), float(eps), code, _stream()))
    return outs[0][0], outs[1][0], outs[2][0], dg, dbeta, ds0


def delta_step(q, k, v, g, beta, s, slots=None, key_heads=None, scale=None, eps: float = 1e-6, out=None):
    """One token of the gated delta rule for a batch: q, k [B, key_heads * DK], v [B, H * DV], g and beta [B, H] fp32; s [pool, H, DK, DV] fp32 is
    updated in place, place b of the batch in row slots[b] as in ``scan_step``.  Returns o like v."""
    done = _fast.delta_step(q, k, v, g, beta, s, slots, key_heads, scale, eps, out)
    if done is not None:
        return done
    B, H, Hk, DK, DV = _heads(q, v, g, key_heads, 2)
    scale = DK ** -0.5 if scale is None else scale
    code, keys, values = _dtype_code(q), (B, Hk * DK), (B, H * DV)
    ins = [_seq(q, "q", keys, q.dtype), _seq(k, "k", keys, q.dtype), _seq(v, "v", values, q.dtype), _seq(g, "g", (B, H), torch.float32),
           _seq(beta, "beta", (B, H), torch.float32)]
    if s.dim() != 4:
        raise ValueError("s must be a [pool, H, DK, DV] tensor")
    sp, lp = _f32(s, "s", (s.shape[0], H, DK, DV)), _index(slots, "slots", B)
    o, os_ = _out(out, "out", values, q)
    _check(lib().dwconv_delta_step(*ins, sp, lp, s.shape[0], os_, B, H, Hk, DK, DV, float(scale), float(eps), code, _stream()))
    return o


# ---- dropout ----

def _dropout(x, name, p, rng, layer, res, scale, tied, out):
    done = _fast.dropout(x, p, rng, layer, res, scale, tied, out)
    if done is not None:
        return done
    shape = B, C, L = _shape3(x, name)
    code = _dtype_code(x)
    xs, rs = _seq(x, name, shape, x.dtype), _NONE if res is None else _seq(res, "res", shape, x.dtype)
    rp = _plain(rng, "rng", (2,), torch.int64)
    o, os_ = _out(out, "out", shape, x)
    _check(lib().dwconv_dropout(xs, rs, os_, rp, int(layer), B, C, L, float(p), float(scale), int(bool(tied)), code, _stream()))
    return o


def dropout_fwd(x, p: float, rng, layer: int = 0, res=None, scale: float = 1.0, tied: bool = False, out=None):
    """res + scale x / (1 - p) where an element of x [B, C, L] is kept, res (None: zeros) where it is dropped, with probability p; scale / (1 - p) is
    finite in 32 bits.  ``tied``: whole channels of a batch entry are.  rng [2] int64 on the GPU, a seed and a step, decides together with ``layer``
    (0 .. 2^24 - 1): the same three give the same mask, which is stored nowhere; a program counts the step up (``rng[1] += 1``, also between replays
    of a graph) and gives every layer its number.  out may be x or res itself."""
    return _dropout(x, "x", p, rng, layer, res, scale, tied, out)


def dropout_bwd(dout, p: float, rng, layer: int = 0, scale: float = 1.0, tied: bool = False, out=None):
    """Gradient of ``dropout_fwd`` with regard to x, from the rng that it had; that with regard to res is dout itself."""
    return _dropout(dout, "dout", p, rng, layer, None, scale, tied, out)


# ---- norms, gate, residual ----

def norm_workspace_bytes(B: int, C: int, L: int, dtype: torch.dtype) -> int:
    return int(lib().dwconv_norm_workspace_bytes(B, C, L, _DTYPE_CODES[dtype]))


def norm_fwd(y, z, res, w, w_next, eps: float = 1e-6, scale: float = 1.0, save: bool = True, out=None, out_n=None):
    """out = res + scale silu(z) y / rms(y) w and n = out / rms(out) w_next, rms over the channels of [B, C, L] tensors; w, w_next [C]
    fp32.  y = z = w = None: no block in front, n is the norm of res and out is None.  Returns (out, n, stats), stats what
    ``norm_bwd`` takes (None without ``save``)."""
    done = _fast.norm_fwd(y, z, res, w, w_next, eps, scale, save, out, out_n)
    if done is not None:
        return done
    shape = B, C, L = _shape3(res, "res")
    code = _dtype_code(res)
    rs, wnp = _seq(res, "res", shape, res.dtype), _f32(w_next, "w_next", (C,))
    ys = zs = os_ = _NONE
    wp = o = None
    if y is None and z is None and w is None:
        if out is not None:
            raise ValueError("there is no out without y, z and w")
    else:
        if y is None or z is None or w is None:
            raise ValueError("y, z and w go together")
        ys, zs, wp = _seq(y, "y", shape, res.dtype), _seq(z, "z", shape, res.dtype), _f32(w, "w", (C,))
        o, os_ = _out(out, "out", shape, res)
    n, ns = _out(out_n, "out_n", shape, res)
    stats = torch.empty((B, 2, L), dtype=torch.float32, device=res.device) if save else None
    _check(lib().dwconv_norm_fwd(ys, zs, rs, wp, wnp, os_, ns, stats.data_ptr() if save else None, B, C, L, float(eps), float(scale), code,
                                 _stream()))
    return o, n, stats


def norm_bwd(dout, dn, y, z, res, w, w_next, stats, scale: float = 1.0, out=None, workspace=None):
    """Gradients of ``norm_fwd`` from dout (None: zeros) and dn: returns (dy, dz, dres, dw, dw_next), the first three like res (or
    into the three tensors of ``out``), the last two [C] fp32.  Without a block (y = z = w = None) dy, dz and dw are None."""
    given = out if out is not None else (None,) * 3
    if len(given) != 3:
        raise ValueError("out must be three tensors (dy, dz, dres)")
    done = _fast.norm_bwd(dout, dn, y, z, res, w, w_next, stats, scale, *given, workspace)
    if done is not None:
        return done
    shape = B, C, L = _shape3(res, "res")
    code = _dtype_code(res)
    ds = _NONE if dout is None else _seq(dout, "dout", shape, res.dtype)
    ns, rs = _seq(dn, "dn", shape, res.dtype), _seq(res, "res", shape, res.dtype)
    wnp, sp = _f32(w_next, "w_next", (C,)), _f32(stats, "stats", (B, 2, L))
    ys = zs = dys = dzs = _NONE
    wp = dy = dz = dw = None
    if y is not None or z is not None or w is not None:
        if y is None or z is None or w is None:
            raise ValueError("y, z and w go together")
        ys, zs, wp = _seq(y, "y", shape, res.dtype), _seq(z, "z", shape, res.dtype), _f32(w, "w", (C,))
        (dy, dys), (dz, dzs) = _out(given[0], "dy", shape, res), _out(given[1], "dz", shape, res)
        dw = torch.empty((C,), dtype=torch.float32, device=res.device)
    dres, drs = _out(given[2], "dres", shape, res)
    dw_next = torch.empty((C,), dtype=torch.float32, device=res.device)
    ws, nbytes, keep = _workspace(workspace, norm_workspace_bytes(B, C, L, res.dtype), res)
    _check(lib().dwconv_norm_bwd(ds, ns, ys, zs, rs, wp, wnp, sp, dys, dzs, drs, None if dw is None else dw.data_ptr(), dw_next.data_ptr(),
                                 ws, nbytes, B, C, L, float(scale), code, _stream()))
    return dy, dz, dres, dw, dw_next


# ---- clipping ----

def _dense(t: torch.Tensor) -> bool:
    """Whether a tensor's elements fill one run of memory, in any order of its axes."""
    if t.is_contiguous():
        return True
    n = 1
    for size, stride in sorted(((s, st) for s, st in zip(t.shape, t.stride()) if s > 1), key=lambda p: p[1]):
        if stride != n:
            return False
        n *= size
    return True


def clip_grad_norm(grads, max_norm: float, out=None, workspace=None) -> torch.Tensor:
    """Scales all tensors of ``grads`` (fp32 or bf16, any mixture, dense) by min(1, max_norm / (norm + 1e-6)), norm the 2-norm of
    everything in them: in place, or into the tensors of ``out``, laid out alike.  max_norm is positive and finite (the largest fp32 value:
    the norm alone).  Returns norm, an fp32 scalar on the GPU."""
    done = _fast.clip_grad_norm(grads, max_norm, out, workspace)
    if done is not None:
        return done
    grads = [grads] if isinstance(grads, torch.Tensor) else list(grads)
    outs = grads if out is None else [out] if isinstance(out, torch.Tensor) else list(out)
    n = len(grads)
    if n == 0:
        raise ValueError("there is nothing to clip")
    if len(outs) != n:
        raise ValueError(f"out must hold {n} tensors, holds {len(outs)}")
    ins, to = (ctypes.c_void_p * n)(), (ctypes.c_void_p * n)()
    sizes, codes = (ctypes.c_longlong * n)(), (ctypes.c_int * n)()
    for k, (g, o) in enumerate(zip(grads, outs)):
        _on_current_device(g, f"grads[{k}]")
        if not _dense(g):
            raise ValueError(f"grads[{k}] must be dense (strides {tuple(g.stride())})")
        if o is not g:
            _on_current_device(o, f"out[{k}]")
            if o.dtype != g.dtype or o.shape != g.shape or o.stride() != g.stride():
                raise ValueError(f"out[{k}] must be shaped, laid out and typed like grads[{k}]")
        ins[k], to[k], sizes[k], codes[k] = g.data_ptr(), o.data_ptr(), g.numel(), _dtype_code(g)
    norm = torch.empty((), dtype=torch.float32, device=grads[0].device)
    ws, nbytes, keep = _workspace(workspace, int(lib().dwconv_clip_workspace_bytes()), grads[0])
    _check(lib().dwconv_clip_grad_norm(ins, to, sizes, codes, n, float(max_norm), norm.data_ptr(), ws, nbytes, _stream()))
    return norm


# ---- the convolution, one token ----

def _ring(ring, C: int, dtype):
    if ring.dim() != 3:
        raise ValueError("ring must be a [pool, C, K] tensor")
    return _plain(ring, "ring", (ring.shape[0], C, ring.shape[2]), dtype)


def conv_step(x, w, ring, pos, slots=None, out=None):
    """The causal convolution (``dwconv_fwd`` with pad_left = K - 1) for one token of every sequence of a batch: x [B, C], w [C, K],
    ring [pool, C, K] (the last K inputs, that of position p at p mod K; updated in place), pos [B] int32 (tokens before this one;
    advanced by the caller, once for all layers), slots as in ``scan_step``.  Returns y like x."""
    done = _fast.conv_step(x, w, ring, pos, slots, out)
    if done is not None:
        return done
    shape = B, C = _shape2(x, "x")
    code = _dtype_code(x)
    xs, rp, pp, sp = _seq(x, "x", shape, x.dtype), _ring(ring, C, x.dtype), _index(pos, "pos", B), _index(slots, "slots", B)
    pool, K = ring.shape[0], ring.shape[2]
    wp = _plain(w, "w", (C, K), x.dtype)
    if pp is None:
        raise ValueError("pos must be a [B] tensor")
    y, ys = _out(out, "out", shape, x)
    _check(lib().dwconv_conv_step(xs, wp, rp, pp, sp, pool, ys, B, C, K, code, _stream()))
    return y


def conv_ring(x, ring, lengths=None, slots=None):
    """Fills ring [pool, C, K] from the prompt x [B, C, L] that ``dwconv_fwd`` has read (its first lengths[b] positions): the next
    position is lengths[b], or L.  Returns ring."""
    shape = B, C, L = _shape3(x, "x")
    xs, rp = _seq(x, "x", shape, x.dtype), _ring(ring, C, x.dtype)
    code = _dtype_code(x)
    lp, sp = _index(lengths, "lengths", B), _index(slots, "slots", B)
    _check(lib().dwconv_conv_ring(xs, rp, lp, sp, ring.shape[0], B, C, L, ring.shape[2], code, _stream()))
    return ring

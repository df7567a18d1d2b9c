"""The gated delta rule in 64 bits on the CPU, chunk by chunk, with bounds on what 32-bit arithmetic may be off; dropout's decisions in
whole numbers.

A value comes with a bound on its error, and both go through every operation (a running error analysis to first order): with u = 2^-24, what one
rounding is off by relative to the value, a product of factors off by ea and eb is off by |a| eb + |b| ea + u |ab|, a sum of n products by the
sum of those and n u times the sum of their sizes, in whatever order it is formed.  (Products of three bf16 limbs per operand leave 2^-24 of a
product: 8 u more for a sum's every size covers them.)  Exponentials, roots and reciprocals are within 4 u, the inverse of a triangular matrix is off by
|T| (error of A + 64 u |I + A|) |T|.  From chunk to chunk a bound by sizes alone would grow without end where the state itself does not, so there
the error is held as a 2-norm: a chunk's own, and the one before times the 2-norm of the matrix that takes a state through the chunk."""
import torch

U = 2.0 ** -24
C = 64
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


class N:
    """A value and the bound of its error."""

    def __init__(self, x, e=None):
        self.x, self.e = x, torch.zeros_like(x) if e is None else e

    def __mul__(self, o):
        o = o if isinstance(o, N) else N(o)
        return N(self.x * o.x, self.x.abs() * o.e + o.x.abs() * self.e + U * (self.x * o.x).abs())

    def __add__(self, o):
        return N(self.x + o.x, self.e + o.e + U * (self.x.abs() + o.x.abs()))

    def __neg__(self):
        return N(-self.x, self.e)

    def __sub__(self, o):
        return self + -o

    def __matmul__(self, o):
        n = self.x.shape[-1] + 8
        a, b = self.x.abs(), o.x.abs()
        return N(self.x @ o.x, a @ o.e + self.e @ b + n * U * (a @ b))

    @property
    def T(self):
        return N(self.x.transpose(-1, -2), self.e.transpose(-1, -2))

    def sum(self, dim):
        return N(self.x.sum(dim), self.e.sum(dim) + 64 * U * self.x.abs().sum(dim))

    def where(self, m):
        return N(torch.where(m, self.x, 0.0), torch.where(m, self.e, 0.0))

    def view(self, *s):
        return N(self.x[s], self.e[s])


def _rel(x, k):
    return N(x, k * U * x.abs())


def rule(q, k, v, g, beta, s0=None, lengths=None, key_heads=None, scale=None, eps=1e-6, do=None, ds_last=None):
    """{name: (value, bound)} of o, s_last and with do all gradients."""
    B, H, L = g.shape
    Hk = H if key_heads is None else key_heads
    each, DK, DV = H // Hk, q.shape[1] // Hk, v.shape[1] // H
    scale = DK ** -0.5 if scale is None else scale
    n = -(-L // C)
    ends = torch.full((B,), L) if lengths is None else lengths.cpu().long().clamp(0, L)
    inside = (torch.arange(n * C) < ends[:, None])[:, None, :]

    def cut(x, h):
        x = x.double().cpu()
        x = torch.cat([x, torch.zeros(B, x.shape[1], n * C - L, dtype=torch.float64)], -1)
        x = torch.where(inside, x, 0.0)
        return x.view(B, h, -1, n, C).permute(0, 1, 3, 4, 2)        # [B, h, n, C, D]
    q, k, v = cut(q, Hk), cut(k, Hk), cut(v, H)
    gs, bs = (cut(x, H)[..., 0] for x in (g, beta))
    G = gs.clamp(min=-1e4).cumsum(-1)
    size = lambda x: 1 / torch.sqrt(x.square().sum(-1, keepdim=True) + eps) if eps else torch.ones_like(x[..., :1])      # noqa: E731
    rq, rk = (_rel(size(x), DK + 8) for x in (q, k))
    qh, kh = N(q) * rq, N(k) * rk
    wide = lambda x: N(x.x.repeat_interleave(each, 1), x.e.repeat_interleave(each, 1))           # noqa: E731
    qs, kw = wide(qh * _rel(torch.full_like(rq.x, scale), 1)), wide(kh)
    low = torch.ones(C, C, dtype=torch.bool).tril()
    D = _rel(torch.where(low, torch.exp(torch.where(low, G[..., :, None] - G[..., None, :], 0.0)), 0.0), 4)
    eG, eC = _rel(torch.exp(G), 4), _rel(torch.exp(G[..., -1:] - G), 4)
    eG, eC = N(eG.x[..., None], eG.e[..., None]), N(eC.x[..., None], eC.e[..., None])
    eA = _rel(torch.exp(G[..., -1])[..., None, None], 4)
    b = N(bs[..., None])
    KK = ((kw @ kw.T) * D).where(low.tril(-1))
    P = (qs @ kw.T) * D
    A, eye = b * KK, torch.eye(C, dtype=torch.float64)
    Tx = torch.linalg.solve_triangular(eye + A.x, eye.expand_as(A.x), upper=False, unitriangular=True)
    T = N(Tx, Tx.abs() @ (A.e + 64 * U * (eye + A.x.abs())) @ Tx.abs())
    kin, kout, qin = eG * kw, eC * kw, eG * qs
    bv, bk = b * N(v), b * kin
    reach = Tx @ bk.x                                           # what w takes of S, as [C, DK]
    norm2 = torch.linalg.matrix_norm(eA.x * torch.eye(DK, dtype=torch.float64) - kout.x.transpose(-1, -2) @ reach, 2)      # [B, H, n]
    rows = lambda x: x.square().sum(-1, keepdim=True).sqrt()    # noqa: E731
    S = torch.zeros(B, H, DK, DV, dtype=torch.float64) if s0 is None else s0.double().cpu()
    off = torch.zeros(B, H, 1, 1, dtype=torch.float64)
    S0, off0, w = [], [], []
    for c in range(n):
        at = (slice(None), slice(None), c)
        S0.append(S), off0.append(off)
        here = T.view(*at) @ (bv.view(*at) - bk.view(*at) @ N(S))
        w.append(N(here.x, here.e + rows(reach[at]) * off))
        new = eA.view(*at) * N(S) + kout.view(*at).T @ here
        S, off = new.x, norm2[at][..., None, None] * off + new.e.square().sum((-1, -2), keepdim=True).sqrt()
    S0, off0 = torch.stack(S0, 2), torch.stack(off0, 2)
    w = N(torch.stack([t.x for t in w], 2), torch.stack([t.e for t in w], 2))
    back = lambda t: t.permute(0, 1, 4, 2, 3).reshape(B, -1, n * C)[..., :L]         # noqa: E731
    cutoff = inside[..., :L]

    def out(x):
        return torch.where(cutoff, back(x.x), 0.0), torch.where(cutoff, back(x.e), 0.0)
    o = qin @ N(S0) + P @ N(w.x, w.e - rows(reach) * off0)      # (what comes of S's own error: by its whole way to o)
    got = {"o": out(N(o.x, o.e + rows(qin.x - P.x @ reach) * off0)), "s_last": (S, off.expand_as(S))}
    if do is None:
        return got
    do = N(cut(do, H))
    dw0 = P.T @ do
    dS = torch.zeros_like(S) if ds_last is None else ds_last.double().cpu()
    off = torch.zeros(B, H, 1, 1, dtype=torch.float64)
    after, off1, dR = [None] * n, [None] * n, [None] * n
    way = T.x.transpose(-1, -2) @ kout.x
    for c in range(n - 1, -1, -1):
        at = (slice(None), slice(None), c)
        after[c], off1[c] = dS, off
        here = T.view(*at).T @ (dw0.view(*at) + kout.view(*at) @ N(dS))
        dR[c] = N(here.x, here.e + rows(way[at]) * off)
        new = eA.view(*at) * N(dS) + qin.view(*at).T @ do.view(*at) - bk.view(*at).T @ here
        dS, off = new.x, norm2[at][..., None, None] * off + new.e.square().sum((-1, -2), keepdim=True).sqrt()
    dR = N(torch.stack([t.x for t in dR], 2), torch.stack([t.e for t in dR], 2))
    S0, after = N(S0, off0.expand_as(S0)), torch.stack(after, 2)
    after = N(after, torch.stack(off1, 2).expand_as(after))
    dP, dA = (do @ w.T).where(low), (-(dR @ w.T)).where(low.tril(-1))
    dAb = dA * b
    dq_in, dk_in, dk_out = do @ S0.T, dR @ S0.T, w @ after.T
    dq = eG * dq_in + (dP * D) @ kw
    dk = (dP * D).T @ qs + (dAb * D) @ kw + (dAb * D).T @ kw - b * eG * dk_in + eC * dk_out
    pairs = dP * P + dAb * KK
    e = (qin * dq_in - bk * dk_in).sum(-1)
    f = (kout * dk_out).sum(-1)
    whole = (eA * after * S0).sum((-1, -2))
    strict, upto = low.tril(-1).double(), low.double()
    # rows i >= t: upto^T e; columns j < t: strict f; pairs of a row i >= t and a column j < t
    lin = lambda M, t: N(t.x @ M.T, t.e @ M.T + 64 * U * (t.x.abs() @ M.T))       # noqa: E731
    X = N(pairs.x @ strict.T, pairs.e @ strict.T + 64 * U * (pairs.x.abs() @ strict.T))       # [i, t]: columns below t
    X = N((X.x * upto).sum(-2), (X.e * upto).sum(-2) + 64 * U * (X.x.abs() * upto).sum(-2))
    dg = N(whole.x[..., None], whole.e[..., None]) + lin(upto.T, e) + lin(strict, f) + X
    # by its three sums, as it is formed
    db = (dR * N(v)).sum(-1) - (kin * dk_in).sum(-1) + (dA * KK).sum(-1)
    group = lambda x: N(x.x.view(B, Hk, each, n, C, DK).sum(2), x.e.view(B, Hk, each, n, C, DK).sum(2) + each * U * x.x.abs().view(B, Hk, each, n, C, DK).sum(2))  # noqa: E731
    sc = _rel(torch.full_like(rq.x, scale), 1)
    dq, dk = group(dq) * sc, group(dk)
    along = lambda x, d: (lambda s: x * N(s.x[..., None], s.e[..., None] + DK * U * (x.x * d.x).abs().sum(-1, keepdim=True)))((x * d).sum(-1))      # noqa: E731
    if eps:
        dq, dk = rq * (dq - along(qh, dq)), rk * (dk - along(kh, dk))
    got["dq"], got["dk"], got["dv"] = out(dq), out(dk), out(b * dR)
    flat = lambda x: tuple(torch.where(cutoff, t.reshape(B, H, n * C)[..., :L], 0.0) for t in (x.x, x.e))      # noqa: E731
    got["dg"], got["dbeta"], got["ds0"] = flat(dg), flat(db), (dS, off.expand_as(dS))
    dead = torch.where(cutoff, g.double().cpu(), 0.0) < -104
    got["dg"] = tuple(torch.where(dead, 0.0, t) for t in got["dg"])
    return got


def one_by_one(q, k, v, g, beta, s0=None, lengths=None, key_heads=None, scale=None, eps=1e-6):
    """o and s_last by the definition, position by position, in the inputs' type (for autograd and differences)."""
    B, H, L = g.shape
    Hk = H if key_heads is None else key_heads
    each, DK, DV = H // Hk, q.shape[1] // Hk, v.shape[1] // H
    scale = DK ** -0.5 if scale is None else scale
    heads = lambda x, h: x.reshape(B, h, -1, L)                 # noqa: E731
    q, k, v = heads(q, Hk), heads(k, Hk), heads(v, H)
    if eps:
        q, k = (x / torch.sqrt(x.square().sum(2, keepdim=True) + eps) for x in (q, k))
    q, k = (x.repeat_interleave(each, 1) for x in (q, k))
    S = torch.zeros(B, H, DK, DV, dtype=q.dtype) if s0 is None else s0
    ends = torch.full((B,), L) if lengths is None else lengths.long().clamp(0, L)
    o = []
    for t in range(L):
        kt, on = k[..., t], (t < ends)[:, None, None, None]
        new = torch.exp(g[..., t])[..., None, None] * S
        u = v[..., t] - (new * kt[..., None]).sum(2)
        new = new + (beta[..., t, None] * kt)[..., None] * u[..., None, :]
        S = torch.where(on, new, S)
        o.append(torch.where(on[..., 0], scale * (new * q[..., t][..., None]).sum(2), 0.0))
    return torch.stack(o, -1).reshape(B, H * DV, L), S


def check(got, want, name):
    """Every element within its bound and the rounding to its storage type."""
    x, e = want
    g = got.detach().double().cpu()
    assert g.shape == x.shape, (name, g.shape, x.shape)
    assert torch.isfinite(g).all(), name
    if not g.numel():
        return
    off = (g - x).abs() - (e + (x.abs() + e) * ROUND[got.dtype] + 1e-37)
    at = int(off.argmax())
    assert off.max() <= 0, (name, "at", at, "got", float(g.reshape(-1)[at]), "wanted", float(x.reshape(-1)[at]), "bound", float(e.reshape(-1)[at]))


# ---- dropout ----

def philox(c, k):
    """philox4x32-10 of four counter words and two key words, in whole numbers."""
    c, k = list(c), list(k)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def bits(seed, step, layer, b, j):
    """The 32 bits that decide element j of entry b."""
    m, at, sh = j >> 3, (j & 7) >> 1, 16 * (j & 1)
    key = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF
    hi, lo = (philox((m & 0xFFFFFFFF, b, step & 0xFFFFFFFF, layer << 8 | m >> 32 << 1 | half), key)[at] >> sh & 0xFFFF for half in (0, 1))
    return hi << 16 | lo


def keeps(seed, step, layer, B, n, p):
    """[B, n] decisions."""
    limit = round(float(torch.tensor(p, dtype=torch.float32)) * 2 ** 32)
    out = torch.empty(B, n, dtype=torch.bool)
    for b in range(B):
        for m in range(-(-n // 8)):
            key = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF
            hi, lo = (philox((m & 0xFFFFFFFF, b, step & 0xFFFFFFFF, layer << 8 | m >> 32 << 1 | half), key) for half in (0, 1))
            for k in range(min(8, n - 8 * m)):
                u = (hi[k >> 1] >> 16 * (k & 1) & 0xFFFF) << 16 | lo[k >> 1] >> 16 * (k & 1) & 0xFFFF
                out[b, 8 * m + k] = u >= limit
    return out

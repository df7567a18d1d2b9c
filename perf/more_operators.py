"""The gated delta rule (forward, backward, one token) and dropout from a counter-based generator (forward, backward), as cases that
can be timed.  Sequences are [B, channels, L] with t the stride-1 index; head h of H has the channels from h D to (h + 1) D.

A case is a dict; ``op`` names the operator and ``dtype`` ("f32" or "bf16") the storage type:
  delta       B, H, Hk (heads of queries and keys, which H / Hk heads of values share), DK, DV, L; ``train`` (forward and backward, else
              forward), ``s0`` (initial states are given), ``ragged`` (lengths)
  delta_step  B, H, Hk, DK, DV; ``slots`` (sequences are rows of a larger pool of states, some places of the batch are empty)
  dropout     B, C, L; ``p``, ``scale``, ``res`` (a residual is added), ``tied`` (one decision for all positions of a channel); forward and backward

The rule, of one head and position, with a state S [DK, DV], a log decay g and a write strength beta; q and k of unit length:
  S <- exp(g) S,   u = v - S^T k,   S <- S + beta k u^T,   o = DK^-1/2 S^T q

Dropout decides by 32 bits an element: those of position j = c L + t (tied: j = c) of batch entry b come from philox4x32-10 with the key
(seed low, seed high) and the counter (m low, b, step, layer << 8 | m high << 1 | half), m = j >> 3: the upper 16 bits of element j & 7
are half-word j & 7 of the block with half = 0, the lower ones that of the block with half = 1.  Below round(p 2^32) it is dropped.

``own`` selects what ``run`` calls: elementary torch operations in 32 bits, or ``paper_2604_25422_amd.block``.
"""
import math
import random
import struct

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ELEM = {"f32": 4, "bf16": 2}
EPS = 1e-6              # under the root of a length
CHUNK = 64              # positions that the plain form takes at a time
LAYER = 5


def _delta_case(name, B, H, Hk, DK, DV, L, dtype, train, s0=False, ragged=False):
    return {"name": name, "op": "delta", "B": B, "H": H, "Hk": Hk, "DK": DK, "DV": DV, "L": L, "dtype": dtype, "train": train, "s0": s0,
            "ragged": ragged}


def _step_case(name, B, H, Hk, DK, DV, dtype, slots):
    return {"name": name, "op": "delta_step", "B": B, "H": H, "Hk": Hk, "DK": DK, "DV": DV, "dtype": dtype, "slots": slots}


def _dropout_case(name, B, C, L, dtype, p, scale=1.0, res=False, tied=False):
    return {"name": name, "op": "dropout", "B": B, "C": C, "L": L, "dtype": dtype, "p": p, "scale": scale, "res": res, "tied": tied}


def listed():
    return [
        # a training step of the small configuration (64 channels as two heads): launches and the way to them
        _delta_case("delta_small_f32", 4, 2, 2, 32, 32, 1024, "f32", True),
        # mixed-precision training at a transformer's width, heads of 128
        _delta_case("delta_train_bf16", 128, 6, 6, 128, 128, 1024, "bf16", True),
        # the headline's tensor as four heads, batches of sequences that continue earlier ones
        _delta_case("delta_train_f32", 32, 4, 4, 64, 64, 4096, "f32", True, s0=True),
        # keys shared by heads, value heads of another width, padded batches of a length nobody rounded
        _delta_case("delta_shared_bf16", 16, 8, 2, 64, 96, 1001, "bf16", True, s0=True, ragged=True),
        # two long prompts of different, odd lengths read before an answer: few heads, a long axis
        _delta_case("delta_prompt_bf16", 2, 2, 2, 128, 128, 65537, "bf16", False, s0=True, ragged=True),
        # one token for each of 256 sequences that live in a pool of states
        _step_case("delta_token_bf16", 256, 6, 6, 128, 128, "bf16", True),
        # one token of one sequence
        _step_case("delta_token_one_f32", 1, 4, 4, 64, 64, "f32", False),
        # a layer's output on its way to the residual, mixed-precision training
        _dropout_case("dropout_train_bf16", 128, 768, 1024, "bf16", 0.1, scale=0.5, res=True),
        # the headline's tensor with one position more, the rate of the paper's model
        _dropout_case("dropout_odd_f32", 32, 256, 4097, "f32", 0.01),
        # the paper's own shape: windows of 48 steps, whole channels dropped
        _dropout_case("dropout_tied_f32", 16384, 128, 48, "f32", 0.01, tied=True),
        # a training step of the small configuration
        _dropout_case("dropout_small_bf16", 4, 64, 1024, "bf16", 0.1, res=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, unit=32):
    """Half of the widths and lengths are multiples of a power of two, as programs like them."""
    n = _log_int(rng, lo, hi)
    return max(lo, n // unit * unit) if rng.random() < 0.5 and n >= unit else n


def draw(rng):
    """Any of the above: one position to sixty-five thousand, a few thousand elements to a hundred million, either type."""
    op = rng.choice(("delta", "delta", "delta", "delta", "delta_step", "dropout", "dropout"))
    dtype = rng.choice(("f32", "bf16"))
    if op == "dropout":
        L = _width(rng, 1, 65536)
        C = _width(rng, 1, 768)
        B = max(1, int(math.exp(rng.uniform(math.log(2.0 ** 12), math.log(9e7))) / (C * L)))
        return {"op": op, "B": B, "C": C, "L": L, "dtype": dtype, "p": rng.choice((0.01, 0.1, 0.25, 0.5)), "scale": rng.choice((1.0, 0.5)),
                "res": rng.random() < 0.5, "tied": rng.random() < 0.3}
    Hk = rng.choice((1, 2, 2, 3, 4))
    H = Hk * rng.choice((1, 1, 1, 2, 4))
    case = {"op": op, "H": H, "Hk": Hk, "DK": _width(rng, 16, 128), "DV": _width(rng, 16, 128), "dtype": dtype}
    if op == "delta_step":
        return {**case, "B": _log_int(rng, 1, 256), "slots": rng.random() < 0.5}
    L = _width(rng, 1, 65536)
    train = rng.random() < 0.6
    top = 3e7 if L <= 8192 else 1e7 if not train else 4e6
    B = max(1, int(math.exp(rng.uniform(math.log(2.0 ** 14), math.log(top))) / (H * max(case["DK"], case["DV"]) * L)))
    return {**case, "B": B, "L": L, "train": train, "s0": rng.random() < 0.5, "ragged": rng.random() < 0.4}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)


def _pool(g, B):
    """A pool of more states than the batch uses (its last row never), rows in any order, every sixteenth place of the batch empty."""
    n = B + B // 4 + 2
    slots = torch.randperm(n - 1, generator=g, device="cuda")[:B].int()
    slots[15::16] = -1
    return n, slots


def _gates(g, *shape):
    """Log decays as such layers have them, some heads forgetting within a few positions and some within a thousand, and strengths of
    writing in (0, 1)."""
    H = shape[1]
    rate = torch.exp(math.log(1e-3) + math.log(1e3) * _uniform(g, H)).view(1, H, *[1] * (len(shape) - 2))
    return -rate * torch.nn.functional.softplus(_normal(g, *shape)), torch.sigmoid(_normal(g, *shape))


def prepare(case, seed):
    g, dt, op = _generator(seed), DTYPES[case["dtype"]], case["op"]
    s, B = dict(case), case["B"]
    if op == "dropout":
        shape = B, case["C"], case["L"]
        s["x"], s["dout"] = _normal(g, *shape).to(dt), _normal(g, *shape).to(dt)
        s["residual"] = _normal(g, *shape).to(dt) if case["res"] else None
        s["rng"] = torch.randint(0, 1 << 62, (2,), generator=g, device="cuda")       # seed and step
        return s
    H, Hk, DK, DV = case["H"], case["Hk"], case["DK"], case["DV"]
    tail = (case["L"],) if op == "delta" else ()
    s["q"], s["k"], s["v"] = (_normal(g, B, n, *tail).to(dt) for n in (Hk * DK, Hk * DK, H * DV))
    s["g"], s["beta"] = _gates(g, B, H, *tail)
    if op == "delta_step":
        n, s["rows"] = _pool(g, B) if case["slots"] else (B, None)
        s["s"] = _normal(g, n, H, DK, DV) / math.sqrt(DK)
        return s
    L = case["L"]
    s["start"] = _normal(g, B, H, DK, DV) / math.sqrt(DK) if case["s0"] else None
    s["lengths"] = None
    if case["ragged"]:                  # at least half of the axis, and every sixteenth sequence empty
        s["lengths"] = torch.randint(L // 2, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        s["lengths"][15::16] = 0
    if case["train"]:
        s["do"] = _normal(g, B, H * DV, L).to(dt)
        s["ds_last"] = _normal(g, B, H, DK, DV) / math.sqrt(DK) if case["s0"] else None
    return s


# ---- the plain forms: elementary torch operations in 32 bits ----

def _split(x, H, n):
    """[B, H D, L] -> [B, H, n, CHUNK, D], zeros behind the end."""
    B, HD, L = x.shape
    x = torch.cat([x.float(), x.new_zeros(B, HD, n * CHUNK - L, dtype=torch.float32)], -1)
    return x.view(B, H, HD // H, n, CHUNK).permute(0, 1, 3, 4, 2).contiguous()


def _join(x, L, dt):
    B, H, n, _, D = x.shape
    return x.permute(0, 1, 4, 2, 3).reshape(B, H * D, n * CHUNK)[..., :L].to(dt)


def _inverse(A):
    """(I + A)^-1 of strictly lower triangular A, a row after the other."""
    T = torch.zeros_like(A) + torch.eye(CHUNK, device=A.device)
    for i in range(1, CHUNK):
        T[..., i, :i] = -(A[..., i, :i, None] * T[..., :i, :i]).sum(-2)
    return T


def _plain_delta(s):
    dt, B, H, Hk, DK, DV, L = s["q"].dtype, s["B"], s["H"], s["Hk"], s["DK"], s["DV"], s["L"]
    n, each, dev = -(-L // CHUNK), H // Hk, s["q"].device
    inside = torch.ones(B, 1, L, dtype=torch.bool, device=dev)
    if s["lengths"] is not None:
        inside = (torch.arange(L, device=dev) < s["lengths"][:, None])[:, None, :]
    cut = lambda x, h: _split(torch.where(inside, x, 0.0), h, n)        # noqa: E731
    q, k, v = cut(s["q"], Hk), cut(s["k"], Hk), cut(s["v"], H)
    rq, rk = (torch.rsqrt((x * x).sum(-1, keepdim=True) + EPS) for x in (q, k))
    q, k = q * rq, k * rk                                               # of unit length
    scale = DK ** -0.5
    qs, kh = (q * scale).repeat_interleave(each, 1), k.repeat_interleave(each, 1)
    gate = lambda x: torch.nn.functional.pad(torch.where(inside, x, 0.0), (0, n * CHUNK - L)).view(B, H, n, CHUNK)      # noqa: E731
    G, beta = gate(s["g"]).double().cumsum(-1), gate(s["beta"])[..., None]
    low = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=dev).tril()
    D = torch.where(low, torch.exp(torch.where(low, G[..., :, None] - G[..., None, :], 0.0)), 0.0).float()
    eG, eC = torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None]
    eA = torch.exp(G[..., -1]).float()[..., None, None]                 # of the whole chunk
    KK = torch.where(low.tril(-1), kh @ kh.transpose(-1, -2) * D, 0.0)
    P = qs @ kh.transpose(-1, -2) * D
    T = _inverse(beta * KK)
    kin, kout, qin = eG * kh, eC * kh, eG * qs
    U, W = T @ (beta * v), T @ (beta * kin)
    S = torch.zeros(B, H, DK, DV, device=dev) if s["start"] is None else s["start"].clone()
    starts, w = [], []
    for c in range(n):
        starts.append(S)
        w.append(U[:, :, c] - W[:, :, c] @ S)
        S = eA[:, :, c] * S + kout[:, :, c].transpose(-1, -2) @ w[-1]
    S0, w = torch.stack(starts, 2), torch.stack(w, 2)
    masked = lambda x, d: torch.where(inside, _join(x, L, torch.float32), 0.0).to(d)        # noqa: E731
    out = {"o": masked(qin @ S0 + P @ w, dt), "s_last": S}
    if not s["train"]:
        return out
    do = cut(s["do"], H)
    dw0, TT = P.transpose(-1, -2) @ do, T.transpose(-1, -2)
    dS = torch.zeros_like(S) if s["ds_last"] is None else s["ds_last"]
    after, dR = [None] * n, [None] * n
    for c in range(n - 1, -1, -1):
        after[c] = dS
        dR[c] = TT[:, :, c] @ (dw0[:, :, c] + kout[:, :, c] @ dS)
        dS = eA[:, :, c] * dS + qin[:, :, c].transpose(-1, -2) @ do[:, :, c] - (beta * kin)[:, :, c].transpose(-1, -2) @ dR[c]
    after, dR = torch.stack(after, 2), torch.stack(dR, 2)
    u = v - kin @ S0 - KK @ w
    dP = torch.where(low, do @ w.transpose(-1, -2), 0.0)
    dA = torch.where(low.tril(-1), -(dR @ w.transpose(-1, -2)), 0.0) * beta
    PD, AD = dP * D, dA * D
    dq_in, dk_in, dk_out = do @ S0.transpose(-1, -2), dR @ S0.transpose(-1, -2), w @ after.transpose(-1, -2)
    dq = eG * dq_in + PD @ kh
    dk = PD.transpose(-1, -2) @ qs + (AD + AD.transpose(-1, -2)) @ kh - beta * eG * dk_in + eC * dk_out
    # what a decay in front of position t scales: the state at the chunk's start, what rows from t on take of it, what is left at the end
    # of columns before t, and every pair of a row from t on and a column before t
    pairs = (dP * P + dA * KK).double()
    e = (qin * dq_in - beta * kin * dk_in).sum(-1).double()
    f = (kout * dk_out).sum(-1).double()
    whole = eA[..., 0, 0].double() * (after * S0).sum((-1, -2)).double()
    from_t = lambda x: x.flip(-1).cumsum(-1).flip(-1)                   # noqa: E731
    dg = whole[..., None] + from_t(e) + f.cumsum(-1) - f
    dg = dg + torch.where(low, pairs.cumsum(-1) - pairs, 0.0).sum(-2)   # (row i >= t: the pairs of columns before t)
    dbeta = (dR * u).sum(-1)
    group = lambda x: x.view(B, Hk, each, n, CHUNK, DK).sum(2)          # noqa: E731
    dq, dk = group(dq) * scale, group(dk)
    out["dq"] = masked(rq * (dq - q * (q * dq).sum(-1, keepdim=True)), dt)
    out["dk"] = masked(rk * (dk - k * (k * dk).sum(-1, keepdim=True)), dt)
    out["dv"] = masked(beta * dR, dt)
    flat = lambda x: torch.where(inside, x.float().view(B, H, n * CHUNK)[..., :L], 0.0)     # noqa: E731
    out["dg"], out["dbeta"], out["ds0"] = flat(dg), flat(dbeta), dS
    return out


def _plain_delta_step(s):
    B, H, Hk, DK, DV, rows, S = s["B"], s["H"], s["Hk"], s["DK"], s["DV"], s["rows"], s["s"]
    q, k, v = s["q"].float().view(B, Hk, DK), s["k"].float().view(B, Hk, DK), s["v"].float().view(B, H, DV)
    q, k = (x * torch.rsqrt((x * x).sum(-1, keepdim=True) + EPS) for x in (q, k))
    q, k = (x.repeat_interleave(H // Hk, 1) for x in (q * DK ** -0.5, k))
    used = torch.ones(B, dtype=torch.bool, device=S.device) if rows is None else rows >= 0
    # (an empty place of the batch takes the pool's last row along, whose values it writes back)
    at = torch.arange(B, device=S.device) if rows is None else torch.where(used, rows.long(), S.shape[0] - 1)
    before = S[at]
    now = torch.exp(s["g"])[..., None, None] * before
    u = v - (now * k[..., None]).sum(-2)
    now = now + s["beta"][..., None, None] * k[..., None] * u[..., None, :]
    o = (now * q[..., None]).sum(-2)
    S[at] = torch.where(used[:, None, None, None], now, before)
    return {"o": torch.where(used[:, None], o.view(B, H * DV), 0.0).to(s["q"].dtype), "s": S}


def _philox(counter, key):
    """philox4x32-10 (Salmon et al., 2011) of four words each in 64 bits."""
    low = 0xFFFFFFFF
    c, (k0, k1) = list(counter), key
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c


def _single(p):
    return struct.unpack("f", struct.pack("f", p))[0]


def _keep(s):
    B, C, L = s["x"].shape
    n, dev = C if s["tied"] else C * L, s["x"].device
    m = torch.arange(-(-n // 8), device=dev)
    b = torch.arange(B, device=dev)[:, None]
    seed, step = s["rng"][0], s["rng"][1]
    low = 0xFFFFFFFF
    key = seed & low, (seed >> 32) & low
    bits = []
    for half in (0, 1):
        words = _philox((m & low, b, step & low, (m >> 32 << 1) + (LAYER << 8 | half)), key)
        words = torch.stack(torch.broadcast_tensors(*words), -1)
        bits.append(torch.stack([words & 0xFFFF, words >> 16], -1).view(B, -1)[:, :n])
    kept = (bits[0] << 16 | bits[1]) >= round(_single(s["p"]) * 2.0 ** 32)
    return kept.view(B, C, -1)


def _plain_dropout(s):
    dt, kept, f = s["x"].dtype, _keep(s), s["scale"] / (1.0 - _single(s["p"]))
    out, dx = torch.where(kept, s["x"].float() * f, 0.0), torch.where(kept, s["dout"].float() * f, 0.0)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return {"out": out.to(dt), "dx": dx.to(dt)}


PLAIN = {"delta": _plain_delta, "delta_step": _plain_delta_step, "dropout": _plain_dropout}


# ---- the framework's operators ----

def _own_delta(s):
    from paper_2604_25422_amd import block
    o, s_last, states = block.delta_fwd(s["q"], s["k"], s["v"], s["g"], s["beta"], s["start"], s["lengths"], key_heads=s["Hk"], eps=EPS,
                                        save=s["train"])
    out = {"o": o, "s_last": s_last}
    if s["train"]:
        out["dq"], out["dk"], out["dv"], out["dg"], out["dbeta"], out["ds0"] = block.delta_bwd(
            s["do"], s["q"], s["k"], s["v"], s["g"], s["beta"], states, s["ds_last"], s["lengths"], key_heads=s["Hk"], eps=EPS)
    return out


def _own_delta_step(s):
    from paper_2604_25422_amd import block
    return {"o": block.delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["s"], s["rows"], key_heads=s["Hk"], eps=EPS), "s": s["s"]}


def _own_dropout(s):
    from paper_2604_25422_amd import block
    return {"out": block.dropout_fwd(s["x"], s["p"], s["rng"], LAYER, s["residual"], scale=s["scale"], tied=s["tied"]),
            "dx": block.dropout_bwd(s["dout"], s["p"], s["rng"], LAYER, scale=s["scale"], tied=s["tied"])}


OWN = {"delta": _own_delta, "delta_step": _own_delta_step, "dropout": _own_dropout}


def run(state):
    return (OWN if own else PLAIN)[state["op"]](state)


def work(case):
    """Per call (forward and backward are two: the rest of a model runs between them): every tensor it takes read once, every tensor it
    returns written once (up to the sequences' ends).  Of a pool, what the batch uses.  Operations as the rule's own sums have them."""
    op, e, B = case["op"], ELEM[case["dtype"]], case["B"]
    if op == "dropout":
        n = B * case["C"] * case["L"]
        return {"bytes": n * e * (5 if case["res"] else 4) + 32, "flops": n * 4}
    H, Hk, DK, DV = case["H"], case["Hk"], case["DK"], case["DV"]
    keys, values, states = Hk * DK * e, H * DV * e, B * H * DK * DV
    if op == "delta_step":
        return {"bytes": B * (2 * keys + 2 * values + 8 * H) + 8 * states, "flops": 7 * states}
    L = case["L"]
    inside = 0.75 if case["ragged"] else 1.0                # what lies behind a sequence's end is written (zeros), not read
    size = B * L * (inside * (2 * keys + values + 8 * H) + values) + 4 * states * (2 if case["s0"] else 1)
    if case["train"]:
        size += B * L * (inside * (2 * keys + 2 * values + 8 * H) + 2 * keys + values + 8 * H) + 4 * states * (2 if case["s0"] else 1)
    return {"bytes": size, "flops": inside * L * states * (29 if case["train"] else 7)}


# ---- from the definitions, in 64 bits ----

def _exact_delta(case, seed):
    """Position by position, and back by the chain rule through every step; states at every 64th position are kept, the rest formed
    again."""
    s = prepare(case, seed)
    B, H, Hk, DK, DV, L = (case[x] for x in ("B", "H", "Hk", "DK", "DV", "L"))
    each, span = H // Hk, 64
    first = lambda x, h: x.double().view(B, h, -1, L).permute(3, 0, 1, 2).contiguous()      # noqa: E731  ([L, B, h, D])
    q0, k0, v = first(s["q"], Hk), first(s["k"], Hk), first(s["v"], H)
    lq, lk = torch.sqrt(q0.pow(2).sum(-1) + EPS), torch.sqrt(k0.pow(2).sum(-1) + EPS)
    wide = lambda x: x.repeat_interleave(each, 2)           # noqa: E731
    q, k = wide(q0 / lq[..., None]) / math.sqrt(DK), wide(k0 / lk[..., None])
    a, beta = (x.double().permute(2, 0, 1).contiguous() for x in (torch.exp(s["g"].double()), s["beta"]))
    if s["lengths"] is not None:
        off = torch.arange(L, device="cuda")[:, None] >= s["lengths"].long()
        for x, value in ((q, 0.0), (k, 0.0), (v, 0.0), (a, 1.0), (beta, 0.0)):
            x[off] = value
    S = torch.zeros(B, H, DK, DV, dtype=torch.float64, device="cuda") if s["start"] is None else s["start"].double()

    def step(S, t):
        fresh = a[t][..., None, None] * S
        u = v[t] - torch.matmul(k[t][..., None, :], fresh)[..., 0, :]
        return fresh.addcmul_(k[t][..., None], (beta[t][..., None] * u)[..., None, :]), u
    o, marks = torch.empty_like(v), []
    for t in range(L):
        if t % span == 0 and case["train"]:
            marks.append(S)
        S, _ = step(S, t)
        o[t] = torch.matmul(q[t][..., None, :], S)[..., 0, :]
    back = lambda x: x.permute(1, 2, 3, 0).reshape(B, -1, L)        # noqa: E731
    out = {"o": back(o), "s_last": S}
    if not case["train"]:
        return out
    do = first(s["do"], H)
    if s["lengths"] is not None:
        do[off] = 0.0
    dS = torch.zeros_like(S) if s["ds_last"] is None else s["ds_last"].double()
    dq, dk, dv, da, db = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(a), torch.empty_like(beta)
    times = lambda M, x: torch.matmul(M, x[..., None])[..., 0]      # noqa: E731
    for c in range(len(marks) - 1, -1, -1):
        kept = [(marks[c], None)]
        for t in range(c * span, min(L, (c + 1) * span)):
            kept.append(step(kept[-1][0], t))
        for t in range(min(L, (c + 1) * span) - 1, c * span - 1, -1):
            after, u = kept.pop()
            before = kept[-1][0]
            dq[t] = times(after, do[t])
            dS = dS.addcmul(q[t][..., None], do[t][..., None, :])
            written = torch.matmul(k[t][..., None, :], dS)[..., 0, :]
            db[t] = (written * u).sum(-1)
            dv[t] = beta[t][..., None] * written
            dk[t] = times(dS, beta[t][..., None] * u) - a[t][..., None] * times(before, dv[t])
            dS = dS.addcmul_(k[t][..., None], dv[t][..., None, :], value=-1)
            da[t] = (dS * before).sum((-1, -2))
            dS = dS * a[t][..., None, None]
    group = lambda x: x.view(L, B, Hk, each, DK).sum(3)     # noqa: E731
    dq, dk = group(dq) / math.sqrt(DK), group(dk)
    # quotient rule: d(x / |x|) = dx / |x| - x (x . dx) / |x|^3
    for x, n, dx in ((q0, lq[..., None], dq), (k0, lk[..., None], dk)):
        dx.copy_(dx / n - x * (x * dx).sum(-1, keepdim=True) / n.pow(3))
    dg = da * a
    if s["lengths"] is not None:
        for x in (dq, dk, dv, dg, db):
            x[off] = 0.0
    return {**out, "dq": back(dq), "dk": back(dk), "dv": back(dv), "dg": dg.permute(1, 2, 0), "dbeta": db.permute(1, 2, 0), "ds0": dS}


def _exact_delta_step(case, seed):
    s = prepare(case, seed)
    B, H, Hk, DK, DV = (case[x] for x in ("B", "H", "Hk", "DK", "DV"))
    S, o = s["s"].double(), torch.zeros(B, H, DV, dtype=torch.float64, device="cuda")
    unit = lambda x: x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) + EPS)       # noqa: E731
    q, k = (unit(s[x].double().view(B, Hk, DK)).repeat_interleave(H // Hk, 1) for x in ("q", "k"))
    v, g, beta = s["v"].double().view(B, H, DV), s["g"].double(), s["beta"].double()
    for b, row in enumerate(range(B) if s["rows"] is None else s["rows"].tolist()):
        if row >= 0:
            kept = S[row] * torch.exp(g[b])[:, None, None]
            u = v[b] - (k[b][..., None] * kept).sum(1)
            S[row] = kept + (beta[b][:, None] * k[b])[..., None] * u[:, None, :]
            o[b] = (q[b][..., None] * S[row]).sum(1) / math.sqrt(DK)
    return {"o": o.view(B, H * DV), "s": S}


def _blocks_of(seed, step, layer, b, m, half):
    """One block of the generator in Python's whole numbers, for checks of the decisions."""
    c, k = [m & 0xFFFFFFFF, b, step & 0xFFFFFFFF, layer << 8 | m >> 32 << 1 | half], [seed & 0xFFFFFFFF, seed >> 32]
    for r in range(10):
        x, y = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        keys = [(w + r * d) & 0xFFFFFFFF for w, d in zip(k, (0x9E3779B9, 0xBB67AE85))]
        c = [y >> 32 ^ c[1] ^ keys[0], y & 0xFFFFFFFF, x >> 32 ^ c[3] ^ keys[1], x & 0xFFFFFFFF]
    return c


def _exact_dropout(case, seed):
    """The decisions are whole numbers and the plain form's; a few thousand of them are formed again, one at a time."""
    s = prepare(case, seed)
    kept = _keep(s)
    B, n, (start, step) = case["B"], kept[0].numel(), s["rng"].tolist()
    rng, limit = random.Random(seed), round(_single(case["p"]) * 2.0 ** 32)
    places = [(rng.randrange(B), rng.randrange(n)) for _ in range(2000)]
    flat = kept.view(B, -1).cpu()
    for b, j in places:
        hi, lo = (_blocks_of(start, step, LAYER, b, j >> 3, half)[(j & 7) >> 1] >> 16 * (j & 1) & 0xFFFF for half in (0, 1))
        if bool(flat[b, j]) != ((hi << 16 | lo) >= limit):
            raise ValueError(f"the decision of element {j} of entry {b} is another one")
    keep = kept.double() * (case["scale"] / (1 - _single(case["p"])))
    out = s["x"].double() * keep
    if s["residual"] is not None:
        out += s["residual"].double()
    return {"out": out, "dx": s["dout"].double() * keep}


def exact(case, seed):
    return {"delta": _exact_delta, "delta_step": _exact_delta_step, "dropout": _exact_dropout}[case["op"]](case, seed)

"""The block operators from their definitions, in 64 bits on the CPU, with bounds on what 32-bit arithmetic may be off.

U is 2^-23, twice the rounding of one 32-bit operation.  A value that is a product of k rounded factors is off by at most k U / 2 of
itself.  A gate (sigmoid of a logit of a few units, through a hardware exponential of a rounded argument and a reciprocal), the
decay and sqrt(1 - a^2) come to fewer than 40 roundings together.  A term of the recurrence that is n steps old has passed n
products with a decay that is itself rounded: 2 n roundings more; `age` sums those ages along with the absolute terms.  Joining
spans adds a logarithm of the length: below 30 roundings for any length that fits memory."""
import torch

U = 2.0 ** -23
BF16 = 2.0 ** -8            # a rounding to bf16 is off by at most half of this


def rounding(dtype):
    return BF16 if dtype == torch.bfloat16 else U


def scan(x, r, i, lam, h0=None, lengths=None, rate=8.0, dy=None, dh_last=None):
    """y, h_last and with dy all gradients, in 64 bits, and {name: bound on the 32-bit error}."""
    x, r, i, lam = (t.double().cpu() for t in (x, r, i, lam))
    B, C, L = x.shape
    h0 = torch.zeros(B, C, dtype=torch.float64) if h0 is None else h0.double().cpu()
    n = torch.full((B,), L) if lengths is None else lengths.cpu().long().clamp(0, L)
    inside = (torch.arange(L) < n[:, None])[:, None, :].expand(B, C, L)
    sr, si = torch.sigmoid(r), torch.sigmoid(i)
    sp = torch.nn.functional.softplus(lam)
    q = rate * sp[:, None] * sr
    a, s = torch.exp(-q), -torch.expm1(-2 * q)
    beta = s.sqrt()
    u = torch.where(inside, beta * si * x, 0.0)
    a = torch.where(inside, a, 1.0)
    h, m, age = h0.clone(), h0.abs(), torch.zeros_like(h0)
    hs, ms, ages = [h], [m], [age]
    for t in range(L):
        age = a[..., t] * (age + m)
        m = a[..., t] * m + u[..., t].abs()
        h = a[..., t] * h + u[..., t]
        hs.append(h), ms.append(m), ages.append(age)
    H, M, A = (torch.stack(v, -1) for v in (hs, ms, ages))
    zero = torch.zeros_like(x)
    out = {"y": torch.where(inside, H[..., 1:], zero), "h_last": H[..., -1]}
    herr = U * (40 * M + 2 * A)
    err = {"y": torch.where(inside, herr[..., 1:], zero), "h_last": herr[..., -1]}
    if dy is None:
        return out, err
    dy = torch.where(inside, dy.double().cpu(), zero)
    v = torch.zeros_like(h0) if dh_last is None else dh_last.double().cpu()
    vm, vage = v.abs(), torch.zeros_like(v)
    g, gm, gage = zero.clone(), zero.clone(), zero.clone()
    for t in range(L - 1, -1, -1):
        g[..., t], gm[..., t], gage[..., t] = dy[..., t] + v, dy[..., t].abs() + vm, vage
        v, vage, vm = a[..., t] * g[..., t], a[..., t] * (vage + gm[..., t]), a[..., t] * gm[..., t]
    gerr = U * (40 * gm + 2 * gage)
    tiny = s <= 0
    pull = torch.where(tiny, 0.0, a / torch.where(tiny, 1.0, s)) * u                 # a u / (1 - a^2)
    e, em = q * a * (pull - H[..., :-1]), q * a * (pull.abs() + M[..., :-1])
    eerr = 40 * U * em + q * a * herr[..., :-1]
    factor = torch.where(lam < -30, 1.0, torch.sigmoid(lam) / torch.where(sp > 0, sp, 1.0))
    d = torch.where(inside, g * e, zero)
    derr = torch.where(inside, gerr * em + gm * eerr, zero)
    for name, f in (("dx", beta * si), ("di", u * torch.sigmoid(-i))):
        out[name], err[name] = torch.where(inside, g * f, zero), torch.where(inside, (gerr + 40 * U * gm) * f.abs(), zero)
    out["dr"], err["dr"] = d * torch.sigmoid(-r), derr * torch.sigmoid(-r)
    out["dlam"], err["dlam"] = d.sum((0, 2)) * factor, (derr + 40 * U * (gm * em) * inside).sum((0, 2)) * factor
    out["dh0"], err["dh0"] = v, U * (40 * vm + 2 * vage)
    return out, err


def norm(y, z, res, w, w_next, eps=1e-6, scale=1.0, dout=None, dn=None, c_axis=1):
    """out, n and with dn all gradients.  Bounds: a sum over C channels in partial sums of at most 64 + log2 terms each way; every
    output is a product of fewer than 40 rounded factors, a mean enters with the roundings of its sum."""
    res, w_next = res.double().cpu(), w_next.double().cpu()[:, None]
    C = res.shape[1]
    k = 40 + C / 32 + 16
    block = y is not None
    if block:
        y, z, w = y.double().cpu(), z.double().cpu(), w.double().cpu()[:, None]
        r1 = 1 / torch.sqrt(y.square().mean(1, keepdim=True) + eps)
        sg = torch.sigmoid(z)
        yh, silu = y * r1, z * sg
        o = res + scale * silu * yh * w
        om = res.abs() + (scale * silu * yh * w).abs()
    else:
        o, om = res, res.abs()
    r2 = 1 / torch.sqrt(o.square().mean(1, keepdim=True) + eps)
    # (the mean of out^2 is off by what out itself is off, relative to its size)
    r2_rel = U * k * (om * om).mean(1, keepdim=True) * r2 * r2
    out, err = {"n": o * r2 * w_next}, {"n": (om * U * k + o.abs() * r2_rel) * r2 * w_next.abs()}
    if block:
        out["out"], err["out"] = o, om * U * k
    if dn is None:
        return out, err
    dn = dn.double().cpu()
    do0 = torch.zeros_like(res) if dout is None else dout.double().cpu()
    oh, dnw = o * r2, dn * w_next
    ohm = om * r2
    m, mm = (dnw * oh).mean(1, keepdim=True), (dnw * ohm).abs().mean(1, keepdim=True)
    do = do0 + r2 * (dnw - oh * m)
    dom = do0.abs() + r2 * (dnw.abs() + ohm * mm)
    derr = (U * k + 3 * r2_rel) * dom
    out["dres"], err["dres"] = do, derr
    out["dw_next"], err["dw_next"] = (dn * oh).sum((0, 2)), ((dn * ohm).abs() * (U * k + 3 * r2_rel)).sum((0, 2)) + U * 200 * (dn * ohm).abs().sum((0, 2))
    if block:
        g = scale * silu
        dyh = do * g * w
        mm1 = (dom * g.abs() * w.abs() * yh.abs()).mean(1, keepdim=True)
        err1 = ((derr + U * k * dom) * (g * w * yh).abs()).mean(1, keepdim=True)
        out["dy"] = r1 * (dyh - yh * (dyh * yh).mean(1, keepdim=True))
        err["dy"] = r1 * ((derr + U * k * dom) * (g * w).abs() + yh.abs() * (err1 + U * k * mm1))
        ds = scale * sg * (1 + z * torch.sigmoid(-z))
        out["dz"] = do * yh * w * ds
        err["dz"] = (derr + U * k * dom) * (yh * w).abs() * scale * sg * (1 + z.abs() * torch.sigmoid(-z))
        out["dw"] = (do * g * yh).sum((0, 2))
        err["dw"] = ((derr + U * k * dom) * (g * yh).abs()).sum((0, 2)) + U * 200 * (dom * (g * yh).abs()).sum((0, 2))
    return out, err


def check(got, ref, err, dtype, name, floor=1e-30):
    """Every element within its bound and the rounding to its storage type."""
    got, ref, err = got.detach().double().cpu(), ref.double(), err.double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert torch.isfinite(got).all(), name
    if got.numel() == 0:
        return
    off = (got - ref).abs() - (err + ref.abs() * rounding(dtype) + floor)
    at = int(off.argmax())
    assert off.max() <= 0, (name, "at", at, "got", float(got.reshape(-1)[at]), "wanted", float(ref.reshape(-1)[at]), "bound", float(err.reshape(-1)[at]))

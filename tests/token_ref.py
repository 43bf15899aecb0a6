"""The operators on rows of tokens in float64 on the CPU, from their definitions (include/revnet.h, "operators on rows of tokens")."""
import math

import numpy as np
import torch

U = 2.0 ** -24                      # half a step of float32, relative
HALF = {"f32": U, "bf16": 2.0 ** -8}  # half a step of an output type, relative
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOP = {"int8": 127.0, "e4m3": 448.0}
GELU_K = 2 * math.sqrt(2 / math.pi)


# ------------------------------------------------------------------ the checkpoint format, byte by byte
def layout(rows, channels):
    pitch = (channels + 31) // 32 * 32
    at = (rows * pitch + 255) // 256 * 256
    groups, padded = (channels + 127) // 128, (rows + 63) // 64 * 64
    return pitch, at, groups, padded, at + groups * padded * 4


def _e4m3_code(q):
    """Nearest e4m3 byte of |q| <= 448, ties to even mantissa, from the list of its 127 magnitudes."""
    mags = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])
    a = np.abs(q)
    hi = np.clip(np.searchsorted(mags, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - mags[lo], mags[hi] - a
    pick = np.where(dl < dh, lo, np.where(dl > dh, hi, np.where(lo % 2 == 0, lo, hi)))
    return (pick | np.where(np.signbit(q), 0x80, 0)).astype(np.uint8)


def encode(x, code):
    """-> (code bytes [rows][pitch], scale bytes [rows][pitch / 32]) of a float64 array."""
    x = np.asarray(x, np.float64)
    rows, channels = x.shape
    pitch = layout(rows, channels)[0]
    v = np.zeros((rows, pitch))
    v[:, :channels] = x
    v = v.reshape(rows, pitch // 32, 32)
    top = np.abs(v).max(2) if rows else np.zeros((0, pitch // 32))
    bad = ~np.isfinite(top)
    e = np.full(top.shape, -117)
    ok = ~bad & (top > 0)
    e[ok] = np.maximum(-117, np.ceil(np.log2(top[ok] / TOP[code])).astype(int))
    with np.errstate(invalid="ignore"):
        e = np.where(ok & (top > TOP[code] * 2.0 ** e), e + 1, e)                      # the logarithm's rounding
        e = np.where(ok & (e > -117) & (top <= TOP[code] * 2.0 ** (e - 1)), e - 1, e)
        q = np.where(bad[..., None], 0.0, v / 2.0 ** e[..., None])
    c = np.rint(q).astype(np.int64).astype(np.int8).view(np.uint8) if code == "int8" else _e4m3_code(q)
    return c.reshape(rows, pitch), np.where(bad, 255, e + 127).astype(np.uint8)


def code_values(c, code):
    c = np.asarray(c, np.uint8)
    if code == "int8":
        return c.view(np.int8).astype(np.float64)
    e, m = (c >> 3) & 15, (c & 7).astype(np.float64)
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(np.float64) - 10)) * np.where(c & 0x80, -1.0, 1.0)


def take_apart(buf, rows, channels):
    """A checkpoint buffer (uint8 tensor) -> (code bytes [rows][pitch], scale bytes [rows][pitch / 32])."""
    b = buf.cpu().numpy()
    pitch, at, groups, padded, size = layout(rows, channels)
    s = b[at:size].reshape(groups, padded, 4)[:, :rows].transpose(1, 0, 2).reshape(rows, groups * 4)[:, :pitch // 32]
    return b[:rows * pitch].reshape(rows, pitch), s


def put_together(c, s, rows, channels, fill=0):
    pitch, at, groups, padded, size = layout(rows, channels)
    b = np.full(size, fill, np.uint8)
    b[:rows * pitch] = c.reshape(-1)
    v = b[at:size].reshape(groups, padded, 4)
    for j in range(pitch // 32):
        v[j // 4, :rows, j % 4] = s[:, j]
    return torch.from_numpy(b)


def decode(c, s, channels, code):
    v = code_values(c, code).reshape(c.shape[0], -1, 32)
    scale = np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127))
    return torch.from_numpy((v * scale[..., None]).reshape(c.shape[0], -1)[:, :channels].copy())


def held(buf, rows, channels, code):
    return decode(*take_apart(buf, rows, channels), channels, code)


def half_step(c, s, channels, code):
    """Half the distance to the next code, of every value held."""
    scale = np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, axis=1)
    if code == "int8":
        h = np.full(c.shape, 0.5)
    else:
        e = np.maximum((c >> 3) & 15, 1).astype(np.float64)
        h = 2.0 ** (e - 10) / 2
        h = np.where((c & 7) == 7, 2 * h, h)         # above the last mantissa of a binade the codes are twice as far apart
    return torch.from_numpy((h * scale)[:, :channels].copy())


# ------------------------------------------------------------------ activations
def act(x, kind):
    if kind == "swiglu":
        g, u = x.chunk(2, 1)
        return g * torch.sigmoid(g) * u
    if kind == "relu":
        return torch.where(x > 0, x, torch.where(x != x, x, 0.0 * torch.ones_like(x)))
    if kind == "silu":
        return x * torch.sigmoid(x)
    if kind == "gelu":
        return x * torch.sigmoid(GELU_K * (x + 0.044715 * x ** 3))
    return x


def act_bwd(x, da, kind):
    """The formulas of the backward pass."""
    if kind == "swiglu":
        g, u = x.chunk(2, 1)
        s = torch.sigmoid(g)
        return torch.cat([da * u * s * (1 + g * (1 - s)), da * g * s], 1)
    if kind == "relu":
        return torch.where(x > 0, da, torch.zeros_like(da))
    if kind == "silu":
        s = torch.sigmoid(x)
        return da * s * (1 + x * (1 - s))
    if kind == "gelu":
        s = torch.sigmoid(GELU_K * (x + 0.044715 * x ** 3))
        return da * (s + x * s * (1 - s) * GELU_K * (1 + 3 * 0.044715 * x * x))
    return da


def _arg(x, kind):
    return GELU_K * (x + 0.044715 * x ** 3) if kind == "gelu" else x


def act_tol(x, kind):
    """Bounds on the float32 errors of act and of its derivative.  e^arg as 2^(arg log2 e) is off by 2 steps of 2^-23 and by 1.17 |arg| through the
    rounded product, arg itself by three roundings, the reciprocal by two steps, the sum 1 + e by half of one: (8 + 2 |arg|) steps for the sigmoid s,
    relative, and as much, absolute, of s for 1 - s; the products add five."""
    if kind in ("none", "relu"):
        return torch.zeros_like(x), torch.zeros_like(x)
    k = GELU_K * (1 + 3 * 0.044715 * x * x) if kind == "gelu" else torch.ones_like(x)
    s = torch.sigmoid(_arg(x, kind))
    eps = (16 + 2 * _arg(x, kind).abs()) * 2.0 ** -23
    tiny = 2.0 ** -120                               # below: the quotient by an infinite denominator is 0
    return eps * (x * s).abs() + tiny, eps * (s + (x * s * k).abs() * (1 + (1 - s))) + tiny


# ------------------------------------------------------------------ norm
def norm_fwd(h, gamma, eps):
    rstd = 1 / torch.sqrt((h * h).mean(1) + eps)
    xh = h * rstd[:, None]
    return rstd, xh, xh * gamma


def norm_bwd(dn, dh, xh, rstd, gamma):
    gd = dn * gamma
    return dh + rstd[:, None] * (gd - xh * (gd * xh).mean(1, keepdim=True)), (dn * xh).sum(0)


# ------------------------------------------------------------------ log probabilities
def logprobs(x, targets):
    """-> (lse, logp, entropy) in float64; target -1: logp 0."""
    m = x.amax(1, keepdim=True)
    lse = torch.where(m[:, 0] == -math.inf, m[:, 0], (m + torch.log(torch.exp(x - m).sum(1, keepdim=True)))[:, 0])
    q = x - lse[:, None]
    p = torch.exp(q)
    ent = -torch.where(p > 0, p * q, torch.where(p != p, p, torch.zeros_like(p))).sum(1)
    none = lse == -math.inf
    ent = torch.where(none, torch.zeros_like(ent), ent)
    logp = x.gather(1, targets.clamp(0, x.shape[1] - 1).long()[:, None])[:, 0] - lse
    logp = torch.where(none, torch.full_like(logp, -math.inf), logp)
    return lse, torch.where(targets == -1, torch.zeros_like(logp), logp), ent


def logprobs_bwd(x, targets, lse, ent, g, ge):
    """Rows of finite lse."""
    q = x - lse[:, None]
    p = torch.exp(q)
    g = torch.where(targets >= 0, g, torch.zeros_like(g))
    d = -p * (g[:, None] + torch.where(p > 0, ge[:, None] * (q + ent[:, None]), torch.zeros_like(p)))
    return d.scatter_add(1, targets.clamp_min(0).long()[:, None], g[:, None])


def top(x, k):
    """Indices of the k largest, the lowest index first among equals, NaN first of all."""
    v = x.numpy().copy()
    nan = np.isnan(v)
    v[nan] = np.inf
    order = np.lexsort((np.broadcast_to(np.arange(v.shape[1]), v.shape), -v, ~nan), axis=1)
    return torch.from_numpy(order[:, :k].astype(np.int32))

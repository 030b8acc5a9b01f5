"""Definitions of a quantized attention block's operators (include/fgq.h), in
numpy and in 64 bits, for the tests: int8 rows with one scale a row, the cache's
groups of channels, attention over the cache's values.  Runs on the CPU and
shares no code with the library."""
import numpy as np
import torch

F32 = np.float32
# unit roundoff and smallest step of the output types
ROUND = {torch.float32: (2.0 ** -24, 2.0 ** -149), torch.float16: (2.0 ** -11, 2.0 ** -24),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -133)}
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def rows(x):
    """Codes (int8) and scales (fp32) of the rows of x (fp32 [M][K])."""
    a = np.abs(x).max(1)
    bad = ~np.isfinite(x).all(1)
    zero = (a < 2.0 ** -120) & ~bad
    with np.errstate(all="ignore"):
        r = np.where(bad | zero, F32(0), F32(127) / a).astype(F32)
        s = np.where(bad, F32(np.nan), np.where(zero, F32(1), a / F32(127))).astype(F32)
        p = np.where((bad | zero)[:, None], F32(0), x * r[:, None])
    return np.rint(p).astype(np.int8), s


def product(q, sx, w, sw, bias):
    """The product in 64 bits, and the magnitude its fp32 roundings are relative to."""
    t = (q.astype(np.int64) @ w.astype(np.int64).T).astype(np.float64)
    t = t * sx.astype(np.float64)[:, None] * sw.astype(np.float64)[None]
    mag = np.abs(t)
    if bias is not None:
        t, mag = t + bias.astype(np.float64), mag + np.abs(bias.astype(np.float64))
    return t, mag


def _bf16(b, up):
    """fp64 values rounded to the bf16 grid, up or down (fp32 range, normal numbers)."""
    e = np.maximum(np.frexp(b)[1], -125)
    grid = np.ldexp(1.0, e - 8)
    return (np.ceil(b / grid) if up else np.floor(b / grid)) * grid


def groups(x, bits, G):
    """Cache codes, lo and step of x (fp32 [...][D], finite): codes int [...][D], fp32 [...][D / G]."""
    L = 15 if bits == 4 else 255
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // G, G)).astype(F32)
    lo = _bf16(g.min(-1).astype(np.float64), False).astype(F32)
    s = (g.max(-1) * F32(0.5) - lo * F32(0.5)) * F32(2.0 / L)
    s = _bf16(s.astype(np.float64), True).astype(F32)
    s[s < 2.0 ** -120] = 0
    with np.errstate(divide="ignore"):
        inv = np.where(s > 0, F32(1) / s, F32(0)).astype(F32)
    with np.errstate(over="ignore"):
        c = np.clip(np.rint((g - lo[..., None]) * inv[..., None]), 0, L).astype(np.int64)
    return c.reshape(x.shape), lo, s


def values(c, lo, s, G):
    """What codes stand for, fp64."""
    g = c.reshape(c.shape[:-1] + (c.shape[-1] // G, G)).astype(np.float64)
    return (lo.astype(np.float64)[..., None] + s.astype(np.float64)[..., None] * g).reshape(c.shape)


def head_bytes(P, D, bits, G):
    return 2 * P * (D * bits // 8 + 4 * (D // G))


def pack_pages(ck, lk, sk, cv, lv, sv, P, bits, G):
    """Whole pages: codes [pages * P][H][D] and their parameters -> uint8 [pages][H][bytes]."""
    n, H, D = ck.shape

    def part(c):
        c = c.reshape(n // P, P, H, D).transpose(0, 2, 1, 3)
        b = c if bits == 8 else c[..., 0::2] | c[..., 1::2] << 4
        return b.astype(np.uint8).reshape(n // P, H, -1)

    def par(lo, s):
        w = (lo.view(np.uint32) >> 16) | (s.view(np.uint32) & 0xFFFF0000)
        w = w.reshape(n // P, P, H, D // G).transpose(0, 2, 3, 1)
        return np.ascontiguousarray(w).view(np.uint8).reshape(n // P, H, -1)

    return np.concatenate([part(ck), part(cv), par(lk, sk), par(lv, sv)], -1)


def attention(q, k, v, n, causal, window, scale):
    """One sequence, one head, fp64: q [nq][D], k and v [n][D].  Returns (o,
    lse, p): p [nq][n] the probabilities, zero where a key is hidden."""
    nq = q.shape[0]
    i, j = np.arange(nq)[:, None] + n - nq, np.arange(n)[None]
    see = np.ones((nq, n), bool)
    if causal:
        see &= j <= i
        if window:
            see &= j > i - window
    s = np.where(see, q @ k[:n].T * scale, -np.inf) if n else np.zeros((nq, 0))
    m = s.max(1, keepdims=True, initial=-np.inf)
    e = np.where(see, np.exp(s - np.where(np.isfinite(m), m, 0)), 0)
    l = e.sum(1, keepdims=True)
    p = e / np.where(l > 0, l, 1)
    with np.errstate(divide="ignore"):
        lse = (np.log(l) + np.where(np.isfinite(m), m, 0))[:, 0]
    return p @ v[:n], lse, p

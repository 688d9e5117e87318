"""Rotary positions, per-head norms and window attention written out in float64, from their formulas."""
import math

import numpy as np


def freqs(sections, base=10000.0, scaling="none", factor=1.0, orig=4096.0, fast=32.0, slow=1.0):
    """Radians a position of every pair, axis after axis."""
    out = []
    for n in sections:
        for i in range(n):
            if scaling == "ntk" and n > 1:
                f = (base * factor ** (n / (n - 1.0))) ** (-i / n)
            else:
                f = base ** (-i / n)
            if scaling == "linear":
                f = f / factor
            if scaling == "yarn":
                first = max(math.floor(n * math.log(orig / (fast * 2 * math.pi)) / math.log(base)), 0)
                last = min(math.ceil(n * math.log(orig / (slow * 2 * math.pi)) / math.log(base)), n - 1)
                r = min(max((i - first) / max(last - first, 0.001), 0.0), 1.0)
                f = f * (1 - r) + f / factor * r
            out.append(f)
    return np.array(out)


def rope(x, pos, sections, f, amp=1.0, layout="interleaved", inverse=False):
    """x [B, L, H, D] float64, pos [axes, B, L]: rotated on its first 2 sum(sections) channels."""
    y = np.array(x, np.float64)
    half = sum(sections)
    i = 0
    for a, n in enumerate(sections):
        for _ in range(n):
            th = pos[a].astype(np.float64) * f[i]
            if inverse:
                th = -th
            c, s = np.cos(th)[..., None], np.sin(th)[..., None]
            p, q = (i, half + i) if layout == "half" else (2 * i, 2 * i + 1)
            u, v = np.array(x[..., p], np.float64), np.array(x[..., q], np.float64)
            y[..., p], y[..., q] = amp * (u * c - v * s), amp * (u * s + v * c)
            i += 1
    return y


def headnorm(x, g, eps):
    x = np.asarray(x, np.float64)
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(g, np.float64)


def seen(p, klen, left, right, sink, group):
    """Keys that the query at position p sees: a truth value for each of klen."""
    j = np.arange(klen)
    ok = np.ones(klen, bool)
    if right >= 0:
        ok &= j // group <= p // group + right
    if left >= 0:
        ok &= (j // group >= p // group - left) | (j < sink)
    return ok


def attention(q, k, v, left=-1, right=0, sink=0, group=1, scale=None, q_len=None, k_len=None, q_start=None):
    """q [B, Lq, H, D], k, v [B, Lk, Hk, D] -> out [B, Lq, H, D], lse [B, H, Lq] (NaN for rows behind the last), and
    sum of weight |v| [B, Lq, H, D] and the largest sum of |scale q k|, which the errors are counted in."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    B, Lq, H, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    n = H // Hk
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse = np.full((B, H, Lq), np.nan)
    big = 0.0
    for b in range(B):
        lq = Lq if q_len is None else int(q_len[b])
        lk = Lk if k_len is None else int(k_len[b])
        start = lk - lq if q_start is None else int(q_start[b])
        if lq == 0:
            continue
        mask = np.stack([seen(start + i, lk, left, right, sink, group) for i in range(lq)])  # [lq, lk]
        used = mask.any(0)
        for h in range(H):
            kk, vv = np.where(used[:, None], k[b, :lk, h // n], 0.0), np.where(used[:, None], v[b, :lk, h // n], 0.0)
            x = np.where(mask, scale * (q[b, :lq, h] @ kk.T), -np.inf)
            if lk:
                big = max(big, float((np.abs(q[b, :lq, h]) @ np.abs(kk).T).max()) * scale)
            m = np.where(mask.any(1), x.max(1, initial=-np.inf), 0.0)
            e = np.exp(x - m[:, None])
            d = e.sum(1)
            w = e / np.where(d > 0, d, 1.0)[:, None]
            out[b, :lq, h] = w @ vv
            mag[b, :lq, h] = w @ np.abs(vv)
            with np.errstate(divide="ignore"):
                lse[b, h, :lq] = m + np.log(d)
    return out, lse, mag, big

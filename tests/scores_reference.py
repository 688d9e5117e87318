"""Attention with capped logits, a bias by distance, documents and prefixes in float64, from its formula."""
import numpy as np


def seen(p, klen, left, right, group, ends=(), prefix=None):
    """Keys that the query at position p sees: a truth value for each of klen.  prefix: one of each document."""
    j = np.arange(klen)
    ends = np.asarray(ends, np.int64)
    doc = int((ends <= p).sum())
    ok = (ends[None, :] <= j[:, None]).sum(1) == doc
    if right >= 0:
        late = j // group <= p // group + right
        if prefix is not None:
            late |= j < (ends[doc - 1] if doc else 0) + prefix[doc]
        ok &= late
    if left >= 0:
        ok &= j // group >= p // group - left
    return ok


def attention(q, k, v, left=-1, right=0, group=1, scale=None, cap=0.0, slopes=None, ends=None, prefix=None, q_len=None,
              k_len=None, q_start=None):
    """q [B, Lq, H, D], k, v [B, Lk, Hk, D] -> out, lse (NaN for rows behind the last), sum of weight |v|, and the largest
    sum of |scale q k| and bias, which the errors are counted in."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    B, Lq, H, D = q.shape
    Lk, n = k.shape[1], H // k.shape[2]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse = np.full((B, H, Lq), np.nan)
    big = far = 0.0
    for b in range(B):
        lq = Lq if q_len is None else int(q_len[b])
        lk = Lk if k_len is None else int(k_len[b])
        start = lk - lq if q_start is None else int(q_start[b])
        if lq == 0:
            continue
        mask = np.stack([seen(start + i, lk, left, right, group, () if ends is None else ends[b],
                              None if prefix is None else prefix[b]) for i in range(lq)])
        dist = np.abs(start + np.arange(lq)[:, None] - np.arange(lk)[None, :])
        used = mask.any(0)
        for h in range(H):
            kk, vv = np.where(used[:, None], k[b, :lk, h // n], 0.0), np.where(used[:, None], v[b, :lk, h // n], 0.0)
            x = scale * (q[b, :lq, h] @ kk.T)
            if lk:
                big = max(big, float((np.abs(q[b, :lq, h]) @ np.abs(kk).T).max()) * scale)
            if cap:
                x = cap * np.tanh(x / cap)
            if slopes is not None:
                x = x - float(slopes[h]) * dist
                far = max(far, abs(float(slopes[h])) * float((dist * mask).max(initial=0)))
            x = np.where(mask, x, -np.inf)
            m = np.where(mask.any(1), x.max(1, initial=-np.inf), 0.0)
            e = np.exp(x - m[:, None])
            d = e.sum(1)
            w = e / np.where(d > 0, d, 1.0)[:, None]
            out[b, :lq, h] = w @ vv
            mag[b, :lq, h] = w @ np.abs(vv)
            with np.errstate(divide="ignore"):
                lse[b, h, :lq] = m + np.log(d)
    return out, lse, mag, big, far

"""The 4-bit cache written out in float64 and bytes, from its definition."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """x [..., D] float64 -> codes [..., D] (sign in bit 3) and exponent bytes [..., D / 32]."""
    y = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    odd = ~np.isfinite(y).all(-1)
    a = np.abs(np.where(odd[..., None], 0.0, y))
    top = a.max(-1)
    e = np.full(top.shape, -124)
    for c in range(-124, 126):          # the smallest at which the largest rounds to 6 or less: it is below 7
        e = np.where((top >= 7.0 * 2.0 ** (c - 1)) & (c > -124), c, e)
    u = a / 2.0 ** e[..., None]
    dist = np.abs(u[..., None] - LEVELS)
    best = dist.min(-1, keepdims=True)
    near = dist == best                 # two at a tie: the even code
    code = np.where(near.sum(-1) == 2, (near & (np.arange(8) % 2 == 0)).argmax(-1), near.argmax(-1))
    code = code + 8 * np.signbit(y)
    code = np.where(odd[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(odd, 255, e + 127).astype(np.uint8)


def values(code, byte):
    """What codes and exponent bytes stand for, float64."""
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127.0))
    return v * np.repeat(scale, 32, axis=-1)


class Pool:
    """Pages as bytes, element by element."""

    def __init__(self, n_pages, heads, D, page_tokens, fill):
        self.heads, self.D, self.P = heads, D, page_tokens
        self.raw = np.full((n_pages, page_tokens // 64, heads, 68 * D), fill, np.uint8)

    def _at(self, tok):
        """Byte offsets of a token's codes (channel pairs) and exponents: K, V, K's, V's."""
        D, G = self.D, self.D // 32
        s, r, c = tok // 32, tok // 8 % 4, tok % 8
        i, g = np.arange(D // 2), np.arange(G)
        k = tok * (D // 2) + i
        v = 32 * D + i // 16 * 1024 + r * 256 + i % 16 * 16 + s * 8 + c
        ke = 64 * D + (((4 * r + c % 4) * G + g) * 2 + s) * 2 + c // 4
        ve = 66 * D + g * 64 + r * 16 + s * 8 + c
        return k, v, ke, ve

    def put(self, page, tok, k, v):
        """k, v: (codes [heads, D], exponents [heads, G])."""
        at = self._at(tok % 64)
        block = self.raw[page, tok // 64]
        for (code, byte), c, e in ((k, at[0], at[2]), (v, at[1], at[3])):
            block[:, c] = code[:, 0::2] | code[:, 1::2] << 4
            block[:, e] = byte

    def get(self, page, tok):
        at = self._at(tok % 64)
        block = self.raw[page, tok // 64]
        out = []
        for c, e in ((at[0], at[2]), (at[1], at[3])):
            code = np.empty((self.heads, self.D), np.uint8)
            code[:, 0::2], code[:, 1::2] = block[:, c] & 15, block[:, c] >> 4
            out.append(values(code, block[:, e]))
        return out

    def places(self, table, count):
        """Values of places 0 .. count - 1 of every sequence [B, count, heads, D], and whether a page holds them [B, count]."""
        B = table.shape[0]
        k = np.zeros((B, count, self.heads, self.D))
        v, there = np.zeros_like(k), np.zeros((B, count), bool)
        for b in range(B):
            for x in range(count):
                page = table[b, x // self.P] if x // self.P < table.shape[1] else -1
                if 0 <= page < len(self.raw):
                    k[b, x], v[b, x] = self.get(page, x % self.P)
                    there[b, x] = True
        return k, v, there


def attention(q, k, v, there, seen, scale, q_len=None, k_len=None, q_start=None):
    """q [B, Lq, H, D]; k, v [B, Lk, Hk, D]; seen(position, keys) -> truth value for each key -> out, lse (NaN behind the
    last row), sum of weight |v|, largest sum of |scale q k|.  Keys that are not `there` are not seen."""
    B, Lq, H, D = q.shape
    Lk, n = k.shape[1], H // k.shape[2]
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse = np.full((B, H, Lq), np.nan)
    big = 0.0
    for b in range(B):
        lq = Lq if q_len is None else int(q_len[b])
        lk = Lk if k_len is None else int(k_len[b])
        start = lk - lq if q_start is None else int(q_start[b])
        if lq == 0:
            continue
        mask = np.stack([seen(start + i, lk) for i in range(lq)]) & there[b, :lk]
        used = mask.any(0)
        for h in range(H):
            kk, vv = np.where(used[:, None], k[b, :lk, h // n], 0.0), np.where(used[:, None], v[b, :lk, h // n], 0.0)
            x = np.where(mask, scale * (q[b, :lq, h] @ kk.T), -np.inf)
            if lk:
                big = max(big, float(np.nan_to_num(np.abs(q[b, :lq, h]) @ np.abs(kk).T).max()) * scale)
            m = np.where(mask.any(1), x.max(1, initial=-np.inf), 0.0)
            e = np.exp(x - m[:, None])
            d = e.sum(1)
            w = e / np.where(d > 0, d, 1.0)[:, None]
            out[b, :lq, h] = w @ vv
            mag[b, :lq, h] = w @ np.abs(vv)
            with np.errstate(divide="ignore"):
                lse[b, h, :lq] = m + np.log(d)
    return out, lse, mag, big

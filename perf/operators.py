"""Operators of streaming and long-video denoisers on one MI355X: rotary positions (``op_rope``), norms of queries and
keys for each head with the rotation in the same pass (``op_headnorm_rope``), and attention with a sliding window and
first tokens that stay visible (``op_attention_window``).

A case is one call.  With ``own`` false ``run`` computes it from elementary torch operations in 32 bits (angles in 64),
with ``own`` true through ``paper_2609_30096_amd.track``.  ``exact`` evaluates the definitions in 64 bits.  Sizes are
the library's widths (12 and 40 heads of 128, 1560 tokens a latent frame, 21 frames, the small float32 pair) and
generic ones; ``draw`` spreads the same calls over their ranges, ragged sizes included.
"""
from __future__ import annotations

import math

import torch

own = False

FRAME = 1560       # tokens of a latent frame of the 480 x 832 video
MAX_FLOPS = 7.0e12  # no drawn attention costs more than attn_video_bf16
MAX_BYTES = 3.5e9   # nor any drawn call moves more than attn_token_long_bf16
LOG2E = 1.4426950408889634


# ---------------------------------------------------------------- the cases
def _rope(kind, dtype, B, L, H, Hk, D, rot, layout, sections, scaling, pos0, factor=1.0, inverse=False, fused=False,
          qlog2=False):
    return {"kind": kind, "dtype": dtype, "B": B, "L": L, "H": H, "Hk": Hk, "D": D, "rot": rot, "layout": layout,
            "sections": sections, "scaling": scaling, "factor": factor, "pos0": pos0, "inverse": inverse,
            "fused": fused, "qlog2": qlog2}


def _attn(dtype, B, H, Hk, D, Lq, Lk, left, right, sink, group, ragged):
    return {"kind": "attn", "dtype": dtype, "B": B, "H": H, "Hk": Hk, "D": D, "Lq": Lq, "Lk": Lk, "left": left,
            "right": right, "sink": sink, "group": group, "ragged": ragged}


def listed():
    return [
        # Serving, one new token for each of 16 sequences far into a stretched context: latency.
        {"name": "rope_tokens_bf16", **_rope("rope", "bf16", 16, 1, 40, 8, 128, 128, "half", "1", "yarn", 180000, 8.0)},
        # Cached keys and queries moved back to position 0 (the inverse), half of each head rotated, odd length.
        {"name": "rope_partial_f32",
         **_rope("rope", "f32", 2, 4099, 8, 8, 64, 32, "interleaved", "1", "linear", 0, 4.0, inverse=True)},
        # The guided video step's queries and keys (cond and negative prompt) at 1.3B width, 3D positions.
        {"name": "rope_video_bf16", **_rope("rope", "bf16", 2, 32760, 12, 12, 128, 128, "interleaved", "3", "none", 0)},
        # One new token for each of 5 sequences, per-head norms, shared key heads: latency.
        {"name": "headnorm_rope_tokens_bf16",
         **_rope("headnorm", "bf16", 5, 1, 40, 8, 128, 128, "half", "1", "none", 9000)},
        # A ragged float32 prompt with part of the head rotated.
        {"name": "headnorm_rope_prompt_f32",
         **_rope("headnorm", "f32", 3, 1777, 10, 2, 128, 64, "half", "1", "ntk", 50, 2.0)},
        # The guided video step at 14B width, read from the fused projection, q in the log2 form of the attention.
        {"name": "headnorm_rope_video_bf16",
         **_rope("headnorm", "bf16", 2, 32760, 40, 40, 128, 128, "interleaved", "3", "none", 0, fused=True,
                 qlog2=True)},
        # The small float32 pair's 64 tokens, frames of 16 tokens that see their neighbours: launches and latency.
        {"name": "attn_small_f32", **_attn("f32", 2, 4, 4, 32, 64, 64, 1, 1, 0, 16, False)},
        # A float32 prompt with a token window and first tokens, odd length.
        {"name": "attn_prompt_f32", **_attn("f32", 1, 8, 4, 64, 1501, 1501, 299, 0, 5, 1, False)},
        # Serving: one token for each of 4 sequences, the last 1024 of 8192 cached keys and 4 first ones.
        {"name": "attn_token_window_bf16", **_attn("bf16", 4, 40, 8, 128, 1, 8192, 1023, 0, 4, 1, True)},
        # Serving over long caches of different lengths, everything visible.
        {"name": "attn_token_long_bf16", **_attn("bf16", 8, 40, 8, 128, 1, 100003, -1, 0, 0, 1, True)},
        # Streaming video: three new frames against the last twelve of a 21-frame cache and the first frame.
        {"name": "attn_stream_bf16", **_attn("bf16", 1, 12, 12, 128, 3 * FRAME, 21 * FRAME, 11, 0, FRAME, FRAME, False)},
        # Whole-video self-attention of the guided step, each frame seeing four on either side and the first.
        {"name": "attn_video_bf16",
         **_attn("bf16", 2, 12, 12, 128, 21 * FRAME, 21 * FRAME, 4, 4, FRAME, FRAME, False)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if rng.random() < 0.5:
            kind = rng.choice(["rope", "headnorm"])
            D = rng.choice([32, 64, 80, 96, 128, 128, 256])
            Hk = rng.choice([1, 2, 3, 4, 8, 12])
            H = Hk * rng.choice([1, 1, 2, 4, 5])
            layout = rng.choice(["interleaved", "half"])
            sections = rng.choice(["1", "1", "3"])
            rot = D if sections == "3" else rng.choice([D, D // 2])
            scaling = "none" if sections == "3" else rng.choice(["none", "linear", "ntk", "yarn"])
            L = 1 if rng.random() < 0.25 else _log(rng, 2, 40000)
            B = rng.randint(1, 24) if L == 1 else rng.randint(1, 3)
            case = _rope(kind, dtype, B, L, H, Hk, D, rot, layout, sections, scaling, _log(rng, 1, 300000),
                         1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]),
                         inverse=kind == "rope" and rng.random() < 0.3, fused=rng.random() < 0.5,
                         qlog2=kind == "headnorm" and rng.random() < 0.5)
        else:
            D = 128 if dtype == "bf16" else rng.choice([32, 64, 128])
            Hk = rng.choice([1, 2, 3, 4, 8, 12])
            H = Hk * rng.choice([1, 1, 2, 4, 5])
            form = rng.choice(["token", "few", "prompt", "frames"])
            top = 100000 if dtype == "bf16" else 8000
            if form == "token":
                Lk = _log(rng, 1, top)
                case = _attn(dtype, rng.randint(1, 8), H, Hk, D, 1, Lk, rng.choice([-1, _log(rng, 1, Lk)]), 0,
                             rng.choice([0, 1, 4, 100]), 1, rng.random() < 0.7)
            elif form == "few":
                Lq = rng.randint(2, 100)
                Lk = Lq + _log(rng, 1, top)
                case = _attn(dtype, rng.randint(1, 4), H, Hk, D, Lq, Lk, rng.choice([-1, _log(rng, 1, Lk)]), 0,
                             rng.choice([0, 1, 4, 100]), 1, rng.random() < 0.5)
            elif form == "prompt":
                Lq = _log(rng, 100, top // 8)
                case = _attn(dtype, rng.randint(1, 3), H, Hk, D, Lq, Lq + rng.choice([0, _log(rng, 1, top // 8)]),
                             rng.choice([-1, _log(rng, 1, Lq)]), rng.choice([0, 0, -1]),
                             rng.choice([0, 1, 4, 100]), 1, rng.random() < 0.5)
            else:
                group = _log(rng, 16, FRAME if dtype == "bf16" else 200)
                frames = rng.randint(2, 21)
                new = rng.choice([1, min(3, frames), frames])
                case = _attn(dtype, rng.randint(1, 2), H, Hk, D, new * group, frames * group,
                             rng.choice([-1, rng.randint(0, frames)]), rng.choice([0, 0, 1, 4]),
                             rng.choice([0, group]), group, False)
        w = work(case)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return case


# ---------------------------------------------------------------- what a pass cannot do without
def _lengths(case):
    """(queries, keys) of each sequence: whole, or shorter by a fixed pattern where ragged."""
    out = []
    for b in range(case["B"]):
        lq, lk = case["Lq"], case["Lk"]
        if case["ragged"] and b:
            lk = max(1, lk - (b * lk) // (2 * case["B"]) - b)
            if lq > 1:
                lq = max(1, lq - (b * lq) // (3 * case["B"]) - b)
        out.append((lq, lk))
    return out


def _seen(case, lq, lk, i):
    """Rows i (a tensor or a number): position and seen key ranges [0, first), [lo, hi)."""
    G = case["group"]
    p = lk - lq + i
    g = p // G
    if case["right"] < 0:
        hi = p * 0 + lk
    else:
        hi = (g + case["right"] + 1) * G
    lo = p * 0 if case["left"] < 0 else (g - case["left"]) * G
    return p, lo, hi


def _clip(x, lo, hi):
    return max(lo, min(x, hi))


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] != "attn":
        n = case["B"] * case["L"] * (case["H"] + case["Hk"]) * case["D"]
        axes = 3 if case["sections"] == "3" else 1
        return {"bytes": 2 * n * e + 4 * axes * case["B"] * case["L"], "flops": (3 if case["kind"] == "rope" else 7) * n}
    H, Hk, D, G = case["H"], case["Hk"], case["D"], case["group"]
    bytes_, pairs = 0, 0
    for lq, lk in _lengths(case):
        keys = set()
        span = None
        n = 0
        i = 0
        while i < lq:  # rows of one group see the same keys
            p, lo, hi = _seen(case, lq, lk, i)
            step = min(lq - i, G - p % G)
            hi = _clip(hi, 0, lk)
            lo = _clip(lo, 0, hi)
            first = min(case["sink"], lo)
            n += step * (hi - lo + first)
            span = (lo, hi, first) if span is None else (min(span[0], lo), max(span[1], hi), max(span[2], first))
            i += step
        keys = span[1] - span[0] + min(span[2], span[0])
        pairs += n
        bytes_ += 2 * lq * H * D * e + 2 * keys * Hk * D * e
    return {"bytes": bytes_, "flops": 4 * D * H * pairs}


# ---------------------------------------------------------------- inputs
def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _sections(case):
    n = case["rot"] // 2
    if case["sections"] == "1":
        return (n,)
    s = case["D"] // 6  # the library's split of a head between frames, height and width
    return (n - 2 * s, s, s)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dt(case)

    def normal(*shape, scale=1.0):
        t = torch.empty(*shape, dtype=dt, device="cuda")
        return t.normal_(0.0, scale, generator=g)

    if case["kind"] != "attn":
        B, L, H, Hk, D = (case[k] for k in ("B", "L", "H", "Hk", "D"))
        if case["fused"]:  # rows of a fused projection: q, k and v beside each other
            rows = normal(B * L, (H + 2 * Hk) * D)
            q = rows[:, :H * D].unflatten(0, (B, L)).unflatten(2, (H, D))
            k = rows[:, H * D:(H + Hk) * D].unflatten(0, (B, L)).unflatten(2, (Hk, D))
        else:
            q, k = normal(B, L, H, D), normal(B, L, Hk, D)
        axes = len(_sections(case))
        t = torch.arange(L, device="cuda", dtype=torch.int64)
        start = torch.randint(0, case["pos0"] + 1, (B, 1), generator=g, device="cuda")
        if axes == 1:
            pos = (start + t)[None]
        else:  # frame, row and column of each token; frames start anywhere
            h, w = 30, 52
            pos = torch.stack([start + t // (h * w), (t // w % h).expand(B, L), (t % w).expand(B, L)])
        st = {"case": case, "q": q, "k": k, "pos": pos.to(torch.int32).contiguous(),
              "freqs": torch.tensor(_freqs(case)[0], dtype=torch.float64, device="cuda"), "amp": _freqs(case)[1]}
        if case["kind"] == "headnorm":
            st["g_q"] = (1.0 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(dt)
            st["g_k"] = (1.0 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(dt)
        if own:
            from paper_2609_30096_amd import track
            st["rope"] = track.Rope(track.RopeConfig(
                head_dim=D, rot_dim=case["rot"], layout=case["layout"], sections=_sections(case), base=10000.0,
                scaling=case["scaling"], factor=case["factor"], orig_len=4096.0))
            st["q_out"] = torch.empty(B, L, H, D, dtype=dt, device="cuda")
            st["k_out"] = torch.empty(B, L, Hk, D, dtype=dt, device="cuda")
        return st
    B, H, Hk, D, Lq, Lk = (case[k] for k in ("B", "H", "Hk", "D", "Lq", "Lk"))
    lens = _lengths(case)
    cap = (Lk + 63) // 64 * 64  # what a cache of this length is rounded up to
    st = {"case": case, "lens": lens,
          # normalised queries and keys: logits of standard deviation about 2
          "q": normal(B, Lq, H, D, scale=1.5), "k": normal(B, cap, Hk, D, scale=1.5), "vt": normal(B, Hk, D, cap),
          "out": torch.zeros(B, Lq, H, D, dtype=dt, device="cuda")}
    if own:
        from paper_2609_30096_amd import track
        st["window"] = track.Window(left=case["left"], right=case["right"], sink=case["sink"], group=case["group"])
        if case["ragged"]:
            st["q_len"] = torch.tensor([a for a, _ in lens], dtype=torch.int32, device="cuda")
            st["k_len"] = torch.tensor([c for _, c in lens], dtype=torch.int32, device="cuda")
        st["ws"] = track.attention_window_workspace(st["window"], st["q"], st["k"][:, :Lk])
    return st


# ---------------------------------------------------------------- plain forms (32 bits; angles in 64)
def _freqs(case):
    """Radians a position of every pair, and the amplitude of the rotation."""
    base, s, orig = 10000.0, case["factor"], 4096.0
    out, amp = [], 1.0
    for n in _sections(case):
        b = base * s ** (n / (n - 1)) if case["scaling"] == "ntk" and n > 1 else base
        for i in range(n):
            f = b ** (-i / n)
            if case["scaling"] == "linear":
                f /= s
            elif case["scaling"] == "yarn":
                # pairs of fewer than beta_slow = 1 turns in the original context are stretched, of more than
                # beta_fast = 32 kept, with a ramp over the pair index between
                lo = max(math.floor(n * math.log(orig / (32.0 * 2 * math.pi)) / math.log(base)), 0)
                hi = min(math.ceil(n * math.log(orig / (1.0 * 2 * math.pi)) / math.log(base)), n - 1)
                r = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
                f = f * (1.0 - r) + f / s * r
            out.append(f)
    if case["scaling"] == "yarn":
        amp = 0.1 * math.log(s) + 1.0
    return out, amp


def _rotate(x, c, s, rot, layout):
    """x [B, L, heads, D] by cos and sin [B, L, 1, rot / 2]."""
    if layout == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        r = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        r = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    return torch.cat([r, x[..., rot:]], dim=-1) if rot < x.shape[-1] else r


def _angles(case, st):
    parts, i = [], 0
    for a, n in enumerate(_sections(case)):
        parts.append(st["pos"][a].double().unsqueeze(-1) * st["freqs"][i:i + n])
        i += n
    th = torch.cat(parts, dim=-1)
    return -th if case["inverse"] else th


def _plain_rope(st):
    case = st["case"]
    th = _angles(case, st)
    c, s = ((f(th) * st["amp"]).float().unsqueeze(2) for f in (torch.cos, torch.sin))
    out = []
    for name in ("q", "k"):
        x = st[name].float()
        if case["kind"] == "headnorm":
            x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6) * st["g_" + name].float()
        x = _rotate(x, c, s, case["rot"], case["layout"])
        if name == "q" and case["qlog2"]:
            x = x * (LOG2E / math.sqrt(case["D"]))
        out.append(x.to(_dt(case)))
    return out


def _plain_attention(st):
    case = st["case"]
    H, Hk, D = case["H"], case["Hk"], case["D"]
    n = H // Hk
    out = st["out"]
    for b, (lq, lk) in enumerate(st["lens"]):
        for i0 in range(0, lq, 512):
            i1 = min(lq, i0 + 512)
            # the keys that any of these rows sees
            _, lo, _ = _seen(case, lq, lk, i0)
            _, _, hi = _seen(case, lq, lk, i1 - 1)
            hi = _clip(hi, 0, lk)
            lo = _clip(lo, 0, hi)
            first = min(case["sink"], lo)
            if hi - lo + first == 0:
                out[b, i0:i1] = 0.0
                continue
            j = torch.arange(lo - first, hi, device="cuda")
            j[:first] -= lo - first
            k = torch.cat([st["k"][b, :first], st["k"][b, lo:hi]]).float().permute(1, 2, 0).contiguous()
            v = torch.cat([st["vt"][b, :, :, :first], st["vt"][b, :, :, lo:hi]], dim=2).float()
            _, rlo, rhi = _seen(case, lq, lk, torch.arange(i0, i1, device="cuda")[:, None])
            seen = (j < rhi) & ((j >= rlo) | (j < case["sink"]))
            q = st["q"][b, i0:i1].float().unflatten(1, (Hk, n)).permute(1, 0, 2, 3).reshape(Hk, (i1 - i0) * n, D)
            x = torch.matmul(q * (1.0 / math.sqrt(D)), k).unflatten(1, (i1 - i0, n))
            x = x.masked_fill(~seen[:, None, :], float("-inf"))
            m = x.amax(dim=-1, keepdim=True).clamp_min(-1e30)
            e = torch.exp(x - m)
            d = e.sum(dim=-1, keepdim=True)
            o = torch.matmul(e.flatten(1, 2), v.transpose(1, 2).contiguous()).unflatten(1, (i1 - i0, n))
            o = o / d.clamp_min(1e-30)
            out[b, i0:i1] = o.permute(1, 0, 2, 3).reshape(i1 - i0, H, D).to(out.dtype)
    return out


def run(state):
    case = state["case"]
    if not own:
        return _plain_attention(state) if case["kind"] == "attn" else _plain_rope(state)
    from paper_2609_30096_amd import track
    if case["kind"] == "attn":
        return track.op_attention_window(state["window"], state["q"], state["k"][:, :case["Lk"]],
                                         state["vt"], state["out"], q_len=state.get("q_len"),
                                         k_len=state.get("k_len"), workspace=state["ws"])
    if case["kind"] == "rope":
        return track.op_rope(state["rope"], state["q"], state["k"], state["pos"], state["q_out"], state["k_out"],
                             inverse=case["inverse"])
    return track.op_headnorm_rope(state["rope"], state["q"], state["k"], state["g_q"], state["g_k"], state["pos"],
                                  state["q_out"], state["k_out"], eps=1e-6,
                                  q_scale=LOG2E / math.sqrt(case["D"]) if case["qlog2"] else 1.0)


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] != "attn":
        return _exact_rope(case, st)
    if work(case)["flops"] > MAX_FLOPS:
        return None
    H, n, D, G = case["H"], case["H"] // case["Hk"], case["D"], case["group"]
    res = torch.zeros(case["B"], case["Lq"], H, D, dtype=torch.float64, device="cuda")
    for b, (lq, lk) in enumerate(st["lens"]):
        keys = torch.arange(lk, device="cuda")
        for h in range(H):
            k = st["k"][b, :lk, h // n].double()
            v = st["vt"][b, h // n, :, :lk].double()
            for r0 in range(0, lq, 2048):
                p = torch.arange(r0, min(lq, r0 + 2048), device="cuda") + (lk - lq)
                dist = keys[None, :].div(G, rounding_mode="floor") - p[:, None].div(G, rounding_mode="floor")
                hide = torch.zeros_like(dist, dtype=torch.bool)
                if case["left"] >= 0:
                    hide |= (dist < -case["left"]) & (keys >= case["sink"])[None, :]
                if case["right"] >= 0:
                    hide |= dist > case["right"]
                z = torch.mm(st["q"][b, r0:r0 + len(p), h].double(), k.t().contiguous()).div_(math.sqrt(D))
                z[hide] = -math.inf
                pr = torch.softmax(z, dim=1).nan_to_num(nan=0.0)  # a row that sees nothing gives zeros
                res[b, r0:r0 + len(p), h] = torch.mm(pr, v.t().contiguous())
    return res


def _exact_rope(case, st):
    """Each pair as a complex number, turned by its angle."""
    w, amp = _freqs(case)
    axis = [a for a, n in enumerate(_sections(case)) for _ in range(n)]
    pos = st["pos"].double()
    turn = torch.stack([pos[a] * f for a, f in zip(axis, w)], dim=-1)
    turn = torch.polar(torch.full_like(turn, amp), -turn if case["inverse"] else turn)[:, :, None, :]
    half = case["rot"] // 2
    res = []
    for name in ("q", "k"):
        y = st[name].double()
        if case["kind"] == "headnorm":
            y = y / (y.pow(2).sum(-1, keepdim=True) / case["D"] + 1e-6).sqrt() * st["g_" + name].double()
        else:
            y = y.clone()
        re, im = (slice(0, half), slice(half, 2 * half)) if case["layout"] == "half" else (
            slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        z = torch.complex(y[..., re].contiguous(), y[..., im].contiguous()) * turn
        y[..., re], y[..., im] = z.real, z.imag
        if name == "q" and case["qlog2"]:
            y = y * LOG2E / math.sqrt(case["D"])
        res.append(y)
    return res

"""Rotary positions, per-head norms with rotation, and window attention against their formulas in float64.

Tolerances (u = eps / 2 of the output type, 2^-24 = one float32 rounding):
 * a rotated pair: the angle is reduced in float64 and rounded once to float32 turns of at most 1/2 (2^-26 turns, 9.4e-8
   radian), sine and cosine are good to 2 units in the last place (1.2e-7), two products and a sum (1.8e-7): 4e-7 of
   the pair's length, times the amplitude, then the output's rounding.
 * the norm: the sum of D squares in chains of at most 16 and 6 levels of lanes, halved by the root, with the division,
   the root and two products: under 18 roundings, 1.1e-6.
 * attention: weights off by a relative eta give |do| <= 2 eta sum w|v| (numerator and denominator).  eta is the logit's
   error (D + 2 roundings of sum |scale q k|), 2^-21 for exp2 and its argument, the rounding to bfloat16 where the
   weights take one, and the float32 sums over the keys.
"""
import ctypes
import math

import numpy as np
import pytest

import window_reference as ref
from gpu_helpers import dev, host, normal, say
from paper_2609_30096_amd import synth, track

F32, BF16 = synth.F32, synth.BF16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
PAIR, NORM = 4e-7, 1.1e-6


@pytest.fixture
def L():
    return track.lib()


# ---------------------------------------------------------------- on the host
@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("yarn", 8.0), ("yarn", 1.0)])
@pytest.mark.parametrize("sections", [(64,), (16,), (1,), (22, 21, 21), (0, 3, 1)])
def test_rope_freqs(scaling, factor, sections):
    rot = 2 * sum(sections)
    cfg = track.RopeConfig(head_dim=rot, sections=sections, scaling=scaling, factor=factor, base=10000.0)
    got, amp = track.rope_freqs(cfg)
    np.testing.assert_allclose(got, ref.freqs(sections, 10000.0, scaling, factor), rtol=1e-13)
    assert amp == pytest.approx(1.0 + 0.1 * math.log(factor) if scaling == "yarn" else 1.0, rel=1e-7)


def test_rope_freqs_properties():
    """NTK keeps the fastest pair and squeezes the slowest by the factor; YaRN leaves fast pairs and squeezes slow ones."""
    plain, _ = track.rope_freqs(track.RopeConfig(head_dim=128))
    ntk, _ = track.rope_freqs(track.RopeConfig(head_dim=128, scaling="ntk", factor=8.0))
    assert ntk[0] == plain[0] and ntk[-1] == pytest.approx(plain[-1] / 8.0, rel=1e-12)
    yarn, _ = track.rope_freqs(track.RopeConfig(head_dim=128, scaling="yarn", factor=8.0))
    ratio = yarn / plain
    assert np.all(ratio[:16] == 1.0) and np.allclose(ratio[-16:], 1 / 8.0, rtol=1e-12)
    assert np.all(np.diff(ratio) <= 0.0)


def _rope_c(**kw):
    a = dict(head_dim=128, sections=(64,))
    a.update(kw)
    return track.RopeConfig(**a).c()


def test_rope_refusals(L):
    p = 1 << 20  # aligned stand-in; never dereferenced
    E = track.DTYPE_BF16

    def rows(heads=4, ldx=512, sx=5120, ldy=512, sy=5120, x=p, y=p):
        return ctypes.byref(track.HeadRowsC(x, ldx, sx, y, ldy, sy, heads))

    def call(c=None, dtype=E, B=2, Ln=10, q=None, k=None, pos=p, freqs=p, amp=1.0, norm=False, gq=p, gk=p, eps=1e-6,
             scale=1.0):
        c = _rope_c() if c is None else c
        q = rows() if q is None else q
        if norm:
            return L.track_op_headnorm_rope(dtype, ctypes.byref(c), B, Ln, q, k, gq, gk, eps, scale, pos, freqs, amp, None)
        return L.track_op_rope(dtype, ctypes.byref(c), B, Ln, q, k, pos, freqs, amp, 0, None)

    S, I = track.E_SHAPE, track.E_INVALID
    assert L.track_op_rope(E, None, 1, 1, rows(), None, p, p, 1.0, 0, None) == I
    assert L.track_op_rope(E, ctypes.byref(_rope_c()), 1, 1, None, None, p, p, 1.0, 0, None) == I
    assert call(dtype=2) == I
    for bad in (dict(head_dim=7, rot_dim=6, sections=(3,)), dict(head_dim=258), dict(rot_dim=130, sections=(65,)),
                dict(rot_dim=63, sections=(31,)), dict(rot_dim=0, sections=(0,)), dict(sections=(63,)),
                dict(sections=(65, -1))):
        assert call(_rope_c(**bad)) == S, bad
    for bad in (dict(base=1.0), dict(base=math.inf), dict(base=math.nan), dict(scaling="linear", factor=0.5),
                dict(scaling="ntk", factor=math.nan), dict(scaling="yarn", factor=2.0, orig_len=0.0),
                dict(scaling="yarn", factor=2.0, beta_fast=math.inf)):
        assert call(_rope_c(**bad)) == I, bad
    c = _rope_c()
    c.layout = 2
    assert call(c) == I
    c = _rope_c()
    c.scaling = 4
    assert call(c) == I
    c = _rope_c()
    c.axes = 0
    assert call(c) == I
    assert call(B=-1) == S and call(Ln=-1) == S and call(B=1 << 20, Ln=1 << 20) == S
    assert call(B=1, Ln=1 << 28) == S  # more tokens than a launch holds
    assert call(q=rows(sy=512 * 10 - 1, y=p + 4096)) == S  # sequences overlap by one element
    assert call(q=rows(heads=0)) == S and call(q=rows(ldx=511)) == S and call(q=rows(ldy=511)) == S
    assert call(q=rows(sx=-1)) == S and call(q=rows(y=p + 4096, sy=511)) == S
    assert call(q=rows(x=0)) == I and call(q=rows(x=p + 1)) == I and call(q=rows(y=p + 1)) == I
    assert call(q=rows(ldx=640)) == I and call(q=rows(sx=6400)) == I  # in place with other strides
    assert call(pos=None) == I and call(freqs=None) == I and call(pos=p + 2) == I and call(freqs=p + 4) == I
    assert call(amp=math.nan) == I
    assert call(k=rows(heads=0)) == S
    assert call(norm=True, gq=None) == I and call(norm=True, k=rows(), gk=None) == I
    assert call(norm=True, eps=0.0) == I and call(norm=True, eps=math.nan) == I and call(norm=True, scale=math.inf) == I
    assert call(norm=True, gq=p + 1) == I
    assert call(B=0) == 0 and call(Ln=0) == 0  # nothing to do, nothing launched
    out = np.zeros(64)
    assert L.track_rope_freqs(ctypes.byref(_rope_c()), None, None) == I
    with pytest.raises(track.TrackError):
        track.rope_freqs(track.RopeConfig(head_dim=128, sections=(10,)))
    for bad in (dict(sections=(16, 16, 16, 16)), dict(layout="whole"), dict(scaling="dynamic")):
        with pytest.raises(ValueError):
            track.RopeConfig(head_dim=128, **bad).c()
    assert np.all(out == 0)


def test_window_refusals(L):
    p = 1 << 20
    E, F = track.DTYPE_BF16, track.DTYPE_F32
    S, I, N, Un = track.E_SHAPE, track.E_INVALID, track.E_NOMEM, track.E_UNSUPPORTED
    base = dict(B=2, H=8, Hk=4, D=128, Lq=1, Lk=5000, ldq=1024, sq=1024, ldk=512, sk=512 * 5000, ldv=5000, sv=512 * 5000,
                ldo=1024, so=1024, q=p, k=p, vt=p, out=p, lse=None, q_len=None, k_len=None, q_start=None, ws=p,
                ws_bytes=1 << 40)

    def call(dtype=E, win=None, **kw):
        a = dict(base, **kw)
        w = track.Window(left=-1, right=0) if win is None else win
        return L.track_op_attention_window(
            dtype, ctypes.byref(w.c()), a["B"], a["H"], a["Hk"], a["D"], a["Lq"], a["Lk"], a["q"], a["ldq"], a["sq"],
            a["k"], a["ldk"], a["sk"], a["vt"], a["ldv"], a["sv"], a["out"], a["ldo"], a["so"], a["lse"], a["q_len"],
            a["k_len"], a["q_start"], a["ws"], a["ws_bytes"], None)

    W = track.Window
    assert L.track_op_attention_window(E, None, *([1] * 6), *([None, 1, 1] * 4), *([None] * 5), 0, None) == I
    assert call(dtype=2) == I
    for w in (W(group=0), W(sink=-1), W(left=-2), W(right=-2), W(scale=-1.0), W(scale=math.nan), W(scale=math.inf),
              W(scale=1e-31), W(scale=1e31)):
        assert call(win=w) == I, w
    for w in (W(group=1 << 31), W(sink=1 << 31), W(left=1 << 31), W(right=1 << 31)):
        assert call(win=w) == S, w
    assert call(B=-1) == S and call(H=0) == S and call(Hk=0) == S and call(H=8, Hk=3) == S
    assert call(Lq=-1) == S and call(Lk=-1) == S and call(Lk=1 << 31) == S and call(Lq=1 << 30) == S
    assert call(D=64) == Un and call(F, D=80) == Un
    for name in ("q", "k", "vt", "out"):
        assert call(**{name: None}) == I, name
        assert call(**{name: p + 8}) == I, name          # bfloat16 rows are 16-byte aligned
        assert call(F, **{name: p + 2}) == I, name
    assert call(ldq=1016) == S and call(ldk=504) == S and call(ldo=1016) == S and call(ldv=4992) == S
    assert call(ldq=1028) == I and call(ldk=516) == I and call(sk=512 * 5000 + 4) == I and call(ldv=5004) == I
    assert call(sq=-8) == S and call(so=512) == S
    assert call(Lq=3, so=3 * 1024 - 8) == S and call(Lq=3, ldo=2040, so=1024) == S  # sequences overlap
    assert call(ldk=(1 << 23) + 8) == S and call(ldv=(1 << 23) + 8) == S
    assert call(lse=p + 2) == I and call(q_len=p + 1) == I and call(k_len=p + 1) == I and call(q_start=p + 1) == I
    need = track.attention_window_workspace_bytes(W(), E, 2, 8, 4, 128, 1, 5000)
    assert need > 0
    assert call(ws=None) == N and call(ws_bytes=need - 1) == N and call(ws=p + 128) == I
    assert call(B=0) == 0 and call(Lq=0) == 0
    assert L.track_attention_window_workspace_bytes(E, None, 1, 1, 1, 128, 1, 1) == -1
    assert L.track_attention_window_workspace_bytes(E, ctypes.byref(W().c()), 1, 1, 1, 96, 1, 1) == -1
    with pytest.raises(track.TrackError):
        track.attention_window_workspace_bytes(W(), E, 1, 3, 2, 128, 1, 1)
    assert track.attention_window_workspace_bytes(W(), E, 1, 8, 8, 128, 0, 100) == 0


def test_binding_refusals():
    import torch
    B, Ln, H, Hk, D = 2, 5, 4, 2, 128
    q, k = torch.zeros(B, Ln, H, D), torch.zeros(B, Ln, Hk, D)
    rope = track.Rope(track.RopeConfig(head_dim=D), device="cpu")
    pos = torch.zeros(1, B, Ln, dtype=torch.int32)

    def raises(*a, **kw):
        with pytest.raises((ValueError, TypeError)):
            track.op_rope(*a, **kw)

    raises(rope, q, k, pos.long())
    raises(rope, q, k, pos[:, :, :4])
    raises(rope, q, k, pos.expand(3, B, Ln))
    raises(rope, q, k[:, :4], pos)
    raises(rope, q, k.bfloat16(), pos)
    raises(rope, q.half(), None, pos)
    raises(rope, q.transpose(1, 2), None, pos)
    raises(rope, q, k, pos, q_out=q[:, :, :2])
    raises(rope, q, None, pos, k_out=k)
    raises(rope, torch.zeros(B, Ln, H, 64), None, pos)
    with pytest.raises(ValueError):
        track.op_headnorm_rope(rope, q, None, torch.ones(64), None, pos)
    vt, out = torch.zeros(B, Hk, D, 8), torch.zeros(B, Ln, H, D)
    w = track.Window()

    def bad(k=k, vt=vt, out=out, **kw):
        with pytest.raises((ValueError, TypeError)):
            track.op_attention_window(w, q, k, vt, out, **kw)

    bad(out=out[:, :4])
    bad(k=k[:1])
    bad(vt=vt[..., :4])
    bad(vt=vt.transpose(2, 3))
    bad(vt=vt.bfloat16())
    bad(lse=torch.zeros(B, H, Ln - 1))
    bad(q_len=torch.zeros(B, dtype=torch.int64))
    bad(k_len=torch.zeros(B + 1, dtype=torch.int32))


def test_sizes_whose_products_wrap(L):
    """Sizes and strides whose products pass 64 (or 32) bits are refused and not taken for small ones."""
    p, S = 1 << 20, track.E_SHAPE

    def rope(B, Ln, heads, ld, sy):
        r = track.HeadRowsC(p, ld, sy, p, ld, sy, heads)
        return L.track_op_rope(track.DTYPE_BF16, ctypes.byref(_rope_c()), B, Ln, ctypes.byref(r), ctypes.byref(r), p, p, 1.0, 0, None)

    assert rope(2, 9, 4, 1 << 61, (1 << 61) + 512) == S       # 8 rows of 2^61 are 2^64
    assert rope(1, 1, (1 << 31) - 1, 1 << 40, 1 << 40) == S   # the heads of q and k in 32 bits
    assert rope(1, 1, (1 << 19) + 1, 1 << 40, 1 << 40) == S

    def window(B, H, Hk, Lq, ldo, so):
        return L.track_op_attention_window(
            track.DTYPE_BF16, ctypes.byref(track.Window().c()), B, H, Hk, 128, Lq, 64, p, 1 << 40, 0, p, 1 << 22, 0, p, 64, 0,
            p, ldo, so, *([None] * 4), p, (1 << 63) - 1, None)

    for B, H in ((1 << 30, 1 << 30), (1 << 30, 1 << 20), (1 << 23, 1), (1 << 12, 1 << 11)):
        assert track.lib().track_attention_window_workspace_bytes(
            track.DTYPE_BF16, ctypes.byref(track.Window().c()), B, H, H, 128, 1 << 28, 64) == -1, (B, H)
    assert window(1 << 30, 1 << 15, 1 << 15, 1, 1 << 40, 1 << 22) == S
    assert window(2, 8, 4, 9, 1 << 61, (1 << 61) + 1024) == S


def test_binding_needs_positions():
    import torch
    rope = track.Rope(track.RopeConfig(head_dim=128), device="cpu")
    q, g = torch.zeros(1, 2, 4, 128), torch.ones(128)
    with pytest.raises(ValueError):
        track.op_rope(rope, q, None, None)
    with pytest.raises(ValueError):
        track.op_headnorm_rope(rope, q, None, g, None, None)


# ---------------------------------------------------------------- rotation on the GPU
gpu = pytest.mark.gpu


def _close(got, want, tol, what):
    err = np.abs(np.asarray(got, np.float64) - want)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.nanmax(err / np.maximum(tol, 1e-300)):.3g} x"


def _pair_len(y, half, layout):
    """Length of the pair that each channel belongs to (0 for copied channels)."""
    out = np.zeros_like(y)
    p, q = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    n = np.hypot(y[..., p], y[..., q])
    out[..., p] = n
    out[..., q] = n
    return out


ROPES = [
    # dtype, B, L, H, Hk, D, sections, layout, scaling, factor, far, inverse
    (BF16, 1, 1, 1, 1, 128, (64,), "half", "none", 1.0, 10, False),
    (BF16, 2, 37, 12, 12, 128, (22, 21, 21), "interleaved", "none", 1.0, 50, False),
    (BF16, 3, 5, 40, 8, 128, (64,), "half", "yarn", 8.0, 1000000, False),
    (BF16, 2, 9, 5, 1, 80, (20,), "half", "linear", 4.0, 2000, True),      # 8-byte units
    (BF16, 2, 9, 5, 1, 80, (40,), "interleaved", "ntk", 2.0, 2000, False),
    (BF16, 1, 300, 3, 2, 64, (5,), "half", "none", 1.0, 300, False),       # single elements
    (BF16, 1, 70, 2, 2, 250, (125,), "interleaved", "none", 1.0, 70, False),  # two units a lane
    (BF16, 1, 70, 2, 1, 250, (33,), "half", "none", 1.0, 70, True),
    (BF16, 1, 33, 7, 1, 256, (128,), "half", "none", 1.0, 33, False),
    (BF16, 1, 3000, 2, 1, 32, (16,), "interleaved", "none", 1.0, 3000, False),
    (BF16, 1, 6, 3, 1, 2, (1,), "half", "none", 1.0, 6, False),
    (F32, 1, 1, 4, 4, 32, (6, 5, 5), "interleaved", "none", 1.0, 4, False),
    (F32, 2, 501, 8, 8, 64, (16,), "interleaved", "linear", 4.0, 100000, True),
    (F32, 3, 77, 10, 2, 128, (32,), "half", "ntk", 2.0, 5000, False),
    (F32, 2, 40, 3, 3, 96, (48,), "half", "yarn", 4.0, 200000, False),
    (F32, 1, 20, 3, 1, 10, (5,), "interleaved", "none", 1.0, 20, False),
    (F32, 1, 20, 2, 1, 254, (127,), "half", "none", 1.0, 20, False),
    (F32, 1, 20, 2, 2, 256, (128,), "interleaved", "none", 1.0, 20, False),
]


def _rope_inputs(case, key):
    dtype, B, Ln, H, Hk, D, sections, layout, scaling, factor, far, inverse = case
    bf = dtype == BF16
    q = normal([key, 1], (B, Ln, H, D), bf16=bf)
    k = normal([key, 2], (B, Ln, Hk, D), bf16=bf)
    rng = np.random.default_rng(key)
    pos = rng.integers(-far, far + 1, (len(sections), B, Ln)).astype(np.int32)
    pos.reshape(-1)[0] = far
    rope = track.Rope(track.RopeConfig(head_dim=D, rot_dim=2 * sum(sections), layout=layout, sections=sections,
                                       scaling=scaling, factor=factor))
    return q, k, pos, rope, ref.freqs(sections, 10000.0, scaling, factor)


@gpu
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("case", ROPES, ids=str)
def test_rope(case, norm):
    import torch
    dtype, B, Ln, H, Hk, D, sections, layout, scaling, factor, far, inverse = case
    if norm and inverse:
        inverse = False
    say(f"rope norm={norm} {case}")
    q, k, pos, rope, f = _rope_inputs(case, 11)
    tq, tk, tp = dev(q, dtype), dev(k, dtype), torch.from_numpy(pos).cuda()
    half, amp, scale = sum(sections), rope.amplitude, 1.0
    want = [q.astype(np.float64), k.astype(np.float64)]
    if norm:
        gains = [1.0 + 0.2 * normal([12, i], (D,)) for i in range(2)]
        if dtype == BF16:
            gains = [synth.bf16_round(g) for g in gains]
        scale = 1.4426950408889634 / math.sqrt(D)
        want = [ref.headnorm(x, g, 1e-5) for x, g in zip(want, gains)]
        oq, ok = torch.empty_like(tq), torch.empty_like(tk)
        got = track.op_headnorm_rope(rope, tq, tk, dev(gains[0], dtype), dev(gains[1], dtype), tp, oq, ok, eps=1e-5,
                                     q_scale=scale)
        assert got[0] is oq and got[1] is ok
    else:
        got = track.op_rope(rope, tq, tk, tp, inverse=inverse)  # in place
        assert got[0] is tq and got[1] is tk
    for name, x, y, m in (("q", want[0], got[0], scale), ("k", want[1], got[1], 1.0)):
        w = m * ref.rope(x, pos, sections, f, amp, layout, inverse)
        calc = m * (PAIR * amp * _pair_len(x, half, layout)) + (NORM + PAIR) * np.abs(w) * norm + \
            m * NORM * amp * _pair_len(x, half, layout) * norm
        _close(host(y), w, calc + U[dtype] * (np.abs(w) + calc), name)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("off", [0, 1, 4])
def test_rope_strided(dtype, off):
    """q and k inside the rows of a fused projection, out into a longer cache, at any alignment: equal to the same call on
    contiguous tensors, everything else untouched.  Equal bit for bit where the rows take units of the same width; single
    elements (an odd offset) put other channels into a lane's part of the sum of squares, and two orders of a float32 sum
    of D squares differ by up to twice its error, 2 NORM relative to the pair's length (at most sqrt(D) max|g|), before the
    output's rounding on either side."""
    import torch
    B, Ln, H, Hk, D = 2, 23, 6, 2, 64
    ld = (H + 2 * Hk) * D + 16
    buf = dev(normal([21], (B * Ln * ld + off,), bf16=dtype == BF16), dtype)
    rows = buf[off:].view(B, Ln, ld)
    q, k = rows[..., :H * D].unflatten(2, (H, D)), rows[..., H * D:(H + Hk) * D].unflatten(2, (Hk, D))
    rope = track.Rope(track.RopeConfig(head_dim=D, layout="half"))
    pos = torch.arange(B * Ln, dtype=torch.int32, device="cuda").view(1, B, Ln)
    g = dev(normal([22], (D,), bf16=dtype == BF16), dtype)
    cache = torch.full((B, Ln + 9, Hk, D), 7.0, dtype=buf.dtype, device="cuda")
    before = buf.clone()
    qo = torch.empty(B, Ln, H, D, dtype=buf.dtype, device="cuda")
    track.op_headnorm_rope(rope, q, k, g, g, pos, qo, cache[:, 4:4 + Ln])
    cq, ck = track.op_headnorm_rope(rope, q.contiguous(), k.contiguous(), g, g, pos)
    assert torch.equal(buf, before)
    if off == 1:
        for a, b in ((qo, cq), (cache[:, 4:4 + Ln], ck)):
            pair = math.sqrt(D) * float(g.abs().max())
            assert bool(((a.double() - b.double()).abs() <= 2.02 * U[dtype] * b.double().abs() + 2 * NORM * pair).all())
    else:
        assert torch.equal(qo, cq) and torch.equal(cache[:, 4:4 + Ln], ck)
    assert bool((cache[:, :4] == 7).all()) and bool((cache[:, 4 + Ln:] == 7).all())
    track.op_rope(rope, q, None, pos)  # in place inside the rows
    assert torch.equal(rows[..., H * D:], before[off:].view(B, Ln, ld)[..., H * D:])
    rq, _ = track.op_rope(rope, before[off:].view(B, Ln, ld)[..., :H * D].unflatten(2, (H, D)).contiguous(), None, pos)
    assert torch.equal(q, rq)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("norm", [False, True])
def test_rope_more_than_the_caches_hold(dtype, layout, norm):
    """Heads of more than 256 MB, which are read past the caches: bit for bit what calls on parts of the tokens give."""
    import torch
    B, H, Hk, D = 2, 70, 40, 128
    Ln = 5003 if dtype == BF16 else 2503
    t = torch.bfloat16 if dtype == BF16 else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(41)
    q = torch.randn(B, Ln, H, D, device="cuda", generator=gen).to(t)
    k = torch.randn(B, Ln, Hk, D, device="cuda", generator=gen).to(t)
    assert q.nbytes + k.nbytes > 256 << 20
    pos = torch.randint(0, 1 << 20, (1, B, Ln), dtype=torch.int32, device="cuda", generator=gen)
    g = torch.randn(D, device="cuda", generator=gen).to(t)
    rope = track.Rope(track.RopeConfig(head_dim=D, layout=layout))

    def call(q, k, pos, qo, ko):
        if norm:
            track.op_headnorm_rope(rope, q, k, g, g, pos, qo, ko)
        else:
            track.op_rope(rope, q, k, pos, qo, ko)

    wq, wk = torch.empty_like(q), torch.empty_like(k)
    for i in range(0, Ln, 1000):
        j = min(Ln, i + 1000)
        call(q[:, i:j], k[:, i:j], pos[..., i:j].contiguous(), wq[:, i:j], wk[:, i:j])
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    call(q, k, pos, qo, ko)
    assert torch.equal(qo, wq) and torch.equal(ko, wk)
    call(q, k, pos, q, k)  # in place
    assert torch.equal(q, wq) and torch.equal(k, wk)


@gpu
def test_rope_far_positions_and_inverse():
    """At position 10^9 the angle still matches float64, and the inverse undoes the rotation."""
    import torch
    x = normal([31], (1, 4, 2, 128))
    pos = np.array([[[0, 1, 10 ** 9 + 7, -(10 ** 9)]]], np.int32)
    rope = track.Rope(track.RopeConfig(head_dim=128))
    tp = torch.from_numpy(pos).cuda()
    y, _ = track.op_rope(rope, dev(x), None, tp, torch.empty(1, 4, 2, 128, device="cuda"))
    w = ref.rope(x, pos, (64,), ref.freqs((64,)))
    # float64 angles of up to 1e9 radian are good to 2^-53 1e9 = 1.1e-7 on both sides
    _close(host(y), w, (PAIR + 4e-7) * _pair_len(x.astype(np.float64), 64, "interleaved") + U[F32] * np.abs(w), "far")
    assert np.array_equal(host(y)[0, 0], x[0, 0])  # position 0
    z, _ = track.op_rope(rope, y, None, tp, inverse=True)
    _close(host(z), x.astype(np.float64), 3 * PAIR * _pair_len(x.astype(np.float64), 64, "interleaved"), "inverse")


@gpu
def test_rope_gradient():
    """The inverse call is the transpose of the forward one, so it is its gradient: against differences of the formula."""
    import torch
    sections, D = (10, 3, 3), 40
    x, gy = normal([32], (1, 3, 2, D)).astype(np.float64), normal([33], (1, 3, 2, D))
    pos = np.arange(9, dtype=np.int32).reshape(3, 1, 3) * 7
    rope = track.Rope(track.RopeConfig(head_dim=D, rot_dim=32, sections=sections, scaling="yarn", factor=4.0))
    f = ref.freqs(sections, 10000.0, "yarn", 4.0)
    gx, _ = track.op_rope(rope, dev(gy), None, torch.from_numpy(pos).cuda(), inverse=True)
    diff = np.zeros_like(x)
    h = 1e-3
    for c in range(D):  # the map is linear: differences are exact up to rounding
        e = np.zeros(D)
        e[c] = h
        up, dn = (ref.rope(x + s * e, pos, sections, f, rope.amplitude) for s in (1, -1))
        diff[..., c] = ((up - dn) / (2 * h) * gy).sum(-1)
    _close(host(gx), diff, 1e-6 * np.abs(gy).max(-1, keepdims=True) + 1e-9, "gradient")


@gpu
def test_headnorm_special_rows():
    """A head of zeros stays zero; NaN and infinity stay inside their head; a head's values do not move its neighbours."""
    import torch
    B, Ln, H, D = 1, 3, 4, 128
    x = normal([41], (B, Ln, H, D), bf16=True)
    x[0, 0, 1] = 0.0
    pos = torch.arange(Ln, dtype=torch.int32, device="cuda").view(1, B, Ln)
    rope = track.Rope(track.RopeConfig(head_dim=D))
    g = dev(np.ones(D, np.float32), BF16)
    clean, _ = track.op_headnorm_rope(rope, dev(x, BF16), None, g, None, pos)
    assert bool((clean[0, 0, 1] == 0).all())
    x[0, 1, 2, 5] = np.nan
    x[0, 2, 0, 9] = np.inf
    got, _ = track.op_headnorm_rope(rope, dev(x, BF16), None, g, None, pos)
    touched = torch.zeros(B, Ln, H, dtype=torch.bool, device="cuda")
    touched[0, 1, 2] = touched[0, 2, 0] = True
    assert torch.equal(got[~touched], clean[~touched])
    assert bool(torch.isnan(got[0, 1, 2]).all())


# ---------------------------------------------------------------- window attention on the GPU
class Case:
    """Seeded inputs of one call, on the host (rounded to the type) and the device."""

    def __init__(self, dtype, B, H, Hk, Lq, Lk, D=128, key=51, cap=None, scale=1.0, poison=None):
        import torch
        bf = dtype == BF16
        self.dtype, self.Lk, self.D = dtype, Lk, D
        self.q = normal([key, 1], (B, Lq, H, D), scale, bf)
        self.k = normal([key, 2], (B, Lk, Hk, D), scale, bf)
        self.v = normal([key, 3], (B, Lk, Hk, D), 1.0, bf)
        cap = (Lk + 7) // 8 * 8 if cap is None else cap
        kc = np.full((B, cap, Hk, D), np.nan if poison is None else poison, np.float32)
        vc = np.full((B, Hk, D, cap), np.nan if poison is None else poison, np.float32)
        kc[:, :Lk] = self.k
        vc[..., :Lk] = self.v.transpose(0, 2, 3, 1)
        self.tq, self.tk, self.tv = dev(self.q, dtype), dev(kc, dtype), dev(vc, dtype)
        self.out = torch.full((B, Lq, H, D), 9.0, dtype=self.tq.dtype, device="cuda")
        self.lse = torch.full((B, H, Lq), 9.0, device="cuda")

    def run(self, win, **lens):
        import torch
        kw = {n: torch.tensor(v, dtype=torch.int32, device="cuda") for n, v in lens.items() if v is not None}
        k = self.tk[:, :self.Lk]
        ws = track.attention_window_workspace(win, self.tq, k)
        track.op_attention_window(win, self.tq, k, self.tv, self.out, lse=self.lse, workspace=ws, **kw)
        return host(self.out), host(self.lse)


def _eta(dtype, D, big, Lk):
    return (D + 2) * 2.0 ** -24 * big + 2.0 ** -21 + (Lk + 16) * 2.0 ** -24 + (U[BF16] if dtype == BF16 else 0.0)


def _check(c, win, got, lse, rows=None, **lens):
    """Against the formula on the host's inputs; of the queries `rows` only, where given."""
    want, wlse, mag, big = ref.attention(c.q, c.k, c.v, win.left, win.right, win.sink, win.group, win.scale, **lens)
    if rows is not None:
        got, lse, want, wlse, mag = got[:, rows], lse[..., rows], want[:, rows], wlse[..., rows], mag[:, rows]
    eta = _eta(c.dtype, c.D, big, c.Lk)
    there = ~np.isnan(want)
    assert np.all(got[~there] == 9.0), "rows behind the last"
    assert np.all(lse[np.isnan(wlse)] == 9.0), "lse behind the last"
    _close(got[there], want[there], (2.1 * eta * mag + U[c.dtype] * np.abs(want) * 1.01)[there], "out")
    ok = ~np.isnan(wlse)
    none = ok & (wlse == -np.inf)
    assert np.array_equal(lse[ok] == -np.inf, none[ok])
    fin = ok & ~none
    _close(lse[fin], wlse[fin], 1.1 * eta + 2.0 ** -22 * np.abs(wlse[fin]) + 1e-6, "lse")
    if none.any():
        assert np.all(got.transpose(0, 2, 1, 3)[none] == 0.0)


W = track.Window
ATTN = [
    # B, H, Hk, Lq, Lk, window, lengths
    (1, 1, 1, 1, 1, W(), {}),
    (1, 4, 4, 1, 7, W(left=2), {}),
    (2, 8, 2, 1, 200, W(left=63, sink=4), {}),
    (3, 10, 2, 1, 1000, W(left=99, sink=70), dict(k_len=[1000, 1, 517])),
    (2, 5, 1, 1, 3000, W(), dict(k_len=[3000, 2048])),                     # shares of the keys
    (1, 40, 8, 1, 5000, W(left=1023, sink=4), {}),
    (2, 4, 1, 4, 300, W(left=40, sink=3), dict(q_len=[4, 2], k_len=[300, 155])),
    (2, 4, 2, 13, 777, W(left=100), {}),
    (1, 6, 2, 16, 130, W(), {}),                                           # 48 rows: two blocks
    (1, 20, 4, 12, 2000, W(left=200, sink=1), {}),
    (2, 3, 3, 65, 65, W(), {}),
    (1, 2, 2, 300, 300, W(left=0), {}),
    (1, 2, 2, 300, 300, W(left=0, right=-1, sink=0), {}),
    (2, 4, 2, 300, 451, W(left=63, sink=5), dict(q_len=[300, 211], k_len=[451, 213])),
    (1, 2, 1, 700, 700, W(left=64, sink=64), {}),
    (1, 2, 1, 700, 700, W(left=200, sink=190), {}),
    (1, 3, 3, 640, 960, W(left=1, right=0, group=160, sink=160), {}),
    (1, 3, 3, 640, 960, W(left=1, right=2, group=100, sink=30), {}),
    (2, 2, 2, 500, 500, W(left=-1, right=-1), {}),
    (2, 2, 2, 500, 333, W(left=5), {}),                                    # the first 167 queries see nothing
    (2, 2, 2, 500, 333, W(left=0, right=3, group=7, sink=9), dict(q_start=[-600, 40])),
    (1, 2, 2, 80, 400, W(left=10), dict(q_start=[1000])),                  # the window is past the last key
    (1, 2, 2, 80, 400, W(left=10, sink=5), dict(q_start=[1000])),
    (3, 2, 1, 100, 256, W(left=20), dict(q_len=[0, 100, 50], k_len=[256, 0, 256])),
    (1, 1, 1, 70, 4000, W(), {}),                                          # shares of the keys, blocks
    (1, 2, 1, 200, 9000, W(left=2500, sink=130), {}),
    (1, 1, 1, 257, 257, W(sink=1000), {}),
    (2, 8, 8, 1040, 1040, W(left=300, sink=5), dict(q_len=[1040, 900], k_len=[1040, 1000])),  # more blocks than CUs hold
    # limits at the ends of their ranges
    (1, 2, 1, 100, 300, W(left=1 << 28, right=1 << 28, group=1 << 28, sink=1 << 28), {}),
    (1, 2, 1, 100, 300, W(left=0, right=0, group=1 << 28), {}),
    (1, 2, 1, 100, 300, W(left=0, right=1 << 28, group=3), {}),
    (3, 2, 1, 20, 300, W(left=100, right=0, sink=7), dict(q_start=[-(1 << 28), 1 << 28, 290])),
    (2, 2, 1, 20, 300, W(left=3, right=0, group=100), dict(q_start=[-250, 250])),
]


@gpu
@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F32, 32), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("case", ATTN, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}_{c[3]}x{c[4]}_l{c[5].left}r{c[5].right}s{c[5].sink}g{c[5].group}{'v' if c[6] else ''}")
def test_window_attention(dtype, D, case):
    B, H, Hk, Lq, Lk, win, lens = case
    say(f"window {dtype} D={D} {case}")
    c = Case(dtype, B, H, Hk, Lq, Lk, D)
    got, lse = c.run(win, **lens)
    _check(c, win, got, lse, **lens)
    again, lse2 = c.run(win, **lens)
    assert np.array_equal(got, again, equal_nan=True) and np.array_equal(lse, lse2)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq,Lk,lens", [(1, 1000, {}), (1, 6000, dict(k_len=[5001])), (9, 700, {}), (400, 900, {}),
                                        (400, 900, dict(k_len=[777]))])
def test_window_masked_places(dtype, Lq, Lk, lens):
    """NaN and infinities in K and V where a query does not look do not reach its output: behind the last key, before
    every window, and at places that other queries of the same block do see."""
    import torch
    win = W(left=49, sink=3)
    lk = lens.get("k_len", [Lk])[0]
    say(f"masked places {dtype} {Lq} {Lk} {lens}")
    c = Case(dtype, 1, 4, 2, Lq, Lk)  # NaN behind Lk already
    first = max(lk - Lq - 49, 3)      # no query looks at 3 .. first - 1
    for value in (float("nan"), float("inf"), torch.finfo(c.tk.dtype).min):
        c.tk[:, 3:first] = value
        c.tv[..., 3:first] = value
        c.tk[:, lk:] = value
        c.tv[..., lk:] = value
        _check(c, win, *c.run(win, **lens), **lens)
    if Lq < 60:
        return
    # one key in the middle: seen by the 50 queries from its place on
    place = lk - Lq + 130
    kept = c.tk[:, place].clone(), c.tv[..., place].clone()
    rows = np.arange(Lq) + lk - Lq
    sees = (rows >= place) & (rows <= place + 49)
    for value in (float("nan"), float("inf")):
        c.tk[:, place], c.tv[..., place] = kept
        c.tv[..., place] = value
        for _ in range(2):  # V alone, then K too
            got, lse = c.run(win, **lens)
            assert np.array_equal(np.isfinite(got).all((0, 2, 3)), ~sees)
            _check(c, win, got, lse, rows=np.nonzero(~sees)[0], **lens)
            c.tk[:, place] = value


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 20, 300])
@pytest.mark.parametrize("scale", [4.0, 12.0])
def test_window_large_logits(dtype, Lq, scale):
    """Logits of some hundreds: the softmax is all but one key, and nothing overflows."""
    c = Case(dtype, 1, 2, 1, Lq, 900, scale=scale)
    win = W(left=400, sink=2)
    got, lse = c.run(win)
    _check(c, win, got, lse)


@gpu
@pytest.mark.parametrize("Lq", [1, 300])
def test_window_log2_queries(Lq):
    """scale = ln 2 takes queries that the norm wrote times log2(e) / sqrt(D)."""
    c = Case(BF16, 2, 4, 2, Lq, 600)
    win = W(left=255, sink=4, scale=math.log(2.0))
    c.q = synth.bf16_round(c.q * np.float32(1.4426950408889634 / math.sqrt(128)))
    c.tq = dev(c.q, BF16)
    got, lse = c.run(win)
    _check(c, win, got, lse)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_window_strides(dtype):
    """Query and output rows inside wider ones, keys inside a longer cache, keys shared by all sequences: the same bits as
    contiguous copies, and nothing else written."""
    import torch
    B, H, Hk, Lq, Lk, D = 3, 4, 2, 90, 150, 128
    win = W(left=70, sink=2)
    c = Case(dtype, B, H, Hk, Lq, Lk)
    want, _ = c.run(win)
    wide = torch.full((B, Lq + 3, H + 2, D), 5.0, dtype=c.tq.dtype, device="cuda")
    qw = wide.clone()
    qw[:, 1:1 + Lq, :H] = c.tq
    cache = torch.full((B, 400, Hk + 1, D), float("nan"), dtype=c.tq.dtype, device="cuda")
    cache[:, 8:8 + Lk, 1:] = c.tk[:, :Lk]
    vc = torch.full((B, Hk, D, 400), float("nan"), dtype=c.tq.dtype, device="cuda")
    vc[..., 16:16 + Lk] = c.tv[..., :Lk]
    q, k, v, out = qw[:, 1:1 + Lq, :H], cache[:, 8:8 + Lk, 1:], vc[..., 16:], wide[:, 1:1 + Lq, :H]
    track.op_attention_window(win, q, k, v, out, workspace=track.attention_window_workspace(win, q, k))
    assert np.array_equal(host(out), want)
    out.fill_(5.0)
    assert bool((wide == 5.0).all())
    ks, vs = c.tk[:1, :Lk].expand(B, -1, -1, -1), c.tv[:1].expand(B, -1, -1, -1)
    shared = torch.empty_like(c.tq)
    track.op_attention_window(win, c.tq, ks, vs, shared, workspace=track.attention_window_workspace(win, c.tq, ks))
    full = torch.empty_like(c.tq)
    kc, vcc = ks.contiguous(), vs.contiguous()
    track.op_attention_window(win, c.tq, kc, vcc, full, workspace=track.attention_window_workspace(win, c.tq, kc))
    assert torch.equal(shared, full)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 3, 90])
def test_window_no_keys(dtype, Lq):
    """Caches without a key yet: zeros, and a log-sum-exp of -inf."""
    import torch
    q = torch.ones(2, Lq, 4, 128, device="cuda").to(track.torch_dtype(dtype))
    k, vt = q.new_empty(2, 0, 2, 128), q.new_empty(2, 2, 128, 0)
    out, lse = torch.full_like(q, 3.0), torch.zeros(2, 4, Lq, device="cuda")
    track.op_attention_window(W(), q, k, vt, out, lse=lse, workspace=track.attention_window_workspace(W(), q, k))
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 70])
def test_sequences_in_turn(dtype, Lq):
    """Rows of the sequences in turn ([tokens, sequences, ..] seen as [sequences, tokens, ..]) for all three operators:
    the same bits as for one sequence after another."""
    import torch
    B, H, Hk, Lk, D = 3, 4, 2, 300, 128
    c = Case(dtype, B, H, Hk, Lq, Lk)
    def turn(t):
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    rope = track.Rope(track.RopeConfig(head_dim=D))
    g = torch.ones(D, dtype=c.tq.dtype, device="cuda")
    pos = torch.arange(B * Lq, dtype=torch.int32, device="cuda").view(1, B, Lq)
    a, b = c.tq.clone(), turn(c.tq)
    track.op_headnorm_rope(rope, a, None, g, None, pos)
    track.op_headnorm_rope(rope, b, None, g, None, pos)
    assert torch.equal(a, b)
    track.op_rope(rope, a, None, pos)
    track.op_rope(rope, b, None, pos)
    assert torch.equal(a, b)
    win = W(left=120, sink=2)
    c.tq.copy_(a)
    want, _ = c.run(win)
    out, k = turn(c.out.clone()), turn(c.tk)[:, :Lk]
    track.op_attention_window(win, b, k, c.tv, out, workspace=track.attention_window_workspace(win, b, k))
    assert np.array_equal(host(out), want)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [4, 300])
def test_window_query_not_finite(dtype, Lq):
    """A query that is not finite gives NaN to its own row alone."""
    c = Case(dtype, 1, 2, 2, Lq, 500)
    win = W(left=77, sink=3)
    c.tq[0, 2, 1, 7] = float("nan")
    got, lse = c.run(win)
    assert np.isnan(got[0, 2, 1]).all() and np.isnan(lse[0, 1, 2])
    rows = np.array([i for i in range(Lq) if i != 2])
    _check(c, win, got, lse, rows=rows)


@gpu
@pytest.mark.parametrize("Lq", [1, 90])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_window_cache_ends_with_its_keys(dtype, Lq):
    """The last V^T row of the last head ends with its keys (rounded up to 16 bytes), the memory behind it is not part
    of any result: the same bits whatever lies there."""
    import torch
    B, H, Hk, D, Lk = 1, 2, 2, 128, 133
    win = W(left=90)
    c = Case(dtype, B, H, Hk, Lq, Lk, cap=136, poison=0.0)
    want, _ = c.run(win)
    n = Hk * D * 136
    flat = torch.full((n + 4096,), float("nan"), dtype=c.tq.dtype, device="cuda")
    flat[:n] = c.tv.reshape(-1)
    c.tv = flat[:n].view(B, Hk, D, 136)
    got, _ = c.run(win)
    assert np.array_equal(got, want)


@gpu
def test_window_f32_unaligned():
    """float32 rows at any 4-byte address."""
    import torch
    B, H, Hk, Lq, Lk, D = 2, 4, 2, 37, 301, 64
    win = W(left=90, sink=3)
    c = Case(F32, B, H, Hk, Lq, Lk, D, cap=301)
    want, _ = c.run(win)
    def odd(t):
        return torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape)
    out = odd(torch.zeros_like(c.out))
    k = odd(c.tk)
    track.op_attention_window(win, odd(c.tq), k, odd(c.tv), out, workspace=track.attention_window_workspace(win, c.tq, k))
    assert np.array_equal(host(out), want)


@gpu
@pytest.mark.parametrize("dtype,H,Lq,Lk", [(BF16, 12, 120, 6000), (F32, 8, 150, 3000)])
def test_window_shares_of_many_rows(dtype, H, Lq, Lk):
    """Rows enough to fill the join by themselves, and shares of the keys all the same; a cut sequence beside a whole one."""
    c = Case(dtype, 1, H, H, Lq, Lk)
    win = W(left=-1, right=-1)
    t = track.DTYPE_BF16 if dtype == BF16 else track.DTYPE_F32
    assert track.attention_window_workspace_bytes(win, t, 1, H, H, 128, Lq, Lk) > 2 * H * Lq * (4 * 128 + 8)
    for lens in ({}, dict(q_len=[Lq - 7], k_len=[Lk // 3 + 1])):
        c.out.fill_(9.0), c.lse.fill_(9.0)
        got, lse = c.run(win, **lens)
        _check(c, win, got, lse, **lens)


@gpu
def test_window_matches_plain_attention():
    """Without limits it is track_op_attention (both within their tolerance of float64)."""
    import torch
    B, H, Lq, Lk, D = 2, 4, 700, 704, 128
    c = Case(BF16, B, H, H, Lq, Lk)
    win = W(left=-1, right=-1)
    got, lse = c.run(win)
    _check(c, win, got, lse)
    plain = torch.empty_like(c.tq)
    track.op_attention(track.DTYPE_BF16, B, H, D, Lq, Lk, c.tq, H * D, c.tk, H * D, c.tv, Lk, plain, H * D)
    want, _, mag, big = ref.attention(c.q, c.k, c.v, -1, -1)
    _close(host(plain), want, 2.1 * _eta(BF16, D, big, Lk) * mag + 1.01 * U[BF16] * np.abs(want), "plain")


@gpu
def test_window_long_cache():
    """A cache of more than 4 GiB: first tokens at its start, a window at its end."""
    import torch
    Hk, D, Lk = 8, 128, 2200000
    k = torch.empty(1, Lk, Hk, D, dtype=torch.bfloat16, device="cuda")
    vt = torch.empty(1, Hk, D, Lk, dtype=torch.bfloat16, device="cuda")
    keep = list(range(4)) + list(range(Lk - 200, Lk))
    rk, rv = normal([61], (1, 204, Hk, D), bf16=True), normal([62], (1, 204, Hk, D), bf16=True)
    k[:, keep] = dev(rk, BF16)
    vt[..., keep] = dev(rv.transpose(0, 2, 3, 1), BF16)
    win = W(left=99, sink=4)
    for Lq, H in ((1, 16), (100, 8)):
        q = normal([63, Lq], (1, Lq, H, D), bf16=True)
        tq = dev(q, BF16)
        out = torch.empty_like(tq)
        track.op_attention_window(win, tq, k, vt, out, workspace=track.attention_window_workspace(win, tq, k))
        want, _, mag, big = ref.attention(q, rk, rv, 99, 0, 4)
        _close(host(out), want, 2.1 * _eta(BF16, D, big, 204) * mag + 1.01 * U[BF16] * np.abs(want), f"Lq {Lq}")


@gpu
@pytest.mark.parametrize("Lq", [1, 200])
def test_window_graph_and_stream(Lq):
    """Captured on a side stream and replayed with new queries, keys, positions and lengths, with eager work between."""
    import torch
    B, H, Hk, Lk, D = 2, 8, 2, 3000, 128
    win = W(left=1500, sink=4)
    c = Case(BF16, B, H, Hk, Lq, Lk)
    k = c.tk[:, :Lk]
    rope = track.Rope(track.RopeConfig(head_dim=D, layout="half"))
    g = dev(normal([71], (D,), bf16=True), BF16)
    pos = torch.zeros(1, B, Lq, dtype=torch.int32, device="cuda")
    k_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    rq = torch.empty_like(c.tq)
    ws = track.attention_window_workspace(win, c.tq, k)

    def step(out):
        track.op_headnorm_rope(rope, c.tq, None, g, None, pos, rq)
        track.op_attention_window(win, rq, k, c.tv, out, k_len=k_len, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(c.out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c.out)
    for i, lens in enumerate(([3000, 1], [2001, 2999], [300, 64], [0, 1024])):
        k_len.copy_(torch.tensor(lens, dtype=torch.int32))
        pos.fill_(1000 * i)
        c.tq.copy_(dev(normal([72, i], (B, Lq, H, D), bf16=True), BF16))
        graph.replay()
        torch.cuda.synchronize()
        got = c.out.clone()
        eager = torch.empty_like(c.out)
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, eager), lens


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_streaming_run(dtype):
    """The three calls as a streaming program uses them: frames arrive in chunks, each chunk's queries and keys are normed
    and rotated (keys into the cache), and attend to the last frames and the first one; then the tokens of one more frame
    come singly, each seeing those of its frame that are there.  The whole frames' result is that of the formulas on the
    whole sequence at once."""
    import torch
    H, Hk, D, group, frames = 4, 2, 128, 48, 9
    total, extra = group * frames, 5
    n = total + extra
    bf = dtype == BF16
    x = normal([81], (1, n, H + 2 * Hk, D), bf16=bf)
    gq, gk = (normal([82, i], (D,), bf16=bf) for i in range(2))
    win = W(left=2, right=0, sink=group, group=group)
    sections = (22, 21, 21)
    rope = track.Rope(track.RopeConfig(head_dim=D, sections=sections))
    t = np.arange(n)
    pos = np.stack([t // group, t % group // 8, t % 8])[:, None].astype(np.int32)
    cap = (n + 63) // 64 * 64
    tx, tp = dev(x, dtype), torch.from_numpy(pos).cuda()
    tgq, tgk = dev(gq, dtype), dev(gk, dtype)
    cache = torch.full((1, cap, Hk, D), float("nan"), dtype=tx.dtype, device="cuda")
    vt = torch.full((1, Hk, D, cap), float("nan"), dtype=tx.dtype, device="cuda")
    out = torch.empty(1, n, H, D, dtype=tx.dtype, device="cuda")
    qr = torch.empty_like(out)
    at = 0
    for step in [group, 3 * group, 2 * group, 3 * group] + [1] * extra:
        s = slice(at, at + step)
        track.op_headnorm_rope(rope, tx[:, s, :H], tx[:, s, H:H + Hk], tgq, tgk, tp[:, :, s].contiguous(), qr[:, s],
                               cache[:, s])
        vt[..., s] = tx[:, s, H + Hk:].permute(0, 2, 3, 1)
        at += step
        k = cache[:, :at]
        track.op_attention_window(win, qr[:, s], k, vt, out[:, s],
                                  workspace=track.attention_window_workspace(win, qr[:, s], k))
    f = ref.freqs(sections)
    q = ref.rope(ref.headnorm(x[:, :, :H], gq, 1e-6), pos, sections, f)
    k = ref.rope(ref.headnorm(x[:, :, H:H + Hk], gk, 1e-6), pos, sections, f)
    # the cache against the formulas, then the attention on what the cache holds
    tol = 1.01 * U[dtype]
    _close(host(qr), q, tol * np.abs(q) + 3e-6 * _pair_len(q, 64, "interleaved"), "q")
    _close(host(cache[:, :n]), k, tol * np.abs(k) + 3e-6 * _pair_len(k, 64, "interleaved"), "k")
    v = x[:, :, H + Hk:]
    for a, b in [(0, total)] + [(i, i + 1) for i in range(total, n)]:
        want, _, mag, big = ref.attention(host(qr)[:, a:b], host(cache)[:, :b], v[:, :b], 2, 0, group, group)
        _close(host(out)[:, a:b], want, 2.1 * _eta(dtype, D, big, b) * mag + 1.01 * U[dtype] * np.abs(want), f"out {a}")


@gpu
@pytest.mark.parametrize("Lq", [1, 40, 500])
def test_two_calls_at_once(Lq):
    """Two streams, each with its outputs and workspace, over one cache, appended to right before: as one after another."""
    import torch
    B, H, Hk, Lk, D = 2, 8, 2, 6000, 128
    win = W(left=-1, right=0, sink=4)
    c = Case(BF16, B, H, Hk, Lq, Lk)
    k = c.tk[:, :Lk]
    qs = [c.tq, c.tq.flip(1).contiguous()]
    rope = track.Rope(track.RopeConfig(head_dim=D))
    pos = torch.arange(Lq, dtype=torch.int32, device="cuda").expand(1, B, Lq).contiguous()
    wss = [track.attention_window_workspace(win, c.tq, k) for _ in qs]

    def call(i, out, rq):
        track.op_rope(rope, qs[i], None, pos, rq)
        return track.op_attention_window(win, rq, k, c.tv, out, workspace=wss[i])

    for turn in range(3):
        k[:, -1] = 0.1 * turn + 1.0  # written on the current stream right before the calls
        want = [call(i, torch.empty_like(c.tq), torch.empty_like(c.tq)) for i in range(2)]
        k[:, -1] = 7.0
        k[:, -1] = 0.1 * turn + 1.0
        outs = [(torch.empty_like(c.tq), torch.empty_like(c.tq)) for _ in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                call(i, *outs[i])
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        for (o, _), w in zip(outs, want):
            assert torch.equal(o, w)


# dtype, H, D, rot, elements a load
COPIED = [(BF16, 3, 128, 64, 8), (BF16, 3, 80, 40, 4), (BF16, 3, 64, 10, 1), (BF16, 2, 250, 66, 1), (F32, 3, 64, 32, 4),
          (F32, 3, 20, 6, 1), (F32, 2, 254, 100, 1)]


@gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("place", ["in place", "out", "norm"])
@pytest.mark.parametrize("case", COPIED, ids=str)
def test_copied_channels(case, place, layout):
    """Channels past rot_dim come out bit for bit, infinities, NaN, -0 and denormals among them, and change no other
    channel's bits; behind the norm an infinity or a NaN stays in its head, and -0 stays -0."""
    import torch
    dtype, H, D, rot, _ = case
    say(f"copied channels {case} {place} {layout}")
    ints = torch.int16 if dtype == BF16 else torch.int32
    Ln = 9
    rope = track.Rope(track.RopeConfig(head_dim=D, rot_dim=rot, sections=(rot // 2,), layout=layout))
    pos = torch.arange(5, 5 + Ln, dtype=torch.int32, device="cuda").view(1, 1, Ln)
    plain = dev(normal([91, D], (1, Ln, H, D), bf16=dtype == BF16), dtype)
    x = plain.clone()
    tiny = 1e-40
    odd = [float("inf"), float("nan"), -float("inf"), -0.0, tiny, -tiny, torch.finfo(x.dtype).max]
    at = [rot, rot + 3, rot + (D - rot) // 2, D - 1]  # in either half of the copied channels
    if place == "norm":
        g = torch.full((D,), 1.25, dtype=x.dtype, device="cuda")
        for i in range(Ln):
            x[0, i, i % H, at[i % 4]] = -0.0
        got, _ = track.op_headnorm_rope(rope, x, None, g, None, pos, torch.empty_like(x))
        zero = x.view(ints) == (-32768 if dtype == BF16 else -2 ** 31)
        assert int(zero.sum()) == Ln and torch.equal(got.view(ints)[zero], x.view(ints)[zero])
        # infinity: the root is infinite, the other channels of the head are 0; NaN: all are NaN
        for value, rest in ((float("inf"), 0.0), (float("nan"), float("nan"))):
            y = plain.clone()
            y[0, 4, 1, rot + 3] = value
            got, _ = track.op_headnorm_rope(rope, y, None, g, None, pos, torch.empty_like(x))
            clean, _ = track.op_headnorm_rope(rope, plain, None, g, None, pos, torch.empty_like(x))
            head = got[0, 4, 1].float()
            assert bool(torch.isnan(head[rot + 3]))
            head = torch.cat([head[:rot + 3], head[rot + 4:]])
            assert bool(torch.isnan(head).all() if math.isnan(rest) else (head == 0).all())
            got[0, 4, 1] = clean[0, 4, 1]
            assert torch.equal(got.view(ints), clean.view(ints))
        return
    for i in range(Ln):
        for h in range(H):
            x[0, i, h, at[(i + h) % 4]] = odd[(i + 2 * h) % len(odd)]
    # a NaN that is not the usual one
    x.view(ints)[0, 0, 0, D - 2] = 0x7fa1 if dtype == BF16 else 0x7fa12345
    want = plain.clone()
    track.op_rope(rope, want, None, pos)
    want[..., rot:] = x[..., rot:]
    want.view(ints)[..., rot:] = x.view(ints)[..., rot:]
    got, _ = track.op_rope(rope, x, None, pos, None if place == "in place" else torch.empty_like(x))
    assert torch.equal(got.view(ints), want.view(ints))


@pytest.mark.parametrize("base,orig,factor", [(256.0, 4096.0, 8.0), (10000.0, 131072.0, 4.0), (10.0, 4096.0, 2.0),
                                              (10000.0, 4096.0, 8.0), (500000.0, 8192.0, 16.0)])
@pytest.mark.parametrize("n", [64, 32, 5])
def test_yarn_one_axis(base, orig, factor, n):
    """The published ramp of one axis: it ends at the pair that makes beta_slow turns over orig_len, also where that is past
    the last pair, and at 2 n - 1 at most.  float64 throughout, some ten roundings."""
    got, _ = track.rope_freqs(track.RopeConfig(head_dim=2 * n, sections=(n,), scaling="yarn", factor=factor, base=base,
                                               orig_len=orig))
    pair = [n * math.log(orig / (turns * 2.0 * math.pi)) / math.log(base) for turns in (32.0, 1.0)]
    low, high = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), 2 * n - 1)
    if (base, orig, n) == (256.0, 4096.0, 64):
        assert high == 75
    if (base, orig, n) == (10000.0, 131072.0, 64):
        assert high == 70
    if base == 10.0:
        assert high == 2 * n - 1
    i = np.arange(n)
    plain = base ** (-i / n)
    ramp = np.clip((i - low) / max(high - low, 0.001), 0.0, 1.0)
    np.testing.assert_allclose(got, plain * (1.0 - ramp) + plain / factor * ramp, rtol=1e-13)


@pytest.mark.parametrize("dtype,B,H,Hk,D,Lq", [
    (BF16, 1, 8, 8, 128, 1), (BF16, 8, 40, 8, 128, 1), (BF16, 64, 8, 1, 128, 1), (BF16, 3, 4, 1, 128, 4), (BF16, 1, 1, 1, 128, 16),
    (F32, 1, 1, 1, 32, 1), (F32, 2, 8, 2, 64, 9), (F32, 1, 4, 4, 128, 40), (F32, 1, 2, 1, 64, 300), (F32, 4, 12, 12, 128, 150),
    (F32, 1, 8, 4, 64, 1501)], ids=str)
@pytest.mark.parametrize("win", [track.Window(), track.Window(left=700, sink=4), track.Window(left=3, right=1, group=64)],
                         ids=lambda w: f"l{w.left}g{w.group}")
def test_workspace_grows_with_the_keys(dtype, B, H, Hk, D, Lq, win):
    """Where a call is refused with less than its size, a size for more keys is enough for fewer (the rest: the next test)."""
    t = track.DTYPE_BF16 if dtype == BF16 else track.DTYPE_F32
    last = 0
    for Lk in [*range(0, 3000, 7), *range(3000, 40000, 97), *range(40000, 400000, 2999)]:
        n = track.attention_window_workspace_bytes(win, t, B, H, Hk, D, Lq, Lk)
        assert n >= last, Lk
        last = n


@gpu
@pytest.mark.parametrize("H,Hk,Lq,Lk,longer", [(12, 12, 200, 512, 576), (40, 8, 60, 510, 576), (2, 1, 200, 3000, 9000)])
def test_workspace_of_more_keys(H, Hk, Lq, Lk, longer):
    """Blocks of rows take the shares that their workspace holds: one made for more keys, less than that, none; the bytes
    behind it stay as they were."""
    import torch
    c = Case(BF16, 1, H, Hk, Lq, Lk)
    win = W(left=-1, right=0, sink=3)
    size = [track.attention_window_workspace_bytes(win, track.DTYPE_BF16, 1, H, Hk, 128, Lq, n) for n in (Lk, longer)]
    assert size[0] > 0
    if longer == 576:
        assert size[1] < size[0]
    share = H * Lq * (4 * 128 + 8)
    for held in sorted({size[0], size[1], size[0] - 1, 2 * share, 2 * share - 1, share, 256, 0}):
        ws = torch.full((held + 4096,), 77, dtype=torch.uint8, device="cuda")
        c.out.fill_(9.0), c.lse.fill_(9.0)
        track.op_attention_window(win, c.tq, c.tk[:, :Lk], c.tv, c.out, lse=c.lse, workspace=ws[:held] if held else None)
        _check(c, win, host(c.out), host(c.lse))
        assert bool((ws[held // share * share if held < size[0] else held:] == 77).all()), held


def test_window_scale_zero():
    """A scale of 0 is not taken for the default one."""
    for scale in (0, 0.0, -0.0):
        with pytest.raises(ValueError, match="scale of 0"):
            W(scale=scale)
    assert W().c().scale == 0.0 and W(scale=0.5).c().scale == 0.5


def _on_cpu():
    """Tensors that op_rope's and op_attention_window's checks accept (but for their device, which is looked at last)."""
    import torch
    B, Ln, Lk, H, Hk, D = 2, 5, 7, 4, 2, 128
    rope = track.Rope(track.RopeConfig(head_dim=D), device="cpu")
    q, k = torch.zeros(B, Ln, H, D), torch.zeros(B, Ln, Hk, D)
    ok = dict(q=q, k=k, q_out=q, k_out=k, pos=torch.zeros(1, B, Ln, dtype=torch.int32), g_q=torch.ones(D), g_k=torch.ones(D))
    win = dict(q=q, k=torch.zeros(B, Lk, Hk, D), vt=torch.zeros(B, Hk, D, 8), out=torch.zeros_like(q), lse=torch.zeros(B, H, Ln),
               q_len=torch.zeros(B, dtype=torch.int32), k_len=torch.zeros(B, dtype=torch.int32),
               q_start=torch.zeros(B, dtype=torch.int32), workspace=torch.zeros(64, dtype=torch.uint8))
    return rope, ok, win


def test_rope_layout_refusals():
    """Each refusal by its own message, behind arguments that are accepted."""
    import torch
    rope, ok, _ = _on_cpu()
    assert rope.check(**ok) == (track.DTYPE_F32, 2, 5, (512, 2560, 512, 2560, 4), (256, 1280, 256, 1280, 2))
    assert rope.check(**dict(ok, k=None, k_out=None, g_q=None, g_k=None))[4] is None
    q, k, pos = ok["q"], ok["k"], ok["pos"]
    for match, kw in (
            (r"^pos: contiguous int32 \(1, 2, 5\)", dict(pos=pos.long())), (r"^pos: contiguous", dict(pos=pos[:, :, :4])),
            (r"^pos: contiguous", dict(pos=pos.expand(3, 2, 5))), (r"^pos: contiguous", dict(pos=pos[0])),
            (r"^pos: contiguous", dict(pos=pos.new_zeros(1, 2, 10)[..., ::2])), (r"^pos: positions are needed", dict(pos=None)),
            (r"^k of shape", dict(k=k[:, :4], k_out=k[:, :4])), (r"^k of shape", dict(k=k[:1], k_out=k[:1])),
            (r"^k: torch.bfloat16 on cpu beside", dict(k=k.bfloat16(), k_out=k.bfloat16())),
            (r"^k: torch.bfloat16 on cpu beside", dict(k_out=k.bfloat16())),
            (r"^q: torch.bfloat16 on cpu beside", dict(q_out=q.bfloat16())),
            (r"^q: output of shape", dict(q_out=q[:, :, :2])), (r"^k: output of shape", dict(k_out=q)),
            (r"^k_out or g_k without k", dict(k=None)), (r"^k_out or g_k without k", dict(k=None, k_out=None)),
            (r"^q: heads of a token must lie side by side", dict(q=q.transpose(1, 2).contiguous().transpose(1, 2))),
            (r"^q: heads of a token must lie side by side", dict(q_out=torch.zeros(2, 5, 4, 256)[..., ::2])),
            (r"^q: \[sequences, tokens, heads, channels\]", dict(q=q[0], q_out=q[0])),
            (r"^q: heads of 64 channels, 128 configured", dict(q=q[..., :64].contiguous(), q_out=q[..., :64].contiguous())),
            (r"^g_q: \[128\]", dict(g_q=torch.ones(64))), (r"^g_k: \[128\]", dict(g_k=torch.ones(256)[::2])),
            (r"^g_q: torch.bfloat16", dict(g_q=torch.ones(128).bfloat16())),
            (r"^float32 or bfloat16", {n: t if n == "pos" else t.half() for n, t in ok.items()})):
        say(f"{match} {list(kw)}")
        with pytest.raises((ValueError, TypeError), match=match):
            rope.check(**dict(ok, **kw))


def test_window_layout_refusals():
    import torch
    _, _, ok = _on_cpu()
    assert track._check_window(**ok) == (track.DTYPE_F32, 2, 4, 2, 128, 5, 7, 512, 2560, 256, 1792, 8, 2048, 512, 2560, 64)
    rest = ("lse", "q_len", "k_len", "q_start", "workspace")
    assert track._check_window(**dict(ok, **dict.fromkeys(rest)))[-1] == 0
    q, k, vt = ok["q"], ok["k"], ok["vt"]
    cases = [
        (r"do not match$", dict(out=ok["out"][:, :4])), (r"do not match$", dict(k=k[:1])),
        (r"do not match$", dict(k=k[..., :64].contiguous())),
        (r"^vt: \[2, 2, 128, >= 7\]", dict(vt=vt[..., :6])), (r"^vt: \[2, 2, 128, >= 7\]", dict(vt=vt[:1])),
        (r"^vt: \[2, 2, 128, >= 7\]", dict(vt=vt[:, :1])), (r"^vt: \[2, 2, 128, >= 7\]", dict(vt=vt[:, :, :64])),
        (r"^vt: \[2, 2, 128, >= 7\]", dict(vt=vt.flatten(1, 2))),
        (r"^vt: rows of keys", dict(vt=torch.zeros(2, 2, 8, 128).transpose(2, 3))),
        (r"^vt: rows of keys", dict(vt=torch.zeros(2, 4, 128, 8)[:, ::2])),
        (r"^vt: torch.bfloat16 on cpu beside", dict(vt=vt.bfloat16())), (r"^k: torch.bfloat16 on", dict(k=k.bfloat16())),
        (r"^out: torch.bfloat16 on", dict(out=q.bfloat16())),
        (r"^k: heads of a token", dict(k=k.transpose(1, 2).contiguous().transpose(1, 2))),
        (r"^out: heads of a token", dict(out=torch.zeros(2, 5, 4, 256)[..., ::2])),
        (r"^lse: contiguous float32 \[2, 4, 5\]", dict(lse=torch.zeros(2, 4, 4))), (r"^lse:", dict(lse=ok["lse"].double())),
        (r"^lse:", dict(lse=torch.zeros(2, 5, 4).transpose(1, 2))),
        (r"^workspace: contiguous", dict(workspace=ok["workspace"][::2])),
        (r"^float32 or bfloat16", dict(q=q.half(), k=k.half(), vt=vt.half(), out=q.half()))]
    for name in ("q_len", "k_len", "q_start"):
        cases += [(rf"^{name}: contiguous int32 \(2,\)", {name: v}) for v in
                  (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32),
                   torch.zeros(4, dtype=torch.int32)[::2])]
    for match, kw in cases:
        say(f"{match} {list(kw)}")
        with pytest.raises((ValueError, TypeError), match=match):
            track._check_window(**dict(ok, **kw))


def test_cpu_tensors_are_refused():
    rope, r, w = _on_cpu()
    with pytest.raises(ValueError, match="^GPU tensors expected"):
        track.op_rope(rope, r["q"], r["k"], r["pos"])
    with pytest.raises(ValueError, match="^GPU tensors expected"):
        track.op_headnorm_rope(rope, r["q"], r["k"], r["g_q"], r["g_k"], r["pos"])
    with pytest.raises(ValueError, match="^GPU tensors expected"):
        track.op_attention_window(W(), **w)


@gpu
def test_tensors_on_other_devices_are_refused():
    """Each tensor in turn on the CPU beside the others on the GPU; nothing is launched."""
    import torch
    _, r, w = _on_cpu()
    r, w = ({n: t.cuda() for n, t in d.items()} for d in (r, w))
    rope = track.Rope(track.RopeConfig(head_dim=128))
    rope.check(**r), track._check_window(**w)
    for check, args in ((rope.check, r), (track._check_window, w)):
        for n in args:
            with pytest.raises((ValueError, TypeError), match="cuda:0"):
                check(**dict(args, **{n: args[n].cpu()}))
    with pytest.raises(ValueError, match="rope on cpu, q on cuda:0"):
        track.op_rope(track.Rope(track.RopeConfig(head_dim=128), device="cpu"), r["q"], r["k"], r["pos"])


def test_rope_freqs_failed_call_writes_nothing(L):
    out, amp = np.full(64, 3.0), ctypes.c_float(5.0)
    p = out.ctypes.data_as(ctypes.POINTER(ctypes.c_double))
    for bad in (dict(sections=(63,)), dict(base=1.0), dict(rot_dim=130, sections=(65,)), dict(scaling="yarn", factor=0.5)):
        assert L.track_rope_freqs(ctypes.byref(_rope_c(**bad)), p, ctypes.byref(amp)) != 0
        assert np.all(out == 3.0) and amp.value == 5.0
    assert L.track_rope_freqs(ctypes.byref(_rope_c()), p, None) == track.E_INVALID and np.all(out == 3.0)
    assert L.track_rope_freqs(ctypes.byref(_rope_c()), p, ctypes.byref(amp)) == 0 and out[0] == 1.0 and amp.value == 1.0


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq,Lk,shares", [(1, 200, False), (1, 6000, True), (4, 6000, True), (70, 300, False), (70, 4000, True),
                                          (300, 451, None)])  # bfloat16 alone takes shares
def test_window_lengths_out_of_range(dtype, Lq, Lk, shares):
    """Lengths and positions in device memory that are out of range are cut to it, in the kernels and in the join: the
    results of the cut ones bit for bit, rows behind them left as they were."""
    import torch
    c = Case(dtype, 3, 4, 2, Lq, Lk)
    win = W(left=-1, right=0, sink=3)
    t = track.DTYPE_BF16 if dtype == BF16 else track.DTYPE_F32
    assert (track.attention_window_workspace_bytes(win, t, 3, 4, 2, 128, Lq, Lk) > 0) == (dtype == BF16 if shares is None else shares)
    big = 2 ** 31 - 1
    lens = [(dict(q_len=[Lq + 5, -3, big], k_len=[Lk + 100, Lk, -1]), dict(q_len=[Lq, 0, Lq], k_len=[Lk, Lk, 0])),
            (dict(q_len=[-big - 1, 1, Lq], k_len=[big, -big - 1, Lk + 1]), dict(q_len=[0, 1, Lq], k_len=[Lk, 0, Lk])),
            (dict(q_start=[big, -big - 1, Lk - Lq]), dict(q_start=[1 << 28, -(1 << 28), Lk - Lq]))]
    for raw, cut in lens:
        c.out.fill_(9.0), c.lse.fill_(9.0)
        got, lse = c.run(win, **raw)
        _check(c, win, got, lse, **cut)
        c.out.fill_(9.0), c.lse.fill_(9.0)
        want, wlse = c.run(win, **cut)
        assert np.array_equal(got, want) and np.array_equal(lse, wlse)


@gpu
@pytest.mark.parametrize("H,Hk,Lq,Lk,lens", [
    (8, 2, 1, 5000, {}), (8, 2, 1, 100003, dict(k_len=[100003, 56000, 17])), (4, 4, 4, 3001, dict(k_len=[3001, 2944, 2945])),
    (4, 2, 20, 5000, {}), (2, 1, 200, 9000, dict(k_len=[9000, 8999, 4097])), (12, 12, 120, 6000, {}),
    (3, 3, 700, 1500, dict(q_len=[700, 511, 1])), (2, 2, 40, 32000, {})], ids=str)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("win", [W(), W(left=1000, sink=70), W(left=3, right=2, group=100, sink=130)],
                         ids=lambda w: f"l{w.left}g{w.group}")
def test_window_counts_each_key_once(dtype, H, Hk, Lq, Lk, lens, win):
    """Queries of zero weigh every key 1, exactly in either type: the log-sum-exp is the log of the keys' number, and V that
    is 1 in one key in 64 (another one for each channel, so every key counts somewhere) gives an exact count over it.
    Sums of whole numbers below 2^24 are exact in any order, so what is left is the logarithm (a unit in the last place, 2^-23),
    its factor and their product (2^-24 each) for lse, and a division and the output's rounding for out: one key too many or too few of 100003 is 1e-5 in the former."""
    import torch
    B, D = 3, 128
    say(f"count {dtype} {H} {Lq} {Lk} {lens} {win}")
    dt = track.torch_dtype(dtype)
    q = torch.zeros(B, Lq, H, D, dtype=dt, device="cuda")
    k = torch.randn(B, Lk, Hk, D, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(dt)
    cap = (Lk + 7) // 8 * 8
    hit = (torch.arange(cap, device="cuda")[None, :] - torch.arange(D, device="cuda")[:, None]) % 64 == 0
    vt = hit.to(dt).expand(B, Hk, D, cap).contiguous()
    out, lse = torch.full_like(q, 9.0), torch.full((B, H, Lq), 9.0, device="cuda")
    dl = {n: torch.tensor(v, dtype=torch.int32, device="cuda") for n, v in lens.items()}
    ws = track.attention_window_workspace(win, q, k)
    track.op_attention_window(win, q, k, vt, out, lse=lse, workspace=ws, **dl)
    got, glse = host(out), host(lse)
    hits = hit[:, :Lk].cpu().numpy().astype(np.float64)  # [D, Lk]
    for b in range(B):
        lq, lk = (lens[n][b] if n in lens else full for n, full in (("q_len", Lq), ("k_len", Lk)))
        seen = np.stack([ref.seen(lk - lq + i, lk, win.left, win.right, win.sink, win.group) for i in range(lq)])
        n = seen.sum(1)
        want = np.where(n[:, None] > 0, (seen @ hits[:, :lk].T) / np.maximum(n, 1)[:, None], 0.0)
        wlse = np.log(np.maximum(n, 1))
        for h in range(H):
            _close(got[b, :lq, h], want, (U[dtype] + 2.0 ** -22) * want, f"out {b} {h}")
            some = n > 0
            _close(glse[b, h, :lq][some], wlse[some], 1.01 * 2.0 ** -22 * wlse[some] + 1e-30, f"lse {b} {h}")
            assert np.all(glse[b, h, :lq][~some] == -np.inf)


@gpu
@pytest.mark.parametrize("B", [15, 16, 40])
@pytest.mark.parametrize("Lq,Lk", [(1, 200), (1, 6000), (3, 1100)])
def test_window_keys_of_many_sequences(B, Lq, Lk):
    """Keys that many sequences share (sequence strides of 0), of ragged lengths: the bits of a copy for each."""
    import torch
    H, Hk, D = 8, 2, 128
    win = W(left=4000, sink=3)
    c = Case(BF16, 1, H, Hk, Lq, Lk)
    q = dev(normal([97, B], (B, Lq, H, D), bf16=True), BF16)
    k_len = torch.tensor([Lk - (b * 37) % Lk for b in range(B)], dtype=torch.int32, device="cuda")
    got = []
    for copies in (False, True):
        k, vt = c.tk[:, :Lk].expand(B, -1, -1, -1), c.tv.expand(B, -1, -1, -1)
        if copies:
            k, vt = k.contiguous(), vt.contiguous()
        out, lse = torch.full_like(q, 9.0), torch.full((B, H, Lq), 9.0, device="cuda")
        ws = track.attention_window_workspace(win, q, k)
        got.append((track.op_attention_window(win, q, k, vt, out, lse=lse, k_len=k_len, workspace=ws), lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert bool(torch.isfinite(got[0][0]).all())


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 20, 300])
@pytest.mark.parametrize("scale", [1.0, 4.0])
def test_window_large_values(dtype, Lq, scale):
    """V up to the documented 2^63 / Lk (5.5 sigma of it) under logits that the weights' reference lags behind: finite, and
    a power of two times the result of V itself."""
    c = Case(dtype, 1, 2, 1, Lq, 900, scale=scale)
    win = W(left=400, sink=2)
    want, _ = c.run(win)
    big = 2.0 ** 50
    assert np.abs(c.v).max() * big < 2.0 ** 63 / 900
    c.tv *= big
    got, _ = c.run(win)
    assert np.array_equal(got, want * np.float32(big))

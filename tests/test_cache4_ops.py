"""The 4-bit paged cache: rows in and out against its definition, byte for byte, and attention on it against the formula in
float64.

Tolerances (u = eps / 2 of the output type): rotation and rounding on the way in are float64, so codes and exponents are
those of the definition but where a rotated value lies within some 1e-13 of a border, which seeded values do not.  The way
out is exact.  Attention: weights off by a relative eta give |do| <= 2 eta sum w|v| (numerator and denominator); eta is
the logit's error ((D + 2) float32 roundings of sum |scale q k|; the cached keys and values are exact in bfloat16), 2^-21 for exp2 and its
argument, the rounding to bfloat16 where the weights take one, and the float32 sums over the keys.
"""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

import cache4_reference as c4
import window_reference as ref
from gpu_helpers import dev, host, normal, say
from paper_2609_30096_amd import synth, track

F32, BF16 = synth.F32, synth.BF16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
W = track.Window
gpu = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_30096_amd", "csrc")


@pytest.fixture
def L():
    return track.lib()


def _close(got, want, tol, what):
    err = np.abs(np.asarray(got, np.float64) - want)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.nanmax(err / np.maximum(tol, 1e-300)):.3g} x"


# ---------------------------------------------------------------- on the host
@pytest.fixture(scope="module")
def program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("cache4") / "cache4_layout")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-include", "initializer_list", "-I", CSRC, "-o", exe,
                    os.path.join(HERE, "cache4_layout.cpp")], check=True)
    return exe


def test_every_thread_takes_its_bytes_of_the_layout(program):
    """All loads of all kernels lie inside their 64 tokens of a head, and page ids out of range are no pages."""
    r = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def test_a_thread_one_byte_off_is_found(program):
    r = subprocess.run([program, "planted"], capture_output=True, text=True, timeout=60)
    assert r.returncode == 1 and "few rows K code: 37" in r.stdout


def test_reference_rounding():
    """The definition on values that can be counted by hand: ties to even codes, the exponent's border at 7, zeros."""
    x = np.zeros((1, 64))
    x[0, :9] = [6.0, 0.25, 0.75, -1.25, 1.75, 2.5, 3.5, -5.0, 0.2500001]
    x[0, 32:35] = [7.0, 0.5, 1.0]
    code, byte = c4.quantise(x)
    assert list(byte[0]) == [127, 128]
    assert list(code[0, :9]) == [7, 0, 2, 8 + 2, 4, 4, 6, 8 + 6, 1]
    assert list(code[0, 32:35]) == [6, 0, 1]  # 3.5, 0.25, 0.5 of 2
    assert list(c4.quantise(np.zeros((1, 32)))[1][0]) == [3]
    assert list(c4.quantise(np.full((1, 32), np.inf))[1][0]) == [255]
    assert list(c4.quantise(np.full((1, 32), 3.38e38))[1][0]) == [252]


def test_page_bytes(L):
    assert L.track_cache4_page_bytes(8, 128, 64) == 8 * 8704 and L.track_cache4_page_bytes(3, 32, 192) == 3 * 3 * 2176
    assert L.track_cache4_page_bytes(1 << 19, 128, 65536) == (1 << 29) * 8704
    for bad in ((0, 128, 64), (-1, 128, 64), (1, 96, 64), (1, 0, 64), (1, 128, 0), (1, 128, 63), (1, 128, 96), (1, 128, 65600),
                ((1 << 19) + 1, 128, 64)):
        assert L.track_cache4_page_bytes(*bad) == 0, bad
        with pytest.raises(ValueError):
            track.cache4_page_bytes(*bad)


P = 1 << 20  # aligned stand-in; never dereferenced


def _cache_c(**kw):
    a = dict(pages=P, n_pages=100, page_tokens=64, heads=4, head_dim=128, table_pages=20, table=P, ld_table=20)
    a.update(kw)
    return track.Cache4C(*[a[n] for n in ("pages", "n_pages", "page_tokens", "heads", "head_dim", "table_pages", "table",
                                          "ld_table")])


BAD_CACHES = [(track.E_UNSUPPORTED, kw) for kw in (dict(page_tokens=0), dict(page_tokens=32), dict(page_tokens=100),
                                                   dict(page_tokens=-64), dict(page_tokens=131072), dict(heads=0),
                                                   dict(heads=(1 << 19) + 1), dict(head_dim=96), dict(head_dim=256))] + \
    [(track.E_SHAPE, kw) for kw in (dict(n_pages=0), dict(n_pages=1 << 31), dict(table_pages=-1), dict(ld_table=-1), dict(table_pages=(1 << 22) + 1, ld_table=1 << 30),
                                    dict(table_pages=1 << 30, page_tokens=65536, ld_table=1 << 30))] + \
    [(track.E_INVALID, kw) for kw in (dict(pages=0), dict(table=0), dict(pages=P + 64), dict(table=P + 2))]


def test_rows_refusals(L):
    E, F, S, I = track.DTYPE_BF16, track.DTYPE_F32, track.E_SHAPE, track.E_INVALID
    base = dict(B=2, Ln=10, k=P, ldk=512, sk=5120, v=P, ldv=512, sv=5120, start=P, n=None, pos=None, freqs=None, amp=1.0)

    def append(dtype=E, cache=None, rope=None, **kw):
        a = dict(base, **kw)
        c = _cache_c() if cache is None else cache
        return L.track_op_cache4_append(dtype, c, rope, a["B"], a["Ln"], a["k"], a["ldk"], a["sk"], a["v"], a["ldv"],
                                        a["sv"], a["start"], a["n"], a["pos"], a["freqs"], a["amp"], None)

    def read(dtype=E, cache=None, **kw):
        a = dict(base, **kw)
        c = _cache_c() if cache is None else cache
        return L.track_op_cache4_read(dtype, c, a["B"], a["Ln"], a["k"], a["ldk"], a["sk"], a["v"], a["ldv"], a["sv"],
                                      a["start"], a["n"], None)

    for call in (append, read):
        assert call(dtype=2) == I and call(dtype=-1) == I
        for want, kw in BAD_CACHES:
            assert call(cache=_cache_c(**kw)) == want, kw
        assert call(B=-1) == S and call(Ln=-1) == S and call(Ln=(1 << 28) + 1, sk=1 << 50, sv=1 << 50) == S
        assert call(ldk=511) == S and call(ldv=511) == S and call(sk=-1) == S and call(sv=-1) == S
        for name in ("k", "v", "start"):
            assert call(**{name: None}) == I, name
            assert call(**{name: P + 1}) == I, name
        assert call(F, k=P + 2) == I and call(n=P + 2) == I
        assert call(B=1 << 16, Ln=1 << 16, sk=1 << 26, sv=1 << 26) == S  # more blocks than a launch holds
        assert call(B=0) == 0 and call(Ln=0) == 0
    assert L.track_op_cache4_append(E, None, None, 1, 1, *([P, 512, 512] * 2), P, None, None, None, 1.0, None) == I
    assert L.track_op_cache4_read(E, None, 1, 1, *([P, 512, 512] * 2), P, None, None) == I
    assert read(sk=512 * 9 + 511) == S and read(sv=100) == S  # sequences overlap in the output
    rope = track.RopeConfig(head_dim=128).c()
    ok = dict(rope=rope, pos=P, freqs=P)
    assert append(**dict(ok, pos=None)) == I and append(**dict(ok, freqs=None)) == I
    assert append(**dict(ok, pos=P + 2)) == I and append(**dict(ok, freqs=P + 4)) == I
    assert append(**ok, amp=math.nan) == I and append(**ok, amp=math.inf) == I
    assert append(**dict(ok, rope=track.RopeConfig(head_dim=64).c())) == S
    bad = track.RopeConfig(head_dim=128).c()
    bad.layout = 2
    assert append(**dict(ok, rope=bad)) == I
    bad = track.RopeConfig(head_dim=128, sections=(10,)).c()
    assert append(**dict(ok, rope=bad)) == S


def test_attention_refusals(L):
    E, F, S, I, N, Un = (track.DTYPE_BF16, track.DTYPE_F32, track.E_SHAPE, track.E_INVALID, track.E_NOMEM,
                         track.E_UNSUPPORTED)
    base = dict(B=2, H=8, Lq=1, Lk=1280, q=P, ldq=1024, sq=1024, out=P, ldo=1024, so=1024, lse=None, q_len=None,
                k_len=None, q_start=None, ws=P, ws_bytes=1 << 40)

    def call(dtype=E, win=None, cache=None, **kw):
        a = dict(base, **kw)
        w, c = W() if win is None else win, _cache_c() if cache is None else cache
        return L.track_op_attention_cache4(dtype, w.c(), c, a["B"], a["H"], a["Lq"], a["Lk"], a["q"], a["ldq"], a["sq"],
                                           a["out"], a["ldo"], a["so"], a["lse"], a["q_len"], a["k_len"], a["q_start"],
                                           a["ws"], a["ws_bytes"], None)

    assert call(dtype=2) == I
    assert L.track_op_attention_cache4(E, None, _cache_c(), 1, 4, 1, 1, *([P, 512, 512] * 2), *([None] * 5), 0, None) == I
    assert L.track_op_attention_cache4(E, W().c(), None, 1, 4, 1, 1, *([P, 512, 512] * 2), *([None] * 5), 0, None) == I
    for want, kw in BAD_CACHES:
        assert call(cache=_cache_c(**kw)) == want, kw
    for w in (W(group=0), W(sink=-1), W(left=-2), W(right=-2), W(scale=-1.0), W(scale=math.nan), W(scale=1e31)):
        assert call(win=w) == I, w
    for w in (W(group=1 << 31), W(sink=1 << 31), W(left=1 << 31), W(right=1 << 31)):
        assert call(win=w) == S, w
    assert call(B=-1) == S and call(H=0) == S and call(H=6) == S and call(Lq=-1) == S and call(Lk=-1) == S
    assert call(Lk=1281) == S and call(Lq=1 << 30) == S
    assert b"places" in L.track_last_error() or call(Lk=1281) == S and b"places" in L.track_last_error()
    assert call(cache=_cache_c(head_dim=64), ldq=512) == Un
    for name in ("q", "out"):
        assert call(**{name: None}) == I and call(**{name: P + 8}) == I and call(F, **{name: P + 2}) == I, name
    assert call(ldq=1016) == S and call(ldo=1016) == S and call(ldq=1028) == I and call(sq=1028) == I
    assert call(sq=-8) == S and call(so=512) == S and call(Lq=3, so=3 * 1024 - 8) == S
    for name in ("lse", "q_len", "k_len", "q_start"):
        assert call(**{name: P + 2}) == I, name
    need = track.attention_cache4_workspace_bytes(W(), E, 2, 8, 4, 128, 1, 1280)
    assert need > 0
    assert call(ws=None) == N and call(ws_bytes=need - 1) == N and call(ws=P + 128) == I
    assert call(B=0) == 0 and call(Lq=0) == 0
    assert L.track_attention_cache4_workspace_bytes(E, None, 1, 1, 1, 128, 1, 1) == -1
    with pytest.raises(track.TrackError):
        track.attention_cache4_workspace_bytes(W(), E, 1, 3, 2, 128, 1, 1)
    for B, H in ((1 << 30, 1 << 30), (1 << 23, 1), (1 << 12, 1 << 11)):
        assert L.track_attention_cache4_workspace_bytes(E, W().c(), B, H, H, 128, 1 << 28, 64) == -1, (B, H)


@pytest.mark.parametrize("dtype,B,H,Hk,D,Lq", [
    (BF16, 1, 8, 8, 128, 1), (BF16, 8, 40, 8, 128, 1), (BF16, 64, 8, 1, 128, 1), (BF16, 3, 4, 1, 128, 4),
    (F32, 1, 1, 1, 32, 1), (F32, 2, 8, 2, 64, 9), (F32, 1, 4, 4, 128, 40), (F32, 4, 12, 12, 128, 150)], ids=str)
@pytest.mark.parametrize("win", [W(), W(left=700, sink=4), W(left=3, right=1, group=64)], ids=lambda w: f"l{w.left}g{w.group}")
def test_workspace_grows_with_the_keys(dtype, B, H, Hk, D, Lq, win):
    t = track.DTYPE_BF16 if dtype == BF16 else track.DTYPE_F32
    last = 0
    for Lk in [*range(0, 3000, 7), *range(3000, 40000, 97), *range(40000, 400000, 2999)]:
        n = track.attention_cache4_workspace_bytes(win, t, B, H, Hk, D, Lq, Lk)
        assert n >= last, Lk
        last = n


def test_no_sequences(L):
    """A call of no sequences does nothing: its table is empty, and an empty tensor's address is null."""
    import torch
    none = _cache_c(table=0)
    for dtype in (track.DTYPE_BF16, track.DTYPE_F32):
        assert L.track_op_cache4_append(dtype, none, None, 0, 5, *([P, 512, 2560] * 2), None, None, None, None, 1.0, None) == 0
        assert L.track_op_cache4_read(dtype, none, 0, 5, *([P, 512, 2560] * 2), None, None, None) == 0
        assert L.track_op_attention_cache4(dtype, W().c(), none, 0, 8, 2, 1280, None, 1024, 2048, None, 1024, 2048, *([None] * 5),
                                           0, None) == 0
        # one sequence has places, and they are in the table
        assert L.track_op_cache4_append(dtype, none, None, 1, 5, *([P, 512, 2560] * 2), P, None, None, None, 1.0,
                                        None) == track.E_INVALID
        assert L.track_op_cache4_read(dtype, none, 1, 5, *([P, 512, 2560] * 2), P, None, None) == track.E_INVALID
        assert L.track_op_attention_cache4(dtype, W().c(), none, 1, 8, 2, 1280, P, 1024, 2048, P, 1024, 2048, *([None] * 4), P,
                                           1 << 40, None) == track.E_INVALID
    cache = track.Cache4(4, 128, 64, torch.zeros(0, 20, dtype=torch.int32), n_pages=2)
    assert cache.c.table is None and cache.tokens == 1280


def _on_cpu():
    import torch
    B, Ln, Hk, D = 2, 5, 2, 128
    table = torch.zeros(B, 3, dtype=torch.int32)
    cache = track.Cache4(Hk, D, 64, table, n_pages=4)
    k = torch.zeros(B, Ln, Hk, D)
    return cache, k, k.clone(), torch.zeros(B, dtype=torch.int32)


def test_binding_refusals():
    import torch
    cache, k, v, start = _on_cpu()
    assert cache.tokens == 192 and cache.pages.shape == (4, 2 * 8704)
    assert cache._rows(k, v, start, None, None, None) == (track.DTYPE_F32, 2, 5, 256, 1280, 256, 1280)
    ok = dict(k=k, v=v, start=start, n=None, pos=None, freqs=None)
    for match, kw in (("^k .*heads of 128$", dict(v=v[:, :4])), ("^k .*heads of 128$", dict(k=k[:1], v=v[:1])),
                      ("^k .*heads of 128$", dict(k=k[:, :, :1], v=v[:, :, :1])),
                      ("^k .*heads of 128$", dict(k=k[..., :64].contiguous(), v=v[..., :64].contiguous())),
                      ("^v: torch.bfloat16", dict(v=v.bfloat16())), ("^start: contiguous int32", dict(start=start.long())),
                      ("^start: contiguous int32", dict(start=start[:1])), ("^start: the first place", dict(start=None)),
                      ("^n: contiguous int32", dict(n=start.float())), (r"^k: \[sequences", dict(k=k[0], v=v[0])),
                      ("^v: heads of a token", dict(v=v.transpose(1, 2).contiguous().transpose(1, 2))),
                      ("^float32 or bfloat16", dict(k=k.half(), v=v.half()))):
        with pytest.raises((ValueError, TypeError), match=match):
            cache._rows(**dict(ok, **kw))
    rope = track.Rope(track.RopeConfig(head_dim=128), device="cpu")
    pos = torch.zeros(1, 2, 5, dtype=torch.int32)
    with pytest.raises(ValueError, match="come together"):
        track.op_cache4_append(cache, k, v, start, rope=rope)
    with pytest.raises(ValueError, match="come together"):
        track.op_cache4_append(cache, k, v, start, pos=pos)
    with pytest.raises(ValueError, match="^pos: contiguous int32"):
        track.op_cache4_append(cache, k, v, start, rope=rope, pos=pos[:, :, :4])
    for call in (lambda: track.op_cache4_append(cache, k, v, start, rope=rope, pos=pos),
                 lambda: track.op_cache4_read(cache, k, v, start),
                 lambda: track.op_attention_cache4(W(), cache, k, v)):
        with pytest.raises(ValueError, match="^GPU tensors expected"):
            call()
    q, out = torch.zeros(2, 1, 4, 128), torch.zeros(2, 1, 4, 128)
    assert cache._queries(q, out, None, None, None, None, None) == (track.DTYPE_F32, 2, 4, 1, 512, 512, 512, 512, 0)
    for match, kw in (("^q .*heads of 128$", dict(out=out[:1])), ("^q .*heads of 128$", dict(q=q[:1], out=out[:1])),
                      ("^out: torch.bfloat16", dict(out=out.bfloat16())), ("^lse", dict(lse=torch.zeros(2, 4))),
                      ("^k_len", dict(k_len=torch.zeros(2)))):
        with pytest.raises((ValueError, TypeError), match=match):
            cache._queries(**dict(dict(q=q, out=out, lse=None, q_len=None, k_len=None, q_start=None, workspace=None), **kw))
    table = cache.table
    for name in ("pages", "table"):  # their addresses are the cache's
        with pytest.raises(AttributeError):
            setattr(cache, name, None)
    assert track.Cache4(2, 128, 64, table[:1].expand(3, -1), n_pages=4).c.ld_table == 0
    for kw in (dict(table=table.long()), dict(table=table[0]), dict(table=torch.zeros(2, 6, dtype=torch.int32)[:, ::2]),
               dict(n_pages=None), dict(pages=cache.pages[:, 1:]), dict(pages=cache.pages.int()), dict(pages=cache.pages, n_pages=3),
               dict(head_dim=80), dict(page_tokens=100)):
        with pytest.raises(ValueError):
            track.Cache4(**dict(dict(heads=2, head_dim=128, page_tokens=64, table=table, n_pages=4), **kw))


# ---------------------------------------------------------------- rows in and out
def _pool(key, n_pages, heads, D, page, B, each):
    """Pages of random bytes on the host, a table without order."""
    rng = np.random.default_rng(key)
    pool = c4.Pool(n_pages, heads, D, page, 0)
    pool.raw[:] = rng.integers(0, 256, pool.raw.shape, dtype=np.uint8)
    table = rng.permutation(n_pages)[:B * each].reshape(B, each).astype(np.int32)
    return pool, table


def _device_cache(pool, table):
    import torch
    return track.Cache4(pool.heads, pool.D, pool.P, torch.from_numpy(table).cuda(),
                        torch.from_numpy(pool.raw.reshape(len(pool.raw), -1)).cuda())


ROWS = [
    # dtype, B, L, heads, D, page, start, n, sections, layout
    (BF16, 1, 1, 1, 128, 64, [0], None, (), ""),
    (BF16, 3, 1, 8, 128, 64, [63, 64, 100], None, (64,), "half"),
    (BF16, 2, 16, 2, 128, 64, [0, 40], None, (64,), "interleaved"),
    (BF16, 2, 200, 3, 128, 128, [5, 70], [200, 131], (22, 21, 21), "interleaved"),
    (BF16, 2, 128, 2, 128, 64, [64, 0], None, (32,), "half"),
    (BF16, 1, 70, 2, 64, 192, [3], None, (5,), "half"),          # pairs that are not whole units
    (BF16, 1, 70, 2, 64, 64, [33], None, (9,), "interleaved"),
    (BF16, 2, 33, 3, 32, 64, [31, 32], [33, 0], (16,), "half"),
    (F32, 2, 1, 4, 64, 64, [17, 0], None, (32,), "interleaved"),
    (F32, 2, 130, 2, 128, 64, [1, 63], [130, 2], (64,), "half"),
    (F32, 1, 300, 1, 32, 256, [200], None, (6, 5, 5), "interleaved"),
    (F32, 1, 65, 5, 64, 64, [64], None, (10,), "half"),
    (F32, 1, 65, 2, 128, 128, [64], None, (), ""),
    # places that the cache does not have
    (BF16, 3, 100, 2, 128, 64, [-50, 180, -200], None, (64,), "half"),
    (F32, 3, 20, 2, 64, 64, [2 ** 31 - 1, -2 ** 31, 250], [20, 20, 2 ** 31 - 1], (), ""),
]


def _rows_inputs(case, key=3):
    dtype, B, Ln, heads, D, page, start, n, sections, layout = case
    bf = dtype == BF16
    k, v = (normal([key, i], (B, Ln, heads, D), bf16=bf) for i in range(2))
    rng = np.random.default_rng(key)
    k *= 2.0 ** rng.integers(-8, 9, (B, Ln, heads, 1))
    pos = rng.integers(-200000, 200001, (max(len(sections), 1), B, Ln)).astype(np.int32)
    rope = track.Rope(track.RopeConfig(head_dim=D, rot_dim=2 * sum(sections), layout=layout, sections=sections)) if sections else None
    return k, v, pos, rope


@gpu
@pytest.mark.parametrize("case", ROWS, ids=str)
def test_append(case):
    """Every byte of the pool against the definition: what is appended, and that nothing else changes."""
    import torch
    dtype, B, Ln, heads, D, page, start, n, sections, layout = case
    say(f"append {case}")
    k, v, pos, rope = _rows_inputs(case)
    each = 512 // page + 1 if page > 64 else 4
    pool, table = _pool(7, B * each + 2, heads, D, page, B, each)
    table[0, -1] = len(pool.raw)      # no page: one past the pool, and a negative id
    if B > 1:
        table[1, 0] = -1
    cache = _device_cache(pool, table)
    tk, tv = dev(k, dtype), dev(v, dtype)
    ts = torch.tensor(start, dtype=torch.int32, device="cuda")
    tn = None if n is None else torch.tensor(n, dtype=torch.int32, device="cuda")
    track.op_cache4_append(cache, tk, tv, ts, n=tn, rope=rope, pos=torch.from_numpy(pos).cuda() if rope else None)
    rk = k.astype(np.float64)
    if sections:
        rk = ref.rope(rk, pos, sections, ref.freqs(sections), 1.0, layout)
    qk, qv = c4.quantise(rk), c4.quantise(v.astype(np.float64))
    for b in range(B):
        for i in range(Ln if n is None else min(n[b], Ln)):
            x = start[b] + i
            if 0 <= x < each * page and 0 <= table[b, x // page] < len(pool.raw):
                pool.put(table[b, x // page], x % page, (qk[0][b, i], qk[1][b, i]), (qv[0][b, i], qv[1][b, i]))
    got = cache.pages.cpu().numpy().reshape(pool.raw.shape)
    bad = got != pool.raw
    assert not bad.any(), f"{bad.sum()} bytes, first {np.argwhere(bad)[:3].tolist()}"


ROTATED = [
    # dtype, B, L, heads, D, start, sections, layout, scaling, factor
    (BF16, 2, 70, 2, 128, [3, 60], (64,), "half", "yarn", 8.0),
    (BF16, 16, 1, 3, 128, list(range(40, 56)), (64,), "half", "yarn", 32.0),
    (BF16, 1, 40, 3, 128, [100], (20,), "interleaved", "yarn", 4.0),        # channels that are not turned
    (BF16, 1, 65, 2, 64, [33], (8,), "half", "yarn", 4.0),
    (BF16, 1, 50, 2, 64, [0], (11,), "half", "yarn", 4.0),                  # pairs that are not whole units
    (BF16, 1, 65, 2, 128, [0], (32, 16, 16), "half", "none", 1.0),
    (BF16, 2, 33, 2, 128, [1, 64], (22, 21, 21), "half", "yarn", 8.0),      # axes that end inside a unit
    (BF16, 1, 40, 5, 32, [30], (4, 2, 2), "half", "linear", 4.0),
    (BF16, 1, 40, 2, 128, [30], (7, 8), "interleaved", "ntk", 8.0),
    (F32, 1, 50, 2, 64, [20], (7, 6, 5), "half", "none", 1.0),
    (F32, 2, 40, 2, 64, [0, 63], (12, 10, 10), "half", "yarn", 8.0),
    (F32, 1, 70, 1, 128, [64], (64,), "interleaved", "yarn", 16.0),
    (F32, 1, 40, 2, 128, [10], (30,), "half", "linear", 4.0),
    (F32, 1, 40, 3, 64, [10], (32,), "interleaved", "ntk", 8.0),
    (F32, 1, 40, 2, 32, [10], (6, 5, 5), "half", "yarn", 2.0),
]


@gpu
@pytest.mark.parametrize("case", ROTATED, ids=str)
def test_append_amplitudes_and_axes(case):
    """Frequencies of every scaling, amplitudes other than one, and axes in halves: every byte against the definition, which
    gives other bytes without the amplitude, without the scaling, and with an axis ending a pair early."""
    import torch
    dtype, B, Ln, heads, D, start, sections, layout, scaling, factor = case
    say(f"append {case}")
    k, v, pos, _ = _rows_inputs((dtype, B, Ln, heads, D, 64, start, None, (), ""), key=17)
    pos = np.random.default_rng(18).integers(-3000, 3001, (len(sections), B, Ln)).astype(np.int32)
    rope = track.Rope(track.RopeConfig(head_dim=D, rot_dim=2 * sum(sections), layout=layout, sections=sections, scaling=scaling,
                                       factor=factor))
    amp = 1.0 + 0.1 * math.log(factor) if scaling == "yarn" else 1.0
    assert rope.amplitude == pytest.approx(amp, rel=2.0 ** -23)
    f = ref.freqs(sections, scaling=scaling, factor=factor)
    pool, table = _pool(19, B * 4, heads, D, 64, B, 4)
    cache = _device_cache(pool, table)
    track.op_cache4_append(cache, dev(k, dtype), dev(v, dtype), torch.tensor(start, dtype=torch.int32, device="cuda"), rope=rope,
                           pos=torch.from_numpy(pos).cuda())

    def want(sections, f, amp):
        return c4.quantise(ref.rope(k.astype(np.float64), pos, sections, f, amp, layout))

    qk, qv = want(sections, f, rope.amplitude), c4.quantise(v.astype(np.float64))
    others = [(sections, ref.freqs(sections), rope.amplitude)] if scaling != "none" else []
    if amp != 1.0:
        others.append((sections, f, 1.0))
    if len(sections) > 1:
        others.append(((sections[0] - 1, sections[1] + 1, *sections[2:]), f, rope.amplitude))
    for other in others:
        assert (want(*other)[0] != qk[0]).any(), other
    for b in range(B):
        for i in range(Ln):
            x = start[b] + i
            pool.put(table[b, x // 64], x % 64, (qk[0][b, i], qk[1][b, i]), (qv[0][b, i], qv[1][b, i]))
    bad = cache.pages.cpu().numpy().reshape(pool.raw.shape) != pool.raw
    assert not bad.any(), f"{bad.sum()} bytes, first {np.argwhere(bad)[:3].tolist()}"


@gpu
@pytest.mark.parametrize("case", ROWS, ids=str)
def test_read(case):
    """Pages of random bytes, every exponent among them, exactly; rows behind the last as they were, missing places zero."""
    import torch
    dtype, B, Ln, heads, D, page, start, n, sections, layout = case
    say(f"read {case}")
    each = 512 // page + 1 if page > 64 else 4
    pool, table = _pool(8, B * each + 2, heads, D, page, B, each)
    table[0, -1] = 2 ** 31 - 1
    if B > 1:
        table[1, 0] = -2 ** 31
    cache = _device_cache(pool, table)
    dt = track.torch_dtype(dtype)
    k, v = (torch.full((B, Ln, heads, D), 9.0, dtype=dt, device="cuda") for _ in range(2))
    ts = torch.tensor(start, dtype=torch.int32, device="cuda")
    tn = None if n is None else torch.tensor(n, dtype=torch.int32, device="cuda")
    got = track.op_cache4_read(cache, k, v, ts, n=tn)
    assert got[0] is k and got[1] is v
    want = np.full((2, B, Ln, heads, D), 9.0)
    for b in range(B):
        for i in range(Ln if n is None else min(n[b], Ln)):
            x = start[b] + i
            want[:, b, i] = 0.0
            if 0 <= x < each * page and 0 <= table[b, x // page] < len(pool.raw):
                want[:, b, i] = pool.get(table[b, x // page], x % page)
    with np.errstate(over="ignore"):
        for name, x, w in (("k", k, want[0]), ("v", v, want[1])):
            np.testing.assert_array_equal(host(x), w.astype(np.float32), name)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rotated", [False, True])
def test_append_special_values(dtype, rotated):
    """Ties, the exponent's border, zeros of both signs, denormals, the largest values, infinities and NaN, in keys and values."""
    import torch
    D, heads, Ln = 64, 2, 40
    dt = track.torch_dtype(dtype)
    x = normal([21], (1, Ln, heads, D), bf16=True).astype(np.float32)
    x[0, 0] = 0.0
    x[0, 1] = -0.0
    x[0, 2, 0, :8] = [6.0, 0.25, 0.75, -1.25, 1.75, 2.5, 3.5, -5.0]
    x[0, 3, 0, :3] = [7.0, 6.96875, -7.0]
    for i, big in enumerate((3.3e38, 2.9e38, 1e-38, 1e-40, 2.0 ** -126, 2.0 ** -125, 6 * 2.0 ** -124, 3.5 * 2.0 ** -124)):
        x[0, 4 + i, 0] *= big / np.abs(x[0, 4 + i, 0]).max()
    x[0, 20, 1, 5] = np.nan
    x[0, 21, 0, 40] = np.inf
    x[0, 22, 0, 31] = -np.inf
    x = torch.from_numpy(x).to(dt)
    h = x.float().numpy().astype(np.float64)
    pool, table = _pool(9, 3, heads, D, 64, 1, 2)
    cache = _device_cache(pool, table)
    rope = track.Rope(track.RopeConfig(head_dim=D, rot_dim=32)) if rotated else None
    pos = torch.zeros(1, 1, Ln, dtype=torch.int32, device="cuda") if rotated else None  # by angle 0: the bits of the values
    track.op_cache4_append(cache, x.cuda(), x.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"), rope=rope, pos=pos)
    code, byte = c4.quantise(h)
    kcode = code.copy()
    if rotated:  # x c - y s with s = 0: the sign of a zero is that of the sum, and inf x 0 is NaN
        with np.errstate(invalid="ignore"):
            r = ref.rope(h, np.zeros((1, 1, Ln), np.int32), (16,), ref.freqs((16,)))
        kcode, kbyte = c4.quantise(r)
        assert np.array_equal(kbyte, byte)
    for i in range(Ln):
        pool.put(table[0, 0], i, (kcode[0, i], byte[0, i]), (code[0, i], byte[0, i]))
    got = cache.pages.cpu().numpy().reshape(pool.raw.shape)
    bad = got != pool.raw
    assert not bad.any(), f"{bad.sum()} bytes, first {np.argwhere(bad)[:3].tolist()}"


def _beside_borders(layout):
    """Float32 keys [1, L, 1, 64] whose rotation lies beside a border of two codes (or, at 7, of two exponents), but rounds to it
    in float32: the rows, positions, and where."""
    Ln, D = 192, 64
    rng = np.random.default_rng(77)
    pos = rng.integers(0, 500, (1, 1, Ln)).astype(np.int32)  # (angles within 2^-43: the rotations within 2^-40)
    f = ref.freqs((D // 2,))
    turn = pos[0, 0][:, None] * f
    c, s = np.cos(turn), np.sin(turn)
    first = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], (Ln, D // 2)) * rng.choice([-1.0, 1.0], (Ln, D // 2))
    first[:, 0::16] = 6.5            # the groups' largest
    first[::3, 0::16] = 7.0
    second = rng.uniform(-1.0, 1.0, first.shape)
    x, z = (first * c + second * s).astype(np.float32), (-first * s + second * c).astype(np.float32)
    # the operand with the smaller factor in small steps, to the first sum that float32 rounds to the border
    fine = np.abs(s) <= np.abs(c)    # z, or x
    hit = np.zeros(first.shape, bool)
    for k in range(-400, 401):
        x1 = np.where(fine, x, x + np.float32(k) * np.spacing(np.abs(x))).astype(np.float32)
        z1 = np.where(fine, z + np.float32(k) * np.spacing(np.abs(z)), z).astype(np.float32)
        r = x1.astype(np.float64) * c - z1.astype(np.float64) * s
        ok = ~hit & (r.astype(np.float32) == first) & (np.abs(r - first) > 2.0 ** -36) & (rng.random(hit.shape) < 0.2)
        x, z, hit = np.where(ok, x1, x), np.where(ok, z1, z), hit | ok
    rows = np.empty((1, Ln, 1, D), np.float32)
    lo, hi = (slice(0, D, 2), slice(1, D, 2)) if layout == "interleaved" else (slice(0, D // 2), slice(D // 2, D))
    rows[0, :, 0, lo], rows[0, :, 0, hi] = x, z
    where = np.zeros((Ln, D), bool)
    where[:, lo] = hit
    return rows, pos, where


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_rows_beside_borders_are_there(layout):
    rows, pos, where = _beside_borders(layout)
    r = ref.rope(rows.astype(np.float64), pos, (32,), ref.freqs((32,)), 1.0, layout)
    once, twice = c4.quantise(r), c4.quantise(r.astype(np.float32).astype(np.float64))
    assert (once[0][0, :, 0] != twice[0][0, :, 0])[where].sum() > 200, "codes that a rounding to float32 first would change"
    assert (once[1] != twice[1]).sum() > 8, "exponents"


@gpu
@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_keys_beside_borders(layout):
    import torch
    rows, pos, _ = _beside_borders(layout)
    Ln, D = rows.shape[1], rows.shape[3]
    rope = track.Rope(track.RopeConfig(head_dim=D, rot_dim=D, layout=layout))
    pool, table = _pool(13, 4, 1, D, 64, 1, 3)
    cache = _device_cache(pool, table)
    k = torch.from_numpy(rows).cuda()
    track.op_cache4_append(cache, k, k, torch.zeros(1, dtype=torch.int32, device="cuda"), rope=rope, pos=torch.from_numpy(pos).cuda())
    qk = c4.quantise(ref.rope(rows.astype(np.float64), pos, (32,), ref.freqs((32,)), 1.0, layout))
    qv = c4.quantise(rows.astype(np.float64))
    for i in range(Ln):
        pool.put(table[0, i // 64], i % 64, (qk[0][0, i], qk[1][0, i]), (qv[0][0, i], qv[1][0, i]))
    bad = cache.pages.cpu().numpy().reshape(pool.raw.shape) != pool.raw
    assert not bad.any(), f"{bad.sum()} bytes, first {np.argwhere(bad)[:3].tolist()}"


@gpu
def test_values_beside_borders():
    """Float32 values one and two steps beside every border, at groups of every exponent, as they are."""
    import torch
    border = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    step = np.spacing(border)
    group = np.concatenate([border + i * step for i in (0, 1, -1, 2, -2)])[:31]
    tops = [np.float32(x) for x in (6.0, np.nextafter(np.float32(7.0), np.float32(0.0)), 7.0, 4.0)]
    x = np.stack([np.append(group * (-1) ** (j + np.arange(31)), tops[j % 4]) for j in range(249)])
    x = (x * 2.0 ** np.arange(-124.0, 125.0)[:, None]).astype(np.float32).reshape(1, 249, 1, 32)
    pool, table = _pool(15, 6, 1, 32, 64, 1, 4)
    cache = _device_cache(pool, table)
    t = torch.from_numpy(x).cuda()
    track.op_cache4_append(cache, t, -t, torch.zeros(1, dtype=torch.int32, device="cuda"))
    qk, qv = c4.quantise(x.astype(np.float64)), c4.quantise(-x.astype(np.float64))
    for i in range(249):
        pool.put(table[0, i // 64], i % 64, (qk[0][0, i], qk[1][0, i]), (qv[0][0, i], qv[1][0, i]))
    bad = cache.pages.cpu().numpy().reshape(pool.raw.shape) != pool.raw
    assert not bad.any(), f"{bad.sum()} bytes, first {np.argwhere(bad)[:3].tolist()}"


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_strides(dtype):
    """Rows of a fused projection, rows at unaligned addresses and sequences in turn: the bytes of contiguous ones, and read back
    into such rows the values of contiguous ones, with nothing else written."""
    import torch
    B, Ln, heads, D = 2, 90, 3, 64
    bf = dtype == BF16
    x = dev(normal([31], (B, Ln, 4 * heads, D), bf16=bf), dtype)
    k, v = x[:, :, heads:2 * heads], x[:, :, 2 * heads:3 * heads]
    start = torch.tensor([10, 33], dtype=torch.int32, device="cuda")
    rope = track.Rope(track.RopeConfig(head_dim=D, layout="half"))
    pos = torch.arange(B * Ln, dtype=torch.int32, device="cuda").view(1, B, Ln)
    pool, table = _pool(10, 6, heads, D, 128, B, 2)

    def put(k, v):
        cache = _device_cache(pool, table)
        track.op_cache4_append(cache, k, v, start, rope=rope, pos=pos)
        return cache

    def odd(t):
        return torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape)

    def turn(t):
        return t.transpose(0, 1).contiguous().transpose(0, 1)

    want = put(k.contiguous(), v.contiguous())
    for a, b in ((k, v), (odd(k.contiguous()), odd(v.contiguous())), (turn(k), turn(v))):
        assert torch.equal(put(a, b).pages, want.pages)
    rk, rv = torch.empty_like(k.contiguous()), torch.empty_like(k.contiguous())
    track.op_cache4_read(want, rk, rv, start)
    wide = torch.full_like(x, 5.0)
    track.op_cache4_read(want, wide[:, :, heads:2 * heads], wide[:, :, 2 * heads:3 * heads], start)
    assert torch.equal(wide[:, :, heads:2 * heads], rk) and torch.equal(wide[:, :, 2 * heads:3 * heads], rv)
    assert bool((wide[:, :, :heads] == 5).all()) and bool((wide[:, :, 3 * heads:] == 5).all())
    for make in (odd, turn):
        a, b = make(torch.zeros_like(rk)), make(torch.zeros_like(rk))
        track.op_cache4_read(want, a, b, start)
        assert torch.equal(a, rk) and torch.equal(b, rv)


@gpu
def test_append_in_pieces():
    """The bytes of one append, for tokens that arrive in pieces of any length."""
    import torch
    B, Ln, heads, D = 2, 300, 2, 128
    k, v = (dev(normal([41, i], (B, Ln, heads, D), bf16=True), BF16) for i in range(2))
    pool, table = _pool(11, 12, heads, D, 64, B, 6)
    pool.raw[:] = 0
    rope = track.Rope(track.RopeConfig(head_dim=D, sections=(22, 21, 21)))
    pos = torch.randint(0, 5000, (3, B, Ln), dtype=torch.int32, device="cuda")
    first = torch.tensor([7, 30], dtype=torch.int32, device="cuda")
    whole, parts = _device_cache(pool, table), _device_cache(pool, table)
    track.op_cache4_append(whole, k, v, first, rope=rope, pos=pos)
    at = 0
    for step in (1, 1, 3, 64, 50, 100, 17, 1, 62, 1):
        s = slice(at, at + step)
        track.op_cache4_append(parts, k[:, s], v[:, s], first + at, rope=rope, pos=pos[:, :, s].contiguous())
        at += step
    assert at == Ln and torch.equal(whole.pages, parts.pages)


# ---------------------------------------------------------------- attention
class Case:
    """Seeded queries and a filled cache of one call, on the host and the device."""

    def __init__(self, dtype, B, H, Hk, Lq, Lk, D=128, page=64, key=51, scale=1.0, missing=()):
        import torch
        self.dtype, self.Lk, self.D, self.B = dtype, Lk, D, B
        each = -(-max(Lk, 1) // page)
        self.pool, self.table = _pool(key, B * each + 1, Hk, D, page, B, each)
        # exponents of ordinary values; what lies past the last key stays random, 255 among it
        rng = np.random.default_rng(key + 1)
        q = self.pool.raw.reshape(len(self.pool.raw), -1, Hk, 68 * D)
        self.q = normal([key, 1], (B, Lq, H, D), scale, dtype == BF16)
        for b in range(B):
            for x in range(Lk):
                at = self.pool._at(x % page % 64)
                block = self.pool.raw[self.table[b, x // page], x % page // 64]
                block[:, at[2]] = rng.integers(124, 128, (Hk, D // 32))
                block[:, at[3]] = rng.integers(124, 128, (Hk, D // 32))
        for b, p, page_id in missing:
            self.table[b, p] = page_id
        self.k, self.v, self.there = self.pool.places(self.table, Lk)
        self.cache = _device_cache(self.pool, self.table)
        self.tq = dev(self.q, dtype)
        self.out = torch.full((B, Lq, H, D), 9.0, dtype=self.tq.dtype, device="cuda")
        self.lse = torch.full((B, H, Lq), 9.0, device="cuda")

    def run(self, win, **lens):
        import torch
        kw = {n: torch.tensor(v, dtype=torch.int32, device="cuda") for n, v in lens.items() if v is not None}
        ws = track.attention_cache4_workspace(win, self.cache, self.tq, self.Lk)
        track.op_attention_cache4(win, self.cache, self.tq, self.out, Lk=self.Lk, lse=self.lse, workspace=ws, **kw)
        return host(self.out), host(self.lse)


def _eta(dtype, D, big, Lk):
    return (D + 2) * 2.0 ** -24 * big + 2.0 ** -21 + (Lk + 16) * 2.0 ** -24 + (U[BF16] if dtype == BF16 else 0.0)


def _check(c, win, got, lse, rows=None, **lens):
    scale = 1.0 / math.sqrt(c.D) if win.scale is None else win.scale
    want, wlse, mag, big = c4.attention(c.q.astype(np.float64), c.k, c.v, c.there,
                                        lambda p, n: ref.seen(p, n, win.left, win.right, win.sink, win.group), scale, **lens)
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


ATTN = [
    # B, H, Hk, Lq, Lk, page, window, lengths
    (1, 1, 1, 1, 1, 64, W(), {}),
    (1, 4, 4, 1, 7, 64, W(left=2), {}),
    (2, 8, 2, 1, 200, 64, W(left=63, sink=4), {}),
    (3, 10, 2, 1, 1000, 192, W(left=99, sink=70), dict(k_len=[1000, 1, 517])),
    (2, 5, 1, 1, 3000, 64, W(), dict(k_len=[3000, 2048])),                     # shares of the keys
    (1, 20, 4, 1, 5000, 1024, W(left=1023, sink=4), {}),
    (2, 4, 1, 4, 300, 64, W(left=40, sink=3), dict(q_len=[4, 2], k_len=[300, 155])),
    (2, 4, 2, 13, 777, 128, W(left=100), {}),
    (1, 6, 2, 16, 130, 64, W(), {}),
    (1, 2, 2, 300, 300, 64, W(left=0), {}),
    (1, 2, 2, 300, 300, 64, W(left=0, right=-1, sink=0), {}),
    (2, 4, 2, 300, 451, 64, W(left=63, sink=5), dict(q_len=[300, 211], k_len=[451, 213])),
    (1, 2, 1, 700, 700, 128, W(left=64, sink=64), {}),
    (1, 3, 3, 640, 960, 64, W(left=1, right=2, group=100, sink=30), {}),
    (2, 2, 2, 500, 500, 192, W(left=-1, right=-1), {}),
    (2, 2, 2, 500, 333, 64, W(left=5), {}),                                    # the first 167 queries see nothing
    (1, 2, 2, 80, 400, 64, W(left=10), dict(q_start=[1000])),                  # the window is past the last key
    (3, 2, 1, 100, 256, 64, W(left=20), dict(q_len=[0, 100, 50], k_len=[256, 0, 256])),
    (1, 1, 1, 70, 4000, 64, W(), {}),                                          # shares of the keys, blocks
    (1, 2, 1, 100, 300, 64, W(left=1 << 28, right=1 << 28, group=1 << 28, sink=1 << 28), {}),
    (3, 2, 1, 20, 300, 64, W(left=100, right=0, sink=7), dict(q_start=[-(1 << 28), 1 << 28, 290])),
    (3, 4, 2, 1, 300, 64, W(), dict(k_len=[2 ** 31 - 1, -5, 64])),
]
KINDS = [(BF16, 128), (F32, 32), (F32, 64), (F32, 128)]


@gpu
@pytest.mark.parametrize("dtype,D", KINDS)
@pytest.mark.parametrize("case", ATTN, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}_{c[3]}x{c[4]}_p{c[5]}l{c[6].left}r{c[6].right}s{c[6].sink}g{c[6].group}{'v' if c[7] else ''}")
def test_attention(dtype, D, case):
    B, H, Hk, Lq, Lk, page, win, lens = case
    say(f"cache attention {dtype} D={D} {case}")
    c = Case(dtype, B, H, Hk, Lq, Lk, D, page)
    got, lse = c.run(win, **lens)
    cut = {n: [min(max(x, 0), Lk) if n == "k_len" else x for x in v] for n, v in lens.items()}
    _check(c, win, got, lse, **cut)
    again, lse2 = c.run(win, **lens)
    assert np.array_equal(got, again) and np.array_equal(lse, lse2)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq,Lk", [(1, 500), (1, 6000), (5, 700), (200, 900)])
def test_missing_pages(dtype, Lq, Lk):
    """Pages that are not there hide their keys, those of a whole sequence too."""
    each = -(-Lk // 64)
    missing = [(0, 0, -1), (0, 2, 1 << 30), (0, each - 1, -2 ** 31)] + [(1, p, -1) for p in range(each)] + [(2, 1, -7)]
    c = Case(dtype, 3, 4, 2, Lq, Lk, missing=missing)
    for win in (W(), W(left=-1, right=-1), W(left=150, sink=70)):
        got, lse = c.run(win)
        _check(c, win, got, lse)
        assert np.all(got[1] == 0.0) and np.all(lse[1] == -np.inf)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq,Lk", [(1, 500), (1, 6000), (6, 700), (200, 900), (400, 1200)])
def test_groups_without_a_number(dtype, Lq, Lk):
    """A NaN group of V reaches the group's channels of the rows that see the key and nothing else; one of K those rows
    whole."""
    win = W(left=49, sink=3)
    c = Case(dtype, 1, 4, 2, Lq, Lk)
    rows = np.arange(Lq) + Lk - Lq

    def put(x, part, group, byte):
        block = c.pool.raw[c.table[0, x // 64], 0]
        block[:, c.pool._at(x % 64)[part][group]] = byte
        c.cache.pages[c.table[0, x // 64]] = dev_bytes(c.pool.raw[c.table[0, x // 64]])

    def dev_bytes(a):
        import torch
        return torch.from_numpy(a.reshape(-1).copy()).cuda()

    clean, clse = c.run(win)
    clean, clse = clean.copy(), clse.copy()
    first = max(Lk - Lq - 49, 3)
    for x in {3, first - 1} - {2}:       # keys that no row sees
        for part in (2, 3):
            put(x, part, 1, 255)
        got, lse = c.run(win)
        assert np.array_equal(got, clean) and np.array_equal(lse, clse)
    for x in sorted({0, Lk - 1, Lk - 1 - Lq // 2, max(Lk - Lq, 3)}):
        sees = (rows >= x) & ((rows <= x + 49) | (x < 3))
        put(x, 3, 2, 255)                # V: channels 64..95
        got, lse = c.run(win)
        nan = np.zeros(got.shape, bool)
        nan[0, sees, :, 64:96] = True
        assert np.array_equal(np.isnan(got), nan), x
        np.testing.assert_allclose(got[~nan], clean[~nan], rtol=2 * U[dtype], atol=1e-6)
        assert np.array_equal(lse, clse)
        put(x, 3, 2, 125)
        put(x, 2, 0, 255)                # K
        got, lse = c.run(win)
        assert np.array_equal(np.isnan(got).all((0, 2, 3)), sees) and np.array_equal(np.isnan(got).any((0, 2, 3)), sees), x
        put(x, 2, 0, 125)
        clean, clse = (t.copy() for t in c.run(win))


@gpu
@pytest.mark.parametrize("D,H,Lq,Lk", [(128, 12, 700, 1100), (64, 20, 840, 1090)])
def test_more_row_blocks_than_places(D, H, Lq, Lk):
    """Float32 row blocks that fill the chip's places once and a little take shares of the keys."""
    win = W()
    c = Case(F32, 1, H, H, Lq, Lk, D=D)
    assert track.attention_cache4_workspace(win, c.cache, c.tq, Lk) is not None
    got, lse = c.run(win)
    _check(c, win, got, lse)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 4, 100])
def test_a_weight_that_falls_to_zero(dtype, Lq):
    """A NaN group of V whose key is seen reaches the rows, though the key's weight is below every float32, in a tile that
    all rows see whole and in one at the end."""
    import torch
    c = Case(dtype, 1, 4, 2, Lq, 230)
    c.tq = c.tq.abs()
    rows = np.arange(Lq) + 230 - Lq
    for x in (70, 229, 230 - Lq):
        page = c.table[0, x // 64]
        block = c.pool.raw[page, 0]
        at = c.pool._at(x % 64)
        kept = block.copy()
        block[:, at[0]] = 0xff           # -6 2^4 in every channel: logits below -500
        block[:, at[2]] = 131
        block[:, at[3][1]] = 255         # V: channels 32..63
        c.cache.pages[page] = torch.from_numpy(c.pool.raw[page].reshape(-1).copy()).cuda()
        got, _ = c.run(W())
        nan = np.zeros(got.shape, bool)
        nan[0, rows >= x, :, 32:64] = True
        assert np.array_equal(np.isnan(got), nan), x
        block[:] = kept
        c.cache.pages[page] = torch.from_numpy(c.pool.raw[page].reshape(-1).copy()).cuda()


@gpu
@pytest.mark.parametrize("dtype,D", KINDS)
@pytest.mark.parametrize("Lq", [1, 7, 300])
def test_every_exponent(dtype, D, Lq):
    """Each query sees its own place only, whose groups have exponents of their own over a hundred octaves: the output is that
    place's value (its weight over itself: exact in bfloat16, three roundings off in float32), the lse its logit.  A query has
    channels of one group only, of a size that brings the logit near one."""
    import torch
    B, Hk, H, Lk, G = 2, 2, 4, 330, D // 32
    rng = np.random.default_rng(23)
    pool, table = _pool(23, B * 6, Hk, D, 64, B, 6)
    ke, ve = rng.integers(60, 191, (B, Lk, Hk, G)), rng.integers(60, 166, (B, Lk, Hk, G))
    for b in range(B):
        for x in range(Lk):
            at = pool._at(x % 64)
            block = pool.raw[table[b, x // 64], 0]
            block[:, at[2]], block[:, at[3]] = ke[b, x], ve[b, x]
    k, v, _ = pool.places(table, Lk)
    cache = _device_cache(pool, table)
    win = W(left=0, right=0)
    base = normal([23, 2], (B, Lq, H, D), bf16=dtype == BF16)
    u = U[dtype]
    for start in range(0, Lk - Lq + 1, Lq if Lq > 1 else 5):
        rows = np.arange(start, start + Lq)
        q = np.zeros((B, Lq, H, D), np.float32)
        for h in range(H):
            g = (rows + h) % G
            for i in range(Lq):
                at = slice(32 * g[i], 32 * g[i] + 32)
                q[:, i, h, at] = base[:, i, h, at] * 2.0 ** (127.0 - ke[:, rows[i], h // 2, g[i], None])
        tq = dev(q, dtype)
        out, lse = torch.empty_like(tq), torch.empty(B, H, Lq, device="cuda")
        ws = track.attention_cache4_workspace(win, cache, tq, Lk)
        track.op_attention_cache4(win, cache, tq, out, Lk=Lk, lse=lse, workspace=ws,
                                  q_start=torch.full((B,), start, dtype=torch.int32, device="cuda"))
        kk, vv = (np.repeat(t[:, rows], 2, axis=2) for t in (k, v))
        x, mag = ((a * b).sum(-1).transpose(0, 2, 1) / math.sqrt(D) for a, b in ((q.astype(np.float64), kk), (np.abs(q).astype(np.float64), np.abs(kk))))
        _close(host(out), vv, (0.0 if dtype == BF16 else 4 * u) * np.abs(vv), f"out {start}")
        # (D + 2 roundings of the logit, those of exp2, log2 and the weight)
        _close(host(lse), x, (D + 2) * 2.0 ** -24 * mag + 2.0 ** -20 + 2.0 ** -22 * np.abs(x) + (u if dtype == BF16 else 0.0), f"lse {start}")


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 4, 100, 300])
def test_places_that_no_query_sees(dtype, Lq):
    """Between the first tokens and the window the pages hold what no append has written: any codes and any exponent bytes,
    whose values pass the largest number too.  No query sees those places, and nothing of them reaches one."""
    import torch
    Lk, sink, left = 900, 5, 210
    c = Case(dtype, 2, 4, 2, Lq, Lk)
    rng = np.random.default_rng(5)
    lo = Lk - Lq - left  # the first query's first
    unseen = np.arange(sink, lo)
    assert len(unseen) > 300 and lo % 64 and sink % 64  # (in tiles that are seen in part as well)
    for b in range(2):
        for x in unseen:
            at = c.pool._at(x % 64)
            block = c.pool.raw[c.table[b, x // 64], 0]
            for i in range(2):
                block[:, at[i]] = rng.choice([0x77, 0xff, 0x00, 0x61], (2, 64))
                block[:, at[2 + i]] = rng.choice([0, 2, 127, 252, 253, 254, 255], (2, 4))
    c.cache.pages.copy_(torch.from_numpy(c.pool.raw.reshape(len(c.pool.raw), -1)))
    c.k, c.v, c.there = c.pool.places(c.table, Lk)
    win = W(left=left, sink=sink)
    got, lse = c.run(win)
    _check(c, win, got, lse)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 4, 100, 300])
def test_places_that_some_queries_see(dtype, Lq):
    """Exponent bytes that no append writes, in keys that the later queries see: the earlier ones have what they would have
    without."""
    import torch
    Lk = 500
    first = Lk - Lq
    c = Case(dtype, 1, 4, 2, Lq, Lk)
    odd = sorted({min(x, Lk - 1) for x in (first + max(1, Lq // 3), first + Lq // 2 + 1, Lk - 1)})
    for i, x in enumerate(odd):
        at = c.pool._at(x % 64)
        block = c.pool.raw[c.table[0, x // 64], 0]
        block[:, at[1]] = 0x77           # 6 in every channel
        block[:, at[3][i % 4]] = 253 + i % 2
    c.cache.pages.copy_(torch.from_numpy(c.pool.raw.reshape(len(c.pool.raw), -1)))
    win = W(left=300)
    got, lse = c.run(win)
    clean = first + np.arange(Lq) < odd[0]
    assert clean.any() == (Lq > 1)
    _check(c, win, got, lse, rows=clean)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 20, 300])
@pytest.mark.parametrize("scale", [4.0, 12.0])
def test_large_logits(dtype, Lq, scale):
    c = Case(dtype, 1, 2, 1, Lq, 900, scale=scale)
    win = W(left=400, sink=2)
    got, lse = c.run(win)
    _check(c, win, got, lse)


@gpu
@pytest.mark.parametrize("Lq", [1, 300])
def test_log2_queries(Lq):
    c = Case(BF16, 2, 4, 2, Lq, 600)
    win = W(left=255, sink=4, scale=math.log(2.0))
    c.q = synth.bf16_round(c.q * np.float32(1.4426950408889634 / math.sqrt(128)))
    c.tq = dev(c.q, BF16)
    got, lse = c.run(win)
    _check(c, win, got, lse)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 90])
def test_attention_strides(dtype, Lq):
    """Queries and outputs inside wider rows, sequences in turn, a table inside a wider one, float32 rows at any 4-byte
    address, sequences that share their pages: the bits of contiguous ones, and nothing else written."""
    import torch
    B, H, Hk, Lk, D = 3, 4, 2, 150, 128
    win = W(left=70, sink=2)
    c = Case(dtype, B, H, Hk, Lq, Lk)
    want, _ = c.run(win)
    wide = torch.full((B, Lq + 3, H + 2, D), 5.0, dtype=c.tq.dtype, device="cuda")
    qw = wide.clone()
    qw[:, 1:1 + Lq, :H] = c.tq
    out = wide[:, 1:1 + Lq, :H]
    tw = torch.full((B, 9), -1, dtype=torch.int32, device="cuda")
    tw[:, 2:2 + c.table.shape[1]] = torch.from_numpy(c.table).cuda()
    cache = track.Cache4(Hk, D, 64, tw[:, 2:2 + c.table.shape[1]], c.cache.pages)
    track.op_attention_cache4(win, cache, qw[:, 1:1 + Lq, :H], out, Lk=Lk, workspace=track.attention_cache4_workspace(win, cache, c.tq, Lk))
    assert np.array_equal(host(out), want)
    out.fill_(5.0)
    assert bool((wide == 5.0).all())

    def turn(t):
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    out = turn(torch.zeros_like(c.out))
    track.op_attention_cache4(win, cache, turn(c.tq), out, Lk=Lk, workspace=track.attention_cache4_workspace(win, cache, c.tq, Lk))
    assert np.array_equal(host(out), want)
    if dtype == F32:
        def odd(t):
            return torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape)
        out = odd(torch.zeros_like(c.out))
        track.op_attention_cache4(win, cache, odd(c.tq), out, Lk=Lk, workspace=track.attention_cache4_workspace(win, cache, c.tq, Lk))
        assert np.array_equal(host(out), want)
    c.table[:] = c.table[0]
    one = track.Cache4(Hk, D, 64, c.cache.table[:1].expand(B, -1), c.cache.pages)  # one row of the table for all
    shared = torch.zeros_like(c.out)
    track.op_attention_cache4(win, one, c.tq, shared, Lk=Lk, workspace=track.attention_cache4_workspace(win, one, c.tq, Lk))
    c.cache.table.copy_(torch.from_numpy(c.table))
    c.k[:], c.v[:] = c.k[0], c.v[0]
    got, lse = c.run(win)
    _check(c, win, got, lse)
    assert np.array_equal(host(shared), got)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 90])
def test_no_keys(dtype, Lq):
    import torch
    cache = track.Cache4(2, 128, 64, torch.zeros(2, 0, dtype=torch.int32, device="cuda"), n_pages=1)
    q = torch.ones(2, Lq, 4, 128, device="cuda").to(track.torch_dtype(dtype))
    out, lse = torch.full_like(q, 3.0), torch.zeros(2, 4, Lq, device="cuda")
    track.op_attention_cache4(W(), cache, q, out, lse=lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@gpu
@pytest.mark.parametrize("H,Hk,Lq,Lk,longer", [(12, 12, 200, 512, 576), (2, 1, 200, 3000, 9000)])
def test_workspace_of_more_keys(H, Hk, Lq, Lk, longer):
    """Blocks of rows take the shares that their workspace holds; the bytes behind it stay as they were."""
    import torch
    c = Case(BF16, 1, H, Hk, Lq, Lk)
    win = W(left=-1, right=0, sink=3)
    size = [track.attention_cache4_workspace_bytes(win, track.DTYPE_BF16, 1, H, Hk, 128, Lq, n) for n in (Lk, longer)]
    assert size[0] > 0
    share = H * Lq * (4 * 128 + 8)
    for held in sorted({size[0], size[1], size[0] - 1, 2 * share, share, 256, 0}):
        ws = torch.full((held + 4096,), 77, dtype=torch.uint8, device="cuda")
        c.out.fill_(9.0), c.lse.fill_(9.0)
        track.op_attention_cache4(win, c.cache, c.tq, c.out, Lk=Lk, lse=c.lse, workspace=ws[:held] if held else None)
        _check(c, win, host(c.out), host(c.lse))
        assert bool((ws[held // share * share if held < size[0] else held:] == 77).all()), held


@gpu
@pytest.mark.parametrize("page,place", [(64, 0), (1024, 200)])
def test_pool_past_32_bits(page, place):
    """Pages whose offsets pass 32 bits, in a pool of more than 4 GiB, and table rows as far apart."""
    import torch
    heads, D, Ln = 8, 128, 130
    size = track.cache4_page_bytes(heads, D, page)
    n = (5 << 30) // size
    pages = torch.empty(n, size, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[n - 1, 3, n - 2], [n // 2, n - 3, 0]], dtype=torch.int32, device="cuda")
    big = track.Cache4(heads, D, page, table, pages)
    small = track.Cache4(heads, D, page, torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3), n_pages=6)
    k, v = (dev(normal([61, i], (2, Ln, heads, D), bf16=True), BF16) for i in range(2))
    start = torch.tensor([place, place + 5], dtype=torch.int32, device="cuda")
    q = dev(normal([62], (2, 1, 16, D), bf16=True), BF16)
    outs = []
    for cache in (big, small):
        pages = cache.pages[cache.table.long()]
        cache.pages[cache.table.long()] = torch.zeros_like(pages)
        track.op_cache4_append(cache, k, v, start)
        back = track.op_cache4_read(cache, torch.empty_like(k), torch.empty_like(v), start)
        out = torch.empty_like(q)
        track.op_attention_cache4(W(left=100), cache, q, out, Lk=place + Ln, workspace=track.attention_cache4_workspace(W(left=100), cache, q, place + Ln))
        outs.append((cache.pages[cache.table.long()], *back, out))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("Lq", [1, 3, 200])
def test_graph(Lq):
    """An append, the attention and a read, captured and replayed with new rows, places, positions, lengths and pages, with eager work between."""
    import torch
    B, H, Hk, D, page = 2, 8, 2, 128, 64
    each = 50
    win = W(left=1500, sink=4)
    pool, table = _pool(71, B * each + 5, Hk, D, page, B, each)
    pool.raw[:] = 0
    cache = _device_cache(pool, table)
    other = _device_cache(pool, table)
    rope = track.Rope(track.RopeConfig(head_dim=D, layout="half"))
    pos = torch.zeros(1, B, Lq, dtype=torch.int32, device="cuda")
    start, k_len = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    q = torch.zeros(B, Lq, H, D, dtype=torch.bfloat16, device="cuda")
    k, v, kb, vb = (torch.zeros(B, Lq, Hk, D, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    ws = track.attention_cache4_workspace(win, cache, q)

    def step(cache, out, kb, vb):
        track.op_cache4_append(cache, k, v, start, rope=rope, pos=pos)
        track.op_attention_cache4(win, cache, q, out, k_len=k_len, workspace=ws)
        track.op_cache4_read(cache, kb, vb, start)

    out = torch.zeros_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache, out, kb, vb)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, out, kb, vb)
    cache.pages.zero_()
    for i, at in enumerate(([2900, 0], [1999, 2700], [299, 63], [0, 1024])):
        start.copy_(torch.tensor(at, dtype=torch.int32))
        k_len.copy_(start + Lq)
        pos.copy_((start[:, None] + torch.arange(Lq, dtype=torch.int32, device="cuda"))[None])
        for j, t in enumerate((q, k, v)):
            t.copy_(dev(normal([72, i, j], tuple(t.shape), bf16=True), BF16))
        if i == 2:  # another sequence's pages
            for x in (cache, other):
                x.table.copy_(x.table.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        got = [out.clone(), kb.clone(), vb.clone()]
        want = [torch.empty_like(t) for t in got]
        step(other, *want)
        torch.cuda.synchronize()
        assert torch.equal(cache.pages, other.pages)
        for a, b in zip(got, want):
            assert torch.equal(a, b), at


@gpu
@pytest.mark.parametrize("Lq", [1, 40, 500])
def test_two_calls_at_once(Lq):
    """Two streams, each with its rows, outputs and workspace, on one pool: as one after another."""
    import torch
    B, H, Hk, Lk, D = 2, 8, 2, 3000, 128
    win = W(left=-1, right=0, sink=4)
    c = Case(BF16, B, H, Hk, Lq, Lk)
    qs = [c.tq, c.tq.flip(1).contiguous()]
    wss = [track.attention_cache4_workspace(win, c.cache, c.tq, Lk) for _ in qs]

    def call(i, out):
        return track.op_attention_cache4(win, c.cache, qs[i], out, Lk=Lk, workspace=wss[i])

    want = [call(i, torch.empty_like(c.tq)) for i in range(2)]
    for _ in range(3):
        outs = [torch.empty_like(c.tq) for _ in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                call(i, outs[i])
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_streaming_run(dtype):
    """The calls as a streaming program uses them: frames arrive in chunks, keys and queries are normed, keys rotated into the
    cache, queries rotated, and they attend to the last frames and the first one; pages behind the window are given back; then tokens
    come singly.  Against the formulas on what the cache holds, and the cache against the definition."""
    import torch
    H, Hk, D, group, frames = 4, 2, 128, 48, 9
    total, extra, page = group * frames, 5, 64
    n = total + extra
    bf = dtype == BF16
    x = normal([81], (1, n, H + 2 * Hk, D), bf16=bf)
    win = W(left=2, right=0, sink=group, group=group)
    sections = (22, 21, 21)
    rope = track.Rope(track.RopeConfig(head_dim=D, sections=sections))
    t = np.arange(n)
    pos = np.stack([t // group, t % group // 8, t % 8])[:, None].astype(np.int32)
    each = -(-n // page)
    rng = np.random.default_rng(82)
    table = torch.from_numpy(rng.permutation(each + 2)[:each].reshape(1, each).astype(np.int32)).cuda()
    cache = track.Cache4(Hk, D, page, table, n_pages=each + 2)
    tx, tp = dev(x, dtype), torch.from_numpy(pos).cuda()
    out = torch.empty(1, n, H, D, dtype=tx.dtype, device="cuda")
    qr = torch.empty_like(out)
    f = ref.freqs(sections)
    k = c4.values(*c4.quantise(ref.rope(x[:, :, H:H + Hk].astype(np.float64), pos, sections, f)))
    v = c4.values(*c4.quantise(x[:, :, H + Hk:].astype(np.float64)))
    at = 0
    for step in [group, 3 * group, 2 * group, 3 * group] + [1] * extra:
        s = slice(at, at + step)
        track.op_cache4_append(cache, tx[:, s, H:H + Hk], tx[:, s, H + Hk:], torch.tensor([at], dtype=torch.int32, device="cuda"),
                               rope=rope, pos=tp[:, :, s].contiguous())
        track.op_rope(rope, tx[:, s, :H], None, tp[:, :, s].contiguous(), qr[:, s])
        back = track.op_cache4_read(cache, torch.empty_like(tx[:, s, :Hk]), torch.empty_like(tx[:, s, :Hk]),
                                    torch.tensor([at], dtype=torch.int32, device="cuda"))
        np.testing.assert_array_equal(host(back[0]), k[:, s])
        np.testing.assert_array_equal(host(back[1]), v[:, s])
        at += step
        track.op_attention_cache4(win, cache, qr[:, s], out[:, s], Lk=at,
                                  workspace=track.attention_cache4_workspace(win, cache, qr[:, s], at))
        done = (at // group - 3) * group // page  # pages that lie whole before the next token's window
        for p in range(-(-group // page), done):
            table[0, p] = -1
    for a, b in [(0, total)] + [(i, i + 1) for i in range(total, n)]:
        want, _, mag, big = c4.attention(host(qr)[:, a:b].astype(np.float64), k[:, :b], v[:, :b], np.ones((1, b), bool),
                                         lambda p, m: ref.seen(p, m, 2, 0, group, group), 1 / math.sqrt(D))
        _close(host(out)[:, a:b], want, 2.1 * _eta(dtype, D, big, b) * mag + 1.01 * U[dtype] * np.abs(want), f"out {a}")

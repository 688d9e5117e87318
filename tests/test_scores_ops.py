"""Attention with capped logits, a bias by distance, documents and prefixes against its formula in float64.

Tolerances (u = eps / 2 of the output type): weights off by a relative eta give |do| <= 2 eta sum w|v|.  eta is the logit's
error: (D + 2) float32 roundings of sum |scale q k| (the cap's slope is 1 at most); of the cap, 5 cap 2^-23 (with t = exp(2 y):
2 t / (t + 1)^2 <= 1/2 of t's error, one unit of exp2 and two roundings of its argument, 0.95; 1.5 units of the sum and the reciprocal, twice;
two roundings; float32's tanh: 5 units); of the bias, 3 float32 roundings of the largest one seen; then 2^-21 for exp2 and its argument, the
rounding to bfloat16 where the weights take one, and the float32 sums over the keys.
"""
import math

import numpy as np
import pytest

import scores_reference as ref
from gpu_helpers import dev, host, normal, say
from paper_2609_30096_amd import synth, track

F32, BF16 = synth.F32, synth.BF16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
S = track.Scores
gpu = pytest.mark.gpu
P = 1 << 20  # aligned stand-in; never dereferenced


@pytest.fixture
def L():
    return track.lib()


# ---------------------------------------------------------------- on the host
def test_refusals(L):
    E, F, Sh, I, N, Un = (track.DTYPE_BF16, track.DTYPE_F32, track.E_SHAPE, track.E_INVALID, track.E_NOMEM,
                          track.E_UNSUPPORTED)
    base = dict(B=2, H=8, Hk=4, D=128, Lq=1, Lk=5000, ldq=1024, sq=1024, ldk=512, sk=512 * 5000, ldv=5000, sv=512 * 5000,
                ldo=1024, so=1024, q=P, k=P, vt=P, out=P, lse=None, slopes=P, doc_end=P, docs=3, prefix=P, q_len=None,
                k_len=None, q_start=None, ws=P, ws_bytes=1 << 40)

    def call(dtype=E, sc=None, **kw):
        a = dict(base, **kw)
        return L.track_op_attention_scores(
            dtype, (S() if sc is None else sc).c(), a["B"], a["H"], a["Hk"], a["D"], a["Lq"], a["Lk"], a["q"], a["ldq"],
            a["sq"], a["k"], a["ldk"], a["sk"], a["vt"], a["ldv"], a["sv"], a["out"], a["ldo"], a["so"], a["lse"],
            a["slopes"], a["doc_end"], a["docs"], a["prefix"], a["q_len"], a["k_len"], a["q_start"], a["ws"],
            a["ws_bytes"], None)

    assert L.track_op_attention_scores(E, None, *([1] * 6), *([None, 1, 1] * 4), *([None] * 3), 0, *([None] * 5), 0, None) == I
    assert b"null scores" in L.track_last_error()
    assert call(dtype=2) == I and b"attention_scores: bad dtype" in L.track_last_error()
    for bad in (dict(group=0), dict(left=-2), dict(right=-2), dict(scale=-1.0), dict(scale=math.nan), dict(scale=1e31),
                dict(cap=-1.0), dict(cap=math.nan), dict(cap=math.inf), dict(cap=1e-4), dict(cap=1.1e3)):
        assert call(sc=S(**bad)) == I, bad
    for bad in (dict(group=1 << 31), dict(left=1 << 31), dict(right=1 << 31)):
        assert call(sc=S(**bad)) == Sh, bad
    assert call(docs=-1) == Sh and call(docs=(1 << 20) + 1) == Sh and call(doc_end=None) == I
    for name in ("slopes", "doc_end", "prefix", "lse", "q_len", "k_len", "q_start"):
        assert call(**{name: P + 2}) == I, name
    assert call(B=-1) == Sh and call(H=0) == Sh and call(Hk=0) == Sh and call(H=8, Hk=3) == Sh
    assert call(Lq=-1) == Sh and call(Lk=-1) == Sh and call(Lk=1 << 31) == Sh and call(Lq=1 << 30) == Sh
    assert call(D=64) == Un and call(F, D=80) == Un
    for name in ("q", "k", "vt", "out"):
        assert call(**{name: None}) == I and call(**{name: P + 8}) == I and call(F, **{name: P + 2}) == I, name
    assert call(ldq=1016) == Sh and call(ldk=504) == Sh and call(ldo=1016) == Sh and call(ldv=4992) == Sh
    assert call(ldq=1028) == I and call(ldk=516) == I and call(ldv=5004) == I
    assert call(sq=-8) == Sh and call(so=512) == Sh and call(ldk=(1 << 23) + 8) == Sh
    need = track.attention_scores_workspace_bytes(S(), E, 2, 8, 4, 128, 1, 5000)
    assert need > 0 and need == track.attention_window_workspace_bytes(track.Window(), E, 2, 8, 4, 128, 1, 5000)
    assert call(ws=None) == N and call(ws_bytes=need - 1) == N and call(ws=P + 128) == I
    assert call(B=0) == 0 and call(Lq=0) == 0 and call(B=0, doc_end=None) == 0
    assert L.track_attention_scores_workspace_bytes(E, None, 1, 1, 1, 128, 1, 1) == -1
    with pytest.raises(track.TrackError):
        track.attention_scores_workspace_bytes(S(cap=-1.0), E, 1, 1, 1, 128, 1, 1)
    with pytest.raises(track.TrackError):
        track.attention_scores_workspace_bytes(S(), E, 1, 3, 2, 128, 1, 1)
    with pytest.raises(ValueError, match="scale of 0"):
        S(scale=0.0)


def test_layout_refusals():
    import torch
    B, Lq, Lk, H, Hk, D = 2, 5, 7, 4, 2, 128
    q = torch.zeros(B, Lq, H, D)
    ok = dict(q=q, k=torch.zeros(B, Lk, Hk, D), vt=torch.zeros(B, Hk, D, 8), out=torch.zeros_like(q), lse=None, q_len=None,
              k_len=None, q_start=None, workspace=None, slopes=torch.zeros(H), doc_end=torch.zeros(B, 3, dtype=torch.int32),
              prefix=torch.zeros(B, 4, dtype=torch.int32))
    assert track._check_scores(**ok)[1] == 3
    assert track._check_scores(**dict(ok, doc_end=None, prefix=ok["prefix"][:, :1].contiguous(), slopes=None))[1] == 0
    for match, kw in ((r"^slopes: contiguous float32 \[4\]", dict(slopes=torch.zeros(2))), ("^slopes", dict(slopes=torch.zeros(4).double())),
                      ("^slopes", dict(slopes=torch.zeros(8)[::2])), (r"^doc_end: \[sequences, documents\]", dict(doc_end=ok["doc_end"][0])),
                      (r"^doc_end: contiguous int32 \(2, 3\)", dict(doc_end=ok["doc_end"].long())),
                      (r"^doc_end: contiguous int32 \(2, 3\)", dict(doc_end=torch.zeros(1, 3, dtype=torch.int32))),
                      (r"^prefix: contiguous int32 \(2, 4\)", dict(prefix=torch.zeros(2, 3, dtype=torch.int32))),
                      (r"^prefix: contiguous int32 \(2, 1\)", dict(doc_end=None)), ("do not match$", dict(out=q[:, :4]))):
        with pytest.raises((ValueError, TypeError), match=match):
            track._check_scores(**dict(ok, **kw))
    with pytest.raises(ValueError, match="^GPU tensors expected"):
        track.op_attention_scores(S(), **ok)


def test_reference_masks():
    """Masks that can be written down by hand."""
    def row(*a, **kw):
        return "".join("x" if v else "." for v in ref.seen(*a, **kw))
    assert row(4, 8, -1, 0, 1) == "xxxxx..."
    assert row(4, 8, 1, 1, 1) == "...xxx.."
    assert row(4, 8, -1, 0, 1, ends=[3, 6]) == "...xx..."
    assert row(4, 8, -1, -1, 1, ends=[3, 6]) == "...xxx.."
    assert row(3, 8, -1, 0, 1, ends=[3, 6], prefix=[0, 2, 0]) == "...xx..."
    assert row(6, 8, -1, 0, 1, ends=[3, 6], prefix=[0, 2, 5]) == "......xx"
    assert row(1, 8, -1, 0, 1, prefix=[4]) == "xxxx...."
    assert row(5, 8, 1, 0, 1, prefix=[8]) == "....xxxx"
    assert row(2, 8, -1, 0, 3) == "xxx....." and row(-1, 4, -1, 1, 2) == "xx.."


# ---------------------------------------------------------------- on the GPU
def _close(got, want, tol, what):
    err = np.abs(np.asarray(got, np.float64) - want)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.nanmax(err / np.maximum(tol, 1e-300)):.3g} x"


class Case:
    def __init__(self, dtype, B, H, Hk, Lq, Lk, D=128, key=51, scale=1.0, slope=0.0, ends=None, prefix=None):
        import torch
        bf = dtype == BF16
        self.dtype, self.Lk, self.D = dtype, Lk, D
        self.q = normal([key, 1], (B, Lq, H, D), scale, bf)
        self.k = normal([key, 2], (B, Lk, Hk, D), scale, bf)
        self.v = normal([key, 3], (B, Lk, Hk, D), 1.0, bf)
        cap = (Lk + 7) // 8 * 8
        kc, vc = np.full((B, cap, Hk, D), np.nan, np.float32), np.full((B, Hk, D, cap), np.nan, np.float32)
        kc[:, :Lk] = self.k
        vc[..., :Lk] = self.v.transpose(0, 2, 3, 1)
        self.tq, self.tk, self.tv = dev(self.q, dtype), dev(kc, dtype), dev(vc, dtype)
        self.out = torch.full((B, Lq, H, D), 9.0, dtype=self.tq.dtype, device="cuda")
        self.lse = torch.full((B, H, Lq), 9.0, device="cuda")
        self.slopes = np.float32(slope) * (1.0 + np.arange(H, dtype=np.float32)) if slope else None
        self.ends = None if ends is None else np.array(ends, np.int32).reshape(B, -1)
        self.prefix = None if prefix is None else np.array(prefix, np.int32).reshape(B, -1)

    def kw(self, **lens):
        import torch
        got = {n: torch.tensor(v, dtype=torch.int32, device="cuda") for n, v in lens.items() if v is not None}
        for n, v in (("slopes", self.slopes), ("doc_end", self.ends), ("prefix", self.prefix)):
            if v is not None:
                got[n] = torch.from_numpy(v).cuda()
        return got

    def run(self, sc, **lens):
        k = self.tk[:, :self.Lk]
        ws = track.attention_scores_workspace(sc, self.tq, k)
        track.op_attention_scores(sc, self.tq, k, self.tv, self.out, lse=self.lse, workspace=ws, **self.kw(**lens))
        return host(self.out), host(self.lse)


def _check(c, sc, got, lse, rows=None, **lens):
    want, wlse, mag, big, far = ref.attention(c.q, c.k, c.v, sc.left, sc.right, sc.group, sc.scale, sc.cap, c.slopes, c.ends,
                                              c.prefix, **lens)
    if rows is not None:
        got, lse, want, wlse, mag = got[:, rows], lse[..., rows], want[:, rows], wlse[..., rows], mag[:, rows]
    eta = (c.D + 2) * 2.0 ** -24 * big + 5 * sc.cap * 2.0 ** -23 + 3 * far * 2.0 ** -24 + 2.0 ** -21 + (c.Lk + 16) * 2.0 ** -24 + \
        (U[BF16] if c.dtype == BF16 else 0.0)
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
    return 2.1 * eta * mag + U[c.dtype] * np.abs(want) * 1.01


CASES = [
    # B, H, Hk, Lq, Lk, scores, slope, ends, prefix, lengths
    (1, 1, 1, 1, 1, S(), 0.0, None, None, {}),
    (1, 4, 4, 1, 7, S(cap=5.0), 0.1, None, None, {}),
    (2, 8, 2, 1, 200, S(left=63, cap=50.0), 0.0, None, None, {}),
    (3, 10, 2, 1, 1000, S(), 0.01, [[400, 800], [1000, 1000], [1, 999]], None, dict(k_len=[1000, 1, 517])),
    (2, 5, 1, 1, 3000, S(cap=30.0), 0.002, None, None, dict(k_len=[3000, 2048])),
    (2, 4, 1, 4, 300, S(right=1, group=7), 0.0, [[100, 298], [10, 150]], [[3, 9, 0], [0, 0, 400]], dict(q_len=[4, 2], k_len=[300, 155])),
    (2, 4, 2, 13, 777, S(left=100, cap=2.0), 0.02, None, [[700], [0]], {}),
    (1, 6, 2, 16, 130, S(), 0.0, None, None, {}),
    (1, 2, 2, 300, 300, S(cap=20.0), 0.0, [[100, 101, 260]], None, {}),
    (1, 2, 2, 300, 300, S(right=-1), 0.05, [[64, 128, 192, 256]], None, {}),
    (1, 2, 2, 300, 300, S(right=0), 0.0, [[77, 90, 255]], [[50, 13, 1, 300]], {}),
    (2, 4, 2, 300, 451, S(left=63), 0.001, [[200], [451]], [[10, 300], [450, 0]], dict(q_len=[300, 211], k_len=[451, 213])),
    (1, 3, 3, 640, 960, S(left=1, right=2, group=100, cap=50.0), 0.003, [[333, 700]], None, {}),
    (1, 2, 1, 700, 700, S(right=0, group=70, cap=30.0), 0.0, [[140, 490]], [[0, 200, 700]], {}),
    (2, 2, 2, 500, 333, S(left=5, right=0), 0.0, None, None, {}),                     # the first 167 queries see nothing
    (1, 2, 2, 80, 400, S(left=10), 0.1, None, None, dict(q_start=[1000])),
    (3, 2, 1, 100, 256, S(), 0.0, [[50]] * 3, [[20, 20]] * 3, dict(q_len=[0, 100, 50], k_len=[256, 0, 256])),
    (1, 1, 1, 70, 4000, S(cap=50.0), 0.001, None, None, {}),                          # shares of the keys
    (1, 2, 1, 200, 9000, S(right=-1), 0.0, [[4000, 8850]], None, {}),
    (1, 2, 1, 600, 600, S(right=-1, cap=10.0), 0.02, [sorted([6 * i + 5 for i in range(99)])], None, {}),  # 99 documents: by halves
    (1, 2, 1, 300, 400, S(), 0.0, [list(range(0, 260, 4))], [[2] * 66], {}),           # 65 of them
    (1, 2, 1, 300, 400, S(), 0.0, [list(range(0, 256, 4))], [[2] * 65], {}),           # 64
    (3, 2, 1, 20, 300, S(left=100, cap=9.0), 0.0, [[0, 290]] * 3, None, dict(q_start=[-(1 << 28), 1 << 28, 290])),
    (2, 2, 1, 40, 300, S(cap=1e3), -0.01, None, [[-5], [2 ** 31 - 1]], {}),
    (2, 2, 1, 40, 300, S(cap=1e-3), 0.0, [[-10, -1], [10, 2 ** 31 - 1]], None, {}),
    (2, 8, 8, 1040, 1040, S(cap=50.0), 0.01, [[500], [999]], [[100, 100], [0, 40]], dict(q_len=[1040, 900], k_len=[1040, 1000])),
]


@gpu
@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F32, 32), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_scores(dtype, D, i):
    B, H, Hk, Lq, Lk, sc, slope, ends, prefix, lens = CASES[i]
    say(f"scores {dtype} D={D} {CASES[i]}")
    c = Case(dtype, B, H, Hk, Lq, Lk, D, slope=slope, ends=ends, prefix=prefix)
    got, lse = c.run(sc, **lens)
    if prefix is not None:
        c.prefix = np.clip(c.prefix, 0, 1 << 28)
    _check(c, sc, got, lse, **lens)
    again, lse2 = c.run(sc, **lens)
    assert np.array_equal(got, again) and np.array_equal(lse, lse2)


@gpu
@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F32, 64)])
@pytest.mark.parametrize("Lq,Lk", [(1, 3000), (9, 700), (400, 900)])
def test_without_changes_it_is_the_window(dtype, D, Lq, Lk):
    """No cap, bias, document or prefix: op_attention_window within both tolerances; in float32 bit for bit."""
    import torch
    c = Case(dtype, 2, 4, 2, Lq, Lk, D)
    sc, win = S(left=77, right=1, group=3), track.Window(left=77, right=1, group=3)
    got, lse = c.run(sc)
    _check(c, sc, got, lse)
    k = c.tk[:, :Lk]
    out = torch.empty_like(c.out)
    track.op_attention_window(win, c.tq, k, c.tv, out, workspace=track.attention_window_workspace(win, c.tq, k))
    np.testing.assert_allclose(host(out), got, rtol=4 * U[dtype], atol=4 * U[dtype])


@gpu
@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F32, 32), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("Lq,Lk", [(1, 3000), (9, 700), (400, 900)])
def test_without_changes_lse_is_the_windows(dtype, D, Lq, Lk):
    """Both are within _check's tolerance of the same number, so they are within twice that of each other (not the same bits: the
    changed logits are scaled before the reference is taken off, the window's in one FMA)."""
    import torch
    c = Case(dtype, 2, 4, 2, Lq, Lk, D)
    sc, win = S(left=77, right=1, group=3), track.Window(left=77, right=1, group=3)
    _, lse = c.run(sc)
    want, wlse, _, big, _ = ref.attention(c.q, c.k, c.v, 77, 1, 3)
    k, out, got = c.tk[:, :Lk], torch.empty_like(c.out), torch.empty_like(c.lse)
    track.op_attention_window(win, c.tq, k, c.tv, out, lse=got, workspace=track.attention_window_workspace(win, c.tq, k))
    eta = (D + 2) * 2.0 ** -24 * big + 2.0 ** -21 + (Lk + 16) * 2.0 ** -24 + (U[BF16] if dtype == BF16 else 0.0)
    _close(host(got), lse, 2 * (1.1 * eta + 2.0 ** -22 * np.abs(wlse) + 1e-6), "lse")


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq,Lk", [(1, 1000), (1, 6000), (9, 700), (400, 900)])
def test_masked_places(dtype, Lq, Lk):
    """NaN and infinities in K and V of other documents, behind the last key and before the window reach no query."""
    import torch
    ends = [[Lk // 4, Lk // 2 + 7]]
    c = Case(dtype, 1, 4, 2, Lq, Lk, slope=0.01, ends=ends)
    sc = S(left=300, right=0, cap=30.0)
    docs = np.searchsorted(ends[0], np.arange(Lk), side="right")
    rows = np.arange(Lq) + Lk - Lq
    first = docs[rows[0]]
    for value in (float("nan"), float("inf"), torch.finfo(c.tk.dtype).min):
        hide = torch.from_numpy((docs < first) | (np.arange(Lk) < rows[0] - 300)).cuda()
        c.tk[:, :Lk][:, hide] = value
        c.tv[..., :Lk][..., hide] = value
        got, lse = c.run(sc)
        _check(c, sc, got, lse)
    if Lq < 60:
        return
    # a key in the middle of the last document: its later rows see it
    place = Lk - 100
    sees = rows >= place
    for value in (float("nan"), float("inf")):
        c.tv[..., place] = value
        got, lse = c.run(sc)
        assert np.array_equal(np.isfinite(got).all((0, 2, 3)), ~sees)
        _check(c, sc, got, lse, rows=np.nonzero(~sees)[0])


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 20, 300])
@pytest.mark.parametrize("cap", [0.0, 5.0, 50.0])
def test_large_logits(dtype, Lq, cap):
    """Logits of some hundreds, capped or not, under a bias of some hundreds."""
    c = Case(dtype, 1, 2, 1, Lq, 900, scale=6.0, slope=0.3)
    sc = S(left=400, cap=cap)
    got, lse = c.run(sc)
    _check(c, sc, got, lse)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 300])
def test_query_not_finite(dtype, Lq):
    """A query of NaN gives NaN to its row alone."""
    c = Case(dtype, 1, 2, 2, Lq, 400)
    sc = S(cap=4.0, right=-1)
    c.tq[0, 0, 1, 3] = float("nan")
    got, lse = c.run(sc)
    assert np.isnan(got[0, 0, 1]).all() and np.isnan(lse[0, 1, 0])
    got[0, 0, 1], lse[0, 1, 0] = 0.0, 0.0
    assert np.isfinite(got).all() and np.isfinite(lse).all()


@gpu
@pytest.mark.parametrize("Lq", [1, 200])
def test_graph(Lq):
    """Captured and replayed with new queries, slopes, documents, prefixes and lengths, with eager work between."""
    import torch
    B, H, Hk, Lk = 2, 8, 2, 3000
    sc = S(cap=30.0)
    c = Case(BF16, B, H, Hk, Lq, Lk, slope=0.01, ends=[[1000, 2000]] * B, prefix=[[5, 5, 5]] * B)
    k = c.tk[:, :Lk]
    kw = c.kw(k_len=[Lk] * B)
    ws = track.attention_scores_workspace(sc, c.tq, k)

    def step(out):
        track.op_attention_scores(sc, c.tq, k, c.tv, out, workspace=ws, **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(c.out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c.out)
    for i, lens in enumerate(([3000, 1], [2001, 2999], [300, 64], [0, 1024])):
        kw["k_len"].copy_(torch.tensor(lens, dtype=torch.int32))
        kw["doc_end"].copy_(torch.tensor([[100 * i, 2000 + i], [50, 60 * i + 50]], dtype=torch.int32))
        kw["prefix"].fill_(300 * i)
        kw["slopes"].mul_(0.5)
        c.tq.copy_(dev(normal([72, i], tuple(c.tq.shape), bf16=True), BF16))
        graph.replay()
        torch.cuda.synchronize()
        got = c.out.clone()
        eager = torch.empty_like(c.out)
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, eager), lens


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_packed_is_each_alone(dtype):
    """Three shots packed in one sequence, with a prefix each, give what each gives alone, and single tokens of the last one
    what their rows of the whole give."""
    import torch
    lens, H, Hk, D = [130, 77, 201], 4, 2, 128
    n = sum(lens)
    ends = np.cumsum(lens)[:-1]
    prefix = [30, 77, 5]
    c = Case(dtype, 1, H, Hk, n, n, slope=0.01, ends=[ends], prefix=[prefix])
    sc = S(cap=20.0, right=0)
    got, lse = c.run(sc)
    tol = _check(c, sc, got, lse)
    at = 0
    for m, px in zip(lens, prefix):
        s = slice(at, at + m)
        alone = Case(dtype, 1, H, Hk, m, m, slope=0.01, prefix=[[px]])
        alone.q, alone.k, alone.v = c.q[:, s], c.k[:, s], c.v[:, s]
        alone.tq, alone.tk = dev(alone.q, dtype), dev(alone.k, dtype)
        alone.tv[..., :m] = c.tv[..., s]
        a, al = alone.run(sc)
        # each is within its tolerance of the same exact value, so they are within both of each other
        _close(a, got[:, s], tol[:, s] + _check(alone, sc, a, al), "alone")
        at += m
    one = Case(dtype, 1, H, Hk, 1, n, slope=0.01, ends=[ends], prefix=[prefix])
    one.k, one.v, one.tk, one.tv = c.k, c.v, c.tk, c.tv
    for i in (0, 129, 130, 206, 207, 300, n - 1):
        one.q = c.q[:, i:i + 1]
        one.tq = dev(one.q, dtype)
        o, ol = one.run(sc, q_start=[i])
        _check(one, sc, o, ol, q_start=[i])


@gpu
@pytest.mark.parametrize("B,H,Hk,Lq,Lk,docs,right,cap", [
    (2, 12, 12, 4200, 4200, 3, -1, 0.0),    # workgroups take the documents' blocks longest first: several sequences,
    (3, 40, 8, 1000, 5000, 7, 0, 30.0),     # shared key heads,
    (1, 12, 12, 5600, 5700, 70, 0, 0.0),    # more documents than lanes,
    (8, 12, 12, 5600, 5600, 5, -1, 0.0),    # more blocks an XCD than are put in order
    (2, 2, 2, 300, 40000, 2, -1, 9.0)])     # shares of the keys
def test_every_row_of_documents_is_taken(B, H, Hk, Lq, Lk, docs, right, cap):
    """Queries of zero weigh every key that they see 1 exactly (the cap of 0 is 0), so the log-sum-exp is the log of their number, and
    V that is 1 in one key in 64 gives an exact count over it: each row once, whatever the order of the workgroups.
    Errors: the logarithm (2^-23), its factor and the product (2^-24 each); a division and the output's rounding; with a cap
    5 cap 2^-23 of the logits, of all the same."""
    import torch
    say(f"documents {B} {H} {Hk} {Lq} {Lk} {docs}")
    D, bf = 128, torch.bfloat16
    q = torch.zeros(B, Lq, H, D, dtype=bf, device="cuda")
    k = torch.randn(B, Lk, Hk, D, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(bf)
    width = (Lk + 7) // 8 * 8
    hit = (torch.arange(width, device="cuda")[None, :] - torch.arange(D, device="cuda")[:, None]) % 64 == 0
    vt = hit.to(bf).expand(B, Hk, D, width).contiguous()
    rng = np.random.default_rng(docs)
    ends = np.sort(rng.integers(0, Lk + 1, (B, docs)), axis=1).astype(np.int32)
    prefix = rng.integers(0, 300, (B, docs + 1)).astype(np.int32)
    q_len = np.array([Lq - 77 * b for b in range(B)], np.int32)
    k_len = np.array([Lk - 50 * b for b in range(B)], np.int32)
    out, lse = torch.full_like(q, 9.0), torch.full((B, H, Lq), 9.0, device="cuda")
    sc = S(right=right, cap=cap)
    track.op_attention_scores(sc, q, k, vt, out, lse=lse, workspace=track.attention_scores_workspace(sc, q, k),
                              **{n: torch.from_numpy(v).cuda() for n, v in
                                 dict(doc_end=ends, prefix=prefix, q_len=q_len, k_len=k_len).items()})
    hits = np.concatenate([np.zeros((1, D)), np.cumsum(hit[:, :Lk].cpu().numpy().T, axis=0)])  # of keys before each
    for b in range(B):
        lq, lk = int(q_len[b]), int(k_len[b])
        p = np.arange(lq) + lk - lq
        bounds = np.concatenate([[0], ends[b].astype(np.int64), [1 << 40]])
        d = np.searchsorted(ends[b], p, side="right")
        lo, hi = np.minimum(bounds[d], lk), np.minimum(bounds[d + 1], lk)
        if right == 0:
            hi = np.minimum(hi, np.maximum(p + 1, bounds[d] + prefix[b][d]))
        n = np.maximum(hi - lo, 0)
        want = (hits[hi] - hits[lo]) / np.maximum(n, 1)[:, None]
        wlse = np.log(np.maximum(n, 1))
        got, glse = host(out[b]), host(lse[b])
        tol = 5 * cap * 2.0 ** -23
        for h in range(H):
            _close(got[:lq, h], want, (U[BF16] + 2.0 ** -22 + 2 * tol) * want, f"out {b} {h}")
            some = n > 0
            _close(glse[h, :lq][some], wlse[some], 1.01 * 2.0 ** -22 * wlse[some] + tol + 1e-30, f"lse {b} {h}")
            assert np.all(glse[h, :lq][~some] == -np.inf) and np.all(got[:lq, h][~some] == 0.0)
        assert np.all(got[lq:] == 9.0) and np.all(glse[:, lq:] == 9.0)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 90])
def test_no_keys(dtype, Lq):
    import torch
    q = torch.ones(2, Lq, 4, 128, device="cuda").to(track.torch_dtype(dtype))
    k, vt = q.new_empty(2, 0, 2, 128), q.new_empty(2, 2, 128, 0)
    out, lse = torch.full_like(q, 3.0), torch.zeros(2, 4, Lq, device="cuda")
    track.op_attention_scores(S(cap=5.0), q, k, vt, out, lse=lse, slopes=torch.ones(4, device="cuda"),
                              doc_end=torch.zeros(2, 2, dtype=torch.int32, device="cuda"))
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@gpu
@pytest.mark.parametrize("ends", [[700, 100, 300], [2 ** 31 - 1, -2 ** 31, 5], [-2 ** 31] * 70, list(range(80, 0, -1))],
                         ids=["mixed", "limits", "lowest", "falling"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [1, 300])
def test_ends_that_do_not_ascend(ends, dtype, Lq):
    """Outputs are unspecified, and nothing else happens: no write behind them."""
    c = Case(dtype, 1, 2, 1, Lq, 900, ends=[ends], prefix=[[2 ** 31 - 1] * (len(ends) + 1)])
    sc = S()
    c.run(sc, q_len=[Lq - Lq // 3])
    assert np.all(host(c.out)[:, Lq - Lq // 3:] == 9.0) and np.all(host(c.lse)[..., Lq - Lq // 3:] == 9.0)

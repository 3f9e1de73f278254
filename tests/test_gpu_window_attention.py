"""Sliding-window attention with sinks over packed sequences against float64: lengths from 0
and 1 to several blocks, windows and sinks at the blocks' edges, grouped heads, types, strides,
rows of no sequence, values that must not reach a result, gradients against differences,
captured graphs.

Tolerances (normwise, 2-norm over an output). fp32: a score is a sum of at most 128 products of
size |q||k|/sqrt(hd), its error below 128 * 2^-24 * |s| ~ 1e-5 in the worst case and a tenth of
that in the mean; weights, sums and outputs follow it: 1e-5. 16 bits: the weights are rounded
once (half a step, 2^-8 in bf16) and so is the result: 2 * 2^-8 for o; a gradient has up to four
such roundings (the weight or score gradient, o inside D, a bf16 copy of an fp16 operand, the
result): 4 * 2^-8."""
import math

import pytest
import torch

from paper_2606_11169_amd import libchunk as lc
from tests.gpu_util import DEV, banner

pytestmark = pytest.mark.gpu
F32, BF16, F16 = lc.LC_FP32, lc.LC_BF16, lc.LC_FP16
DT = {F32: torch.float32, BF16: torch.bfloat16, F16: torch.float16}
TOL_O = {F32: 1e-5, BF16: 2 * 2.0 ** -8, F16: 2 * 2.0 ** -8}
TOL_G = {F32: 1e-5, BF16: 4 * 2.0 ** -8, F16: 4 * 2.0 ** -8}


def seen(lens, first, T, W, S):
    """[T, T] which key each row sees."""
    start = torch.full((T,), T, dtype=torch.long)
    at = first
    for n in lens:
        start[at:at + n] = at
        at += n
    i, j = torch.arange(T)[:, None], torch.arange(T)[None, :]
    s = start[:, None]
    return ((j <= i) & (j >= s) & ((i - j < W) | (j < s + S)) & (s < T)).to(DEV)


def reference(q, k, v, dout, see, H, Hkv, hd):
    """o, lse, dq, dk, dv in float64; a masked place contributes nothing, whatever it holds."""
    T, G = q.shape[0], H // Hkv
    q, k, v, dout = (t.double() for t in (q, k, v, dout))
    o, lse = torch.zeros_like(q), torch.zeros((H, T), dtype=torch.float64, device=DEV)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    some = see.any(1)
    for h in range(H):
        a, b = slice(h * hd, (h + 1) * hd), slice(h // G * hd, (h // G + 1) * hd)
        s = (q[:, a] @ k[:, b].T / math.sqrt(hd)).masked_fill(~see, -math.inf)
        L = torch.logsumexp(s, 1)
        P = torch.where(see, torch.exp(s - L[:, None]), 0.0)
        o[:, a], lse[h] = P @ v[:, b], torch.where(some, L, 0.0)
        dP = dout[:, a] @ v[:, b].T
        dS = torch.where(see, P * (dP - (dout[:, a] * o[:, a]).sum(1, keepdim=True)), 0.0) / math.sqrt(hd)
        do = torch.where(some[:, None], dout[:, a], 0.0)
        dq[:, a] = dS @ k[:, b]
        dk[:, b] += dS.T @ q[:, a]
        dv[:, b] += P.T @ do
    return o, lse, dq, dk, dv


def make(lens, H, Hkv, hd, dt, first=0, tail=0, seed=1, pad=0, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    T = first + sum(lens) + tail
    out = F32 if dt == F32 else BF16

    def t(width, ty, s=scale):
        buf = torch.full((T, width + pad), 5.0, device=DEV, dtype=DT[ty])
        buf[:, :width] = (torch.randn((T, width), generator=g, device=DEV) * s).to(DT[ty])
        return buf

    off = [first]
    for n in lens:
        off.append(off[-1] + n)
    return dict(T=T, out=out, q=t(H * hd, dt), k=t(Hkv * hd, dt), v=t(Hkv * hd, dt), dout=t(H * hd, out),
                off=torch.tensor(off, dtype=torch.int32, device=DEV), pad=pad, dt=dt, H=H, Hkv=Hkv, hd=hd,
                lens=lens, first=first)


def run(m, W, S, offsets=True, stream=None, scratch=None, fill=9.0):
    T, H, Hkv, hd, dt, out, pad = (m[x] for x in ("T", "H", "Hkv", "hd", "dt", "out", "pad"))
    qw, kw = H * hd + pad, Hkv * hd + pad
    o, dq = (torch.full((T, qw), fill, device=DEV, dtype=DT[out]) for _ in range(2))
    dk, dv = (torch.full((T, kw), fill, device=DEV, dtype=DT[out]) for _ in range(2))
    lse = torch.full((H, T), fill, device=DEV)
    n = lc.lc_window_attention_scratch_bytes(dt, T, H, Hkv, hd, W, S)
    if scratch is None:
        scratch = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device=DEV)  # (NaN as floats)
    B, off = (len(m["lens"]), m["off"]) if offsets else (len(m["lens"]), None)
    lc.lc_window_attention_forward(dt, out, T, B, off, H, Hkv, hd, W, S, m["q"], qw, m["k"], kw, m["v"], kw, o, qw,
                                   lse, stream=stream)
    lc.lc_window_attention_backward(dt, out, T, B, off, H, Hkv, hd, W, S, m["q"], qw, m["k"], kw, m["v"], kw, o, qw,
                                    lse, m["dout"], qw, dq, qw, dk, kw, dv, kw, scratch, n, stream=stream)
    assert bool((scratch[n:] == 0xFF).all())
    return o, lse, dq, dk, dv


def rel(a, b):
    n = float(b.norm())
    return float((a.double() - b).norm()) / (n if n else 1.0)


def verify(m, W, S, got, rows=None, keys=None):
    """Every output against float64; rows / keys: only those (where others hold what they like)."""
    o, lse, dq, dk, dv = got
    H, Hkv, hd, dt, T = (m[x] for x in ("H", "Hkv", "hd", "dt", "T"))
    see = seen(m["lens"], m["first"], T, W, S)
    q, k, v, dout = m["q"][:, :H * hd], m["k"][:, :Hkv * hd], m["v"][:, :Hkv * hd], m["dout"][:, :H * hd]
    ref = reference(q, k, v, dout, see, H, Hkv, hd)
    on = torch.zeros(T, dtype=torch.bool, device=DEV)
    on[m["first"]:m["first"] + sum(m["lens"])] = True
    for t, w in ((o, H), (dq, H), (dk, Hkv), (dv, Hkv)):  # padding columns and rows of no sequence
        assert bool((t[:, w * hd:] == 9.0).all()) and bool((t[~on] == 9.0).all())
    assert bool((lse[:, ~on] == 9.0).all())
    r = on if rows is None else on & rows
    c = on if keys is None else on & keys
    assert rel(o[r][:, :H * hd], ref[0][r]) < TOL_O[dt], "o"
    assert float((lse[:, r].double() - ref[1][:, r]).abs().max() if r.any() else 0.0) < 2e-4, "lse"
    # a row that sees one key has no score gradient: what is left of it there is o's rounding
    # inside D, half a step of |dout|, so a quarter of those rows' |dout| counts as its size
    single = 0.25 * float(dout[on & (see.sum(1) == 1)].double().norm())
    for name, t, u, at, w in (("dq", dq, ref[2], r, H), ("dk", dk, ref[3], c, Hkv), ("dv", dv, ref[4], c, Hkv)):
        if not at.any():
            continue
        d = t[at][:, :w * hd].double() - u[at]
        assert bool(torch.isfinite(d).all()), name
        assert float(d.norm()) < TOL_G[dt] * max(float(u[at].norm()), single), name


SHAPES = [([1], 1, 0), ([2, 1, 0, 5], 3, 1), ([63], 16, 2), ([64], 64, 0), ([65], 64, 1), ([128, 1], 30, 30),
          ([129], 1, 0), ([130], 1, 3), ([127, 0, 1, 300], 100, 4), ([500, 700], 128, 0), ([333, 64, 64, 200], 65, 70),
          ([600], 1000, 5), ([400, 41], 50, 1000), ([1, 1, 1, 1, 1, 1, 1], 5, 2), ([31, 33, 32, 97, 5, 250], 64, 16),
          ([0, 700, 0], 257, 64), ([1100], 200, 129)]


@pytest.mark.parametrize("dt,H,Hkv,hd", [(BF16, 2, 2, 128), (BF16, 6, 2, 64), (F16, 4, 1, 128), (F16, 2, 2, 64),
                                         (F32, 3, 3, 64), (F32, 4, 2, 18), (F32, 2, 1, 128), (BF16, 5, 1, 128)])
@pytest.mark.parametrize("lens,W,S", SHAPES, ids=[f"{'_'.join(map(str, a))}w{b}s{c}" for a, b, c in SHAPES])
def test_forward_and_backward(lens, W, S, dt, H, Hkv, hd):
    banner(f"window attention {lens} W={W} S={S} {dt} {H}/{Hkv} x {hd}")
    m = make(lens, H, Hkv, hd, dt, seed=len(lens) + W)
    verify(m, W, S, run(m, W, S))


LONG = [([5000], 64, 5, 2, 1), ([2100, 1, 2047, 3000], 100, 33, 2, 2), ([4500, 2500], 1024, 4, 1, 1),
        ([3300], 2000, 0, 2, 1), ([1030, 1024, 1025, 2050], 37, 128, 3, 1), ([6200], 20, 140, 1, 1)]


@pytest.mark.parametrize("dt,hd", [(BF16, 128), (BF16, 64), (F16, 128), (F32, 32)])
@pytest.mark.parametrize("lens,W,S,H,Hkv", LONG, ids=[f"{'_'.join(map(str, a[0]))}w{a[1]}s{a[2]}" for a in LONG])
def test_long_sequences(lens, W, S, H, Hkv, dt, hd):
    banner(f"window attention long {lens} W={W} S={S} {dt} {H}/{Hkv} x {hd}")
    m = make(lens, H, Hkv, hd, dt, seed=W, tail=9)
    verify(m, W, S, run(m, W, S))


@pytest.mark.parametrize("dt,H,Hkv,hd", [(BF16, 16, 2, 128), (BF16, 24, 24, 64), (F16, 8, 8, 128), (F32, 8, 2, 64)])
def test_rows_of_no_sequence_and_strides(dt, H, Hkv, hd):
    """Offsets that begin after row 0 and end before T, rows wider than the heads."""
    banner(f"window attention first/tail rows {dt} {H}/{Hkv} x {hd}")
    for first, tail in ((0, 1), (70, 0), (130, 200)):
        m = make([150, 0, 90, 260], H, Hkv, hd, dt, first=first, tail=tail, pad=8, seed=first)
        verify(m, 48, 7, run(m, 48, 7))
    m = make([0, 0], 2, 2, 64 if dt != F32 else 16, dt, first=5, tail=6)  # no sequence holds a row
    verify(m, 4, 1, run(m, 4, 1))


@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_equal_sequences_without_offsets(dt):
    banner(f"window attention without offsets {dt}")
    m = make([96] * 5, 4, 2, 128, dt)
    a, b = run(m, 40, 3), run(m, 40, 3, offsets=False)
    verify(m, 40, 3, b)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_full_window_equals_causal_attention():
    """A window over the whole sequence is lc_attention's result (both against the same tolerance)."""
    banner("window attention against lc_attention")
    B, S, H, hd = 2, 256, 3, 128
    m = make([S] * B, H, H, hd, BF16)
    o, lse, _, _, _ = run(m, S, 0, offsets=False)
    o2, lse2 = torch.empty_like(o), torch.empty((B, H, S), device=DEV)
    lc.lc_attention_forward(BF16, BF16, B, S, H, hd, m["q"], m["k"], m["v"], H * hd, o2, H * hd, lse2)
    assert rel(o, o2.double()) < TOL_O[BF16]
    assert float((lse.view(H, B, S).transpose(0, 1) - lse2).abs().max()) < 1e-5


@pytest.mark.parametrize("dt,H,Hkv,hd", [(BF16, 2, 2, 128), (BF16, 4, 2, 64), (F16, 2, 1, 128), (F32, 2, 2, 64)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_masked_places_reach_nothing(bad, dt, H, Hkv, hd):
    """Infinite and NaN values in one token of the middle sequence and in the rows behind the
    last: rows that do not see it, and keys that it does not see, are what they were."""
    banner(f"window attention masked places {bad} {dt}")
    lens, W, S, at = [90, 300, 70], 40, 3, 90 + 150
    for what in ("q", "k", "v", "dout"):
        m = make(lens, H, Hkv, hd, dt, tail=30, seed=6)
        clean = {x: m[x].clone() for x in ("q", "k", "v", "dout")}
        m[what][at, ::3] = bad
        for x in ("q", "k", "v", "dout"):
            m[x][sum(lens):] = bad
        got = run(m, W, S)
        m.update({x: clean[x] for x in clean})
        see = seen(lens, 0, m["T"], W, S)
        rows = ~see[:, at] if what in ("k", "v") else torch.arange(m["T"], device=DEV) != at
        # keys that some row sees which sees the bad one (or is it) carry its gradient
        hit = see[~rows].any(0)
        verify(m, W, S, got, rows=rows, keys=~hit)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_a_bad_sink_is_seen_by_all_later_rows(dt):
    banner(f"window attention bad sink {dt}")
    m = make([400, 100], 2, 2, 64, dt, seed=3)
    clean = m["v"].clone()
    m["v"][0, :] = math.nan
    o, lse, dq, dk, dv = run(m, 32, 1)
    assert bool(torch.isnan(o[:400, :128]).all()) and bool(torch.isfinite(o[400:]).all())
    m["v"] = clean
    rows = torch.arange(m["T"], device=DEV) >= 400
    verify(m, 32, 1, (o, lse, dq, dk, dv), rows=rows, keys=rows)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_large_and_equal_scores(dt):
    """Scores of some hundreds (weights of one key), and equal ones (q = 0)."""
    banner(f"window attention large scores {dt}")
    m = make([200, 55], 2, 2, 64, dt, seed=2, scale=6.0)
    see = seen(m["lens"], 0, m["T"], 50, 2)
    o, lse, dq, dk, dv = run(m, 50, 2)
    ref = reference(m["q"], m["k"], m["v"], m["dout"], see, 2, 2, 64)
    # scores of size 36 * 8 = 300: the fp32 sums of 64 products are off by up to 300 * 2^-20
    assert rel(o, ref[0]) < TOL_O[dt] + 3e-4 and float((lse.double() - ref[1]).abs().max()) < 1e-3
    m["q"].zero_()
    got = run(m, 50, 2)
    assert rel(got[0], reference(m["q"], m["k"], m["v"], m["dout"], see, 2, 2, 64)[0]) < TOL_O[dt]


@pytest.mark.parametrize("dt,H,Hkv", [(BF16, 8, 2), (F16, 4, 4), (F32, 4, 2)])
def test_the_same_bits_every_run(dt, H, Hkv):
    banner(f"window attention determinism {dt}")
    m = make([3000, 500, 77], H, Hkv, 64, dt)
    a = run(m, 200, 9)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(a, run(m, 200, 9)))


def test_gradient_against_differences():
    banner("window attention differences")
    H, Hkv, hd, W, S = 4, 2, 16, 9, 2
    m = make([30, 41], H, Hkv, hd, F32, seed=12)
    _, _, dq, dk, dv = run(m, W, S)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    h = 1e-2  # truncation of order h^2, rounding 1e3 * 2^-24 / h: below 5e-3 of a gradient's size
    for name, grad in (("q", dq), ("k", dk), ("v", dv)):
        u, base, val = torch.randn(m[name].shape, generator=g, device=DEV), m[name], []
        for sign in (1, -1):
            m[name] = base + sign * h * u
            val.append(float((run(m, W, S)[0].double() * m["dout"].double()).sum()))
        m[name] = base
        want = float((grad.double() * u.double()).sum())
        assert abs((val[0] - val[1]) / (2 * h) - want) < 5e-3 * max(1.0, abs(want)), name


@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_captured_and_replayed_on_another_stream(dt):
    banner(f"window attention graph {dt}")
    H, Hkv, hd, W, S = 4, 2, 64, 60, 4
    m = make([1500, 300, 33], H, Hkv, hd, dt)
    T, out, qw, kw = m["T"], m["out"], H * hd, Hkv * hd
    o, dq = (torch.empty((T, qw), device=DEV, dtype=DT[out]) for _ in range(2))
    dk, dv = (torch.empty((T, kw), device=DEV, dtype=DT[out]) for _ in range(2))
    lse = torch.empty((H, T), device=DEV)
    n = lc.lc_window_attention_scratch_bytes(dt, T, H, Hkv, hd, W, S)
    scratch = torch.empty(n, dtype=torch.uint8, device=DEV)
    outs = (o, lse, dq, dk, dv)

    def calls(st):
        lc.lc_window_attention_forward(dt, out, T, 3, m["off"], H, Hkv, hd, W, S, m["q"], qw, m["k"], kw, m["v"], kw,
                                       o, qw, lse, stream=st)
        lc.lc_window_attention_backward(dt, out, T, 3, m["off"], H, Hkv, hd, W, S, m["q"], qw, m["k"], kw, m["v"], kw,
                                        o, qw, lse, m["dout"], qw, dq, qw, dk, kw, dv, kw, scratch, n, stream=st)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls(side)
    for i, cuts in enumerate(([0, 1500, 1800, 1833], [0, 10, 10, 1800], [3, 600, 1700, 1833])):
        m["off"].copy_(torch.tensor(cuts, dtype=torch.int32))  # the lengths are the replay's own
        m["q"].mul_(-1.0)
        scratch.fill_(0xFF)
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        calls(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs)), i


def test_offsets_out_of_range_are_clamped():
    banner("window attention clamped offsets")
    m = make([100, 60], 2, 2, 64, BF16)
    m["off"] = torch.tensor([-7, 100, 4000], dtype=torch.int32, device=DEV)
    verify(m, 30, 2, run(m, 30, 2))


def test_no_rows():
    banner("window attention T=0")
    lc.lc_window_attention_forward(BF16, BF16, 0, 1, None, 2, 2, 64, 4, 0, None, 128, None, 128, None, 128, None, 128, None)
    torch.cuda.synchronize()


# What a call's number of rows and heads chooses: 128 rows per workgroup, its waves over one or two
# groups of keys, 64 keys per dK/dV workgroup, a group's query heads over some workgroups and sinks
# over chunks of queries (few rows, as in most tests above: 32 rows, 32 keys, every head of its own)
WIDE = [([700, 1, 0, 333, 466], 100, 5, 24, 24),    # 128 rows; 64 keys, sinks split
        ([65, 200, 63, 64, 129, 1200, 31], 64, 70, 24, 24),
        ([1000, 0, 1000], 300, 4, 32, 8),           # a group's four heads over two workgroups
        ([900, 511, 589], 1500, 0, 32, 8),
        ([1500, 1501], 600, 3, 10, 5),              # two groups of keys
        ([2999], 5000, 0, 10, 2),
        ([2500, 100], 513, 1000, 12, 12),
        ([1, 1, 3, 2, 200, 77, 1800], 33, 2, 32, 16)]
SOME = [WIDE[0], WIDE[4], WIDE[2]]


@pytest.mark.parametrize("dt,hd", [(BF16, 128), (BF16, 64), (F16, 128), (F16, 64), (F32, 40)])
@pytest.mark.parametrize("lens,W,S,H,Hkv", WIDE, ids=[f"{'_'.join(map(str, a[0]))}w{a[1]}s{a[2]}h{a[3]}" for a in WIDE])
def test_many_heads(lens, W, S, H, Hkv, dt, hd):
    banner(f"window attention wide {lens} W={W} S={S} {dt} {H}/{Hkv} x {hd}")
    m = make(lens, H, Hkv, hd, dt, seed=W, first=3, tail=70)
    a = run(m, W, S)
    verify(m, W, S, a)
    assert all(torch.equal(x, y) for x, y in zip(a, run(m, W, S)))


@pytest.mark.parametrize("dt,hd", [(BF16, 128), (BF16, 64), (F16, 128)])
@pytest.mark.parametrize("lens,W,S,H,Hkv", SOME, ids=[f"w{a[1]}s{a[2]}h{a[3]}" for a in SOME])
def test_many_heads_masked_places(lens, W, S, H, Hkv, dt, hd):
    banner(f"window attention wide masked places {lens} W={W} S={S} {dt} {H}/{Hkv} x {hd}")
    at = lens[0] // 2
    for what, bad in (("k", math.inf), ("v", math.nan), ("q", math.nan), ("dout", -math.inf)):
        m = make(lens, H, Hkv, hd, dt, tail=30, seed=6)
        clean = {x: m[x].clone() for x in ("q", "k", "v", "dout")}
        m[what][at, ::3] = bad
        for x in ("q", "k", "v", "dout"):
            m[x][sum(lens):] = bad
        got = run(m, W, S)
        m.update(clean)
        see = seen(lens, 0, m["T"], W, S)
        rows = ~see[:, at] if what in ("k", "v") else torch.arange(m["T"], device=DEV) != at
        verify(m, W, S, got, rows=rows, keys=~see[~rows].any(0))


MANY = [(64, 40, 16, 2), (100, 30, 7, 3), (63, 35, 9, 1), (1000, 9, 4, 1), (5000, 3, 2, 1), (4097, 1, 1, 0),
        (129, 60, 200, 4)]


@pytest.mark.parametrize("dt,H,Hkv,hd", [(BF16, 4, 2, 64), (F16, 2, 2, 128), (F32, 2, 1, 32), (BF16, 16, 16, 128)])
@pytest.mark.parametrize("B,most,W,S", MANY)
def test_many_sequences(B, most, W, S, dt, H, Hkv, hd):
    """Sequence counts at and past what one load of a wave holds, lengths from 0 to `most`."""
    banner(f"window attention {B} sequences of up to {most} W={W} S={S} {dt} {H}/{Hkv} x {hd}")
    g = torch.Generator()
    g.manual_seed(B)
    lens = torch.randint(0, most + 1, (B,), generator=g).tolist()
    lens[-1] = lens[-1] or 1
    m = make(lens, H, Hkv, hd, dt, seed=B, first=2, tail=5)
    verify(m, W, S, run(m, W, S))


def test_many_long_sequences_with_split_sinks():
    banner("window attention 70 sequences of which some are long")
    lens = [3000, 1, 2048, 0] + [30] * 65 + [1500]
    m = make(lens, 4, 2, 64, BF16, seed=4)
    verify(m, 50, 6, run(m, 50, 6))


@pytest.mark.parametrize("dt", [BF16, F32])
def test_many_equal_sequences_without_offsets(dt):
    banner(f"window attention 200 sequences without offsets {dt}")
    m = make([17] * 200, 4, 2, 64, dt)
    a, b = run(m, 6, 2), run(m, 6, 2, offsets=False)
    verify(m, 6, 2, b)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens,W,S,H,Hkv", [([700, 300], 8, 0, 4, 4), ([8] * 50, 100, 0, 4, 4), ([2000], 8, 1, 24, 24),
                                            ([1000], 100, 2, 4, 2)])
def test_dk_and_dv_are_two_roundings_off(lens, W, S, H, Hkv, hd):
    """bf16: the weights (or their gradients) are rounded and the result is; independent
    roundings of one relative size add up to sqrt(2) of one, which is the exact result's own."""
    banner(f"window attention roundings {lens[:3]} W={W} S={S} {H}/{Hkv} x {hd}")
    m = make(lens, H, Hkv, hd, BF16, seed=1)
    got = run(m, W, S)
    ref = reference(m["q"], m["k"], m["v"], m["dout"], seen(lens, 0, m["T"], W, S), H, Hkv, hd)
    for i in (3, 4):
        one = float((ref[i].to(torch.bfloat16).double() - ref[i]).norm())
        assert float((got[i].double() - ref[i]).norm()) < 1.05 * math.sqrt(2) * one, i


def dq_given_o(m, W, S, o):
    """dq by its formula in float64, D from the given o; per value the size (root of the sum of
    squares) of the products that it sums; per row and head the size of what its fp32 sums dP and D
    come from, |dout| times the weighted mean of |v| |k| / sqrt(hd)."""
    T, H, Hkv, hd, lens = (m[x] for x in ("T", "H", "Hkv", "hd", "lens"))
    see = seen(lens, m["first"], T, W, S)
    q, k, v, dout = (m[x].double() for x in ("q", "k", "v", "dout"))
    dq, size, sums = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((T, H), dtype=torch.float64, device=DEV)
    for h in range(H):
        a, b = slice(h * hd, (h + 1) * hd), slice(h // (H // Hkv) * hd, (h // (H // Hkv) + 1) * hd)
        s = (q[:, a] @ k[:, b].T / math.sqrt(hd)).masked_fill_(~see, -math.inf)
        P = torch.exp(s.sub_(torch.logsumexp(s, 1, keepdim=True)))
        dS = P * (dout[:, a] @ v[:, b].T - (dout[:, a] * o[:, a].double()).sum(1, keepdim=True)) / math.sqrt(hd)
        dS = torch.where(see, dS, 0.0)
        dq[:, a], size[:, a] = dS @ k[:, b], (dS.square() @ k[:, b].square()).sqrt()
        sums[:, h] = dout[:, a].norm(dim=1) * (P @ (v[:, b].norm(dim=1) * k[:, b].norm(dim=1))) / math.sqrt(hd)
    return dq, size, sums


# (lens, W, S, H, Hkv): what a call's rows and heads choose; see WIDE
DQ = [([8192], 8192, 0, 2, 1), ([4096], 512, 4, 1, 1), ([4100], 5000, 0, 4, 2), ([300, 1, 2700], 700, 3, 16, 16)]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("size", [1.0, 0.02, 1e-3, 3000.0])
@pytest.mark.parametrize("lens,W,S,H,Hkv", DQ, ids=[f"{'_'.join(map(str, a[0]))}w{a[1]}h{a[3]}" for a in DQ])
@pytest.mark.parametrize("bad", ["none", "tail", "token"])
def test_fp16_dq_is_as_exact_for_any_size_of_v_and_number_of_keys(bad, lens, W, S, H, Hkv, size, hd):
    """fp16, v of any size and weights of thousands of keys, also in workgroups that hold rows of NaN
    (behind the last sequence; one key that the rows compared do not see).

    dq is rounded to bf16, each value by at most half a step: 2^-8 of a row's norm, and over all
    rows as far off as the exact one rounded. Besides that dS is rounded to fp16, each of its products
    with k by at most 2^-11: independent, so 2^-11 of their root of the sum of squares. And dP and D are
    fp32 sums of hd products: the n-th step rounds by 2^-24 of a partial sum of size sqrt(n / hd)
    |dout||v| / sqrt(hd) (independent terms), which add up to less than 2^-24 |dout||v| for each of
    the two, however much of them cancels in dP - D: 2^-23 of `sums`. (Found to be needed where a
    row sees one key and D is off by nearly nothing: |dq| 5e-6 where |dout||v| is 2.7, off by 4e-8.)"""
    banner(f"window attention fp16 dq {bad} {lens} W={W} S={S} {H}/{Hkv} x {hd} v {size}")
    m = make(lens, H, Hkv, hd, F16, seed=W, tail=40 if bad == "tail" else 0)
    m["v"].mul_(size)
    clean = {x: m[x].clone() for x in ("q", "k", "v", "dout")}
    T, n, at = m["T"], sum(lens), sum(lens) // 2 + 5
    for x in ("q", "k", "v", "dout"):
        m[x][n:] = math.nan
    if bad == "token":
        m["k"][at], m["v"][at] = math.nan, math.inf
    o, _, dq, _, _ = run(m, W, S)
    m.update({x: clean[x] for x in clean})
    rows = torch.arange(T, device=DEV) < n
    if bad == "token":
        rows &= ~seen(lens, 0, T, W, S)[:, at]
    o[~rows] = 0.0
    want, parts, sums = dq_given_o(m, W, S, o)
    off, want, parts = (x[rows].view(-1, H, hd) for x in (dq.double() - want, want, parts))
    most = 2.0 ** -8 * want.norm(dim=2) + 2.0 ** -11 * parts.norm(dim=2) + 2.0 ** -23 * sums[rows]
    assert bool((off.norm(dim=2) <= most).all()), float((off.norm(dim=2) / most).max())
    one = float((want.to(torch.bfloat16).double() - want).norm())
    assert float(off.norm()) < 1.05 * one + 2.0 ** -11 * float(parts.norm())


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens,W,S,H,Hkv", [([300, 100], 64, 2, 2, 1), ([2000], 300, 0, 24, 24)])
def test_fp16_a_dominant_value_of_dout(lens, W, S, H, Hkv, hd):
    """One value of every dout row 2^15 times the others, in a column where v is 1: its part of dP - D
    cancels, and the gradients are those of the others.

    dP and D are fp32 sums whose terms include the dominant one, 2^12: each of their hd steps rounds by
    at most 2^-24 of 2^13, sqrt(hd) of them 2^-8 at most, where dP - D has the size sqrt(hd) / 8: less than
    2^-8 of it at hd = 64. The rest as everywhere: 4 * 2^-8 for a gradient."""
    banner(f"window attention fp16 dominant dout {lens} {H}/{Hkv} x {hd}")
    m = make(lens, H, Hkv, hd, F16, seed=5)
    T = m["T"]
    m["dout"].mul_(0.125)
    m["dout"].view(T, H, hd)[:, :, 7] = 4096.0
    m["v"].view(T, Hkv, hd)[:, :, 7] = 1.0
    o, lse, dq, dk, dv = run(m, W, S)
    assert bool((o.view(T, H, hd)[:, :, 7] == 1.0).all())  # (a mean of ones: within 2^-11 of 1, so rounded to it)
    ref = reference(m["q"], m["k"], m["v"], m["dout"], seen(lens, 0, T, W, S), H, Hkv, hd)
    for name, got, want in (("dq", dq, ref[2]), ("dk", dk, ref[3])):
        assert rel(got, want) < 5 * 2.0 ** -8, name


def test_more_workgroups_than_a_launch_holds():
    """2080 tokens of 2^18 heads are 65 x 2^16 workgroups, over the 2^22 of one launch: 130 GB of q and o."""
    banner("window attention forward of 2^18 heads")
    T, H, hd, W = 2080, 1 << 18, 64, 40
    if torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved() - torch.cuda.memory_allocated() < 160e9:
        pytest.skip("less than 160 GB of memory are free")
    torch.cuda.empty_cache()
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    q = torch.empty((T, H * hd), dtype=torch.bfloat16, device=DEV)
    for rows in q.split(130):
        rows.normal_(generator=g)
    k, v = (torch.randn((T, hd), generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    o, lse = torch.empty_like(q), torch.empty((H, T), device=DEV)
    lc.lc_window_attention_forward(BF16, BF16, T, 1, None, H, 1, hd, W, 2, q, H * hd, k, hd, v, hd, o, H * hd, lse)
    torch.cuda.synchronize()
    heads = [0, 1, 5, 4095, 100001, H // 2, H - 2, H - 1]
    qs = torch.stack([q[:, h * hd:(h + 1) * hd] for h in heads], 1).view(T, -1)
    os = torch.stack([o[:, h * hd:(h + 1) * hd] for h in heads], 1).view(T, -1)
    ref = reference(qs, k, v, torch.zeros_like(qs), seen([T], 0, T, W, 2), len(heads), 1, hd)
    assert rel(os, ref[0]) < TOL_O[BF16] and float((lse[heads].double() - ref[1]).abs().max()) < 2e-4
    del q, o, lse
    torch.cuda.empty_cache()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("tail", [0, 37])
@pytest.mark.parametrize("lens,W,S,H,Hkv", [([700, 300], 40, 0, 4, 4), ([2000, 1, 500], 300, 3, 24, 24),
                                            ([3000], 3000, 0, 10, 5), ([1000], 100, 2, 4, 2)])
def test_gradients_are_their_roundings_off(lens, W, S, H, Hkv, tail, dt, hd):
    """Independent roundings of one relative size add up in squares to that of the exact result alone:
    two for dq of bf16 (dS and the result; D given o), dv (the weights and the result) and dk of bf16 (dS
    and the result), three for dk of fp16, whose q is rounded to bf16; one for dq of fp16, whose dS has
    an eighth of its step. Rows of NaN behind the last sequence change nothing."""
    banner(f"window attention gradient roundings {lens} +{tail} W={W} S={S} {dt} {H}/{Hkv} x {hd}")
    m = make(lens, H, Hkv, hd, dt, seed=3, tail=tail)
    n = sum(lens)
    clean = {x: m[x].clone() for x in ("q", "k", "v", "dout")}
    for x in clean:
        m[x][n:] = math.nan
    o, _, dq, dk, dv = run(m, W, S)
    m.update(clean)
    ref = reference(m["q"], m["k"], m["v"], m["dout"], seen(lens, 0, m["T"], W, S), H, Hkv, hd)
    want = (dq_given_o(m, W, S, o)[0], ref[3], ref[4])
    for name, a, b, k in zip(("dq", "dk", "dv"), (dq, dk, dv), want, (2, 2, 2) if dt == BF16 else (1 + 1 / 64, 3, 2)):
        one = float((b[:n].to(torch.bfloat16).double() - b[:n]).norm())
        assert float((a[:n].double() - b[:n]).norm()) < 1.05 * math.sqrt(k) * one, name

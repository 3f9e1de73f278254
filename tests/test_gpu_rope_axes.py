"""Rotary positions with several axes against float64: head widths and sections, both
frequency layouts, far and negative positions, types, strides, in place, the table, and the
table in the projection's epilogue and the q/k norm.

Tolerances: cos and sin are within 2^-23; a rotated value a c - b s in fp32 is then off by at
most 2^-22 (|a| + |b|) with its own roundings; a 16-bit result by half a step more."""
import math

import pytest
import torch

from paper_2606_11169_amd import libchunk as lc
from tests.gpu_util import DEV, banner

pytestmark = pytest.mark.gpu
F32, BF16, F16 = lc.LC_FP32, lc.LC_BF16, lc.LC_FP16
DT = {F32: torch.float32, BF16: torch.bfloat16, F16: torch.float16}
STEP = {F32: 0.0, BF16: 2.0 ** -8, F16: 2.0 ** -11}
HEAD, AXIS = lc.LC_ROPE_FREQ_HEAD, lc.LC_ROPE_FREQ_AXIS


def angles(pos, hd, sections, freq, base):
    """[T, hd/2] angles in float64."""
    half = hd // 2
    a = torch.zeros((pos.shape[1], half), dtype=torch.float64, device=DEV)
    i = 0
    for ax, n in enumerate(sections):
        for j in range(n):
            f = base ** (-(j / n if freq == AXIS else i / half))
            a[:, i] = pos[ax].double() * f
            i += 1
    return a


def rotated(x, T, heads, hd, a, sign):
    z = x.double().view(T, heads, 2, hd // 2)
    c, s = torch.cos(a)[:, None], sign * torch.sin(a)[:, None]
    return torch.stack([z[:, :, 0] * c - z[:, :, 1] * s, z[:, :, 1] * c + z[:, :, 0] * s], 2).view(T, heads * hd)


@pytest.mark.parametrize("T,heads,hd,sections,freq,base", [
    (1, 1, 2, [1], HEAD, 10000.0), (5, 3, 128, [16, 24, 24], HEAD, 1e6), (33, 40, 128, [16, 24, 24], HEAD, 1e6),
    (130, 24, 64, [8, 10, 10], AXIS, 10000.0), (17, 5, 72, [12, 12, 12], AXIS, 100.0), (9, 2, 80, [40], HEAD, 5e5),
    (64, 7, 96, [10, 0, 9, 20], HEAD, 10000.0), (3, 1, 256, [32, 48, 48], HEAD, 1e6), (21, 3, 20, [3, 3, 3], AXIS, 1.0),
    (11, 65, 16, [1, 2, 3], AXIS, 10000.0), (2049, 2, 32, [4, 6, 6], HEAD, 10000.0), (6, 9, 6, [1, 1], HEAD, 50.0)])
@pytest.mark.parametrize("xt,yt", [(BF16, BF16), (F16, F16), (F32, F32), (F32, BF16)])
def test_forward_and_backward(T, heads, hd, sections, freq, base, xt, yt):
    banner(f"rope axes T={T} heads={heads} hd={hd} {sections} {freq} {xt}{yt}")
    g = torch.Generator(device=DEV)
    g.manual_seed(T + heads)
    width = heads * hd
    pos = torch.randint(-40, 5000, (len(sections), T + 3), generator=g, device=DEV, dtype=torch.int32)
    a = angles(pos[:, :T], hd, sections, freq, base)
    for ldx, ldy in ((width, width), (width + 8, width + 16), (width + 3, width + 1)):
        x = torch.full((T, ldx), 3.0, device=DEV, dtype=DT[xt])
        x[:, :width] = torch.randn((T, width), generator=g, device=DEV).to(DT[xt])
        for fn, sign in ((lc.lc_rope_axes_forward, 1), (lc.lc_rope_axes_backward, -1)):
            y = torch.full((T, ldy), 7.0, device=DEV, dtype=DT[yt])
            fn(T, heads, hd, sections, pos, T + 3, x, ldx, y, ldy, xt, yt, base=base, freq=freq)
            ref = rotated(x[:, :width].contiguous(), T, heads, hd, a, sign)
            far = (x[:, :width].double().abs().view(T, heads, 2, hd // 2).sum(2, keepdim=True)
                   .expand(-1, -1, 2, -1).reshape(T, width))
            bound = far * 2.0 ** -22 + ref.abs() * STEP[yt] + (2.0 ** -25 if yt == F16 else 0)
            assert bool(((y[:, :width].double() - ref).abs() <= bound).all())
            assert bool((y[:, width:] == 7.0).all())
            if xt == yt and ldx == ldy:  # in place: the same bits
                z = x.clone()
                fn(T, heads, hd, sections, pos, T + 3, z, ldx, z, ldx, xt, yt, base=base, freq=freq)
                assert torch.equal(z, y)


@pytest.mark.parametrize("hd,sections,freq,base", [(128, [16, 24, 24], HEAD, 1e6), (64, [8, 12, 12], AXIS, 10000.0),
                                                   (10, [2, 1], HEAD, 10000.0), (256, [128], HEAD, 1.0)])
def test_table_at_far_positions(hd, sections, freq, base):
    """Positions over the whole int32 range; the reference's angles are reduced with integers
    of any size: pos * f / (2 pi) as a fraction with 200 bits."""
    banner(f"rope axes table hd={hd} {sections}")
    from fractions import Fraction
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    half, T = hd // 2, 9
    vals = [0, 1, -1, 1 << 20, (1 << 24) + 1, 123456789, (1 << 31) - 1, -(1 << 31), -77777777]
    pos = torch.tensor([vals] * len(sections), dtype=torch.int32, device=DEV)
    cos, sin = (torch.full((T, half), 9.0, device=DEV) for _ in range(2))
    lc.lc_rope_axes_table(T, hd, sections, pos, T, cos, sin, base=base, freq=freq)
    pi = Fraction(Decimal("3.14159265358979323846264338327950288419716939937510582097494"))
    i, worst = 0, 0.0
    for ax, n in enumerate(sections):
        for j in range(n):
            e = Fraction(j, n) if freq == AXIS else Fraction(i, half)
            f = Decimal(base) ** (-(Decimal(e.numerator) / Decimal(e.denominator)))
            for t, p in enumerate(vals):
                x = p * Fraction(f) / (2 * pi)
                x -= round(x)
                ang = float(2 * pi * x)
                worst = max(worst, abs(float(cos[t, i]) - math.cos(ang)), abs(float(sin[t, i]) - math.sin(ang)))
            i += 1
    assert worst <= 2.0 ** -23
    assert bool((cos[:, i:] == 1).all()) and bool((sin[:, i:] == 0).all())


def test_table_makes_the_fused_rotations_turn_by_axes():
    """The projection's epilogue (rope_seq = T) and the q/k norm (seq_len = T) with the table."""
    banner("rope axes table in lc_gemm and lc_qk_norm_rope_forward")
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    T, H, Hkv, hd, d = 200, 4, 2, 128, 256
    cols, rope_cols = (H + 2 * Hkv) * hd, (H + Hkv) * hd
    sections, base = [16, 24, 24], 1e6
    pos = torch.randint(0, 3000, (3, T), generator=g, device=DEV, dtype=torch.int32)
    cos, sin = (torch.empty((T, hd // 2), device=DEV) for _ in range(2))
    lc.lc_rope_axes_table(T, hd, sections, pos, T, cos, sin, base=base)
    x = torch.randn((T, d), generator=g, device=DEV).to(torch.bfloat16)
    w = (torch.randn((cols, d), generator=g, device=DEV) * 0.06).to(torch.bfloat16)
    fused, plain = (torch.empty((T, cols), dtype=torch.float32, device=DEV) for _ in range(2))
    lc.lc_gemm(BF16, lc.LC_EPI_ROPE, T, cols, d, x, d, 1, w, d, 1, fused, cols, rope_cos=cos, rope_sin=sin,
               rope_seq=T, rope_cols=rope_cols, head_dim=hd, c_dtype=F32)
    lc.lc_gemm(BF16, lc.LC_EPI_STORE_F32, T, cols, d, x, d, 1, w, d, 1, plain, cols)
    a = angles(pos, hd, sections, HEAD, base)
    ref = rotated(plain[:, :rope_cols].contiguous(), T, H + Hkv, hd, a, 1)
    assert float((fused[:, :rope_cols].double() - ref).norm() / ref.norm()) < 1e-6
    lc.lc_rope_axes_forward(T, H + Hkv, hd, sections, pos, T, plain, cols, plain, cols, F32, F32, base=base)
    assert float((plain[:, :rope_cols].double() - ref).norm() / ref.norm()) < 1e-6
    assert torch.equal(plain[:, rope_cols:], fused[:, rope_cols:])
    qk = torch.randn((T, rope_cols), generator=g, device=DEV)
    y, raw, rstd = qk.clone(), torch.empty_like(qk), torch.empty((T, H + Hkv), device=DEV)
    one = torch.ones(hd, device=DEV)
    lc.lc_qk_norm_rope_forward(T, H, Hkv, hd, T, 1e-6, y, rope_cols, raw, rstd, one, one, F32, F32, cos, sin)
    n = qk.double().view(T, H + Hkv, hd)
    n = n * (n.square().mean(2, keepdim=True) + 1e-6).rsqrt()
    ref = rotated(n.reshape(T, -1), T, H + Hkv, hd, a, 1)
    assert float((y.double() - ref).norm() / ref.norm()) < 1e-6


def test_captured_and_replayed():
    banner("rope axes graph")
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    T, heads, hd = 77, 10, 64
    pos = torch.randint(0, 100, (3, T), generator=g, device=DEV, dtype=torch.int32)
    x = torch.randn((T, heads * hd), generator=g, device=DEV).to(torch.bfloat16)
    y, z = torch.empty_like(x), torch.empty_like(x)
    cos, sin = (torch.empty((T, hd // 2), device=DEV) for _ in range(2))

    def calls(st):
        lc.lc_rope_axes_forward(T, heads, hd, [8, 12, 12], pos, T, x, heads * hd, y, heads * hd, BF16, BF16, stream=st)
        lc.lc_rope_axes_backward(T, heads, hd, [8, 12, 12], pos, T, x, heads * hd, z, heads * hd, BF16, BF16, stream=st)
        lc.lc_rope_axes_table(T, hd, [8, 12, 12], pos, T, cos, sin, stream=st)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls(side)
    for i in range(3):
        pos.copy_(torch.randint(0, 1000, (3, T), generator=g, device=DEV, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, z, cos, sin)]
        for t in (y, z, cos, sin):
            t.zero_()
        calls(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, z, cos, sin)))


def test_no_tokens():
    banner("rope axes T=0")
    lc.lc_rope_axes_forward(0, 2, 64, [32], None, 0, None, 128, None, 128, BF16, BF16)
    lc.lc_rope_axes_table(0, 64, [32], None, 0, None, None)
    torch.cuda.synchronize()


@pytest.mark.parametrize("T,heads,hd,sections", [(5, 3, 128, [16, 24, 10]), (40, 9, 64, [8, 9, 10]), (7, 2, 6, [1, 1]),
                                                 (9, 4, 256, [30, 0, 40, 20]), (3, 5, 130, [64]), (33, 2, 72, [7])])
@pytest.mark.parametrize("dt", [F32, BF16, F16])
def test_pairs_past_the_sections_stay_as_they_are(T, heads, hd, sections, dt):
    """Bit for bit (NaN: NaN), also beside an infinite, NaN or negative value of their pair, and with
    the sign of zero."""
    banner(f"rope axes pairs past the sections T={T} heads={heads} hd={hd} {sections} {dt}")
    g = torch.Generator(device=DEV)
    g.manual_seed(hd)
    n, half, width = sum(sections), hd // 2, heads * hd
    pos = torch.randint(-40, 5000, (len(sections), T), generator=g, device=DEV, dtype=torch.int32)
    x = torch.randn((T, heads, 2, half), generator=g, device=DEV).to(DT[dt])
    for i, v in enumerate((math.inf, -math.inf, math.nan, -0.0, 0.0)):
        x[i % T, :, 0, n + i % (half - n)] = v
        x[(i + 1) % T, :, 1, n + (i + 2) % (half - n)] = v
    for fn in (lc.lc_rope_axes_forward, lc.lc_rope_axes_backward):
        y = torch.full_like(x, 3.0)
        fn(T, heads, hd, sections, pos, T, x, width, y, width, dt, dt)
        a, b = x[..., n:], y[..., n:]
        ints = torch.int32 if dt == F32 else torch.int16
        same = a.contiguous().view(ints) == b.contiguous().view(ints)
        assert bool((same | (a.isnan() & b.isnan())).all())
        assert bool(y[..., :n].isfinite().all())

"""LayerNorm forward and backward against float64: row lengths around the kernels' row
shapes and block edges, odd widths, strides, type mixes, in-place calls, constant and
far-off-zero rows, gradients against differences, captured graphs.

Tolerances: fp32 results are sums of d (or T) terms in fp32; with the partial sums of a
few dozen terms each that the kernels use, their error is some 2^-24 times the root of
the number of steps, 1e-6 normwise with room. A 16-bit result is off by at most half a
step more (bf16 2^-8, fp16 2^-11). dx is a difference: r (t - mean t - xh mean(t xh)) with each
term rounded by 2^-24 of its size, however much of them cancels (of two values all but
eps / variance does: xh = +-1 and t lies in the span of the two terms taken off), so its fp32
error is measured against the size of r t where that is larger than dx itself."""
import math

import pytest
import torch

from paper_2606_11169_amd import libchunk as lc
from tests.gpu_util import DEV, banner

pytestmark = pytest.mark.gpu
F32, BF16, F16 = lc.LC_FP32, lc.LC_BF16, lc.LC_FP16
DT = {F32: torch.float32, BF16: torch.bfloat16, F16: torch.float16}
STEP = {F32: 1e-6, BF16: 2.0 ** -8 + 1e-6, F16: 2.0 ** -11 + 1e-6}
EPS = 1e-5


def rel(a, b):
    n = float(b.norm())
    return float((a.double() - b).norm()) / (n if n else 1.0)


def rel_dx(a, b, r, dy, gain, ot):
    """The error of dx in units of its tolerance: the fp32 part against max(|dx|, |r t|), the
    rounding to a 16-bit type against |dx|."""
    t = float((r[:, None] * (dy.double() * gain.double())).norm())
    n = float(b.norm())
    return float((a.double() - b).norm()) / (1e-6 * max(n, t) + (STEP[ot] - 1e-6) * n)


def rows(g, T, d, dt, ld, scale=1.0, shift=0.0):
    """[T, d] values of type dt at row stride ld (a view of a larger buffer)."""
    buf = torch.full((T, ld), 77.0, device=DEV, dtype=DT[dt])
    buf[:, :d] = (torch.randn((T, d), generator=g, device=DEV) * scale + shift).to(DT[dt])
    return buf


def reference(x, g, b, dy, dres):
    mu = x.mean(1, keepdim=True)
    r = ((x - mu).square().mean(1, keepdim=True) + EPS).rsqrt()
    xh = (x - mu) * r
    y = xh * g + (0 if b is None else b)
    t = dy * g
    dx = r * (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True))
    return y, mu[:, 0], r[:, 0], dx + (0 if dres is None else dres), (dy * xh).sum(0), dy.sum(0)


def run(T, d, x, g, b, dy, dres, types, lds=(0, 0, 0, 0, 0), dg=None, db=None, copy=None, store=0,
        y=None, dx=None, stream=None):
    xt, wt, yt, dyt, rt, ot = types
    lx, ly, ldy, lr, lo = lds
    y = torch.empty((T, ly or d), dtype=DT[yt], device=DEV) if y is None else y
    dx = torch.empty((T, lo or d), dtype=DT[ot], device=DEV) if dx is None else dx
    mean, rstd = (torch.empty(T, device=DEV) for _ in range(2))
    n = lc.lc_layernorm_scratch_bytes(T, d)
    scratch = torch.full((n // 4 + 64,), -3.0, device=DEV)
    lc.lc_layernorm_forward(T, d, x, g, b, EPS, y, mean, rstd, xt, wt, yt, ld_x=lx, ld_y=ly, stream=stream)
    lc.lc_layernorm_backward(T, d, dy, x, mean, rstd, g, dres, dx, dg, db, scratch, n, dyt, xt, wt,
                             rt, ot, dx_copy=copy, store_dg=store, ld_x=lx, ld_dy=ldy, ld_dres=lr,
                             ld_dx=lo, stream=stream)
    return y, mean, rstd, dx, scratch, n


@pytest.mark.parametrize("types", [(F32, BF16, BF16, F32, F32, F32), (BF16, BF16, BF16, BF16, BF16, BF16),
                                   (F32, F32, F32, F32, F32, F32), (F16, F32, F16, BF16, F16, F16)],
                         ids=["stream", "bf16", "fp32", "mixed"])
@pytest.mark.parametrize("T,d", [(1, 1), (3, 2), (1, 8), (17, 63), (9, 64), (33, 520), (16, 768), (7, 1025),
                                 (40, 2048), (5, 2056), (31, 4104), (18, 8192), (6, 8200), (3, 16385),
                                 (2, 40000), (1200, 96), (2500, 24)])
def test_forward_and_backward(T, d, types):
    banner(f"layernorm T={T} d={d} {types}")
    g = torch.Generator(device=DEV)
    g.manual_seed(T * 7 + d)
    xt, wt, yt, dyt, rt, ot = types
    x, dy, dres = rows(g, T, d, xt, d, 1.5, 0.7), rows(g, T, d, dyt, d), rows(g, T, d, rt, d)
    gain = (1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(DT[wt])
    bias = (0.1 * torch.randn(d, generator=g, device=DEV)).to(DT[wt])
    dg0, db0 = torch.randn(d, generator=g, device=DEV), torch.randn(d, generator=g, device=DEV)
    dg, db = dg0.clone(), db0.clone()
    copy = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    y, mean, rstd, dx, scratch, n = run(T, d, x, gain, bias, dy, dres, types, dg=dg, db=db, copy=copy)
    ry, rm, rr, rdx, rdg, rdb = reference(x.double(), gain.double(), bias.double(), dy.double(), dres.double())
    assert rel(y, ry) < STEP[yt]
    assert rel(mean, rm) < 1e-6 and rel(rstd, rr) < 1e-6
    assert rel_dx(dx, rdx, rr, dy, gain, ot) < 1
    assert rel_dx(copy, rdx, rr, dy, gain, BF16) < 1
    assert rel(dg, dg0.double() + rdg) < 1e-6 and rel(db, db0.double() + rdb) < 1e-6
    assert bool((scratch[n // 4:] == -3.0).all())
    # again, stored, without a residual, bias and copy, into the same values every run
    a, b = torch.full((d,), 9.0, device=DEV), torch.full((d,), 9.0, device=DEV)
    y, _, _, dx, _, _ = run(T, d, x, gain, None, dy, None, types, dg=a, db=b, store=1)
    assert rel(y, ry - bias.double()) < STEP[yt]
    assert rel_dx(dx, rdx - dres.double(), rr, dy, gain, ot) < 1
    assert rel(a, rdg) < 1e-6 and rel(b, rdb) < 1e-6
    a2, b2 = torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    dx2 = run(T, d, x, gain, None, dy, None, types, dg=a2, db=b2, store=1)[3]
    assert torch.equal(a, a2) and torch.equal(b, b2) and torch.equal(dx, dx2)


@pytest.mark.parametrize("T,d,lds", [(33, 512, (520, 528, 536, 544, 552)), (33, 512, (513, 512, 515, 0, 517)),
                                     (9, 77, (80, 78, 77, 79, 81)), (5, 9000, (9008, 9008, 0, 9016, 9000))])
def test_strides_and_one_gradient_alone(T, d, lds):
    banner(f"layernorm strides T={T} d={d} {lds}")
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    full = [v or d for v in lds]
    types = (BF16, F32, F32, F32, BF16, BF16)
    x, dy, dres = rows(g, T, d, BF16, full[0]), rows(g, T, d, F32, full[2]), rows(g, T, d, BF16, full[3])
    gain, bias = 1 + 0.1 * torch.randn(d, generator=g, device=DEV), torch.randn(d, generator=g, device=DEV)
    y = torch.full((T, full[1]), 5.0, device=DEV)
    dx = torch.full((T, full[4]), 5.0, dtype=torch.bfloat16, device=DEV)
    dg = torch.zeros(d, device=DEV)
    run(T, d, x, gain, bias, dy, dres, types, lds=lds, dg=dg, y=y, dx=dx)
    ry, _, _, rdx, rdg, rdb = reference(x[:, :d].double(), gain.double(), bias.double(), dy[:, :d].double(),
                                        dres[:, :d].double())
    assert rel(y[:, :d], ry) < 1e-6 and rel(dx[:, :d], rdx) < STEP[BF16] and rel(dg, rdg) < 1e-6
    assert bool((y[:, d:] == 5.0).all()) and bool((dx[:, d:] == 5.0).all())
    db = torch.zeros(d, device=DEV)
    run(T, d, x, gain, bias, dy, dres, types, lds=lds, db=db)
    assert rel(db, rdb) < 1e-6


@pytest.mark.parametrize("T,d", [(37, 1024), (20, 331), (6, 9216)])
def test_in_place(T, d):
    banner(f"layernorm in place T={T} d={d}")
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    types = (F32,) * 6
    x, dy, dres = rows(g, T, d, F32, d), rows(g, T, d, F32, d), rows(g, T, d, F32, d)
    gain, bias = 1 + 0.1 * torch.randn(d, generator=g, device=DEV), torch.randn(d, generator=g, device=DEV)
    dg, db = torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    y, _, _, dx, _, _ = run(T, d, x, gain, bias, dy, dres, types, dg=dg, db=db)
    for over in (dy, dres):
        a, b, r = torch.zeros(d, device=DEV), torch.zeros(d, device=DEV), over.clone()
        args = [r if over is t else t for t in (dy, dres)]
        run(T, d, x, gain, bias, *args, types, dg=a, db=b, dx=r)
        assert torch.equal(r, dx) and torch.equal(a, dg) and torch.equal(b, db)
    xs = x.clone()
    mean, rstd = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    lc.lc_layernorm_forward(T, d, xs, gain, bias, EPS, xs, mean, rstd, F32, F32, F32)
    assert torch.equal(xs, y)


@pytest.mark.parametrize("d", [64, 1000, 4096, 10000])
def test_rows_far_from_zero_and_constant_rows(d):
    """The variance comes from differences to the mean: rows at 4096 with a spread of 1 (their
    squares' sum would lose it), and constant rows (variance 0: y = b, finite gradients)."""
    banner(f"layernorm far rows d={d}")
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    T = 6
    x = rows(g, T, d, F32, d, 1.0, 4096.0)
    x[3] = 0.5
    dy = rows(g, T, d, F32, d)
    gain, bias = torch.ones(d, device=DEV), torch.zeros(d, device=DEV)
    y, mean, rstd, dx, _, _ = run(T, d, x, gain, bias, dy, None, (F32,) * 6)
    ry, rm, rr, rdx, _, _ = reference(x.double(), gain.double(), bias.double(), dy.double(), None)
    keep = [0, 1, 2, 4, 5]
    # the mean itself is held to half a step of 4096 (2^-12), which shifts a row of spread 1 by that
    assert rel(y[keep], ry[keep]) < 2.0 ** -11 and rel(rstd[keep], rr[keep]) < 1e-5
    assert rel(dx[keep], rdx[keep]) < 2.0 ** -10
    assert float(y[3].abs().max()) < 1e-3 and bool(torch.isfinite(dx).all())


def test_gradient_against_differences():
    banner("layernorm differences")
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    T, d = 7, 72
    x, dy, u = (rows(g, T, d, F32, d) for _ in range(3))
    gain, bias = 1 + 0.1 * torch.randn(d, generator=g, device=DEV), torch.randn(d, generator=g, device=DEV)
    dg, db = torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    dx = run(T, d, x, gain, bias, dy, None, (F32,) * 6, dg=dg, db=db)[3]

    def loss(xx, gg, bb):
        y = torch.empty_like(xx)
        m, r = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        lc.lc_layernorm_forward(T, d, xx, gg, bb, EPS, y, m, r, F32, F32, F32)
        return float((y.double() * dy.double()).sum())

    h = 1e-2  # truncation h^2, rounding 500 * 2^-24 / h: both well under 1e-3 of the gradient's size
    ug, ub = torch.randn(d, generator=g, device=DEV), torch.randn(d, generator=g, device=DEV)
    for num, ana in (((loss(x + h * u, gain, bias) - loss(x - h * u, gain, bias)) / (2 * h), (dx * u).sum()),
                     ((loss(x, gain + h * ug, bias) - loss(x, gain - h * ug, bias)) / (2 * h), (dg * ug).sum()),
                     ((loss(x, gain, bias + h * ub) - loss(x, gain, bias - h * ub)) / (2 * h), (db * ub).sum())):
        assert abs(num - float(ana)) < 5e-3 * max(1.0, abs(float(ana)))


def test_captured_and_replayed_on_another_stream():
    banner("layernorm graph")
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    T, d = 300, 640
    types = (BF16, BF16, BF16, BF16, BF16, BF16)
    x, dy, dres = (rows(g, T, d, BF16, d) for _ in range(3))
    gain, bias = torch.ones(d, dtype=torch.bfloat16, device=DEV), torch.zeros(d, dtype=torch.bfloat16, device=DEV)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    dg, db = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    n = lc.lc_layernorm_scratch_bytes(T, d)
    scratch = torch.empty(n, dtype=torch.uint8, device=DEV)

    def calls(st):
        lc.lc_layernorm_forward(T, d, x, gain, bias, EPS, y, mean, rstd, BF16, BF16, BF16, stream=st)
        lc.lc_layernorm_backward(T, d, dy, x, mean, rstd, gain, dres, dx, dg, db, scratch, n, BF16, BF16, BF16,
                                 BF16, BF16, store_dg=1, stream=st)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls(side)
    for i in range(4):
        x.copy_((torch.randn((T, d), generator=g, device=DEV) * (i + 1)).to(torch.bfloat16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, mean, rstd, dg, db)]
        for t in (y, dx, mean, rstd, dg, db):
            t.fill_(3.0)
        scratch.fill_(255)
        calls(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, mean, rstd, dg, db)))


def test_no_rows():
    banner("layernorm T=0")
    dg = torch.full((8,), 2.0, device=DEV)
    one = torch.ones(8, device=DEV)
    lc.lc_layernorm_forward(0, 8, None, one, None, EPS, None, None, None, F32, F32, F32)
    lc.lc_layernorm_backward(0, 8, None, None, None, None, one, None, None, dg, None, None, 0, F32, F32, F32,
                             F32, F32)
    torch.cuda.synchronize()
    assert bool((dg == 2.0).all())


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("T,d", [(300, 1155), (40, 2049), (40, 4099), (300, 8195), (20, 9001), (20, 12289), (20, 16383)])
def test_dx_over_dres_in_rows_of_no_whole_runs(T, d, out):
    """The last run of such a row shares values with the one before, which other lanes hold."""
    banner(f"layernorm dx over dres T={T} d={d} {out}")
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    x, dy, dres = rows(g, T, d, BF16, d), rows(g, T, d, BF16, d), rows(g, T, d, out, d)
    gain = rows(g, 1, d, F32, d)[0]
    types = (BF16, F32, BF16, BF16, out, out)
    want = run(T, d, x, gain, None, dy, dres, types)[3]
    for _ in range(3):
        over = dres.clone()
        run(T, d, x, gain, None, dy, over, types, dx=over)
        assert torch.equal(over, want)


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("T,d", [(40, 1537), (40, 4097), (30, 8191), (30, 8193), (30, 8195), (20, 8711), (20, 12289), (9, 16383)])
def test_copy_of_dx_over_dres_in_rows_of_no_whole_runs(T, d, out):
    """dx_copy where dx lies over dres, at lengths whose last run shares values with another wave's
    (8193 to 8199, 8705 to 8711, ...: with the wave of another of its runs)."""
    banner(f"layernorm copy of dx over dres T={T} d={d} {out}")
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    x, dy, dres = rows(g, T, d, BF16, d), rows(g, T, d, BF16, d), rows(g, T, d, out, d)
    gain = rows(g, 1, d, F32, d)[0]
    types = (BF16, F32, BF16, BF16, out, out)
    copy = torch.full((T + 1, d), 5.0, dtype=torch.bfloat16, device=DEV)
    want = run(T, d, x, gain, None, dy, dres, types, copy=copy)[3]
    assert torch.equal(copy[:T], want.to(torch.bfloat16)) and bool((copy[T] == 5.0).all())
    for _ in range(3):
        over, copy = dres.clone(), torch.full((T + 1, d), 5.0, dtype=torch.bfloat16, device=DEV)
        run(T, d, x, gain, None, dy, over, types, dx=over, copy=copy)
        assert torch.equal(over, want)
        assert torch.equal(copy[:T], want.to(torch.bfloat16)) and bool((copy[T] == 5.0).all())


@pytest.mark.parametrize("d", [70001, 1 << 20, (1 << 24) - 3])
def test_long_rows_of_equal_values(d):
    """Rows of one value: y is the bias, and with equal dy g the row's dx is 0. A thread's compensated sum
    is off by some 2^-23 of itself and eight more additions join the threads' (2^-24 each), so the mean is
    off by less than 2^-20 of the value, y by that over sqrt(eps), which also bounds xh; dx = r (t - mean t
    - xh mean(t xh)): 2^-20 |t| r for the first two terms, less for the third."""
    banner(f"layernorm long rows of equal values d={d}")
    T, r = 3, EPS ** -0.5
    x = torch.tensor([0.1, -0.7, 0.3], device=DEV)[:, None].expand(T, d).contiguous()
    dy = torch.tensor([0.3, 0.1, -1.1], device=DEV)[:, None].expand(T, d).contiguous()
    gain, bias = torch.ones(d, device=DEV), torch.zeros(d, device=DEV)
    y, mean, _, dx, _, _ = run(T, d, x, gain, bias, dy, None, (F32,) * 6)
    at = 2.0 ** -20
    assert bool(((mean - x[:, 0]).abs() <= at * x[:, 0].abs()).all())
    assert float(y.abs().max()) <= at * 0.7 * r
    assert float(dx.abs().max()) <= 2 * at * 1.1 * r


def test_more_long_rows_than_a_launch_holds():
    """Rows of over 8192 values are a workgroup of 1024 threads each: 2^22 of them (69 GB, in place) are
    2^32 work-items, one more than a launch takes."""
    T, d = (1 << 22) + 3, 8200
    banner(f"layernorm forward T={T} d={d}")
    if torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved() - torch.cuda.memory_allocated() < 100e9:
        pytest.skip("less than 100 GB of memory are free")
    torch.cuda.empty_cache()
    g = torch.Generator(device=DEV)
    g.manual_seed(9)
    x = torch.empty((T, d), dtype=torch.bfloat16, device=DEV)
    for part in x.split(1 << 17):
        part.normal_(generator=g)
    gain = 1 + 0.1 * torch.randn(d, generator=g, device=DEV)
    at = torch.tensor([0, 1, (1 << 21) - 1, 1 << 21, (1 << 22) - 1, 1 << 22, T - 1], device=DEV)
    was = x[at].double()
    mean, rstd = (torch.full((T,), -7.0, device=DEV) for _ in range(2))
    lc.lc_layernorm_forward(T, d, x, gain, None, EPS, x, mean, rstd, BF16, F32, BF16)
    torch.cuda.synchronize()
    y, m, r = reference(was, gain.double(), None, was, None)[:3]
    assert rel(x[at], y) < STEP[BF16] and rel(mean[at], m) < 1e-5 and rel(rstd[at], r) < 1e-6
    assert bool((rstd > 0).all())
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("d", [3, 300, 70001, 1 << 20])
def test_infinite_values_stay_in_their_row(d):
    """Rows with an infinite value have an infinite mean, whatever holds them, and a NaN output; both
    signs, or a NaN, a NaN mean. Their neighbours are what they were."""
    banner(f"layernorm infinite values d={d}")
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    T, gain, bias = 6, torch.ones(d, device=DEV), torch.zeros(d, device=DEV)
    x, dy = rows(g, T, d, F32, d), rows(g, T, d, F32, d)
    y, mean, rstd, dx, _, _ = run(T, d, x, gain, bias, dy, None, (F32,) * 6)
    bad = x.clone()
    bad[1, d // 2], bad[2, d - 1], bad[4, 0] = math.inf, -math.inf, math.nan
    bad[5, 0], bad[5, d - 1] = math.inf, -math.inf
    yb, mb, rb, dxb, _, _ = run(T, d, bad, gain, bias, dy, None, (F32,) * 6)
    assert float(mb[1]) == math.inf and float(mb[2]) == -math.inf and bool(mb[4:].isnan().all())
    assert bool(yb[[1, 2, 4, 5]].isnan().all())
    keep = [0, 3]
    assert torch.equal(yb[keep], y[keep]) and torch.equal(mb[keep], mean[keep])
    assert torch.equal(rb[keep], rstd[keep]) and torch.equal(dxb[keep], dx[keep])

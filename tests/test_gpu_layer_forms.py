"""LayerNorm, the projection, rotary positions of three axes and sliding-window attention as
a layer's attention half uses them, forward and backward, on a packed batch with a padded end,
against float64 with autograd.

Tolerance: every tensor between the operators is rounded to bf16 once (half a step, 2^-8); the
forward passes five of them (n, qkv, rotated qkv, o, weights), the backward five more, each
adding in squares: sqrt(10) * 2^-8 * (their mean of 0.6 of a half step) < 2^-7 forward, and twice
that backward."""
import math

import pytest
import torch

from paper_2606_11169_amd import libchunk as lc
from tests.gpu_util import DEV, banner

pytestmark = pytest.mark.gpu
F32, BF16 = lc.LC_FP32, lc.LC_BF16


@pytest.mark.parametrize("fused", [False, True])
def test_attention_half_of_a_layer(fused):
    banner(f"layer forms fused={fused}")
    g = torch.Generator(device=DEV)
    g.manual_seed(21)
    lens, tail, H, Hkv, hd, W, S = [150, 1, 210], 7, 4, 2, 128, 64, 4
    T, d, cols, rc = sum(lens) + tail, 512, (H + 2 * Hkv) * hd, (H + Hkv) * hd
    sections, base = [16, 24, 24], 1e6
    off = torch.tensor([0, 150, 151, 361], dtype=torch.int32, device=DEV)
    pos = torch.randint(0, 500, (3, T), generator=g, device=DEV, dtype=torch.int32)
    x = torch.randn((T, d), generator=g, device=DEV)
    dy = torch.randn((T, d), generator=g, device=DEV)
    dy[sum(lens):] = 0
    gain, bias = 1 + 0.1 * torch.randn(d, generator=g, device=DEV), 0.1 * torch.randn(d, generator=g, device=DEV)
    w = (torch.randn((cols, d), generator=g, device=DEV) * d ** -0.5).to(torch.bfloat16)
    wo = (torch.randn((d, H * hd), generator=g, device=DEV) * d ** -0.5).to(torch.bfloat16)
    bf = dict(dtype=torch.bfloat16, device=DEV)

    # forward
    n, mean, rstd = torch.empty((T, d), **bf), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    lc.lc_layernorm_forward(T, d, x, gain, bias, 1e-5, n, mean, rstd, F32, F32, BF16)
    qkv = torch.empty((T, cols), **bf)
    if fused:
        cos, sin = (torch.empty((T, hd // 2), device=DEV) for _ in range(2))
        lc.lc_rope_axes_table(T, hd, sections, pos, T, cos, sin, base=base)
        lc.lc_gemm(BF16, lc.LC_EPI_ROPE, T, cols, d, n, d, 1, w, d, 1, qkv, cols, rope_cos=cos, rope_sin=sin,
                   rope_seq=T, rope_cols=rc, head_dim=hd)
    else:
        lc.lc_gemm(BF16, lc.LC_EPI_STORE, T, cols, d, n, d, 1, w, d, 1, qkv, cols)
        lc.lc_rope_axes_forward(T, H + Hkv, hd, sections, pos, T, qkv, cols, qkv, cols, BF16, BF16, base=base)
    q, k, v = qkv, qkv[:, H * hd:], qkv[:, rc:]
    o, lse = torch.zeros((T, H * hd), **bf), torch.empty((H, T), device=DEV)
    lc.lc_window_attention_forward(BF16, BF16, T, 3, off, H, Hkv, hd, W, S, q, cols, k, cols, v, cols, o, H * hd, lse)
    y = torch.empty((T, d), device=DEV)
    lc.lc_gemm(BF16, lc.LC_EPI_RESIDUAL, T, d, H * hd, o, H * hd, 1, wo, H * hd, 1, y, d, R=x, ldr=d, c_dtype=F32,
               r_dtype=F32)
    # backward
    dy16, do = dy.to(torch.bfloat16), torch.empty((T, H * hd), **bf)
    lc.lc_gemm(BF16, lc.LC_EPI_STORE, T, H * hd, d, dy16, d, 1, wo, H * hd, 0, do, H * hd)
    dqkv = torch.zeros((T, cols), **bf)
    nb = lc.lc_window_attention_scratch_bytes(BF16, T, H, Hkv, hd, W, S)
    scratch = torch.empty(nb, dtype=torch.uint8, device=DEV)
    lc.lc_window_attention_backward(BF16, BF16, T, 3, off, H, Hkv, hd, W, S, q, cols, k, cols, v, cols, o, H * hd, lse,
                                    do, H * hd, dqkv, cols, dqkv[:, H * hd:], cols, dqkv[:, rc:], cols, scratch, nb)
    lc.lc_rope_axes_backward(T, H + Hkv, hd, sections, pos, T, dqkv, cols, dqkv, cols, BF16, BF16, base=base)
    dn = torch.empty((T, d), device=DEV)
    lc.lc_gemm(BF16, lc.LC_EPI_STORE_F32, T, d, cols, dqkv, cols, 1, w, d, 0, dn, d)
    # (a product over the batch's rows wants a multiple of 8: 368)
    dw = torch.zeros((cols, d), device=DEV)
    lc.lc_gemm(BF16, lc.LC_EPI_ACCUM_F32, cols, d, T, dqkv, cols, 0, n, d, 0, dw, d)
    dx, dg, db = torch.empty((T, d), device=DEV), torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    ns = lc.lc_layernorm_scratch_bytes(T, d)
    sc = torch.empty(ns, dtype=torch.uint8, device=DEV)
    lc.lc_layernorm_backward(T, d, dn, x, mean, rstd, gain, dy, dx, dg, db, sc, ns, F32, F32, F32, F32, F32)
    torch.cuda.synchronize()

    # float64, on the CPU
    X, Gn, Bn, Wq = (t.double().cpu().requires_grad_() for t in (x, gain, bias, w))
    mu = X.mean(1, keepdim=True)
    N = (X - mu) * ((X - mu).square().mean(1, keepdim=True) + 1e-5).rsqrt() * Gn + Bn
    Z = (N @ Wq.T).view(T, H + 2 * Hkv, hd)
    ang = torch.zeros((T, hd // 2), dtype=torch.float64)
    for i in range(hd // 2):
        ang[:, i] = pos[0 if i < 16 else 1 if i < 40 else 2].double().cpu() * base ** (-i / (hd // 2))
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    a, b = Z[:, :H + Hkv, :64], Z[:, :H + Hkv, 64:]
    R = torch.cat([a * c - b * s, b * c + a * s], 2)
    Q, K, V = R[:, :H], R[:, H:].repeat_interleave(H // Hkv, 1), Z[:, H + Hkv:].repeat_interleave(H // Hkv, 1)
    st = torch.repeat_interleave(torch.tensor([0, 150, 151, 361]), torch.tensor([150, 1, 210, tail]))
    i, j = torch.arange(T)[:, None], torch.arange(T)[None, :]
    see = (j <= i) & (j >= st[:, None]) & ((i - j < W) | (j < st[:, None] + S))
    sc = torch.einsum("ihe,jhe->hij", Q, K) / math.sqrt(hd)
    P = torch.softmax(sc.masked_fill(~see, -math.inf), -1)
    O = torch.einsum("hij,jhe->ihe", P, V).reshape(T, H * hd)
    live = (torch.arange(T) < sum(lens)).double()[:, None]
    Y = X + (O * live) @ wo.double().cpu().T
    (Y * dy.double().cpu()).sum().backward()

    def rel(a, b):
        return float((a.double().cpu() - b).norm() / b.norm())

    assert rel(y, Y.detach()) < 2.0 ** -7
    assert rel(dx, X.grad) < 2.0 ** -6 and rel(dw, Wq.grad) < 2.0 ** -6
    assert rel(dg, Gn.grad) < 2.0 ** -6 and rel(db, Bn.grad) < 2.0 ** -6


class Pass:
    """A LayerNorm and a window attention, forward and backward, with tensors of their own."""

    def __init__(self, seed, lens, dt, H, Hkv, hd, W, S):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.T, self.lens, self.a = sum(lens), lens, (H, Hkv, hd, W, S)
        self.dt, self.out = dt, F32 if dt == F32 else BF16
        ty, to = (torch.float32, torch.float32) if dt == F32 else (torch.bfloat16, torch.bfloat16)
        r = lambda w, t: torch.randn((self.T, w), generator=g, device=DEV).to(t)
        self.q, self.k, self.v, self.do = r(H * hd, ty), r(Hkv * hd, ty), r(Hkv * hd, ty), r(H * hd, to)
        self.off = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)
        self.x, self.dy, self.gain = r(1000, to), r(1000, to), torch.randn(1000, generator=g, device=DEV)
        e = torch.empty_like
        self.outs = [e(self.do), torch.empty((H, self.T), device=DEV), e(self.do), e(self.k, dtype=to), e(self.v, dtype=to),
                     e(self.x), torch.empty(self.T, device=DEV), torch.empty(self.T, device=DEV), e(self.x),
                     torch.empty(1000, device=DEV), torch.empty(1000, device=DEV)]
        self.need = (lc.lc_window_attention_scratch_bytes(dt, self.T, H, Hkv, hd, W, S),
                     lc.lc_layernorm_scratch_bytes(self.T, 1000))

    def __call__(self, scratch, st=None):
        H, Hkv, hd, W, S = self.a
        o, lse, dq, dk, dv, y, mean, rstd, dx, dg, db = self.outs
        a, b, T, B = H * hd, Hkv * hd, self.T, len(self.lens)
        lc.lc_window_attention_forward(self.dt, self.out, T, B, self.off, H, Hkv, hd, W, S, self.q, a, self.k, b,
                                       self.v, b, o, a, lse, stream=st)
        lc.lc_layernorm_forward(T, 1000, self.x, self.gain, None, 1e-5, y, mean, rstd, self.out, F32, self.out, stream=st)
        lc.lc_window_attention_backward(self.dt, self.out, T, B, self.off, H, Hkv, hd, W, S, self.q, a, self.k, b,
                                        self.v, b, o, a, lse, self.do, a, dq, a, dk, b, dv, b, scratch, self.need[0],
                                        stream=st)
        lc.lc_layernorm_backward(T, 1000, self.dy, self.x, mean, rstd, self.gain, None, dx, dg, db, scratch,
                                 self.need[1], self.out, self.out, F32, F32, self.out, store_dg=1, stream=st)

    def scratch(self):
        return torch.full((max(self.need),), 0xFF, dtype=torch.uint8, device=DEV)

    def clear(self):
        for t in self.outs:
            t.fill_(7.0)
        torch.cuda.synchronize()

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.outs]


def passes():
    return [Pass(1, [700, 3, 900], BF16, 16, 4, 128, 100, 3), Pass(2, [40] * 70, F32, 4, 2, 64, 30, 2),
            Pass(3, [2000], lc.LC_FP16, 8, 8, 128, 300, 5)]


def test_calls_at_once_on_three_streams():
    banner("layer forms on three streams")
    ps, streams = passes(), [torch.cuda.Stream() for _ in range(3)]
    ws = [p.scratch() for p in ps]
    want = []
    for p, w in zip(ps, ws):
        p(w)
        want.append(p.results())
        p.clear()
    for _ in range(5):
        for p, w, s in zip(ps, ws, streams):
            p(w, s)
    for p, ref in zip(ps, want):
        assert all(torch.equal(a, b) for a, b in zip(p.results(), ref))


def test_captured_graphs_that_share_a_workspace():
    banner("layer forms, graphs that share a workspace")
    ps = passes()
    w = max((p.scratch() for p in ps), key=len)
    want, graphs, side = [], [], torch.cuda.Stream()
    for p in ps:
        p(w)
        want.append(p.results())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            p(w, side)
    for order in ((0, 1, 2), (2, 0, 1), (1, 1, 0, 2)):
        for p in ps:
            p.clear()
        w.fill_(0xFF)
        for i in order:  # (one after the other, on one stream)
            graphs[i].replay()
        for p, ref in zip(ps, want):
            assert all(torch.equal(a, b) for a, b in zip(p.results(), ref))
        ps[order[0]](w)  # eager work of the program's own between the replays


@pytest.mark.parametrize("dt", [BF16, F32])
def test_rows_past_32_bit_offsets(dt):
    """Tensors whose rows lie 2^24 values apart (the last ones past 2^31 values, 2^32 bytes) give the
    same bits as packed ones."""
    banner(f"layer forms, rows 2^24 values apart {dt}")
    p = Pass(5, [150, 60], dt, 4, 2, 64, 40, 3)
    H, Hkv, hd, W, S = p.a
    T, ld, d, w = p.T, 1 << 24, 1000, p.scratch()
    p(w)
    want = p.results()
    t = torch.float32 if dt == F32 else torch.bfloat16
    big = torch.empty((T, ld), dtype=t, device=DEV)
    assert big.numel() > 1 << 31
    cols = 0

    def wide(src=None, width=0):
        nonlocal cols
        v = big[:, cols:cols + (width or src.shape[1])]
        cols += (v.shape[1] + 63) // 64 * 64
        if src is not None:
            v.copy_(src)
        return v

    q, k, v, do, x, dy = (wide(s) for s in (p.q, p.k, p.v, p.do, p.x, p.dy))
    o, dq, dk, dv, y, dx = (wide(width=n) for n in (H * hd, H * hd, Hkv * hd, Hkv * hd, d, d))
    lse, mean, rstd, dg, db = (torch.empty_like(want[i]) for i in (1, 6, 7, 9, 10))
    lc.lc_window_attention_forward(dt, dt, T, 2, p.off, H, Hkv, hd, W, S, q, ld, k, ld, v, ld, o, ld, lse)
    lc.lc_window_attention_backward(dt, dt, T, 2, p.off, H, Hkv, hd, W, S, q, ld, k, ld, v, ld, o, ld, lse, do, ld,
                                    dq, ld, dk, ld, dv, ld, w, p.need[0])
    lc.lc_layernorm_forward(T, d, x, p.gain, None, 1e-5, y, mean, rstd, dt, F32, dt, ld_x=ld, ld_y=ld)
    lc.lc_layernorm_backward(T, d, dy, x, mean, rstd, p.gain, None, dx, dg, db, w, p.need[1], dt, dt, F32, F32, dt,
                             store_dg=1, ld_x=ld, ld_dy=ld, ld_dx=ld)
    torch.cuda.synchronize()
    for a, b in zip((o, lse, dq, dk, dv, y, mean, rstd, dx, dg, db), want):
        assert torch.equal(a, b)
    pos = torch.arange(2 * T, dtype=torch.int32, device=DEV)
    packed, apart = torch.empty_like(p.q), wide(width=H * hd)
    lc.lc_rope_axes_forward(T, H, hd, [20, 12], pos, T, p.q, H * hd, packed, H * hd, dt, dt)
    lc.lc_rope_axes_forward(T, H, hd, [20, 12], pos, T, q, ld, apart, ld, dt, dt)
    assert torch.equal(packed, apart)

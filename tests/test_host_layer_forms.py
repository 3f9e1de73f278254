"""Argument checking of LayerNorm, the rotary positions with several axes and the
sliding-window attention, without a GPU: every call breaks one documented rule and must return
its status from the host-side checks, before anything is enqueued (addresses are aligned fakes
that are never dereferenced; calls without rows return LC_OK). Host-only, like
test_host_ops.py."""
import pytest
import torch

from paper_2606_11169_amd import libchunk as lc

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: host-only checks")

A, B, C, D, E, F = ((i + 1) << 24 for i in range(6))
BF16, FP16, FP32 = lc.LC_BF16, lc.LC_FP16, lc.LC_FP32
BAD, UNSUP, WS, OK = lc.LC_ERR_INVALID_ARG, lc.LC_ERR_UNSUPPORTED, lc.LC_ERR_WORKSPACE, lc.LC_OK


def status_of(fn, **k):
    try:
        fn(**k)
    except lc.LibchunkError as e:
        assert str(e)
        return e.status
    return OK


LN_F = dict(T=16, d=100, x=A, g=B, b=C, eps=1e-5, y=D, mean=E, rstd=F, x_dtype=FP32, w_dtype=BF16, out_dtype=BF16)
LN_B = dict(T=16, d=100, dy=A, x=B, mean=C, rstd=D, g=E, dres=None, dx=F, dg_accum=A, db_accum=B, scratch=C,
            scratch_bytes=1 << 22, dy_dtype=FP32, x_dtype=FP32, w_dtype=BF16, dres_dtype=FP32, out_dtype=FP32)


@pytest.mark.parametrize("over,want", [
    (dict(T=-1), BAD), (dict(d=0), BAD), (dict(x=None), BAD), (dict(x=A + 4), BAD), (dict(g=None), BAD),
    (dict(b=C + 8), BAD), (dict(y=None), BAD), (dict(mean=None), BAD), (dict(rstd=F + 4), BAD),
    (dict(x_dtype=3), BAD), (dict(out_dtype=-1), BAD), (dict(ld_x=99), BAD), (dict(ld_y=-100), BAD),
    (dict(ld_x=1 << 61), BAD), (dict(d=1 << 31), UNSUP), (dict(T=1 << 31), UNSUP),
    (dict(T=0), OK), (dict(T=0, x=None, y=None, mean=None), OK)], ids=str)
def test_layernorm_forward(over, want):
    assert status_of(lc.lc_layernorm_forward, **{**LN_F, **over}) == want


@pytest.mark.parametrize("over,want", [
    (dict(dy=None), BAD), (dict(dx=None), BAD), (dict(dx=F + 2), BAD), (dict(dy_dtype=5), BAD),
    (dict(dres=A, dres_dtype=7), BAD), (dict(dres=A + 4), BAD), (dict(dx_copy=A + 8), BAD), (dict(dg_accum=A + 4), BAD),
    (dict(ld_dy=50), BAD), (dict(ld_dx=99), BAD), (dict(dres=A, ld_dres=10), BAD),
    (dict(scratch=None), WS), (dict(scratch_bytes=7), WS), (dict(dg_accum=None, scratch_bytes=7), WS),
    (dict(scratch=C + 4), WS), (dict(T=0), OK)], ids=str)
def test_layernorm_backward(over, want):
    assert status_of(lc.lc_layernorm_backward, **{**LN_B, **over}) == want


def test_layernorm_scratch():
    assert lc.lc_layernorm_scratch_bytes(0, 8) == 0 and lc.lc_layernorm_scratch_bytes(8, 0) == 0
    n = lc.lc_layernorm_scratch_bytes(4096, 4096)
    assert 0 < n <= 4096 * 4096 * 2  # far below the rows themselves
    need = lc.lc_layernorm_scratch_bytes(LN_B["T"], LN_B["d"])
    assert status_of(lc.lc_layernorm_backward, **{**LN_B, "scratch_bytes": need - 1}) == WS


ROPE = dict(T=10, n_heads=4, hd=128, sections=[16, 24, 24], pos=A, ld_pos=10, x=B, ld_x=512, y=C, ld_y=512,
            x_dtype=BF16, y_dtype=BF16)


@pytest.mark.parametrize("over,want", [
    (dict(T=-1), BAD), (dict(T=1 << 31), UNSUP), (dict(hd=127), UNSUP), (dict(hd=0), UNSUP), (dict(hd=258), UNSUP),
    (dict(n_heads=0), BAD), (dict(sections=[]), BAD), (dict(sections=[1] * 5), BAD), (dict(sections=[0, 0]), BAD),
    (dict(sections=[40, 25]), BAD), (dict(sections=[-1, 9]), BAD), (dict(freq=2), BAD), (dict(base=0.5), BAD),
    (dict(base=float("nan")), BAD), (dict(base=float("inf")), BAD), (dict(ld_pos=9), BAD), (dict(pos=None), BAD),
    (dict(pos=A + 2), BAD), (dict(x=None), BAD), (dict(y=C + 8), BAD), (dict(ld_x=511), BAD), (dict(ld_y=0), BAD),
    (dict(x_dtype=9), BAD), (dict(y_dtype=-1), BAD), (dict(ld_x=1 << 61), BAD), (dict(T=0, ld_pos=0, pos=None), OK)], ids=str)
def test_rope_axes(over, want):
    for fn in (lc.lc_rope_axes_forward, lc.lc_rope_axes_backward):
        assert status_of(fn, **{**ROPE, **over}) == want


@pytest.mark.parametrize("over,want", [(dict(cos=None), BAD), (dict(sin=C + 4), BAD), (dict(hd=130, sections=[66]), BAD),
                                       (dict(T=0, ld_pos=0), OK)], ids=str)
def test_rope_table(over, want):
    args = dict(T=10, hd=128, sections=[16, 24, 24], pos=A, ld_pos=10, cos=B, sin=C)
    assert status_of(lc.lc_rope_axes_table, **{**args, **over}) == want


WIN_F = dict(dtype=BF16, o_dtype=BF16, T=100, B=2, seq_offsets=A, H=4, Hkv=2, hd=128, window=32, n_sink=4, q=B,
             ld_q=1024, k=B + 1024, ld_k=1024, v=B + 1536, ld_v=1024, o=C, ld_o=512, lse=D)


@pytest.mark.parametrize("over,want", [
    (dict(T=-1), BAD), (dict(T=1 << 30), UNSUP), (dict(B=0), BAD), (dict(B=(1 << 20) + 1), UNSUP), (dict(H=0), BAD),
    (dict(Hkv=3), BAD), (dict(Hkv=-1), BAD), (dict(hd=96), UNSUP), (dict(hd=0), BAD), (dict(window=0), BAD),
    (dict(n_sink=-1), BAD), (dict(seq_offsets=None, B=3), BAD), (dict(seq_offsets=A + 2), BAD), (dict(dtype=4), BAD),
    (dict(o_dtype=FP16), UNSUP), (dict(dtype=FP16, o_dtype=FP16), UNSUP), (dict(dtype=FP32), UNSUP),
    (dict(dtype=FP32, o_dtype=FP32, hd=130), UNSUP), (dict(dtype=FP32, o_dtype=FP32, hd=33), UNSUP),
    (dict(ld_q=511), BAD), (dict(ld_q=1020), BAD), (dict(ld_k=128), BAD), (dict(ld_v=(1 << 30) + 8), BAD),
    (dict(ld_o=504), BAD), (dict(q=None), BAD), (dict(k=B + 2), BAD), (dict(o=None), BAD), (dict(lse=None), BAD),
    (dict(T=0), OK), (dict(T=0, q=None, seq_offsets=None), OK)], ids=str)
def test_window_attention_forward(over, want):
    assert status_of(lc.lc_window_attention_forward, **{**WIN_F, **over}) == want


@pytest.mark.parametrize("over,want", [
    (dict(dout=None), BAD), (dict(dq=None), BAD), (dict(dk=E + 8), BAD), (dict(dv=None), BAD), (dict(ld_dout=100), BAD),
    (dict(ld_dq=508), BAD), (dict(ld_dk=8), BAD), (dict(ld_dv=252), BAD), (dict(scratch=None), WS),
    (dict(scratch_bytes=16), WS), (dict(scratch=F + 4), WS), (dict(window=0), BAD), (dict(T=0), OK)], ids=str)
def test_window_attention_backward(over, want):
    args = dict(WIN_F, dout=D, ld_dout=512, dq=E, ld_dq=1024, dk=E + 1024, ld_dk=1024, dv=E + 1536, ld_dv=1024,
                scratch=F, scratch_bytes=1 << 23)
    assert status_of(lc.lc_window_attention_backward, **{**args, **over}) == want
    need = lc.lc_window_attention_scratch_bytes(BF16, 100, 4, 2, 128, 32, 4)
    assert status_of(lc.lc_window_attention_backward, **{**args, "scratch_bytes": need - 1}) == WS


@pytest.mark.parametrize("d,want", [((1 << 24) + 1, UNSUP), (1 << 30, UNSUP)])
def test_layernorm_long_rows(d, want):
    assert status_of(lc.lc_layernorm_forward, **{**LN_F, "d": d}) == want
    assert status_of(lc.lc_layernorm_backward, **{**LN_B, "d": d}) == want
    assert lc.lc_layernorm_scratch_bytes(16, d) == 0 < lc.lc_layernorm_scratch_bytes(16, 1 << 24)


def test_window_attention_of_too_many_workgroups():
    """2^29 rows of 2^18 heads: refused before a launch, and no workgroup count wraps."""
    T, H, hd, ld = 1 << 29, 1 << 18, 64, 1 << 24
    n = lc.lc_window_attention_scratch_bytes(BF16, T, H, H, hd, 100, 4)
    assert n >= T * H * 8
    rows = dict(dtype=BF16, o_dtype=BF16, T=T, B=1, seq_offsets=None, H=H, Hkv=H, hd=hd, window=100, n_sink=4, q=A,
                ld_q=ld, k=B, ld_k=ld, v=C, ld_v=ld, o=D, ld_o=ld, lse=E)
    assert status_of(lc.lc_window_attention_forward, **rows) == UNSUP
    assert status_of(lc.lc_window_attention_backward, **rows, dout=F, ld_dout=ld, dq=A, ld_dq=ld, dk=B, ld_dk=ld,
                     dv=C, ld_dv=ld, scratch=D, scratch_bytes=n) == UNSUP


def test_null_argument_structs():
    L = lc.lib()
    for name in ("lc_layernorm_forward", "lc_layernorm_backward", "lc_rope_axes_forward", "lc_rope_axes_backward",
                 "lc_rope_axes_table", "lc_window_attention_forward", "lc_window_attention_backward"):
        assert getattr(L, name)(None, None) == BAD and lc.lib().lc_last_error()

"""Argument checking of the 8-bit quantisation, the products of its operands and the router's
balance loss, without a GPU: every call breaks one documented rule and must return its status from
the host-side checks, before anything is enqueued (addresses are aligned fakes that are never
dereferenced; calls without rows return LC_OK)."""
import ctypes

import pytest
import torch

from paper_2606_11169_amd import libchunk as lc

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0,
                                reason="fake device addresses: host-only checks")

A, B, C, D, E, F, G, H = ((i + 1) << 24 for i in range(8))
BF16, FP16, FP32, E4, E5 = lc.LC_BF16, lc.LC_FP16, lc.LC_FP32, lc.LC_FP8_E4M3, lc.LC_FP8_E5M2
BAD, UNSUP, WS, OK = lc.LC_ERR_INVALID_ARG, lc.LC_ERR_UNSUPPORTED, lc.LC_ERR_WORKSPACE, lc.LC_OK


def status_of(fn, **k):
    try:
        fn(**k)
    except lc.LibchunkError as e:
        assert str(e)
        return e.status
    return OK


QUANT = dict(T=200, d=100, x=A, x_dtype=BF16, q_dtype=E4, q=B, ld_q=112, scale=C, ld_scale=200, qt=D,
             ld_qt=256, scale_t=E, ld_scale_t=100)
GROUPS = dict(group_offsets=F, n_groups=3, ld_qt=512)


@pytest.mark.parametrize("over,want", [
    (dict(T=-1), BAD), (dict(d=0), BAD), (dict(T=1 << 31), UNSUP), (dict(d=(1 << 24) + 1), UNSUP),
    (dict(x=None), BAD), (dict(x=A + 8), BAD), (dict(x_dtype=E4), BAD), (dict(x_dtype=-1), BAD),
    (dict(q_dtype=BF16), BAD), (dict(q_dtype=5), BAD), (dict(block_rows=2), BAD), (dict(block_rows=0), BAD),
    (dict(q=None), BAD), (dict(scale=None), BAD), (dict(qt=None), BAD), (dict(scale_t=None), BAD),
    (dict(q=None, scale=None, qt=None, scale_t=None), BAD), (dict(q=B + 8), BAD), (dict(scale_t=E + 4), BAD),
    (dict(ld_x=99), BAD), (dict(ld_x=-100), BAD), (dict(ld_q=96), BAD), (dict(ld_q=120), BAD),
    (dict(ld_scale=196), BAD), (dict(ld_scale=202), BAD), (dict(ld_qt=192), BAD), (dict(ld_qt=264), BAD),
    (dict(ld_scale_t=96), BAD), (dict(ld_scale_t=101), BAD), (dict(n_groups=-1), BAD),
    (dict(n_groups=65, group_offsets=F), BAD), (dict(n_groups=2), BAD), ({**GROUPS, "group_offsets": F + 2}, BAD),
    ({**GROUPS, "block_rows": 128}, UNSUP), ({**GROUPS, "ld_qt": 496}, BAD), (dict(row_index=F, x_rows=-1), BAD),
    (dict(row_index=F + 1, x_rows=4), BAD), (dict(row_weight=F + 2), BAD),
    (dict(T=0, x=None), OK), (dict(T=0, x=None, **GROUPS), OK)], ids=str)
def test_quantize(over, want):
    assert status_of(lc.lc_fp8_quantize, **{**QUANT, **over}) == want


def test_padded_rows():
    """The most columns that n groups of T rows in all can need."""
    for T in (0, 1, 127, 128, 129, 1000):
        assert lc.lc_fp8_padded_rows(T) == lc.lc_fp8_padded_rows(T, 1) == -(-T // 128) * 128
    for T, n in ((1, 3), (2, 3), (3, 3), (130, 2), (384, 3), (1000, 7), (5000, 64)):
        k = min(T, n)  # k groups of one row, the rest in the last of them: whole blocks there waste least
        most = max(128 * ((k - 1 - j) + -(-(T - (k - 1 - j)) // 128)) for j in range(k))
        assert most <= lc.lc_fp8_padded_rows(T, n) <= 128 * (T // 128 + n)
        assert lc.lc_fp8_padded_rows(T, n) % 128 == 0
    for T, n in ((-1, 1), (1 << 31, 1), (5, -1), (5, 65)):
        assert lc.lc_fp8_padded_rows(T, n) == 0


GEMM = dict(epilogue=lc.LC_EPI_STORE, M=100, N=200, K=256, A=A, lda=256, a_scale=B, ld_a_scale=100, B=C, ldb=256,
            b_scale=D, ld_b_scale=4, Cm=E, ldc=200)
ROWS = dict(group_mode=lc.LC_GROUP_ROWS, n_groups=3, group_offsets=F, group_stride_b=200 * 256,
            group_stride_b_scale=8)
KGRP = dict(group_mode=lc.LC_GROUP_K, n_groups=3, group_offsets=F, group_stride_c=100 * 200)


@pytest.mark.parametrize("over,want", [
    (dict(M=-1), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(K=250), BAD), (dict(M=1 << 30, ld_a_scale=1 << 30), UNSUP),
    (dict(N=1 << 30), UNSUP), (dict(K=1 << 30), UNSUP), (dict(A=None), BAD), (dict(B=C + 8), BAD),
    (dict(a_scale=None), BAD), (dict(b_scale=D + 4), BAD), (dict(Cm=None), BAD), (dict(Cm=E + 4), BAD),
    (dict(a_dtype=BF16), BAD), (dict(b_dtype=5), BAD), (dict(a_block_rows=64), BAD), (dict(b_block_rows=0), BAD),
    (dict(epilogue=-1), BAD), (dict(epilogue=7), BAD), (dict(epilogue=lc.LC_EPI_ROPE), UNSUP),
    (dict(epilogue=lc.LC_EPI_SWIGLU), UNSUP), (dict(epilogue=lc.LC_EPI_SWIGLU_BWD), UNSUP),
    (dict(c_dtype=E4), BAD), (dict(lda=264), BAD), (dict(ldb=240), BAD), (dict(ldb=1 << 23), UNSUP),
    (dict(ld_a_scale=96), BAD), (dict(ld_a_scale=102), BAD), (dict(ld_b_scale=0), BAD), (dict(ldc=199), BAD),
    (dict(b_block_rows=1), BAD), (dict(ldc=(1 << 30) + 4), UNSUP),
    (dict(ld_a_scale=1 << 30), UNSUP), (dict(K=512, lda=512, ldb=512, ld_b_scale=1 << 29), UNSUP),
    (dict(epilogue=lc.LC_EPI_RESIDUAL), BAD), (dict(epilogue=lc.LC_EPI_RESIDUAL, R=F, ldr=199), BAD),
    (dict(epilogue=lc.LC_EPI_RESIDUAL, R=F, ldr=200, r_dtype=9), BAD), (dict(group_mode=3), BAD),
    ({**ROWS, "n_groups": 0}, BAD), ({**ROWS, "n_groups": 65}, BAD), ({**ROWS, "group_offsets": None}, BAD),
    ({**ROWS, "group_offsets": F + 1}, BAD), ({**ROWS, "group_stride_b": 8}, BAD), ({**ROWS, "group_stride_b": -16}, BAD),
    ({**ROWS, "group_stride_b_scale": -4}, BAD), ({**ROWS, "a_block_rows": 128}, UNSUP),
    ({**ROWS, "epilogue": lc.LC_EPI_RESIDUAL, "R": G, "ldr": 200}, UNSUP), ({**KGRP, "group_stride_c": -1}, BAD),
    (dict(M=0, A=None, Cm=None), OK), ({**ROWS, "M": 0}, OK)], ids=str)
def test_gemm(over, want):
    assert status_of(lc.lc_gemm_fp8, **{**GEMM, **over}) == want


FWD = dict(T=10, d=64, E=8, n=A, wr=B, sel=C, probs=D, lse=E, counts=F, loss=G, scratch=H, scratch_bytes=1 << 20,
           n_dtype=BF16, w_dtype=FP32)
BWD = dict(T=10, d=64, E=8, n=A, wr=B, sel=C, probs=D, lse=E, counts=F, coef=0.1, z_coef=0.0, dn=G, dwr_accum=H,
           scratch=A, scratch_bytes=1 << 24, n_dtype=BF16, w_dtype=FP32, dn_dtype=FP32)


@pytest.mark.parametrize("over,want", [
    (dict(T=-1), BAD), (dict(T=1 << 30), UNSUP), (dict(d=0), BAD), (dict(d=60), UNSUP),
    (dict(d=(1 << 20) + 8, scratch_bytes=1 << 40), UNSUP), (dict(E=1), BAD),
    (dict(E=65), BAD), (dict(n=None), BAD), (dict(wr=B + 4), BAD), (dict(sel=None), BAD), (dict(probs=None), BAD),
    (dict(lse=E + 8), BAD), (dict(counts=None), BAD), (dict(loss=None), BAD), (dict(n_dtype=E4), BAD),
    (dict(w_dtype=7), BAD), (dict(scratch=None), BAD), (dict(scratch=H + 4), BAD), (dict(scratch_bytes=100), WS)],
    ids=str)
def test_balance_forward(over, want):
    assert status_of(lc.lc_moe_balance_forward, **{**FWD, **over}) == want


@pytest.mark.parametrize("over,want", [
    (dict(T=-1), BAD), (dict(d=60), UNSUP), (dict(d=(1 << 20) + 8, scratch_bytes=1 << 40), UNSUP), (dict(E=65), BAD),
    (dict(n=None), BAD), (dict(counts=None), BAD),
    (dict(w=A), BAD), (dict(dw=A), BAD), (dict(w=A + 4, dw=B), BAD), (dict(dn=G + 2), BAD), (dict(dn_dtype=E5), BAD),
    (dict(dres=A, dres_dtype=8), BAD), (dict(dres=A + 8), BAD), (dict(dwr_accum=H + 4), BAD),
    (dict(coef=float("nan")), BAD), (dict(z_coef=float("nan")), BAD),
    (dict(T=1000, scratch=None), BAD), (dict(T=1000, scratch_bytes=64), WS),
    (dict(dn=None, dwr_accum=None), OK), (dict(T=0, n=None, sel=None, probs=None, dwr_accum=None), OK)], ids=str)
def test_balance_backward(over, want):
    assert status_of(lc.lc_moe_balance_backward, **{**BWD, **over}) == want


def test_balance_scratch_bytes():
    assert all(lc.lc_moe_balance_scratch_bytes(*a) == 0 for a in ((-1, 8, 8), (1 << 30, 8, 8), (5, 0, 8), (5, 8, 1), (5, 8, 65)))
    assert lc.lc_moe_balance_scratch_bytes(0, 8, 2) > 0
    # the backward's partial sums stay a small part of what it reads
    assert lc.lc_moe_balance_scratch_bytes(1 << 20, 4096, 64) <= 64 << 20


def test_packed_arguments_have_the_structs_layout():
    """The calls pack their arguments as bytes: sizes, and the place of every field, as in the structs."""
    for packed, cls in ((lc._FP8_QUANTIZE, lc.lc_fp8_quantize_args), (lc._GEMM_FP8, lc.lc_gemm_fp8_args),
                        (lc._MOE_BALANCE, lc.lc_moe_balance_args)):
        assert packed.size == ctypes.sizeof(cls)
        values = [i + 1 for i in range(len(cls._fields_))]
        got = cls.from_buffer_copy(packed.pack(*values))
        assert [getattr(got, f[0]) for f in cls._fields_] == values


@pytest.mark.parametrize("over,want", [
    (dict(group_stride_c=0), BAD), (dict(group_stride_c=199), BAD), (dict(group_stride_c=200), BAD),
    (dict(group_stride_c=99 * 200 + 199), BAD), (dict(group_stride_c=99 * 200 + 200, M=0), OK),
    (dict(group_stride_c=0, n_groups=1, M=0), OK),
    # side by side in wider rows: three groups of 200 columns in rows of 600, not of 599; by whole rows
    (dict(group_stride_c=200, ldc=600, M=0), OK), (dict(group_stride_c=200, ldc=599), BAD),
    (dict(group_stride_c=600, ldc=200), BAD), (dict(group_stride_c=700, ldc=400), BAD)], ids=str)
def test_groups_of_k_do_not_overlap(over, want):
    """Results of two groups in one place would be written in any order."""
    assert status_of(lc.lc_gemm_fp8, **{**GEMM, **KGRP, **over}) == want


def test_groups_of_k_overlap_as_counted():
    """The refusal against every element's place, for small sizes (what
    is not refused goes on to the launch, which fails without a GPU)."""
    for M, N, ldc, G in ((3, 16, 16, 3), (3, 16, 40, 2), (4, 20, 50, 3), (1, 16, 16, 2), (5, 16, 35, 2)):
        for stride in range(0, (M + 1) * ldc, 3):
            places = [g * stride + m * ldc + n for g in range(G) for m in range(M) for n in range(N)]
            got = status_of(lc.lc_gemm_fp8, **{**GEMM, **KGRP, "M": M, "N": N, "ldc": ldc, "n_groups": G, "ld_a_scale": 8,
                                               "ld_b_scale": 4, "b_block_rows": 128, "group_stride_c": stride})
            assert (got == BAD) == (len(set(places)) < len(places)), (M, N, ldc, G, stride)

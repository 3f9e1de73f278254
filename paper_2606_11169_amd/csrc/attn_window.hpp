// What the sliding-window attention kernels share: the call's checked parameters and the
// search for the sequence that holds a row.
#pragma once

#include "common.hpp"

namespace lc {

// Where the backward's scratch holds what (bytes from its start; -1: not needed), and the
// split of its work that this follows from (k_attn_window.hip)
struct WindowPlan {
  int64_t D, nl2;          // fp32 [H, T] each
  int64_t kb, vb, qb;      // fp16 inputs: bf16 rows of k, v [T, Hkv hd] and q [T, H hd]
  int64_t share;           // fp32 dk, then dv [parts, T, Hkv hd]
  int64_t slots;           // fp32 sums of sinks: [2, chunks, Hkv, parts, n_sink, 2, hd]
  int64_t total;
  int parts;               // workgroups that share a key block's query heads
  int chunk, chunks;       // query rows of a chunk; chunks of T (1: sinks are not split)
};
WindowPlan window_plan(int dtype, int64_t T, int H, int Hkv, int hd, int window, int n_sink);

// fp32 path (arguments already checked)
lc_status window_f32_fwd_launch(const lc_window_attn_args &a, hipStream_t s);
lc_status window_f32_bwd_launch(const lc_window_attn_args &a, hipStream_t s);

namespace {

// Offset b of the sequences' rows (S: rows of each without an offset array)
__device__ __forceinline__ int offset_of(const int32_t *off, int S, int T, int b) {
  return off ? min(max(off[b], 0), T) : b * S;
}

// The sequence that holds `row` (one row per wave, the same in every lane): its rows
// [start, end) and number; false if none does. 64 offsets per step, one load per lane.
// (Offsets that decrease against the documentation give some sequence inside [0, T).)
__device__ __forceinline__ bool wave_sequence(const int32_t *off, int S, int T, int B, int row, int lane, int &b,
                                              int &start, int &end) {
  if (!off) {
    b = row / S;
    start = b * S;
    end = start + S;
    return b < B;
  }
  const int first = offset_of(off, S, T, 0), last = offset_of(off, S, T, B);
  int lo = 0, hi = B;  // offset(lo) <= row < offset(hi)
  b = start = end = 0;
  if (row < first || row >= last) return false;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64;
    const int at = min(lo + (lane + 1) * step, hi);
    const uint64_t le = __ballot(at < hi && offset_of(off, S, T, at) <= row);
    lo = min(lo + (int)__popcll(le) * step, hi - 1);
    hi = min(hi, lo + step);
  }
  b = __builtin_amdgcn_readfirstlane(lo);
  start = __builtin_amdgcn_readfirstlane(offset_of(off, S, T, b));
  end = __builtin_amdgcn_readfirstlane(offset_of(off, S, T, b + 1));
  return true;
}

// The same for a row of each lane, none before sequence b0's first row
__device__ __forceinline__ bool lane_sequence(const int32_t *off, int S, int T, int B, int row, int b0, int &start,
                                              int &end) {
  if (!off) {
    start = row / S * S;
    end = start + S;
    return row < B * S;
  }
  int lo = b0, hi = B;
  start = end = 0;
  if (row < offset_of(off, S, T, b0) || row >= offset_of(off, S, T, B)) return false;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offset_of(off, S, T, mid) <= row) lo = mid;
    else hi = mid;
  }
  start = offset_of(off, S, T, lo);
  end = offset_of(off, S, T, hi);
  return true;
}

}  // namespace
}  // namespace lc

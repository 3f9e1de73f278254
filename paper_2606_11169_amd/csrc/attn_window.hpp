// What the sliding-window attention kernels share: the scratch's layout and the search for
// the sequence that holds a row.
#pragma once

#include "common.hpp"

namespace lc {

// Where the backward's scratch holds what (bytes from its start), and the split of its work
// that this follows from (k_attn_window.hip)
struct WindowPlan {
  int64_t D, nl2;          // fp32 [H, T] each
  int64_t inv;             // fp16 inputs: fp32 [H, T]
  int64_t share;           // fp32 dk, then dv [parts, T, Hkv hd]
  int64_t slots;           // fp32 sums of sinks: [2, chunks, Hkv, parts, n_sink, 2, hd]
  int64_t total;
  int krows, parts;        // keys per dK/dV workgroup; workgroups that share their query heads
  int chunk, chunks;       // query rows of a chunk; chunks of T (1: sinks are not split)
};
WindowPlan window_plan(int dtype, int64_t T, int H, int Hkv, int hd, int window, int n_sink);

// fp32 path (arguments already checked)
lc_status window_f32_fwd_launch(const lc_window_attn_args &a, hipStream_t s);
lc_status window_f32_bwd_launch(const lc_window_attn_args &a, hipStream_t s);

namespace {

// The packed sequences as a wave sees them. Up to 63 sequences' offsets are held one per
// lane, so that finding a row's sequence costs one load's latency in all; more are searched for
// in memory. (Offsets that decrease against the documentation give some sequence inside
// [0, T).)
struct Sequences {
  const int32_t *off;
  int S, T, B;       // S: rows of each without an offset array
  int first, last;   // rows [first, last) belong to sequences
  int mine;          // offset `lane`, for up to 63 sequences
  __device__ __forceinline__ bool held() const { return B < 64; }
  __device__ __forceinline__ int at(int b) const { return off ? min(max(off[b], 0), T) : b * S; }

  __device__ __forceinline__ Sequences(const int32_t *off_, int S_, int T_, int B_, int lane)
      : off(off_), S(S_), T(T_), B(B_), mine(0) {
    if (!off) {
      first = 0;
      last = B * S;
    } else if (held()) {
      mine = at(min(lane, B));
      first = __builtin_amdgcn_readlane(mine, 0);
      last = __builtin_amdgcn_readlane(mine, B);
    } else {
      first = at(0);
      last = at(B);
    }
  }

  // The sequence that holds `row` (one row per wave): number b, rows [start, end); false if none does
  __device__ __forceinline__ bool of_wave(int row, int lane, int &b, int &start, int &end) const {
    b = start = end = 0;
    if (row < first || row >= last) return false;
    if (!off) {
      b = row / S;
      start = b * S;
      end = start + S;
    } else if (held()) {
      b = min((int)__popcll(__ballot(lane < B && mine <= row)), B) - 1;
      b = max(b, 0);
      start = __builtin_amdgcn_readlane(mine, b);
      end = __builtin_amdgcn_readlane(mine, b + 1);
    } else {
      int lo = 0, hi = B;  // at(lo) <= row < at(hi); 64 offsets per step
      while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64;
        const int x = min(lo + (lane + 1) * step, hi);
        const uint64_t le = __ballot(x < hi && at(x) <= row);
        lo = min(lo + (int)__popcll(le) * step, hi - 1);
        hi = min(hi, lo + step);
      }
      b = __builtin_amdgcn_readfirstlane(lo);
      start = __builtin_amdgcn_readfirstlane(at(b));
      end = __builtin_amdgcn_readfirstlane(at(b + 1));
    }
    return true;
  }

  // The same for a row of each lane (every lane of the wave calls it; rows before sequence b0 are of
  // no interest)
  __device__ __forceinline__ bool of_lane(int row, int b0, int &start, int &end) const {
    start = end = 0;
    const bool in = row >= first && row < last;
    if (!off) {
      start = row / S * S;
      end = start + S;
    } else if (held()) {
      for (int b = b0; b < B; ++b) {
        const int s = __builtin_amdgcn_readlane(mine, b), e = __builtin_amdgcn_readlane(mine, b + 1);
        if (row >= s) {
          start = s;
          end = e;
        }
        if (!__any(in && row >= e)) break;
      }
    } else if (in) {
      int lo = b0, hi = B;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at(mid) <= row) lo = mid;
        else hi = mid;
      }
      start = at(lo);
      end = at(hi);
    }
    return in && row >= start && row < end;
  }
};

}  // namespace
}  // namespace lc

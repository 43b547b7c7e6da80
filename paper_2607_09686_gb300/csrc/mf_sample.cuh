// Which entries of a row of logits are kept, as sampling finds them and verification uses them (not part of the C ABI).
#pragma once

#include "mf_attn.cuh"

namespace mf {

constexpr int kMaxVocab = 1 << 20;

// The temperature and its inverse are kept where 0 and -inf times the inverse (also in units of log2 e and of bins) are 0 and
// -inf: T from 2^-120 up (below it what differs from M weighs nothing, unless by less than 2^-113), the inverse above 0 for
// T = inf (times the largest number it is below 1e-6).
__device__ __forceinline__ float bounded(float t) { return fmaxf(t, 0x1p-120f); }
__device__ __forceinline__ float inverse(float unit, float t) { return fmaxf(unit / t, 1e-45f); }
// (what is no number, -inf / inf, is -inf)
__device__ __forceinline__ float z_of(float x, float m, float t) { return x == m ? 0.f : fmaxf(__fdiv_rn(x - m, t), -INFINITY); }

// A row's kept entries: those above xc and, where equal to it, up to index ic, with w = exp(z) >= min_p, z = z_of(x, m, t).
struct Kept {
  float m, t, xc, min_p;
  int ic;
  float log_sum;  // of w over them
  int any;        // 0: none
  int unused;
};

// Rows of several sequences: the target's (where `target` is set) and, where draft is given, the drafter's (not the last of a sequence),
// with settings by sequence.  The n_rows target rows' sets are left in kept, the drafter's behind their place.
struct KeptRows {
  const void *logits, *draft;
  int64_t logits_stride, draft_stride;
  const int32_t* row_start;
  mf_cuts_t cuts, draft_cuts;
  Kept* kept;
  int* fall;  // is set to whether a start lies below the one before it
  int n_seqs, n_rows, vocab, dtype, target;
};
cudaError_t launch_kept(const KeptRows& rows, cudaStream_t s);
int sample_hold();  // mf_sample_test_hold

// The rows of a sequence, inside [0, n_rows], where the starts rise.
struct RowSpan {
  int b, e;
};
__device__ __forceinline__ int row_at(const int32_t* row_start, int n_rows, int i) { return min(max(__ldg(row_start + i), 0), n_rows); }
__device__ __forceinline__ RowSpan row_span(const int32_t* row_start, int n_rows, int s) {
  const int b = row_at(row_start, n_rows, s);
  return {b, max(row_at(row_start, n_rows, s + 1), b)};
}
// Where they do not, a start is the largest so far, and rows still have one sequence at most.  Whether one of starts 1 .. n lies below
// the one before it, as far as this thread of the block looks.
__device__ __forceinline__ bool starts_fall(const int32_t* row_start, int n) {
  bool fall = false;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += blockDim.x) fall |= __ldg(row_start + i) > __ldg(row_start + i + 1);
  return fall;
}
// Then the rows of a sequence (every lane of the warp).
static __device__ __noinline__ RowSpan row_span_fallen(const int32_t* row_start, int n_rows, int s) {
  int b = 0;
  for (int i = threadIdx.x & 31; i <= s; i += 32) b = max(b, row_at(row_start, n_rows, i));
  b = __reduce_max_sync(0xffffffffu, b);
  return {b, max(b, row_at(row_start, n_rows, s + 1))};
}
// A row's sequence (-1: none), which is the last that begins at or before it, the one before the first that begins behind it where starts
// fall, and where that ends (every lane of the warp).
static __device__ __noinline__ int2 row_owner(const int32_t* row_start, int n_rows, int n_seqs, int row, bool fall) {
  if (!fall) {
    int lo = 0, hi = n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (__ldg(row_start + mid) <= row) lo = mid;
      else hi = mid - 1;
    }
    const RowSpan sp = row_span(row_start, n_rows, lo);
    return make_int2(row >= sp.b && row < sp.e ? lo : -1, sp.e);
  }
  for (int base = 0; base <= n_seqs; base += 32) {
    const int i = base + (int)(threadIdx.x & 31), at = i <= n_seqs ? row_at(row_start, n_rows, i) : 0;
    const unsigned behind = __ballot_sync(0xffffffffu, at > row);
    if (behind) return make_int2(base + __ffs(behind) - 2, __shfl_sync(0xffffffffu, at, __ffs(behind) - 1));
  }
  return make_int2(-1, 0);
}
// The same in either case, by every thread of the block: of few sequences all starts are read at once.
constexpr int kFewStarts = 4 * 32;
__device__ __forceinline__ int2 row_owner_any(const int32_t* row_start, int n_rows, int n_seqs, int row) {
  if (n_seqs >= kFewStarts) return row_owner(row_start, n_rows, n_seqs, row, __syncthreads_or(starts_fall(row_start, n_seqs)));
  const int lane = threadIdx.x & 31;
  int at[kFewStarts / 32];
#pragma unroll
  for (int k = 0; k < kFewStarts / 32; ++k) at[k] = 32 * k + lane <= n_seqs ? row_at(row_start, n_rows, 32 * k + lane) : 0;
  int2 own = make_int2(-1, 0);
#pragma unroll
  for (int k = kFewStarts / 32 - 1; k >= 0; --k) {
    const unsigned behind = __ballot_sync(0xffffffffu, at[k] > row);
    if (behind) own = make_int2(32 * k + __ffs(behind) - 2, __shfl_sync(0xffffffffu, at[k], __ffs(behind) - 1));
  }
  return own;
}

}  // namespace mf

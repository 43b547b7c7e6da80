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
  int n_seqs, n_rows, vocab, dtype, target;
};
cudaError_t launch_kept(const KeptRows& rows, cudaStream_t s);
int sample_hold();  // mf_sample_test_hold

// The rows of a sequence, inside [0, n_rows].
struct RowSpan {
  int b, e;
};
__device__ __forceinline__ RowSpan row_span(const int32_t* row_start, int n_rows, int s) {
  const int b = min(max(__ldg(row_start + s), 0), n_rows);
  return {b, min(max(__ldg(row_start + s + 1), b), n_rows)};
}

}  // namespace mf

// Verification of drafted tokens: the drafts that the target takes, and the token that ends each sequence.  Contract: mawforge.h.
//
// Two launches.  The first finds what each row of the target's logits keeps and the sum of its weights (k_sample's steps, without the
// draw), and the same of the drafter's rows, so that p and q of any entry are a few operations on its logit.  In the second
// a cluster of 1 to 8 blocks has a sequence: the drafts' p and q, one row a thread, the first row whose draft is not taken; then one
// pass over that row for the largest log(p - q) + noise.
#include <cooperative_groups.h>

#include <cmath>

#include "mf_sample.cuh"

namespace cg = cooperative_groups;

namespace mf {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;

struct VerifyCall {
  const void *logits, *draft;
  int64_t logits_stride, draft_stride, noise_stride;
  const int32_t *row_start, *tokens;
  const float *u, *noise;
  int32_t *token, *accepted;
  float* logprob;
  const Kept* kept;
  int n_rows, vocab, slice;
};

// log p of the entry of index i, -inf where it is not kept
__device__ __forceinline__ float log_p(const Kept& k, float x, int i) {
  x = fmaxf(x, -INFINITY);  // NaN as -inf
  if (!k.any || x == -INFINITY || !(x > k.xc || (x == k.xc && i <= k.ic))) return -INFINITY;
  const float z = z_of(x, k.m, k.t);
  return k.min_p > 0.f && expf(z) < k.min_p ? -INFINITY : z - k.log_sum;
}

struct Best {  // the largest key so far, the lowest index where equal
  float v, lp;
  int i;
  __device__ __forceinline__ void take(float ov, float olp, int oi) {
    if (ov > v || (ov == v && oi < i)) v = ov, lp = olp, i = oi;
  }
};

template <class T>
__global__ void __launch_bounds__(kThreads) k_verify(const __grid_constant__ VerifyCall c) {
  __shared__ Best s_best[kWarps + 1];
  __shared__ int s_stop;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), s = blockIdx.x / C;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  const RowSpan sp = row_span(c.row_start, c.n_rows, s);
  if (sp.b == sp.e) {
    if (rank == 0 && tid == 0) c.accepted[s] = 0;
    return;
  }
  const int drafts = sp.e - sp.b - 1;
  const T* logits = static_cast<const T*>(c.logits);
  const T* draft = static_cast<const T*>(c.draft);
  auto draft_log_p = [&](int row) -> float {
    const int x = __ldg(c.tokens + row + 1);
    if (x < 0 || x >= c.vocab) return -INFINITY;
    return log_p(c.kept[row], (float)logits[(int64_t)row * c.logits_stride + x], x);
  };
  // ---- the drafts that are taken
  if (tid == 0) s_stop = drafts;
  __syncthreads();
  for (int j = tid; j < drafts; j += kThreads) {
    const int row = sp.b + j, x = __ldg(c.tokens + row + 1);
    const float p = expf(draft_log_p(row));
    float q = 1.f;
    if (draft && x >= 0 && x < c.vocab) q = expf(log_p(c.kept[c.n_rows + row], (float)draft[(int64_t)row * c.draft_stride + x], x));
    if (!(__ldg(c.u + row) * q < p)) atomicMin(&s_stop, j);
  }
  __syncthreads();
  const int stop = s_stop, row = sp.b + stop, one = stop < drafts && !draft ? __ldg(c.tokens + row + 1) : -1;
  const Kept kp = c.kept[row];
  const bool less = stop < drafts && draft;
  Kept kq = {};
  if (less) kq = c.kept[c.n_rows + row];

  // ---- the token after them
  const int i0 = rank * c.slice, i1 = min(c.vocab, i0 + c.slice);
  const T* x = logits + (int64_t)row * c.logits_stride;
  const T* y = less ? draft + (int64_t)row * c.draft_stride : nullptr;
  const float* noise = c.noise + (int64_t)s * c.noise_stride;
  const Best none = {-INFINITY, -INFINITY, 0x7FFFFFFF};
  auto warp_best = [&](Best b) -> Best {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      b.take(__shfl_xor_sync(0xffffffffu, b.v, d), __shfl_xor_sync(0xffffffffu, b.lp, d), __shfl_xor_sync(0xffffffffu, b.i, d));
    return b;
  };
  Best b;
  for (int turn = 0; turn < 2; ++turn) {  // (the second where no entry has p > q: with p alone)
    b = none;
    for (int i = i0 + tid; i < i1; i += kThreads) {
      const float lp = log_p(kp, (float)x[i], i);
      if (lp == -INFINITY) continue;
      float key = lp;
      if (turn == 0) {
        if (i == one) continue;
        if (less) {
          const float lq = log_p(kq, (float)y[i], i);
          if (lq > -INFINITY) {
            const float d = expf(lp) - expf(lq);
            if (!(d > 0.f)) continue;
            key = logf(d);
          }
        }
      }
      b.take(fmaxf(key + noise[i], -INFINITY), lp, i);
    }
    b = warp_best(b);
    __syncthreads();
    if (lane == 0) s_best[warp] = b;
    __syncthreads();
    if (warp == 0) {
      b = warp_best(lane < kWarps ? s_best[lane] : none);
      if (lane == 0) s_best[kWarps] = b;
    }
    cl.sync();
    b = warp_best(lane < C ? cl.map_shared_rank(s_best, lane)[kWarps] : none);
    cl.sync();  // no block writes its best again, or leaves, while another reads it
    if (b.i != none.i) break;
  }

  if (rank != 0) return;
  for (int j = tid; j <= drafts; j += kThreads) {
    const int at = sp.b + j;
    const bool empty = b.i == none.i;
    c.token[at] = j < stop ? __ldg(c.tokens + at + 1) : j > stop || empty ? -1 : b.i;
    if (c.logprob) c.logprob[at] = j < stop ? draft_log_p(at) : j > stop || empty ? -INFINITY : b.lp;
  }
  if (tid == 0) c.accepted[s] = stop;
}

template <class T>
cudaError_t run(VerifyCall c, int n_seqs, cudaStream_t s) {
  int C = 1;
  while (C < 8 && (int64_t)n_seqs * C < 304 && c.vocab / C > 8192) C *= 2;
  c.slice = (c.vocab + C - 1) / C;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_seqs * (unsigned)C);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)C, 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_verify<T>, c);
}

bool bad_word(const void* p) { return ((uintptr_t)p & 3) != 0; }
bool bad_cuts(const mf_cuts_t& c) { return bad_word(c.temperature) || bad_word(c.top_p) || bad_word(c.min_p) || bad_word(c.top_k); }

}  // namespace
}  // namespace mf

using namespace mf;

extern "C" int mf_verify_bytes(int n_seqs, int n_rows, int vocab, uint64_t* out) {
  if (!out || n_seqs < 0 || n_rows < 0 || n_seqs > (1 << 26) || n_rows > (1 << 26) || vocab < 1 || vocab > kMaxVocab) return MF_E_INVAL;
  *out = (uint64_t)(n_rows > 0 ? n_rows : 1) * 2 * sizeof(Kept);
  return MF_OK;
}

extern "C" int mf_verify(const mf_verify_args_t* a, void* stream) {
  uint64_t bytes;
  if (!a || mf_verify_bytes(a->n_seqs, a->n_rows, a->vocab, &bytes) != MF_OK) return MF_E_INVAL;
  if (a->dtype != MF_F32 && a->dtype != MF_F16 && a->dtype != MF_BF16) return MF_E_INVAL;
  if (a->n_seqs == 0) return a->n_rows == 0 ? MF_OK : MF_E_INVAL;
  if (!a->row_start || !a->accepted || bad_word(a->row_start) || bad_word(a->accepted)) return MF_E_INVAL;
  if (a->n_rows > 0) {
    if (!a->logits || !a->tokens || !a->u || !a->noise || !a->token || !a->work) return MF_E_INVAL;
    if (bad_word(a->tokens) || bad_word(a->u) || bad_word(a->noise) || bad_word(a->token) || bad_word(a->logprob) ||
        bad_cuts(a->cuts) || bad_cuts(a->draft_cuts) || ((uintptr_t)a->work & 15))
      return MF_E_INVAL;
    const uintptr_t odd = a->dtype == MF_F32 ? 3 : 1;
    if (((uintptr_t)a->logits | (uintptr_t)a->draft_logits) & odd) return MF_E_INVAL;
    if (a->n_rows > 1 && (a->logits_stride < a->vocab || (a->draft_logits && a->draft_stride < a->vocab))) return MF_E_INVAL;
    if (a->n_seqs > 1 && a->noise_stride < a->vocab) return MF_E_INVAL;
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  Kept* kept = static_cast<Kept*>(a->work);
  const KeptRows rows = {a->logits, a->draft_logits, a->logits_stride, a->draft_stride, a->row_start, a->cuts, a->draft_cuts,
                         kept,      a->n_seqs,       a->n_rows,        a->vocab,        a->dtype};
  const VerifyCall c = {a->logits, a->draft_logits, a->logits_stride, a->draft_stride, a->noise_stride, a->row_start, a->tokens, a->u,
                        a->noise,  a->token,        a->accepted,      a->logprob,      kept,            a->n_rows,    a->vocab,  0};
  cudaError_t e = a->n_rows > 0 ? launch_kept(rows, s) : cudaSuccess;
  if (e == cudaSuccess)
    e = a->dtype == MF_F32   ? run<float>(c, a->n_seqs, s)
        : a->dtype == MF_F16 ? run<__half>(c, a->n_seqs, s)
                             : run<__nv_bfloat16>(c, a->n_seqs, s);
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_verify");
}

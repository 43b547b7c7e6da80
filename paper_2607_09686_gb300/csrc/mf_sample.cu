// One token from each row of logits: temperature, top-k, top-p, min-p, and an argmax with the caller's Gumbel
// noise.  Contract: mawforge.h.
//
// The kept entries are a prefix of the row in the order (x falling, index rising), so they are described by a
// value and an index: all entries with a larger x, and those equal to it up to that index.  One block per row finds
// both by bisection over the 32 bits of the value's ordered key (counts for top-k, sums of w for top-p), then over the
// index, and takes the argmax in a last pass.
#include <cmath>

#include "mf_attn.cuh"

namespace mf {
namespace {

constexpr int kThreads = 1024;
constexpr int kMaxVocab = 1 << 20;

struct SampleCall {
  const void* logits;
  const float *noise, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* token;
  float* logprob;
  int64_t logits_stride, noise_stride;
  int vocab;
};

// x in fp32 with NaN as -inf
template <class T>
__device__ __forceinline__ float logit(const void* row, int i) {
  float x;
  if constexpr (sizeof(T) == 4) x = static_cast<const float*>(row)[i];
  else if constexpr (sizeof(T) == 2) x = (float)static_cast<const T*>(row)[i];
  return x == x ? x : -INFINITY;
}
// larger floats have larger keys (-0 and +0 compare equal as floats: one key)
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float z_of(float x, float m, float t) { return x == m ? 0.f : __fdiv_rn(x - m, t); }

// (sum, count) over the block, the same in every thread; partial sums in a fixed order
__device__ __forceinline__ void block_sum(double& s, int& n, double* buf, int* nbuf) {
  for (int d = 16; d; d >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, d);
    n += __shfl_xor_sync(0xffffffffu, n, d);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = s, nbuf[threadIdx.x >> 5] = n;
  __syncthreads();
  s = 0, n = 0;
  for (int i = 0; i < kThreads / 32; ++i) s += buf[i], n += nbuf[i];
}

template <class T>
__global__ void __launch_bounds__(kThreads) k_sample_simple(SampleCall c) {
  __shared__ double buf[32];
  __shared__ int nbuf[32];
  __shared__ float fbuf[32];
  const int r = blockIdx.x, tid = threadIdx.x, V = c.vocab;
  const void* row = static_cast<const T*>(c.logits) + (int64_t)r * c.logits_stride;
  const float* g = c.noise + (int64_t)r * c.noise_stride;
  const float t = c.temperature ? c.temperature[r] : 1.f;
  const bool greedy = !(t > 0.f);
  float m = -INFINITY;
  for (int i = tid; i < V; i += kThreads) m = fmaxf(m, logit<T>(row, i));
  for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  if ((tid & 31) == 0) fbuf[tid >> 5] = m;
  __syncthreads();
  for (int i = 0; i < kThreads / 32; ++i) m = fmaxf(m, fbuf[i]);
  if (m == -INFINITY) {
    if (tid == 0) {
      c.token[r] = -1;
      if (c.logprob) c.logprob[r] = -INFINITY;
    }
    return;
  }
  const float top_p = c.top_p ? c.top_p[r] : 1.f, min_p = c.min_p ? fminf(fmaxf(c.min_p[r], 0.f), 1.f) : 0.f;
  const int top_k = greedy ? 1 : c.top_k ? c.top_k[r] : 0;
  const float td = greedy ? 1.f : t;

  // entries with a key above `key`, and the first `ties` of those at it, are kept
  uint32_t key = order_key(-INFINITY) + 1;  // all but -inf
  int64_t ties = V;
  auto scan = [&](uint32_t from, double& s, int& n) {  // keys >= from
    s = 0, n = 0;
    float part = 0.f;
    for (int i = tid; i < V; i += kThreads) {
      const float x = logit<T>(row, i);
      if (order_key(x) >= from) part += expf(z_of(x, m, td)), ++n;
    }
    s = part;
    block_sum(s, n, buf, nbuf);
  };
  double s;
  int n;
  scan(key, s, n);
  if (top_k > 0 && top_k < n) {
    uint32_t lo = key, hi = order_key(m);  // largest key with at least top_k entries at or above
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo + 1) / 2;
      scan(mid, s, n);
      if (n >= top_k) lo = mid;
      else hi = mid - 1;
    }
    key = lo;
    double s1;
    int n1;
    scan(key, s, n);
    scan(key + 1, s1, n1);
    ties = top_k - n1;
    s = s1 + (s - s1) / (n - n1) * (double)ties;
  }
  if (top_p < 1.f) {
    const double want = (double)top_p * s;
    uint32_t lo = key, hi = order_key(m);  // largest key whose mass above it is below want ... and the first tie past it
    while (lo < hi) {  // smallest key such that the mass above it is < want
      const uint32_t mid = lo + (hi - lo) / 2;
      double sm;
      int nm;
      scan(mid + 1, sm, nm);
      if (sm < want) hi = mid;
      else lo = mid + 1;
    }
    double s0, s1;
    int n0, n1;
    scan(lo, s0, n0);
    scan(lo + 1, s1, n1);
    int64_t keep = n0 > n1 ? (int64_t)ceil((want - s1) / ((s0 - s1) / (n0 - n1))) : 0;
    keep = keep < 1 ? 1 : keep;
    if (lo > key || keep < ties) ties = lo > key ? keep : (keep < ties ? keep : ties);
    key = lo;
  }
  // index of the last kept tie
  int last = V - 1;
  {
    int lo = 0, hi = V - 1;  // smallest index with at least `ties` ties at or before it
    double sd;
    int nt;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      sd = 0, nt = 0;
      for (int i = tid; i <= mid; i += kThreads) nt += order_key(logit<T>(row, i)) == key;
      block_sum(sd, nt, buf, nbuf);
      if (nt >= ties) hi = mid;
      else lo = mid + 1;
    }
    last = lo;
  }
  // argmax over the kept
  float best = -INFINITY, zbest = 0.f, part = 0.f;
  int at = V;
  for (int i = tid; i < V; i += kThreads) {
    const float x = logit<T>(row, i);
    const uint32_t k = order_key(x);
    if (!(k > key || (k == key && i <= last))) continue;
    const float z = z_of(x, m, td), w = expf(z);
    if (!(w >= min_p)) continue;
    part += w;
    const float gi = g[i], v = gi == gi ? z + gi : -INFINITY;
    if (at == V || v > best) best = v, at = i, zbest = z;
  }
  s = part, n = 0;
  block_sum(s, n, buf, nbuf);
  __shared__ int ibuf[32];
  __shared__ float zbuf[32];
  for (int d = 16; d; d >>= 1) {
    const float b = __shfl_xor_sync(0xffffffffu, best, d), zb = __shfl_xor_sync(0xffffffffu, zbest, d);
    const int a = __shfl_xor_sync(0xffffffffu, at, d);
    if (b > best || (b == best && a < at)) best = b, at = a, zbest = zb;
  }
  if ((tid & 31) == 0) fbuf[tid >> 5] = best, ibuf[tid >> 5] = at, zbuf[tid >> 5] = zbest;
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < kThreads / 32; ++i)
      if (fbuf[i] > best || (fbuf[i] == best && ibuf[i] < at)) best = fbuf[i], at = ibuf[i], zbest = zbuf[i];
    c.token[r] = at;
    if (c.logprob) c.logprob[r] = (float)((double)zbest - log(s));
  }
}

}  // namespace
}  // namespace mf

using namespace mf;

extern "C" int mf_sample(const mf_sample_args_t* a, void* stream) {
  if (!a || a->n_rows < 0 || a->vocab < 1 || a->vocab > kMaxVocab) return MF_E_INVAL;
  if (a->dtype != MF_F32 && a->dtype != MF_F16 && a->dtype != MF_BF16) return MF_E_INVAL;
  if (a->n_rows == 0) return MF_OK;
  if (!a->logits || !a->noise || !a->token) return MF_E_INVAL;
  const uintptr_t word = (uintptr_t)a->noise | (uintptr_t)a->temperature | (uintptr_t)a->top_p | (uintptr_t)a->min_p |
                         (uintptr_t)a->top_k | (uintptr_t)a->token | (uintptr_t)a->logprob;
  if ((word & 3) || ((uintptr_t)a->logits & (a->dtype == MF_F32 ? 3 : 1))) return MF_E_INVAL;
  if (a->n_rows > 1 && (a->logits_stride < a->vocab || a->noise_stride < a->vocab)) return MF_E_INVAL;
  SampleCall c = {a->logits, a->noise, a->temperature, a->top_p, a->min_p, a->top_k, a->token, a->logprob,
                  a->logits_stride, a->noise_stride, a->vocab};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a->dtype == MF_F32) k_sample_simple<float><<<a->n_rows, kThreads, 0, s>>>(c);
  else if (a->dtype == MF_F16) k_sample_simple<__half><<<a->n_rows, kThreads, 0, s>>>(c);
  else k_sample_simple<__nv_bfloat16><<<a->n_rows, kThreads, 0, s>>>(c);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_sample");
}

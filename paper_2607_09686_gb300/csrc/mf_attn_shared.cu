// Paged attention of sequences that share their first lines.  Contract: mawforge.h.
//
// A warp has a (token, head): its row of q in registers, the lines one after the other, those that the group shares from the pages of
// the group's first sequence.  A running maximum and sum.
#include "mf_attn.cuh"

namespace mf {
namespace {

template <class T, int D>
__global__ void __launch_bounds__(128) k_attn_shared_simple(const __grid_constant__ AttnCall c, const __grid_constant__ SharedGroups g) {
  constexpr int kE = D / 32;
  const AttnStep& st = c.st;
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  pdl_wait();
  if (unit >= (int64_t)st.n_tokens * st.Hq) return;
  const int t = (int)(unit / st.Hq), head = (int)(unit % st.Hq), h = head / st.G;
  int s = t;
  if (st.q_start) {
    s = 0;
    for (int i = 0; i < st.n_seqs; ++i) s += __ldg(st.q_start + i + 1) <= t;
  }
  if (s >= st.n_seqs) return;
  const SeqSpan sp = seq_span(st, s);
  if (t < sp.q0 || t >= sp.q0 + sp.n) return;
  int from = s, skip = 0;
  for (int i = 0; i < g.n; ++i) {
    const int a0 = __ldg(g.first + i), b0 = __ldg(g.first + i + 1);
    const int a = min(max(a0, 0), st.n_seqs), b = min(max(b0, a), st.n_seqs);
    if (a != a0 || b != b0) attn_report(st, kAttnRange);
    if (s < a || s >= b) continue;
    int len = __ldg(g.len + i);
    const int asked = len;
    for (int q = a; q < b; ++q) {
      const SeqSpan o = seq_span(st, q);
      len = min(len, o.len - o.n);
    }
    len = max(len, 0);
    if (len != asked) attn_report(st, kAttnRange);
    from = a, skip = len / st.page_size * st.page_size;
  }
  const int pos = sp.len - sp.n + t - sp.q0, hi = vis_hi(c, pos, sp.len);
  float q[kE], o[kE];
  const T* src = static_cast<const T*>(c.q) + (int64_t)t * c.q_stride + (int64_t)head * D + lane * kE;
#pragma unroll
  for (int i = 0; i < kE; ++i) q[i] = (float)src[i], o[i] = 0.f;
  float m = -INFINITY, l = 0.f;
  for (int x = 0; x < hi; ++x) {
    const int64_t at = line_offset(st, x < skip ? from : s, x) + (int64_t)h * st.head_stride + lane * kE;
    const T *k = static_cast<const T*>(c.k) + at, *v = static_cast<const T*>(c.v) + at;
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < kE; ++i) z += q[i] * (float)k[i];
#pragma unroll
    for (int d = 16; d; d >>= 1) z += __shfl_xor_sync(0xffffffffu, z, d);
    z *= c.scale;
    const float mn = fmaxf(m, z), ms = mn == -INFINITY ? 0.f : mn, f = expf(m - ms), p = expf(z - ms);
    m = mn, l = l * f + p;
#pragma unroll
    for (int i = 0; i < kE; ++i) o[i] = o[i] * f + p * (float)v[i];
  }
  T* dst = static_cast<T*>(c.out) + (int64_t)t * c.out_stride + (int64_t)head * D + lane * kE;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < kE; ++i) dst[i] = T(o[i] * inv);
  if (c.lse && lane == 0) c.lse[(int64_t)t * st.Hq + head] = l == 0.f ? -INFINITY : m + logf(l);
}

template <class T, int D>
cudaError_t run(const AttnCall& c, const SharedGroups& g, cudaStream_t s) {
  const int64_t units = (int64_t)c.st.n_tokens * c.st.Hq;
  return launch_pdl(true, k_attn_shared_simple<T, D>, dim3((unsigned)((units + 3) / 4)), dim3(128), 0, s, c, g);
}

}  // namespace

cudaError_t launch_attn_shared(const AttnCall& c, const SharedGroups& g, int head_dim, bool bf16, cudaStream_t s) {
  if (bf16)
    return head_dim == 64    ? run<__nv_bfloat16, 64>(c, g, s)
           : head_dim == 128 ? run<__nv_bfloat16, 128>(c, g, s)
                             : run<__nv_bfloat16, 256>(c, g, s);
  return head_dim == 64 ? run<__half, 64>(c, g, s) : head_dim == 128 ? run<__half, 128>(c, g, s) : run<__half, 256>(c, g, s);
}

}  // namespace mf

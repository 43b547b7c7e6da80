// Paged attention, one warp per (token, query head): o = sum_j softmax_j(scale q.k_j) v_j over the lines the token
// sees, in one pass with the running maximum m and sum l: when m grows to m', what was summed is scaled by
// exp(m - m').  Each lane holds D / 32 elements of q and o; a score is a warp sum.
#include "mf_attn.cuh"

namespace mf {
namespace {

template <class T, int D>
__global__ void __launch_bounds__(256) k_attn_rows(AttnCall c) {
  constexpr int W = D / 64;  // 32-bit words of a row per lane
  const AttnStep& st = c.st;
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int t = (int)(row / st.Hq), h = (int)(row % st.Hq);
  if (t >= st.n_tokens) return;
  int s = t;
  if (st.q_start) {
    s = 0;
    for (int base = 0; base < st.n_seqs; base += 32) {
      const int i = base + lane;
      s += __popc(__ballot_sync(0xffffffffu, i < st.n_seqs && __ldg(st.q_start + i + 1) <= t));
    }
  }
  if (s >= st.n_seqs) return;
  const SeqSpan sp = seq_span(st, s);
  if (t < sp.q0 || t >= sp.q0 + sp.n) return;
  const int pos = sp.len - sp.n + t - sp.q0;
  const int lo = vis_lo(c, pos), hi = vis_hi(c, pos, sp.len);
  const uint32_t* q = reinterpret_cast<const uint32_t*>(static_cast<const T*>(c.q) + (int64_t)t * c.q_stride + (int64_t)h * D);
  float2 qv[W], o[W];
#pragma unroll
  for (int i = 0; i < W; ++i) qv[i] = Half2<T>::up(q[i * 32 + lane]), o[i] = make_float2(0.f, 0.f);
  float m = -INFINITY, l = 0.f;
  for (int j = lo; j < hi; ++j) {
    const int64_t at = line_offset(st, s, j) + (int64_t)(h / st.G) * st.head_stride;
    const uint32_t* k = reinterpret_cast<const uint32_t*>(static_cast<const T*>(c.k) + at);
    const uint32_t* v = reinterpret_cast<const uint32_t*>(static_cast<const T*>(c.v) + at);
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float2 kv = Half2<T>::up(k[i * 32 + lane]);
      x += qv[i].x * kv.x + qv[i].y * kv.y;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    x *= c.scale;
    const float mn = fmaxf(m, x), f = expf(m - mn), p = expf(x - mn);
    m = mn;
    l = l * f + p;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float2 vv = Half2<T>::up(v[i * 32 + lane]);
      o[i].x = o[i].x * f + p * vv.x;
      o[i].y = o[i].y * f + p * vv.y;
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<T*>(c.out) + (int64_t)t * c.out_stride + (int64_t)h * D);
#pragma unroll
  for (int i = 0; i < W; ++i) out[i * 32 + lane] = Half2<T>::down(o[i].x * inv, o[i].y * inv);
  if (c.lse && lane == 0) c.lse[(int64_t)t * st.Hq + h] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace

cudaError_t launch_attn(const AttnCall& c, int head_dim, bool bf16, cudaStream_t s) {
  const unsigned blocks = (unsigned)(((int64_t)c.st.n_tokens * c.st.Hq + 7) / 8);
  if (bf16) {
    if (head_dim == 64) k_attn_rows<__nv_bfloat16, 64><<<blocks, 256, 0, s>>>(c);
    else if (head_dim == 128) k_attn_rows<__nv_bfloat16, 128><<<blocks, 256, 0, s>>>(c);
    else k_attn_rows<__nv_bfloat16, 256><<<blocks, 256, 0, s>>>(c);
  } else {
    if (head_dim == 64) k_attn_rows<__half, 64><<<blocks, 256, 0, s>>>(c);
    else if (head_dim == 128) k_attn_rows<__half, 128><<<blocks, 256, 0, s>>>(c);
    else k_attn_rows<__half, 256><<<blocks, 256, 0, s>>>(c);
  }
  return cudaGetLastError();
}

}  // namespace mf

// Append of new tokens with the norms of q and k: for each head y = x / sqrt(mean(x^2) + eps) * (w + offset), then the rotation by
// position, q to its place, k and v into their lines.
//
// Everything is read and written once: a copy, bounded by memory (few tokens: by its launch and a chain of look-ups).  A head's
// 4, 8 or 16 lanes hold it whole, 16 elements each (two 16-byte vectors: the two halves of eight rotated pairs, or 16
// neighbours when interleaved or not rotated), so that the mean is a few shuffles.  A block has kTB tokens, as in the append without norms: its
// threads ask for their first vectors, then a warp a token looks up where it goes, the weights and the tokens' angles come into
// shared memory, laid out as the lanes read them, and each thread takes two items at a time.  Arithmetic on pairs of floats (f32x2).
//
// Measured, in a graph: 8192 tokens of 32 + 2 x 4 heads of 128 (168 MB and the angles) 38.2 us, 4.5 TB/s, 65 % of the issue slots (the
// append without norms 36.2); three prompts, 5400 tokens in all, of 16 + 2 x 4 heads of 256, fp16, a quarter rotated by three axes 35.0
// us, 3.8 TB/s (28.5); one token 3.1 us, 64 tokens 3.9.  Four tokens a block where that gives two blocks an SM (two tokens 45.6 and 39.7
// us, eight 36.6 and 38.9), else one, for latency; four blocks an SM (three 43.8 and 35.7, five, with registers spilled, 40.1 and 35.0).
#include "mf_attn.cuh"
#include "mf_tc.cuh"

namespace mf {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t neg2(uint64_t a) { return a ^ 0x8000000080000000ull; }

template <class T, int D, int kTB>
__global__ void __launch_bounds__(kThreads, 4) k_append_norm(const __grid_constant__ AppendCall c, const __grid_constant__ AppendNorm n,
                                                             FastDiv by_items) {
  constexpr int kPer = D / 16;  // lanes of a head
  const AttnStep& st = c.st;
  __shared__ int64_t s_at[kTB];
  __shared__ int s_line[kTB];  // the token's line; -1: not stored
  __shared__ float4 s_angle[kTB][4][16];  // (cos, cos, sin, sin) of pairs 2u and 2u + 1 of a lane's eight, by u and lane
  __shared__ float4 s_weight[2][4][16];   // four of a lane's 16 weights of q, of k, offset added
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, t0 = blockIdx.x * kTB, tokens = min(kTB, st.n_tokens - t0);
  const int q_heads = c.q ? st.Hq : 0, n_items = (q_heads + 2 * st.Hkv) * kPer, total = tokens * n_items;
  pdl_wait();

  struct Item {
    uint4 a, b;
    int64_t at;          // element of the destination (a head of a cache line: from the line's beginning)
    int e0, e1, k, j;    // elements of the two vectors; token, place in the head
    int kind;            // 0: q, 1: k, 2: v, 3: none
  };
  auto load = [&](int i, Item& it) {
    it.kind = 3, it.a = it.b = make_uint4(0, 0, 0, 0), it.k = 0, it.j = i % kPer;
    const bool split = it.j * 8 < c.half && !c.interleaved;
    it.e0 = split ? it.j * 8 : it.j * 16, it.e1 = split ? it.e0 + c.half : it.e0 + 8;
    if (i >= total) return;
    const int k = kTB == 1 ? 0 : (int)fast_div((uint32_t)i, by_items.mul, by_items.shift), head = (i - k * n_items) / kPer;
    it.k = k;
    it.kind = head < q_heads ? 0 : head < q_heads + st.Hkv ? 1 : 2;
    const int h = it.kind == 0 ? head : it.kind == 1 ? head - q_heads : head - q_heads - st.Hkv;
    const T* src = static_cast<const T*>(it.kind == 0 ? c.q : it.kind == 1 ? c.k : c.v) +
                   (int64_t)(t0 + k) * (it.kind == 0 ? c.q_stride : it.kind == 1 ? c.k_stride : c.v_stride) + h * D;
    it.at = it.kind == 0 ? (int64_t)(t0 + k) * c.q_out_stride + h * D : (int64_t)h * st.head_stride;
    it.a = *reinterpret_cast<const uint4*>(src + it.e0), it.b = *reinterpret_cast<const uint4*>(src + it.e1);
  };
  auto store = [&](Item& it) {  // (every lane of the warp)
    uint32_t wa[4] = {it.a.x, it.a.y, it.a.z, it.a.w}, wb[4] = {it.b.x, it.b.y, it.b.z, it.b.w};
    const bool normed = it.kind == 0 ? n.q_weight != nullptr : it.kind == 1 && n.k_weight, turn = it.kind < 2 && it.j * 8 < c.half;
    uint64_t x[4], y[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float2 f = Half2<T>::up(wa[u]), g = Half2<T>::up(wb[u]);
      x[u] = tc::pack2(f.x, f.y), y[u] = tc::pack2(g.x, g.y);
    }
    // the sum of squares in fp32 (a tree: its error is some 20 roundings'); where it passes the largest float the values are
    // taken times 2^-70, whose squares fit, and eps is nothing beside them
    auto sum_of = [&](float f) {
      const uint64_t f2 = tc::pack2(f, f);
      uint64_t s0 = 0, s1 = 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint64_t v = mul2(x[u], f2), z = mul2(y[u], f2);
        s0 = tc::fma2(v, v, s0), s1 = tc::fma2(z, z, s1);
      }
      float lo, hi;
      tc::unpack2(tc::add2(s0, s1), lo, hi);
      float ss = lo + hi;
#pragma unroll
      for (int d = 1; d < kPer; d <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
      return ss;
    };
    const float ss = sum_of(1.f);
    float rs = rsqrtf(ss * (1.f / D) + n.eps);
    if (__any_sync(0xffffffffu, ss == INFINITY)) {
      const float big = sum_of(0x1p-70f);
      if (ss == INFINITY) rs = rsqrtf(big * (1.f / D)) * 0x1p-70f;
    }
    if (it.kind == 3 || (it.kind > 0 && s_line[it.k] < 0)) return;
    if (normed) {
      const uint64_t rs2 = tc::pack2(rs, rs);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const ulonglong2 p = *reinterpret_cast<const ulonglong2*>(&s_weight[it.kind][u][it.j]),
                         q = *reinterpret_cast<const ulonglong2*>(&s_weight[it.kind][2 + u][it.j]);
        x[2 * u] = mul2(mul2(x[2 * u], rs2), p.x), x[2 * u + 1] = mul2(mul2(x[2 * u + 1], rs2), p.y);
        y[2 * u] = mul2(mul2(y[2 * u], rs2), q.x), y[2 * u + 1] = mul2(mul2(y[2 * u + 1], rs2), q.y);
      }
    }
    if (turn && !c.interleaved) {  // (a, b): (a cos - b sin, b cos + a sin)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const ulonglong2 cs = *reinterpret_cast<const ulonglong2*>(&s_angle[it.k][u][it.j]);
        const uint64_t v = tc::fma2(x[u], cs.x, neg2(mul2(y[u], cs.y)));
        y[u] = tc::fma2(y[u], cs.x, mul2(x[u], cs.y));
        x[u] = v;
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float p0, p1, q0, q1;
      tc::unpack2(x[u], p0, p1), tc::unpack2(y[u], q0, q1);
      if (turn && c.interleaved) {  // each word is a pair
        const float4 f = s_angle[it.k][u >> 1][it.j], g = s_angle[it.k][2 + (u >> 1)][it.j];
        const float cp = u & 1 ? f.y : f.x, sp = u & 1 ? f.w : f.z, cq = u & 1 ? g.y : g.x, sq = u & 1 ? g.w : g.z;
        const float v = p0 * cp - p1 * sp, z = q0 * cq - q1 * sq;
        p1 = p1 * cp + p0 * sp, q1 = q1 * cq + q0 * sq;
        p0 = v, q0 = z;
      }
      if (normed || turn) wa[u] = Half2<T>::down(p0, p1), wb[u] = Half2<T>::down(q0, q1);
    }
    T* to = static_cast<T*>(it.kind == 0 ? c.q_out : it.kind == 1 ? c.kc : c.vc) + it.at + (it.kind == 0 ? 0 : s_at[it.k]);
    *reinterpret_cast<uint4*>(to + it.e0) = make_uint4(wa[0], wa[1], wa[2], wa[3]);
    *reinterpret_cast<uint4*>(to + it.e1) = make_uint4(wb[0], wb[1], wb[2], wb[3]);
  };

  Item x, y;  // both items' loads before the first store, the first ones' before the look-ups
  load(tid, x);
  load(tid + kThreads, y);
  if (warp < tokens) {
    const int t = t0 + warp;
    int s = t;
    if (st.q_start) {
      s = 0;
      for (int base = 0; base < st.n_seqs; base += 32) {
        const int i = base + lane;
        s += __popc(__ballot_sync(0xffffffffu, i < st.n_seqs && __ldg(st.q_start + i + 1) <= t));
      }
    }
    if (lane == 0) {
      int line = -1;
      int64_t at = 0;
      if (s < st.n_seqs) {
        const SeqSpan sp = seq_span(st, s);
        const int at_line = sp.len - sp.n + t - sp.q0;
        if (t >= sp.q0 && t < sp.q0 + sp.n && at_line >= 0) {
          const int pi = (int)fast_div((uint32_t)at_line, st.page_mul, st.page_shift);
          const int page = __ldg(st.pages + (int64_t)s * st.pages_per_seq + pi);
          if (page >= 0 && page < st.n_pages) {
            line = at_line;
            at = (int64_t)page * st.page_stride + (int64_t)(at_line - pi * st.page_size) * st.token_stride;
          }
        }
      }
      if (line < 0) attn_report(st, kAttnRange);
      s_line[warp] = line;
      s_at[warp] = at;
    }
  } else {
    for (int i = tid - 32 * tokens; i < 2 * D; i += kThreads - 32 * tokens) {
      const int kind = i / D, e = i % D;  // which lane's, which of its elements
      const bool low = e < 2 * c.half && !c.interleaved, second = low && e >= c.half;
      const int j = low ? (second ? e - c.half : e) / 8 : e / 16, u = low ? (second ? 8 : 0) + e % 8 : e % 16;
      const void* from = kind ? n.k_weight : n.q_weight;
      const float f = !from ? 0.f : n.f32 ? __ldg(static_cast<const float*>(from) + e) : (float)static_cast<const T*>(from)[e];
      reinterpret_cast<float*>(&s_weight[kind][u >> 2][j])[u & 3] = f + n.offset;
    }
  }
  __syncthreads();
  if (c.half) {
    for (int i = tid; i < tokens * c.half; i += kThreads) {
      const int k = i / c.half, pair = i - k * c.half;
      int p = s_line[k];
      if (c.pos) {
        const int axis = c.n_axes == 1 ? 0 : (pair >= c.end0) + (pair >= c.end1) + (pair >= c.end2);
        p = __ldg(c.pos + (int64_t)axis * st.n_tokens + t0 + k);
      }
      const int pc = min(max(p, 0), c.n_pos - 1);
      if (pc != p) attn_report(st, kAttnRange);
      float* to = reinterpret_cast<float*>(&s_angle[k][(pair & 7) >> 1][pair >> 3]) + (pair & 1);
      to[0] = __ldg(c.cos + (int64_t)pc * c.half + pair), to[2] = __ldg(c.sin + (int64_t)pc * c.half + pair);
    }
    __syncthreads();
  }
  for (int i = tid;;) {  // (a warp's lanes together)
    store(x);
    store(y);
    i += 2 * kThreads;
    if (i - lane >= total) break;
    load(i, x);
    load(i + kThreads, y);
  }
}

template <class T, int D>
cudaError_t run(const AppendCall& c, const AppendNorm& n, cudaStream_t s) {
  const int t = c.st.n_tokens;
  const FastDiv by_items = make_fast_div((uint32_t)(((c.q ? c.st.Hq : 0) + 2 * c.st.Hkv) * (D / 16)));
  auto launch = [&](auto kernel, int tb) { return launch_pdl(true, kernel, dim3((unsigned)((t + tb - 1) / tb)), dim3(kThreads), 0, s, c, n, by_items); };
  return t < 8 * 152 ? launch(k_append_norm<T, D, 1>, 1) : launch(k_append_norm<T, D, 4>, 4);
}

}  // namespace

cudaError_t launch_append_norm(const AppendCall& c, const AppendNorm& n, int head_dim, bool bf16, cudaStream_t s) {
  if (bf16)
    return head_dim == 64    ? run<__nv_bfloat16, 64>(c, n, s)
           : head_dim == 128 ? run<__nv_bfloat16, 128>(c, n, s)
                             : run<__nv_bfloat16, 256>(c, n, s);
  return head_dim == 64 ? run<__half, 64>(c, n, s) : head_dim == 128 ? run<__half, 128>(c, n, s) : run<__half, 256>(c, n, s);
}

}  // namespace mf

// Append of new tokens with the norms of q and k: for each head y = x / sqrt(mean(x^2) + eps) * (w + offset), then the rotation by
// position, q to its place, k and v into their lines.
//
// Everything is read and written once: a copy, bounded by memory (few tokens: by its launch and a chain of look-ups).  A head's
// 4, 8 or 16 lanes hold it whole, 16 elements each (two 16-byte vectors: the two halves of eight rotated pairs, or 16
// neighbours when interleaved or not rotated), so that the mean is a few shuffles.  A row is 32 lanes' worth of a token's heads, 1 KiB; the
// step's rows are one list, shared out evenly over all warps that find room.  A warp copies its rows ahead, kAhead of them under way, into shared
// memory that each lane reads back itself, so nothing waits for another lane: 24 warps of 8 KiB an SM.  (Loads into registers, four rows a
// warp and a warp for each four rows: 106 registers, 16 warps an SM, whose heads were under way for a third of their time; 8192 tokens of 40
// heads of 128 49.6 us.)  At a new token a warp looks up where it goes, its sequence (the ends at or before it are counted), its
// line and its page, and its lanes' angles: a lane has the same place in each of its heads.
#include "mf_attn.cuh"

namespace mf {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kAhead = 8;
constexpr uint32_t kRowBytes = 1024;

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 3) k_append_norm(const __grid_constant__ AppendCall c, const __grid_constant__ AppendNorm n,
                                                             int per_token) {
  constexpr int kPer = D / 16, kHeads = 32 / kPer;  // lanes of a head, heads of a row
  extern __shared__ __align__(128) unsigned char smem[];
  const AttnStep& st = c.st;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // this warp's rows of the list, neighbouring runs on different SMs
  const int64_t total = (int64_t)st.n_tokens * per_token, W = min((int64_t)gridDim.x * kWarps, total);
  const int64_t w = (int64_t)warp * gridDim.x + blockIdx.x, f0 = w < W ? total * w / W : 0, f1 = w < W ? total * (w + 1) / W : 0;
  pdl_wait();
  if (f0 >= f1) return;
  const int j = lane % kPer, q_heads = c.q ? st.Hq : 0, heads = q_heads + 2 * st.Hkv;
  const bool turned = j * 8 < c.half, split = turned && !c.interleaved;
  const int e0 = split ? j * 8 : j * 16, e1 = split ? e0 + c.half : e0 + 8;
  unsigned char* mine = smem + warp * (kAhead * kRowBytes) + lane * 16;
  const uint32_t mine_s = smem_u32(mine);

  // ---- the copies' side
  int rows = (int)(f1 - f0), lt = (int)(f0 / per_token), lr = (int)(f0 - (int64_t)lt * per_token), asked = 0;
  auto ask = [&]() {  // the next row, if there is one; a group either way
    const int head = lr * kHeads + lane / kPer;
    if (asked < rows && head < heads) {
      const bool is_q = head < q_heads, is_v = head >= q_heads + st.Hkv;
      const T* src = is_q   ? static_cast<const T*>(c.q) + (int64_t)lt * c.q_stride + (int64_t)head * D
                     : is_v ? static_cast<const T*>(c.v) + (int64_t)lt * c.v_stride + (int64_t)(head - q_heads - st.Hkv) * D
                            : static_cast<const T*>(c.k) + (int64_t)lt * c.k_stride + (int64_t)(head - q_heads) * D;
      const uint32_t dst = mine_s + (uint32_t)(asked % kAhead) * kRowBytes;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src + e0) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + 512), "l"(src + e1) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ++asked;
    if (++lr == per_token) lr = 0, ++lt;
  };
#pragma unroll 1
  for (int i = 0; i < kAhead; ++i) ask();

  int t = (int)(f0 / per_token), r = (int)(f0 - (int64_t)t * per_token), line = -1;
  int64_t at = 0;
  float co[8], si[8];
  bool fresh = true;
#pragma unroll 1
  for (int i = 0; i < rows; ++i) {
    if (fresh) {
      fresh = false;
      // ---- the token's line and where that lies (every lane the same)
      line = -1, at = 0;
      int s = t;
      if (st.q_start) {
        s = 0;
        for (int base = 0; base < st.n_seqs; base += 32) {
          const int q = base + lane;
          s += __popc(__ballot_sync(0xffffffffu, q < st.n_seqs && __ldg(st.q_start + q + 1) <= t));
        }
      }
      if (s < st.n_seqs) {
        const SeqSpan sp = seq_span(st, s);
        const int x = sp.len - sp.n + t - sp.q0;
        if (t >= sp.q0 && t < sp.q0 + sp.n && x >= 0) {
          const int pi = (int)fast_div((uint32_t)x, st.page_mul, st.page_shift);
          const int page = __ldg(st.pages + (int64_t)s * st.pages_per_seq + pi);
          if (page >= 0 && page < st.n_pages) {
            line = x;
            at = (int64_t)page * st.page_stride + (int64_t)(x - pi * st.page_size) * st.token_stride;
          }
        }
      }
      if (line < 0 && lane == 0) attn_report(st, kAttnRange);
      // ---- this lane's eight angles
      if (turned) {
        auto clamped = [&](int p) {
          const int pc = min(max(p, 0), c.n_pos - 1);
          if (pc != p) attn_report(st, kAttnRange);
          return (int64_t)pc * c.half;
        };
        if (c.n_axes == 1) {
          const int64_t row = clamped(c.pos ? __ldg(c.pos + t) : line) + j * 8;
#pragma unroll
          for (int u = 0; u < 8; u += 4) {
            *reinterpret_cast<float4*>(co + u) = __ldg(reinterpret_cast<const float4*>(c.cos + row + u));
            *reinterpret_cast<float4*>(si + u) = __ldg(reinterpret_cast<const float4*>(c.sin + row + u));
          }
        } else {
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const int pair = j * 8 + u, axis = (pair >= c.end0) + (pair >= c.end1) + (pair >= c.end2);
            const int64_t row = clamped(__ldg(c.pos + (int64_t)axis * st.n_tokens + t));
            co[u] = __ldg(c.cos + row + pair), si[u] = __ldg(c.sin + row + pair);
          }
        }
      }
    }
    const int head = r * kHeads + lane / kPer;
    const bool in = head < heads, is_q = head < q_heads, is_v = head >= q_heads + st.Hkv;
    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
    const unsigned char* slot = mine + (i % kAhead) * kRowBytes;
    const uint4 a = *reinterpret_cast<const uint4*>(slot), b = *reinterpret_cast<const uint4*>(slot + 512);
    uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
    ask();
    float x[8], y[8];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float2 p = Half2<T>::up(in ? wa[u] : 0u), q = Half2<T>::up(in ? wb[u] : 0u);
      x[2 * u] = p.x, x[2 * u + 1] = p.y, y[2 * u] = q.x, y[2 * u + 1] = q.y;
    }
    const void* weight = is_q ? n.q_weight : n.k_weight;
    const bool normed = in && !is_v && weight;
    // the sum of squares in fp32 (a tree: its error is some 20 roundings'); where it passes the largest float the values are
    // taken times 2^-70, whose squares fit, and eps is nothing beside them
    auto sum_of = [&](float f) {
      float ss = 0.f, s2 = 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) ss = fmaf(x[u] * f, x[u] * f, ss), s2 = fmaf(y[u] * f, y[u] * f, s2);
      ss += s2;
#pragma unroll
      for (int d = 1; d < kPer; d <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
      return ss;
    };
    float ss = sum_of(1.f), rs = rsqrtf(ss * (1.f / D) + n.eps);
    if (__any_sync(0xffffffffu, ss == INFINITY)) {
      const float big = sum_of(0x1p-70f);
      if (ss == INFINITY) rs = rsqrtf(big * (1.f / D)) * 0x1p-70f;
    }
    if (normed) {
      auto scaled = [&](float (&v)[8], int e) {
        if (n.f32) {
          const float* q = static_cast<const float*>(weight) + e;
#pragma unroll
          for (int u = 0; u < 8; ++u) v[u] = v[u] * rs * (__ldg(q + u) + n.offset);
        } else {
          const uint4 q = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(weight) + e));
          const uint32_t ws[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float2 f = Half2<T>::up(ws[u]);
            v[2 * u] = v[2 * u] * rs * (f.x + n.offset), v[2 * u + 1] = v[2 * u + 1] * rs * (f.y + n.offset);
          }
        }
      };
      scaled(x, e0), scaled(y, e1);
    }
    if (turned && !is_v) {
      if (c.interleaved) {
#pragma unroll
        for (int u = 0; u < 8; u += 2) {
          const float p = x[u] * co[u / 2] - x[u + 1] * si[u / 2], q = y[u] * co[4 + u / 2] - y[u + 1] * si[4 + u / 2];
          x[u + 1] = x[u + 1] * co[u / 2] + x[u] * si[u / 2], y[u + 1] = y[u + 1] * co[4 + u / 2] + y[u] * si[4 + u / 2];
          x[u] = p, y[u] = q;
        }
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float p = x[u] * co[u] - y[u] * si[u];
          y[u] = y[u] * co[u] + x[u] * si[u];
          x[u] = p;
        }
      }
    }
    if (in && (is_q || line >= 0)) {
      if (normed || (turned && !is_v)) {
#pragma unroll
        for (int u = 0; u < 4; ++u) wa[u] = Half2<T>::down(x[2 * u], x[2 * u + 1]), wb[u] = Half2<T>::down(y[2 * u], y[2 * u + 1]);
      }
      T* dst = is_q   ? static_cast<T*>(c.q_out) + (int64_t)t * c.q_out_stride + (int64_t)head * D
               : is_v ? static_cast<T*>(c.vc) + at + (int64_t)(head - q_heads - st.Hkv) * st.head_stride
                      : static_cast<T*>(c.kc) + at + (int64_t)(head - q_heads) * st.head_stride;
      *reinterpret_cast<uint4*>(dst + e0) = make_uint4(wa[0], wa[1], wa[2], wa[3]);
      *reinterpret_cast<uint4*>(dst + e1) = make_uint4(wb[0], wb[1], wb[2], wb[3]);
    }
    if (++r == per_token) r = 0, ++t, fresh = true;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <class T, int D>
cudaError_t run(const AppendCall& c, const AppendNorm& n, cudaStream_t s) {
  constexpr int kHeads = 32 * 16 / D;
  constexpr size_t smem = kWarps * kAhead * kRowBytes;
  const int per_token = ((c.q ? c.st.Hq : 0) + 2 * c.st.Hkv + kHeads - 1) / kHeads;
  const int64_t blocks = ((int64_t)c.st.n_tokens * per_token + kWarps - 1) / kWarps, fit = 3 * 152;  // (this GPU's SMs)
  const cudaError_t e = cudaFuncSetAttribute(k_append_norm<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  return e == cudaSuccess ? launch_pdl(true, k_append_norm<T, D>, dim3((unsigned)(blocks < fit ? blocks : fit)), dim3(kThreads), smem, s, c, n, per_token)
                          : e;
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

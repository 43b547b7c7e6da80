// Append of new tokens with the norms of q and k: for each head y = x / sqrt(mean(x^2) + eps) * (w + offset), then the rotation by
// position, q to its place, k and v into their lines.
//
// Everything is read and written once: a copy, bounded by memory (few tokens: by its launch and a chain of look-ups).  A head's
// 4, 8 or 16 lanes hold it whole, 16 elements each (two 16-byte vectors: the two halves of eight rotated pairs, or 16
// neighbours when interleaved or not rotated), so that the mean is a few shuffles and nothing passes through shared memory.  A warp takes
// part of one token's heads, and asks for them before it looks up where the token goes: its sequence (the ends at or
// before it are counted), its line and its page lie one behind the other, and the heads arrive meanwhile.  A lane
// has the same place in each of its heads, so their angles are fetched once.
#include "mf_attn.cuh"

namespace mf {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMost = 4;  // rows (32 lanes' worth of heads) of a warp

template <class T, int D>
__global__ void __launch_bounds__(kThreads) k_append_norm(const __grid_constant__ AppendCall c, const __grid_constant__ AppendNorm n,
                                                          int parts, int rows_per) {
  constexpr int kPer = D / 16, kHeads = 32 / kPer;  // lanes of a head, heads of a row
  const AttnStep& st = c.st;
  const int lane = threadIdx.x & 31, unit = (int)blockIdx.x * kWarps + (int)(threadIdx.x >> 5);
  const int t = unit / parts, part = unit - t * parts;
  pdl_wait();
  if (t >= st.n_tokens) return;
  const int j = lane % kPer, q_heads = c.q ? st.Hq : 0, heads = q_heads + 2 * st.Hkv;
  const int head0 = part * rows_per * kHeads + lane / kPer;
  const bool turned = j * 8 < c.half, split = turned && !c.interleaved;
  const int e0 = split ? j * 8 : j * 16, e1 = split ? e0 + c.half : e0 + 8;

  uint4 a[kMost], b[kMost];
#pragma unroll
  for (int u = 0; u < kMost; ++u) {
    const int head = head0 + u * kHeads;
    a[u] = b[u] = make_uint4(0, 0, 0, 0);
    if (u < rows_per && head < heads) {
      const bool is_q = head < q_heads, is_v = head >= q_heads + st.Hkv;
      const T* src = is_q   ? static_cast<const T*>(c.q) + (int64_t)t * c.q_stride + (int64_t)head * D
                     : is_v ? static_cast<const T*>(c.v) + (int64_t)t * c.v_stride + (int64_t)(head - q_heads - st.Hkv) * D
                            : static_cast<const T*>(c.k) + (int64_t)t * c.k_stride + (int64_t)(head - q_heads) * D;
      a[u] = *reinterpret_cast<const uint4*>(src + e0), b[u] = *reinterpret_cast<const uint4*>(src + e1);
    }
  }

  // ---- the token's line and where that lies (every lane the same)
  int s = t, line = -1;
  int64_t at = 0;
  if (st.q_start) {
    s = 0;
    for (int base = 0; base < st.n_seqs; base += 32) {
      const int i = base + lane;
      s += __popc(__ballot_sync(0xffffffffu, i < st.n_seqs && __ldg(st.q_start + i + 1) <= t));
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
  float co[8], si[8];
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

#pragma unroll
  for (int u = 0; u < kMost; ++u) {
    const int head = head0 + u * kHeads;
    const bool in = u < rows_per && head < heads, is_q = head < q_heads, is_v = head >= q_heads + st.Hkv;
    if (u >= rows_per) break;
    uint32_t wa[4] = {a[u].x, a[u].y, a[u].z, a[u].w}, wb[4] = {b[u].x, b[u].y, b[u].z, b[u].w};
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = Half2<T>::up(wa[i]), q = Half2<T>::up(wb[i]);
      x[2 * i] = p.x, x[2 * i + 1] = p.y, y[2 * i] = q.x, y[2 * i + 1] = q.y;
    }
    const void* weight = is_q ? n.q_weight : n.k_weight;
    const bool normed = in && !is_v && weight;
    // the sum of squares in fp32 (a tree: its error is some 20 roundings'); where it passes the largest float the values are
    // taken times 2^-70, whose squares fit, and eps is nothing beside them
    auto sum_of = [&](float f) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i] * f, x[i] * f, fmaf(y[i] * f, y[i] * f, ss));
#pragma unroll
      for (int d = 1; d < kPer; d <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
      return ss;
    };
    float ss = sum_of(1.f), r = rsqrtf(ss * (1.f / D) + n.eps);
    if (__any_sync(0xffffffffu, ss == INFINITY)) {
      const float big = sum_of(0x1p-70f);
      if (ss == INFINITY) r = rsqrtf(big * (1.f / D)) * 0x1p-70f;
    }
    if (normed) {
      auto scaled = [&](float (&v)[8], int e) {
        if (n.f32) {
          const float* w = static_cast<const float*>(weight) + e;
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = v[i] * r * (__ldg(w + i) + n.offset);
        } else {
          const uint4 w = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(weight) + e));
          const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 f = Half2<T>::up(ws[i]);
            v[2 * i] = v[2 * i] * r * (f.x + n.offset), v[2 * i + 1] = v[2 * i + 1] * r * (f.y + n.offset);
          }
        }
      };
      scaled(x, e0), scaled(y, e1);
    }
    if (turned && !is_v) {
      if (c.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float p = x[i] * co[i / 2] - x[i + 1] * si[i / 2], q = y[i] * co[4 + i / 2] - y[i + 1] * si[4 + i / 2];
          x[i + 1] = x[i + 1] * co[i / 2] + x[i] * si[i / 2], y[i + 1] = y[i + 1] * co[4 + i / 2] + y[i] * si[4 + i / 2];
          x[i] = p, y[i] = q;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float p = x[i] * co[i] - y[i] * si[i];
          y[i] = y[i] * co[i] + x[i] * si[i];
          x[i] = p;
        }
      }
    }
    if (!in || (!is_q && line < 0)) continue;
    if (normed || (turned && !is_v)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) wa[i] = Half2<T>::down(x[2 * i], x[2 * i + 1]), wb[i] = Half2<T>::down(y[2 * i], y[2 * i + 1]);
    }
    T* dst = is_q   ? static_cast<T*>(c.q_out) + (int64_t)t * c.q_out_stride + (int64_t)head * D
             : is_v ? static_cast<T*>(c.vc) + at + (int64_t)(head - q_heads - st.Hkv) * st.head_stride
                    : static_cast<T*>(c.kc) + at + (int64_t)(head - q_heads) * st.head_stride;
    *reinterpret_cast<uint4*>(dst + e0) = make_uint4(wa[0], wa[1], wa[2], wa[3]);
    *reinterpret_cast<uint4*>(dst + e1) = make_uint4(wb[0], wb[1], wb[2], wb[3]);
  }
}

template <class T, int D>
cudaError_t run(const AppendCall& c, const AppendNorm& n, cudaStream_t s) {
  constexpr int kHeads = 32 * 16 / D;
  const int rows = ((c.q ? c.st.Hq : 0) + 2 * c.st.Hkv + kHeads - 1) / kHeads;
  const int parts = (rows + kMost - 1) / kMost, rows_per = (rows + parts - 1) / parts;
  const int64_t units = (int64_t)c.st.n_tokens * parts;
  return launch_pdl(true, k_append_norm<T, D>, dim3((unsigned)((units + kWarps - 1) / kWarps)), dim3(kThreads), 0, s, c, n, parts,
                    rows_per);
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

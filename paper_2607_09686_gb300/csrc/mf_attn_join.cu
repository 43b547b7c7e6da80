// The partials of paged attention joined: out = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p over a row's pieces in their
// order, M the largest m_p.  A copy's work: bounded by the launch for the few pieces of a balanced split, by reading them
// where one sequence is cut for all blocks.  Threads hold four columns each.  A block takes one row, its groups of threads
// the pieces in turn (many pieces), or one row a group (few pieces).  After one token over 1001 lines (104 pieces) some 3 us with
// its launch.
#include "mf_attn.cuh"

namespace mf {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kFew = 8;  // pieces up to which a row is one group of threads' work

template <int D>
struct Join {
  static constexpr int kCols = D / 4, kThreads = D == 256 ? 512 : 256, kGroups = kThreads / kCols;
};

template <class T, int D, bool kOneRow, bool kTiles>
__device__ __forceinline__ void join_row(const AttnCall& c, const AttnParts& parts, int part_rows, const AttnRec& rec, int b, int r,
                                         int col, int g) {
  using J = Join<D>;
  const int tid = threadIdx.x;
  auto o_of = [&](int64_t row) -> const float4* {  // the row's four columns (kTiles: column group by column group)
    const int64_t part0 = row - r;
    return reinterpret_cast<const float4*>(parts.o + part0 * D + (kTiles ? (col * part_rows + r) * 4 : r * D + col * 4));
  };
  auto row_of = [&](int p) { return (int64_t)(p == 0 ? b * 2 + 1 : (b + p) * 2) * part_rows + r; };
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  float mx = -INFINITY, ls = 0.f;
  if constexpr (kOneRow) {
    __syncthreads();  // the row before this one has been read
    __shared__ float s_w[kMaxParts];
    __shared__ float4 s_o[J::kThreads];
    __shared__ float s_red[2][J::kThreads / 32];
    for (int p = tid; p < rec.n; p += J::kThreads) mx = fmaxf(mx, parts.ml[row_of(p)].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    if ((tid & 31) == 0) s_red[0][tid >> 5] = mx;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < J::kThreads / 32; ++i) mx = fmaxf(mx, s_red[0][i]);
    const float ms = mx == -INFINITY ? 0.f : mx;
    for (int p = tid; p < rec.n; p += J::kThreads) {
      const float2 ml = parts.ml[row_of(p)];
      const float w = exp2f(ml.x - ms);
      s_w[p] = w;
      ls += w * ml.y;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) ls += __shfl_xor_sync(0xffffffffu, ls, d);
    if ((tid & 31) == 0) s_red[1][tid >> 5] = ls;
    __syncthreads();
    ls = 0.f;
#pragma unroll
    for (int i = 0; i < J::kThreads / 32; ++i) ls += s_red[1][i];
#pragma unroll 8
    for (int p = g; p < rec.n; p += J::kGroups) {
      const float w = s_w[p];
      const float4 v = *o_of(row_of(p));
      sum.x += w * v.x, sum.y += w * v.y, sum.z += w * v.z, sum.w += w * v.w;
    }
    s_o[tid] = sum;
    __syncthreads();
    if (g != 0) return;
#pragma unroll
    for (int i = 1; i < J::kGroups; ++i) {
      const float4 v = s_o[i * J::kCols + col];
      sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
    }
  } else {
    for (int p = 0; p < rec.n; ++p) mx = fmaxf(mx, parts.ml[row_of(p)].x);
    const float ms = mx == -INFINITY ? 0.f : mx;
#pragma unroll 2
    for (int p = 0; p < rec.n; ++p) {
      const float2 ml = parts.ml[row_of(p)];
      const float w = exp2f(ml.x - ms);
      const float4 v = *o_of(row_of(p));
      sum.x += w * v.x, sum.y += w * v.y, sum.z += w * v.z, sum.w += w * v.w;
      ls += w * ml.y;
    }
  }
  const int R = rec.row0 + r, tok = rec.q0 + R / c.st.G, head = rec.h * c.st.G + R % c.st.G;
  const float inv = ls == 0.f ? 0.f : 1.f / ls;  // (a NaN in the scores stays NaN)
  T* out = static_cast<T*>(c.out) + (int64_t)tok * c.out_stride + (int64_t)head * D + col * 4;
  *reinterpret_cast<uint2*>(out) =
      make_uint2(Half2<T>::down(sum.x * inv, sum.y * inv), Half2<T>::down(sum.z * inv, sum.w * inv));
  if (c.lse && col == 0) c.lse[(int64_t)tok * c.st.Hq + head] = ls == 0.f ? -INFINITY : (mx + log2f(ls)) * kLn2;
}

// Bounds of groups that fall or lie outside the step, and lengths that a sequence of the group does not have, are reported.
__device__ void look_at_groups(const AttnStep& st, const SharedGroups& g) {
  bool bad = false;
  for (int i = threadIdx.x; i <= g.n; i += blockDim.x) {
    const int x = g.first[i];
    bad |= x < 0 || x > st.n_seqs || (i > 0 && x < g.first[i - 1]);
  }
  if (!__syncthreads_or(bad)) {
    for (int s = threadIdx.x; s < st.n_seqs; s += blockDim.x) {
      int lo = -1, hi = g.n - 1;  // the last group that begins at or before the sequence
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (g.first[mid] <= s) lo = mid;
        else hi = mid - 1;
      }
      if (lo < 0 || s >= g.first[lo + 1]) continue;
      const SeqSpan sp = seq_span(st, s);
      const int len = g.len[lo];
      bad |= len < 0 || len > max(sp.len - sp.n, 0);
    }
  }
  if (bad) attn_report(st, kAttnRange);
}
__global__ void __launch_bounds__(256) k_look(const __grid_constant__ AttnCall c) {
  pdl_wait();
  look_at_groups(c.st, c.look);
}

// kLook: the last block looks at the call's groups.
template <class T, int D, bool kOneRow, bool kTiles, bool kLook>
__global__ void __launch_bounds__(Join<D>::kThreads, 2)
    k_attn_join(const __grid_constant__ AttnCall c, const __grid_constant__ AttnParts parts, int part_rows) {
  using J = Join<D>;
  const int b = blockIdx.x, tid = threadIdx.x;
  pdl_wait();
  if (kLook && b + 1 == gridDim.x) {
    if (blockIdx.y == 0) look_at_groups(c.st, c.look);
    return;
  }
  const AttnRec rec = parts.rec[b];
  if (rec.n == 0) return;
  if (kOneRow && rec.n > kFew) {
    for (int r = blockIdx.y; r < rec.rows; r += gridDim.y)
      join_row<T, D, true, kTiles>(c, parts, part_rows, rec, b, r, tid % J::kCols, tid / J::kCols);
  } else {  // (neighbouring threads take what neighbours in memory: columns, or rows as tiles leave them)
    const int col = kTiles ? tid / J::kGroups : tid % J::kCols, g = kTiles ? tid % J::kGroups : tid / J::kCols;
    for (int r = blockIdx.y * J::kGroups + g; r < rec.rows; r += gridDim.y * J::kGroups)
      join_row<T, D, false, kTiles>(c, parts, part_rows, rec, b, r, col, g);
  }
}

template <class T, int D, bool kLook>
cudaError_t run(const AttnCall& c, const AttnParts& parts, int rows, bool tiles, int blocks, cudaStream_t s) {
  using J = Join<D>;
  // up to 64 rows there may be many pieces of each; with more, a record has few pieces
  const int64_t most = (int64_t)c.st.max_q * c.st.G;
  const int held = (int)(most < rows ? most : rows);
  const int x = blocks + kLook;
  const dim3 one(x, held < 8 ? held : 8), each(x, (held + J::kGroups - 1) / J::kGroups), threads(J::kThreads);
  if (!tiles) return launch_pdl(true, k_attn_join<T, D, true, false, kLook>, one, threads, 0, s, c, parts, rows);
  if (held <= 64) return launch_pdl(true, k_attn_join<T, D, true, true, kLook>, one, threads, 0, s, c, parts, rows);
  return launch_pdl(true, k_attn_join<T, D, false, true, kLook>, each, threads, 0, s, c, parts, rows);
}

template <class T, int D>
cudaError_t pick(const AttnCall& c, const AttnParts& parts, int rows, bool tiles, int blocks, cudaStream_t s) {
  return c.look.n ? run<T, D, true>(c, parts, rows, tiles, blocks, s) : run<T, D, false>(c, parts, rows, tiles, blocks, s);
}

}  // namespace

cudaError_t launch_attn_join(const AttnCall& c, const AttnParts& parts, int head_dim, bool bf16, int rows, bool tiles, int blocks,
                             cudaStream_t s) {
  if (bf16)
    return head_dim == 64    ? pick<__nv_bfloat16, 64>(c, parts, rows, tiles, blocks, s)
           : head_dim == 128 ? pick<__nv_bfloat16, 128>(c, parts, rows, tiles, blocks, s)
                             : pick<__nv_bfloat16, 256>(c, parts, rows, tiles, blocks, s);
  return head_dim == 64    ? pick<__half, 64>(c, parts, rows, tiles, blocks, s)
         : head_dim == 128 ? pick<__half, 128>(c, parts, rows, tiles, blocks, s)
                           : pick<__half, 256>(c, parts, rows, tiles, blocks, s);
}

cudaError_t launch_look(const AttnCall& c, cudaStream_t s) { return launch_pdl(true, k_look, dim3(1), dim3(256), 0, s, c); }

}  // namespace mf

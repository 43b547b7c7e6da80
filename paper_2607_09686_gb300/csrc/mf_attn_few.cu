// Paged attention of few query rows: one token a sequence, or a few whose heads share kv heads, at most 16 rows
// (token, head of the group) for each kv head.
//
// With so few rows every line of K and V is read for a handful of products, so the time is that of reading the
// cache: 2 L Hkv D elements.  Each line is read once per kv head, the rows of its group taking their products from one
// copy on chip (mma.sync m16n8k16: its 16 rows fit; a tcgen05 tile has 128 and its set-up costs more than these
// products).  The scores' softmax runs in one pass: a running maximum m and sum l per row, o scaled by 2^(m - m') when m
// grows to m' (log2 domain, scale folded in).
//
// Split.  The step's work is one list of tiles of 64 lines, sequence by sequence, kv head by kv head; block b of B
// takes the b-th B-th of it, wherever that starts or ends, so lengths may differ as they like.  What a block holds of
// a (sequence, head) it does not have whole it leaves as a partial (o, m, l), and k_attn_join adds those up in
// their order (no atomics: the same bits every time).  A block has at most two partials: its first and its last piece.
//
// Inside a block four warps take 16 lines of each tile each, with pipelines of their own (cp.async into slots that
// only this warp touches, so nothing in the loop waits for another warp); at a piece's end they put their o into the
// slots just freed and add up.
#include "mf_attn.cuh"

namespace mf {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kUnit = 16;               // lines a warp takes at once
constexpr int kTile = kWarps * kUnit;   // lines of a tile
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int D>
struct Cfg {
  static constexpr int kStages = D == 64 ? 5 : 3;
  static constexpr int kBlocksPerSm = D == 64 ? 2 : D == 128 ? 2 : 1;
  static constexpr uint32_t kRow = D * 2;                  // bytes of a line
  static constexpr uint32_t kSlot = 2 * kUnit * kRow;      // K then V of a unit; = 16 rows of o in fp32
  static constexpr uint32_t kSmem = kWarps * kStages * kSlot;
};

// the tiles of a sequence: lines from `start` (a multiple of 16) to its length
struct Span {
  SeqSpan sp;
  int start, nt;
};
__device__ __forceinline__ Span span_of(const AttnCall& c, int s) {
  Span r;
  r.sp = seq_span(c.st, s);
  const int first = r.sp.len - r.sp.n;  // line of the first new token
  r.start = c.window > 0 ? max(0, first - c.window + 1) & ~(kUnit - 1) : 0;
  r.nt = r.sp.n == 0 ? 0 : max(1, (r.sp.len - r.start + kTile - 1) / kTile);
  return r;
}

// a place in the list of tiles
struct Cursor {
  Span sn;
  int s, h, j;
  __device__ __forceinline__ void settle(const AttnCall& c) {  // to the next sequence that has tiles
    while (s < c.st.n_seqs) {
      sn = span_of(c, s);
      if (sn.nt) return;
      ++s;
    }
    sn.nt = 0;
  }
  __device__ __forceinline__ void next(const AttnCall& c) {
    if (++j < sn.nt) return;
    j = 0;
    if (++h < c.st.Hkv) return;
    h = 0;
    ++s;
    settle(c);
  }
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
template <class T>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (Half2<T>::kBf16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, Cfg<D>::kBlocksPerSm) k_attn_few(AttnCall c, AttnParts parts) {
  using C = Cfg<D>;
  constexpr int kS = C::kStages, kSteps = D / 16, kChunks = D / 8, kRowsPer = 32 / (kChunks < 32 ? kChunks : 32);
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int64_t s_sum[kWarps];
  __shared__ int64_t s_at;
  __shared__ int s_seq;
  __shared__ float s_m[kWarps][16], s_l[kWarps][16];
  const AttnStep& st = c.st;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();

  // ---- this block's share [t0, t1) of the list, and where it starts
  int64_t total = 0;
  for (int base = 0; base < st.n_seqs; base += kThreads) {
    const int s = base + tid;
    total += s < st.n_seqs ? span_of(c, s).nt : 0;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  if (lane == 0) s_sum[warp] = total;
  __syncthreads();
  total = (s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]) * st.Hkv;
  const int64_t B = min((int64_t)gridDim.x, total);  // every block that works has a tile
  if (tid == 0) parts.rec[blockIdx.x].n = 0;
  if (blockIdx.x >= B) return;
  const int64_t t0 = total * blockIdx.x / B, t1 = total * (blockIdx.x + 1) / B;
  {
    int64_t before = 0;  // tiles of the sequences before this round's
    for (int base = 0; base < st.n_seqs; base += kThreads) {
      const int s = base + tid;
      const int64_t nt = s < st.n_seqs ? (int64_t)span_of(c, s).nt * st.Hkv : 0;
      int64_t pre = nt;  // inclusive prefix
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, pre, d);
        if (lane >= d) pre += o;
      }
      __syncthreads();
      if (lane == 31) s_sum[warp] = pre;
      __syncthreads();
      int64_t round = 0, mine = before;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) mine += s_sum[w];
        round += s_sum[w];
      }
      pre += mine;
      if (nt && t0 >= pre - nt && t0 < pre) s_seq = s, s_at = t0 - (pre - nt);
      before += round;
      if (t0 < before) break;
    }
    __syncthreads();
  }
  Cursor cur;
  cur.s = s_seq;
  cur.sn = span_of(c, cur.s);
  cur.h = (int)(s_at / cur.sn.nt);
  cur.j = (int)(s_at % cur.sn.nt);
  const int n_tiles = (int)(t1 - t0);
  pdl_trigger();  // k_attn_join's blocks may start to wait

  // ---- the copies' side, kS - 1 units ahead
  const uint32_t slots = smem_u32(smem) + warp * (kS * C::kSlot);
  Cursor ld = cur;
  int ld_left = n_tiles;
  int64_t line_at = 0;  // offset of line lane % 16 of the unit to copy next
  bool line_ok = false;
  auto look_up = [&]() {
    const int line = ld.sn.start + ld.j * kTile + warp * kUnit + (lane & 15);
    const int lo = c.window > 0 ? max(0, ld.sn.sp.len - ld.sn.sp.n - c.window + 1) : 0;
    line_ok = ld_left > 0 && line >= lo && line < ld.sn.sp.len;
    if (line_ok) line_at = line_offset(st, ld.s, line) + (int64_t)ld.h * st.head_stride;
  };
  auto copy_unit = [&](int slot) {
    if (ld_left > 0) {
      const uint32_t k0 = slots + slot * C::kSlot;
      const int ok = line_ok;
#pragma unroll
      for (int i = 0; i < kUnit / kRowsPer; ++i) {
        const int row = i * kRowsPer + lane / kChunks, ch = lane % kChunks;
        const int64_t at = __shfl_sync(0xffffffffu, line_at, row) + ch * 8;
        const uint32_t n = __shfl_sync(0xffffffffu, ok, row) ? 16u : 0u;  // other lines: zeros
        const uint32_t o = row * C::kRow + ((ch ^ (row & 7)) << 4);
        cp16(k0 + o, static_cast<const T*>(c.k) + (n ? at : 0), n);
        cp16(k0 + kUnit * C::kRow + o, static_cast<const T*>(c.v) + (n ? at : 0), n);
      }
      --ld_left;
      if (ld_left > 0) ld.next(c);
      look_up();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  look_up();
#pragma unroll
  for (int i = 0; i < kS - 1; ++i) copy_unit(i);

  const float scale = c.scale * kLog2e;
  uint32_t qf[kSteps][4];
  float o[D / 8][4];
  float m[2], l[2];
  int lo[2], hi[2];  // the lines that this thread's two rows see
  int slot = 0, j0 = 0;
  bool fresh = true;
  for (int t = 0; t < n_tiles; ++t) {
    if (fresh) {  // a new (sequence, head): its query rows
      fresh = false;
      j0 = cur.j;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = lane / 4 + 8 * u, i = r / st.G, pos = cur.sn.sp.len - cur.sn.sp.n + i;
        const bool ok = r < cur.sn.sp.n * st.G;
        lo[u] = vis_lo(c, pos);
        hi[u] = ok ? vis_hi(c, pos, cur.sn.sp.len) : 0;
        m[u] = -INFINITY, l[u] = 0.f;
        const T* q = static_cast<const T*>(c.q) + (int64_t)(cur.sn.sp.q0 + (ok ? i : 0)) * c.q_stride +
                     (int64_t)(cur.h * st.G + (ok ? r % st.G : 0)) * D + (lane & 3) * 2;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
          qf[kk][u] = ok ? *reinterpret_cast<const uint32_t*>(q + kk * 16) : 0u;
          qf[kk][2 + u] = ok ? *reinterpret_cast<const uint32_t*>(q + kk * 16 + 8) : 0u;
        }
      }
#pragma unroll
      for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    }
    // this unit's copies have landed (the kS - 2 groups after it may still fly)
    asm volatile("cp.async.wait_group %0;" ::"n"(kS - 2) : "memory");
    __syncwarp();
    copy_unit(slot == 0 ? kS - 1 : slot - 1);  // into the slot that the previous unit left
    const uint32_t kb = slots + slot * C::kSlot, vb = kb + kUnit * C::kRow;
    const int line0 = cur.sn.start + cur.j * kTile + warp * kUnit;
    if (line0 < cur.sn.sp.len) {
      float x[2][2][4];  // [half of the sum][8 lines][fragment]: two chains of products for each
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i >> 3][(i >> 2) & 1][i & 3] = 0.f;
      const int key = (lane >> 4) * 8 + (lane & 7);
#pragma unroll
      for (int kk = 0; kk < kSteps; ++kk) {
        uint32_t b[4];
        ldsm4(kb + key * C::kRow + (((kk * 2 + ((lane >> 3) & 1)) ^ (key & 7)) << 4), b);
        mma16816<T>(x[kk & 1][0], qf[kk], b[0], b[1]);
        mma16816<T>(x[kk & 1][1], qf[kk], b[2], b[3]);
      }
      float sc[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int line = line0 + n * 8 + (lane & 3) * 2 + (i & 1);
          const float v = (x[0][n][i] + x[1][n][i]) * scale;
          sc[n][i] = line >= lo[i >> 1] && line < hi[i >> 1] ? v : -INFINITY;
        }
      float f[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float mx = fmaxf(fmaxf(sc[0][2 * u], sc[0][2 * u + 1]), fmaxf(sc[1][2 * u], sc[1][2 * u + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        const float mn = fmaxf(m[u], mx), ms = mn == -INFINITY ? 0.f : mn;
        f[u] = exp2f(m[u] - ms);
        m[u] = mn;
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) sum += sc[n][2 * u + i] = exp2f(sc[n][2 * u + i] - ms);
        l[u] = l[u] * f[u] + sum;
      }
      if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] *= f[0], o[i][1] *= f[0], o[i][2] *= f[1], o[i][3] *= f[1];
      }
      // the probabilities, rounded to the cache's type (an MMA multiplies equal types): the A operand's layout is
      // that of the scores
      const uint32_t a[4] = {Half2<T>::down(sc[0][0], sc[0][1]), Half2<T>::down(sc[0][2], sc[0][3]),
                             Half2<T>::down(sc[1][0], sc[1][1]), Half2<T>::down(sc[1][2], sc[1][3])};
      const int vkey = ((lane >> 3) & 1) * 8 + (lane & 7);
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        uint32_t b[4];
        ldsm4t(vb + vkey * C::kRow + (((n + (lane >> 4)) ^ (vkey & 7)) << 4), b);
        mma16816<T>(o[n], a, b[0], b[1]);
        mma16816<T>(o[n + 1], a, b[2], b[3]);
      }
    }
    __syncwarp();
    if (cur.j + 1 == cur.sn.nt || t + 1 == n_tiles) {
      // ---- the piece's end: the four warps' parts added up
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        l[u] += __shfl_xor_sync(0xffffffffu, l[u], 1);
        l[u] += __shfl_xor_sync(0xffffffffu, l[u], 2);
        if ((lane & 3) == 0) s_m[warp][lane / 4 + 8 * u] = m[u], s_l[warp][lane / 4 + 8 * u] = l[u];
      }
      float* mine = reinterpret_cast<float*>(smem + (warp * kS + slot) * C::kSlot);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const int col = i * 8 + (lane & 3) * 2;
        *reinterpret_cast<float2*>(mine + (lane / 4) * D + col) = make_float2(o[i][0], o[i][1]);
        *reinterpret_cast<float2*>(mine + (lane / 4 + 8) * D + col) = make_float2(o[i][2], o[i][3]);
      }
      __syncthreads();
      const bool whole = j0 == 0 && cur.j + 1 == cur.sn.nt;
      const int part = blockIdx.x * 2 + (j0 == 0);  // a piece that starts before this block is its first
      const int rows = cur.sn.sp.n * st.G;
      if (j0 == 0 && !whole && tid == 0) {  // the block of the last tile has the last piece
        const int64_t end = t0 + t - cur.j + cur.sn.nt;
        parts.rec[blockIdx.x] = {cur.sn.sp.q0, cur.h, 0, rows, (int)((B * end - 1) / total) - (int)blockIdx.x + 1};
      }
      for (int i = tid; i < rows * (D / 4); i += kThreads) {
        const int r = i / (D / 4), col = i % (D / 4) * 4;
        float mx = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) mx = fmaxf(mx, s_m[w][r]);
        const float ms = mx == -INFINITY ? 0.f : mx;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        float ls = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = exp2f(s_m[w][r] - ms);
          const float4 v = *reinterpret_cast<const float4*>(smem + (w * kS + slot) * C::kSlot + (r * D + col) * 4);
          sum.x += f * v.x, sum.y += f * v.y, sum.z += f * v.z, sum.w += f * v.w;
          ls += f * s_l[w][r];
        }
        if (whole) {
          const float inv = ls > 0.f ? 1.f / ls : 0.f;
          const int tok = cur.sn.sp.q0 + r / st.G, head = cur.h * st.G + r % st.G;
          T* out = static_cast<T*>(c.out) + (int64_t)tok * c.out_stride + (int64_t)head * D + col;
          *reinterpret_cast<uint2*>(out) =
              make_uint2(Half2<T>::down(sum.x * inv, sum.y * inv), Half2<T>::down(sum.z * inv, sum.w * inv));
          if (c.lse && col == 0) c.lse[(int64_t)tok * st.Hq + head] = ls > 0.f ? (mx + log2f(ls)) * kLn2 : -INFINITY;
        } else {
          *reinterpret_cast<float4*>(parts.o + ((int64_t)part * 16 + r) * D + col) = sum;
          if (col == 0) parts.ml[part * 16 + r] = make_float2(mx, ls);
        }
      }
      __syncthreads();
      fresh = true;
    }
    if (++slot == kS) slot = 0;
    if (t + 1 < n_tiles) cur.next(c);
  }
}

template <class T, int D>
cudaError_t run(const AttnCall& c, const AttnParts& parts, int sms, cudaStream_t s) {
  // no more blocks than tiles there can be: the lengths are on the device, the pages they fit in are known
  const int64_t most = (int64_t)c.st.n_seqs * c.st.Hkv * (((int64_t)c.st.cap + kTile - 1) / kTile);
  const int64_t fit = (int64_t)sms * Cfg<D>::kBlocksPerSm;
  const unsigned grid = (unsigned)(most < fit ? most : fit);
  cudaError_t e = cudaFuncSetAttribute(k_attn_few<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<D>::kSmem);
  if (e == cudaSuccess) e = launch_pdl(false, k_attn_few<T, D>, dim3(grid), dim3(kThreads), Cfg<D>::kSmem, s, c, parts);
  if (e == cudaSuccess && grid > 1) e = launch_attn_join(c, parts, D, Half2<T>::kBf16, kFewRows, (int)grid, s);
  return e;
}

}  // namespace

int attn_few_blocks(int sms) { return sms * 2; }

cudaError_t launch_attn_few(const AttnCall& c, const AttnParts& parts, int head_dim, bool bf16, int sms, cudaStream_t s) {
  if (bf16)
    return head_dim == 64    ? run<__nv_bfloat16, 64>(c, parts, sms, s)
           : head_dim == 128 ? run<__nv_bfloat16, 128>(c, parts, sms, s)
                             : run<__nv_bfloat16, 256>(c, parts, sms, s);
  return head_dim == 64    ? run<__half, 64>(c, parts, sms, s)
         : head_dim == 128 ? run<__half, 128>(c, parts, sms, s)
                           : run<__half, 256>(c, parts, sms, s);
}

}  // namespace mf

// Paged attention of few query rows: one token a sequence, or a few whose heads share kv heads, at most 16 MT rows
// (token, head of the group) for each kv head (MT = 1, 2, 3 fragments of rows: as many as registers hold).
//
// With so few rows every line of K and V is read for a handful of products, so the time is that of reading the
// cache: 2 L Hkv D elements.  Each line is read once per kv head, the rows of its group taking their products from one
// copy on chip (mma.sync m16n8k16; a tcgen05 tile has 128 rows and its set-up costs more than these
// products).  The scores' softmax runs in one pass: a running maximum m and sum l per row, o scaled by 2^(m - m') when m
// grows to m' (log2 domain, scale folded in).
//
// Split.  The step's work is one list of tiles of 64 lines, sequence by sequence, kv head by kv head, each (sequence,
// head) preceded by kOver empty tiles for what its beginning and end cost; block b of B takes the b-th B-th of the list,
// wherever that starts or ends, so lengths may differ as they like.  What a block holds of
// a (sequence, head) it does not have whole it leaves as a partial (o, m, l), and mf_attn_join.cu adds those up in
// their order (no atomics: the same bits every time).  A block has at most two partials: its first and its last piece.
//
// Inside a block four warps take 16 lines of each tile each, with pipelines of their own: cp.async into slots that
// only this warp touches, so nothing in the loop waits for another warp, K and V apart, so that a slot is filled again as
// soon as its products are done (128 KiB and more in flight per SM; the copies' depth sets the rate).  At a piece's end
// the warps put their o into the slots just freed and add up.
//
// Measured: 64 sequences of 166 to 8192 lines, 32/4 heads of 128, 395 MB: 74.5 us with the join, 5.3 TB/s (78 % of the copy
// rate; that rate once it runs, 6 us before the first lines are there); one sequence of 131071 lines, 16/2 heads of 256:
// 54.9 us, 4.9 TB/s; one of 1001 lines: 9.8 us, of which 5 are this kernel's and the rest the join's and the launches'.
#include "mf_attn.cuh"

namespace mf {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kUnit = 16;               // lines a warp takes at once
constexpr int kTile = kWarps * kUnit;   // lines of a tile
constexpr int kOver = 3;                // tiles that a (sequence, head) costs besides its own
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int D>
struct Cfg {
  static constexpr int kStages = D == 64 ? 5 : 3;
  static constexpr int kBlocksPerSm = D == 64 ? 2 : D == 128 ? 2 : 1;
  static constexpr uint32_t kRow = D * 2;                  // bytes of a line
  static constexpr uint32_t kHalf = kUnit * kRow, kSlot = 2 * kHalf;  // K, then V of a unit; together 16 rows of o in fp32
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

// a place in a block's share of the list
struct Cursor {
  Span sn;
  int s, h, j, j_end;   // tile j of this (sequence, head), which the block has to j_end
  int64_t at, t1;       // the place of its first (empty) tile in the list, the end of the share
  __device__ __forceinline__ void limit() { j_end = (int)max((int64_t)0, min((int64_t)sn.nt, t1 - at - kOver)); }
  __device__ __forceinline__ void next(const AttnCall& c) {
    if (++j < j_end) return;
    at += sn.nt + kOver;
    j = j_end = 0;
    if (at + kOver >= t1) return;  // (nothing of what follows is this block's)
    if (++h == c.st.Hkv) {
      h = 0;
      do sn = span_of(c, ++s);  // (there is one with tiles: the list goes on)
      while (sn.nt == 0);
    }
    limit();
  }
  __device__ __forceinline__ bool live() const { return j < j_end; }
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
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
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

template <class T, int D, int MT>
__global__ void __launch_bounds__(kThreads, Cfg<D>::kBlocksPerSm) k_attn_few(AttnCall c, AttnParts parts) {
  using C = Cfg<D>;
  constexpr int kS = C::kStages, kSteps = D / 16, kChunks = D / 8, kRowsPer = 32 / (kChunks < 32 ? kChunks : 32);
  constexpr bool kQShared = MT * kSteps > 12;  // the query rows in shared memory, registers being short
  constexpr int kChains = MT == 1 ? 2 : 1;  // independent sums of a score: enough products in flight either way
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int64_t s_sum[kWarps];
  __shared__ int64_t s_at;
  __shared__ int s_seq;
  __shared__ float s_m[kWarps][16], s_l[kWarps][16];
  const AttnStep& st = c.st;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();

  // ---- this block's share [t0, t1) of the list, and where it starts
  auto cost_of = [&](int s) -> int64_t {  // of a kv head of sequence s
    if (s >= st.n_seqs) return 0;
    const int nt = span_of(c, s).nt;
    return nt ? nt + kOver : 0;
  };
  int64_t total = 0;
  for (int base = 0; base < st.n_seqs; base += kThreads) total += cost_of(base + tid);
#pragma unroll
  for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  if (lane == 0) s_sum[warp] = total;
  __syncthreads();
  total = (s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]) * st.Hkv;
  const int64_t B = min((int64_t)gridDim.x, total);
  if (tid == 0) parts.rec[blockIdx.x].n = 0;
  if (blockIdx.x >= B) return;
  const int64_t t0 = total * blockIdx.x / B, t1 = total * (blockIdx.x + 1) / B;
  {
    int64_t before = 0;  // tiles of the sequences before these
    for (int base = 0; base < st.n_seqs; base += kThreads) {
      const int64_t nt = cost_of(base + tid) * st.Hkv;
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
      if (nt && t0 >= pre - nt && t0 < pre) s_seq = base + tid, s_at = pre - nt;
      before += round;
      if (t0 < before) break;
    }
    __syncthreads();
  }
  Cursor cur;
  cur.s = s_seq;
  cur.sn = span_of(c, cur.s);
  cur.h = (int)((t0 - s_at) / (cur.sn.nt + kOver));
  cur.at = s_at + (int64_t)cur.h * (cur.sn.nt + kOver);
  cur.t1 = t1;
  cur.j = (int)max((int64_t)0, t0 - cur.at - kOver);
  cur.limit();
  pdl_trigger();  // k_attn_join's blocks may start to wait
  if (!cur.live()) return;  // (a share of empty tiles alone)

  // ---- the copies' side, kS units ahead
  const uint32_t slots = smem_u32(smem) + warp * (kS * C::kSlot);
  Cursor ld = cur;
  // Where pages hold a multiple of 8 lines, lane L knows where the halves of unit L of 32 begin, from tile `win` of the
  // (sequence, head) on, else lane L % 16 where that line of the unit to copy lies.
  const bool whole_pages = st.page_size % 8 == 0;
  int64_t line_at = 0, half_at = 0, unit_at[2] = {0, 0};
  int win = 0, lo_at = 0, hi_at = 0;  // lines of the unit from lo_at to hi_at are copied, others become zeros
  bool fresh_win = true;
  auto look_up = [&]() {
    if (!ld.live()) return;
    const int line0 = ld.sn.start + ld.j * kTile + warp * kUnit, len = ld.sn.sp.len;
    const int lo = c.window > 0 ? max(0, len - ld.sn.sp.n - c.window + 1) : 0;
    lo_at = lo - line0, hi_at = len - line0;
    if (whole_pages) {
      if (fresh_win || ld.j - win >= 32) {
        fresh_win = false;
        win = ld.j;
        const int line = line0 + lane * kTile;
        if (ld.j + lane < ld.j_end) {
          if (line < len && line + 8 > lo) line_at = line_offset(st, ld.s, line) + (int64_t)ld.h * st.head_stride;
          if (line + 8 < len) half_at = line_offset(st, ld.s, line + 8) + (int64_t)ld.h * st.head_stride;
        }
      }
    } else {
      const int line = line0 + (lane & 15);
      if (line >= lo && line < len) line_at = line_offset(st, ld.s, line) + (int64_t)ld.h * st.head_stride;
    }
  };
  const int sub = lane / kChunks, ch = lane % kChunks;  // this lane's line (of kRowsPer) and chunk in a copy
  const int64_t lane_off = (int64_t)sub * st.token_stride + ch * 8, step = (int64_t)kRowsPer * st.token_stride;
  // K (then V, after which the cursor moves on) of the unit at `ld` to `dst`; one group each, empty past the end
  auto copy_half = [&](uint32_t dst, const void* cache, bool is_v) {
    if (ld.live()) {
      const T* base = static_cast<const T*>(cache);
      if (whole_pages) {
        if (!is_v) {
          unit_at[0] = __shfl_sync(0xffffffffu, line_at, ld.j - win) + lane_off;
          unit_at[1] = __shfl_sync(0xffffffffu, half_at, ld.j - win) + lane_off;
        }
        if (lo_at <= 0 && hi_at >= kUnit) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const T* p = base + unit_at[half];
#pragma unroll
            for (int i = 0; i < 8 / kRowsPer; ++i) {
              const int row = half * 8 + i * kRowsPer + sub;
              cp16(dst + row * C::kRow + ((ch ^ (row & 7)) << 4), p, 16u);
              p += step;
            }
          }
        } else {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const T* p = base + unit_at[half];
#pragma unroll 1
            for (int i = 0; i < 8 / kRowsPer; ++i) {
              const int row = half * 8 + i * kRowsPer + sub;
              const bool in = row >= lo_at && row < hi_at;
              cp16(dst + row * C::kRow + ((ch ^ (row & 7)) << 4), in ? p : base, in ? 16u : 0u);
              p += step;
            }
          }
        }
      } else {
#pragma unroll 1
        for (int i = 0; i < kUnit / kRowsPer; ++i) {
          const int row = i * kRowsPer + sub;
          const int64_t at = __shfl_sync(0xffffffffu, line_at, row) + ch * 8;
          const bool in = row >= lo_at && row < hi_at;
          cp16(dst + row * C::kRow + ((ch ^ (row & 7)) << 4), base + (in ? at : 0), in ? 16u : 0u);
        }
      }
      if (is_v) {
        const int64_t was = ld.at;
        ld.next(c);
        if (ld.at != was) fresh_win = true;
        look_up();
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  look_up();
#pragma unroll 1
  for (int i = 0; i < kS; ++i) {
    copy_half(slots + i * C::kSlot, c.k, false);
    copy_half(slots + i * C::kSlot + C::kHalf, c.v, true);
  }

  const float scale = c.scale * kLog2e;
  uint32_t qf[kQShared ? 1 : MT][kQShared ? 1 : kSteps][4];
  const uint32_t q_at = smem_u32(smem) + C::kSmem;  // [16 MT rows], chunks XORed with the row as in K
  float o[MT][D / 8][4];
  float m[MT][2], l[MT][2];
  int lo[MT][2], hi[MT][2];  // the lines that this thread's rows see
  int slot = 0, j0 = 0;
  bool fresh = true;
#pragma unroll 1
  while (cur.live()) {
    if (fresh) {  // a new (sequence, head): its query rows
      fresh = false;
      j0 = cur.j;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int r = t * 16 + lane / 4 + 8 * u, i = r / st.G, pos = cur.sn.sp.len - cur.sn.sp.n + i;
          const bool ok = r < cur.sn.sp.n * st.G;
          lo[t][u] = vis_lo(c, pos);
          hi[t][u] = ok ? vis_hi(c, pos, cur.sn.sp.len) : 0;
          m[t][u] = -INFINITY, l[t][u] = 0.f;
          if constexpr (!kQShared) {
            const T* q = static_cast<const T*>(c.q) + (int64_t)(cur.sn.sp.q0 + (ok ? i : 0)) * c.q_stride +
                         (int64_t)(cur.h * st.G + (ok ? r % st.G : 0)) * D + (lane & 3) * 2;
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk) {
              qf[t][kk][u] = ok ? *reinterpret_cast<const uint32_t*>(q + kk * 16) : 0u;
              qf[t][kk][2 + u] = ok ? *reinterpret_cast<const uint32_t*>(q + kk * 16 + 8) : 0u;
            }
          }
        }
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[t][i][0] = o[t][i][1] = o[t][i][2] = o[t][i][3] = 0.f;
      }
      if constexpr (kQShared) {  // (the last piece's end has seen every warp past its rows)
        for (int i = tid; i < MT * 16 * kChunks; i += kThreads) {
          const int r = i / kChunks, x = i % kChunks, tok = r / st.G;
          const bool ok = r < cur.sn.sp.n * st.G;
          uint4 v = make_uint4(0, 0, 0, 0);
          if (ok)
            v = *reinterpret_cast<const uint4*>(static_cast<const T*>(c.q) + (int64_t)(cur.sn.sp.q0 + tok) * c.q_stride +
                                                (int64_t)(cur.h * st.G + r % st.G) * D + x * 8);
          *reinterpret_cast<uint4*>(smem + C::kSmem + r * C::kRow + ((x ^ (r & 7)) << 4)) = v;
        }
        __syncthreads();
      }
    }
    const bool ends = cur.j + 1 == cur.j_end;  // the piece's last unit: its slot serves the adding up first
    const uint32_t kb = slots + slot * C::kSlot, vb = kb + C::kHalf;
    const int line0 = cur.sn.start + cur.j * kTile + warp * kUnit;
    const bool some = line0 < cur.sn.sp.len;
    asm volatile("cp.async.wait_group %0;" ::"n"(2 * kS - 1) : "memory");  // this unit's K has landed
    __syncwarp();
    float x[MT][kChains][2][4];
    uint32_t a[MT][4];
    if (some) {
#pragma unroll
      for (int i = 0; i < MT * kChains * 8; ++i) x[i / (kChains * 8)][i / 8 % kChains][(i >> 2) & 1][i & 3] = 0.f;
      const int key = (lane >> 4) * 8 + (lane & 7);
#pragma unroll
      for (int kk = 0; kk < kSteps; ++kk) {
        uint32_t b[4];
        ldsm4(kb + key * C::kRow + (((kk * 2 + ((lane >> 3) & 1)) ^ (key & 7)) << 4), b);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          uint32_t q[4];
          if constexpr (kQShared) {  // matrices: rows 0-7 and 8-15 of the first eight elements, then of the next
            const int r = t * 16 + (lane & 15);
            ldsm4(q_at + r * C::kRow + (((kk * 2 + (lane >> 4)) ^ (r & 7)) << 4), q);
          } else {
            q[0] = qf[t][kk][0], q[1] = qf[t][kk][1], q[2] = qf[t][kk][2], q[3] = qf[t][kk][3];
          }
          mma16816<T>(x[t][kk % kChains][0], q, b[0], b[1]);
          mma16816<T>(x[t][kk % kChains][1], q, b[2], b[3]);
        }
      }
    }
    __syncwarp();
    if (!ends) copy_half(kb, c.k, false);
    if (some) {
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        if constexpr (kChains == 2)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[t][0][i >> 2][i & 3] += x[t][kChains - 1][i >> 2][i & 3];
      }
      // (step by step over all fragments: their chains of shuffles and exponentials run beside each other)
      float f[MT][2], ms[MT][2];
      bool grown = false;
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int line = line0 + n * 8 + (lane & 3) * 2 + (i & 1);
            float& v = x[t][0][n][i];
            v = line >= lo[t][i >> 1] && line < hi[t][i >> 1] ? v * scale : -INFINITY;
          }
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          ms[t][u] = fmaxf(fmaxf(x[t][0][0][2 * u], x[t][0][0][2 * u + 1]), fmaxf(x[t][0][1][2 * u], x[t][0][1][2 * u + 1]));
#pragma unroll
      for (int d = 1; d <= 2; d <<= 1)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int u = 0; u < 2; ++u) ms[t][u] = fmaxf(ms[t][u], __shfl_xor_sync(0xffffffffu, ms[t][u], d));
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float mn = fmaxf(m[t][u], ms[t][u]);
          ms[t][u] = mn == -INFINITY ? 0.f : mn;
          f[t][u] = ex2(m[t][u] - ms[t][u]);
          m[t][u] = mn;
          grown |= f[t][u] != 1.f;
        }
#pragma unroll
      for (int t = 0; t < MT; ++t) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float sum = 0.f;
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) sum += x[t][0][n][2 * u + i] = ex2(x[t][0][n][2 * u + i] - ms[t][u]);
          l[t][u] = l[t][u] * f[t][u] + sum;
        }
        // the probabilities, rounded to the cache's type (an MMA multiplies equal types): the A operand's layout is
        // that of the scores
        a[t][0] = Half2<T>::down(x[t][0][0][0], x[t][0][0][1]), a[t][1] = Half2<T>::down(x[t][0][0][2], x[t][0][0][3]);
        a[t][2] = Half2<T>::down(x[t][0][1][0], x[t][0][1][1]), a[t][3] = Half2<T>::down(x[t][0][1][2], x[t][0][1][3]);
      }
      if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int i = 0; i < D / 8; ++i)
            o[t][i][0] *= f[t][0], o[t][i][1] *= f[t][0], o[t][i][2] *= f[t][1], o[t][i][3] *= f[t][1];
      }
    }
    // this unit's V has landed
    if (ends) asm volatile("cp.async.wait_group %0;" ::"n"(2 * kS - 2) : "memory");
    else asm volatile("cp.async.wait_group %0;" ::"n"(2 * kS - 1) : "memory");
    __syncwarp();
    if (some) {
      const int vkey = ((lane >> 3) & 1) * 8 + (lane & 7);
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        uint32_t b[4];
        ldsm4t(vb + vkey * C::kRow + (((n + (lane >> 4)) ^ (vkey & 7)) << 4), b);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          mma16816<T>(o[t][n], a[t], b[0], b[1]);
          mma16816<T>(o[t][n + 1], a[t], b[2], b[3]);
        }
      }
    }
    __syncwarp();
    if (ends) {
      // ---- the piece's end: the four warps' parts added up, 16 rows at a time
      const bool whole = j0 == 0 && cur.j_end == cur.sn.nt;
      const int part = blockIdx.x * 2 + (j0 == 0);  // a piece that starts before this block is its first
      const int rows = cur.sn.sp.n * st.G;
      if (j0 == 0 && !whole && tid == 0) {  // the block of the last tile has the last piece
        const int64_t end = cur.at + kOver + cur.sn.nt;
        parts.rec[blockIdx.x] = {cur.sn.sp.q0, cur.h, 0, rows, (int)((B * end - 1) / total) - (int)blockIdx.x + 1};
      }
      float* mine = reinterpret_cast<float*>(smem + (warp * kS + slot) * C::kSlot);
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        if (t * 16 >= rows) break;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          l[t][u] += __shfl_xor_sync(0xffffffffu, l[t][u], 1);
          l[t][u] += __shfl_xor_sync(0xffffffffu, l[t][u], 2);
          if ((lane & 3) == 0) s_m[warp][lane / 4 + 8 * u] = m[t][u], s_l[warp][lane / 4 + 8 * u] = l[t][u];
        }
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const int col = i * 8 + (lane & 3) * 2;
          *reinterpret_cast<float2*>(mine + (lane / 4) * D + col) = make_float2(o[t][i][0], o[t][i][1]);
          *reinterpret_cast<float2*>(mine + (lane / 4 + 8) * D + col) = make_float2(o[t][i][2], o[t][i][3]);
        }
        __syncthreads();
        for (int i = tid; i < min(rows - t * 16, 16) * (D / 4); i += kThreads) {
          const int r = i / (D / 4), col = i % (D / 4) * 4, R = t * 16 + r;
          float mx = s_m[0][r];
#pragma unroll
          for (int w = 1; w < kWarps; ++w) mx = fmaxf(mx, s_m[w][r]);
          const float ms = mx == -INFINITY ? 0.f : mx;
          float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
          float ls = 0.f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float f = ex2(s_m[w][r] - ms);
            const float4 v = *reinterpret_cast<const float4*>(smem + (w * kS + slot) * C::kSlot + (r * D + col) * 4);
            sum.x += f * v.x, sum.y += f * v.y, sum.z += f * v.z, sum.w += f * v.w;
            ls += f * s_l[w][r];
          }
          if (whole) {
            const float inv = ls == 0.f ? 0.f : 1.f / ls;  // (a NaN in the scores stays NaN)
            const int tok = cur.sn.sp.q0 + R / st.G, head = cur.h * st.G + R % st.G;
            T* out = static_cast<T*>(c.out) + (int64_t)tok * c.out_stride + (int64_t)head * D + col;
            *reinterpret_cast<uint2*>(out) =
                make_uint2(Half2<T>::down(sum.x * inv, sum.y * inv), Half2<T>::down(sum.z * inv, sum.w * inv));
            if (c.lse && col == 0) c.lse[(int64_t)tok * st.Hq + head] = ls == 0.f ? -INFINITY : (mx + log2f(ls)) * kLn2;
          } else {
            *reinterpret_cast<float4*>(parts.o + ((int64_t)part * (MT * 16) + R) * D + col) = sum;
            if (col == 0) parts.ml[part * (MT * 16) + R] = make_float2(mx, ls);
          }
        }
        __syncthreads();
      }
      fresh = true;
      copy_half(kb, c.k, false);
    }
    copy_half(vb, c.v, true);
    if (++slot == kS) slot = 0;
    cur.next(c);
  }
}

template <class T, int D, int MT>
cudaError_t run(const AttnCall& c, const AttnParts& parts, int sms, cudaStream_t s) {
  // no more blocks than tiles there can be: the lengths are on the device, the pages they fit in are known
  const int64_t most = (int64_t)c.st.n_seqs * c.st.Hkv * (((int64_t)c.st.cap + kTile - 1) / kTile);
  const int64_t fit = (int64_t)sms * Cfg<D>::kBlocksPerSm;
  const unsigned grid = (unsigned)(most < fit ? most : fit);
  constexpr size_t smem = Cfg<D>::kSmem + MT * 16 * Cfg<D>::kRow;  // the pipelines, the query rows
  cudaError_t e = cudaFuncSetAttribute(k_attn_few<T, D, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) e = launch_pdl(true, k_attn_few<T, D, MT>, dim3(grid), dim3(kThreads), smem, s, c, parts);
  if (e == cudaSuccess && grid > 1) e = launch_attn_join(c, parts, D, Half2<T>::kBf16, MT * 16, false, (int)grid, s);
  return e;
}

template <class T>
cudaError_t pick(const AttnCall& c, const AttnParts& parts, int head_dim, int sms, cudaStream_t s) {
  const int rows = c.st.max_q * c.st.G;
  if (head_dim == 256) return run<T, 256, 1>(c, parts, sms, s);
  if (head_dim == 128) return rows <= 16 ? run<T, 128, 1>(c, parts, sms, s) : run<T, 128, 2>(c, parts, sms, s);
  return rows <= 16 ? run<T, 64, 1>(c, parts, sms, s) : rows <= 32 ? run<T, 64, 2>(c, parts, sms, s) : run<T, 64, 3>(c, parts, sms, s);
}

}  // namespace

int attn_few_blocks(int sms) { return sms * 2; }
int attn_few_rows(int head_dim) { return head_dim == 256 ? 16 : head_dim == 128 ? 32 : 48; }

cudaError_t launch_attn_few(const AttnCall& c, const AttnParts& parts, int head_dim, bool bf16, int sms, cudaStream_t s) {
  return bf16 ? pick<__nv_bfloat16>(c, parts, head_dim, sms, s) : pick<__half>(c, parts, head_dim, sms, s);
}

}  // namespace mf

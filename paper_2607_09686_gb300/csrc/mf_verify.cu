// Verification of drafted tokens: the drafts that the target takes, and the token that ends each sequence.  Contract: mawforge.h.
//
// First what each row of the target's logits keeps and the sum of its weights, and the same of the drafter's rows, so that p and q of any entry are a
// few operations on its logit: by k_sample's steps without the draw where rows are cut, else (k_rows) by maxima and sums of
// pieces of them.  Then (k_verify) a cluster of 1 to 8 blocks has a sequence: a warp a draft, p and q of it; the first row whose
// draft is not taken; one pass over that row for the largest log(p - q) + noise.  In that pass log p + noise, a bound of it that
// takes no exponential, is compared with the largest key so far, and only what lies above it is worked out.
// What bounds it: reading the logits (k_rows), then of the rows that decide the logits again and the noise; few sequences, the
// chain of launches and look-ups.  Where rows are cut, k_sample.
//
// Measured, in graphs: 64 sequences of up to 4 drafts and a drafter's rows, 131072 bf16, by temperature: 36.7 us, about 16 of them k_rows'
// (79 MB, 5 TB/s); 64 of up to 8 drafts without a drafter, 50001 bf16: 22.3.  Cut rows: one sequence of 4 drafts, 131072 fp32: 20.8, of
// them 12 k_sample's; 24 of up to 4, 200001 fp16: 77.6, of which k_sample, with 116 rows, has most (by itself 73, the caches cold).
#include <cooperative_groups.h>

#include <cfloat>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "mf_sample.cuh"
#include "mf_tc.cuh"

namespace cg = cooperative_groups;

namespace mf {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// Of a piece of a row: the largest logit, its first index (rows without a temperature), the sum of w against it; in a row's first piece
// their number.
struct Piece {
  float m, s;
  int first, n;
};

struct VerifyCall {
  const void *logits, *draft;
  int64_t logits_stride, draft_stride, noise_stride;
  const int32_t *row_start, *tokens;
  const float *u, *noise;
  const float* temperature[2];  // the target's, the drafter's
  int32_t *token, *accepted;
  float* logprob;
  const Kept* kept;   // [2][rows], of rows that are cut
  Piece* pieces;      // [2][rows][n_units], of others
  int* fall;          // the kernels before k_verify set it to whether row starts fall (of one sequence: they cannot matter)
  int whole[2];       // the target's, the drafter's are not cut
  int n_seqs, n_rows, vocab, n_units, slice;  // units of a row (k_rows); slice: entries of a block of k_verify
  int stages;  // of k_verify's ring
  int hold;    // (a test's) copies are not issued
};

// ---- rows that are not cut
//
// The rows' units of 128 16-byte vectors are one list, shared out evenly: a warp takes a run of units, four vectors a lane at a time while the
// next four are under way, with a running maximum and sum a lane, and leaves a piece where a row or its run ends (which depends on
// the row starts alone).  The list has the target's rows and those of the drafter's that have a draft: every block adds up the sequences' rows
// in shared memory (of more than kSeqs sequences, or starts that fall: all rows, of which some are passed over).  Bounded by
// reading the logits once; of an entry's four instructions (pairs of floats) one is an exponential.
constexpr int kRowThreads = 256, kUnit = 128, kVecs = kUnit / 32, kSeqs = 2048;
template <class T>
constexpr int kUnitEntries = kUnit * 16 / (int)sizeof(T);

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// the largest of the vectors' numbers (-inf: there is none)
template <class T>
__device__ __forceinline__ float largest(const uint4 (&v)[kVecs]) {
  if constexpr (sizeof(T) == 4) {
    float most = -INFINITY;
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      most = fmaxf(most, fmaxf(fmaxf(__uint_as_float(v[k].x), __uint_as_float(v[k].y)), fmaxf(__uint_as_float(v[k].z), __uint_as_float(v[k].w))));
    return most;
  } else {  // pair by pair, as they are
    using P = typename std::conditional<Half2<T>::kBf16, __nv_bfloat162, __half2>::type;
    const uint32_t low = Half2<T>::kBf16 ? 0xFF80FF80u : 0xFC00FC00u;
    P most;
    memcpy(&most, &low, 4);
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      P e[4];
      memcpy(e, &v[k], 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) most = __hmax2(most, e[i]);
    }
    uint32_t w;
    memcpy(&w, &most, 4);
    const float2 f = Half2<T>::up(w);
    return fmaxf(f.x, f.y);
  }
}

template <class T>
__global__ void __launch_bounds__(kRowThreads, 3) k_rows(const __grid_constant__ VerifyCall c, int side0, int rows) {
  constexpr int kV = 16 / sizeof(T);
  const int lane = threadIdx.x & 31;
  // rows before a sequence: the target's, the drafter's
  __shared__ int s_rows[kSeqs + 1], s_drafts[kSeqs + 1];
  __shared__ int2 s_sum[kRowThreads / 32];
  pdl_wait();
  pdl_trigger();
  int listed = rows, target = side0 ? 0 : c.n_rows;  // rows of the list; the target's among them
  bool packed = c.n_seqs <= kSeqs, fall = !packed && starts_fall(c.row_start, c.n_seqs);
  if (packed) {
    int2 done = make_int2(0, 0);
    for (int base = 0; base < c.n_seqs; base += kRowThreads) {
      const int q = base + (int)threadIdx.x;
      int n = 0;
      if (q < c.n_seqs) {
        const RowSpan sp = row_span(c.row_start, c.n_rows, q);
        n = sp.e - sp.b;
        fall |= __ldg(c.row_start + q) > __ldg(c.row_start + q + 1);
      }
      int2 x = make_int2(n, max(n - 1, 0));  // inclusive prefixes
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int2 o = make_int2(__shfl_up_sync(0xffffffffu, x.x, d), __shfl_up_sync(0xffffffffu, x.y, d));
        if (lane >= d) x.x += o.x, x.y += o.y;
      }
      __syncthreads();
      if (lane == 31) s_sum[threadIdx.x >> 5] = x;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kRowThreads / 32; ++i) {
        const int2 o = s_sum[i];
        if (i < (int)(threadIdx.x >> 5)) x.x += o.x, x.y += o.y;
      }
      if (q < c.n_seqs) s_rows[q + 1] = done.x + x.x, s_drafts[q + 1] = done.y + x.y;
      for (int i = 0; i < kRowThreads / 32; ++i) done.x += s_sum[i].x, done.y += s_sum[i].y;
    }
    if (threadIdx.x == 0) s_rows[0] = s_drafts[0] = 0;
  }
  fall = __syncthreads_or(fall);
  packed = packed && !fall;
  if (blockIdx.x == 0 && threadIdx.x == 0) *c.fall = fall;
  if (packed) {
    target = side0 ? 0 : s_rows[c.n_seqs];
    listed = target + (rows > c.n_rows || side0 ? s_drafts[c.n_seqs] : 0);
  }
  // runs: no more than units, so that each has one and a row no more pieces than units
  const int64_t U = (int64_t)listed * c.n_units, S = min((int64_t)gridDim.x * (kRowThreads / 32), U);
  const int64_t w = (int64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x, u0 = w < S ? U * w / S : 0, u1 = w < S ? U * (w + 1) / S : 0;
  if (u0 >= u1) return;
  const float none = -INFINITY;
  int at = (int)(u0 / c.n_units), q = (int)(u0 - (int64_t)at * c.n_units);  // row of the list, unit of the row
  const T* x = nullptr;
  int lead_in = 0;
  // the last sequence that has a place at or before i (of those that begin there too: the last, which has rows)
  auto search = [&](const int* before, int i) {
    int lo = 0, hi = c.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (before[mid] <= i) lo = mid;
      else hi = mid - 1;
    }
    return lo;
  };
  auto load = [&](uint4 (&v)[kVecs], int unit) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int i = (unit * kUnit + k * 32 + lane) * kV - lead_in;
      if (i >= 0 && i + kV <= c.vocab) {
        v[k] = *reinterpret_cast<const uint4*>(x + i);
      } else {
        T e[kV];
#pragma unroll
        for (int j = 0; j < kV; ++j) e[j] = i + j >= 0 && i + j < c.vocab ? x[i + j] : T(none);
        memcpy(&v[k], e, 16);
      }
    }
  };
  for (int64_t u = u0; u < u1; ++at, q = 0) {  // row by row
    const int end = (int)min((int64_t)c.n_units, q + u1 - u), side = side0 || at >= target, i = at >= target ? at - target : at;
    u += end - q;
    uint4 v[kVecs], next[kVecs];
    int row = i, lo;
    if (packed) {
      lo = search(side ? s_drafts : s_rows, i);
      row = row_span(c.row_start, c.n_rows, lo).b + i - (side ? s_drafts : s_rows)[lo];
    }
    x = side ? static_cast<const T*>(c.draft) + (int64_t)row * c.draft_stride : static_cast<const T*>(c.logits) + (int64_t)row * c.logits_stride;
    lead_in = (int)(((uintptr_t)x & 15) / sizeof(T));
    load(next, q);
    if (!packed) {
      const int2 own = row_owner(c.row_start, c.n_rows, c.n_seqs, row, fall);
      if (own.x < 0 || (side && row + 1 == own.y)) continue;
      lo = own.x;
    }
    const float temp = c.temperature[side] ? c.temperature[side][lo] : 1.f;
    const bool greedy = !(temp > 0.f);
    const float inv_e = inverse(1.4426950408889634f, greedy ? 1.f : bounded(temp));
    float m = none, s = 0.f;
    int first = 0x7FFFFFFF;
    for (int j = q; j < end; ++j) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) v[k] = next[k];
      if (j + 1 < end) load(next, j + 1);
      auto each = [&](auto&& f) {
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
          T e[kV];
          memcpy(e, &v[k], 16);
#pragma unroll
          for (int i = 0; i < kV; ++i) f((float)e[i], (j * kUnit + k * 32 + lane) * kV - lead_in + i);
        }
      };
      const float most = largest<T>(v);  // (a NaN is passed over)
      if (most > m) {
        if (m > none) s *= exp2f((m - most) * inv_e);
        m = most;
        if (greedy) first = 0x7FFFFFFF;
      }
      if (greedy) {
        each([&](float y, int i) {
          if (y == m) first = min(first, i);
        });
      } else if (m == INFINITY) {  // (what came before it, and is finite, weighs nothing)
        each([&](float y, int) { s += y == INFINITY ? 1.f : 0.f; });
      } else if (m > none) {
        // (pairs of floats; where a NaN among them spoils the sum, once more with -inf in its place)
        const uint64_t by = tc::pack2(-m, -m), inv2 = tc::pack2(inv_e, inv_e);
        uint64_t part[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
          const uint32_t word[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
          for (int i = 0; i < kV / 2; ++i) {
            float2 y;
            if constexpr (sizeof(T) == 2) y = Half2<T>::up(word[i]);
            else y = make_float2(__uint_as_float(word[2 * i]), __uint_as_float(word[2 * i + 1]));
            float y0, y1;
            tc::unpack2(mul2(tc::add2(tc::pack2(y.x, y.y), by), inv2), y0, y1);
            part[i & 1] = tc::add2(part[i & 1], tc::pack2(ex2(y0), ex2(y1)));
          }
        }
        float s0, s1;
        tc::unpack2(tc::add2(part[0], part[1]), s0, s1);
        s0 += s1;
        if (s0 != s0) {
          s0 = 0.f;
          each([&](float y, int) { s0 += ex2((fmaxf(y, none) - m) * inv_e); });
        }
        s += s0;
      }
    }
    float all = m;
#pragma unroll
    for (int d = 16; d; d >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, d));
    if (m < all) s = m == none ? 0.f : s * exp2f((m - all) * inv_e), first = 0x7FFFFFFF;
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    first = __reduce_min_sync(0xffffffffu, first);
    if (lane == 0) {
      const int64_t r0 = (int64_t)at * c.n_units;  // the row's first unit; the runs that hold that and its last
      const int64_t w0 = (S * (r0 + 1) - 1) / U, w1 = (S * (r0 + c.n_units) - 1) / U;
      c.pieces[((int64_t)side * c.n_rows + row) * c.n_units + (w - w0)] = {all, s, first, (int)(w1 - w0) + 1};
    }
  }
}

// log p of the entry of index i, -inf where it is not kept
__device__ __forceinline__ float log_p(const Kept& k, float x, int i) {
  x = fmaxf(x, -INFINITY);  // NaN as -inf
  if (!k.any || x == -INFINITY || !(x > k.xc || (x == k.xc && i <= k.ic))) return -INFINITY;
  const float z = z_of(x, k.m, k.t);
  return k.min_p > 0.f && expf(z) < k.min_p ? -INFINITY : z - k.log_sum;
}

// floats in the order of unsigned integers (0: below all)
__device__ __forceinline__ unsigned ordered(float x) {
  const unsigned b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_of(unsigned k) { return k == 0 ? -INFINITY : __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

struct Best {  // the largest key so far, the lowest index where equal
  float v, lp;
  int i;
  __device__ __forceinline__ void take(float ov, float olp, int oi) {
    if (ov > v || (ov == v && oi < i)) v = ov, lp = olp, i = oi;
  }
};

// ---- the drafts and the token that follows
//
// The pass over the row that decides goes through a ring of chunks in shared memory that a warp of its own fills by bulk copies: logits, the
// drafter's where they count, and the noise.  A copy covers whole 16-byte vectors inside its row; what is left of a row's ends, and
// chunks whose copies do not arrive in time, are read where they lie.  Each thread keeps the two largest bounds of its keys: log p + noise
// + log(1 - q / p) by approximate exponentials, with a margin for all roundings; an entry that the drafter may not have kept counts as if it had
// not.  The first chunk's largest key spares most of what follows all but the bound by p alone.  With the largest bound's key worked out, no
// entry whose bound lies below the block's largest key can be the one; a thread whose second does not looks at all its entries.
constexpr int kU = 8, kChunk = kU * kThreads, kMostStages = 8;  // entries of a thread, of a chunk
constexpr int kTogether = kWarps;               // rows that are looked at together, a warp each
template <class T>
struct Stage {
  static constexpr uint32_t kLogits = kChunk * sizeof(T) + 128, kNoise = 2 * kLogits, kBytes = kNoise + kChunk * 4 + 128;
};

// A row's entries e0 .. e1 - 1 in a buffer: entry e at place + (e - e0) * sizeof(E), those from lo to hi - 1 by a copy.
template <class E>
struct Part {
  const E* row;
  uint32_t place;
  int lo, hi;
  // (n: entries of the row)
  __device__ __forceinline__ void set(const E* r, int n, int e0, int e1, uint32_t buffer) {
    row = r;
    const uintptr_t p = (uintptr_t)r, first = (p + 15) & ~uintptr_t(15), last = (uintptr_t)(r + n) & ~uintptr_t(15);  // whole vectors
    const uintptr_t a = (uintptr_t)(r + e0) & ~uintptr_t(15), b = ((uintptr_t)(r + e1) + 15) & ~uintptr_t(15);
    const uintptr_t from = a > first ? a : first, to = b < last ? b : last;
    place = buffer + (uint32_t)((uintptr_t)(r + e0) & 15);
    lo = to > from ? (int)((int64_t)(from - p) / (int)sizeof(E)) : 0;  // (from may lie before e0)
    hi = to > from ? (int)((int64_t)(to - p) / (int)sizeof(E)) : 0;
  }
  __device__ __forceinline__ uint32_t bytes() const { return (uint32_t)(hi - lo) * (uint32_t)sizeof(E); }
  __device__ __forceinline__ void copy(unsigned char* smem, int e0, uint64_t* bar) const {
    if (hi > lo) bulk_g2s(smem + (int)place + (lo - e0) * (int)sizeof(E), row + lo, bytes(), bar);
  }
  __device__ __forceinline__ E at(const unsigned char* smem, int e, int e0, bool there) const {
    return there && e >= lo && e < hi ? *reinterpret_cast<const E*>(smem + place + (uint32_t)(e - e0) * (uint32_t)sizeof(E)) : row[e];
  }
};

template <class T>
__global__ void __launch_bounds__(kThreads + 32, 3) k_verify(const __grid_constant__ VerifyCall c) {
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ Best s_best[kWarps], s_all[2][8];  // of the warps; of the cluster's blocks, by turn
  __shared__ Kept s_kept[2][kTogether];
  __shared__ float s_lp[2][kTogether];
  __shared__ uint64_t s_full[kMostStages], s_free[kMostStages];
  const int stages = c.stages;
  __shared__ volatile int s_lost;
  __shared__ volatile unsigned s_floor;  // the largest key that is known
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), s = blockIdx.x / C;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < kMostStages; ++i) mbar_init(&s_full[i], 1), mbar_init(&s_free[i], kWarps);
    s_lost = 0, s_floor = 0;
    mbar_fence_init();
  }
  // The kernels before this one let it start when what comes before them is done: the call's inputs may be read, what they find not yet.
  if (c.n_rows == 0) pdl_wait();  // (there are none)
  RowSpan sp = row_span(c.row_start, c.n_rows, s);  // (where starts fall it begins later or has no rows: looked at below)
  if (sp.b == sp.e) {
    pdl_wait();
    if (rank == 0 && tid == 0) c.accepted[s] = 0;
    return;
  }
  cl.barrier_arrive();  // (before any block writes to another's shared memory that one has to run: waited for below)
  int drafts = sp.e - sp.b - 1;
  const T* logits = static_cast<const T*>(c.logits);
  const T* draft = static_cast<const T*>(c.draft);
  const int i0 = rank * c.slice, i1 = min(c.vocab, i0 + c.slice);
  const float* noise = c.noise + (int64_t)s * c.noise_stride;
  if (tid == 32 && c.whole[0] && i1 > i0) {  // all of the noise will be asked for: into the L2 cache meanwhile
    const uintptr_t a = ((uintptr_t)(noise + i0) + 15) & ~uintptr_t(15), e = (uintptr_t)(noise + i1) & ~uintptr_t(15);
    if (e > a) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a), "r"((uint32_t)(e - a)) : "memory");
  }
  // the drafts of the first kTogether rows, and their logits
  const int my_side = draft && warp < drafts ? lane >> 4 : 0;
  int my_x = warp < min(kTogether, drafts) ? c.tokens[sp.b + warp + 1] : -1;
  auto logit_of = [&](int side, int row, int x) -> float {
    const T* from = side ? draft + (int64_t)row * c.draft_stride : logits + (int64_t)row * c.logits_stride;
    return x >= 0 && x < c.vocab ? (float)from[x] : -INFINITY;
  };
  float my_v = logit_of(my_side, sp.b + warp, my_x);
  pdl_wait();
  bool fall = s > 0 && *c.fall != 0;
  // what a row keeps, in 16 lanes of the target's and 16 of the drafter's, all lanes together (ordinary loads: read-only ones may be moved
  // ahead of the wait)
  auto kept_of = [&](int side, int row) -> Kept {
    if (!c.whole[0] && !c.whole[1]) return c.kept[(int64_t)side * c.n_rows + row];
    const int sub = lane & 15;
    const Piece* pieces = c.pieces + ((int64_t)side * c.n_rows + row) * c.n_units;
    Piece x = {-INFINITY, 0.f, 0x7FFFFFFF, 0};
    if (c.whole[side] && sub < c.n_units) x = pieces[sub];  // (asked for before their number is known)
    const int n = min(max(__shfl_sync(0xffffffffu, x.n, lane & 16), 0), c.n_units);
    if (sub >= n) x = {-INFINITY, 0.f, 0x7FFFFFFF, 0};
    const float temp = c.temperature[side] ? c.temperature[side][s] : 1.f;
    const bool greedy = !(temp > 0.f);
    const float t = greedy ? 1.f : bounded(temp), inv_e = inverse(1.4426950408889634f, t);
    for (int q = sub + 16; q < n; q += 16) {
      const Piece y = pieces[q];
      const float to = fmaxf(x.m, y.m);
      x.s = to == -INFINITY ? 0.f : x.s * (x.m == to ? 1.f : exp2f((x.m - to) * inv_e)) + y.s * (y.m == to ? 1.f : exp2f((y.m - to) * inv_e));
      x.first = x.m == y.m ? min(x.first, y.first) : x.m > y.m ? x.first : y.first;
      x.m = to;
    }
    __syncwarp();
    float m = x.m;
#pragma unroll
    for (int d = 8; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    float sum = x.m == m ? x.s : x.m == -INFINITY ? 0.f : x.s * exp2f((x.m - m) * inv_e);
    int first = x.m == m ? x.first : 0x7FFFFFFF;
#pragma unroll
    for (int d = 8; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d), first = min(first, __shfl_xor_sync(0xffffffffu, first, d));
    if (!c.whole[side]) return c.kept[(int64_t)side * c.n_rows + row];
    return {m, t, greedy ? m : -INFINITY, 0.f, greedy ? first : 0x7FFFFFFF, greedy ? 0.f : logf(sum), m > -INFINITY, 0};
  };
  // ---- the drafts that are taken: kTogether rows at a time, until one stops
  int stop = drafts, j0 = 0;
  for (;; j0 += kTogether) {
    const int j = j0 + warp;
    if (warp < kTogether && j <= drafts) {
      const int side = draft && j < drafts ? lane >> 4 : 0, row = sp.b + j;
      const int x = j0 == 0 ? my_x : j < drafts ? c.tokens[row + 1] : -1;
      const float v = j0 == 0 ? my_v : logit_of(side, row, x);
      const Kept k = kept_of(side, row);
      if (lane == 16 * side) s_kept[side][warp] = k, s_lp[side][warp] = log_p(k, v, x);
    }
    __syncthreads();
    if (fall) {  // once more with the rows that the sequence has
      fall = false;
      sp = row_span_fallen(c.row_start, c.n_rows, s);
      if (sp.b == sp.e) {
        cl.barrier_wait();
        if (rank == 0 && tid == 0) c.accepted[s] = 0;
        return;
      }
      stop = drafts = sp.e - sp.b - 1;
      my_x = warp < min(kTogether, drafts) ? c.tokens[sp.b + warp + 1] : -1;
      my_v = logit_of(draft && warp < drafts ? lane >> 4 : 0, sp.b + warp, my_x);
      j0 = -kTogether;
      __syncthreads();
      continue;
    }
    if (lane < kTogether && j0 + lane < drafts) {  // (in every warp)
      const float q = draft ? expf(s_lp[1][lane]) : 1.f;
      if (!(c.u[sp.b + j0 + lane] * q < expf(s_lp[0][lane]))) stop = j0 + lane;
    }
    stop = __reduce_min_sync(0xffffffffu, stop);
    if (rank == 0 && tid < kTogether && j0 + tid < stop) {
      const int at = sp.b + j0 + tid;
      c.token[at] = c.tokens[at + 1];
      if (c.logprob) c.logprob[at] = s_lp[0][tid];
    }
    if (stop < j0 + kTogether) break;
    __syncthreads();
  }
  const int row = sp.b + stop, one = stop < drafts && !draft ? c.tokens[row + 1] : -1;
  const bool less = stop < drafts && draft;
  const Kept kp = s_kept[0][stop - j0], kq = less ? s_kept[1][stop - j0] : Kept{};

  // ---- the token after them
  const T* x = logits + (int64_t)row * c.logits_stride;
  const T* y = less ? draft + (int64_t)row * c.draft_stride : x;
  // logits below this are surely not kept (NaN and -inf never are; a bound that is no number bounds nothing)
  const float inv_t = inverse(1.f, kp.t),
              low = fmaxf(fmaxf(kp.xc, kp.min_p > 0.f ? kp.m + kp.t * (logf(kp.min_p) - 1e-3f) - 1e-6f * fabsf(kp.m) : -INFINITY), -FLT_MAX);
  const int chunks = i1 > i0 && kp.any ? (i1 - i0 + kChunk - 1) / kChunk : 0;
  const Best none = {-INFINITY, -INFINITY, 0x7FFFFFFF};
  auto warp_best = [&](Best b) -> Best {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      b.take(__shfl_xor_sync(0xffffffffu, b.v, d), __shfl_xor_sync(0xffffffffu, b.lp, d), __shfl_xor_sync(0xffffffffu, b.i, d));
    return b;
  };
  struct Parts {
    Part<T> x, y;
    Part<float> g;
  };
  auto parts_of = [&](int k, int stage) -> Parts {
    const int e0 = i0 + k * kChunk, e1 = min(i1, e0 + kChunk);
    const uint32_t at = (uint32_t)stage * Stage<T>::kBytes;
    Parts p;
    p.x.set(x, c.vocab, e0, e1, at + 64);
    p.y.set(y, c.vocab, e0, e1, at + Stage<T>::kLogits + 64);
    p.g.set(noise, c.vocab, e0, e1, at + Stage<T>::kNoise + 64);
    if (!less) p.y.lo = p.y.hi = 0;
    return p;
  };
  auto fill = [&](int k, int stage) {  // (one thread)
    const Parts p = parts_of(k, stage);
    const int e0 = i0 + k * kChunk;
    uint64_t* bar = &s_full[stage];
    mbar_arrive_tx(bar, c.hold ? 1 : p.x.bytes() + p.y.bytes() + p.g.bytes());
    if (c.hold) return;
    p.x.copy(ring, e0, bar), p.y.copy(ring, e0, bar), p.g.copy(ring, e0, bar);
  };
  // The bound of a key: z + noise - log_sum with a margin several times that of all roundings, 8e-6 of their sizes and of M / T.
  const float inv_tq = less ? inverse(1.f, kq.t) : 0.f, shift = -kp.m * inv_t - kp.log_sum, shift_q = less ? -kq.m * inv_tq - kq.log_sum : 0.f;
  const float size = 1.f + 2.f * (fabsf(kp.log_sum) + fabsf(kq.log_sum)) + 4.f * (fabsf(kp.m * inv_t) + fabsf(kq.m * inv_tq));
  const bool bounded_keys = size < INFINITY;  // (else every entry is looked at)
  // logits above this are surely kept by the drafter
  const float sure_q = !less || !kq.any      ? INFINITY
                       : kq.min_p > 0.f ? fmaxf(kq.xc, kq.m + kq.t * (logf(kq.min_p) + 1e-3f) + 1e-6f * fabsf(kq.m))
                                        : fmaxf(kq.xc, -FLT_MAX);
  Best b = none;
  auto work_out = [&](int e, bool minus) {
    const float lp = log_p(kp, (float)x[e], e);
    if (lp == -INFINITY || (minus && e == one)) return;
    float key = lp;
    if (minus && less) {
      const float lq = log_p(kq, (float)y[e], e);
      if (lq > -INFINITY) {
        const float rest = expf(lp) - expf(lq);
        if (!(rest > 0.f)) return;
        key = logf(rest);
      }
    }
    b.take(fmaxf(key + noise[e], -INFINITY), lp, e);
  };
  float reach = -INFINITY, reach2 = -INFINITY, floor = -INFINITY;
  int at = -1, filled = 0;  // chunks whose copies were issued
  if (warp == kWarps) {
    // ================= copies
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 1;  // (the first turn of the ring waits for nothing)
      for (int k = 0; k < chunks; ++k) {
        if (k >= stages && !mbar_wait(&s_free[stage], phase, kDefaultWaitNs)) s_lost = 1;
        if (s_lost) break;  // (the stage may have been let go without its copies, which may be on their way)
        fill(k, stage);
        filled = k + 1;
        if (++stage == stages) stage = 0, phase ^= 1;
      }
    }
    __syncwarp();
  } else {
    // chunks that are copied whole: entries from in_lo to in_hi; an entry's place in its chunk's buffers is the same in all chunks
    int in_lo, in_hi;
    {
      Part<T> a;
      Part<float> g;
      a.set(x, c.vocab, 0, c.vocab, 0), g.set(noise, c.vocab, 0, c.vocab, 0);
      in_lo = max(a.lo, g.lo), in_hi = min(i1, min(a.hi, g.hi));
      a.set(y, c.vocab, 0, c.vocab, 0);
      in_lo = max(in_lo, a.lo), in_hi = min(in_hi, a.hi);
    }
    const uint32_t x_off = 64 + (uint32_t)((uintptr_t)(x + i0) & 15), y_off = Stage<T>::kLogits + 64 + (uint32_t)((uintptr_t)(y + i0) & 15),
                   g_off = Stage<T>::kNoise + 64 + (uint32_t)((uintptr_t)(noise + i0) & 15);
    int stage = 0;
    uint32_t phase = 0;
    for (int k = 0; k < chunks; ++k) {
      const int e0 = i0 + k * kChunk, e1 = min(i1, e0 + kChunk);
      bool there = !s_lost;
      if (there && !mbar_wait(&s_full[stage], phase, kDefaultWaitNs)) there = false, s_lost = 1;
      const unsigned char* buf = ring + stage * Stage<T>::kBytes;
      // (without the drafter's part the bound is higher, and nearly always enough)
      const float over = floor - 8e-6f * size;
      auto may_be = [&](float v, float g) -> bool {
        const float a = fmaf(v, inv_t, shift);
        return v >= low && !(fmaf(8e-6f, fabsf(a) + fabsf(g), a + g) < over);
      };
      auto take = [&](int e, float v, float w, float g) {
        const float a = fmaf(v, inv_t, shift), sum = a + g;
        float r = fmaf(8e-6f, fabsf(a) + fabsf(g) + size, sum);
        bool out = e == one;  // or p is surely not above q
        if (less) {
          const float b = fmaf(w, inv_tq, shift_q);
          float ratio, lg;  // q / p; the bound of log(1 - q / p)
          asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ratio) : "f"((b - a) * 1.4426950408889634f));
          const float rest = fmaxf(fmaf(ratio, 8e-6f * (fabsf(a) + fabsf(b) + size), 1.f - ratio), 0.f);
          asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(lg) : "f"(rest));
          out |= bounded_keys && w > sure_q && rest == 0.f;
          r = w > sure_q ? fmaf(lg, 0.6931471805599453f, r) : r;
        }
        r = bounded_keys && r == r ? fmaxf(r, -FLT_MAX) : INFINITY;
        if (!out) {
          const bool more = r > reach || at < 0;
          reach2 = fmaxf(reach2, more ? reach : r);
          if (more) reach = r, at = e;
        }
      };
      if (there && e0 >= in_lo && e0 + kChunk <= in_hi) {
        const T* px = reinterpret_cast<const T*>(buf + x_off) + tid;
        const T* py = reinterpret_cast<const T*>(buf + y_off) + tid;
        const float* pg = reinterpret_cast<const float*>(buf + g_off) + tid;
        uint32_t some = 0;
#pragma unroll
        for (int u = 0; u < kU; ++u) some |= (uint32_t)may_be((float)px[u * kThreads], pg[u * kThreads]) << u;
        for (; some; some &= some - 1) {
          const int u = __ffs(some) - 1;
          take(e0 + u * kThreads + tid, (float)px[u * kThreads], less ? (float)py[u * kThreads] : 0.f, pg[u * kThreads]);
        }
      } else {
        const Parts p = parts_of(k, stage);
        for (int e = e0 + tid; e < e1; e += kThreads) {
          const float v = (float)p.x.at(ring, e, e0, there), g = p.g.at(ring, e, e0, there);
          if (may_be(v, g)) take(e, v, less ? (float)p.y.at(ring, e, e0, there) : 0.f, g);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&s_free[stage]);
      if (++stage == stages) stage = 0, phase ^= 1;
      // The block's largest key of the first chunk (of what warps know when they ask): few of what follows reach it.
      if (k == 0 && chunks > 1) {
        if (at >= 0) work_out(at, true);
        const unsigned mine = __reduce_max_sync(0xffffffffu, ordered(b.v));
        if (lane == 0) atomicMax(const_cast<unsigned*>(&s_floor), mine);
        b = none;
      }
      floor = key_of(s_floor);
    }
  }
  auto block_best = [&]() {  // in every warp
    b = warp_best(b);
    __syncthreads();
    if (lane == 0 && warp < kWarps) s_best[warp] = b;
    __syncthreads();
    b = warp_best(lane < kWarps ? s_best[lane] : none);
  };
  if (at >= 0) work_out(at, true);
  block_best();
  {
    const Best found = b;
    b = none;
    const bool again = reach2 > -INFINITY && !(reach2 < found.v);
    if (__syncthreads_or(again)) {
      if (again)
        for (int e = i0 + tid; e < i1; e += kThreads) work_out(e, true);
      b.take(found.v, found.lp, found.i);
      block_best();
    } else {
      b = found;
    }
  }
  cl.barrier_wait();
  for (int turn = 0;; ++turn) {  // (the second where no entry has p > q: with p alone)
    // the cluster's: every block tells every other
    if (warp == 0 && lane < C) cl.map_shared_rank(&s_all[turn][0], lane)[rank] = b;
    cl.sync();
    b = none;
    for (int q = 0; q < C; ++q) b.take(s_all[turn][q].v, s_all[turn][q].lp, s_all[turn][q].i);
    if (b.i != none.i || turn == 1) break;
    if (warp < kWarps && kp.any)
      for (int e = i0 + tid; e < i1; e += kThreads) work_out(e, false);
    block_best();
  }
  // no copy may be in flight when the block exits (one that was not waited for: its chunk was read without it)
  if (tid == kThreads && s_lost && !c.hold)
    for (int k = max(0, filled - stages); k < filled; ++k) mbar_wait(&s_full[k % stages], (k / stages) & 1, kDefaultWaitNs);

  if (rank != 0) return;
  const bool empty = b.i == none.i;
  for (int j = stop + tid; j <= drafts; j += kThreads + 32) {
    const int at = sp.b + j;
    c.token[at] = j > stop || empty ? -1 : b.i;
    if (c.logprob) c.logprob[at] = j > stop || empty ? -INFINITY : b.lp;
  }
  if (tid == 0) c.accepted[s] = stop;
}

template <class T>
cudaError_t run(VerifyCall c, cudaStream_t s) {
  const int n_seqs = c.n_seqs;
  if (c.n_rows > 0 && (c.whole[0] || (c.draft && c.whole[1]))) {
    c.n_units = (c.vocab + 16 / (int)sizeof(T) - 1 + kUnitEntries<T> - 1) / kUnitEntries<T>;  // (a row may begin anywhere in a vector)
    const int rows = (c.whole[0] + (c.draft && c.whole[1])) * c.n_rows;
    const int64_t most = ((int64_t)rows * c.n_units + kRowThreads / 32 - 1) / (kRowThreads / 32);
    const cudaError_t e = launch_pdl(true, k_rows<T>, dim3((unsigned)(most < 456 ? most : 456)), dim3(kRowThreads), 0, s, c,
                                     c.whole[0] ? 0 : 1, rows);
    if (e != cudaSuccess) return e;
  }
  // Blocks of a sequence: as many as find room on the GPU at once (clusters of up to 8 that lie on some SMs together: 64 sequences of
  // 131072 entries, 6 blocks each 48 us, 4 55, 7 and 8, in two turns, 56 and 53; 128 sequences, 3 83, 4 86), where each has some thousand
  // entries.
  int C = 400 / n_seqs < 8 ? 400 / n_seqs : 8;
  while (C > 1 && c.vocab / C < 4096) --C;
  if (C < 1) C = 1;
  c.slice = (c.vocab + C - 1) / C;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_seqs * (unsigned)C);
  cfg.blockDim = dim3(kThreads + 32);
  // The ring: what shared memory holds of the blocks that an SM gets.
  const int64_t per_sm = ((int64_t)n_seqs * C + 151) / 152, fit = (int64_t)(220 * 1024) / Stage<T>::kBytes / (per_sm < 3 ? per_sm : 3);
  c.stages = fit < kMostStages ? (int)fit : kMostStages;
  cfg.dynamicSmemBytes = c.stages * Stage<T>::kBytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)C, 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaFuncSetAttribute(k_verify<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
  return e == cudaSuccess ? cudaLaunchKernelEx(&cfg, k_verify<T>, c) : e;
}

constexpr uint64_t kFallBytes = 16;  // of the workspace, before the rows' kept

bool bad_word(const void* p) { return ((uintptr_t)p & 3) != 0; }
bool bad_cuts(const mf_cuts_t& c) { return bad_word(c.temperature) || bad_word(c.top_p) || bad_word(c.min_p) || bad_word(c.top_k); }

}  // namespace
}  // namespace mf

using namespace mf;

extern "C" int mf_verify_bytes(int n_seqs, int n_rows, int vocab, uint64_t* out) {
  if (!out || n_seqs < 0 || n_rows < 0 || n_seqs > (1 << 26) || n_rows > (1 << 26) || vocab < 1 || vocab > kMaxVocab) return MF_E_INVAL;
  const uint64_t units = ((uint64_t)vocab + kUnitEntries<float> + 2) / kUnitEntries<float>;
  *out = kFallBytes + (uint64_t)(n_rows > 0 ? n_rows : 1) * 2 * (sizeof(Kept) + units * sizeof(Piece));
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
  auto whole = [](const mf_cuts_t& c) { return !c.top_p && !c.min_p && !c.top_k; };
  const bool whole_p = whole(a->cuts), whole_q = whole(a->draft_cuts);
  int* fall = static_cast<int*>(a->work);
  Kept* kept = reinterpret_cast<Kept*>(static_cast<unsigned char*>(a->work) + kFallBytes);
  const VerifyCall c = {a->logits, a->draft_logits, a->logits_stride, a->draft_stride, a->noise_stride, a->row_start, a->tokens, a->u, a->noise,
                        {a->cuts.temperature, a->draft_cuts.temperature}, a->token, a->accepted, a->logprob, kept,
                        reinterpret_cast<Piece*>(kept + 2 * (int64_t)a->n_rows), fall, {whole_p, whole_q}, a->n_seqs, a->n_rows, a->vocab, 0, 0, 0,
                        sample_hold()};
  cudaError_t e = cudaSuccess;
  if (a->n_rows > 0 && (!whole_p || (a->draft_logits && !whole_q))) {
    const KeptRows rows = {a->logits,  whole_q ? nullptr : a->draft_logits, a->logits_stride, a->draft_stride, a->row_start, a->cuts, a->draft_cuts,
                           kept, fall, a->n_seqs, a->n_rows, a->vocab, a->dtype, !whole_p};
    e = launch_kept(rows, s);
  }
  if (e == cudaSuccess) e = a->dtype == MF_F32 ? run<float>(c, s) : a->dtype == MF_F16 ? run<__half>(c, s) : run<__nv_bfloat16>(c, s);
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_verify");
}

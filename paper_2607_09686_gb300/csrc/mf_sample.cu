// One token from each row of logits: temperature, top-k, top-p, min-p, and an argmax with the caller's Gumbel
// noise.  Contract: mawforge.h.
//
// The kept entries are a prefix of the row in the order (x falling, index rising), so they are described by a value and an
// index: all entries with a larger x, and those equal to it up to that index (and w >= min_p, which needs no order).
//
// A cluster of 1 to 8 blocks has a row, each block a slice of it in shared memory: the logits cross the memory bus
// once, whatever the steps that follow.  Sums and choices of the blocks meet in distributed shared memory.  Steps:
//   1. load (bulk copies), M = max.
//   2. top-k: the k-th largest of the threads' own maxima is a floor of the k-th largest entry, and hardly more than k
//      entries reach it; these go to the leading block, which sorts them and finishes alone: top-p, min-p, argmax.  (Where k
//      is large for that, a histogram of counts over bins of 1/64 in z takes the maxima's place.)
//   3. top-p of what may be many entries: a histogram of masses.  A bin's mass is a sum of integers, w / e^(-bin / 64)
//      in units of 2^-q, so it hangs on no order of additions; the border bin's entries are sorted as above.
//      (Bits: a slice of 2^s entries, s >= 15, leaves q = 31 - s.  A mass is rounded up or down by a number that hangs on
//      the entry's place alone, evenly spread: up as often as its fraction says.  So N equal logits, which to the nearest
//      unit would all be rounded alike, up to N 2^-(q + 1) of an entry too much or too little, err by some sqrt(8 N) 2^-(q + 2)
//      together: 0.05 of an entry for the 2^20 of the largest vocabulary, whose q is 14, as a sum in fp32 does.)
//      What lies so low that it cannot hold the border is summed by ex2 alone.
//   4. a border bin that is too large is cut by bisection over the value's 32-bit key, and equal values by counting them
//      in the order of their index.
//   5. what is kept: sum of w and the largest z + noise, with z as a product; then the entries that come near that one
//      again, with z as the exact quotient.
// What bounds it: with top-k the cluster's barriers and one pass over the slice; else passes of ten to twenty-five
// instructions an entry.  One row of 131072 fp32, T = 0.8, in a graph: top-k of 50 11.2 us, of 1000 20.0 (a longer list to sort),
// top-p of 0.9 21.9.  262144 bf16: one row 11.8, 20.5, 26.1; by top-p 38 rows, as many clusters as the GPU holds at a time, 51 and
// 64 rows 67; 64 rows, each with settings of its own, 54.  Rows by temperature alone have a kernel of their own, in one pass
// (k_sample_plain).
#include <cooperative_groups.h>

#include <atomic>
#include <cfloat>
#include <cmath>

#include "mf_attn.cuh"

namespace cg = cooperative_groups;

namespace mf {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxVocab = 1 << 20;
constexpr int kBins = 2048, kList = 4096, kShort = 512;
constexpr int kCounted = 256;  // entries of a list up to which they are sorted by counting (80: 11.2 us a row against 12.1, 345: 14.3 against 13.8)
constexpr float kBinsPerUnit = 64.f;
constexpr size_t kListAt = (kBins + 4) * 4, kRowAt = kListAt + kList * 8;  // bytes of shared memory before the list, the row
constexpr size_t kResident = 128 * 1024;  // bytes of a slice that are kept in shared memory

struct SampleCall {
  const void* logits;
  const float *noise, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* token;
  float* logprob;
  int64_t logits_stride, noise_stride;
  int vocab;
  int slice;  // entries of a block
  int qbits;  // bits of a mass unit
  int keep;   // the slice's logits lie in shared memory
  int hold;   // (a test's) their copies are not issued
};

// larger floats have larger keys (-0 and +0 compare equal as floats: one key)
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
// The temperature and its inverse are kept where 0 and -inf times the inverse (also in units of log2 e and of bins) are 0 and
// -inf: T from 2^-120 up (below it what differs from M weighs nothing, unless by less than 2^-113), the inverse above 0 for
// T = inf (times the largest number it is below 1e-6).
__device__ __forceinline__ float bounded(float t) { return fmaxf(t, 0x1p-120f); }
__device__ __forceinline__ float inverse(float unit, float t) { return fmaxf(unit / t, 1e-45f); }
// (what is no number, -inf / inf, is -inf)
__device__ __forceinline__ float z_of(float x, float m, float t) { return x == m ? 0.f : fmaxf(__fdiv_rn(x - m, t), -INFINITY); }
// bin of an entry `d` = x - M, the nearest of those at multiples of 1/64 in z; monotonic in d (inv: bins per unit of d).
// Rounded by adding 2^23: conversions share a slow pipe with ex2.
__device__ __forceinline__ float bin_at(float d, float inv) {
  return fminf(-d * inv, (float)(kBins - 1)) + 8388608.f;
}
__device__ __forceinline__ int bin_of(float d, float inv) { return (int)(__float_as_uint(bin_at(d, inv)) & (kBins - 1)); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct Best {  // the largest z + noise so far, the lowest index where equal
  float v, z;
  int i;
  __device__ __forceinline__ void take(float ov, float oz, int oi) {
    if (ov > v || (ov == v && oi < i)) v = ov, z = oz, i = oi;
  }
};

struct Shared {
  float d[kWarps];       // sums of the warps
  float pub[2];          // sums of the block, which the cluster reads
  float f[kWarps], mx;   // maxima of the warps, of the block
  float top[2];          // the block's largest key
  int n[kWarps + 1];
  Best best[kWarps + 1];
  // the leading block's answers
  float above, goal;
  int bin, count;             // border bin (-1: nothing is cut), entries down to it
  unsigned listed, kmin, kmax;  // entries put on the list, and their keys' range
  unsigned place;               // of this block's entries on the leading block's list
  uint32_t key;
  int index;
  int here;
  uint64_t bar;  // the bulk copies' barrier
};

template <class T>
__global__ void __launch_bounds__(kThreads, 2) k_sample(SampleCall c) {
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ Shared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), r = blockIdx.x / C;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t* hist = reinterpret_cast<uint32_t*>(dyn);
  unsigned long long* list = reinterpret_cast<unsigned long long*>(dyn + kListAt);
  const int base = rank * c.slice, n = max(0, min(c.slice, c.vocab - base));
  const T* row = static_cast<const T*>(c.logits) + (int64_t)r * c.logits_stride + base;
  const float* noise = c.noise + (int64_t)r * c.noise_stride + base;
  Shared* lead = cl.map_shared_rank(&sh, 0);
  unsigned long long* lead_list = cl.map_shared_rank(list, 0);

  pdl_wait();
  // ---- 1. the slice into shared memory, at the same place modulo 16 bytes: whole vectors by bulk copies, the ends by hand
  auto up = [](T v) -> float { return fmaxf((float)v, -INFINITY); };  // NaN as -inf
  const T* src = row;
  // A copy that does not arrive in time costs time, no answer: the slice is read where it lies then.
  bool keep = c.keep, lost = false;
  if (keep) {
    T* x0 = reinterpret_cast<T*>(dyn + kRowAt + ((uintptr_t)row & 15));
    const int head = min(n, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T)),
              body = (n - head) * (int)sizeof(T) / 16 * 16 / (int)sizeof(T);
    if (tid == 0) {
      mbar_init(&sh.bar, 1);
      mbar_fence_init();
      const uint32_t bytes = (uint32_t)(body * sizeof(T));
      mbar_arrive_tx(&sh.bar, bytes);
      // pieces of 32 KiB: several copies in flight
      for (uint32_t o = 0; o < bytes && !c.hold; o += 32768)
        bulk_g2s(reinterpret_cast<unsigned char*>(x0 + head) + o, reinterpret_cast<const unsigned char*>(row + head) + o, min(bytes - o, 32768u),
                 &sh.bar);
    }
    for (int i = tid; i < n - body; i += kThreads) {
      const int at = i < head ? i : body + i;
      x0[at] = row[at];
    }
    __syncthreads();
    lost = __syncthreads_or(!mbar_wait(&sh.bar, 0, kDefaultWaitNs));
    keep = !lost;
    if (keep) src = x0;
  }
  auto leave = [&]() {  // no copy may be in flight when the block exits
    if (lost) mbar_wait(&sh.bar, 0, kDefaultWaitNs);
  };
  // every thread's entries, f(index, logit, vector): whole vectors of the slice where it lies in shared memory
  auto for_each = [&](auto&& f) {
    if (keep) {
      constexpr int kV = 16 / sizeof(T);
      const int lead_in = (int)(((uintptr_t)src & 15) / sizeof(T)), total = lead_in + n;
      for (int v = tid; v * kV < total; v += kThreads) {
        const uint4 q = reinterpret_cast<const uint4*>(src - lead_in)[v];
        const T* e = reinterpret_cast<const T*>(&q);
        const int i0 = v * kV - lead_in;
        if (i0 >= 0 && i0 + kV <= n) {
#pragma unroll
          for (int u = 0; u < kV; ++u) f(i0 + u, up(e[u]), v);
        } else {
          for (int i = max(i0, 0); i < min(i0 + kV, n); ++i) f(i, up(src[i]), v);
        }
      }
    } else {
      for (int i = tid; i < n; i += kThreads) f(i, up(row[i]), i);
    }
  };
  // Those from lo to hi (a bound that is no number bounds nothing), where they are few: of 64 entries at a time a thread's are
  // picked out first, then taken four by four, with what get() loads for them under way together.
  auto for_some = [&](float lo, float hi, auto&& get, auto&& f) {
    auto within = [&](float x) { return !(x < lo) && !(x > hi); };
    if (keep) {
      constexpr int kV = 16 / sizeof(T), kGroup = 64 / kV;
      const int lead_in = (int)(((uintptr_t)src & 15) / sizeof(T)), total = lead_in + n;
      const T* from = src - lead_in;
      for (int v0 = tid; v0 * kV < total; v0 += kGroup * kThreads) {
        uint32_t some[2] = {0, 0};
#pragma unroll
        for (int g = 0; g < kGroup; ++g) {
          const int v = v0 + g * kThreads;
          if (v * kV >= total) break;
          const uint4 q = reinterpret_cast<const uint4*>(from)[v];
          const T* e = reinterpret_cast<const T*>(&q);
#pragma unroll
          for (int u = 0; u < kV; ++u) some[g * kV / 32] |= (uint32_t)within((float)e[u]) << (g * kV % 32 + u);
        }
        unsigned long long left = (unsigned long long)some[1] << 32 | some[0];
        while (left) {
          int at[4];
          float x[4], y[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int bit = __ffsll((long long)left) - 1;
            at[u] = left ? (v0 + (bit / kV) * kThreads) * kV + bit % kV - lead_in : -1;
            left &= left - 1;
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            if (at[u] >= n) at[u] = -1;
            x[u] = at[u] >= 0 ? up(src[at[u]]) : 0.f;
            y[u] = at[u] >= 0 ? get(at[u]) : 0.f;
          }
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (at[u] >= 0) f(at[u], x[u], y[u]);
        }
      }
    } else {
      for (int i = tid; i < n; i += kThreads) {
        const float x = up(row[i]);
        if (within(x)) f(i, x, get(i));
      }
    }
  };
  auto get_none = [](int) { return 0.f; };
  float mx = -INFINITY;
  for_each([&](int, float x, int) { mx = fmaxf(mx, x); });
  const float own_max = mx;
#pragma unroll
  for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
  if (lane == 0) sh.f[warp] = mx;
  if (tid == 0) sh.listed = 0, sh.kmin = 0xFFFFFFFFu, sh.kmax = 0;
  __syncthreads();
  auto warp_max = [&](float v) -> float {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
  };
  auto warp_sum = [&](float v) -> float {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
  };
  if (warp == 0) {
    mx = warp_max(lane < kWarps ? sh.f[lane] : -INFINITY);
    if (lane == 0) sh.mx = mx;
  }
  cl.sync();
  const float theirs = lane < C ? cl.map_shared_rank(&sh, lane)->mx : -INFINITY;
  const float m = warp_max(theirs);

  const float temp = c.temperature ? c.temperature[r] : 1.f;
  const bool greedy = !(temp > 0.f);
  const float t = greedy ? 1.f : bounded(temp);
  const int top_k = c.top_k && !greedy ? c.top_k[r] : 0;
  const float top_p = c.top_p && !greedy ? c.top_p[r] : 1.f;
  const float min_p = c.min_p && !greedy ? fminf(fmaxf(c.min_p[r], 0.f), 1.f) : 0.f;
  const float inv = inverse(kBinsPerUnit, t);
  float xc = -INFINITY;  // kept: larger entries, and equal ones up to index ic
  int ic = -1;
  auto kept = [&](float x, int i) { return x > xc || (x == xc && i <= ic); };

  // a sum and a maximum over the cluster, the same in every thread and whatever the order of execution
  int flip = 0;
  auto cluster_sum = [&](float v, float& top) -> float {
    v = warp_sum(v), top = warp_max(top);
    __syncthreads();
    if (lane == 0) sh.d[warp] = v, sh.f[warp] = top;
    __syncthreads();
    if (warp == 0) {
      v = warp_sum(lane < kWarps ? sh.d[lane] : 0.f), top = warp_max(lane < kWarps ? sh.f[lane] : -INFINITY);
      if (lane == 0) sh.pub[flip] = v, sh.top[flip] = top;
    }
    cl.sync();
    const Shared* o = cl.map_shared_rank(&sh, lane < C ? lane : 0);
    v = warp_sum(lane < C ? o->pub[flip] : 0.f), top = warp_max(o->top[flip]);
    flip ^= 1;
    return v;
  };
  // exclusive prefix over the block's threads, and the sum
  auto block_scan = [&](float v, float& all) -> float {
    float x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const float o = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += o;
    }
    __syncthreads();
    if (lane == 31) sh.d[warp] = x;
    __syncthreads();
    float before = 0;
    all = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += sh.d[w];
      all += sh.d[w];
    }
    return before + x - v;
  };
  // The last bin that is not empty and begins below `goal`, of bins tid * 4 + u of v[u], this thread's first beginning at `at` (-1:
  // none), in every thread; its owner gets its span.  A border that is sought so is found whatever the rounding: the ends of a
  // thread's bins and the beginning of the next thread's are different sums, with gaps and overlaps of a last bit, in which no
  // bin, or two, would hold the goal.  (sh.here is -1 before.)
  auto last_below = [&](const float (&v)[4], float at, float goal, bool& own, float2& span) -> int {
    int mine = -1;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (v[u] > 0.f && at < goal) mine = tid * 4 + u, span = make_float2(at, at + v[u]);
      at += v[u];
    }
    const int most = __reduce_max_sync(0xffffffffu, mine);
    if (lane == 0) atomicMax(&sh.here, most);
    __syncthreads();
    own = mine >= 0 && mine == sh.here;
    return sh.here;
  };
  // Counts (or masses, in units of 2^-qbits) of the kept entries by bin, or counts of the threads' maxima; the leading block finds
  // the first bin down to which they reach `want` (mass: want * their total), and tells all blocks: bin, above, goal, and for
  // counts count.  Counts are whole numbers below 2^24: exact in fp32.
  // Masses: entries of less than (1 - want) / vocab of the largest one's cannot hold the border, whatever they are together;
  // theirs is summed in units of 2^-30 (hist[kBins]) and joins the total alone.
  enum { kCounts, kMasses, kMaxima };
  auto find_bin = [&](int what, float want) {
    const bool mass = what == kMasses;
    for (int i = tid; i <= kBins; i += kThreads) hist[i] = 0;
    __syncthreads();
    const float unit = (float)(1 << c.qbits);
    if (what == kMaxima) {
      if (own_max > -INFINITY) atomicAdd(hist + bin_of(own_max == m ? 0.f : own_max - m, inv), 1u);
    } else if (mass) {
      const bool all = xc == -INFINITY;
      const float low = all ? m + t * (logf((1.f - want) / (float)c.vocab) - 0.01f) - 1e-6f * fabsf(m) : xc;
      const float inv_e = inverse(1.4426950408889634f, t);
      const uint32_t seed = (uint32_t)rank * 0x85EBCA6Bu;
      float rest = 0.f;
      for_each([&](int i, float x, int v) {  // (without branches: both sides cost less than their divergence)
        const bool below = x < low;
        const float d = x == m ? 0.f : x - m, at = bin_at(d, inv);
        // (w against that at the bin's middle: near 1)
        const float w = ex2(fmaf(d, inv, at - 8388608.f) * (1.4426950408889634f / kBinsPerUnit)), tail = ex2(d * inv_e);
        rest += below && all ? tail : 0.f;
        // rounded down after a number of [0, 1) is added, the vector's own (multiples of the golden ratio, their fractions):
        // whole masses stay what they are
        const float part = __uint_as_float(0x3F800000u | ((uint32_t)v * 0x9E3779B9u + seed) >> 9) - 1.f;
        if (!below && (all || kept(x, base + i)))
          atomicAdd(hist + (__float_as_uint(at) & (kBins - 1)), __float_as_uint(__fadd_rd(__fmaf_rd(w, unit, part), 8388608.f)) & 0x7FFFFFu);
      });
      rest = warp_sum(rest);
      if (lane == 0 && rest > 0.f) atomicAdd(hist + kBins, (uint32_t)(fminf(rest, 1.f) * 1073741824.f / (float)(kWarps) + 0.5f));
    } else {
      for_each([&](int i, float x, int) {
        if (kept(x, base + i)) atomicAdd(hist + bin_of(x == m ? 0.f : x - m, inv), 1u);
      });
    }
    cl.sync();
    if (rank == 0) {
      constexpr int kPer = kBins / kThreads;
      float v[kPer], sum = 0, total;
      static_assert(kPer == 4, "a vector of bins a thread");
      uint4 h[8];
#pragma unroll
      for (int q = 0; q < 8; ++q)
        h[q] = q < C ? reinterpret_cast<const uint4*>(cl.map_shared_rank(hist, q))[tid] : make_uint4(0, 0, 0, 0);
      const float rest = mass ? warp_sum(lane < C ? (float)cl.map_shared_rank(hist, lane)[kBins] : 0.f) * ((float)kWarps / 1073741824.f) : 0.f;
      unsigned long long s[kPer] = {0, 0, 0, 0};
#pragma unroll
      for (int q = 0; q < 8; ++q) s[0] += h[q].x, s[1] += h[q].y, s[2] += h[q].z, s[3] += h[q].w;
#pragma unroll
      for (int u = 0; u < kPer; ++u) {
        const int b = tid * kPer + u;
        v[u] = mass ? (float)s[u] * expf(-(float)b * (1.f / kBinsPerUnit)) : (float)s[u];
        sum += v[u];
      }
      if (tid == 0) sh.bin = sh.here = -1;
      const float at = block_scan(sum, total), goal = mass ? want * (total + rest * unit) : want;
      bool own;
      float2 span;
      const int bin = last_below(v, at, goal, own, span);
      // (counts: fewer entries than are wanted cut nothing; a part of the mass is always reached)
      if (own && (mass || total >= want)) sh.bin = bin, sh.above = span.x, sh.count = (int)span.y;
      if (tid == 0) sh.goal = goal;
      __syncthreads();
      if (warp == 0 && lane > 0 && lane < C) {
        Shared* o = cl.map_shared_rank(&sh, lane);
        o->bin = sh.bin, o->above = sh.above, o->count = sh.count, o->goal = sh.goal;
      }
    }
    cl.sync();
  };
  // The entries from `lo` to `hi` that are wanted onto the leading block's list (as many as there is room for; all are
  // counted), in no certain order: each block collects its own first, so that whole runs and one counter cross to the leading
  // block.  kmin, kmax: the range of their keys.
  auto gather = [&](float lo, float hi, auto&& wanted) {
    if (rank != 0 && tid == 0) sh.listed = 0, sh.kmin = 0xFFFFFFFFu, sh.kmax = 0;
    __syncthreads();
    if (!(own_max < lo)) {
      unsigned kmin = 0xFFFFFFFFu, kmax = 0;
      for_some(lo, hi, get_none, [&](int i, float x, float) {
        if (!wanted(x, base + i)) return;
        const uint32_t k = order_key(x);
        const unsigned at = atomicAdd(&sh.listed, 1u);
        if (at < kList) list[at] = (unsigned long long)k << 32 | (0xFFFFFFFFu - (unsigned)(base + i));
        kmin = min(kmin, k), kmax = max(kmax, k);
      });
      if (kmax) atomicMin(&sh.kmin, kmin), atomicMax(&sh.kmax, kmax);
    }
    __syncthreads();
    const unsigned own = sh.listed;
    if (rank != 0 && own) {
      if (tid == 0) {
        sh.place = atomicAdd(&lead->listed, own);
        atomicMin(&lead->kmin, sh.kmin), atomicMax(&lead->kmax, sh.kmax);
      }
      __syncthreads();
      for (unsigned i = tid; i < own && sh.place + i < kList; i += kThreads) lead_list[sh.place + i] = list[i];
    }
    cl.sync();
  };
  // The leading block's list sorted: keys falling, indices rising.  A short one: each thread counts those before its entry (no
  // two are equal).  Else bitonic; entries up to 64 apart meet in the registers of a warp that has 128, without barriers.
  auto sort_list = [&](int len) {
    __syncthreads();
    if (len <= kCounted) {
      if (tid == 0) list[len] = 0;
      __syncthreads();
      const unsigned long long e = tid < len ? list[tid] : 0;
      int before = 0;
      if (warp * 32 < len) {
#pragma unroll 4
        for (int i = 0; i < len; i += 2) {
          const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(list + i);
          before += (int)(o.x > e) + (int)(o.y > e);
        }
      }
      __syncthreads();
      if (tid < len) list[before] = e;
      __syncthreads();
      return;
    }
    int p2 = 2 * kCounted;
    while (p2 < len) p2 <<= 1;
    for (int i = len + tid; i < p2; i += kThreads) list[i] = 0;
    __syncthreads();
    for (int k = 128; k <= p2; k <<= 1) {
      for (int j = k >> 1; j > 64; j >>= 1) {
        for (int i = tid; i < p2 / 2; i += kThreads) {
          const int a = 2 * i - (i & (j - 1)), b = a + j;
          const unsigned long long x = list[a], y = list[b];
          if ((x < y) == ((a & k) == 0)) list[a] = y, list[b] = x;
        }
        __syncthreads();
      }
      for (int at = warp * 128 + lane * 4; at < p2; at += kWarps * 128) {  // four neighbours a lane
        ulonglong2* mine = reinterpret_cast<ulonglong2*>(list + at);
        const ulonglong2 lo = mine[0], hi = mine[1];
        unsigned long long e[4] = {lo.x, lo.y, hi.x, hi.y};
        auto meet = [&](int u, int w, bool fall) {
          const unsigned long long x = e[u], y = e[w];
          if ((x < y) == fall) e[u] = y, e[w] = x;
        };
        if (k == 128) meet(0, 1, true), meet(2, 3, false);
        for (int k2 = k == 128 ? 4 : k; k2 <= k; k2 <<= 1) {
          const bool fall = (at & k2) == 0;
          for (int j = min(k2 >> 1, 64); j > 2; j >>= 1) {
            const bool larger = fall == ((at & j) == 0);  // this lane keeps the larger ones
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const unsigned long long o = __shfl_xor_sync(0xffffffffu, e[u], j >> 2);
              if ((e[u] < o) == larger) e[u] = o;
            }
          }
          meet(0, 2, fall), meet(1, 3, fall), meet(0, 1, fall), meet(2, 3, fall);
        }
        mine[0] = make_ulonglong2(e[0], e[1]), mine[1] = make_ulonglong2(e[2], e[3]);
      }
      __syncthreads();
    }
  };
  auto clear_list = [&]() {  // (after which a barrier of the cluster comes before the next gather: find_bin's)
    if (rank == 0 && tid == 0) sh.listed = 0, sh.kmin = 0xFFFFFFFFu, sh.kmax = 0;
  };
  auto warp_best = [&](Best b) -> Best {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      b.take(__shfl_xor_sync(0xffffffffu, b.v, d), __shfl_xor_sync(0xffffffffu, b.z, d), __shfl_xor_sync(0xffffffffu, b.i, d));
    return b;
  };
  const Best none = {-INFINITY, 0.f, 0x7FFFFFFF};
  auto block_best = [&](Best b) -> Best {  // (in warp 0)
    b = warp_best(b);
    __syncthreads();
    if (lane == 0) sh.best[warp] = b;
    __syncthreads();
    return warp == 0 ? warp_best(lane < kWarps ? sh.best[lane] : none) : none;
  };
  auto answer = [&](const Best& b, float sum) {
    c.token[r] = b.i;
    if (c.logprob) c.logprob[r] = b.z - logf(sum);
  };
  // the border among entries too many for the list, keys lo .. hi: the largest key down to which value() reaches want,
  // then the index of the last of its equals that is kept
  auto cut_by_key = [&](bool mass, double want, uint32_t lo, uint32_t hi) {
    auto value = [&](uint32_t from) -> double {  // of the kept entries with keys >= from
      float part = 0.f;
      int cnt = 0;
      for (int i = tid; i < n; i += kThreads) {
        const float x = up(src[i]);
        const uint32_t k = order_key(x);
        if (k < from || !kept(x, base + i)) continue;
        if (mass) part += expf(z_of(x, m, t));
        else ++cnt;
      }
      float unused = 0.f;
      return cluster_sum(mass ? part : (float)cnt, unused);
    };
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo + 1) / 2;
      if (value(mid) >= want) lo = mid;
      else hi = mid - 1;
    }
    const double over = value(lo + 1);
    const double left = mass ? ceil((want - over) / (double)expf(z_of(key_value(lo), m, t))) : want - over;
    const int ties = left < 1 ? 1 : left > 2e9 ? 2000000000 : (int)left;
    // the ties-th of the equal ones in the order of their index: warp w has entries w * seg .. of the slice
    const int seg = ((n + kWarps - 1) / kWarps + 31) & ~31, s0 = min(n, warp * seg), s1 = min(n, s0 + seg);
    int mine = 0;
    for (int i = s0 + lane; i < s1; i += 32) {
      const float x = up(src[i]);
      mine += order_key(x) == lo && kept(x, base + i);
    }
    mine = __reduce_add_sync(0xffffffffu, mine);
    __syncthreads();
    if (lane == 0) sh.n[warp] = mine;
    if (tid == 0) sh.here = -1;
    __syncthreads();
    if (tid == 0) {
      int s = 0;
      for (int w = 0; w < kWarps; ++w) s += sh.n[w];
      sh.n[kWarps] = s;
    }
    cl.sync();
    int before = 0, all = 0;
    for (int b = 0; b < C; ++b) {
      const int v = cl.map_shared_rank(&sh, b)->n[kWarps];
      if (b < rank) before += v;
      all += v;
    }
    for (int w = 0; w < warp; ++w) before += sh.n[w];
    const int nth = min(ties, all);
    if (mine && before < nth && nth <= before + mine) {
      for (int i0 = s0; i0 < s1; i0 += 32) {
        const int i = i0 + lane;
        bool in = false;
        if (i < s1) {
          const float x = up(src[i]);
          in = order_key(x) == lo && kept(x, base + i);
        }
        const unsigned who = __ballot_sync(0xffffffffu, in);
        if (nth <= before + __popc(who)) {
          if (lane == 0) {
            unsigned left_of = who;
            for (int q = 1; q < nth - before; ++q) left_of &= left_of - 1;
            lead->index = base + i0 + __ffs(left_of) - 1;
          }
          break;
        }
        before += __popc(who);
      }
    }
    cl.sync();
    xc = key_value(lo);
    ic = lead->index;
    cl.sync();
  };

  if (m == -INFINITY) {
    if (rank == 0 && tid == 0) {
      c.token[r] = -1;
      if (c.logprob) c.logprob[r] = -INFINITY;
    }
    leave();
    cl.sync();
    return;
  }
  if (!greedy && top_k > 0 && top_k < c.vocab) {
    // ---- 2. top-k
    // The bin down to which top_k of the threads' maxima reach holds top_k entries at least; if the list has no room for all
    // down to it, the bin that top_k entries reach.
    bool few = false;
    if (top_k <= kThreads * C / 2) {
      find_bin(kMaxima, (float)top_k);
      if (sh.bin >= 0) {
        // the bin's lower end, a little lower for the rounding (more entries than needed do no harm)
        const float low = m - ((float)sh.bin + 0.5f) * (1.f / inv) * 1.00001f;
        gather(sh.bin < kBins - 1 && low > -INFINITY ? low : -FLT_MAX, INFINITY, [](float x, int) { return x > -INFINITY; });
        few = lead->listed <= kList;
        if (!few) {
          cl.sync();
          clear_list();
        }
      }
    }
    if (!few) find_bin(kCounts, (float)top_k);
    const int bin = sh.bin, above = bin < 0 ? 0 : (int)sh.above;
    if (bin >= 0) {
      if (!few) {
        few = sh.count <= kList;
        const int first = few ? 0 : bin;
        gather(-INFINITY, INFINITY, [&](float x, int i) {
          const int b = bin_of(x == m ? 0.f : x - m, inv);
          return b >= first && b <= bin && kept(x, i);
        });
      }
      if (few) {
        // the other blocks are done: nothing of theirs is read any more, and the leading block waits for their last look at it
        cl.barrier_arrive();
        if (rank == 0) {
          const int count = (int)sh.listed;
          sort_list(count);
          constexpr int kPer = kList / kThreads;
          const int len = min(top_k, count), per = (len + kThreads - 1) / kThreads;
          float w[kPer], z[kPer];
          float sum = 0, all;
#pragma unroll
          for (int u = 0; u < kPer; ++u) {
            const int i = tid * per + u;
            w[u] = z[u] = 0.f;
            if (u < per && i < len) z[u] = z_of(key_value((uint32_t)(list[i] >> 32)), m, t), w[u] = expf(z[u]);
            sum += w[u];
          }
          if (tid == 0) sh.here = 0;
          float at = block_scan(sum, all);
          int last = len - 1;  // kept by top-p
          if (top_p < 1.f) {
            const float want = top_p * all;
            int mine = 0;
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
              if (u < per && tid * per + u < len && at < want) mine = tid * per + u;
              at += w[u];
            }
            mine = __reduce_max_sync(0xffffffffu, mine);
            if (lane == 0) atomicMax(&sh.here, mine);
            __syncthreads();
            last = sh.here;
          }
          Best b = none;
          sum = 0;
#pragma unroll
          for (int u = 0; u < kPer; ++u) {
            const int i = tid * per + u;
            if (u < per && i <= last && (i == 0 || w[u] >= min_p)) {
              const int idx = (int)(0xFFFFFFFFu - (uint32_t)list[i]);
              const float g = noise[idx];
              b.take(g == g ? z[u] + g : -INFINITY, z[u], idx);
              sum += w[u];
            }
          }
          block_scan(sum, all);
          b = block_best(b);
          if (tid == 0) answer(b, all);
        }
        leave();
        cl.barrier_wait();
        return;
      }
      if (lead->listed <= kList) {
        if (rank == 0) {
          sort_list((int)lead->listed);
          if (tid == 0) {
            const unsigned long long e = list[top_k - above - 1];
            sh.key = (uint32_t)(e >> 32), sh.index = (int)(0xFFFFFFFFu - (uint32_t)e);
          }
        }
        cl.sync();
        xc = key_value(lead->key), ic = lead->index;
      } else {
        cut_by_key(false, (double)top_k, lead->kmin, lead->kmax);
      }
      cl.sync();
      clear_list();
    }
  }
  if (!greedy && tid == 0 && n > 0) {  // much of the noise will be asked for: into the L2 cache meanwhile
    const uintptr_t a = ((uintptr_t)noise + 15) & ~uintptr_t(15), e = (uintptr_t)(noise + n) & ~uintptr_t(15);
    if (e > a) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a), "r"((uint32_t)(e - a)) : "memory");
  }
  if (!greedy && top_p < 1.f) {
    // ---- 3. top-p
    if (!(top_p > 0.f)) {  // the first entry alone: the lowest of the largest
      xc = m;
      ic = -1;
    } else {
      find_bin(kMasses, top_p);
      const int bin = sh.bin;
      if (bin >= 0) {
        // the bin's ends, somewhat farther apart for the rounding
        const float wide = 1e-5f * (float)(bin + 1) / inv + 1e-6f * fabsf(m);
        gather(bin < kBins - 1 ? m - ((float)bin + 0.5f) / inv - wide : -INFINITY, m - ((float)bin - 0.5f) / inv + wide,
               [&](float x, int i) { return bin_of(x == m ? 0.f : x - m, inv) == bin && kept(x, i); });
        const unsigned len = lead->listed;
        if (len <= kList) {
          if (rank == 0) {
            // In units of an entry's w: the list's entries are cut down to those around the border, by histograms of masses over
            // the range of their keys, then (equal keys) over that of their indices, until a short list is left to sort.
            const float unit = 1.f / (float)(1 << c.qbits), want = sh.goal * unit;
            float above = sh.above * unit;
            uint32_t lo = sh.kmin, hi = sh.kmax;      // keys of the entries around the border
            uint32_t i_lo = 0, i_hi = (uint32_t)c.vocab - 1;  // and their indices, once the keys are equal
            int left = (int)len;
            const float w_top = expf(z_of(key_value(hi), m, t));
            auto around = [&](unsigned long long e) {
              const uint32_t k = (uint32_t)(e >> 32), i = 0xFFFFFFFFu - (uint32_t)e;
              return k >= lo && k <= hi && i >= i_lo && i <= i_hi;
            };
            while (left > kShort && (lo < hi || i_lo < i_hi)) {
              const bool by_key = lo < hi;
              const uint32_t range = by_key ? hi - lo : i_hi - i_lo;
              const int shift = max(0, 32 - __clz(range) - 11);  // 2048 bins
              for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
              __syncthreads();
              for (int i = tid; i < (int)len; i += kThreads) {
                const unsigned long long e = list[i];
                if (!around(e)) continue;
                const uint32_t k = (uint32_t)(e >> 32), bin = (by_key ? hi - k : 0xFFFFFFFFu - (uint32_t)e - i_lo) >> shift;
                // 19 bits of w against the largest of the list (of 2^12 entries), the low bit kept for "not empty"
                atomicAdd(hist + bin, (uint32_t)(expf(z_of(key_value(k), m, t)) / w_top * 524287.f + 0.5f));
              }
              __syncthreads();
              float v[4], sum = 0, all;
#pragma unroll
              for (int u = 0; u < 4; ++u) sum += v[u] = (float)hist[tid * 4 + u] * (w_top / 524287.f);
              if (tid == 0) sh.here = -1;
              const float at = above + block_scan(sum, all);
              bool own;
              float2 span;
              const int bin = last_below(v, at, want, own, span);
              if (bin < 0) break;  // (the sums' last bits: the border is the range's beginning; sorted below as it is)
              if (own) sh.above = span.x;
              __syncthreads();
              above = sh.above;
              if (by_key) {
                const uint32_t top = hi - ((uint32_t)bin << shift), step = (1u << shift) - 1;
                hi = top, lo = top - lo > step ? top - step : lo;
              } else {
                const uint32_t first = i_lo + ((uint32_t)bin << shift), step = (1u << shift) - 1;
                i_lo = first, i_hi = i_hi - first > step ? first + step : i_hi;
              }
              int cnt = 0;
              for (int i = tid; i < (int)len; i += kThreads) cnt += around(list[i]);
              block_scan((float)cnt, all);
              left = (int)all;
            }
            // those around the border to the list's front, sorted
            unsigned long long mine[kList / kThreads];
            int cnt = 0;
#pragma unroll
            for (int u = 0; u < kList / kThreads; ++u) {
              const int i = tid + u * kThreads;
              mine[u] = i < (int)len && around(list[i]) ? list[i] : 0;
              cnt += mine[u] != 0;
            }
            float all;
            int to = (int)block_scan((float)cnt, all);
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kList / kThreads; ++u)
              if (mine[u]) list[to++] = mine[u];
            left = (int)all;
            __syncthreads();
            sort_list(left);
            constexpr int kPer = kList / kThreads;
            const int per = (left + kThreads - 1) / kThreads;
            float w[kPer], sum = 0;
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
              const int i = tid * per + u;
              w[u] = u < per && i < left ? expf(z_of(key_value((uint32_t)(list[i] >> 32)), m, t)) : 0.f;
              sum += w[u];
            }
            float at = above + block_scan(sum, all);
            if (tid == 0) sh.here = -1;
            __syncthreads();
            int lastk = -1;
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
              const int i = tid * per + u;
              if (u < per && i < left && at < want) lastk = i;
              at += w[u];
            }
            if (lastk >= 0) atomicMax(&sh.here, lastk);
            __syncthreads();
            if (tid == 0) {
              const unsigned long long e = list[max(sh.here, 0)];
              sh.key = (uint32_t)(e >> 32), sh.index = (int)(0xFFFFFFFFu - (uint32_t)e);
            }
          }
          cl.sync();
          xc = key_value(lead->key), ic = lead->index;
        } else {
          // the bin's share of the mass, with sums in floating point throughout
          float part = 0.f;
          for (int i = tid; i < n; i += kThreads) {
            const float x = up(src[i]);
            if (kept(x, base + i)) part += expf(z_of(x, m, t));
          }
          float unused = 0.f;
          const double total = cluster_sum(part, unused);
          cut_by_key(true, (double)top_p * total, lead->kmin, lead->kmax);
        }
      }
    }
  }
  // ---- 5. what is kept
  const bool first_only = greedy || top_p <= 0.f;
  Best b = none;
  float sum = 1.f;
  if (first_only) {
    for_each([&](int i, float x, int) {
      if (x == m) b.take(0.f, 0.f, base + i);
    });
  } else {
    const float inv_t = inverse(1.f, t), inv_e = inv_t * 1.4426950408889634f;
    // z as a product and w of an entry, and whether it is in: w >= min_p is decided on the exact w where the other comes near.
    // (w is off by the rounding of z log2(e), by a few 2^-24 |z|, and by ex2's 2^-22.)
    const float eps = 4e-7f * (8.f + fabsf(logf(fmaxf(min_p, FLT_MIN)))), p_hi = min_p * (1.f + eps), p_lo = min_p * (1.f - eps);
    auto in_with = [&](float x, int i, float& near, float& w) -> bool {
      const float d = x == m ? 0.f : x - m;
      near = d * inv_t;
      w = ex2(d * inv_e);
      return kept(x, i) && w >= p_lo && (w >= p_hi || expf(z_of(x, m, t)) >= min_p);
    };
    // sum of w; the largest key with its margin (the key and the exact one differ by less than 1e-6 (|z| + |noise|), and 4e-6 is
    // allowed for), whose it is and its |z| + |noise|, and the second largest of them.  The key less its margin is a floor of the
    // largest exact key; the sum of a large z and a large noise may be small, its margin is theirs.
    float part, reach, reach2, size;
    int at;
    auto clear = [&]() { part = size = 0.f, reach = reach2 = -INFINITY, at = -1; };
    auto add = [&](float near, float w, float g, int i) {
      const float mag = fabsf(near) + fabsf(g), far = fmaf(4e-6f, mag, near + g);
      part += w;
      const bool more = far > reach;
      reach2 = fmaxf(reach2, more ? reach : far);
      if (more) reach = far, size = mag, at = i;
    };
    clear();
    // (the smallest x that may be in, somewhat less for the rounding)
    const float low = fmaxf(xc, min_p > 0.f ? m + t * (logf(p_lo) - 1e-3f) - 1e-6f * fabsf(m) : -INFINITY);
    const bool all = low == -INFINITY && m < INFINITY;  // nothing is cut
    bool sure = m < INFINITY;
    if (sure && !all) {  // (every pass gives a thread the same entries)
      for_some(low, INFINITY, [&](int i) { return noise[i]; }, [&](int i, float x, float g) {
        const float d = x - m, w = ex2(d * inv_e);
        if (kept(x, base + i) && w >= p_lo) {
          sure = sure && w >= p_hi;
          add(d * inv_t, w, g, i);
        }
      });
    } else if (sure) {
#pragma unroll 8
      for (int i = tid; i < n; i += kThreads) {
        const float x = up(src[i]), d = x - m;
        if (x > -INFINITY) add(d * inv_t, ex2(d * inv_e), noise[i], i);
      }
    }
    if (!sure) {
      clear();
      for_some(low, INFINITY, [&](int i) { return noise[i]; }, [&](int i, float x, float g) {
        float near, w;
        if (in_with(x, base + i, near, w)) add(near, w, g, i);
      });
    }
    float floor = fmaf(-8e-6f, size, reach);
    sum = cluster_sum(part, floor);
    // the entries near the largest with z as the exact quotient: a thread has one at most, if its second is not near (a reach or
    // floor that is no number: it looks at all)
    if (!(reach2 < floor)) {
      auto look = [&](int i, float x, float g) {
        float near, w;
        const bool in = in_with(x, base + i, near, w);
        g = fmaxf(g, -INFINITY);
        if (!in || fmaf(4e-6f, fabsf(near) + fabsf(g), near + g) < floor) return;
        const float z = z_of(x, m, t);
        b.take(z + g, z, base + i);
      };
      if (all)
        for (int i = tid; i < n; i += kThreads) look(i, up(src[i]), noise[i]);
      else
        for_some(low, INFINITY, [&](int i) { return noise[i]; }, look);
    } else if (!(reach < floor)) {
      const float z = z_of(up(src[at]), m, t);
      b.take(z + noise[at], z, base + at);
    }
  }
  b = block_best(b);
  if (tid == 0) sh.best[kWarps] = b;
  cl.sync();
  if (rank == 0 && warp == 0) {
    b = warp_best(lane < C ? cl.map_shared_rank(&sh, lane)->best[kWarps] : none);
    if (lane == 0) answer(b, sum);
  }
  leave();
  cl.sync();  // no block leaves while another reads its shared memory
}

// ---- rows by temperature alone: no entry is cut, so that one pass over logits and noise will do
//
// Each thread keeps the running maximum of its logits and its sum of w against that (scaled when the maximum grows), and of
// its keys, with M / T left in (x / T + noise), the two largest with their margins, as above: rounding aside the keys'
// order needs no M.  With the row's M known, a thread whose key comes near the largest forms that one again, with z as the exact
// quotient, or looks at all its entries where its second comes near too.  Bounded by reading logits and noise once, and by two cluster barriers a row.
// 256 rows of 50001 fp16: 22.9 us, 3.4 TB/s (half of the copy rate: 256 blocks where 304 find room, two thirds of the issue slots
// taken, 4 us of barriers and joining at the end).
struct PlainShared {
  float m[kWarps], s[kWarps], top[kWarps];
  int i[kWarps];
  float bm, bs, btop;  // of the block
  int bi;
  float sum;
  Best best[kWarps], block_best;
};

template <class T>
__global__ void __launch_bounds__(kThreads, 2) k_sample_plain(SampleCall c) {
  __shared__ PlainShared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), r = blockIdx.x / C;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int base = rank * c.slice, n = max(0, min(c.slice, c.vocab - base));
  const T* row = static_cast<const T*>(c.logits) + (int64_t)r * c.logits_stride + base;
  const float* noise = c.noise + (int64_t)r * c.noise_stride + base;
  pdl_wait();
  const float temp = c.temperature ? c.temperature[r] : 1.f;
  const bool greedy = !(temp > 0.f);
  const float t = greedy ? 1.f : bounded(temp), inv_t = inverse(1.f, t), inv_e = inv_t * 1.4426950408889634f;
  auto up = [](T v) -> float { return fmaxf((float)v, -INFINITY); };  // NaN as -inf
  auto scaled = [&](float s, float from, float to) { return from == to ? s : s * ex2((from - to) * inv_e); };
  float m = -INFINITY, s = 0.f, reach = -INFINITY, reach2 = -INFINITY, size = 0.f;
  int first = 0x7FFFFFFF, at = 0;  // of this thread's largest, of its key with the largest reach
  constexpr int kU = 8;  // entries whose logits and noise are under way in each thread while it takes as many
  T x[kU], x2[kU];
  float g[kU], g2[kU];
  auto load = [&](T* xs, float* gs, int k0) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int k = k0 + u * kThreads;
      xs[u] = k < n ? row[k] : T(-INFINITY), gs[u] = k < n ? noise[k] : 0.f;
    }
  };
  load(x2, g2, tid);
  for (int k0 = tid; k0 < n; k0 += kU * kThreads) {
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < kU; ++u) x[u] = x2[u], g[u] = g2[u];
    load(x2, g2, k0 + kU * kThreads);
#pragma unroll
    for (int u = 0; u < kU; ++u) most = fmaxf(most, up(x[u]));
    if (most > m) {  // the sum is scaled once for all of them
      s = m == -INFINITY ? 0.f : scaled(s, m, most);
      m = most;
#pragma unroll
      for (int u = kU - 1; u >= 0; --u)
        if ((float)x[u] == m) first = base + k0 + u * kThreads;
    }
    const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const float v = up(x[u]), near = v * inv_t, mag = fabsf(near) + fabsf(g[u]), far = fmaf(4e-6f, mag, near + g[u]);
      s += ex2((v - from) * inv_e);
      const bool more = far > reach;
      reach2 = fmaxf(reach2, more ? reach : far);
      if (more) reach = far, size = mag, at = base + k0 + u * kThreads;
    }
  }
  float top = fmaf(-8e-6f, size, reach);  // a floor of the largest exact key

  // the block's, then the row's
  auto join = [&](float& am, float& as, float& atop, int& ai, float bm, float bs, float btop, int bi) {
    const float to = fmaxf(am, bm);
    as = to == -INFINITY ? 0.f : scaled(as, am, to) + scaled(bs, bm, to);
    ai = am == bm ? min(ai, bi) : am > bm ? ai : bi;
    am = to, atop = fmaxf(atop, btop);
  };
  auto warp_join = [&](float& am, float& as, float& atop, int& ai) {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      join(am, as, atop, ai, __shfl_xor_sync(0xffffffffu, am, d), __shfl_xor_sync(0xffffffffu, as, d),
           __shfl_xor_sync(0xffffffffu, atop, d), __shfl_xor_sync(0xffffffffu, ai, d));
  };
  warp_join(m, s, top, first);
  if (lane == 0) sh.m[warp] = m, sh.s[warp] = s, sh.top[warp] = top, sh.i[warp] = first;
  __syncthreads();
  if (warp == 0) {
    const bool in = lane < kWarps;
    m = in ? sh.m[lane] : -INFINITY, s = in ? sh.s[lane] : 0.f, top = in ? sh.top[lane] : -INFINITY, first = in ? sh.i[lane] : 0x7FFFFFFF;
    warp_join(m, s, top, first);
    if (lane == 0) sh.bm = m, sh.bs = s, sh.btop = top, sh.bi = first;
  }
  cl.sync();
  {
    const PlainShared* o = cl.map_shared_rank(&sh, lane < C ? lane : 0);
    const bool in = lane < C;
    m = in ? o->bm : -INFINITY, s = in ? o->bs : 0.f, top = in ? o->btop : -INFINITY, first = in ? o->bi : 0x7FFFFFFF;
    warp_join(m, s, top, first);
  }
  Best b = {-INFINITY, 0.f, 0x7FFFFFFF};
  if (!greedy && m == INFINITY) {  // the entries of +inf share the mass: their number, and the largest of their noise
    float num = 0.f;
    for (int k = tid; k < n; k += kThreads)
      if ((float)row[k] == INFINITY) {
        num += 1.f;
        b.take(fmaxf(noise[k], -INFINITY), 0.f, base + k);
      }
#pragma unroll
    for (int d = 16; d; d >>= 1) num += __shfl_xor_sync(0xffffffffu, num, d);
    __syncthreads();
    if (lane == 0) sh.s[warp] = num;
    __syncthreads();
    if (tid == 0) {
      num = 0.f;
      for (int w = 0; w < kWarps; ++w) num += sh.s[w];
      sh.sum = num;
    }
  } else if (!greedy && m > -INFINITY) {
    const float slack = 4e-6f * fabsf(m * inv_t), floor = top - slack;
    if (!(reach2 + slack < floor)) {  // (no number: look)
      for (int k0 = tid; k0 < n; k0 += kU * kThreads) {
        float x[kU], g[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {  // all loads before their use: few threads are here, and the row waits for them
          const int k = k0 + u * kThreads;
          x[u] = k < n ? up(row[k]) : -INFINITY, g[u] = k < n ? fmaxf(noise[k], -INFINITY) : -INFINITY;
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          if (x[u] == -INFINITY) continue;
          const float near = x[u] * inv_t;
          if (fmaf(4e-6f, fabsf(near) + fabsf(g[u]), near + g[u]) + slack < floor) continue;
          const float z = z_of(x[u], m, t);
          b.take(z + g[u], z, base + k0 + u * kThreads);
        }
      }
    } else if (!(reach + slack < floor)) {
      const float z = z_of(up(row[at - base]), m, t);
      b.take(z + noise[at - base], z, at);
    }
  }
  auto warp_best = [&](Best v) -> Best {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      v.take(__shfl_xor_sync(0xffffffffu, v.v, d), __shfl_xor_sync(0xffffffffu, v.z, d), __shfl_xor_sync(0xffffffffu, v.i, d));
    return v;
  };
  const Best none = {-INFINITY, 0.f, 0x7FFFFFFF};
  b = warp_best(b);
  if (lane == 0) sh.best[warp] = b;
  __syncthreads();
  if (warp == 0) {
    b = warp_best(lane < kWarps ? sh.best[lane] : none);
    if (lane == 0) sh.block_best = b;
  }
  cl.sync();
  if (rank == 0 && warp == 0) {
    b = warp_best(lane < C ? cl.map_shared_rank(&sh, lane)->block_best : none);
    if (lane == 0) {
      if (m == INFINITY) {
        s = 0.f;
        for (int q = 0; q < C; ++q) s += cl.map_shared_rank(&sh, q)->sum;
      }
      c.token[r] = m == -INFINITY ? -1 : greedy ? first : b.i;
      if (c.logprob) c.logprob[r] = m == -INFINITY ? -INFINITY : greedy ? 0.f : b.z - logf(s);
    }
  }
  cl.sync();  // no block leaves while another reads its shared memory
}

std::atomic<int> g_hold{0};  // mf_sample_test_hold

int ceil_log2(int v) {
  int l = 0;
  while ((1 << l) < v) ++l;
  return l;
}

template <class T>
cudaError_t run(SampleCall c, int rows, cudaStream_t s) {
  // Blocks of a row: as many as leave each some ten thousand entries while they find room on the GPU at once (few rows),
  // at least so many that the slices stay in shared memory.  By temperature alone: no more than find room at once (256
  // rows of 50001: one block a row 25 us, two a row 31, four 54, whose barriers leave the memory idle).  152 and 304 are this
  // GPU's SMs and the blocks that find room on them, two an SM.
  const bool plain = !c.top_k && !c.top_p && !c.min_p;
  int C = 1;
  while (C < 8 && (plain ? (int64_t)rows * C * 2 <= 304 && c.vocab / C > 8192
                         : (size_t)((c.vocab + C - 1) / C) * sizeof(T) > 64 * 1024 || ((int64_t)rows * C < 152 && c.vocab / C > 8192)))
    C *= 2;
  c.slice = (c.vocab + C - 1) / C;
  c.qbits = 31 - ceil_log2(c.slice > 32768 ? c.slice : 32768);
  const size_t bytes = (size_t)c.slice * sizeof(T);
  c.keep = bytes <= kResident;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)rows * (unsigned)C);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = plain ? 0 : kRowAt + (c.keep ? bytes + 64 : 0);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)C, 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (plain) return cudaLaunchKernelEx(&cfg, k_sample_plain<T>, c);
  const cudaError_t e = cudaFuncSetAttribute(k_sample<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)(kRowAt + kResident + 64));
  return e == cudaSuccess ? cudaLaunchKernelEx(&cfg, k_sample<T>, c) : e;
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
  if (a->n_rows > (1 << 27)) return MF_E_INVAL;
  SampleCall c = {a->logits, a->noise, a->temperature, a->top_p, a->min_p, a->top_k, a->token, a->logprob,
                  a->logits_stride, a->noise_stride, a->vocab, 0, 0, 0, g_hold.load()};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = a->dtype == MF_F32   ? run<float>(c, a->n_rows, s)
                        : a->dtype == MF_F16 ? run<__half>(c, a->n_rows, s)
                                             : run<__nv_bfloat16>(c, a->n_rows, s);
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_sample");
}

extern "C" int mf_sample_test_hold(int hold) {
  if (hold != 0 && hold != 1) return MF_E_INVAL;
  g_hold = hold;
  return MF_OK;
}

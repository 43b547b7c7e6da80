// One token from each row of logits: temperature, top-k, top-p, min-p, and an argmax with the caller's Gumbel
// noise.  Contract: mawforge.h.
//
// The kept entries are a prefix of the row in the order (x falling, index rising), so they are described by a value and an
// index: all entries with a larger x, and those equal to it up to that index (and w >= min_p, which needs no order).
//
// A cluster of 1 to 8 blocks has a row, each block a slice of it in shared memory: the logits cross the memory bus
// once, whatever the steps that follow (a step reads shared memory, 64 entries a thread; noise is read for kept entries
// alone).  Sums and choices of the blocks meet in distributed shared memory.  Steps:
//   1. load, M = max.
//   2. top-k: a histogram of counts over bins of 1/64 in z; the bin where the count passes k.  If the entries down to
//      that bin are few (kList), they go to the leading block, which sorts them and finishes alone: top-p, min-p, argmax.
//   3. top-p of what may be many entries: a histogram of masses.  A bin's mass is a sum of integers, w / e^(-bin / 64)
//      in units of 2^-q, so it hangs on no order of additions; the border bin's entries are sorted as above.
//      (Bits: a slice of 2^s entries leaves q = 31 - s; rounding to a unit is random and below 2^-16 of an entry.)
//   4. a border bin that is too large is cut by bisection over the value's 32-bit key, and equal values by counting them
//      in the order of their index.
//   5. one pass over what is kept: sum of w, argmax of z + noise.
// What bounds it: a few passes of some ten instructions an entry and the cluster's barriers, about 1 us each; not
// the memory.
#include <cooperative_groups.h>

#include <cmath>

#include "mf_attn.cuh"

namespace cg = cooperative_groups;

namespace mf {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxVocab = 1 << 20;
constexpr int kBins = 2048, kList = 4096;
constexpr float kBinsPerUnit = 64.f;
constexpr size_t kResident = 128 * 1024;  // bytes of a slice that are kept in shared memory
constexpr uint32_t kKeyNone = 0x007FFFFFu;  // the key of -inf

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
};

// larger floats have larger keys (-0 and +0 compare equal as floats: one key)
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ float z_of(float x, float m, float t) { return x == m ? 0.f : __fdiv_rn(x - m, t); }
__device__ __forceinline__ int bin_of(float z) { return (int)fminf(-z * kBinsPerUnit, (float)(kBins - 1)); }

struct Best {  // the largest z + noise so far, the lowest index where equal
  float v, z;
  int i;
  __device__ __forceinline__ void take(float ov, float oz, int oi) {
    if (ov > v || (ov == v && oi < i)) v = ov, z = oz, i = oi;
  }
};

struct Shared {
  float d[2][kWarps];    // sums of the warps
  double pub[2];         // sums of the block, which the cluster reads
  float f[kWarps + 1];
  int n[kWarps + 1];
  Best best[kWarps + 1];
  // the leading block's answers
  float above, goal;
  int bin, count;             // border bin (-1: nothing is cut), entries down to it
  unsigned listed, kmin, kmax;  // entries put on the list, and their keys' range
  uint32_t key;
  int index;
  int here;
};

template <class T>
__global__ void __launch_bounds__(kThreads, 2) k_sample(SampleCall c) {
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ Shared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), r = blockIdx.x / C;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t* hist = reinterpret_cast<uint32_t*>(dyn);
  unsigned long long* list = reinterpret_cast<unsigned long long*>(dyn + kBins * 4);
  const int base = rank * c.slice, n = max(0, min(c.slice, c.vocab - base));
  const T* row = static_cast<const T*>(c.logits) + (int64_t)r * c.logits_stride + base;
  const float* noise = c.noise + (int64_t)r * c.noise_stride + base;
  Shared* lead = cl.map_shared_rank(&sh, 0);
  unsigned long long* lead_list = cl.map_shared_rank(list, 0);

  // ---- 1. the slice into shared memory (at the same place modulo 16 bytes, so that whole vectors are copied)
  const T* src = row;
  float mx = -INFINITY;
  auto up = [](T v) -> float {  // NaN as -inf
    const float x = (float)v;
    return x == x ? x : -INFINITY;
  };
  if ((size_t)c.slice * sizeof(T) <= kResident) {
    constexpr int kV = 16 / sizeof(T);
    T* keep = reinterpret_cast<T*>(dyn + kBins * 4 + kList * 8) + (((uintptr_t)row & 15) / sizeof(T));
    const int head = min(n, (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(T)), vecs = (n - head) / kV;
    const uint4* from = reinterpret_cast<const uint4*>(row + head);
    uint4* to = reinterpret_cast<uint4*>(keep + head);
#pragma unroll 4
    for (int i = tid; i < vecs; i += kThreads) {
      const uint4 v = ld_stream(from + i);
      to[i] = v;
      const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
      for (int u = 0; u < kV; ++u) mx = fmaxf(mx, up(e[u]));
    }
    const int rest = head + vecs * kV;
    for (int i = tid; i < head + n - rest; i += kThreads) {
      const int at = i < head ? i : rest + i - head;
      keep[at] = row[at];
      mx = fmaxf(mx, up(row[at]));
    }
    src = keep;
  } else {
    for (int i = tid; i < n; i += kThreads) mx = fmaxf(mx, up(row[i]));
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
  if (lane == 0) sh.f[warp] = mx;
  if (tid == 0) sh.listed = 0, sh.kmin = 0xFFFFFFFFu, sh.kmax = 0;
  __syncthreads();
  if (warp == 0) {
    mx = lane < kWarps ? sh.f[lane] : -INFINITY;
#pragma unroll
    for (int d = 16; d; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    if (lane == 0) sh.f[kWarps] = mx;
  }
  cl.sync();
  float m = -INFINITY;
  for (int b = 0; b < C; ++b) m = fmaxf(m, cl.map_shared_rank(&sh, b)->f[kWarps]);

  const float temp = c.temperature ? c.temperature[r] : 1.f;
  const bool greedy = !(temp > 0.f);
  const float t = greedy ? 1.f : temp;
  const int top_k = c.top_k && !greedy ? c.top_k[r] : 0;
  const float top_p = c.top_p && !greedy ? c.top_p[r] : 1.f;
  const float min_p = c.min_p && !greedy ? fminf(fmaxf(c.min_p[r], 0.f), 1.f) : 0.f;
  uint32_t kc = kKeyNone;  // kept: larger keys, and this one up to index ic
  int ic = -1;
  auto kept = [&](uint32_t k, int i) { return k > kc || (k == kc && i <= ic); };

  // a sum over the cluster, the same in every thread and whatever the order of execution (doubles only where one thread
  // adds: there are few units for them)
  int flip = 0;
  auto cluster_sum = [&](float v) -> double {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (lane == 0) sh.d[flip][warp] = v;
    __syncthreads();
    if (tid == 0) {
      double s = 0;
      for (int w = 0; w < kWarps; ++w) s += (double)sh.d[flip][w];
      sh.pub[flip] = s;
    }
    cl.sync();
    double s = 0;
    for (int b = 0; b < C; ++b) s += cl.map_shared_rank(&sh, b)->pub[flip];
    flip ^= 1;
    return s;
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
    if (lane == 31) sh.d[0][warp] = x;
    __syncthreads();
    float before = 0;
    all = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += sh.d[0][w];
      all += sh.d[0][w];
    }
    return before + x - v;
  };
  // counts (or masses, in units of 2^-qbits) of the kept entries by bin; the leading block finds the first bin down to
  // which they reach `want` (mass: want * their total); then lead->bin, above, goal, and for counts count.  Counts are whole
  // numbers below 2^24: exact in fp32.
  auto find_bin = [&](bool mass, float want) {
    for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
    __syncthreads();
    const float unit = (float)(1 << c.qbits);
    for (int i = tid; i < n; i += kThreads) {
      const float x = up(src[i]);
      if (!kept(order_key(x), base + i)) continue;
      const float z = z_of(x, m, t);
      const int b = bin_of(z);
      atomicAdd(hist + b, mass ? (uint32_t)(__expf(z + (float)b * (1.f / kBinsPerUnit)) * unit + 0.5f) : 1u);
    }
    cl.sync();
    if (rank == 0) {
      constexpr int kPer = kBins / kThreads;
      float v[kPer], sum = 0, total;
#pragma unroll
      for (int u = 0; u < kPer; ++u) {
        const int b = tid * kPer + u;
        unsigned long long s = 0;
        for (int q = 0; q < C; ++q) s += cl.map_shared_rank(hist, q)[b];
        v[u] = mass ? (float)s * expf(-(float)b * (1.f / kBinsPerUnit)) : (float)s;
        sum += v[u];
      }
      if (tid == 0) sh.bin = -1;
      float at = block_scan(sum, total);
      const float goal = mass ? want * total : want;
#pragma unroll
      for (int u = 0; u < kPer; ++u) {
        if (at < goal && at + v[u] >= goal) sh.bin = tid * kPer + u, sh.above = at, sh.count = (int)(at + v[u]);
        at += v[u];
      }
      if (tid == 0) sh.goal = goal;
    }
    cl.sync();
  };
  // the kept entries of bins lo .. hi onto the leading block's list (as many as there is room for; all are counted)
  auto gather = [&](int lo, int hi) {
    for (int i0 = 0; i0 < n; i0 += kThreads) {
      const int i = i0 + tid;
      uint32_t k = 0;
      bool in = false;
      if (i < n) {
        const float x = up(src[i]);
        k = order_key(x);
        if (kept(k, base + i)) {
          const int b = bin_of(z_of(x, m, t));
          in = b >= lo && b <= hi;
        }
      }
      const unsigned who = __ballot_sync(0xffffffffu, in);
      if (!who) continue;
      unsigned at = 0;
      if (lane == 0) at = atomicAdd(&lead->listed, (unsigned)__popc(who));
      at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1));
      if (in && at < kList) lead_list[at] = (unsigned long long)k << 32 | (0xFFFFFFFFu - (unsigned)(base + i));
      const unsigned kmin = __reduce_min_sync(0xffffffffu, in ? k : 0xFFFFFFFFu), kmax = __reduce_max_sync(0xffffffffu, in ? k : 0u);
      if (lane == 0) atomicMin(&lead->kmin, kmin), atomicMax(&lead->kmax, kmax);
    }
    cl.sync();
  };
  // the leading block's list sorted: keys falling, indices rising
  auto sort_list = [&](int len) {
    int p2 = 1;
    while (p2 < len) p2 <<= 1;
    for (int i = len + tid; i < p2; i += kThreads) list[i] = 0;
    for (int k = 2; k <= p2; k <<= 1)
      for (int j = k >> 1; j; j >>= 1) {
        __syncthreads();
        for (int i = tid; i < p2 / 2; i += kThreads) {
          const int a = 2 * i - (i & (j - 1)), b = a + j;
          const unsigned long long x = list[a], y = list[b];
          if ((x < y) == ((a & k) == 0)) list[a] = y, list[b] = x;
        }
      }
    __syncthreads();
  };
  auto block_best = [&](Best b) -> Best {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      b.take(__shfl_xor_sync(0xffffffffu, b.v, d), __shfl_xor_sync(0xffffffffu, b.z, d), __shfl_xor_sync(0xffffffffu, b.i, d));
    __syncthreads();
    if (lane == 0) sh.best[warp] = b;
    __syncthreads();
    for (int w = 0; w < kWarps; ++w) b.take(sh.best[w].v, sh.best[w].z, sh.best[w].i);
    return b;
  };
  const Best none = {-INFINITY, 0.f, 0x7FFFFFFF};
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
        if (k < from || !kept(k, base + i)) continue;
        if (mass) part += expf(z_of(x, m, t));
        else ++cnt;
      }
      return cluster_sum(mass ? part : (float)cnt);
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
      const uint32_t k = order_key(up(src[i]));
      mine += k == lo && kept(k, base + i);
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
        uint32_t k = 0;
        bool in = false;
        if (i < s1) {
          k = order_key(up(src[i]));
          in = k == lo && kept(k, base + i);
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
    kc = lo;
    ic = lead->index;
    cl.sync();
  };

  if (m == -INFINITY) {
    if (rank == 0 && tid == 0) {
      c.token[r] = -1;
      if (c.logprob) c.logprob[r] = -INFINITY;
    }
    cl.sync();
    return;
  }
  if (!greedy && top_k > 0 && top_k < c.vocab) {
    // ---- 2. top-k
    find_bin(false, (float)top_k);
    const int bin = lead->bin, count = lead->count, above = bin < 0 ? 0 : (int)lead->above;
    if (bin >= 0) {
      const bool few = count <= kList;
      gather(few ? 0 : bin, bin);
      if (few) {
        if (rank == 0) {
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
          float at = block_scan(sum, all);
          const float want = top_p * all;
          Best b = none;
          sum = 0;
#pragma unroll
          for (int u = 0; u < kPer; ++u) {
            const int i = tid * per + u;
            if (u < per && i < len && (i == 0 || ((!(top_p < 1.f) || at < want) && w[u] >= min_p))) {
              const int idx = (int)(0xFFFFFFFFu - (uint32_t)list[i]);
              const float g = noise[idx];
              b.take(g == g ? z[u] + g : -INFINITY, z[u], idx);
              sum += w[u];
            }
            at += w[u];
          }
          block_scan(sum, all);
          b = block_best(b);
          if (tid == 0) answer(b, all);
        }
        cl.sync();
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
        kc = lead->key, ic = lead->index;
      } else {
        cut_by_key(false, (double)top_k, lead->kmin, lead->kmax);
      }
      cl.sync();
      if (rank == 0 && tid == 0) sh.listed = 0, sh.kmin = 0xFFFFFFFFu, sh.kmax = 0;
    }
  }
  if (!greedy && top_p < 1.f) {
    // ---- 3. top-p
    if (!(top_p > 0.f)) {  // the first entry alone: the lowest of the largest
      kc = order_key(m);
      ic = -1;
    } else {
      find_bin(true, top_p);
      const int bin = lead->bin;
      if (bin >= 0) {
        gather(bin, bin);
        const unsigned len = lead->listed;
        if (len <= kList) {
          if (rank == 0) {
            sort_list((int)len);
            constexpr int kPer = kList / kThreads;
            const float unit = 1.f / (float)(1 << c.qbits), above = sh.above * unit, want = sh.goal * unit;
            const int per = ((int)len + kThreads - 1) / kThreads;
            float w[kPer];
            float sum = 0, all;
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
              const int i = tid * per + u;
              w[u] = u < per && i < (int)len ? expf(z_of(key_value((uint32_t)(list[i] >> 32)), m, t)) : 0.f;
              sum += w[u];
            }
            float at = above + block_scan(sum, all);
            if (tid == 0) sh.here = -1;
            __syncthreads();
            int lastk = -1;
#pragma unroll
            for (int u = 0; u < kPer; ++u) {
              const int i = tid * per + u;
              if (u < per && i < (int)len && at < want) lastk = i;
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
          kc = lead->key, ic = lead->index;
        } else {
          // the bin's share of the mass, with sums in floating point throughout
          float part = 0.f;
          for (int i = tid; i < n; i += kThreads) {
            const float x = up(src[i]);
            if (kept(order_key(x), base + i)) part += expf(z_of(x, m, t));
          }
          const double total = cluster_sum(part);
          cut_by_key(true, (double)top_p * total, lead->kmin, lead->kmax);
        }
      }
    }
  }
  // ---- 5. what is kept
  const bool first_only = greedy || top_p <= 0.f;
  Best b = none;
  float part = 0.f;
  if (first_only) {
    for (int i = tid; i < n; i += kThreads)
      if (up(src[i]) == m) b.take(0.f, 0.f, base + i);
    part = 0.f;
  } else {
#pragma unroll 4
    for (int i = tid; i < n; i += kThreads) {
      const float x = up(src[i]);
      if (!kept(order_key(x), base + i)) continue;
      const float z = z_of(x, m, t), w = expf(z);
      if (!(w >= min_p)) continue;
      const float g = noise[i];
      part += w;
      b.take(g == g ? z + g : -INFINITY, z, base + i);
    }
  }
  b = block_best(b);
  if (tid == 0) sh.best[kWarps] = b;
  const double sum = cluster_sum(part);
  if (rank == 0 && tid == 0) {
    for (int q = 1; q < C; ++q) {
      const Best o = cl.map_shared_rank(&sh, q)->best[kWarps];
      b.take(o.v, o.z, o.i);
    }
    answer(b, first_only ? 1.f : (float)sum);
  }
  cl.sync();  // no block leaves while another reads its shared memory
}

int ceil_log2(int v) {
  int l = 0;
  while ((1 << l) < v) ++l;
  return l;
}

template <class T>
cudaError_t run(SampleCall c, int rows, cudaStream_t s) {
  // Blocks of a row: as many as leave each some ten thousand entries while they find room on the GPU at once (few rows),
  // at least so many that the slices stay in shared memory.
  int C = 1;
  while (C < 8 && ((size_t)((c.vocab + C - 1) / C) * sizeof(T) > 64 * 1024 || ((int64_t)rows * C < 152 && c.vocab / C > 8192))) C *= 2;
  c.slice = (c.vocab + C - 1) / C;
  c.qbits = 31 - ceil_log2(c.slice > 32768 ? c.slice : 32768);
  const size_t keep = (size_t)c.slice * sizeof(T);
  const size_t smem = kBins * 4 + kList * 8 + (keep <= kResident ? keep + 32 : 0);
  cudaError_t e = cudaFuncSetAttribute(k_sample<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kBins * 4 + kList * 8 + kResident + 32));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)rows * (unsigned)C);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)C, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_sample<T>, c);
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
                  a->logits_stride, a->noise_stride, a->vocab, 0, 0};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = a->dtype == MF_F32   ? run<float>(c, a->n_rows, s)
                        : a->dtype == MF_F16 ? run<__half>(c, a->n_rows, s)
                                             : run<__nv_bfloat16>(c, a->n_rows, s);
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_sample");
}

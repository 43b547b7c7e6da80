// Verification of drafted tokens: the drafts that the target takes, and the token that ends each sequence.  Contract: mawforge.h.
//
// First what each row of the target's logits keeps and the sum of its weights, and the same of the drafter's rows, so that p and q of any entry are a
// few operations on its logit: by k_sample's steps without the draw where rows are cut, else (k_rows) by maxima and sums of
// pieces of them.  Then (k_verify) a cluster of 1 to 8 blocks has a sequence: a warp a draft, p and q of it; the first row whose
// draft is not taken; one pass over that row for the largest log(p - q) + noise.  In that pass log p + noise, a bound of it that
// takes no exponential, is compared with the largest key so far, and only what lies above it is worked out.
// What bounds it: reading the logits (k_rows), then of the rows that decide the logits again and the noise.
#include <cooperative_groups.h>

#include <cfloat>
#include <cmath>
#include <cstring>

#include "mf_sample.cuh"

namespace cg = cooperative_groups;

namespace mf {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;

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
  int whole[2];       // the target's, the drafter's are not cut
  int n_seqs, n_rows, vocab, n_units, slice;  // units of a row (k_rows); slice: entries of a block of k_verify
};

// ---- rows that are not cut
//
// The rows' units of 128 16-byte vectors are one list, shared out evenly: a warp takes a run of units, four vectors a lane at a time while the
// next four are under way, with a running maximum and sum a lane, and leaves a piece where a row or its run ends (which depends on
// the sizes alone).  Neighbouring runs lie on different SMs: some rows are not needed, and what is left stays evenly spread.  Bounded by
// reading the logits once; of an entry's some six instructions one is an exponential.
constexpr int kRowThreads = 256, kUnit = 128, kVecs = kUnit / 32;
template <class T>
constexpr int kUnitEntries = kUnit * 16 / (int)sizeof(T);

template <class T>
__global__ void __launch_bounds__(kRowThreads, 3) k_rows(const __grid_constant__ VerifyCall c, int side0, int rows) {
  constexpr int kV = 16 / sizeof(T);
  const int lane = threadIdx.x & 31;
  // runs: no more than units, so that each has one and a row no more pieces than units
  const int64_t U = (int64_t)rows * c.n_units, S = min((int64_t)gridDim.x * (kRowThreads / 32), U);
  const int64_t w = (int64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x, u0 = w < S ? U * w / S : 0, u1 = w < S ? U * (w + 1) / S : 0;
  pdl_wait();
  pdl_trigger();
  if (u0 >= u1) return;
  const float none = -INFINITY;
  int at = (int)(u0 / c.n_units), q = (int)(u0 - (int64_t)at * c.n_units);  // row of the list, unit of the row
  const T* x = nullptr;
  int lead_in = 0;
  auto row_of = [&](int r) {  // where a row of the list begins
    const bool second = side0 || r >= c.n_rows;
    const int row = r >= c.n_rows ? r - c.n_rows : r;
    x = second ? static_cast<const T*>(c.draft) + (int64_t)row * c.draft_stride : static_cast<const T*>(c.logits) + (int64_t)row * c.logits_stride;
    lead_in = (int)(((uintptr_t)x & 15) / sizeof(T));
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
    const int end = (int)min((int64_t)c.n_units, q + u1 - u), side = side0 || at >= c.n_rows, row = at >= c.n_rows ? at - c.n_rows : at;
    u += end - q;
    uint4 v[kVecs], next[kVecs];
    row_of(at);
    load(next, q);
    int lo = 0, hi = c.n_seqs - 1;  // the last sequence that begins at or before the row
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (c.row_start[mid] <= row) lo = mid;
      else hi = mid - 1;
    }
    const RowSpan sp = row_span(c.row_start, c.n_rows, lo);
    if (row < sp.b || row >= sp.e || (side && row + 1 == sp.e)) continue;
    const float temp = c.temperature[side] ? c.temperature[side][lo] : 1.f;
    const bool greedy = !(temp > 0.f);
    const float inv_e = inverse(1.4426950408889634f, greedy ? 1.f : bounded(temp));
    float m = none, s = 0.f;
    int first = 0x7FFFFFFF;
    for (int j = q; j < end; ++j) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) v[k] = next[k];
      if (j + 1 < end) load(next, j + 1);
      float most = none;
      auto each = [&](auto&& f) {
#pragma unroll
        for (int k = 0; k < kVecs; ++k) {
          T e[kV];
          memcpy(e, &v[k], 16);
#pragma unroll
          for (int i = 0; i < kV; ++i) f((float)e[i], (j * kUnit + k * 32 + lane) * kV - lead_in + i);
        }
      };
      each([&](float y, int) { most = fmaxf(most, y); });  // (a NaN is passed over)
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
        float part[2] = {0.f, 0.f};
        each([&](float y, int i) {
          float z;
          asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(z) : "f"((fmaxf(y, none) - m) * inv_e));
          part[i & 1] += z;
        });
        s += part[0] + part[1];
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

struct Best {  // the largest key so far, the lowest index where equal
  float v, lp;
  int i;
  __device__ __forceinline__ void take(float ov, float olp, int oi) {
    if (ov > v || (ov == v && oi < i)) v = ov, lp = olp, i = oi;
  }
};

template <class T>
__global__ void __launch_bounds__(kThreads, 2) k_verify(const __grid_constant__ VerifyCall c) {
  __shared__ Best s_best[kWarps + 1];
  __shared__ Kept s_kept[2];
  __shared__ int s_stop;
  cg::cluster_group cl = cg::this_cluster();
  const int C = (int)cl.num_blocks(), rank = (int)cl.block_rank(), s = blockIdx.x / C;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();
  const RowSpan sp = row_span(c.row_start, c.n_rows, s);
  if (sp.b == sp.e) {
    if (rank == 0 && tid == 0) c.accepted[s] = 0;
    return;
  }
  const int drafts = sp.e - sp.b - 1;
  const T* logits = static_cast<const T*>(c.logits);
  const T* draft = static_cast<const T*>(c.draft);
  // what a row keeps, in every lane of a warp (ordinary loads: read-only ones may be moved ahead of the wait)
  auto kept_of = [&](int side, int row) -> Kept {
    if (!c.whole[side]) return c.kept[(int64_t)side * c.n_rows + row];
    const Piece* pieces = c.pieces + ((int64_t)side * c.n_rows + row) * c.n_units;
    const int n = min(max(pieces->n, 0), c.n_units);
    const float temp = c.temperature[side] ? c.temperature[side][s] : 1.f;
    const bool greedy = !(temp > 0.f);
    const float t = greedy ? 1.f : bounded(temp), inv_e = inverse(1.4426950408889634f, t);
    float m = -INFINITY, sum = 0.f;
    int first = 0x7FFFFFFF;
    auto join = [&](float om, float os, int oi) {
      const float to = fmaxf(m, om);
      sum = to == -INFINITY ? 0.f : sum * (m == to ? 1.f : exp2f((m - to) * inv_e)) + os * (om == to ? 1.f : exp2f((om - to) * inv_e));
      first = m == om ? min(first, oi) : m > om ? first : oi;
      m = to;
    };
    for (int q = lane; q < n; q += 32) {
      const Piece x = pieces[q];
      join(x.m, x.s, x.first);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1)
      join(__shfl_xor_sync(0xffffffffu, m, d), __shfl_xor_sync(0xffffffffu, sum, d), __shfl_xor_sync(0xffffffffu, first, d));
    return {m, t, greedy ? m : -INFINITY, 0.f, greedy ? first : 0x7FFFFFFF, greedy ? 0.f : logf(sum), m > -INFINITY, 0};
  };
  // ---- the drafts that are taken
  if (tid == 0) s_stop = drafts;
  __syncthreads();
  for (int j = warp; j < drafts; j += kWarps) {
    const int row = sp.b + j, x = c.tokens[row + 1];
    const bool there = x >= 0 && x < c.vocab;
    const float vp = there ? (float)logits[(int64_t)row * c.logits_stride + x] : -INFINITY,
                vq = there && draft ? (float)draft[(int64_t)row * c.draft_stride + x] : -INFINITY;
    const Kept kp = kept_of(0, row);
    const float lp = log_p(kp, vp, x);
    float q = 1.f;
    if (draft) q = expf(log_p(kept_of(1, row), vq, x));
    if (lane == 0) {
      if (!(c.u[row] * q < expf(lp))) atomicMin(&s_stop, j);
      if (rank == 0) {  // (what is not taken after all is written over below)
        c.token[row] = x;
        if (c.logprob) c.logprob[row] = lp;
      }
    }
  }
  __syncthreads();
  const int stop = s_stop, row = sp.b + stop, one = stop < drafts && !draft ? c.tokens[row + 1] : -1;
  const bool less = stop < drafts && draft;
  if (warp == 0) {
    const Kept k = kept_of(0, row);
    if (lane == 0) s_kept[0] = k;
  } else if (warp == 1 && less) {
    const Kept k = kept_of(1, row);
    if (lane == 0) s_kept[1] = k;
  }
  __syncthreads();
  const Kept kp = s_kept[0], kq = s_kept[1];

  // ---- the token after them
  const int i0 = rank * c.slice, i1 = min(c.vocab, i0 + c.slice);
  const T* x = logits + (int64_t)row * c.logits_stride;
  const T* y = less ? draft + (int64_t)row * c.draft_stride : x;
  const float* noise = c.noise + (int64_t)s * c.noise_stride;
  const Best none = {-INFINITY, -INFINITY, 0x7FFFFFFF};
  auto warp_best = [&](Best b) -> Best {
#pragma unroll
    for (int d = 16; d; d >>= 1)
      b.take(__shfl_xor_sync(0xffffffffu, b.v, d), __shfl_xor_sync(0xffffffffu, b.lp, d), __shfl_xor_sync(0xffffffffu, b.i, d));
    return b;
  };
  const float inv_t = inverse(1.f, kp.t), low = fmaxf(kp.xc, -FLT_MAX);  // (NaN and -inf are never kept)
  Best b;
  for (int turn = 0; turn < 2; ++turn) {  // (the second where no entry has p > q: with p alone)
    b = none;
    const bool minus = less && turn == 0;
    constexpr int kU = 4;  // entries of a thread that are under way while it takes as many
    float floor = -INFINITY;
    T vx[kU], vy[kU], wx[kU], wy[kU];
    float g[kU], h[kU];
    auto load = [&](T* ax, T* ay, float* ag, int k0) {
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int i = k0 + u * kThreads;
        const bool in = i < i1;
        ax[u] = in ? x[i] : T(-INFINITY), ag[u] = in ? noise[i] : -INFINITY;
        ay[u] = in && minus ? y[i] : T(-INFINITY);
      }
    };
    load(wx, wy, h, i0 + tid);
    for (int kb = i0; kb < i1; kb += kU * kThreads) {  // (a warp's lanes together)
      const int k0 = kb + tid;
#pragma unroll
      for (int u = 0; u < kU; ++u) vx[u] = wx[u], vy[u] = wy[u], g[u] = h[u];
      load(wx, wy, h, k0 + kU * kThreads);
      // The bound of a key: z as a product differs from the quotient by a few 2^-24 of it; the margin is several times that of all
      // roundings.  (A bound that is no number is looked at.)
      float ub[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const float v = (float)vx[u], z = (v - kp.m) * inv_t;
        const int i = k0 + u * kThreads;
        ub[u] = fmaf(4e-6f, fabsf(z) + fabsf(kp.log_sum) + fabsf(g[u]) + 1.f, z - kp.log_sum + g[u]);
        ub[u] = ub[u] != ub[u] ? INFINITY : fmaxf(ub[u], -FLT_MAX);
        if (!(v >= low) || i >= i1 || (turn == 0 && i == one)) ub[u] = -INFINITY;
      }
      // each thread's most promising entry in turn, until none of the warp's reaches its largest key
      for (;;) {
        float most = -INFINITY, cg = 0.f;
        T cx = T(0.f), cy = T(0.f);
        int ci = -1;
#pragma unroll
        for (int u = 0; u < kU; ++u)
          if (ub[u] > most) most = ub[u], cx = vx[u], cy = vy[u], cg = g[u], ci = u;
        const bool look = ci >= 0 && !(most < floor);
        if (!__any_sync(0xffffffffu, look)) break;
        if (look) {
#pragma unroll
          for (int u = 0; u < kU; ++u)
            if (u == ci) ub[u] = -INFINITY;
          const int i = k0 + ci * kThreads;
          const float lp = log_p(kp, (float)cx, i);
          float key = lp;
          bool in = lp > -INFINITY;
          if (in && minus) {
            const float lq = log_p(kq, (float)cy, i);
            if (lq > -INFINITY) {
              const float rest = expf(lp) - expf(lq);
              in = rest > 0.f;
              key = logf(rest);
            }
          }
          if (in) b.take(fmaxf(key + cg, -INFINITY), lp, i);
        }
        floor = b.v;
#pragma unroll
        for (int d = 16; d; d >>= 1) floor = fmaxf(floor, __shfl_xor_sync(0xffffffffu, floor, d));
      }
    }
    b = warp_best(b);
    __syncthreads();
    if (lane == 0) s_best[warp] = b;
    __syncthreads();
    if (warp == 0) {
      b = warp_best(lane < kWarps ? s_best[lane] : none);
      if (lane == 0) s_best[kWarps] = b;
    }
    cl.sync();
    b = warp_best(lane < C ? cl.map_shared_rank(s_best, lane)[kWarps] : none);
    cl.sync();  // no block writes its best again, or leaves, while another reads it
    if (b.i != none.i) break;
  }

  if (rank != 0) return;
  const bool empty = b.i == none.i;
  for (int j = stop + tid; j <= drafts; j += kThreads) {
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
  int C = 1;
  while (C < 8 && (int64_t)n_seqs * C * 2 <= 304 && c.vocab / C > 8192) C *= 2;
  c.slice = (c.vocab + C - 1) / C;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_seqs * (unsigned)C);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)C, 1, 1};
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_verify<T>, c);
}

bool bad_word(const void* p) { return ((uintptr_t)p & 3) != 0; }
bool bad_cuts(const mf_cuts_t& c) { return bad_word(c.temperature) || bad_word(c.top_p) || bad_word(c.min_p) || bad_word(c.top_k); }

}  // namespace
}  // namespace mf

using namespace mf;

extern "C" int mf_verify_bytes(int n_seqs, int n_rows, int vocab, uint64_t* out) {
  if (!out || n_seqs < 0 || n_rows < 0 || n_seqs > (1 << 26) || n_rows > (1 << 26) || vocab < 1 || vocab > kMaxVocab) return MF_E_INVAL;
  const uint64_t units = ((uint64_t)vocab + kUnitEntries<float> + 2) / kUnitEntries<float>;
  *out = (uint64_t)(n_rows > 0 ? n_rows : 1) * 2 * (sizeof(Kept) + units * sizeof(Piece));
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
  Kept* kept = static_cast<Kept*>(a->work);
  const VerifyCall c = {a->logits, a->draft_logits, a->logits_stride, a->draft_stride, a->noise_stride, a->row_start, a->tokens, a->u, a->noise,
                        {a->cuts.temperature, a->draft_cuts.temperature}, a->token, a->accepted, a->logprob, kept,
                        reinterpret_cast<Piece*>(kept + 2 * (int64_t)a->n_rows), {whole_p, whole_q}, a->n_seqs, a->n_rows, a->vocab, 0, 0};
  cudaError_t e = cudaSuccess;
  if (a->n_rows > 0 && (!whole_p || (a->draft_logits && !whole_q))) {
    const KeptRows rows = {a->logits,  whole_q ? nullptr : a->draft_logits, a->logits_stride, a->draft_stride, a->row_start, a->cuts, a->draft_cuts, kept,
                           a->n_seqs, a->n_rows, a->vocab, a->dtype, !whole_p};
    e = launch_kept(rows, s);
  }
  if (e == cudaSuccess) e = a->dtype == MF_F32 ? run<float>(c, s) : a->dtype == MF_F16 ? run<__half>(c, s) : run<__nv_bfloat16>(c, s);
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_verify");
}

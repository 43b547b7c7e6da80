// Paged attention of many query rows (prefill chunks, verification batches) on the fifth-generation tensor cores.
//
// Rows.  The tokens of a sequence times the query heads that share a kv head are one list of rows (token major), cut into
// row tiles of 128, so K and V are read once for the whole group and short chunks fill a tile with several heads.
// A work item ("segment") is one or two row tiles of a (sequence, kv head) and the 128-line key tiles that
// any of their rows sees; per key tile and row tile ("job")
//   S = Q K^T (tcgen05, both operands in shared memory)  ->  tensor memory, 128 fp32 columns
//   P = 2^(scale log2e S - m), rounded to the cache's type, written over S      (one thread a row; the first 64 lines'
//                                                              products with V begin while the others are computed)
//   O += P V  (A from tensor memory, V read as it lies: its lines are the K dimension, an MN-major operand)
// with a running maximum m and sum l per row.  O is rescaled only when m grows by more than 2^8 (until then the old m
// serves: p stays below 2^8, and o and l carry the same factor); so most key tiles touch O not at all.
//
// Two jobs are always under way: while the tensor cores run one's products the softmax of the other is computed,
// S and P in two buffers.  With head_dim 64 and 128 they are the two row tiles of a segment (they share K and V in
// shared memory, which halves the cache's traffic), each with a warpgroup of its own; with head_dim 256, whose O fills
// half of the tensor memory, or where a segment has one row tile, they are successive key tiles of it.
//
// 12 warps: 0-3 and 4-7 softmax (thread = row; the maximum and the sum need no shuffles), 8 issues the MMAs of S, 9 those of O
// (one warp for both left the tensor cores idle while it waited between products: their queue covers a few hundred
// cycles), 10 copies Q and K, 11 V, each into a ring of its own.  A barrier has one waiting role, which sees every phase of
// it.  Copies are TMA boxes of as many lines as the largest power of two that divides the page (8 to 128); a tile that
// reaches past its sequence's lines (where anything may lie, NaN among it, which a product with p = 0 would pass on)
// or before every window is copied line by line with cp.async, such lines becoming zeros.  So are all tiles of pages that
// are no multiple of 8 lines, and Q where the group does not divide 128.
//
// Split.  As for few rows: the step's jobs are one list shared out evenly over one block per SM; pieces of segments that
// a block does not have whole are left as partials and joined in order.
//
// Measured: 2048 tokens over 14336 lines, 32/8 heads of 128, causal: 360 to 375 us, 1.4 PFLOP/s (72 % of the library's rate; the
// tensor pipe is busy 66 % of the time, the rest is softmax and the waits between a job's two products); eight prompts of 1494 to
// 4001 tokens, 32/4 heads of 128: 457 to 464 us, 1.13 PFLOP/s (beginnings and ends of segments); 8192 tokens, 16/8 heads of 256,
// window 1024: 173 us, 0.75 PFLOP/s (segments of 9 to 10 key tiles, two of them masked; 4096 tokens over 16384 without a window: 881 us,
// 1.40 PFLOP/s).
#include <cstring>

#include "mf_attn.cuh"
#include "mf_tc.cuh"

namespace mf {
namespace {

constexpr int kThreads = 384, kQkWarp = 8, kPvWarp = 9, kKWarp = 10;
constexpr int kKeys = 128;                  // lines of a key tile
constexpr uint32_t kUnitBytes = 128 * 128;  // 128 lines x 64 elements
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kGrow = 8.f;  // growth of the maximum (log2) that o is rescaled for

template <int D>
struct Cfg {
  static constexpr int kU = D / 64;                   // units of a K or V tile
  static constexpr int kSlotU = D == 64 ? 1 : 2;      // units of a ring slot: what one barrier and one product of O cover
  static constexpr int kTileSlots = kU / kSlotU;
  static constexpr int kKSlots = D == 64 ? 5 : 3, kVSlots = D == 64 ? 5 : 2;  // 160 KiB of rings
  static constexpr uint32_t kSlotBytes = kSlotU * kUnitBytes;
  static constexpr int kRowTiles = D == 256 ? 1 : 2;  // row tiles of a segment
  static constexpr int kRows = kRowTiles * 128;
  static constexpr uint32_t kQBytes = kRowTiles * kU * kUnitBytes;
  // jobs that a segment's beginning and end cost (first scores without a product beside them, O to memory)
  static constexpr int kOver = 4;
  static constexpr uint32_t kTail = kQBytes + (kKSlots + kVSlots) * kSlotBytes;  // then a Tail
};
constexpr uint32_t kTmemCols = 512, kColS = 0, kColO = 256;

// ---- the step's segments

// One block: for each sequence the index of its first row tile, for each row tile its description and the jobs before it.
template <int D>
__global__ void __launch_bounds__(1024) k_attn_plan(AttnCall c, AttnPlan p) {
  __shared__ int64_t s_warp[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_trigger();
  auto scan = [&](int64_t v, int64_t& all) -> int64_t {  // exclusive prefix over the block, and the sum
    int64_t x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += o;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    int64_t before = 0;
    all = 0;
    for (int w = 0; w < 32; ++w) {
      if (w < warp) before += s_warp[w];
      all += s_warp[w];
    }
    return before + x - v;
  };
  int64_t done = 0;
  for (int base = 0; base < c.st.n_seqs; base += 1024) {
    const int s = base + tid;
    int n = 0;
    if (s < c.st.n_seqs) n = (seq_span(c.st, s).n * c.st.G + Cfg<D>::kRows - 1) / Cfg<D>::kRows;
    int64_t all;
    const int64_t at = done + scan(n, all);
    if (s < c.st.n_seqs) p.first[s] = (int)min(at, (int64_t)p.max_tiles);
    done += all;
  }
  const int tiles = (int)min(done, (int64_t)p.max_tiles);
  if (tid == 0) p.first[c.st.n_seqs] = tiles;
  __syncthreads();
  int64_t jobs = 0;
  for (int base = 0; base < tiles; base += 1024) {
    const int i = base + tid;
    int64_t n = 0;
    if (i < tiles) {
      int lo = 0, hi = c.st.n_seqs - 1;  // the last sequence whose first tile is at or before i
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.first[mid] <= i) lo = mid;
        else hi = mid - 1;
      }
      const SeqSpan sp = seq_span(c.st, lo);
      const int qt = i - p.first[lo], R0 = qt * Cfg<D>::kRows, G = c.st.G;
      const int rows = min(Cfg<D>::kRows, sp.n * G - R0), first = sp.len - sp.n;
      int start = vis_lo(c, first + R0 / G);
      if (c.box) start &= ~(c.box - 1);
      const int end = max(0, vis_hi(c, first + (R0 + rows - 1) / G, sp.len));
      p.tile[2 * i] = make_int4(lo, sp.q0, sp.n, sp.len);
      p.tile[2 * i + 1] = make_int4(qt, rows, start, end);
      n = ((int64_t)max(1, (end - start + kKeys - 1) / kKeys) << (Cfg<D>::kRowTiles == 2 && rows > 128)) + Cfg<D>::kOver;
    }
    int64_t all;
    const int64_t at = jobs + scan(n, all);
    if (i < tiles) p.before[i] = at;
    jobs += all;
  }
  if (tid == 0) p.before[tiles] = jobs;
}

// The walk over a block's segments: key tiles j0 .. j1 - 1 of a row tile (of all: `tile`) and kv head h.  The list is
// ordered by sequence, kv head, row tile.  The next tile's description is asked for when the walk comes to a segment, and
// has long arrived when the segment ends.  The roles' loops together have to fit the instruction cache (with walks that
// looked everything up inline, two fifths of the fetches missed and a job took five times as long).
template <int kRows, int kOver>
struct Walk {
  int s, q0, n, len;          // the sequence: new tokens, lines
  int qt, rows, start, end;   // the row tile: its place, rows, lines that any of them sees
  int h, tile, j0, j1, nt;
  int two;                    // 1: two row tiles, two jobs a key tile
  int4 na, nb;                // the next tile's description
  int64_t at, t0, t1;         // place of the segment's first job in the list; the block's share
  bool more;                  // this is a segment of the block

  __device__ __forceinline__ void set(int4 a, int4 b) {
    s = a.x, q0 = a.y, n = a.z, len = a.w, qt = b.x, rows = b.y, start = b.z, end = b.w;
    two = rows > 128;
    nt = max(1, (end - start + kKeys - 1) / kKeys);
    // a key tile belongs to the block that its first job falls to; the segment's kOver come before its jobs
    const int64_t up0 = (t0 - at - kOver + two) >> two, up1 = (t1 - at - kOver + two) >> two;
    j0 = (int)max((int64_t)0, up0);
    j1 = (int)min((int64_t)nt, up1);
  }
  // the tile after this one in the list (of this kv head or the next)
  __device__ __forceinline__ int following(const AttnCall& c) const {
    return (qt + 1) * kRows >= n * c.st.G && h + 1 < c.st.Hkv ? tile - qt : tile + 1;
  }
  __device__ __forceinline__ void ask(const AttnCall& c, const AttnPlan& p) {
    const int f = min(following(c), p.max_tiles - 1);  // (past the last tile: anything, not used)
    na = __ldg(p.tile + 2 * f), nb = __ldg(p.tile + 2 * f + 1);
  }
  __device__ __forceinline__ void next(const AttnCall& c, const AttnPlan& p) {
#pragma unroll 1
    do {
      at += ((int64_t)nt << two) + kOver;
      if (at >= t1) {
        more = false;
        return;
      }
      const int f = following(c);
      if ((qt + 1) * kRows >= n * c.st.G) h = f > tile ? 0 : h + 1;
      tile = f;
      set(na, nb);
      ask(c, p);
    } while (j0 >= j1);
  }
};
// to the block's first segment
template <int kRows, int kOver>
__device__ __noinline__ void walk_start(Walk<kRows, kOver>& w, const AttnCall& c, const AttnPlan& p, int tiles, int64_t a, int64_t b) {
  w.t0 = a, w.t1 = b;
  w.more = a < b;
  if (!w.more) return;
  // the last tile whose sequence starts at or before a, then the kv head, then the tile
  int lo = 0, hi = tiles - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    const int first = mid - __ldg(p.tile + 2 * mid + 1).x;
    if (__ldg(p.before + first) * c.st.Hkv <= a) lo = mid;
    else hi = mid - 1;
  }
  const int first = lo - __ldg(p.tile + 2 * lo + 1).x, end = lo + 1;
  const int64_t b0 = __ldg(p.before + first), len = __ldg(p.before + end) - b0;
  w.h = (int)((a - b0 * c.st.Hkv) / len);
  const int64_t head = b0 * c.st.Hkv + w.h * len;
  lo = first, hi = end - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (head + __ldg(p.before + mid) - b0 <= a) lo = mid;
    else hi = mid - 1;
  }
  w.tile = lo;
  w.at = head + __ldg(p.before + lo) - b0;
  w.set(__ldg(p.tile + 2 * lo), __ldg(p.tile + 2 * lo + 1));
  w.ask(c, p);
  if (w.j0 >= w.j1) w.next(c, p);
}

// The jobs of the walk one by one: (key tile, row tile), row tile inner.
struct Jobs {
  int i, n, two;  // job in its segment, of n; two row tiles
  bool live;
  template <class W>
  __device__ __forceinline__ void take(const W& w) {
    live = w.more;
    i = 0;
    two = w.two;
    n = (w.j1 - w.j0) << two;
  }
  __device__ __forceinline__ int row_tile() const { return two & i; }  // also: which of the tile's jobs
  __device__ __forceinline__ bool first_of_tile() const { return !(two & i); }
  __device__ __forceinline__ bool last_of_tile() const { return !two || (i & 1); }
};

// What the softmax needs of a segment, told by the warp that copies K: it comes to a segment a few key tiles ahead, and the
// softmax, which has no registers to walk with, finds it in shared memory.
struct Piece {
  int nj, two, k_start, R0, rows, h, q0, first, len, nt, j0, more;
  int64_t last;  // place of the last key tile's first job
  template <int kRows, int kOver>
  __device__ __forceinline__ void take(const Walk<kRows, kOver>& w) {
    more = w.more, two = w.two, nj = w.j1 - w.j0, k_start = w.start + w.j0 * kKeys, R0 = w.qt * kRows, rows = w.rows;
    h = w.h, q0 = w.q0, first = w.len - w.n, len = w.len, nt = w.nt, j0 = w.j0;
    last = w.at + kOver + ((int64_t)(nt - 1) << two);
  }
};

// A wait whose first poll failed; false, with the block's flag and the error word set, once any wait gave up.
__device__ __noinline__ bool wait_slow(uint64_t* bar, uint32_t parity, volatile int* flag, unsigned* err) {
  if (*flag) return false;
  if (mbar_wait(bar, parity, kDefaultWaitNs)) return true;
  *flag = 1;
  atomicOr(err, kAttnTimeout);
  return false;
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// 4-D tiled TMA load of the box at (element, head, line, page), completing on `bar`
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* tm, int x, int h, int line, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(h), "r"(line), "r"(page), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
// 64 lines x 64 elements to `dst`, swizzled; a0, a1: element offsets of lines lane, lane + 32 (negative: a line of zeros)
template <class T>
__device__ __noinline__ void copy_lines(uint32_t dst, const T* base, int64_t a0, int64_t a1) {
  const int lane = threadIdx.x & 31, ch = lane & 7, sub = lane >> 3;
  dst += sub * 128;
  const uint32_t even = (uint32_t)(ch ^ sub) << 4, odd = (uint32_t)(ch ^ (sub + 4)) << 4;  // lines sub, sub + 4 of eight
#pragma unroll 1
  for (int q = 0; q < 2; ++q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t o = __shfl_sync(0xffffffffu, a0, i * 4 + sub);
      cp16(dst + i * 512 + (i & 1 ? odd : even), base + (o < 0 ? 0 : o + ch * 8), o < 0 ? 0u : 16u);
    }
    dst += 4096;
    a0 = a1;
  }
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// shared memory: [Q][ring of K][ring of V]; barriers: slots full and free, Q full and free, S and P by (warpgroup,
// buffer; kBP2: the second half of P), O by who reads it, the buffers free again, the end of all MMAs, and for segments of
// one row tile m and l written, read, O read; segments told, done with
constexpr int kBKFull = 0, kBKFree = 5, kBVFull = 10, kBVFree = 15, kBQFull = 20, kBQFree = 21, kBS = 22, kBP = 26, kBO = 30,
              kBBuf = 32, kBDrain = 34, kBP2 = 36, kBStat = 40, kBStatFree = 41, kBOFree = 42,
              kBPiece = 43, kBPieceFree = 47, kBars = 51;
constexpr int kPieces = 4;

struct Tail {
  uint64_t bars[kBars];
  Piece piece[kPieces];
  float2 stat[128];  // m and l of the rows of a segment of one row tile
  uint32_t tmem;
  int flag;
};

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1) k_attn_many(const __grid_constant__ AttnCall c, const __grid_constant__ AttnMaps maps,
                                                           const __grid_constant__ AttnPlan p,
                                                           const __grid_constant__ AttnParts parts) {
  using C = Cfg<D>;
  constexpr bool kBf = Half2<T>::kBf16;
  extern __shared__ __align__(1024) unsigned char smem[];  // (nothing static beside it: it begins at a multiple of 1024)
  Tail& tail = *reinterpret_cast<Tail*>(smem + C::kTail);
  uint64_t* bars = tail.bars;
  uint32_t& s_tmem = tail.tmem;
  volatile int& s_flag = tail.flag;
  const uint32_t smem0 = smem_u32(smem);
  const uint32_t kring = smem0 + C::kQBytes, vring = kring + C::kKSlots * C::kSlotBytes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const AttnStep& st = c.st;
  if (tid == 0) {
    for (int i = 0; i < kBars; ++i) mbar_init(&bars[i], i >= kBPieceFree ? 8 : i >= kBPiece ? 1 : (i >= kBP && i < kBP + 4) || i >= kBP2 ? 4 : 1);
    s_flag = 0;
    mbar_fence_init();
  }
  if (warp == kQkWarp) tc::alloc(&s_tmem, kTmemCols);
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  const uint32_t tmem = s_tmem;
  pdl_wait();
  pdl_trigger();

  const int tiles = __ldg(p.first + st.n_seqs);
  const int64_t total = tiles ? __ldg(p.before + tiles) * st.Hkv : 0;
  // every block that works has at least two jobs, so that it has a key tile's start
  const int64_t B = max((int64_t)1, min((int64_t)gridDim.x, total / 2));
  const int64_t b = blockIdx.x;
  const int64_t t0 = b < B ? total * b / B : 0, t1 = b < B ? total * (b + 1) / B : 0;

  auto wait = [&](int bar, uint32_t parity) -> bool {  // bounded
    return mbar_try_wait(&bars[bar], parity) || wait_slow(&bars[bar], parity, &s_flag, st.err);
  };
  auto wait_all = [&](int bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, wait(bar, parity)); };

  if (warp < kQkWarp) {
    // ================= softmax: warpgroup wg has row tile wg of two; of the only one, 0 the softmax and 1 the storing of
    // O, while 0 has begun the next segment
    const int wg = warp >> 2, row = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const float sc2 = c.scale * kLog2e;
    int par = 0;                     // buffer of the segment's first job
    uint32_t sph[2] = {0, 0};        // phases of this warpgroup's S barriers, by buffer
    uint32_t oph = 0, lph = wg ^ 1;      // phases of its O barrier, of that of m and l (0 waits for them to be read)
    int rec_n = 0;
    bool alive = true;
    int at = 0;
    uint32_t pph = 0;
    for (;;) {
      if (!(alive = wait_all(kBPiece + at, pph))) break;
      const Piece& cur = tail.piece[at];
      if (!cur.more) break;
      const int nj = cur.nj, two = cur.two, k_start = cur.k_start, tile_row = (two ? wg * 128 : 0) + row;
      const uint32_t col_o = tmem + lanes + kColO + (two ? wg * D : 0);
      const bool ok = tile_row < cur.rows;
      float m = -INFINITY, l = 0.f;
      if (two || wg == 0) {
        const int pos = cur.first + (cur.R0 + tile_row) / st.G;
        const int lo = ok ? vis_lo(c, pos) : 0, hi = ok ? vis_hi(c, pos, cur.len) : 0;
        for (int j = 0; j < nj; ++j) {
          const int buf = (par + (two ? wg : j)) & 1;
          if (!(alive = wait_all(kBS + wg * 2 + buf, sph[buf] & 1))) break;
          ++sph[buf];
          tc::fence_after();
          const uint32_t col_s = tmem + lanes + kColS + buf * 128;
          const int k0 = k_start + j * kKeys, a = lo - k0, z = hi - k0;  // columns [a, z) are seen
          if (__any_sync(0xffffffffu, a > 0 || z < kKeys)) {
            // a tile at an edge (one or two of a segment): -inf written over the others
#pragma unroll
            for (int i = 0; i < 128; i += 32) {
              uint32_t v[32];
              tc::ld32(col_s + i, v);
              tc::wait_ld();
              tc::pin32(v);
              const int za = min(max(z - i, 0), 32), aa = min(max(a - i, 0), 32);
              const uint32_t bits = (uint32_t)((1ull << za) - 1) & ~(uint32_t)((1ull << aa) - 1);
#pragma unroll
              for (int u = 0; u < 32; ++u) v[u] = bits >> u & 1 ? v[u] : 0xFF800000u;
              tc::st32(col_s + i, v);
            }
            tc::wait_st();
          }
          // the row's scores: the first 64 stay in registers, the others are read again when their turn comes
          uint32_t sa[64], sb[64];
          tc::ld32(col_s, sa);
          tc::ld32(col_s + 32, sa + 32);
          tc::ld32(col_s + 64, sb);
          tc::ld32(col_s + 96, sb + 32);
          tc::wait_ld();
          tc::pin32(sa), tc::pin32(sa + 32), tc::pin32(sb), tc::pin32(sb + 32);
          float mx[4] = {m, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 64; i += 4)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              mx[u] = fmaxf(mx[u], fmaxf(__uint_as_float(sa[i + 2 * u]), __uint_as_float(sa[i + 2 * u + 1])));
              mx[2 + u] = fmaxf(mx[2 + u], fmaxf(__uint_as_float(sb[i + 2 * u]), __uint_as_float(sb[i + 2 * u + 1])));
            }
          const float mn = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
          bool waited = two || j == 0;  // two row tiles: S(g + 2) is formed after O(g)
          if (j == 0) {
            m = mn;
          } else if (__any_sync(0xffffffffu, (mn - m) * sc2 > kGrow)) {
            if (!waited) {
              if (!(alive = wait_all(kBO + wg, oph))) break;
              oph ^= 1;
              tc::fence_after();
              waited = true;
            }
            const float f = mn == -INFINITY ? 1.f : ex2((m - mn) * sc2);
            m = mn;
            l *= f;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
              uint32_t o[32];
              tc::ld32(col_o + i * 32, o);
              tc::wait_ld();
              tc::pin32(o);
#pragma unroll
              for (int u = 0; u < 32; ++u) o[u] = __float_as_uint(__uint_as_float(o[u]) * f);
              tc::st32(col_o + i * 32, o);
            }
          }
          const float ms = m == -INFINITY ? 0.f : m * sc2;
          const uint64_t sc2x2 = tc::pack2(sc2, sc2), nms2 = tc::pack2(-ms, -ms);
          uint64_t sum[2] = {0, 0};
          auto exps = [&](uint32_t* s, uint32_t col) {  // 64 scores -> P, written over S
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t pk[16];
#pragma unroll
              for (int u = 0; u < 16; ++u) {
                float e0, e1;
                tc::unpack2(tc::fma2(tc::pack2(__uint_as_float(s[32 * i + 2 * u]), __uint_as_float(s[32 * i + 2 * u + 1])), sc2x2, nms2),
                            e0, e1);
                e0 = ex2(e0), e1 = ex2(e1);
                sum[u & 1] = tc::add2(sum[u & 1], tc::pack2(e0, e1));
                pk[u] = Half2<T>::down(e0, e1);
              }
              tc::st16(col_s + col + i * 16, pk);
            }
          };
          tc::ld32(col_s + 64, sb);
          tc::ld32(col_s + 96, sb + 32);
          exps(sa, 0);
          tc::wait_st();
          if (!waited) {  // keeps this barrier's phases in step
            if (!(alive = wait_all(kBO + wg, oph))) break;
            oph ^= 1;
          }
          tc::fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[kBP + wg * 2 + buf]);
          tc::wait_ld();
          tc::pin32(sb), tc::pin32(sb + 32);
          exps(sb, 32);
          float l0, l1;
          tc::unpack2(tc::add2(sum[0], sum[1]), l0, l1);
          l += l0 + l1;
          tc::wait_st();
          tc::fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[kBP2 + wg * 2 + buf]);
        }
        if (!alive) break;
        if (tid == 0 && cur.j0 == 0 && nj != cur.nt) {
          // the block of the segment's last key tile, by the place of its first job
          rec_n = (int)((B * (cur.last + 1) - 1) / total) - (int)b + 1;
          parts.rec[b] = {cur.q0, cur.h, cur.R0, cur.rows, rec_n};
        }
        if (!two) {  // m and l to the other warpgroup
          if (!(alive = wait_all(kBStatFree, lph))) break;
          lph ^= 1;
          tail.stat[row] = make_float2(m, l);
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[kBStat]);
        }
      } else {
        if (!(alive = wait_all(kBStat, lph))) break;
        lph ^= 1;
        const float2 ml = tail.stat[row];
        m = ml.x, l = ml.y;
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[kBStatFree]);
      }
      if (two || wg == 1) {
        // ---- the piece's o
        if (!(alive = wait_all(kBO + wg, oph))) break;
        oph ^= 1;
        tc::fence_after();
        const int R = cur.R0 + tile_row, tok = R / st.G, q0 = cur.q0, h = cur.h, j0 = cur.j0;
        const bool whole = nj == cur.nt;
        // partials column group by column group, so that a warp's rows are neighbours
        const int64_t pr0 = ((int64_t)b * 2 + (j0 == 0)) * C::kRows, pr = pr0 + tile_row;
        float* po = parts.o + pr0 * D + tile_row * 4;
        const int head = h * st.G + R % st.G;
        if (whole) {
          // 64 columns at a time: 32 bytes of a row and lane, transposed among four lanes, so that these store 128
          // neighbouring bytes of one row after the other (a row a lane, the stores took 4000 cycles a segment)
          const float inv = l == 0.f ? 0.f : 1.f / l;  // (a NaN in the scores stays NaN)
          const bool wide = (((uintptr_t)c.out | (uintptr_t)(c.out_stride * 2)) & 31) == 0;
          const int64_t at = ok ? (int64_t)(q0 + tok) * c.out_stride + (int64_t)head * D : -1;
          T* out[4];  // where the rows of this lane's four begin, this lane's quarter of 64 columns; null: no row
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t o = __shfl_sync(0xffffffffu, at, (lane & ~3) + i);
            out[i] = o < 0 ? nullptr : static_cast<T*>(c.out) + o + (lane & 3) * 16;
          }
#pragma unroll
          for (int i = 0; i < D / 64; ++i) {
            uint32_t o[64], v[4][8];
            tc::ld32(col_o + i * 64, o);
            tc::ld32(col_o + i * 64 + 32, o + 32);
            tc::wait_ld();
            tc::pin32(o), tc::pin32(o + 32);
#pragma unroll
            for (int u = 0; u < 32; ++u) v[u >> 3][u & 7] = Half2<T>::down(__uint_as_float(o[2 * u]) * inv, __uint_as_float(o[2 * u + 1]) * inv);
#pragma unroll
            for (int bit = 1; bit <= 2; bit <<= 1) {
              const bool up = lane & bit;
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                if (q & bit) continue;
#pragma unroll
                for (int x = 0; x < 8; ++x) {  // blocks q and q + bit: the one that belongs to the other lane changes places
                  const uint32_t give = up ? v[q][x] : v[q + bit][x];
                  const uint32_t got = __shfl_xor_sync(0xffffffffu, give, bit);
                  if (up) v[q][x] = got;
                  else v[q + bit][x] = got;
                }
              }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {  // v[r]: columns 16 (lane % 4) .. of the 64, row r of the four
              if (!out[r]) continue;
              T* to = out[r] + i * 64;
              if (wide) {
                asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(v[r][0]), "r"(v[r][1]), "r"(v[r][2]),
                             "r"(v[r][3]), "r"(v[r][4]), "r"(v[r][5]), "r"(v[r][6]), "r"(v[r][7])
                             : "memory");
              } else {
                *reinterpret_cast<uint4*>(to) = make_uint4(v[r][0], v[r][1], v[r][2], v[r][3]);
                *reinterpret_cast<uint4*>(to + 8) = make_uint4(v[r][4], v[r][5], v[r][6], v[r][7]);
              }
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < D / 32; ++i) {
            uint32_t o[32];
            tc::ld32(col_o + i * 32, o);
            tc::wait_ld();
            tc::pin32(o);
            if (!ok) continue;
#pragma unroll
            for (int u = 0; u < 8; ++u)
              *reinterpret_cast<uint4*>(po + (int64_t)(i * 8 + u) * (C::kRows * 4)) =
                  make_uint4(o[4 * u], o[4 * u + 1], o[4 * u + 2], o[4 * u + 3]);
          }
        }
        if (ok) {
          const float mm = m == -INFINITY ? m : m * sc2;
          if (!whole) parts.ml[pr] = make_float2(mm, l);
          else if (c.lse) c.lse[(int64_t)(q0 + tok) * st.Hq + head] = l == 0.f ? -INFINITY : (mm + log2f(l)) * kLn2;
        }
        if (!two) {  // O may be written again
          tc::fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[kBOFree]);
        }
      }
      par = (par + (nj << two)) & 1;
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[kBPieceFree + at]);
      if (++at == kPieces) at = 0, pph ^= 1;
    }
    if (tid == 0 && rec_n == 0) parts.rec[b].n = 0;
  } else if (warp <= kPvWarp) {
    // ================= MMA issue: the whole warp walks the jobs, one elected lane issues.  Operands of an MMA come from
    // uniform registers: what they derive from is read from one lane, so that the compiler knows it to be uniform (moved
    // there one by one they cost as much as the products).
    auto uniform = [](uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); };
    const uint32_t bars0 = uniform(smem_u32(bars)), tm = uniform(tmem);
    Walk<C::kRows, C::kOver> w0;
    walk_start(w0, c, p, tiles, t0, t1);
    Walk<C::kRows, C::kOver> w = w0;
    Jobs jb{};
    jb.take(w);
    uint32_t slot = 0, sph = 0, buf = 0, g = 0;  // next ring slot and its phase, buffer of S and P, job
    if (warp == kQkWarp) {
      constexpr uint32_t kId = tc::idesc_f16(kBf, 128, false);
      const uint32_t q0 = uniform(smem0), r0 = uniform(kring);
      uint32_t first = 0, seg_ph = 0;
#pragma unroll 1
      for (; jb.live; ++g, buf ^= 1) {  // S = Q K^T
        bool ok = true;
        if (jb.i == 0) {
          ok = wait_all(kBQFull, seg_ph);
          seg_ph ^= 1;
        }
        if (jb.first_of_tile()) {
          first = slot;
          if (C::kTileSlots == 1) {
            ok = ok && wait_all(kBKFull + (int)slot, sph);
            if (++slot == C::kKSlots) slot = 0, sph ^= 1;
          }
        }
        const uint32_t x = uniform(jb.row_tile()), b_ = uniform(buf), end = uniform(jb.i == jb.n - 1),
                       last = uniform(jb.last_of_tile()), f = uniform(first);
        if (g >= 2) ok = ok && wait_all(kBBuf + (int)buf, (g >> 1) + 1 & 1);  // P of job g - 2 has been read
        if (!ok) break;
        tc::fence_after();
#pragma unroll
        for (int v = 0; v < C::kTileSlots; ++v) {
          const uint32_t sl = f + v >= C::kKSlots ? f + v - C::kKSlots : f + v;
          if (C::kTileSlots > 1) {  // slot by slot: one row tile, so each is used once
            if (!(ok = wait_all(kBKFull + (int)slot, sph))) break;
            if (++slot == C::kKSlots) slot = 0, sph ^= 1;
            tc::fence_after();
          }
          if (tc::elect_one()) {
#pragma unroll
            for (int u = 0; u < C::kSlotU; ++u) {
              const uint64_t a = tc::desc_sw128(q0 + (x * C::kU + v * C::kSlotU + u) * kUnitBytes, 0),
                             bd = tc::desc_sw128(r0 + sl * C::kSlotBytes + u * kUnitBytes, 0);
#pragma unroll
              for (int k = 0; k < 4; ++k)  // 16 elements: 32 bytes along the rows
                tc::mma_ss(tm + kColS + b_ * 128, a + k * 2, bd + k * 2, kId, v + u + k > 0);
            }
            if (v == C::kTileSlots - 1) {
              tc::commit(bars0 + (kBS + x * 2 + b_) * 8);
              if (end) tc::commit(bars0 + kBQFree * 8);
            }
            if (last) tc::commit(bars0 + (kBKFree + sl) * 8);
          }
          __syncwarp();
        }
        if (!ok) break;
        if (++jb.i == jb.n) {
          w.next(c, p);
          jb.take(w);
        }
      }
    } else {
      constexpr uint32_t kId = tc::idesc_f16(kBf, D == 64 ? 64 : 128, true);
      const uint32_t r0 = uniform(vring);
      uint32_t first = 0, pph = 0, oph = 0;  // pph: phases of the four P barriers, a bit each
      bool read_by_other = false;            // the last segment's O is read by warpgroup 1 while this one's P is formed
#pragma unroll 1
      for (; jb.live; ++g, buf ^= 1) {  // O += P V
        bool ok = true;
        if (jb.first_of_tile()) {
          first = slot;
          if (C::kTileSlots == 1) {
            ok = wait_all(kBVFull + (int)slot, sph);
            if (++slot == C::kVSlots) slot = 0, sph ^= 1;
          }
        }
        if (jb.i == 0) {
          if (read_by_other) {
            ok = ok && wait_all(kBOFree, oph);
            oph ^= 1;
          }
          read_by_other = !jb.two;
        }
        const int pb = jb.row_tile() * 2 + (int)buf;
        const uint32_t x = uniform(jb.row_tile()), b_ = uniform(buf), acc = uniform(jb.i > jb.two), f = uniform(first);
        // two row tiles: only their last product is waited for (their next S is formed after it); one: each, the last by
        // warpgroup 1
        const uint32_t tell = uniform(!jb.two || jb.i + 2 >= jb.n), who = uniform(jb.two ? jb.row_tile() : jb.i == jb.n - 1), last = uniform(jb.last_of_tile());
        ok = ok && wait_all(kBP + pb, pph >> pb & 1);
        if (!ok) break;
        pph ^= 1u << pb;
        tc::fence_after();
#pragma unroll
        for (int v = 0; v < C::kTileSlots; ++v) {
          const uint32_t sl = f + v >= C::kVSlots ? f + v - C::kVSlots : f + v;
          if (C::kTileSlots > 1) {
            if (!(ok = wait_all(kBVFull + (int)slot, sph))) break;
            if (++slot == C::kVSlots) slot = 0, sph ^= 1;
            tc::fence_after();
          }
          const uint64_t bd = tc::desc_sw128(r0 + sl * C::kSlotBytes, kUnitBytes);
          if (tc::elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)  // 16 lines: two groups of eight
              tc::mma_ts(tm + kColO + x * D + v * 128, tm + kColS + b_ * 128 + k * 8, bd + k * (2048 >> 4), kId, acc | (k > 0));
          }
          __syncwarp();
          if (v == 0) {
            if (!(ok = wait_all(kBP2 + pb, pph >> pb & 1 ^ 1))) break;
            tc::fence_after();
          }
          if (tc::elect_one()) {
#pragma unroll
            for (int k = 4; k < 8; ++k)
              tc::mma_ts(tm + kColO + x * D + v * 128, tm + kColS + b_ * 128 + k * 8, bd + k * (2048 >> 4), kId, 1);
            if (v == C::kTileSlots - 1) {
              tc::commit(bars0 + (kBBuf + b_) * 8);
              if (tell) tc::commit(bars0 + (kBO + who) * 8);
            }
            if (last) tc::commit(bars0 + (kBVFree + sl) * 8);
          }
          __syncwarp();
        }
        if (!ok) break;
        if (++jb.i == jb.n) {
          w.next(c, p);
          jb.take(w);
        }
      }
    }
    // nothing may be in flight when the tensor memory is freed
    const int drain = kBDrain + warp - kQkWarp;
    if (tc::elect_one()) tc::commit(bars0 + drain * 8);
    __syncwarp();
    if (!mbar_wait(&bars[drain], 0, kDefaultWaitNs)) attn_report(st, kAttnTimeout);
  } else {
    // ================= copies: warp kKWarp Q and K, the next one V
    const bool is_k = warp == kKWarp;
    const uint32_t bars0 = smem_u32(bars), ring = is_k ? kring : vring;
    const int full = is_k ? kBKFull : kBVFull, empty = is_k ? kBKFree : kBVFree, slots = is_k ? C::kKSlots : C::kVSlots;
    const CUtensorMap* tm = is_k ? &maps.k : &maps.v;
    const T* cache = static_cast<const T*>(is_k ? c.k : c.v);
    const int n_box = c.box ? kKeys / c.box : 0;
    int slot = 0, pending = -1;         // pending: barrier of the cp.async copies that are not announced yet
    uint32_t sph = 1, seg_ph = 1;       // parities of "it is free" (at first it is)
    uint32_t tx = 0;                    // slots that TMA has been asked to fill last
    bool ok = true;
    auto announce = [&](bool last) {  // the copies of the pending barrier, once they have landed (last: the newest group's)
      if (pending < 0) return;
      if (last) asm volatile("cp.async.wait_group 0;" ::: "memory");
      else asm volatile("cp.async.wait_group 1;" ::: "memory");
      tc::fence_proxy();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[pending]);
      pending = -1;
    };
    auto wait_free = [&](int bar, uint32_t parity) -> bool {  // no copy stays unannounced while this warp sleeps
      if (__all_sync(0xffffffffu, mbar_try_wait(&bars[bar], parity))) return true;
      announce(true);
      return wait_all(bar, parity);
    };
    auto copied = [&](int bar) {
      asm volatile("cp.async.commit_group;" ::: "memory");
      announce(false);
      pending = bar;
    };
    Walk<C::kRows, C::kOver> w0;
    walk_start(w0, c, p, tiles, t0, t1);
    Walk<C::kRows, C::kOver> w = w0;
    int told = 0;
    uint32_t tph = 1;
    auto tell = [&]() -> bool {  // the softmax what comes
      if (!wait_free(kBPieceFree + told, tph)) return false;
      if (lane == 0) {
        tail.piece[told].take(w);
        mbar_arrive(&bars[kBPiece + told]);
      }
      __syncwarp();
      if (++told == kPieces) told = 0, tph ^= 1;
      return true;
    };
#pragma unroll 1
    for (; w.more && ok; w.next(c, p)) {
      if (is_k && !(ok = tell())) break;
      if (is_k) {  // the segment's rows of q
        if (!(ok = wait_free(kBQFree, seg_ph))) break;
        seg_ph ^= 1;
        if (c.q_box) {
          const int n = (w.two + 1) * C::kU;
          announce(true);
          if (lane == 0) mbar_arrive_tx(&bars[kBQFull], n * kUnitBytes);
          __syncwarp();
          if (lane < n)
            tma_load_3d(smem0 + lane * kUnitBytes, &maps.q, lane % C::kU * 64, w.h * st.G,
                        w.q0 + (w.qt * C::kRows + lane / C::kU * 128) / st.G, bars0 + kBQFull * 8);
        } else {
          const int n = 2 * (w.two + 1) * C::kU;  // halves of units
#pragma unroll 1
          for (int v = 0; v < n; ++v) {
            const int x = (v >> 1) / C::kU, u = (v >> 1) % C::kU;
            int64_t at[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int r = x * 128 + (v & 1) * 64 + i * 32 + lane, R = w.qt * C::kRows + r;
              at[i] = r < w.rows ? (int64_t)(w.q0 + R / st.G) * c.q_stride + (int64_t)(w.h * st.G + R % st.G) * D : -1;
            }
            copy_lines<T>(smem0 + (uint32_t)v * (kUnitBytes / 2), static_cast<const T*>(c.q) + u * 64, at[0], at[1]);
          }
          copied(kBQFull);
          announce(true);
        }
      }
      const int lo0 = vis_lo(c, w.len - w.n);  // the sequence's first line that any token of the step sees
      const int un = lane / max(n_box, 1), bx = lane - un * n_box;  // TMA: this lane's box bx of unit un of a slot
#pragma unroll 1
      for (int j = w.j0; j < w.j1 && ok; ++j) {
        const int k0 = w.start + j * kKeys;
        // TMA where all the tile's lines are the sequence's, and seen by some token of the step
        const bool tma = n_box && k0 >= lo0 && k0 + kKeys <= w.len;
        int page = 0, line = 0;
        int64_t at[4] = {-1, -1, -1, -1};
        if (tma) {
          if (un < C::kSlotU) {
            const int l0 = k0 + bx * c.box, pi = (int)fast_div((uint32_t)l0, st.page_mul, st.page_shift);
            const int raw = __ldg(st.pages + (int64_t)w.s * st.pages_per_seq + pi);
            page = min(max(raw, 0), st.n_pages - 1);
            if (page != raw) attn_report(st, kAttnRange);
            line = l0 - pi * st.page_size;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int l0 = k0 + i * 32 + lane;
            if (l0 >= lo0 && l0 < w.end) at[i] = line_offset(st, w.s, l0) + (int64_t)w.h * st.head_stride;
          }
        }
#pragma unroll 1
        for (int u = 0; u < C::kTileSlots; ++u) {
          if (!(ok = wait_free(empty + slot, sph))) break;
          const uint32_t dst = ring + slot * C::kSlotBytes;
          if (tma) {
            if (lane == 0) mbar_arrive_tx(&bars[full + slot], C::kSlotBytes);
            __syncwarp();
            if (un < C::kSlotU)
              tma_load_4d(dst + un * kUnitBytes + bx * c.box * 128, tm, (u * C::kSlotU + un) * 64, w.h, line, page,
                          bars0 + (full + slot) * 8);
            tx |= 1u << slot;
          } else {
#pragma unroll 1
            for (int x = 0; x < 2 * C::kSlotU; ++x)
              copy_lines<T>(dst + x * (kUnitBytes / 2), cache + (u * C::kSlotU + (x >> 1)) * 64, at[x & 1 ? 2 : 0], at[x & 1 ? 3 : 1]);
            copied(full + slot);
            tx &= ~(1u << slot);
          }
          if (++slot == slots) slot = 0, sph ^= 1;
        }
      }
    }
    if (is_k && ok) tell();  // the end
    announce(true);
    asm volatile("cp.async.wait_all;" ::: "memory");
    // no copy may be in flight when the block exits: the MMA warps have waited for every slot they used, and use all unless a
    // wait gave up; then the slots' last phases are waited for here (the one before `slot` was filled in this turn)
    if (!ok)
      for (int i = 0; i < slots; ++i)
        if (tx >> i & 1) mbar_wait(&bars[full + i], i < slot ? sph ^ 1 : sph, kDefaultWaitNs);
  }
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  if (warp == kQkWarp) tc::dealloc(tmem, kTmemCols);
}

template <class T, int D>
cudaError_t run(const AttnCall& c, const AttnMaps& maps, AttnPlan plan, const AttnParts& parts, int sms, cudaStream_t s) {
  using C = Cfg<D>;
  const int64_t rows = (int64_t)c.st.n_tokens * c.st.G;
  const int64_t tiles = rows / C::kRows + c.st.n_seqs;
  plan.max_tiles = tiles < plan.max_tiles ? (int)tiles : plan.max_tiles;
  const int64_t most = tiles * c.st.Hkv * (((int64_t)c.st.cap + kKeys - 1) / kKeys);
  const unsigned grid = (unsigned)(most < sms ? most : sms);
  constexpr size_t smem = C::kTail + sizeof(Tail);
  static_assert(smem <= 232448, "shared memory of a block");
  cudaError_t e = cudaFuncSetAttribute(k_attn_many<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) e = launch_pdl(true, k_attn_plan<D>, dim3(1), dim3(1024), 0, s, c, plan);
  if (e == cudaSuccess) e = launch_pdl(true, k_attn_many<T, D>, dim3(grid), dim3(kThreads), smem, s, c, maps, plan, parts);
  if (e == cudaSuccess && grid > 1) e = launch_attn_join(c, parts, D, Half2<T>::kBf16, C::kRows, true, (int)grid, s);
  return e;
}

}  // namespace

void attn_maps(AttnCall& c, int head_dim, AttnMaps* maps) {
  using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const EncodeTiled encode = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
    return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiled>(fn) : nullptr;
  }();
  memset(maps, 0, sizeof(*maps));
  c.box = c.q_box = 0;
  const AttnStep& st = c.st;
  if (!encode) return;
  auto make = [&](CUtensorMap* tm, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
                  const cuuint32_t* box) {
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    return encode(tm, CU_TENSOR_MAP_DATA_TYPE_UINT16, rank, const_cast<void*>(base), dims, strides, box, ones,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  const cuuint64_t d = (cuuint64_t)head_dim;
  int box = kKeys;
  while (st.page_size % box) box /= 2;
  if (box >= 8) {
    const cuuint64_t dims[4] = {d, (cuuint64_t)st.Hkv, (cuuint64_t)st.page_size, (cuuint64_t)st.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)st.head_stride * 2, (cuuint64_t)st.token_stride * 2, (cuuint64_t)st.page_stride * 2};
    const cuuint32_t boxes[4] = {64, 1, (cuuint32_t)box, 1};
    if (make(&maps->k, c.k, 4, dims, strides, boxes) && make(&maps->v, c.v, 4, dims, strides, boxes)) c.box = box;
  }
  if (128 % st.G == 0) {  // a row tile is the group's heads of 128 / G tokens
    const cuuint64_t dims[3] = {d, (cuuint64_t)st.Hq, (cuuint64_t)st.n_tokens};
    const cuuint64_t strides[2] = {d * 2, (cuuint64_t)c.q_stride * 2};
    const cuuint32_t boxes[3] = {64, (cuuint32_t)st.G, (cuuint32_t)(128 / st.G)};
    c.q_box = make(&maps->q, c.q, 3, dims, strides, boxes);
  }
}

int attn_tile_rows(int head_dim) { return head_dim == 256 ? 128 : 256; }

cudaError_t launch_attn_many(const AttnCall& c, const AttnMaps& maps, const AttnPlan& plan, const AttnParts& parts, int head_dim, bool bf16, int sms,
                             cudaStream_t s) {
  if (bf16)
    return head_dim == 64    ? run<__nv_bfloat16, 64>(c, maps, plan, parts, sms, s)
           : head_dim == 128 ? run<__nv_bfloat16, 128>(c, maps, plan, parts, sms, s)
                             : run<__nv_bfloat16, 256>(c, maps, plan, parts, sms, s);
  return head_dim == 64    ? run<__half, 64>(c, maps, plan, parts, sms, s)
         : head_dim == 128 ? run<__half, 128>(c, maps, plan, parts, sms, s)
                           : run<__half, 256>(c, maps, plan, parts, sms, s);
}

}  // namespace mf

// Internal declarations of the paged attention operators (not part of the C ABI).
#pragma once

#include <cuda_bf16.h>

#include "mf_internal.cuh"

namespace mf {

// Bits of a handle's error word.
constexpr unsigned kAttnRange = 1u, kAttnTimeout = 2u;

// A step and the cache it works on, as the kernels take them (by value).
struct AttnStep {
  const int32_t *q_start, *kv_len, *pages;
  int n_seqs, n_tokens, max_q, pages_per_seq;
  int page_size, n_pages, cap;  // cap: lines a sequence's pages can hold
  uint32_t page_mul, page_shift;  // line / page_size = (line * page_mul) >> (32 + page_shift), see fast_div
  int64_t page_stride, token_stride, head_stride;
  int Hq, Hkv, G;
  unsigned* err;
};

// n / d for 0 <= n < 2^31 from a multiplier chosen on the host (Granlund and Montgomery, 1994: m = ceil(2^(32+l) / d)
// with 2^l >= d fits 33 bits; its low 32 bits are kept and the top one added back by the sum below).
struct FastDiv {
  uint32_t mul, shift;
};
__host__ __device__ __forceinline__ uint32_t mulhi_u32(uint32_t a, uint32_t b) {
#ifdef __CUDA_ARCH__
  return __umulhi(a, b);
#else
  return (uint32_t)(((uint64_t)a * b) >> 32);
#endif
}
inline FastDiv make_fast_div(uint32_t d) {
  uint32_t l = 0;
  while (l < 31 && (1u << l) < d) ++l;
  const uint64_t m = ((uint64_t(1) << 32) * ((uint64_t(1) << l) - d)) / d + 1;
  return {(uint32_t)m, l};
}
__host__ __device__ __forceinline__ uint32_t fast_div(uint32_t n, uint32_t mul, uint32_t shift) {
  return (uint32_t)(((uint64_t)mulhi_u32(n, mul) + n) >> shift);
}

// One sequence's part of the step: its new tokens q0 .. q0 + n - 1 of the step, its lines in the cache.
struct SeqSpan {
  int q0, n, len;
};

__device__ __forceinline__ void attn_report(const AttnStep& a, unsigned bit) { atomicOr(a.err, bit); }

__device__ __forceinline__ SeqSpan seq_span(const AttnStep& a, int s) {
  int b = s, e = s + 1;
  if (a.q_start) b = __ldg(a.q_start + s), e = __ldg(a.q_start + s + 1);
  const int len0 = __ldg(a.kv_len + s);
  const int q0 = min(max(b, 0), a.n_tokens), q1 = min(max(e, q0), a.n_tokens);
  SeqSpan r = {q0, min(q1 - q0, a.max_q), min(max(len0, 0), a.cap)};
  // (tokens before the first sequence's or after the last one's are nobody's)
  const bool nobodys = (s == 0 && b != 0) || (s + 1 == a.n_seqs && e != a.n_tokens);
  if (r.q0 != b || r.q0 + r.n != e || r.len != len0 || r.len < r.n || nobodys) attn_report(a, kAttnRange);
  return r;
}

// Element offset of line c of sequence s in the cache (head 0); a page outside the pool is taken as the nearest.
__device__ __forceinline__ int64_t line_offset(const AttnStep& a, int s, int c) {
  const int pi = (int)fast_div((uint32_t)c, a.page_mul, a.page_shift);
  const int raw = __ldg(a.pages + (int64_t)s * a.pages_per_seq + pi), page = min(max(raw, 0), a.n_pages - 1);
  if (page != raw) attn_report(a, kAttnRange);
  return (int64_t)page * a.page_stride + (int64_t)(c - pi * a.page_size) * a.token_stride;
}

// Groups of sequences that share their first lines (mf_shared_t).
struct SharedGroups {
  const int32_t *first, *len;
  int n;
};

// An attention call.
struct AttnCall {
  AttnStep st;
  const void *k, *v, *q;
  void* out;
  float* lse;
  int64_t q_stride, out_stride;
  float scale;
  int window, causal;
  int box;  // lines of a tensor-map box (mf_attn_many.cu): a power of two that divides the page; 0: no tensor maps
  int q_box;  // Q has a tensor map
  SharedGroups look;  // groups that are looked at (are bounds and lengths in range?) and not used; n = 0: none
};

// The caches as 4-D tensors (element, head, line, page), boxes of 64 elements x `box` lines, 128-byte swizzled.
// Q as a 3-D tensor (element, head, token), boxes of 64 elements x a group's heads x 128 / G tokens.
struct AttnMaps {
  CUtensorMap k, v, q;
};

// An append of new tokens.
struct AppendCall {
  AttnStep st;
  const void *q, *k, *v;
  void *q_out, *kc, *vc;
  int64_t q_stride, k_stride, v_stride, q_out_stride;
  const float *cos, *sin;
  const int32_t* pos;
  int n_pos, half, interleaved, n_axes;  // half = rot_dim / 2 (0: no rotation)
  int end0, end1, end2;  // first pair after axes 0, 1, 2
};
// Norms that come before the rotation: weights [head_dim] (of the caches' type, or float where f32 is set; null: that one is not
// normed), to which `offset` is added.
struct AppendNorm {
  const void *q_weight, *k_weight;
  float eps, offset;
  int f32;
};

// The lines [lo, hi) that the token at line `pos` of a sequence of `len` lines sees.
__device__ __forceinline__ int vis_lo(const AttnCall& c, int pos) { return c.window > 0 ? max(0, pos - c.window + 1) : 0; }
__device__ __forceinline__ int vis_hi(const AttnCall& c, int pos, int len) { return c.causal ? min(len, pos + 1) : len; }

// The two 16-bit types.
template <class T>
struct Half2;
template <>
struct Half2<__half> {
  static constexpr bool kBf16 = false;
  static __device__ __forceinline__ float2 up(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
  static __device__ __forceinline__ uint32_t down(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <>
struct Half2<__nv_bfloat16> {
  static constexpr bool kBf16 = true;
  static __device__ __forceinline__ float2 up(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint32_t down(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

// A (sequence, kv head)'s rows that several blocks share: `rows` of them from row0 on (row r: token q0 + r / G of the
// step, head r % G of kv head h's group), in n pieces of successive blocks (0: none starts here).
struct AttnRec {
  int q0, h, row0, rows, n;
};
// What blocks leave of work that they do not have whole.  Block b's last piece, where it starts the work, is part
// 2b + 1 and rec[b] describes it; the pieces that go on with it are parts 2(b + 1), 2(b + 2), ...
struct AttnParts {
  float* o;     // [parts][rows][head_dim] (few rows) or [parts][head_dim / 4][rows][4] (tiles), not yet divided by l
  float2* ml;   // [parts][rows]  running maximum (log2 domain) and sum
  AttnRec* rec;  // [blocks]
  // Of a step whose groups share lines, what blocks have whole of the groups' rows and then of the sequences', each [kv heads][tokens *
  // heads of a group]: o of a row tile as [head_dim / 4][its rows][4] where its rows begin.
  float* whole;
  float2* whole_ml;
};
constexpr int kMaxParts = 1024; // pieces of one record
int attn_few_blocks(int sms);
int attn_few_rows(int head_dim);   // the most rows (token, head of the group) that launch_attn_few takes: rows of a part
int attn_tile_rows(int head_dim);  // rows of a part of launch_attn_many (one block per SM)

// What k_attn_plan finds of a step for launch_attn_many: the row tiles of the sequences and the jobs before each.
struct AttnPlan {
  int* first;       // [max_seqs + 1]  first row tile of a sequence; then the number of tiles
  int4* tile;       // [max_tiles][2]  its sequence, that one's first new token, new tokens and lines; its place among the
                    //                 sequence's tiles, rows, first and end of the lines that any of them sees
  int64_t* before;  // [max_tiles + 1] jobs (of one kv head) before the tile
  int max_tiles;
  // of a step whose groups share lines: the virtual sequences of the list, groups and then sequences, and for each row tile and kv
  // head the block that has its first key tile and how many have one
  int groups, seqs;
  int2* runs;       // [max_tiles][kv heads]
  // where each block begins: {row tile, kv head, blocks that have work, -}, {place of the tile's segment, beginning of the share}, {its end, all}
  longlong2* start;  // [blocks][3]
};

// What k_attn_plan_shared finds of groups of sequences that share their first lines.
struct SharedPlan {
  int* bound;   // [max_groups + 1] first sequence of a group
  int4* group;  // [max_groups]     that, its first token, tokens (0: nothing is shared), lines that are shared
  int2* seq;    // [2][max_seqs]    a sequence's group (-1: none), the lines it shares, for each of the plan's blocks
  // for the join: a sequence's first token and tokens, its group's; the group's place in the list of few rows or its first row tile,
  // its row tiles
  int4* join;   // [max_seqs][2]
  // the list of launch_attn_few_shared: a (virtual) sequence's first new token, new tokens, end and beginning of its lines; the
  // places before it; for each and a kv head the block that has its first tile and how many have one
  int4* span;       // [max_groups + max_seqs]
  int64_t* before;  // [max_groups + max_seqs + 1]
  int2* runs;       // [max_groups + max_seqs][kv heads]
  // where its blocks begin: {sequence, kv head, row of the page table, blocks that have work}, its span, {place, beginning of the share}, {its
  // end, all}
  int4* start;      // [blocks][4]
};
// A step whose groups share lines, as launch_attn_few_shared takes it.
struct FewShared {
  const int4 *span, *group, *start;
  int2* runs;
  int groups;  // virtual sequences before the step's
  int wait;    // the kernel before this one is the plan
  int blocks;
};
constexpr int kFewTile = 64, kFewOver = 3;  // lines of a tile, tiles that a (sequence, head) costs besides its own
// What mf_attn_share allots.
struct AttnShared {
  int max_groups;  // 0: it was not called
  unsigned char* mem;
  SharedPlan found;
  AttnPlan plan;
  AttnParts parts, few;  // of the two kernels, which may run side by side (what is whole: one place)
};
cudaError_t launch_append_norm(const AppendCall& c, const AppendNorm& n, int head_dim, bool bf16, cudaStream_t s);
int attn_few_part_rows(int rows);            // rows of a part of launch_attn_few_shared for that many rows
int attn_few_fit(int head_dim, int sms);     // its blocks that find room at once
cudaError_t launch_attn_few_shared(const AttnCall& c, const AttnParts& parts, const FewShared& shared, int rows, int head_dim, bool bf16,
                                   int sms, cudaStream_t s);
cudaError_t launch_attn_few(const AttnCall& c, const AttnParts& parts, int head_dim, bool bf16, int sms, cudaStream_t s);
// Fills `maps`, c.box and c.q_box where the cache and Q can be described so (0 where not).
void attn_maps(AttnCall& c, int head_dim, AttnMaps* maps);
cudaError_t launch_attn_many(const AttnCall& c, const AttnMaps& maps, const AttnPlan& plan, const AttnParts& parts, int head_dim, bool bf16, int sms,
                             cudaStream_t s);
cudaError_t launch_attn_shared(const AttnCall& c, const AttnMaps& maps, const SharedGroups& groups, const AttnShared& sh, int head_dim, bool bf16,
                               int sms, cudaStream_t s);
// Rows of a sequence, on the average, from which launch_attn_many does not gain by shared lines.
int attn_alone_rows(int head_dim);
cudaError_t launch_look(const AttnCall& c, cudaStream_t s);  // c.look, where no join does it
// the records of `blocks` blocks joined; rows: rows of a part; tiles: left by launch_attn_many
cudaError_t launch_attn_join(const AttnCall& c, const AttnParts& parts, int head_dim, bool bf16, int rows, bool tiles, int blocks,
                             cudaStream_t s);

}  // namespace mf

struct mf_attn {
  mf_attn_shape_t shape;
  int max_seqs, max_tokens, device;
  int sms;
  unsigned* err;  // device error word, at the workspace's start
  mf::AttnParts parts;
  mf::AttnPlan plan;
  mf::AttnShared shared;
};

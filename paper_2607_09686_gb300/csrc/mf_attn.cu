// Attention over a paged key/value cache: entry points, and the append of new tokens.  Declarations and
// contracts: mawforge.h.
#include <cmath>
#include <cstring>
#include <new>

#include "mf_attn.cuh"

namespace mf {
namespace {

// ---- append: q and k rotated by position, k and v into their lines
//
// A pair (a, b) turned by an angle is (a cos - b sin, b cos + a sin).  Every element is read and written once,
// so the kernel is a copy bounded by memory (few tokens: by its launch).  A block has kTB tokens (one where there are few
// tokens, four else, so that a thread has several loads under way): a warp finds a token's sequence (the ends at or before
// it are counted) and its line, the threads fetch the angles' cosines and sines once for all heads, then each takes pairs
// of 16-byte vectors of a head: the two halves of eight rotated pairs (elements j.. and j + rot / 2.., or 16 neighbours when
// interleaved), or 16 neighbours of what is only copied.  5366 tokens of 16 + 2 x 4 heads of 256: 29.6 us, 4.5 TB/s; one
// token: 2.6 to 2.8 us in a graph.
constexpr int kAppendThreads = 256;

template <class T, int kTB>
__global__ void __launch_bounds__(kAppendThreads) k_append(const __grid_constant__ AppendCall c, int D) {
  const AttnStep& st = c.st;
  __shared__ int64_t s_at[kTB];
  __shared__ int s_line[kTB];  // the token's line; -1: not stored
  __shared__ float2 s_cs[kTB][128];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, t0 = blockIdx.x * kTB, tokens = min(kTB, st.n_tokens - t0);
  pdl_wait();
  if (warp < tokens) {
    const int t = t0 + warp;
    int s = t;
    if (st.q_start) {
      s = 0;
      for (int base = 0; base < st.n_seqs; base += 32) {
        const int i = base + lane;
        s += __popc(__ballot_sync(0xffffffffu, i < st.n_seqs && __ldg(st.q_start + i + 1) <= t));
      }
    }
    if (lane == 0) {
      int line = -1;
      int64_t at = 0;
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
      if (line < 0) attn_report(st, kAttnRange);
      s_line[warp] = line;
      s_at[warp] = at;
    }
  }
  __syncthreads();
  if (c.half) {
    for (int i = tid; i < tokens * c.half; i += kAppendThreads) {
      const int k = i / c.half, pair = i - k * c.half;
      int p = s_line[k];
      if (c.pos) {
        const int axis = c.n_axes == 1 ? 0 : (pair >= c.end0) + (pair >= c.end1) + (pair >= c.end2);
        p = __ldg(c.pos + (int64_t)axis * st.n_tokens + t0 + k);
      }
      const int pc = min(max(p, 0), c.n_pos - 1);
      if (pc != p) attn_report(st, kAttnRange);
      s_cs[k][pair] = make_float2(__ldg(c.cos + (int64_t)pc * c.half + pair), __ldg(c.sin + (int64_t)pc * c.half + pair));
    }
    __syncthreads();
  }

  const int per = D / 16, q_heads = c.q ? st.Hq : 0, n_items = (q_heads + 2 * st.Hkv) * per;
  struct Item {
    T* dst;
    uint4 a, b;
    int e0, e1, k, j;  // elements of the two vectors; token, place in the head
    bool turn, ok;
  };
  auto load = [&](int i, Item& it) {
    it.ok = i < tokens * n_items;
    if (!it.ok) return;
    const int k = i / n_items, x = i - k * n_items, head = x / per, j = x - head * per, t = t0 + k;
    const bool is_q = head < q_heads, is_v = head >= q_heads + st.Hkv;
    const int h = is_q ? head : is_v ? head - q_heads - st.Hkv : head - q_heads;
    it.ok = is_q || s_line[k] >= 0;
    if (!it.ok) return;
    const T* src = static_cast<const T*>(is_q ? c.q : is_v ? c.v : c.k) +
                   (int64_t)t * (is_q ? c.q_stride : is_v ? c.v_stride : c.k_stride) + (int64_t)h * D;
    it.dst = is_q ? static_cast<T*>(c.q_out) + (int64_t)t * c.q_out_stride + (int64_t)h * D
                  : static_cast<T*>(is_v ? c.vc : c.kc) + s_at[k] + (int64_t)h * st.head_stride;
    it.turn = !is_v && j * 8 < c.half;
    it.e0 = it.turn && !c.interleaved ? j * 8 : j * 16, it.e1 = it.turn && !c.interleaved ? it.e0 + c.half : it.e0 + 8;
    it.k = k, it.j = j;
    it.a = *reinterpret_cast<const uint4*>(src + it.e0), it.b = *reinterpret_cast<const uint4*>(src + it.e1);
  };
  auto store = [&](Item& it) {
    if (!it.ok) return;
    if (it.turn) {
      uint32_t wa[4] = {it.a.x, it.a.y, it.a.z, it.a.w}, wb[4] = {it.b.x, it.b.y, it.b.z, it.b.w};
      const float2* cs = &s_cs[it.k][it.j * 8];
      if (c.interleaved) {  // words hold (a, b) of a pair
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float2 x = Half2<T>::up(wa[u]), y = Half2<T>::up(wb[u]), p = cs[u], q = cs[4 + u];
          wa[u] = Half2<T>::down(x.x * p.x - x.y * p.y, x.y * p.x + x.x * p.y);
          wb[u] = Half2<T>::down(y.x * q.x - y.y * q.y, y.y * q.x + y.x * q.y);
        }
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float2 x = Half2<T>::up(wa[u]), y = Half2<T>::up(wb[u]), p = cs[2 * u], q = cs[2 * u + 1];
          wa[u] = Half2<T>::down(x.x * p.x - y.x * p.y, x.y * q.x - y.y * q.y);
          wb[u] = Half2<T>::down(y.x * p.x + x.x * p.y, y.y * q.x + x.y * q.y);
        }
      }
      it.a = make_uint4(wa[0], wa[1], wa[2], wa[3]);
      it.b = make_uint4(wb[0], wb[1], wb[2], wb[3]);
    }
    *reinterpret_cast<uint4*>(it.dst + it.e0) = it.a;
    *reinterpret_cast<uint4*>(it.dst + it.e1) = it.b;
  };
  for (int i = tid; i < tokens * n_items; i += 2 * kAppendThreads) {  // both items' loads before the first store
    Item x, y;
    load(i, x);
    load(i + kAppendThreads, y);
    store(x);
    store(y);
  }
}

// ---- arguments

bool shape_ok(const mf_attn_shape_t* s) {
  return s && s->n_kv_heads >= 1 && s->n_heads >= s->n_kv_heads && s->n_heads <= 4096 && s->n_heads % s->n_kv_heads == 0 &&
         s->n_heads / s->n_kv_heads <= 128 && (s->head_dim == 64 || s->head_dim == 128 || s->head_dim == 256) &&
         (s->dtype == MF_F16 || s->dtype == MF_BF16);
}

bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }
bool bad_rows(const void* p, int64_t stride) { return !p || off16(p) || stride < 0 || stride % 8; }

// false where the cache or the step does not fit the handle
bool make_step(const mf_attn_t* h, const mf_kv_cache_t* c, const mf_step_t* t, AttnStep* st) {
  if (!h || !c || !t || !c->k || !c->v || off16(c->k) || off16(c->v)) return false;
  if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0 ||
      (c->page_stride | c->token_stride | c->head_stride) % 8 || c->n_pages < 1 || c->page_size < 1)
    return false;
  if (t->n_seqs < 0 || t->n_tokens < 0 || t->n_seqs > h->max_seqs || t->n_tokens > h->max_tokens) return false;
  if (t->n_tokens > 0 && (t->n_seqs < 1 || !t->kv_len || !t->pages || t->pages_per_seq < 1 || t->max_q < 1)) return false;
  if (!t->q_start && t->n_tokens != t->n_seqs) return false;
  st->q_start = t->q_start;
  st->kv_len = t->kv_len;
  st->pages = t->pages;
  st->n_seqs = t->n_seqs;
  st->n_tokens = t->n_tokens;
  st->max_q = t->max_q < t->n_tokens ? t->max_q : t->n_tokens;
  st->pages_per_seq = t->pages_per_seq;
  st->page_size = c->page_size;
  st->n_pages = c->n_pages;
  const int64_t cap = (int64_t)t->pages_per_seq * c->page_size;
  st->cap = cap < (1 << 30) ? (int)cap : 1 << 30;
  const FastDiv fd = make_fast_div((uint32_t)c->page_size);
  st->page_mul = fd.mul;
  st->page_shift = fd.shift;
  st->page_stride = c->page_stride;
  st->token_stride = c->token_stride;
  st->head_stride = c->head_stride;
  st->Hq = h->shape.n_heads;
  st->Hkv = h->shape.n_kv_heads;
  st->G = st->Hq / st->Hkv;
  st->err = h->err;
  return true;
}

struct Carve {  // places in one allocation
  size_t off = 0;
  size_t take(size_t bytes) {
    const size_t o = off;
    off = (off + bytes + 255) & ~size_t(255);
    return o;
  }
};

struct OnDevice {
  int prev = -1;
  bool ok;
  explicit OnDevice(int dev) {
    ok = cudaGetDevice(&prev) == cudaSuccess && (prev == dev || cudaSetDevice(dev) == cudaSuccess);
    if (prev == dev) prev = -1;
  }
  ~OnDevice() {
    if (prev >= 0) cudaSetDevice(prev);
  }
};

}  // namespace
}  // namespace mf

using namespace mf;

extern "C" int mf_kv_bytes(const mf_attn_shape_t* shape, int n_layers, int64_t n_tokens, int page_size, uint64_t* out) {
  if (!shape_ok(shape) || !out || n_layers < 1 || n_tokens < 0 || page_size < 1) return MF_E_INVAL;
  const uint64_t pages = ((uint64_t)n_tokens + (uint64_t)page_size - 1) / (uint64_t)page_size;
  const unsigned __int128 b = (unsigned __int128)pages * (unsigned)page_size * 4u * (unsigned)shape->n_kv_heads *
                              (unsigned)shape->head_dim * (unsigned)n_layers;
  if (b >> 64) return MF_E_INVAL;
  *out = (uint64_t)b;
  return MF_OK;
}

extern "C" int mf_attn_create(mf_attn_t** out, const mf_attn_shape_t* shape, int max_seqs, int max_tokens, int device) {
  if (!out) return MF_E_INVAL;
  *out = nullptr;
  if (!shape_ok(shape) || max_seqs < 1 || max_tokens < 1 || device < 0) return MF_E_INVAL;
  if ((int64_t)max_tokens * (shape->n_heads / shape->n_kv_heads) > (1 << 30)) return MF_E_INVAL;  // rows are counted in 32 bits
  OnDevice on(device);
  if (!on.ok) return cuda_fail(cudaGetLastError(), "cudaSetDevice");
  mf_attn_t* h = new (std::nothrow) mf_attn_t();
  if (!h) return MF_E_OOM;
  h->shape = *shape;
  h->max_seqs = max_seqs;
  h->max_tokens = max_tokens;
  h->device = device;
  cudaError_t e = cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, device);
  // parts of either path (a step takes one): rows of a part times parts
  const int G = shape->n_heads / shape->n_kv_heads, tile = attn_tile_rows(shape->head_dim);
  const size_t few = (size_t)attn_few_blocks(h->sms) * 2 * attn_few_rows(shape->head_dim);
  const size_t many = (int64_t)max_tokens * G > attn_few_rows(shape->head_dim) ? (size_t)h->sms * 2 * tile : 0;
  const size_t rows = few > many ? few : many, tiles = (size_t)((int64_t)max_tokens * G / tile) + max_seqs;
  Carve w;
  const size_t o_err = w.take(256), o_o = w.take(rows * shape->head_dim * 4), o_ml = w.take(rows * 8),
               o_rec = w.take((size_t)attn_few_blocks(h->sms) * sizeof(AttnRec)), o_first = w.take(((size_t)max_seqs + 1) * 4),
               o_tile = w.take(tiles * 32), o_before = w.take((tiles + 1) * 8);
  unsigned char* ws = nullptr;
  if (e == cudaSuccess) e = tiles < (1u << 30) ? cudaMalloc(&ws, w.off) : cudaErrorMemoryAllocation;
  h->err = reinterpret_cast<unsigned*>(ws + o_err);
  h->parts = {reinterpret_cast<float*>(ws + o_o), reinterpret_cast<float2*>(ws + o_ml), reinterpret_cast<AttnRec*>(ws + o_rec), nullptr, nullptr};
  h->plan = {reinterpret_cast<int*>(ws + o_first), reinterpret_cast<int4*>(ws + o_tile), reinterpret_cast<int64_t*>(ws + o_before),
             (int)tiles, 0, 0, nullptr, nullptr};
  if (e == cudaSuccess) e = cudaMemset(h->err, 0, 256);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    const int rc = cuda_fail(e, "mf_attn_create");
    cudaGetLastError();
    cudaFree(h->err);
    delete h;
    return rc;
  }
  *out = h;
  return MF_OK;
}

namespace {

// The arguments of an append, but its norms, as the kernels take them; *work: there is something to do.
int make_append(const mf_attn_t* attn, const mf_kv_cache_t* cache, const mf_step_t* step, const mf_rope_t* rope,
                const mf_append_args_t* args, AppendCall* call, bool* work) {
  AppendCall& c = *call;
  memset(&c, 0, sizeof(c));
  *work = false;
  if (!args || !make_step(attn, cache, step, &c.st)) return MF_E_INVAL;
  const int D = attn->shape.head_dim;
  if (rope) {
    if (!rope->cos || !rope->sin || off16(rope->cos) || off16(rope->sin) || rope->n_pos < 1 || rope->rot_dim < 16 ||
        rope->rot_dim % 16 || rope->rot_dim > D || rope->n_axes < 1 || rope->n_axes > 4 || (rope->n_axes > 1 && !rope->pos))
      return MF_E_INVAL;
    c.half = rope->rot_dim / 2;
    int end[4] = {c.half, c.half, c.half, c.half}, at = 0;
    for (int a = 0; a < rope->n_axes && rope->n_axes > 1; ++a) {
      if (rope->section[a] < 0 || rope->section[a] > c.half - at) return MF_E_INVAL;
      end[a] = at += rope->section[a];
    }
    if (rope->n_axes > 1 && at != c.half) return MF_E_INVAL;
    c.end0 = end[0], c.end1 = end[1], c.end2 = end[2];
    c.cos = rope->cos, c.sin = rope->sin, c.pos = rope->pos;
    c.n_pos = rope->n_pos, c.interleaved = rope->interleaved != 0, c.n_axes = rope->n_axes;
  }
  if (c.st.n_tokens == 0) return MF_OK;
  if (bad_rows(args->k, args->k_stride) || bad_rows(args->v, args->v_stride) || !args->q != !args->q_out) return MF_E_INVAL;
  if (args->q && (bad_rows(args->q, args->q_stride) || bad_rows(args->q_out, args->q_out_stride))) return MF_E_INVAL;
  c.q = args->q, c.k = args->k, c.v = args->v, c.q_out = args->q_out, c.kc = cache->k, c.vc = cache->v;
  c.q_stride = args->q_stride, c.k_stride = args->k_stride, c.v_stride = args->v_stride, c.q_out_stride = args->q_out_stride;
  *work = true;
  return MF_OK;
}

}  // namespace

extern "C" int mf_kv_append(mf_attn_t* attn, const mf_kv_cache_t* cache, const mf_step_t* step, const mf_rope_t* rope,
                            const mf_append_args_t* args, void* stream) {
  AppendCall c;
  bool work;
  const int rc = make_append(attn, cache, step, rope, args, &c, &work);
  if (rc != MF_OK || !work) return rc;
  const int D = attn->shape.head_dim;
  OnDevice on(attn->device);
  if (!on.ok) return cuda_fail(cudaGetLastError(), "cudaSetDevice");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // Single tokens keep latency low; from some eight blocks an SM on there are blocks enough to give each more tokens (heads
  // of 256, one against four a block: 160 tokens 12.5 and 15.3 us, 600 14.8 and 16.0, 1200 17.8 and 15.9, 3000 26.8 and 22.0,
  // event to event).
  const int T = c.st.n_tokens;
  auto launch = [&](auto kernel, int tb) {
    return launch_pdl(true, kernel, dim3((unsigned)((T + tb - 1) / tb)), dim3(kAppendThreads), 0, s, c, D);
  };
  cudaError_t e;
  if (attn->shape.dtype == MF_BF16)
    e = T < 8 * attn->sms ? launch(k_append<__nv_bfloat16, 1>, 1) : launch(k_append<__nv_bfloat16, 4>, 4);
  else
    e = T < 8 * attn->sms ? launch(k_append<__half, 1>, 1) : launch(k_append<__half, 4>, 4);
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_kv_append");
}

extern "C" int mf_kv_append_norm(mf_attn_t* attn, const mf_kv_cache_t* cache, const mf_step_t* step, const mf_qk_norm_t* norm,
                                 const mf_rope_t* rope, const mf_append_args_t* args, void* stream) {
  AppendCall c;
  bool work;
  if (!attn || !norm || (norm->dtype != MF_F32 && norm->dtype != attn->shape.dtype) || off16(norm->q_weight) || off16(norm->k_weight) ||
      !(norm->eps >= 0x1p-100f) || !std::isfinite(norm->eps) || !std::isfinite(norm->offset))
    return MF_E_INVAL;
  const int rc = make_append(attn, cache, step, rope, args, &c, &work);
  if (rc != MF_OK || !work) return rc;
  const AppendNorm n = {norm->q_weight, norm->k_weight, norm->eps, norm->offset, norm->dtype == MF_F32};
  OnDevice on(attn->device);
  if (!on.ok) return cuda_fail(cudaGetLastError(), "cudaSetDevice");
  const cudaError_t e = launch_append_norm(c, n, attn->shape.head_dim, attn->shape.dtype == MF_BF16, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_kv_append_norm");
}

namespace {

// The arguments of an attention call as the kernels take them; *work: there is something to do.
int make_attn(const mf_attn_t* attn, const mf_kv_cache_t* cache, const mf_step_t* step, const mf_attn_args_t* args, AttnCall* call,
              bool* work) {
  AttnCall& c = *call;
  memset(&c, 0, sizeof(c));
  *work = false;
  if (!args || !make_step(attn, cache, step, &c.st) || args->window < 0 || !std::isfinite(args->scale) ||
      !(args->scale > 0.f))
    return MF_E_INVAL;
  if (c.st.n_tokens == 0) return MF_OK;
  if (bad_rows(args->q, args->q_stride) || bad_rows(args->out, args->out_stride) || ((uintptr_t)args->lse & 3)) return MF_E_INVAL;
  c.k = cache->k, c.v = cache->v, c.q = args->q, c.out = args->out, c.lse = args->lse;
  c.q_stride = args->q_stride, c.out_stride = args->out_stride;
  c.scale = args->scale, c.causal = args->causal != 0;
  // a window of 2^30 lines holds every line there can be, and the line it begins at is counted in 32 bits also from a
  // token whose own line would lie before the first (no more than 2^30 before it)
  c.window = args->window < (1 << 30) ? args->window : 1 << 30;
  *work = true;
  return MF_OK;
}

// Each sequence from its own pages.
cudaError_t each_alone(const mf_attn_t* attn, AttnCall& c, cudaStream_t s) {
  const int D = attn->shape.head_dim;
  const bool bf16 = attn->shape.dtype == MF_BF16;
  // (few rows: as many as their kernel's registers hold.  There it is the faster one, but for heads of 64 without a window.  16
  // sequences of 4093 lines and 8 heads a kv head, in a graph, few against many, with a window of 1024 and without: 48 rows of 64
  // 20.8 us against 31.1, 38.5 against 35.5; 32 rows of 128 21.7 against 33.2, 44.2 against 46.3; 16 rows of 256 24.2 against
  // 42.7, 62.2 against 70.7.  One token a sequence more goes to the other kernel: 40 rows of 128 34.0 and 48.4, 24 rows of 256 43.3 and
  // 71.9)
  if ((int64_t)c.st.max_q * c.st.G <= attn_few_rows(D)) return launch_attn_few(c, attn->parts, D, bf16, attn->sms, s);
  AttnMaps maps;
  attn_maps(c, D, &maps);
  return launch_attn_many(c, maps, attn->plan, attn->parts, D, bf16, attn->sms, s);
}

}  // namespace

extern "C" int mf_attn_forward(mf_attn_t* attn, const mf_kv_cache_t* cache, const mf_step_t* step,
                               const mf_attn_args_t* args, void* stream) {
  AttnCall c;
  bool work;
  const int rc = make_attn(attn, cache, step, args, &c, &work);
  if (rc != MF_OK || !work) return rc;
  OnDevice on(attn->device);
  if (!on.ok) return cuda_fail(cudaGetLastError(), "cudaSetDevice");
  const cudaError_t e = each_alone(attn, c, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_attn_forward");
}

extern "C" int mf_attn_share(mf_attn_t* attn, int max_groups) {
  if (!attn || max_groups < 1 || max_groups > (1 << 20)) return MF_E_INVAL;
  OnDevice on(attn->device);
  if (!on.ok) return cuda_fail(cudaGetLastError(), "cudaSetDevice");
  const mf_attn_shape_t& sh = attn->shape;
  const int64_t rows = (int64_t)attn->max_tokens * sh.n_heads, group_rows = rows / sh.n_kv_heads, tile = attn_tile_rows(sh.head_dim);
  const int64_t tiles = 2 * (group_rows / tile) + attn->max_seqs + max_groups, part_rows = (int64_t)attn->sms * 2 * tile;
  Carve w;
  const size_t o_bound = w.take(((size_t)max_groups + 1) * 4), o_group = w.take((size_t)max_groups * 16),
               o_seq = w.take((size_t)attn->max_seqs * 16), o_first = w.take(((size_t)attn->max_seqs + max_groups + 1) * 4),
               o_tile = w.take((size_t)tiles * 32), o_before = w.take(((size_t)tiles + 1) * 8),
               o_o = w.take((size_t)part_rows * sh.head_dim * 4), o_ml = w.take((size_t)part_rows * 8),
               o_few = w.take((size_t)attn_few_blocks(attn->sms) * 2 * attn_few_rows(sh.head_dim) * sh.head_dim * 4),
               o_few_ml = w.take((size_t)attn_few_blocks(attn->sms) * 2 * attn_few_rows(sh.head_dim) * 8),
               o_span = w.take(((size_t)max_groups + attn->max_seqs) * 16), o_fbefore = w.take(((size_t)max_groups + attn->max_seqs + 1) * 8),
               o_join = w.take((size_t)attn->max_seqs * 32), o_runs = w.take((size_t)tiles * sh.n_kv_heads * 8),
               o_fruns = w.take(((size_t)max_groups + attn->max_seqs) * sh.n_kv_heads * 8),
               o_start = w.take((size_t)attn->sms * 48), o_fstart = w.take((size_t)attn_few_blocks(attn->sms) * 64),
               o_whole = w.take((size_t)rows * 2 * sh.head_dim * 4), o_whole_ml = w.take((size_t)rows * 2 * 8);
  unsigned char* ws = nullptr;
  // (the join counts its vectors in 32 bits)
  cudaError_t e = tiles < (1 << 30) && w.off < ((size_t)1 << 36) ? cudaMalloc(&ws, w.off) : cudaErrorMemoryAllocation;
  // (runs that a step does not write, for lack of tiles where its bounds overlap, hold zeros or what an earlier step wrote: a wrong answer to a
  // step that is reported, from inside the workspace)
  if (e == cudaSuccess) e = cudaMemset(ws + o_runs, 0, (size_t)tiles * sh.n_kv_heads * 8);
  if (e == cudaSuccess) e = cudaMemset(ws + o_fruns, 0, ((size_t)max_groups + attn->max_seqs) * sh.n_kv_heads * 8);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    const int rc = cuda_fail(e, "mf_attn_share");
    cudaGetLastError();
    cudaFree(ws);
    return rc;
  }
  cudaFree(attn->shared.mem);
  AttnShared& a = attn->shared;
  a.max_groups = max_groups;
  a.mem = ws;
  a.found = {reinterpret_cast<int*>(ws + o_bound), reinterpret_cast<int4*>(ws + o_group), reinterpret_cast<int2*>(ws + o_seq),
             reinterpret_cast<int4*>(ws + o_join), reinterpret_cast<int4*>(ws + o_span), reinterpret_cast<int64_t*>(ws + o_fbefore),
             reinterpret_cast<int2*>(ws + o_fruns), reinterpret_cast<int4*>(ws + o_fstart)};
  a.plan = {reinterpret_cast<int*>(ws + o_first), reinterpret_cast<int4*>(ws + o_tile), reinterpret_cast<int64_t*>(ws + o_before),
            (int)tiles, 0, 0, reinterpret_cast<int2*>(ws + o_runs), reinterpret_cast<longlong2*>(ws + o_start)};
  a.parts = {reinterpret_cast<float*>(ws + o_o), reinterpret_cast<float2*>(ws + o_ml), nullptr, reinterpret_cast<float*>(ws + o_whole),
             reinterpret_cast<float2*>(ws + o_whole_ml)};
  a.few = {reinterpret_cast<float*>(ws + o_few), reinterpret_cast<float2*>(ws + o_few_ml), nullptr, a.parts.whole, a.parts.whole_ml};
  return MF_OK;
}

extern "C" int mf_attn_forward_shared(mf_attn_t* attn, const mf_kv_cache_t* cache, const mf_step_t* step, const mf_shared_t* shared,
                                      const mf_attn_args_t* args, void* stream) {
  AttnCall c;
  bool work;
  if (!shared || shared->n_groups < 0 || (shared->n_groups > 0 && (!shared->first || !shared->len)) ||
      (((uintptr_t)shared->first | (uintptr_t)shared->len) & 3))
    return MF_E_INVAL;
  const int rc = make_attn(attn, cache, step, args, &c, &work);
  if (rc != MF_OK) return rc;
  if (args->window) return MF_E_INVAL;
  if (!attn->shared.max_groups) return MF_E_STATE;
  if (shared->n_groups > attn->shared.max_groups) return MF_E_INVAL;
  if (!work) return MF_OK;
  OnDevice on(attn->device);
  if (!on.ok) return cuda_fail(cudaGetLastError(), "cudaSetDevice");
  const SharedGroups g = {shared->first, shared->len, shared->n_groups};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // Sharing costs a plan, a launch and a longer join.  Where all that the sequences' tables can hold is soon read (of lines that share pages
  // most come from the L2 cache), or the sequences have rows enough to fill tiles of their own (a group's tiles then spare no products
  // and hardly any reading, and the partials cost), each sequence reads all its lines itself, from its own pages, which hold the same.
  // Shared against alone, 4 kv heads with 8 heads each, in a graph: one token a sequence, 2 to 64 sequences, 66 MB 22 to 27 us and 20 to 22, 100
  // MB 24 to 30 and 21 to 25, 131 MB 25 to 29 and 25 to 29; heads of 64 17 MB 18 and 13, 99 MB 22 and 26.  8 sequences of 100 and
  // 8192 shared lines, rows of a sequence on the average: heads of 128, 58 32 us and 38, 77 40 and 39, 154 59 and 54; of 64, 77 52 and 51;
  // of 256, 77 52 and 55, 154 66 and 75, 3400 430 and 376.
  const int D = attn->shape.head_dim;
  const int64_t rows = (int64_t)c.st.n_tokens * c.st.G, held = (int64_t)c.st.n_seqs * c.st.cap * c.st.Hkv * D * 4;
  cudaError_t e;
  if (held <= (D == 64 ? 80 : 128) * (int64_t)1000000 ||
      ((int64_t)c.st.max_q * c.st.G > attn_few_rows(D) && rows >= (int64_t)attn_alone_rows(D) * c.st.n_seqs)) {
    c.look = g;
    e = each_alone(attn, c, s);
  } else {
    AttnMaps maps;
    attn_maps(c, D, &maps);
    e = launch_attn_shared(c, maps, g, attn->shared, D, attn->shape.dtype == MF_BF16, attn->sms, s);
  }
  return e == cudaSuccess ? MF_OK : cuda_fail(e, "mf_attn_forward_shared");
}

extern "C" int mf_attn_check(mf_attn_t* attn) {
  if (!attn) return MF_E_INVAL;
  OnDevice on(attn->device);
  unsigned err = 0;
  cudaError_t e = on.ok ? cudaDeviceSynchronize() : cudaGetLastError();
  if (e == cudaSuccess) e = cudaMemcpy(&err, attn->err, sizeof(err), cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && err) e = cudaMemset(attn->err, 0, sizeof(err));
  if (e == cudaSuccess && err) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return cuda_fail(e, "mf_attn_check");
  return err & kAttnTimeout ? MF_E_TIMEOUT : err ? MF_E_INVAL : MF_OK;
}

extern "C" void mf_attn_destroy(mf_attn_t* attn) {
  if (!attn) return;
  OnDevice on(attn->device);
  cudaDeviceSynchronize();
  cudaFree(attn->shared.mem);
  cudaFree(attn->err);
  delete attn;
}

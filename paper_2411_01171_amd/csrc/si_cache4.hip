// A cache of keys and values in 4 bits (see include/si.h): storing and reading back, attention over it, eviction from it.
// Checks, plans and launches.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "k_cache4.h"
#include "k_cache4_attn.h"
#include "k_cache4_evict.h"
#include "si_attn_ops.h"
#include "si_host.h"

namespace si {

static HeadsView view_of(const si_heads* t) { return HeadsView{t->ptr, t->stride_b, t->stride_n, t->stride_h}; }

static int cache_groups(const si_cache4* c) { return (int)((c->dim_head + 31) / 32); }
static int64_t code_bytes(const si_cache4* c) { return 16 * cache_groups(c); }
static int64_t scale_bytes(const si_cache4* c) { return cache4_scale_bytes(cache_groups(c)); }
static size_t cache_rows(const si_cache4* c) { return (size_t)(c->B * c->heads * c->capacity); }

static Cache4View view_of(const si_cache4* c) {
  return Cache4View{static_cast<uint8_t*>(c->k_codes), static_cast<uint8_t*>(c->k_scales), static_cast<uint8_t*>(c->v_codes),
                    static_cast<uint8_t*>(c->v_scales), (int)c->heads, (int)c->capacity};
}

// Memory that a call reads or writes, for the question whether two of them meet.
struct Span {
  const void* p;
  size_t bytes;
};
static bool meet(const Span& a, const Span& b) { return a.p && b.p && a.bytes && b.bytes && ranges_overlap(a.p, a.bytes, b.p, b.bytes); }
struct CacheSpans {
  Span s[4];
  explicit CacheSpans(const si_cache4* c)
      : s{{c->k_codes, cache_rows(c) * code_bytes(c)}, {c->k_scales, cache_rows(c) * scale_bytes(c)},
          {c->v_codes, cache_rows(c) * code_bytes(c)}, {c->v_scales, cache_rows(c) * scale_bytes(c)}} {}
  bool meets(const Span& o) const {
    for (const Span& x : s)
      if (meet(x, o)) return true;
    return false;
  }
  bool meets(const si_heads* t) const {
    for (const Span& x : s)
      if (x.p && heads_overlap_range(t, x.p, x.bytes)) return true;
    return false;
  }
};

// `written`: the four arrays must be apart.
static si_status check_cache(const si_cache4* c, bool written) {
  if (!c) return SI_ERR_NULL;
  if (c->B < 1 || c->heads < 1 || c->capacity < 0 || c->dim_head < 8 || c->dim_head > 128 || c->dim_head % 8) return SI_ERR_SHAPE;
  if (c->B > (1 << 24) || c->capacity > kMostTokens || c->heads > 65535 || c->B * c->heads > (1 << 28)) return SI_ERR_SHAPE;
  if ((double)(c->B * c->heads) * (double)c->capacity >= 1099511627776.0) return SI_ERR_SHAPE;  // 2^40 tokens
  if (c->capacity == 0) return SI_OK;
  for (const void* p : {c->k_codes, c->k_scales, c->v_codes, c->v_scales}) {
    if (!p) return SI_ERR_NULL;
    if (!aligned16(p)) return SI_ERR_ALIGN;
  }
  if (written) {
    const CacheSpans a(c);
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < i; ++j)
        if (meet(a.s[i], a.s[j])) return SI_ERR_ARG;
  }
  return SI_OK;
}

static bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Calls f(integral_constant<groups>).
template <class Fn>
static void by_groups(const si_cache4* c, Fn f) {
  switch (cache_groups(c)) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 3: f(std::integral_constant<int, 3>()); break;
    default: f(std::integral_constant<int, 4>()); break;
  }
}

// ----------------------------------------------------------------------------- storing and reading back

// k, v are heads of the cache's shape; `out`: they are written.
static si_status check_copy(const si_heads* k, const si_heads* v, const si_cache4* c, const int32_t* first, const int32_t* length,
                            const float* weight, bool out, int64_t* chunks) {
  si_status s = check_heads(k, out);
  if (s == SI_OK) s = check_heads(v, out);
  if (s == SI_OK) s = check_cache(c, !out);
  if (s != SI_OK) return s;
  if (v->dtype != k->dtype) return SI_ERR_DTYPE;
  for (const si_heads* t : {k, v})
    if (t->B != c->B || t->heads != c->heads || t->dim_head != c->dim_head || t->N != k->N) return SI_ERR_SHAPE;
  if (!aligned4(first) || !aligned4(length) || !aligned4(weight)) return SI_ERR_ALIGN;
  const int64_t tokens = kCache4Threads / (4 * cache_groups(c)) * kCache4Deep;
  *chunks = (k->N + tokens - 1) / tokens;
  if ((double)*chunks * (double)(c->B * c->heads) >= 4294967296.0 - kGridMost) return SI_ERR_SHAPE;
  const CacheSpans spans(c);
  const Span w{weight, cache_rows(c) * 4}, lens[] = {{first, (size_t)c->B * 4}, {length, (size_t)c->B * 4}};
  for (const si_heads* t : {k, v}) {
    if (spans.meets(t) || (w.p && heads_overlap_range(t, w.p, w.bytes))) return SI_ERR_ARG;
    for (const Span& l : lens)
      if (out && l.p && heads_overlap_range(t, l.p, l.bytes)) return SI_ERR_ARG;
  }
  if (out && !heads_apart(k, v)) return SI_ERR_ARG;
  if (spans.meets(w)) return SI_ERR_ARG;
  for (const Span& l : lens)
    if (!out && (spans.meets(l) || meet(w, l))) return SI_ERR_ARG;
  return SI_OK;
}

template <typename T>
static void launch_copy(const Cache4CopyArgs& a, const si_cache4* c, bool out, hipStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>(a.work, kGridMost);
  by_groups(c, [&](auto g) {
    if (out) cache4_load_kernel<T, g.value><<<grid, kCache4Threads, 0, st>>>(a);
    else cache4_store_kernel<T, g.value><<<grid, kCache4Threads, 0, st>>>(a);
  });
}

static si_status enqueue_copy(const si_heads* k, const si_heads* v, const si_cache4* c, const int32_t* first, const int32_t* length,
                              float* weight, bool out, int64_t chunks, hipStream_t st) {
  if (k->N == 0 || c->capacity == 0) return SI_OK;
  Cache4CopyArgs a;
  a.x[0] = view_of(k);
  a.x[1] = view_of(v);
  a.c = view_of(c);
  a.weight = weight;
  a.first = first;
  a.length = length;
  a.N = (int)k->N;
  a.d = (int)k->dim_head;
  a.chunks = (int)chunks;
  a.work = (unsigned)(chunks * c->B * c->heads);
  StageScope scope(out ? "cache4_load" : "cache4_store", st);
  if (k->dtype == SI_F32) launch_copy<float>(a, c, out, st);
  else launch_copy<bf16>(a, c, out, st);
  SI_CHECK_LAUNCH();
  return SI_OK;
}

// ----------------------------------------------------------------------------- attention

struct CachePlan {
  int group, tile_rows;  // query heads of a key head; rows of a tile: up to 32 by the few kernel, 128 and 256 (bfloat16) by the other
  int64_t runs, run_len, tiles_per_run, work, rows, weight_chunks;
  int weight_rows;  // that the weights' kernel keeps, or 0: it keeps keys
  int nsplit;
  size_t part_bytes, stat_bytes, row_bytes;
  size_t bytes() const { return part_bytes + stat_bytes + row_bytes + 256; }
};

// Into how many shares the keys of a tile are dealt out.
// Few rows: as many workgroups as the chip holds at once (`held` per CU), 256 keys at least to each; a third more than that took 110 us for one
// token of 32 heads against 115200 slots, and takes 99 so.
// Many: the busiest CU's number of workgroups bounds the time, and the shares cost their way through memory.  360 tiles on 256 CUs leave the
// busiest with 2 where the mean is 1.4 (9216 tokens of 5 heads over 64512 slots, two batch entries: 2214 us); in seven shares it has 10 of
// 9.8 (1639).  A workgroup alone on a CU is taken for three quarters of the time that two take, and 64 keys of a row and channel for
// cell_us: 0.073 ns, the rate of a whole chip's; float32's is 0.16, but its shares cost more at their beginnings, which 0.1 stands for (1500 tokens of 8 heads of
// 64 over 14000 slots: 120 us, with 0.16 136).
static int64_t shares_of_tiles(int64_t tiles, int tile_rows, int held, int64_t capacity, int64_t rows, int64_t d, double cell_us) {
  if (tiles == 0) return 1;
  const int64_t most = std::min<int64_t>(64, std::max<int64_t>(1, capacity / 256));
  if (tile_rows <= 32) return std::max<int64_t>(1, std::min<int64_t>(256 * held / tiles, most));
  int64_t best = 1;
  double least = 0.0;
  for (int64_t n = 1; n <= most && n * tiles <= 4096; ++n) {
    const double on_cu = (double)((tiles * n + 255) / 256);
    const double us = std::max(on_cu, 1.5) / (double)n * (double)((capacity + 63) / 64) * (double)(tile_rows * d) * cell_us +
                      (n > 1 ? 5.0 + (double)(rows * n) * (double)(d + 4) * 8.0 / 4e6 : 0.0);
    if (n == 1 || us < least) { least = us; best = n; }
  }
  return best;
}

static si_status plan_cache_attn(const si_heads* q, const si_cache4* c, int64_t run, bool weights, CachePlan* p) {
  si_status s = check_heads(q, false);
  if (s == SI_OK) s = check_cache(c, false);
  if (s != SI_OK) return s;
  if (q->B != c->B || q->dim_head != c->dim_head || q->heads % c->heads) return SI_ERR_SHAPE;
  if (run < 0 || run > kMostTokens) return SI_ERR_SHAPE;
  p->group = (int)(q->heads / c->heads);
  if ((double)p->group * (double)q->N >= 2147483648.0 - kGridMost) return SI_ERR_SHAPE;  // rows of a key head in 31 bits
  const int64_t rows_of_run = p->group * (run > 0 && run < q->N ? run : std::max<int64_t>(q->N, 1)), rows = p->group * std::max<int64_t>(q->N, 1);
  // float32 heads of 64, 8 of them over 30000 slots: 65 rows 30 us in tiles of 32, 33 in one of 128; 97 rows 35 and 33; 128 39 and 37.
  const bool many = rows > (q->dtype == SI_BF16 ? 64 : 96);
  p->tile_rows = !many ? (rows <= 16 ? 16 : 32) : q->dtype == SI_BF16 && cache_groups(c) <= 2 && rows > 128 ? 256 : 128;
  // A tile ends with its run, so that its rows see the same keys; runs shorter than a tile share them.
  const bool own = run > 0 && run < q->N && rows_of_run >= p->tile_rows;
  p->run_len = own ? run : std::max<int64_t>(q->N, 1);
  p->runs = q->N == 0 ? 0 : (q->N + p->run_len - 1) / p->run_len;
  p->tiles_per_run = (p->group * p->run_len + p->tile_rows - 1) / p->tile_rows;
  const int64_t lists = c->B * c->heads;
  const double tiles = (double)lists * (double)p->runs * (double)p->tiles_per_run;
  if (tiles >= 2147483648.0 - kGridMost) return SI_ERR_SHAPE;
  // The shares, and with them the workspace, do not depend on the runs.
  const int64_t whole = q->N == 0 ? 0 : lists * ((rows + p->tile_rows - 1) / p->tile_rows);
  const int groups = cache_groups(c), held = p->tile_rows == 32 ? (groups == 1 ? 3 : 2) : q->dtype == SI_BF16 ? (groups <= 2 ? 4 : 3) : groups == 1 ? 4 : groups == 2 ? 3 : 2;
  p->nsplit = (int)shares_of_tiles(whole, p->tile_rows, held, c->capacity, q->B * q->N * q->heads, q->dim_head, q->dtype == SI_BF16 ? 0.073e-3 : 0.1e-3);
  if (tiles * p->nsplit >= 2147483648.0 - kGridMost) return SI_ERR_SHAPE;
  p->work = (int64_t)tiles * p->nsplit;
  p->rows = q->B * q->N * q->heads;
  p->part_bytes = p->nsplit > 1 ? align_up((size_t)(p->rows * p->nsplit * q->dim_head) * 4, 256) : 0;
  p->stat_bytes = p->nsplit > 1 ? align_up((size_t)(p->rows * p->nsplit) * 16, 256) : 0;
  p->row_bytes = weights ? align_up((size_t)p->rows * 8, 256) : 0;
  // Weights: rows that fit operands are kept, and the keys dealt out like those of the attention (eight tokens of 32 heads, 57600 padded slots, all
  // of the call: 63 us with 768 workgroups, 65 with 512, 71 with 1024); otherwise keys are kept.
  p->weight_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 0;
  if (p->weight_rows) p->weight_chunks = std::min<int64_t>(std::max<int64_t>(1, 768 / lists), std::max<int64_t>(1, (c->capacity + 255) / 256));
  else p->weight_chunks = (c->capacity + 128 * kWeightTiles - 1) / (128 * kWeightTiles);
  if ((double)(c->B * c->heads) * (double)p->weight_chunks >= 4294967296.0 - kGridMost) return SI_ERR_SHAPE;
  return SI_OK;
}

static unsigned grid_of(int64_t work) { return (unsigned)((std::min<int64_t>(work, kGridMost) + 7) / 8 * 8); }

template <typename T>
static si_status launch_cache_attn(const CacheAttnArgs& a, const CacheWeightArgs* w, const si_cache4* c, const CachePlan& p, hipStream_t st) {
  if (p.work > 0) {
    StageScope scope("cache4_attn", st);
    const unsigned grid = grid_of(p.work);
    by_groups(c, [&](auto g) {
      if (p.tile_rows == 16) cache4_attn_few_kernel<T, g.value, 1><<<grid, 256, 0, st>>>(a);
      else if (p.tile_rows == 32) cache4_attn_few_kernel<T, g.value, 2><<<grid, 256, 0, st>>>(a);
      else if constexpr (sizeof(T) == 4) cache4_attn_many_kernel<T, g.value, 1, false><<<grid, 256, 0, st>>>(a);
      else {
        auto launch = [&](auto ct) {
          if (w) cache4_attn_many_kernel<T, g.value, ct.value, true><<<grid, 256, 0, st>>>(a);
          else cache4_attn_many_kernel<T, g.value, ct.value, false><<<grid, 256, 0, st>>>(a);
        };
        if (p.tile_rows == 128) launch(std::integral_constant<int, 1>());
        else if constexpr (g.value <= 2) launch(std::integral_constant<int, 2>());
      }
    });
    if (p.nsplit > 1) cache4_join_kernel<T><<<(unsigned)((p.rows + 3) / 4), 256, 0, st>>>(a, (int)p.rows);
    SI_CHECK_LAUNCH();
  }
  if (w && w->work > 0 && c->capacity > 0) {
    StageScope scope("cache4_weight", st);
    const unsigned grid = grid_of(w->work);
    by_groups(c, [&](auto g) {
      if (p.weight_rows == 16) cache4_weight_few_kernel<T, g.value, 1><<<grid, 256, 0, st>>>(*w);
      else if (p.weight_rows == 32) cache4_weight_few_kernel<T, g.value, 2><<<grid, 256, 0, st>>>(*w);
      else cache4_weight_many_kernel<T, g.value><<<grid, 256, 0, st>>>(*w);
    });
    SI_CHECK_LAUNCH();
  }
  return SI_OK;
}

// ----------------------------------------------------------------------------- eviction

struct EvictPlan {
  int64_t lists, chunks, parts, part_slots;
  size_t count_bytes, least_bytes, search_bytes, hist_bytes, bytes;
};

static si_status plan_evict(const si_cache4* c, int64_t keep, EvictPlan* p) {
  const si_status s = check_cache(c, false);
  if (s != SI_OK) return s;
  if (keep < 1 || keep > kMostTokens) return SI_ERR_SHAPE;
  p->lists = c->B * c->heads;
  p->chunks = (c->capacity + kEvictChunk - 1) / kEvictChunk;
  if ((double)p->lists * (double)p->chunks >= 4294967296.0 - kGridMost || (double)p->lists * (double)keep >= 1099511627776.0) return SI_ERR_SHAPE;
  p->count_bytes = align_up((size_t)(p->lists * p->chunks) * sizeof(int2), 256);
  p->least_bytes = align_up((size_t)p->lists * sizeof(uint2), 256);
  // Lists that do not fit a workgroup's registers are cut into up to 16 parts, as long as there are few lists: every part adds up all parts' counts.
  const int64_t batches = (c->capacity + kEvictPart - 1) / kEvictPart;
  p->parts = c->capacity <= kEvictWhole ? 0 : std::min<int64_t>(std::min<int64_t>(kEvictParts, batches), std::max<int64_t>(1, 1024 / p->lists));
  p->part_slots = p->parts ? (batches + p->parts - 1) / p->parts * kEvictPart : 0;
  p->search_bytes = p->parts ? align_up((size_t)p->lists * 2 * sizeof(EvictSearch), 256) : 0;
  p->hist_bytes = (size_t)(p->lists * p->parts) * kEvictBins * sizeof(int);
  p->bytes = p->count_bytes + p->least_bytes + p->search_bytes + 2 * p->hist_bytes + 256;
  return SI_OK;
}

}  // namespace si

// ============================================================================= C ABI

extern "C" {

si_status si_cache4_store(const si_heads* k, const si_heads* v, const int32_t* first, const int32_t* length, const si_cache4* cache,
                          float* weight, void* stream) {
  int64_t chunks;
  const si_status s = si::check_copy(k, v, cache, first, length, weight, false, &chunks);
  if (s != SI_OK) return s;
  return si::enqueue_copy(k, v, cache, first, length, weight, false, chunks, static_cast<hipStream_t>(stream));
}

si_status si_cache4_load(const si_cache4* cache, const int32_t* first, const int32_t* length, si_heads* k, si_heads* v, void* stream) {
  int64_t chunks;
  const si_status s = si::check_copy(k, v, cache, first, length, nullptr, true, &chunks);
  if (s != SI_OK) return s;
  return si::enqueue_copy(k, v, cache, first, length, nullptr, true, chunks, static_cast<hipStream_t>(stream));
}

size_t si_cache4_attn_workspace_bytes(const si_heads* q, const si_cache4* cache, int32_t weights) {
  si::CachePlan p;
  return si::plan_cache_attn(q, cache, 0, weights != 0, &p) == SI_OK ? p.bytes() : 0;
}

si_status si_cache4_attn_forward(const si_heads* q, const si_cache4* cache, float scale, int64_t run, const int32_t* q_len,
                                 const int32_t* k_len, const float* weight_in, float decay, float* weight_out, si_heads* out,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  si::CachePlan p;
  si_status s = si::plan_cache_attn(q, cache, run, weight_out != nullptr, &p);
  if (s == SI_OK) s = si::check_heads(out, true);
  if (s != SI_OK) return s;
  if (out->dtype != q->dtype) return SI_ERR_DTYPE;
  if (out->B != q->B || out->N != q->N || out->heads != q->heads || out->dim_head != q->dim_head) return SI_ERR_SHAPE;
  if (!(scale > 0.f) || !(scale <= 1e38f)) return SI_ERR_ARG;  // times log2(e) it is a float32
  if (weight_in && !weight_out) return SI_ERR_ARG;
  if (weight_in && !(decay >= 0.f && decay <= 3e38f)) return SI_ERR_ARG;
  if (!workspace) return SI_ERR_NULL;
  if (!si::aligned4(q_len) || !si::aligned4(k_len) || !si::aligned4(weight_in) || !si::aligned4(weight_out) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return SI_ERR_ALIGN;
  if (workspace_bytes < p.bytes()) return SI_ERR_WORKSPACE;
  const size_t weight_bytes = si::cache_rows(cache) * 4;
  const si::Span ws{workspace, p.bytes()}, win{weight_in, weight_bytes}, wout{weight_out, weight_bytes}, lens[] = {{q_len, (size_t)q->B * 4}, {k_len, (size_t)q->B * 4}};
  const si::CacheSpans spans(cache);
  if (!si::heads_apart(q, out) || spans.meets(out) || spans.meets(ws) || spans.meets(wout)) return SI_ERR_ARG;
  for (const si_heads* t : {q, static_cast<const si_heads*>(out)})
    if (si::heads_overlap_range(t, ws.p, ws.bytes) || (weight_out && si::heads_overlap_range(t, wout.p, wout.bytes))) return SI_ERR_ARG;
  if (weight_in && si::heads_overlap_range(out, win.p, win.bytes)) return SI_ERR_ARG;
  if (si::meet(ws, win) || si::meet(ws, wout) || (weight_in != weight_out && si::meet(win, wout))) return SI_ERR_ARG;
  for (const si::Span& l : lens)
    if (l.p && (si::meet(l, ws) || si::meet(l, wout) || si::heads_overlap_range(out, l.p, l.bytes))) return SI_ERR_ARG;

  si::CacheAttnArgs a;
  a.q = q->ptr; a.o = out->ptr;
  a.qb = q->stride_b; a.qn = q->stride_n; a.qh = q->stride_h;
  a.ob = out->stride_b; a.on = out->stride_n; a.oh = out->stride_h;
  a.c = si::view_of(cache);
  a.q_len = q_len; a.k_len = k_len;
  a.Nq = (int)q->N; a.group = p.group; a.d = (int)q->dim_head;
  a.run = run < q->N ? (int)run : 0;
  a.runs = (int)p.runs; a.run_len = (int)p.run_len; a.tiles_per_run = (int)p.tiles_per_run;
  a.work = (unsigned)p.work; a.nsplit = p.nsplit;
  a.scale_log2 = scale * 1.4426950408889634f;
  char* at = static_cast<char*>(workspace);
  a.part = reinterpret_cast<float*>(at);
  a.part_stat = reinterpret_cast<si::f32x4_t*>(at + p.part_bytes);
  a.row_stat = weight_out ? reinterpret_cast<float2*>(at + p.part_bytes + p.stat_bytes) : nullptr;
  si::CacheWeightArgs w;
  if (weight_out) {
    w.q = a.q; w.qb = a.qb; w.qn = a.qn; w.qh = a.qh;
    w.c = a.c; w.q_len = q_len; w.k_len = k_len;
    w.Nq = a.Nq; w.group = a.group; w.d = a.d; w.run = a.run;
    w.chunks = (int)p.weight_chunks;
    w.work = (unsigned)(p.weight_chunks * cache->B * cache->heads);
    w.scale_log2 = a.scale_log2; w.decay = decay;
    w.row_stat = a.row_stat; w.in = weight_in; w.out = weight_out;
  }
  const hipStream_t st = static_cast<hipStream_t>(stream);
  return q->dtype == SI_F32 ? si::launch_cache_attn<float>(a, weight_out ? &w : nullptr, cache, p, st)
                            : si::launch_cache_attn<si::bf16>(a, weight_out ? &w : nullptr, cache, p, st);
}

size_t si_cache4_evict_workspace_bytes(const si_cache4* cache, int64_t keep) {
  si::EvictPlan p;
  return si::plan_evict(cache, keep, &p) == SI_OK ? p.bytes : 0;
}

si_status si_cache4_evict(const si_cache4* cache, const int32_t* k_len, const float* weight, int64_t keep, int64_t first, int64_t last,
                          const si_cache4* out, float* weight_out, int32_t* kept, int32_t* out_len, void* workspace,
                          size_t workspace_bytes, void* stream) {
  si::EvictPlan p;
  si_status s = si::plan_evict(cache, keep, &p);
  if (s == SI_OK) s = si::check_cache(out, true);
  if (s != SI_OK) return s;
  if (out->B != cache->B || out->heads != cache->heads || out->dim_head != cache->dim_head || out->capacity < std::min(keep, cache->capacity)) return SI_ERR_SHAPE;
  if (first < 0 || last < 0 || first > keep || last > keep - first) return SI_ERR_ARG;
  if (!out_len || !workspace || (cache->capacity > 0 && (!weight || !weight_out || !kept))) return SI_ERR_NULL;
  for (const void* q : {static_cast<const void*>(k_len), static_cast<const void*>(weight), static_cast<const void*>(weight_out), static_cast<const void*>(kept),
                        static_cast<const void*>(out_len)})
    if (!si::aligned4(q)) return SI_ERR_ALIGN;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return SI_ERR_ALIGN;
  if (workspace_bytes < p.bytes) return SI_ERR_WORKSPACE;
  const si::CacheSpans from(cache), to(out);
  const si::Span in[] = {from.s[0], from.s[1], from.s[2], from.s[3], {weight, si::cache_rows(cache) * 4}, {k_len, (size_t)cache->B * 4}};
  const si::Span written[] = {to.s[0], to.s[1], to.s[2], to.s[3], {weight_out, si::cache_rows(out) * 4}, {kept, (size_t)(p.lists * keep) * 4},
                              {out_len, (size_t)cache->B * 4}, {workspace, p.bytes}};
  for (size_t i = 0; i < std::size(written); ++i) {
    for (const si::Span& x : in)
      if (si::meet(x, written[i])) return SI_ERR_ARG;
    for (size_t j = 0; j < i; ++j)
      if (si::meet(written[j], written[i])) return SI_ERR_ARG;
  }
  si::EvictArgs a;
  a.from = si::view_of(cache);
  a.to = si::view_of(out);
  a.weight = weight; a.weight_out = weight_out;
  a.kept = kept; a.out_len = out_len; a.k_len = k_len;
  a.keep = (int)keep; a.first = (int)first; a.last = (int)last;
  a.lists = (unsigned)p.lists;
  a.chunks = (unsigned)p.chunks;
  a.work = (unsigned)(p.lists * p.chunks);
  a.counts = static_cast<int2*>(workspace);
  char* at = static_cast<char*>(workspace) + p.count_bytes;
  a.least = reinterpret_cast<uint2*>(at);
  a.parts = (unsigned)p.parts;
  a.part_slots = p.part_slots;
  a.search = reinterpret_cast<si::EvictSearch*>(at += p.least_bytes);
  a.hist[0] = reinterpret_cast<int*>(at += p.search_bytes);
  a.hist[1] = reinterpret_cast<int*>(at + p.hist_bytes);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  si::StageScope scope("cache4_evict", st);
  if (p.parts == 0) {
    const unsigned grid = (unsigned)std::min<int64_t>(p.lists, si::kGridMost);
    if (cache->capacity <= 4 * si::kEvictThreads) si::cache4_pick_kernel<4><<<grid, si::kEvictThreads, 0, st>>>(a);
    else if (cache->capacity <= si::kEvictPart) si::cache4_pick_kernel<si::kEvictPer><<<grid, si::kEvictThreads, 0, st>>>(a);
    else si::cache4_pick_kernel<si::kEvictPerMost><<<grid, si::kEvictThreads, 0, st>>>(a);
  } else {
    const unsigned grid = (unsigned)std::min<int64_t>(p.lists * p.parts, si::kGridMost);
    si::cache4_search_kernel<0><<<grid, si::kEvictThreads, 0, st>>>(a);
    si::cache4_search_kernel<1><<<grid, si::kEvictThreads, 0, st>>>(a);
    si::cache4_search_kernel<2><<<grid, si::kEvictThreads, 0, st>>>(a);
    si::cache4_search_kernel<3><<<grid, si::kEvictThreads, 0, st>>>(a);
  }
  if (a.work > 0)
    si::by_groups(cache, [&](auto g) { si::cache4_move_kernel<g.value><<<(unsigned)std::min<int64_t>(a.work, si::kGridMost), si::kMoveThreads, 0, st>>>(a); });
  SI_CHECK_LAUNCH();
  return SI_OK;
}

}  // extern "C"

// Operators on heads of video tokens (see include/si.h): rotary positions, key-block selection, attention over key blocks.
// Checks, plans and launches, for their own entry points below and for the spatial block that uses them (si_api.hip).
#include "si_attn_ops.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "k_attn_select.h"
#include "k_attn_sparse.h"
#include "k_rope.h"
#include "si_host.h"

namespace si {

constexpr int64_t kMostOfBlock = 1 << 20;               // tokens of a run or a key block

static inline HeadsView view_of(const si_heads* t) { return HeadsView{t->ptr, t->stride_b, t->stride_n, t->stride_h}; }
static inline int heads_esize(const si_heads* t) { return t->dtype == SI_F32 ? 4 : 2; }
static inline bool heads_empty(const si_heads* t) { return t->N == 0; }

int64_t heads_extent(const si_heads* t, int64_t below) {
  int64_t e = t->dim_head;
  const int64_t n[] = {t->B, t->N, t->heads}, s[] = {t->stride_b, t->stride_n, t->stride_h};
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1 && s[i] < below) e += (n[i] - 1) * s[i];
  return e;
}

si_status check_heads(const si_heads* t, bool written) {
  if (!t) return SI_ERR_NULL;
  if (t->dtype != SI_F32 && t->dtype != SI_BF16) return SI_ERR_DTYPE;
  if (t->B < 1 || t->N < 0 || t->heads < 1 || t->dim_head < 8 || t->dim_head > 128 || t->dim_head % 8) return SI_ERR_SHAPE;
  if (t->B > (1 << 24) || t->N > kMostTokens || t->heads > 65535 || t->B * t->heads > (1 << 28)) return SI_ERR_SHAPE;
  const int64_t n[] = {t->B, t->N, t->heads}, s[] = {t->stride_b, t->stride_n, t->stride_h};
  const int vec = 16 / heads_esize(t);
  double far = (double)t->dim_head;
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (s[i] < 0 || s[i] >= (1LL << 44)) return SI_ERR_SHAPE;
    far += (double)(n[i] - 1) * (double)s[i];
  }
  if (far >= 70368744177664.0) return SI_ERR_SHAPE;  // 2^46 elements
  if (heads_empty(t)) return SI_OK;
  if (!t->ptr) return SI_ERR_NULL;
  if (!aligned16(t->ptr)) return SI_ERR_ALIGN;
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1 && s[i] % vec) return SI_ERR_ALIGN;
  if (written) {
    for (int i = 0; i < 3; ++i)  // every dimension steps over all that the smaller ones span
      if (n[i] > 1) {
        if (s[i] < heads_extent(t, s[i])) return SI_ERR_ARG;
        for (int j = 0; j < i; ++j)
          if (n[j] > 1 && s[j] == s[i]) return SI_ERR_ARG;
      }
  }
  return SI_OK;
}

static bool same_heads(const si_heads* a, const si_heads* b) {
  return a->ptr == b->ptr && a->dtype == b->dtype && a->B == b->B && a->N == b->N && a->heads == b->heads && a->dim_head == b->dim_head &&
         (a->B <= 1 || a->stride_b == b->stride_b) && (a->N <= 1 || a->stride_n == b->stride_n) && (a->heads <= 1 || a->stride_h == b->stride_h);
}

// Their ranges are apart, or they repeat with a common period
// (rows of one projection, halves of one buffer) and occupy different parts of it.
bool heads_apart(const si_heads* a, const si_heads* b) {
  if (heads_empty(a) || heads_empty(b)) return true;
  const int64_t ea = heads_esize(a), eb = heads_esize(b);
  if (!ranges_overlap(a->ptr, (size_t)(heads_extent(a) * ea), b->ptr, (size_t)(heads_extent(b) * eb))) return true;
  const int64_t periods[] = {a->stride_b, a->stride_n, a->stride_h};
  const int64_t counts[] = {a->B, a->N, a->heads};
  auto repeats = [](const si_heads* t, int64_t bytes, int64_t e) {
    const int64_t n[] = {t->B, t->N, t->heads}, s[] = {t->stride_b, t->stride_n, t->stride_h};
    for (int i = 0; i < 3; ++i)
      if (n[i] > 1 && s[i] * e >= bytes && (s[i] * e) % bytes) return false;
    return true;
  };
  for (int i = 0; i < 3; ++i) {
    const int64_t period = periods[i] * ea;
    if (counts[i] <= 1 || period <= 0 || period % eb) continue;
    if (!repeats(a, period, ea) || !repeats(b, period, eb)) continue;
    const int64_t wa = heads_extent(a, period / ea) * ea, wb = heads_extent(b, period / eb) * eb;
    const int64_t d = (int64_t)((reinterpret_cast<uintptr_t>(b->ptr) - reinterpret_cast<uintptr_t>(a->ptr)) % (uintptr_t)period);
    const int64_t delta = reinterpret_cast<uintptr_t>(b->ptr) >= reinterpret_cast<uintptr_t>(a->ptr)
                              ? d
                              : (period - (int64_t)((reinterpret_cast<uintptr_t>(a->ptr) - reinterpret_cast<uintptr_t>(b->ptr)) % (uintptr_t)period)) % period;
    if (delta >= wa && delta + wb <= period) return true;
  }
  return false;
}

bool heads_overlap_range(const si_heads* t, const void* p, size_t bytes) {
  return !heads_empty(t) && bytes && ranges_overlap(t->ptr, (size_t)heads_extent(t) * (size_t)heads_esize(t), p, bytes);
}

// ----------------------------------------------------------------------------- rotary positions

si_status check_rope(const si_rope* r, int d) {
  if (!r) return SI_ERR_NULL;
  int64_t pairs = 0;
  double tokens = 1.0;
  if (!(r->theta > 0.0) || !std::isnormal(r->theta)) return SI_ERR_ARG;  // 1 / theta is finite
  const double most = 1e12 * std::min(1.0, r->theta);  // frequencies are at most max(1, 1 / theta)
  for (int i = 0; i < 3; ++i) {
    if (r->extent[i] < 1 || r->extent[i] > INT32_MAX || r->pairs[i] < 0 || r->pairs[i] > d / 2) return SI_ERR_SHAPE;
    tokens *= (double)r->extent[i];
    pairs += r->pairs[i];
    // further out, a position times a frequency has no digits left behind the point
    if (!(std::fabs(r->origin[i]) <= most) || !(std::fabs(r->step[i]) * (double)r->extent[i] <= most)) return SI_ERR_ARG;
  }
  if (tokens > (double)kMostTokens) return SI_ERR_SHAPE;
  if (pairs < 1 || pairs % 4 || 2 * pairs > d) return SI_ERR_SHAPE;
  if (r->layout != SI_ROPE_INTERLEAVED && r->layout != SI_ROPE_HALVES) return SI_ERR_ARG;
  if (!std::isfinite(r->norm_eps)) return SI_ERR_ARG;
  if (r->norm_eps >= 0.f) {
    if ((r->q_gain && !aligned16(r->q_gain)) || (r->k_gain && !aligned16(r->k_gain))) return SI_ERR_ALIGN;
  }
  return SI_OK;
}

template <typename T>
static void launch_rope(const RopeArgs& a, bool halves, bool norm, dim3 grid, hipStream_t st) {
  if (halves) {
    if (norm) rope_kernel<T, true, true><<<grid, kRopeThreads, 0, st>>>(a);
    else rope_kernel<T, true, false><<<grid, kRopeThreads, 0, st>>>(a);
  } else {
    if (norm) rope_kernel<T, false, true><<<grid, kRopeThreads, 0, st>>>(a);
    else rope_kernel<T, false, false><<<grid, kRopeThreads, 0, st>>>(a);
  }
}

// Whether a gain that the norm reads (d elements of esize bytes) has a byte in [p, p + bytes).
bool rope_gain_in(const si_rope* r, int d, int esize, const void* p, size_t bytes) {
  if (r->norm_eps < 0.f) return false;
  for (const void* g : {r->q_gain, r->k_gain})
    if (g && ranges_overlap(g, (size_t)d * (size_t)esize, p, bytes)) return true;
  return false;
}

// Operands and descriptor have been checked; k and ko may be NULL.
si_status enqueue_rope(const si_heads* q, const si_heads* k, const si_rope* r, int64_t first, const si_heads* qo, const si_heads* ko,
                              hipStream_t st) {
  if (q->N == 0) return SI_OK;
  RopeArgs a;
  a.q = view_of(q);
  a.qo = view_of(qo);
  a.k = view_of(k ? k : q);
  a.ko = view_of(ko ? ko : qo);
  a.q_gain = r->q_gain;
  a.k_gain = r->k_gain;
  a.tokens = q->B * q->N;
  a.N = (int)q->N;
  a.H = (int)r->extent[1];
  a.W = (int)r->extent[2];
  a.first = (int)first;
  a.heads_q = (int)q->heads;
  a.heads = (int)(q->heads + (k ? k->heads : 0));
  a.d = (int)q->dim_head;
  a.pairs = r->pairs[0] + r->pairs[1] + r->pairs[2];
  a.end_f = r->pairs[0];
  a.end_y = r->pairs[0] + r->pairs[1];
  a.eps = r->norm_eps;
  a.inv_d = 1.f / (float)a.d;
  a.tokens_per_wg = kRopeThreads / (a.d / 8);
  int p = 0;
  for (int ax = 0; ax < 3; ++ax) {
    a.origin[ax] = r->origin[ax];
    a.step[ax] = r->step[ax];
    if (r->pairs[ax] == 0) continue;
    // powers by products of 64-bit significands: nearer than a power function in float64, and one of them instead of many
    const long double ratio = std::pow((long double)r->theta, -1.0L / r->pairs[ax]);
    long double f = 0.159154943091895335768883763372514362L;  // 1 / (2 pi)
    for (int i = 0; i < r->pairs[ax]; ++i, f *= ratio) a.freq[p++] = (double)f;
  }
  for (; p < kRopeMaxPairs; ++p) a.freq[p] = 0.0;
  // A workgroup takes every head of its tokens, so that their sines are computed once, unless that leaves CUs idle.
  const int64_t wgs = (a.tokens + a.tokens_per_wg - 1) / a.tokens_per_wg;
  if (wgs > (1 << 23)) return SI_ERR_SHAPE;
  const int shares = (int)std::min<int64_t>((a.heads + kRopeHeads - 1) / kRopeHeads, std::max<int64_t>(1, 1024 / wgs));
  a.heads_per_wg = ((a.heads + shares - 1) / shares + kRopeHeads - 1) / kRopeHeads * kRopeHeads;
  const dim3 grid((unsigned)wgs, (unsigned)((a.heads + a.heads_per_wg - 1) / a.heads_per_wg));
  StageScope scope("rope", st);
  if (q->dtype == SI_F32) launch_rope<float>(a, r->layout == SI_ROPE_HALVES, r->norm_eps >= 0.f, grid, st);
  else launch_rope<bf16>(a, r->layout == SI_ROPE_HALVES, r->norm_eps >= 0.f, grid, st);
  SI_CHECK_LAUNCH();
  return SI_OK;
}

// ----------------------------------------------------------------------------- runs and blocks

// Sizes that the selection and the attention share.
si_status plan_blocks(const si_heads* q, const si_heads* k, int64_t q_block, int64_t k_block, BlocksPlan* p) {
  if (q->dtype != k->dtype) return SI_ERR_DTYPE;
  if (q->B != k->B || q->dim_head != k->dim_head || q->heads % k->heads) return SI_ERR_SHAPE;
  if (q_block < 1 || q_block > kMostOfBlock || k_block < 64 || k_block > kMostOfBlock || k_block % 64) return SI_ERR_SHAPE;
  p->group = (int)(q->heads / k->heads);
  if (p->group * q_block >= (1 << 24)) return SI_ERR_SHAPE;
  if (k->N > 1 && k->stride_n >= (1 << 23)) return SI_ERR_SHAPE;  // 64 rows of keys inside 31 bits of bytes
  p->runs = (q->N + q_block - 1) / q_block;
  p->blocks = (k->N + k_block - 1) / k_block;
  p->words = (p->blocks + 31) / 32;
  // kernels count lists, blocks and pieces of rows in 32 bits
  const double lists = (double)q->B * (double)k->heads, most = 2147483648.0 - kGridMost;
  if (lists * (double)p->runs * 16 >= most || lists * (double)p->blocks * 16 >= most) return SI_ERR_SHAPE;
  if (lists * (double)p->runs * (double)(p->words + 1) >= 1e12) return SI_ERR_SHAPE;
  return SI_OK;
}

// ----------------------------------------------------------------------------- selection

size_t select_bytes(const si_heads* q, const si_heads* k, const BlocksPlan& p) {
  return align_up((size_t)(q->B * k->heads * p.runs * q->dim_head) * sizeof(double), 256) +
         align_up((size_t)(q->B * k->heads * p.blocks * q->dim_head) * sizeof(double), 256);
}

static MeansOf means_of(const si_heads* x, int64_t heads_kv, int64_t block, int64_t runs, int64_t chunks, const int32_t* len, double* out) {
  return MeansOf{view_of(x), len, out, (int)x->N, (int)(x->heads / heads_kv), (int)block, (int)runs, (unsigned)(x->B * runs * chunks)};
}

si_status enqueue_select(const si_heads* q, const si_heads* k, const BlocksPlan& p, int64_t q_block, int64_t k_block, int64_t keep,
                                const int32_t* q_len, const int32_t* k_len, uint32_t* blocks, char* ws, hipStream_t st) {
  if (p.runs == 0 || p.words == 0) return SI_OK;
  StageScope scope("attn_select", st);
  double* qm = reinterpret_cast<double*>(ws);
  double* km = reinterpret_cast<double*>(ws + align_up((size_t)(q->B * k->heads * p.runs * q->dim_head) * sizeof(double), 256));
  MeansArgs m;
  m.heads_kv = (int)k->heads;
  m.d = (int)q->dim_head;
  m.chunks = (int)((k->heads * q->dim_head * heads_esize(q) / 16 + kMeanPieces - 1) / kMeanPieces);
  m.of[0] = means_of(q, k->heads, q_block, p.runs, m.chunks, q_len, qm);
  m.of[1] = means_of(k, k->heads, k_block, p.blocks, m.chunks, k_len, km);
  const unsigned grid = (unsigned)std::min<int64_t>((int64_t)m.of[0].work + m.of[1].work, kGridMost);
  if (q->dtype == SI_F32) block_means_kernel<float><<<grid, kMeanPieces * kMeanSlices, 0, st>>>(m);
  else block_means_kernel<bf16><<<grid, kMeanPieces * kMeanSlices, 0, st>>>(m);
  SI_CHECK_LAUNCH();
  SelectArgs a;
  a.qm = qm; a.km = km; a.out = blocks;
  a.q_len = q_len; a.k_len = k_len;
  a.Nq = (int)q->N; a.Nk = (int)k->N;
  a.heads_kv = (int)k->heads; a.d = (int)q->dim_head;
  a.q_block = (int)q_block; a.k_block = (int)k_block;
  a.runs = (int)p.runs; a.blocks = (int)p.blocks; a.words = (int)p.words;
  a.keep = (int)std::min<int64_t>(keep, p.blocks);
  a.pitch = (int)((p.blocks + 15) / 16 * 16 + 2);
  auto launch = [&](auto cap, auto kpl, auto threads) {
    a.rows = std::min(16, cap.value / a.pitch);
    a.tiles = (int)((p.runs + a.rows - 1) / a.rows);
    a.work = (unsigned)(q->B * k->heads * a.tiles);
    const unsigned grid = (unsigned)((std::min<int64_t>((int64_t)a.work, kGridMost) + 7) / 8 * 8);
    switch ((a.d + 31) / 32) {
      case 1: block_select_kernel<cap.value, kpl.value, threads.value, 1><<<grid, threads.value, 0, st>>>(a); break;
      case 2: block_select_kernel<cap.value, kpl.value, threads.value, 2><<<grid, threads.value, 0, st>>>(a); break;
      case 3: block_select_kernel<cap.value, kpl.value, threads.value, 3><<<grid, threads.value, 0, st>>>(a); break;
      default: block_select_kernel<cap.value, kpl.value, threads.value, 4><<<grid, threads.value, 0, st>>>(a); break;
    }
  };
  // The smallest store of scores that holds 16 runs, for as many workgroups on a CU as possible, and a wavefront for every run;
  // lists of up to 32 blocks have too little work for that many.  Calls with 512 and with 1024 threads: 16 blocks (32 batch entries
  // of 1024 tokens) 22.8 and 25.4 us, 64 (float32, padded) 15.1 and 14.7, 144 (9216 tokens) 22.5 and 21.7, 400 (25600 tokens) 49.2
  // and 54.8 (there alone fewer would be better), 900 (57600 tokens) 139 and 134.
  using std::integral_constant;
  if (p.blocks <= 32) launch(integral_constant<int, 16 * 34>(), integral_constant<int, 1>(), integral_constant<int, 512>());
  else if (p.blocks <= 64) launch(integral_constant<int, 16 * 66>(), integral_constant<int, 1>(), integral_constant<int, 1024>());
  else if (p.blocks <= 128) launch(integral_constant<int, 16 * 130>(), integral_constant<int, 2>(), integral_constant<int, 1024>());
  else if (p.blocks <= 256) launch(integral_constant<int, 16 * 258>(), integral_constant<int, 4>(), integral_constant<int, 1024>());
  else if (p.blocks <= 512) launch(integral_constant<int, 16 * 514>(), integral_constant<int, 8>(), integral_constant<int, 1024>());
  else if (p.blocks <= 1024) launch(integral_constant<int, 16 * 1026>(), integral_constant<int, 16>(), integral_constant<int, 1024>());
  else launch(integral_constant<int, 16 * 1028>(), integral_constant<int, 0>(), integral_constant<int, 1024>());
  static_assert(16 * 1028 >= kSelectMaxBlocks + 2, "one run of the longest list");
  SI_CHECK_LAUNCH();
  return SI_OK;
}

// ----------------------------------------------------------------------------- attention over blocks

// Rows of a workgroup and shares of a run's blocks.  bf16: 32 rows per wavefront, up to 128 of a run together.  float32: 16
// per wavefront, 32 in runs of more than 64 rows.  Blocks are dealt out to several workgroups while there are fewer than two
// for every CU.
si_status plan_sparse(const si_heads* q, const si_heads* k, int64_t q_block, const BlocksPlan& b, bool may_split, SparsePlan* p) {
  const int64_t rows = b.group * std::min<int64_t>(q_block, std::max<int64_t>(q->N, 1));
  p->tile_rows = q->dtype == SI_F32 && rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  p->tiles_per_run = (rows + p->tile_rows - 1) / p->tile_rows;
  if ((double)q->B * k->heads * b.runs * (double)p->tiles_per_run >= 2147483648.0 - kGridMost) return SI_ERR_SHAPE;
  p->tiles = q->B * k->heads * b.runs * p->tiles_per_run;
  const int64_t want = p->tile_rows <= 32 ? 1024 : 512;
  p->nsplit = 1;
  if (may_split && p->tiles > 0 && p->tiles * 2 <= want) p->nsplit = (int)std::min<int64_t>(std::min<int64_t>(want / p->tiles, 64), std::max<int64_t>(1, b.blocks / 2));
  p->work = p->tiles * p->nsplit;
  p->rows = q->B * q->N * q->heads;
  p->part_bytes = p->nsplit > 1 ? (size_t)(q->B * q->N * q->heads) * p->nsplit * (q->dim_head + 2) * sizeof(float) : 0;
  return SI_OK;
}

// Calls f(integral_constant<d / 8>) for a head of d channels.
template <int D8 = 1, class Fn>
static void by_head(int d, Fn f) {
  if constexpr (D8 <= 16) {
    if (d == 8 * D8) f(std::integral_constant<int, D8>());
    else by_head<D8 + 1>(d, f);
  }
}

template <typename T>
static void dispatch_sparse(const SparseArgs& a, const SparsePlan& p, hipStream_t st) {
  const unsigned grid = (unsigned)((std::min<int64_t>((int64_t)a.work, kGridMost) + 7) / 8 * 8);
  using std::integral_constant;
  if constexpr (sizeof(T) == 4) {
    by_head(a.d, [&](auto d8) {
      if (p.tile_rows == 16) sparse_attn_f32_kernel<d8.value, 1, 1><<<grid, 64, 0, st>>>(a);
      else if (p.tile_rows == 32) sparse_attn_f32_kernel<d8.value, 2, 1><<<grid, 128, 0, st>>>(a);
      else if (p.tile_rows == 64) sparse_attn_f32_kernel<d8.value, 4, 1><<<grid, 256, 0, st>>>(a);
      else sparse_attn_f32_kernel<d8.value, 4, 2><<<grid, 256, 0, st>>>(a);
    });
  } else {
    // steps of 16 channels; one form for 8 to 32 channels and one for 104 to 128
    auto launch_pad = [&](auto ks, auto pad) {
      if (p.tile_rows == 32) sparse_attn_bf16_kernel<ks.value, 1, pad.value, 1><<<grid, 64, 0, st>>>(a);
      else if (p.tile_rows == 64) sparse_attn_bf16_kernel<ks.value, 4, pad.value, 2><<<grid, 256, 0, st>>>(a);
      else sparse_attn_bf16_kernel<ks.value, 4, pad.value, 1><<<grid, 256, 0, st>>>(a);
    };
    auto launch = [&](auto ks) {
      if (a.d < 16 * ks.value) launch_pad(ks, std::true_type());
      else launch_pad(ks, std::false_type());
    };
    const int ks = (a.d + 15) / 16;
    if (ks <= 2) launch(integral_constant<int, 2>());
    else if (ks == 3) launch(integral_constant<int, 3>());
    else if (ks == 4) launch(integral_constant<int, 4>());
    else if (ks == 5) launch(integral_constant<int, 5>());
    else if (ks == 6) launch(integral_constant<int, 6>());
    else launch(integral_constant<int, 8>());
  }
  if (a.nsplit > 1) {
    const int rows = (int)p.rows;  // at most 128 for each of 256 tiles: a split call has few
    sparse_join_kernel<T><<<(unsigned)((rows + 3) / 4), 256, 0, st>>>(a, rows);
  }
}

si_status enqueue_sparse(const si_heads* q, const si_heads* k, const si_heads* v, const BlocksPlan& b, const SparsePlan& p, int64_t q_block,
                                int64_t k_block, float scale, const int32_t* q_len, const int32_t* k_len, const uint32_t* blocks,
                                const si_heads* out, char* ws, hipStream_t st, int o_frag) {
  if (p.tiles == 0) return SI_OK;
  SparseArgs a;
  a.q = q->ptr; a.k = k->ptr; a.v = v->ptr; a.o = out->ptr;
  a.qb = q->stride_b; a.qn = q->stride_n; a.qh = q->stride_h;
  a.kb = k->stride_b; a.kn = k->stride_n; a.kh = k->stride_h;
  a.vb = v->stride_b; a.vn = v->stride_n; a.vh = v->stride_h;
  a.ob = out->stride_b; a.on = out->stride_n; a.oh = out->stride_h;
  a.mask = blocks;
  a.q_len = q_len; a.k_len = k_len;
  a.Nq = (int)q->N; a.Nk = (int)k->N;
  a.heads_kv = (int)k->heads; a.group = b.group; a.d = (int)q->dim_head;
  a.q_block = (int)q_block; a.k_block = (int)k_block;
  a.runs = (int)b.runs; a.words = (int)b.words;
  a.tiles_per_run = (int)p.tiles_per_run;
  a.work = (unsigned)p.work; a.nsplit = p.nsplit;
  a.c = scale * 1.4426950408889634f;
  a.part = reinterpret_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(a.part + (p.nsplit > 1 ? p.rows * p.nsplit * q->dim_head : 0));
  a.o_frag = o_frag;
  StageScope scope("attn_sparse", st);
  if (q->dtype == SI_F32) dispatch_sparse<float>(a, p, st);
  else dispatch_sparse<bf16>(a, p, st);
  SI_CHECK_LAUNCH();
  return SI_OK;
}

}  // namespace si

// ============================================================================= C ABI

extern "C" {

si_status si_rope_forward(const si_heads* q, const si_heads* k, const si_rope* rope, int64_t first, si_heads* q_out, si_heads* k_out,
                          void* stream) {
  if (!q || !q_out || !rope || (!k) != (!k_out)) return SI_ERR_NULL;
  const si_heads *in[] = {q, k}, *out[] = {q_out, k_out};
  const int n = k ? 2 : 1;
  for (int i = 0; i < n; ++i) {
    si_status s = si::check_heads(in[i], false);
    if (s == SI_OK) s = si::check_heads(out[i], true);
    if (s != SI_OK) return s;
    if (in[i]->dtype != q->dtype || out[i]->dtype != q->dtype) return SI_ERR_DTYPE;
    if (in[i]->B != q->B || in[i]->N != q->N || in[i]->dim_head != q->dim_head) return SI_ERR_SHAPE;
    if (out[i]->B != q->B || out[i]->N != q->N || out[i]->dim_head != q->dim_head || out[i]->heads != in[i]->heads) return SI_ERR_SHAPE;
  }
  const si_status s = si::check_rope(rope, (int)q->dim_head);
  if (s != SI_OK) return s;
  if (first < 0 || (double)first + (double)q->N > (double)rope->extent[0] * (double)rope->extent[1] * (double)rope->extent[2]) return SI_ERR_SHAPE;
  for (int i = 0; i < n; ++i) {  // an output is its own input or apart from every input and output
    for (int j = 0; j < n; ++j) {
      if (!(i == j && si::same_heads(in[j], out[i])) && !si::heads_apart(in[j], out[i])) return SI_ERR_ARG;
      if (i != j && !si::heads_apart(out[i], out[j])) return SI_ERR_ARG;
    }
    const int es = si::heads_esize(q);
    if (!si::heads_empty(out[i]) && si::rope_gain_in(rope, (int)q->dim_head, es, out[i]->ptr, (size_t)si::heads_extent(out[i]) * es)) return SI_ERR_ARG;
  }
  return si::enqueue_rope(q, k, rope, first, q_out, k_out, static_cast<hipStream_t>(stream));
}

int64_t si_attn_block_words(int64_t n_keys, int64_t k_block) {
  if (n_keys < 0 || n_keys > si::kMostTokens || k_block < 64 || k_block > si::kMostOfBlock || k_block % 64) return 0;
  return ((n_keys + k_block - 1) / k_block + 31) / 32;
}

static si_status check_select(const si_heads* q, const si_heads* k, int64_t q_block, int64_t k_block, si::BlocksPlan* p) {
  si_status s = si::check_heads(q, false);
  if (s == SI_OK) s = si::check_heads(k, false);
  if (s == SI_OK) s = si::plan_blocks(q, k, q_block, k_block, p);
  if (s != SI_OK) return s;
  return p->blocks > si::kSelectMaxBlocks ? SI_ERR_SHAPE : SI_OK;
}

size_t si_attn_select_workspace_bytes(const si_heads* q, const si_heads* k, int64_t q_block, int64_t k_block) {
  si::BlocksPlan p;
  if (check_select(q, k, q_block, k_block, &p) != SI_OK) return 0;
  return si::select_bytes(q, k, p) + 256;
}

si_status si_attn_select(const si_heads* q, const si_heads* k, int64_t q_block, int64_t k_block, int64_t keep, const int32_t* q_len,
                         const int32_t* k_len, uint32_t* blocks, void* workspace, size_t workspace_bytes, void* stream) {
  si::BlocksPlan p;
  const si_status s = check_select(q, k, q_block, k_block, &p);
  if (s != SI_OK) return s;
  if (keep < 1) return SI_ERR_ARG;
  const size_t bits = (size_t)(q->B * k->heads * p.runs * p.words) * 4, need = si::select_bytes(q, k, p) + 256;
  if ((!blocks && bits) || !workspace) return SI_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(q_len) & 3u) || (reinterpret_cast<uintptr_t>(k_len) & 3u) || (reinterpret_cast<uintptr_t>(blocks) & 3u) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return SI_ERR_ALIGN;
  if (workspace_bytes < need) return SI_ERR_WORKSPACE;
  if (si::ranges_overlap(workspace, need, blocks, bits) || si::heads_overlap_range(q, workspace, need) || si::heads_overlap_range(k, workspace, need) ||
      si::heads_overlap_range(q, blocks, bits) || si::heads_overlap_range(k, blocks, bits))
    return SI_ERR_ARG;
  const size_t lens = (size_t)q->B * 4;
  for (const int32_t* l : {q_len, k_len})
    if (l && (si::ranges_overlap(l, lens, workspace, need) || si::ranges_overlap(l, lens, blocks, bits))) return SI_ERR_ARG;
  return si::enqueue_select(q, k, p, q_block, k_block, keep, q_len, k_len, blocks, static_cast<char*>(workspace), static_cast<hipStream_t>(stream));
}

static si_status check_sparse(const si_heads* q, const si_heads* k, int64_t q_block, int64_t k_block, si::BlocksPlan* b, si::SparsePlan* p) {
  si_status s = si::check_heads(q, false);
  if (s == SI_OK) s = si::check_heads(k, false);
  if (s == SI_OK) s = si::plan_blocks(q, k, q_block, k_block, b);
  if (s == SI_OK) s = si::plan_sparse(q, k, q_block, *b, true, p);
  return s;
}

size_t si_attn_sparse_workspace_bytes(const si_heads* q, const si_heads* k, int64_t q_block, int64_t k_block) {
  si::BlocksPlan b;
  si::SparsePlan p;
  if (check_sparse(q, k, q_block, k_block, &b, &p) != SI_OK) return 0;
  return p.part_bytes + 256;
}

si_status si_attn_sparse_forward(const si_heads* q, const si_heads* k, const si_heads* v, int64_t q_block, int64_t k_block, float scale,
                                 const int32_t* q_len, const int32_t* k_len, const uint32_t* blocks, si_heads* out, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  si::BlocksPlan b;
  si::SparsePlan p;
  si_status s = check_sparse(q, k, q_block, k_block, &b, &p);
  if (s == SI_OK) s = si::check_heads(v, false);
  if (s == SI_OK) s = si::check_heads(out, true);
  if (s != SI_OK) return s;
  if (v->dtype != q->dtype || out->dtype != q->dtype) return SI_ERR_DTYPE;
  if (v->B != k->B || v->N != k->N || v->heads != k->heads || v->dim_head != k->dim_head) return SI_ERR_SHAPE;
  if (v->N > 1 && v->stride_n >= (1 << 23)) return SI_ERR_SHAPE;
  if (out->B != q->B || out->N != q->N || out->heads != q->heads || out->dim_head != q->dim_head) return SI_ERR_SHAPE;
  if (!(scale > 0.f) || !(scale <= 1e38f)) return SI_ERR_ARG;  // times log2(e) it is a float32
  const size_t need = p.part_bytes + 256, bits = blocks ? (size_t)(q->B * k->heads * b.runs * b.words) * 4 : 0;
  if (!workspace) return SI_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(q_len) & 3u) || (reinterpret_cast<uintptr_t>(k_len) & 3u) || (reinterpret_cast<uintptr_t>(blocks) & 3u) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return SI_ERR_ALIGN;
  if (workspace_bytes < need) return SI_ERR_WORKSPACE;
  for (const si_heads* t : {q, k, v}) {
    if (!si::heads_apart(t, out)) return SI_ERR_ARG;
    if (si::heads_overlap_range(t, workspace, need)) return SI_ERR_ARG;
  }
  const size_t lens = (size_t)q->B * 4;
  if (si::heads_overlap_range(out, workspace, need) || (bits && (si::heads_overlap_range(out, blocks, bits) || si::ranges_overlap(workspace, need, blocks, bits))))
    return SI_ERR_ARG;
  for (const int32_t* l : {q_len, k_len})
    if (l && (si::ranges_overlap(l, lens, workspace, need) || si::heads_overlap_range(out, l, lens))) return SI_ERR_ARG;
  return si::enqueue_sparse(q, k, v, b, p, q_block, k_block, scale, q_len, k_len, blocks, out, static_cast<char*>(workspace),
                            static_cast<hipStream_t>(stream), 0);
}

}  // extern "C"

// Attention of new tokens over a cache in 4 bits (k_cache4.h), and the weight that every cached token received.
//
// All queries of a key head walk the same keys, or with runs those up to the end of their own run.  The rows of a key head
// (tokens times the query heads that share it) are cut into tiles, a tile's keys into steps of 32 that are dealt out to the
// wavefronts of a workgroup and, where there are few tiles, to several workgroups.  Every wavefront keeps the running maximum
// and sum of a softmax and its own output; they are joined in a fixed order.
// An output is divided by its sum at the end.  Until then it is a sum over up to 2^31 slots of weights up to kSparseTrigger = 2^8 (2^64 at scores of
// 1e9, where the maximum's own rounding is that large), so values of up to 2^88 (2^32) stay finite.
//   S^T[key, row] = K Q^T       row operand: keys, column operand: rows
//   O^T[chan, row] += V^T P^T   column operand: the softmax result registers as they stand
// Codes are read once, become bf16 (exactly) in registers, and go to the matrix cores: keys straight from where they were
// loaded, as a lane's channels of a key lie next to each other there; values by way of LDS, which transposes them.
// float32 queries are three bf16 parts whose sum is the value, and so are their probabilities: the products are exact and
// the sums float32.
#pragma once
#include "k_attn_sparse.h"
#include "k_cache4.h"

namespace si {

struct CacheAttnArgs {
  const void* q;
  void* o;
  int64_t qb, qn, qh, ob, on, oh;  // strides in elements
  Cache4View c;
  const int *q_len, *k_len;  // per batch entry, or NULL
  int Nq, group, d;
  int run;                   // tokens of a run, 0: every query sees every key
  int runs, run_len;         // of the tiling: tiles end with a run unless a run is shorter than a tile
  int tiles_per_run;
  unsigned work;             // B * heads * runs * tiles_per_run * nsplit
  int nsplit;
  float scale_log2;          // softmax scale * log2(e)
  float* part;               // nsplit > 1: outputs [query row][nsplit][d]; query row = (b Nq + n) heads + h
  f32x4_t* part_stat;        // nsplit > 1: (maximum, sum of the rounded weights, sum of the weights) [query row][nsplit]
  float2* row_stat;          // or NULL: row_stat() of every query row
};

// Batch entry, key head, tile and share of a piece of work, and which keys its rows see.
struct CacheTile {
  int part, tile, run, hk, b, q_len, k_len;
  __device__ __forceinline__ CacheTile(const CacheAttnArgs& a, unsigned work) {
    auto pop = [&](int n) {  // the fastest index
      const unsigned up = work / (unsigned)n;
      const int i = (int)(work - up * n);
      work = up;
      return i;
    };
    part = a.nsplit > 1 ? pop(a.nsplit) : 0;
    tile = a.tiles_per_run > 1 ? pop(a.tiles_per_run) : 0;
    run = a.runs > 1 ? pop(a.runs) : 0;
    hk = pop(a.c.heads);
    b = (int)work;
    q_len = a.q_len ? min(max(a.q_len[b], 0), a.Nq) : a.Nq;
    k_len = a.k_len ? min(max(a.k_len[b], 0), a.c.cap) : a.c.cap;
  }
  // token of row `rho` of the tiling's run, or -1; sub: its head among those of the key head
  __device__ __forceinline__ int token(const CacheAttnArgs& a, int rho, int& sub) const {
    const int in_run = a.group > 1 ? rho / a.group : rho;
    const int64_t n = (int64_t)run * a.run_len + in_run;
    sub = rho - in_run * a.group;
    return in_run < a.run_len && n < q_len ? (int)n : -1;
  }
  // keys that token n sees, the first so many
  __device__ __forceinline__ int seen(const CacheAttnArgs& a, int n) const { return cache_seen(a.run, n, q_len, k_len); }
  __device__ __forceinline__ static int cache_seen(int run, int n, int q_len, int k_len) {
    if (run == 0) return k_len;
    const int64_t end = min(((int64_t)(n / run) + 1) * run, (int64_t)q_len);
    return (int)max((int64_t)0, k_len - q_len + end);
  }
};

// What turns a score s of a row into its softmax weight, 2^(c s - x) y: the maximum and 1 / sum of the weights.  No keys: y = 0; NaN: x is NaN and
// y is not, so that what the row does not see can be left out by a weight of zero.
__device__ __forceinline__ float2 row_stat(float maximum, float sum) {
  if (!(sum == sum)) return make_float2(NAN, 1.f);
  return make_float2(maximum, sum == 0.f ? 0.f : 1.f / sum);
}

// A pair of values as bf16 parts: one, rounded, or three that add up to it, eight of its 24 bits each.
template <int TERMS>
__device__ __forceinline__ void bf16_parts(float lo, float hi, unsigned (&out)[TERMS]) {
  if constexpr (TERMS == 1) {
    out[0] = pack_bf16x2(lo, hi);
  } else {
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
      out[t] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);  // upper halves
      lo -= __uint_as_float(out[t] << 16);
      hi -= __uint_as_float(out[t] & 0xFFFF0000u);
    }
  }
}

// Eight float32 channels as operands.
template <int TERMS>
__device__ __forceinline__ void query_parts(const f32x4_t& x, const f32x4_t& y, u32x4_t (&out)[TERMS]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned w[TERMS];
    const float lo = i < 2 ? x[2 * i] : y[2 * i - 4], hi = i < 2 ? x[2 * i + 1] : y[2 * i - 3];
    bf16_parts<TERMS>(lo, hi, w);
    // an infinity's rest would be a NaN: it has none
    if (__builtin_isinf(lo) || __builtin_isinf(hi))
#pragma unroll
      for (int t = 1; t < TERMS; ++t) w[t] &= (__builtin_isinf(lo) ? 0xFFFF0000u : ~0u) & (__builtin_isinf(hi) ? 0x0000FFFFu : ~0u);
#pragma unroll
    for (int t = 0; t < TERMS; ++t) out[t][i] = w[t];
  }
}
// The same of a query's row in either type.
template <typename T, int TERMS>
__device__ __forceinline__ void query_parts(const T* p, u32x4_t (&out)[TERMS]) {
  if constexpr (sizeof(T) == 2) out[0] = *reinterpret_cast<const u32x4_t*>(p);
  else query_parts(*reinterpret_cast<const f32x4_t*>(p), *reinterpret_cast<const f32x4_t*>(p + 4), out);
}

// The codes of two tiles of 16 keys as the lanes of a row operand hold them: lane (r, g) channels 8 G g .. 8 G g + 8 G - 1 of keys
// r and 16 + r, and the two keys' scales.
template <int G>
struct KeyCodes {
  static constexpr int S = cache4_scale_bytes(G);
  unsigned w[2][G];
  unsigned s[2];
  // The key's row begins at codes + at[t] * 16 G, with an offset that lanes have of their own from a base that they share.
  __device__ __forceinline__ void load_rows(const uint8_t* codes, const uint8_t* scales, const unsigned (&at)[2], int g) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const unsigned* p = reinterpret_cast<const unsigned*>(codes + (at[t] * (16u * G) + g * (4u * G)));
      if constexpr (G == 4) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[t][i] = v[i];
      } else if constexpr (G == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[t][0] = v.x; w[t][1] = v.y;
      } else {
#pragma unroll
        for (int i = 0; i < G; ++i) w[t][i] = p[i];
      }
      if constexpr (S == 4) s[t] = *reinterpret_cast<const unsigned*>(scales + at[t] * 4u);
      else if constexpr (S == 2) s[t] = *reinterpret_cast<const unsigned short*>(scales + at[t] * 2u);
      else s[t] = scales[at[t]];
    }
  }
  // Keys key0 .. key0 + 31 of a head, those at and behind `end` as the last one before it.
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int key0, int end, int r, int g) {
    const int last = end - 1 - key0;
    const unsigned at[2] = {(unsigned)min(r, last), (unsigned)min(16 + r, last)};
    load_rows(codes + (int64_t)key0 * (16 * G), scales + (int64_t)key0 * S, at, g);
  }
  // Channels 8 G g + 8 i .. + 7 of key tile t.  Groups of 32 channels are 4 / G lanes' or, with three of them, end inside a lane's.
  __device__ __forceinline__ u32x4_t operand(int t, int i, int g) const {
    const unsigned group = G == 4 ? g : G == 2 ? g / 2 : G == 1 ? 0 : (3 * g + i) / 4;
    return cache4_bf16x8(w[t][i], __uint_as_float(((s[t] >> (8 * group)) & 255u) << 23));
  }
};

// A NaN among the values would make one of every row's weight of zero as well.  It is stored as zeros instead, and the lowest slot that has one
// in a group is noted: rows that see it receive NaN in that group in the end.
__device__ __forceinline__ void note_nan(int* bad_key, int group, int key, u32x4_t& codes, unsigned& scale) {
  atomicMin(&bad_key[group], key);
  codes = u32x4_t{0, 0, 0, 0};
  scale = 127u;
}

// Rows of up to 32 of a tile: four wavefronts that each take every fourth step of 32 keys, on their own until the end.
// T: of queries and outputs.  G: groups of 32 channels of a head.  NT: columns of rows, 16 each.
// One token of 32 heads against 115200 slots of 8 heads of 128, four batch entries: 502 MB in 92 us, 5.4 TB/s, bound by HBM (with
// registers spilled to scratch, whose reloads wait for every load in flight, 197 us).  Eight such tokens, 32 rows, 57600 slots and fewer, two batch
// entries: 116 MB in 36 us: a step's chain of latencies on two wavefronts per SIMD.  float32 rows beyond 16 of heads of 104 to 128 do spill, 29
// registers: eight such tokens over 60000 slots take 92 us.
template <typename T, int G, int NT>
__global__ __launch_bounds__(256, sizeof(T) == 2 && NT == 1 ? (G > 2 ? 3 : 4) : 2) void cache4_attn_few_kernel(CacheAttnArgs a) {
  constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;
  constexpr int ROW = G == 1 ? 64 : G == 2 ? 128 : 256;  // bytes of a key's values in LDS
  constexpr int UNITS = 32 * G, PER = (UNITS + 63) / 64;  // groups of a step's values, and a lane's share
  constexpr int KEEP = 2 * G * 4 * NT + 3 * NT;           // what a wavefront hands over at the end, a lane
  constexpr int BYTES = 4 * 32 * ROW > 2 * KEEP * 256 ? 4 * 32 * ROW : 2 * KEEP * 256;
  constexpr int SB = cache4_scale_bytes(G);
  __shared__ __align__(1024) u32x4_t lds[BYTES / 16];
  __shared__ int bad_key[4];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % 16, g = lane / 16;
  // A key's values lie in 16-byte pieces; piece p in slot p ^ swizzle(key).  LDS has 64 banks of 4 bytes: the transposing reads of 32 lanes take
  // two pieces of eight keys, and 16 lanes write one of every four pieces of the keys that key_of gives them; both fall on different banks.
  auto swizzle = [](int key) { return ROW == 64 ? ((key >> 2) & 1) << 1 | ((key >> 3) & 1) : ROW == 128 ? (key & 6) | ((key >> 3) & 1) : (key & 7) << 1 | ((key >> 3) & 1); };
  auto key_of = [](int unit) {  // a step's values in groups of 32 channels: unit / G with some of its bits in another order
    const int n = unit / G;
    return G == 4 ? (n & 17) | (n & 2) << 2 | (n & 12) >> 1 : G == 2 ? (n & 19) | (n & 4) << 1 | (n & 8) >> 1 : n;
  };
  const unsigned vals = (unsigned)(size_t)(__attribute__((address_space(3))) void*)(&lds[0]) + wave * 32 * ROW;

  const unsigned chunk = (a.work + 7) / 8;  // contiguous per XCD: a head's codes are fetched into one L2
  const unsigned chunk_end = min(a.work, (blockIdx.x % 8 + 1) * chunk);
  for (unsigned work = blockIdx.x % 8 * chunk + blockIdx.x / 8; work < chunk_end; work += gridDim.x / 8) {
    const CacheTile t(a, work);
    int first_sub;
    const int first = t.token(a, t.tile * 16 * NT, first_sub);
    if (first < 0) continue;  // the tile's first row is its earliest token
    if (threadIdx.x < 4) bad_key[threadIdx.x] = INT32_MAX;
    __syncthreads();
    // keys that every row sees, and that any sees
    const int64_t last = min(min((int64_t)t.run * a.run_len + min((t.tile * 16 * NT + 16 * NT - 1) / a.group, a.run_len - 1), (int64_t)t.q_len - 1), (int64_t)a.Nq - 1);
    const int all = t.seen(a, first), any = t.seen(a, (int)last);
    int token[NT], sub[NT], seen[NT];
    u32x4_t q[NT][G][TERMS];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      token[c] = t.token(a, (t.tile * NT + c) * 16 + r, sub[c]);
      seen[c] = token[c] < 0 ? any : t.seen(a, token[c]);
      const T* row = static_cast<const T*>(a.q) + t.b * a.qb + (int64_t)max(token[c], 0) * a.qn + (int64_t)(t.hk * a.group + (token[c] < 0 ? 0 : sub[c])) * a.qh;
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const int ch = 8 * (G * g + i);
#pragma unroll
        for (int x = 0; x < TERMS; ++x) q[c][i][x] = u32x4_t{0, 0, 0, 0};
        if (ch < a.d && token[c] >= 0) query_parts<T, TERMS>(row + ch, q[c][i]);
      }
    }
    const int64_t head = ((int64_t)t.b * a.c.heads + t.hk) * a.c.cap;
    const uint8_t *kc = a.c.kc + head * (16 * G), *ks = a.c.ks + head * SB, *vc = a.c.vc + head * (16 * G), *vs = a.c.vs + head * SB;

    f32x4_t o[2 * G][NT];
    float mref[NT], lsum[NT], lwt[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      mref[c] = kSparseLow;
      lsum[c] = lwt[c] = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) o[i][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const unsigned steps = ((unsigned)any + 31u) / 32u;
    const unsigned lo = (unsigned)((uint64_t)steps * t.part / a.nsplit), hi = (unsigned)((uint64_t)steps * (t.part + 1) / a.nsplit);
    KeyCodes<G> kn;
    u32x4_t vn[PER];
    unsigned vsn[PER];
    auto fetch = [&](unsigned step) {
      const int key0 = (int)(step * 32), left = any - key0;
      kn.load(kc, ks, key0, any, r, g);
      const uint8_t *codes = vc + (int64_t)key0 * (16 * G), *scales = vs + (int64_t)key0 * SB;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int unit = i * 64 + lane, key = key_of(unit), group = unit % G;
        vn[i] = u32x4_t{0, 0, 0, 0};
        vsn[i] = 127u;  // what no row sees counts as zero
        if ((UNITS % 64 == 0 || unit < UNITS) && key < left) {
          vn[i] = *reinterpret_cast<const u32x4_t*>(codes + (unsigned)((key * G + group) * 16));
          vsn[i] = scales[(unsigned)(key * SB + group)];
        }
      }
    };
    if (lo + wave < hi) fetch(lo + wave);
    for (unsigned step = lo + wave; step < hi; step += 4) {
      const int key0 = (int)(step * 32);
      const KeyCodes<G> k = kn;
      u32x4_t v[PER];
      unsigned vsc[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) { v[i] = vn[i]; vsc[i] = vsn[i]; }
      if (step + 4 < hi) fetch(step + 4);

      // ---- values to LDS
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int unit = i * 64 + lane, key = key_of(unit), group = unit % G;
        if (UNITS % 64 && unit >= UNITS) continue;
        if (vsc[i] == 255u) note_nan(bad_key, group, key0 + key, v[i], vsc[i]);
#pragma unroll
        for (int p = 0; p < 4; ++p)
          *reinterpret_cast<__attribute__((address_space(3))) u32x4_t*>((size_t)(vals + key * ROW + ((4 * group + p) ^ swizzle(key)) * 16)) =
              cache4_bf16x8(v[i][p], __uint_as_float(vsc[i] << 23));
      }
      asm volatile("" ::: "memory");

      // ---- scores
      f32x4_t sc[2][NT];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < NT; ++c) sc[u][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, k.operand(u, i, g));
#pragma unroll
          for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int x = TERMS - 1; x >= 0; --x)  // the smallest part first
              sc[u][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, __builtin_bit_cast(bf16x8_t, q[c][i][x]), sc[u][c], 0, 0, 0);
        }
      if (key0 + 32 > all) {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          const int lim = seen[c] - key0 - 4 * g;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (16 * u + j >= lim) sc[u][c][j] = -INFINITY;
        }
      }

      // ---- probabilities against a reference maximum that is raised only when a partial sum has grown past it
      u32x4_t pk[NT][TERMS];
      float rs[NT], rw[NT];
      auto exponentiate = [&]() {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          rs[c] = rw[c] = 0.f;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
              const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[u][c][j], a.scale_log2, -mref[c])), p1 = __builtin_amdgcn_exp2f(fmaf(sc[u][c][j + 1], a.scale_log2, -mref[c]));
              unsigned w[TERMS];
              bf16_parts<TERMS>(p0, p1, w);
#pragma unroll
              for (int x = 0; x < TERMS; ++x) pk[c][x][2 * u + j / 2] = w[x];
              if constexpr (TERMS == 1) rs[c] = dot2_ones(w[0], rs[c]);
              rw[c] += p0 + p1;
            }
          if constexpr (TERMS > 1) rs[c] = rw[c];
        }
      };
      exponentiate();
      bool grown = false;
#pragma unroll
      for (int c = 0; c < NT; ++c) grown = grown || !(rs[c] <= kSparseTrigger);
      if (__builtin_amdgcn_ballot_w64(grown) != 0) {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          float mx = sc[0][c][0];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) mx = fmaxf(mx, sc[u][c][j]);
          mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
          mx = fmaxf(mx, __shfl_xor(mx, 32, kWave)) * a.scale_log2;  // the four parts of the row agree on the new reference
          const float up = fmaxf(mx, mref[c]), alpha = __builtin_amdgcn_exp2f(mref[c] - up);
          mref[c] = up;
          lsum[c] *= alpha;
          lwt[c] *= alpha;
#pragma unroll
          for (int i = 0; i < 2 * G; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][c][j] *= alpha;
        }
        exponentiate();
      }
#pragma unroll
      for (int c = 0; c < NT; ++c) { lsum[c] += rs[c]; lwt[c] += rw[c]; }

      // ---- O^T += V^T P^T: slots e < 4 of group g are keys 4 g + e, the others 16 + 4 g + e - 4
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) {
        if (i == 2 * G - 1 && a.d <= 16 * i) break;  // no channels of the head
        const int row = 4 * g + r / 4, piece = 2 * i + (r % 4) / 2;
        const uint2 x = lds_read_tr(vals + row * ROW + (piece ^ swizzle(row)) * 16 + (r % 2) * 8);
        const uint2 y = lds_read_tr(vals + (16 + row) * ROW + (piece ^ swizzle(16 + row)) * 16 + (r % 2) * 8);
        const u32x4_t vf{x.x, x.y, y.x, y.y};
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int x2 = TERMS - 1; x2 >= 0; --x2)
            o[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vf), __builtin_bit_cast(bf16x8_t, pk[c][x2]), o[i][c], 0, 0, 0);
      }
      asm volatile("" ::: "memory");
    }
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      lsum[c] += __shfl_xor(lsum[c], 16, kWave);
      lsum[c] += __shfl_xor(lsum[c], 32, kWave);
      lwt[c] += __shfl_xor(lwt[c], 16, kWave);
      lwt[c] += __shfl_xor(lwt[c], 32, kWave);
    }

    // ---- four wavefronts' results become one: 2 and 3 into 0 and 1, then 1 into 0
    float* img = reinterpret_cast<float*>(&lds[0]) + lane;
#pragma unroll
    for (int half = 2; half >= 1; half /= 2) {
      __syncthreads();
      if (wave >= half && wave < 2 * half) {
        float* to = img + (wave - half) * KEEP * kWave;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
#pragma unroll
          for (int i = 0; i < 2 * G; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) to[((c * 2 * G + i) * 4 + j) * kWave] = o[i][c][j];
          to[(8 * G * NT + 3 * c) * kWave] = mref[c];
          to[(8 * G * NT + 3 * c + 1) * kWave] = lsum[c];
          to[(8 * G * NT + 3 * c + 2) * kWave] = lwt[c];
        }
      }
      __syncthreads();
      if (wave < half) {
        const float* from = img + wave * KEEP * kWave;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          const float m2 = from[(8 * G * NT + 3 * c) * kWave], top = fmaxf(mref[c], m2);
          const float w1 = __builtin_amdgcn_exp2f(mref[c] - top), w2 = __builtin_amdgcn_exp2f(m2 - top);
          mref[c] = top;
          lsum[c] = lsum[c] * w1 + from[(8 * G * NT + 3 * c + 1) * kWave] * w2;
          lwt[c] = lwt[c] * w1 + from[(8 * G * NT + 3 * c + 2) * kWave] * w2;
#pragma unroll
          for (int i = 0; i < 2 * G; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][c][j] = o[i][c][j] * w1 + from[((c * 2 * G + i) * 4 + j) * kWave] * w2;
        }
      }
    }
    if (wave == 0) {
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        if (token[c] < 0) continue;
        const int h = t.hk * a.group + sub[c];
        const int64_t row = ((int64_t)t.b * a.Nq + token[c]) * (a.c.heads * a.group) + h;
        const float inv = lsum[c] == 0.f ? 0.f : 1.f / lsum[c];  // a row without keys gives zero
        T* dst = static_cast<T*>(a.o) + t.b * a.ob + (int64_t)token[c] * a.on + (int64_t)h * a.oh;
#pragma unroll
        for (int i = 0; i < 2 * G; ++i) {
          const int ch = 16 * i + 4 * g;
          if (ch >= a.d) continue;
          f32x4_t y = o[i][c];
          if (seen[c] > bad_key[i / 2]) y = f32x4_t{NAN, NAN, NAN, NAN};
          if (a.nsplit > 1) {
            *reinterpret_cast<f32x4_t*>(a.part + (row * a.nsplit + t.part) * a.d + ch) = y;
            continue;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = lsum[c] == 0.f ? 0.f : y[j] * inv;
          if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst + ch) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
          else *reinterpret_cast<f32x4_t*>(dst + ch) = y;
        }
        if (g == 0) {
          if (a.nsplit > 1) a.part_stat[row * a.nsplit + t.part] = f32x4_t{mref[c], lsum[c], lwt[c], 0.f};
          else if (a.row_stat) a.row_stat[row] = row_stat(mref[c], lwt[c]);
        }
      }
    }
    __syncthreads();  // the next tile's values overwrite what was handed over
  }
}

// Rows by the hundred: tiles of 128 CT rows (float32: CT = 1), 32 CT to each of four wavefronts, that share stages of 64 keys.  A stage's codes are
// fetched into registers one stage ahead, a quarter of a key's and of a value's row to a thread, and become bf16 in LDS while
// the stage before is multiplied.
// W: the sums of the unrounded weights are wanted too; float32's are those.
// 9216 tokens of 5 heads of 64 over 64512 slots, two batch entries: 1559 us, 976 TFLOP/s; matrix cores 40 % and vector ALUs 57 % of the cycles,
// at 2.33 of 2.4 GHz.  The two add up to nearly all of them, as matrix and vector time does on this chip: fewer vector instructions would
// help, and other orders of them do not: with wavefronts of 32 rows at twice the number (four per SIMD), with keys read a piece ahead, without the
// scheduling barriers it takes 1575 to 1650, with products and exponentials of neighbouring pieces interleaved instruction by
// instruction 1960.  Heads of 96 and 128: 850 and 800 to 860 TFLOP/s.
// float32, 4050 rows of 8 heads of 80 over 14175 slots: 363 us, 376 TFLOP/s of the operation's own, 1130 with the three parts; matrix cores
// 58 %, vector ALUs 53 %, at 2.12 GHz (the kernel above, which converts codes anew for every 32 rows, 395, 45 % and 60 %).  Pieces of two tiles
// save nothing with the registers of three parts (371 us).
template <typename T, int G, int CT, bool W>
__global__ __launch_bounds__(256, sizeof(T) == 2 && G == 1 && CT == 1 ? 3 : 2) void cache4_attn_many_kernel(CacheAttnArgs a) {
  using Geo = SparseGeo<bf16, 2 * G, 4>;  // rows of LDS and their swizzle
  constexpr int ROW = Geo::ROW, HALF = 64 * ROW, KS = 2 * G, SB = cache4_scale_bytes(G);
  constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;
  constexpr int UT = CT == 1 && G < (TERMS > 1 ? 2 : 4) ? 2 : 1;  // 32-key tiles that are in work together, as far as registers go
  __shared__ __align__(1024) u32x4_t ring[4 * HALF / 16];
  __shared__ int bad_key[4];
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) void*)(&ring[0]);
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % 32, g = lane / 32;
  // LDS addresses of the first fragments, as in k_attn_sparse.h
  const unsigned kat = lds0 + r * ROW + (g ^ Geo::swizzle(r)) * 16;  // piece 2 s + g: ^ 32 s
  const int vr = 4 * g + (lane % 16) / 4;
  const unsigned vat = lds0 + HALF + vr * ROW + ((2 * ((lane / 16) % 2) + (lane % 4) / 2) ^ Geo::swizzle(vr)) * 16 + (lane % 2) * 8;
  // This thread's part of a stage: 8 G channels of one key.  The keys are dealt out so that 16 lanes' pieces fall on different banks.
  const int n = threadIdx.x / 4, quarter = threadIdx.x % 4;
  const int key = G >= 3 ? (n & 3) << 2 | ((n >> 2) & 3) | (n & 48) : G == 2 ? (n & 1) | (n & 2) << 2 | (n & 12) >> 1 | (n & 48) : n;
  const unsigned wat = lds0 + key * ROW;
  const unsigned code_at = key * (16 * G) + quarter * (4 * G), scale_at = key * SB;

  const unsigned chunk = (a.work + 7) / 8;  // contiguous per XCD
  const unsigned chunk_end = min(a.work, (blockIdx.x % 8 + 1) * chunk);
  for (unsigned work = blockIdx.x % 8 * chunk + blockIdx.x / 8; work < chunk_end; work += gridDim.x / 8) {
    const CacheTile t(a, work);
    int first_sub;
    const int rho0 = t.tile * 128 * CT, first = t.token(a, rho0, first_sub);
    if (first < 0) continue;
    if (threadIdx.x < 4) bad_key[threadIdx.x] = INT32_MAX;
    const int64_t last = min(min((int64_t)t.run * a.run_len + min((rho0 + 128 * CT - 1) / a.group, a.run_len - 1), (int64_t)t.q_len - 1), (int64_t)a.Nq - 1);
    const int all = t.seen(a, first), any = t.seen(a, (int)last);
    int token[CT], sub[CT], seen[CT];
    u32x4_t q[CT][KS][TERMS];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      token[c] = t.token(a, rho0 + (wave * CT + c) * 32 + r, sub[c]);
      seen[c] = token[c] < 0 ? any : t.seen(a, token[c]);
      const T* row = static_cast<const T*>(a.q) + t.b * a.qb + (int64_t)max(token[c], 0) * a.qn + (int64_t)(t.hk * a.group + (token[c] < 0 ? 0 : sub[c])) * a.qh;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int ch = 16 * s + 8 * g;
#pragma unroll
        for (int x = 0; x < TERMS; ++x) q[c][s][x] = u32x4_t{0, 0, 0, 0};
        if (ch < a.d && token[c] >= 0) query_parts<T, TERMS>(row + ch, q[c][s]);
      }
    }
    const int64_t head = ((int64_t)t.b * a.c.heads + t.hk) * a.c.cap;
    const uint8_t *kc = a.c.kc + head * (16 * G), *ks = a.c.ks + head * SB, *vc = a.c.vc + head * (16 * G), *vs = a.c.vs + head * SB;
    const unsigned stages = ((unsigned)any + 63u) / 64u;
    const unsigned lo = (unsigned)((uint64_t)stages * t.part / a.nsplit), hi = (unsigned)((uint64_t)stages * (t.part + 1) / a.nsplit);

    unsigned kn[G], vn[G], ksn, vsn;
    auto fetch = [&](unsigned st) {
      const int key0 = (int)(st * 64), left = any - key0;
      const bool in = key < left;
      auto words = [&](const uint8_t* p, unsigned (&w)[G]) {
        if constexpr (G == 4) {
          const u32x4_t v = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = v[i];
        } else if constexpr (G == 2) {
          const uint2 v = *reinterpret_cast<const uint2*>(p);
          w[0] = v.x; w[1] = v.y;
        } else {
#pragma unroll
          for (int i = 0; i < G; ++i) w[i] = reinterpret_cast<const unsigned*>(p)[i];
        }
      };
      auto scale = [&](const uint8_t* p) -> unsigned {
        if constexpr (SB == 4) return *reinterpret_cast<const unsigned*>(p);
        else if constexpr (SB == 2) return *reinterpret_cast<const unsigned short*>(p);
        else return *p;
      };
      ksn = vsn = 0x7F7F7F7Fu;  // what no row sees counts as zero
#pragma unroll
      for (int i = 0; i < G; ++i) kn[i] = vn[i] = 0u;
      if (in) {
        words(kc + (int64_t)key0 * (16 * G) + code_at, kn);
        ksn = scale(ks + (int64_t)key0 * SB + scale_at);
        words(vc + (int64_t)key0 * (16 * G) + code_at, vn);
        vsn = scale(vs + (int64_t)key0 * SB + scale_at);
      }
    };
    auto place = [&](unsigned st, unsigned slot) {  // the fetched codes, as bf16
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const unsigned group = G == 4 ? quarter : G == 2 ? quarter / 2 : G == 1 ? 0 : (3 * quarter + i) / 4;
        const unsigned kscale = (ksn >> (8 * group)) & 255u;
        unsigned vscale = (vsn >> (8 * group)) & 255u, vw = vn[i];
        if (vscale == 255u) {
          u32x4_t none;
          note_nan(bad_key, group, (int)(st * 64) + key, none, vscale);
          vw = 0u;
        }
        const unsigned at = wat + slot + ((G * quarter + i) ^ Geo::swizzle(key)) * 16;
        *reinterpret_cast<__attribute__((address_space(3))) u32x4_t*>((size_t)at) = cache4_bf16x8(kn[i], __uint_as_float(kscale << 23));
        *reinterpret_cast<__attribute__((address_space(3))) u32x4_t*>((size_t)(at + HALF)) = cache4_bf16x8(vw, __uint_as_float(vscale << 23));
      }
    };

    f32x16_t o[CT][G];
    float mref[CT], lsum[CT], lwt[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      mref[c] = kSparseLow;
      lsum[c] = lwt[c] = 0.f;
#pragma unroll
      for (int i = 0; i < G; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[c][i][e] = 0.f;
    }
    unsigned slot = 0;
    __syncthreads();  // bad_key
    if (lo < hi) {
      fetch(lo);
      place(lo, 0);
      if (lo + 1 < hi) fetch(lo + 1);
    }
    __syncthreads();
    for (unsigned st = lo; st < hi; ++st) {
      if (st + 1 < hi) {
        place(st + 1, slot ^ (2 * HALF));
        if (st + 2 < hi) fetch(st + 2);
      }
#pragma unroll
      for (int part = 0; part < 2 / UT; ++part) {
        const unsigned at = slot + part * 32 * UT * ROW;
        u32x4_t kf[KS][UT];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int u = 0; u < UT; ++u) kf[s][u] = lds_read<u32x4_t>(((kat + at) ^ (32 * s)) + 32 * u * ROW);
        __builtin_amdgcn_sched_barrier(0);
        f32x16_t sc[CT][UT];
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
          for (int u = 0; u < UT; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[c][u][e] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          if (TERMS > 1 && s == KS - 1 && a.d <= 16 * s) break;  // no channels of the head: three products less (bf16 multiplies one with zeros)
#pragma unroll
          for (int u = 0; u < UT; ++u)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
              for (int x = TERMS - 1; x >= 0; --x)  // the smallest part first
                sc[c][u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[s][u]), __builtin_bit_cast(bf16x8_t, q[c][s][x]), sc[c][u], 0, 0, 0);
        }
        const int key0 = (int)(st * 64) + part * 32 * UT;
        if (key0 + 32 * UT > all) {
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            const int lim = seen[c] - key0 - 4 * g;  // register e of tile u is key 32 u + 8 (e / 4) + e % 4 + 4 g
#pragma unroll
            for (int u = 0; u < UT; ++u)
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if (32 * u + 8 * (e / 4) + e % 4 >= lim) sc[c][u][e] = -INFINITY;
          }
        }
        // the values are on their way while the exponentials are taken
        uint2 vlo[2 * UT][G], vhi[2 * UT][G];
#pragma unroll
        for (int k16 = 0; k16 < 2 * UT; ++k16)
#pragma unroll
          for (int i = 0; i < G; ++i) {
            vlo[k16][i] = lds_read_tr(((vat + at) ^ (64 * i)) + 16 * k16 * ROW);
            vhi[k16][i] = lds_read_tr(((vat + at) ^ (64 * i) ^ (Geo::swizzle(8) * 16)) + (16 * k16 + 8) * ROW);
          }
        __builtin_amdgcn_sched_barrier(0);

        // ---- probabilities, as in the kernel above
        u32x4_t pk[CT][2 * UT][TERMS];
        float rs[CT], rw[CT];
        auto exponentiate = [&]() {
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            rs[c] = rw[c] = 0.f;
#pragma unroll
            for (int u = 0; u < UT; ++u)
#pragma unroll
              for (int e = 0; e < 16; e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[c][u][e], a.scale_log2, -mref[c])), p1 = __builtin_amdgcn_exp2f(fmaf(sc[c][u][e + 1], a.scale_log2, -mref[c]));
                unsigned w[TERMS];
                bf16_parts<TERMS>(p0, p1, w);
#pragma unroll
                for (int x = 0; x < TERMS; ++x) pk[c][2 * u + e / 8][x][e % 8 / 2] = w[x];
                if constexpr (TERMS == 1) rs[c] = dot2_ones(w[0], rs[c]);
                else rs[c] += p0 + p1;
                if constexpr (W) rw[c] += p0 + p1;
              }
          }
        };
        exponentiate();
        bool grown = false;
#pragma unroll
        for (int c = 0; c < CT; ++c) grown = grown || !(rs[c] <= kSparseTrigger);
        if (__builtin_amdgcn_ballot_w64(grown) != 0) {
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            float mx = sc[c][0][0];
#pragma unroll
            for (int u = 0; u < UT; ++u)
#pragma unroll
              for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[c][u][e]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, kWave)) * a.scale_log2;
            const float up = fmaxf(mx, mref[c]), alpha = __builtin_amdgcn_exp2f(mref[c] - up);
            mref[c] = up;
            lsum[c] *= alpha;
            if constexpr (W) lwt[c] *= alpha;
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
              for (int e = 0; e < 16; ++e) o[c][i][e] *= alpha;
          }
          exponentiate();
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          lsum[c] += rs[c];
          if constexpr (W) lwt[c] += rw[c];
        }

        // ---- O^T += V^T P^T
#pragma unroll
        for (int k16 = 0; k16 < 2 * UT; ++k16)
#pragma unroll
          for (int i = 0; i < G; ++i) {
            const u32x4_t vf{vlo[k16][i].x, vlo[k16][i].y, vhi[k16][i].x, vhi[k16][i].y};
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
              for (int x = TERMS - 1; x >= 0; --x)
                o[c][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf), __builtin_bit_cast(bf16x8_t, pk[c][k16][x]), o[c][i], 0, 0, 0);
          }
      }
      slot ^= 2 * HALF;
      __syncthreads();
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      lsum[c] += __shfl_xor(lsum[c], 32, kWave);
      lwt[c] = W ? lwt[c] + __shfl_xor(lwt[c], 32, kWave) : lsum[c];
      if (token[c] < 0) continue;
      const int h = t.hk * a.group + sub[c];
      const int64_t row = ((int64_t)t.b * a.Nq + token[c]) * (a.c.heads * a.group) + h;
      const float inv = lsum[c] == 0.f ? 0.f : 1.f / lsum[c];  // a row without keys gives zero
      T* dst = static_cast<T*>(a.o) + t.b * a.ob + (int64_t)token[c] * a.on + (int64_t)h * a.oh;
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const bool bad = seen[c] > bad_key[i];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const int ch = 32 * i + 8 * p + 4 * g;
          if (ch >= a.d) continue;
          f32x4_t y{o[c][i][4 * p], o[c][i][4 * p + 1], o[c][i][4 * p + 2], o[c][i][4 * p + 3]};
          if (bad) y = f32x4_t{NAN, NAN, NAN, NAN};
          if (a.nsplit > 1) {
            *reinterpret_cast<f32x4_t*>(a.part + (row * a.nsplit + t.part) * a.d + ch) = y;
            continue;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = lsum[c] == 0.f ? 0.f : y[j] * inv;
          if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst + ch) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
          else *reinterpret_cast<f32x4_t*>(dst + ch) = y;
        }
      }
      if (g == 0) {
        if (a.nsplit > 1) a.part_stat[row * a.nsplit + t.part] = f32x4_t{mref[c], lsum[c], lwt[c], 0.f};
        else if (a.row_stat) a.row_stat[row] = row_stat(mref[c], lwt[c]);
      }
    }
    __syncthreads();  // bad_key and the ring are the next tile's
  }
}

// The shares of a query row joined: weights 2^(m - max m).  92160 rows of 7 shares: 36 us, HBM.  A wavefront per row: its lanes hold one share's maximum and sums
// each (nsplit <= 64), then 64 / (d / 4) shares' outputs at a time, four channels per lane; the order of the sums is fixed.
template <typename T>
__global__ __launch_bounds__(256) void cache4_join_kernel(CacheAttnArgs a, int rows) {
  const int lane = threadIdx.x % kWave, heads = a.c.heads * a.group, quads = a.d / 4;
  // lanes of one share: the next power of two of quads
  const int width = quads <= 2 ? 2 : quads <= 4 ? 4 : quads <= 8 ? 8 : quads <= 16 ? 16 : 32, at_once = kWave / width;
  const int quad = lane % width, which = lane / width;
  const int row = (int)blockIdx.x * 4 + threadIdx.x / kWave;
  if (row >= rows) return;
  const int bn = row / heads;
  const int h = row - bn * heads, b = bn / a.Nq, token = bn - b * a.Nq;
  if (a.q_len && token >= a.q_len[b]) return;
  const f32x4_t stat = lane < a.nsplit ? a.part_stat[(int64_t)row * a.nsplit + lane] : f32x4_t{kSparseLow, 0.f, 0.f, 0.f};
  const float top = wave_max(stat[0]), w = __builtin_amdgcn_exp2f(stat[0] - top);
  const float l = wave_sum(stat[1] * w), lw = wave_sum(stat[2] * w);
  const float* src = a.part + (int64_t)row * a.nsplit * a.d + 4 * quad;
  f32x4_t o{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.nsplit; s0 += 4 * at_once) {
    f32x4_t x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = s0 + u * at_once + which;
      x[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (s < a.nsplit && quad < quads) x[u] = *reinterpret_cast<const f32x4_t*>(src + (int64_t)s * a.d);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float ws = __shfl(w, (s0 + u * at_once + which) % kWave, kWave);  // past the last share: times zero
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = fmaf(x[u][j], ws, o[j]);
    }
  }
  for (int step = width; step < kWave; step <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += __shfl_xor(o[j], step, kWave);
  if (a.row_stat && lane == 0) a.row_stat[row] = row_stat(top, lw);
  if (which != 0 || quad >= quads) return;
  const float inv = 1.f / l;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = l == 0.f ? 0.f : o[j] * inv;
  T* dst = static_cast<T*>(a.o) + b * a.ob + (int64_t)token * a.on + (int64_t)h * a.oh + 4 * quad;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
  else *reinterpret_cast<f32x4_t*>(dst) = o;
}

constexpr int kWeightTiles = 2;  // of 32 keys, that a wavefront of the kernel for many rows keeps (1, 3 and 4 are up to 4 % slower)

struct CacheWeightArgs {
  const void* q;
  int64_t qb, qn, qh;
  Cache4View c;
  const int *q_len, *k_len;
  int Nq, group, d, run;
  int chunks;                // pieces of a head's keys: of 128 kWeightTiles, or shares
  unsigned work;             // B * heads * chunks
  float scale_log2, decay;
  const float2* row_stat;
  const float* in;           // or NULL: zeros
  float* out;
};

// out[key] = decay in[key] + sum over the rows that see it of their softmax weight, in an order that depends on sizes only.  The scores are
// taken again, against the rows' maxima and sums of the whole call: keys come from memory a second time, where keeping
// the scores would write and read 8 bytes of every row.
//   S[row, key] = Q K^T         row operand: rows, column operand: keys
// Up to 16 NT rows, kept as operands with their statistics; a wavefront walks every fourth step of 32 keys of its workgroup's share.  32 rows, 57600
// slots and fewer of 8 heads of 128, two batch entries: 61 MB in 22 us.
template <typename T, int G, int NT>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? (NT == 1 ? 4 : 3) : 2) void cache4_weight_few_kernel(CacheWeightArgs a) {
  constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;
  constexpr int SB = cache4_scale_bytes(G);
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % 16, g = lane / 16;
  const unsigned part = (a.work + 7) / 8, part_end = min(a.work, (blockIdx.x % 8 + 1) * part);
  for (unsigned work = blockIdx.x % 8 * part + blockIdx.x / 8; work < part_end; work += gridDim.x / 8) {
    const unsigned bh = work / (unsigned)a.chunks, share = work % (unsigned)a.chunks;
    const int b = (int)(bh / (unsigned)a.c.heads), hk = (int)(bh % (unsigned)a.c.heads), heads = a.c.heads * a.group;
    const int q_len = a.q_len ? min(max(a.q_len[b], 0), a.Nq) : a.Nq, k_len = a.k_len ? min(max(a.k_len[b], 0), a.c.cap) : a.c.cap;
    const unsigned steps = ((unsigned)k_len + 31u) / 32u;
    const unsigned lo = (unsigned)((uint64_t)steps * share / (unsigned)a.chunks), hi = (unsigned)((uint64_t)steps * (share + 1) / (unsigned)a.chunks);
    if (lo + wave >= hi) continue;
    const int64_t head = ((int64_t)b * a.c.heads + hk) * a.c.cap;
    const uint8_t *codes = a.c.kc + head * (16 * G), *scales = a.c.ks + head * SB;
    KeyCodes<G> kn;
    kn.load(codes, scales, (int)((lo + wave) * 32), k_len, r, g);
    const int rows = q_len * a.group;
    u32x4_t q[NT][G][TERMS];
    float2 stat[NT][4];
    int seen[NT][4], all = k_len;  // keys that every row sees
#pragma unroll
    for (int c = 0; c < NT; ++c) {
      const int rho = 16 * c + r, n = rho / a.group, h = hk * a.group + rho - n * a.group;
      const T* row = static_cast<const T*>(a.q) + b * a.qb + (int64_t)n * a.qn + (int64_t)h * a.qh;
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const int ch = 8 * (G * g + i);
#pragma unroll
        for (int x = 0; x < TERMS; ++x) q[c][i][x] = u32x4_t{0, 0, 0, 0};
        if (ch < a.d && rho < rows) query_parts<T, TERMS>(row + ch, q[c][i]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // of row 4 g + j, as the scores lie
        const int of = 16 * c + 4 * g + j, token = of / a.group;
        stat[c][j] = make_float2(INFINITY, 0.f);  // no row: 2^-inf
        seen[c][j] = 0;
        if (of < rows) {
          stat[c][j] = a.row_stat[((int64_t)b * a.Nq + token) * heads + hk * a.group + of - token * a.group];
          seen[c][j] = CacheTile::cache_seen(a.run, token, q_len, k_len);
        }
      }
    }
    if (rows < 16 * NT) all = 0;
    else if (a.run) all = CacheTile::cache_seen(a.run, 0, q_len, k_len);
    for (unsigned step = lo + wave; step < hi; step += 4) {
      const int key0 = (int)(step * 32);
      const KeyCodes<G> k = kn;
      if (step + 4 < hi) kn.load(codes, scales, key0 + 128, k_len, r, g);
      float total[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        bf16x8_t kf[G];
#pragma unroll
        for (int i = 0; i < G; ++i) kf[i] = __builtin_bit_cast(bf16x8_t, k.operand(u, i, g));
        f32x4_t sc[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) sc[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
          for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int x = TERMS - 1; x >= 0; --x)  // the smallest part first
              sc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, q[c][i][x]), kf[i], sc[c], 0, 0, 0);
        float p[NT][4];
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int j = 0; j < 4; ++j) p[c][j] = __builtin_amdgcn_exp2f(fmaf(sc[c][j], a.scale_log2, -stat[c][j].x));
        if (key0 + 32 > all) {
#pragma unroll
          for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (key0 + 16 * u + r >= seen[c][j]) p[c][j] = 0.f;
        }
        float t = 0.f;
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int j = 0; j < 4; ++j) t = fmaf(p[c][j], stat[c][j].y, t);
        t += __shfl_xor(t, 16, kWave);
        total[u] = t + __shfl_xor(t, 32, kWave);
      }
      const int key = key0 + lane;  // lanes of the first two groups write a tile's keys each
      if (lane < 32 && key < k_len) a.out[head + key] = (a.in ? a.decay * a.in[head + key] : 0.f) + (g == 0 ? total[0] : total[1]);
    }
  }
}

// The same for more rows.  A wavefront keeps 32 KT keys as bf16 column operands and walks the rows in tiles of 32 that the
// workgroup's four share in LDS (direct global->LDS loads, one tile ahead), with their statistics.  A lane holds one key of every 32, so that a
// sum over the rows is one register.  Bound by the vector ALUs: an fma, an exponential and an fma for every score, beside 2 G
// matrix instructions of 32 clocks for 16 of a lane's.  A row's statistics, and the address of a wavefront's first load of a tile, are found by
// steps from tile to tile, without a division; bfloat16 heads of up to 64 channels and float32 ones of up to 32 have that load only, others
// divide for the second to fourth.
// 1024 rows over 26624 slots of 10 heads of 64, two batch entries: 122 us (every key's sum in registers of its own: 134; with divisions: 155).
// Rows are not dealt out to workgroups: short caches leave most of the chip idle (747 tokens of 16 heads over 747 slots of 2, two batch
// entries: 149 us in 12 workgroups).
// Equal rows give a key the same number again and again, and a running sum then rounds the same way every time: 73728 of them were 5e-4 of the
// weight off.  A lane's 16 terms of a tile are added up first, and collected with what every rounding added (Kahan's compensated summation):
// 4 additions for 48 instructions, below what the time can tell.
template <typename T, int G>
__global__ __launch_bounds__(256, sizeof(T) == 2 && G <= 2 ? 3 : 2) void cache4_weight_many_kernel(CacheWeightArgs a) {
  using Geo = SparseGeo<T, 2 * G, 4>;
  constexpr int KT = kWeightTiles, TERMS = sizeof(T) == 2 ? 1 : 3;
  constexpr int ROW = Geo::ROW, TILE = 32 * ROW, KS = 2 * G, SB = cache4_scale_bytes(G);
  constexpr int LOADS = TILE / 4096 > 0 ? TILE / 4096 : 1;  // of a wavefront and tile, 1 KiB each; tiles of 2 KiB leave two wavefronts without
  __shared__ __align__(1024) u32x4_t ring[2 * TILE / 16];
  __shared__ __align__(16) float maxima[2][32], factors[2][32];
  __shared__ __align__(16) int ends[2][32];
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) void*)(&ring[0]);
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % 32, g = lane / 32, heads = a.c.heads * a.group;
  // piece 2 s + g (float32: pieces 4 s + 2 g and one more) of row r: ^ 32 s (^ 64 s, and ^ 16)
  const unsigned qat = lds0 + r * ROW + ((sizeof(T) == 2 ? g : 2 * g) ^ Geo::swizzle(r)) * 16;
  const int step_n = 32 / a.group, step_sub = 32 % a.group;          // from a tile to the next
  // Row rho of a key head, as a token and one of its query heads, and an offset that grows with both.
  struct Row {
    int rho, n, sub;
    int64_t at;
    __device__ __forceinline__ Row(int rho_, int group, int64_t per_token, int64_t per_head) : rho(rho_) {
      n = group > 1 ? rho / group : rho;
      sub = rho - n * group;
      at = n * per_token + sub * per_head;
    }
    __device__ __forceinline__ void step(int group, int dn, int s, int64_t per_token, int64_t per_head) {
      rho += 32;
      n += dn;
      sub += s;
      at += dn * per_token + s * per_head;
      if (sub >= group) {
        sub -= group;
        ++n;
        at += per_token - group * per_head;
      }
    }
  };
  const unsigned part = (a.work + 7) / 8, part_end = min(a.work, (blockIdx.x % 8 + 1) * part);
  for (unsigned work = blockIdx.x % 8 * part + blockIdx.x / 8; work < part_end; work += gridDim.x / 8) {
    const unsigned bh = work / (unsigned)a.chunks;
    const int b = (int)(bh / (unsigned)a.c.heads), hk = (int)(bh % (unsigned)a.c.heads);
    const int q_len = a.q_len ? min(max(a.q_len[b], 0), a.Nq) : a.Nq, k_len = a.k_len ? min(max(a.k_len[b], 0), a.c.cap) : a.c.cap;
    const int64_t first_key = (int64_t)(work % (unsigned)a.chunks) * (128 * KT);
    if (first_key >= k_len) continue;
    const int key0 = (int)first_key + wave * 32 * KT, last_key = (int)min(first_key + 128 * KT, (int64_t)k_len);  // behind the workgroup's last
    const int64_t head = ((int64_t)b * a.c.heads + hk) * a.c.cap;

    // ---- this wavefront's keys: tile u, step s: channels 16 s + 8 g .. + 7 of key 32 u + r
    u32x4_t kf[KT][KS];
#pragma unroll
    for (int u = 0; u < KT; ++u) {
      const int64_t key = head + min(key0 + 32 * u + r, k_len - 1);
      const uint8_t* codes = a.c.kc + key * (16 * G);
#pragma unroll
      for (int s = 0; s < KS; ++s)
        kf[u][s] = cache4_bf16x8(*reinterpret_cast<const unsigned*>(codes + (16 * s + 8 * g) / 2), __uint_as_float((unsigned)a.c.ks[key * SB + s / 2] << 23));
    }
    float sum[KT], over[KT];  // over: what the roundings have added to sum
#pragma unroll
    for (int u = 0; u < KT; ++u) sum[u] = over[u] = 0.f;

    // ---- rows: q_len tokens times `group` heads; the first that see one of these keys
    const int rows = q_len * a.group;
    int begin = 0;
    if (a.run) {
      // token n sees key j iff the end of its run, min((n / run + 1) run, q_len), is beyond j + q_len - k_len
      const int64_t over = first_key + q_len - k_len;
      begin = over < 0 ? 0 : (int)(over / a.run * a.run) * a.group;
    }
    const int tiles = rows > begin ? (rows - begin + 31) / 32 : 0;
    // what a wavefront's loads bring: rows of 16-byte pieces, by neighbouring lanes
    const T* q0 = static_cast<const T*>(a.q) + b * a.qb + (int64_t)hk * a.group * a.qh;
    auto load_row = [&](int l) { return (wave + 4 * l) * (64 / Geo::PR) + lane / Geo::PR; };
    auto load_piece = [&](int l) {
      const int at = (lane % Geo::PR) ^ Geo::swizzle(load_row(l));
      return at * Geo::VEC < a.d ? at * Geo::VEC : 0;
    };
    Row of(begin + load_row(0), a.group, a.qn, a.qh);
    Row mine(begin + r, a.group, heads, 1);  // whose statistics the first wavefront's lanes bring
    const float2* stat0 = a.row_stat + (int64_t)b * a.Nq * heads + hk * a.group;
    float2 stat = make_float2(INFINITY, 0.f);
    int end = 0;
    auto issue = [&](unsigned slot) {
      if (wave == 0) {
        stat = stat0[mine.rho < rows ? mine.at : 0];
        end = CacheTile::cache_seen(a.run, mine.n, q_len, k_len);
        if (mine.rho >= rows) {  // no row: 2^-inf
          stat = make_float2(INFINITY, 0.f);
          end = 0;
        }
        mine.step(a.group, step_n, step_sub, heads, 1);
      }
#pragma unroll
      for (int l = 0; l < LOADS; ++l) {
        const Row row = l == 0 ? of : Row(of.rho + load_row(l) - load_row(0), a.group, a.qn, a.qh);
        if (TILE >= 4096 || wave * 1024 < TILE)
          load_to_lds(q0 + (row.rho < rows ? row.at : 0) + load_piece(l), lds0 + slot * TILE + (wave + 4 * l) * 1024);
      }
      of.step(a.group, step_n, step_sub, a.qn, a.qh);
    };
    auto put_stat = [&](unsigned slot) {
      if (wave == 0 && g == 0) {
        maxima[slot][r] = stat.x;
        factors[slot][r] = stat.y;
        ends[slot][r] = end;
      }
    };
    __syncthreads();  // nobody reads the ring of the piece before
    if (tiles > 0) {
      issue(0);
      put_stat(0);
    }
    for (int i = 0; i < tiles; ++i) {
      const int slot = i & 1;
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // tile i
      __syncthreads();
      if (i + 1 < tiles) issue(slot ^ 1);
      u32x4_t qf[KS][TERMS];
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        if constexpr (TERMS == 1) {
          qf[s][0] = lds_read<u32x4_t>((qat ^ (32 * s)) + slot * TILE);
        } else {
          query_parts(lds_read<f32x4_t>((qat ^ (64 * s)) + slot * TILE), lds_read<f32x4_t>((qat ^ (64 * s) ^ 16) + slot * TILE), qf[s]);
        }
      }
      if (a.d < 32 * G) {  // channels past the head
#pragma unroll
        for (int s = KS - 2; s < KS; ++s)
          if (16 * s + 8 * g >= a.d)
#pragma unroll
            for (int x = 0; x < TERMS; ++x) qf[s][x] = u32x4_t{0, 0, 0, 0};
      }
      f32x4_t top[4], factor[4];  // of rows 8 p + 4 g + j, as registers 4 p + j of the scores lie
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        top[p] = *reinterpret_cast<const f32x4_t*>(&maxima[slot][8 * p + 4 * g]);
        factor[p] = *reinterpret_cast<const f32x4_t*>(&factors[slot][8 * p + 4 * g]);
      }
      f32x16_t sc[KT];
#pragma unroll
      for (int u = 0; u < KT; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[u][e] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int x = TERMS - 1; x >= 0; --x)  // the smallest part first
#pragma unroll
          for (int u = 0; u < KT; ++u)
            sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, qf[s][x]), __builtin_bit_cast(bf16x8_t, kf[u][s]), sc[u], 0, 0, 0);
#pragma unroll
      for (int u = 0; u < KT; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[u][e] = __builtin_amdgcn_exp2f(fmaf(sc[u][e], a.scale_log2, -top[e / 4][e % 4]));
      // Is one of these rows behind the last, or is there one, then the first, that does not see all of the workgroup's keys?
      if (begin + 32 * i + 32 > rows || (a.run && __builtin_amdgcn_readfirstlane(ends[slot][0]) < last_key)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int lim = ends[slot][8 * (e / 4) + 4 * g + e % 4] - key0 - r;
#pragma unroll
          for (int u = 0; u < KT; ++u)
            if (32 * u >= lim) sc[u][e] = 0.f;
        }
      }
      float of_tile[KT];
#pragma unroll
      for (int u = 0; u < KT; ++u) of_tile[u] = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int u = 0; u < KT; ++u) of_tile[u] = fmaf(sc[u][e], factor[e / 4][e % 4], of_tile[u]);
#pragma unroll
      for (int u = 0; u < KT; ++u) {
        const float more = of_tile[u] - over[u], up = sum[u] + more;
        over[u] = (up - sum[u]) - more;
        sum[u] = up;
      }
      if (i + 1 < tiles) put_stat(slot ^ 1);
    }
#pragma unroll
    for (int u = 0; u < KT; ++u) {
      const float total = sum[u] + __shfl_xor(sum[u], 32, kWave);
      const int key = key0 + 32 * u + r;
      if (g == 0 && key < k_len) a.out[head + key] = (a.in ? a.decay * a.in[head + key] : 0.f) + total;
    }
  }
}

}  // namespace si

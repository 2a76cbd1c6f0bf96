// Key blocks for runs of queries by a cheap score: the product of the run's mean query and the block's mean key.
//
//   block_means_kernel   means over the rows of a run / block (and the heads that share a key / value head), float64
//   block_select_kernel  scores of 16 runs against every block on the float64 matrix cores, kept in LDS; then, per run,
//                        the `keep` largest, ties to the lowest block, as a bitmap
//
// Everything behind the loads is float64: which block is the last one kept can hang on any digit of its score, and the
// result is discrete.  The means are bound by HBM: every query and key is read once, 57600 tokens of 10 heads of 64, two batch
// entries (295 MB), in 50 us (5.9 TB/s).  The scores take 2 d flop per (run, block) at some 60 TFLOP/s (450 runs x 900 blocks x
// 20 heads: 16 us of matrix cores); the second kernel's 81 us there are latency: one workgroup fills a CU's LDS with the scores
// of 16 runs, about half of the time goes to fetching means from the L2 and the rest to the search for the threshold.  2032
// blocks, 1016 runs of 4 heads: 177 us a call; 16384 blocks, 8192 runs: 15.7 ms, with one run to a workgroup, whose search a
// single wavefront walks.  Means laid out as the
// matrix cores' fragments made that kernel 15 us shorter and the first one 7 longer, and calls of one frame 6 % slower; means of
// the next blocks fetched ahead of the products made it 10 us longer.
#pragma once
#include "k_rope.h"
#include "k_select_search.h"

#include <type_traits>

namespace si {

typedef double f64x2_t __attribute__((ext_vector_type(2)));
typedef double f64x4_t __attribute__((ext_vector_type(4)));

constexpr int kMeanPieces = 32, kMeanSlices = 8;  // 16-byte pieces of a row x rows in flight of one workgroup

struct MeansOf {
  HeadsView x;
  const int* len;
  double* out;  // [B][heads_kv][runs][d]
  int N, group, block, runs;
  unsigned work;   // B * runs * chunks
};
struct MeansArgs {
  MeansOf of[2];   // queries in runs, keys in blocks: one launch
  int heads_kv, d;
  int chunks;      // of kMeanPieces pieces of a row
};

template <typename T>
__global__ __launch_bounds__(kMeanPieces* kMeanSlices) void block_means_kernel(MeansArgs args) {
  constexpr int VEC = 16 / sizeof(T);
  __shared__ double part[kMeanSlices][kMeanPieces][VEC];
  const int px = threadIdx.x % kMeanPieces, slice = threadIdx.x / kMeanPieces;
  const int per_head = args.d / VEC;
  for (unsigned w = blockIdx.x; w < args.of[0].work + args.of[1].work; w += gridDim.x) {
    const bool keys = w >= args.of[0].work;
    const MeansOf& a = args.of[keys ? 1 : 0];
    const unsigned work = keys ? w - args.of[0].work : w, br = work / (unsigned)args.chunks;
    const int chunk = (int)(work - br * args.chunks), b = (int)(br / (unsigned)a.runs), run = (int)(br - (unsigned)b * a.runs);
    const int item = chunk * kMeanPieces + px;
    const bool live = item < args.heads_kv * per_head;
    const int hk = live ? item / per_head : 0, ch = live ? (item - hk * per_head) * VEC : 0;
    const int len = a.len ? min(max(a.len[b], 0), a.N) : a.N;
    const int64_t n0 = (int64_t)run * a.block;
    const int rows = (int)min((int64_t)a.block, max((int64_t)0, len - n0));
    double sum[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] = 0.0;
    if (live) {
      const T* p = static_cast<const T*>(a.x.p) + b * a.x.sb + n0 * a.x.sn + (int64_t)hk * a.group * a.x.sh + ch;
      for (int s = 0; s < a.group; ++s, p += a.x.sh)
#pragma unroll 4
        for (int n = slice; n < rows; n += kMeanSlices) {
          const T* q = p + n * a.x.sn;
          if constexpr (sizeof(T) == 2) {
            const u32x4_t v = *reinterpret_cast<const u32x4_t*>(q);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              sum[2 * i] += (double)__uint_as_float(v[i] << 16);
              sum[2 * i + 1] += (double)__uint_as_float(v[i] & 0xffff0000u);
            }
          } else {
            const f32x4_t v = *reinterpret_cast<const f32x4_t*>(q);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += (double)v[i];
          }
        }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) part[slice][px][i] = sum[i];
    __syncthreads();
    const double of = rows > 0 ? (double)((int64_t)rows * a.group) : 1.0;
    for (int e = threadIdx.x; e < kMeanPieces * VEC; e += kMeanPieces * kMeanSlices) {
      const int it = chunk * kMeanPieces + e / VEC;
      if (it >= args.heads_kv * per_head) continue;
      double s = 0.0;
#pragma unroll
      for (int k = 0; k < kMeanSlices; ++k) s += part[k][e / VEC][e % VEC];
      const int h = it / per_head, c = (it - h * per_head) * VEC + e % VEC;
      a.out[(((int64_t)b * args.heads_kv + h) * a.runs + run) * args.d + c] = s / of;
    }
    __syncthreads();
  }
}

struct SelectArgs {
  const double *qm, *km;  // [B][heads_kv][runs][d], [B][heads_kv][blocks][d]
  unsigned* out;          // [B][heads_kv][runs][words]
  const int *q_len, *k_len;
  int Nq, Nk, heads_kv, d, q_block, k_block, runs, blocks, words;
  int keep, rows;         // blocks to keep; runs of a workgroup
  int pitch;              // scores of one run in LDS
  int tiles;              // of `rows` runs; a workgroup takes one tile of one (b, kv head)
  unsigned work;          // B * heads_kv * tiles
};

// v of all lanes of the wavefront joined (identity 0) by data-parallel primitives, in a scalar register.
template <class Join>
__device__ __forceinline__ unsigned lanes_join(unsigned v, Join join) {
  auto step = [&](auto ctrl, auto rows) { v = join(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, ctrl.value, rows.value, 0xf, rows.value == 0xf)); };
  using std::integral_constant;
  using All = integral_constant<int, 0xf>;
  step(integral_constant<int, 0x111>(), All());  // from lane - 1, - 2, - 4, - 8 of a row of 16
  step(integral_constant<int, 0x112>(), All());
  step(integral_constant<int, 0x114>(), All());
  step(integral_constant<int, 0x118>(), All());
  step(integral_constant<int, 0x142>(), integral_constant<int, 0xa>());  // the last lane of row 0 to row 1, of row 2 to row 3
  step(integral_constant<int, 0x143>(), integral_constant<int, 0xc>());  // lane 31 to rows 2 and 3
  return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}

// CAP: scores (float64) of a workgroup in LDS.  KPL: keys of a run per lane in registers (64 KPL >= blocks), or 0: read from
// LDS every time.  NC: channels in steps of 32, so that all loads of a tile's means are in flight before its products.
template <int CAP, int KPL, int NT, int NC>
__global__ __launch_bounds__(NT) void block_select_kernel(SelectArgs a) {
  __shared__ unsigned long long keys[CAP];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  constexpr int nw = NT / kWave, STEPS = 4 * NC;  // of 8 channels
  // the tiles of one (b, kv head) on one XCD: its L2 holds their key means
  const unsigned chunk = (a.work + 7) / 8;
  const unsigned chunk_end = min(a.work, (blockIdx.x % 8 + 1) * chunk);
  for (unsigned work = blockIdx.x % 8 * chunk + blockIdx.x / 8; work < chunk_end; work += gridDim.x / 8) {
    const unsigned pr = work / (unsigned)a.tiles;  // (b, kv head)
    const int64_t pair = pr;
    const int b = (int)(pr / (unsigned)a.heads_kv), run0 = (int)(work - pr * a.tiles) * a.rows;
    const int q_len = a.q_len ? min(max(a.q_len[b], 0), a.Nq) : a.Nq, k_len = a.k_len ? min(max(a.k_len[b], 0), a.Nk) : a.Nk;
    const int nblk = (k_len + a.k_block - 1) / a.k_block;  // blocks with a key

    // ---- scores: 16 blocks (rows) x 16 runs (columns) per step; lane (m, g) supplies row / column m's channels 8 s + 2 g + {0, 1}
    {
      const int m = lane % 16, g = lane / 16;
      const int qrow = min(run0 + min(m, a.rows - 1), a.runs - 1);
      const double* qp = a.qm + (pair * a.runs + qrow) * a.d + 2 * g;
      // channels past the head: any of the head's, made zero on both sides
      auto means = [&](const double* p, f64x2_t (&v)[STEPS]) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) v[s] = *reinterpret_cast<const f64x2_t*>(p + min(8 * s, a.d - 8));
#pragma unroll
        for (int s = 4 * NC - 4; s < STEPS; ++s)
          if (8 * s >= a.d) v[s] = f64x2_t{0.0, 0.0};
      };
      f64x2_t qv[STEPS], kv[STEPS];
      if (wave * 16 < nblk) means(qp, qv);
      for (int j0 = wave * 16; j0 < nblk; j0 += nw * 16) {
        means(a.km + (pair * a.blocks + min(j0 + m, a.blocks - 1)) * a.d + 2 * g, kv);
        f64x4_t acc{0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          acc = __builtin_amdgcn_mfma_f64_16x16x4f64(kv[s][0], qv[s][0], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f64_16x16x4f64(kv[s][1], qv[s][1], acc, 0, 0, 0);
        }
        if (m < a.rows) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // result register i: row 4 i + g
            const int j = j0 + 4 * i + g;
            if (j < a.pitch) keys[m * a.pitch + j] = j < nblk ? order_key(acc[i]) : 0ull;
          }
        }
      }
    }
    __syncthreads();

    // ---- the `keep` largest of each run
    for (int row = wave; row < a.rows; row += nw) {
      const int run = run0 + row;
      if (run >= a.runs) break;
      unsigned* out = a.out + (pair * a.runs + run) * a.words;
      unsigned long long* key = keys + row * a.pitch;
      const bool none = (int64_t)run * a.q_block >= q_len;
      if (none || nblk <= a.keep) {  // nothing, or all
        for (int w = lane; w < a.words; w += kWave) {
          const int n = none ? 0 : nblk - 32 * w;
          out[w] = n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u;
        }
        continue;
      }
      unsigned long long held[KPL ? KPL : 1];
      if constexpr (KPL > 0) {
#pragma unroll
        for (int i = 0; i < KPL; ++i) held[i] = i * kWave + lane < nblk ? key[i * kWave + lane] : 0ull;  // 0: below every score
      }
      auto tally = [&](auto pred) {
        int n = 0;
        if constexpr (KPL > 0 && KPL <= 4) {
#pragma unroll
          for (int i = 0; i < KPL; ++i) n += __popcll(__builtin_amdgcn_ballot_w64(pred(held[i])));
          return n;
        } else if constexpr (KPL > 0) {
#pragma unroll
          for (int i = 0; i < KPL; ++i) n += pred(held[i]) ? 1 : 0;
        } else {
          for (int j = lane; j < nblk; j += kWave) n += pred(key[j]) ? 1 : 0;
        }
        return (int)lanes_join((unsigned)n, [](unsigned x, unsigned y) { return x + y; });
      };
      // The upper words first.  (From zero on, by the bits of a threshold, all candidates counted to the end: 144 us a call against
      // 134 for 450 runs x 900 blocks x 20 heads.)
      unsigned top = 0;
      if constexpr (KPL > 0) {
#pragma unroll
        for (int i = 0; i < KPL; ++i) top = max(top, (unsigned)(held[i] >> 32));
      } else {
        for (int j = lane; j < nblk; j += kWave) top = max(top, (unsigned)(key[j] >> 32));
      }
      top = lanes_join(top, [](unsigned x, unsigned y) { return max(x, y); });
      constexpr int WAYS = KPL > 0 && KPL <= 4 ? 4 : 2;
      UpperBounds bounds = upper_bounds<WAYS>(top, nblk, a.keep, KPL > 1 ? kWave : 0,
                                              [&](unsigned c) { return tally([&](unsigned long long k) { return (unsigned)(k >> 32) >= c; }); });
      int &n_lo = bounds.n_lo, &n_hi = bounds.n_hi;
      unsigned long long least = (unsigned long long)bounds.lo << 32;  // everything >= least is kept, except some of the equal ones
      bool exact = n_lo == a.keep;
      int need_equal = 0;  // of the values == least, when not exact
      if (!exact) {
        unsigned long long end = (unsigned long long)bounds.hi << 32;
        if (KPL > 0 && n_lo - n_hi <= kWave) {  // one candidate per lane: a count is a ballot
          unsigned long long mine = 0;
          if constexpr (KPL == 1) {
            mine = is_candidate(held[0], least, end) ? held[0] : 0ull;
          } else if constexpr (KPL > 0) {
            int at = 0;
#pragma unroll
            for (int i = 0; i < KPL; ++i) {  // the run's scores in LDS are in registers: their place is free, and holds more than the
                                             // kWave candidates at most (KPL > 1: more than kWave blocks)
              const bool in = is_candidate(held[i], least, end);
              const unsigned long long ins = __builtin_amdgcn_ballot_w64(in);
              if (in) key[at + __popcll(ins & ((1ull << lane) - 1ull))] = held[i];
              at += __popcll(ins);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (lane < at) mine = key[lane];
          }
          const int above = n_hi;
          narrow<4>(least, end, n_lo, n_hi, a.keep, 0, [&](unsigned long long c) { return above + __popcll(__builtin_amdgcn_ballot_w64(mine >= c)); });
        } else {  // many of one upper word
          narrow<WAYS>(least, end, n_lo, n_hi, a.keep, 0, [&](unsigned long long c) { return tally([&](unsigned long long k) { return k >= c; }); });
        }
        exact = n_lo == a.keep;
        need_equal = a.keep - n_hi;
      }
      int equal = 0;
      auto taken = [&](unsigned long long k) {
        bool take = exact ? k >= least : k > least;
        if (!exact) {
          const unsigned long long eqs = __builtin_amdgcn_ballot_w64(k == least);
          const int rank = equal + __popcll(eqs & ((1ull << lane) - 1ull));
          take = take || (k == least && rank < need_equal);
          equal += __popcll(eqs);
        }
        return __builtin_amdgcn_ballot_w64(take);
      };
      if constexpr (KPL > 0) {  // lane w collects word w
        unsigned word = 0;
#pragma unroll
        for (int i = 0; i < KPL; ++i) {
          const unsigned long long bits = taken(held[i]);
          if (lane / 2 == i) word = (unsigned)(lane % 2 ? bits >> 32 : bits);
        }
        if (lane < a.words) out[lane] = word;
      } else {
        for (int j0 = 0; j0 < 32 * a.words; j0 += kWave) {
          const unsigned long long bits = taken(j0 + lane < nblk ? key[j0 + lane] : 0ull);
          if (lane < 2 && j0 / 32 + lane < a.words) out[j0 / 32 + lane] = (unsigned)(bits >> (32 * lane));
        }
      }
    }
    __syncthreads();
  }
}

}  // namespace si

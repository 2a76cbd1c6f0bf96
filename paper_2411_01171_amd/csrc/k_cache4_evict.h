// Eviction from a cache in 4 bits: which slots stay, by the weight they received, and their move to another cache.
//
// Weights are ordered as unsigned integers.  The least weight that stays is found digit by digit from the top, by counting in
// LDS; then how many slots of every 1024 are above it and how many equal it.  From these counts the last kernel's workgroups, one
// for every 1024 slots, know where what they keep begins.  All counts are whole numbers: no order changes them.
#pragma once
#include <type_traits>

#include "k_cache4.h"

namespace si {

struct EvictArgs {
  Cache4View from, to;
  const float* weight;
  float* weight_out;
  int *kept, *out_len;
  const int* k_len;  // or NULL
  int keep, first, last;
  unsigned lists;    // B * heads
  unsigned chunks;   // of 1024 slots of a list
  unsigned work;     // lists * chunks
  int2* counts;      // [lists][chunks]: slots that stay without question, slots that equal the threshold
  uint2* least;      // [lists]: the threshold, and how many of those that equal it stay
  unsigned parts;    // workgroups of a list of more than 32768 slots
  int64_t part_slots;
  int* hist[2];      // [lists][parts][2048], of one step and the next
  struct EvictSearch* search;  // [2][lists]
};

// Order of a weight as an unsigned integer: NaN as -infinity, -0 as +0.  At least 0x007fffff, at most 0xff800000.
__device__ __forceinline__ unsigned weight_key(float x) {
  if (!(x == x)) x = -INFINITY;
  const unsigned b = __float_as_uint(x + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}

constexpr int kEvictThreads = 1024;
constexpr int kEvictPer = 16, kEvictPerMost = 32;            // weights of a thread at a time; of the lists with a workgroup each at most
constexpr int kEvictPart = kEvictThreads * kEvictPer;
constexpr int kEvictWhole = kEvictThreads * kEvictPerMost;   // longer lists are searched by several workgroups
constexpr unsigned kEvictParts = 16;                         // so many at most
constexpr int kEvictChunk = kEvictThreads;                   // slots that are counted together; the second kernel's piece
constexpr int kEvictBins = 2048;                             // digits of 11, 11 and 10 bits

// Whether the weight of a slot of a list of n > keep counts; of those whose weight does not, all stay.
__device__ __forceinline__ bool evict_open(const EvictArgs& a, int n, int64_t i) { return i >= a.first && i < n - a.last; }

__host__ __device__ constexpr int evict_shift(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }

// The threshold as far as it is known: its upper digits, and how many weights of those that share them stay.
struct EvictSearch {
  unsigned least;
  int left;
};

// What a workgroup of kEvictThreads shares.
struct EvictShared {
  int hist[kEvictBins];
  int wave_total[kEvictThreads / kWave];
  int count[kEvictPerMost][2];
  EvictSearch found;
};

// Inclusive sums over the lanes of a wavefront.
__device__ __forceinline__ int wave_upto(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);  // row_shr 1, 2, 4, 8: within 16 lanes
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast 15: lane 15 to row 1, 47 to row 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast 31: to rows 2 and 3
  return v;
}

// The next digit, from the thread's two counts: those of digits 2047 - 2 t and 2046 - 2 t.  It is the one with which the count from the top
// reaches what is left.
__device__ __forceinline__ EvictSearch evict_digit(EvictShared& sh, EvictSearch at, int digit, int h0, int h1) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  int upto = wave_upto(h0 + h1);
  if (lane == kWave - 1) sh.wave_total[wave] = upto;
  __syncthreads();
  // the wavefronts before this one, a lane each
  upto += __builtin_amdgcn_readlane(wave_upto(lane < wave ? sh.wave_total[lane & 15] : 0), 15);
  const int before = upto - h0 - h1;
  if (before < at.left && at.left <= upto) {  // one thread's
    const bool second = before + h0 < at.left;
    sh.found.least = at.least | (unsigned)(second ? 2046 - 2 * tid : 2047 - 2 * tid) << evict_shift(digit);
    sh.found.left = at.left - before - (second ? h0 : 0);
  }
  __syncthreads();
  return sh.found;
}

// A batch of up to 32768 slots, base + 1024 j + t: which of them there are and which weights count, from its first slot on.
struct EvictBatch {
  int there, lo, hi;
  __device__ __forceinline__ EvictBatch(const EvictArgs& a, int n, int64_t base, int64_t end) {
    auto from_base = [&](int64_t i) { return (int)min(max(i - base, (int64_t)0), (int64_t)kEvictWhole); };
    there = from_base(end);
    lo = min(from_base(a.first), there);
    hi = max(lo, min(from_base((int64_t)n - a.last), there));
  }
  __device__ __forceinline__ bool any(int j) const { return j * kEvictThreads < there; }  // of a thread's slot j, over the workgroup
  __device__ __forceinline__ bool open(int i) const { return i >= lo && i < hi; }
};

// The weights in their order; 0: no weight that counts.
template <int PER>
__device__ __forceinline__ void evict_load(const EvictArgs& a, const float* w, const EvictBatch& of, int64_t base, unsigned (&key)[PER]) {
  float x[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = j * kEvictThreads + (int)threadIdx.x;
    x[j] = 0.f;
    if (of.any(j) && i < of.there) x[j] = w[base + i];
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) key[j] = of.any(j) && of.open(j * kEvictThreads + (int)threadIdx.x) ? weight_key(x[j]) : 0u;
}

// Adds the weights that share the digits found so far to sh.hist, which is zero.
template <int PER>
__device__ __forceinline__ void evict_count(EvictShared& sh, const unsigned (&key)[PER], const EvictBatch& of, EvictSearch at, int digit) {
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (!of.any(j)) continue;
    const bool counts = key[j] != 0u && (digit == 0 || (key[j] ^ at.least) >> evict_shift(digit - 1) == 0u);
    if (counts) atomicAdd(&sh.hist[(key[j] >> evict_shift(digit)) & (digit == 2 ? 1023u : 2047u)], 1);
  }
}

// For every 1024 slots from `base` on, those that stay without question and those that equal the threshold.
template <int PER>
__device__ __forceinline__ void evict_counts(const EvictArgs& a, EvictShared& sh, const unsigned (&key)[PER], const EvictBatch& of, unsigned least, unsigned list,
                                             int64_t base) {
  const int tid = threadIdx.x;
  if (tid < 2 * PER) sh.count[tid / 2][tid % 2] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (!of.any(j)) continue;
    const int i = j * kEvictThreads + tid;
    const int above = (int)__popcll(__builtin_amdgcn_ballot_w64(of.open(i) ? key[j] > least : i < of.there));  // of slots that are not open all stay
    const int equal = (int)__popcll(__builtin_amdgcn_ballot_w64(key[j] == least && key[j] != 0u));
    if (tid % kWave == 0) {
      if (above) atomicAdd(&sh.count[j][0], above);
      if (equal) atomicAdd(&sh.count[j][1], equal);
    }
  }
  __syncthreads();
  if (tid < PER && of.any(tid)) a.counts[(int64_t)list * a.chunks + (unsigned)(base / kEvictChunk) + tid] = make_int2(sh.count[tid][0], sh.count[tid][1]);
  __syncthreads();
}

__device__ __forceinline__ int evict_length(const EvictArgs& a, unsigned list) {
  const int b = (int)(list / (unsigned)a.from.heads);
  return a.k_len ? min(max(a.k_len[b], 0), a.from.cap) : a.from.cap;
}
__device__ __forceinline__ void evict_put_length(const EvictArgs& a, unsigned list, int n) {
  if (threadIdx.x == 0 && list % (unsigned)a.from.heads == 0) a.out_len[list / (unsigned)a.from.heads] = min(n, a.keep);
}
// Where a search begins.  Nothing that counts stays: no weight is above the highest number.
__device__ __forceinline__ EvictSearch evict_begin(const EvictArgs& a) {
  const int left = a.keep - a.first - a.last;
  return EvictSearch{left > 0 ? 0u : ~0u, left};
}

// Lists of up to 1024 PER slots, one workgroup each; the weights stay in registers.  A chain of latencies, that of fetching the code among
// them: the digits are a loop, and short lists have a form of their own (4096 slots 7 us; with digits unrolled and 16 weights of a thread 12).
// With 32 weights of a thread 24000 and 32768 slots of 8 lists take 28 and 32 us with their move, in two pieces 36 and 37, with 64 of a
// thread 38 and 43; 60000 slots take 57 with 64, and 38 in pieces.
template <int PER>
__global__ __launch_bounds__(kEvictThreads) void cache4_pick_kernel(EvictArgs a) {
  __shared__ EvictShared sh;
  const int tid = threadIdx.x;
  for (unsigned list = blockIdx.x; list < a.lists; list += gridDim.x) {
    const int n = evict_length(a, list);
    evict_put_length(a, list, n);
    if (n <= a.keep) {  // all: above a threshold of zero
      if (tid == 0) a.least[list] = make_uint2(0u, 0u);
      continue;
    }
    unsigned key[PER];
    const EvictBatch of(a, n, 0, n);
    evict_load(a, a.weight + (int64_t)list * a.from.cap, of, 0, key);
    sh.hist[tid] = 0;
    sh.hist[tid + kEvictThreads] = 0;
    EvictSearch at = evict_begin(a);
    if (at.left > 0)
#pragma unroll 1
      for (int digit = 0; digit < 3; ++digit) {
        __syncthreads();
        evict_count(sh, key, of, at, digit);
        __syncthreads();
        const int h0 = sh.hist[2047 - 2 * tid], h1 = sh.hist[2046 - 2 * tid];
        sh.hist[2047 - 2 * tid] = sh.hist[2046 - 2 * tid] = 0;
        at = evict_digit(sh, at, digit, h0, h1);
      }
    if (tid == 0) a.least[list] = make_uint2(at.least, (unsigned)at.left);
    evict_counts(a, sh, key, of, at.least, list, 0);
  }
}

// Longer lists, a workgroup for each of a.parts pieces of one.  STEP 0, 1, 2: the counts of that digit of a piece's weights; 1, 2, 3: before
// that, the digit before it from all pieces' counts; 3: the counts of every 1024 slots.  A launch per step, 9 to 11 us each for 32 lists
// of 115200 slots: latencies of memory, and of fetching the code (pieces of 4096 and 8192 slots are slower; a workgroup per list took 98 us).
template <int STEP>
__global__ __launch_bounds__(kEvictThreads) void cache4_search_kernel(EvictArgs a) {
  __shared__ EvictShared sh;
  const int tid = threadIdx.x;
  for (unsigned work = blockIdx.x; work < a.lists * a.parts; work += gridDim.x) {
    const unsigned list = work / a.parts, part = work % a.parts;
    const int n = evict_length(a, list);
    if (STEP == 0 && part == 0) evict_put_length(a, list, n);
    if (n <= a.keep) {
      if (STEP == 3 && part == 0 && tid == 0) a.least[list] = make_uint2(0u, 0u);
      continue;
    }
    const int64_t begin = (int64_t)part * a.part_slots, end = min((int64_t)n, begin + a.part_slots);
    unsigned key[kEvictPer];
    const float* w = a.weight + (int64_t)list * a.from.cap;
    EvictBatch of(a, n, begin, end);
    evict_load(a, w, of, begin, key);      // on its way while the digit is found
    __syncthreads();                       // the piece before has been counted
    if (STEP < 3) {
      sh.hist[tid] = 0;
      sh.hist[tid + kEvictThreads] = 0;
    }
    EvictSearch at = evict_begin(a);
    if (STEP > 0 && at.left > 0) {
      if (STEP > 1) at = a.search[(STEP % 2) * a.lists + list];
      const int2* counts = reinterpret_cast<const int2*>(a.hist[(STEP + 1) % 2] + (int64_t)list * a.parts * kEvictBins) + (kEvictThreads - 1 - tid);
      int h0 = 0, h1 = 0;
#pragma unroll 1
      for (unsigned p0 = 0; p0 < a.parts; p0 += 8) {
        int2 v[8];
#pragma unroll
        for (unsigned p = 0; p < 8; ++p)
          if (p0 + p < a.parts) v[p] = counts[(p0 + p) * (kEvictBins / 2)];
#pragma unroll
        for (unsigned p = 0; p < 8; ++p)
          if (p0 + p < a.parts) {
            h1 += v[p].x;
            h0 += v[p].y;
          }
      }
      at = evict_digit(sh, at, STEP - 1, h0, h1);
      if (part == 0 && tid == 0) a.search[((STEP + 1) % 2) * a.lists + list] = at;
    }
    if (STEP == 3 && part == 0 && tid == 0) a.least[list] = make_uint2(at.least, (unsigned)at.left);
    __syncthreads();
#pragma unroll 1
    for (int64_t base = begin; base < end; base += kEvictPart) {
      if (base != begin) {
        of = EvictBatch(a, n, base, end);
        evict_load(a, w, of, base, key);
      }
      if constexpr (STEP < 3) {
        if (at.left > 0) evict_count(sh, key, of, at, STEP);
      } else {
        evict_counts(a, sh, key, of, at.least, list, base);
      }
    }
    if constexpr (STEP < 3) {
      __syncthreads();
      int2* out = reinterpret_cast<int2*>(a.hist[STEP % 2] + ((int64_t)list * a.parts + part) * kEvictBins);
      out[tid] = make_int2(sh.hist[2 * tid], sh.hist[2 * tid + 1]);
    }
  }
}

constexpr int kMoveThreads = 256;

// The slots of a chunk that stay: listed in LDS in their order, then moved, 16 bytes of codes to a thread.  Bound by HBM: a quarter of 115200 slots and fewer
// of 32 heads of 128 in 78 us, 233 MB read (rows of 64 bytes in lines of 128) and 134 written, 4.7 TB/s.
template <int G>
__global__ __launch_bounds__(kMoveThreads) void cache4_move_kernel(EvictArgs a) {
  constexpr int WAVES = kMoveThreads / kWave, PER = kEvictChunk / kMoveThreads, S = cache4_scale_bytes(G);
  __shared__ int stays[kEvictChunk];
  __shared__ int sums[3][WAVES];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const unsigned long long below = lane ? ~0ull >> (64 - lane) : 0ull;
  for (unsigned work = blockIdx.x; work < a.work; work += gridDim.x) {
    const unsigned list = work / a.chunks, chunk = work % a.chunks;
    const int n = evict_length(a, list);
    const int64_t slot0 = (int64_t)chunk * kEvictChunk;
    if (slot0 >= n) continue;
    const float* w = a.weight + (int64_t)list * a.from.cap;
    const uint2 least = a.least[list];
    float x[PER];
    unsigned long long sure[PER], tie[PER];
    int my_ties = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int64_t i = slot0 + (wave * PER + j) * kWave + lane;
      x[j] = i < n ? w[i] : 0.f;
    }
    int above = 0, equal = 0;  // of the chunks before
    if (n > a.keep)
      for (unsigned c = tid; c < chunk; c += kMoveThreads) {
        const int2 v = a.counts[(int64_t)list * a.chunks + c];
        above += v.x;
        equal += v.y;
      }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int64_t i = slot0 + (wave * PER + j) * kWave + lane;
      const unsigned key = weight_key(x[j]);
      const bool open = n > a.keep && evict_open(a, n, i);
      sure[j] = __builtin_amdgcn_ballot_w64(open ? key > least.x : i < n);  // of slots that are not open all stay
      tie[j] = __builtin_amdgcn_ballot_w64(open && key == least.x);
      my_ties += __popcll(tie[j]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      above += __shfl_xor(above, o, kWave);
      equal += __shfl_xor(equal, o, kWave);
    }
    __syncthreads();  // the piece before has been moved
    if (lane == 0) {
      sums[0][wave] = above;
      sums[1][wave] = equal;
      sums[2][wave] = my_ties;
    }
    __syncthreads();
    int base = 0, ties = 0, left;  // slots that stayed and ties before this chunk
#pragma unroll
    for (int v = 0; v < WAVES; ++v) {
      base += sums[0][v];
      ties += sums[1][v];
    }
    left = (int)least.y - ties;  // ties of this chunk and later ones that stay; below zero where they ended before
    base = n > a.keep ? base + min(ties, (int)least.y) : (int)slot0;
    int ties_before = 0, at = 0, in_chunk = 0;
    for (int v = 0; v < wave; ++v) ties_before += sums[2][v];
    unsigned long long stay[PER];
    int mine = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const bool in = (tie[j] >> lane & 1ull) && ties_before + (int)__popcll(tie[j] & below) < left;
      stay[j] = sure[j] | __builtin_amdgcn_ballot_w64(in);
      ties_before += __popcll(tie[j]);
      mine += __popcll(stay[j]);
    }
    __syncthreads();
    if (lane == 0) sums[0][wave] = mine;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < WAVES; ++v) {
      if (v < wave) at += sums[0][v];
      in_chunk += sums[0][v];
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (stay[j] >> lane & 1ull) {
        const int k = at + (int)__popcll(stay[j] & below), i = (int)(slot0 + (wave * PER + j) * kWave + lane);
        stays[k] = i;
        a.kept[(int64_t)list * a.keep + base + k] = i;
        a.weight_out[(int64_t)list * a.to.cap + base + k] = x[j];
      }
      at += __popcll(stay[j]);
    }
    __syncthreads();
    const int64_t src0 = (int64_t)list * a.from.cap, dst0 = (int64_t)list * a.to.cap + base;
    const int pieces = in_chunk * G;
    for (int u0 = 0; u0 < pieces; u0 += 2 * kMoveThreads) {
      u32x4_t kv[2][2];
      int64_t to[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int u = u0 + i * kMoveThreads + tid, t = u / G;
        to[i] = -1;
        if (u >= pieces) continue;
        const int64_t src = (src0 + stays[t]) * (16 * G) + (u % G) * 16;
        to[i] = (dst0 + t) * (16 * G) + (u % G) * 16;
        kv[i][0] = *reinterpret_cast<const u32x4_t*>(a.from.kc + src);
        kv[i][1] = *reinterpret_cast<const u32x4_t*>(a.from.vc + src);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (to[i] >= 0) {
          *reinterpret_cast<u32x4_t*>(a.to.kc + to[i]) = kv[i][0];
          *reinterpret_cast<u32x4_t*>(a.to.vc + to[i]) = kv[i][1];
        }
    }
    using Word = std::conditional_t<S == 4, unsigned, std::conditional_t<S == 2, unsigned short, uint8_t>>;
    for (int t = tid; t < in_chunk; t += kMoveThreads) {
      const int64_t src = (src0 + stays[t]) * S, dst = (dst0 + t) * S;
      const Word k = *reinterpret_cast<const Word*>(a.from.ks + src), v = *reinterpret_cast<const Word*>(a.from.vs + src);
      *reinterpret_cast<Word*>(a.to.ks + dst) = k;
      *reinterpret_cast<Word*>(a.to.vs + dst) = v;
    }
  }
}

}  // namespace si

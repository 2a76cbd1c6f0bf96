// Eviction from a cache in 4 bits: which tokens stay, by the weight they received, and their move to another cache.
#pragma once
#include "k_cache4.h"

namespace si {

struct EvictArgs {
  Cache4View from, to;
  const float* weight;
  float* weight_out;
  int *kept, *out_len;
  const int* k_len;  // or NULL
  int keep, first, last, code_bytes, scale_bytes;
  unsigned lists;    // B * heads
  unsigned chunks, work;  // of the move
};

// Order of a weight as an unsigned integer: NaN as -infinity, -0 as +0.  At least 0x007fffff.
__device__ __forceinline__ unsigned weight_key(float x) {
  if (!(x == x)) x = -INFINITY;
  const unsigned b = __float_as_uint(x + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}

constexpr int kEvictThreads = 1024;

// One workgroup per list: the threshold's 32 bits, eight at a time by counting, then the tokens that stay in their order.
__global__ __launch_bounds__(kEvictThreads) void cache4_pick_kernel(EvictArgs a) {
  __shared__ int hist[256], above[kEvictThreads / kWave], equal[kEvictThreads / kWave];
  __shared__ unsigned found_digit;
  __shared__ int found_left;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  for (unsigned list = blockIdx.x; list < a.lists; list += gridDim.x) {
    const int b = (int)(list / (unsigned)a.from.heads);
    const int n = a.k_len ? min(max(a.k_len[b], 0), a.from.cap) : a.from.cap;
    const float* w = a.weight + (int64_t)list * a.from.cap;
    int* kept = a.kept + (int64_t)list * a.keep;
    float* wo = a.weight_out + (int64_t)list * a.to.cap;
    if (tid == 0 && list % (unsigned)a.from.heads == 0) a.out_len[b] = min(n, a.keep);
    if (n <= a.keep) {
      for (int i = tid; i < n; i += kEvictThreads) {
        kept[i] = i;
        wo[i] = w[i];
      }
      continue;
    }
    const int lo = a.first, hi = n - a.last;  // candidates
    int left = a.keep - a.first - a.last;     // of them that stay
    unsigned prefix = 0u;
    for (int shift = 24; shift >= 0 && left > 0; shift -= 8) {
      for (int i = tid; i < 256; i += kEvictThreads) hist[i] = 0;
      __syncthreads();
      for (int64_t i = (int64_t)lo + tid; i < hi; i += kEvictThreads) {
        const unsigned key = weight_key(w[i]);
        if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[(key >> shift) & 255u], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int d = 255, more = left;
        for (; d > 0 && hist[d] < more; --d) more -= hist[d];
        found_digit = (unsigned)d;
        found_left = more;
      }
      __syncthreads();
      prefix |= found_digit << shift;
      left = found_left;
    }
    // what is above `prefix` stays, and the first `left` that equal it; none at all if nothing was to be found
    const bool none = a.keep - a.first - a.last == 0;
    int done = 0, eq = 0;
    for (int64_t i0 = 0; i0 < n; i0 += kEvictThreads) {
      const int64_t i = i0 + tid;
      const float x = i < n ? w[i] : 0.f;
      const unsigned key = weight_key(x);
      const bool open = i >= lo && i < hi && !none;
      const bool sure = i < n && (i < lo || i >= hi || (open && key > prefix)), tie = open && key == prefix;
      const unsigned long long ties = __builtin_amdgcn_ballot_w64(tie), below = lane ? ~0ull >> (64 - lane) : 0ull;
      if (lane == 0) equal[wave] = __popcll(ties);
      __syncthreads();
      int ties_before = eq + __popcll(ties & below);
      for (int v = 0; v < kEvictThreads / kWave; ++v) {
        if (v < wave) ties_before += equal[v];
        eq += equal[v];
      }
      const bool stay = sure || (tie && ties_before < left);
      const unsigned long long stays = __builtin_amdgcn_ballot_w64(stay);
      if (lane == 0) above[wave] = __popcll(stays);
      __syncthreads();
      int at = done + __popcll(stays & below);
      for (int v = 0; v < kEvictThreads / kWave; ++v) {
        if (v < wave) at += above[v];
        done += above[v];
      }
      if (stay) {
        kept[at] = (int)i;
        wo[at] = x;
      }
    }
    __syncthreads();
  }
}

// The tokens that stay, 16 bytes of codes to a thread.
__global__ __launch_bounds__(256) void cache4_move_kernel(EvictArgs a) {
  const int pieces = a.code_bytes / 16, tokens = 256 / (2 * pieces);
  const int t = threadIdx.x / (2 * pieces), x = threadIdx.x % (2 * pieces) / pieces, piece = threadIdx.x % pieces;
  const uint8_t *fc = x ? a.from.vc : a.from.kc, *fs = x ? a.from.vs : a.from.ks;
  uint8_t *tc = x ? a.to.vc : a.to.kc, *ts = x ? a.to.vs : a.to.ks;
  for (unsigned work = blockIdx.x; work < a.work; work += gridDim.x) {
    const unsigned list = work / a.chunks;
    const int b = (int)(list / (unsigned)a.from.heads);
    const int n = min(a.k_len ? min(max(a.k_len[b], 0), a.from.cap) : a.from.cap, a.keep);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t slot = ((int64_t)(work % a.chunks) * 4 + i) * tokens + t;
      if (t >= tokens || slot >= n) continue;
      const int64_t src = (int64_t)list * a.from.cap + a.kept[(int64_t)list * a.keep + slot], dst = (int64_t)list * a.to.cap + slot;
      *reinterpret_cast<u32x4_t*>(tc + dst * a.code_bytes + piece * 16) = *reinterpret_cast<const u32x4_t*>(fc + src * a.code_bytes + piece * 16);
      if (piece == 0) {
        if (a.scale_bytes == 4) *reinterpret_cast<unsigned*>(ts + dst * 4) = *reinterpret_cast<const unsigned*>(fs + src * 4);
        else if (a.scale_bytes == 2) *reinterpret_cast<unsigned short*>(ts + dst * 2) = *reinterpret_cast<const unsigned short*>(fs + src * 2);
        else ts[dst] = fs[src];
      }
    }
  }
}

}  // namespace si

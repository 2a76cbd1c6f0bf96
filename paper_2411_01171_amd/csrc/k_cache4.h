// A cache of keys and values in 4 bits: storing tokens and reading them back.
//
// A head's channels are held in groups of 32: e2m1 codes c (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) and one byte s, value
// c 2^(s - 127).  Both the codes' type and the power of two are what this chip's conversions take and give, so that a value comes back by
// one instruction per two of them, exactly, in bf16 as in float32.
//   s = the smallest with max |x| <= 7 * 2^(s - 127): between 6 and 7 the nearest code is 6, as the grid's next value would be 8
//   c = the nearest code to x / 2^(s - 127), ties to the even code, no further than 6
// Every step is exact or the one rounding to c, so the result is the definition's, bit for bit.
#pragma once
#include "si_common.h"

namespace si {

struct Cache4View {
  uint8_t *kc, *ks, *vc, *vs;
  int heads, cap;
};

// Bytes of a token's scales: room for whole words.
__host__ __device__ constexpr int cache4_scale_bytes(int groups) { return groups == 3 ? 4 : groups; }

struct Cache4CopyArgs {
  HeadsView x[2];  // keys, values
  Cache4View c;
  float* weight;             // [B][heads][cap] or NULL (store: zeroed where a token lands)
  const int *first, *length;  // per batch entry, or NULL: 0, N
  int N, d;
  int chunks;                // of tokens
  unsigned work;             // chunks * heads * B, the heads fastest
};

constexpr int kCache4Threads = 256;
constexpr int kCache4Deep = 4;  // tokens of a thread

template <int G> constexpr int cache4_tokens() { return kCache4Threads / (4 * G) * kCache4Deep; }  // of a workgroup

// the largest of the four lanes of a quad
__device__ __forceinline__ unsigned quad_max(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
  return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
}

// Scale byte of a group whose largest magnitude has these float32 bits: up from its own binade's where the fraction passes
// 1.75.  2 and 252 at the ends keep every value a normal, finite bf16; 255 where a NaN or an infinity is among the values.
__device__ __forceinline__ unsigned cache4_scale(unsigned bits) {
  if (bits >= 0x7F800000u) return 255u;
  const int s = (int)((bits + 0x1FFFFFu) >> 23) - 2;
  return (unsigned)min(max(s, 2), 252);
}

// Eight channels on their way: 16 bytes of bf16, 32 of float32.
template <typename T> struct Eight;
template <> struct Eight<bf16> {
  u32x4_t w;
  __device__ __forceinline__ void load(const bf16* p) { w = *reinterpret_cast<const u32x4_t*>(p); }
  __device__ __forceinline__ void clear() { w = u32x4_t{0, 0, 0, 0}; }
  __device__ __forceinline__ unsigned top() const {  // largest magnitude, as float32 bits
    typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
    u16x2_t m = __builtin_bit_cast(u16x2_t, w[0] & 0x7FFF7FFFu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, w[i] & 0x7FFF7FFFu));
    return (unsigned)max(m[0], m[1]) << 16;
  }
  __device__ __forceinline__ unsigned codes(float scale) const {
    auto pair = [&](int i) {  // by way of a plain value: the bit cast of a vector's element takes the vector's first
      const unsigned x = w[i];
      return __builtin_bit_cast(bf16x2_t, x);
    };
    unsigned r = 0u;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(0), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(1), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(2), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair(3), scale, 3);
  }
};
template <> struct Eight<float> {
  u32x4_t w[2];
  __device__ __forceinline__ void load(const float* p) {
    w[0] = *reinterpret_cast<const u32x4_t*>(p);
    w[1] = *reinterpret_cast<const u32x4_t*>(p + 4);
  }
  __device__ __forceinline__ void clear() { w[0] = w[1] = u32x4_t{0, 0, 0, 0}; }
  __device__ __forceinline__ unsigned top() const {
    unsigned m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, w[i / 4][i % 4] & 0x7FFFFFFFu);
    return m;
  }
  __device__ __forceinline__ unsigned codes(float scale) const {
    auto f = [&](int i) { return __uint_as_float(w[i / 4][i % 4]); };
    unsigned r = 0u;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f(0), f(1), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f(2), f(3), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f(4), f(5), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f(6), f(7), scale, 3);
  }
};

// Eight codes as bf16, in pairs.  A scale of byte 255 makes every one of them NaN.
__device__ __forceinline__ u32x4_t cache4_bf16x8(unsigned codes, float scale) {
  return u32x4_t{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                 __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                 __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                 __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// Where a workgroup's thread works: eight channels of kCache4Deep tokens of one head.
template <int G>
struct Cache4Place {
  int piece, at, h, b, len;
  int64_t first, row;  // first slot; rows of the arrays before this head's
  __device__ __forceinline__ Cache4Place(const Cache4CopyArgs& a, unsigned work) {
    const int t = threadIdx.x / (4 * G);
    piece = threadIdx.x % (4 * G);
    unsigned up = work / (unsigned)a.c.heads;
    h = (int)(work - up * (unsigned)a.c.heads);
    b = (int)(up / (unsigned)a.chunks);
    at = (int)(up % (unsigned)a.chunks) * cache4_tokens<G>() + t;
    len = a.length ? min(max(a.length[b], 0), a.N) : a.N;
    first = a.first ? a.first[b] : 0;
    row = ((int64_t)b * a.c.heads + h) * a.c.cap;
    if (t >= kCache4Threads / (4 * G)) len = 0;  // groups of three leave four threads over
  }
  __device__ __forceinline__ int token(int i) const { return at + i * (kCache4Threads / (4 * G)); }
  __device__ __forceinline__ bool there(const Cache4CopyArgs& a, int n) const { return n < len && first + n >= 0 && first + n < a.c.cap; }
};

// Four lanes share a group of 32 channels, and a thread takes eight channels of four tokens, whose loads are in flight together.  Workgroups go
// through the heads of some tokens before the next tokens, so that rows of one projection are read to their end.  Bound by HBM:
// 230400 tokens of 5 heads of 64, two batch entries, 172 us (756 MB, 4.4 TB/s); one token 3.6 us.
template <typename T, int G>
__global__ __launch_bounds__(kCache4Threads) void cache4_store_kernel(Cache4CopyArgs a) {
  constexpr int S = cache4_scale_bytes(G);
  for (unsigned work = blockIdx.x; work < a.work; work += gridDim.x) {
    const Cache4Place<G> p(a, work);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const T* src = static_cast<const T*>(a.x[x].p) + p.b * a.x[x].sb + p.h * a.x[x].sh + p.piece * 8;
      uint8_t *codes = x ? a.c.vc : a.c.kc, *scales = x ? a.c.vs : a.c.ks;
      Eight<T> e[kCache4Deep];
#pragma unroll
      for (int i = 0; i < kCache4Deep; ++i) {
        const int n = p.token(i);
        e[i].clear();
        if (p.there(a, n) && p.piece * 8 < a.d) e[i].load(src + (int64_t)n * a.x[x].sn);
      }
#pragma unroll
      for (int i = 0; i < kCache4Deep; ++i) {
        const int n = p.token(i);
        const unsigned s = cache4_scale(quad_max(e[i].top()));
        const unsigned c = s == 255u ? 0u : e[i].codes(__uint_as_float(s << 23));
        if (p.there(a, n)) {
          const int64_t row = p.row + p.first + n;
          *reinterpret_cast<unsigned*>(codes + row * (16 * G) + p.piece * 4) = c;
          if (p.piece % 4 == 0) scales[row * S + p.piece / 4] = (uint8_t)s;
          if (S > G && p.piece == 0) scales[row * S + G] = 0;
          if (x == 0 && a.weight && p.piece == 0) a.weight[row] = 0.f;
        }
      }
    }
  }
}

// The same way back: 129 us (747 MB, 5.8 TB/s).
template <typename T, int G>
__global__ __launch_bounds__(kCache4Threads) void cache4_load_kernel(Cache4CopyArgs a) {
  constexpr int S = cache4_scale_bytes(G);
  for (unsigned work = blockIdx.x; work < a.work; work += gridDim.x) {
    const Cache4Place<G> p(a, work);
    if (p.piece * 8 >= a.d) continue;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      T* dst = static_cast<T*>(a.x[x].p) + p.b * a.x[x].sb + p.h * a.x[x].sh + p.piece * 8;
      const uint8_t *codes = x ? a.c.vc : a.c.kc, *scales = x ? a.c.vs : a.c.ks;
      unsigned c[kCache4Deep], s[kCache4Deep];
#pragma unroll
      for (int i = 0; i < kCache4Deep; ++i) {
        const int n = p.token(i);
        c[i] = s[i] = 0u;
        if (p.there(a, n)) {
          const int64_t row = p.row + p.first + n;
          c[i] = *reinterpret_cast<const unsigned*>(codes + row * (16 * G) + p.piece * 4);
          s[i] = scales[row * S + p.piece / 4];
        }
      }
#pragma unroll
      for (int i = 0; i < kCache4Deep; ++i) {
        const int n = p.token(i);
        if (!p.there(a, n)) continue;
        const u32x4_t v = cache4_bf16x8(c[i], __uint_as_float(s[i] << 23));
        T* at = dst + (int64_t)n * a.x[x].sn;
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<u32x4_t*>(at) = v;
        } else {  // what a code stands for fits bf16
          *reinterpret_cast<u32x4_t*>(at) = u32x4_t{v[0] << 16, v[0] & 0xFFFF0000u, v[1] << 16, v[1] & 0xFFFF0000u};
          *reinterpret_cast<u32x4_t*>(at + 4) = u32x4_t{v[2] << 16, v[2] & 0xFFFF0000u, v[3] << 16, v[3] & 0xFFFF0000u};
        }
      }
    }
  }
}

}  // namespace si

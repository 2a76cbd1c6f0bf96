// Shared device helpers: storage types, conversions, wavefront reductions.
// gfx950 only: 64-wide wavefronts are assumed throughout.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace si {

constexpr int kWave = 64;

// bf16 storage: upper 16 bits of an IEEE float.
struct bf16 {
  unsigned short v;
};

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));  // 16-byte register staging (a plain vector, not a struct)

__device__ __forceinline__ float bf16_bits_to_float(unsigned short b) {
  return __uint_as_float(((unsigned)b) << 16);
}

// Round-to-nearest-even via the hardware conversion (v_cvt_pk_bf16_f32); NaN stays NaN.
__device__ __forceinline__ unsigned short float_to_bf16_bits(float f) {
  return __builtin_bit_cast(unsigned short, (__bf16)f);
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return bf16_bits_to_float(v.v); }

template <typename T> __device__ __forceinline__ T from_float(float f);
template <> __device__ __forceinline__ float from_float<float>(float f) { return f; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float f) {
  bf16 r;
  r.v = float_to_bf16_bits(f);
  return r;
}

// Optional parameter vectors: NULL gain = 1, NULL shift / bias = 0.
template <typename T> __device__ __forceinline__ float param_or(const T* p, int64_t i, float dflt) {
  return p ? to_float(p[i]) : dflt;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// Direct global->LDS loads: every lane brings 16 bytes from base + off (from an address of its own) to LDS at lds + 16 lane.
// As assembly, so that the compiler's wait-count pass does not place a full vector-memory wait in front of every later LDS
// read: whoever calls them awaits their completion.  The LDS address goes through M0, and one wait state has to lie between a
// scalar write of M0 and the load that reads it; nothing inside a string of assembly adds it, hence the s_nop.  The
// compiler reserves M0 and takes no clobber of it; nothing else in the library uses it.
__device__ __forceinline__ void load_to_lds(unsigned off, const void* base, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(lds) : "memory");
}
__device__ __forceinline__ void load_to_lds(const void* p, unsigned lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds) : "memory");
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// two floats -> packed bf16 pair, round-to-nearest-even (one v_cvt_pk_bf16_f32)
__device__ __forceinline__ unsigned pack_bf16x2(float lo, float hi) {
  const f32x2_t v = {lo, hi};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2_t));
}

// sum of a bf16 pair's values onto acc
__device__ __forceinline__ float dot2_ones(unsigned packed_bf16x2, float acc) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, packed_bf16x2), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), acc,
                                         false);
}

// Fragment order of a 16-bit activation operand of the ring kernels (k_conv.h): granule
// act_granule(t, c8) holds the 16 bytes (channels 8*c8 .. +7) of token t; a 1 KiB fragment is the
// 64 granules of (32-token block, 16-channel step), 16-channel steps fastest; the buffer starts with
// a 256-byte block of zeros.
constexpr int kActZeroBytes = 256;
__host__ __device__ __forceinline__ int64_t act_granule(int64_t t, int c8, int C) {
  return ((t >> 5) * (C / 16) + (c8 >> 1)) * 64 + (c8 & 1) * 32 + (t & 31);
}
// element offset (16-bit elements) of channel c of token t in such a buffer
__host__ __device__ __forceinline__ int64_t act_offset(int64_t t, int c, int C) {
  return kActZeroBytes / 2 + act_granule(t, c >> 3, C) * 8 + (c & 7);
}

__device__ __forceinline__ float gelu_erf(float u) {
  return 0.5f * u * (1.0f + erff(u * 0.70710678118654752440f));
}

// Coefficients of Phi(x) - 0.5 = xc * R(xc^2), xc = clamp(x, -4.2, 4.2), R of degree 8 (minimax fit of
// erf(x / sqrt 2) / x on [0, 4.2], |erf error| <= 2.2e-5 everywhere, coefficients pre-halved).
constexpr float kGeluClamp = 4.2f;
constexpr int kGeluDeg = 8;
__device__ constexpr float kGeluC[kGeluDeg + 1] = {
    0.5f * 0.7978148460388184f,     0.5f * -0.1327207386493683f,    0.5f * 0.019660256803035736f,
    0.5f * -0.0022282942663878202f, 0.5f * 0.00018914842803496867f, 0.5f * -1.1521495252964087e-05f,
    0.5f * 4.6873191195118125e-07f, 0.5f * -1.1266531707576632e-08f, 0.5f * 1.199598614887165e-10f};
// GELU(x) = x * Phi(x) from that polynomial: 13 full-rate instructions, no transcendental ones
__device__ __forceinline__ float gelu_poly(float x) {
  const float xc = __builtin_amdgcn_fmed3f(x, -kGeluClamp, kGeluClamp), t = xc * xc;
  float p = fmaf(kGeluC[kGeluDeg], t, kGeluC[kGeluDeg - 1]);
#pragma unroll
  for (int k = kGeluDeg - 2; k >= 0; --k) p = fmaf(p, t, kGeluC[k]);
  return x * fmaf(p, xc, 0.5f);
}

}  // namespace si

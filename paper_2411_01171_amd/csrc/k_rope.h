// Rotary positions on three axes (frame, row, column) for heads of video tokens, with the heads' root-mean-square norm in
// the same pass.
//
// Token n lies at coordinates (f, y, x) of an F x H x W grid, raster order.  Pair i of an axis turns by
//   angle = (origin + step * coordinate) * theta^(-i / pairs of that axis),
// (x1, x2) -> (x1 cos - x2 sin, x1 sin + x2 cos).  The angle is formed in float64 and in revolutions (the host divides the
// frequencies by 2 pi), so that its whole part drops out exactly before the sine and cosine are taken in float32: positions
// of 10^6 lose nothing, and the digits that the rest loses in float32 come back to first order.  Everything else is float32
// with one rounding at the store.
//
// Bound by HBM: every head is read and written once.  A thread owns eight channels (four pairs) of one token and walks the
// heads of q and k: the sines of a token are computed once for all of them, and the loads of kRopeHeads heads are in
// flight together.  25 frames of 72x128, two batch entries, 5 heads of 64 (1180 MB in and out): 219 us (5.4 TB/s; a copy of
// 2 GiB reaches 4.9), channel halves 238, with the norm 216 and 237; float32, 14 frames of 45x50, 8 heads of 80 (323 MB) 72 us.
// The norm's sums over a head's threads go by lane primitives where those are 1, 2, 4, 8 or 16 lanes of a row, else by LDS;
// 1 / sqrt is the hardware's (one step of float32), and the gains stay as they lie in memory: both took the vector ALUs from
// 79 % of the cycles (halves: 267 us).  One 16x16 frame takes the kernel 4.4 us and its call 9, on the host.
#pragma once
#include "si_common.h"

namespace si {

constexpr int kRopeThreads = 256, kRopeHeads = 4, kRopeMaxPairs = 64;

struct HeadsView {  // element (b, n, h, c) at p + b*sb + n*sn + h*sh + c
  void* p;
  int64_t sb, sn, sh;
};

struct RopeArgs {
  HeadsView q, k, qo, ko;
  const void *q_gain, *k_gain;
  int64_t tokens;            // B * N
  int N, H, W, first;        // token n of a batch entry is grid point first + n
  int heads_q, heads, d;     // heads of q; of q and k
  int heads_per_wg;          // a workgroup's share of the heads (blockIdx.y)
  int pairs, end_f, end_y;   // all pairs; pairs [0, end_f) turn with the frame, [end_f, end_y) with the row
  int tokens_per_wg;         // kRopeThreads / (d / 8)
  float eps, inv_d;          // inv_d: 1 / d
  double origin[3], step[3];
  double freq[kRopeMaxPairs];  // revolutions per position
};

template <typename T> struct Raw8;  // eight channels as they lie in memory
template <> struct Raw8<bf16> { u32x4_t v; };
template <> struct Raw8<float> { f32x4_t v[2]; };

// channels [c0, c0 + 4) and [c1, c1 + 4) of a head; ONE: c1 == c0 + 4
template <bool ONE> __device__ __forceinline__ void load8(const bf16* p, int c0, int c1, Raw8<bf16>& r) {
  if constexpr (ONE) r.v = *reinterpret_cast<const u32x4_t*>(p + c0);
  else {
    const uint2 a = *reinterpret_cast<const uint2*>(p + c0), b = *reinterpret_cast<const uint2*>(p + c1);
    r.v = u32x4_t{a.x, a.y, b.x, b.y};
  }
}
template <bool ONE> __device__ __forceinline__ void load8(const float* p, int c0, int c1, Raw8<float>& r) {
  r.v[0] = *reinterpret_cast<const f32x4_t*>(p + c0);
  r.v[1] = *reinterpret_cast<const f32x4_t*>(p + c1);
}
__device__ __forceinline__ void unpack8(const Raw8<bf16>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(r.v[i] << 16);
    x[2 * i + 1] = __uint_as_float(r.v[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = r.v[i / 4][i % 4];
}
__device__ __forceinline__ void ones8(Raw8<bf16>& r) { r.v = u32x4_t{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}; }
__device__ __forceinline__ void ones8(Raw8<float>& r) { r.v[0] = r.v[1] = f32x4_t{1.f, 1.f, 1.f, 1.f}; }
template <bool ONE> __device__ __forceinline__ void store8(bf16* p, int c0, int c1, const float (&y)[8]) {
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (unsigned)float_to_bf16_bits(y[2 * i]) | ((unsigned)float_to_bf16_bits(y[2 * i + 1]) << 16);
  if constexpr (ONE) *reinterpret_cast<u32x4_t*>(p + c0) = u32x4_t{w[0], w[1], w[2], w[3]};
  else {
    *reinterpret_cast<uint2*>(p + c0) = make_uint2(w[0], w[1]);
    *reinterpret_cast<uint2*>(p + c1) = make_uint2(w[2], w[3]);
  }
}
template <bool ONE> __device__ __forceinline__ void store8(float* p, int c0, int c1, const float (&y)[8]) {
  *reinterpret_cast<f32x4_t*>(p + c0) = f32x4_t{y[0], y[1], y[2], y[3]};
  *reinterpret_cast<f32x4_t*>(p + c1) = f32x4_t{y[4], y[5], y[6], y[7]};
}

// v of the lane that a data-parallel primitive names, added to v
template <int CTRL> __device__ __forceinline__ float add_dpp(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// HALVES: pair p is channels (p, pairs + p), else (2p, 2p + 1).  The channels behind the pairs pass through.
template <typename T, bool HALVES, bool NORM>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  __shared__ f32x4_t sums[2][NORM ? kRopeThreads : 1];
  static_assert(kRopeHeads == 4, "one float4 of partial sums per thread");
  const int nchunk = a.d / 8, slot = threadIdx.x / nchunk, c = threadIdx.x % nchunk;
  const int64_t token = (int64_t)blockIdx.x * a.tokens_per_wg + slot;
  const bool live = slot < a.tokens_per_wg && token < a.tokens;
  const int64_t tk = live ? token : 0;
  const int64_t b = tk / a.N;
  const int n = (int)(tk - b * a.N);
  const bool turned = 4 * c < a.pairs;
  // this thread's channels: two runs of four
  const int c0 = HALVES && turned ? 4 * c : 8 * c, c1 = HALVES && turned ? a.pairs + 4 * c : 8 * c + 4;
  float cs[4], sn[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
  if (turned) {
    const int at = a.first + n, row = at / a.W, f = row / a.H, y = row - f * a.H, x = at - row * a.W;
    const double pf = fma(a.step[0], (double)f, a.origin[0]), py = fma(a.step[1], (double)y, a.origin[1]),
                 px = fma(a.step[2], (double)x, a.origin[2]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = 4 * c + i;
      const double rev = (p < a.end_f ? pf : p < a.end_y ? py : px) * a.freq[p];
      const double turn = rev - rint(rev);  // the whole turns drop out exactly
      const float near = (float)turn, rest = (float)(turn - (double)near) * 6.283185307f;  // what float32 cannot hold, in radians
      float s, co;
      sincospif(2.f * near, &s, &co);
      sn[i] = fmaf(co, rest, s);
      cs[i] = fmaf(-s, rest, co);
    }
  }
  Raw8<T> gq, gk;  // as they lie in memory: half the registers for bf16
  if constexpr (NORM) {
    auto gain = [&](const void* p, Raw8<T>& g) {
      if (!p) ones8(g);
      else if (HALVES && turned) load8<false>(static_cast<const T*>(p), c0, c1, g);
      else load8<true>(static_cast<const T*>(p), c0, c1, g);
    };
    gain(a.q_gain, gq);
    gain(a.k_gain, gk);
  }
  const int h_end = min(a.heads, (int)(blockIdx.y + 1) * a.heads_per_wg);
  int flip = 0;
  for (int h0 = blockIdx.y * a.heads_per_wg; h0 < h_end; h0 += kRopeHeads, flip ^= 1) {
    Raw8<T> raw[kRopeHeads] = {};
#pragma unroll
    for (int u = 0; u < kRopeHeads; ++u) {
      const int h = h0 + u < h_end ? h0 + u : h_end - 1;
      const HeadsView& s = h < a.heads_q ? a.q : a.k;
      const T* p = static_cast<const T*>(s.p) + b * s.sb + n * s.sn + (h < a.heads_q ? h : h - a.heads_q) * s.sh;
      if (live) {
        if (HALVES && turned) load8<false>(p, c0, c1, raw[u]);
        else load8<true>(p, c0, c1, raw[u]);
      }
    }
    float inv[kRopeHeads];
    if constexpr (NORM) {
      f32x4_t part;
#pragma unroll
      for (int u = 0; u < kRopeHeads; ++u) {
        float x[8];
        unpack8(raw[u], x);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(x[i], x[i], s);
        part[u] = s;
      }
      f32x4_t all = part;
      if ((nchunk & (nchunk - 1)) == 0) {  // a head's threads are neighbouring lanes, 1 to 16 of a row
#pragma unroll
        for (int u = 0; u < kRopeHeads; ++u) {
          if (nchunk > 1) all[u] = add_dpp<0xB1>(all[u]);   // lane ^ 1
          if (nchunk > 2) all[u] = add_dpp<0x4E>(all[u]);   // lane ^ 2
          if (nchunk > 4) all[u] = add_dpp<0x141>(all[u]);  // the other half of 8
          if (nchunk > 8) all[u] = add_dpp<0x140>(all[u]);  // the other half of 16
        }
      } else {
        sums[flip][threadIdx.x] = part;
        __syncthreads();
        all = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (live)
          for (int i = 0; i < nchunk; ++i) all += sums[flip][slot * nchunk + i];
      }
#pragma unroll
      for (int u = 0; u < kRopeHeads; ++u) inv[u] = rsqrtf(fmaf(all[u], a.inv_d, a.eps));
    }
    if (!live) continue;
#pragma unroll
    for (int u = 0; u < kRopeHeads; ++u) {
      const int h = h0 + u;
      if (h >= h_end) break;
      const bool is_q = h < a.heads_q;
      float x[8], y[8];
      unpack8(raw[u], x);
      if constexpr (NORM) {
        float gain[8];
        unpack8(is_q ? gq : gk, gain);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= inv[u] * gain[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int i1 = HALVES ? i : 2 * i, i2 = HALVES ? i + 4 : 2 * i + 1;
        y[i1] = x[i1] * cs[i] - x[i2] * sn[i];
        y[i2] = x[i1] * sn[i] + x[i2] * cs[i];
      }
      if (!turned) {  // passes through, also where a value is infinite
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i];
      }
      const HeadsView& s = is_q ? a.qo : a.ko;
      T* p = static_cast<T*>(s.p) + b * s.sb + n * s.sn + (is_q ? h : h - a.heads_q) * s.sh;
      if (HALVES && turned) store8<false>(p, c0, c1, y);
      else store8<true>(p, c0, c1, y);
    }
  }
}

}  // namespace si

// Attention of runs of queries over listed key blocks.
//
// A run is q_block consecutive queries of the `group` heads that share a key / value head: group * q_block rows, one list of
// key blocks (a bitmap).  One workgroup takes NW x 32 rows of a run and walks the run's blocks, a stage of kStageKeys keys at
// a time, with the running maximum and sum of a softmax:
//   S^T[key, row] = K Q^T       row operand: 32 keys, column operand: 32 rows (one wavefront's)
//   O^T[chan, row] += V^T P^T   column operand: the softmax result registers as they stand
// With queries as columns a lane holds 16 scores of one query, its running maximum and its half of the sum (the other half is
// lane ^ 32's), so the softmax needs no cross-lane traffic in the steady state.
//
// Keys and values go from their own rows to LDS with direct global->LDS loads, whole rows by neighbouring lanes (full
// cache lines), and lie there in rows of 16-byte pieces that lds_swizzle spreads over the banks.  bf16 values are transposed
// on their way out of LDS (ds_read_b64_tr_b16), so nothing has to be laid out before the call.
//
// When there are few rows (single new tokens) a run's blocks are dealt out to `nsplit` workgroups; each leaves its
// unnormalised output, maximum and sum, and sparse_join_kernel adds them in a fixed order.
#pragma once
#include "si_common.h"

namespace si {

struct SparseArgs {
  const void *q, *k, *v;
  void* o;
  int64_t qb, qn, qh, kb, kn, kh, vb, vn, vh, ob, on, oh;  // strides in elements
  const unsigned* mask;      // [B][kv heads][runs][words], or NULL: every block
  const int *q_len, *k_len;  // per batch entry, or NULL
  int Nq, Nk, heads_kv, group, d;
  int q_block, k_block, runs, words;
  int tiles_per_run;         // row tiles of a run
  int64_t work;              // B * heads_kv * runs * tiles_per_run * nsplit
  int nsplit;
  float c;                   // softmax scale * log2(e)
  float* part;               // nsplit > 1: [work][wave][OB * 4 + 1][64] of 16 bytes
  int o_frag;                // 0, or o is a fragment-order buffer of that many channels per token
};

// s_waitcnt immediate (gfx9 encoding): vmcnt <= n, other counters unconstrained
constexpr int vmcnt_imm(int n) { return (n & 0xF) | 0x70 | 0xF00 | ((n >> 4) << 14); }

constexpr float kSparseLow = -1e30f;  // reference maximum before the first key: below every score, and finite
constexpr float kSparseTrigger = 256.f;

// zero rows for keys past the end and channels past the head
static __device__ __align__(16) const unsigned kSparseZero[4] = {0, 0, 0, 0};

// The key blocks of one run, as the first keys of stages of SK keys in ascending order.  Every wavefront walks the list
// with scalar registers: 64 words of the bitmap (2048 blocks) lie one per lane.
template <int SK>
struct BlockWalk {
  const unsigned* words;
  int nwords, nblk, k_block, k_len;
  int base, lane;
  unsigned mine;             // this lane's word of the chunk
  unsigned long long left;   // lanes of the chunk whose word has not been opened
  unsigned bits;             // of the open word
  int word, rem;             // open word; blocks still to hand out
  int key, key_end;          // of the open block

  __device__ __forceinline__ unsigned load(int at) const {
    if (at >= nwords) return 0u;
    unsigned w = words ? words[at] : ~0u;
    const int n = nblk - 32 * at;  // bits past the last block are nobody's
    if (n < 32) w = n <= 0 ? 0u : w & ((1u << n) - 1u);
    return w;
  }
  __device__ __forceinline__ void open_chunk(int at) {
    base = at;
    mine = load(base + lane);
    left = __builtin_amdgcn_ballot_w64(mine != 0u);
    bits = 0u;
  }
  // share `part` of `parts` of the list
  __device__ __forceinline__ void begin(const unsigned* w, int nw, int nb, int kb, int kl, int part, int parts) {
    words = w; nwords = nw; nblk = nb; k_block = kb; k_len = kl;
    lane = threadIdx.x % kWave;
    key = key_end = 0;
    open_chunk(0);
    if (parts == 1) {  // all of it: the walk ends when the words do
      rem = 0x7fffffff;
      return;
    }
    int count = 0;
    for (int at = 0; at < nwords; at += kWave) {
      int n = __popc(load(at + lane));
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, kWave);
      count += n;
    }
    count = __builtin_amdgcn_readfirstlane(count);
    int skip = (int)((int64_t)count * part / parts);
    rem = (int)((int64_t)count * (part + 1) / parts) - skip;
    for (;;) {  // to the word that holds block number `skip` of the list
      int upto = __popc(mine);
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int n = __shfl_up(upto, o, kWave);
        if (lane >= o) upto += n;
      }
      const unsigned long long past = __builtin_amdgcn_ballot_w64(upto > skip);
      if (past) {
        word = __builtin_ctzll(past);
        const int before = __builtin_amdgcn_readlane(upto, word) - __popc(__builtin_amdgcn_readlane(mine, word));
        bits = __builtin_amdgcn_readlane(mine, word);
        for (int i = before; i < skip; ++i) bits &= bits - 1u;
        left &= word == 63 ? 0ull : ~0ull << (word + 1);
        break;
      }
      skip -= __builtin_amdgcn_readlane(upto, kWave - 1);
      if (base + kWave >= nwords) { rem = 0; break; }
      open_chunk(base + kWave);
    }
  }
  // first key of the next stage, or -1
  __device__ __forceinline__ int next() {
    if (key >= key_end) {
      if (rem <= 0) return -1;
      while (bits == 0u) {
        if (left == 0ull) {
          if (base + kWave >= nwords) { rem = 0; return -1; }
          open_chunk(base + kWave);
          continue;
        }
        word = __builtin_ctzll(left);
        left &= left - 1ull;
        bits = __builtin_amdgcn_readlane(mine, word);
      }
      const int j = 32 * (base + word) + __builtin_ctz(bits);
      bits &= bits - 1u;
      --rem;
      key = j * k_block;
      key_end = k_len - key < k_block ? k_len : key + k_block;  // a listed block has a key: nblk counts those that do
    }
    const int at = key;
    key += SK;
    return at;
  }
};

template <typename T> struct SparseShape;
template <> struct SparseShape<bf16> {
  static constexpr int SK = 64, VEC = 8;  // keys of a stage, elements of a 16-byte piece
};
template <> struct SparseShape<float> {
  static constexpr int SK = 32, VEC = 4;
};

// Piece p of row r lies in slot p ^ lds_swizzle(r) of its row.  LDS reads 256 bytes per clock.  Keys: 16 lanes read one piece of
// 16 rows, which have to fall on 16 different groups of four banks.  bf16 values: 32 lanes read four pieces of four rows, so
// the rows' lowest bits have to move the slot by four; float32 values: 64 lanes read eight pieces of rows that differ in
// bit 2.  (The first form, p ^ (r & 7), lost half of the LDS's cycles to conflicts: 57600 tokens 1930 us.)
// Every bit of the row moves bits of the slot by itself: lds_swizzle(a | b) = lds_swizzle(a) ^ lds_swizzle(b) for disjoint a, b.
template <int ROW, bool F32>
__device__ constexpr int lds_swizzle(int r) {
  if (ROW == 64) return (r >> 2) & 3;
  if (ROW == 128) return ((r >> 1) & 1) << 2 | ((r >> 2) & 1) << 1 | ((r >> 3) & 1);
  if (F32) return (r & 3) | ((r >> 3) & 1) << 2 | ((r >> 2) & 1) << 3;
  return (r & 3) << 2 | ((r >> 2) & 3);
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));

template <typename V> __device__ __forceinline__ V lds_read(unsigned at) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V*>((size_t)at);
}
// ds_read_b64_tr_b16: of the 16 lanes of a group, lane i reads 8 bytes of its own address (row i / 4, columns
// 4 (i % 4) .. + 3 of a 4 x 16 tile) and receives column i: four rows' values of one channel
__device__ __forceinline__ uint2 lds_read_tr(unsigned at) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4_t*>((size_t)at)));
}

// Output of one wavefront: lane (r, g) holds query row r's channels 32 b + 8 q + 4 g + j in register 16 b + 4 q + j.
template <typename T, int OB>
__device__ __forceinline__ void sparse_store(const SparseArgs& a, const f32x16_t (&o)[OB], float lsum, int b, int hk, int token, int sub,
                                             bool valid, int g) {
  if (!valid) return;
  const float inv = lsum > 0.f ? 1.f / lsum : 0.f;  // a row without keys gives zero
  const int h = hk * a.group + sub;
  T* row = static_cast<T*>(a.o) + b * a.ob + (int64_t)token * a.on + (int64_t)h * a.oh;
#pragma unroll
  for (int i = 0; i < OB; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int ch = 32 * i + 8 * q + 4 * g;
      if (ch >= a.d) continue;
      float y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = lsum > 0.f ? o[i][4 * q + j] * inv : 0.f;
      if constexpr (sizeof(T) == 2) {
        bf16* dst = a.o_frag ? static_cast<bf16*>(a.o) + act_offset((int64_t)b * a.Nq + token, h * a.d + ch, a.o_frag)
                             : reinterpret_cast<bf16*>(row) + ch;
        *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
      } else {
        *reinterpret_cast<f32x4_t*>(row + ch) = f32x4_t{y[0], y[1], y[2], y[3]};
      }
    }
}

// KS: head channels in steps of 16 (d <= 16 KS).
template <typename T, int KS, int NW>
__global__ __launch_bounds__(64 * NW, NW < 4 ? 1 : KS <= 4 && sizeof(T) == 2 ? 3 : 2) void sparse_attn_kernel(SparseArgs a) {
  using Shape = SparseShape<T>;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int SK = Shape::SK, VEC = Shape::VEC;
  constexpr int NP = KS * 16 / VEC;                               // 16-byte pieces of a padded head
  constexpr int PR = NP <= 4 ? 4 : NP <= 8 ? 8 : NP <= 16 ? 16 : 32;  // pieces of a row in LDS
  constexpr int ROW = PR * 16;                                    // bytes
  constexpr int OB = (KS + 1) / 2;                                // 32-channel blocks of the output
  constexpr int HALF = SK * ROW;                                  // bytes of a stage's keys; its values follow
  constexpr int NS = HALF <= 8192 ? 3 : 2;                        // stages in LDS
  constexpr int LOADS = HALF / 1024;                              // wave-wide loads of a stage's keys
  constexpr int PER = LOADS / NW;                                 // per wavefront
  constexpr int QS = F32 ? KS * 2 : KS;                           // pieces of a query per lane
  static_assert(LOADS % NW == 0, "every wavefront issues the same number of loads, the waits count them");
  __shared__ __align__(1024) u32x4_t ring[NS * 2 * HALF / 16];
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) void*)(&ring[0]);
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = lane % 32, g = lane / 32;
  auto swizzle = [](int row) { return lds_swizzle<ROW, F32>(row); };

  // ---- what stays the same through all stages, per lane.  Load i of a half: rows (wave + NW i) (64 / PR) .., lane l takes
  // slot l % PR of row l / PR of them.
  unsigned koff[PER], voff[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int row = (wave + NW * i) * (64 / PR) + lane / PR, piece = (lane % PR) ^ swizzle(row);
    koff[i] = (unsigned)(row * (int)a.kn + piece * VEC) * (unsigned)sizeof(T);  // the host keeps this inside 31 bits
    voff[i] = (unsigned)(row * (int)a.vn + piece * VEC) * (unsigned)sizeof(T);
  }
  const bool whole_rows = a.d == PR * VEC;
  // LDS addresses of the first fragments; pieces further on are exclusive-ors (rows are aligned to their length), and so is
  // what a row further on changes in the slot
  const unsigned kat = lds0 + r * ROW + (g ^ swizzle(r)) * 16;  // piece 2 s + g: ^ 32 s
  // bf16: step t of 16 keys: slots e < 4 of group g are keys 16 t + 4 g + e, the others 16 t + 8 + 4 g + e - 4; channel block i: ^ 64 i
  // f32: register (q, j) of the scores is key 8 q + 4 g + j; channel block i: ^ 128 i
  const int vr = F32 ? 4 * g : 4 * g + (lane % 16) / 4;
  const unsigned vat = lds0 + HALF + vr * ROW +
                       (F32 ? ((r / 4) ^ swizzle(vr)) * 16 + (r % 4) * 4 : ((2 * ((lane / 16) % 2) + (lane % 4) / 2) ^ swizzle(vr)) * 16 + (lane % 2) * 8);

  // Work goes to the 8 XCDs in contiguous chunks, so that the keys and values of a head are fetched into one L2.
  const int64_t chunk = (a.work + 7) / 8;
  const int64_t chunk_end = min(a.work, ((int64_t)(blockIdx.x % 8) + 1) * chunk);
  for (int64_t work = (int64_t)(blockIdx.x % 8) * chunk + blockIdx.x / 8; work < chunk_end; work += gridDim.x / 8) {
    const int part = (int)(work % a.nsplit);
    int64_t at = work / a.nsplit;
    const int tile = (int)(at % a.tiles_per_run);
    at /= a.tiles_per_run;
    const int run = (int)(at % a.runs);
    at /= a.runs;
    const int hk = (int)(at % a.heads_kv), b = (int)(at / a.heads_kv);
    const int q_len = a.q_len ? min(max(a.q_len[b], 0), a.Nq) : a.Nq, k_len = a.k_len ? min(max(a.k_len[b], 0), a.Nk) : a.Nk;
    // this lane's query row
    const int rho = (tile * NW + wave) * 32 + r, in_run = rho / a.group, sub = rho - in_run * a.group;
    const int64_t token64 = (int64_t)run * a.q_block + in_run;
    const bool valid = in_run < a.q_block && token64 < q_len;
    const int token = valid ? (int)token64 : 0;

    BlockWalk<SK> walk;
    const unsigned* mrow = a.mask ? a.mask + (((int64_t)b * a.heads_kv + hk) * a.runs + run) * a.words : nullptr;
    // a tile without a query walks nothing (the first row of the tile is its earliest token)
    const int first_row = tile * NW * 32, first_tok = first_row / a.group;
    const bool any = first_tok < a.q_block && (int64_t)run * a.q_block + first_tok < q_len;
    walk.begin(mrow, any ? a.words : 0, (k_len + a.k_block - 1) / a.k_block, a.k_block, k_len, part, a.nsplit);

    const char* const kbase = static_cast<const char*>(a.k) + ((int64_t)b * a.kb + (int64_t)hk * a.kh) * (int64_t)sizeof(T);
    const char* const vbase = static_cast<const char*>(a.v) + ((int64_t)b * a.vb + (int64_t)hk * a.vh) * (int64_t)sizeof(T);
    int issued = 0, last_keys = SK;
    unsigned islot = 0;
    // assembly: completion is awaited explicitly, the compiler would wait for all of it before the next LDS read
    auto issue = [&]() {
      const int key0 = walk.next();
      if (key0 < 0) return;
      const int nkeys = min(SK, k_len - key0);
      last_keys = nkeys;
      const char* ksrc = kbase + (int64_t)key0 * a.kn * (int64_t)sizeof(T);
      const char* vsrc = vbase + (int64_t)key0 * a.vn * (int64_t)sizeof(T);
      const unsigned dst = lds0 + islot + wave * 1024;
      if (nkeys == SK && whole_rows) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(koff[i]), "s"(ksrc), "s"(dst + NW * i * 1024) : "memory");
          asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(voff[i]), "s"(vsrc), "s"(dst + HALF + NW * i * 1024) : "memory");
        }
      } else {  // keys past the end and channels past the head as zeros
        int l = lane;
        asm volatile("" : "+v"(l));  // rows and pieces are formed here again: kept through the loop they cost registers
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int row = (wave + NW * i) * (64 / PR) + l / PR, piece = (l % PR) ^ swizzle(row);
          const bool in = piece * VEC < a.d && row < nkeys;
          const char* ks = in ? ksrc + koff[i] : reinterpret_cast<const char*>(kSparseZero);
          const char* vs = in ? vsrc + voff[i] : reinterpret_cast<const char*>(kSparseZero);
          asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(ks), "s"(dst + NW * i * 1024) : "memory");
          asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(vs), "s"(dst + HALF + NW * i * 1024) : "memory");
        }
      }
      islot = islot == (NS - 1) * 2 * HALF ? 0 : islot + 2 * HALF;
      ++issued;
    };
    for (int i = 0; i < NS - 1; ++i) issue();

    // ---- this lane's query as column operand: pieces as the keys' fragments have them
    u32x4_t qop[QS];
    {
      const T* qrow = static_cast<const T*>(a.q) + b * a.qb + (int64_t)token * a.qn + (int64_t)(hk * a.group + (valid ? sub : 0)) * a.qh;
#pragma unroll
      for (int s = 0; s < QS; ++s) {
        const int piece = 2 * s + g;
        qop[s] = u32x4_t{0, 0, 0, 0};
        if (piece * VEC < a.d && q_len > 0) qop[s] = *reinterpret_cast<const u32x4_t*>(qrow + piece * VEC);
      }
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // the query: nothing that the compiler tracks stays pending in the loop

    f32x16_t oacc[OB];
    float mref = kSparseLow, lsum = 0.f;
#pragma unroll
    for (int i = 0; i < OB; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) oacc[i][e] = 0.f;
    unsigned cslot = 0;
    for (int st = 0; st < issued; ++st) {
      const int younger = issued - 1 - st;  // stages in flight behind this one: at most NS - 2
      if (NS == 3 && younger >= 1) __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * PER));
      else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      __syncthreads();  // the stage is there for all, and nobody reads the slot that is filled next
      issue();
      const int nkeys = st + 1 == issued ? last_keys : SK;  // only the list's last stage can hold fewer

      // ---- scores of SK / 32 tiles of 32 keys
      f32x16_t sc[SK / 32];
#pragma unroll
      for (int u = 0; u < SK / 32; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[u][e] = 0.f;
      constexpr int KF = F32 ? 1 : QS;  // pieces of a key that are read ahead of the products
      u32x4_t kf[KF][SK / 32];
#pragma unroll
      for (int s = 0; s < QS; ++s) {
        if (s % KF == 0) {
#pragma unroll
          for (int i = 0; i < KF; ++i)
#pragma unroll
            for (int u = 0; u < SK / 32; ++u) kf[i][u] = lds_read<u32x4_t>(((kat + cslot) ^ (32 * (s + i))) + 32 * u * ROW);
          if constexpr (!F32) __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int u = 0; u < SK / 32; ++u) {
          if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              sc[u] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[0][u][j]), __uint_as_float(qop[s][j]), sc[u], 0, 0, 0);
          } else {
            sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[s][u]), __builtin_bit_cast(bf16x8_t, qop[s]), sc[u], 0, 0, 0);
          }
        }
      }
      if (nkeys < SK) {
        const int lim = nkeys - 4 * g;  // register e of tile u is key 32 u + 8 (e / 4) + e % 4 + 4 g
#pragma unroll
        for (int u = 0; u < SK / 32; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (32 * u + 8 * (e / 4) + e % 4 >= lim) sc[u][e] = -INFINITY;
      }
      // bf16 values on their way while the exponentials are taken
      constexpr int VT = F32 ? 1 : SK / 16;
      uint2 vlo[VT][OB], vhi[VT][OB];
      if constexpr (!F32) {
#pragma unroll
        for (int t = 0; t < VT; ++t)
#pragma unroll
          for (int i = 0; i < OB; ++i) {
            vlo[t][i] = lds_read_tr(((vat + cslot) ^ (64 * i)) + 16 * t * ROW);
            vhi[t][i] = lds_read_tr(((vat + cslot) ^ (64 * i) ^ (lds_swizzle<ROW, F32>(8) * 16)) + (16 * t + 8) * ROW);
          }
        __builtin_amdgcn_sched_barrier(0);
      }

      // ---- probabilities against the lazy reference maximum: it is raised only when the partial sums say that an
      // exponent has grown past it, so that the steady state has no maximum and no rescaling.  exp2 of up to 2^8 is
      // harmless in float32 and, relative as bf16 rounds, in bf16.
      u32x4_t pk[F32 ? 1 : SK / 16];
      float pf[F32 ? 16 : 1];
      auto exponentiate = [&]() {
        float rs = 0.f;
#pragma unroll
        for (int u = 0; u < SK / 32; ++u)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[u][e], a.c, -mref)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[u][e + 1], a.c, -mref));
            if constexpr (F32) {
              pf[e] = p0;
              pf[e + 1] = p1;
              rs += p0 + p1;
            } else {  // the sum is of the rounded values, those that weigh V
              const unsigned w = pack_bf16x2(p0, p1);
              pk[2 * u + e / 8][e % 8 / 2] = w;
              rs = dot2_ones(w, rs);
            }
          }
        return rs;
      };
      float rs = exponentiate();
      if (__builtin_amdgcn_ballot_w64(!(rs <= kSparseTrigger)) != 0) {
        float mx = sc[0][0];
#pragma unroll
        for (int u = 0; u < SK / 32; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[u][e]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave)) * a.c;  // both halves of the row agree on the new reference
        const float up = fmaxf(mx, mref), alpha = __builtin_amdgcn_exp2f(mref - up);
        mref = up;
        lsum *= alpha;
#pragma unroll
        for (int i = 0; i < OB; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[i][e] *= alpha;
        rs = exponentiate();
      }
      lsum += rs;

      // ---- O^T += V^T P^T
      if constexpr (F32) {
        // one step of two keys: the lane's own and lane ^ 32's
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < OB; ++i)
              oacc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(lds_read<float>(((vat + cslot) ^ (lds_swizzle<ROW, F32>(8 * q + j) * 16) ^ (128 * i)) + (8 * q + j) * ROW), pf[4 * q + j], oacc[i], 0, 0, 0);
      } else {
#pragma unroll
        for (int t = 0; t < SK / 16; ++t)
#pragma unroll
          for (int i = 0; i < OB; ++i) {
            const u32x4_t vf{vlo[t][i].x, vlo[t][i].y, vhi[t][i].x, vhi[t][i].y};
            oacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf), __builtin_bit_cast(bf16x8_t, pk[t]), oacc[i], 0, 0, 0);
          }
      }
      cslot = cslot == (NS - 1) * 2 * HALF ? 0 : cslot + 2 * HALF;
    }
    lsum += __shfl_xor(lsum, 32, kWave);
    if (a.nsplit == 1) {
      sparse_store<T, OB>(a, oacc, lsum, b, hk, token, sub, valid, g);
    } else if (valid) {  // rows that hold no query are not read back either
      f32x4_t* img = reinterpret_cast<f32x4_t*>(a.part) + (work * NW + wave) * (OB * 4 + 1) * kWave + lane;
#pragma unroll
      for (int i = 0; i < OB * 4; ++i)
        img[i * kWave] = f32x4_t{oacc[i / 4][i % 4 * 4], oacc[i / 4][i % 4 * 4 + 1], oacc[i / 4][i % 4 * 4 + 2], oacc[i / 4][i % 4 * 4 + 3]};
      img[OB * 4 * kWave] = f32x4_t{mref, lsum, 0.f, 0.f};
    }
    __syncthreads();  // the next tile's loads overwrite the ring
  }
}

// The shares of a row tile joined: weights 2^(m - max m), in the order of the shares.  A wavefront takes four channels per
// lane of one 32-row image; blockIdx.y * 4 + wavefront says which.
template <typename T, int OB, int NW>
__global__ __launch_bounds__(256) void sparse_join_kernel(SparseArgs a) {
  const int lane = threadIdx.x % kWave, i = blockIdx.y * 4 + threadIdx.x / kWave, r = lane % 32, g = lane / 32;
  const int64_t images = a.work / a.nsplit * NW, pitch = (int64_t)NW * (OB * 4 + 1) * kWave;
  for (int64_t im = blockIdx.x; im < images; im += gridDim.x) {
    const int64_t t = im / NW;
    const int wave = (int)(im % NW);
    int64_t at = t;
    const int tile = (int)(at % a.tiles_per_run);
    at /= a.tiles_per_run;
    const int run = (int)(at % a.runs);
    at /= a.runs;
    const int hk = (int)(at % a.heads_kv), b = (int)(at / a.heads_kv);
    const int q_len = a.q_len ? min(max(a.q_len[b], 0), a.Nq) : a.Nq;
    const int rho = (tile * NW + wave) * 32 + r, in_run = rho / a.group, sub = rho - in_run * a.group;
    const int64_t token = (int64_t)run * a.q_block + in_run;
    const int ch = 32 * (i / 4) + 8 * (i % 4) + 4 * g;
    if (in_run >= a.q_block || token >= q_len || ch >= a.d) continue;
    const f32x4_t* img = reinterpret_cast<const f32x4_t*>(a.part) + (t * a.nsplit * NW + wave) * (OB * 4 + 1) * kWave + lane;
    float top = kSparseLow;
#pragma unroll 8
    for (int s = 0; s < a.nsplit; ++s) top = fmaxf(top, img[s * pitch + OB * 4 * kWave][0]);
    float l = 0.f;
    f32x4_t o{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < a.nsplit; ++s) {
      const f32x4_t ml = img[s * pitch + OB * 4 * kWave], x = img[s * pitch + i * kWave];
      const float w = __builtin_amdgcn_exp2f(ml[0] - top);
      l = fmaf(ml[1], w, l);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = fmaf(x[j], w, o[j]);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    T* dst = static_cast<T*>(a.o) + b * a.ob + token * a.on + (int64_t)(hk * a.group + sub) * a.oh + ch;
    if constexpr (sizeof(T) == 2) {
      if (a.o_frag) dst = static_cast<T*>(a.o) + act_offset((int64_t)b * a.Nq + token, (hk * a.group + sub) * a.d + ch, a.o_frag);
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    } else {
      *reinterpret_cast<f32x4_t*>(dst) = f32x4_t{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    }
  }
}

}  // namespace si

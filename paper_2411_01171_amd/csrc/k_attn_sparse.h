// Attention of runs of queries over listed key blocks.
//
// A run is q_block consecutive queries of the `group` heads that share a key / value head: group * q_block rows, one list of
// key blocks (a bitmap).  One workgroup takes 16 to 128 rows of a run and walks the run's blocks, a stage of 64 (float32: 32)
// keys at a time, with the running maximum and sum of a softmax.  bf16: 32 rows on one wavefront, 64 on four (two to the same
// rows, SPLIT), 128 on four; float32: 16 rows to a wavefront, in workgroups of 16, 32 and 64, or 32 to each of four (H).
//   S^T[key, row] = K Q^T       row operand: keys, column operand: rows
//   O^T[chan, row] += V^T P^T   column operand: the softmax result registers as they stand
// With queries as columns a lane holds scores of one query (float32: of H), its running maximum and its part of the sum, so
// the softmax needs no cross-lane traffic in the steady state.
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
  unsigned work;             // B * heads_kv * runs * tiles_per_run * nsplit
  int nsplit;
  float c;                   // softmax scale * log2(e)
  float* part;               // nsplit > 1: outputs [query row][nsplit][d], then (maximum, sum) [query row][nsplit]; query row = (b Nq + n) heads + h
  float2* part_ml;
  int o_frag;                // 0, or o is a fragment-order buffer of that many channels per token
};

// s_waitcnt immediate (gfx9 encoding): vmcnt <= n, other counters unconstrained
constexpr int vmcnt_imm(int n) { return (n & 0xF) | 0x70 | 0xF00 | ((n >> 4) << 14); }

constexpr float kSparseLow = -1e30f;  // reference maximum before the first key: below every score, and finite
constexpr float kSparseTrigger = 256.f;

// zero rows for keys past the end
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

// What all kernels share: where a head's rows lie in LDS.
template <typename T, int KS, int NW>
struct SparseGeo {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int SK = F32 ? 32 : 64;                            // keys of a stage
  static constexpr int VEC = 16 / sizeof(T);                          // elements of a 16-byte piece
  static constexpr int NP = KS * 16 / VEC;                            // pieces of a padded head
  static constexpr int PR = NP <= 4 ? 4 : NP <= 8 ? 8 : NP <= 16 ? 16 : 32;  // pieces of a row in LDS
  static constexpr int ROW = PR * 16;                                 // bytes
  static constexpr int HALF = SK * ROW;                               // bytes of a stage's keys; its values follow
  // Stages in LDS.  A wavefront on its own has no other that waits with it: two, and more workgroups (runs of 32 rows, heads of
  // 64, 164 -> 142 us; one token against 16384 keys of 8 heads of 64, 39 -> 33 us).
  static constexpr int NS = !F32 && HALF <= 8192 && NW > 1 ? 3 : 2;
  static constexpr int LOADS = HALF / 1024;                           // wave-wide loads of a stage's keys

  // Piece p of row r lies in slot p ^ swizzle(r) of its row.  LDS reads 256 bytes per clock.  Keys: the lanes of a clock read
  // one piece of 16 rows, which have to fall on 16 different groups of four banks (float32 still has conflicts).  Values: they read the pieces of 32 (bf16)
  // or 16 (float32) channels of four rows, which differ in bits 0 and 1 (bf16) or 2 and 3 (float32): those bits have to move
  // the slot by four.  (p ^ (r & 7) lost half of the LDS's cycles to conflicts: heads of 128, padded batch, 429 us against 388.)
  // Every bit of the row moves bits of the slot by itself: swizzle(a | b) = swizzle(a) ^ swizzle(b) for disjoint a and b.
  static __host__ __device__ constexpr int swizzle(int r) {
    return ROW == 64 ? (r >> 2) & 3
           : ROW == 128 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 1) << 1 | ((r >> 3) & 1)
           : F32 ? r & 15
                 : (r & 3) << 2 | ((r >> 2) & 3);
  }
};

typedef short s16x4_t __attribute__((ext_vector_type(4)));

template <typename V> __device__ __forceinline__ V lds_read(unsigned at) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V*>((size_t)at);
}
// ds_read_b64_tr_b16: of the 16 lanes of a group, lane i reads 8 bytes of its own address (row i / 4, columns
// 4 (i % 4) .. + 3 of a 4 x 16 tile) and receives column i: four rows' values of one channel
__device__ __forceinline__ uint2 lds_read_tr(unsigned at) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4_t*>((size_t)at)));
}

// One row tile of a run, or a share of its blocks.
struct SparseTile {
  int part, tile, run, hk, b, q_len, k_len;
  __device__ __forceinline__ SparseTile(const SparseArgs& a, unsigned work) {
    auto pop = [&](int n) {  // the fastest index
      const unsigned up = work / (unsigned)n;
      const int i = (int)(work - up * n);
      work = up;
      return i;
    };
    part = a.nsplit > 1 ? pop(a.nsplit) : 0;
    tile = a.tiles_per_run > 1 ? pop(a.tiles_per_run) : 0;
    run = pop(a.runs);
    hk = pop(a.heads_kv);
    b = (int)work;
    q_len = a.q_len ? min(max(a.q_len[b], 0), a.Nq) : a.Nq;
    k_len = a.k_len ? min(max(a.k_len[b], 0), a.Nk) : a.Nk;
  }
  // token of row `rho` of the run, or -1; sub: its head among those of the key head
  __device__ __forceinline__ int token(const SparseArgs& a, int rho, int& sub) const {
    const int in_run = a.group > 1 ? rho / a.group : rho;
    const int64_t n = (int64_t)run * a.q_block + in_run;
    sub = rho - in_run * a.group;
    return in_run < a.q_block && n < q_len ? (int)n : -1;
  }
  template <int SK>
  __device__ __forceinline__ void begin(const SparseArgs& a, int rows, BlockWalk<SK>& walk) const {
    const unsigned* list = a.mask ? a.mask + (((int64_t)b * a.heads_kv + hk) * a.runs + run) * a.words : nullptr;
    int sub;
    const bool any = token(a, tile * rows, sub) >= 0;  // the tile's first row is its earliest token; without one it walks nothing
    walk.begin(list, any ? a.words : 0, (k_len + a.k_block - 1) / a.k_block, a.k_block, k_len, part, a.nsplit);
  }
};

// The stages of a workgroup's list on their way to LDS, by direct global->LDS loads whose completion is awaited explicitly.
template <typename T, int KS, int NW>
struct StageLoads {
  using G = SparseGeo<T, KS, NW>;
  static constexpr int PER = G::LOADS / NW;  // loads of a stage's keys per wavefront, and of its values
  static_assert(G::LOADS % NW == 0, "every wavefront issues the same number of loads, the waits count them");
  unsigned lds0, slot;
  int lane, wave;
  // Load i: rows (wave + NW i) (64 / PR) .., lane l takes slot l % PR of row l / PR of them; slots of channels past the head
  // receive the row's first piece, and whoever reads them does not use it.
  unsigned koff[PER], voff[PER];
  const char *kbase, *vbase;
  int issued, last_keys;

  __device__ __forceinline__ void setup(const SparseArgs& a, unsigned at) {
    lds0 = at;
    lane = threadIdx.x % kWave;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int row = (wave + NW * i) * (64 / G::PR) + lane / G::PR, at = (lane % G::PR) ^ G::swizzle(row), piece = at * G::VEC < a.d ? at : 0;
      koff[i] = (unsigned)(row * (int)a.kn + piece * G::VEC) * (unsigned)sizeof(T);  // the host keeps this inside 31 bits
      voff[i] = (unsigned)(row * (int)a.vn + piece * G::VEC) * (unsigned)sizeof(T);
    }
  }
  __device__ __forceinline__ void begin(const SparseArgs& a, const SparseTile& t) {
    kbase = static_cast<const char*>(a.k) + ((int64_t)t.b * a.kb + (int64_t)t.hk * a.kh) * (int64_t)sizeof(T);
    vbase = static_cast<const char*>(a.v) + ((int64_t)t.b * a.vb + (int64_t)t.hk * a.vh) * (int64_t)sizeof(T);
    issued = 0;
    last_keys = G::SK;
    slot = 0;
  }
  __device__ __forceinline__ void issue(const SparseArgs& a, BlockWalk<G::SK>& walk) {
    const int key0 = walk.next();
    if (key0 < 0) return;
    const int nkeys = min(G::SK, walk.k_len - key0);
    last_keys = nkeys;
    const char* ksrc = kbase + (int64_t)key0 * a.kn * (int64_t)sizeof(T);
    const char* vsrc = vbase + (int64_t)key0 * a.vn * (int64_t)sizeof(T);
    const unsigned dst = lds0 + slot + wave * 1024;
    if (nkeys == G::SK) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        load_to_lds(koff[i], ksrc, dst + NW * i * 1024);
        load_to_lds(voff[i], vsrc, dst + G::HALF + NW * i * 1024);
      }
    } else {  // keys past the end as zeros
      int l = lane;
      asm volatile("" : "+v"(l));  // rows are formed here again: kept through the loop they cost registers
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const bool in = (wave + NW * i) * (64 / G::PR) + l / G::PR < nkeys;
        const char* ks = in ? ksrc + koff[i] : reinterpret_cast<const char*>(kSparseZero);
        const char* vs = in ? vsrc + voff[i] : reinterpret_cast<const char*>(kSparseZero);
        load_to_lds(ks, dst + NW * i * 1024);
        load_to_lds(vs, dst + G::HALF + NW * i * 1024);
      }
    }
    slot = slot == (G::NS - 1) * 2 * G::HALF ? 0 : slot + 2 * G::HALF;
    ++issued;
  }
  // Stage st is there for all, and nobody reads the slot that is filled next; returns its keys.
  __device__ __forceinline__ int open(const SparseArgs& a, BlockWalk<G::SK>& walk, int st) {
    const int younger = issued - 1 - st;  // stages in flight behind this one: at most NS - 2
    if (G::NS == 3 && younger >= 1) __builtin_amdgcn_s_waitcnt(vmcnt_imm(2 * PER));
    else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    __syncthreads();
    issue(a, walk);
    return st + 1 == issued ? last_keys : G::SK;  // only the list's last stage can hold fewer
  }
};

// Four channels of a query row: the result, or (nsplit > 1) its share.
template <typename T>
__device__ __forceinline__ void sparse_put(const SparseArgs& a, const SparseTile& t, int token, int sub, int ch, f32x4_t o, float lsum) {
  const int h = t.hk * a.group + sub;
  if (a.nsplit > 1) {
    const int64_t share = (((int64_t)t.b * a.Nq + token) * (a.heads_kv * a.group) + h) * a.nsplit + t.part;
    *reinterpret_cast<f32x4_t*>(a.part + share * a.d + ch) = o;
    return;
  }
  const float inv = 1.f / lsum;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = lsum == 0.f ? 0.f : o[j] * inv;  // a row without keys gives zero; a sum that is NaN stays one
  T* dst = static_cast<T*>(a.o) + t.b * a.ob + (int64_t)token * a.on + (int64_t)h * a.oh + ch;
  if constexpr (sizeof(T) == 2) {
    if (a.o_frag) dst = static_cast<T*>(a.o) + act_offset((int64_t)t.b * a.Nq + token, h * a.d + ch, a.o_frag);
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
  } else {
    *reinterpret_cast<f32x4_t*>(dst) = o;
  }
}
__device__ __forceinline__ void sparse_put_ml(const SparseArgs& a, const SparseTile& t, int token, int sub, float m, float l) {
  const int64_t share = (((int64_t)t.b * a.Nq + token) * (a.heads_kv * a.group) + t.hk * a.group + sub) * a.nsplit + t.part;
  a.part_ml[share] = make_float2(m, l);
}

// bf16.  KS: head channels in steps of 16 (d <= 16 KS).  v_mfma_f32_32x32x16_bf16: a wavefront's 32 rows are its columns; a
// result lane (r, g) holds column r and, in register 4 q + j, row 8 q + 4 g + j.
//
// Bound by the vector ALUs and the matrix cores together: per 32 rows x 64 keys and head of 64, 512 clocks of MFMA and, beside
// them, 32 exponentials (8 clocks each), 32 fma (the scale stays in float32: folded into q before a second rounding of q it
// would save 4 % at 57600 tokens), 16 conversions and 16 sums of pairs; the two hardly overlap, whatever the number of
// wavefronts (four per SIMD, sharing rows in pairs, 1958 us at 57600 tokens against 1858 with three); and by power: in long
// launches the clock falls to 1.8 GHz.  72x128 frame over a quarter of its keys 69 us (784 TFLOP/s, 10 of them before the first
// product and behind the last), 57600 tokens over a tenth 1867 us (910); a library product of 8192^3 reaches 1420.  Heads of
// 128 in runs of 128: 9216 tokens of 5 heads 870 TFLOP/s, 28800 of 8 heads 1046; in runs of 400 rows, whose last tile of 128
// holds 16, 750.  s_setprio around either half changes nothing.
// PAD: d < 16 KS; what the keys' fragments hold past the head is made zero, as the queries are there.
// SPLIT 2: two wavefronts share 32 rows and take half of a stage's keys each, joined at the end: a run of 64 rows then has four
// wavefronts on a CU for every stage in its LDS, not two (72x128 frame, runs of 64: 112 -> 79 us).
template <int KS, int NW, bool PAD, int SPLIT>
__global__ __launch_bounds__(64 * NW, NW < 4 ? 1 : KS <= 4 ? 3 : 2) void sparse_attn_bf16_kernel(SparseArgs a) {
  constexpr int UT = 2 / SPLIT;  // 32-key tiles of a stage per wavefront
  using G = SparseGeo<bf16, KS, NW>;
  constexpr int SK = G::SK, ROW = G::ROW;
  constexpr int OB = (KS + 1) / 2;  // 32-channel blocks of the output
  __shared__ __align__(1024) u32x4_t ring[G::NS * 2 * G::HALF / 16];
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) void*)(&ring[0]);
  StageLoads<bf16, KS, NW> loads;
  loads.setup(a, lds0);
  const int lane = loads.lane, r = lane % 32, g = lane / 32;
  const int rows_of = loads.wave % (NW / SPLIT), share = loads.wave / (NW / SPLIT);  // this wavefront's rows, and its half of the keys
  // LDS addresses of the first fragments; pieces further on are exclusive-ors (rows are aligned to their length), and so is
  // what a row further on changes in the slot
  const unsigned kat = lds0 + (32 * share + r) * ROW + (g ^ G::swizzle(r)) * 16;  // piece 2 s + g: ^ 32 s
  // step t of 16 keys: slots e < 4 of group g are keys 16 t + 4 g + e, the others 16 t + 8 + 4 g + e - 4; channel block i: ^ 64 i
  const int vr = 4 * g + (lane % 16) / 4;
  const unsigned vat = lds0 + G::HALF + (32 * share + vr) * ROW + ((2 * ((lane / 16) % 2) + (lane % 4) / 2) ^ G::swizzle(vr)) * 16 + (lane % 2) * 8;

  // Work goes to the 8 XCDs in contiguous chunks, so that the keys and values of a head are fetched into one L2.
  const unsigned chunk = (a.work + 7) / 8;
  const unsigned chunk_end = min(a.work, (blockIdx.x % 8 + 1) * chunk);
  for (unsigned work = blockIdx.x % 8 * chunk + blockIdx.x / 8; work < chunk_end; work += gridDim.x / 8) {
    const SparseTile t(a, work);
    int sub;
    const int token = t.token(a, (t.tile * (NW / SPLIT) + rows_of) * 32 + r, sub);  // this lane's query row
    BlockWalk<SK> walk;
    t.begin(a, NW / SPLIT * 32, walk);
    loads.begin(a, t);
    for (int i = 0; i < G::NS - 1; ++i) loads.issue(a, walk);

    // ---- this lane's query as column operand: pieces as the keys' fragments have them
    u32x4_t qop[KS];
    {
      const bf16* qrow = static_cast<const bf16*>(a.q) + t.b * a.qb + (int64_t)max(token, 0) * a.qn + (int64_t)(t.hk * a.group + (token < 0 ? 0 : sub)) * a.qh;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int piece = 2 * s + g;
        qop[s] = u32x4_t{0, 0, 0, 0};
        if (piece * 8 < a.d && t.q_len > 0) qop[s] = *reinterpret_cast<const u32x4_t*>(qrow + piece * 8);
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
    // a wavefront whose rows all lie past the run's end loads its share of the stages, no more
    if (__builtin_amdgcn_ballot_w64(token >= 0) == 0)
      for (int st = 0; st < loads.issued; ++st) loads.open(a, walk, st);
    else for (int st = 0; st < loads.issued; ++st) {
      const int nkeys = loads.open(a, walk, st);

      // ---- scores of two tiles of 32 keys; all fragments are on their way before the first product
      u32x4_t kf[KS][UT];
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int u = 0; u < UT; ++u) kf[s][u] = lds_read<u32x4_t>(((kat + cslot) ^ (32 * s)) + 32 * u * ROW);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (PAD) {
#pragma unroll
        for (int s = KS == 2 ? 0 : KS == 8 ? 6 : KS - 1; s < KS; ++s)
#pragma unroll
          for (int u = 0; u < UT; ++u)
            if (16 * s + 8 * g >= a.d) kf[s][u] = u32x4_t{0, 0, 0, 0};
      }
      f32x16_t sc[UT];
#pragma unroll
      for (int u = 0; u < UT; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[u][e] = 0.f;
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int u = 0; u < UT; ++u)
          sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[s][u]), __builtin_bit_cast(bf16x8_t, qop[s]), sc[u], 0, 0, 0);
      if (nkeys < SK) {
        const int lim = nkeys - 32 * share - 4 * g;  // register e of tile u is key 32 u + 8 (e / 4) + e % 4 + 4 g
#pragma unroll
        for (int u = 0; u < UT; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (32 * u + 8 * (e / 4) + e % 4 >= lim) sc[u][e] = -INFINITY;
      }
      // the values are on their way while the exponentials are taken
      uint2 vlo[2 * UT][OB], vhi[2 * UT][OB];
#pragma unroll
      for (int k16 = 0; k16 < 2 * UT; ++k16)
#pragma unroll
        for (int i = 0; i < OB; ++i) {
          vlo[k16][i] = lds_read_tr(((vat + cslot) ^ (64 * i)) + 16 * k16 * ROW);
          vhi[k16][i] = lds_read_tr(((vat + cslot) ^ (64 * i) ^ (G::swizzle(8) * 16)) + (16 * k16 + 8) * ROW);
        }
      __builtin_amdgcn_sched_barrier(0);

      // ---- probabilities against the lazy reference maximum: it is raised only when the partial sums say that an
      // exponent has grown past it, so that the steady state has no maximum and no rescaling.  exp2 of up to 2^8 is
      // harmless in float32 and, relative as bf16 rounds, in bf16.  They are rounded to bf16, the matrix cores' type for V:
      // half a step of 2^-8 of each weight, which the sums over the keys average out; the row sum is of the rounded
      // values, those that weigh V.
      u32x4_t pk[2 * UT];
      auto exponentiate = [&]() {
        float rs = 0.f;
#pragma unroll
        for (int u = 0; u < UT; ++u)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const unsigned w = pack_bf16x2(__builtin_amdgcn_exp2f(fmaf(sc[u][e], a.c, -mref)), __builtin_amdgcn_exp2f(fmaf(sc[u][e + 1], a.c, -mref)));
            pk[2 * u + e / 8][e % 8 / 2] = w;
            rs = dot2_ones(w, rs);
          }
        return rs;
      };
      float rs = exponentiate();
      if (__builtin_amdgcn_ballot_w64(!(rs <= kSparseTrigger)) != 0) {
        float mx = sc[0][0];
#pragma unroll
        for (int u = 0; u < UT; ++u)
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
#pragma unroll
      for (int k16 = 0; k16 < 2 * UT; ++k16)
#pragma unroll
        for (int i = 0; i < OB; ++i) {
          const u32x4_t vf{vlo[k16][i].x, vlo[k16][i].y, vhi[k16][i].x, vhi[k16][i].y};
          oacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vf), __builtin_bit_cast(bf16x8_t, pk[k16]), oacc[i], 0, 0, 0);
        }
      cslot = cslot == (G::NS - 1) * 2 * G::HALF ? 0 : cslot + 2 * G::HALF;
    }
    lsum += __shfl_xor(lsum, 32, kWave);
    if constexpr (SPLIT == 2) {
      // the second half's wavefront leaves its output, maximum and sum in LDS, the first adds them to its own
      constexpr int IMG = (OB * 16 + 2) * kWave;
      static_assert(NW / 2 * IMG * 4 <= G::NS * 2 * G::HALF, "the outputs fit the ring");
      float* img = reinterpret_cast<float*>(&ring[0]) + rows_of * IMG + lane;
      __syncthreads();
      if (share == 1) {
#pragma unroll
        for (int i = 0; i < OB; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) img[(16 * i + e) * kWave] = oacc[i][e];
        img[OB * 16 * kWave] = mref;
        img[(OB * 16 + 1) * kWave] = lsum;
      }
      __syncthreads();
      if (share == 0) {
        const float m2 = img[OB * 16 * kWave], top = fmaxf(mref, m2);
        const float w1 = __builtin_amdgcn_exp2f(mref - top), w2 = __builtin_amdgcn_exp2f(m2 - top);
        lsum = lsum * w1 + img[(OB * 16 + 1) * kWave] * w2;
        mref = top;
#pragma unroll
        for (int i = 0; i < OB; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[i][e] = oacc[i][e] * w1 + img[(16 * i + e) * kWave] * w2;
      }
    }
    if (token >= 0 && share == 0) {
#pragma unroll
      for (int i = 0; i < OB; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int ch = 32 * i + 8 * q + 4 * g;
          if (ch < a.d) sparse_put<bf16>(a, t, token, sub, ch, f32x4_t{oacc[i][4 * q], oacc[i][4 * q + 1], oacc[i][4 * q + 2], oacc[i][4 * q + 3]}, lsum);
        }
      if (a.nsplit > 1 && g == 0) sparse_put_ml(a, t, token, sub, mref, lsum);
    }
    __syncthreads();  // the next tile's loads overwrite the ring
  }
}

// float32 throughout, on v_mfma_f32_16x16x4_f32: a wavefront's rows are H column tiles of 16; with two of them a key or value
// operand serves two products, with one there are twice the wavefronts to hide each other's waits (runs of 64 rows, 64x64, heads
// of 40: 121 -> 118 us).  A result lane (c, g), g = lane / 16, holds column c and rows 4 g + j.  Those four keys are, register by
// register, the column operand of four steps of the second product.  16-channel tiles: heads of 40 contract 40 and produce
// 48 channels (32 x 32 tiles: 48 and 64).  Bound by the float32 matrix rate, 256 flop per clock and CU: heads of 64 and 128
// run at 123 and 124 TFLOP/s (a library product of 8192^3 at 153), heads of 40 at 103 of their own and 112 with the padded
// channels; there 31 % of the active LDS cycles are conflicts.  One token against 115200 keys, 256 blocks: 4.35 TB/s.
// D8: head channels / 8, exactly: the products of a stage are one block of instructions with its reads ahead of it.
template <int D8, int NW, int H>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 2 : 1) void sparse_attn_f32_kernel(SparseArgs a) {
  constexpr int KS = (D8 + 1) / 2, KL = KS < 2 ? 2 : KS;  // channels in steps of 16: of the output, and of a row in LDS
  using G = SparseGeo<float, KL, NW>;
  constexpr int SK = G::SK, ROW = G::ROW;
  __shared__ __align__(1024) u32x4_t ring[G::NS * 2 * G::HALF / 16];
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) void*)(&ring[0]);
  StageLoads<float, KL, NW> loads;
  loads.setup(a, lds0);
  const int lane = loads.lane, c = lane % 16, g = lane / 16;
  const unsigned kat = lds0 + c * ROW + ((g / 2) ^ G::swizzle(c)) * 16 + (g % 2) * 8;  // channels 8 s + 2 g ..: ^ 32 s
  const unsigned vat = lds0 + G::HALF + 4 * g * ROW + ((c / 4) ^ G::swizzle(4 * g)) * 16 + (c % 4) * 4;  // channel tile i: ^ 64 i

  const unsigned chunk = (a.work + 7) / 8;  // contiguous per XCD, as above
  const unsigned chunk_end = min(a.work, (blockIdx.x % 8 + 1) * chunk);
  for (unsigned work = blockIdx.x % 8 * chunk + blockIdx.x / 8; work < chunk_end; work += gridDim.x / 8) {
    const SparseTile t(a, work);
    int token[H], sub[H];
#pragma unroll
    for (int h = 0; h < H; ++h) token[h] = t.token(a, ((t.tile * NW + loads.wave) * H + h) * 16 + c, sub[h]);
    BlockWalk<SK> walk;
    t.begin(a, NW * H * 16, walk);
    loads.begin(a, t);
    for (int i = 0; i < G::NS - 1; ++i) loads.issue(a, walk);

    float2 qop[H][D8];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const float* qrow = static_cast<const float*>(a.q) + t.b * a.qb + (int64_t)max(token[h], 0) * a.qn +
                          (int64_t)(t.hk * a.group + (token[h] < 0 ? 0 : sub[h])) * a.qh + 2 * g;
#pragma unroll
      for (int s = 0; s < D8; ++s) {
        qop[h][s] = make_float2(0.f, 0.f);
        if (t.q_len > 0) qop[h][s] = *reinterpret_cast<const float2*>(qrow + 8 * s);
      }
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // the queries: nothing that the compiler tracks stays pending in the loop

    f32x4_t oacc[H][KS];
    float mref[H], lsum[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      mref[h] = kSparseLow;
      lsum[h] = 0.f;
#pragma unroll
      for (int i = 0; i < KS; ++i) oacc[h][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    unsigned cslot = 0;
    // a wavefront whose rows all lie past the run's end loads its share of the stages, no more
    if (__builtin_amdgcn_ballot_w64(max(token[0], token[H - 1]) >= 0) == 0)
      for (int st = 0; st < loads.issued; ++st) loads.open(a, walk, st);
    else for (int st = 0; st < loads.issued; ++st) {
      const int nkeys = loads.open(a, walk, st);
      f32x4_t sc[2][H];  // [key tile][column tile]
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int h = 0; h < H; ++h) sc[u][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < D8; ++s) {
        f32x2_t kf[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) kf[u] = lds_read<f32x2_t>(((kat + cslot) ^ (32 * s)) + 16 * u * ROW);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int h = 0; h < H; ++h)
              sc[u][h] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[u][j], j ? qop[h][s].y : qop[h][s].x, sc[u][h], 0, 0, 0);
      }
      if (nkeys < SK) {
        const int lim = nkeys - 4 * g;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (16 * u + j >= lim) sc[u][h][j] = -INFINITY;
      }

      // the first key tile's values are on their way while the exponentials are taken, the second's during its products
      float vf[2][4][KS];
      auto values = [&](int u) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < KS; ++i) vf[u][j][i] = lds_read<float>(((vat + cslot) ^ (G::swizzle(j) * 16) ^ (64 * i)) + (16 * u + j) * ROW);
      };
      values(0);
      __builtin_amdgcn_sched_barrier(0);

      // ---- probabilities against the lazy reference maximum, as above
      float p[2][H][4], rs[H];
      auto exponentiate = [&]() {
#pragma unroll
        for (int h = 0; h < H; ++h) {
          rs[h] = 0.f;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              p[u][h][j] = __builtin_amdgcn_exp2f(fmaf(sc[u][h][j], a.c, -mref[h]));
              rs[h] += p[u][h][j];
            }
        }
      };
      exponentiate();
      if (__builtin_amdgcn_ballot_w64(!(rs[0] <= kSparseTrigger) || !(rs[H - 1] <= kSparseTrigger)) != 0) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
          float mx = sc[0][h][0];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) mx = fmaxf(mx, sc[u][h][j]);
          mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
          mx = fmaxf(mx, __shfl_xor(mx, 32, kWave)) * a.c;  // the four parts of the row agree on the new reference
          const float up = fmaxf(mx, mref[h]), alpha = __builtin_amdgcn_exp2f(mref[h] - up);
          mref[h] = up;
          lsum[h] *= alpha;
#pragma unroll
          for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) oacc[h][i][j] *= alpha;
        }
        exponentiate();
      }
#pragma unroll
      for (int h = 0; h < H; ++h) lsum[h] += rs[h];

      // ---- O^T += V^T P^T: step (u, j) takes keys 16 u + 4 g + j
      values(1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int h = 0; h < H; ++h) oacc[h][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[u][j][i], p[u][h][j], oacc[h][i], 0, 0, 0);
      cslot = cslot == (G::NS - 1) * 2 * G::HALF ? 0 : cslot + 2 * G::HALF;
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
      lsum[h] += __shfl_xor(lsum[h], 16, kWave);
      lsum[h] += __shfl_xor(lsum[h], 32, kWave);
      if (token[h] >= 0) {
#pragma unroll
        for (int i = 0; i < KS; ++i)
          if (16 * i + 4 * g < a.d) sparse_put<float>(a, t, token[h], sub[h], 16 * i + 4 * g, oacc[h][i], lsum[h]);
        if (a.nsplit > 1 && g == 0) sparse_put_ml(a, t, token[h], sub[h], mref[h], lsum[h]);
      }
    }
    __syncthreads();
  }
}

// The shares of a query row joined: weights 2^(m - max m).  A wavefront per row: its lanes hold one share's maximum and sum
// each (nsplit <= 64), then 64 / (d / 4) shares' outputs at a time, four channels per lane; the order of the sums is fixed.
template <typename T>
__global__ __launch_bounds__(256) void sparse_join_kernel(SparseArgs a, int rows) {
  const int lane = threadIdx.x % kWave, heads = a.heads_kv * a.group, quads = a.d / 4;
  // lanes of one share: the next power of two of quads
  const int width = quads <= 2 ? 2 : quads <= 4 ? 4 : quads <= 8 ? 8 : quads <= 16 ? 16 : 32, at_once = kWave / width;
  const int quad = lane % width, which = lane / width;
  const int row = (int)blockIdx.x * 4 + threadIdx.x / kWave;
  if (row >= rows) return;
  const int bn = row / heads;
  const int h = row - bn * heads, b = bn / a.Nq, token = bn - b * a.Nq;
  if (a.q_len && token >= a.q_len[b]) return;
  const float2 ml = lane < a.nsplit ? a.part_ml[(int64_t)row * a.nsplit + lane] : make_float2(kSparseLow, 0.f);
  const float w = __builtin_amdgcn_exp2f(ml.x - wave_max(ml.x));
  const float l = wave_sum(ml.y * w);
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
  if (which != 0 || quad >= quads) return;
  const float inv = 1.f / l;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = l == 0.f ? 0.f : o[j] * inv;
  T* dst = static_cast<T*>(a.o) + b * a.ob + (int64_t)token * a.on + (int64_t)h * a.oh + 4 * quad;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
  else *reinterpret_cast<f32x4_t*>(dst) = o;
}

}  // namespace si

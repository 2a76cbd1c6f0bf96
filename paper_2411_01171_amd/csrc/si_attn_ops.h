// Operators on heads of video tokens, as the spatial block's path calls them, and checks of heads (defined in si_attn_ops.hip).
#pragma once
#include "../../include/si.h"

#include <hip/hip_runtime.h>

namespace si {

constexpr int64_t kMostTokens = INT32_MAX - (1 << 22);  // of a sequence: kernels add tiles to token numbers in 31 bits
constexpr int64_t kGridMost = 1 << 20;                  // workgroups of a launch; kernels walk longer lists
constexpr int64_t kSelectMaxBlocks = 16384;  // one run's scores fill the LDS of a workgroup

struct BlocksPlan {
  int64_t runs, blocks, words;
  int group;
};

struct SparsePlan {
  int tile_rows, nsplit;
  int64_t tiles_per_run, tiles, work;
  int64_t rows;  // of all queries and heads
  size_t part_bytes;
};

// Elements from the first to behind the last one, over the dimensions whose stride is below `below`.
int64_t heads_extent(const si_heads* t, int64_t below = INT64_MAX);
// Sizes, strides and alignment of one operand.  `written`: its elements must have addresses of their own.
si_status check_heads(const si_heads* t, bool written);
// Whether no element of one lies on an element of the other.
bool heads_apart(const si_heads* a, const si_heads* b);
bool heads_overlap_range(const si_heads* t, const void* p, size_t bytes);

si_status check_rope(const si_rope* r, int d);
bool rope_gain_in(const si_rope* r, int d, int esize, const void* p, size_t bytes);
si_status plan_blocks(const si_heads* q, const si_heads* k, int64_t q_block, int64_t k_block, BlocksPlan* p);
si_status plan_sparse(const si_heads* q, const si_heads* k, int64_t q_block, const BlocksPlan& b, bool may_split, SparsePlan* p);
size_t select_bytes(const si_heads* q, const si_heads* k, const BlocksPlan& p);

// The operands of these have been checked.  k and ko may be NULL.
si_status enqueue_rope(const si_heads* q, const si_heads* k, const si_rope* r, int64_t first, const si_heads* qo, const si_heads* ko,
                       hipStream_t st);
si_status enqueue_select(const si_heads* q, const si_heads* k, const BlocksPlan& p, int64_t q_block, int64_t k_block, int64_t keep,
                         const int32_t* q_len, const int32_t* k_len, uint32_t* blocks, char* ws, hipStream_t st);
// o_frag: 0, or out is a fragment-order operand buffer of that many channels per token (bf16)
si_status enqueue_sparse(const si_heads* q, const si_heads* k, const si_heads* v, const BlocksPlan& b, const SparsePlan& p, int64_t q_block,
                         int64_t k_block, float scale, const int32_t* q_len, const int32_t* k_len, const uint32_t* blocks,
                         const si_heads* out, char* ws, hipStream_t st, int o_frag);

}  // namespace si

// Argument blocks and launchers of the kernels around a model's attention:
// per-head norms with the position rotation, and attention of query blocks with
// windows and drafted trees.
//
// The launchers are weak: the API's host side also builds without CUDA kernels,
// over a stand-in of the runtime, and need not name them all there.  A call
// whose kernels are not linked in is refused (SQ_ERR_UNSUPPORTED).
#pragma once

#include "launch.hpp"

#define SQ_OPTIONAL __attribute__((weak))

namespace sq {

// ---- norms of queries and keys, position rotation ------------------------------
// Where a token's K/V row goes (page * page_size + slot) and its position.
struct RowPlace {
    int32_t row, pos;
};
// Tokens whose places go with the launch; more are uploaded.
constexpr int kNormInline = 240;

struct NormRopeArgs {
    const __nv_bfloat16 *q, *k, *v;          // rows of a token: [heads][D], contiguous
    int64_t q_stride, k_stride, v_stride;    // elements between tokens
    const int32_t* positions;                // [n] or null: RowPlace::pos
    const RowPlace* places;                  // [n] or null: inline_place
    __nv_bfloat16 *q_out, *k_out;            // [n][heads][D]; k_out null: into the pool
    __nv_bfloat16* pool;
    const void *q_weight, *k_weight;         // [D] or null (ones)
    const float2* rope;                      // [max_pos][rot / 2] (cos, sin)
    int64_t num_pages;
    int32_t n, Hq, Hkv, P, layer;
    int32_t rot, interleaved, max_pos, weight_f32;
    float eps;
    int* err;
};
struct NormRopeInlineArgs : NormRopeArgs {
    RowPlace inline_place[kNormInline];
};

struct NormRopeGradArgs {
    const __nv_bfloat16 *q, *k;
    int64_t q_stride, k_stride;
    const int32_t* positions;
    const __nv_bfloat16 *dq_out, *dk_out;    // [n][heads][D], of the rotated outputs
    __nv_bfloat16 *dq, *dk;                  // [n][heads][D], of the inputs
    int64_t dq_stride, dk_stride;
    float *dq_weight, *dk_weight;            // [D] or null
    const void *q_weight, *k_weight;
    const float2* rope;
    float* part;                             // [ctas][2][D] partial weight gradients
    int32_t n, Hq, Hkv, rot, interleaved, max_pos, weight_f32;
    int32_t ctas;
    float eps;
    int* err;
};

SQ_OPTIONAL cudaError_t launch_norm_rope(const NormRopeArgs& a, int D, bool store, cudaStream_t st);
SQ_OPTIONAL cudaError_t launch_norm_rope_inline(const NormRopeInlineArgs& a, int D, cudaStream_t st);
// CTAs of the backward kernel for n tokens of a geometry on a device of num_sms.
SQ_OPTIONAL int norm_rope_grad_ctas(int32_t n, int32_t Hq, int32_t Hkv, int D, int num_sms);
SQ_OPTIONAL cudaError_t launch_norm_rope_grad(const NormRopeGradArgs& a, int D, cudaStream_t st);

// ---- attention of query blocks ---------------------------------------------------
// The prefill kernel's arguments, of which items and tiles are the blocks' own;
// n, n_q and n_tiles are the items'.
struct BlockArgs : PrefillArgs {
    const int2* rows;       // [queries] first and last slot of each one's window, or
                            // null: low0 + i and pos0 + i of the item
    const uint32_t* bits;   // [queries][n_words] drafted trees' visibility from the
                            // item's base on
    int32_t n_words;
    // as the tensor maps have them (rows that are taken once more read them plainly)
    const void* pool;       // bf16 [layers][num_pages][2][Hkv][P][D]
    const void* q;          // bf16 [queries][Hq][D]
    int32_t n_ctas;         // CTAs launched (one-tile blocks are dealt out to them;
                            // otherwise one for each item)
};
// Calls whose items' queries all fit in one query tile.
struct BlockShortArgs : BlockArgs {
    int32_t kv_early;       // as DecodeArgs::kv_early
    int32_t n_unsafe;
    int32_t unsafe[kMaxUnsafe];
};
// The same with two producer warps (instances of their own).
struct BlockArgs2 : BlockArgs {};
struct BlockShortArgs2 : BlockShortArgs {};
struct BlockCombineArgs {
    const BlockMerge* merges;
    int32_t n_merges;
    const float* part_o;
    const float* part_ml;
    void* out;
    int32_t out_f32;
    float* lse;
    int32_t Hq, G, BP;
    int32_t max_splits;
    int32_t rows;           // rows of a unit that can hold queries
};
SQ_OPTIONAL cudaError_t blocks_prepare(int D);
// one: every item's queries fit in one query tile
SQ_OPTIONAL cudaError_t launch_blocks(const CUtensorMap& pool_map, const CUtensorMap& qmap,
                                      const BlockShortArgs& a, int D, bool one, cudaStream_t st);
SQ_OPTIONAL cudaError_t launch_blocks_combine(const BlockCombineArgs& a, int D, cudaStream_t st);

}  // namespace sq

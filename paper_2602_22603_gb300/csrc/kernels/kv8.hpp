// Rows held in 8 bits: their layout, and the argument blocks and launchers of the
// kernels on them (weak, as operators.hpp has them).
#pragma once

#include "operators.hpp"

namespace sq {

// The pool of an 8-bit cache: e4m3 codes [L][num_pages][2 (K, V)][Hkv][P][D], then
// fp32 scales [L][num_pages][2][Hkv][P / kScaleRows].  A row's value is its code
// times the scale of its block, kScaleRows slots of one page, plane and head.  A
// scale is the least power of two, from 2^kLeastScale on, with which the largest
// finite element of the block's rows (new ones before they are rounded, others as
// they are held) is at most 448: codes of any scale then share
// one grid but for the smallest (below 2^-6), so that taking a row to another scale
// changes nothing but what falls below that.
constexpr int kScaleRows = 8;
constexpr int kLeastScale = -100;
constexpr int kMostScale = 120;  // of elements up to 2^128

// Rows in consecutive slots of one page, none over a border of kRunRows (row: page * P +
// slot of the first), the call's from `first` on; pos: the first one's position.
struct RowRun {
    int32_t row, first, n, pos;
};
constexpr int kRunRows = 64;
// Runs that go with the launch; more are uploaded.
constexpr int kRunsInline = 236;

struct Kv8Pool {
    uint8_t* codes;
    float* scales;
    int64_t num_pages;
    int32_t Hkv, P;
};
struct Kv8StoreArgs {
    const __nv_bfloat16 *q, *k, *v;          // rows of a token: [heads][D], contiguous
    int64_t q_stride, k_stride, v_stride;    // elements between tokens
    int64_t layer_stride;                    // ... between layers (k and v)
    const int32_t* positions;                // [n] or null: the runs'
    const RowRun* runs;                      // or null: inline_run
    __nv_bfloat16* q_out;                    // [n][Hq][D]
    Kv8Pool pool;
    const void *q_weight, *k_weight;         // [D] or null (ones)
    const float2* rope;                      // [max_pos][rot / 2] (cos, sin)
    int32_t n_runs, blocks, most;            // most blocks of any run, most rows in any block
    int32_t Hq, Hkv, layer, n_layers;        // Hq 0: no queries
    int32_t plain;                           // 1: keys as they are, like values
    int32_t rot, interleaved, max_pos, weight_f32;
    float eps;
    int* err;
};
struct Kv8StoreInlineArgs : Kv8StoreArgs {
    RowRun inline_run[kRunsInline];
};
static_assert(sizeof(Kv8StoreInlineArgs) <= 4096, "launch arguments");

// Copies of pages' first rows, and words of decode plans (see AppendBatchArgs).
struct Kv8CopyArgs {
    Kv8Pool pool;
    int32_t L;
    AppendLens lens;
    int32_t n_cow;
    CowCopy cow[kAppendBatchMax];
    int* err;
};
// Rows as bf16, [n][Hkv][D].
struct Kv8ReadArgs {
    Kv8Pool pool;
    const __nv_bfloat16* wide;  // the pool where rows are bf16 (codes null)
    const RowRun* runs;         // or null: inline_run
    __nv_bfloat16 *k, *v;
    int32_t n_runs, most, layer;
    int* err;
};
struct Kv8ReadInlineArgs : Kv8ReadArgs {
    RowRun inline_run[kRunsInline];
};
// Pages of one layer as bf16, out [n][2][Hkv][P][D].
struct Kv8WidenArgs {
    Kv8Pool pool;
    const int32_t* pages;
    int32_t n, layer;
    __nv_bfloat16* out;
    int* err;
};
// As EvictArgs; a page's moved rows are one tile.
struct Kv8EvictArgs {
    Kv8Pool pool;
    int32_t L;
    const EvictTile* tiles;
    const EvictPiece* pieces;
    const int32_t* chunk;       // [n_chunks + 1]
    int32_t n_chunks, n_tiles, n_pieces;
    int* err;
};

// Single tokens over such rows (tmap: the codes', 5-D: head dim, slot, KV head, K or V,
// page of a layer; a box has min(P, kStageTokens) rows of both).
struct DecodeKv8Args : DecodeArgs {
    const float* scales;
};
SQ_OPTIONAL cudaError_t launch_decode_kv8(const CUtensorMap& tmap, const DecodeKv8Args& a, int n_ctas, int D,
                                          cudaStream_t st);

// Query blocks of one tile over such rows, as BlockShortArgs and BlockShortArgs2.
struct BlockShortKv8Args : BlockShortArgs {
    const float* scales;
};
struct BlockShortKv8Args2 : BlockShortKv8Args {};
SQ_OPTIONAL cudaError_t blocks_kv8_prepare(int D);
SQ_OPTIONAL cudaError_t launch_blocks_kv8(const CUtensorMap& pool_map, const CUtensorMap& qmap,
                                          const BlockShortKv8Args& a, int D, cudaStream_t st);

SQ_OPTIONAL cudaError_t kv8_prepare(int D);
SQ_OPTIONAL cudaError_t launch_kv8_store(const Kv8StoreInlineArgs& a, int D, cudaStream_t st);
SQ_OPTIONAL cudaError_t launch_kv8_copy(const Kv8CopyArgs& a, int D, cudaStream_t st);
SQ_OPTIONAL cudaError_t launch_kv8_read(const Kv8ReadInlineArgs& a, int D, cudaStream_t st);
SQ_OPTIONAL cudaError_t launch_kv8_widen(const Kv8WidenArgs& a, int D, cudaStream_t st);
SQ_OPTIONAL cudaError_t launch_kv8_evict(const Kv8EvictArgs& a, int D, cudaStream_t st);

}  // namespace sq

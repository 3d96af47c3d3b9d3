// Shared declarations of the 8-bit cache's operators and of the attention over shared prefixes.
#pragma once

#include "common.h"

namespace specv {

// What the pages of a cache hold.
enum CacheKind : int {
    kCacheTiles = 0,    // bf16, SPEC_KV_MFMA
    kCacheTokens = 1,   // bf16, SPEC_KV_TOKEN_MAJOR
    kCacheE4M3 = 2,
    kCacheInt8 = 3,
};
constexpr bool is_8bit(int kind) { return kind >= kCacheE4M3; }

constexpr float kMaxE4M3 = 448.0f, kMaxInt8 = 127.0f;
constexpr float kSmallestRow = 8.673617379884035e-19f;   // 2^-60: see spec_kv8_append
constexpr float kSmallestScale = kSmallestRow / 512.0f;  // below every scale that an append writes

struct Kv8AppendParams {
    int32_t B, Hkv, d, max_blocks_per_req, num_blocks, T, src_f32, int8;
    int64_t token_stride;
    const void *new_k, *new_v;
    unsigned char *k_cache, *v_cache;
    float *kv_scale;
    const int32_t *block_table, *kv_len, *cu_q_len;
    unsigned long long *errors;
};
hipError_t launch_kv8_append(const Kv8AppendParams &p, hipStream_t stream);

struct Kv8ReadParams {
    int32_t B, Hkv, d, max_blocks_per_req, num_blocks, T, out_f32, int8;
    const unsigned char *k_cache, *v_cache;
    const float *kv_scale;
    const int32_t *block_table, *start, *cu_len;
    void *out_k, *out_v;
    unsigned long long *errors;
};
hipError_t launch_kv8_read(const Kv8ReadParams &p, hipStream_t stream);

// Attention over a paged cache in one launch or two.
//   prefix   one block per (row block of a group, KV head, chunk of the group's prefix): partial results of all the group's
//            query rows, which see the whole prefix.  Groups with more than 48 rows have a kernel of their own (many rows).
//   own      one block per (request, row block, KV head, chunk of the tokens after the prefix, or of all tokens where there is no
//            prefix launch), causal inside the draft.  A request whose tokens are one chunk takes its prefix partials in and
//            writes the output; otherwise the last of its blocks to finish joins its partials first (tickets).
// Partial results of query row r (token row * Hq + head), chunk (or piece) c:
//   acc [r][max chunks][d]  sum_t 2^(x_t - m) V_t, un-normalised    ml [r][max chunks][2]  m and sum_t 2^(x_t - m)
// in fp32.
constexpr int kMaxChunkTokens = 4096;   // the block-table entries of a block's four wavefronts: 64 pages each

constexpr int kPrefixRows = 32;         // many rows: rows of a wavefront; a block has 4 of them, or 8
constexpr int kStepPages = 4;           // ... pages of a step
constexpr int kMaxPrefixSteps = 64;     // ... most steps of a block
constexpr int kMaxPrefixBlocks = 1 << 24;   // ... most blocks of a launch

struct CacheAttnParams {
    int32_t B, Hq, Hkv, group, num_blocks, max_blocks_per_req, T, G;
    int32_t kind, d, out_f32;
    int32_t row_tiles, row_blocks;              // own: 16-row tiles of a block, blocks that cover a request's rows
    int32_t chunk_tokens, max_chunks;           // own tokens
    int32_t whole_context;                      // own: of the prefix too, which no other launch takes then
    int32_t capacity_tokens;                    // longest kv_len planned for
    int32_t prefix_tiles, prefix_row_blocks;    // prefix: 16-row tiles of a block, blocks over all groups
    int32_t prefix_chunk_tokens, max_prefix_chunks;   // 0: no group has a prefix
    int32_t prefix_many_rows, prefix_piece_steps;   // the launch for many rows: steps of a block, prefix_row_blocks blocks
    int32_t prefix_rows_log2;                   // ... log2 of a block's rows
    int32_t prefix_capacity;                    // longest prefix planned for
    int32_t max_q_rows;                         // rows of the largest request
    uint32_t generation;
    uint32_t group_inverse;                     // 2^32 / group, rounded up
    float scale_log2;
    int64_t q_stride;                           // elements per token
    const void *q, *k_cache, *v_cache;
    const float *kv_scale;
    const int32_t *block_table, *kv_len, *cu_q_len, *cu_group, *prefix_len;
    void *out;
    float *acc, *ml;                            // own partials
    float *prefix_acc, *prefix_ml;
    unsigned long long *tickets;                // [B][Hkv][row_blocks]
    unsigned long long *errors;
};
hipError_t launch_cache_attn(const CacheAttnParams &p, hipStream_t stream);

// The tuning switch SPEC_VERIFY_PREFIX_SHARED: 0 / 1, or -1: the planner's choice.
int prefix_shared_switch();

}  // namespace specv

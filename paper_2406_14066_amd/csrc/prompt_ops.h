// Shared declarations of the operators around prompts and bounded caches.
#pragma once

#include "cache_ops.h"

namespace specv {

// r / group for r < 2^28 and group <= 16: a product with a rounded-up reciprocal.
inline uint32_t inverse_of_group(int group) { return (uint32_t)((((uint64_t)1 << 32) + group - 1) / group); }   // (unused where the group is 1)
constexpr int64_t kMaxHeadRows = (int64_t)1 << 28;   // query rows of a KV head
__device__ __forceinline__ int divide_by_group(int r, int group, uint32_t inverse) { return group == 1 ? r : (int)__umulhi((uint32_t)r, inverse); }

struct QkNormRopeParams {
    int32_t T, Hq, Hkv, d, f32, weight_f32, rot_dim, interleaved;
    int32_t passes, per_wave;   // passes over a token's heads, passes of a wavefront
    float eps, scale;
    int64_t q_stride, k_stride, out_q_stride, out_k_stride;
    const void *q, *k, *q_weight, *k_weight;
    void *out_q, *out_k;
    const int32_t *positions;
    const float *inv_freq;
};
hipError_t launch_qk_norm_rope(const QkNormRopeParams &p, hipStream_t stream);

constexpr int kMostPromptChunks = 64;   // of a row's tokens

// Prompt attention.  The query rows of a request and KV head are counted token by token, the group's heads side by side: row r is head
// r % group of token r / group.  A block takes 2^rows_log2 of them through a chunk of the tokens they see.  Request b owns the
// items row_item(cu[b], b) .. row_item(cu[b + 1], b + 1) - 1 of the grid, which are enough for its row blocks; those left over have no work.
struct PromptAttnParams {
    int32_t B, Hq, Hkv, group, num_blocks, max_blocks_per_req, T, kind;
    int32_t d, out_f32, rows_log2, items, chunk_tokens, max_chunks, even, capacity_tokens;
    uint32_t group_inverse;
    float scale_log2;
    int32_t reserved;
    int64_t q_stride;
    const void *q, *k_cache, *v_cache;
    const float *kv_scale;
    const int32_t *block_table, *kv_len, *cu_q_len;
    void *out;
    float *lse;
    float *acc, *ml;      // partial results [T * Hq][max_chunks][d], [..][2]
    unsigned long long *errors;
};
// Whether a request's rows, by offsets from device memory, are among the T packed ones, or there are none.
__device__ __forceinline__ bool offsets_fit(int begin, int end, int T) { return begin == end || (begin >= 0 && end > begin && end <= T); }
__host__ __device__ inline int row_item(int packed, int b, int group, int rows_log2) { return (int)(((int64_t)packed * group) >> rows_log2) + b; }
hipError_t launch_prompt_attn(const PromptAttnParams &p, hipStream_t stream);

constexpr int kWeightTokens = 32;   // tokens of a wavefront (or block) of the weight kernel
enum : int32_t {
    kWeightOwn = 0,      // a block's wavefronts have tokens of their own and go through the same rows
    kWeightShared = 1,   // ... have the same tokens and share the rows
    kWeightFew = 2,      // at most kWeightFewRows rows: they stay in LDS, and the wavefronts go through many tokens
    kWeightSome = 3,     // ... kWeightSomeRows
};
constexpr int kWeightFewRows = 64, kWeightSomeRows = 256;
struct KvWeightParams {
    int32_t B, Hq, Hkv, group, num_blocks, max_blocks_per_req, T, kind;
    int32_t d, max_tiles, capacity_tokens;
    int32_t form;           // one of kWeight*
    int32_t groups;         // kWeightFew, kWeightSome: times 32 tokens that a wavefront takes one after another
    uint32_t group_inverse;
    float scale_log2;
    int32_t reserved;
    int64_t q_stride;
    const void *q, *k_cache;
    const float *lse, *kv_scale, *weight_in;
    float *weight;
    const int32_t *block_table, *kv_len, *cu_q_len;
    unsigned long long *errors;
};
hipError_t launch_kv_weight(const KvWeightParams &p, hipStream_t stream);

constexpr int kEvictTurn = 4096;   // tokens of which the choice's threads hold four each
struct KvEvictParams {
    int32_t B, Hkv, d, num_blocks, max_blocks_per_req, dst_max_blocks;
    int32_t kv_dtype, kv_layout, first, recent, capacity_tokens, score_stride;
    int32_t held;           // times 4 tokens of a thread of the choice: 1, 4 or 8 (the last for any length)
    int32_t reserved;
    void *k_cache, *v_cache;
    float *kv_scale, *weight;
    const int32_t *block_table, *kv_len, *keep, *dst_block_table;
    int32_t *new_kv_len, *kept;
    uint32_t *score;        // workspace: [B][score_stride] ordered bits of the scores
    int32_t *chosen;        // workspace: [B][16 * dst_max_blocks] where the kept tokens lie: page * 16 + slot, -1 outside the pool
    unsigned long long *errors;
};
hipError_t launch_kv_evict(const KvEvictParams &p, hipStream_t stream);

}  // namespace specv

// C entry points of the operators around prompts and bounded caches: argument checks, launch plans.
#include "api_util.h"
#include "prompt_ops.h"

#include <math.h>
#include <string.h>

#include <algorithm>

namespace specv {

namespace {

constexpr int kMostGrid = 65535, kMostKvHeads = 65535;
constexpr int64_t kMostThreads = (int64_t)1 << 32;   // of a launch, fewer
constexpr int64_t kMostSplitRows = (int64_t)1 << 22;   // (token, head) rows whose tokens may be split: the partial results of two chunks are 4 GB

// Whether two arrays of so many bytes share some.
bool overlap(const void *a, const void *b, size_t bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return (x < y ? y - x : x - y) < bytes;
}

bool float_or_bf16(int32_t dtype) { return dtype == SPEC_F32 || dtype == SPEC_BF16; }

spec_status check_rope(const spec_qk_norm_rope_args *a)
{
    if (a == nullptr || a->T < 0 || a->Hq < 0 || a->Hkv < 0 || (a->Hq == 0 && a->Hkv == 0) || a->d < 1) return SPEC_EINVAL;
    if (!float_or_bf16(a->dtype) || !float_or_bf16(a->weight_dtype)) return SPEC_EINVAL;
    if (a->rot_dim < 0 || a->rot_dim > a->d || a->interleaved < 0 || a->interleaved > 1) return SPEC_EINVAL;
    if (!(a->eps >= 0.0f) || isinf(a->eps) || isnan(a->scale) || isinf(a->scale)) return SPEC_EINVAL;
    if (a->T > 0) {
        if ((a->Hq > 0 && (a->q == nullptr || a->out_q == nullptr)) || (a->Hkv > 0 && (a->k == nullptr || a->out_k == nullptr))) return SPEC_EINVAL;
        if (a->rot_dim > 0 && (a->positions == nullptr || a->inv_freq == nullptr)) return SPEC_EINVAL;
    }
    for (const void *ptr : {a->q, a->k, (const void *)a->out_q, (const void *)a->out_k, a->q_weight, a->k_weight})
        if (!aligned(ptr, 16)) return SPEC_EINVAL;
    const int64_t per = a->dtype == SPEC_F32 ? 4 : 8;   // elements of 16 bytes
    const int64_t stride[4] = {a->q_stride, a->out_q_stride, a->k_stride, a->out_k_stride};
    for (int i = 0; i < 4; ++i)
        if (stride[i] != 0 && (stride[i] < (int64_t)(i < 2 ? a->Hq : a->Hkv) * a->d || stride[i] % per != 0)) return SPEC_EINVAL;
    if (a->T > 1) {   // rows that lie on their outputs lie on their own
        const int64_t q_row = (int64_t)a->Hq * a->d, k_row = (int64_t)a->Hkv * a->d;
        auto moved = [](const void *from, const void *to, int64_t x, int64_t y, int64_t row) { return from != nullptr && from == to && (x != 0 ? x : row) != (y != 0 ? y : row); };
        if (moved(a->q, a->out_q, a->q_stride, a->out_q_stride, q_row) || moved(a->k, a->out_k, a->k_stride, a->out_k_stride, k_row)) return SPEC_EINVAL;
    }
    if (a->d != 64 && a->d != 128) return SPEC_EUNSUPPORTED;
    if (a->rot_dim % 16 != 0) return SPEC_EUNSUPPORTED;
    if ((int64_t)a->T * ((int64_t)a->Hq + a->Hkv) > kMaxPacked || a->T > 1 << 25) return SPEC_EUNSUPPORTED;
    if (((int64_t)a->Hq + a->Hkv) * a->d >= (int64_t)1 << 31) return SPEC_EUNSUPPORTED;   // (a head's place in its token)
    return SPEC_OK;
}

// The longest request that the launch allows for.
int capacity_of(int B, int max_kv_len, const int32_t *host_kv_len, const int32_t *host_cu_q_len)
{
    if (max_kv_len > 0) return max_kv_len;
    int most = 0;
    for (int b = 0; b < B; ++b)
        if (host_cu_q_len == nullptr || host_cu_q_len[b + 1] > host_cu_q_len[b]) most = std::max(most, host_kv_len[b]);
    return most;
}

// What the attention and the weights have in common: query rows over paged K.
spec_status check_rows(int32_t B, int32_t Hq, int32_t Hkv, int32_t d, int32_t num_blocks, int32_t max_blocks_per_req, int32_t T, int32_t kv_dtype, int32_t kv_layout,
                       int32_t max_kv_len, int64_t q_token_stride, const void *q, const void *k_cache, const float *kv_scale, const int32_t *block_table,
                       const int32_t *kv_len, const int32_t *cu_q_len, const int32_t *host_kv_len, const int32_t *host_cu_q_len, float softmax_scale)
{
    if (B < 1 || Hq < 1 || Hkv < 1 || num_blocks < 1 || max_blocks_per_req < 1 || T < 0) return SPEC_EINVAL;
    if (k_cache == nullptr || block_table == nullptr || kv_len == nullptr || cu_q_len == nullptr || host_cu_q_len == nullptr) return SPEC_EINVAL;
    if (T > 0 && q == nullptr) return SPEC_EINVAL;
    if (kv_dtype != SPEC_BF16 && kv_dtype != SPEC_E4M3 && kv_dtype != SPEC_INT8) return SPEC_EINVAL;
    const bool b8 = kv_dtype != SPEC_BF16;
    if ((kv_scale != nullptr) != b8) return SPEC_EINVAL;
    if (kv_layout != SPEC_KV_MFMA && (b8 || kv_layout != SPEC_KV_TOKEN_MAJOR)) return SPEC_EINVAL;
    if (!aligned(k_cache, 32) || !aligned(kv_scale, 32) || !aligned(q, 16)) return SPEC_EINVAL;
    if (max_kv_len < 0 || (max_kv_len == 0 && host_kv_len == nullptr) || pages_of(max_kv_len) > max_blocks_per_req) return SPEC_EINVAL;
    if (Hq % Hkv != 0) return SPEC_EINVAL;
    if (!(softmax_scale >= 0.0f) || isinf(softmax_scale)) return SPEC_EINVAL;
    if (q_token_stride != 0 && (q_token_stride < (int64_t)Hq * d || q_token_stride % 8 != 0)) return SPEC_EINVAL;
    if (!prefix_sum_ok(host_cu_q_len, B, T)) return SPEC_EINVAL;
    for (int b = 0; b < B; ++b) {
        if (host_kv_len == nullptr || host_cu_q_len[b + 1] == host_cu_q_len[b]) continue;
        const int len = host_kv_len[b];
        if (len < 0 || pages_of(len) > max_blocks_per_req || (max_kv_len > 0 && len > max_kv_len)) return SPEC_EINVAL;
    }
    if (d != 64 && d != 128) return SPEC_EUNSUPPORTED;
    if (capacity_of(B, max_kv_len, host_kv_len, host_cu_q_len) > kMaxPacked) return SPEC_EUNSUPPORTED;   // (places of tokens, rounded up to steps and groups of them)
    if (Hq / Hkv > 16 || Hkv > kMostKvHeads || B > kMostGrid) return SPEC_EUNSUPPORTED;
    if ((int64_t)T * Hq > kMaxPacked || (int64_t)T * (Hq / Hkv) >= kMaxHeadRows) return SPEC_EUNSUPPORTED;   // (of T: whatever the offsets in device memory say)
    return SPEC_OK;
}

int kind_of(int32_t kv_dtype, int32_t kv_layout)
{
    return kv_dtype == SPEC_E4M3 ? kCacheE4M3 : kv_dtype == SPEC_INT8 ? kCacheInt8 : kv_layout == SPEC_KV_MFMA ? kCacheTiles : kCacheTokens;
}

float scale_log2_of(float softmax_scale, int d) { return (float)((softmax_scale > 0.0f ? (double)softmax_scale : 1.0 / sqrt((double)d)) * kLog2eD); }

spec_status check_prompt(const spec_prompt_attn_args *a)
{
    if (a == nullptr) return SPEC_EINVAL;
    const spec_status st = check_rows(a->B, a->Hq, a->Hkv, a->d, a->num_blocks, a->max_blocks_per_req, a->T, a->kv_dtype, a->kv_layout, a->max_kv_len,
                                      a->q_token_stride, a->q, a->k_cache, a->kv_scale, a->block_table, a->kv_len, a->cu_q_len, a->host_kv_len,
                                      a->host_cu_q_len, a->softmax_scale);
    if (st == SPEC_EINVAL) return st;
    if (a->v_cache == nullptr || (a->T > 0 && a->out == nullptr) || !float_or_bf16(a->out_dtype)) return SPEC_EINVAL;
    if (!aligned(a->v_cache, 32) || !aligned(a->out, 32) || !aligned(a->lse, 4)) return SPEC_EINVAL;
    return st;
}

// The launch of the attention, from a model of it in steps of 64 tokens, kStepUs or (256 rows) kWideStepUs each.  A block takes kBlockSteps' worth besides its
// steps.  Two blocks of four wavefronts fit a compute unit and slow each other down by kTogether; blocks beyond the ones that the device holds end at
// different times, which costs half of the longest one.  Each chunk of a row's tokens is a partial result to write and to read back; the
// join is a launch and looks at the chunks in turn.  Measured, us, by chunks of the longest request (planned: *): one token behind 32000, 64/8
// heads: 8 86, 16 52, 32 38 *, 64 45; 8 requests of 1 .. 9 rows behind 2000 .. 30000: 4 131, 8 104 *, 12 101, 24 109; 512 rows behind 8000: 1 206, 2 140 *, 3 167;
// a prompt of 4000 tokens: 1 130 *, 2 156, 4 189.  (With a join that took 4 us more for 32 chunks: the first is 34 now.)
struct PromptPlan {
    int rows_log2, items, chunk_tokens, max_chunks, even, capacity;
    size_t acc, ml, total;   // offsets into the workspace
};
constexpr int kStep = 64;
constexpr double kStepUs = 1.35, kWideStepUs = 1.7, kBlockSteps = 3.0, kTogether = 1.4, kJoinBytesPerUs = 4e6, kJoinUs = 4.0, kJoinChunkUs = 0.15;

PromptPlan plan_prompt(const spec_prompt_attn_args *a, bool whole)
{
    PromptPlan pl;
    memset(&pl, 0, sizeof pl);
    const int group = a->Hq / a->Hkv;
    whole = whole || (int64_t)a->T * a->Hq > kMostSplitRows;
    pl.capacity = capacity_of(a->B, a->max_kv_len, a->host_kv_len, a->host_cu_q_len);
    auto each_request = [&](auto request) {   // (query rows of a KV head, tokens, rows in tokens)
        for (int b = 0; b < a->B; ++b) {
            const int n = a->host_cu_q_len[b + 1] - a->host_cu_q_len[b];
            if (n > 0) request((int64_t)n * group, a->max_kv_len > 0 ? a->max_kv_len : a->host_kv_len[b], n);
        }
    };
    const int most_steps = std::max((pl.capacity + kStep - 1) / kStep, 1);
    // Blocks of eight wavefronts and 256 rows, or of four and 128: the first bring pages in half as often, which is the faster the more blocks
    // there are (a prompt of 4000 tokens, 32/8 heads: 130 against 149 us), unless they walk many more absent rows; the second are done earlier where
    // there is less than one for each compute unit (1000 tokens: 31 against 27).
    double padded[2] = {0.0, 0.0};
    each_request([&](int64_t rows, int tokens, int) {
        for (int wide = 0; wide < 2; ++wide) padded[wide] += (double)((rows + (128 << wide) - 1) >> (7 + wide) << (7 + wide)) * tokens;
    });
    const double units = compute_units();
    int best = most_steps;
    double best_cost = 1e300;
    pl.rows_log2 = 7;
    pl.even = 1;
    for (int wide = 0; wide <= (a->d == 128 && padded[1] <= 1.1 * padded[0] ? 1 : 0); ++wide) {
        const double slots = units * (wide ? 1.0 : 2.0), together = wide ? 1.0 : kTogether;
        for (int chunks = 1, last = 0; chunks <= (whole ? 1 : kMostPromptChunks); chunks = std::max(chunks + 1, chunks * 5 / 4)) {
            const int length = (most_steps + chunks - 1) / chunks;
            if (length == last) continue;
            last = length;
            double sum = 0.0, count = 0.0, longest = 0.0, bytes = 0.0;
            each_request([&](int64_t rows, int tokens, int n) {
                const int64_t blocks = ((rows + (128 << wide) - 1) >> (7 + wide)) * a->Hkv;
                const double steps = std::max(tokens - 0.5 * n, 1.0) / kStep, pieces = ceil(steps / length);
                sum += blocks * (steps + pieces * kBlockSteps);
                count += blocks * pieces;
                longest = std::max(longest, std::min((double)length, ceil((double)tokens / kStep)) + kBlockSteps);
                if (tokens > length * kStep) bytes += (double)rows * a->Hkv * pieces * a->d * 8.0;
            });
            double cost = (wide ? kWideStepUs : kStepUs) * (count <= units ? longest : together * (count <= slots ? longest : std::max(longest, sum / slots + 0.5 * longest)));
            if (bytes > 0.0) cost += kJoinUs + kJoinChunkUs * ceil((double)most_steps / length) + bytes / kJoinBytesPerUs;
            if (cost < (length == most_steps ? 1.0 : 0.97) * best_cost) {   // (more chunks only for something)
                best_cost = cost;
                best = length;
                pl.rows_log2 = 7 + wide;
            }
        }
    }
    // Wide blocks, more than half as many as there are units: the longest are cut, and units left over take what remains of them, two of those
    // each and with time to spare (blocks are handed to parts of the device in turn, whichever is free).  Four chunks of 340 .. 421 rows behind 7100 .. 9800 tokens
    // of e4m3, 208 blocks of 118 .. 159 steps, by the steps of a first piece: 159 308, 145 293, 135 277, 124 260 *, 119 (every request cut) 303; halves 326.
    // Forty other batches for which it is chosen, of 1 .. 10 requests of 40 .. 1100 rows behind 1300 .. 20000 tokens, bf16, e4m3 and int8, 64/8, 64/4, 32/8 and 32/32 heads, against even
    // shares: 0.83 .. 1.03 of the time, 0.93 in the mean, 36 of them less; 17 of 29 rows behind 5869 187 -> 152, 205 -> 163, 211 -> 167.
    // (Blocks of 128 rows, two a unit: between 0.94 and 1.09 of the time, and are left alone.)
    double first = 0.0;
    const double best_even = best_cost;
    each_request([&](int64_t rows, int, int) { first += (double)((rows + 255) >> 8) * a->Hkv; });
    const bool cut = a->d == 128 && padded[1] <= 1.1 * padded[0] && !whole && first > 0.5 * units && first < units;
    for (int part = 1; part <= 16 && cut; ++part) {
        const int length = most_steps - most_steps * part / 32;
        double rests = 0.0, rest = 0.0, bytes = 0.0;
        each_request([&](int64_t rows, int tokens, int) {
            const int steps = (tokens + kStep - 1) / kStep;
            if (steps <= length) return;
            const double blocks = (double)((rows + 255) >> 8) * a->Hkv;
            rests += blocks;
            rest += blocks * (steps - length + kBlockSteps);
            bytes += (double)rows * a->Hkv * 2 * a->d * 8.0;
        });
        if (rests == 0.0 || rests > 2.0 * (units - first) || rest > 0.6 * (units - first) * length) continue;
        const double cost = kWideStepUs * (length + kBlockSteps) + kJoinUs + 2 * kJoinChunkUs + bytes / kJoinBytesPerUs;
        if (cost < best_cost && cost < 0.93 * best_even) {
            best_cost = cost;
            best = length;
            pl.rows_log2 = 8;
            pl.even = 0;
        }
    }
    pl.items = row_item(a->T, a->B, group, pl.rows_log2);
    pl.chunk_tokens = best * kStep;
    pl.max_chunks = (most_steps + best - 1) / best;
    size_t at = 0;
    if (pl.max_chunks > 1) {
        const size_t partials = (size_t)a->T * a->Hq * pl.max_chunks;
        pl.acc = at;
        at += align_up(partials * a->d * 4);
        pl.ml = at;
        at += align_up(partials * 8);
    }
    pl.total = std::max(at, kAlign);
    return pl;
}

spec_status check_weight(const spec_kv_weight_args *a)
{
    if (a == nullptr) return SPEC_EINVAL;
    const spec_status st = check_rows(a->B, a->Hq, a->Hkv, a->d, a->num_blocks, a->max_blocks_per_req, a->T, a->kv_dtype, a->kv_layout, a->max_kv_len,
                                      a->q_token_stride, a->q, a->k_cache, a->kv_scale, a->block_table, a->kv_len, a->cu_q_len, a->host_kv_len,
                                      a->host_cu_q_len, a->softmax_scale);
    if (st == SPEC_EINVAL) return st;
    if (a->weight == nullptr || (a->T > 0 && a->lse == nullptr)) return SPEC_EINVAL;
    if (!aligned(a->weight, 32) || !aligned(a->weight_in, 32) || !aligned(a->lse, 4)) return SPEC_EINVAL;
    if (a->weight_in != nullptr && a->weight_in != a->weight && overlap(a->weight_in, a->weight, (size_t)a->num_blocks * a->Hkv * SPEC_BLOCK_SIZE * 4)) return SPEC_EINVAL;
    return st;
}

constexpr int kWeightFewWaves = 16;   // wavefronts a compute unit that kWeightFew's blocks of several groups of tokens leave at least

spec_status check_evict(const spec_kv_evict_args *a)
{
    if (a == nullptr || a->B < 1 || a->Hkv < 1 || a->num_blocks < 1 || a->max_blocks_per_req < 1 || a->dst_max_blocks < 1 || a->first < 0 || a->recent < 0)
        return SPEC_EINVAL;
    if (a->k_cache == nullptr || a->v_cache == nullptr || a->weight == nullptr || a->block_table == nullptr || a->kv_len == nullptr || a->keep == nullptr ||
        a->dst_block_table == nullptr || a->new_kv_len == nullptr)
        return SPEC_EINVAL;
    if (a->dst_block_table == a->block_table) return SPEC_EINVAL;   // (the pages read would be written)
    for (const int32_t *lengths : {a->kv_len, a->keep})
        if (overlap(a->new_kv_len, lengths, (size_t)a->B * 4)) return SPEC_EINVAL;   // (a block's wavefronts read them while its first writes)
    const bool b8 = a->kv_dtype == SPEC_E4M3 || a->kv_dtype == SPEC_INT8;
    if (!b8 && !float_or_bf16(a->kv_dtype)) return SPEC_EINVAL;
    if ((a->kv_scale != nullptr) != b8) return SPEC_EINVAL;
    if (a->kv_layout != SPEC_KV_MFMA && a->kv_layout != SPEC_KV_TOKEN_MAJOR) return SPEC_EINVAL;
    if ((b8 && a->kv_layout != SPEC_KV_MFMA) || (a->kv_dtype == SPEC_F32 && a->kv_layout != SPEC_KV_TOKEN_MAJOR)) return SPEC_EINVAL;
    if (!aligned(a->k_cache, 32) || !aligned(a->v_cache, 32) || !aligned(a->kv_scale, 32) || !aligned(a->weight, 32)) return SPEC_EINVAL;
    if (a->max_kv_len < 0 || (a->max_kv_len == 0 && a->host_kv_len == nullptr) || pages_of(a->max_kv_len) > a->max_blocks_per_req) return SPEC_EINVAL;
    if (a->host_kv_len != nullptr)
        for (int b = 0; b < a->B; ++b)
            if (a->host_kv_len[b] < 0 || pages_of(a->host_kv_len[b]) > a->max_blocks_per_req || (a->max_kv_len > 0 && a->host_kv_len[b] > a->max_kv_len))
                return SPEC_EINVAL;
    if (a->d != 64 && a->d != 128) return SPEC_EUNSUPPORTED;
    if (a->num_blocks > INT32_MAX / SPEC_BLOCK_SIZE || a->max_blocks_per_req > kMaxPacked / SPEC_BLOCK_SIZE) return SPEC_EUNSUPPORTED;
    if (a->B > kMostGrid || a->Hkv > kMostKvHeads || (int64_t)a->dst_max_blocks * a->Hkv * 64 >= kMostThreads || a->dst_max_blocks > kMaxPacked / SPEC_BLOCK_SIZE)
        return SPEC_EUNSUPPORTED;
    return SPEC_OK;
}

struct EvictPlan {
    int capacity, score_stride, held;
    size_t chosen, total;
};
EvictPlan plan_evict(const spec_kv_evict_args *a)
{
    EvictPlan pl;
    pl.capacity = capacity_of(a->B, a->max_kv_len, a->host_kv_len, nullptr);
    pl.held = pl.capacity <= kEvictTurn ? 1 : pl.capacity <= 4 * kEvictTurn ? 4 : 8;
    const int64_t segment = (int64_t)pl.held * kEvictTurn;   // (of requests up to kEvictTurn tokens no scores are handed over)
    pl.score_stride = pl.held == 1 ? 0 : (int)((pl.capacity + segment - 1) / segment * segment);
    pl.chosen = align_up((size_t)a->B * pl.score_stride * 4);
    pl.total = pl.chosen + align_up((size_t)a->B * a->dst_max_blocks * SPEC_BLOCK_SIZE * 4);
    return pl;
}

}  // namespace

}  // namespace specv

using namespace specv;

extern "C" {

spec_status spec_qk_norm_rope(const spec_qk_norm_rope_args *a, void *hip_stream)
{
    const spec_status st = check_rope(a);
    if (st != SPEC_OK || a->T == 0) return st;
    QkNormRopeParams p;
    memset(&p, 0, sizeof p);
    p.T = a->T; p.Hq = a->Hq; p.Hkv = a->Hkv; p.d = a->d; p.f32 = a->dtype == SPEC_F32; p.weight_f32 = a->weight_dtype == SPEC_F32;
    p.rot_dim = a->rot_dim; p.interleaved = a->interleaved;
    p.eps = a->eps;
    p.scale = a->scale == 0.0f ? 1.0f : a->scale;
    const int64_t q_row = (int64_t)a->Hq * a->d, k_row = (int64_t)a->Hkv * a->d;
    p.q_stride = a->q_stride != 0 ? a->q_stride : q_row;
    p.k_stride = a->k_stride != 0 ? a->k_stride : k_row;
    p.out_q_stride = a->out_q_stride != 0 ? a->out_q_stride : q_row;
    p.out_k_stride = a->out_k_stride != 0 ? a->out_k_stride : k_row;
    p.q = a->q; p.k = a->k; p.out_q = a->out_q; p.out_k = a->out_k; p.q_weight = a->q_weight; p.k_weight = a->k_weight;
    p.positions = a->positions; p.inv_freq = a->inv_freq;
    return launch_qk_norm_rope(p, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? SPEC_OK : SPEC_EHIP;
}

size_t spec_prompt_attn_workspace_bytes(const spec_prompt_attn_args *a) { return check_prompt(a) == SPEC_OK ? plan_prompt(a, false).total : 0; }

spec_status spec_prompt_attn(const spec_prompt_attn_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const spec_status st = check_prompt(a);
    if (st != SPEC_OK) return st;
    if (workspace == nullptr || !aligned(workspace, kAlign)) return SPEC_EWORKSPACE;
    PromptPlan pl = plan_prompt(a, false);
    if (workspace_bytes < pl.total) pl = plan_prompt(a, true);   // (sized for another call: tokens are not split)
    if (workspace_bytes < pl.total) return SPEC_EWORKSPACE;
    if (a->T == 0) return SPEC_OK;
    if (((int64_t)pl.items * a->Hkv + 1) * (2 << pl.rows_log2) >= kMostThreads) return SPEC_EUNSUPPORTED;   // (two threads a row)
    char *ws = static_cast<char *>(workspace);
    PromptAttnParams p;
    memset(&p, 0, sizeof p);
    p.B = a->B; p.Hq = a->Hq; p.Hkv = a->Hkv; p.group = a->Hq / a->Hkv; p.num_blocks = a->num_blocks; p.max_blocks_per_req = a->max_blocks_per_req; p.T = a->T;
    p.kind = kind_of(a->kv_dtype, a->kv_layout);
    p.d = a->d; p.out_f32 = a->out_dtype == SPEC_F32;
    p.rows_log2 = pl.rows_log2; p.items = pl.items; p.even = pl.even; p.chunk_tokens = pl.chunk_tokens; p.max_chunks = pl.max_chunks; p.capacity_tokens = pl.capacity;
    p.group_inverse = inverse_of_group(p.group);
    p.scale_log2 = scale_log2_of(a->softmax_scale, a->d);
    p.q_stride = a->q_token_stride != 0 ? a->q_token_stride : (int64_t)a->Hq * a->d;
    p.q = a->q; p.k_cache = a->k_cache; p.v_cache = a->v_cache; p.kv_scale = a->kv_scale;
    p.block_table = a->block_table; p.kv_len = a->kv_len; p.cu_q_len = a->cu_q_len;
    p.out = a->out; p.lse = a->lse;
    p.acc = reinterpret_cast<float *>(ws + pl.acc);
    p.ml = reinterpret_cast<float *>(ws + pl.ml);
    p.errors = reinterpret_cast<unsigned long long *>(a->error_count);
    return launch_prompt_attn(p, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? SPEC_OK : SPEC_EHIP;
}

spec_status spec_kv_weight(const spec_kv_weight_args *a, void *hip_stream)
{
    const spec_status st = check_weight(a);
    if (st != SPEC_OK || a->T == 0) return st;
    KvWeightParams p;
    memset(&p, 0, sizeof p);
    p.B = a->B; p.Hq = a->Hq; p.Hkv = a->Hkv; p.group = a->Hq / a->Hkv; p.num_blocks = a->num_blocks; p.max_blocks_per_req = a->max_blocks_per_req; p.T = a->T;
    p.kind = kind_of(a->kv_dtype, a->kv_layout);
    p.d = a->d;
    p.capacity_tokens = capacity_of(a->B, a->max_kv_len, a->host_kv_len, a->host_cu_q_len);
    p.max_tiles = std::max((p.capacity_tokens + kWeightTokens - 1) / kWeightTokens, 1);
    if ((int64_t)p.max_tiles * a->Hkv * 4 * 64 >= kMostThreads) return SPEC_EUNSUPPORTED;
    int64_t units = 0;
    int most_rows = 0;
    for (int b = 0; b < a->B; ++b) {
        const int n = a->host_cu_q_len[b + 1] - a->host_cu_q_len[b];
        most_rows = std::max(most_rows, n * p.group);
        if (n > 0) units += (int64_t)((a->max_kv_len > 0 ? a->max_kv_len : a->host_kv_len[b]) + kWeightTokens - 1) / kWeightTokens * a->Hkv;
    }
    // A block for each 32 tokens as long as all of them run at once (two a unit): 32 rows of 64/8 heads behind 500 tokens 5.9 us against 9.2 and 9.3 of the
    // other two forms, 2000 tokens 6.4, 9.7, 9.3; 4000 tokens 11.2, 9.7, 9.6.  Rows that fit LDS stay there: four requests of 4000 .. 12000 tokens 22 against 27.
    p.form = most_rows <= kWeightFewRows ? kWeightFew : units <= 2 * compute_units() ? kWeightShared : most_rows <= kWeightSomeRows ? kWeightSome : kWeightOwn;
    p.groups = (int)std::min<int64_t>(std::max<int64_t>(units / (kWeightFewWaves * compute_units()), 1), 16);
    if (p.form == kWeightSome) {
        // As few groups as let all blocks run at once (two a unit), else two: four requests of 4500 .. 9400 tokens, by groups: 25.3, 22.1 *, 27.2, 33.8; of 8500: 30.8, 32.2, 28.7 *,
        // 34.1; two of 30000, int8: 44.2, 40.9, -, 39.8 *; 32/8 heads, sixteen of 4000 .. 12000: 73, 63.7 *, -, 64.6.
        // Nine more batches that four groups do not fit (4 .. 64 requests of 1000 .. 30000 tokens, bf16, e4m3 and int8, 64/8, 32/8 and 32/32 heads), 1, 2, 3, 4 and 6 groups: two are within 6% of the best.
        auto blocks = [&](int groups) {
            int64_t n = 0;
            for (int b = 0; b < a->B; ++b)
                if (a->host_cu_q_len[b + 1] > a->host_cu_q_len[b]) n += (a->max_kv_len > 0 ? a->max_kv_len : a->host_kv_len[b]) / (8 * kWeightTokens * groups) + 1;
            return n * a->Hkv;
        };
        for (p.groups = 1; p.groups < 5 && blocks(p.groups) > 2 * compute_units(); ++p.groups) {}
        if (p.groups == 5) p.groups = 2;
    }
    p.group_inverse = inverse_of_group(p.group);
    p.scale_log2 = scale_log2_of(a->softmax_scale, a->d);
    p.q_stride = a->q_token_stride != 0 ? a->q_token_stride : (int64_t)a->Hq * a->d;
    p.q = a->q; p.lse = a->lse; p.k_cache = a->k_cache; p.kv_scale = a->kv_scale; p.weight_in = a->weight_in; p.weight = a->weight;
    p.block_table = a->block_table; p.kv_len = a->kv_len; p.cu_q_len = a->cu_q_len;
    p.errors = reinterpret_cast<unsigned long long *>(a->error_count);
    return launch_kv_weight(p, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? SPEC_OK : SPEC_EHIP;
}

size_t spec_kv_evict_workspace_bytes(const spec_kv_evict_args *a) { return check_evict(a) == SPEC_OK ? plan_evict(a).total : 0; }

spec_status spec_kv_evict(const spec_kv_evict_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const spec_status st = check_evict(a);
    if (st != SPEC_OK) return st;
    const EvictPlan pl = plan_evict(a);
    if (workspace == nullptr || !aligned(workspace, kAlign) || workspace_bytes < pl.total) return SPEC_EWORKSPACE;
    KvEvictParams p;
    memset(&p, 0, sizeof p);
    p.B = a->B; p.Hkv = a->Hkv; p.d = a->d; p.num_blocks = a->num_blocks; p.max_blocks_per_req = a->max_blocks_per_req; p.dst_max_blocks = a->dst_max_blocks;
    p.kv_dtype = a->kv_dtype; p.kv_layout = a->kv_layout; p.first = a->first; p.recent = a->recent;
    p.capacity_tokens = pl.capacity; p.score_stride = pl.score_stride; p.held = pl.held;
    p.k_cache = a->k_cache; p.v_cache = a->v_cache; p.kv_scale = a->kv_scale; p.weight = a->weight;
    p.block_table = a->block_table; p.kv_len = a->kv_len; p.keep = a->keep; p.dst_block_table = a->dst_block_table;
    p.new_kv_len = a->new_kv_len; p.kept = a->kept;
    p.score = static_cast<uint32_t *>(workspace);
    p.chosen = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + pl.chosen);
    p.errors = reinterpret_cast<unsigned long long *>(a->error_count);
    return launch_kv_evict(p, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? SPEC_OK : SPEC_EHIP;
}

}  // extern "C"

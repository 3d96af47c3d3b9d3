// C entry points of the 8-bit cache and of the attention over shared prefixes: argument checks, launch plans.
#include "cache_ops.h"

#include <math.h>
#include <string.h>

#include <algorithm>
#include <atomic>

namespace specv {

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxPacked = (int64_t)1 << 30;   // packed (token, head) rows and work items are 32-bit in the kernels
constexpr int kPairTokens = 4 * 2 * SPEC_BLOCK_SIZE;   // tokens that a block's wavefronts take at a time

int compute_units()
{
    static int cached = 0;
    if (cached == 0) {
        int dev = 0, n = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1)
            n = 256;   // MI355X
        cached = n;
    }
    return cached;
}

bool aligned(const void *ptr, uintptr_t to) { return (reinterpret_cast<uintptr_t>(ptr) & (to - 1)) == 0; }
int pages_of(int64_t tokens) { return (int)((tokens + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE); }
size_t align_up(size_t n) { return (n + kAlign - 1) & ~(kAlign - 1); }

// cu[0] = 0 <= cu[1] <= ... <= cu[n] = total
bool prefix_sum_ok(const int32_t *cu, int n, int total)
{
    if (cu[0] != 0 || cu[n] != total) return false;
    for (int i = 0; i < n; ++i)
        if (cu[i + 1] < cu[i]) return false;
    return true;
}

// ---------------------------------------------------------------------------
// Append and read
// ---------------------------------------------------------------------------
spec_status check_append(const spec_kv8_append_args *a)
{
    if (a == nullptr || a->B < 1 || a->Hkv < 1 || a->T < 0 || a->num_blocks < 1 || a->max_blocks_per_req < 1) return SPEC_EINVAL;
    if (a->k_cache == nullptr || a->v_cache == nullptr || a->kv_scale == nullptr || a->block_table == nullptr || a->kv_len == nullptr ||
        a->cu_q_len == nullptr || a->host_cu_q_len == nullptr)
        return SPEC_EINVAL;
    if (a->T > 0 && (a->new_k == nullptr || a->new_v == nullptr)) return SPEC_EINVAL;   // (no rows need no address)
    if (a->src_dtype != SPEC_F32 && a->src_dtype != SPEC_BF16) return SPEC_EINVAL;
    if (a->kv_dtype != SPEC_E4M3 && a->kv_dtype != SPEC_INT8) return SPEC_EINVAL;
    if (!aligned(a->k_cache, 32) || !aligned(a->v_cache, 32) || !aligned(a->kv_scale, 32) || !aligned(a->new_k, 16) || !aligned(a->new_v, 16))
        return SPEC_EINVAL;
    const int64_t esz = a->src_dtype == SPEC_F32 ? 4 : 2, row = (int64_t)a->Hkv * a->d;
    if (a->token_stride != 0 && (a->token_stride < row || a->token_stride * esz % 16 != 0)) return SPEC_EINVAL;
    if (!prefix_sum_ok(a->host_cu_q_len, a->B, a->T)) return SPEC_EINVAL;
    if (a->host_kv_len != nullptr)
        for (int b = 0; b < a->B; ++b) {
            const int n = a->host_cu_q_len[b + 1] - a->host_cu_q_len[b];
            if (n > 0 && (a->host_kv_len[b] < n || pages_of(a->host_kv_len[b]) > a->max_blocks_per_req)) return SPEC_EINVAL;
        }
    if (a->d != 64 && a->d != 128) return SPEC_EUNSUPPORTED;
    if (((int64_t)a->T / SPEC_BLOCK_SIZE + 2 * (int64_t)a->B) * a->Hkv > kMaxPacked) return SPEC_EUNSUPPORTED;
    return SPEC_OK;
}

spec_status check_read(const spec_kv8_read_args *a)
{
    if (a == nullptr || a->B < 1 || a->Hkv < 1 || a->T < 0 || a->num_blocks < 1 || a->max_blocks_per_req < 1) return SPEC_EINVAL;
    if (a->k_cache == nullptr || a->v_cache == nullptr || a->kv_scale == nullptr || a->block_table == nullptr || a->cu_len == nullptr ||
        a->host_cu_len == nullptr)
        return SPEC_EINVAL;
    if (a->T > 0 && (a->out_k == nullptr || a->out_v == nullptr)) return SPEC_EINVAL;
    if (a->kv_dtype != SPEC_E4M3 && a->kv_dtype != SPEC_INT8) return SPEC_EINVAL;
    if (a->out_dtype != SPEC_F32 && a->out_dtype != SPEC_BF16) return SPEC_EINVAL;
    if (!aligned(a->k_cache, 32) || !aligned(a->v_cache, 32) || !aligned(a->kv_scale, 32) || !aligned(a->out_k, 32) || !aligned(a->out_v, 32))
        return SPEC_EINVAL;
    if (!prefix_sum_ok(a->host_cu_len, a->B, a->T)) return SPEC_EINVAL;
    if (a->d != 64 && a->d != 128) return SPEC_EUNSUPPORTED;
    if (((int64_t)a->T / SPEC_BLOCK_SIZE + 2 * (int64_t)a->B) * a->Hkv > kMaxPacked) return SPEC_EUNSUPPORTED;
    return SPEC_OK;
}

// ---------------------------------------------------------------------------
// Attention: one set of checks and one plan for both entry points
// ---------------------------------------------------------------------------
spec_prefix_attn_args as_prefix_args(const spec_kv8_attn_args *a)   // no groups: G == 0
{
    spec_prefix_attn_args x;
    memset(&x, 0, sizeof x);
    x.B = a->B; x.Hq = a->Hq; x.Hkv = a->Hkv; x.d = a->d; x.num_blocks = a->num_blocks; x.max_blocks_per_req = a->max_blocks_per_req; x.T = a->T;
    x.kv_dtype = a->kv_dtype; x.kv_layout = SPEC_KV_MFMA; x.out_dtype = a->out_dtype; x.max_kv_len = a->max_kv_len;
    x.q_token_stride = a->q_token_stride;
    x.q = a->q; x.k_cache = a->k_cache; x.v_cache = a->v_cache; x.kv_scale = a->kv_scale;
    x.block_table = a->block_table; x.kv_len = a->kv_len; x.cu_q_len = a->cu_q_len; x.out = a->out;
    x.host_kv_len = a->host_kv_len; x.host_cu_q_len = a->host_cu_q_len;
    x.error_count = a->error_count; x.softmax_scale = a->softmax_scale;
    return x;
}

spec_status check_attn(const spec_prefix_attn_args *a)
{
    if (a->B < 1 || a->Hq < 1 || a->Hkv < 1 || a->num_blocks < 1 || a->max_blocks_per_req < 1 || a->T < 1) return SPEC_EINVAL;
    if (a->q == nullptr || a->k_cache == nullptr || a->v_cache == nullptr || a->block_table == nullptr || a->kv_len == nullptr ||
        a->cu_q_len == nullptr || a->out == nullptr || a->host_cu_q_len == nullptr)
        return SPEC_EINVAL;
    if (a->kv_dtype != SPEC_BF16 && a->kv_dtype != SPEC_E4M3 && a->kv_dtype != SPEC_INT8) return SPEC_EINVAL;
    const bool b8 = a->kv_dtype != SPEC_BF16;
    if ((a->kv_scale != nullptr) != b8) return SPEC_EINVAL;
    if (a->kv_layout != SPEC_KV_MFMA && (b8 || a->kv_layout != SPEC_KV_TOKEN_MAJOR)) return SPEC_EINVAL;
    if (a->out_dtype != SPEC_F32 && a->out_dtype != SPEC_BF16) return SPEC_EINVAL;
    if (!aligned(a->k_cache, 32) || !aligned(a->v_cache, 32) || !aligned(a->kv_scale, 32) || !aligned(a->out, 32) || !aligned(a->q, 16))
        return SPEC_EINVAL;
    if (a->max_kv_len < 0 || (a->max_kv_len == 0 && a->host_kv_len == nullptr)) return SPEC_EINVAL;
    if (pages_of(a->max_kv_len) > a->max_blocks_per_req) return SPEC_EINVAL;
    if (a->Hq % a->Hkv != 0) return SPEC_EINVAL;
    if (!(a->softmax_scale >= 0.0f) || isinf(a->softmax_scale)) return SPEC_EINVAL;
    if (a->q_token_stride != 0 && (a->q_token_stride < (int64_t)a->Hq * a->d || a->q_token_stride % 8 != 0)) return SPEC_EINVAL;
    if (!prefix_sum_ok(a->host_cu_q_len, a->B, a->T)) return SPEC_EINVAL;
    if (a->G > 0) {
        if (a->G > a->B || a->cu_group == nullptr || a->prefix_len == nullptr || a->host_cu_group == nullptr || a->host_prefix_len == nullptr)
            return SPEC_EINVAL;
        if (!prefix_sum_ok(a->host_cu_group, a->G, a->B)) return SPEC_EINVAL;
    }
    for (int b = 0, g = 0; b < a->B; ++b) {
        const int n = a->host_cu_q_len[b + 1] - a->host_cu_q_len[b];
        if (n > SPEC_K_MAX + 1) return SPEC_EINVAL;
        int prefix = 0;
        if (a->G > 0) {
            while (g + 1 < a->G && a->host_cu_group[g + 1] <= b) ++g;
            prefix = a->host_prefix_len[g];
            if (b == a->host_cu_group[g] && (prefix < 0 || prefix % SPEC_BLOCK_SIZE != 0 || prefix / SPEC_BLOCK_SIZE > a->max_blocks_per_req))
                return SPEC_EINVAL;
            if (a->max_kv_len > 0 && n > 0 && prefix > 0 && prefix + n > a->max_kv_len) return SPEC_EINVAL;
        }
        if (a->host_kv_len == nullptr || n == 0) continue;
        const int len = a->host_kv_len[b];
        if (len < 0 || pages_of(len) > a->max_blocks_per_req || (a->max_kv_len > 0 && len > a->max_kv_len)) return SPEC_EINVAL;
        if (prefix > 0 && len - n < prefix) return SPEC_EINVAL;
    }
    for (int g = 0; g < a->G; ++g)
        if (a->host_cu_group[g + 1] == a->host_cu_group[g]) return SPEC_EINVAL;
    if (a->d != 64 && a->d != 128) return SPEC_EUNSUPPORTED;
    if (a->Hq / a->Hkv > 16) return SPEC_EUNSUPPORTED;
    if ((int64_t)a->T * a->Hq > kMaxPacked) return SPEC_EUNSUPPORTED;
    return SPEC_OK;
}

constexpr int kMostTiles = 3;   // row tiles of a block

struct Plan {
    int whole_context, row_tiles, row_blocks, chunk_tokens, max_chunks, capacity, max_q_rows;
    int prefix_tiles, prefix_many_rows, prefix_piece_steps, prefix_rows_log2, prefix_row_blocks, prefix_chunk_tokens, max_prefix_chunks, prefix_capacity;
    size_t acc, ml, tickets, prefix_acc, prefix_ml, total;   // offsets into the workspace
    int64_t blocks, prefix_blocks;
};

// Row tiles of a block and chunk length for jobs of some tokens and query rows, from a model of the launch, fitted to single
// requests and batches of 4 and 16 with 300 .. 16000 tokens (40 rows, d = 128) at every number of tiles and chunks.
//
// With n row tiles a block takes kBlockUs[n] and kTokenUs[n] for a token: more rows are more to multiply and to merge, and all wait
// for the slowest wavefront (700 tokens of one request, 8-bit, n = 1, 2, 3: 8.3 / 10.0 / 12.2 us), but fewer tiles mean more blocks
// that read the same pages.  A job of c chunks waits for its partial results and a ticket, and its last block reads c times its rows
// (6000 tokens of one request, n = 1, c = 3, 6, 12, 24, 48: 19.0 / 15.6 / 18.0 / 36.6 / 56.7 us).  A second block on a compute
// unit shares its issue slots and its share of the memory with the first, and adds a tenth to the rate; blocks beyond the first on each
// unit end at different times, which costs half of the longest one.
struct Split {
    int tiles, length;
    double us;
};
constexpr double kBlockUs[4] = {0.0, 4.7, 5.5, 6.7}, kTokenUs[4] = {0.0, 0.0052, 0.0064, 0.0078};
constexpr double kFullFactor = 1.4, kShortFactor = 0.7;                              // of a token, with weights in more than one term; with d = 64
constexpr double kTicketUs = 2.5, kJoinUs[4] = {0.0, 0.55, 0.75, 0.95};              // of a split job; of each of its chunks
constexpr double kSecondBlock = 1.1;

// A prefix is walked once for all of its group's rows by a launch of its own, whose results the own launch takes in; or each request
// walks its whole context, which is one launch and reads the prefix again for every request, mostly from the caches.  The second is
// less work than it seems while prefixes are short or groups small (64/8 heads, bf16 pages: two requests behind 512 tokens 13.1 -> 8.1 us, 64
// behind 512 tokens 32 -> 16; 32/8 heads, 8-bit, 4 x 16 requests behind 2048 tokens 37 -> 25), the first where they are long
// and groups large (64/8 heads, 64 requests behind 4096 tokens 74 against 81; 32/8 heads, 2 x 64 behind 8192 115 against 279; 16 x 12
// requests without drafts behind 8192 125 against 499).  The model of the second: a token that comes from the caches costs a busy compute
// unit kCachedTokens of its time alone, kFarTokens of it when the prefixes of a KV head do not fit an XCD's L2 well (kNearBytes) or
// are bf16, twice the bytes; it was found too low by kWhole*; and the caches give kCacheBytesPerUs.  Of the first: the sum of its launches
// was found too low by kTwoLaunches, and memory gives kMemoryBytesPerUs.
constexpr double kCachedTokens = 0.5, kFarTokens = 0.7, kNearBytes = 3e6, kWholeBf16 = 1.15, kWholeInt8 = 1.25, kCacheBytesPerUs = 9e6;
constexpr double kTwoLaunches = 1.1, kLaunchUs = 2.5, kMemoryBytesPerUs = 5.3e6;
template <typename F>
Split split_jobs(int most_rows, int most_tokens, int Hkv, double token_factor, double ticket_us, double busy_tokens, bool least, F for_each_job)   // for_each_job(f): f(tokens, rows)
{
    const int most = std::min(kMaxChunkTokens, std::max((most_tokens + kPairTokens - 1) / kPairTokens * kPairTokens, kPairTokens));
    const double units = compute_units();
    const int most_tiles = std::min((most_rows + 15) / 16, kMostTiles);
    Split best = {most_tiles, most, 1e30};
    if (least) return best;   // the fewest chunks
    for (int tiles = most_tiles; tiles >= 1; --tiles) {
        const double token_us = kTokenUs[tiles] * token_factor;
        for (int len = most; len >= kPairTokens; len = len * 3 / 4 / kPairTokens * kPairTokens) {
            double longest = 0.0, sum = 0.0, count = 0.0;
            for_each_job([&](int tokens, int64_t rows) {
                const int chunks = std::max((tokens + len - 1) / len, 1), each = (tokens + chunks - 1) / chunks;
                const double blocks = (double)((rows + 16 * tiles - 1) / (16 * tiles)) * Hkv * chunks;
                const double us = kBlockUs[tiles] + each * token_us, join_us = chunks > 1 ? ticket_us + chunks * kJoinUs[tiles] : 0.0;
                longest = std::max(longest, us + join_us);
                sum += blocks * (kBlockUs[tiles] + each * token_us * busy_tokens);
                count += blocks;
            });
            const double busy = sum / (units * kSecondBlock), us = std::max(longest, count > units ? busy + 0.5 * longest : 0.0);
            if (us < best.us * 0.97) best = {tiles, len, us};   // (fewer tiles or shorter chunks only for something)
            if (busy >= best.us) break;   // (shorter chunks are more work in all)
        }
    }
    return best;
}

// Most steps of a piece of the launch for prefixes with many rows, from a model of it.  A block takes kPieceUs besides its steps; a step
// takes kStepUs while the block has its compute unit for itself, and kSharedStepUs where two share one, which is what fits: matrix cores and
// vector units are busy at the same time more often (d = 128, weights in one term, bf16 pages without the second one; measured behind one prefix of 4096
// tokens, 64 requests, 64/8 heads, k = 2: 24 steps alone 32 us, 12 and 12 together 22 us; wide: a block of eight wavefronts has the unit, 13 steps 22 us,
// and 31 with the second term).  More blocks than that take turns.  Each piece of a prefix is
// partial results to write and to read back.
constexpr double kPieceUs = 7.0, kStepUs = 1.35, kSharedStepUs = 1.87, kWideStepUs = 1.7, kPieceJoinUs = 0.35;
template <typename F>
int prefix_piece_steps(int most_steps, int Hkv, int d, bool full, bool codes, bool wide, bool least, double &best_us, F for_each_group)   // for_each_group(f): f(row blocks, steps)
{
    const double units = compute_units(), slots = wide ? units : 2 * units, busy_us = wide ? kWideStepUs : kSharedStepUs, factor = d / 128.0 * (codes ? (full ? 1.5 : 1.0) : (full ? 2.0 : 1.45));   // (more terms: more products with V)
    int best = std::min(most_steps, kMaxPrefixSteps);
    best_us = 1e30;
    if (least) return best;   // the fewest pieces
    for (int len = best; len >= 1; len = std::min(len - 1, len * 7 / 8)) {
        double count = 0.0, sum = 0.0, longest = 0.0, pieces = 0.0;
        for_each_group([&](int64_t row_blocks, int steps) {
            if (steps == 0) return;
            const int n = (steps + len - 1) / len, each = (steps + n - 1) / n;
            count += (double)row_blocks * n * Hkv;
            sum += (double)row_blocks * n * Hkv * (kPieceUs + each * busy_us * factor);
            longest = std::max(longest, (double)each);
            pieces = std::max(pieces, (double)n);
        });
        double us = kPieceUs + longest * factor * (count <= units && !wide ? kStepUs : busy_us);
        if (count > slots) us = std::max(us, sum / slots + 0.5 * longest * factor * busy_us);
        us += pieces * kPieceJoinUs;
        if (us < best_us) {
            best_us = us;
            best = len;
        }
        if (sum / slots > best_us) break;   // (shorter pieces are more work in all)
    }
    return best;
}

// The plan that the models above find the fastest, or the one that leaves the least in the workspace.
Plan make_plan(const spec_prefix_attn_args *a, bool least)
{
    Plan pl;
    memset(&pl, 0, sizeof pl);
    const int group = a->Hq / a->Hkv;
    const bool full = a->out_dtype == SPEC_F32;
    const double token_factor = (full ? kFullFactor : 1.0) * (a->d == 64 ? kShortFactor : 1.0);
    int max_q = 0, max_own = 0, max_len = 0;
    auto prefix_of = [&](int &g, int b) {
        if (a->G == 0) return 0;
        while (g + 1 < a->G && a->host_cu_group[g + 1] <= b) ++g;
        return (int)a->host_prefix_len[g];
    };
    for (int b = 0, g = 0; b < a->B; ++b) {
        const int n = a->host_cu_q_len[b + 1] - a->host_cu_q_len[b], prefix = prefix_of(g, b);
        if (n == 0) continue;
        const int len = a->max_kv_len > 0 ? a->max_kv_len : a->host_kv_len[b];
        max_q = std::max(max_q, n);
        max_own = std::max(max_own, len - prefix);
        max_len = std::max(max_len, len);
    }
    const int max_rows = std::max(max_q * group, 1);
    pl.max_q_rows = max_rows;
    pl.capacity = a->max_kv_len > 0 ? a->max_kv_len : max_len;
    auto split_own = [&](int most_tokens, bool whole, double busy_tokens) {
        return split_jobs(max_rows, most_tokens, a->Hkv, token_factor, kTicketUs, busy_tokens, least, [&](auto job) {
            for (int b = 0, g = 0; b < a->B; ++b) {
                const int q = a->host_cu_q_len[b + 1] - a->host_cu_q_len[b], prefix = whole ? 0 : prefix_of(g, b);
                if (q > 0) job((a->max_kv_len > 0 ? a->max_kv_len : a->host_kv_len[b]) - prefix, q * group);
            }
        });
    };
    const size_t rows = (size_t)a->T * a->Hq;
    auto chunks_of = [](const Split &split, int tokens) { return std::max((tokens + split.length - 1) / split.length, 1); };
    auto row_blocks_of = [&](const Split &split) { return (max_rows + 16 * split.tiles - 1) / (16 * split.tiles); };
    auto partial_bytes = [&](int chunks) { return align_up(rows * chunks * a->d * 4) + align_up(rows * chunks * 8); };
    auto ticket_bytes = [&](const Split &split) { return (size_t)a->B * a->Hkv * row_blocks_of(split) * 8; };
    auto own_bytes = [&](const Split &split, int tokens) {
        const int chunks = chunks_of(split, tokens);
        return chunks > 1 ? partial_bytes(chunks) + align_up(ticket_bytes(split)) : 0;
    };
    Split own = split_own(max_own, false, 1.0);
    int max_prefix = 0;
    int64_t most_rows = 0;
    for (int g = 0; g < a->G; ++g) {
        max_prefix = std::max(max_prefix, a->host_prefix_len[g]);
        most_rows = std::max<int64_t>(most_rows, (int64_t)(a->host_cu_q_len[a->host_cu_group[g + 1]] - a->host_cu_q_len[a->host_cu_group[g]]) * group);
    }
    if (max_prefix > 0 && most_rows > 0) {
        pl.prefix_capacity = max_prefix;
        double prefix_us = 0.0;
        pl.prefix_many_rows = most_rows > 16 * kMostTiles;
        auto rows_of = [&](int g) { return (int64_t)(a->host_cu_q_len[a->host_cu_group[g + 1]] - a->host_cu_q_len[a->host_cu_group[g]]) * group; };
        if (pl.prefix_many_rows) {
            constexpr int kStepTokens = kStepPages * SPEC_BLOCK_SIZE;
            auto steps_of = [&](int tokens) { return (tokens + kStepTokens - 1) / kStepTokens; };
            auto each_group = [&](auto group) {
                for (int g = 0; g < a->G; ++g) group((rows_of(g) + (1 << pl.prefix_rows_log2) - 1) >> pl.prefix_rows_log2, steps_of(a->host_prefix_len[g]));
            };
            // Blocks of eight wavefronts and 256 rows where that does not walk many more absent rows: pages are brought in and converted
            // half as often (calls with 64 requests behind 4096 tokens, 64/8 heads, k = 2, bf16: 78.1 -> 75.6 us; with three documents of 6000 ..
            // 20000 tokens, e4m3: 161 -> 156.5).  Near the limit there is little between them (one group behind 6144 tokens, bf16: 1632 rows, 1.08 times
            // as many, 91.6 -> 86.3; 1104, 1.11, 65.7 -> 65.4; 600, 1.2, 46.3 -> 47.5; 320 behind 2048, 1.33, 22.9 -> 28.0).  With d = 64 more, smaller blocks are as good (15.7 us against 18.4, 18.0 against 16.5 in the next launch).
            double padded[2] = {0.0, 0.0};
            for (int wide = 0; wide < 2; ++wide) {
                pl.prefix_rows_log2 = 7 + wide;
                each_group([&](int64_t row_blocks, int steps) { padded[wide] += (double)(row_blocks << pl.prefix_rows_log2) * steps; });
            }
            const bool wide = a->d == 128 && padded[1] <= 1.1 * padded[0];
            pl.prefix_rows_log2 = wide ? 8 : 7;
            pl.prefix_piece_steps = prefix_piece_steps(steps_of(max_prefix), a->Hkv, a->d, full, a->kv_dtype != SPEC_BF16, pl.prefix_rows_log2 == 8, least, prefix_us, each_group);
            each_group([&](int64_t row_blocks, int steps) {
                pl.prefix_blocks += row_blocks * ((steps + pl.prefix_piece_steps - 1) / pl.prefix_piece_steps) * a->Hkv;
            });
            pl.prefix_blocks = (pl.prefix_blocks + kXcdCount - 1) / kXcdCount * kXcdCount;
            pl.prefix_row_blocks = (int)std::min<int64_t>(pl.prefix_blocks, INT32_MAX);
            pl.max_prefix_chunks = (steps_of(max_prefix) + pl.prefix_piece_steps - 1) / pl.prefix_piece_steps;
        } else {
            const Split split = split_jobs((int)most_rows, max_prefix, a->Hkv, token_factor, 0.0, 1.0, least, [&](auto job) {   // (no ticket: the next launch joins)
                for (int g = 0; g < a->G; ++g)
                    if (a->host_prefix_len[g] > 0) job(a->host_prefix_len[g], rows_of(g));
            });
            prefix_us = split.us;
            pl.prefix_tiles = split.tiles;
            pl.prefix_chunk_tokens = split.length;
            // (as many row blocks as the rows can make however they are spread over the groups)
            pl.prefix_row_blocks = (int)((int64_t)a->T * group / (16 * pl.prefix_tiles)) + a->G;
            pl.max_prefix_chunks = (max_prefix + pl.prefix_chunk_tokens - 1) / pl.prefix_chunk_tokens;
            pl.prefix_blocks = (int64_t)pl.prefix_row_blocks * a->Hkv * pl.max_prefix_chunks;
        }
        const double token_bytes = a->kv_dtype == SPEC_BF16 ? 4.0 * a->d : 2.0 * a->d + 8.0;   // of a KV head
        double prefix_tokens = 0.0, walked_tokens = 0.0;   // of the prefixes; of what the requests walk of them
        for (int g = 0; g < a->G; ++g) {
            prefix_tokens += a->host_prefix_len[g];
            for (int b = a->host_cu_group[g]; b < a->host_cu_group[g + 1]; ++b)
                if (a->host_cu_q_len[b + 1] > a->host_cu_q_len[b]) walked_tokens += a->host_prefix_len[g];
        }
        const bool near = a->kv_dtype != SPEC_BF16 && prefix_tokens * token_bytes <= kNearBytes;
        const Split whole = split_own(max_len, true, near ? kCachedTokens : kFarTokens);
        const double more = a->kv_dtype == SPEC_BF16 ? kWholeBf16 : a->kv_dtype == SPEC_INT8 ? kWholeInt8 : 1.0;
        const double whole_us = std::max(whole.us * more, walked_tokens * token_bytes * a->Hkv / kCacheBytesPerUs);
        const double shared_us = std::max((own.us + prefix_us) * kTwoLaunches, prefix_tokens * token_bytes * a->Hkv / kMemoryBytesPerUs) + kLaunchUs;
        const int shared = prefix_shared_switch();
        const bool whole_wins = least ? own_bytes(whole, max_len) < own_bytes(own, max_own) + partial_bytes(pl.max_prefix_chunks) : whole_us < shared_us;
        if (shared < 0 ? whole_wins : shared == 0) {
            own = whole;
            max_own = max_len;
            pl.whole_context = 1;
            pl.max_prefix_chunks = 0;
            pl.prefix_blocks = pl.prefix_row_blocks = 0;
        }
    }
    pl.row_tiles = own.tiles;
    pl.row_blocks = row_blocks_of(own);
    pl.chunk_tokens = own.length;
    pl.max_chunks = chunks_of(own, max_own);
    pl.blocks = (int64_t)pl.row_blocks * a->B * a->Hkv * pl.max_chunks;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += align_up(bytes); return here; };
    if (pl.max_chunks > 1) {
        pl.acc = take(rows * pl.max_chunks * a->d * 4);
        pl.ml = take(rows * pl.max_chunks * 8);
        pl.tickets = take(ticket_bytes(own));
    }
    if (pl.max_prefix_chunks > 0) {
        pl.prefix_acc = take(rows * pl.max_prefix_chunks * a->d * 4);
        pl.prefix_ml = take(rows * pl.max_prefix_chunks * 8);
    }
    pl.total = std::max(at, kAlign);
    return pl;
}

// Tag of a call's tickets (see ticket_arrive).  The workspace may hold what any other call left in it, partial results above all, so
// the tags are bits that no fp32 result has: negative NaNs whose lower half is not zero (arithmetic makes 0x7FC00000, or hands on
// the NaN of a bf16 input).  They recur after 8 million calls, which leaves nothing behind: the last block to arrive clears its ticket.
uint32_t next_generation()
{
    static std::atomic<uint32_t> calls{0u};
    for (;;) {
        const uint32_t tag = 0xFF800000u | (calls++ & 0x007FFFFFu);
        if ((tag & 0xFFFFu) != 0) return tag;
    }
}

spec_status run_attn(const spec_prefix_attn_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    Plan pl = make_plan(a, false);
    if (workspace_bytes < pl.total) pl = make_plan(a, true);   // (sized for another batch: fewer chunks may still fit)
    if (workspace == nullptr || !aligned(workspace, kAlign) || workspace_bytes < pl.total) return SPEC_EWORKSPACE;
    if (a->B > 65535 || (!pl.prefix_many_rows && pl.prefix_row_blocks > 65535) || pl.row_blocks * pl.max_chunks > 65535) return SPEC_EUNSUPPORTED;   // (grid)
    if (pl.blocks > kMaxPacked || pl.prefix_blocks > (pl.prefix_many_rows ? kMaxPrefixBlocks : kMaxPacked)) return SPEC_EUNSUPPORTED;
    // (a request's partial results are addressed with 32-bit offsets)
    if (pl.max_chunks > 1 && (int64_t)pl.max_q_rows * a->Hkv * pl.max_chunks * a->d * 4 > UINT32_MAX) return SPEC_EUNSUPPORTED;
    char *ws = static_cast<char *>(workspace);
    CacheAttnParams p;
    memset(&p, 0, sizeof p);
    p.B = a->B; p.Hq = a->Hq; p.Hkv = a->Hkv; p.group = a->Hq / a->Hkv; p.num_blocks = a->num_blocks; p.max_blocks_per_req = a->max_blocks_per_req;
    p.T = a->T;
    p.G = pl.max_prefix_chunks > 0 || pl.whole_context ? a->G : 0;   // (groups without a prefix are single requests)
    p.kind = a->kv_dtype == SPEC_E4M3 ? kCacheE4M3 : a->kv_dtype == SPEC_INT8 ? kCacheInt8 : a->kv_layout == SPEC_KV_MFMA ? kCacheTiles : kCacheTokens;
    p.d = a->d;
    p.out_f32 = a->out_dtype == SPEC_F32;
    p.whole_context = pl.whole_context;
    p.row_tiles = pl.row_tiles; p.row_blocks = pl.row_blocks; p.chunk_tokens = pl.chunk_tokens; p.max_chunks = pl.max_chunks;
    p.capacity_tokens = pl.capacity; p.max_q_rows = pl.max_q_rows;
    p.prefix_tiles = pl.prefix_tiles; p.prefix_many_rows = pl.prefix_many_rows; p.prefix_piece_steps = pl.prefix_piece_steps; p.prefix_row_blocks = pl.prefix_row_blocks; p.prefix_chunk_tokens = pl.prefix_chunk_tokens;
    p.prefix_rows_log2 = pl.prefix_rows_log2;
    p.max_prefix_chunks = pl.max_prefix_chunks; p.prefix_capacity = pl.prefix_capacity;
    p.generation = next_generation();
    p.group_inverse = (uint32_t)((((uint64_t)1 << 32) + p.group - 1) / p.group);   // (unused where the group is 1)
    const double scale = a->softmax_scale > 0.0f ? (double)a->softmax_scale : 1.0 / sqrt((double)a->d);
    p.scale_log2 = (float)(scale * kLog2eD);
    p.q_stride = a->q_token_stride != 0 ? a->q_token_stride : (int64_t)a->Hq * a->d;
    p.q = a->q; p.k_cache = a->k_cache; p.v_cache = a->v_cache; p.kv_scale = a->kv_scale;
    p.block_table = a->block_table; p.kv_len = a->kv_len; p.cu_q_len = a->cu_q_len; p.cu_group = a->cu_group; p.prefix_len = a->prefix_len;
    p.out = a->out;
    p.acc = reinterpret_cast<float *>(ws + pl.acc);
    p.ml = reinterpret_cast<float *>(ws + pl.ml);
    p.tickets = reinterpret_cast<unsigned long long *>(ws + pl.tickets);
    p.prefix_acc = reinterpret_cast<float *>(ws + pl.prefix_acc);
    p.prefix_ml = reinterpret_cast<float *>(ws + pl.prefix_ml);
    p.errors = reinterpret_cast<unsigned long long *>(a->error_count);
    return launch_cache_attn(p, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? SPEC_OK : SPEC_EHIP;
}

spec_status check_kv8_attn(const spec_kv8_attn_args *a)
{
    if (a == nullptr || (a->kv_dtype != SPEC_E4M3 && a->kv_dtype != SPEC_INT8)) return SPEC_EINVAL;
    const spec_prefix_attn_args x = as_prefix_args(a);
    return check_attn(&x);
}

spec_status check_prefix_attn(const spec_prefix_attn_args *a)
{
    if (a == nullptr || a->G < 1) return SPEC_EINVAL;
    return check_attn(a);
}

}  // namespace

}  // namespace specv

using namespace specv;

extern "C" {

spec_status spec_kv8_append(const spec_kv8_append_args *a, void *hip_stream)
{
    const spec_status st = check_append(a);
    if (st != SPEC_OK || a->T == 0) return st;
    Kv8AppendParams p;
    memset(&p, 0, sizeof p);
    p.B = a->B; p.Hkv = a->Hkv; p.d = a->d; p.max_blocks_per_req = a->max_blocks_per_req; p.num_blocks = a->num_blocks; p.T = a->T;
    p.src_f32 = a->src_dtype == SPEC_F32;
    p.int8 = a->kv_dtype == SPEC_INT8;
    p.token_stride = a->token_stride != 0 ? a->token_stride : (int64_t)a->Hkv * a->d;
    p.new_k = a->new_k; p.new_v = a->new_v;
    p.k_cache = static_cast<unsigned char *>(a->k_cache); p.v_cache = static_cast<unsigned char *>(a->v_cache); p.kv_scale = a->kv_scale;
    p.block_table = a->block_table; p.kv_len = a->kv_len; p.cu_q_len = a->cu_q_len;
    p.errors = reinterpret_cast<unsigned long long *>(a->error_count);
    return launch_kv8_append(p, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? SPEC_OK : SPEC_EHIP;
}

spec_status spec_kv8_read(const spec_kv8_read_args *a, void *hip_stream)
{
    const spec_status st = check_read(a);
    if (st != SPEC_OK || a->T == 0) return st;
    Kv8ReadParams p;
    memset(&p, 0, sizeof p);
    p.B = a->B; p.Hkv = a->Hkv; p.d = a->d; p.max_blocks_per_req = a->max_blocks_per_req; p.num_blocks = a->num_blocks; p.T = a->T;
    p.out_f32 = a->out_dtype == SPEC_F32;
    p.int8 = a->kv_dtype == SPEC_INT8;
    p.k_cache = static_cast<const unsigned char *>(a->k_cache); p.v_cache = static_cast<const unsigned char *>(a->v_cache);
    p.kv_scale = a->kv_scale;
    p.block_table = a->block_table; p.start = a->start; p.cu_len = a->cu_len;
    p.out_k = a->out_k; p.out_v = a->out_v;
    p.errors = reinterpret_cast<unsigned long long *>(a->error_count);
    return launch_kv8_read(p, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? SPEC_OK : SPEC_EHIP;
}

size_t spec_kv8_attn_workspace_bytes(const spec_kv8_attn_args *a)
{
    if (check_kv8_attn(a) != SPEC_OK) return 0;
    const spec_prefix_attn_args x = as_prefix_args(a);
    return make_plan(&x, false).total;
}

spec_status spec_kv8_attn(const spec_kv8_attn_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const spec_status st = check_kv8_attn(a);
    if (st != SPEC_OK) return st;
    const spec_prefix_attn_args x = as_prefix_args(a);
    return run_attn(&x, workspace, workspace_bytes, hip_stream);
}

size_t spec_prefix_attn_workspace_bytes(const spec_prefix_attn_args *a)
{
    return check_prefix_attn(a) == SPEC_OK ? make_plan(a, false).total : 0;
}

spec_status spec_prefix_attn(const spec_prefix_attn_args *a, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const spec_status st = check_prefix_attn(a);
    if (st != SPEC_OK) return st;
    return run_attn(a, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"

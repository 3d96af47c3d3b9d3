// Causal attention of any number of query rows per request over a paged cache (spec_prompt_attn).
#include "code8.h"
#include "prompt_ops.h"

#include <type_traits>

#ifndef SPEC_PROMPT_PART
#error "compiled once per kind of cache: SPEC_PROMPT_PART is the kind, or 4 for the launch functions"
#endif

namespace specv {

template <int KIND>
hipError_t launch_prompt_kind(const PromptAttnParams &p, hipStream_t stream);

namespace {

// Tokens that the rows of the row block see, and its request's lengths; false: the block has no work.
struct RowBlock {
    int b, row0, q_len, past;   // request, its first packed token row, its rows, its tokens before them
    int row_lo, rows;           // first of the block's fused rows; the request's fused rows
    int seen;                   // tokens that the block's last row sees
    bool last;                  // the request's last rows, which see all its tokens
};

__device__ __forceinline__ int seen_by(int past, int q_len, int rows, int row_lo, int rows_log2, int group, uint32_t inverse)
{
    const int last = min(rows, row_lo + (1 << rows_log2)) - 1;
    return max(past + divide_by_group(last, group, inverse) + 1, 0);
}
__device__ __forceinline__ int chunks_of(int seen, int chunk_tokens) { return max((seen + chunk_tokens - 1) / chunk_tokens, 1); }
__device__ __forceinline__ bool length_fits(int kv_len, int capacity, int max_blocks)
{
    return kv_len >= 0 && kv_len <= capacity && (kv_len + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE <= max_blocks;
}

}  // namespace

#if SPEC_PROMPT_PART < 4

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr float kRescaleSlack = 8.0f;   // the running reference follows the maximum when it is this much behind
constexpr float kLift = 0x1p22f, kLower = 0x1p-22f;   // 8-bit pages: of the sums of weights
constexpr int kStepPages = 4, kStepTokens = kStepPages * SPEC_BLOCK_SIZE;
constexpr int kWaveRows = 32;
constexpr int v_row_bytes(int D) { return D * 2 + 16; }   // token rows of V in LDS (token-major pages)

// The IEEE 754-2019 maximum: no canonicalising multiplication per operand that a matrix instruction made, and a NaN stays one.
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

// The request that owns an item (see row_item): the last one whose first item is not beyond it.  A wavefront asks 64 places at a time.
__device__ __forceinline__ int request_of_rows(const PromptAttnParams &p, int item)
{
    const int lane = threadIdx.x % kWave;
    int lo = 0, n = p.B;
    while (n > 1) {
        const int stride = (n + kWave - 1) / kWave, at = lo + lane * stride;
        const bool begun = lane * stride < n && row_item(p.cu_q_len[min(at, p.B - 1)], at, p.group, p.rows_log2) <= item;
        const int count = max(__builtin_popcountll(__builtin_amdgcn_ballot_w64(begun)), 1);
        lo += (count - 1) * stride;
        n = min(stride, n - (count - 1) * stride);
    }
    return lo;
}

__device__ __forceinline__ size_t packed_row(const PromptAttnParams &p, int row0, int kvh, int r)
{
    const int j = divide_by_group(r, p.group, p.group_inverse);
    return (size_t)(row0 + j) * p.Hq + kvh * p.group + (r - j * p.group);
}

// A block takes 128 or 256 rows of a request and KV head (the group's heads side by side, so that K and V are brought in once for all of them)
// through a chunk of the tokens they see; row blocks that see most go first.  Its four or eight wavefronts have 32 rows each and walk the
// same pages, which pass through LDS once for all, a step (64 tokens) at a time, two buffers, one barrier a step.  In LDS the pages lie as the operands of
// v_mfma_f32_32x32x16 want them, as 16-bit values whatever the cache holds; token-major V by rows, read through the transposing read.
// (lane = 32 half + c; pair: two of the step's pages)
//   S^T[token][row] = K[token][:] . Q[row][:]: a pair, 16 dims an instruction, lane (half, c) holds row c, tokens 4 half + 8 i + 0 .. 3
//   O^T[dim][row] += V^T[dim][token] . P^T[token][row]: a page an instruction, its tokens in that order, so that P goes from one product to the
//   other without leaving its lane
// The two pairs' score products take turns (chains on one accumulator wait for themselves: 16384 tokens 3982 -> 3890 us), operands are read six reads ahead.
//
// What bounds it: one prompt of 16384 tokens, 64/8 heads, d = 128, bf16: 3.8 .. 4.3 ms from card to card, 1.02 .. 1.15 PFLOP/s of visible pairs (a product of two 8192 x 8192 bf16
// matrices 1.31).  Matrix cores are busy 55% of the cycles and vector instructions take 40% more; the two wavefronts of a SIMD are in the same phase
// after each barrier.  The clock is 1.95 GHz under this load and falls further where the phases overlap more (half of the wavefronts half a step
// behind: as many cycles, 4.0 .. 4.35 ms).  A block takes about 5 us to start and to end, which packed prompts of 700 .. 5000 tokens see ten times a
// unit (410 .. 460 us for 389 GFLOP).  Four wavefronts a block bring pages in twice as often (4.27 ms), but are done earlier where there are few.
// Weights of bf16 outputs are one term: a second one of bf16 pages is half as many products again and their conversions, for errors of 1.65e-3 instead of 2.1e-3 of the
// output's norm (16384 tokens 3.9 -> 5.4 ms, packed prompts 428 -> 573 us; for requests of up to 96 rows alone: one token behind 32000 37.7 -> 43 us, 64 of five rows, 64/8 heads, behind
// 2000 128 -> 141, 8 of 1 .. 9 rows behind 2000 .. 30000 103 either way; a batch of both kinds up to a fifth more).  It goes by the types alone, so that a row's
// error does not depend on what else is in the batch.  Those of fp32 outputs are three (8-bit pages: two): 2.6e-7 on Gaussian rows.  Each term's products are added to the sum by
// themselves, the small ones rounded to its steps: with equal weights and a V of one sign up to 3.5e-5 of it after 16384 tokens that are not split.
template <int KIND, int D, int W>
struct PromptShared {
    static constexpr int kK = kStepTokens * D * 2;   // of a step
    static constexpr int kV = kStepTokens * (KIND == kCacheTokens ? v_row_bytes(D) : D * 2);
    static constexpr int kOutRow = D * 2 + 16;       // a bf16 result row, or half an fp32 one
    union {
        struct {
            alignas(16) unsigned char k[2][kK];   // [pair][16 dims][lane][16]
            alignas(16) unsigned char v[2][kV];   // [page][32-dim slice][lane][tokens 4 half .. + 3, 8 + 4 half .. + 3]; token-major: [page][token] rows
        };
        alignas(16) unsigned char o[W][kWaveRows * kOutRow];   // results on their way out
    };
    // 8-bit pages, per token: K's scale with the softmax scale, log2 of V's, its lifted reciprocal
    float scale[is_8bit(KIND) ? 2 : 1][3][is_8bit(KIND) ? kStepTokens : 1];
    int odd[2];   // the last step whose V in this buffer had infinities or NaN
};

template <int KIND, int D, bool FULL, int W>
__global__ __launch_bounds__(W *kWave, D == 64 && !is_8bit(KIND) ? 3 : 2) void prompt_attn_kernel(PromptAttnParams p)
{
    constexpr int kPerPage = W / kStepPages;             // wavefronts that bring in a page
    constexpr bool B8 = is_8bit(KIND), INT8 = KIND == kCacheInt8, TM = KIND == kCacheTokens;
    constexpr int KS = D / 16, SL = D / 32;
    constexpr int kPageBytes = SPEC_BLOCK_SIZE * D * (B8 ? 1 : 2);
    constexpr int N = B8 ? D / 64 : D / 32;              // 1 KB pieces of a page's K, of its V
    constexpr int TERMS = FULL ? (B8 ? 2 : 3) : 1;
    constexpr float kTop = B8 ? 7.0f : 0.0f;             // fp16 weights go up to 2^(7 + slack): their small ones stay normal numbers
    typedef std::conditional_t<B8, f16x8, bf16x8> Weights;
    typedef PromptShared<KIND, D, W> Sh;
    __shared__ Sh sh;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, c32 = lane & 31, n16 = lane & 15, g = lane >> 4;
    const int item = (int)(blockIdx.x / (unsigned)p.Hkv), kvh = (int)blockIdx.x - item * p.Hkv;

    // Offsets that lie outside the rows may be no request's that an item leads to: one block, behind all items, looks at them.
    if (item >= p.items) {
        if (blockIdx.y == 0)
            for (int b = tid; b < p.B; b += W * kWave) {
                const unsigned long long found = __builtin_amdgcn_ballot_w64(!offsets_fit(p.cu_q_len[b], p.cu_q_len[b + 1], p.T));
                if (found != 0 && lane == __builtin_ctzll(found)) atomicAdd(p.errors, (unsigned long long)__builtin_popcountll(found));
            }
        return;
    }

    // the row block and its tokens
    const int b = request_of_rows(p, item);
    const int row0 = uniform_load(p.cu_q_len, b), end = uniform_load(p.cu_q_len, b + 1);
    if (row0 < 0 || end <= row0 || end > p.T) return;
    const int q_len = end - row0, all_rows = q_len * p.group;
    const int blocks = (all_rows + (1 << p.rows_log2) - 1) >> p.rows_log2, which = item - row_item(row0, b, p.group, p.rows_log2);
    if (which < 0 || which >= blocks) return;
    const int kv_len = uniform_load(p.kv_len, b);
    if (!length_fits(kv_len, p.capacity_tokens, p.max_blocks_per_req)) {
        if (which == 0 && kvh == 0 && blockIdx.y == 0 && tid == 0 && p.errors != nullptr) atomicAdd(p.errors, 1ull);
        return;
    }
    const int past = kv_len - q_len, block_lo = (blocks - 1 - which) << p.rows_log2;   // (the rows that see most go first)
    const int seen = seen_by(past, q_len, all_rows, block_lo, p.rows_log2, p.group, p.group_inverse);
    const int chunks = chunks_of(seen, p.chunk_tokens), chunk = blockIdx.y;
    if (chunk >= chunks) return;
    const int all_steps = (seen + kStepTokens - 1) / kStepTokens;
    // (even shares, or whole chunks and what is left)
    const int first_step = p.even ? (int)((int64_t)all_steps * chunk / chunks) : chunk * (p.chunk_tokens / kStepTokens);
    const int steps = (p.even ? (int)((int64_t)all_steps * (chunk + 1) / chunks) : min(first_step + p.chunk_tokens / kStepTokens, all_steps)) - first_step;
    const int tok0 = first_step * kStepTokens, tok1 = min(seen, tok0 + steps * kStepTokens);

    // this wavefront's rows: lane c32 holds row row_lo + c32, which sees the tokens up to `limit`
    const int row_lo = block_lo + wave * kWaveRows, rows = min(max(all_rows - row_lo, 0), kWaveRows);
    const int my_row = rows > 0 ? row_lo + min(c32, rows - 1) : 0;
    const int limit = past + divide_by_group(my_row, p.group, p.group_inverse);
    const int most = __builtin_amdgcn_readfirstlane(rows > 0 ? past + divide_by_group(row_lo + rows - 1, p.group, p.group_inverse) : -1);

    bf16x8 q[KS];
    {
        const int j = divide_by_group(my_row, p.group, p.group_inverse);
        const __bf16 *row = static_cast<const __bf16 *>(p.q) + (size_t)(row0 + j) * p.q_stride + (size_t)(kvh * p.group + (my_row - j * p.group)) * D;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const bf16x8 *>(row + 16 * ks + 8 * half);
    }

    // Block-table entries of the chunk's pages, 64 at a time, a lane each; -1: past the end or outside the pool (reads as zeros).
    const int32_t *table = p.block_table + (size_t)b * p.max_blocks_per_req + tok0 / SPEC_BLOCK_SIZE;
    const int pages = (tok1 - tok0 + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE;
    const bool counts = which == 0 && kvh == 0 && wave == 0;
    auto look_up = [&](int base) {
        int entry = -1;
        bool bad = false;
        if (base + lane < pages) {
            entry = table[base + lane];
            bad = (unsigned)entry >= (unsigned)p.num_blocks;
            if (bad) entry = -1;
        }
        if (counts && p.errors != nullptr) {
            const unsigned long long found = __builtin_amdgcn_ballot_w64(bad);
            if (found != 0 && lane == 0) atomicAdd(p.errors, (unsigned long long)__builtin_popcountll(found));
        }
        return entry;
    };
    // Wavefront w brings in page w of a step (of eight: half of page w / 2).
    static_assert(N % kPerPage == 0, "whole pieces");
    constexpr int PN = N / kPerPage;
    const int my_page = wave / kPerPage, j0 = wave % kPerPage * PN;
    int entries = look_up(0), entries_next = look_up(kWave);
    auto entry_of = [&](int step) {   // asked for step after step
        if (step > 0 && step % (kWave / kStepPages) == 0) {
            entries = entries_next;
            entries_next = look_up(kStepPages * step + kWave);
        }
        return __builtin_amdgcn_readlane(entries, (kStepPages * step + my_page) % kWave);
    };

    const char *khead = static_cast<const char *>(p.k_cache) + (size_t)kvh * kPageBytes;
    const char *vhead = static_cast<const char *>(p.v_cache) + (size_t)kvh * kPageBytes;
    const uint32_t page_stride = (uint32_t)p.Hkv * kPageBytes;
    struct {
        u32x4 k[PN], v[PN];
        float scale;   // 8-bit: the page's record, an entry per lane
    } in;
    auto load = [&](int entry) {
        const uint64_t at = (uint64_t)(uint32_t)entry * page_stride;
        const int bytes = entry < 0 ? 0 : kPageBytes;
        const __amdgpu_buffer_rsrc_t kd = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(khead + at), 0, bytes, kBufferFlags);
        const __amdgpu_buffer_rsrc_t vd = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(vhead + at), 0, bytes, kBufferFlags);
#pragma unroll
        for (int i = 0; i < PN; ++i) {
            in.k[i] = TM ? __builtin_amdgcn_raw_buffer_load_b128(kd, n16 * (D * 2) + g * 16, (j0 + i) * 64, 0)
                         : __builtin_amdgcn_raw_buffer_load_b128(kd, lane * 16, (j0 + i) * 1024, 0);
            in.v[i] = __builtin_amdgcn_raw_buffer_load_b128(vd, lane * 16, (j0 + i) * 1024, 0);
        }
        if constexpr (B8) {
            const __amdgpu_buffer_rsrc_t sd = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<float *>(p.kv_scale + ((uint64_t)(uint32_t)entry * (uint32_t)p.Hkv + kvh) * 32), 0, entry < 0 ? 0 : 128, kBufferFlags);
            in.scale = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sd, c32 * 4, 0, 0));
        }
    };
    // V of the tokens past the end is cleared (those slots may hold anything, and 0 times it has to be 0): `left` tokens are there.
    auto clear_tail = [&](int left) {
        const int n = min(max(left - 4 * g, 0), 4);   // of the lane's four tokens
#pragma unroll
        for (int i = 0; i < PN; ++i) {
            if constexpr (TM) {
                constexpr int LR = D / 8;
                if ((kWave / LR) * (j0 + i) + lane / LR >= left) in.v[i] = (u32x4){0, 0, 0, 0};
            } else if constexpr (B8) {
                const uint32_t mask = n == 4 ? 0xFFFFFFFFu : (1u << 8 * n) - 1u;
#pragma unroll
                for (int e = 0; e < 4; ++e) in.v[i][e] &= mask;
            } else {
                const uint32_t lo = n >= 2 ? 0xFFFFFFFFu : n == 1 ? 0xFFFFu : 0u, hi = n == 4 ? 0xFFFFFFFFu : n == 3 ? 0xFFFFu : 0u;
                in.v[i] = (u32x4){in.v[i][0] & lo, in.v[i][1] & hi, in.v[i][2] & lo, in.v[i][3] & hi};
            }
        }
    };
    // Infinities and NaN in V are cleared too; true: there were some.
    auto clear_odd = [&] {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        u16x2 largest = {0, 0};   // magnitudes order as integers, infinities and NaN last
#pragma unroll
        for (int i = 0; i < PN; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, in.v[i][e] & 0x7FFF7FFFu));
        if (__builtin_amdgcn_ballot_w64(max(largest.x, largest.y) >= 0x7F80) == 0) return false;
#pragma unroll
        for (int i = 0; i < PN; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = in.v[i][e];
                const uint32_t lo = (w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u, hi = (w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u;
                in.v[i][e] = w & ~(lo | hi);
            }
        return true;
    };
    auto store = [&](int buf) {
        unsigned char *ks = sh.k[buf] + (my_page >> 1) * (KS * 1024) + (my_page & 1) * 256, *vs = sh.v[buf];
#pragma unroll
        for (int i = 0; i < PN; ++i) {
            const int j = j0 + i;
            if constexpr (B8) {   // token n16, dims 64 j + 16 g .. + 15; tokens 4 g .. + 3, dims 64 j + 16 e + n16
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x2 a = codes_to_bf16<INT8>(in.k[i][2 * e]), c = codes_to_bf16<INT8>(in.k[i][2 * e + 1]);
                    *reinterpret_cast<u32x4 *>(ks + (4 * j + g) * 1024 + (e * 32 + n16) * 16) = (u32x4){a.x, a.y, c.x, c.y};
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<u32x2 *>(vs + (my_page * SL + 2 * j + e / 2) * 1024 + ((g & 1) * 32 + (e % 2) * 16 + n16) * 16 + (g >> 1) * 8) =
                        codes_to_f16<INT8>(in.v[i][e]);
            } else {              // token n16, dims 32 j + 8 g .. + 7
                *reinterpret_cast<u32x4 *>(ks + (2 * j + (g >> 1)) * 1024 + ((g & 1) * 32 + n16) * 16) = in.k[i];
                if constexpr (TM) {
                    constexpr int LR = D / 8;   // lanes per token row of a 1 KB load
                    *reinterpret_cast<u32x4 *>(vs + (my_page * SPEC_BLOCK_SIZE + (kWave / LR) * j + lane / LR) * v_row_bytes(D) + (lane % LR) * 16) = in.v[i];
                } else {          // tokens 4 g .. + 3, dims 32 j + 16 e + n16
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        *reinterpret_cast<u32x2 *>(vs + (my_page * SL + j) * 1024 + ((g & 1) * 32 + e * 16 + n16) * 16 + (g >> 1) * 8) =
                            (u32x2){in.v[i][2 * e], in.v[i][2 * e + 1]};
                }
            }
        }
        if constexpr (B8) {
            if (lane < 32 && wave % kPerPage == 0) {   // 16 scales of K, 16 of V
                float *to = &sh.scale[buf][0][my_page * 16 + n16];
                if (lane < 16) to[0] = in.scale * p.scale_log2;
                else {   // (a NaN reaches the rows that see the token through its logarithm; the reciprocal, which masked tokens meet as 0 times it, stays finite)
                    to[kStepTokens] = __builtin_amdgcn_logf(__builtin_elementwise_maximum(in.scale, kSmallestScale));
                    to[2 * kStepTokens] = __builtin_amdgcn_rcpf(fmaxf(in.scale, kSmallestScale) * kLower);
                }
            }
        }
    };

    f32x16 acc[SL];
    float m_run = -INFINITY, m_use = 0.0f;     // the reference, and what it is while no key has been seen
    float l_run = 0.0f, l_lost = 0.0f;         // the lane's part of the sum, what its additions have lost
    f32x4 l_step = {0.0f, 0.0f, 0.0f, 0.0f};   // parts of the step's
#pragma unroll
    for (int sl = 0; sl < SL; ++sl)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[sl][e] = 0.0f;

    f32x16 s[2];                 // of the step's pairs of pages
    Weights pw[2][2][TERMS];     // ... and their pages
    // Operands come from LDS kAhead reads ahead of the products that take them.
    constexpr int kAhead = D == 128 ? 6 : 4;
    u32x4 operand[kAhead];
    auto read_k = [&](int buf, int i) { return *reinterpret_cast<const u32x4 *>(sh.k[buf] + (i % 2 * KS + i / 2) * 1024 + lane * 16); };   // pair i % 2, dims 16 (i / 2) ..
    auto read_v = [&](int buf, int i) {   // page i / SL, dims 32 (i % SL) ..
        if constexpr (TM) {
            const unsigned char *src = sh.v[buf] + (i / SL * SPEC_BLOCK_SIZE + 4 * half + (n16 >> 2)) * v_row_bytes(D) + (i % SL * 32 + 16 * (g & 1) + 4 * (n16 & 3)) * 2;
            const u32x2 a = read_transposed(src), c = read_transposed(src + 8 * v_row_bytes(D));
            return (u32x4){a.x, a.y, c.x, c.y};
        } else {
            return *reinterpret_cast<const u32x4 *>(sh.v[buf] + i * 1024 + lane * 16);
        }
    };
    auto multiply = [&](u32x4 v, Weights w, f32x16 c) {
        if constexpr (B8) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, w), c, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, w), c, 0, 0, 0);
    };
    // products of the K in buffer `buf` with the queries
    auto scores = [&](int buf) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[h][e] = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * KS; ++i) {
            s[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, operand[i % kAhead]), q[i / 2], s[i % 2], 0, 0, 0);
            if (i + kAhead < 2 * KS) operand[i % kAhead] = read_k(buf, i + kAhead);
        }
    };
    // scores to base-2 exponents (8-bit; bf16: up to the scale, which the exponent's multiply-add applies), and the running
    // reference raised where it has fallen behind; token 32 h + 8 i + 4 half + r of the step is s[h][4 i + r]
    auto exponents = [&](int buf, int t0, auto masked) {
        if constexpr (B8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f32x4 ks = *reinterpret_cast<const f32x4 *>(&sh.scale[buf][0][8 * i + 4 * half]);
                const f32x4 lv = *reinterpret_cast<const f32x4 *>(&sh.scale[buf][1][8 * i + 4 * half]);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[i / 4][4 * (i % 4) + r] = fmaf(s[i / 4][4 * (i % 4) + r], ks[r], lv[r]);
            }
        }
        if constexpr (masked) {
            const int from = limit - t0 - 4 * half;   // the lane's tokens after this one are hidden
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (8 * i + r > from) s[i / 4][4 * (i % 4) + r] = -INFINITY;
        }
        float mx = max3(s[0][0], s[0][1], s[0][2]), m2 = max3(s[1][0], s[1][1], s[1][2]);
#pragma unroll
        for (int e = 3; e < 15; e += 2) {
            mx = max3(mx, s[0][e], s[0][e + 1]);
            m2 = max3(m2, s[1][e], s[1][e + 1]);
        }
        mx = max3(max3(mx, s[0][15], s[1][15]), m2, m2);
        mx = B8 ? mx - kTop : mx * p.scale_log2;   // (the scale is positive: the maximum commutes with it)
        if (__builtin_amdgcn_ballot_w64(mx > m_run + kRescaleSlack) != 0) {
            mx = max_across_xor32(mx);
            const bool up = mx > m_run + kRescaleSlack;
            const float alpha = up ? fast_exp2(m_run - mx) : 1.0f;
            l_run *= alpha;
            l_lost *= alpha;
#pragma unroll
            for (int sl = 0; sl < SL; ++sl) acc[sl] *= alpha;
            if (up) m_run = m_use = mx;
        }
    };
    // weights of pair h
    auto weigh = [&](int buf, int h) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 rv = {0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (B8) rv = *reinterpret_cast<const f32x4 *>(&sh.scale[buf][2][32 * h + 8 * i + 4 * half]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = s[h][4 * i + r];
                const float e = fast_exp2(B8 ? x - m_use : fmaf(x, p.scale_log2, -m_use));
                if constexpr (B8) l_step[r] = h + i > 0 ? fmaf(e, rv[r], l_step[r]) : e * rv[r];
                else l_step[r] = h + i > 0 ? l_step[r] + e : e;
                float rest = e;
#pragma unroll
                for (int t = 0; t < TERMS; ++t) {
                    pw[h][i / 2][t][4 * (i % 2) + r] = (std::conditional_t<B8, _Float16, __bf16>)rest;
                    if (t + 1 < TERMS) rest -= (float)pw[h][i / 2][t][4 * (i % 2) + r];
                }
            }
        }
        if (h == 1) {   // a step's weights in a few levels, and steps with what each addition loses: thousands of equal ones would lose the same each time
            const float add = ((l_step[0] + l_step[1]) + (l_step[2] + l_step[3])) - l_lost, next = l_run + add;
            l_lost = (next - l_run) - add;
            l_run = next;
        }
    };
    // product of pair h's weights with its V in buffer `buf`
    auto product = [&](int buf, int h) {
#pragma unroll
        for (int k = 0; k < 2 * SL; ++k) {
            const int i = 2 * SL * h + k;
            const u32x4 v = operand[i % kAhead];
#pragma unroll
            for (int t = 0; t < TERMS; ++t) acc[k % SL] = multiply(v, pw[h][k / SL][t], acc[k % SL]);
            if (i + kAhead < 4 * SL) operand[i % kAhead] = read_v(buf, i + kAhead);
        }
    };
    // bf16 pages, a step that some rows do not see whole: an infinity or NaN in V would reach those as 0 times it; and weights in several terms, some of them zero or
    // negative, would make NaN of an infinity.  Such values are cleared on their way to LDS (see `clear_odd`), and the rows that see them get them here, from memory.
    auto add_odd = [&](int t0) __attribute__((always_inline)) {
#pragma unroll 1
        for (int i = 0; i < min(kStepTokens, tok1 - t0); ++i) {
            const int entry = uniform_load(table, (t0 - tok0 + i) / SPEC_BLOCK_SIZE);
            if ((unsigned)entry >= (unsigned)p.num_blocks) continue;
            const __bf16 *from = reinterpret_cast<const __bf16 *>(vhead + (uint64_t)(uint32_t)entry * page_stride);
            const int slot = i % SPEC_BLOCK_SIZE;
#pragma unroll
            for (int sl = 0; sl < SL; ++sl)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int c = 8 * (e / 4) + 4 * half + e % 4;   // of the 32 dims
                    const float v = (float)from[TM ? slot * D + 32 * sl + c : (((sl * 4 + slot / 4) * 16 + c % 16) * 2 + c / 16) * 4 + slot % 4];
                    if (!(fabsf(v) < INFINITY) && t0 + i <= limit) acc[sl][e] += v;
                    if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (rare: no registers of the steps for it)
                }
        }
    };

    const int seen_whole = max(past + divide_by_group(block_lo, p.group, p.group_inverse) + 1 - tok0, 0) / kStepTokens;   // steps that all rows see whole
    auto bring = [&](int step, int buf) {   // what was loaded for `step` goes to LDS
        const int left = tok1 - tok0 - step * kStepTokens - my_page * SPEC_BLOCK_SIZE;
        if (left < SPEC_BLOCK_SIZE) clear_tail(left);
        if constexpr (!B8)
            if ((FULL || step >= seen_whole) && clear_odd()) sh.odd[buf] = step;
        store(buf);
    };
    auto walk = [&](int u, auto masked) __attribute__((always_inline)) {
        const int buf = u & 1, t0 = tok0 + u * kStepTokens;
        __syncthreads();        // step u is in LDS, and no wavefront reads step u - 1 any more
        const bool active = masked ? t0 <= most : rows > 0;
        const bool odd = !B8 && (masked || FULL) && sh.odd[buf] == u;
        if (active) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) operand[i] = read_k(buf, i);
        }
        bring(u + 1, buf ^ 1);
        load(entry_of(u + 2));
        if (!active) return;
        scores(buf);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) operand[i] = read_v(buf, i);
        exponents(buf, t0, masked);
        weigh(buf, 0);
        product(buf, 0);
        weigh(buf, 1);
        product(buf, 1);
        if constexpr ((masked || FULL) && !B8)
            if (odd) add_odd(t0);
    };
    if (tid < 2) sh.odd[tid] = -1;
    __syncthreads();
    load(entry_of(0));
    bring(0, 0);
    load(entry_of(1));
    int u = 0;
    for (; u < min(steps, seen_whole); ++u) walk(u, std::false_type{});
    for (; u < steps; ++u) walk(u, std::true_type{});

    // Results, and partial results where the tokens are split, go through LDS so that they go out in long pieces.  (Which lane
    // this is, is found again: no registers for that in the steps.)
    int end_tid = threadIdx.x;
    asm volatile("" : "+v"(end_tid));
    const int end_lane = end_tid & 63, end_half = end_lane >> 5, end_c32 = end_lane & 31;
    l_run -= l_lost;
    l_run += __uint_as_float(__builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false)[end_half ^ 1]);
    const bool whole = chunks == 1;
    const size_t my_index = packed_row(p, row0, kvh, my_row);
    if (end_half == 0 && end_c32 < rows) {
        if (!whole) *reinterpret_cast<f32x2 *>(p.ml + (my_index * p.max_chunks + chunk) * 2) = (f32x2){m_run, l_run};
        else if (p.lse != nullptr) p.lse[my_index] = l_run == 0.0f ? -INFINITY : (m_run + __builtin_amdgcn_logf(B8 ? l_run * kLower : l_run)) * kLn2;
    }
    if (whole) {
        const float inv = limit < 0 ? 0.0f : (B8 ? kLift : 1.0f) / l_run;   // (a row that sees no key is zero)
#pragma unroll
        for (int sl = 0; sl < SL; ++sl) acc[sl] *= inv;
    }
    __syncthreads();
    unsigned char *o = sh.o[wave];
    auto lds_order = [] {   // (a region for each wavefront, and LDS executes a wavefront's accesses in order)
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    constexpr int OP = D / 8;   // 16-byte pieces of a bf16 row, or of half an fp32 row
    if (FULL || !whole) {
#pragma unroll
        for (int d2 = 0; d2 < 2; ++d2) {
#pragma unroll
            for (int sl = 0; sl < SL / 2; ++sl)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x16 &x = acc[d2 * (SL / 2) + sl];
                    *reinterpret_cast<f32x4 *>(o + end_c32 * Sh::kOutRow + (32 * sl + 8 * i + 4 * end_half) * 4) = (f32x4){x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
                }
            lds_order();
#pragma unroll
            for (int piece = end_lane; piece < kWaveRows * OP; piece += kWave) {
                const int r = piece / OP, c = piece % OP;
                if (r < rows) {
                    const size_t index = packed_row(p, row0, kvh, row_lo + r);
                    float *to = whole ? static_cast<float *>(p.out) + index * D : p.acc + (index * p.max_chunks + chunk) * D;
                    *reinterpret_cast<u32x4 *>(to + d2 * (D / 2) + c * 4) = *reinterpret_cast<const u32x4 *>(o + r * Sh::kOutRow + c * 16);
                }
            }
            lds_order();
        }
    } else {
#pragma unroll
        for (int sl = 0; sl < SL; ++sl)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x16 &x = acc[sl];
                const f32x4 four = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
                *reinterpret_cast<u32x2 *>(o + end_c32 * Sh::kOutRow + (32 * sl + 8 * i + 4 * end_half) * 2) = __builtin_bit_cast(u32x2, __builtin_convertvector(four, bf16x4));
            }
        lds_order();
#pragma unroll
        for (int piece = end_lane; piece < kWaveRows * OP; piece += kWave) {
            const int r = piece / OP, c = piece % OP;
            if (r < rows)
                *reinterpret_cast<u32x4 *>(static_cast<__bf16 *>(p.out) + packed_row(p, row0, kvh, row_lo + r) * D + c * 8) =
                    *reinterpret_cast<const u32x4 *>(o + r * Sh::kOutRow + c * 16);
        }
    }
}

template <int KIND, int D, bool FULL>
hipError_t go(const PromptAttnParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)p.items * (unsigned)p.Hkv + (p.errors != nullptr ? 1u : 0u), (unsigned)p.max_chunks);
    if constexpr (D == 128) {
        if (p.rows_log2 == 8) {
            hipLaunchKernelGGL((prompt_attn_kernel<KIND, D, FULL, 8>), grid, dim3(8 * kWave), 0, stream, p);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((prompt_attn_kernel<KIND, D, FULL, 4>), grid, dim3(4 * kWave), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

template <>
hipError_t launch_prompt_kind<SPEC_PROMPT_PART>(const PromptAttnParams &p, hipStream_t stream)
{
    if (p.d == 128) return p.out_f32 ? go<SPEC_PROMPT_PART, 128, true>(p, stream) : go<SPEC_PROMPT_PART, 128, false>(p, stream);
    return p.out_f32 ? go<SPEC_PROMPT_PART, 64, true>(p, stream) : go<SPEC_PROMPT_PART, 64, false>(p, stream);
}

#else

namespace {

// Joins the partial results of the rows whose tokens are split: four rows a wavefront, 16 lanes and D / 16 dims a lane each.  A lane looks at every
// 16th chunk's reference and sum; the chunks' factors go round through LDS, and four chunks' results are asked for at a time.  (A
// wavefront per row took 10 us and more where rows are few, five dependent latencies of which little ran at once.)
template <int D>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptAttnParams p)
{
    constexpr int N = D / 16, kRows = 4;
    __shared__ float factors[4][kRows][kMostPromptChunks];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, sub = lane / 16, at = lane % 16;
    const int64_t all = (int64_t)p.T * p.Hq, index = ((int64_t)blockIdx.x * 4 + wave) * kRows + sub;
    const int row = (int)(min(index, all - 1) / p.Hq), head = (int)(min(index, all - 1) - (int64_t)row * p.Hq);
    const int b = request_of(p.cu_q_len, p.B, row, (int)((int64_t)row * p.B / p.T));
    const int row0 = p.cu_q_len[b], end = p.cu_q_len[b + 1], kv_len = p.kv_len[b];
    int chunks = 0;
    if (index < all && row0 >= 0 && row >= row0 && end > row && end <= p.T && length_fits(kv_len, p.capacity_tokens, p.max_blocks_per_req)) {
        const int r = (row - row0) * p.group + head % p.group;
        const int seen = seen_by(kv_len - (end - row0), end - row0, (end - row0) * p.group, r >> p.rows_log2 << p.rows_log2, p.rows_log2, p.group, p.group_inverse);
        chunks = chunks_of(seen, p.chunk_tokens);
        if (chunks == 1 || chunks > p.max_chunks) chunks = 0;   // (a single chunk's results are in place)
    }
    if (__builtin_amdgcn_ballot_w64(chunks > 0) == 0) return;

    constexpr int kEach = kMostPromptChunks / 16;
    f32x2 mine[kEach];
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        mine[i] = (f32x2){-INFINITY, 0.0f};
        if (at + 16 * i < chunks) mine[i] = *reinterpret_cast<const f32x2 *>(p.ml + (index * p.max_chunks + at + 16 * i) * 2);
        top = fmaxf(top, mine[i].x);
    }
#pragma unroll
    for (int step = 1; step < 16; step *= 2) top = fmaxf(top, __shfl_xor(top, step));
    float l = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        // a chunk in which the row sees nothing, or nothing but scores of -infinity, has no part; one whose sum is NaN has
        const bool none = mine[i].x == -INFINITY;
        const float factor = none ? (mine[i].y == 0.0f ? 0.0f : 1.0f) : fast_exp2(mine[i].x - top);
        l += none ? mine[i].y : mine[i].y * factor;
        factors[wave][sub][at + 16 * i] = factor;
    }
#pragma unroll
    for (int step = 1; step < 16; step *= 2) l += __shfl_xor(l, step);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if (chunks == 0) return;
    f32x4 sum[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) sum[i] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    const float *from = p.acc + index * p.max_chunks * D + at * 4;
    constexpr int kAtOnce = 4;
    for (int c = 0; c < chunks; c += kAtOnce) {
        f32x4 x[kAtOnce][N / 4];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
            for (int i = 0; i < N / 4; ++i) x[k][i] = *reinterpret_cast<const f32x4 *>(from + (size_t)min(c + k, chunks - 1) * D + i * 64);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const bool there = c + k < chunks;   // (a factor of zero counts: an infinity or NaN of tokens with weights below fp32's range is not lost)
            const float w = factors[wave][sub][c + k];
#pragma unroll
            for (int i = 0; i < N / 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[i][e] = fmaf(w, there ? x[k][i][e] : 0.0f, sum[i][e]);
        }
    }
    const bool b8 = is_8bit(p.kind);
    const float inv = kv_len - end + row < 0 ? 0.0f : (b8 ? 0x1p22f : 1.0f) / l;
    if (at == 0 && p.lse != nullptr) p.lse[index] = l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(b8 ? l * 0x1p-22f : l)) * kLn2;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const f32x4 o = sum[i] * inv;
        if (p.out_f32) *reinterpret_cast<f32x4 *>(static_cast<float *>(p.out) + index * D + at * 4 + i * 64) = o;
        else *reinterpret_cast<u32x2 *>(static_cast<__bf16 *>(p.out) + index * D + at * 4 + i * 64) = __builtin_bit_cast(u32x2, __builtin_convertvector(o, bf16x4));
    }
}

}  // namespace

hipError_t launch_prompt_attn(const PromptAttnParams &p, hipStream_t stream)
{
    hipError_t e;
    switch (p.kind) {
    case kCacheTiles: e = launch_prompt_kind<kCacheTiles>(p, stream); break;
    case kCacheTokens: e = launch_prompt_kind<kCacheTokens>(p, stream); break;
    case kCacheE4M3: e = launch_prompt_kind<kCacheE4M3>(p, stream); break;
    default: e = launch_prompt_kind<kCacheInt8>(p, stream); break;
    }
    if (e != hipSuccess || p.max_chunks == 1) return e;
    const dim3 grid((unsigned)(((int64_t)p.T * p.Hq + 15) / 16));
    if (p.d == 128) hipLaunchKernelGGL((prompt_join_kernel<128>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((prompt_join_kernel<64>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

#endif

}  // namespace specv

// Attention over a paged cache of bf16 or 8-bit pages for the query rows of single requests or of groups of
// requests that share a prefix (spec_kv8_attn, spec_prefix_attn).
//
// Arithmetic, per pair of 16-token pages and 16-row tile (lane = 16 g + n):
//   S^T[token][row] = K[token][:] . Q[row][:]             v_mfma_f32_16x16x32_bf16, a page each
//   base-2 online softmax on the lane's tokens 4 g .. + 3 of both pages, query row n
//   O^T[dim][row] += V^T[dim][token] . P^T[token][row]    16x16x32, both pages' tokens in one contraction; P^T is
//   S^T's own accumulator layout
// 8-bit pages: K's codes become bf16 and V's fp16, both exactly.  With the scales k_t and v_t of token t
//   x_t = (q . K_t) k_t softmax_scale log2 e,   y_t = x_t + log2 v_t,   w_t = 2^(y_t - m),  m: running maximum of y
//   O = sum w_t V_t,   l = sum w_t / v_t
// so that the weights of the product are at most one whatever the scales are, and V's scale costs an addition in
// the exponent; they fit fp16, whose 11 bits keep their rounding (2^-12) below that of a bf16 output.
#include "code8.h"

#include <math.h>

#include <type_traits>

#ifndef SPEC_CACHE_PART
#error "compiled once per kind of cache: SPEC_CACHE_PART is the kind, or 4 for the launch functions"
#endif

namespace specv {

// Variants are chosen by (row tiles, head dim, weights in more than one term); one set per kind of cache.
struct CacheLaunch {
    unsigned blocks;
    int prefix;   // which of the two launches
};
template <int KIND>
hipError_t launch_cache_kind(const CacheAttnParams &p, int tiles, bool full, CacheLaunch at, hipStream_t stream);

#if SPEC_CACHE_PART < 4

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr float kRescaleSlack = 8.0f;   // the running reference follows the maximum when it is this much behind

constexpr int v_row_bytes(int D) { return D * 2 + 16; }   // token rows of V in LDS (token-major pages)
constexpr int o_row_bytes(int D) { return D * 4 + 16; }   // result rows in LDS

template <int KIND, int D>
struct Pair {   // two pages
    static constexpr int N = is_8bit(KIND) ? D / 64 : D / 32;   // 1 KB loads of K, of V
    u32x4 k[2][N], v[2][N];
    f32x4 ks[is_8bit(KIND) ? 2 : 1], vs[is_8bit(KIND) ? 2 : 1];
};

template <int KIND, int NT, int D>
struct Shared {
    union {
        unsigned char v[KIND == kCacheTokens ? kWaves : 1][KIND == kCacheTokens ? 2 * SPEC_BLOCK_SIZE * v_row_bytes(D) : 16];
        f32x4 acc[2][NT][D / 16][kWave];                 // results of the wavefronts being merged
        unsigned char o[NT * 16 * o_row_bytes(D)];       // the block's result, by rows
    };
    float m[2][NT][kWave], l[2][NT][kWave];
    float row_m[NT * 16], row_l[NT * 16];
    int last;
};

// The block's place in the work.
struct Work {
    int b;             // request whose block-table row says where the pages are
    int kvh, chunk, nchunks;
    int row0, rows;    // first packed token row, fused query rows from there on
    int row_lo;        // first of them that is this block's
    int tok0, tok1;    // its tokens
    int hide_from;     // row r of the block's rows sees tokens < hide_from + r / group; all of them: INT_MAX
    int group_index, prefix_chunks;   // partial results that come in from the prefix launch
    int row_block;
};

__device__ __forceinline__ void count_error(const CacheAttnParams &p, bool first)
{
    if (first && threadIdx.x == 0 && p.errors != nullptr) atomicAdd(p.errors, 1ull);
}

// Group of request b: the number of groups that end at or before it.
__device__ __forceinline__ int group_of(const CacheAttnParams &p, int b)
{
    const int lane = threadIdx.x % kWave;
    int g = 0;
    for (int base = 0; base < p.G; base += kWave) {
        const bool before = base + lane < p.G && p.cu_group[base + lane + 1] <= b;
        const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(before));
        g += n;
        if (n < kWave) break;
    }
    return min(g, p.G - 1);
}

__device__ __forceinline__ bool prefix_ok(const CacheAttnParams &p, int len)
{
    return len >= 0 && len <= p.prefix_capacity && len % SPEC_BLOCK_SIZE == 0 && len / SPEC_BLOCK_SIZE <= p.max_blocks_per_req;
}

__device__ __forceinline__ int chunk_count(int tokens, int chunk_tokens) { return (tokens + chunk_tokens - 1) / chunk_tokens; }

// One block of the own launch.  Items: chunk-major, then row blocks, requests, KV heads innermost.
template <int NT>
__device__ __forceinline__ bool place_own(const CacheAttnParams &p, int item, Work &w)
{
    w.kvh = item % p.Hkv;
    item /= p.Hkv;
    w.b = item % p.B;
    item /= p.B;
    w.row_block = item % p.row_blocks;
    w.chunk = item / p.row_blocks;
    const int L = uniform_load(p.kv_len, w.b);
    w.row0 = uniform_load(p.cu_q_len, w.b);
    const int q_len = uniform_load(p.cu_q_len, w.b + 1) - w.row0;
    if (q_len == 0) return false;   // a padded slot
    const bool first = w.chunk == 0 && w.kvh == 0 && w.row_block == 0;
    int P = 0;
    w.group_index = 0;
    if (p.G > 0) {
        w.group_index = group_of(p, w.b);
        P = uniform_load(p.prefix_len, w.group_index);
    }
    // The lengths come from device memory and bound every loop and index below: a request whose lengths do not fit
    // the launch is left out and reported.
    if (q_len < 0 || q_len > SPEC_K_MAX + 1 || w.row0 < 0 || w.row0 + q_len > p.T || q_len * p.group > p.max_q_rows || L < 0 ||
        L > p.capacity_tokens || (L + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE > p.max_blocks_per_req || !prefix_ok(p, P) ||
        (P > 0 && L - q_len < P)) {
        count_error(p, first);
        return false;
    }
    w.rows = q_len * p.group;
    w.row_lo = w.row_block * (NT * 16);
    if (w.row_lo >= w.rows) return false;
    w.prefix_chunks = P > 0 ? chunk_count(P, p.prefix_chunk_tokens) : 0;
    // even chunks per request, page aligned; a request without tokens has one that is empty
    const int tokens = L - P;
    w.nchunks = max(min(chunk_count(tokens, p.chunk_tokens), p.max_chunks), 1);
    if (w.chunk >= w.nchunks) return false;
    const int C = ((tokens + w.nchunks - 1) / w.nchunks + SPEC_BLOCK_SIZE - 1) & ~(SPEC_BLOCK_SIZE - 1);
    if (C > kMaxChunkTokens) {   // (a prefix that is shorter on the device than planned for)
        count_error(p, first);
        return false;
    }
    w.tok0 = min(P + w.chunk * C, L);
    w.tok1 = min(w.tok0 + C, L);
    w.hide_from = L - q_len + 1;
    return true;
}

// One block of the prefix launch.  Items: chunk-major, then row blocks of all groups, KV heads innermost.
template <int NT>
__device__ __forceinline__ bool place_prefix(const CacheAttnParams &p, int item, Work &w)
{
    w.kvh = item % p.Hkv;
    item /= p.Hkv;
    const int block = item % p.prefix_row_blocks;
    w.chunk = item / p.prefix_row_blocks;
    // the group that holds row block `block`: a lane counts the blocks of a group, 64 groups at a time
    const int lane = threadIdx.x % kWave;
    int before = 0, g = -1;
    for (int base = 0; base < p.G && g < 0; base += kWave) {
        int n = 0;
        if (base + lane < p.G) {
            const int b0 = p.cu_group[base + lane], b1 = p.cu_group[base + lane + 1];
            if (b0 >= 0 && b0 <= b1 && b1 <= p.B) {
                const int rows = (p.cu_q_len[b1] - p.cu_q_len[b0]) * p.group;
                n = rows > 0 ? (rows + NT * 16 - 1) / (NT * 16) : 0;
            }
        }
        int sum = n;   // inclusive prefix sum over the lanes
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const int up = __shfl_up(sum, off);
            if (lane >= off) sum += up;
        }
        const unsigned long long holds = __builtin_amdgcn_ballot_w64(before + sum > block);
        if (holds != 0) {
            const int at = __builtin_ctzll(holds);
            g = base + at;
            w.row_block = block - before - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(n, at));
        } else {
            before += __builtin_amdgcn_readlane(sum, kWave - 1);
        }
    }
    if (g < 0) return false;
    w.group_index = g;
    w.row_block = __builtin_amdgcn_readfirstlane(w.row_block);
    const int P = uniform_load(p.prefix_len, g);
    const int b0 = uniform_load(p.cu_group, g), b1 = uniform_load(p.cu_group, g + 1);
    w.b = b0;
    w.row0 = uniform_load(p.cu_q_len, b0);
    const int tokens = uniform_load(p.cu_q_len, b1) - w.row0;
    if (!prefix_ok(p, P) || P == 0 || w.row0 < 0 || tokens < 0 || w.row0 + tokens > p.T) return false;   // (counted by the own launch)
    w.rows = tokens * p.group;
    w.row_lo = w.row_block * (NT * 16);
    if (w.row_lo >= w.rows) return false;
    w.nchunks = chunk_count(P, p.prefix_chunk_tokens);
    if (w.chunk >= w.nchunks) return false;
    const int C = ((P + w.nchunks - 1) / w.nchunks + SPEC_BLOCK_SIZE - 1) & ~(SPEC_BLOCK_SIZE - 1);
    w.tok0 = min(w.chunk * C, P);
    w.tok1 = min(w.tok0 + C, P);
    w.hide_from = 0x7FFFFFFF - SPEC_K_MAX - 1;
    w.prefix_chunks = 0;
    return true;
}

// Weighted sum of the partial results of a row, four head dims per thread.
struct RowSum {
    float m = kEmptyMax, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    __device__ __forceinline__ void add(float pm, float pl, f32x4 po)
    {
        const float mn = fmaxf(m, pm);
        const float keep = fast_exp2(m - mn), take = fast_exp2(pm - mn);
        l = l * keep + pl * take;
        o = o * keep + po * take;
        m = mn;
    }
};

template <int D>
__device__ __forceinline__ void add_prefix(const CacheAttnParams &p, RowSum &sum, size_t rh, int chunks, int dim)
{
    for (int c = 0; c < chunks; ++c) {
        const size_t slot = rh * p.max_prefix_chunks + c;
        const f32x2 ml = *reinterpret_cast<const f32x2 *>(p.prefix_ml + slot * 2);
        sum.add(ml.x, ml.y, *reinterpret_cast<const f32x4 *>(p.prefix_acc + slot * D + dim));
    }
}

template <int D>
__device__ __forceinline__ void write_row(const CacheAttnParams &p, size_t rh, int dim, const RowSum &sum)
{
    const float inv = sum.l == 0.0f ? 0.0f : 1.0f / sum.l;   // (a row that has seen no key is zero)
    const f32x4 o = sum.o * inv;
    if (p.out_f32)
        __builtin_nontemporal_store(o, reinterpret_cast<f32x4 *>(static_cast<float *>(p.out) + rh * D + dim));
    else
        __builtin_nontemporal_store(__builtin_bit_cast(u32x2, __builtin_convertvector(o, bf16x4)),
                                    reinterpret_cast<u32x2 *>(static_cast<__bf16 *>(p.out) + rh * D + dim));
}

template <int KIND, int NT, int D, bool FULL>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_kernel(CacheAttnParams p, int prefix)
{
    constexpr bool B8 = is_8bit(KIND), INT8 = KIND == kCacheInt8, TM = KIND == kCacheTokens;
    constexpr int KK = D / 32, MT = D / 16;
    constexpr int kPageBytes = SPEC_BLOCK_SIZE * D * (B8 ? 1 : 2);   // of one KV head
    constexpr int TERMS = FULL ? (B8 ? 2 : 3) : 1;   // 16-bit terms of a softmax weight: 22 bits of fp16's, 24 of bf16's
    constexpr float kTop = B8 ? 7.0f : 0.0f;         // fp16 weights go up to 2^(7 + slack): their small ones stay normal numbers
    typedef std::conditional_t<B8, f16x8, bf16x8> Weights;
    __shared__ Shared<KIND, NT, D> sh;

    Work w;
    if (!(prefix ? place_prefix<NT>(p, blockIdx.x, w) : place_own<NT>(p, blockIdx.x, w))) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n16 = lane & 15, g = lane >> 4;
    const int rows = min(w.rows - w.row_lo, NT * 16);   // this block's
    auto out_index = [&](int r) {   // packed (token row, query head) of the block's row r
        const int rr = w.row_lo + r;
        return (size_t)(w.row0 + rr / p.group) * p.Hq + w.kvh * p.group + rr % p.group;
    };

    // block-table entries of this wavefront's pages: pairs wave, wave + 4, ...; lane 2 i + h holds page h of its pair i
    const int npages = (w.tok1 - w.tok0 + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE;   // <= 64 * kWaves
    const int mine = 2 * (wave + kWaves * (lane >> 1)) + (lane & 1);
    int bt = -1;
    {
        const bool used = mine < npages;
        if (used) bt = p.block_table[(size_t)w.b * p.max_blocks_per_req + w.tok0 / SPEC_BLOCK_SIZE + mine];
        const bool bad = used && (unsigned)bt >= (unsigned)p.num_blocks;   // never turned into an address: reads as zeros
        if (bad) bt = -1;
        const unsigned long long bad_lanes = __builtin_amdgcn_ballot_w64(bad);
        if (bad_lanes != 0 && w.kvh == 0 && w.row_block == 0 && lane == 0 && p.errors != nullptr)
            atomicAdd(p.errors, (unsigned long long)__builtin_popcountll(bad_lanes));
    }
    const int npairs = (npages + 1) / 2;
    const int my_pairs = npairs > wave ? (npairs - wave + kWaves - 1) / kWaves : 0;

    // Q as the B operand of S^T = K Q^T: lane (g, n) holds row n, the 8 dims that the lane's K holds (token-major and tiled
    // bf16 pages: 32 kk + 8 g ..; 8-bit pages, 16 bytes of which are two operands: 64 (kk / 2) + 16 g + 8 (kk % 2) ..)
    bf16x8 q[NT][KK];
    int limit[NT];   // last token that the lane's row sees
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 16 + n16;
        const bool on = r < rows;
        const int rr = w.row_lo + (on ? r : 0);
        limit[nt] = on ? w.hide_from - 1 + (prefix ? 0 : rr / p.group) : -1;
        const __bf16 *row = static_cast<const __bf16 *>(p.q) + (size_t)(w.row0 + rr / p.group) * p.q_stride + (size_t)(w.kvh * p.group + rr % p.group) * D;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
            q[nt][kk] = *reinterpret_cast<const bf16x8 *>(row + (B8 ? 64 * (kk / 2) + 16 * g + 8 * (kk % 2) : 32 * kk + 8 * g));
    }

    // Pages are read through descriptors that cover exactly one (page, KV head); a page that is not there has length 0,
    // for which the hardware returns zeros without touching memory.
    const char *khead = static_cast<const char *>(p.k_cache) + (size_t)w.kvh * kPageBytes;
    const char *vhead = static_cast<const char *>(p.v_cache) + (size_t)w.kvh * kPageBytes;
    const size_t page_stride = (size_t)p.Hkv * kPageBytes;
    auto load = [&](int i, Pair<KIND, D> &r) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int entry = __builtin_amdgcn_readlane(bt, i < my_pairs ? 2 * i + h : 0);
            const bool valid = i < my_pairs && entry >= 0;
            const size_t page = (size_t)(valid ? entry : 0);
            const int bytes = valid ? kPageBytes : 0;
            const __amdgpu_buffer_rsrc_t kd = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(khead + page * page_stride), 0, bytes, kBufferFlags);
            const __amdgpu_buffer_rsrc_t vd = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(vhead + page * page_stride), 0, bytes, kBufferFlags);
#pragma unroll
            for (int j = 0; j < Pair<KIND, D>::N; ++j)
                r.k[h][j] = TM ? __builtin_amdgcn_raw_buffer_load_b128(kd, n16 * (D * 2) + g * 16, j * 64, 0)
                               : __builtin_amdgcn_raw_buffer_load_b128(kd, lane * 16, j * 1024, kStreamPolicy);
#pragma unroll
            for (int j = 0; j < Pair<KIND, D>::N; ++j) r.v[h][j] = __builtin_amdgcn_raw_buffer_load_b128(vd, lane * 16, j * 1024, kStreamPolicy);
            if constexpr (B8) {
                const __amdgpu_buffer_rsrc_t sd = __builtin_amdgcn_make_buffer_rsrc(
                    const_cast<float *>(p.kv_scale + (page * p.Hkv + w.kvh) * 32), 0, valid ? 128 : 0, kBufferFlags);
                r.ks[h] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(sd, g * 16, 0, 0));
                r.vs[h] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(sd, g * 16, 64, 0));
            }
        }
    };

    f32x4 acc[NT][MT];
    float m_run[NT], l_run[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m_run[nt] = kEmptyMax;
        l_run[nt] = 0.0f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    }

    auto consume = [&](Pair<KIND, D> &cur, int i) {
        const int first = w.tok0 + 2 * (wave + kWaves * i) * SPEC_BLOCK_SIZE;
        const bool need_mask = first + 2 * SPEC_BLOCK_SIZE > min(w.tok1, w.hide_from);
        // scores
        f32x4 s[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 a;
                if constexpr (B8) {
                    const u32x2 lo = codes_to_bf16<INT8>(cur.k[h][kk / 2][2 * (kk % 2)]), hi = codes_to_bf16<INT8>(cur.k[h][kk / 2][2 * (kk % 2) + 1]);
                    a = (u32x4){lo.x, lo.y, hi.x, hi.y};
                } else {
                    a = cur.k[h][kk];
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    s[nt][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), q[nt][kk], s[nt][h], 0, 0, 0);
            }
        }
        // to base-2 exponents; per token: k = scale of x, lv = log2 of V's scale, rv = its reciprocal
        f32x4 ks[2], lv[2], rv[2];
        if constexpr (B8) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float v = cur.vs[h][r] < kSmallestScale ? kSmallestScale : cur.vs[h][r];   // (a page that reads as zeros)
                    ks[h][r] = cur.ks[h][r] * p.scale_log2;
                    lv[h][r] = __builtin_amdgcn_logf(v);
                    rv[h][r] = __builtin_amdgcn_rcpf(v);
                }
        }
        Weights pw[NT][TERMS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mx = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[nt][h][r] = B8 ? fmaf(s[nt][h][r], ks[h][r], lv[h][r]) : s[nt][h][r] * p.scale_log2;
                    if (need_mask && first + h * SPEC_BLOCK_SIZE + 4 * g + r > min(limit[nt], w.tok1 - 1)) s[nt][h][r] = -INFINITY;
                    mx = fmaxf(mx, s[nt][h][r]);
                }
            }
            mx -= kTop;
            const float most = m_run[nt] + kRescaleSlack;
            if (__builtin_amdgcn_ballot_w64(mx > most) != 0) {
                mx = max_across_xor32(max_across_xor16(mx));
                const float m_new = mx > most ? mx : m_run[nt];
                const float alpha = fast_exp2(m_run[nt] - m_new);
                l_run[nt] *= alpha;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) acc[nt][mt] *= alpha;
                m_run[nt] = m_new;
            }
            float sum = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = fast_exp2(s[nt][h][r] - m_run[nt]);
                    float part = e;
                    if constexpr (B8) {
                        part = e * rv[h][r];
                        if (need_mask && first + h * SPEC_BLOCK_SIZE + 4 * g + r > min(limit[nt], w.tok1 - 1)) part = 0.0f;
                    }
                    sum += part;
                    float rest = e;
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) {
                        pw[nt][t][4 * h + r] = (std::conditional_t<B8, _Float16, __bf16>)rest;
                        rest -= (float)pw[nt][t][4 * h + r];
                    }
                }
            }
            l_run[nt] += sum;
        }

        // V's operands: v[mt] holds dim 16 mt + n of the first page's tokens 4 g .. + 3, then of the second's
        u32x4 v[MT];
        if constexpr (TM) {
            // through this wavefront's LDS region: token rows in, operand order out (LDS executes a wavefront's
            // accesses in order, so the reads see the writes without a barrier)
            unsigned char *st = sh.v[wave];
            constexpr int LR = D / 8;   // lanes per token row of a 1 KB load
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < KK; ++j)
                    *reinterpret_cast<u32x4 *>(st + (h * SPEC_BLOCK_SIZE + (kWave / LR) * j + lane / LR) * v_row_bytes(D) + (lane % LR) * 16) = cur.v[h][j];
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const unsigned char *src = st + (4 * g + (n16 >> 2)) * v_row_bytes(D) + (n16 & 3) * 8 + mt * 32;
                const u32x2 v0 = read_transposed(src), v1 = read_transposed(src + SPEC_BLOCK_SIZE * v_row_bytes(D));
                v[mt] = (u32x4){v0.x, v0.y, v1.x, v1.y};
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        } else if constexpr (KIND == kCacheTiles) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const u32x4 a = cur.v[0][mt / 2], b = cur.v[1][mt / 2];
                v[mt] = (mt & 1) ? (u32x4){a.z, a.w, b.z, b.w} : (u32x4){a.x, a.y, b.x, b.y};
            }
        }
        // slots past the end may hold anything, NaN too: their V is cleared (`keep`: bits of the lane's tokens that stay)
        int n0 = 4, n1 = 4;
        if (need_mask) {
            n0 = min(max(w.tok1 - (first + 4 * g), 0), 4);
            n1 = min(max(w.tok1 - (first + SPEC_BLOCK_SIZE + 4 * g), 0), 4);
        }
        if constexpr (B8) {
            const uint32_t keep0 = n0 >= 4 ? 0xFFFFFFFFu : (1u << (8 * n0)) - 1u, keep1 = n1 >= 4 ? 0xFFFFFFFFu : (1u << (8 * n1)) - 1u;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                uint32_t c0 = cur.v[0][mt / 4][mt % 4], c1 = cur.v[1][mt / 4][mt % 4];
                if (need_mask) { c0 &= keep0; c1 &= keep1; }
                const u32x2 v0 = codes_to_f16<INT8>(c0), v1 = codes_to_f16<INT8>(c1);
                const f16x8 va = __builtin_bit_cast(f16x8, (u32x4){v0.x, v0.y, v1.x, v1.y});
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) acc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, __builtin_bit_cast(f16x8, pw[nt][t]), acc[nt][mt], 0, 0, 0);
            }
        } else {
            if (need_mask) {
                const u32x4 keep = {n0 >= 2 ? 0xFFFFFFFFu : (n0 == 1 ? 0x0000FFFFu : 0u), n0 >= 4 ? 0xFFFFFFFFu : (n0 == 3 ? 0x0000FFFFu : 0u),
                                    n1 >= 2 ? 0xFFFFFFFFu : (n1 == 1 ? 0x0000FFFFu : 0u), n1 >= 4 ? 0xFFFFFFFFu : (n1 == 3 ? 0x0000FFFFu : 0u)};
                bool odd = false;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    v[mt] &= keep;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        odd = odd || (v[mt][e] & 0x7F80u) == 0x7F80u || (v[mt][e] & 0x7F800000u) == 0x7F800000u;
                }
                // An infinity or NaN in a token that some rows do not see would reach them as 0 * inf: such values leave the
                // product, and are added to the rows that see them (any positive weight leaves them what they are).
                if (__builtin_amdgcn_ballot_w64(odd) != 0) {
                    const int at[2] = {__builtin_amdgcn_readlane(bt, 2 * i), __builtin_amdgcn_readlane(bt, 2 * i + 1)};
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if ((v[mt][e] & 0x7F80u) == 0x7F80u) v[mt][e] &= 0xFFFF0000u;
                            if ((v[mt][e] & 0x7F800000u) == 0x7F800000u) v[mt][e] &= 0x0000FFFFu;
                        }
#pragma unroll 1
                    for (int t = 0; t < 2 * SPEC_BLOCK_SIZE; ++t) {
                        const int slot = t % SPEC_BLOCK_SIZE, entry = at[t / SPEC_BLOCK_SIZE];
                        if (first + t >= w.tok1 || entry < 0) continue;
                        const uint16_t *page = reinterpret_cast<const uint16_t *>(vhead + (size_t)entry * page_stride);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {   // the dims that this lane accumulates: 16 mt + 4 g + e
                                const int c = 16 * mt + 4 * g + e;
                                const uint32_t bits = page[TM ? slot * D + c : ((((c / 32) * 4 + slot / 4) * 16 + c % 16) * 2 + (c / 16) % 2) * 4 + slot % 4];
                                if ((bits & 0x7F80u) != 0x7F80u) continue;
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
                                    if (first + t <= limit[nt]) acc[nt][mt][e] += __uint_as_float(bits << 16);
                            }
                    }
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int t = 0; t < TERMS; ++t)
                        acc[nt][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[mt]), __builtin_bit_cast(bf16x8, pw[nt][t]), acc[nt][mt], 0, 0, 0);
            }
        }
    };

    {
        Pair<KIND, D> a, b;
        load(0, a);
        for (int i = 0; i < my_pairs; i += 2) {
            load(i + 1, b);
            consume(a, i);
            load(i + 2, a);
            if (i + 1 < my_pairs) consume(b, i + 1);
        }
    }

    // merge the wavefronts: 2, 3 into 0, 1, then 1 into 0
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) l_run[nt] = sum_across_rows(l_run[nt]);
    auto put = [&](int buf) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sh.acc[buf][nt][mt][lane] = acc[nt][mt];
            sh.m[buf][nt][lane] = m_run[nt];
            sh.l[buf][nt][lane] = l_run[nt];
        }
    };
    auto merge = [&](int buf) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float mo = sh.m[buf][nt][lane], mn = fmaxf(m_run[nt], mo);
            const float wa = fast_exp2(m_run[nt] - mn), wb = fast_exp2(mo - mn);
            l_run[nt] = l_run[nt] * wa + sh.l[buf][nt][lane] * wb;
            m_run[nt] = mn;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = acc[nt][mt] * wa + sh.acc[buf][nt][mt][lane] * wb;
        }
    };
    __syncthreads();   // (the regions of the walk are free)
    if (wave >= 2) put(wave - 2);
    __syncthreads();
    if (wave < 2) merge(wave);
    __syncthreads();
    if (wave == 1) put(0);
    __syncthreads();
    if (wave == 0) {
        merge(0);   // (its reads precede the writes below in program order)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                *reinterpret_cast<f32x4 *>(sh.o + (nt * 16 + n16) * o_row_bytes(D) + (mt * 16 + 4 * g) * 4) = acc[nt][mt];
            if (g == 0) {
                sh.row_m[nt * 16 + n16] = m_run[nt];
                sh.row_l[nt * 16 + n16] = l_run[nt];
            }
        }
    }
    __syncthreads();

    constexpr int OP = D / 4;   // pieces of four dims in a row
    if (prefix || w.nchunks > 1) {
        float *const acc_out = prefix ? p.prefix_acc : p.acc, *const ml_out = prefix ? p.prefix_ml : p.ml;
        const int chunks = prefix ? p.max_prefix_chunks : p.max_chunks;
        for (int piece = tid; piece < rows * OP; piece += kThreads) {
            const int r = piece / OP, c = piece % OP;
            const size_t slot = out_index(r) * chunks + w.chunk;
            const f32x4 o = *reinterpret_cast<const f32x4 *>(sh.o + r * o_row_bytes(D) + c * 16);
            unsigned long long *dst = reinterpret_cast<unsigned long long *>(acc_out + slot * D + c * 4);
            publish_u64(dst, pack_f32x2(o[0], o[1]));
            publish_u64(dst + 1, pack_f32x2(o[2], o[3]));
            if (c == 0) publish_u64(reinterpret_cast<unsigned long long *>(ml_out + slot * 2), pack_f32x2(sh.row_m[r], sh.row_l[r]));
        }
        if (prefix) return;
        writes_complete();   // the partials are in memory before the ticket is taken
        __syncthreads();
        if (tid == 0) {
            unsigned long long *ticket = &p.tickets[((size_t)w.b * p.Hkv + w.kvh) * p.row_blocks + w.row_block];
            const int last = ticket_arrive(ticket, p.generation) + 1u == (uint32_t)w.nchunks ? 1 : 0;
            if (last) ticket_reset(ticket);
            sh.last = last;
        }
        __syncthreads();
        if (!sh.last) return;
        order_after_ticket();
    }
    // the rows' results: the prefix's partials, then the own ones in chunk order
    for (int piece = tid; piece < rows * OP; piece += kThreads) {
        const int r = piece / OP, c = piece % OP;
        const size_t rh = out_index(r);
        RowSum sum;
        add_prefix<D>(p, sum, rh, w.prefix_chunks, c * 4);
        if (w.nchunks == 1) {
            sum.add(sh.row_m[r], sh.row_l[r], *reinterpret_cast<const f32x4 *>(sh.o + r * o_row_bytes(D) + c * 16));
        } else {
#pragma unroll 4
            for (int k = 0; k < w.nchunks; ++k) {
                const size_t slot = rh * p.max_chunks + k;
                const unsigned long long *src = reinterpret_cast<const unsigned long long *>(p.acc + slot * D + c * 4);
                const unsigned long long ml = fetch_u64(reinterpret_cast<const unsigned long long *>(p.ml + slot * 2));
                const unsigned long long o0 = fetch_u64(src), o1 = fetch_u64(src + 1);
                sum.add(__uint_as_float((uint32_t)ml), __uint_as_float((uint32_t)(ml >> 32)),
                        (f32x4){__uint_as_float((uint32_t)o0), __uint_as_float((uint32_t)(o0 >> 32)), __uint_as_float((uint32_t)o1),
                                __uint_as_float((uint32_t)(o1 >> 32))});
            }
        }
        write_row<D>(p, rh, c * 4, sum);
    }
}

template <int KIND, int NT, int D, bool FULL>
void go(const CacheAttnParams &p, CacheLaunch at, hipStream_t stream)
{
    hipLaunchKernelGGL((cache_attn_kernel<KIND, NT, D, FULL>), dim3(at.blocks), dim3(kThreads), 0, stream, p, at.prefix);
}

}  // namespace

template <int KIND>
hipError_t launch_cache_kind(const CacheAttnParams &p, int tiles, bool full, CacheLaunch at, hipStream_t stream)
{
    auto by_dim = [&](auto nt) {
        constexpr int NT = decltype(nt)::value;
        if (p.d == 128) { if (full) go<KIND, NT, 128, true>(p, at, stream); else go<KIND, NT, 128, false>(p, at, stream); }
        else { if (full) go<KIND, NT, 64, true>(p, at, stream); else go<KIND, NT, 64, false>(p, at, stream); }
    };
    if (tiles == 1) by_dim(std::integral_constant<int, 1>());
    else if (tiles == 2) by_dim(std::integral_constant<int, 2>());
    else if (tiles == 3) by_dim(std::integral_constant<int, 3>());
    else return hipErrorInvalidValue;
    return hipGetLastError();
}
template hipError_t launch_cache_kind<SPEC_CACHE_PART>(const CacheAttnParams &p, int tiles, bool full, CacheLaunch at, hipStream_t stream);

#else   // the launch functions

namespace {

hipError_t launch_kind(const CacheAttnParams &p, int tiles, CacheLaunch at, hipStream_t stream)
{
    const bool full = p.out_f32 != 0;
    switch (p.kind) {
        case kCacheTiles: return launch_cache_kind<kCacheTiles>(p, tiles, full, at, stream);
        case kCacheTokens: return launch_cache_kind<kCacheTokens>(p, tiles, full, at, stream);
        case kCacheE4M3: return launch_cache_kind<kCacheE4M3>(p, tiles, full, at, stream);
        case kCacheInt8: return launch_cache_kind<kCacheInt8>(p, tiles, full, at, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnParams &p, hipStream_t stream)
{
    if (p.max_prefix_chunks > 0) {
        const unsigned blocks = (unsigned)(p.prefix_row_blocks * p.Hkv * p.max_prefix_chunks);
        const hipError_t err = launch_kind(p, p.prefix_tiles, CacheLaunch{blocks, 1}, stream);
        if (err != hipSuccess) return err;
    }
    return launch_kind(p, p.row_tiles, CacheLaunch{(unsigned)(p.row_blocks * p.B * p.Hkv * p.max_chunks), 0}, stream);
}

#endif

}  // namespace specv

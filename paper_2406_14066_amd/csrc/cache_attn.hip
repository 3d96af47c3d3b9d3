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
// the exponent; they fit fp16, whose 11 bits keep their rounding (2^-12) below that of a bf16 output.  l is kept times 2^22: 2^22 / v_t is
// between 2^-99 and 2^91, so that weights from 2^-34 of the largest on up to those of a million tokens stay normal numbers in it
// whatever the scales are (denormals are flushed).
#include "code8.h"

#include <math.h>

#include <type_traits>

#ifndef SPEC_CACHE_PART
#error "compiled once per kind of cache: SPEC_CACHE_PART is the kind, or 4 for the launch functions"
#endif

namespace specv {

// Variants are chosen by (row tiles or wavefronts, head dim, type of the output); one set per kind of cache.
struct CacheLaunch {
    dim3 blocks;
    int prefix;      // which of the two launches
    int tiles;       // cache_attn_kernel's row tiles; 0: the launch is prefix_rows_kernel's
    int waves;       // prefix_rows_kernel's wavefronts
};
template <int KIND>
hipError_t launch_cache_kind(const CacheAttnParams &p, CacheLaunch at, hipStream_t stream);

#if SPEC_CACHE_PART < 4

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kDeviceScope = 16;        // "sc1" bit of a raw buffer access: coherent over the device's caches
constexpr float kRescaleSlack = 8.0f;   // the running reference follows the maximum when it is this much behind
constexpr float kLift = 0x1p22f, kLower = 0x1p-22f;   // 8-bit pages: of the sums of weights (see above)

// Partial results of the launch for many rows keep a row's dims in the order in which the wavefronts that merge them hold
// them: four groups of 4 from each 16-dim slice of a wavefront (D = 128: two slices), a lane's dims side by side.
template <int D>
__device__ __forceinline__ constexpr int partial_place(int dim)   // of four dims
{
    if constexpr (D == 128) return dim / 32 * 32 + dim % 16 / 4 * 8 + dim % 32 / 16 * 4;
    return dim;
}

constexpr int v_row_bytes(int D) { return D * 2 + 16; }   // token rows of V in LDS (token-major pages)
constexpr int q_row_bytes(int D) { return D * 2 + 16; }   // query rows in LDS

// The IEEE 754-2019 maximum: unlike fmaxf it needs no canonicalising multiplication per operand that a matrix
// instruction made.  A NaN stays one: the row it belongs to is NaN whatever its reference is.
__device__ __forceinline__ float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }

template <int KIND, int D>
struct Pair {   // two pages
    static constexpr int N = is_8bit(KIND) ? D / 64 : D / 32;   // 1 KB loads of K, of V
    u32x4 k[2][N], v[2][N];
    float ks, vs;   // 8-bit: the scales of one token: lane (g, n) has token 4 g + n % 4 of page n / 4 % 2
};

// Lane N of the 16-lane row, to all lanes of the row.
template <int N>
__device__ __forceinline__ float row_broadcast(float x)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), 0x150 + N, 0xF, 0xF, true));
}

template <int KIND, int NT, int D>
struct Shared {
    static constexpr int kSlices = D / 16 / kWaves;          // 16-dim slices that a wavefront merges
    union {
        struct {
            alignas(16) unsigned char q[NT * 16 * q_row_bytes(D)];   // the block's query rows
            unsigned char v[KIND == kCacheTokens ? kWaves : 1][KIND == kCacheTokens ? 2 * SPEC_BLOCK_SIZE * v_row_bytes(D) : 16];
        };
        f32x4 acc[kWaves][kWaves - 1][NT][kSlices][kWave];   // for each wavefront, the others' results for its slices
    };
    float m[kWaves][NT][16], l[kWaves][NT][16];
    int last;
};

// The block's place in the work.
struct Work {
    int b;             // request whose block-table row says where the pages are
    int head, head_pages;   // ... but for its first pages another one's
    int kvh, chunk, nchunks;
    int row0, rows;    // first packed token row, fused query rows from there on
    int row_lo;        // first of them that is this block's
    int tok0, tok1;    // its tokens
    int hide_from;     // row r of the block's rows sees tokens < hide_from + r / group; all of them: INT_MAX
    int prefix;        // tokens of its group's prefix
    int group_index, first_of_group, end_of_group;    // its group, and (lane-wise, groups 0 .. 63) every group's requests and prefix
    int prefix_of_group;
    int prefix_chunks;                // partial results that come in from the prefix launch
    int row_block;
};

// r / group for rows: a product with a rounded-up reciprocal, exact for r < 2^32 / 16.
__device__ __forceinline__ int by_group(const CacheAttnParams &p, int r) { return p.group == 1 ? r : (int)__umulhi((uint32_t)r, p.group_inverse); }

// Packed (token row, query head) of fused row r of the rows that begin at packed token row row0.
__device__ __forceinline__ size_t packed_row(const CacheAttnParams &p, int row0, int kvh, int r)
{
    const int j = by_group(p, r);
    return (size_t)(row0 + j) * p.Hq + kvh * p.group + (r - j * p.group);
}
__device__ __forceinline__ const __bf16 *query_row(const CacheAttnParams &p, int row0, int kvh, int r)
{
    const int j = by_group(p, r);
    return static_cast<const __bf16 *>(p.q) + (size_t)(row0 + j) * p.q_stride + (size_t)(kvh * p.group + (r - j * p.group)) * (p.d);
}

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

// A group of the launch for prefixes with many query rows (see prefix_rows_kernel): its row blocks, and the pieces that each of
// them walks the prefix in.
struct GroupWork {
    int request, row0, rows, pages;   // first request, first packed token row, fused query rows, pages of the prefix
    int pieces, blocks;               // ... row blocks times pieces: the blocks of a KV head; 0: none (or not valid, which the own launch reports)
    __device__ __forceinline__ void set(const CacheAttnParams &p, int b0, int b1, int P)
    {
        request = row0 = rows = pages = pieces = blocks = 0;
        if (b0 < 0 || b0 > b1 || b1 > p.B || !prefix_ok(p, P)) return;
        request = b0;
        row0 = p.cu_q_len[b0];
        const int end = p.cu_q_len[b1];
        if (row0 < 0 || end <= row0 || end > p.T) return;
        rows = (end - row0) * p.group;
        pages = P / SPEC_BLOCK_SIZE;
        const int steps = (pages + kStepPages - 1) / kStepPages;
        pieces = (steps + p.prefix_piece_steps - 1) / p.prefix_piece_steps;
        // (more than there can be, from rows that several groups claim, stays more: sums of 64 of them do not wrap)
        blocks = (int)min((int64_t)((rows + (1 << p.prefix_rows_log2) - 1) >> p.prefix_rows_log2) * pieces, (int64_t)kMaxPrefixBlocks + 1);
    }
    __device__ __forceinline__ void look(const CacheAttnParams &p, int g)
    {
        if (g < p.G) set(p, p.cu_group[g], p.cu_group[g + 1], p.prefix_len[g]);
        else request = row0 = rows = pages = pieces = blocks = 0;
    }
};

// The sum over the lanes, and over this lane and those before it.
__device__ __forceinline__ int running_sum(int x, int &all)
{
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const int up = __shfl_up(x, off);
        if (lane >= off) x += up;
    }
    all = __builtin_amdgcn_readlane(x, kWave - 1);
    return x;
}

// Blocks of a KV head, all groups.
__device__ __forceinline__ int group_blocks(const CacheAttnParams &p)
{
    int total = 0;
    for (int base = 0; base < p.G; base += kWave) {
        GroupWork work;
        work.look(p, base + threadIdx.x % kWave);
        int all;
        (void)running_sum(work.blocks, all);
        total = min(total + all, kMaxPrefixBlocks + 1);
    }
    return total;
}

// Row blocks of requests b0 .. b1 - 1 in the prefix launch for few rows, of `size` rows each; 0: none, or not valid.
__device__ __forceinline__ int few_rows_blocks(const CacheAttnParams &p, int b0, int b1, int size)
{
    if (b0 < 0 || b0 > b1 || b1 > p.B) return 0;
    const int row0 = p.cu_q_len[b0], end = p.cu_q_len[b1];
    return row0 < 0 || end <= row0 || end > p.T ? 0 : ((end - row0) * p.group + size - 1) / size;
}

// One block of the own launch: grid (KV heads, requests, row blocks x chunks).
template <int NT>
__device__ __forceinline__ bool place_own(const CacheAttnParams &p, Work &w)
{
    w.kvh = blockIdx.x;
    w.b = blockIdx.y;
    w.chunk = p.row_blocks == 1 ? blockIdx.z : blockIdx.z / p.row_blocks;
    w.row_block = blockIdx.z - w.chunk * p.row_blocks;
    // (up to 64 groups, a lane each, are looked up with the loads that the lengths take anyway)
    const int lane = threadIdx.x % kWave;
    w.first_of_group = w.end_of_group = w.prefix_of_group = 0;
    if (p.G <= kWave && lane < p.G) {
        w.first_of_group = p.cu_group[lane];
        w.end_of_group = p.cu_group[lane + 1];
        w.prefix_of_group = p.prefix_len[lane];
    }
    const int L = uniform_load(p.kv_len, w.b);
    w.row0 = uniform_load(p.cu_q_len, w.b);
    const int q_len = uniform_load(p.cu_q_len, w.b + 1) - w.row0;
    if (q_len == 0) return false;   // a padded slot
    const bool first = w.chunk == 0 && w.kvh == 0 && w.row_block == 0;
    int P = 0;
    w.group_index = 0;
    w.head = w.b;
    if (p.G > kWave) {
        w.group_index = group_of(p, w.b);
        P = uniform_load(p.prefix_len, w.group_index);
        w.head = uniform_load(p.cu_group, w.group_index);
    } else if (p.G > 0) {
        w.group_index = min(__builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < p.G && w.end_of_group <= w.b)), p.G - 1);
        P = __builtin_amdgcn_readlane(w.prefix_of_group, w.group_index);
        w.head = __builtin_amdgcn_readlane(w.first_of_group, w.group_index);
    }
    const int own_from = p.whole_context ? 0 : P;
    w.prefix = own_from;
    w.head_pages = p.whole_context ? P / SPEC_BLOCK_SIZE : 0;
    // The lengths come from device memory and bound every loop and index below: a request whose lengths do not fit
    // the launch is left out and reported.
    if (q_len < 0 || q_len > SPEC_K_MAX + 1 || w.row0 < 0 || w.row0 + q_len > p.T || q_len * p.group > p.max_q_rows || L < 0 ||
        L > p.capacity_tokens || (L + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE > p.max_blocks_per_req || !prefix_ok(p, P) ||
        (P > 0 && (L - q_len < P || w.head < 0 || w.head > w.b))) {
        count_error(p, first);
        return false;
    }
    w.rows = q_len * p.group;
    w.row_lo = w.row_block * (NT * 16);
    if (w.row_lo >= w.rows) return false;
    // even chunks per request, page aligned; a request without tokens has one that is empty
    const int tokens = L - own_from;
    w.nchunks = p.max_chunks == 1 ? 1 : max(min(chunk_count(tokens, p.chunk_tokens), p.max_chunks), 1);
    if (w.chunk >= w.nchunks) return false;
    const int C = w.nchunks == 1 ? tokens : ((tokens + w.nchunks - 1) / w.nchunks + SPEC_BLOCK_SIZE - 1) & ~(SPEC_BLOCK_SIZE - 1);
    if (C > kMaxChunkTokens) {   // (a prefix that is shorter on the device than planned for)
        count_error(p, first);
        return false;
    }
    w.tok0 = min(own_from + w.chunk * C, L);
    w.tok1 = min(w.tok0 + C, L);
    w.hide_from = L - q_len + 1;
    return true;
}

// Which partial results of the prefix launch are this block's (not needed before its own rows are done, so it is found out while
// the first pages are on their way).  False: they are not there; reported.
__device__ __forceinline__ bool place_partials(const CacheAttnParams &p, Work &w)
{
    w.prefix_chunks = 0;
    if (w.prefix == 0) return true;
    const bool first = w.chunk == 0 && w.kvh == 0 && w.row_block == 0;
    if (!p.prefix_many_rows) {
        // (scalar loads, which do not wait for the pages)
        const int b1 = uniform_load(p.cu_group, w.group_index + 1);
        bool there = b1 > w.b && b1 <= p.B;
        if (there) {
            const int row0 = uniform_load(p.cu_q_len, w.head), end = uniform_load(p.cu_q_len, b1);
            there = row0 >= 0 && row0 <= w.row0 && w.row0 + by_group(p, w.rows) <= end && end <= p.T;
        }
        if (!there) {
            count_error(p, first);
            return false;
        }
        w.prefix_chunks = chunk_count(w.prefix, p.prefix_chunk_tokens);
        return true;
    }
    GroupWork work;
    int total, rows, row0;
    if (p.G <= kWave) {
        if ((int)(threadIdx.x % kWave) < p.G) work.set(p, w.first_of_group, w.end_of_group, w.prefix_of_group);
        else work.look(p, p.G);
        (void)running_sum(work.blocks, total);
        w.prefix_chunks = __builtin_amdgcn_readlane(work.pieces, w.group_index);
        rows = __builtin_amdgcn_readlane(work.rows, w.group_index);
        row0 = __builtin_amdgcn_readlane(work.row0, w.group_index);
    } else {
        total = group_blocks(p);
        work.look(p, w.group_index);
        w.prefix_chunks = __builtin_amdgcn_readfirstlane(work.pieces);
        rows = __builtin_amdgcn_readfirstlane(work.rows);
        row0 = __builtin_amdgcn_readfirstlane(work.row0);
    }
    const int after = (w.row0 - row0) * p.group;   // the request's rows lie in its group's
    if ((int64_t)total * p.Hkv > p.prefix_row_blocks || w.prefix_chunks == 0 || after < 0 || after + w.rows > rows) {
        count_error(p, first);
        return false;
    }
    return true;
}

// One block of the prefix launch: grid (KV heads, row blocks of all groups, chunks).
template <int ROWS>
__device__ __forceinline__ bool place_prefix(const CacheAttnParams &p, Work &w)
{
    w.kvh = blockIdx.x;
    const int block = blockIdx.y;
    w.chunk = blockIdx.z;
    // the group that holds row block `block`: a lane counts the blocks of a group, 64 groups at a time
    const int lane = threadIdx.x % kWave;
    int before = 0, g = -1;
    for (int base = 0; base < p.G && g < 0; base += kWave) {
        const int n = base + lane < p.G ? few_rows_blocks(p, p.cu_group[base + lane], p.cu_group[base + lane + 1], ROWS) : 0;
        int all;
        const int sum = running_sum(n, all);
        const unsigned long long holds = __builtin_amdgcn_ballot_w64(before + sum > block);
        if (holds != 0) {
            const int at = __builtin_ctzll(holds);
            g = base + at;
            w.row_block = block - before - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(n, at));
        } else {
            before += all;
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
    if (!prefix_ok(p, P) || P == 0) return false;   // (counted by the own launch)
    w.rows = tokens * p.group;
    w.row_lo = w.row_block * ROWS;
    if (w.row_lo >= w.rows) return false;
    w.nchunks = chunk_count(P, p.prefix_chunk_tokens);
    if (w.chunk >= w.nchunks) return false;
    const int C = ((P + w.nchunks - 1) / w.nchunks + SPEC_BLOCK_SIZE - 1) & ~(SPEC_BLOCK_SIZE - 1);
    w.tok0 = min(w.chunk * C, P);
    w.tok1 = min(w.tok0 + C, P);
    w.hide_from = 0x7FFFFFFF - SPEC_K_MAX - 1;
    w.prefix = w.head = w.head_pages = 0;
    return true;
}

// Weighted sum of partial results: N times four head dims of a row.
template <int N>
struct RowSum {
    float m, l;
    f32x4 o[N];
    __device__ __forceinline__ void clear()
    {
        m = kEmptyMax;
        l = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    }
    __device__ __forceinline__ void add(float pm, float pl, const f32x4 (&po)[N])
    {
        const float mn = fmaxf(m, pm);
        const float keep = fast_exp2(m - mn), take = fast_exp2(pm - mn);
        l = l * keep + pl * take;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = o[i] * keep + po[i] * take;
        m = mn;
    }
};

// ---------------------------------------------------------------------------
// One block: a row block of NT 16-row tiles through a chunk of a request's tokens (or, prefix = 1, of a group's prefix, with at most 48 query
// rows behind it).  Four wavefronts take the chunk's pairs of pages in turn and never wait for each other before the end: K and V go
// from memory into a wavefront's registers in operand order, and each part of them asks for the next pair as soon as it has been used.
//
// What bounds it: with many blocks the bytes of the cache (256 requests of 256 .. 1024 tokens on 64/8 heads, 8-bit, k = 2: 371 MB in
// 72 us, 5.1 TB/s); with wide rows the instructions of a step, which are conversions and softmax more than matrix products (4 requests of
// 6000 .. 32768 tokens, int8, 36 rows, fp32 output: 58 us, 3.8 TB/s; counters: vector instructions 53% of the wavefronts' cycles, matrix
// instructions 27%, waits 23%); with few blocks latency (one request of 687 tokens: 6.9 us, of which 3.8 is an empty launch).
// Hence one wavefront a SIMD with as many registers as that allows, the queries in LDS (NT > 1), descriptors and scales by a
// few instructions, masks only in the steps that need them.  Eight wavefronts a block, a block order that keeps a request on an XCD, and
// three blocks on a compute unit (registers spilled) were all slower.
// ---------------------------------------------------------------------------
template <int KIND, int NT, int D, bool FULL>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_kernel(CacheAttnParams p, int prefix)
{
    constexpr bool B8 = is_8bit(KIND), INT8 = KIND == kCacheInt8, TM = KIND == kCacheTokens;
    constexpr int KK = D / 32, MT = D / 16;
    constexpr int kPageBytes = SPEC_BLOCK_SIZE * D * (B8 ? 1 : 2);   // of one KV head
    constexpr int TERMS = FULL ? (B8 ? 2 : 3) : (B8 ? 1 : 2);   // 16-bit terms of a softmax weight: 11 or 22 bits of fp16's, 16 or 24 of bf16's
    constexpr float kTop = B8 ? 7.0f : 0.0f;         // fp16 weights go up to 2^(7 + slack): their small ones stay normal numbers
    typedef std::conditional_t<B8, f16x8, bf16x8> Weights;
    __shared__ Shared<KIND, NT, D> sh;

    Work w;
    if (!(prefix ? place_prefix<NT * 16>(p, w) : place_own<NT>(p, w))) return;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n16 = lane & 15, g = lane >> 4;
    const int rows = min(w.rows - w.row_lo, NT * 16);   // this block's

    // Q goes to LDS and comes back as the B operand of S^T = K Q^T when it is needed (a single tile: once, for good), which keeps
    // registers for pages on their way: lane (g, n) takes row n, the 8 dims that the lane's K holds (bf16 pages: 32 kk + 8 g ..; 8-bit pages, 16
    // bytes of which are two operands: 64 (kk / 2) + 16 g + 8 (kk % 2) ..)
    constexpr int QP = D / 8, QN = (NT * 16 * QP + kThreads - 1) / kThreads;   // 16-byte pieces of a row, of a thread
    u32x4 q_piece[QN];
#pragma unroll
    for (int k = 0; k < QN; ++k) {
        const int piece = k * kThreads + tid, r = piece / QP;
        q_piece[k] = (u32x4){0u, 0u, 0u, 0u};
        if (r < rows) q_piece[k] = *reinterpret_cast<const u32x4 *>(query_row(p, w.row0, w.kvh, w.row_lo + r) + piece % QP * 8);
    }

    // block-table entries of this wavefront's pages: pairs wave, wave + 4, ...; lane 2 i + h holds page h of its pair i
    const int npages = (w.tok1 - w.tok0 + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE;   // <= 64 * kWaves
    const int mine = 2 * (wave + kWaves * (lane >> 1)) + (lane & 1);
    int bt = -1;
    bool some_bad;
    {
        const bool used = mine < npages;
        const int page = w.tok0 / SPEC_BLOCK_SIZE + mine;
        if (used) bt = p.block_table[(size_t)(page < w.head_pages ? w.head : w.b) * p.max_blocks_per_req + page];
        const bool bad = used && (unsigned)bt >= (unsigned)p.num_blocks;   // never turned into an address: reads as zeros
        if (bad) bt = -1;
        const unsigned long long bad_lanes = __builtin_amdgcn_ballot_w64(bad);
        some_bad = bad_lanes != 0;
        if (some_bad && w.kvh == 0 && w.row_block == 0 && p.errors != nullptr) {   // (a shared page: by the group's first rows)
            const unsigned long long shared = __builtin_amdgcn_ballot_w64(bad && page < w.head_pages);
            const int n = __builtin_popcountll(w.row0 == uniform_load(p.cu_q_len, w.head) ? bad_lanes : bad_lanes & ~shared);
            if (lane == 0 && n > 0) atomicAdd(p.errors, (unsigned long long)n);
        }
    }
    const int npairs = (npages + 1) / 2;
    const int my_pairs = npairs > wave ? (npairs - wave + kWaves - 1) / kWaves : 0;

    int limit[NT];   // last token that the lane's row sees
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 16 + n16;
        limit[nt] = r < rows ? w.hide_from - 1 + (prefix ? 0 : by_group(p, w.row_lo + r)) : -1;
    }
    int q_at = 0;   // (0, but the compiler does not know: it would hold Q in registers throughout)
    auto q_operand = [&](int nt, int kk) {
        return *reinterpret_cast<const bf16x8 *>(sh.q + q_at + (nt * 16 + n16) * q_row_bytes(D) + (B8 ? 128 * (kk / 2) + 32 * g + 16 * (kk % 2) : 64 * kk + 16 * g));
    };

    // Pages are read through descriptors that cover exactly one (page, KV head); a page that is not there has length 0,
    // for which the hardware returns zeros without touching memory.
    const char *khead = static_cast<const char *>(p.k_cache) + (size_t)w.kvh * kPageBytes;
    const char *vhead = static_cast<const char *>(p.v_cache) + (size_t)w.kvh * kPageBytes;
    const uint32_t page_stride = (uint32_t)p.Hkv * kPageBytes;
    Pair<KIND, D> cur;
    auto page_of = [&](int i, int h) {   // -1: none.  (past the last pair that a wavefront can have: that one again, and not used)
        return __builtin_amdgcn_readlane(bt, 2 * min(i, kWave / 2 - 1) + h);
    };
    auto page_descriptor = [&](const char *head, int page) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(head + (uint64_t)(uint32_t)page * page_stride), 0, page < 0 ? 0 : kPageBytes, kBufferFlags);
    };
    auto load_k = [&](int i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const __amdgpu_buffer_rsrc_t kd = page_descriptor(khead, page_of(i, h));
#pragma unroll
            for (int j = 0; j < Pair<KIND, D>::N; ++j)
                cur.k[h][j] = TM ? __builtin_amdgcn_raw_buffer_load_b128(kd, n16 * (D * 2) + g * 16, j * 64, 0)
                                 : __builtin_amdgcn_raw_buffer_load_b128(kd, lane * 16, j * 1024, kStreamPolicy);
        }
    };
    const char *scales_at = reinterpret_cast<const char *>(p.kv_scale + w.kvh * 32 + 4 * g + (n16 & 3));
    auto load_scales = [&](int i) {
        if constexpr (B8) {   // (no branch: a page that is not there is read as page 0, and not used)
            const uint32_t page0 = max(page_of(i, 0), 0), page1 = max(page_of(i, 1), 0);
            const float *at = reinterpret_cast<const float *>(scales_at + (uint64_t)((n16 & 4) ? page1 : page0) * (uint32_t)(p.Hkv * 128));
            cur.ks = at[0];
            cur.vs = at[16];
        }
    };
    auto load_v = [&](int i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const __amdgpu_buffer_rsrc_t vd = page_descriptor(vhead, page_of(i, h));
#pragma unroll
            for (int j = 0; j < Pair<KIND, D>::N; ++j) cur.v[h][j] = __builtin_amdgcn_raw_buffer_load_b128(vd, lane * 16, j * 1024, kStreamPolicy);
        }
    };
    load_k(0);
    load_scales(0);
    load_v(0);
    if (!place_partials(p, w)) return;
#pragma unroll
    for (int k = 0; k < QN; ++k) {
        const int piece = k * kThreads + tid;
        if (NT * 16 * QP % kThreads == 0 || piece < NT * 16 * QP)
            *reinterpret_cast<u32x4 *>(sh.q + piece / QP * q_row_bytes(D) + piece % QP * 16) = q_piece[k];
    }
    __syncthreads();   // Q is in LDS

    f32x4 acc[NT][MT];
    float m_run[NT], l_run[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m_run[nt] = kEmptyMax;
        l_run[nt] = 0.0f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[nt][mt] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    }

    // Each part of a pair's registers takes the next pair as soon as it has been used.
    // (masked: some of the pair's tokens are hidden from some row, or past the end, or some page is not there)
    auto step = [&](int i, auto masked) {
        constexpr bool need_mask = decltype(masked)::value;
        const int first = w.tok0 + 2 * (wave + kWaves * i) * SPEC_BLOCK_SIZE;
        if constexpr (NT > 1) asm volatile("" : "+v"(q_at));   // (the query rows are read from LDS in every step, not kept in registers)
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
                    s[nt][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), q_operand(nt, kk), s[nt][h], 0, 0, 0);
            }
        }
        load_k(i + 1);
        // to base-2 exponents; per token: k = scale of x, lv = log2 of V's scale, rv = its lifted reciprocal (each made by one lane of
        // the row and handed to the others)
        f32x4 ks[2], lv[2], rv[2];
        if constexpr (B8) {
            float k1 = cur.ks * p.scale_log2, v1 = __builtin_elementwise_maximum(cur.vs, kSmallestScale);
            if (need_mask) {
                const bool on = ((n16 & 4) ? page_of(i, 1) : page_of(i, 0)) >= 0;   // (a page that reads as zeros)
                k1 = on ? k1 : 0.0f;
                v1 = on ? v1 : kSmallestScale;
            }
            const float l1 = __builtin_amdgcn_logf(v1), r1 = __builtin_amdgcn_rcpf(v1 * kLower);
            auto hand_out = [&](float x, f32x4(&to)[2]) {
                to[0] = (f32x4){row_broadcast<0>(x), row_broadcast<1>(x), row_broadcast<2>(x), row_broadcast<3>(x)};
                to[1] = (f32x4){row_broadcast<4>(x), row_broadcast<5>(x), row_broadcast<6>(x), row_broadcast<7>(x)};
            };
            hand_out(k1, ks);
            hand_out(l1, lv);
            hand_out(r1, rv);
        }
        load_scales(i + 1);
        Weights pw[NT][TERMS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if constexpr (B8) s[nt][h][r] = fmaf(s[nt][h][r], ks[h][r], lv[h][r]);
                    if (need_mask && first + h * SPEC_BLOCK_SIZE + 4 * g + r > min(limit[nt], w.tok1 - 1)) s[nt][h][r] = -INFINITY;
                }
            }
            float mx = max3(max3(s[nt][0][0], s[nt][0][1], s[nt][0][2]), max3(s[nt][0][3], s[nt][1][0], s[nt][1][1]), __builtin_elementwise_maximum(s[nt][1][2], s[nt][1][3]));
            mx = B8 ? mx - kTop : mx * p.scale_log2;   // (the scale is positive: the maximum commutes with it)
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
                    const float e = fast_exp2(B8 ? s[nt][h][r] - m_run[nt] : fmaf(s[nt][h][r], p.scale_log2, -m_run[nt]));
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
                        const uint16_t *page = reinterpret_cast<const uint16_t *>(vhead + (uint64_t)entry * page_stride);
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
        load_v(i + 1);
    };

    const int all_see = min(w.tok1, w.hide_from) - w.tok0;   // tokens that every row sees
    const int plain = some_bad ? 0 : min(my_pairs, all_see / (2 * SPEC_BLOCK_SIZE) > wave ? (all_see / (2 * SPEC_BLOCK_SIZE) - wave + kWaves - 1) / kWaves : 0);
    int i = 0;
    for (; i < plain; ++i) step(i, std::false_type());
    for (; i < my_pairs; ++i) step(i, std::true_type());

    // Merge the wavefronts: each takes a quarter of the head dims of all rows and finds the others' results for them in LDS.
    constexpr int SN = Shared<KIND, NT, D>::kSlices;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) l_run[nt] = sum_across_rows(l_run[nt]);
    __syncthreads();   // (the walk's regions are free)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        if (g == 0) {
            sh.m[wave][nt][n16] = m_run[nt];
            sh.l[wave][nt][n16] = l_run[nt];
        }
    }
    RowSum<SN> sum[NT];   // row nt * 16 + n16, dims (wave * SN + i) * 16 + 4 g .. + 3
#pragma unroll
    for (int to = 0; to < kWaves; ++to) {
        if (to == wave) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < SN; ++i) sum[nt].o[i] = acc[nt][to * SN + i];
        } else {
            const int from = wave - (wave > to ? 1 : 0);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < SN; ++i) sh.acc[to][from][nt][i][lane] = acc[nt][to * SN + i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float m[kWaves], top = m_run[nt];
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            m[k] = sh.m[k][nt][n16];
            top = fmaxf(top, m[k]);
        }
        const float own = fast_exp2(m_run[nt] - top);
        sum[nt].m = top;
        sum[nt].l = 0.0f;
#pragma unroll
        for (int i = 0; i < SN; ++i) sum[nt].o[i] *= own;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) sum[nt].l = fmaf(sh.l[k][nt][n16], fast_exp2(m[k] - top), sum[nt].l);
#pragma unroll
        for (int k = 0; k < kWaves - 1; ++k) {
            const float take = fast_exp2((k < wave ? m[k] : m[k + 1]) - top);
#pragma unroll
            for (int i = 0; i < SN; ++i) sum[nt].o[i] += sh.acc[wave][k][nt][i][lane] * take;
        }
    }

    size_t rh[NT];   // packed (token row, query head) of the lane's rows (past the last: the last one's, not written)
    bool on[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 16 + n16;
        on[nt] = r < rows;
        rh[nt] = packed_row(p, w.row0, w.kvh, w.row_lo + min(r, rows - 1));
    }
    const int dim0 = wave * (SN * 16) + 4 * g;
    // Partial results are read in rounds, whose loads are all on their way together: as many as the walk's registers hold, or a few
    // where a few are left.
    constexpr int kFew = NT <= 2 ? 4 : 2, kMany = (NT * D >= 256 ? 160 : 80) / (NT * (4 * SN + 2));
    if (prefix) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (!on[nt]) continue;
            const size_t slot = rh[nt] * p.max_prefix_chunks + w.chunk;
#pragma unroll
            for (int i = 0; i < SN; ++i) *reinterpret_cast<f32x4 *>(p.prefix_acc + slot * D + dim0 + i * 16) = sum[nt].o[i];
            if (wave == 0 && g == 0) *reinterpret_cast<f32x2 *>(p.prefix_ml + slot * 2) = (f32x2){sum[nt].m, sum[nt].l};
        }
        return;
    }
    if (w.nchunks > 1) {
        // Partial results go from block to block inside the launch: past the cache levels that are not coherent
        // (kDeviceScope), 16 bytes at a time through descriptors of the request's part of the workspace.
        const size_t part = (size_t)w.row0 * p.Hq * p.max_chunks;
        const __amdgpu_buffer_rsrc_t acc_d = __builtin_amdgcn_make_buffer_rsrc(p.acc + part * D, 0, 0xFFFFFFFFu, kBufferFlags);
        const __amdgpu_buffer_rsrc_t ml_d = __builtin_amdgcn_make_buffer_rsrc(p.ml + part * 2, 0, 0xFFFFFFFFu, kBufferFlags);
        uint32_t at[NT];   // the row's first slot in it
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) at[nt] = (uint32_t)(rh[nt] - (size_t)w.row0 * p.Hq) * (uint32_t)p.max_chunks;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (!on[nt]) continue;
#pragma unroll
            for (int i = 0; i < SN; ++i)
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, sum[nt].o[i]), acc_d, ((at[nt] + w.chunk) * D + dim0 + i * 16) * 4, 0, kDeviceScope);
            if (wave == 0 && g == 0)
                __builtin_amdgcn_raw_buffer_store_b64((u32x2){__float_as_uint(sum[nt].m), __float_as_uint(sum[nt].l)}, ml_d, (at[nt] + w.chunk) * 8, 0, kDeviceScope);
        }
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
        // the last chunk to finish: all of them in chunk order
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sum[nt].clear();
        auto add_chunks = [&](auto count, int c0) {
            constexpr int U = decltype(count)::value;
            u32x2 ml[NT][U];
            u32x4 o[NT][U][SN];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const uint32_t slot = at[nt] + min(c0 + u, w.nchunks - 1);
                    ml[nt][u] = __builtin_amdgcn_raw_buffer_load_b64(ml_d, slot * 8, 0, kDeviceScope);
#pragma unroll
                    for (int i = 0; i < SN; ++i) o[nt][u][i] = __builtin_amdgcn_raw_buffer_load_b128(acc_d, (slot * D + dim0 + i * 16) * 4, 0, kDeviceScope);
                }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    f32x4 x[SN];
#pragma unroll
                    for (int i = 0; i < SN; ++i) x[i] = __builtin_bit_cast(f32x4, o[nt][u][i]);
                    if (c0 + u < w.nchunks) sum[nt].add(__uint_as_float(ml[nt][u].x), __uint_as_float(ml[nt][u].y), x);
                }
        };
        for (int c0 = 0; c0 < w.nchunks;) {
            if (w.nchunks - c0 > kFew) {
                add_chunks(std::integral_constant<int, kMany>(), c0);
                c0 += kMany;
            } else {
                add_chunks(std::integral_constant<int, kFew>(), c0);
                c0 += kFew;
            }
        }
    }
    // the prefix's partial results
    if (w.prefix > 0) {
        const bool many = p.prefix_many_rows != 0;
        auto add_pieces = [&](auto count, int c0) {
            constexpr int U = decltype(count)::value;
            f32x2 ml[NT][U];
            f32x4 o[NT][U][SN];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const size_t slot = rh[nt] * p.max_prefix_chunks + min(c0 + u, w.prefix_chunks - 1);
                    const float *from = p.prefix_acc + slot * D;
                    ml[nt][u] = *reinterpret_cast<const f32x2 *>(p.prefix_ml + slot * 2);
#pragma unroll
                    for (int i = 0; i < SN; ++i)
                        o[nt][u][i] = *reinterpret_cast<const f32x4 *>(from + (many ? partial_place<D>(dim0) + 4 * i : dim0 + i * 16));
                }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (c0 + u < w.prefix_chunks) sum[nt].add(ml[nt][u].x, ml[nt][u].y, o[nt][u]);
        };
        for (int c0 = 0; c0 < w.prefix_chunks;) {
            if (w.prefix_chunks - c0 > kFew) {
                add_pieces(std::integral_constant<int, kMany>(), c0);
                c0 += kMany;
            } else {
                add_pieces(std::integral_constant<int, kFew>(), c0);
                c0 += kFew;
            }
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        if (!on[nt]) continue;
        const float inv = sum[nt].l == 0.0f ? 0.0f : (B8 ? kLift : 1.0f) / sum[nt].l;   // (a row that has seen no key is zero)
#pragma unroll
        for (int i = 0; i < SN; ++i) {
            const f32x4 o = sum[nt].o[i] * inv;
            if (p.out_f32)
                *reinterpret_cast<f32x4 *>(static_cast<float *>(p.out) + rh[nt] * D + dim0 + i * 16) = o;
            else
                *reinterpret_cast<u32x2 *>(static_cast<__bf16 *>(p.out) + rh[nt] * D + dim0 + i * 16) =
                    __builtin_bit_cast(u32x2, __builtin_convertvector(o, bf16x4));
        }
    }
}

// ---------------------------------------------------------------------------
// Prefixes of groups with many query rows.
//
// A block takes a row block of 128 or 256 rows through a piece of its group's prefix, counted in steps of four pages: the pieces of a prefix are
// as even as they can be, and at most so long that the blocks of all groups fill the device (the host's choice).  Blocks lie KV head by KV
// head, group by group, row block by row block, and consecutive ones on one XCD, which share their KV head's pages in its L2.
//
// A block's wavefronts, four or eight, have 32 rows each and walk the same pages, which pass through LDS once for all of them, a step
// (64 tokens, a page brought in by each wavefront or by two) at a time.  In LDS the pages lie as the operands of v_mfma_f32_32x32x16 want
// them, 16 bytes per lane and 1 KB per read, as 16-bit values whatever the cache holds (8-bit codes are converted once on the
// way in); token-major V is stored by rows and read through the transposing read.  (lane = 32 half + c; pair: two of the pages)
//   S^T[token][row] = K[token][:] . Q[row][:]: a pair, 16 dims per instruction, lane (half, c) holds row c, tokens
//   4 half + 8 i + 0..3, i = 0, 1 of the first page, 2, 3 of the second
//   O^T[dim][row] += V^T[dim][token] . P^T[token][row]: a page per instruction, its tokens in that order
// Two LDS buffers and one barrier per step; operands are read four reads ahead of the products that take them, and both pairs'
// scores come before one look at the running maximum, so that the second pair's weights are made under the first one's products.
//
// What bounds it: behind one prefix of 4096 tokens, 64 requests, 64/8 heads, k = 2, bf16, the launch takes 45 us.  A block of eight
// wavefronts on each compute unit walks a step in 2.4 us, 1.24 PFLOP/s over the device counting the weights' second term and 0.83 without (a product
// of two 8192 x 8192 bf16 matrices reaches 1.31, of 4096 x 4096 1.10), for 31 of them; the rest is the start (finding the group, the table, the
// first pages: 5), the partial results (5) and the launch.  With one term the call took 64 instead of 73, and the error of its bf16 output was
// 1.35 times what rounding leaves.
// 8-bit pages add the conversions and the scales (three prefixes of 6000 .. 20000 tokens, 40 rows a request: 132 us for 113 GFLOP, of which 26 are of
// rows that are not there: groups of 648, 320 and 216 rows in blocks of 256); a second term of their weights, whose first has 11 bits,
// would take a call with them from 147 to 190.  Two blocks of four wavefronts a unit bring in and convert every page twice as
// often (calls 78 against 75.6, 161 against 156.5).  64 rows a wavefront would halve the operand reads, but its accumulators go to the second register file
// and come back for every use of the others; three blocks of four wavefronts with one pair a step do as well as two of these but leave half as
// many partial results again.
// ---------------------------------------------------------------------------
typedef float f32x16 __attribute__((ext_vector_type(16)));
template <int KIND, int D, int W>
struct RowsShared {
    static constexpr int kK = kStepPages * SPEC_BLOCK_SIZE * D * 2;   // of a step
    static constexpr int kV = kStepPages * SPEC_BLOCK_SIZE * (KIND == kCacheTokens ? v_row_bytes(D) : D * 2);
    static constexpr int kOutRow = D * 2 + 16;               // half a result row
    union {
        struct {
            alignas(16) unsigned char k[2][kK];   // [pair][16 dims][lane][16]
            alignas(16) unsigned char v[2][kV];   // [page][32-dim slice][lane][tokens 4 half .. + 3, 8 + 4 half .. + 3]; token-major: [page][token] rows
        };
        alignas(16) unsigned char o[W][kPrefixRows * kOutRow];   // results on their way out, by half rows
    };
    // 8-bit pages, per token: K's scale with the softmax scale, log2 of V's, its lifted reciprocal
    float scale[is_8bit(KIND) ? 2 : 1][3][is_8bit(KIND) ? kStepPages * SPEC_BLOCK_SIZE : 1];
    int page[kStepPages * (kMaxPrefixSteps + 4)];   // the steps' block-table entries, and four more steps'; -1: outside the pool, or past the end
    static_assert(kStepPages * kMaxPrefixSteps <= W * kWave, "a thread per page");
};

template <int KIND, int D, bool FULL, int W>
__global__ __launch_bounds__(W * kWave, 2) void prefix_rows_kernel(CacheAttnParams p)
{
    constexpr int kPerPage = W / kStepPages;             // wavefronts that bring in a page
    constexpr bool B8 = is_8bit(KIND), INT8 = KIND == kCacheInt8, TM = KIND == kCacheTokens;
    constexpr int KS = D / 16, SL = D / 32;
    constexpr int kPageBytes = SPEC_BLOCK_SIZE * D * (B8 ? 1 : 2);
    constexpr int N = B8 ? D / 64 : D / 32;              // 1 KB pieces of a page's K, of its V
    constexpr int TERMS = FULL ? (B8 ? 2 : 3) : (B8 ? 1 : 2);   // as in cache_attn_kernel: a row's error does not depend on the kernel that takes it
    constexpr float kTop = B8 ? 7.0f : 0.0f;
    typedef std::conditional_t<B8, f16x8, bf16x8> Weights;
    typedef RowsShared<KIND, D, W> Sh;
    __shared__ Sh sh;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, c32 = lane & 31, n16 = lane & 15, g = lane >> 4;
    // consecutive blocks go to different XCDs; consecutive steps stay on one
    const int block = (int)(blockIdx.x % kXcdCount) * (gridDim.x / kXcdCount) + blockIdx.x / kXcdCount;

    // the group, row block and piece
    int total = 0, rest = block, first = 0, steps = 0, row_block = 0;   // blocks of a KV head; its how-many-th block; the piece
    GroupWork work;
    work.look(p, lane);
    int all, upto = running_sum(work.blocks, all);
    total = p.G > kWave ? group_blocks(p) : all;
    if (total == 0 || (int64_t)total * p.Hkv > gridDim.x) return;   // (not the groups planned for: the own launch reports it)
    const int kvh = block / total;
    if (kvh >= p.Hkv) return;
    rest -= kvh * total;
    for (int base = kWave; rest >= all && base < p.G; base += kWave) {   // (more than 64 groups)
        rest -= all;
        work.look(p, base + lane);
        upto = running_sum(work.blocks, all);
    }
    if (rest >= all) return;
    {
        const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > rest));
        rest -= __builtin_amdgcn_readlane(upto - work.blocks, who);
        work.request = __builtin_amdgcn_readlane(work.request, who);
        work.row0 = __builtin_amdgcn_readlane(work.row0, who);
        work.rows = __builtin_amdgcn_readlane(work.rows, who);
        work.pages = __builtin_amdgcn_readlane(work.pages, who);
        work.pieces = __builtin_amdgcn_readlane(work.pieces, who);
    }
    row_block = rest / work.pieces;
    const int slot = rest - row_block * work.pieces;
    {
        const int all_steps = (work.pages + kStepPages - 1) / kStepPages, each = (all_steps + work.pieces - 1) / work.pieces;
        first = slot * each;
        steps = min(all_steps - first, each);
    }
    const int row0 = work.row0;                                 // the group's first packed token row
    const int row_lo = (row_block * W + wave) * kPrefixRows;
    const int rows = min(max(work.rows - row_lo, 0), 32);       // this wavefront's
    auto out_index = [&](int r) {
        return packed_row(p, row0, kvh, row_lo + r);
    };
    {
        const bool used = tid < kStepPages * steps && tid < work.pages - kStepPages * first;   // pages from the first one of these steps on
        int entry = -1;
        if (used) entry = p.block_table[(size_t)work.request * p.max_blocks_per_req + kStepPages * first + tid];
        const int last_pages = work.pages - kStepPages * (first + steps - 1);   // of the last step: 1 .. 4 (or more follow)
        bf16x8 q[KS];
        {
            const __bf16 *row = query_row(p, row0, kvh, c32 < rows ? row_lo + c32 : 0);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const bf16x8 *>(row + 16 * ks + 8 * half);
        }
        {
            const bool bad = used && (unsigned)entry >= (unsigned)p.num_blocks;   // never turned into an address: reads as zeros
            if (tid < kStepPages * (kMaxPrefixSteps + 4)) sh.page[tid] = bad ? -1 : entry;
            if (W * kWave < kStepPages * (kMaxPrefixSteps + 4) && tid < 4 * kStepPages) sh.page[kStepPages * kMaxPrefixSteps + tid] = -1;
            const unsigned long long bad_lanes = __builtin_amdgcn_ballot_w64(bad);
            if (bad_lanes != 0 && kvh == 0 && row_block == 0 && lane == 0 && p.errors != nullptr)
                atomicAdd(p.errors, (unsigned long long)__builtin_popcountll(bad_lanes));
        }
        __syncthreads();

        // Wavefront w brings in page w of a step (of eight: half of page w / 2).
        static_assert(N % kPerPage == 0, "whole pieces");
        constexpr int PN = N / kPerPage;
        const int my_page = wave / kPerPage, j0 = wave % kPerPage * PN;
        const char *khead = static_cast<const char *>(p.k_cache) + (size_t)kvh * kPageBytes;
        const char *vhead = static_cast<const char *>(p.v_cache) + (size_t)kvh * kPageBytes;
        const uint32_t page_stride = (uint32_t)p.Hkv * kPageBytes;
        struct {
            u32x4 k[PN], v[PN];
            float scale;   // 8-bit: the page's record, an entry per lane
        } in;
        auto load = [&](int page_entry) {
            const int entry = __builtin_amdgcn_readfirstlane(page_entry);
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
        auto store = [&](int buf) {
            unsigned char *ks = sh.k[buf] + (my_page >> 1) * (KS * 1024) + (my_page & 1) * 256, *vs = sh.v[buf];
#pragma unroll
            for (int i = 0; i < PN; ++i) {
                const int j = j0 + i;
                if constexpr (B8) {   // token n16, dims 64 j + 16 g .. + 15; tokens 4 g .. + 3, dims 64 j + 16 e + n16
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const u32x2 a = codes_to_bf16<INT8>(in.k[i][2 * e]), b = codes_to_bf16<INT8>(in.k[i][2 * e + 1]);
                        *reinterpret_cast<u32x4 *>(ks + (4 * j + g) * 1024 + (e * 32 + n16) * 16) = (u32x4){a.x, a.y, b.x, b.y};
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
                if (lane < 32 && wave % kPerPage == 0) {   // 16 scales of K, 16 of V (a page that reads as zeros: the smallest one)
                    const float x = __builtin_elementwise_maximum(in.scale, kSmallestScale);
                    float *to = &sh.scale[buf][0][my_page * 16 + n16];
                    constexpr int kRow = kStepPages * SPEC_BLOCK_SIZE;
                    if (lane < 16) to[0] = in.scale * p.scale_log2;
                    else {
                        to[kRow] = __builtin_amdgcn_logf(x);
                        to[2 * kRow] = __builtin_amdgcn_rcpf(x * kLower);
                    }
                }
            }
        };

        f32x16 acc[SL];
        float m_run = kEmptyMax, l_run = 0.0f;
#pragma unroll
        for (int sl = 0; sl < SL; ++sl)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[sl][e] = 0.0f;

        f32x16 s[2];                 // of the step's pairs
        Weights pw[2][2][TERMS];     // ... and their pages
        // Operands come from LDS kAhead reads ahead of the products that take them.
        constexpr int kAhead = 4;
        u32x4 operand[kAhead];
        auto read_k = [&](int buf, int i) { return *reinterpret_cast<const u32x4 *>(sh.k[buf] + i * 1024 + lane * 16); };   // pair i / KS, dims 16 (i % KS) ..
        auto read_v = [&](int buf, int i) {   // page i / SL, dims 32 (i % SL) ..
            if constexpr (TM) {
                const unsigned char *src = sh.v[buf] + (i / SL * SPEC_BLOCK_SIZE + 4 * half + (n16 >> 2)) * v_row_bytes(D) + (i % SL * 32 + 16 * (g & 1) + 4 * (n16 & 3)) * 2;
                const u32x2 a = read_transposed(src), b = read_transposed(src + 8 * v_row_bytes(D));
                return (u32x4){a.x, a.y, b.x, b.y};
            } else {
                return *reinterpret_cast<const u32x4 *>(sh.v[buf] + i * 1024 + lane * 16);
            }
        };
        // products of the K in buffer `buf` with the queries
        auto scores = [&](int buf) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[h][e] = 0.0f;
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i) {
                s[i / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, operand[i % kAhead]), q[i % KS], s[i / KS], 0, 0, 0);
                if (i + kAhead < 2 * KS) operand[i % kAhead] = read_k(buf, i + kAhead);
            }
        };
        // scores to base-2 exponents (8-bit; bf16: up to the scale, which the exponent's multiply-add applies), and the running
        // reference raised where it has fallen behind
        auto exponents = [&](int buf, int pages) {
            if constexpr (B8) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const f32x4 ks = *reinterpret_cast<const f32x4 *>(&sh.scale[buf][0][8 * i + 4 * half]);
                    const f32x4 lv = *reinterpret_cast<const f32x4 *>(&sh.scale[buf][1][8 * i + 4 * half]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[i / 4][4 * (i % 4) + r] = fmaf(s[i / 4][4 * (i % 4) + r], ks[r], lv[r]);
                }
            }
            if (pages < kStepPages) {
#pragma unroll
                for (int i = 1; i < kStepPages; ++i)
                    if (i >= pages) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) s[i / 2][8 * (i % 2) + e] = -INFINITY;
                    }
            }
            float mx = max3(s[0][0], s[0][1], s[0][2]), b = max3(s[1][0], s[1][1], s[1][2]);
#pragma unroll
            for (int e = 3; e < 15; e += 2) {
                mx = max3(mx, s[0][e], s[0][e + 1]);
                b = max3(b, s[1][e], s[1][e + 1]);
            }
            mx = max3(max3(mx, s[0][15], s[1][15]), b, b);
            mx = B8 ? mx - kTop : mx * p.scale_log2;   // (the scale is positive: the maximum commutes with it)
            const float limit = m_run + kRescaleSlack;
            if (__builtin_amdgcn_ballot_w64(mx > limit) != 0) {
                mx = max_across_xor32(mx);
                const float m_new = mx > limit ? mx : m_run;
                const float alpha = fast_exp2(m_run - m_new);
                l_run *= alpha;
#pragma unroll
                for (int sl = 0; sl < SL; ++sl) acc[sl] *= alpha;
                m_run = m_new;
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
                    const float e = fast_exp2(B8 ? x - m_run : fmaf(x, p.scale_log2, -m_run));
                    if constexpr (B8) l_run = fmaf(e, rv[r], l_run);
                    else l_run += e;
                    float rest = e;
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) {
                        pw[h][i / 2][t][4 * (i % 2) + r] = (std::conditional_t<B8, _Float16, __bf16>)rest;
                        rest -= (float)pw[h][i / 2][t][4 * (i % 2) + r];
                    }
                }
            }
        };
        // product of pair h's weights with its V in buffer `buf`
        auto product = [&](int buf, int h) {
#pragma unroll
            for (int k = 0; k < 2 * SL; ++k) {
                const int i = 2 * SL * h + k;
                const u32x4 v = operand[i % kAhead];
#pragma unroll
                for (int t = 0; t < TERMS; ++t) {
                    const Weights w8 = pw[h][k / SL][t];
                    if constexpr (B8) acc[k % SL] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, w8), acc[k % SL], 0, 0, 0);
                    else acc[k % SL] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, w8), acc[k % SL], 0, 0, 0);
                }
                if (i + kAhead < 4 * SL) operand[i % kAhead] = read_v(buf, i + kAhead);
            }
        };

        load(sh.page[my_page]);
        store(0);
        load(sh.page[kStepPages + my_page]);
        int entry_ahead = sh.page[2 * kStepPages + my_page];
        for (int u = 0; u < steps; ++u) {
            const int buf = u & 1;
            __syncthreads();        // step u is in LDS, and no wavefront reads step u - 1 any more
#pragma unroll
            for (int i = 0; i < kAhead; ++i) operand[i] = read_k(buf, i);
            store(buf ^ 1);
            load(entry_ahead);
            entry_ahead = sh.page[kStepPages * (u + 3) + my_page];
            scores(buf);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) operand[i] = read_v(buf, i);
            exponents(buf, u == steps - 1 ? last_pages : kStepPages);
            weigh(buf, 0);
            product(buf, 0);
            weigh(buf, 1);
            product(buf, 1);
        }

        // The rows' partial results, half of the dims at a time through LDS so that they go out in long pieces.
        l_run += __uint_as_float(__builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false)[half ^ 1]);
        if (half == 0 && c32 < rows)
            *reinterpret_cast<f32x2 *>(p.prefix_ml + (out_index(c32) * p.max_prefix_chunks + slot) * 2) = (f32x2){m_run, l_run};
        __syncthreads();
        unsigned char *o = sh.o[wave];
        constexpr int OP = D / 2 * 4 / 16;            // 16-byte pieces of half a row
#pragma unroll
        for (int d2 = 0; d2 < 2; ++d2) {   // (a region for each wavefront, and LDS executes a wavefront's accesses in order)
#pragma unroll
            for (int sl = 0; sl < SL / 2; ++sl)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x16 &x = acc[d2 * (SL / 2) + sl];
                    const f32x4 four = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
                    *reinterpret_cast<f32x4 *>(o + c32 * Sh::kOutRow + partial_place<D>(32 * sl + 8 * i + 4 * half) * 4) = four;
                }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
            for (int piece = lane; piece < 32 * OP; piece += kWave) {
                const int r = piece / OP, c = piece % OP;
                if (r < rows)
                    *reinterpret_cast<u32x4 *>(p.prefix_acc + (out_index(r) * p.max_prefix_chunks + slot) * D + d2 * (D / 2) + c * 4) =
                        *reinterpret_cast<const u32x4 *>(o + r * Sh::kOutRow + c * 16);
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    }
}

template <int KIND, int D, bool FULL>
hipError_t go(const CacheAttnParams &p, CacheLaunch at, hipStream_t stream)
{
    auto rows = [&](auto waves) {
        constexpr int W = decltype(waves)::value;
        hipLaunchKernelGGL((prefix_rows_kernel<KIND, D, FULL, W>), at.blocks, dim3(W * kWave), 0, stream, p);
        return hipGetLastError();
    };
    auto own = [&](auto tiles) {
        hipLaunchKernelGGL((cache_attn_kernel<KIND, decltype(tiles)::value, D, FULL>), at.blocks, dim3(kThreads), 0, stream, p, at.prefix);
        return hipGetLastError();
    };
    if (at.tiles == 0 && at.waves == 4) return rows(std::integral_constant<int, 4>());
    if constexpr (D == 128)
        if (at.tiles == 0 && at.waves == 8) return rows(std::integral_constant<int, 8>());
    if (at.tiles == 1) return own(std::integral_constant<int, 1>());
    if (at.tiles == 2) return own(std::integral_constant<int, 2>());
    if (at.tiles == 3) return own(std::integral_constant<int, 3>());
    return hipErrorInvalidValue;
}

}  // namespace

template <int KIND>
hipError_t launch_cache_kind(const CacheAttnParams &p, CacheLaunch at, hipStream_t stream)
{
    if (p.d == 128) return p.out_f32 ? go<KIND, 128, true>(p, at, stream) : go<KIND, 128, false>(p, at, stream);
    return p.out_f32 ? go<KIND, 64, true>(p, at, stream) : go<KIND, 64, false>(p, at, stream);
}
template hipError_t launch_cache_kind<SPEC_CACHE_PART>(const CacheAttnParams &p, CacheLaunch at, hipStream_t stream);

#else   // the launch functions

namespace {

hipError_t launch_kind(const CacheAttnParams &p, CacheLaunch at, hipStream_t stream)
{
    switch (p.kind) {
        case kCacheTiles: return launch_cache_kind<kCacheTiles>(p, at, stream);
        case kCacheTokens: return launch_cache_kind<kCacheTokens>(p, at, stream);
        case kCacheE4M3: return launch_cache_kind<kCacheE4M3>(p, at, stream);
        case kCacheInt8: return launch_cache_kind<kCacheInt8>(p, at, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_cache_attn(const CacheAttnParams &p, hipStream_t stream)
{
    if (p.max_prefix_chunks > 0) {
        const CacheLaunch at = p.prefix_many_rows ? CacheLaunch{dim3(p.prefix_row_blocks), 1, 0, (1 << p.prefix_rows_log2) / kPrefixRows}
                                                  : CacheLaunch{dim3(p.Hkv, p.prefix_row_blocks, p.max_prefix_chunks), 1, p.prefix_tiles, 0};
        const hipError_t err = launch_kind(p, at, stream);
        if (err != hipSuccess) return err;
    }
    return launch_kind(p, CacheLaunch{dim3(p.Hkv, p.B, p.row_blocks * p.max_chunks), 0, p.row_tiles, 0}, stream);
}

#endif

}  // namespace specv

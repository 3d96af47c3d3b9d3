// The attention weight that every cached token gets from given query rows (spec_kv_weight).
#include "code8.h"
#include "prompt_ops.h"

namespace specv {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kTileRows = 32;
constexpr int waves_of(int form) { return form == kWeightSome ? 8 : 4; }

// 32 tokens of a request and KV head are a wavefront's, or, where there are too few of them for the device (kWeightShared), a block's, whose
// wavefronts take the rows in turn.  The query rows that see any of the block's tokens pass through LDS, 64 (shared: 128) at a time, as rows: read from
// memory in operand order they would be 64 lanes in 64 cache lines each time (32 rows of four requests of 4500 .. 9400 tokens, 64/8 heads: 42 us, with rows in LDS 28, all of them at once 22).
// S[row][token] = Q[row][:] . K[token][:] with v_mfma_f32_32x32x16_bf16, K's 32 tokens held in registers: lane (half, c) holds token c,
// rows 8 i + 4 half .. + 3, so that a token's sum is the lane's own additions, one exchange with the other half, and
// (shared) four wavefronts through LDS, in a fixed order.  A tile's 16 weights of a lane are added in a few levels, and tiles, of which a long prompt has thousands, with
// what each addition loses kept (one after another, 48000 weights of about the same size lost 1e-4 of their sum, all in one direction).
// kWeightFew: at most 64 rows, a step's: they stay in LDS, and the wavefronts go through several groups of tokens whose K is asked for two groups
// ahead; nothing in between waits for a load (five rows of 64 requests, 1000 .. 3000 tokens of e4m3: 40 us for 150 MB, 3.8 TB/s; one group a block 55).
// kWeightSome: at most 256 rows, the same with eight wavefronts a block and K asked for where the group before it ends, which leaves registers for four wavefronts
// a SIMD (a group ahead: 24 us instead of 22).  Bound by the exponentials and their sums (32 rows of four requests of 4500 .. 9400 tokens: about 13 us of the 22).
template <int KIND, int D, int FORM>
__global__ __launch_bounds__(waves_of(FORM) *kWave, FORM == kWeightSome ? 4 : 2) void kv_weight_kernel(KvWeightParams p)
{
    constexpr bool B8 = is_8bit(KIND), INT8 = KIND == kCacheInt8, SHARED = FORM == kWeightShared, SOME = FORM == kWeightSome, FEW = FORM == kWeightFew || SOME;
    constexpr int kWeightWaves = waves_of(FORM);
    constexpr int kAhead = FORM == kWeightFew ? 2 : 1;     // groups whose K is asked for ahead
    constexpr int KS = D / 16, kPageBytes = SPEC_BLOCK_SIZE * D * (B8 ? 1 : 2);
    constexpr int kThreads = kWeightWaves * kWave, kRows = SOME ? kWeightSomeRows : SHARED ? 128 : kWeightFewRows, kStageTiles = kRows / kTileRows, kRowBytes = D * 2 + 16;
    constexpr int kRowPieces = D / 8, kPieces = kRows * kRowPieces / kThreads;   // 16-byte pieces of a row, of a thread
    constexpr int kBuffers = FEW ? 1 : 2;
    __shared__ alignas(16) unsigned char rows[kBuffers][kRows * kRowBytes];
    __shared__ alignas(16) float row_lse[kBuffers][kRows];
    __shared__ alignas(16) int row_limit[kBuffers][kRows];
    __shared__ float sums[SHARED ? kWeightWaves : 1][kWeightTokens];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, c32 = lane & 31;
    const int place = (int)(blockIdx.x / (unsigned)p.Hkv), kvh = (int)blockIdx.x - place * p.Hkv, b = blockIdx.y;
    const int row0 = uniform_load(p.cu_q_len, b), end = uniform_load(p.cu_q_len, b + 1), kv_len = uniform_load(p.kv_len, b);
    if (end == row0) return;
    // (kWeightFew and kWeightSome are chosen by the host's offsets: rows beyond a stage's, from others in device memory, would be lost)
    if (!offsets_fit(row0, end, p.T) || kv_len < 0 || kv_len > p.capacity_tokens || (kv_len + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE > p.max_blocks_per_req ||
        (FEW && (end - row0) * p.group > kRows)) {
        if (blockIdx.x == 0 && tid == 0 && p.errors != nullptr) atomicAdd(p.errors, 1ull);
        return;
    }
    // the block's tokens: in groups, as many as it has wavefronts times 32 (SHARED: 32)
    constexpr int kGroupTokens = (SHARED ? 1 : kWeightWaves) * kWeightTokens;
    const int most_groups = FEW ? p.groups : 1, block_t0 = place * most_groups * kGroupTokens;
    if (block_t0 >= kv_len) return;
    const int groups = min(most_groups, (kv_len - block_t0 + kGroupTokens - 1) / kGroupTokens);
    const int q_len = end - row0, past = kv_len - q_len, all_rows = q_len * p.group;
    const int all_pages = (kv_len + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE;
    const int32_t *table = p.block_table + (size_t)b * p.max_blocks_per_req;
    auto first_token = [&](int group) { return block_t0 + group * kGroupTokens + (SHARED ? 0 : wave * kWeightTokens); };   // of this wavefront's
    // This lane's token is the first one + c32.  The entries of this wavefront's pages (two a group, at most 16 groups) are asked for at once, a lane
    // each; -1: no token there, or outside the pool (page 0 is read in its place, and nothing is written).
    int entries = -1;
    {
        const int page = first_token(lane / 2) / SPEC_BLOCK_SIZE + lane % 2;
        if (lane < 2 * groups && page < all_pages) {
            entries = table[page];
            if ((unsigned)entries >= (unsigned)p.num_blocks) {
                entries = -1;
                if (kvh == 0 && p.errors != nullptr && (!SHARED || wave == 0)) atomicAdd(p.errors, 1ull);
            }
        }
    }
    auto entry_of = [&](int group) {
        const int e0 = __builtin_amdgcn_readlane(entries, 2 * group % kWave), e1 = __builtin_amdgcn_readlane(entries, (2 * group + 1) % kWave);
        return group >= groups ? -1 : c32 < SPEC_BLOCK_SIZE ? e0 : e1;
    };
    // tiles of 32 rows: the first that sees a token, and how many there are
    auto first_of = [&](int token) { return max(token - past, 0) * p.group / kTileRows; };
    const int tiles = (all_rows + kTileRows - 1) / kTileRows, stages = (tiles + kStageTiles - 1) / kStageTiles;

    u32x4 piece[kPieces];
    float lse = 0.0f;
    int limit = -1;          // a row's last visible token; -1 for rows that count nothing
    auto load_rows = [&](int stage) {
        if (stage >= stages) return;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int at = i * kThreads + tid, r = stage * kRows + at / kRowPieces, j = divide_by_group(r, p.group, p.group_inverse);
            if (r < all_rows) piece[i] = *reinterpret_cast<const u32x4 *>(static_cast<const __bf16 *>(p.q) + (size_t)(row0 + j) * p.q_stride +
                                                        (size_t)(kvh * p.group + (r - j * p.group)) * D + at % kRowPieces * 8);
        }
        if (tid < kRows) {
            const int r = stage * kRows + tid, j = divide_by_group(min(r, all_rows - 1), p.group, p.group_inverse);
            lse = p.lse[(size_t)(row0 + j) * p.Hq + kvh * p.group + (min(r, all_rows - 1) - j * p.group)];
            limit = r < all_rows && fabsf(lse) < INFINITY ? past + j : -1;
        }
    };
    auto store_rows = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int at = i * kThreads + tid;
            *reinterpret_cast<u32x4 *>(&rows[buf][at / kRowPieces * kRowBytes + at % kRowPieces * 16]) = piece[i];
        }
        if (tid < kRows) {
            row_lse[buf][tid] = limit >= 0 ? lse * kLog2e : 0.0f;
            row_limit[buf][tid] = limit;
        }
    };
    const int first_stage = FEW ? 0 : first_of(block_t0) / kStageTiles;
    load_rows(first_stage);

    // K of a group, as it lies
    constexpr int kRaw = B8 ? KS / 2 : KS;
    u32x4 raw[kAhead][kRaw];
    float raw_scale[kAhead], before[kAhead];
    auto load_k = [&](int group, int at) {
        const int entry = max(entry_of(group), 0), slot = c32 & 15;
        const size_t head = (size_t)entry * p.Hkv + kvh;
        before[at] = p.weight_in != nullptr ? p.weight_in[head * SPEC_BLOCK_SIZE + slot] : 0.0f;
        if (B8) raw_scale[at] = p.kv_scale[head * 32 + slot];
        const char *page = static_cast<const char *>(p.k_cache) + head * kPageBytes;
#pragma unroll
        for (int i = 0; i < kRaw; ++i)
            raw[at][i] = *reinterpret_cast<const u32x4 *>(page + (KIND == kCacheTokens ? slot * (D * 2) + i * 32 + half * 16 : (2 * i + half) * 256 + slot * 16));
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load_k(i, i);
    if (FEW) {
        store_rows(0);
        __syncthreads();
    }

    auto one_group = [&](int group, int at_ring) {
        const int t0 = first_token(group), last_token = min(t0 + kWeightTokens, kv_len) - 1;
        const int first_tile = t0 < kv_len ? first_of(t0) : INT32_MAX;   // this wavefront's
        const float factor = B8 ? raw_scale[at_ring] * p.scale_log2 : p.scale_log2;   // of a product, to base-2 exponents
        bf16x8 k[KS];
#pragma unroll
        for (int i = 0; i < kRaw; ++i) {
            if constexpr (B8) {   // 16 dims
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x2 lo = codes_to_bf16<INT8>(raw[at_ring][i][2 * e]), hi = codes_to_bf16<INT8>(raw[at_ring][i][2 * e + 1]);
                    k[2 * i + e] = __builtin_bit_cast(bf16x8, (u32x4){lo.x, lo.y, hi.x, hi.y});
                }
            } else {
                k[i] = __builtin_bit_cast(bf16x8, raw[at_ring][i]);
            }
        }
        const float old = before[at_ring];
        if (FEW && !SOME) load_k(group + kAhead, at_ring);
        float sum = 0.0f, lost = 0.0f;   // so far; what its additions have lost
        for (int stage = first_stage, buf = 0; stage < (FEW ? 1 : stages); ++stage, buf ^= FEW ? 0 : 1) {
            if (!FEW) {
                store_rows(buf);
                __syncthreads();     // the rows are there, and no wavefront reads the stage before any more
                if (stage + 1 < stages) load_rows(stage + 1);
            }
#pragma unroll 1
            for (int i = SHARED ? wave : 0; i < kStageTiles; i += SHARED ? kWeightWaves : 1) {
                const int at = stage * kStageTiles + i;
                if (at < first_tile || at >= tiles) continue;
                const bool all_see = __builtin_amdgcn_ballot_w64(row_limit[buf][i * kTileRows + c32] < last_token) == 0;
                const unsigned char *row = &rows[buf][(i * kTileRows + c32) * kRowBytes];
                f32x16 s;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.0f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        *reinterpret_cast<const bf16x8 *>(row + (B8 ? 64 * (ks / 2) + 32 * half + 16 * (ks % 2) : 32 * ks + 16 * half)), k[ks], s, 0, 0, 0);
                f32x4 parts;   // of the tile's 16 weights
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4) {
                    const int at4 = i * kTileRows + 8 * e4 + 4 * half;
                    const f32x4 off = *reinterpret_cast<const f32x4 *>(&row_lse[buf][at4]);
                    if (all_see) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = fast_exp2(fmaf(s[4 * e4 + e], factor, -off[e]));
                            parts[e] = e4 > 0 ? parts[e] + x : x;
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float all = fast_exp2(fmaf(s[4 * e4 + e], factor, -off[e])), x = row_limit[buf][at4 + e] >= t0 + c32 ? all : 0.0f;
                            parts[e] = e4 > 0 ? parts[e] + x : x;
                        }
                    }
                }
                const float tile = (parts[0] + parts[1]) + (parts[2] + parts[3]);
                if constexpr (FEW) {
                    sum += tile;
                } else {
                    const float add = tile - lost, next = sum + add;
                    lost = next < INFINITY ? (next - sum) - add : 0.0f;   // (rows with an lse of other scores: infinite weights stay infinite)
                    sum = next;
                }
            }
        }
        if (SOME) load_k(group + kAhead, at_ring);
        if (!FEW) sum -= lost;
        const u32x2_t both = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        sum = __uint_as_float(both[0]) + __uint_as_float(both[1]);
        if constexpr (SHARED) {   // (one group)
            if (half == 0) sums[wave][c32] = sum;
            __syncthreads();
            if (wave > 0) return;
            sum = (sums[0][c32] + sums[1][c32]) + (sums[2][c32] + sums[3][c32]);
        }
        const int t = t0 + c32, entry = entry_of(group);
        if (half == 0 && t < kv_len && entry >= 0) p.weight[((size_t)entry * p.Hkv + kvh) * SPEC_BLOCK_SIZE + c32 % SPEC_BLOCK_SIZE] = (t < past ? old : 0.0f) + sum;
    };
    if constexpr (FEW) {
        for (int group = 0; group < groups; group += kAhead)
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (group + i < groups) one_group(group + i, i);
    } else {
        one_group(0, 0);
    }
}

template <int KIND, int D>
void go(const KvWeightParams &p, hipStream_t stream)
{
    const unsigned waves = (unsigned)waves_of(p.form), each = p.form == kWeightShared ? 1u : waves * (p.form >= kWeightFew ? (unsigned)p.groups : 1u);   // times 32 tokens of a block
    const dim3 grid(((unsigned)p.max_tiles + each - 1) / each * (unsigned)p.Hkv, (unsigned)p.B), threads(waves * kWave);
    if (p.form == kWeightShared) hipLaunchKernelGGL((kv_weight_kernel<KIND, D, kWeightShared>), grid, threads, 0, stream, p);
    else if (p.form == kWeightSome) hipLaunchKernelGGL((kv_weight_kernel<KIND, D, kWeightSome>), grid, threads, 0, stream, p);
    else if (p.form == kWeightFew) hipLaunchKernelGGL((kv_weight_kernel<KIND, D, kWeightFew>), grid, threads, 0, stream, p);
    else hipLaunchKernelGGL((kv_weight_kernel<KIND, D, kWeightOwn>), grid, threads, 0, stream, p);
}
template <int KIND>
void go(const KvWeightParams &p, hipStream_t stream)
{
    if (p.d == 128) go<KIND, 128>(p, stream);
    else go<KIND, 64>(p, stream);
}

}  // namespace

hipError_t launch_kv_weight(const KvWeightParams &p, hipStream_t stream)
{
    switch (p.kind) {
    case kCacheTiles: go<kCacheTiles>(p, stream); break;
    case kCacheTokens: go<kCacheTokens>(p, stream); break;
    case kCacheE4M3: go<kCacheE4M3>(p, stream); break;
    default: go<kCacheInt8>(p, stream); break;
    }
    return hipGetLastError();
}

}  // namespace specv

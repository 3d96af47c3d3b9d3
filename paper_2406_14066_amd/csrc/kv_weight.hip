// The attention weight that every cached token gets from given query rows (spec_kv_weight).
#include "code8.h"
#include "prompt_ops.h"

namespace specv {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kWeightWaves = 4, kTileRows = 32, kTilePages = kWeightTokens / SPEC_BLOCK_SIZE;

// A block has 64 tokens of a request and KV head; its wavefronts go through the query rows that see any of them, 32 at a time, in turn.
// S[row][token] = Q[row][:] . K[token][:] with v_mfma_f32_32x32x16_bf16, K's 64 tokens held in registers: lane (half, c) holds token c of
// each 32, rows 8 i + 4 half .. + 3, so that a token's sum is the lane's own additions, one exchange with the other half, and
// four wavefronts through LDS, in a fixed order.
template <int KIND, int D>
__global__ __launch_bounds__(kWeightWaves *kWave, 2) void kv_weight_kernel(KvWeightParams p)
{
    constexpr bool B8 = is_8bit(KIND), INT8 = KIND == kCacheInt8;
    constexpr int KS = D / 16, kPageBytes = SPEC_BLOCK_SIZE * D * (B8 ? 1 : 2);
    __shared__ alignas(16) float row_lse[kWeightWaves][kTileRows];
    __shared__ alignas(16) int row_limit[kWeightWaves][kTileRows];
    __shared__ float sums[kWeightWaves][kWeightTokens];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, c32 = lane & 31;
    const int tile = (int)(blockIdx.x / (unsigned)p.Hkv), kvh = (int)blockIdx.x - tile * p.Hkv, b = blockIdx.y;
    const int row0 = uniform_load(p.cu_q_len, b), end = uniform_load(p.cu_q_len, b + 1), kv_len = uniform_load(p.kv_len, b);
    if (row0 < 0 || end <= row0 || end > p.T) return;
    if (kv_len < 0 || kv_len > p.capacity_tokens || (kv_len + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE > p.max_blocks_per_req) {
        if (blockIdx.x == 0 && tid == 0 && p.errors != nullptr) atomicAdd(p.errors, 1ull);
        return;
    }
    const int t0 = tile * kWeightTokens;
    if (t0 >= kv_len) return;
    const int q_len = end - row0, past = kv_len - q_len, all_rows = q_len * p.group;
    const int last_token = min(t0 + kWeightTokens, kv_len) - 1;

    // this lane's tokens: t0 + c32 and t0 + 32 + c32
    const int pages = (kv_len + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE - t0 / SPEC_BLOCK_SIZE;
    const int32_t *table = p.block_table + (size_t)b * p.max_blocks_per_req + t0 / SPEC_BLOCK_SIZE;
    auto entry_of = [&](int page) {   // -1: no tokens there, or outside the pool
        const int entry = page < pages ? table[page] : -1;
        return (unsigned)entry < (unsigned)p.num_blocks ? entry : -1;
    };
    float factor[2];     // of a product, to base-2 exponents
    const int first_tile = max(t0 - past, 0) * p.group / kTileRows;   // of 32 rows: the first that sees token t0
    const int tiles = (all_rows + kTileRows - 1) / kTileRows;
    bf16x8 k[2][KS];
    if (first_tile + wave < tiles) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int entry = entry_of(2 * h + (c32 >> 4)), slot = c32 & 15;
            const char *page = static_cast<const char *>(p.k_cache) + ((size_t)max(entry, 0) * p.Hkv + kvh) * kPageBytes;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                u32x4 x = {0, 0, 0, 0};
                if (entry >= 0) {
                    if constexpr (B8) {
                        const u32x2 codes = *reinterpret_cast<const u32x2 *>(page + ks * 256 + slot * 16 + half * 8);
                        const u32x2 lo = codes_to_bf16<INT8>(codes.x), hi = codes_to_bf16<INT8>(codes.y);
                        x = (u32x4){lo.x, lo.y, hi.x, hi.y};
                    } else if constexpr (KIND == kCacheTiles) {
                        x = *reinterpret_cast<const u32x4 *>(page + (2 * ks + half) * 256 + slot * 16);
                    } else {
                        x = *reinterpret_cast<const u32x4 *>(page + slot * (D * 2) + ks * 32 + half * 16);
                    }
                }
                k[h][ks] = __builtin_bit_cast(bf16x8, x);
            }
            factor[h] = p.scale_log2;
            if constexpr (B8) factor[h] *= entry >= 0 ? p.kv_scale[((size_t)entry * p.Hkv + kvh) * 32 + slot] : 0.0f;
        }
    }

    float sum[2] = {0.0f, 0.0f};
    bf16x8 q[KS];
    float lse = 0.0f;
    auto load_rows = [&](int rows_at) {
        const int r = min(rows_at * kTileRows + c32, all_rows - 1), j = divide_by_group(r, p.group, p.group_inverse);
        const int head = kvh * p.group + (r - j * p.group);
        const __bf16 *row = static_cast<const __bf16 *>(p.q) + (size_t)(row0 + j) * p.q_stride + (size_t)head * D;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const bf16x8 *>(row + 16 * ks + 8 * half);
        lse = p.lse[(size_t)(row0 + j) * p.Hq + head];
    };
    if (first_tile + wave < tiles) load_rows(first_tile + wave);
    for (int at = first_tile + wave; at < tiles; at += kWeightWaves) {
        // the rows' log-sum-exp and last visible token; -1 for rows that count nothing
        const int r = at * kTileRows + c32;
        const bool counts = r < all_rows && fabsf(lse) < INFINITY;
        const int limit = counts ? past + divide_by_group(r, p.group, p.group_inverse) : -1;
        if (half == 0) {
            row_lse[wave][c32] = counts ? lse * kLog2e : 0.0f;
            row_limit[wave][c32] = limit;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const bool all_see = __builtin_amdgcn_ballot_w64(limit < last_token) == 0;
        f32x16 s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[h][e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int h = 0; h < 2; ++h) s[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q[ks], k[h][ks], s[h], 0, 0, 0);
        f32x4 off[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) off[i] = *reinterpret_cast<const f32x4 *>(&row_lse[wave][8 * i + 4 * half]);
        if (at + kWeightWaves < tiles) load_rows(at + kWeightWaves);
        if (all_see) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[h] += fast_exp2(fmaf(s[h][e], factor[h], -off[e / 4][e % 4]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int most = row_limit[wave][8 * i + 4 * half + e] - t0 - c32;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float x = fast_exp2(fmaf(s[h][4 * i + e], factor[h], -off[i][e]));
                        sum[h] += 32 * h <= most ? x : 0.0f;
                    }
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const u32x2_t x = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[h]), __float_as_uint(sum[h]), false, false);
        if (half == 0) sums[wave][32 * h + c32] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    __syncthreads();
    if (tid < kWeightTokens) {
        const int t = t0 + tid, entry = entry_of(tid / SPEC_BLOCK_SIZE);
        if (t < kv_len && entry >= 0) {
            const size_t at = ((size_t)entry * p.Hkv + kvh) * SPEC_BLOCK_SIZE + tid % SPEC_BLOCK_SIZE;
            const float before = p.weight_in != nullptr && t < past ? p.weight_in[at] : 0.0f;
            p.weight[at] = before + ((sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]));
        }
        if (kvh == 0 && p.errors != nullptr && tid < kTilePages && tid < pages && entry_of(tid) < 0) atomicAdd(p.errors, 1ull);
    }
}

template <int KIND>
void go(const KvWeightParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)p.max_tiles * (unsigned)p.Hkv, (unsigned)p.B);
    if (p.d == 128) hipLaunchKernelGGL((kv_weight_kernel<KIND, 128>), grid, dim3(kWeightWaves * kWave), 0, stream, p);
    else hipLaunchKernelGGL((kv_weight_kernel<KIND, 64>), grid, dim3(kWeightWaves * kWave), 0, stream, p);
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

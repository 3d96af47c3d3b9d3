// Eviction: a request's tokens with the largest weights, its first and its latest ones go into other pages (spec_kv_evict).
// Three launches: scores, the choice (a block per request), the copies.
#include "device_util.h"
#include "prompt_ops.h"

namespace specv {

namespace {

constexpr int kScoreWaves = 4, kChoiceThreads = 1024, kChoiceWaves = kChoiceThreads / kWave, kCopyWaves = 4;

// (The library flushes fp32's denormals, and weights may be: their conversions to 64 bits and back are done on the bits.)
__device__ __forceinline__ double wide(float x)
{
    const uint32_t bits = __float_as_uint(x);
    if ((bits & 0x7F800000u) != 0) return (double)x;
    const double v = (double)(bits & 0x7FFFFFu) * 0x1p-149;
    return bits >> 31 ? -v : v;
}
// A score as a word that orders like it, 0 for NaN: the sum rounded to fp32, both zeros alike.
__device__ __forceinline__ uint32_t ordered(double x)
{
    if (!(x == x)) return 0;
    uint32_t bits;
    if (fabs(x) < 0x1p-126) bits = (uint32_t)rint(fabs(x) * 0x1p149) | (x < 0.0 ? 0x80000000u : 0u);
    else bits = __float_as_uint((float)x);
    if (bits == 0x80000000u) bits = 0;
    return bits >> 31 ? ~bits : bits | 0x80000000u;
}

// What a request's lengths come to; false: they do not fit.
struct Choice {
    int n, keep, first, recent;
};
__device__ __forceinline__ bool choice_of(const KvEvictParams &p, int b, Choice &c)
{
    const int n = uniform_load(p.kv_len, b), keep = uniform_load(p.keep, b);
    if (n < 0 || n > p.capacity_tokens || (n + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE > p.max_blocks_per_req || keep < 0) return false;
    c.n = n;
    c.keep = min(n, keep);
    if ((c.keep + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE > p.dst_max_blocks) return false;
    c.first = min(p.first, c.keep);
    c.recent = min(p.recent, c.keep - c.first);
    return true;
}

// A wavefront takes four pages, a lane a token: the KV heads' weights in order.  Bound by the bytes, and by latency where they are few.
__global__ __launch_bounds__(kScoreWaves *kWave) void evict_score_kernel(KvEvictParams p)
{
    const int lane = threadIdx.x % kWave, b = blockIdx.y, t = (blockIdx.x * kScoreWaves + threadIdx.x / kWave) * kWave + lane;
    Choice c;
    if (!choice_of(p, b, c) || t >= c.n || c.n == c.keep) return;
    const int entry = p.block_table[(size_t)b * p.max_blocks_per_req + t / SPEC_BLOCK_SIZE];
    uint32_t key = 0;
    if ((unsigned)entry < (unsigned)p.num_blocks) {
        const float *from = p.weight + (size_t)entry * p.Hkv * SPEC_BLOCK_SIZE + t % SPEC_BLOCK_SIZE;
        double sum = 0.0;
#pragma unroll 8
        for (int h = 0; h < p.Hkv; ++h) sum += wide(from[h * SPEC_BLOCK_SIZE]);
        key = ordered(sum);
    }
    p.score[(size_t)b * p.score_stride + t] = key;
}

// A block per request: the smallest score that stays is found digit by digit (8 bits each, the largest first) from counts; then the
// tokens are gone through in order, and those that stay find their places from running counts of the scores above and at the smallest
// one (of which the earliest stay).
__global__ __launch_bounds__(kChoiceThreads) void evict_choice_kernel(KvEvictParams p)
{
    __shared__ int count[kChoiceWaves][256];
    __shared__ int total[256];
    __shared__ uint32_t wave_sum[2][kChoiceWaves];
    __shared__ uint32_t found_digit;
    __shared__ int found_rest;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, b = blockIdx.x;
    const int width = p.dst_max_blocks * SPEC_BLOCK_SIZE;
    int32_t *chosen = p.chosen + (size_t)b * width, *kept = p.kept != nullptr ? p.kept + (size_t)b * width : nullptr;
    Choice c;
    const bool ok = choice_of(p, b, c);
    if (tid == 0) {
        p.new_kv_len[b] = ok ? c.keep : -1;
        if (!ok && p.errors != nullptr) atomicAdd(p.errors, 1ull);
    }
    if (kept != nullptr)
        for (int i = (ok ? c.keep : 0) + tid; i < width; i += kChoiceThreads) kept[i] = -1;
    if (!ok) return;
    if (c.keep == c.n) {
        for (int i = tid; i < c.n; i += kChoiceThreads) {
            chosen[i] = i;
            if (kept != nullptr) kept[i] = i;
        }
        return;
    }
    const uint32_t *score = p.score + (size_t)b * p.score_stride;
    const int lo = c.first, hi = c.n - c.recent;
    int rest = c.keep - c.first - c.recent;   // of the tokens lo .. hi - 1, fewer than there are
    uint32_t least = 0;                       // the digits found
    if (rest > 0) {
        for (int digit = 0; digit < 4; ++digit) {
            const int shift = 24 - 8 * digit;
            for (int i = tid; i < kChoiceWaves * 256; i += kChoiceThreads) (&count[0][0])[i] = 0;
            __syncthreads();
            for (int i = lo + tid; i < hi; i += kChoiceThreads) {
                const uint32_t s = score[i];
                if (digit == 0 || s >> (shift + 8) == least) atomicAdd(&count[wave][s >> shift & 255u], 1);
            }
            __syncthreads();
            if (tid < 256) {
                int sum = 0;
#pragma unroll
                for (int w = 0; w < kChoiceWaves; ++w) sum += count[w][tid];
                total[tid] = sum;
            }
            __syncthreads();
            if (wave == 0) {   // lane l has the digits 255 - 4 l .. 252 - 4 l
                int mine[4], sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += mine[e] = total[255 - 4 * lane - e];
                int upto = sum;
                for (int step = 1; step < kWave; step *= 2) {
                    const int other = __shfl_up(upto, step);
                    if (lane >= step) upto += other;
                }
                int above = upto - sum;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (above < rest && above + mine[e] >= rest) {
                        found_digit = 255 - 4 * lane - e;
                        found_rest = rest - above;
                    }
                    above += mine[e];
                }
            }
            __syncthreads();
            least = least << 8 | found_digit;
            rest = found_rest;
        }
    }
    // scores above `least` stay, and the first `rest` that equal it (none where only protected tokens stay)
    const bool any = c.keep > c.first + c.recent;
    int above = 0, equal = 0;    // so far
    for (int base = 0, turn = 0; base < c.n; base += 4 * kChoiceThreads, turn ^= 1) {
        const int i0 = base + 4 * tid;
        uint32_t flags = 0;      // bit e: stays; bit 4 + e: equals
        uint32_t mine = 0;       // counts: stays << 16 | equals
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = i0 + e;
            if (i >= c.n) continue;
            bool stays = i < lo || i >= hi, same = false;
            if (!stays && any) {
                const uint32_t s = score[i];
                stays = s > least;
                same = s == least;
            }
            flags |= (stays ? 1u : 0u) << e | (same ? 16u : 0u) << e;
            mine += (stays ? 0x10000u : 0u) + (same ? 1u : 0u);
        }
        uint32_t upto = mine;
        for (int step = 1; step < kWave; step *= 2) {
            const uint32_t other = __shfl_up(upto, step);
            if (lane >= step) upto += other;
        }
        if (lane == kWave - 1) wave_sum[turn][wave] = upto;
        __syncthreads();
        uint32_t before = upto - mine, all = 0;
#pragma unroll
        for (int w = 0; w < kChoiceWaves; ++w) {
            const uint32_t x = wave_sum[turn][w];
            if (w < wave) before += x;
            all += x;
        }
        int a = above + (int)(before >> 16), q = equal + (int)(before & 0xFFFFu);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool stays = flags >> e & 1u, same = flags >> (4 + e) & 1u;
            if (stays || (same && q < rest)) {
                const int place = a + min(q, rest);
                chosen[place] = i0 + e;
                if (kept != nullptr) kept[place] = i0 + e;
            }
            a += stays;
            q += same;
        }
        above += (int)(all >> 16);
        equal += (int)(all & 0xFFFFu);
    }
}

// A wavefront per (page filled, KV head): 16 tokens from wherever they are.  K's 16-byte pieces hold one token each in every layout, so do
// token-major V's; a tiled V's 16-byte cell holds four tokens, which are picked from their four cells.  Cells that the last page does not fill go out
// element by element, so that what lies behind the last token stays as it was.
__global__ __launch_bounds__(kCopyWaves *kWave) void evict_copy_kernel(KvEvictParams p)
{
    const int lane = threadIdx.x % kWave, b = blockIdx.y, s = lane & 15, g = lane >> 4;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * kCopyWaves + threadIdx.x / kWave);
    const int index = unit / p.Hkv, kvh = unit - index * p.Hkv;
    if (index >= p.dst_max_blocks) return;
    const int keep = uniform_load(p.new_kv_len, b), here = min(keep - index * SPEC_BLOCK_SIZE, SPEC_BLOCK_SIZE);
    if (here <= 0) return;
    const int to = uniform_load(p.dst_block_table + (size_t)b * p.dst_max_blocks, index);
    if ((unsigned)to >= (unsigned)p.num_blocks) {
        if (kvh == 0 && lane == 0 && p.errors != nullptr) atomicAdd(p.errors, (unsigned long long)here);
        return;
    }
    // lane s % 16: where token s comes from
    int from = -1, slot = 0;
    if (s < here) {
        const int t = p.chosen[((size_t)b * p.dst_max_blocks + index) * SPEC_BLOCK_SIZE + s];
        from = p.block_table[(size_t)b * p.max_blocks_per_req + t / SPEC_BLOCK_SIZE];
        slot = t % SPEC_BLOCK_SIZE;
        if ((unsigned)from >= (unsigned)p.num_blocks) from = -1;
        const unsigned long long bad = __builtin_amdgcn_ballot_w64(from < 0) & 0xFFFFull;
        if (bad != 0 && kvh == 0 && lane == 0 && p.errors != nullptr) atomicAdd(p.errors, (unsigned long long)__builtin_popcountll(bad));
    }
    const int esz = p.kv_dtype == SPEC_F32 ? 4 : p.kv_dtype == SPEC_BF16 ? 2 : 1;
    const bool tiled = p.kv_dtype == SPEC_E4M3 || p.kv_dtype == SPEC_INT8 || p.kv_layout == SPEC_KV_MFMA;
    const int page_bytes = SPEC_BLOCK_SIZE * p.d * esz, pieces = p.d * esz / 16;   // 16-byte pieces of a token
    const size_t head_to = (size_t)to * p.Hkv + kvh, head_from = (size_t)max(from, 0) * p.Hkv + kvh;
    const u32x4 none = {0, 0, 0, 0};
    auto copy_pieces = [&](void *pool, bool by_piece) {
        unsigned char *base = static_cast<unsigned char *>(pool), *page = base + head_to * page_bytes;
        if (by_piece) {          // [piece][token]: lane (piece, token)
            if (s < here)
                for (int c = g; c < pieces; c += 4)
                    *reinterpret_cast<u32x4 *>(page + (c * SPEC_BLOCK_SIZE + s) * 16) =
                        from < 0 ? none : *reinterpret_cast<const u32x4 *>(base + head_from * page_bytes + (c * SPEC_BLOCK_SIZE + slot) * 16);
        } else {                 // [token][piece]: consecutive lanes, consecutive pieces
            for (int i = lane; i < SPEC_BLOCK_SIZE * pieces; i += kWave) {
                const int token = i / pieces, c = i - token * pieces;
                const int f = __shfl(from, token), sl = __shfl(slot, token);
                if (token < here)
                    *reinterpret_cast<u32x4 *>(page + (token * pieces + c) * 16) =
                        f < 0 ? none : *reinterpret_cast<const u32x4 *>(base + ((size_t)f * p.Hkv + kvh) * page_bytes + (sl * pieces + c) * 16);
            }
        }
    };
    copy_pieces(p.k_cache, tiled);
    if (!tiled) {
        copy_pieces(p.v_cache, false);
    } else {
        // lane (g, s): the cells of tokens 4 g .. + 3, place s of 16
        unsigned char *base = static_cast<unsigned char *>(p.v_cache), *page = base + head_to * page_bytes;
        const unsigned char *cell[4];
        int at[4];
        bool there[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int f = __shfl(from, 4 * g + e), sl = __shfl(slot, 4 * g + e);
            there[e] = f >= 0;
            cell[e] = base + ((size_t)max(f, 0) * p.Hkv + kvh) * page_bytes + (sl / 4 * 16 + s) * 16;
            at[e] = sl % 4;
        }
        const int n = min(max(here - 4 * g, 0), 4);   // of the lane's four tokens
        for (int i = 0; i < page_bytes / 1024; ++i) {
            u32x4 x[4], out = none;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = there[e] ? *reinterpret_cast<const u32x4 *>(cell[e] + i * 1024) : none;
            unsigned char *dst = page + i * 1024 + (g * 16 + s) * 16;
            if (esz == 1) {      // [4 dims][4 tokens]
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t v = x[e][q] >> 8 * at[e] & 0xFFu;
                        out[q] |= v << 8 * e;
                        if (n < 4 && e < n) dst[4 * q + e] = (unsigned char)v;
                    }
            } else {             // [2 dims][4 tokens]
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t word = at[e] / 2 ? x[e][2 * h + 1] : x[e][2 * h], v = word >> 16 * (at[e] & 1) & 0xFFFFu;
                        out[2 * h + e / 2] |= v << 16 * (e & 1);
                        if (n < 4 && e < n) *reinterpret_cast<uint16_t *>(dst + 8 * h + 2 * e) = (uint16_t)v;
                    }
            }
            if (n == 4) *reinterpret_cast<u32x4 *>(dst) = out;
        }
    }
    if (s < here) {
        if (p.kv_scale != nullptr && g < 2) p.kv_scale[head_to * 32 + g * 16 + s] = from < 0 ? 0.0f : p.kv_scale[head_from * 32 + g * 16 + slot];
        if (g == 2) p.weight[head_to * SPEC_BLOCK_SIZE + s] = from < 0 ? 0.0f : p.weight[head_from * SPEC_BLOCK_SIZE + slot];
    }
}

}  // namespace

hipError_t launch_kv_evict(const KvEvictParams &p, hipStream_t stream)
{
    const unsigned B = (unsigned)p.B;
    constexpr int kScoreTokens = kScoreWaves * kWave;
    hipLaunchKernelGGL(evict_score_kernel, dim3(p.capacity_tokens / kScoreTokens + 1, B), dim3(kScoreTokens), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(evict_choice_kernel, dim3(B), dim3(kChoiceThreads), 0, stream, p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(evict_copy_kernel, dim3((unsigned)(((int64_t)p.dst_max_blocks * p.Hkv + kCopyWaves - 1) / kCopyWaves), B), dim3(kCopyWaves * kWave), 0, stream, p);
    return hipGetLastError();
}

}  // namespace specv

// Eviction: a request's tokens with the largest weights, its first and its latest ones go into other pages (spec_kv_evict).
// Three launches: scores, the choice (a block per request), the copies; short requests' choices make their scores themselves.
#include "device_util.h"
#include "prompt_ops.h"

namespace specv {

namespace {

constexpr int kScoreWaves = 4, kChoiceThreads = kEvictTurn / 4, kChoiceWaves = kChoiceThreads / kWave, kCopyWaves = 4;

constexpr uint32_t kNoScore = 1, kProtected = 0xFFFFFFFFu;   // below and above every score; 0: no token there

// A score as a word that orders like it, kNoScore for NaN: the sum rounded to fp32, both zeros alike.
__device__ __forceinline__ uint32_t ordered(double x)
{
    if (!(x == x)) return kNoScore;
    uint32_t bits = __float_as_uint((float)x);   // (this file is compiled with fp32's denormals: small weights are told apart)
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

__device__ __forceinline__ uint32_t score_of(const KvEvictParams &p, int entry, int slot)
{
    if ((unsigned)entry >= (unsigned)p.num_blocks) return kNoScore;
    const float *from = p.weight + (size_t)entry * p.Hkv * SPEC_BLOCK_SIZE + slot;
    double sum = 0.0;
#pragma unroll 8
    for (int h = 0; h < p.Hkv; ++h) sum += (double)from[h * SPEC_BLOCK_SIZE];
    return ordered(sum);
}

// Where the score of token t is handed over: the choice's threads have 4 * held tokens side by side of each 4096 * held and read them 16 bytes a thread at a time.
__device__ __forceinline__ int score_place(int t, int held)
{
    const int per = 4 * held, all = per * kChoiceThreads, segment = t / all, in = t - segment * all, thread = in / per, e = in - thread * per;
    return segment * all + (e / 4 * kChoiceThreads + thread) * 4 + e % 4;
}

// A wavefront takes four pages, a lane a token: the KV heads' weights in order.  Bound by the bytes, and by latency where they are few.
__global__ __launch_bounds__(kScoreWaves *kWave) void evict_score_kernel(KvEvictParams p)
{
    const int lane = threadIdx.x % kWave, b = blockIdx.y, t = (blockIdx.x * kScoreWaves + threadIdx.x / kWave) * kWave + lane;
    Choice c;
    if (!choice_of(p, b, c) || t >= c.n || c.n == c.keep) return;
    p.score[(size_t)b * p.score_stride + score_place(t, p.held)] = score_of(p, p.block_table[(size_t)b * p.max_blocks_per_req + t / SPEC_BLOCK_SIZE], t % SPEC_BLOCK_SIZE);
}

// A block per request: the smallest score that stays is found from counts over 2048 even parts of the interval that it lies in, first that of all
// scores, then the part in which it was found, and so on (three times at the most, fewer where all of a part stays); then the tokens that stay find their places from the numbers,
// before them, of scores above it and at it (of which the earliest stay).  A thread has 4 * HELD tokens side by side; they are in
// registers throughout, or, longer requests (LONG), fetched again for each pass.  HELD == 1 makes the scores itself.
// What is handed to the copies is where a token lies: page * 16 + slot, -1 outside the pool.
// Additions to one counter in LDS go one after another, which is why the parts are even: counts by the scores' leading 8 or 11 bits, which are of
// a few binary orders, took 44 us for 16 requests of 8500 .. 30000 tokens, votes (no counters, two bits a pass) 76.
template <int HELD, bool LONG>
__global__ __launch_bounds__(kChoiceThreads) void evict_choice_kernel(KvEvictParams p)
{
    constexpr int kBins = 2048, kCopies = 4, kPer = 4 * HELD, kSegment = kPer * kChoiceThreads;
    __shared__ alignas(16) int count[kCopies][kBins];
    __shared__ int wave_sum[2][2][kChoiceWaves];
    __shared__ uint32_t wave_least[kChoiceWaves], wave_most[kChoiceWaves];
    __shared__ int found_digit, found_rest;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, b = blockIdx.x;
    const int width = p.dst_max_blocks * SPEC_BLOCK_SIZE;
    int32_t *chosen = p.chosen + (size_t)b * width, *kept = p.kept != nullptr ? p.kept + (size_t)b * width : nullptr;
    const int32_t *table = p.block_table + (size_t)b * p.max_blocks_per_req;
    Choice c;
    const bool ok = choice_of(p, b, c);
    if (tid == 0) {
        p.new_kv_len[b] = ok ? c.keep : -1;
        if (!ok && p.errors != nullptr) atomicAdd(p.errors, 1ull);
    }
    if (kept != nullptr)
        for (int i = (ok ? c.keep : 0) + tid; i < width; i += kChoiceThreads) kept[i] = -1;
    if (!ok) return;
    auto put = [&](int place, int t, int entry) {
        chosen[place] = (unsigned)entry < (unsigned)p.num_blocks ? entry * SPEC_BLOCK_SIZE + t % SPEC_BLOCK_SIZE : -1;
        if (kept != nullptr) kept[place] = t;
    };
    if (c.keep == 0) return;
    if (c.keep == c.n) {
        for (int i = tid; i < c.n; i += kChoiceThreads) put(i, i, table[i / SPEC_BLOCK_SIZE]);
        return;
    }
    const uint32_t *score = p.score + (size_t)b * p.score_stride;   // (rows begin at multiples of 16 bytes)
    const int lo = c.first, hi = c.n - c.recent, segments = LONG ? (c.n + kSegment - 1) / kSegment : 1;
    uint32_t x[kPer];
    auto fetch = [&](int segment) {
        const int i0 = segment * kSegment + tid * kPer;
        if constexpr (HELD == 1) {
            const int entry = i0 < c.n ? table[i0 / SPEC_BLOCK_SIZE] : -1;
            double sum[4] = {0.0, 0.0, 0.0, 0.0};
            const float *from = p.weight + (size_t)max(entry, 0) * p.Hkv * SPEC_BLOCK_SIZE + i0 % SPEC_BLOCK_SIZE;
            const bool inside = (unsigned)entry < (unsigned)p.num_blocks;
            if (inside) {
#pragma unroll 8
                for (int h = 0; h < p.Hkv; ++h) {
                    const f32x4 w = *reinterpret_cast<const f32x4 *>(from + h * SPEC_BLOCK_SIZE);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] += (double)w[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = inside ? ordered(sum[e]) : kNoScore;
        } else {
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                const u32x4 v = *reinterpret_cast<const u32x4 *>(score + segment * kSegment + (k * kChoiceThreads + tid) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * k + e] = v[e];
            }
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) x[e] = i0 + e >= c.n ? 0 : i0 + e < lo || i0 + e >= hi ? kProtected : x[e];
    };
    if (!LONG) fetch(0);
    int rest = c.keep - c.first - c.recent;   // of the scores in the interval least .. least + span; fewer than there are
    uint32_t least = kProtected - 1, span = 0;
    if (rest > 0) {
        uint32_t most = 0;
        for (int segment = 0; segment < segments; ++segment) {
            if (LONG) fetch(segment);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                least = min(least, x[e] - 1);                        // (no place: 0, which becomes the largest)
                most = max(most, x[e] == kProtected ? 0u : x[e]);
            }
        }
#pragma unroll
        for (int step = 1; step < kWave; step *= 2) {
            least = min(least, (uint32_t)__shfl_xor((int)least, step));
            most = max(most, (uint32_t)__shfl_xor((int)most, step));
        }
        if (lane == 0) {
            wave_least[wave] = least;
            wave_most[wave] = most;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kChoiceWaves; ++w) {
            least = min(least, wave_least[w]);
            most = max(most, wave_most[w]);
        }
        least += 1;
        span = most - least;
#pragma unroll 1
        for (;;) {
            const int shift = max(21 - (span != 0 ? __builtin_clz(span) : 32), 0);   // span >> shift < 2048
            for (int i = tid; i < kCopies * kBins / 4; i += kChoiceThreads) reinterpret_cast<u32x4 *>(&count[0][0])[i] = (u32x4){0, 0, 0, 0};
            __syncthreads();
            int *mine_count = count[wave % kCopies];
            for (int segment = 0; segment < segments; ++segment) {
                if (LONG) fetch(segment);
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (x[e] - least <= span) atomicAdd(&mine_count[(x[e] - least) >> shift], 1);
            }
            __syncthreads();
            // thread t has the parts 2047 - 2 t and 2046 - 2 t
            int mine[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                mine[e] = 0;
#pragma unroll
                for (int w = 0; w < kCopies; ++w) mine[e] += count[w][kBins - 1 - 2 * tid - e];
            }
            int upto = mine[0] + mine[1];
#pragma unroll
            for (int step = 1; step < kWave; step *= 2) {
                const int other = __shfl_up(upto, step);
                if (lane >= step) upto += other;
            }
            if (lane == kWave - 1) wave_sum[0][0][wave] = upto;
            __syncthreads();
            int over = upto - mine[0] - mine[1];
#pragma unroll
            for (int w = 0; w < kChoiceWaves; ++w)
                if (w < wave) over += wave_sum[0][0][w];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (over < rest && over + mine[e] >= rest) {
                    found_digit = kBins - 1 - 2 * tid - e;
                    found_rest = over + mine[e] == rest ? 0 : rest - over;
                }
                over += mine[e];
            }
            __syncthreads();
            const uint32_t from = (uint32_t)found_digit << shift;
            least += from;
            span = min(span - from, (1u << shift) - 1u);
            rest = found_rest;
            if (rest == 0) {   // all of the part stays: whatever is above the score before its first
                least -= 1;
                break;
            }
            if (shift == 0) break;
            __syncthreads();   // (found_* and the counts have been read)
        }
    }
    // scores above `least` stay, and the first `rest` that equal it
    int above = 0, equal = 0;    // so far
    for (int segment = 0; segment < segments; ++segment) {
        if (LONG) fetch(segment);
        int more = 0, same = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            more += x[e] > least;
            same += x[e] == least;
        }
        int more_upto = more, same_upto = same;
#pragma unroll
        for (int step = 1; step < kWave; step *= 2) {
            const int m = __shfl_up(more_upto, step), q = __shfl_up(same_upto, step);
            if (lane >= step) {
                more_upto += m;
                same_upto += q;
            }
        }
        if (lane == kWave - 1) {
            wave_sum[segment & 1][0][wave] = more_upto;
            wave_sum[segment & 1][1][wave] = same_upto;
        }
        __syncthreads();
        int a = above + more_upto - more, q = equal + same_upto - same;
#pragma unroll
        for (int w = 0; w < kChoiceWaves; ++w) {
            const int m = wave_sum[segment & 1][0][w], s = wave_sum[segment & 1][1][w];
            if (w < wave) {
                a += m;
                q += s;
            }
            above += m;
            equal += s;
        }
        const int i0 = segment * kSegment + tid * kPer;
        int entry = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (e % SPEC_BLOCK_SIZE == 0 && i0 + e < c.n) entry = table[(i0 + e) / SPEC_BLOCK_SIZE];   // (kPer divides a page or is a multiple of it)
            const bool stays = x[e] > least, ties = x[e] == least;
            if (stays || (ties && q < rest)) put(a + min(q, rest), i0 + e, entry);
            a += stays;
            q += ties;
        }
    }
}

// A wavefront per (page filled, KV head): 16 tokens from wherever they are.  K's 16-byte pieces hold one token each in every layout, so do
// token-major V's; a tiled V's 16-byte cell holds four tokens, which are picked from their four cells.  Cells that the last page does not fill go out
// element by element, so that what lies behind the last token stays as it was.
// Bound by the cache lines that the tokens lie in: 4096 of 8500 .. 30000 tokens of 16 requests, 8 heads, e4m3: 117 us, about four fifths of the pages' lines in and 138 MB out.
__global__ __launch_bounds__(kCopyWaves *kWave) void evict_copy_kernel(KvEvictParams p)
{
    const int lane = threadIdx.x % kWave, b = blockIdx.y, s = lane & 15, g = lane >> 4;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * kCopyWaves + threadIdx.x / kWave);
    const int index = unit / p.Hkv, kvh = unit - index * p.Hkv;
    if (index >= p.dst_max_blocks) return;
    // (all asked for before the first is looked at)
    const int keep = uniform_load(p.new_kv_len, b), to = uniform_load(p.dst_block_table + (size_t)b * p.dst_max_blocks, index);
    const int place = p.chosen[((size_t)b * p.dst_max_blocks + index) * SPEC_BLOCK_SIZE + s];
    const int here = min(keep - index * SPEC_BLOCK_SIZE, SPEC_BLOCK_SIZE);
    if (here <= 0) return;
    if ((unsigned)to >= (unsigned)p.num_blocks) {
        if (kvh == 0 && lane == 0 && p.errors != nullptr) atomicAdd(p.errors, (unsigned long long)here);
        return;
    }
    // lane s % 16: where token s comes from
    const int from = s < here && place >= 0 ? place / SPEC_BLOCK_SIZE : -1, slot = place & (SPEC_BLOCK_SIZE - 1);
    if (kvh == 0 && p.errors != nullptr) {
        const unsigned long long bad = __builtin_amdgcn_ballot_w64(s < here && from < 0) & 0xFFFFull;
        if (bad != 0 && lane == 0) atomicAdd(p.errors, (unsigned long long)__builtin_popcountll(bad));
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
    hipError_t e;
    // Short requests' choices make their scores: a launch less.  (A block reads the weights of 4096 tokens in about the time that a launch takes.)
    if (p.held > 1) {
        hipLaunchKernelGGL(evict_score_kernel, dim3(p.capacity_tokens / kScoreTokens + 1, B), dim3(kScoreTokens), 0, stream, p);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.held == 1) hipLaunchKernelGGL((evict_choice_kernel<1, false>), dim3(B), dim3(kChoiceThreads), 0, stream, p);
    else if (p.held == 4) hipLaunchKernelGGL((evict_choice_kernel<4, false>), dim3(B), dim3(kChoiceThreads), 0, stream, p);
    else if (p.capacity_tokens <= p.held * kEvictTurn) hipLaunchKernelGGL((evict_choice_kernel<8, false>), dim3(B), dim3(kChoiceThreads), 0, stream, p);
    else hipLaunchKernelGGL((evict_choice_kernel<8, true>), dim3(B), dim3(kChoiceThreads), 0, stream, p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(evict_copy_kernel, dim3((unsigned)(((int64_t)p.dst_max_blocks * p.Hkv + kCopyWaves - 1) / kCopyWaves), B), dim3(kCopyWaves * kWave), 0, stream, p);
    return hipGetLastError();
}

}  // namespace specv

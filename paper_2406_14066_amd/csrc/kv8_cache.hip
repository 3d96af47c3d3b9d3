// The 8-bit KV cache: rows are quantised as they enter the pages (spec_kv8_append), and tokens are read back as
// rows (spec_kv8_read).  Formats and page layout: spec_verify.h.
#include "code8.h"

#include <type_traits>

namespace specv {

namespace {

constexpr int kPageWaves = 4;

// What a wavefront of a kernel that goes by pages works on.
struct PageWork {
    int b, kvh, first;    // request, KV head, packed row of slot 0 (negative where the tokens begin later in the page)
    int s0, s1;           // slots [s0, s1) hold the request's tokens
    int page;             // -1: position or table entry out of range
};

// tokens `pos0 .. pos0 + n - 1` of request b are packed rows row0 .. row0 + n - 1; `i`: the how-many-th page they touch
__device__ __forceinline__ bool place_page(PageWork &w, int pos0, int n, int row0, int i, const int32_t *table, int max_blocks, int num_blocks)
{
    // (a negative first position, from lengths that do not fit, rounds towards minus infinity)
    const int index = (pos0 >> 4) + i;
    const int begin = index * SPEC_BLOCK_SIZE;
    w.s0 = max(pos0 - begin, 0);
    w.s1 = min(pos0 + n - begin, SPEC_BLOCK_SIZE);
    if (w.s0 >= w.s1) return false;
    w.first = row0 + begin - pos0;
    w.page = -1;
    if (index >= 0 && index < max_blocks) {
        const int page = table[(size_t)w.b * max_blocks + index];
        if ((unsigned)page < (unsigned)num_blocks) w.page = page;
    }
    return true;
}

// Append: a wavefront per (page that a request's rows touch, KV head).  Lane (s, g) = (lane % 16, lane / 16) takes token slot s,
// dims g D/4 .. + D/4 - 1: a token's maximum is one exchange between four lanes.  K's codes are 16-byte pieces of the page
// as they are; V's, four tokens to a word, are transposed between the lanes of a quad and gathered through LDS into the page's
// 16-byte cells (4 tokens of 4 dims), which go out whole where all four tokens are new and by halves and bytes of words where some
// are not (their old neighbours stay untouched without being read).
// Rows of long prompts are bound by the bytes (16000 tokens, 8 heads, d = 128, bf16 rows inside a fused projection: 64 MB in 13.7 us,
// 4.7 TB/s; 16.0 with V's words stored one by one), a step's five rows of 256 requests by the chain lengths -> table -> rows -> stores and the partly written lines
// (8.4 us; an empty launch takes 3.8, one row of one request 5).
template <typename T, bool INT8, int D>
__global__ __launch_bounds__(kPageWaves *kWave) void kv8_append_kernel(Kv8AppendParams p, int items)
{
    constexpr int N = D / 4;        // dims per lane
    __shared__ alignas(16) unsigned char stage[kPageWaves][SPEC_BLOCK_SIZE * D];
    constexpr float kMost = INT8 ? kMaxInt8 : kMaxE4M3;
    const int lane = threadIdx.x % kWave, s = lane & 15, g = lane >> 4;
    const int unit = (int)(blockIdx.x * kPageWaves + threadIdx.x / kWave);
    const int item = __builtin_amdgcn_readfirstlane(unit / p.Hkv);
    if (item >= items) return;   // (the wavefronts of a block are independent)
    PageWork w;
    w.kvh = __builtin_amdgcn_readfirstlane(unit - item * p.Hkv);
    w.b = request_of_item(p.cu_q_len, p.B, item, items);
    const int row0 = p.cu_q_len[w.b], end = p.cu_q_len[w.b + 1], n = end - row0;
    if (row0 < 0 || end <= row0 || end > p.T) return;
    const int pos0 = p.kv_len[w.b] - n;
    if (!place_page(w, pos0, n, row0, item - page_item(row0, w.b), p.block_table, p.max_blocks_per_req, p.num_blocks)) return;

    const bool on = s >= w.s0 && s < w.s1;
    const int64_t from = (int64_t)(w.first + (on ? s : w.s0)) * p.token_stride + w.kvh * D + g * N;
    constexpr int kPieces = N * (int)sizeof(T) / 16, kPer = 16 / (int)sizeof(T);
    u32x4 raw[2][kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) raw[0][i] = *reinterpret_cast<const u32x4 *>(static_cast<const T *>(p.new_k) + from + i * kPer);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) raw[1][i] = *reinterpret_cast<const u32x4 *>(static_cast<const T *>(p.new_v) + from + i * kPer);
    if (w.page < 0) {
        if (w.kvh == 0 && lane == 0 && p.errors != nullptr) atomicAdd(p.errors, (unsigned long long)(w.s1 - w.s0));
        return;
    }

    const size_t head = (size_t)w.page * p.Hkv + w.kvh;
    float scale[2];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        f32x4 x[N / 4];
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const uint32_t word = raw[kv][e / kPer][e % kPer * (int)sizeof(T) / 4];
            const uint32_t bits = sizeof(T) == 4 ? word : e % 2 == 0 ? word << 16 : word & 0xFFFF0000u;
            x[e / 4][e % 4] = __uint_as_float(bits);
            most = max(most, bits & 0x7FFFFFFFu);   // magnitudes order as integers, infinities and NaN last
        }
        {   // over the token's four lanes
            u32x2_t r = __builtin_amdgcn_permlane16_swap(most, most, false, false);
            most = max(r[0], r[1]);
            r = __builtin_amdgcn_permlane32_swap(most, most, false, false);
            most = max(r[0], r[1]);
        }
        const bool finite = most < 0x7F800000u;
        const float a = fmaxf(__uint_as_float(most), kSmallestRow);
        // (the two quotients as products with rounded reciprocals, as fp32 tensor arithmetic does them: codes at a tie agree with it;
        // 1 / a as 2^8 times itself, which has the same bits and is a normal number for every a: above 2^126 1 / a is not, and denormals
        // are flushed)
        scale[kv] = finite ? a * (1.0f / kMost) : __uint_as_float(0x7FC00000u);
        const float inv = kMost * 0x1p-8f * (1.0f / (a * 0x1p-8f));
        uint32_t code[N / 4];
#pragma unroll
        for (int j = 0; j < N / 4; ++j) {
            code[j] = f32_to_codes<INT8>(x[j] * inv);
            if (!finite) code[j] = 0;
        }
        if (kv == 0) {
            unsigned char *page = p.k_cache + head * (SPEC_BLOCK_SIZE * D);
            if (on) {
#pragma unroll
                for (int j = 0; j < N / 16; ++j)
                    *reinterpret_cast<u32x4 *>(page + (g * (N / 16) + j) * 256 + s * 16) =
                        (u32x4){code[4 * j], code[4 * j + 1], code[4 * j + 2], code[4 * j + 3]};
            }
        } else {
            // after the transposition lane (s, g) holds, per j, dim g N + 4 j + s % 4 of the tokens s & ~3 .. + 3
            unsigned char *page = p.v_cache + head * (SPEC_BLOCK_SIZE * D), *st = stage[threadIdx.x / kWave];
            const int a4 = s & 3;
#pragma unroll
            for (int j = 0; j < N / 4; ++j) {
                const int dim = g * N + 4 * j + a4;
                *reinterpret_cast<uint32_t *>(st + ((dim / 64 * 4 + (s >> 2)) * 16 + dim % 16) * 16 + dim % 64 / 16 * 4) = transpose_quad(code[j], a4);
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            // lane (n, g) takes the cells of tokens 4 g .. + 3: those from t0 up to t1 are new
            const int t0 = min(max(w.s0 - 4 * g, 0), 4), t1 = min(max(w.s1 - 4 * g, 0), 4);
            const bool whole = t0 == 0 && t1 == 4, low = t0 == 0 && t1 >= 2, high = t0 <= 2 && t1 == 4;   // both tokens of a half
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                const u32x4 cell = *reinterpret_cast<const u32x4 *>(st + i * 1024 + lane * 16);
                unsigned char *at = page + i * 1024 + lane * 16;
                if (whole) {
                    *reinterpret_cast<u32x4 *>(at) = cell;
                } else if (t0 < t1) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (low) *reinterpret_cast<uint16_t *>(at + 4 * e) = (uint16_t)cell[e];
                        else if (t0 == 0) at[4 * e] = (unsigned char)cell[e];
                        else if (t0 == 1) at[4 * e + 1] = (unsigned char)(cell[e] >> 8);
                        if (high) *reinterpret_cast<uint16_t *>(at + 4 * e + 2) = (uint16_t)(cell[e] >> 16);
                        else if (t0 <= 2 && t1 == 3) at[4 * e + 2] = (unsigned char)(cell[e] >> 16);
                        else if (t0 == 3) at[4 * e + 3] = (unsigned char)(cell[e] >> 24);
                    }
                }
            }
        }
    }
    if (on && g < 2) p.kv_scale[head * 32 + g * 16 + s] = g == 0 ? scale[0] : scale[1];
}

// Read: a wavefront per (page, KV head).  Codes come in as they lie, and go through LDS as values, a row per token, so
// that the rows go out whole and past the caches.  Bound by the bytes: 32 requests of 500 .. 8000 tokens, 8 heads, d = 128, to bf16:
// 673 MB in 119 us, 5.7 TB/s, more than a device copy's 5.1.
template <typename T, bool INT8, int D>
__global__ __launch_bounds__(kPageWaves *kWave) void kv8_read_kernel(Kv8ReadParams p, int items)
{
    constexpr int kRow = D * sizeof(T) + 16;   // bytes of a token row in LDS
    __shared__ alignas(16) unsigned char stage[kPageWaves][SPEC_BLOCK_SIZE * kRow];
    const int lane = threadIdx.x % kWave, n16 = lane & 15, g = lane >> 4;
    const int unit = (int)(blockIdx.x * kPageWaves + threadIdx.x / kWave);
    const int item = __builtin_amdgcn_readfirstlane(unit / p.Hkv);
    if (item >= items) return;   // (the wavefronts of a block are independent)
    PageWork w;
    w.kvh = __builtin_amdgcn_readfirstlane(unit - item * p.Hkv);
    w.b = request_of_item(p.cu_len, p.B, item, items);
    const int row0 = p.cu_len[w.b], end = p.cu_len[w.b + 1], n = end - row0;
    if (row0 < 0 || end <= row0 || end > p.T) return;
    const int pos0 = p.start != nullptr ? p.start[w.b] : 0;
    if (!place_page(w, pos0, n, row0, item - page_item(row0, w.b), p.block_table, p.max_blocks_per_req, p.num_blocks)) return;
    if (w.page < 0 && w.kvh == 0 && lane == 0 && p.errors != nullptr) atomicAdd(p.errors, (unsigned long long)(w.s1 - w.s0));
    const bool there = w.page >= 0;
    const size_t head = (size_t)(there ? w.page : 0) * p.Hkv + w.kvh;
    const unsigned char *kp = p.k_cache + head * (SPEC_BLOCK_SIZE * D), *vp = p.v_cache + head * (SPEC_BLOCK_SIZE * D);
    const float *sc = p.kv_scale + head * 32;
    u32x4 k[D / 64], v[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        k[i] = *reinterpret_cast<const u32x4 *>(kp + i * 1024 + lane * 16);   // token n16, dims 64 i + 16 g .. + 15
        v[i] = *reinterpret_cast<const u32x4 *>(vp + i * 1024 + lane * 16);   // tokens 4 g .. + 3, dims 64 i + 16 q + n16
    }
    if (!there) {   // (not some other page times zero: that page may hold anything)
#pragma unroll
        for (int i = 0; i < D / 64; ++i) k[i] = v[i] = (u32x4){0u, 0u, 0u, 0u};
    }
    const float ks = there ? sc[n16] : 0.0f;
    const f32x4 vs = there ? *reinterpret_cast<const f32x4 *>(sc + 16 + 4 * g) : (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    unsigned char *st = stage[threadIdx.x / kWave];
    auto put = [&](int token, int dim, f32x4 x) {   // four dims of a token
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4 *>(st + token * kRow + dim * 4) = x;
        } else {
            *reinterpret_cast<bf16x4 *>(st + token * kRow + dim * 2) = __builtin_convertvector(x, bf16x4);
        }
    };
    auto rows_out = [&](void *out) {
        constexpr int kLanes = D * sizeof(T) / 16;   // lanes per row
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int i = 0; i < SPEC_BLOCK_SIZE * kLanes / kWave; ++i) {
            const int piece = i * kWave + lane, token = piece / kLanes, part = piece % kLanes;
            if (token >= w.s0 && token < w.s1)
                __builtin_nontemporal_store(*reinterpret_cast<const u32x4 *>(st + token * kRow + part * 16),
                                            reinterpret_cast<u32x4 *>(static_cast<T *>(out) +
                                                                      ((size_t)(w.first + token) * p.Hkv + w.kvh) * D + part * (16 / sizeof(T))));
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) put(n16, 64 * i + 16 * g + 4 * j, codes_to_f32<INT8>(k[i][j]) * ks);
    rows_out(p.out_k);
    const int a4 = n16 & 3;
    const float vsa = a4 == 0 ? vs[0] : a4 == 1 ? vs[1] : a4 == 2 ? vs[2] : vs[3];
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)   // after the transposition: token 4 g + n16 % 4, dims 64 i + 16 q + (n16 & ~3) .. + 3
            put(4 * g + a4, 64 * i + 16 * q + (n16 & ~3), codes_to_f32<INT8>(transpose_quad(v[i][q], a4)) * vsa);
    rows_out(p.out_v);
}

template <typename F>
void by_type(bool f32, bool int8, int d, F go)
{
    if (f32) {
        if (int8) { if (d == 128) go(0.0f, std::true_type(), std::integral_constant<int, 128>()); else go(0.0f, std::true_type(), std::integral_constant<int, 64>()); }
        else { if (d == 128) go(0.0f, std::false_type(), std::integral_constant<int, 128>()); else go(0.0f, std::false_type(), std::integral_constant<int, 64>()); }
    } else {
        if (int8) { if (d == 128) go(__bf16(), std::true_type(), std::integral_constant<int, 128>()); else go(__bf16(), std::true_type(), std::integral_constant<int, 64>()); }
        else { if (d == 128) go(__bf16(), std::false_type(), std::integral_constant<int, 128>()); else go(__bf16(), std::false_type(), std::integral_constant<int, 64>()); }
    }
}

}  // namespace

hipError_t launch_kv8_append(const Kv8AppendParams &p, hipStream_t stream)
{
    const int items = page_item(p.T, p.B);
    const unsigned blocks = (unsigned)(((int64_t)items * p.Hkv + kPageWaves - 1) / kPageWaves);
    by_type(p.src_f32 != 0, p.int8 != 0, p.d, [&](auto type, auto int8, auto d) {
        hipLaunchKernelGGL((kv8_append_kernel<decltype(type), decltype(int8)::value, decltype(d)::value>), dim3(blocks),
                           dim3(kPageWaves * kWave), 0, stream, p, items);
    });
    return hipGetLastError();
}

hipError_t launch_kv8_read(const Kv8ReadParams &p, hipStream_t stream)
{
    const int items = page_item(p.T, p.B);
    const unsigned blocks = (unsigned)(((int64_t)items * p.Hkv + kPageWaves - 1) / kPageWaves);
    by_type(p.out_f32 != 0, p.int8 != 0, p.d, [&](auto type, auto int8, auto d) {
        hipLaunchKernelGGL((kv8_read_kernel<decltype(type), decltype(int8)::value, decltype(d)::value>), dim3(blocks),
                           dim3(kPageWaves * kWave), 0, stream, p, items);
    });
    return hipGetLastError();
}

}  // namespace specv

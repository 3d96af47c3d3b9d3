// 8-bit codes of the cache and the matrix operands they become.
#pragma once

#include "cache_ops.h"
#include "device_util.h"

namespace specv {

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Four codes (bytes) as fp32.
template <bool INT8>
__device__ __forceinline__ f32x4 codes_to_f32(uint32_t w)
{
    if constexpr (INT8)
        return (f32x4){(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)};
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return (f32x4){lo.x, lo.y, hi.x, hi.y};
}

// ... as bf16.  Exact: 4 (8) significant bits fit bf16's 8.
template <bool INT8>
__device__ __forceinline__ u32x2 codes_to_bf16(uint32_t w)
{
    if constexpr (INT8) {
        const f32x4 x = codes_to_f32<true>(w);
        // the upper halves of two fp32 side by side
        return (u32x2){__builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u),
                       __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u)};
    }
    return (u32x2){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true))};
}

// ... as fp16, exact too.
template <bool INT8>
__device__ __forceinline__ u32x2 codes_to_f16(uint32_t w)
{
    if constexpr (INT8) {
        // 0x6400 | u is 1024 + u in fp16, u = code + 128
        const uint32_t u = w ^ 0x80808080u;
        const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
        const f16x2 lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - bias;
        const f16x2 hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - bias;
        return (u32x2){__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
    }
    return (u32x2){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true))};
}

// Four fp32 that are codes already scaled, to bytes: nearest, ties to even; a product that was rounded past the
// largest code is brought back to it.
template <bool INT8>
__device__ __forceinline__ uint32_t f32_to_codes(f32x4 x)
{
    if constexpr (INT8) {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w |= ((uint32_t)(int)fminf(fmaxf(__builtin_rintf(x[e]), -kMaxInt8), kMaxInt8) & 0xFFu) << (8 * e);
        return w;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = fminf(fmaxf(x[e], -kMaxE4M3), kMaxE4M3);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
}

// The request that holds packed row `row`: the first guess is right where all requests have as many rows.
__device__ __forceinline__ int request_of(const int32_t *cu, int B, int row, int guess)
{
    if (cu[guess] <= row && row < cu[guess + 1]) return guess;
    int lo = 0, hi = B - 1;   // largest b with cu[b] <= row; of equal ones the last, which is the one with rows
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu[mid] <= row) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Work of a kernel that goes by pages: request b owns the items page_item(cu[b], b) .. page_item(cu[b+1], b+1) - 1, which are
// enough for n = cu[b+1] - cu[b] tokens from any position: those touch at most n / 16 + 2 pages.
__host__ __device__ __forceinline__ int page_item(int packed, int b) { return packed / SPEC_BLOCK_SIZE + 2 * b; }

// The request that owns an item: the last one whose first item is not beyond it.  A wavefront asks 64 places at a time: those about
// the place where it is if all requests are alike, then all of them at even distances (256 requests: two more loads one after
// another, where halving takes eight).
__device__ __forceinline__ int request_of_item(const int32_t *cu, int B, int item, int items)
{
    const int lane = threadIdx.x % kWave;
    if (B > kWave) {
        const int base = min(max((int)((int64_t)item * B / items) - kWave / 2, 0), B - kWave), at = base + lane;
        const int count = __builtin_popcountll(__builtin_amdgcn_ballot_w64(page_item(cu[at], at) <= item));
        if (count > 0 && (count < kWave || base == B - kWave)) return base + count - 1;
    }
    int lo = 0, n = B;
    while (n > 1) {
        const int stride = (n + kWave - 1) / kWave, at = lo + lane * stride;
        const bool begun = lane * stride < n && page_item(cu[min(at, B - 1)], at) <= item;
        const int count = max(__builtin_popcountll(__builtin_amdgcn_ballot_w64(begun)), 1);
        lo += (count - 1) * stride;
        n = min(stride, n - (count - 1) * stride);
    }
    return lo;
}

// Transposes the 4 x 4 bytes that the four lanes of a quad hold: lane a gets byte a of each lane's word, in lane order.
__device__ __forceinline__ uint32_t transpose_quad(uint32_t w, int a)
{
    const uint32_t w0 = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, 0x00, 0xF, 0xF, true);
    const uint32_t w1 = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, 0x55, 0xF, 0xF, true);
    const uint32_t w2 = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, 0xAA, 0xF, 0xF, true);
    const uint32_t w3 = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, 0xFF, 0xF, 0xF, true);
    const uint32_t pick = 0x0C0C0400u + (uint32_t)a * 0x0101u;   // bytes {second operand's a, first's a, zero, zero}
    const uint32_t lo = __builtin_amdgcn_perm(w1, w0, pick), hi = __builtin_amdgcn_perm(w3, w2, pick);
    return lo | (hi << 16);
}

}  // namespace

}  // namespace specv

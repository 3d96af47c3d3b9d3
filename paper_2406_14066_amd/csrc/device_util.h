// Device helpers shared by the kernels of this library.
#pragma once

#include "common.h"

namespace specv {

namespace {

constexpr int kBufferFlags = 0x00020000;   // raw 32-bit buffer descriptor, word 3
// Cache policy of the loads that stream data read once (KV pages, the race's logit rows):
// non-temporal, i.e. the lines are first in line for replacement in the L2.  Without it the
// stream pushes out what the blocks do come back to (code, block tables, queries, hand-off
// words); measured on the four large workloads the hint alone takes 8-10% off the step.
constexpr int kStreamPolicy = 2;           // "nt" bit of a raw buffer load

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Exchanges between the four 16-lane rows of a wavefront with the gfx950 row-swap instructions
// (vector ALU, a few cycles) instead of a round trip through the LDS crossbar, which is what a
// generic lane shuffle by 16 or 32 compiles to: v_permlane16_swap trades the odd rows of its
// first operand with the even rows of its second, v_permlane32_swap the upper half of the first
// with the lower half of the second.  Fed the same value twice, the two results hold, in every
// lane l, the values of lanes l and l ^ 16 (l ^ 32).
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float max_across_xor16(float v)
{
    const u32x2_t r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_across_xor32(float v)
{
    const u32x2_t r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_across_rows(float v)   // over lanes l, l ^ 16, l ^ 32, l ^ 48
{
    u32x2_t r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// One gfx950 transposing LDS read: the 16 lanes of a row give the addresses of a 4 x 16 block of 16-bit
// elements, 8 bytes each (lane n: block row n / 4, elements 4 (n % 4) .. + 3), and lane n receives block
// column n.
typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x2 read_transposed(const unsigned char *src)
{
    typedef __attribute__((address_space(3))) s16x4 *lds_s16x4_ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)src));
}

// ---------------------------------------------------------------------------
// Tickets.  Word = generation << 32 | arrivals.  Returns how many blocks arrived
// before this one.  The common case is one atomic add: the word carries this call's
// generation already.  The first arrivals of a call find something else (garbage, the
// zero its last user left, or either plus what other early arrivals added) and replace
// it; the last arrival, which is the one the merge waits for, is never among them.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t ticket_arrive(unsigned long long *ticket, uint32_t generation)
{
    const unsigned long long got = atomicAdd(ticket, 1ull);
    if ((uint32_t)(got >> 32) == generation) return (uint32_t)got;
    unsigned long long cur = got + 1ull;
    for (;;) {
        const unsigned long long first = ((unsigned long long)generation << 32) | 1ull;
        const unsigned long long seen = atomicCAS(ticket, cur, first);
        if (seen == cur) return 0u;
        if ((uint32_t)(seen >> 32) == generation) return (uint32_t)atomicAdd(ticket, 1ull);
        cur = seen;
    }
}

__device__ __forceinline__ void ticket_reset(unsigned long long *ticket)
{
    __hip_atomic_store(ticket, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Data handed from one block to another inside the launch (chunk partials, row
// statistics) is written and read with relaxed agent-scope atomic accesses, which
// go past the non-coherent cache levels, and published by waiting for the
// writes to complete before the ticket is taken.  A full agent-scope fence would
// also write back and invalidate the whole L2 of the XCD on every block; that is
// far too slow for thousands of blocks.
__device__ __forceinline__ void publish_u64(unsigned long long *dst, unsigned long long v)
{
    __hip_atomic_store(dst, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ unsigned long long fetch_u64(const unsigned long long *src)
{
    return __hip_atomic_load(src, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ unsigned long long pack_f32x2(float a, float b)
{
    return (unsigned long long)__float_as_uint(a) | ((unsigned long long)__float_as_uint(b) << 32);
}

// A 32-bit payload and the call's generation tag in one 8-byte word: written and read
// atomically, so a reader that finds this call's tag also has the payload, with no
// ordering needed between the words of a record.
__device__ __forceinline__ void publish_tagged(unsigned long long *dst, uint32_t payload, uint32_t generation)
{
    publish_u64(dst, (unsigned long long)payload | ((unsigned long long)generation << 32));
}

__device__ __forceinline__ bool tagged_ok(unsigned long long word, uint32_t generation)
{
    return (uint32_t)(word >> 32) == generation;
}

__device__ __forceinline__ void writes_complete()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);  // every outstanding store of this wavefront has been acknowledged
}

__device__ __forceinline__ void order_after_ticket()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

// Read-only inputs indexed by a block-uniform value (lengths, row offsets) are read through
// the constant address space, which makes them scalar loads: they are served by the scalar
// cache (these arrays are small and every block reads them) instead of a round trip to
// the L2 under load, and they have a wait counter of their own.
typedef const int32_t __attribute__((address_space(4))) *uniform_i32_ptr;
__device__ __forceinline__ int uniform_load(const int32_t *base, int index)
{
    return ((uniform_i32_ptr)(uintptr_t)base)[__builtin_amdgcn_readfirstlane(index)];
}

}  // namespace

}  // namespace specv

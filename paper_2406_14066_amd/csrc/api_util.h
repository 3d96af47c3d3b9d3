// Host helpers of the C entry points.
#pragma once

#include "common.h"

namespace specv {

namespace {

constexpr size_t kAlign = 256;
constexpr int64_t kMaxPacked = (int64_t)1 << 30;   // packed (token, head) rows and work items are 32-bit in the kernels

int compute_units()
{
    static int cached = 0;
    if (cached == 0) {
        int dev = 0, n = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1)
            n = 256;   // MI355X
        cached = n;
    }
    return cached;
}

bool aligned(const void *ptr, uintptr_t to) { return (reinterpret_cast<uintptr_t>(ptr) & (to - 1)) == 0; }
int pages_of(int64_t tokens) { return (int)((tokens + SPEC_BLOCK_SIZE - 1) / SPEC_BLOCK_SIZE); }
size_t align_up(size_t n) { return (n + kAlign - 1) & ~(kAlign - 1); }

// cu[0] = 0 <= cu[1] <= ... <= cu[n] = total
bool prefix_sum_ok(const int32_t *cu, int n, int total)
{
    if (cu[0] != 0 || cu[n] != total) return false;
    for (int i = 0; i < n; ++i)
        if (cu[i + 1] < cu[i]) return false;
    return true;
}

}  // namespace

}  // namespace specv

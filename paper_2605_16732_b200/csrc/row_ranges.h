// Whether tensors given by address, rows and stride can share memory.  Plain C++.
#pragma once
#include <stdint.h>

namespace dirotq {

// Whether the rows [0, rows) of `width` bytes at `stride` bytes from a, and the rows of b, can share a byte: their whole ranges are compared,
// and where both have the same stride, the columns as well.
inline bool rows_overlap(const void* a, long long rows_a, long long width_a, long long stride_a, const void* b, long long rows_b, long long width_b,
                         long long stride_b) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    const uintptr_t a1 = a0 + static_cast<uintptr_t>((rows_a - 1) * stride_a + width_a), b1 = b0 + static_cast<uintptr_t>((rows_b - 1) * stride_b + width_b);
    if (a1 <= b0 || b1 <= a0) return false;
    if (stride_a == stride_b) {
        const uintptr_t s = static_cast<uintptr_t>(stride_a);
        const uintptr_t off = (b0 >= a0 ? b0 - a0 : s - (a0 - b0) % s) % s;  // b's columns relative to a's
        if (off >= static_cast<uintptr_t>(width_a) && off + static_cast<uintptr_t>(width_b) <= s) return false;
    }
    return true;
}

}  // namespace dirotq

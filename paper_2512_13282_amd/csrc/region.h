// region.h -- operands as the entry points check them on the host, before any HIP call.
#pragma once

#include <stdint.h>

namespace gemm {

constexpr int64_t kMaxSize = int64_t(1) << 55;      // sizes and stride products stay in 64-bit byte offsets

// One operand: rows of `used` bytes at a stride of `stride` bytes from `p`.
struct Region {
    uintptr_t p;
    int64_t rows, used, stride;
    int64_t align;
    bool empty() const { return rows <= 0 || used <= 0; }
    bool valid() const {
        if (empty()) return true;
        if (p == 0 || p % uintptr_t(align) != 0 || stride < used) return false;
        return rows <= kMaxSize && stride <= kMaxSize / rows;
    }
    uint64_t span() const { return empty() ? 0 : uint64_t((rows - 1) * stride + used); }
    bool overlaps(const Region &o) const {
        return !empty() && !o.empty() && p < o.p + o.span() && o.p < p + span();
    }
};

inline Region region(const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t esize) {
    // Strides past the limit and negative ones, whose bytes may not fit 64 bits, become ones that valid() refuses.
    const bool big = ld > kMaxSize || cols > kMaxSize;
    return Region{reinterpret_cast<uintptr_t>(p), rows, big ? kMaxSize : cols * esize, big ? kMaxSize + 1 : ld < 0 ? -1 : ld * esize, esize};
}

}  // namespace gemm

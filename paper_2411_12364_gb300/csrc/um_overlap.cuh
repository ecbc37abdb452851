// um_overlap.cuh -- whether an output of a call shares memory with its inputs.
#pragma once

#include <stdint.h>

namespace um {

// A tensor's memory: `rows` runs of `bytes`, `step` bytes apart.
struct Memory {
    const void *at;             // null: no tensor
    int64_t bytes;
    int64_t rows = 1, step = 0;

    bool contiguous() const { return rows <= 1 || step == bytes; }
    int64_t total() const { return bytes * rows; }
};

// whether `a`, which is contiguous, and `b` have a byte in common
inline bool overlap(const Memory &a, const Memory &b) {
    if (!a.at || !b.at || a.total() <= 0 || b.total() <= 0) return false;
    const uintptr_t lo = (uintptr_t)a.at, hi = lo + a.total(), start = (uintptr_t)b.at;
    // the first run of b that ends behind lo
    int64_t i = 0;
    if (lo >= start + b.bytes) {
        if (b.rows <= 1) return false;
        i = (int64_t)((lo - start - b.bytes) / (uintptr_t)b.step) + 1;
    }
    return i < b.rows && start + (uintptr_t)(i * b.step) < hi;
}

// whether `a` is `b` itself, or shares nothing with it
inline bool same_or_apart(const Memory &a, const Memory &b) {
    return !overlap(a, b) || (a.at == b.at && b.contiguous() && a.total() == b.total());
}

}  // namespace um

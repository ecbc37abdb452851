// um_overlap.cuh -- whether an output of a call shares memory with its inputs.
#pragma once

#include <stdint.h>

#include <initializer_list>

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

// Whether two tensors of rows have a byte in common.  Rows of one lie in the
// gaps between rows of the other when both step alike (slices of one tensor's
// rows); with other steps the whole ranges have to be apart, or one of the
// tensors contiguous.
inline bool rows_overlap(const Memory &a, const Memory &b) {
    if (a.contiguous()) return overlap(a, b);
    if (b.contiguous()) return overlap(b, a);
    if (!a.at || !b.at || a.bytes <= 0 || b.bytes <= 0) return false;
    const uintptr_t a0 = (uintptr_t)a.at, b0 = (uintptr_t)b.at;
    const uintptr_t a1 = a0 + (uintptr_t)((a.rows - 1) * a.step + a.bytes);
    const uintptr_t b1 = b0 + (uintptr_t)((b.rows - 1) * b.step + b.bytes);
    if (a1 <= b0 || b1 <= a0) return false;
    if (a.step != b.step) return true;
    // where a row of the later tensor starts within the earlier one's step
    const Memory &lo = a0 <= b0 ? a : b, &hi = a0 <= b0 ? b : a;
    const int64_t at = (int64_t)((uintptr_t)hi.at - (uintptr_t)lo.at) % a.step;
    return at < lo.bytes || at + hi.bytes > a.step;
}

// Whether a call's outputs (contiguous) share no memory with one another or
// with its inputs.
inline bool apart(std::initializer_list<Memory> outputs, std::initializer_list<Memory> inputs) {
    for (const Memory *o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Memory *p = outputs.begin(); p != o; ++p)
            if (overlap(*o, *p)) return false;
        for (const Memory &in : inputs)
            if (overlap(*o, in)) return false;
    }
    return true;
}

// whether `a` is `b` itself, or shares nothing with it
inline bool same_or_apart(const Memory &a, const Memory &b) {
    return !overlap(a, b) || (a.at == b.at && b.contiguous() && a.total() == b.total());
}

}  // namespace um

// um_planes.cuh -- rows as the copies to planes read them (um_ce.cu), on the
// host as well, where a test puts a matrix at the end of its memory.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

namespace um {

// 8 entries of a row as they are stored
template <typename T> struct Piece {
    uint4 x[sizeof(T) / 2];
};

// The entries c .. c + 7 of a row of D, c a multiple of 8: nothing past the row is
// read, and zeros stand for it.  `wide`: D is a multiple of 8 and rows start on
// 16 bytes, so that a piece lies in the row as a whole or not at all.
template <typename T>
__host__ __device__ __forceinline__ Piece<T> read_piece(const T *row, int c, int D, bool wide) {
    Piece<T> p = {};
    if (c >= D) return p;
    if (wide) {
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
            p.x[i] = reinterpret_cast<const uint4 *>(row + c)[i];
    } else {
        T v[8];
        for (int k = 0; k < 8; ++k) v[k] = c + k < D ? row[c + k] : T(0.f);
        memcpy(&p, v, sizeof v);
    }
    return p;
}

}  // namespace um

// um_norm.cu -- the norms before and after a block, fused with the block's
// gate and the residual scale, and their gradient.
//
//   z = N_post(y),  u = res_scale r + out_scale gate (.) z,  n = N_pre(u)
//
// closes one block (its output y, the residual stream r) and opens the next
// one (the new stream u, the next input n).  N is x rstd w (rms, rstd =
// 1 / sqrt(mean x^2 + eps)) or (x - mean) rstd w + b (layer, the population
// variance under the root).
//
// What bounds it: every entry of y and r is read once and every entry of u
// and n written once, about 30 operations apart, so the bound is memory.  A
// row lies in the registers of one warp (up to 256 entries) or one block (in
// the gradient, which needs 128 registers a thread, past 4096 entries a cluster
// of two), 8 entries a thread, between its two norms.
// The rows' sums are chains of barriers, so the bytes in flight must not
// depend on them: each thread copies its own 16-byte pieces of the next rows
// into shared memory (cp.async), two or three rows ahead, and waits for its own copies
// only.  Blocks are persistent, so that the gains, biases and the per-channel
// gate are read once per block, into registers.  Measured at 16384 x 2048 in
// bf16 with a full gate: 57 us forward, 5.9 TB/s of what has to move; the
// gradient with a channel gate 80 us, 5.0 TB/s.  These two keep everything in
// registers.  LayerNorm spills: forward rows of 512 and 1024 threads 64 to 120
// bytes of stores, others up to 36; gradients to 76, of odd widths to 196.
#include "um_device.cuh"
#include "um_internal.cuh"
#include "um_overlap.cuh"
#include "um_pair.cuh"
#include "um_tc.cuh"

namespace um {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kSumSlots = 32 * 4;   // warps of a row x values of a sum

struct NormArgs {
    const void *y, *r, *gate;      // r: the residual (forward), u as stored (backward)
    const void *du, *dn;           // backward: gradients of u and n, either may be null
    const float *w_post, *b_post, *w_pre, *b_pre;
    void *u, *n;                   // forward outputs (n null without the second norm)
    void *dy, *dr, *dgate_rows;    // backward outputs; dgate of a token or full gate
    float *part;                   // backward: [blocks][n_cols][D] column partial sums
    int64_t T, ld_y, ld_r, ld_du, ld_dn;
    int D, post, pre, gate_mode;
    float res_scale, out_scale, eps;
};

// ---- a row in registers ------------------------------------------------
// Thread t of the NT CL threads of a row holds 8 entries as 4 pairs.  Rows on
// 16-byte boundaries (kRun): one run, entries 8 t.., in one or two 16-byte
// accesses.  Rows on 4-byte boundaries (kWord: any fp32 row, bf16 rows of even
// width): 4-byte words t + NT CL i, so that a warp's accesses are still
// consecutive.  Other bf16 rows (kHalf; every second row of an odd width
// starts inside a word): the same pairs of entries, from the one or two words
// that hold them.
enum { kRun = 16, kWord = 4, kHalf = 2 };
constexpr int kP = 4;

template <typename T, int MODE, int TPR> __device__ __forceinline__ int col_of(int t, int e) {
    if constexpr (MODE == kRun) return 8 * t + e;
    if constexpr (sizeof(T) == 2) return 2 * (t + TPR * (e >> 1)) + (e & 1);
    return t + TPR * e;
}

__device__ __forceinline__ void widen(F2 (&x)[kP], const uint4 *q, __nv_bfloat16) {
    const uint32_t w[4] = {q[0].x, q[0].y, q[0].z, q[0].w};
#pragma unroll
    for (int i = 0; i < kP; ++i)
        x[i] = f2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ void widen(F2 (&x)[kP], const uint4 *q, float) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[2 * i] = f2(__uint_as_float(q[i].x), __uint_as_float(q[i].y));
        x[2 * i + 1] = f2(__uint_as_float(q[i].z), __uint_as_float(q[i].w));
    }
}

// the pair as stored
__device__ __forceinline__ uint32_t pack(F2 x) {
    const float2 v = split(x);
    const __nv_bfloat162 b = __floats2bfloat162_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t *>(&b);
}
__device__ __forceinline__ F2 as_stored(F2 x, __nv_bfloat16) {
    const uint32_t w = pack(x);
    return f2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ F2 as_stored(F2 x, float) { return x; }

// Rows in flight ahead of the one at work.  At 16384 x 2048 in bf16 the
// forward took 60.2 us with two and 61.4 with three (57 with two since), the
// gradient 80.4 and 78.2 (fp32 and odd rows of 4096 entries leave room for two): the blocks of
// an SM together keep enough bytes in flight.
constexpr int kAhead = 2;
template <typename T, int MODE>
constexpr int kAheadBack = sizeof(T) == 2 && MODE != kHalf ? 3 : 2;

// A thread's way to the rows of up to MAXK tensors: a ring of its own copies
// in shared memory.  THREADS: of the block.  Addresses are kept per tensor and
// advanced from row to row.
template <typename T, int MODE, int NT, int CL, int THREADS, int S, int MAXK> struct Feed {
    static constexpr int kTpr = NT * CL;
    static constexpr int kBytes = MODE == kRun ? 16 : 4;                     // of a copy
    // copies of 8 entries (kHalf: two words a pair)
    static constexpr int kCopies = MODE == kHalf ? 8 : 8 * (int)sizeof(T) / kBytes;
    static constexpr int kPer = kBytes / (int)sizeof(T);                     // entries of a copy
    static constexpr uint32_t kStage = (uint32_t)MAXK * kCopies * kBytes * THREADS;
    const T *src[MAXK];                                      // this thread's next row to copy
    int64_t hop[MAXK];                                       // entries from one of its rows to the next
    int64_t first, step, T_rows, next;                       // next: the row src points at
    int t, D, copies;                                        // copies: that lie inside the row
    uint32_t ring, fill;                                     // shared addresses: base, next stage
    const char *mine;                                        // the base as a pointer
    int drain;                                               // the stage at hand, from there
    uint32_t inside, flips;                                  // kHalf: bit k, the row at hand starts
                                                             // inside a word, and its rows alternate

    static constexpr size_t smem_bytes() { return (size_t)S * kStage; }
    // entries between a thread's copies
    __device__ static constexpr int apart() { return MODE == kRun ? kPer : kPer * kTpr; }
    __device__ __forceinline__ int start() const {           // of this thread's entries
        return MODE == kRun ? 8 * t : MODE == kWord ? kPer * t : 0;
    }
    __device__ __forceinline__ void tensor(int k, const void *base, int64_t ld) {
        src[k] = base ? static_cast<const T *>(base) + first * ld + (copies ? start() : 0) : nullptr;
        hop[k] = step * ld;
        if constexpr (MODE == kHalf) {
            inside |= (uint32_t)(((uintptr_t)src[k] >> 1) & 1) << k;
            flips |= (uint32_t)(hop[k] & 1) << k;
        }
    }
    // before tensor(): rows first, first + step, ..
    __device__ __forceinline__ void rows(int64_t first_, int64_t step_, int64_t T_rows_, int t_,
                                         int D_, void *smem) {
        first = next = first_;
        step = step_;
        T_rows = T_rows_;
        t = t_;
        D = D_;
        copies = 0;
        inside = flips = 0;
        if constexpr (MODE != kHalf)
#pragma unroll
            for (int i = 0; i < kCopies; ++i) copies += start() + i * apart() < D ? 1 : 0;
        mine = static_cast<char *>(smem) + kBytes * threadIdx.x;
        drain = 0;
        ring = fill = (uint32_t)__cvta_generic_to_shared(mine);
    }
    // starts the copies of this thread's next row
    __device__ __forceinline__ void issue() {
        if (next < T_rows) {
#pragma unroll
            for (int k = 0; k < MAXK; ++k) {
                if (!src[k]) continue;
                const uint32_t dst = fill + k * kCopies * THREADS * kBytes;
                if constexpr (MODE == kHalf) {
                    copy_pairs(dst, src[k]);
                } else {
#pragma unroll
                    for (int i = 0; i < kCopies; ++i)
                        if (i < copies) copy(dst + i * THREADS * kBytes, src[k] + i * apart());
                }
                src[k] += hop[k];
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        next += step;
        fill += kStage;
        if (fill == ring + S * kStage) fill = ring;
    }
    __device__ __forceinline__ static void copy(uint32_t dst, const void *from) {
        if constexpr (kBytes == 16)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(from)
                         : "memory");
        else
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(from)
                         : "memory");
    }
    // The words of pair t + kTpr i.  A row that starts inside a word shares its
    // first word with what precedes it, and the last word may reach past the
    // row's end: neither outer half is read unless it is the row's own or
    // (before a later row's start) the previous row's.
    __device__ __forceinline__ void copy_pairs(uint32_t dst, const T *row) const {
        const bool in = ((uintptr_t)row >> 1) & 1;
        const char *word = reinterpret_cast<const char *>((uintptr_t)row & ~(uintptr_t)3);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int q = t + kTpr * i;
            if (2 * q >= D) break;
            const uint32_t lo = dst + 2 * i * THREADS * 4, hi = lo + THREADS * 4;
            if (in && q == 0) {              // the entry alone, in the word's upper half
                const uint32_t x = (uint32_t)*reinterpret_cast<const uint16_t *>(row) << 16;
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(lo), "r"(x) : "memory");
            } else if (!in && 2 * q + 1 >= D) {   // the entry alone, in the lower half
                const uint32_t x = *reinterpret_cast<const uint16_t *>(row + 2 * q);
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(lo), "r"(x) : "memory");
            } else {
                copy(lo, word + 4 * (int64_t)q);
            }
            if (in && 2 * q + 1 < D) {
                if (2 * q + 2 >= D) {        // the pair's second entry ends the row
                    const uint32_t x = *reinterpret_cast<const uint16_t *>(row + 2 * q + 1);
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(hi), "r"(x) : "memory");
                } else {
                    copy(hi, word + 4 * (int64_t)q + 4);
                }
            }
        }
    }
    __device__ __forceinline__ void wait() {
        asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
    }
    // the row's entries of tensor k (zeros past D and without a tensor)
    __device__ __forceinline__ void take(F2 (&x)[kP], int k) {
        const char *from = mine + drain + k * kCopies * THREADS * kBytes;
        if constexpr (MODE == kRun) {
            uint4 q[kCopies];
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                q[i] = make_uint4(0u, 0u, 0u, 0u);
                if (src[k] && i < copies)
                    q[i] = *reinterpret_cast<const uint4 *>(from + i * THREADS * kBytes);
            }
            widen(x, q, T());
        } else {
            uint32_t q[kCopies];
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                // kHalf: words 2 i and 2 i + 1 of pair i, the second for entries of
                // a row that starts inside a word
                const bool have = MODE == kHalf
                    ? 2 * (t + kTpr * (i >> 1)) + (i & 1) < D && (!(i & 1) || (inside >> k & 1))
                    : i < copies;
                q[i] = 0u;
                if (src[k] && have)
                    q[i] = *reinterpret_cast<const uint32_t *>(from + i * THREADS * kBytes);
            }
#pragma unroll
            for (int e = 0; e < kP; ++e) {
                if constexpr (sizeof(T) == 4) {
                    x[e] = f2(__uint_as_float(q[2 * e]), __uint_as_float(q[2 * e + 1]));
                } else {
                    uint32_t v = q[MODE == kHalf ? 2 * e : e];
                    if (MODE == kHalf && (inside >> k & 1)) v = __funnelshift_r(v, q[2 * e + 1], 16);
                    x[e] = f2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
                }
            }
        }
    }
    // the row is taken: its place gets a further row
    __device__ __forceinline__ void taken() {
        drain += kStage;
        if (drain == (int)(S * kStage)) drain = 0;
        if constexpr (MODE == kHalf) inside ^= flips;
        issue();
    }
    // a contiguous output's row, dst its start
    __device__ __forceinline__ void put(T *dst, const F2 (&x)[kP]) const {
        if constexpr (MODE == kRun && sizeof(T) == 2) {
            if (copies)
                *reinterpret_cast<uint4 *>(dst + 8 * t) =
                    make_uint4(pack(x[0]), pack(x[1]), pack(x[2]), pack(x[3]));
        } else if constexpr (MODE == kRun) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i < copies) {
                    const float2 lo = split(x[2 * i]), hi = split(x[2 * i + 1]);
                    *reinterpret_cast<float4 *>(dst + 8 * t + 4 * i) =
                        make_float4(lo.x, lo.y, hi.x, hi.y);
                }
        } else if constexpr (MODE == kWord && sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < kP; ++i)
                if (i < copies)
                    *reinterpret_cast<uint32_t *>(dst + 2 * (t + kTpr * i)) = pack(x[i]);
        } else {
#pragma unroll
            for (int e = 0; e < kP; ++e) {
                const float2 v = split(x[e]);
                const int c0 = col_of<T, MODE, kTpr>(t, 2 * e), c1 = col_of<T, MODE, kTpr>(t, 2 * e + 1);
                if (c0 < D) dst[c0] = from_f<T>(v.x);
                if (c1 < D) dst[c1] = from_f<T>(v.y);
            }
        }
    }
};

// a parameter vector, or `fill` everywhere without one; zeros past D
template <typename T, int MODE, int TPR>
__device__ __forceinline__ void param(F2 (&x)[kP], const float *p, float fill, int t, int D) {
    if constexpr (MODE == kRun) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (8 * t + 4 * i < D)
                v = p ? *reinterpret_cast<const float4 *>(p + 8 * t + 4 * i)
                      : make_float4(fill, fill, fill, fill);
            x[2 * i] = f2(v.x, v.y);
            x[2 * i + 1] = f2(v.z, v.w);
        }
    } else {
        float v[2 * kP];
#pragma unroll
        for (int e = 0; e < 2 * kP; ++e) {
            const int c = col_of<T, MODE, TPR>(t, e);
            v[e] = c < D ? (p ? p[c] : fill) : 0.f;
        }
#pragma unroll
        for (int e = 0; e < kP; ++e) x[e] = f2(v[2 * e], v[2 * e + 1]);
    }
}

// clears the entries past D
template <typename T, int MODE, int TPR>
__device__ __forceinline__ void clip(F2 (&x)[kP], int t, int D) {
    if (col_of<T, MODE, TPR>(t, 7) < D) return;   // the thread's last entry is its largest column
#pragma unroll
    for (int e = 0; e < kP; ++e) {
        const float2 v = split(x[e]);
        x[e] = f2(col_of<T, MODE, TPR>(t, 2 * e) < D ? v.x : 0.f,
                  col_of<T, MODE, TPR>(t, 2 * e + 1) < D ? v.y : 0.f);
    }
}

// Sums of K (1 or 3) values over the threads of a row, returned to all of them.
// The warps of a row leave their sums in shared memory (both blocks' of a
// cluster), in one of two buffers in turn, so that one barrier serves a sum.
// Within a warp the lanes first share the values out (half of the lanes keep
// half of the values), so that three values take 6 shuffles, not 15.
template <int NT, int CL> struct RowSum {
    float (*buf)[kSumSlots];
    int turn;
    template <int K> __device__ __forceinline__ void operator()(float (&v)[K]) {
        const int lane = threadIdx.x & 31;
        if constexpr (NT * CL == 32) {
#pragma unroll
            for (int off = 16; off > 0; off >>= 1)
#pragma unroll
                for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(kFull, v[k], off);
            return;
        }
        constexpr int kWarps = NT * CL / 32;
        float r;
        int mine = 0;                        // the value that this lane ends up with
        if constexpr (K == 1) {
            r = v[0] + __shfl_xor_sync(kFull, v[0], 16);
            r += __shfl_xor_sync(kFull, r, 8);
        } else {
            static_assert(K == 3, "one or three values");
            const bool high = lane & 16, odd = lane & 8;
            float a = high ? v[2] : v[0], b = high ? 0.f : v[1];
            a += __shfl_xor_sync(kFull, high ? v[0] : v[2], 16);
            b += __shfl_xor_sync(kFull, high ? v[1] : 0.f, 16);
            r = odd ? b : a;
            r += __shfl_xor_sync(kFull, odd ? a : b, 8);
            mine = (high ? 2 : 0) + (odd ? 1 : 0);
        }
#pragma unroll
        for (int off = 4; off > 0; off >>= 1) r += __shfl_xor_sync(kFull, r, off);
        float *b = buf[turn];
        turn ^= 1;
        const int w = threadIdx.x >> 5;
        if constexpr (CL == 1) {
            if ((lane & 7) == 0 && mine < K) b[mine * kWarps + w] = r;
            __syncthreads();
        } else {
            if ((lane & 7) < CL && mine < K) {   // lanes 0 and 1 of 8: one block each
                const uint32_t dst = tc::mapa_shared(
                    tc::smem_u32(b + mine * kWarps + tc::cluster_ctarank() * (NT / 32) + w),
                    lane & 7);
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst), "f"(r) : "memory");
            }
            tc::cluster_sync();
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if constexpr (kWarps % 4 == 0) {
                F2 s = f2(0.f);
#pragma unroll 2   // more loads at once cost registers that wide rows do not have
                for (int i = 0; i < kWarps; i += 4) {
                    const float4 x = *reinterpret_cast<const float4 *>(b + k * kWarps + i);
                    s = s + (f2(x.x, x.y) + f2(x.z, x.w));
                }
                v[k] = both(s);
            } else {
                v[k] = 0.f;
#pragma unroll
                for (int i = 0; i < kWarps; ++i) v[k] += b[k * kWarps + i];
            }
        }
    }
};

// x <- the normalised row (entries past D stay 0); the mean (layer) is
// subtracted before the squares are summed, so nothing cancels
template <typename T, int MODE, int NT, int CL, bool LAYER, typename Sum>
__device__ __forceinline__ void normalise(F2 (&x)[kP], int D, float inv, float eps, int t,
                                          Sum &sum) {
    float s[1];
    if constexpr (LAYER) {
        s[0] = both((x[0] + x[1]) + (x[2] + x[3]));
        sum(s);
        const F2 mean = f2(-s[0] * inv);
#pragma unroll
        for (int e = 0; e < kP; ++e) x[e] = x[e] + mean;
        clip<T, MODE, NT * CL>(x, t, D);
    }
    F2 q = x[0] * x[0];
#pragma unroll
    for (int e = 1; e < kP; ++e) q = fma2(x[e], x[e], q);
    s[0] = both(q);
    sum(s);
    const F2 rstd = f2(rsqrtf(fmaf(s[0], inv, eps)));
#pragma unroll
    for (int e = 0; e < kP; ++e) x[e] = x[e] * rstd;
}

// What the first norm's gain and bias, the per-channel gate and the output's
// scale make of a normalised row, as one factor and one offset a channel:
// out_scale gate (.) (w x + b) = W x + B.  (x itself without the first norm.)
template <typename T, int MODE, int TPR, bool LAYER>
__device__ __forceinline__ void fold_post(F2 (&W)[kP], F2 (&B)[kP], const NormArgs &a, int t) {
    F2 g[kP];
    const bool channel = a.gate_mode == ULTRAMEM_GATE_CHANNEL;
    param<T, MODE, TPR>(g, channel ? static_cast<const float *>(a.gate) : nullptr, 1.f, t, a.D);
    param<T, MODE, TPR>(W, a.post ? a.w_post : nullptr, 1.f, t, a.D);
    if constexpr (LAYER) param<T, MODE, TPR>(B, a.post ? a.b_post : nullptr, 0.f, t, a.D);
    const F2 s = f2(a.out_scale);
#pragma unroll
    for (int e = 0; e < kP; ++e) {
        g[e] = g[e] * s;
        W[e] = W[e] * g[e];
        if constexpr (LAYER) B[e] = B[e] * g[e];
    }
}

// Blocks of the forward that an SM is to have registers for, 640 to 1024
// threads.  (Layer norms take 86 to 98 registers without the bound: 72 us
// against 62 at 16384 x 2048.)
template <int NT> constexpr int kBlocks = NT > 512 ? 1 : NT >= 384 ? 2 : NT == 32 ? 5 : 768 / NT;

// A row per NT threads, grid-stride; rows of one warp go four to a block.
template <typename T, int MODE, int NT, bool LAYER>
__global__ void __launch_bounds__(NT == 32 ? 128 : NT, kBlocks<NT>)
    block_norm_kernel(NormArgs a) {
    constexpr int TPR = NT;
    extern __shared__ uint4 ring[];
    __shared__ __align__(16) float buf[2][kSumSlots];
    RowSum<NT, 1> sum{buf, 0};
    const int t = NT == 32 ? (threadIdx.x & 31) : threadIdx.x;
    const int rows = NT == 32 ? blockDim.x >> 5 : 1;
    const bool full = a.gate_mode == ULTRAMEM_GATE_FULL;
    const float inv = 1.f / (float)a.D;
    Feed<T, MODE, NT, 1, NT == 32 ? 128 : NT, kAhead, 3> in;
    in.rows((int64_t)blockIdx.x * rows + (NT == 32 ? threadIdx.x >> 5 : 0),
            (int64_t)gridDim.x * rows, a.T, t, a.D, ring);
    in.tensor(0, a.y, a.ld_y);
    in.tensor(1, a.r, a.ld_r);
    in.tensor(2, full ? a.gate : nullptr, a.D);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) in.issue();
    F2 W[kP], B[kP], wn[kP], bn[kP];
    fold_post<T, MODE, TPR, LAYER>(W, B, a, t);
    param<T, MODE, TPR>(wn, a.w_pre, 1.f, t, a.D);
    if constexpr (LAYER) param<T, MODE, TPR>(bn, a.b_pre, 0.f, t, a.D);
    const F2 res = f2(a.res_scale);
    T *u_row = static_cast<T *>(a.u) + in.first * a.D, *n_row = nullptr;
    if (a.pre) n_row = static_cast<T *>(a.n) + in.first * a.D;
    const int64_t hop = in.step * a.D;
    for (int64_t row = in.first; row < a.T; row += in.step, u_row += hop, n_row += hop) {
        F2 z[kP], u[kP], g[kP];
        in.wait();
        in.take(z, 0);
        in.take(u, 1);
        if (full) in.take(g, 2);
        in.taken();
        if (a.post) normalise<T, MODE, NT, 1, LAYER>(z, a.D, inv, a.eps, t, sum);
#pragma unroll
        for (int e = 0; e < kP; ++e) z[e] = LAYER ? fma2(z[e], W[e], B[e]) : z[e] * W[e];
        if (full) {
#pragma unroll
            for (int e = 0; e < kP; ++e) z[e] = z[e] * g[e];
        } else if (a.gate_mode == ULTRAMEM_GATE_TOKEN) {
            const F2 gt = f2(to_f(static_cast<const T *>(a.gate)[row]));
#pragma unroll
            for (int e = 0; e < kP; ++e) z[e] = z[e] * gt;
        }
#pragma unroll
        for (int e = 0; e < kP; ++e) u[e] = fma2(res, u[e], z[e]);
        in.put(u_row, u);
        if (a.pre) {
            // The second norm reads the stream as stored, so that the
            // gradient taken from the stored stream is that of this function.
#pragma unroll
            for (int e = 0; e < kP; ++e) u[e] = as_stored(u[e], T());
            normalise<T, MODE, NT, 1, LAYER>(u, a.D, inv, a.eps, t, sum);
#pragma unroll
            for (int e = 0; e < kP; ++e) u[e] = LAYER ? fma2(u[e], wn[e], bn[e]) : u[e] * wn[e];
            in.put(n_row, u);
        }
    }
}

// ---- the gradient ------------------------------------------------------
// With û, ŷ the normalised rows and g = w (.) d for the gradient d of a
// norm's output, the gradient of its input is
//   rstd (g - mean(g) - û mean(g û))      (rms: without mean(g)).
// One pass over y, u, du and dn gives everything: the rows' statistics are
// taken again from the rows themselves.  With gv the gradient gu of the
// stream times a token's or entry's gate, two column sums serve the first
// norm and a per-channel gate together,
//   P = sum gv ŷ,  Q = sum gv:   dw_post = out_scale gate P,
//   db_post = out_scale gate Q,  dgate = out_scale (w_post P + b_post Q),
// and sum dn û, sum dn are those of the second norm.  They stay in registers
// over a block's rows and leave as one partial row per block, which a second
// kernel adds in the blocks' order (no atomics: the result does not depend on
// the schedule).
enum { kColP, kColPre, kColQ, kColBPre };   // order of the partial rows (the last two: layer)

template <typename T, int MODE, int NT, int CL, bool LAYER>
__global__ void __launch_bounds__(NT, NT < 512 ? 512 / NT : 1)
    block_norm_backward_kernel(NormArgs a) {
    constexpr int TPR = NT * CL;
    extern __shared__ uint4 ring[];
    __shared__ __align__(16) float buf[2][kSumSlots];
    // the peer's shared memory may be written only once the peer runs: arrive
    // here and wait below, behind the first copies and the parameters' loads
    if constexpr (CL > 1) tc::cluster_arrive_relaxed();
    RowSum<NT, CL> sum{buf, 0};
    const int t = threadIdx.x + (CL > 1 ? NT * (int)tc::cluster_ctarank() : 0);
    const bool full = a.gate_mode == ULTRAMEM_GATE_FULL;
    const bool token = a.gate_mode == ULTRAMEM_GATE_TOKEN;
    const float inv = 1.f / (float)a.D;
    Feed<T, MODE, NT, CL, NT, kAheadBack<T, MODE>, 5> in;
    in.rows(blockIdx.x / CL, gridDim.x / CL, a.T, t, a.D, ring);
    in.tensor(0, a.y, a.ld_y);
    in.tensor(1, a.pre ? a.r : nullptr, a.ld_r);
    in.tensor(2, a.pre ? a.dn : nullptr, a.ld_dn);
    in.tensor(3, a.du, a.ld_du);
    in.tensor(4, full ? a.gate : nullptr, a.D);
#pragma unroll
    for (int i = 0; i < kAheadBack<T, MODE>; ++i) in.issue();
    F2 W[kP], B[kP], wn[kP];
    F2 c_p[kP], c_pre[kP], c_q[kP], c_bpre[kP];
    fold_post<T, MODE, TPR, LAYER>(W, B, a, t);
    param<T, MODE, TPR>(wn, a.w_pre, 1.f, t, a.D);
#pragma unroll
    for (int e = 0; e < kP; ++e) c_p[e] = c_pre[e] = c_q[e] = c_bpre[e] = f2(0.f);
    const F2 res = f2(a.res_scale);
    if constexpr (CL > 1) tc::cluster_wait();   // before the first sum stores into the peer

    auto row_of = [&](void *base) { return static_cast<T *>(base) + in.first * a.D; };
    T *dr_row = a.dr ? row_of(a.dr) : nullptr, *dy_row = a.dy ? row_of(a.dy) : nullptr;
    T *dg_row = full && a.dgate_rows ? row_of(a.dgate_rows) : nullptr;
    const int64_t hop = in.step * a.D;
    for (int64_t row = in.first; row < a.T; row += in.step) {
        F2 y[kP], u[kP], gu[kP], dn[kP], g[kP];
        in.wait();
        in.take(y, 0);
        in.take(u, 1);
        in.take(dn, 2);
        in.take(gu, 3);
        if (full) in.take(g, 4);
        in.taken();
        const float gt = token ? to_f(static_cast<const T *>(a.gate)[row]) : 1.f;

        // statistics of y and u, and the sums of the second norm's gradient
        float s[3], mean_g = 0.f;
        if constexpr (LAYER) {
#pragma unroll
            for (int e = 0; e < kP; ++e) c_bpre[e] = c_bpre[e] + dn[e];
        }
        F2 wd[kP];
#pragma unroll
        for (int e = 0; e < kP; ++e) wd[e] = wn[e] * dn[e];
        if constexpr (LAYER) {
            s[0] = both((y[0] + y[1]) + (y[2] + y[3]));
            s[1] = both((u[0] + u[1]) + (u[2] + u[3]));
            s[2] = both((wd[0] + wd[1]) + (wd[2] + wd[3]));
            sum(s);
            const F2 my = f2(a.post ? -s[0] * inv : 0.f), mu = f2(-s[1] * inv);
            mean_g = s[2] * inv;
#pragma unroll
            for (int e = 0; e < kP; ++e) {
                y[e] = y[e] + my;
                u[e] = u[e] + mu;
            }
            clip<T, MODE, TPR>(y, t, a.D);
            clip<T, MODE, TPR>(u, t, a.D);
        }
        {
            F2 q0 = y[0] * y[0], q1 = u[0] * u[0], q2 = wd[0] * u[0];
#pragma unroll
            for (int e = 1; e < kP; ++e) {
                q0 = fma2(y[e], y[e], q0);
                q1 = fma2(u[e], u[e], q1);
                q2 = fma2(wd[e], u[e], q2);
            }
            s[0] = both(q0);
            s[1] = both(q1);
            s[2] = both(q2);
        }
        sum(s);
        const float ry = a.post ? rsqrtf(fmaf(s[0], inv, a.eps)) : 1.f;
        const float ru = a.pre ? rsqrtf(fmaf(s[1], inv, a.eps)) : 0.f;
        const F2 ry2 = f2(ry), ru2 = f2(ru), m_gu = f2(-s[2] * ru * inv), m_g = f2(-mean_g);
        F2 gy[kP];
        F2 q0 = f2(0.f), q1 = f2(0.f), q2 = f2(0.f);
#pragma unroll
        for (int e = 0; e < kP; ++e) {
            const F2 uh = u[e] * ru2;
            c_pre[e] = fma2(dn[e], uh, c_pre[e]);
            F2 d = fma2(uh, m_gu, wd[e]);
            if constexpr (LAYER) d = d + m_g;
            gu[e] = fma2(ru2, d, gu[e]);
            y[e] = y[e] * ry2;                 // from here the normalised row
            u[e] = res * gu[e];
        }
        if constexpr (LAYER) clip<T, MODE, TPR>(gu, t, a.D);
        if (dr_row) {
            in.put(dr_row, u);
            dr_row += hop;
        }
        if (full || token) {
            // through a gate of the row: its gradient out_scale z gu, and gv
#pragma unroll
            for (int e = 0; e < kP; ++e) {
                u[e] = (LAYER ? fma2(W[e], y[e], B[e]) : W[e] * y[e]) * gu[e];
                q2 = q2 + u[e];
                gu[e] = gu[e] * (full ? g[e] : f2(gt));
            }
            if (dg_row) {
                in.put(dg_row, u);
                dg_row += hop;
            }
        }
#pragma unroll
        for (int e = 0; e < kP; ++e) {
            c_p[e] = fma2(gu[e], y[e], c_p[e]);
            if constexpr (LAYER) c_q[e] = c_q[e] + gu[e];
            gy[e] = W[e] * gu[e];
            if constexpr (LAYER) q0 = q0 + gy[e];
            q1 = fma2(gy[e], y[e], q1);
        }
        float s1 = 0.f, s0 = 0.f;
        if (LAYER || token) {
            float v[3] = {both(q1), both(q2), both(q0)};
            sum(v);
            if (token && a.dgate_rows && t == 0)
                static_cast<T *>(a.dgate_rows)[row] = from_f<T>(v[1]);
            s1 = v[0];
            s0 = v[2];
        } else {
            float v[1] = {both(q1)};
            sum(v);
            s1 = v[0];
        }
        const F2 m1 = f2(a.post ? -s1 * inv : 0.f);
        const F2 m0 = f2(LAYER && a.post ? -s0 * inv : 0.f);
#pragma unroll
        for (int e = 0; e < kP; ++e) {
            F2 d = fma2(y[e], m1, gy[e]);
            if constexpr (LAYER) d = d + m0;
            gy[e] = ry2 * d;
        }
        if (dy_row) {
            in.put(dy_row, gy);
            dy_row += hop;
        }
    }

    pdl_trigger();
    float *part = a.part + (int64_t)(blockIdx.x / CL) * (LAYER ? 4 : 2) * a.D;
    auto leave = [&](int k, const F2 (&c)[kP]) {
        float *dst = part + (int64_t)k * a.D;
        if constexpr (MODE == kRun) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (8 * t + 4 * i < a.D) {
                    const float2 lo = split(c[2 * i]), hi = split(c[2 * i + 1]);
                    *reinterpret_cast<float4 *>(dst + 8 * t + 4 * i) =
                        make_float4(lo.x, lo.y, hi.x, hi.y);
                }
        } else {
#pragma unroll
            for (int e = 0; e < kP; ++e) {
                const float2 v = split(c[e]);
                const int x = col_of<T, MODE, TPR>(t, 2 * e), y = col_of<T, MODE, TPR>(t, 2 * e + 1);
                if (x < a.D) dst[x] = v.x;
                if (y < a.D) dst[y] = v.y;
            }
        }
    };
    leave(kColP, c_p);
    leave(kColPre, c_pre);
    if constexpr (LAYER) {
        leave(kColQ, c_q);
        leave(kColBPre, c_bpre);
    }
}

struct ColOut {
    float *dw_post, *db_post, *dgate, *dw_pre, *db_pre;   // null: not wanted
    const float *w_post, *b_post, *gate;                  // null: ones, zeros, ones
    float out_scale;
};

// The column sums over the blocks' partial rows, 32 columns a block, 32 warps
// over the rows; blockIdx.y 0: the first norm's and the gate's, 1: the second's.
__global__ void __launch_bounds__(1024) column_sum_kernel(const float *part, int blocks,
                                                          int layer, int D, ColOut o) {
    __shared__ float s[2][32][33];
    const int n_cols = layer ? 4 : 2, which = blockIdx.y;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    pdl_wait();
    float v = 0.f, q = 0.f;
    if (c < D) {
#pragma unroll 4
        for (int b = w; b < blocks; b += 32) {
            const float *row = part + ((int64_t)b * n_cols + which) * D + c;
            v += row[0];
            if (layer) q += row[2 * (int64_t)D];
        }
    }
    s[0][w][lane] = v;
    s[1][w][lane] = q;
    __syncthreads();
    if (w != 0 || c >= D) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) {
        v += s[0][i][lane];
        q += s[1][i][lane];
    }
    if (which == 1) {
        if (o.dw_pre) o.dw_pre[c] = v;
        if (o.db_pre) o.db_pre[c] = q;
        return;
    }
    // all read before the first write: a gradient may take its vector's place
    const float g = o.out_scale * (o.gate ? o.gate[c] : 1.f);
    const float wp = o.w_post ? o.w_post[c] : 1.f, bp = o.b_post ? o.b_post[c] : 0.f;
    if (o.dw_post) o.dw_post[c] = g * v;
    if (o.db_post) o.db_post[c] = g * q;
    if (o.dgate) o.dgate[c] = o.out_scale * fmaf(wp, v, bp * q);
}

// ---- launches ----------------------------------------------------------

constexpr int kMaxDim = 8192;

// Threads of a row: 8 entries each, in steps of a third to a half, so that few
// idle, each a kernel of its own: with the number known at run time only, the
// gradient at 16384 x 2048 took 97 us instead of 78.
int row_threads(int D) {
    const int v = (D + 7) / 8;
    for (const int t : {32, 64, 128, 192, 256, 384, 512, 768})
        if (v <= t) return t;
    return 1024;
}

// Dynamic shared memory and grid of a persistent kernel: as many blocks as
// the SMs hold, asked of the driver once per kernel and device.
template <auto K> cudaError_t resident_blocks(int threads, size_t smem, int *n) {
    static PerDevice<int> blocks;
    return blocks.get(n, [&](int, int *b) {
        cudaError_t e =
            cudaFuncSetAttribute(K, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e == cudaSuccess)
            e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(b, K, threads, smem);
        return e == cudaSuccess && *b < 1 ? cudaErrorInvalidConfiguration : e;
    });
}

template <auto K> cudaError_t run_rows(const NormArgs &a, int64_t units, int threads, int cl,
                                       size_t smem, int64_t most, int *groups, cudaStream_t st) {
    int fit = 0;
    const cudaError_t e = resident_blocks<K>(threads, smem, &fit);
    if (e != cudaSuccess) return e;
    int64_t grid = (int64_t)device_sm_count() * fit / cl;   // clusters (or blocks)
    grid = grid < most ? grid : most;
    grid = grid < units ? grid : units;
    grid = grid < 1 ? 1 : grid;
    *groups = (int)grid;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(grid * cl));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = cl;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = cl > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, K, a);
}

template <typename T, int MODE, bool LAYER> struct Forward {
    template <int NT> static cudaError_t go(const NormArgs &a, int *groups, cudaStream_t st) {
        constexpr int threads = NT == 32 ? 128 : NT;
        constexpr size_t smem = Feed<T, MODE, NT, 1, threads, kAhead, 3>::smem_bytes();
        const int64_t units = NT == 32 ? (a.T + 3) / 4 : a.T;
        return run_rows<block_norm_kernel<T, MODE, NT, LAYER>>(a, units, threads, 1, smem,
                                                              INT64_MAX, groups, st);
    }
    // Past 4096 entries one wide block: a cluster of two of 512 threads pays its
    // barrier up to four times a row (4096 x 8192 in bf16: 94 us against 57).
    static cudaError_t launch(const NormArgs &a, int *groups, cudaStream_t st) {
        switch (row_threads(a.D)) {
        case 32: return go<32>(a, groups, st);
        case 64: return go<64>(a, groups, st);
        case 128: return go<128>(a, groups, st);
        case 192: return go<192>(a, groups, st);
        case 256: return go<256>(a, groups, st);
        case 384: return go<384>(a, groups, st);
        case 512: return go<512>(a, groups, st);
        case 768: return go<768>(a, groups, st);
        default: return go<1024>(a, groups, st);
        }
    }
};

// Partial rows of the gradient's column sums, one per block (or cluster): as
// many as the SMs hold at 128 registers a thread (64 at rows of one warp, so
// that the second kernel's sums stay short), and no more than rows.  A partial
// row is written and read again, so a block gets at least 4 rows once every SM
// has a block.  With 1, 2, 4 or 8 instead: 1000 x 1000 fp32 15.3, 15.1, 15.1,
// 16.3 us; 300 x 2048 bf16 7.7, 7.0, 6.9, 7.0; 500 x 512 6.9, 6.4, 7.2, 7.2;
// 4000 x 512 12.5, 12.5, 12.3, 12.6.
int64_t partial_rows(int64_t T, int D) {
    const int threads = row_threads(D);
    int per_sm2 = threads > 512 ? 1 : 2 * (512 / threads);   // per two SMs
    if (per_sm2 > 16) per_sm2 = 16;
    const int64_t sms = device_sm_count(), most = sms * per_sm2 / 2;
    int64_t n = (T + 3) / 4;
    if (n < sms) n = T < sms ? T : sms;
    return n < most ? n : most;
}

template <typename T, int MODE, bool LAYER> struct Backward {
    template <int NT, int CL> static cudaError_t go(const NormArgs &a, int *groups, cudaStream_t st) {
        constexpr size_t smem = Feed<T, MODE, NT, CL, NT, kAheadBack<T, MODE>, 5>::smem_bytes();
        return run_rows<block_norm_backward_kernel<T, MODE, NT, CL, LAYER>>(
            a, a.T, NT, CL, smem, partial_rows(a.T, a.D), groups, st);
    }
    static cudaError_t launch(const NormArgs &a, int *groups, cudaStream_t st) {
        switch (row_threads(a.D)) {
        case 32: return go<32, 1>(a, groups, st);
        case 64: return go<64, 1>(a, groups, st);
        case 128: return go<128, 1>(a, groups, st);
        case 192: return go<192, 1>(a, groups, st);
        case 256: return go<256, 1>(a, groups, st);
        case 384: return go<384, 1>(a, groups, st);
        case 512: return go<512, 1>(a, groups, st);
        case 768: return go<384, 2>(a, groups, st);
        default: return go<512, 2>(a, groups, st);
        }
    }
};

// groups: the blocks (or clusters) launched
template <template <typename, int, bool> class Op>
cudaError_t dispatch(const NormArgs &a, int dtype, bool layer, int mode, int *groups,
                     cudaStream_t st) {
    using B = __nv_bfloat16;
    if (dtype == ULTRAMEM_BF16 && mode == kRun)
        return layer ? Op<B, kRun, true>::launch(a, groups, st)
                     : Op<B, kRun, false>::launch(a, groups, st);
    if (dtype == ULTRAMEM_BF16 && mode == kWord)
        return layer ? Op<B, kWord, true>::launch(a, groups, st)
                     : Op<B, kWord, false>::launch(a, groups, st);
    if (dtype == ULTRAMEM_BF16)
        return layer ? Op<B, kHalf, true>::launch(a, groups, st)
                     : Op<B, kHalf, false>::launch(a, groups, st);
    if (mode == kRun)
        return layer ? Op<float, kRun, true>::launch(a, groups, st)
                     : Op<float, kRun, false>::launch(a, groups, st);
    return layer ? Op<float, kWord, true>::launch(a, groups, st)
                 : Op<float, kWord, false>::launch(a, groups, st);
}

bool valid(const ultramem_block_norm_args *p) {
    if (!p || p->n_tokens < 0 || p->dim < 1 || p->dim > kMaxDim) return false;
    if (p->dtype != ULTRAMEM_F32 && p->dtype != ULTRAMEM_BF16) return false;
    if (p->kind != ULTRAMEM_NORM_RMS && p->kind != ULTRAMEM_NORM_LAYER) return false;
    if ((p->post != 0 && p->post != 1) || (p->pre != 0 && p->pre != 1)) return false;
    if (p->gate_mode < ULTRAMEM_GATE_NONE || p->gate_mode > ULTRAMEM_GATE_FULL) return false;
    if ((p->gate_mode == ULTRAMEM_GATE_NONE) != (p->gate == nullptr)) return false;
    if (!(p->eps >= 0.f) || !(p->eps < INFINITY) || !isfinite(p->res_scale) ||
        !isfinite(p->out_scale))
        return false;
    if (p->kind == ULTRAMEM_NORM_RMS && (p->b_post || p->b_pre)) return false;
    return true;
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

NormArgs args_of(const ultramem_block_norm_args *p) {
    NormArgs a = {};
    a.y = p->y;
    a.gate = p->gate;
    a.w_post = p->w_post;
    a.b_post = p->b_post;
    a.w_pre = p->w_pre;
    a.b_pre = p->b_pre;
    a.T = p->n_tokens;
    a.D = p->dim;
    a.ld_y = p->ld_y;
    a.ld_r = p->ld_r;
    a.post = p->post;
    a.pre = p->pre;
    a.gate_mode = p->gate_mode;
    a.res_scale = p->res_scale;
    a.out_scale = p->out_scale;
    a.eps = p->eps;
    return a;
}

// The widest access that all rows allow: `rows` and `lds` are the row tensors
// and their row distances, `vectors` fp32 vectors that kRun reads by 16 bytes.
int mode_of(int dtype, int D, std::initializer_list<const void *> rows,
            std::initializer_list<int64_t> lds, std::initializer_list<const void *> vectors) {
    const int es = dtype == ULTRAMEM_BF16 ? 2 : 4;
    uintptr_t low = (uintptr_t)D * es;
    for (const void *p : rows) low |= (uintptr_t)p;
    for (int64_t ld : lds) low |= (uintptr_t)(ld * es);
    uintptr_t wide = low;
    for (const void *p : vectors) wide |= (uintptr_t)p;
    return wide % 16 == 0 ? kRun : low % 4 == 0 ? kWord : kHalf;
}

// Whether all pointers lie on boundaries of `size` bytes.
bool on_boundary(int size, std::initializer_list<const void *> pointers) {
    uintptr_t low = 0;
    for (const void *p : pointers) low |= (uintptr_t)p;
    return low % size == 0;
}
// The same of a call's parameters and its gate (and the gate's gradient).
bool params_on_boundary(const ultramem_block_norm_args *p, const void *dgate) {
    const bool channel = p->gate_mode == ULTRAMEM_GATE_CHANNEL;
    return on_boundary(4, {p->w_post, p->b_post, p->w_pre, p->b_pre}) &&
           on_boundary(channel || p->dtype == ULTRAMEM_F32 ? 4 : 2, {p->gate, dgate});
}

// A row tensor, and the call's vectors and gate.
Memory rows_of(const ultramem_block_norm_args *p, const void *at, int64_t ld) {
    const int64_t es = p->dtype == ULTRAMEM_BF16 ? 2 : 4;
    return {at, p->dim * es, p->n_tokens, ld * es};
}
Memory vector_of(const ultramem_block_norm_args *p, const void *at) {
    return {at, p->dim * (int64_t)sizeof(float)};
}
// the gate, or its gradient
Memory gate_of(const ultramem_block_norm_args *p, const void *at) {
    if (p->gate_mode == ULTRAMEM_GATE_FULL) return rows_of(p, at, p->dim);
    if (p->gate_mode == ULTRAMEM_GATE_CHANNEL) return vector_of(p, at);
    return {at, (int64_t)p->n_tokens * (p->dtype == ULTRAMEM_BF16 ? 2 : 4)};
}

// A row of an output is written after that row of every input was read and
// while other rows are not: an output may be a row tensor itself.  Anything
// else that outputs share, with one another or with an input, goes wrong.
bool forward_apart(const ultramem_block_norm_args *p, const void *r, const void *u,
                   const void *n) {
    const Memory out[2] = {rows_of(p, u, p->dim), rows_of(p, n, p->dim)};
    if (overlap(out[0], out[1])) return false;
    for (const Memory &o : out) {
        if (!same_or_apart(o, rows_of(p, p->y, p->ld_y)) ||
            !same_or_apart(o, rows_of(p, r, p->ld_r)))
            return false;
        const Memory gate = gate_of(p, p->gate);
        if (p->gate_mode == ULTRAMEM_GATE_FULL ? !same_or_apart(o, gate) : overlap(o, gate))
            return false;
        for (const void *v : {p->w_post, p->b_post, p->w_pre, p->b_pre})
            if (overlap(o, vector_of(p, v))) return false;
    }
    return true;
}

// The same of the gradient.  A sum over the tokens and a gate's gradient may
// also take the place of the vector or gate that it is the gradient of; the
// partial sums' workspace shares nothing.
bool backward_apart(const ultramem_block_norm_args *p, const void *u, const void *du,
                    int64_t ld_du, const void *dn, int64_t ld_dn, const void *dy, const void *dr,
                    const void *dgate, const float *dw_post, const float *db_post,
                    const float *dw_pre, const float *db_pre, const void *workspace,
                    int64_t workspace_bytes) {
    enum { kDy, kDr, kDgate, kDwPost, kDbPost, kDwPre, kDbPre, kWorkspace, kOut };
    const Memory out[kOut] = {rows_of(p, dy, p->dim), rows_of(p, dr, p->dim), gate_of(p, dgate),
                              vector_of(p, dw_post),  vector_of(p, db_post),
                              vector_of(p, dw_pre),   vector_of(p, db_pre),
                              {workspace, workspace_bytes}};
    for (int i = 0; i < kOut; ++i)
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return false;
    const bool full = p->gate_mode == ULTRAMEM_GATE_FULL;
    const Memory rows[4] = {rows_of(p, p->y, p->ld_y), rows_of(p, p->pre ? u : nullptr, p->ld_r),
                            rows_of(p, du, ld_du), rows_of(p, dn, ld_dn)};
    // what an output may be itself: -1 the row tensors, else the one of that gradient
    const struct {
        Memory in;
        int own;
    } others[5] = {{gate_of(p, p->gate), full ? -1 : kDgate},  {vector_of(p, p->w_post), kDwPost},
                   {vector_of(p, p->b_post), kDbPost},         {vector_of(p, p->w_pre), kDwPre},
                   {vector_of(p, p->b_pre), kDbPre}};
    for (int i = 0; i < kOut; ++i) {
        const bool is_rows = i == kDy || i == kDr || (full && i == kDgate);
        for (const Memory &in : rows)
            if (is_rows ? !same_or_apart(out[i], in) : overlap(out[i], in)) return false;
        for (const auto &o : others) {
            const bool itself = o.own == i || (o.own == -1 && is_rows);
            if (itself ? !same_or_apart(out[i], o.in) : overlap(out[i], o.in)) return false;
        }
    }
    return true;
}

}  // namespace
}  // namespace um

extern "C" ultramem_status ultramem_block_norm(const ultramem_block_norm_args *p, const void *r,
                                               void *u, void *n, void *stream) {
    if (!um::valid(p)) return ULTRAMEM_EINVAL;
    if (p->n_tokens == 0) return ULTRAMEM_OK;
    if (!p->y || !r || !u || (p->pre != 0) != (n != nullptr) || p->ld_y < p->dim ||
        p->ld_r < p->dim)
        return ULTRAMEM_EINVAL;
    const int es = p->dtype == ULTRAMEM_BF16 ? 2 : 4;
    if (!um::on_boundary(es, {p->y, r, u, n}) || !um::params_on_boundary(p, nullptr) ||
        !um::forward_apart(p, r, u, n))
        return ULTRAMEM_EINVAL;
    um::NormArgs a = um::args_of(p);
    a.r = r;
    a.u = u;
    a.n = n;
    const void *full = p->gate_mode == ULTRAMEM_GATE_FULL ? p->gate : nullptr;
    const void *channel = p->gate_mode == ULTRAMEM_GATE_CHANNEL ? p->gate : nullptr;
    const int mode = um::mode_of(p->dtype, p->dim, {p->y, r, u, n, full}, {p->ld_y, p->ld_r},
                                 {p->w_post, p->b_post, p->w_pre, p->b_pre, channel});
    cudaGetLastError();
    int groups = 0;
    return um::status_from_cuda(um::dispatch<um::Forward>(
        a, p->dtype, p->kind == ULTRAMEM_NORM_LAYER, mode, &groups, (cudaStream_t)stream));
}

extern "C" int64_t ultramem_block_norm_backward_workspace(int64_t n_tokens, int32_t dim) {
    if (n_tokens < 0 || dim < 1 || dim > um::kMaxDim) return 0;
    return um::partial_rows(n_tokens, dim) * 4 * dim * (int64_t)sizeof(float);
}

extern "C" ultramem_status ultramem_block_norm_backward(
    const ultramem_block_norm_args *p, const void *u, const void *du, int64_t ld_du,
    const void *dn, int64_t ld_dn, void *dy, void *dr, void *dgate, float *dw_post, float *db_post,
    float *dw_pre, float *db_pre, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!um::valid(p)) return ULTRAMEM_EINVAL;
    if (dgate && p->gate_mode == ULTRAMEM_GATE_NONE) return ULTRAMEM_EINVAL;
    if (p->kind == ULTRAMEM_NORM_RMS && (db_post || db_pre)) return ULTRAMEM_EINVAL;
    if ((!p->post && (dw_post || db_post)) || (!p->pre && (dw_pre || db_pre || dn)))
        return ULTRAMEM_EINVAL;
    const int D = p->dim;
    cudaStream_t st = (cudaStream_t)stream;
    float *channel_gate = p->gate_mode == ULTRAMEM_GATE_CHANNEL ? static_cast<float *>(dgate) : nullptr;
    const um::ColOut cols = {dw_post, db_post, channel_gate, dw_pre, db_pre,
                             p->post ? p->w_post : nullptr, p->post ? p->b_post : nullptr,
                             p->gate_mode == ULTRAMEM_GATE_CHANNEL ? static_cast<const float *>(p->gate)
                                                                   : nullptr,
                             p->out_scale};
    float *const sums[5] = {dw_post, db_post, channel_gate, dw_pre, db_pre};
    cudaGetLastError();
    if (p->n_tokens == 0) {   // empty sums
        for (float *o : sums)
            if (o) {
                cudaError_t e = cudaMemsetAsync(o, 0, sizeof(float) * D, st);
                if (e != cudaSuccess) return um::status_from_cuda(e);
            }
        return ULTRAMEM_OK;
    }
    if (!p->y || p->ld_y < D || (p->pre && (!u || !dn || p->ld_r < D || ld_dn < D)) ||
        (du && ld_du < D) || (!du && !dn) || !workspace || !um::aligned16(workspace) ||
        workspace_bytes < ultramem_block_norm_backward_workspace(p->n_tokens, D))
        return ULTRAMEM_EINVAL;
    const int es = p->dtype == ULTRAMEM_BF16 ? 2 : 4;
    if (!um::on_boundary(es, {p->y, p->pre ? u : nullptr, du, dn, dy, dr}) ||
        !um::on_boundary(4, {dw_post, db_post, dw_pre, db_pre}) ||
        !um::params_on_boundary(p, dgate) ||
        !um::backward_apart(p, u, du, ld_du, dn, ld_dn, dy, dr, dgate, dw_post, db_post, dw_pre,
                            db_pre, workspace,
                            ultramem_block_norm_backward_workspace(p->n_tokens, D)))
        return ULTRAMEM_EINVAL;
    um::NormArgs a = um::args_of(p);
    a.r = u;
    a.du = du;
    a.dn = dn;
    a.ld_du = ld_du;
    a.ld_dn = ld_dn;
    a.dy = dy;
    a.dr = dr;
    a.dgate_rows = channel_gate ? nullptr : dgate;
    a.part = static_cast<float *>(workspace);
    const bool full = p->gate_mode == ULTRAMEM_GATE_FULL;
    const void *channel = p->gate_mode == ULTRAMEM_GATE_CHANNEL ? p->gate : nullptr;
    const int mode = um::mode_of(
        p->dtype, D,
        {p->y, p->pre ? u : nullptr, du, dn, dy, dr, full ? p->gate : nullptr, full ? dgate : nullptr},
        {p->ld_y, p->pre ? p->ld_r : 0, du ? ld_du : 0, dn ? ld_dn : 0},
        {p->w_post, p->b_post, p->w_pre, p->b_pre, channel});
    const bool layer = p->kind == ULTRAMEM_NORM_LAYER;
    int groups = 0;
    cudaError_t e = um::dispatch<um::Backward>(a, p->dtype, layer, mode, &groups, st);
    if (e != cudaSuccess) return um::status_from_cuda(e);
    bool any = false;
    for (float *o : sums) any = any || o;
    if (any) {
        e = um::launch_kernel(true, um::column_sum_kernel, dim3((D + 31) / 32, 2), 1024, 0, st,
                              (const float *)a.part, groups, layer ? 1 : 0, D, cols);
    }
    return um::status_from_cuda(e);
}

// um_attn_grad.cu -- the gradient of the attention of whole sequences: the call
// itself, the pass that prepares it (the sums d_i = dout_i . out_i and the
// list of blocks), and the kernel of the storages and head widths that the
// tensor-core kernels do not take.
//
// With P_ij = e^(scale q_i k_j - lse_i) and dS_ij = scale P_ij (dout_i v_j - d_i):
//   dv_j = sum_i P_ij dout_i,  dk_j = sum_i dS_ij q_i,  dq_i = sum_j dS_ij k_j
// P is computed again from the stored lse, so nothing of the size of the
// scores is read or written.  dk and dv are sums over rows, dq over keys: two
// kernels, one that holds a block of keys and streams the rows that see them
// (of all query heads of the key/value head), one that holds a block of rows
// and streams the keys they see.  Both compute P and dS; in return no sum is
// shared between blocks, there is no second pass over partial sums, and the
// order of every sum is fixed.
#include "um_attn_grad.cuh"

#include "um_device.cuh"
#include "um_overlap.cuh"
#include "um_paged.cuh"
#include "um_tc.cuh"

namespace um {
namespace attn_grad {
namespace {

// ---- preparation -------------------------------------------------------------

// 8 entries of a row as they are loaded, in 16-byte pieces or one by one
template <typename T, bool WIDE> struct Eight {
    uint4 x[sizeof(T) / 2];
    __device__ __forceinline__ void get(const T *p) {
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i)
                x[i] = reinterpret_cast<const uint4 *>(p)[i];
        } else {
            T v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = p[k];
            memcpy(x, v, sizeof v);
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) x[i] = make_uint4(0, 0, 0, 0);
    }
};
__device__ __forceinline__ float dot4(uint4 a, uint4 b, float s, const float *) {
    s = fmaf(__uint_as_float(a.x), __uint_as_float(b.x), s);
    s = fmaf(__uint_as_float(a.y), __uint_as_float(b.y), s);
    s = fmaf(__uint_as_float(a.z), __uint_as_float(b.z), s);
    return fmaf(__uint_as_float(a.w), __uint_as_float(b.w), s);
}
__device__ __forceinline__ float dot4(uint4 a, uint4 b, float s, const __nv_bfloat16 *) {
    const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), s);
        s = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), s);
    }
    return s;
}

// The lists of blocks, by one thread block.  A sequence of n blocks has one of
// each length 1..n, in rows that see a key block and in keys that a row
// block sees, so that one count by length places both lists, the longest first
// (lengths past kLengths count as that).
constexpr int kLengths = 1024;
__device__ void list_blocks(const Args &a) {
    __shared__ int count[kLengths + 1], at[2][kLengths + 1], scan[8];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    auto sequence = [&](int64_t r, int &tok0, int &n) {
        tok0 = max(0, a.q_start[r]);
        n = max(0, min(a.T, a.q_start[r + 1]) - tok0);
        return (int)(((int64_t)n + a.block - 1) / a.block);
    };
    for (int i = tid; i <= kLengths; i += 256) count[i] = 0;
    __syncthreads();
    // by a sequence's own number of blocks, and what lies past the last length
    for (int64_t r = tid; r < a.n_seqs; r += 256) {
        int tok0, n;
        const int blocks = sequence(r, tok0, n);
        if (blocks) atomicAdd(&count[min(blocks, kLengths)], 1);
        if (blocks > kLengths) atomicAdd(&count[0], blocks - kLengths);
    }
    __syncthreads();
    // blocks of length l: sequences of at least l blocks; four lengths a thread,
    // from the longest, sums over threads by a scan
    const int top = kLengths - 4 * tid;
    int own[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += own[i] = count[top - i];
    auto before = [&](int v) {
        int upto = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        __syncthreads();
        if (lane == 31) scan[w] = upto;
        __syncthreads();
        int base = upto - v;
        for (int i = 0; i < w; ++i) base += scan[i];
        return base;
    };
    int longer = before(sum), of[4], total = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) total += of[i] = longer += own[i];
    if (tid == 0) {
        total += count[0];                  // the blocks past the last length, counted as that
        of[0] += count[0];
    }
    int start = before(total);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        at[0][top - i] = at[1][top - i] = start;
        start += of[i];
    }
    if (tid == 255) *a.count = min(start, a.most);
    __syncthreads();
    // a warp a sequence, so that a long one is listed in few steps
    for (int64_t r0 = 0; r0 < a.n_seqs; r0 += 256) {
        int tok0 = 0, n = 0, blocks = 0;
        if (r0 + tid < a.n_seqs) blocks = sequence(r0 + tid, tok0, n);
        for (int i = 0; i < 32; ++i) {
            const int t0 = __shfl_sync(0xffffffffu, tok0, i);
            const int tn = __shfl_sync(0xffffffffu, n, i);
            const int nb = __shfl_sync(0xffffffffu, blocks, i);
            for (int b = lane; b < nb; b += 32) {
                const int k = atomicAdd(&at[0][min(nb - b, kLengths)], 1);
                if (k < a.most) a.blocks[k] = make_int4(t0, tn, b, 0);
                const int q = atomicAdd(&at[1][min(b + 1, kLengths)], 1);
                if (q < a.most) a.blocks[a.most + q] = make_int4(t0, tn, b, 0);
            }
        }
    }
}

// Block 0 lists the sequences' blocks; the others compute d_i: 2^lanes_log2 lanes
// a row and head, 8 entries each (a warp takes as many rows as fit, four times
// over, so that enough loads are in flight).  Bound by reading dout and out.
template <typename T, bool WIDE> __global__ void __launch_bounds__(256)
    prepare_kernel(Args a, int lanes_log2) {
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0) {
        list_blocks(a);
        return;
    }
    constexpr int kAhead = 4;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int per_row = 1 << lanes_log2, part = lane & (per_row - 1);
    const int64_t rows = (int64_t)a.T * a.q_heads;
    const int64_t per_warp = 32 >> lanes_log2;
    const int64_t step = (int64_t)(gridDim.x - 1) * 8 * per_warp * kAhead;
    const int64_t first =
        ((int64_t)(blockIdx.x - 1) * 8 + w) * per_warp * kAhead + (lane >> lanes_log2);
    for (int64_t i0 = first; i0 - (lane >> lanes_log2) < rows; i0 += step) {
        Eight<T, WIDE> x[kAhead], y[kAhead];
        int64_t t[kAhead];
        int h[kAhead];
        t[0] = i0 / a.q_heads;
        h[0] = (int)(i0 - t[0] * a.q_heads);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t i = i0 + k * per_warp;
            if (k > 0) {
                t[k] = t[k - 1];
                h[k] = h[k - 1] + (int)per_warp;
                while (h[k] >= a.q_heads) {
                    h[k] -= a.q_heads;
                    ++t[k];
                }
            }
            if (i < rows && part * 8 < a.D) {
                const int64_t at = (int64_t)h[k] * a.D + part * 8;
                x[k].get(static_cast<const T *>(a.dout) + t[k] * a.dout_stride + at);
                y[k].get(static_cast<const T *>(a.out) + t[k] * a.out_stride + at);
            } else {
                x[k].zero();
                y[k].zero();
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float s = 0.f;
#pragma unroll
            for (int c = 0; c < (int)sizeof(T) / 2; ++c)
                s = dot4(x[k].x[c], y[k].x[c], s, static_cast<const T *>(nullptr));
            for (int o = per_row / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (part == 0 && i0 + k * per_warp < rows) {
                const float lse = a.lse[i0 + k * per_warp];
                // weights e^(score - inf) = 0 for a row that saw nothing
                a.rows[(int64_t)h[k] * a.T + t[k]] =
                    make_float2(lse == -INFINITY ? INFINITY : lse, s);
            }
        }
    }
}

// ---- the CUDA-core kernel ----------------------------------------------------
// 256 threads hold a block of HELD rows and stream blocks of 32.  A thread
// computes HELD / 16 x 2 scores and as many dout . v from shared memory, then,
// with P and dS in shared memory, its part of the held rows' sums.  The next block
// is on its way into registers meanwhile (heads up to 128 wide).  Bound by the fp32
// pipes and shared-memory reads, and in a short batch by the steps of its
// longest block: there blocks are half as high (5 sequences of up to 300 tokens,
// 4 heads x 80: 54 us; 133 with blocks of 64, columns padded to 128, no loads ahead
// and a load for each of the sums' operands).

constexpr int kStream = 32;
constexpr int kThreads = 256;

template <int DP, int HELD> struct Shape {
    static constexpr int kPad = DP + 4;                  // conflict-free rows
    static constexpr int kWPad = HELD + 4;
    static constexpr bool kPrefetch = DP <= 128;
    static constexpr size_t kSmem =
        sizeof(float) * ((size_t)2 * (HELD + kStream) * kPad + 2 * kStream * kWPad + 2 * 64);
};

__device__ __forceinline__ float4 load4(const float *p, bool wide) {
    if (wide) return *reinterpret_cast<const float4 *>(p);
    return make_float4(p[0], p[1], p[2], p[3]);
}
__device__ __forceinline__ float4 load4(const __nv_bfloat16 *p, bool wide) {
    if (wide) {
        const uint2 x = *reinterpret_cast<const uint2 *>(p);
        return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u),
                           __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u));
    }
    return make_float4(to_f(p[0]), to_f(p[1]), to_f(p[2]), to_f(p[3]));
}

// 2 or 4 neighbours of shared memory, in one load
template <int N> __device__ __forceinline__ void load_shared(const float *p, float *v) {
    if constexpr (N == 4) {
        const float4 x = *reinterpret_cast<const float4 *>(p);
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
    } else {
        static_assert(N == 2, "pairs");
        const float2 x = *reinterpret_cast<const float2 *>(p);
        v[0] = x.x, v[1] = x.y;
    }
}

// ROWS rows of a tensor from row `first` on, zeros past `end`, in registers on
// their way to shared memory.
template <typename T, int DP, int ROWS> struct Block {
    static constexpr int kN = ROWS * DP / 4 / kThreads;
    static_assert(kN * kThreads * 4 == ROWS * DP, "whole pieces");
    float4 v[kN];
    __device__ __forceinline__ void get(const void *src, int64_t stride, int64_t head, int64_t first,
                                        int64_t end, int D, bool wide) {
        const T *p = static_cast<const T *>(src) + head;
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            const int i = k * kThreads + threadIdx.x, r = i / (DP / 4), c = i % (DP / 4) * 4;
            v[k] = first + r < end && c < D ? load4(p + (first + r) * stride + c, wide)
                                            : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    __device__ __forceinline__ void put(float *dst) const {
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            const int i = k * kThreads + threadIdx.x, r = i / (DP / 4), c = i % (DP / 4) * 4;
            *reinterpret_cast<float4 *>(dst + r * (DP + 4) + c) = v[k];
        }
    }
};

// KEYS: holds keys and values, streams queries and output gradients, writes dk
// and dv; else the other way round, and dq.  `ranks` CTAs of a cluster may share
// out the steps of a block of keys, and then its rows, of which each adds the sums
// of all in their order.
template <typename T, int DP, int HELD, bool KEYS>
__device__ __forceinline__ void rows_run(float *sm, const Args &a, unsigned cta, int rank,
                                         int ranks) {
    using S = Shape<DP, HELD>;
    constexpr int kPad = S::kPad, kWPad = S::kWPad;
    constexpr int kH = HELD / 16;                        // held rows of a thread's scores
    constexpr int kC = DP / 16, kV = kC % 4 ? 2 : 4;     // columns of a thread's sums, neighbours
    float *h0 = sm, *h1 = h0 + HELD * kPad;              // K and V, or Q and dout
    float *s0 = h1 + HELD * kPad, *s1 = s0 + kStream * kPad;
    float *wp = s1 + kStream * kPad, *wd = wp + kStream * kWPad;   // P and dS, [streamed][held]
    float *lse = wd + kStream * kWPad, *di = lse + 64;
    const int heads = KEYS ? a.kv_heads : a.q_heads;
    const int index = (int)(cta / heads), head = (int)(cta % heads);
    if (index >= *a.count) return;
    const int4 blk = a.blocks[KEYS ? index : a.most + index];   // the longest first
    const int64_t tok0 = blk.x, end = tok0 + blk.y;
    const int64_t first = tok0 + (int64_t)blk.z * HELD;
    const int kv = KEYS ? head : head / a.group;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const bool wide = a.wide;
    float acc0[kH][kC], acc1[kH][kC];                    // dv and dk, or (acc1) dq
#pragma unroll
    for (int i = 0; i < kH; ++i)
#pragma unroll
        for (int c = 0; c < kC; ++c) acc0[i][c] = acc1[i][c] = 0.f;
    // what is streamed: Q and dout of the group's heads, or K and V
    const void *src0 = KEYS ? a.q : a.k, *src1 = KEYS ? a.dout : a.v;
    const int64_t st0 = KEYS ? a.q_stride : a.k_stride, st1 = KEYS ? a.dout_stride : a.v_stride;
    const int64_t from = KEYS ? first : tok0, to = KEYS ? end : min(end, first + HELD);
    const int per_head = (int)((to - from + kStream - 1) / kStream);
    const int steps = (KEYS ? a.group : 1) * per_head;
    Block<T, DP, kStream> n0, n1;
    float2 row = make_float2(0.f, 0.f);
    auto fetch = [&](int j) {
        const int h = KEYS ? kv * a.group + j / per_head : kv;
        const int64_t r0 = from + (int64_t)(j % per_head) * kStream;
        n0.get(src0, st0, (int64_t)h * a.D, r0, end, a.D, wide);
        n1.get(src1, st1, (int64_t)h * a.D, r0, end, a.D, wide);
        if (KEYS && threadIdx.x < kStream && r0 + threadIdx.x < end)
            row = a.rows[(int64_t)h * a.T + r0 + threadIdx.x];
    };
    {
        Block<T, DP, HELD> b;
        b.get(KEYS ? a.k : a.q, KEYS ? a.k_stride : a.q_stride, (int64_t)head * a.D, first, end, a.D,
              wide);
        b.put(h0);
        b.get(KEYS ? a.v : a.dout, KEYS ? a.v_stride : a.dout_stride, (int64_t)head * a.D, first, end,
              a.D, wide);
        b.put(h1);
        if (!KEYS && threadIdx.x < HELD && first + threadIdx.x < end) {
            const float2 r = a.rows[(int64_t)head * a.T + first + threadIdx.x];
            lse[threadIdx.x] = r.x;
            di[threadIdx.x] = r.y;
        }
    }
    if (S::kPrefetch && rank < steps) fetch(rank);
    for (int j = rank; j < steps; j += ranks) {
        const int64_t r0 = from + (int64_t)(j % per_head) * kStream;
        if (!S::kPrefetch) fetch(j);
        __syncthreads();
        n0.put(s0);
        n1.put(s1);
        if (KEYS && threadIdx.x < kStream) {
            lse[threadIdx.x] = row.x;
            di[threadIdx.x] = row.y;
        }
        __syncthreads();
        if (S::kPrefetch && j + ranks < steps) fetch(j + ranks);
        const int live = (int)min((int64_t)kStream, to - r0);    // streamed rows
        float s[kH][2], dp[kH][2];
#pragma unroll
        for (int i = 0; i < kH; ++i) s[i][0] = s[i][1] = dp[i][0] = dp[i][1] = 0.f;
#pragma unroll 4
        for (int c = 0; c < a.D; c += 4) {
            float4 x0[2], x1[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                x0[q] = *reinterpret_cast<const float4 *>(s0 + (ty + 16 * q) * kPad + c);
                x1[q] = *reinterpret_cast<const float4 *>(s1 + (ty + 16 * q) * kPad + c);
            }
#pragma unroll
            for (int i = 0; i < kH; ++i) {
                const float4 y0 = *reinterpret_cast<const float4 *>(h0 + (tx + 16 * i) * kPad + c);
                const float4 y1 = *reinterpret_cast<const float4 *>(h1 + (tx + 16 * i) * kPad + c);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    s[i][q] = fmaf(x0[q].x, y0.x, s[i][q]);
                    s[i][q] = fmaf(x0[q].y, y0.y, s[i][q]);
                    s[i][q] = fmaf(x0[q].z, y0.z, s[i][q]);
                    s[i][q] = fmaf(x0[q].w, y0.w, s[i][q]);
                    dp[i][q] = fmaf(x1[q].x, y1.x, dp[i][q]);
                    dp[i][q] = fmaf(x1[q].y, y1.y, dp[i][q]);
                    dp[i][q] = fmaf(x1[q].z, y1.z, dp[i][q]);
                    dp[i][q] = fmaf(x1[q].w, y1.w, dp[i][q]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kH; ++i)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int held = tx + 16 * i, str = ty + 16 * q;
                const int64_t at_row = KEYS ? r0 + str : first + held;
                const int64_t key = KEYS ? first + held : r0 + str;
                const int at = KEYS ? str : held;
                float p = 0.f, d = 0.f;
                if (key <= at_row && at_row < end) {
                    p = expf(fmaf(s[i][q], a.scale, -lse[at]));
                    d = a.scale * p * (dp[i][q] - di[at]);
                }
                wp[str * kWPad + held] = p;
                wd[str * kWPad + held] = d;
            }
        __syncthreads();
#pragma unroll 4
        for (int r = 0; r < live; ++r) {
            float p[kH], d[kH], x0[kC], x1[kC];
            if (KEYS) load_shared<kH>(wp + r * kWPad + ty * kH, p);
            load_shared<kH>(wd + r * kWPad + ty * kH, d);
#pragma unroll
            for (int c = 0; c < kC; c += kV) {
                const int col = (c / kV * 16 + tx) * kV;
                load_shared<kV>(s0 + r * kPad + col, x0 + c);
                if (KEYS) load_shared<kV>(s1 + r * kPad + col, x1 + c);
            }
#pragma unroll
            for (int i = 0; i < kH; ++i)
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    if (KEYS) acc0[i][c] = fmaf(p[i], x1[c], acc0[i][c]);
                    acc1[i][c] = fmaf(d[i], x0[c], acc1[i][c]);
                }
        }
    }
    T *o1 = static_cast<T *>(KEYS ? a.dk : a.dq), *o0 = static_cast<T *>(a.dv);
    const int64_t out1 = KEYS ? a.dk_stride : a.dq_stride;
    if (KEYS && ranks > 1) {
        __syncthreads();                                 // what the sums read may go
#pragma unroll
        for (int i = 0; i < kH; ++i)
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                const int at = (ty * kH + i) * kPad + (c / kV * 16 + tx) * kV + c % kV;
                h0[at] = acc0[i][c];
                h1[at] = acc1[i][c];
            }
        tc::cluster_sync();
        const int pieces = a.D / 4;
        for (int k = threadIdx.x; k < HELD / ranks * pieces; k += kThreads) {
            const int r = rank + k / pieces * ranks, col = k % pieces * 4;
            if (first + r >= end) continue;
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const float *from = (o ? h1 : h0) + r * kPad + col;
                float4 v = load_peer(from, 0);
                for (int p = 1; p < ranks; ++p) {
                    const float4 x = load_peer(from, p);
                    v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
                }
                T *out = o ? o1 + (first + r) * out1 : o0 + (first + r) * a.dv_stride;
                out += (int64_t)head * a.D + col;
                out[0] = from_f<T>(v.x), out[1] = from_f<T>(v.y);
                out[2] = from_f<T>(v.z), out[3] = from_f<T>(v.w);
            }
        }
        __syncwarp();
        tc::cluster_sync();                              // peers have read this CTA's sums
        return;
    }
#pragma unroll
    for (int i = 0; i < kH; ++i) {
        const int64_t at = first + ty * kH + i;
        if (at >= end) continue;
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            const int col = (c / kV * 16 + tx) * kV + c % kV;
            if (col >= a.D) continue;
            o1[at * out1 + (int64_t)head * a.D + col] = from_f<T>(acc1[i][c]);
            if (KEYS) o0[at * a.dv_stride + (int64_t)head * a.D + col] = from_f<T>(acc0[i][c]);
        }
    }
}

// Both roles in one launch, held keys first: a cluster a block of keys, or as many
// blocks of rows as it has CTAs.
template <typename T, int DP, int HELD>
__global__ void __launch_bounds__(kThreads) rows_kernel(Args a) {
    extern __shared__ float sm[];
    pdl_wait();
    pdl_trigger();
    const unsigned keys = (unsigned)a.most * a.kv_heads;
    if (blockIdx.x < keys)
        rows_run<T, DP, HELD, true>(sm, a, blockIdx.x, blockIdx.z, gridDim.z);
    else
        rows_run<T, DP, HELD, false>(sm, a, (blockIdx.x - keys) * gridDim.z + blockIdx.z, 0, 1);
}

template <typename T, int DP, int HELD> cudaError_t rows_go(const Args &a, cudaStream_t st) {
    constexpr size_t smem = Shape<DP, HELD>::kSmem;
    const cudaError_t e = allow_dynamic_smem<rows_kernel<T, DP, HELD>>(smem);
    if (e != cudaSuccess) return e;
    return launch_kernel(true, (unsigned)a.ranks, rows_kernel<T, DP, HELD>, grid_of(a), kThreads, smem,
                         st, a);
}
template <typename T, int DP> cudaError_t rows_held(const Args &a, cudaStream_t st) {
    return a.block == 32 ? rows_go<T, DP, 32>(a, st) : rows_go<T, DP, 64>(a, st);
}
template <typename T> cudaError_t rows_dim(const Args &a, cudaStream_t st) {
    if (a.D <= 64) return rows_held<T, 64>(a, st);
    if (a.D <= 96) return rows_held<T, 96>(a, st);
    if (a.D <= 128) return rows_held<T, 128>(a, st);
    return rows_go<T, 256, 32>(a, st);
}

template <typename T> cudaError_t launch_prepare(const Args &a, cudaStream_t st) {
    int lanes = 0;                         // log2 of the lanes of a row: 8 entries each
    while ((8 << lanes) < a.D) ++lanes;
    const int64_t rows = (int64_t)a.T * a.q_heads, per_block = (8 * 4 * 32) >> lanes;
    const int64_t want = (rows + per_block - 1) / per_block;
    const int64_t most = (int64_t)device_sm_count() * 8;
    const unsigned grid = (unsigned)(1 + (want < most ? want : most));
    const bool wide =
        ((uintptr_t)a.dout | (uintptr_t)a.out | (uintptr_t)((a.dout_stride | a.out_stride) * sizeof(T))) %
            16 == 0;
    if (wide)
        prepare_kernel<T, true><<<grid, 256, 0, st>>>(a, lanes);
    else
        prepare_kernel<T, false><<<grid, 256, 0, st>>>(a, lanes);
    return cudaGetLastError();
}

// Rows of a block on the CUDA cores: 64, or 32 for wide heads and batches whose
// higher blocks would leave SMs idle.
int block_of(int32_t T, int32_t heads, int32_t dim) {
    return dim > 128 || (int64_t)T / 64 * heads < 2 * device_sm_count() ? 32 : 64;
}

// CTAs that share out the steps of a block of held keys, with streamed blocks of
// `stream` rows and room for `slots` CTAs.  A block of keys has the query heads'
// steps one after another, `group` times those of a block of rows: where that is
// far more than a slot's part of the whole batch, it is divided until it is not, and
// no more, because each CTA holds and adds the block again.  (By 1, 2, 4 CTAs: bf16, one
// sequence of 4096, 8 heads on 1 x 128, 323, 172, 99 us, 32 heads on 8, 320, 341, 424;
// fp32, 4 sequences of 512, 8 heads on 2 x 64, 358, 184, 179, 16 of 1000, 2353, 2394,
// 2564.)  More than `group` CTAs help only while `spare` SMs would be idle.  By the
// mean length: the host does not know the others.
int ranks_of(const Args &a, int stream, int64_t slots, int64_t spare) {
    const int64_t mean = (a.T / a.n_seqs + stream - 1) / stream, steps = a.group * mean;
    const int64_t all = (int64_t)a.most * a.q_heads * (mean + 1);    // of both roles
    auto ctas = [&](int n) { return (int64_t)a.most * ((int64_t)n * a.kv_heads + a.q_heads); };
    int n = 1;
    while (n < 8 && 2 * n <= steps && 5 * steps * slots > 8 * n * all &&
           (2 * n <= a.group || ctas(2 * n) <= spare))
        n *= 2;
    return n;
}

// Blocks of the sequences, at most: whole ones, and a short one for each that
// has tokens.
int64_t most_blocks(int32_t T, int32_t n_seqs, int block) {
    return (int64_t)T / block + (n_seqs < T ? n_seqs : T);
}

struct Layout {
    int64_t rows, blocks, count, total;
};
Layout layout_of(int32_t T, int32_t n_seqs, int32_t q_heads) {
    Layout l = {};
    // room for the lower blocks, whichever the call takes
    const int64_t most = most_blocks(T, n_seqs, 32);
    l.rows = 0;
    l.blocks = ((int64_t)T * q_heads * 8 + 15) & ~15ll;
    l.count = l.blocks + 2 * most * 16;
    l.total = l.count + 16;
    return l;
}

bool heads_ok(int32_t dtype, int32_t q_heads, int32_t kv_heads, int32_t dim) {
    return (dtype == ULTRAMEM_F32 || dtype == ULTRAMEM_BF16) && kv_heads > 0 && kv_heads <= 1024 &&
           q_heads > 0 && q_heads % kv_heads == 0 && q_heads / kv_heads <= 64 && dim > 0 &&
           dim <= kMaxHeadDim && dim % 8 == 0;
}
// what grids and offsets hold
bool sizes_ok(int32_t T, int32_t n_seqs, int32_t q_heads) {
    return T >= 0 && n_seqs >= 0 && most_blocks(T, n_seqs, 32) * 2 * q_heads <= INT32_MAX;
}

}  // namespace
}  // namespace attn_grad
}  // namespace um

using namespace um::attn_grad;

extern "C" int64_t ultramem_paged_attention_backward_workspace(int32_t dtype, int32_t n_tokens,
                                                               int32_t n_seqs, int32_t q_heads,
                                                               int32_t kv_heads,
                                                               int32_t head_dim) {
    if (!heads_ok(dtype, q_heads, kv_heads, head_dim) ||
        !sizes_ok(n_tokens, n_seqs, q_heads))
        return 0;
    return layout_of(n_tokens, n_seqs, q_heads).total;
}

extern "C" ultramem_status ultramem_paged_attention_backward(const ultramem_attention_grad *p,
                                                             void *workspace,
                                                             int64_t workspace_bytes,
                                                             void *stream) {
    if (!p || !heads_ok(p->dtype, p->q_heads, p->kv_heads, p->head_dim) ||
        !sizes_ok(p->n_tokens, p->n_seqs, p->q_heads) || !(p->scale > 0.f) ||
        !(p->scale * kLog2e < INFINITY))
        return ULTRAMEM_EINVAL;
    if (p->n_tokens == 0 || p->n_seqs == 0) return ULTRAMEM_OK;
    const int es = p->dtype == ULTRAMEM_BF16 ? 2 : 4;
    const int64_t qr = (int64_t)p->q_heads * p->head_dim, kr = (int64_t)p->kv_heads * p->head_dim;
    if (!p->q || !p->k || !p->v || !p->out || !p->dout || !p->dq || !p->dk || !p->dv || !p->lse ||
        !p->q_start || !workspace || ((uintptr_t)workspace & 15))
        return ULTRAMEM_EINVAL;
    if (((uintptr_t)p->q | (uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->out |
         (uintptr_t)p->dout | (uintptr_t)p->dq | (uintptr_t)p->dk | (uintptr_t)p->dv) % es ||
        ((uintptr_t)p->lse | (uintptr_t)p->q_start) % 4)
        return ULTRAMEM_EINVAL;
    if (p->q_stride < qr || p->out_stride < qr || p->dout_stride < qr || p->dq_stride < qr ||
        p->k_stride < kr || p->v_stride < kr || p->dk_stride < kr || p->dv_stride < kr)
        return ULTRAMEM_EINVAL;
    const Layout l = layout_of(p->n_tokens, p->n_seqs, p->q_heads);
    if (workspace_bytes < l.total) return ULTRAMEM_EINVAL;
    const int64_t T = p->n_tokens;
    auto rows_of = [&](const void *at, int64_t row, int64_t stride) {
        return um::Memory{at, row * es, T, stride * es};
    };
    const um::Memory in[7] = {rows_of(p->q, qr, p->q_stride),
                              rows_of(p->k, kr, p->k_stride),
                              rows_of(p->v, kr, p->v_stride),
                              rows_of(p->out, qr, p->out_stride),
                              rows_of(p->dout, qr, p->dout_stride),
                              {p->lse, T * p->q_heads * 4},
                              {p->q_start, ((int64_t)p->n_seqs + 1) * 4}};
    const um::Memory out[3] = {rows_of(p->dq, qr, p->dq_stride), rows_of(p->dk, kr, p->dk_stride),
                               rows_of(p->dv, kr, p->dv_stride)};
    const um::Memory ws = {workspace, l.total};
    for (int i = 0; i < 3; ++i) {
        if (um::overlap(ws, out[i])) return ULTRAMEM_EINVAL;
        for (int j = 0; j < i; ++j)
            if (um::rows_overlap(out[i], out[j])) return ULTRAMEM_EINVAL;
        for (const um::Memory &m : in)
            if (um::rows_overlap(out[i], m)) return ULTRAMEM_EINVAL;
    }
    for (const um::Memory &m : in)
        if (um::overlap(ws, m)) return ULTRAMEM_EINVAL;
    Args a = {};
    a.q = p->q;
    a.k = p->k;
    a.v = p->v;
    a.out = p->out;
    a.dout = p->dout;
    a.dq = p->dq;
    a.dk = p->dk;
    a.dv = p->dv;
    a.lse = p->lse;
    a.q_start = p->q_start;
    a.q_stride = p->q_stride;
    a.k_stride = p->k_stride;
    a.v_stride = p->v_stride;
    a.out_stride = p->out_stride;
    a.dout_stride = p->dout_stride;
    a.dq_stride = p->dq_stride;
    a.dk_stride = p->dk_stride;
    a.dv_stride = p->dv_stride;
    char *at = static_cast<char *>(workspace);
    a.rows = reinterpret_cast<float2 *>(at + l.rows);
    a.blocks = reinterpret_cast<int4 *>(at + l.blocks);
    a.count = reinterpret_cast<int *>(at + l.count);
    a.n_seqs = p->n_seqs;
    a.T = p->n_tokens;
    a.q_heads = p->q_heads;
    a.kv_heads = p->kv_heads;
    a.group = p->q_heads / p->kv_heads;
    a.D = p->head_dim;
    a.block = block_of(p->n_tokens, p->q_heads + p->kv_heads, p->head_dim);
    a.most = (int)most_blocks(p->n_tokens, p->n_seqs, a.block);
    a.scale = p->scale;
    a.scale_log2 = p->scale * kLog2e;
    const int64_t sms = um::device_sm_count();
    a.ranks = ranks_of(a, kStream, 2 * sms, sms);
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    cudaError_t e;
    // TMA reads the inputs, and the outputs leave, in 16-byte pieces
    const uintptr_t in_low = (uintptr_t)p->q | (uintptr_t)p->k | (uintptr_t)p->v |
                             (uintptr_t)p->dout |
                             (uintptr_t)((p->q_stride | p->k_stride | p->v_stride | p->dout_stride) * es);
    a.wide = in_low % (4 * es) == 0;
    const uintptr_t low = in_low | (uintptr_t)p->dq | (uintptr_t)p->dk | (uintptr_t)p->dv |
                          (uintptr_t)((p->dq_stride | p->dk_stride | p->dv_stride) * es);
    if (p->dtype == ULTRAMEM_BF16 && p->head_dim <= 128 && low % 16 == 0) {
        if (!(a.err = um::paged::error_word())) return ULTRAMEM_ENODEV;
        a.block = kTensorBlock;
        a.most = (int)most_blocks(p->n_tokens, p->n_seqs, kTensorBlock);
        a.ranks = ranks_of(a, kTensorBlock, sms, 0);       // <= group, as the kernel needs
        CUtensorMap q, k, v, dout;
        auto map = [&](CUtensorMap *m, const void *x, int heads, int64_t stride) {
            return um::paged::encode(m, x, a.D, heads, T, a.D, stride, 1, kTensorBlock);
        };
        if (!map(&q, a.q, a.q_heads, a.q_stride) || !map(&k, a.k, a.kv_heads, a.k_stride) ||
            !map(&v, a.v, a.kv_heads, a.v_stride) || !map(&dout, a.dout, a.q_heads, a.dout_stride))
            return um::status_from_cuda(cudaErrorInvalidValue);
        e = launch_prepare<__nv_bfloat16>(a, st);
        if (e == cudaSuccess) e = launch_tensor(a, q, k, v, dout, st);
    } else if (p->dtype == ULTRAMEM_BF16) {
        e = launch_prepare<__nv_bfloat16>(a, st);
        if (e == cudaSuccess) e = rows_dim<__nv_bfloat16>(a, st);
    } else {
        e = launch_prepare<float>(a, st);
        if (e == cudaSuccess) e = rows_dim<float>(a, st);
    }
    return um::status_from_cuda(e);
}

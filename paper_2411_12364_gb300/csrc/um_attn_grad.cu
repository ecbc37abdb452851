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
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) x[i] = reinterpret_cast<const uint4 *>(p)[i];
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
    const int64_t per_warp = 32 >> lanes_log2, step = (int64_t)(gridDim.x - 1) * 8 * per_warp * kAhead;
    const int64_t first = ((int64_t)(blockIdx.x - 1) * 8 + w) * per_warp * kAhead + (lane >> lanes_log2);
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
                a.rows[(int64_t)h[k] * a.T + t[k]] = make_float2(lse == -INFINITY ? INFINITY : lse, s);
            }
        }
    }
}

// ---- the CUDA-core kernel ----------------------------------------------------
// 256 threads hold a block of HELD rows and stream blocks of 32.  A thread
// computes HELD / 16 x 2 scores and as many dout . v from shared memory, then,
// with P and dS in shared memory, its part of the held rows' sums.  Bound by
// the fp32 pipes and shared-memory reads.

constexpr int kStream = 32;
constexpr int kThreads = 256;

template <int DP> struct Shape {
    static constexpr int kHeld = DP == 256 ? 32 : 64;
    static constexpr int kPad = DP + 4;                  // conflict-free rows
    static constexpr int kWPad = kHeld + 4;
    static constexpr size_t kSmem =
        sizeof(float) * ((size_t)2 * (kHeld + kStream) * kPad + 2 * kStream * kWPad + 2 * 64);
};

// `rows` rows of a tensor from row `first` into dst, zeros past `end`.
template <typename T, int DP>
__device__ __forceinline__ void load_rows(float *dst, const void *src, int64_t stride, int64_t head,
                                          int64_t first, int rows, int64_t end, int D) {
    constexpr int kPad = Shape<DP>::kPad;
    const T *p = static_cast<const T *>(src) + head;
    for (int i = threadIdx.x; i < rows * DP; i += kThreads) {
        const int r = i / DP, c = i % DP;
        dst[r * kPad + c] = first + r < end && c < D ? to_f(p[(first + r) * stride + c]) : 0.f;
    }
}

// KEYS: holds keys and values, streams queries and output gradients, writes dk
// and dv; else the other way round, and dq.
template <typename T, int DP, bool KEYS>
__device__ __forceinline__ void rows_run(float *sm, const Args &a, unsigned cta) {
    using S = Shape<DP>;
    constexpr int kHeld = S::kHeld, kPad = S::kPad, kWPad = S::kWPad;
    constexpr int kH = kHeld / 16;                       // held rows of a thread's scores
    constexpr int kC = DP / 16;                          // columns of a thread's sums
    float *h0 = sm, *h1 = h0 + kHeld * kPad;             // K and V, or Q and dout
    float *s0 = h1 + kHeld * kPad, *s1 = s0 + kStream * kPad;
    float *wp = s1 + kStream * kPad, *wd = wp + kStream * kWPad;   // P and dS, [streamed][held]
    float *lse = wd + kStream * kWPad, *di = lse + 64;
    const int heads = KEYS ? a.kv_heads : a.q_heads;
    const int index = (int)(cta / heads), head = (int)(cta % heads);
    if (index >= *a.count) return;
    const int4 blk = a.blocks[KEYS ? index : a.most + index];   // the longest first
    const int64_t tok0 = blk.x, end = tok0 + blk.y;
    const int64_t first = tok0 + (int64_t)blk.z * kHeld;
    const int kv = KEYS ? head : head / a.group;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc0[kH][kC], acc1[kH][kC];                    // dv and dk, or (acc1) dq
#pragma unroll
    for (int i = 0; i < kH; ++i)
#pragma unroll
        for (int c = 0; c < kC; ++c) acc0[i][c] = acc1[i][c] = 0.f;
    if (KEYS) {
        load_rows<T, DP>(h0, a.k, a.k_stride, (int64_t)kv * a.D, first, kHeld, end, a.D);
        load_rows<T, DP>(h1, a.v, a.v_stride, (int64_t)kv * a.D, first, kHeld, end, a.D);
    } else {
        load_rows<T, DP>(h0, a.q, a.q_stride, (int64_t)head * a.D, first, kHeld, end, a.D);
        load_rows<T, DP>(h1, a.dout, a.dout_stride, (int64_t)head * a.D, first, kHeld, end, a.D);
        if (threadIdx.x < kHeld && first + threadIdx.x < end) {
            const float2 r = a.rows[(int64_t)head * a.T + first + threadIdx.x];
            lse[threadIdx.x] = r.x;
            di[threadIdx.x] = r.y;
        }
    }
    const int64_t from = KEYS ? first : tok0, to = KEYS ? end : min(end, first + kHeld);
    for (int g = 0; g < (KEYS ? a.group : 1); ++g) {
        const int h = KEYS ? kv * a.group + g : head;
        for (int64_t r0 = from; r0 < to; r0 += kStream) {
            __syncthreads();
            if (KEYS) {
                load_rows<T, DP>(s0, a.q, a.q_stride, (int64_t)h * a.D, r0, kStream, end, a.D);
                load_rows<T, DP>(s1, a.dout, a.dout_stride, (int64_t)h * a.D, r0, kStream, end,
                                 a.D);
                if (threadIdx.x < kStream && r0 + threadIdx.x < end) {
                    const float2 r = a.rows[(int64_t)h * a.T + r0 + threadIdx.x];
                    lse[threadIdx.x] = r.x;
                    di[threadIdx.x] = r.y;
                }
            } else {
                load_rows<T, DP>(s0, a.k, a.k_stride, (int64_t)kv * a.D, r0, kStream, end, a.D);
                load_rows<T, DP>(s1, a.v, a.v_stride, (int64_t)kv * a.D, r0, kStream, end, a.D);
            }
            __syncthreads();
            float s[kH][2], dp[kH][2];
#pragma unroll
            for (int i = 0; i < kH; ++i) s[i][0] = s[i][1] = dp[i][0] = dp[i][1] = 0.f;
#pragma unroll 4
            for (int c = 0; c < DP; c += 4) {
                float4 x0[2], x1[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    x0[j] = *reinterpret_cast<const float4 *>(s0 + (ty + 16 * j) * kPad + c);
                    x1[j] = *reinterpret_cast<const float4 *>(s1 + (ty + 16 * j) * kPad + c);
                }
#pragma unroll
                for (int i = 0; i < kH; ++i) {
                    const float4 y0 =
                        *reinterpret_cast<const float4 *>(h0 + (tx + 16 * i) * kPad + c);
                    const float4 y1 =
                        *reinterpret_cast<const float4 *>(h1 + (tx + 16 * i) * kPad + c);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        s[i][j] = fmaf(x0[j].x, y0.x, s[i][j]);
                        s[i][j] = fmaf(x0[j].y, y0.y, s[i][j]);
                        s[i][j] = fmaf(x0[j].z, y0.z, s[i][j]);
                        s[i][j] = fmaf(x0[j].w, y0.w, s[i][j]);
                        dp[i][j] = fmaf(x1[j].x, y1.x, dp[i][j]);
                        dp[i][j] = fmaf(x1[j].y, y1.y, dp[i][j]);
                        dp[i][j] = fmaf(x1[j].z, y1.z, dp[i][j]);
                        dp[i][j] = fmaf(x1[j].w, y1.w, dp[i][j]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kH; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int held = tx + 16 * i, str = ty + 16 * j;
                    const int64_t row = KEYS ? r0 + str : first + held;
                    const int64_t key = KEYS ? first + held : r0 + str;
                    const int at = KEYS ? str : held;
                    float p = 0.f, d = 0.f;
                    if (key <= row && row < end) {
                        p = expf(fmaf(s[i][j], a.scale, -lse[at]));
                        d = a.scale * p * (dp[i][j] - di[at]);
                    }
                    wp[str * kWPad + held] = p;
                    wd[str * kWPad + held] = d;
                }
            __syncthreads();
#pragma unroll 2
            for (int r = 0; r < kStream; ++r) {
                float p[kH], d[kH], x0[kC], x1[kC];
#pragma unroll
                for (int i = 0; i < kH; ++i) {
                    p[i] = wp[r * kWPad + ty * kH + i];
                    d[i] = wd[r * kWPad + ty * kH + i];
                }
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    x0[c] = s0[r * kPad + (c / 4 * 16 + tx) * 4 + c % 4];
                    x1[c] = s1[r * kPad + (c / 4 * 16 + tx) * 4 + c % 4];
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
    }
    T *o1 = static_cast<T *>(KEYS ? a.dk : a.dq), *o0 = static_cast<T *>(a.dv);
    const int64_t st1 = KEYS ? a.dk_stride : a.dq_stride;
#pragma unroll
    for (int i = 0; i < kH; ++i) {
        const int64_t row = first + ty * kH + i;
        if (row >= end) continue;
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            const int col = (c / 4 * 16 + tx) * 4 + c % 4;
            if (col >= a.D) continue;
            o1[row * st1 + (int64_t)head * a.D + col] = from_f<T>(acc1[i][c]);
            if (KEYS)
                o0[row * a.dv_stride + (int64_t)head * a.D + col] = from_f<T>(acc0[i][c]);
        }
    }
}

// Both roles in one launch, held keys first.
template <typename T, int DP>
__global__ void __launch_bounds__(kThreads) rows_kernel(Args a) {
    extern __shared__ float sm[];
    pdl_wait();
    pdl_trigger();
    const unsigned keys = (unsigned)a.most * a.kv_heads;
    if (blockIdx.x < keys)
        rows_run<T, DP, true>(sm, a, blockIdx.x);
    else
        rows_run<T, DP, false>(sm, a, blockIdx.x - keys);
}

template <typename T, int DP> cudaError_t rows_go(const Args &a, cudaStream_t st) {
    const cudaError_t e = allow_dynamic_smem<rows_kernel<T, DP>>(Shape<DP>::kSmem);
    if (e != cudaSuccess) return e;
    return launch_kernel(true, rows_kernel<T, DP>,
                         dim3((unsigned)a.most * (a.kv_heads + a.q_heads)), kThreads,
                         Shape<DP>::kSmem, st, a);
}
template <typename T> cudaError_t rows_dim(const Args &a, cudaStream_t st) {
    return a.D <= 64 ? rows_go<T, 64>(a, st)
                     : a.D <= 128 ? rows_go<T, 128>(a, st) : rows_go<T, 256>(a, st);
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

int block_of(int32_t dim) { return dim > 128 ? 32 : 64; }

// Blocks of the sequences, at most: whole ones, and a short one for each that
// has tokens.
int64_t most_blocks(int32_t T, int32_t n_seqs, int block) {
    return (int64_t)T / block + (n_seqs < T ? n_seqs : T);
}

struct Layout {
    int block, most;
    int64_t rows, blocks, count, total;
};
Layout layout_of(int32_t T, int32_t n_seqs, int32_t q_heads, int32_t dim) {
    Layout l = {};
    l.block = block_of(dim);
    const int64_t most = most_blocks(T, n_seqs, l.block);
    l.most = (int)most;
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
bool sizes_ok(int32_t T, int32_t n_seqs, int32_t q_heads, int32_t dim) {
    return T >= 0 && n_seqs >= 0 && most_blocks(T, n_seqs, block_of(dim)) * 2 * q_heads <= INT32_MAX;
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
        !sizes_ok(n_tokens, n_seqs, q_heads, head_dim))
        return 0;
    return layout_of(n_tokens, n_seqs, q_heads, head_dim).total;
}

extern "C" ultramem_status ultramem_paged_attention_backward(const ultramem_attention_grad *p,
                                                             void *workspace,
                                                             int64_t workspace_bytes,
                                                             void *stream) {
    if (!p || !heads_ok(p->dtype, p->q_heads, p->kv_heads, p->head_dim) ||
        !sizes_ok(p->n_tokens, p->n_seqs, p->q_heads, p->head_dim) || !(p->scale > 0.f) ||
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
    const Layout l = layout_of(p->n_tokens, p->n_seqs, p->q_heads, p->head_dim);
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
    a.block = l.block;
    a.most = l.most;
    a.scale = p->scale;
    a.scale_log2 = p->scale * kLog2e;
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    cudaError_t e;
    // TMA reads the inputs, and the outputs leave, in 16-byte pieces
    const uintptr_t low = (uintptr_t)p->q | (uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->dout |
                          (uintptr_t)p->dq | (uintptr_t)p->dk | (uintptr_t)p->dv |
                          (uintptr_t)((p->q_stride | p->k_stride | p->v_stride | p->dout_stride |
                                       p->dq_stride | p->dk_stride | p->dv_stride) * es);
    if (p->dtype == ULTRAMEM_BF16 && p->head_dim <= 128 && low % 16 == 0) {
        if (!(a.err = um::paged::error_word())) return ULTRAMEM_ENODEV;
        a.block = kTensorBlock;
        a.most = (int)most_blocks(p->n_tokens, p->n_seqs, kTensorBlock);
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

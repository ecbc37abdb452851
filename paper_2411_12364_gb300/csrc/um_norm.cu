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
// and n written once, about 30 operations apart, so the bound is memory.
// A row stays in registers between its two norms: a warp owns a row of up to
// 1024 entries (no block barrier), a block a wider one.  Blocks are
// persistent, so that the gains, biases and the per-channel gate are read
// once per block, into registers.
#include "um_internal.cuh"

namespace um {
namespace {

constexpr unsigned kFull = 0xffffffffu;

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
// Thread t of the TPR threads of a row holds 8 NV entries.  With 16-byte
// aligned rows (VEC) these are NV runs of 8 (run v: entries 8 (t + TPR v)..),
// one or two 16-byte accesses each; otherwise single entries t + TPR e, so
// that a warp's accesses are still consecutive.
template <int NV, bool VEC, int TPR> struct Row {
    static constexpr int kN = 8 * NV;
    __device__ static __forceinline__ int col(int t, int e) {
        return VEC ? 8 * (t + TPR * (e >> 3)) + (e & 7) : t + TPR * e;
    }
    template <typename T>
    __device__ static __forceinline__ void load(float (&x)[kN], const T *row, int t, int D) {
        if constexpr (VEC) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = 8 * (t + TPR * v);
                if constexpr (sizeof(T) == 2) {
                    uint4 q = make_uint4(0, 0, 0, 0);
                    if (c < D) q = *reinterpret_cast<const uint4 *>(row + c);
                    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[8 * v + 2 * i] = __uint_as_float(w[i] << 16);
                        x[8 * v + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (c + 4 * i < D) q = *reinterpret_cast<const float4 *>(row + c + 4 * i);
                        x[8 * v + 4 * i] = q.x;
                        x[8 * v + 4 * i + 1] = q.y;
                        x[8 * v + 4 * i + 2] = q.z;
                        x[8 * v + 4 * i + 3] = q.w;
                    }
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const int c = t + TPR * e;
                x[e] = c < D ? to_f(row[c]) : 0.f;
            }
        }
    }
    template <typename T>
    __device__ static __forceinline__ void store(T *row, const float (&x)[kN], int t, int D) {
        if constexpr (VEC) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = 8 * (t + TPR * v);
                if constexpr (sizeof(T) == 2) {
                    if (c < D) {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const __nv_bfloat162 b =
                                __floats2bfloat162_rn(x[8 * v + 2 * i], x[8 * v + 2 * i + 1]);
                            w[i] = *reinterpret_cast<const uint32_t *>(&b);
                        }
                        *reinterpret_cast<uint4 *>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (c + 4 * i < D)
                            *reinterpret_cast<float4 *>(row + c + 4 * i) =
                                make_float4(x[8 * v + 4 * i], x[8 * v + 4 * i + 1],
                                            x[8 * v + 4 * i + 2], x[8 * v + 4 * i + 3]);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) {
                const int c = t + TPR * e;
                if (c < D) row[c] = from_f<T>(x[e]);
            }
        }
    }
    // a parameter vector, or `fill` everywhere without one
    __device__ static __forceinline__ void param(float (&x)[kN], const float *p, float fill, int t,
                                                 int D) {
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const int c = col(t, e);
            x[e] = c < D ? (p ? p[c] : fill) : 0.f;
        }
    }
};

// Sums of K values over the TPR threads of a row, returned to all of them.
// A block of several warps leaves its warps' sums in shared memory, in one
// of two buffers in turn, so that one barrier serves each sum.
template <int K, int TPR> struct RowSum {
    float (*buf)[32 * 3];
    int turn;
    __device__ __forceinline__ void operator()(float (&v)[K]) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1)
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(kFull, v[k], off);
        if constexpr (TPR > 32) {
            float *b = buf[turn];
            turn ^= 1;
            const int w = threadIdx.x >> 5;
            if ((threadIdx.x & 31) == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) b[w * K + k] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = 0.f;
#pragma unroll
                for (int i = 0; i < TPR / 32; ++i) v[k] += b[i * K + k];
            }
        }
    }
};

// x <- the normalised row (entries past D stay 0); the mean (0 for rms) is
// subtracted before the squares are summed, so nothing cancels
template <int NV, bool VEC, int TPR, bool LAYER, typename Sum>
__device__ __forceinline__ void normalise(float (&x)[8 * NV], const NormArgs &a, int t, Sum &sum) {
    using R = Row<NV, VEC, TPR>;
    float s[1];
    if constexpr (LAYER) {
        s[0] = 0.f;
#pragma unroll
        for (int e = 0; e < R::kN; ++e) s[0] += x[e];
        sum(s);
        const float mean = s[0] / (float)a.D;
#pragma unroll
        for (int e = 0; e < R::kN; ++e) x[e] = R::col(t, e) < a.D ? x[e] - mean : 0.f;
    }
    s[0] = 0.f;
#pragma unroll
    for (int e = 0; e < R::kN; ++e) s[0] = fmaf(x[e], x[e], s[0]);
    sum(s);
    const float rstd = 1.f / sqrtf(s[0] / (float)a.D + a.eps);
#pragma unroll
    for (int e = 0; e < R::kN; ++e) x[e] *= rstd;
}

// One row per TPR threads; block = max(TPR, 32 * warps), grid-stride rows.
template <typename T, int NV, bool VEC, int TPR, bool LAYER>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) block_norm_kernel(NormArgs a) {
    using R = Row<NV, VEC, TPR>;
    constexpr int N = R::kN;
    __shared__ float buf[2][32 * 3];
    RowSum<1, TPR> sum{buf, 0};
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
    const int64_t groups = TPR == 32 ? (int64_t)gridDim.x * (blockDim.x >> 5) : gridDim.x;
    const int64_t first = TPR == 32 ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)
                                    : blockIdx.x;
    float wp[N], bp[N], wn[N], bn[N], gc[N];
    R::param(wp, a.w_post, 1.f, t, a.D);
    R::param(wn, a.w_pre, 1.f, t, a.D);
    if constexpr (LAYER) {
        R::param(bp, a.b_post, 0.f, t, a.D);
        R::param(bn, a.b_pre, 0.f, t, a.D);
    }
    R::param(gc, a.gate_mode == ULTRAMEM_GATE_CHANNEL ? static_cast<const float *>(a.gate) : nullptr,
             1.f, t, a.D);
    for (int64_t row = first; row < a.T; row += groups) {
        float z[N], u[N];
        R::load(z, static_cast<const T *>(a.y) + row * a.ld_y, t, a.D);
        R::load(u, static_cast<const T *>(a.r) + row * a.ld_r, t, a.D);
        float gt = a.out_scale;
        float g[N];
        if (a.gate_mode == ULTRAMEM_GATE_FULL)
            R::load(g, static_cast<const T *>(a.gate) + row * a.D, t, a.D);
        else if (a.gate_mode == ULTRAMEM_GATE_TOKEN)
            gt *= to_f(static_cast<const T *>(a.gate)[row]);
        if (a.post) {
            normalise<NV, VEC, TPR, LAYER>(z, a, t, sum);
#pragma unroll
            for (int e = 0; e < N; ++e) z[e] = LAYER ? fmaf(z[e], wp[e], bp[e]) : z[e] * wp[e];
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            z[e] *= a.gate_mode == ULTRAMEM_GATE_FULL ? g[e] : gc[e];
            u[e] = fmaf(gt, z[e], a.res_scale * u[e]);
        }
        R::store(static_cast<T *>(a.u) + row * a.D, u, t, a.D);
        if (a.pre) {
            // The second norm reads the stream as stored, so that the
            // gradient taken from the stored stream is that of this function.
#pragma unroll
            for (int e = 0; e < N; ++e) u[e] = to_f(from_f<T>(u[e]));
            normalise<NV, VEC, TPR, LAYER>(u, a, t, sum);
#pragma unroll
            for (int e = 0; e < N; ++e) u[e] = LAYER ? fmaf(u[e], wn[e], bn[e]) : u[e] * wn[e];
            R::store(static_cast<T *>(a.n) + row * a.D, u, t, a.D);
        }
    }
}

// ---- the gradient ------------------------------------------------------
// With û, ŷ the normalised rows and g = w (.) d for the gradient d of a
// norm's output, the gradient of its input is
//   rstd (g - mean(g) - û mean(g û))      (rms: without mean(g)),
// d û summed over the rows is the gain's gradient and d the bias's.  One
// pass over y, u, du and dn gives everything: the rows' statistics are taken
// again from the rows themselves.  The column sums stay in registers over a
// block's rows and leave as one partial row per block, which a second kernel
// adds in the blocks' order (no atomics: the result does not depend on the
// schedule).
enum { kColWPost, kColWPre, kColGate, kColBPost, kColBPre };   // order of the partial rows

template <typename T, int NV, bool VEC, int TPR, bool LAYER>
__global__ void __launch_bounds__(TPR) block_norm_backward_kernel(NormArgs a) {
    using R = Row<NV, VEC, TPR>;
    constexpr int N = R::kN;
    __shared__ float buf[2][32 * 3];
    RowSum<3, TPR> sum{buf, 0};
    const int t = threadIdx.x;
    float wp[N], bp[N], wn[N], gc[N];
    float c_wp[N], c_wn[N], c_g[N], c_bp[N], c_bn[N];
    R::param(wp, a.w_post, 1.f, t, a.D);
    R::param(wn, a.w_pre, 1.f, t, a.D);
    if constexpr (LAYER) R::param(bp, a.b_post, 0.f, t, a.D);
    const bool channel = a.gate_mode == ULTRAMEM_GATE_CHANNEL;
    R::param(gc, channel ? static_cast<const float *>(a.gate) : nullptr, 1.f, t, a.D);
#pragma unroll
    for (int e = 0; e < N; ++e) c_wp[e] = c_wn[e] = c_g[e] = c_bp[e] = c_bn[e] = 0.f;
    const float inv = 1.f / (float)a.D;

    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
        float y[N], u[N], gu[N], dn[N], g[N];
        R::load(y, static_cast<const T *>(a.y) + row * a.ld_y, t, a.D);
        if (a.pre) {
            R::load(u, static_cast<const T *>(a.r) + row * a.ld_r, t, a.D);
            R::load(dn, static_cast<const T *>(a.dn) + row * a.ld_dn, t, a.D);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) u[e] = dn[e] = 0.f;
        }
        if (a.du)
            R::load(gu, static_cast<const T *>(a.du) + row * a.ld_du, t, a.D);
        else
#pragma unroll
            for (int e = 0; e < N; ++e) gu[e] = 0.f;
        float gt = a.out_scale;
        if (a.gate_mode == ULTRAMEM_GATE_FULL)
            R::load(g, static_cast<const T *>(a.gate) + row * a.D, t, a.D);
        else if (a.gate_mode == ULTRAMEM_GATE_TOKEN)
            gt *= to_f(static_cast<const T *>(a.gate)[row]);

        // statistics of y and u, and the sums of the second norm's gradient
        float s[3], mean_g = 0.f;
        if constexpr (LAYER) {
            s[0] = s[1] = s[2] = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                s[0] += y[e];
                s[1] += u[e];
                s[2] = fmaf(wn[e], dn[e], s[2]);
            }
            sum(s);
            const float my = a.post ? s[0] * inv : 0.f, mu = s[1] * inv;
            mean_g = s[2] * inv;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const bool in = R::col(t, e) < a.D;
                y[e] = in ? y[e] - my : 0.f;
                u[e] = in ? u[e] - mu : 0.f;
            }
        }
        s[0] = s[1] = s[2] = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            s[0] = fmaf(y[e], y[e], s[0]);
            s[1] = fmaf(u[e], u[e], s[1]);
            s[2] = fmaf(wn[e] * dn[e], u[e], s[2]);
        }
        sum(s);
        const float ry = a.post ? 1.f / sqrtf(s[0] * inv + a.eps) : 1.f;
        const float ru = a.pre ? 1.f / sqrtf(s[1] * inv + a.eps) : 0.f;
        const float mean_gu = s[2] * ru * inv;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float uh = u[e] * ru;
            gu[e] = fmaf(ru, fmaf(wn[e], dn[e], -fmaf(uh, mean_gu, mean_g)), gu[e]);
            c_wn[e] = fmaf(dn[e], uh, c_wn[e]);
            if constexpr (LAYER) c_bn[e] += dn[e];
            y[e] *= ry;   // from here the normalised row
            u[e] = a.res_scale * gu[e];
        }
        if (a.dr) R::store(static_cast<T *>(a.dr) + row * a.D, u, t, a.D);

        // through the gate: d gate = out_scale z gu, d z = out_scale gate gu
        s[0] = s[1] = s[2] = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float z = LAYER ? fmaf(y[e], wp[e], bp[e]) : y[e] * wp[e];
            const float zg = (a.post ? z : y[e]) * gu[e];
            if (channel) c_g[e] = fmaf(a.out_scale, zg, c_g[e]);
            s[2] += zg;
            u[e] = a.out_scale * zg;
            gu[e] *= gt * (a.gate_mode == ULTRAMEM_GATE_FULL ? g[e] : gc[e]);
            if (a.post) {
                c_wp[e] = fmaf(gu[e], y[e], c_wp[e]);
                if constexpr (LAYER) c_bp[e] += R::col(t, e) < a.D ? gu[e] : 0.f;
                gu[e] *= wp[e];
                if constexpr (LAYER) s[0] += R::col(t, e) < a.D ? gu[e] : 0.f;
                s[1] = fmaf(gu[e], y[e], s[1]);
            }
        }
        if (a.gate_mode == ULTRAMEM_GATE_FULL && a.dgate_rows)
            R::store(static_cast<T *>(a.dgate_rows) + row * a.D, u, t, a.D);
        sum(s);
        if (a.gate_mode == ULTRAMEM_GATE_TOKEN && a.dgate_rows && t == 0)
            static_cast<T *>(a.dgate_rows)[row] = from_f<T>(a.out_scale * s[2]);
        if (a.post) {
            const float m0 = s[0] * inv, m1 = s[1] * inv;
#pragma unroll
            for (int e = 0; e < N; ++e) gu[e] = ry * (gu[e] - fmaf(y[e], m1, m0));
        }
        if (a.dy) R::store(static_cast<T *>(a.dy) + row * a.D, gu, t, a.D);
    }

    const int n_cols = LAYER ? 5 : 3;
    float *part = a.part + (int64_t)blockIdx.x * n_cols * a.D;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const int c = R::col(t, e);
        if (c >= a.D) continue;
        part[kColWPost * a.D + c] = c_wp[e];
        part[kColWPre * a.D + c] = c_wn[e];
        part[kColGate * a.D + c] = c_g[e];
        if constexpr (LAYER) {
            part[kColBPost * a.D + c] = c_bp[e];
            part[kColBPre * a.D + c] = c_bn[e];
        }
    }
}

struct ColOut {
    float *out[5];
};

// out[k][c] = sum over the blocks of part[b][k][c]: 32 columns a block, 8
// warps over the partial rows.
__global__ void __launch_bounds__(256) column_sum_kernel(const float *part, int blocks, int n_cols,
                                                         int D, ColOut o) {
    __shared__ float s[8][33];
    const int k = blockIdx.y;
    if (!o.out[k]) return;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float v = 0.f;
    if (c < D)
        for (int b = w; b < blocks; b += 8) v += part[((int64_t)b * n_cols + k) * D + c];
    s[w][lane] = v;
    __syncthreads();
    if (w == 0 && c < D) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += s[i][lane];
        o.out[k][c] = v;
    }
}

// ---- launches ----------------------------------------------------------

constexpr int kMaxDim = 8192;

template <typename T, bool VEC, bool LAYER> struct Forward {
    template <int NV, int TPR> static cudaError_t go(const NormArgs &a, cudaStream_t st) {
        // up to 2048 threads an SM; few rows spread over the SMs first
        const int sms = device_sm_count();
        int rows = TPR == 32 ? 4 : 1;
        if (TPR == 32 && a.T < 4 * (int64_t)sms) rows = 1;
        const int threads = rows * TPR;
        const int64_t want = (a.T + rows - 1) / rows, most = (int64_t)sms * (2048 / (TPR < 128 ? 128 : TPR));
        const unsigned grid = (unsigned)(want < most ? want : most);
        block_norm_kernel<T, NV, VEC, TPR, LAYER><<<grid, threads, 0, st>>>(a);
        return cudaGetLastError();
    }
    static cudaError_t launch(const NormArgs &a, cudaStream_t st) {
        const int v = (a.D + 7) / 8;
        if (v <= 32) return go<1, 32>(a, st);
        if (v <= 64) return go<2, 32>(a, st);
        if (v <= 128) return go<1, 128>(a, st);
        if (v <= 256) return go<1, 256>(a, st);
        if (v <= 512) return go<1, 512>(a, st);
        return go<1, 1024>(a, st);
    }
};

int backward_tpr(int D) {
    const int v = (D + 7) / 8;
    int t = 32;
    while (t < v && t < 1024) t *= 2;
    return t;
}

// Blocks of the gradient's first kernel: as many as fit at about 96
// registers a thread, and no more than 8 an SM (each leaves a partial row).
int backward_blocks(int64_t T, int D) {
    const int tpr = backward_tpr(D);
    int per_sm = 640 / tpr;
    per_sm = per_sm < 1 ? 1 : per_sm > 8 ? 8 : per_sm;
    const int64_t most = (int64_t)device_sm_count() * per_sm;
    return (int)(T < most ? T : most);
}

template <typename T, bool VEC, bool LAYER> struct Backward {
    template <int NV, int TPR> static cudaError_t go(const NormArgs &a, cudaStream_t st) {
        block_norm_backward_kernel<T, NV, VEC, TPR, LAYER>
            <<<backward_blocks(a.T, a.D), TPR, 0, st>>>(a);
        return cudaGetLastError();
    }
    static cudaError_t launch(const NormArgs &a, cudaStream_t st) {
        switch (backward_tpr(a.D)) {
        case 32: return go<1, 32>(a, st);
        case 64: return go<1, 64>(a, st);
        case 128: return go<1, 128>(a, st);
        case 256: return go<1, 256>(a, st);
        case 512: return go<1, 512>(a, st);
        default: return go<1, 1024>(a, st);
        }
    }
};

template <template <typename, bool, bool> class Op>
cudaError_t dispatch(const NormArgs &a, int dtype, bool layer, bool vec, cudaStream_t st) {
    if (dtype == ULTRAMEM_BF16) {
        if (vec)
            return layer ? Op<__nv_bfloat16, true, true>::launch(a, st)
                         : Op<__nv_bfloat16, true, false>::launch(a, st);
        return layer ? Op<__nv_bfloat16, false, true>::launch(a, st)
                     : Op<__nv_bfloat16, false, false>::launch(a, st);
    }
    if (vec)
        return layer ? Op<float, true, true>::launch(a, st) : Op<float, true, false>::launch(a, st);
    return layer ? Op<float, false, true>::launch(a, st) : Op<float, false, false>::launch(a, st);
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

// rows of whole 16-byte words that start on 16-byte boundaries
bool rows_aligned(int dtype, int D, std::initializer_list<const void *> ptrs,
                  std::initializer_list<int64_t> lds) {
    const int per = dtype == ULTRAMEM_BF16 ? 8 : 4;
    if (D % per) return false;
    for (const void *p : ptrs)
        if (!aligned16(p)) return false;
    for (int64_t ld : lds)
        if (ld % per) return false;
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
    um::NormArgs a = um::args_of(p);
    a.r = r;
    a.u = u;
    a.n = n;
    const void *gate_rows = p->gate_mode == ULTRAMEM_GATE_FULL ? p->gate : nullptr;
    const bool vec = um::rows_aligned(p->dtype, p->dim, {p->y, r, u, n, gate_rows},
                                      {p->ld_y, p->ld_r});
    cudaGetLastError();
    return um::status_from_cuda(um::dispatch<um::Forward>(
        a, p->dtype, p->kind == ULTRAMEM_NORM_LAYER, vec, (cudaStream_t)stream));
}

extern "C" int64_t ultramem_block_norm_backward_workspace(int64_t n_tokens, int32_t dim) {
    if (n_tokens < 0 || dim < 1 || dim > um::kMaxDim) return 0;
    return (int64_t)um::backward_blocks(n_tokens, dim) * 5 * dim * (int64_t)sizeof(float);
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
    um::ColOut cols = {{dw_post, dw_pre, channel_gate, db_post, db_pre}};
    cudaGetLastError();
    if (p->n_tokens == 0) {   // empty sums
        for (float *o : cols.out)
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
    const bool vec = um::rows_aligned(
        p->dtype, D,
        {p->y, p->pre ? u : nullptr, du, dn, dy, dr, full ? p->gate : nullptr, full ? dgate : nullptr},
        {p->ld_y, p->pre ? p->ld_r : 0, du ? ld_du : 0, dn ? ld_dn : 0});
    const bool layer = p->kind == ULTRAMEM_NORM_LAYER;
    cudaError_t e = um::dispatch<um::Backward>(a, p->dtype, layer, vec, st);
    if (e != cudaSuccess) return um::status_from_cuda(e);
    bool any = false;
    for (float *o : cols.out) any = any || o;
    if (any) {
        const int n_cols = layer ? 5 : 3;
        um::column_sum_kernel<<<dim3((D + 31) / 32, n_cols), 256, 0, st>>>(
            a.part, um::backward_blocks(p->n_tokens, D), n_cols, D, cols);
        e = cudaGetLastError();
    }
    return um::status_from_cuda(e);
}

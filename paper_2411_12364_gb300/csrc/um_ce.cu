// um_ce.cu -- the softmax cross entropy of hidden states against a vocabulary's
// output weights, without the logits in memory, and its gradient.
//
// Forward: a block makes a 64 x 64 tile of logits and leaves, for each of its
// tokens, the maximum and the sum of e^(z - maximum) over the tile's columns
// (and the label's logit, in the tile that has it); a second kernel joins the
// tiles' pairs.  Gradient: the logits again, in pieces of the vocabulary; a
// piece's G = scale dloss (e^(z - lse) - onehot) goes to the workspace, and
// two products read it: dx += G W, dw = G^T x.
#include "um_device.cuh"
#include "um_internal.cuh"
#include "um_overlap.cuh"

namespace um {
namespace ce {
namespace {

constexpr int kMaxVocab = 1 << 30;
constexpr int kMaxDim = 65536;
constexpr int kTile = 64, kStep = 16;
constexpr int64_t kPieceBytes = 512ll << 20;

struct Args {
    const void *x, *w, *labels;
    int64_t ld_x, ld_w;
    int T, V, D, wide;
    float scale;
    const float *lse_in, *dloss;
    float *loss, *lse, *target;
    float2 *part;             // [tiles][T]
    float *g;                 // [T][piece]
    float *dx_sum;            // [T][D]
    void *dx, *dw;
    int v0, vn, piece;        // the piece at hand
};

__device__ __forceinline__ int label_of(const Args &a, int64_t t) {
    const int64_t l = a.wide ? static_cast<const int64_t *>(a.labels)[t]
                             : (int64_t) static_cast<const int32_t *>(a.labels)[t];
    return l >= 0 && l < a.V ? (int)l : -1;
}

// C[i][j] = sum_k A(i, k) B(j, k) of a 64 x 64 tile, 4 x 4 a thread: row
// ty * 4 + r, column tx * 4 + c.
template <typename FA, typename FB>
__device__ __forceinline__ void tile_product(int m, int n, int k, FA a, FB b, float (&c)[4][4]) {
    __shared__ float sa[kStep][kTile + 4], sb[kStep][kTile + 4];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[i][j] = 0.f;
    for (int k0 = 0; k0 < k; k0 += kStep) {
        for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
            const int r = i / kStep, kk = i % kStep;
            sa[kk][r] = r < m && k0 + kk < k ? a(r, k0 + kk) : 0.f;
            sb[kk][r] = r < n && k0 + kk < k ? b(r, k0 + kk) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kStep; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    c[i][j] = fmaf(sa[kk][ty * 4 + i], sb[kk][tx * 4 + j], c[i][j]);
        __syncthreads();
    }
}

template <typename T> __device__ __forceinline__ void logits(const Args &a, int t0, int v0, int vn,
                                                             float (&z)[4][4]) {
    const T *x = static_cast<const T *>(a.x) + (int64_t)t0 * a.ld_x;
    const T *w = static_cast<const T *>(a.w) + (int64_t)v0 * a.ld_w;
    tile_product(min(kTile, a.T - t0), vn, a.D, [&](int i, int k) { return to_f(x[i * a.ld_x + k]); },
                 [&](int j, int k) { return to_f(w[j * a.ld_w + k]); }, z);
}

template <typename T> __global__ void __launch_bounds__(256) lse_kernel(Args a) {
    const int t0 = blockIdx.y * kTile, v0 = blockIdx.x * kTile, vn = min(kTile, a.V - v0);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float z[4][4];
    logits<T>(a, t0, v0, vn, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t t = t0 + ty * 4 + i;
        const int label = t < a.T ? label_of(a, t) : -1;
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            z[i][j] *= a.scale;
            if (tx * 4 + j < vn) {
                m = fmaxf(m, z[i][j]);
                if (label == v0 + tx * 4 + j) a.target[t] = z[i][j];
            }
        }
#pragma unroll
        for (int o = 8; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (m > -INFINITY)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (tx * 4 + j < vn) l += expf(z[i][j] - m);
#pragma unroll
        for (int o = 8; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (tx == 0 && t < a.T) a.part[(int64_t)blockIdx.x * a.T + t] = make_float2(m, l);
    }
}

__global__ void __launch_bounds__(256) join_kernel(Args a, int tiles) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= a.T) return;
    float m = -INFINITY, l = 0.f;
    for (int i = 0; i < tiles; ++i) {
        const float2 p = a.part[(int64_t)i * a.T + t];
        const float top = fmaxf(m, p.x);
        if (top == -INFINITY) continue;
        l = l * expf(m - top) + p.y * expf(p.x - top);
        m = top;
    }
    const float lse = m + logf(l);
    a.lse[t] = lse;
    a.loss[t] = label_of(a, t) >= 0 ? lse - a.target[t] : 0.f;
}

template <typename T> __global__ void __launch_bounds__(256) g_kernel(Args a) {
    const int t0 = blockIdx.y * kTile, c0 = blockIdx.x * kTile, vn = min(kTile, a.vn - c0);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float z[4][4];
    logits<T>(a, t0, a.v0 + c0, vn, z);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t t = t0 + ty * 4 + i;
        if (t >= a.T) continue;
        const int label = label_of(a, t);
        const float d = label >= 0 ? a.dloss[t] * a.scale : 0.f, lse = a.lse_in[t];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = c0 + tx * 4 + j;
            if (c >= a.vn) continue;
            const float p = expf(z[i][j] * a.scale - lse) - (label == a.v0 + c ? 1.f : 0.f);
            const float g = label >= 0 ? to_f(from_f<T>(p * d)) : 0.f;
            a.g[t * a.piece + c] = g;
        }
    }
}

template <typename T> __global__ void __launch_bounds__(256) dx_kernel(Args a) {
    const int t0 = blockIdx.y * kTile, c0 = blockIdx.x * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const T *w = static_cast<const T *>(a.w) + (int64_t)a.v0 * a.ld_w + c0;
    const float *g = a.g + (int64_t)t0 * a.piece;
    float c[4][4];
    tile_product(min(kTile, a.T - t0), min(kTile, a.D - c0), a.vn,
                 [&](int i, int k) { return g[(int64_t)i * a.piece + k]; },
                 [&](int j, int k) { return to_f(w[k * a.ld_w + j]); }, c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t t = t0 + ty * 4 + i;
            const int col = c0 + tx * 4 + j;
            if (t >= a.T || col >= a.D) continue;
            const float v = c[i][j] + (a.v0 ? a.dx_sum[t * a.D + col] : 0.f);
            if (a.v0 + a.vn == a.V)
                static_cast<T *>(a.dx)[t * a.D + col] = from_f<T>(v);
            else
                a.dx_sum[t * a.D + col] = v;
        }
}

template <typename T> __global__ void __launch_bounds__(256) dw_kernel(Args a) {
    const int r0 = blockIdx.y * kTile, c0 = blockIdx.x * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const T *x = static_cast<const T *>(a.x) + c0;
    const float *g = a.g + r0;
    float c[4][4];
    tile_product(min(kTile, a.vn - r0), min(kTile, a.D - c0), a.T,
                 [&](int i, int k) { return g[(int64_t)k * a.piece + i]; },
                 [&](int j, int k) {   // a token that does not count: whatever x holds
                     return label_of(a, k) >= 0 ? to_f(x[k * a.ld_x + j]) : 0.f;
                 }, c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t v = (int64_t)a.v0 + r0 + ty * 4 + i;
            const int col = c0 + tx * 4 + j;
            if (r0 + ty * 4 + i < a.vn && col < a.D)
                static_cast<T *>(a.dw)[v * a.D + col] = from_f<T>(c[i][j]);
        }
}

// ---- the calls' plans --------------------------------------------------------

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

bool sizes_ok(int32_t dtype, int32_t T, int32_t V, int32_t D) {
    return (dtype == ULTRAMEM_F32 || dtype == ULTRAMEM_BF16) && T >= 0 && V >= 1 &&
           V <= kMaxVocab && D >= 1 && D <= kMaxDim;
}

int piece_of(int32_t T, int32_t V) {
    int64_t n = kPieceBytes / 4 / (T > 0 ? T : 1) / kTile * kTile;
    if (n < kTile) n = kTile;
    return (int)(n < V ? n : V);
}

bool args_ok(const ultramem_cross_entropy_args *p) {
    return p && sizes_ok(p->dtype, p->n_tokens, p->vocab, p->dim) &&
           (p->labels_bytes == 4 || p->labels_bytes == 8) && isfinite(p->logit_scale);
}
bool inputs_ok(const ultramem_cross_entropy_args *p) {
    const int es = p->dtype == ULTRAMEM_BF16 ? 2 : 4;
    return p->x && p->w && p->labels && p->ld_x >= p->dim && p->ld_w >= p->dim &&
           ((uintptr_t)p->x | (uintptr_t)p->w) % es == 0 &&
           (uintptr_t)p->labels % p->labels_bytes == 0;
}
Memory rows_of(const ultramem_cross_entropy_args *p, const void *at, int64_t n, int64_t ld) {
    const int64_t es = p->dtype == ULTRAMEM_BF16 ? 2 : 4;
    return {at, p->dim * es, n, ld * es};
}
Args args_of(const ultramem_cross_entropy_args *p) {
    Args a = {};
    a.x = p->x;
    a.w = p->w;
    a.labels = p->labels;
    a.ld_x = p->ld_x;
    a.ld_w = p->ld_w;
    a.T = p->n_tokens;
    a.V = p->vocab;
    a.D = p->dim;
    a.wide = p->labels_bytes == 8;
    a.scale = p->logit_scale;
    return a;
}

}  // namespace
}  // namespace ce
}  // namespace um

using namespace um::ce;

extern "C" int64_t ultramem_cross_entropy_workspace(int32_t dtype, int32_t n_tokens,
                                                    int32_t vocab, int32_t dim) {
    if (!sizes_ok(dtype, n_tokens, vocab, dim)) return 0;
    return (int64_t)n_tokens * (8ll * ceil_div(vocab, kTile) + 4);
}

extern "C" ultramem_status ultramem_cross_entropy(const ultramem_cross_entropy_args *p,
                                                  float *loss, float *lse, void *workspace,
                                                  int64_t workspace_bytes, void *stream) {
    if (!args_ok(p)) return ULTRAMEM_EINVAL;
    if (p->n_tokens == 0) return ULTRAMEM_OK;
    const int64_t need = ultramem_cross_entropy_workspace(p->dtype, p->n_tokens, p->vocab, p->dim);
    if (!inputs_ok(p) || !loss || !lse || ((uintptr_t)loss | (uintptr_t)lse) % 4 || !workspace ||
        ((uintptr_t)workspace & 15) || workspace_bytes < need)
        return ULTRAMEM_EINVAL;
    const int64_t T = p->n_tokens;
    if (!um::apart({{loss, T * 4}, {lse, T * 4}, {workspace, need}},
                   {rows_of(p, p->x, T, p->ld_x), rows_of(p, p->w, p->vocab, p->ld_w),
                    {p->labels, T * p->labels_bytes}}))
        return ULTRAMEM_EINVAL;
    Args a = args_of(p);
    a.loss = loss;
    a.lse = lse;
    const int tiles = ceil_div(a.V, kTile);
    a.part = static_cast<float2 *>(workspace);
    a.target = reinterpret_cast<float *>(a.part + T * tiles);
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    const dim3 grid(tiles, ceil_div(T, kTile));
    if (p->dtype == ULTRAMEM_BF16)
        lse_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(a);
    else
        lse_kernel<float><<<grid, 256, 0, st>>>(a);
    join_kernel<<<ceil_div(T, 256), 256, 0, st>>>(a, tiles);
    return um::status_from_cuda(cudaGetLastError());
}

extern "C" int64_t ultramem_cross_entropy_backward_workspace(int32_t dtype, int32_t n_tokens,
                                                             int32_t vocab, int32_t dim) {
    if (!sizes_ok(dtype, n_tokens, vocab, dim)) return 0;
    return 4ll * n_tokens * ((int64_t)piece_of(n_tokens, vocab) + dim);
}

extern "C" ultramem_status ultramem_cross_entropy_backward(const ultramem_cross_entropy_args *p,
                                                           const float *lse, const float *dloss,
                                                           void *dx, void *dw, void *workspace,
                                                           int64_t workspace_bytes, void *stream) {
    if (!args_ok(p)) return ULTRAMEM_EINVAL;
    const int es = p->dtype == ULTRAMEM_BF16 ? 2 : 4;
    if (((uintptr_t)dx | (uintptr_t)dw) % es) return ULTRAMEM_EINVAL;
    const int64_t dw_bytes = (int64_t)p->vocab * p->dim * es;
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    if (p->n_tokens == 0)
        return dw ? um::status_from_cuda(cudaMemsetAsync(dw, 0, dw_bytes, st)) : ULTRAMEM_OK;
    if (!dx && !dw) return ULTRAMEM_OK;
    const int64_t need =
        ultramem_cross_entropy_backward_workspace(p->dtype, p->n_tokens, p->vocab, p->dim);
    if (!inputs_ok(p) || !lse || !dloss || ((uintptr_t)lse | (uintptr_t)dloss) % 4 || !workspace ||
        ((uintptr_t)workspace & 15) || workspace_bytes < need)
        return ULTRAMEM_EINVAL;
    const int64_t T = p->n_tokens;
    if (!um::apart({{dx, T * p->dim * es}, {dw, dw_bytes}, {workspace, need}},
                   {rows_of(p, p->x, T, p->ld_x), rows_of(p, p->w, p->vocab, p->ld_w),
                    {p->labels, T * p->labels_bytes}, {lse, T * 4}, {dloss, T * 4}}))
        return ULTRAMEM_EINVAL;
    Args a = args_of(p);
    a.lse_in = lse;
    a.dloss = dloss;
    a.dx = dx;
    a.dw = dw;
    a.piece = piece_of(a.T, a.V);
    a.g = static_cast<float *>(workspace);
    a.dx_sum = a.g + T * a.piece;
    for (a.v0 = 0; a.v0 < a.V; a.v0 += a.piece) {
        a.vn = a.V - a.v0 < a.piece ? a.V - a.v0 : a.piece;
        const dim3 g_grid(ceil_div(a.vn, kTile), ceil_div(T, kTile));
        const dim3 dx_grid(ceil_div(a.D, kTile), ceil_div(T, kTile));
        const dim3 dw_grid(ceil_div(a.D, kTile), ceil_div(a.vn, kTile));
        auto go = [&](auto t) {
            using E = decltype(t);
            g_kernel<E><<<g_grid, 256, 0, st>>>(a);
            if (dx) dx_kernel<E><<<dx_grid, 256, 0, st>>>(a);
            if (dw) dw_kernel<E><<<dw_grid, 256, 0, st>>>(a);
        };
        p->dtype == ULTRAMEM_BF16 ? go(__nv_bfloat16()) : go(float());
    }
    return um::status_from_cuda(cudaGetLastError());
}

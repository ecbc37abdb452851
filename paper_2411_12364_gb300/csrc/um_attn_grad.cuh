// um_attn_grad.cuh -- the gradient of the attention of whole sequences: the
// call's arguments and the list of tiles, shared by its kernels.
#pragma once

#include <cuda.h>

#include "um_internal.cuh"
#include "um_tc.cuh"

namespace um {
namespace attn_grad {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxHeadDim = 256;

struct Args {
    const void *q, *k, *v, *out, *dout;
    void *dq, *dk, *dv;
    const float *lse;
    const int32_t *q_start;
    int64_t q_stride, k_stride, v_stride, out_stride, dout_stride, dq_stride, dk_stride, dv_stride;
    float2 *rows;             // [q_heads][T]: (lse, +inf where it is -inf; d_i)
    int4 *blocks;             // [2][most]: tok0, n, b of each block of `block` rows, by the
                              // rows behind it, and by the keys before it, longest first
    int *count;               // of them
    int *err;
    int n_seqs, T, q_heads, kv_heads, group, D;
    int block;                // rows of a block
    int most;                 // blocks that a list holds
    int ranks;                // CTAs that share out a block of keys
    int wide;                 // inputs whose rows allow loads of 4 entries
    float scale, scale_log2;
};

// Clusters of `ranks` CTAs: one for each block of held keys, and one for as many
// blocks of held rows as it has CTAs.
inline dim3 grid_of(const Args &a) {
    const unsigned ranks = (unsigned)a.ranks, most = (unsigned)a.most;
    return dim3(most * a.kv_heads + (most * a.q_heads + ranks - 1) / ranks, 1, ranks);
}

// 4 floats of shared memory at the same place of another CTA of the cluster
__device__ __forceinline__ float4 load_peer(const float *p, uint32_t rank) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(tc::mapa_shared(tc::smem_u32(p), rank))
                 : "memory");
    return v;
}

// bf16, heads up to 128 wide (um_attn_grad_tc.cu): maps of boxes of 64 columns x
// a head x 128 tokens over the inputs as [tokens][heads][width].
constexpr int kTensorBlock = 128;
cudaError_t launch_tensor(const Args &a, const CUtensorMap &q, const CUtensorMap &k,
                          const CUtensorMap &v, const CUtensorMap &dout, cudaStream_t st);

}  // namespace attn_grad
}  // namespace um

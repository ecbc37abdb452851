// um_attn_grad.cuh -- the gradient of the attention of whole sequences: the
// call's arguments and the list of tiles, shared by its kernels.
#pragma once

#include <cuda.h>

#include "um_internal.cuh"

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
    int ranks;                // CTAs to a block (CUDA cores)
    int wide;                 // inputs whose rows allow loads of 4 entries
    float scale, scale_log2;
};

// bf16, heads up to 128 wide (um_attn_grad_tc.cu): maps of boxes of 64 columns x
// a head x 128 tokens over the inputs as [tokens][heads][width].
constexpr int kTensorBlock = 128;
cudaError_t launch_tensor(const Args &a, const CUtensorMap &q, const CUtensorMap &k,
                          const CUtensorMap &v, const CUtensorMap &dout, cudaStream_t st);

}  // namespace attn_grad
}  // namespace um

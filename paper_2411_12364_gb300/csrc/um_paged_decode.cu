// um_paged_decode.cu -- attention over the paged cache for few rows a request
// (bf16, heads up to 128 wide, at most 16 rows of new tokens x query heads a
// key/value head): single-token decode and short drafts.
//
// Every key and value is read once for at most 16 rows, 4 to 64 flops a byte,
// so the bound is memory; the work is to keep enough bytes in flight and to
// give every SM an equal share of keys whatever the requests' lengths are
// (place_share).  One producer warp streams blocks of 64 keys and values by
// TMA, a box per page, into a ring of 3 stages (96 KB; two CTAs an SM keep
// 192 KB in flight).  Four warps take 16 keys of each block each: both
// products run on mma.sync m16n8k16 with the 16 rows as M (a tcgen05 tile
// would be 128 rows for the same bytes), the running maximum and sum stay in
// registers, and the warps never wait for one another inside a tile; their
// partial outputs are joined at its end.
//
// Measured: 64 requests of up to 8192 keys (16 / 4 heads x 128, pages of 16)
// 84 us without the join of split tiles, 6.3 TB/s; one request of 131072 keys
// 46 us, 5.8 TB/s.
#include "um_device.cuh"
#include "um_paged.cuh"
#include "um_tc.cuh"

namespace um {
namespace paged {
namespace {

constexpr int kRows = 16;
constexpr int kKeys = 64;                 // keys of a block
constexpr int kWarps = 4;                 // consumer warps, 16 keys each
constexpr int kThreads = 32 * (kWarps + 1);
constexpr uint32_t kHalfBytes = kKeys * 128;   // 64 keys x 64 columns of bf16

template <int DP> struct Cfg {
    static constexpr int kHalves = DP / 64;
    static constexpr uint32_t kTile = kHalfBytes * kHalves;   // K or V of a block
    static constexpr int kStages = DP == 128 ? 3 : 6;
    // stages, the warps' join buffer (2 warps x 16 rows x 64 columns), alignment
    static constexpr size_t kSmem = (size_t)2 * kTile * kStages + 2 * kRows * 64 * 4 + 1024;
};

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}
// 16-byte word `chunk` of row `key` of a 64-column half written by TMA with
// the 128-byte swizzle (the half starts on a 1024-byte boundary)
__device__ __forceinline__ uint32_t swizzled(uint32_t half, int key, int chunk) {
    return half + key * 128 + ((chunk ^ (key & 7)) << 4);
}
__device__ __forceinline__ void consumers_sync() {
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
}
// the same, and whether every consumer warp still goes on
__device__ __forceinline__ bool consumers_all(bool ok) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.and.pred q, 1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)ok), "n"(32 * kWarps)
        : "memory");
    return r != 0;
}

template <int DP>
__global__ void __launch_bounds__(kThreads, 2)
    decode_kernel(const __grid_constant__ CUtensorMap map_k,
                  const __grid_constant__ CUtensorMap map_v, AttnArgs a, int box_rows) {
    using C = Cfg<DP>;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[C::kStages], empty[C::kStages];
    __shared__ int64_t scratch[kThreads / 32 + 1];
    __shared__ Cursor cur;
    __shared__ float2 stat[kWarps][kRows];
    uint8_t *ring = raw + ((1024 - (tc::smem_u32(raw) & 1023)) & 1023);
    float *join = reinterpret_cast<float *>(ring + (size_t)2 * C::kTile * C::kStages);
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            tc::mbar_init(&full[s], 1);
            tc::mbar_init(&empty[s], kWarps);
        }
        tc::fence_mbar_init();
    }
    pdl_wait();
    place_share<kThreads>(a, blockIdx.x, gridDim.x, kKeys, 2 * kKeys, scratch, &cur);
    pdl_trigger();
    int4 *desc = a.part_desc + 2 * blockIdx.x;
    Walk wk;
    wk.begin(a, cur);
    int stage = 0;
    uint32_t phase = 0;

    if (w == kWarps) {
        // ---- producer: the whole warp, a lane per page of the block ----
        if (lane == 0) {
            tc::prefetch_tensormap(&map_k);
            tc::prefetch_tensormap(&map_v);
        }
        const int pages = kKeys / box_rows;                 // boxes of a block
        const int page_mask = (1 << a.page_shift) - 1;
        bool ok = true;
        int issued = 0;
        while (ok && wk.next(a, kKeys)) {
            // the table's entry for a block is read a block ahead
            int page = lane < pages ? page_of(a, wk.c.r, wk.j0 * kKeys + lane * box_rows, wk.kv)
                                    : -1;
            for (int j = wk.j0; ok && j < wk.j1; ++j) {
                const int key = j * kKeys + lane * box_rows;
                // outside the cache: reads zeros
                const int z = page < 0 ? a.n_pages * a.kv_heads : page * a.kv_heads + wk.h;
                page = lane < pages ? page_of(a, wk.c.r, key + kKeys, wk.kv) : -1;
                if (!__all_sync(0xffffffffu, tc::mbar_wait(&empty[stage], phase ^ 1))) {
                    ok = false;
                    break;
                }
                if (lane == 0) tc::mbar_arrive_expect_tx(&full[stage], 2 * C::kTile);
                __syncwarp();
                if (lane < pages) {
                    uint8_t *dst = ring + (size_t)stage * 2 * C::kTile + lane * box_rows * 128;
#pragma unroll
                    for (int i = 0; i < C::kHalves; ++i) {
                        tc::tma_load_3d(dst + i * kHalfBytes, &map_k, &full[stage], 64 * i,
                                        key & page_mask, z);
                        tc::tma_load_3d(dst + C::kTile + i * kHalfBytes, &map_v, &full[stage],
                                        64 * i, key & page_mask, z);
                    }
                }
                ++issued;
                if (++stage == C::kStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }
        }
        if (!ok) {   // leave nothing in flight: wait for the copies issued last
            if (lane == 0) atomicOr(a.err, kErrTimeout);
            for (int i = 0; i < C::kStages && i < issued; ++i) {
                if (--stage < 0) {
                    stage = C::kStages - 1;
                    phase ^= 1;
                }
                tc::mbar_wait(&full[stage], phase);
            }
        }
        return;
    }

    // ---- consumers ----
    if (tid == 0) desc[0] = desc[1] = make_int4(kPartNone, 0, 0, 0);
    const int r0 = lane >> 2, kk = (lane & 3) * 2;          // rows r0, r0 + 8; key pair kk
    bool ok = true;
    while (ok && wk.next(a, kKeys)) {
        const int n_rows = wk.n_tok * a.group;
        // the rows' queries as A fragments (zeros past the tile's rows and width)
        uint32_t qf[DP / 16][4];
        int limit[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = r0 + 8 * i, tok = row / a.group;
            limit[i] = row < n_rows ? min(wk.kv, wk.pos0 + tok + 1) : 0;
            const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(a.q) +
                                     (int64_t)(wk.tok0 + tok) * a.q_stride +
                                     (int64_t)(wk.h * a.group + row - tok * a.group) * a.D;
#pragma unroll
            for (int s = 0; s < DP / 16; ++s)
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const int c = 16 * s + 8 * g + kk;
                    qf[s][i + 2 * g] = row < n_rows && c < a.D
                                           ? *reinterpret_cast<const uint32_t *>(q + c) : 0u;
                }
        }
        float o[DP / 8][4];
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

        for (int j = wk.j0; j < wk.j1; ++j) {
            if (!__all_sync(0xffffffffu, tc::mbar_wait(&full[stage], phase))) {
                ok = false;
                break;
            }
            const uint32_t ks = tc::smem_u32(ring + (size_t)stage * 2 * C::kTile);
            const uint32_t vs = ks + C::kTile;
            float s[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[t][i] = 0.f;
            {   // scores of the warp's 16 keys: matrices (keys 0-7 | 8-15) x (8 columns | next 8)
                const int key = 16 * w + (lane >> 4) * 8 + (lane & 7), sub = (lane >> 3) & 1;
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) {
                    uint32_t b[4];
                    ldsm4(b, swizzled(ks + (c >> 2) * kHalfBytes, key, (c & 3) * 2 + sub));
                    mma16816(s[0], qf[c], b[0], b[1]);
                    mma16816(s[1], qf[c], b[2], b[3]);
                }
            }
            const int key0 = j * kKeys + 16 * w + kk;       // + 8 t + (i & 1)
            float mx[2] = {m[0], m[1]};
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[t][i] = key0 + 8 * t + (i & 1) < limit[i >> 1] ? s[t][i] * a.scale_log2
                                                                     : -INFINITY;
                    mx[i >> 1] = fmaxf(mx[i >> 1], s[t][i]);
                }
            float f[2], base[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
                base[i] = mx[i] == -INFINITY ? 0.f : mx[i];
                f[i] = exp2f(m[i] - base[i]);
                m[i] = mx[i];
                l[i] *= f[i];
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[t][i] = exp2f(s[t][i] - base[i >> 1]);
                    l[i >> 1] += s[t][i];
                }
            if (!__all_sync(0xffffffffu, f[0] == 1.f && f[1] == 1.f)) {
#pragma unroll
                for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[n][i] *= f[i >> 1];
            }
            // weights as the A operand: one rounding to bf16, as large as that
            // of the values themselves; the sum l keeps fp32
            const uint32_t p[4] = {pack_bf16(s[0][0], s[0][1]), pack_bf16(s[0][2], s[0][3]),
                                   pack_bf16(s[1][0], s[1][1]), pack_bf16(s[1][2], s[1][3])};
            // a block's places past the request's length may hold anything:
            // weight 0 times that could be NaN, so they are cleared
            uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;
            const bool tail = (j + 1) * kKeys > wk.kv;
            if (tail) {
                const int left = wk.kv - key0;
                keep0 = left <= 0 ? 0u : left == 1 ? 0xffffu : 0xffffffffu;
                keep1 = left <= 8 ? 0u : left == 9 ? 0xffffu : 0xffffffffu;
            }
            {
                const int key = 16 * w + ((lane >> 3) & 1) * 8 + (lane & 7), sub = lane >> 4;
#pragma unroll
                for (int n = 0; n < DP / 16; ++n) {
                    uint32_t b[4];
                    ldsm4_t(b, swizzled(vs + (n >> 2) * kHalfBytes, key, (n & 3) * 2 + sub));
                    if (tail) {
                        b[0] &= keep0;
                        b[1] &= keep1;
                        b[2] &= keep0;
                        b[3] &= keep1;
                    }
                    mma16816(o[2 * n], p, b[0], b[1]);
                    mma16816(o[2 * n + 1], p, b[2], b[3]);
                }
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&empty[stage]);
            if (++stage == C::kStages) {
                stage = 0;
                phase ^= 1;
            }
        }

        // ---- join the warps: their maxima and sums, then the outputs added
        // two by two through shared memory, 64 columns at a time ----
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
            if ((lane & 3) == 0) stat[w][r0 + 8 * i] = make_float2(m[i], l[i]);
        }
        if (!ok && lane == 0) atomicOr(a.err, kErrTimeout);
        ok = consumers_all(ok);
        if (!ok) break;
        float top[2], sum[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            top[i] = -INFINITY;
            sum[i] = 0.f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) top[i] = fmaxf(top[i], stat[k][r0 + 8 * i].x);
            const float b = top[i] == -INFINITY ? 0.f : top[i];
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                const float2 x = stat[k][r0 + 8 * i];
                sum[i] = fmaf(exp2f(x.x - b), x.y, sum[i]);
            }
            const float f = exp2f(m[i] - b);
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) {
                o[n][2 * i] *= f;
                o[n][2 * i + 1] *= f;
            }
        }
#pragma unroll
        for (int step = 2; step >= 1; step >>= 1)
#pragma unroll
            for (int half = 0; half < C::kHalves; ++half) {
                if (w >= step && w < 2 * step) {
                    float4 *dst = reinterpret_cast<float4 *>(join) + (w - step) * 256 + lane;
#pragma unroll
                    for (int n = 0; n < 8; ++n)
                        dst[32 * n] = make_float4(o[8 * half + n][0], o[8 * half + n][1],
                                                  o[8 * half + n][2], o[8 * half + n][3]);
                }
                consumers_sync();
                if (w < step) {
                    const float4 *src = reinterpret_cast<const float4 *>(join) + w * 256 + lane;
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        const float4 x = src[32 * n];
                        o[8 * half + n][0] += x.x;
                        o[8 * half + n][1] += x.y;
                        o[8 * half + n][2] += x.z;
                        o[8 * half + n][3] += x.w;
                    }
                }
                consumers_sync();
            }
        if (w != 0) continue;
        if (wk.part != kPartNone && lane == 0)
            desc[wk.slot] = make_int4(wk.part, wk.tok0, wk.n_tok, wk.h);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = r0 + 8 * i;
            if (row >= n_rows) continue;
            if (wk.part != kPartNone) {
                const int64_t rec = ((int64_t)blockIdx.x * 2 + wk.slot) * kRows + row;
#pragma unroll
                for (int n = 0; n < DP / 8; ++n)
                    *reinterpret_cast<float2 *>(a.part_o + rec * DP + 8 * n + kk) =
                        make_float2(o[n][2 * i], o[n][2 * i + 1]);
                if ((lane & 3) == 0) a.part_ml[rec] = make_float2(top[i], sum[i]);
                continue;
            }
            const int64_t head = (int64_t)(wk.tok0 + row / a.group) * a.q_heads +
                                 wk.h * a.group + row % a.group;
            const bool none = sum[i] == 0.f;
            const float r = none ? 0.f : 1.f / sum[i];
            __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.out) + head * a.D;
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
                if (8 * n < a.D)
                    *reinterpret_cast<uint32_t *>(dst + 8 * n + kk) =
                        none ? 0u : pack_bf16(o[n][2 * i] * r, o[n][2 * i + 1] * r);
            if (a.lse && (lane & 3) == 0)
                a.lse[head] = none ? -INFINITY : (top[i] + log2f(sum[i])) / kLog2e;
        }
    }
}

template <int DP> cudaError_t go(const AttnArgs &a, const CUtensorMap &k, const CUtensorMap &v,
                                 int box_rows, int ctas, cudaStream_t st) {
    const cudaError_t e = allow_dynamic_smem<decode_kernel<DP>>(Cfg<DP>::kSmem);
    if (e != cudaSuccess) return e;
    decode_kernel<DP><<<ctas, kThreads, Cfg<DP>::kSmem, st>>>(k, v, a, box_rows);
    return cudaGetLastError();
}

}  // namespace

int decode_box_rows(int page_size) { return page_size < kKeys ? page_size : kKeys; }

cudaError_t launch_decode(const AttnArgs &a, const CUtensorMap &k, const CUtensorMap &v, int ctas,
                          cudaStream_t st) {
    const int box = decode_box_rows(1 << a.page_shift);
    return a.D <= 64 ? go<64>(a, k, v, box, ctas, st) : go<128>(a, k, v, box, ctas, st);
}

}  // namespace paged
}  // namespace um

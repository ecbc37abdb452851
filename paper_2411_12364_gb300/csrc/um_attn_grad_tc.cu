// um_attn_grad_tc.cu -- the gradient of the attention of whole sequences on the
// tensor cores (bf16, heads up to 128 wide).
//
// One kernel, two roles.  A CTA holds 128 keys (K, V) and streams the blocks of
// 128 rows that see them, for all query heads of the key/value head:
//   S^T = K Q^T, P^T = 2^(S^T - lse)     dP^T = V dO^T, dS^T = P^T (dP^T - d)
//   dV += P^T dO                         dK += dS^T Q
// or it holds 128 rows (Q, dO) of a head and streams the keys they see:
//   S = Q K^T, dP = dO V^T, dS as above  dQ += dS K
// In a short batch a cluster shares out the steps of a block of keys, and its CTAs
// add one another's sums from shared memory, each for a part of the rows.
// Scores have the held rows on TMEM lanes, so that P and dS, written back to
// TMEM as bf16, are the A operands of the sums, whose accumulators stay in
// TMEM for the whole tile; the streamed tiles serve both as K-major B operands
// (scores) and as MN-major ones (sums).  dS leaves the scale out; the sums take it.
//
// Per block of 128 x 128 the products take 2048 (keys held) and 1536 (rows held)
// cycles of the tensor pipe at width 128, the exponentials 1024 of the
// special-function units.  What overlaps them is the order of issue: with
// keys held dP_j, [P_j] dV_j, S_{j+1}, [dS_j] dK_j (brackets: what the product
// waits for), so that P_{j+1} is computed under dK_j and dP_{j+1} and dS_j
// under dV_j and S_{j+1}.  Narrow heads and held rows leave room in TMEM for a
// second block of scores, issued one block ahead.
//
// Warps: 0-15 P and dS (a thread a held row, four warps for each quarter of the
// streamed columns) and the output, 16 products, 17 copies (TMA), 18 the streamed
// rows' lse and d, and zeros over what a last block holds past the sequence
// (weight 0 times anything there must stay 0), 19 the sums of held rows.  P and dS are
// a chain of loads from TMEM, exponentials, stores and barriers; eight warps for
// them took 2500 cycles a block, waiting for one another's latencies.
//
// 4 sequences of 4096, 16 heads on 4 x 128: 610 us, 1.6 PFLOP/s of the seven
// products, tensor pipe 71 % active; 24 of up to 2048, 16 heads on 2 x 64: 438 us,
// 38 % active, bound by that chain.
#include "um_attn_grad.cuh"

#include <type_traits>

#include "um_device.cuh"
#include "um_pair.cuh"
#include "um_tc.cuh"

namespace um {
namespace attn_grad {
namespace {

constexpr int kSoftmax = 16;                     // warps that make P and dS
constexpr int kThreads = (kSoftmax + 4) * 32;
constexpr int kRows = 128;                       // held, and streamed at a time
constexpr uint32_t kHalfBytes = 128 * 128;       // 128 rows x 64 columns of bf16

template <int DP, bool KEYS> struct Cfg {
    static constexpr int kHalves = DP / 64;
    static constexpr uint32_t kTile = kHalfBytes * kHalves;
    // blocks of scores in TMEM (128 columns each) beside dP and the sums
    static constexpr int kScores = KEYS && DP == 128 ? 1 : 2;
    // streamed tiles that the sums read last (Q or K), and the others (dO or V)
    static constexpr int kLong = DP == 128 ? 3 : 4;
    static constexpr int kShort = DP == 128 ? 2 : 3;
    // a second warp for the sums, where a commit may stand between them and
    // the scores that take their operands' place
    static constexpr bool kTwo = !KEYS;
    static constexpr int kTiles = 2 + kLong + kShort;
    static constexpr size_t kSmem = (size_t)kTile * kTiles + 2 * 2 * kRows * 4 + 512;
    // dV and dK in fp32 over the tiles, rows without bank conflicts
    static constexpr int kSumRow = DP + 4;
    static_assert(2 * kRows * kSumRow * 4 <= kTile * kTiles, "room for the sums");
};

struct Bars {
    uint64_t held, long_full[4], long_raw[4], long_empty[4], short_full[4], short_raw[4],
        short_empty[4], s_full[2], dp_full, p_full[2], ds_full[2], row_full[2], row_empty[2],
        out_full, drained[2];
    uint32_t tmem;
};
static_assert(sizeof(Bars) <= 512, "barriers");

// A place in a ring of N stages and the phase of its barriers.
template <int N> struct Stage {
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++at == N) {
            at = 0;
            phase ^= 1;
        }
    }
};

// What a CTA works on: `steps` streamed blocks.
struct Work {
    int tok0, n, b;            // the sequence's first token and tokens, the held block
    int blocks, steps;         // blocks of the sequence, streamed blocks
    int kv, head;              // key/value head; the query head of held rows
    int rank, ranks;           // of a cluster that shares out the steps of held keys
    __device__ __forceinline__ int of_all(int j) const { return rank + j * ranks; }
    __device__ __forceinline__ int group_of(int j) const { return of_all(j) / (blocks - b); }
    // the streamed block of step j
    template <bool KEYS> __device__ __forceinline__ int block(int j) const {
        return KEYS ? b + of_all(j) % (blocks - b) : j;
    }
    __device__ __forceinline__ bool tail(int block) const {
        return block == blocks - 1 && (n & (kRows - 1));
    }
};

__device__ __forceinline__ void clear_rows(uint8_t *tile, int halves, int from, int lane) {
    for (int x = 0; x < halves; ++x)
        for (int i = from * 8 + lane; i < kRows * 8; i += 32)
            *reinterpret_cast<uint4 *>(tile + x * kHalfBytes + i * 16) = make_uint4(0, 0, 0, 0);
    tc::fence_proxy_async_smem();
    __syncwarp();
}

__device__ __forceinline__ uint32_t pack(float x, float y) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&b);
}

template <int DP, bool KEYS>
__device__ __forceinline__ void run(uint8_t *sm, const CUtensorMap &map_h0,
                                    const CUtensorMap &map_h1, const CUtensorMap &map_l,
                                    const CUtensorMap &map_s, const Args &a, unsigned cta,
                                    int rank, int ranks) {
    using C = Cfg<DP, KEYS>;
    uint8_t *held0 = sm, *held1 = sm + C::kTile, *ring_l = sm + 2 * C::kTile,
            *ring_s = ring_l + C::kLong * C::kTile;
    float *row_lse = reinterpret_cast<float *>(ring_s + C::kShort * C::kTile);   // [2][kRows]
    float *row_d = row_lse + 2 * kRows;
    Bars &bar = *reinterpret_cast<Bars *>(row_d + 2 * kRows);
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;

    const int heads = KEYS ? a.kv_heads : a.q_heads;
    const int index = (int)(cta / heads);
    if (index >= *a.count) return;
    const int4 blk = a.blocks[KEYS ? index : a.most + index];   // the longest first
    Work wk;
    wk.tok0 = blk.x;
    wk.n = blk.y;
    wk.b = blk.z;
    wk.blocks = (blk.y + kRows - 1) / kRows;
    wk.head = (int)(cta % heads);
    wk.kv = KEYS ? wk.head : wk.head / a.group;
    wk.rank = rank;
    wk.ranks = ranks;
    // ranks <= group: every CTA has a step
    wk.steps = KEYS ? (a.group * (wk.blocks - wk.b) - rank + ranks - 1) / ranks : wk.b + 1;
    const int steps = wk.steps;

    if (tid == 0) {
        tc::mbar_init(&bar.held, 1);
        for (int i = 0; i < 4; ++i) {
            tc::mbar_init(&bar.long_full[i], 1);
            tc::mbar_init(&bar.long_raw[i], 1);
            tc::mbar_init(&bar.long_empty[i], 1);
            tc::mbar_init(&bar.short_full[i], 1);
            tc::mbar_init(&bar.short_raw[i], 1);
            tc::mbar_init(&bar.short_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&bar.s_full[i], 1);
            // two of each, in turns: the warp that waits for one may be a step late
            tc::mbar_init(&bar.p_full[i], kSoftmax);
            tc::mbar_init(&bar.ds_full[i], kSoftmax);
            tc::mbar_init(&bar.row_full[i], 32);
            tc::mbar_init(&bar.row_empty[i], kSoftmax);
        }
        tc::mbar_init(&bar.dp_full, 1);
        tc::mbar_init(&bar.out_full, 1);
        tc::mbar_init(&bar.drained[0], 1);
        tc::mbar_init(&bar.drained[1], 1);
        tc::fence_mbar_init();
    }
    if (w == kSoftmax) tc::tmem_alloc(&bar.tmem, 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    pdl_trigger();
    const uint32_t tmem = bar.tmem;
    const uint32_t t_dp = 128 * C::kScores, t_o0 = t_dp + 128, t_o1 = t_o0 + (KEYS ? DP : 0);
    bool ok = true;

    if (w < kSoftmax) {
        const int part = w >> 2, row = (w & 3) * 32 + lane;    // quarter of the columns, held row
        const uint32_t lanes = tmem + ((uint32_t)((w & 3) * 32) << 16);
        const int held = wk.b * kRows + row;                   // in the sequence
        const F2 scale = f2(a.scale_log2);
        F2 own_lse = f2(0.f), own_d = f2(0.f);
        if (!KEYS) {
            float2 r = make_float2(INFINITY, 0.f);
            if (held < wk.n) r = a.rows[(int64_t)wk.head * a.T + wk.tok0 + held];
            own_lse = f2(-r.x * kLog2e);
            own_d = f2(-r.y);
        }
        uint32_t s_phase = 0;                                  // a bit a block of scores
        // A block's P and dS; MASKED: the diagonal block, whose rows see the keys
        // up to their own, and a short last one.
        auto block = [&](auto masked, int j) {
            constexpr bool MASKED = decltype(masked)::value;
            const int sb = j % C::kScores, st = j & 1;
            const int str0 = wk.block<KEYS>(j) * kRows + 32 * part;   // the first streamed column
            const float *lse = row_lse + st * kRows + 32 * part, *d = row_d + st * kRows + 32 * part;
            auto sees = [&](int k) {
                const int at = str0 + k;
                return KEYS ? held <= at && at < wk.n : at <= held;
            };
            if (KEYS && !tc::warp_wait(&bar.row_full[st], (j >> 1) & 1)) return false;
            if (!tc::warp_wait(&bar.s_full[sb], (s_phase >> sb) & 1)) return false;
            s_phase ^= 1u << sb;
            // these scores were issued behind dV of kScores steps before, and dP
            // behind dK of the step before: their stages are free
            if (!C::kTwo && j >= C::kScores && w == 0) {
                if (lane == 0) tc::mbar_arrive(&bar.short_empty[(j - C::kScores) % C::kShort]);
                __syncwarp();
            }
            tc::tc_fence_after();
            const uint32_t ts = lanes + 128 * sb + 32 * part, tdp = lanes + t_dp + 32 * part;
            uint32_t s[32], p[16];
            tc::tmem_ld32_nowait(ts, s);
            tc::tmem_ld_wait();
            tc::arrived(s);
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
                F2 l0 = own_lse, l1 = own_lse;
                if (KEYS) {
                    const float4 v = *reinterpret_cast<const float4 *>(lse + k);
                    l0 = f2(v.x, v.y);
                    l1 = f2(v.z, v.w);
                }
                const float2 y0 =
                    split(fma2(f2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), scale, l0));
                const float2 y1 =
                    split(fma2(f2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])), scale, l1));
                float e[4] = {tc::ex2(y0.x), tc::ex2(y0.y), tc::ex2(y1.x), tc::ex2(y1.y)};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (MASKED) e[i] = sees(k + i) ? e[i] : 0.f;
                    s[k + i] = __float_as_uint(e[i]);
                }
                // weights as an operand: one rounding to bf16, as large as that
                // of the values they multiply
                p[k / 2] = pack(e[0], e[1]);
                p[k / 2 + 1] = pack(e[2], e[3]);
            }
            if (KEYS) {
                tc::tmem_st16(ts, p);
                tc::tmem_st_wait();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&bar.p_full[st]);
            }
            if (!tc::warp_wait(&bar.dp_full, j & 1)) return false;
            if (!C::kTwo && j > 0 && w == 0) {
                if (lane == 0) tc::mbar_arrive(&bar.long_empty[(j - 1) % C::kLong]);
                __syncwarp();
            }
            tc::tc_fence_after();
            uint32_t g[32];
            tc::tmem_ld32_nowait(tdp, g);
            tc::tmem_ld_wait();
            tc::arrived(g);
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
                F2 d0 = own_d, d1 = own_d;
                if (KEYS) {
                    const float4 v = *reinterpret_cast<const float4 *>(d + k);
                    d0 = f2(v.x, v.y);
                    d1 = f2(v.z, v.w);
                }
                const F2 x0 = f2(__uint_as_float(g[k]), __uint_as_float(g[k + 1])) + d0;
                const F2 x1 = f2(__uint_as_float(g[k + 2]), __uint_as_float(g[k + 3])) + d1;
                float2 y0 = split(f2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])) * x0);
                float2 y1 = split(f2(__uint_as_float(s[k + 2]), __uint_as_float(s[k + 3])) * x1);
                if (MASKED && !KEYS) {     // V past the sequence may be anything
                    y0.x = sees(k) ? y0.x : 0.f;
                    y0.y = sees(k + 1) ? y0.y : 0.f;
                    y1.x = sees(k + 2) ? y1.x : 0.f;
                    y1.y = sees(k + 3) ? y1.y : 0.f;
                }
                p[k / 2] = pack(y0.x, y0.y);
                p[k / 2 + 1] = pack(y1.x, y1.y);
            }
            tc::tmem_st16(KEYS ? tdp : ts, p);
            tc::tmem_st_wait();
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                tc::mbar_arrive(&bar.ds_full[st]);
                if (KEYS) tc::mbar_arrive(&bar.row_empty[st]);
            }
            return true;
        };
        for (int j = 0; ok && j < steps; ++j) {
            const int b = wk.block<KEYS>(j);
            ok = b == wk.b || wk.tail(b) ? block(std::true_type(), j) : block(std::false_type(), j);
        }
        if (ok) ok = tc::warp_wait(&bar.out_full, 0);
        if (ok && KEYS && ranks > 1) {
            // every product is done and every tile read: the sums take their place
            tc::tc_fence_after();
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                float *to = reinterpret_cast<float *>(sm) + (o * kRows + row) * C::kSumRow;
#pragma unroll
                for (int c = 0; c < DP / 64; ++c) {
                    const int col = part * (DP / 4) + 16 * c;
                    float v[16];
                    tc::tmem_ld16(lanes + (o == 0 ? t_o0 : t_o1) + col, v);
#pragma unroll
                    for (int k = 0; k < 16; ++k) asm volatile("" : "+f"(v[k]));   // after the wait
#pragma unroll
                    for (int k = 0; k < 16; k += 4)
                        *reinterpret_cast<float4 *>(to + col + k) =
                            make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
                }
            }
            tc::tc_fence_before();
        } else if (ok) {
            tc::tc_fence_after();
            const int64_t tok = (int64_t)wk.tok0 + held;
#pragma unroll
            for (int o = 0; o < (KEYS ? 2 : 1); ++o) {
                // dV, then dK, or dQ
                const bool scaled = !KEYS || o == 1;
                __nv_bfloat16 *to =
                    KEYS ? (o == 0 ? static_cast<__nv_bfloat16 *>(a.dv) + tok * a.dv_stride
                                   : static_cast<__nv_bfloat16 *>(a.dk) + tok * a.dk_stride)
                         : static_cast<__nv_bfloat16 *>(a.dq) + tok * a.dq_stride;
                to += (int64_t)wk.head * a.D;
                const float f = scaled ? a.scale : 1.f;
#pragma unroll
                for (int c = 0; c < DP / 64; ++c) {
                    const int col = part * (DP / 4) + 16 * c;
                    float v[16];
                    __syncwarp();                              // rows past the end go on below
                    tc::tmem_ld16(lanes + (o == 0 ? t_o0 : t_o1) + col, v);
#pragma unroll
                    for (int k = 0; k < 16; ++k) asm volatile("" : "+f"(v[k]));   // after the wait
                    if (held >= wk.n) continue;
#pragma unroll
                    for (int k = 0; k < 16; k += 8) {
                        if (col + k >= a.D) break;
                        uint32_t x[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            x[i] = pack(v[k + 2 * i] * f, v[k + 2 * i + 1] * f);
                        *reinterpret_cast<uint4 *>(to + col + k) =
                            make_uint4(x[0], x[1], x[2], x[3]);
                    }
                }
            }
            tc::tc_fence_before();
        }
        if (!ok && lane == 0) atomicOr(a.err, kErrTimeout);
    } else if (w == kSoftmax || (C::kTwo && w == kSoftmax + 3)) {
        // ---- products: the whole warp waits, one elected thread issues.  A
        // wait costs the issuing warp about 100 cycles, a commit as much and a
        // product 24.  With keys held one warp issues everything, in the order
        // that the buffers allow without a wait for a product's end; with rows held
        // it would be busy for longer than the products run (2600 cycles a
        // block at width 128), and a second one issues the sums ----
        constexpr uint32_t idesc_s = tc::idesc_bf16_f32(128, 128);
        constexpr uint32_t idesc_o = tc::idesc_bf16_f32(128, DP) | tc::kBColumns;
        const bool leader = tc::elect_one();
        const uint32_t base = tc::uniform(tmem);
        const uint64_t h0 = tc::desc_k_sw128(tc::smem_u32(held0));
        const uint64_t h1 = tc::desc_k_sw128(tc::smem_u32(held1));
        const uint64_t l_k = tc::desc_k_sw128(tc::smem_u32(ring_l));
        const uint64_t s_k = tc::desc_k_sw128(tc::smem_u32(ring_s));
        const uint64_t l_mn = tc::desc_mn_sw128(tc::smem_u32(ring_l), kHalfBytes);
        const uint64_t s_mn = tc::desc_mn_sw128(tc::smem_u32(ring_s), kHalfBytes);
        auto commit = [&](uint64_t *b) {
            if (leader) tc::mma_commit(b);
        };
        auto product = [&](uint32_t to, uint64_t x, uint64_t y) {   // over the head width
            if (leader) {
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const uint32_t off = ((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
                    tc::mma_bf16(base + to, x + off, y + off, idesc_s, k > 0);
                }
            }
        };
        auto sum = [&](uint32_t to, uint32_t x, uint64_t y, bool add) {   // over the block's rows
            if (leader) {
#pragma unroll
                for (int k = 0; k < kRows / 16; ++k)
                    // each quarter of the columns was written where its scores were
                    tc::mma_bf16_ts(base + to, base + x + (k >> 1) * 32 + (k & 1) * 8,
                                    y + k * (16 * 128 >> 4), idesc_o, add || k > 0);
            }
        };
        Stage<C::kLong> l;
        Stage<C::kShort> h;
        auto scores = [&](int j) {               // S of step j, the l-th stage
            if (!tc::warp_wait(&bar.long_full[l.at], l.phase)) return false;
            tc::tc_fence_after();
            product(128 * (j % C::kScores), h0, l_k + (uint32_t)l.at * (C::kTile >> 4));
            commit(&bar.s_full[j % C::kScores]);
            l.next();
            return true;
        };
        auto other = [&] {                       // dP of the next step
            if (!tc::warp_wait(&bar.short_full[h.at], h.phase)) return false;
            tc::tc_fence_after();
            product(t_dp, h1, s_k + (uint32_t)h.at * (C::kTile >> 4));
            commit(&bar.dp_full);
            if (!KEYS) commit(&bar.short_empty[h.at]);
            h.next();
            return true;
        };
        auto sum_short = [&](int j, const Stage<C::kShort> &st) {   // dV
            if (!tc::warp_wait(&bar.p_full[j & 1], (j >> 1) & 1)) return false;
            tc::tc_fence_after();
            sum(t_o0, 128 * (j % C::kScores), s_mn + (uint32_t)st.at * (C::kTile >> 4), j > 0);
            return true;
        };
        auto sum_long = [&](int j, const Stage<C::kLong> &st) {     // dK or dQ
            if (!tc::warp_wait(&bar.ds_full[j & 1], (j >> 1) & 1)) return false;
            tc::tc_fence_after();
            sum(KEYS ? t_o1 : t_o0, KEYS ? t_dp : 128 * (j % C::kScores),
                l_mn + (uint32_t)st.at * (C::kTile >> 4), j > 0);
            if (C::kTwo) commit(&bar.long_empty[st.at]);
            return true;
        };
        if (!C::kTwo) {
            // what a step's stages are free of is told to the copies by the warps
            // that wait for the commits behind it
            Stage<C::kLong> ls;
            Stage<C::kShort> hs;
            ok = tc::warp_wait(&bar.held, 0);
            for (int j = 0; ok && j < C::kScores && j < steps; ++j) ok = scores(j);
            for (int j = 0; ok && j < steps; ++j, ls.next(), hs.next())
                ok = other() && sum_short(j, hs) &&
                     (j + C::kScores >= steps || scores(j + C::kScores)) && sum_long(j, ls);
            if (ok) commit(&bar.out_full);
        } else if (w == kSoftmax) {
            Stage<C::kLong> ls;
            ok = tc::warp_wait(&bar.held, 0);
            for (int j = 0; ok && j < C::kScores && j < steps; ++j) ok = scores(j);
            if (ok) ok = other();
            for (int j = 0; ok && j + 1 < steps; ++j, ls.next())
                // dP was read, and dS by the sum, whose place S of step j + 2 takes
                ok = tc::warp_wait(&bar.ds_full[j & 1], (j >> 1) & 1) && other() &&
                     (j + C::kScores >= steps ||
                      (tc::warp_wait(&bar.long_empty[ls.at], ls.phase) && scores(j + C::kScores)));
        } else {
            Stage<C::kLong> ls;
            for (int j = 0; ok && j < steps; ++j, ls.next()) ok = sum_long(j, ls);
            if (ok) commit(&bar.out_full);
        }
        if (!ok) {
            if (leader) atomicOr(a.err, kErrTimeout);
            uint64_t *drained = &bar.drained[w == kSoftmax ? 0 : 1];
            commit(drained);                   // products in flight end before TMEM is freed
            tc::warp_wait(drained, 0);
        }
    } else if (w == kSoftmax + 1) {
        // ---- copies, in the order in which the products read them ----
        if (lane == 0) {
            tc::prefetch_tensormap(&map_h0);
            tc::prefetch_tensormap(&map_h1);
            tc::prefetch_tensormap(&map_l);
            tc::prefetch_tensormap(&map_s);
            auto load = [&](uint8_t *to, const CUtensorMap *map, uint64_t *b, int head, int tok) {
                tc::mbar_arrive_expect_tx(b, C::kTile);
#pragma unroll
                for (int x = 0; x < C::kHalves; ++x)
                    tc::tma_load_3d(to + x * kHalfBytes, map, b, 64 * x, head, tok);
            };
            const int at = wk.tok0 + wk.b * kRows;
            tc::mbar_arrive_expect_tx(&bar.held, 2 * C::kTile);
#pragma unroll
            for (int x = 0; x < C::kHalves; ++x) {
                tc::tma_load_3d(held0 + x * kHalfBytes, &map_h0, &bar.held, 64 * x, wk.head, at);
                tc::tma_load_3d(held1 + x * kHalfBytes, &map_h1, &bar.held, 64 * x, wk.head, at);
            }
            auto stream = [&](int j, bool is_long) {
                const int n = is_long ? C::kLong : C::kShort, st = j % n;
                const uint32_t parity = ((j / n) & 1) ^ 1;
                if (!tc::mbar_wait(is_long ? &bar.long_empty[st] : &bar.short_empty[st], parity))
                    return false;
                const int b = wk.block<KEYS>(j);
                const int head = KEYS ? wk.kv * a.group + wk.group_of(j) : wk.kv;
                // a short last block is cleared past its end before it is used
                const bool raw = wk.tail(b) && (is_long || KEYS);
                if (is_long)
                    load(ring_l + st * C::kTile, &map_l, raw ? &bar.long_raw[st] : &bar.long_full[st],
                         head, wk.tok0 + b * kRows);
                else
                    load(ring_s + st * C::kTile, &map_s,
                         raw ? &bar.short_raw[st] : &bar.short_full[st], head, wk.tok0 + b * kRows);
                return true;
            };
            for (int j = 0; ok && j < C::kScores && j < steps; ++j) ok = stream(j, true);
            for (int j = 0; ok && j < steps; ++j) {
                ok = stream(j, false);
                if (ok && j + C::kScores < steps) ok = stream(j + C::kScores, true);
            }
            if (!ok) {
                atomicOr(a.err, kErrTimeout);
                // copies in flight end by themselves: give them far longer than they take
                const long long start = clock64();
                while (clock64() - start < 4000000ll) __nanosleep(1000);
            }
        }
        __syncwarp();
    } else if (w == kSoftmax + 2) {
        uint32_t l_raw = 0, s_raw = 0;         // phases, a bit a stage
        const int from = wk.n & (kRows - 1);
        float2 ahead[kRows / 32];              // of the next step: in flight while this one runs
        auto rows_of = [&](int j) {
            const float2 *rows = a.rows + (int64_t)(wk.kv * a.group + wk.group_of(j)) * a.T + wk.tok0;
#pragma unroll
            for (int i = 0; i < kRows / 32; ++i) {
                const int r = wk.block<KEYS>(j) * kRows + 32 * i + lane;
                ahead[i] = r < wk.n ? rows[r] : make_float2(INFINITY, 0.f);
            }
        };
        if (KEYS) rows_of(0);
        for (int j = 0; ok && j < steps; ++j) {
            const int b = wk.block<KEYS>(j);
            if (wk.tail(b)) {
                int st = j % C::kLong;
                if (!(ok = tc::warp_wait(&bar.long_raw[st], (l_raw >> st) & 1))) break;
                l_raw ^= 1u << st;
                clear_rows(ring_l + st * C::kTile, C::kHalves, from, lane);
                if (lane == 0) tc::mbar_arrive(&bar.long_full[st]);
                if (KEYS) {
                    st = j % C::kShort;
                    if (!(ok = tc::warp_wait(&bar.short_raw[st], (s_raw >> st) & 1))) break;
                    s_raw ^= 1u << st;
                    clear_rows(ring_s + st * C::kTile, C::kHalves, from, lane);
                    if (lane == 0) tc::mbar_arrive(&bar.short_full[st]);
                }
            }
            if (!KEYS) continue;
            const int st = j & 1;
            if (!(ok = tc::warp_wait(&bar.row_empty[st], ((j >> 1) & 1) ^ 1))) break;
#pragma unroll
            for (int i = 0; i < kRows / 32; ++i) {
                row_lse[st * kRows + 32 * i + lane] = -ahead[i].x * kLog2e;
                row_d[st * kRows + 32 * i + lane] = -ahead[i].y;
            }
            tc::mbar_arrive(&bar.row_full[st]);
            if (j + 1 < steps) rows_of(j + 1);
        }
        if (!ok && lane == 0) atomicOr(a.err, kErrTimeout);
    }
    __syncwarp();
    __syncthreads();
    if (w == kSoftmax) tc::tmem_dealloc(tmem, 512);
    if (KEYS && ranks > 1) {
        // a CTA's part of the rows: the sums of all, in their order
        tc::cluster_sync();
        const int pieces = a.D / 8;
        for (int k = tid; k < 2 * (kRows / ranks) * pieces; k += kThreads) {
            const int i = k / pieces, col = k % pieces * 8;
            const int o = i & 1, row = rank + (i >> 1) * ranks, held = wk.b * kRows + row;
            if (held >= wk.n) continue;
            const float *from = reinterpret_cast<float *>(sm) + (o * kRows + row) * C::kSumRow + col;
            float4 x = load_peer(from, 0), y = load_peer(from + 4, 0);
            for (int p = 1; p < ranks; ++p) {
                const float4 u = load_peer(from, p), v = load_peer(from + 4, p);
                x.x += u.x, x.y += u.y, x.z += u.z, x.w += u.w;
                y.x += v.x, y.y += v.y, y.z += v.z, y.w += v.w;
            }
            const float f = o ? a.scale : 1.f;
            const int64_t tok = (int64_t)wk.tok0 + held;
            __nv_bfloat16 *to = o ? static_cast<__nv_bfloat16 *>(a.dk) + tok * a.dk_stride
                                  : static_cast<__nv_bfloat16 *>(a.dv) + tok * a.dv_stride;
            *reinterpret_cast<uint4 *>(to + (int64_t)wk.head * a.D + col) =
                make_uint4(pack(x.x * f, x.y * f), pack(x.z * f, x.w * f), pack(y.x * f, y.y * f),
                           pack(y.z * f, y.w * f));
        }
        __syncwarp();
        tc::cluster_sync();                  // peers have read this CTA's sums
    }
}

// Both roles in one launch: the long tiles of held keys first, and the many
// short ones of held rows fill the SMs that those leave.  A cluster takes one
// tile of keys, or as many of rows as it has CTAs.
template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
    grad_kernel(const __grid_constant__ CUtensorMap q, const __grid_constant__ CUtensorMap k,
                const __grid_constant__ CUtensorMap v, const __grid_constant__ CUtensorMap dout,
                Args a) {
    extern __shared__ __align__(1024) uint8_t sm[];
    pdl_wait();
    const unsigned keys = (unsigned)a.most * a.kv_heads;
    if (blockIdx.x < keys)
        run<DP, true>(sm, k, v, q, dout, a, blockIdx.x, blockIdx.z, gridDim.z);
    else
        run<DP, false>(sm, q, dout, k, v, a, (blockIdx.x - keys) * gridDim.z + blockIdx.z, 0, 1);
}

template <int DP>
cudaError_t go(const Args &a, const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v,
               const CUtensorMap &dout, cudaStream_t st) {
    static_assert(Cfg<DP, true>::kSmem == Cfg<DP, false>::kSmem, "one launch");
    const cudaError_t e = allow_dynamic_smem<grad_kernel<DP>>(Cfg<DP, true>::kSmem);
    if (e != cudaSuccess) return e;
    return launch_kernel(true, (unsigned)a.ranks, grad_kernel<DP>, grid_of(a), kThreads,
                         Cfg<DP, true>::kSmem, st, q, k, v, dout, a);
}

}  // namespace

cudaError_t launch_tensor(const Args &a, const CUtensorMap &q, const CUtensorMap &k,
                          const CUtensorMap &v, const CUtensorMap &dout, cudaStream_t st) {
    return a.D <= 64 ? go<64>(a, q, k, v, dout, st) : go<128>(a, q, k, v, dout, st);
}

}  // namespace attn_grad
}  // namespace um

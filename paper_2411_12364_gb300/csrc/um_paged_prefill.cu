// um_paged_prefill.cu -- attention over the paged cache for chunks of new
// tokens (bf16, heads up to 128 wide), on the tensor cores.
//
// One persistent CTA an SM works on tiles of 2 x 128 rows (new tokens x the
// query heads of one key/value head, token-major, so that a key block is read
// once for the whole group) against blocks of 128 keys:
//   S_i = Q_i K^T        tcgen05.mma, both operands from shared memory
//   P_i = 2^(S_i - m)    128 threads a half, one row each, S read from TMEM
//   O_i += P_i V         tcgen05.mma, P from TMEM, V from shared memory
// with S_0, S_1, O_0, O_1 in TMEM (512 columns at width 128); P_i takes S_i's
// columns as bf16.  The two halves are what keeps the tensor cores busy: while
// the threads of one half turn S into P, the tensor cores run the other
// half's products.  Per block and half the products take 1024 cycles of the
// tensor pipe at width 128 and the exponentials and their bookkeeping about
// as many issue slots of one warp a scheduler, so the kernel is bound by
// these two together.
//
// The maximum that the exponents refer to is not raised for every block, only
// when a row's new maximum passes it by 2^8: the output and the sum refer to
// the same value, so the quotient is the same, and the pass over O in TMEM
// that a raise costs is rare.
//
// Measured: 4 prompts of 4096 tokens (16 / 4 heads x 128) 197 us without the
// join of split tiles, 1396 TFLOP/s of what the causal rows need, the tensor
// pipe 64 % active; 8 ragged chunks over up to 31 k keys at width 64 264 us,
// 985 TFLOP/s.  The softmax threads spill 22 of their registers (88 bytes a
// thread; the compiler holds the kernel to the 168 of the launch, of which a
// row's scores take 128); the other roles spill none.
//
// Warps: 0-3 and 4-7 the halves' softmax and output, 8 and 11 the halves'
// products (one elected thread each), 9 the copies (TMA: K and V blocks, a box
// per page, in a ring; Q per tile), 10 clears what a last page holds past the
// request's length.
#include "um_device.cuh"
#include "um_paged.cuh"
#include "um_pair.cuh"
#include "um_tc.cuh"

namespace um {
namespace paged {
namespace {

constexpr int kKeys = 128;
constexpr int kHalfRows = 128;
constexpr int kThreads = 384;
// registers of a thread: 384 x 168 at launch, split 2 x 128 x 208 + 128 x 88
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(256 * kSoftmaxRegs + 128 * kOtherRegs <= kThreads * 168, "register split");
constexpr uint32_t kHalfBytes = 128 * 128;     // 128 rows x 64 columns of bf16
constexpr float kRaise = 8.f;                  // log2 units

template <int DP> struct Cfg {
    static constexpr int kHalves = DP / 64;                   // 64-column halves of a row
    static constexpr uint32_t kTile = kHalfBytes * kHalves;   // 128 rows
    // Width 64: a stage holds a block's K and V together, which saves the
    // issuing warps a wait and a commit a block (295 -> 273 us for the ragged
    // chunks below).  Width 128 has room for two such stages and a half, so it
    // takes K and V one by one (two whole stages: 305 instead of 223 us).
    static constexpr bool kPaired = DP == 64;
    static constexpr int kParts = kPaired ? 2 : 1;            // tiles of a stage
    static constexpr int kStages = 5;
    static constexpr uint32_t kStage = kTile * kParts;
    static constexpr size_t kSmem = (size_t)kTile * 2 + (size_t)kStage * kStages + 1024;
};

// What each role needs of the tile at hand: blocks [j0, e[i]) of half i.
struct Halves {
    int n_tok[2], e[2], end;
    __device__ __forceinline__ Halves(const Walk &wk, int tq_half) {
        n_tok[0] = min(wk.n_tok, tq_half);
        n_tok[1] = max(0, wk.n_tok - tq_half);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int sees = n_tok[i] ? wk.pos0 + i * tq_half + n_tok[i] : 0;   // keys
            e[i] = max(wk.j0, min(wk.j1, (max(0, sees) + kKeys - 1) / kKeys));
        }
        end = max(e[0], e[1]);
    }
    __device__ __forceinline__ bool live(const Walk &wk) const { return end > wk.j0; }
    // the block that holds the request's last page, when that page has places
    // past the length; -1 without one among [j0, end)
    __device__ __forceinline__ int tail(const Walk &wk, int page_mask) const {
        const int j = wk.kv / kKeys;
        return (wk.kv & page_mask) && j >= wk.j0 && j < end ? j : -1;
    }
};

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
    prefill_kernel(const __grid_constant__ CUtensorMap map_q,
                   const __grid_constant__ CUtensorMap map_k,
                   const __grid_constant__ CUtensorMap map_v, AttnArgs a, int box_rows) {
    using C = Cfg<DP>;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t kv_full[C::kStages], kv_empty[C::kStages], kv_raw[C::kStages];
    __shared__ uint64_t q_full, q_empty, s_full[2], p_full[2], o_full[2], turn[2];
    __shared__ uint64_t drained[2];
    __shared__ int64_t scratch[kThreads / 32 + 1];
    __shared__ Cursor cur;
    __shared__ uint32_t tmem_base;
    uint8_t *qs = raw + ((1024 - (tc::smem_u32(raw) & 1023)) & 1023);
    uint8_t *ring = qs + 2 * C::kTile;
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            tc::mbar_init(&kv_full[s], 1);
            tc::mbar_init(&kv_empty[s], 2);      // both halves' products
            tc::mbar_init(&kv_raw[s], 1);
        }
        tc::mbar_init(&q_full, 1);
        tc::mbar_init(&q_empty, 2);
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&s_full[i], 1);
            tc::mbar_init(&p_full[i], kHalfRows);
            tc::mbar_init(&o_full[i], 1);
            tc::mbar_init(&turn[i], 1);
            tc::mbar_init(&drained[i], 1);
        }
        tc::fence_mbar_init();
    }
    pdl_wait();
    place_share<kThreads>(a, blockIdx.x, gridDim.x, kKeys, 2 * kKeys, scratch, &cur);
    if (w == 8) tc::tmem_alloc(&tmem_base, 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_base;
    const uint32_t tmem_s[2] = {tmem, tmem + 128}, tmem_o[2] = {tmem + 256, tmem + 256 + DP};
    const int tq_half = a.tq / 2;
    const int page_mask = (1 << a.page_shift) - 1;
    Walk wk;
    wk.begin(a, cur);
    bool ok = true;

    if (w < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // ---- softmax and output of half i: thread = row ----
        const int i = w >> 2, row = (w & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((w & 3) * 32) << 16;
        const uint32_t ts = tmem_s[i] + lanes, to = tmem_o[i] + lanes;
        int4 *desc = a.part_desc + 2 * blockIdx.x;
        if (tid == 0) desc[0] = desc[1] = make_int4(kPartNone, 0, 0, 0);
        const int tok = row / a.group, g = row - tok * a.group;
        const F2 scale = f2(a.scale_log2);
        const bool wide = a.D % 16 == 0 && ((uintptr_t)a.out & 31) == 0;
        uint32_t blocks = 0, tiles = 0;      // done so far by this half: barrier phases
        while (ok && wk.next(a, kKeys)) {
            const Halves hv(wk, tq_half);
            const bool mine = tok < hv.n_tok[i] && tok < tq_half;
            const int pos = wk.pos0 + i * tq_half + tok;
            const int limit = mine ? min(wk.kv, pos + 1) : 0;   // keys this row sees
            // keys that all rows of the half see: below it no masking (rows past
            // the tile's tokens hold whatever lies there and are not stored)
            const int all_see = wk.pos0 + i * tq_half + 1;
            float m = -INFINITY, l = 0.f;
            for (int j = wk.j0; j < hv.e[i]; ++j) {
                if (!tc::warp_wait(&s_full[i], blocks & 1)) {
                    ok = false;
                    break;
                }
                ++blocks;
                tc::tc_fence_after();
                uint32_t s[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tc::tmem_ld32_nowait(ts + 32 * c, s[c]);
                tc::tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 4; ++c) tc::arrived(s[c]);
                if ((j + 1) * kKeys > all_see) {
                    const int left = limit - j * kKeys;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (32 * c + k >= left) s[c][k] = 0xff800000u;   // -inf
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = fmaxf(__uint_as_float(s[c][0]), __uint_as_float(s[c][1]));
#pragma unroll
                    for (int k = 2; k < 32; k += 2)
                        mx[c] = max3(mx[c], __uint_as_float(s[c][k]), __uint_as_float(s[c][k + 1]));
                }
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                const bool raise = (top - m) * a.scale_log2 > kRaise ||
                                   (m == -INFINITY && top > -INFINITY);
                if (__any_sync(0xffffffffu, raise)) {
                    const float f = raise ? tc::ex2((m - top) * a.scale_log2) : 1.f;
                    if (raise) m = top;
                    l *= f;
                    if (j > wk.j0) {   // S_i is there, so all earlier products are done
#pragma unroll
                        for (int c = 0; c < DP / 16; ++c) {
                            float o[16];
                            uint32_t x[16];
                            tc::tmem_ld16(to + 16 * c, o);
#pragma unroll
                            for (int k = 0; k < 16; ++k) {
                                asm volatile("" : "+f"(o[k]));   // after the load's wait
                                x[k] = __float_as_uint(o[k] * f);
                            }
                            tc::tmem_st16(to + 16 * c, x);
                        }
                    }
                }
                const F2 shift = f2(m == -INFINITY ? 0.f : -m * a.scale_log2);
                F2 sum[2] = {f2(0.f), f2(0.f)};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t p[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float2 y = split(fma2(f2(__uint_as_float(s[c][2 * k]),
                                                       __uint_as_float(s[c][2 * k + 1])),
                                                    scale, shift));
                        const float e0 = tc::ex2(y.x), e1 = tc::ex2(y.y);
                        sum[k & 1] = sum[k & 1] + f2(e0, e1);
                        // weights as the A operand: one rounding to bf16, as
                        // large as that of the values; the sum keeps fp32
                        const __nv_bfloat162 b = __floats2bfloat162_rn(e0, e1);
                        p[k] = *reinterpret_cast<const uint32_t *>(&b);
                    }
                    tc::tmem_st16(ts + 16 * c, p);
                }
                l += both(sum[0] + sum[1]);
                tc::tmem_st_wait();
                tc::tc_fence_before();
                tc::mbar_arrive(&p_full[i]);
            }
            if (!ok) break;
            const bool any = hv.e[i] > wk.j0;
            if (any) {
                if (!tc::warp_wait(&o_full[i], tiles & 1)) {
                    ok = false;
                    break;
                }
                ++tiles;
                tc::tc_fence_after();
            }
            if (wk.part != kPartNone && tid == 0)
                desc[wk.slot] = make_int4(wk.part, wk.tok0, wk.n_tok, wk.h);
            const int64_t rec = ((int64_t)blockIdx.x * 2 + wk.slot) * a.rows +
                                i * tq_half * a.group + row;
            const int64_t head = (int64_t)(wk.tok0 + i * tq_half + tok) * a.q_heads +
                                 wk.h * a.group + g;
            const bool none = l == 0.f;
            const float r = none ? 0.f : 1.f / l;
            const float top = m == -INFINITY ? -INFINITY : m * a.scale_log2;
            if (mine) {
                if (wk.part != kPartNone)
                    a.part_ml[rec] = make_float2(top, l);
                else if (a.lse)
                    a.lse[head] = none ? -INFINITY : (top + log2f(l)) / kLog2e;
            }
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
                uint32_t o[32];
                if (any) {
                    __syncwarp();                     // rows past the tile go on below
                    tc::tmem_ld32_nowait(to + 32 * c, o);
                    tc::tmem_ld_wait();
                    tc::arrived(o);
                } else {
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = 0u;
                }
                if (!mine) continue;
                if (wk.part != kPartNone) {
                    float *dst = a.part_o + rec * DP + 32 * c;
#pragma unroll
                    for (int k = 0; k < 4; ++k) tc::store_sector(dst + 8 * k, &o[8 * k]);
                    continue;
                }
                __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.out) + head * a.D + 32 * c;
                uint32_t q[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const __nv_bfloat162 b = __floats2bfloat162_rn(
                        none ? 0.f : __uint_as_float(o[2 * k]) * r,
                        none ? 0.f : __uint_as_float(o[2 * k + 1]) * r);
                    q[k] = *reinterpret_cast<const uint32_t *>(&b);
                }
                if (wide) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        if (32 * c + 16 * k < a.D) tc::store_sector(dst + 16 * k, &q[8 * k]);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (32 * c + 8 * k < a.D)
                            *reinterpret_cast<uint4 *>(dst + 8 * k) =
                                make_uint4(q[4 * k], q[4 * k + 1], q[4 * k + 2], q[4 * k + 3]);
                }
            }
            tc::tc_fence_before();   // O is read: the next tile's products may write it
        }
        if (!ok && lane == 0) atomicOr(a.err, kErrTimeout);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    }
    if (w == 8 || w == 11) {
        // ---- products of half i, issued by one elected thread.  A warp for
        // each half, because a wait, a commit and a product cost the issuing
        // warp 60 to 110, 100 and 24 cycles: one warp for both halves was
        // busy for longer than the products run.  The whole warp walks and
        // waits, so that descriptors and bounds are warp-uniform (with one
        // thread in this branch a product took 115 cycles to issue).  The halves
        // take turns, a block's output product and the next scores at a time:
        // left to themselves they may fall into step, and then their softmax
        // and their products collide (3090 instead of 2410 cycles a block) ----
        constexpr uint32_t idesc_s = tc::idesc_bf16_f32(128, kKeys);
        constexpr uint32_t idesc_o = tc::idesc_bf16_f32(128, DP) | tc::kBColumns;
        const int i = w == 8 ? 0 : 1;
        const bool leader = tc::elect_one();
        const uint64_t q_desc = tc::desc_k_sw128(tc::smem_u32(qs + i * C::kTile));
        const uint64_t k_desc = tc::desc_k_sw128(tc::smem_u32(ring));
        const uint64_t v_desc =
            tc::desc_mn_sw128(tc::smem_u32(ring + (C::kPaired ? C::kTile : 0)), kHalfBytes);
        const uint32_t t_s = tc::uniform(tmem) + 128 * i, t_o = tc::uniform(tmem) + 256 + DP * i;
        int stage = 0;
        uint32_t phase = 0, tiles = 0, p_phase = 0, turns = 0;
        auto advance = [&] {
            if (++stage == C::kStages) {
                stage = 0;
                phase ^= 1;
            }
        };
        auto commit = [&](uint64_t *bar) {
            if (leader) tc::mma_commit(bar);
        };
        auto scores = [&](int st) {
            const uint64_t kd = k_desc + (uint32_t)st * (C::kStage >> 4);
            if (leader) {
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const uint32_t off = ((k >> 2) * kHalfBytes + (k & 3) * 32) >> 4;
                    tc::mma_bf16(t_s, q_desc + off, kd + off, idesc_s, k > 0);
                }
                tc::mma_commit(&s_full[i]);
            }
        };
        auto output = [&](int st, bool add) {
            const uint64_t vd = v_desc + (uint32_t)st * (C::kStage >> 4);
            if (leader) {
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k)
                    tc::mma_bf16_ts(t_o, t_s + 8 * k, vd + k * (16 * 128 >> 4), idesc_o,
                                    add || k > 0);
            }
        };
        while (ok && wk.next(a, kKeys)) {
            const Halves hv(wk, tq_half);
            if (!hv.live(wk)) continue;
            const int j0 = tc::uniform(wk.j0), end = tc::uniform(hv.end);
            const int e = tc::uniform(i == 0 ? hv.e[0] : hv.e[1]);   // blocks past e: no products
            if (!(ok = tc::warp_wait(&q_full, tiles & 1))) break;
            ++tiles;
            if (!(ok = tc::warp_wait(&kv_full[stage], phase))) break;
            tc::tc_fence_after();
            if (j0 < e) scores(stage);
            if constexpr (!C::kPaired) {
                commit(&kv_empty[stage]);
                advance();
            }
            if (j0 + 1 == end) commit(&q_empty);
            for (int j = j0; j < end; ++j) {
                const int sv = stage;            // V of this block, then K of the next
                if (!C::kPaired && !(ok = tc::warp_wait(&kv_full[stage], phase))) break;
                advance();
                const bool more = j + 1 < end;
                const int sk = stage;
                if (more && !(ok = tc::warp_wait(&kv_full[stage], phase))) break;
                // half 0 goes first: it waits for half 1's turn before, half 1
                // for half 0's at this block
                if (!(ok = tc::warp_wait(&turn[i ^ 1], (turns & 1) ^ (i == 0)))) break;
                ++turns;
                if (j < e) {
                    if (!(ok = tc::warp_wait(&p_full[i], p_phase))) break;
                    p_phase ^= 1;
                    tc::tc_fence_after();
                    output(sv, j > j0);
                    if (j + 1 == e) commit(&o_full[i]);
                }
                if (j + 1 < e) scores(sk);
                if (leader) tc::mbar_arrive(&turn[i]);
                commit(&kv_empty[sv]);
                if (more) {
                    if (!C::kPaired) commit(&kv_empty[sk]);
                    if (j + 2 == end) commit(&q_empty);
                    if (!C::kPaired) advance();
                }
            }
        }
        if (!ok) {
            if (leader) atomicOr(a.err, kErrTimeout);
            commit(&drained[i]);               // products in flight end before TMEM is freed
            tc::warp_wait(&drained[i], 0);
        }
    } else if (w == 9) {
        // ---- copies: the lanes read the table, one elected thread issues ----
        if (lane == 0) {
            tc::prefetch_tensormap(&map_q);
            tc::prefetch_tensormap(&map_k);
            tc::prefetch_tensormap(&map_v);
        }
        const bool leader = tc::elect_one();
        const int pages = kKeys / box_rows;
        const uint32_t q_bytes = (uint32_t)(tq_half * a.group) * 128 * C::kHalves;
        int stage = 0, issued = 0;
        uint32_t phase = 0, tiles = 0;
        while (ok && wk.next(a, kKeys)) {
            const Halves hv(wk, tq_half);
            if (!hv.live(wk)) continue;
            const int tail = hv.tail(wk, page_mask);
            if (!(ok = tc::warp_wait(&q_empty, (tiles & 1) ^ 1))) break;
            ++tiles;
            if (lane == 0) {
                const int n = hv.n_tok[1] ? 2 : 1;
                tc::mbar_arrive_expect_tx(&q_full, n * q_bytes);
                for (int i = 0; i < n; ++i)
#pragma unroll
                    for (int x = 0; x < C::kHalves; ++x)
                        tc::tma_load_3d(qs + i * C::kTile + x * kHalfBytes, &map_q, &q_full,
                                        64 * x, wk.h * a.group, wk.tok0 + i * tq_half);
            }
            // the table's entry for a block is read a block ahead
            int page = lane < pages ? page_of(a, wk.c.r, wk.j0 * kKeys + lane * box_rows, wk.kv)
                                    : -1;
            for (int j = wk.j0; ok && j < hv.end; ++j) {
                const int key = j * kKeys + lane * box_rows;
                // outside the cache: reads zeros
                const int z = page < 0 ? a.n_pages * a.kv_heads : page * a.kv_heads + wk.h;
                page = lane < pages ? page_of(a, wk.c.r, key + kKeys, wk.kv) : -1;
#pragma unroll
                for (int part = 0; part < 2; ++part) {   // K, then V
                    if (part == 0 || !C::kPaired) {
                        if (!(ok = tc::warp_wait(&kv_empty[stage], phase ^ 1))) break;
                    }
                    uint64_t *bar = (part || C::kPaired) && j == tail ? &kv_raw[stage]
                                                                      : &kv_full[stage];
                    if (leader && (part == 0 || !C::kPaired))
                        tc::mbar_arrive_expect_tx(bar, C::kStage);
                    // the pages one by one with uniform coordinates: a copy a
                    // lane took longer to issue than a block of 16-token pages
                    // takes to compute
                    uint8_t *at = ring + (size_t)stage * C::kStage +
                                  (C::kPaired ? part * C::kTile : 0);
#pragma unroll 8
                    for (int p = 0; p < pages; ++p) {
                        const int zp = (int)__shfl_sync(0xffffffffu, z, p);
                        const int rp = (j * kKeys + p * box_rows) & page_mask;
                        if (leader) {
#pragma unroll
                            for (int x = 0; x < C::kHalves; ++x)
                                tc::tma_load_3d(at + p * box_rows * 128 + x * kHalfBytes,
                                                part ? &map_v : &map_k, bar, 64 * x, rp, zp);
                        }
                    }
                    if (part == 1 || !C::kPaired) {
                        ++issued;
                        if (++stage == C::kStages) {
                            stage = 0;
                            phase ^= 1;
                        }
                    }
                }
            }
        }
        if (!ok) {   // leave nothing in flight: wait for the copies issued last
            if (lane == 0) atomicOr(a.err, kErrTimeout);
            if (tiles) tc::mbar_wait(&q_full, (tiles - 1) & 1);
            for (int k = 0; k < C::kStages && k < issued; ++k) {
                if (--stage < 0) {
                    stage = C::kStages - 1;
                    phase ^= 1;
                }
                tc::mbar_wait(&kv_full[stage], phase);
            }
        }
    } else if (w == 10) {
        // ---- the last page's places past the length may hold anything, and
        // weight 0 times that could be NaN: clear them in V's copy ----
        int stage = 0;
        uint32_t raw_phase = 0;               // a bit a stage
        while (ok && wk.next(a, kKeys)) {
            const Halves hv(wk, tq_half);
            if (!hv.live(wk)) continue;
            const int tail = hv.tail(wk, page_mask);
            const int each = C::kPaired ? 1 : 2;             // stages of a block
            const int n = each * (hv.end - wk.j0);           // and of this tile
            if (tail >= 0) {
                const int st = (stage + each * (tail - wk.j0) + each - 1) % C::kStages;
                if (!(ok = tc::warp_wait(&kv_raw[st], (raw_phase >> st) & 1))) break;
                raw_phase ^= 1u << st;
                const int from = wk.kv - tail * kKeys;
                const int to = min(kKeys, (from | page_mask) + 1);
                uint8_t *v = ring + (size_t)st * C::kStage + (C::kPaired ? C::kTile : 0);
                for (int x = 0; x < C::kHalves; ++x)
                    for (int k = from * 8 + lane; k < to * 8; k += 32)
                        *reinterpret_cast<uint4 *>(v + x * kHalfBytes + k * 16) =
                            make_uint4(0, 0, 0, 0);
                tc::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&kv_full[st]);
            }
            stage = (stage + n) % C::kStages;
        }
        if (!ok && lane == 0) atomicOr(a.err, kErrTimeout);
    }
    __syncwarp();
    __syncthreads();
    if (w == 8) tc::tmem_dealloc(tmem, 512);
}

template <int DP>
cudaError_t go(const AttnArgs &a, const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v,
               int ctas, cudaStream_t st) {
    const cudaError_t e = allow_dynamic_smem<prefill_kernel<DP>>(Cfg<DP>::kSmem);
    if (e != cudaSuccess) return e;
    prefill_kernel<DP><<<ctas, kThreads, Cfg<DP>::kSmem, st>>>(
        q, k, v, a, prefill_box_rows(1 << a.page_shift));
    return cudaGetLastError();
}

}  // namespace

int prefill_box_rows(int page_size) { return page_size < kKeys ? page_size : kKeys; }

cudaError_t launch_prefill(const AttnArgs &a, const CUtensorMap &q, const CUtensorMap &k,
                           const CUtensorMap &v, int ctas, cudaStream_t st) {
    return a.D <= 64 ? go<64>(a, q, k, v, ctas, st) : go<128>(a, q, k, v, ctas, st);
}

}  // namespace paged
}  // namespace um

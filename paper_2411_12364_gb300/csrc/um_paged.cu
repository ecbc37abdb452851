// um_paged.cu -- the paged key/value cache: pages for a step's new tokens
// (paged_plan), the new keys and values into their pages (paged_append), and
// the attention kernel of the storages and head widths that the tensor-core
// kernels do not take, with the kernels that join split tiles.
#include <initializer_list>
#include <mutex>

#include "um_device.cuh"
#include "um_overlap.cuh"
#include "um_paged.cuh"
#include "um_pair.cuh"
#include "um_tc.cuh"

namespace um {
namespace paged {
namespace {

// ---- plan ----------------------------------------------------------------
// One integer pass over the requests' lengths: prefix sums of the new tokens
// (q_start) and of the pages they need.  It is bound by latency, so it is one
// launch: every block of the grid takes both prefix sums over all requests
// itself (a few KB from L2) and then serves its own run of the new tokens.
// The thread that holds the first token of a new page enters that page in
// the table, so the table's writes are spread like the tokens; the pages that
// a token reads from the table are the context's, which nothing writes.
// Measured (graph replay): 6 us for 64 requests with a token each, 10 us for
// 2048 requests with 32 k tokens.
struct PlanArgs {
    const int32_t *ctx, *fresh, *free_pages, *free_count;
    int32_t *table, *q_start, *kv_lens, *slots, *free_left, *balance;
    int n_seqs, n_tokens, page_shift, table_width, n_free;
};

struct PlanRequest {
    int ctx, n;
    int64_t need;               // new pages; 0 when the table is too narrow
    bool fits;
    __device__ __forceinline__ void read(const PlanArgs &a, int r) {
        ctx = max(0, a.ctx[r]);
        n = max(0, a.fresh[r]);
        const int mask = (1 << a.page_shift) - 1;
        const int64_t full = ((int64_t)ctx + n + mask) >> a.page_shift;
        fits = full <= a.table_width && (int64_t)ctx + n <= INT32_MAX;
        need = fits ? full - (((int64_t)ctx + mask) >> a.page_shift) : 0;
    }
    // upto: the pages needed by this and all earlier requests
    __device__ __forceinline__ bool granted(const PlanArgs &a, int64_t upto, int64_t tok0,
                                            int free) const {
        return fits && (need == 0 || upto <= free) && tok0 + n <= a.n_tokens;
    }
};

template <int THREADS> __global__ void __launch_bounds__(THREADS) plan_kernel(PlanArgs a) {
    __shared__ int64_t warp_need[THREADS / 32], warp_tok[THREADS / 32];
    __shared__ int64_t need_at[THREADS], tok_at[THREADS + 1];   // before thread i's run
    __shared__ unsigned long long taken, asked;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int64_t per = ((int64_t)a.n_seqs + THREADS - 1) / THREADS;
    const int r0 = (int)min((int64_t)a.n_seqs, tid * per);
    const int r1 = (int)min((int64_t)a.n_seqs, r0 + per);
    const int free = max(0, min(*a.free_count, a.n_free));
    PlanRequest q;
    int64_t need = 0, tok = 0;
    for (int r = r0; r < r1; ++r) {
        q.read(a, r);
        need += q.need;
        tok += q.n;
    }
    int64_t need_to = need, tok_to = tok;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, need_to, o);
        const int64_t y = __shfl_up_sync(0xffffffffu, tok_to, o);
        if (lane >= o) {
            need_to += x;
            tok_to += y;
        }
    }
    if (lane == 31) {
        warp_need[w] = need_to;
        warp_tok[w] = tok_to;
    }
    if (tid == 0) taken = asked = 0;
    __syncthreads();
    int64_t need_b = need_to - need, tok_b = tok_to - tok, total = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
        if (i < w) {
            need_b += warp_need[i];
            tok_b += warp_tok[i];
        }
        total += warp_tok[i];
    }
    need_at[tid] = need_b;
    tok_at[tid] = tok_b;
    if (tid == 0) tok_at[THREADS] = total;

    if (blockIdx.x == 0) {   // the requests' own outputs
        int64_t upto = need_b, at = tok_b, last = 0, served = 0;
        for (int r = r0; r < r1; ++r) {
            q.read(a, r);
            upto += q.need;
            const bool ok = q.granted(a, upto, at, free);
            if (ok && q.need) last = upto;
            if (ok) served = upto;
            a.q_start[r] = (int32_t)min(at, (int64_t)INT32_MAX);
            a.kv_lens[r] = ok ? q.ctx + q.n : 0;
            at += q.n;
        }
        if (last) atomicMax(&taken, (unsigned long long)last);
        if (served) atomicMax(&asked, (unsigned long long)served);
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        a.q_start[a.n_seqs] = (int32_t)min(total, (int64_t)INT32_MAX);
        if (a.free_left) *a.free_left = free - (int)taken;
        *a.balance = (int32_t)max((int64_t)INT32_MIN, (int64_t)free - (int64_t)asked);
    }

    const int tokens = (int)min(total, (int64_t)a.n_tokens);
    for (int64_t i = (int64_t)blockIdx.x * THREADS + tid; i < a.n_tokens;
         i += (int64_t)gridDim.x * THREADS) {
        if (i >= tokens) {   // past the batch's tokens
            a.slots[i] = -1;
            continue;
        }
        int lo = 0, hi = THREADS - 1;   // the last run that starts at or before i
        while (lo < hi) {
            const int m = (lo + hi + 1) >> 1;
            if (tok_at[m] <= i)
                lo = m;
            else
                hi = m - 1;
        }
        int64_t upto = need_at[lo], at = tok_at[lo];
        int r = (int)(lo * per);
        for (;; ++r) {
            q.read(a, r);
            upto += q.need;
            if (at + q.n > i) break;
            at += q.n;
        }
        int64_t slot = -1;
        if (q.granted(a, upto, at, free)) {
            const int mask = (1 << a.page_shift) - 1;
            const int pos = q.ctx + (int)(i - at), col = pos >> a.page_shift;
            const int old = (int)(((int64_t)q.ctx + mask) >> a.page_shift);
            int32_t *entry = a.table + (int64_t)r * a.table_width + col;
            int page;
            if (col < old) {
                page = *entry;
            } else {
                page = a.free_pages[free - 1 - (upto - q.need + (col - old))];
                if ((pos & mask) == 0) *entry = page;
            }
            slot = page < 0 ? -1 : ((int64_t)page << a.page_shift) + (pos & mask);
        }
        a.slots[i] = slot <= INT32_MAX ? (int32_t)slot : -1;
    }
}

// ---- append --------------------------------------------------------------
// A scatter of whole rows: each thread moves one piece (16 bytes where the
// rows are aligned to that, else one element) of a token's keys and the same
// piece of its values.  Each byte is read and written once, 9.9 us of memory
// traffic for 16384 tokens of 4 heads x 128 in bf16; calls in a row take 14.4
// us, 4.7 TB/s.  What it waits for is latency: each thread has a 64-bit
// division, then the slot's load, then one piece in flight (issue 60 % active,
// the largest stall a load's).  64 tokens: a launch.
template <typename W>
__global__ void __launch_bounds__(256) append_kernel(const W *k, const W *v, int64_t k_stride,
                                                     int64_t v_stride, const int32_t *slots,
                                                     W *k_cache, W *v_cache, int n_tokens,
                                                     int heads, int words, int page_shift,
                                                     int64_t n_slots) {
    const int per_token = heads * words;
    const int64_t total = (int64_t)n_tokens * per_token;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const int t = (int)(i / per_token), j = (int)(i - (int64_t)t * per_token);
        const int slot = slots[t];
        if (slot < 0 || slot >= n_slots) continue;
        const W x = k[t * k_stride + j], y = v[t * v_stride + j];
        const int h = j / words, c = j - h * words;
        const int page = slot >> page_shift, at = slot & ((1 << page_shift) - 1);
        const int64_t dst = ((((int64_t)page * heads + h) << page_shift) + at) * words + c;
        k_cache[dst] = x;
        v_cache[dst] = y;
    }
}

// ---- attention, CUDA cores --------------------------------------------------
// fp32 storage, and bf16 heads that the tensor-core kernels do not take.  A
// block holds a tile of ROWS rows and walks its keys in blocks of kKeys, which
// cp.async brings in as stored, one block ahead: the scores by dot products
// from shared memory, the running maximum and sum of each row, the values
// added into registers.  Sums are fp32 throughout.
//
// What bounds it: reads of shared memory and the fp32 pipes, on which the
// products run as packed pairs.  Many rows (64) share every read among 8 rows
// of a warp; a thread accumulates 4 rows x 4 ND columns.  Few rows (8, 16:
// single tokens) leave nothing to share, so there the threads of one column
// group split the keys between them, each with 8 rows, and add up at the
// tile's end, and warps whose rows are not there take no scores (each reads
// all keys: 295 -> 238 us for the first case below).  Blocks of 64 keys are for
// up to 256 bytes a key, 32 keep two CTAs an SM beyond (238 -> 183 us).
// Measured in fp32: 6 single tokens over up to 31 k keys (16 / 8 heads x 128)
// 183 us, 4.5 TB/s; 8 chunks of up to 45 tokens over up to 24 k keys (8 / 2
// heads x 128) 418 us.
constexpr int kThreads = 256;

template <typename T, int ROWS, int ND> struct RowsCfg {
    static constexpr int DP = 64 * ND;
    static constexpr int kKeys = ND * (int)sizeof(T) <= 4 ? 64 : 32;   // of a block
    static constexpr bool kFew = ROWS <= 16;
    static constexpr int kPitch = DP * (int)sizeof(T) + 16;      // of a key, bytes
    static constexpr int kLdQ = DP + 4, kLdP = ROWS + 4;         // floats
    static_assert(kKeys * DP * (int)sizeof(T) / 16 % kThreads == 0, "whole rounds of copies");
    static constexpr int kQuads = 16 * ND;                       // groups of 4 columns
    static constexpr int kRowGroups = kFew ? ROWS / 8 : 16;      // of 8 or 4 rows
    static constexpr int kGroups =                               // that split the keys
        kFew ? kThreads / (kQuads * kRowGroups) : 1;
    static constexpr size_t kStage = (size_t)2 * kKeys * kPitch; // K and V of a block
    static constexpr size_t kJoin = kFew ? (size_t)kGroups * ROWS * DP * 4 : 0;
    static constexpr size_t kRing = 2 * kStage > kJoin ? 2 * kStage : kJoin;
    static constexpr size_t kSmem =
        sizeof(float) * ((size_t)ROWS * kLdQ + (size_t)kKeys * kLdP) + kRing;
    static constexpr int kPerSm = kSmem <= 115000 ? 2 : 1;
};

__device__ __forceinline__ float4 load4(const float *p) {
    return *reinterpret_cast<const float4 *>(p);
}
__device__ __forceinline__ float4 load4(const __nv_bfloat16 *p) {
    const uint2 q = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xffff0000u),
                       __uint_as_float(q.y << 16), __uint_as_float(q.y & 0xffff0000u));
}

template <typename T, int ROWS, int ND>
__global__ void __launch_bounds__(kThreads, RowsCfg<T, ROWS, ND>::kPerSm) rows_kernel(AttnArgs a) {
    using C = RowsCfg<T, ROWS, ND>;
    constexpr int DP = C::DP, kKeys = C::kKeys;
    constexpr int TPR = kThreads / ROWS;         // threads of a row's softmax
    constexpr int KPT = kKeys / TPR;             // keys each of them holds
    constexpr int RPT = C::kFew ? 8 : 4;         // rows a thread accumulates
    constexpr int NQ = C::kFew ? 1 : ND;         // groups of 4 columns of each
    extern __shared__ __align__(16) float smem[];
    float *qs = smem, *ps = qs + ROWS * C::kLdQ;              // p [key][row]
    char *ring = reinterpret_cast<char *>(ps + kKeys * C::kLdP);
    __shared__ float alpha[ROWS], denom[ROWS], top[ROWS];
    __shared__ int64_t scratch[kThreads / 32 + 1];
    __shared__ Cursor cur;
    const int tid = threadIdx.x, page_mask = (1 << a.page_shift) - 1;
    place_share<kThreads>(a, blockIdx.x, gridDim.x, kKeys, kKeys, scratch, &cur);
    pdl_trigger();
    int4 *desc = a.part_desc + 2 * blockIdx.x;
    if (tid == 0) desc[0] = desc[1] = make_int4(kPartNone, 0, 0, 0);
    Walk wk;
    wk.begin(a, cur);
    const int srow = tid / TPR, spos = tid % TPR;
    const int quad = C::kFew ? tid % C::kQuads : tid & 15;
    const int group = C::kFew ? tid / (C::kQuads * C::kRowGroups) : 0;   // of the keys
    const int row0 = C::kFew ? tid / C::kQuads % C::kRowGroups * 8 : (tid >> 4) * 4;

    // starts the copies of block j into a stage: 16-byte pieces, zeros for keys
    // without a page and columns past the width.  All of a thread's table reads
    // come first, so that they wait for memory once.
    auto fetch = [&](int j, int stage) {
        constexpr int kPieces = DP * (int)sizeof(T) / 16, kEach = 16 / (int)sizeof(T);
        constexpr int kTimes = kKeys * kPieces / kThreads;
        const uint32_t dst0 = (uint32_t)__cvta_generic_to_shared(ring + stage * C::kStage);
        int page[kTimes];
#pragma unroll
        for (int n = 0; n < kTimes; ++n) {
            const int i = tid + n * kThreads, key = i / kPieces, c = (i % kPieces) * kEach;
            page[n] = c < a.D ? page_of(a, wk.c.r, j * kKeys + key, wk.kv) : -1;
        }
#pragma unroll
        for (int n = 0; n < kTimes; ++n) {
            const int i = tid + n * kThreads, key = i / kPieces, c = (i % kPieces) * kEach;
            const int64_t row = ((((int64_t)page[n] * a.kv_heads + wk.h) << a.page_shift) +
                                 ((j * kKeys + key) & page_mask)) * a.D + c;
            const int64_t from = page[n] < 0 ? 0 : row;
            const uint32_t dst = dst0 + key * C::kPitch + c * (int)sizeof(T);
            const int bytes = page[n] < 0 ? 0 : 16;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst),
                         "l"(static_cast<const T *>(a.k) + from), "r"(bytes) : "memory");
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                             dst + kKeys * C::kPitch),
                         "l"(static_cast<const T *>(a.v) + from), "r"(bytes) : "memory");
        }
    };
    auto key_at = [&](int stage, int which, int key) {        // which 0: K, 1: V
        return reinterpret_cast<const T *>(ring + stage * C::kStage +
                                           (which * kKeys + key) * C::kPitch);
    };

    while (wk.next(a, kKeys)) {
        const int n_rows = wk.n_tok * a.group;
        __syncthreads();                         // the tile before is done with shared memory
        fetch(wk.j0, 0);
        asm volatile("cp.async.commit_group;" ::: "memory");
        // queries: a warp a row, the lanes over its columns
#pragma unroll 4
        for (int row = tid >> 5; row < ROWS; row += kThreads / 32) {
            const int tok = row / a.group;
            const T *q = static_cast<const T *>(a.q) + (wk.tok0 + tok) * a.q_stride +
                         (int64_t)(wk.h * a.group + row - tok * a.group) * a.D;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i) {
                const int c = (tid & 31) + 32 * i;
                qs[row * C::kLdQ + c] = row < n_rows && c < a.D ? to_f(q[c]) : 0.f;
            }
        }
        F2 acc[RPT][2 * NQ];
#pragma unroll
        for (int i = 0; i < RPT; ++i)
#pragma unroll
            for (int c = 0; c < 2 * NQ; ++c) acc[i][c] = f2(0.f);
        // each thread of a row keeps the row's maximum; the sum is its share
        float m = -INFINITY, l = 0.f, base = 0.f;
        const int limit = min(wk.kv, wk.pos0 + srow / a.group + 1);   // keys this row sees
        int stage = 0;
        for (int j = wk.j0; j < wk.j1; ++j, stage ^= 1) {
            if (j + 1 < wk.j1) fetch(j + 1, stage ^ 1);
            asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncthreads();
            // a warp has ROWS / 8 rows' scores: one without any rows goes on to
            // the values (of 64 rows it has the same rows there, and none)
            const bool live = ROWS / 8 * (tid >> 5) < n_rows;
            if (!C::kFew && !live) {
                __syncthreads();
                __syncthreads();
                continue;
            }
            if (live) {
                // scores: this thread's row, keys spos + TPR i
                F2 dot[KPT];
#pragma unroll
                for (int i = 0; i < KPT; ++i) dot[i] = f2(0.f);
#pragma unroll 4
                for (int c = 0; c < DP; c += 4) {
                    const float4 x = load4(qs + srow * C::kLdQ + c);
                    const F2 x0 = f2(x.x, x.y), x1 = f2(x.z, x.w);
#pragma unroll
                    for (int i = 0; i < KPT; ++i) {
                        const float4 y = load4(key_at(stage, 0, spos + TPR * i) + c);
                        dot[i] = fma2(x0, f2(y.x, y.y), dot[i]);
                        dot[i] = fma2(x1, f2(y.z, y.w), dot[i]);
                    }
                }
                float s[KPT];
#pragma unroll
                for (int i = 0; i < KPT; ++i) s[i] = both(dot[i]);
                float mx = m;
#pragma unroll
                for (int i = 0; i < KPT; ++i) {
                    s[i] = j * kKeys + spos + TPR * i < limit ? s[i] : -INFINITY;
                    mx = fmaxf(mx, s[i]);
                }
#pragma unroll
                for (int o = TPR / 2; o > 0; o >>= 1)
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                // exponents as one product and difference: what rounds is the
                // difference, not the score; a row without keys so far refers to 0
                const float before = base;
                base = mx == -INFINITY ? 0.f : -mx * a.scale_log2;
                const float f = m == -INFINITY ? 0.f : exp2f(base - before);
                m = mx;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < KPT; ++i) {
                    const float p = exp2f(fmaf(s[i], a.scale_log2, base));
                    sum += p;
                    ps[(spos + TPR * i) * C::kLdP + srow] = p;
                }
                l = fmaf(l, f, sum);
                if (spos == 0) alpha[srow] = f;
            }
            __syncthreads();
            if (!C::kFew || group < C::kGroups) {
                // a block's sum is taken by itself and then added, so that a long
                // axis is a sum of short ones
                F2 blk[RPT][2 * NQ];
#pragma unroll
                for (int i = 0; i < RPT; ++i)
#pragma unroll
                    for (int c = 0; c < 2 * NQ; ++c) blk[i][c] = f2(0.f);
#pragma unroll 2
                for (int key = group; key < kKeys; key += C::kGroups) {
                    F2 p[RPT];
#pragma unroll
                    for (int i = 0; i < RPT; i += 4) {
                        const float4 x = load4(ps + key * C::kLdP + row0 + i);
                        p[i] = f2(x.x);
                        p[i + 1] = f2(x.y);
                        p[i + 2] = f2(x.z);
                        p[i + 3] = f2(x.w);
                    }
#pragma unroll
                    for (int d = 0; d < NQ; ++d) {
                        const float4 y = load4(key_at(stage, 1, key) + 4 * quad + 64 * d);
                        const F2 y0 = f2(y.x, y.y), y1 = f2(y.z, y.w);
#pragma unroll
                        for (int i = 0; i < RPT; ++i) {
                            blk[i][2 * d] = fma2(p[i], y0, blk[i][2 * d]);
                            blk[i][2 * d + 1] = fma2(p[i], y1, blk[i][2 * d + 1]);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < RPT; ++i) {
                    const F2 g = f2(alpha[row0 + i]);
#pragma unroll
                    for (int c = 0; c < 2 * NQ; ++c) acc[i][c] = fma2(acc[i][c], g, blk[i][c]);
                }
            }
            __syncthreads();                     // the stage is free for the block after next
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (spos == 0) {
            denom[srow] = l;
            top[srow] = m * a.scale_log2;        // in log2 units, -inf without keys
        }
        if constexpr (C::kFew) {                 // the groups' sums, through the ring
            float *join = reinterpret_cast<float *>(ring);
            if (group < C::kGroups)
#pragma unroll
                for (int i = 0; i < RPT; ++i) {
                    const float2 lo = split(acc[i][0]), hi = split(acc[i][1]);
                    *reinterpret_cast<float4 *>(join + (group * ROWS + row0 + i) * DP + 4 * quad) =
                        make_float4(lo.x, lo.y, hi.x, hi.y);
                }
        }
        __syncthreads();
        if (wk.part != kPartNone && tid == 0)
            desc[wk.slot] = make_int4(wk.part, wk.tok0, wk.n_tok, wk.h);
        auto write = [&](int row, int col, float4 x) {
            if (wk.part != kPartNone) {
                const int64_t rec = ((int64_t)blockIdx.x * 2 + wk.slot) * a.rows + row;
                *reinterpret_cast<float4 *>(a.part_o + rec * DP + col) = x;
                if (col == 0) a.part_ml[rec] = make_float2(top[row], denom[row]);
                return;
            }
            const int64_t head = (int64_t)(wk.tok0 + row / a.group) * a.q_heads +
                                 wk.h * a.group + row % a.group;
            const bool none = denom[row] == 0.f;
            const float r = none ? 0.f : 1.f / denom[row];
            T *o = static_cast<T *>(a.out) + head * a.D + col;
            if (col < a.D) {                     // widths are multiples of 8
                o[0] = from_f<T>(none ? 0.f : x.x * r);
                o[1] = from_f<T>(none ? 0.f : x.y * r);
                o[2] = from_f<T>(none ? 0.f : x.z * r);
                o[3] = from_f<T>(none ? 0.f : x.w * r);
            }
            if (a.lse && col == 0)
                a.lse[head] = none ? -INFINITY : (top[row] + log2f(denom[row])) / kLog2e;
        };
        if constexpr (C::kFew) {
            const float *join = reinterpret_cast<const float *>(ring);
            for (int i = tid; i < n_rows * C::kQuads; i += kThreads) {
                const int row = i / C::kQuads, col = 4 * (i - row * C::kQuads);
                float4 x = load4(join + row * DP + col);
#pragma unroll
                for (int g = 1; g < C::kGroups; ++g) {
                    const float4 y = load4(join + (g * ROWS + row) * DP + col);
                    x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
                }
                write(row, col, x);
            }
        } else {
#pragma unroll
            for (int i = 0; i < RPT; ++i)
#pragma unroll
                for (int d = 0; d < NQ; ++d)
                    if (row0 + i < n_rows) {
                        const float2 lo = split(acc[i][2 * d]), hi = split(acc[i][2 * d + 1]);
                        write(row0 + i, 4 * quad + 64 * d, make_float4(lo.x, lo.y, hi.x, hi.y));
                    }
        }
    }
}

// ---- join of split tiles ----------------------------------------------------
// Weights 2^(m_i - max m) over the shares' partials of a tile, added in a
// fixed order, so the result does not depend on which share finished first.
// The work is a chain of dependent loads (records, statistics, outputs), so
// each step is one round of loads.
//
// Up to 16 rows a tile (single tokens: one request of 131072 keys leaves 76
// partials of 4 rows): block (c, y) takes row y of the tile that begins in
// share c, its 8 warps split the partials (10 us; by one warp 82).  Taller
// tiles: every block lists the split tiles and takes its part of all (tile,
// rows) units, a warp one row or four.  One row where tiles are few and
// their partials many, so that a row's loads over the partials fill the
// flight (29 and 64 tokens over 48 k and 65 k keys: 33 and 54 us with the
// attention, four rows 77 and 76); four rows where most tiles have two or
// three partials (4 prompts of 4096, 213 us with the attention, and 8 ragged
// chunks, 280: 7 and 8 us less than with one row).
struct Span {
    int slot, n;                // place of the first partial, shares of the tile
    int tok0, n_rows, h;
};

// The tile that begins in share c, the same for the whole block; false
// without one.  kind[i]: what share c + i holds of it (n values, shared).
__device__ __forceinline__ bool find_span(const AttnArgs &a, int c, int ctas, int *kind,
                                          int *last, Span *s) {
    int4 d = a.part_desc[2 * c];
    s->slot = 0;
    if (threadIdx.x == 0) *last = ctas - 1;
    for (int i = c + 1 + (int)threadIdx.x; i < ctas; i += blockDim.x)
        kind[i - c] = a.part_desc[2 * i].x;
    if (d.x != kPartFirst) {
        d = a.part_desc[2 * c + 1];
        s->slot = 1;
    }
    if (d.x != kPartFirst) return false;
    s->tok0 = d.y;
    s->n_rows = d.z * a.group;
    s->h = d.w;
    __syncthreads();
    for (int i = 1 + (int)threadIdx.x; i < ctas - c; i += blockDim.x)
        if (kind[i] == kPartLast) {
            atomicMin(last, c + i);
            break;
        }
    if (threadIdx.x == 0) kind[0] = kPartFirst;
    __syncthreads();
    s->n = *last - c + 1;
    return true;
}
__device__ __forceinline__ int64_t record_of(const AttnArgs &a, const Span &s, int c, int i,
                                             int row) {
    return ((int64_t)2 * (c + i) + (i ? 0 : s.slot)) * a.rows + row;
}
__device__ __forceinline__ int64_t head_of(const AttnArgs &a, const Span &s, int row) {
    return (int64_t)(s.tok0 + row / a.group) * a.q_heads + s.h * a.group + row % a.group;
}
__device__ __forceinline__ float lse_of(float m, float sum) {   // m in log2 units
    return sum == 0.f ? -INFINITY : (m + log2f(sum)) / kLog2e;
}

template <typename T, int DP>
__global__ void __launch_bounds__(256) join_row_kernel(AttnArgs a, int ctas) {
    constexpr int kC = DP / 32;
    extern __shared__ int shared[];
    int *kind = shared;
    float *weight = reinterpret_cast<float *>(shared + ctas);
    __shared__ int last;
    __shared__ float warp_max[8], warp_sum[8], part[8][DP];
    pdl_wait();
    const int c = blockIdx.x, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    Span s;
    if (!find_span(a, c, ctas, kind, &last, &s)) return;
    for (int row = blockIdx.y; row < s.n_rows; row += gridDim.y) {
        float m = -INFINITY;
        float2 ml[2];                        // up to 512 shares
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = tid + 256 * k;
            ml[k] = make_float2(-INFINITY, 0.f);
            if (i < s.n && kind[i] != kPartNone) ml[k] = a.part_ml[record_of(a, s, c, i, row)];
            m = fmaxf(m, ml[k].x);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (lane == 0) warp_max[w] = m;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, warp_max[k]);
        const float base = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = tid + 256 * k;
            const float f = exp2f(ml[k].x - base);
            if (i < s.n) weight[i] = f;      // 0 for a share without a block of this tile
            sum = fmaf(f, ml[k].y, sum);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) warp_sum[w] = sum;
        __syncthreads();
        float acc[kC];
#pragma unroll
        for (int k = 0; k < kC; ++k) acc[k] = 0.f;
#pragma unroll 8
        for (int i = w; i < s.n; i += 8) {
            const float f = weight[i];
            if (f == 0.f) continue;          // an absent partial holds anything
            const float *o = a.part_o + record_of(a, s, c, i, row) * DP + lane;
#pragma unroll
            for (int k = 0; k < kC; ++k) acc[k] = fmaf(f, o[32 * k], acc[k]);
        }
#pragma unroll
        for (int k = 0; k < kC; ++k) part[w][lane + 32 * k] = acc[k];
        __syncthreads();
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += warp_sum[k];
        const int64_t head = head_of(a, s, row);
        if (tid < a.D) {
            float x = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) x += part[k][tid];
            static_cast<T *>(a.out)[head * a.D + tid] = from_f<T>(sum == 0.f ? 0.f : x / sum);
        }
        if (a.lse && tid == 0) a.lse[head] = lse_of(m, sum);
        __syncthreads();                     // the next row reuses the shared arrays
    }
}

// A place of join_rows_kernel's list of split tiles.
struct Split {
    int4 desc;                  // of the tile's first partial
    int first, slot, last;      // its share and place, the tile's last share
    int pad;
};

// RW: rows a warp takes at a time.
template <typename T, int DP, int RW>
__global__ void __launch_bounds__(256, DP > 128 ? 2 : 3)
    join_rows_kernel(AttnArgs a, int ctas, int groups) {
    constexpr int V = DP % 128 == 0 ? 4 : 2, kN = DP / (32 * V);   // a lane's columns: kN runs of V
    constexpr int kRows = 8 * RW, kSub = 32 / RW;
    using W = std::conditional_t<V == 4, float4, float2>;
    extern __shared__ __align__(16) char joined[];
    Split *split = reinterpret_cast<Split *>(joined);
    int *kind = reinterpret_cast<int *>(split + ctas);
    __shared__ int2 count[8];
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    // the split tiles in order: tiles follow one another on the axis, so the
    // k-th first partial and the k-th last one are of the same tile
    int n_first = 0, n_last = 0;
    for (int c0 = 0; c0 < ctas; c0 += 256) {
        const int c = c0 + tid;
        int4 d0 = make_int4(kPartNone, 0, 0, 0), d1 = d0;
        if (c < ctas) {
            d0 = a.part_desc[2 * c];
            d1 = a.part_desc[2 * c + 1];
            kind[c] = d0.x;
        }
        const bool is_first = d0.x == kPartFirst || d1.x == kPartFirst, is_last = d0.x == kPartLast;
        const unsigned f = __ballot_sync(0xffffffffu, is_first);
        const unsigned l = __ballot_sync(0xffffffffu, is_last);
        if (lane == 0) count[w] = make_int2(__popc(f), __popc(l));
        __syncthreads();
        const unsigned below = (1u << lane) - 1;
        int kf = n_first + __popc(f & below), kl = n_last + __popc(l & below);
        for (int i = 0; i < 8; ++i) {
            const int2 x = count[i];
            if (i < w) {
                kf += x.x;
                kl += x.y;
            }
            n_first += x.x;
            n_last += x.y;
        }
        if (is_first) {
            const int slot = d0.x == kPartFirst ? 0 : 1;
            split[kf].desc = slot ? d1 : d0;
            split[kf].first = c;
            split[kf].slot = slot;
        }
        if (is_last) split[kl].last = c;
        __syncthreads();
    }
    for (int unit = blockIdx.x; unit < n_first * groups; unit += gridDim.x) {
        const Split &p = split[unit / groups];
        const int c = p.first, n_rows = p.desc.z * a.group;
        const int n = (unit / groups < n_last ? p.last : ctas - 1) - c + 1;
        const Span s = {p.slot, n, p.desc.y, n_rows, p.desc.w};
        for (int row0 = unit % groups * kRows + w * RW; row0 < n_rows; row0 += groups * kRows) {
            // lane (sub, r): partials sub, sub + kSub .. of row row0 + r
            const int mine = row0 + lane % RW, sub = lane / RW;
            auto stat = [&](int i) {
                float2 ml = make_float2(-INFINITY, 0.f);   // without a block of this tile
                if (i < n && mine < n_rows && (i == 0 || kind[c + i] != kPartNone))
                    ml = a.part_ml[record_of(a, s, c, i, mine)];
                return ml;
            };
            const float2 head = stat(sub);
            float m = head.x, sum = 0.f;
            for (int i = sub + kSub; i < n; i += kSub) m = fmaxf(m, stat(i).x);
#pragma unroll
            for (int o = 16; o >= RW; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float base = m == -INFINITY ? 0.f : m;
            float acc[RW][kN][V];
#pragma unroll
            for (int r = 0; r < RW; ++r)
#pragma unroll
                for (int k = 0; k < kN; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[r][k][e] = 0.f;
            for (int i0 = 0; i0 < n; i0 += kSub) {
                const float2 ml = i0 ? stat(i0 + sub) : head;
                const float weight = exp2f(ml.x - base);
                sum = fmaf(weight, ml.y, sum);
                const int left = min(kSub, n - i0);
#pragma unroll(8 / RW)
                for (int i = 0; i < left; ++i)
#pragma unroll
                    for (int r = 0; r < RW; ++r) {
                        const float f = __shfl_sync(0xffffffffu, weight, i * RW + r);
                        if (row0 + r >= n_rows) continue;
                        const int64_t rec = record_of(a, s, c, i0 + i, row0 + r);
                        const W *o = reinterpret_cast<const W *>(a.part_o + rec * DP) + lane;
#pragma unroll
                        for (int k = 0; k < kN; ++k) {
                            const W x = o[32 * k];
                            const float *v = reinterpret_cast<const float *>(&x);
#pragma unroll
                            for (int e = 0; e < V; ++e) {   // an absent partial holds anything
                                const float y = fmaf(f, v[e], acc[r][k][e]);
                                acc[r][k][e] = f == 0.f ? acc[r][k][e] : y;
                            }
                        }
                    }
            }
#pragma unroll
            for (int o = 16; o >= RW; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (a.lse && sub == 0 && mine < n_rows) a.lse[head_of(a, s, mine)] = lse_of(m, sum);
            const float inverse = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const float x = __shfl_sync(0xffffffffu, inverse, r);
                if (row0 + r >= n_rows) continue;
                T *o = static_cast<T *>(a.out) + head_of(a, s, row0 + r) * a.D;
#pragma unroll
                for (int k = 0; k < kN; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int col = 32 * V * k + V * lane + e;
                        if (col < a.D) o[col] = from_f<T>(acc[r][k][e] * x);
                    }
            }
        }
    }
}

template <typename T, int DP, int RW>
cudaError_t join_rows(const AttnArgs &a, int ctas, int rows, bool pdl, cudaStream_t st) {
    const int groups = (rows + 8 * RW - 1) / (8 * RW);
    const int most = device_sm_count() * (RW == 1 ? 8 : 4), units = ctas * groups;
    return launch_kernel(pdl, join_rows_kernel<T, DP, RW>, dim3(units < most ? units : most), 256,
                         (size_t)ctas * (sizeof(Split) + 4), st, a, ctas, groups);
}

// max_new and the batch bound the number of tiles: a few tiles on all CTAs
// leave many partials each.
template <typename T, int DP>
cudaError_t combine_dim(const AttnArgs &a, int ctas, int max_new, bool pdl, cudaStream_t st) {
    // blocks for the rows that the caller's bound announces; a block goes on
    // to further rows where there are more
    const int rows = a.rows < a.rows_hint ? a.rows : a.rows_hint;
    if (rows <= 16)
        return launch_kernel(pdl, join_row_kernel<T, DP>, dim3(ctas, rows), 256, (size_t)8 * ctas,
                             st, a, ctas);
    const int64_t of_max = (int64_t)a.n_seqs * ((max_new + (int64_t)a.tq - 1) / a.tq);
    const int64_t of_all = (int64_t)a.n_seqs + a.n_tokens / a.tq;
    const int64_t tiles = (of_max < of_all ? of_max : of_all) * a.kv_heads;
    return 2 * tiles <= ctas ? join_rows<T, DP, 1>(a, ctas, rows, pdl, st)
                             : join_rows<T, DP, 4>(a, ctas, rows, pdl, st);
}

template <typename T> cudaError_t combine(const AttnArgs &a, int ctas, int dp, int max_new,
                                          bool pdl, cudaStream_t st) {
    switch (dp) {
    case 64: return combine_dim<T, 64>(a, ctas, max_new, pdl, st);
    case 128: return combine_dim<T, 128>(a, ctas, max_new, pdl, st);
    case 192: return combine_dim<T, 192>(a, ctas, max_new, pdl, st);
    default: return combine_dim<T, 256>(a, ctas, max_new, pdl, st);
    }
}

template <typename T, int ROWS, int ND> cudaError_t rows_go(const AttnArgs &a, int ctas,
                                                            cudaStream_t st) {
    constexpr size_t smem = RowsCfg<T, ROWS, ND>::kSmem;
    const cudaError_t e = allow_dynamic_smem<rows_kernel<T, ROWS, ND>>(smem);
    if (e != cudaSuccess) return e;
    rows_kernel<T, ROWS, ND><<<ctas, kThreads, smem, st>>>(a);
    return cudaGetLastError();
}

// Calls f with the kernel's types for a storage type, tile height and width.
struct RowsPlan {
    int per_sm, keys;
};
template <typename F> auto rows_variant(int32_t dtype, int rows, int dim, F &&f) {
    auto width = [&](auto t, auto r) {
        using T = decltype(t);
        constexpr int R = decltype(r)::value;
        switch ((dim + 63) / 64) {
        case 1: return f(RowsCfg<T, R, 1>(), t, r, std::integral_constant<int, 1>());
        case 2: return f(RowsCfg<T, R, 2>(), t, r, std::integral_constant<int, 2>());
        case 3: return f(RowsCfg<T, R, 3>(), t, r, std::integral_constant<int, 3>());
        default: return f(RowsCfg<T, R, 4>(), t, r, std::integral_constant<int, 4>());
        }
    };
    auto height = [&](auto t) {
        if (rows <= 8) return width(t, std::integral_constant<int, 8>());
        if (rows <= 16) return width(t, std::integral_constant<int, 16>());
        return width(t, std::integral_constant<int, 64>());
    };
    return dtype == ULTRAMEM_BF16 ? height(__nv_bfloat16()) : height(float());
}
RowsPlan rows_plan(int32_t dtype, int rows, int dim) {
    return rows_variant(dtype, rows, dim, [](auto cfg, auto, auto, auto) {
        return RowsPlan{decltype(cfg)::kPerSm, decltype(cfg)::kKeys};
    });
}
cudaError_t launch_rows(const AttnArgs &a, int32_t dtype, int ctas, cudaStream_t st) {
    return rows_variant(dtype, a.rows, a.D, [&](auto, auto t, auto r, auto nd) {
        return rows_go<decltype(t), decltype(r)::value, decltype(nd)::value>(a, ctas, st);
    });
}

// ---- the call's plan --------------------------------------------------------

// Which kernel serves a call.  The tensor-core kernels take bf16 heads up to
// 128 wide; a call of at most 16 rows a request and key/value head reads each
// key for those rows alone and goes to the decode kernel (M = 16), any other
// to the 2 x 128-row kernel.  Everything else runs on the CUDA cores.
enum Path { kRows, kDecode, kPrefill };

Path path_of(int32_t dtype, int32_t q_heads, int32_t kv_heads, int32_t dim, int32_t max_new,
             bool tensor) {
    const bool few = (int64_t)max_new * (q_heads / kv_heads) <= 16;
    if (dtype == ULTRAMEM_BF16 && dim <= 128 && tensor) return few ? kDecode : kPrefill;
    return kRows;
}

struct Layout {
    int ctas, rows, tq, dp, extra;
    int64_t o, ml, desc, total;     // byte offsets in the workspace
};

Layout layout_of(Path path, int32_t dtype, int32_t group, int32_t dim, int32_t max_new) {
    Layout l = {};
    const int sms = device_sm_count();
    l.dp = (dim + 63) / 64 * 64;
    if (path == kPrefill) {
        l.ctas = sms;
        l.tq = 2 * (128 / group);
        l.rows = l.tq * group;
        // what reading the queries and writing the output of a tile measured,
        // in the time of so many keys
        l.extra = l.dp == 128 ? 384 : 256;
    } else if (path == kDecode) {
        l.ctas = 2 * sms;
        l.rows = 16;
        l.extra = 64;
    } else {
        const int64_t rows = (int64_t)max_new * group;
        l.rows = rows <= 8 ? 8 : rows <= 16 ? 16 : 64;
        const RowsPlan p = rows_plan(dtype, l.rows, dim);
        l.ctas = p.per_sm * sms;
        l.extra = p.keys;
    }
    if (path != kPrefill) l.tq = l.rows / group;
    // what the join kernels hold: join_row_kernel two shares a thread (512),
    // join_rows_kernel 36 bytes of shared memory a share (17 KB)
    if (l.ctas > 480) l.ctas = 480;
    l.o = 0;
    l.ml = l.o + (int64_t)l.ctas * 2 * l.rows * l.dp * 4;
    l.desc = (l.ml + (int64_t)l.ctas * 2 * l.rows * 8 + 15) & ~15ll;
    l.total = l.desc + (int64_t)l.ctas * 2 * 16 + 128;   // and room to align the start to 128
    return l;
}

// Set by a kernel whose bounded wait gave up; read and cleared by
// ultramem_paged_check.  Each device has its own.
__device__ int g_error;
__device__ int g_taken;         // what the check at hand read; checks take turns
std::mutex g_check;

template <int &SYMBOL> int *word_of() {
    static PerDevice<int *> word;
    int *p = nullptr;
    const cudaError_t e = word.get(&p, [](int, int **at) {
        void *a = nullptr;
        const cudaError_t found = cudaGetSymbolAddress(&a, SYMBOL);
        *at = static_cast<int *>(a);
        return found;
    });
    if (e == cudaSuccess) return p;
    cudaGetLastError();
    return nullptr;
}
// Reads and clears the word in one step: a timeout that a kernel of another
// stream records meanwhile is in this answer or in the next one.
__global__ void take_error_kernel(int *word, int *taken) { *taken = atomicExch(word, 0); }

__global__ void probe_kernel(int *err) {
    __shared__ uint64_t never;
    tc::probe_timeout(&never, err, kErrTimeout);
}

int shift_of(int32_t page_size) {
    int s = 0;
    while ((1 << s) < page_size) ++s;
    return s;
}

bool page_size_ok(int32_t p) { return p >= 16 && p <= 256 && (p & (p - 1)) == 0; }

bool cache_ok(const ultramem_kv_cache *c) {
    return c && c->k && c->v && c->n_pages > 0 && c->kv_heads > 0 && c->kv_heads <= 1024 &&
           c->head_dim > 0 && c->head_dim <= kMaxHeadDim && c->head_dim % 8 == 0 &&
           page_size_ok(c->page_size) &&
           (c->dtype == ULTRAMEM_F32 || c->dtype == ULTRAMEM_BF16) &&
           ((uintptr_t)c->k & 15) == 0 && ((uintptr_t)c->v & 15) == 0 &&
           (int64_t)c->n_pages * c->page_size <= INT32_MAX &&
           (int64_t)c->n_pages * c->kv_heads <= INT32_MAX;
}

bool heads_ok(int32_t dtype, int32_t q_heads, int32_t kv_heads, int32_t dim, int32_t max_new) {
    return (dtype == ULTRAMEM_F32 || dtype == ULTRAMEM_BF16) && kv_heads > 0 && kv_heads <= 1024 &&
           q_heads > 0 && q_heads % kv_heads == 0 && q_heads / kv_heads <= 64 && dim > 0 &&
           dim <= kMaxHeadDim && dim % 8 == 0 && max_new >= 0;
}

Memory ints(const int32_t *p, int64_t n) { return {p, n * (int64_t)sizeof(int32_t)}; }

}  // namespace

int *error_word() { return word_of<g_error>(); }

// A map of 64-column boxes over a bf16 tensor [outer][mid][inner] with the
// given strides in elements; zeros outside.
bool encode(CUtensorMap *map, const void *base, uint64_t inner, uint64_t mid, uint64_t outer,
            uint64_t mid_stride, uint64_t outer_stride, uint32_t box_mid, uint32_t box_outer) {
    using Fn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                            const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                            const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<Fn> known{nullptr};   // the driver's, the same for every device
    Fn fn = known.load();
    if (!fn) {
        cudaDriverEntryPointQueryResult q;
        void *f = nullptr;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000,
                                             cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess || !f) {
            cudaGetLastError();
            return false;
        }
        fn = reinterpret_cast<Fn>(f);
        known.store(fn);
    }
    const cuuint64_t dims[3] = {inner, mid, outer};
    const cuuint64_t strides[2] = {mid_stride * 2, outer_stride * 2};
    const cuuint32_t box[3] = {64, box_mid, box_outer}, step[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides,
              box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
           CUDA_SUCCESS;
}

cudaError_t launch_combine(const AttnArgs &a, int ctas, int dp, int dtype, int max_new, bool pdl,
                           cudaStream_t st) {
    return dtype == ULTRAMEM_BF16 ? combine<__nv_bfloat16>(a, ctas, dp, max_new, pdl, st)
                                  : combine<float>(a, ctas, dp, max_new, pdl, st);
}

}  // namespace paged
}  // namespace um

using namespace um::paged;

extern "C" ultramem_status ultramem_paged_plan(const int32_t *ctx_lens, const int32_t *new_lens,
                                               int32_t n_seqs, int32_t page_size,
                                               int32_t *block_table, int32_t table_width,
                                               const int32_t *free_pages,
                                               const int32_t *free_count, int32_t n_free,
                                               int32_t n_tokens, int32_t *q_start,
                                               int32_t *kv_lens, int32_t *slots,
                                               int32_t *free_left, int32_t *balance,
                                               void *stream) {
    if (n_seqs < 0 || n_tokens < 0 || table_width < 0 || n_free < 0 ||
        !page_size_ok(page_size) || !free_count || !q_start || !balance)
        return ULTRAMEM_EINVAL;
    if (n_seqs > 0 && (!ctx_lens || !new_lens || !kv_lens || (table_width > 0 && !block_table)))
        return ULTRAMEM_EINVAL;
    if ((n_tokens > 0 && !slots) || (n_free > 0 && !free_pages)) return ULTRAMEM_EINVAL;
    if (!um::apart({ints(q_start, (int64_t)n_seqs + 1), ints(kv_lens, n_seqs),
                    ints(slots, n_tokens), ints(free_left, 1), ints(balance, 1),
                    ints(block_table, (int64_t)n_seqs * table_width)},
                   {ints(ctx_lens, n_seqs), ints(new_lens, n_seqs), ints(free_pages, n_free),
                    ints(free_count, 1)}))
        return ULTRAMEM_EINVAL;
    PlanArgs a = {ctx_lens, new_lens,  free_pages, free_count, block_table,
                  q_start,  kv_lens,   slots,      free_left,  balance,
                  n_seqs,   n_tokens,  shift_of(page_size),    table_width, n_free};
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    // more than 256 requests: wider blocks, so that no thread walks many
    const int threads = n_seqs <= 256 ? 256 : 1024;
    int64_t grid = ((int64_t)n_tokens + threads - 1) / threads;
    const int64_t most = um::device_sm_count();
    grid = grid < 1 ? 1 : grid > most ? most : grid;
    if (threads == 256)
        plan_kernel<256><<<(unsigned)grid, 256, 0, st>>>(a);
    else
        plan_kernel<1024><<<(unsigned)grid, 1024, 0, st>>>(a);
    return um::status_from_cuda(cudaGetLastError());
}

extern "C" ultramem_status ultramem_paged_append(const ultramem_kv_cache *c, const void *k,
                                                 int64_t k_stride, const void *v, int64_t v_stride,
                                                 const int32_t *slots, int32_t n_tokens,
                                                 void *stream) {
    if (!cache_ok(c) || n_tokens < 0) return ULTRAMEM_EINVAL;
    if (n_tokens == 0) return ULTRAMEM_OK;
    const int row = c->kv_heads * c->head_dim;
    if (!k || !v || !slots || k_stride < row || v_stride < row) return ULTRAMEM_EINVAL;
    const int es = c->dtype == ULTRAMEM_BF16 ? 2 : 4;
    if (((uintptr_t)k | (uintptr_t)v) % es) return ULTRAMEM_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    const int shift = shift_of(c->page_size);
    const int64_t n_slots = (int64_t)c->n_pages << shift;
    const bool wide = (((uintptr_t)k | (uintptr_t)v) & 15) == 0 && k_stride * es % 16 == 0 &&
                      v_stride * es % 16 == 0;
    const int per = wide ? 16 / es : 1;
    const int64_t total = (int64_t)n_tokens * (row / per);
    const int64_t most = (int64_t)um::device_sm_count() * 64;
    const int64_t blocks = (total + 255) / 256;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    const int words = c->head_dim / per;
    if (wide)
        append_kernel<uint4><<<grid, 256, 0, st>>>(
            static_cast<const uint4 *>(k), static_cast<const uint4 *>(v), k_stride / per,
            v_stride / per, slots, static_cast<uint4 *>(c->k), static_cast<uint4 *>(c->v),
            n_tokens, c->kv_heads, words, shift, n_slots);
    else if (es == 2)
        append_kernel<uint16_t><<<grid, 256, 0, st>>>(
            static_cast<const uint16_t *>(k), static_cast<const uint16_t *>(v), k_stride, v_stride,
            slots, static_cast<uint16_t *>(c->k), static_cast<uint16_t *>(c->v), n_tokens,
            c->kv_heads, words, shift, n_slots);
    else
        append_kernel<uint32_t><<<grid, 256, 0, st>>>(
            static_cast<const uint32_t *>(k), static_cast<const uint32_t *>(v), k_stride, v_stride,
            slots, static_cast<uint32_t *>(c->k), static_cast<uint32_t *>(c->v), n_tokens,
            c->kv_heads, words, shift, n_slots);
    return um::status_from_cuda(cudaGetLastError());
}

extern "C" int64_t ultramem_paged_attention_workspace(int32_t dtype, int32_t q_heads,
                                                      int32_t kv_heads, int32_t head_dim,
                                                      int32_t max_new) {
    if (!heads_ok(dtype, q_heads, kv_heads, head_dim, max_new)) return 0;
    // the largest of the kernels that the call may take: a query or output that
    // is not aligned for the tensor-core ones goes to the CUDA cores
    int64_t most = 0;
    for (const bool tensor : {false, true}) {
        const Path p = path_of(dtype, q_heads, kv_heads, head_dim, max_new, tensor);
        const int64_t n = layout_of(p, dtype, q_heads / kv_heads, head_dim, max_new).total;
        most = n > most ? n : most;
    }
    return most;
}

extern "C" ultramem_status ultramem_paged_attention(
    const ultramem_kv_cache *c, const void *q, int64_t q_stride, int32_t q_heads,
    const int32_t *q_start, const int32_t *kv_lens, const int32_t *block_table,
    int32_t table_width, int32_t n_seqs, int32_t n_tokens, int32_t max_new, float scale, void *out,
    float *lse, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!cache_ok(c) || !heads_ok(c->dtype, q_heads, c->kv_heads, c->head_dim, max_new) ||
        n_seqs < 0 || n_tokens < 0 || table_width < 0 || !(scale > 0.f) || !(scale * kLog2e < INFINITY))
        return ULTRAMEM_EINVAL;
    if (n_tokens == 0 || n_seqs == 0 || max_new == 0) return ULTRAMEM_OK;
    const int es = c->dtype == ULTRAMEM_BF16 ? 2 : 4;
    if (!q || !q_start || !kv_lens || !out || q_stride < (int64_t)q_heads * c->head_dim ||
        (uintptr_t)q % es || (uintptr_t)out % es || (table_width > 0 && !block_table) ||
        !workspace || ((uintptr_t)workspace & 15))
        return ULTRAMEM_EINVAL;
    const int64_t need = ultramem_paged_attention_workspace(c->dtype, q_heads, c->kv_heads,
                                                            c->head_dim, max_new);
    if (workspace_bytes < need) return ULTRAMEM_EINVAL;
    // a token's head is written after its query was read: out may be q itself
    const int64_t row = (int64_t)q_heads * c->head_dim * es;
    const um::Memory mem_q = {q, row, n_tokens, q_stride * es}, mem_out = {out, row * n_tokens},
                     mem_lse = ints(reinterpret_cast<int32_t *>(lse), (int64_t)n_tokens * q_heads),
                     mem_ws = {workspace, need};
    if (!um::same_or_apart(mem_out, mem_q) || um::overlap(mem_lse, mem_q) ||
        um::overlap(mem_ws, mem_q) ||
        !um::apart({mem_out, mem_lse, mem_ws},
                   {ints(q_start, (int64_t)n_seqs + 1), ints(kv_lens, n_seqs),
                    ints(block_table, (int64_t)n_seqs * table_width)}))
        return ULTRAMEM_EINVAL;
    const int group = q_heads / c->kv_heads;
    // 4-byte fragments of q and out suffice for the decode kernel; TMA wants
    // rows of q on 16-byte boundaries
    const bool few = (int64_t)max_new * group <= 16;
    const int align = few ? 4 : 16;
    const bool tensor = ((uintptr_t)q | (uintptr_t)out) % align == 0 && q_stride * es % align == 0;
    const Path path = path_of(c->dtype, q_heads, c->kv_heads, c->head_dim, max_new, tensor);
    const Layout l = layout_of(path, c->dtype, group, c->head_dim, max_new);
    AttnArgs a = {};
    a.q = q;
    a.k = c->k;
    a.v = c->v;
    a.table = block_table;
    a.q_start = q_start;
    a.kv_lens = kv_lens;
    a.out = out;
    a.lse = lse;
    char *ws = reinterpret_cast<char *>(((uintptr_t)workspace + 127) & ~(uintptr_t)127);
    a.part_o = reinterpret_cast<float *>(ws + l.o);
    a.part_ml = reinterpret_cast<float2 *>(ws + l.ml);
    a.part_desc = reinterpret_cast<int4 *>(ws + l.desc);
    a.q_stride = q_stride;
    a.n_seqs = n_seqs;
    a.n_tokens = n_tokens;
    a.q_heads = q_heads;
    a.kv_heads = c->kv_heads;
    a.group = group;
    a.D = c->head_dim;
    a.page_shift = shift_of(c->page_size);
    a.table_width = table_width;
    a.n_pages = c->n_pages;
    a.rows = l.rows;
    a.tq = l.tq;
    a.extra = l.extra;
    a.rows_hint = (int)((int64_t)max_new * group < l.rows ? (int64_t)max_new * group : l.rows);
    a.scale_log2 = scale * kLog2e;
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    cudaError_t e = cudaSuccess;
    if (path == kDecode || path == kPrefill) {
        if (!(a.err = error_word())) return ULTRAMEM_ENODEV;
        CUtensorMap mq, mk, mv;
        const uint64_t D = c->head_dim, P = c->page_size;
        const uint64_t outer = (uint64_t)c->n_pages * c->kv_heads;
        const uint32_t box = path == kDecode ? decode_box_rows(c->page_size)
                                             : prefill_box_rows(c->page_size);
        if (!encode(&mk, c->k, D, P, outer, D, P * D, box, 1) ||
            !encode(&mv, c->v, D, P, outer, D, P * D, box, 1))
            return um::status_from_cuda(cudaErrorInvalidValue);
        if (path == kDecode) {
            e = launch_decode(a, mk, mv, l.ctas, st);
        } else {
            if (!encode(&mq, q, D, q_heads, n_tokens, D, q_stride, group, l.tq / 2))
                return um::status_from_cuda(cudaErrorInvalidValue);
            e = launch_prefill(a, mq, mk, mv, l.ctas, st);
        }
    } else {
        e = launch_rows(a, c->dtype, l.ctas, st);
    }
    // tables that hold no more keys than a tile keeps whole leave nothing to
    // join (a launch less: 3 us of a call of 10 to 20)
    const int64_t held = (int64_t)table_width << a.page_shift;
    if (e == cudaSuccess && held > whole_keys(a))
        e = launch_combine(a, l.ctas, l.dp, c->dtype, max_new, true, st);
    return um::status_from_cuda(e);
}

extern "C" ultramem_status ultramem_paged_check(void *stream) {
    int *word = error_word(), *taken = word_of<g_taken>();
    if (!word || !taken) return ULTRAMEM_ENODEV;
    int err = 0;
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    const std::lock_guard<std::mutex> turn(g_check);
    take_error_kernel<<<1, 1, 0, st>>>(word, taken);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) e = cudaMemcpyAsync(&err, taken, sizeof err, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return um::status_from_cuda(e);
    return err & um::kErrTimeout ? ULTRAMEM_ETIMEOUT : ULTRAMEM_OK;
}

extern "C" ultramem_status ultramem_debug_paged_probe(void *stream) {
    int *word = error_word();
    if (!word) return ULTRAMEM_ENODEV;
    cudaGetLastError();
    probe_kernel<<<1, 32, 0, (cudaStream_t)stream>>>(word);
    return um::status_from_cuda(cudaGetLastError());
}

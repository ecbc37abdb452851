// um_ce.cu -- the softmax cross entropy of hidden states against a vocabulary's
// output weights, without the logits in memory, and its gradient.
//
// Forward: z = x W^T in 256 x n tiles on pairs of SMs (um_pair_gemm.cuh); the
// epilogue leaves, for each token, the maximum and the sum of e^(z - maximum)
// over the tile's columns (and the label's logit, in the tile that has it),
// and a second kernel joins the tiles' pairs.
//
// Gradient: the logits again, in pieces of the vocabulary; a piece's
// G = scale dloss (e^(z - lse) - onehot) goes to the workspace in the storage
// type, and two products read it: dx = G W (summed over the pieces) and
// dw = G^T x (a piece's rows).  Bound by the tensor cores: 2 T V D operations
// a product.  16384 tokens x 32000 x 2048 bf16: 1170 us (1.84 PFLOP/s) and, with the
// gradient under the power cap, 4080 (1.58).
//
// Storage in fp32 enters the products as three bf16 terms a value, v = a + b + c
// with residues of 2^-9, 2^-17 and 2^-25 of |v|; the six products of terms that
// reach 2^-24 of the result are added, the smallest first.
#include "um_device.cuh"
#include "um_overlap.cuh"
#include "um_paged.cuh"
#include "um_pair.cuh"
#include "um_pair_gemm.cuh"
#include "um_planes.cuh"

#include <atomic>

namespace um {
namespace ce {
namespace {

constexpr int kMaxVocab = 1 << 30;
constexpr int kMaxDim = 65536;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// bytes of a piece's G, and of its weights where they are rearranged: large
// enough that a piece's products fill the GPU many times over, and a
// small part of its memory.  Tests set fewer (ultramem_debug_cross_entropy_piece).
constexpr int64_t kPieceBytes = 512ll << 20;
std::atomic<int64_t> g_piece_bytes{kPieceBytes};

struct Labels {
    const void *at;
    int wide, V;
    // the label of token t, or -1 for one that does not count
    __device__ __forceinline__ int operator()(int64_t t) const { return of(load(t)); }
    // the same in two steps: what a load gives, and what it says
    __device__ __forceinline__ int64_t load(int64_t t) const {
        return wide ? static_cast<const int64_t *>(at)[t]
                    : (int64_t) static_cast<const int32_t *>(at)[t];
    }
    __device__ __forceinline__ int of(int64_t l) const { return l >= 0 && l < V ? (int)l : -1; }
};

// The next of the bf16 terms that add up to v, and v less it.  A value that rounds
// to infinity is cut instead, and an infinity or NaN is its own first term.
__device__ __forceinline__ __nv_bfloat16 take_term(float &v) {
    __nv_bfloat16 b = __float2bfloat16_rn(v);
    if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) {
        v = 0.f;
        return b;
    }
    if (fabsf(__bfloat162float(b)) == INFINITY)
        b = __ushort_as_bfloat16((unsigned short)(__float_as_uint(v) >> 16));
    v -= __bfloat162float(b);
    return b;
}

// ---- operands as planes --------------------------------------------------------
// src [R][D] (rows ld apart) -> dst [planes][R][Dp], Dp = D rounded up to 64, so
// that rows start on 128 bytes, with zeros behind a row: fp32 values as three bf16
// terms, bf16 ones as they are, for operands that TMA cannot read well where they
// lie.  With `labels`, rows of tokens that do not count become zeros, so that
// weight 0 never meets what they hold.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256)
    planes_kernel(const T *src, int64_t ld, int64_t R, int D, int Dp, __nv_bfloat16 *dst,
                  Labels labels) {
    constexpr int P = sizeof(T) == 4 ? 3 : 1;
    pdl_wait();
    pdl_trigger();
    const int pieces = Dp / 8;
    const int64_t total = R * pieces, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += step) {
        const int64_t r = i / pieces;
        const int c = (int)(i - r * pieces) * 8;
        const bool counts = !labels.at || labels(r) >= 0;
        const Piece<T> from = counts ? read_piece(src + r * ld, c, D, ALIGNED) : Piece<T>{};
        if constexpr (P == 1) {
            *reinterpret_cast<uint4 *>(dst + r * Dp + c) = from.x[0];
            continue;
        }
        float v[8];
        memcpy(v, &from, sizeof v);
#pragma unroll
        for (int q = 0; q < P; ++q) {
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const __nv_bfloat162 b = {take_term(v[2 * k]), take_term(v[2 * k + 1])};
                o[k] = *reinterpret_cast<const uint32_t *>(&b);
            }
            *reinterpret_cast<uint4 *>(dst + ((int64_t)q * R + r) * Dp + c) =
                make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

// ---- forward -------------------------------------------------------------------

// Its results are fp32: past kLongSum entries a row the sums in the tensor cores
// are cut (lse of 2048 entries off by 6e-7 of its size, growing with the
// entries; in sums of 1024 by 4e-7, and 16384 x 32000 x 2048 in 1366 instead of 1314 us).
constexpr int kLongSum = 2048;
// what exponents are taken relative to: the maximum, or 0 beside an infinite one,
// whose differences would be NaN
__device__ __forceinline__ float shift_of(float top) {
    return fabsf(top) == INFINITY ? 0.f : top;
}
// what turns a difference of products (of the scale's sign) into one of exponents
__device__ __forceinline__ float log2_units(float scale_log2) {
    return scale_log2 == 0.f ? 1.f : fabsf(scale_log2);
}
template <int SUM> struct LseEpi {
    static constexpr int kSumBlocks = SUM;
    Labels labels;
    // Maxima and the label's product are kept as the products come (their sign
    // turned where the scale is negative, 0 where it is 0): differences of them
    // are then 0 or of one sign without an error, and so is the loss made of them.
    float2 *part;             // [half tiles][T]: maximum, sum of e^(|scale| (product - maximum))
    float *target;            // [T]: the label's product
    int T, vn, v0, tile0;     // columns of the piece, its first one, its first half tile
    int n_tile;
    float scale_log2;

    template <int N> LseEpi<N> cut() const {
        return {labels, part, target, T, vn, v0, tile0, n_tile, scale_log2};
    }
    __device__ __forceinline__ int64_t fetch(const pair::Tile &t, int row) const {
        const int64_t tok = t.m0 + row;
        return tok < T ? labels.load(tok) : -1;
    }
    template <class Sums, class Turn>
    __device__ __forceinline__ void operator()(const pair::Tile &t, int row, Sums &sums,
                                               int half, int c0, int c1, int64_t loaded,
                                               Turn &scratch) const {
        const int64_t tok = t.m0 + row;
        const int label = labels.of(loaded) - (v0 + t.n0);       // the tile's column
        const int cols = min(c1, vn - t.n0);
        const float by = log2_units(scale_log2);
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int i = 0; i < Sums::kChunks; ++i) {
            const int c = c0 + 32 * i;
            if (c >= cols) break;
            float place[32];
            float (&z)[32] = sums.get(i, place);
            if (scale_log2 <= 0.f) {
#pragma unroll
                for (int k = 0; k < 32; ++k) z[k] = scale_log2 < 0.f ? -z[k] : z[k] * 0.f;
            }
            if (label >= c && label < c + 32) {
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (label == c + k) target[tok] = z[k];
            }
            if (c + 32 > cols) {
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (c + k >= cols) z[k] = -INFINITY;
            }
            float top = fmaxf(z[0], z[1]);
#pragma unroll
            for (int k = 2; k < 32; k += 2) top = max3(top, z[k], z[k + 1]);
            top = fmaxf(m, top);
            const float shift = shift_of(top);
            const F2 f = f2(by), less = f2(-shift);
            F2 s[2] = {f2(0.f), f2(0.f)};
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
                const float2 y = split((f2(z[k], z[k + 1]) + less) * f);
                s[(k >> 1) & 1] = s[(k >> 1) & 1] + f2(tc::ex2(y.x), tc::ex2(y.y));
            }
            l = fmaf(l, tc::ex2((m - shift) * by), both(s[0] + s[1]));
            m = top;
        }
        if (tok < T)
            part[(int64_t)(tile0 + 2 * (t.n0 / n_tile) + half) * T + tok] = make_float2(m, l);
    }
};

// A block joins the tiles' pairs of 32 tokens, a warp every 32nd tile.  The largest
// product's term of the sum is exactly 1, so
//   loss = |scale| (maximum - label's product) + ln(sum)
// adds two values that are at least 0.  (As lse less the label's logit, each
// rounded for itself, it came out as low as -4e-6 where a label of logit 60 held
// nearly all the probability.  Exponents as differences times the scale instead of
// one multiply-add: 5563 tokens x 107918 x 128 in 251 instead of 247.5 us.)
__global__ void __launch_bounds__(1024)
    join_kernel(const float2 *part, const float *target, Labels labels, int T, int tiles,
                float scale, float scale_log2, float *loss, float *lse) {
    __shared__ float2 got[32][33];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const float by = log2_units(scale_log2);
    auto add = [by](float2 &a, float2 b) {
        const float top = fmaxf(a.x, b.x), shift = shift_of(top);
        a.y = a.y * tc::ex2((a.x - shift) * by) + b.y * tc::ex2((b.x - shift) * by);
        a.x = top;
    };
    for (int64_t t0 = (int64_t)blockIdx.x * 32; t0 < T; t0 += (int64_t)gridDim.x * 32) {
        float2 a = make_float2(-INFINITY, 0.f);
        if (t0 + lane < T)
            for (int i = w; i < tiles; i += 32) add(a, part[(int64_t)i * T + t0 + lane]);
        got[w][lane] = a;
        __syncthreads();
        const int64_t t = t0 + w;       // now a warp a token
        a = got[lane][w];
#pragma unroll
        for (int o = 16; o; o >>= 1)
            add(a, make_float2(__shfl_xor_sync(0xffffffffu, a.x, o),
                               __shfl_xor_sync(0xffffffffu, a.y, o)));
        if (lane == 0 && t < T) {
            const float size = fabsf(scale), rest = kLn2 * log2f(a.y);
            lse[t] = fmaf(size, a.x, rest);
            loss[t] = labels(t) >= 0 ? fmaf(size, a.x - target[t], rest) : 0.f;
        }
        __syncthreads();
    }
}

// ---- gradient ------------------------------------------------------------------

// 32 values to a row of T, on a 32-byte boundary
template <typename T> __device__ __forceinline__ void store32(T *to, const float (&v)[32]) {
#pragma unroll
    for (int k = 0; k < (int)sizeof(T); ++k) {
        uint32_t o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (sizeof(T) == 4) {
                o[j] = __float_as_uint(v[8 * k + j]);
            } else {
                const __nv_bfloat162 b =
                    __floats2bfloat162_rn(v[16 * k + 2 * j], v[16 * k + 2 * j + 1]);
                o[j] = *reinterpret_cast<const uint32_t *>(&b);
            }
        }
        tc::store_sector(to + 32 / sizeof(T) * k, o);
    }
}

// P planes of G [P][T][ld]; ld is a multiple of 32, and columns up to the next
// multiple of 32 past vn are written (as zeros).
template <int P> struct GradEpi {
    static constexpr int kSumBlocks = 0;
    Labels labels;
    const float *lse, *dloss;
    __nv_bfloat16 *g;
    int64_t ld;
    int T, vn, v0;
    float scale, scale_log2;

    struct Row {
        int64_t label;
        float dloss, lse;
    };
    __device__ __forceinline__ Row fetch(const pair::Tile &t, int row) const {
        const int64_t tok = t.m0 + row;
        if (tok >= T) return {-1, 0.f, 0.f};
        return {labels.load(tok), dloss[tok], lse[tok]};
    }
    template <class Sums, class Turn>
    __device__ __forceinline__ void operator()(const pair::Tile &t, int row, Sums &sums,
                                               int half, int c0, int c1, const Row &r,
                                               Turn &scratch) const {
        const int64_t tok = t.m0 + row;
        const bool live = tok < T;
        const int label = labels.of(r.label), at = label - (v0 + t.n0);
        const float d = label >= 0 ? r.dloss * scale : 0.f;
        const float shift = label >= 0 ? -r.lse * kLog2e : 0.f;
        const int cols = min(c1, vn - t.n0);
#pragma unroll
        for (int i = 0; i < Sums::kChunks; ++i) {
            const int c = c0 + 32 * i;
            if (c >= cols) break;
            float place[32];
            float (&z)[32] = sums.get(i, place);
            if (!live) continue;
#pragma unroll
            for (int k = 0; k < 32; ++k) z[k] = tc::ex2(fmaf(z[k], scale_log2, shift));
            if (at >= c && at < c + 32) {
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (at == c + k) z[k] -= 1.f;
            }
            if (label < 0 || c + 32 > cols) {
#pragma unroll
                for (int k = 0; k < 32; ++k) z[k] = label >= 0 && c + k < cols ? z[k] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < 32; ++k) z[k] *= d;
            __nv_bfloat16 *to = g + tok * ld + t.n0 + c;
#pragma unroll
            for (int q = 0; q < P; ++q) {
                store32(to + (int64_t)q * T * ld, z);
                if (q + 1 < P)
#pragma unroll
                    for (int k = 0; k < 32; ++k) z[k] -= __bfloat162float(__float2bfloat16_rn(z[k]));
            }
        }
    }
};

// A product's rows [M][N], with `add` on top of what part [splits][M][ld] (fp32,
// ld a multiple of 8) holds: to `out` in T, or without it back to part.  Where
// out's rows allow 32-byte stores (`wide`), each thread stores its row; else a
// warp turns 8 or 16 columns of its 32 rows at a time, so that lanes store
// neighbours (each thread along its row: gradient of 333 tokens against 5003 x
// 509 111 us, so 96).
template <typename T> struct StoreEpi {
    static constexpr int kSumBlocks = 0;
    T *out;
    float *part;
    int64_t M, N, ld;
    int add, wide;

    __device__ __forceinline__ int fetch(const pair::Tile &, int) const { return 0; }
    template <class Sums, class Turn>
    __device__ __forceinline__ void operator()(const pair::Tile &t, int row, Sums &sums,
                                               int half, int c0, int c1, int, Turn &scratch) const {
        const int64_t r = t.m0 + row;
        const int cols = (int)min((int64_t)c1, N - t.n0), lane = threadIdx.x & 31;
#pragma unroll
        for (int j = 0; j < Sums::kChunks; ++j) {
            const int c = c0 + 32 * j;
            if (c >= cols) break;
            float place[32];
            float (&x)[32] = sums.get(j, place);
            const int left = cols - c;
            if (r < M) {
                float *sum = part + ((int64_t)t.split * M + r) * ld + t.n0 + c;
                if (add) {
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        if (k >= left) break;            // rows are padded to 8
                        const float4 y = *reinterpret_cast<const float4 *>(sum + k);
                        x[k] += y.x, x[k + 1] += y.y, x[k + 2] += y.z, x[k + 3] += y.w;
                    }
                }
                if (!out) {
#pragma unroll
                    for (int k = 0; k < 32; k += 8) {
                        if (k >= left) break;
                        const uint32_t o[8] = {__float_as_uint(x[k]),     __float_as_uint(x[k + 1]),
                                               __float_as_uint(x[k + 2]), __float_as_uint(x[k + 3]),
                                               __float_as_uint(x[k + 4]), __float_as_uint(x[k + 5]),
                                               __float_as_uint(x[k + 6]), __float_as_uint(x[k + 7])};
                        tc::store_sector(sum + k, o);
                    }
                } else if (wide && left >= 32) {
                    store32(out + r * N + t.n0 + c, x);
                }
            }
            if (!out || (wide && left >= 32)) continue;
            const int64_t row0 = r - lane;
            constexpr int W = Turn::kCols, kRows = 32 / W;
#pragma unroll
            for (int h = 0; h < 32; h += W) {
                if (h >= left) break;
                __syncwarp();
#pragma unroll
                for (int k = 0; k < W; ++k) scratch.v[lane][k] = x[h + k];
                __syncwarp();
                const int k = lane % W;
#pragma unroll 8
                for (int i = lane / W; i < 32; i += kRows)
                    if (row0 + i < M && h + k < left)
                        out[(row0 + i) * N + t.n0 + c + h + k] = from_f<T>(scratch.v[i][k]);
            }
        }
    }
};

// out [M][N] = sum of part [splits][M][ld] over the splits, in order; four
// columns a thread
template <typename T>
__global__ void __launch_bounds__(256)
    sum_splits_kernel(const float *part, int splits, int64_t M, int N, int ld, T *out, int wide) {
    pdl_wait();
    pdl_trigger();
    const int pieces = ld / 4;
    const int64_t n = M * pieces, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += step) {
        const int64_t r = i / pieces;
        const int c = (int)(i - r * pieces) * 4;
        const float *from = part + r * ld + c;
        float4 s = *reinterpret_cast<const float4 *>(from);
#pragma unroll 4
        for (int k = 1; k < splits; ++k) {
            const float4 x = *reinterpret_cast<const float4 *>(from + k * M * ld);
            s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
        }
        T *to = out + r * N + c;
        if (!wide) {
            const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (c + k < N) to[k] = from_f<T>(v[k]);
        } else if constexpr (sizeof(T) == 4) {
            if (c < N) *reinterpret_cast<float4 *>(to) = s;
        } else if (c < N) {
            const __nv_bfloat162 b[2] = {__floats2bfloat162_rn(s.x, s.y),
                                         __floats2bfloat162_rn(s.z, s.w)};
            *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(b);
        }
    }
}

// ---- the calls' plans ------------------------------------------------------------

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t pad256(int64_t n) { return (n + 255) & ~255ll; }
int pairs_of_sms() {
    const int n = device_sm_count() / 2;
    return n < 1 ? 1 : n;
}
int planes_of(int32_t dtype) { return dtype == ULTRAMEM_F32 ? 3 : 1; }

// The product of [M][K] and [N][K]: tiles, and splits of K where there are
// fewer tiles than pairs of SMs.
// n_tile: the widest tile, unless narrower ones share out among the pairs more
// evenly; `step` 32, or 128 where the columns are MN-major (boxes of 64 columns a CTA).
// splits (at most `most`, 64 or fewer): as many as keep a sum below kMostSum terms in
// the tensor cores, and more by time: a tile's time is its k blocks (2 cycles a
// column, and no less than 480 for the copies: 128 columns took 615) and about 3000
// cycles; a split costs a pass over the output in fp32.
// kMostSum: the tensor cores cut off what a step of 16 terms loses in a sum's last
// place, less than 2^-23 of it; 65536 terms of one sign lose less than 2^-11, an
// eighth of half a step of bf16.  (fp32 storage adds its sums in fp32 after each k
// block.)
constexpr int64_t kMostSum = 65536;
pair::Plan plan_of(int64_t M, int64_t N, int64_t K, int planes, int step, int most) {
    pair::Plan p = {};
    const int64_t pairs = pairs_of_sms();
    p.m_tiles = (int)ceil_div(M, pair::kTileM);
    p.k_blocks = (int)ceil_div(K, 64);
    const int pairs_of_planes = planes == 3 ? 6 : 1;
    int least = planes == 3 ? 1 : (int)ceil_div(p.k_blocks, kMostSum / 64);
    if (least > 64) least = 64;
    if (most < least) most = least;
    double best = 0;
    const int widest = planes == 3 ? pair::Shape<true>::kMaxN : pair::Shape<false>::kMaxN;
    for (int n = widest; n >= 128; n -= step) {
        const int64_t nt = ceil_div(N, n);
        // a second share of a pair's time is the last that a split can save
        for (int s = least; s <= most && s <= p.k_blocks; ++s) {
            if (s > least && p.m_tiles * nt * (s - 1) >= 2 * pairs) break;
            const int64_t waves = ceil_div(p.m_tiles * nt * s, pairs);
            const double block = pairs_of_planes * 2.0 * n;
            const double tile =
                (double)ceil_div(p.k_blocks, s) * (block > 480. ? block : 480.) + 3000.0;
            // 2000 cycles and s writes and reads of the output at 3 KB a cycle
            const double join = s > 1 ? 2000.0 + (double)M * N * 8.0 * s / 3000.0 : 0.0;
            const double cost = waves * tile + join;
            if (best == 0 || cost < 0.97 * best) {
                best = cost;
                p.n_tile = n;
                p.n_tiles = (int)nt;
                p.splits = s;
            }
        }
    }
    p.group_m = 8;
    return p;
}

// rows x [K or columns]: K-major boxes of `rows` rows, or MN-major ones of 64 k
bool operand(CUtensorMap *map, const void *at, int64_t inner, int64_t rows, int64_t ld, int planes,
             int64_t plane, uint32_t box) {
    return paged::encode(map, at, inner, rows, planes, ld, plane, box, 1);
}

template <class Epi, bool A_MN, bool B_MN, bool EXACT>
cudaError_t multiply(const CUtensorMap &a, const CUtensorMap &b, const pair::Plan &p,
                     const Epi &epi, cudaStream_t st) {
    constexpr size_t smem = pair::Shape<EXACT>::kSmem;
    const cudaError_t e = allow_dynamic_smem<pair::gemm_kernel<Epi, A_MN, B_MN, EXACT>>(smem);
    if (e != cudaSuccess) return e;
    const int64_t items = (int64_t)p.m_tiles * p.n_tiles * p.splits, pairs = pairs_of_sms();
    return launch_kernel(true, pair::gemm_kernel<Epi, A_MN, B_MN, EXACT>,
                         dim3((unsigned)(2 * (items < pairs ? items : pairs))), pair::kThreads,
                         smem, st, a, b, p, epi);
}

// Whether a matrix is read where it lies: TMA wants rows on 16-byte boundaries.
// Off 128 bytes it reads two lines for each row of a box; a copy costs a launch and
// a pass over the matrix, which pays from about 4096 tokens on and against as long a
// vocabulary.  Read where they lie / copied, us, loss and gradient: 2048 tokens x
// 14297 x 1400 57 / 68 and 196 / 205, x 32000 x 1000 94 / 111 and 285 / 298; 4096 x 60000
// x 1000 355 / 337 and 1013 / 977; 8192 x 50000 x 328 228 / 242 and 900 / 844; 16384 x
// 32000 x 1000 765 / 658 and 2215 / 2180.
constexpr int64_t kShortSide = 4096;
bool as_it_lies(int32_t dtype, const void *at, int64_t ld, int64_t T, int64_t V) {
    const int align = T < kShortSide || V < kShortSide ? 16 : 128;
    return dtype == ULTRAMEM_BF16 && (uintptr_t)at % align == 0 && ld * 2 % align == 0;
}
int64_t padded(int64_t D) { return (D + 63) & ~63ll; }

template <typename T>
cudaError_t planes_t(const void *src, int64_t ld, int64_t R, int D, void *dst, Labels labels,
                     bool pdl, cudaStream_t st) {
    const int Dp = (int)padded(D);
    const int64_t blocks = ceil_div(R * (Dp / 8), 256), most = (int64_t)device_sm_count() * 16;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    const bool aligned = D % 8 == 0 && (uintptr_t)src % 16 == 0 && ld * sizeof(T) % 16 == 0;
    const T *s = static_cast<const T *>(src);
    __nv_bfloat16 *d = static_cast<__nv_bfloat16 *>(dst);
    return aligned ? launch_kernel(pdl, planes_kernel<T, true>, grid, 256, 0, st, s, ld, R, D, Dp, d,
                                   labels)
                   : launch_kernel(pdl, planes_kernel<T, false>, grid, 256, 0, st, s, ld, R, D, Dp,
                                   d, labels);
}
cudaError_t to_planes(int32_t dtype, const void *src, int64_t ld, int64_t R, int D, void *dst,
                      Labels labels, bool pdl, cudaStream_t st) {
    return dtype == ULTRAMEM_BF16
               ? planes_t<__nv_bfloat16>(src, ld, R, D, dst, labels, pdl, st)
               : planes_t<float>(src, ld, R, D, dst, labels, pdl, st);
}

// A matrix as the products read it: where it lies, or its planes.
struct Matrix {
    const void *at;
    int64_t ld, plane;
    int planes;
};

bool sizes_ok(int32_t dtype, int32_t T, int32_t V, int32_t D) {
    return (dtype == ULTRAMEM_F32 || dtype == ULTRAMEM_BF16) && T >= 0 && V >= 1 &&
           V <= kMaxVocab && D >= 1 && D <= kMaxDim &&
           ceil_div(T, pair::kTileM) * ceil_div(V, 128) <= INT32_MAX &&     // tiles
           ceil_div(T, pair::kTileM) * ceil_div(D, 128) * 64 <= INT32_MAX;
}

// Rows of the vocabulary whose planes fit a piece's bytes.
int64_t rows_in_planes(int32_t dtype, int32_t D) {
    const int64_t n = g_piece_bytes.load() / (planes_of(dtype) * padded(D) * 2) / 256 * 256;
    return n < 256 ? 256 : n;
}
// `limit` rows or fewer a piece, in equal pieces of whole tiles
int64_t piece_of(int64_t V, int64_t limit) {
    if (V <= limit) return V;
    const int64_t n = ceil_div(V, limit);
    return ceil_div(ceil_div(V, n), 256) * 256;
}

struct ForwardLayout {
    int64_t piece;            // of the vocabulary, when the weights are rearranged
    int64_t tiles;            // half tiles of all pieces, at most
    int64_t part, target, x, w, total;
};
ForwardLayout forward_layout(int32_t dtype, int64_t T, int64_t V, int32_t D) {
    ForwardLayout l = {};
    l.piece = piece_of(V, rows_in_planes(dtype, D));
    // of the weights where they lie, or in pieces, the last of which may choose any width
    const int P = planes_of(dtype);
    const int64_t t = T > 0 ? T : 1, last = V % l.piece ? V % l.piece : l.piece;
    const int64_t whole = ceil_div(V, plan_of(t, V, D, P, 32, 1).n_tile);
    const int64_t each = ceil_div(l.piece, plan_of(t, l.piece, D, P, 32, 1).n_tile);
    const int64_t pieces = (V - last) / l.piece * each + ceil_div(last, 128);
    l.tiles = 2 * (whole > pieces ? whole : pieces);
    const int64_t es = planes_of(dtype) * padded(D) * 2;
    l.part = 0;
    l.target = pad256(l.tiles * T * 8);
    l.x = l.target + pad256(T * 4);
    l.w = l.x + pad256(T * es);
    l.total = l.w + pad256(l.piece * es) + 256;
    return l;
}

struct BackwardLayout {
    int64_t piece, ld;        // ld: of G
    int64_t x, w, g, dx, dw, total;
    int dx_splits, dw_splits; // at most
    pair::Plan logits, x_plan, w_plan;       // of a whole piece
};
BackwardLayout backward_layout(int32_t dtype, int64_t T, int64_t V, int32_t D) {
    BackwardLayout l = {};
    const int P = planes_of(dtype);
    const int64_t bytes = g_piece_bytes.load();
    int64_t limit = bytes / (2 * P * (T > 0 ? T : 1)) / 256 * 256;
    if (limit < 256) limit = 256;
    const int64_t rows = rows_in_planes(dtype, D);
    l.piece = piece_of(V, limit < rows ? limit : rows);
    l.ld = (l.piece + 31) & ~31ll;
    // partial sums stay below a piece's bytes, but for as many as long sums need
    auto most = [bytes](int64_t m, int64_t n) {
        const int64_t s = bytes / (m * n * 4);
        return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
    };
    const int64_t t = T > 0 ? T : 1;
    l.logits = plan_of(t, l.piece, D, P, 32, 1);
    l.x_plan = plan_of(t, D, l.piece, P, 128, most(t, padded(D)));
    l.w_plan = plan_of(l.piece, D, t, P, 128, most(l.piece, padded(D)));
    l.dx_splits = l.x_plan.splits;
    l.dw_splits = l.w_plan.splits;
    const int64_t es = P * padded(D) * 2;
    l.x = 0;
    l.w = pad256(T * es);
    l.g = l.w + pad256(l.piece * es);
    l.dx = l.g + pad256(P * T * l.ld * 2);
    l.dw = l.dx + (l.dx_splits > 1 || l.piece < V ? pad256(4 * l.dx_splits * T * padded(D)) : 0);
    l.total = l.dw + (l.dw_splits > 1 ? pad256(4 * l.dw_splits * l.piece * padded(D)) : 0) + 256;
    return l;
}

bool args_ok(const ultramem_cross_entropy_args *p) {
    return p && sizes_ok(p->dtype, p->n_tokens, p->vocab, p->dim) &&
           (p->labels_bytes == 4 || p->labels_bytes == 8) && isfinite(p->logit_scale) &&
           isfinite(p->logit_scale * kLog2e);
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
Labels labels_of(const ultramem_cross_entropy_args *p) {
    return {p->labels, p->labels_bytes == 8, p->vocab};
}
char *aligned256(void *p) {
    return reinterpret_cast<char *>(((uintptr_t)p + 255) & ~(uintptr_t)255);
}
const char *row_at(const ultramem_cross_entropy_args *p, int64_t v) {
    return static_cast<const char *>(p->w) + v * p->ld_w * (p->dtype == ULTRAMEM_BF16 ? 2 : 4);
}

cudaError_t forward(const ultramem_cross_entropy_args *p, const ForwardLayout &l, float *loss,
                    float *lse, char *ws, int *err, cudaStream_t st) {
    const int P = planes_of(p->dtype), D = p->dim;
    const int64_t T = p->n_tokens, Dp = padded(D);
    cudaError_t e = cudaSuccess;
    bool pdl = false;
    Matrix x = {p->x, p->ld_x, T * p->ld_x, 1};
    if (!as_it_lies(p->dtype, p->x, p->ld_x, T, p->vocab)) {
        x = {ws + l.x, Dp, T * Dp, P};
        e = to_planes(p->dtype, p->x, p->ld_x, T, D, ws + l.x, {}, false, st);
        pdl = true;
    }
    const bool direct = as_it_lies(p->dtype, p->w, p->ld_w, T, p->vocab);
    const int64_t piece = direct ? p->vocab : l.piece;
    LseEpi<0> epi = {};
    epi.labels = labels_of(p);
    epi.part = reinterpret_cast<float2 *>(ws + l.part);
    epi.target = reinterpret_cast<float *>(ws + l.target);
    epi.T = p->n_tokens;
    epi.scale_log2 = p->logit_scale * kLog2e;
    for (int64_t v0 = 0; v0 < p->vocab && e == cudaSuccess; v0 += piece) {
        const int64_t vn = p->vocab - v0 < piece ? p->vocab - v0 : piece;
        Matrix w = {row_at(p, v0), p->ld_w, vn * p->ld_w, 1};
        if (!direct) {
            w = {ws + l.w, Dp, vn * Dp, P};
            e = to_planes(p->dtype, row_at(p, v0), p->ld_w, vn, D, ws + l.w, {}, pdl, st);
            if (e != cudaSuccess) break;
        }
        pair::Plan plan = plan_of(T, vn, D, P, 32, 1);
        plan.err = err;
        CUtensorMap ma, mb;
        if (!operand(&ma, x.at, D, T, x.ld, x.planes, x.plane, 128) ||
            !operand(&mb, w.at, D, vn, w.ld, w.planes, w.plane, plan.n_tile / 2))
            return cudaErrorInvalidValue;
        epi.vn = (int)vn;
        epi.v0 = (int)v0;
        epi.n_tile = plan.n_tile;
        if (P == 3)
            e = multiply<LseEpi<0>, false, false, true>(ma, mb, plan, epi, st);
        else if (D <= kLongSum)
            e = multiply<LseEpi<0>, false, false, false>(ma, mb, plan, epi, st);
        else
            e = multiply<LseEpi<16>, false, false, false>(ma, mb, plan, epi.cut<16>(), st);
        epi.tile0 += 2 * plan.n_tiles;
        pdl = true;
    }
    if (e != cudaSuccess) return e;
    const int64_t blocks = ceil_div(T, 32);
    return launch_kernel(true, join_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), 1024, 0,
                         st, (const float2 *)epi.part, (const float *)epi.target, epi.labels,
                         p->n_tokens, epi.tile0, p->logit_scale, epi.scale_log2, loss, lse);
}

template <typename T, int P>
cudaError_t backward(const ultramem_cross_entropy_args *p, const BackwardLayout &l,
                     const float *lse, const float *dloss, void *dx, void *dw, char *ws, int *err,
                     cudaStream_t st) {
    const int D = p->dim;
    const int64_t N = p->n_tokens, Dp = padded(D);
    cudaError_t e = cudaSuccess;
    // dw reads x with weights that are 0 for tokens that do not count
    bool pdl = false;
    Matrix x = {p->x, p->ld_x, N * p->ld_x, 1};
    if (dw || !as_it_lies(p->dtype, p->x, p->ld_x, N, p->vocab)) {
        x = {ws + l.x, Dp, N * Dp, P};
        e = to_planes(p->dtype, p->x, p->ld_x, N, D, ws + l.x, labels_of(p), false, st);
        pdl = true;
    }
    const bool direct = as_it_lies(p->dtype, p->w, p->ld_w, N, p->vocab);
    GradEpi<P> ge = {};
    ge.labels = labels_of(p);
    ge.lse = lse;
    ge.dloss = dloss;
    ge.g = reinterpret_cast<__nv_bfloat16 *>(ws + l.g);
    ge.ld = l.ld;
    ge.T = p->n_tokens;
    ge.scale = p->logit_scale;
    ge.scale_log2 = p->logit_scale * kLog2e;
    const bool dx_parts = l.dx_splits > 1 || l.piece < p->vocab;
    float *dx_sum = dx_parts ? reinterpret_cast<float *>(ws + l.dx) : nullptr;
    float *dw_sum = l.dw_splits > 1 ? reinterpret_cast<float *>(ws + l.dw) : nullptr;
    auto wide = [&](const void *at) { return (uintptr_t)at % 32 == 0 && D * sizeof(T) % 32 == 0; };
    auto sum_splits = [&](const float *part, int splits, int64_t m, T *out) {
        const int64_t blocks = ceil_div(m * (Dp / 4), 256), most = (int64_t)device_sm_count() * 32;
        return launch_kernel(true, sum_splits_kernel<T>,
                             dim3((unsigned)(blocks < most ? blocks : most)), 256, 0, st, part,
                             splits, m, D, (int)Dp, out,
                             (int)((uintptr_t)out % 16 == 0 && D % 4 == 0));
    };
    for (int64_t v0 = 0; v0 < p->vocab && e == cudaSuccess; v0 += l.piece) {
        const int64_t vn = p->vocab - v0 < l.piece ? p->vocab - v0 : l.piece;
        Matrix w = {row_at(p, v0), p->ld_w, vn * p->ld_w, 1};
        if (!direct) {
            w = {ws + l.w, Dp, vn * Dp, P};
            e = to_planes(p->dtype, row_at(p, v0), p->ld_w, vn, D, ws + l.w, {}, pdl, st);
            if (e != cudaSuccess) break;
        }
        CUtensorMap ma, mb;
        pair::Plan plan = l.logits;
        plan.n_tiles = (int)ceil_div(vn, plan.n_tile);
        plan.err = err;
        if (!operand(&ma, x.at, D, N, x.ld, x.planes, x.plane, 128) ||
            !operand(&mb, w.at, D, vn, w.ld, w.planes, w.plane, plan.n_tile / 2))
            return cudaErrorInvalidValue;
        ge.vn = (int)vn;
        ge.v0 = (int)v0;
        e = multiply<GradEpi<P>, false, false, P == 3>(ma, mb, plan, ge, st);
        pdl = true;
        if (dx && e == cudaSuccess) {            // [N][D] = G [N][vn] W [vn][D]
            plan = l.x_plan;
            plan.k_blocks = (int)ceil_div(vn, 64);
            // a short last piece: fewer splits, the other sums stay as they are
            if (plan.splits > plan.k_blocks) plan.splits = plan.k_blocks;
            plan.err = err;
            if (!operand(&ma, ge.g, vn, N, l.ld, P, N * l.ld, 128) ||
                !operand(&mb, w.at, D, vn, w.ld, w.planes, w.plane, 64))
                return cudaErrorInvalidValue;
            // one split: the last piece adds the others' sums and writes dx itself
            const bool here = l.dx_splits == 1 && v0 + vn == p->vocab;
            const StoreEpi<T> se = {here ? static_cast<T *>(dx) : nullptr, dx_sum, N, D, Dp, v0 > 0,
                                    wide(dx)};
            e = multiply<StoreEpi<T>, false, true, P == 3>(ma, mb, plan, se, st);
        }
        if (dw && e == cudaSuccess) {            // [vn][D] = G^T [vn][N] x [N][D]
            plan = l.w_plan;
            plan.m_tiles = (int)ceil_div(vn, pair::kTileM);
            plan.err = err;
            if (!operand(&ma, ge.g, vn, N, l.ld, P, N * l.ld, 64) ||
                !operand(&mb, x.at, D, N, x.ld, x.planes, x.plane, 64))
                return cudaErrorInvalidValue;
            T *out = static_cast<T *>(dw) + v0 * D;
            const StoreEpi<T> se = {dw_sum ? nullptr : out, dw_sum, vn, D, Dp, 0, wide(out)};
            e = multiply<StoreEpi<T>, true, true, P == 3>(ma, mb, plan, se, st);
            if (dw_sum && e == cudaSuccess) e = sum_splits(dw_sum, l.dw_splits, vn, out);
        }
    }
    if (dx && l.dx_splits > 1 && e == cudaSuccess)
        e = sum_splits(dx_sum, l.dx_splits, N, static_cast<T *>(dx));
    return e;
}

}  // namespace
}  // namespace ce
}  // namespace um

using namespace um::ce;

extern "C" int64_t ultramem_cross_entropy_workspace(int32_t dtype, int32_t n_tokens,
                                                    int32_t vocab, int32_t dim) {
    if (!sizes_ok(dtype, n_tokens, vocab, dim)) return 0;
    return forward_layout(dtype, n_tokens, vocab, dim).total;
}

extern "C" ultramem_status ultramem_cross_entropy(const ultramem_cross_entropy_args *p,
                                                  float *loss, float *lse, void *workspace,
                                                  int64_t workspace_bytes, void *stream) {
    if (!args_ok(p)) return ULTRAMEM_EINVAL;
    if (p->n_tokens == 0) return ULTRAMEM_OK;
    const ForwardLayout l = forward_layout(p->dtype, p->n_tokens, p->vocab, p->dim);
    const int64_t need = l.total;
    if (!inputs_ok(p) || !loss || !lse || ((uintptr_t)loss | (uintptr_t)lse) % 4 || !workspace ||
        ((uintptr_t)workspace & 15) || workspace_bytes < need)
        return ULTRAMEM_EINVAL;
    const int64_t T = p->n_tokens;
    if (!um::apart({{loss, T * 4}, {lse, T * 4}, {workspace, need}},
                   {rows_of(p, p->x, T, p->ld_x), rows_of(p, p->w, p->vocab, p->ld_w),
                    {p->labels, T * p->labels_bytes}}))
        return ULTRAMEM_EINVAL;
    cudaGetLastError();
    int *err = um::paged::error_word();
    if (!err) return ULTRAMEM_ENODEV;
    return um::status_from_cuda(
        forward(p, l, loss, lse, aligned256(workspace), err, (cudaStream_t)stream));
}

extern "C" int64_t ultramem_cross_entropy_backward_workspace(int32_t dtype, int32_t n_tokens,
                                                             int32_t vocab, int32_t dim) {
    if (!sizes_ok(dtype, n_tokens, vocab, dim)) return 0;
    return backward_layout(dtype, n_tokens, vocab, dim).total;
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
    const BackwardLayout l = backward_layout(p->dtype, p->n_tokens, p->vocab, p->dim);
    const int64_t need = l.total;
    if (!inputs_ok(p) || !lse || !dloss || ((uintptr_t)lse | (uintptr_t)dloss) % 4 || !workspace ||
        ((uintptr_t)workspace & 15) || workspace_bytes < need)
        return ULTRAMEM_EINVAL;
    const int64_t T = p->n_tokens;
    if (!um::apart({{dx, T * p->dim * es}, {dw, dw_bytes}, {workspace, need}},
                   {rows_of(p, p->x, T, p->ld_x), rows_of(p, p->w, p->vocab, p->ld_w),
                    {p->labels, T * p->labels_bytes}, {lse, T * 4}, {dloss, T * 4}}))
        return ULTRAMEM_EINVAL;
    int *err = um::paged::error_word();
    if (!err) return ULTRAMEM_ENODEV;
    char *ws = aligned256(workspace);
    return um::status_from_cuda(
        p->dtype == ULTRAMEM_BF16
            ? backward<__nv_bfloat16, 1>(p, l, lse, dloss, dx, dw, ws, err, st)
            : backward<float, 3>(p, l, lse, dloss, dx, dw, ws, err, st));
}

extern "C" ultramem_status ultramem_debug_cross_entropy_piece(int64_t bytes) {
    if (bytes < 0) return ULTRAMEM_EINVAL;
    g_piece_bytes.store(bytes ? bytes : kPieceBytes);
    return ULTRAMEM_OK;
}

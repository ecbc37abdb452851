// um_paged.cuh -- what the kernels over the paged key/value cache share: the
// call's arguments, the split of the work over a fixed number of CTAs, and
// the partial results that CTAs leave when a split falls inside a tile.
//
// The rows of a request that read one key/value head are its new tokens x
// the query heads of that head's group, token-major.  A tile is TQ tokens of
// one request for one key/value head.  Its length is the number of keys its
// last token sees (at least 1) and a fixed cost in keys (reading the queries,
// writing the output), and the lengths of all tiles, laid end to end in the
// order (request, head, tile), form one axis.  CTA c of C takes the
// c-th of C equal shares of that axis, so the CTAs finish together whatever
// the requests' lengths are, without any table made on the host.  A share
// boundary inside a tile is moved to the next block of KB keys, and a tile of
// at most twice its fixed cost in keys is not split (its halves would cost
// more than they save) but goes with the share it starts in.  A tile that
// lies in one share is written straight to the output; one that crosses
// shares leaves a partial (maximum, sum, unnormalised output) per share,
// which the join kernels add in share order.
#pragma once

#include "um_internal.cuh"

namespace um {
namespace paged {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxHeadDim = 256;
// The most keys of a request: whole blocks, and the block after the last one
// has numbers below 2^31 too (the table is read a block ahead).
constexpr int kMaxKeys = INT32_MAX - 1023;

struct AttnArgs {
    const void *q, *k, *v;
    const int32_t *table, *q_start, *kv_lens;
    void *out;
    float *lse;                 // [T][q_heads] or null
    float *part_o;              // [C][2][rows][DP] unnormalised outputs
    float2 *part_ml;            // [C][2][rows] (maximum in log2 units, sum)
    int4 *part_desc;            // [C][2] (kind, first token, tokens, head)
    int *err;
    int64_t q_stride;           // elements between tokens of q
    int n_seqs, n_tokens, q_heads, kv_heads, group, D;
    int page_shift, table_width, n_pages;
    int rows;                   // rows of a tile, padded (the partials' stride)
    int rows_hint;              // rows that tiles are expected to have
    int tq;                     // tokens of a tile
    int extra;                  // a tile's fixed cost, in keys
    float scale_log2;           // the scores' factor times log2(e)
};

enum { kPartNone = 0, kPartFirst = 1, kPartMiddle = 2, kPartLast = 3 };

// The most keys of a tile that is not split.
__host__ __device__ inline int whole_keys(const AttnArgs &a) { return 2 * a.extra; }

// One request's part of the axis.
struct Request {
    int tok0, n, kv;            // first token in the batch, new tokens, keys
    __device__ __forceinline__ void read(const AttnArgs &a, int r) {
        tok0 = a.q_start[r];
        int end = a.q_start[r + 1];
        if (tok0 < 0) tok0 = 0;
        if (end > a.n_tokens) end = a.n_tokens;
        n = end > tok0 ? end - tok0 : 0;
        kv = a.kv_lens[r];
        int64_t held = (int64_t)a.table_width << a.page_shift;
        if (held > kMaxKeys) held = kMaxKeys;
        if (kv > held) kv = (int)held;
        if (kv < 0) kv = 0;
    }
    __device__ __forceinline__ int tiles(int tq) const { return (n + tq - 1) / tq; }
    // keys the last token of tile t sees, at least 1
    __device__ __forceinline__ int keys(int t, int tq) const {
        const int last = min((t + 1) * tq, n);
        return max(1, kv - n + last);
    }
    // where tile t < tiles() starts: the keys and fixed costs of the tiles
    // before it, kv - n + (i + 1) tq keys each, but 1 where that is below 1
    __device__ __forceinline__ int64_t before(int t, const AttnArgs &a) const {
        const int64_t c = (int64_t)kv - n;
        const int64_t flat = c < 0 ? min((int64_t)t, -c / a.tq) : 0;   // tiles of 1 key
        const int64_t m = t - flat;
        return flat + m * c + (int64_t)a.tq * (m * flat + m * (m + 1) / 2) + (int64_t)t * a.extra;
    }
    __device__ __forceinline__ int64_t per_head(const AttnArgs &a) const {
        const int t = tiles(a.tq);
        return t ? before(t - 1, a) + keys(t - 1, a.tq) + a.extra : 0;
    }
};

// Where a CTA's share starts, found by the whole block (THREADS threads).
struct Cursor {
    int r, h, t;                // request, key/value head, tile
    int64_t off;                // keys into the tile
    int64_t left;               // keys left of the share
};

// Block-wide: sums the requests' parts of the axis, thread i over a
// contiguous run of requests, and places the share of CTA `c` of `ctas`.
// `scratch` holds THREADS / 32 + 1 values in shared memory; `cur` is shared.
template <int THREADS>
__device__ __forceinline__ void place_share(const AttnArgs &a, int c, int ctas, int kb,
                                            int64_t min_share, int64_t *scratch, Cursor *cur) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int64_t per = ((int64_t)a.n_seqs + THREADS - 1) / THREADS;
    const int r0 = (int)min((int64_t)a.n_seqs, tid * per);
    const int r1 = (int)min((int64_t)a.n_seqs, r0 + per);
    int64_t mine = 0;
    Request q;
    for (int r = r0; r < r1; ++r) {
        q.read(a, r);
        mine += q.per_head(a) * a.kv_heads;
    }
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) scratch[w] = upto;
    if (tid == 0) cur->left = 0;
    __syncthreads();
    int64_t total = 0, base = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
        if (i == w) base = total;
        total += scratch[i];
    }
    int64_t share = (total + ctas - 1) / ctas;
    if (share < min_share) share = min_share;
    share = (share + kb - 1) / kb * kb;
    const int64_t lo = share * c, hi = min(total, lo + share);
    int64_t at = base + upto - mine;
    if (lo < hi && lo >= at && lo < at + mine) {   // this thread's run holds the start
        int r = r0;
        int64_t rest = lo - at, head = 0;
        for (; r < r1; ++r) {
            q.read(a, r);
            head = q.per_head(a);
            if (rest < head * a.kv_heads) break;
            rest -= head * a.kv_heads;
        }
        const int h = (int)(rest / head);
        rest -= h * head;
        int t0 = 0, t1 = q.tiles(a.tq) - 1;   // the last tile that starts at or before rest
        while (t0 < t1) {
            const int m = (t0 + t1 + 1) >> 1;
            if (q.before(m, a) <= rest)
                t0 = m;
            else
                t1 = m - 1;
        }
        cur->r = r;
        cur->h = h;
        cur->t = t0;
        cur->off = rest - q.before(t0, a);
        cur->left = hi - lo;
    }
    __syncthreads();
}

// A CTA's walk over its share, the same in every thread that runs it.
struct Walk {
    Cursor c;
    Request q;
    bool first;                 // the next tile is the share's first
    // the tile at hand
    int tok0, n_tok, h, kv, pos0;   // first token, tokens, head, keys, position of the first token
    int j0, j1, blocks;             // blocks of KB keys: [j0, j1) of this share, of the tile
    int part;                       // kPart*: whether the tile is this share's alone
    int slot;                       // 0: the share's first tile, else 1 (the partials' place)

    __device__ __forceinline__ void begin(const AttnArgs &a, const Cursor &cur) {
        c = cur;
        first = true;
        if (c.left > 0) q.read(a, c.r);
    }
    // The next tile with blocks in this share; false at the share's end.
    __device__ __forceinline__ bool next(const AttnArgs &a, int kb) {
        while (c.left > 0) {
            while (c.t >= q.tiles(a.tq)) {   // next head, next request with rows
                c.t = 0;
                if (++c.h >= a.kv_heads) {
                    c.h = 0;
                    q.read(a, ++c.r);
                } else if (q.n == 0) {
                    c.h = a.kv_heads - 1;
                }
            }
            const int keys = q.keys(c.t, a.tq);
            const bool whole = keys <= whole_keys(a);
            const int64_t len = (int64_t)keys + a.extra;
            if (whole && c.off > 0) {        // begun and finished by an earlier share
                c.left -= len - c.off;
                c.off = 0;
                ++c.t;
                continue;
            }
            const int64_t take = whole ? len : min(c.left, len - c.off);
            tok0 = q.tok0 + c.t * a.tq;
            n_tok = min(a.tq, q.n - c.t * a.tq);
            h = c.h;
            kv = q.kv;
            pos0 = q.kv - q.n + c.t * a.tq;
            blocks = (keys + kb - 1) / kb;
            j0 = (int)min((int64_t)blocks, (c.off + kb - 1) / kb);
            j1 = (int)min((int64_t)blocks, (c.off + take + kb - 1) / kb);
            slot = first ? 0 : 1;
            first = false;
            c.left -= take;
            c.off += take;
            if (c.off >= len) {
                c.off = 0;
                ++c.t;
            }
            if (j0 < j1) {
                part = j0 == 0 ? (j1 == blocks ? kPartNone : kPartFirst)
                               : (j1 == blocks ? kPartLast : kPartMiddle);
                return true;
            }
        }
        return false;
    }
};

// The page of key `key` of request r, or -1 past its length and where the
// table names no page of the cache (read as zeros).
__device__ __forceinline__ int page_of(const AttnArgs &a, int r, int key, int kv) {
    if (key >= kv) return -1;
    const int p = a.table[(int64_t)r * a.table_width + (key >> a.page_shift)];
    return p < 0 || p >= a.n_pages ? -1 : p;
}

// The current device's error word of the calls without a handle (null when it
// cannot be found): kernels whose bounded wait gave up set kErrTimeout.
int *error_word();
// A map of 64-column boxes over a bf16 tensor [outer][mid][inner] with the
// given strides in elements; zeros outside.  False when it cannot be made.
bool encode(CUtensorMap *map, const void *base, uint64_t inner, uint64_t mid, uint64_t outer,
            uint64_t mid_stride, uint64_t outer_stride, uint32_t box_mid, uint32_t box_outer);

// bf16, heads up to 128 wide: at most 16 rows a tile (um_paged_decode.cu), or
// two halves of 128 rows (um_paged_prefill.cu).  The maps are over the cache
// as [pages x heads][page size][head width] with boxes of 64 columns x
// *_box_rows tokens, and over q as [tokens][heads][width].
int decode_box_rows(int page_size);
int prefill_box_rows(int page_size);
cudaError_t launch_decode(const AttnArgs &a, const CUtensorMap &k, const CUtensorMap &v, int ctas,
                          cudaStream_t st);
cudaError_t launch_prefill(const AttnArgs &a, const CUtensorMap &q, const CUtensorMap &k,
                           const CUtensorMap &v, int ctas, cudaStream_t st);
cudaError_t launch_combine(const AttnArgs &a, int ctas, int dp, int dtype, int max_new, bool pdl,
                           cudaStream_t st);

}  // namespace paged
}  // namespace um

// um_embed.cu -- the embedding of token ids and its gradient.
//
// Forward: out[t] = scale table[id_t], one read and one write of a row a
// token (16384 x 2048 bf16: 20.4 us, 6.6 TB/s).
//
// Gradient: dtable[v] = scale sum_{t: id_t = v} dout[t].  The tokens are sorted
// by id (stable, so a row's tokens stay in their order), the sorted list is
// cut into chunks of equal length, and a block sums the runs of equal ids in
// its chunk in fp32.  A run inside one chunk is written at once; one that
// crosses chunks leaves a partial sum a chunk, which a last kernel adds in
// chunk order.  No sum depends on the order in which blocks run, and a
// frequent id costs no more than rare ones.  16384 x 2048 into 32000 rows, bf16: 57 us,
// 29 of them the bytes at the copy rate; the zeros beside the sort 20, sums 21, join 8.
// Short batches go another way (short_kernel).
#include "um_device.cuh"
#include "um_internal.cuh"
#include "um_overlap.cuh"
#include "um_tc.cuh"

namespace um {
namespace embed {
namespace {

constexpr int kMaxVocab = 1 << 30;
constexpr int kMaxDim = 65536;

// ---- values, 8 at a time where rows allow 16-byte accesses -------------------

// Ordinary loads: the rows that sums are added to are written by the same kernel, and
// partial sums by one that may still run when theirs starts.
__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0];
    const float4 b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
// N values (8, or 1 where rows are not aligned)
template <typename T, int N> __device__ __forceinline__ void load(const T *p, float (&v)[N]) {
    if constexpr (N == 8) {
        load8(p, v);
    } else {
        v[0] = to_f(p[0]);
    }
}
template <typename T, int N> __device__ __forceinline__ void store(T *p, const float (&v)[N]) {
    if constexpr (N == 8) {
        store8(p, v);
    } else {
        p[0] = from_f<T>(v[0]);
    }
}

// the id of token t, or -1 outside [0, vocab)
__device__ __forceinline__ int id_of(const void *ids, int wide, int64_t t, int vocab) {
    const int64_t id = wide ? static_cast<const int64_t *>(ids)[t]
                            : (int64_t) static_cast<const int32_t *>(ids)[t];
    return id >= 0 && id < vocab ? (int)id : -1;
}

// ---- forward -------------------------------------------------------------

// A thread an N-wide piece of a row.
template <typename T, int N>
__global__ void __launch_bounds__(256)
    embed_kernel(const T *table, int64_t ld, int vocab, int D, const void *ids, int wide,
                 int64_t n_tokens, float scale, T *out) {
    const int pieces = D / N;
    const int64_t total = n_tokens * pieces, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += step) {
        const int64_t t = i / pieces;
        const int c = (int)(i - t * pieces) * N;
        const int id = id_of(ids, wide, t, vocab);
        float v[N];
        if (id >= 0) {
            load<T, N>(table + (int64_t)id * ld + c, v);
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] *= scale;
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = 0.f;
        }
        store<T, N>(out + t * D + c, v);
    }
}

// ---- the tokens sorted by id -------------------------------------------------
// A radix sort from the lowest digit, 8 bits or less at a time.  A block takes
// kTile keys in order, a warp 32 x kRounds of them at most: a key's place among the
// keys of its digit is the number of equal digits before it in its warp (by
// ballots in a round, and a counter a warp and digit from round to round), in the
// warps before, and in the blocks before.

constexpr int kSortThreads = 1024;
constexpr int kRounds = 4;
constexpr int kTile = kSortThreads * kRounds;
constexpr int kDigits = 256;
constexpr int kCluster = 8;               // blocks that sort together
constexpr int kWarps = kSortThreads / 32;

struct SortArgs {
    const void *ids;
    int *key[2], *tok[2];     // [T], in turns
    int *hist;                // [tiles][kDigits] of a pass
    int T, vocab, wide, bits, passes, tiles;
    int tile;                 // keys of a tile, at most kTile
};

__host__ __device__ __forceinline__ int pass_bits(int bits, int passes) {
    return (bits + passes - 1) / passes;
}

// key `i` before pass `p`; an id outside the table sorts behind all others
__device__ __forceinline__ int key_at(const SortArgs &a, int p, int i) {
    if (p > 0) return (p & 1 ? a.key[0] : a.key[1])[i];
    const int id = id_of(a.ids, a.wide, i, a.vocab);
    return id < 0 ? a.vocab : id;
}

struct SortShared {
    int count[kWarps][kDigits];
    int first[kDigits];       // of a digit's keys in the tile's order
    int move[kDigits];        // from there to their place among all tiles' keys
    int scan[2][kDigits / 32];
    int part[2][kSortThreads / kDigits][kDigits];
    int key[kTile], tok[kTile];          // the tile in order
};

// The exclusive sum of `v` over threads 0..kDigits - 1, two block barriers.
__device__ __forceinline__ int digits_before(int v, int *scan) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int upto = v;
    if (threadIdx.x < kDigits) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (lane == 31) scan[w] = upto;
    }
    __syncthreads();
    int at = upto - v;
    if (threadIdx.x < kDigits)
        for (int i = 0; i < w; ++i) at += scan[i];
    return at;
}

// Ranks of the keys among the equal digits before them in their warp, whose
// counts are left in count[warp]; a warp holds 32 x rounds keys in order.
__device__ __forceinline__ void rank_keys(const int (&key)[kRounds], int (&rank)[kRounds],
                                          int rounds, int mine, int n, int shift, int db,
                                          int (&count)[kDigits]) {
    const int lane = threadIdx.x & 31;
    const uint32_t mask = (1u << db) - 1u;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        if (r >= rounds) break;
        const bool live = mine + r * 32 < n;
        const uint32_t d = ((uint32_t)key[r] >> shift) & mask;
        // the lanes with this digit, a ballot a bit
        uint32_t same = __ballot_sync(0xffffffffu, live);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            if (b >= db) break;
            const bool set = d & (1u << b);
            const uint32_t lanes = __ballot_sync(0xffffffffu, set);
            same &= set ? lanes : ~lanes;
        }
        const int before = live ? count[d] : 0;
        __syncwarp();
        if (live && lane == __ffs(same) - 1) count[d] = before + __popc(same);
        __syncwarp();
        rank[r] = before + __popc(same & ((1u << lane) - 1u));
    }
}
// Thread d < kDigits: the warps' counts of digit d become their sums before a
// warp; returns the block's count.
__device__ __forceinline__ int sum_warps(int (&count)[kWarps][kDigits]) {
    int here = 0;
    for (int i = 0; i < kWarps; ++i) {
        const int c = count[i][threadIdx.x];
        count[i][threadIdx.x] = here;
        here += c;
    }
    return here;
}

// Pass p of tile `tile`, whose digits' counts are in hist with those of the
// others.  The keys go to their places by way of shared memory, because a
// warp's 32 keys scatter over as many sectors.
__device__ __forceinline__ void sort_pass(const SortArgs &a, int p, int tile, SortShared &s) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int db = pass_bits(a.bits, a.passes), shift = p * db;
    const uint32_t mask = (1u << db) - 1u;
    for (int i = tid; i < kWarps * kDigits; i += kSortThreads) (&s.count[0][0])[i] = 0;
    int *key_to = p & 1 ? a.key[1] : a.key[0], *tok_to = p & 1 ? a.tok[1] : a.tok[0];
    const int *tok_from = p & 1 ? a.tok[0] : a.tok[1];
    const int64_t start = (int64_t)tile * a.tile;
    const int n = (int)min((int64_t)a.tile, a.T - start);
    const int rounds = a.tile / kSortThreads;
    int key[kRounds], rank[kRounds];
    const int mine = w * 32 * rounds + lane;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = mine + r * 32;
        key[r] = r < rounds && i < n ? key_at(a, p, (int)(start + i)) : -1;
    }
    __syncthreads();
    rank_keys(key, rank, rounds, mine, n, shift, db, s.count[w]);
    __syncthreads();
    int here = 0, all = 0, tiles_before = 0;
    if (tid < kDigits) here = sum_warps(s.count);
    {   // four threads a digit share the tiles
        int c_all = 0, c_before = 0;
        const int d = tid & (kDigits - 1);
#pragma unroll 8
        for (int i = tid / kDigits; i < a.tiles; i += 4) {
            const int c = a.hist[(int64_t)i * kDigits + d];
            if (i < tile) c_before += c;
            c_all += c;
        }
        s.part[0][tid / kDigits][d] = c_all;
        s.part[1][tid / kDigits][d] = c_before;
        __syncthreads();
        if (tid < kDigits)
            for (int i = 0; i < 4; ++i) {
                all += s.part[0][i][tid];
                tiles_before += s.part[1][i][tid];
            }
    }
    const int first = digits_before(here, s.scan[0]), global = digits_before(all, s.scan[1]);
    if (tid < kDigits) {
        s.first[tid] = first;
        s.move[tid] = global + tiles_before - first;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = mine + r * 32;
        if (r >= rounds || i >= n) continue;
        const uint32_t d = ((uint32_t)key[r] >> shift) & mask;
        const int to = s.first[d] + s.count[w][d] + rank[r];
        s.key[to] = key[r];
        s.tok[to] = p > 0 ? tok_from[start + i] : (int)(start + i);
    }
    __syncthreads();
    for (int i = tid; i < n; i += kSortThreads) {
        const int k = s.key[i], to = i + s.move[((uint32_t)k >> shift) & mask];
        key_to[to] = k;
        tok_to[to] = s.tok[i];
    }
}

// zeros over dtable, the blocks `block` of `blocks` sharing it
__device__ __forceinline__ void fill_zeros(uint4 *at, int64_t n16, void *rest, int rest_bytes,
                                           int block, int blocks) {
    const int64_t step = (int64_t)blocks * blockDim.x;
    for (int64_t i = (int64_t)block * blockDim.x + threadIdx.x; i < n16; i += step)
        at[i] = make_uint4(0, 0, 0, 0);
    if (block == 0 && threadIdx.x < rest_bytes) static_cast<uint8_t *>(rest)[threadIdx.x] = 0;
}

struct FillArgs {
    uint8_t *at;              // null: nothing to fill
    int64_t bytes;
};

// The part `part` of `parts` of the fill.
__device__ __forceinline__ void fill(const FillArgs &f, int part, int parts, int block,
                                     int blocks) {
    if (!f.at) return;
    // whole 16-byte pieces from the first boundary on; the ends byte by byte
    const int64_t head = min(f.bytes, (int64_t)(-(uintptr_t)f.at & 15));
    const int64_t n16 = (f.bytes - head) / 16;
    const int64_t lo = n16 * part / parts, hi = n16 * (part + 1) / parts;
    uint4 *body = reinterpret_cast<uint4 *>(f.at + head);
    if (part == 0 && block == 0 && threadIdx.x < head) f.at[threadIdx.x] = 0;
    const int tail = part == parts - 1 ? (int)(f.bytes - head - n16 * 16) : 0;
    fill_zeros(body + lo, hi - lo, f.at + f.bytes - tail, tail, block, blocks);
}

// Zeros over dtable by one block an SM, all resident at once, so that the sort
// starts beside it (inside the sort's launch, whose blocks hold 80 KB of shared
// memory, 200 MB took 43 us instead of 34).
__global__ void __launch_bounds__(1024) fill_kernel(FillArgs f) {
    pdl_trigger();
    fill(f, 0, 1, blockIdx.x, gridDim.x);
}

// The whole sort of at most kCluster tiles by a cluster: block b holds places
// b * tile .. of the list in its shared memory, and the blocks send their
// digits' counts and their keys to one another's, so that the sort does not
// wait for a memory that the fill keeps busy.  (By a single block the sort of
// 16384 tokens took 40 us, bound by issuing its 160000 instructions; 15 so.)
// It reads and writes nothing of the fill's and runs beside it; it ends after
// it, and so what follows finds both done.
struct ClusterShared {
    int count[kWarps][kDigits];
    int counts[kCluster][kDigits];       // of the blocks
    int base[kDigits];                   // of a digit's keys of this block in the list
    int scan[kDigits / 32];
    int key[2][kTile], tok[2][kTile];    // this block's places, before and after a pass
};
__device__ __forceinline__ void store_peer(int *at, int rank, int v) {
    const uint32_t to = tc::mapa_shared(tc::smem_u32(at), (uint32_t)rank);
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(to), "r"(v) : "memory");
}
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kSortThreads)
    sort_small_kernel(SortArgs a) {
    extern __shared__ __align__(16) uint8_t raw[];
    ClusterShared &s = *reinterpret_cast<ClusterShared *>(raw);
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, block = blockIdx.x;
    const int db = pass_bits(a.bits, a.passes);
    const uint32_t mask = (1u << db) - 1u;
    const int start = block * a.tile, n = max(0, min(a.tile, a.T - start));
    const int rounds = a.tile / kSortThreads, mine = w * 32 * rounds + lane;
    tc::cluster_sync();                  // the peers have started
    for (int p = 0; p < a.passes; ++p) {
        const int shift = p * db;
        for (int i = tid; i < kWarps * kDigits; i += kSortThreads) (&s.count[0][0])[i] = 0;
        int key[kRounds], tok[kRounds], rank[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = mine + r * 32;
            const bool live = r < rounds && i < n;
            key[r] = !live ? -1 : p ? s.key[p & 1][i] : key_at(a, 0, start + i);
            tok[r] = !live ? 0 : p ? s.tok[p & 1][i] : start + i;
        }
        __syncthreads();
        rank_keys(key, rank, rounds, mine, n, shift, db, s.count[w]);
        __syncthreads();
        if (tid < kDigits) {
            const int here = sum_warps(s.count);
            for (int i = 0; i < kCluster; ++i) store_peer(&s.counts[block][tid], i, here);
        }
        tc::cluster_sync();
        int all = 0, before = 0;
        if (tid < kDigits)
            for (int i = 0; i < kCluster; ++i) {
                const int c = s.counts[i][tid];
                if (i < block) before += c;
                all += c;
            }
        const int first = digits_before(all, s.scan);
        if (tid < kDigits) s.base[tid] = first + before;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            if (r >= rounds || mine + r * 32 >= n) continue;
            const uint32_t d = ((uint32_t)key[r] >> shift) & mask;
            const int to = s.base[d] + s.count[w][d] + rank[r];
            const int peer = to / a.tile, at = to - peer * a.tile;
            store_peer(&s.key[(p + 1) & 1][at], peer, key[r]);
            store_peer(&s.tok[(p + 1) & 1][at], peer, tok[r]);
        }
        tc::cluster_sync();
    }
    const int last = a.passes & 1;
    for (int i = tid; i < n; i += kSortThreads) {
        a.key[0][start + i] = s.key[last][i];
        a.tok[0][start + i] = s.tok[last][i];
    }
    pdl_wait();
}

// Digit counts of pass p, a block a tile; blocks past them zero a part of dtable.
__global__ void __launch_bounds__(kSortThreads)
    sort_count_kernel(SortArgs a, int p, FillArgs f, int part, int parts) {
    __shared__ int count[kDigits];
    pdl_wait();
    pdl_trigger();
    const int tile = blockIdx.x;
    if (tile >= a.tiles) {
        fill(f, part, parts, tile - a.tiles, gridDim.x - a.tiles);
        return;
    }
    const int db = pass_bits(a.bits, a.passes);
    if (threadIdx.x < kDigits) count[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll 4
    for (int r = 0; r < kRounds; ++r) {
        const int64_t i = (int64_t)tile * a.tile + r * kSortThreads + threadIdx.x;
        if (i < a.T)
            atomicAdd(&count[((uint32_t)key_at(a, p, (int)i) >> (p * db)) & ((1u << db) - 1u)], 1);
    }
    __syncthreads();
    if (threadIdx.x < kDigits) a.hist[(int64_t)tile * kDigits + threadIdx.x] = count[threadIdx.x];
}

__global__ void __launch_bounds__(kSortThreads)
    sort_place_kernel(SortArgs a, int p, FillArgs f, int part, int parts) {
    extern __shared__ __align__(16) uint8_t raw[];
    SortShared &s = *reinterpret_cast<SortShared *>(raw);
    pdl_wait();
    pdl_trigger();
    if ((int)blockIdx.x < a.tiles)
        sort_pass(a, p, blockIdx.x, s);
    else
        fill(f, part, parts, blockIdx.x - a.tiles, gridDim.x - a.tiles);
}

// ---- the sums ----------------------------------------------------------------

struct SumArgs {
    const int *key, *tok;     // sorted
    const void *dout;
    int64_t ld;
    void *dtable;
    float *part;              // [chunks][2][D]: a chunk's first and last run, where they cross
    int T, D, vocab, chunk, chunks, accumulate;
    float scale;
};

template <typename O, int N>
__device__ __forceinline__ void write_row(const SumArgs &a, int id, int c, const float (&s)[N]) {
    O *to = static_cast<O *>(a.dtable) + (int64_t)id * a.D + c;
    float v[N];
    if (a.accumulate) {
        load<O, N>(to, v);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = fmaf(a.scale, s[k], v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = a.scale * s[k];
    }
    store<O, N>(to, v);
}

// values as they are loaded: 8 (16 or 32 bytes), or one
template <typename T, int N> struct Raw {
    uint4 x[N == 8 ? sizeof(T) / 2 : 1];
    __device__ __forceinline__ void get(const T *p) {
        if constexpr (N == 8) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i)
                x[i] = __ldg(reinterpret_cast<const uint4 *>(p) + i);
        } else {
            x[0].x = __float_as_uint(to_f(p[0]));
        }
    }
    __device__ __forceinline__ void add_to(float (&s)[N]) const {
        if constexpr (N == 1) {
            s[0] += __uint_as_float(x[0].x);
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
                const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (sizeof(T) == 4) {
                        s[4 * i + k] += __uint_as_float(w[k]);
                    } else {
                        s[2 * k] += __uint_as_float(w[k] << 16);
                        s[2 * k + 1] += __uint_as_float(w[k] & 0xffff0000u);
                    }
                }
            }
        }
    }
};

// blockDim.x x N columns of blockDim.y chunks of the sorted tokens; the list in
// steps of 32 tokens by way of shared memory, the rows two sets ahead,
// because the time is that of the loads' latency.
template <typename T, typename O, int N>
__global__ void __launch_bounds__(256, sizeof(T) == 4 ? 2 : 4) sum_kernel(SumArgs a) {
    constexpr int kList = 32, kAhead = 4;
    __shared__ int keys[32][kList + 1], toks[32][kList];
    pdl_wait();
    pdl_trigger();
    int *key = keys[threadIdx.y], *tok = toks[threadIdx.y];
    const int c = (blockIdx.y * blockDim.x + threadIdx.x) * N;
    const int64_t chunk = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int lo = (int)min((int64_t)a.T, chunk * a.chunk);
    const int hi = (int)min((int64_t)a.T, (int64_t)lo + a.chunk);
    const bool live = c < a.D;
    const T *dout = static_cast<const T *>(a.dout) + c;
    const bool joined = lo > 0 && lo < hi && a.key[lo - 1] == a.key[lo];
    float *part = a.part + chunk * 2 * a.D + c;
    bool head = true;         // the run at hand starts the chunk
    float sum[N];
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = 0.f;
    for (int64_t i0 = lo; i0 < (int64_t)lo + a.chunk; i0 += kList) {    // as often in all rows
        const int n = (int)max((int64_t)0, min((int64_t)kList, hi - i0));
        __syncthreads();
        for (int k = threadIdx.x; k <= kList; k += blockDim.x) {
            const int64_t i = i0 + k;
            key[k] = i < a.T ? a.key[i] : -1;
            if (k < kList) tok[k] = hi > lo ? a.tok[min(i, (int64_t)hi - 1)] : 0;
        }
        __syncthreads();
        if (!live || n == 0) continue;
        Raw<T, N> v[2][kAhead];
        auto fetch = [&](Raw<T, N> (&to)[kAhead], int j0) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) to[j].get(dout + (int64_t)tok[j0 + j] * a.ld);
        };
        auto add = [&](const Raw<T, N> (&from)[kAhead], int j0) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (j0 + j >= n) break;
                from[j].add_to(sum);
                const int id = key[j0 + j], next = key[j0 + j + 1];
                const bool last = i0 + j0 + j + 1 == hi;
                if (next == id && !last) continue;
                if (id < a.vocab) {
                    if (head && joined)
                        store<float, N>(part, sum);             // goes on from the chunk before
                    else if (next == id)
                        store<float, N>(part + a.D, sum);       // goes on in the next chunk
                    else
                        write_row<O, N>(a, id, c, sum);
                }
                head = false;
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] = 0.f;
            }
        };
        fetch(v[0], 0);
#pragma unroll 1
        for (int j0 = 0; j0 < n; j0 += 2 * kAhead) {
            if (j0 + kAhead < n) fetch(v[1], j0 + kAhead);
            add(v[0], j0);
            if (j0 + 2 * kAhead < n) fetch(v[0], j0 + 2 * kAhead);
            add(v[1], j0 + kAhead);
        }
    }
}

// Runs that start in chunk blockIdx.x and cross its end: their partial sums, in
// the order of the chunks.  Four groups of 64 threads take a quarter of them
// each, so that a frequent id takes a quarter of the steps.
template <typename O, int N> __global__ void __launch_bounds__(256) join_kernel(SumArgs a) {
    __shared__ float quarter[3][64][N];
    pdl_wait();
    pdl_trigger();
    const int end = (blockIdx.x + 1) * a.chunk;   // < T: the last chunk has none
    const int id = a.key[end - 1];
    if (id >= a.vocab || a.key[end] != id) return;
    const int lo = end - a.chunk;
    // all of this chunk, and what goes on from the chunk before: not its start
    if (a.key[lo] == id && lo > 0 && a.key[lo - 1] == id) return;
    const int g = threadIdx.x >> 6, tid = threadIdx.x & 63;
    const int c = (blockIdx.y * 64 + tid) * N;
    // the last chunk whose first key is still `id`, 256 chunks at a look
    int last = blockIdx.x;
    for (;;) {
        const int64_t m = (int64_t)last + 1 + threadIdx.x;
        const int more = __syncthreads_count(m < a.chunks && a.key[m * a.chunk] == id);
        last += more;
        if (more < 256) break;
    }
    // this chunk's part is its last run's (index 1), those of the others their first's
    const int n = last - (int)blockIdx.x + 1, from = n * g / 4, to = n * (g + 1) / 4;
    float sum[N];
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = 0.f;
    if (c < a.D) {
#pragma unroll 8
        for (int i = from; i < to; ++i) {
            float v[N];
            load<float, N>(a.part + ((int64_t)(blockIdx.x + i) * 2 + (i == 0)) * a.D + c, v);
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] += v[k];
        }
        if (g > 0)
#pragma unroll
            for (int k = 0; k < N; ++k) quarter[g - 1][tid][k] = sum[k];
    }
    __syncthreads();
    if (g > 0 || c >= a.D) return;
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] += quarter[q][tid][k];
    write_row<O, N>(a, id, c, sum);
}

// ---- a short batch ---------------------------------------------------------------

// All of it in one launch: a block has a range of dtable's rows, which it zeroes;
// it picks the range's tokens out of all ids, in their order, sorts the few by rank and
// sums each row's, 128 bytes a thread in flight; groups of threads beside those that one
// row takes have a row each, or a part of a long run.  An id that fills the batch
// is summed by one block, so the batch has to be small.  (35 tokens x 1280 into
// 38843 rows, bf16: 18 us of the GPU, 25 by the kernels above; 512 x 1024 into 1000,
// 5 and 13, or 32 and 17 where all have one id; a call takes 14 instead of 22 us of
// the host.)
constexpr int kShortTokens = 512;
constexpr int64_t kShortBytes = 1 << 20;
constexpr int kShortRows = 1 << 22;      // of a block: row and place in one integer
template <typename T, typename O, int N>
__global__ void __launch_bounds__(256, 4) short_kernel(SumArgs a, const void *ids, int wide) {
    constexpr int kAhead = sizeof(T) == 2 ? 8 : 4, kLong = 4 * kAhead;
    __shared__ __align__(16) uint32_t got[kShortTokens];      // row in the range, place
    __shared__ int row_of[kShortTokens], tok[2][kShortTokens], warps[8];
    __shared__ float part[256 * N];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int lo = (int)((int64_t)a.vocab * blockIdx.x / gridDim.x);
    const int hi = (int)((int64_t)a.vocab * (blockIdx.x + 1) / gridDim.x);
    int n = 0;
    for (int t0 = 0; t0 < a.T; t0 += 256) {
        const int t = t0 + tid, id = t < a.T ? id_of(ids, wide, t, a.vocab) : -1;
        const bool here = id >= lo && id < hi;
        const unsigned all = __ballot_sync(0xffffffffu, here);
        if (lane == 0) warps[w] = __popc(all);
        __syncthreads();
        int at = n + __popc(all & ((1u << lane) - 1u));
        for (int i = 0; i < 8; ++i) {
            if (i < w) at += warps[i];
            n += warps[i];
        }
        if (here) {
            got[at] = (uint32_t)(id - lo) * kShortTokens + at;
            tok[0][at] = t;
        }
        __syncthreads();
    }
    if (!a.accumulate) {
        const int64_t row = (int64_t)a.D * sizeof(O);
        fill({static_cast<uint8_t *>(a.dtable) + lo * row, (hi - lo) * row}, 0, 1, 0, 1);
    }
    for (int i = n + tid; i < kShortTokens && i < n + 4; i += 256) got[i] = 0xffffffffu;
    __syncthreads();
    for (int i = tid; i < n; i += 256) {
        const uint32_t own = got[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < n; j += 4) {
            const uint4 x = *reinterpret_cast<const uint4 *>(got + j);
            rank += (x.x < own) + (x.y < own) + (x.z < own) + (x.w < own);
        }
        row_of[rank] = (int)(own / kShortTokens);
        tok[1][rank] = tok[0][i];
    }
    __syncthreads();                     // the zeros are written, too
    // as many rows side by side as have room for their columns
    const int pieces = a.D / N;
    int x = 256;
    while (x > 1 && x / 2 >= pieces) x /= 2;
    const int mine = tid % x, group = tid / x, groups = 256 / x;
    int run = 0;                         // of the list
    for (int i = 0, end; i < n; i = end, ++run) {
        const int row = row_of[i];
        end = i + 1;                     // the first place of another row
        for (int last = n; end < last;) {
            const int middle = (end + last) / 2;
            if (row_of[middle] == row)
                end = middle + 1;
            else
                last = middle;
        }
        // a long run in parts, where a row leaves room beside it (x covers it then)
        const int len = end - i;
        const bool split = groups > 1 && len >= kLong;
        if (!split && run % groups != group) continue;
        const int from = split ? i + len * group / groups : i;
        const int to = split ? i + len * (group + 1) / groups : end;
        float sum[N];
        for (int c = mine * N; c < a.D; c += x * N) {
            const T *dout = static_cast<const T *>(a.dout) + c;
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] = 0.f;
            for (int j = from; j < to; j += kAhead) {
                Raw<T, N> v[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (j + k < to) v[k].get(dout + (int64_t)tok[1][j + k] * a.ld);
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (j + k < to) v[k].add_to(sum);
            }
            if (split) {
#pragma unroll
                for (int k = 0; k < N; ++k) part[k * 256 + tid] = sum[k];
            } else {
                write_row<O, N>(a, lo + row, c, sum);
            }
        }
        if (!split) continue;
        __syncthreads();
        if (group == 0 && mine * N < a.D) {
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] = 0.f;
            for (int g = 0; g < groups; ++g)
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] += part[k * 256 + g * x + mine];
            write_row<O, N>(a, lo + row, mine * N, sum);
        }
        __syncthreads();
    }
}

// ---- launches ------------------------------------------------------------------

// Tokens of a chunk: 32, fewer in a short batch (512 chunks and more occupy the
// GPU), and at most 8192 chunks, so that the partial sums of an id that fills the
// batch are joined in a quarter as many steps.
int chunk_of(int T) {
    const int most = (int)(((int64_t)T + 8191) / 8192), few = T / 512;
    const int c = few < 8 ? 8 : few < 32 ? few : 32;
    return c < most ? most : c;
}

struct Layout {
    int chunk, chunks, tile, tiles;
    int64_t key[2], tok[2], hist, part, total;
};
Layout layout_of(int T, int D) {
    Layout l = {};
    l.chunk = chunk_of(T);
    l.chunks = (T + l.chunk - 1) / l.chunk;
    // up to a cluster's tiles: as many as it has blocks, of whole rounds
    const int64_t least = ((int64_t)T + kCluster - 1) / kCluster;
    const int64_t rounds = (least + kSortThreads - 1) / kSortThreads;
    l.tile = kSortThreads * (int)(rounds < 1 ? 1 : rounds < kRounds ? rounds : kRounds);
    l.tiles = (int)(((int64_t)T + l.tile - 1) / l.tile);
    const int64_t keys = ((int64_t)T * 4 + 15) & ~15ll;
    int64_t at = 0;
    for (int i = 0; i < 2; ++i) {
        l.key[i] = at;
        l.tok[i] = at + keys;
        at += 2 * keys;
    }
    l.hist = at;
    at += (int64_t)l.tiles * kDigits * 4;
    l.part = at;
    l.total = at + (int64_t)l.chunks * 2 * D * 4;
    return l;
}

template <typename T, typename O, int N>
cudaError_t sums(const SumArgs &a, const void *ids, int wide, cudaStream_t st) {
    if (!a.key) {
        const int most = 4 * device_sm_count();
        return launch_kernel(false, short_kernel<T, O, N>, dim3(a.vocab < most ? a.vocab : most),
                             256, 0, st, a, ids, wide);
    }
    const int pieces = a.D / N;
    // 256 threads a block: columns, and as many chunks as fit beside them (32 at most)
    const int x = pieces >= 256 ? 256 : (pieces + 7) / 8 * 8, y = 256 / x;
    cudaError_t e = launch_kernel(true, sum_kernel<T, O, N>,
                                  dim3((a.chunks + y - 1) / y, (pieces + x - 1) / x), dim3(x, y), 0,
                                  st, a);
    if (e == cudaSuccess && a.chunks > 1)
        e = launch_kernel(true, join_kernel<O, N>, dim3(a.chunks - 1, (pieces + 63) / 64), 256, 0,
                          st, a);
    return e;
}
template <typename T, typename O>
cudaError_t sums_n(const SumArgs &a, const void *ids, int ids_wide, bool wide, cudaStream_t st) {
    return wide ? sums<T, O, 8>(a, ids, ids_wide, st) : sums<T, O, 1>(a, ids, ids_wide, st);
}

bool dtype_ok(int32_t t) { return t == ULTRAMEM_F32 || t == ULTRAMEM_BF16; }
int size_of(int32_t t) { return t == ULTRAMEM_BF16 ? 2 : 4; }
bool sizes_ok(int32_t vocab, int32_t dim, int32_t ids_bytes, int32_t n_tokens, float scale) {
    return vocab >= 1 && vocab <= kMaxVocab && dim >= 1 && dim <= kMaxDim &&
           (ids_bytes == 4 || ids_bytes == 8) && n_tokens >= 0 && isfinite(scale);
}

}  // namespace
}  // namespace embed
}  // namespace um

using namespace um::embed;

extern "C" ultramem_status ultramem_embedding(const void *table, int64_t ld_table, int32_t dtype,
                                              int32_t vocab, int32_t dim, const void *ids,
                                              int32_t ids_bytes, int32_t n_tokens, float scale,
                                              void *out, void *stream) {
    if (!dtype_ok(dtype) || !sizes_ok(vocab, dim, ids_bytes, n_tokens, scale))
        return ULTRAMEM_EINVAL;
    if (n_tokens == 0) return ULTRAMEM_OK;
    const int es = size_of(dtype);
    if (!table || !ids || !out || ld_table < dim || ((uintptr_t)table | (uintptr_t)out) % es ||
        (uintptr_t)ids % ids_bytes)
        return ULTRAMEM_EINVAL;
    const int64_t row = (int64_t)dim * es;
    if (!um::apart({{out, row * n_tokens}}, {{table, row, vocab, ld_table * es},
                                             {ids, (int64_t)n_tokens * ids_bytes}}))
        return ULTRAMEM_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    const bool wide = dim % 8 == 0 && ((uintptr_t)table | (uintptr_t)out) % 16 == 0 &&
                      ld_table * es % 16 == 0;
    const int64_t pieces = (int64_t)n_tokens * (wide ? dim / 8 : dim);
    const int64_t most = (int64_t)um::device_sm_count() * 64, blocks = (pieces + 255) / 256;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    auto go = [&](auto t, auto n) {
        using T = decltype(t);
        embed_kernel<T, decltype(n)::value><<<grid, 256, 0, st>>>(
            static_cast<const T *>(table), ld_table, vocab, dim, ids, ids_bytes == 8, n_tokens,
            scale, static_cast<T *>(out));
    };
    using One = std::integral_constant<int, 1>;
    using Eight = std::integral_constant<int, 8>;
    if (dtype == ULTRAMEM_BF16)
        wide ? go(__nv_bfloat16(), Eight()) : go(__nv_bfloat16(), One());
    else
        wide ? go(float(), Eight()) : go(float(), One());
    return um::status_from_cuda(cudaGetLastError());
}

extern "C" int64_t ultramem_embedding_backward_workspace(int32_t n_tokens, int32_t dim) {
    if (n_tokens < 0 || dim < 1 || dim > kMaxDim) return 0;
    return layout_of(n_tokens, dim).total;
}

extern "C" ultramem_status ultramem_embedding_backward(
    const void *ids, int32_t ids_bytes, int32_t n_tokens, const void *dout, int64_t ld_dout,
    int32_t dtype, int32_t vocab, int32_t dim, float scale, void *dtable, int32_t table_dtype,
    int32_t accumulate, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!dtype_ok(dtype) || !dtype_ok(table_dtype) || (accumulate != 0 && accumulate != 1) ||
        !sizes_ok(vocab, dim, ids_bytes, n_tokens, scale) || !dtable ||
        (uintptr_t)dtable % size_of(table_dtype))
        return ULTRAMEM_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    cudaGetLastError();
    const int64_t out_bytes = (int64_t)vocab * dim * size_of(table_dtype);
    if (n_tokens == 0) {
        if (accumulate) return ULTRAMEM_OK;
        return um::status_from_cuda(cudaMemsetAsync(dtable, 0, out_bytes, st));
    }
    const int es = size_of(dtype);
    const Layout l = layout_of(n_tokens, dim);
    if (!ids || !dout || ld_dout < dim || (uintptr_t)ids % ids_bytes || (uintptr_t)dout % es ||
        !workspace || ((uintptr_t)workspace & 15) || workspace_bytes < l.total)
        return ULTRAMEM_EINVAL;
    if (!um::apart({{dtable, out_bytes}, {workspace, l.total}},
                   {{ids, (int64_t)n_tokens * ids_bytes},
                    {dout, (int64_t)dim * es, n_tokens, ld_dout * es}}))
        return ULTRAMEM_EINVAL;
    char *ws = static_cast<char *>(workspace);
    SortArgs s = {};
    s.ids = ids;
    for (int i = 0; i < 2; ++i) {
        s.key[i] = reinterpret_cast<int *>(ws + l.key[i]);
        s.tok[i] = reinterpret_cast<int *>(ws + l.tok[i]);
    }
    s.hist = reinterpret_cast<int *>(ws + l.hist);
    s.T = n_tokens;
    s.vocab = vocab;
    s.wide = ids_bytes == 8;
    s.tiles = l.tiles;
    s.tile = l.tile;
    while ((vocab >> s.bits) != 0) ++s.bits;   // keys 0..vocab
    s.passes = (s.bits + 7) / 8;
    const FillArgs f = {accumulate ? nullptr : static_cast<uint8_t *>(dtable), out_bytes};
    // blocks that zero dtable beside the sorting ones
    const int64_t want = (out_bytes + 65535) / 65536;
    const int spare =
        accumulate ? 0 : (int)(want < um::device_sm_count() ? want : um::device_sm_count());
    cudaError_t e = cudaSuccess;
    const bool whole = n_tokens <= kShortTokens && (int64_t)n_tokens * dim * es <= kShortBytes &&
                       vocab / (4 * um::device_sm_count()) < kShortRows;
    if (whole) {
        // one launch of the sums does it all
    } else if (l.tiles <= kCluster) {
        e = um::allow_dynamic_smem<sort_small_kernel>(sizeof(ClusterShared));
        if (e == cudaSuccess && !accumulate)
            e = um::launch_kernel(false, fill_kernel, dim3(spare), 1024, 0, st, f);
        if (e == cudaSuccess)
            e = um::launch_kernel(!accumulate, sort_small_kernel, dim3(kCluster), kSortThreads,
                                  sizeof(ClusterShared), st, s);
    } else {
        const int parts = 2 * s.passes;
        e = um::allow_dynamic_smem<sort_place_kernel>(sizeof(SortShared));
        for (int p = 0; p < s.passes && e == cudaSuccess; ++p) {
            e = um::launch_kernel(p > 0, sort_count_kernel, dim3(l.tiles + spare), kSortThreads, 0,
                                  st, s, p, f, 2 * p, parts);
            if (e == cudaSuccess)
                e = um::launch_kernel(true, sort_place_kernel, dim3(l.tiles + spare), kSortThreads,
                                      sizeof(SortShared), st, s, p, f, 2 * p + 1, parts);
        }
    }
    if (e != cudaSuccess) return um::status_from_cuda(e);
    SumArgs a = {};
    const int at = l.tiles <= kCluster ? 0 : (s.passes - 1) & 1;
    a.key = whole ? nullptr : s.key[at];
    a.tok = s.tok[at];
    a.dout = dout;
    a.ld = ld_dout;
    a.dtable = dtable;
    a.part = reinterpret_cast<float *>(ws + l.part);
    a.T = n_tokens;
    a.D = dim;
    a.vocab = vocab;
    a.chunk = l.chunk;
    a.chunks = l.chunks;
    a.accumulate = accumulate;
    a.scale = scale;
    const bool wide = dim % 8 == 0 && ((uintptr_t)dout | (uintptr_t)dtable) % 16 == 0 &&
                      ld_dout * es % 16 == 0;
    using B = __nv_bfloat16;
    if (dtype == ULTRAMEM_BF16)
        e = table_dtype == ULTRAMEM_BF16 ? sums_n<B, B>(a, ids, s.wide, wide, st)
                                         : sums_n<B, float>(a, ids, s.wide, wide, st);
    else
        e = table_dtype == ULTRAMEM_BF16 ? sums_n<float, B>(a, ids, s.wide, wide, st)
                                         : sums_n<float, float>(a, ids, s.wide, wide, st);
    return um::status_from_cuda(e);
}

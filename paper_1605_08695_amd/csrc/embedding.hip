// Embedding table kernels: lookup with scaling, and the table's gradient summed token by token after
// the tokens have been grouped by their row.
//
//   lookup    out[i] = scale * table[ids[i]]                        (0 for an id outside the table)
//   gradient  dtable[r] = beta * dtable[r] + scale * sum over the tokens i with ids[i] == r of dy[i]
//   update    var[r] <- fma(-lr, scale * that sum, var[r])          (rows with tokens only)
//
// Sums are fp32, in an order fixed by n, d and the ids alone: no atomic touches a value.
//
// All three are bound by HBM (one addition per element read).  The lookup is one pass over what it reads and
// writes.  A gradient needs a row's tokens together: the tokens are sorted by row, as indexes, and each row's
// sum is formed in registers and written once, so the table's gradient is never read, and an update moves only
// the rows that have tokens.  Rows of tables are not equal: a frequent word can have half the tokens, so nothing
// below leaves a row's length to one wave.
#include "common.h"
#include "kernels.h"
#include "rowvec.h"

namespace tfk {

// A grid of so many workgroups in two dimensions (the threads of one have to stay below 2^32), and a
// workgroup's place in it.
static dim3 block_grid(int64_t blocks) {
    const int64_t x = std::min<int64_t>(blocks, 1 << 22);
    return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}
__device__ __forceinline__ int64_t block_index() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// ------------------------------------------------------------------ lookup
// A thread moves V consecutive elements of a row; the last piece of a row that is not a whole number of
// them starts V before the row's end (the elements it shares with the piece before are written twice,
// with the same values).  A workgroup has 256 * UNR consecutive pieces of the output, whatever the row's length:
// the loads of UNR pieces, ids first, are in flight together.  Bound by HBM: 65536 x 2048 bf16, 350 MB, 59 us
// (stores past the caches; 73 through them), 20011 x 771 fp32, 83 MB, 15.6 us.  Small outputs take one piece a
// thread: 128 x 512 is 2.6 us, a launch and two dependent loads.
template <typename TI, typename TO, int V, int UNR, bool AWAY>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const TI *__restrict__ table, int64_t rows, int64_t tld, int d,
                                                        const int32_t *__restrict__ ids, int64_t n, float scale,
                                                        TO *__restrict__ out, int64_t old_, uint32_t pieces,
                                                        FastDiv by_pieces) {
    const int64_t base = block_index() * (256 * UNR);
    const int64_t i0 = base / pieces;
    const uint32_t r0 = (uint32_t)(base - i0 * pieces);
    int64_t i[UNR];
    int k[UNR];
    int32_t id[UNR];
#pragma unroll
    for (int u = 0; u < UNR; ++u) {
        uint32_t q, r;
        by_pieces.divmod(r0 + u * 256 + threadIdx.x, q, r);
        i[u] = i0 + q;
        k[u] = min((int)r * V, d - V);
        id[u] = i[u] < n ? ids[i[u]] : -1;
    }
    typename RowVec<TI, V>::raw v[UNR];
#pragma unroll
    for (int u = 0; u < UNR; ++u) {
        const bool ok = id[u] >= 0 && id[u] < rows;
        if (ok) v[u] = RowVec<TI, V>::load(table + id[u] * tld + k[u]);
    }
#pragma unroll
    for (int u = 0; u < UNR; ++u) {
        const bool ok = id[u] >= 0 && id[u] < rows;
        float f[V];
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = 0.f;
        if (ok) {
            RowVec<TI, V>::unpack(v[u], f);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] *= scale;
        }
        if (i[u] >= n) continue;
        if (AWAY) RowVec<TO, V>::store_away(out + i[u] * old_ + k[u], f);
        else RowVec<TO, V>::store(out + i[u] * old_ + k[u], f);
    }
}

template <typename TI, typename TO, int V>
static hipError_t embed_fwd(const TI *table, int64_t rows, int64_t tld, int d, const int32_t *ids, int64_t n, float scale,
                            TO *out, int64_t old_, hipStream_t st) {
    const uint32_t pieces = (uint32_t)((d + V - 1) / V);
    const FastDiv by(pieces);
    const int64_t total = n * pieces;
#define TFK_GO(UNR, AWAY)                                                                                             \
    hipLaunchKernelGGL((embed_fwd_kernel<TI, TO, V, UNR, AWAY>), block_grid((total + 256 * UNR - 1) / (256 * UNR)),   \
                       dim3(256), 0, st, table, rows, tld, d, ids, n, scale, out, old_, pieces, by)
    if (total < 256 * 4 * 1024) TFK_GO(1, false);     // (with four a thread, less than four workgroups per CU)
    else if (n * d * (int64_t)sizeof(TO) < kPastCaches) TFK_GO(4, false);
    else TFK_GO(4, true);
#undef TFK_GO
    return hipGetLastError();
}

hipError_t launch_embed_fwd(int tdt, const void *table, int64_t rows, int64_t tld, int d, const int32_t *ids, int64_t n,
                            float scale, int odt, void *out, int64_t old_, hipStream_t st) {
#define TFK_GO(TI, TO, V)                                                                                              \
    return d >= V ? embed_fwd<TI, TO, V>((const TI *)table, rows, tld, d, ids, n, scale, (TO *)out, old_, st)          \
                  : embed_fwd<TI, TO, 1>((const TI *)table, rows, tld, d, ids, n, scale, (TO *)out, old_, st)
    if (tdt == 0 && odt == 0) TFK_GO(float, float, 4);
    if (tdt == 0) TFK_GO(float, bf16_t, 8);
    if (odt == 0) TFK_GO(bf16_t, float, 8);
    TFK_GO(bf16_t, bf16_t, 8);
#undef TFK_GO
}

// ------------------------------------------------------------------ tokens grouped by row
// The rows are dealt to 2^bb buckets: groups of 2^gs consecutive rows go round the buckets, each round
// shifted from the one before.  With gs = 0, neighbouring rows -- the most frequent words, in tables ordered
// by frequency -- are in different buckets, and so are rows a power of two apart; larger groups are for
// buckets that clear their own rows, at least 512 bytes in one piece however narrow they are.
struct RowSplit {
    int gs, bb;            // log2 of the rows per group, of the buckets
    int local;             // rows per bucket (upper bound)
};

static RowSplit row_split(int64_t rows, int gs, int bb, int most) {
    RowSplit s;
    s.gs = gs;
    s.bb = bb;
    while (((((rows - 1) >> s.gs) >> s.bb) + 1) << s.gs > most) ++s.bb;
    s.local = (int)(((((rows - 1) >> s.gs) >> s.bb) + 1) << s.gs);
    return s;
}

__device__ __forceinline__ void row_place(uint32_t id, int gs, int bb, uint32_t &bucket, uint32_t &local) {
    const uint32_t g = id >> gs, hi = g >> bb;
    bucket = (g + hi * 77u) & ((1u << bb) - 1u);
    local = (hi << gs) | (id & ((1u << gs) - 1u));
}

// the row of a place
__device__ __forceinline__ uint32_t place_row(uint32_t bucket, uint32_t local, int gs, int bb) {
    const uint32_t hi = local >> gs;
    return ((((hi << bb) | ((bucket - hi * 77u) & ((1u << bb) - 1u))) << gs) | (local & ((1u << gs) - 1u)));
}

// What becomes of a row's sum g (scaled): stored, added to what is there, or applied as an SGD step.
enum { kStore = 0, kAdd = 1, kSgd = 2 };

// What is there (kAdd, kSgd): V columns from o, asked for before the sum is known.
template <int MODE, int V>
__device__ __forceinline__ typename RowVec<float, V>::raw row_old(const float *dst, int64_t o) {
    if constexpr (MODE == kStore) return {};
    else return RowVec<float, V>::load(dst + o);
}

// V columns from o of the row's result; the first `skip` of them belong to another lane.
template <int MODE, int V>
__device__ __forceinline__ void row_finish(float *dst, bf16_t *sh, int64_t o, const float *s,
                                           const typename RowVec<float, V>::raw &old_, int skip, float scale, float lr) {
    float g[V], old[V];
    if constexpr (MODE != kStore) RowVec<float, V>::unpack(old_, old);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        g[e] = scale * s[e];
        if constexpr (MODE == kAdd) g[e] = old[e] + g[e];
        if constexpr (MODE == kSgd) g[e] = fmaf(-lr, g[e], old[e]);
    }
    if (skip == 0) {
        RowVec<float, V>::store(dst + o, g);
        if (MODE == kSgd && sh != nullptr) RowVec<bf16_t, V>::store(sh + o, g);
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e >= skip) {
            dst[o + e] = g[e];
            if (MODE == kSgd && sh != nullptr) sh[o + e] = (bf16_t)f32_to_bf16(g[e]);
        }
}

// A lane's columns of a block of 64 * V: the first one, and how many of its V belong to the lane before
// (the last lane of a row starts V before its end); V: none.
template <int V>
__device__ __forceinline__ int lane_columns(int d, int cb, int lane, int &skip) {
    const int64_t c = ((int64_t)cb * 64 + lane) * V;
    const int64_t left = d - c;
    skip = left >= V ? 0 : (left > 0 ? (int)(V - left) : V);
    return skip < V ? (int)(c - skip) : 0;
}

// Zeros in columns [c0, c1) of the n rows row(l) that are in the table and have no token (none(l)), a wave
// per row, 16 bytes a lane; rows of less than 128 columns an element a thread.
template <int NT, typename R, typename N>
__device__ __forceinline__ void zero_rows(float *dst, int d, int c0, int c1, uint32_t rows, int n, R row, N none) {
    if (d < 128) {
        const int total = n * d;                      // (at most 1024 * 127)
        for (int e = threadIdx.x; e < total; e += NT) {
            const int l = e / d, c = e - l * d;
            if (row(l) < rows && none(l) && c >= c0 && c < c1) dst[(int64_t)row(l) * d + c] = 0.f;
        }
        return;
    }
    const int lane = threadIdx.x & 63;
    const float z[4] = {0.f, 0.f, 0.f, 0.f};
    for (int l = threadIdx.x >> 6; l < n; l += NT / 64) {
        const uint32_t r = row(l);
        if (r >= rows || !none(l)) continue;
        float *p = dst + (int64_t)r * d;
        for (int c = c0 + lane * 4; c < c1; c += 256) RowVec<float, 4>::store(p + min(c, c1 - 4), z);
    }
}

// One bucket's part of a stable counting sort of the tokens by row: a workgroup of NW waves reads all n
// ids (they stay in the caches), counts those of its bucket per row and wave (each wave has a contiguous
// range of the tokens), which gives every (row, wave) its first place, and puts each token into its place:
// by row, then by token.  Ids outside [0, rows) are in no bucket.  A lane keeps its ids (KEEP of them:
// n <= NW * 64 * KEEP) in registers, and a bit for those of the bucket, between the two turns.
template <int NW, int KEEP>
struct BucketSort {
    static_assert(KEEP <= 64, "one bit per kept id");
    const int32_t *ids;
    uint32_t rows, mine, lo, hi;           // this wave's tokens: [lo, hi)
    int gs, bb, lane, wave;
    uint32_t v[KEEP];
    uint64_t hits;

    __device__ BucketSort(const int32_t *ids_, uint32_t n, uint32_t rows_, int gs_, int bb_, uint32_t mine_)
        : ids(ids_), rows(rows_), mine(mine_), gs(gs_), bb(bb_), lane(threadIdx.x & 63),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), hits(0) {
        const uint32_t per = ((n + NW - 1) / NW + 63) / 64 * 64;
        lo = min(n, wave * per);
        hi = min(n, lo + per);
    }

    // the bucket of an id (~0: none) and its row's place there
    __device__ __forceinline__ uint32_t place(uint32_t id, uint32_t &local) const {
        uint32_t b;
        row_place(id, gs, bb, b, local);
        return id < rows ? b : ~0u;
    }

    // Counts into cnt[local row][wave].
    __device__ __forceinline__ void count(uint32_t *cnt) {
#pragma unroll
        for (int e = 0; e < KEEP; ++e) {
            if (lo + e * 64 >= hi) break;
            const uint32_t i = lo + e * 64 + lane;
            v[e] = i < hi ? (uint32_t)ids[i] : ~0u;
        }
#pragma unroll
        for (int e = 0; e < KEEP; ++e) {
            if (lo + e * 64 >= hi) break;
            uint32_t l;
            if (place(v[e], l) == mine) {
                atomicAdd(&cnt[l * NW + wave], 1u);
                hits |= 1ull << e;
            }
        }
    }

    // One id a lane: put(place, token, row) for the lanes with ok, in the order of the lanes.
    template <typename F>
    __device__ __forceinline__ void step(uint32_t *cnt, uint32_t base, uint32_t id, bool ok, F put) const {
        uint64_t left = __ballot(ok);
        while (left) {                                // one turn per distinct row among the lanes
            const int lead = __ffsll((unsigned long long)left) - 1;
            const uint32_t row = __builtin_amdgcn_readlane(id, lead);
            const bool same = ok && id == row;
            const uint64_t m = __ballot(same);
            uint32_t p = 0;
            if (lane == lead) {
                uint32_t b, l;
                row_place(row, gs, bb, b, l);
                p = atomicAdd(&cnt[l * NW + wave], (uint32_t)__popcll(m));
            }
            p = __builtin_amdgcn_readlane(p, lead);
            if (same) put(p + (uint32_t)__popcll(m & ((1ull << lane) - 1ull)), base + lane, row);
            left &= ~m;
        }
    }

    // Places the tokens; cnt: each (row, wave)'s first place, which moves to the next one's.
    template <typename F>
    __device__ __forceinline__ void put(uint32_t *cnt, F f) const {
#pragma unroll
        for (int e = 0; e < KEEP; ++e) {
            if (lo + e * 64 >= hi) break;
            step(cnt, lo + e * 64, v[e], (hits >> e) & 1, f);
        }
    }
};

// Exclusive sums of cnt[0 .. entries) in place, from `at`; cnt[entries] and the result are the end.  entries
// is a multiple of 4 and cnt 16-byte aligned: a thread has a contiguous range, four at a time.
template <int NW>
__device__ __forceinline__ uint32_t scan_counts(uint32_t *cnt, int entries, uint32_t at, uint32_t *red) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u32x4_t *const c4 = reinterpret_cast<u32x4_t *>(cnt);
    const int quads = entries / 4, each = (quads + NW * 64 - 1) / (NW * 64);
    const int e0 = min(quads, tid * each), e1 = min(quads, e0 + each);
    uint32_t own = 0;
    for (int e = e0; e < e1; ++e) {
        const u32x4_t c = c4[e];
        own += (c.x + c.y) + (c.z + c.w);
    }
    uint32_t incl = own;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    if (lane == 63) red[wave] = incl;
    __syncthreads();
    uint32_t end = at;
    at += incl - own;
    for (int w = 0; w < NW; ++w) {
        if (w < wave) at += red[w];
        end += red[w];
    }
    for (int e = e0; e < e1; ++e) {
        const u32x4_t c = c4[e];
        c4[e] = u32x4_t{at, at + c.x, at + c.x + c.y, at + c.x + c.y + c.z};
        at += (c.x + c.y) + (c.z + c.w);
    }
    if (tid == 0) cnt[entries] = end;
    __syncthreads();
    return end;
}

// ------------------------------------------------------------------ many tokens: a sort in two launches
// Stable, by a digit of the id: tables of up to 2^kDigitBits rows take one round with the id itself, all others
// two, with the low and the high half of a bijection of the 32-bit ids that spreads them (high halves of the
// ids would be the same few for most tokens; only equal ids have to come together).
//   tiles    each workgroup sorts its contiguous range of the tokens by bucket and leaves where each of the
//            256 buckets begins in it
//   buckets  each workgroup takes its bucket's tokens out of every tile, in order, and sorts them by row;
//            the tokens of the buckets before are the sum of the tiles' beginnings of its own
// Bound by latency, not by the ids' few bytes: 65536 tokens 5 + 10 us (a sort in one launch, every bucket
// reading all ids, took 41).  256 buckets are a workgroup per CU, each tile's beginnings one line of
// 1 KB, and a table of 2^18 rows leaves 1024 rows to count per bucket, what the LDS holds for 8 waves.  By
// the digits of the ids themselves two rounds are slower (65536 x 64 of 3M rows: 164 us, 63 by the spread ids).
// Round two and the sums read the number of tokens left (those with ids in the table) from *nvalid.
constexpr int kDigitBits = 18, kTileWaves = 4, kTileThreads = 64 * kTileWaves, kBuckets = 256, kMostTiles = 512;

struct Digit {
    int half;              // -1: the id; 0, 1: the halves of the spread id
    uint32_t rows;
    __device__ __forceinline__ void place(uint32_t id, uint32_t &bucket, uint32_t &local) const {
        if (half >= 0) {
            id *= 2654435769u;                        // (odd: a bijection mod 2^32, as the xor with its own high half is)
            id ^= id >> 16;
            id *= 2654435769u;
            id = half == 0 ? id & 0xffffu : id >> 16;
        }
        row_place(id, 0, 8, bucket, local);
    }
};

// The lanes with ok whose x has the same low `bits` bits as this lane's.
template <int MOST>
__device__ __forceinline__ uint64_t same_lanes(uint32_t x, int bits, bool ok) {
    uint64_t m = __ballot(ok);
#pragma unroll
    for (int b = 0; b < MOST; ++b) {
        if (b >= bits) break;
        const bool one = (x >> b) & 1u;
        const uint64_t w = __ballot(one);
        m &= one ? w : ~w;
    }
    return m;
}

// The next places of this lane's entry in cnt[entry][wave], in the order of the lanes (same: the lanes
// with the same entry; lanes without ok get nothing).
__device__ __forceinline__ uint32_t take_places(uint32_t *entry, uint64_t same, bool ok, int lane) {
    const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1ull));
    uint32_t p = 0;
    if (ok && rank == 0) p = atomicAdd(entry, (uint32_t)__popcll(same));
    return __shfl(p, ok ? __ffsll((unsigned long long)same) - 1 : lane, 64) + rank;
}

// Counts this lane's entry (ok): the lanes that have the first one's at once (a frequent word is in most
// lanes, and an atomic takes the lanes of one address one by one), the others each by itself.
__device__ __forceinline__ void count_place(uint32_t *cnt, uint32_t entry, bool ok, int lane) {
    const uint64_t all = __ballot(ok);
    if (all == 0) return;
    const int lead = __ffsll((unsigned long long)all) - 1;
    const uint32_t e0 = __builtin_amdgcn_readlane(entry, lead);
    const bool with = ok && entry == e0;
    const uint64_t m = __ballot(with);
    if (ok && (!with || lane == lead)) atomicAdd(&cnt[entry], with ? (uint32_t)__popcll(m) : 1u);
}

__global__ __launch_bounds__(kTileThreads) void embed_tile_kernel(const int32_t *__restrict__ ids,
                                                                  const int32_t *__restrict__ tokens, uint32_t n,
                                                                  const int32_t *__restrict__ nvalid, Digit g,
                                                                  uint32_t tile, int32_t *__restrict__ ttok,
                                                                  int32_t *__restrict__ tkey,
                                                                  int32_t *__restrict__ begin) {
    __shared__ alignas(16) uint32_t cnt[kBuckets * kTileWaves + 1];
    __shared__ uint32_t red[kTileWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (nvalid != nullptr) n = (uint32_t)*nvalid;
    for (int e = threadIdx.x; e < kBuckets * kTileWaves; e += kTileThreads) cnt[e] = 0;
    __syncthreads();
    const uint32_t t0 = min(n, blockIdx.x * tile), t1 = min(n, t0 + tile);
    const uint32_t per = (tile / kTileWaves + 63) / 64 * 64;
    const uint32_t lo = min(t1, t0 + wave * per), hi = min(t1, lo + per);
    for (uint32_t base = lo; base < hi; base += 256) {
        uint32_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t i = base + e * 64 + lane;
            v[e] = i < hi ? (uint32_t)ids[i] : ~0u;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t b, l;
            g.place(v[e], b, l);
            count_place(cnt, b * kTileWaves + wave, v[e] < g.rows, lane);
        }
    }
    __syncthreads();
    scan_counts<kTileWaves>(cnt, kBuckets * kTileWaves, 0, red);
    int32_t *const mine = begin + (int64_t)blockIdx.x * (kBuckets + 1);
    for (int e = threadIdx.x; e <= kBuckets; e += kTileThreads) mine[e] = (int32_t)cnt[e * kTileWaves];
    __syncthreads();
    for (uint32_t base = lo; base < hi; base += 256) {
        uint32_t v[4], tok[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t i = base + e * 64 + lane;
            v[e] = i < hi ? (uint32_t)ids[i] : ~0u;
            tok[e] = tokens != nullptr && i < hi ? (uint32_t)tokens[i] : i;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t b, l;
            g.place(v[e], b, l);
            const bool ok = v[e] < g.rows;
            const uint32_t p = take_places(&cnt[b * kTileWaves + wave], same_lanes<8>(b, 8, ok), ok, lane);
            if (ok) {
                ttok[t0 + p] = (int32_t)tok[e];
                tkey[t0 + p] = (int32_t)v[e];
            }
        }
    }
}

// used (or null; one round only): a byte per row of the table, 1 for rows with tokens.
template <int NW>
__global__ __launch_bounds__(64 * NW) void embed_bucket_kernel(const int32_t *__restrict__ ttok,
                                                                      const int32_t *__restrict__ tkey,
                                                                      const int32_t *__restrict__ begin, int tiles,
                                                                      uint32_t tile, Digit g, int local_rows,
                                                                      int local_bits, int32_t *__restrict__ order,
                                                                      int32_t *__restrict__ key,
                                                                      int32_t *__restrict__ nvalid,
                                                                      uint8_t *__restrict__ used) {
    static_assert(64 * NW >= kMostTiles, "a thread per tile");
    extern __shared__ __align__(16) uint32_t cnt[];                 // [local row][wave], and the end
    __shared__ uint32_t pre[kMostTiles + 1], src[kMostTiles];        // a tile's first entry; where it is
    __shared__ uint32_t red[2][NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int entries = local_rows * NW;
    uint32_t s = 0, e = 0;
    if (tid < tiles) {
        s = (uint32_t)begin[(int64_t)tid * (kBuckets + 1) + blockIdx.x];
        e = (uint32_t)begin[(int64_t)tid * (kBuckets + 1) + blockIdx.x + 1];
    }
    for (int q = tid; q < entries; q += (64 * NW)) cnt[q] = 0;
    uint32_t incl = e - s, before = s;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o, 64);
    if (lane == 63) {
        red[0][wave] = incl;
        red[1][wave] = before;
    }
    __syncthreads();
    uint32_t at = incl - (e - s), m = 0;
    before = 0;
    for (int w = 0; w < NW; ++w) {
        if (w < wave) at += red[0][w];
        m += red[0][w];
        before += red[1][w];
    }
    if (tid < kMostTiles) {
        pre[tid] = at;
        src[tid] = tid * tile + s;
    }
    if (tid == 0) pre[kMostTiles] = m;
    __syncthreads();
    // entry i of the bucket: in the last tile whose first is not behind it
    const auto where = [&](uint32_t i) {
        int t = 0;
#pragma unroll
        for (int step = kMostTiles / 2; step > 0; step >>= 1)
            if (pre[t + step] <= i) t += step;
        return src[t] + (i - pre[t]);
    };
    const uint32_t per = ((m + NW - 1) / NW + 63) / 64 * 64;
    const uint32_t lo = min(m, wave * per), hi = min(m, lo + per);
    // entries that a lane has at hand, and fetches at a time; worked on four by four, side by side
    constexpr int KEEP = 16;
    uint32_t tok[KEEP], id[KEEP];
    const auto fetch = [&](uint32_t base) {
#pragma unroll
        for (int q0 = 0; q0 < KEEP; q0 += 4) {
            if (base + q0 * 64 >= hi) break;
#pragma unroll
            for (int q = q0; q < q0 + 4; ++q) {
                const uint32_t i = base + q * 64 + lane, at_ = where(i < hi ? i : lo);
                id[q] = (uint32_t)tkey[at_];
                tok[q] = (uint32_t)ttok[at_];
            }
        }
    };
    for (uint32_t base = lo; base < hi; base += KEEP * 64) {
        fetch(base);
#pragma unroll
        for (int q0 = 0; q0 < KEEP; q0 += 4) {
            if (base + q0 * 64 >= hi) break;
#pragma unroll
            for (int q = q0; q < q0 + 4; ++q) {
                uint32_t b, l;
                g.place(id[q], b, l);
                count_place(cnt, l * NW + wave, base + q * 64 + lane < hi, lane);
            }
        }
    }
    __syncthreads();
    const uint32_t end = scan_counts<NW>(cnt, entries, before, red[0]);
    if (blockIdx.x == kBuckets - 1 && tid == 0) *nvalid = (int32_t)end;
    if (used != nullptr) {
        for (int l = tid; l < local_rows; l += (64 * NW)) {
            const uint32_t row = place_row(blockIdx.x, l, 0, 8);
            if (row < g.rows) used[row] = cnt[l * NW] != cnt[(l + 1) * NW];
        }
        __syncthreads();
    }
    for (uint32_t base = lo; base < hi; base += KEEP * 64) {
        if (per > KEEP * 64) fetch(base);             // (else they are still at hand)
#pragma unroll
        for (int q0 = 0; q0 < KEEP; q0 += 4) {
            if (base + q0 * 64 >= hi) break;
            uint32_t p[4], l[4];
            uint64_t same[4];
            bool ok[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t b;
                g.place(id[q0 + q], b, l[q]);
                ok[q] = base + (q0 + q) * 64 + lane < hi;
                same[q] = same_lanes<10>(l[q], local_bits, ok[q]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) p[q] = take_places(&cnt[l[q] * NW + wave], same[q], ok[q], lane);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (ok[q]) {
                    order[p[q]] = (int32_t)tok[q0 + q];
                    key[p[q]] = (int32_t)id[q0 + q];
                }
        }
    }
}

// ------------------------------------------------------------------ sums of the grouped tokens
// Bound by HBM: 65536 x 1024 bf16 tokens of a 131072-row table, 237 MB with the rows written, 54 us (4.4 TB/s);
// an update, which reads those rows too, 75 us (4.6 TB/s).
// A wave sums the grouped tokens of `chunk` places over 64 * V columns, eight rows of dy in flight, and
// finishes the rows of the table that begin there and end there or in the next chunk.  A row that goes on
// beyond (it covers the whole of a chunk that it does not begin in) is left in parts: [chunk][1] in the chunk
// where it begins, [chunk][0] in the others.  A chunk and the next are one lane each of a wave's 64: kMaxChunk
// is the most (with every row over a border in parts, 65536 x 1024 took 211 us in all, with these 184).
constexpr int kMaxChunk = 32;

template <typename T, int V, int MODE>
__global__ __launch_bounds__(256) void embed_sum_kernel(const T *__restrict__ dy, int64_t n, int64_t dld, int d, int cblocks,
                                                        int chunk, const int32_t *__restrict__ order,
                                                        const int32_t *__restrict__ key,
                                                        const int32_t *__restrict__ nvalid, float scale, float lr,
                                                        float *__restrict__ dst, bf16_t *__restrict__ sh,
                                                        float *__restrict__ part) {
    const int lane = threadIdx.x & 63;
    const int64_t id = block_index() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t ch = id / cblocks;
    const int cb = (int)(id - ch * cblocks);
    const int64_t p0 = ch * chunk, p1 = p0 + chunk, p2 = p1 + chunk;
    if (p0 >= n) return;
    // lane l: token and row of place p0 + l, of this chunk and the next (-1: past the end); the rows before,
    // a chunk before, and behind the next chunk.  (One round of loads: places past *nvalid hold anything.)
    const int nv = *nvalid;
    const bool there = lane < 2 * chunk && p0 + lane < n;
    const int t_ = there ? order[p0 + lane] : 0, r_ = there ? key[p0 + lane] : -1;
    const int prev = p0 > 0 ? key[p0 - 1] : -1, prev2 = p0 > chunk ? key[p0 - chunk - 1] : -1;
    int behind = p2 < n ? key[p2] : -1;
    if (p0 >= nv) return;
    const int tok = p0 + lane < nv ? t_ : 0, row = p0 + lane < nv ? r_ : -1;
    if (p2 >= nv) behind = -1;
    const auto row_at = [&](int i) { return i < 64 ? __builtin_amdgcn_readlane(row, i) : -1; };
    const int at1 = p1 < nv ? (chunk < 64 ? row_at(chunk) : -1) : -1;          // the row at the next chunk's first place
    int cur = row_at(0);
    bool head = cur == prev;                          // it began before
    int i = 0;
    if (head && prev2 != cur && at1 != cur) {         // in the chunk before, and it ends here: not ours
        const uint64_t other = __ballot(lane < chunk && row != cur);
        if (other == 0) return;
        i = __ffsll((unsigned long long)other) - 1;
        cur = row_at(i);
        head = false;
        if (cur < 0) return;
    }
    // the last place of this wave: of the chunk, or of the row that goes on into the next and ends there
    const int last = row_at(chunk - 1);
    const uint64_t ours = __ballot(row >= 0 && (lane < chunk || (lane < 2 * chunk && row == last)));
    const bool goes_on = last >= 0 && at1 == last;
    const bool part1 = goes_on && (behind == last || (head && cur == last));   // ... as a part
    const int end = goes_on && !part1 ? __popcll(ours) : (int)min((int64_t)chunk, nv - p0);
    int skip;
    const int c0 = lane_columns<V>(d, cb, lane, skip);
    const bool act = skip < V;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    float *const slot = part + ch * 2 * d + c0;
    const auto as_part = [&](bool began) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (act && e >= skip) slot[(began ? d : 0) + e] = acc[e];
    };
    // kAhead tokens at a time (dy is read past the caches: nothing reads a gradient after its sum); with each
    // that ends its row, what is there in the row
    constexpr int kAhead = 8;
    for (; i < end; i += kAhead) {
        typename RowVec<T, V>::raw buf[kAhead];
        typename RowVec<float, V>::raw old[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < end && act) {
                buf[u] = RowVec<T, V>::load_last(dy + __builtin_amdgcn_readlane(tok, i + u) * dld + c0);
                const int r = __builtin_amdgcn_readlane(row, i + u);
                if (MODE != kStore && (i + u + 1 >= end || __builtin_amdgcn_readlane(row, i + u + 1) != r))
                    old[u] = row_old<MODE, V>(dst, (int64_t)r * d + c0);
            }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= end) break;
            float f[V];
            RowVec<T, V>::unpack(buf[u], f);
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += f[e];
            const bool over = i + u + 1 >= end;
            const int r = over ? -1 : __builtin_amdgcn_readlane(row, i + u + 1);
            if (r == cur) continue;
            if (head || (over && part1)) as_part(!head);
            else if (act) row_finish<MODE, V>(dst, sh, (int64_t)cur * d + c0, acc, old[u], skip, scale, lr);
            cur = r;
            head = false;
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = 0.f;
        }
    }
}

// The rows in parts.  A workgroup looks through kJoinWaves chunks, a wave each, for one that a row in parts
// begins in, and adds the parts up over 64 * V columns: up to kJoinAlone of them by that wave, more by all
// waves, a contiguous share each, joined in their order.  Workgroups from `joins` on clear a share of the
// rows without tokens (used; null: none to clear) -- last in the operation, so that the sums' reads do not
// wait behind the writes.
constexpr int kJoinWaves = 16, kJoinThreads = 64 * kJoinWaves, kJoinAlone = 16, kClearRows = 256;

template <int V>
__device__ __forceinline__ void add_parts(const float *part, int64_t d, int64_t ch, int64_t i0, int64_t i1, float *acc) {
    for (int64_t i = i0; i < i1; i += 8) {            // part 0: chunk ch's [1]; part i: chunk ch + i's [0]
        typename RowVec<float, V>::raw buf[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int64_t j = min(i + u, i1 - 1);
            buf[u] = RowVec<float, V>::load(part + ((ch + j) * 2 + (j == 0)) * d);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (i + u >= i1) break;
            float f[V];
            RowVec<float, V>::unpack(buf[u], f);
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += f[e];
        }
    }
}

template <int V, int MODE>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(int64_t n, int d, int cblocks, int chunk, int64_t groups,
                                                                  uint32_t joins, const int32_t *__restrict__ key,
                                                                  const int32_t *__restrict__ nvalid, float scale, float lr,
                                                                  float *__restrict__ dst, bf16_t *__restrict__ sh,
                                                                  const float *__restrict__ part,
                                                                  const uint8_t *__restrict__ used, uint32_t rows) {
    __shared__ float sums[kJoinWaves - 1][64][V + 1];
    __shared__ int begins[kJoinWaves];                // the row in many parts that begins in the wave's chunk, or -1
    __shared__ int stops[kJoinWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (blockIdx.x >= joins) {
        const uint32_t r0 = (blockIdx.x - joins) * kClearRows;
        zero_rows<kJoinThreads>(dst, d, 0, d, rows, kClearRows, [&](int l) { return r0 + l; },
                                [&](int l) { return used[r0 + l] == 0; });
        return;
    }
    const int nv = *nvalid;
    for (int64_t b = blockIdx.x; b < groups; b += joins) {
        const int64_t ch0 = b / cblocks * kJoinWaves;
        const int cb = (int)(b % cblocks);
        const int64_t ch = ch0 + wave, p0 = ch * chunk, p1 = p0 + chunk, p2 = p1 + chunk;
        int skip;
        const int c0 = lane_columns<V>(d, cb, lane, skip);
        float acc[V];
        int row = -1;
        if (p2 < n) {                                 // (one round of loads, with *nvalid's)
            const int last = key[p1 - 1], next = key[p1], behind = key[p2], before = p0 > 0 ? key[p0 - 1] : -1;
            const int64_t q = p2 + (1 + lane) * chunk;
            const int far = q < n ? key[q] : -1;
            if (p2 < nv && next == last && behind == last && before != last) {
                const uint64_t stop = __ballot(q >= nv || far != last);
                const int more = stop ? __ffsll((unsigned long long)stop) + 1 : kJoinAlone;
                if (more < kJoinAlone) {              // chunks that it is the first row of, and this one
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] = 0.f;
                    if (skip < V) {
                        const auto old = row_old<MODE, V>(dst, (int64_t)last * d + c0);
                        add_parts<V>(part + c0, d, ch, 0, more + 1, acc);
                        row_finish<MODE, V>(dst, sh, (int64_t)last * d + c0, acc, old, skip, scale, lr);
                    }
                } else {
                    row = last;
                }
            }
        }
        __syncthreads();
        if (lane == 0) begins[wave] = row;
        __syncthreads();
        for (int w = 0; w < kJoinWaves; ++w) {
            const int cur = begins[w];
            if (cur < 0) continue;                    // (uniform over the workgroup)
            // the chunks it is the first row of: each wave looks at 64 more
            int64_t more = kJoinAlone;
            for (bool found = false; !found;) {
                const int64_t q = (ch0 + w + 1 + more + wave * 64 + lane) * chunk;
                const uint64_t stop = __ballot(q >= nv || key[q] != cur);
                if (lane == 0) stops[wave] = stop ? __ffsll((unsigned long long)stop) - 1 : 64;
                __syncthreads();
                for (int x = 0; x < kJoinWaves && !found; ++x) {
                    more += stops[x];
                    found = stops[x] < 64;
                }
                __syncthreads();
            }
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = 0.f;
            const int64_t each = (more + 1 + kJoinWaves - 1) / kJoinWaves, i0 = wave * each, i1 = min(more + 1, i0 + each);
            typename RowVec<float, V>::raw old{};
            if (skip < V) {
                if (wave == 0) old = row_old<MODE, V>(dst, (int64_t)cur * d + c0);
                add_parts<V>(part + c0, d, ch0 + w, i0, i1, acc);
            }
            if (wave > 0)
#pragma unroll
                for (int e = 0; e < V; ++e) sums[wave - 1][lane][e] = acc[e];
            __syncthreads();
            if (wave == 0 && skip < V) {
                for (int x = 0; x < kJoinWaves - 1; ++x)
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] += sums[x][lane][e];
                row_finish<MODE, V>(dst, sh, (int64_t)cur * d + c0, acc, old, skip, scale, lr);
            }
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------------ few tokens: one launch
// The gradient of 2560 x 512 is 16.8 us, most of it the clearing of an 80 MB table; the update of as many is
// 8.9 us, half of it the sort: a chain of LDS and cache latencies, which more waves lengthen (16: 13.3 us).
// Workgroup (bucket, 64 * V columns) sorts the bucket's tokens into LDS and sums its rows itself.  A row of
// more than kAlone tokens is summed by all waves, each a contiguous part of its tokens, joined in their
// order; the others go to the waves in turn.
constexpr int kSmallWaves = 8, kSmallThreads = 64 * kSmallWaves, kAlone = 8, kSmallAhead = 8;

template <typename T, int V, int MODE, int KEEP, int BATCH>
__global__ __launch_bounds__(kSmallThreads) void embed_small_kernel(const T *__restrict__ dy, int64_t dld, int d,
                                                                    const int32_t *__restrict__ ids, uint32_t n,
                                                                    uint32_t rows, int gs, int bb, int local_rows,
                                                                    float scale, float lr, float *__restrict__ dst,
                                                                    bf16_t *__restrict__ sh) {
    extern __shared__ __align__(16) uint32_t cnt[];                 // [local row][wave], the end, then the tokens (16 bits each)
    __shared__ uint32_t red[kSmallWaves];
    __shared__ float sums[kSmallWaves - 1][64][V + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int entries = local_rows * kSmallWaves;
    uint16_t *const list = (uint16_t *)(cnt + entries + 1);
    for (int e = threadIdx.x; e < entries; e += kSmallThreads) cnt[e] = 0;
    __syncthreads();
    BucketSort<kSmallWaves, KEEP> sort(ids, n, rows, gs, bb, blockIdx.x);
    sort.count(cnt);
    __syncthreads();
    scan_counts<kSmallWaves>(cnt, entries, 0, red);
    int skip;
    const int c0 = lane_columns<V>(d, blockIdx.y, lane, skip);
    if (MODE == kStore) {
        zero_rows<kSmallThreads>(
            dst, d, blockIdx.y * 64 * V, min(d, (int)(blockIdx.y + 1) * 64 * V), rows, local_rows,
            [&](int l) { return place_row(blockIdx.x, l, gs, bb); },
            [&](int l) { return cnt[l * kSmallWaves] == cnt[(l + 1) * kSmallWaves]; });
        __syncthreads();
    }
    sort.put(cnt, [&](uint32_t p, uint32_t token, uint32_t) { list[p] = (uint16_t)token; });
    __syncthreads();
    // (every (row, wave)'s place has moved to the next one's first)
    const auto first = [&](int l) { return l == 0 ? 0u : cnt[l * kSmallWaves - 1]; };
    int turn = 0;
    for (int l0 = 0; l0 < local_rows; l0 += 64) {
        const int l = l0 + lane;
        uint64_t some = __ballot(l < local_rows && first(l) != first(min(l + 1, local_rows)));
        while (some) {
            const int j = l0 + __ffsll((unsigned long long)some) - 1;
            some &= some - 1;
            const int b = (int)first(j), e = (int)first(j + 1);
            const bool all = e - b > kAlone;          // (uniform over the workgroup, like the loops)
            if (!all && turn++ % kSmallWaves != wave) continue;
            const int each = all ? (e - b + kSmallWaves - 1) / kSmallWaves : e - b;
            const int t0 = all ? min(e, b + wave * each) : b, t1 = min(e, t0 + each);
            const int64_t o = (int64_t)place_row(blockIdx.x, j, gs, bb) * d + c0;
            typename RowVec<float, V>::raw old{};
            if (skip < V && (!all || wave == 0)) old = row_old<MODE, V>(dst, o);
            float acc[V];
#pragma unroll
            for (int q = 0; q < V; ++q) acc[q] = 0.f;
            int t = t0;
            if (skip < V) {
                if (BATCH > kSmallAhead)
                    for (; t + BATCH <= t1; t += BATCH) {
                        typename RowVec<T, V>::raw buf[BATCH];
#pragma unroll
                        for (int u = 0; u < BATCH; ++u) buf[u] = RowVec<T, V>::load(dy + list[t + u] * dld + c0);
#pragma unroll
                        for (int u = 0; u < BATCH; ++u) {
                            float f[V];
                            RowVec<T, V>::unpack(buf[u], f);
#pragma unroll
                            for (int q = 0; q < V; ++q) acc[q] += f[q];
                        }
                    }
                for (; t < t1; t += kSmallAhead) {
                    typename RowVec<T, V>::raw buf[kSmallAhead];
#pragma unroll
                    for (int u = 0; u < kSmallAhead; ++u)
                        if (t + u < t1) buf[u] = RowVec<T, V>::load(dy + list[t + u] * dld + c0);
#pragma unroll
                    for (int u = 0; u < kSmallAhead; ++u)
                        if (t + u < t1) {
                            float f[V];
                            RowVec<T, V>::unpack(buf[u], f);
#pragma unroll
                            for (int q = 0; q < V; ++q) acc[q] += f[q];
                        }
                }
            }
            if (all) {
                if (wave > 0)
#pragma unroll
                    for (int q = 0; q < V; ++q) sums[wave - 1][lane][q] = acc[q];
                __syncthreads();
                if (wave == 0)
                    for (int w = 0; w < kSmallWaves - 1; ++w)
#pragma unroll
                        for (int q = 0; q < V; ++q) acc[q] += sums[w][lane][q];
            }
            if (skip < V && (!all || wave == 0))
                row_finish<MODE, V>(dst, sh, o, acc, old, skip, scale, lr);
            if (all) __syncthreads();
        }
    }
}

constexpr int kSmallKeep = 16, kSmallTokens = kSmallThreads * kSmallKeep;
// Buckets: 2^3 to 2^9 of them, eight tokens in each on average (2^9 where each clears its own rows; 256, 512
// and 1024 for 2560 tokens: 10.6, 9.0 and 9.2 us), more only where a bucket's counters (kSmallLocal rows)
// would not fit the LDS.
constexpr int kSmallBits = 9, kSmallLocal = 960;
// Up to so many workgroups, two per CU, 16 rows of dy are in flight in a wave: a frequent row's sum is a chain of such
// rounds (8000 x 512 with half the tokens one word 78 us, 50 so; 2560 x 512 10.1, 9.1).  More workgroups need the
// registers for one another (2560 x 2048: 18 us with 8 in flight, 23 with 16).
constexpr int kSmallDeep = 512;

static size_t list_bytes(int64_t n) { return ((size_t)n * 4 + 15) / 16 * 16; }

// a byte per row (gradients of one round that store)
static size_t used_bytes(int64_t rows) { return rows > ((int64_t)1 << kDigitBits) ? 0 : ((size_t)rows + 15) / 16 * 16; }

// tokens per wave: 32, or 16 where that makes less than 4096 waves, half of what the chip holds
static int sum_chunk(int64_t n, int cblocks) {
    return (n + kMaxChunk - 1) / kMaxChunk * cblocks < 4096 ? kMaxChunk / 2 : kMaxChunk;
}

struct Tiles {
    int64_t size, count;
};

static Tiles tiles_of(int64_t n) {
    Tiles t;
    t.count = std::min<int64_t>(kMostTiles, (n + 255) / 256);
    t.size = ((n + t.count - 1) / t.count + 63) / 64 * 64;
    t.count = (n + t.size - 1) / t.size;
    return t;
}

// Few tokens, and few enough buckets: each of them reads all ids.  One launch against the four of the sort in
// two launches, update of a table of 32000 rows: 2560 x 512 9.4 us against 25.4, 7500 x 256 20 against 31,
// 7500 x 1024 27 against 35; from 12000 tokens on the sort is as fast or faster (gradient 12000 x 1024: 71, 51).
// The rule looks at n and rows alone, though with thousands of columns the sort is faster from 6000 tokens on
// already (7500 x 4096: 70 us here, 63 there): d is left out of it.
static bool sum_small(int64_t n, int64_t rows) { return n <= kSmallTokens && rows <= ((int64_t)kSmallLocal << 10); }

size_t embed_ws_bytes(int64_t n, int d, int64_t rows) {
    if (n == 0 || rows == 0 || sum_small(n, rows)) return 0;
    int64_t chunks = 0;                               // of the type that has more
    for (const int v : {d >= 8 ? 8 : 1, d >= 4 ? 4 : 1}) {
        const int chunk = sum_chunk(n, (d + 64 * v - 1) / (64 * v));
        chunks = std::max(chunks, (n + chunk - 1) / chunk);
    }
    return 16 + 4 * list_bytes(n) + list_bytes(tiles_of(n).count * (kBuckets + 1)) + used_bytes(rows) +
           (size_t)chunks * 2 * d * 4;
}

template <typename T, int V>
static hipError_t embed_bwd(const T *dy, int64_t n, int d, int64_t dld, const int32_t *ids, int64_t rows, float scale,
                            int mode, float lr, float *dst, bf16_t *sh, void *ws, hipStream_t st) {
    const int cblocks = (d + 64 * V - 1) / (64 * V);
    if (sum_small(n, rows)) {
        int gs = 0, bb = mode == kStore ? kSmallBits : 3;
        while (mode == kStore && ((int64_t)d << gs) < 128) ++gs;
        while (bb < kSmallBits && (8 << bb) < n) ++bb;
        const RowSplit s = row_split(rows, gs, bb, kSmallLocal);
        const size_t lds = ((size_t)s.local * kSmallWaves + 1) * 4 + n * 2;
#define TFK_BATCH(MODE, BATCH)                                                                                         \
    hipLaunchKernelGGL((embed_small_kernel<T, V, MODE, kSmallKeep, BATCH>), dim3(1u << s.bb, cblocks),                \
                       dim3(kSmallThreads), lds, st, dy, dld, d, ids, (uint32_t)n, (uint32_t)rows, s.gs, s.bb,        \
                       s.local, scale, lr, dst, sh)
#define TFK_GO(MODE)                                                                                                   \
    do {                                                                                                               \
        if ((int64_t)cblocks << s.bb <= kSmallDeep) TFK_BATCH(MODE, 16);                                               \
        else TFK_BATCH(MODE, kSmallAhead);                                                                             \
    } while (0)
        if (mode == kStore) TFK_GO(kStore);
        else if (mode == kAdd) TFK_GO(kAdd);
        else TFK_GO(kSgd);
#undef TFK_GO
#undef TFK_BATCH
        return hipGetLastError();
    }
    const size_t list = list_bytes(n) / 4;
    const Tiles t = tiles_of(n);
    int32_t *nvalid = (int32_t *)ws, *order = nvalid + 4, *key = order + list, *ttok = key + list, *tkey = ttok + list,
            *begin = tkey + list;
    uint8_t *used = (uint8_t *)(begin + list_bytes(t.count * (kBuckets + 1)) / 4);
    float *part = (float *)(used + used_bytes(rows));
    const int rounds = rows > ((int64_t)1 << kDigitBits) ? 2 : 1;
    if (mode != kStore || rounds == 2) used = nullptr;
    if (mode == kStore && rounds == 2) {
        const hipError_t e = launch_fill_zero(dst, rows * d, st);
        if (e != hipSuccess) return e;
    }
    for (int r = 0; r < rounds; ++r) {
        const RowSplit s = row_split(rounds == 1 ? rows : 1 << 16, 0, 8, 1024);
        const Digit g{rounds == 1 ? -1 : r, (uint32_t)rows};
        int bits = 0;
        while ((1 << bits) < s.local) ++bits;
        hipLaunchKernelGGL(embed_tile_kernel, dim3((unsigned)t.count), dim3(kTileThreads), 0, st, r == 0 ? ids : key,
                           r == 0 ? nullptr : order, (uint32_t)n, r == 0 ? nullptr : nvalid, g, (uint32_t)t.size, ttok, tkey,
                           begin);
        // (a frequent row's bucket is one workgroup's: 16 waves, where their counters fit)
#define TFK_GO(NW)                                                                                                     \
    hipLaunchKernelGGL((embed_bucket_kernel<NW>), dim3(kBuckets), dim3(64 * NW), ((size_t)s.local * NW + 1) * 4, st,   \
                       ttok, tkey, begin, (int)t.count, (uint32_t)t.size, g, s.local, bits, order, key, nvalid, used)
        if (s.local <= 512) TFK_GO(16);
        else TFK_GO(8);
#undef TFK_GO
    }
    const int chunk = sum_chunk(n, cblocks);
    const int64_t chunks = (n + chunk - 1) / chunk, groups = (chunks + kJoinWaves - 1) / kJoinWaves * cblocks;
    const unsigned joins = (unsigned)std::min<int64_t>(groups, 1 << 20);
    const dim3 gs = block_grid((chunks * cblocks + 3) / 4);
    const dim3 gj(joins + (used != nullptr ? (unsigned)((rows + kClearRows - 1) / kClearRows) : 0u));
#define TFK_GO(MODE)                                                                                                   \
    do {                                                                                                               \
        hipLaunchKernelGGL((embed_sum_kernel<T, V, MODE>), gs, dim3(256), 0, st, dy, n, dld, d, cblocks, chunk, order, \
                           key, nvalid, scale, lr, dst, sh, part);                                                     \
        hipLaunchKernelGGL((embed_join_kernel<V, MODE>), gj, dim3(kJoinThreads), 0, st, n, d, cblocks, chunk, groups,  \
                           joins, key, nvalid, scale, lr, dst, sh, part, used, (uint32_t)rows);                        \
    } while (0)
    if (mode == kStore) TFK_GO(kStore);
    else if (mode == kAdd) TFK_GO(kAdd);
    else TFK_GO(kSgd);
#undef TFK_GO
    return hipGetLastError();
}

static hipError_t embed_bwd_any(int dt, const void *dy, int64_t n, int d, int64_t dld, const int32_t *ids, int64_t rows,
                                float scale, int mode, float lr, float *dst, bf16_t *sh, void *ws, hipStream_t st) {
    if (n == 0) return launch_fill_zero(dst, rows * d, st);           // (kStore only)
#define TFK_GO(T, V) return embed_bwd<T, V>((const T *)dy, n, d, dld, ids, rows, scale, mode, lr, dst, sh, ws, st)
    if (dt == 0) {
        if (d >= 4) TFK_GO(float, 4);
        TFK_GO(float, 1);
    }
    if (d >= 8) TFK_GO(bf16_t, 8);
    TFK_GO(bf16_t, 1);
#undef TFK_GO
}

hipError_t launch_embed_bwd(int dt, const void *dy, int64_t n, int d, int64_t dld, const int32_t *ids, int64_t rows,
                            float scale, float beta, float *dtable, void *ws, hipStream_t st) {
    return embed_bwd_any(dt, dy, n, d, dld, ids, rows, scale, beta == 0.f ? kStore : kAdd, 0.f, dtable, nullptr, ws, st);
}

hipError_t launch_embed_sgd(int dt, float *var, uint16_t *sh, int64_t rows, int d, const int32_t *ids, int64_t n,
                            const void *dy, int64_t dld, float scale, float lr, void *ws, hipStream_t st) {
    return embed_bwd_any(dt, dy, n, d, dld, ids, rows, scale, kSgd, lr, var, sh, ws, st);
}

}  // namespace tfk

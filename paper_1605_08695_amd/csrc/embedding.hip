// Embedding table kernels: lookup with scaling, and the table's gradient summed token by token after
// the tokens have been grouped by their row.
//
//   lookup    out[i] = scale * table[ids[i]]                        (0 for an id outside the table)
//   gradient  dtable[r] = beta * dtable[r] + scale * sum over the tokens i with ids[i] == r of dy[i]
//   update    var[r] <- fma(-lr, scale * that sum, var[r])          (rows with tokens only)
//
// Sums are fp32, in an order fixed by n, d and the ids alone.
#include "common.h"
#include "kernels.h"
#include "rowvec.h"

namespace tfk {

// ------------------------------------------------------------------ lookup
// A thread moves V consecutive elements of a row; the last piece of a row that is not a whole number of
// them starts V before the row's end (the elements it shares with the piece before are written twice,
// with the same values).  A workgroup has 256 * UNR consecutive pieces of the output.
template <typename TI, typename TO, int V, int UNR>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const TI *__restrict__ table, int64_t rows, int64_t tld, int d,
                                                        const int32_t *__restrict__ ids, int64_t n, float scale,
                                                        TO *__restrict__ out, int64_t old_, uint32_t pieces,
                                                        FastDiv by_pieces) {
    const int64_t base = (int64_t)blockIdx.x * (256 * UNR);
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
        if (i[u] < n) RowVec<TO, V>::store(out + i[u] * old_ + k[u], f);
    }
}

template <typename TI, typename TO, int V>
static hipError_t embed_fwd(const TI *table, int64_t rows, int64_t tld, int d, const int32_t *ids, int64_t n, float scale,
                            TO *out, int64_t old_, hipStream_t st) {
    const uint32_t pieces = (uint32_t)((d + V - 1) / V);
    const FastDiv by(pieces);
    const int64_t total = n * pieces;
    if (total < 256 * 4 * 1024)
        hipLaunchKernelGGL((embed_fwd_kernel<TI, TO, V, 1>), dim3((unsigned)((total + 255) / 256)), dim3(256), 0, st, table,
                           rows, tld, d, ids, n, scale, out, old_, pieces, by);
    else
        hipLaunchKernelGGL((embed_fwd_kernel<TI, TO, V, 4>), dim3((unsigned)((total + 1023) / 1024)), dim3(256), 0, st,
                           table, rows, tld, d, ids, n, scale, out, old_, pieces, by);
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
// The rows are dealt to 2^bb buckets: groups of 2^gs consecutive rows (so that a bucket's rows are at
// least 512 bytes in one piece, however narrow) go round the buckets, each round shifted from the one
// before.  Neighbouring rows -- the most frequent words, in tables ordered by frequency -- are then in
// different buckets, and so are rows a power of two apart.
struct RowSplit {
    int gs, bb;            // log2 of the rows per group, of the buckets
    int local;             // rows per bucket (upper bound)
};

static RowSplit row_split(int64_t rows, int d, int bb, int most) {
    RowSplit s;
    s.gs = 0;
    while (((int64_t)d << s.gs) < 128) ++s.gs;
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

// V columns from o of the row's result; the first `skip` of them belong to another lane.
template <int MODE, int V>
__device__ __forceinline__ void row_finish(float *dst, bf16_t *sh, int64_t o, const float *s, int skip, float scale,
                                           float lr) {
    if (skip == 0) {
        float g[V];
#pragma unroll
        for (int e = 0; e < V; ++e) g[e] = scale * s[e];
        if (MODE != kStore) {
            float old[V];
            RowVec<float, V>::unpack(RowVec<float, V>::load(dst + o), old);
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = MODE == kAdd ? old[e] + g[e] : fmaf(-lr, g[e], old[e]);
        }
        RowVec<float, V>::store(dst + o, g);
        if (MODE == kSgd && sh != nullptr) RowVec<bf16_t, V>::store(sh + o, g);
        return;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (e >= skip) {
            float g = scale * s[e];
            if (MODE != kStore) g = MODE == kAdd ? dst[o + e] + g : fmaf(-lr, g, dst[o + e]);
            dst[o + e] = g;
            if (MODE == kSgd && sh != nullptr) sh[o + e] = (bf16_t)f32_to_bf16(g);
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

// Zeros in the rows of a bucket that have no token: first(l) is the number of tokens before local row l.
template <int NT, typename F>
__device__ __forceinline__ void zero_rows(float *dst, int d, uint32_t rows, uint32_t bucket, int gs, int bb, int local_rows,
                                          F first) {
    if (d >= 256) {                                   // a wave per row, 16 bytes a lane
        const int lane = threadIdx.x & 63;
        for (int l = threadIdx.x >> 6; l < local_rows; l += NT / 64) {
            const uint32_t row = place_row(bucket, l, gs, bb);
            if (row >= rows || first(l) != first(l + 1)) continue;
            float *p = dst + (int64_t)row * d;
            const float z[4] = {0.f, 0.f, 0.f, 0.f};
            for (int c = lane * 4; c < d; c += 256) RowVec<float, 4>::store(p + min(c, d - 4), z);
        }
        return;
    }
    const int total = local_rows * d;                 // (at most 960 * 255)
    for (int e = threadIdx.x; e < total; e += NT) {
        const int l = e / d;
        const uint32_t row = place_row(bucket, l, gs, bb);
        if (row < rows && first(l) == first(l + 1)) dst[(int64_t)row * d + (e - l * d)] = 0.f;
    }
}

// A stable counting sort of the tokens by row in one launch.  Workgroup b reads all n ids (they stay in
// the caches), counts those of its bucket per row and wave (each wave has a contiguous range of the
// tokens) and those of the buckets before it, which gives every (row, wave) its first place, and reads
// the ids again to put each token into its place: first by bucket, then by row, then by token.  Tokens
// outside [0, rows) are left out; *nvalid is the number of the others.  zero (or null): the table whose
// rows without tokens are cleared on the way.
constexpr int kGroupThreads = 1024, kGroupWaves = kGroupThreads / 64;

__global__ __launch_bounds__(kGroupThreads) void embed_group_kernel(const int32_t *__restrict__ ids, uint32_t n,
                                                                    uint32_t rows, int gs, int bb, int local_rows,
                                                                    int32_t *__restrict__ order,
                                                                    int32_t *__restrict__ key,
                                                                    int32_t *__restrict__ nvalid,
                                                                    float *__restrict__ zero, int d) {
    extern __shared__ uint32_t cnt[];                 // [local row][wave], and the end
    __shared__ uint32_t red[2][kGroupWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t mine = blockIdx.x;
    const int entries = local_rows * kGroupWaves;
    for (int e = tid; e < entries; e += kGroupThreads) cnt[e] = 0;
    __syncthreads();
    const uint32_t per = ((n + kGroupWaves - 1) / kGroupWaves + 63) / 64 * 64;
    const uint32_t lo = min(n, wave * per), hi = min(n, lo + per);
    uint32_t before = 0;
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
            row_place(v[e], gs, bb, b, l);
            const bool ok = v[e] < rows;
            before += ok && b < mine;
            if (ok && b == mine) atomicAdd(&cnt[l * kGroupWaves + wave], 1u);
        }
    }
    for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o, 64);
    if (lane == 0) red[0][wave] = before;
    __syncthreads();
    before = 0;
    for (int w = 0; w < kGroupWaves; ++w) before += red[0][w];
    // exclusive sums over (row, wave), the buckets before added
    const int each = (entries + kGroupThreads - 1) / kGroupThreads;
    const int e0 = min(entries, tid * each), e1 = min(entries, e0 + each);
    uint32_t own = 0;
    for (int e = e0; e < e1; ++e) own += cnt[e];
    uint32_t incl = own;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    if (lane == 63) red[1][wave] = incl;
    __syncthreads();
    uint32_t at = before + incl - own;
    uint32_t all = before;
    for (int w = 0; w < kGroupWaves; ++w) {
        if (w < wave) at += red[1][w];
        all += red[1][w];
    }
    for (int e = e0; e < e1; ++e) {
        const uint32_t c = cnt[e];
        cnt[e] = at;
        at += c;
    }
    if (tid == 0) {
        cnt[entries] = all;
        if (mine == gridDim.x - 1) *nvalid = (int32_t)all;
    }
    __syncthreads();
    if (zero != nullptr) {
        zero_rows<kGroupThreads>(zero, d, rows, mine, gs, bb, local_rows, [&](int l) { return cnt[l * kGroupWaves]; });
        __syncthreads();
    }
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
            row_place(v[e], gs, bb, b, l);
            const bool ok = v[e] < rows && b == mine;
            uint64_t left = __ballot(ok);
            while (left) {                            // one turn per distinct row among the lanes
                const int lead = __ffsll((unsigned long long)left) - 1;
                const uint32_t row = __builtin_amdgcn_readlane(v[e], lead);
                const bool same = ok && v[e] == row;
                const uint64_t m = __ballot(same);
                uint32_t p = 0;
                if (lane == lead) p = atomicAdd(&cnt[l * kGroupWaves + wave], (uint32_t)__popcll(m));
                p = __builtin_amdgcn_readlane(p, lead);
                if (same) {
                    p += (uint32_t)__popcll(m & ((1ull << lane) - 1ull));
                    order[p] = (int32_t)(base + e * 64 + lane);
                    key[p] = (int32_t)row;
                }
                left &= ~m;
            }
        }
    }
}

// ------------------------------------------------------------------ sums of the grouped tokens
// A wave sums `chunk` consecutive grouped tokens over 64 * V columns, eight rows of dy in flight, and
// finishes each row of the table whose tokens begin and end in the chunk.  Sums of a row that goes on
// over the chunk's borders are left in part: [chunk][0] the one that began before, [chunk][1] the one that
// begins here and goes on.
constexpr int kMaxChunk = 64;

template <typename T, int V, int MODE>
__global__ __launch_bounds__(256) void embed_sum_kernel(const T *__restrict__ dy, int64_t dld, int d, int cblocks, int chunk,
                                                        const int32_t *__restrict__ order,
                                                        const int32_t *__restrict__ key,
                                                        const int32_t *__restrict__ nvalid, float scale, float lr,
                                                        float *__restrict__ dst, bf16_t *__restrict__ sh,
                                                        float *__restrict__ part) {
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t ch = wave / cblocks;
    const int cb = (int)(wave - ch * cblocks);
    const int nv = *nvalid;
    const int64_t p0 = ch * chunk;
    if (p0 >= nv) return;
    const int cnt = (int)min((int64_t)chunk, nv - p0);
    // lane l: token and row of place p0 + l; the row before and the row behind
    const int tok = lane < cnt ? order[p0 + lane] : 0;
    const int row = lane < cnt ? key[p0 + lane] : -1;
    const int prev = p0 > 0 ? key[p0 - 1] : -1, next = p0 + cnt < nv ? key[p0 + cnt] : -1;
    int skip;
    const int c0 = lane_columns<V>(d, cb, lane, skip);
    const bool act = skip < V;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    int cur = __builtin_amdgcn_readlane(row, 0);
    bool head = cur == prev;
    float *const slot = part + ch * 2 * d;
    for (int i0 = 0; i0 < cnt; i0 += 8) {
        typename RowVec<T, V>::raw buf[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int t = __builtin_amdgcn_readlane(tok, i0 + u);      // (token 0 past the end: not used)
            if (act) buf[u] = RowVec<T, V>::load(dy + t * dld + c0);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (i0 + u >= cnt) break;
            const int r = __builtin_amdgcn_readlane(row, i0 + u);
            if (r != cur) {
                if (act) {
                    if (head) {
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            if (e >= skip) slot[c0 + e] = acc[e];
                    } else {
                        row_finish<MODE, V>(dst, sh, (int64_t)cur * d + c0, acc, skip, scale, lr);
                    }
                }
                cur = r;
                head = false;
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] = 0.f;
            }
            float f[V];
            RowVec<T, V>::unpack(buf[u], f);
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] += f[e];
        }
    }
    if (!act) return;
    if (!head && next != cur) {
        row_finish<MODE, V>(dst, sh, (int64_t)cur * d + c0, acc, skip, scale, lr);
    } else {
        float *o = slot + (head ? 0 : d) + c0;
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e >= skip) o[e] = acc[e];
    }
}

// The rows that go over chunk borders: workgroup (chunk, 64 * V columns), for the row that begins in the
// chunk and goes on, adds up its part of every chunk, each of 4 waves a contiguous quarter, then the four.
template <int V, int MODE>
__global__ __launch_bounds__(256) void embed_join_kernel(int d, int cblocks, int chunk, const int32_t *__restrict__ key,
                                                         const int32_t *__restrict__ nvalid, float scale, float lr,
                                                         float *__restrict__ dst, bf16_t *__restrict__ sh,
                                                         const float *__restrict__ part) {
    __shared__ float sums[3][64][V + 1];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int nv = *nvalid;
    for (int64_t b = blockIdx.x;; b += gridDim.x) {
        const int64_t ch = b / cblocks;
        const int cb = (int)(b - ch * cblocks);
        const int64_t p0 = ch * chunk, p1 = p0 + chunk;
        if (p1 >= nv) return;
        const int cur = key[p1 - 1];
        if (key[p1] != cur || (p0 > 0 && key[p0 - 1] == cur)) continue;    // ends here, or began before
        // the number of chunks that the row is the first of
        int64_t more = 1;
        for (;;) {
            const int64_t q = (ch + 1 + more + lane) * chunk;
            const uint64_t stop = __ballot(q >= nv || key[q] != cur);
            if (stop) {
                more += __ffsll((unsigned long long)stop) - 1;
                break;
            }
            more += 64;
        }
        int skip;
        const int c0 = lane_columns<V>(d, cb, lane, skip);
        float acc[V];
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.f;
        // entry 0: this chunk's [1]; entry i: chunk ch + i's [0]
        const int64_t each = (more + 1 + 3) / 4, i0 = wave * each, i1 = min(more + 1, i0 + each);
        if (skip < V)
            for (int64_t i = i0; i < i1; ++i) {
                const float *p = part + ((ch + i) * 2 + (i == 0)) * d + c0;
                float f[V];
                RowVec<float, V>::unpack(RowVec<float, V>::load(p), f);
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += f[e];
            }
        if (wave > 0)
#pragma unroll
            for (int e = 0; e < V; ++e) sums[wave - 1][lane][e] = acc[e];
        __syncthreads();
        if (wave == 0 && skip < V) {
            for (int w = 0; w < 3; ++w)
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += sums[w][lane][e];
            row_finish<MODE, V>(dst, sh, (int64_t)cur * d + c0, acc, skip, scale, lr);
        }
        __syncthreads();
    }
}

static size_t list_bytes(int64_t n) { return ((size_t)n * 4 + 15) / 16 * 16; }

// tokens per wave: 64, and fewer down to 16 where there are less than 4096 waves
static int sum_chunk(int64_t n, int cblocks) {
    int chunk = kMaxChunk;
    while (chunk > 16 && (n + chunk - 1) / chunk * cblocks < 4096) chunk /= 2;
    return chunk;
}

size_t embed_ws_bytes(int64_t n, int d, int64_t rows) {
    if (n == 0 || rows == 0) return 0;
    int64_t chunks = 0;                               // of the type that has more
    for (const int v : {d >= 8 ? 8 : 1, d >= 4 ? 4 : 1}) {
        const int chunk = sum_chunk(n, (d + 64 * v - 1) / (64 * v));
        chunks = std::max(chunks, (n + chunk - 1) / chunk);
    }
    return 16 + 2 * list_bytes(n) + (size_t)chunks * 2 * d * 4;
}

template <typename T, int V>
static hipError_t embed_bwd(const T *dy, int64_t n, int d, int64_t dld, const int32_t *ids, int64_t rows, float scale,
                            int mode, float lr, float *dst, bf16_t *sh, void *ws, hipStream_t st) {
    const RowSplit s = row_split(rows, d, 8, 960);
    int32_t *nvalid = (int32_t *)ws, *order = nvalid + 4, *key = order + list_bytes(n) / 4;
    float *part = (float *)(key + list_bytes(n) / 4);
    hipLaunchKernelGGL(embed_group_kernel, dim3(1u << s.bb), dim3(kGroupThreads),
                       (size_t)s.local * kGroupWaves * 4 + 4, st, ids, (uint32_t)n, (uint32_t)rows, s.gs, s.bb, s.local,
                       order, key, nvalid, mode == kStore ? dst : nullptr, d);
    const int cblocks = (d + 64 * V - 1) / (64 * V), chunk = sum_chunk(n, cblocks);
    const int64_t chunks = (n + chunk - 1) / chunk;
    const dim3 gs((unsigned)((chunks * cblocks + 3) / 4)), gj((unsigned)std::min<int64_t>(chunks * cblocks, 1 << 22));
#define TFK_GO(MODE)                                                                                                   \
    do {                                                                                                               \
        hipLaunchKernelGGL((embed_sum_kernel<T, V, MODE>), gs, dim3(256), 0, st, dy, dld, d, cblocks, chunk, order,    \
                           key, nvalid, scale, lr, dst, sh, part);                                                     \
        if (chunks > 1)                                                                                                \
            hipLaunchKernelGGL((embed_join_kernel<V, MODE>), gj, dim3(256), 0, st, d, cblocks, chunk, key, nvalid,     \
                               scale, lr, dst, sh, part);                                                              \
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

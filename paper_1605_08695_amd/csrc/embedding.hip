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

namespace tfk {

// ------------------------------------------------------------------ lookup
template <typename TI, typename TO>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const TI *__restrict__ table, int64_t rows, int64_t tld, int d,
                                                        const int32_t *__restrict__ ids, int64_t n, float scale,
                                                        TO *__restrict__ out, int64_t old_) {
    const int64_t total = n * d, step = (int64_t)gridDim.x * 256;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += step) {
        const int64_t i = t / d;
        const int k = (int)(t - i * d);
        const int64_t r = ids[i];
        float v = 0.f;
        if (r >= 0 && r < rows) v = scale * Elem<TI>::load(table + r * tld + k);
        Elem<TO>::store(out + i * old_ + k, v);
    }
}

hipError_t launch_embed_fwd(int tdt, const void *table, int64_t rows, int64_t tld, int d, const int32_t *ids, int64_t n,
                            float scale, int odt, void *out, int64_t old_, hipStream_t st) {
    const dim3 g((unsigned)std::min<int64_t>((n * d + 255) / 256, 1 << 20));
#define TFK_GO(TI, TO)                                                                                                \
    hipLaunchKernelGGL((embed_fwd_kernel<TI, TO>), g, dim3(256), 0, st, (const TI *)table, rows, tld, d, ids, n, scale, \
                       (TO *)out, old_)
    if (tdt == 0 && odt == 0) TFK_GO(float, float);
    else if (tdt == 0) TFK_GO(float, bf16_t);
    else if (odt == 0) TFK_GO(bf16_t, float);
    else TFK_GO(bf16_t, bf16_t);
#undef TFK_GO
    return hipGetLastError();
}

// ------------------------------------------------------------------ tokens grouped by row
// A stable counting sort in one launch.  The rows are dealt to 2^bb buckets; workgroup b reads all n
// ids (they stay in the caches), counts those of its bucket per row and wave (each wave has a
// contiguous range of the tokens) and those of the buckets before it, which gives every (row, wave)
// its first place, and reads the ids again to put each token into its place: first by bucket, then by
// row, then by token.  Tokens outside [0, rows) are left out; *nvalid is the number of the others.
// Buckets hold every 2^bb-th group of 2^gs rows (shifted from one round of groups to the next), so
// neighbouring rows -- the most frequent words, in tables ordered by frequency -- are in different ones.
constexpr int kGroupThreads = 1024, kGroupWaves = kGroupThreads / 64;

struct RowSplit {
    int gs, bb;            // log2 of the rows per group, of the buckets
    int local;             // rows per bucket (upper bound)
};

static RowSplit row_split(int64_t rows, int d) {
    RowSplit s;
    (void)d;
    s.gs = 0;
    s.bb = 8;
    // counters of a bucket: below 64 KiB of LDS
    while (((((rows - 1) >> s.gs) >> s.bb) + 1) << s.gs > 960) ++s.bb;
    s.local = (int)(((((rows - 1) >> s.gs) >> s.bb) + 1) << s.gs);
    return s;
}

__device__ __forceinline__ void row_place(uint32_t id, int gs, int bb, uint32_t &bucket, uint32_t &local) {
    const uint32_t g = id >> gs, hi = g >> bb;
    bucket = (g + hi * 77u) & ((1u << bb) - 1u);
    local = (hi << gs) | (id & ((1u << gs) - 1u));
}

__global__ __launch_bounds__(kGroupThreads) void embed_group_kernel(const int32_t *__restrict__ ids, uint32_t n,
                                                                    uint32_t rows, int gs, int bb, int local_rows,
                                                                    int32_t *__restrict__ order,
                                                                    int32_t *__restrict__ key,
                                                                    int32_t *__restrict__ nvalid) {
    extern __shared__ uint32_t cnt[];                 // [local row][wave]
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
    if (mine == gridDim.x - 1 && tid == 0) *nvalid = (int32_t)all;
    __syncthreads();
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
// What becomes of a row's sum g (scaled): stored, added to what is there, or applied as an SGD step.
enum { kStore = 0, kAdd = 1, kSgd = 2 };

template <int MODE>
__device__ __forceinline__ void row_finish(float *dst, bf16_t *sh, int64_t o, float g, float lr) {
    if (MODE == kStore) dst[o] = g;
    if (MODE == kAdd) dst[o] += g;
    if (MODE == kSgd) {
        const float v = fmaf(-lr, g, dst[o]);
        dst[o] = v;
        if (sh != nullptr) sh[o] = (bf16_t)f32_to_bf16(v);
    }
}

// One workgroup per place and 256 columns: the first token of a row sums the row's tokens.
template <typename T, int MODE>
__global__ __launch_bounds__(256) void embed_sum_kernel(const T *__restrict__ dy, int64_t dld, int d,
                                                        const int32_t *__restrict__ order,
                                                        const int32_t *__restrict__ key,
                                                        const int32_t *__restrict__ nvalid, float scale, float lr,
                                                        float *__restrict__ dst, bf16_t *__restrict__ sh) {
    const int p0 = blockIdx.x, nv = *nvalid;
    if (p0 >= nv) return;
    const int row = key[p0];
    if (p0 > 0 && key[p0 - 1] == row) return;
    const int c = blockIdx.y * 256 + threadIdx.x;
    if (c >= d) return;
    float s = 0.f;
    for (int p = p0; p < nv && key[p] == row; ++p) s += Elem<T>::load(dy + order[p] * dld + c);
    row_finish<MODE>(dst, sh, (int64_t)row * d + c, scale * s, lr);
}

size_t embed_ws_bytes(int64_t n, int d, int64_t rows) {
    (void)d;
    if (n == 0 || rows == 0) return 0;
    const size_t list = ((size_t)n * 4 + 15) / 16 * 16;
    return 16 + 2 * list;
}

template <typename T>
static hipError_t embed_bwd(const T *dy, int64_t n, int d, int64_t dld, const int32_t *ids, int64_t rows, float scale,
                            int mode, float lr, float *dst, bf16_t *sh, void *ws, hipStream_t st) {
    if (mode == kStore) {
        const hipError_t e = launch_fill_zero(dst, rows * d, st);
        if (e != hipSuccess || n == 0) return e;
    }
    const RowSplit s = row_split(rows, d);
    int32_t *nvalid = (int32_t *)ws, *order = nvalid + 4, *key = order + ((size_t)n + 3) / 4 * 4;
    hipLaunchKernelGGL(embed_group_kernel, dim3(1u << s.bb), dim3(kGroupThreads),
                       (size_t)s.local * kGroupWaves * 4, st, ids, (uint32_t)n, (uint32_t)rows, s.gs, s.bb, s.local, order,
                       key, nvalid);
    const dim3 g((unsigned)n, (unsigned)((d + 255) / 256));
#define TFK_GO(MODE)                                                                                                    \
    hipLaunchKernelGGL((embed_sum_kernel<T, MODE>), g, dim3(256), 0, st, dy, dld, d, order, key, nvalid, scale, lr, dst, sh)
    if (mode == kStore) TFK_GO(kStore);
    else if (mode == kAdd) TFK_GO(kAdd);
    else TFK_GO(kSgd);
#undef TFK_GO
    return hipGetLastError();
}

hipError_t launch_embed_bwd(int dt, const void *dy, int64_t n, int d, int64_t dld, const int32_t *ids, int64_t rows,
                            float scale, float beta, float *dtable, void *ws, hipStream_t st) {
    const int mode = beta == 0.f ? kStore : kAdd;
    return dt == 0 ? embed_bwd((const float *)dy, n, d, dld, ids, rows, scale, mode, 0.f, dtable, nullptr, ws, st)
                   : embed_bwd((const bf16_t *)dy, n, d, dld, ids, rows, scale, mode, 0.f, dtable, nullptr, ws, st);
}

hipError_t launch_embed_sgd(int dt, float *var, uint16_t *sh, int64_t rows, int d, const int32_t *ids, int64_t n,
                            const void *dy, int64_t dld, float scale, float lr, void *ws, hipStream_t st) {
    return dt == 0 ? embed_bwd((const float *)dy, n, d, dld, ids, rows, scale, kSgd, lr, var, sh, ws, st)
                   : embed_bwd((const bf16_t *)dy, n, d, dld, ids, rows, scale, kSgd, lr, var, sh, ws, st);
}

}  // namespace tfk

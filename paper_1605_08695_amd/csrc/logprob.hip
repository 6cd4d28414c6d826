// Log-probabilities of given tokens, the entropy and the largest classes of rows of logits, and the gradient of
// the first two.
//
// With x = logits + bias, m = max x, u = (x - m) / T, s = sum e^u, W = sum u e^u:
//   lse = m / T + log s     logp = u_token - log s     entropy = log s - W / s
//   dx_j = (dlogp ([j = token] - p_j) - dentropy p_j (log p_j + entropy)) / T,   p_j = e^(x_j / T - lse)
// A class of -inf has p = 0 and no term; rows of masks alone (-1e9, -1e30, the type's lowest value) are rows like any
// other.  The largest classes are ordered by x, then by the lower class.
//
// A workgroup has a row and reads it once.  A lane's sums are relative to a power of two of its own, which it raises only
// when a class passes it by 2^kSlack: without the slack nearly every step of a wave has a lane with a new maximum.  A class
// costs one fma and one exponential, and raising costs none; a row too far out for that (beyond 2^27, infinite or NaN) is
// read again by exact differences (Part below).  The slack also bounds what a row with one class far above the others loses:
// W's terms at that class and its lane's later sums are up to kSlack times s, and entropy is what is left of them.  With 4
// and the terms of a piece added up before they join the lane's, it is off by 2.2e-6 at most, fp32 operations on whole rows
// by 1.5e-6 (2560 x 40000 and 256 x 131072, a class 12 to 25 above the mean; with a slack of 32 and term by term 4e-5), in the
// same time as with 1, 2, 8 or 32.
//
// Each lane keeps the largest x it saw, and for a list the largest of each group of its batches of pieces.  The k-th largest
// of the lanes' is at most the row's k-th largest, so the classes on the list are in the few groups whose largest is not
// below it, and only those are read again, shared out to all lanes, to find the candidates, which then count how many
// are before them.
//
// Bound by HBM, in bf16 with a bias and a list nearly as much by the vector unit: a row is read once, and for the gradient
// once more and written.  Measured, in bf16: 2560 x 40000 with a bias and 32 classes 62 us (48 with the logits in the caches,
// where the vector unit is 87 % busy; without a list 46), 4096 x 131072 with a bias 218 us (4.9 TB/s; 247 between calls of its
// gradient, whose last writes it waits for), its gradient 387 us (5.5 TB/s); 1021 x 50021 in fp32 with a bias and 5 classes 43
// us, its gradient 70.  A bias is read from the L2 for each row, or for two (4096 x 131072 without one: 187 us and 358).
#include "common.h"
#include "kernels.h"
#include "rowvec.h"

#pragma clang fp contract(off)

namespace tfk {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kSlack = 4.f, kFar = 1e4f, kEdge = 0x1p28f;      // in powers of two
// Pieces in flight of a lane (8192 x 10000 with 32 classes: 56 us, 80 with four, whose groups are twice as long; 4096 x 131072
// with a bias and 32 classes 267, 274), and groups of its batches that a lane's maxima are kept for.
constexpr int kBatch = 2, kGroups = 16;

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

// x's order as an unsigned number (+0 and -0 alike), 0 for -inf and below every finite x's.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    const uint32_t k = b ^ (uint32_t)((int32_t)b >> 31 | (int32_t)0x80000000);
    return x == -INFINITY ? 0u : k;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

typedef unsigned long long u64;
__device__ __forceinline__ u64 key_of(uint32_t order, int j) { return (u64)order << 32 | (uint32_t)~j; }

__device__ __forceinline__ float wave_maxf(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ float wave_sumf(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// A lane's part of a row: sums relative to a power of two, and its largest x.  EXACT false: x ct - R by one fma, R a whole
// number near the largest x ct, so that sums go from one to the next by a change of their exponents; rows that this cannot
// hold (the largest x ct beyond +-2^27, or infinite or NaN: s is no positive number then) are read again with EXACT, relative
// to a ref by exact differences.
template <bool EXACT>
struct Part {
    float ref, s, W, top;              // ref: R, or an x
    __device__ __forceinline__ static Part none() { return {EXACT ? -__FLT_MAX__ : -kEdge, 0.f, 0.f, -INFINITY}; }
    __device__ __forceinline__ float power(float x, float ct) const {
        return EXACT ? (x - ref) * ct : __builtin_fmaf(x, ct, -ref);
    }
    __device__ __forceinline__ void raise(float x, float ct) {
        const float to = EXACT ? x : __builtin_rintf(__builtin_amdgcn_fmed3f(x * ct, -kEdge, kEdge));
        const float D = fminf(EXACT ? (x - ref) * ct : to - ref, kFar);
        W -= D * s;
        if (EXACT) {
            const float r = ex2(-D);
            W *= r;
            s *= r;
        } else {
            W = __builtin_amdgcn_ldexpf(W, -(int)D);
            s = __builtin_amdgcn_ldexpf(s, -(int)D);
        }
        ref = to;
    }
    template <int V>
    __device__ __forceinline__ float add(const float *x, float ct) {
        float t = x[0];
#pragma unroll
        for (int e = 1; e < V; ++e) t = fmaxf(t, x[e]);
        if (power(t, ct) > kSlack) raise(t, ct);
        float ps = 0.f, pW = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float u = power(x[e], ct), p = ex2(u);
            ps = e ? ps + p : p;
            pW = __builtin_fmaf(p, fmaxf(u, -kFar), pW);    // (p is 0 where the bound is reached)
        }
        s += ps;
        W += pW;
        return t;
    }
};

template <typename T>
__device__ __forceinline__ float logit(const T *z, const float *bias, int j) {
    return Elem<T>::load(z + j) + (bias ? bias[j] : 0.f);
}

// 16 bytes at the same classes of each of R rows, and the bias beside them, read once.
template <typename T, int R>
struct Pieces {
    static constexpr int V = Elem<T>::kPerChunk;
    typename RowVec<T, V>::raw z[R];
    typename RowVec<float, V>::raw b;
    __device__ __forceinline__ void load(const T *const (&zp)[R], const float *bias, int j) {
#pragma unroll
        for (int i = 0; i < R; ++i) z[i] = RowVec<T, V>::load(zp[i] + j);
        if (bias) b = RowVec<float, V>::load(bias + j);
    }
    __device__ __forceinline__ void values(int i, const float *bias, float *x) const {
        RowVec<T, V>::unpack(z[i], x);
        if (bias) {
            float y[V];
            RowVec<float, V>::unpack(b, y);
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] += y[e];
        }
    }
};

// All of the workgroup's NT lanes' parts of R rows of c classes: pieces lane, lane + NT ..., in batches of kBatch, and
// single classes behind the last whole piece.  groups, if given: the upper halves of the orders of each lane's largest in
// each kGroups-th batch, kGroups rows of them for each row.
template <bool EXACT, typename T, int NT, int R>
__device__ __forceinline__ void read_rows(const T *const (&z)[R], const float *bias, int c, float ct, uint16_t (*groups)[NT],
                                          Part<EXACT> (&p)[R]) {
    constexpr int V = Pieces<T, R>::V;
#pragma unroll
    for (int k = 0; k < R; ++k) p[k] = Part<EXACT>::none();
    const int n = c / V;
    int g = 0;
    const auto note = [&](const float (&t)[R]) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            p[k].top = fmaxf(p[k].top, t[k]);
            if (groups) {
                const uint16_t o = (uint16_t)(order_of(t[k]) >> 16);
                uint16_t *const at = &groups[k * kGroups + g % kGroups][threadIdx.x];
                *at = g < kGroups ? o : max(*at, o);
            }
        }
        ++g;
    };
    const auto add = [&](const Pieces<T, R> &b, float (&t)[R]) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            float x[V];
            b.values(k, bias, x);
            t[k] = fmaxf(t[k], p[k].template add<V>(x, ct));
        }
    };
    int q = threadIdx.x;
    for (; q + (kBatch - 1) * NT < n; q += kBatch * NT) {
        Pieces<T, R> b[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) b[i].load(z, bias, (q + i * NT) * V);
        float t[R];
#pragma unroll
        for (int k = 0; k < R; ++k) t[k] = -INFINITY;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) add(b[i], t);
        note(t);
    }
    if (q < n) {
        float t[R];
#pragma unroll
        for (int k = 0; k < R; ++k) t[k] = -INFINITY;
        for (; q < n; q += NT) {
            Pieces<T, R> b;
            b.load(z, bias, q * V);
            add(b, t);
        }
        note(t);
    }
    if (threadIdx.x < c - n * V) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const float x = logit(z[k], bias, n * V + threadIdx.x);
            p[k].top = fmaxf(p[k].top, p[k].template add<1>(&x, ct));
        }
    }
}

template <bool EXACT, typename T, int NT>
__device__ __forceinline__ Part<EXACT> read_row(const T *z, const float *bias, int c, float ct, uint16_t (*groups)[NT]) {
    const T *const one[1] = {z};
    Part<EXACT> p[1];
    read_rows<EXACT, T, NT, 1>(one, bias, c, ct, groups, p);
    return p[0];
}

template <int NT>
struct RowStats {
    float top[NT / 64], s[NT / 64], W[NT / 64];
};

// The row's maximum m, sum s and weighted sum W (in powers of two) relative to it, in all lanes, from the lanes' parts.
template <bool EXACT, int NT>
__device__ __forceinline__ void join_row(const Part<EXACT> &p, float ct, RowStats<NT> &sh, float &m, float &s, float &W) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const float wm = wave_maxf(p.top);
    __syncthreads();
    if (lane == 0) sh.top[w] = wm;
    __syncthreads();
    m = sh.top[0];
#pragma unroll
    for (int v = 1; v < NT / 64; ++v) m = fmaxf(m, sh.top[v]);
    // what the lane's sums are relative to is at most kSlack below its largest class, or far below m
    const float D = m == -INFINITY ? 0.f : fminf(p.power(m, ct), kFar), r = ex2(-D);
    s = wave_sumf(p.s * r);
    W = wave_sumf((p.W - D * p.s) * r);
    if (lane == 0) {
        sh.s[w] = s;
        sh.W[w] = W;
    }
    __syncthreads();
    s = sh.s[0];
    W = sh.W[0];
#pragma unroll
    for (int v = 1; v < NT / 64; ++v) {
        s += sh.s[v];
        W += sh.W[v];
    }
}

// The same, and the row again with exact differences where it needs them.
template <typename T, int NT>
__device__ __forceinline__ void join_sums(const T *z, const float *bias, int c, float ct, const Part<false> &p, RowStats<NT> &sh,
                                          float &m, float &s, float &W) {
    join_row<false, NT>(p, ct, sh, m, s, W);
    // (towards the edge terms and W leave fp32's exponents before s does)
    if (!(s > 0.f && s < INFINITY && __builtin_fabsf(m) * ct < kEdge / 2))
        join_row<true, NT>(read_row<true, T, NT>(z, bias, c, ct, nullptr), ct, sh, m, s, W);
}

// The largest number, of those whose bits below `low` are 0, that at least k of a wave's orders (U a lane) are not below (0:
// fewer than k are above 0), from its highest bit down; exactly k of them stop the search.
template <int U>
__device__ __forceinline__ uint32_t kth_of(const uint32_t (&mine)[U], int k, int low) {
    uint32_t t = 0;
    for (int bit = 31; bit >= low; --bit) {
        const uint32_t trial = t | 1u << bit;
        int n = 0;
#pragma unroll
        for (int i = 0; i < U; ++i) n += __popcll(__ballot(mine[i] >= trial));
        if (n >= k) t = trial;
        if (n == k) break;
    }
    return t;
}

template <int NT>
struct Trials {
    u64 differ[NT / 64];
    int counts[2][NT / 64];
};

template <int NT, int CANDS>
struct ListShared {
    static constexpr int kCands = CANDS;       // candidates for the list
    uint32_t orders[NT];       // of each lane's largest class
    int hot[NT];               // lanes whose largest is on the list, at most k, or more of equal ones
    uint32_t tau;
    int nhot, n;
    int counts[NT / 64];
    u64 best[NT / 64];
    Trials<NT> trials;
    u64 cand[kCands];
};

// Classes of the row whose order is at least `least` into sh.cand; sh.n counts them all.  The batches of the hot lanes in
// which such a class can be are shared out to all lanes.  (A hot lane's pieces lie NT pieces apart, so reading all of them
// again would fetch as many lines as the row has.)
template <typename T, int NT, int CANDS>
__device__ __forceinline__ void collect(const T *z, const float *bias, int c, const uint16_t (*groups)[NT],
                                        ListShared<NT, CANDS> &sh, uint32_t least) {
    constexpr int V = Pieces<T, 1>::V, kCands = CANDS;
    const T *const row[1] = {z};
    const int n = c / V, per = (n + kBatch * NT - 1) / (kBatch * NT), all = sh.nhot * per;
    const auto take = [&](float x, int j) {
        const uint32_t o = order_of(x);
        if (o < least) return;
        const int i = atomicAdd(&sh.n, 1);
        if (i < kCands) sh.cand[i] = key_of(o, j);
    };
    for (int q = threadIdx.x; q < all; q += NT) {
        const int h = q / per, g = q - h * per, lane = sh.hot[h];
        if (groups[g % kGroups][lane] < (uint16_t)(least >> 16)) continue;
        const int at = g * kBatch * NT + lane;
        Pieces<T, 1> b[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (at + i * NT < n) b[i].load(row, bias, (at + i * NT) * V);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (at + i * NT >= n) continue;
            float x[V];
            b[i].values(0, bias, x);
#pragma unroll
            for (int e = 0; e < V; ++e) take(x[e], (at + i * NT) * V + e);
        }
    }
    // single classes behind the last piece
    if (threadIdx.x < c - n * V) take(logit(z, bias, n * V + threadIdx.x), n * V + threadIdx.x);
}

// The first `want` classes of the row whose order is tau, in the row's order, behind the n candidates in sh.cand.
template <typename T, int NT, int CANDS>
__device__ __forceinline__ void first_equal(const T *z, const float *bias, int c, ListShared<NT, CANDS> &sh, int n, int want) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int base = 0; base < c && want > 0; base += NT) {
        const int j = base + threadIdx.x;
        const bool eq = j < c && order_of(logit(z, bias, j)) == sh.tau;
        const u64 all = __ballot(eq);
        __syncthreads();
        if (lane == 0) sh.counts[w] = __popcll(all);
        __syncthreads();
        int before = 0, total = 0;
#pragma unroll
        for (int v = 0; v < NT / 64; ++v) {
            before += v < w ? sh.counts[v] : 0;
            total += sh.counts[v];
        }
        before += __popcll(all & ((1ull << lane) - 1));
        if (eq && before < want) sh.cand[n + before] = key_of(sh.tau, j);
        n += min(total, want);
        want -= total;
    }
}

// The row's largest class below key `last`, by all lanes.
template <typename T, int NT, int CANDS>
__device__ __forceinline__ u64 next_below(const T *z, const float *bias, int c, ListShared<NT, CANDS> &sh, u64 last) {
    u64 mine = 0;
    for (int j = threadIdx.x; j < c; j += NT) {
        const u64 key = key_of(order_of(logit(z, bias, j)), j);
        if (key < last && key > mine) mine = key;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const u64 other = __shfl_xor(mine, o, 64);
        mine = other > mine ? other : mine;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = mine;
    __syncthreads();
    for (int v = 0; v < NT / 64; ++v) mine = sh.best[v] > mine ? sh.best[v] : mine;
    return mine;
}

// Of n > kRankAll candidates, all different and none 0, the k < n largest to the front of cand, in any order, found by all
// waves bit by bit of those that differ (each round counts the candidates that are not below a trial), where a rank for
// each would look at n^2 (2560 x 1000 with 128 classes: 29 us, 283).
constexpr int kRankAll = 256;

template <int NT, int MOST>
__device__ __forceinline__ void shrink(u64 *cand, int n, int k, Trials<NT> &sh, int *next) {
    constexpr int U = MOST / NT;
    static_assert(MOST % NT == 0);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const u64 one = cand[0];
    u64 mine[U], differ = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const bool there = (int)threadIdx.x + i * NT < n;
        mine[i] = there ? cand[threadIdx.x + i * NT] : 0;
        differ |= there ? mine[i] ^ one : 0;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) differ |= __shfl_xor(differ, o, 64);
    if (lane == 0) sh.differ[w] = differ;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < NT / 64; ++v) differ |= sh.differ[v];
    u64 t = one & ~differ;                   // bits that all have alike change no count
    for (int round = 0; differ; ++round) {
        const u64 bit = 1ull << (63 - __builtin_clzll(differ)), trial = t | bit;
        differ ^= bit;
        int c = 0;
#pragma unroll
        for (int i = 0; i < U; ++i) c += __popcll(__ballot(mine[i] >= trial));
        if (NT > 64) {
            if (lane == 0) sh.counts[round & 1][w] = c;
            __syncthreads();
            c = 0;
#pragma unroll
            for (int v = 0; v < NT / 64; ++v) c += sh.counts[round & 1][v];
        }
        if (c >= k) t = trial;
        if (c == k) break;
    }
    __syncthreads();
    if (threadIdx.x == 0) *next = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < U; ++i)
        if (mine[i] >= t) cand[atomicAdd(next, 1)] = mine[i];
    __syncthreads();
}

// The k largest classes of a row (or of a part of one) that has one, largest first, to emit(rank, key); behind the
// last class that is not -inf emit(rank, 0).  top: each lane's largest.
template <typename T, int NT, int CANDS, typename Emit>
__device__ __forceinline__ void largest(const T *z, const float *bias, int c, int k, float top, const uint16_t (*groups)[NT],
                                        ListShared<NT, CANDS> &sh, const Emit &emit) {
    constexpr int kCands = CANDS;
    constexpr bool kGroupwise = NT == 64 && CANDS >= 1024;
    const int lane = threadIdx.x & 63;
    sh.orders[threadIdx.x] = order_of(top);
    __syncthreads();
    // sixteen bits of it will do, but where too many classes have the same ones: then all, the classes above it, and the
    // first of those equal to it (masks of a finite number)
    const auto set_tau = [&](int low) {
        if (threadIdx.x < 64) {
            uint32_t t;
            if (kGroupwise && low == 16) {
                // a wave's maxima are too few to tell: those of its groups (2560 x 4000 with 64 classes 25 us, 1200 by the
                // lanes' own, which let most classes be candidates)
                constexpr int V = Pieces<T, 1>::V;
                uint32_t mine[kGroups];
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
                    mine[g] = g * kBatch * NT + lane < c / V ? (uint32_t)groups[g][lane] << 16 : 0;
                t = kth_of(mine, k, low);
            } else if (kGroupwise) {
                // exactly, of all classes
                t = 0;
                for (int bit = 31; bit >= 0; --bit) {
                    int n = 0;
                    for (int j = lane; j < c; j += 64) n += order_of(logit(z, bias, j)) >= (t | 1u << bit);
                    if (wave_sum(n) >= k) t |= 1u << bit;
                }
            } else {
                uint32_t mine[NT / 64];
#pragma unroll
                for (int i = 0; i < NT / 64; ++i) mine[i] = sh.orders[i * 64 + lane];
                t = kth_of(mine, k, low);
            }
            if (lane == 0) {
                sh.tau = max(t, 1u);
                sh.nhot = sh.n = 0;
            }
        }
        __syncthreads();
        if (sh.orders[threadIdx.x] >= sh.tau) sh.hot[atomicAdd(&sh.nhot, 1)] = threadIdx.x;
        __syncthreads();
    };
    set_tau(16);
    collect<T, NT, CANDS>(z, bias, c, groups, sh, sh.tau);
    __syncthreads();
    int n = sh.n;
    if (n > kCands) {
        __syncthreads();
        set_tau(0);
        collect<T, NT, CANDS>(z, bias, c, groups, sh, sh.tau + 1);
        __syncthreads();
        n = sh.n;
        if (n <= kCands - 128) {
            const int want = max(k - n, 0);
            first_equal<T, NT, CANDS>(z, bias, c, sh, n, want);
            n += want;
            __syncthreads();
        }
    }
    if (n <= kCands) {
        if (n > kRankAll) {
            shrink<NT, CANDS>(sh.cand, n, k, sh.trials, &sh.n);
            n = k;
        }
        for (int i = threadIdx.x; i < n; i += NT) {
            const u64 key = sh.cand[i];
            int rank = 0;
            for (int q = 0; q < n; ++q) rank += sh.cand[q] > key;
            if (rank < k) emit(rank, key);
        }
        for (int q = n + threadIdx.x; q < k; q += NT) emit(q, 0ull);
        return;
    }
    // the largest classes crowd in few lanes: one after the other, each by a reading of the row
    u64 last = ~0ull;
    for (int q = 0; q < k; ++q) {
        if (last != 0) last = next_below<T, NT, CANDS>(z, bias, c, sh, last);
        if ((last >> 32) == 0) last = 0;             // nothing but -inf is left
        if (threadIdx.x == 0) emit(q, last);
    }
}

// A row that is padding: its logits are not looked at.
template <int NT>
__device__ __forceinline__ bool padding(const LogprobArgs &a, int64_t r, int token) {
    if (token >= 0 && token < a.c) return false;
    if (threadIdx.x == 0) {
        if (a.logp) a.logp[r] = 0.f;
        if (a.entropy) a.entropy[r] = 0.f;
        if (a.lse) a.lse[r] = 0.f;
    }
    for (int q = threadIdx.x; q < a.k; q += NT) {
        a.top_idx[r * a.k + q] = -1;
        a.top_logp[r * a.k + q] = -INFINITY;
    }
    return true;
}

// What a row's maximum and sums say, and whether it has a list (else that is written, too).
template <int NT>
__device__ __forceinline__ bool finish_row(const LogprobArgs &a, int64_t r, float xt, float m, float s, float W, float &ls) {
    const bool empty = m == -INFINITY && s == 0.f, nan = !(s < INFINITY);
    const float invT = 1.f / a.temperature;
    ls = __builtin_amdgcn_logf(fmaxf(s, 1.f)) * kLn2;       // (the largest class alone adds 1, but for a rounding)
    if (threadIdx.x == 0) {
        if (a.logp) a.logp[r] = empty ? -INFINITY : nan ? NAN : (xt - m) * invT - ls;
        if (a.entropy) a.entropy[r] = empty ? 0.f : nan ? NAN : fmaxf(ls - W / s * kLn2, 0.f);
        if (a.lse) a.lse[r] = empty ? -INFINITY : nan ? NAN : m * invT + ls;
    }
    if (!empty && !nan) return a.k > 0;
    for (int q = threadIdx.x; q < a.k; q += NT) {
        a.top_idx[r * a.k + q] = -1;
        a.top_logp[r * a.k + q] = nan ? NAN : -INFINITY;
    }
    return false;
}

__device__ __forceinline__ void put_class(const LogprobArgs &a, int64_t r, int rank, u64 key, float m, float ls) {
    a.top_idx[r * a.k + rank] = key ? (int32_t)~(uint32_t)key : -1;
    a.top_logp[r * a.k + rank] = key ? (value_of((uint32_t)(key >> 32)) - m) * (1.f / a.temperature) - ls : -INFINITY;
}

template <typename T, int NT, int CANDS>
__global__ __launch_bounds__(NT) void logprob_kernel(LogprobArgs a) {
    __shared__ RowStats<NT> st;
    __shared__ ListShared<NT, CANDS> sh;
    __shared__ uint16_t groups[kGroups][NT];
    const int64_t r = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (r >= a.n) return;
    const float ct = kLog2e / a.temperature;
    const int token = a.tokens ? a.tokens[r] : 0;
    if (padding<NT>(a, r, token)) return;
    const T *const z = (const T *)a.z + r * a.zld;
    const float xt = logit(z, a.bias, token);
    float m, s, W, ls;
    const Part<false> p = read_row<false, T, NT>(z, a.bias, a.c, ct, a.k > 0 ? groups : nullptr);
    join_sums<T, NT>(z, a.bias, a.c, ct, p, st, m, s, W);
    if (finish_row<NT>(a, r, xt, m, s, W, ls))
        largest<T, NT, CANDS>(z, a.bias, a.c, a.k, p.top, groups, sh, [&](int rank, u64 key) { put_class(a, r, rank, key, m, ls); });
}

// R neighbouring rows by one workgroup, without lists: read together, which reads the bias once, unless one of them is padding.
template <typename T, int NT, int R>
__global__ __launch_bounds__(NT) void logprob_rows_kernel(LogprobArgs a) {
    __shared__ RowStats<NT> st;
    const int64_t r0 = (blockIdx.x + (int64_t)blockIdx.y * gridDim.x) * R;
    if (r0 >= a.n) return;
    const float ct = kLog2e / a.temperature;
    const T *z[R];
    int token[R], rows = 0;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int64_t r = min(r0 + k, a.n - 1);
        token[k] = a.tokens ? a.tokens[r] : 0;
        z[k] = (const T *)a.z + r * a.zld;
        rows += r0 + k < a.n && token[k] >= 0 && token[k] < a.c;
    }
    Part<false> p[R];
    if (rows == R) read_rows<false, T, NT, R>(z, a.bias, a.c, ct, nullptr, p);
#pragma unroll
    for (int k = 0; k < R; ++k) {
        if (r0 + k >= a.n || padding<NT>(a, r0 + k, token[k])) continue;
        const float xt = logit(z[k], a.bias, token[k]);
        if (rows < R) p[k] = read_row<false, T, NT>(z[k], a.bias, a.c, ct, nullptr);
        float m, s, W, ls;
        join_sums<T, NT>(z[k], a.bias, a.c, ct, p[k], st, m, s, W);
        finish_row<NT>(a, r0 + k, xt, m, s, W, ls);
    }
}

// Few long rows: each cut into parts, a workgroup each, which leave their maximum, sums and k largest classes in the
// workspace; then a workgroup joins each row's parts.  Both are chains of waits: 16 x 131072 in bf16 takes 6.6 us without
// a list, 12.9 with 20 classes, 24 with 128.
struct PartStats {
    float m, s, W;
};
constexpr int kPartLeast = 8192, kPartMost = 32;

template <typename T>
__global__ __launch_bounds__(256) void logprob_part_kernel(LogprobArgs a, PartStats *stats, u64 *lists, int parts, int part_len) {
    constexpr int NT = 256;
    __shared__ RowStats<NT> st;
    __shared__ ListShared<NT, 1024> sh;
    __shared__ uint16_t groups[kGroups][NT];
    const int64_t r = blockIdx.y;
    const int part = blockIdx.x, j0 = part * part_len, c = min(part_len, a.c - j0);
    const float ct = kLog2e / a.temperature;
    if (a.tokens && (a.tokens[r] < 0 || a.tokens[r] >= a.c)) return;
    const T *const z = (const T *)a.z + r * a.zld + j0;
    const float *const bias = a.bias ? a.bias + j0 : nullptr;
    float m, s, W;
    const Part<false> p = read_row<false, T, NT>(z, bias, c, ct, a.k > 0 ? groups : nullptr);
    join_sums<T, NT>(z, bias, c, ct, p, st, m, s, W);
    if (threadIdx.x == 0) stats[r * parts + part] = PartStats{m, s, W};
    if (a.k == 0 || !(s < INFINITY)) return;         // (a NaN row has no list)
    u64 *const list = lists + (r * parts + part) * a.k;
    largest<T, NT, 1024>(z, bias, c, a.k, p.top, groups, sh, [&](int rank, u64 key) { list[rank] = key ? key - (u64)j0 : 0ull; });
}

template <typename T>
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobArgs a, const PartStats *stats, const u64 *lists, int parts) {
    constexpr int NT = 256, U = 4;
    __shared__ u64 cand[kPartMost * 128];
    __shared__ Trials<NT> trials;
    __shared__ int count;
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x & 63, total = parts * a.k;
    const int token = a.tokens ? a.tokens[r] : 0;
    // what is to be known about the row is asked for at once
    const PartStats own = lane < parts ? stats[r * parts + lane] : PartStats{-INFINITY, 0.f, 0.f};
    const u64 *const list = lists + r * total;
    u64 key[U];
#pragma unroll
    for (int i = 0; i < U; ++i) key[i] = (int)threadIdx.x + i * NT < total ? list[threadIdx.x + i * NT] : 0;
    const int half = min(a.k, (parts + 1) / 2), deep = half > 0 ? (a.k + half - 1) / half : 0;
    const u64 bar = deep > 0 && lane < parts ? list[lane * a.k + deep - 1] : 0;
    if (padding<NT>(a, r, token)) return;
    const float ct = kLog2e / a.temperature;
    const float xt = logit((const T *)a.z + r * a.zld, a.bias, token);
    const float m = wave_maxf(own.m);
    const float D = own.m == -INFINITY ? 0.f : fminf((m - own.m) * ct, kFar), e = ex2(-D);
    const float s = wave_sumf(own.s * e), W = wave_sumf((own.W - D * own.s) * e);
    float ls;
    if (!finish_row<NT>(a, r, xt, m, s, W, ls)) return;
    // of half the parts, those with the largest ones, each has `deep` classes that are not below the least of these
    int before = 0;
    for (int v = 0; v < parts; ++v) before += (u64)__shfl(bar, v, 64) > bar;
    u64 t = before < half ? bar : ~0ull;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) t = min(t, (u64)__shfl_xor(t, o, 64));
    t = max(t, (u64)1);
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < U; ++i)
        if (key[i] >= t) cand[atomicAdd(&count, 1)] = key[i];
    for (int q = threadIdx.x + U * NT; q < total; q += NT) {
        const u64 x = list[q];
        if (x >= t) cand[atomicAdd(&count, 1)] = x;
    }
    __syncthreads();
    int n = count;
    if (n > kRankAll) {
        shrink<NT, kPartMost * 128>(cand, n, a.k, trials, &count);
        n = a.k;
    }
    for (int i = threadIdx.x; i < n; i += NT) {
        const u64 x = cand[i];
        int rank = 0;
        for (int q = 0; q < n; ++q) rank += cand[q] > x;
        if (rank < a.k) put_class(a, r, rank, x, m, ls);
    }
    for (int q = n + threadIdx.x; q < a.k; q += NT) put_class(a, r, q, 0ull, m, ls);
}

// The gradient.  Where lse is so large that fp32 no longer tells x / T from it (a row of masks alone; past fp32's range,
// m / T is infinite), the row's maximum and sum are formed again from the row.
// (Each part of a row does: 4096 x 131072 bf16 2742 us, where 393 without; a row that is one workgroup's, as in place, 698,
// 445 without.)
constexpr float kFarLse = 128.f;
constexpr int kBwdPart = 1024;             // pieces of 16 bytes of a part

// What a row's gradient is made of: log p = (x - m) / T - ls, then -p (de log p + base), and dl where the token is.
struct RowGrad {
    int token;
    bool there, none;              // whether there is such a row; whether its gradient is 0
    float m, ls, dl, de, base;
    __device__ __forceinline__ float of(float x, float invT) const {
        const float lp = __builtin_fmaf(x - m, invT, -ls), p = ex2(lp * kLog2e);
        return -p * __builtin_fmaf(de, fmaxf(lp, -kFar), base);
    }
};

// A part of R neighbouring rows by each workgroup, with one reading of the bias.
template <typename T, int NT, int R>
__global__ __launch_bounds__(NT) void logprob_bwd_kernel(LogprobBwdArgs a, int parts, int part_len) {
    constexpr int V = Pieces<T, R>::V, U = 4 / R;
    __shared__ RowStats<NT> st;
    const int64_t job = blockIdx.x + (int64_t)blockIdx.y * gridDim.x, r0 = job / parts * R;
    if (r0 >= a.n) return;
    const int j0 = (int)(job % parts) * part_len, j1 = min(a.c, j0 + part_len);
    const float invT = 1.f / a.temperature, ct = kLog2e / a.temperature;
    const T *z[R];
    T *dz[R];
    RowGrad g[R];
    bool all_none = true;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int64_t r = min(r0 + k, a.n - 1);
        z[k] = (const T *)a.z + r * a.zld;
        dz[k] = (T *)a.dz + r * a.dld;
        g[k].there = r0 + k < a.n;
        g[k].token = a.tokens[r];
        g[k].none = g[k].token < 0 || g[k].token >= a.c || !g[k].there;
        const float lse = a.lse[r];
        g[k].dl = g[k].none ? 0.f : a.dlogp[r] * invT;
        g[k].de = g[k].none || !a.dentropy ? 0.f : a.dentropy[r] * invT;
        g[k].base = g[k].none || !a.dentropy ? g[k].dl : g[k].dl + g[k].de * a.entropy[r];
        g[k].m = 0.f;
        g[k].ls = lse;
        if (!g[k].none && __builtin_fabsf(lse) > kFarLse) {
            float s, W;
            join_row<true, NT>(read_row<true, T, NT>(z[k], a.bias, a.c, ct, nullptr), ct, st, g[k].m, s, W);
            g[k].none = g[k].m == -INFINITY && s == 0.f;                  // -inf throughout
            g[k].ls = __builtin_amdgcn_logf(fmaxf(s, 1.f)) * kLn2;
        }
        all_none = all_none && g[k].none;
    }
    const int n = (j1 - j0) / V;
    for (int q = threadIdx.x; q < n; q += U * NT) {
        Pieces<T, R> b[U];
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (!all_none && q + i * NT < n) b[i].load(z, a.bias, j0 + (q + i * NT) * V);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int j = j0 + (q + i * NT) * V;
            if (q + i * NT >= n) break;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                float x[V];
                if (g[k].none) {
#pragma unroll
                    for (int e = 0; e < V; ++e) x[e] = 0.f;
                } else {
                    b[i].values(k, a.bias, x);
#pragma unroll
                    for (int e = 0; e < V; ++e) x[e] = g[k].of(x[e], invT);
                    if ((unsigned)(g[k].token - j) < (unsigned)V) {
#pragma unroll
                        for (int e = 0; e < V; ++e) x[e] += g[k].token == j + e ? g[k].dl : 0.f;
                    }
                }
                if (g[k].there) RowVec<T, V>::store(dz[k] + j, x);
            }
        }
    }
    const int j = j0 + n * V + threadIdx.x;
    if (j >= j1) return;
#pragma unroll
    for (int k = 0; k < R; ++k)
        if (g[k].there)
            Elem<T>::store(dz[k] + j, g[k].none ? 0.f : g[k].of(logit(z[k], a.bias, j), invT) + (j == g[k].token ? g[k].dl : 0.f));
}

// Parts of a row, 0 for rows that one workgroup reads: enough for two workgroups a CU, of at least kPartLeast classes.
// (The list asked for has no say in it, nor below in how many waves read a row, and so none in the sums' order.)
// Measured with 20 classes, in parts and by one workgroup a row: 131072 classes, 16 rows 12.9 and 18.7 us, 128 rows 17.9
// and 20.3, 256 rows 25.7 and 21.0; 40000 classes, 16 rows 12.3 and 13.1, 128 rows 13.7 and 14.0, 256 rows 16.2 and 14.9.
static int row_parts(int64_t n, int c) {
    if (n > 128 || c < 4 * kPartLeast) return 0;
    return (int)std::min<int64_t>({kPartMost, c / kPartLeast, (512 + n - 1) / n});
}

size_t logprob_ws_bytes(int64_t n, int c, int k) {
    const int64_t parts = n > 0 ? row_parts(n, c) : 0;
    return (size_t)(n * parts * (sizeof(u64) * k + sizeof(PartStats)));
}

// Short rows by one wave, for lists up to 32 with room for few candidates (65536 x 1024: 38 us without a list, 84 with 20
// classes; by four waves 84 and 197; with room for 1024 candidates 49 and 123, as fewer rows fit a CU).  Up to 4096
// classes, where there are rows enough (65536 x 1500: 50 us and with 10 classes 94, by four waves 94 and 202; 2560 x 4000 8.2
// and 12.2, 9.0 and 16.1; but 256 x 2000 4.3, 3.8), with lists of more than 64 with room for 2048 candidates (2560 x 1100
// with 128 classes 65 us: its 74 groups are too few, so that all classes are candidates).
// With a bias and no list two rows by four waves (4096 x 131072 218 us, 250 by one row; 2560 x 40000 46, 54; 20000 x 10000
// 87, 98; but 1500 x 10000 12.4, 11.7; with lists, which follow one another then, 2560 x 40000 76, 64).  Few rows too long for
// four waves, and too many to be cut, by sixteen (256 x 131072 with 20 classes 21 us, 31 by four; 200 x 50000 15.0, 17.3;
// but 200 x 20000 12.2, 10.6).
template <typename T>
static void launch_rows(const LogprobArgs &a, void *ws, hipStream_t st) {
    const int parts = row_parts(a.n, a.c);
    if (parts) {
        // parts begin at whole pieces of 16 bytes of the row
        const int len = ((a.c + parts - 1) / parts + 63) / 64 * 64;
        u64 *const lists = (u64 *)ws;
        PartStats *const stats = (PartStats *)(lists + a.n * parts * a.k);
        const int used = (a.c + len - 1) / len;
        hipLaunchKernelGGL((logprob_part_kernel<T>), dim3(used, (unsigned)a.n), dim3(256), 0, st, a, stats, lists, used, len);
        hipLaunchKernelGGL((logprob_join_kernel<T>), dim3((unsigned)a.n), dim3(256), 0, st, a, stats, lists, used);
    } else if (a.c <= 1024 || (a.c <= 4096 && a.n >= 1024)) {
        if (a.k <= 32) hipLaunchKernelGGL((logprob_kernel<T, 64, 320>), grid_2d(a.n), dim3(64), 0, st, a);
        else if (a.c <= 1024 || a.k <= 64) hipLaunchKernelGGL((logprob_kernel<T, 64, 1024>), grid_2d(a.n), dim3(64), 0, st, a);
        else hipLaunchKernelGGL((logprob_kernel<T, 64, 2048>), grid_2d(a.n), dim3(64), 0, st, a);
    } else if (a.n > 256 || a.c < 4 * kPartLeast) {
        if (a.k == 0 && a.bias && a.n >= 1024 && a.n * a.c >= (int64_t)1 << 25)
            hipLaunchKernelGGL((logprob_rows_kernel<T, 256, 2>), grid_2d((a.n + 1) / 2), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((logprob_kernel<T, 256, 1024>), grid_2d(a.n), dim3(256), 0, st, a);
    } else {
        hipLaunchKernelGGL((logprob_kernel<T, 1024, 1024>), grid_2d(a.n), dim3(1024), 0, st, a);
    }
}

hipError_t launch_logprob(int dt, const LogprobArgs &a, void *ws, hipStream_t st) {
    if (dt == 0) launch_rows<float>(a, ws, st);
    else launch_rows<bf16_t>(a, ws, st);
    return hipGetLastError();
}

// Short rows by one wave (65536 x 1000: 46 us, 87 by four); longer ones in parts of the same length, a workgroup each
// (20000 x 10000 in two halves 152 us, in 8192 and 1808 163).  Two rows a workgroup where one is not much work for it
// (65536 x 1500 76 us, 145), or has a bias to read (4096 x 131072 387, 410; 20000 x 10000 160; but 1600 x 131072 181, 166).
template <typename T>
static void launch_bwd_rows(const LogprobBwdArgs &a, hipStream_t st) {
    // parts of a row read the whole of it where lse is far out: in place a row is one workgroup's (4096 x 131072 445 us, apart 393;
    // 1021 x 50021 fp32 92, 81; but 64 x 131072 35, 11)
    const int most = kBwdPart * 16 / (int)sizeof(T), parts = a.dz == a.z ? 1 : (a.c + most - 1) / most;
    const int len = ((a.c + parts - 1) / parts + 63) / 64 * 64;
    const bool pairs = (a.n >= 1024 && a.c * sizeof(T) <= 6144) || (a.bias && a.n >= 2048 && a.n * a.c >= (int64_t)1 << 25);
    if (a.c <= 1024) {
        hipLaunchKernelGGL((logprob_bwd_kernel<T, 64, 1>), grid_2d(a.n), dim3(64), 0, st, a, 1, a.c);
    } else if (pairs) {
        hipLaunchKernelGGL((logprob_bwd_kernel<T, 256, 2>), grid_2d((a.n + 1) / 2 * parts), dim3(256), 0, st, a, parts, len);
    } else {
        hipLaunchKernelGGL((logprob_bwd_kernel<T, 256, 1>), grid_2d(a.n * parts), dim3(256), 0, st, a, parts, len);
    }
}

hipError_t launch_logprob_bwd(int dt, const LogprobBwdArgs &a, hipStream_t st) {
    if (dt == 0) launch_bwd_rows<float>(a, st);
    else launch_bwd_rows<bf16_t>(a, st);
    return hipGetLastError();
}

}  // namespace tfk

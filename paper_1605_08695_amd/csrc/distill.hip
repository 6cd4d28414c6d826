// Distillation from a teacher's top logits: per row, the loss and its gradient in one launch.
//
// With x = logits + bias, K the distinct classes in the row's list, P_j the sum of the teacher's
// probabilities of class j's entries, P_r what the teacher gives to all other classes (0 where its list
// is renormalised), q = softmax(x / T), q_r = sum of q over the classes outside K:
//   soft = sum_K P_j (log P_j - log q_j) + P_r (log P_r - log q_r)        (terms with P = 0 are 0)
//   hard = logsumexp(x) - x_label
//   loss = w (alpha T^2 soft + (1 - alpha) hard)
//   dx_j = scale w (alpha T (q_j - P_j)              + (1 - alpha) (softmax(x)_j - [j = label]))   j in K
//   dx_j = scale w (alpha T q_j (q_r - P_r) / q_r    + (1 - alpha) (softmax(x)_j - [j = label]))   else
// The classes outside K have their own maximum m_r and sum S_r = sum exp((x - m_r) / T), so that
// q_j / q_r = exp((x_j - m_r) / T) / S_r and log q_r lose nothing where the listed classes hold nearly
// all of the student's probability.  In the bulk of a row a listed class is -inf (a bit per class, in LDS,
// tells them apart), its exponential 0; the first wave looks after the listed ones and the label, whose
// gradients it stores after the bulk's.
//
// Exponentials are powers of two, exp(y / T) = 2^(y ct): 2^(x ct - R) by one fma and one exp instruction,
// with R = m_r ct rounded once and used as it is wherever the sum is.  R's rounding error is then a factor of
// all of the sum's terms, and has to stay a small one: up to |R| = 2^24 it is at most half a power of two (two,
// of the fourth powers below).  Rows whose maximum is further out (a mask throughout, -1e9 as well as the
// type's lowest value, infinities, NaN) are shifted first, by exact differences; in a running sum classes that
// far below count as 0 until a nearer one comes.
//
// Bound by HBM: a row's logits are read once and its gradient written once, with everything between in
// registers; what the loss needs besides (the list, the label, the bias) is small or comes from the caches.  A
// workgroup has a row, so nothing is exchanged between workgroups and no workspace is needed.
//   c <= 40960 in bf16, 20480 in fp32: x in fp32 registers, its exponential in the same ones; 2560 x 40000 bf16
//     with bias 99 us a call (4.2 TB/s; in place 100)
//   c <= 131072, 65536: the logits as they were read; 1021 x 50021 with bias 55 us (3.7 TB/s; in place 63); one
//     workgroup per CU from 65536 on: 4096 x 131072 with labels at T = 2 582 us (3.7 TB/s; in place 597;
//     exponentials twice, VALU 60 % busy; read twice instead: 664 us)
//   longer rows: read twice
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "rowvec.h"

// R is a rounded product: an fma that formed it anew inside a difference would see another one.  Where an fma
// is wanted, it is written.
#pragma clang fp contract(off)

namespace tfk {

// Where the T = 1 exponentials of the hard term come from: those at T themselves (no hard term, or T = 1),
// their square (T = 2), their fourth power (T = 4), or exponentials of their own.  (4096 x 40000, T = 2, labels:
// 159 us by squares, 179 with exponentials of their own.)
enum { kSame = 0, kSquare = 1, kFourth = 2, kOwn = 3 };

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f, kHuge = 1e30f;

// The largest |x| whose exponents, at T and at 1, stay within 2^24.
__device__ __forceinline__ float far_of(float temperature) { return 0x1p24f * kLn2 * fminf(temperature, 1.f); }

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

// Reductions of a wave, the same in all its lanes (which are all here): within 16 lanes by exchanges in the
// operand's own read -- neighbours, pairs, mirrored eights and sixteens -- and the four sixteens by scalars.  (A
// row's chain holds about ten of them: 128 rows of 1000 8.0 us by exchanges through the LDS, 7.2 so; 2560 x 40000 92.5, 90.)
template <int CTRL>
__device__ __forceinline__ float lane_swap(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
__device__ __forceinline__ float wave_maxf(float v) {
    v = fmaxf(v, lane_swap<0xb1>(v));
    v = fmaxf(v, lane_swap<0x4e>(v));
    v = fmaxf(v, lane_swap<0x141>(v));
    v = fmaxf(v, lane_swap<0x140>(v));
    return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
__device__ __forceinline__ float wave_sumf(float v) {
    v += lane_swap<0xb1>(v);
    v += lane_swap<0x4e>(v);
    v += lane_swap<0x141>(v);
    v += lane_swap<0x140>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

// The same number, as one that nothing computed from it before is known for: what a later phase computes
// from it (addresses, exponentials) is then computed there, not kept in registers from an earlier one.
template <typename X>
__device__ __forceinline__ X fresh(X x) {
    asm volatile("" : "+v"(x));
    return x;
}

// LDS written by other lanes of this wave is there, and nothing moves across.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// What the first wave finds out about a row and all waves need.
struct RowShared {
    float mtop;            // the largest x on the list (-inf: none)
    float psum;            // sum of the listed P
    float top[2];          // sums of the listed exponentials at T and at 1, relative to m
    int soft;              // whether there is a soft term
    float max[16];         // per wave: maximum outside the list
    float sum[16][2];      // per wave: sums outside the list at T and at 1
};

// The row's list in LDS.
struct RowList {
    int32_t *cls;          // [k] the entry's class; -1: none, or another entry stands for it
    float *P;              // [k] its class's probability
    float *x;              // [k] the student's x there
    uint32_t *bits;        // a bit per class of a segment
};

__device__ __forceinline__ void clear_bits(uint32_t *bits, int seg) {
    u32x4_t *const b4 = reinterpret_cast<u32x4_t *>(bits);
#pragma unroll 1
    for (int q = threadIdx.x & 63; q < (seg + 127) / 128; q += 64) b4[q] = u32x4_t{0, 0, 0, 0};
}

// A lane's first entry of the list, asked for before anything else is known about the row.
struct ListHead {
    int32_t idx;
    float t;
};
__device__ __forceinline__ float top_at(const DistillArgs &a, int64_t i) {
    return a.top_dt == 0 ? ((const float *)a.top)[i] : bf16_to_f32(((const bf16_t *)a.top)[i]);
}
__device__ __forceinline__ ListHead list_head(const DistillArgs &a, int64_t row) {
    const int64_t i = row * a.k + min((int)(threadIdx.x & 63), a.k - 1);
    return {a.top_idx[i], top_at(a, i)};
}

// The first wave: reads the list, forms P, adds up the entries of one class under the first of them, marks
// the bits of classes [0, seg), and gathers x.
template <typename T>
__device__ __forceinline__ void read_list(const DistillArgs &a, int64_t row, const ListHead &head, const T *z, int seg,
                                          const RowList &l, RowShared &sh) {
    const int lane = threadIdx.x & 63, k = a.k, c = a.c;
    const int32_t *idx = a.top_idx + row * k;
    float tm = -INFINITY;
#pragma unroll 1
    for (int j = lane; j < k; j += 64) {
        const int32_t i = j < 64 ? head.idx : idx[j];
        const bool ok = i >= 0 && i < c;
        const float t = !ok ? -INFINITY : j < 64 ? head.t : top_at(a, row * k + j);
        l.cls[j] = ok ? i : -1;
        l.P[j] = t;
        tm = fmaxf(tm, t != t ? INFINITY : t);
    }
    clear_bits(l.bits, seg);
    wave_sync();
    tm = wave_maxf(tm);
    const float invt = 1.f / a.temperature;
    float ref = 0.f, lse = 0.f;                       // log p = (t - ref) / T - lse
    if (a.top_lse) {
        lse = a.top_lse[row];
    } else {
        ref = tm;
#pragma unroll 1
        for (int j = lane; j < k; j += 64)
            if (l.cls[j] >= 0) lse += expf((l.P[j] - ref) * invt);
        lse = logf(wave_sumf(lse));
    }
    float psum = 0.f, mtop = -INFINITY;
    bool twice = false;
#pragma unroll 1
    for (int j = lane; j < k; j += 64) {
        const int32_t i = l.cls[j];
        float p = 0.f, x = 0.f;
        if (i >= 0) {
            p = expf((l.P[j] - ref) * invt - lse);
            x = Elem<T>::load(z + i) + (a.bias ? a.bias[i] : 0.f);
            mtop = fmaxf(mtop, x);
            if (i < seg) twice |= (atomicOr(&l.bits[i >> 5], 1u << (i & 31)) >> (i & 31)) & 1u;
        }
        l.P[j] = p;
        l.x[j] = x;
        psum += p;
    }
    wave_sync();
    if (__any(twice) || seg < c) {                    // (classes past the segment have no bits to tell by)
#pragma unroll 1
        for (int j0 = 0; j0 < k; j0 += 64) {
            const int j = j0 + lane;
            const int32_t i = j < k ? l.cls[j] : -1;
            float p = 0.f;
            bool first = true;
            if (i >= 0)
#pragma unroll 1
                for (int q = 0; q < k; ++q)
                    if (l.cls[q] == i) {
                        if (q < j) {
                            first = false;
                            break;
                        }
                        p += l.P[q];
                    }
            wave_sync();
            if (i >= 0) l.P[j] = first ? p : -1.f;    // (p adds entries from j on: none of them overwritten yet)
            wave_sync();
        }
#pragma unroll 1
        for (int j = lane; j < k; j += 64)
            if (l.P[j] < 0.f) l.cls[j] = -1;
    }
    psum = wave_sumf(psum);
    mtop = wave_maxf(mtop);
    if (lane == 0) {
        sh.psum = psum;
        sh.mtop = mtop;
        sh.soft = a.top_lse != nullptr || tm > -INFINITY;
    }
}

// What the divergence is formed times: next to a listed class of the type's lowest value x / T may have no fp32 value
// (T < 1), nor the sum of its terms (the probabilities add up to one and a rounding), where alpha T^2 of it has.
__device__ __forceinline__ float loss_unit(float temperature) { return 0.5f * fminf(temperature, 1.f); }

// A row's sums and what follows from them, the same in every thread.
struct RowTotals {
    float m, mr;           // maxima: of all, outside the list (0: none)
    bool huge;             // whether x outside the list is taken relative to mr before anything else
    float ct;              // log2(e) / T
    float R, R1;           // exponents' references outside the list, at T and at 1 (0 where huge)
    float relt, rel1;      // 2^(those - m's)
    float ln_rel;          // log relt, times loss_unit
    float st, s1, logst, qr;
    float co, ch;          // gradients outside the list: co e + ch e1
    float gs, at, gb;      // scale w, alpha T, scale w (1 - alpha)

    // x outside the list, as its exponentials want it
    __device__ __forceinline__ float e(float x) const { return huge ? ex2((x - mr) * ct) : ex2(fmaf(x, ct, -R)); }
    __device__ __forceinline__ float e1(float x) const { return huge ? ex2((x - mr) * kLog2e) : ex2(fmaf(x, kLog2e, -R1)); }

    __device__ __forceinline__ void maxima(float outside, float mtop, float temperature, int kind) {
        m = fmaxf(outside, mtop);
        ct = kLog2e / temperature;
        mr = outside > -INFINITY ? outside : 0.f;
        huge = !(fabsf(mr) < far_of(temperature) && !(m >= kHuge));        // (m ct itself could overflow)
        R = huge ? 0.f : mr * ct;
        R1 = huge ? 0.f : (kind == kOwn ? mr * kLog2e : R * temperature);   // (exact: T is 1, 2 or 4 otherwise)
        const bool none = !(outside > -INFINITY);
        relt = none ? 0.f : ex2(huge ? (mr - m) * ct : fmaf(-m, ct, R));
        rel1 = none ? 0.f : ex2(huge ? (mr - m) * kLog2e : fmaf(-m, kLog2e, R1));
        ln_rel = none ? 0.f : huge ? 0.5f * (mr - m) / fmaxf(temperature, 1.f) : fmaf(-m, ct, R) * (kLn2 * loss_unit(temperature));
    }

    __device__ __forceinline__ void sums(const DistillArgs &a, float w, float rest, float rest1, const RowShared &sh,
                                         bool hard, float pr) {
        st = sh.top[0] + rest * relt;
        s1 = sh.top[1] + rest1 * rel1;
        logst = logf(st);
        qr = rest * relt / st;
        gs = a.scale * w;
        at = a.alpha * a.temperature;
        gb = gs * (1.f - a.alpha);
        co = !sh.soft ? 0.f : (rest != 0.f ? gs * at * (qr - pr) / rest : gs * at * qr);
        ch = hard ? gb * rel1 / s1 : 0.f;
    }
};

// What the teacher gives to the classes outside the list.
__device__ __forceinline__ float rest_of(const DistillArgs &a, const RowShared &sh) {
    const float pr = 1.f - sh.psum;
    return !a.top_lse || pr < 0.f ? 0.f : pr;         // (NaN stays NaN)
}

// The first wave: sums of the listed exponentials, relative to m.
__device__ __forceinline__ void sum_list(const DistillArgs &a, const RowTotals &t, const RowList &l, bool hard, RowShared &sh) {
    const int lane = threadIdx.x & 63;
    float s = 0.f, s1 = 0.f;
#pragma unroll 1
    for (int j = lane; j < a.k; j += 64)
        if (l.cls[j] >= 0) {
            s += ex2((l.x[j] - t.m) * t.ct);
            if (hard) s1 += ex2((l.x[j] - t.m) * kLog2e);
        }
    s = wave_sumf(s);
    s1 = wave_sumf(s1);
    if (lane == 0) {
        sh.top[0] = s;
        sh.top[1] = s1;
    }
}

// The first wave: the loss.
__device__ __forceinline__ void row_loss(const DistillArgs &a, int64_t row, const RowTotals &t, const RowList &l,
                                         const RowShared &sh, float rest, float pr, float w, bool hard, float xlab) {
    const int lane = threadIdx.x & 63;
    const float unit = loss_unit(a.temperature), invt = unit / a.temperature, logst = t.logst * unit;
    float kl = 0.f;                                   // (times unit)
    if (sh.soft) {
#pragma unroll 1
        for (int j = lane; j < a.k; j += 64)
            if (l.cls[j] >= 0) {
                const float p = l.P[j];
                if (p != 0.f) kl += p * (logf(p) * unit - ((l.x[j] - t.m) * invt - logst));
            }
        kl = wave_sumf(kl);
        if (pr != 0.f) kl += pr * (logf(pr) * unit - (logf(rest) * unit + t.ln_rel - logst));
    }
    if (lane == 0) {
        float loss = sh.soft ? a.alpha * a.temperature * (a.temperature / unit) * kl : 0.f;
        if (hard) loss += (1.f - a.alpha) * (t.m - xlab + logf(t.s1));
        a.loss[row] = w * loss;
    }
}

// The first wave, after the bulk's stores: the gradients of the listed classes and of the label.
template <typename T>
__device__ __forceinline__ void store_list(const DistillArgs &a, const RowTotals &t, const RowList &l, const RowShared &sh,
                                           bool hard, int lab, float xlab, T *dz) {
    const int lane = threadIdx.x & 63;
    bool found = !hard;
#pragma unroll 1
    for (int j = lane; j < a.k; j += 64) {
        const int32_t i = l.cls[j];
        if (i < 0) continue;
        float g = sh.soft ? t.gs * t.at * (ex2((l.x[j] - t.m) * t.ct) / t.st - l.P[j]) : 0.f;
        if (hard) g += t.gb * (ex2((l.x[j] - t.m) * kLog2e) / t.s1 - (i == lab ? 1.f : 0.f));
        found |= hard && i == lab;
        Elem<T>::store(dz + i, g);
    }
    if (!__any(found) && lane == 0) Elem<T>::store(dz + lab, t.co * t.e(xlab) + t.ch * t.e1(xlab) - t.gb);
}

template <int POW>
__device__ __forceinline__ float power(float e) {
    if (POW == kSquare) return e * e;
    if (POW == kFourth) return (e * e) * (e * e);
    return e;
}

// s + power(e)
template <int POW>
__device__ __forceinline__ float add_power(float e, float s) {
    if (POW == kSquare) return fmaf(e, e, s);
    if (POW == kFourth) return fmaf(e * e, e * e, s);
    return s + e;
}

// The gradient outside the list from the exponential at T (not kOwn).
template <int POW>
__device__ __forceinline__ float slope_of(const RowTotals &t, float y) {
    if (POW == kSquare) return y * fmaf(t.ch, y, t.co);
    if (POW == kFourth) return y * fmaf(t.ch * y, y * y, t.co);
    return (t.co + t.ch) * y;                         // (one exponential for both)
}

// ------------------------------------------------------------------ rows in registers
// A workgroup of NT threads has a row of up to NT * NCH * V classes in registers, in fp32: one read of the
// logits and one write of the gradient.  Piece i of thread t is V classes from head + (i NT + t) V; the classes
// before and behind the whole pieces are one each in the first lanes of the last wave (xt).
//
// A row of bf16 that begins between two words leaves its first class to them (head = 1): pieces at any word are
// read as fast as aligned ones, pieces between two words are not (4096 x 50001: 244 us; 205 with a head).
template <typename T>
__device__ __forceinline__ int row_head(const T *z) {
    return sizeof(T) == 2 ? (int)(((uintptr_t)z >> 1) & 1) : 0;
}

// The bits of V classes from j on.  (A piece's may lie in two words; what follows the last word is the list.)
template <int V>
__device__ __forceinline__ uint32_t bits_at(const uint32_t *bits, uint32_t j) {
    const uint32_t lo = bits[j >> 5], hi = V == 8 ? bits[(j >> 5) + 1] : 0;
    return __builtin_amdgcn_alignbit(hi, lo, j & 31) & ((1u << V) - 1u);
}

template <typename T>
__device__ __forceinline__ T *at32(T *p, uint32_t i) {     // (a uniform base and a 32-bit offset)
    typedef typename std::conditional<std::is_const<T>::value, const char, char>::type C;
    return reinterpret_cast<T *>(reinterpret_cast<C *>(p) + i * (uint32_t)sizeof(T));
}

template <typename T, int NT, int NCH, int POW>
__global__ __launch_bounds__(NT) void distill_row_kernel(DistillArgs a, int64_t n, int bit_words) {
    constexpr int V = 16 / sizeof(T), NW = NT / 64;
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ RowShared sh;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = a.c, k = a.k;
    RowList l;
    l.bits = smem;
    l.cls = (int32_t *)(smem + bit_words);
    l.P = (float *)(l.cls + k);
    l.x = l.P + k;
    const bool hard = a.labels != nullptr;
    const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (row >= n) return;
    int tid = fresh(threadIdx.x);
    const T *z = (const T *)a.z + row * a.zld;
    T *dz = (T *)a.dz + row * a.dld;
    const int head = row_head(z), whole = (c - head) / V;
    // this lane's class outside the pieces, which start at zp, dzp, bp
    const int jt = wave == NW - 1 && lane < c - whole * V ? (lane < head ? lane : whole * V + lane) : -1;
    const T *const zp = z + head;
    T *const dzp = dz + head;
    const float *const bp = a.bias ? a.bias + head : nullptr;
    ListHead first{};
    if (wave == 0) first = list_head(a, row);
    const float w = a.weight ? a.weight[row] : 1.f;
    const int lab = hard ? a.labels[row] : -1;
    const bool bad = hard && (lab < 0 || lab >= c);
    bool done = w == 0.f || bad;                  // (uniform) a row that counts for nothing, or has no loss
    float fill = w == 0.f ? 0.f : __builtin_nanf("");
    const bool read_last = a.z != a.dz;           // (in place, the lines are written again at once)
    typename RowVec<T, V>::raw raw[NCH];
    float xt = -INFINITY, xlab = 0.f;
    const auto read = [&]() {
        if (read_last) {
#pragma unroll
            for (int i = 0; i < NCH; ++i)
                if (i * NT + tid < whole) raw[i] = RowVec<T, V>::load_last(at32(zp, (i * NT + tid) * V));
        } else {
            const int tid_ = fresh(tid);              // (equal addresses would make one plain load of the two)
#pragma unroll
            for (int i = 0; i < NCH; ++i)
                if (i * NT + tid_ < whole) raw[i] = RowVec<T, V>::load(at32(zp, (i * NT + tid_) * V));
        }
    };
    constexpr bool kShort = NT == 64;             // short rows: the reads, the bias's too, not after the weight and the label
    typename RowVec<float, V>::raw braw[kShort ? NCH : 1];
    if (kShort) {
        read();
        if (a.bias)
#pragma unroll
            for (int i = 0; i < (kShort ? NCH : 1); ++i)
                if (i * NT + tid < whole) braw[i] = RowVec<float, V>::load(at32(bp, (i * NT + tid) * V));
    }
    if (!done) {
        if (!kShort) read();
        if (jt >= 0) xt = Elem<T>::load(z + jt) + (a.bias ? a.bias[jt] : 0.f);
        if (wave == 0) {
            if (hard) xlab = Elem<T>::load(z + lab) + (a.bias ? a.bias[lab] : 0.f);
            read_list<T>(a, row, first, z, c, l, sh);
        }
        __syncthreads();
        if (!sh.soft && !hard) {
            done = true;
            fill = 0.f;
        }
    }
    if (done) {
        float f[V];
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = fill;
        for (int p = tid; p < whole; p += NT) RowVec<T, V>::store(at32(dzp, p * V), f);
        if (jt >= 0) Elem<T>::store(dz + jt, fill);
        if (tid == 0) a.loss[row] = fill;
        return;
    }

    // x, -inf where listed or past the end; its maximum
    tid = fresh(tid);
    float x[NCH][V];
    if (jt >= 0 && ((l.bits[jt >> 5] >> (jt & 31)) & 1u)) xt = -INFINITY;
    float mx = xt;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
#pragma unroll
        for (int e = 0; e < V; ++e) x[i][e] = -INFINITY;
        if (i * NT + tid < whole) {
            const uint32_t j = (i * NT + tid) * V;
            RowVec<T, V>::unpack(raw[i], x[i]);
            if (a.bias) {
                float b[V];
                RowVec<float, V>::unpack(kShort ? braw[kShort ? i : 0] : RowVec<float, V>::load(at32(bp, j)), b);
#pragma unroll
                for (int e = 0; e < V; ++e) x[i][e] += b[e];
            }
            const uint32_t on = bits_at<V>(l.bits, j + head);
            if (on != 0) {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if ((on >> e) & 1u) x[i][e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) mx = fmaxf(mx, x[i][e]);
        }
        if (i % 2 == 1) __builtin_amdgcn_sched_barrier(0);       // (two pieces' bias at a time in registers)
    }
    mx = wave_maxf(mx);
    if (lane == 0) sh.max[wave] = mx;
    __syncthreads();
    mx = sh.max[0];
#pragma unroll
    for (int q = 1; q < NW; ++q) mx = fmaxf(mx, sh.max[q]);
    RowTotals t;
    t.maxima(mx, sh.mtop, a.temperature, POW);
    if (t.huge) {
        xt -= t.mr;
#pragma unroll
        for (int i = 0; i < NCH; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) x[i][e] -= t.mr;
    }
    // sums; x becomes its exponential, unless both of them are needed again
    float s = 0.f, s1 = 0.f;
    const auto add = [&](float &v) {
        const float y = ex2(fmaf(v, t.ct, -t.R));
        s += y;
        if (POW == kOwn) {
            s1 += ex2(fmaf(v, kLog2e, -t.R1));
            return;
        }
        if (POW != kSame) s1 = add_power<POW>(POW == kFourth ? fresh(y) : y, s1);  // (its square is not kept for the slope)
        v = y;
    };
    add(xt);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
#pragma unroll
        for (int e = 0; e < V; ++e) add(x[i][e]);
        __builtin_amdgcn_sched_barrier(0);
    }
    s = wave_sumf(s);
    if (POW != kSame) s1 = wave_sumf(s1);
    if (lane == 0) {
        sh.sum[wave][0] = s;
        sh.sum[wave][1] = s1;
    }
    if (wave == 0) sum_list(a, t, l, hard, sh);
    __syncthreads();
    s = sh.sum[0][0];
    s1 = sh.sum[0][1];
#pragma unroll
    for (int q = 1; q < NW; ++q) {
        s += sh.sum[q][0];
        s1 += sh.sum[q][1];
    }
    if (POW == kSame) s1 = s;                     // (T = 1, or not used)
    const float pr = rest_of(a, sh);
    t.sums(a, w, s, s1, sh, hard, pr);
    tid = fresh(tid);
    const float R = fresh(t.R), R1 = fresh(t.R1);
    const auto slope = [&](float v) {
        if (POW == kOwn) return fmaf(t.ch, ex2(fmaf(v, kLog2e, -R1)), t.co * ex2(fmaf(v, t.ct, -R)));
        return slope_of<POW>(t, v);
    };
#pragma unroll
    for (int i = 0; i < NCH; ++i)
        if (i * NT + tid < whole) {
            float g[V];
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = slope(x[i][e]);
            RowVec<T, V>::store(at32(dzp, (i * NT + tid) * V), g);
            __builtin_amdgcn_sched_barrier(0);
        }
    if (jt >= 0) Elem<T>::store(dz + jt, slope(xt));
    if (wave == 0) row_loss(a, row, t, l, sh, s, pr, w, hard, xlab);
    __syncthreads();
    if (wave == 0) store_list<T>(a, t, l, sh, hard, lab, xlab, dz);
}

// ------------------------------------------------------------------ wider rows in registers
// The running maximum and sums of a thread, relative to the maximum: exponents r at T, r1 at 1.
template <int POW>
struct Running {
    float M, ct, far, r, r1, s, s1;
    __device__ explicit Running(float temperature)
        : M(-INFINITY), ct(kLog2e / temperature), far(far_of(temperature)), r(-far * ct), r1(-far * kLog2e), s(0.f), s1(0.f) {}

    template <int N>
    __device__ __forceinline__ void add(const float (&x)[N]) {
        float cm = M;
#pragma unroll
        for (int e = 0; e < N; ++e) cm = fmaxf(cm, x[e]);
        M = cm;
        const float at = fminf(fmaxf(cm, -far), far), rn = at * ct, f = ex2(r - rn);
        s *= f;
        if (POW == kOwn) {
            const float rn1 = at * kLog2e;
            s1 *= ex2(r1 - rn1);
            r1 = rn1;
        } else if (POW != kSame) {
            s1 *= power<POW>(f);
        }
        r = rn;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float y = ex2(fmaf(x[e], ct, -rn));
            s += y;
            if (POW == kOwn) s1 += ex2(fmaf(x[e], kLog2e, -r1));
            else if (POW != kSame) s1 = add_power<POW>(y, s1);
        }
    }

    // x as an exact difference from the row's maximum, where t.huge
    __device__ __forceinline__ void add_shifted(float d) {
        const float y = ex2(d * ct);
        s += y;
        if (POW == kOwn) s1 += ex2(d * kLog2e);
        else if (POW != kSame) s1 = add_power<POW>(y, s1);
    }

    // relative to the row's maximum
    __device__ __forceinline__ void settle(const RowTotals &t) {
        const float f = ex2(r - t.R);
        s *= f;
        if (POW == kOwn) s1 *= ex2(r1 - t.R1);
        else if (POW != kSame) s1 *= power<POW>(f);
    }
};

// The gradient outside the list at x (less t.mr where t.huge).
template <int POW>
__device__ __forceinline__ float slope_at(const RowTotals &t, float x) {
    const float y = ex2(fmaf(x, t.ct, -t.R));
    if (POW == kOwn) return fmaf(t.ch, ex2(fmaf(x, kLog2e, -t.R1)), t.co * y);
    return slope_of<POW>(t, y);
}

// Pieces of the logits as they were read, with the listed classes made -inf.
__device__ __forceinline__ void make_inf(u32x4_t &raw, uint32_t on) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if ((on >> (2 * e)) & 1u) raw[e] = (raw[e] & 0xffff0000u) | 0xff80u;
        if ((on >> (2 * e + 1)) & 1u) raw[e] = (raw[e] & 0xffffu) | 0xff800000u;
    }
}
__device__ __forceinline__ void make_inf(f32x4_t &raw, uint32_t on) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if ((on >> e) & 1u) raw[e] = -INFINITY;
}

// As distill_row_kernel, with the logits in registers as they were read (half the registers in bf16, so twice the
// classes, or two workgroups per CU where x in fp32 leaves one): the bias is added twice, and the maximum and
// the sums are formed in one pass, piece by piece.
template <typename T, int NT, int NCH, int POW>
__global__ __launch_bounds__(NT, NT / 256) void distill_raw_kernel(DistillArgs a, int64_t n, int bit_words) {
    constexpr int V = 16 / sizeof(T), NW = NT / 64;
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ RowShared sh;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = a.c, k = a.k;
    RowList l;
    l.bits = smem;
    l.cls = (int32_t *)(smem + bit_words);
    l.P = (float *)(l.cls + k);
    l.x = l.P + k;
    const bool hard = a.labels != nullptr;
    const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (row >= n) return;
    int tid = threadIdx.x;
    const T *z = (const T *)a.z + row * a.zld;
    T *dz = (T *)a.dz + row * a.dld;
    const int head = row_head(z), whole = (c - head) / V;
    // this lane's class outside the pieces, which start at zp, dzp, bp
    const int jt = wave == NW - 1 && lane < c - whole * V ? (lane < head ? lane : whole * V + lane) : -1;
    const T *const zp = z + head;
    T *const dzp = dz + head;
    const float *const bp = a.bias ? a.bias + head : nullptr;
    ListHead first{};
    if (wave == 0) first = list_head(a, row);
    const float w = a.weight ? a.weight[row] : 1.f;
    const int lab = hard ? a.labels[row] : -1;
    const bool bad = hard && (lab < 0 || lab >= c);
    bool done = w == 0.f || bad;                  // (uniform) a row that counts for nothing, or has no loss
    float fill = w == 0.f ? 0.f : __builtin_nanf("");
    typename RowVec<T, V>::raw raw[NCH];
    float xt = -INFINITY, xlab = 0.f;
    if (!done) {
        if (a.z != a.dz) {                        // (in place, the lines are written again at once)
#pragma unroll
            for (int i = 0; i < NCH; ++i)
                if (i * NT + tid < whole) raw[i] = RowVec<T, V>::load_last(at32(zp, (i * NT + tid) * V));
        } else {
            const int tid_ = fresh(tid);          // (equal addresses would make one plain load of the two)
#pragma unroll
            for (int i = 0; i < NCH; ++i)
                if (i * NT + tid_ < whole) raw[i] = RowVec<T, V>::load(at32(zp, (i * NT + tid_) * V));
        }
        if (jt >= 0) xt = Elem<T>::load(z + jt) + (a.bias ? a.bias[jt] : 0.f);
        if (wave == 0) {
            if (hard) xlab = Elem<T>::load(z + lab) + (a.bias ? a.bias[lab] : 0.f);
            read_list<T>(a, row, first, z, c, l, sh);
        }
        __syncthreads();
        if (!sh.soft && !hard) {
            done = true;
            fill = 0.f;
        }
    }
    if (done) {
        float f[V];
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = fill;
        for (int p = tid; p < whole; p += NT) RowVec<T, V>::store(at32(dzp, p * V), f);
        if (jt >= 0) Elem<T>::store(dz + jt, fill);
        if (tid == 0) a.loss[row] = fill;
        return;
    }
    tid = fresh(tid);
    const auto x_of = [&](int i, float(&x)[V]) {
        RowVec<T, V>::unpack(raw[i], x);
        if (a.bias) {
            float b[V];
            RowVec<float, V>::unpack(RowVec<float, V>::load(at32(bp, (i * NT + tid) * V)), b);
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] += b[e];
        }
    };
    if (jt >= 0 && ((l.bits[jt >> 5] >> (jt & 31)) & 1u)) xt = -INFINITY;
    Running<POW> run(a.temperature);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
        if (i * NT + tid < whole) {
            const uint32_t on = bits_at<V>(l.bits, (i * NT + tid) * V + head);
            if (on != 0) make_inf(raw[i], on);
            float x[V];
            x_of(i, x);
            run.add(x);
        }
        if (i % 2 == 1) __builtin_amdgcn_sched_barrier(0);       // (two pieces' bias at a time in registers)
    }
    {
        const float x[1] = {xt};
        run.add(x);
    }
    float mx = wave_maxf(run.M);
    if (lane == 0) sh.max[wave] = mx;
    __syncthreads();
    mx = sh.max[0];
#pragma unroll
    for (int q = 1; q < NW; ++q) mx = fmaxf(mx, sh.max[q]);
    RowTotals t;
    t.maxima(mx, sh.mtop, a.temperature, POW);
    const bool huge = __builtin_amdgcn_readfirstlane(t.huge);
    if (huge) {
        run.s = run.s1 = 0.f;
#pragma unroll
        for (int i = 0; i < NCH; ++i)
            if (i * NT + tid < whole) {
                float x[V];
                x_of(i, x);
#pragma unroll
                for (int e = 0; e < V; ++e) run.add_shifted(x[e] - t.mr);
            }
        xt -= t.mr;
        run.add_shifted(xt);
    } else {
        run.settle(t);
    }
    float s = wave_sumf(run.s), s1 = POW != kSame ? wave_sumf(run.s1) : 0.f;
    if (lane == 0) {
        sh.sum[wave][0] = s;
        sh.sum[wave][1] = s1;
    }
    if (wave == 0) sum_list(a, t, l, hard, sh);
    __syncthreads();
    s = sh.sum[0][0];
    s1 = sh.sum[0][1];
#pragma unroll
    for (int q = 1; q < NW; ++q) {
        s += sh.sum[q][0];
        s1 += sh.sum[q][1];
    }
    if (POW == kSame) s1 = s;                     // (T = 1, or not used)
    const float pr = rest_of(a, sh);
    t.sums(a, w, s, s1, sh, hard, pr);
    tid = fresh(tid);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
        if (i * NT + tid < whole) {
            float g[V];
            x_of(i, g);
            if (huge)
#pragma unroll
                for (int e = 0; e < V; ++e) g[e] -= t.mr;
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = slope_at<POW>(t, g[e]);
            RowVec<T, V>::store(at32(dzp, (i * NT + tid) * V), g);
        }
        if (i % 2 == 1) __builtin_amdgcn_sched_barrier(0);
    }
    if (jt >= 0) Elem<T>::store(dz + jt, slope_at<POW>(t, xt));
    if (wave == 0) row_loss(a, row, t, l, sh, s, pr, w, hard, xlab);
    __syncthreads();
    if (wave == 0) store_list<T>(a, t, l, sh, hard, lab, xlab, dz);
}

// ------------------------------------------------------------------ long rows
// Rows that do not fit the registers are read twice: once for the maximum and the sums together (each thread
// keeps its own running maximum and sums relative to it), once for the gradient; the second read of a row
// follows the first closely enough to come from the caches (1024 x 262144 bf16 361 us, 3.0 TB/s).  The bits are
// those of kSeg classes at a time.
constexpr int kSeg = 262144, kLongThreads = 1024, kLongPieces = 4;

// f(j, x) for the pieces of V classes from j0 on, j0 + NT V, ... below j1 (whole pieces), UN at a time; their
// loads come before all else.
template <typename T, int V, int UN, int NT, typename F>
__device__ __forceinline__ void for_pieces(const T *z, const float *bias, int j0, int j1, bool last, F f) {
    for (int j = j0 + (int)threadIdx.x * V; j < j1; j += UN * NT * V) {
        typename RowVec<T, V>::raw raw[UN];
        typename RowVec<float, V>::raw b[UN];
        if (last) {
#pragma unroll
            for (int u = 0; u < UN; ++u) raw[u] = RowVec<T, V>::load_last(z + min(j + u * NT * V, j1 - V));
        } else {
            const int j_ = fresh(j);                  // (equal addresses would make one plain load of the two)
#pragma unroll
            for (int u = 0; u < UN; ++u) raw[u] = RowVec<T, V>::load(z + min(j_ + u * NT * V, j1 - V));
        }
        if (bias)
#pragma unroll
            for (int u = 0; u < UN; ++u) b[u] = RowVec<float, V>::load(bias + min(j + u * NT * V, j1 - V));
        float x[UN][V];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            RowVec<T, V>::unpack(raw[u], x[u]);
            if (bias) {
                float w[V];
                RowVec<float, V>::unpack(b[u], w);
#pragma unroll
                for (int e = 0; e < V; ++e) x[u][e] += w[e];
            }
        }
        f(j, x);
    }
}

template <typename T, int POW>
__global__ __launch_bounds__(kLongThreads) void distill_long_kernel(DistillArgs a, int64_t n, int bit_words) {
    constexpr int V = 16 / sizeof(T), NT = kLongThreads, NW = NT / 64, UN = kLongPieces;
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ RowShared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = a.c, k = a.k, whole = c / V * V;
    const int jt = wave == NW - 1 && lane < c - whole ? whole + lane : -1;              // this lane's class past the pieces
    RowList l;
    l.bits = smem;
    l.cls = (int32_t *)(smem + bit_words);
    l.P = (float *)(l.cls + k);
    l.x = l.P + k;
    const bool hard = a.labels != nullptr;
    const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (row >= n) return;
    const T *z = (const T *)a.z + row * a.zld;
    T *dz = (T *)a.dz + row * a.dld;
    ListHead first{};
    if (wave == 0) first = list_head(a, row);
    const float w = a.weight ? a.weight[row] : 1.f;
    const int lab = hard ? a.labels[row] : -1;
    const bool bad = hard && (lab < 0 || lab >= c);
    bool done = w == 0.f || bad;                  // (uniform) a row that counts for nothing, or has no loss
    float fill = w == 0.f ? 0.f : __builtin_nanf("");
    float xt = -INFINITY, xlab = 0.f;
    if (!done) {
        if (jt >= 0) xt = Elem<T>::load(z + jt) + (a.bias ? a.bias[jt] : 0.f);
        if (wave == 0) {
            if (hard) xlab = Elem<T>::load(z + lab) + (a.bias ? a.bias[lab] : 0.f);
            read_list<T>(a, row, first, z, min(c, kSeg), l, sh);
        }
        __syncthreads();
        if (!sh.soft && !hard) {
            done = true;
            fill = 0.f;
        }
    }
    if (done) {
        float f[V];
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = fill;
        for (int j = tid * V; j < whole; j += NT * V) RowVec<T, V>::store(dz + j, f);
        if (jt >= 0) Elem<T>::store(dz + jt, fill);
        if (tid == 0) a.loss[row] = fill;
        return;
    }
    // f(x) for the pieces' classes, listed ones and those past the end -inf
    const auto outside = [&](bool marked, auto f) {
        for (int s0 = 0; s0 < c; s0 += kSeg) {
            if (s0 > 0 || !marked) {              // (read_list has marked the first segment)
                __syncthreads();
                if (wave == 0) {
                    clear_bits(l.bits, min(c, kSeg));
                    wave_sync();
#pragma unroll 1
                    for (int j = lane; j < k; j += 64) {
                        const int32_t i = l.cls[j];
                        if (i >= s0 && i - s0 < kSeg) atomicOr(&l.bits[(i - s0) >> 5], 1u << ((i - s0) & 31));
                    }
                }
                __syncthreads();
            }
            const int s1 = min(whole, s0 + kSeg);
            for_pieces<T, V, UN, NT>(z, a.bias, s0, s1, false, [&](int j, float(&x)[UN][V]) {
#pragma unroll
                for (int u = 0; u < UN; ++u) {
                    const int q = j + u * NT * V - s0;
                    const uint32_t on = q < s1 - s0 ? (l.bits[q >> 5] >> (q & 31)) & ((1u << V) - 1u) : (1u << V) - 1u;
                    if (on != 0) {
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            if ((on >> e) & 1u) x[u][e] = -INFINITY;
                    }
                }
                f(x);
            });
            if (s0 + kSeg >= c && jt >= 0 && ((l.bits[(jt - s0) >> 5] >> ((jt - s0) & 31)) & 1u)) xt = -INFINITY;
        }
    };
    Running<POW> run(a.temperature);
    outside(true, [&](float(&x)[UN][V]) { run.add(*reinterpret_cast<float(*)[UN * V]>(&x)); });
    {
        const float x[1] = {xt};
        run.add(x);
    }
    float mx = wave_maxf(run.M);
    if (lane == 0) sh.max[wave] = mx;
    __syncthreads();
    mx = sh.max[0];
#pragma unroll
    for (int q = 1; q < NW; ++q) mx = fmaxf(mx, sh.max[q]);
    RowTotals t;
    t.maxima(mx, sh.mtop, a.temperature, POW);
    const bool huge = __builtin_amdgcn_readfirstlane(t.huge);
    if (huge) {                                   // (read again)
        run.s = run.s1 = 0.f;
        outside(c <= kSeg, [&](float(&x)[UN][V]) {
#pragma unroll
            for (int u = 0; u < UN; ++u)
#pragma unroll
                for (int e = 0; e < V; ++e) run.add_shifted(x[u][e] - t.mr);
        });
        xt -= t.mr;
        run.add_shifted(xt);
    } else {
        run.settle(t);
    }
    float s = wave_sumf(run.s), s1 = POW != kSame ? wave_sumf(run.s1) : 0.f;
    if (lane == 0) {
        sh.sum[wave][0] = s;
        sh.sum[wave][1] = s1;
    }
    if (wave == 0) sum_list(a, t, l, hard, sh);
    __syncthreads();
    s = sh.sum[0][0];
    s1 = sh.sum[0][1];
#pragma unroll
    for (int q = 1; q < NW; ++q) {
        s += sh.sum[q][0];
        s1 += sh.sum[q][1];
    }
    if (POW == kSame) s1 = s;                     // (T = 1, or not used)
    const float pr = rest_of(a, sh);
    t.sums(a, w, s, s1, sh, hard, pr);
    for_pieces<T, V, UN, NT>(z, a.bias, 0, whole, a.z != a.dz, [&](int j, float(&x)[UN][V]) {
        if (huge)
#pragma unroll
            for (int u = 0; u < UN; ++u)
#pragma unroll
                for (int e = 0; e < V; ++e) x[u][e] -= t.mr;
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            float g[V];
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = slope_at<POW>(t, x[u][e]);
            if (j + u * NT * V >= whole) break;
            RowVec<T, V>::store(dz + j + u * NT * V, g);
        }
    });
    if (jt >= 0) Elem<T>::store(dz + jt, slope_at<POW>(t, xt));
    if (wave == 0) row_loss(a, row, t, l, sh, s, pr, w, hard, xlab);
    __syncthreads();
    if (wave == 0) store_list<T>(a, t, l, sh, hard, lab, xlab, dz);
}

// ------------------------------------------------------------------ launch
// A workgroup per row; the threads of one grid dimension have to stay below 2^32.
static dim3 row_grid(int64_t n) {
    const int64_t x = std::min<int64_t>(n, 1 << 20);
    return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

// (Short rows are bound by latencies: exponentials of their own cost them nothing.)
template <typename T, int NT, int NCH>
static void launch_rows(const DistillArgs &a, int64_t n, int kind, size_t lds, int words, hipStream_t st) {
    const dim3 g = row_grid(n);
#define TFK_GO(POW) hipLaunchKernelGGL((distill_row_kernel<T, NT, NCH, POW>), g, dim3(NT), lds, st, a, n, words)
    if (kind == kSame) TFK_GO(kSame);
    else if (NT >= 512 && kind == kSquare) TFK_GO(NT >= 512 ? kSquare : kOwn);
    else if (NT >= 512 && kind == kFourth) TFK_GO(NT >= 512 ? kFourth : kOwn);
    else TFK_GO(kOwn);
#undef TFK_GO
}

// The least threads that hold the row with two, three or more workgroups per CU: a wave for rows of up to 256
// pieces (4096 x 1000 bf16: 14 us; 22 by 256 threads), then 256 (4096 x 4000: 27 us; 52 by 512) and 512, each
// with the least pieces a thread that suffice (4096 x 32000: 152 us with 10; 238 in one workgroup of 1024).
// From 5120 pieces on the row as it was read keeps two workgroups per CU (4096 x 50000 with labels: 208 us; x
// in fp32 and one workgroup 290), unless there is a row per CU at most: then 1024 threads have it sooner
// (256 x 50000: 17 us; 21.6).
constexpr int kCUs = 256;

template <typename T>
static hipError_t launch_typed(const DistillArgs &a, int64_t n, hipStream_t st) {
    const int pieces = (a.c + (int)(16 / sizeof(T)) - 1) / (int)(16 / sizeof(T));
    const int words = (std::min(a.c, kSeg) + 127) / 128 * 4;
    const size_t lds = (size_t)words * 4 + (size_t)a.k * 12;
    const int kind = a.labels == nullptr || a.temperature == 1.f ? kSame
                     : a.temperature == 2.f ? kSquare : a.temperature == 4.f ? kFourth : kOwn;
    if (pieces <= 64 * 2) launch_rows<T, 64, 2>(a, n, kind, lds, words, st);
    else if (pieces <= 64 * 4) launch_rows<T, 64, 4>(a, n, kind, lds, words, st);
    else if (pieces <= 256 * 2) launch_rows<T, 256, 2>(a, n, kind, lds, words, st);
    else if (pieces <= 256 * 4) launch_rows<T, 256, 4>(a, n, kind, lds, words, st);
    else if (pieces <= 512 * 4) launch_rows<T, 512, 4>(a, n, kind, lds, words, st);
    else if (pieces <= 512 * 7) launch_rows<T, 512, 7>(a, n, kind, lds, words, st);
    else if (pieces <= 512 * 10) launch_rows<T, 512, 10>(a, n, kind, lds, words, st);
    else if (pieces <= 1024 * 8 && n <= kCUs) launch_rows<T, 1024, 8>(a, n, kind, lds, words, st);
    else {
        const dim3 g = row_grid(n);
#define TFK_GO(POW)                                                                                                   \
    do {                                                                                                              \
        if (pieces <= 512 * 16)                                                                                       \
            hipLaunchKernelGGL((distill_raw_kernel<T, 512, 16, POW>), g, dim3(512), lds, st, a, n, words);            \
        else if (pieces <= 1024 * 16)                                                                                 \
            hipLaunchKernelGGL((distill_raw_kernel<T, 1024, 16, POW>), g, dim3(1024), lds, st, a, n, words);          \
        else                                                                                                          \
            hipLaunchKernelGGL((distill_long_kernel<T, POW>), g, dim3(kLongThreads), lds, st, a, n, words);           \
    } while (0)
        if (kind == kSame) TFK_GO(kSame);
        else if (kind == kSquare) TFK_GO(kSquare);
        else if (kind == kFourth) TFK_GO(kFourth);
        else TFK_GO(kOwn);
#undef TFK_GO
    }
    return hipGetLastError();
}

hipError_t launch_distill(int dt, int64_t n, const DistillArgs &a, hipStream_t st) {
    return dt == 0 ? launch_typed<float>(a, n, st) : launch_typed<bf16_t>(a, n, st);
}

}  // namespace tfk

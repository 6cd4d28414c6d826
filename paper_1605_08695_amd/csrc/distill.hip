// Distillation from a teacher's top logits: per row, the loss and its gradient in one launch.
//
// With x = logits + bias, u = x / T, K the distinct classes in the row's list, P_j the sum of the
// teacher's probabilities of class j's entries, P_r what the teacher gives to all other classes (0
// where its list is renormalised), q = softmax(u), q_r = sum of q over the classes outside K:
//   soft = sum_K P_j (log P_j - log q_j) + P_r (log P_r - log q_r)        (terms with P = 0 are 0)
//   hard = logsumexp(x) - x_label
//   loss = w (alpha T^2 soft + (1 - alpha) hard)
//   dx_j = scale w (alpha T (q_j - P_j)              + (1 - alpha) (softmax(x)_j - [j = label]))   j in K
//   dx_j = scale w (alpha T q_j (q_r - P_r) / q_r    + (1 - alpha) (softmax(x)_j - [j = label]))   else
// The classes outside K have their own maximum m_r and sum S_r = sum exp((x - m_r) / T), so that
// q_j / q_r = exp((x_j - m_r) / T) / S_r and log q_r lose nothing where the listed classes hold nearly
// all of the student's probability.  A bit per class, in LDS, tells the listed ones apart.
#include "common.h"
#include "kernels.h"

namespace tfk {

constexpr int kDistillThreads = 256;
constexpr int kDistillSeg = 65536;                    // classes whose bits are in LDS at a time

// Block-wide maxima / sums of NV values at once, in a fixed order; every thread gets the results.
template <int NV, bool MAX>
__device__ __forceinline__ void block_reduce(float (&v)[NV], float *red) {
    constexpr int nw = kDistillThreads / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        for (int o = 32; o > 0; o >>= 1) {
            const float w = __shfl_xor(v[i], o, 64);
            v[i] = MAX ? fmaxf(v[i], w) : v[i] + w;
        }
    __syncthreads();                                  // red may still be read
    if (lane == 0)
        for (int i = 0; i < NV; ++i) red[i * nw + wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        v[i] = red[i * nw];
        for (int w = 1; w < nw; ++w) v[i] = MAX ? fmaxf(v[i], red[i * nw + w]) : v[i] + red[i * nw + w];
    }
}

template <typename T, typename TT>
__global__ __launch_bounds__(kDistillThreads) void distill_kernel(DistillArgs a) {
    extern __shared__ uint32_t smem[];
    __shared__ float red[4 * kDistillThreads / 64];
    constexpr int NT = kDistillThreads;
    const int tid = threadIdx.x, c = a.c, k = a.k;
    const int seg_words = (min(c, kDistillSeg) + 31) / 32;
    int32_t *cls = (int32_t *)smem;                   // [k] the entry's class; -1: none, or another entry stands for it
    float *lp = (float *)(cls + k);                   // [k] the entry's log-probability
    float *P = lp + k;                                // [k] its class's probability
    float *xs = P + k;                                // [k] the student's x there
    uint32_t *bits = (uint32_t *)(xs + k);            // [seg_words]
    const int64_t row = blockIdx.x;
    const T *z = (const T *)a.z + row * a.zld;
    T *dz = (T *)a.dz + row * a.dld;
    const float w = a.weight ? a.weight[row] : 1.f;
    const bool hard = a.labels != nullptr;
    const int lab = hard ? a.labels[row] : -1;
    const bool bad = hard && (lab < 0 || lab >= c);
    if (w == 0.f || bad) {                            // (uniform) a row that counts for nothing, or has no loss
        const float v = w == 0.f ? 0.f : __builtin_nanf("");
        for (int j = tid; j < c; j += NT) Elem<T>::store(dz + j, v);
        if (tid == 0) a.loss[row] = v;
        return;
    }
    const float invt = 1.f / a.temperature, beta = 1.f - a.alpha;
    const float c1 = 1.44269504088896341f, ct = c1 / a.temperature;   // exp(y / T) = 2^(y ct)
    const auto load_x = [&](int j) { return Elem<T>::load(z + j) + (a.bias ? a.bias[j] : 0.f); };
    const float xlab = hard ? load_x(lab) : 0.f;

    // ---- the teacher
    const int32_t *idx = a.top_idx + row * k;
    const TT *top = (const TT *)a.top + row * k;
    float tm[1] = {-INFINITY};
    for (int j = tid; j < k; j += NT) {
        const int32_t i = idx[j];
        const bool ok = i >= 0 && i < c;
        const float t = ok ? Elem<TT>::load(top + j) : -INFINITY;
        cls[j] = ok ? i : -1;
        lp[j] = t;
        tm[0] = fmaxf(tm[0], t != t ? INFINITY : t);
    }
    block_reduce<1, true>(tm, red);
    const bool soft = a.top_lse != nullptr || tm[0] > -INFINITY;
    float ref = 0.f, lse[1] = {0.f};                  // log p = (t - ref) / T - lse
    if (a.top_lse) {
        lse[0] = a.top_lse[row];
    } else {
        ref = tm[0];
        for (int j = tid; j < k; j += NT)
            if (cls[j] >= 0) lse[0] += expf((lp[j] - ref) * invt);
        block_reduce<1, false>(lse, red);
        lse[0] = logf(lse[0]);
    }
    for (int j = tid; j < k; j += NT)
        if (cls[j] >= 0) {
            lp[j] = (lp[j] - ref) * invt - lse[0];
            xs[j] = load_x(cls[j]);
        }
    __syncthreads();
    for (int j = tid; j < k; j += NT) {               // entries of one class are added up by the first
        const int32_t i = cls[j];
        float p = 0.f;
        for (int q = 0; q < k && i >= 0; ++q)
            if (cls[q] == i) {
                if (q < j) {
                    p = -1.f;
                    break;
                }
                p += expf(lp[q]);
            }
        P[j] = p;
    }
    __syncthreads();
    for (int j = tid; j < k; j += NT)
        if (P[j] < 0.f) cls[j] = -1;

    // ---- the student: maxima, then sums, outside the list (relative to mr) and on it (relative to m)
    const auto mark = [&](int s0) {                   // the bits of the listed among classes s0 ...
        __syncthreads();
        for (int q = tid; q < seg_words; q += NT) bits[q] = 0;
        __syncthreads();
        for (int j = tid; j < k; j += NT) {
            const int32_t i = cls[j];
            if (i >= s0 && i - s0 < kDistillSeg) atomicOr(&bits[(i - s0) >> 5], 1u << ((i - s0) & 31));
        }
        __syncthreads();
    };
    const auto listed = [&](int j) { return ((bits[j >> 5] >> (j & 31)) & 1u) != 0; };
    float mx[2] = {-INFINITY, -INFINITY};
    for (int s0 = 0; s0 < c; s0 += kDistillSeg) {
        mark(s0);
        for (int j = tid; j < min(c - s0, kDistillSeg); j += NT)
            if (!listed(j)) mx[0] = fmaxf(mx[0], load_x(s0 + j));
    }
    for (int j = tid; j < k; j += NT)
        if (cls[j] >= 0) mx[1] = fmaxf(mx[1], xs[j]);
    block_reduce<2, true>(mx, red);
    const float m = fmaxf(mx[0], mx[1]), mr = mx[0] > -INFINITY ? mx[0] : 0.f;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};              // outside at T, at 1; listed at T, at 1
    for (int s0 = 0; s0 < c; s0 += kDistillSeg) {
        if (c > kDistillSeg) mark(s0);
        for (int j = tid; j < min(c - s0, kDistillSeg); j += NT)
            if (!listed(j)) {
                const float x = load_x(s0 + j) - mr;
                sum[0] += exp2f(x * ct);
                if (hard) sum[1] += exp2f(x * c1);
            }
    }
    for (int j = tid; j < k; j += NT)
        if (cls[j] >= 0) {
            sum[2] += exp2f((xs[j] - m) * ct);
            if (hard) sum[3] += exp2f((xs[j] - m) * c1);
        }
    block_reduce<4, false>(sum, red);
    const float relt = mx[0] > -INFINITY ? exp2f((mr - m) * ct) : 0.f, rel1 = mx[0] > -INFINITY ? exp2f((mr - m) * c1) : 0.f;
    const float st = sum[2] + sum[0] * relt, s1 = sum[3] + sum[1] * rel1;
    const float logst = logf(st), qr = sum[0] * relt / st;

    // ---- the loss
    float pl[2] = {0.f, 0.f};                         // the listed P; their terms
    for (int j = tid; j < k; j += NT)
        if (cls[j] >= 0) {
            const float p = P[j];
            pl[0] += p;
            if (p != 0.f) pl[1] += p * (logf(p) - ((xs[j] - m) * invt - logst));
        }
    block_reduce<2, false>(pl, red);
    float pr = a.top_lse ? 1.f - pl[0] : 0.f;
    if (pr < 0.f) pr = 0.f;
    if (tid == 0) {
        float loss = 0.f;
        if (soft) {
            if (pr != 0.f) pl[1] += pr * (logf(pr) - (logf(sum[0]) + (mr - m) * invt - logst));
            loss = a.alpha * a.temperature * a.temperature * pl[1];
        }
        if (hard) loss += beta * (m - xlab + logf(s1));
        a.loss[row] = w * loss;
    }

    // ---- the gradient, as if no class were listed, then the listed ones
    const float gs = a.scale * w, at = a.alpha * a.temperature, gb = gs * beta;
    const float co = !soft ? 0.f : (sum[0] != 0.f ? gs * at * (qr - pr) / sum[0] : gs * at * qr);
    const float ch = hard ? gb * rel1 / s1 : 0.f;
    for (int j = tid; j < c; j += NT) {
        const float x = load_x(j) - mr;
        float g = soft ? co * exp2f(x * ct) : 0.f;
        if (hard) g += ch * exp2f(x * c1);
        if (j == lab) g -= gb;
        Elem<T>::store(dz + j, g);
    }
    __syncthreads();
    for (int j = tid; j < k; j += NT) {
        const int32_t i = cls[j];
        if (i < 0) continue;
        float g = soft ? gs * at * (exp2f((xs[j] - m) * ct) / st - P[j]) : 0.f;
        if (hard) g += gb * (exp2f((xs[j] - m) * c1) / s1 - (i == lab ? 1.f : 0.f));
        Elem<T>::store(dz + i, g);
    }
}

hipError_t launch_distill(int dt, int top_dt, int64_t n, const DistillArgs &a, hipStream_t st) {
    const size_t lds = (size_t)a.k * 16 + (size_t)(std::min(a.c, kDistillSeg) + 31) / 32 * 4;
#define TFK_GO(T, TT) \
    hipLaunchKernelGGL((distill_kernel<T, TT>), dim3((unsigned)n), dim3(kDistillThreads), lds, st, a)
    if (dt == 0 && top_dt == 0) TFK_GO(float, float);
    else if (dt == 0) TFK_GO(float, bf16_t);
    else if (top_dt == 0) TFK_GO(bf16_t, float);
    else TFK_GO(bf16_t, bf16_t);
#undef TFK_GO
    return hipGetLastError();
}

}  // namespace tfk

// Log-probabilities of given tokens, the entropy and the largest classes of rows of logits, and the gradient of
// the first two.
//
// With x = logits + bias, m = max x, u = (x - m) / T, s = sum e^u, W = sum u e^u:
//   lse = m / T + log s     logp = u_token - log s     entropy = log s - W / s
//   dx_j = (dlogp ([j = token] - p_j) - dentropy p_j (log p_j + entropy)) / T,   p_j = e^(x_j / T - lse)
// A class of -inf has p = 0 and no term.  The sums run with the maximum seen so far: where it rises by D, W
// becomes (W - D s) e^-D.  The largest classes are ordered by x, then by the lower class.
#include "common.h"
#include "kernels.h"

#pragma clang fp contract(off)

namespace tfk {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

__device__ __forceinline__ float exp_of(float u) { return __builtin_amdgcn_exp2f(u * kLog2e); }

// x's order as an unsigned number (+0 and -0 alike), 0 for -inf and below every finite x's.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    const uint32_t k = b ^ (uint32_t)((int32_t)b >> 31 | (int32_t)0x80000000);
    return x == -INFINITY ? 0u : k;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// Maximum, sum and weighted sum of a part of a row.
struct Part {
    float m, s, W;
    // Terms further than 200 below the maximum are 0, and so is their share of W.
    __device__ void add(float x, float invT) {
        if (x > m) {
            const float D = m == -INFINITY ? 0.f : (x - m) * invT, r = m == -INFINITY ? 0.f : exp_of(-D);
            W = (W - fminf(D, 200.f) * s) * r;
            s *= r;
            m = x;
        }
        const float u = m == -INFINITY ? x : (x - m) * invT;
        const float e = exp_of(u);
        s += e;
        W = __builtin_fmaf(u < -200.f ? 0.f : u, e, W);
    }
    __device__ void join(const Part &o, float invT) {
        const float M = fmaxf(m, o.m);
        const float D = m == -INFINITY ? 0.f : (M - m) * invT, E = o.m == -INFINITY ? 0.f : (M - o.m) * invT;
        const float r = exp_of(-D), t = exp_of(-E);
        W = (W - fminf(D, 200.f) * s) * r + (o.W - fminf(E, 200.f) * o.s) * t;
        s = s * r + o.s * t;
        m = M;
    }
};

template <typename T>
__global__ __launch_bounds__(256) void logprob_kernel(LogprobArgs a) {
    __shared__ Part parts[4];
    __shared__ unsigned long long best[4];
    const int64_t r = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (r >= a.n) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const float invT = 1.f / a.temperature;
    const int token = a.tokens ? a.tokens[r] : 0;
    if (a.tokens && (token < 0 || token >= a.c)) {       // padding: the logits are not looked at
        if (threadIdx.x == 0) {
            if (a.logp) a.logp[r] = 0.f;
            if (a.entropy) a.entropy[r] = 0.f;
            if (a.lse) a.lse[r] = 0.f;
        }
        for (int q = threadIdx.x; q < a.k; q += 256) {
            a.top_idx[r * a.k + q] = -1;
            a.top_logp[r * a.k + q] = -INFINITY;
        }
        return;
    }
    const T *const z = (const T *)a.z + r * a.zld;
    Part p{-INFINITY, 0.f, 0.f};
    for (int j = threadIdx.x; j < a.c; j += 256) p.add(Elem<T>::load(z + j) + (a.bias ? a.bias[j] : 0.f), invT);
    for (int o = 32; o > 0; o >>= 1) p.join(Part{__shfl_xor(p.m, o), __shfl_xor(p.s, o), __shfl_xor(p.W, o)}, invT);
    if (lane == 0) parts[w] = p;
    __syncthreads();
    p = parts[0];
    for (int v = 1; v < 4; ++v) p.join(parts[v], invT);
    const bool empty = p.m == -INFINITY && p.s == 0.f, nan = !(p.s < INFINITY);
    const float ls = __builtin_amdgcn_logf(p.s) * kLn2;
    if (threadIdx.x == 0) {
        if (a.logp) {
            const float x = Elem<T>::load(z + token) + (a.bias ? a.bias[token] : 0.f);
            a.logp[r] = empty ? -INFINITY : nan ? NAN : (x - p.m) * invT - ls;
        }
        if (a.entropy) a.entropy[r] = empty ? 0.f : nan ? NAN : fmaxf(ls - p.W / p.s, 0.f);
        if (a.lse) a.lse[r] = empty ? -INFINITY : nan ? NAN : p.m * invT + ls;
    }
    unsigned long long last = ~0ull;
    for (int q = 0; q < a.k; ++q) {
        unsigned long long mine = 0;
        if (!nan && !empty && last != 0)
            for (int j = threadIdx.x; j < a.c; j += 256) {
                const unsigned long long key =
                    (unsigned long long)order_of(Elem<T>::load(z + j) + (a.bias ? a.bias[j] : 0.f)) << 32 | (uint32_t)~j;
                if (key < last && key > mine) mine = key;
            }
        for (int o = 32; o > 0; o >>= 1) {
            const unsigned long long other = __shfl_xor(mine, o);
            mine = other > mine ? other : mine;
        }
        __syncthreads();
        if (lane == 0) best[w] = mine;
        __syncthreads();
        for (int v = 0; v < 4; ++v) mine = best[v] > mine ? best[v] : mine;
        if ((mine >> 32) == 0) mine = 0;             // nothing but -inf is left
        if (threadIdx.x == 0) {
            a.top_idx[r * a.k + q] = mine ? (int32_t)~(uint32_t)mine : -1;
            a.top_logp[r * a.k + q] = nan ? NAN : mine ? (value_of((uint32_t)(mine >> 32)) - p.m) * invT - ls : -INFINITY;
        }
        last = mine;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void logprob_bwd_kernel(LogprobBwdArgs a) {
    const int64_t r = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (r >= a.n) return;
    const T *const z = (const T *)a.z + r * a.zld;
    T *const dz = (T *)a.dz + r * a.dld;
    const int token = a.tokens[r];
    const float lse = a.lse[r];
    const bool none = token < 0 || token >= a.c || lse == -INFINITY;
    const float invT = 1.f / a.temperature, dl = a.dlogp[r] * invT, de = a.dentropy ? a.dentropy[r] * invT : 0.f;
    const float H = a.dentropy ? a.entropy[r] : 0.f;
    for (int j = threadIdx.x; j < a.c; j += 256) {
        float g = 0.f;
        if (!none) {
            const float lp = (Elem<T>::load(z + j) + (a.bias ? a.bias[j] : 0.f)) * invT - lse;
            const float p = exp_of(lp);
            g = -p * (dl + de * ((lp < -200.f ? -200.f : lp) + H)) + (j == token ? dl : 0.f);
        }
        Elem<T>::store(dz + j, g);
    }
}

hipError_t launch_logprob(int dt, const LogprobArgs &a, hipStream_t st) {
    if (dt == 0) hipLaunchKernelGGL(logprob_kernel<float>, grid_2d(a.n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(logprob_kernel<bf16_t>, grid_2d(a.n), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_logprob_bwd(int dt, const LogprobBwdArgs &a, hipStream_t st) {
    if (dt == 0) hipLaunchKernelGGL(logprob_bwd_kernel<float>, grid_2d(a.n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(logprob_bwd_kernel<bf16_t>, grid_2d(a.n), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace tfk

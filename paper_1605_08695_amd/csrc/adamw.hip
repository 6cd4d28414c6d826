// AdamW over many variables in one launch per batch of them, moments in fp32 or in 8 bits.
//
//   m <- b1 m + (1 - b1) g          v <- b2 v + (1 - b2) g^2
//   var <- var - lr wd var - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
// In 8 bits a moment is an e4m3 value (four significant bits, 18 powers of two) times its block's scale, one fp32
// number for each 256 values of a variable: scale = largest / 448, so that the largest is e4m3's largest.  The
// second moment is kept as its square root, which halves its range in powers of two, and never becomes 0 where it
// was not: its smallest value is e4m3's smallest, 2^-9 of 448, so that a rounded moment makes a step smaller and
// not larger.  The step itself is made with the moments before they are rounded.
#include "common.h"
#include "kernels.h"

#pragma clang fp contract(off)

namespace tfk {

constexpr float kTop = 448.f, kLeast = 0x1p-9f, kNothing = 0x1p-100f;

__device__ __forceinline__ float wave_max_bits(float v) {
    uint32_t b = __float_as_uint(v) & 0x7fffffffu;        // as whole numbers NaN is the largest
    for (int o = 32; o > 0; o >>= 1) b = max(b, (uint32_t)__shfl_xor((int)b, o));
    return __uint_as_float(b);
}

__device__ __forceinline__ float step_of(float m, float v, const AdamwParams &p) {
    return p.lr * m / (__builtin_sqrtf(v * p.rc2) + p.eps);
}

// One wave has one block of 256 values, four a lane.
template <bool BITS8>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwBatch b, AdamwParams p) {
    const int64_t blk0 = (blockIdx.x + (int64_t)blockIdx.y * gridDim.x) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (blk0 >= b.blk_start[b.count]) return;
    int i = 0;
    while (blk0 >= b.blk_start[i + 1]) ++i;
    const int64_t blk = blk0 - b.blk_start[i], n = b.n[i];
    float m[4], v[4];
    float ms = 0.f, vs = 0.f;
    if (BITS8) {
        ms = b.m_scale[i][blk];
        vs = b.v_scale[i][blk];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t at = blk * 256 + lane + 64 * e;
        m[e] = v[e] = 0.f;
        if (at >= n) continue;
        const float g = b.grad[i][at];
        float var = b.var[i][at];
        if (BITS8) {
            m[e] = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)b.m[i])[at], 0) * ms;
            const float root = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)b.v[i])[at], 0) * vs;
            v[e] = root * root;
        } else {
            m[e] = ((const float *)b.m[i])[at];
            v[e] = ((const float *)b.v[i])[at];
        }
        m[e] = p.b1 * m[e] + p.omb1 * g;
        v[e] = p.b2 * v[e] + p.omb2 * g * g;
        var = __builtin_fmaf(-b.decay[i], var, var) - step_of(m[e], v[e], p);
        b.var[i][at] = var;
        if (b.shadow[i]) b.shadow[i][at] = (uint16_t)f32_to_bf16(var);
        if (!BITS8) {
            ((float *)b.m[i])[at] = m[e];
            ((float *)b.v[i])[at] = v[e];
        }
    }
    if (!BITS8) return;
    float root[4], mt = 0.f, vt = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        root[e] = __builtin_sqrtf(v[e]);
        mt = __uint_as_float(max(__float_as_uint(mt), __float_as_uint(m[e]) & 0x7fffffffu));
        vt = __uint_as_float(max(__float_as_uint(vt), __float_as_uint(root[e]) & 0x7fffffffu));
    }
    mt = wave_max_bits(mt);
    vt = wave_max_bits(vt);
    const float mi = mt < kNothing ? 0.f : kTop / mt, vi = vt < kNothing ? 0.f : kTop / vt;
    if (lane == 0) {
        b.m_scale[i][blk] = mt < kNothing ? 0.f : mt < INFINITY ? mt / kTop : NAN;
        b.v_scale[i][blk] = vt < kNothing ? 0.f : vt < INFINITY ? vt / kTop : NAN;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t at = blk * 256 + lane + 64 * e;
        if (at >= n) continue;
        const float x = fminf(fmaxf(m[e] * mi, -kTop), kTop);
        const float r = root[e] > 0.f && vi > 0.f ? fminf(fmaxf(root[e] * vi, kLeast), kTop) : 0.f;
        const int two = __builtin_amdgcn_cvt_pk_fp8_f32(x, r, 0, false);
        ((uint8_t *)b.m[i])[at] = (uint8_t)(two & 0xff);
        ((uint8_t *)b.v[i])[at] = (uint8_t)(two >> 8 & 0xff);
    }
}

hipError_t launch_adamw(bool bits8, const AdamwBatch &b, const AdamwParams &p, hipStream_t st) {
    const int64_t blocks = (b.blk_start[b.count] + 3) / 4;
    if (bits8) hipLaunchKernelGGL(adamw_kernel<true>, grid_2d(blocks), dim3(256), 0, st, b, p);
    else hipLaunchKernelGGL(adamw_kernel<false>, grid_2d(blocks), dim3(256), 0, st, b, p);
    return hipGetLastError();
}

}  // namespace tfk

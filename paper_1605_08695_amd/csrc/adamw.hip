// AdamW over many variables in one launch per batch of them, moments in fp32 or in 8 bits.
//
//   m <- b1 m + (1 - b1) g          v <- b2 v + (1 - b2) g^2
//   var <- var - lr wd var - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
// In 8 bits a moment is an e4m3 value (four significant bits, 18 powers of two) times its block's scale, one fp32
// number for each 256 values of a variable: scale = largest / 448, so that the largest is e4m3's largest.  The
// second moment is kept as its square root, which halves its range in powers of two, and never becomes 0 where it
// was not: its smallest value is e4m3's smallest, 2^-9 of 448, so that there a rounded moment makes a step smaller.
// Elsewhere it is rounded either way, by up to 2^-4 of itself, and a change of less than half a code is rounded off again
// in each step: a root r stays where it is relative to its block's largest until one step moves it by 2^-4, that is until
// g^2 > (1 + (2^-3 + 2^-8) / (1 - b2)) r^2: it may be too small by 11 at b2 = 0.999, by 3.7 at 0.99, by 1.5 at 0.9 (and
// too large by any factor), a first moment by 1 + 2^-4 / (1 - b1).  The step itself is made with the moments before they
// are rounded.
//
// One pass, bound by HBM: 277 million values in 9 variables with bf16 copies, in 8 bits 842 us (5.9 TB/s); 24 million in 190
// variables, in fp32 134 us (5.4 TB/s); two of 0.8 million in all 5.8 us, which the caches hold.
#include "common.h"
#include "kernels.h"
#include "rowvec.h"

#pragma clang fp contract(off)

namespace tfk {

constexpr float kTop = 448.f, kLeast = 0x1p-9f, kNothing = 0x1p-100f;

// The largest magnitude of a wave's values, by whole numbers: NaN is the largest of all.
template <int CTRL>
__device__ __forceinline__ uint32_t lane_swap(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ float wave_top(const float *x) {
    uint32_t b = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) b = max(b, __float_as_uint(x[e]) & 0x7fffffffu);
    b = max(b, lane_swap<0xb1>(b));                       // neighbours, pairs, mirrored eights and sixteens
    b = max(b, lane_swap<0x4e>(b));
    b = max(b, lane_swap<0x141>(b));
    b = max(b, lane_swap<0x140>(b));
    const uint32_t lo = max((uint32_t)__builtin_amdgcn_readlane((int)b, 0), (uint32_t)__builtin_amdgcn_readlane((int)b, 16));
    const uint32_t hi = max((uint32_t)__builtin_amdgcn_readlane((int)b, 32), (uint32_t)__builtin_amdgcn_readlane((int)b, 48));
    return __uint_as_float(max(lo, hi));
}

// One value's step.  The moments are rounded operation by operation, as they are written: an e4m3 value then does not
// depend on how a compiler joins a product and a sum.
__device__ __forceinline__ void step_of(float &var, float g, float &m, float &v, float &root, float decay, const AdamwParams &p) {
    m = p.b1 * m + p.omb1 * g;
    v = p.b2 * v + p.omb2 * g * g;
    root = __builtin_sqrtf(v);
    const float den = __builtin_fmaf(root, p.rrc2, p.eps);
    var = __builtin_fmaf(-decay, var, var) - p.lr * m * __builtin_amdgcn_rcpf(den);
}

// The factor of a block whose largest magnitude is top, and what its values are multiplied by: by the reciprocals, as
// elementary tensor operations divide by one number, so that values next to a border between two codes go to the same
// side there and here (each product is within an ulp of the quotient, 2^-20 of a code's step).
__device__ __forceinline__ float factor(float top, float &inv) {
    const bool none = top < kNothing;
    inv = none ? 0.f : 1.f / top * kTop;
    return none ? 0.f : top < INFINITY ? top * (1.f / kTop) : NAN;
}
__device__ __forceinline__ float code_m(float m, float inv) { return __builtin_amdgcn_fmed3f(m * inv, -kTop, kTop); }
__device__ __forceinline__ float code_v(float root, float inv) {
    return root > 0.f && inv > 0.f ? __builtin_amdgcn_fmed3f(root * inv, kLeast, kTop) : 0.f;
}

template <bool AWAY>
__device__ __forceinline__ f32x4_t get4(const float *p) {
    return AWAY ? RowVec<float, 4>::load_last(p) : RowVec<float, 4>::load(p);
}
template <bool AWAY>
__device__ __forceinline__ void put4(float *p, const float *v) {
    if (AWAY) RowVec<float, 4>::store_away(p, v);
    else RowVec<float, 4>::store(p, v);
}
typedef uint32_t u32_a1_t __attribute__((aligned(1)));

// One wave has one block of 256 values, four neighbouring ones a lane.  AWAY: past the caches, which the whole is too
// much for.
template <bool BITS8, bool AWAY>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwBatch b, AdamwParams p) {
    const int64_t blk0 = (blockIdx.x + (int64_t)blockIdx.y * gridDim.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (blk0 >= b.blk_start[b.count]) return;
    int i = 0;
    for (int half = 32; half > 0; half >>= 1)             // the last variable that begins at or before blk0
        if (i + half < b.count && blk0 >= b.blk_start[i + half]) i += half;
    const int64_t blk = blk0 - b.blk_start[i];
    const int64_t at = blk * 256 + 4 * lane;
    const int there = (int)min((int64_t)4, max((int64_t)0, b.n[i] - at));      // of the lane's four
    const bool whole = b.n[i] - blk * 256 >= 256;
    const float decay = b.decay[i];
    float *const pv = b.var[i] + at;
    const float *const pg = b.grad[i] + at;
    uint16_t *const ps = b.shadow[i] ? b.shadow[i] + at : nullptr;
    float var[4], g[4], m[4], v[4], root[4];
    float ms = 0.f, vs = 0.f;
    if (BITS8) {
        ms = b.m_scale[i][blk];
        vs = b.v_scale[i][blk];
    }
    if (whole) {
        RowVec<float, 4>::unpack(get4<AWAY>(pv), var);
        RowVec<float, 4>::unpack(get4<AWAY>(pg), g);
        if (BITS8) {
            const uint32_t cm = *reinterpret_cast<const u32_a1_t *>((const uint8_t *)b.m[i] + at);
            const uint32_t cv = *reinterpret_cast<const u32_a1_t *>((const uint8_t *)b.v[i] + at);
            m[0] = __builtin_amdgcn_cvt_f32_fp8(cm, 0), m[1] = __builtin_amdgcn_cvt_f32_fp8(cm, 1);
            m[2] = __builtin_amdgcn_cvt_f32_fp8(cm, 2), m[3] = __builtin_amdgcn_cvt_f32_fp8(cm, 3);
            v[0] = __builtin_amdgcn_cvt_f32_fp8(cv, 0), v[1] = __builtin_amdgcn_cvt_f32_fp8(cv, 1);
            v[2] = __builtin_amdgcn_cvt_f32_fp8(cv, 2), v[3] = __builtin_amdgcn_cvt_f32_fp8(cv, 3);
        } else {
            RowVec<float, 4>::unpack(get4<AWAY>((const float *)b.m[i] + at), m);
            RowVec<float, 4>::unpack(get4<AWAY>((const float *)b.v[i] + at), v);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            var[e] = g[e] = m[e] = v[e] = 0.f;
            if (e >= there) continue;
            var[e] = pv[e];
            g[e] = pg[e];
            if (BITS8) {
                m[e] = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)b.m[i])[at + e], 0);
                v[e] = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)b.v[i])[at + e], 0);
            } else {
                m[e] = ((const float *)b.m[i])[at + e];
                v[e] = ((const float *)b.v[i])[at + e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (BITS8) {
            m[e] *= ms;
            v[e] *= vs;
            v[e] *= v[e];
        }
        step_of(var[e], g[e], m[e], v[e], root[e], decay, p);
        if (!whole && e >= there) m[e] = root[e] = 0.f;     // beyond the variable, whatever its block's factors are
    }
    uint32_t cm = 0, cv = 0;
    if (BITS8) {
        float mi, vi;
        const float fm = factor(wave_top(m), mi), fv = factor(wave_top(root), vi);
        if (lane == 0) {
            b.m_scale[i][blk] = fm;
            b.v_scale[i][blk] = fv;
        }
        cm = __builtin_amdgcn_cvt_pk_fp8_f32(code_m(m[0], mi), code_m(m[1], mi), 0, false);
        cm = __builtin_amdgcn_cvt_pk_fp8_f32(code_m(m[2], mi), code_m(m[3], mi), cm, true);
        cv = __builtin_amdgcn_cvt_pk_fp8_f32(code_v(root[0], vi), code_v(root[1], vi), 0, false);
        cv = __builtin_amdgcn_cvt_pk_fp8_f32(code_v(root[2], vi), code_v(root[3], vi), cv, true);
    }
    if (whole) {
        put4<AWAY>(pv, var);
        if (ps) RowVec<bf16_t, 4>::store(ps, var);
        if (BITS8) {
            *reinterpret_cast<u32_a1_t *>((uint8_t *)b.m[i] + at) = cm;
            *reinterpret_cast<u32_a1_t *>((uint8_t *)b.v[i] + at) = cv;
        } else {
            put4<AWAY>((float *)b.m[i] + at, m);
            put4<AWAY>((float *)b.v[i] + at, v);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (e >= there) break;
        pv[e] = var[e];
        if (ps) ps[e] = (uint16_t)f32_to_bf16(var[e]);
        if (BITS8) {
            ((uint8_t *)b.m[i])[at + e] = (uint8_t)(cm >> 8 * e);
            ((uint8_t *)b.v[i])[at + e] = (uint8_t)(cv >> 8 * e);
        } else {
            ((float *)b.m[i])[at + e] = m[e];
            ((float *)b.v[i])[at + e] = v[e];
        }
    }
}

hipError_t launch_adamw(bool bits8, const AdamwBatch &b, const AdamwParams &p, bool away, hipStream_t st) {
    const dim3 grid = grid_2d((b.blk_start[b.count] + 3) / 4);
    if (bits8 && away) hipLaunchKernelGGL((adamw_kernel<true, true>), grid, dim3(256), 0, st, b, p);
    else if (bits8) hipLaunchKernelGGL((adamw_kernel<true, false>), grid, dim3(256), 0, st, b, p);
    else if (away) hipLaunchKernelGGL((adamw_kernel<false, true>), grid, dim3(256), 0, st, b, p);
    else hipLaunchKernelGGL((adamw_kernel<false, false>), grid, dim3(256), 0, st, b, p);
    return hipGetLastError();
}

}  // namespace tfk

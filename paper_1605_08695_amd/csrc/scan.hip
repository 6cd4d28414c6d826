// Gated linear recurrence: forward and backward over whole sequences, and one token of many sequences.
//
// With x, a, b the columns of z + bias (b only with an output gate), f = 1 / (1 + e^-a), o = 1 / (1 + e^-b):
//   h_t = f_t h_(t-1) + (1 - f_t) x_t          y_t = h_t, or o_t h_t
//   g_t = o_t dy_t + f_(t+1) g_(t+1)           (the last one: + dh_last)
//   dx = (1 - f) g     da = f (1 - f) (h_(t-1) - x) g     db = o (1 - o) dy h     dh0 = f_1 g_1
// Of a gate's two shares f and 1 - f the smaller is formed, e / (1 + e) with e = e^-|a|, and kept with a's sign: s >= 0
// is 1 - f, s < 0 is -f.  A state moves from where it is by s (x - h), or from x by -f (x - h): one that forgets a
// part in a million a token (of 1 - f, fp32 holds four bits beside f) keeps its steady value and its time constant,
// and one that is forgotten leaves nothing behind.  A span of tokens maps h to S + P h with S its states begun at 0
// and P = prod f, kept as 1 - P or P, whichever is smaller, in the same way.  Backwards, a span maps what comes from
// behind, c, to R + P c.
//
// A workgroup has a strip of channels of one sequence, each wave a run of kSteps tokens of it in registers; the
// waves' spans are joined through LDS, and the workgroup goes on to the next kWaves * kSteps tokens with the
// state they leave.  Bound by HBM: z is read once and y written once; the backward pass reads z and dy and
// writes dz, with the states of each kScanBlock-th token from the forward pass.
#include "common.h"
#include "kernels.h"

#pragma clang fp contract(off)

namespace tfk {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kSteps = 16;                         // tokens a wave has in registers
constexpr int kWaves = kScanBlock / kSteps;        // waves of a workgroup

// The smaller share of a gate, with the sign of its argument.
__device__ __forceinline__ float gate(float a) {
    const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(a));
    return __builtin_copysignf(e * __builtin_amdgcn_rcpf(1.f + e), a);
}
// Whether the share is f (the sign alone tells: -0 is a gate that keeps nothing).
__device__ __forceinline__ bool shut(float s) { return __float_as_int(s) < 0; }
__device__ __forceinline__ float keeps(float s) { return shut(s) ? -s : 1.f - s; }          // f
__device__ __forceinline__ float takes(float s) { return shut(s) ? 1.f + s : s; }           // 1 - f
__device__ __forceinline__ float slope(float s) { return __builtin_fabsf(s) * (1.f - __builtin_fabsf(s)); }

// f h + (1 - f) x
__device__ __forceinline__ float move(float h, float s, float x) { return __builtin_fmaf(s, x - h, shut(s) ? x : h); }
// f g
__device__ __forceinline__ float kept(float g, float s) { return __builtin_fmaf(-s, g, shut(s) ? 0.f : g); }
// S + P h
__device__ __forceinline__ float join(float h, float s, float S) { return (shut(s) ? 0.f : h) + __builtin_fmaf(-s, h, S); }
// The smaller of 1 - P and P of a span, from both.
__device__ __forceinline__ float span(float Q, float P) { return Q < 0.5f ? Q : -P; }

__device__ __forceinline__ int span_of(const int32_t *lengths, int64_t b, int t) {
    return lengths == nullptr ? t : min(max(lengths[b], 0), t);
}

template <typename T, bool OUT>
__global__ __launch_bounds__(64 * kWaves) void scan_fwd_kernel(ScanArgs a) {
    __shared__ float2 spans[2][kWaves][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int strips = (a.d + 63) / 64;
    const int64_t job = blockIdx.x + (int64_t)blockIdx.y * gridDim.x, b = job / strips;
    if (b >= a.b) return;
    const int c = (int)(job - b * strips) * 64 + lane;
    const bool live = c < a.d;
    const int cc = live ? c : a.d - 1;
    const int len = span_of(a.lengths, b, a.t);
    const float bx = a.bias ? a.bias[cc] : 0.f, bf = a.bias ? a.bias[a.d + cc] : 0.f;
    const float bo = OUT && a.bias ? a.bias[2 * a.d + cc] : 0.f;
    const T *const z = (const T *)a.z + b * a.z_bs + cc;
    T *const y = (T *)a.y + b * a.y_bs + cc;
    const int blocks = (a.t + kScanBlock - 1) / kScanBlock;
    float H = a.h0 ? a.h0[b * a.d + cc] : 0.f;
    for (int blk = 0; blk < blocks; ++blk) {
        const int t0 = blk * kScanBlock + w * kSteps;
        if (blk * kScanBlock >= len) {             // padding from here on
            for (int i = 0; i < kSteps; ++i)
                if (live && t0 + i < a.t) Elem<T>::store(y + (t0 + i) * a.y_ts, 0.f);
            continue;
        }
        float s[kSteps], x[kSteps], o[OUT ? kSteps : 1];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = t0 + i < len;
            const T *const p = z + (in ? t0 + i : 0) * a.z_ts;
            x[i] = Elem<T>::load(p) + bx;
            s[i] = gate(Elem<T>::load(p + a.d) + bf);
            if (OUT) o[i] = keeps(gate(Elem<T>::load(p + 2 * a.d) + bo));
            if (!in) s[i] = x[i] = 0.f;            // a state stays as it is
        }
        float S = 0.f, Q = 0.f, P = 1.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            S = move(S, s[i], x[i]);
            Q = move(Q, s[i], 1.f);
            P = kept(P, s[i]);
        }
        spans[blk & 1][w][lane] = make_float2(S, span(Q, P));
        __syncthreads();
        float h = H;
        for (int v = 0; v < kWaves; ++v) {
            if (v == w) h = H;
            const float2 m = spans[blk & 1][v][lane];
            H = join(H, m.y, m.x);
        }
        if (a.states && w == 0 && live) a.states[((int64_t)b * blocks + blk) * a.d + c] = h;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            h = move(h, s[i], x[i]);
            if (live && t0 + i < a.t) Elem<T>::store(y + (t0 + i) * a.y_ts, t0 + i < len ? (OUT ? o[i] * h : h) : 0.f);
        }
    }
    if (a.h_last && w == 0 && live) a.h_last[b * a.d + c] = H;
}

template <typename T, bool OUT>
__global__ __launch_bounds__(64 * kWaves) void scan_bwd_kernel(ScanBwdArgs a) {
    __shared__ float spans[2][kWaves][3][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int strips = (a.d + 63) / 64;
    const int64_t job = blockIdx.x + (int64_t)blockIdx.y * gridDim.x, b = job / strips;
    if (b >= a.b) return;
    const int c = (int)(job - b * strips) * 64 + lane;
    const bool live = c < a.d;
    const int cc = live ? c : a.d - 1;
    const int len = span_of(a.lengths, b, a.t);
    const float bx = a.bias ? a.bias[cc] : 0.f, bf = a.bias ? a.bias[a.d + cc] : 0.f;
    const float bo = OUT && a.bias ? a.bias[2 * a.d + cc] : 0.f;
    const T *const z = (const T *)a.z + b * a.z_bs + cc;
    const T *const dy = (const T *)a.dy + b * a.dy_bs + cc;
    T *const dz = (T *)a.dz + b * a.dz_bs + cc;
    const int blocks = (a.t + kScanBlock - 1) / kScanBlock;
    float C = a.dh_last ? a.dh_last[b * a.d + cc] : 0.f;     // what comes from behind
    for (int blk = blocks - 1; blk >= 0; --blk) {
        const int t0 = blk * kScanBlock + w * kSteps;
        if (blk * kScanBlock >= len) {
            for (int i = 0; i < kSteps; ++i)
                if (live && t0 + i < a.t)
                    for (int k = 0; k < (OUT ? 3 : 2); ++k) Elem<T>::store(dz + (t0 + i) * a.dz_ts + k * a.d, 0.f);
            continue;
        }
        float s[kSteps], x[kSteps], up[kSteps], so[OUT ? kSteps : 1], h1[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = t0 + i < len;
            const int at = in ? t0 + i : 0;
            const T *const p = z + at * a.z_ts;
            x[i] = Elem<T>::load(p) + bx;
            s[i] = gate(Elem<T>::load(p + a.d) + bf);
            up[i] = Elem<T>::load(dy + at * a.dy_ts);
            if (OUT) so[i] = gate(Elem<T>::load(p + 2 * a.d) + bo);
            if (!in) s[i] = x[i] = up[i] = 0.f;
        }
        float S = 0.f, Q = 0.f, P = 1.f, R = 0.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            S = move(S, s[i], x[i]);
            Q = move(Q, s[i], 1.f);
            P = kept(P, s[i]);
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) R = kept(R + (OUT ? keeps(so[i]) * up[i] : up[i]), s[i]);
        float(*const sp)[3][64] = spans[blk & 1];
        sp[w][0][lane] = S;
        sp[w][1][lane] = span(Q, P);
        sp[w][2][lane] = R;
        __syncthreads();
        float h = a.states[((int64_t)b * blocks + blk) * a.d + cc], cin = C;
        for (int v = 0; v < w; ++v) h = join(h, sp[v][1][lane], sp[v][0][lane]);
        for (int v = kWaves - 1; v >= 0; --v) {
            if (v == w) cin = C;
            C = join(C, sp[v][1][lane], sp[v][2][lane]);
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            h1[i] = h;
            h = move(h, s[i], x[i]);
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            const float g = cin + (OUT ? keeps(so[i]) * up[i] : up[i]);
            cin = kept(g, s[i]);
            if (live && t0 + i < a.t) {
                const bool in = t0 + i < len;
                T *const p = dz + (t0 + i) * a.dz_ts;
                Elem<T>::store(p, in ? takes(s[i]) * g : 0.f);
                Elem<T>::store(p + a.d, in ? (h1[i] - x[i]) * (slope(s[i]) * g) : 0.f);
                if (OUT) Elem<T>::store(p + 2 * a.d, in ? slope(so[i]) * up[i] * move(h1[i], s[i], x[i]) : 0.f);
            }
        }
    }
    if (a.dh0 && w == 0 && live) a.dh0[b * a.d + c] = C;
}

// One token of each row: the row's state, in its slot, moves on.  A row whose slot is none gets zeros.
template <typename T, bool OUT>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanStepArgs a) {
    const int c = (int)blockIdx.x * 256 + threadIdx.x;
    const int64_t r = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
    if (r >= a.n || c >= a.d) return;
    T *const y = (T *)a.y + r * a.y_ld + c;
    const int64_t slot = a.slots ? (int64_t)a.slots[r] : r;
    if (slot < 0 || slot >= a.nslots) {
        Elem<T>::store(y, 0.f);
        return;
    }
    const T *const z = (const T *)a.z + r * a.z_ld + c;
    float *const st = a.state + slot * a.d + c;
    const float s = gate(Elem<T>::load(z + a.d) + (a.bias ? a.bias[a.d + c] : 0.f));
    const float h = move(*st, s, Elem<T>::load(z) + (a.bias ? a.bias[c] : 0.f));
    *st = h;
    float o = 1.f;
    if (OUT) o = keeps(gate(Elem<T>::load(z + 2 * a.d) + (a.bias ? a.bias[2 * a.d + c] : 0.f)));
    Elem<T>::store(y, OUT ? o * h : h);
}

#define SCAN_LAUNCH(kernel, grid, threads, a)                                                               \
    do {                                                                                                    \
        if (dt == 0 && gates == 2) hipLaunchKernelGGL((kernel<float, false>), grid, dim3(threads), 0, st, a); \
        if (dt == 0 && gates == 3) hipLaunchKernelGGL((kernel<float, true>), grid, dim3(threads), 0, st, a);  \
        if (dt == 1 && gates == 2) hipLaunchKernelGGL((kernel<bf16_t, false>), grid, dim3(threads), 0, st, a); \
        if (dt == 1 && gates == 3) hipLaunchKernelGGL((kernel<bf16_t, true>), grid, dim3(threads), 0, st, a);  \
    } while (0)

size_t scan_ws_bytes(bool bwd, int64_t b, int64_t t, int d) { return 0; }

hipError_t launch_scan_fwd(int dt, int gates, const ScanArgs &a, void *ws, hipStream_t st) {
    SCAN_LAUNCH(scan_fwd_kernel, grid_2d(a.b * ((a.d + 63) / 64)), 64 * kWaves, a);
    return hipGetLastError();
}

hipError_t launch_scan_bwd(int dt, int gates, const ScanBwdArgs &a, void *ws, hipStream_t st) {
    SCAN_LAUNCH(scan_bwd_kernel, grid_2d(a.b * ((a.d + 63) / 64)), 64 * kWaves, a);
    return hipGetLastError();
}

hipError_t launch_scan_step(int dt, int gates, const ScanStepArgs &a, hipStream_t st) {
    const unsigned gy = (unsigned)std::min<int64_t>(a.n, 32768);
    SCAN_LAUNCH(scan_step_kernel, dim3((a.d + 255) / 256, gy, (unsigned)((a.n + gy - 1) / gy)), 256, a);
    return hipGetLastError();
}

}  // namespace tfk

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
// A workgroup has a strip of 64 channels of one sequence and takes it in blocks of four runs of 32 tokens (of 8, where the
// plan below says so), each wave one run in registers (with two bf16 channels a lane each half wave half of it); the
// waves' spans are joined through LDS, and the workgroup goes on to the next block with the state they leave.  Where
// there are too few strips for the chip, the time axis is cut into segments: a first launch reads all segments but the
// last for what each makes of the state before it (x and the gate; backwards the gate and dy), and in the second each
// workgroup joins those of the segments before its own.  Nothing waits for another workgroup, and sums go the same way
// each time.
//
// Bound by HBM and, with two bf16 channels a lane, nearly as much by the vector unit (a gate is an exponential and a
// reciprocal; with the output gate 46 vector instructions a channel and token forwards, 23 for a segment, 72 backwards, 35 for
// a segment): z is read once and y written once; the backward pass reads z and dy and writes dz, with the states of each
// kScanBlock-th token from the forward pass.  Measured, in bf16 with the output gate at 65536 x 768: segments 50 us, forward
// 97 us (4.2 TB/s, vector unit 76 % busy), segments backwards 78 us, backward 177 us (4.0 TB/s, 63 %).
//
// Tried and slower: the next block's loads before a block is joined (spills, or half the waves); 16 waves of short runs or
// 8 waves of runs of 16 tokens (5 to 30 %); blocks of the time in turn, so that the second launch finds what the first read
// in the caches (no gain).  The backward kernel has 124 registers of 256: three waves a SIMD in its launch bounds spill.
#include <type_traits>

#include "common.h"
#include "kernels.h"

#pragma clang fp contract(off)

namespace tfk {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int kWaves = 4;                          // waves of a workgroup
constexpr int kRun = 32, kShort = 8;               // tokens of a wave's run, or of its half waves' two
constexpr int kStrip = 64;                         // channels of a workgroup
constexpr int kSegments = 64;                      // the most a sequence is cut into

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

// The same number, as one that nothing computed from it before is known for: each pass over a run's gates then looks at
// their signs anew, where the compiler else keeps them all, a pair of scalar registers each, and runs out of those.
__device__ __forceinline__ float fresh(float s) {
    asm volatile("" : "+v"(s));
    return s;
}

// The nearest finite number: what an infinity may be multiplied by a share as, where it stays as a summand (its difference
// from a finite number, or from itself, would be NaN).  Finite results are the same bits with and without it.
__device__ __forceinline__ float finite(float x) { return __builtin_amdgcn_fmed3f(x, -__FLT_MAX__, __FLT_MAX__); }

// f h + (1 - f) x: from the one with the larger share towards the other
__device__ __forceinline__ float move(float h, float s, float x) {
    const float most = shut(s) ? x : h, least = shut(s) ? h : x;
    return __builtin_fmaf(__builtin_fabsf(s), least - finite(most), most);
}
// f g
__device__ __forceinline__ float kept(float g, float s) {
    return __builtin_fmaf(-s, shut(s) ? g : finite(g), shut(s) ? 0.f : g);
}
// The same of a product of gates, which is finite: P f, and 1 - P with what 1 - f adds to it.
__device__ __forceinline__ float kept_of(float P, float s) { return __builtin_fmaf(-s, P, shut(s) ? 0.f : P); }
__device__ __forceinline__ float gone_of(float Q, float s) { return __builtin_fmaf(s, 1.f - Q, shut(s) ? 1.f : Q); }
// S + P h (an infinite h stays where P is too small for fp32: no gate's f is 0)
__device__ __forceinline__ float join(float h, float s, float S) {
    const float c = finite(h);
    return (shut(s) ? h - c : h) + __builtin_fmaf(-s, c, S);
}
// The smaller of 1 - P and P of a span, from both.
__device__ __forceinline__ float span(float Q, float P) { return Q < 0.5f ? Q : -P; }

__device__ __forceinline__ int span_of(const int32_t *lengths, int64_t b, int t) {
    return lengths == nullptr ? t : min(max(lengths[b], 0), t);
}

// V neighbouring channels of a row of d (V <= d) from channel c on.  The last lanes of a row of an odd number of channels
// read the pair that ends with it.
template <typename T, int V>
struct Chans {
    typedef T raw;
    int at, live;
    __device__ __forceinline__ Chans(int c, int d) : at(min(c, d - 1)), live(c < d ? 1 : 0) {}
    __device__ __forceinline__ static raw load(const T *p) { return *p; }
    __device__ __forceinline__ void unpack(raw r, float *v) const { v[0] = Elem<T>::load(&r); }
};
template <>
struct Chans<bf16_t, 2> {
    typedef uint32_t raw;
    int at, live;
    uint32_t low;                      // where the first channel's two bytes are in a pair
    __device__ __forceinline__ Chans(int c, int d)
        : at(min(c, d - 2)), live(min(max(d - c, 0), 2)), low(c > d - 2 ? 0x03020c0c : 0x01000c0c) {}
    __device__ __forceinline__ static raw load(const bf16_t *p) {
        typedef uint32_t __attribute__((aligned(2))) pair_t;
        return *reinterpret_cast<const pair_t *>(p);
    }
    __device__ __forceinline__ void unpack(raw r, float *v) const {
        v[0] = __uint_as_float(__builtin_amdgcn_perm(r, r, low));
        v[1] = __uint_as_float(r & 0xffff0000u);
    }
};

// The strip, sequence and run of tokens of a lane.  w, segment, b and whole (whether the strip has all its channels)
// are the same for a wave.
template <typename T, int V, int RUN>
struct Lane {
    static constexpr int kRow = 64 / V;                       // lanes of a row of the strip
    static constexpr int kSteps = RUN / V;                      // tokens a lane has in registers
    int sub, w, c, segment;
    int64_t b;
    bool whole;
    Chans<T, V> ch;
    __device__ __forceinline__ Lane(int64_t job, int strips, int segments, int d)
        : sub((threadIdx.x & 63) / kRow), w(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)),
          c((int)(job % strips) * kStrip + (threadIdx.x % kRow) * V), segment((int)(job / strips % segments)),
          b(job / strips / segments), whole((int)(job % strips) * kStrip + kStrip <= d), ch(c, d) {}
};

// Rows of a sequence, read and written through buffer descriptors: an address that the wave's lanes share, in scalar
// registers, and an offset of 32 bits of each lane (rows are at most kScanRowStep elements apart).  A lane whose token or
// channel is not there gives kNowhere, past the descriptor's end: it reads 0 and writes nothing, without a branch.
constexpr uint32_t kNowhere = 0x80000000u;

template <typename T, int V, int RUN>
struct Rows {
    typedef std::remove_const_t<T> E;
    typedef Lane<E, V, RUN> L;
    T *p;
    int64_t ts;
    uint32_t off, off_all, off_half;   // where a lane reads, writes all of its channels, and the first one alone
    __device__ __forceinline__ Rows(T *base, int64_t ts, const L &l)
        : p(base), ts(ts), off((uint32_t)((l.sub * L::kSteps * ts + l.ch.at) * sizeof(T))) {
        off_all = l.ch.live == V ? off : kNowhere;
        off_half = V == 2 && l.ch.live == 1 ? off + (uint32_t)sizeof(T) : kNowhere;
    }
    // Token t of the wave's first run.
    __device__ __forceinline__ T *row(int t) const { return p + t * ts; }
    __device__ __forceinline__ static __amdgpu_buffer_rsrc_t desc(T *r) {
        return __builtin_amdgcn_make_buffer_rsrc((void *)const_cast<E *>(r), 0, 0x7fffffff, 0x00027000);
    }
    // The lane's channels in the columns that begin at r, of the wave's first run's row or the same one of the lane's.
    __device__ __forceinline__ typename Chans<E, V>::raw load(T *r, bool there) const {
        const uint32_t o = there ? off : kNowhere;
        if constexpr (sizeof(E) * V == 4) {
            return __builtin_bit_cast(typename Chans<E, V>::raw, __builtin_amdgcn_raw_buffer_load_b32(desc(r), o, 0, 0));
        } else {
            return (E)__builtin_amdgcn_raw_buffer_load_b16(desc(r), o, 0, 0);
        }
    }
    __device__ __forceinline__ void store(T *r, const float *v, bool there, bool whole) const {
        const uint32_t o = there ? off_all : kNowhere;
        if constexpr (sizeof(E) == 4) {
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[0]), desc(r), o, 0, 0);
        } else if constexpr (V == 2) {
            __builtin_amdgcn_raw_buffer_store_b32(pack_bf16x2(v[0], v[1]), desc(r), o, 0, 0);
            if (!whole) __builtin_amdgcn_raw_buffer_store_b16((short)f32_to_bf16(v[0]), desc(r), there ? off_half : kNowhere, 0, 0);
        } else {
            __builtin_amdgcn_raw_buffer_store_b16((short)f32_to_bf16(v[0]), desc(r), o, 0, 0);
        }
    }
};

// What the runs of a block make of a channel's state: S + P h, s the smaller of 1 - P and P (see above).
struct Span {
    float S, Q, P;
    __device__ __forceinline__ void add(float s, float x) {
        S = move(S, s, x);
        Q = gone_of(Q, s);
        P = kept_of(P, s);
    }
    // This span, then o.
    __device__ __forceinline__ Span then(const Span &o) const {
        return {join(S, span(o.Q, o.P), o.S), Q + o.Q - Q * o.Q, P * o.P};
    }
    __device__ __forceinline__ Span other_half() const {
        return {__shfl_xor(S, 32, 64), __shfl_xor(Q, 32, 64), __shfl_xor(P, 32, 64)};
    }
};

struct ScanSegArgs {
    const void *z;
    int64_t z_bs, z_ts;
    const float *bias;
    const int32_t *lengths;
    const void *dy;
    int64_t dy_bs, dy_ts, b;
    int t, d;
};

// A strip's state (or what comes from behind) at the border of a segment: h0 (dh_last), then the segments between.
template <int V>
__device__ __forceinline__ void join_segments(const float2 *agg, int64_t at, int64_t step, int n, int c, int d, float *H) {
    for (int g = 0; g < n; g += 8) {
        float2 m[8][V];
#pragma unroll
        for (int q = 0; q < 8; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) m[q][e] = agg[at + min(g + q, n - 1) * step + min(c + e, d - 1)];
#pragma unroll
        for (int q = 0; q < 8; ++q)
#pragma unroll
            for (int e = 0; e < V; ++e) H[e] = g + q < n ? join(H[e], m[q][e].y, m[q][e].x) : H[e];
    }
}

// What each segment but the last makes of the state before it (BWD: each but the first of what comes from behind it, where
// OUT says whether there is an output gate),
// to agg[b][segment][channel].  Each wave takes a part of the segment, run by run.
template <typename T, int V, bool OUT, bool BWD, int RUN>
__global__ __launch_bounds__(64 * kWaves) void scan_segments_kernel(ScanSegArgs a, float2 *agg, int segments, int seg_len) {
    typedef Lane<T, V, RUN> L;
    constexpr int kSteps = L::kSteps;
    __shared__ Span spans[kWaves][kStrip];
    const int d = a.d, strips = (d + kStrip - 1) / kStrip;
    const int64_t job = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (job >= a.b * strips * (segments - 1)) return;
    L l(job, strips, segments - 1, d);
    if (BWD) ++l.segment;
    const int len = span_of(a.lengths, l.b, a.t);
    float bx[V], bf[V], bo[V];
    Span m[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = min(l.c + e, d - 1);
        bx[e] = a.bias ? a.bias[c] : 0.f;
        bf[e] = a.bias ? a.bias[d + c] : 0.f;
        bo[e] = OUT && a.bias ? a.bias[2 * d + c] : 0.f;
        m[e] = Span{0.f, 0.f, 1.f};
    }
    const Rows<const T, V, RUN> z((const T *)a.z + l.b * a.z_bs, a.z_ts, l), dy((const T *)a.dy + l.b * a.dy_bs, a.dy_ts, l);
    const int part = l.segment * seg_len + l.w * (seg_len / kWaves);
    const auto run = [&](int tw, auto inside) {
        constexpr bool INSIDE = decltype(inside)::value;
        const int t0 = tw + l.sub * kSteps;
        typename Chans<T, V>::raw rx[kSteps], rf[kSteps], ro[OUT && BWD ? kSteps : 1];
        const T *r = z.row(tw), *ry = BWD ? dy.row(tw) : nullptr;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const bool in = INSIDE || t0 + i < len;
            rx[i] = BWD ? dy.load(ry, in) : z.load(r, in);
            rf[i] = z.load(r + d, in);
            if (OUT && BWD) ro[i] = z.load(r + 2 * d, in);
            r += z.ts;
            if (BWD) ry += dy.ts;
        }
        Span n[V];
#pragma unroll
        for (int e = 0; e < V; ++e) n[e] = Span{0.f, 0.f, 1.f};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int i = BWD ? kSteps - 1 - k : k;
            float x[V], f[V], o[V];
            l.ch.unpack(rx[i], x);
            l.ch.unpack(rf[i], f);
            if (OUT && BWD) l.ch.unpack(ro[i], o);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float s = gate(f[e] + bf[e]), v = BWD ? x[e] : x[e] + bx[e];
                if (OUT && BWD) v *= keeps(gate(o[e] + bo[e]));
                if (!INSIDE && t0 + i >= len) s = v = 0.f;
                if (BWD) n[e].S = kept(n[e].S + v, s);
                else n[e].S = move(n[e].S, s, v);
                n[e].Q = gone_of(n[e].Q, s);
                n[e].P = kept_of(n[e].P, s);
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (V == 2) {
                const Span o = n[e].other_half();
                const bool first = (l.sub == 0) != BWD;
                n[e] = (first ? n[e] : o).then(first ? o : n[e]);
            }
            m[e] = m[e].then(n[e]);
        }
    };
    const int runs = seg_len / kWaves / RUN;
    for (int k = 0; k < runs; ++k) {
        const int tw = part + (BWD ? runs - 1 - k : k) * RUN;
        if (tw + RUN <= len) run(tw, std::true_type{});
        else if (tw < len) run(tw, std::false_type{});
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
        if (V == 1 || l.sub == e) spans[l.w][threadIdx.x % L::kRow * V + e] = m[e];
    __syncthreads();
    if (threadIdx.x >= kStrip) return;
    Span n = spans[BWD ? kWaves - 1 : 0][threadIdx.x];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) n = n.then(spans[BWD ? kWaves - 1 - v : v][threadIdx.x]);
    const int c = (int)(job % strips) * kStrip + threadIdx.x;
    if (c < d) agg[(l.b * segments + l.segment) * d + c] = make_float2(n.S, span(n.Q, n.P));
}

template <typename T, int V, bool OUT, int RUN>
__global__ __launch_bounds__(64 * kWaves, RUN == kShort ? 4 : 3) void scan_fwd_kernel(ScanArgs a, const float2 *agg,
                                                                                        int segments, int seg_len) {
    typedef Lane<T, V, RUN> L;
    constexpr int kSteps = L::kSteps, kBlock = kWaves * RUN;
    __shared__ float2 spans[2][kWaves][kStrip];
    const int d = a.d, strips = (d + kStrip - 1) / kStrip;
    const int64_t job = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (job >= a.b * strips * segments) return;
    const L l(job, strips, segments, d);
    const int len = span_of(a.lengths, l.b, a.t);
    float bx[V], bf[V], bo[V], H[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = min(l.c + e, d - 1);
        bx[e] = a.bias ? a.bias[c] : 0.f;
        bf[e] = a.bias ? a.bias[d + c] : 0.f;
        bo[e] = OUT && a.bias ? a.bias[2 * d + c] : 0.f;
        H[e] = a.h0 ? a.h0[l.b * d + c] : 0.f;
    }
    if (l.segment > 0) join_segments<V>(agg, l.b * segments * d, d, l.segment, l.c, d, H);
    const Rows<const T, V, RUN> z((const T *)a.z + l.b * a.z_bs, a.z_ts, l);
    const Rows<T, V, RUN> y((T *)a.y + l.b * a.y_bs, a.y_ts, l);
    const int blocks = (a.t + kBlock - 1) / kBlock, saved = (a.t + kScanBlock - 1) / kScanBlock;
    const int col = threadIdx.x % L::kRow * V;
    // INSIDE: all of the block's tokens and channels are there
    const auto block = [&](int blk, auto inside) {
        constexpr bool INSIDE = decltype(inside)::value;
        const int tw = blk * kBlock + l.w * RUN, t0 = tw + l.sub * kSteps;
        float s[kSteps][V], x[kSteps][V], o[OUT ? kSteps : 1][V];
        {
            typename Chans<T, V>::raw rx[kSteps], rf[kSteps], ro[OUT ? kSteps : 1];
            const T *r = z.row(tw);
#pragma unroll
            for (int i = 0; i < kSteps; ++i, r += z.ts) {
                const bool in = INSIDE || t0 + i < len;
                rx[i] = z.load(r, in);
                rf[i] = z.load(r + d, in);
                if (OUT) ro[i] = z.load(r + 2 * d, in);
            }
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                l.ch.unpack(rx[i], x[i]);
                l.ch.unpack(rf[i], s[i]);
                if (OUT) l.ch.unpack(ro[i], o[i]);
            }
        }
        Span m[V];
#pragma unroll
        for (int e = 0; e < V; ++e) m[e] = Span{0.f, 0.f, 1.f};
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[i][e] += bx[e];
                s[i][e] = gate(s[i][e] + bf[e]);
                if (OUT) o[i][e] = keeps(gate(o[i][e] + bo[e]));
                if (!INSIDE && t0 + i >= len) s[i][e] = x[i][e] = 0.f;            // a state stays as it is
                m[e].add(s[i][e], x[i][e]);
            }
        float2 half[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (V == 2) {
                const Span other = m[e].other_half();
                half[e] = make_float2(other.S, span(other.Q, other.P));
                m[e] = l.sub == 0 ? m[e].then(other) : other.then(m[e]);
            }
            if (V == 1 || l.sub == e) spans[blk & 1][l.w][col + e] = make_float2(m[e].S, span(m[e].Q, m[e].P));
        }
        __syncthreads();
        float h[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
#pragma unroll
            for (int v = 0; v < kWaves; ++v) {
                if (v == l.w) h[e] = H[e];
                const float2 q = spans[blk & 1][v][col + e];
                H[e] = join(H[e], q.y, q.x);
            }
            if (V == 2) h[e] = l.sub == 1 ? join(h[e], half[e].y, half[e].x) : h[e];
        }
        T *r = y.row(tw);
#pragma unroll
        for (int i = 0; i < kSteps; ++i, r += y.ts) {
            if (i % kScanBlock == 0 && a.states && (kSteps >= kScanBlock || t0 % kScanBlock == 0) && (INSIDE || t0 + i < a.t)) {
                float *const st = a.states + (l.b * saved + (t0 + i) / kScanBlock) * d + l.c;
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (INSIDE || l.c + e < d) st[e] = h[e];
            }
            float out[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                h[e] = move(h[e], fresh(s[i][e]), x[i][e]);
                out[e] = OUT ? o[i][e] * h[e] : h[e];
                if (!INSIDE && t0 + i >= len) out[e] = 0.f;
            }
            y.store(r, out, INSIDE || t0 + i < a.t, INSIDE || l.whole);
        }
    };
    for (int blk = l.segment * (seg_len / kBlock); blk < min(blocks, (l.segment + 1) * (seg_len / kBlock)); ++blk) {
        if (l.whole && (blk + 1) * kBlock <= len) {
            block(blk, std::true_type{});
        } else if (blk * kBlock < len) {
            block(blk, std::false_type{});
        } else {                                   // padding from here on
            const int tw = blk * kBlock + l.w * RUN, t0 = tw + l.sub * kSteps;
            const float none[2] = {0.f, 0.f};
            for (int i = 0; i < kSteps; ++i)
                y.store(y.row(tw + i), none, t0 + i < a.t, l.whole);
        }
    }
    if (a.h_last && l.segment == segments - 1 && threadIdx.x < L::kRow)
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (l.c + e < d) a.h_last[l.b * d + l.c + e] = H[e];
}

template <typename T, int V, bool OUT, int RUN>
__global__ __launch_bounds__(64 * kWaves, RUN == kShort ? 4 : 2) void scan_bwd_kernel(ScanBwdArgs a, const float2 *agg,
                                                                                        int segments, int seg_len) {
    typedef Lane<T, V, RUN> L;
    // DIRECT: a state was saved for each lane's first token; else the runs since the last one are joined
    constexpr int kSteps = L::kSteps, kBlock = kWaves * RUN;
    constexpr bool DIRECT = kSteps >= kScanBlock;
    constexpr int kSince = DIRECT ? 1 : kScanBlock / RUN;          // waves since a saved state
    __shared__ float2 spans[2][kWaves][kStrip];                    // backwards: R, and the smaller of 1 - P and P
    __shared__ float fronts[2][DIRECT ? 1 : kWaves][kStrip];       // forwards: S
    const int d = a.d, strips = (d + kStrip - 1) / kStrip;
    const int64_t job = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (job >= a.b * strips * segments) return;
    const L l(job, strips, segments, d);
    const int len = span_of(a.lengths, l.b, a.t);
    float bx[V], bf[V], bo[V], C[V];                             // C: what comes from behind
#pragma unroll
    for (int e = 0; e < V; ++e) {
        const int c = min(l.c + e, d - 1);
        bx[e] = a.bias ? a.bias[c] : 0.f;
        bf[e] = a.bias ? a.bias[d + c] : 0.f;
        bo[e] = OUT && a.bias ? a.bias[2 * d + c] : 0.f;
        C[e] = a.dh_last ? a.dh_last[l.b * d + c] : 0.f;
    }
    if (l.segment < segments - 1)
        join_segments<V>(agg, (l.b * segments + segments - 1) * d, -(int64_t)d, segments - 1 - l.segment, l.c, d, C);
    const Rows<const T, V, RUN> z((const T *)a.z + l.b * a.z_bs, a.z_ts, l), dy((const T *)a.dy + l.b * a.dy_bs, a.dy_ts, l);
    const Rows<T, V, RUN> dz((T *)a.dz + l.b * a.dz_bs, a.dz_ts, l);
    const int blocks = (a.t + kBlock - 1) / kBlock, saved = (a.t + kScanBlock - 1) / kScanBlock;
    const int col = threadIdx.x % L::kRow * V;
    const auto block = [&](int blk, auto inside) {
        constexpr bool INSIDE = decltype(inside)::value;
        const int tw = blk * kBlock + l.w * RUN, t0 = tw + l.sub * kSteps;
        float s[kSteps][V], x[kSteps][V], up[kSteps][V], o[OUT ? kSteps : 1][V], h[V];
        {
            typename Chans<T, V>::raw rx[kSteps], rf[kSteps], ru[kSteps], ro[OUT ? kSteps : 1];
            const T *r = z.row(tw), *ry = dy.row(tw);
#pragma unroll
            for (int i = 0; i < kSteps; ++i, r += z.ts, ry += dy.ts) {
                const bool in = INSIDE || t0 + i < len;
                rx[i] = z.load(r, in);
                rf[i] = z.load(r + d, in);
                ru[i] = dy.load(ry, in);
                if (OUT) ro[i] = z.load(r + 2 * d, in);
            }
            const int at = min((t0 - (DIRECT ? 0 : (l.w % kSince) * RUN + l.sub * kSteps)) / kScanBlock, saved - 1);
#pragma unroll
            for (int e = 0; e < V; ++e) h[e] = a.states[(l.b * saved + at) * d + min(l.c + e, d - 1)];
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                l.ch.unpack(rx[i], x[i]);
                l.ch.unpack(rf[i], s[i]);
                l.ch.unpack(ru[i], up[i]);
                if (OUT) l.ch.unpack(ro[i], o[i]);
            }
        }
        // Forwards with the states: x becomes h_(t-1) - x, dy becomes what reaches h_t, and the output gate's gradient
        // is done.
        T *r = dz.row(tw);
        const auto forward = [&](int i, float(&out)[V]) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float before = h[e];
                h[e] = move(before, fresh(s[i][e]), x[i][e]);
                x[i][e] = before - x[i][e];
                if (OUT) {
                    const float so = fresh(o[i][e]);
                    out[e] = INSIDE || t0 + i < len ? slope(so) * up[i][e] * h[e] : 0.f;
                    up[i][e] *= keeps(so);
                }
            }
            if (OUT) dz.store(r + 2 * d, out, INSIDE || t0 + i < a.t, INSIDE || l.whole);
            r += dz.ts;
        };
        Span m[V];
        float R[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            m[e] = Span{0.f, 0.f, 1.f};
            R[e] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[i][e] += bx[e];
                s[i][e] = gate(s[i][e] + bf[e]);
                if (OUT) o[i][e] = gate(o[i][e] + bo[e]);
                if (!INSIDE && t0 + i >= len) s[i][e] = x[i][e] = up[i][e] = 0.f;
                if (!DIRECT) m[e].S = move(m[e].S, s[i][e], x[i][e]);
                m[e].Q = gone_of(m[e].Q, s[i][e]);
                m[e].P = kept_of(m[e].P, s[i][e]);
            }
            float out[V];
            if (DIRECT) forward(i, out);
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i)
#pragma unroll
            for (int e = 0; e < V; ++e)
                R[e] = kept(R[e] + (OUT && !DIRECT ? keeps(fresh(o[i][e])) * up[i][e] : up[i][e]), fresh(s[i][e]));
        float half_S[V], half_s[V], half_R[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float back = R[e];
            if (V == 2) {
                const Span other = m[e].other_half();
                half_S[e] = other.S;
                half_s[e] = span(other.Q, other.P);
                half_R[e] = __shfl_xor(R[e], 32, 64);
                // the earlier half is the later one of the way back
                back = l.sub == 0 ? join(half_R[e], span(m[e].Q, m[e].P), R[e]) : join(R[e], half_s[e], half_R[e]);
                m[e] = l.sub == 0 ? m[e].then(other) : other.then(m[e]);
            }
            if (V == 1 || l.sub == e) {
                spans[blk & 1][l.w][col + e] = make_float2(back, span(m[e].Q, m[e].P));
                if (!DIRECT) fronts[blk & 1][l.w][col + e] = m[e].S;
            }
        }
        __syncthreads();
        float c[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
#pragma unroll
            for (int v = kWaves - 1; v >= 0; --v) {
                if (v == l.w) c[e] = C[e];
                const float2 q = spans[blk & 1][v][col + e];
                C[e] = join(C[e], q.y, q.x);
            }
            if (!DIRECT) {
#pragma unroll
                for (int v = 0; v < kWaves; ++v)
                    if (v < l.w && v / kSince == l.w / kSince)
                        h[e] = join(h[e], spans[blk & 1][v][col + e].y, fronts[blk & 1][v][col + e]);
                if (V == 2) h[e] = l.sub == 1 ? join(h[e], half_s[e], half_S[e]) : h[e];
            }
            if (V == 2) c[e] = l.sub == 0 ? join(c[e], half_s[e], half_R[e]) : c[e];
        }
        if (!DIRECT) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                float out[V];
                forward(i, out);
            }
        }
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            r -= dz.ts;
            float dx[V], df[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float g = c[e] + up[i][e], si = fresh(s[i][e]);
                c[e] = kept(g, si);
                const bool in = INSIDE || t0 + i < len;
                dx[e] = in ? takes(si) * g : 0.f;
                df[e] = in ? x[i][e] * (slope(si) * g) : 0.f;
            }
            dz.store(r, dx, INSIDE || t0 + i < a.t, INSIDE || l.whole);
            dz.store(r + d, df, INSIDE || t0 + i < a.t, INSIDE || l.whole);
        }
    };
    const int first = l.segment * (seg_len / kBlock);
    for (int blk = min(blocks, first + seg_len / kBlock) - 1; blk >= first; --blk) {
        if (l.whole && (blk + 1) * kBlock <= len) {
            block(blk, std::true_type{});
        } else if (blk * kBlock < len) {
            block(blk, std::false_type{});
        } else {                                   // padding
            const int tw = blk * kBlock + l.w * RUN, t0 = tw + l.sub * kSteps;
            const float none[2] = {0.f, 0.f};
            for (int i = 0; i < kSteps; ++i)
                for (int k = 0; k < (OUT ? 3 : 2); ++k) dz.store(dz.row(tw + i) + k * d, none, t0 + i < a.t, l.whole);
        }
    }
    if (a.dh0 && l.segment == 0 && threadIdx.x < L::kRow)
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (l.c + e < d) a.dh0[l.b * d + l.c + e] = C[e];
}

// One token of each row: the row's state, in its slot, moves on.  A row whose slot is none gets zeros.  Slots are distinct.
// Bound by two dependent loads (128 rows x 512: 2.7 us).
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

// How the time axis is cut: segments of seg_len tokens, a whole number of blocks.  Measured, forward and backward in bf16 with
// the output gate, replayed as a graph:
//   blocks of four short runs: for up to 32 tokens (128 x 20 x 512: 22 us, 48 by blocks of 128), and for more than 128
//     where blocks of 128 are fewer than 512 (1 x 500 x 512: 25 us, 49; 4 x 200 x 1024: 27, 35; but a single block of 128
//     is better read by one workgroup: 8 x 128 x 1024: 21 us, 27 by short runs)
//   segments: below 512 strips, towards 2048 workgroups (65536 x 768: 377 us, 410 towards 512; 8 x 4096 x 2048 without the
//     output gate, ragged: 309 to 320, 323 to 326; but of full lengths 369, 338); from 512 on one workgroup reads all of a
//     strip (32 x 2048 x 1024: 356 us, 478 in segments)
struct ScanPlan {
    bool fine;
    int segments, seg_len;
};

static ScanPlan scan_plan(int64_t b, int64_t t, int d) {
    const int64_t strips = b * ((d + kStrip - 1) / kStrip);
    const int64_t whole = strips * ((t + kWaves * kRun - 1) / (kWaves * kRun));
    const bool fine = t <= kWaves * kShort || (t > kWaves * kRun && whole < 512);
    const int block = kWaves * (fine ? kShort : kRun);
    const int64_t blocks = std::max<int64_t>((t + block - 1) / block, 1);
    int64_t want = 1;
    if (strips < 512) want = std::min<int64_t>({kSegments, fine ? blocks : blocks / 2, (2048 + strips - 1) / strips});
    const int64_t per = (blocks + std::max<int64_t>(want, 1) - 1) / std::max<int64_t>(want, 1);
    return {fine, (int)((blocks + per - 1) / per), (int)(per * block)};
}

// (Forward and backward are cut alike.)
size_t scan_ws_bytes(int64_t b, int64_t t, int d) {
    const ScanPlan p = scan_plan(b, t, d);
    return p.segments > 1 ? (size_t)b * p.segments * d * sizeof(float2) : 0;
}

template <typename T, int V, bool OUT, int RUN>
static void launch_fwd_run(const ScanArgs &a, float2 *ws, const ScanPlan &p, hipStream_t st) {
    const int64_t strips = a.b * ((a.d + kStrip - 1) / kStrip);
    if (p.segments > 1) {
        const ScanSegArgs g{a.z, a.z_bs, a.z_ts, a.bias, a.lengths, nullptr, 0, 0, a.b, a.t, a.d};
        hipLaunchKernelGGL((scan_segments_kernel<T, V, false, false, RUN>), grid_2d(strips * (p.segments - 1)), dim3(64 * kWaves),
                           0, st, g, ws, p.segments, p.seg_len);
    }
    hipLaunchKernelGGL((scan_fwd_kernel<T, V, OUT, RUN>), grid_2d(strips * p.segments), dim3(64 * kWaves), 0, st, a, ws, p.segments,
                       p.seg_len);
}

template <typename T, int V, bool OUT, int RUN>
static void launch_bwd_run(const ScanBwdArgs &a, float2 *ws, const ScanPlan &p, hipStream_t st) {
    const int64_t strips = a.b * ((a.d + kStrip - 1) / kStrip);
    if (p.segments > 1) {
        const ScanSegArgs g{a.z, a.z_bs, a.z_ts, a.bias, a.lengths, a.dy, a.dy_bs, a.dy_ts, a.b, a.t, a.d};
        hipLaunchKernelGGL((scan_segments_kernel<T, V, OUT, true, RUN>), grid_2d(strips * (p.segments - 1)), dim3(64 * kWaves), 0,
                           st, g, ws, p.segments, p.seg_len);
    }
    hipLaunchKernelGGL((scan_bwd_kernel<T, V, OUT, RUN>), grid_2d(strips * p.segments), dim3(64 * kWaves), 0, st, a, ws, p.segments,
                       p.seg_len);
}

// Two channels a lane in bf16, but for a single channel.
template <typename T, int V, bool OUT>
static void launch_fwd(const ScanArgs &a, float2 *ws, hipStream_t st) {
    const ScanPlan p = scan_plan(a.b, a.t, a.d);
    if (p.fine) launch_fwd_run<T, V, OUT, kShort>(a, ws, p, st);
    else launch_fwd_run<T, V, OUT, kRun>(a, ws, p, st);
}

template <typename T, int V, bool OUT>
static void launch_bwd(const ScanBwdArgs &a, float2 *ws, hipStream_t st) {
    const ScanPlan p = scan_plan(a.b, a.t, a.d);
    if (p.fine) launch_bwd_run<T, V, OUT, kShort>(a, ws, p, st);
    else launch_bwd_run<T, V, OUT, kRun>(a, ws, p, st);
}

#define SCAN_CASES(fn, ...)                                                         \
    do {                                                                            \
        if (dt == 0) {                                                              \
            if (gates == 2) fn<float, 1, false>(__VA_ARGS__);                       \
            else fn<float, 1, true>(__VA_ARGS__);                                   \
        } else if (a.d == 1) {                                                      \
            if (gates == 2) fn<bf16_t, 1, false>(__VA_ARGS__);                      \
            else fn<bf16_t, 1, true>(__VA_ARGS__);                                  \
        } else {                                                                    \
            if (gates == 2) fn<bf16_t, 2, false>(__VA_ARGS__);                      \
            else fn<bf16_t, 2, true>(__VA_ARGS__);                                  \
        }                                                                           \
    } while (0)

hipError_t launch_scan_fwd(int dt, int gates, const ScanArgs &a, void *ws, hipStream_t st) {
    SCAN_CASES(launch_fwd, a, (float2 *)ws, st);
    return hipGetLastError();
}

hipError_t launch_scan_bwd(int dt, int gates, const ScanBwdArgs &a, void *ws, hipStream_t st) {
    SCAN_CASES(launch_bwd, a, (float2 *)ws, st);
    return hipGetLastError();
}

template <typename T, bool OUT>
static void launch_step(const ScanStepArgs &a, hipStream_t st) {
    const unsigned gy = (unsigned)std::min<int64_t>(a.n, 32768);
    hipLaunchKernelGGL((scan_step_kernel<T, OUT>), dim3((a.d + 255) / 256, gy, (unsigned)((a.n + gy - 1) / gy)), dim3(256), 0, st,
                       a);
}

hipError_t launch_scan_step(int dt, int gates, const ScanStepArgs &a, hipStream_t st) {
    if (dt == 0 && gates == 2) launch_step<float, false>(a, st);
    else if (dt == 0) launch_step<float, true>(a, st);
    else if (gates == 2) launch_step<bf16_t, false>(a, st);
    else launch_step<bf16_t, true>(a, st);
    return hipGetLastError();
}

}  // namespace tfk

// 16-byte pieces of rows that start at any element: gfx950 reads and writes 16 bytes at any element
// address (LLVM's unaligned-access-mode, on for HIP), so rows need no alignment of their own.
#pragma once
#include "common.h"

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t u32x4_a2_t __attribute__((aligned(2)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x2_t u32x2_a2_t __attribute__((aligned(2)));
typedef f32x4_t f32x4_a4_t __attribute__((aligned(4)));

// A result of this size or more is stored past the caches: the last of them, 256 MB, could not hold it until
// its reader comes.  (Lookup and the matrix product that reads it, 512 MB of bf16: 334 us through the caches,
// 306 past them; 256 MB 156, 151; 128 MB 75, 78.)
constexpr int64_t kPastCaches = (int64_t)256 << 20;

// V elements of T at p as fp32 and back; V = 1, 4 or 8.  load_last and store_away: past the caches, for
// what is not read again, or is too much for them.
template <typename T, int V>
struct RowVec;

template <typename T>
struct RowVec<T, 1> {
    typedef float raw;
    __device__ static raw load(const T *p) { return Elem<T>::load(p); }
    __device__ static raw load_last(const T *p) { return load(p); }
    __device__ static void unpack(raw r, float *v) { v[0] = r; }
    __device__ static void store(T *p, const float *v) { Elem<T>::store(p, v[0]); }
    __device__ static void store_away(T *p, const float *v) { store(p, v); }
};

template <>
struct RowVec<float, 4> {
    typedef f32x4_t raw;
    __device__ static raw load(const float *p) { return *reinterpret_cast<const f32x4_a4_t *>(p); }
    __device__ static void unpack(raw r, float *v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = r[e];
    }
    __device__ static void store(float *p, const float *v) {
        *reinterpret_cast<f32x4_a4_t *>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
    }
    __device__ static raw load_last(const float *p) { return __builtin_nontemporal_load(reinterpret_cast<const f32x4_a4_t *>(p)); }
    __device__ static void store_away(float *p, const float *v) {
        const f32x4_a4_t r = f32x4_t{v[0], v[1], v[2], v[3]};
        __builtin_nontemporal_store(r, reinterpret_cast<f32x4_a4_t *>(p));
    }
};

template <>
struct RowVec<float, 8> {
    struct raw {
        f32x4_t a, b;
    };
    __device__ static raw load(const float *p) { return {RowVec<float, 4>::load(p), RowVec<float, 4>::load(p + 4)}; }
    __device__ static void unpack(const raw &r, float *v) {
        RowVec<float, 4>::unpack(r.a, v);
        RowVec<float, 4>::unpack(r.b, v + 4);
    }
    __device__ static void store(float *p, const float *v) {
        RowVec<float, 4>::store(p, v);
        RowVec<float, 4>::store(p + 4, v + 4);
    }
    __device__ static void store_away(float *p, const float *v) {
        RowVec<float, 4>::store_away(p, v);
        RowVec<float, 4>::store_away(p + 4, v + 4);
    }
};

template <>
struct RowVec<bf16_t, 4> {
    typedef u32x2_t raw;
    __device__ static raw load(const bf16_t *p) { return *reinterpret_cast<const u32x2_a2_t *>(p); }
    __device__ static void store(bf16_t *p, const float *v) {
        *reinterpret_cast<u32x2_a2_t *>(p) = u32x2_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
};

template <>
struct RowVec<bf16_t, 8> {
    typedef u32x4_t raw;
    __device__ static raw load(const bf16_t *p) { return *reinterpret_cast<const u32x4_a2_t *>(p); }
    __device__ static void unpack(raw r, float *v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = bf16_to_f32(r[e] & 0xffffu);
            v[2 * e + 1] = __uint_as_float(r[e] & 0xffff0000u);
        }
    }
    __device__ static void store(bf16_t *p, const float *v) {
        u32x4_t r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
        *reinterpret_cast<u32x4_a2_t *>(p) = r;
    }
    __device__ static raw load_last(const bf16_t *p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2_t *>(p)); }
    __device__ static void store_away(bf16_t *p, const float *v) {
        u32x4_a2_t r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
        __builtin_nontemporal_store(r, reinterpret_cast<u32x4_a2_t *>(p));
    }
};

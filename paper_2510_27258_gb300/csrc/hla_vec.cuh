// Loads and stores of V consecutive elements (fp32 or bf16) as fp32 values: one 16- or 8-byte
// access where V > 1 (the caller guarantees V-element alignment), else scalar.
#pragma once

#include <string.h>

#include "hla_internal.h"

namespace hla {

template <typename T, int V>
struct VecIo;

template <typename T>
struct VecIo<T, 1> {
    static __device__ __forceinline__ void load(const T *p, float (&v)[1]) { v[0] = to_f32(*p); }
    static __device__ __forceinline__ void store(T *p, const float (&v)[1]) { from_f32(p, v[0]); }
};

template <>
struct VecIo<float, 4> {
    static __device__ __forceinline__ void load(const float *p, float (&v)[4]) {
        const float4 u = *reinterpret_cast<const float4 *>(p);
        v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    }
    static __device__ __forceinline__ void store(float *p, const float (&v)[4]) {
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};

// two bf16 in one word: the low half is the first element
__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

template <>
struct VecIo<__nv_bfloat16, 4> {
    static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float (&v)[4]) {
        const uint2 u = *reinterpret_cast<const uint2 *>(p);
        v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float (&v)[4]) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    }
};

template <>
struct VecIo<__nv_bfloat16, 8> {
    static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float (&v)[8]) {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
        v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
        v[4] = bf16_lo(u.z); v[5] = bf16_hi(u.z); v[6] = bf16_lo(u.w); v[7] = bf16_hi(u.w);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float (&v)[8]) {
        *reinterpret_cast<uint4 *>(p) =
            make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    }
};

// V elements as they are stored (for loads issued well before their use), and as fp32 pairs
template <typename T, int V>
struct Raw {
    T v[V];
};
template <>
struct Raw<float, 4> {
    float4 v;
};
template <>
struct Raw<__nv_bfloat16, 4> {
    uint2 v;
};
template <>
struct Raw<__nv_bfloat16, 8> {
    uint4 v;
};

template <typename T, int V>
__device__ __forceinline__ Raw<T, V> raw_load(const T *p) {
    return *reinterpret_cast<const Raw<T, V> *>(p);
}
template <typename T, int V>
__device__ __forceinline__ Raw<T, V> raw_zero() {
    Raw<T, V> r;
    memset(&r, 0, sizeof(r));
    return r;
}
__device__ __forceinline__ void raw_floats(const Raw<float, 1> &r, float (&f)[1]) { f[0] = r.v[0]; }
__device__ __forceinline__ void raw_floats(const Raw<__nv_bfloat16, 1> &r, float (&f)[1]) { f[0] = to_f32(r.v[0]); }
__device__ __forceinline__ void raw_floats(const Raw<float, 4> &r, float (&f)[4]) {
    f[0] = r.v.x; f[1] = r.v.y; f[2] = r.v.z; f[3] = r.v.w;
}
__device__ __forceinline__ void raw_floats(const Raw<__nv_bfloat16, 4> &r, float (&f)[4]) {
    f[0] = bf16_lo(r.v.x); f[1] = bf16_hi(r.v.x); f[2] = bf16_lo(r.v.y); f[3] = bf16_hi(r.v.y);
}
__device__ __forceinline__ void raw_floats(const Raw<__nv_bfloat16, 8> &r, float (&f)[8]) {
    f[0] = bf16_lo(r.v.x); f[1] = bf16_hi(r.v.x); f[2] = bf16_lo(r.v.y); f[3] = bf16_hi(r.v.y);
    f[4] = bf16_lo(r.v.z); f[5] = bf16_hi(r.v.z); f[6] = bf16_lo(r.v.w); f[7] = bf16_hi(r.v.w);
}

// whether a base pointer and a row stride (elements of `eb` bytes) keep every row aligned to `bytes`
inline bool rows_aligned(const void *p, long long stride, size_t eb, size_t bytes) {
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (static_cast<size_t>(stride) * eb) % bytes == 0;
}

}  // namespace hla

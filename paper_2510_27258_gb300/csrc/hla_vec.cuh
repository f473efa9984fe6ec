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
struct VecIo<float, 2> {
    static __device__ __forceinline__ void load(const float *p, float (&v)[2]) {
        const float2 u = *reinterpret_cast<const float2 *>(p);
        v[0] = u.x; v[1] = u.y;
    }
    static __device__ __forceinline__ void store(float *p, const float (&v)[2]) {
        *reinterpret_cast<float2 *>(p) = make_float2(v[0], v[1]);
    }
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
struct VecIo<__nv_bfloat16, 2> {
    static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float (&v)[2]) {
        const uint32_t u = *reinterpret_cast<const uint32_t *>(p);
        v[0] = bf16_lo(u); v[1] = bf16_hi(u);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float (&v)[2]) {
        *reinterpret_cast<uint32_t *>(p) = bf16_pair(v[0], v[1]);
    }
};

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
struct Raw<float, 2> {
    float2 v;
};
template <>
struct Raw<__nv_bfloat16, 2> {
    uint32_t v;
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

// A ring of rows in flight per thread: slot s of thread t is the Raw at s * blockDim.x + t of a
// shared array, written by the thread's own asynchronous copies (one group a row) and read by it
// alone, so no barrier is needed.  One-element rows are copied through a register.
template <typename T, int V>
__device__ __forceinline__ void ring_copy(Raw<T, V> *slot, const T *src, bool on) {
    if constexpr (sizeof(Raw<T, V>) >= 4) {
        if (on)
            asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(
                             static_cast<uint32_t>(__cvta_generic_to_shared(slot))),
                         "l"(src), "n"((int)sizeof(Raw<T, V>))
                         : "memory");
    } else {
        if (on) *slot = raw_load<T, V>(src);
    }
}
__device__ __forceinline__ void ring_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void ring_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// two fp32 values in a 64-bit register, and the paired operations on them (one issue slot for two)
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ uint64_t pair(uint32_t lo, uint32_t hi) { return pair(__uint_as_float(lo), __uint_as_float(hi)); }
__device__ __forceinline__ void unpair(uint64_t v, float &lo, float &hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint32_t bf16_of(uint64_t v) {
    float lo, hi;
    unpair(v, lo, hi);
    return bf16_pair(lo, hi);
}
__device__ __forceinline__ uint64_t of_bf16(uint32_t u) { return pair(bf16_lo(u), bf16_hi(u)); }

// a row's V elements as (V + 1) / 2 pairs (V = 1: the second half of the pair is zero), and back
__device__ __forceinline__ void to_pairs(const Raw<float, 1> &r, uint64_t (&f)[1]) { f[0] = pair(r.v[0], 0.f); }
__device__ __forceinline__ void to_pairs(const Raw<__nv_bfloat16, 1> &r, uint64_t (&f)[1]) { f[0] = pair(to_f32(r.v[0]), 0.f); }
__device__ __forceinline__ void to_pairs(const Raw<float, 2> &r, uint64_t (&f)[1]) { f[0] = pair(r.v.x, r.v.y); }
__device__ __forceinline__ void to_pairs(const Raw<__nv_bfloat16, 2> &r, uint64_t (&f)[1]) { f[0] = of_bf16(r.v); }
__device__ __forceinline__ void to_pairs(const Raw<float, 4> &r, uint64_t (&f)[2]) {
    f[0] = pair(r.v.x, r.v.y);
    f[1] = pair(r.v.z, r.v.w);
}
__device__ __forceinline__ void to_pairs(const Raw<__nv_bfloat16, 4> &r, uint64_t (&f)[2]) {
    f[0] = of_bf16(r.v.x);
    f[1] = of_bf16(r.v.y);
}
__device__ __forceinline__ void to_pairs(const Raw<__nv_bfloat16, 8> &r, uint64_t (&f)[4]) {
    f[0] = of_bf16(r.v.x);
    f[1] = of_bf16(r.v.y);
    f[2] = of_bf16(r.v.z);
    f[3] = of_bf16(r.v.w);
}
template <typename T, int V>
__device__ __forceinline__ void store_pairs(T *p, const uint64_t (&f)[(V + 1) / 2]) {
    float v[V + 1];
#pragma unroll
    for (int i = 0; i < V; i += 2) unpair(f[i / 2], v[i], v[i + 1]);
    float out[V];
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = v[i];
    VecIo<T, V>::store(p, out);
}

// whether a base pointer and a row stride (elements of `eb` bytes) keep every row aligned to `bytes`
inline bool rows_aligned(const void *p, long long stride, size_t eb, size_t bytes) {
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (static_cast<size_t>(stride) * eb) % bytes == 0;
}

}  // namespace hla

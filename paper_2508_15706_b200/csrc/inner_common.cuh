// Typed vector loads and stores, block sums: shared by the operators of the inner phase (inner.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace {

typedef __nv_bfloat16 bf16;

constexpr unsigned kFullMask = 0xFFFFFFFFu;

template <int BYTES>
struct RawVec;
template <>
struct RawVec<16> { typedef uint4 type; };
template <>
struct RawVec<8> { typedef uint2 type; };
template <>
struct RawVec<4> { typedef unsigned type; };
template <>
struct RawVec<2> { typedef unsigned short type; };

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16 x) { return __bfloat162float(x); }
template <class T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ bf16 narrow<bf16>(float x) { return __float2bfloat16_rn(x); }

// N values of T in registers, moved by accesses of at most 16 bytes; `p` is aligned to min(16, N * sizeof(T)).
template <class T, int N>
struct Pack {
    static constexpr int kBytes = N * (int)sizeof(T);
    static constexpr int kPiece = kBytes < 16 ? kBytes : 16;
    static constexpr int kPieces = kBytes / kPiece;
    typedef typename RawVec<kPiece>::type Raw;
    union {
        Raw raw[kPieces];
        T v[N];
    };
    __device__ __forceinline__ Pack() {}
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) raw[i] = reinterpret_cast<const Raw*>(p)[i];
    }
    __device__ __forceinline__ void load_stream(const T* p) {  // read once: first to leave the caches
#pragma unroll
        for (int i = 0; i < kPieces; ++i) raw[i] = __ldcs(reinterpret_cast<const Raw*>(p) + i);
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) reinterpret_cast<Raw*>(p)[i] = raw[i];
    }
    __device__ __forceinline__ void store_stream(T* p) const {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) __stcs(reinterpret_cast<Raw*>(p) + i, raw[i]);
    }
    // (bfloat16 by pairs: a shift and a mask one way, one conversion of two values the other)
    __device__ __forceinline__ void get(float (&f)[N]) const {
        if constexpr (sizeof(T) == 2 && N % 2 == 0) {
            const unsigned* w = reinterpret_cast<const unsigned*>(raw);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                f[i] = __uint_as_float(w[i / 2] << 16);
                f[i + 1] = __uint_as_float(w[i / 2] & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = widen(v[i]);
        }
    }
    __device__ __forceinline__ void set(const float (&f)[N]) {
        if constexpr (sizeof(T) == 2 && N % 2 == 0) {
            unsigned* w = reinterpret_cast<unsigned*>(raw);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(f[i], f[i + 1]);
                w[i / 2] = *reinterpret_cast<const unsigned*>(&b);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = narrow<T>(f[i]);
        }
    }
};

// Two fp32 operations in one instruction; each half is rounded as the single one is.
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }

// 32 bits that hold two bfloat16, the first one low, as floats and back
__device__ __forceinline__ float2 widen2(unsigned w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ unsigned narrow2(float2 f) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const unsigned*>(&b);
}

template <class V>
__device__ __forceinline__ V warp_sum(V x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
    return x;
}
__device__ __forceinline__ float warp_max(float x) {  // NaN only where all are
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}

template <int BYTES>
__device__ __forceinline__ void copy_async(unsigned shared, const void* global) {
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(shared), "l"(global) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(shared), "l"(global), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int BYTES>
__device__ __forceinline__ void shared_load(unsigned at, void* to) {
    unsigned* w = static_cast<unsigned*>(to);
    if (BYTES == 16) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
    else if (BYTES == 8) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    else if (BYTES == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
    else {
        unsigned short h;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at));
        *static_cast<unsigned short*>(to) = h;
    }
}

inline bool fits(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes) == 0; }

}  // namespace

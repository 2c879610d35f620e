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
    __device__ __forceinline__ void get(float (&f)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = widen(v[i]);
    }
    __device__ __forceinline__ void set(const float (&f)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = narrow<T>(f[i]);
    }
};

template <class V>
__device__ __forceinline__ V warp_sum(V x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
    return x;
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kFullMask, x, o));
    return x;
}

inline bool fits(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes) == 0; }

}  // namespace

// AdamW over a tensor table: global gradient norm, then one pass over parameters, gradients and moments.
// Part of libsparseloco (inner.cu).
//
// Bound: HBM.  A step reads theta, g, m, v once and writes theta, m, v once (28 bytes per element with 32-bit moments and
// fp32 gradients, 16 with 8-bit ones), plus the pass over g that the norm needs before anything can be updated.  The
// update kernel walks the table from its end to its beginning: the part of g that the norm pass read last is still in
// the 126 MB L2 and is not fetched again.
#pragma once
#include <cuda_fp8.h>

#include "inner_common.cuh"

namespace {

constexpr int kAdamTile = 4096;   // elements of one tensor that a CTA updates
constexpr int kAdamThreads = 256;
constexpr int kAdamVec = 8;       // consecutive elements of a thread
constexpr int kAdamBlock = 128;   // elements under one scale of an 8-bit moment: 16 threads
constexpr int kAdamMaxParts = 2048;
constexpr int kAdamNormCtas = 8;  // of the norm pass per SM, all resident

struct AdamTile {
    long long base;    // element offset in the flat buffers
    long long block0;  // first scale block
    int len;
    int tensor;
    long long pad;
};
static_assert(sizeof(AdamTile) == 32, "AdamTile layout");

struct AdamClip {  // what the norm pass leaves for the update
    float coef;
    int ok;
    unsigned ticket;  // CTAs that are done; the last one puts it back to 0
    int pad;
};

// 32-bit integer hash, Chris Wellons' published two-multiplication mix: bijective, every input bit reaches every output bit.
__device__ __forceinline__ unsigned mix32(unsigned x) {
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}
// 19 random bits of element i under a seed: mix32(i ^ key) >> 13.  Of four elements i, i + 1, .. from a multiple of 4 on, only the two
// lowest bits differ, which the first shift leaves alone: `lot_base` is common to them.
__device__ __forceinline__ unsigned hash_key(unsigned seed, unsigned long long i) {
    return mix32(seed) ^ mix32((unsigned)(i >> 32) * 0x9E3779B9u);
}
__device__ __forceinline__ unsigned lot_base(unsigned key, unsigned i) { return (i ^ key) ^ ((i ^ key) >> 16); }
__device__ __forceinline__ unsigned lot19(unsigned base, unsigned j) {  // j: 0..3
    unsigned x = (base ^ j) * 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return (x ^ (x >> 16)) >> 13;
}

__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a <= 3.402823466e38f ? a : 0.0f;  // false for NaN too
}
__device__ __forceinline__ float pow2_byte(int byte) { return __uint_as_float((unsigned)byte << 23); }  // 2^(byte - 127), byte 1..254
__device__ __forceinline__ float inv_pow2_byte(int byte) {  // 2^(127 - byte), byte 1..254 (2^-127 is no normal number)
    const unsigned b = (unsigned)(254 - byte) << 23;
    return __uint_as_float(b > (1u << 22) ? b : 1u << 22);
}
__device__ __forceinline__ int scale_byte_m(float top) {
    const unsigned b = __float_as_uint(top);
    const int e = (int)(b >> 23) + ((b & 0x7FFFFFu) > 0x600000u) - 8;  // 1.75 * 2^8 = 448 is the largest e4m3
    return e < 1 ? 1 : e;
}
__device__ __forceinline__ int scale_byte_v(float top) {
    const unsigned b = __float_as_uint(top);
    const int e = (int)(b >> 23) + ((b & 0x7FFFFFu) > 0x780000u);  // at most 31/16, the largest code's value: rounding up is never cut off
    return e < 1 ? 1 : (e > 254 ? 254 : e);
}
// Code of a finite v >= 0 in units of its scale, at most 31/16: the exponent and the first 4 mantissa bits after the lot is added
// below them; what lies under the smallest code becomes it, only 0 becomes 0.
__device__ __forceinline__ unsigned code_v(float scaled, unsigned lot) {
    const unsigned b = __float_as_uint(scaled);
    const int c = (int)(b + lot - (1792u << 19)) >> 19, least = (int)min(b, 1u);
    return (unsigned)max(c, least);
}
// ... of any value: what is not finite becomes 255
__device__ __forceinline__ unsigned code_v_any(float scaled, unsigned lot) { return scaled <= 3.402823466e38f ? min(code_v(scaled, lot), 255u) : 255u; }
__device__ __forceinline__ float value_v(unsigned c) {
    const float f = __uint_as_float((c << 19) + (1792u << 19));
    return c ? f : 0.0f;
}
__device__ __forceinline__ unsigned code_m2(float a, float b) { return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ unsigned code_m2_any(float a, float b) {  // no infinity in the format: NaN
    return code_m2(a, b) | (fabsf(a) <= 3.402823466e38f ? 0u : 0x007Fu) | (fabsf(b) <= 3.402823466e38f ? 0u : 0x7F00u);
}
__device__ __forceinline__ float2 value_m2(unsigned c) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c, __NV_E4M3);
    return __half22float2(__half2(h));
}

// 8 elements at p; A8: p is aligned to 8 elements, else to 4 only.
template <class T, bool A8, bool STREAM = true>
__device__ __forceinline__ void load8(const T* p, float (&f)[kAdamVec]) {
    if (A8) {
        Pack<T, 8> a;
        if (STREAM) a.load_stream(p);
        else a.load(p);
        a.get(f);
    } else {
        Pack<T, 4> a, b;
        if (STREAM) a.load_stream(p), b.load_stream(p + 4);
        else a.load(p), b.load(p + 4);
        float x[4], y[4];
        a.get(x);
        b.get(y);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = x[i], f[i + 4] = y[i];
    }
}
template <class T, bool A8>
__device__ __forceinline__ void store8(T* p, const float (&f)[kAdamVec]) {
    if (A8) {
        Pack<T, 8> a;
        a.set(f);
        a.store_stream(p);
    } else {
        Pack<T, 4> a, b;
        const float x[4] = {f[0], f[1], f[2], f[3]}, y[4] = {f[4], f[5], f[6], f[7]};
        a.set(x);
        b.set(y);
        a.store_stream(p);
        b.store_stream(p + 4);
    }
}
template <class T, bool A8>
__device__ __forceinline__ void load_some(const T* p, int n, float (&f)[kAdamVec]) {
    if (n >= kAdamVec) {
        load8<T, A8>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < kAdamVec; ++i) f[i] = i < n ? widen(p[i]) : 0.0f;
    }
}
template <class T, bool A8>
__device__ __forceinline__ void store_some(T* p, int n, const float (&f)[kAdamVec]) {
    if (n >= kAdamVec) {
        store8<T, A8>(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < kAdamVec; ++i)
            if (i < n) p[i] = narrow<T>(f[i]);
    }
}
// 8 code bytes as two words
template <bool A8>
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, int n) {
    uint2 w = make_uint2(0u, 0u);
    if (n >= kAdamVec) {
        if (A8) {
            w = __ldcs(reinterpret_cast<const uint2*>(p));
        } else {
            w.x = __ldcs(reinterpret_cast<const unsigned*>(p));
            w.y = __ldcs(reinterpret_cast<const unsigned*>(p) + 1);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kAdamVec; ++i)
            if (i < n) (i < 4 ? w.x : w.y) |= (unsigned)p[i] << (8 * (i & 3));
    }
    return w;
}
template <bool A8>
__device__ __forceinline__ void store_codes(uint8_t* p, int n, uint2 w) {
    if (n >= kAdamVec) {
        if (A8) {
            __stcs(reinterpret_cast<uint2*>(p), w);
        } else {
            __stcs(reinterpret_cast<unsigned*>(p), w.x);
            __stcs(reinterpret_cast<unsigned*>(p) + 1, w.y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kAdamVec; ++i)
            if (i < n) p[i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}
__device__ __forceinline__ void values_m(uint2 w, float scale, float (&m)[kAdamVec]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = value_m2(((i < 2 ? w.x : w.y) >> (16 * (i & 1))) & 0xFFFFu);
        m[2 * i] = f.x * scale;
        m[2 * i + 1] = f.y * scale;
    }
}
__device__ __forceinline__ void values_v(uint2 w, float scale, float (&v)[kAdamVec]) {
#pragma unroll
    for (int i = 0; i < kAdamVec; ++i) v[i] = value_v(((i < 4 ? w.x : w.y) >> (8 * (i & 3))) & 0xFFu) * scale;
}
// Codes of the thread's 8 moments; the 16 threads of a block agree on its scales.  Every lane of the warp takes part.
// NAN_V: a v may be NaN though its m is not (never after a step, where both come from one gradient).
template <bool NAN_V>
__device__ __forceinline__ void encode_moments(const float (&m)[kAdamVec], const float (&v)[kAdamVec], unsigned seed, unsigned long long at,
                                               uint2& cm, uint2& cv, int& bm, int& bv) {
    float tm = 0.0f, tv = 0.0f, odd = 0.0f;  // odd: 0, or NaN where an m is not finite
#pragma unroll
    for (int i = 0; i < kAdamVec; ++i) {
        tm = fmaxf(tm, fabsf(m[i]));
        tv = fmaxf(tv, v[i]);
        odd = fmaf(m[i], 0.0f, odd);
        if (NAN_V) odd = fmaf(v[i], 0.0f, odd);
    }
    const bool all_finite = __all_sync(kFullMask, odd == 0.0f && tv <= 3.402823466e38f);
    if (!all_finite) {
        tm = tv = 0.0f;
#pragma unroll
        for (int i = 0; i < kAdamVec; ++i) {
            tm = fmaxf(tm, finite_abs(m[i]));
            tv = fmaxf(tv, finite_abs(v[i]));
        }
    }
    // scale bytes grow with the largest value: the block's are the largest of its threads', found for both moments at once
    unsigned scales = (unsigned)scale_byte_m(tm) | ((unsigned)scale_byte_v(tv) << 16);
#pragma unroll
    for (int o = 8; o; o >>= 1) scales = __vmaxu2(scales, __shfl_xor_sync(kFullMask, scales, o));
    bm = (int)(scales & 0xFFFFu);
    bv = (int)(scales >> 16);
    const float im = inv_pow2_byte(bm), iv = inv_pow2_byte(bv);
    // (8 consecutive offsets that begin at a multiple of 4 may cross a multiple of 2^32)
    const unsigned base0 = lot_base(hash_key(seed, at), (unsigned)at), base1 = lot_base(hash_key(seed, at + 4), (unsigned)at + 4u);
    unsigned c[kAdamVec];
    if (all_finite && bv < 254) {
        cm.x = code_m2(m[0] * im, m[1] * im) | (code_m2(m[2] * im, m[3] * im) << 16);
        cm.y = code_m2(m[4] * im, m[5] * im) | (code_m2(m[6] * im, m[7] * im) << 16);
#pragma unroll
        for (int i = 0; i < kAdamVec; ++i) c[i] = code_v(v[i] * iv, lot19(i < 4 ? base0 : base1, (unsigned)(i & 3)));
    } else {
        cm.x = code_m2_any(m[0] * im, m[1] * im) | (code_m2_any(m[2] * im, m[3] * im) << 16);
        cm.y = code_m2_any(m[4] * im, m[5] * im) | (code_m2_any(m[6] * im, m[7] * im) << 16);
#pragma unroll
        for (int i = 0; i < kAdamVec; ++i) c[i] = code_v_any(v[i] * iv, lot19(i < 4 ? base0 : base1, (unsigned)(i & 3)));
    }
    cv.x = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
    cv.y = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
}

constexpr double kAdamTwo896 = 5.2829453113566525e269;  // 2^896

// acc + 2^896 small gains the squares of 8 values, each exact.  A conversion to fp64 runs at 16 per SM and clock, too few for
// bfloat16 at the memory's rate; but a bfloat16's square is exact in fp32, with zeros in the 8 lowest bits, and the bits of a fp32
// shifted right by 3 are the upper word of the fp64 2^-896 times as large.  What that does not hold for (squares that overflow
// or come near underflow) is converted.
template <class G>
__device__ __forceinline__ void add_squares(const float (&f)[kAdamVec], double& acc, double& small) {
    if (sizeof(G) == 2) {
        unsigned top = 0u;
#pragma unroll
        for (int j = 0; j < kAdamVec; ++j) top = max(top, __float_as_uint(f[j]) & 0x7FFFFFFFu);
        if (top - 0x30000000u < 0x5F000000u - 0x30000000u) {  // the largest is in 2^-31 .. 2^63: a square that underflows beside it is nothing
            double s[2] = {0.0, 0.0};
#pragma unroll
            for (int j = 0; j < kAdamVec; ++j) s[j & 1] += __hiloint2double((int)(__float_as_uint(f[j] * f[j]) >> 3), 0);
            small += s[0] + s[1];
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < kAdamVec; ++j) acc = fma((double)f[j], (double)f[j], acc);
}

// Sum of squares of the gradient in fp64: every CTA leaves one partial sum, the last one to finish adds them in index
// order and turns the norm into the coefficient of the update.  The assignment of tiles to CTAs is fixed, so is the sum.
template <class G, bool A8>
__global__ void __launch_bounds__(kAdamThreads, kAdamNormCtas)
adamw_norm_kernel(const AdamTile* __restrict__ tiles, long long n_tiles, const G* __restrict__ grad, double grad_scale, double max_norm,
                  double* __restrict__ parts, AdamClip* __restrict__ clip, float* __restrict__ norm_out) {
    __shared__ double warp_part[kAdamThreads / 32];
    __shared__ int last;
    const int tid = threadIdx.x;
    cudaTriggerProgrammaticLaunchCompletion();  // the update's CTAs may come and load their operands
    double acc = 0.0, small = 0.0;
    AdamTile next = tiles[blockIdx.x];
    for (long long t = blockIdx.x; t < n_tiles; t += gridDim.x) {
        const AdamTile tile = next;
        if (t + gridDim.x < n_tiles) next = tiles[t + gridDim.x];  // known before its loads are due
        const G* g = grad + tile.base;
        constexpr int kIters = kAdamTile / (kAdamThreads * kAdamVec);
        float f[kIters][kAdamVec];
        if (tile.len == kAdamTile) {
#pragma unroll
            for (int it = 0; it < kIters; ++it) load8<G, A8, false>(g + (it * kAdamThreads + tid) * kAdamVec, f[it]);
        } else {
#pragma unroll
            for (int it = 0; it < kIters; ++it) load_some<G, A8>(g + (it * kAdamThreads + tid) * kAdamVec, tile.len - (it * kAdamThreads + tid) * kAdamVec, f[it]);
        }
#pragma unroll
        for (int it = 0; it < kIters; ++it) {
            add_squares<G>(f[it], acc, small);
        }
    }
    acc = fma(small, kAdamTwo896, acc);
    acc = warp_sum(acc);
    if ((tid & 31) == 0) warp_part[tid >> 5] = acc;
    __syncthreads();
    if (tid == 0) {
        double s = 0.0;
        for (int w = 0; w < kAdamThreads / 32; ++w) s += warp_part[w];
        parts[blockIdx.x] = s;
        __threadfence();
        last = atomicAdd(&clip->ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double s = 0.0;
    for (int p = tid; p < (int)gridDim.x; p += kAdamThreads) s += __ldcg(parts + p);
    s = warp_sum(s);
    if ((tid & 31) == 0) warp_part[tid >> 5] = s;
    __syncthreads();
    if (tid == 0) {
        s = 0.0;
        for (int w = 0; w < kAdamThreads / 32; ++w) s += warp_part[w];
        const double n = fabs(grad_scale) * sqrt(s);
        double c = grad_scale;
        if (max_norm > 0.0) {
            const double q = max_norm / (n + 1e-6);
            if (q < 1.0) c *= q;  // (false for NaN: the coefficient stays, the gradient carries the NaN)
        }
        clip->coef = (float)c;
        clip->ok = n <= 1.7976931348623157e308;
        clip->ticket = 0u;
        if (norm_out) *norm_out = (float)n;
    }
}

struct AdamArgs {
    void* theta;
    const void* grad;
    void* m;
    void* v;
    uint8_t* scales;
    bf16* copy;
    const AdamClip* clip;  // NULL: no norm pass ran
    long long blocks;
    float coef, beta1, omb1, beta2, omb2, eps, inv_sqrt_bc2, step_size, lr;
    unsigned seed;
    int skip, flush;
};
// What counting a denormal v as 0 leaves out of the denominator, up to 2^-63 / sqrt(1 - beta2^t), is below 2^-23 of eps.
inline bool adamw_may_flush(float eps, float inv_sqrt_bc2) { return eps >= 9.094947017729282e-13f * inv_sqrt_bc2; }  // 2^-40

// The moments are formed by single-rounded operations in the order of the formula, so that the 8-bit codes do not depend
// on how a compiler contracts them.  (Not by the paired ones: their products and sums are contracted, explicit rounding or not.)
__device__ __forceinline__ void adamw_moments(float g, float& m, float& v, const AdamArgs& a, float c) {
    g = __fmul_rn(g, c);
    m = __fadd_rn(__fmul_rn(m, a.beta1), __fmul_rn(g, a.omb1));
    v = __fadd_rn(__fmul_rn(v, a.beta2), __fmul_rn(__fmul_rn(g, g), a.omb2));
}
// sqrt and reciprocal are the fast ones (2^-22 relative): theta's own rounding is coarser.
__device__ __forceinline__ void adamw_element(float& p, float g, float& m, float& v, const AdamArgs& a, float c, float decay) {
    adamw_moments(g, m, v, a, c);
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    p = fmaf(-a.step_size, __fdividef(m, fmaf(r, a.inv_sqrt_bc2, a.eps)), fmaf(-decay, p, p));
}
// ... where eps hides a denormal v, which the root here takes for 0 (AdamArgs::flush).
__device__ __forceinline__ void adamw_pair(float2& p, float2 g, float2& m, float2& v, const AdamArgs& a, float c, float2 decay) {
    adamw_moments(g.x, m.x, v.x, a, c);
    adamw_moments(g.y, m.y, v.y, a, c);
    float2 r, q;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(v.x));
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(v.y));
    r = fma2(r, both(a.inv_sqrt_bc2), both(a.eps));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q.x) : "f"(r.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q.y) : "f"(r.y));
    p = fma2(both(-a.step_size), mul2(q, m), fma2(decay, p, p));  // decay: -lr * weight decay
}

// What a thread reads for its 8 elements.
template <class P, class G, int BITS, bool A8>
struct AdamLoads {
    float p[kAdamVec], g[kAdamVec];
    float m[BITS == 32 ? kAdamVec : 1], v[BITS == 32 ? kAdamVec : 1];
    uint2 wm, wv;
    int bm, bv;
    __device__ __forceinline__ void load(const P* theta, const G* grad, const AdamArgs& a, const AdamTile& tile, int i) {
        const int n = tile.len - i;
        load_some<P, A8>(theta + i, n, p);
        load_some<G, A8>(grad + i, n, g);
        if constexpr (BITS == 32) {
            load_some<float, A8>(static_cast<const float*>(a.m) + tile.base + i, n, m);
            load_some<float, A8>(static_cast<const float*>(a.v) + tile.base + i, n, v);
        } else {
            wm = load_codes<A8>(static_cast<const uint8_t*>(a.m) + tile.base + i, n);
            wv = load_codes<A8>(static_cast<const uint8_t*>(a.v) + tile.base + i, n);
            const long long blk = tile.block0 + i / kAdamBlock;
            bm = n > 0 ? a.scales[blk] : 0;
            bv = n > 0 ? a.scales[a.blocks + blk] : 0;
        }
    }
    __device__ __forceinline__ void moments(float (&m_)[kAdamVec], float (&v_)[kAdamVec]) const {
        if constexpr (BITS == 32) {
#pragma unroll
            for (int j = 0; j < kAdamVec; ++j) m_[j] = m[j], v_[j] = v[j];
        } else {
            values_m(wm, pow2_byte(bm), m_);
            values_v(wv, pow2_byte(bv), v_);
        }
    }
};

template <class P, class G, int BITS, bool A8>
__global__ void __launch_bounds__(kAdamThreads)
adamw_step_kernel(const AdamTile* __restrict__ tiles, const float* __restrict__ weight_decay, const AdamArgs a) {
    const AdamTile tile = tiles[gridDim.x - 1 - blockIdx.x];  // last tiles first: their gradients are still in L2
    const int tid = threadIdx.x;
    P* theta = static_cast<P*>(a.theta) + tile.base;
    const G* grad = static_cast<const G*>(a.grad) + tile.base;
    const float decay = a.lr * weight_decay[tile.tensor];
    constexpr int kIters = kAdamTile / (kAdamThreads * kAdamVec);
    // everything that does not depend on the norm is fetched first, both iterations at once where that is few bytes: 160 a thread
    // (one at a time with a CTA more per SM: 1304 us for a step of 200 M elements and its read-out, 1103 this way)
    constexpr int kAhead = BITS == 8 ? kIters : 1;
    AdamLoads<P, G, BITS, A8> in[kAhead];
#pragma unroll
    for (int it = 0; it < kAhead; ++it) in[it].load(theta, grad, a, tile, (it * kAdamThreads + tid) * kAdamVec);
    if (a.clip) cudaGridDependencySynchronize();
    const float c = a.clip ? __ldcg(&a.clip->coef) : a.coef;
    if (a.clip && a.skip && !__ldcg(&a.clip->ok)) return;
#pragma unroll
    for (int it = 0; it < kIters; ++it) {
        const int i = (it * kAdamThreads + tid) * kAdamVec;
        if ((it * kAdamThreads + (tid & ~31)) * kAdamVec >= tile.len) return;  // whole warps only
        if (it >= kAhead) in[0].load(theta, grad, a, tile, i);
        const AdamLoads<P, G, BITS, A8>& x = in[it < kAhead ? it : 0];
        const int n = tile.len - i;  // elements of this thread (more than 8: 8; below 1: none)
        float p[kAdamVec], m[kAdamVec], v[kAdamVec];
        x.moments(m, v);
#pragma unroll
        for (int j = 0; j < kAdamVec; ++j) p[j] = x.p[j];
        if (a.flush) {
#pragma unroll
            for (int j = 0; j < kAdamVec; j += 2) {
                float2 pp = make_float2(p[j], p[j + 1]), mm = make_float2(m[j], m[j + 1]), vv = make_float2(v[j], v[j + 1]);
                adamw_pair(pp, make_float2(x.g[j], x.g[j + 1]), mm, vv, a, c, both(-decay));
                p[j] = pp.x, p[j + 1] = pp.y, m[j] = mm.x, m[j + 1] = mm.y, v[j] = vv.x, v[j + 1] = vv.y;
            }
        } else {
#pragma unroll
            for (int j = 0; j < kAdamVec; ++j) adamw_element(p[j], x.g[j], m[j], v[j], a, c, decay);
        }
        store_some<P, A8>(theta + i, n, p);
        if (a.copy) store_some<bf16, A8>(a.copy + tile.base + i, n, p);
        if (BITS == 32) {
            store_some<float, A8>(static_cast<float*>(a.m) + tile.base + i, n, m);
            store_some<float, A8>(static_cast<float*>(a.v) + tile.base + i, n, v);
        } else {
            if (n < kAdamVec) {  // what lies behind the tensor's end has no part in the scale
#pragma unroll
                for (int j = 0; j < kAdamVec; ++j)
                    if (j >= n) m[j] = v[j] = 0.0f;
            }
            uint2 cm, cv;
            int bm, bv;
            encode_moments<false>(m, v, a.seed, (unsigned long long)(tile.base + i), cm, cv, bm, bv);
            store_codes<A8>(static_cast<uint8_t*>(a.m) + tile.base + i, n, cm);
            store_codes<A8>(static_cast<uint8_t*>(a.v) + tile.base + i, n, cv);
            if (n > 0 && (tid & 15) == 0) {
                const long long blk = tile.block0 + i / kAdamBlock;
                a.scales[blk] = (uint8_t)bm;
                a.scales[a.blocks + blk] = (uint8_t)bv;
            }
        }
    }
}

// fp32 moments -> codes and scales.
template <bool A8>
__global__ void __launch_bounds__(kAdamThreads)
adamw_write_kernel(const AdamTile* __restrict__ tiles, const float* __restrict__ m32, const float* __restrict__ v32, uint8_t* m8, uint8_t* v8, uint8_t* scales,
                   long long blocks, unsigned seed) {
    const AdamTile tile = tiles[blockIdx.x];
    const int tid = threadIdx.x;
#pragma unroll
    for (int it = 0; it < kAdamTile / (kAdamThreads * kAdamVec); ++it) {
        const int i = (it * kAdamThreads + tid) * kAdamVec;
        if ((it * kAdamThreads + (tid & ~31)) * kAdamVec >= tile.len) return;  // whole warps only
        const int n = tile.len - i;
        const long long blk = tile.block0 + i / kAdamBlock;
        float m[kAdamVec], v[kAdamVec];
        load_some<float, A8>(m32 + tile.base + i, n, m);
        load_some<float, A8>(v32 + tile.base + i, n, v);
        uint2 cm, cv;
        int bm, bv;
        encode_moments<true>(m, v, seed, (unsigned long long)(tile.base + i), cm, cv, bm, bv);
        store_codes<A8>(m8 + tile.base + i, n, cm);
        store_codes<A8>(v8 + tile.base + i, n, cv);
        if (n > 0 && (tid & 15) == 0) {
            scales[blk] = (uint8_t)bm;
            scales[blocks + blk] = (uint8_t)bv;
        }
    }
}

// Codes and scales -> fp32 moments.  Mostly stores: 4 elements per thread, so that a warp's store fills whole sectors (8 per thread,
// two stores of half sectors: 70 us more for 200 M elements).
__global__ void __launch_bounds__(kAdamThreads)
adamw_read_kernel(const AdamTile* __restrict__ tiles, float* m32, float* v32, const uint8_t* m8, const uint8_t* v8, const uint8_t* scales,
                  long long blocks) {
    constexpr int kIters = kAdamTile / (kAdamThreads * 4);
    const AdamTile tile = tiles[blockIdx.x];
    unsigned wm[kIters], wv[kIters];
    int bm[kIters], bv[kIters];
#pragma unroll
    for (int it = 0; it < kIters; ++it) {
        const int i = (it * kAdamThreads + (int)threadIdx.x) * 4;
        if (i + 4 <= tile.len) {
            const long long blk = tile.block0 + i / kAdamBlock;
            wm[it] = __ldcs(reinterpret_cast<const unsigned*>(m8 + tile.base + i));
            wv[it] = __ldcs(reinterpret_cast<const unsigned*>(v8 + tile.base + i));
            bm[it] = scales[blk];
            bv[it] = scales[blocks + blk];
        }
    }
#pragma unroll
    for (int it = 0; it < kIters; ++it) {
        const int i = (it * kAdamThreads + (int)threadIdx.x) * 4;
        if (i + 4 <= tile.len) {
            const float sm = pow2_byte(bm[it]), sv = pow2_byte(bv[it]);
            const float2 a = value_m2(wm[it] & 0xFFFFu), b = value_m2(wm[it] >> 16);
            __stcs(reinterpret_cast<float4*>(m32 + tile.base + i), make_float4(a.x * sm, a.y * sm, b.x * sm, b.y * sm));
            __stcs(reinterpret_cast<float4*>(v32 + tile.base + i),
                   make_float4(value_v(wv[it] & 255u) * sv, value_v((wv[it] >> 8) & 255u) * sv, value_v((wv[it] >> 16) & 255u) * sv, value_v(wv[it] >> 24) * sv));
        } else {
            for (int j = i; j < tile.len; ++j) {
                const long long blk = tile.block0 + j / kAdamBlock;
                m32[tile.base + j] = value_m2(m8[tile.base + j]).x * pow2_byte(scales[blk]);
                v32[tile.base + j] = value_v(v8[tile.base + j]) * pow2_byte(scales[blocks + blk]);
            }
        }
    }
}

}  // namespace

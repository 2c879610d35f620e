// Next-token loss and its gradient.  Part of libsparseloco (inner.cu).
//
// Bound: HBM (logits read once, gradient written once).  A CTA takes a row: one pass with a running maximum and sum, a
// second one that forms the gradient from the row again, which by then comes from L2 (a row is 64 or 128 KB at a
// vocabulary of 32000, the rows in flight a fraction of the 126 MB).
#pragma once
#include "inner_common.cuh"

namespace {

constexpr int kLossThreads = 512;

struct LossWork {
    int valid;        // rows that count
    unsigned ticket;  // CTAs that are done
    int pad[2];
};

struct LossArgs {
    long long rows, ld_logits, ld_grad, ignore_index;
    int vocab, target_bits, mean;
    float smoothing, z, scale;
    const void* targets;
    float *row_loss, *lse, *total;
    LossWork* work;
};

__device__ __forceinline__ long long target_of(const LossArgs& a, long long row) {
    return a.target_bits == 64 ? static_cast<const long long*>(a.targets)[row] : (long long)static_cast<const int*>(a.targets)[row];
}

__global__ void __launch_bounds__(1024)
loss_count_kernel(const LossArgs a) {
    __shared__ int part[32];
    int n = 0;
    for (long long r = threadIdx.x; r < a.rows; r += 1024) n += target_of(a, r) != a.ignore_index;
    n = warp_sum(n);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
        n = 0;
        for (int w = 0; w < 32; ++w) n += part[w];
        a.work->valid = n;
        a.work->ticket = 0u;
        if (a.rows == 0 && a.total) *a.total = 0.0f;
    }
}

// Running maximum and sum of exponentials; sum is relative to the maximum.  -inf with 0 = nothing seen.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
    const float top = fmaxf(m, m2);
    if (top == -INFINITY) {  // nothing but -inf on both sides (or NaN, which the sums carry)
        s += s2;
        return;
    }
    s = s * expf(m - top) + s2 * expf(m2 - top);
    m = top;
}

template <class T, int VEC>
__global__ void __launch_bounds__(kLossThreads)
token_loss_kernel(const LossArgs a, const T* logits, T* grad) {
    __shared__ float sm[32], ss[32], sx[32];
    __shared__ int last;
    const int tid = threadIdx.x;
    const long long row = blockIdx.x;
    const T* x = logits + row * a.ld_logits;
    // the vector body begins at the row's first 16-byte boundary
    int head = 0;
    if (VEC > 1) {
        head = (int)((16u - (unsigned)(reinterpret_cast<uintptr_t>(x) & 15u)) & 15u) / (int)sizeof(T);
        if (head > a.vocab) head = a.vocab;
    }
    const int body = VEC > 1 ? (a.vocab - head) / VEC : 0;  // vectors
    const int rest = head + body * VEC;                     // scalars from here on
    const long long target = target_of(a, row);
    const bool counts = target != a.ignore_index, inside = target >= 0 && target < a.vocab;
    float m = -INFINITY, s = 0.0f, sum = 0.0f;
    auto see = [&](float v) {
        sum += v;
        if (v > m) {
            s = s * expf(m - v) + 1.0f;
            m = v;
        } else if (v == -INFINITY) {
        } else {
            s += expf(v - m);  // (NaN and +inf end here and stay in the sum)
        }
    };
    for (int i = tid; i < head; i += kLossThreads) see(widen(x[i]));
    for (int i = tid; i < body; i += kLossThreads) {
        Pack<T, VEC> p;
        p.load(x + head + i * VEC);
        float f[VEC];
        p.get(f);
        float top = f[0];
#pragma unroll
        for (int j = 1; j < VEC; ++j) top = fmaxf(top, f[j]);
        if (top > m) {
            s = s * expf(m - top);
            m = top;
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            sum += f[j];
            if (f[j] != -INFINITY) s += expf(f[j] - m);
        }
    }
    for (int i = rest + tid; i < a.vocab; i += kLossThreads) see(widen(x[i]));
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float m2 = __shfl_xor_sync(kFullMask, m, o), s2 = __shfl_xor_sync(kFullMask, s, o);
        join(m, s, m2, s2);
    }
    sum = warp_sum(sum);
    if ((tid & 31) == 0) sm[tid >> 5] = m, ss[tid >> 5] = s, sx[tid >> 5] = sum;
    const float xt = counts && inside ? widen(x[target]) : 0.0f;  // (read before any thread writes a gradient in its place)
    __syncthreads();
    m = sm[0], s = ss[0], sum = sx[0];
    for (int w = 1; w < kLossThreads / 32; ++w) {
        join(m, s, sm[w], ss[w]);
        sum += sx[w];
    }
    const bool empty = m == -INFINITY && s == 0.0f;  // every logit is -inf
    const float lse = empty ? -INFINITY : m + logf(s);
    const int valid = a.work->valid;
    const float w = a.mean ? a.scale / (float)(valid > 0 ? valid : 1) : a.scale;
    if (tid == 0) {
        float loss = 0.0f;
        if (counts) {
            if (!inside) loss = __int_as_float(0x7FC00000);
            else if (empty) loss = INFINITY;
            else {
                loss = lse - (1.0f - a.smoothing) * xt + a.z * lse * lse;
                if (a.smoothing != 0.0f) loss -= a.smoothing * (sum / (float)a.vocab);
            }
        }
        a.row_loss[row] = loss;
        if (a.lse) a.lse[row] = lse;
    }
    if (grad) {
        T* g = grad + row * a.ld_grad;
        if (!counts || !inside || empty) {
            // zeros; the stores go where the loads went, by the same alignment
            for (int i = tid; i < head; i += kLossThreads) g[i] = narrow<T>(0.0f);
            for (int i = tid; i < body; i += kLossThreads) {
                Pack<T, VEC> p;
#pragma unroll
                for (int j = 0; j < VEC; ++j) p.v[j] = narrow<T>(0.0f);
                p.store(g + head + i * VEC);
            }
            for (int i = rest + tid; i < a.vocab; i += kLossThreads) g[i] = narrow<T>(0.0f);
        } else {
            const float k = w * fmaf(2.0f * a.z, lse, 1.0f) / s, off = w * a.smoothing / (float)a.vocab, hit = w * (1.0f - a.smoothing);
            const int t = (int)target;
            auto of = [&](float v, int i) {
                float d = fmaf(k, expf(v - m), -off);
                if (i == t) d -= hit;
                return d;
            };
            for (int i = tid; i < head; i += kLossThreads) g[i] = narrow<T>(of(widen(x[i]), i));
            for (int i = tid; i < body; i += kLossThreads) {
                Pack<T, VEC> p;
                p.load(x + head + i * VEC);
#pragma unroll
                for (int j = 0; j < VEC; ++j) p.v[j] = narrow<T>(of(widen(p.v[j]), head + i * VEC + j));
                p.store(g + head + i * VEC);
            }
            for (int i = rest + tid; i < a.vocab; i += kLossThreads) g[i] = narrow<T>(of(widen(x[i]), i));
        }
    }
    // the last CTA adds the rows' losses in their order: thread by thread, then thread after thread
    if (!a.total) return;
    if (tid == 0) {
        __threadfence();
        last = atomicAdd(&a.work->ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double t = 0.0;
    for (long long r = tid; r < a.rows; r += kLossThreads) t += (double)__ldcg(a.row_loss + r);
    t = warp_sum(t);
    __shared__ double st[32];
    if ((tid & 31) == 0) st[tid >> 5] = t;
    __syncthreads();
    if (tid == 0) {
        t = 0.0;
        for (int i = 0; i < kLossThreads / 32; ++i) t += st[i];
        *a.total = valid > 0 ? (float)(t * (double)w) : 0.0f;
    }
}

}  // namespace

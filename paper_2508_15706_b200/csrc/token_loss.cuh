// Next-token loss and its gradient.  Part of libsparseloco (inner.cu).
//
// Bound: HBM (logits read once, gradient written once).  A row stays in the registers of its CTA, or of the CTAs of a cluster where
// one CTA cannot hold it or there are fewer rows than SMs: one pass for a maximum and a sum of exponentials per thread, one
// exchange, then the gradient from the same registers.
// Exponentials are 2^(x log2 e - M), one fused multiply-add and one instruction: M stands for the maximum in that scale, and its
// rounding moves nothing as long as it is the same M everywhere.  Where |x log2 e| could overflow (a row of the type's lowest
// value) the factor is 1 instead: numbers of that size are equal or differ by more than any exponential can show.
// Rows that eight CTAs cannot hold, and gradients that sit elsewhere relative to 16 bytes than their logits, go through a kernel that
// reads the row twice (the second time from L2).
#pragma once
#include <cooperative_groups.h>

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

// The number of rows that count; also puts the ticket back.
__global__ void __launch_bounds__(1024)
loss_count_kernel(const LossArgs a) {
    __shared__ int part[32];
    cudaTriggerProgrammaticLaunchCompletion();  // the rows' CTAs may come and read their logits
    int n = 0;
#pragma unroll 4
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

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {  // 2^x, relative error 2^-22; 0 for -inf
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float loss_scale(float top) { return fabsf(top) < 1e30f ? kLog2e : 1.0f; }  // (1 for infinities)
__device__ __forceinline__ float loss_offset(float top) { return top == -INFINITY ? 0.0f : top * loss_scale(top); }

// Scaled maximum and sum of exponentials relative to it; -inf with 0 = nothing seen, NaN and +inf end in the sum.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
    const float top = fmaxf(m, m2);
    if (top == -INFINITY) {
        s += s2;
        return;
    }
    s = s * exp2_fast(m - top) + s2 * exp2_fast(m2 - top);
    m = top;
}

// What a row comes to, from its maximum, sum and target.
struct LossRow {
    float m, s, sum, lse, w, scale;
    long long target;
    int valid;
    bool counts, inside, empty;
    __device__ __forceinline__ bool has_gradient() const { return counts && inside && !empty; }
};
__device__ __forceinline__ void finish_row(const LossArgs& a, LossRow& r) {
    r.empty = r.m == -INFINITY && r.s == 0.0f;  // every logit is -inf
    r.scale = fabsf(r.m) < 1e30f ? kLog2e : 1.0f;
    r.lse = r.empty ? -INFINITY : r.scale == 1.0f ? r.m + logf(r.s) : (r.m + log2f(r.s)) * kLn2;
    cudaGridDependencySynchronize();
    r.valid = __ldcg(&a.work->valid);
    r.w = a.mean ? a.scale / (float)(r.valid > 0 ? r.valid : 1) : a.scale;
}
__device__ __forceinline__ void write_row(const LossArgs& a, const LossRow& r, long long row, float xt) {
    float loss = 0.0f;
    if (r.counts) {
        if (!r.inside) loss = __int_as_float(0x7FC00000);
        else if (r.empty) loss = INFINITY;
        else {
            loss = r.lse - (1.0f - a.smoothing) * xt + a.z * r.lse * r.lse;
            if (a.smoothing != 0.0f) loss -= a.smoothing * (r.sum / (float)a.vocab);
        }
    }
    a.row_loss[row] = loss;
    if (a.lse) a.lse[row] = r.lse;
}
// The last of `rows` callers adds the rows' losses in a fixed order: thread by thread, then thread after thread.
__device__ __forceinline__ void add_rows(const LossArgs& a, const LossRow& r) {
    __shared__ int last;
    __shared__ double st[32];
    if (!a.total) return;
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(&a.work->ticket, 1u) == (unsigned)(a.rows - 1);
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double t = 0.0;
    for (long long i = threadIdx.x; i < a.rows; i += blockDim.x) t += (double)__ldcg(a.row_loss + i);
    t = warp_sum(t);
    if ((threadIdx.x & 31) == 0) st[threadIdx.x >> 5] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        t = 0.0;
        for (int i = 0; i < (int)(blockDim.x >> 5); ++i) t += st[i];
        *a.total = r.valid > 0 ? (float)(t * (double)r.w) : 0.0f;
    }
}

// A row in registers: NV accesses of VEC values per thread, `cluster` CTAs per row.  The vector body begins at the row's first
// 16-byte boundary; the values before it belong to the first CTA, those behind it to the last, one per thread.
template <class T, int VEC, int NV>
__global__ void __launch_bounds__(kLossThreads, NV * VEC * (int)sizeof(T) <= 128 ? 2 : 1)
loss_row_kernel(const LossArgs a, const T* logits, T* grad, int cluster) {
    __shared__ float sm[32], ss[32], sx[32];
    __shared__ float mine[4];  // this CTA's maximum, sum of exponentials, sum: read by the cluster
    const int tid = threadIdx.x, threads = blockDim.x;
    const long long row = blockIdx.x / (unsigned)cluster;
    const int rank = (int)(blockIdx.x - (unsigned)row * (unsigned)cluster);
    const T* x = logits + row * a.ld_logits;
    int head = (int)((16u - (unsigned)(reinterpret_cast<uintptr_t>(x) & 15u)) & 15u) / (int)sizeof(T);
    if (head > a.vocab) head = a.vocab;
    const int body = (a.vocab - head) / VEC, tail = head + body * VEC, per = (body + cluster - 1) / cluster;
    const int begin = rank * per, end = min(body, begin + per);
    Pack<T, VEC> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = begin + i * threads + tid;
        if (at < end) {
            v[i].load_stream(x + head + at * VEC);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i].v[j] = narrow<T>(-INFINITY);
        }
    }
    // a single value before or behind the body (each at most VEC - 1 of them; both ends may be in one CTA)
    const int before = rank == 0 && tid < head ? tid : -1, behind = rank == cluster - 1 && tail + tid < a.vocab ? tail + tid : -1;
    const float first = before >= 0 ? widen(x[before]) : -INFINITY, last_one = behind >= 0 ? widen(x[behind]) : -INFINITY;
    LossRow r;
    r.target = target_of(a, row);
    r.counts = r.target != a.ignore_index;
    r.inside = r.target >= 0 && r.target < a.vocab;
    const float xt = r.counts && r.inside ? widen(x[r.target]) : 0.0f;  // (before any gradient takes its place: a barrier follows)

    float m = fmaxf(first, last_one);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float f[VEC];
        v[i].get(f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) m = fmaxf(m, f[j]);
    }
    const float scale = loss_scale(m), ref = loss_offset(m);
    float s = exp2_fast(fmaf(first, scale, -ref)) + exp2_fast(fmaf(last_one, scale, -ref)), sum = 0.0f;
    if (a.smoothing != 0.0f) {
        sum = (before >= 0 ? first : 0.0f) + (behind >= 0 ? last_one : 0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (begin + i * threads + tid < end) {
                float f[VEC];
                v[i].get(f);
#pragma unroll
                for (int j = 0; j < VEC; ++j) sum += f[j];
            }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float f[VEC], part = 0.0f;  // (short chains of additions)
        v[i].get(f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) part += exp2_fast(fmaf(f[j], scale, -ref));
        s += part;
    }
    m *= scale;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float m2 = __shfl_xor_sync(kFullMask, m, o), s2 = __shfl_xor_sync(kFullMask, s, o);
        join(m, s, m2, s2);
        if (a.smoothing != 0.0f) sum += __shfl_xor_sync(kFullMask, sum, o);
    }
    if ((tid & 31) == 0) sm[tid >> 5] = m, ss[tid >> 5] = s, sx[tid >> 5] = sum;
    __syncthreads();
    r.m = sm[0], r.s = ss[0], r.sum = sx[0];
    for (int w = 1; w < threads / 32; ++w) {
        join(r.m, r.s, sm[w], ss[w]);
        r.sum += sx[w];
    }
    if (cluster > 1) {
        namespace cg = cooperative_groups;
        auto group = cg::this_cluster();
        if (tid == 0) mine[0] = r.m, mine[1] = r.s, mine[2] = r.sum;
        group.sync();
        for (int c = 0; c < cluster; ++c) {  // in the same order in every CTA
            const float* other = group.map_shared_rank(mine, (unsigned)c);
            const float m2 = other[0], s2 = other[1], x2 = other[2];
            if (c == 0) r.m = m2, r.s = s2, r.sum = x2;
            else join(r.m, r.s, m2, s2), r.sum += x2;
        }
        group.sync();  // nobody leaves while its values are read
    }
    finish_row(a, r);
    if (rank == 0 && tid == 0) write_row(a, r, row, xt);
    if (grad) {
        T* g = grad + row * a.ld_grad;
        const bool some = r.has_gradient();
        const float k = some ? r.w * fmaf(2.0f * a.z, r.lse, 1.0f) / r.s : 0.0f, off = some ? r.w * a.smoothing / (float)a.vocab : 0.0f,
                    hit = r.w * (1.0f - a.smoothing);
        const int t = some ? (int)r.target : -1;
        const int tv = t >= head && t < tail ? (t - head) / VEC : -1, te = t - head - tv * VEC;  // the target's vector and place in it
        const float top = some ? r.m : 0.0f, scale = r.scale;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = begin + i * threads + tid;
            if (at < end) {
                float f[VEC];
                v[i].get(f);
#pragma unroll
                for (int j = 0; j < VEC; ++j) f[j] = fmaf(k, exp2_fast(fmaf(f[j], scale, -top)), -off);
                if (at == tv) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        if (j == te) f[j] -= hit;
                }
                if (!some) {  // (0 times what overflows or is NaN would not be 0)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) f[j] = 0.0f;
                }
                Pack<T, VEC> o;
                o.set(f);
                o.store_stream(g + head + at * VEC);
            }
        }
        auto one = [&](int at, float val) {
            float d = some ? fmaf(k, exp2_fast(fmaf(val, scale, -top)), -off) : 0.0f;
            if (at == t) d -= hit;
            g[at] = narrow<T>(d);
        };
        if (before >= 0) one(before, first);
        if (behind >= 0) one(behind, last_one);
    }
    if (rank == 0) add_rows(a, r);
}

// The row read twice: a running maximum and sum, then the gradient.

template <class T, int VEC>
__global__ void __launch_bounds__(kLossThreads)
loss_stream_kernel(const LossArgs a, const T* logits, T* grad) {
    __shared__ float sm[32], ss[32], sx[32];
    const int tid = threadIdx.x;
    const long long row = blockIdx.x;
    const T* x = logits + row * a.ld_logits;
    int head = 0;
    if (VEC > 1) {
        head = (int)((16u - (unsigned)(reinterpret_cast<uintptr_t>(x) & 15u)) & 15u) / (int)sizeof(T);
        if (head > a.vocab) head = a.vocab;
    }
    const int body = VEC > 1 ? (a.vocab - head) / VEC : 0;  // vectors
    const int rest = head + body * VEC;                     // scalars from here on
    LossRow r;
    r.target = target_of(a, row);
    r.counts = r.target != a.ignore_index;
    r.inside = r.target >= 0 && r.target < a.vocab;
    float m = -INFINITY, s = 0.0f, sum = 0.0f;
    float scale = kLog2e, ref = 0.0f;           // m in the scale of the exponentials
    auto rise = [&](float top) {                // the maximum so far goes up to top
        if (top > m) {
            const float to = loss_offset(top);
            s *= exp2_fast(m == -INFINITY ? m : ref - to);
            m = top;
            scale = loss_scale(top);
            ref = to;
        }
    };
    auto see = [&](float v) {
        sum += v;
        s += exp2_fast(fmaf(v, scale, -ref));   // (0 for -inf; NaN and +inf end here and stay in the sum)
    };
    for (int i = tid; i < head; i += kLossThreads) rise(widen(x[i])), see(widen(x[i]));
    for (int i = tid; i < body; i += kLossThreads) {
        Pack<T, VEC> p;
        p.load(x + head + i * VEC);
        float f[VEC];
        p.get(f);
        float top = f[0];
#pragma unroll
        for (int j = 1; j < VEC; ++j) top = fmaxf(top, f[j]);
        rise(top);
#pragma unroll
        for (int j = 0; j < VEC; ++j) see(f[j]);
    }
    for (int i = rest + tid; i < a.vocab; i += kLossThreads) rise(widen(x[i])), see(widen(x[i]));
    m = m == -INFINITY ? m : ref;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const float m2 = __shfl_xor_sync(kFullMask, m, o), s2 = __shfl_xor_sync(kFullMask, s, o);
        join(m, s, m2, s2);
    }
    sum = warp_sum(sum);
    if ((tid & 31) == 0) sm[tid >> 5] = m, ss[tid >> 5] = s, sx[tid >> 5] = sum;
    const float xt = r.counts && r.inside ? widen(x[r.target]) : 0.0f;  // (read before any thread writes a gradient in its place)
    __syncthreads();
    r.m = sm[0], r.s = ss[0], r.sum = sx[0];
    for (int w = 1; w < kLossThreads / 32; ++w) {
        join(r.m, r.s, sm[w], ss[w]);
        r.sum += sx[w];
    }
    finish_row(a, r);
    if (tid == 0) write_row(a, r, row, xt);
    if (grad) {
        T* g = grad + row * a.ld_grad;
        const bool some = r.has_gradient();
        const float k = some ? r.w * fmaf(2.0f * a.z, r.lse, 1.0f) / r.s : 0.0f, off = r.w * a.smoothing / (float)a.vocab, hit = r.w * (1.0f - a.smoothing);
        auto of = [&](float v, int i) {
            if (!some) return 0.0f;
            const float d = fmaf(k, exp2_fast(fmaf(v, r.scale, -r.m)), -off);
            return i == (int)r.target ? d - hit : d;
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
    add_rows(a, r);
}

}  // namespace

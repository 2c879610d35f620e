// Next-token loss and its gradient.  Part of libsparseloco (inner.cu).
//
// Bound: HBM (logits read once, gradient written once).  CTAs stay and walk over rows.  A row, or the part of it that a CTA of a cluster
// has, comes through a ring in shared memory two rows ahead; its exponentials relative to each thread's own maximum stay in
// registers until the row's maximum and sum are known, and the gradient is those times one factor per thread: one exponential per
// logit.  (Computed a second time instead, with the row's bits in registers, they bound the kernel: 318 us at 8192 x 32000.)
// Exponentials are 2^(x log2 e - M), one fused multiply-add and one instruction: M stands for the maximum in that scale, and its
// rounding moves nothing as long as it is the same M everywhere and is small beside an exponential's range: up to 2^30, where it is
// 64 at most.  Beyond (a mask of -1e10, a row of the type's lowest value) the factor is 1 instead: numbers of that size are equal
// or 64 and more apart, and 2^-64 is nothing in a sum.  Maxima are compared as M / 2 and, beyond 2^30, as they are: an order that
// is theirs on both sides of 2^30 and passes no number's range.
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
constexpr float kLossFar = 1073741824.0f;  // 2^30
__device__ __forceinline__ float loss_scale(float top) { return fabsf(top) < kLossFar ? kLog2e : 1.0f; }  // (1 for infinities)
__device__ __forceinline__ float loss_offset(float top) { return top == -INFINITY ? 0.0f : top * loss_scale(top); }
// The rank of a maximum: half of its offset, or, beyond 2^30, the maximum itself.  `lift` is what sums relative to `from` are
// multiplied with to be relative to `to`: 2 to the difference of the offsets.
__device__ __forceinline__ float loss_rank(float top) { return fabsf(top) < kLossFar ? 0.5f * (top * kLog2e) : top; }
__device__ __forceinline__ float lift(float from, float to) { return exp2_fast((from - to) + (from - to)); }

// Rank of the maximum and sum of exponentials relative to it; -inf with 0 = nothing seen, NaN and +inf end in the sum.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
    const float top = fmaxf(m, m2);
    if (top == -INFINITY) {
        s += s2;
        return;
    }
    s = s * lift(m, top) + s2 * lift(m2, top);
    m = top;
}

// The CTA's maximum, sum and plain sum from its threads', the same in every thread, each exchange one scaling per thread: first the
// maximum, then the sums relative to it.  `buf`: [3][32], not to be written again before every thread has read it: callers alternate.
__device__ __forceinline__ void block_join(float& m, float& s, float& sum, bool with_sum, float (*buf)[32]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    float top = warp_max(m);
    s = top == -INFINITY ? warp_sum(s) : warp_sum(s * lift(m, top));
    if (with_sum) sum = warp_sum(sum);
    if (lane == 0) buf[0][warp] = top, buf[1][warp] = s, buf[2][warp] = sum;
    __syncthreads();
    m = lane < warps ? buf[0][lane] : -INFINITY;
    s = lane < warps ? buf[1][lane] : 0.0f;
    top = warp_max(m);
    s = top == -INFINITY ? warp_sum(s) : warp_sum(s * lift(m, top));
    if (with_sum) sum = warp_sum(lane < warps ? buf[2][lane] : 0.0f);
    m = top;
}

// What a row comes to, from its maximum, sum and target.
struct LossRow {
    float m, s, sum;   // m: the maximum's rank
    float scale, ref;  // exponentials are 2^(x scale - ref)
    long long target;
    bool counts, inside, empty;
    __device__ __forceinline__ bool has_gradient() const { return counts && inside && !empty; }
    __device__ __forceinline__ void aim(const LossArgs& a, long long its_target) {
        target = its_target;
        counts = target != a.ignore_index;
        inside = target >= 0 && target < a.vocab;
    }
    __device__ __forceinline__ void finish() {
        empty = m == -INFINITY && s == 0.0f;  // every logit is -inf
        scale = loss_scale(m);  // (the rank of a maximum below 2^30 is below 2^30)
        ref = scale == 1.0f ? m : m + m;
    }
    __device__ __forceinline__ float log_sum() const { return scale == 1.0f ? logf(s) : log2f(s); }
    __device__ __forceinline__ float lse(float log_s) const { return empty ? -INFINITY : scale == 1.0f ? ref + log_s : (ref + log_s) * kLn2; }
    // lse - x for a logit x (or their mean): from the parts, since lse is rounded at its own size, which may be any.  The rounding of
    // ref is in s and in ref - x log2 e alike and goes out between them.  What is below 2^-21, twice the accuracy of an exponential, is 0.
    __device__ __forceinline__ float above(float x, float log_s) const {
        const float d = scale == 1.0f ? ref - x + log_s : fabsf(x) < kLossFar ? (log_s + fmaf(-x, scale, ref)) * kLn2 : lse(log_s) - x;
        return d < 4.76837158203125e-7f ? 0.0f : d;  // (NaN stays)
    }
    // ... within 2^-21 of lse or so: what the gradient's factor of p needs
    __device__ __forceinline__ float near_lse() const { return scale == 1.0f ? ref + __logf(s) : (ref + __log2f(s)) * kLn2; }
    // (the quotient within 2 ulp: s is at most 2^95, far below where the fast division gives up, and at least 2^-65)
    __device__ __forceinline__ float factor(const LossArgs& a, float w) const { return __fdividef(a.z == 0.0f ? w : w * fmaf(2.0f * a.z, near_lse(), 1.0f), s); }
};
// 1 / (rows that count), or 1, times the caller's scale; the count comes from the kernel before
__device__ __forceinline__ float row_weight(const LossArgs& a, int& valid) {
    cudaGridDependencySynchronize();
    valid = __ldcg(&a.work->valid);
    return a.mean ? a.scale / (float)(valid > 0 ? valid : 1) : a.scale;
}
__device__ __forceinline__ void write_row(const LossArgs& a, const LossRow& r, long long row, float xt) {
    float loss = 0.0f;
    const float log_s = r.log_sum(), lse = r.lse(log_s);
    if (r.counts) {
        if (!r.inside) loss = __int_as_float(0x7FC00000);
        else if (r.empty) loss = INFINITY;
        else {
            loss = a.z == 0.0f ? 0.0f : a.z * lse * lse;
            if (a.smoothing != 1.0f) loss += (1.0f - a.smoothing) * r.above(xt, log_s);
            if (a.smoothing != 0.0f) loss += a.smoothing * r.above(r.sum / (float)a.vocab, log_s);
        }
    }
    a.row_loss[row] = loss;
    if (a.lse) a.lse[row] = lse;
}
// The last of `callers` CTAs adds the rows' losses in a fixed order: thread by thread, then thread after thread.
__device__ __forceinline__ void add_rows(const LossArgs& a, unsigned callers, float w, int valid) {
    __shared__ int last;
    __shared__ double st[32];
    if (!a.total) return;
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(&a.work->ticket, 1u) == callers - 1;
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
        *a.total = valid > 0 ? (float)(t * (double)w) : 0.0f;
    }
}

// The largest of a vector's values (never NaN unless all are).
template <class T, int VEC>
__device__ __forceinline__ float top_of(const unsigned (&w)[4]) {
    if (sizeof(T) == 2) {
        __nv_bfloat162 t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = *reinterpret_cast<const __nv_bfloat162*>(&w[j]);
        t[0] = __hmax2(__hmax2(t[0], t[1]), __hmax2(t[2], t[3]));
        const float2 f = widen2(*reinterpret_cast<const unsigned*>(&t[0]));
        return fmaxf(f.x, f.y);
    }
    return fmaxf(fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])), fmaxf(__uint_as_float(w[2]), __uint_as_float(w[3])));
}
template <class T, int VEC>
__device__ __forceinline__ void unpack(const unsigned (&w)[4], float2 (&f)[VEC / 2]) {
#pragma unroll
    for (int j = 0; j < VEC / 2; ++j) f[j] = sizeof(T) == 2 ? widen2(w[j]) : make_float2(__uint_as_float(w[(2 * j) & 3]), __uint_as_float(w[(2 * j + 1) & 3]));
}

// A CTA's part of a row.  The vector body begins at the row's first 16-byte boundary; the values before it belong to the first CTA
// of the cluster, those behind it to the last, one per thread.  RAGGED: there may be such values, else every row is all vectors.
template <class T, int VEC, bool RAGGED>
struct LossPart {
    int head, begin, vectors, tail;  // this CTA's vectors begin at value head + begin * VEC of the row; single values from `tail` on
    __device__ __forceinline__ LossPart(const LossArgs& a, const T* x, int rank, int cluster) {
        head = RAGGED ? (int)((16u - (unsigned)(reinterpret_cast<uintptr_t>(x) & 15u)) & 15u) / (int)sizeof(T) : 0;
        if (RAGGED && head > a.vocab) head = a.vocab;
        const int body = (a.vocab - head) / VEC, per = cluster == 1 ? body : (body + cluster - 1) / cluster;
        begin = rank * per;
        vectors = min(body, begin + per) - begin;
        tail = head + body * VEC;
    }
    __device__ __forceinline__ int base() const { return head + begin * VEC; }
    __device__ __forceinline__ int before(int rank) const { return RAGGED && rank == 0 && (int)threadIdx.x < head ? (int)threadIdx.x : -1; }
    __device__ __forceinline__ int behind(const LossArgs& a, int rank, int cluster) const {
        return RAGGED && rank == cluster - 1 && tail + (int)threadIdx.x < a.vocab ? tail + (int)threadIdx.x : -1;
    }
};

constexpr int kLossStages = 3;
constexpr unsigned kLossPolls = 1u << 22;  // of a wait for a copy; if one ever runs out, nothing more is asked or waited for, and the losses from there on are NaN

__device__ __forceinline__ void bulk_expect(unsigned barrier, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(barrier), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_copy(unsigned to, const void* from, unsigned bytes, unsigned barrier) {
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(barrier) : "memory");
}
__device__ __forceinline__ bool bulk_wait(unsigned barrier, unsigned phase) {
    unsigned done = 0;
    for (unsigned n = 0; !done && n < kLossPolls; ++n)
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(barrier), "r"(phase) : "memory");
    return done != 0;
}

__device__ __forceinline__ void shared_value(unsigned at, float& x) { asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at)); }
__device__ __forceinline__ void shared_value(unsigned at, bf16& x) {
    unsigned short h;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at));
    x = __ushort_as_bfloat16(h);
}

// NV vectors of VEC values per thread; all but a thread's last one exist in every row (the launch sees to it).
template <class T, int VEC, int NV, bool RAGGED>
__global__ void __launch_bounds__(kLossThreads, NV * VEC <= 32 ? 2 : 1)
loss_row_kernel(const LossArgs a, const T* logits, T* grad, int cluster) {
    extern __shared__ __align__(16) char ring[];  // [stages][NV * threads] vectors
    __shared__ __align__(8) unsigned long long landed[kLossStages];
    __shared__ float buf[2][3][32], xts[2];
    __shared__ float mine[2][4];  // this CTA's maximum, sum of exponentials, sum of two rows in turn: read by the cluster
    const int tid = threadIdx.x, threads = blockDim.x;
    const unsigned teams = gridDim.x / (unsigned)cluster;
    long long row = blockIdx.x / (unsigned)cluster;
    const int rank = (int)(blockIdx.x - (unsigned)row * (unsigned)cluster);
    const unsigned ring_at = (unsigned)__cvta_generic_to_shared(ring), place = ring_at + (unsigned)tid * 16u, pitch = (unsigned)threads * 16u, stage_bytes = (unsigned)NV * pitch;
    const unsigned landed_at = (unsigned)__cvta_generic_to_shared(landed);
    // one thread asks for a CTA's whole part of a row in one copy
    auto fetch = [&](long long i, unsigned stage) {
        if (i >= a.rows) return;
        const T* x = logits + i * a.ld_logits;
        const LossPart<T, VEC, RAGGED> p(a, x, rank, cluster);
        const unsigned bytes = (unsigned)p.vectors * 16u;
        bulk_expect(landed_at + stage * 8u, bytes);
        if (bytes) bulk_copy(ring_at + stage * stage_bytes, x + p.base(), bytes, landed_at + stage * 8u);
    };
    if (tid == 0) {
        for (int k = 0; k < kLossStages; ++k) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(landed_at + k * 8u) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int k = 0; k < kLossStages; ++k) fetch(row + (long long)k * teams, (unsigned)k);
    }
    __syncthreads();
    float w = 0.0f;
    int valid = 0;
    bool weighed = false;
    unsigned at = 0, stage = 0, phase = 0;
    bool arrived = true;
    auto target_at = [&](long long i) { return i < a.rows ? target_of(a, i) : -1ll; };
    long long its_target = target_at(row);
    // single values of the next row, asked for a row ahead
    float first = -INFINITY, last_one = -INFINITY, first_next = -INFINITY, last_next = -INFINITY;
    auto singles = [&](long long i, float& front, float& back) {
        if (!RAGGED || i >= a.rows) return;
        const T* x = logits + i * a.ld_logits;
        const LossPart<T, VEC, RAGGED> p(a, x, rank, cluster);
        const int f = p.before(rank), b = p.behind(a, rank, cluster);
        front = f >= 0 ? widen(x[f]) : -INFINITY;
        back = b >= 0 ? widen(x[b]) : -INFINITY;
    };
    singles(row, first, last_one);
    const float inv_threads = 1.0f / (float)threads;
    float off_all = 0.0f;
    for (int turn = 0; row < a.rows; row += teams, turn ^= 1) {
        const long long target_next = target_at(row + teams);
        singles(row + teams, first_next, last_next);
        const T* x = logits + row * a.ld_logits;
        const LossPart<T, VEC, RAGGED> part(a, x, rank, cluster);
        const int before = part.before(rank), behind = part.behind(a, rank, cluster);
        const bool last_too = (NV - 1) * threads + tid < part.vectors;
        float m = -INFINITY, s, sum = 0.0f, rank_own;
        float2 e[NV][VEC / 2];
        arrived = arrived && bulk_wait(landed_at + stage * 8u, phase);
        LossRow r;
        r.aim(a, its_target);
        // the target's place in this CTA's part, its vector there, whose it is; the CTA that has it writes the row's loss
        const int t = r.counts && r.inside ? (int)r.target - part.base() : -1;
        const bool in_body = t >= 0 && t < part.vectors * VEC;
        const int tv = in_body ? t / VEC : 0, ti = (int)(((float)tv + 0.5f) * inv_threads), te = t - tv * VEC;
        const bool owner = in_body && tid == tv - ti * threads;  // of the target: value te of its vector ti
        const bool writes = r.counts && r.inside ? in_body || (rank == 0 && r.target < part.head) || (rank == cluster - 1 && r.target >= part.tail) : rank == 0;
        {
            m = fmaxf(first, last_one);
            unsigned v[NV][4];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[i][0]), "=r"(v[i][1]), "=r"(v[i][2]), "=r"(v[i][3]) : "r"(place + at + i * pitch));
                if (i == NV - 1 && !last_too) v[i][0] = v[i][1] = v[i][2] = v[i][3] = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;  // -inf
                m = fmaxf(m, top_of<T, VEC>(v[i]));
            }
            if (r.counts && r.inside) {
                if (before == (int)r.target) xts[turn] = first;
                if (behind == (int)r.target) xts[turn] = last_one;
                if (owner) {
                    T own;
                    shared_value(place + at + (unsigned)ti * pitch + (unsigned)te * (unsigned)sizeof(T), own);
                    xts[turn] = widen(own);
                }
            }
            const float scale = loss_scale(m), ref = loss_offset(m);
            s = exp2_fast(fmaf(first, scale, -ref)) + exp2_fast(fmaf(last_one, scale, -ref));
            if (a.smoothing != 0.0f) {
                sum = (before >= 0 ? first : 0.0f) + (behind >= 0 ? last_one : 0.0f);
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float2 f[VEC / 2];
                    unpack<T, VEC>(v[i], f);
                    if (i < NV - 1 || last_too)
#pragma unroll
                        for (int j = 0; j < VEC / 2; ++j) sum += f[j].x + f[j].y;
                }
            }
            const float2 sc = both(scale), of = both(-ref);
            float2 acc[2] = {both(0.0f), both(0.0f)};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                unpack<T, VEC>(v[i], e[i]);
#pragma unroll
                for (int j = 0; j < VEC / 2; ++j) {
                    const float2 t = fma2(e[i][j], sc, of);
                    e[i][j] = make_float2(exp2_fast(t.x), exp2_fast(t.y));
                    acc[j & 1] = add2(acc[j & 1], e[i][j]);
                }
            }
            acc[0] = add2(acc[0], acc[1]);
            s += acc[0].x + acc[0].y;
            m = rank_own = loss_rank(m);
            if (!arrived) s = __int_as_float(0x7FC00000);
        }
        block_join(m, s, sum, a.smoothing != 0.0f, buf[turn]);
        // (behind the barrier in there nobody reads this stage any more)
        if (tid == 0 && arrived) fetch(row + (long long)kLossStages * teams, stage);
        r.m = m, r.s = s, r.sum = sum;
        if (cluster > 1) {
            namespace cg = cooperative_groups;
            auto group = cg::this_cluster();
            if (tid == 0) mine[turn][0] = r.m, mine[turn][1] = r.s, mine[turn][2] = r.sum;
            group.sync();
            for (int c = 0; c < cluster; ++c) {  // in the same order in every CTA
                const float* other = group.map_shared_rank(mine[turn], (unsigned)c);
                const float m2 = other[0], s2 = other[1], x2 = other[2];
                if (c == 0) r.m = m2, r.s = s2, r.sum = x2;
                else join(r.m, r.s, m2, s2), r.sum += x2;
            }
        }
        r.finish();
        if (!weighed) {
            w = row_weight(a, valid);
            off_all = w * a.smoothing / (float)a.vocab;
            weighed = true;
        }
        if (writes && tid == 0) write_row(a, r, row, xts[turn]);
        T* g = grad + row * a.ld_grad;
        T* gb = g + part.base() + tid * VEC;
        if (!grad) {
        } else if (r.has_gradient()) {
            const float k = r.factor(a, w), off = off_all, hit = w * (1.0f - a.smoothing);
            // from the thread's maximum to the row's, which is not below it (a thread of nothing but -inf: 0)
            const float2 k2 = both(k * lift(rank_own, r.m)), off2 = both(-off);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float2 q[VEC / 2];
#pragma unroll
                for (int j = 0; j < VEC / 2; ++j) q[j] = fma2(k2, e[i][j], off2);
                if (owner && ti == i) {
#pragma unroll
                    for (int j = 0; j < VEC / 2; ++j) {
                        if (2 * j == te) q[j].x -= hit;
                        if (2 * j + 1 == te) q[j].y -= hit;
                    }
                }
                if (i < NV - 1 || last_too) {
                    uint4 o;
                    if (sizeof(T) == 2) o = make_uint4(narrow2(q[0]), narrow2(q[1]), narrow2(q[(VEC / 2 - 1) & 2]), narrow2(q[VEC / 2 - 1]));
                    else o = make_uint4(__float_as_uint(q[0].x), __float_as_uint(q[0].y), __float_as_uint(q[1].x), __float_as_uint(q[1].y));
                    __stcs(reinterpret_cast<uint4*>(gb + i * threads * VEC), o);
                }
            }
            auto one = [&](int i) {
                const float d = fmaf(k, exp2_fast(fmaf(widen(x[i]), r.scale, -r.ref)), -off);
                g[i] = narrow<T>(i == (int)r.target ? d - hit : d);
            };
            if (before >= 0) one(before);
            if (behind >= 0) one(behind);
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < NV - 1 || last_too) __stcs(reinterpret_cast<uint4*>(gb + i * threads * VEC), make_uint4(0u, 0u, 0u, 0u));
            if (before >= 0) g[before] = narrow<T>(0.0f);
            if (behind >= 0) g[behind] = narrow<T>(0.0f);
        }
        first = first_next, last_one = last_next, its_target = target_next;
        stage = stage + 1 == kLossStages ? 0u : stage + 1;
        if (stage == 0) phase ^= 1u;
        at = stage * stage_bytes;
    }
    if (cluster > 1) cooperative_groups::this_cluster().sync();  // nobody leaves while its values are read
    if (!arrived && tid == 0)  // (a last bounded wait for what may still be on its way into this CTA's memory)
        for (int k = 0; k < kLossStages; ++k, stage = stage + 1 == kLossStages ? 0u : stage + 1, phase ^= stage == 0) bulk_wait(landed_at + stage * 8u, phase);
    add_rows(a, gridDim.x, w, valid);
}

// What autograd asks for behind the loss: the gradient times the number that arrives from above, which stays on the device.  fp32
// products, rounded once.  Bound: HBM (read once, written once: floor 161 us at 8192 x 32000 bf16; forward and backward together 352 us,
// 197 of them the loss itself).
constexpr int kUpThreads = 256, kUpVectors = 4;  // (of a thread, all on their way at once)
template <class T, int VEC>
__global__ void __launch_bounds__(kUpThreads)
loss_backward_kernel(const T* grad, const float* __restrict__ upstream, T* out, long long n) {
    const long long vectors = n / VEC, first = (long long)blockIdx.x * (kUpThreads * kUpVectors) + threadIdx.x;
    Pack<T, VEC> p[kUpVectors];
#pragma unroll
    for (int i = 0; i < kUpVectors; ++i)
        if (first + i * kUpThreads < vectors) p[i].load_stream(grad + (first + i * kUpThreads) * VEC);
    const float up = *upstream;
#pragma unroll
    for (int i = 0; i < kUpVectors; ++i) {
        if (first + i * kUpThreads >= vectors) continue;
        float f[VEC];
        p[i].get(f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] *= up;
        p[i].set(f);
        p[i].store_stream(out + (first + i * kUpThreads) * VEC);
    }
    const long long rest = vectors * VEC + (blockIdx.x ? n : threadIdx.x);
    if (rest < n) out[rest] = narrow<T>(widen(grad[rest]) * up);
}

// The row read twice: a running maximum and sum, then the gradient.

template <class T, int VEC>
__global__ void __launch_bounds__(kLossThreads)
loss_stream_kernel(const LossArgs a, const T* logits, T* grad) {
    __shared__ float buf[3][32];
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
    r.aim(a, target_of(a, row));
    const bool smoothed = a.smoothing != 0.0f;
    float m = -INFINITY, s = 0.0f;
    double logits_sum = 0.0;                    // (hundreds of terms a thread)
    float scale = kLog2e, ref = 0.0f;           // of the exponentials
    auto rise = [&](float top) {                // the maximum so far goes up to top
        if (top > m) {
            s *= lift(loss_rank(m), loss_rank(top));
            m = top;
            scale = loss_scale(top);
            ref = loss_offset(top);
        }
    };
    auto see = [&](float v) {
        s += exp2_fast(fmaf(v, scale, -ref));   // (0 for -inf; NaN and +inf end here and stay in the sum)
    };
    auto one = [&](float v) {
        rise(v);
        see(v);
        if (smoothed) logits_sum += v;
    };
    for (int i = tid; i < head; i += kLossThreads) one(widen(x[i]));
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
        if (smoothed) {
            float part = f[0];
#pragma unroll
            for (int j = 1; j < VEC; ++j) part += f[j];
            logits_sum += part;
        }
    }
    for (int i = rest + tid; i < a.vocab; i += kLossThreads) one(widen(x[i]));
    float sum = (float)logits_sum;
    m = loss_rank(m);
    const float xt = r.counts && r.inside ? widen(x[r.target]) : 0.0f;  // (read before any thread writes a gradient in its place)
    block_join(m, s, sum, true, buf);
    r.m = m, r.s = s, r.sum = sum;
    r.finish();
    int valid;
    const float w = row_weight(a, valid);
    if (tid == 0) write_row(a, r, row, xt);
    if (grad) {
        T* g = grad + row * a.ld_grad;
        const bool some = r.has_gradient();
        const float k = some ? r.factor(a, w) : 0.0f, off = w * a.smoothing / (float)a.vocab, hit = w * (1.0f - a.smoothing);
        auto of = [&](float v, int i) {
            if (!some) return 0.0f;
            const float d = fmaf(k, exp2_fast(fmaf(v, r.scale, -r.ref)), -off);
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
    add_rows(a, gridDim.x, w, valid);
}

}  // namespace

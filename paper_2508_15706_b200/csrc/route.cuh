// Router of a mixture of experts: choice, weights, counts, places in expert order, balance and z loss, and their gradient.
// Part of libsparseloco (experts.cu).
//
// Bound: launches for the sizes a layer has (8 experts x 32768 tokens are 1 MB); HBM for wide fp32 logits.  A token's logits sit in the
// registers of G lanes, 8 (up to 32) to a lane, so that one lane holds all of 8 experts; choosing is k rounds of a maximum over 64-bit keys
// (logit in order-keeping form, then the index complemented), which settles ties and NaN in one comparison.
// Places need counts of all tokens before a token.  Tokens are cut into chunks, one CTA each, whose counts per expert go to the
// workspace; a second kernel adds up the table of counts in every CTA for itself (chunks x experts integers from L2, less than a
// launch costs) and ranks its chunk's choices; a single chunk goes on in the first.  No floating atomics: sums of p and lse^2 go through the table
// too, in a fixed order.
// Measured (a graph of one small kernel replays in 2.3 us): 37 x 8 6.3 us, one CTA's chain of loads, choices, counts and places; 32768 x 8 bfloat16 8.6 us,
// the two kernels; gradients of 30011 x 128 fp32 13.5 us (33 MB: 2.4 TB/s), bound by what is done per logit; by shuffles, one choice after the other,
// 20.4.  Forward with 8 of 128 experts, 30011 tokens: 150 us, fp32 and bfloat16 alike, the 8 rounds of 64-bit maxima over 16 lanes.
#pragma once
#include "inner_common.cuh"

namespace {

constexpr int kRouteThreads = 256, kRouteWarps = kRouteThreads / 32;
constexpr int kRouteMaxExperts = 1024, kRouteMaxK = 32;

struct RouteArgs {
    const void* logits;
    void* dlogits;
    const uint8_t* mask;
    float* weights;
    int* experts;
    int* slots;
    int* counts;
    int* offsets;
    float* lse;
    float* balance;
    float* z;
    const float* dweights;
    const float* dbalance;
    const float* dz;
    int* chunk_counts;   // [chunks][E]
    float* chunk_share;  // [chunks][E], sums of p
    double* chunk_z;     // [chunks]
    long long ld, ld_d;
    int rows, E, k, chunk, chunks;  // tokens per chunk
    int renormalize, wide;          // wide: a lane's logits may be read by 16-byte accesses
};

// order-keeping form of a float; -0 as +0, NaN above +inf
__device__ __forceinline__ unsigned ordered(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const unsigned u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <class T, int V>
__device__ __forceinline__ void route_load(float (&x)[V], const T* row, int first, int E, int wide) {
    if (wide && first + V <= E) {
        Pack<T, V> p;
        p.load(row + first);
        p.get(x);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = first + i < E ? widen(row[first + i]) : -INFINITY;
    }
}

template <int G, class X>
__device__ __forceinline__ X group_sum(X x) {
#pragma unroll
    for (int o = G / 2; o; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
    return x;
}
template <int G>
__device__ __forceinline__ unsigned long long group_max(unsigned long long x) {
#pragma unroll
    for (int o = G / 2; o; o >>= 1) {
        const unsigned long long y = __shfl_xor_sync(kFullMask, x, o);
        x = y > x ? y : x;
    }
    return x;
}

// Places: one CTA per chunk.  Shared: total[E], before[E], count[warps][E].
__device__ __forceinline__ void route_place(const RouteArgs& a, int* s_int, bool behind) {
    int* total = s_int;                // [E]
    int* before = s_int + a.E;         // [E], in the chunks before this one
    int* count = s_int + 2 * a.E;      // [kRouteWarps][E]
    __shared__ int s_warp[kRouteWarps];
    __shared__ double s_sum[kRouteWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int e = tid; e < (2 + kRouteWarps) * a.E; e += kRouteThreads) s_int[e] = 0;
    __syncthreads();
    if (behind) asm volatile("griddepcontrol.wait;" ::: "memory");
    // The table of counts, added up by experts: threads side by side take neighbouring experts, teams of them every n-th chunk.
    const int across = min(a.E, kRouteThreads), teams = kRouteThreads / across, team = tid / across;
    if (team < teams)
        for (int e = tid % across; e < a.E; e += across) {
            int all = 0, own = 0;
#pragma unroll 8
            for (int c = team; c < a.chunks; c += teams) {
                const int n = __ldcg(&a.chunk_counts[(long long)c * a.E + e]);
                all += n;
                own += c < (int)blockIdx.x ? n : 0;
            }
            atomicAdd(&total[e], all);
            atomicAdd(&before[e], own);
        }
    // counts of every warp's part of the chunk
    const int begin = blockIdx.x * a.chunk, tokens = min(a.chunk, a.rows - begin);
    const int n = tokens * a.k, part = (n + kRouteThreads - 1) / kRouteThreads * 32;  // choices per warp, whole rounds of 32
    const int* ex = a.experts + (long long)begin * a.k;
    int* out = a.slots + (long long)begin * a.k;
    const int from = min(n, warp * part), to = min(n, from + part);
    for (int i = from; i < to; i += 32) {
        const int e = i + lane < to ? __ldcg(&ex[i + lane]) : -1;
        if (e >= 0) atomicAdd(&count[warp * a.E + e], 1);
    }
    __syncthreads();
    // first place of every expert: a running sum over the experts, 256 of them at a time
    int carry = 0;
    for (int e0 = 0; e0 < a.E; e0 += kRouteThreads) {
        const int e = e0 + tid, mine = e < a.E ? total[e] : 0;
        int run = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(kFullMask, run, o);
            if (lane >= o) run += y;
        }
        if (lane == 31) s_warp[warp] = run;
        __syncthreads();
        int ahead = carry, all = 0;
#pragma unroll
        for (int w = 0; w < kRouteWarps; ++w) {
            if (w < warp) ahead += s_warp[w];
            all += s_warp[w];
        }
        carry += all;
        if (e < a.E) {
            const int start = ahead + run - mine;
            int at = start + before[e];
            for (int w = 0; w < kRouteWarps; ++w) {  // a warp's count becomes its first place
                const int c = count[w * a.E + e];
                count[w * a.E + e] = at;
                at += c;
            }
            if (blockIdx.x == 0) {
                a.offsets[e] = start;
                a.counts[e] = mine;
            }
        }
        __syncthreads();
    }
    for (int i = from; i < to; i += 32) {
        const int e = i + lane < to ? __ldcg(&ex[i + lane]) : -1;
        const unsigned same = __match_any_sync(kFullMask, e);
        const int rank = __popc(same & ((1u << lane) - 1u));
        int at = 0;
        if (e >= 0) at = count[warp * a.E + e];
        __syncwarp();
        if (e >= 0 && rank == 0) count[warp * a.E + e] = at + __popc(same);
        __syncwarp();
        if (i + lane < to) out[i + lane] = e >= 0 ? at + rank : -1;
    }
    if (blockIdx.x != 0) return;
    // the losses, by the first CTA: sums over the chunks in a fixed order, 64 bits
    if (tid == 0) a.offsets[a.E] = carry;
    const double N = (double)carry / a.k;
    double s = 0.0, zz = 0.0;
    for (int e = warp; e < a.E; e += kRouteWarps) {
        double share = 0.0;
        for (int c = lane; c < a.chunks; c += 32) share += (double)__ldcg(&a.chunk_share[(long long)c * a.E + e]);
        share = warp_sum(share);
        s += share * (double)total[e];
    }
    if (warp == 0) {
        for (int c = lane; c < a.chunks; c += 32) zz += __ldcg(&a.chunk_z[c]);
        zz = warp_sum(zz);
    }
    if (lane == 0) s_sum[warp] = s;
    __syncthreads();
    if (tid == 0) {
        double b = 0.0;
        for (int w = 0; w < kRouteWarps; ++w) b += s_sum[w];
        a.balance[0] = carry ? (float)((double)a.E * b / ((double)a.k * N * N)) : 0.0f;
        a.z[0] = carry ? (float)(zz / N) : 0.0f;
    }
}
__global__ void __launch_bounds__(kRouteThreads) route_place_kernel(RouteArgs a) {
    extern __shared__ __align__(16) int s_place[];
    route_place(a, s_place, true);
}

template <class T, int G, int V>
__global__ void __launch_bounds__(kRouteThreads) route_choose_kernel(RouteArgs a) {
    constexpr int kTokens = kRouteThreads / G;  // at a time
    extern __shared__ int s_count[];            // [E], then the groups' sums of p: [kRouteWarps][E] floats
    float* s_share = reinterpret_cast<float*>(s_count + a.E);
    __shared__ double s_z[kRouteWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, member = tid % G, first = member * V;
    for (int e = tid; e < a.E; e += kRouteThreads) s_count[e] = 0;
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    float share[V];
    double z = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) share[i] = 0.0f;
    const int begin = blockIdx.x * a.chunk, end = min(a.rows, begin + a.chunk);
    // (every lane of a warp takes part in all rounds: the shuffles need them)
    for (int t0 = begin; t0 < end; t0 += kTokens) {
        const int t = t0 + tid / G;
        const bool there = t < end;
        float x[V];
        if (there) {
            route_load<T, V>(x, static_cast<const T*>(a.logits) + (long long)t * a.ld, first, a.E, a.wide);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = -INFINITY;
        }
        unsigned long long key[V], best = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            key[i] = first + i < a.E ? ((unsigned long long)ordered(x[i]) << 32) | (unsigned)~(first + i) : 0ull;
            best = key[i] > best ? key[i] : best;
        }
        best = group_max<G>(best);
        // the row's maximum from its key (a NaN stays one)
        const unsigned top_bits = (unsigned)(best >> 32);
        const float top = top_bits == 0xFFFFFFFFu ? NAN : __uint_as_float(top_bits & 0x80000000u ? top_bits & 0x7FFFFFFFu : ~top_bits);
        const bool alive = there && top != -INFINITY;
        const bool counts = alive && (!a.mask || a.mask[t]);
        float p[V], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            p[i] = alive && first + i < a.E ? expf(x[i] - top) : 0.0f;
            sum += p[i];
        }
        sum = group_sum<G>(sum);
        const float lse = alive ? top + logf(sum) : -INFINITY, inv = alive ? 1.0f / sum : 0.0f;
        if (there && member == 0) a.lse[t] = lse;
        if (counts) {
#pragma unroll
            for (int i = 0; i < V; ++i) share[i] += p[i] * inv;
            if (member == 0) z += (double)lse * (double)lse;
        }
        // k rounds: the largest key that is left; its lane drops it
        const long long at = (long long)t * a.k;
        float chosen_sum = 0.0f;
        for (int j = 0; j < a.k; ++j) {
            if (j) {
                best = 0;
#pragma unroll
                for (int i = 0; i < V; ++i) best = key[i] > best ? key[i] : best;
                best = group_max<G>(best);
            }
            const int e = (int)~(unsigned)best;
            float pe = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (key[i] == best) {
                    key[i] = 0ull;
                    pe = p[i];
                }
            pe = group_sum<G>(pe);
            chosen_sum += pe;
            if (there && member == 0) {
                a.experts[at + j] = counts ? e : -1;
                a.weights[at + j] = counts ? (a.renormalize ? pe : pe * inv) : 0.0f;
                if (counts) atomicAdd(&s_count[e], 1);
            }
        }
        if (a.renormalize && counts && member == 0)
            for (int j = 0; j < a.k; ++j) a.weights[at + j] /= chosen_sum;  // (its own writes)
    }
    // sums of p: over the warp's groups (lanes that hold the same experts), then over the warps, each in a fixed order
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int o = G; o < 32; o <<= 1) share[i] += __shfl_xor_sync(kFullMask, share[i], o);
        if (lane < G && first + i < a.E) s_share[warp * a.E + first + i] = share[i];
    }
    z = warp_sum(z);
    if (lane == 0) s_z[warp] = z;
    __syncthreads();
    for (int e = tid; e < a.E; e += kRouteThreads) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kRouteWarps; ++w) s += s_share[w * a.E + e];
        a.chunk_share[(long long)blockIdx.x * a.E + e] = s;
        a.chunk_counts[(long long)blockIdx.x * a.E + e] = s_count[e];
    }
    if (tid == 0) {
        double s = 0.0;
        for (int w = 0; w < kRouteWarps; ++w) s += s_z[w];
        a.chunk_z[blockIdx.x] = s;
    }
    if (a.chunks == 1) {  // a single chunk needs no second kernel
        __syncthreads();
        route_place(a, s_count, false);
    }
}

template <class T, int G, int V>
__global__ void __launch_bounds__(kRouteThreads) route_backward_kernel(RouteArgs a) {
    constexpr int kTokens = kRouteThreads / G;
    extern __shared__ __align__(16) float s_route[];  // every lane's V values of the chosen weights' gradients, then [E], the balance loss's derivative by p
    float* s_even = s_route + kRouteThreads * V;
    __shared__ int s_n[kRouteWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, member = tid % G, first = member * V;
    int n = 0;
    for (int e = tid; e < a.E; e += kRouteThreads) n += a.counts[e];
    n = warp_sum(n);
    if (lane == 0) s_n[warp] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < kRouteWarps; ++w) n += s_n[w];
    const double N = n > 0 ? (double)n / a.k : 1.0;
    const double per = a.dbalance ? (double)a.dbalance[0] * a.E / (a.k * N * N) : 0.0;
    const float zf = a.dz ? (float)(2.0 * (double)a.dz[0] / N) : 0.0f;
    for (int e = tid; e < a.E; e += kRouteThreads) s_even[e] = (float)(per * (double)a.counts[e]);
    __syncthreads();
    for (long long t0 = (long long)blockIdx.x * kTokens; t0 < a.rows; t0 += (long long)gridDim.x * kTokens) {
        const long long t = t0 + tid / G, at = t * a.k;
        const bool there = t < a.rows;
        float x[V];
        if (there) {
            route_load<T, V>(x, static_cast<const T*>(a.logits) + t * a.ld, first, a.E, a.wide);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = -INFINITY;
        }
        // the choices, one to a lane of the group, kMine of them to each
        constexpr int kMine = (kRouteMaxK + G - 1) / G;
        int chosen[kMine];
        float d[kMine], w[kMine];
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            const int j = m * G + member;
            const bool here = there && j < a.k;
            chosen[m] = here ? a.experts[at + j] : -1;
            d[m] = here && a.dweights ? a.dweights[at + j] : 0.0f;
            w[m] = here && a.dweights && a.renormalize ? a.weights[at + j] : 0.0f;
        }
        const float row_lse = there ? a.lse[t] : 0.0f;
        const bool counts = __shfl_sync(kFullMask, chosen[0], lane - member) >= 0;
        const float lse = counts ? row_lse : 0.0f;
        // (p from the logits again, not as exp(x - lse): beside a logit of the type's lowest value lse cannot hold its logarithm)
        float p[V], g[V], dot = 0.0f, top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) top = x[i] > top || x[i] != x[i] ? x[i] : top;
#pragma unroll
        for (int o = G / 2; o; o >>= 1) {
            const float y = __shfl_xor_sync(kFullMask, top, o);
            top = y > top || y != y ? y : top;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            p[i] = counts && first + i < a.E ? expf(x[i] - top) : 0.0f;
            sum += p[i];
        }
        sum = group_sum<G>(sum);
        const float inv = counts ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            p[i] *= inv;
            g[i] = first + i < a.E ? s_even[first + i] : 0.0f;
        }
        // what reaches the chosen logits: put in its place by the lane that holds the choice, read by the lane that holds the logit
        float extra[V];
#pragma unroll
        for (int i = 0; i < V; ++i) extra[i] = 0.0f;
        if (a.dweights) {
            float mean = 0.0f;  // of dweights under the weights
#pragma unroll
            for (int m = 0; m < kMine; ++m) mean += w[m] * d[m];
            mean = group_sum<G>(mean);
            float4* own = reinterpret_cast<float4*>(s_route + tid * V);
#pragma unroll
            for (int i = 0; i < V / 4; ++i) own[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            __syncwarp();
#pragma unroll
            for (int m = 0; m < kMine; ++m)
                if ((unsigned)chosen[m] < (unsigned)a.E) s_route[(tid - member) * V + chosen[m]] = a.renormalize ? w[m] * (d[m] - mean) : d[m];
            __syncwarp();
#pragma unroll
            for (int i = 0; i < V / 4; ++i) {
                const float4 e = own[i];
                extra[4 * i] = e.x;
                extra[4 * i + 1] = e.y;
                extra[4 * i + 2] = e.z;
                extra[4 * i + 3] = e.w;
            }
            if (!a.renormalize) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    g[i] += extra[i];
                    extra[i] = 0.0f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) dot += p[i] * g[i];
        dot = group_sum<G>(dot);
        if (!there) continue;  // (whole groups; the shuffles of a round are behind)
        const float zl = zf * lse;
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = counts ? p[i] * (g[i] - dot + zl) + extra[i] : 0.0f;
        T* row = static_cast<T*>(a.dlogits) + t * a.ld_d;
        if (a.wide && first + V <= a.E) {
            Pack<T, V> o;
            o.set(g);
            o.store(row + first);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (first + i < a.E) row[first + i] = narrow<T>(g[i]);
        }
    }
}

}  // namespace

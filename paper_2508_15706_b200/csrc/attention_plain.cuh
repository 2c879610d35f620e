// Attention in fp32 multiply-adds: fp32 heads, heads of more than 128 values, and what the tensor-core kernels hand over.
// Part of libsparseloco (attention.cu).
//
// 256 threads as 16 x 16.  A CTA owns TILE rows (queries, or keys for dk and dv) and takes the rows they meet STEP at a time, all as fp32 in
// shared memory.  A thread holds the scores of rows ty R + r against rows tx + 16 c (neighbouring threads read rows a padded pitch apart: no bank
// conflicts), and of the sums R of the own rows, 4 neighbouring values every 64.  Bound: fp32 multiply-adds, two to an instruction, fed by one shared access of
// 16 bytes for every 4 to 8 of them.  STEP is 32 for heads of 128 so that two CTAs fit an SM: one alone left most cycles without an instruction.
// Measured, gradients in fp32 without a mask: 4096 tokens, 16 heads of 128 17.4 ms (20 TFLOP/s counting 5 products, 28 with the 7 that run, of 74);
// 1501 tokens in 4 sequences, 10 heads on 5, 0.78 ms: tiles that only part of their rows see, and shared memory 59 % busy.  Causal, 4096 tokens, 16 heads of 128: forward 2.4 ms
// (29 TFLOP/s), gradients 7.8 ms (22, counting 5 products); heads of 64 1.24 and 3.7 ms.
//
// Masked scores have p = 0, which passes over finite values.  Whether all values loaded so far are finite is noted on the way into shared
// memory; once one is not, the products of steps that are not full take each row's own range: what stands in a masked row, NaN or
// infinity, never meets a factor of 0.
#pragma once
#include "attention_common.cuh"

namespace {

constexpr int kPlainThreads = 256;

__device__ __forceinline__ void plain_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// rows taken at a time by a kernel for heads of up to `dmax` values
__host__ __device__ constexpr int plain_step_of(int dmax) { return dmax == 64 ? 64 : 32; }

// rows first .. first + ROWS - 1 of a head into shared memory as fp32, zeros behind the last token and behind the head's end
template <class T, int DMAX, int ROWS>
__device__ __forceinline__ void plain_load(float* to, const void* from, AttnPlace st, int head, int first, const AttnArgs& a, int tid, volatile int* odd) {
    constexpr int P = DMAX + 4;
    const T* base = static_cast<const T*>(from) + head * st.head;
    bool fine = true;
    if (a.vec) {
#pragma unroll 8
        for (int i = tid; i < ROWS * (DMAX / 4); i += kPlainThreads) {
            const int r = i / (DMAX / 4), d = i % (DMAX / 4) * 4;
            float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (first + r < a.tokens && d < a.dim) {
                Pack<T, 4> p;
                p.load(base + (first + r) * st.token + d);
                p.get(f);
                fine = fine && isfinite(f[0]) && isfinite(f[1]) && isfinite(f[2]) && isfinite(f[3]);
            }
            *reinterpret_cast<float4*>(to + r * P + d) = make_float4(f[0], f[1], f[2], f[3]);
        }
    } else {
        for (int i = tid; i < ROWS * DMAX; i += kPlainThreads) {
            const int r = i / DMAX, d = i % DMAX;
            const float f = first + r < a.tokens && d < a.dim ? widen(base[(first + r) * st.token + d]) : 0.0f;
            fine = fine && isfinite(f);
            to[r * P + d] = f;
        }
    }
    if (!fine) *odd = 1;
}

template <class T, int DMAX, int R>
__device__ __forceinline__ void plain_store(const float (&acc)[R][DMAX / 64][4], int r, void* to, AttnPlace st, int head, int token, float by, const AttnArgs& a, int tx) {
    T* row = static_cast<T*>(to) + head * st.head + token * st.token;
#pragma unroll
    for (int c = 0; c < DMAX / 64; ++c) {
        const int d = tx * 4 + 64 * c;
        float f[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) f[x] = acc[r][c][x] * by;
        if (a.vec) {
            if (d < a.dim) {
                Pack<T, 4> p;
                p.set(f);
                p.store(row + d);
            }
        } else {
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (d + x < a.dim) row[d + x] = narrow<T>(f[x]);
        }
    }
}
// the same unscaled, as a part
template <int DMAX, int R>
__device__ __forceinline__ void plain_store_part(const float (&acc)[R][DMAX / 64][4], int r, float* row, const AttnArgs& a, int tx) {
#pragma unroll
    for (int c = 0; c < DMAX / 64; ++c) {
        const int d = tx * 4 + 64 * c;
        if (d < a.width) *reinterpret_cast<float4*>(row + d) = make_float4(acc[r][c][0], acc[r][c][1], acc[r][c][2], acc[r][c][3]);
    }
}

// scores of rows ty R + r (of x) against rows tx + 16 c (of y); even and odd values' products are summed apart, two to an instruction
template <int DMAX, int R, int C>
__device__ __forceinline__ void plain_scores(float (&s)[R][C], const float* x, const float* y, int tx, int ty, int dim) {
    constexpr int P = DMAX + 4;
    float2 t[R][C];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) t[r][c] = make_float2(0.0f, 0.0f);
#pragma unroll 4
    for (int d = 0; d < dim; d += 4) {
        float4 u[R], w[C];
#pragma unroll
        for (int r = 0; r < R; ++r) u[r] = *reinterpret_cast<const float4*>(x + (ty * R + r) * P + d);
#pragma unroll
        for (int c = 0; c < C; ++c) w[c] = *reinterpret_cast<const float4*>(y + (tx + 16 * c) * P + d);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < C; ++c) {
                t[r][c] = fma2(make_float2(u[r].x, u[r].y), make_float2(w[c].x, w[c].y), t[r][c]);
                t[r][c] = fma2(make_float2(u[r].z, u[r].w), make_float2(w[c].z, w[c].w), t[r][c]);
            }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) s[r][c] = t[r][c].x + t[r][c].y;
}

template <int R, int C>
__device__ __forceinline__ void plain_add(float (&acc)[R][C][4], int r, float f, const float4 (&w)[C]) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const float2 lo = fma2(both(f), make_float2(w[c].x, w[c].y), make_float2(acc[r][c][0], acc[r][c][1]));
        const float2 hi = fma2(both(f), make_float2(w[c].z, w[c].w), make_float2(acc[r][c][2], acc[r][c][3]));
        acc[r][c][0] = lo.x;
        acc[r][c][1] = lo.y;
        acc[r][c][2] = hi.x;
        acc[r][c][3] = hi.y;
    }
}

// acc[r] += sum_n f(ty R + r, n) y[n] over STEP rows of y, tokens n0 ...  f is [row][n] in shared memory, or (DOWN) [n][row], a padded pitch apart.  With
// `apart` only the tokens of the row's range.
template <int DMAX, int R, int STEP, bool DOWN>
__device__ __forceinline__ void plain_product(float (&acc)[R][DMAX / 64][4], const float* f, const float* y, int tx, int ty, bool apart, const int2* range, int n0) {
    constexpr int P = DMAX + 4, kScore = (DOWN ? R * 16 : STEP) + 4, C = DMAX / 64;
    static_assert(R == 4 || R == 2, "rows of a thread as one access");
    if (!apart) {
        constexpr int N = DOWN ? 1 : R;  // n at a time: as many as one access of f brings
        typedef typename RawVec<R * 4>::type Raw;
#pragma unroll 4
        for (int n = 0; n < STEP; n += N) {
            float g[N][R];
            if (DOWN) {
                const Raw v = *reinterpret_cast<const Raw*>(f + n * kScore + ty * R);
#pragma unroll
                for (int r = 0; r < R; ++r) g[0][r] = __uint_as_float(reinterpret_cast<const unsigned*>(&v)[r]);
            } else {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const Raw v = *reinterpret_cast<const Raw*>(f + (ty * R + r) * kScore + n);
#pragma unroll
                    for (int x = 0; x < N; ++x) g[x][r] = __uint_as_float(reinterpret_cast<const unsigned*>(&v)[x]);
                }
            }
#pragma unroll
            for (int x = 0; x < N; ++x) {
                float4 w[C];
#pragma unroll
                for (int c = 0; c < C; ++c) w[c] = *reinterpret_cast<const float4*>(y + (n + x) * P + tx * 4 + 64 * c);
#pragma unroll
                for (int r = 0; r < R; ++r) plain_add(acc, r, g[x][r], w);
            }
        }
        return;
    }
#pragma unroll 1
    for (int n = 0; n < STEP; ++n) {
        float4 w[C];
#pragma unroll
        for (int c = 0; c < C; ++c) w[c] = *reinterpret_cast<const float4*>(y + n * P + tx * 4 + 64 * c);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int2 see = range[ty * R + r];
            if (n0 + n >= see.x && n0 + n < see.y) plain_add(acc, r, f[DOWN ? n * kScore + ty * R + r : (ty * R + r) * kScore + n], w);
        }
    }
}

template <class X>
__device__ __forceinline__ X lanes16_sum(X x) {
#pragma unroll
    for (int o = 8; o; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
    return x;
}

// The ranges of a tile's rows into shared memory, and over all of them: the first and the last token seen, and the largest
// beginning and smallest end (steps of tokens between those are full for every row).  All threads get the four numbers.  The note of values that
// are not finite is cleared between the two barriers: a thread still in the last round of a tile before this one reads that tile's.
template <int TILE, bool KEYS>
__device__ __forceinline__ int4 plain_ranges(const AttnArgs& a, int first, int2* range, volatile int* odd, int tid) {
    plain_sync();
    if (tid == 0) *odd = 0;
    if (tid < TILE) range[tid] = KEYS ? keys_of(a, first + tid) : queries_of(a, first + tid);
    plain_sync();
    int4 all = make_int4(0x7FFFFFFF, 0, 0, 0x7FFFFFFF);
    for (int r = 0; r < TILE; ++r) {
        const int2 x = range[r];
        if (x.y > 0) {
            all.x = min(all.x, x.x);
            all.y = max(all.y, x.y);
        }
        all.z = max(all.z, x.y > 0 ? x.x : 0x7FFFFFFF);  // (a row that sees nothing makes no step full)
        all.w = min(all.w, x.y);
    }
    return all;
}

// floats of shared memory: `own` and `met` matrices, one of scores, ranges, statistics, the note of values that are not finite
constexpr int plain_floats(int dmax, int tile, int own, int met) {
    return (own * tile + met * plain_step_of(dmax)) * (dmax + 4) + (tile + 4) * (plain_step_of(dmax) + 4) + 4 * tile + 2 * plain_step_of(dmax) + 4;
}

template <class T, int R, int C>
__device__ __forceinline__ void plain_zero(T (&acc)[R][C][4]) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int x = 0; x < 4; ++x) acc[r][c][x] = 0.0f;
}

// out and lse of the queries q0 .. of one head.  `smem`: plain_floats(DMAX, TILE, 1, 2) floats.
template <class T, int DMAX, int TILE>
__device__ __noinline__ void plain_forward_tile(const AttnArgs& a, int q0, int head, float* smem, int tid) {
    constexpr int STEP = plain_step_of(DMAX), R = TILE / 16, C = STEP / 16, P = DMAX + 4, kScore = STEP + 4;
    float *sq = smem, *sk = sq + TILE * P, *sv = sk + STEP * P, *sp = sv + STEP * P;
    int2* range = reinterpret_cast<int2*>(sp + TILE * kScore);
    volatile int* odd = reinterpret_cast<int*>(range + TILE);
    int unused = 0;  // (q and k meet masked scores only before they are masked)
    const int tx = tid & 15, ty = tid >> 4;
    const int4 all = plain_ranges<TILE, true>(a, q0, range, odd, tid);
    plain_load<T, DMAX, TILE>(sq, a.q, a.sq, head, q0, a, tid, &unused);
    float acc[R][DMAX / 64][4], top[R], sum[R];
    plain_zero(acc);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        top[r] = -INFINITY;
        sum[r] = 0.0f;
    }
    for (int k0 = all.x / STEP * STEP; k0 < all.y; k0 += STEP) {
        plain_sync();  // (the last step's products are done)
        plain_load<T, DMAX, STEP>(sk, a.k, a.sk, head / a.group, k0, a, tid, &unused);
        plain_load<T, DMAX, STEP>(sv, a.v, a.sv, head / a.group, k0, a, tid, odd);
        plain_sync();
        const bool some = k0 < all.z || k0 + STEP > all.w;
        float s[R][C];
        plain_scores<DMAX, R, C>(s, sq, sk, tx, ty, a.dim);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int2 see = range[ty * R + r];
            float best = -INFINITY;
            bool in[C];
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int j = k0 + tx + 16 * c;
                in[c] = !some || (j >= see.x && j < see.y);
                if (in[c]) best = s[r][c] > best || s[r][c] != s[r][c] ? s[r][c] : best;
            }
#pragma unroll
            for (int o = 8; o; o >>= 1) {
                const float y = __shfl_xor_sync(kFullMask, best, o);
                best = y > best || y != y ? y : best;
            }
            const float next = best > top[r] || best != best ? best : top[r];  // (NaN stays)
            const float old = top[r] == next || sum[r] == 0.0f ? 1.0f : exp2f((top[r] - next) * a.c);
            const float base = next == -INFINITY ? 0.0f : next;  // (nothing but scores of -inf so far: weights of 0)
            float part = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const float p = in[c] ? exp2f((s[r][c] - base) * a.c) : 0.0f;
                sp[(ty * R + r) * kScore + tx + 16 * c] = p;
                part += p;
            }
            sum[r] = sum[r] * old + lanes16_sum(part);
            top[r] = next;
#pragma unroll
            for (int c = 0; c < DMAX / 64; ++c)
#pragma unroll
                for (int x = 0; x < 4; ++x) acc[r][c][x] *= old;
        }
        plain_sync();
        plain_product<DMAX, R, STEP, false>(acc, sp, sv, tx, ty, some && *odd, range, k0);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = q0 + ty * R + r;
        const bool in = range[ty * R + r].y > 0;
        if (i >= a.tokens || (!in && !a.fill)) continue;
        plain_store<T, DMAX, R>(acc, r, a.o, a.so, head, i, in ? 1.0f / sum[r] : 0.0f, a, tx);
        if (tx == 0) a.lse[(long long)head * a.tokens + i] = !in ? -INFINITY : top[r] == INFINITY ? INFINITY : top[r] * a.scale + logf(sum[r]);  // (the sum is NaN beside a score of inf)
    }
}

// p of queries against keys, kept in registers: rows are queries (ty R + r), columns keys (tx + 16 c); KEYS is which of the two the ranges are of.
// Masked ones are -0, which no exponential is, so that plain_ds knows them.
template <int R, int C, bool KEYS>
__device__ __forceinline__ void plain_p(const AttnArgs& a, float (&p)[R][C], const int2* range, const float* lse, int q0, int k0, bool some, int tx, int ty) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = ty * R + r, i = q0 + row;
        const float l = lse[row];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = tx + 16 * c, j = k0 + col;
            const int2 see = KEYS ? range[row] : range[col];
            const bool in = !some || (KEYS ? j >= see.x && j < see.y : i >= see.x && i < see.y);
            p[r][c] = in ? exp2f(fmaf(p[r][c], a.c, l)) : -0.0f;
        }
    }
}
// ds = p (dp - delta); 0 where masked, whatever dp.  (Not wherever p is 0: a weight that vanishes passes a NaN on all the same.)
template <int R, int C>
__device__ __forceinline__ void plain_ds(float (&dp)[R][C], const float (&p)[R][C], const float* delta, int ty) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) dp[r][c] = __float_as_uint(p[r][c]) == 0x80000000u ? 0.0f : p[r][c] * (dp[r][c] + delta[ty * R + r]);
}
template <int R, int C>
__device__ __forceinline__ void plain_keep(float* to, const float (&x)[R][C], int pitch, int tx, int ty) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) to[(ty * R + r) * pitch + tx + 16 * c] = x[r][c];
}

template <int ROWS>
__device__ __forceinline__ void plain_stats(float* lse, float* delta, const AttnArgs& a, int head, int q0, int tid) {
    if (tid < ROWS) {
        const long long at = (long long)head * a.pitch + q0 + tid;  // (padded to whole tiles)
        lse[tid] = __ldcg(&a.nlse2[at]);  // (from L2, for the kernels that begin before the one that wrote them is waited for)
        delta[tid] = __ldcg(&a.ndelta[at]);
    }
}

// dk and dv of the keys k0 .. of one key/value head, or of one part of their queries.  `smem`: plain_floats(DMAX, TILE, 2, 2) floats.  The rounds are the
// steps of queries from `from.x` on, from.y of them to every head; rounds.x .. rounds.y - 1 of them are taken (from.y < 0: found here, the
// part's share).
template <class T, int DMAX, int TILE>
__device__ __noinline__ void plain_dkv_tile(const AttnArgs& a, int k0, int kv, int part, int2 from, int2 rounds, float* smem, int tid) {
    constexpr int STEP = plain_step_of(DMAX), R = TILE / 16, RQ = STEP / 16, P = DMAX + 4, kScore = TILE + 4;
    float *sk = smem, *sv = sk + TILE * P, *sq = sv + TILE * P, *sdo = sq + STEP * P, *sp = sdo + STEP * P;
    int2* range = reinterpret_cast<int2*>(sp + STEP * kScore);
    float *lse = reinterpret_cast<float*>(range + TILE), *delta = lse + STEP;
    volatile int* odd = reinterpret_cast<int*>(delta + STEP);
    int unused = 0;
    const int tx = tid & 15, ty = tid >> 4;
    const int4 all = plain_ranges<TILE, false>(a, k0, range, odd, tid);
    plain_load<T, DMAX, TILE>(sk, a.k, a.sk, kv, k0, a, tid, &unused);
    plain_load<T, DMAX, TILE>(sv, a.v, a.sv, kv, k0, a, tid, &unused);
    float gk[R][DMAX / 64][4], gv[R][DMAX / 64][4];
    plain_zero(gk);
    plain_zero(gv);
    if (from.y < 0) {
        from = all.y > 0 ? make_int2(all.x / STEP, (all.y + STEP - 1) / STEP - all.x / STEP) : make_int2(0, 0);
        rounds = share_of(from.y * a.group, part, a.parts_kv);
    }
    for (int n = rounds.x; n < rounds.y; ++n) {
        const int head = kv * a.group + n / from.y, q0 = (from.x + n % from.y) * STEP;
        plain_sync();
        plain_load<T, DMAX, STEP>(sq, a.q, a.sq, head, q0, a, tid, odd);
        plain_load<T, DMAX, STEP>(sdo, a.dout, a.sdo, head, q0, a, tid, odd);
        plain_stats<STEP>(lse, delta, a, head, q0, tid);
        plain_sync();
        const bool some = q0 < all.z || q0 + STEP > all.w, apart = some && *odd;
        float p[RQ][R], ds[RQ][R];
        plain_scores<DMAX, RQ, R>(p, sq, sk, tx, ty, a.dim);
        plain_p<RQ, R, false>(a, p, range, lse, q0, k0, some, tx, ty);
        plain_keep(sp, p, kScore, tx, ty);
        plain_scores<DMAX, RQ, R>(ds, sdo, sv, tx, ty, a.dim);
        plain_ds(ds, p, delta, ty);
        plain_sync();
        plain_product<DMAX, R, STEP, true>(gv, sp, sdo, tx, ty, apart, range, q0);
        plain_sync();
        plain_keep(sp, ds, kScore, tx, ty);
        plain_sync();
        plain_product<DMAX, R, STEP, true>(gk, sp, sq, tx, ty, apart, range, q0);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = k0 + ty * R + r;
        const bool in = range[ty * R + r].y > 0;
        if (j >= a.tokens || (!in && !a.fill)) continue;
        if (a.parts_kv > 1) {
            plain_store_part<DMAX, R>(gk, r, part_row(a.part_dk, part, a.kv_heads, kv, j, a), a, tx);
            plain_store_part<DMAX, R>(gv, r, part_row(a.part_dv, part, a.kv_heads, kv, j, a), a, tx);
            continue;
        }
        plain_store<T, DMAX, R>(gk, r, a.dk, a.sdk, kv, j, a.scale, a, tx);
        plain_store<T, DMAX, R>(gv, r, a.dv, a.sdv, kv, j, 1.0f, a, tx);
    }
}

// dq of the queries q0 .. of one head, or of one part of their keys: the steps rounds.x .. rounds.y - 1 (rounds.y < 0: found here).  `smem` as for dk
// and dv.
template <class T, int DMAX, int TILE>
__device__ __noinline__ void plain_dq_tile(const AttnArgs& a, int q0, int head, int part, int2 rounds, float* smem, int tid) {
    constexpr int STEP = plain_step_of(DMAX), R = TILE / 16, C = STEP / 16, P = DMAX + 4, kScore = STEP + 4;
    float *sq = smem, *sdo = sq + TILE * P, *sk = sdo + TILE * P, *sv = sk + STEP * P, *sds = sv + STEP * P;
    int2* range = reinterpret_cast<int2*>(sds + TILE * kScore);
    float *lse = reinterpret_cast<float*>(range + TILE), *delta = lse + TILE;
    volatile int* odd = reinterpret_cast<int*>(delta + TILE);
    int unused = 0;
    const int tx = tid & 15, ty = tid >> 4;
    const int4 all = plain_ranges<TILE, true>(a, q0, range, odd, tid);
    plain_load<T, DMAX, TILE>(sq, a.q, a.sq, head, q0, a, tid, &unused);
    plain_load<T, DMAX, TILE>(sdo, a.dout, a.sdo, head, q0, a, tid, &unused);
    plain_stats<TILE>(lse, delta, a, head, q0, tid);
    float g[R][DMAX / 64][4];
    plain_zero(g);
    if (rounds.y < 0) {
        const int first = all.y > 0 ? all.x / STEP : 0;
        rounds = share_of((all.y + STEP - 1) / STEP - first, part, a.parts_q);
        rounds.x += first;
        rounds.y += first;
    }
    for (int k0 = rounds.x * STEP; k0 < rounds.y * STEP; k0 += STEP) {
        plain_sync();
        plain_load<T, DMAX, STEP>(sk, a.k, a.sk, head / a.group, k0, a, tid, odd);
        plain_load<T, DMAX, STEP>(sv, a.v, a.sv, head / a.group, k0, a, tid, &unused);
        plain_sync();
        const bool some = k0 < all.z || k0 + STEP > all.w;
        float p[R][C], ds[R][C];
        plain_scores<DMAX, R, C>(p, sq, sk, tx, ty, a.dim);
        plain_p<R, C, true>(a, p, range, lse, q0, k0, some, tx, ty);
        plain_scores<DMAX, R, C>(ds, sdo, sv, tx, ty, a.dim);
        plain_ds(ds, p, delta, ty);
        plain_keep(sds, ds, kScore, tx, ty);
        plain_sync();
        plain_product<DMAX, R, STEP, false>(g, sds, sk, tx, ty, some && *odd, range, k0);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = q0 + ty * R + r;
        const bool in = range[ty * R + r].y > 0;
        if (i >= a.tokens || (!in && !a.fill)) continue;
        if (a.parts_q > 1) plain_store_part<DMAX, R>(g, r, part_row(a.part_dq, part, a.q_heads, head, i, a), a, tx);
        else plain_store<T, DMAX, R>(g, r, a.dq, a.sdq, head, i, a.scale, a, tx);
    }
}

// CTA x: tile x / heads, head x % heads; the tiles with the most to do first (the last queries, the first keys of a causal sequence).
template <class T, int DMAX, int TILE>
__global__ void __launch_bounds__(kPlainThreads, 2) plain_forward_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ __align__(16) float plain_smem[];
    const int tiles = (a.tokens + TILE - 1) / TILE, x = blockIdx.x;
    plain_forward_tile<T, DMAX, TILE>(a, (tiles - 1 - x / a.q_heads) * TILE, x % a.q_heads, plain_smem, threadIdx.x);
}
template <class T, int DMAX, int TILE>
__global__ void __launch_bounds__(kPlainThreads, 2) plain_dkv_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ __align__(16) float plain_smem[];
    plain_dkv_tile<T, DMAX, TILE>(a, (int)(blockIdx.x / a.kv_heads) * TILE, blockIdx.x % a.kv_heads, blockIdx.y, make_int2(0, -1), make_int2(0, 0), plain_smem, threadIdx.x);
}
template <class T, int DMAX, int TILE>
__global__ void __launch_bounds__(kPlainThreads, 2) plain_dq_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ __align__(16) float plain_smem[];
    const int tiles = (a.tokens + TILE - 1) / TILE, x = blockIdx.x;
    plain_dq_tile<T, DMAX, TILE>(a, (tiles - 1 - x / a.q_heads) * TILE, x % a.q_heads, blockIdx.y, make_int2(0, -1), plain_smem, threadIdx.x);
}

// The parts of one gradient added up in order: 4 values to a thread.
template <class T>
__global__ void __launch_bounds__(kPlainThreads) attention_join_kernel(const __grid_constant__ AttnArgs a, const float* from, void* to, AttnPlace st, int heads, int parts, float by) {
    const int per_row = a.width / 4;
    const long long n = (long long)a.tokens * heads * per_row, apart = (long long)heads * a.tokens * a.width;
    for (long long x = (long long)blockIdx.x * kPlainThreads + threadIdx.x; x < n; x += (long long)gridDim.x * kPlainThreads) {
        const int d = (int)(x % per_row) * 4;
        const long long row = x / per_row;
        const int token = (int)(row % a.tokens), head = (int)(row / a.tokens);
        const bool in = sequence_of(a, token).y > 0;
        if ((!in && !a.fill) || d >= a.dim) continue;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (in)
            for (int p = 0; p < parts; ++p) {
                const float4 v = __ldcs(reinterpret_cast<const float4*>(from + p * apart + row * a.width + d));
                sum.x += v.x;
                sum.y += v.y;
                sum.z += v.z;
                sum.w += v.w;
            }
        T* out = static_cast<T*>(to) + head * st.head + token * st.token + d;
        const float f[4] = {sum.x * by, sum.y * by, sum.z * by, sum.w * by};
        if (a.vec) {
            Pack<T, 4> o;
            o.set(f);
            o.store(out);
        } else {
#pragma unroll
            for (int y = 0; y < 4; ++y)
                if (d + y < a.dim) out[y] = narrow<T>(f[y]);
        }
    }
}

// -lse / ln 2 and -delta of every query, delta = sum do o; zeros for tokens outside every sequence and behind the last one.  16 lanes take a token's head, 8 values to a lane and
// turn, as 16-byte accesses where everything lies on such boundaries.  Bound: HBM (o and do once); 4 tokens a group of lanes, loads first, keep
// enough of them in flight.
constexpr int kStatTokens = 4;
template <class T, int VEC>
__global__ void __launch_bounds__(kPlainThreads) attention_stats_kernel(const __grid_constant__ AttnArgs a) {
    const int lane = threadIdx.x & 15, h = blockIdx.y;
    const long long t0 = ((long long)blockIdx.x * (kPlainThreads / 16) + (threadIdx.x >> 4)) * kStatTokens;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (the next kernel waits for what it needs of this one)
    const int2 live = live_tokens(a);
    if (t0 >= a.pitch) return;  // (whole warps or their halves: pitch is a multiple of 8 tokens)
    float s[kStatTokens];
#pragma unroll
    for (int x = 0; x < kStatTokens; ++x) s[x] = 0.0f;
    const T* o = static_cast<const T*>(a.o_in) + h * a.so.head;
    const T* d = static_cast<const T*>(a.dout) + h * a.sdo.head;
    for (int i = lane * VEC; i < a.dim; i += 16 * VEC) {
        Pack<T, VEC> u[kStatTokens], w[kStatTokens];
#pragma unroll
        for (int x = 0; x < kStatTokens; ++x)
            if (t0 + x < a.tokens) {
                u[x].load(o + (t0 + x) * a.so.token + i);
                w[x].load(d + (t0 + x) * a.sdo.token + i);
            }
#pragma unroll
        for (int x = 0; x < kStatTokens; ++x)
            if (t0 + x < a.tokens) {
                float f[VEC], g[VEC];
                u[x].get(f);
                w[x].get(g);
#pragma unroll
                for (int y = 0; y < VEC; ++y) s[x] = fmaf(f[y], g[y], s[x]);
            }
    }
#pragma unroll
    for (int x = 0; x < kStatTokens; ++x) s[x] = lanes16_sum(s[x]);
    if (lane < kStatTokens) {
        const long long t = t0 + lane;
        float mine = s[0];
#pragma unroll
        for (int x = 1; x < kStatTokens; ++x) mine = lane == x ? s[x] : mine;
        const bool in = t >= live.x && t < live.y;
        a.nlse2[h * a.pitch + t] = in ? -a.lse[(long long)h * a.tokens + t] * kLog2e : 0.0f;
        a.ndelta[h * a.pitch + t] = in ? -mine : 0.0f;
    }
}

}  // namespace

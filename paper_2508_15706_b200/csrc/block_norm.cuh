// Residual update and norms around a block, forward and backward, row by row.  Part of libsparseloco (block_norm.cu).
//
// Bound: HBM.  Forward reads x and branch and writes y and h; backward reads dy, dh, y, branch and writes dx, dbranch:
// every matrix once.  A row lives in the registers of its threads between its sums and its outputs (a warp for narrow
// rows, a CTA for wide ones), so a row is fetched once and in-place outputs are safe.  CTAs stay and walk over rows: a thread
// keeps its columns, so weights and column sums stay in its registers too, and the next row's loads are under way while the
// present one is reduced.
#pragma once
#include "inner_common.cuh"

namespace {

// Not tuned: rows wider than the team kernels' shared memory allows in the backward pass (from 4104 columns in fp32, 8200 in bfloat16),
// and rows of many single values a thread: the general backward kernels keep 32 columns of six arrays a thread and spill 1700 to 3900 bytes.
// The one-warp backward teams of up to 512 columns spill 90 to 720 bytes.

constexpr int kNormMaxCols = 16384;
constexpr int kNormMaxThreads = 512;
constexpr int kNormWarpRows = 8;   // rows (warps) of a CTA where a warp takes a row
// registers of a thread, by its columns and the launch bounds below (1024, 640, 512 threads): what decides how many CTAs are resident
inline int norm_regs(int columns, bool backward) { return columns <= 8 ? (backward ? 96 : 64) : columns <= 16 && !backward ? 96 : 128; }

struct NormArgs {
    long long rows;
    int cols;
    int gate_kind;
    float alpha, eps, inv_cols;
    long long ld_x, ld_branch, ld_gate, ld_y, ld_h, ld_dy, ld_dh;
    const void *x, *branch, *branch_weight, *gate, *weight;
    void *y, *h;
    float *branch_rstd, *rstd;
    // backward: x = the forward pass's y
    const void *dy, *dh;
    void *dx, *dbranch, *dgate;
    int stages;   // rows in a CTA's ring
    float* part;  // [CTAs][2][cols] column sums: of dh yhat, and of alpha dx bhat (times a row or element gate)
};

// Sum of K (1 or 3) values over the threads of a row, the same in all of them: lanes, then (rows wider than a warp) up to 16 warps
// through `buf` (K * 16 floats; those of absent warps are 0).  `buf` must not be written again before every thread has read it:
// callers alternate between two.
template <int K>
__device__ __forceinline__ void row_sums(float (&s)[K], float* buf) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (K == 1 || blockDim.x <= 32) {
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] = warp_sum(s[k]);
        if (blockDim.x <= 32) return;
        if (lane == 0) buf[warp] = s[0];
    } else {
        // three sums at once: with every halving of the lanes that share a value, each lane keeps half of the values
        const bool high = lane & 16, odd = lane & 8;
        const float p = (high ? s[K - 1] : s[0]) + __shfl_xor_sync(kFullMask, high ? s[0] : s[K - 1], 16);
        const float q = (high ? 0.0f : s[K / 2]) + __shfl_xor_sync(kFullMask, high ? s[K / 2] : 0.0f, 16);
        float v = (odd ? q : p) + __shfl_xor_sync(kFullMask, odd ? p : q, 8);
        v += __shfl_xor_sync(kFullMask, v, 4);
        v += __shfl_xor_sync(kFullMask, v, 2);
        v += __shfl_xor_sync(kFullMask, v, 1);
        if ((lane & 7) == 0 && lane != 24) buf[(high ? 2 : odd ? 1 : 0) * 16 + warp] = v;
    }
    __syncthreads();
    const int mask = blockDim.x > 256 ? 15 : blockDim.x > 128 ? 7 : blockDim.x > 64 ? 3 : 1;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        s[k] = buf[k * 16 + (lane & mask)];
        if (mask > 7) s[k] += __shfl_xor_sync(kFullMask, s[k], 8);
        if (mask > 3) s[k] += __shfl_xor_sync(kFullMask, s[k], 4);
        if (mask > 1) s[k] += __shfl_xor_sync(kFullMask, s[k], 2);
        s[k] += __shfl_xor_sync(kFullMask, s[k], 1);
    }
}
__device__ __forceinline__ void clear_sums(float* buf, int n) {
    if (blockDim.x <= 32) return;
    for (int i = threadIdx.x; i < n; i += blockDim.x) buf[i] = 0.0f;
    __syncthreads();
}

__device__ __forceinline__ float reciprocal_root(float x) { return rsqrtf(x); }  // 2 ulp

// A thread's columns: `pieces` of at most NV pieces of VEC columns, piece i from column (i * blockDim.x + threadIdx.x) * VEC on.
template <int VEC>
__device__ __forceinline__ int norm_column(int i) { return (i * (int)blockDim.x + (int)threadIdx.x) * VEC; }
template <int VEC, int NV>
__device__ __forceinline__ int norm_pieces(int cols) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) n += norm_column<VEC>(i) < cols;
    return n;
}

__device__ __forceinline__ void copy_wait(int behind) {  // all but the `behind` last groups have landed, for this thread
    if (behind == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (behind == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 3;" ::: "memory");
}
// One matrix as a thread sees it.  RING: a ring of rows in shared memory that the thread fills for itself, asynchronously and rows
// ahead (a piece is read by the thread that copied it, so nothing is waited for but the copy); places of absent matrices and of
// columns beyond the row's end are zeroed once.  Else (many columns per thread): global memory.
template <class T, int VEC, int NV, bool RING>
struct NormMatrix {
    typedef Pack<T, VEC> Piece;
    static constexpr bool kLate = Piece::kBytes < 4;  // too small for an asynchronous copy: in registers for a row, then into the ring
    const T* row;    // the thread's first column in the row to be copied (RING) or used next; null: absent
    long long step;  // elements from one of the CTA's rows to the next
    unsigned place;  // shared address of its first piece in the ring's first row
    unsigned short held[kLate ? NV : 1];
    __device__ __forceinline__ NormMatrix(const void* base, long long ld, long long first, long long stride, const char* ring, int array) {
        row = base ? static_cast<const T*>(base) + first * ld + norm_column<VEC>(0) : nullptr;
        step = base ? stride * ld : 0;
        place = (unsigned)__cvta_generic_to_shared(ring) + (unsigned)((array * NV * blockDim.x * blockDim.y + threadIdx.y * blockDim.x + threadIdx.x) * sizeof(Piece));
    }
    static __device__ __forceinline__ int offset(int i) { return i * (int)blockDim.x * VEC; }
    static __device__ __forceinline__ unsigned pitch(int i) { return (unsigned)i * (unsigned)(blockDim.x * blockDim.y * sizeof(Piece)); }
    __device__ __forceinline__ void clear(int stages, unsigned stage_bytes, int pieces) const {
        for (int s = 0; s < stages; ++s)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (!row || i >= pieces)
#pragma unroll
                    for (int j = 0; j < VEC * (int)sizeof(T); j += 2)
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(place + (unsigned)s * stage_bytes + pitch(i) + (unsigned)j), "h"((unsigned short)0) : "memory");
    }
    // the next row on its way to stage_at (kLate: into `held`, which settle() then puts there)
    __device__ __forceinline__ void fetch(unsigned stage_at, int pieces) {
        if (!row) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i < pieces) {
                if constexpr (kLate) held[i] = *reinterpret_cast<const unsigned short*>(row + offset(i));
                else copy_async<Piece::kBytes>(place + stage_at + pitch(i), row + offset(i));
            }
        }
        row += step;
    }
    __device__ __forceinline__ void settle(unsigned held_at, int pieces) const {
        if constexpr (kLate) {
            if (!row) return;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < pieces) asm volatile("st.shared.u16 [%0], %1;" ::"r"(place + held_at + pitch(i)), "h"(held[i]) : "memory");
        }
    }
    // all of the thread's values as pairs, 0 beyond the row's end or without a matrix
    __device__ __forceinline__ void get(unsigned stage_at, int pieces, float2 (&f)[NV * VEC / 2]) const {
        float g[NV * VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Piece t;
            if constexpr (RING) {
                shared_load<Piece::kBytes>(place + stage_at + pitch(i), &t);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) t.v[j] = narrow<T>(0.0f);
                if (row && i < pieces) t.load(row + offset(i));
            }
            float x[VEC];
            t.get(x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) g[i * VEC + j] = x[j];
        }
#pragma unroll
        for (int i = 0; i < NV * VEC / 2; ++i) f[i] = make_float2(g[2 * i], g[2 * i + 1]);
    }
    __device__ __forceinline__ void next() {
        if (!RING) row += step;
    }
};

// A row of an output, by the same pieces.
template <class T, int VEC, int NV>
__device__ __forceinline__ void norm_store(T* row, int pieces, const float2 (&f)[NV * VEC / 2]) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i < pieces) {
            float x[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[j] = (i * VEC + j) % 2 ? f[(i * VEC + j) / 2].y : f[(i * VEC + j) / 2].x;
            Pack<T, VEC> t;
            t.set(x);
            t.store(row + i * (int)blockDim.x * VEC);
        }
    }
}

// Weights of a thread's columns (times those of `times`), 1 where there are none.
template <class W, int VEC, int NV>
__device__ __forceinline__ void norm_weights(const void* w, const void* times, int pieces, float2 (&f)[NV * VEC / 2]) {
    float g[NV * VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) g[i * VEC + j] = 1.0f;
        if (i < pieces) {
            Pack<W, VEC> t;
            if (w) {
                t.load(static_cast<const W*>(w) + norm_column<VEC>(i));
#pragma unroll
                for (int j = 0; j < VEC; ++j) g[i * VEC + j] = widen(t.v[j]);
            }
            if (times) {
                t.load(static_cast<const W*>(times) + norm_column<VEC>(i));
#pragma unroll
                for (int j = 0; j < VEC; ++j) g[i * VEC + j] *= widen(t.v[j]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NV * VEC / 2; ++i) f[i] = make_float2(g[2 * i], g[2 * i + 1]);
}

// Few columns per thread: their weights stay in registers and rows come through the ring.
template <int VEC, int NV>
constexpr bool kNormFew = NV * VEC <= 16;
template <int VEC, int NV>
constexpr bool kNormFewBackward = NV * VEC <= 8;

// T: activations, W: weights; VEC values per access, NV accesses per thread: blockDim.x * VEC * NV >= cols; FULL: a gate per element.
// blockDim.y rows per CTA, more than one only where blockDim.x is a warp.
template <class T, class W, int VEC, int NV, bool FULL>
__global__ void __launch_bounds__(NV* VEC <= 8 ? 1024 : NV * VEC <= 16 ? 640 : kNormMaxThreads)
norm_forward_kernel(const NormArgs a) {
    constexpr bool kFew = kNormFew<VEC, NV>;
    constexpr int P = NV * VEC / 2;
    constexpr bool kLate = VEC * sizeof(T) < 4;
    extern __shared__ __align__(16) char ring[];
    __shared__ float sums[2][16];
    clear_sums(sums[0], 32);
    const long long stride = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool normed = a.branch_weight != nullptr, has_branch = a.branch != nullptr;
    const void* column_gate = a.gate_kind == SL_GATE_COLUMN ? a.gate : nullptr;
    const int pieces = norm_pieces<VEC, NV>(a.cols);
    NormMatrix<T, VEC, NV, kFew> mx(a.x, a.ld_x, row, stride, ring, 0), mb(a.branch, a.ld_branch, row, stride, ring, 1), mg(FULL ? a.gate : nullptr, a.ld_gate, row, stride, ring, 2);
    const unsigned stage_bytes = (unsigned)((FULL ? 3 : 2) * NV * VEC * sizeof(T) * blockDim.x * blockDim.y), ring_bytes = (unsigned)a.stages * stage_bytes;
    long long coming = row;  // the row to be copied next
    auto fetch = [&](unsigned stage_at) {
        if (kLate && coming > row && coming - stride < a.rows) {  // the row before, held until now
            const unsigned held_at = stage_at ? stage_at - stage_bytes : ring_bytes - stage_bytes;
            mx.settle(held_at, pieces);
            mb.settle(held_at, pieces);
            if (FULL) mg.settle(held_at, pieces);
        }
        if (coming < a.rows) {
            mx.fetch(stage_at, pieces);
            mb.fetch(stage_at, pieces);
            if (FULL) mg.fetch(stage_at, pieces);
        }
        coming += stride;
        copy_commit();
    };
    if constexpr (kFew) {
        mx.clear(a.stages, stage_bytes, pieces);
        mb.clear(a.stages, stage_bytes, pieces);
        if (FULL) mg.clear(a.stages, stage_bytes, pieces);
        for (int k = 0; k < a.stages - 1; ++k) fetch((unsigned)k * stage_bytes);
    }
    float2 w[P], c[P];
    if (kFew) {
        norm_weights<W, VEC, NV>(a.weight, nullptr, pieces, w);
        norm_weights<W, VEC, NV>(a.branch_weight, column_gate, pieces, c);
    }
    T* y = static_cast<T*>(a.y) + (a.y ? row * a.ld_y + norm_column<VEC>(0) : 0);
    T* h = static_cast<T*>(a.h) + (a.h ? row * a.ld_h + norm_column<VEC>(0) : 0);
    int turn = 0;  // of the exchanges, one or two in a row
    for (unsigned at = 0; row < a.rows; row += stride) {
        if (kFew) {
            fetch(at ? at - stage_bytes : ring_bytes - stage_bytes);
            copy_wait(a.stages - 1);
        }
        float2 v[P];
        if (has_branch) {
            float2 z[P];
            float rb = 1.0f;
            mb.get(at, pieces, z);
            if (normed) {
                float2 q = both(0.0f);
#pragma unroll
                for (int i = 0; i < P; ++i) q = fma2(z[i], z[i], q);
                float s[1] = {q.x + q.y};
                row_sums<1>(s, sums[turn]);
                turn ^= 1;
                rb = reciprocal_root(fmaf(s[0], a.inv_cols, a.eps));
                if (a.branch_rstd && threadIdx.x == 0) a.branch_rstd[row] = rb;
            }
            float scale = a.alpha * rb;
            if (a.gate_kind == SL_GATE_ROW) scale *= widen(static_cast<const T*>(a.gate)[row * a.ld_gate]);
            mx.get(at, pieces, v);
            float2 g[P];
            if (FULL) mg.get(at, pieces, g);
            if (!kFew) norm_weights<W, VEC, NV>(a.branch_weight, column_gate, pieces, c);
#pragma unroll
            for (int i = 0; i < P; ++i) v[i] = fma2(mul2(z[i], both(scale)), FULL ? mul2(c[i], g[i]) : c[i], v[i]);
            norm_store<T, VEC, NV>(y, pieces, v);
            y += stride * a.ld_y;
        } else {
            mx.get(at, pieces, v);
        }
        at = at + stage_bytes == ring_bytes ? 0u : at + stage_bytes;
        mx.next(), mb.next(), mg.next();
        if (!a.h) continue;
        float2 q = both(0.0f);
#pragma unroll
        for (int i = 0; i < P; ++i) q = fma2(v[i], v[i], q);  // (0 beyond the row's end)
        float s[1] = {q.x + q.y};
        row_sums<1>(s, sums[turn]);
        turn ^= 1;
        const float r = reciprocal_root(fmaf(s[0], a.inv_cols, a.eps));
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = r;
        if (!kFew) norm_weights<W, VEC, NV>(a.weight, nullptr, pieces, w);
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = mul2(mul2(v[i], both(r)), w[i]);
        norm_store<T, VEC, NV>(h, pieces, v);
        h += stride * a.ld_h;
    }
}

// Backward.  Three sums of a row at once (one exchange between its warps): with u = dh weight, yhat = y r, c = branch_weight times a
// column gate, q = bhat c times an element gate,
//     s0 = sum u yhat;   s1 = sum q (dy + r u);   s2 = sum q yhat
// give mean(u yhat) = s0 / cols and sum q dx = s1 - r s0 / cols s2, from which both mean(dz branch_weight bhat) and a row gate's
// gradient follow.  Two column sums serve three gradients: dbranch_weight and a column gate's are the sum of alpha dx bhat times the
// other one's weight.
template <class T, class W, int VEC, int NV, bool FULL>
__global__ void __launch_bounds__(NV* VEC <= 8 ? 640 : kNormMaxThreads)
norm_backward_kernel(const NormArgs a) {
    constexpr bool kFew = kNormFewBackward<VEC, NV>;
    constexpr int P = NV * VEC / 2;
    constexpr bool kLate = VEC * sizeof(T) < 4;
    extern __shared__ __align__(16) char ring[];  // afterwards [2][cols] column sums, only where blockDim.y > 1
    __shared__ float sums[2][3 * 16];
    clear_sums(sums[0], 2 * 3 * 16);
    const long long stride = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool normed = a.branch_weight != nullptr, row_gate = a.gate_kind == SL_GATE_ROW;
    const void* column_gate = a.gate_kind == SL_GATE_COLUMN ? a.gate : nullptr;
    const int pieces = norm_pieces<VEC, NV>(a.cols);
    NormMatrix<T, VEC, NV, kFew> mdy(a.dy, a.ld_dy, row, stride, ring, 0), mdh(a.dh, a.ld_dh, row, stride, ring, 1), my(a.dh ? a.x : nullptr, a.ld_y, row, stride, ring, 2),
        mb(a.branch, a.ld_branch, row, stride, ring, 3), mg(FULL ? a.gate : nullptr, a.ld_gate, row, stride, ring, 4);
    const unsigned stage_bytes = (unsigned)((FULL ? 5 : 4) * NV * VEC * sizeof(T) * blockDim.x * blockDim.y), ring_bytes = (unsigned)a.stages * stage_bytes;
    long long coming = row;
    auto fetch = [&](unsigned stage_at) {
        if (kLate && coming > row && coming - stride < a.rows) {  // the row before, held until now
            const unsigned held_at = stage_at ? stage_at - stage_bytes : ring_bytes - stage_bytes;
            mdy.settle(held_at, pieces);
            mdh.settle(held_at, pieces);
            my.settle(held_at, pieces);
            mb.settle(held_at, pieces);
            if (FULL) mg.settle(held_at, pieces);
        }
        if (coming < a.rows) {
            mdy.fetch(stage_at, pieces);
            mdh.fetch(stage_at, pieces);
            my.fetch(stage_at, pieces);
            mb.fetch(stage_at, pieces);
            if (FULL) mg.fetch(stage_at, pieces);
        }
        coming += stride;
        copy_commit();
    };
    float r_next = 0.0f, rb_next = 1.0f, rg_next = 1.0f;
    auto scalars = [&](long long at) {
        if (a.dh) r_next = a.rstd[at];
        if (normed) rb_next = a.branch_rstd[at];
        if (row_gate) rg_next = widen(static_cast<const T*>(a.gate)[at * a.ld_gate]);
    };
    if constexpr (kFew) {
        mdy.clear(a.stages, stage_bytes, pieces);
        mdh.clear(a.stages, stage_bytes, pieces);
        my.clear(a.stages, stage_bytes, pieces);
        mb.clear(a.stages, stage_bytes, pieces);
        if (FULL) mg.clear(a.stages, stage_bytes, pieces);
        for (int k = 0; k < a.stages - 1; ++k) fetch((unsigned)k * stage_bytes);
    }
    if (row < a.rows) scalars(row);
    float2 w[P], c[P], acc[2][P];
    if (kFew) {
        norm_weights<W, VEC, NV>(a.weight, nullptr, pieces, w);
        norm_weights<W, VEC, NV>(a.branch_weight, column_gate, pieces, c);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) acc[0][i] = acc[1][i] = both(0.0f);
    T* dx = static_cast<T*>(a.dx) + (a.dx ? row * a.ld_x + norm_column<VEC>(0) : 0);
    T* dbranch = static_cast<T*>(a.dbranch) + (a.dbranch ? row * a.ld_branch + norm_column<VEC>(0) : 0);
    T* dgate = static_cast<T*>(a.dgate) + (FULL && a.dgate ? row * a.ld_gate + norm_column<VEC>(0) : 0);
    int turn = 0;
    for (unsigned at = 0; row < a.rows; row += stride, turn ^= 1) {
        if (kFew) {
            fetch(at ? at - stage_bytes : ring_bytes - stage_bytes);
            copy_wait(a.stages - 1);
        } else {
            norm_weights<W, VEC, NV>(a.weight, nullptr, pieces, w);
            norm_weights<W, VEC, NV>(a.branch_weight, column_gate, pieces, c);
        }
        const float r = r_next, rb = rb_next, rg = rg_next;
        if (row + stride < a.rows) scalars(row + stride);
        float2 dy[P], dh[P], yh[P], bh[P], g[P];
        mdy.get(at, pieces, dy);
        mdh.get(at, pieces, dh);
        my.get(at, pieces, yh);
        mb.get(at, pieces, bh);
        if (FULL) mg.get(at, pieces, g);
        float2 t0 = both(0.0f), t1 = t0, t2 = t0;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            yh[i] = mul2(yh[i], both(r));
            bh[i] = mul2(bh[i], both(rb));
            const float2 u = mul2(dh[i], w[i]), q = FULL ? mul2(mul2(bh[i], c[i]), g[i]) : mul2(bh[i], c[i]);
            t0 = fma2(u, yh[i], t0);
            t1 = fma2(q, fma2(both(r), u, dy[i]), t1);
            t2 = fma2(q, yh[i], t2);
        }
        float s[3] = {t0.x + t0.y, t1.x + t1.y, t2.x + t2.y};
        row_sums<3>(s, sums[turn]);
        const float mean = s[0] * a.inv_cols;
        const float qdx = fmaf(-r * mean, s[2], s[1]);         // sum q dx
        const float bmean = a.alpha * rg * qdx * a.inv_cols;    // mean(dz branch_weight bhat)
        if (row_gate && a.dgate && threadIdx.x == 0) static_cast<T*>(a.dgate)[row * a.ld_gate] = narrow<T>(a.alpha * qdx);
        const float scale = a.alpha * rg, rbm = normed ? rb * bmean : 0.0f;
        mdy.get(at, pieces, dy);  // (read again rather than kept over the exchange: registers decide how many CTAs are resident)
        mdh.get(at, pieces, dh);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            acc[0][i] = fma2(dh[i], yh[i], acc[0][i]);
            dy[i] = fma2(both(r), fma2(yh[i], both(-mean), mul2(dh[i], w[i])), dy[i]);  // dx
            float2 e = mul2(dy[i], both(scale));
            if (FULL) {
                const float2 up = e;
                e = mul2(e, g[i]);
                g[i] = mul2(up, mul2(bh[i], c[i]));                                       // the element gate's (c is branch_weight then)
            }
            acc[1][i] = fma2(e, bh[i], acc[1][i]);
            dh[i] = fma2(mul2(e, both(rb)), c[i], mul2(bh[i], both(-rbm)));                // dbranch (rb is 1 and rbm 0 without its norm)
        }
        if (a.dx) norm_store<T, VEC, NV>(dx, pieces, dy);
        if (a.dbranch) norm_store<T, VEC, NV>(dbranch, pieces, dh);
        if (FULL && a.dgate) norm_store<T, VEC, NV>(dgate, pieces, g);
        dx += stride * a.ld_x;
        dbranch += stride * a.ld_branch;
        if (FULL) dgate += stride * a.ld_gate;
        at = at + stage_bytes == ring_bytes ? 0u : at + stage_bytes;
        mdy.next(), mdh.next(), my.next(), mb.next(), mg.next();
    }
    cudaTriggerProgrammaticLaunchCompletion();
    if (!a.part) return;
    float* part = a.part + (long long)blockIdx.x * 2 * a.cols;
    float* colsum = reinterpret_cast<float*>(ring);
    if (blockDim.y > 1) __syncthreads();  // every warp is through with the ring
    for (int t = 0; t < (int)blockDim.y; ++t) {  // the warps of a CTA add up in their order
        if ((int)threadIdx.y == t) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int col = norm_column<VEC>(i);
                    if (col < a.cols) {
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            const int at = k * a.cols + col + j;
                            const float own = (i * VEC + j) % 2 ? acc[k][(i * VEC + j) / 2].y : acc[k][(i * VEC + j) / 2].x;
                            const float sum = t ? colsum[at] + own : own;
                            if (t == (int)blockDim.y - 1) part[at] = sum;
                            else colsum[at] = sum;
                        }
                    }
                }
        }
        if (blockDim.y > 1) __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------------------------------------
// Rows that divide into pieces of 8 values on 16-byte boundaries (what models have): a warp takes a whole row of up to 512 columns, two
// warps wider ones, up to 8 pieces per lane.  What a row costs besides its values (its sums' exchange, addresses, loop) is paid once per
// warp, so few warps per row it is; two rather than one, since twice the warps fit the registers and shared memory of the same rows.
// Weights sit in shared memory as fp32, column sums in registers, rows come through a ring that every lane fills for itself.
// ------------------------------------------------------------------------------------------------------------------------------
constexpr int kTeamMaxPieces = 8;
__host__ __device__ constexpr int norm_team_threads(int nv, bool backward) {  // of a CTA: what its registers allow
    return backward ? (nv <= 1 ? 640 : nv <= 3 ? 512 : nv <= 5 ? 384 : 256) : (nv <= 2 ? 1024 : nv <= 4 ? 640 : nv <= 6 ? 512 : 384);
}

// Threads of a row: 32 or 64, known when compiling (offsets become immediate), or (TEAM = 0) as many as the launch says, the CTA's.
template <int TEAM>
__device__ __forceinline__ int team_width() { return TEAM ? TEAM : (int)blockDim.x; }

// Sums over a row's threads, the same in all of them.  Two warps meet at a barrier of their own (one per row of the CTA); `buf` holds
// [2 K] floats per row for them and must not be written again before both have read: callers alternate.
template <int K, int TEAM>
__device__ __forceinline__ void team_sums(float (&s)[K], float* buf) {
    if (TEAM == 0) {
        row_sums<K>(s, buf);
        return;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = warp_sum(s[k]);
    if (TEAM == 64) {
        float* own = buf + threadIdx.y * 2 * K;
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) own[2 * k + (threadIdx.x >> 5)] = s[k];
        }
        asm volatile("bar.sync %0, 64;" ::"r"(threadIdx.y + 1) : "memory");
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] = own[2 * k] + own[2 * k + 1];
    }
}

// A piece is 8 values: one 16-byte chunk of bfloat16, or two of fp32 that lie a team apart, so that every access of a warp is one
// contiguous stretch.  Chunk k of thread x begins at column (k * threads + x) * (values of a chunk).
template <class T>
struct Chunks {
    static constexpr int kNum = 8 * (int)sizeof(T) / 16, kValues = 16 / (int)sizeof(T);
};
template <class T, int NV, int TEAM>
__device__ __forceinline__ int team_chunks(int cols) {  // of this thread that the row has
    const int all = cols / Chunks<T>::kValues, x = (int)threadIdx.x;
    return all > x ? min(NV * Chunks<T>::kNum, (all - x - 1) / team_width<TEAM>() + 1) : 0;
}

// The 8 values of a piece from shared memory: chunk 0 at `at`, chunk 1 `plane` bytes on.
template <class T>
__device__ __forceinline__ void team_get(unsigned at, unsigned plane, float2 (&f)[4]) {
    unsigned w[4 * Chunks<T>::kNum];
#pragma unroll
    for (int h = 0; h < Chunks<T>::kNum; ++h) shared_load<16>(at + h * plane, w + 4 * h);
    if (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = widen2(w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + (sizeof(T) == 4 ? 1 : 0)]));
    }
}
// Piece i into the row whose first column of this thread is at p.
template <class T, int TEAM>
__device__ __forceinline__ void team_put(T* p, int i, int chunks, const float2 (&f)[4]) {
    if (sizeof(T) == 2) {
        if (i < chunks) *reinterpret_cast<uint4*>(p + i * team_width<TEAM>() * 8) = make_uint4(narrow2(f[0]), narrow2(f[1]), narrow2(f[2]), narrow2(f[3]));
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (2 * i + h < chunks) *reinterpret_cast<float4*>(p + (2 * i + h) * team_width<TEAM>() * 4) = make_float4(f[2 * h].x, f[2 * h].y, f[2 * h + 1].x, f[2 * h + 1].y);
    }
}

// The thread's pieces of a matrix, row by row.
template <class T, int NV, int TEAM>
struct TeamMatrix {
    const T* row;    // null: absent
    long long step;
    unsigned place;  // in the ring's first row
    __device__ __forceinline__ TeamMatrix(const void* base, long long ld, long long first, long long stride, unsigned ring, int array) {
        row = base ? static_cast<const T*>(base) + first * ld + threadIdx.x * Chunks<T>::kValues : nullptr;
        step = base ? stride * ld : 0;
        place = ring + (unsigned)(array * NV * Chunks<T>::kNum * team_width<TEAM>() + (int)threadIdx.x) * 16u;
    }
    __device__ __forceinline__ unsigned at(int k) const { return place + (unsigned)(k * team_width<TEAM>()) * 16u; }  // chunk k
    __device__ __forceinline__ void clear(int stages, unsigned stage_bytes, int chunks) const {
        for (int s = 0; s < stages; ++s)
#pragma unroll
            for (int k = 0; k < NV * Chunks<T>::kNum; ++k)
                if (!row || k >= chunks) asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at(k) + (unsigned)s * stage_bytes), "r"(0u) : "memory");
    }
    __device__ __forceinline__ void fetch(unsigned stage_at, int chunks) {
        if (!row) return;
#pragma unroll
        for (int k = 0; k < NV * Chunks<T>::kNum; ++k)
            if (k < chunks) copy_async<16>(at(k) + stage_at, row + k * team_width<TEAM>() * Chunks<T>::kValues);
        row += step;
    }
    __device__ __forceinline__ void get(unsigned stage_at, int i, float2 (&f)[4]) const { team_get<T>(at(i * Chunks<T>::kNum) + stage_at, (unsigned)team_width<TEAM>() * 16u, f); }
};

// fp32 weights (times those of `times`) of all columns into shared memory at `to`, by the CTA, in the order in which threads read
// them: plane 2 i + h holds values 4 h .. 4 h + 3 of every thread's piece i.
template <class T, class W, int NV, int TEAM>
__device__ __forceinline__ void team_weights(unsigned to, const void* w, const void* times, int cols) {
    for (int v = threadIdx.y * blockDim.x + threadIdx.x; v < 2 * NV * team_width<TEAM>(); v += blockDim.x * blockDim.y) {
        const int plane = v / team_width<TEAM>(), x = v - plane * team_width<TEAM>();
        const int col = sizeof(T) == 2 ? ((plane >> 1) * team_width<TEAM>() + x) * 8 + (plane & 1) * 4 : (plane * team_width<TEAM>() + x) * 4;
        float f[4] = {1.0f, 1.0f, 1.0f, 1.0f};
        if (col < cols) {
            Pack<W, 4> t;
            if (w) {
                t.load(static_cast<const W*>(w) + col);
                t.get(f);
            }
            if (times) {
                float g[4];
                t.load(static_cast<const W*>(times) + col);
                t.get(g);
#pragma unroll
                for (int j = 0; j < 4; ++j) f[j] *= g[j];
            }
        }
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + (unsigned)v * 16u), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]) : "memory");
    }
}

// blockDim = (threads of a row, rows of the CTA); shared memory: weights [2][NV][2][blockDim.x] chunks, then every row's ring.
template <class T, class W, int NV, bool FULL, int TEAM>
__global__ void __launch_bounds__(norm_team_threads(NV, false), 1)
norm_forward_team_kernel(const NormArgs a) {
    extern __shared__ __align__(16) char shared[];
    __shared__ float sums[2][32];
    if (TEAM == 0) clear_sums(sums[0], 64);
    const unsigned weights = (unsigned)__cvta_generic_to_shared(shared), table = 2u * NV * (unsigned)team_width<TEAM>() * 16u;
    const unsigned stage_bytes = (FULL ? 3u : 2u) * NV * Chunks<T>::kNum * (unsigned)team_width<TEAM>() * 16u, ring_bytes = (unsigned)a.stages * stage_bytes;
    const unsigned ring = weights + 2u * table + threadIdx.y * ring_bytes;
    const long long stride = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool normed = a.branch_weight != nullptr, has_branch = a.branch != nullptr;
    const int chunks = team_chunks<T, NV, TEAM>(a.cols);
    constexpr int kFirst = Chunks<T>::kValues;
    TeamMatrix<T, NV, TEAM> mx(a.x, a.ld_x, row, stride, ring, 0), mb(a.branch, a.ld_branch, row, stride, ring, 1), mg(FULL ? a.gate : nullptr, a.ld_gate, row, stride, ring, 2);
    mx.clear(a.stages, stage_bytes, chunks);
    mb.clear(a.stages, stage_bytes, chunks);
    if (FULL) mg.clear(a.stages, stage_bytes, chunks);
    long long coming = row;
    auto fetch = [&](unsigned stage_at) {
        if (coming < a.rows) {
            mx.fetch(stage_at, chunks);
            mb.fetch(stage_at, chunks);
            if (FULL) mg.fetch(stage_at, chunks);
        }
        coming += stride;
        copy_commit();
    };
    for (int k = 0; k < a.stages - 1; ++k) fetch((unsigned)k * stage_bytes);
    team_weights<T, W, NV, TEAM>(weights, a.weight, nullptr, a.cols);
    team_weights<T, W, NV, TEAM>(weights + table, a.branch_weight, a.gate_kind == SL_GATE_COLUMN ? a.gate : nullptr, a.cols);
    __syncthreads();
    const unsigned mine = weights + threadIdx.x * 16u, plane = (unsigned)team_width<TEAM>() * 16u;  // this thread's weights: piece i at mine + 2 i plane
    T* y = static_cast<T*>(a.y) + (a.y ? row * a.ld_y + threadIdx.x * kFirst : 0);
    T* h = static_cast<T*>(a.h) + (a.h ? row * a.ld_h + threadIdx.x * kFirst : 0);
    int turn = 0;  // of the exchanges, one or two in a row
    for (unsigned at = 0; row < a.rows; row += stride) {
        fetch(at ? at - stage_bytes : ring_bytes - stage_bytes);
        copy_wait(a.stages - 1);
        float2 v[NV][4], q = both(0.0f);
        if (has_branch) {
            float rb = 1.0f;
            if (normed) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float2 z[4];
                    mb.get(at, i, z);
#pragma unroll
                    for (int j = 0; j < 4; ++j) q = fma2(z[j], z[j], q);
                }
                float s[1] = {q.x + q.y};
                team_sums<1, TEAM>(s, sums[turn]);
                turn ^= 1;
                rb = reciprocal_root(fmaf(s[0], a.inv_cols, a.eps));
                if (a.branch_rstd && threadIdx.x == 0) a.branch_rstd[row] = rb;
                q = both(0.0f);
            }
            float scale = a.alpha * rb;
            if (a.gate_kind == SL_GATE_ROW) scale *= widen(static_cast<const T*>(a.gate)[row * a.ld_gate]);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float2 z[4], c[4], g[4];
                mx.get(at, i, v[i]);
                mb.get(at, i, z);
                if (FULL) mg.get(at, i, g);
                team_get<float>(mine + table + 2u * i * plane, plane, c);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[i][j] = fma2(mul2(z[j], both(scale)), FULL ? mul2(c[j], g[j]) : c[j], v[i][j]);
                    q = fma2(v[i][j], v[i][j], q);
                }
                team_put<T, TEAM>(y, i, chunks, v[i]);
            }
            y += stride * a.ld_y;
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                mx.get(at, i, v[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) q = fma2(v[i][j], v[i][j], q);
            }
        }
        at = at + stage_bytes == ring_bytes ? 0u : at + stage_bytes;
        if (!a.h) continue;
        float s[1] = {q.x + q.y};
        team_sums<1, TEAM>(s, sums[turn]);
        turn ^= 1;
        const float r = reciprocal_root(fmaf(s[0], a.inv_cols, a.eps));
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = r;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float2 w[4];
            team_get<float>(mine + 2u * i * plane, plane, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = mul2(mul2(v[i][j], both(r)), w[j]);
            team_put<T, TEAM>(h, i, chunks, w);
        }
        h += stride * a.ld_h;
    }
}

// The formulas are norm_backward_kernel's; a row's pieces and weights are read again for the second half.
template <class T, class W, int NV, bool FULL, int TEAM>
__global__ void __launch_bounds__(norm_team_threads(NV, true), 1)
norm_backward_team_kernel(const NormArgs a) {
    extern __shared__ __align__(16) char shared[];  // the rings become [rows of the CTA][2][cols] column sums at the end
    __shared__ float sums[2][3 * 32];
    if (TEAM == 0) clear_sums(sums[0], 2 * 3 * 32);
    const unsigned weights = (unsigned)__cvta_generic_to_shared(shared), table = 2u * NV * (unsigned)team_width<TEAM>() * 16u;
    const unsigned stage_bytes = (FULL ? 5u : 4u) * NV * Chunks<T>::kNum * (unsigned)team_width<TEAM>() * 16u, ring_bytes = (unsigned)a.stages * stage_bytes;
    const unsigned ring = weights + 2u * table + threadIdx.y * ring_bytes;
    const long long stride = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool normed = a.branch_weight != nullptr, row_gate = a.gate_kind == SL_GATE_ROW;
    const int chunks = team_chunks<T, NV, TEAM>(a.cols);
    constexpr int kFirst = Chunks<T>::kValues;
    TeamMatrix<T, NV, TEAM> mdy(a.dy, a.ld_dy, row, stride, ring, 0), mdh(a.dh, a.ld_dh, row, stride, ring, 1), my(a.dh ? a.x : nullptr, a.ld_y, row, stride, ring, 2),
        mb(a.branch, a.ld_branch, row, stride, ring, 3), mg(FULL ? a.gate : nullptr, a.ld_gate, row, stride, ring, 4);
    mdy.clear(a.stages, stage_bytes, chunks);
    mdh.clear(a.stages, stage_bytes, chunks);
    my.clear(a.stages, stage_bytes, chunks);
    mb.clear(a.stages, stage_bytes, chunks);
    if (FULL) mg.clear(a.stages, stage_bytes, chunks);
    long long coming = row;
    auto fetch = [&](unsigned stage_at) {
        if (coming < a.rows) {
            mdy.fetch(stage_at, chunks);
            mdh.fetch(stage_at, chunks);
            my.fetch(stage_at, chunks);
            mb.fetch(stage_at, chunks);
            if (FULL) mg.fetch(stage_at, chunks);
        }
        coming += stride;
        copy_commit();
    };
    float r_next = 0.0f, rb_next = 1.0f, rg_next = 1.0f;
    auto scalars = [&](long long at) {
        if (a.dh) r_next = a.rstd[at];
        if (normed) rb_next = a.branch_rstd[at];
        if (row_gate) rg_next = widen(static_cast<const T*>(a.gate)[at * a.ld_gate]);
    };
    for (int k = 0; k < a.stages - 1; ++k) fetch((unsigned)k * stage_bytes);
    if (row < a.rows) scalars(row);
    team_weights<T, W, NV, TEAM>(weights, a.weight, nullptr, a.cols);
    team_weights<T, W, NV, TEAM>(weights + table, a.branch_weight, a.gate_kind == SL_GATE_COLUMN ? a.gate : nullptr, a.cols);
    __syncthreads();
    const unsigned mine = weights + threadIdx.x * 16u, plane = (unsigned)team_width<TEAM>() * 16u;
    float2 acc[2][NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[0][i][j] = acc[1][i][j] = both(0.0f);
    T* dx = static_cast<T*>(a.dx) + (a.dx ? row * a.ld_x + threadIdx.x * kFirst : 0);
    T* dbranch = static_cast<T*>(a.dbranch) + (a.dbranch ? row * a.ld_branch + threadIdx.x * kFirst : 0);
    T* dgate = static_cast<T*>(a.dgate) + (FULL && a.dgate ? row * a.ld_gate + threadIdx.x * kFirst : 0);
    int turn = 0;
    for (unsigned at = 0; row < a.rows; row += stride, turn ^= 1) {
        fetch(at ? at - stage_bytes : ring_bytes - stage_bytes);
        copy_wait(a.stages - 1);
        const float r = r_next, rb = rb_next, rg = rg_next;
        if (row + stride < a.rows) scalars(row + stride);
        float2 t0 = both(0.0f), t1 = t0, t2 = t0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float2 dy[4], dh[4], yh[4], bh[4], g[4], w[4], c[4];
            mdy.get(at, i, dy);
            mdh.get(at, i, dh);
            my.get(at, i, yh);
            mb.get(at, i, bh);
            if (FULL) mg.get(at, i, g);
            team_get<float>(mine + 2u * i * plane, plane, w);
            team_get<float>(mine + table + 2u * i * plane, plane, c);
#pragma unroll
            for (int j = 0; j < 4; ++j) {  // (r and rb come in after the sums)
                const float2 u = mul2(dh[j], w[j]), q = FULL ? mul2(mul2(bh[j], c[j]), g[j]) : mul2(bh[j], c[j]);
                t0 = fma2(u, yh[j], t0);
                t1 = fma2(q, fma2(both(r), u, dy[j]), t1);
                t2 = fma2(q, yh[j], t2);
            }
        }
        float s[3] = {t0.x + t0.y, t1.x + t1.y, t2.x + t2.y};
        team_sums<3, TEAM>(s, sums[turn]);
        const float mean = s[0] * r * a.inv_cols;
        const float qdx = rb * fmaf(-r * mean, s[2] * r, s[1]);  // sum q dx
        const float bmean = a.alpha * rg * qdx * a.inv_cols;      // mean(dz branch_weight bhat)
        if (row_gate && a.dgate && threadIdx.x == 0) static_cast<T*>(a.dgate)[row * a.ld_gate] = narrow<T>(a.alpha * qdx);
        const float scale = a.alpha * rg, rbm = normed ? rb * rb * bmean : 0.0f;
        const float2 r2 = both(r), ry = both(-r * mean), rs = both(rb), sc = both(scale), nb = both(-rbm);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float2 dy[4], dh[4], yh[4], bh[4], g[4], w[4], c[4];
            mdy.get(at, i, dy);
            mdh.get(at, i, dh);
            my.get(at, i, yh);
            mb.get(at, i, bh);
            if (FULL) mg.get(at, i, g);
            team_get<float>(mine + 2u * i * plane, plane, w);
            team_get<float>(mine + table + 2u * i * plane, plane, c);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[0][i][j] = fma2(mul2(dh[j], r2), yh[j], acc[0][i][j]);
                dy[j] = fma2(r2, fma2(yh[j], ry, mul2(dh[j], w[j])), dy[j]);  // dx
                float2 e = mul2(dy[j], sc);
                if (FULL) {
                    const float2 up = e;
                    e = mul2(e, g[j]);
                    g[j] = mul2(mul2(up, rs), mul2(bh[j], c[j]));               // the element gate's (c is branch_weight then)
                }
                e = mul2(e, rs);
                acc[1][i][j] = fma2(e, bh[j], acc[1][i][j]);
                dh[j] = fma2(e, c[j], mul2(bh[j], nb));                          // dbranch (rb is 1 and rbm 0 without its norm)
            }
            if (a.dx) team_put<T, TEAM>(dx, i, chunks, dy);
            if (a.dbranch) team_put<T, TEAM>(dbranch, i, chunks, dh);
            if (FULL && a.dgate) team_put<T, TEAM>(dgate, i, chunks, g);
        }
        dx += stride * a.ld_x;
        dbranch += stride * a.ld_branch;
        if (FULL) dgate += stride * a.ld_gate;
        at = at + stage_bytes == ring_bytes ? 0u : at + stage_bytes;
    }
    cudaTriggerProgrammaticLaunchCompletion();
    if (!a.part) return;
    // every row of the CTA lays its sums down in shared memory; the columns are then added up row after row
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    const unsigned down = weights + 2u * table;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int col = sizeof(T) == 2 ? (i * team_width<TEAM>() + (int)threadIdx.x) * 8 + 4 * h : ((2 * i + h) * team_width<TEAM>() + (int)threadIdx.x) * 4;
                if (col < a.cols)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(down + ((threadIdx.y * 2u + k) * (unsigned)a.cols + (unsigned)col) * 4u), "f"(acc[k][i][2 * h].x),
                                 "f"(acc[k][i][2 * h].y), "f"(acc[k][i][2 * h + 1].x), "f"(acc[k][i][2 * h + 1].y) : "memory");
            }
    __syncthreads();
    float* part = a.part + (long long)blockIdx.x * 2 * a.cols;
    for (int col = threadIdx.y * blockDim.x + threadIdx.x; col < 2 * a.cols; col += blockDim.x * blockDim.y) {
        float sum = 0.0f;
        for (int t = 0; t < (int)blockDim.y; ++t) {
            float x;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(down + (unsigned)(t * 2 * a.cols + col) * 4u));
            sum += x;
        }
        part[col] = sum;
    }
}

// Column sums of the CTAs' parts in a fixed order: 32 columns per CTA, 32 strands of parts, then the strands in order.
template <class W>
__global__ void __launch_bounds__(1024)
norm_columns_kernel(const float* __restrict__ part, int parts, int cols, const W* branch_weight, const W* column_gate, W* dweight, W* dbranch_weight, W* dgate) {
    __shared__ float strand[32][33];
    const int lane = threadIdx.x & 31, s = threadIdx.x >> 5;
    const int at = blockIdx.x * 32 + lane, col = at < cols ? at : at - cols;  // among 2 * cols
    const bool first = at < cols, wanted = at < 2 * cols && (first ? dweight != nullptr : dbranch_weight || dgate);
    float sum = 0.0f;
    cudaGridDependencySynchronize();
    if (wanted) {
#pragma unroll 4
        for (int p = s; p < parts; p += 32) sum += __ldcg(part + (long long)p * 2 * cols + at);
    }
    strand[s][lane] = sum;
    __syncthreads();
    if (s == 0 && wanted) {
        sum = strand[0][lane];
#pragma unroll
        for (int k = 1; k < 32; ++k) sum += strand[k][lane];
        if (first) {
            dweight[col] = narrow<W>(sum);
        } else {
            if (dbranch_weight) dbranch_weight[col] = narrow<W>(column_gate ? sum * widen(column_gate[col]) : sum);
            if (dgate) dgate[col] = narrow<W>(branch_weight ? sum * widen(branch_weight[col]) : sum);
        }
    }
}

}  // namespace

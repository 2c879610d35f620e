// Residual update and norms around a block, forward and backward, row by row.  Part of libsparseloco (inner.cu).
//
// Bound: HBM.  Forward reads x and branch and writes y and h; backward reads dy, dh, y, branch and writes dx, dbranch:
// every matrix once.  A row lives in the registers of its threads between its sums and its outputs (a warp for narrow
// rows, a CTA for wide ones), so a row is fetched once and in-place outputs are safe.  CTAs stay and walk over rows: a thread
// keeps its columns, so weights and column sums stay in its registers too, and the next row's loads are under way while the
// present one is reduced.
#pragma once
#include "inner_common.cuh"

namespace {

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

// Sum of K values over the threads of a row, the same in all of them: lanes, then (rows wider than a warp) up to 16 warps through
// `buf` (K * 16 floats; those of absent warps are 0).  `buf` must not be written again before every thread has read it: callers
// alternate between two.
template <int K>
__device__ __forceinline__ void row_sums(float (&s)[K], float* buf) {
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = warp_sum(s[k]);
    if (blockDim.x <= 32) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) buf[k * 16 + warp] = s[k];
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

// The columns of a thread: vector i begins at column (i * blockDim.x + threadIdx.x) * VEC.
template <int VEC>
__device__ __forceinline__ int norm_column(int i) { return (i * (int)blockDim.x + (int)threadIdx.x) * VEC; }

template <int BYTES>
__device__ __forceinline__ void copy_async(void* shared, const void* global) {
    const unsigned at = (unsigned)__cvta_generic_to_shared(shared);
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(global) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(global), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait(int behind) {  // all but the `behind` last groups have landed, for this thread
    if (behind == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (behind == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// Where a thread finds its pieces of a row.  RING: a ring of rows in shared memory that it fills for itself, asynchronously and
// rows ahead (a piece is read by the thread that copied it, so nothing is waited for but the copy); places of absent matrices and
// of columns beyond the row's end are zeroed once.  Else (many columns per thread): global memory.
template <class T, int VEC, int NV, bool RING>
struct NormMatrix {
    typedef Pack<T, VEC> Piece;
    const T* ahead;     // the thread's first column in the row to be copied next (null: absent)
    const T* now;       // ... in the present row (where there is no ring)
    long long step;     // elements from one of the CTA's rows to the next
    char* places;       // this thread's first piece of stage 0
    __device__ __forceinline__ NormMatrix(const void* base, long long ld, long long row, long long stride, char* ring, int array) {
        ahead = base ? static_cast<const T*>(base) + row * ld + norm_column<VEC>(0) : nullptr;
        now = ahead;
        step = stride * ld;
        places = ring + ((size_t)array * NV * blockDim.x * blockDim.y + threadIdx.y * blockDim.x + threadIdx.x) * sizeof(Piece);
    }
    static __device__ __forceinline__ int offset(int i) { return i * (int)blockDim.x * VEC; }
    __device__ __forceinline__ Piece* place(int stage_bytes, int i) const {
        return reinterpret_cast<Piece*>(places + stage_bytes + i * (int)(blockDim.x * blockDim.y * sizeof(Piece)));
    }
    __device__ __forceinline__ void clear(int stages, int stage_bytes, int cols) const {
        for (int s = 0; s < stages; ++s)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (!ahead || norm_column<VEC>(i) >= cols)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) place(s * stage_bytes, i)->v[j] = narrow<T>(0.0f);
    }
    __device__ __forceinline__ void fetch(int stage_at, int cols) {
        if (!ahead) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (norm_column<VEC>(i) < cols) {
                if constexpr (Piece::kBytes >= 4) copy_async<Piece::kBytes>(place(stage_at, i), ahead + offset(i));
                else place(stage_at, i)->v[0] = ahead[offset(i)];
            }
        }
        ahead += step;
    }
    __device__ __forceinline__ void get(int stage_at, int i, int cols, float (&f)[VEC]) const {
        Piece t;
        if constexpr (RING) {
            t = *place(stage_at, i);
            t.get(f);
        } else if (now && norm_column<VEC>(i) < cols) {
            t.load(now + offset(i));
            t.get(f);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[j] = 0.0f;
        }
    }
    __device__ __forceinline__ void next() { now += now ? step : 0; }
};

// Weights of a thread's columns, 1 where there are none.
template <class W, int VEC, int NV>
struct NormWeights {
    float f[NV][VEC];
    __device__ __forceinline__ void set(const void* w, const void* times, int cols) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[i][j] = 1.0f;
            const int c = norm_column<VEC>(i);
            if (c < cols) {
                Pack<W, VEC> t;
                if (w) {
                    t.load(static_cast<const W*>(w) + c);
                    t.get(f[i]);
                }
                if (times) {
                    t.load(static_cast<const W*>(times) + c);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) f[i][j] *= widen(t.v[j]);
                }
            }
        }
    }
};

// Weights of piece i: kept, or (many columns per thread) fetched again.
template <class W, int VEC, int NV, bool KEEP>
__device__ __forceinline__ void norm_weights(const NormWeights<W, VEC, NV>& kept, const void* w, const void* times, int i, int cols, float (&f)[VEC]) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) f[j] = KEEP ? kept.f[i][j] : 1.0f;
    const int c = norm_column<VEC>(i);
    if (!KEEP && c < cols) {
        Pack<W, VEC> t;
        if (w) {
            t.load(static_cast<const W*>(w) + c);
            t.get(f);
        }
        if (times) {
            t.load(static_cast<const W*>(times) + c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[j] *= widen(t.v[j]);
        }
    }
}

// Few columns per thread: their weights stay in registers and rows come through the ring.
template <int VEC, int NV>
constexpr bool kNormFew = NV * VEC <= 16;

// T: activations, W: weights; VEC values per access, NV accesses per thread: blockDim.x * VEC * NV >= cols; FULL: a gate per element.
// blockDim.y rows per CTA, more than one only where blockDim.x is a warp.
template <class T, class W, int VEC, int NV, bool FULL>
__global__ void __launch_bounds__(NV* VEC <= 8 ? 1024 : NV * VEC <= 16 ? 640 : kNormMaxThreads)
norm_forward_kernel(const NormArgs a) {
    constexpr bool kFew = kNormFew<VEC, NV>;
    extern __shared__ __align__(16) char ring[];
    __shared__ float sums[2][16];
    clear_sums(sums[0], 32);
    const long long stride = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool normed = a.branch_weight != nullptr, has_branch = a.branch != nullptr;
    const void* column_gate = a.gate_kind == SL_GATE_COLUMN ? a.gate : nullptr;
    NormMatrix<T, VEC, NV, kFew> x(a.x, a.ld_x, row, stride, ring, 0), b(a.branch, a.ld_branch, row, stride, ring, 1), g(FULL ? a.gate : nullptr, a.ld_gate, row, stride, ring, 2);
    const int stage_bytes = (FULL ? 3 : 2) * NV * VEC * (int)(sizeof(T) * blockDim.x * blockDim.y), ring_bytes = a.stages * stage_bytes;
    if constexpr (kFew) {
        x.clear(a.stages, stage_bytes, a.cols);
        b.clear(a.stages, stage_bytes, a.cols);
        if (FULL) g.clear(a.stages, stage_bytes, a.cols);
    }
    long long coming = row;  // the row to be copied next
    auto fetch = [&](int stage_at) {
        if (coming < a.rows) {
            x.fetch(stage_at, a.cols);
            b.fetch(stage_at, a.cols);
            if (FULL) g.fetch(stage_at, a.cols);
        }
        coming += stride;
        copy_commit();
    };
    if (kFew)
        for (int k = 0; k < a.stages - 1; ++k) fetch(k * stage_bytes);
    NormWeights<W, VEC, NV> w, c;
    if (kFew) {
        w.set(a.weight, nullptr, a.cols);
        c.set(a.branch_weight, column_gate, a.cols);
    }
    T* y = static_cast<T*>(a.y) + (a.y ? row * a.ld_y + norm_column<VEC>(0) : 0);
    T* h = static_cast<T*>(a.h) + (a.h ? row * a.ld_h + norm_column<VEC>(0) : 0);
    for (int at = 0; row < a.rows; row += stride) {
        if (kFew) {
            fetch(at ? at - stage_bytes : ring_bytes - stage_bytes);
            copy_wait(a.stages - 1);
        }
        float v[NV][VEC];
        if (has_branch) {
            float z[NV][VEC], rb = 1.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) b.get(at, i, a.cols, z[i]);
            if (normed) {
                float s[1] = {0.0f};
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) s[0] = fmaf(z[i][j], z[i][j], s[0]);
                row_sums<1>(s, sums[0]);
                rb = reciprocal_root(fmaf(s[0], a.inv_cols, a.eps));
                if (a.branch_rstd && threadIdx.x == 0) a.branch_rstd[row] = rb;
            }
            float scale = a.alpha * rb;
            if (a.gate_kind == SL_GATE_ROW) scale *= widen(static_cast<const T*>(a.gate)[row * a.ld_gate]);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float gi[VEC], ci[VEC];
                x.get(at, i, a.cols, v[i]);
                if (FULL) g.get(at, i, a.cols, gi);
                norm_weights<W, VEC, NV, kFew>(c, a.branch_weight, column_gate, i, a.cols, ci);
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[i][j] = fmaf(FULL ? ci[j] * gi[j] : ci[j], scale * z[i][j], v[i][j]);
                if (norm_column<VEC>(i) < a.cols) {
                    Pack<T, VEC> t;
                    t.set(v[i]);
                    t.store(y + x.offset(i));
                }
            }
            y += stride * a.ld_y;
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) x.get(at, i, a.cols, v[i]);
        }
        at = at + stage_bytes == ring_bytes ? 0 : at + stage_bytes;
        x.next(), b.next(), g.next();
        if (!a.h) continue;
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] = fmaf(v[i][j], v[i][j], s[0]);  // (0 beyond the row's end)
        row_sums<1>(s, sums[1]);
        const float r = reciprocal_root(fmaf(s[0], a.inv_cols, a.eps));
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = r;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (norm_column<VEC>(i) < a.cols) {
                float wi[VEC];
                norm_weights<W, VEC, NV, kFew>(w, a.weight, nullptr, i, a.cols, wi);
#pragma unroll
                for (int j = 0; j < VEC; ++j) wi[j] *= v[i][j] * r;
                Pack<T, VEC> t;
                t.set(wi);
                t.store(h + x.offset(i));
            }
        }
        h += stride * a.ld_h;
    }
}

// Backward.  Three sums of a row at once (one exchange between its warps): with u = dh weight, yhat = y r, c = branch_weight times a
// column gate, q = bhat c times an element gate,
//     s0 = sum u yhat;   s1 = sum q (dy + r u);   s2 = sum q yhat
// give mean(u yhat) = s0 / cols and sum q dx = s1 - r s0 / cols s2, from which both mean(dz branch_weight bhat) and a row gate's
// gradient follow.  Two column sums serve three gradients: dbranch_weight and a column gate's are the sum of alpha dx bhat times the
// other one's weight.  The row's pieces are read again for the second half rather than kept: registers decide how many rows are
// under way.
template <class T, class W, int VEC, int NV, bool FULL>
__global__ void __launch_bounds__(NV* VEC <= 8 ? 640 : kNormMaxThreads)
norm_backward_kernel(const NormArgs a) {
    constexpr bool kFew = NV * VEC <= 8;
    extern __shared__ __align__(16) char ring[];  // afterwards [2][cols] column sums, only where blockDim.y > 1
    __shared__ float sums[2][3 * 16];
    clear_sums(sums[0], 2 * 3 * 16);
    const long long stride = (long long)gridDim.x * blockDim.y;
    long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool normed = a.branch_weight != nullptr, row_gate = a.gate_kind == SL_GATE_ROW;
    const void* column_gate = a.gate_kind == SL_GATE_COLUMN ? a.gate : nullptr;
    NormMatrix<T, VEC, NV, kFew> mdy(a.dy, a.ld_dy, row, stride, ring, 0), mdh(a.dh, a.ld_dh, row, stride, ring, 1), my(a.dh ? a.x : nullptr, a.ld_y, row, stride, ring, 2),
        mb(a.branch, a.ld_branch, row, stride, ring, 3), mg(FULL ? a.gate : nullptr, a.ld_gate, row, stride, ring, 4);
    const int stage_bytes = (FULL ? 5 : 4) * NV * VEC * (int)(sizeof(T) * blockDim.x * blockDim.y), ring_bytes = a.stages * stage_bytes;
    if constexpr (kFew) {
        mdy.clear(a.stages, stage_bytes, a.cols);
        mdh.clear(a.stages, stage_bytes, a.cols);
        my.clear(a.stages, stage_bytes, a.cols);
        mb.clear(a.stages, stage_bytes, a.cols);
        if (FULL) mg.clear(a.stages, stage_bytes, a.cols);
    }
    long long coming = row;
    auto fetch = [&](int stage_at) {
        if (coming < a.rows) {
            mdy.fetch(stage_at, a.cols);
            mdh.fetch(stage_at, a.cols);
            my.fetch(stage_at, a.cols);
            mb.fetch(stage_at, a.cols);
            if (FULL) mg.fetch(stage_at, a.cols);
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
    if (kFew)
        for (int k = 0; k < a.stages - 1; ++k) fetch(k * stage_bytes);
    if (row < a.rows) scalars(row);
    NormWeights<W, VEC, NV> w, c;
    if (kFew) {
        w.set(a.weight, nullptr, a.cols);
        c.set(a.branch_weight, column_gate, a.cols);
    }
    float acc[2][NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[0][i][j] = acc[1][i][j] = 0.0f;
    T* dx = static_cast<T*>(a.dx) + (a.dx ? row * a.ld_x + norm_column<VEC>(0) : 0);
    T* dbranch = static_cast<T*>(a.dbranch) + (a.dbranch ? row * a.ld_branch + norm_column<VEC>(0) : 0);
    T* dgate = static_cast<T*>(a.dgate) + (FULL && a.dgate ? row * a.ld_gate + norm_column<VEC>(0) : 0);
    int turn = 0;
    for (int at = 0; row < a.rows; row += stride, turn ^= 1) {
        if (kFew) {
            fetch(at ? at - stage_bytes : ring_bytes - stage_bytes);
            copy_wait(a.stages - 1);
        }
        const float r = r_next, rb = rb_next, rg = rg_next;
        if (row + stride < a.rows) scalars(row + stride);
        auto piece = [&](int i, float (&dy)[VEC], float (&dh)[VEC], float (&yh)[VEC], float (&bh)[VEC], float (&g)[VEC], float (&wi)[VEC], float (&ci)[VEC]) {
            mdy.get(at, i, a.cols, dy);
            mdh.get(at, i, a.cols, dh);
            my.get(at, i, a.cols, yh);
            mb.get(at, i, a.cols, bh);
            if (FULL) mg.get(at, i, a.cols, g);
            norm_weights<W, VEC, NV, kFew>(w, a.weight, nullptr, i, a.cols, wi);
            norm_weights<W, VEC, NV, kFew>(c, a.branch_weight, column_gate, i, a.cols, ci);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                yh[j] *= r;
                bh[j] *= rb;
            }
        };
        float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float dy[VEC], dh[VEC], yh[VEC], bh[VEC], g[VEC], wi[VEC], ci[VEC];
            piece(i, dy, dh, yh, bh, g, wi, ci);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float u = dh[j] * wi[j], q = FULL ? bh[j] * ci[j] * g[j] : bh[j] * ci[j];
                s[0] = fmaf(u, yh[j], s[0]);
                s[1] = fmaf(q, fmaf(r, u, dy[j]), s[1]);
                s[2] = fmaf(q, yh[j], s[2]);
            }
        }
        row_sums<3>(s, sums[turn]);
        const float mean = s[0] * a.inv_cols;
        const float qdx = fmaf(-r * mean, s[2], s[1]);         // sum q dx
        const float bmean = a.alpha * rg * qdx * a.inv_cols;    // mean(dz branch_weight bhat)
        if (row_gate && a.dgate && threadIdx.x == 0) static_cast<T*>(a.dgate)[row * a.ld_gate] = narrow<T>(a.alpha * qdx);
        const float scale = a.alpha * rg, rbm = normed ? rb * bmean : 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (norm_column<VEC>(i) >= a.cols) continue;
            float dy[VEC], dh[VEC], yh[VEC], bh[VEC], g[VEC], wi[VEC], ci[VEC];
            piece(i, dy, dh, yh, bh, g, wi, ci);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                acc[0][i][j] = fmaf(dh[j], yh[j], acc[0][i][j]);
                dy[j] = fmaf(r, fmaf(dh[j], wi[j], -yh[j] * mean), dy[j]);     // dx
                const float up = scale * dy[j], e = FULL ? up * g[j] : up;
                acc[1][i][j] = fmaf(e, bh[j], acc[1][i][j]);
                dh[j] = fmaf(rb * e, ci[j], -bh[j] * rbm);                      // dbranch (rb is 1 and rbm 0 without its norm)
                if (FULL) g[j] = up * bh[j] * ci[j];                            // the element gate's (c is branch_weight then)
            }
            Pack<T, VEC> t;
            if (a.dx) {
                t.set(dy);
                t.store(dx + mdy.offset(i));
            }
            if (a.dbranch) {
                t.set(dh);
                t.store(dbranch + mdy.offset(i));
            }
            if (FULL && a.dgate) {
                t.set(g);
                t.store(dgate + mdy.offset(i));
            }
        }
        dx += stride * a.ld_x;
        dbranch += stride * a.ld_branch;
        if (FULL) dgate += stride * a.ld_gate;
        at = at + stage_bytes == ring_bytes ? 0 : at + stage_bytes;
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
                            const float sum = t ? colsum[at] + acc[k][i][j] : acc[k][i][j];
                            if (t == (int)blockDim.y - 1) part[at] = sum;
                            else colsum[at] = sum;
                        }
                    }
                }
        }
        if (blockDim.y > 1) __syncthreads();
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

// Residual update and norms around a block, forward and backward, row by row.  Part of libsparseloco (inner.cu).
//
// Bound: HBM.  Forward reads x and branch and writes y and h; backward reads dy, dh, y, branch and writes dx, dbranch:
// every matrix once.  A row lives in the registers of its threads between its sums and its outputs (a warp for narrow
// rows, a CTA for wide ones), so a row is fetched once and in-place outputs are safe.
#pragma once
#include "inner_common.cuh"

namespace {

constexpr int kNormMaxCols = 16384;
constexpr int kNormMaxThreads = 512;
constexpr int kNormWarpRows = 4;   // rows (warps) of a forward CTA where a warp takes a row

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
    float* part;  // [CTAs][3][cols] column sums: dweight, dbranch_weight, dgate
    int row_gate_stride;
};

// Sum of K values over the threads of a row: lanes, then (rows wider than a warp) warps through `buf` (K * 32 floats).
// `buf` must not be written again before every thread has read it: callers alternate between two.
template <int K>
__device__ __forceinline__ void row_sums(float (&s)[K], float* buf) {
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = warp_sum(s[k]);
    if (blockDim.x <= 32) return;
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) buf[k * 32 + warp] = s[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = 0.0f;
    for (int w = 0; w < warps; ++w) {
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] += buf[k * 32 + w];
    }
}

// 1/sqrt with the result correct to an ulp or so (the approximate instruction plus one Newton step would do the same)
__device__ __forceinline__ float reciprocal_root(float x) { return 1.0f / sqrtf(x); }

// T: activations, W: weights; VEC values per access, NV accesses per thread: blockDim.x * VEC * NV >= cols.
// blockDim.y rows per CTA, more than one only where blockDim.x is a warp.
template <class T, class W, int VEC, int NV>
__global__ void __launch_bounds__(kNormMaxThreads)
norm_forward_kernel(const NormArgs a) {
    __shared__ float sums[2][32];
    const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= a.rows) return;  // (a whole warp, or the whole CTA)
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    float v[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        if (c < a.cols) {
            Pack<T, VEC> t;
            t.load(x + c);
            t.get(v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = 0.0f;
        }
    }
    if (a.branch) {
        const T* br = static_cast<const T*>(a.branch) + row * a.ld_branch;
        const W* bw = static_cast<const W*>(a.branch_weight);
        float b[NV][VEC];
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
            if (c < a.cols) {
                Pack<T, VEC> t;
                t.load(br + c);
                t.get(b[i]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) b[i][j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[0] = fmaf(b[i][j], b[i][j], s[0]);
        }
        float rb = 1.0f;
        if (bw) {
            row_sums<1>(s, sums[0]);
            rb = reciprocal_root(fmaf(s[0], a.inv_cols, a.eps));
            if (a.branch_rstd && threadIdx.x == 0) a.branch_rstd[row] = rb;
        }
        float scale = a.alpha;
        if (a.gate_kind == SL_GATE_ROW) scale *= widen(static_cast<const T*>(a.gate)[row * a.ld_gate]);
        T* y = static_cast<T*>(a.y) + row * a.ld_y;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
            if (c < a.cols) {
                float f[VEC];
                if (bw) {
                    Pack<W, VEC> t;
                    t.load(bw + c);
                    t.get(f);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) b[i][j] *= rb * f[j];
                }
                if (a.gate_kind == SL_GATE_COLUMN) {
                    Pack<W, VEC> t;
                    t.load(static_cast<const W*>(a.gate) + c);
                    t.get(f);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) b[i][j] *= f[j];
                } else if (a.gate_kind == SL_GATE_FULL) {
                    Pack<T, VEC> t;
                    t.load(static_cast<const T*>(a.gate) + row * a.ld_gate + c);
                    t.get(f);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) b[i][j] *= f[j];
                }
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[i][j] = fmaf(scale, b[i][j], v[i][j]);
                Pack<T, VEC> t;
                t.set(v[i]);
                t.store(y + c);
            }
        }
    }
    if (!a.h) return;
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[0] = fmaf(v[i][j], v[i][j], s[0]);
    row_sums<1>(s, sums[1]);
    const float r = reciprocal_root(fmaf(s[0], a.inv_cols, a.eps));
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = r;
    T* h = static_cast<T*>(a.h) + row * a.ld_h;
    const W* w = static_cast<const W*>(a.weight);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        if (c < a.cols) {
            float f[VEC];
            if (w) {
                Pack<W, VEC> t;
                t.load(w + c);
                t.get(f);
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[j] = w ? v[i][j] * r * f[j] : v[i][j] * r;
            Pack<T, VEC> t;
            t.set(f);
            t.store(h + c);
        }
    }
}

// Backward.  Three sums of a row at once (one exchange between its warps): with u = dh weight, yhat = y r, z as in the
// forward pass and q = z, times the column or element gate,
//     s0 = sum u yhat;   s1 = sum q (dy + r u);   s2 = sum q yhat
// give mean(u yhat) = s0 / cols and sum q dx = s1 - r s0 / cols s2, from which both mean(dz branch_weight bhat) and a row gate's
// gradient follow.  A thread keeps its columns from row to row, so the column sums stay in its registers until the end.
template <class T, class W, int VEC, int NV>
__global__ void __launch_bounds__(kNormMaxThreads)
norm_backward_kernel(const NormArgs a) {
    extern __shared__ float colsum[];  // [3][cols], only where blockDim.y > 1
    __shared__ float sums[2][3 * 32];
    float acc[3][NV][VEC], w[NV][VEC], bw[NV][VEC], cg[NV][VEC];
    const bool normed = a.branch_weight != nullptr, has_branch = a.branch != nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            acc[0][i][j] = acc[1][i][j] = acc[2][i][j] = 0.0f;
            w[i][j] = bw[i][j] = cg[i][j] = 1.0f;
        }
        if (c < a.cols) {
            Pack<W, VEC> t;
            if (a.weight) {
                t.load(static_cast<const W*>(a.weight) + c);
                t.get(w[i]);
            }
            if (normed) {
                t.load(static_cast<const W*>(a.branch_weight) + c);
                t.get(bw[i]);
            }
            if (a.gate_kind == SL_GATE_COLUMN) {
                t.load(static_cast<const W*>(a.gate) + c);
                t.get(cg[i]);
            }
        }
    }
    int turn = 0;
    for (long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y; row < a.rows; row += (long long)gridDim.x * blockDim.y, turn ^= 1) {
        const float r = a.dh ? a.rstd[row] : 0.0f, rb = normed ? a.branch_rstd[row] : 1.0f;
        const float rg = a.gate_kind == SL_GATE_ROW ? widen(static_cast<const T*>(a.gate)[row * a.ld_gate]) : 1.0f;
        float dy[NV][VEC], dh[NV][VEC], yh[NV][VEC], bh[NV][VEC], fg[NV][VEC];
        float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
#pragma unroll
            for (int j = 0; j < VEC; ++j) dy[i][j] = dh[i][j] = yh[i][j] = bh[i][j] = 0.0f, fg[i][j] = cg[i][j];
            if (c < a.cols) {
                Pack<T, VEC> t;
                if (a.dy) {
                    t.load(static_cast<const T*>(a.dy) + row * a.ld_dy + c);
                    t.get(dy[i]);
                }
                if (a.dh) {
                    t.load(static_cast<const T*>(a.dh) + row * a.ld_dh + c);
                    t.get(dh[i]);
                    t.load(static_cast<const T*>(a.x) + row * a.ld_y + c);
                    t.get(yh[i]);
                }
                if (has_branch) {
                    t.load(static_cast<const T*>(a.branch) + row * a.ld_branch + c);
                    t.get(bh[i]);
                }
                if (a.gate_kind == SL_GATE_FULL) {
                    t.load(static_cast<const T*>(a.gate) + row * a.ld_gate + c);
                    t.get(fg[i]);
                }
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                yh[i][j] *= r;
                bh[i][j] *= rb;
                const float u = dh[i][j] * w[i][j], q = bh[i][j] * bw[i][j] * fg[i][j];
                s[0] = fmaf(u, yh[i][j], s[0]);
                s[1] = fmaf(q, fmaf(r, u, dy[i][j]), s[1]);
                s[2] = fmaf(q, yh[i][j], s[2]);
            }
        }
        row_sums<3>(s, sums[turn]);
        const float mean = s[0] * a.inv_cols;
        const float qdx = fmaf(-r * mean, s[2], s[1]);             // sum q dx
        const float bmean = a.alpha * rg * qdx * a.inv_cols;        // mean(dz branch_weight bhat)
        if (a.gate_kind == SL_GATE_ROW && a.dgate && threadIdx.x == 0) static_cast<T*>(a.dgate)[row * a.ld_gate] = narrow<T>(a.alpha * qdx);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
            if (c >= a.cols) continue;
            float f[VEC], g[VEC], d[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                acc[0][i][j] = fmaf(dh[i][j], yh[i][j], acc[0][i][j]);
                f[j] = fmaf(r, fmaf(dh[i][j], w[i][j], -yh[i][j] * mean), dy[i][j]);  // dx
                const float up = a.alpha * f[j];
                g[j] = up * bh[i][j] * bw[i][j];                                      // the gate's gradient here
                acc[2][i][j] += g[j];
                const float dz = up * fg[i][j] * rg;
                acc[1][i][j] = fmaf(dz, bh[i][j], acc[1][i][j]);
                d[j] = normed ? rb * fmaf(dz, bw[i][j], -bh[i][j] * bmean) : dz;
            }
            Pack<T, VEC> t;
            if (a.dx) {
                t.set(f);
                t.store(static_cast<T*>(a.dx) + row * a.ld_x + c);
            }
            if (a.dbranch) {
                t.set(d);
                t.store(static_cast<T*>(a.dbranch) + row * a.ld_branch + c);
            }
            if (a.gate_kind == SL_GATE_FULL && a.dgate) {
                t.set(g);
                t.store(static_cast<T*>(a.dgate) + row * a.ld_gate + c);
            }
        }
    }
    if (!a.part) return;
    float* part = a.part + (long long)blockIdx.x * 3 * a.cols;
    for (int y = 0; y < (int)blockDim.y; ++y) {  // the warps of a CTA add up in their order
        if ((int)threadIdx.y == y) {
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = (i * blockDim.x + threadIdx.x) * VEC;
                    if (c < a.cols) {
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            const int at = k * a.cols + c + j;
                            const float sum = y ? colsum[at] + acc[k][i][j] : acc[k][i][j];
                            if (y == (int)blockDim.y - 1) part[at] = sum;
                            else colsum[at] = sum;
                        }
                    }
                }
        }
        if (blockDim.y > 1) __syncthreads();
    }
}

// Column sums of the CTAs' parts in a fixed order: 32 columns per CTA, 8 strands of parts, then the strands in order.
template <class W>
__global__ void __launch_bounds__(256)
norm_columns_kernel(const float* __restrict__ part, int parts, int cols, W* dweight, W* dbranch_weight, W* dgate) {
    __shared__ float strand[8][32];
    const int lane = threadIdx.x & 31, s = threadIdx.x >> 5;
    const int at = blockIdx.x * 32 + lane;  // among 3 * cols
    W* out = nullptr;
    if (at < 3 * cols) out = at < cols ? dweight : (at < 2 * cols ? dbranch_weight : dgate);
    float sum = 0.0f;
    if (out)
        for (int p = s; p < parts; p += 8) sum += part[(long long)p * 3 * cols + at];
    strand[s][lane] = sum;
    __syncthreads();
    if (s == 0 && out) {
        sum = strand[0][lane];
#pragma unroll
        for (int k = 1; k < 8; ++k) sum += strand[k][lane];
        out[at % cols] = narrow<W>(sum);
    }
}

}  // namespace

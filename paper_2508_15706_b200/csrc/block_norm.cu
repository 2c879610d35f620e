// Residual update and norms around a block (sl_norm_forward, sl_norm_backward): host side of the C ABI declared in
// include/sparseloco.h, over the kernels in block_norm.cuh.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <initializer_list>

#include "sparseloco.h"

#include "host.cuh"
#include "inner_common.cuh"
#include "block_norm.cuh"

namespace {

struct NormShape {
    int vec, nv, threads, rows_per_cta, stages;
    bool team;  // the kernels with whole rows per warp
    unsigned grid;
    size_t smem;
};

constexpr long long kNormShared = 220 * 1024;

// Pieces of 8 on 16-byte boundaries: a warp per row up to 512 columns, two up to 4096, as many as it takes beyond; with no more rows than
// a few per SM, as many threads as the row has pieces (up to 256).  A CTA per SM with as many rows as registers and a ring of two rows
// each allow.  False where shared memory does not hold two rows of everything.
bool norm_team_shape(NormShape* s, int cols, int bytes, int arrays, long long rows, int n_sms, bool backward) {
    const int vectors = cols / 8;
    int threads = vectors <= 64 ? 32 : vectors <= 64 * kTeamMaxPieces ? 64 : (vectors + 32 * kTeamMaxPieces - 1) / (32 * kTeamMaxPieces) * 32;
    if (rows <= 4ll * n_sms) threads = std::min(256, std::max(threads, (vectors + 31) / 32 * 32));
    int nv = (vectors + threads - 1) / threads;
    if (nv == 7 || (threads > 64 && nv > 4)) nv = 8;
    if (threads > 64 && nv == 3) nv = 4;
    const long long table = 2ll * 2 * nv * threads * 16, one = (long long)arrays * nv * threads * 8 * bytes;
    if (threads > norm_team_threads(nv, backward) || table + 2 * one > kNormShared) return false;
    long long r = threads > 64 ? 1 : std::min(15, norm_team_threads(nv, backward) / threads);  // (15: a barrier for each)
    r = std::min(r, (kNormShared - table) / (2 * one));
    r = std::max(1ll, std::min(r, (rows + n_sms - 1) / n_sms));
    // of the counts near the largest one, that whose last round of rows is fullest
    long long best = r;
    const auto filled = [&](long long k) { return (double)rows / (double)((rows + n_sms * k - 1) / (n_sms * k) * n_sms * k); };
    for (long long k = r; k >= 1 && 3 * k >= 2 * r; --k)
        if (filled(k) > filled(best) + 0.02) best = k;
    r = best;
    s->team = true;
    s->vec = 8;
    s->nv = nv;
    s->threads = threads;
    s->rows_per_cta = (int)r;
    // one row per CTA (wide rows, few rows): as many CTAs per SM as threads and shared memory allow
    const long long ctas = r > 1 ? 1 : std::max(1ll, std::min((long long)norm_team_threads(nv, backward) / threads, kNormShared / (table + 2 * one + 2048)));
    s->grid = (unsigned)std::min((rows + r - 1) / r, (long long)n_sms * ctas);
    const long long per = (long long)std::max(1u, s->grid) * r;  // (no more stages than a CTA has rows, and one)
    s->stages = (int)std::max(2ll, std::min(std::min(4ll, (rows + per - 1) / per + 1), (kNormShared / ctas - table) / (r * one)));
    s->smem = (size_t)(table + r * s->stages * one);
    if (backward) s->smem = std::max(s->smem, (size_t)(table + r * 2 * cols * 4));
    return true;
}

// Other rows: a warp takes a row of up to 32 vectors; wider rows are spread over a CTA of at most 512 threads, with as few vectors per
// thread as that allows.  (Single values: four per thread at least.)
NormShape norm_shape(int cols, int vec, int bytes, int arrays, long long rows, int n_sms, bool backward) {
    NormShape s = {};
    if (vec == 8 && norm_team_shape(&s, cols, bytes, arrays, rows, n_sms, backward)) return s;
    s.vec = vec == 8 ? 16 / bytes : vec;
    const int vectors = (cols + s.vec - 1) / s.vec;
    const int need = (vectors + kNormMaxThreads - 1) / kNormMaxThreads;
    if (s.vec >= 4) s.nv = 32 / s.vec;  // (wide rows only)
    else if (s.vec == 2) s.nv = need <= 4 ? 4 : 16;
    else s.nv = need <= 4 ? 4 : need <= 8 ? 8 : 32;
    s.threads = ((vectors + s.nv - 1) / s.nv + 31) / 32 * 32;
    s.rows_per_cta = s.threads == 32 ? kNormWarpRows : 1;
    // CTAs per SM: the registers of a thread decide (the kernels' launch bounds hold them to this)
    const int threads = s.threads * s.rows_per_cta;
    const long long ctas = std::max(1, std::min(32, 65536 / norm_regs(s.nv * s.vec, backward) / threads));
    s.grid = (unsigned)std::min((rows + s.rows_per_cta - 1) / s.rows_per_cta, n_sms * ctas);
    // rows in a CTA's ring: up to four, as many as the SM's shared memory holds for its CTAs, two at least (one being used, one on its
    // way), but no more than a CTA has rows
    const bool few = s.nv * s.vec <= (backward ? 8 : 16);
    const long long one = (long long)threads * s.nv * s.vec * bytes * arrays, per = (long long)std::max(1u, s.grid) * s.rows_per_cta;
    s.stages = (int)std::max(2ll, std::min(std::min(4ll, kNormShared / ctas / one), (rows + per - 1) / per + 1));
    s.smem = few ? (size_t)(one * s.stages) : 0;
    if (backward && s.rows_per_cta > 1) s.smem = std::max(s.smem, sizeof(float) * 2 * (size_t)cols);
    return s;
}

template <class K>
sl_status launch_norm_kernel(K kern, const NormArgs& a, const NormShape& s, cudaStream_t st) {
    if (s.smem > 47 * 1024) SL_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024));  // (1 KB stays for the sums)
    kern<<<s.grid, dim3((unsigned)s.threads, (unsigned)s.rows_per_cta), s.smem, st>>>(a);
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}

template <class T, class W, int NV, int TEAM>
sl_status launch_norm_team(const NormArgs& a, const NormShape& s, bool backward, cudaStream_t st) {
    const bool full = a.gate_kind == SL_GATE_FULL;
    if (backward) return full ? launch_norm_kernel(norm_backward_team_kernel<T, W, NV, true, TEAM>, a, s, st) : launch_norm_kernel(norm_backward_team_kernel<T, W, NV, false, TEAM>, a, s, st);
    return full ? launch_norm_kernel(norm_forward_team_kernel<T, W, NV, true, TEAM>, a, s, st) : launch_norm_kernel(norm_forward_team_kernel<T, W, NV, false, TEAM>, a, s, st);
}

template <class T, class W, int VEC, int NV>
sl_status launch_norm(const NormArgs& a, const NormShape& s, bool backward, cudaStream_t st) {
    const bool full = a.gate_kind == SL_GATE_FULL;
    if (backward) return full ? launch_norm_kernel(norm_backward_kernel<T, W, VEC, NV, true>, a, s, st) : launch_norm_kernel(norm_backward_kernel<T, W, VEC, NV, false>, a, s, st);
    return full ? launch_norm_kernel(norm_forward_kernel<T, W, VEC, NV, true>, a, s, st) : launch_norm_kernel(norm_forward_kernel<T, W, VEC, NV, false>, a, s, st);
}

template <class T, class W>
sl_status launch_norm_shape(const NormArgs& given, const NormShape& s, bool backward, cudaStream_t st) {
    NormArgs a = given;
    a.stages = s.stages;
    if (s.team && s.rows_per_cta == 1 && s.threads > 64) {
        switch (s.nv) {
            case 1: return launch_norm_team<T, W, 1, 0>(a, s, backward, st);
            case 2: return launch_norm_team<T, W, 2, 0>(a, s, backward, st);
            case 4: return launch_norm_team<T, W, 4, 0>(a, s, backward, st);
            default: return launch_norm_team<T, W, 8, 0>(a, s, backward, st);
        }
    }
    if (s.team && s.threads == 32) return s.nv == 1 ? launch_norm_team<T, W, 1, 32>(a, s, backward, st) : launch_norm_team<T, W, 2, 32>(a, s, backward, st);
    if (s.team) {
        switch (s.nv) {
            case 1: return launch_norm_team<T, W, 1, 64>(a, s, backward, st);
            case 2: return launch_norm_team<T, W, 2, 64>(a, s, backward, st);
            case 3: return launch_norm_team<T, W, 3, 64>(a, s, backward, st);
            case 4: return launch_norm_team<T, W, 4, 64>(a, s, backward, st);
            case 5: return launch_norm_team<T, W, 5, 64>(a, s, backward, st);
            case 6: return launch_norm_team<T, W, 6, 64>(a, s, backward, st);
            default: return launch_norm_team<T, W, 8, 64>(a, s, backward, st);
        }
    }
    if (s.vec == 1) return s.nv == 4 ? launch_norm<T, W, 1, 4>(a, s, backward, st) : s.nv == 8 ? launch_norm<T, W, 1, 8>(a, s, backward, st) : launch_norm<T, W, 1, 32>(a, s, backward, st);
    if (s.vec == 2) return s.nv == 4 ? launch_norm<T, W, 2, 4>(a, s, backward, st) : launch_norm<T, W, 2, 16>(a, s, backward, st);
    return launch_norm<T, W, 16 / (int)sizeof(T), 2 * (int)sizeof(T)>(a, s, backward, st);
}

sl_status launch_norm_types(const sl_norm_desc* d, const NormArgs& a, const NormShape& s, bool backward, cudaStream_t st) {
    if (d->dtype == SL_F32) return launch_norm_shape<float, float>(a, s, backward, st);
    if (d->weight_dtype == SL_F32) return launch_norm_shape<bf16, float>(a, s, backward, st);
    return launch_norm_shape<bf16, bf16>(a, s, backward, st);
}

template <class W>
sl_status launch_norm_columns(const NormArgs& a, unsigned parts, const void* column_gate, void* dweight, void* dbranch_weight, void* dgate, cudaStream_t st) {
    cudaLaunchConfig_t lc;
    memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3((unsigned)((2 * a.cols + 31) / 32));
    lc.blockDim = dim3(1024);
    lc.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = parts ? 1 : 0;  // only behind the backward kernel, which waits for what came before it
    SL_CUDA(cudaLaunchKernelEx(&lc, norm_columns_kernel<W>, (const float*)a.part, (int)parts, a.cols, static_cast<const W*>(a.branch_weight),
                               static_cast<const W*>(column_gate), static_cast<W*>(dweight), static_cast<W*>(dbranch_weight), static_cast<W*>(dgate)));
    return SL_OK;
}

sl_status norm_check(const sl_norm_desc* d) {
    if (!d || d->rows < 0 || d->cols < 1 || !isfinite(d->alpha) || !finite_at_least(d->eps, 0.0)) return SL_ERR_INVALID_ARG;
    if (!known_dtype(d->dtype) || !known_dtype(d->weight_dtype)) return SL_ERR_UNSUPPORTED;
    if (d->dtype == SL_F32 && d->weight_dtype != SL_F32) return SL_ERR_UNSUPPORTED;
    if (d->gate_kind < SL_GATE_NONE || d->gate_kind > SL_GATE_FULL) return SL_ERR_INVALID_ARG;
    if (d->cols > kNormMaxCols || d->rows > 0x7FFFFFFFll) return SL_ERR_TOO_LARGE;
    const int64_t ld[] = {d->ld_x, d->ld_branch, d->ld_y, d->ld_h, d->ld_dy, d->ld_dh};
    for (int64_t l : ld)
        if (l != 0 && l < d->cols) return SL_ERR_INVALID_ARG;
    if (d->ld_gate < 0 || (d->gate_kind == SL_GATE_FULL && d->ld_gate != 0 && d->ld_gate < d->cols)) return SL_ERR_INVALID_ARG;
    return SL_OK;
}

void norm_strides(const sl_norm_desc* d, NormArgs* a) {
    memset(a, 0, sizeof(*a));
    a->rows = d->rows;
    a->cols = (int)d->cols;
    a->gate_kind = d->gate_kind;
    a->alpha = d->alpha;
    a->eps = d->eps;
    a->inv_cols = 1.0f / (float)d->cols;
    a->ld_x = d->ld_x ? d->ld_x : d->cols;
    a->ld_branch = d->ld_branch ? d->ld_branch : d->cols;
    a->ld_y = d->ld_y ? d->ld_y : d->cols;
    a->ld_h = d->ld_h ? d->ld_h : d->cols;
    a->ld_dy = d->ld_dy ? d->ld_dy : d->cols;
    a->ld_dh = d->ld_dh ? d->ld_dh : d->cols;
    a->ld_gate = d->ld_gate ? d->ld_gate : (d->gate_kind == SL_GATE_FULL ? d->cols : 1);
}

// The values per piece that columns, row strides and pointers of everything allow: 8 (on 16-byte boundaries), or two, or one.
struct NormAlign {
    int bytes, vec;
    bool element;
    explicit NormAlign(const sl_norm_desc* d) : bytes(dtype_bytes(d->dtype)), vec(8), element(true) { all(d->cols, 8); }
    void all(long long n, int whole) { vec = n % whole == 0 ? vec : n % 2 == 0 ? std::min(vec, 2) : 1; }
    void matrix(const void* p, long long ld) {
        if (!p) return;
        element = element && fits(p, bytes);
        all(ld, 16 / bytes);
        all((long long)(reinterpret_cast<uintptr_t>(p) / (unsigned)bytes), 16 / bytes);
    }
    void vector(const void* p, int b) {  // weights: 16 bytes at a time, or as many values
        if (!p) return;
        element = element && fits(p, b);
        if (vec > 2 && !fits(p, 16)) vec = 2;
        if (vec == 2 && !fits(p, 2 * b)) vec = 1;
    }
};

// A matrix that is written where another one is read has to be the very same rows: others would be written before they are read.
struct NormPlace {
    const void* p;
    long long ld;
};
bool in_place_by_rows(long long rows, std::initializer_list<NormPlace> read, std::initializer_list<NormPlace> written) {
    for (const NormPlace& w : written)
        for (const NormPlace& r : read)
            if (rows > 1 && w.p && w.p == r.p && w.ld != r.ld) return false;
    return true;
}

}  // namespace

extern "C" {

sl_status sl_norm_forward(const sl_norm_desc* d, const void* x, const void* branch, const void* branch_weight, const void* gate, const void* weight,
                          void* y, void* h, float* branch_rstd, float* rstd, void* stream) {
    sl_status s = norm_check(d);
    if (s != SL_OK || d->rows == 0) return s;  // (matrices without rows have no address to check)
    if (!x || (!y && !h) || (branch != nullptr) != (y != nullptr) || (branch_weight && !branch) || (weight && !h)) return SL_ERR_INVALID_ARG;
    if ((d->gate_kind != SL_GATE_NONE) != (gate != nullptr) || (gate && !branch)) return SL_ERR_INVALID_ARG;
    NormArgs a;
    norm_strides(d, &a);
    a.x = x;
    a.branch = branch;
    a.branch_weight = branch_weight;
    a.gate = gate;
    a.weight = weight;
    a.y = y;
    a.h = h;
    a.branch_rstd = branch_rstd;
    a.rstd = rstd;
    const bool full = d->gate_kind == SL_GATE_FULL;
    if (!in_place_by_rows(d->rows, {{x, a.ld_x}, {branch, a.ld_branch}, {full ? gate : nullptr, a.ld_gate}}, {{y, a.ld_y}, {h, a.ld_h}})) return SL_ERR_INVALID_ARG;
    const int wb = dtype_bytes(d->weight_dtype);
    NormAlign al(d);
    al.matrix(x, a.ld_x);
    al.matrix(branch, a.ld_branch);
    al.matrix(y, a.ld_y);
    al.matrix(h, a.ld_h);
    al.vector(branch_weight, wb);
    al.vector(weight, wb);
    if (d->gate_kind == SL_GATE_COLUMN) al.vector(gate, wb);
    else if (d->gate_kind == SL_GATE_FULL) al.matrix(gate, a.ld_gate);
    else if (!fits(gate, al.bytes)) return SL_ERR_ALIGNMENT;
    if (!al.element || !fits(branch_rstd, 4) || !fits(rstd, 4)) return SL_ERR_ALIGNMENT;
    int n_sms = 0;
    s = sm_count(&n_sms);
    if (s != SL_OK) return s;
    const NormShape sh = norm_shape(a.cols, al.vec, al.bytes, d->gate_kind == SL_GATE_FULL ? 3 : 2, d->rows, n_sms, false);
    return launch_norm_types(d, a, sh, false, static_cast<cudaStream_t>(stream));
}

sl_status sl_norm_workspace_bytes(const sl_norm_desc* d, size_t* bytes) {
    sl_status s = norm_check(d);
    if (s != SL_OK) return s;
    if (!bytes) return SL_ERR_INVALID_ARG;
    int n_sms = 0;
    s = sm_count(&n_sms);
    if (s != SL_OK) return s;
    // the largest of the launch shapes that alignment and the gate decide between
    size_t most = 0;
    for (int vec : {1, 2, 8}) {
        if (vec == 8 && d->cols % 8) continue;
        for (int arrays : {4, 5}) {
            const NormShape sh = norm_shape((int)d->cols, vec, dtype_bytes(d->dtype), arrays, d->rows, n_sms, true);
            most = std::max(most, sizeof(float) * 2 * (size_t)d->cols * sh.grid);
        }
    }
    *bytes = up256(most);
    return SL_OK;
}

sl_status sl_norm_backward(const sl_norm_desc* d, const void* dy, const void* dh, const void* y, const void* branch, const void* branch_weight,
                           const void* gate, const void* weight, const float* branch_rstd, const float* rstd, void* dx, void* dbranch, void* dweight,
                           void* dbranch_weight, void* dgate, void* workspace, size_t workspace_bytes, void* stream) {
    sl_status s = norm_check(d);
    if (s != SL_OK) return s;
    const bool rows = d->rows > 0;  // (matrices without rows have no address to check)
    if (rows && ((!dy && !dh) || (dh && (!y || !rstd)) || (branch_weight && (!branch || !branch_rstd)) || (weight && !dh))) return SL_ERR_INVALID_ARG;
    if (rows && ((d->gate_kind != SL_GATE_NONE) != (gate != nullptr) || (gate && !branch) || (dbranch && !branch))) return SL_ERR_INVALID_ARG;
    if ((dweight && !weight) || (dbranch_weight && !branch_weight) || (rows && dgate && !gate)) return SL_ERR_INVALID_ARG;
    if (rows && !dx && !dbranch && !dweight && !dbranch_weight && !dgate) return SL_ERR_INVALID_ARG;
    NormArgs a;
    norm_strides(d, &a);
    a.dy = dy;
    a.dh = dh;
    a.x = y;
    a.branch = branch;
    a.branch_weight = branch_weight;
    a.gate = gate;
    a.weight = weight;
    a.branch_rstd = const_cast<float*>(branch_rstd);
    a.rstd = const_cast<float*>(rstd);
    a.dx = dx;
    a.dbranch = dbranch;
    a.dgate = d->gate_kind == SL_GATE_COLUMN ? nullptr : dgate;
    const bool full = d->gate_kind == SL_GATE_FULL;
    if (!in_place_by_rows(d->rows, {{dy, a.ld_dy}, {dh, a.ld_dh}, {y, a.ld_y}, {branch, a.ld_branch}, {full ? gate : nullptr, a.ld_gate}},
                          {{dx, a.ld_x}, {dbranch, a.ld_branch}, {full ? dgate : nullptr, a.ld_gate}}))
        return SL_ERR_INVALID_ARG;
    const int wb = dtype_bytes(d->weight_dtype);
    NormAlign al(d);
    al.matrix(dy, a.ld_dy);
    al.matrix(dh, a.ld_dh);
    if (dh) al.matrix(y, a.ld_y);
    al.matrix(branch, a.ld_branch);
    al.matrix(dx, a.ld_x);
    al.matrix(dbranch, a.ld_branch);
    al.vector(branch_weight, wb);
    al.vector(weight, wb);
    if (d->gate_kind == SL_GATE_COLUMN) al.vector(gate, wb);
    else if (d->gate_kind == SL_GATE_FULL) al.matrix(gate, a.ld_gate), al.matrix(dgate, a.ld_gate);
    else if (!fits(gate, al.bytes) || !fits(dgate, al.bytes)) return SL_ERR_ALIGNMENT;
    if (!al.element || !fits(branch_rstd, 4) || !fits(rstd, 4) || !fits(dweight, wb) || !fits(dbranch_weight, wb) || misaligned(workspace) ||
        (d->gate_kind == SL_GATE_COLUMN && !fits(dgate, wb)))
        return SL_ERR_ALIGNMENT;
    const bool columns = dweight || dbranch_weight || (d->gate_kind == SL_GATE_COLUMN && dgate);
    int n_sms = 0;
    s = sm_count(&n_sms);
    if (s != SL_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const NormShape sh = norm_shape(a.cols, al.vec, al.bytes, d->gate_kind == SL_GATE_FULL ? 5 : 4, d->rows, n_sms, true);
    const unsigned grid = d->rows ? sh.grid : 0;
    if (columns) {
        if (grid && (!workspace || workspace_bytes < sizeof(float) * 2 * (size_t)a.cols * grid)) return SL_ERR_NOMEM;
        a.part = static_cast<float*>(workspace);
    }
    if (grid) {
        s = launch_norm_types(d, a, sh, true, st);
        if (s != SL_OK) return s;
    }
    if (columns) {
        void* dg = d->gate_kind == SL_GATE_COLUMN ? dgate : nullptr;
        const void* cg = d->gate_kind == SL_GATE_COLUMN ? gate : nullptr;
        s = d->weight_dtype == SL_F32 ? launch_norm_columns<float>(a, grid, cg, dweight, dbranch_weight, dg, st)
                                      : launch_norm_columns<bf16>(a, grid, cg, dweight, dbranch_weight, dg, st);
        if (s != SL_OK) return s;
    }
    return SL_OK;
}

}  // extern "C"

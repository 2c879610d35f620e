// The operators of the inner phase (Alg. 1, the worker's local steps) for sm_100a: host side of the C ABI declared in
// include/sparseloco.h, over the kernels in the .cuh files beside it.  (The norms' host side is block_norm.cu: their many
// instances compile beside this file.)
//   adamw.cuh       AdamW over the tensor table, clipping by the global norm, moments in 32 or 8 bits
//   rotary.cuh      rotary positions of queries and keys
//   token_loss.cuh  next-token loss and its gradient
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "sparseloco.h"

#include "host.cuh"
#include "inner_common.cuh"
#include "adamw.cuh"
#include "rotary.cuh"
#include "token_loss.cuh"

struct sl_adamw {
    sl_adamw_config cfg;
    int device, n_sms;
    bool aligned8;  // every tensor begins on a multiple of 8 elements
    long long n_tiles, blocks, flat_elems;
    AdamTile* d_tiles;
    float* d_decay;
    double* d_parts;
    AdamClip* d_clip;
};

struct sl_rotary {
    sl_rotary_config cfg;
    int device;
    unsigned long long* d_turns;
};

namespace {

// ---- AdamW
template <class G>
sl_status launch_adamw_norm(const sl_adamw* c, const void* grad, double grad_scale, float* norm, cudaStream_t st) {
    const long long want = c->n_tiles, most = (long long)c->n_sms * kAdamNormCtas;
    const unsigned grid = (unsigned)std::min(std::min(want, most), (long long)kAdamMaxParts);
    auto kern = c->aligned8 ? adamw_norm_kernel<G, true> : adamw_norm_kernel<G, false>;
    kern<<<grid, kAdamThreads, 0, st>>>(c->d_tiles, c->n_tiles, static_cast<const G*>(grad), grad_scale, c->cfg.max_norm, c->d_parts, c->d_clip, norm);
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}

template <class P, class G, int BITS>
sl_status launch_adamw_step(const sl_adamw* c, const AdamArgs& a, cudaStream_t st) {
    auto kern = c->aligned8 ? adamw_step_kernel<P, G, BITS, true> : adamw_step_kernel<P, G, BITS, false>;
    cudaLaunchConfig_t lc;
    memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3((unsigned)c->n_tiles);
    lc.blockDim = dim3(kAdamThreads);
    lc.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = a.clip ? 1 : 0;  // only behind the norm kernel, which waits for what came before it
    SL_CUDA(cudaLaunchKernelEx(&lc, kern, (const AdamTile*)c->d_tiles, (const float*)c->d_decay, a));
    return SL_OK;
}

template <class P, class G>
sl_status launch_adamw_bits(const sl_adamw* c, const AdamArgs& a, cudaStream_t st) {
    return c->cfg.state_bits == 32 ? launch_adamw_step<P, G, 32>(c, a, st) : launch_adamw_step<P, G, 8>(c, a, st);
}

// ---- rotary
template <class T, int VEC>
sl_status launch_rotary(const RopeArgs& a, bool half, unsigned grid, size_t smem, cudaStream_t st) {
    constexpr bool kMayBeWide = VEC * sizeof(T) < 16;
    if (kMayBeWide && a.copy != VEC && a.slots > a.rot_slots) {
        if (half) rotary_kernel<T, VEC, true, kMayBeWide><<<grid, kRopeThreads, smem, st>>>(a);
        else rotary_kernel<T, VEC, false, kMayBeWide><<<grid, kRopeThreads, smem, st>>>(a);
    } else {
        if (half) rotary_kernel<T, VEC, true, false><<<grid, kRopeThreads, smem, st>>>(a);
        else rotary_kernel<T, VEC, false, false><<<grid, kRopeThreads, smem, st>>>(a);
    }
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}

// ---- loss
template <class T, int NV, bool RAGGED>
sl_status launch_loss_rows(const LossArgs& a, const T* logits, T* grad, int threads, int cluster, int n_sms, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    // as many CTAs as are resident: threads (by the launch bounds' registers) and shared memory
    const size_t smem = (size_t)kLossStages * threads * NV * 16;
    const long long ctas = std::max(1ll, std::min(32ll, std::min((NV * V <= 32 ? 1024ll : 512ll) / threads, 222ll * 1024 / ((long long)smem + 2048))));
    const long long teams = std::min((long long)a.rows, std::max(1ll, n_sms * ctas / cluster));
    const auto kern = loss_row_kernel<T, V, NV, RAGGED>;
    if (smem > 47 * 1024) SL_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024));
    cudaLaunchConfig_t lc;
    memset(&lc, 0, sizeof(lc));
    lc.gridDim = dim3((unsigned)(teams * cluster));
    lc.blockDim = dim3((unsigned)threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // behind the count, which waits for what came before it
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = cluster > 1 ? 2 : 1;
    SL_CUDA(cudaLaunchKernelEx(&lc, kern, a, logits, grad, cluster));
    return SL_OK;
}

template <class T, int VEC>
sl_status launch_loss_stream(const LossArgs& a, const T* logits, T* grad, cudaStream_t st) {
    loss_stream_kernel<T, VEC><<<(unsigned)a.rows, kLossThreads, 0, st>>>(a, logits, grad);
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}

template <class T, bool RAGGED>
sl_status launch_loss_nv(const LossArgs& a, const T* logits, T* grad, int nv, int threads, int cluster, int n_sms, cudaStream_t st) {
    return nv == 1 ? launch_loss_rows<T, 1, RAGGED>(a, logits, grad, threads, cluster, n_sms, st) : nv == 2 ? launch_loss_rows<T, 2, RAGGED>(a, logits, grad, threads, cluster, n_sms, st)
         : nv == 4 ? launch_loss_rows<T, 4, RAGGED>(a, logits, grad, threads, cluster, n_sms, st) : launch_loss_rows<T, 8, RAGGED>(a, logits, grad, threads, cluster, n_sms, st);
}

template <class T>
sl_status launch_loss(const LossArgs& a, const T* logits, T* grad, bool same, int n_sms, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T), kMaxNv = 8;
    const long long vectors = std::max(1, a.vocab / V);
    if (!same) return launch_loss_stream<T, 1>(a, logits, grad, st);
    if (vectors > 8ll * kLossThreads * kMaxNv || a.rows * 8 > 0x7FFFFFFFll) return launch_loss_stream<T, V>(a, logits, grad, st);
    // as few CTAs as hold the row; more while there are SMs without one and every thread would keep a vector
    int cluster = 1;
    while (vectors > (long long)cluster * kLossThreads * kMaxNv) cluster *= 2;
    while (cluster < 8 && a.rows * cluster < n_sms && vectors >= 2ll * cluster * kLossThreads) cluster *= 2;
    const long long per = (vectors + cluster - 1) / cluster;
    // as many vectors per thread as there are (what a row costs besides its values is paid by every thread), unless there are so few
    // rows that the SMs are better filled with threads
    const int least = a.rows * cluster > 2 * n_sms ? 32 : 256;
    int nv = 8;
    while (nv > 1 && per < (long long)nv * least) nv /= 2;
    while (per > (long long)nv * kLossThreads) nv *= 2;
    // (a thread's last vector may be missing, the others are there in every part of every row: parts are at most cluster + 1 vectors
    // shorter than `per`)
    int threads = (int)((per + nv - 1) / nv + 31) / 32 * 32;
    while (nv > 1 && (long long)(nv - 1) * threads > per - cluster - 1) {
        nv /= 2;
        threads = (int)((per + nv - 1) / nv + 31) / 32 * 32;
    }
    const bool ragged = !fits(logits, 16) || a.ld_logits % V || a.vocab % V;
    return ragged ? launch_loss_nv<T, true>(a, logits, grad, nv, threads, cluster, n_sms, st) : launch_loss_nv<T, false>(a, logits, grad, nv, threads, cluster, n_sms, st);
}

template <class T>
sl_status launch_loss_backward(const T* grad, const float* upstream, T* out, long long n, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    const bool whole = fits(grad, 16) && fits(out, 16);
    const long long items = whole ? std::max(1ll, n / V) : n, per = (long long)kUpThreads * kUpVectors;
    const unsigned grid = (unsigned)((items + per - 1) / per);
    if (whole) loss_backward_kernel<T, V><<<grid, kUpThreads, 0, st>>>(grad, upstream, out, n);
    else loss_backward_kernel<T, 1><<<grid, kUpThreads, 0, st>>>(grad, upstream, out, n);
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}

bool overlaps_no(const sl_tensor_desc* tensors, int n) {
    std::vector<std::pair<long long, long long>> span((size_t)n);
    for (int j = 0; j < n; ++j) span[(size_t)j] = {(long long)tensors[j].offset, (long long)tensors[j].offset + tensors[j].rows * tensors[j].cols};
    std::sort(span.begin(), span.end());
    for (int j = 1; j < n; ++j)
        if (span[(size_t)j].first < span[(size_t)j - 1].second) return false;
    return true;
}

void adamw_free(sl_adamw* c) {
    cudaFree(c->d_tiles);
    cudaFree(c->d_decay);
    cudaFree(c->d_parts);
    cudaFree(c->d_clip);
    delete c;
}

sl_status adamw_upload(sl_adamw* c, const std::vector<AdamTile>& tiles, const float* decay, int n) {
    SL_CUDA(cudaMalloc(&c->d_tiles, tiles.size() * sizeof(AdamTile)));
    SL_CUDA(cudaMalloc(&c->d_decay, (size_t)n * sizeof(float)));
    SL_CUDA(cudaMalloc(&c->d_parts, kAdamMaxParts * sizeof(double)));
    SL_CUDA(cudaMalloc(&c->d_clip, sizeof(AdamClip)));
    SL_CUDA(cudaMemcpy(c->d_tiles, tiles.data(), tiles.size() * sizeof(AdamTile), cudaMemcpyHostToDevice));
    SL_CUDA(cudaMemcpy(c->d_decay, decay, (size_t)n * sizeof(float), cudaMemcpyHostToDevice));
    SL_CUDA(cudaMemset(c->d_clip, 0, sizeof(AdamClip)));
    SL_CUDA(cudaDeviceSynchronize());
    return SL_OK;
}

}  // namespace

extern "C" {

sl_status sl_adamw_create(const sl_adamw_config* cfg, const sl_tensor_desc* tensors, const float* weight_decay, int32_t n_tensors, sl_adamw** out) {
    if (!out) return SL_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || !tensors || !weight_decay || n_tensors < 1) return SL_ERR_INVALID_ARG;
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return SL_ERR_INVALID_ARG;
    if (!finite_at_least(cfg->eps, 0.0) || !finite_at_least(cfg->max_norm, 0.0)) return SL_ERR_INVALID_ARG;
    if (cfg->skip_nonfinite != 0 && cfg->skip_nonfinite != 1) return SL_ERR_INVALID_ARG;
    if ((cfg->state_bits != 32 && cfg->state_bits != 8) || !known_dtype(cfg->param_dtype) || !known_dtype(cfg->grad_dtype)) return SL_ERR_UNSUPPORTED;
    long long total = 0;
    for (int j = 0; j < n_tensors; ++j) {
        const sl_tensor_desc& t = tensors[j];
        if (t.rows < 1 || t.cols < 1 || t.offset < 0 || !finite_at_least(weight_decay[j], 0.0)) return SL_ERR_INVALID_ARG;
        if (t.rows > (1ll << 40) / t.cols || t.offset > (1ll << 46)) return SL_ERR_TOO_LARGE;
        if (t.offset % 4 != 0) return SL_ERR_ALIGNMENT;
        total += (t.rows * t.cols + kAdamTile - 1) / kAdamTile;
        if (total > 0x7FFFFFFFll) return SL_ERR_TOO_LARGE;
    }
    try {
        if (!overlaps_no(tensors, n_tensors)) return SL_ERR_INVALID_ARG;
        std::vector<AdamTile> tiles;
        tiles.reserve((size_t)total);
        long long blocks = 0, flat = 0;
        bool a8 = true;
        for (int j = 0; j < n_tensors; ++j) {
            const long long n = tensors[j].rows * tensors[j].cols, off = tensors[j].offset;
            a8 = a8 && off % 8 == 0;
            flat = std::max(flat, off + n);
            for (long long i = 0; i < n; i += kAdamTile) {
                AdamTile t;
                t.base = off + i;
                t.block0 = blocks + i / kAdamBlock;
                t.len = (int)std::min((long long)kAdamTile, n - i);
                t.tensor = j;
                t.pad = 0;
                tiles.push_back(t);
            }
            blocks += (n + kAdamBlock - 1) / kAdamBlock;
        }
        sl_adamw* c = new (std::nothrow) sl_adamw();
        if (!c) return SL_ERR_NOMEM;
        c->cfg = *cfg;
        c->aligned8 = a8;
        c->n_tiles = total;
        c->blocks = blocks;
        c->flat_elems = flat;
        sl_status s = SL_OK;
        const cudaError_t e = cudaGetDevice(&c->device);
        s = e == cudaSuccess ? sm_count(&c->n_sms) : cuda_fail(e, "cudaGetDevice");
        if (s == SL_OK) s = adamw_upload(c, tiles, weight_decay, n_tensors);
        if (s != SL_OK) {
            adamw_free(c);
            return s;
        }
        *out = c;
        return SL_OK;
    } catch (const std::bad_alloc&) {
        return SL_ERR_NOMEM;
    }
}

sl_status sl_adamw_destroy(sl_adamw* c) {
    if (!c) return SL_ERR_INVALID_ARG;
    DeviceGuard g(c->device);
    const cudaError_t e = cudaDeviceSynchronize();
    adamw_free(c);
    return e == cudaSuccess ? SL_OK : cuda_fail(e, "cudaDeviceSynchronize");
}

sl_status sl_adamw_sizes(const sl_adamw* c, int64_t* flat_elems, int64_t* blocks) {
    if (!c || !flat_elems || !blocks) return SL_ERR_INVALID_ARG;
    *flat_elems = c->flat_elems;
    *blocks = c->blocks;
    return SL_OK;
}

sl_status sl_adamw_step(sl_adamw* c, void* theta, const void* grad, void* m, void* v, uint8_t* scales, uint16_t* copy, float* norm, int64_t step,
                        double lr, double grad_scale, uint32_t seed, void* stream) {
    if (!c || !theta || !grad || !m || !v || step < 1 || !isfinite(lr) || !isfinite(grad_scale)) return SL_ERR_INVALID_ARG;
    if ((c->cfg.state_bits == 8) != (scales != nullptr)) return SL_ERR_INVALID_ARG;
    if (copy && c->cfg.param_dtype != SL_F32) return SL_ERR_INVALID_ARG;
    const void* p[] = {theta, grad, m, v, scales, copy};
    for (int i = 0; i < 6; ++i)
        for (int j = 0; j < i; ++j)
            if (p[i] && p[i] == p[j]) return SL_ERR_INVALID_ARG;
    for (const void* x : p)
        if (misaligned(x)) return SL_ERR_ALIGNMENT;
    if (!fits(norm, 4)) return SL_ERR_ALIGNMENT;
    DeviceGuard guard(c->device);
    if (!guard.ok) return SL_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    AdamArgs a;
    memset(&a, 0, sizeof(a));
    a.theta = theta;
    a.grad = grad;
    a.m = m;
    a.v = v;
    a.scales = scales;
    a.copy = reinterpret_cast<bf16*>(copy);
    a.blocks = c->blocks;
    a.coef = (float)grad_scale;
    a.beta1 = (float)c->cfg.beta1;
    a.omb1 = (float)(1.0 - c->cfg.beta1);
    a.beta2 = (float)c->cfg.beta2;
    a.omb2 = (float)(1.0 - c->cfg.beta2);
    a.eps = (float)c->cfg.eps;
    a.inv_sqrt_bc2 = (float)(1.0 / sqrt(1.0 - pow(c->cfg.beta2, (double)step)));
    a.flush = adamw_may_flush(a.eps, a.inv_sqrt_bc2);
    a.step_size = (float)(lr / (1.0 - pow(c->cfg.beta1, (double)step)));
    a.lr = (float)lr;
    a.seed = seed;
    a.skip = c->cfg.skip_nonfinite;
    if (c->cfg.max_norm > 0.0 || c->cfg.skip_nonfinite || norm) {
        sl_status s = c->cfg.grad_dtype == SL_F32 ? launch_adamw_norm<float>(c, grad, grad_scale, norm, st) : launch_adamw_norm<bf16>(c, grad, grad_scale, norm, st);
        if (s != SL_OK) return s;
        a.clip = c->d_clip;
    }
    if (c->cfg.param_dtype == SL_F32) return c->cfg.grad_dtype == SL_F32 ? launch_adamw_bits<float, float>(c, a, st) : launch_adamw_bits<float, bf16>(c, a, st);
    return c->cfg.grad_dtype == SL_F32 ? launch_adamw_bits<bf16, float>(c, a, st) : launch_adamw_bits<bf16, bf16>(c, a, st);
}

static sl_status adamw_state(sl_adamw* c, bool write, float* m32, float* v32, uint8_t* m8, uint8_t* v8, uint8_t* scales, uint32_t seed, void* stream) {
    if (!c || !m32 || !v32 || !m8 || !v8 || !scales) return SL_ERR_INVALID_ARG;
    if (c->cfg.state_bits != 8) return SL_ERR_UNSUPPORTED;
    const void* p[] = {m32, v32, m8, v8, scales};
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < i; ++j)
            if (p[i] == p[j]) return SL_ERR_INVALID_ARG;
        if (misaligned(p[i])) return SL_ERR_ALIGNMENT;
    }
    DeviceGuard guard(c->device);
    if (!guard.ok) return SL_ERR_CUDA;
    const unsigned grid = (unsigned)c->n_tiles;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!write) adamw_read_kernel<<<grid, kAdamThreads, 0, st>>>(c->d_tiles, m32, v32, m8, v8, scales, c->blocks);
    else if (c->aligned8) adamw_write_kernel<true><<<grid, kAdamThreads, 0, st>>>(c->d_tiles, m32, v32, m8, v8, scales, c->blocks, seed);
    else adamw_write_kernel<false><<<grid, kAdamThreads, 0, st>>>(c->d_tiles, m32, v32, m8, v8, scales, c->blocks, seed);
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}

sl_status sl_adamw_read_state(sl_adamw* c, const uint8_t* m, const uint8_t* v, const uint8_t* scales, float* m_out, float* v_out, void* stream) {
    return adamw_state(c, false, m_out, v_out, const_cast<uint8_t*>(m), const_cast<uint8_t*>(v), const_cast<uint8_t*>(scales), 0u, stream);
}

sl_status sl_adamw_write_state(sl_adamw* c, const float* m_in, const float* v_in, uint8_t* m, uint8_t* v, uint8_t* scales, uint32_t seed, void* stream) {
    return adamw_state(c, true, const_cast<float*>(m_in), const_cast<float*>(v_in), m, v, scales, seed, stream);
}

sl_status sl_rotary_create(const sl_rotary_config* cfg, sl_rotary** out) {
    if (!out) return SL_ERR_INVALID_ARG;
    *out = nullptr;
    if (!cfg || cfg->rot_dim < 2 || cfg->rot_dim % 2 || cfg->rot_dim > 1024) return SL_ERR_INVALID_ARG;
    if (cfg->layout != SL_ROPE_HALF && cfg->layout != SL_ROPE_INTERLEAVED) return SL_ERR_INVALID_ARG;
    if (cfg->scaling < SL_ROPE_PLAIN || cfg->scaling > SL_ROPE_BY_PARTS) return SL_ERR_INVALID_ARG;
    if (!(isfinite(cfg->base) && cfg->base > 1.0) || !isfinite(cfg->magnitude)) return SL_ERR_INVALID_ARG;
    if (cfg->scaling != SL_ROPE_PLAIN && !(finite_at_least(cfg->factor, 1.0))) return SL_ERR_INVALID_ARG;
    if (cfg->scaling == SL_ROPE_BASE && cfg->rot_dim < 4) return SL_ERR_INVALID_ARG;
    if (cfg->scaling == SL_ROPE_BY_PARTS && !(finite_at_least(cfg->original_length, 1.0) && finite_at_least(cfg->low_turns, 0.0) && isfinite(cfg->high_turns) &&
                                              cfg->high_turns > cfg->low_turns))
        return SL_ERR_INVALID_ARG;
    const int half = cfg->rot_dim / 2;
    const long double two_pi = 6.283185307179586476925286766559005768L;
    std::vector<unsigned long long> turns;
    try {
        turns.resize((size_t)half);
    } catch (const std::bad_alloc&) {
        return SL_ERR_NOMEM;
    }
    long double base = cfg->base;
    if (cfg->scaling == SL_ROPE_BASE) base *= powl((long double)cfg->factor, (long double)cfg->rot_dim / (cfg->rot_dim - 2));
    for (int i = 0; i < half; ++i) {
        long double f = powl(base, -2.0L * i / cfg->rot_dim);
        if (cfg->scaling == SL_ROPE_LINEAR) f /= cfg->factor;
        if (cfg->scaling == SL_ROPE_BY_PARTS) {
            long double k = (cfg->original_length * f / two_pi - cfg->low_turns) / ((long double)cfg->high_turns - cfg->low_turns);
            k = k < 0.0L ? 0.0L : (k > 1.0L ? 1.0L : k);
            f = f * k + f / cfg->factor * (1.0L - k);
        }
        // f <= 1 radian, so below a turn; the fraction keeps 64 bits behind the point
        turns[(size_t)i] = (unsigned long long)(f / two_pi * 18446744073709551616.0L + 0.5L);
    }
    sl_rotary* c = new (std::nothrow) sl_rotary();
    if (!c) return SL_ERR_NOMEM;
    c->cfg = *cfg;
    c->d_turns = nullptr;
    cudaError_t e = cudaGetDevice(&c->device);
    if (e == cudaSuccess) e = cudaMalloc(&c->d_turns, turns.size() * sizeof(unsigned long long));
    if (e == cudaSuccess) e = cudaMemcpy(c->d_turns, turns.data(), turns.size() * sizeof(unsigned long long), cudaMemcpyHostToDevice);
    if (e != cudaSuccess) {
        cudaFree(c->d_turns);
        delete c;
        return cuda_fail(e, "sl_rotary_create");
    }
    *out = c;
    return SL_OK;
}

sl_status sl_rotary_destroy(sl_rotary* c) {
    if (!c) return SL_ERR_INVALID_ARG;
    DeviceGuard g(c->device);
    const cudaError_t e = cudaDeviceSynchronize();
    cudaFree(c->d_turns);
    delete c;
    return e == cudaSuccess ? SL_OK : cuda_fail(e, "cudaDeviceSynchronize");
}

sl_status sl_rotary_apply(sl_rotary* c, const sl_rotary_desc* d, const sl_rotary_heads* q, const sl_rotary_heads* k, const void* positions, void* stream) {
    if (!c || !d || !q || !q->in || !q->out) return SL_ERR_INVALID_ARG;
    if (!known_dtype(d->dtype)) return SL_ERR_UNSUPPORTED;
    if (d->batch < 0 || d->seq < 0 || d->head_dim < c->cfg.rot_dim || q->heads < 1) return SL_ERR_INVALID_ARG;
    if (positions && d->position_bits != 32 && d->position_bits != 64) return SL_ERR_INVALID_ARG;
    const sl_rotary_heads none = {nullptr, nullptr, 0, 0, 0, 0, 0, 0, 0};
    if (!k) k = &none;
    if ((k->in != nullptr) != (k->out != nullptr) || (k->in != nullptr) != (k->heads != 0) || k->heads < 0) return SL_ERR_INVALID_ARG;
    if (d->head_dim > 65536 || d->seq > 0x7FFFFFFFll || d->batch > 0x7FFFFFFFll || d->batch * d->seq > 0x7FFFFFFFll || q->heads > 65536 ||
        k->heads > 65536 || (q->heads + k->heads) * d->head_dim > (1ll << 27))
        return SL_ERR_TOO_LARGE;
    for (const sl_rotary_heads* h : {q, k}) {  // in place means the very same elements: dimensions of one element may have any stride
        const int64_t extent[] = {d->batch, d->seq, h->heads}, in[] = {h->in_batch, h->in_token, h->in_head}, out[] = {h->out_batch, h->out_token, h->out_head};
        for (int i = 0; i < 3; ++i)
            if (h->in && extent[i] > 1 && ((h->in == h->out && in[i] != out[i]) || out[i] == 0)) return SL_ERR_INVALID_ARG;
    }
    const int bytes = dtype_bytes(d->dtype), rot = c->cfg.rot_dim;
    const bool half = c->cfg.layout == SL_ROPE_HALF;
    // the widest accesses that every offset of the turned part, and of what is passed through, is a multiple of
    int vec = 16 / bytes, copy = 16 / bytes;
    auto divides = [&](int v, int64_t part, int64_t begin) {
        if (part % v || begin % v) return false;
        for (const sl_rotary_heads* h : {q, k}) {
            if (!h->in) continue;
            for (int64_t st : {h->in_batch, h->in_token, h->in_head, h->out_batch, h->out_token, h->out_head})
                if (st % v) return false;
            if (!fits(h->in, v * bytes) || !fits(h->out, v * bytes)) return false;
        }
        return true;
    };
    while (copy > 1 && !divides(copy, d->head_dim - rot, rot)) copy /= 2;
    while (vec > 1 && (vec > copy || !divides(vec, half ? rot / 2 : rot, 0))) vec /= 2;  // (never wider than the rest's)
    for (const sl_rotary_heads* h : {q, k})
        if (!fits(h->in, bytes) || !fits(h->out, bytes)) return SL_ERR_ALIGNMENT;
    if (positions && !fits(positions, d->position_bits / 8)) return SL_ERR_ALIGNMENT;
    DeviceGuard guard(c->device);
    if (!guard.ok) return SL_ERR_CUDA;
    RopeArgs a;
    memset(&a, 0, sizeof(a));
    auto heads = [](const sl_rotary_heads* h) {
        RopeHeads r = {h->in, h->out, (int)h->heads, h->in_batch, h->in_token, h->in_head, h->out_batch, h->out_token, h->out_head};
        return r;
    };
    a.q = heads(q);
    a.k = heads(k);
    a.turns = c->d_turns;
    a.positions = positions;
    a.pos_batch = d->pos_batch;
    a.pos_token = d->pos_token;
    a.first = d->first;
    a.rows = d->batch * d->seq;
    a.position_bits = d->position_bits;
    a.seq = (int)d->seq;
    a.head_dim = (int)d->head_dim;
    a.rot = rot;
    a.magnitude = (float)c->cfg.magnitude;
    a.sign = d->inverse ? -1.0f : 1.0f;
    a.rot_slots = half ? rot / 2 / vec : (vec > 1 ? rot / vec : rot / 2);
    a.copy = copy;
    a.slots = a.rot_slots + (int)(d->head_dim - rot) / copy;
    if (a.rows == 0) return SL_OK;
    int n_sms = 0;
    sl_status s = sm_count(&n_sms);
    if (s != SL_OK) return s;
    // more tokens per CTA even out its last round of accesses; few tokens are spread over the SMs first
    a.tokens = (int)std::max(1ll, std::min(8ll, (long long)(a.rows / (4 * n_sms))));
    const unsigned grid = (unsigned)((a.rows + a.tokens - 1) / a.tokens);
    const size_t smem = sizeof(float2) * (size_t)a.tokens * (rot / 2);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (d->dtype == SL_F32)
        return vec == 4 ? launch_rotary<float, 4>(a, half, grid, smem, st) : vec == 2 ? launch_rotary<float, 2>(a, half, grid, smem, st) : launch_rotary<float, 1>(a, half, grid, smem, st);
    return vec == 8 ? launch_rotary<bf16, 8>(a, half, grid, smem, st) : vec == 4 ? launch_rotary<bf16, 4>(a, half, grid, smem, st)
         : vec == 2 ? launch_rotary<bf16, 2>(a, half, grid, smem, st) : launch_rotary<bf16, 1>(a, half, grid, smem, st);
}

size_t sl_loss_workspace_bytes(void) { return 256; }

sl_status sl_token_loss(const sl_loss_desc* d, const void* logits, const void* targets, void* grad, float* row_loss, float* lse, float* total,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (!d || d->rows < 0 || d->vocab < 1) return SL_ERR_INVALID_ARG;
    if (!known_dtype(d->dtype) || (d->target_bits != 32 && d->target_bits != 64)) return SL_ERR_UNSUPPORTED;
    if (d->rows > 0 && (!logits || !targets || !row_loss)) return SL_ERR_INVALID_ARG;
    if (!(d->smoothing >= 0.0f && d->smoothing <= 1.0f) || !isfinite(d->z) || !isfinite(d->scale)) return SL_ERR_INVALID_ARG;
    if (d->vocab > (1ll << 30) || d->rows > 0x7FFFFFFFll) return SL_ERR_TOO_LARGE;
    if ((d->ld_logits != 0 && d->ld_logits < d->vocab) || (d->ld_grad != 0 && d->ld_grad < d->vocab)) return SL_ERR_INVALID_ARG;
    const int bytes = dtype_bytes(d->dtype);
    if (!fits(logits, bytes) || !fits(grad, bytes) || !fits(targets, d->target_bits / 8) || !fits(row_loss, 4) || !fits(lse, 4) || !fits(total, 4) ||
        misaligned(workspace))
        return SL_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < sizeof(LossWork)) return SL_ERR_NOMEM;
    LossArgs a;
    memset(&a, 0, sizeof(a));
    a.rows = d->rows;
    a.ld_logits = d->ld_logits ? d->ld_logits : d->vocab;
    a.ld_grad = d->ld_grad ? d->ld_grad : d->vocab;
    if (grad && grad == logits && a.ld_grad != a.ld_logits) return SL_ERR_INVALID_ARG;
    a.ignore_index = d->ignore_index;
    a.vocab = (int)d->vocab;
    a.target_bits = d->target_bits;
    a.mean = d->mean;
    a.smoothing = d->smoothing;
    a.z = d->z;
    a.scale = d->scale;
    a.targets = targets;
    a.row_loss = row_loss;
    a.lse = lse;
    a.total = total;
    a.work = static_cast<LossWork*>(workspace);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    loss_count_kernel<<<1, 1024, 0, st>>>(a);
    SL_CUDA(cudaGetLastError());
    if (d->rows == 0) return SL_OK;
    // 16-byte accesses from the first boundary of a row on: every row of logits and gradient has to meet it at the same column
    const bool same = !grad || ((reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(grad)) % 16 == 0 && (a.ld_logits - a.ld_grad) * bytes % 16 == 0);
    int n_sms = 0;
    sl_status s = sm_count(&n_sms);
    if (s != SL_OK) return s;
    return d->dtype == SL_F32 ? launch_loss<float>(a, (const float*)logits, (float*)grad, same, n_sms, st) : launch_loss<bf16>(a, (const bf16*)logits, (bf16*)grad, same, n_sms, st);
}

sl_status sl_token_loss_backward(int32_t dtype, int64_t n, const void* grad, const float* upstream, void* out, void* stream) {
    if (n < 0 || (n > 0 && (!grad || !upstream || !out))) return SL_ERR_INVALID_ARG;
    if (!known_dtype(dtype)) return SL_ERR_UNSUPPORTED;
    if (n > (1ll << 40)) return SL_ERR_TOO_LARGE;
    const int bytes = dtype_bytes(dtype);
    if (!fits(grad, bytes) || !fits(out, bytes) || !fits(upstream, 4)) return SL_ERR_ALIGNMENT;
    if (n == 0) return SL_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == SL_F32 ? launch_loss_backward<float>((const float*)grad, upstream, (float*)out, n, st) : launch_loss_backward<bf16>((const bf16*)grad, upstream, (bf16*)out, n, st);
}

}  // extern "C"

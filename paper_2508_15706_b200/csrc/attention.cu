// Attention over a packed batch for sm_100a: host side of the C ABI declared in include/sparseloco.h, over the kernels in
//   attention_forward.cuh   bfloat16 heads of up to 128 values on the tensor cores
//   attention_backward.cuh  their gradients
//   attention_plain.cuh     fp32 multiply-adds: any type, any strides, heads of up to 256 values
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <atomic>

#include "sparseloco.h"

#include "host.cuh"
#include "inner_common.cuh"
#include "attention_common.cuh"
#include "attention_plain.cuh"
#include "attention_forward.cuh"
#include "attention_backward.cuh"

namespace {

enum { kForward, kBackward };

sl_status attention_check(const sl_attention_desc* d) {
    if (!d || d->tokens < 0 || d->q_heads < 1 || d->kv_heads < 1 || d->head_dim < 1 || d->q_heads % d->kv_heads) return SL_ERR_INVALID_ARG;
    if (!known_dtype(d->dtype)) return SL_ERR_UNSUPPORTED;
    if ((d->causal != 0 && d->causal != 1) || (d->fill_rest != 0 && d->fill_rest != 1) || !(isfinite(d->scale) && d->scale > 0.0f)) return SL_ERR_INVALID_ARG;
    if (d->head_dim > 256 || d->tokens > (1ll << 30) || d->q_heads > 65535 || d->sequences > (1ll << 30)) return SL_ERR_TOO_LARGE;
    if ((d->tokens + 31) / 32 * d->q_heads > 0x7FFFFFFFll) return SL_ERR_TOO_LARGE;
    return SL_OK;
}

// How many CTAs share a tile of keys (dk, dv) or of queries (dq).  Where the tiles are fewer than fill the GPU some times over, and a tile has
// rounds enough (of 128 x 128 on the tensor cores, 3000 cycles each, or of 64 x 32 in fp32, 20000), its rounds are split: what that costs are fp32 sums
// through memory, 1 KB a token and part.  The lengths are on the device; their mean stands in for them.  Wanted are 3 CTAs for each of 148 SMs on the tensor cores and 12 in fp32
// (8: 1501 tokens, 10 heads of 128 on 5, 801 us in place of 780), numbers and not the device's, so that the workspace's size needs no device.
struct Parts {
    int kv, q;
};
int parts_of(double rounds, double least, double ctas, double wanted) {
    const double p = std::min(std::min(wanted / ctas, rounds / least), 8.0);
    return p >= 2.0 ? (int)p : 1;
}
Parts attention_parts(const sl_attention_desc* d, bool with_offsets, bool tensor) {
    const double length = with_offsets ? (double)d->tokens / (double)std::max<int64_t>(1, d->sequences) : (double)d->seq, group = (double)d->q_heads / d->kv_heads;
    const int64_t tile = tensor ? 128 : d->head_dim <= 128 ? 64 : 32, step = tensor ? 128 : d->head_dim <= 64 ? 64 : 32;
    const double tiles = (double)((d->tokens + tile - 1) / tile), rounds = std::max(1.0, length / (double)step * (d->causal ? 0.5 : 1.0)), least = tensor ? 8.0 : 2.0, wanted = 148.0 * (tensor ? 3.0 : 12.0);
    Parts p;
    p.kv = parts_of(rounds * group, least, tiles * d->kv_heads, wanted);
    p.q = parts_of(rounds, least, tiles * d->q_heads, wanted);
    return p;
}
int part_width(const sl_attention_desc* d) { return (d->head_dim + 3) / 4 * 4; }
// floats behind the statistics
size_t part_floats(const sl_attention_desc* d, const Parts& p) {
    const size_t row = (size_t)d->tokens * part_width(d);
    return (p.kv > 1 ? 2 * (size_t)p.kv * d->kv_heads * row : 0) + (p.q > 1 ? (size_t)p.q * d->q_heads * row : 0);
}

int64_t stat_pitch(const sl_attention_desc* d) { return (d->tokens + 127) / 128 * 128; }

struct Operand {
    const void* p;
    int64_t token, head;
    int heads;
    bool out;
};

// Strides that are never used (one head, one token) count as the head's width; an output's rows must lie apart.
sl_status attention_operand(const sl_attention_desc* d, Operand& o) {
    if (o.token < 0 || o.head < 0 || o.token > (1ll << 40) || o.head > (1ll << 40)) return SL_ERR_INVALID_ARG;
    if (o.heads == 1) o.head = d->head_dim;
    if (d->tokens == 1) o.token = (int64_t)o.heads * d->head_dim;
    if (!fits(o.p, dtype_bytes(d->dtype))) return SL_ERR_ALIGNMENT;
    if (!o.out) return SL_OK;
    const bool token_outer = d->tokens > 1 && (o.heads == 1 || o.token >= o.head);
    const int64_t inner = token_outer ? o.head : o.token, outer = token_outer ? o.token : o.head;
    const int64_t n_inner = token_outer ? o.heads : d->tokens, n_outer = token_outer ? d->tokens : o.heads;
    if ((n_inner > 1 && inner < d->head_dim) || (n_outer > 1 && outer < (n_inner - 1) * inner + d->head_dim)) return SL_ERR_INVALID_ARG;
    return SL_OK;
}

sl_status attention_args(AttnArgs& a, const sl_attention_desc* d, const int32_t* offsets) {
    memset(&a, 0, sizeof(a));
    a.parts_kv = a.parts_q = 1;
    if (offsets ? d->sequences < 0 : (d->tokens > 0 && (d->seq < 1 || d->tokens % d->seq))) return SL_ERR_INVALID_ARG;
    if (!fits(offsets, 4)) return SL_ERR_ALIGNMENT;
    a.offsets = offsets;
    a.sequences = (int)d->sequences;
    a.tokens = (int)d->tokens;
    a.seq = (int)std::min<int64_t>(d->seq, 1ll << 30);
    a.q_heads = d->q_heads;
    a.kv_heads = d->kv_heads;
    a.group = d->q_heads / d->kv_heads;
    a.dim = d->head_dim;
    a.causal = d->causal;
    a.fill = d->fill_rest;
    a.scale = d->scale;
    a.c = (float)((double)d->scale * 1.4426950408889634);
    return SL_OK;
}

// whether every row of every matrix may be taken by 4 elements at a time
bool by_fours(const sl_attention_desc* d, const Operand* ops, int n) {
    bool ok = d->head_dim % 4 == 0;
    for (int i = 0; i < n; ++i) ok = ok && fits(ops[i].p, 4 * dtype_bytes(d->dtype)) && ops[i].token % 4 == 0 && ops[i].head % 4 == 0;
    return ok;
}

AttnPlace place(const Operand& o) {
    AttnPlace p = {o.token, o.head};
    return p;
}

// Leave for a kernel's shared memory, asked for once per device (the call costs as much as a third of a launch).
template <auto KERNEL>
sl_status allow_shared(int bytes) {
    static std::atomic<uint64_t> asked{0};
    int dev = 0;
    SL_CUDA(cudaGetDevice(&dev));
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (bit && (asked.load(std::memory_order_relaxed) & bit)) return SL_OK;
    SL_CUDA(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    asked.fetch_or(bit, std::memory_order_relaxed);
    return SL_OK;
}
#define SL_TRY(call)                         \
    do {                                     \
        const sl_status s_ = (call);         \
        if (s_ != SL_OK) return s_;          \
    } while (0)

template <auto KERNEL>
sl_status launch_plain(const AttnArgs& a, long long ctas, int parts, size_t floats, cudaStream_t st) {
    SL_TRY(allow_shared<KERNEL>((int)(floats * 4)));
    KERNEL<<<dim3((unsigned)ctas, (unsigned)parts), kPlainThreads, floats * 4, st>>>(a);
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}

template <class T, int DMAX, int TILE>
sl_status plain_launches(const AttnArgs& a, int what, cudaStream_t st) {
    const long long tiles = (a.tokens + TILE - 1) / TILE;
    if (what == kForward) return launch_plain<plain_forward_kernel<T, DMAX, TILE>>(a, tiles * a.q_heads, 1, plain_floats(DMAX, TILE, 1, 2), st);
    SL_TRY((launch_plain<plain_dkv_kernel<T, DMAX, TILE>>(a, tiles * a.kv_heads, a.parts_kv, plain_floats(DMAX, TILE, 2, 2), st)));
    return launch_plain<plain_dq_kernel<T, DMAX, TILE>>(a, tiles * a.q_heads, a.parts_q, plain_floats(DMAX, TILE, 2, 2), st);
}

template <class T>
sl_status attention_plain(const AttnArgs& a, int what, cudaStream_t st) {
    return a.dim <= 64 ? plain_launches<T, 64, 64>(a, what, st) : a.dim <= 128 ? plain_launches<T, 128, 64>(a, what, st) : plain_launches<T, 256, 32>(a, what, st);
}

// Whether a matrix can be copied by tiles: bfloat16, heads of whole 16-byte pieces, and everything on 16-byte boundaries.
bool by_tiles(const sl_attention_desc* d, const Operand* ops, int n) {
    bool ok = d->dtype == SL_BF16 && d->head_dim <= 128 && d->head_dim % 8 == 0;
    for (int i = 0; i < n; ++i) ok = ok && !misaligned(ops[i].p) && ops[i].token % 8 == 0 && ops[i].head % 8 == 0 && ops[i].token > 0 && ops[i].head > 0 && ops[i].token < (1ll << 38) && ops[i].head < (1ll << 38);
    return ok;
}

// 64 values by `rows` tokens of one head; the outer dimensions in the order of their strides (*swapped: tokens lie inside heads)
bool tile_map(TileMap* m, int* swapped, const sl_attention_desc* d, const Operand& o, int rows) {
    const TmaEncodeFn encode = tma_encode_fn();
    if (!encode) return false;
    *swapped = o.token < o.head;
    const cuuint64_t tokens = (cuuint64_t)d->tokens, heads = (cuuint64_t)o.heads;
    const cuuint64_t dims[3] = {(cuuint64_t)d->head_dim, *swapped ? tokens : heads, *swapped ? heads : tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)(*swapped ? o.token : o.head) * 2, (cuuint64_t)(*swapped ? o.head : o.token) * 2};
    const cuuint32_t box[3] = {64, *swapped ? (cuuint32_t)rows : 1u, *swapped ? 1u : (cuuint32_t)rows}, steps[3] = {1, 1, 1};
    return encode(&m->map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
sl_status launch_forward(const AttnArgs& a, const TileMap* m, int swapped, cudaStream_t st) {
    SL_TRY(allow_shared<attention_forward_kernel<D>>(FwdShape<D>::kSmem));
    const long long ctas = (long long)((a.tokens + 255) / 256) * a.q_heads;
    attention_forward_kernel<D><<<(unsigned)ctas, kFwdThreads, FwdShape<D>::kSmem, st>>>(a, m[0], m[1], m[2], swapped);
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}

// A kernel of the backward pass, which may begin before the one in front of it has ended.
template <auto KERNEL>
sl_status launch_early(dim3 grid, int smem, cudaStream_t st, const AttnArgs& a, const TileMap* m, int swapped) {
    cudaLaunchConfig_t lc;
    memset(&lc, 0, sizeof(lc));
    lc.gridDim = grid;
    lc.blockDim = dim3(kBwdThreads);
    lc.dynamicSmemBytes = (size_t)smem;
    lc.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 1;
    SL_CUDA(cudaLaunchKernelEx(&lc, KERNEL, a, m[0], m[1], m[2], m[3], swapped));
    return SL_OK;
}

template <int D>
sl_status launch_backward(const AttnArgs& a, const TileMap* m, int swapped, cudaStream_t st) {
    SL_TRY(allow_shared<attention_dkv_kernel<D>>(BwdShape<D>::kSmem));
    SL_TRY(allow_shared<attention_dq_kernel<D>>(BwdShape<D>::kSmem));
    const long long tiles = (a.tokens + 127) / 128;
    SL_TRY((launch_early<attention_dkv_kernel<D>>(dim3((unsigned)(tiles * a.kv_heads), (unsigned)a.parts_kv), BwdShape<D>::kSmem, st, a, m, swapped)));
    SL_TRY((launch_early<attention_dq_kernel<D>>(dim3((unsigned)(tiles * a.q_heads), (unsigned)a.parts_q), BwdShape<D>::kSmem, st, a, m, swapped)));
    return SL_OK;
}

template <class T>
sl_status launch_stats(const AttnArgs& a, bool wide, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T), kPer = kPlainThreads / 16 * kStatTokens;  // tokens of a CTA
    const dim3 grid((unsigned)((a.pitch + kPer - 1) / kPer), (unsigned)a.q_heads);
    if (wide) attention_stats_kernel<T, V><<<grid, kPlainThreads, 0, st>>>(a);
    else attention_stats_kernel<T, 1><<<grid, kPlainThreads, 0, st>>>(a);
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}

template <class T>
sl_status launch_join(const AttnArgs& a, const float* from, void* to, AttnPlace st, int heads, int parts, float by, cudaStream_t stream) {
    int n_sms = 0;
    const sl_status s = sm_count(&n_sms);
    if (s != SL_OK) return s;
    const long long items = (long long)a.tokens * heads * (a.width / 4);
    attention_join_kernel<T><<<(unsigned)std::min<long long>((items + kPlainThreads - 1) / kPlainThreads, 16ll * n_sms), kPlainThreads, 0, stream>>>(a, from, to, st, heads, parts, by);
    SL_CUDA(cudaGetLastError());
    return SL_OK;
}
template <class T>
sl_status launch_joins(const AttnArgs& a, cudaStream_t st) {
    sl_status s = SL_OK;
    if (a.parts_kv > 1) {
        s = launch_join<T>(a, a.part_dk, a.dk, a.sdk, a.kv_heads, a.parts_kv, a.scale, st);
        if (s == SL_OK) s = launch_join<T>(a, a.part_dv, a.dv, a.sdv, a.kv_heads, a.parts_kv, 1.0f, st);
    }
    if (s == SL_OK && a.parts_q > 1) s = launch_join<T>(a, a.part_dq, a.dq, a.sdq, a.q_heads, a.parts_q, a.scale, st);
    return s;
}

}  // namespace

extern "C" {

sl_status sl_attention_forward(const sl_attention_desc* d, const void* q, const void* k, const void* v, const int32_t* offsets, void* o, float* lse, void* stream) {
    sl_status s = attention_check(d);
    if (s != SL_OK) return s;
    AttnArgs a;
    s = attention_args(a, d, offsets);
    if (s != SL_OK) return s;
    if (d->tokens == 0) return SL_OK;
    if (!q || !k || !v || !o || !lse) return SL_ERR_INVALID_ARG;
    for (const void* p : {q, k, v, (const void*)offsets})
        if (p == o || p == (const void*)lse) return SL_ERR_INVALID_ARG;
    if (o == (void*)lse) return SL_ERR_INVALID_ARG;
    if (!fits(lse, 4)) return SL_ERR_ALIGNMENT;
    Operand ops[] = {{q, d->q_token, d->q_head, d->q_heads, false}, {k, d->k_token, d->k_head, d->kv_heads, false}, {v, d->v_token, d->v_head, d->kv_heads, false},
                     {o, d->o_token, d->o_head, d->q_heads, true}};
    for (Operand& x : ops)
        if ((s = attention_operand(d, x)) != SL_OK) return s;
    a.q = q;
    a.k = k;
    a.v = v;
    a.o = o;
    a.lse = lse;
    a.sq = place(ops[0]);
    a.sk = place(ops[1]);
    a.sv = place(ops[2]);
    a.so = place(ops[3]);
    a.vec = by_fours(d, ops, 4);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (by_tiles(d, ops, 4)) {
        TileMap m[3];
        int swapped = 0, one = 0;
        bool ok = true;
        for (int i = 0; i < 3 && ok; ++i) {
            ok = tile_map(&m[i], &one, d, ops[i], 128);
            swapped |= one << i;
        }
        if (ok) return d->head_dim <= 64 ? launch_forward<64>(a, m, swapped, st) : launch_forward<128>(a, m, swapped, st);
    }
    return d->dtype == SL_F32 ? attention_plain<float>(a, kForward, st) : attention_plain<bf16>(a, kForward, st);
}

sl_status sl_attention_workspace_bytes(const sl_attention_desc* d, size_t* bytes) {
    const sl_status s = attention_check(d);
    if (s != SL_OK) return s;
    if (!bytes) return SL_ERR_INVALID_ARG;
    // (enough for either kind of kernels, with or without offsets: which it is depends on the addresses)
    size_t most = 0;
    for (int i = 0; i < 4; ++i) most = std::max(most, part_floats(d, attention_parts(d, i & 1, i >> 1)));
    *bytes = up256((2 * (size_t)stat_pitch(d) * d->q_heads + most) * 4);
    return SL_OK;
}

sl_status sl_attention_backward(const sl_attention_desc* d, const void* dout, const void* q, const void* k, const void* v, const void* o, const float* lse, const int32_t* offsets, void* dq,
                                void* dk, void* dv, void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    sl_status s = sl_attention_workspace_bytes(d, &need);
    if (s != SL_OK) return s;
    AttnArgs a;
    s = attention_args(a, d, offsets);
    if (s != SL_OK) return s;
    if (d->tokens == 0) return SL_OK;
    if (!dout || !q || !k || !v || !o || !lse || !dq || !dk || !dv) return SL_ERR_INVALID_ARG;
    const void* outs[] = {dq, dk, dv};
    for (int i = 0; i < 3; ++i) {
        for (const void* p : {dout, q, k, v, o, (const void*)lse, (const void*)offsets, (const void*)workspace})
            if (p == outs[i]) return SL_ERR_INVALID_ARG;
        if (outs[i] == outs[(i + 1) % 3]) return SL_ERR_INVALID_ARG;
    }
    if (!fits(lse, 4) || misaligned(workspace)) return SL_ERR_ALIGNMENT;
    Operand ops[] = {{q, d->q_token, d->q_head, d->q_heads, false},     {k, d->k_token, d->k_head, d->kv_heads, false},   {v, d->v_token, d->v_head, d->kv_heads, false},
                     {o, d->o_token, d->o_head, d->q_heads, false},     {dout, d->do_token, d->do_head, d->q_heads, false}, {dq, d->dq_token, d->dq_head, d->q_heads, true},
                     {dk, d->dk_token, d->dk_head, d->kv_heads, true}, {dv, d->dv_token, d->dv_head, d->kv_heads, true}};
    for (Operand& x : ops)
        if ((s = attention_operand(d, x)) != SL_OK) return s;
    if (!workspace || workspace_bytes < need) return SL_ERR_NOMEM;
    a.q = q;
    a.k = k;
    a.v = v;
    a.o_in = o;
    a.dout = dout;
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    a.lse = const_cast<float*>(lse);
    a.pitch = stat_pitch(d);
    a.nlse2 = static_cast<float*>(workspace);
    a.ndelta = a.nlse2 + a.pitch * d->q_heads;
    a.sq = place(ops[0]);
    a.sk = place(ops[1]);
    a.sv = place(ops[2]);
    a.so = place(ops[3]);
    a.sdo = place(ops[4]);
    a.sdq = place(ops[5]);
    a.sdk = place(ops[6]);
    a.sdv = place(ops[7]);
    a.vec = by_fours(d, ops, 8);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int piece = 16 / dtype_bytes(d->dtype);
    bool wide = d->head_dim % piece == 0;
    for (int i : {3, 4}) wide = wide && !misaligned(ops[i].p) && ops[i].token % piece == 0 && ops[i].head % piece == 0;
    s = d->dtype == SL_F32 ? launch_stats<float>(a, wide, st) : launch_stats<bf16>(a, wide, st);
    if (s != SL_OK) return s;
    TileMap m[4];
    const int which[4] = {0, 1, 2, 4};  // q, k, v, dout
    int swapped = 0;
    bool tensor = by_tiles(d, ops, 8);
    for (int i = 0; i < 4 && tensor; ++i) {
        int one = 0;
        tensor = tile_map(&m[i], &one, d, ops[which[i]], d->head_dim <= 64 ? BwdShape<64>::kRound : BwdShape<128>::kRound);
        swapped |= one << i;
    }
    const Parts parts = attention_parts(d, offsets != nullptr, tensor);
    a.parts_kv = parts.kv;
    a.parts_q = parts.q;
    a.width = part_width(d);
    const size_t row = (size_t)d->tokens * a.width;
    a.part_dk = a.ndelta + a.pitch * d->q_heads;
    a.part_dv = a.part_dk + (parts.kv > 1 ? parts.kv * d->kv_heads * row : 0);
    a.part_dq = a.part_dv + (parts.kv > 1 ? parts.kv * d->kv_heads * row : 0);
    if (tensor) s = d->head_dim <= 64 ? launch_backward<64>(a, m, swapped, st) : launch_backward<128>(a, m, swapped, st);
    else s = d->dtype == SL_F32 ? attention_plain<float>(a, kBackward, st) : attention_plain<bf16>(a, kBackward, st);
    if (s != SL_OK) return s;
    return d->dtype == SL_F32 ? launch_joins<float>(a, st) : launch_joins<bf16>(a, st);
}

}  // extern "C"

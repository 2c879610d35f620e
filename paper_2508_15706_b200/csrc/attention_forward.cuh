// Attention forward on the tensor cores: bfloat16 heads of up to 64 or 128 values.  Part of libsparseloco (attention.cu).
//
// One CTA: two tiles of 128 queries of one head.  Per tile of 128 keys, for each of the two: S = Q K^T (tensor memory, 128 columns), a warpgroup
// turns S into P = exp2(c S - c m) with one row per thread and writes it as bfloat16 pairs over S, then O += P V (128 or 64 columns).  A
// third group of warps feeds them: one thread issues every product, one every copy (K and V tiles through a ring), one warp clears rows.  While one
// tile's S is with its warpgroup, the tensor cores work on the other's, so the two take turns, and K and V are read once for 256 queries.  With
// D = 128 a tile pair costs 2048 cycles of products and 2 x 16384 exponentials, 2048 cycles at 16 a cycle: both bound.  So part of the exponentials are
// formed by multiply-adds (1 of 8: 32768 tokens 3.75 -> 3.60 ms in a short run; 2 of 8 3.77 ms, 4 of 8 3.99), and m, the row's reference, follows the
// maximum only when that has moved by more than 2^8 (P may be as large as that; sums and O are fp32), which spares O's rescaling.
// P is rounded to bfloat16 as an operand: 2^-8 of its size at most on either side, beside the output's own rounding.
//
// Measured, 16 heads of 128 on 4, bfloat16, causal: 32768 tokens 3.50 ms from a graph (1258 TFLOP/s, 77 % of what a library product reaches in a
// burst, 91 % of what it holds), 4.0 ms in a loop at the power limit; 4 x 4096 tokens 275 to 340 us with the clock, 12 heads of 64 190 to 225 us.  37 tokens 7.4 us: one
// CTA's way from the launch through offsets, copies, two products and the store.  Steps: issuing behind elect.sync 4.39 -> 4.04 ms; no select for masked exponentials
// 3.62 -> 3.48.  V of a round and K of the next behind one barrier made no difference.  The compiler fits 168 registers, those of the launch, and spills 144
// bytes a thread, though the split leaves 216.
//
// Masked scores become -inf.  Their P is 0, but 0 times an infinity or NaN in V is not.  (A NaN score stays NaN on either way to an exponential, so that the row's sums show it.)  Rows of V outside every sequence (padding may hold
// anything) are set to 0 in shared memory; for the rest, a row whose output is not finite is taken again, with its whole tile, by the
// fp32 code, which passes over what is masked.
#pragma once
#include "attention_common.cuh"
#include "attention_plain.cuh"
#include "tensor_core.cuh"

namespace {

constexpr int kFwdThreads = 384;  // two warpgroups for P, one that issues (168 registers a thread at launch: 64512; after the split 2 x 128 x 216 + 128 x 72, the same)
constexpr float kFwdSlack = 8.0f;
constexpr int kFwdPoly = 1;  // of 8 exponentials by multiply-adds

template <int D>
struct FwdShape {
    static constexpr int kTile = D / 64 * 16384;         // bytes of 128 rows
    static constexpr int kStages = D == 128 ? 5 : 6;     // K and V tiles in flight
    static constexpr int kSmem = (2 + kStages) * kTile + 1024;
};

struct FwdShared {
    unsigned long long q_full[2], s_full[2], p_full[2], o_full[2], kv_full[6], kv_empty[6], drained;
    Cleaner cleaner;
    int4 ranges[8];
    int failed, again[2];
    unsigned tmem;
};

// first and last tile of keys that rows of a tile see, the largest beginning and the smallest end, from those of its four warps
__device__ __forceinline__ int4 tile_ranges(const int4* w) {
    int4 r = w[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) r = make_int4(min(r.x, w[i].x), max(r.y, w[i].y), max(r.z, w[i].z), min(r.w, w[i].w));
    return r;
}
// of a warp's rows: rows that see nothing do not count
__device__ __forceinline__ int4 warp_ranges(int2 see) {
    const bool in = see.y > 0;
    return make_int4(__reduce_min_sync(kFullMask, in ? see.x : 0x7FFFFFFF), __reduce_max_sync(kFullMask, in ? see.y : 0), __reduce_max_sync(kFullMask, in ? see.x : 0),
                     __reduce_min_sync(kFullMask, in ? see.y : 0x7FFFFFFF));
}

// A warp's 32 rows of an accumulator as bfloat16, N columns; returns whether all values of the thread's row are finite.  Rows go through 4 KB
// of shared memory (16-byte pieces, exchanged within a row's 8 by the row's number, so that neither side meets a bank twice), from where neighbouring
// lanes store neighbouring pieces: by one row per lane every store touched 32 lines, 3000 cycles a tile.  `first`: the token of lane 0.
template <int N>
__device__ __forceinline__ bool store_rows(unsigned at, bool any, bool in, bool store, float by, bf16* rows, long long token, int first, int dim, unsigned buffer, int lane) {
    constexpr int kPart = N < 64 ? N : 64, kPieces = kPart / 8, kRows = 32 / kPieces;  // columns at a time, pieces of a row, rows of one store
    const unsigned stored = __ballot_sync(kFullMask, store);
    bool fine = true;
#pragma unroll
    for (int c = 0; c < N; c += kPart) {
#pragma unroll
        for (int b = 0; b < kPart; b += 32) {
            float o[32];
            if (any) {
                tmem_load32(at + c + b, o);
                tmem_loaded(o);
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                o[j] = in ? o[j] * by : 0.0f;
                fine = fine && fabsf(o[j]) <= 3.4e38f;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned piece = (unsigned)(b / 8 + j) ^ (lane & (kPieces - 1));
                asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(buffer + lane * (kPieces * 16) + piece * 16), "r"(narrow2(make_float2(o[8 * j], o[8 * j + 1]))),
                             "r"(narrow2(make_float2(o[8 * j + 2], o[8 * j + 3]))), "r"(narrow2(make_float2(o[8 * j + 4], o[8 * j + 5]))), "r"(narrow2(make_float2(o[8 * j + 6], o[8 * j + 7])))
                             : "memory");
            }
        }
        __syncwarp();
        const int piece = lane % kPieces, d = c + piece * 8;
#pragma unroll
        for (int r = lane / kPieces; r < 32; r += kRows) {
            uint4 w;
            shared_load<16>(buffer + r * (kPieces * 16) + ((unsigned)piece ^ (r & (kPieces - 1))) * 16, &w);
            if ((stored >> r & 1) && d < dim) *reinterpret_cast<uint4*>(rows + (first + r) * token + d) = w;
        }
        __syncwarp();
    }
    return fine;
}

template <int D>
__global__ void __launch_bounds__(kFwdThreads, 1) attention_forward_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ TileMap mq, const __grid_constant__ TileMap mk,
                                                                           const __grid_constant__ TileMap mv, int swapped) {
    typedef FwdShape<D> Shape;
    extern __shared__ __align__(1024) unsigned char fwd_smem[];
    __shared__ FwdShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int pairs = (a.tokens + 255) / 256, head = blockIdx.x % a.q_heads, q0 = (pairs - 1 - (int)(blockIdx.x / a.q_heads)) * 256;
    const unsigned base = (shared_address(fwd_smem) + 1023u) & ~1023u;
    const unsigned sq = base, ring = base + 2 * Shape::kTile;
    auto bar = [&](const unsigned long long* b) { return shared_address(b); };
    volatile int* failed = &sh.failed;

    if (tid == 0) {
        sh.failed = sh.again[0] = sh.again[1] = 0;
        for (int i = 0; i < 2; ++i) {
            bar_init(bar(&sh.q_full[i]), 1);
            bar_init(bar(&sh.s_full[i]), 1);
            bar_init(bar(&sh.p_full[i]), 4);
            bar_init(bar(&sh.o_full[i]), 1);
        }
        for (int i = 0; i < Shape::kStages; ++i) {
            bar_init(bar(&sh.kv_full[i]), 1);
            bar_init(bar(&sh.kv_empty[i]), 1);
        }
        bar_init(bar(&sh.drained), 1);
        cleaner_init(sh.cleaner);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 8) tmem_alloc(shared_address(&sh.tmem), 512);
    int2 see = make_int2(0, 0);
    if (warp < 8) {
        see = keys_of(a, q0 + tid);
        const int4 r = warp_ranges(see);
        if (lane == 0) sh.ranges[warp] = r;
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const unsigned tmem = sh.tmem;
    int begin[2], end[2];  // tiles of keys of each tile of queries
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int4 r = tile_ranges(sh.ranges + 4 * x);
        begin[x] = r.y > 0 ? r.x / 128 : 0;
        end[x] = (r.y + 127) / 128;
    }
    const bool has[2] = {end[0] > begin[0], end[1] > begin[1]};
    const int first = has[0] ? (has[1] ? min(begin[0], begin[1]) : begin[0]) : begin[1], last = max(end[0], end[1]);
    const unsigned s_at[2] = {tmem, tmem + 128}, o_at[2] = {tmem + 256, tmem + 256 + D};

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 9 && elected()) {
            for (int x = 0; x < 2; ++x)
                if (has[x]) {
                    bar_expect(bar(&sh.q_full[x]), Shape::kTile);
                    for (int p = 0; p < D / 64; ++p) tile_load(sq + x * Shape::kTile + p * 16384, &mq, swapped & 1, p * 64, head, q0 + 128 * x, bar(&sh.q_full[x]));
                }
            const int kv = head / a.group;
            int n = 0;  // tiles issued: K, V, K, V ..
            bool ok = true;
            for (int t = first; t < last && ok; ++t)
                for (int v = 0; v < 2 && ok; ++v, ++n) {
                    const int st = n % Shape::kStages;
                    ok = bar_wait(bar(&sh.kv_empty[st]), ((n / Shape::kStages) & 1) ^ 1, failed);
                    if (!ok) break;
                    bar_expect(bar(&sh.kv_full[st]), Shape::kTile);
                    for (int p = 0; p < D / 64; ++p)
                        tile_load(ring + st * Shape::kTile + p * 16384, v ? &mv : &mk, swapped >> (1 + v) & 1, p * 64, kv, t * 128, bar(&sh.kv_full[st]));
                }
            if (!ok) {  // no copy may be on its way when the CTA ends
                const long long from = clock64();
                for (int m = max(0, n - Shape::kStages); m < n; ++m)
                    bar_settle(bar(&sh.kv_full[m % Shape::kStages]), (m / Shape::kStages) & 1, from);
                for (int x = 0; x < 2; ++x)
                    if (has[x]) bar_settle(bar(&sh.q_full[x]), 0, from);
            }
        }
        const int2 live = live_tokens(a);
        const bool dead = last > first && dead_rows(first * 128, (last - first) * 128, live, a.tokens);  // V has rows outside every sequence
        if (warp == 10 && dead) cleaner_run<D, 128>(sh.cleaner, live, lane, failed);
        if (warp == 8 && last > first && elected()) {
            int n = 0;              // tiles of the ring taken
            unsigned asked = 0;
            bool ok = true;
            auto take = [&]() {
                const int st = n % Shape::kStages;
                ok = ok && bar_wait(bar(&sh.kv_full[st]), (n / Shape::kStages) & 1, failed);
                ++n;
                return st;
            };
            for (int x = 0; x < 2; ++x)
                if (has[x]) ok = ok && bar_wait(bar(&sh.q_full[x]), 0, failed);
            int k_stage = take(), used[2] = {0, 0};
            if (ok) {
                for (int x = 0; x < 2; ++x)
                    if (has[x] && begin[x] == first) {
                        product_rows<D>(s_at[x], sq + x * Shape::kTile, ring + k_stage * Shape::kTile);
                        products_to(bar(&sh.s_full[x]));
                    }
                products_to(bar(&sh.kv_empty[k_stage]));
            }
            for (int t = first; t < last && ok; ++t) {
                const int v_stage = take();
                if (t + 1 < last) k_stage = take();
                if (dead && dead_rows(t * 128, 128, live, a.tokens)) ok = ok && cleaner_ask(sh.cleaner, ring + v_stage * Shape::kTile, t * 128, asked, failed);
                if (!ok) break;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (has[x] && t >= begin[x] && t < end[x]) {
                        ok = ok && bar_wait(bar(&sh.p_full[x]), used[x] & 1, failed);
                        if (!ok) break;
                        ++used[x];
                        tmem_fence_after();
                        product_down<D>(o_at[x], s_at[x], ring + v_stage * Shape::kTile, t > begin[x]);
                        if (t == end[x] - 1) products_to(bar(&sh.o_full[x]));
                    }
                    if (has[x] && t + 1 >= begin[x] && t + 1 < end[x]) {
                        product_rows<D>(s_at[x], sq + x * Shape::kTile, ring + k_stage * Shape::kTile);
                        products_to(bar(&sh.s_full[x]));
                    }
                }
                products_to(bar(&sh.kv_empty[v_stage]));
                if (t + 1 < last) products_to(bar(&sh.kv_empty[k_stage]));
            }
            if (dead) cleaner_ask(sh.cleaner, 0, 0, asked, failed);
            if (!ok) {
                products_to(bar(&sh.drained));
                bar_settle(bar(&sh.drained), 0, clock64());
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int x = warp >> 2;  // which tile of queries
        const unsigned lanes = (unsigned)(warp & 3) << 21, s_t = s_at[x] + lanes, o_t = o_at[x] + lanes;
        const int4 mine = sh.ranges[warp];
        const bool in = see.y > 0;
        float top = -INFINITY;  // the reference that P and O are scaled by
        float2 sum2 = make_float2(0.0f, 0.0f);
        bool ok = true;
        int round = 0;
        if (has[x])
            for (int t = begin[x]; t < end[x]; ++t, ++round) {
                ok = bar_wait(bar(&sh.s_full[x]), round & 1, failed) && ok;  // (after a failure the rest of the waits end at once)
                __syncwarp();
                tmem_fence_after();
                float s[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_load32(s_t + 32 * i, s[i]);
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_loaded(s[i]);
                const int k0 = t * 128;
                if (k0 < mine.z) {
                    const int lo = see.x - k0;
#pragma unroll
                    for (int i = 0; i < 128; ++i) s[i / 32][i % 32] = i >= lo ? s[i / 32][i % 32] : -INFINITY;
                }
                if (k0 + 128 > mine.w) {
                    const int hi = see.y - k0;
#pragma unroll
                    for (int i = 0; i < 128; ++i) s[i / 32][i % 32] = i < hi ? s[i / 32][i % 32] : -INFINITY;
                }
                float best[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    best[i] = s[i][0];
#pragma unroll
                    for (int j = 1; j < 32; ++j) best[i] = fmaxf(best[i], s[i][j]);
                }
                const float high = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
                if (round == 0) {
                    top = high;
                } else if (__any_sync(kFullMask, (high - top) * a.c > kFwdSlack)) {  // (-inf to -inf: NaN, not above)
                    const float next = fmaxf(high, top);
                    const float by = next == top ? 1.0f : exp2_fast((top - next) * a.c);
                    top = next;
                    sum2 = mul2(sum2, both(by));
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        float o[32];
                        tmem_load32(o_t + 32 * i, o);
                        tmem_loaded(o);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] *= by;
                        tmem_store32(o_t + 32 * i, o);
                    }
                }
                const float from = top == -INFINITY ? 0.0f : -top * a.c;
                const float2 c2 = both(a.c), from2 = both(from);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    unsigned w[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float2 e = fma2(make_float2(s[i][2 * j], s[i][2 * j + 1]), c2, from2);
                        const float2 p = exp2_pair<kFwdPoly>(e, j);  // (0 of -inf, and NaN stays: a row with one is found by its sums)
                        sum2 = add2(sum2, p);
                        w[j] = narrow2(p);
                    }
                    tmem_store16(s_t + 16 * i, w);
                }
                tmem_stored();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(bar(&sh.p_full[x]));
            }
        const int i = q0 + tid;
        if (has[x]) ok = bar_wait(bar(&sh.o_full[x]), 0, failed) && ok;
        __syncwarp();
        tmem_fence_after();
        const float sum = sum2.x + sum2.y, inv = in ? (ok ? 1.0f / sum : NAN) : 0.0f;
        const bool store = i < a.tokens && (in || a.fill);
        bf16* rows = static_cast<bf16*>(a.o) + head * a.so.head;
        bool fine = store_rows<D>(o_t, has[x], in, store, inv, rows, a.so.token, i - lane, a.dim, sq + x * Shape::kTile + (warp & 3) * 4096, lane);
        fine = fine && isfinite(top);
        if (store) a.lse[(long long)head * a.tokens + i] = in ? (ok ? logf(sum) - (top == -INFINITY ? 0.0f : -top * a.c) * kLn2 : NAN) : -INFINITY;
        if (in && ok && !fine) sh.again[x] = 1;
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 8) {
        tmem_fence_after();
        tmem_free(tmem, 512);
    }
    if (sh.failed || tid >= 256) return;
    for (int x = 0; x < 2; ++x)
        if (sh.again[x])
            for (int half = 0; half < 2; ++half) plain_forward_tile<bf16, D, 64>(a, q0 + 128 * x + 64 * half, head, reinterpret_cast<float*>(fwd_smem), tid);
}

}  // namespace

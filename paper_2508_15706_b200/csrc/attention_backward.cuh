// Attention backward on the tensor cores: bfloat16 heads of up to 64 or 128 values.  Part of libsparseloco (attention.cu).
//
// Two kernels that each form P and dS anew, so that every gradient is summed inside one CTA, in a fixed order, without atomics or fp32
// copies of dq: 7 products per tile where one kernel would need 5, but one of those five (dq of all keys) would go through memory.
//   dk, dv   one CTA: 128 keys of one key/value head, over all queries of its group.  Keys are the rows throughout:
//            S^T = K Q^T, dP^T = V dO^T (128 columns each), dV += P^T dO, dK += dS^T Q, P^T and dS^T bfloat16 pairs over S^T and dP^T.
//            512 columns of tensor memory with D = 128, all of them.
//   dq       one CTA: 128 queries of one head.  S = Q K^T (two buffers), dP = dO V^T, dQ += dS K, dS over S.
// Two warpgroups form P and dS, each half of the columns, one row per thread and half; one thread issues the products, one the copies.
// The products of the next tile run while exponentials of this one are formed.  Per tile of 128 x 128 and D = 128: dk, dv 2048 cycles of products,
// dq 1536, 16384 exponentials 1024 cycles each.
//
// dq needs nothing of dk and dv: its kernel begins as soon as the other's last CTAs have begun, and fills the SMs that run out of tiles of keys.
//
// Measured, bfloat16, causal, with the statistics: 4 x 4096 tokens, 16 heads of 128 on 4, 807 us from a graph (852 TFLOP/s counting the 5 products, 1193
// with the 7 that run), 915 to 960 in a loop; 6007 tokens in 23 sequences, 12 heads of 64, 80 us (two CTAs an SM leave 80 registers a thread: dk, dv spills 84 bytes, dq 60).  A round of dk, dv takes 3200 cycles, of dq 2400, with the
// tensor cores at work 63 % of them.  What was tried: two streams of 64-row items with a warpgroup each (4190 and 3390 cycles: a wait costs the
// issuing thread 200 cycles even when there is nothing to wait for, and there were twice as many); four warpgroups to a round in place of two (the same
// within 3 %); `lane == 0` in place of elect.sync (3990 and 3080).  Of 8 exponentials 1 goes by multiply-adds (0: 2 % slower, 3: 3 % with heads of 64).
//
// The rows' statistics come as -lse / ln 2 and -delta, fp32, padded to whole tiles, with the tile they belong to.
#pragma once
#include "attention_common.cuh"
#include "attention_forward.cuh"
#include "attention_plain.cuh"
#include "tensor_core.cuh"

namespace {

constexpr int kBwdThreads = 384;
constexpr int kBwdPoly = 1;  // of 8 exponentials by multiply-adds

// Rings: Q (K in dq) is needed from its scores to its part of the sum, a whole round, dO (V) for half of one; a copy takes more than 1000 cycles to
// arrive.  So Q and K have three stages and dO and V two, which fills shared memory with D = 128 (a common ring of 4 had the products wait 800 cycles a round).
//
// Heads of up to 64 values take rounds of 64 (R) instead, half of everything, so that two CTAs share an SM: their products are too short for one's threads to
// hide, and a ragged batch's tiles have few rounds between a beginning and an end of 4000 cycles each.
template <int D>
struct BwdShape {
    static constexpr int kRound = D == 128 ? 128 : 64, kCtas = D == 128 ? 1 : 2;  // rows of a round, CTAs an SM
    static constexpr int kOwn = D / 64 * 16384;                                   // bytes of the CTA's own 128 rows
    static constexpr int kTile = D / 64 * kRound * 128;                           // of a round's
    static constexpr int kA = D == 128 ? 3 : 4, kB = D == 128 ? 2 : 4;            // stages
    static constexpr int kStats = 8 * kRound;                                     // -lse / ln 2 and -delta of a round's queries, two stages
    static constexpr int kPlain = plain_floats(D, 64, 2, 2) * 4;
    static constexpr int kColumns = 2 * kRound + 2 * D;                           // of tensor memory: scores, dP, two sums (or two buffers of scores, dP, one sum)
    static constexpr int most(int x, int y) { return x > y ? x : y; }
    static constexpr int kShared = most(2 * kOwn + (kA + kB) * kTile + 2 * kStats, kPlain);  // where the shared state lies
    static constexpr int kSmem = kShared + 512;
};
static_assert(BwdShape<128>::kColumns == 512 && BwdShape<64>::kColumns == 256, "powers of two");

struct BwdShared {  // behind the tiles
    unsigned long long own_full, a_full[4], a_empty[4], b_full[4], b_empty[4], stat_full[2], stat_empty[2], s_full[2], p_full, dp_full, ds_full, done, drained;
    Cleaner cleaner;
    int4 ranges[4];
    int failed, again;
    unsigned tmem;
};
static_assert(sizeof(BwdShared) <= 512, "the shared state has 512 bytes");

__device__ __forceinline__ void bulk_load(unsigned to, const void* from, unsigned bytes, unsigned bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}

// a thread's half of a row as bfloat16 pairs, 16 to a store
template <int N>
__device__ __forceinline__ void store_pairs(unsigned at, const float2 (&p)[N]) {
#pragma unroll
    for (int i = 0; i < N / 16; ++i) {
        unsigned w[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = narrow2(p[16 * i + j]);
        tmem_store16(at + 16 * i, w);
    }
    tmem_stored();
    tmem_fence_before();
    __syncwarp();
}
// N columns of a row
template <int N>
__device__ __forceinline__ void load_columns(unsigned at, float (&s)[N / 32][32]) {
#pragma unroll
    for (int i = 0; i < N / 32; ++i) tmem_load32(at + 32 * i, s[i]);
#pragma unroll
    for (int i = 0; i < N / 32; ++i) tmem_loaded(s[i]);
}

// to[128, R] = a b^T over D values: a of 128 rows, b of R
template <int D, int R>
__device__ __forceinline__ void product_round(unsigned to, unsigned a, unsigned b) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        const unsigned step = (unsigned)(i % 4) * 32u, panel = (unsigned)(i / 4);
        product(to, tile_desc(a + panel * 16384u + step, 0), tile_desc(b + panel * (R * 128u) + step, 0), product_kind(R, false), i > 0);
    }
}
// to[128, D] (+)= p b over b's R rows; p's halves lie R / 2 columns apart
template <int D, int R>
__device__ __forceinline__ void product_halves(unsigned to, unsigned p, unsigned b, bool add) {
#pragma unroll
    for (int i = 0; i < R / 16; ++i) product_tmem(to, p + (i / (R / 32)) * (R / 2) + (i % (R / 32)) * 8u, tile_desc(b + 2048u * i, R * 128u), product_kind(D, true), add || i > 0);
}

// One row of an accumulator as fp32, N columns; returns whether all values are finite.
template <int N>
__device__ __forceinline__ bool store_part(unsigned at, bool any, bool in, bool store, bool ok, float* row, int width) {
    bool fine = true;
#pragma unroll
    for (int b = 0; b < N / 32; ++b) {
        float o[32];
        if (any) {
            tmem_load32(at + 32 * b, o);
            tmem_loaded(o);
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            o[j] = !in ? 0.0f : !ok ? NAN : any ? o[j] : 0.0f;
            fine = fine && fabsf(o[j]) <= 3.4e38f;
        }
#pragma unroll
        for (int j = 0; j < 32; j += 4)
            if (store && b * 32 + j < width) *reinterpret_cast<float4*>(row + b * 32 + j) = make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
    }
    return fine;
}

// The tiles' swizzle counts from multiples of 1024 bytes.  The kernels have no static shared memory, so that the dynamic one begins on such an address, as its
// declaration asks; with D = 128 it is too full for rounding up.  Should it ever lie elsewhere, nothing is copied and the results are NaN.
__device__ __forceinline__ bool swizzle_placed(unsigned at) { return (at & 1023u) == 0u; }

__device__ __forceinline__ void bwd_init(BwdShared& sh) {
    sh.failed = sh.again = 0;
    bar_init(shared_address(&sh.own_full), 1);
    for (int i = 0; i < 4; ++i) {
        bar_init(shared_address(&sh.a_full[i]), 1);
        bar_init(shared_address(&sh.a_empty[i]), 1);
        bar_init(shared_address(&sh.b_full[i]), 1);
        bar_init(shared_address(&sh.b_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
        bar_init(shared_address(&sh.stat_full[i]), 1);
        bar_init(shared_address(&sh.stat_empty[i]), 8);
        bar_init(shared_address(&sh.s_full[i]), 1);
    }
    bar_init(shared_address(&sh.p_full), 8);
    bar_init(shared_address(&sh.dp_full), 1);
    bar_init(shared_address(&sh.ds_full), 8);
    bar_init(shared_address(&sh.done), 1);
    bar_init(shared_address(&sh.drained), 1);
    cleaner_init(sh.cleaner);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// A ring's next stage and the parity of its barriers.
template <int STAGES>
struct Ring {
    unsigned at = 0, phase = 0;
    __device__ __forceinline__ void step() {
        if (++at == STAGES) {
            at = 0;
            phase ^= 1;
        }
    }
};
// No copy may be on its way when the CTA ends: after a failed wait, those issued are waited for, for as long again.
__device__ __forceinline__ void bwd_settle(const unsigned long long* full, int issued, int stages, long long from) {
    for (int m = max(0, issued - stages); m < issued; ++m) bar_settle(shared_address(&full[m % stages]), (m / stages) & 1, from);
}
__device__ __forceinline__ void bwd_drain(BwdShared& sh) {
    products_to(shared_address(&sh.drained));
    bar_settle(shared_address(&sh.drained), 0, clock64());
}

// Of a thread's columns those below `lo` and from `hi` on become 0.  A warp's rows mostly need one side only (the diagonal of a causal
// sequence, its first tile), which halves the comparisons.
template <int N>
__device__ __forceinline__ void mask_pairs(float2 (&p)[N], int lo, int hi, bool below, bool above) {
    if (below) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            p[i].x = 2 * i >= lo ? p[i].x : 0.0f;
            p[i].y = 2 * i + 1 >= lo ? p[i].y : 0.0f;
        }
    }
    if (above) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            p[i].x = 2 * i < hi ? p[i].x : 0.0f;
            p[i].y = 2 * i + 1 < hi ? p[i].y : 0.0f;
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kBwdThreads, BwdShape<D>::kCtas) attention_dkv_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ TileMap mq, const __grid_constant__ TileMap mk,
                                                                       const __grid_constant__ TileMap mv, const __grid_constant__ TileMap mdo, int swapped) {
    typedef BwdShape<D> Shape;
    constexpr int kA = Shape::kA, kB = Shape::kB, kTile = Shape::kTile, kOwn = Shape::kOwn, R = Shape::kRound, H = R / 2;  // H: columns of a thread
    extern __shared__ __align__(1024) unsigned char bwd_smem[];
    BwdShared& sh = *reinterpret_cast<BwdShared*>(bwd_smem + Shape::kShared);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int kv = blockIdx.x % a.kv_heads, k0 = (int)(blockIdx.x / a.kv_heads) * 128, part = blockIdx.y;
    const unsigned sk = shared_address(bwd_smem), sv = sk + kOwn, sq = sk + 2 * kOwn, sdo = sq + kA * kTile, stats = sdo + kB * kTile;
    volatile int* failed = &sh.failed;
    if (tid == 0) bwd_init(sh);
    if (warp == 8) tmem_alloc(shared_address(&sh.tmem), Shape::kColumns);
    int2 see = make_int2(0, 0);
    if (warp < 8) {
        see = queries_of(a, k0 + (tid & 127));
        const int4 r = warp_ranges(see);
        if (lane == 0 && warp < 4) sh.ranges[warp] = r;
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const unsigned tmem = sh.tmem, s_at = tmem, dp_at = tmem + R, dv_at = tmem + 2 * R, dk_at = tmem + 2 * R + D;
    const int4 all = tile_ranges(sh.ranges);
    const int first = all.y > 0 ? all.x / R : 0, tiles = (all.y + R - 1) / R - first;
    const int2 share = share_of(tiles * a.group, part, a.parts_kv);  // of the heads' tiles one after the other
    const bool placed = swizzle_placed(sk);
    const int round0 = share.x, rounds = placed ? share.y - share.x : 0;

    if (warp >= 8) {
        if (warp == 9 && elected()) {
            if (rounds > 0) {
                bar_expect(shared_address(&sh.own_full), 2 * kOwn);
                for (int p = 0; p < D / 64; ++p)
                    for (int r = 0; r < 128; r += R) {
                        tile_load(sk + p * 16384 + r * 128, &mk, swapped >> 1 & 1, p * 64, kv, k0 + r, shared_address(&sh.own_full));
                        tile_load(sv + p * 16384 + r * 128, &mv, swapped >> 2 & 1, p * 64, kv, k0 + r, shared_address(&sh.own_full));
                    }
            }
            // (A CTA without rounds waits too: that this kernel has ended has to mean that the one in front of it has, since dq waits for this one alone.)
            earlier_done();    // the statistics are there, for the loads below and for dq,
            next_may_begin();  // which may begin when every CTA has come as far
            bool ok = true;
            int round = 0, b_issued = 0;
            Ring<kA> ra;
            Ring<kB> rb;
            for (; round < rounds; ++round) {
                const int head = kv * a.group + (round0 + round) / tiles, t = (first + (round0 + round) % tiles) * R;
                const unsigned qb = shared_address(&sh.a_full[ra.at]), dob = shared_address(&sh.b_full[rb.at]), tb = shared_address(&sh.stat_full[round & 1]);
                if (!(ok = bar_wait(shared_address(&sh.a_empty[ra.at]), ra.phase ^ 1, failed))) break;
                bar_expect(qb, kTile);
                for (int p = 0; p < D / 64; ++p) tile_load(sq + ra.at * kTile + p * (R * 128), &mq, swapped & 1, p * 64, head, t, qb);
                ra.step();
                ok = bar_wait(shared_address(&sh.b_empty[rb.at]), rb.phase ^ 1, failed) && bar_wait(shared_address(&sh.stat_empty[round & 1]), (round >> 1 & 1) ^ 1, failed);
                if (!ok) {
                    ++round;
                    break;
                }
                bar_expect(dob, kTile);
                for (int p = 0; p < D / 64; ++p) tile_load(sdo + rb.at * kTile + p * (R * 128), &mdo, swapped >> 3 & 1, p * 64, head, t, dob);
                rb.step();
                const unsigned to = stats + (round & 1) * Shape::kStats;
                bar_expect(tb, Shape::kStats);
                bulk_load(to, a.nlse2 + head * a.pitch + t, 4 * R, tb);
                bulk_load(to + 4 * R, a.ndelta + head * a.pitch + t, 4 * R, tb);
                b_issued = round + 1;
            }
            if (!ok) {
                const long long from = clock64();
                bwd_settle(sh.a_full, round, kA, from);
                bwd_settle(sh.b_full, b_issued, kB, from);
                bwd_settle(sh.stat_full, b_issued, 2, from);
                bar_settle(shared_address(&sh.own_full), 0, from);
            }
        }
        const int2 live = live_tokens(a);
        const bool dead = rounds > 0 && dead_rows(first * R, tiles * R, live, a.tokens);  // there are rows outside every sequence
        if (warp == 10 && dead) cleaner_run<D, R>(sh.cleaner, live, lane, failed);
        if (warp == 8 && rounds > 0 && elected()) {
            // (A wait takes this thread some 200 cycles when there is nothing to wait for, a product 20 to 30, and its time is part of every round: no
            // more in it than has to be.  After a failed wait the others end at once, and what is issued then is of no use but does no harm.)
            unsigned asked = 0;
            const unsigned a_full = shared_address(&sh.a_full[0]), a_empty = shared_address(&sh.a_empty[0]), b_full = shared_address(&sh.b_full[0]), b_empty = shared_address(&sh.b_empty[0]);
            const unsigned s_full = shared_address(&sh.s_full[0]), p_full = shared_address(&sh.p_full), dp_full = shared_address(&sh.dp_full), ds_full = shared_address(&sh.ds_full);
            auto clear = [&](unsigned tile, int round) {
                const int t = (first + (round0 + round) % tiles) * R;
                if (dead_rows(t, R, live, a.tokens)) cleaner_ask(sh.cleaner, tile, t, asked, failed);
            };
            Ring<kA> ra;  // of the next round
            Ring<kB> rb;
            unsigned q_now = 0, do_now = 0;  // stages of this round
            auto q_there = [&](int round) {
                bar_wait(a_full + 8 * ra.at, ra.phase, failed);
                if (dead) clear(sq + ra.at * kTile, round);
            };
            auto do_there = [&](int round) {
                bar_wait(b_full + 8 * rb.at, rb.phase, failed);
                if (dead) clear(sdo + rb.at * kTile, round);
            };
            auto scores = [&]() {
                product_round<D, R>(s_at, sk, sq + ra.at * kTile);
                products_to(s_full);
                ra.step();
            };
            auto gradient = [&]() {
                product_round<D, R>(dp_at, sv, sdo + rb.at * kTile);
                products_to(dp_full);
                rb.step();
            };
            bar_wait(shared_address(&sh.own_full), 0, failed);
            q_there(0);
            scores();
            do_there(0);
            gradient();
            for (int round = 0; round < rounds; ++round) {
                const bool more = round + 1 < rounds;
                const unsigned q_next = ra.at, do_next = rb.at;
                if (more) q_there(round + 1);
                bar_wait(p_full, round & 1, failed);
                tmem_fence_after();
                product_halves<D, R>(dv_at, s_at, sdo + do_now * kTile, round > 0);
                if (more) scores();
                products_to(b_empty + 8 * do_now);
                if (more) do_there(round + 1);
                bar_wait(ds_full, round & 1, failed);
                tmem_fence_after();
                product_halves<D, R>(dk_at, dp_at, sq + q_now * kTile, round > 0);
                if (more) gradient();
                products_to(more ? a_empty + 8 * q_now : shared_address(&sh.done));
                q_now = q_next;
                do_now = do_next;
            }
            if (dead) cleaner_ask(sh.cleaner, 0, 0, asked, failed);
            if (*failed) bwd_drain(sh);
        }
    } else {
        const int half = warp >> 2, j = k0 + (tid & 127);
        const unsigned lanes = (unsigned)(warp & 3) << 21, s_t = s_at + lanes + H * half, dp_t = dp_at + lanes + H * half;
        const int4 mine = sh.ranges[warp & 3];
        const float2 c2 = both(a.c);
        bool ok = placed;
        for (int round = 0; round < rounds; ++round) {
            const int q0 = (first + (round0 + round) % tiles) * R + H * half;
            // (after a failure the rest of the waits end at once)
            ok = bar_wait(shared_address(&sh.s_full[0]), round & 1, failed) && ok;
            ok = bar_wait(shared_address(&sh.stat_full[round & 1]), round >> 1 & 1, failed) && ok;
            __syncwarp();
            tmem_fence_after();
            float s[H / 32][32];
            const unsigned at = stats + (round & 1) * Shape::kStats + half * (H * 4);
            load_columns<H>(s_t, s);
            float2 p[H / 2];
#pragma unroll
            for (int i = 0; i < H / 4; ++i) {
                float4 l;
                shared_load<16>(at + 16 * i, &l);
                const float2 e = fma2(make_float2(s[i / 8][i % 8 * 4], s[i / 8][i % 8 * 4 + 1]), c2, make_float2(l.x, l.y));
                const float2 f = fma2(make_float2(s[i / 8][i % 8 * 4 + 2], s[i / 8][i % 8 * 4 + 3]), c2, make_float2(l.z, l.w));
                p[2 * i] = exp2_pair<kBwdPoly>(e, 2 * i);
                p[2 * i + 1] = exp2_pair<kBwdPoly>(f, 2 * i + 1);
            }
            mask_pairs(p, see.x - q0, see.y - q0, q0 < mine.z, q0 + H > mine.w);
            store_pairs(s_t, p);
            if (lane == 0) bar_arrive(shared_address(&sh.p_full));
            ok = bar_wait(shared_address(&sh.dp_full), round & 1, failed) && ok;
            __syncwarp();
            tmem_fence_after();
            load_columns<H>(dp_t, s);
#pragma unroll
            for (int i = 0; i < H / 4; ++i) {
                float4 l;
                shared_load<16>(at + 4 * R + 16 * i, &l);
                const float2 e = add2(make_float2(s[i / 8][i % 8 * 4], s[i / 8][i % 8 * 4 + 1]), make_float2(l.x, l.y));
                const float2 f = add2(make_float2(s[i / 8][i % 8 * 4 + 2], s[i / 8][i % 8 * 4 + 3]), make_float2(l.z, l.w));
                p[2 * i] = mul2(p[2 * i], e);
                p[2 * i + 1] = mul2(p[2 * i + 1], f);
            }
            // (0 where p is: dP of rows outside every sequence is finite, and of others that are not the fp32 code hears)
            store_pairs(dp_t, p);
            if (lane == 0) {
                bar_arrive(shared_address(&sh.ds_full));
                bar_arrive(shared_address(&sh.stat_empty[round & 1]));
            }
        }
        if (rounds > 0) ok = bar_wait(shared_address(&sh.done), 0, failed) && ok;
        __syncwarp();
        tmem_fence_after();
        const bool in = see.y > 0;
        if (a.parts_kv > 1) {
            const bool fine = store_part<D>((half ? dk_at : dv_at) + lanes, rounds > 0, in, j < a.tokens && in, ok, part_row(half ? a.part_dk : a.part_dv, part, a.kv_heads, kv, min(j, a.tokens - 1), a), a.width);
            if (in && ok && !fine) sh.again = 1;
        } else {
        const AttnPlace to = half ? a.sdk : a.sdv;
        bf16* rows = static_cast<bf16*>(half ? a.dk : a.dv) + kv * to.head;
        const bool fine = store_rows<D>((half ? dk_at : dv_at) + lanes, rounds > 0, in, j < a.tokens && (in || a.fill), ok ? (half ? a.scale : 1.0f) : NAN, rows, to.token, j - lane, a.dim,
                                        shared_address(bwd_smem) + warp * 4096, lane);
        if (in && ok && !fine) sh.again = 1;
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 8) {
        tmem_fence_after();
        tmem_free(tmem, Shape::kColumns);
    }
    if (sh.failed || !sh.again || tid >= 256) return;
    constexpr int kSteps = R / plain_step_of(D);  // of the fp32 code to a round
    for (int x = 0; x < 2; ++x)
        plain_dkv_tile<bf16, D, 64>(a, k0 + 64 * x, kv, part, make_int2(kSteps * first, kSteps * tiles), make_int2(kSteps * round0, kSteps * (round0 + rounds)), reinterpret_cast<float*>(bwd_smem), tid);
}

template <int D>
__global__ void __launch_bounds__(kBwdThreads, BwdShape<D>::kCtas) attention_dq_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ TileMap mq, const __grid_constant__ TileMap mk,
                                                                      const __grid_constant__ TileMap mv, const __grid_constant__ TileMap mdo, int swapped) {
    typedef BwdShape<D> Shape;
    constexpr int kA = Shape::kA, kB = Shape::kB, kTile = Shape::kTile, kOwn = Shape::kOwn, R = Shape::kRound, H = R / 2;  // H: columns of a thread
    extern __shared__ __align__(1024) unsigned char bwd_smem[];
    BwdShared& sh = *reinterpret_cast<BwdShared*>(bwd_smem + Shape::kShared);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int tiles_all = (a.tokens + 127) / 128, head = blockIdx.x % a.q_heads, q0 = (tiles_all - 1 - (int)(blockIdx.x / a.q_heads)) * 128, part = blockIdx.y;
    const unsigned sq = shared_address(bwd_smem), sdo = sq + kOwn, sk = sq + 2 * kOwn, sv = sk + kA * kTile;
    volatile int* failed = &sh.failed;
    if (tid == 0) bwd_init(sh);
    if (warp == 8) tmem_alloc(shared_address(&sh.tmem), Shape::kColumns);
    int2 see = make_int2(0, 0);
    if (warp < 8) {
        see = keys_of(a, q0 + (tid & 127));
        const int4 r = warp_ranges(see);
        if (lane == 0 && warp < 4) sh.ranges[warp] = r;
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const unsigned tmem = sh.tmem, dp_at = tmem + 2 * R, dq_at = tmem + 3 * R;  // scores of even and odd rounds in front
    const int4 all = tile_ranges(sh.ranges);
    const int2 share = all.y > 0 ? share_of((all.y + R - 1) / R - all.x / R, part, a.parts_q) : make_int2(0, 0);
    const bool placed = swizzle_placed(sq);
    const int first = (all.y > 0 ? all.x / R : 0) + share.x, rounds = placed ? share.y - share.x : 0;

    if (warp >= 8) {
        if (warp == 9 && rounds > 0 && elected()) {
            bar_expect(shared_address(&sh.own_full), 2 * kOwn);
            for (int p = 0; p < D / 64; ++p)
                for (int r = 0; r < 128; r += R) {
                    tile_load(sq + p * 16384 + r * 128, &mq, swapped & 1, p * 64, head, q0 + r, shared_address(&sh.own_full));
                    tile_load(sdo + p * 16384 + r * 128, &mdo, swapped >> 3 & 1, p * 64, head, q0 + r, shared_address(&sh.own_full));
                }
            const int kv = head / a.group;
            bool ok = true;
            int round = 0, b_issued = 0;
            Ring<kA> ra;
            Ring<kB> rb;
            for (; round < rounds; ++round) {
                const unsigned kb = shared_address(&sh.a_full[ra.at]), vb = shared_address(&sh.b_full[rb.at]);
                // (V's stage is free before K's)
                if (!(ok = bar_wait(shared_address(&sh.b_empty[rb.at]), rb.phase ^ 1, failed))) break;
                bar_expect(vb, kTile);
                for (int p = 0; p < D / 64; ++p) tile_load(sv + rb.at * kTile + p * (R * 128), &mv, swapped >> 2 & 1, p * 64, kv, (first + round) * R, vb);
                rb.step();
                b_issued = round + 1;
                if (!(ok = bar_wait(shared_address(&sh.a_empty[ra.at]), ra.phase ^ 1, failed))) break;
                bar_expect(kb, kTile);
                for (int p = 0; p < D / 64; ++p) tile_load(sk + ra.at * kTile + p * (R * 128), &mk, swapped >> 1 & 1, p * 64, kv, (first + round) * R, kb);
                ra.step();
            }
            if (!ok) {
                const long long from = clock64();
                bwd_settle(sh.a_full, round, kA, from);
                bwd_settle(sh.b_full, b_issued, kB, from);
                bar_settle(shared_address(&sh.own_full), 0, from);
            }
        }
        const int2 live = live_tokens(a);
        const bool dead = rounds > 0 && dead_rows(first * R, rounds * R, live, a.tokens);  // K has rows outside every sequence, and dq sums over them
        if (warp == 10 && dead) cleaner_run<D, R>(sh.cleaner, live, lane, failed);
        if (warp == 8 && rounds > 0 && elected()) {
            unsigned asked = 0, k_now = 0, k_then = 0, v_at = 0;  // stages of K of this round and the next, and of V
            const unsigned a_full = shared_address(&sh.a_full[0]), a_empty = shared_address(&sh.a_empty[0]), b_full = shared_address(&sh.b_full[0]), b_empty = shared_address(&sh.b_empty[0]);
            const unsigned s_full = shared_address(&sh.s_full[0]), dp_full = shared_address(&sh.dp_full), ds_full = shared_address(&sh.ds_full);
            Ring<kA> ra;
            Ring<kB> rb;
            auto scores = [&](int round) {  // of the next K
                const unsigned st = ra.at;
                bar_wait(a_full + 8 * st, ra.phase, failed);
                if (dead && dead_rows((first + round) * R, R, live, a.tokens)) cleaner_ask(sh.cleaner, sk + st * kTile, (first + round) * R, asked, failed);
                product_round<D, R>(tmem + R * (round & 1), sq, sk + st * kTile);
                products_to(s_full + 8 * (round & 1));
                ra.step();
                return st;
            };
            auto v_there = [&]() {
                v_at = rb.at;
                bar_wait(b_full + 8 * rb.at, rb.phase, failed);
                rb.step();
            };
            auto gradient = [&]() {
                product_round<D, R>(dp_at, sdo, sv + v_at * kTile);
                products_to(dp_full);
            };
            bar_wait(shared_address(&sh.own_full), 0, failed);
            k_now = scores(0);
            v_there();
            gradient();
            products_to(b_empty + 8 * v_at);
            if (rounds > 1) k_then = scores(1);
            for (int round = 0; round < rounds; ++round) {
                const bool more = round + 1 < rounds;
                if (more) v_there();
                bar_wait(ds_full, round & 1, failed);
                tmem_fence_after();
                if (more) gradient();
                product_halves<D, R>(dq_at, tmem + R * (round & 1), sk + k_now * kTile, round > 0);
                products_to(more ? a_empty + 8 * k_now : shared_address(&sh.done));
                if (more) products_to(b_empty + 8 * v_at);
                k_now = k_then;
                if (round + 2 < rounds) k_then = scores(round + 2);
            }
            if (dead) cleaner_ask(sh.cleaner, 0, 0, asked, failed);
            if (*failed) bwd_drain(sh);
        }
    } else {
        const int half = warp >> 2, i = q0 + (tid & 127);
        const unsigned lanes = (unsigned)(warp & 3) << 21;
        const int4 mine = sh.ranges[warp & 3];
        const bool in = see.y > 0;
        const long long at = (long long)head * a.pitch + i;  // (the statistics are padded to whole tiles)
        const float2 c2 = both(a.c), l2 = both(__ldcg(&a.nlse2[at])), d2 = both(__ldcg(&a.ndelta[at]));  // (from L2: written by a kernel that this one has not waited for itself)
        bool ok = placed;
        for (int round = 0; round < rounds; ++round) {
            const int j0 = (first + round) * R + H * half;
            const unsigned s_t = tmem + R * (round & 1) + lanes + H * half, dp_t = dp_at + lanes + H * half;
            ok = bar_wait(shared_address(&sh.s_full[round & 1]), (round >> 1) & 1, failed) && ok;
            __syncwarp();
            tmem_fence_after();
            float s[H / 32][32];
            load_columns<H>(s_t, s);
            float2 p[H / 2];
#pragma unroll
            for (int x = 0; x < H / 2; ++x) {
                const float2 e = fma2(make_float2(s[x / 16][x % 16 * 2], s[x / 16][x % 16 * 2 + 1]), c2, l2);
                p[x] = exp2_pair<kBwdPoly>(e, x);
            }
            ok = bar_wait(shared_address(&sh.dp_full), round & 1, failed) && ok;
            __syncwarp();
            tmem_fence_after();
            load_columns<H>(dp_t, s);
#pragma unroll
            for (int x = 0; x < H / 2; ++x) p[x] = mul2(p[x], add2(make_float2(s[x / 16][x % 16 * 2], s[x / 16][x % 16 * 2 + 1]), d2));
            mask_pairs(p, see.x - j0, see.y - j0, j0 < mine.z, j0 + H > mine.w);
            store_pairs(s_t, p);
            if (lane == 0) bar_arrive(shared_address(&sh.ds_full));
        }
        if (rounds > 0) ok = bar_wait(shared_address(&sh.done), 0, failed) && ok;
        __syncwarp();
        tmem_fence_after();
        // each half of the threads stores half of the row
        constexpr int W = D / 2;
        if (a.parts_q > 1) {
            const bool fine = store_part<W>(dq_at + lanes + half * W, rounds > 0, in, i < a.tokens && in, ok, part_row(a.part_dq, part, a.q_heads, head, min(i, a.tokens - 1), a) + half * W, a.width - half * W);
            if (in && ok && !fine) sh.again = 1;
        } else {
        const AttnPlace to = a.sdq;
        bf16* rows = static_cast<bf16*>(a.dq) + head * to.head + half * W;
        const bool fine = store_rows<W>(dq_at + lanes + half * W, rounds > 0, in, i < a.tokens && (in || a.fill), ok ? a.scale : NAN, rows, to.token, i - lane, a.dim - half * W,
                                        shared_address(bwd_smem) + warp * 4096, lane);
        if (in && ok && !fine) sh.again = 1;
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 8) {
        tmem_fence_after();
        tmem_free(tmem, Shape::kColumns);
    }
    // (the last CTA, which has the least to do, ends after dk and dv have, and with them the statistics: what follows in the stream waits for this kernel alone)
    if (tid == 0 && blockIdx.x + 1 == gridDim.x && blockIdx.y + 1 == gridDim.y) earlier_done();
    if (sh.failed || !sh.again || tid >= 256) return;
    constexpr int kSteps = R / plain_step_of(D);  // of the fp32 code to a round
    for (int x = 0; x < 2; ++x) plain_dq_tile<bf16, D, 64>(a, q0 + 64 * x, head, part, make_int2(kSteps * first, kSteps * (first + rounds)), reinterpret_cast<float*>(bwd_smem), tid);
}

}  // namespace

// tcgen05 products, tensor memory, tile copies and the barriers between them, as the attention kernels use them.
// Part of libsparseloco (attention.cu).
//
// Operand tiles lie in shared memory as the tile copies leave them with a 128-byte swizzle: panels of 64 bfloat16 (128 bytes) by R rows,
// 8 rows to a 1024-byte group, panels R * 128 bytes apart.  The same panel serves as an operand whose summed dimension runs
// along the 128 bytes ("along": steps of 16 values are 32 bytes) or down the rows ("down": steps of 16 rows are 2048 bytes).
#pragma once
#include <cuda.h>

#include "inner_common.cuh"

namespace {

__device__ __forceinline__ unsigned shared_address(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }

// ---- kernels that begin before the one in front of them ends
__device__ __forceinline__ void earlier_done() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void next_may_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- barriers
__device__ __forceinline__ void bar_init(unsigned bar, unsigned arrivals) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(arrivals) : "memory"); }
__device__ __forceinline__ void bar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(unsigned bar, unsigned bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }
__device__ __forceinline__ bool bar_try(unsigned bar, unsigned parity) {
    unsigned done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}
// Waits for at most 2^32 cycles (two to four seconds), then marks the CTA as failed; every other wait of the CTA then ends too.  (The
// SM's own cycle counter: reading the global timer took longer than most waits.)
constexpr long long kWaitCycles = 1ll << 32;
__device__ __forceinline__ bool bar_wait(unsigned bar, unsigned parity, volatile int* failed) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
        if (bar_try(bar, parity)) return true;
    const long long from = clock64();
#pragma unroll 1
    for (unsigned i = 1; i < (1u << 26); ++i) {
        if (bar_try(bar, parity)) return true;
        if ((i & 63u) == 0u && (*failed || clock64() - from > kWaitCycles)) break;
    }
    *failed = 1;
    return false;
}
// After a failure: waits for what is on its way, as long again.
__device__ __forceinline__ void bar_settle(unsigned bar, unsigned parity, long long from) {
    while (!bar_try(bar, parity) && clock64() - from < kWaitCycles) {
    }
}

// ---- tile copies
struct TileMap {
    CUtensorMap map;
};
// 64 values by the map's rows at (x, head, token) of a [token, head, value] matrix; `swapped`: the map has tokens inside heads
__device__ __forceinline__ void tile_load(unsigned to, const TileMap* m, int swapped, int x, int head, int token, unsigned bar) {
    const int y = swapped ? token : head, z = swapped ? head : token;
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y),
                 "r"(z), "r"(bar)
                 : "memory");
}

// ---- tensor memory
__device__ __forceinline__ void tmem_alloc(unsigned to, int columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(unsigned at, int columns) { asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of this warp's lanes, one lane per thread.  The loaded values may be used only behind tmem_loaded().
__device__ __forceinline__ void tmem_load32(unsigned at, float (&f)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]), "=f"(f[8]), "=f"(f[9]), "=f"(f[10]), "=f"(f[11]), "=f"(f[12]), "=f"(f[13]), "=f"(f[14]),
          "=f"(f[15]), "=f"(f[16]), "=f"(f[17]), "=f"(f[18]), "=f"(f[19]), "=f"(f[20]), "=f"(f[21]), "=f"(f[22]), "=f"(f[23]), "=f"(f[24]), "=f"(f[25]), "=f"(f[26]), "=f"(f[27]), "=f"(f[28]),
          "=f"(f[29]), "=f"(f[30]), "=f"(f[31])
        : "r"(at)
        : "memory");
}
// (the values pass through the wait, so that no use of them moves in front of it)
__device__ __forceinline__ void tmem_loaded(float (&f)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]), "+f"(f[4]), "+f"(f[5]), "+f"(f[6]), "+f"(f[7]), "+f"(f[8]), "+f"(f[9]), "+f"(f[10]), "+f"(f[11]), "+f"(f[12]), "+f"(f[13]),
                   "+f"(f[14]), "+f"(f[15]), "+f"(f[16]), "+f"(f[17]), "+f"(f[18]), "+f"(f[19]), "+f"(f[20]), "+f"(f[21]), "+f"(f[22]), "+f"(f[23]), "+f"(f[24]), "+f"(f[25]), "+f"(f[26]),
                   "+f"(f[27]), "+f"(f[28]), "+f"(f[29]), "+f"(f[30]), "+f"(f[31])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_store32(unsigned at, const float (&f)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
        "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]), "f"(f[8]), "f"(f[9]), "f"(f[10]), "f"(f[11]), "f"(f[12]), "f"(f[13]), "f"(f[14]), "f"(f[15]), "f"(f[16]),
        "f"(f[17]), "f"(f[18]), "f"(f[19]), "f"(f[20]), "f"(f[21]), "f"(f[22]), "f"(f[23]), "f"(f[24]), "f"(f[25]), "f"(f[26]), "f"(f[27]), "f"(f[28]), "f"(f[29]), "f"(f[30]), "f"(f[31])
        : "memory");
}
// 16 columns of two bfloat16 each
__device__ __forceinline__ void tmem_store16(unsigned at, const unsigned (&w)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                 "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(w[8]), "r"(w[9]), "r"(w[10]), "r"(w[11]), "r"(w[12]), "r"(w[13]), "r"(w[14]), "r"(w[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- products
// One lane of a converged warp, the same every time.  (Behind `lane == 0` the compiler does not know that a single thread goes on, and every product
// took some 110 cycles to issue in place of 30.)
__device__ __forceinline__ bool elected() {
    unsigned one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
// 128-byte swizzle, rows of 128 bytes, 8-row groups 1024 bytes apart, panels `panel` bytes apart (read only where the rows are summed over)
__device__ __forceinline__ uint64_t tile_desc(unsigned at, unsigned panel) {
    return (uint64_t)((at & 0x3FFFF) >> 4) | (uint64_t)((panel & 0x3FFFF) >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// bfloat16 x bfloat16 into fp32, 128 rows, n columns; B summed along its 128 bytes or (down) down its rows
__host__ __device__ constexpr unsigned product_kind(int n, bool down) { return 1u << 4 | 1u << 7 | 1u << 10 | (down ? 1u << 16 : 0u) | (unsigned)(n >> 3) << 17 | (128u >> 4) << 24; }

__device__ __forceinline__ void product(unsigned to, uint64_t a, uint64_t b, unsigned kind, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(to), "l"(a), "l"(b), "r"(kind), "r"((unsigned)add) : "memory");
}
__device__ __forceinline__ void product_tmem(unsigned to, unsigned a, uint64_t b, unsigned kind, bool add) {  // A in tensor memory
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(to), "r"(a), "l"(b), "r"(kind), "r"((unsigned)add) : "memory");
}
// the barrier gets one arrival when all products issued so far by this thread are done
__device__ __forceinline__ void products_to(unsigned bar) { asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory"); }

// to[128, 128] = a b^T over D values, both tiles along their rows; 128-row tiles, so panels are 16 KB
template <int D>
__device__ __forceinline__ void product_rows(unsigned to, unsigned a, unsigned b) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        const unsigned at = (unsigned)(i / 4) * 16384u + (unsigned)(i % 4) * 32u;
        product(to, tile_desc(a + at, 0), tile_desc(b + at, 0), product_kind(128, false), i > 0);
    }
}
// to[128, D] (+)= p b over b's 128 rows, p of bfloat16 pairs in tensor memory
template <int D>
__device__ __forceinline__ void product_down(unsigned to, unsigned p, unsigned b, bool add) {
#pragma unroll
    for (int i = 0; i < 8; ++i) product_tmem(to, p + 8u * i, tile_desc(b + 2048u * i, 16384u), product_kind(D, true), add || i > 0);
}

// Rows of a tile that stand for tokens outside `live` are set to 0 before a product sums over them: what lies behind the last sequence
// may be anything, and 0 times NaN is NaN.  A warp of its own does it, when the issuing thread asks: only the few tiles that have such rows
// (rows behind the last token are zeros already) are asked for.
__device__ __forceinline__ bool dead_rows(int first, int rows, int2 live, int tokens) { return first < live.x || (first + rows > live.y && live.y < tokens); }
struct Cleaner {
    unsigned long long asked, cleared;  // one arrival each
    unsigned tile;                      // 0: no more
    int first;
};
__device__ __forceinline__ void cleaner_init(Cleaner& c) {
    bar_init(shared_address(&c.asked), 1);
    bar_init(shared_address(&c.cleared), 1);
}
template <int D, int ROWS>
__device__ __forceinline__ void cleaner_run(Cleaner& c, int2 live, int lane, volatile int* failed) {
    for (unsigned k = 0;; ++k) {
        const bool ok = bar_wait(shared_address(&c.asked), k & 1, failed);
        if (__any_sync(kFullMask, !ok)) return;
        const unsigned tile = *(volatile unsigned*)&c.tile;
        const int first = *(volatile int*)&c.first;
        if (tile == 0) return;
        for (int r = lane >> 3; r < ROWS; r += 4)
            if (first + r < live.x || first + r >= live.y)
#pragma unroll
                for (int p = 0; p < D / 64; ++p) asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + p * (ROWS * 128u) + r * 128u + (lane & 7) * 16u), "r"(0u) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) bar_arrive(shared_address(&c.cleared));
    }
}
__device__ __forceinline__ bool cleaner_ask(Cleaner& c, unsigned tile, int first, unsigned& asked, volatile int* failed) {
    *(volatile unsigned*)&c.tile = tile;
    *(volatile int*)&c.first = first;
    bar_arrive(shared_address(&c.asked));
    return tile == 0 || bar_wait(shared_address(&c.cleared), asked++ & 1, failed);
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The larger of two, NaN where either is.
__device__ __forceinline__ float max_nan(float x, float y) {
    float z;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
// The same of two values by multiply-adds, for part of a tile's exponentials (the instruction above takes 8 cycles a warp): x = n + f with n the
// nearest integer, 2^f on [-1/2, 1/2] by the polynomial of degree 5 with the smallest relative error that is 1 at 0 (1.1e-7, a linear
// programme over 4001 points), times 2^n.  What is added to round x leaves n + 127 in the lowest bits, the exponent of 2^n.  x may be up to 127; below -126.5
// (-inf too) the factor's exponent is 0 and the result 0, as the instruction's is, and NaN goes through every step.
__device__ __forceinline__ float2 exp2_poly(float2 x) {
    constexpr float kRound = 12582912.0f + 127.0f;  // 3 * 2^22
    x.x = max_nan(x.x, -127.0f);
    x.y = max_nan(x.y, -127.0f);
    const float2 t = add2(x, both(kRound)), n = add2(t, both(-kRound)), f = fma2(n, both(-1.0f), x);
    float2 p = fma2(both(0.001326465280726552f), f, both(0.009671511128544807f));
    p = fma2(p, f, both(0.05550733953714371f));
    p = fma2(p, f, both(0.24022242426872253f));
    p = fma2(p, f, both(0.6931470036506653f));
    p = fma2(p, f, both(1.0f));
    return mul2(p, make_float2(__int_as_float(__float_as_int(t.x) << 23), __int_as_float(__float_as_int(t.y) << 23)));
}
// pair i of a row: which of the two ways
template <int OF8>
__device__ __forceinline__ float2 exp2_pair(float2 x, int i) {
    return ((i * OF8) & 7) + OF8 > 7 ? exp2_poly(x) : make_float2(exp2_fast(x.x), exp2_fast(x.y));
}

}  // namespace

// Rotary positions of queries and keys.  Part of libsparseloco (inner.cu).
//
// Bound: HBM (q and k read and written once).  Sine and cosine depend on the token and the pair only: a CTA computes
// them once for its tokens, into shared memory, and uses them for every head.
#pragma once
#include "inner_common.cuh"

namespace {

constexpr int kRopeThreads = 256;

struct RopeHeads {
    const void* in;
    void* out;
    int heads;
    long long in_batch, in_token, in_head, out_batch, out_token, out_head;
};

struct RopeArgs {
    RopeHeads q, k;
    const unsigned long long* turns;  // 2^64 f_i / (2 pi)
    const void* positions;
    long long pos_batch, pos_token, first, rows;  // rows = batch * seq
    int position_bits, seq, head_dim, rot, tokens;  // tokens per CTA
    int slots, rot_slots;                           // accesses per head, those of them that turn
    int copy;                                       // values per access of the rest, which is passed through
    float magnitude, sign;
};

// One item: a slot of a head of a token.  VEC consecutive values per access.  Half layout: a turning slot is two accesses, rot / 2
// apart; interleaved: one access of VEC / 2 pairs (one pair of single values where VEC is 1).  The slots behind them copy what is
// passed through; WIDE: by wider accesses than those that turn.
template <class T, int VEC, bool HALF, bool WIDE>
struct RopeItem {
    Pack<T, VEC> a, b;
    uint4 c;  // WIDE: what is passed through
    __device__ __forceinline__ void load(const T* in, int slot, const RopeArgs& r) {
        if (!WIDE && slot >= r.rot_slots) {
            a.load(in + r.rot + (slot - r.rot_slots) * VEC);
        } else if (slot >= r.rot_slots) {
            const T* p = in + r.rot + (slot - r.rot_slots) * r.copy;
            const int bytes = r.copy * (int)sizeof(T);
            if (bytes == 16) c = *reinterpret_cast<const uint4*>(p);
            else if (bytes == 8) c.x = reinterpret_cast<const uint2*>(p)->x, c.y = reinterpret_cast<const uint2*>(p)->y;
            else if (bytes == 4) c.x = *reinterpret_cast<const unsigned*>(p);
            else c.x = *reinterpret_cast<const unsigned short*>(p);
        } else if (HALF) {
            a.load(in + slot * VEC);
            b.load(in + r.rot / 2 + slot * VEC);
        } else if (VEC > 1) {
            a.load(in + slot * VEC);
        } else {
            a.v[0] = in[2 * slot];
            b.v[0] = in[2 * slot + 1];
        }
    }
    // cs: sines and cosines of the slot's first pair; those of the next pair are rot_slots further on (so that neighbouring slots
    // read neighbouring words)
    __device__ __forceinline__ void turn_store(T* out, int slot, const RopeArgs& r, const float2* cs, bool in_place) {
        if (slot >= r.rot_slots) {
            if (in_place) return;
            if (!WIDE) {
                a.store(out + r.rot + (slot - r.rot_slots) * VEC);
                return;
            }
            T* p = out + r.rot + (slot - r.rot_slots) * r.copy;
            const int bytes = r.copy * (int)sizeof(T);
            if (bytes == 16) *reinterpret_cast<uint4*>(p) = c;
            else if (bytes == 8) *reinterpret_cast<uint2*>(p) = make_uint2(c.x, c.y);
            else if (bytes == 4) *reinterpret_cast<unsigned*>(p) = c.x;
            else *reinterpret_cast<unsigned short*>(p) = (unsigned short)c.x;
        } else if (HALF) {
            const int c = slot * VEC;
            float x[VEC], y[VEC];
            a.get(x);
            b.get(y);
            if constexpr (VEC > 1) {
#pragma unroll
                for (int j = 0; j < VEC; j += 2) {
                    const float2 e = cs[j * r.rot_slots], f = cs[(j + 1) * r.rot_slots];
                    const float2 co = make_float2(e.x, f.x), si = make_float2(e.y, f.y), p = make_float2(x[j], x[j + 1]), q = make_float2(y[j], y[j + 1]);
                    const float2 u = fma2(p, co, mul2(q, make_float2(-si.x, -si.y))), v = fma2(q, co, mul2(p, si));
                    x[j] = u.x, x[j + 1] = u.y, y[j] = v.x, y[j + 1] = v.y;
                }
            } else {
                turn(x[0], y[0], cs[0]);
            }
            a.set(x);
            b.set(y);
            a.store(out + c);
            b.store(out + r.rot / 2 + c);
        } else if (VEC > 1) {
            const int c = slot * VEC;
            float x[VEC];
            a.get(x);
#pragma unroll
            for (int j = 0; j + 1 < VEC; j += 2) turn(x[j], x[j + 1], cs[(j / 2) * r.rot_slots]);
            a.set(x);
            a.store(out + c);
        } else {
            float x = widen(a.v[0]), y = widen(b.v[0]);
            turn(x, y, cs[0]);
            out[2 * slot] = narrow<T>(x);
            out[2 * slot + 1] = narrow<T>(y);
        }
    }
    static __device__ __forceinline__ void turn(float& x, float& y, float2 e) {
        const float p = x, q = y;
        x = fmaf(p, e.x, -q * e.y);
        y = fmaf(q, e.x, p * e.y);
    }
};

// A thread keeps its slot and walks over the (token, head) pairs of the CTA, a few of them at a time, all loads before the
// first use; the first batch is on its way while sines and cosines are computed.
template <class T, int VEC, bool HALF, bool WIDE>
__global__ void __launch_bounds__(kRopeThreads)
rotary_kernel(const RopeArgs a) {
    constexpr int kBatch = HALF && VEC > 1 ? 2 : 4, kPairs = HALF ? VEC : (VEC > 1 ? VEC / 2 : 1);  // pairs of a slot
    extern __shared__ float2 turn[];  // [tokens][pair of a slot][slot]: magnitude * (cos, sin)
    const int half = a.rot / 2, heads = a.q.heads + a.k.heads;
    const long long row0 = (long long)blockIdx.x * a.tokens;
    const int n_tok = (int)(a.rows - row0 < a.tokens ? a.rows - row0 : a.tokens);
    const int span = a.slots < kRopeThreads ? a.slots : kRopeThreads;  // threads of a (token, head) pair
    const int groups = kRopeThreads / span, group = threadIdx.x / span;
    const bool works = group < groups;
    const int pairs = n_tok * heads;

    struct Place {
        int tok, head;
    };
    const int step_tok = groups / heads, step_head = groups - step_tok * heads;
    auto step = [&](Place& p) {
        p.tok += step_tok;
        p.head += step_head;
        if (p.head >= heads) p.head -= heads, ++p.tok;
    };
    const unsigned b0 = (unsigned)row0 / (unsigned)a.seq, s0 = (unsigned)row0 - b0 * (unsigned)a.seq;
    auto where = [&](int tok, long long& b, long long& s) {  // (tokens per CTA are few)
        unsigned bb = b0, ss = s0 + (unsigned)tok;
        while (ss >= (unsigned)a.seq) ss -= (unsigned)a.seq, ++bb;
        b = bb;
        s = ss;
    };
    auto in_of = [&](const Place& p) {
        const bool k = p.head >= a.q.heads;
        const RopeHeads& x = k ? a.k : a.q;
        long long b, s;
        where(p.tok, b, s);
        return static_cast<const T*>(x.in) + b * x.in_batch + s * x.in_token + (long long)(k ? p.head - a.q.heads : p.head) * x.in_head;
    };
    auto out_of = [&](const Place& p) {
        const bool k = p.head >= a.q.heads;
        const RopeHeads& x = k ? a.k : a.q;
        long long b, s;
        where(p.tok, b, s);
        return static_cast<T*>(x.out) + b * x.out_batch + s * x.out_token + (long long)(k ? p.head - a.q.heads : p.head) * x.out_head;
    };

    bool ready = false;
    for (int slot = threadIdx.x - group * span; slot < a.slots || !ready; slot += span) {
        RopeItem<T, VEC, HALF, WIDE> item[kBatch];
        Place at;
        at.tok = group / heads;
        at.head = group - at.tok * heads;
        const bool mine = works && slot < a.slots;
        for (int pair = group; pair < pairs || !ready; pair += groups * kBatch) {
            Place p = at;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if (mine && pair + u * groups < pairs) item[u].load(in_of(p), slot, a);
                step(p);
            }
            if (!ready) {
                for (int i = threadIdx.x; i < n_tok * half; i += kRopeThreads) {
                    const int t = i / half, f = i - t * half;
                    long long b, s;
                    where(t, b, s);
                    long long pos = a.first + s;
                    if (a.positions) {
                        const long long w = b * a.pos_batch + s * a.pos_token;
                        pos = a.position_bits == 64 ? static_cast<const long long*>(a.positions)[w] : (long long)static_cast<const int*>(a.positions)[w];
                    }
                    // position * frequency in turns, modulo 1 by the 64-bit product; the nearest quarter turn is taken off before
                    // what is left is rounded to fp32, as half turns in [-1/4, 1/4): sine and cosine stay accurate where they are small
                    const unsigned long long phase = (unsigned long long)pos * a.turns[f], quarter = (phase + (1ull << 61)) >> 62;
                    float sn, cs;
                    sincospif((float)(long long)(phase - (quarter << 62)) * 1.0842021724855044e-19f, &sn, &cs);  // 2^-63
                    if (quarter & 1) {
                        const float s0 = sn;
                        sn = cs;
                        cs = -s0;
                    }
                    if (quarter & 2) sn = -sn, cs = -cs;
                    turn[t * half + (f % kPairs) * a.rot_slots + f / kPairs] = make_float2(cs * a.magnitude, sn * a.sign * a.magnitude);
                }
                __syncthreads();
                ready = true;
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if (mine && pair + u * groups < pairs) {
                    const bool k = at.head >= a.q.heads;
                    item[u].turn_store(out_of(at), slot, a, turn + at.tok * half + slot, (k ? a.k.in : a.q.in) == (k ? a.k.out : a.q.out));
                }
                step(at);
            }
        }
    }
}

}  // namespace

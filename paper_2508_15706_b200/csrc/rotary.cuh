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
    float magnitude, sign;
};

// VEC consecutive values per access.  Half layout: a turning slot is two accesses, rot / 2 apart; interleaved: one access of
// VEC / 2 pairs (one pair of single values where VEC is 1).  The slots behind them copy what is passed through.
template <class T, int VEC, bool HALF>
__global__ void __launch_bounds__(kRopeThreads)
rotary_kernel(const RopeArgs a) {
    extern __shared__ float2 turn[];  // [tokens][rot / 2]: magnitude * (cos, sin)
    const int half = a.rot / 2;
    const long long row0 = (long long)blockIdx.x * a.tokens;
    const int n_tok = (int)(a.rows - row0 < a.tokens ? a.rows - row0 : a.tokens);
    for (int i = threadIdx.x; i < n_tok * half; i += kRopeThreads) {
        const int t = i / half, f = i - t * half;
        const long long row = row0 + t, b = row / a.seq, s = row - b * a.seq;
        long long pos = a.first + s;
        if (a.positions) {
            const long long at = b * a.pos_batch + s * a.pos_token;
            pos = a.position_bits == 64 ? static_cast<const long long*>(a.positions)[at] : (long long)static_cast<const int*>(a.positions)[at];
        }
        // position * frequency in turns, modulo 1 by the 64-bit product; as half turns in [-1, 1)
        const long long phase = (long long)((unsigned long long)pos * a.turns[f]);
        float sn, cs;
        sincospif((float)phase * 1.0842021724855044e-19f, &sn, &cs);  // 2^-63
        turn[i] = make_float2(cs * a.magnitude, sn * a.sign * a.magnitude);
    }
    __syncthreads();
    const int heads = a.q.heads + a.k.heads, per_tok = heads * a.slots;
    for (int i = threadIdx.x; i < n_tok * per_tok; i += kRopeThreads) {
        const int t = i / per_tok, u = i - t * per_tok;
        int h = u / a.slots;
        const int slot = u - h * a.slots;
        const bool is_k = h >= a.q.heads;
        const RopeHeads& x = is_k ? a.k : a.q;
        if (is_k) h -= a.q.heads;
        const long long row = row0 + t, b = row / a.seq, s = row - b * a.seq;
        const T* in = static_cast<const T*>(x.in) + b * x.in_batch + s * x.in_token + h * x.in_head;
        T* out = static_cast<T*>(x.out) + b * x.out_batch + s * x.out_token + h * x.out_head;
        const float2* cs = turn + t * half;
        if (slot < a.rot_slots) {
            if (HALF) {
                const int c = slot * VEC;
                Pack<T, VEC> lo, hi;
                lo.load(in + c);
                hi.load(in + half + c);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float p = widen(lo.v[j]), q = widen(hi.v[j]);
                    const float2 e = cs[c + j];
                    lo.v[j] = narrow<T>(fmaf(p, e.x, -q * e.y));
                    hi.v[j] = narrow<T>(fmaf(q, e.x, p * e.y));
                }
                lo.store(out + c);
                hi.store(out + half + c);
            } else if (VEC > 1) {
                const int c = slot * VEC;
                Pack<T, VEC> v;
                v.load(in + c);
#pragma unroll
                for (int j = 0; j + 1 < VEC; j += 2) {
                    const float p = widen(v.v[j]), q = widen(v.v[j + 1]);
                    const float2 e = cs[(c + j) / 2];
                    v.v[j] = narrow<T>(fmaf(p, e.x, -q * e.y));
                    v.v[j + 1] = narrow<T>(fmaf(q, e.x, p * e.y));
                }
                v.store(out + c);
            } else {
                const float p = widen(in[2 * slot]), q = widen(in[2 * slot + 1]);
                const float2 e = cs[slot];
                out[2 * slot] = narrow<T>(fmaf(p, e.x, -q * e.y));
                out[2 * slot + 1] = narrow<T>(fmaf(q, e.x, p * e.y));
            }
        } else if (in != out) {
            const int c = a.rot + (slot - a.rot_slots) * VEC;
            Pack<T, VEC> v;
            v.load(in + c);
            v.store(out + c);
        }
    }
}

}  // namespace

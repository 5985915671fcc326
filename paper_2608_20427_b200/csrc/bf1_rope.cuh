// Rotary positions: what the rotation kernel (bf1_rope.cu) and the cache write (bf1_cache.cu), which rotates on the way into
// the pages, share.
#pragma once

#include "bf1_common.cuh"

namespace bf1 {

// The tables of a bf1_rope as a kernel takes them.
struct RopeTable {
    const double* turns;   // [dim / 2]: turns of a pair per position
    int32_t dim;           // rotated dimensions of a head; 0: nothing is rotated
    int32_t half;          // 1: pairs (i, i + dim / 2); 0: pairs (2 i, 2 i + 1)
    float magnitude;       // factor on the rotated values
};

// (cos, sin) of a pair's angle, times the magnitude.  The angle is position * turns in 64 bits, of which only the part of a turn
// counts: table and product are each off by 2^-53 of the whole at most, so that a position of 2^31 still has its angle to 4e-7 of a radian (at a
// pair of one radian per position), where 32 bits lose all of it beyond 2^24 turns.  In 32 bits the sine and cosine are those of the rounded angle, corrected by their slopes times what the rounding
// took (which would be as large as their own error).  In 64 bits a call costs 2.5 times as much: it is for numbers that are rounded
// to three bits of fraction next, where an error of 2^-24 may turn a tie.
__device__ __forceinline__ double rope_half_turns(const RopeTable& r, int position, int pair) {
    const double t = (double)position * r.turns[pair];
    return 2.0 * (t - rint(t));
}
__device__ __forceinline__ float2 rope_angle(const RopeTable& r, int position, int pair) {
    const double t = rope_half_turns(r, position, pair);
    const float hi = (float)t, lo = 3.14159265f * (float)(t - (double)hi);
    float s, c;
    sincospif(hi, &s, &c);
    return make_float2(__fmaf_rn(-lo, s, c) * r.magnitude, __fmaf_rn(lo, c, s) * r.magnitude);
}
__device__ __forceinline__ double2 rope_angle64(const RopeTable& r, int position, int pair) {
    double s, c;
    sincospi(rope_half_turns(r, position, pair), &s, &c);
    return make_double2(c * r.magnitude, s * r.magnitude);
}

__device__ __forceinline__ void unpack_bf16x8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack_bf16x8(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// One pair turned.  The products are rounded in a stated order, so that every kernel gives the same bits (of 32-bit angles; the
// one below is for those of 64 bits: single tokens, or a few that share a page, into pages of 8 bits).
__device__ __forceinline__ void rope_turn(float& x, float& y, float c, float s) {
    const float p = x, q = y;
    x = __fmaf_rn(p, c, -__fmul_rn(q, s));
    y = __fmaf_rn(p, s, __fmul_rn(q, c));
}

__device__ __forceinline__ void rope_turn(float& x, float& y, double c, double s) {
    const double p = x, q = y;
    x = (float)(p * c - q * s);
    y = (float)(p * s + q * c);
}

// Rows of heads in global memory: bf16, the dimensions of a head side by side, strides in elements.
struct Rows {
    __nv_bfloat16* p;
    int64_t row, head;
    __device__ __forceinline__ __nv_bfloat16* at(int64_t token, int h) const { return p + token * row + h * head; }
};

// What a CTA of 128 threads does: kRopeTokens tokens from `token0`, a lane to sixteen dimensions of one, and for each warp the heads h0 + warp, h0 + warp +
// step, ...: the eight pairs 8 c .. 8 c + 7, or sixteen dimensions that are carried over.  The angles of the tokens are made once, two to a thread, and
// handed out through shared memory (each thread making its own eight: 4096 tokens of 24 heads 12.1 us, 9.9 as it is).  kAhead heads are asked for before
// the first is turned.  sign -1 turns back, which is the gradient (a rotation's transpose; the magnitude stays).  With kSplit = 4 every warp has
// tokens of its own and all the heads, of which there are fewer than four then.
constexpr int kRopeThreads = 128;
template <int D, int kSplit = 1>
constexpr int kRopeTokens = kSplit * 32 / (D / 16);
template <int D, int kAhead, int kSplit = 1>
__device__ __forceinline__ void rope_block(const RopeTable& r, const int32_t* positions, int64_t token0, int tokens, float sign, const Rows& in_q,
                                           const Rows& in_k, const Rows& out_q, const Rows& out_k, int hq, int heads, int h0, int step) {
    constexpr int kLanes = D / 16;                       // to a token
    constexpr int kTokens = kRopeTokens<D, kSplit>;
    __shared__ float2 angles[kTokens][8][kLanes];        // [token][pair of the lane][lane]
    const int warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < kTokens * kLanes * 8; i += kRopeThreads) {
        const int t = i / (kLanes * 8), pair = i % (kLanes * 8);
        if (2 * pair < r.dim && token0 + t < tokens) angles[t][pair % 8][pair / 8] = rope_angle(r, positions[token0 + t], pair);
    }
    const int lane = threadIdx.x & 31, t = (kSplit > 1 ? warp * (32 / kLanes) : 0) + lane / kLanes, c = lane % kLanes;
    const int64_t token = token0 + t;
    const bool live = token < tokens && positions[token] >= 0;   // padding: its rows stay as they are
    __syncthreads();
    if (!live) return;
    const bool turn = 16 * c < r.dim;
    const int lo = turn && r.half ? 8 * c : 16 * c, hi = turn && r.half ? r.dim / 2 + 8 * c : 16 * c + 8;
    float cs[8], sn[8];
    if (turn) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 a = angles[t][i][c];
            cs[i] = a.x;
            sn[i] = a.y * sign;
        }
    }
    for (int h = kSplit > 1 ? h0 : h0 + warp; h < heads; h += kAhead * step) {
        uint4 a[kAhead], b[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int hh = h + u * step;
            if (hh >= heads) break;
            const __nv_bfloat16* x = hh < hq ? in_q.at(token, hh) : in_k.at(token, hh - hq);
            a[u] = *reinterpret_cast<const uint4*>(x + lo);
            b[u] = *reinterpret_cast<const uint4*>(x + hi);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int hh = h + u * step;
            if (hh >= heads) break;
            __nv_bfloat16* y = hh < hq ? out_q.at(token, hh) : out_k.at(token, hh - hq);
            if (turn) {
                float x0[8], x1[8];
                unpack_bf16x8(a[u], x0);
                unpack_bf16x8(b[u], x1);
                if (r.half) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) rope_turn(x0[i], x1[i], cs[i], sn[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        rope_turn(x0[2 * i], x0[2 * i + 1], cs[i], sn[i]);
                        rope_turn(x1[2 * i], x1[2 * i + 1], cs[4 + i], sn[4 + i]);
                    }
                }
                a[u] = pack_bf16x8(x0);
                b[u] = pack_bf16x8(x1);
            }
            *reinterpret_cast<uint4*>(y + lo) = a[u];
            *reinterpret_cast<uint4*>(y + hi) = b[u];
        }
    }
}

// Dimensions 8 c .. 8 c + 7 of a row, rotated by angle(pair) = (cos, sin), in place of x.  With pairs of halves `other` are the eight dimensions that
// they are paired with, 8 rope_other(r, c) and up.
__device__ __forceinline__ int rope_other(const RopeTable& r, int c) { return 16 * c < r.dim ? c + r.dim / 16 : c - r.dim / 16; }
template <typename F>
__device__ __forceinline__ void rope_chunk(const RopeTable& r, int c, float (&x)[8], const uint4& other, F&& angle) {
    if (r.half) {
        const bool second = 16 * c >= r.dim;
        const int pair = second ? 8 * c - r.dim / 2 : 8 * c;
        float y[8];
        unpack_bf16x8(other, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const auto a = angle(pair + i);
            float p = second ? y[i] : x[i], q = second ? x[i] : y[i];
            rope_turn(p, q, a.x, a.y);
            x[i] = second ? q : p;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const auto a = angle(4 * c + i);
            rope_turn(x[2 * i], x[2 * i + 1], a.x, a.y);
        }
    }
}

// Host checks of a bf1_rope and of rows of heads (bf1_rope.cu).
int check_rope(const bf1_rope* rope, int32_t d);
int check_rows(const bf1_rows* rows, const char* name);
inline Rows rows_of(const bf1_rows* r) { return {static_cast<__nv_bfloat16*>(r->data), r->row_stride, r->head_stride}; }
inline RopeTable table_of(const bf1_rope* r) { return {r->turns, r->dim, r->layout == BF1_ROPE_HALF ? 1 : 0, r->magnitude}; }

}  // namespace bf1

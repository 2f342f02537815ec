// Angles of rotary positions.
//
// Pair i of a head turns by p f_i at position p.  The descriptor holds f_i / 2 pi as a 64-bit fraction F_i of a turn, so that the low 64 bits of p F_i are
// the angle modulo a whole turn, off by the rounding of F_i alone: 2^-65 turns a position, 4.7e-8 rad at p = 2^38 (fp32 products p f_i are off by 0.008 rad at
// p = 131072).  Its upper 32 bits are kept (1.5e-9 rad).  The nearest quarter turn is taken off, the rest lies within an eighth, |x| <= pi / 4, where the power
// series of sine and cosine up to x^9 and x^10 are within 2e-9.
#pragma once
#include "common.hpp"

namespace qarl {

// amplitude (cos, sin) of the angle at position p
__device__ __forceinline__ float2 rope_turn(uint64_t turns, int64_t p, float amplitude)
{
    const uint64_t phase = (uint64_t)p * turns;
    const uint32_t top = (uint32_t)(phase >> 32), quarter = (top + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(top - (quarter << 30)) * (float)(6.283185307179586 / 4294967296.0), x2 = x * x;
    float s = 1.f / 362880.f, c = -1.f / 3628800.f;
    s = fmaf(s, x2, -1.f / 5040.f);
    s = fmaf(s, x2, 1.f / 120.f);
    s = fmaf(s, x2, -1.f / 6.f);
    s = fmaf(s * x2, x, x);
    c = fmaf(c, x2, 1.f / 40320.f);
    c = fmaf(c, x2, -1.f / 720.f);
    c = fmaf(c, x2, 1.f / 24.f);
    c = fmaf(c, x2, -0.5f);
    c = fmaf(c, x2, 1.f);
    const bool odd = quarter & 1u;
    const float cs = odd ? s : c, sn = odd ? c : s;
    // quarters 1 and 2 have a negative cosine, 2 and 3 a negative sine
    return make_float2(((quarter + 1u) & 2u ? -cs : cs) * amplitude, (quarter & 2u ? -sn : sn) * amplitude);
}

// What a lane holds of a head: two runs of 16 bytes, E elements each, at `at`.  Lane c of a head's first rotary_dim / 2 E has E whole pairs; neighbouring lanes'
// runs are neighbours.  `pair`: of the first pair of either run (HALF: the runs are the pairs' two halves, and the second number is not used).
struct RopeRuns {
    int at[2], pair[2];
    bool turned;
};
template <int E>
__device__ __forceinline__ RopeRuns rope_runs(int c, int head_dim, int rot, int layout)
{
    const int lanes = rot / (2 * E), rest = (head_dim - rot) / (2 * E), j = c - lanes;
    RopeRuns r;
    r.turned = c < lanes;
    if (!r.turned) {
        r.at[0] = rot + E * j;
        r.at[1] = rot + E * (rest + j);
        r.pair[0] = r.pair[1] = 0;
    } else if (layout == QARL_ROPE_HALF) {
        r.at[0] = r.pair[0] = r.pair[1] = E * c;
        r.at[1] = rot / 2 + E * c;
    } else {
        r.at[0] = E * c;
        r.at[1] = E * (c + lanes);
        r.pair[0] = E / 2 * c;
        r.pair[1] = E / 2 * (c + lanes);
    }
    return r;
}

// The lane's cosines and sines, out of a token's
template <int E>
__device__ __forceinline__ void rope_turns(const float2 *turns, const RopeRuns &r, int layout, float2 (&t)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) t[i] = make_float2(1.f, 0.f);
    if (!r.turned) return;
#pragma unroll
    for (int i = 0; i < E; ++i) t[i] = turns[layout == QARL_ROPE_HALF || i < E / 2 ? r.pair[0] + i : r.pair[1] + i - E / 2];
}

// The lane's values turned: y = (a cos - b sin, b cos + a sin) of each pair (a, b)
template <int E>
__device__ __forceinline__ void rope_apply(float (&x)[2 * E], const float2 (&t)[E], int layout)
{
    if (layout == QARL_ROPE_HALF) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float a = x[i], b = x[E + i];
            x[i] = fmaf(a, t[i].x, -(b * t[i].y));
            x[E + i] = fmaf(b, t[i].x, a * t[i].y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = fmaf(a, t[i].x, -(b * t[i].y));
            x[2 * i + 1] = fmaf(b, t[i].x, a * t[i].y);
        }
    }
}

}  // namespace qarl

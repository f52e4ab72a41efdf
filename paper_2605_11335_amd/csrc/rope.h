// cos and sin of rotary positions from whole turns in 64-bit fixed point (host plan: cf_rope_plan).
//
// A pair turns by pos * f radians.  turn = f / 2 pi as a fraction of 2^64 is rounded once (2^-65 turns), and pos * turn modulo 2^64 is
// exact in integers: the fraction of a turn comes out to |pos| * 2^-65 turns (3e-9 rad at the ends of int32), where a product in fp32
// would be off by 0.06 rad at position 10^6.  The nearest quarter turn goes into the choice of signs; what is left, at most an eighth
// of a turn, goes through the Taylor series of sin and cos (first terms left out: x^11 / 11! = 2e-9, x^12 / 12! = 1e-10 at x = pi / 4).
#pragma once
#include "common.h"
#include "../../include/chunkflow.h"

__device__ __forceinline__ void rope_sincos(uint64_t turn, int32_t pos, float& c, float& s) {
    const uint32_t ph = (uint32_t)((turn * (uint64_t)(int64_t)pos + 0x80000000ull) >> 32);      // fraction of a turn, 2^-32
    const uint32_t quarter = (ph + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(ph - (quarter << 30)) * 1.46291807926715968e-9f;           // 2 pi / 2^32
    const float x2 = x * x;
    const float sn = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 2.7557319224e-6f, -1.9841269841e-4f), 8.3333333333e-3f), -1.6666666667e-1f), x);
    const float cs = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -2.7557319224e-7f, 2.4801587302e-5f), -1.3888888889e-3f), 4.1666666667e-2f), -0.5f), 1.0f);
    const float a = quarter & 1u ? sn : cs, b = quarter & 1u ? cs : sn;
    c = (quarter + 1u) & 2u ? -a : a;                                                            // quarters 1 and 2
    s = quarter & 2u ? -b : b;                                                                   // quarters 2 and 3
}

__device__ __forceinline__ void rope_turn(float& a, float& b, float c, float s) {
    const float x = fmaf(a, c, -b * s), y = fmaf(a, s, b * c);
    a = x;
    b = y;
}

// argument checks shared by the entry points that take a plan
inline const char* rope_bad(const cf_rope* r) {
    if (!r) return "null plan";
    if (r->head_dim != 64 && r->head_dim != 128) return "not a plan (cf_rope_plan)";
    if (r->n_axes < 1 || r->n_axes > CF_ROPE_AXES || r->n_pairs < 1 || r->n_pairs > r->head_dim / 2) return "not a plan (cf_rope_plan)";
    for (int p = 0; p < 64; ++p)
        if (r->axis[p] >= r->n_axes) return "not a plan (cf_rope_plan)";
    return nullptr;
}

// Rounding of 4-bit quantisation, shared by the weights and the key / value cache: scales and codes as if computed exactly.
#pragma once
#include "../../include/eesd.h"
#include "common.cuh"

namespace eesd {

// The quotient's nearest value of the scale's type (ties to even).  For bf16 it is rounded once: towards zero in fp32 with what is lost
// kept in the last bit, then to nearest.
__device__ __forceinline__ float round_scale(float x, float by, int scale_dtype) {
    if (scale_dtype == EESD_F32) return __fdiv_rn(x, by);
    float f = __fdiv_rz(x, by);
    if (__fmaf_rn(-f, by, x) != 0.f) f = __uint_as_float(__float_as_uint(f) | 1u);
    return __bfloat162float(__float2bfloat16_rn(f));
}
// (hi - lo) / 15 with hi >= 0 >= lo, likewise.  The difference may take more than the 53 bits of a double and its quotient more again: both
// remainders are exact, and they tell the side where the rounded quotient lies on the border between two scales (the true one lies on
// the same side of a border as the rounded one, or that is the border itself, since rounding keeps order and a border times 15 is a double).
__device__ __forceinline__ float round_range(float hi, float lo, int scale_dtype) {
    const double a = fmax((double)hi, -(double)lo), b = fmin((double)hi, -(double)lo);
    const double sum = a + b, lost = b - (sum - a);
    const double q = sum / 15.0, rest = fma(-q, 15.0, sum) + lost;
    const uint32_t step = scale_dtype == EESD_F32 ? 1u : 0x10000u;
    const uint32_t below = __float_as_uint(__double2float_rz(q)) & ~(step - 1u);   // the scale at or below q
    const double at = __uint_as_float(below), next = __uint_as_float(below + step);
    double side = q - (at + next) * 0.5;
    if (side == 0.0) side = rest;
    return __uint_as_float(side > 0.0 || (side == 0.0 && (below & step)) ? below + step : below);
}

// nearest integer (ties to even) to the exact quotient x / s.  The rounded quotient can only be off by one, and only when x / s
// is within rounding of a half: the exact remainder (one fused multiply-add) settles it.
__device__ __forceinline__ float nearest_quotient(float x, float s) {
    float q = rintf(__fdiv_rn(x, s));
    q = fminf(fmaxf(q, -17.f), 17.f);
    const float rem = __fmaf_rn(-q, s, x), twice = rem + rem;
    if (twice > s || (twice == s && ((int)q & 1))) q += 1.f;
    else if (-twice > s || (-twice == s && ((int)q & 1))) q -= 1.f;
    return q;
}
__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

}  // namespace eesd

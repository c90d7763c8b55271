// The nonlinearity between two layers, its value and slope, two values at a time.
#pragma once
#include "row_ops.cuh"

namespace lrbi {

constexpr int ACT_NONE = LRBI_ACT_NONE;

__device__ __forceinline__ F2 exp2_2(F2 p)      // the hardware's estimate, 2^-22 off
{
    float a, b;
    split(p, a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    return f2(a, b);
}
__device__ __forceinline__ F2 inverse2(F2 p)    // 2^-23 off
{
    float a, b;
    split(p, a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return f2(a, b);
}

// Value and slope of the nonlinearity.  gelu(h) = h Phi(h), Phi the normal distribution; slope Phi(h) + h phi(h).
// With tail = Phi(-|h|): value = max(h, 0) - |h| tail, slope = [h >= 0] - sign(h) tail + h phi(h), no branch and no
// cancellation in the value for h < 0.  tail = erfc(z) / 2 with z = |h| / sqrt(2), phi = exp(-z^2) / sqrt(2 pi), and
// erfc(z) = t (a0 + t (a1 + ...)) exp(-z^2), t = 1 / (1 + p z), Hastings' form.  p and the a (halved here) were fitted to
// exp(z^2) erfc(z) on 0 .. 9.4 for the smallest largest error (least squares, reweighted by the errors).  FINE, for results in
// 32 bits: eight a, off by 7.7e-8 of the tail.  For bf16: five, off by 1.2e-6 absolutely and by 2^-13 of the tail, a 32nd of a
// step; with eight the forward pass of 16384 x 4096 takes 46.1 us, not 43.7, with the copy 63.8, not 60.4; results in fp32 take
// as long with either.  (Hastings' own five, Abramowitz and Stegun 7.1.26, are off by 5e-4 of the tail at h = -4, 1e-2 at -8.)
template <bool FINE> __device__ __forceinline__ F2 half_erfc_factor(F2 m)      // erfc(z) exp(z^2) / 2, m = |h|
{
    const F2 t = inverse2(fma2(m, f2(FINE ? 0.233056586f : 0.358236255f), f2(1.f)));      // p / sqrt(2)
    F2 p;
    if (FINE) {
        p = fma2(t, f2(-0.0686676508f), f2(0.235281272f));
        p = fma2(t, p, f2(-0.183808087f));
        p = fma2(t, p, f2(0.211417088f));
        p = fma2(t, p, f2(0.019920065f));
        p = fma2(t, p, f2(0.101591877f));
        p = fma2(t, p, f2(0.0911900968f));
        p = fma2(t, p, f2(0.0930753007f));
    } else {
        p = fma2(t, f2(-0.092899649f), f2(0.241409861f));
        p = fma2(t, p, f2(0.0510323927f));
        p = fma2(t, p, f2(0.158783556f));
        p = fma2(t, p, f2(0.141672657f));
    }
    return t * p;
}
template <int ACT, bool SLOPE, bool FINE, bool FINE_SLOPE>      // FINE: of the value
__device__ __forceinline__ void activate(F2 h, F2 &value, F2 &slope)
{
    constexpr float LOG2E = 1.44269504f;
    float a, b;
    split(h, a, b);
    if (ACT == LRBI_ACT_RELU) {
        value = f2(a < 0.f ? 0.f : a, b < 0.f ? 0.f : b);                       // a NaN stays
        if (SLOPE) slope = f2(a > 0.f ? 1.f : (a <= 0.f ? 0.f : a), b > 0.f ? 1.f : (b <= 0.f ? 0.f : b));
    } else if (ACT == LRBI_ACT_SILU) {
        const F2 s = inverse2(exp2_2(h * f2(-LOG2E)) + f2(1.f));
        value = h * s;
        if (SLOPE) slope = fma2(value, fma2(s, f2(-1.f), f2(1.f)), s);
    } else {
        const F2 m = f2(fabsf(a), fabsf(b)), e = exp2_2(h * h * f2(-0.5f * LOG2E));
        // The tail of 64 is zero already: +inf would give infinity times zero.  (A NaN comes through the tail.)
        value = fma2(f2(-fabsf(fminf(a, 64.f)), -fabsf(fminf(b, 64.f))), half_erfc_factor<FINE>(m) * e, f2(fmaxf(a, 0.f), fmaxf(b, 0.f)));
        if (SLOPE) {
            float x, y;
            split(half_erfc_factor<FINE_SLOPE>(m) * e, x, y);
            slope = fma2(h * f2(0.39894228f), e, f2((a >= 0.f ? 1.f : 0.f) - copysignf(x, a), (b >= 0.f ? 1.f : 0.f) - copysignf(y, b)));
        }
    }
}

}  // namespace lrbi

// gate.h -- the activation of the gated feed-forward and its gradient.
//
// act(g) = g sigma(z(g)) with z = g (SiLU) or 2 sqrt(2/pi) (g + 0.044715 g^3)
// (GELU in its tanh form, since (1 + tanh y) / 2 = sigma(2 y)).
#pragma once

#include <hip/hip_runtime.h>

#include "mxnorm.h"

#pragma clang fp contract(off)

namespace mxk {

// sigma(z(g)) from the hardware's exp2 and reciprocal, one unit in the last
// place each: for |z| up to 20 the result is within 2^-19 (SiLU) or 2^-18 (GELU,
// whose polynomial is rounded too) of its value relatively, by the argument's
// rounding, far below a bf16 or MX rounding.  z
// beyond the exponential's range gives exactly 0 or 1.
template <int ACT> __device__ __forceinline__ float gate_sigma(float g)
{
    constexpr float kLog2e = 1.44269504f;
    float t; // -z log2(e)
    if constexpr (ACT == MX_ACT_SILU) {
        t = g * -kLog2e;
    } else {
        constexpr float c = 1.5957691216f * kLog2e; // 2 sqrt(2/pi) log2(e)
        t = g * __builtin_fmaf(g * g, -c * 0.044715f, -c);
    }
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
}

// Gradients of act(g) u: dg = gh u act'(g), act' = sigma (1 + g (1 - sigma)
// z'(g)), and du = gh act(g).  Beyond |g| = 128 the second term is 0 in float,
// or sigma is: its g is held there, a finite polynomial times 0, also for
// infinite g.  (A NaN g, which the clamp would drop, is in sigma.)
template <int ACT>
__device__ __forceinline__ void gate_gradient(float g, float u, float gh, float &dg, float &du)
{
    const float s = gate_sigma<ACT>(g);
    const float gc = __builtin_amdgcn_fmed3f(g, -128.0f, 128.0f);
    float t = gc;
    if constexpr (ACT == MX_ACT_GELU_TANH) {
        constexpr float c = 1.5957691216f;
        t *= __builtin_fmaf(gc * gc, c * 3.0f * 0.044715f, c);
    }
    const float hs = gh * s;
    dg = hs * u * __builtin_fmaf(t, 1.0f - s, 1.0f);
    du = hs * g;
}

// gate_gradient of 8 bf16 columns, rounded to bf16: what the casts of a
// backward take, like every gradient that reaches them.
template <int ACT>
__device__ __forceinline__ void gate_gradients(const uint4 &g, const uint4 &u, const uint4 &gh,
                                               uint4 &dg, uint4 &du)
{
    const uint32_t gw[4] = {g.x, g.y, g.z, g.w}, uw[4] = {u.x, u.y, u.z, u.w};
    const uint32_t hw[4] = {gh.x, gh.y, gh.z, gh.w};
    uint32_t a[4], b[4];
    auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
    auto hi = [](uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); };
    auto pack = [](float x, float y) {
        const __bf16 p = (__bf16)x, q = (__bf16)y;
        return (uint32_t)__builtin_bit_cast(uint16_t, p) | ((uint32_t)__builtin_bit_cast(uint16_t, q) << 16);
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float g0, g1, u0, u1;
        gate_gradient<ACT>(lo(gw[i]), lo(uw[i]), lo(hw[i]), g0, u0);
        gate_gradient<ACT>(hi(gw[i]), hi(uw[i]), hi(hw[i]), g1, u1);
        a[i] = pack(g0, g1);
        b[i] = pack(u0, u1);
    }
    dg = make_uint4(a[0], a[1], a[2], a[3]);
    du = make_uint4(b[0], b[1], b[2], b[3]);
}

} // namespace mxk

// The gated product of a feed-forward block, H = act(G) * U, where gate and up are stored as ONE projection whose output
// channels alternate (channel 2 i is gate i, channel 2 i + 1 is up i), so that the two factors of a product are neighbours
// in every linear kernel's epilogue: in adjacent lanes of a warp.
//
// Both activations are g times a logistic function of g (c0 + c1 g^2):
//   silu       g / (1 + exp(-g))                                         c0 = 1, c1 = 0
//   gelu_tanh  g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2           c0 = sqrt(8/pi), c1 = 0.044715 c0
//              (because (1 + tanh(z / 2)) / 2 = 1 / (1 + exp(-z)))
// so the choice is two numbers: k0, k1 = -c0 log2(e), -c1 log2(e), and with them act(g) = g / (1 + 2^(g (k0 + k1 g^2))).  G and U are the
// fp16 outputs of the two projections, the product is formed in fp32 (MUFU exponential and reciprocal: 2^-21 relative at |g| below
// 8, far below the 2^-11 of the result) and rounded to fp16 once.
#pragma once
#include "aser_common.cuh"

namespace aser {

__device__ __forceinline__ float ex2_approx(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp_approx_ftz(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// SILU: k1 is zero.
template <bool SILU>
__device__ __forceinline__ float gated_product(float g, float u, const GluForm& f) {
    // (the square is kept finite: at an infinite gate k1 g^2 is to have the sign of k1)
    const float z = g * (SILU ? f.k0 : fmaf(f.k1, fminf(g * g, 1e10f), f.k0));
    return g * rcp_approx_ftz(1.f + ex2_approx(z)) * u;
}

// `pair` holds this lane's channel at two tokens (low half: the first).  Even lanes hold gate, odd lanes the up channel of
// the lane before; an even lane returns H of the first token, an odd lane that of the second (fp16 bits).  Warp-wide.
template <bool SILU>
__device__ __forceinline__ unsigned short gated_exchange(uint32_t pair, int lane, const GluForm& f) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, pair, 1);
    // {gate, up} of this lane's token: the low halves of both words, or the high halves the other way round
    const uint32_t gu = __byte_perm(pair, other, (lane & 1) ? 0x3276 : 0x5410);
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&gu));
    return __half_as_ushort(__float2half_rn(gated_product<SILU>(v.x, v.y, f)));
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace aser

// The gated product of a feed-forward block, H = act(G) * U, where gate and up are stored as ONE projection whose output
// channels alternate (channel 2 i is gate i, channel 2 i + 1 is up i), so that the two factors of a product are neighbours
// in every linear kernel's epilogue: in adjacent lanes of a warp.
//
// Both activations are g times a logistic function of g (c0 + c1 g^2):
//   silu       g / (1 + exp(-g))                                         c0 = 1, c1 = 0
//   gelu_tanh  g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2           c0 = sqrt(8/pi), c1 = 0.044715 c0
//              (because (1 + tanh(z / 2)) / 2 = 1 / (1 + exp(-z)))
// so the choice is two numbers and no branch.  G and U are the fp16 outputs of the two projections, the product is formed in
// fp32 and rounded to fp16 once.
#pragma once
#include "aser_common.cuh"

namespace aser {

__device__ __forceinline__ float gated_product(float g, float u, const GluForm& f) {
    // (the square is kept finite: 0 * inf would make silu of an infinite gate a NaN)
    const float z = g * fmaf(f.c1, fminf(g * g, 1e10f), f.c0);
    return __fdividef(g, 1.f + __expf(-z)) * u;
}

// `pair` holds this lane's channel at two tokens (low half: the first).  Even lanes hold gate, odd lanes the up channel of
// the lane before; an even lane returns H of the first token, an odd lane that of the second (fp16 bits).  Warp-wide.
__device__ __forceinline__ unsigned short gated_exchange(uint32_t pair, int lane, const GluForm& f) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, pair, 1);
    const bool odd = lane & 1;
    const unsigned short g = (unsigned short)(odd ? other >> 16 : pair & 0xffffu);
    const unsigned short u = (unsigned short)(odd ? pair >> 16 : other & 0xffffu);
    return __half_as_ushort(__float2half_rn(gated_product(__half2float(__ushort_as_half(g)), __half2float(__ushort_as_half(u)), f)));
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace aser

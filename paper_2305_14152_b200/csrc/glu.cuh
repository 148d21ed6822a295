// The gated feed-forward block, H = act(X Wg^T) * (X Wu^T), as the kernels see it: gate and up projection are one quantized
// linear of 2 F rows, in which runs of eight gate rows alternate with the eight up rows of the same channels.  So the two sums of a
// channel are made by one tile, wherever the tile begins, and mostly in one thread; and all that is done with a linear (its
// gradients, AdamW, the prepared copy) is done with the block.
#pragma once

#include "common.cuh"

namespace peqa {

constexpr int kGluRun = 8;       // rows of a run

// What a forward kernel makes of the block's sums beside storing them.
//
// Scales of groups lie on the contraction, so they go into the operand, and rounded to bf16 there they and the products are off by 2^-9 of themselves in the
// mean: two such sums multiplied had twice the error that the rounding of H has.  So with groups the operands are binary16 (2^-12): X times a power of two
// per token, scales times one per row, which glu_operands_kernel (glu.cu) makes and the epilogue takes off.
struct GluOut {
  __nv_bfloat16* H;              // [tokens, F]; nullptr: an ordinary linear
  int act;                       // peqa_activation
  const float* factors;          // groups: what the sums are multiplied by, [2F] and behind them [tokens]
};

inline bool glu_act_ok(int act) { return act == PEQA_ACT_SILU || act == PEQA_ACT_GELU_TANH; }

#ifdef __CUDACC__
// Both activations are x p(v) with p the logistic function: v = x, or 2 sqrt(2/pi) (x + 0.044715 x^3), since (1 + tanh(u)) / 2 =
// p(2u).  Exponential and reciprocal are the approximate ones (good to 2^-18 of p for |v| up to 88), far below bf16's step.
constexpr float kGeluInner = 1.5957691216057308f, kGeluCubic = 0.044715f;
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// v of x
template <int ACT>
__device__ __forceinline__ float glu_inner(float x) {
  return ACT == PEQA_ACT_SILU ? x : kGeluInner * fmaf(kGeluCubic * x * x, x, x);
}
template <int ACT>
__device__ __forceinline__ float glu_value(float x, float up) {
  return x * rcp_approx(1.0f + __expf(-glu_inner<ACT>(x))) * up;      // (0 where the exponential is too large)
}
__device__ __forceinline__ float glu_value(float x, float up, int act) {
  return act == PEQA_ACT_SILU ? glu_value<PEQA_ACT_SILU>(x, up) : glu_value<PEQA_ACT_GELU_TANH>(x, up);
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}
// Eight channels: their gate sums, then their up sums, in y.  (One reciprocal for four of them, 1/a = bcd / abcd, is three quarters of the
// special functions and more multiplications: 4096 tokens at 22016 x 1024, where the epilogue shows, 169 -> 174 us.)
template <int ACT>
__device__ __forceinline__ void glu_pack(const float (&y)[16], uint32_t* o) {
#pragma unroll
  for (int q = 0; q < 4; ++q) o[q] = bf16_pair(glu_value<ACT>(y[2 * q], y[2 * q + 8]), glu_value<ACT>(y[2 * q + 1], y[2 * q + 9]));
}
#endif

}  // namespace peqa

// The gated feed-forward block's forward entry point, and the backward pass of its activation (HBM bound).
//
// With Y [T, 2F] the block's two sums (glu.cuh), a = act(gate) = x p(v) and dH [T, F]:
//   dY[gate] = dH * up * (p + x p q v'),   dY[up] = dH * x p,   q = 1 - p
// p and q come from one exponential of -|v|, so neither cancels.  A thread takes eight channels: 32 bytes of Y, which are their gate and up
// sums side by side, 16 of dH, and writes 32 of dY; ten bytes a channel is all the traffic there is (4096 x 22016: 130 us, 6.9 TB/s).
#include <cuda_bf16.h>

#include "common.cuh"
#include "glu.cuh"
#include "sm100_ptx.cuh"

namespace peqa {

namespace {

constexpr int kBackThreads = 256;

__device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t both(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <int ACT>
__device__ __forceinline__ void glu_slopes(float x, float up, float dh, float& d_gate, float& d_up) {
  float v = x, dv = 1.0f;
  if (ACT == PEQA_ACT_GELU_TANH) {
    v = kGeluInner * fmaf(kGeluCubic * x * x, x, x);
    dv = kGeluInner * fmaf(3.0f * kGeluCubic * x, x, 1.0f);
  }
  const float t = __expf(-fabsf(v)), r = __fdividef(1.0f, 1.0f + t);
  const float p = v < 0.0f ? t * r : r, q = v < 0.0f ? r : t * r;
  d_up = dh * (x * p);
  // far out q is 0, where dv may have overflowed
  d_gate = dh * up * (ACT == PEQA_ACT_GELU_TANH && q == 0.0f ? p : fmaf(x * p, q * dv, p));
}

template <int ACT>
__global__ void __launch_bounds__(kBackThreads) glu_bwd_kernel(const uint4* Y, const uint4* dH, uint4* dY, long long units) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const long long u = (long long)blockIdx.x * kBackThreads + threadIdx.x;
  if (u >= units) return;
  const uint4 g4 = ptx::ld_global(Y + 2 * u), u4 = ptx::ld_global(Y + 2 * u + 1), h4 = ptx::ld_global(dH + u);
  const uint32_t g[4] = {g4.x, g4.y, g4.z, g4.w}, w[4] = {u4.x, u4.y, u4.z, u4.w}, h[4] = {h4.x, h4.y, h4.z, h4.w};
  uint32_t a[4], b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float g0, g1, u0, u1;
    glu_slopes<ACT>(low(g[e]), low(w[e]), low(h[e]), g0, u0);
    glu_slopes<ACT>(high(g[e]), high(w[e]), high(h[e]), g1, u1);
    a[e] = both(g0, g1);
    b[e] = both(u0, u1);
  }
  dY[2 * u] = make_uint4(a[0], a[1], a[2], a[3]);
  dY[2 * u + 1] = make_uint4(b[0], b[1], b[2], b[3]);
}

}  // namespace

}  // namespace peqa

using namespace peqa;

extern "C" int peqa_qglu_fwd(const peqa_qweight_t* w, int activation, const void* X, int T, void* Y, void* H, void* stream) {
  int g = 0, G = 0;
  PEQA_TRY(check_qweight(w, &g, &G));
  if (!X || !H) return PEQA_ERR_NULL;
  if (T <= 0 || w->in_features % 64 != 0 || w->out_features % 16 != 0 || !fwd_pair_supported(w) || !glu_act_ok(activation))
    return PEQA_ERR_BAD_SHAPE;
  if (!aligned16(X) || !aligned16(Y) || !aligned16(H)) return PEQA_ERR_ALIGNMENT;
  PEQA_TRY(check_arch());
  return launch_glu_fwd(w, g, X, T, Y, GluOut{static_cast<__nv_bfloat16*>(H), activation}, as_stream(stream));
}

extern "C" int peqa_glu_bwd(int activation, const void* Y, const void* dH, int T, int F, void* dY, void* stream) {
  if (!Y || !dH || !dY) return PEQA_ERR_NULL;
  if (T <= 0 || F <= 0 || F % kGluRun != 0 || !glu_act_ok(activation)) return PEQA_ERR_BAD_SHAPE;
  if (!aligned16(Y) || !aligned16(dH) || !aligned16(dY)) return PEQA_ERR_ALIGNMENT;
  const long long units = (long long)T * (F / kGluRun), blocks = (units + kBackThreads - 1) / kBackThreads;
  if (blocks > INT32_MAX) return PEQA_ERR_TOO_LARGE;
  PEQA_TRY(check_arch());
  return launch_after(activation == PEQA_ACT_SILU ? glu_bwd_kernel<PEQA_ACT_SILU> : glu_bwd_kernel<PEQA_ACT_GELU_TANH>, (int)blocks,
                      kBackThreads, as_stream(stream), static_cast<const uint4*>(Y), static_cast<const uint4*>(dH),
                      static_cast<uint4*>(dY), units);
}

// The gated feed-forward block's forward entry point, and the backward pass of its activation (HBM bound).
//
// With Y [T, 2F] the block's two sums (glu.cuh), a = act(gate) = x p(v) and dH [T, F]:
//   dY[gate] = dH * up * (p + x p q v'),   dY[up] = dH * x p,   q = 1 - p
// p and q come from one exponential of -|v|, so neither cancels.  A thread takes eight channels: 32 bytes of Y, which are their gate and up
// sums side by side, 16 of dH, and writes 32 of dY; ten bytes a channel is all the traffic there is (4096 x 22016: 130 us, 6.9 TB/s).
#include <cuda_bf16.h>

#include "common.cuh"
#include "dequant.cuh"
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
  // far out p or q is 0, where dv may have overflowed; the slope is p then
  const bool flat = ACT == PEQA_ACT_GELU_TANH && (p == 0.0f || q == 0.0f);
  d_gate = dh * up * (flat ? p : fmaf(x * p, q * dv, p));
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

// Operands of a block with groups, in binary16 (see GluOut).  A CTA a token: its largest channel brought to [2^14, 2^15), so that all that is more than
// 2^-28 of it keeps its bits.  Behind the tokens' CTAs the rows: a row's largest scale brought to [2^11, 2^12), which fifteen steps of a code leave within
// binary16 (65504), so that all that is 2^-25 of it or more keeps its bits; by as many lanes as hold its groups in kRowHeld registers each, so that every scale is asked for before the first is used.  (Against a warp for eight rows, one after the other, the
// forward of 77 tokens, us: 4096 rows of 172 groups 34.4 / 22.0, 8192 of 128 at 300 tokens 64.1 / 51.8, 22016 of 32 38.4 / 37.5.)
constexpr int kRowHeld = 8;
constexpr int kHeld = 4;                          // 16-byte pieces of a token that a thread keeps between the two passes
// lanes of a row, a power of two
__host__ __device__ inline int row_lanes(int G) {
  int lanes = 1;
  while (lanes < 32 && lanes * kRowHeld < G) lanes *= 2;
  return lanes;
}

// 2^e for |e| <= 126, and the exponent that takes the largest of these bits to 2^target; what is not finite stays so.
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
__device__ __forceinline__ int shift_to(uint32_t largest, int target) {
  const int e = (int)(largest >> 23 & 255u);
  return e == 255 ? 0 : max(-126, min(126, target + 127 - e));
}
__device__ __forceinline__ uint32_t largest_of(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t most = 0u;
#pragma unroll
  for (int e = 0; e < 4; ++e) most = max(most, max(w[e] << 16 & 0x7FFF0000u, w[e] & 0x7FFF0000u));
  return most;
}
// Eight channels, in the order of the codes' (dq::half_column).
template <int BITS>
__device__ __forceinline__ uint4 to_half(const uint4& v, float by) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float x[8];
#pragma unroll
  for (int q = 0; q < 4; ++q) x[2 * q] = low(w[q]) * by, x[2 * q + 1] = high(w[q]) * by;
  uint32_t o[4];
#pragma unroll
  for (int q = 0; q < 4; ++q)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(o[q]) : "f"(x[dq::half_column(BITS, 2 * q + 1)]), "f"(x[dq::half_column(BITS, 2 * q)]));
  return make_uint4(o[0], o[1], o[2], o[3]);
}

template <int BITS>
__global__ void __launch_bounds__(kBackThreads) glu_operands_kernel(const uint4* X, const float* scales, int T, int K, int N, int G,
                                                                    uint4* halves, float* scaled, float* factors) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (blockIdx.x < T) {
    __shared__ uint32_t part[kBackThreads / 32];
    const int pieces = K / 8;
    const uint4* x = X + (size_t)blockIdx.x * pieces;
    uint4 held[kHeld];
    uint32_t most = 0u;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int c = (int)threadIdx.x + i * kBackThreads;
      held[i] = c < pieces ? ptx::ld_global(x + c) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int i = 0; i < kHeld; ++i) most = max(most, largest_of(held[i]));
    for (int c = (int)threadIdx.x + kHeld * kBackThreads; c < pieces; c += kBackThreads) most = max(most, largest_of(ptx::ld_global(x + c)));
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) part[warp] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBackThreads / 32; ++w) most = max(most, part[w]);
    const int e = shift_to(most, 14);
    const float by = power_of_two(e);
    uint4* out = halves + (size_t)blockIdx.x * pieces;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int c = (int)threadIdx.x + i * kBackThreads;
      if (c < pieces) out[c] = to_half<BITS>(held[i], by);
    }
    for (int c = (int)threadIdx.x + kHeld * kBackThreads; c < pieces; c += kBackThreads) out[c] = to_half<BITS>(ptx::ld_global(x + c), by);
    if (threadIdx.x == 0) factors[N + blockIdx.x] = power_of_two(-e);
    return;
  }
  const int lanes = row_lanes(G), at = lane & (lanes - 1);
  const int row = (((int)blockIdx.x - T) * kBackThreads + (int)threadIdx.x) / lanes;
  const float* from = scales + (size_t)row * G;
  float* to = scaled + (size_t)row * G;
  // group of register i; rows of a multiple of four begin on 16 bytes
  const bool fours = G % 4 == 0;
  auto group = [&](int i) { return fours ? (at + i / 4 * lanes) * 4 + i % 4 : at + i * lanes; };
  float s[kRowHeld];
  if (fours) {
#pragma unroll
    for (int i = 0; i < kRowHeld; i += 4) {
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (row < N && group(i) < G) v = ptx::ld_global(reinterpret_cast<const float4*>(from + group(i)));
      s[i] = v.x, s[i + 1] = v.y, s[i + 2] = v.z, s[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kRowHeld; ++i) s[i] = row < N && group(i) < G ? ptx::ld_global(from + group(i)) : 0.0f;
  }
  uint32_t most = 0u;
#pragma unroll
  for (int i = 0; i < kRowHeld; ++i) most = max(most, __float_as_uint(s[i]) & 0x7FFFFFFFu);
  if (row < N)                                    // (more than 256 groups: a warp is one row)
    for (int g = at + kRowHeld * lanes; g < G; g += lanes) most = max(most, __float_as_uint(ptx::ld_global(from + g)) & 0x7FFFFFFFu);
  for (int o = lanes >> 1; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (row >= N) return;
  const int e = shift_to(most, 11);
  const float by = power_of_two(e);
  if (fours) {
#pragma unroll
    for (int i = 0; i < kRowHeld; i += 4)
      if (group(i) < G) *reinterpret_cast<float4*>(to + group(i)) = make_float4(s[i] * by, s[i + 1] * by, s[i + 2] * by, s[i + 3] * by);
  } else {
#pragma unroll
    for (int i = 0; i < kRowHeld; ++i)
      if (group(i) < G) to[group(i)] = s[i] * by;
  }
  for (int g = at + kRowHeld * lanes; g < G; g += lanes) to[g] = ptx::ld_global(from + g) * by;
  if (at == 0) factors[row] = power_of_two(-e);
}

// The workspace of a block with groups.
struct GluWorkspace {
  size_t halves, scaled, factors, bytes;
};
GluWorkspace glu_workspace(const peqa_qweight_t* w, int G, int T) {
  GluWorkspace ws = {};
  if (G == 1) return ws;
  auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  const size_t N = (size_t)w->out_features;
  ws.scaled = up((size_t)T * w->in_features * 2);
  ws.factors = ws.scaled + up(N * G * sizeof(float));
  ws.bytes = ws.factors + up((N + T) * sizeof(float));
  return ws;
}

}  // namespace

size_t glu_workspace_bytes(const peqa_qweight_t* w, int g, int T) { return glu_workspace(w, w->in_features / g, T).bytes; }

}  // namespace peqa

using namespace peqa;

extern "C" int peqa_qglu_fwd(const peqa_qweight_t* w, int activation, const void* X, int T, void* Y, void* H, void* workspace,
                             size_t workspace_bytes, void* stream) {
  int g = 0, G = 0;
  PEQA_TRY(check_qweight(w, &g, &G));
  if (!X || !H) return PEQA_ERR_NULL;
  if (T <= 0 || w->in_features % 64 != 0 || w->out_features % 16 != 0 || !fwd_pair_supported(w) || !glu_act_ok(activation))
    return PEQA_ERR_BAD_SHAPE;
  if (!aligned16(X) || !aligned16(Y) || !aligned16(H)) return PEQA_ERR_ALIGNMENT;
  PEQA_TRY(check_arch());
  const GluWorkspace at = glu_workspace(w, G, T);
  GluOut glu = {static_cast<__nv_bfloat16*>(H), activation, nullptr};
  cudaStream_t st = as_stream(stream);
  if (at.bytes == 0) return launch_glu_fwd(w, g, X, T, Y, glu, st);
  if (!workspace || workspace_bytes < at.bytes) return PEQA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return PEQA_ERR_ALIGNMENT;
  char* ws = static_cast<char*>(workspace);
  float *scaled = reinterpret_cast<float*>(ws + at.scaled), *factors = reinterpret_cast<float*>(ws + at.factors);
  const int rows_of_cta = kBackThreads / row_lanes(G);
  const long long ctas = (long long)T + (w->out_features + rows_of_cta - 1) / rows_of_cta;
  if (ctas > INT32_MAX) return PEQA_ERR_TOO_LARGE;
  PEQA_TRY(launch_after(w->bits == 4 ? glu_operands_kernel<4> : glu_operands_kernel<3>, (int)ctas, kBackThreads, st, static_cast<const uint4*>(X), w->scales, T, (int)w->in_features,
                        (int)w->out_features, G, reinterpret_cast<uint4*>(ws + at.halves), scaled, factors));
  peqa_qweight_t half = *w;
  half.scales = scaled;
  glu.factors = factors;
  return launch_glu_fwd(&half, g, ws + at.halves, T, Y, glu, st);
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

// What the kernels of the vocabulary projection's loss share (head_loss.cu, and head_loss_few.cu for few tokens).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "common.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

namespace peqa {
namespace loss {

using namespace ptx;

constexpr int kTile = 256;                      // tokens, and vocabulary entries or features, of a tile
constexpr int kDepth = 64;                      // contraction elements of a stage
constexpr int kOperandBytes = 128 * kDepth * 2;     // this CTA's half of a stage's A or B
constexpr int kLossThreads = 384;               // warps: 0 TMA, 1 MMA, 2 tensor memory, 4-11 epilogue
constexpr float kFarAbove = 60.0f;              // exp(60) V |W| is far below binary32's largest number
constexpr float kLog2e = 1.4426950408889634f;

// What the kernel before leaves of the tokens that count, in their order.
struct LiveTokens {
  int* count;        // [1]
  int* index;        // token
  int* label;
  float* ref;        // logit of the label
  int* above;        // bits of the largest l - ref beyond kFarAbove, 0 if there is none
};

struct LossParams {
  LiveTokens live;
  int* again;            // the chunk's flag
  bool second;           // the repetition
  float* sums;           // [halves (few tokens: eighths) of tiles, rows]: s, or (without gradient) pairs of largest logit and sum relative to it
  int row0, rows;        // first live token of the chunk, rows that its buffers have (a multiple of 256)
  int V, K, k_blocks;    // stages of a tile of logits
  int width;             // entries of a tile of the vocabulary, a multiple of 32
  int tile0, tiles;      // tiles of the vocabulary in this launch's piece
  int back0, back_blocks;    // first entry and stages of the piece before, whose gradient is summed; 0 stages: none
  bool first_back;       // nothing has been summed yet
  int splits;            // parts that the sum over a piece is cut into, each with sums of its own
  int group, back_group; // blocks of 256 tokens whose tiles are worked through together
  int* status;
};

int loss_map(CUtensorMap* m, CUtensorMapDataType type, const void* base, uint64_t inner, uint64_t outer, int size, uint32_t box_x,
             uint32_t box_y, CUtensorMapSwizzle swizzle, uint64_t pitch = 0);
inline int bf16_map(CUtensorMap* m, const void* base, uint64_t inner, uint64_t outer, uint32_t box_y, uint64_t pitch = 0) {
  return loss_map(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, inner, outer, 2, 64, box_y, CU_TENSOR_MAP_SWIZZLE_128B, pitch);
}

// Few tokens (head_loss_few.cu): tokens at most, partial sums of a tile, its buffers.
constexpr int kFewTokens = 256;
constexpr int kFewParts = 8;
// Without gradient nothing is known or counted beforehand: the tokens are the call's own, and the labels' logits are left in live.ref.
struct FewCall {
  const void* rows;            // [256, K], or the call's X
  const void* W;
  const int32_t* labels;
  float* grads;                // [splits, 256, K]
  void* e[2];                  // exponentials of a piece [256, pitch]; by turns, if there are several
  int pitch, tokens;
  CUtensorMap w, x, wt, e_out[2];
};
int few_maps(FewCall& call, int width, int V, int K, bool grad);
// turn: which of e this piece's exponentials go to; in_entries: of the piece before, in the other
int launch_few(const LossParams& p, const FewCall& call, int turn, int in_entries, bool grad, int pairs, cudaStream_t st);
int finish_few(const LossParams& p, const FewCall& call, int parts, float* loss, cudaStream_t st);

#ifdef __CUDACC__
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}
__device__ __forceinline__ void tma_add_2d(const CUtensorMap* m, uint32_t src_smem, int x, int y) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(src_smem), "r"(x), "r"(y)
               : "memory");
}
__device__ __forceinline__ void wait_for_kernel_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_kernel_behind_in() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// This lane's share of <x, w>, K a multiple of 8: columns first, first + step, ... of eight; copy: where x is to be left too, or nullptr.
__device__ __forceinline__ float dot_share(const __nv_bfloat16* x, const __nv_bfloat16* w, __nv_bfloat16* copy, int K, int first, int step) {
  float dot = 0.0f;
#pragma unroll 4
  for (int c = first; c < K; c += step) {
    const uint4 a = ld_global(reinterpret_cast<const uint4*>(x + c)), b = ld_global(reinterpret_cast<const uint4*>(w + c));
    if (copy) *reinterpret_cast<uint4*>(copy + c) = a;
    const uint32_t xs[4] = {a.x, a.y, a.z, a.w}, ws[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      dot = fmaf(__uint_as_float(xs[e] << 16), __uint_as_float(ws[e] << 16), dot);
      dot = fmaf(__uint_as_float(xs[e] & 0xFFFF0000u), __uint_as_float(ws[e] & 0xFFFF0000u), dot);
    }
  }
  return dot;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_dot(const __nv_bfloat16* x, const __nv_bfloat16* w, int K, int lane) {
  return warp_sum(dot_share(x, w, nullptr, K, lane * 8, 256));
}

// A largest logit and a sum relative to it.
struct LogSum {
  float most, sum;
};
__device__ __forceinline__ LogSum join_sums(LogSum a, LogSum b) {
  const float most = fmaxf(a.most, b.most), by = most == -INFINITY ? 0.0f : most;
  return {most, a.sum * exp2_approx((a.most - by) * kLog2e) + b.sum * exp2_approx((b.most - by) * kLog2e)};
}
// Whether a label's logit is a number that others can be held against.  What is not finite among the others shows in their sum, but against +infinity
// every other entry counts 0, and of a vocabulary of one there are no others.
__device__ __forceinline__ bool finite_label(float logit) { return fabsf(logit) < INFINITY; }
// loss = log(sum over all entries of exp(l)) - label's logit, from the sum over the others
__device__ __forceinline__ float loss_of(LogSum others, float label) {
  if (!finite_label(label)) return NAN;
  const float above = others.most - label;
  return above <= 0.0f ? log1pf(others.sum * expf(above)) : above + logf(others.sum + expf(-above));
}

// Reference of a live token: the label's logit, or in the repetition the row's largest if that is far above.
__device__ __forceinline__ float above_of(const LiveTokens& live, int row) { return __int_as_float(ld_global(live.above + row)); }
#endif

}  // namespace loss
}  // namespace peqa

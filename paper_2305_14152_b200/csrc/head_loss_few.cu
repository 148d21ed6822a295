// The loss of the vocabulary projection for up to 256 tokens (see head_loss.cu for the formulas and the launches around this one).
//
// Here the head is what there is to move, and with tokens as the matrix instruction's 256 rows most of it would be padding: 150 tokens took
// 56 us for the logits and as long for the gradient (32000 x 4096), one token no less.  So the head is its first operand, entries of the vocabulary
// (logits) or features (gradient) its rows, and the tokens, cut to a multiple of 16, its columns:
//   logits    D[entry, token]   = W[entry, :] X[token, :]
//   gradient  D[feature, token] = sum over the piece's entries of W[entry, feature] e[token, entry]
// An epilogue thread is an entry or a feature.  Sums over the entries go across the lanes: at distance o a lane keeps the tokens that
// agree with it in bit o and hands the others over, 31 exchanges for 32 tokens.  Every warp of a tile leaves its own.
//
// HBM bounds it: one token at 32000 x 4096 takes 49 us (46 for the kernel, 5.7 TB/s, of 40), 150 with gradient 129 to 133, of which 108 are the two passes
// over the head.  For the second to find in L2 what the first read last, all parts of the gradient's sums go through the vocabulary together, from its end.
#include "head_loss.cuh"
#include "kv_cache.cuh"

namespace peqa {

namespace {

using namespace loss;

constexpr int kMaxStages = 12;
constexpr int kFewSmemLimit = 216 * 1024;       // beside which a CTA of the kernel behind can already stand (100 tokens at 5000 x 2048 16.0 -> 13.9 us)

struct FewBarriers {
  uint64_t full[kMaxStages];     // leader: both CTAs' operands landed
  uint64_t empty[kMaxStages];    // each CTA: MMAs that read the stage completed
  uint64_t acc_full[2];          // each CTA
  uint64_t acc_empty[2];         // leader: both CTAs' epilogues drained it
  uint32_t tmem_base;
  int abort_flag;
  int wait_limit_us;             // must follow abort_flag (read by the bounded waits)
  float ref[kFewTokens];
  int label[kFewTokens];         // -1 where there is no token
};
constexpr int kFewStaging = 2048;        // of an epilogue warp: 32 tokens x 16 entries, twice
constexpr int kFewSmemFixed = 1024 + 8 * kFewStaging + (int)((sizeof(FewBarriers) + 127) / 128 * 128);

struct FewParams {
  LossParams p;
  float* grads;                  // [splits, 256, K]
  // without gradient: the call's tokens, `tokens` of them, and their labels
  const int32_t* labels;
  const __nv_bfloat16* x;
  const __nv_bfloat16* W;
  int tokens;
  int nt;                        // columns: tokens, a multiple of 16
  int stages, stage_bytes;
};

// Items of a launch: the gradient's, then logits, dealt out in turns.
struct FewItem {
  bool grad;
  int col, kbs, split;
};
struct FewWalk {
  int n1, n2, features;
  __device__ __forceinline__ FewWalk(const LossParams& p, bool any) {
    features = (p.K + kTile - 1) / kTile;
    n1 = any ? p.tiles : 0;
    n2 = any && p.back_blocks ? features * p.splits : 0;
  }
  __device__ __forceinline__ bool get(const LossParams& p, int i, FewItem& it) const {
    int e = (int)(blockIdx.x >> 1) + i * (int)(gridDim.x >> 1);
    if (e >= n1 + n2) return false;
    it.grad = e < n2;
    if (it.grad) {
      it.split = e / features;
      it.col = e - it.split * features;
      it.kbs = (p.back_blocks - it.split + p.splits - 1) / p.splits;
    } else {
      it.split = 0;
      it.col = e - n2;
      it.kbs = p.k_blocks;
    }
    return true;
  }
};

// Joins 32 lanes' 32 values: lane j ends with value j's.
template <typename F>
__device__ __forceinline__ float fold32(float (&v)[32], int lane, F&& join) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int j = 0; j < o; ++j) {
      const float keep = up ? v[j + o] : v[j], give = up ? v[j] : v[j + o];
      v[j] = join(keep, __shfl_xor_sync(0xffffffffu, give, o));
    }
  }
  return v[0];
}

template <bool GRAD>
__global__ void __launch_bounds__(kLossThreads, 1)
head_loss_few_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x,
                     const __grid_constant__ CUtensorMap tmap_wt, const __grid_constant__ CUtensorMap tmap_e,
                     const __grid_constant__ CUtensorMap tmap_e_out, const FewParams q) {
  const LossParams& p = q.p;
  if (GRAD && p.second) {
    wait_for_kernel_before();
    if (ld_global(p.again) == 0) {
      let_kernel_behind_in();
      return;
    }
  }
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* staging = base + q.stages * q.stage_bytes;
  FewBarriers* bars = reinterpret_cast<FewBarriers*>(staging + 8 * kFewStaging);
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  volatile int* abort_flag = &bars->abort_flag;

  if (threadIdx.x == 0) {
    for (int s = 0; s < q.stages; ++s) {
      mbar_init(smem_u32(&bars->full[s]), 1);
      mbar_init(smem_u32(&bars->empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&bars->acc_full[b]), 1);
      mbar_init(smem_u32(&bars->acc_empty[b]), 16);          // 8 epilogue warps in each CTA
    }
    bars->abort_flag = 0;
    bars->wait_limit_us = p.status[4];
    fence_mbar_init();
    prefetch_tmap(&tmap_w);
    prefetch_tmap(&tmap_x);
    if (GRAD) {
      prefetch_tmap(&tmap_wt);
      prefetch_tmap(&tmap_e);
      prefetch_tmap(&tmap_e_out);
    }
  }
  if (warp == 2) {
    tmem_alloc_pair(smem_u32(&bars->tmem_base), 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  wait_for_kernel_before();
  let_next_in(false);
  const uint32_t tmem_base = bars->tmem_base;
  const int live = GRAD ? min(kFewTokens, ld_global(p.live.count)) : q.tokens;
  const FewWalk walk(p, live > 0);
  const int half_entries = p.width >> 1, half_tokens = q.nt >> 1;     // of a CTA
  const uint32_t b_bytes = half_tokens * (kDepth * 2);

  if (warp == 0) {
    // ------------------------------------------ operands (one lane)
    if (const uint32_t lane = elect_lane(); lane == 0) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      FewItem item;
      // self-test knob (peqa_selftest_configure): one byte more is announced than will arrive
      const uint32_t starve = p.status[5] != 0 ? 1u : 0u;
      for (int i = 0; ok && walk.get(p, i, item); ++i) {
        const uint32_t bytes = 2 * ((item.grad ? (uint32_t)kOperandBytes : half_entries * (kDepth * 2)) + b_bytes) + starve;
        for (int kb = 0; kb < item.kbs; ++kb) {
          if (!mbar_wait_cluster(smem_u32(&bars->empty[s]), ph ^ 1u, abort_flag)) { ok = false; break; }
          if (leader) mbar_arrive_expect_tx(smem_u32(&bars->full[s]), bytes);
          const uint32_t bar = mapa_shared(smem_u32(&bars->full[s]), 0), a = smem_u32(base + s * q.stage_bytes);
          // All parts of the gradient's sum go through the piece together, from its end: what the logits were made of last is still in L2.
          const int k = (item.grad ? p.back_blocks - 1 - item.split - kb * p.splits : kb) * kDepth;
          if (!item.grad) {
            tma_load_2d_pair(a, &tmap_w, bar, k, (p.tile0 + item.col) * p.width + (int)rank * half_entries);
            tma_load_2d_pair(a + kOperandBytes, &tmap_x, bar, k, (int)rank * half_tokens);
          } else if (GRAD) {
            const int m0 = item.col * kTile + (int)rank * 128;
#pragma unroll
            for (int m = 0; m < 2; ++m) tma_load_2d_pair(a + m * 8192, &tmap_wt, bar, m0 + 64 * m, p.back0 + k);
            tma_load_2d_pair(a + kOperandBytes, &tmap_e, bar, k, (int)rank * half_tokens);
          }
          if (++s == q.stages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------ MMA issuer (leader CTA, one lane)
    if (leader) if (const uint32_t lane = elect_lane(); lane == 0) {
      const uint32_t idesc_logits = idesc_bf16_f32(256, q.nt, 0, 0), idesc_grad = idesc_bf16_f32(256, q.nt, 1, 0);
      const uint32_t a0 = smem_u32(base);
      const uint64_t adesc_logits = smem_desc_sw128(a0, 16, 1024), adesc_grad = smem_desc_sw128(a0, 8192, 1024);
      const uint64_t bdesc0 = smem_desc_sw128(a0 + kOperandBytes, 16, 1024);
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      FewItem item;
      for (int i = 0; ok && walk.get(p, i, item); ++i) {
        const int buf = i & 1;
        if (!mbar_wait_cluster(smem_u32(&bars->acc_empty[buf]), ((i >> 1) & 1u) ^ 1u, abort_flag)) break;
        tc_fence_after();
        const uint32_t d = tmem_base + buf * 256;
        for (int kb = 0; kb < item.kbs; ++kb) {
          if (!mbar_wait_cluster(smem_u32(&bars->full[s]), ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint64_t by = (uint64_t)(s * (q.stage_bytes >> 4)), bdesc = bdesc0 + by;
          if (!item.grad) {
#pragma unroll
            for (int k = 0; k < kDepth / 16; ++k)
              mma_bf16_ss_pair(d, adesc_logits + by + k * (32 / 16), bdesc + k * (32 / 16), idesc_logits, (kb | k) != 0 ? 1u : 0u);
          } else if (GRAD) {
#pragma unroll
            for (int k = 0; k < kDepth / 16; ++k)
              mma_bf16_ss_pair(d, adesc_grad + by + k * (16 * 128 / 16), bdesc + k * (32 / 16), idesc_grad, (kb | k) != 0 ? 1u : 0u);
          }
          mma_commit_pair(smem_u32(&bars->empty[s]), 3);
          if (++s == q.stages) {
            s = 0;
            ph ^= 1u;
          }
        }
        if (ok) mma_commit_pair(smem_u32(&bars->acc_full[buf]), 3);
      }
    }
  } else if (warp == 3) {
    // ------------------------------------------ without gradient: the labels' logits, while the tiles are worked on.  In binary32: a tile's
    // sums drop what is below their last bit, always towards zero, which the label's, the largest as a rule, shows most (a loss of 1e-3 off by 3e-5 of
    // itself).
    if (!GRAD) {
      for (int t = blockIdx.x; t < live; t += gridDim.x) {
        const int label = ld_global(q.labels + t);
        if ((unsigned)label >= (unsigned)p.V) continue;
        const float dot = warp_dot(q.x + (size_t)t * p.K, q.W + (size_t)label * p.K, p.K, lane);
        if (lane == 0) p.live.ref[t] = dot;
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------ epilogue: thread = entry or feature, every other 32 tokens
    {
      const int t = (int)threadIdx.x - 128;
      float ref = 0.0f;
      int label = -1;
      if (GRAD && t < live) {
        ref = ld_global(p.live.ref + t);
        if (p.second) ref += above_of(p.live, t);
        label = ld_global(p.live.label + t);
      }
      if (!GRAD && t < live) label = ld_global(q.labels + t);
      bars->ref[t] = ref;
      bars->label[t] = label;
      named_barrier_sync(1, 256);
    }
    const int quarter = warp & 3, half = (warp - 4) >> 2, in_half = quarter * 32 + lane;
    const int chunks = (q.nt + 31) >> 5;
    FewItem item;
    for (int i = 0; walk.get(p, i, item); ++i) {
      const int buf = i & 1;
      const uint32_t from = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * 256;
      const uint32_t acc_empty = mapa_shared(smem_u32(&bars->acc_empty[buf]), 0);
      if (!warp_wait_cluster(smem_u32(&bars->acc_full[buf]), (uint32_t)(i >> 1) & 1u, abort_flag)) break;
      tc_fence_after();
      const int in_piece = item.col * p.width + (int)rank * half_entries + in_half;       // logits: this thread's entry
      const int entry = p.tile0 * p.width + in_piece;
      const bool mine = in_half < half_entries, valid = mine && entry < p.V;
      const int feature = item.col * kTile + (int)rank * 128 + in_half;                   // gradient: its feature
#pragma unroll 1
      for (int c = half; c < chunks; c += 2) {
        uint32_t r[32];
        tmem_ld_32x32(from + c * 32, r);
        tmem_ld_wait();
        if (c + 2 >= chunks) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(acc_empty);
        }
        const int t0 = c * 32;
        if (!item.grad) {
          float v[32];
          const size_t slot = ((size_t)((p.tile0 + item.col) * 2 + (int)rank) * 4 + quarter) * kFewTokens + t0 + lane;
          if (!GRAD) {
            float x[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = x[j] = valid && bars->label[t0 + j] != entry ? __uint_as_float(r[j]) : -INFINITY;
            const float most = fold32(v, lane, [](float a, float b) { return fmaxf(a, b); });
            const float by = most == -INFINITY ? 0.0f : most;
#pragma unroll
            for (int j = 0; j < 32; ++j) x[j] = exp2_approx((x[j] - __shfl_sync(0xffffffffu, by, j)) * kLog2e);
            const float sum = fold32(x, lane, [](float a, float b) { return a + b; });
            reinterpret_cast<float2*>(p.sums)[slot] = make_float2(most, sum);
          } else {
            bool far = false;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              const float x = __uint_as_float(r[j]) - bars->ref[t0 + j];
              const bool on = valid && bars->label[t0 + j] != entry;
              v[j] = on ? exp2_approx(x * kLog2e) : 0.0f;
              far |= on && x > kFarAbove;
            }
            if (far && !p.second) {
              // rare: each token's largest is noted, and the whole is done once more
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                const float x = __uint_as_float(r[j]) - bars->ref[t0 + j];
                if (t0 + j < live && bars->label[t0 + j] != entry && x > kFarAbove) {
                  atomicMax(p.live.above + t0 + j, __float_as_int(x));
                  *p.again = 1;
                }
              }
            }
            // [token][entry] in two boxes of 16 entries, which a CTA's share of a tile is a multiple of
            if (lane == 0) bulk_wait_group_read0();
            __syncwarp();
            uint8_t* at = staging + (warp - 4) * kFewStaging + (lane >> 4) * 1024 + (lane & 15) * 2;
#pragma unroll
            for (int j = 0; j < 32; ++j) *reinterpret_cast<__nv_bfloat16*>(at + j * 32) = __float2bfloat16_rn(v[j]);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              const int first = in_piece;                     // of the warp's entries
#pragma unroll
              for (int b = 0; b < 2; ++b)
                if (t0 < live && quarter * 32 + b * 16 < half_entries)
                  tma_store_2d(&tmap_e_out, smem_u32(staging + (warp - 4) * kFewStaging + b * 1024), first + b * 16, t0);
              bulk_commit_group();
            }
            p.sums[slot] = fold32(v, lane, [](float a, float b) { return a + b; });
          }
        } else if (GRAD) {
          if (feature < p.K) {
            float* at = q.grads + ((size_t)item.split * kFewTokens + t0) * p.K + feature;
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (t0 + j < live) {
                float* to = at + (size_t)j * p.K;
                *to = p.first_back ? __uint_as_float(r[j]) : *to + __uint_as_float(r[j]);
              }
          }
        }
      }
      if (half >= chunks) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(acc_empty);
      }
    }
    if (GRAD && lane == 0) bulk_wait_group0();
  }

  if (*abort_flag) {
    // let copies and MMAs already in flight finish before memory is released
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
  if (threadIdx.x == 0 && bars->abort_flag) {
    atomicExch(p.status, (int)PEQA_ERR_DEVICE_TIMEOUT);
    p.status[1] = (int)blockIdx.x;
  }
}

template <bool GRAD>
int launch_few_t(const CUtensorMap& w, const CUtensorMap& x, const CUtensorMap& wt, const CUtensorMap& e_in, const CUtensorMap& e_out,
                 const FewParams& q, int pairs, size_t smem, cudaStream_t st) {
  auto kern = head_loss_few_kernel<GRAD>;
  static std::atomic<uint64_t> done{0};
  PEQA_TRY(allow_smem(kern, kFewSmemLimit, done));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * pairs, 1, 1);
  cfg.blockDim = dim3(kLossThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  PEQA_CUDA(cudaLaunchKernelEx(&cfg, kern, w, x, wt, e_in, e_out, q));
  return PEQA_OK;
}

// The losses of few tokens without gradient, a token a CTA.
__global__ void __launch_bounds__(256) loss_few_finish_kernel(const float2* sums, int parts, const int32_t* labels, int V, const float* ref,
                                                              float* loss, int* status) {
  wait_for_kernel_before();
  let_kernel_behind_in();
  __shared__ LogSum part[8];
  const int token = blockIdx.x, lane = threadIdx.x & 31;
  const int label = ld_global(labels + token);
  const float own = ld_global(ref + token);
  if ((unsigned)label >= (unsigned)V) {
    if (threadIdx.x == 0) {
      if (label >= V) note_bad_index(status);
      loss[token] = 0.0f;
    }
    return;
  }
  LogSum v = {-INFINITY, 0.0f};
#pragma unroll 4
  for (int h = threadIdx.x; h < parts; h += 256) {
    const float2 u = ld_global(sums + (size_t)h * kFewTokens + token);
    v = join_sums(v, {u.x, u.y});
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = join_sums(v, {__shfl_xor_sync(0xffffffffu, v.most, o), __shfl_xor_sync(0xffffffffu, v.sum, o)});
  if (lane == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < 8; ++w) v = join_sums(v, part[w]);
  loss[token] = loss_of(v, own);
}

}  // namespace

int loss::few_maps(FewCall& call, int width, int V, int K, bool grad) {
  const uint32_t half_tokens = ((call.tokens + 15) & ~15) / 2;
  PEQA_TRY(bf16_map(&call.w, call.W, K, V, width / 2));
  PEQA_TRY(bf16_map(&call.x, call.rows, K, grad ? kFewTokens : call.tokens, half_tokens));
  if (!grad) return PEQA_OK;
  PEQA_TRY(bf16_map(&call.wt, call.W, K, V, 64));
  for (int b = 0; b < (call.e[0] == call.e[1] ? 1 : 2); ++b)
    PEQA_TRY(loss_map(&call.e_out[b], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, call.e[b], call.pitch, kFewTokens, 2, 16, 32, CU_TENSOR_MAP_SWIZZLE_NONE));
  return PEQA_OK;
}

int loss::launch_few(const LossParams& p, const FewCall& call, int turn, int in_entries, bool grad, int pairs, cudaStream_t st) {
  FewParams q;
  q.p = p;
  q.grads = call.grads;
  q.labels = call.labels;
  q.x = static_cast<const __nv_bfloat16*>(call.rows);
  q.W = static_cast<const __nv_bfloat16*>(call.W);
  q.tokens = call.tokens;
  q.nt = (call.tokens + 15) & ~15;
  q.stage_bytes = kOperandBytes + q.nt / 2 * (kDepth * 2);
  q.stages = (kFewSmemLimit - kFewSmemFixed) / q.stage_bytes;
  if (q.stages > kMaxStages) q.stages = kMaxStages;
  const size_t smem = (size_t)q.stages * q.stage_bytes + kFewSmemFixed;
  if (!grad) return launch_few_t<false>(call.w, call.x, call.w, call.w, call.w, q, pairs, smem, st);
  CUtensorMap e_in = call.w;
  // of the piece's own width: what its last stage has beyond that is read as zeros
  if (in_entries > 0) PEQA_TRY(bf16_map(&e_in, call.e[turn ^ 1], in_entries, kFewTokens, q.nt / 2, (uint64_t)call.pitch * 2));
  return launch_few_t<true>(call.w, call.x, call.wt, e_in, call.e_out[call.e[0] == call.e[1] ? 0 : turn], q, pairs, smem, st);
}

int loss::finish_few(const LossParams& p, const FewCall& call, int parts, float* loss, cudaStream_t st) {
  return launch_after(loss_few_finish_kernel, call.tokens, 256, st, reinterpret_cast<const float2*>(p.sums), parts, call.labels, p.V,
                      static_cast<const float*>(p.live.ref), loss, p.status);
}

}  // namespace peqa

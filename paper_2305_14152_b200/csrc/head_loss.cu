// Softmax cross entropy of the vocabulary projection, with its gradient, in pieces of the vocabulary:
//
//   l[t,v] = sum_j X[t,j] W[v,j]          loss[t] = log sum_v exp(l[t,v] - l[t,y_t])
//   dX[t]  = g[t] * (sum_v p[t,v] W[v] - W[y_t]),   p = softmax of l[t]
//
// W [V, K] is the frozen head in bf16, so dX is all there is to a gradient.  The logits are formed once and never stored:
// a contraction costs 2 T V K operations, and with a second one for the gradient these two are all.  What allows that is a reference
// r[t] that is known before the first logit is: r = l[t,y_t], the label's own, one dot product per token.  With e[t,v] = exp(l[t,v] - r[t]),
// the label left out, and s[t] their sum,
//
//   loss[t] = r[t] - l[t,y_t] + log(s[t] + exp(l[t,y_t] - r[t]))       (= log1p(s[t]) when r is the label's logit)
//   dX[t]   = g[t] * (sum_{v != y_t} e[t,v] W[v] - s[t] W[y_t]) / (s[t] + exp(l[t,y_t] - r[t]))
//
// and neither cancels: a token whose label is all but certain keeps the relative precision of its loss and gradient.  e is rounded to bf16 for
// the second contraction (off by 2^-8 of itself at most, whatever its size, since bf16 has binary32's exponents; s is summed in binary32 before
// that).  Nothing overflows while no logit lies more than kFarAbove above r.  Where one does, the epilogue notes the row's largest and raises
// the chunk's flag, and the chunk's launches, which follow once more and otherwise return at once, repeat it with that as r.
//
// Launches.  loss_gather_kernel copies the tokens that count (labels of instruction samples are mostly ignored) side by
// side and takes r.  Then, piece by piece of the vocabulary, head_loss_kernel works through two kinds of tiles of 256 x 256: logits
// of piece p, whose epilogue leaves e in bf16 and its sums, and the gradient's sums over piece p - 1, added to binary32 [T, K].  Both
// kinds in one launch share out evenly where one would leave a last round half empty; no CTA waits for another but for the
// one that it shares its tiles with.  loss_finish_kernel adds up s and writes loss and dX.
//
// A tile belongs to a pair of CTAs (cta_group::2), operands come by TMA through a ring of six stages of 64, and two accumulators of
// 256 columns fill tensor memory, so that one tile's epilogue runs under the next one's contraction.
//
// The tensor cores bound it, under the power limit: 4096 tokens at 32000 x 8192 take 3350 to 3430 us, 1.25 to 1.28 PFLOP/s (losses alone, 2048 tokens at 32000 x 4096,
// 406 to 417; their kernel 1.4 PFLOP/s, what a library's product of the size sustains).  A launch with both kinds of tiles keeps the tensor pipe busy 90 to 93 %
// of the time.  Tiles of the gradient dealt out column by column in groups of token blocks instead of row by row: 3551 -> 3435 us, as a piece's
// rows of the head (134 MB at 8192 features) were read once for every 74 tiles before.
#include <cuda.h>
#include <cuda_bf16.h>

#include "common.cuh"
#include "head_loss.cuh"
#include "kv_cache.cuh"

namespace peqa {

int loss::loss_map(CUtensorMap* m, CUtensorMapDataType type, const void* base, uint64_t inner, uint64_t outer, int size, uint32_t box_x,
             uint32_t box_y, CUtensorMapSwizzle swizzle, uint64_t pitch) {
  EncodeTiledFn enc = nullptr;
  PEQA_TRY(tensor_map_encoder(&enc));
  cuuint64_t dims[2] = {inner, outer};
  cuuint64_t strides[1] = {pitch ? pitch : inner * size};
  cuuint32_t box[2] = {box_x, box_y};
  cuuint32_t estr[2] = {1, 1};
  if (enc(m, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cuda_fail(cudaErrorInvalidValue);
  return PEQA_OK;
}

namespace {

using namespace ptx;
using namespace loss;

constexpr int kStages = 6;
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kStagingBytes = 4096;             // of an epilogue warp
constexpr int kLossSmem = kStages * kStageBytes + 8 * kStagingBytes + 1024 + 512;
constexpr int kSideThreads = 256;               // of the kernels before and behind
constexpr int kChunkRows = 8192;

struct LossBarriers {
  uint64_t full[kStages];        // leader: both CTAs' operands landed
  uint64_t empty[kStages];       // each CTA: MMAs that read the stage completed
  uint64_t acc_full[2];          // each CTA
  uint64_t acc_empty[2];         // leader: both CTAs' epilogues drained it
  uint32_t tmem_base;
  int abort_flag;
  int wait_limit_us;             // must follow abort_flag (read by the bounded waits)
};

// How the tokens that count share a chunk's buffers and pairs, known where they have been counted.  Where they fill half of the buffers, a
// quarter or an eighth, as of instruction samples, of which the answers count alone, several pieces of the vocabulary are taken at once, and where their tiles
// of the gradient are fewer than the pairs, the sum over a piece is cut into parts with sums of their own.
constexpr int kFolds = 4;
struct Share {
  int blocks;            // of 256 tokens
  int fold;              // log2 of the pieces taken at once
  int splits;            // parts
};
struct ShareRule {
  int blocks, pieces, features, pairs;     // features: tiles of 256
  int splits;            // parts that the buffer has room for when all tokens count
  int least;             // stages of the narrowest piece
};
__host__ __device__ inline Share share_of(const ShareRule& r, int rows_live) {
  Share s = {(rows_live + kTile - 1) / kTile, 0, 1};
  if (s.blocks == 0) return s;
  while (s.fold + 1 < kFolds && (2 << s.fold) * s.blocks <= r.blocks && (1 << s.fold) < r.pieces) ++s.fold;
  const int tiles = s.blocks * r.features, room = r.splits * r.blocks / s.blocks;
  if (tiles < r.pairs) s.splits = r.pairs / tiles;
  s.splits = s.splits < 16 ? s.splits : 16;
  s.splits = s.splits < r.least ? s.splits : r.least;
  s.splits = s.splits < room ? s.splits : room;
  return s;
}

// What a launch of the ordinary kernel is given beside LossParams, whose piece is its own here.
struct LossLaunch {
  ShareRule rule;
  int number;            // of the launch: logits of piece `number`, the gradient's sum over the one before (pieces as many as are taken at once)
  int all_tiles, pieces;
  __host__ __device__ int piece_tile(int i) const { return (int)((long long)all_tiles * (i < pieces ? i : pieces) / pieces); }
};
struct LossMaps {
  CUtensorMap x, w, wt, sum;
  CUtensorMap e_out[kFolds], e_in[kFolds];
};

struct Item {
  bool grad;
  int row;               // block of 256 tokens of the chunk
  int col;               // tile of the piece (logits), 256 features (gradient)
  int split;
  int kb0, kbs;          // stages of 64: the first (gradient), how many
};

// A pair's items, one after the other.  Tiles of the gradient, the longer ones as a rule, are dealt out first; the pairs that get one less
// begin with as many tiles of logits as take its time, and the others are dealt to all.
struct Walk {
  int pair, pairs, n1, n2, n2_mine, lo_first, lo_pairs, lo_mine, lo_total;
  int rows, features, splits, fold, back_group;
  int tile0, tiles, back0, back_blocks;
  __device__ __forceinline__ Walk(const LossParams& p, const LossLaunch& l, int rows_live) {
    const Share share = share_of(l.rule, rows_live);
    pair = blockIdx.x >> 1;
    pairs = gridDim.x >> 1;
    rows = share.blocks;
    features = l.rule.features;
    splits = share.splits;
    fold = share.fold;
    back_group = max(4, p.back_group >> fold);
    const int before = l.piece_tile((l.number - 1) << fold), behind = l.piece_tile((l.number + 1) << fold);
    tile0 = l.piece_tile(l.number << fold);
    tiles = behind - tile0;
    back0 = before * p.width;
    back_blocks = l.number > 0 ? ((tile0 - before) * p.width + kDepth - 1) / kDepth : 0;
    n1 = rows * tiles;
    n2 = back_blocks ? rows * features * splits : 0;
    n2_mine = n2 > pair ? (n2 - pair - 1) / pairs + 1 : 0;
    lo_first = n2 % pairs;
    lo_pairs = lo_first ? pairs - lo_first : 0;
    const int each = lo_pairs ? (back_blocks / splits + p.k_blocks / 2) / p.k_blocks : 0;
    lo_total = min(n1, each * lo_pairs);
    const int e = pair - lo_first;
    lo_mine = lo_pairs && e >= 0 && lo_total > e ? (lo_total - e - 1) / lo_pairs + 1 : 0;
  }
  // Groups of token blocks, in them column by column of tiles: what the pairs read at a time stays in L2.
  __device__ __forceinline__ void deal(int e, int group, int cols, Item& it) const {
    const int g = e / (group * cols), first = g * group, in_group = min(group, rows - first);
    e -= first * cols;
    it.col = e / in_group;
    it.row = first + e - it.col * in_group;
  }
  __device__ __forceinline__ bool get(const LossParams& p, int i, Item& it) const {
    if (i < n2_mine) {
      int e = pair + i * pairs;
      it.grad = true;
      it.split = e / (rows * features);
      deal(e - it.split * rows * features, back_group, features, it);
      it.kb0 = (int)((long long)it.split * back_blocks / splits);
      it.kbs = (int)((long long)(it.split + 1) * back_blocks / splits) - it.kb0;
      return true;
    }
    i -= n2_mine;
    int e;
    if (i < lo_mine) {
      e = pair - lo_first + i * lo_pairs;
    } else {
      const long long at = (long long)lo_total + pair + (long long)(i - lo_mine) * pairs;
      if (at >= n1) return false;
      e = (int)at;
    }
    it.grad = false;
    deal(e, p.group, tiles, it);
    it.split = 0;
    it.kb0 = 0;
    it.kbs = p.k_blocks;
    return true;
  }
};

template <bool GRAD>
__global__ void __launch_bounds__(kLossThreads, 1)
head_loss_kernel(const __grid_constant__ LossMaps maps, const LossParams p, const LossLaunch l) {
  if (GRAD && p.second) {
    wait_for_kernel_before();
    if (ld_global(p.again) == 0) {
      let_kernel_behind_in();
      return;
    }
  }
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* staging = base + kStages * kStageBytes;
  LossBarriers* bars = reinterpret_cast<LossBarriers*>(staging + 8 * kStagingBytes);
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  volatile int* abort_flag = &bars->abort_flag;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
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
    prefetch_tmap(&maps.x);
    prefetch_tmap(&maps.w);
    if (GRAD) {
      prefetch_tmap(&maps.wt);
      prefetch_tmap(&maps.sum);
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
  const int rows_live = min(p.rows, ld_global(p.live.count) - p.row0);     // none or fewer: no items
  const Walk walk(p, l, rows_live > 0 ? rows_live : 0);
  const CUtensorMap *tmap_e_out = &maps.e_out[walk.fold], *tmap_e_in = &maps.e_in[walk.fold];

  if (warp == 0) {
    // ------------------------------------------ operands (one lane)
    if (const uint32_t lane = elect_lane(); lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      Item item;
      // self-test knob (peqa_selftest_configure): one byte more is announced than will arrive
      const uint32_t starve = p.status[5] != 0 ? 1u : 0u;
      const uint32_t logits_bytes = 2 * kOperandBytes + p.width * (kDepth * 2);      // of both CTAs
      for (int i = 0; ok && walk.get(p, i, item); ++i) {
        const int row = item.row * kTile + (int)rank * 128;
        for (int kb = 0; kb < item.kbs; ++kb, ++it) {
          const int s = it % kStages;
          if (!mbar_wait_cluster(smem_u32(&bars->empty[s]), ((it / kStages) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
          if (leader) mbar_arrive_expect_tx(smem_u32(&bars->full[s]), (item.grad ? 2 * kStageBytes : logits_bytes) + starve);
          const uint32_t bar = mapa_shared(smem_u32(&bars->full[s]), 0), a = smem_u32(base + s * kStageBytes);
          if (!item.grad) {
            tma_load_2d_pair(a, &maps.x, bar, kb * kDepth, p.row0 + row);
            tma_load_2d_pair(a + kOperandBytes, &maps.w, bar, kb * kDepth, (walk.tile0 + item.col) * p.width + (int)rank * (p.width >> 1));
          } else if (GRAD) {
            const int k = (item.kb0 + kb) * kDepth, n0 = item.col * kTile + (int)rank * 128;
            tma_load_2d_pair(a, tmap_e_in, bar, k, row);
#pragma unroll
            for (int m = 0; m < 2; ++m)
              tma_load_2d_pair(a + kOperandBytes + m * 8192, &maps.wt, bar, n0 + 64 * m, walk.back0 + k);
          }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------ MMA issuer (leader CTA, one lane)
    if (leader) if (const uint32_t lane = elect_lane(); lane == 0) {
      const uint32_t idesc_logits = idesc_bf16_f32(256, p.width, 0, 0);
      constexpr uint32_t idesc_grad = idesc_bf16_f32(256, 256, 0, 1);
      const uint32_t a0 = smem_u32(base);
      const uint64_t adesc0 = smem_desc_sw128(a0, 16, 1024);
      const uint64_t bdesc_logits = smem_desc_sw128(a0 + kOperandBytes, 16, 1024);
      const uint64_t bdesc_grad = smem_desc_sw128(a0 + kOperandBytes, 8192, 1024);
      uint32_t s = 0, ph = 0;
      bool ok = true;
      Item item;
      for (int i = 0; ok && walk.get(p, i, item); ++i) {
        const int buf = i & 1;
        if (!mbar_wait_cluster(smem_u32(&bars->acc_empty[buf]), ((i >> 1) & 1u) ^ 1u, abort_flag)) break;
        tc_fence_after();
        const uint32_t d = tmem_base + buf * 256;
        for (int kb = 0; kb < item.kbs; ++kb) {
          if (!mbar_wait_cluster(smem_u32(&bars->full[s]), ph, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint64_t adesc = adesc0 + s * (kStageBytes >> 4);
          const uint32_t at = s;
          if (!item.grad) {
            const uint64_t bdesc = bdesc_logits + s * (kStageBytes >> 4);
#pragma unroll
            for (int k = 0; k < kDepth / 16; ++k)
              mma_bf16_ss_pair(d, adesc + k * (32 / 16), bdesc + k * (32 / 16), idesc_logits, (kb | k) != 0 ? 1u : 0u);
          } else if (GRAD) {
            const uint64_t bdesc = bdesc_grad + s * (kStageBytes >> 4);
#pragma unroll
            for (int k = 0; k < kDepth / 16; ++k)
              mma_bf16_ss_pair(d, adesc + k * (32 / 16), bdesc + k * (16 * 128 / 16), idesc_grad, (kb | k) != 0 ? 1u : 0u);
          }
          if (++s == kStages) {
            s = 0;
            ph ^= 1u;
          }
          mma_commit_pair(smem_u32(&bars->empty[at]), 3);
        }
        if (ok) mma_commit_pair(smem_u32(&bars->acc_full[buf]), 3);
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------ epilogue: thread = token, 128 of the tile's columns
    const int quarter = warp & 3, half = (warp - 4) >> 2;
    uint8_t* mine = staging + (warp - 4) * kStagingBytes;
    Item item;
    for (int i = 0; walk.get(p, i, item); ++i) {
      const int buf = i & 1;
      const int row_w = item.row * kTile + (int)rank * 128 + quarter * 32, row = row_w + lane;
      const bool live = row < rows_live;
      const uint32_t from = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * 256 + half * 128;
      const uint32_t acc_empty = mapa_shared(smem_u32(&bars->acc_empty[buf]), 0);
      float ref = 0.0f;
      int label = -1, cols = 0;                             // both counted from this half tile's first entry
      const int entry0 = (walk.tile0 + item.col) * p.width + half * 128;
      const int chunks = item.grad ? 4 : min(4, (p.width - half * 128) >> 5);      // none: 0 or less
      if (!item.grad) {
        cols = min(p.V - entry0, chunks * 32);
        if (live) {
          ref = ld_global(p.live.ref + p.row0 + row);
          if (GRAD && p.second) ref += above_of(p.live, p.row0 + row);
          label = ld_global(p.live.label + p.row0 + row) - entry0;
        }
      }
      if (!warp_wait_cluster(smem_u32(&bars->acc_full[buf]), (uint32_t)(i >> 1) & 1u, abort_flag)) break;
      tc_fence_after();
      float most = -INFINITY, sum = 0.0f;
#pragma unroll 1
      for (int c = 0; c < chunks; ++c) {
        uint32_t v[32];
        tmem_ld_32x32(from + c * 32, v);
        tmem_ld_wait();
        if (c + 1 == chunks) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(acc_empty);
        }
        if (!item.grad) {
          // entries beyond the vocabulary, and the label's own, are not among the others
          if (cols < c * 32 + 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (c * 32 + j >= cols) v[j] = __float_as_uint(-INFINITY);
          }
          if ((unsigned)(label - c * 32) < 32u) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (c * 32 + j == label) v[j] = __float_as_uint(-INFINITY);
          }
          float here = -INFINITY;
#pragma unroll
          for (int j = 0; j < 32; ++j) here = fmaxf(here, __uint_as_float(v[j]));
          if (!GRAD) {
            // sums relative to the largest so far; a number that is not finite makes both so
            const float next = fmaxf(most, here), by = next == -INFINITY ? 0.0f : next;
            sum *= exp2_approx((most - by) * kLog2e);
#pragma unroll
            for (int j = 0; j < 32; ++j) sum += exp2_approx((__uint_as_float(v[j]) - by) * kLog2e);
            most = next;
          } else {
            most = fmaxf(most, here);
            uint8_t* at = mine + (c & 1) * 2048;
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            __syncwarp();
            uint8_t* out = at + lane * 64;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              float e[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                e[j] = exp2_approx((__uint_as_float(v[8 * q + j]) - ref) * kLog2e);
                sum += e[j];
              }
              *reinterpret_cast<uint4*>(out + ((q ^ ((lane >> 1) & 3)) << 4)) =
                  make_uint4(bf16_pair(e[0], e[1]), bf16_pair(e[2], e[3]), bf16_pair(e[4], e[5]), bf16_pair(e[6], e[7]));
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              if (row_w < rows_live) tma_store_2d(tmap_e_out, smem_u32(at), item.col * p.width + half * 128 + c * 32, row_w);
              bulk_commit_group();
            }
          }
        } else if (GRAD) {
          if (lane == 0) bulk_wait_group_read0();
          __syncwarp();
          uint8_t* out = mine + lane * 128;
#pragma unroll
          for (int q = 0; q < 8; ++q)
            *reinterpret_cast<uint4*>(out + ((q ^ (lane & 7)) << 4)) = make_uint4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            const int x = item.col * kTile + half * 128 + c * 32, y = item.split * walk.rows * kTile + row_w;
            if (row_w < rows_live && x < p.K) {
              if (l.number == 1) tma_store_2d(&maps.sum, smem_u32(mine), x, y);
              else tma_add_2d(&maps.sum, smem_u32(mine), x, y);
            }
            bulk_commit_group();
          }
        }
      }
      if (chunks <= 0) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(acc_empty);
      }
      if (!item.grad) {
        const size_t slot = ((size_t)(walk.tile0 + item.col) * 2 + half) * p.rows + row;
        if (!GRAD) {
          reinterpret_cast<float2*>(p.sums)[slot] = make_float2(most, sum);
        } else {
          p.sums[slot] = sum;
          if (live && !p.second && most - ref > kFarAbove) {
            atomicMax(p.live.above + p.row0 + row, __float_as_int(most - ref));
            *p.again = 1;
          }
        }
      }
      if (GRAD) {
        // the halves of the staging memory change hands by turns of c; the next tile may be of the other kind
        if (lane == 0) bulk_wait_group_read0();
        __syncwarp();
      }
    }
    if (lane == 0) bulk_wait_group0();
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

struct GatherParams {
  const __nv_bfloat16* X;
  const __nv_bfloat16* W;
  const int32_t* labels;
  int T, V, K;
  LiveTokens live;
  __nv_bfloat16* rows;     // live tokens' X, side by side
  int* again;              // flags of the chunks
  int chunks;
  const int* counts;       // of spans of kCountSpan tokens, or nullptr
  float* loss;
  __nv_bfloat16* dX;       // or nullptr
  int* status;
};

// Sum over the CTA (kSideThreads), in one order, to all threads.  part: 8 floats of shared memory that nobody reads any more.
template <typename V, typename F>
__device__ __forceinline__ V over_block(V v, V* part, F&& join) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = join(v, __shfl_xor_sync(0xffffffffu, v, o));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int w = 1; w < kSideThreads / 32; ++w) v = join(v, part[w]);
  return v;
}
__device__ __forceinline__ float add_floats(float a, float b) { return a + b; }

// Tokens that count, span by span, where there are so many that a gathering CTA would not count them all itself.
constexpr int kCountSpan = 4096;
constexpr int kCountFrom = 16 * kCountSpan;
__global__ void __launch_bounds__(kSideThreads) loss_count_kernel(const int32_t* labels, int T, int V, int* counts) {
  wait_for_kernel_before();
  let_kernel_behind_in();
  __shared__ int part[kSideThreads / 32];
  const int first = blockIdx.x * kCountSpan, behind = min(T, first + kCountSpan);
  int n = 0;
  for (int i = first + (int)threadIdx.x; i < behind; i += kSideThreads) n += (unsigned)ld_global(labels + i) < (unsigned)V;
  n = over_block(n, part, [](int a, int b) { return a + b; });
  if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// ROWS tokens a CTA, 8 / ROWS warps a token: its place among those that count, its row beside theirs, and the logit of its label.
// A CTA counts the tokens before its own itself (16 KB of labels at 4096 tokens), or those of its span.  One token a CTA where there are few.
template <int ROWS>
__global__ void __launch_bounds__(kSideThreads) loss_gather_kernel(const GatherParams p) {
  wait_for_kernel_before();
  let_kernel_behind_in();
  constexpr int kSpan = kSideThreads / ROWS;         // threads of a token
  __shared__ int counts[8];
  __shared__ float dots[8];
  const int lane = threadIdx.x & 31, t0 = blockIdx.x * ROWS, mine = threadIdx.x / kSpan, at_thread = threadIdx.x % kSpan;
  const int32_t near = lane < ROWS && t0 + lane < p.T ? ld_global(p.labels + t0 + lane) : -1;
  const uint32_t alive = __ballot_sync(0xffffffffu, (unsigned)near < (unsigned)p.V);
  const int t = t0 + mine, label = __shfl_sync(0xffffffffu, near, mine);
  const bool live = alive >> mine & 1u;
  const size_t own = (size_t)t * p.K;
  int before = 0, from = 0;
  if (p.counts) {
    const int spans = t0 / kCountSpan;
    for (int i = threadIdx.x; i < spans; i += kSideThreads) before += ld_global(p.counts + i);
    from = spans * kCountSpan;
  }
  for (int i = from + (int)threadIdx.x; i < t0; i += kSideThreads) before += (unsigned)ld_global(p.labels + i) < (unsigned)p.V;
  before = over_block(before, counts, [](int a, int b) { return a + b; });
  if (blockIdx.x == 0)
    for (int c = threadIdx.x; c < p.chunks; c += kSideThreads) p.again[c] = 0;
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *p.live.count = before + __popc(alive);

  const int at = before + __popc(alive & ((1u << mine) - 1u));
  float dot = 0.0f;
  if (live) {
    dot = dot_share(p.X + own, p.W + (size_t)label * p.K, p.rows + (size_t)at * p.K, p.K, at_thread * 8, kSpan * 8);
  } else if (t < p.T) {
    if (at_thread == 0) {
      if (label >= p.V) note_bad_index(p.status);
      p.loss[t] = 0.0f;
    }
    if (p.dX)
      for (int c = at_thread * 8; c < p.K; c += kSpan * 8) *reinterpret_cast<uint4*>(p.dX + own + c) = make_uint4(0u, 0u, 0u, 0u);
  }
  if constexpr (ROWS == 1) {
    dot = over_block(dot, dots, add_floats);
  } else {
    dot = warp_sum(dot);
  }
  if (live && at_thread == 0) {
    p.live.index[at] = t;
    p.live.label[at] = label;
    p.live.ref[at] = dot;
    p.live.above[at] = 0;
  }
}

struct FinishParams {
  LiveTokens live;
  const float* sums;
  int parts;               // that the vocabulary's sums come in
  int row0, rows;
  const float* grads;      // [splits, rows, K]: rows of the blocks of 256 that count
  ShareRule rule;
  int splits, K;           // splits: of few tokens, whose sums are 256 rows each; 0: by the rule
  const __nv_bfloat16* W;
  const float* weight;     // or nullptr
  float* loss;
  __nv_bfloat16* dX;
};

// ROWS tokens a CTA: their sums over the vocabulary, added in one order whatever the timing, then 8 / ROWS warps a token.
template <bool GRAD, int ROWS>
__global__ void __launch_bounds__(kSideThreads) loss_finish_kernel(const FinishParams p) {
  wait_for_kernel_before();
  let_kernel_behind_in();
  constexpr int kSpan = kSideThreads / ROWS, kParts = kSideThreads / ROWS;
  __shared__ LogSum part[kParts][ROWS];
  const int row_b = blockIdx.x * ROWS, live = min(p.rows, ld_global(p.live.count) - p.row0);
  if (row_b >= live) return;
  // everything that the sums are not needed for is asked for before them
  const int mine = threadIdx.x / kSpan, at_thread = threadIdx.x % kSpan, lane = threadIdx.x & 31, row = min(row_b + mine, live - 1);
  const int token = ld_global(p.live.index + p.row0 + row), label = ld_global(p.live.label + p.row0 + row);
  const float of_label = ld_global(p.live.ref + p.row0 + row), above = GRAD ? above_of(p.live, p.row0 + row) : 0.0f;
  const float weight = GRAD && p.weight ? ld_global(p.weight + token) : 1.0f;
  const __nv_bfloat16* w = p.W + (size_t)label * p.K;
  const float* g = p.grads + (size_t)row * p.K;
  const Share share = GRAD && !p.splits ? share_of(p.rule, live) : Share{1, 0, p.splits};
  const size_t per_split = (size_t)share.blocks * kTile * p.K;
  struct Eight {
    float v[8];       // the first part's sums
    uint4 w;          // the label's row of the head
  };
  auto load = [&](int c) {
    Eight e = {};
    if (GRAD && c < p.K) {
      const float4 a = ld_global(reinterpret_cast<const float4*>(g + c)), b = ld_global(reinterpret_cast<const float4*>(g + c + 4));
      e = {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, ld_global(reinterpret_cast<const uint4*>(w + c))};
    }
    return e;
  };
  Eight now = load(at_thread * 8);
  {
    const int r = threadIdx.x % ROWS, first = threadIdx.x / ROWS;
    LogSum v = {-INFINITY, 0.0f};
#pragma unroll 4
    for (int h = first; h < p.parts; h += kParts) {
      const size_t at = (size_t)h * p.rows + row_b + r;
      if (GRAD) {
        v.sum += ld_global(p.sums + at);
      } else {
        const float2 u = ld_global(reinterpret_cast<const float2*>(p.sums) + at);
        v = join_sums(v, {u.x, u.y});
      }
    }
    part[first][r] = v;
  }
  __syncthreads();
  if (row_b + mine >= live) return;
  LogSum v = {-INFINITY, 0.0f};
#pragma unroll
  for (int h = 0; h < kParts; h += 32) {
    const LogSum u = part[h + lane][mine];
    if (GRAD) v.sum += u.sum;
    else v = join_sums(v, u);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const LogSum u = {__shfl_xor_sync(0xffffffffu, v.most, o), __shfl_xor_sync(0xffffffffu, v.sum, o)};
    if (GRAD) v.sum += u.sum;
    else v = join_sums(v, u);
  }
  const float sum = v.sum;
  if (!GRAD) {
    if (at_thread == 0) p.loss[token] = loss_of(v, of_label);
    return;
  }
  // above: the reference above the label's logit; own: the label's term, 1 if there is no such distance
  const float own = finite_label(of_label) ? expf(-above) : NAN;
  if (at_thread == 0) p.loss[token] = above == 0.0f ? log1pf(sum * own) : above + logf(sum + own);
  const float by = weight / (sum + own);
  __nv_bfloat16* out = p.dX + (size_t)token * p.K;
#pragma unroll 1
  for (int c = at_thread * 8; c < p.K; c += kSpan * 8) {
    const Eight next = load(c + kSpan * 8);
#pragma unroll 4
    for (int s = 1; s < share.splits; ++s) {
      const float4 a = ld_global(reinterpret_cast<const float4*>(g + s * per_split + c));
      const float4 b = ld_global(reinterpret_cast<const float4*>(g + s * per_split + c + 4));
      now.v[0] += a.x; now.v[1] += a.y; now.v[2] += a.z; now.v[3] += a.w;
      now.v[4] += b.x; now.v[5] += b.y; now.v[6] += b.z; now.v[7] += b.w;
    }
    const uint32_t y[4] = {now.w.x, now.w.y, now.w.z, now.w.w};
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      o[e] = bf16_pair(fmaf(-sum, __uint_as_float(y[e] << 16), now.v[2 * e]) * by,
                       fmaf(-sum, __uint_as_float(y[e] & 0xFFFF0000u), now.v[2 * e + 1]) * by);
    *reinterpret_cast<uint4*>(out + c) = make_uint4(o[0], o[1], o[2], o[3]);
    now = next;
  }
}

// ------------------------------------------------------------- host side

struct LossPlan {
  int rows;                  // live tokens of a chunk at most, a multiple of 256
  int chunks;
  int width, tiles, pieces, splits;      // width: entries of a tile
  int group, back_group;
  bool few;                  // head_loss_few.cu
  // offsets into the workspace
  size_t count, again, counts, index, label, ref, above, x, sums, e[2], grads, bytes;
  ShareRule rule(int K, int pairs) const {
    return {rows / kTile, pieces, (K + kTile - 1) / kTile, pairs, splits, tiles / pieces * width / kDepth};
  }
  int piece_tile(int i) const { return (int)((long long)tiles * i / pieces); }
  int piece_width() const { return ((tiles + pieces - 1) / pieces) * width; }     // entries of the widest
};

// Sizes and cuts, by the sizes of the call alone.
LossPlan plan_loss(int T, int V, int K, bool grad, int sms) {
  LossPlan c = {};
  const int pairs = sms / 2 > 0 ? sms / 2 : 1;
  // tokens of a chunk: their sums of the gradient are 256 MB at most (or 256 tokens')
  long long most = ((1ll << 26) / K) & ~255ll;
  most = most < 256 ? 256 : most > kChunkRows ? kChunkRows : most;
  const long long all = ((long long)T + 255) & ~255ll;
  c.rows = (int)(all < most ? all : most);
  c.chunks = (int)((all + c.rows - 1) / c.rows);
  const int blocks = c.rows / kTile;
  c.few = T <= kFewTokens;
  // 96 MB of exponentials a piece (4096 tokens at 32000 x 8192, us: 32 MB 3540, 64 3390, 96 3350, 128 3330; every piece's sums of the gradient go to memory
  // once more); few tokens' 128, since what their launches do is read the head, which one pass over it, logits, and another, gradient, do
  // best (four pieces of 32000 x 4096, whose second reads would be L2's: 150 tokens 133 -> 172)
  const long long wide = ((c.few ? 128ll : 96ll) << 20) / (2ll * c.rows);
  c.pieces = grad ? (int)((V + wide - 1) / wide) : 1;
  // Where all tiles of logits are one launch's, they are as wide as shares them out best: rounds of the pairs, each a tile's contraction,
  // which takes a time proportional to its width, and a sixteenth of a full one's for what does not.
  c.width = kTile;
  if (c.pieces == 1) {
    long long best = 0;
    for (int width = kTile; width >= 128; width -= 32) {
      const long long rounds = ((long long)blocks * ((V + width - 1) / width) + pairs - 1) / pairs, cost = rounds * (width + 16);
      if (best == 0 || cost < best) {
        best = cost;
        c.width = width;
      }
    }
  }
  c.tiles = (int)(((long long)V + c.width - 1) / c.width);
  if (c.pieces > c.tiles) c.pieces = c.tiles;
  c.splits = 1;
  // token blocks whose operands, 32 MB, share the L2 with a few tiles of the other side
  auto group_of = [](long long depth) {
    const int g = (int)((32ll << 20) / (512ll * depth));
    return g < 4 ? 4 : g;
  };
  c.group = group_of(K);
  c.back_group = group_of(c.piece_width());
  if (grad && c.few) {
    // rounds of the pairs, each the stages of a part and eight stages' time for what does not grow with them, one more for each part
    const long long features = (K + kTile - 1) / kTile, stages = (long long)c.piece_width() / kDepth;
    const int least = c.tiles / c.pieces * c.width / kDepth;
    long long best = 0;
    for (int splits = 1; splits <= 16 && splits <= least; ++splits) {
      const long long cost = (features * splits + pairs - 1) / pairs * (stages / splits + 8) + splits;
      if (best == 0 || cost < best) {
        best = cost;
        c.splits = splits;
      }
    }
  } else if (grad) {
    const int back = blocks * ((K + kTile - 1) / kTile);
    if (back < pairs) {
      c.splits = pairs / back;
      const int least = c.tiles / c.pieces * c.width / kDepth;
      if (c.splits > least) c.splits = least;
      if (c.splits > 16) c.splits = 16;
    }
  }
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at = (at + bytes + 255) & ~(size_t)255;
    return here;
  };
  const size_t rows_all = (size_t)c.chunks * c.rows;
  c.count = take(4);
  c.again = take((size_t)c.chunks * 4);
  c.counts = take(T > kCountFrom ? (size_t)(T + kCountSpan - 1) / kCountSpan * 4 : 0);
  c.index = take(rows_all * 4);
  c.label = take(rows_all * 4);
  c.ref = take(rows_all * 4);
  c.above = take(rows_all * 4);
  c.x = take(rows_all * K * 2);
  c.sums = take((size_t)c.tiles * (c.few ? kFewParts : 2) * c.rows * (grad ? 4 : 8));
  if (grad) {
    c.e[0] = take((size_t)c.rows * c.piece_width() * 2);
    c.e[1] = c.pieces > 1 ? take((size_t)c.rows * c.piece_width() * 2) : c.e[0];
    c.grads = take((size_t)c.splits * c.rows * K * 4);
  }
  c.bytes = at;
  return c;
}

template <bool GRAD>
int launch_loss(const LossMaps& maps, const LossParams& p, const LossLaunch& l, int pairs, cudaStream_t st) {
  auto kern = head_loss_kernel<GRAD>;
  static std::atomic<uint64_t> done{0};
  PEQA_TRY(allow_smem(kern, kLossSmem, done));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * pairs, 1, 1);
  cfg.blockDim = dim3(kLossThreads, 1, 1);
  cfg.dynamicSmemBytes = kLossSmem;
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
  PEQA_CUDA(cudaLaunchKernelEx(&cfg, kern, maps, p, l));
  return PEQA_OK;
}

}  // namespace

}  // namespace peqa

using namespace peqa;

static bool loss_shape_ok(int T, int V, int K) { return T > 0 && V > 0 && K > 0 && K % 8 == 0; }
// K and V so that no count below passes 31 bits
static bool loss_size_ok(int T, int V, int K) { return T <= (1 << 24) && V <= (1 << 24) && K <= (1 << 20); }

extern "C" size_t peqa_head_loss_workspace_bytes(int T, int V, int K, int need_grad) {
  if (!loss_shape_ok(T, V, K) || !loss_size_ok(T, V, K)) return 0;
  const int sms = sm_count_or(148);
  const LossPlan c = plan_loss(T, V, K, need_grad != 0, sms);
  // A shorter batch may want more: its exponentials are rounded to other pieces, its sums of the gradient come in parts where tiles are few, those of
  // the vocabulary in eighths of a tile up to 256 tokens.  So that one workspace serves them all: the most of any batch up to T, by blocks of 256 tokens within a chunk.
  size_t bytes = c.bytes;
  for (int t = kTile; t <= c.rows && t < T; t += kTile) {
    const size_t shorter = plan_loss(t, V, K, need_grad != 0, sms).bytes;
    bytes = shorter > bytes ? shorter : bytes;
  }
  return bytes;
}

extern "C" int peqa_head_loss(const void* X, const void* W, const int32_t* labels, const float* weight, int T, int V, int K,
                              float* loss, void* dX, void* workspace, size_t workspace_bytes, void* stream) {
  if (!X || !W || !labels || !loss) return PEQA_ERR_NULL;
  if (!loss_shape_ok(T, V, K)) return PEQA_ERR_BAD_SHAPE;
  if (!loss_size_ok(T, V, K)) return PEQA_ERR_TOO_LARGE;
  if (!aligned16(X) || !aligned16(W) || !aligned16(labels) || !aligned16(loss) || !aligned16(dX) || !aligned16(weight))
    return PEQA_ERR_ALIGNMENT;
  PEQA_TRY(check_arch());
  const int sms = sm_count_or(148), pairs = sms / 2;
  const LossPlan c = plan_loss(T, V, K, dX != nullptr, sms);
  if (!workspace || workspace_bytes < c.bytes) return PEQA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return PEQA_ERR_ALIGNMENT;
  cudaStream_t st = as_stream(stream);
  char* ws = static_cast<char*>(workspace);
  int* status = nullptr;
  PEQA_TRY(status_word(st, &status));

  LiveTokens live;
  live.count = reinterpret_cast<int*>(ws + c.count);
  live.index = reinterpret_cast<int*>(ws + c.index);
  live.label = reinterpret_cast<int*>(ws + c.label);
  live.ref = reinterpret_cast<float*>(ws + c.ref);
  live.above = reinterpret_cast<int*>(ws + c.above);

  LossParams p = {};
  p.live = live;
  p.sums = reinterpret_cast<float*>(ws + c.sums);
  p.rows = c.rows;
  p.V = V;
  p.K = K;
  p.k_blocks = (K + kDepth - 1) / kDepth;
  p.splits = c.splits;
  p.group = c.group;
  p.back_group = c.back_group;
  p.width = c.width;
  p.status = status;
  const uint64_t width = c.piece_width();
  LossMaps maps = {};
  FewCall few = {};
  if (c.few) {
    few.rows = dX ? ws + c.x : X;
    few.W = W;
    few.labels = labels;
    few.grads = reinterpret_cast<float*>(ws + c.grads);
    few.pitch = (int)width;
    few.tokens = T;
    for (int b = 0; b < 2; ++b) few.e[b] = ws + c.e[b];
    PEQA_TRY(few_maps(few, c.width, V, K, dX != nullptr));
    if (!dX) {
      p.tiles = c.tiles;
      PEQA_TRY(launch_few(p, few, 0, 0, false, pairs, st));
      return finish_few(p, few, kFewParts * c.tiles, loss, st);
    }
  } else {
    PEQA_TRY(bf16_map(&maps.x, ws + c.x, K, (uint64_t)c.chunks * c.rows, 128));
    PEQA_TRY(bf16_map(&maps.w, W, K, V, c.width / 2));
    if (dX) {
      PEQA_TRY(bf16_map(&maps.wt, W, K, V, 64));
      PEQA_TRY(loss_map(&maps.sum, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, ws + c.grads, K, (uint64_t)c.splits * c.rows, 4, 32, 32,
                        CU_TENSOR_MAP_SWIZZLE_128B));
    }
  }
  // [turn][fold]; several pieces' entries are whole stages, one's may not be: what its last stage has beyond it is read as zeros
  CUtensorMap e_out[2][kFolds] = {}, e_in[2][kFolds] = {};
  if (dX && !c.few)
    for (int b = 0; b < (c.pieces > 1 ? 2 : 1); ++b)
      for (int f = 0; f < kFolds && c.rows / kTile >> f > 0; ++f) {
        PEQA_TRY(loss_map(&e_out[b][f], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, ws + c.e[b], width << f, c.rows >> f, 2, 32, 32,
                          CU_TENSOR_MAP_SWIZZLE_64B));
        PEQA_TRY(bf16_map(&e_in[b][f], ws + c.e[b], width << f, c.rows >> f, 128));
      }

  GatherParams gp = {};
  gp.X = static_cast<const __nv_bfloat16*>(X);
  gp.W = static_cast<const __nv_bfloat16*>(W);
  gp.labels = labels;
  gp.T = T;
  gp.V = V;
  gp.K = K;
  gp.live = live;
  gp.rows = reinterpret_cast<__nv_bfloat16*>(ws + c.x);
  gp.again = reinterpret_cast<int*>(ws + c.again);
  gp.chunks = c.chunks;
  gp.loss = loss;
  gp.dX = static_cast<__nv_bfloat16*>(dX);
  gp.status = status;
  if (T > kCountFrom) {
    int* counts = reinterpret_cast<int*>(ws + c.counts);
    PEQA_TRY(launch_after(loss_count_kernel, (T + kCountSpan - 1) / kCountSpan, kSideThreads, st, labels, T, V, counts));
    gp.counts = counts;
  }
  // one token a CTA while that fills no more than two rounds of the SMs
  const bool alone = T <= 2 * 8 * sms;
  PEQA_TRY(alone ? launch_after(loss_gather_kernel<1>, T, kSideThreads, st, gp)
                 : launch_after(loss_gather_kernel<8>, (T + 7) / 8, kSideThreads, st, gp));

  FinishParams fp = {};
  fp.live = live;
  fp.sums = p.sums;
  fp.parts = (c.few ? kFewParts : 2) * c.tiles;
  fp.rows = c.rows;
  fp.grads = reinterpret_cast<const float*>(ws + c.grads);
  fp.splits = c.few ? c.splits : 0;
  const ShareRule rule = c.rule(K, pairs);
  fp.rule = rule;
  fp.K = K;
  fp.W = gp.W;
  fp.weight = weight;
  fp.loss = loss;
  fp.dX = gp.dX;
  for (int ch = 0; ch < c.chunks; ++ch) {
    p.row0 = fp.row0 = ch * c.rows;
    p.again = gp.again + ch;
    for (int turn = 0; turn < (dX ? 2 : 1); ++turn) {
      p.second = turn == 1;
      for (int i = 0; i <= (dX ? c.pieces : 0); ++i) {
        if (c.few) {
          p.tile0 = i < c.pieces ? c.piece_tile(i) : 0;
          p.tiles = i < c.pieces ? c.piece_tile(i + 1) - p.tile0 : 0;
          const int before = i > 0 ? c.piece_tile(i - 1) : 0, entries = i > 0 ? (c.piece_tile(i) - before) * c.width : 0;
          p.back0 = before * c.width;
          p.back_blocks = (entries + kDepth - 1) / kDepth;
          p.first_back = i == 1;
          PEQA_TRY(launch_few(p, few, i & 1, entries, dX != nullptr, pairs, st));
          continue;
        }
        const LossLaunch l = {rule, i, c.tiles, c.pieces};
        if (dX) {
          for (int f = 0; f < kFolds; ++f) {
            maps.e_out[f] = e_out[c.pieces > 1 ? i & 1 : 0][f];
            maps.e_in[f] = e_in[c.pieces > 1 ? (i & 1) ^ 1 : 0][f];
          }
          PEQA_TRY(launch_loss<true>(maps, p, l, pairs, st));
        } else {
          PEQA_TRY(launch_loss<false>(maps, p, l, pairs, st));
        }
      }
    }
    const int rows = c.rows < T ? c.rows : T;
    if (alone) PEQA_TRY(launch_after(dX ? loss_finish_kernel<true, 1> : loss_finish_kernel<false, 1>, rows, kSideThreads, st, fp));
    else PEQA_TRY(launch_after(dX ? loss_finish_kernel<true, 8> : loss_finish_kernel<false, 8>, (rows + 7) / 8, kSideThreads, st, fp));
  }
  return PEQA_OK;
}

// New keys and values into the paged cache, rotated by their positions, and the rotation of the queries beside them.
//
//   y[a] = x[a] c - x[b] s,   y[b] = x[b] c + x[a] s     (c, s) = cos_sin[position, i], (a, b) the i-th pair of channels
//
// Bound by memory: each row of a head is read once and written once.  head_dim / 16 adjacent lanes take a head of a token, 16 channels
// each, in two pieces of 16 bytes that hold whole pairs: channels 8 i and R/2 + 8 i on (pairs a half apart), or
// 16 i on (adjacent pairs, channels behind R, values).  What a row needs of its token, its place in the cache and its
// angles, is found while the rows themselves are on their way.
#include "common.cuh"
#include "kv_cache.cuh"
#include "sm100_ptx.cuh"

#include <cuda_bf16.h>

namespace peqa {

int check_kv_cache(const peqa_kv_cache_t* c, CacheView* view) {
  if (!c) return PEQA_ERR_NULL;
  if (c->type != PEQA_KV_BF16 && c->type != PEQA_KV_INT8) return PEQA_ERR_BAD_BITS;
  const bool codes = c->type == PEQA_KV_INT8;
  if (!c->k || !c->v || !c->page_table || (codes && (!c->k_scales || !c->v_scales))) return PEQA_ERR_NULL;
  if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->n_seqs < 1 || c->max_pages < 1) return PEQA_ERR_BAD_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return PEQA_ERR_BAD_SHAPE;
  if (!aligned16(c->k) || !aligned16(c->v)) return PEQA_ERR_ALIGNMENT;
  if (!aligned16(c->k_scales) || !aligned16(c->v_scales) || (reinterpret_cast<uintptr_t>(c->page_table) & 3u)) return PEQA_ERR_ALIGNMENT;
  if ((long long)c->max_pages * c->page_size > 0x7fffffffll) return PEQA_ERR_TOO_LARGE;
  // the three outer dimensions from the nearest to the furthest: each steps over all that lies within
  struct Dim {
    long long size, stride;
  } dims[3] = {{c->n_pages, c->page_stride}, {c->page_size, c->token_stride}, {c->n_kv_heads, c->head_stride}};
  const int bytes = codes ? 1 : 2, unit = 16 / bytes;
  for (int i = 0; i < 3; ++i) {
    if (dims[i].size == 1) dims[i].stride = 0;
    else if (dims[i].stride < 1) return PEQA_ERR_BAD_SHAPE;
    else if (dims[i].stride % unit != 0) return PEQA_ERR_ALIGNMENT;
    else if (dims[i].stride > (1ll << 36)) return PEQA_ERR_TOO_LARGE;
  }
  view->page16 = (uint32_t)(dims[0].stride / unit);
  view->token16 = (uint32_t)(dims[1].stride / unit);
  view->head16 = (uint32_t)(dims[2].stride / unit);
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (dims[j].stride > dims[j + 1].stride) {
        const Dim d = dims[j];
        dims[j] = dims[j + 1];
        dims[j + 1] = d;
      }
  long long extent = c->head_dim;
  for (int i = 0; i < 3; ++i) {
    if (dims[i].size == 1) continue;
    if (dims[i].stride < extent) return PEQA_ERR_BAD_SHAPE;
    if (dims[i].stride > (1ll << 36) / (dims[i].size - 1)) return PEQA_ERR_TOO_LARGE;
    extent += dims[i].stride * (dims[i].size - 1);
  }
  if (extent > (1ll << 36) / bytes) return PEQA_ERR_TOO_LARGE;
  view->k = c->k;
  view->v = c->v;
  view->k_scales = c->k_scales;
  view->v_scales = c->v_scales;
  view->table = c->page_table;
  view->by_page = make_divider((uint32_t)c->page_size);
  view->page_size = c->page_size;
  view->n_pages = c->n_pages;
  view->n_seqs = c->n_seqs;
  view->max_pages = c->max_pages;
  view->n_kv_heads = c->n_kv_heads;
  view->capacity = c->max_pages * c->page_size;
  return PEQA_OK;
}

int check_rows(const peqa_rows_t* r, int rows, int heads, int dim, bool written) {
  if (!r->data) return PEQA_ERR_NULL;
  if (!aligned16(r->data)) return PEQA_ERR_ALIGNMENT;
  const long long a = rows > 1 ? r->row_stride : 0, b = heads > 1 ? r->head_stride : 0;
  if (a < 0 || b < 0) return PEQA_ERR_BAD_SHAPE;
  if (a % 8 != 0 || b % 8 != 0) return PEQA_ERR_ALIGNMENT;
  if (a > (1ll << 30) || b > (1ll << 30)) return PEQA_ERR_TOO_LARGE;
  if (!written) return PEQA_OK;
  if (heads > 1 && b < dim) return PEQA_ERR_BAD_SHAPE;
  if (rows > 1 && a < dim) return PEQA_ERR_BAD_SHAPE;
  if (rows > 1 && heads > 1 && a < b * (heads - 1) + dim && b < a * (rows - 1) + dim) return PEQA_ERR_BAD_SHAPE;
  return PEQA_OK;
}

namespace {

constexpr int kThreads = 256;

struct Rows {
  uint16_t* data;
  long long row, head;
};

struct AppendParams {
  CacheView cache;
  Rows q, k, v, q_out;
  int n_heads, rotary;               // query heads (0: none); channels that turn
  bool interleaved;
  const float* cos_sin;
  int n_positions;
  const int32_t* seq_lens;
  const int32_t* starts;
  int* status;
};

// Eight channels of bf16.
__device__ __forceinline__ void widen(const uint4& u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 narrow(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float larger(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// One pair.  Each operation rounded by itself: the codes of an 8-bit cache are decided by these bits.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float y = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = y;
}

template <int D, bool I8>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const AppendParams p) {
  constexpr int kLanes = D / 16, kRows = kThreads / kLanes;    // of a head of a token; heads that a CTA takes at once
  constexpr int kAtOnce = 2;                                   // heads of a thread whose loads are in flight together
  __shared__ int s_seq;
  const int tid = threadIdx.x, i = tid % kLanes;
  const int t = blockIdx.x;
  const int kv_heads = p.cache.n_kv_heads, rows = p.n_heads + 2 * kv_heads;
  const bool turns = 16 * i < p.rotary;
  const bool apart = turns && !p.interleaved;
  const int d0 = apart ? 8 * i : 16 * i, d1 = apart ? p.rotary / 2 + 8 * i : 16 * i + 8;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  uint4 x0[kAtOnce], x1[kAtOnce];
  auto load = [&](int first) {
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) {
      const int r = first + e * gridDim.y * kRows;
      x0[e] = x1[e] = make_uint4(0, 0, 0, 0);
      if (r >= rows) continue;
      const bool is_q = r < p.n_heads, is_k = !is_q && r < p.n_heads + kv_heads;
      const Rows& from = is_q ? p.q : is_k ? p.k : p.v;
      const int h = is_q ? r : is_k ? r - p.n_heads : r - p.n_heads - kv_heads;
      const uint16_t* x = from.data + t * from.row + h * from.head;
      const bool value = !is_q && !is_k;                       // not turned: its 16 channels lie side by side
      x0[e] = ptx::ld_global(reinterpret_cast<const uint4*>(x + (value ? 16 * i : d0)));
      x1[e] = ptx::ld_global(reinterpret_cast<const uint4*>(x + (value ? 16 * i + 8 : d1)));
    }
  };
  int r0 = blockIdx.y * kRows + tid / kLanes;
  load(r0);

  // ---- the token's sequence and position
  int b = t, position;
  if (p.starts) {
    if (tid == 0) s_seq = -1;
    __syncthreads();
    for (int k = tid; k < p.cache.n_seqs; k += kThreads)
      if (ptx::ld_global(p.starts + k) <= t && t < ptx::ld_global(p.starts + k + 1)) s_seq = k;
    __syncthreads();
    b = s_seq;
    if (b < 0) return;
  }
  const int len = ptx::ld_global(p.seq_lens + b);
  if (len == 0) return;
  position = p.starts ? len - ptx::ld_global(p.starts + b + 1) + t : len - 1;
  if (len < 0 || len > p.cache.capacity || position < 0 || position >= p.n_positions) {
    if (tid == 0) note_bad_index(p.status);
    return;
  }
  const int entry = divide(position, p.cache.by_page);
  const int page = ptx::ld_global(p.cache.table + (long long)b * p.cache.max_pages + entry);
  const int place = position - entry * p.cache.page_size;
  const bool there = (uint32_t)page < (uint32_t)p.cache.n_pages;
  if (!there && tid == 0) note_bad_index(p.status);
  float c[8], s[8];
  if (turns) {
    const float* at = p.cos_sin + (long long)position * p.rotary + 8 * i;
    *reinterpret_cast<float4*>(c) = ptx::ld_global(reinterpret_cast<const float4*>(at));
    *reinterpret_cast<float4*>(c + 4) = ptx::ld_global(reinterpret_cast<const float4*>(at + 4));
    *reinterpret_cast<float4*>(s) = ptx::ld_global(reinterpret_cast<const float4*>(at + p.rotary / 2));
    *reinterpret_cast<float4*>(s + 4) = ptx::ld_global(reinterpret_cast<const float4*>(at + p.rotary / 2 + 4));
  }

  while (true) {
#pragma unroll
    for (int e = 0; e < kAtOnce; ++e) {
      const int r = r0 + e * gridDim.y * kRows;
      const bool is_q = r < p.n_heads, is_k = !is_q && r < p.n_heads + kv_heads;
      float a[8], z[8];
      widen(x0[e], a);
      widen(x1[e], z);
      if (turns && (is_q || is_k)) {
        if (p.interleaved) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            turn(a[2 * k], a[2 * k + 1], c[k], s[k]);
            turn(z[2 * k], z[2 * k + 1], c[4 + k], s[4 + k]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) turn(a[k], z[k], c[k], s[k]);
        }
      }
      const int e0 = is_q || is_k ? d0 : 16 * i, e1 = is_q || is_k ? d1 : 16 * i + 8;
      if constexpr (I8) {
        // the largest of the head, over the lanes that have it (all lanes of the warp take part)
        float most = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) most = larger(most, larger(fabsf(a[k]), fabsf(z[k])));
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) most = larger(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (r >= p.n_heads && r < rows && there) {
          const int h = is_k ? r - p.n_heads : r - p.n_heads - kv_heads;
          const float step = most == 0.f ? 1.f : __fdiv_rn(most, 127.f);
          uint32_t codes[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t word = 0;
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              const float y = k < 2 ? a[4 * k + m] : z[4 * (k - 2) + m];
              const int code = min(max(__float2int_rn(__fdiv_rn(y, step)), -127), 127);
              word |= (uint32_t)(code & 0xff) << (8 * m);
            }
            codes[k] = word;
          }
          int8_t* to = static_cast<int8_t*>(const_cast<void*>(is_k ? p.cache.k : p.cache.v)) +
                       ((uint64_t)page * p.cache.page16 + (uint64_t)place * p.cache.token16 + (uint64_t)h * p.cache.head16) * 16;
          *reinterpret_cast<uint2*>(to + e0) = make_uint2(codes[0], codes[1]);
          *reinterpret_cast<uint2*>(to + e1) = make_uint2(codes[2], codes[3]);
          if (i == 0)
            const_cast<float*>(is_k ? p.cache.k_scales : p.cache.v_scales)[((long long)page * kv_heads + h) * p.cache.page_size + place] = step;
        }
      }
      if (r < rows && (is_q || (!I8 && there))) {
        const int h = is_q ? r : is_k ? r - p.n_heads : r - p.n_heads - kv_heads;
        uint16_t* to = is_q ? p.q_out.data + t * p.q_out.row + h * p.q_out.head
                            : static_cast<uint16_t*>(const_cast<void*>(is_k ? p.cache.k : p.cache.v)) +
                                  ((uint64_t)page * p.cache.page16 + (uint64_t)place * p.cache.token16 + (uint64_t)h * p.cache.head16) * 8;
        *reinterpret_cast<uint4*>(to + e0) = narrow(a);
        *reinterpret_cast<uint4*>(to + e1) = narrow(z);
      }
    }
    // (the whole CTA goes on together)
    r0 += kAtOnce * gridDim.y * kRows;
    if (r0 - tid / kLanes >= rows) return;
    load(r0);
  }
}

template <int D, bool I8>
int launch(const AppendParams& p, int n_tokens, cudaStream_t st) {
  constexpr int kRows = kThreads / (D / 16);
  const int rows = p.n_heads + 2 * p.cache.n_kv_heads, passes = (rows + kRows - 1) / kRows;
  // a CTA for every so many heads where there are few tokens, for every token where there are many
  const int split = n_tokens * (long long)passes <= 4 * sm_count_or(148) ? passes : (passes + 1) / 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_tokens, min(split, 65535), 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  PEQA_CUDA(cudaLaunchKernelEx(&cfg, kv_append_kernel<D, I8>, p));
  return PEQA_OK;
}

template <bool I8>
int launch_dim(const AppendParams& p, int dim, int n_tokens, cudaStream_t st) {
  switch (dim) {
    case 64: return launch<64, I8>(p, n_tokens, st);
    case 128: return launch<128, I8>(p, n_tokens, st);
    default: return launch<256, I8>(p, n_tokens, st);
  }
}

Rows rows_of(const peqa_rows_t* r, int rows, int heads) {
  return Rows{static_cast<uint16_t*>(r->data), rows > 1 ? (long long)r->row_stride : 0, heads > 1 ? (long long)r->head_stride : 0};
}

}  // namespace
}  // namespace peqa

using namespace peqa;

extern "C" int peqa_kv_append(const peqa_kv_cache_t* c, const peqa_rows_t* q, int n_heads, const peqa_rows_t* k,
                              const peqa_rows_t* v, int n_tokens, const float* cos_sin, int n_positions, int rotary_dim,
                              int interleaved, const int32_t* seq_lens, const int32_t* starts, const peqa_rows_t* q_out,
                              void* stream) {
  AppendParams p = {};
  PEQA_TRY(check_kv_cache(c, &p.cache));
  if (!k || !v || !cos_sin || !seq_lens || (q == nullptr) != (q_out == nullptr)) return PEQA_ERR_NULL;
  if (n_tokens < 1 || n_positions < 1 || (!starts && n_tokens != c->n_seqs)) return PEQA_ERR_BAD_SHAPE;
  if (rotary_dim < 16 || rotary_dim % 16 != 0 || rotary_dim > c->head_dim) return PEQA_ERR_BAD_SHAPE;
  if (q && n_heads < 1) return PEQA_ERR_BAD_SHAPE;
  if (n_heads > (1 << 20) || c->n_kv_heads > (1 << 20)) return PEQA_ERR_TOO_LARGE;
  if (q) {
    PEQA_TRY(check_rows(q, n_tokens, n_heads, c->head_dim, false));
    PEQA_TRY(check_rows(q_out, n_tokens, n_heads, c->head_dim, true));
    p.q = rows_of(q, n_tokens, n_heads);
    p.q_out = rows_of(q_out, n_tokens, n_heads);
    p.n_heads = n_heads;
  }
  PEQA_TRY(check_rows(k, n_tokens, c->n_kv_heads, c->head_dim, false));
  PEQA_TRY(check_rows(v, n_tokens, c->n_kv_heads, c->head_dim, false));
  if (!aligned16(cos_sin)) return PEQA_ERR_ALIGNMENT;
  if ((reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(starts)) & 3u) return PEQA_ERR_ALIGNMENT;
  PEQA_TRY(check_arch());
  p.k = rows_of(k, n_tokens, c->n_kv_heads);
  p.v = rows_of(v, n_tokens, c->n_kv_heads);
  p.rotary = rotary_dim;
  p.interleaved = interleaved != 0;
  p.cos_sin = cos_sin;
  p.n_positions = n_positions;
  p.seq_lens = seq_lens;
  p.starts = starts;
  cudaStream_t st = as_stream(stream);
  PEQA_TRY(status_word(st, &p.status));
  return c->type == PEQA_KV_INT8 ? launch_dim<true>(p, c->head_dim, n_tokens, st) : launch_dim<false>(p, c->head_dim, n_tokens, st);
}

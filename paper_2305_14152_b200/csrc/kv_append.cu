// New keys and values into the paged cache, rotated by their positions, and the rotation of the queries beside them.
//
//   y[a] = x[a] c - x[b] s,   y[b] = x[b] c + x[a] s     (c, s) = cos_sin[position, i], (a, b) the i-th pair of channels
//
// Bound by memory: each row of a head is read once and written once.  head_dim / 16 adjacent lanes take a head of a token, 16 channels
// each, in two pieces of 16 bytes that hold whole pairs: channels 8 i and R/2 + 8 i on (pairs a half apart), or
// 16 i on (adjacent pairs, channels behind R, values).
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

constexpr int kThreads = 128;

struct Rows {
  uint16_t* data;
  uint32_t row, head;                // strides in elements
};

struct AppendParams {
  CacheView cache;
  Rows q, k, v, q_out;
  int n_tokens, n_heads, rotary;     // query heads (0: none); channels that turn
  int passes;                        // of kThreads over the heads of a token
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

// Codes of a lane's 16 channels, rint(y / step) of the IEEE quotient.  Values of half the largest are frequent among 16-bit numbers, and
// their quotient, 63.5, lies between two codes: it has to be the quotient to the last bit.  By Markstein's theorem (IBM J. Res. Dev. 34, 1990): with
// inv the reciprocal rounded to nearest and q one of the two numbers next to y / step, the remainder r = y - q step is exact, and q + r inv
// rounded once is the quotient rounded to nearest.  The product y inv is off by less than two units in the last place; once
// corrected in the same way by less than one, as the theorem wants it, twice it is the quotient.  (Exponents far from the ends of their range;
// quotients that are far below 1/2 may be off and round to 0 all the same.)
__device__ __forceinline__ void encode(const float (&a)[8], const float (&z)[8], float step, uint32_t (&codes)[4]) {
  constexpr float kMagic = 12582912.f;                         // 1.5 * 2^23: the sum's lowest bits are the rounded number
  if (step > 0x1p-100f && step < 0x1p100f) {
    const float inv = __frcp_rn(step);
    auto rounded = [&](float y) {
      float q = __fmul_rn(y, inv);
#pragma unroll
      for (int k = 0; k < 2; ++k) q = __fmaf_rn(__fmaf_rn(-q, step, y), inv, q);
      return __float_as_uint(__fadd_rn(q, kMagic));
    };
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float* y = k < 2 ? a + 4 * k : z + 4 * (k - 2);
      const uint32_t lo = __byte_perm(rounded(y[0]), rounded(y[1]), 0x0040), hi = __byte_perm(rounded(y[2]), rounded(y[3]), 0x0040);
      codes[k] = __byte_perm(lo, hi, 0x5410);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    codes[k] = 0;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const float q = __fdiv_rn(k < 2 ? a[4 * k + m] : z[4 * (k - 2) + m], step);
      codes[k] |= (uint32_t)(min(max(__float2int_rn(q), -127), 127) & 0xff) << (8 * m);
    }
  }
}

// An item is the heads of a token that a CTA takes at once: a pass over its rows (queries, keys, values) has several.
// A thread's head in a pass, for token t.
template <int D>
struct Head {
  static constexpr int kLanes = D / 16, kRows = kThreads / kLanes;   // of a head of a token; heads of an item
  bool there, is_q, is_k, turns, apart;
  uint32_t h, at0, at1;              // its 16 channels, in bytes: two pieces of whole pairs
  const char* from;
  uint64_t from_step;
  char *to_q, *to_cache;

  __device__ __forceinline__ Head(const AppendParams& p, int pass, int t) {
    const int r = pass * kRows + threadIdx.x / kLanes, i = threadIdx.x % kLanes, kv_heads = p.cache.n_kv_heads;
    there = r < p.n_heads + 2 * kv_heads, is_q = r < p.n_heads, is_k = !is_q && r < p.n_heads + kv_heads;
    h = is_q ? r : is_k ? r - p.n_heads : r - p.n_heads - kv_heads;
    const Rows rows = is_q ? p.q : is_k ? p.k : p.v;
    turns = (is_q || is_k) && 16 * i < p.rotary, apart = turns && !p.interleaved;
    at0 = apart ? 16 * i : 32 * i, at1 = apart ? p.rotary + 16 * i : 32 * i + 16;
    from = reinterpret_cast<const char*>(rows.data + (uint64_t)(uint32_t)t * rows.row + (uint64_t)h * rows.head);
    from_step = (uint64_t)rows.row * 2;
    to_q = reinterpret_cast<char*>(p.q_out.data + (uint64_t)(uint32_t)t * p.q_out.row + (uint64_t)h * p.q_out.head);
    to_cache = static_cast<char*>(const_cast<void*>(is_k ? p.cache.k : p.cache.v)) + (uint64_t)(h * p.cache.head16) * 16;
  }
  __device__ __forceinline__ void load(uint4& x0, uint4& x1) const {
    if (!there) return;
    x0 = ptx::ld_global(reinterpret_cast<const uint4*>(from + at0));
    x1 = ptx::ld_global(reinterpret_cast<const uint4*>(from + at1));
  }
};

// state of a token: 0 left out, 1 its place is in no page, 2 it has one: `unit` in the cache, in units of 16 bytes, and `scale` in the scales (fewer than
// 2^30: the codes have less than 2^36 bytes).  All lanes of a warp take part.
template <int D, bool I8>
__device__ __forceinline__ void put_row(const AppendParams& p, const Head<D>& head, uint4 x0, uint4 x1, const float* angles, int state, uint32_t unit,
                                        uint32_t scale) {
  constexpr int kLanes = Head<D>::kLanes;
  const int i = threadIdx.x % kLanes;
  float a[8], z[8];
  widen(x0, a);
  widen(x1, z);
  if (head.turns) {
    float c[8], s[8];
    const float4 *cos = reinterpret_cast<const float4*>(angles + 8 * i), *sin = reinterpret_cast<const float4*>(angles + p.rotary / 2 + 8 * i);
    *reinterpret_cast<float4*>(c) = cos[0], *reinterpret_cast<float4*>(c + 4) = cos[1];
    *reinterpret_cast<float4*>(s) = sin[0], *reinterpret_cast<float4*>(s + 4) = sin[1];
    if (head.apart) {
#pragma unroll
      for (int k = 0; k < 8; ++k) turn(a[k], z[k], c[k], s[k]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        turn(a[2 * k], a[2 * k + 1], c[k], s[k]);
        turn(z[2 * k], z[2 * k + 1], c[4 + k], s[4 + k]);
      }
    }
  }
  if (I8 && __any_sync(0xffffffffu, !head.is_q)) {
    // the largest of the head, over the lanes that have it
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = larger(most, larger(fabsf(a[k]), fabsf(z[k])));
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) most = larger(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (!head.is_q && head.there && state == 2) {
      const float step = most == 0.f ? 1.f : __fdiv_rn(most, 127.f);
      uint32_t codes[4];
      encode(a, z, step, codes);
      char* const to = head.to_cache + (uint64_t)unit * 16;
      *reinterpret_cast<uint2*>(to + head.at0 / 2) = make_uint2(codes[0], codes[1]);
      *reinterpret_cast<uint2*>(to + head.at1 / 2) = make_uint2(codes[2], codes[3]);
      if (i == 0) const_cast<float*>(head.is_k ? p.cache.k_scales : p.cache.v_scales)[scale + head.h * p.cache.page_size] = step;
    }
  }
  if (head.there && (head.is_q ? state > 0 : !I8 && state == 2)) {
    char* const to = head.is_q ? head.to_q : head.to_cache + (uint64_t)unit * 16;
    *reinterpret_cast<uint4*>(to + head.at0) = narrow(a);
    *reinterpret_cast<uint4*>(to + head.at1) = narrow(z);
  }
}

// The sequence of a row: the first that ends behind it, if it has begun there, else -1.  By a warp, 32 ends at a time ...
__device__ __forceinline__ int sequence_by_warp(const AppendParams& p, int t) {
  if (!p.starts) return t;
  int lo = 0, n = p.cache.n_seqs;            // among n sequences from lo on
  for (;;) {
    const int step = (n + 31) / 32;
    const uint32_t end = min(lo + ((threadIdx.x & 31) + 1) * step, (uint32_t)(lo + n));
    const int before = __popc(__ballot_sync(0xffffffffu, ptx::ld_global(p.starts + end) <= t)) * step;
    if (before >= n) return -1;
    lo += before, n = min(step, n - before);
    if (step == 1) break;
  }
  return ptx::ld_global(p.starts + lo) <= t && t < ptx::ld_global(p.starts + lo + 1) ? lo : -1;
}
// ... and by a thread, for many rows at once.
__device__ __forceinline__ int sequence_of(const AppendParams& p, int t) {
  if (!p.starts) return t;
  int lo = 0, hi = p.cache.n_seqs;
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (ptx::ld_global(p.starts + mid + 1) <= t) lo = mid + 1;
    else hi = mid;
  }
  return lo < p.cache.n_seqs && ptx::ld_global(p.starts + lo) <= t ? lo : -1;
}
// A token's position: -1 if it is left out.
__device__ __forceinline__ int position_of(const AppendParams& p, int t, int b) {
  const int len = b < 0 ? 0 : ptx::ld_global(p.seq_lens + b);
  if (len == 0) return -1;
  const int position = p.starts ? len - ptx::ld_global(p.starts + b + 1) + t : len - 1;
  if (len > 0 && len <= p.cache.capacity && position >= 0 && position < p.n_positions) return position;
  note_bad_index(p.status);
  return -1;
}
// Its state, its place in the cache and in the scales.
__device__ __forceinline__ int place_of(const AppendParams& p, int b, int position, uint32_t& unit, uint32_t& scale) {
  const uint32_t entry = divide(position, p.cache.by_page), place = position - entry * p.cache.page_size;
  const uint32_t page = (uint32_t)ptx::ld_global(p.cache.table + (long long)b * p.cache.max_pages + entry);
  unit = page * p.cache.page16 + place * p.cache.token16;
  scale = page * (uint32_t)p.cache.n_kv_heads * p.cache.page_size + place;
  if (page < (uint32_t)p.cache.n_pages) return 2;
  note_bad_index(p.status);
  return 1;
}

// A CTA for each item, which finds the token's place while its row is on its way.  (Of 128 threads: with 256, 512 tokens of 96 rows of 128
// 6.7 us, now 6.1.  A search of all `starts` for the row's sequence by the CTA's threads together: 4096 tokens of 80 rows in 1024 pieces 39.2 us, by
// warps 37.8, by each thread alone 44.1.)
template <int D, bool I8>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const AppendParams p) {
  const int t = blockIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Head<D> head(p, blockIdx.y, t);
  uint4 x0 = make_uint4(0, 0, 0, 0), x1 = x0;
  head.load(x0, x1);
  const int b = sequence_by_warp(p, t), position = position_of(p, t, b);
  if (position < 0) return;
  uint32_t unit, scale;
  const int state = place_of(p, b, position, unit, scale);
  put_row<D, I8>(p, head, x0, x1, p.cos_sin + (long long)position * p.rotary, state, unit, scale);
}

// Many items of an 8-bit cache, whose codes take more instructions than the copies leave time for: items are numbered through the
// tokens, then the passes, and the CTAs take equal runs.  So a thread has the same head of one token after another: where it reads and writes moves by
// a stride.  A CTA resolves the places of its next kBatch tokens together (4096 tokens of 80 rows: by eights 39.3 us, 16 36.6, 32 34.0) and copies
// their angles to shared memory; the row of the next token is asked for before the one at hand is used.
template <int D>
__global__ void __launch_bounds__(kThreads, 8) kv_append_runs_kernel(const AppendParams p) {
  constexpr int kBatch = D <= 64 ? 64 : D <= 128 ? 32 : 16;    // tokens whose places are resolved together
  __shared__ int s_position[kBatch], s_state[kBatch];
  __shared__ uint32_t s_unit[kBatch], s_scale[kBatch];
  __shared__ __align__(16) float s_angles[kBatch][D];
  const int tid = threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  const long long items = (long long)p.n_tokens * p.passes;
  const long long first = items * blockIdx.x / gridDim.x, end = items * (blockIdx.x + 1) / gridDim.x;
  int left = (int)(end - first), pass = (int)(first / p.n_tokens), t = (int)(first - (long long)pass * p.n_tokens);

  for (; left > 0; ++pass, t = 0) {
    Head<D> head(p, pass, t);
    uint4 x0 = make_uint4(0, 0, 0, 0), x1 = x0;
    head.load(x0, x1);
    for (int tokens = min(left, p.n_tokens - t); tokens > 0;) {
      // ---- the places of the next tokens
      const int n = min(kBatch, tokens);
      __syncthreads();                                         // those of the ones before have been read
      int b = -1, position = -1;
      if (tid < n) {
        b = sequence_of(p, t + tid);
        position = position_of(p, t + tid, b);
        s_position[tid] = max(position, 0);
      }
      __syncthreads();
      if (tid < n) s_state[tid] = position < 0 ? 0 : place_of(p, b, position, s_unit[tid], s_scale[tid]);
      for (int token = tid / Head<D>::kLanes; token < n; token += Head<D>::kRows)
        for (int e = tid % Head<D>::kLanes; e < p.rotary / 4; e += Head<D>::kLanes)
          reinterpret_cast<float4*>(s_angles[token])[e] =
              ptx::ld_global(reinterpret_cast<const float4*>(p.cos_sin + (long long)s_position[token] * p.rotary) + e);
      __syncthreads();

      for (int e = 0; e < n; ++e) {
        const uint4 y0 = x0, y1 = x1;
        head.from += head.from_step;
        if (--tokens > 0) head.load(x0, x1);
        put_row<D, true>(p, head, y0, y1, s_angles[e], s_state[e], s_unit[e], s_scale[e]);
        head.to_q += (uint64_t)p.q_out.row * 2;
      }
      t += n;
      left -= n;
    }
  }
}

template <int D, bool I8>
int launch(AppendParams& p, cudaStream_t st) {
  p.passes = (p.n_heads + 2 * p.cache.n_kv_heads + Head<D>::kRows - 1) / Head<D>::kRows;
  const long long items = (long long)p.n_tokens * p.passes, sms = sm_count_or(148);
  if (items > 0x7fffffffll) return PEQA_ERR_TOO_LARGE;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.n_tokens, p.passes, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  // A CTA for each item / runs of items, us.  8 bits: 700 tokens of 96 rows of 128 (4200 items) 9.7 / 11.4, 1400 (8400) 18.3 / 18.1, 2600 31.5 / 28.6; 1400 of
  // 80 rows 14.5 / 15.2, 1700 (8500) 16.9 / 16.7, 4000 35.3 / 31.9.  bf16: 4000 of 96 37.6 / 38.6, 4096 of 192 71.0 / 73.3, of 96 rows of 64 21.4 / 22.7.
  if constexpr (I8)
    if (items > 56 * sms) {
      cfg.gridDim = dim3((unsigned)min(items, 8 * sms), 1, 1);   // as many as can be at once
      PEQA_CUDA(cudaLaunchKernelEx(&cfg, kv_append_runs_kernel<D>, p));
      return PEQA_OK;
    }
  PEQA_CUDA(cudaLaunchKernelEx(&cfg, kv_append_kernel<D, I8>, p));
  return PEQA_OK;
}

template <bool I8>
int launch_dim(AppendParams& p, int dim, cudaStream_t st) {
  switch (dim) {
    case 64: return launch<64, I8>(p, st);
    case 128: return launch<128, I8>(p, st);
    default: return launch<256, I8>(p, st);
  }
}

Rows rows_of(const peqa_rows_t* r, int rows, int heads) {
  return Rows{static_cast<uint16_t*>(r->data), rows > 1 ? (uint32_t)r->row_stride : 0u, heads > 1 ? (uint32_t)r->head_stride : 0u};
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
  if ((q ? n_heads : 0) + 2ll * c->n_kv_heads > (1 << 18)) return PEQA_ERR_TOO_LARGE;
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
  p.n_tokens = n_tokens;
  p.rotary = rotary_dim;
  p.interleaved = interleaved != 0;
  p.cos_sin = cos_sin;
  p.n_positions = n_positions;
  p.seq_lens = seq_lens;
  p.starts = starts;
  cudaStream_t st = as_stream(stream);
  PEQA_TRY(status_word(st, &p.status));
  return c->type == PEQA_KV_INT8 ? launch_dim<true>(p, c->head_dim, st) : launch_dim<false>(p, c->head_dim, st);
}

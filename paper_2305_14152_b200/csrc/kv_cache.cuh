// The paged key-value cache as the kernels address it, and the host's checks of its descriptor.
//
// A token of a sequence lies in page page_table[seq][t / page_size] at place t % page_size.  k and v are two tensors of
// the same shape [n_pages, page_size, n_kv_heads, head_dim] and strides, in any order of the first three dimensions.
// An 8-bit cache (PEQA_KV_INT8) holds codes in [-127, 127] and one binary32 scale per token and head, [n_pages, n_kv_heads,
// page_size]; a value is scale * code.
#pragma once

#include "common.cuh"

namespace peqa {

// t / d for 0 <= t < 2^31 and 1 <= d < 2^31.  With s = ceil(log2 d) and mul = floor(2^32 (2^s - d) / d) + 1 (< 2^32, as
// 2^s < 2d), m = 2^32 + mul is 2^(32+s)/d rounded up: m = (2^(32+s) + e)/d with 0 < e <= d <= 2^s.  So m t / 2^(32+s) exceeds
// t/d by e t / (d 2^(32+s)) <= t / (2^32 d) < 1/(2d), too little to reach the next multiple of 1/d.  m t / 2^32 = umulhi(t, mul) + t
// up to a fraction that the shift drops, and stays below 2^32.
struct Divider {
  uint32_t mul, shift;
};
inline Divider make_divider(uint32_t d) {
  uint32_t s = 0;
  while ((1ull << s) < d) ++s;
  Divider r;
  r.mul = (uint32_t)(((1ull << 32) * ((1ull << s) - d)) / d + 1);
  r.shift = s;
  return r;
}

// Strides in units of 16 bytes: places in a cache of less than 64 GiB are 32-bit numbers of such units.
struct CacheView {
  const void* k;
  const void* v;
  const float* k_scales;
  const float* v_scales;
  const int32_t* table;
  uint32_t page16, token16, head16;
  Divider by_page;
  int page_size, n_pages, n_seqs, max_pages, n_kv_heads;
  int capacity;                  // tokens a sequence can have: max_pages * page_size
};

// Checks a descriptor and fills the view; nothing is read on the device.
int check_kv_cache(const peqa_kv_cache_t* c, CacheView* view);
// Rows of heads: 16-byte aligned, strides of 16 bytes; `written`: no two elements in one place.
int check_rows(const peqa_rows_t* r, int rows, int heads, int dim, bool written);

constexpr int kStatusIndexWord = 6;    // of a status slot (common.cuh)

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t divide(uint32_t t, const Divider& d) { return (__umulhi(t, d.mul) + t) >> d.shift; }

// A length, page number or position that does not fit is noted in the stream's status slot and nothing is accessed by it.
__device__ __forceinline__ void note_bad_index(int* status) { atomicExch(status + kStatusIndexWord, 1); }

// Tokens of a sequence, 0 for a length that is none.
__device__ __forceinline__ int checked_length(int len, int capacity, int* status) {
  if (len < 0 || len > capacity) {
    note_bad_index(status);
    return 0;
  }
  return len;
}
#endif

}  // namespace peqa

// Attention of one new token per sequence to its paged cache (Sec. 3.1: generation is bound by what it reads).
//
//   out[b,h] = sum_t p_t v_t,   p_t = exp(s_t - lse),   s_t = scale <q[b,h], k_t>,   lse = log sum_t exp(s_t)
//
// Every cached key and value is read once, by one warp, for all query heads that share it (a row of work: a sequence, a
// key-value head and up to NH = 8 or 16 of its query heads).  4 NH flops per cached element are too few to bind anything
// but memory, and the rest is laid out to keep copies in flight:
//   * A tile is 16 tokens of a row.  Tiles are numbered through all sequences, heads and lengths, and dealt evenly: every CTA
//     takes an equal run of them, every warp an equal run of its CTA's.  Nothing depends on how uneven the lengths are.
//   * A warp copies its own tiles into its own ring of shared memory (cp.async, several units of 16 keys or values ahead), whole
//     tokens at a time, and reads them as operands of the tensor cores' m16n8k16 product: the channels of the contraction and
//     the tokens of a tile are taken in whatever order makes one 16-byte load serve several products without bank conflicts.  So there
//     is no barrier between warps and no transposition in the loop.
//       S = Q K^T      Q [16 heads x 16 channels] in registers, K the other operand: a lane holds 4 adjacent channels of a token
//       O^T = V^T P^T  V^T [16 channels x 16 tokens]: a lane loads the same channels of four tokens and pairs them byte by byte (prmt);
//                      S leaves the first product laid out as the operand P^T of the second
//   * Running maximum and sum per row, as the softmax allows: the sums are rescaled only when the maximum has risen by more than
//     kSlack (a factor of 2^8 that the binary32 sums carry easily).
//   * p goes into the second product as the sum of two 16-bit numbers: with one, its rounding (2^-9 of p) would double the
//     error variance that the rounding of the output has.  v and q are 16-bit numbers already, and 8-bit codes are exact ones.
//   * A row that a warp has from its first tile to its last is written out.  Parts of rows are joined within the CTA in shared
//     memory, and what crosses CTAs by a second kernel, which stands ready when the first ends (launch_after).
#include "common.cuh"
#include "kv_cache.cuh"
#include "sm100_ptx.cuh"

#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace peqa {
namespace {

constexpr int kTile = 16;            // tokens
#ifndef MINT
#define MINT 4
#endif
constexpr float kSlack = 8.f;        // of the running maximum, in powers of two
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_huge_valf();

struct AttnParams {
  CacheView cache;
  const uint16_t* q;                 // bf16 [n_seqs, n_heads, D]
  long long q_row, q_head;
  const int32_t* seq_lens;
  int n_heads, group;                // query heads in all, and of one key-value head
  int chunks, rows_of_seq;           // of NH query heads per key-value head; n_kv_heads * chunks
  float scale_log2;
  int window;
  uint16_t* out;
  float* lse;
  int4* headers;                     // [2 * CTAs]: row, whether its last tile is in the part
  float* parts;                      // [2 * CTAs][Shape::kPart]
  float* first_parts;                // [CTAs][warps][Shape::kPart]
  int* status;
};

// Everything that follows from the channels D, the query heads NH of a row, the type of the cache and whether a tile lies in
// one page (WHOLE: the page size is a multiple of 16).
template <int D_, int NH_, bool I8_, bool WHOLE_>
struct Shape {
  static constexpr int D = D_, NH = NH_;
  static constexpr bool I8 = I8_, WHOLE = WHOLE_;
  static constexpr bool kHalves = NH == 4;                      // the two numbers that p is are columns of one product
  static constexpr int kCols = NH > 8 ? 2 : 1;                  // of eight heads (kHalves: of four, twice)
  static constexpr int kBytes = D * (I8 ? 1 : 2);               // of a token
  static constexpr int kKC = kBytes / 64;                       // 16-byte pieces per lane of a token's key, 4 lanes side by side
  static constexpr int kVB = kBytes >= 128 ? 16 : 8;            // bytes per lane of a token's value, 8 lanes side by side
  static constexpr int kVC = kBytes / (8 * kVB);
  static constexpr int kEV = kVB / (I8 ? 1 : 2);                // channels in them
  static constexpr int kPieces = kBytes / 16;                   // 16-byte pieces of a token
  static constexpr int kRows = 32 / kPieces;                    // tokens that a warp copies with one instruction
  static constexpr int kUnit = kTile * kBytes;                  // keys or values of a tile
  static constexpr int kWarps = D > 128 || NH > 8 ? 8 : 16;     // by the registers that a thread needs
  static constexpr int kFit = 192 * 1024 / (kWarps * (kUnit + (I8 ? 64 : 0)));
  static constexpr int kUnits = kFit >= 9 ? 9 : kFit >= 7 ? 7 : kFit >= 5 ? 5 : 3;   // odd: keys follow keys, values values
  static constexpr int kRing = kUnits * kUnit;
  static constexpr int kSmem = kWarps * (kRing + (I8 ? kUnits * 64 : 0));            // and the scales of a unit's 16 tokens
  static constexpr int kPart = NH * (D + 2);                    // floats of a part: sums, maxima, sums of p
  static_assert(kFit >= 3 && kRing >= kPart * 4 && kRing % 1024 == 0 && kPart % 4 == 0, "shared memory");
};

__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, std::integral_constant<int, 16>) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, uint32_t bytes, std::integral_constant<int, 16>) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, uint32_t bytes, std::integral_constant<int, 8>) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, uint32_t bytes, std::integral_constant<int, 4>) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}
__device__ __forceinline__ float lds_float(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
  return v;
}

template <bool F16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <bool F16>
__device__ __forceinline__ void mma0(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// 2^x, 0 below 2^-126
__device__ __forceinline__ float power_of_two(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Codes of 8 bits as binary16: with its sign bit turned a code c is the byte c + 128, and 0x6400 | byte is 1024 + 128 + c.
__device__ __forceinline__ uint32_t less_bias(uint32_t h) {
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&h), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// two bytes of x, the lower pair or the higher
__device__ __forceinline__ uint32_t low_codes(uint32_t x) { return less_bias(__byte_perm(x, 0x64646464u, 0x4140)); }
__device__ __forceinline__ uint32_t high_codes(uint32_t x) { return less_bias(__byte_perm(x, 0x64646464u, 0x4342)); }

// Two numbers rounded to 16 bits, and what that leaves of them; lower half: p0.
template <bool F16>
__device__ __forceinline__ uint32_t round16(float& p0, float& p1) {
  uint32_t w;
  if constexpr (F16) {
    const __half2 h = __floats2half2_rn(p0, p1);
    const float2 f = __half22float2(h);
    p0 -= f.x, p1 -= f.y;
    w = *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
    w = *reinterpret_cast<const uint32_t*>(&h);
    p0 -= __uint_as_float(w << 16), p1 -= __uint_as_float(w & 0xffff0000u);
  }
  return w;
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// The tokens of a sequence that are seen, and their tiles.
struct Span {
  int first, end;                    // tokens
  __device__ __forceinline__ int tiles() const { return end > first ? (end - 1) / kTile + 1 - first / kTile : 0; }
};
__device__ __forceinline__ Span span_of(const AttnParams& p, int b) {
  Span s;
  s.end = checked_length(ptx::ld_global(p.seq_lens + b), p.cache.capacity, p.status);
  s.first = p.window > 0 && s.end > p.window ? s.end - p.window : 0;
  return s;
}

// Where a warp is: the tile from token t0 on of row (b, r), of which `left` tiles are to come with this one.
struct Cursor {
  int b, r, t0, left;
  Span span;

  __device__ __forceinline__ int tile0() const { return span.first & ~(kTile - 1); }
  __device__ __forceinline__ void begin(const AttnParams& p, int seq, int tiles_before) {
    b = seq;
    span = span_of(p, b);
    const int tiles = span.tiles();
    r = tiles_before / tiles;
    const int tile = tiles_before - r * tiles;
    t0 = tile0() + tile * kTile;
    left = tiles - tile;
  }
  // true: at another row
  __device__ __forceinline__ bool next(const AttnParams& p) {
    t0 += kTile;
    if (--left > 0) return false;
    if (++r >= p.rows_of_seq) {
      r = 0;
      do {
        if (++b >= p.cache.n_seqs) {   // behind the last tile there is none
          span.first = span.end = 0;
          left = 0x7fffffff;
          return true;
        }
        span = span_of(p, b);
      } while (span.end <= span.first);
    }
    t0 = tile0();
    left = span.tiles();
    return true;
  }
};

// Sums of a row, or of a part of one, in a part's memory: O [NH][D], then the maxima and the sums of p.  Within a CTA four channels of
// a head lie in the place of others of their eight times four, so that the lanes of a warp write to different banks.
template <typename S, bool MIXED>
struct Part {
  float* at;
  __device__ __forceinline__ float4& sums(int head, int d4) const {
    const int lc = (head >> 1) & 3, mix = S::kEV == 16 ? lc : (lc & 1) + 4 * (lc >> 1);
    return reinterpret_cast<float4*>(at + head * S::D)[MIXED ? d4 ^ mix : d4];
  }
  __device__ __forceinline__ float& most(int head) const { return at[S::NH * S::D + head]; }
  __device__ __forceinline__ float& total(int head) const { return at[S::NH * (S::D + 1) + head]; }
};

__device__ __forceinline__ float weight(float m, float most) { return m == kNegInf ? 0.f : exp2f(m - most); }

// First query head of a row, and how many there are.
template <typename S>
__device__ __forceinline__ int first_head(const AttnParams& p, int r, int& heads) {
  const int kv = r / p.chunks, chunk = r - kv * p.chunks;
  heads = min(S::NH, p.group - chunk * S::NH);
  return kv * p.group + chunk * S::NH;
}

template <typename S>
__global__ void __launch_bounds__(S::kWarps * 32, 1) attn_decode_kernel(const AttnParams p) {
  constexpr int D = S::D, NH = S::NH, kCols = S::kCols, kThreads = S::kWarps * 32;
  constexpr bool I8 = S::I8;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ int s_scan[kThreads];
  __shared__ int s_warp[S::kWarps];
  __shared__ int4 s_head[2 * S::kWarps];   // of a warp's parts: row (-1: none), begins its row, ends it

  const int tid = threadIdx.x, lane = tid & 31, warp = ptx::warp_index();
  const int lr = lane >> 2, lc = lane & 3;
  const uint32_t ring = ptx::smem_u32(smem) + warp * S::kRing;
  // a warp's parts of rows: one that it goes on from lies in the workspace, its last in its ring
  const auto first_part = [&](int w) { return Part<S, true>{p.first_parts + ((long long)blockIdx.x * S::kWarps + w) * S::kPart}; };
  const auto last_part = [&](int w) { return Part<S, true>{reinterpret_cast<float*>(smem + w * S::kRing)}; };

  if (tid < 2 * S::kWarps) s_head[tid] = make_int4(-1, 0, 0, 0);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // ---- the tiles of all sequences, and this warp's share of them: [begin, end)
  const int B = p.cache.n_seqs;
  int total = 0, begin = 0, end = 0;
  auto share = [&]() {
    // no CTA without a tile for a warp of each scheduler, while there are enough
    const int busy = min((int)gridDim.x, max(1, total / MINT)), cta = blockIdx.x;
    if (cta >= busy) return;
    const int each = total / busy, more = total - each * busy;             // the first `more` CTAs have one more
    const int first = each * cta + min(cta, more), n = each + (cta < more);
    const int each_warp = n / S::kWarps, more_warp = n - each_warp * S::kWarps;
    begin = first + each_warp * warp + min(warp, more_warp);
    end = begin + each_warp + (warp < more_warp);
  };
  auto tiles_of = [&](int b) { return b < B ? span_of(p, b).tiles() * p.rows_of_seq : 0; };
  if (B > kThreads) {
    for (int b = tid; b < B; b += kThreads) total += tiles_of(b);
    total = __reduce_add_sync(0xffffffffu, total);
    if (lane == 0) s_warp[warp] = total;
    __syncthreads();
    total = __reduce_add_sync(0xffffffffu, lane < S::kWarps ? s_warp[lane] : 0);
    share();
  }
  Cursor in;                                // of the copies; the sums follow with `at`
  in.b = in.r = in.t0 = in.left = in.span.first = in.span.end = 0;
  int before = 0;                           // tiles of the sequences before this round's
  if (B <= 32) {                            // every warp for itself
    int upto = tiles_of(lane);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += up;
    }
    total = __shfl_sync(0xffffffffu, upto, 31);
    share();
    if (begin < end) {
      const int b = __popc(__ballot_sync(0xffffffffu, upto <= begin));
      in.begin(p, b, begin - (b > 0 ? __shfl_sync(0xffffffffu, upto, b - 1) : 0));
    }
  } else for (int base = 0; base < B; base += kThreads) {
    int sum = tiles_of(base + tid);         // of the sequences up to this one, within the warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    __syncthreads();                        // s_scan and s_warp of the round before have been read
    s_scan[tid] = sum;
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    int upto = lane < S::kWarps ? s_warp[lane] : 0;     // of the warps up to warp `lane`
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += up;
    }
    const int round = __shfl_sync(0xffffffffu, upto, 31);
    if (B <= kThreads) {
      total = round;
      share();
    }
    int left = begin - before;              // tiles before this warp's first in its sequence, once the ones before are taken off
    if (begin < end && left >= 0 && left < round) {
      const int w = __popc(__ballot_sync(0xffffffffu, upto <= left));      // warps whose sequences end before it
      if (w > 0) left -= __shfl_sync(0xffffffffu, upto, w - 1);
      const int in_warp = s_scan[w * 32 + lane], l = __popc(__ballot_sync(0xffffffffu, in_warp <= left));
      if (l > 0) left -= __shfl_sync(0xffffffffu, in_warp, l - 1);
      in.begin(p, base + w * 32 + l, left);
    }
    before += round;
  }

  if (begin < end) {
    Cursor at = in;
    const int count = end - begin;

    // ---- copies.  Units of keys and of values follow one another through the ring, kUnits - 1 of them under way.
    int page = 0, issued = 0;
    uint32_t put = ring, get = ring;         // next unit to fill, and to read
    const uint32_t scales_of = ptx::smem_u32(smem) + S::kWarps * S::kRing + warp * S::kUnits * 64;
    uint32_t put_scales = scales_of, get_scales = scales_of;
    // Piece c of token t lies in place c ^ (t & 7): the eight lanes that a load serves at a time read eight different places of 128 bytes,
    // of two tokens four apart (keys) or of two times four tokens (values).  (64-byte tokens lie as they come.)
    auto place_of = [](int t, int c) { return (uint32_t)(t * S::kPieces + (S::kPieces >= 8 ? c ^ (t & 7) : c)) * 16; };
    const int copy_row = lane / S::kPieces, copy_piece = lane % S::kPieces;
    const uint32_t copy_to = place_of(copy_row, copy_piece);
    const int key_token = (lr >> 1) + 4 * (lr & 1);         // of column lr of the first product, and 8 more
    const uint32_t key_at = place_of(key_token, lc), key_at2 = key_at ^ 64;
    const uint32_t value_at = S::kVB == 16 ? place_of(lc + 4 * (lr & 1), lr) : place_of(lc + 4 * (lr & 1), 0) + lr * 8;
    const uint32_t value_at2 = S::kVB == 16 ? place_of(lc + 4 * (1 - (lr & 1)), lr) : place_of(lc + 4 * (1 - (lr & 1)), 0) + lr * 8;
    const uint32_t pick_low = I8 ? (lr & 1 ? 0x1504u : 0x5140u) : (lr & 1 ? 0x1054u : 0x5410u);
    const uint32_t pick_high = I8 ? (lr & 1 ? 0x3726u : 0x7362u) : (lr & 1 ? 0x3276u : 0x7632u);
    uint32_t unit = 0;                       // place of the copies' tile (WHOLE) or of its token (lane & 15)
    uint32_t scale = 0;                      // the same in the scales (fewer than 2^30: each has 64 bytes of codes, and they have less than 2^36)
    int kv = in.r / p.chunks;                // head of keys and values
    // Page of the copies' tile or of its token (lane & 15), asked for a tile ahead of its use.
    auto look_up = [&](bool there) {
      const int t = in.t0 + (S::WHOLE ? 0 : lane & 15);
      page = 0;
      if (there && (S::WHOLE || (t >= in.span.first && t < in.span.end)))
        page = ptx::ld_global(p.cache.table + (long long)in.b * p.cache.max_pages + divide(t, p.cache.by_page));
    };
    auto in_span = [&](int t) { return t >= in.span.first && t < in.span.end; };
    // A warp copies whole tokens, 512 bytes an instruction: in pieces of 64 bytes, as the products take keys, the same copies reach 4.9
    // TB/s of 6.6 (blocks of 4 KB in no order).
    auto copy_tokens = [&](const void* from, bool all) {
      const char* const base = static_cast<const char*>(from) + copy_piece * 16;
      const char* src = base + (uint64_t)(unit + copy_row * p.cache.token16) * 16;
      const uint64_t step = (uint64_t)p.cache.token16 * (S::kRows * 16);
#pragma unroll
      for (int j = 0; j < kTile / S::kRows; ++j) {
        if constexpr (!S::WHOLE) src = base + (uint64_t)__shfl_sync(0xffffffffu, unit, copy_row + j * S::kRows) * 16;
        const uint32_t to = ((put + copy_to) ^ (S::kPieces >= 8 ? ((j * S::kRows) & 7) * 16 : 0)) + j * 512;
        if (all) cp_async(to, src, std::integral_constant<int, 16>());
        else cp_async(to, src, in_span(in.t0 + copy_row + j * S::kRows) ? 16 : 0, std::integral_constant<int, 16>());
        if constexpr (S::WHOLE) src += step;
      }
    };
    auto copy_scales = [&](const float* scales) {
      if constexpr (I8)
        if (lane < 16) cp_async(put_scales + lane * 4, scales + scale, in_span(in.t0 + lane) ? 4 : 0, std::integral_constant<int, 4>());
    };
    auto copy_keys = [&]() {
      const int t = in.t0 + (S::WHOLE ? 0 : lane & 15);
      const uint32_t place = t - divide(t, p.cache.by_page) * p.cache.page_size;
      if ((uint32_t)page >= (uint32_t)p.cache.n_pages) {
        note_bad_index(p.status);
        page = 0;
      }
      unit = page * p.cache.page16 + place * p.cache.token16 + kv * p.cache.head16;
      if constexpr (I8) scale = (page * p.cache.n_kv_heads + kv) * p.cache.page_size + place + (S::WHOLE ? lane & 15 : 0);
      copy_tokens(p.cache.k, S::WHOLE);   // keys behind a sequence's end have no score, whatever they are, but may be in no page
    };
    auto copy_values = [&]() {
      // 0 for what is not seen: its p is 0, and must stay so
      copy_tokens(p.cache.v, in.t0 >= in.span.first && in.span.end - in.t0 >= kTile);
    };
    auto filled = [&]() {
      asm volatile("cp.async.commit_group;" ::: "memory");
      put += S::kUnit, put_scales += 64;
      if (put == ring + S::kRing) put = ring, put_scales = scales_of;
    };
    auto issue_keys = [&]() {
      if (issued < count) {
        copy_keys();
        copy_scales(p.cache.k_scales);
      }
      filled();
    };
    auto issue_values = [&]() {
      if (issued < count) {
        copy_values();
        copy_scales(p.cache.v_scales);
        if (in.next(p)) kv = in.r / p.chunks;
        look_up(issued + 1 < count);
      }
      ++issued;
      filled();
    };
    auto landed = [&]() { asm volatile("cp.async.wait_group %0;" ::"n"(S::kUnits - 2) : "memory"); };
    auto read = [&]() {
      get += S::kUnit, get_scales += 64;
      if (get == ring + S::kRing) get = ring, get_scales = scales_of;
    };
    look_up(true);
#pragma unroll 1
    for (int i = 0; i < S::kUnits / 2; ++i) {
      issue_keys();
      issue_values();
    }

    uint32_t q[kCols][D / 16][2];                            // heads lr (+ 8): words of adjacent channels
    float to_log2[2] = {p.scale_log2, p.scale_log2};         // of a product of the tensor cores, per head
    float most[2], sum[2];                                   // of heads lr (+ 8); sum: of this lane's tokens
    float acc[D / 16][kCols][4];                             // rows: channels, columns: heads 2 lc, 2 lc + 1 (+ 8)
    float v_ref = 1.f, inv_ref = 1.f;                        // I8: acc is in units of it
    float q_bias[2] = {0.f, 0.f};                            // I8: what the sums of products have too much
    bool from_start;

    auto begin_row = [&]() {
      int heads;
      const int h0 = first_head<S>(p, at.r, heads);
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        const int h = (S::kHalves ? lr & 3 : lr) + 8 * n;
        const uint16_t* from = p.q + at.b * p.q_row + (long long)(h0 + h) * p.q_head;
        constexpr int kAdjacent = I8 ? 16 : 8;               // channels of a 16-byte piece of a key
#pragma unroll
        for (int j = 0; j < S::kKC; ++j)
#pragma unroll
          for (int e = 0; e < kAdjacent / 8; ++e) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (h < heads) x = ptx::ld_global(reinterpret_cast<const uint4*>(from + (j * 4 + lc) * kAdjacent + e * 8));
            const int s = (j * kAdjacent + e * 8) / 4;
            q[n][s][0] = x.x, q[n][s][1] = x.y, q[n][s + 1][0] = x.z, q[n][s + 1][1] = x.w;
          }
        if constexpr (I8) {
          // bf16 as binary16: times a power of two that brings the head's largest below 4.  What becomes subnormal there is
          // 2^-14 of the largest or less, and off by 2^-25 of it at most.
          float big = 0.f;
#pragma unroll
          for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&q[n][s][e]));
              big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
          big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
          big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
          const int e = min(max((int)(__float_as_uint(big) >> 23) - 127, -126), 126);
          const float down = __uint_as_float((uint32_t)(127 - e) << 23);
          // Codes come as c + 128 in the lowest bits of a binary16, (c + 128) 2^-24: 128 2^-24 times the sum of q is taken off each sum.
          // (The bias is about three times as large as the sums themselves, so their last bits weigh as much more.)
          to_log2[n] = p.scale_log2 * __uint_as_float((uint32_t)(127 + e) << 23) * 16777216.f;
          q_bias[n] = 0.f;
#pragma unroll
          for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&q[n][s][w]));
              const __half2 x = __floats2half2_rn(f.x * down, f.y * down);
              q[n][s][w] = *reinterpret_cast<const uint32_t*>(&x);
              const float2 g = __half22float2(x);
              q_bias[n] += g.x + g.y;
            }
          q_bias[n] += __shfl_xor_sync(0xffffffffu, q_bias[n], 1);
          q_bias[n] += __shfl_xor_sync(0xffffffffu, q_bias[n], 2);
          q_bias[n] *= 0x1p-17f;
        }
        most[n] = kNegInf;
        sum[n] = 0.f;
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int n = 0; n < kCols; ++n) acc[d][n][0] = acc[d][n][1] = acc[d][n][2] = acc[d][n][3] = 0.f;
      if constexpr (I8) v_ref = 0.f;
      from_start = at.t0 == at.tile0();
    };

    // acc times a factor per head; lanes have those of heads lr (+ 8)
    auto rescale = [&](const float (&f)[2]) {
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        const float f0 = __shfl_sync(0xffffffffu, f[n], lc * 8), f1 = __shfl_sync(0xffffffffu, f[n], lc * 8 + 4);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          acc[d][n][0] *= f0, acc[d][n][1] *= f1, acc[d][n][2] *= f0, acc[d][n][3] *= f1;
        }
      }
    };

    auto add_tile = [&]() {
      const int t0 = at.t0;
      landed();
      __syncwarp();                          // for all lanes, and all have read what is filled next
      issue_keys();
      // ---- S = Q K^T, tokens 0..7 and 8..15; two sums each, so that a product waits for the one before the last
      float s[2][2][4];
#pragma unroll
      for (int j = 0; j < S::kKC; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 x = lds16(get + (j & 1 ? key_at2 : key_at) + i * 8 * S::kBytes + (j >> 1) * 128);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
          constexpr int kSteps = I8 ? 4 : 2;
#pragma unroll
          for (int e = 0; e < kSteps; ++e) {
            const int k = kSteps * j + e;
            uint32_t b0, b1;
            if constexpr (I8) {
              const uint32_t u = w[e] ^ 0x80808080u;
              b0 = __byte_perm(u, 0u, 0x4140), b1 = __byte_perm(u, 0u, 0x4342);
            } else {
              b0 = w[2 * e], b1 = w[2 * e + 1];
            }
            const uint32_t a1 = kCols > 1 ? q[kCols - 1][k][0] : 0u, a3 = kCols > 1 ? q[kCols - 1][k][1] : 0u;
            if (k < 2) mma0<I8>(s[i][e & 1], q[0][k][0], a1, q[0][k][1], a3, b0, b1);
            else mma<I8>(s[i][e & 1], q[0][k][0], a1, q[0][k][1], a3, b0, b1);
          }
        }
      // ---- scores in powers of two: x[n][i] of heads lr + 8 n and tokens lc + 4 {0, 1} + 8 {0, 1}
      float x[kCols][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float k_scale = 1.f;
        if constexpr (I8) k_scale = lds_float(get_scales + (lc + 4 * i) * 4);
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
          float y = s[i >> 1][0][2 * n + (i & 1)] + s[i >> 1][1][2 * n + (i & 1)];
          if constexpr (I8) y = (y - q_bias[n]) * k_scale;
          x[n][i] = y * to_log2[n];
        }
      }
      if (t0 < at.span.first || at.span.end - t0 < kTile) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + lc + 4 * i < at.span.first || t0 + lc + 4 * i >= at.span.end)
#pragma unroll
            for (int n = 0; n < kCols; ++n) x[n][i] = kNegInf;
      }
      // ---- running maximum
      float top[kCols];
      bool higher = false;
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        top[n] = fmaxf(fmaxf(x[n][0], x[n][1]), fmaxf(x[n][2], x[n][3]));
        top[n] = fmaxf(top[n], __shfl_xor_sync(0xffffffffu, top[n], 1));
        top[n] = fmaxf(top[n], __shfl_xor_sync(0xffffffffu, top[n], 2));
        higher |= top[n] > most[n] + kSlack;
      }
      if (__any_sync(0xffffffffu, higher)) {
        float f[2] = {1.f, 1.f};
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
          const float next = fmaxf(most[n], top[n]);
          f[n] = weight(most[n], next);
          sum[n] *= f[n];
          most[n] = next;
        }
        rescale(f);
      }
      // ---- p and its sum
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        const float base = most[n] == kNegInf ? 0.f : most[n];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[n][i] = power_of_two(x[n][i] - base);
          sum[n] += x[n][i];
        }
      }
      read();
      // ---- O^T += V^T P^T
      landed();
      __syncwarp();
      issue_values();
      if constexpr (I8) {
        float v_scale[4], big = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v_scale[i] = lds_float(get_scales + (lc + 4 * i) * 4);
          big = fmaxf(big, fabsf(v_scale[i]));
        }
        // Values in units of 2^-6 of the largest scale so far, cut to a power of two: p (at most 2^kSlack) times what is left of its
        // token's scale (below 2^7) is a binary16, and as two of them off by 2^-25 of a unit at most, 2^-31 of the largest.
        const uint32_t exponent = __reduce_max_sync(0xffffffffu, __float_as_uint(big)) & 0x7f800000u;
        const float ref = __uint_as_float(exponent > (7u << 23) ? exponent - (6u << 23) : 1u << 23);
        if (ref > v_ref) {
          if (v_ref > 0.f) {
            const float both[2] = {v_ref / ref, v_ref / ref};
            rescale(both);
          }
          v_ref = ref;
          inv_ref = 1.f / ref;
        }
#pragma unroll
        for (int n = 0; n < kCols; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[n][i] *= v_scale[i] * inv_ref;
      }
      uint32_t hi[kCols][2], lo[kCols][2];
#pragma unroll
      for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          hi[n][i] = round16<I8>(x[n][2 * i], x[n][2 * i + 1]);
          lo[n][i] = round16<I8>(x[n][2 * i], x[n][2 * i + 1]);
          if (S::kHalves && lr >= 4) hi[n][i] = lo[n][i];
        }
#pragma unroll
      for (int j = 0; j < S::kVC; ++j) {
        constexpr int kWords = S::kVB / 4;
        uint32_t w[4][kWords];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t from = get + (i & 1 ? value_at2 : value_at) + (i >> 1) * 8 * S::kBytes + j * 128;
          if constexpr (S::kVB == 16) {
            const uint4 v = lds16(from);
            w[i][0] = v.x, w[i][1] = v.y, w[i][kWords - 2] = v.z, w[i][kWords - 1] = v.w;
          } else {
            const uint2 v = lds8(from);
            w[i][0] = v.x, w[i][1] = v.y;
          }
        }
        auto product = [&](int d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
          for (int n = 0; n < kCols; ++n) {
            mma<I8>(acc[d][n], a0, a1, a2, a3, hi[n][0], hi[n][1]);
            if constexpr (!S::kHalves) mma<I8>(acc[d][n], a0, a1, a2, a3, lo[n][0], lo[n][1]);
          }
        };
#pragma unroll
        for (int e = 0; e < kWords; ++e) {
          if constexpr (I8) {
            // bytes of two tokens side by side: channels 0, 0, 1, 1 and 2, 2, 3, 3 of the word
            const uint32_t a = __byte_perm(w[0][e], w[1][e], pick_low) ^ 0x80808080u, b = __byte_perm(w[2][e], w[3][e], pick_low) ^ 0x80808080u;
            const uint32_t c = __byte_perm(w[0][e], w[1][e], pick_high) ^ 0x80808080u, f = __byte_perm(w[2][e], w[3][e], pick_high) ^ 0x80808080u;
            product(2 * (j * kWords + e), low_codes(a), high_codes(a), low_codes(b), high_codes(b));
            product(2 * (j * kWords + e) + 1, low_codes(c), high_codes(c), low_codes(f), high_codes(f));
          } else {
            product(j * kWords + e, __byte_perm(w[0][e], w[1][e], pick_low), __byte_perm(w[0][e], w[1][e], pick_high),
                    __byte_perm(w[2][e], w[3][e], pick_low), __byte_perm(w[2][e], w[3][e], pick_high));
          }
        }
      }
      read();
    };

    // The row's sums, or what this warp has of them, are complete.  acc[d] holds channels base + 2 e and base + 2 e + 1 in its
    // rows lr and lr + 8, where d = j * kEV / 2 + e and base = (j * 8 + lr) * kEV.
    auto end_row = [&](bool to_end, bool more) {
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 1);
        sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 2);
      }
      if constexpr (S::kHalves) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[d][0][i] += __shfl_xor_sync(0xffffffffu, acc[d][0][i], 2);
      }
      int heads;
      const int h0 = first_head<S>(p, at.r, heads);
      if (from_start && to_end) {
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
          const float inv = 1.f / sum[n];
          const long long out0 = (long long)at.b * p.n_heads + h0 + 8 * n;
          if (p.lse && lc == 0 && lr + 8 * n < heads) p.lse[out0 + lr] = kLn2 * (most[n] + log2f(sum[n]));
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int h = 2 * lc + c;
            const float f = __shfl_sync(0xffffffffu, inv, lc * 8 + c * 4) * v_ref;
            if (h + 8 * n < heads) {
              uint16_t* out = p.out + (out0 + h) * D + lr * S::kEV;
#pragma unroll
              for (int j = 0; j < S::kVC; ++j)
#pragma unroll
                for (int e = 0; e < S::kEV / 2; e += 4) {
                  uint32_t o[4];
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    const float* a = acc[j * (S::kEV / 2) + e + i][n];
                    o[i] = bf16_pair(a[c] * f, a[c + 2] * f);
                  }
                  *reinterpret_cast<uint4*>(out + j * 8 * S::kEV + e * 2) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
          }
        }
        return;
      }
      if (!more) asm volatile("cp.async.wait_group 0;" ::: "memory");   // the ring is no longer filled
      __syncwarp();
      const Part<S, true> part = more ? first_part(warp) : last_part(warp);
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        if (lc == 0 && lr + 8 * n < NH) {
          part.most(lr + 8 * n) = most[n];
          part.total(lr + 8 * n) = sum[n];
        }
#pragma unroll
        for (int d = 0; d < D / 16; d += 2) {
          const int j = d / (S::kEV / 2), e = d % (S::kEV / 2);
          const int d4 = ((j * 8 + lr) * S::kEV + 2 * e) / 4;
#pragma unroll
          for (int c = 0; c < 2; ++c)
            if (!S::kHalves || lc < 2)
              part.sums(2 * lc + c + 8 * n, d4) = make_float4(acc[d][n][c] * v_ref, acc[d][n][c + 2] * v_ref, acc[d + 1][n][c] * v_ref, acc[d + 1][n][c + 2] * v_ref);
        }
      }
      if (lane == 0) s_head[2 * warp + (more ? 0 : 1)] = make_int4(at.b * p.rows_of_seq + at.r, from_start, to_end, 0);
    };

    bool fresh = true;
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      if (fresh) begin_row();
      add_tile();
      fresh = at.left == 1;
      if (fresh || i + 1 == count) end_row(fresh, i + 1 < count);
      at.next(p);
    }
  }
  __syncthreads();

  // ---- rows that no warp has alone.  Lane i has the i-th part of the CTA (two for each warp, of the rows in order); a warp takes a head of
  // a row at a time.
  const int4 own = lane < 2 * S::kWarps ? s_head[lane] : make_int4(-1, 0, 0, 0);
  const Part<S, true> own_part = lane & 1 ? last_part(lane >> 1) : first_part(lane >> 1);
  const uint32_t there = __ballot_sync(0xffffffffu, own.x >= 0);
  int4* const headers = p.headers + 2 * blockIdx.x;
  int task = 0, crossing0 = -1, crossing1 = -1, ends0 = 0;
  for (uint32_t rest = there; rest;) {
    const int leader = __ffs(rest) - 1;
    const int row = __shfl_sync(0xffffffffu, own.x, leader);
    const uint32_t parts = __ballot_sync(0xffffffffu, own.x == row);
    rest &= ~parts;
    const int starts = __shfl_sync(0xffffffffu, own.y, leader), ends = __shfl_sync(0xffffffffu, own.z, 31 - __clz(parts));
    if (!starts) crossing0 = row, ends0 = ends;
    else if (!ends) crossing1 = row;
    const int b = row / p.rows_of_seq;
    int heads;
    const int h0 = first_head<S>(p, row - b * p.rows_of_seq, heads);
    for (int head = 0; head < heads; ++head, ++task) {
      if (task % S::kWarps != warp) continue;
      const bool mine = own.x == row;
      const float m = mine ? own_part.most(head) : kNegInf;
      float most = m;
#pragma unroll
      for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      const float f = weight(m, most);
      float total_p = mine ? f * own_part.total(head) : 0.f;
#pragma unroll
      for (int o = 16; o; o >>= 1) total_p += __shfl_xor_sync(0xffffffffu, total_p, o);
      for (int d4 = lane; d4 < (D / 4 + 31) / 32 * 32; d4 += 32) {         // (the whole warp goes round)
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        for (uint32_t of = parts; of;) {
          float fi[4];
          float4 v[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {      // (the last one again, with a factor of 0, where there are fewer)
            const int i = of ? __ffs(of) - 1 : leader;
            fi[u] = __shfl_sync(0xffffffffu, f, i);
            if (!of) fi[u] = 0.f;
            of &= of - 1;
            v[u] = (i & 1 ? last_part(i >> 1) : first_part(i >> 1)).sums(head, d4 % (D / 4));
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) sum.x += v[u].x * fi[u], sum.y += v[u].y * fi[u], sum.z += v[u].z * fi[u], sum.w += v[u].w * fi[u];
        }
        if (d4 >= D / 4) continue;
        if (!starts || !ends) {
          Part<S, false>{p.parts + (2ll * blockIdx.x + (starts ? 1 : 0)) * S::kPart}.sums(head, d4) = sum;
        } else {
          const float inv = 1.f / total_p;
          reinterpret_cast<uint2*>(p.out)[((long long)b * p.n_heads + h0 + head) * (D / 4) + d4] =
              make_uint2(bf16_pair(sum.x * inv, sum.y * inv), bf16_pair(sum.z * inv, sum.w * inv));
        }
      }
      if (lane == 0) {
        if (!starts || !ends) {
          const Part<S, false> part{p.parts + (2ll * blockIdx.x + (starts ? 1 : 0)) * S::kPart};
          part.most(head) = most;
          part.total(head) = total_p;
        } else if (p.lse) {
          p.lse[(long long)b * p.n_heads + h0 + head] = kLn2 * (most + log2f(total_p));
        }
      }
    }
  }
  if (tid == 0) {
    headers[0] = make_int4(crossing0, ends0, 0, 0);
    headers[1] = make_int4(crossing1, 0, 0, 0);
  }

  // ---- sequences that are not there have outputs all the same
  for (int b = blockIdx.x; b < B; b += gridDim.x)
    if (span_of(p, b).tiles() == 0) {
      for (int i = tid; i < p.n_heads * (D / 8); i += kThreads)
        reinterpret_cast<uint4*>(p.out)[(long long)b * p.n_heads * (D / 8) + i] = make_uint4(0, 0, 0, 0);
      if (p.lse)
        for (int i = tid; i < p.n_heads; i += kThreads) p.lse[(long long)b * p.n_heads + i] = kNegInf;
    }
}

// Joins the rows that cross CTAs.  CTA i takes the row that begins in CTA i of the kernel before and goes on in the next ones.
constexpr int kMaxCtas = 256;
template <int D, int NH>
__global__ void __launch_bounds__(256) attn_join_kernel(const AttnParams p, const int ctas) {
  using S = Shape<D, NH, false, true>;
  __shared__ float s_weight[NH][kMaxCtas];
  __shared__ float s_inv[NH];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int4 own = ptx::behind_wait(p.headers)[2 * blockIdx.x + 1];
  const int row = own.x;
  if (row < 0) return;
  // parts of the row: the own one, then the first ones of the CTAs behind, up to the one that has the row's end
  int n = 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int base = blockIdx.x + 1; base < ctas; base += 32) {
    const int c = base + lane;
    const int4 h = c < ctas ? ptx::behind_wait(p.headers)[2 * c] : make_int4(-1, 1, 0, 0);
    const uint32_t stop = __ballot_sync(0xffffffffu, h.x != row || h.y);
    if (stop) {
      const int l = __ffs(stop) - 1;
      n += l + (__shfl_sync(0xffffffffu, h.x, l) == row ? 1 : 0);
      break;
    }
    n += 32;
  }
  auto part_of = [&](int i) { return Part<S, false>{p.parts + (i == 0 ? 2ll * blockIdx.x + 1 : 2ll * (blockIdx.x + i)) * S::kPart}; };
  const int b = row / p.rows_of_seq;
  int heads;
  const int h0 = first_head<S>(p, row - b * p.rows_of_seq, heads);
  for (int head = warp; head < heads; head += 8) {
    float most = kNegInf;
    for (int i = lane; i < n; i += 32) most = fmaxf(most, part_of(i).most(head));
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    float total = 0.f;
    for (int i = lane; i < n; i += 32) {
      const float w = weight(part_of(i).most(head), most);
      s_weight[head][i] = w;
      total += w * part_of(i).total(head);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    if (lane == 0) {
      s_inv[head] = 1.f / total;
      if (p.lse) p.lse[(long long)b * p.n_heads + h0 + head] = kLn2 * (most + log2f(total));
    }
  }
  __syncthreads();
  for (int item = tid; item < heads * (D / 4); item += 256) {
    const int head = item / (D / 4), d = item % (D / 4) * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float w = s_weight[head][i];
      const float4 v = part_of(i).sums(head, d / 4);
      sum.x += w * v.x, sum.y += w * v.y, sum.z += w * v.z, sum.w += w * v.w;
    }
    const float inv = s_inv[head];
    const long long o = (long long)b * p.n_heads + h0 + head;
    *reinterpret_cast<uint2*>(p.out + o * D + d) = make_uint2(bf16_pair(sum.x * inv, sum.y * inv), bf16_pair(sum.z * inv, sum.w * inv));
  }
}

int attn_ctas() { return min(sm_count_or(148), kMaxCtas); }

// Query heads of a row of work.
int heads_of_row(int group, int dim) { return group <= 4 ? 4 : group <= 8 || dim > 128 ? 8 : 16; }

template <int D, int NH, bool I8, bool WHOLE>
int launch(const AttnParams& p, cudaStream_t st) {
  using S = Shape<D, NH, I8, WHOLE>;
  static std::atomic<uint64_t> allowed{0};
  PEQA_TRY(allow_smem(attn_decode_kernel<S>, S::kSmem, allowed));
  const int ctas = attn_ctas();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas, 1, 1);
  cfg.blockDim = dim3(S::kWarps * 32, 1, 1);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  PEQA_CUDA(cudaLaunchKernelEx(&cfg, attn_decode_kernel<S>, p));
  return launch_after(attn_join_kernel<D, NH>, ctas, 256, st, p, ctas);
}

template <int D, int NH>
int launch_type(const AttnParams& p, bool codes, cudaStream_t st) {
  const bool whole = p.cache.page_size % kTile == 0;
  if (codes) return whole ? launch<D, NH, true, true>(p, st) : launch<D, NH, true, false>(p, st);
  return whole ? launch<D, NH, false, true>(p, st) : launch<D, NH, false, false>(p, st);
}

template <int D>
int launch_heads(const AttnParams& p, int nh, bool codes, cudaStream_t st) {
  if (nh == 4) return launch_type<D, 4>(p, codes, st);
  if constexpr (D <= 128)
    if (nh == 16) return launch_type<D, 16>(p, codes, st);
  return launch_type<D, 8>(p, codes, st);
}

// headers, parts of CTAs, parts of warps
size_t workspace_bytes(int dim, int nh) {
  const int warps = dim > 128 || nh > 8 ? 8 : 16;
  static_assert(Shape<128, 8, false, true>::kWarps == 16 && Shape<64, 16, false, true>::kWarps == 8 && Shape<256, 4, true, true>::kWarps == 8, "");
  return (size_t)attn_ctas() * (2 * sizeof(int4) + (2 + warps) * (size_t)nh * (dim + 2) * sizeof(float));
}

}  // namespace
}  // namespace peqa

using namespace peqa;

extern "C" size_t peqa_attn_workspace_bytes(const peqa_kv_cache_t* c, int n_heads) {
  if (!c || c->n_kv_heads < 1 || n_heads < 1 || n_heads % c->n_kv_heads != 0) return 0;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return 0;
  return workspace_bytes(c->head_dim, heads_of_row(n_heads / c->n_kv_heads, c->head_dim));
}

extern "C" int peqa_attn_decode(const peqa_kv_cache_t* c, const peqa_rows_t* q, int n_heads, const int32_t* seq_lens,
                                float scale, int window, void* out, float* lse, void* workspace, size_t bytes,
                                void* stream) {
  AttnParams p = {};
  PEQA_TRY(check_kv_cache(c, &p.cache));
  if (!q || !seq_lens || !out) return PEQA_ERR_NULL;
  if (n_heads < 1 || n_heads % c->n_kv_heads != 0 || window < 0) return PEQA_ERR_BAD_SHAPE;
  PEQA_TRY(check_rows(q, c->n_seqs, n_heads, c->head_dim, false));
  if (!aligned16(out)) return PEQA_ERR_ALIGNMENT;
  if ((reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(lse)) & 3u) return PEQA_ERR_ALIGNMENT;
  p.group = n_heads / c->n_kv_heads;
  const int nh = heads_of_row(p.group, c->head_dim);
  p.chunks = (p.group + nh - 1) / nh;
  // tiles and rows are numbered in 31 bits
  const long long rows_of_seq = (long long)c->n_kv_heads * p.chunks, rows = c->n_seqs * rows_of_seq;
  if (rows > 0x7fffffffll || rows > 0x7fffffffll / (p.cache.capacity / kTile + 2)) return PEQA_ERR_TOO_LARGE;
  p.rows_of_seq = (int)rows_of_seq;
  PEQA_TRY(check_arch());
  if (!workspace || bytes < workspace_bytes(c->head_dim, nh)) return PEQA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return PEQA_ERR_ALIGNMENT;
  p.q = static_cast<const uint16_t*>(q->data);
  p.q_row = c->n_seqs > 1 ? q->row_stride : 0;
  p.q_head = n_heads > 1 ? q->head_stride : 0;
  p.seq_lens = seq_lens;
  p.n_heads = n_heads;
  p.scale_log2 = scale * kLog2e;
  p.window = window;
  p.out = static_cast<uint16_t*>(out);
  p.lse = lse;
  p.headers = static_cast<int4*>(workspace);
  p.parts = reinterpret_cast<float*>(p.headers + 2 * attn_ctas());
  p.first_parts = p.parts + (size_t)attn_ctas() * 2 * nh * (c->head_dim + 2);
  cudaStream_t st = as_stream(stream);
  PEQA_TRY(status_word(st, &p.status));
  const bool codes = c->type == PEQA_KV_INT8;
  switch (c->head_dim) {
    case 64: return launch_heads<64>(p, nh, codes, st);
    case 128: return launch_heads<128>(p, nh, codes, st);
    default: return launch_heads<256>(p, nh, codes, st);
  }
}

// Attention of one new token per sequence to its paged cache (Sec. 3.1: generation is bound by what it reads).
//
//   out[b,h] = sum_t p_t v_t,   p_t = exp(s_t - lse),   s_t = scale <q[b,h], k_t>,   lse = log sum_t exp(s_t)
//
// Every cached key and value of a row of work is read once, by one warp.  A row is a sequence, a key-value head and up to NH = 4, 8 or 16 of the
// query heads that share it (8 where D is 256): a larger group is several rows, ceil(group / NH) readings.  4 NH flops per cached element are too few to
// bind anything but memory, and the rest is laid out to keep copies in flight:
//   * A tile is 16 tokens of a row.  Tiles are numbered through all sequences, heads and lengths, and dealt evenly: every CTA
//     takes an equal run of them, every warp an equal run of its CTA's.  Nothing depends on how uneven the lengths are.  (With few
//     and short rows a CTA has a row to itself.)
//   * A warp copies its own tiles into its own ring of shared memory, several units of 16 keys or values ahead (tensor copies, or
//     cp.async where pages end within tiles), and reads them with ldmatrix as the 16-row operand of the tensor cores' m16n8k16 product, the
//     heads as its 8 columns:
//       S^T = K Q^T     K [16 tokens x 16 channels] as it lies, Q in registers
//       O^T = V^T P^T   V^T [16 channels x 16 tokens] by the transposing ldmatrix; P^T from S^T by movmatrix
//     So there is no barrier between warps in the loop, and a lane has the factors of the sums that it holds.
//   * With bf16 up to four query heads stand in the columns twice, and p's two numbers (below) in the two places.
//   * Running maximum and sum per row, as the softmax allows: the sums are rescaled only when the maximum has risen by more than
//     kSlack (a factor of 2^8 that the binary32 sums carry easily).
//   * With bf16 values p goes into the second product as the sum of two of them (off by 2^-16 of p): with one, its rounding (2^-8 of p at most) would
//     double the error variance that the rounding of the output has.  8-bit codes are exact in binary16, and p in it is off by 2^-11 of itself at
//     most, an eighth of that (the error of outputs against 64 bits grows by 0.6 % of itself; a second binary16 for the rest costs 4 to 6 % of time).
//   * A row that a warp has from its first tile to its last is written out.  Parts of rows are joined within the CTA in shared
//     memory, and what crosses CTAs by a second kernel, which stands ready when the first ends.
#include "common.cuh"
#include "kv_cache.cuh"
#include "sm100_ptx.cuh"
#include "tensor_map.cuh"

#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace peqa {
namespace {

constexpr int kTile = 16;            // tokens
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
  bool row_each;                     // a CTA has a row to itself
  bool halves;                       // bf16: a tile of which 8 tokens or fewer are there is copied by half
  uint16_t* out;
  float* lse;
  // [CTAs][2]: row that an earlier CTA began, row that a later one goes on with (-1: none).  (Whole sectors: one that is written in part is
  // filled from memory before it is read, 0.4 to 0.7 us of every call.)
  int4* headers;
  float* parts;                      // [CTAs][2][Shape::kPart]: of those rows
  float* first_parts;                // [CTAs][warps][D][NH]
  int* status;
};

// By the registers that a thread needs.
constexpr int warps_of(int dim, int nh) { return dim > 128 ? 8 : nh <= 8 ? 16 : dim <= 64 ? 12 : 8; }

// Everything that follows from the channels D, the query heads NH of a row, the type of the cache and whether a tile comes by
// tensor copies (WHOLE: it lies in one page).
template <int D_, int NH_, bool I8_, bool WHOLE_>
struct Shape {
  static constexpr int D = D_, NH = NH_;
  static constexpr bool I8 = I8_, WHOLE = WHOLE_;
  static constexpr bool kHalves = NH == 4 && !I8;               // the two numbers that p is are columns of one product
  static constexpr int kCols = NH > 8 ? 2 : 1;                  // of eight heads (kHalves: of four, twice)
  static constexpr int kBytes = D * (I8 ? 1 : 2);               // of a token
  static constexpr int kPieces = kBytes / 16;                   // 16-byte pieces of a token
  static constexpr int kLine = kBytes < 128 ? kBytes : 128;     // bytes of a token that lie together in shared memory
  static constexpr int kRows = 32 / kPieces;                    // tokens that a warp copies with one instruction
  static constexpr int kUnit = kTile * kBytes;                  // keys or values of a tile
  static constexpr int kWarps = warps_of(D, NH);
  static constexpr int kFit = 192 * 1024 / (kWarps * (kUnit + (I8 ? 64 : 0)));
  static constexpr int kUnits = kFit >= 9 ? 9 : kFit >= 7 ? 7 : kFit >= 5 ? 5 : 3;   // odd: keys follow keys, values values
  static constexpr int kRing = kUnits * kUnit;
  static constexpr int kSmem = kWarps * (kRing + (I8 ? kUnits * 64 : 0));            // and the scales of a unit's 16 tokens
  static constexpr int kPart = NH * (D + 2);                    // floats of a part: sums, maxima, sums of p
  static_assert(kFit >= 3 && kRing >= 2 * NH * D * 4 && kRing % 1024 == 0 && kPart % 4 == 0, "shared memory");
};

// A box of 16 tokens (8) from token y on: channels from x on of head `head` in page `page`.
__device__ __forceinline__ void tensor_copy(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int head, int y, int page) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(head), "r"(y), "r"(page)
      : "memory");
}
__device__ __forceinline__ void bulk_copy_64(uint32_t dst, const void* src, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], 64, [%2];" ::"r"(dst), "l"(src), "r"(bar) : "memory");
}
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, uint32_t bytes, std::integral_constant<int, 16>) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, uint32_t bytes, std::integral_constant<int, 4>) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// Four 8 x 8 matrices of 16-bit elements, their rows at the addresses that the lanes give (lanes 8 i .. 8 i + 7: matrix i).  Lane (r, c) gets
// elements 2 c and 2 c + 1 of row r, or (transposed) of column r.
__device__ __forceinline__ void ldmatrix(uint32_t (&x)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix_transposed(uint32_t (&x)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
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
// the same from sums c0, c1 of the columns on
__device__ __forceinline__ void mma_from(float (&d)[4], float c0, float c1, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%10,%11};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1));
}
// 2^x, 0 below 2^-126
__device__ __forceinline__ float power_of_two(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Codes of 8 bits, with their sign bits turned: c + 128 as a byte.  Two of them as binary16: 0x6400 | byte is 1024 + 128 + c.
__device__ __forceinline__ uint32_t codes(uint32_t x, uint32_t which) {
  const uint32_t h = __byte_perm(x, 0x64646464u, which);
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&h), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// Two numbers as 16 bits; lower half: p0.
__device__ __forceinline__ uint32_t half_pair(float p0, float p1) {
  const __half2 h = __floats2half2_rn(p0, p1);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The upper 16 bits of two numbers that are not negative, as bf16, and what they leave.  Cut and not rounded, and with the lowest bit set: both
// parts are then above 0 wherever p is (from 2^-110 on), so that p times an infinite value is that infinity, and not 0 inf or inf - inf.  What
// is left, below 2^-7 of p, is rounded to bf16 where it is used: 2^-16 of p at most.
__device__ __forceinline__ uint32_t upper_halves(float& p0, float& p1) {
  const uint32_t a = __float_as_uint(p0), b = __float_as_uint(p1);
  p0 = __uint_as_float(a | 1u) - __uint_as_float(a & 0xffff0000u);
  p1 = __uint_as_float(b | 1u) - __uint_as_float(b & 0xffff0000u);
  return __byte_perm(a, b, 0x7632);
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
    if (--left > 0) {
      t0 += kTile;
      return false;
    }
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

// Sums of a row, or of a part of one, in a part's memory: O^T [D][NH], then the maxima and the sums of p.
template <int D, int NH>
struct Part {
  float* at;
  __device__ __forceinline__ float2& two(int d, int head) const { return *reinterpret_cast<float2*>(at + d * NH + head); }
  // four heads of a channel, by their place
  __device__ __forceinline__ float4& four(int i) const { return reinterpret_cast<float4*>(at)[i]; }
  __device__ __forceinline__ float4& most4(int head) const { return *reinterpret_cast<float4*>(at + D * NH + head); }
  __device__ __forceinline__ float4& total4(int head) const { return *reinterpret_cast<float4*>(at + (D + 1) * NH + head); }
};
__device__ __forceinline__ float4 operator*(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
__device__ __forceinline__ float4 operator+(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

__device__ __forceinline__ float4 larger(float4 a, float4 b) {
  return make_float4(fmaxf(a.x, b.x), fmaxf(a.y, b.y), fmaxf(a.z, b.z), fmaxf(a.w, b.w));
}
__device__ __forceinline__ float4 shuffled(float4 a, int o) {
  return make_float4(__shfl_xor_sync(0xffffffffu, a.x, o), __shfl_xor_sync(0xffffffffu, a.y, o), __shfl_xor_sync(0xffffffffu, a.z, o),
                     __shfl_xor_sync(0xffffffffu, a.w, o));
}
__device__ __forceinline__ float weight(float m, float most) { return m == kNegInf ? 0.f : exp2f(m - most); }

// Channel d of heads h0 + head .. + 3, as far as there are heads, and their log-sums where d is 0.
template <int D>
__device__ __forceinline__ void put_out(const AttnParams& p, long long row0, int heads, int head, int d, float4 sum, float4 most, float4 total) {
  const float o[4] = {sum.x, sum.y, sum.z, sum.w}, m[4] = {most.x, most.y, most.z, most.w}, t[4] = {total.x, total.y, total.z, total.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (head + i < heads) {
      const __nv_bfloat16 x = __float2bfloat16_rn(o[i] * __fdividef(1.f, t[i]));
      p.out[(row0 + head + i) * D + d] = *reinterpret_cast<const uint16_t*>(&x);
      if (p.lse && d == 0) p.lse[row0 + head + i] = kLn2 * (m[i] + log2f(t[i]));
    }
}

// First query head of a row, and how many there are.
template <int NH>
__device__ __forceinline__ int first_head(const AttnParams& p, int r, int& heads) {
  const int kv = r / p.chunks, chunk = r - kv * p.chunks;
  heads = min(NH, p.group - chunk * NH);
  return kv * p.group + chunk * NH;
}

template <typename S>
__global__ void __launch_bounds__(S::kWarps * 32, 1) attn_decode_kernel(const AttnParams p, const __grid_constant__ CUtensorMap keys,
                                                                        const __grid_constant__ CUtensorMap values,
                                                                        const __grid_constant__ CUtensorMap keys8,
                                                                        const __grid_constant__ CUtensorMap values8) {
  constexpr int D = S::D, NH = S::NH, kCols = S::kCols, kThreads = S::kWarps * 32;
  constexpr bool I8 = S::I8;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ int s_scan[kThreads];
  __shared__ int s_warp[S::kWarps];
  __shared__ __align__(16) float s_weight[32][NH], s_most[32][NH], s_total[32][NH];   // of a part and head; s_most: at last of its row
  __shared__ int4 s_head[2 * S::kWarps];   // of a warp's parts: row (-1: none), 1 if it begins its row + 2 if it ends it + 4 times its heads, its first head's place in out
  __shared__ __align__(8) uint64_t s_full[S::WHOLE ? S::kWarps * S::kUnits : 1];
  __shared__ uint32_t s_empty;             // of sequences blockIdx.x + i gridDim.x, i < 32: those without tiles
  __shared__ int s_abort[2];               // as the bounded waits of sm100_ptx.cuh have it

  const int tid = threadIdx.x, lane = tid & 31, warp = ptx::warp_index();
  const int lr = lane >> 2, lc = lane & 3;
  const uint32_t ring = ptx::smem_u32(smem) + warp * S::kRing;
  // a warp's parts of rows in its ring, when that is free: the one that it began with (i even; until then it lies in the workspace), its last
  const auto part_of = [&](int i) { return Part<D, NH>{reinterpret_cast<float*>(smem + (i >> 1) * S::kRing) + (i & 1 ? 0 : NH * D)}; };
  const auto first_part = [&]() { return Part<D, NH>{p.first_parts + ((long long)blockIdx.x * S::kWarps + warp) * (NH * D)}; };

  volatile int* const abort_flag = s_abort;
  if (lane < 2) s_head[2 * warp + lane] = make_int4(-1, 0, 0, 0);   // each warp its own: no barrier is sure to come before its parts
  __syncwarp();
  if constexpr (S::WHOLE) {
    // self-test knob (peqa_selftest_configure): one arrival more than will come, so that no unit is ever full
    if (lane < S::kUnits) ptx::mbar_init(ptx::smem_u32(&s_full[warp * S::kUnits + lane]), p.status[5] ? 2 : 1);
    ptx::fence_mbar_init();
    if (tid == 0) {
      s_abort[0] = 0;
      s_abort[1] = p.status[4];
      ptx::prefetch_tmap(&keys);
      ptx::prefetch_tmap(&values);
    }
    __syncthreads();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  const int B = p.cache.n_seqs;
  if (warp == S::kWarps - 1) {               // at the end their lengths would be waited for once more
    const long long b = blockIdx.x + (long long)lane * gridDim.x;
    const uint32_t empty = __ballot_sync(0xffffffffu, b < B && span_of(p, (int)b).tiles() == 0);
    if (lane == 0) s_empty = empty;
  }
  // ---- the tiles of all sequences, and this warp's share of them: [begin, end)
  int total = 0, begin = 0, end = 0;
  auto among_warps = [&](int first, int n) {
    const int each = n / S::kWarps, more = n - each * S::kWarps;           // the first `more` warps have one more
    begin = first + each * warp + min(warp, more);
    end = begin + each + (warp < more);
  };
  auto share = [&]() {
    // no CTA without a tile for a warp of each scheduler, while there are enough
    const int busy = min((int)gridDim.x, max(1, total / 4)), cta = blockIdx.x;
    if (cta >= busy) return;
    const int each = total / busy, more = total - each * busy;             // the first `more` CTAs have one more
    among_warps(each * cta + min(cta, more), each + (cta < more));
  };
  auto tiles_of = [&](int b) { return b < B ? span_of(p, b).tiles() * p.rows_of_seq : 0; };
  if (B > kThreads && !p.row_each) {
    for (int b = tid; b < B; b += kThreads) total += tiles_of(b);
    total = __reduce_add_sync(0xffffffffu, total);
    if (lane == 0) s_warp[warp] = total;
    __syncthreads();
    total = __reduce_add_sync(0xffffffffu, lane < S::kWarps ? s_warp[lane] : 0);
    share();
  }
  Cursor in;                                // of the copies; the sums follow with `at`
  in.b = in.r = in.t0 = in.left = in.span.first = in.span.end = 0;
  int before = 0;                           // tiles of the sequences before these
  if (p.row_each) {
    const int b = blockIdx.x / p.rows_of_seq, r = blockIdx.x - b * p.rows_of_seq;
    const int tiles = span_of(p, b).tiles();
    among_warps(r * tiles, tiles);          // of the sequence's tiles
    if (begin < end) in.begin(p, b, begin);
  } else if (B <= 32) {                     // every warp for itself
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
    const uint32_t full_of = ptx::smem_u32(&s_full[S::WHOLE ? warp * S::kUnits : 0]);
    uint32_t put_full = full_of, get_full = full_of, get_phase = 0;
    // A token's 16-byte pieces lie in lines of 128 bytes, the lines of the unit's tokens one behind another; piece c of token t in place
    // c ^ (t & 7) of its line (lines of 64 bytes: c ^ (t / 2 & 3)), as tensor copies mix them: the eight rows of a matrix are in different banks.
    auto turn_of = [](int t) { return S::kLine == 128 ? t & 7 : t >> 1 & 3; };
    auto place_of = [&](int t, int c) { return (uint32_t)(c / 8 * kTile * S::kLine + t * S::kLine + ((c & 7) ^ turn_of(t)) * 16); };
    // matrices of keys, and of 8-bit values: tokens 0..7 and 8..15 of a piece, then of the next; of values: two pieces of tokens 0..7, then of 8..15
    const uint32_t key_at = place_of((lane & 7) + (lane & 8), lane >> 4);
    const uint32_t value_at = I8 ? key_at : place_of((lane & 7) + (lane >> 4) * 8, lane >> 3 & 1);
    auto pair_at = [](uint32_t at, int j) { return (at ^ ((2 * j & 7) * 16)) + j / 4 * kTile * S::kLine; };   // pieces 2 j and 2 j + 1
    int entry = 0, place = 0;                // of the copies' tile: of the page table, and in the page (WHOLE)
    uint32_t unit = 0;                       // else place of token (lane & 15) of it in the cache
    uint32_t scale = 0;                      // and in the scales (fewer than 2^30: each has 64 bytes of codes, and they have less than 2^36)
    int kv = in.r / p.chunks;                // head of keys and values
    auto table_of = [&](int e) { return ptx::ld_global(p.cache.table + (long long)in.b * p.cache.max_pages + e); };
    // Page of the copies' tile or of its token (lane & 15), asked for a tile ahead of its use.
    auto look_up = [&](bool new_row, bool there) {
      if constexpr (S::WHOLE) {
        place += kTile;
        if (new_row) {
          entry = divide(in.t0, p.cache.by_page);
          place = in.t0 - entry * p.cache.page_size;
          kv = in.r / p.chunks;
        } else if (place == p.cache.page_size) {
          ++entry;
          place = 0;
        } else {
          return;                            // the page it has
        }
        page = there ? table_of(entry) : 0;
      } else {
        if (new_row) kv = in.r / p.chunks;
        const int t = in.t0 + (lane & 15);
        page = there && t >= in.span.first && t < in.span.end ? table_of(divide(t, p.cache.by_page)) : 0;
      }
    };
    auto in_span = [&](int t) { return t >= in.span.first && t < in.span.end; };
    auto check_page = [&]() {
      if ((uint32_t)page >= (uint32_t)p.cache.n_pages) {
        note_bad_index(p.status);
        page = 0;
      }
    };
    // Keys or values of the tile, by tensor copies: a page has all of them, or places of its own for what is behind the sequence's end.
    auto copy_whole = [&](const CUtensorMap* map, const CUtensorMap* map8, const float* scales) {
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (ptx::elect_lane() == 0) {
        const bool half = !I8 && p.halves && in.span.end - in.t0 <= kTile / 2;
        ptx::mbar_arrive_expect_tx(put_full, (half ? S::kUnit / 2 : S::kUnit) + (I8 ? 64 : 0));
#pragma unroll
        for (int c = 0; c < S::kBytes / S::kLine; ++c)
          tensor_copy(put + c * kTile * S::kLine, half ? map8 : map, put_full, c * (S::kLine / (I8 ? 1 : 2)), kv, place, page);
        if constexpr (I8) bulk_copy_64(put_scales, scales + (uint32_t)((page * p.cache.n_kv_heads + kv) * p.cache.page_size + place), put_full);
      }
      __syncwarp();
    };
    // The same where pages end within tiles, token by token: 512 bytes an instruction.  (In pieces of 64 bytes, as the products take keys,
    // copies of blocks of 4 KB reach 4.9 TB/s of 6.6.)  0 for what is not seen.
    auto copy_tokens = [&](const void* from, const float* scales) {
      const int row = lane / S::kPieces, piece = lane % S::kPieces;
      const char* const base = static_cast<const char*>(from) + piece * 16;
      const uint32_t to = put + place_of(row, piece);
#pragma unroll
      for (int j = 0; j < kTile / S::kRows; ++j)
        cp_async((to ^ (turn_of(j * S::kRows) * 16)) + j * S::kRows * S::kLine,
                 base + (uint64_t)__shfl_sync(0xffffffffu, unit, row + j * S::kRows) * 16, in_span(in.t0 + row + j * S::kRows) ? 16 : 0,
                 std::integral_constant<int, 16>());
      if constexpr (I8)
        if (lane < 16) cp_async(put_scales + lane * 4, scales + scale, in_span(in.t0 + lane) ? 4 : 0, std::integral_constant<int, 4>());
    };
    auto filled = [&]() {
      if constexpr (!S::WHOLE) asm volatile("cp.async.commit_group;" ::: "memory");
      put += S::kUnit, put_scales += 64, put_full += 8;
      if (put == ring + S::kRing) put = ring, put_scales = scales_of, put_full = full_of;
    };
    auto issue_keys = [&]() {
      if (issued < count) {
        check_page();
        if constexpr (S::WHOLE) {
          copy_whole(&keys, &keys8, p.cache.k_scales);
        } else {
          const int t = in.t0 + (lane & 15);
          const uint32_t at_place = t - divide(t, p.cache.by_page) * p.cache.page_size;
          unit = page * p.cache.page16 + at_place * p.cache.token16 + kv * p.cache.head16;
          scale = (page * p.cache.n_kv_heads + kv) * p.cache.page_size + at_place;
          copy_tokens(p.cache.k, p.cache.k_scales);
        }
      }
      filled();
    };
    auto issue_values = [&]() {
      if (issued < count) {
        if constexpr (S::WHOLE) copy_whole(&values, &values8, p.cache.v_scales);
        else copy_tokens(p.cache.v, p.cache.v_scales);
        const bool new_row = in.next(p);
        look_up(new_row, issued + 1 < count);
      }
      ++issued;
      filled();
    };
    bool sound = true;                       // no wait has run out
    auto landed = [&]() {
      if constexpr (S::WHOLE) sound = ptx::warp_wait(get_full, get_phase, abort_flag) && sound;
      else asm volatile("cp.async.wait_group %0;" ::"n"(S::kUnits - 2) : "memory");
      __syncwarp();                          // for all lanes, and all have read what is filled next
    };
    auto read = [&]() {
      get += S::kUnit, get_scales += 64, get_full += 8;
      if (get == ring + S::kRing) get = ring, get_scales = scales_of, get_full = full_of, get_phase ^= 1;
    };
    uint32_t q[kCols][D / 16][2];                            // head lr (+ 8): two and two channels for each product
    auto load_q = [&]() {
      int heads;
      const int h0 = first_head<NH>(p, at.r, heads);
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        const int h = (S::kHalves ? lr & 3 : lr) + 8 * n;
        const uint16_t* from = p.q + at.b * p.q_row + (long long)(h0 + h) * p.q_head;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
          uint2 x = make_uint2(0u, 0u);
          if (h < heads) {
            // as the matrices have the channels: 2 lc and 8 + 2 lc of a product's sixteen, of 8-bit keys 4 lc .. 4 lc + 3
            if constexpr (I8) x = ptx::ld_global(reinterpret_cast<const uint2*>(from + 16 * s + 4 * lc));
            else x = make_uint2(ptx::ld_global(reinterpret_cast<const uint32_t*>(from + 16 * s + 2 * lc)),
                                ptx::ld_global(reinterpret_cast<const uint32_t*>(from + 16 * s + 8 + 2 * lc)));
          }
          q[n][s][0] = x.x, q[n][s][1] = x.y;
        }
      }
    };
    load_q();                                // before the first copies: behind those of all CTAs they come 2 us later (16 sequences of up to 300 tokens 8.9 -> 8.6 us)
    look_up(true, true);
#pragma unroll 1
    for (int i = 0; i < S::kUnits / 2; ++i) {
      issue_keys();
      issue_values();
    }

    float to_log2[kCols][2];                                 // of a product of the tensor cores; here and below: heads 2 lc, 2 lc + 1 (+ 8)
    float q_bias[kCols][2];                                  // I8: what the sums of products begin with
    float most[kCols][2], sum[kCols][2];                     // sum: of this lane's tokens
    float base[kCols][2];                                    // most, or 0 where there is none
    float acc[D / 16][kCols][4];                             // two channels of each of the two heads
    float v_ref = 1.f, inv_ref = 1.f;                        // I8: acc is in units of it
    bool from_start, behind = false;         // behind: this warp has the end of a row that the ones before began

    auto begin_row = [&]() {
#pragma unroll
      for (int n = 0; n < kCols; ++n) {
        float scale = p.scale_log2, bias = 0.f;
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
          // Codes come as c + 128 in the lowest bits of a binary16, (c + 128) 2^-24: each sum begins with -128 2^-24 times the sum of q.
          // (The bias is about three times as large as the sums themselves, so their last bits weigh as much more.)
          scale = p.scale_log2 * __uint_as_float((uint32_t)(127 + e) << 23) * 16777216.f;
#pragma unroll
          for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&q[n][s][w]));
              const __half2 x = __floats2half2_rn(f.x * down, f.y * down);
              q[n][s][w] = *reinterpret_cast<const uint32_t*>(&x);
              const float2 g = __half22float2(x);
              bias += g.x + g.y;
            }
          bias += __shfl_xor_sync(0xffffffffu, bias, 1);
          bias += __shfl_xor_sync(0xffffffffu, bias, 2);
          bias *= -0x1p-17f;
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {                        // from the lanes of head lr to those of its column
          to_log2[n][c] = I8 ? __shfl_sync(0xffffffffu, scale, lc * 8 + c * 4) : scale;
          q_bias[n][c] = I8 ? __shfl_sync(0xffffffffu, bias, lc * 8 + c * 4) : 0.f;
          most[n][c] = kNegInf;
          sum[n][c] = base[n][c] = 0.f;
        }
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int n = 0; n < kCols; ++n) acc[d][n][0] = acc[d][n][1] = acc[d][n][2] = acc[d][n][3] = 0.f;
      if constexpr (I8) v_ref = 0x1p-126f, inv_ref = 0x1p126f;
      from_start = at.t0 == at.tile0();
    };

    auto rescale = [&](const float (&f)[kCols][2]) {
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int n = 0; n < kCols; ++n) acc[d][n][0] *= f[n][0], acc[d][n][1] *= f[n][1], acc[d][n][2] *= f[n][0], acc[d][n][3] *= f[n][1];
    };

    auto add_tile = [&]() {
      const int t0 = at.t0;
      landed();
      issue_keys();
      // ---- S^T = K Q^T, in two sums, so that a product waits for the one before the last
      float s[2][kCols][4];
#pragma unroll
      for (int j = 0; j < S::kPieces / 2; ++j) {
        uint32_t k[4];
        ldmatrix(k, pair_at(get + key_at, j));
        if constexpr (I8) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t u = k[2 * e] ^ 0x80808080u, w = k[2 * e + 1] ^ 0x80808080u;
            const uint32_t a0 = __byte_perm(u, 0u, 0x4140), a1 = __byte_perm(w, 0u, 0x4140), a2 = __byte_perm(u, 0u, 0x4342), a3 = __byte_perm(w, 0u, 0x4342);
#pragma unroll
            for (int n = 0; n < kCols; ++n) {
              if (j == 0 && e == 0) mma_from(s[e][n], q_bias[n][0], q_bias[n][1], a0, a1, a2, a3, q[n][0][0], q[n][0][1]);
              else if (j == 0) mma0<true>(s[e][n], a0, a1, a2, a3, q[n][e][0], q[n][e][1]);
              else mma<true>(s[e][n], a0, a1, a2, a3, q[n][2 * j + e][0], q[n][2 * j + e][1]);
            }
          }
        } else {
#pragma unroll
          for (int n = 0; n < kCols; ++n) {
            if (j < 2) mma0<false>(s[j & 1][n], k[0], k[1], k[2], k[3], q[n][j][0], q[n][j][1]);
            else mma<false>(s[j & 1][n], k[0], k[1], k[2], k[3], q[n][j][0], q[n][j][1]);
          }
        }
      }
      // ---- scores in powers of two: x[n][i] of head 2 lc + (i & 1) + 8 n and token lr + 8 (i >> 1)
      float x[kCols][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float k_scale = 1.f;
        if constexpr (I8) k_scale = lds_float(get_scales + (lr + 8 * (i >> 1)) * 4);
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
          float y = s[0][n][i] + s[1][n][i];
          if constexpr (I8) y *= k_scale;
          x[n][i] = y * to_log2[n][i & 1];
        }
      }
      const bool cut = t0 < at.span.first || at.span.end - t0 < kTile;     // not all of the tile is seen
      if (cut) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + lr + 8 * (i >> 1) < at.span.first || t0 + lr + 8 * (i >> 1) >= at.span.end)
#pragma unroll
            for (int n = 0; n < kCols; ++n) x[n][i] = kNegInf;
      }
      // ---- running maximum, brought up to date where one is passed by more than kSlack
      bool higher = false;
#pragma unroll
      for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) higher |= fmaxf(x[n][c], x[n][c + 2]) > most[n][c] + kSlack;
      if (__any_sync(0xffffffffu, higher)) {
        float f[kCols][2];
#pragma unroll
        for (int n = 0; n < kCols; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float next = fmaxf(x[n][c], x[n][c + 2]);
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) next = fmaxf(next, __shfl_xor_sync(0xffffffffu, next, o));
            next = fmaxf(next, most[n][c]);
            f[n][c] = weight(most[n][c], next);
            sum[n][c] *= f[n][c];
            most[n][c] = next;
            base[n][c] = next == kNegInf ? 0.f : next;
          }
        rescale(f);
      }
      // ---- p and its sum
#pragma unroll
      for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[n][i] = power_of_two(x[n][i] - base[n][i & 1]);
          sum[n][i & 1] += x[n][i];
        }
      // ---- O^T += V^T P^T
      read();
      landed();
      issue_values();
      if (S::WHOLE && !I8 && cut) {          // p is 0 there, and must stay so whatever the page has
        for (int i = lane; i < kTile * S::kPieces; i += 32) {
          const int t = i / S::kPieces;
          if (t0 + t < at.span.first || t0 + t >= at.span.end)
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(get + place_of(t, i % S::kPieces)), "r"(0u) : "memory");
        }
        __syncwarp();
      }
      if constexpr (I8) {
        float v_scale[2] = {lds_float(get_scales + lr * 4), lds_float(get_scales + lr * 4 + 32)};
        if (cut)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (t0 + lr + 8 * i < at.span.first || t0 + lr + 8 * i >= at.span.end) v_scale[i] = 0.f;
        // Values in units of 2^-6 of the largest scale so far, cut to a power of two: p (at most 2^kSlack) times what is left of its
        // token's scale (below 2^7) is a binary16, off by 2^-11 of it, or by 2^-25 of a unit, 2^-31 of the largest.
        float v_rest[2] = {v_scale[0] * inv_ref, v_scale[1] * inv_ref};
        if (__any_sync(0xffffffffu, fmaxf(fabsf(v_rest[0]), fabsf(v_rest[1])) >= 128.f)) {
          const uint32_t exponent = __reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(fabsf(v_scale[0]), fabsf(v_scale[1])))) & 0x7f800000u;
          const float ref = __uint_as_float(exponent - (6u << 23));
          float f[kCols][2];
#pragma unroll
          for (int n = 0; n < kCols; ++n) f[n][0] = f[n][1] = v_ref / ref;
          rescale(f);
          v_ref = ref;
          inv_ref = 1.f / ref;
          v_rest[0] = v_scale[0] * inv_ref, v_rest[1] = v_scale[1] * inv_ref;
        }
#pragma unroll
        for (int n = 0; n < kCols; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[n][i] *= v_rest[i >> 1];
      }
      uint32_t hi[kCols][2], lo[kCols][2];                   // tokens 0..7, 8..15
#pragma unroll
      for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          hi[n][i] = I8 ? half_pair(x[n][2 * i], x[n][2 * i + 1]) : upper_halves(x[n][2 * i], x[n][2 * i + 1]);
          lo[n][i] = I8 ? 0u : bf16_pair(x[n][2 * i], x[n][2 * i + 1]);
          if (S::kHalves && lc >= 2) hi[n][i] = lo[n][i];
          hi[n][i] = transposed(hi[n][i]);
          if constexpr (!I8 && !S::kHalves) lo[n][i] = transposed(lo[n][i]);
        }
      auto product = [&](int d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
          mma<I8>(acc[d][n], a0, a1, a2, a3, hi[n][0], hi[n][1]);
          if constexpr (!I8 && !S::kHalves) mma<I8>(acc[d][n], a0, a1, a2, a3, lo[n][0], lo[n][1]);
        }
      };
#pragma unroll
      for (int j = 0; j < S::kPieces / 2; ++j) {
        uint32_t v[4];
        ldmatrix_transposed(v, pair_at(get + value_at, j));
        if constexpr (I8) {
          // a lane has channels 2 lr and 2 lr + 1 of two tokens, byte by byte
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t u = v[2 * e] ^ 0x80808080u, w = v[2 * e + 1] ^ 0x80808080u;
            product(2 * j + e, codes(u, 0x4240), codes(u, 0x4341), codes(w, 0x4240), codes(w, 0x4341));
          }
        } else {
          product(j, v[0], v[1], v[2], v[3]);
        }
      }
      read();
    };

    // The row's sums, or what this warp has of them, are complete.  acc[d][n]: channels 16 d + lr and 16 d + lr + 8 (I8: 16 d + 2 lr and + 1).
    auto end_row = [&](bool to_end, bool more) {
#pragma unroll
      for (int n = 0; n < kCols; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) sum[n][c] += __shfl_xor_sync(0xffffffffu, sum[n][c], o);
      if constexpr (S::kHalves) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[d][0][i] += __shfl_xor_sync(0xffffffffu, acc[d][0][i], 2);
      }
      int heads;
      const int h0 = first_head<NH>(p, at.r, heads);
      if (from_start && to_end) {
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
          const float f[2] = {__fdividef(v_ref, sum[n][0]), __fdividef(v_ref, sum[n][1])};
          const long long row0 = (long long)at.b * p.n_heads + h0 + 8 * n;
          if (p.lse && lr == 0)
#pragma unroll
            for (int c = 0; c < 2; ++c)
              if (2 * lc + c + 8 * n < heads) p.lse[row0 + 2 * lc + c] = kLn2 * (most[n][c] + log2f(sum[n][c]));
          uint16_t* const out = p.out + (row0 + lr) * D;     // head lr, once transposed
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {
            const uint32_t a = transposed(bf16_pair(acc[d][n][0] * f[0], acc[d][n][1] * f[1]));
            const uint32_t b = transposed(bf16_pair(acc[d][n][2] * f[0], acc[d][n][3] * f[1]));
            if (lr + 8 * n < heads) {
              if constexpr (I8) {                            // a: channels 4 lc and 4 lc + 2, b: the ones behind them
                *reinterpret_cast<uint2*>(out + 16 * d + 4 * lc) = make_uint2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
              } else {
                *reinterpret_cast<uint32_t*>(out + 16 * d + 2 * lc) = a;
                *reinterpret_cast<uint32_t*>(out + 16 * d + 8 + 2 * lc) = b;
              }
            }
          }
        }
        return;
      }
      if (!more) asm volatile("cp.async.wait_group 0;" ::: "memory");   // the ring is no longer filled
      __syncwarp();
      behind = behind || more;
      const Part<D, NH> part = more ? first_part() : part_of(2 * warp + 1);
      if (NH > 4 || lc < 2)
#pragma unroll
        for (int n = 0; n < kCols; ++n) {
          const int head = 2 * lc + 8 * n;
          if (lr == 0) {
            *reinterpret_cast<float2*>(&s_most[2 * warp + (more ? 0 : 1)][head]) = make_float2(most[n][0], most[n][1]);
            *reinterpret_cast<float2*>(&s_total[2 * warp + (more ? 0 : 1)][head]) = make_float2(sum[n][0], sum[n][1]);
          }
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {
            part.two(16 * d + (I8 ? 2 * lr : lr), head) = make_float2(acc[d][n][0] * v_ref, acc[d][n][1] * v_ref);
            part.two(16 * d + (I8 ? 2 * lr + 1 : lr + 8), head) = make_float2(acc[d][n][2] * v_ref, acc[d][n][3] * v_ref);
          }
        }
      if (lane == 0)
        s_head[2 * warp + (more ? 0 : 1)] =
            make_int4(at.b * p.rows_of_seq + at.r, (from_start ? 1 : 0) + (to_end ? 2 : 0) + heads * 4, at.b * p.n_heads + h0, 0);
    };

    bool fresh = true;
#pragma unroll 1
    for (int i = 0; i < count && sound; ++i) {
      if (fresh) {
        if (i > 0) load_q();
        begin_row();
      }
      add_tile();
      fresh = at.left == 1;
      if (fresh || i + 1 == count) end_row(fresh, i + 1 < count);
      at.next(p);
    }
    // The join below reads parts again and again: from shared memory, as the loads from here come while the other warps have tiles left.
    if (behind) {
      constexpr int kEach = NH * D / 128;
      float4 x[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) x[i] = first_part().four(i * 32 + lane);
#pragma unroll
      for (int i = 0; i < kEach; ++i) part_of(2 * warp).four(i * 32 + lane) = x[i];
    }
  }
  __syncthreads();
  if (S::WHOLE && *abort_flag) {
    // copies still in flight must land before the shared memory is given back
    for (int i = 0; i < 64; ++i) __nanosleep(1000);
    if (tid == 0) {
      atomicExch(p.status, (int)PEQA_ERR_DEVICE_TIMEOUT);
      p.status[1] = (int)blockIdx.x;
    }
  }

  // ---- rows that no warp has alone.  Lane i has the i-th part of the CTA (two for each warp, of the rows in order).  A warp finds the weights
  // of all parts for a head, then takes 128 sums of a row at a time, a lane four heads of a channel.
  constexpr int kSlices = NH * D / 128;
  const int4 own = lane < 2 * S::kWarps ? s_head[lane] : make_int4(-1, 0, 0, 0);
  const uint32_t parts_of_own = __match_any_sync(0xffffffffu, own.x);
  for (int head = warp; head < NH; head += S::kWarps) {
    float m = kNegInf;
    if (own.x >= 0) m = s_most[lane][head];
    // the largest of the row's: as whole numbers that have the order of the floats
    const int bits = __float_as_int(m), key = bits ^ (bits >> 31 & 0x7fffffff);
    const int most_key = __reduce_max_sync(parts_of_own, key);
    const float most = __int_as_float(most_key ^ (most_key >> 31 & 0x7fffffff));
    s_weight[lane][head] = weight(m, most);
    s_most[lane][head] = most;
  }
  // of the row that a lane's part is of: whether the CTA has its first tile and its last
  const int run_starts = __shfl_sync(0xffffffffu, own.y, __ffs(parts_of_own) - 1) & 1;
  const int run_ends = __shfl_sync(0xffffffffu, own.y, 31 - __clz(parts_of_own)) & 2;
  const uint32_t leaders = __ballot_sync(0xffffffffu, own.x >= 0 && lane == __ffs(parts_of_own) - 1);
  if (warp == 0 && !p.row_each) {
    const uint32_t behind = __ballot_sync(0xffffffffu, own.x >= 0 && !run_starts), before = __ballot_sync(0xffffffffu, own.x >= 0 && run_starts && !run_ends);
    const int row0 = __shfl_sync(0xffffffffu, own.x, behind ? __ffs(behind) - 1 : 0), row1 = __shfl_sync(0xffffffffu, own.x, before ? __ffs(before) - 1 : 0);
    if (lane == 0) {
      p.headers[2 * blockIdx.x] = make_int4(behind ? row0 : -1, 0, 0, 0);
      p.headers[2 * blockIdx.x + 1] = make_int4(before ? row1 : -1, 0, 0, 0);
    }
  }
  __syncthreads();
  for (int task = warp; task < __popc(leaders) * kSlices; task += S::kWarps) {
    uint32_t from = leaders;
    for (int i = task / kSlices; i > 0; --i) from &= from - 1;
    const int leader = __ffs(from) - 1;
    const uint32_t parts = __shfl_sync(0xffffffffu, parts_of_own, leader);
    const int starts = __shfl_sync(0xffffffffu, run_starts, leader), ends = __shfl_sync(0xffffffffu, run_ends, leader);
    const int out_row = __shfl_sync(0xffffffffu, own.z, leader), heads = __shfl_sync(0xffffffffu, own.y, leader) >> 2;
    const int place = task % kSlices * 32 + lane, head = place * 4 % NH, d = place * 4 / NH;
    float4 total_p = make_float4(0.f, 0.f, 0.f, 0.f), sums = total_p;
    for (uint32_t of = parts; of;) {
      constexpr int kAtOnce = 2;               // parts at once; for one that is not there the leader is read, and counts as 0 (its sums may be infinite)
      const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
      float4 f[kAtOnce], t[kAtOnce], v[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const bool there = of != 0;
        const int i = there ? __ffs(of) - 1 : leader;
        of &= of - 1;
        f[u] = *reinterpret_cast<const float4*>(&s_weight[i][head]);
        t[u] = *reinterpret_cast<const float4*>(&s_total[i][head]);
        v[u] = part_of(i).four(place);
        if (!there) f[u] = v[u] = none;
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) total_p = total_p + f[u] * t[u], sums = sums + f[u] * v[u];
    }
    const float4 top = *reinterpret_cast<const float4*>(&s_most[leader][head]);
    if (starts && ends) {
      put_out<D>(p, out_row, heads, head, d, sums, top, total_p);
    } else {
      const Part<D, NH> part{p.parts + (2ll * blockIdx.x + (starts ? 1 : 0)) * S::kPart};
      part.four(place) = sums;
      if (d == 0) part.most4(head) = top, part.total4(head) = total_p;
    }
  }

  // ---- sequences that are not there have outputs all the same
  for (int i = 0, b = blockIdx.x; b < B; b += gridDim.x, ++i)
    if (i < 32 ? s_empty >> i & 1 : span_of(p, b).tiles() == 0) {
      for (int at = tid; at < p.n_heads * (D / 8); at += kThreads)
        reinterpret_cast<uint4*>(p.out)[(long long)b * p.n_heads * (D / 8) + at] = make_uint4(0, 0, 0, 0);
      if (p.lse)
        for (int at = tid; at < p.n_heads; at += kThreads) p.lse[(long long)b * p.n_heads + at] = kNegInf;
    }
}

// Joins the rows that cross CTAs.  CTAs (i, .) take the row that begins in CTA i of the kernel before and goes on in the next ones, CTA
// (i, j) 32 channels of four of its heads: a thread finds the weights of a part, then a lane sums a channel, the warps the parts in
// turn.  (One row of 16 heads over all CTAs: by one CTA 50 us.)
constexpr int kMaxCtas = 256;
template <int D, int NH>
__global__ void __launch_bounds__(kMaxCtas) attn_join_kernel(const AttnParams p, const int ctas) {
  constexpr int kPart = NH * (D + 2), kWarps = kMaxCtas / 32;
  __shared__ float4 s_weight[kMaxCtas], s_top[kWarps], s_total[kWarps], s_sums[kWarps][32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // The row's parts: the own one, then the first ones of the CTAs behind that have it too.  Thread i sees to part i + 1, the last thread (there are
  // fewer parts) to part 0.  What a warp sums first is asked for before it is known whether the row has it.
  const int4* const headers = ptx::behind_wait(p.headers);
  const int group = blockIdx.y % (NH / 4), d = blockIdx.y / (NH / 4) * 32 + lane, head = group * 4, place = d * (NH / 4) + group;
  auto part_of = [&](int i) { return Part<D, NH>{p.parts + (i == 0 ? 2ll * blockIdx.x + 1 : 2ll * (blockIdx.x + i)) * kPart}; };
  const int row = headers[2 * blockIdx.x + 1].x, c = blockIdx.x + 1 + tid;
  const int its_row = c < ctas ? headers[2 * c].x : -1;
  float4 sums = make_float4(0.f, 0.f, 0.f, 0.f), m = make_float4(kNegInf, kNegInf, kNegInf, kNegInf), total = sums;
  if ((int)blockIdx.x + warp < ctas) sums = part_of(warp).four(place);
  if (row < 0) return;
  const int own = tid == kMaxCtas - 1 ? 0 : tid + 1;
  if (own == 0 || its_row == row) m = part_of(own).most4(head), total = part_of(own).total4(head);
  const int n = 1 + __syncthreads_count(its_row == row);
  float4 top = m;
#pragma unroll
  for (int o = 16; o; o >>= 1) top = larger(top, shuffled(top, o));
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) top = larger(top, s_top[w]);
  const float4 f = make_float4(weight(m.x, top.x), weight(m.y, top.y), weight(m.z, top.z), weight(m.w, top.w));
  s_weight[own] = f;
  total = total * f;
#pragma unroll
  for (int o = 16; o; o >>= 1) total = total + shuffled(total, o);
  if (lane == 0) s_total[warp] = total;
  __syncthreads();
  sums = warp < n ? s_weight[warp] * sums : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = warp + kWarps; i < n; i += kWarps) sums = sums + s_weight[i] * part_of(i).four(place);
  s_sums[warp][lane] = sums;
  __syncthreads();
  if (warp > 0) return;
#pragma unroll
  for (int w = 1; w < kWarps; ++w) sums = sums + s_sums[w][lane];
  total = s_total[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) total = total + s_total[w];
  const int b = row / p.rows_of_seq;
  int heads;
  const int h0 = first_head<NH>(p, row - b * p.rows_of_seq, heads);
  put_out<D>(p, (long long)b * p.n_heads + h0, heads, head, d, sums, top, total);
}

int attn_ctas() { return min(sm_count_or(148), kMaxCtas); }

// Query heads of a row of work.
int heads_of_row(int group, int dim) { return group <= 4 ? 4 : group <= 8 || dim > 128 ? 8 : 16; }

// Keys or values [n_pages, page_size, n_kv_heads, D] in boxes of some tokens and a line of their channels.
template <typename S>
int tensor_map_of(const CacheView& c, const void* at, uint32_t tokens, CUtensorMap* map) {
  EncodeTiledFn encode = nullptr;
  PEQA_TRY(tensor_map_encoder(&encode));
  // (the stride of a dimension of one says nothing, and 0 is none)
  auto bytes = [](uint32_t stride16) { return stride16 ? (cuuint64_t)stride16 * 16 : (cuuint64_t)16; };
  const cuuint64_t dims[4] = {(cuuint64_t)S::D, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.page_size, (cuuint64_t)c.n_pages};
  const cuuint64_t strides[3] = {bytes(c.head16), bytes(c.token16), bytes(c.page16)};
  const cuuint32_t box[4] = {(cuuint32_t)(S::kLine / (S::I8 ? 1 : 2)), 1, tokens, 1}, steps[4] = {1, 1, 1, 1};
  if (encode(map, S::I8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(at), dims, strides, box, steps,
             CU_TENSOR_MAP_INTERLEAVE_NONE, S::kLine == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             // no more than a head has of a token: what lies beside it may be another head's
             S::kBytes >= 256 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B
                              : S::kBytes == 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_64B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cuda_fail(cudaErrorInvalidValue);
  return PEQA_OK;
}

template <int D, int NH, bool I8, bool WHOLE>
int launch(const AttnParams& p, cudaStream_t st) {
  using S = Shape<D, NH, I8, WHOLE>;
  static std::atomic<uint64_t> allowed{0};
  PEQA_TRY(allow_smem(attn_decode_kernel<S>, S::kSmem, allowed));
  const int ctas = attn_ctas();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.row_each ? p.cache.n_seqs * p.rows_of_seq : ctas, 1, 1);
  cfg.blockDim = dim3(S::kWarps * 32, 1, 1);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  CUtensorMap keys = {}, values = {}, keys8 = {}, values8 = {};
  if constexpr (WHOLE) {
    PEQA_TRY(tensor_map_of<S>(p.cache, p.cache.k, kTile, &keys));
    PEQA_TRY(tensor_map_of<S>(p.cache, p.cache.v, kTile, &values));
    if (p.halves) {
      PEQA_TRY(tensor_map_of<S>(p.cache, p.cache.k, kTile / 2, &keys8));
      PEQA_TRY(tensor_map_of<S>(p.cache, p.cache.v, kTile / 2, &values8));
    }
  }
  PEQA_CUDA(cudaLaunchKernelEx(&cfg, attn_decode_kernel<S>, p, keys, values, keys8, values8));
  if (p.row_each) return PEQA_OK;
  cfg.gridDim = dim3(ctas, NH * D / 128, 1);
  cfg.blockDim = dim3(kMaxCtas, 1, 1);
  cfg.dynamicSmemBytes = 0;
  PEQA_CUDA(cudaLaunchKernelEx(&cfg, attn_join_kernel<D, NH>, p, ctas));
  return PEQA_OK;
}

template <int D, int NH>
int launch_type(const AttnParams& p, bool codes, cudaStream_t st) {
  // Tensor copies take fewer instructions than copies token by token, which the clock feels where the power limit holds it: 64 sequences of up to
  // 8190 tokens in 8 bits 138 -> 123 us.  But lines of 128 bytes that lie apart come slower by them: 4 sequences of up to 32003, all
  // heads of a token together, 286 -> 355 us; 16 of up to 8000, heads of 64 channels in bf16, 134 -> 192 us.
  const bool whole = p.cache.page_size % kTile == 0 && (D * (codes ? 1 : 2) >= 256 || p.cache.token16 == D * (codes ? 1 : 2) / 16);
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
  return (size_t)attn_ctas() * (2 * sizeof(int4) + (2 * (size_t)(dim + 2) + (size_t)warps_of(dim, nh) * dim) * nh * sizeof(float));
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
  if (rows > 0x7fffffffll / (p.cache.capacity / kTile + 2) || (long long)c->n_seqs * n_heads > 0x7fffffffll) return PEQA_ERR_TOO_LARGE;
  p.rows_of_seq = (int)rows_of_seq;
  PEQA_TRY(check_arch());
  if (!workspace || bytes < workspace_bytes(c->head_dim, nh)) return PEQA_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return PEQA_ERR_ALIGNMENT;
  p.q = static_cast<const uint16_t*>(q->data);
  p.q_row = c->n_seqs > 1 ? q->row_stride : 0;
  p.q_head = n_heads > 1 ? q->head_stride : 0;
  p.seq_lens = seq_lens;
  p.n_heads = n_heads;
  // A CTA for every row needs no second kernel, but is as long as the longest row.  Rows of T tiles, rows x T: dealt out evenly / a CTA each, us:
  // 8 x 9 8.0 / 5.6, 8 x 16 7.9 / 6.9, 8 x 32 7.9 / 8.0, 8 x 64 8.4 / 9.9; 32 x 9 8.0 / 5.5, 32 x 32 8.2 / 7.5, 32 x 64 9.3 / 9.4; 128 x 9 8.5 / 5.6, 128 x
  // 64 16.1 / 12.5, 128 x 128 22.4 / 19.4 (four sequences of uneven lengths).  What is known here of the lengths is what they can be at most.
  const long long ctas = attn_ctas(), capacity = p.cache.capacity;
  const long long most = (min(capacity, window > 0 ? window + kTile - 1ll : capacity) + kTile - 1) / kTile;
  p.row_each = rows <= ctas && (most < 32 || (4 * rows >= ctas && most * (ctas - rows) <= 48 * ctas && most <= 129));
  // A row's last tile is half empty on average, which rows of few tiles feel: 256 sequences of up to 16 tokens, 32 heads, 19.8 -> 18.6 us, of up to 50
  // 40.7 -> 39.0, of up to 513 219.4 -> 217.6.  (8 bits: by the registers that it takes 64 of up to 300 16.9 -> 17.9.)
  p.halves = c->type == PEQA_KV_BF16 && !p.row_each && most <= 64;
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

// The paged 8-bit cache but for its attention (gfx950): storing, the index, copies, tables.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "eta_device.h"
#include "eta_lanes.h"
#include "eta_page.h"
#include "eta_page_codes.h"

namespace eta {
namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef int64_t i64x2_t __attribute__((ext_vector_type(2)));

// the largest value over the wavefront, in every lane
__device__ __forceinline__ float wave_max64(float x) {
  auto over = [&](uint32_t y) { x = fmaxf(x, __uint_as_float(y)); };
  over(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0xB1, 0xf, 0xf, false));    // quad_perm [1,0,3,2]
  over(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x4E, 0xf, 0xf, false));    // quad_perm [2,3,0,1]
  over(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x141, 0xf, 0xf, false));   // row_half_mirror
  over(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x140, 0xf, 0xf, false));   // row_mirror
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// ---------------------------------------------------------------- storing
//
// A page's scale is a power of two, so that a page whose scale grows, as tokens come one by one,
// keeps its codes' values: E4M3 has as many fraction bits at every exponent, so only codes that
// fall below 2^-6 of the new scale are rounded again, and x / scale is exact.  (A scale of
// amax / 448 would round every code again at each growth, for less than one bit of range.)

// Exponent e of the least 2^e with amax <= 448 * 2^e (448 = 1.75 * 2^8), at least -126.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < -126 ? -126 : e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// |x|, or 0 where x is NaN or infinite
__device__ __forceinline__ float finite_abs(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? __uint_as_float(u) : 0.f;
}

// x / scale as it is coded: infinities become NaN (the conversion rounds to nearest, ties to
// even, and |x| / scale never passes 448)
__device__ __forceinline__ float coded(float x, float inv) {
  return (__float_as_uint(x) & 0x7fffffffu) == 0x7f800000u ? __builtin_nanf("") : x * inv;
}

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// A page may hold any scale (one coded elsewhere by amax / 448).  With one that is no power of two a
// quotient x / scale, or a product of a code and the ratio of two scales, can round to the middle between
// two codes that it only lies next to, and the tie would go to the wrong one.  So both are rounded to odd:
// y, the nearest to the exact value, with the sign of what that leaves in `rest`, becomes the one of its
// two neighbours in 32 bits whose last bit is set, which rounds to a code as the exact value does.
__device__ __forceinline__ float to_odd(float y, float rest) {
  if (!(rest < 0.f || rest > 0.f)) return y;         // (exact, or not finite)
  const uint32_t u = __float_as_uint(y), beyond = (u ^ __float_as_uint(rest)) >> 31;
  return __uint_as_float((u - beyond) | 1u);
}
// x / scale for a scale that is no power of two, as it is coded.  (`up` keeps the rest above the least float.)
__device__ __forceinline__ float quotient(float x, float scale) {
  const float up = scale < 0x1p-60f ? 0x1p64f : 1.0f, y = (x * up) / (scale * up);
  return to_odd(y, fmaf(-y, scale * up, x * up));
}
__device__ __forceinline__ bool is_power_of_two(float s) { return (__float_as_uint(s) & 0x7fffffu) == 0; }

// the codes of a word times r, rounded again
__device__ __forceinline__ uint32_t scaled4(uint32_t w, float r) {
  const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  auto times = [r](float c) {
    const float y = c * r;
    return to_odd(y, fmaf(c, r, -y));
  };
  return pack4(times(lo[0]), times(lo[1]), times(hi[0]), times(hi[1]));
}

// Eight elements of a row in 32 bits.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = __builtin_bit_cast(float4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p))), b = __builtin_bit_cast(float4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p) + 1));
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    const uint4 a = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}

struct StoreArgs {
  uint8_t* code[2];              // k, v
  float* scale[2];
  const void* rows[2];
  int64_t sb[2], sh[2], st[2];
  const int32_t* table;
  const int32_t* start;
  const int32_t* new_lens;
  PageGeom pg;
  int new_tokens;
};

// New tokens [first, end) of a sequence, in positions.
__device__ __forceinline__ void new_span(const StoreArgs& a, int b, int64_t* first, int64_t* end) {
  int64_t s = a.start != nullptr ? a.start[b] : 0;
  int64_t n = a.new_lens != nullptr ? a.new_lens[b] : a.new_tokens;
  s = s < 0 ? 0 : s;
  n = n < 0 ? 0 : (n > a.new_tokens ? a.new_tokens : n);
  *first = s;
  *end = s + n;
}

// One workgroup for a page and head of K or of V (blockIdx.x even, odd).  A thread holds 8 dims
// of 4 consecutive tokens, so that V's transposed codes form whole words of 4 tokens, which go
// through LDS to rows of the page.  Bound by HBM: 16K tokens, 8 kv heads, d = 128, bf16: 100.7 MB in
// 19.0 us.  Rows and codes go past the caches (us through them / rows past / both past: 22.6, 21.6,
// 19.6; 4 x 16K 59.5, 51.6, 51.8; with the index read behind it 30.2 rows past, 29.9 both).
template <int D, int BS, typename T>
__global__ __launch_bounds__(D / 8 * (BS / 4)) void page_store_kernel(StoreArgs a) {
  constexpr int TPR = D / 8, NT = TPR * (BS / 4), NW = NT / 64;
  __shared__ float red_s[NW];
  __shared__ uint32_t v_s[D][BS / 4 + 1];
  const int kv = blockIdx.x & 1, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int c = tid % TPR, q4 = tid / TPR;            // dims 8 c .., tokens 4 q4 .. of the page
  int64_t first, end;
  new_span(a, b, &first, &end);
  const int64_t j = first / BS + (blockIdx.x >> 1), base = j * BS;
  const int64_t lo64 = first > base ? first - base : 0, hi64 = end - base < BS ? end - base : BS;
  if (hi64 <= lo64) return;
  const int lo = (int)lo64, hi = (int)hi64;
  const int64_t page = page_of(a.table + (int64_t)b * a.pg.table_stride, j, a.pg.table_blocks, a.pg.pages);
  if (page < 0) return;
  const int64_t si = page * a.pg.scale_stride + h;
  const float held = a.scale[kv][si];
  const T* src = reinterpret_cast<const T*>(a.rows[kv]) + b * a.sb[kv] + h * a.sh[kv];
  uint8_t* dst = a.code[kv] + page * a.pg.page_stride + (int64_t)h * BS * D;
  float x[4][8], amax = 0.f;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = 4 * q4 + r;
    const int64_t i = (t >= lo && t < hi ? t : lo) + base - first;      // (others read a new row too)
    load8<T>(src + i * a.st[kv] + 8 * c, x[r]);
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, finite_abs(x[r][e]));
  }
  amax = wave_max64(amax);
  if ((tid & 63) == 0) red_s[tid >> 6] = amax;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NW; ++k) amax = fmaxf(amax, red_s[k]);
  const int e2 = scale_exponent(amax);
  const float need = power_of_two(e2);
  // (a scale held that is no power of two, or NaN, is kept where it is not less)
  const bool grows = lo == 0 || need > held;
  const float scale = grows ? need : held;
  float inv = grows ? power_of_two(-e2) : 1.0f / held;
  const float again = held / scale;
  if (!grows && !is_power_of_two(held)) {            // (the whole workgroup)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[r][e] = quotient(x[r][e], held);
    inv = 1.0f;
  }
  const bool round_held = lo > 0 && grows;
  if (tid == 0 && grows) a.scale[kv][si] = scale;
  if (kv == 0) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = 4 * q4 + r;
      uint2* p = reinterpret_cast<uint2*>(dst + t * D + 8 * c);
      if (t >= lo && t < hi) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = coded(x[r][e], inv);
        __builtin_nontemporal_store((uint64_t)pack4(y[0], y[1], y[2], y[3]) | (uint64_t)pack4(y[4], y[5], y[6], y[7]) << 32, reinterpret_cast<uint64_t*>(p));
      } else if (t < lo && round_held) {
        const uint2 w = *p;
        *p = make_uint2(scaled4(w.x, again), scaled4(w.y, again));
      }
    }
    return;
  }
  const int t0 = 4 * q4;
  const bool whole = t0 >= lo && t0 + 4 <= hi;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint32_t w = pack4(coded(x[0][e], inv), coded(x[1][e], inv), coded(x[2][e], inv), coded(x[3][e], inv));
    if (!whole) {
      const uint32_t old = *reinterpret_cast<const uint32_t*>(dst + (8 * c + e) * BS + t0);
      const uint32_t rounded = round_held ? scaled4(old, again) : old;
      uint32_t m = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t byte = 0xffu << (8 * r);
        m |= (t0 + r < lo ? rounded : (t0 + r < hi ? w : old)) & byte;
      }
      w = m;
    }
    v_s[8 * c + e][q4] = w;
  }
  __syncthreads();
  constexpr int WPR = BS / 16;                        // 16-byte pieces of a row of V
  for (int k = tid; k < D * WPR; k += NT) {
    const int d = k / WPR, p = k % WPR;
    const uint32_t* s = &v_s[d][4 * p];
    __builtin_nontemporal_store(u32x4_t{s[0], s[1], s[2], s[3]}, reinterpret_cast<u32x4_t*>(dst + d * BS + 16 * p));
  }
}

// One token of each sequence: one workgroup for a head of K or of V, every wavefront with the
// token's row (a lane D / 64 of its values), so that its scale needs no exchange.  Where the page's
// scale grows, the workgroup rounds the codes held again; else it writes the row.  All latency:
// three round trips (start, table and row, scale).  32 sequences, 8 kv heads, d = 128: 3.6 us, 7.2
// with the kernel above.
template <int D, int BS, typename T>
__global__ __launch_bounds__(256) void page_token_kernel(StoreArgs a) {
  constexpr int PL = D / 64;
  const int kv = blockIdx.x & 1, h = blockIdx.x >> 1, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const T* src = reinterpret_cast<const T*>(a.rows[kv]) + b * a.sb[kv] + h * a.sh[kv] + lane * PL;
  float x[PL];
#pragma unroll
  for (int e = 0; e < PL; ++e) {
    if constexpr (sizeof(T) == 4)
      x[e] = src[e];
    else
      x[e] = __uint_as_float((uint32_t)src[e] << 16);
  }
  int64_t first, end;
  new_span(a, b, &first, &end);
  if (end <= first) return;
  const int64_t j = first / BS, page = page_of(a.table + (int64_t)b * a.pg.table_stride, j, a.pg.table_blocks, a.pg.pages);
  if (page < 0) return;
  const int lo = (int)(first - j * BS);
  const int64_t si = page * a.pg.scale_stride + h;
  const float held = a.scale[kv][si];
  uint8_t* dst = a.code[kv] + page * a.pg.page_stride + (int64_t)h * BS * D;
  float amax = 0.f;
#pragma unroll
  for (int e = 0; e < PL; ++e) amax = fmaxf(amax, finite_abs(x[e]));
  const int e2 = scale_exponent(wave_max64(amax));
  const float need = power_of_two(e2);
  const bool grows = lo == 0 || need > held;
  float inv = grows ? power_of_two(-e2) : 1.0f / held;
  if (!grows && !is_power_of_two(held)) {
#pragma unroll
    for (int e = 0; e < PL; ++e) x[e] = quotient(x[e], held);
    inv = 1.0f;
  }
  if (lo > 0 && grows) {
    const float again = held / need;
    for (int k = tid; k < BS * D / 16; k += 256) {
      uint4* p = reinterpret_cast<uint4*>(dst) + k;
      if (kv == 0) {
        if (k >= lo * (D / 16)) break;
        uint4 w = *p;
        *p = make_uint4(scaled4(w.x, again), scaled4(w.y, again), scaled4(w.z, again), scaled4(w.w, again));
      } else {
        const int t0 = 16 * (k % (BS / 16));         // tokens t0 .. of a dimension
        if (t0 >= lo) continue;
        const uint4 v = *p;
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int nv = lo - t0 - 4 * i;              // tokens of the word that are held
          const uint32_t m = nv >= 4 ? ~0u : (nv <= 0 ? 0u : (1u << (8 * nv)) - 1u);
          w[i] = (scaled4(w[i], again) & m) | (w[i] & ~m);
        }
        *p = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    // (the words of V rounded again hold the new token's place)
    __threadfence_block();
    __syncthreads();
  }
  if (tid >= 64) return;
  if (grows && lane == 0) a.scale[kv][si] = need;
  const uint32_t w = pack4(coded(x[0], inv), coded(x[PL - 1], inv), 0.f, 0.f);
  if (kv == 0) {
    if constexpr (PL == 2)
      reinterpret_cast<uint16_t*>(dst + lo * D)[lane] = (uint16_t)w;
    else
      dst[lo * D + lane] = (uint8_t)w;
  } else {
#pragma unroll
    for (int e = 0; e < PL; ++e) dst[(lane * PL + e) * BS + lo] = (uint8_t)(w >> (8 * e));
  }
}

// ---------------------------------------------------------------- the index
//
// mu = s m, sigma = s sqrt(mean((c - m)^2)), M = s max |c_t| over the codes c of a block, m their
// mean and s the page's scale.  A byte read would cost the vector unit five operations (widen
// twice, add, subtract, square, and the row's norm), about what it can do in the time HBM takes
// for it; the matrix cores take all but the square.  A tile of 16 tokens x 32 dims of codes, as
// it is loaded, is the A operand of
//   A I     against columns of the unit matrix: the codes widened, each 16 dims a result whose
//           rows are the tile's tokens; added up over the tiles in the accumulator (the sums are
//           exact: codes are multiples of 2^-9), and in the second pass, with -m as the
//           accumulator's start, the deviations;
//   A A^T   the tokens' products, whose diagonal has the squared norms: of rows of 64 dims no
//           element is larger than the largest of them, so nothing looks for it; the two parts
//           of rows of 128 are added.  (With the codes widened to bf16: sums of 8-bit products
//           come back 5e-6 off, of bf16 ones 3e-8.)
// The block stays in registers for both passes (two passes: mean first, so that a coordinate
// whose mean is far larger than its spread loses nothing).  A lane's squares go to two sums in turn
// (blocks of 128 x 128: deviations 7.1e-8 off; one sum of 64 squares 1.2e-7 at the same time, four 4.6e-8 at
// 2% more for 8 x 16K tokens).  Results are staged in LDS and leave
// as rows of the dimension-major records.  (NaN times a zero of the unit matrix is NaN: a key with
// NaN makes the means and deviations of the 32 dims of its step NaN too, and may leave the norms of
// other tokens out; the block's bound is NaN with one of them.)

struct IndexArgs {
  const uint8_t* k;
  const float* k_scale;
  const int32_t* table;
  const int32_t* prev_lens;
  const int32_t* seq_lens;
  void* mu;
  void* sigma;
  float* mx;
  PageGeom pg;
  int max_new;
  unsigned run, runs, rounds;    // neighbours of a run, runs of a (sequence, kv head), rounds along x
};

// fp32 -> E4M3, nearest even, saturating at 448; NaN stays
__device__ __forceinline__ uint8_t to_record8(float f) {
  const float a = fabsf(f) > 448.0f ? copysignf(448.0f, f) : f;
  return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, a, 0, false);
}

template <int D, int BS, int NB, bool STREAM>
__global__ __launch_bounds__(256, 2) void page_summaries_kernel(IndexArgs a) {
  constexpr int HALF = D / 64, RT = 16 / HALF;         // parts of a row, tokens of a load
  constexpr int NL = BS / RT;                          // loads of a block
  __shared__ float mu_s[D][NB + 1];
  __shared__ float sg_s[D][NB + 1];
  __shared__ float mx_s[NB];
  __shared__ bool there_s[NB];
  const Geom& g = a.pg.g;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int col = lane & 15, g4 = lane >> 4;
  // Workgroups go to the XCDs round robin.  Each XCD takes runs of neighbours, whose records share
  // cache lines (at most eight runs of a sequence and head; 130K tokens 38.5 us in eight, 40.8 in
  // 64), and the runs of all sequences and heads are dealt to the XCDs in turn (with every one's
  // first run on the first XCD, short ones left the others idle: 64 times 9 blocks of 128 tokens
  // 11.2 us, so 8.1; one block each of 128 heads 7.3, 5.0).
  const unsigned i8 = blockIdx.x >> 3, r = (i8 / a.run + blockIdx.y * a.rounds) * 8 + (blockIdx.x & 7);
  const unsigned bh = r / a.runs, at = r % a.runs * a.run + i8 % a.run;
  if (bh >= (unsigned)(g.B * g.Hkv)) return;
  const int b = bh / g.Hkv, h = bh % g.Hkv;
  int64_t N = clamp_len(a.seq_lens, b, g.cap) / BS, j0 = (int64_t)at * NB;
  if (N > g.ncap) N = g.ncap;
  if (a.prev_lens != nullptr) {
    const int64_t first = clamp_len(a.prev_lens, b, g.cap) / BS;
    j0 += first;
    if (N > first + a.max_new) N = first + a.max_new;
  }
  if (j0 >= N) return;
  // columns 16 u .. of the unit matrix of a step's 32 dims: this lane's rows are 8 g4 .. + 7
  int64_t unit[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = 16 * u + col - 8 * g4;
    unit[u] = i >= 0 && i < 8 ? (int64_t)0x38 << (8 * i) : 0;      // 0x38: 1.0
  }
  // 1 where register r of a 16 x 16 result is the lane's element of the diagonal
  float diag[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) diag[r] = col == 4 * g4 + r ? 1.0f : 0.f;
  const int32_t* row = a.table + (int64_t)b * a.pg.table_stride;
  // Block jj of this workgroup; its loads (row i of the A operand: token i % RT, part i / RT of
  // its row, so that a load covers whole rows) are in flight while the wavefront's block before
  // it is worked on.  Returns whether it is there.
  float scale_n = 0.f;
  i64x2_t x[NL], xn[NL];
  auto load = [&](int jj) {
    const int64_t j = j0 + jj;
    if (jj >= NB || j >= N) return false;
    const int64_t page = page_of(row, j, a.pg.table_blocks, a.pg.pages);
    if (lane == 0) there_s[jj] = page >= 0;
    const int64_t from = page < 0 ? 0 : page;          // (no page: another is read and not recorded)
    const uint8_t* p = a.k + from * a.pg.page_stride + (int64_t)h * BS * D + (col % RT) * D + (col / RT) * 64 + 16 * g4;
    scale_n = a.k_scale[from * a.pg.scale_stride + h];
#pragma unroll
    for (int t = 0; t < NL; ++t) {
      const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p + t * RT * D);
      xn[t] = __builtin_bit_cast(i64x2_t, STREAM ? __builtin_nontemporal_load(q) : *q);
    }
    return true;
  };
  bool more = load(w);
  for (int jj = w; more; jj += 4) {
    const float scale = scale_n;
#pragma unroll
    for (int t = 0; t < NL; ++t) x[t] = xn[t];
    more = NB > 4 && load(jj + 4);
    __builtin_amdgcn_sched_barrier(0);
    float n2 = 0.f;
#pragma unroll
    for (int t = 0; t < NL; ++t) {
      f32x4 aa = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const bf16x8 wide = widen((uint32_t)x[t][e], (uint32_t)(x[t][e] >> 32));
        aa = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide, wide, aa, 0, 0, 0);
      }
      if constexpr (HALF == 1) {
#pragma unroll
        for (int r = 0; r < 4; ++r) n2 = fmaxf(n2, aa[r]);
      } else {
        // the diagonal's element of a token's first part is in lane (token, row token / 4), that
        // of its second in (8 + token, row 2 + token / 4); every other lane has 0
        float y = aa[0] * diag[0];
#pragma unroll
        for (int r = 1; r < 4; ++r) y = fmaf(aa[r], diag[r], y);
        y = dpp_add<0x128>(y);                         // row_ror:8
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
        n2 = fmaxf(n2, __uint_as_float(r[0]) + __uint_as_float(r[1]));
      }
    }
    // the sum over the lanes of a column that hold the same part of a row, in each of them
    auto column_sum = [](float y) {
      auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
      y = __uint_as_float(r[0]) + __uint_as_float(r[1]);
      if constexpr (HALF == 1) {
        r = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
        y = __uint_as_float(r[0]) + __uint_as_float(r[1]);
      }
      return y;
    };
    // step e, columns u: dim 16 (2 u + col / 8) + 8 e + col % 8 of the lane's part
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      __builtin_amdgcn_sched_barrier(0);               // (32 dims at a time: few registers)
      f32x4 y[2], from[2];
      f32x2_t v[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) y[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NL; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) y[u] = __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(x[t][e], unit[u], y[u], 0, 0, 0);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float mean = column_sum((y[u][0] + y[u][1]) + (y[u][2] + y[u][3])) * (1.0f / BS);
        from[u] = f32x4{-mean, -mean, -mean, -mean};
        v[u] = f32x2_t{0.f, 0.f};
      }
#pragma unroll
      for (int t = 0; t < NL; ++t)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const f32x4 d = __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(x[t][e], unit[u], from[u], 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) v[u][r & 1] = fmaf(d[r], d[r], v[u][r & 1]);
        }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float sd = sqrtf(column_sum(v[u][0] + v[u][1]) * (1.0f / BS));
        if (HALF == 1 ? g4 == 0 : (g4 & 1) == 0) {
          const int i = 64 * (g4 >> 1) + 16 * (2 * u + (col >> 3)) + 8 * e + (col & 7);
          mu_s[i][jj] = -from[u][0] * scale;
          sg_s[i][jj] = sd * scale;
        }
      }
    }
    n2 = wave_max64(n2);
    if (lane == 0) mx_s[jj] = sqrtf(n2) * scale;
  }
  __syncthreads();
  const int nv = N - j0 < NB ? (int)(N - j0) : NB;
  const int64_t bg = (int64_t)b * g.Hkv + h, ob = bg * D * g.ncap + j0;
  for (int idx = tid; idx < D * NB; idx += 256) {
    const int i = idx / NB, jj = idx % NB;
    if (jj >= nv || !there_s[jj]) continue;
    const int64_t o = ob + (int64_t)i * g.ncap + jj;
    if (g.stat_dtype == ETA_DT_F16) {
      reinterpret_cast<_Float16*>(a.mu)[o] = (_Float16)mu_s[i][jj];
      reinterpret_cast<_Float16*>(a.sigma)[o] = (_Float16)sg_s[i][jj];
    } else if (g.stat_dtype == ETA_DT_FP8) {
      reinterpret_cast<uint8_t*>(a.mu)[o] = to_record8(mu_s[i][jj]);
      reinterpret_cast<uint8_t*>(a.sigma)[o] = to_record8(sg_s[i][jj]);
    } else {
      reinterpret_cast<float*>(a.mu)[o] = mu_s[i][jj];
      reinterpret_cast<float*>(a.sigma)[o] = sg_s[i][jj];
    }
  }
  if (tid < nv && there_s[tid]) a.mx[bg * g.ncap + j0 + tid] = mx_s[tid];
}

// ---------------------------------------------------------------- copies

// One workgroup for a pair, a head, and K or V: b d codes (N x 256 x 16) and their scale.  Past
// the caches when read (a copied page is not read next; 1200 pages of 256 KB: 37 us through them, 30
// past them; written past them too: 33).
template <int N>
__global__ __launch_bounds__(256) void page_copy_kernel(eta_page_pool_t pool, PageGeom pg, const int32_t* src,
                                                        const int32_t* dst, int64_t n) {
  const int h = blockIdx.y >> 1;
  const bool isv = blockIdx.y & 1;
  uint8_t* code = reinterpret_cast<uint8_t*>(isv ? pool.v : pool.k) + (int64_t)h * (N * 4096) + threadIdx.x * 16;
  float* scale = (isv ? pool.v_scale : pool.k_scale) + h;
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const int64_t a = src[i], b = dst[i];
    if (a < 0 || a >= pg.pages || b < 0 || b >= pg.pages) continue;
    const u32x4_t* from = reinterpret_cast<const u32x4_t*>(code + a * pg.page_stride);
    u32x4_t* to = reinterpret_cast<u32x4_t*>(code + b * pg.page_stride);
    u32x4_t x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = __builtin_nontemporal_load(from + 256 * k);
#pragma unroll
    for (int k = 0; k < N; ++k) to[256 * k] = x[k];
    if (threadIdx.x == 0) scale[b * pg.scale_stride] = scale[a * pg.scale_stride];
  }
}

// ---------------------------------------------------------------- tables
//
// Integer bookkeeping of a few hundred kilobytes at most: what counts is the number of launches
// and of round trips (a fork of 32 rows in one launch 7.5 us, in three 1.6 + 3.2 + 4.0 and two more
// launches, which the host takes 4 us each for).  Work over the table's entries is spread over the card; what has to know
// the order of the free pages runs in one workgroup, which reads refs 4096 pages at a time.

constexpr int kTableThreads = 1024;
// Entries and counts up to which one workgroup goes over the table too: a launch less.
constexpr int64_t kOneWorkgroup = 16384;

// Exclusive prefix over the workgroup's kTableThreads threads; *total gets the sum.
__device__ __forceinline__ int wide_excl_scan(int x, int* wsum, int* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int incl = wave_incl_scan(x);
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  int off = 0, tot = 0;
#pragma unroll
  for (int k = 0; k < kTableThreads / 64; ++k) {
    off += k < w ? wsum[k] : 0;
    tot += wsum[k];
  }
  __syncthreads();
  *total = tot;
  return off + incl - x;
}

// Calls f(rank, page) for the pages that `in` holds for, ranks ascending with the pages' numbers
// from `rank` on, until `most` are found.  Returns the rank after the last.  Every thread of the
// workgroup takes part.
template <typename In, typename F>
__device__ __forceinline__ int64_t ranked(int64_t pages, int64_t most, int* wsum, In in, F f) {
  int64_t rank = 0;
  for (int64_t base = 0; base < pages && rank < most; base += 4 * kTableThreads) {
    bool is[4];
    int cnt = 0, tot;
    const int64_t p0 = base + 4 * threadIdx.x;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      is[e] = p0 + e < pages && in(p0 + e);
      cnt += is[e];
    }
    int64_t r = rank + wide_excl_scan(cnt, wsum, &tot);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (is[e]) {
        if (r < most) f(r, p0 + e);
        ++r;
      }
    rank += tot;
  }
  return rank;
}

__device__ __forceinline__ int64_t blocks_of(const eta_table_desc_t& td, int64_t len, int64_t* full) {
  const int64_t cap = td.table_blocks * td.block_size;
  len = len < 0 ? 0 : (len > cap ? cap : len);
  *full = len / td.block_size;
  return (len + td.block_size - 1) / td.block_size;
}

// The pages that each row lacks.
__global__ __launch_bounds__(256) void extend_count_kernel(eta_table_desc_t td, const int32_t* table,
                                                           const int32_t* seq_lens, int32_t* need) {
  __shared__ int red[4];
  const int b = blockIdx.x, tid = threadIdx.x;
  int64_t full;
  const int64_t nb = blocks_of(td, seq_lens[b], &full);
  int cnt = 0;
  for (int64_t j = tid; j < nb; j += 256) cnt += table[b * td.table_stride + j] < 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) cnt += __shfl_xor(cnt, o, 64);
  if ((tid & 63) == 0) red[tid >> 6] = cnt;
  __syncthreads();
  if (tid == 0) need[b] = red[0] + red[1] + red[2] + red[3];
}

// Free pages in order (free_list), then row by row the entries that lack one.
__global__ __launch_bounds__(kTableThreads) void extend_kernel(eta_table_desc_t td, int32_t* table, int32_t* refs,
                                                               const int32_t* seq_lens, int32_t* missing,
                                                               int32_t* need, int32_t* free_list) {
  __shared__ int wsum[kTableThreads / 64];
  const int tid = threadIdx.x;
  int64_t want = 0;
  for (int base = 0; base < td.batch; base += kTableThreads) {
    int tot;
    const int x = base + tid < td.batch ? need[base + tid] : 0;
    const int ex = wide_excl_scan(x, wsum, &tot);
    // (a row that lacks none is marked, the others get the rank of their first new page)
    if (base + tid < td.batch) need[base + tid] = x == 0 ? -1 : (int)(want + ex);
    want += tot;
  }
  const int64_t found = ranked(td.num_pages, want, wsum, [&](int64_t p) { return refs[p] <= 0; },
                               [&](int64_t r, int64_t p) { free_list[r] = (int32_t)p; });
  const int64_t have = found < want ? found : want;
  if (tid == 0) missing[0] = (int32_t)(want - have);
  __threadfence_block();
  __syncthreads();
  // a wavefront takes a row, 64 entries at a time
  for (int b = tid >> 6; b < td.batch; b += kTableThreads / 64) {
    int64_t r = need[b], full;
    if (r < 0) continue;
    const int64_t nb = blocks_of(td, seq_lens[b], &full);
    for (int64_t j0 = 0; j0 < nb; j0 += 64) {
      const int64_t j = j0 + (tid & 63);
      const bool lacks = j < nb && table[b * td.table_stride + j] < 0;
      const unsigned long long bal = __ballot(lacks);
      const int64_t k = r + __popcll(bal & ((1ull << (tid & 63)) - 1ull));
      if (lacks && k < have) {
        const int32_t p = free_list[k];
        table[b * td.table_stride + j] = p;
        refs[p] = 1;
      }
      r += __popcll(bal);
    }
  }
}

__global__ __launch_bounds__(256) void fork_init_kernel(eta_table_desc_t td, const int32_t* refs, int32_t* refs_out) {
  const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (p < td.num_pages) refs_out[p] = refs[p];
}

// Rows of the new table and the counts' changes; need[b]: the page to copy for the row, or -1.
__global__ __launch_bounds__(256) void fork_rows_kernel(eta_table_desc_t td, const int32_t* table,
                                                        const int32_t* seq_lens, const int32_t* parents,
                                                        int32_t* table_out, int32_t* refs_out,
                                                        int32_t* seq_lens_out, int32_t* need) {
  const int b = blockIdx.y, tid = threadIdx.x;
  const int64_t j = (int64_t)blockIdx.x * 256 + tid;
  const int a = parents[b];
  const bool is = a >= 0 && a < td.batch;
  const int64_t len = is ? seq_lens[a] : 0;
  int64_t full;
  const int64_t nb = blocks_of(td, len, &full);
  __shared__ int earlier_s;
  if (tid == 0) earlier_s = 0;
  __syncthreads();
  if (is && full < nb) {             // whether an earlier row takes the last block already
    for (int o = tid; o < b; o += 256)
      if (parents[o] == a) earlier_s = 1;
  }
  __syncthreads();
  const bool copies = full < nb && earlier_s != 0;
  if (blockIdx.x == 0 && tid == 0) {
    const int64_t cap = td.table_blocks * td.block_size;
    seq_lens_out[b] = (int32_t)(len < 0 ? 0 : (len > cap ? cap : len));
    const int32_t p = copies ? table[a * td.table_stride + full] : -1;
    need[b] = p >= 0 && p < td.num_pages ? p : -1;
  }
  if (j >= td.table_blocks) return;
  const int32_t old = table[b * td.table_stride + j];
  int32_t now = is && j < nb && !(copies && j == full) ? table[a * td.table_stride + j] : -1;
  if (now < 0 || now >= td.num_pages) now = -1;
  table_out[b * td.table_stride + j] = now;
  if (old != now) {
    if (old >= 0 && old < td.num_pages) atomicSub(refs_out + old, 1);
    if (now >= 0) atomicAdd(refs_out + now, 1);
  }
}

// Gives the rows that copy a page their new one (one workgroup).
__device__ __forceinline__ void fork_pages(const eta_table_desc_t& td, const int32_t* seq_lens_out, int32_t* table_out,
                                           int32_t* refs_out, int32_t* src, int32_t* dst, int32_t* missing,
                                           const int32_t* need, int32_t* free_list, int* wsum) {
  const int tid = threadIdx.x;
  int64_t want = 0;
  for (int base = 0; base < td.batch; base += kTableThreads) {
    int tot;
    wide_excl_scan(base + tid < td.batch && need[base + tid] >= 0, wsum, &tot);
    want += tot;
  }
  const int64_t found = ranked(td.num_pages, want, wsum, [&](int64_t p) {
                                 // (atomics changed the counts past this compute unit's cache)
                                 return __hip_atomic_load(refs_out + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) <= 0;
                               },
                               [&](int64_t r, int64_t p) { free_list[r] = (int32_t)p; });
  const int64_t have = found < want ? found : want;
  if (tid == 0) missing[0] = (int32_t)(want - have);
  __threadfence_block();
  __syncthreads();
  int64_t rank = 0;
  for (int base = 0; base < td.batch; base += kTableThreads) {
    const int b = base + tid;
    const int32_t from = b < td.batch ? need[b] : -1;
    int tot;
    const int64_t r = rank + wide_excl_scan(from >= 0, wsum, &tot);
    if (b < td.batch) {
      const bool got = from >= 0 && r < have;
      const int32_t p = got ? free_list[r] : -1;
      src[b] = got ? from : -1;
      dst[b] = p;
      if (got) {
        int64_t full;
        blocks_of(td, seq_lens_out[b], &full);
        table_out[b * td.table_stride + full] = p;
        refs_out[p] = 1;
      }
    }
    rank += tot;
  }
}

__global__ __launch_bounds__(kTableThreads) void fork_pages_kernel(eta_table_desc_t td, const int32_t* seq_lens_out,
                                                                   int32_t* table_out, int32_t* refs_out, int32_t* src,
                                                                   int32_t* dst, int32_t* missing,
                                                                   const int32_t* need, int32_t* free_list) {
  __shared__ int wsum[kTableThreads / 64];
  fork_pages(td, seq_lens_out, table_out, refs_out, src, dst, missing, need, free_list, wsum);
}

// The whole of it in one workgroup, for tables of at most kTableThreads rows and few entries.
__global__ __launch_bounds__(kTableThreads) void fork_kernel(eta_table_desc_t td, const int32_t* table,
                                                             const int32_t* refs, const int32_t* seq_lens,
                                                             const int32_t* parents, int32_t* table_out,
                                                             int32_t* refs_out, int32_t* seq_lens_out, int32_t* src,
                                                             int32_t* dst, int32_t* missing, int32_t* need,
                                                             int32_t* free_list) {
  __shared__ int wsum[kTableThreads / 64];
  __shared__ int parent_s[kTableThreads], blocks_s[kTableThreads], copy_s[kTableThreads];
  const int tid = threadIdx.x;
  int a = -1;
  int64_t full = 0, nb = 0;
  if (tid < td.batch) {
    a = parents[tid];
    if (a < 0 || a >= td.batch) a = -1;
    const int64_t cap = td.table_blocks * td.block_size;
    int64_t len = a >= 0 ? seq_lens[a] : 0;
    len = len < 0 ? 0 : (len > cap ? cap : len);
    nb = blocks_of(td, len, &full);
    seq_lens_out[tid] = (int32_t)len;
    parent_s[tid] = a;
    blocks_s[tid] = (int)nb;
  }
  for (int64_t p = tid; p < td.num_pages; p += kTableThreads) refs_out[p] = refs[p];
  __threadfence_block();
  __syncthreads();
  if (tid < td.batch) {
    bool copies = false;
    if (full < nb)                   // whether an earlier row takes the last block already
      for (int o = 0; o < tid; ++o) copies |= parent_s[o] == a;
    copy_s[tid] = copies ? (int)full : -1;
    const int32_t p = copies ? table[a * td.table_stride + full] : -1;
    need[tid] = p >= 0 && p < td.num_pages ? p : -1;
  }
  __threadfence_block();
  __syncthreads();
  const int64_t entries = td.batch * td.table_blocks;
  for (int64_t e = tid; e < entries; e += kTableThreads) {
    const int b = (int)((uint32_t)e / (uint32_t)td.table_blocks);
    const int64_t j = e - b * td.table_blocks;
    const int32_t old = table[b * td.table_stride + j];
    int32_t now = j < blocks_s[b] && j != copy_s[b] ? table[parent_s[b] * td.table_stride + j] : -1;
    if (now < 0 || now >= td.num_pages) now = -1;
    table_out[b * td.table_stride + j] = now;
    if (old != now) {
      if (old >= 0 && old < td.num_pages) atomicSub(refs_out + old, 1);
      if (now >= 0) atomicAdd(refs_out + now, 1);
    }
  }
  __threadfence_block();
  __syncthreads();
  fork_pages(td, seq_lens_out, table_out, refs_out, src, dst, missing, need, free_list, wsum);
}

// New numbers of the pages (map: -1 for free ones), the counts by them, and the pairs to copy.
__global__ __launch_bounds__(kTableThreads) void compact_kernel(eta_table_desc_t td, const int32_t* refs,
                                                                int32_t* refs_out, int32_t* src, int32_t* dst,
                                                                int32_t* live, int32_t* map, const int32_t* table,
                                                                int32_t* table_out) {
  __shared__ int wsum[kTableThreads / 64];
  const int tid = threadIdx.x;
  const int64_t P = td.num_pages;
  int cnt = 0, n;
  for (int64_t p = tid; p < P; p += kTableThreads) cnt += refs[p] > 0;
  wide_excl_scan(cnt, wsum, &n);
  if (tid == 0) live[0] = n;
  // free numbers below n, in order, and as many pages in use from n on
  const int64_t moves = ranked(n, P, wsum, [&](int64_t p) { return refs[p] <= 0; },
                               [&](int64_t r, int64_t p) { dst[r] = (int32_t)p; });
  __threadfence_block();
  __syncthreads();
  ranked(P - n, P, wsum, [&](int64_t p) { return refs[n + p] > 0; },
         [&](int64_t r, int64_t p) {
           const int32_t to = dst[r];
           src[r] = (int32_t)(n + p);
           map[n + p] = to;
           refs_out[to] = refs[n + p];
         });
  for (int64_t p = tid; p < P; p += kTableThreads) {
    const int32_t c = refs[p];
    if (p < n && c > 0) {
      map[p] = (int32_t)p;
      refs_out[p] = c;
    }
    if (c <= 0) map[p] = -1;
    if (p >= n) refs_out[p] = 0;
  }
  for (int64_t r = moves + tid; r < P / 2; r += kTableThreads) src[r] = dst[r] = -1;
  if (table == nullptr) return;      // (its launch of its own follows)
  __threadfence_block();
  __syncthreads();
  const int64_t entries = td.batch * td.table_blocks;
  for (int64_t e = tid; e < entries; e += kTableThreads) {
    const int b = (int)((uint32_t)e / (uint32_t)td.table_blocks);
    const int64_t at = b * td.table_stride + (e - b * td.table_blocks);
    const int32_t p = table[at];
    table_out[at] = p >= 0 && p < P ? map[p] : -1;
  }
}

__global__ __launch_bounds__(256) void compact_table_kernel(eta_table_desc_t td, const int32_t* table,
                                                            int32_t* table_out, const int32_t* map) {
  const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x, b = blockIdx.y;
  if (j >= td.table_blocks) return;
  const int32_t p = table[b * td.table_stride + j];
  table_out[b * td.table_stride + j] = p >= 0 && p < td.num_pages ? map[p] : -1;
}

template <int D, int BS>
void launch_store(const StoreArgs& a, bool f32, dim3 grid, hipStream_t stream) {
  const dim3 threads(D / 8 * (BS / 4));
  if (a.new_tokens == 1) {
    const Geom& g = a.pg.g;
    if (f32)
      hipLaunchKernelGGL((page_token_kernel<D, BS, float>), dim3(2 * g.Hkv, g.B), dim3(256), 0, stream, a);
    else
      hipLaunchKernelGGL((page_token_kernel<D, BS, uint16_t>), dim3(2 * g.Hkv, g.B), dim3(256), 0, stream, a);
    return;
  }
  if (f32)
    hipLaunchKernelGGL((page_store_kernel<D, BS, float>), grid, threads, 0, stream, a);
  else
    hipLaunchKernelGGL((page_store_kernel<D, BS, uint16_t>), grid, threads, 0, stream, a);
}

}  // namespace

hipError_t launch_page_store(const PageGeom& pg, const eta_page_pool_t& pool, const int32_t* table,
                             const eta_page_rows_t& rows, const void* k, const void* v, const int32_t* start,
                             const int32_t* new_lens, hipStream_t stream, LaunchHook hook) {
  const Geom& g = pg.g;
  const StoreArgs a{{(uint8_t*)pool.k, (uint8_t*)pool.v}, {pool.k_scale, pool.v_scale}, {k, v},
                    {rows.k_stride_b, rows.v_stride_b}, {rows.k_stride_h, rows.v_stride_h},
                    {rows.k_stride_t, rows.v_stride_t}, table, start, new_lens, pg, rows.new_tokens};
  // the pages that new_tokens tokens can touch, wherever they begin
  const int64_t touched = ((int64_t)rows.new_tokens + g.BS - 2) / g.BS + 1;
  const dim3 grid((unsigned)(2 * (touched < pg.table_blocks ? touched : pg.table_blocks)), g.Hkv, g.B);
  const bool f32 = rows.dtype == ETA_DT_F32;
  return with_hook(hook, ETA_KERNEL_PAGE_STORE, stream, [&] {
    if (g.D == 64 && g.BS == 64) launch_store<64, 64>(a, f32, grid, stream);
    if (g.D == 64 && g.BS == 128) launch_store<64, 128>(a, f32, grid, stream);
    if (g.D == 128 && g.BS == 64) launch_store<128, 64>(a, f32, grid, stream);
    if (g.D == 128 && g.BS == 128) launch_store<128, 128>(a, f32, grid, stream);
  });
}

hipError_t launch_page_summaries(const PageGeom& pg, const eta_page_pool_t& pool, const int32_t* table,
                                 const int32_t* prev_lens, const int32_t* seq_lens, int max_new,
                                 const eta_summary_t& s, hipStream_t stream, LaunchHook hook) {
  const Geom& g = pg.g;
  const int64_t most = g.cap / g.BS < g.ncap ? g.cap / g.BS : g.ncap;
  const int64_t nblk = prev_lens != nullptr && max_new < most ? max_new : most;
  if (nblk <= 0) return hipSuccess;
  // Large caches (past what the last-level cache holds): 32 blocks to a workgroup, whose records
  // leave as whole rows, the keys read past the caches.  Below, one block to a wavefront, four to a
  // workgroup, so that as many start as there are.  us with 32 and the hint / 4 without, fp32
  // records: 256 MiB of keys (128 x 128 blocks) 57 / 69; 469 MiB (128 dims x 64) 111 / 117, 469 MiB
  // (64 x 64) 114 / 119; 98 MiB (128 x 64) 33 / 29; 49 MiB (64 x 128) 20 / 14; 4 MiB 23 / 7.
  // Between, four with the hint: 127 MiB (128 x 64) 39.1 without, 35.2 with it, 146 MiB 41.5 / 39.0, 128
  // MiB of different lengths 30.9 / 31.3; below, keys just stored are still in the caches.
  const int64_t keys = nblk * g.Hkv * g.B * g.BS * g.D;
  const bool large = nblk >= 32 && keys > (int64_t(200) << 20), hint = keys > (int64_t(96) << 20);
  const int nb = large ? 32 : 4;
  const unsigned wgs = (unsigned)((nblk + nb - 1) / nb), runs = wgs < 64 ? (wgs + 7) / 8 : 8, run = (wgs + runs - 1) / runs;
  const int64_t rounds = ((int64_t)g.B * g.Hkv * runs + 7) / 8, most_x = run < 16 ? 65536 : (1 << 20) / run,
                along = rounds < most_x ? rounds : most_x;
  const IndexArgs a{(const uint8_t*)pool.k, pool.k_scale, table, prev_lens, seq_lens, s.mu, s.sigma, s.max_norm, pg, max_new,
                    run, runs, (unsigned)along};
  const dim3 grid((unsigned)along * 8 * run, (unsigned)((rounds + along - 1) / along));
  return with_hook(hook, ETA_KERNEL_PAGE_SUMMARIES, stream, [&] {
#define ETA_PSUM(D_, BS_)                                                                                    \
  if (g.D == D_ && g.BS == BS_) {                                                                            \
    if (large)                                                                                               \
      hipLaunchKernelGGL((page_summaries_kernel<D_, BS_, 32, true>), grid, dim3(256), 0, stream, a);         \
    else if (hint)                                                                                           \
      hipLaunchKernelGGL((page_summaries_kernel<D_, BS_, 4, true>), grid, dim3(256), 0, stream, a);          \
    else                                                                                                     \
      hipLaunchKernelGGL((page_summaries_kernel<D_, BS_, 4, false>), grid, dim3(256), 0, stream, a);         \
  }
    ETA_PSUM(64, 64) ETA_PSUM(64, 128) ETA_PSUM(128, 64) ETA_PSUM(128, 128)
#undef ETA_PSUM
  });
}

hipError_t launch_page_copy(const PageGeom& pg, const eta_page_pool_t& pool, const int32_t* src,
                            const int32_t* dst, int64_t n, hipStream_t stream, LaunchHook hook) {
  if (n <= 0) return hipSuccess;
  const dim3 grid((unsigned)(n < 65536 ? n : 65536), 2 * pg.g.Hkv);
  return with_hook(hook, ETA_KERNEL_PAGE_COPY, stream, [&] {
    const int kb = pg.g.BS * pg.g.D / 4096;            // 4 KB pieces: 1, 2 or 4
    if (kb == 1) hipLaunchKernelGGL(page_copy_kernel<1>, grid, dim3(256), 0, stream, pool, pg, src, dst, n);
    if (kb == 2) hipLaunchKernelGGL(page_copy_kernel<2>, grid, dim3(256), 0, stream, pool, pg, src, dst, n);
    if (kb == 4) hipLaunchKernelGGL(page_copy_kernel<4>, grid, dim3(256), 0, stream, pool, pg, src, dst, n);
  });
}

hipError_t launch_page_extend(const eta_table_desc_t& td, int32_t* table, int32_t* refs,
                              const int32_t* seq_lens, int32_t* missing, const TableWs& ws,
                              hipStream_t stream, LaunchHook hook) {
  hipError_t e = with_hook(hook, ETA_KERNEL_PAGE_TABLE, stream, [&] {
    hipLaunchKernelGGL(extend_count_kernel, dim3(td.batch), dim3(256), 0, stream, td, table, seq_lens, ws.need);
  });
  if (e != hipSuccess) return e;
  return with_hook(hook, ETA_KERNEL_PAGE_TABLE, stream, [&] {
    hipLaunchKernelGGL(extend_kernel, dim3(1), dim3(kTableThreads), 0, stream, td, table, refs, seq_lens, missing,
                       ws.need, ws.map);
  });
}

hipError_t launch_page_fork(const eta_table_desc_t& td, const int32_t* table, const int32_t* refs,
                            const int32_t* seq_lens, const int32_t* parents, int32_t* table_out,
                            int32_t* refs_out, int32_t* seq_lens_out, int32_t* src, int32_t* dst,
                            int32_t* missing, const TableWs& ws, hipStream_t stream, LaunchHook hook) {
  if (td.batch <= kTableThreads && td.batch * td.table_blocks + td.num_pages <= kOneWorkgroup)
    return with_hook(hook, ETA_KERNEL_PAGE_TABLE, stream, [&] {
      hipLaunchKernelGGL(fork_kernel, dim3(1), dim3(kTableThreads), 0, stream, td, table, refs, seq_lens, parents,
                         table_out, refs_out, seq_lens_out, src, dst, missing, ws.need, ws.map);
    });
  hipError_t e = with_hook(hook, ETA_KERNEL_PAGE_TABLE, stream, [&] {
    hipLaunchKernelGGL(fork_init_kernel, dim3((unsigned)((td.num_pages + 255) / 256)), dim3(256), 0, stream, td, refs,
                       refs_out);
  });
  if (e != hipSuccess) return e;
  e = with_hook(hook, ETA_KERNEL_PAGE_TABLE, stream, [&] {
    hipLaunchKernelGGL(fork_rows_kernel, dim3((unsigned)((td.table_blocks + 255) / 256), td.batch), dim3(256), 0,
                       stream, td, table, seq_lens, parents, table_out, refs_out, seq_lens_out, ws.need);
  });
  if (e != hipSuccess) return e;
  return with_hook(hook, ETA_KERNEL_PAGE_TABLE, stream, [&] {
    hipLaunchKernelGGL(fork_pages_kernel, dim3(1), dim3(kTableThreads), 0, stream, td, seq_lens_out, table_out,
                       refs_out, src, dst, missing, ws.need, ws.map);
  });
}

hipError_t launch_page_compact(const eta_table_desc_t& td, const int32_t* table, const int32_t* refs,
                               int32_t* table_out, int32_t* refs_out, int32_t* src, int32_t* dst,
                               int32_t* live, const TableWs& ws, hipStream_t stream, LaunchHook hook) {
  const bool one = td.batch * td.table_blocks <= kOneWorkgroup;
  hipError_t e = with_hook(hook, ETA_KERNEL_PAGE_TABLE, stream, [&] {
    hipLaunchKernelGGL(compact_kernel, dim3(1), dim3(kTableThreads), 0, stream, td, refs, refs_out, src, dst, live,
                       ws.map, one ? table : nullptr, table_out);
  });
  if (e != hipSuccess || one) return e;
  return with_hook(hook, ETA_KERNEL_PAGE_TABLE, stream, [&] {
    hipLaunchKernelGGL(compact_table_kernel, dim3((unsigned)((td.table_blocks + 255) / 256), td.batch), dim3(256), 0,
                       stream, td, table, table_out, ws.map);
  });
}

}  // namespace eta

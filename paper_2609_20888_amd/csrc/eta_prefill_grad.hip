// Gradients of the gated prefill (gfx950, wave64): from the gradients of its
// output, gate row sums and log-sum-exp to those of q, k, v and tau.  The
// probabilities are formed again from q, k, tau and the saved log-sum-exp.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "eta_lanes.h"
#include "eta_tile.h"
#include "eta_train.h"
#include "eta_train_index.h"

namespace eta {
namespace {

// With S = q.k / sqrt(d), sg = sigmoid(beta (S - tau_i)), sg' = sg (1 - sg) and S~ as in the
// forward, P = exp(S~ - L_i), D_i = dO_i.O_i - dL_i:
//   dS~ = P (dO_i.v_j - D_i),   m = beta (S dS~ + dR_i)  (additive: beta (C dS~ + dR_i)),
//   dS  = dS~ sg + sg' m  (additive: dS~ + sg' m),   dtau_i = - sum_j sg' m,
//   dq_i = sum_j dS k_j / sqrt(d),  dk_j = sum_i dS q_i / sqrt(d),  dv_j = sum_i P dO_i;
// on the diagonal S~ = S, so dS = dS~ + sg' beta dR_i.
//
// Every sum has one owner and a fixed order: a workgroup owns either 128 query rows and walks over
// the keys (dq, dtau), or 128 keys and walks over the query rows and the heads of its group (dk,
// dv).  Each kind forms S and dO.v anew: seven products for the five that one walk would need, whose
// dq would have to be added up in memory from every block of keys (512 bytes a row for each 128
// keys, in an order that changes).  Both kinds run in one launch, the longest walks first, so that
// short ones fill the compute units beside the last long ones; the row scalars that both read (D
// among them) come from a small launch before.
// What bounds it: vector-ALU issue (three transcendentals and 10 to 12 other instructions for a score of
// either kind; 84% of the time at d = 64) and at d = 128 the card's power: 16K tokens, 32/8 heads:
// 8.2 to 8.4 ms, 660 TFLOP/s of the five products and 925 of the seven that run (a plain library product:
// 1260), the vector unit 69% and the matrix cores 52% busy at 1.85 GHz.  d = 64: 5.3 ms.  4096
// tokens, 16/4 heads, d = 128: 306 us (dR and dL given).

constexpr int kGrQ = 128;    // rows (queries or keys) a workgroup owns, 32 per wavefront
constexpr int kGrT = 64;     // rows of a streamed tile

struct GradArgs {
  const uint16_t *q, *k, *v, *out, *dout;
  const float *tau, *L, *dR, *dL;
  const int32_t* seq_lens;
  uint16_t *dq, *dk, *dv;
  float* dtau;
  float* stats;              // [B Hq][Tp / 32][4][32]: -L', beta tau' + log2(kd is2), -D, sqrt(d) dR or dR (Gate)
  float* part;               // [2][nsplit][B Hkv][T][d] partial dk, dv (nsplit > 1)
  int64_t part_step;         // nsplit B Hkv T d
  int B, Hq, Hkv, T, Tp, nsplit;
  float beta, C;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

extern "C" __device__ float eta_mul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");

// A score's gate and gradient, in base-2 units (S' = S log2 e = s2 c, c the raw product), with kd = beta /
// sqrt(d) (additive: beta), the factor of m, folded into the exponential:
//   E = kd is2 2^(-beta (S' - tau')) (is2 = 1 / s2),  u = 1 / (E / kd + is2) = s2 sg,  u E = kd (1 - sg),
//   m / kd = c dS~ + sqrt(d) dR (additive: C dS~ + dR),  s2 sg' m = u (u E) (m / kd).
// sg' keeps its relative accuracy where the gate is nearly open or nearly shut (the legacy product
// gives 0 for 0 x inf, the shut gate).  A beta below kLeastBeta, whose kd would leave E no room in
// fp32, takes part in the gate alone: kd is kLeastBeta's, dR counts as 0, m (dS~ times 1e-30) is lost in dS~'s
// rounding, and dtau is 0.
constexpr float kLeastBeta = 1e-30f;
struct Gate {
  float s2, is2, nbs, kd, ikd, C, C2, C2is;
  template <int D, bool ADD>
  static __device__ __forceinline__ Gate make(float beta, float C) {
    Gate g;
    g.s2 = kLog2e / sqrtf((float)D);
    g.is2 = 1.0f / g.s2;
    g.nbs = -beta * g.s2;
    g.kd = fmaxf(beta, kLeastBeta) * (ADD ? 1.0f : 1.0f / sqrtf((float)D));
    g.ikd = 1.0f / g.kd;
    g.C = C;
    g.C2 = C * kLog2e;
    g.C2is = g.C2 * g.is2;
    return g;
  }
};

// The row scalars of a score: t: beta tau' + log2(kd is2); nl: -L'; kap: sqrt(d) dR (additive: dR).
struct RowScalars {
  float t, nl, kap;
};

// The vector work of a unit: 16 scores of a lane, raw products in s and dO.v - D in dp, two
// scores a step, the four stages of a score one step apart so that no step waits for its own
// transcendentals.  row(j) gives score j's scalars, mask(j, valid, diag) its place (MASKED),
// done(j, p, ds, n) takes P, s2 dS and s2 sg' m (the last with TAU only); beside(step) is the matrix work of a step.
template <bool ADD, bool MASKED, bool TAU, typename Row, typename Mask, typename Done, typename Beside>
__device__ __forceinline__ void unit_scores(const Gate& g, const f32x16& s, const f32x16& dp, Row row, Mask mask,
                                            Done done, Beside beside) {
  float e[16], u[16], w[16], p[16];       // (a few of each are alive at a time)
#pragma unroll
  for (int st = 0; st < 11; ++st) {
    beside(st);
    if (st >= 3) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j = 2 * (st - 3) + i, o = j;
        const float d = p[o] * dp[j], kap = row(j).kap;
        float m = fmaf(d, ADD ? g.C : s[j], kap), lin = ADD ? g.s2 : u[o];
        if constexpr (MASKED) {
          bool valid, diag;
          mask(j, valid, diag);
          m = diag ? kap : m;
          lin = diag ? g.s2 : lin;
          m = valid ? m : 0.f;
        }
        const float n = w[o] * m;
        if constexpr (TAU || ADD || MASKED) done(j, p[o], fmaf(d, lin, n), n);
        else done(j, p[o], u[o] * fmaf(w[o], m, d), 0.f);
      }
    }
    if (st >= 2 && st < 10) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j = 2 * (st - 2) + i, o = j;
        w[o] = eta_mul_legacy(u[o], e[o]);              // kd (1 - sg)
        if constexpr (TAU || ADD || MASKED) w[o] *= u[o];
        const float nl = row(j).nl;
        float y = ADD ? fmaf(g.C2is, u[o], fmaf(s[j], g.s2, nl - g.C2)) : fmaf(s[j], u[o], nl);
        if constexpr (MASKED) {
          bool valid, diag;
          mask(j, valid, diag);
          y = diag ? fmaf(s[j], g.s2, nl) : y;
          y = valid ? y : kNegInf;
        }
        p[o] = __builtin_amdgcn_exp2f(y);
      }
    }
    if (st >= 1 && st < 9) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int o = 2 * (st - 1) + i;
        u[o] = __builtin_amdgcn_rcpf(fmaf(e[o], g.ikd, g.is2));
      }
    }
    if (st < 8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j = 2 * st + i;
        e[j] = __builtin_amdgcn_exp2f(fmaf(g.nbs, s[j], row(j).t));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A tile of rows of D bf16 in LDS: groups of 1 KiB (what a wavefront's direct load writes), 16 bytes
// apart, and in a row the 16-byte chunks XORed by row, so that (a) the same chunk of 16
// consecutive rows (row reads) and (b) an aligned run of four chunks of four consecutive rows
// (transpose reads) both cover all 64 banks once.  The padding takes the part of the row that
// would otherwise be XORed too: a lane's operands lie at four addresses plus constants.
template <int D>
struct Tile {
  static constexpr int GR = 512 / D, GB = 1040;      // rows and bytes of a group
  static constexpr int HALF = 32 / GR * GB, BYTES = 2 * HALF;   // of 32 and 64 rows
  static constexpr int NR = 4;                       // row addresses of a lane
  static __device__ __forceinline__ int swizzle(int row) {
    if constexpr (D == 128) return (row & 3) << 2;
    return ((row >> 1) & 1) << 2;
  }
  static __device__ __forceinline__ uint32_t at(int row, int chunk) {
    return (uint32_t)(row / GR * GB + row % GR * 2 * D + 16 * (chunk ^ swizzle(row)));
  }
  // dims 16 kc + 8 (lane / 32) .. of row lane & 31: row_base(lane, kc / per) + row_step(kc)
  static constexpr int PER = D / 16 / NR;
  static __device__ __forceinline__ uint32_t row_base(int lane, int i) { return at(lane & 31, 2 * PER * i + (lane >> 5)); }
  static constexpr int row_step(int kc) { return 32 * (kc % PER); }
  // dims 32 db + (lane & 31) of rows 16 c + 8 hi + 4 (lane / 32) .. + 3: turn_base(lane, db) + turn_step(c, hi)
  static __device__ __forceinline__ uint32_t turn_base(int lane, int db) {
    const int row = 4 * (lane >> 5) + ((lane & 15) >> 2), chunk = 4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    return at(row, chunk) + 8 * (lane & 1);
  }
  static constexpr int turn_step(int c, int hi) { return (16 * c + 8 * hi) / GR * GB; }
};

// Streams tiles of R rows of a [rows][D] tensor into LDS; rows from `rows` on repeat the last one
// (what the tensor holds there, NaN too, must reach no product).
template <int D, int R = kGrT>
struct TileLoad {
  static constexpr int CPR = D / 8, NI = R * CPR / 256, RPJ = 256 / CPR;
  static_assert(RPJ % 8 == 0, "the swizzle takes row bits 0 .. 2");
  int grow0;
  uint32_t goff;
  __device__ __forceinline__ explicit TileLoad(int tid)
      : grow0(tid / CPR), goff((uint32_t)(grow0 * D + 8 * ((tid % CPR) ^ Tile<D>::swizzle(grow0))) * 2u) {}
  __device__ __forceinline__ void operator()(const uint16_t* src, char* tile, int w, int blk, int rows) const {
    const int row0 = min(blk * R, rows - 1), over = blk * R + R - rows;
    const char* base = reinterpret_cast<const char*>(src + (int64_t)row0 * D);
    char* dst = tile + w * Tile<D>::GB;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      uint32_t off = goff + 4096u * j;
      if (over > 0) off -= (uint32_t)max(RPJ * j + grow0 - (rows - 1 - row0), 0) * (2u * D);
      __builtin_amdgcn_global_load_lds((const void*)(base + off),
                                       (__attribute__((address_space(3))) void*)(dst + 4 * Tile<D>::GB * j), 16, 0, 0);
    }
  }
};

typedef __attribute__((address_space(3))) char LdsBytes;
__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(LdsBytes*)p; }
__device__ __forceinline__ u32x4 lds_rows(uint32_t at) {
  return *(__attribute__((address_space(3))) const u32x4*)(uintptr_t)at;
}
__device__ __forceinline__ f32x4 lds_floats(uint32_t at) {
  return *(__attribute__((address_space(3))) const f32x4*)(uintptr_t)at;
}
__device__ __forceinline__ u32x4 lds_turned(uint32_t lo, uint32_t hi) {
  const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)lo);
  const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(uintptr_t)hi);
  const uint2 a2 = __builtin_bit_cast(uint2, a), b2 = __builtin_bit_cast(uint2, b);
  return u32x4{a2.x, a2.y, b2.x, b2.y};
}

__device__ __forceinline__ f32x16 mfma(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                 0, 0, 0);
}

// A unit's 16 values of a lane, given in order, as the two B operands of a product over the
// unit's 32 rows (bf16 pairs).  P and dS are rounded to bf16 here, once, for the products into dv, dq and dk (the
// sums stay fp32): the matrix cores take both operands in one type, and K, Q and dO are bf16.  In fp32
// these three products would run at a sixteenth of the bf16 rate; as two bf16 parts, high and low, they would be
// six.  It costs a half step of each term, which average: relative 2-norms of the results against 64 bits
// 2.3e-3 to 2.4e-3, with fp32 P and dS 1.7e-3, the rounding of the results alone.  dtau takes neither.
struct Packer {
  u32x4 o[2];
  float hold;
  __device__ __forceinline__ void put(int j, float x) {
    if (j & 1) {
      // (taken here: the work behind it is otherwise moved to where the pair is used, a unit
      // later, and its operands stay in registers)
      uint32_t both = pack_bf16x2(hold, x);
      asm volatile("" : "+v"(both));
      o[j >> 3][(j >> 1) & 3] = both;
    } else {
      hold = x;
    }
  }
};

// The row scalars (GradArgs::stats): D_i = dO_i.O_i - dL_i, the lanes of a row 16 bytes each, 64 rows of a head a
// workgroup.  Rows at or past the sequence's end, up to a whole block, get P = 0 and no gradient.  Bound by
// reading O and dO.
template <int D, bool ADD>
__global__ __launch_bounds__(256) void grad_rows_kernel(GradArgs a) {
  constexpr int LPR = D / 8, RPP = 256 / LPR, NP = 64 / RPP;       // lanes of a row, rows of a pass, passes
  __shared__ float d_s[64];
  const int blk = (int)(blockIdx.x % (uint32_t)(a.Tp / 64));
  const int64_t head = blockIdx.x / (uint32_t)(a.Tp / 64);
  const int n = (int)clamp_len(a.seq_lens, (int)(head / a.Hq), a.T) - 64 * blk;   // rows of the block that count
  const int r = threadIdx.x / LPR, c = threadIdx.x % LPR;
  const int64_t row0 = head * a.T + 64 * blk;
  u32x4 x[NP], y[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int64_t at = (row0 + r + RPP * i) * D + 8 * c;
    x[i] = y[i] = u32x4{0, 0, 0, 0};
    if (r + RPP * i < n) {
      x[i] = *reinterpret_cast<const u32x4*>(a.dout + at);
      y[i] = *reinterpret_cast<const u32x4*>(a.out + at);
    }
  }
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s = fmaf(__uint_as_float(x[i][j] << 16), __uint_as_float(y[i][j] << 16), s);
      s = fmaf(__uint_as_float(x[i][j] & 0xffff0000u), __uint_as_float(y[i][j] & 0xffff0000u), s);
    }
    s = lanes_sum<LPR>(s);
    if (c == 0) d_s[r + RPP * i] = s;
  }
  __syncthreads();
  const int which = threadIdx.x >> 6, t = threadIdx.x & 63;        // one scalar of 64 rows a wavefront
  float v = which == 0 ? kNegInf : 0.f;
  if (t < n) {
    if (which == 0) v = -a.L[row0 + t] * kLog2e;
    if (which == 1) v = a.beta * kLog2e * a.tau[row0 + t];
    if (which == 2) v = a.dL ? a.dL[row0 + t] - d_s[t] : -d_s[t];
    if (which == 3) v = a.dR && a.beta >= kLeastBeta ? a.dR[row0 + t] * (ADD ? 1.0f : sqrtf((float)D)) : 0.f;
  }
  if (which == 1) {
    const Gate g = Gate::make<D, ADD>(a.beta, a.C);
    v += log2f(g.kd * g.is2);
  }
  a.stats[(head * a.Tp + 64 * blk + (t & 32)) * 4 + 32 * which + (t & 31)] = v;
}

// dq, dtau of 128 query rows.  As in the forward each lane owns a query row: S^T = K Q^T and dP^T =
// V dO^T - D with A from LDS, dq^T += K^T dS^T with the lane's own dS (bf16) as B and K^T from transpose
// reads.
template <int D>
constexpr int kGradQLds = 4 * Tile<D>::BYTES;
template <int D, bool ADD>
__device__ __forceinline__ void grad_q(const GradArgs& a, char* lds, int qblk, int h, int b) {
  constexpr int KC = D / 16, DB = D / 32;
  using TL = Tile<D>;
  constexpr int BUF = 2 * TL::BYTES;                                // K, V; two buffers
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, g2 = lane >> 5;
  const int Tb = (int)clamp_len(a.seq_lens, b, a.T);
  const int64_t head = (int64_t)b * a.Hq + h, qrow0 = head * a.T;
  const int64_t kvoff = ((int64_t)b * a.Hkv + h / (a.Hq / a.Hkv)) * a.T * D;
  const Gate g = Gate::make<D, ADD>(a.beta, a.C);

  const int wrow0 = qblk * kGrQ + 32 * w, t = wrow0 + r32, tq = min(t, max(Tb, 1) - 1);
  u32x4 qb[KC], dob[KC];
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) {
    const int64_t at = (qrow0 + tq) * D + 16 * kc + 8 * g2;
    qb[kc] = *reinterpret_cast<const u32x4*>(a.q + at);
    dob[kc] = *reinterpret_cast<const u32x4*>(a.dout + at);
  }
  const bool in = t < Tb;
  const float* st = a.stats + (head * a.Tp + wrow0) * 4 + r32;
  const RowScalars rs{st[32], st[0], st[96]};
  const float nd = st[64];

  const TileLoad<D> load(tid);
  uint32_t ra[TL::NR], ta[DB];
#pragma unroll
  for (int i = 0; i < TL::NR; ++i) ra[i] = lds_address(lds) + TL::row_base(lane, i);
#pragma unroll
  for (int db = 0; db < DB; ++db) ta[db] = lds_address(lds) + TL::turn_base(lane, db);
  const uint16_t *kh = a.k + kvoff, *vh = a.v + kvoff;
  const int last_row = min(qblk * kGrQ + kGrQ, Tb) - 1;
  const int nkb = last_row >= qblk * kGrQ ? last_row / kGrT + 1 : 0;
  const int nu = wrow0 < Tb ? (min(wrow0 + 32, Tb) - 1) / 32 + 1 : 0;
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x16{};
  float nsum = 0.f;

  // One unit of 32 keys: the score products, the vector work, the product into dq.  Nothing of a
  // wavefront overlaps with its own vector work; the other wavefront of the SIMD's does.
  constexpr int LA = 4;                              // LDS operands ahead of their MFMA
  auto unit = [&](int u, int kt, auto masked_tag) {      // kt: byte offset of the unit's keys
    constexpr bool MASKED = decltype(masked_tag)::value;
    u32x4 op[LA];
    f32x16 s{}, dp;
#pragma unroll
    for (int i = 0; i < 16; ++i) dp[i] = nd;
    auto rd = [&](int x) {
      if (x < 2 * KC)
        op[x % LA] = lds_rows(ra[(x >> 1) / TL::PER] + kt + (x & 1 ? TL::BYTES : 0) + TL::row_step(x >> 1));
    };
#pragma unroll
    for (int x = 0; x < LA; ++x) rd(x);
#pragma unroll
    for (int x = 0; x < 2 * KC; ++x) {
      if (x & 1) dp = mfma(op[x % LA], dob[x >> 1], dp);
      else s = mfma(op[x % LA], qb[x >> 1], s);
      rd(x + LA);
      __builtin_amdgcn_sched_barrier(0);
    }
    Packer pk;
    float un = 0.f;
    unit_scores<ADD, MASKED, true>(
        g, s, dp, [&](int) { return rs; },
        [&](int i, bool& valid, bool& diag) {
          const int j = u * 32 + 8 * (i >> 2) + 4 * g2 + (i & 3);
          valid = j <= t && in;
          diag = j == t;
        },
        [&](int i, float, float ds, float n) {
          pk.put(i, ds);
          un += n;
          if (i & 1) asm volatile("" : "+v"(un));
        },
        [](int) {});
    nsum += un;
    auto rt = [&](int x) {
      if (x < 2 * DB)
        op[x % LA] = lds_turned(ta[x % DB] + kt + TL::turn_step(x / DB, 0), ta[x % DB] + kt + TL::turn_step(x / DB, 1));
    };
#pragma unroll
    for (int x = 0; x < LA; ++x) rt(x);
#pragma unroll
    for (int x = 0; x < 2 * DB; ++x) {
      acc[x % DB] = mfma(op[x % LA], pk.o[x / DB], acc[x % DB]);
      rt(x + LA);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // Blocks of 64 keys, two buffers: at the start of a block its tiles have arrived (the barrier says
  // so for every wavefront's part) and every wavefront is done with the other buffer.
  auto arrive = [&](int kb, int buf) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (kb + 1 < nkb) {
      load(kh, lds + (buf ^ 1) * BUF, w, kb + 1, Tb);
      load(vh, lds + (buf ^ 1) * BUF + TL::BYTES, w, kb + 1, Tb);
    }
  };
  if (nkb > 0) {
    load(kh, lds, w, 0, Tb);
    load(vh, lds + TL::BYTES, w, 0, Tb);
    constexpr std::integral_constant<bool, false> plain{};
    constexpr std::integral_constant<bool, true> masked{};
    // the blocks before the workgroup's rows (an even number of them) need no mask
    for (int kb = 0; kb < 2 * qblk; kb += 2) {
#pragma unroll
      for (int buf = 0; buf < 2; ++buf) {
        arrive(kb + buf, buf);
#pragma unroll
        for (int x = 0; x < 2; ++x)
          unit(2 * (kb + buf) + x, buf * BUF + x * TL::HALF, plain);
      }
    }
#pragma unroll 1
    for (int kb = 2 * qblk; kb < nkb; ++kb) {
      arrive(kb, kb & 1);
#pragma unroll 1
      for (int u = 2 * kb; u < min(2 * kb + 2, nu); ++u)
        unit(u, (kb & 1) * BUF + (u & 1) * TL::HALF, masked);
    }
  }

  nsum = row2_sum(nsum);
  if (t < a.T) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const uint32_t lo = in ? pack_bf16x2(acc[db][i] * kLn2, acc[db][i + 1] * kLn2) : 0u;
        const uint32_t hi = in ? pack_bf16x2(acc[db][i + 2] * kLn2, acc[db][i + 3] * kLn2) : 0u;
        *reinterpret_cast<uint2*>(a.dq + (qrow0 + t) * D + 32 * db + 2 * i + 4 * g2) = make_uint2(lo, hi);
      }
    if (g2 == 0) a.dtau[qrow0 + t] = in && a.beta >= kLeastBeta ? -nsum * g.is2 : 0.f;
  }
}

// dk, dv of 128 keys: each lane owns a key.  S = Q K^T and dP = dO V^T - D with A from LDS (rows of
// Q and dO) and B the wavefront's keys; dv^T += dO^T P and dk^T += Q^T dS with the lane's own P and
// dS (bf16) as B and dO^T, Q^T from transpose reads.  The tiles run from the sequence's end down to
// the keys' own rows, so that the workgroups of one kv head, which start together, read the same
// tiles at the same time.
//
// At d = 128 the sums take 128 registers; V stays in LDS (a B operand read each time), so that two
// wavefronts fit a SIMD and the matrix work of one runs beside the vector work of the other.
// (With V in registers too only one fits: 3.2K cycles a unit with all its matrix work threaded
// through the vector work, a quarter of them waits.)
template <int D>
struct KeyWalk {
  static constexpr bool VLDS = D == 128;
  static constexpr int TR = D == 128 ? 32 : 64, UT = TR / 32;      // rows and units of a tile
  static constexpr int NKL = VLDS ? 3 : 0;                         // K operands kept in LDS
  static constexpr int TILE = UT * Tile<D>::HALF, BUF = 2 * TILE + 4 * TR * 4;
  static constexpr int VB = VLDS ? 4 * (D / 16 + NKL) * 1024 : 0;
  static constexpr int LDS = VB + 2 * BUF;                         // V (and K operands), then twice: Q, dO, row scalars
};
template <int D, bool ADD>
__device__ __forceinline__ void grad_kv(const GradArgs& a, char* lds, int kblk, int hs, int b) {
  constexpr int KC = D / 16, DB = D / 32;
  using TL = Tile<D>;
  using KW = KeyWalk<D>;
  constexpr bool VLDS = KW::VLDS;
  constexpr int TR = KW::TR, UT = KW::UT, NKL = KW::NKL, TILE = KW::TILE, BUF = KW::BUF, VB = KW::VB;
  const int kvh = hs / a.nsplit, split = hs % a.nsplit;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, g2 = lane >> 5;
  const int Tb = (int)clamp_len(a.seq_lens, b, a.T);
  const int GH = a.Hq / a.Hkv / a.nsplit, h0 = kvh * (a.Hq / a.Hkv) + split * GH;   // this workgroup's heads
  const Gate g = Gate::make<D, ADD>(a.beta, a.C);
  const int wrow0 = kblk * kGrQ + 32 * w, j = wrow0 + r32, jk = min(j, max(Tb, 1) - 1);
  const int64_t kvrow0 = ((int64_t)b * a.Hkv + kvh) * a.T;
  u32x4 kf[KC - NKL], vf[VLDS ? 1 : KC];
  const uint32_t va = lds_address(lds) + w * (KC + NKL) * 1024 + lane * 16;   // operands of 1 KiB, as they are read
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) {
    const int64_t at = (kvrow0 + jk) * D + 16 * kc + 8 * g2;
    const u32x4 kk = *reinterpret_cast<const u32x4*>(a.k + at), vv = *reinterpret_cast<const u32x4*>(a.v + at);
    auto put = [&](int n, const u32x4& x) { *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(va + n * 1024) = x; };
    if (kc < NKL) put(KC + kc, kk);
    else kf[kc - NKL] = kk;
    if constexpr (VLDS) put(kc, vv);
    else vf[kc] = vv;
  }
  f32x16 dka[DB], dva[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dka[db] = dva[db] = f32x16{};

  // Tiles of each head: from the pair of tiles that holds the sequence's last row (rows past the end
  // have P = 0) down to the keys' own rows, an even number of them.
  const TileLoad<D, TR> load(tid);
  const int t0 = kblk * (kGrQ / TR), nt = 2 * ((Tb + 2 * TR - 1) / (2 * TR)), nb = max(nt - t0, 0), steps = nb * GH;
  const int ku = wrow0 / 32;                                       // the unit of the wavefront's diagonal
  int fh = 0, ft = nt - 1;                                         // next tile to fetch
  auto fetch = [&](int buf) {
    const int64_t head = (int64_t)b * a.Hq + h0 + fh;
    char* dst = lds + VB + buf * BUF;
    load(a.q + head * a.T * D, dst, w, ft, Tb);
    load(a.dout + head * a.T * D, dst + TILE, w, ft, Tb);
    if (w < 4 * TR / 64)                                           // 64 of the 4 TR scalars
      __builtin_amdgcn_global_load_lds((const void*)(a.stats + (head * a.Tp + ft * TR) * 4 + tid),
                                       (__attribute__((address_space(3))) void*)(dst + 2 * TILE + 256 * w), 4, 0, 0);
    if (ft-- == t0) {
      ft = nt - 1;
      ++fh;
    }
  };

  uint32_t ra[TL::NR], ta[DB];
#pragma unroll
  for (int i = 0; i < TL::NR; ++i) ra[i] = lds_address(lds) + VB + TL::row_base(lane, i);
#pragma unroll
  for (int db = 0; db < DB; ++db) ta[db] = lds_address(lds) + VB + TL::turn_base(lane, db);
  const uint32_t sa = lds_address(lds) + VB + 2 * TILE + 16 * g2;

  // One unit of 32 query rows (half a tile where the tile has 64).  Its MFMAs in order: S, dP, the
  // products into dv and dk, those of the rows whose P and dS come first beside the last steps of the
  // vector work.  (The rest overlaps with the vector work of the SIMD's other wavefront.)
  constexpr int LA = 3;                                            // LDS operands ahead of their MFMA
  constexpr int NM = 2 * KC + 4 * DB;
  auto unit = [&](int row0, int buf, int half, auto masked_tag) {
    constexpr bool MASKED = decltype(masked_tag)::value;
    const int at = buf * BUF + half * TL::HALF;
    auto scalars = [&](int which, int x) {                         // rows 8 x + 4 g2 .. + 3
      return lds_floats(sa + buf * BUF + half * 512 + which * 128 + 32 * x);
    };
    u32x4 op[LA], ov[LA];
    f32x16 s{}, dp;
    Packer pp, pd;
    auto rd = [&](int x) {
      if (x < 2 * KC) {
        const int kc = x % KC;
        op[x % LA] = lds_rows(ra[kc / TL::PER] + at + (x < KC ? 0 : TILE) + TL::row_step(kc));
        if (x < NKL) ov[x % LA] = lds_rows(va + (KC + kc) * 1024);
        if (VLDS && x >= KC) ov[x % LA] = lds_rows(va + kc * 1024);
      } else if (x < NM) {
        const int y = x - 2 * KC, c = y / (2 * DB), db = y % (2 * DB) / 2;
        const uint32_t o = ta[db] + at + (y & 1 ? 0 : TILE);
        op[x % LA] = lds_turned(o + TL::turn_step(c, 0), o + TL::turn_step(c, 1));
      }
    };
    auto step = [&](int x) {
      if (x < KC) {
        s = mfma(op[x % LA], x < NKL ? ov[x % LA] : kf[x < NKL ? 0 : x - NKL], s);
      } else if (x < 2 * KC) {
        dp = mfma(op[x % LA], VLDS ? ov[x % LA] : vf[VLDS ? 0 : x - KC], dp);
      } else {
        const int y = x - 2 * KC, c = y / (2 * DB), db = y % (2 * DB) / 2;
        if (y & 1) dka[db] = mfma(op[x % LA], pd.o[c], dka[db]);
        else dva[db] = mfma(op[x % LA], pp.o[c], dva[db]);
      }
      rd(x + LA);
    };
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const f32x4 nd = scalars(2, x);
#pragma unroll
      for (int i = 0; i < 4; ++i) dp[4 * x + i] = nd[i];
    }
#pragma unroll
    for (int x = 0; x < LA; ++x) rd(x);
#pragma unroll
    for (int x = 0; x < 2 * KC; ++x) {
      step(x);
      __builtin_amdgcn_sched_barrier(0);
    }
    f32x4 nl[4], bt[4], kap[4];
    bt[0] = scalars(1, 0);
    unit_scores<ADD, MASKED, false>(
        g, s, dp, [&](int i) { return RowScalars{bt[i >> 2][i & 3], nl[i >> 2][i & 3], kap[i >> 2][i & 3]}; },
        [&](int i, bool& valid, bool& diag) {
          const int row = row0 + 8 * (i >> 2) + 4 * g2 + (i & 3);
          valid = j <= row;
          diag = j == row;
        },
        [&](int i, float p, float ds, float) {
          pp.put(i, p);
          pd.put(i, ds);
        },
        [&](int st) {        // the scalars of four rows are read a step before the first of them is due
          if (st % 2 == 1 && st < 7) bt[(st + 1) / 2] = scalars(1, (st + 1) / 2);
          if (st % 2 == 1 && st < 8) nl[st / 2] = scalars(0, st / 2);
          if (st >= 2 && st % 2 == 0 && st < 10) kap[st / 2 - 1] = scalars(3, st / 2 - 1);
#pragma unroll
          for (int x = 2 * KC; x < 2 * KC + 2 * DB; ++x)           // (the first half is packed in step 6)
            if (7 + (x - 2 * KC) * 4 / (2 * DB) == st) step(x);
        });
#pragma unroll
    for (int x = 2 * KC + 2 * DB; x < NM; ++x) {
      step(x);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // At the start of a tile it has arrived (the barrier says so for every wavefront's part) and every
  // wavefront is done with the other buffer.
  int it = 0;
  auto arrive = [&](int buf) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (++it < steps) fetch(buf ^ 1);
  };
  if (steps > 0) {
    fetch(0);
    constexpr std::integral_constant<bool, false> plain{};
    constexpr std::integral_constant<bool, true> masked{};
    for (int hh = 0; hh < GH; ++hh) {
      int t = nt - 1;
      for (; t >= t0 + kGrQ / TR; t -= 2) {
#pragma unroll
        for (int buf = 0; buf < 2; ++buf) {
          arrive(buf);
#pragma unroll
          for (int x = UT - 1; x >= 0; --x) unit((t - buf) * TR + 32 * x, buf, x, plain);
        }
      }
      // the keys' own rows: a wavefront's units before its diagonal hold no pair
#pragma unroll 1
      for (; t >= t0; --t) {
        const int buf = (t & 1) ^ 1;
        arrive(buf);
#pragma unroll 1
        for (int x = UT - 1; x >= 0; --x)
          if (UT * t + x >= ku) unit(t * TR + 32 * x, buf, x, masked);
      }
    }
  }

  if (j >= Tb)       // (no pair reached these sums; a NaN of the sequence's last row, which stood in for the key, may have)
#pragma unroll
    for (int db = 0; db < DB; ++db) dka[db] = dva[db] = f32x16{};
  if (j < a.T) {
    if (a.nsplit > 1) {
      float* o = a.part + (((int64_t)(split * a.B + b) * a.Hkv + kvh) * a.T + j) * D + 4 * g2;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          *reinterpret_cast<f32x4*>(o + 32 * db + 2 * i) = f32x4{dka[db][i], dka[db][i + 1], dka[db][i + 2], dka[db][i + 3]};
          *reinterpret_cast<f32x4*>(o + a.part_step + 32 * db + 2 * i) =
              f32x4{dva[db][i], dva[db][i + 1], dva[db][i + 2], dva[db][i + 3]};
        }
    } else {
      const int64_t o = (kvrow0 + j) * D + 4 * g2;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          *reinterpret_cast<uint2*>(a.dk + o + 32 * db + 2 * i) =
              make_uint2(pack_bf16x2(dka[db][i] * kLn2, dka[db][i + 1] * kLn2),
                         pack_bf16x2(dka[db][i + 2] * kLn2, dka[db][i + 3] * kLn2));
          *reinterpret_cast<uint2*>(a.dv + o + 32 * db + 2 * i) =
              make_uint2(pack_bf16x2(dva[db][i], dva[db][i + 1]), pack_bf16x2(dva[db][i + 2], dva[db][i + 3]));
        }
    }
  }
}

template <int D, bool ADD>
__global__ __launch_bounds__(256, 2) void grad_kernel(GradArgs a, int blocks) {
  __shared__ __attribute__((aligned(16))) char lds[kGradQLds<D> > KeyWalk<D>::LDS ? kGradQLds<D> : KeyWalk<D>::LDS];
  const GradWork x = grad_work(blockIdx.x, (uint32_t)blocks, (uint32_t)a.B, (uint32_t)a.Hq, (uint32_t)a.Hkv, (uint32_t)a.nsplit);
  if (x.keys) grad_kv<D, ADD>(a, lds, x.blk, x.h, x.b);
  else grad_q<D, ADD>(a, lds, x.blk, x.h, x.b);
}

// dk (blockIdx.y 0) or dv (1) from the head splits' partials, added in order; four values a thread.
__global__ __launch_bounds__(256) void grad_join_kernel(GradArgs a, int64_t n4) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n4) return;
  const f32x4* p = reinterpret_cast<const f32x4*>(a.part + blockIdx.y * a.part_step) + i;
  f32x4 s = p[0];
  for (int x = 1; x < a.nsplit; ++x) s += p[x * n4];
  const float f = blockIdx.y ? 1.0f : kLn2;
  reinterpret_cast<uint2*>(blockIdx.y ? a.dv : a.dk)[i] =
      make_uint2(pack_bf16x2(s[0] * f, s[1] * f), pack_bf16x2(s[2] * f, s[3] * f));
}

}  // namespace

hipError_t launch_prefill_grad(const eta_prefill_desc_t& pd, const GradPlan& p, const PrefillGradPtrs& x,
                               hipStream_t stream, LaunchHook hook) {
  GradArgs a{};
  a.q = (const uint16_t*)x.q;
  a.k = (const uint16_t*)x.k;
  a.v = (const uint16_t*)x.v;
  a.out = (const uint16_t*)x.out;
  a.dout = (const uint16_t*)x.dout;
  a.tau = x.tau;
  a.L = x.L;
  a.dR = x.dR;
  a.dL = x.dL;
  a.seq_lens = x.seq_lens;
  a.dq = (uint16_t*)x.dq;
  a.dk = (uint16_t*)x.dk;
  a.dv = (uint16_t*)x.dv;
  a.dtau = x.dtau;
  a.stats = x.stats;
  a.part = x.part;
  a.B = pd.batch;
  a.Hq = pd.num_q_heads;
  a.Hkv = pd.num_kv_heads;
  a.T = pd.capacity_tokens;
  a.Tp = p.rows;
  a.nsplit = p.nsplit;
  a.part_step = (int64_t)p.nsplit * pd.batch * pd.num_kv_heads * pd.capacity_tokens * pd.head_dim;
  a.beta = pd.beta;
  a.C = pd.additive ? pd.C : 0.f;
  hipError_t e = with_hook(hook, ETA_KERNEL_PREFILL_GRAD_ROWS, stream, [&] {
    const int64_t rows = (int64_t)pd.batch * pd.num_q_heads * p.rows;
    const dim3 grid((uint32_t)(rows / 64));
    if (pd.additive) {
      if (pd.head_dim == 64) hipLaunchKernelGGL((grad_rows_kernel<64, true>), grid, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((grad_rows_kernel<128, true>), grid, dim3(256), 0, stream, a);
    } else {
      if (pd.head_dim == 64) hipLaunchKernelGGL((grad_rows_kernel<64, false>), grid, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((grad_rows_kernel<128, false>), grid, dim3(256), 0, stream, a);
    }
  });
  if (e != hipSuccess) return e;
  const dim3 grid((uint32_t)((int64_t)p.blocks * pd.batch * (pd.num_q_heads + pd.num_kv_heads * p.nsplit)));
  e = with_hook(hook, ETA_KERNEL_PREFILL_GRAD, stream, [&] {
    if (pd.additive) {
      if (pd.head_dim == 64) hipLaunchKernelGGL((grad_kernel<64, true>), grid, dim3(256), 0, stream, a, p.blocks);
      else hipLaunchKernelGGL((grad_kernel<128, true>), grid, dim3(256), 0, stream, a, p.blocks);
    } else {
      if (pd.head_dim == 64) hipLaunchKernelGGL((grad_kernel<64, false>), grid, dim3(256), 0, stream, a, p.blocks);
      else hipLaunchKernelGGL((grad_kernel<128, false>), grid, dim3(256), 0, stream, a, p.blocks);
    }
  });
  if (e != hipSuccess || p.nsplit == 1) return e;
  const int64_t n4 = a.part_step / p.nsplit / 4;
  return with_hook(hook, ETA_KERNEL_PREFILL_GRAD_JOIN, stream, [&] {
    hipLaunchKernelGGL(grad_join_kernel, dim3((uint32_t)((n4 + 255) / 256), 2), dim3(256), 0, stream, a, n4);
  });
}

}  // namespace eta

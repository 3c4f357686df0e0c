// Gradients of the gated prefill (gfx950, wave64): from the gradients of its
// output, gate row sums and log-sum-exp to those of q, k, v and tau.  The
// probabilities are formed again from q, k, tau and the saved log-sum-exp.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "eta_tile.h"
#include "eta_train.h"

namespace eta {
namespace {

// With S = q.k / sqrt(d), sg = sigmoid(beta (S - tau_i)), sg' = sg (1 - sg) and S~ as in the
// forward, P = exp(S~ - L_i), D_i = dO_i.O_i - dL_i:
//   dS~ = P (dO_i.v_j - D_i),   m = beta (S dS~ + dR_i)  (additive: beta (C dS~ + dR_i)),
//   dS  = dS~ sg + sg' m  (additive: dS~ + sg' m),   dtau_i = - sum_j sg' m,
//   dq_i = sum_j dS k_j / sqrt(d),  dk_j = sum_i dS q_i / sqrt(d),  dv_j = sum_i P dO_i;
// on the diagonal S~ = S, so dS = dS~ + sg' beta dR_i.
//
// Two passes, so that every sum has one owner and a fixed order: grad_q_kernel owns 128 query
// rows and walks over the keys (dq, dtau), grad_kv_kernel owns 128 keys and walks over the
// query rows and the heads of its group (dk, dv).  Each forms S and dO.v anew: seven products
// for the five that one pass would need, whose dq would have to be added up in memory from
// every block of keys (512 bytes a row for each 128 keys, in an order that changes).
// What bounds them: vector-ALU issue, as in the forward (three transcendentals and about
// twelve other instructions for a score in either pass).

constexpr int kGrQ = 128;    // rows (queries or keys) a workgroup owns, 32 per wavefront
constexpr int kGrT = 64;     // rows of a streamed tile

struct GradArgs {
  const uint16_t *q, *k, *v, *out, *dout;
  const float *tau, *L, *dR, *dL;
  const int32_t* seq_lens;
  uint16_t *dq, *dk, *dv;
  float* dtau;
  float* stats;              // [4][B Hq][Tp]: -L and tau in base-2 units, -D, beta dR
  float* part;               // [2][nsplit][B Hkv][T][d] partial dk, dv (nsplit > 1)
  int64_t stat_step;         // B Hq Tp
  int64_t part_step;         // nsplit B Hkv T d
  int Hq, Hkv, T, Tp, nsplit;
  float beta, C;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

extern "C" __device__ float eta_mul_legacy(float, float) __asm("llvm.amdgcn.fmul.legacy");

// A score's gate and gradient, in base-2 units (S' = S log2 e = s2 c, c the raw product):
// E = is2 2^(-beta (S' - tau')) (the factor is2 = 1 / s2 is in the exponent), u = 1 / (E + is2)
// = s2 sg, u E = 1 - sg, so sg' keeps its relative accuracy where the gate is nearly open or
// nearly shut (the legacy product gives 0 for 0 x inf, the shut gate).
struct Gate {
  float s2, is2, nbs, lis2, kd, C2is;   // kd: beta / sqrt(d) (additive: beta C)
  template <int D>
  static __device__ __forceinline__ Gate make(float beta, float C, bool add) {
    Gate g;
    g.s2 = kLog2e / sqrtf((float)D);
    g.is2 = 1.0f / g.s2;
    g.nbs = -beta * g.s2;
    g.lis2 = log2f(g.is2);
    g.kd = add ? beta * C : beta / sqrtf((float)D);
    g.C2is = C * kLog2e * g.is2;
    return g;
  }
};

// c: raw product, t: beta tau' + log2 is2, nl: -L' (additive: -L' - C'), dp: dO.v - D, kap: beta dR.
// Gives P, s2 dS and s2 sg' m.
template <bool ADD, bool MASKED>
__device__ __forceinline__ void score_grad(const Gate& g, float c, float t, float nl, float nl_diag, float dp,
                                           float kap, bool valid, bool diag, float& p, float& ds, float& n) {
  const float e = __builtin_amdgcn_exp2f(fmaf(g.nbs, c, t));
  const float u = __builtin_amdgcn_rcpf(e + g.is2);
  const float w = u * eta_mul_legacy(u, e);
  float y = ADD ? fmaf(g.C2is, u, fmaf(c, g.s2, nl)) : fmaf(c, u, nl);
  if constexpr (MASKED) {
    if (diag) y = fmaf(c, g.s2, nl_diag);
    if (!valid) y = kNegInf;
  }
  p = __builtin_amdgcn_exp2f(y);
  const float d = p * dp;
  float m = fmaf(ADD ? d : d * c, g.kd, kap);
  float lin = ADD ? g.s2 : u;
  if constexpr (MASKED) {
    if (diag) {
      m = kap;
      lin = g.s2;
    }
    if (!valid) m = 0.f;
  }
  n = w * m;
  ds = fmaf(d, lin, n);
}

// The work of workgroup `wg` of nb blocks and NH (head, sequence) pairs: blocks in order of
// `blk` (the caller puts the longest first), and with a multiple of eight heads neighbouring
// heads on one XCD (workgroups are dealt to the eight XCDs round robin).
__device__ __forceinline__ void grad_work(uint32_t wg, uint32_t H, uint32_t NH, int& blk, int& h, int& b) {
  blk = (int)(wg / NH);
  const uint32_t hi = wg % NH;
  if ((H & 7) == 0) {
    const uint32_t hpx = H / 8, r = hi / 8;
    h = (int)((hi % 8) * hpx + r % hpx);
    b = (int)(r / hpx);
  } else {
    h = (int)(hi % H);
    b = (int)(hi / H);
  }
}

// Streams 64-row tiles of a [rows][D] tensor into swizzled LDS; rows from `rows` on repeat the
// last one (what the tensor holds there, NaN too, must reach no product).
template <int D>
struct TileLoad {
  static constexpr int CPR = D / 8, NI = kGrT * CPR / 256, RPJ = 256 / CPR;
  static_assert(RPJ % 16 == 0, "the swizzle takes row bits 0 .. 3");
  int grow0;
  uint32_t goff;
  __device__ __forceinline__ explicit TileLoad(int tid)
      : grow0(tid / CPR), goff((uint32_t)(grow0 * D + 8 * pf_chunk<D>(grow0, tid % CPR)) * 2u) {}
  __device__ __forceinline__ void operator()(const uint16_t* src, uint16_t* tile, int w, int blk, int rows) const {
    const char* base = reinterpret_cast<const char*>(src + (int64_t)blk * kGrT * D);
    uint16_t* dst = tile + 8 * 64 * w;
    if ((blk + 1) * kGrT <= rows) {
#pragma unroll
      for (int j = 0; j < NI; ++j)
        __builtin_amdgcn_global_load_lds((const void*)(base + goff + 4096 * j),
                                         (__attribute__((address_space(3))) void*)(dst + 8 * 256 * j), 16, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int row = RPJ * j + grow0;
        const uint32_t off =
            goff + 4096u * j - (uint32_t)(row - (min(blk * kGrT + row, rows - 1) - blk * kGrT)) * (2u * D);
        __builtin_amdgcn_global_load_lds((const void*)(base + off),
                                         (__attribute__((address_space(3))) void*)(dst + 8 * 256 * j), 16, 0, 0);
      }
    }
  }
};

// Operands from a swizzled half tile (32 rows): rows as they are (row lane & 31, dims 16 kc + 8 g2 ..),
// and transposed (dims 32 db + lane & 31 of the 16 rows of chunk c, in the order of pack_units).
template <int D>
struct TileRead {
  int row_off, r32, g2, vt_row, vt_c, vt_half;
  __device__ __forceinline__ explicit TileRead(int lane)
      : r32(lane & 31), g2(lane >> 5), vt_row(4 * (lane >> 5) + ((lane & 15) >> 2)),
        vt_c(2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)), vt_half(4 * (lane & 1)) {}
  __device__ __forceinline__ u32x4 rows(const uint16_t* t, int kc) const {
    return *reinterpret_cast<const u32x4*>(&t[r32 * D + 8 * pf_chunk<D>(r32, 2 * kc + g2)]);
  }
  __device__ __forceinline__ int off(int c, int db, int hi8) const {
    const int row = vt_row + 8 * hi8;
    return (16 * c + row) * D + 8 * pf_chunk<D>(row, 4 * db + vt_c) + vt_half;
  }
  __device__ __forceinline__ u32x4 turned(const uint16_t* t, int c, int db) const {
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) i16x4*)(&t[off(c, db, 0)]));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) i16x4*)(&t[off(c, db, 1)]));
    const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
    return u32x4{l2.x, l2.y, h2.x, h2.y};
  }
};

__device__ __forceinline__ f32x16 mfma(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                 0, 0, 0);
}

// A unit's 16 values of a lane as the two B operands of a product over the unit's 32 rows
__device__ __forceinline__ void pack_units(const float (&x)[16], u32x4 (&o)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[i >> 1][2 * (i & 1)] = pack_bf16x2(x[4 * i], x[4 * i + 1]);
    o[i >> 1][2 * (i & 1) + 1] = pack_bf16x2(x[4 * i + 2], x[4 * i + 3]);
  }
}

__device__ __forceinline__ float dot_bf16(const u32x4& a, const u32x4& b, float s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s = fmaf(__uint_as_float(a[i] << 16), __uint_as_float(b[i] << 16), s);
    s = fmaf(__uint_as_float(a[i] & 0xffff0000u), __uint_as_float(b[i] & 0xffff0000u), s);
  }
  return s;
}

// dq, dtau of 128 query rows, and the row scalars that grad_kv_kernel reads.  As in the forward
// each lane owns a query row: S^T = K Q^T and dP^T = V dO^T with A from LDS, dq^T += K^T dS^T with
// the lane's own dS (bf16) as B and K^T from transpose reads.
template <int D, bool ADD>
__global__ __launch_bounds__(256, 2) void grad_q_kernel(GradArgs a) {
  constexpr int KC = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) uint16_t k_s[2][kGrT * D];
  __shared__ __attribute__((aligned(16))) uint16_t v_s[2][kGrT * D];
  const uint32_t nqb = gridDim.x, NH = gridDim.y * gridDim.z;
  int blk, h, b;
  grad_work(blockIdx.x + nqb * (blockIdx.y + gridDim.y * blockIdx.z), (uint32_t)a.Hq, NH, blk, h, b);
  const int qblk = (int)nqb - 1 - blk;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, g2 = lane >> 5;
  const int Tb = (int)clamp_len(a.seq_lens, b, a.T);
  const int64_t head = (int64_t)b * a.Hq + h, qrow0 = head * a.T;
  const int64_t kvoff = ((int64_t)b * a.Hkv + h / (a.Hq / a.Hkv)) * a.T * D;
  const Gate g = Gate::make<D>(a.beta, a.C, ADD);

  const int wrow0 = qblk * kGrQ + 32 * w, t = wrow0 + r32, tq = min(t, max(Tb, 1) - 1);
  u32x4 qb[KC], dob[KC];
  float dsum = 0.f;
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) {
    const int64_t at = (qrow0 + tq) * D + 16 * kc + 8 * g2;
    qb[kc] = *reinterpret_cast<const u32x4*>(a.q + at);
    dob[kc] = *reinterpret_cast<const u32x4*>(a.dout + at);
    dsum = dot_bf16(dob[kc], *reinterpret_cast<const u32x4*>(a.out + at), dsum);
  }
  // row scalars; rows at or past the sequence's end take P = 0 and no gradient
  const bool in = t < Tb;
  float nl = kNegInf, bt = 0.f, nd = 0.f, kap = 0.f;
  if (in) {
    nl = -a.L[qrow0 + t] * kLog2e;
    bt = a.beta * a.tau[qrow0 + t] * kLog2e;
    nd = -row2_sum(dsum);
    if (a.dL) nd += a.dL[qrow0 + t];
    if (a.dR) kap = a.beta * a.dR[qrow0 + t];
  }
  if (g2 == 0) {
    float* st = a.stats + head * a.Tp + t;
    st[0] = nl;
    st[a.stat_step] = bt;
    st[2 * a.stat_step] = nd;
    st[3 * a.stat_step] = kap;
  }
  const float nlg = ADD ? nl - a.C * kLog2e : nl, btl = bt + g.lis2;

  const TileLoad<D> load(tid);
  const TileRead<D> rd(lane);
  const uint16_t *kh = a.k + kvoff, *vh = a.v + kvoff;
  const int last_row = min(qblk * kGrQ + kGrQ, Tb) - 1;
  const int nkb = last_row >= qblk * kGrQ ? last_row / kGrT + 1 : 0;
  const int nu = wrow0 < Tb ? (min(wrow0 + 32, Tb) - 1) / 32 + 1 : 0;
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x16{};
  float nsum = 0.f;

  auto unit = [&](int u, const uint16_t* kt, const uint16_t* vt, auto masked_tag) {
    constexpr bool MASKED = decltype(masked_tag)::value;
    f32x16 s{}, dp;
#pragma unroll
    for (int i = 0; i < 16; ++i) dp[i] = nd;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) s = mfma(rd.rows(kt, kc), qb[kc], s);
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) dp = mfma(rd.rows(vt, kc), dob[kc], dp);
    float ds[16], un = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = u * 32 + 8 * (i >> 2) + 4 * g2 + (i & 3);
      float p, n;
      score_grad<ADD, MASKED>(g, s[i], btl, nlg, nl, dp[i], kap, j <= t && in, j == t, p, ds[i], n);
      un += n;
    }
    nsum += un;
    u32x4 x[2];
    pack_units(ds, x);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] = mfma(rd.turned(kt, c, db), x[c], acc[db]);
  };

  if (nkb > 0) {
    load(kh, k_s[0], w, 0, Tb);
    load(vh, v_s[0], w, 0, Tb);
  }
  for (int kb = 0; kb < nkb; ++kb) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (kb + 1 < nkb) {
      load(kh, k_s[(kb + 1) & 1], w, kb + 1, Tb);
      load(vh, v_s[(kb + 1) & 1], w, kb + 1, Tb);
    }
#pragma unroll 1
    for (int u = 2 * kb; u < min(2 * kb + 2, nu); ++u) {
      const uint16_t *kt = k_s[kb & 1] + (u & 1) * 32 * D, *vt = v_s[kb & 1] + (u & 1) * 32 * D;
      if (u < nu - 1) unit(u, kt, vt, std::integral_constant<bool, false>{});
      else unit(u, kt, vt, std::integral_constant<bool, true>{});
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
    if (g2 == 0) a.dtau[qrow0 + t] = in ? -nsum * g.is2 : 0.f;
  }
}

// dk, dv of 128 keys: each lane owns a key.  S = Q K^T and dP = dO V^T - D with A from LDS (rows of
// Q and dO) and B the wavefront's keys in registers; dv^T += dO^T P and dk^T += Q^T dS with the
// lane's own P and dS (bf16) as B and dO^T, Q^T from transpose reads.  The tiles run from the
// sequence's end down to the keys' own rows, so that the workgroups of one kv head, which start
// together, read the same tiles at the same time.
template <int D, bool ADD>
__global__ __launch_bounds__(256, 1) void grad_kv_kernel(GradArgs a) {
  constexpr int KC = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) uint16_t q_s[2][kGrT * D];
  __shared__ __attribute__((aligned(16))) uint16_t do_s[2][kGrT * D];
  __shared__ __attribute__((aligned(16))) float st_s[2][4][kGrT];
  const uint32_t NH = gridDim.y * gridDim.z;
  int kblk, hs, b;
  grad_work(blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z), (uint32_t)gridDim.y, NH, kblk, hs, b);
  const int kvh = hs / a.nsplit, split = hs % a.nsplit;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, g2 = lane >> 5;
  const int Tb = (int)clamp_len(a.seq_lens, b, a.T);
  const int GH = a.Hq / a.Hkv / a.nsplit, h0 = kvh * (a.Hq / a.Hkv) + split * GH;   // this workgroup's heads
  const Gate g = Gate::make<D>(a.beta, a.C, ADD);
  const int wrow0 = kblk * kGrQ + 32 * w, j = wrow0 + r32, jk = min(j, max(Tb, 1) - 1);
  const int64_t kvrow0 = ((int64_t)b * a.Hkv + kvh) * a.T;
  u32x4 kf[KC], vf[KC];
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) {
    const int64_t at = (kvrow0 + jk) * D + 16 * kc + 8 * g2;
    kf[kc] = *reinterpret_cast<const u32x4*>(a.k + at);
    vf[kc] = *reinterpret_cast<const u32x4*>(a.v + at);
  }
  f32x16 dka[DB], dva[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dka[db] = dva[db] = f32x16{};

  const TileLoad<D> load(tid);
  const TileRead<D> rd(lane);
  // tiles of 64 query rows of a head: from nqb - 1 down to qb0; units from the wavefront's own (ku) on
  const int qb0 = kblk * (kGrQ / kGrT), nqb = (Tb + kGrT - 1) / kGrT, nb = max(nqb - qb0, 0);
  const int ku = wrow0 / 32, steps = nb * GH;

  auto fetch = [&](int it, int buf) {
    const int hh = it / nb, qb = nqb - 1 - (it - hh * nb);
    const int64_t head = (int64_t)b * a.Hq + h0 + hh;
    load(a.q + head * a.T * D, q_s[buf], w, qb, Tb);
    load(a.dout + head * a.T * D, do_s[buf], w, qb, Tb);
    if (w == 0)      // lane l: four rows of scalar l / 16
      __builtin_amdgcn_global_load_lds(
          (const void*)(a.stats + (lane >> 4) * a.stat_step + head * a.Tp + qb * kGrT + 4 * (lane & 15)),
          (__attribute__((address_space(3))) void*)&st_s[buf][0][0], 16, 0, 0);
  };
  auto unit = [&](int row0, const uint16_t* qt, const uint16_t* dt, const float* st, auto masked_tag) {
    constexpr bool MASKED = decltype(masked_tag)::value;
    f32x16 s{}, dp;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const f32x4 nd = *reinterpret_cast<const f32x4*>(st + 2 * kGrT + 8 * x + 4 * g2);
#pragma unroll
      for (int i = 0; i < 4; ++i) dp[4 * x + i] = nd[i];
    }
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) s = mfma(rd.rows(qt, kc), kf[kc], s);
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) dp = mfma(rd.rows(dt, kc), vf[kc], dp);
    float p[16], ds[16];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const f32x4 nl = *reinterpret_cast<const f32x4*>(st + 8 * x + 4 * g2);
      const f32x4 bt = *reinterpret_cast<const f32x4*>(st + kGrT + 8 * x + 4 * g2);
      const f32x4 kap = *reinterpret_cast<const f32x4*>(st + 3 * kGrT + 8 * x + 4 * g2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = row0 + 8 * x + 4 * g2 + i;
        float n;
        score_grad<ADD, MASKED>(g, s[4 * x + i], bt[i] + g.lis2, ADD ? nl[i] - a.C * kLog2e : nl[i], nl[i],
                                dp[4 * x + i], kap[i], j <= row, j == row, p[4 * x + i], ds[4 * x + i], n);
      }
    }
    u32x4 pp[2], pd[2];
    pack_units(p, pp);
    pack_units(ds, pd);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        dva[db] = mfma(rd.turned(dt, c, db), pp[c], dva[db]);
        dka[db] = mfma(rd.turned(qt, c, db), pd[c], dka[db]);
      }
  };

  if (steps > 0) fetch(0, 0);
  for (int it = 0; it < steps; ++it) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (it + 1 < steps) fetch(it + 1, (it + 1) & 1);
    const int qb = nqb - 1 - it % nb, buf = it & 1;
#pragma unroll 1
    for (int x = 0; x < 2; ++x) {
      const int u = 2 * qb + x;
      if (u < ku) continue;
      const uint16_t *qt = q_s[buf] + x * 32 * D, *dt = do_s[buf] + x * 32 * D;
      const float* st = &st_s[buf][0][32 * x];
      if (u == ku) unit(32 * u, qt, dt, st, std::integral_constant<bool, true>{});
      else unit(32 * u, qt, dt, st, std::integral_constant<bool, false>{});
    }
  }

  if (j < a.T) {
    if (a.nsplit > 1) {
      float* o = a.part + (((int64_t)split * gridDim.z * a.Hkv + (int64_t)b * a.Hkv + kvh) * a.T + j) * D + 4 * g2;
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
  a.Hq = pd.num_q_heads;
  a.Hkv = pd.num_kv_heads;
  a.T = pd.capacity_tokens;
  a.Tp = p.rows;
  a.nsplit = p.nsplit;
  a.stat_step = (int64_t)pd.batch * pd.num_q_heads * p.rows;
  a.part_step = (int64_t)p.nsplit * pd.batch * pd.num_kv_heads * pd.capacity_tokens * pd.head_dim;
  a.beta = pd.beta;
  a.C = pd.additive ? pd.C : 0.f;
  const dim3 gq(p.blocks, pd.num_q_heads, pd.batch), gk(p.blocks, pd.num_kv_heads * p.nsplit, pd.batch);
  hipError_t e = with_hook(hook, ETA_KERNEL_PREFILL_GRAD_Q, stream, [&] {
    if (pd.additive) {
      if (pd.head_dim == 64) hipLaunchKernelGGL((grad_q_kernel<64, true>), gq, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((grad_q_kernel<128, true>), gq, dim3(256), 0, stream, a);
    } else {
      if (pd.head_dim == 64) hipLaunchKernelGGL((grad_q_kernel<64, false>), gq, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((grad_q_kernel<128, false>), gq, dim3(256), 0, stream, a);
    }
  });
  if (e != hipSuccess) return e;
  e = with_hook(hook, ETA_KERNEL_PREFILL_GRAD_KV, stream, [&] {
    if (pd.additive) {
      if (pd.head_dim == 64) hipLaunchKernelGGL((grad_kv_kernel<64, true>), gk, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((grad_kv_kernel<128, true>), gk, dim3(256), 0, stream, a);
    } else {
      if (pd.head_dim == 64) hipLaunchKernelGGL((grad_kv_kernel<64, false>), gk, dim3(256), 0, stream, a);
      else hipLaunchKernelGGL((grad_kv_kernel<128, false>), gk, dim3(256), 0, stream, a);
    }
  });
  if (e != hipSuccess || p.nsplit == 1) return e;
  const int64_t n4 = a.part_step / p.nsplit / 4;
  return with_hook(hook, ETA_KERNEL_PREFILL_GRAD_JOIN, stream, [&] {
    hipLaunchKernelGGL(grad_join_kernel, dim3((uint32_t)((n4 + 255) / 256), 2), dim3(256), 0, stream, a, n4);
  });
}

}  // namespace eta

// Split decode over a paged 8-bit cache (gfx950): the gated step's, over the union that screening
// left, and the dense one's, over every block.
//
//   S_t = s_k / sqrt(d) <q, c_t>,  S~_t = S_t sigmoid(beta (S_t - tau_eff))  (dense: S~ = S),
//   partial of a split: m = a reference maximum, l = sum 2^(x_t - m), acc = sum 2^(x_t - m) s_v v_t,
//   x_t = S~_t log2 e; the partials are merged as those of the contiguous caches are.
//
// A wavefront takes a unit of 64 tokens of a page at a time, on the matrix cores from end to end
// and without LDS.  Scores: A = 16 keys x 32 dims (codes widened to bf16, exactly), B = 32 dims x
// 16 columns, four tiles of 16 keys.  Row i of tile t is token 16 (i / 4) + 4 t + i % 4, so that
// the result hands lane (column, lane group g) the tokens 16 g + 4 t + r.  The columns repeat the
// group's heads (column G j + h: head h), and replica j takes the gate and the softmax of its
// share of the tiles alone, so that a lane has 4 scores (eight heads: 8) to work on, not 16 in a
// quarter of the lanes.  The weights are, as they lie, the B operand of p.V, with zeros for the
// other replicas' tokens: A = 16 dims x 32 tokens of V, which lies by dimension in the page, so
// that lane (dim, g) reads its 16 tokens with one 16-byte load.  The result is the output's
// transpose, columns as before: the softmax state and the rescaling stay in the lane, each replica
// has its own, and they are merged once at the end.  The contraction runs in the order the loads
// give (any order does that both operands share).
//
// The weights go to p.V as three bf16 parts, which keep all 24 bits, and fp32 queries to the scores as
// three too.  Two parts (16 bits) would be 2^-18 of a weight off, more than fp32 sums are: where weights
// nearly cancel that shows in bf16 outputs too, and one in a thousand of a long context's rounds the
// other way.  Two / three parts, us in a graph: 512K tokens 73.3 / 73.5, 16 x 64K 76.8 / 77.4, dense 8 x
// 32K 40.9 / 41.6, 16 x 3400 of 64 dims in groups of eight 19.2 / 19.8.
//
// Bound by HBM once the caches are long: without the gate, the softmax and p.V the same loads take
// the same time.  512K tokens, 4 kv heads, d = 128, 283.7 MB of a step's union: 49.2 us (5.8 TB/s; a
// device copy reads and writes 5.16); 8 ragged sequences of up to 32K, dense: 185 MB in 33.0 us;
// 16 of up to 64K, 232.5 MB of unions in 49.5 us.  Of these 4 to 6 us are the way to the first
// load (length, tile counts, union ids, page, keys: each needs the one before) and the merge; short
// calls are nothing else.  Tried and not faster: values a unit further ahead in a second buffer,
// eight wavefronts, three per SIMD, the merge by the last workgroup of a group instead of a launch
// (69 -> 82 us a step: every workgroup's release writes its L2 back).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eta_device.h"
#include "eta_index.h"
#include "eta_lanes.h"
#include "eta_page.h"
#include "eta_page_codes.h"

namespace eta {

struct PageSplitArgs {
  const void* q;
  const uint8_t* k;
  const uint8_t* v;
  const float* k_scale;
  const float* v_scale;
  const int32_t* table;
  const int32_t* seq_lens;
  const float* tau;
  const int32_t* ids;
  const int32_t* tile_cnt;
  float2* part_ml;           // [splits][G]
  float* part_acc;           // [splits][G][D]
  const float* resc_best;    // screening's window parts
  const int32_t* resc_info;
  const uint8_t* wbits;
  uint8_t* mask;
  int32_t* resc_out;
  int32_t* extra_union;
  int2* plan;
  const int32_t* head_cnt;
  void* out;
  int32_t* counts;
  int32_t* union_counts;
  PageGeom pg;
  int q_dtype;
  float beta, offset_a;
  int self_ungated;
  int c;                     // rescue window (blocks)
};

namespace {

constexpr int kMaxGroup = 8;                 // query heads of a kv head
constexpr int kItems = 256;                  // 64-token units resolved at a time
constexpr uint32_t kIdMask = 0x00ffffffu;    // union id: block index | head bits << 24
constexpr float kLog2e = 1.4426950408889634f;

// x in N bf16 parts, the largest first, as packed words: each part is the nearest to what the
// ones before it leave, so N = 2 keep 16 bits of x and N = 3 all 24.
template <int M, int N>
__device__ __forceinline__ void in_parts(const float (&x)[M], uint32_t (&out)[N][M / 2]) {
  float r[M];
#pragma unroll
  for (int e = 0; e < M; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < M; e += 2) {
      const uint32_t w = pack_bf16x2(r[e], r[e + 1]);
      out[n][e / 2] = w;
      if (n + 1 < N) {
        r[e] -= __uint_as_float(w << 16);
        r[e + 1] -= __uint_as_float(w & 0xffff0000u);
      }
    }
}
__device__ __forceinline__ bf16x8 as_bf16(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8, make_uint4(a, b, c, d));
}

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load16(const uint8_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ uint4 load16_nt(const uint8_t* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
}

// Exclusive prefix over the workgroup's threads; *total gets the sum.  Holds two barriers.
template <int kWaves>
__device__ __forceinline__ int block_excl_scan(int x, int* wsum, int* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int incl = wave_incl_scan(x);
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  int off = 0, tot = 0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    off += k < w ? wsum[k] : 0;
    tot += wsum[k];
  }
  __syncthreads();
  *total = tot;
  return off + incl - x;
}

// Online softmax in base 2 of one head (the lane's column), against a reference maximum m that
// moves only when a score passes it by more than 8 (t = m + 8; -inf before the first key).
// m and t are the same in a column's four lanes; l is the lane's share of the sum.
template <int D>
struct Column {
  float m, t, l;
  f32x4 acc[D / 16];
};

template <int D, bool DENSE, bool F32, int REP>
struct Attend {
  static constexpr int NQ = F32 ? 3 : 1;     // bf16 parts of the queries
  static constexpr int NP = 3;               // and of the weights
  static constexpr int NC = D / 32;          // steps of a score's contraction
  static constexpr int TS = 4 / REP;         // tiles of a replica
  static constexpr int NS = 4 * TS;          // scores of a lane
  bf16x8 q[NC][NQ];
  float s2, beta, bt;                        // log2 e / sqrt d; gate exponent: bt - beta x
  int lane, rep;                             // rep: the lane's replica (REP and more: idle)

  // This lane's share of the queries: head h's dims 64 k + 16 g + 8 e .. + 7 in step 2 k + e.
  __device__ __forceinline__ void load_q(const PageSplitArgs& a, int64_t row) {
    const int g4 = lane >> 4;
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      const int at = 64 * (s >> 1) + 16 * g4 + 8 * (s & 1);
      if constexpr (F32) {
        const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + row + at);
        const float4 u = p[0], w = p[1];
        const float x[8] = {u.x, u.y, u.z, u.w, w.x, w.y, w.z, w.w};
        uint32_t y[NQ][4];
        in_parts<8, NQ>(x, y);
#pragma unroll
        for (int n = 0; n < NQ; ++n) q[s][n] = as_bf16(y[n][0], y[n][1], y[n][2], y[n][3]);
      } else {
        q[s][0] = __builtin_bit_cast(
            bf16x8, *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.q) + row + at));
      }
    }
  }

  // The scores' products <q, c> of the lane's tokens.
  __device__ __forceinline__ void scores(const uint4 (&k)[4][D / 64], float (&c)[NS]) const {
    f32x4 all[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f32x4 part[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) part[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NC; ++s) {
        const uint4& x = k[t][s >> 1];
        const bf16x8 kb = (s & 1) ? widen(x.z, x.w) : widen(x.x, x.y);
#pragma unroll
        for (int n = 0; n < NQ; ++n) part[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, q[s][n], part[n], 0, 0, 0);
      }
      all[t] = part[NQ - 1];                 // the low parts' sums first
#pragma unroll
      for (int n = NQ - 2; n >= 0; --n) all[t] += part[n];
    }
#pragma unroll
    for (int e = 0; e < NS; ++e) {
      const int i = e >> 2, r = e & 3;
      if constexpr (REP == 4)
        c[e] = rep < 2 ? (rep == 0 ? all[0][r] : all[1][r]) : (rep == 2 ? all[2][r] : all[3][r]);
      else
        c[e] = rep == 0 ? all[i][r] : all[2 + i][r];
    }
  }

  // Scores -> weights.  n: tokens of the unit that are there; on: whether the lane's head
  // attends it; self: the unit's token that is not gated (or none of 0..63).
  __device__ __forceinline__ void weights(const float (&c)[NS], int n, bool on, int self, float ks,
                                          Column<D>& st, float (&p)[NS]) const {
    const int tok = 16 * (lane >> 4) + NS * rep;
    const int nl = on ? n - tok : 0, sl = self - tok;
    const float f = ks * s2;
    float y[NS], x[NS];
    bool over = false;
#pragma unroll
    for (int e = 0; e < NS; ++e) {
      y[e] = c[e];
      if constexpr (!DENSE) {
        const float sig = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(fmaf(-beta, c[e] * f, bt)));
        // (an open gate passes any score, -inf too, where the gate's own sum is NaN)
        y[e] = (e == sl || bt == kNegInf) ? c[e] : c[e] * sig;
      }
      x[e] = e < nl ? y[e] * f : kNegInf;
      over |= x[e] > st.t;
    }
    if (__ballot(over) != 0ull) {
      float bm = x[0];
#pragma unroll
      for (int e = 1; e < NS; ++e) bm = fmaxf(bm, x[e]);
      bm = fmaxf(bm, __shfl_xor(bm, 16, 64));
      bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
      const bool first = st.t == kNegInf;
      // (a reference is a number: where every score is NaN, the weights are)
      const float mn = first ? (bm > kNegInf ? bm : 0.f) : fmaxf(st.m, bm);
      const float alpha = first ? 1.0f : __builtin_amdgcn_exp2f(st.m - mn);   // (before the first key: of zeros)
      st.m = mn;
      if (!first || bm > kNegInf) st.t = mn + 8.0f;
      st.l *= alpha;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) st.acc[k] *= alpha;
    }
#pragma unroll
    for (int e = 0; e < NS; ++e) {
      p[e] = e < nl ? __builtin_amdgcn_exp2f(fmaf(y[e], f, -st.m)) : 0.f;
      st.l += p[e];
    }
  }

  __device__ __forceinline__ void values(const uint4 (&v)[D / 16], const float (&p)[NS], bool on, float vs,
                                         Column<D>& st) const {
    uint32_t y[NP][NS / 2];
    in_parts<NS, NP>(p, y);
    bf16x8 w[2][NP];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        if constexpr (REP == 4) {
          const bool lo = rep == 2 * m, hi = rep == 2 * m + 1;
          w[m][n] = as_bf16(lo ? y[n][0] : 0u, lo ? y[n][1] : 0u, hi ? y[n][0] : 0u, hi ? y[n][1] : 0u);
        } else {
          const bool in = rep == m;
          w[m][n] = as_bf16(in ? y[n][0] : 0u, in ? y[n][1] : 0u, in ? y[n][2] : 0u, in ? y[n][3] : 0u);
        }
      }
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const bf16x8 v0 = widen(v[k].x, v[k].y), v1 = widen(v[k].z, v[k].w);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = NP - 1; n >= 0; --n) {
        o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, w[0][n], o, 0, 0, 0);
        o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, w[1][n], o, 0, 0, 0);
      }
      // (a head that does not attend the unit takes nothing, whatever V holds there)
      if (on) {
#pragma unroll
        for (int r = 0; r < 4; ++r) st.acc[k][r] = fmaf(o[r], vs, st.acc[k][r]);
      }
    }
  }
};

// Tokens from n on of a unit's values weigh 0, but what lies there may be NaN: made zero.
template <int D>
__device__ __forceinline__ void clear_behind(uint4 (&v)[D / 16], int n, int lane) {
  const int nl = n - 16 * (lane >> 4);
  uint32_t keep[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int nv = nl - 4 * w;
    keep[w] = nv >= 4 ? ~0u : (nv <= 0 ? 0u : (1u << (8 * nv)) - 1u);
  }
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    v[k].x &= keep[0];
    v[k].y &= keep[1];
    v[k].z &= keep[2];
    v[k].w &= keep[3];
  }
}

__device__ __forceinline__ void store_o(void* o, int q_dtype, int64_t idx, float x) {
  if (q_dtype == ETA_DT_F32)
    reinterpret_cast<float*>(o)[idx] = x;
  else
    reinterpret_cast<__bf16*>(o)[idx] = (__bf16)x;
}

template <int D, int BS, bool DENSE, bool PROP, bool F32, int REP, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void page_split_kernel(PageSplitArgs a) {
  constexpr int kThreads = 64 * kWaves;
  constexpr int GPT = kPropMaxGroups / kThreads, CPT = kPropMaxCounts / kThreads;
  const Geom& g = a.pg.g;
  const int G = g.G, tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  constexpr int spb = BS >> 6, spb_log = BS >> 7;  // units of a block: 1 or 2
  __shared__ int wsum_s[kWaves];
  __shared__ int pref_s[DENSE ? 1 : (PROP ? kPropMaxCounts : kMaxTiles) + 1];
  __shared__ int own_s[3];
  __shared__ int item_page[kItems];
  __shared__ uint32_t item_meta[kItems];           // head bits | sub << 8 | tokens << 16 | own token << 24
  __shared__ float mrg_m[kWaves][16], mrg_l[kWaves][16], sum_s[kMaxGroup];
  __shared__ __attribute__((aligned(16))) float mrg_acc[kWaves][16][D];
  __shared__ float rbest_s[DENSE ? 1 : kMaxGroup][kRescueTiles];
  __shared__ int rinfo_s[DENSE ? 1 : kMaxGroup][kRescueTiles];
  __shared__ int resc_s[kMaxGroup], rxw_s[kMaxGroup], rx_s[kMaxGroup][2], nrx_s;

  // ---- which (sequence, kv head) and which split of it.  Uniform plan: grid (S, Hkv, B).
  // Proportional plan (several sequences): a 1-D grid dealt to the groups by their units.  Loads
  // that do not wait for each other are requested together: a step on its own is mostly their
  // round trips.
  int b, gh, s, S, first, UI, tc0 = 0;
  int pbase = 0;                     // the group's tile prefix is pref[], offset by pbase
  const int* pref = pref_s;
  const int32_t* tc = nullptr;
  if constexpr (!PROP) {
    s = blockIdx.x;
    gh = blockIdx.y;
    b = blockIdx.z;
    S = gridDim.x;
    first = (b * g.Hkv + gh) * S;
    if constexpr (!DENSE) {
      tc = a.tile_cnt + ((int64_t)b * g.Hkv + gh) * g.n_tiles;
      tc0 = tid < g.n_tiles ? tc[tid] : 0;
    }
  } else {
    const int BG = g.B * g.Hkv, nct = g.n_tiles, nc = BG * nct, W = gridDim.x, me = blockIdx.x;
    if (tid == 0) own_s[0] = -1;
    int work[GPT], len[GPT], cv[CPT], tot;
    if constexpr (!DENSE) {
#pragma unroll
      for (int k = 0; k < CPT; ++k) {
        const int i = tid * CPT + k;
        cv[k] = a.tile_cnt[i < nc ? i : 0];
      }
    }
    {
      GroupStepper gs((unsigned)(tid * GPT), 1u, (unsigned)g.Hkv);
#pragma unroll
      for (int r = 0; r < GPT; ++r) {
        len[r] = a.seq_lens[tid * GPT + r < BG ? gs.q : 0u];
        gs.next();
      }
    }
    // (all of them are needed here, so that none is moved into a branch)
#pragma unroll
    for (int r = 0; r < GPT; ++r) asm volatile("" ::"v"(len[r]));
    if constexpr (!DENSE) {
      int run = 0;
#pragma unroll
      for (int k = 0; k < CPT; ++k) {
        const int x = tid * CPT + k < nc ? cv[k] : 0;
        cv[k] = run;
        run += x;
      }
      const int ex = block_excl_scan<kWaves>(run, wsum_s, &tot);
#pragma unroll
      for (int k = 0; k < CPT; ++k) pref_s[tid * CPT + k] = ex + cv[k];
      if (tid == 0) pref_s[kPropMaxCounts] = tot;
      __syncthreads();
    }
    // the groups' units (thread tid: groups GPT tid ..), and splits in proportion to them
    int mine = 0;
#pragma unroll
    for (int r = 0; r < GPT; ++r) {
      const int x = tid * GPT + r;
      work[r] = 0;
      if (x < BG) {
        const int64_t t = len[r] < 0 ? 0 : (len[r] > g.cap ? g.cap : len[r]);
        const int blocks = DENSE ? (int)(t / BS) : pref_s[(x + 1) * nct] - pref_s[x * nct];
        work[r] = group_work(blocks, spb, t, BS);
      }
      mine += work[r];
    }
    block_excl_scan<kWaves>(mine, wsum_s, &tot);
    int nsp[GPT], sum = 0, dummy;
#pragma unroll
    for (int r = 0; r < GPT; ++r) {
      nsp[r] = tid * GPT + r < BG ? group_splits(work[r], tot, W, BG) : 0;
      sum += nsp[r];
    }
    int f = block_excl_scan<kWaves>(sum, wsum_s, &dummy);
#pragma unroll
    for (int r = 0; r < GPT; ++r) {
      if (tid * GPT + r < BG && owns_split(f, nsp[r], me)) {
        own_s[0] = tid * GPT + r;
        own_s[1] = f;
        own_s[2] = nsp[r];
      }
      f += nsp[r];
    }
    __syncthreads();
    const int x = own_s[0];
    if (x < 0) return;               // past the allocation (the whole workgroup)
    b = x / g.Hkv;
    gh = x % g.Hkv;
    first = own_s[1];
    s = me - first;
    S = own_s[2];
    if constexpr (!DENSE) {
      pref = pref_s + x * nct;
      pbase = pref[0];
      UI = pref[nct] - pbase;
    }
    if (s == 0 && tid == 0) a.plan[x] = make_int2(first, S);
  }
  const int64_t hq0 = (int64_t)b * g.Hq + (int64_t)gh * G, bg = (int64_t)b * g.Hkv + gh;
  const bool single = !PROP && S == 1;             // no partials, no combine
  const int col = lane & 15, head = col % G;       // (G divides 16)
  Attend<D, DENSE, F32, REP> at;
  at.lane = lane;
  at.rep = col / G;
  at.s2 = kLog2e / sqrtf((float)D);
  at.beta = a.beta;
  at.bt = kNegInf;
  int t_raw = a.seq_lens[b];
  float tau = 0.f, rb = 0.f;
  int ri = 0;
  if constexpr (!DENSE) {
    tau = a.tau[hq0 + head];
    // (the parts of every window tile: those past the window are not used)
    const int64_t e = hq0 * kRescueTiles + (tid < G * kRescueTiles ? tid : 0);
    rb = a.resc_best[e];
    ri = a.resc_info[e];
  }
  at.load_q(a, (hq0 + head) * D);
  asm volatile("" : "+v"(t_raw) : "v"(tau), "v"(rb), "v"(ri), "v"(tc0));
  t_raw = __builtin_amdgcn_readfirstlane(t_raw);
  const int64_t T = t_raw < 0 ? 0 : (t_raw > g.cap ? g.cap : (int64_t)t_raw);
  const int64_t N = T / BS;
  const int ntail = (int)(T - N * BS);
  if constexpr (DENSE) UI = (int)N;
  if constexpr (!DENSE) {
    const float teff = tau - a.offset_a;
    at.bt = teff == kNegInf ? kNegInf : a.beta * teff * kLog2e;
    if (tid < G * kRescueTiles) {
      rbest_s[tid / kRescueTiles][tid % kRescueTiles] = rb;
      rinfo_s[tid / kRescueTiles][tid % kRescueTiles] = ri;
    }
    if constexpr (!PROP) {
      int carry = 0;
      for (int base = 0; base < g.n_tiles; base += kThreads) {
        const int t = base + tid;
        int tot;
        const int ex = block_excl_scan<kWaves>(base == 0 ? tc0 : (t < g.n_tiles ? tc[t] : 0), wsum_s, &tot);
        if (t < g.n_tiles) pref_s[t] = carry + ex;
        carry += tot;
      }
      if (tid == 0) pref_s[g.n_tiles] = carry;
      UI = carry;
    }
    __syncthreads();
  }

  // ---- top-1 rescue: for each head, when no block of the window is selected, the first of the
  // window's largest bounds (tiles in order) is attended too; each distinct one is a further item
  // of the list, with the heads that rescued it
  int jr_h = -1, wb_rescued = 1, nrx = 0;
  const int UI_union = UI;
  if constexpr (!DENSE) {
    const int64_t Wn = (int64_t)a.c < N ? (int64_t)a.c : N;
    const int nwt = (int)((Wn + kScreenTile - 1) / kScreenTile);
    if (lane < G) {                  // (every wavefront, so that all know whether there is any)
      float best = kNegInf;
      bool any = false;
      for (int t = 0; t < nwt; ++t) {
        const int inf = rinfo_s[lane][t];
        const float v = rbest_s[lane][t];
        if (inf == kRescueAny) {
          any = true;
        } else if (inf >= 0 && (jr_h < 0 || v > best)) {
          best = v;
          jr_h = inf;
        }
      }
      if (any) jr_h = -1;
    }
    if (__ballot(jr_h >= 0) != 0ull) {
      if (tid < G) {
        resc_s[tid] = jr_h;
        if (s == S - 1 && jr_h >= 0) wb_rescued = a.wbits[bg * kMaxRescueWindow + jr_h];
      }
      __syncthreads();
      if (tid == 0) {
        int nb = 0;
        for (int h = 0; h < G; ++h) {
          const int j = resc_s[h];
          if (j < 0) continue;
          int k = 0;
          while (k < nb && rx_s[k][0] != j) ++k;
          if (k == nb) {
            rx_s[nb][0] = j;
            rx_s[nb][1] = 0;
            ++nb;
          }
          rx_s[k][1] |= 1 << h;
        }
        nrx_s = nb;
      }
      __syncthreads();
      nrx = nrx_s;
      UI += nrx;
    }
  }

  // ---- the list: its items' blocks, then the tail.  This split has items s, s + S, ..; the units
  // of an item are neighbours, so that the wavefronts that take them read the halves of V's lines
  // (blocks of 128 tokens) at about the same time
  const uint32_t all_bits = (1u << G) - 1u;
  const int total = UI + (ntail > 0);
  const int64_t self_t = (!DENSE && a.self_ungated) ? T - 1 : -1;
  const int32_t* row = a.table + (int64_t)b * a.pg.table_stride;
  auto resolve = [&](int unit, int slot) {
    const int it = s + S * (unit >> spb_log), sub = unit & (spb - 1);
    int64_t j = it;
    int n = 64;
    uint32_t bits = all_bits;
    if (it >= UI) {
      j = N;
      n = ntail - 64 * sub;
      n = n < 0 ? 0 : (n > 64 ? 64 : n);
    } else if constexpr (!DENSE) {
      if (it >= UI_union) {
        j = rx_s[it - UI_union][0];
        bits = (uint32_t)rx_s[it - UI_union][1];
      } else {
        int tl, sl;
        resolve_item(pref, g.n_tiles, it + pbase, &tl, &sl);
        const uint32_t id = (uint32_t)a.ids[bg * g.ncap + (int64_t)tl * kScreenTile + sl];
        j = id & kIdMask;
        bits = id >> 24;
      }
    }
    int64_t page = page_of(row, j, a.pg.table_blocks, a.pg.pages);
    if (page < 0) {                  // no page: nothing of it is attended, page 0 is read in its place
      page = 0;
      n = 0;
    }
    const int64_t own = self_t - (j * BS + 64 * sub);
    item_page[slot] = (int)page;
    item_meta[slot] = bits | (uint32_t)sub << 8 | (uint32_t)n << 16 | (own >= 0 && own < 64 ? (uint32_t)own : 255u) << 24;
  };

  Column<D> st;
  st.m = st.l = 0.f;
  st.t = kNegInf;
#pragma unroll
  for (int k = 0; k < D / 16; ++k) st.acc[k] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int g4 = lane >> 4;
  const int64_t head_off = (int64_t)gh * BS * D;
  const uint8_t* kl = a.k + head_off + (16 * (col >> 2) + (col & 3)) * D + 16 * g4;
  const uint8_t* vl = a.v + head_off + col * BS + 16 * g4;
  uint4 kr[4][D / 64], vr[D / 16];
  auto load_k = [&](int64_t off) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int h = 0; h < D / 64; ++h) kr[t][h] = load16(kl + off + 4 * t * D + 64 * h);
  };
  // (a block's 64 tokens of a row of V: whole lines, read once, past the caches; halves of the
  // lines of 128 tokens, whose other halves a neighbour reads, through them)
  auto load_v = [&](int64_t off) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      if constexpr (BS == 64)
        vr[k] = load16_nt(vl + off + 16 * k * BS);
      else
        vr[k] = load16(vl + off + 16 * k * BS);
    }
  };
  // The unit that is worked on and the next one: page, part of the block, the page's scales (which
  // come while its keys do).
  int64_t at_n = 0;                  // the next unit's page
  int sub_n = 0;
  float ks_n = 0.f, vs_n = 0.f;
  auto next = [&](int x) {
    at_n = __builtin_amdgcn_readfirstlane(item_page[x]);
    sub_n = (__builtin_amdgcn_readfirstlane(item_meta[x]) >> 8) & 255;
    ks_n = a.k_scale[at_n * a.pg.scale_stride + gh];
    vs_n = a.v_scale[at_n * a.pg.scale_stride + gh];
  };
  // The next unit's keys are requested as soon as this one's scores have taken theirs, its values
  // when p.V has.  The last unit is peeled (more false), so that the loads in the loop are
  // unconditional.
  auto unit = [&](int x, auto more_tag) {
    constexpr bool more = decltype(more_tag)::value;
    const uint32_t meta = __builtin_amdgcn_readfirstlane(item_meta[x]);
    const float ks = ks_n, vs = vs_n;
    const int n = (meta >> 16) & 255;
    // (a unit without a page is not attended: what was read in its place weighs nothing, NaN or not)
    const bool on = at.rep < REP && n > 0 && ((meta >> head) & 1u);
    constexpr int NS = Attend<D, DENSE, F32, REP>::NS;
    float c[NS], p[NS];
    if constexpr (more) next(x + kWaves);
    at.scores(kr, c);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (more) load_k(at_n * a.pg.page_stride + sub_n * 64 * D);
    __builtin_amdgcn_sched_barrier(0);
    at.weights(c, n, on, (int)(meta >> 24), ks, st, p);
    if (n < 64) clear_behind<D>(vr, n, lane);
    at.values(vr, p, on, vs, st);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (more) load_v(at_n * a.pg.page_stride + sub_n * 64);
    __builtin_amdgcn_sched_barrier(0);
  };
  const int nt = strided_share(total, s, S) * spb;
  for (int k0 = 0; k0 < nt; k0 += kItems) {
    const int n = nt - k0 < kItems ? nt - k0 : kItems;
    if (tid < n) resolve(k0 + tid, tid);
    __syncthreads();
    if (w < n) {
      next(w);
      load_k(at_n * a.pg.page_stride + sub_n * 64 * D);
      load_v(at_n * a.pg.page_stride + sub_n * 64);
      int x = w;
      for (; x + kWaves < n; x += kWaves) unit(x, std::integral_constant<bool, true>{});
      unit(x, std::integral_constant<bool, false>{});
    }
    __syncthreads();
  }

  if constexpr (!DENSE) {
    if (s == S - 1) {
      // the rescued blocks' mask bits; each head's rescued block and how many are outside the union
      int extra = 0;
      if (nrx > 0) {
        if (tid < G) rxw_s[tid] = jr_h >= 0 ? wb_rescued : 1;
        __syncthreads();
        for (int k = 0; k < nrx; ++k) {
          bool in_union = false;
          for (int h = 0; h < G; ++h) in_union |= resc_s[h] == rx_s[k][0] && rxw_s[h] != 0;
          extra += !in_union;
        }
        if (tid < G && jr_h >= 0) a.mask[(hq0 + tid) * g.ncap + jr_h] = 1;
      }
      if (tid == 0) {
        if (!single)
          a.extra_union[bg] = extra;
        else if (a.union_counts != nullptr)
          a.union_counts[bg] = UI_union + extra;
      }
      if (!single && tid < G) a.resc_out[hq0 + tid] = jr_h;
    }
  }

  // ---- merge of the wavefronts' replicas
  st.l += __shfl_xor(st.l, 16, 64);
  st.l += __shfl_xor(st.l, 32, 64);
  if (g4 == 0) {
    // (no key: no weight; keys whose scores are all NaN leave t as it was, and a sum of NaN)
    mrg_m[w][col] = st.t == kNegInf && st.l == 0.f ? kNegInf : st.m;
    mrg_l[w][col] = st.l;
  }
#pragma unroll
  for (int k = 0; k < D / 16; ++k) *reinterpret_cast<f32x4*>(&mrg_acc[w][col][16 * k + 4 * g4]) = st.acc[k];
  __syncthreads();
  // wavefront 0, lane (w', column): the weights of the replicas of wavefronts w', w' + 4, ..; the
  // heads' maxima and sums
  if (w == 0) {
    float mk[kWaves / 4], ms = kNegInf, L = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves / 4; ++k) {
      mk[k] = mrg_m[4 * k + g4][col];
      ms = fmaxf(ms, mk[k]);
    }
    for (int o = G; o < 64; o <<= 1) ms = fmaxf(ms, __shfl_xor(ms, o, 64));
#pragma unroll
    for (int k = 0; k < kWaves / 4; ++k) {
      const float wk = mk[k] == kNegInf ? 0.f : __builtin_amdgcn_exp2f(mk[k] - ms);
      if (mk[k] != kNegInf) L = fmaf(wk, mrg_l[4 * k + g4][col], L);
      mrg_m[4 * k + g4][col] = wk;
    }
    for (int o = G; o < 64; o <<= 1) L += __shfl_xor(L, o, 64);
    if (lane < G) {
      sum_s[lane] = L;
      // (the merge takes a sum that is not positive for no key: NaN goes on in the accumulators)
      if (!single) a.part_ml[(int64_t)(first + s) * G + lane] = make_float2(ms, L != L ? 1.0f : L);
    }
  }
  __syncthreads();
  for (int idx = tid; idx < G * D; idx += kThreads) {
    const int h = idx / D, i = idx % D;
    float o = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k)
#pragma unroll
      for (int j = 0; j < REP; ++j) o = fmaf(mrg_acc[k][j * G + h][i], mrg_m[k][j * G + h], o);
    const float L = sum_s[h];
    if (single) {
      store_o(a.out, a.q_dtype, (hq0 + h) * D + i, L == 0.f ? 0.f : o / L);
    } else {
      a.part_acc[((int64_t)(first + s) * G + h) * D + i] = L != L ? L : o;
    }
  }
  if constexpr (!DENSE) {
    if (single && a.counts != nullptr) {
      for (int h = w; h < G; h += kWaves) {
        int cnt = 0;
        for (int t = lane; t < g.n_tiles; t += 64) cnt += a.head_cnt[(hq0 + h) * g.n_tiles + t];
#pragma unroll
        for (int o2 = 32; o2 > 0; o2 >>= 1) cnt += __shfl_xor(cnt, o2, 64);
        if (lane == 0) a.counts[hq0 + h] = (int32_t)(((int64_t)cnt + (nrx > 0 && resc_s[h] >= 0 ? 1 : 0)) * BS + ntail);
      }
    }
  }
}

template <bool DENSE>
void launch_split(const PageSplitArgs& a, const SplitPlan& pl, hipStream_t stream) {
  const Geom& g = a.pg.g;
  const dim3 grid = pl.S > 0 ? dim3(pl.S, g.Hkv, g.B) : dim3(pl.W);
#define ETA_PSPL_R(D_, BS_, P_, F_, R_, W_) \
  hipLaunchKernelGGL((page_split_kernel<D_, BS_, DENSE, P_, F_, R_, W_>), grid, dim3(64 * W_), 0, stream, a);
#define ETA_PSPL(D_, BS_, P_, F_)                                                          \
  if (g.D == D_ && g.BS == BS_ && (pl.S == 0) == P_ && (a.q_dtype == ETA_DT_F32) == F_) {  \
    if (g.G == 8) {                                                                        \
      if (pl.S == 1) ETA_PSPL_R(D_, BS_, false, F_, 2, 8)                                  \
      else ETA_PSPL_R(D_, BS_, P_, F_, 2, 4)                                               \
    } else {                                                                               \
      if (pl.S == 1) ETA_PSPL_R(D_, BS_, false, F_, 4, 8)                                  \
      else ETA_PSPL_R(D_, BS_, P_, F_, 4, 4)                                               \
    }                                                                                      \
  }
#define ETA_PSPL_P(D_, BS_)                                           \
  ETA_PSPL(D_, BS_, false, false) ETA_PSPL(D_, BS_, false, true)      \
  ETA_PSPL(D_, BS_, true, false) ETA_PSPL(D_, BS_, true, true)
  ETA_PSPL_P(64, 64) ETA_PSPL_P(64, 128) ETA_PSPL_P(128, 64) ETA_PSPL_P(128, 128)
#undef ETA_PSPL_P
#undef ETA_PSPL
#undef ETA_PSPL_R
}

}  // namespace

hipError_t launch_page_split(const PageGeom& pg, const DecodeCfg& c, int q_dtype, const void* q,
                             const eta_page_pool_t& pool, const int32_t* table, const int32_t* seq_lens,
                             const float* tau, void* out, uint8_t* mask, int32_t* counts,
                             int32_t* union_counts, const DecodeWs& ws, hipStream_t stream, LaunchHook hook) {
  const PageSplitArgs a{q, (const uint8_t*)pool.k, (const uint8_t*)pool.v, pool.k_scale, pool.v_scale, table,
                        seq_lens, tau, ws.ids, ws.tile_cnt, ws.part_ml, ws.part_acc, ws.resc_best, ws.resc_info,
                        ws.wbits, mask, ws.resc_out, ws.extra_union, ws.plan, ws.head_cnt, out, counts,
                        union_counts, pg, q_dtype, c.beta, c.offset_a, c.self_ungated, c.rescue_window};
  return with_hook(hook, ETA_KERNEL_PAGE_SPLIT, stream, [&] { launch_split<false>(a, c.plan, stream); });
}

hipError_t launch_page_dense(const PageGeom& pg, const SplitPlan& plan, int q_dtype, const void* q,
                             const eta_page_pool_t& pool, const int32_t* table, const int32_t* seq_lens,
                             void* out, const DecodeWs& ws, hipStream_t stream, LaunchHook hook) {
  const PageSplitArgs a{q, (const uint8_t*)pool.k, (const uint8_t*)pool.v, pool.k_scale, pool.v_scale, table,
                        seq_lens, nullptr, nullptr, nullptr, ws.part_ml, ws.part_acc, nullptr, nullptr, nullptr,
                        nullptr, nullptr, nullptr, ws.plan, nullptr, out, nullptr, nullptr, pg, q_dtype, 0.f,
                        0.f, 0, 0};
  return with_hook(hook, ETA_KERNEL_PAGE_DENSE_SPLIT, stream, [&] { launch_split<true>(a, plan, stream); });
}

}  // namespace eta

// Split decode over a paged 8-bit cache (gfx950): the gated step's, over the union that screening
// left, and the dense one's, over every block.
//
//   S_t = s_k / sqrt(d) <q, c_t>,  S~_t = S_t sigmoid(beta (S_t - tau_eff))  (dense: S~ = S),
//   partial of a split: m = a reference maximum, l = sum 2^(x_t - m), acc = sum 2^(x_t - m) s_v v_t,
//   x_t = S~_t log2 e; the partials are merged as those of the contiguous caches are.
//
// A wavefront takes 64 tokens of a page at a time, on the matrix cores from end to end and
// without LDS.  Scores: A = 16 keys x 32 dims (codes widened to bf16, exactly), B = 32 dims x 16
// query heads (columns past the group's heads are zero), four tiles of 16 keys.  Row i of tile t
// is token 16 (i / 4) + 4 t + i % 4, so that the result hands lane (column c, lane group g) the
// 16 consecutive tokens 16 g .. 16 g + 15 of head c, which after the gate and the softmax are,
// as they lie, the B operand of p.V: A = 16 dims x 32 tokens of V, B = 32 tokens x 16 heads.  V
// lies by dimension in the page, so lane (dim, g) reads its 16 tokens with one 16-byte load, and
// the result is the output's transpose, whose columns are heads again: the softmax state and the
// rescaling stay in the lane.  The contraction runs in the order the loads give (any order does
// that both operands share).
//
// The weights go to p.V as two bf16 parts (16 bits), and fp32 queries as three with weights of
// three: MFMA time is not what bounds these kernels.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eta_device.h"
#include "eta_index.h"
#include "eta_lanes.h"
#include "eta_page.h"

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

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kMaxGroup = 8;                 // query heads of a kv head
constexpr int kItems = 256;                  // 64-token units resolved at a time
constexpr uint32_t kIdMask = 0x00ffffffu;    // union id: block index | head bits << 24
constexpr float kLog2e = 1.4426950408889634f;

// Eight codes -> eight bf16, exactly.
__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b) {
  union {
    bf16x2_t p[4];
    bf16x8 v;
  } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  return u.v;
}

// x in N bf16 parts, the largest first: each is the nearest to what the ones before it leave, so
// N = 2 keep 16 bits of x and N = 3 all 24.
template <int N>
__device__ __forceinline__ void in_parts(const float (&x)[8], bf16x8 (&out)[N]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    union {
      uint32_t w[4];
      bf16x8 v;
    } u;
#pragma unroll
    for (int e = 0; e < 8; e += 2) u.w[e / 2] = pack_bf16x2(r[e], r[e + 1]);
    out[n] = u.v;
    if (n + 1 < N) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        r[e] -= __uint_as_float(u.w[e / 2] << 16);
        r[e + 1] -= __uint_as_float(u.w[e / 2] & 0xffff0000u);
      }
    }
  }
}

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load16(const uint8_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ uint4 load16_nt(const uint8_t* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p)));
}

// Exclusive prefix over the workgroup's threads; *total gets the sum.  Holds two barriers.
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

// One unit of 64 tokens as its loads left it, with what the loop has to know of it.
template <int D>
struct Unit {
  uint4 k[4][D / 64];
  uint4 v[D / 16];
};

template <int D, bool DENSE, bool F32>
struct Attend {
  static constexpr int NQ = F32 ? 3 : 1;     // bf16 parts of the queries
  static constexpr int NP = F32 ? 3 : 2;     // and of the weights
  static constexpr int NC = D / 32;          // steps of a score's contraction
  bf16x8 q[NC][NQ];
  float s2, beta, bt;                        // log2 e / sqrt d; gate exponent: bt - beta x
  int lane;

  // This lane's share of the queries: column c's dims 64 h + 16 g + 8 e .. + 7 in step 2 h + e.
  __device__ __forceinline__ void load_q(const PageSplitArgs& a, int64_t hq0, int G) {
    const int col = lane & 15, g4 = lane >> 4;
    const bool in = col < G;
    const int64_t row = (hq0 + (in ? col : 0)) * D;
#pragma unroll
    for (int s = 0; s < NC; ++s) {
      const int at = 64 * (s >> 1) + 16 * g4 + 8 * (s & 1);
      if constexpr (F32) {
        const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + row + at);
        const float4 u = p[0], w = p[1];
        const float x[8] = {in ? u.x : 0.f, in ? u.y : 0.f, in ? u.z : 0.f, in ? u.w : 0.f,
                            in ? w.x : 0.f, in ? w.y : 0.f, in ? w.z : 0.f, in ? w.w : 0.f};
        in_parts<NQ>(x, q[s]);
      } else {
        uint4 u = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.q) + row + at);
        if (!in) u = make_uint4(0u, 0u, 0u, 0u);
        q[s][0] = __builtin_bit_cast(bf16x8, u);
      }
    }
  }

  __device__ __forceinline__ void scores(const Unit<D>& u, f32x4 (&c)[4]) const {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f32x4 part[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) part[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NC; ++s) {
        const uint4& x = u.k[t][s >> 1];
        const bf16x8 kb = (s & 1) ? widen(x.z, x.w) : widen(x.x, x.y);
#pragma unroll
        for (int n = 0; n < NQ; ++n) part[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, q[s][n], part[n], 0, 0, 0);
      }
      c[t] = part[NQ - 1];                   // the low parts' sums first
#pragma unroll
      for (int n = NQ - 2; n >= 0; --n) c[t] += part[n];
    }
  }

  // Scores -> weights.  n: tokens of the unit that are there; on: whether the lane's head
  // attends it; self: the unit's token that is not gated (or none of 0..63).
  __device__ __forceinline__ void weights(const f32x4 (&c)[4], int n, bool on, int self, float ks,
                                          Column<D>& st, float (&p)[16]) const {
    const int nl = on ? n - 16 * (lane >> 4) : 0, sl = self - 16 * (lane >> 4);
    const float f = ks * s2;
    float y[16], x[16];
    bool over = false;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float ce = c[e >> 2][e & 3];
      y[e] = ce;
      if constexpr (!DENSE) {
        const float sig = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(fmaf(-beta, ce * f, bt)));
        // (an open gate passes any score, -inf too, where the gate's own sum is NaN)
        y[e] = (e == sl || bt == kNegInf) ? ce : ce * sig;
      }
      x[e] = e < nl ? y[e] * f : kNegInf;
      over |= x[e] > st.t;
    }
    if (__ballot(over) != 0ull) {
      float bm = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) bm = fmaxf(bm, x[e]);
      bm = fmaxf(bm, __shfl_xor(bm, 16, 64));
      bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
      const bool first = st.t == kNegInf;
      const float mn = first ? (bm == kNegInf ? 0.f : bm) : fmaxf(st.m, bm);
      const float alpha = first ? 1.0f : __builtin_amdgcn_exp2f(st.m - mn);   // (before the first key: of zeros)
      st.m = mn;
      if (!first || bm != kNegInf) st.t = mn + 8.0f;
      st.l *= alpha;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) st.acc[k] *= alpha;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = e < nl ? __builtin_amdgcn_exp2f(fmaf(y[e], f, -st.m)) : 0.f;
      st.l += p[e];
    }
  }

  __device__ __forceinline__ void values(const Unit<D>& u, const float (&p)[16], bool on, float vs,
                                         Column<D>& st) const {
    bf16x8 w[2][NP];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = p[8 * m + e];
      in_parts<NP>(x, w[m]);
    }
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const bf16x8 v0 = widen(u.v[k].x, u.v[k].y), v1 = widen(u.v[k].z, u.v[k].w);
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
__device__ __forceinline__ void clear_behind(Unit<D>& u, int n, int lane) {
  const int nl = n - 16 * (lane >> 4);
  uint32_t keep[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int nv = nl - 4 * w;
    keep[w] = nv >= 4 ? ~0u : (nv <= 0 ? 0u : (1u << (8 * nv)) - 1u);
  }
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    u.v[k].x &= keep[0];
    u.v[k].y &= keep[1];
    u.v[k].z &= keep[2];
    u.v[k].w &= keep[3];
  }
}

__device__ __forceinline__ void store_o(void* o, int q_dtype, int64_t idx, float x) {
  if (q_dtype == ETA_DT_F32)
    reinterpret_cast<float*>(o)[idx] = x;
  else
    reinterpret_cast<__bf16*>(o)[idx] = (__bf16)x;
}

template <int D, bool DENSE, bool PROP, bool F32>
__global__ __launch_bounds__(kThreads, 2) void page_split_kernel(PageSplitArgs a) {
  constexpr int GPT = kPropMaxGroups / kThreads, CPT = kPropMaxCounts / kThreads;
  const Geom& g = a.pg.g;
  const int G = g.G, BS = g.BS, tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  const int spb = BS >> 6, spb_log = BS >> 7;      // units of a block: 1 or 2
  __shared__ int wsum_s[kWaves];
  __shared__ int pref_s[DENSE ? 1 : (PROP ? kPropMaxCounts : kMaxTiles) + 1];
  __shared__ int own_s[3];
  __shared__ int item_page[kItems];
  __shared__ uint32_t item_meta[kItems];           // head bits | sub << 8 | tokens << 16 | own token << 24
  __shared__ float item_ks[kItems], item_vs[kItems];
  __shared__ float mrg_ml[kWaves][kMaxGroup][2];
  __shared__ __attribute__((aligned(16))) float mrg_acc[kWaves][kMaxGroup][D];
  __shared__ int resc_s[kMaxGroup], rxw_s[kMaxGroup], rx_s[kMaxGroup][2], nrx_s;

  // ---- which (sequence, kv head) and which split of it.  Uniform plan: grid (S, Hkv, B).
  // Proportional plan (several sequences): a 1-D grid dealt to the groups by their units.
  int b, gh, s, S, first, UI;
  int pbase = 0;                     // the group's prefix within pref_s starts at pref0, offset by pbase
  const int* pref = pref_s;
  if constexpr (!PROP) {
    s = blockIdx.x;
    gh = blockIdx.y;
    b = blockIdx.z;
    S = gridDim.x;
    first = (b * g.Hkv + gh) * S;
    if constexpr (!DENSE) {
      const int32_t* tc = a.tile_cnt + ((int64_t)b * g.Hkv + gh) * g.n_tiles;
      int carry = 0;
      for (int base = 0; base < g.n_tiles; base += kThreads) {
        const int t = base + tid;
        int tot;
        const int ex = block_excl_scan(t < g.n_tiles ? tc[t] : 0, wsum_s, &tot);
        if (t < g.n_tiles) pref_s[t] = carry + ex;
        carry += tot;
      }
      if (tid == 0) pref_s[g.n_tiles] = carry;
      UI = carry;
    }
  } else {
    const int BG = g.B * g.Hkv, nct = g.n_tiles, nc = BG * nct, W = gridDim.x, me = blockIdx.x;
    if (tid == 0) own_s[0] = -1;
    int work[GPT], tot;
    if constexpr (!DENSE) {
      int cv[CPT], run = 0;
#pragma unroll
      for (int k = 0; k < CPT; ++k) {
        const int i = tid * CPT + k;
        cv[k] = a.tile_cnt[i < nc ? i : 0];
      }
#pragma unroll
      for (int k = 0; k < CPT; ++k) {
        const int x = tid * CPT + k < nc ? cv[k] : 0;
        cv[k] = run;
        run += x;
      }
      const int ex = block_excl_scan(run, wsum_s, &tot);
#pragma unroll
      for (int k = 0; k < CPT; ++k) pref_s[tid * CPT + k] = ex + cv[k];
      if (tid == 0) pref_s[kPropMaxCounts] = tot;
      __syncthreads();
    }
    // the groups' units (thread tid: groups GPT tid ..), and splits in proportion to them
    int mine = 0;
    GroupStepper gs((unsigned)(tid * GPT), 1u, (unsigned)g.Hkv);
#pragma unroll
    for (int r = 0; r < GPT; ++r) {
      const int x = tid * GPT + r;
      work[r] = 0;
      if (x < BG) {
        const int64_t len = clamp_len(a.seq_lens, (int)gs.q, g.cap);
        const int blocks = DENSE ? (int)(len / BS) : pref_s[(x + 1) * nct] - pref_s[x * nct];
        work[r] = group_work(blocks, spb, len, BS);
      }
      mine += work[r];
      gs.next();
    }
    block_excl_scan(mine, wsum_s, &tot);
    int nsp[GPT], sum = 0, dummy;
#pragma unroll
    for (int r = 0; r < GPT; ++r) {
      nsp[r] = tid * GPT + r < BG ? group_splits(work[r], tot, W, BG) : 0;
      sum += nsp[r];
    }
    int f = block_excl_scan(sum, wsum_s, &dummy);
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
  const int64_t T = clamp_len(a.seq_lens, b, g.cap);
  const int64_t N = T / BS;
  const int ntail = (int)(T - N * BS);
  if constexpr (DENSE) UI = (int)N;

  Attend<D, DENSE, F32> at;
  at.lane = lane;
  at.s2 = kLog2e / sqrtf((float)D);
  at.beta = a.beta;
  at.bt = kNegInf;
  at.load_q(a, hq0, G);
  const int col = lane & 15;
  if constexpr (!DENSE) {
    const float teff = (col < G ? a.tau[hq0 + col] : 0.f) - a.offset_a;
    at.bt = teff == kNegInf ? kNegInf : a.beta * teff * kLog2e;
  }

  // ---- top-1 rescue: for each head, when no block of the window is selected, the first of the
  // window's largest bounds (tiles in order) is attended too; each distinct one is a further item
  // of the list, with the heads that rescued it
  int jr_h = -1, wb_rescued = 1;
  const int UI_union = UI;
  if constexpr (!DENSE) {
    const int64_t Wn = (int64_t)a.c < N ? (int64_t)a.c : N;
    const int nwt = (int)((Wn + kScreenTile - 1) / kScreenTile);
    if (tid < G) {
      float best = kNegInf;
      bool any = false;
      for (int t = 0; t < nwt; ++t) {
        const int64_t e = (hq0 + tid) * kRescueTiles + t;
        const int inf = a.resc_info[e];
        const float v = a.resc_best[e];
        if (inf == kRescueAny) {
          any = true;
        } else if (inf >= 0 && (jr_h < 0 || v > best)) {
          best = v;
          jr_h = inf;
        }
      }
      if (any) jr_h = -1;
      resc_s[tid] = jr_h;
      if (s == S - 1 && jr_h >= 0) wb_rescued = a.wbits[bg * kMaxRescueWindow + jr_h];
    }
    if (!PROP && s == 0 && tid == 0) a.plan[bg] = make_int2(first, S);
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
    UI += nrx_s;
  }

  // ---- the list's units: the items' blocks, then the tail; this split has units s, s + S, ...
  const uint32_t all_bits = (1u << G) - 1u;
  const int64_t units = (int64_t)UI * spb, total = units + (ntail + 63) / 64;
  const int64_t self_t = (!DENSE && a.self_ungated) ? T - 1 : -1;
  const int32_t* row = a.table + (int64_t)b * a.pg.table_stride;
  auto resolve = [&](int64_t t, int slot) {
    int64_t j = N;
    int sub, n = 64;
    uint32_t bits = all_bits;
    if (t >= units) {
      sub = (int)(t - units);
      n = ntail - 64 * sub < 64 ? ntail - 64 * sub : 64;
    } else {
      const int it = (int)(t >> spb_log);
      sub = (int)(t & (spb - 1));
      if constexpr (DENSE) {
        j = it;
      } else if (it >= UI_union) {
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
    item_ks[slot] = a.k_scale[page * a.pg.scale_stride + gh];
    item_vs[slot] = a.v_scale[page * a.pg.scale_stride + gh];
  };

  Column<D> st;
  st.m = st.l = 0.f;
  st.t = kNegInf;
#pragma unroll
  for (int k = 0; k < D / 16; ++k) st.acc[k] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int ri = lane & 15, g4 = lane >> 4;
  const int64_t head_off = (int64_t)gh * BS * D;
  const uint8_t* kl = a.k + head_off + (16 * (ri >> 2) + (ri & 3)) * D + 16 * g4;
  const uint8_t* vl = a.v + head_off + ri * BS + 16 * g4;
  Unit<D> u;
  auto unit_of = [&](int x, int64_t* koff, int64_t* voff) {
    const int64_t page = __builtin_amdgcn_readfirstlane(item_page[x]);
    const int sub = (__builtin_amdgcn_readfirstlane(item_meta[x]) >> 8) & 255;
    *koff = page * a.pg.page_stride + sub * 64 * D;
    *voff = page * a.pg.page_stride + sub * 64;
  };
  auto load_k = [&](int64_t off) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int h = 0; h < D / 64; ++h) u.k[t][h] = load16(kl + off + 4 * t * D + 64 * h);
  };
  auto load_v = [&](int64_t off) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) u.v[k] = load16_nt(vl + off + 16 * k * BS);
  };
  auto tile = [&](int x, int64_t kn, int64_t vn, auto more_tag) {
    constexpr bool MORE = decltype(more_tag)::value;
    const uint32_t meta = __builtin_amdgcn_readfirstlane(item_meta[x]);
    const float ks = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(item_ks[x])));
    const float vs = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(item_vs[x])));
    const int n = (meta >> 16) & 255;
    const bool on = (meta >> col) & 1u & (col < G);
    f32x4 c[4];
    at.scores(u, c);
    if constexpr (MORE) {
      __builtin_amdgcn_sched_barrier(0);
      load_k(kn);
      __builtin_amdgcn_sched_barrier(0);
    }
    float p[16];
    at.weights(c, n, on, (int)(meta >> 24), ks, st, p);
    if (n < 64) clear_behind<D>(u, n, lane);
    at.values(u, p, on, vs, st);
    if constexpr (MORE) {
      __builtin_amdgcn_sched_barrier(0);
      load_v(vn);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const int nt = strided_share(total, s, S);
  for (int k0 = 0; k0 < nt; k0 += kItems) {
    const int n = nt - k0 < kItems ? nt - k0 : kItems;
    if (tid < n) resolve(s + (int64_t)S * (k0 + tid), tid);
    __syncthreads();
    if (w < n) {
      int64_t ko, vo;
      unit_of(w, &ko, &vo);
      load_k(ko);
      load_v(vo);
      int x = w;
      for (; x + kWaves < n; x += kWaves) {
        unit_of(x + kWaves, &ko, &vo);
        tile(x, ko, vo, std::integral_constant<bool, true>{});
      }
      tile(x, 0, 0, std::integral_constant<bool, false>{});
    }
    __syncthreads();
  }

  if constexpr (!DENSE) {
    if (s == S - 1) {
      // the rescued blocks' mask bits; each head's rescued block and how many are outside the union
      if (tid < G) rxw_s[tid] = jr_h >= 0 ? wb_rescued : 1;
      __syncthreads();
      if (tid == 0) {
        int extra = 0;
        for (int k = 0; k < nrx_s; ++k) {
          bool in_union = false;
          for (int h = 0; h < G; ++h) in_union |= resc_s[h] == rx_s[k][0] && rxw_s[h] != 0;
          extra += !in_union;
        }
        if (!single)
          a.extra_union[bg] = extra;
        else if (a.union_counts != nullptr)
          a.union_counts[bg] = UI_union + extra;
      }
      if (tid < G) {
        if (!single) a.resc_out[hq0 + tid] = jr_h;
        if (jr_h >= 0) a.mask[(hq0 + tid) * g.ncap + jr_h] = 1;
      }
    }
  }

  // ---- merge of the four wavefronts
  st.l += __shfl_xor(st.l, 16, 64);
  st.l += __shfl_xor(st.l, 32, 64);
  if (col < G) {
    if (g4 == 0) {
      mrg_ml[w][col][0] = st.t == kNegInf ? kNegInf : st.m;
      mrg_ml[w][col][1] = st.l;
    }
#pragma unroll
    for (int k = 0; k < D / 16; ++k) *reinterpret_cast<f32x4*>(&mrg_acc[w][col][16 * k + 4 * g4]) = st.acc[k];
  }
  __syncthreads();
  for (int idx = tid; idx < G * D; idx += kThreads) {
    const int h = idx / D, i = idx % D;
    float ms = kNegInf;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) ms = fmaxf(ms, mrg_ml[k][h][0]);
    float L = 0.f, o = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float mk = mrg_ml[k][h][0];
      if (mk == kNegInf) continue;
      const float wk = __builtin_amdgcn_exp2f(mk - ms);
      L = fmaf(mrg_ml[k][h][1], wk, L);
      o = fmaf(mrg_acc[k][h][i], wk, o);
    }
    if (single) {
      store_o(a.out, a.q_dtype, (hq0 + h) * D + i, ms == kNegInf ? 0.f : o / L);
    } else {
      const int64_t pidx = (int64_t)(first + s) * G + h;
      a.part_acc[pidx * D + i] = o;
      if (i == 0) a.part_ml[pidx] = make_float2(ms, L);
    }
  }
  if constexpr (!DENSE) {
    if (single && a.counts != nullptr) {
      for (int h = w; h < G; h += kWaves) {
        int cnt = 0;
        for (int t = lane; t < g.n_tiles; t += 64) cnt += a.head_cnt[(hq0 + h) * g.n_tiles + t];
#pragma unroll
        for (int o2 = 32; o2 > 0; o2 >>= 1) cnt += __shfl_xor(cnt, o2, 64);
        if (lane == 0) a.counts[hq0 + h] = (int32_t)(((int64_t)cnt + (resc_s[h] >= 0 ? 1 : 0)) * BS + ntail);
      }
    }
  }
}

template <bool DENSE>
void launch_split(const PageSplitArgs& a, const SplitPlan& pl, hipStream_t stream) {
  const Geom& g = a.pg.g;
  const dim3 grid = pl.S > 0 ? dim3(pl.S, g.Hkv, g.B) : dim3(pl.W);
#define ETA_PSPL(D_, P_, F_)                                                                             \
  if (g.D == D_ && (pl.S == 0) == P_ && (a.q_dtype == ETA_DT_F32) == F_)                                 \
    hipLaunchKernelGGL((page_split_kernel<D_, DENSE, P_, F_>), grid, dim3(kThreads), 0, stream, a);
  ETA_PSPL(64, false, false) ETA_PSPL(64, false, true) ETA_PSPL(64, true, false) ETA_PSPL(64, true, true)
  ETA_PSPL(128, false, false) ETA_PSPL(128, false, true) ETA_PSPL(128, true, false) ETA_PSPL(128, true, true)
#undef ETA_PSPL
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

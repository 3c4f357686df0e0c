// Norms of the queries and keys of each head and their rotation by position, in
// one pass from the projections' layout into q [B][Hq][T][d] and the K / V
// caches, and the gradients of that pass (gfx950, wave64).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "eta_device.h"
#include "eta_lanes.h"
#include "eta_train.h"

namespace eta {
namespace {

// A row is one head of one token: n = x r w with r = 1 / sqrt(mean x^2 + eps) (n = x
// without a weight), then the pairs (a, b) of its first rotary_dim values become
// (a cos - b sin, a sin + b cos) at the angle position x frequency.  Values and sums are
// fp32; the result is rounded once.  The angle is taken in turns in 64 bits (at position
// 2^19 an fp32 angle is off by up to 2^-6 radians), its fraction in fp32.
//
// What bounds it: memory, each row read once and written once (16K tokens, 32/8 heads, d = 128, bf16:
// 82 us, 4.9 TB/s, where a device copy reaches 5.2; the gradients 116 us, 4.9 TB/s).  A lane holds 16 bytes
// of a row, so a row of 256 bytes is 16 lanes and its sum of squares four DPP steps; the
// lanes of a row keep one token and walk over heads, so that sines, cosines and weights
// stay in registers (16 heads a workgroup: 90 us before the hints below, 8: 95, 4: 116).

// 16 bytes of a row, read once: with the non-temporal hint (16K tokens, 32/8 heads, d = 128, bf16,
// backward into the same results each time: 125 -> 108 us; 4 x 2000, 32/4, d = 64, fp32: 46.5 -> 42.6 us).
// With STREAM the results are written with it too (plan_rope has the rule and what it measured).
typedef uint32_t u32x4n __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 get16(const char* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4n*>(p)));
}
template <bool STREAM>
__device__ __forceinline__ void put16(char* p, const uint4& x) {
  if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(u32x4n, x), reinterpret_cast<u32x4n*>(p));
  else *reinterpret_cast<uint4*>(p) = x;
}

template <typename T>
struct Piece;                     // 16 bytes of a row
template <>
struct Piece<uint16_t> {
  static constexpr int E = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                      pack_bf16x2(x[6], x[7]));
  }
};
template <>
struct Piece<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float (&x)[4]) {
    x[0] = __uint_as_float(r.x);
    x[1] = __uint_as_float(r.y);
    x[2] = __uint_as_float(r.z);
    x[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                      __float_as_uint(x[3]));
  }
};

struct RopeArgs {
  const char *q, *k, *v;          // projections [B][Tn][H][d] (byte strides below)
  char *q_out, *k_out, *v_out;    // q [B][Hq][Tn][d], caches
  const char *gq, *gk, *gv;       // gradients of those (backward)
  char *dq, *dk, *dv;             // gradients of the projections (backward)
  const float *qw, *kw, *freqs;
  const int32_t *start, *lens;
  float* part;
  int64_t qb, qt, kb, kt, vb, vt;         // strides of the projections, bytes
  int64_t dqb, dqt, dkb, dkt, dvb, dvt;   // and of their gradients
  int64_t cb, ch, ct;                     // cache strides, bytes
  int64_t cap;
  int Hq, Hkv, Tn, N;                     // N = B Tn tokens
  int heads, nq, nk, tiles;
  int rot, interleaved;
  float eps;
};

// A token's place: sequence, row among its new tokens, cache row, whether it is there.
struct Token {
  int b, i;
  int64_t row;
  bool there;                     // the row is new (i < new_lens[b])
  bool kept;                      // and the cache has a row for it
};
__device__ __forceinline__ Token token_of(const RopeArgs& a, int n) {
  Token t;
  const int nn = n < a.N ? n : a.N - 1;
  t.b = nn / a.Tn;
  t.i = nn - t.b * a.Tn;
  const int len = a.lens ? a.lens[t.b] : a.Tn;
  int64_t s = a.start ? a.start[t.b] : 0;
  if (s < 0) s = 0;
  t.row = s + t.i;
  t.there = n < a.N && t.i < len;
  t.kept = t.there && t.row < a.cap;
  return t;
}

// The turn of a lane's E values: y = x c + other s, other the pair's other value (s carries
// its sign); lanes past the rotated part keep x.
template <int E, int LPR>
struct Turn {
  float c[E], s[E];
  int partner;                    // lane that holds the pairs' other values (halves)
  bool rotated;
  __device__ __forceinline__ void set(const RopeArgs& a, int chunk, int lane, int64_t pos) {
    const int rc = a.rot / E, hc = rc / 2;
    rotated = chunk < rc;
    const bool first = chunk < hc;
    partner = lane;
    if (!a.interleaved && rotated) partner = first ? lane + hc : lane - hc;
    const double p = (double)pos;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      c[e] = 1.f;
      s[e] = 0.f;
    }
    if (!rotated) return;
    auto angle = [&](int j, float& cc, float& ss) {
      const double turns = p * ((double)a.freqs[j] * 0.15915494309189533577);
      sincospif((float)(2.0 * (turns - rint(turns))), &ss, &cc);
    };
    if (a.interleaved) {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        float cc, ss;
        angle((chunk * E + e) / 2, cc, ss);
        c[e] = c[e + 1] = cc;
        s[e] = -ss;
        s[e + 1] = ss;
      }
    } else {
      const int j0 = (first ? chunk : chunk - hc) * E;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        angle(j0 + e, c[e], s[e]);
        if (first) s[e] = -s[e];
      }
    }
  }
  __device__ __forceinline__ uint4 other_raw(const uint4& r) const {
    return make_uint4((uint32_t)__shfl((int)r.x, partner), (uint32_t)__shfl((int)r.y, partner),
                      (uint32_t)__shfl((int)r.z, partner), (uint32_t)__shfl((int)r.w, partner));
  }
};

// Which heads a workgroup takes: kind 0 q, 1 k, 2 v.
struct Share {
  int kind, h0, h1;
};
__device__ __forceinline__ Share share_of(const RopeArgs& a, int y) {
  Share s;
  s.kind = y < a.nq ? 0 : y < a.nq + a.nk ? 1 : 2;
  s.h0 = (y - (s.kind == 0 ? 0 : s.kind == 1 ? a.nq : a.nq + a.nk)) * a.heads;
  s.h1 = min(s.h0 + a.heads, s.kind == 0 ? a.Hq : a.Hkv);
  return s;
}

constexpr int kRopeAhead = 4;     // rows of a lane in flight

template <typename T, int D, bool STREAM>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int E = Piece<T>::E, LPR = D / E, TPW = 256 / LPR;
  constexpr int64_t ROW = D * sizeof(T);
  const int lane = threadIdx.x & 63, chunk = threadIdx.x % LPR;
  const Token t = token_of(a, blockIdx.x * TPW + threadIdx.x / LPR);
  const Share sh = share_of(a, blockIdx.y);
  const bool live = sh.kind == 0 ? t.there : t.kept;
  const char* in;
  char* out;
  int64_t step;
  if (sh.kind == 0) {
    in = a.q + t.b * a.qb + t.i * a.qt;
    out = a.q_out + ((int64_t)t.b * a.Hq * a.Tn + t.i) * ROW;
    step = a.Tn * ROW;
  } else {
    in = sh.kind == 1 ? a.k + t.b * a.kb + t.i * a.kt : a.v + t.b * a.vb + t.i * a.vt;
    out = (sh.kind == 1 ? a.k_out : a.v_out) + t.b * a.cb + (t.kept ? t.row : 0) * a.ct;
    step = a.ch;
  }
  in += chunk * 16;
  out += chunk * 16;
  if (sh.kind == 2) {
    for (int h = sh.h0; h < sh.h1; h += kRopeAhead) {
      uint4 r[kRopeAhead];
#pragma unroll
      for (int u = 0; u < kRopeAhead; ++u)
        r[u] = get16(in + min(h + u, sh.h1 - 1) * ROW);
#pragma unroll
      for (int u = 0; u < kRopeAhead; ++u)
        if (live && h + u < sh.h1) put16<STREAM>(out + (h + u) * step, r[u]);
    }
    return;
  }
  const float* wt = sh.kind == 0 ? a.qw : a.kw;
  // the first rows are on their way while the sines are formed
  uint4 r[kRopeAhead];
  auto fetch = [&](int h) {
#pragma unroll
    for (int u = 0; u < kRopeAhead; ++u) r[u] = get16(in + min(h + u, sh.h1 - 1) * ROW);
  };
  fetch(sh.h0);
  Turn<E, LPR> turn;
  turn.set(a, chunk, lane, t.row);
  float w[E], wo[E];              // weights of the lane's values and of their pairs' others
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int at = a.interleaved ? chunk * E + (e ^ 1) : (chunk + turn.partner - lane) * E + e;
    w[e] = wt ? wt[chunk * E + e] : 1.f;
    wo[e] = (wt ? wt[at] : 1.f) * turn.s[e];
    w[e] *= turn.c[e];
  }
  for (int h = sh.h0; h < sh.h1; h += kRopeAhead) {
    if (h > sh.h0) fetch(h);
#pragma unroll
    for (int u = 0; u < kRopeAhead; ++u) {
      float x[E], o[E];
      Piece<T>::unpack(r[u], x);
      float rs = 1.f;
      if (wt) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) ss = fmaf(x[e], x[e], ss);
        rs = rsqrtf(lanes_sum<LPR>(ss) * (1.0f / D) + a.eps);
      }
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = x[e ^ 1];
      } else {
        Piece<T>::unpack(turn.other_raw(r[u]), o);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float n = x[e] * rs;
        x[e] = turn.rotated ? fmaf(o[e] * rs, wo[e], n * w[e]) : n * w[e];
      }
      if (live && h + u < sh.h1) put16<STREAM>(out + (h + u) * step, Piece<T>::pack(x));
    }
  }
}

// Gradients of rope_kernel.  With g the rotation's transpose of dy (the turn by the
// opposite angle) and n = x r: dx = r (w g - n mean(n w g)), dw = sum over the rows of
// g n.  x and dy are read once, dx written once; r is formed again from x.  The sums of
// dw stay in a lane's registers over all its rows; a workgroup adds its token groups in
// order and leaves one row of partials, which rope_weight_kernel adds in order, so the
// result does not depend on the order of the workgroups.
template <typename T, int D, bool STREAM>
__global__ __launch_bounds__(256) void rope_grad_kernel(RopeArgs a) {
  constexpr int E = Piece<T>::E, LPR = D / E, TPW = 256 / LPR;
  constexpr int64_t ROW = D * sizeof(T);
  __shared__ float sums[TPW][D];
  const int lane = threadIdx.x & 63, chunk = threadIdx.x % LPR;
  const Share sh = share_of(a, blockIdx.y);
  const float* wt = sh.kind == 0 ? a.qw : sh.kind == 1 ? a.kw : nullptr;
  float dw[E], w[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    dw[e] = 0.f;
    w[e] = wt ? wt[chunk * E + e] : 1.f;
  }
  for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const int n0 = tile * TPW + threadIdx.x / LPR;
    const Token t = token_of(a, n0);
    const bool live = sh.kind == 0 ? t.there : t.kept;
    const char *x_in, *g_in;
    char* out;
    int64_t step;
    if (sh.kind == 0) {
      x_in = a.q + t.b * a.qb + t.i * a.qt;
      g_in = a.gq + ((int64_t)t.b * a.Hq * a.Tn + t.i) * ROW;
      out = a.dq + t.b * a.dqb + t.i * a.dqt;
      step = a.Tn * ROW;
    } else {
      x_in = a.k + t.b * a.kb + t.i * a.kt;
      g_in = (sh.kind == 1 ? a.gk : a.gv) + t.b * a.cb + (t.kept ? t.row : 0) * a.ct;
      out = sh.kind == 1 ? a.dk + t.b * a.dkb + t.i * a.dkt : a.dv + t.b * a.dvb + t.i * a.dvt;
      step = a.ch;
    }
    x_in += chunk * 16;
    g_in += chunk * 16;
    out += chunk * 16;
    const bool in_range = n0 < a.N;
    Turn<E, LPR> turn;
    if (sh.kind != 2) turn.set(a, chunk, lane, t.row);
    for (int h = sh.h0; h < sh.h1; h += kRopeAhead) {
      uint4 rg[kRopeAhead], rx[kRopeAhead];
#pragma unroll
      for (int u = 0; u < kRopeAhead; ++u) {
        const int hh = min(h + u, sh.h1 - 1);
        rg[u] = get16(g_in + hh * step);
        if (wt) rx[u] = get16(x_in + hh * ROW);
      }
#pragma unroll
      for (int u = 0; u < kRopeAhead; ++u) {
        uint4 res = rg[u];
        const bool row = live && h + u < sh.h1;
        if (sh.kind != 2) {
          float g[E], o[E];
          Piece<T>::unpack(rg[u], g);
          if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = g[e ^ 1];
          } else {
            Piece<T>::unpack(turn.other_raw(rg[u]), o);
          }
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (turn.rotated) g[e] = fmaf(-o[e], turn.s[e], g[e] * turn.c[e]);
          if (wt) {
            float x[E], ss = 0.f, sg = 0.f;
            Piece<T>::unpack(rx[u], x);
#pragma unroll
            for (int e = 0; e < E; ++e) ss = fmaf(x[e], x[e], ss);
            const float rs = rsqrtf(lanes_sum<LPR>(ss) * (1.0f / D) + a.eps);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              x[e] *= rs;
              const float p = g[e] * x[e];
              if (row) dw[e] += p;
              sg = fmaf(p, w[e], sg);
            }
            sg = lanes_sum<LPR>(sg) * (1.0f / D);
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = rs * fmaf(-x[e], sg, g[e] * w[e]);
          }
          res = Piece<T>::pack(g);
        }
        if (!live) res = make_uint4(0, 0, 0, 0);
        if (in_range && h + u < sh.h1) put16<STREAM>(out + (h + u) * ROW, res);
      }
    }
  }
  if (wt) {
#pragma unroll
    for (int e = 0; e < E; ++e) sums[threadIdx.x / LPR][chunk * E + e] = dw[e];
    __syncthreads();
    if (threadIdx.x < D) {
      float s = 0.f;
#pragma unroll
      for (int r = 0; r < TPW; ++r) s += sums[r][threadIdx.x];
      a.part[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * D + threadIdx.x] = s;
    }
  }
}

// Sums of the rows of partials: one workgroup per 16 columns of q's or k's weight.  Thread (r, c) adds
// rows r, r + 64, ... of its column, sixteen loads at once (they, not the adds, are the time), and the
// 64 sums are added in order.
__global__ __launch_bounds__(1024) void rope_weight_kernel(const float* part, int rows_q, int rows_k,
                                                           int D, float* dqw, float* dkw) {
  static_assert(kRopePartials <= 64 * 16, "one batch of loads");
  __shared__ float s[64][17];
  const int r = threadIdx.x / 16, c = threadIdx.x % 16;
  const bool key = blockIdx.y == 1;
  float* out = key ? dkw : dqw;
  if (out == nullptr) return;
  const float* p = part + (key ? (int64_t)rows_q * D : 0) + blockIdx.x * 16 + c;
  const int rows = key ? rows_k : rows_q;
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int row = r + 64 * i;
    x[i] = row < rows ? p[(int64_t)row * D] : 0.f;
  }
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) t += x[i];
  s[r][c] = t;
  __syncthreads();
  if (r == 0) {
    t = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) t += s[i][c];
    out[blockIdx.x * 16 + c] = t;
  }
}

RopeArgs rope_args(const eta_rope_desc_t& rd, const RopePlan& p, const float* qw, const float* kw,
                   const float* freqs, const int32_t* start, const int32_t* lens) {
  const int64_t e = rd.dtype == ETA_DT_F32 ? 4 : 2;
  RopeArgs a{};
  a.qw = qw;
  a.kw = kw;
  a.freqs = freqs;
  a.start = start;
  a.lens = lens;
  a.qb = rd.q_stride_b * e;
  a.qt = rd.q_stride_t * e;
  a.kb = rd.k_stride_b * e;
  a.kt = rd.k_stride_t * e;
  a.vb = rd.v_stride_b * e;
  a.vt = rd.v_stride_t * e;
  a.dqb = rd.dq_stride_b * e;
  a.dqt = rd.dq_stride_t * e;
  a.dkb = rd.dk_stride_b * e;
  a.dkt = rd.dk_stride_t * e;
  a.dvb = rd.dv_stride_b * e;
  a.dvt = rd.dv_stride_t * e;
  a.cb = rd.cache_stride_b * e;
  a.ch = rd.cache_stride_h * e;
  a.ct = rd.cache_stride_t * e;
  a.cap = rd.capacity_tokens;
  a.Hq = rd.num_q_heads;
  a.Hkv = rd.num_kv_heads;
  a.Tn = rd.new_tokens;
  a.N = rd.batch * rd.new_tokens;
  a.heads = p.heads;
  a.nq = p.nq;
  a.nk = p.nk;
  a.tiles = p.tiles;
  a.rot = rd.rotary_dim;
  a.interleaved = rd.interleaved;
  a.eps = rd.eps;
  return a;
}

// Launches a kernel for the descriptor's type and head dimension.
#define ETA_ROPE_LAUNCH(kernel, STREAM)                                                                         \
  do {                                                                                                          \
    if (rd.dtype == ETA_DT_F32) {                                                                               \
      if (rd.head_dim == 64) hipLaunchKernelGGL((kernel<float, 64, STREAM>), grid, dim3(256), 0, stream, a);    \
      else hipLaunchKernelGGL((kernel<float, 128, STREAM>), grid, dim3(256), 0, stream, a);                     \
    } else {                                                                                                    \
      if (rd.head_dim == 64) hipLaunchKernelGGL((kernel<uint16_t, 64, STREAM>), grid, dim3(256), 0, stream, a); \
      else hipLaunchKernelGGL((kernel<uint16_t, 128, STREAM>), grid, dim3(256), 0, stream, a);                  \
    }                                                                                                           \
  } while (0)

}  // namespace

hipError_t launch_rope(const eta_rope_desc_t& rd, const RopePlan& p, const void* q, const void* k,
                       const void* v, const float* qw, const float* kw, const float* freqs,
                       const int32_t* start, const int32_t* new_lens, void* q_out, void* k_cache,
                       void* v_cache, hipStream_t stream, LaunchHook hook) {
  RopeArgs a = rope_args(rd, p, qw, kw, freqs, start, new_lens);
  a.q = (const char*)q;
  a.k = (const char*)k;
  a.v = (const char*)v;
  a.q_out = (char*)q_out;
  a.k_out = (char*)k_cache;
  a.v_out = (char*)v_cache;
  const dim3 grid(p.tiles, p.nq + p.nk + p.nv);
  return with_hook(hook, ETA_KERNEL_QK_ROPE, stream, [&] {
    if (p.stream) ETA_ROPE_LAUNCH(rope_kernel, true);
    else ETA_ROPE_LAUNCH(rope_kernel, false);
  });
}

hipError_t launch_rope_grad(const eta_rope_desc_t& rd, const RopePlan& p, const void* dq_out,
                            const void* dk_cache, const void* dv_cache, const void* q, const void* k,
                            const float* qw, const float* kw, const float* freqs,
                            const int32_t* start, const int32_t* new_lens, void* dq, void* dk,
                            void* dv, float* dqw, float* dkw, float* part, hipStream_t stream,
                            LaunchHook hook) {
  RopeArgs a = rope_args(rd, p, qw, kw, freqs, start, new_lens);
  a.q = (const char*)q;
  a.k = (const char*)k;
  a.gq = (const char*)dq_out;
  a.gk = (const char*)dk_cache;
  a.gv = (const char*)dv_cache;
  a.dq = (char*)dq;
  a.dk = (char*)dk;
  a.dv = (char*)dv;
  a.part = part;
  const dim3 grid(p.steps, p.nq + p.nk + p.nv);
  hipError_t e = with_hook(hook, ETA_KERNEL_QK_ROPE_GRAD, stream, [&] {
    if (p.stream) ETA_ROPE_LAUNCH(rope_grad_kernel, true);
    else ETA_ROPE_LAUNCH(rope_grad_kernel, false);
  });
  if (e != hipSuccess || (!qw && !kw)) return e;
  return with_hook(hook, ETA_KERNEL_QK_WEIGHT_GRAD, stream, [&] {
    hipLaunchKernelGGL(rope_weight_kernel, dim3(rd.head_dim / 16, 2), dim3(1024), 0, stream, part,
                       p.nq * p.steps, p.nk * p.steps, rd.head_dim, qw ? dqw : nullptr, kw ? dkw : nullptr);
  });
}

}  // namespace eta

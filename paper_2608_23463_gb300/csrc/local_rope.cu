// Queries and keys of the local stream's attention: RMSNorm of every head and
// the position rotation in one pass over the rows, its backward, and the same
// pass writing keys and values into a paged cache.
//
// A head x of dh values (r = 1 / sqrt(mean x^2 + eps), weights w):
//   y = w x r;   pair (2 j, 2 j + 1) of y turned by angle_j = pos_a f_j,
//   f_j = theta^(-i / n_a) for pair i of the n_a that axis a turns.
// Backward, from the gradient dz of the turned head (dy = dz turned back):
//   dw = sum over rows and heads of dy x r,
//   dx = r (w dy - x r mean(w dy x r)).
//
// HBM traffic bounds all of them, a row read once and written once, and the
// instructions come next.  A head's values lie on dh / 8 (bf16) or dh / 4
// (fp32) lanes, 16 bytes each, so that a warp holds several heads and a head's
// sum takes three to five shuffles; a warp takes a token, makes its sines (a
// pair or two on each lane, handed round by shuffles), folds the weights into
// them and walks the token's heads.  Arithmetic is in packed pairs: the first
// halves of two turned pairs side by side, and the second halves.  With few
// tokens a token's heads are spread over several warps (`parts`): latency
// counts there, and the sines made twice do not.
// Measured: four images of 512 x 512 tokens, 8 + 8 heads of 64, 694 us (6.2
// TB/s, 91 % of a plain copy); backward, 65536 tokens of 16 + 4 heads, 97 us
// (5.2 TB/s); eight prompts of 11738 tokens in all, 16 + 2 heads of 128, into
// the cache 25.5 us (4.7 TB/s), quantised 27.6.  fp32: the images 1283 us (6.7 TB/s), the
// backward 158 us (6.4 TB/s).  Scalar arithmetic with the weights applied
// apart took 843 us for the images, three quarters of the issue slots busy.
//
// Angles: the frequency is held as a 64-bit fraction of a turn, and
// pos * f modulo 2^64 is exact integer arithmetic; a position of a million
// loses nothing, where a product in fp32 would be off by 0.06 radians.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "local.h"
#include "paged_q8.cuh"

namespace pf {

static Launched launched;
int take_dev_error_local_rope() { return launched.take(take_dev_error_tu); }
int set_wait_limit_local_rope(unsigned long long ns) { return set_wait_limit_tu(ns); }

namespace {

constexpr int RW_THREADS = 256;
constexpr int RW_WARPS = RW_THREADS / 32;
// Resident CTAs an SM and passes in flight per lane.  Forward, four images of 512 x 512 tokens and 8 + 8
// heads of 64: 694 us so, 723 with 4 CTAs, 802 with one pass, 877 with three and 4 CTAs.  Backward,
// 65536 tokens of 16 + 4 heads: 97 us so, 102 with 2 CTAs and four passes, 110 with one.  Rows asked into
// L2 a token ahead: 799 and 103.
constexpr int RW_FWD_CTAS = 5, RW_FWD_U = 2;
constexpr int RW_BWD_CTAS = 3, RW_BWD_U = 2;
constexpr int RW_MAX_PAIRS = 64;

struct RopeFreq {
  unsigned long long f[RW_MAX_PAIRS];  // turns per position, in 2^-64
  unsigned char axis[RW_MAX_PAIRS];
  int n_axes;
};

struct RopeArgs {
  const void *q, *k;   // [rows, ld], head h at column h * dh
  void *qo, *ko;
  long ldq, ldk, ldqo, ldko;
  const float *w_q, *w_k;  // [dh] or null: no norm
  const int* pos;          // [rows, n_axes] or null: row % seq_len (cache row when appending)
  int rows, seq_len, H, KV;
  int parts;  // warps that share a token
  float eps;
  // backward: gradients of qo and ko, and the CTAs' sums of the weights' gradients
  const void *dqo, *dko;
  long lddqo, lddko;
  float* part;  // [grid][2][dh]
  // append
  const void* v;
  long ldv;
  bf16 *K, *V;                       // [n_pages, KV, page, dh]
  signed char *Ke, *Ve;              // quantised: their exponents [n_pages, KV, page] (K and V are bytes then)
  const int *table, *len, *start;
  int B, page, max_pages;
  long n_pages;
};

// 16 bytes of a head as packed pairs: e[i] holds the first halves of the turned
// pairs 2 i and 2 i + 1 (of the lane's), o[i] their second halves.
template <class T>
struct Vec;
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(uint4 u, float2* e, float2* o) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      e[i] = make_float2(__uint_as_float(w[2 * i] << 16), __uint_as_float(w[2 * i + 1] << 16));
      o[i] = make_float2(__uint_as_float(w[2 * i] & 0xffff0000u),
                         __uint_as_float(w[2 * i + 1] & 0xffff0000u));
    }
  }
  static __device__ __forceinline__ uint4 put(const float2* e, const float2* o) {
    return make_uint4(pack_bf16(e[0].x, o[0].x), pack_bf16(e[0].y, o[0].y),
                      pack_bf16(e[1].x, o[1].x), pack_bf16(e[1].y, o[1].y));
  }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(uint4 u, float2* e, float2* o) {
    e[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.z));
    o[0] = make_float2(__uint_as_float(u.y), __uint_as_float(u.w));
  }
  static __device__ __forceinline__ uint4 put(const float2* e, const float2* o) {
    return make_uint4(__float_as_uint(e[0].x), __float_as_uint(o[0].x), __float_as_uint(e[0].y),
                      __float_as_uint(o[0].y));
  }
};

// How a warp holds heads of DH values of type T.
template <class T, int DH>
struct Lay {
  static constexpr int N = Vec<T>::N;       // values per lane
  static constexpr int G = N / 4;           // packed groups of two pairs
  static constexpr int LANES = DH / N;      // lanes per head
  static constexpr int HEADS = 32 / LANES;  // heads per pass of the warp
  static constexpr int PPL = DH / 64;       // pairs whose sines a lane makes
};

struct RopeSmem {
  unsigned long long f[RW_MAX_PAIRS];
  float2 w[2][RW_MAX_PAIRS];  // w_q, w_k: group i's (first halves, second halves) at 2 i, 2 i + 1
  unsigned char axis[RW_MAX_PAIRS];
};

// (The table comes from parameter space, which serves a warp one address at a
// time: each thread fetches one entry.)
template <int DH>
__device__ __forceinline__ void stage_freq(RopeSmem& s, const RopeFreq& fr) {
  const int i = threadIdx.x;
  if (i < DH / 2) {
    s.f[i] = fr.f[i];
    s.axis[i] = fr.axis[i];
  }
}
template <int DH>
__device__ __forceinline__ void stage_weights(RopeSmem& s, const RopeArgs& a) {
  const int i = threadIdx.x;
  if (i < DH) {
    const float* w = i < DH / 2 ? a.w_q : a.w_k;
    const int c = i % (DH / 2), j = c / 2 * 4 + (c & 1);  // values j and j + 2 of a head
    s.w[i / (DH / 2)][c] = w ? make_float2(w[j], w[j + 2]) : make_float2(1.f, 1.f);
  }
  __syncthreads();
}

// cos and sin of the lane's pairs at the token's position(s), packed as the
// values.  bf16 rows take the hardware sine (absolute error below 2^-20 for
// |angle| <= pi, a 2000th of the rounding of the result); fp32 rows, and those that
// are quantised (whole numbers come out as they would of exact values but for one in
// some ten thousand), the library's.
template <class T, int DH, bool EXACT = sizeof(T) == 4>
__device__ __forceinline__ void turn_of(const RopeSmem& s, const int* pos3, int lane, float2* cs,
                                        float2* sn) {
  using Ly = Lay<T, DH>;
  float oc[Ly::PPL], os[Ly::PPL];
#pragma unroll
  for (int i = 0; i < Ly::PPL; ++i) {
    const int p = lane * Ly::PPL + i, ax = s.axis[p];
    const int ps = ax == 0 ? pos3[0] : ax == 1 ? pos3[1] : pos3[2];
    const unsigned long long ph = (unsigned long long)(long long)ps * s.f[p];
    const float h = (float)(int)(ph >> 32) * 4.656612873077393e-10f;  // half turns, [-1, 1]
    if (!EXACT)
      __sincosf(h * 3.14159265358979f, &os[i], &oc[i]);
    else
      sincospif(h, &os[i], &oc[i]);
  }
  const int sub = lane % Ly::LANES;
#pragma unroll
  for (int i = 0; i < Ly::N / 2; ++i) {
    const int src = (sub * (Ly::N / 2) + i) / Ly::PPL;
    const float c = __shfl_sync(0xffffffffu, oc[i % Ly::PPL], src);
    const float t = __shfl_sync(0xffffffffu, os[i % Ly::PPL], src);
    (i & 1 ? cs[i / 2].y : cs[i / 2].x) = c;
    (i & 1 ? sn[i / 2].y : sn[i / 2].x) = t;
  }
}

template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// A head's 8 values of a lane (e, o as above) quantised: row and exponent.  All lanes of the head
// take part; `in`: it is one to be written.
template <int LANES>
__device__ __forceinline__ void put_q8(const float2* e, const float2* o, signed char* row, signed char* ex, int sub,
                                       bool in) {
  const float y[8] = {e[0].x, o[0].x, e[0].y, o[0].y, e[1].x, o[1].x, e[1].y, o[1].y};
  int m = 0;  // of the bits: NaN counts as larger than all else
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_int(y[i]) & 0x7fffffff);
#pragma unroll
  for (int s = LANES / 2; s > 0; s >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, s));
  const int x = pq_exp(__int_as_float(m));
  const float f = pq_inverse(x);
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t n[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) n[k] = (uint32_t)__float2int_rn(y[4 * i + k] * f);
    w[i] = __byte_perm(__byte_perm(n[0], n[1], 0x0040), __byte_perm(n[2], n[3], 0x0040), 0x5410);
  }
  if (!in) return;
  *reinterpret_cast<uint2*>(row) = make_uint2(w[0], w[1]);
  if (sub == 0) *ex = (signed char)x;
}

// n passes, U at a time without a branch between them, so that their shuffles overlap, and
// what is left of them singly.
template <int U, class F>
__device__ __forceinline__ void in_passes(int n, F pass) {
  for (; n >= U; n -= U) pass(std::integral_constant<int, U>{});
  if (U > 1)
    for (; n > 0; --n) pass(std::integral_constant<int, 1>{});
}

// Passes [p0, p1) of one token's heads (head p * HEADS + the lane's slot, below
// nh), normed and turned: src + head * DH -> dst + head * dst_stride; Q8: quantised, dst of bytes,
// the exponents to ex + head * dst_stride / DH.
template <class T, int DH, bool Q8 = false, class D = T>
__device__ __forceinline__ void rope_heads(const T* src, D* dst, long dst_stride, int p0, int p1,
                                           int nh, const float2* w, bool norm, float eps,
                                           const float2* cs, const float2* sn, int lane, signed char* ex = nullptr) {
  using Ly = Lay<T, DH>;
  constexpr int G = Ly::G;
  const int sub = lane % Ly::LANES, slot = lane / Ly::LANES;
  // w folded into the turn: z_e = x_e (w_e c) - x_o (w_o s), z_o = x_e (w_e s) + x_o (w_o c)
  float2 ec[G], os[G], es[G], oc[G];
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const float2 we = w[(sub * G + i) * 2], wo = w[(sub * G + i) * 2 + 1];
    ec[i] = __fmul2_rn(we, cs[i]);
    es[i] = __fmul2_rn(we, sn[i]);
    oc[i] = __fmul2_rn(wo, cs[i]);
    os[i] = __fmul2_rn(wo, make_float2(-sn[i].x, -sn[i].y));
  }
  int h = p0 * Ly::HEADS + slot;
  const T* sp = src + (long)h * DH + sub * Ly::N;
  D* dp = dst + h * dst_stride + sub * Ly::N;
  const long dstep = Ly::HEADS * dst_stride;
  auto pass = [&](auto count) {
    constexpr int U = decltype(count)::value;
    uint4 u[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      u[i] = make_uint4(0, 0, 0, 0);
      if (h + i * Ly::HEADS < nh)
        u[i] = *reinterpret_cast<const uint4*>(sp + i * Ly::HEADS * DH);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float2 e[G], o[G];
      Vec<T>::get(u[i], e, o);
      float r = 1.f;
      if (norm) {
        float2 ss = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < G; ++k) ss = __ffma2_rn(e[k], e[k], __ffma2_rn(o[k], o[k], ss));
        r = rsqrtf(fmaf(head_sum<Ly::LANES>(ss.x + ss.y), 1.f / DH, eps));
      }
      float2 ze[G], zo[G];
#pragma unroll
      for (int k = 0; k < G; ++k) {
        ze[k] = __ffma2_rn(e[k], ec[k], __fmul2_rn(o[k], os[k]));
        zo[k] = __ffma2_rn(e[k], es[k], __fmul2_rn(o[k], oc[k]));
        if (norm) {
          ze[k] = __fmul2_rn(ze[k], both(r));
          zo[k] = __fmul2_rn(zo[k], both(r));
        }
      }
      if constexpr (Q8)
        put_q8<Ly::LANES>(ze, zo, dp + i * dstep, ex + (h + i * Ly::HEADS) * (dst_stride / DH), sub, h + i * Ly::HEADS < nh);
      else if (h + i * Ly::HEADS < nh)
        *reinterpret_cast<uint4*>(dp + i * dstep) = Vec<T>::put(ze, zo);
    }
    h += U * Ly::HEADS;
    sp += U * Ly::HEADS * DH;
    dp += U * dstep;
  };
  in_passes<RW_FWD_U>(p1 - p0, pass);
}

// Forward (APPEND: keys and values go to their cache pages; Q8: quantised).  A unit is part
// `pt` of a token's passes: q heads, then k heads, then (APPEND) v heads.
template <class T, int DH, bool APPEND, bool Q8 = false>
__global__ void __launch_bounds__(RW_THREADS, RW_FWD_CTAS)
    rope_fwd_kernel(RopeArgs a, const __grid_constant__ RopeFreq fr) {
  using Ly = Lay<T, DH>;
  __shared__ __align__(16) RopeSmem s;
  stage_freq<DH>(s, fr);
  pdl_enter();
  stage_weights<DH>(s, a);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int nq = (a.H + Ly::HEADS - 1) / Ly::HEADS, nk = (a.KV + Ly::HEADS - 1) / Ly::HEADS;
  const int passes = nq + nk + (APPEND ? nk : 0);
  const long units = (long)a.rows * a.parts;
  for (long un = (long)blockIdx.x * RW_WARPS + warp; un < units; un += (long)gridDim.x * RW_WARPS) {
    const int row = a.parts == 1 ? (int)un : (int)(un / a.parts), pt = (int)(un - (long)row * a.parts);
    const int p0 = pt * passes / a.parts, p1 = (pt + 1) * passes / a.parts;
    int pos3[3] = {0, 0, 0};
    bf16 *kd = nullptr, *vd = nullptr;
    long at = 0;  // the token's row of the pool, of its first head
    if (APPEND) {
      // the token's sequence: how many of them end at or before it
      int b = row;
      if (a.start) {
        b = 0;
        for (int i = 0; i < a.B; i += 32) {
          const bool past = i + lane < a.B && a.start[i + lane + 1] <= row;
          b += __popc(__ballot_sync(0xffffffffu, past));
        }
      }
      int crow = -1;
      if (b < a.B) crow = a.len[b] - (a.start ? a.start[b + 1] - row : 1);
      pos3[0] = crow;
      long pg = -1;
      if (crow >= 0 && crow / a.page < a.max_pages)
        pg = a.table[(long)b * a.max_pages + crow / a.page];
      if (pg < 0 || pg >= a.n_pages) {
        if (lane == 0) set_dev_error(DEVERR_CAPACITY);
      } else {
        at = pg * a.KV * a.page + crow % a.page;
        kd = a.K + at * DH;
        vd = a.V + at * DH;
      }
    } else if (!a.pos) {
      pos3[0] = row % a.seq_len;
    }
    if (a.pos) {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < fr.n_axes) pos3[i] = a.pos[(long)row * fr.n_axes + i];
    }
    float2 cs[Ly::G], sn[Ly::G];
    turn_of<T, DH, Q8 || sizeof(T) == 4>(s, pos3, lane, cs, sn);
    if (p0 < nq)
      rope_heads<T, DH>(static_cast<const T*>(a.q) + row * a.ldq, static_cast<T*>(a.qo) + row * a.ldqo,
                        DH, p0, min(p1, nq), a.H, s.w[0], a.w_q != nullptr, a.eps, cs, sn, lane);
    const int k0 = max(p0, nq) - nq, k1 = min(p1, nq + nk) - nq;
    const T* ks = static_cast<const T*>(a.k) + row * a.ldk;
    if (!APPEND) {
      if (k0 < k1)
        rope_heads<T, DH>(ks, static_cast<T*>(a.ko) + row * a.ldko, DH, k0, k1, a.KV, s.w[1],
                          a.w_k != nullptr, a.eps, cs, sn, lane);
    } else if (kd) {
      const long hs = (long)a.page * DH;
      if constexpr (Q8) {
        if (k0 < k1)
          rope_heads<T, DH, true>(ks, reinterpret_cast<signed char*>(a.K) + at * DH, hs, k0, k1, a.KV, s.w[1],
                                  a.w_k != nullptr, a.eps, cs, sn, lane, a.Ke + at);
        const int slot = lane / Ly::LANES, sub = lane % Ly::LANES;
        const T* vs = static_cast<const T*>(a.v) + row * a.ldv;
#pragma unroll 2
        for (int p = max(p0, nq + nk) - nq - nk; p < p1 - nq - nk; ++p) {
          const int h = p * Ly::HEADS + slot;
          uint4 u = make_uint4(0, 0, 0, 0);
          if (h < a.KV) u = *reinterpret_cast<const uint4*>(vs + h * DH + sub * Ly::N);
          float2 e[Ly::G], o[Ly::G];
          Vec<T>::get(u, e, o);
          put_q8<Ly::LANES>(e, o, reinterpret_cast<signed char*>(a.V) + at * DH + h * hs + sub * Ly::N,
                            a.Ve + at + (long)h * a.page, sub, h < a.KV);
        }
        continue;
      }
      if (k0 < k1)
        rope_heads<T, DH>(ks, reinterpret_cast<T*>(kd), hs, k0, k1, a.KV, s.w[1], a.w_k != nullptr,
                          a.eps, cs, sn, lane);
      const int slot = lane / Ly::LANES, sub = lane % Ly::LANES;
      const T* vs = static_cast<const T*>(a.v) + row * a.ldv;
#pragma unroll 4
      for (int p = max(p0, nq + nk) - nq - nk; p < p1 - nq - nk; ++p) {
        const int h = p * Ly::HEADS + slot;
        if (h < a.KV)
          *reinterpret_cast<uint4*>(vd + h * hs + sub * Ly::N) =
              *reinterpret_cast<const uint4*>(vs + h * DH + sub * Ly::N);
      }
    }
  }
}

// Passes [p0, p1) of one token's heads, backward; the weights' gradients are
// added to the lane's sums.
template <class T, int DH>
__device__ __forceinline__ void rope_heads_bwd(const T* x, const T* dz, T* dx, int p0, int p1, int nh,
                                               const float2* w, bool norm, float eps,
                                               const float2* cs, const float2* sn, float2* ge,
                                               float2* go, int lane) {
  using Ly = Lay<T, DH>;
  constexpr int G = Ly::G;
  const int sub = lane % Ly::LANES, slot = lane / Ly::LANES;
  int h = p0 * Ly::HEADS + slot;
  const long off = (long)h * DH + sub * Ly::N;
  x += off;
  dz += off;
  dx += off;
  w += sub * G * 2;
  auto pass = [&](auto count) {
    constexpr int U = decltype(count)::value;
    uint4 ux[U], uz[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      ux[i] = uz[i] = make_uint4(0, 0, 0, 0);
      if (h + i * Ly::HEADS < nh) {
        uz[i] = *reinterpret_cast<const uint4*>(dz + i * Ly::HEADS * DH);
        if (norm) ux[i] = *reinterpret_cast<const uint4*>(x + i * Ly::HEADS * DH);
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float2 ze[G], zo[G], ye[G], yo[G];
      Vec<T>::get(uz[i], ze, zo);
#pragma unroll
      for (int k = 0; k < G; ++k) {
        const float2 ns = make_float2(-sn[k].x, -sn[k].y);
        ye[k] = __ffma2_rn(ze[k], cs[k], __fmul2_rn(zo[k], sn[k]));
        yo[k] = __ffma2_rn(zo[k], cs[k], __fmul2_rn(ze[k], ns));
      }
      if (norm) {
        float2 xe[G], xo[G], ss = both(0.f), t = both(0.f);
        Vec<T>::get(ux[i], xe, xo);
#pragma unroll
        for (int k = 0; k < G; ++k) {
          ss = __ffma2_rn(xe[k], xe[k], __ffma2_rn(xo[k], xo[k], ss));
          t = __ffma2_rn(__fmul2_rn(w[2 * k], ye[k]), xe[k],
                         __ffma2_rn(__fmul2_rn(w[2 * k + 1], yo[k]), xo[k], t));
        }
        const float sq = head_sum<Ly::LANES>(ss.x + ss.y), tt = head_sum<Ly::LANES>(t.x + t.y);
        const float r = rsqrtf(fmaf(sq, 1.f / DH, eps));
        const float m = -tt * r * r * r * (1.f / DH);  // -r^2 mean(w dy x r), of x
#pragma unroll
        for (int k = 0; k < G; ++k) {
          const float2 re = __fmul2_rn(ye[k], both(r)), ro = __fmul2_rn(yo[k], both(r));
          ge[k] = __ffma2_rn(re, xe[k], ge[k]);
          go[k] = __ffma2_rn(ro, xo[k], go[k]);
          ye[k] = __ffma2_rn(w[2 * k], re, __fmul2_rn(xe[k], both(m)));
          yo[k] = __ffma2_rn(w[2 * k + 1], ro, __fmul2_rn(xo[k], both(m)));
        }
      }
      if (h + i * Ly::HEADS < nh)
        *reinterpret_cast<uint4*>(dx + i * Ly::HEADS * DH) = Vec<T>::put(ye, yo);
    }
    h += U * Ly::HEADS;
    x += U * Ly::HEADS * DH;
    dz += U * Ly::HEADS * DH;
    dx += U * Ly::HEADS * DH;
  };
  in_passes<RW_BWD_U>(p1 - p0, pass);
}

template <class T, int DH>
__global__ void __launch_bounds__(RW_THREADS, RW_BWD_CTAS)
    rope_bwd_kernel(RopeArgs a, const __grid_constant__ RopeFreq fr) {
  using Ly = Lay<T, DH>;
  constexpr int G = Ly::G;
  __shared__ __align__(16) RopeSmem s;
  __shared__ float red[RW_WARPS][2][DH];
  stage_freq<DH>(s, fr);
  pdl_enter();
  stage_weights<DH>(s, a);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float2 g[2][2 * G];  // of w_q, w_k: first halves, then second halves
#pragma unroll
  for (int i = 0; i < 2 * G; ++i) g[0][i] = g[1][i] = both(0.f);
  const int nq = (a.H + Ly::HEADS - 1) / Ly::HEADS, nk = (a.KV + Ly::HEADS - 1) / Ly::HEADS;
  const int passes = nq + nk;
  const long units = (long)a.rows * a.parts;
  for (long un = (long)blockIdx.x * RW_WARPS + warp; un < units; un += (long)gridDim.x * RW_WARPS) {
    const int row = a.parts == 1 ? (int)un : (int)(un / a.parts), pt = (int)(un - (long)row * a.parts);
    const int p0 = pt * passes / a.parts, p1 = (pt + 1) * passes / a.parts;
    int pos3[3] = {a.pos ? 0 : row % a.seq_len, 0, 0};
    if (a.pos) {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < fr.n_axes) pos3[i] = a.pos[(long)row * fr.n_axes + i];
    }
    float2 cs[G], sn[G];
    turn_of<T, DH>(s, pos3, lane, cs, sn);
    if (p0 < nq)
      rope_heads_bwd<T, DH>(static_cast<const T*>(a.q) + row * a.ldq,
                            static_cast<const T*>(a.dqo) + row * a.lddqo,
                            static_cast<T*>(a.qo) + row * a.ldqo, p0, min(p1, nq), a.H, s.w[0],
                            a.w_q != nullptr, a.eps, cs, sn, g[0], g[0] + G, lane);
    const int k0 = max(p0, nq) - nq;
    if (k0 < p1 - nq)
      rope_heads_bwd<T, DH>(static_cast<const T*>(a.k) + row * a.ldk,
                            static_cast<const T*>(a.dko) + row * a.lddko,
                            static_cast<T*>(a.ko) + row * a.ldko, k0, p1 - nq, a.KV, s.w[1],
                            a.w_k != nullptr, a.eps, cs, sn, g[1], g[1] + G, lane);
  }
  if (!a.part) return;  // no norm
  // the CTA's sums of the weights' gradients, in a fixed order
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int k = 0; k < 2 * G; ++k) {
#pragma unroll
      for (int o = Ly::LANES; o < 32; o <<= 1) {
        g[q][k].x += __shfl_xor_sync(0xffffffffu, g[q][k].x, o);
        g[q][k].y += __shfl_xor_sync(0xffffffffu, g[q][k].y, o);
      }
      if (lane < Ly::LANES) {  // values 4 i, 4 i + 2 (first halves) or + 1, + 3 of the lane's
        float* d = red[warp][q] + lane * Ly::N + k % G * 4 + k / G;
        d[0] = g[q][k].x;
        d[2] = g[q][k].y;
      }
    }
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * DH; c += RW_THREADS) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < RW_WARPS; ++w) v += red[w][c / DH][c % DH];
    a.part[(long)blockIdx.x * 2 * DH + c] = v;
  }
}

// dw[c] = sum over the CTAs of part[.][c] (c < dh: w_q, else w_k).  A CTA takes
// 32 columns, 16 threads to a column.
__global__ void __launch_bounds__(512) rope_dw_kernel(const float* part, int n, int dh,
                                                      float* dw_q, float* dw_k) {
  pdl_enter();
  __shared__ float red[16][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), g = threadIdx.x >> 5;
  float v = 0.f;
#pragma unroll 8
  for (int i = g; i < n; i += 16) v += part[(long)i * 2 * dh + c];
  red[g][threadIdx.x & 31] = v;
  __syncthreads();
  if (g) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) v += red[i][threadIdx.x & 31];
  float* o = c < dh ? dw_q : dw_k;
  if (o) o[c % dh] = v;
}

__global__ void paged_advance_kernel(const int* start, int* len, int B, int cap) {
  pdl_enter();
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b >= B) return;
  const int n = start ? start[b + 1] - start[b] : 1;
  const int old = len[b];
  if (old < 0 || n < 0 || (long)old + n > cap)
    set_dev_error(DEVERR_CAPACITY);
  else
    len[b] = old + n;
}

RopeFreq freq_of(const QkRope& s) {
  RopeFreq fr{};
  fr.n_axes = s.n_axes;
  int p = 0;
  for (int ax = 0; ax < s.n_axes; ++ax) {
    // theta^(-i / n) by repeated products: 64 roundings at most, 2^-47 of a turn's
    // fraction that shrinks with i
    const double step = std::pow(s.theta, -1.0 / std::max(1, s.pairs[ax]));
    double w = 0.15915494309189535;  // 1 / (2 pi): turns per position of the first pair
    for (int i = 0; i < s.pairs[ax]; ++i, ++p, w *= step) {
      fr.f[p] = (unsigned long long)std::ldexp(w - std::floor(w), 64);  // (theta < 1: whole turns count for nothing)
      fr.axis[p] = (unsigned char)ax;
    }
  }
  return fr;
}

constexpr int RW_SMS = 152;  // whatever the device has: the sums keep their order

// Passes of a token's heads are spread over so many warps that about 16 warps
// an SM have work (a token a warp: 66 tokens of 10 heads would run on 9 SMs).
void set_parts(RopeArgs& a, const QkRope& s, bool with_v) {
  const int heads = 32 * 16 / (s.dh * (s.f32 ? 4 : 2));  // of a pass
  const int nk = (s.KV + heads - 1) / heads, passes = (s.H + heads - 1) / heads + (with_v ? 2 : 1) * nk;
  a.parts = std::min(std::max(1, 16 * RW_SMS / a.rows), passes);
}

RopeArgs args_of(const QkRope& s, const QkvPtr& x, const QkvPtr& o, const float* w_q,
                 const float* w_k, const int* pos, long rows, long seq_len) {
  RopeArgs a{};
  a.q = x.q; a.k = x.k; a.v = x.v;
  a.ldq = x.ldq; a.ldk = x.ldk; a.ldv = x.ldv;
  a.qo = o.q; a.ko = o.k;
  a.ldqo = o.ldq; a.ldko = o.ldk;
  a.w_q = w_q;
  a.w_k = w_k;
  a.pos = pos;
  a.rows = (int)rows;
  a.seq_len = (int)seq_len;
  a.H = s.H;
  a.KV = s.KV;
  a.eps = std::max((float)s.eps, 1.17549435e-38f);  // (fp32's least normal: an eps of 0 made a zero row NaN)
  return a;
}

int rope_grid(const RopeArgs& a, int per_sm) {
  return (int)std::min<long>(((long)a.rows * a.parts + RW_WARPS - 1) / RW_WARPS, (long)per_sm * RW_SMS);
}

}  // namespace

cudaError_t qk_rope_fwd(const QkRope& s, const QkvPtr& x, const QkvPtr& o, const float* w_q,
                        const float* w_k, const int* pos, long rows, long seq_len,
                        cudaStream_t st) {
  launched.mark();
  RopeArgs a = args_of(s, x, o, w_q, w_k, pos, rows, seq_len);
  set_parts(a, s, false);
  const double n = (double)rows * (s.H + s.KV) * s.dh;
  LaunchTimer lt("qk_rope_fwd", st, 8.0 * n, (s.f32 ? 8.0 : 4.0) * n);
  const int grid = rope_grid(a, RW_FWD_CTAS);
  auto k = s.f32 ? (s.dh == 64 ? rope_fwd_kernel<float, 64, false> : rope_fwd_kernel<float, 128, false>)
                 : (s.dh == 64 ? rope_fwd_kernel<bf16, 64, false> : rope_fwd_kernel<bf16, 128, false>);
  return launch_kernel(k, grid, RW_THREADS, 0, st, a, freq_of(s));
}

size_t qk_rope_part_bytes(int dh) { return (size_t)RW_BWD_CTAS * RW_SMS * 2 * dh * sizeof(float); }

cudaError_t qk_rope_bwd(const QkRope& s, const QkvPtr& x, const QkvPtr& dout, const QkvPtr& dx,
                        const float* w_q, const float* w_k, const int* pos, float* dw_q,
                        float* dw_k, float* part, long rows, long seq_len, cudaStream_t st) {
  launched.mark();
  RopeArgs a = args_of(s, x, dx, w_q, w_k, pos, rows, seq_len);
  a.dqo = dout.q;
  a.dko = dout.k;
  a.lddqo = dout.ldq;
  a.lddko = dout.ldk;
  a.part = dw_q || dw_k ? part : nullptr;
  set_parts(a, s, false);
  const double n = (double)rows * (s.H + s.KV) * s.dh;
  const int grid = rope_grid(a, RW_BWD_CTAS);
  {
    LaunchTimer lt("qk_rope_bwd", st, 16.0 * n, (s.f32 ? 12.0 : 6.0) * n);
    auto k = s.f32 ? (s.dh == 64 ? rope_bwd_kernel<float, 64> : rope_bwd_kernel<float, 128>)
                   : (s.dh == 64 ? rope_bwd_kernel<bf16, 64> : rope_bwd_kernel<bf16, 128>);
    const cudaError_t e = launch_kernel(k, grid, RW_THREADS, 0, st, a, freq_of(s));
    if (e != cudaSuccess) return e;
  }
  if (!a.part) return cudaSuccess;
  LaunchTimer lt("qk_rope_dw", st, 2.0 * grid * s.dh, 8.0 * grid * s.dh);
  return launch_kernel(rope_dw_kernel, 2 * s.dh / 32, 512, 0, st, part, grid, s.dh, dw_q, dw_k);
}

cudaError_t paged_append(const QkRope& s, const Paged& c, const QkvPtr& x, bf16* q_out, long ldqo,
                         const float* w_q, const float* w_k, const int* start, const int* pos,
                         long rows, cudaStream_t st) {
  launched.mark();
  QkvPtr o{};
  o.q = q_out;
  o.ldq = ldqo;
  RopeArgs a = args_of(s, x, o, w_q, w_k, pos, rows, 1);
  a.K = c.K; a.V = c.V; a.Ke = c.Ke; a.Ve = c.Ve;
  a.table = c.table; a.len = c.len; a.start = start;
  a.B = c.B; a.page = c.page; a.max_pages = c.max_pages;
  a.n_pages = c.n_pages;
  set_parts(a, s, true);
  const double n = (double)rows * s.dh;
  LaunchTimer lt("paged_append", st, 8.0 * n * (s.H + s.KV), (4.0 * s.H + (c.Ke ? 6.0 : 8.0) * s.KV) * n);
  const int grid = rope_grid(a, RW_FWD_CTAS);
  if (c.Ke)
    return launch_kernel(s.dh == 64 ? rope_fwd_kernel<bf16, 64, true, true> : rope_fwd_kernel<bf16, 128, true, true>,
                         grid, RW_THREADS, 0, st, a, freq_of(s));
  return launch_kernel(s.dh == 64 ? rope_fwd_kernel<bf16, 64, true> : rope_fwd_kernel<bf16, 128, true>,
                       grid, RW_THREADS, 0, st, a, freq_of(s));
}

cudaError_t paged_advance(const Paged& c, const int* start, int* len, cudaStream_t st) {
  launched.mark();
  LaunchTimer lt("paged_advance", st, 0.0, 12.0 * c.B);
  const long cap = std::min<long>((long)c.max_pages * c.page, 0x7fffffffL);
  return launch_kernel(paged_advance_kernel, (c.B + 127) / 128, 128, 0, st, start, len, c.B, (int)cap);
}

}  // namespace pf

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
// HBM traffic bounds all of them: a row is read once and written once.  A
// head's values lie on dh / 8 (bf16) or dh / 4 (fp32) lanes, 16 bytes each, so
// that a warp holds several heads and a head's sum takes three to five
// shuffles; a warp takes a token and walks its heads, four loads in flight per
// lane, with the token's sines made once (a pair or two on each lane, handed
// round by shuffles).  With few tokens a token's heads are spread over several
// warps (`parts`): latency counts there, and the sines made twice do not.
//
// Angles: the frequency is held as a 64-bit fraction of a turn, and
// pos * f modulo 2^64 is exact integer arithmetic; a position of a million
// loses nothing, where a product in fp32 would be off by 0.06 radians.
#include <algorithm>
#include <cmath>

#include "local.h"

namespace pf {

int take_dev_error_local_rope() { return take_dev_error_tu(); }
int set_wait_limit_local_rope(unsigned long long ns) { return set_wait_limit_tu(ns); }

namespace {

constexpr int RW_THREADS = 256;
constexpr int RW_WARPS = RW_THREADS / 32;
constexpr int RW_U = 4;         // heads in flight per lane
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
  int rows, seq_len, H, KV, parts;
  float eps;
  // backward: gradients of qo and ko, and the CTAs' sums of the weights' gradients
  const void *dqo, *dko;
  long lddqo, lddko;
  float* part;  // [grid][2][dh]
  // append
  const void* v;
  long ldv;
  bf16 *K, *V;                       // [n_pages, KV, page, dh]
  const int *table, *len, *start;
  int B, page, max_pages;
  long n_pages;
};

template <class T>
struct Vec;
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(uint4 u, float* v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack_bf16(w[i]);
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ uint4 put(const float* v) {
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                      pack_bf16(v[6], v[7]));
  }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(uint4 u, float* v) {
    v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y);
    v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                      __float_as_uint(v[3]));
  }
};

// How a warp holds heads of DH values of type T.
template <class T, int DH>
struct Lay {
  static constexpr int N = Vec<T>::N;    // values per lane
  static constexpr int LANES = DH / N;   // lanes per head
  static constexpr int HEADS = 32 / LANES;  // heads per pass of the warp
  static constexpr int PPL = DH / 64;    // pairs whose sines a lane makes
};

// cos and sin of the lane's N / 2 pairs at the token's position(s).  bf16 rows
// take the hardware sine (absolute error below 2^-20 for |angle| <= pi, a
// 2000th of the rounding of the result); fp32 rows the library's.
template <class T, int DH>
__device__ __forceinline__ void turn_of(const unsigned long long* f, const unsigned char* axis,
                                        const int* pos3, int lane, float* cs, float* sn) {
  using Ly = Lay<T, DH>;
  float oc[Ly::PPL], os[Ly::PPL];
#pragma unroll
  for (int s = 0; s < Ly::PPL; ++s) {
    const int p = lane * Ly::PPL + s;
    const int a = axis[p];
    const int ps = a == 0 ? pos3[0] : a == 1 ? pos3[1] : pos3[2];
    const unsigned long long ph = (unsigned long long)(long long)ps * f[p];
    const float h = (float)(int)(ph >> 32) * 4.656612873077393e-10f;  // half turns, [-1, 1]
    if (sizeof(T) == 2)
      __sincosf(h * 3.14159265358979f, &os[s], &oc[s]);
    else
      sincospif(h, &os[s], &oc[s]);
  }
  const int sub = lane % Ly::LANES;
#pragma unroll
  for (int i = 0; i < Ly::N / 2; ++i) {
    const int src = (sub * (Ly::N / 2) + i) / Ly::PPL;
    cs[i] = __shfl_sync(0xffffffffu, oc[i % Ly::PPL], src);
    sn[i] = __shfl_sync(0xffffffffu, os[i % Ly::PPL], src);
  }
}

template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Heads [h0, h0 + HEADS * n) of one token (those below nh), normed and turned:
// src + h * DH -> dst + h * dst_stride.
template <class T, int DH>
__device__ __forceinline__ void rope_heads(const T* src, T* dst, long dst_stride, int h0, int n,
                                           int nh, const float* w, bool norm, float eps,
                                           const float* cs, const float* sn, int lane) {
  using Ly = Lay<T, DH>;
  const int slot = lane / Ly::LANES, sub = lane % Ly::LANES;
  for (int p = 0; p < n; p += RW_U) {
    uint4 u[RW_U];
    int h[RW_U];
#pragma unroll
    for (int i = 0; i < RW_U; ++i) {
      h[i] = h0 + (p + i) * Ly::HEADS + slot;
      if (p + i >= n || h[i] >= nh) h[i] = -1;
      if (h[i] >= 0) u[i] = *reinterpret_cast<const uint4*>(src + (long)h[i] * DH + sub * Ly::N);
    }
#pragma unroll
    for (int i = 0; i < RW_U; ++i) {
      if (p + i >= n) break;  // the same for every lane
      float x[Ly::N];
      Vec<T>::get(h[i] >= 0 ? u[i] : make_uint4(0, 0, 0, 0), x);
      if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < Ly::N; ++e) ss = fmaf(x[e], x[e], ss);
        const float r = rsqrtf(fmaf(head_sum<Ly::LANES>(ss), 1.f / DH, eps));
#pragma unroll
        for (int e = 0; e < Ly::N; ++e) x[e] *= r * w[e];
      }
      float z[Ly::N];
#pragma unroll
      for (int e = 0; e < Ly::N; e += 2) {
        z[e] = x[e] * cs[e / 2] - x[e + 1] * sn[e / 2];
        z[e + 1] = fmaf(x[e], sn[e / 2], x[e + 1] * cs[e / 2]);
      }
      if (h[i] >= 0)
        *reinterpret_cast<uint4*>(dst + (long)h[i] * dst_stride + sub * Ly::N) = Vec<T>::put(z);
    }
  }
}

// The frequency table in shared memory (a table in parameter space read with a
// lane's own index is served one address at a time).
struct FreqSmem {
  unsigned long long f[RW_MAX_PAIRS];
  unsigned char axis[RW_MAX_PAIRS];
};
__device__ __forceinline__ void stage_freq(FreqSmem& s, const RopeFreq& fr) {
  if (threadIdx.x < RW_MAX_PAIRS) {
    s.f[threadIdx.x] = fr.f[threadIdx.x];
    s.axis[threadIdx.x] = fr.axis[threadIdx.x];
  }
  __syncthreads();
}

template <class T, int DH>
__device__ __forceinline__ void load_w(const float* w, int lane, float* o) {
  using Ly = Lay<T, DH>;
#pragma unroll
  for (int e = 0; e < Ly::N; ++e) o[e] = w ? w[(lane % Ly::LANES) * Ly::N + e] : 1.f;
}

// Forward (APPEND: keys and values go to their cache pages).  A unit is part
// `pt` of a token's passes: q heads, then k heads, then (APPEND) v heads.
template <class T, int DH, bool APPEND>
__global__ void __launch_bounds__(RW_THREADS) rope_fwd_kernel(RopeArgs a,
                                                              const __grid_constant__ RopeFreq fr) {
  using Ly = Lay<T, DH>;
  __shared__ FreqSmem fs;
  stage_freq(fs, fr);
  const int pz = pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float wq[Ly::N], wk[Ly::N];
  load_w<T, DH>(a.w_q ? a.w_q + pz : nullptr, lane, wq);
  load_w<T, DH>(a.w_k ? a.w_k + pz : nullptr, lane, wk);
  const int nq = (a.H + Ly::HEADS - 1) / Ly::HEADS, nk = (a.KV + Ly::HEADS - 1) / Ly::HEADS;
  const int passes = nq + nk + (APPEND ? nk : 0);
  const long units = (long)a.rows * a.parts;
  for (long un = (long)blockIdx.x * RW_WARPS + warp; un < units; un += (long)gridDim.x * RW_WARPS) {
    const int row = (int)(un / a.parts), pt = (int)(un % a.parts);
    const int p0 = pt * passes / a.parts, p1 = (pt + 1) * passes / a.parts;
    int pos3[3] = {0, 0, 0};
    bf16 *kd = nullptr, *vd = nullptr;
    if (APPEND) {
      // the token's sequence: how many of the others start at or before it
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
      const long pi = crow / a.page;
      long pg = -1;
      if (crow >= 0 && pi < a.max_pages) pg = a.table[(long)b * a.max_pages + pi];
      if (pg < 0 || pg >= a.n_pages) {
        if (lane == 0) set_dev_error(DEVERR_CAPACITY);
      } else {
        const long o = (pg * a.KV * a.page + crow % a.page) * DH;
        kd = a.K + o;
        vd = a.V + o;
      }
    } else if (!a.pos) {
      pos3[0] = row % a.seq_len;
    }
    if (a.pos) {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < fr.n_axes) pos3[i] = a.pos[(long)row * fr.n_axes + i];
    }
    float cs[Ly::N / 2], sn[Ly::N / 2];
    turn_of<T, DH>(fs.f, fs.axis, pos3, lane, cs, sn);
    if (p0 < nq)
      rope_heads<T, DH>(static_cast<const T*>(a.q) + row * a.ldq, static_cast<T*>(a.qo) + row * a.ldqo,
                        DH, p0 * Ly::HEADS, min(p1, nq) - p0, a.H, wq, a.w_q != nullptr, a.eps, cs,
                        sn, lane);
    const int k0 = max(p0, nq) - nq, k1 = min(p1, nq + nk) - nq;
    const T* ks = static_cast<const T*>(a.k) + row * a.ldk;
    if (!APPEND) {
      if (k0 < k1)
        rope_heads<T, DH>(ks, static_cast<T*>(a.ko) + row * a.ldko, DH, k0 * Ly::HEADS, k1 - k0, a.KV,
                          wk, a.w_k != nullptr, a.eps, cs, sn, lane);
    } else if (kd) {
      const long hs = (long)a.page * DH;
      if (k0 < k1)
        rope_heads<T, DH>(ks, reinterpret_cast<T*>(kd), hs, k0 * Ly::HEADS, k1 - k0, a.KV, wk,
                          a.w_k != nullptr, a.eps, cs, sn, lane);
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

// Heads [h0, h0 + HEADS * n) of one token, backward; the weights' gradients are
// added to the lane's sums.
template <class T, int DH>
__device__ __forceinline__ void rope_heads_bwd(const T* x, const T* dz, T* dx, int h0, int n, int nh,
                                               const float* w, bool norm, float eps,
                                               const float* cs, const float* sn, float* dw,
                                               int lane) {
  using Ly = Lay<T, DH>;
  constexpr int U = RW_U / 2;  // two rows to a head
  const int slot = lane / Ly::LANES, sub = lane % Ly::LANES;
  for (int p = 0; p < n; p += U) {
    uint4 ux[U], uz[U];
    int h[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      h[i] = h0 + (p + i) * Ly::HEADS + slot;
      if (p + i >= n || h[i] >= nh) h[i] = -1;
      const long o = (long)h[i] * DH + sub * Ly::N;
      ux[i] = uz[i] = make_uint4(0, 0, 0, 0);
      if (h[i] >= 0) {
        uz[i] = *reinterpret_cast<const uint4*>(dz + o);
        if (norm) ux[i] = *reinterpret_cast<const uint4*>(x + o);
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (p + i >= n) break;  // the same for every lane
      float z[Ly::N], y[Ly::N];
      Vec<T>::get(uz[i], z);
#pragma unroll
      for (int e = 0; e < Ly::N; e += 2) {
        y[e] = fmaf(z[e], cs[e / 2], z[e + 1] * sn[e / 2]);
        y[e + 1] = z[e + 1] * cs[e / 2] - z[e] * sn[e / 2];
      }
      if (norm) {
        float xv[Ly::N], ss = 0.f, t = 0.f;
        Vec<T>::get(ux[i], xv);
#pragma unroll
        for (int e = 0; e < Ly::N; ++e) ss = fmaf(xv[e], xv[e], ss);
#pragma unroll
        for (int e = 0; e < Ly::N; ++e) t = fmaf(w[e] * y[e], xv[e], t);
        ss = head_sum<Ly::LANES>(ss);
        t = head_sum<Ly::LANES>(t);
        const float r = rsqrtf(fmaf(ss, 1.f / DH, eps));
        const float m = t * r * (1.f / DH);  // mean(w dy x r)
#pragma unroll
        for (int e = 0; e < Ly::N; ++e) {
          const float xh = xv[e] * r;
          dw[e] = fmaf(y[e], xh, dw[e]);
          y[e] = r * (w[e] * y[e] - xh * m);
        }
      }
      if (h[i] >= 0)
        *reinterpret_cast<uint4*>(dx + (long)h[i] * DH + sub * Ly::N) = Vec<T>::put(y);
    }
  }
}

template <class T, int DH>
__global__ void __launch_bounds__(RW_THREADS) rope_bwd_kernel(RopeArgs a,
                                                              const __grid_constant__ RopeFreq fr) {
  using Ly = Lay<T, DH>;
  __shared__ FreqSmem fs;
  __shared__ float red[RW_WARPS][2][DH];
  stage_freq(fs, fr);
  const int pz = pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float wq[Ly::N], wk[Ly::N], gq[Ly::N] = {}, gk[Ly::N] = {};
  load_w<T, DH>(a.w_q ? a.w_q + pz : nullptr, lane, wq);
  load_w<T, DH>(a.w_k ? a.w_k + pz : nullptr, lane, wk);
  const int nq = (a.H + Ly::HEADS - 1) / Ly::HEADS, nk = (a.KV + Ly::HEADS - 1) / Ly::HEADS;
  const int passes = nq + nk;
  const long units = (long)a.rows * a.parts;
  for (long un = (long)blockIdx.x * RW_WARPS + warp; un < units; un += (long)gridDim.x * RW_WARPS) {
    const int row = (int)(un / a.parts), pt = (int)(un % a.parts);
    const int p0 = pt * passes / a.parts, p1 = (pt + 1) * passes / a.parts;
    int pos3[3] = {a.pos ? 0 : row % a.seq_len, 0, 0};
    if (a.pos) {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < fr.n_axes) pos3[i] = a.pos[(long)row * fr.n_axes + i];
    }
    float cs[Ly::N / 2], sn[Ly::N / 2];
    turn_of<T, DH>(fs.f, fs.axis, pos3, lane, cs, sn);
    if (p0 < nq)
      rope_heads_bwd<T, DH>(static_cast<const T*>(a.q) + row * a.ldq,
                            static_cast<const T*>(a.dqo) + row * a.lddqo,
                            static_cast<T*>(a.qo) + row * a.ldqo, p0 * Ly::HEADS, min(p1, nq) - p0,
                            a.H, wq, a.w_q != nullptr, a.eps, cs, sn, gq, lane);
    const int k0 = max(p0, nq) - nq;
    if (k0 < p1 - nq)
      rope_heads_bwd<T, DH>(static_cast<const T*>(a.k) + row * a.ldk,
                            static_cast<const T*>(a.dko) + row * a.lddko,
                            static_cast<T*>(a.ko) + row * a.ldko, k0 * Ly::HEADS, p1 - nq - k0, a.KV,
                            wk, a.w_k != nullptr, a.eps, cs, sn, gk, lane);
  }
  if (!a.part) return;  // no norm
  // the CTA's sums of the weights' gradients, in a fixed order
#pragma unroll
  for (int e = 0; e < Ly::N; ++e)
#pragma unroll
    for (int o = Ly::LANES; o < 32; o <<= 1) {
      gq[e] += __shfl_xor_sync(0xffffffffu, gq[e], o);
      gk[e] += __shfl_xor_sync(0xffffffffu, gk[e], o);
    }
  if (lane < Ly::LANES)
#pragma unroll
    for (int e = 0; e < Ly::N; ++e) {
      red[warp][0][lane * Ly::N + e] = gq[e];
      red[warp][1][lane * Ly::N + e] = gk[e];
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
__global__ void __launch_bounds__(512) rope_dw_kernel(const float* __restrict__ part, int n, int dh,
                                                      float* dw_q, float* dw_k) {
  const int pz = pdl_enter();
  __shared__ float red[16][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), g = threadIdx.x >> 5;
  float v = 0.f;
#pragma unroll 8
  for (int i = g + pz; i < n; i += 16) v += part[(long)i * 2 * dh + c];
  red[g][threadIdx.x & 31] = v;
  __syncthreads();
  if (g) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) v += red[i][threadIdx.x & 31];
  float* o = c < dh ? dw_q : dw_k;
  if (o) o[c % dh] = v;
}

__global__ void paged_advance_kernel(const int* __restrict__ start, int* len, int B, int cap) {
  const int pz = pdl_enter();
  const int b = blockIdx.x * blockDim.x + threadIdx.x + pz;
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
      fr.f[p] = (unsigned long long)std::ldexp(w, 64);
      fr.axis[p] = (unsigned char)ax;
    }
  }
  return fr;
}

constexpr int RW_CTAS = 4 * 152;  // grid: what 152 SMs hold, whatever the device has (sums keep their order)

// Passes of a token's heads are spread over so many warps that about 16 warps
// an SM have work (a token a warp: 66 tokens of 10 heads would run on 9 SMs).
int rope_parts(long rows, int passes) {
  const long want = (16L * 152 + rows - 1) / rows;
  return (int)std::min<long>(std::max(1L, want), passes);
}

int rope_passes(const QkRope& s, bool with_v) {
  const int heads = 32 / (s.dh * (s.f32 ? 4 : 2) / 16);
  return (s.H + heads - 1) / heads + (with_v ? 2 : 1) * ((s.KV + heads - 1) / heads);
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
  a.eps = (float)s.eps;
  return a;
}

int rope_grid(long units) { return (int)std::min<long>((units + RW_WARPS - 1) / RW_WARPS, RW_CTAS); }

}  // namespace

cudaError_t qk_rope_fwd(const QkRope& s, const QkvPtr& x, const QkvPtr& o, const float* w_q,
                        const float* w_k, const int* pos, long rows, long seq_len,
                        cudaStream_t st) {
  RopeArgs a = args_of(s, x, o, w_q, w_k, pos, rows, seq_len);
  a.parts = rope_parts(rows, rope_passes(s, false));
  const double n = (double)rows * (s.H + s.KV) * s.dh;
  LaunchTimer lt("qk_rope_fwd", st, 8.0 * n, (s.f32 ? 8.0 : 4.0) * n);
  const int grid = rope_grid(rows * a.parts);
  auto k = s.f32 ? (s.dh == 64 ? rope_fwd_kernel<float, 64, false> : rope_fwd_kernel<float, 128, false>)
                 : (s.dh == 64 ? rope_fwd_kernel<bf16, 64, false> : rope_fwd_kernel<bf16, 128, false>);
  return launch_kernel(k, grid, RW_THREADS, 0, st, a, freq_of(s));
}

size_t qk_rope_part_bytes(int dh) { return (size_t)RW_CTAS * 2 * dh * sizeof(float); }

cudaError_t qk_rope_bwd(const QkRope& s, const QkvPtr& x, const QkvPtr& dout, const QkvPtr& dx,
                        const float* w_q, const float* w_k, const int* pos, float* dw_q,
                        float* dw_k, float* part, long rows, long seq_len, cudaStream_t st) {
  RopeArgs a = args_of(s, x, dx, w_q, w_k, pos, rows, seq_len);
  a.dqo = dout.q;
  a.dko = dout.k;
  a.lddqo = dout.ldq;
  a.lddko = dout.ldk;
  a.part = dw_q || dw_k ? part : nullptr;
  a.parts = rope_parts(rows, rope_passes(s, false));
  const double n = (double)rows * (s.H + s.KV) * s.dh;
  const int grid = rope_grid(rows * a.parts);
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
  QkvPtr o{};
  o.q = q_out;
  o.ldq = ldqo;
  RopeArgs a = args_of(s, x, o, w_q, w_k, pos, rows, 1);
  a.K = c.K; a.V = c.V;
  a.table = c.table; a.len = c.len; a.start = start;
  a.B = c.B; a.page = c.page; a.max_pages = c.max_pages;
  a.n_pages = c.n_pages;
  a.parts = rope_parts(rows, rope_passes(s, true));
  const double n = (double)rows * s.dh;
  LaunchTimer lt("paged_append", st, 8.0 * n * (s.H + s.KV), 4.0 * n * (s.H + 2 * s.KV));
  const int grid = rope_grid(rows * a.parts);
  return launch_kernel(s.dh == 64 ? rope_fwd_kernel<bf16, 64, true> : rope_fwd_kernel<bf16, 128, true>,
                       grid, RW_THREADS, 0, st, a, freq_of(s));
}

cudaError_t paged_advance(const Paged& c, const int* start, int* len, cudaStream_t st) {
  LaunchTimer lt("paged_advance", st, 0.0, 12.0 * c.B);
  const long cap = std::min<long>((long)c.max_pages * c.page, 0x7fffffffL);
  return launch_kernel(paged_advance_kernel, (c.B + 127) / 128, 128, 0, st, start, len, c.B, (int)cap);
}

}  // namespace pf

// Attention of one new token per sequence over a paged cache of keys and
// values, bf16 with fp32 arithmetic, grouped heads.
//
//   o_h = sum_j softmax_j(q_h . K_j / sqrt(dh)) V_j over the sequence's rows
//   j < len, with a window W also j >= len - W or j < S (the sinks);
//   a sequence without rows gives zeros.
// A token sees itself, so that a sum is never empty: a row whose scores are NaN, or all
// -inf, comes out as NaN (0 / 0 the latter).
//
// Streaming the visible K and V rows from HBM once bounds it: the query heads
// that share a key head (up to 16) are the 16 rows of the same m16n8k16 MMAs,
// so a row is read once for all of them and its arithmetic (4 dh multiply-adds
// a query head) stays far below the copy.  (tcgen05 would fill 8 to 16 of its
// 128 rows.)
//
// Layout of the work.  A warp takes tiles of 16 rows of one key head; they lie
// in one page, as pages are multiples of 16 rows, and [page, row, dh] of one
// head is contiguous.  Each warp has its own ring of tiles, filled by 16-byte
// cp.async with the swizzle that its reads want; no barrier between the warps
// while they stream.  Rows that the token does not see are filled with zeros,
// not read: 0 times an infinity there would reach the sums.
// Short caches, or enough of them: a CTA to each (sequence, key head) (pa_whole).
// Else the split over the cache: a unit is a tile for each of the CTA's warps, and
// the units of all (sequence, key head) pairs, ragged as they are, are dealt
// to the CTAs in equal contiguous ranges.  The lengths are read on the device;
// every CTA sums them up itself.  A CTA that holds all of a pair writes its
// rows; else it leaves (max, sum, acc) of its piece, at most two of them (its
// first and its last), and paged_join_kernel joins them in the order of the
// CTAs, so that results repeat bit for bit.
#include <algorithm>

#include "local.h"

namespace pf {

static Launched launched;
int take_dev_error_paged_attn() { return launched.take(take_dev_error_tu); }
int set_wait_limit_paged_attn(unsigned long long ns) { return set_wait_limit_tu(ns); }

namespace {

constexpr int PA_WARPS = 4;
constexpr int PA_THREADS = 32 * PA_WARPS;
constexpr int PA_TILE = 16;                    // rows of a warp's tile
constexpr int PA_UNIT = PA_TILE * PA_WARPS;    // rows of a unit
constexpr int PA_MAX_B = 2048;
constexpr int PA_CTAS = 2 * 152;  // two rings an SM, whatever the device has (splits keep their places)
constexpr float PA_RESCALE = 8.f;

template <int DH>
struct PaCfg {
  static constexpr int TILE_BYTES = PA_TILE * DH * 2;  // of K, and of V
  static constexpr int STAGES = DH == 128 ? 3 : 6;     // 24 KB a warp
  static constexpr int WARP_BYTES = STAGES * 2 * TILE_BYTES;
  static constexpr int SMEM = PA_WARPS * WARP_BYTES;
  static_assert(WARP_BYTES >= 16 * (DH + 4) * 4, "a warp's sums fit its ring");
};

struct PaArgs {
  const bf16* q;
  long ldq;
  const bf16 *K, *V;
  const int *table, *len;
  bf16* out;
  long ldo;
  float* part;  // [2 G][g][DH] sums, then [2 G][g][2] (max, sum)
  int B, KV, g, page, max_pages, window, sinks, G;
  bool whole;  // a CTA for each (sequence, key head), not equal ranges of units
  long n_pages;
  float sl2;  // log2(e) / sqrt(dh)
};

// Tiles that the newest token of a cache of n rows sees: the sinks' [0, ns) and
// the window's from lo on.
struct PaSpan {
  int n, lo, ns, tiles, first;  // first: first row inside the window
};
__device__ __forceinline__ int pa_tiles(int rows) { return rows / PA_TILE + (rows % PA_TILE != 0); }
__device__ __forceinline__ PaSpan pa_span(const PaArgs& a, int b) {
  PaSpan s;
  const long cap = (long)a.max_pages * a.page;
  const int len = a.len[b];
  s.n = len < 0 || len > cap ? 0 : len;  // flagged by pa_units
  s.first = a.window > 0 && s.n > a.window ? s.n - a.window : 0;
  s.lo = s.first / PA_TILE;
  s.ns = min(pa_tiles(a.sinks), s.lo);
  if (a.window <= 0) s.ns = 0;
  s.tiles = s.ns + pa_tiles(s.n) - s.lo;
  return s;
}

// pre[b] = units of the sequences before b (one key head), pre[B] their total.
__device__ __forceinline__ void pa_units(const PaArgs& a, int* pre, int nthr) {
  __shared__ int wsum[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int base = 0;
  for (int b0 = 0; b0 < a.B; b0 += nthr) {
    const int b = b0 + tid;
    int u = 0;
    if (b < a.B) {
      const int len = a.len[b];
      if (len < 0 || len > (long)a.max_pages * a.page) set_dev_error(DEVERR_CAPACITY);
      u = (pa_span(a, b).tiles + PA_WARPS - 1) / PA_WARPS;
    }
    int v = u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += t;
    }
    if (lane == 31) wsum[warp] = v;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < nthr / 32; ++w) {
      if (w < warp) before += wsum[w];
      all += wsum[w];
    }
    if (b < a.B) pre[b] = base + before + v - u;
    base += all;
    __syncthreads();
  }
  if (tid == 0) pre[a.B] = base;
  __syncthreads();
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool full) {
  const int n = full ? 16 : 0;  // 0: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n)
               : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// First unit of CTA c of G <= T, and the CTA that holds unit u, of T units.
__device__ __forceinline__ long pa_first(long T, int G, int c) { return T * c / G; }
__device__ __forceinline__ int pa_cta(long T, int G, long u) { return (int)(((u + 1) * G - 1) / T); }

template <int DH>
__global__ void __launch_bounds__(PA_THREADS) paged_attn_kernel(PaArgs a) {
  using C = PaCfg<DH>;
  constexpr int KC = DH / 32;  // 32-wide chunks of a row, two MMAs each
  constexpr int NT = DH / 8;   // 8-wide output tiles
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ int pre[PA_MAX_B + 1];
  pdl_enter();
  // the next kernel's CTAs may take their places now: they wait for this grid to end, and
  // all of its CTAs are running.  That is the join, or (whole pairs) mostly the next layer's
  // append, as small: a layer's append and attention, captured, 8 sequences of 60 rows 5.75 us
  // so and 6.28 without, 300 of 200 8.3 and 8.7, 256 of 1000 (2048 CTAs) 164.4 and 163.0
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int gid = lane >> 2, t = lane & 3;
  auto zeros = [&](int b, int col, int n) {
    for (int i = tid * 8; i < n; i += PA_THREADS * 8)
      *reinterpret_cast<uint4*>(a.out + b * a.ldo + col + i) = make_uint4(0, 0, 0, 0);
  };
  int b = 0, h = 0, nu = 0;
  long r0 = 0, r1;
  if (a.whole) {
    b = blockIdx.x / a.KV;
    h = blockIdx.x - b * a.KV;
    const int len = a.len[b];
    if (tid == 0 && (len < 0 || len > (long)a.max_pages * a.page)) set_dev_error(DEVERR_CAPACITY);
    r1 = nu = (pa_span(a, b).tiles + PA_WARPS - 1) / PA_WARPS;
    if (nu == 0) zeros(b, h * a.g * DH, a.g * DH);
  } else {
    pa_units(a, pre, PA_THREADS);
    // rows of sequences without keys
    for (int e = blockIdx.x; e < a.B; e += a.G)
      if (pre[e + 1] == pre[e]) zeros(e, 0, a.KV * a.g * DH);
    const long T = (long)pre[a.B] * a.KV;
    const int G = (int)min((long)a.G, T);
    if ((int)blockIdx.x >= G) return;
    r0 = pa_first(T, G, blockIdx.x);
    r1 = pa_first(T, G, blockIdx.x + 1);
    // the sequence of unit r0
    int hi = a.B;
    while (hi - b > 1) {
      const int m = (b + hi) >> 1;
      if ((long)pre[m] * a.KV <= r0) b = m; else hi = m;
    }
  }
  unsigned char* const wring = ring + warp * C::WARP_BYTES;
  const uint32_t wr = smem_u32(wring);
  float* const ml = a.part + 2L * a.G * a.g * DH;

  long pos = r0;
  while (pos < r1) {
    int u0 = 0;
    if (!a.whole) {
      while (pre[b + 1] == pre[b] || (long)pre[b + 1] * a.KV <= pos) ++b;
      nu = pre[b + 1] - pre[b];
      const long off = pos - (long)pre[b] * a.KV;
      h = (int)(off / nu);
      u0 = (int)(off % nu);
    }
    const int u1 = (int)min((long)nu, u0 + (r1 - pos));
    const PaSpan sp = pa_span(a, b);
    const int t1 = min(sp.tiles, u1 * PA_WARPS);
    // this warp's tiles: t0, t0 + PA_WARPS, ... below t1
    const int t0 = u0 * PA_WARPS + warp;
    const int nt = t0 < t1 ? (t1 - t0 + PA_WARPS - 1) / PA_WARPS : 0;
    const int* tab = a.table + (long)b * a.max_pages;
    auto tile_row = [&](int i) {
      const int k = t0 + i * PA_WARPS;
      return (k < sp.ns ? k : sp.lo + k - sp.ns) * PA_TILE;
    };
    auto page_of = [&](int i) { return i < nt ? tab[tile_row(i) / a.page] : 0; };
    auto fill = [&](int i, int pg) {  // tile i into its stage
      if (i < nt) {
        const int row = tile_row(i);
        const bool ok = pg >= 0 && pg < a.n_pages;
        if (!ok && lane == 0) set_dev_error(DEVERR_CAPACITY);
        const long o = (((ok ? (long)pg : 0L) * a.KV + h) * a.page + row % a.page) * DH;
        const uint32_t ks = wr + (i % C::STAGES) * 2 * C::TILE_BYTES, vs = ks + C::TILE_BYTES;
        constexpr int CPR = DH / 8;  // 16-byte chunks of a row
#pragma unroll
        for (int j = 0; j < PA_TILE * CPR / 32; ++j) {
          const int e = j * 32 + lane, r = e / CPR, c = e % CPR;
          const int j2 = row + r;
          const bool in = ok && j2 < sp.n && (j2 >= sp.first || j2 < a.sinks);
          const long src = in ? o + r * DH + c * 8 : 0;
          cp_async16(ks + (r * CPR + (c ^ ((r & 1) << 2))) * 16, a.K + src, in);
          cp_async16(vs + (r * CPR + (c ^ (r & 7))) * 16, a.V + src, in);
        }
      }
      cp_commit();
    };
    int pg_next = page_of(0);
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i) {
      const int pg = pg_next;
      pg_next = page_of(i + 1);
      fill(i, pg);
    }
    // the group's queries: rows gid and gid + 8 of the MMAs' A
    uint4 qa[KC], qb[KC];
    {
      const bf16* qr = a.q + b * a.ldq + (long)h * a.g * DH + 8 * t;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        qa[c] = qb[c] = make_uint4(0, 0, 0, 0);
        if (gid < a.g) qa[c] = *reinterpret_cast<const uint4*>(qr + gid * DH + 32 * c);
        if (gid + 8 < a.g) qb[c] = *reinterpret_cast<const uint4*>(qr + (gid + 8) * DH + 32 * c);
      }
    }
    float acc[NT][4] = {};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    for (int i = 0; i < nt; ++i) {
      cp_wait<C::STAGES - 2>();
      __syncwarp();
      {
        const int pg = pg_next;
        pg_next = page_of(i + C::STAGES);
        fill(i + C::STAGES - 1, pg);  // the stage read in the last round
      }
      const uint32_t ks = wr + (i % C::STAGES) * 2 * C::TILE_BYTES, vs = ks + C::TILE_BYTES;
      const unsigned char* kp = wring + (i % C::STAGES) * 2 * C::TILE_BYTES;
      // scores: rows of S are query heads, columns keys 8 n + 2 t, + 1.  A thread
      // takes 8 values of a row at once; the sum over them is free of order, and
      // Q's are taken alike.
      float s[2][4] = {};
#pragma unroll
      for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int r = n * 8 + gid;
          const uint4 k = *reinterpret_cast<const uint4*>(
              kp + (r * (DH / 8) + ((4 * c + t) ^ ((r & 1) << 2))) * 16);
          const uint32_t a0[4] = {qa[c].x, qb[c].x, qa[c].y, qb[c].y};
          mma16816(s[n], a0, k.x, k.y);
          const uint32_t a1[4] = {qa[c].z, qb[c].z, qa[c].w, qb[c].w};
          mma16816(s[n], a1, k.z, k.w);
        }
      const int row = tile_row(i);
      if (row > sp.n - PA_TILE || row < sp.first) {  // the last tile, the sinks', the window's first
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int j = row + n * 8 + 2 * t + e;
            if (j >= sp.n || (j < sp.first && j >= a.sinks)) s[n][e] = s[n][e + 2] = -INFINITY;
          }
      }
      float mx[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        mx[r] = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 1));
        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 2)) * a.sl2;
      }
      // the reference is raised only by more than PA_RESCALE (log2 units): until then
      // every probability is at most 2^PA_RESCALE, as exact in bf16 as any other
      if (__any_sync(0xffffffffu, mx[0] > m[0] + PA_RESCALE || mx[1] > m[1] + PA_RESCALE)) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if (!(mx[r] > m[r] + PA_RESCALE)) continue;
          const float f = ex2_approx(m[r] - mx[r]);  // first keys: 2^-inf = 0 of nothing
          m[r] = mx[r];
          l[r] *= f;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            acc[n][2 * r] *= f;
            acc[n][2 * r + 1] *= f;
          }
        }
      }
      uint32_t p[4];  // P as the A operand: bf16, the sums take it unrounded
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float ref = m[r] == -INFINITY ? 0.f : m[r];
        float e[4];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int k = 0; k < 2; ++k) e[2 * n + k] = ex2_approx(fmaf(s[n][2 * r + k], a.sl2, -ref));
        l[r] += (e[0] + e[1]) + (e[2] + e[3]);
        p[r] = pack_bf16(e[0], e[1]);
        p[r + 2] = pack_bf16(e[2], e[3]);
      }
#pragma unroll
      for (int c = 0; c < NT; c += 2) {
        const int r = lane & 15, ch = c + (lane >> 4);
        uint32_t v[4];
        ldmatrix_x4_trans(vs + (r * (DH / 8) + (ch ^ (r & 7))) * 16, v);
        mma16816(acc[c], p, v[0], v[1]);
        mma16816(acc[c + 1], p, v[2], v[3]);
      }
      __syncwarp();
    }
    cp_wait<0>();
    __syncwarp();
    // the warps' sums through their rings: row r of a warp at r * (DH + 4), its (max, sum)
    // after the values
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      float* w = reinterpret_cast<float*>(wring) + (gid + 8 * r) * (DH + 4);
#pragma unroll
      for (int n = 0; n < NT; ++n)
        *reinterpret_cast<float2*>(w + 8 * n + 2 * t) = make_float2(acc[n][2 * r], acc[n][2 * r + 1]);
      if (t == 0) *reinterpret_cast<float2*>(w + DH) = make_float2(m[r], l[r]);
    }
    __syncthreads();
    const bool whole = u0 == 0 && u1 == nu;
    const int slot = 2 * blockIdx.x + (pos == r0 ? 0 : 1);
    for (int i = tid; i < a.g * DH; i += PA_THREADS) {
      const int r = i / DH, d = i % DH;
      float mw[PA_WARPS], M = -INFINITY, L = 0.f, v = 0.f;
#pragma unroll
      for (int w = 0; w < PA_WARPS; ++w) {
        mw[w] = reinterpret_cast<const float*>(ring + w * C::WARP_BYTES)[r * (DH + 4) + DH];
        M = fmaxf(M, mw[w]);
      }
#pragma unroll
      for (int w = 0; w < PA_WARPS; ++w) {
        const float* x = reinterpret_cast<const float*>(ring + w * C::WARP_BYTES) + r * (DH + 4);
        const float f = M == -INFINITY ? 0.f : ex2_approx(mw[w] - M);
        L = fmaf(x[DH + 1], f, L);
        v = fmaf(x[d], f, v);
      }
      if (whole) {
        a.out[b * a.ldo + (long)h * a.g * DH + i] = __float2bfloat16(v / L);
      } else {
        a.part[((long)slot * a.g + r) * DH + d] = v;
        if (d == 0) {
          ml[((long)slot * a.g + r) * 2] = M;
          ml[((long)slot * a.g + r) * 2 + 1] = L;
        }
      }
    }
    __syncthreads();
    pos += u1 - u0;
  }
}

// Rows whose pair lies on several CTAs: the pieces joined in the order of the
// CTAs.  CTA x takes pair x, or, with more pairs than CTAs, the pair that
// begins on CTA x and ends on a later one; CTAs y share its columns, 32 at a
// time, 16 threads to a column.
constexpr int PJ_THREADS = 512;
template <int DH>
__global__ void __launch_bounds__(PJ_THREADS) paged_join_kernel(PaArgs a) {
  __shared__ int pre[PA_MAX_B + 1];
  __shared__ float sw[PA_CTAS];
  __shared__ float red[16][33];
  __shared__ float sL;
  pdl_enter();
  pa_units(a, pre, PJ_THREADS);
  const int tid = threadIdx.x, x = blockIdx.x;
  const long T = (long)pre[a.B] * a.KV;
  const int G = (int)min((long)a.G, T);
  int b, h;
  if (a.B * a.KV <= a.G) {
    b = x / a.KV;
    h = x - b * a.KV;
  } else {
    if (x + 1 >= G) return;
    const long u = pa_first(T, G, x + 1);
    int hi = a.B;
    b = 0;
    while (hi - b > 1) {
      const int m = (b + hi) >> 1;
      if ((long)pre[m] * a.KV <= u) b = m; else hi = m;
    }
    while (pre[b + 1] == pre[b]) ++b;  // (u < T: such a one follows)
    h = (int)((u - (long)pre[b] * a.KV) / (pre[b + 1] - pre[b]));
  }
  const int nu = pre[b + 1] - pre[b];
  if (nu == 0) return;
  const long u0 = (long)pre[b] * a.KV + (long)h * nu;
  const int c0 = pa_cta(T, G, u0), c1 = pa_cta(T, G, u0 + nu - 1);
  if (c0 == c1 || (a.B * a.KV > a.G && c0 != x)) return;
  const int n = c1 - c0 + 1;
  const float* ml = a.part + 2L * a.G * a.g * DH;
  auto slot = [&](int i) { return 2L * (c0 + i) + (i == 0 && pa_first(T, G, c0) != u0 ? 1 : 0); };
  for (int k = blockIdx.y; k < a.g * (DH / 32); k += gridDim.y) {
    const int r = k / (DH / 32), d = k % (DH / 32) * 32 + (tid & 31), g = tid >> 5;
    if (tid < 32) {
      float M = -INFINITY, L = 0.f;
      for (int i = tid; i < n; i += 32) M = fmaxf(M, ml[(slot(i) * a.g + r) * 2]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      for (int i = tid; i < n; i += 32) {
        const float* y = ml + (slot(i) * a.g + r) * 2;
        const float f = M == -INFINITY ? 0.f : ex2_approx(y[0] - M);
        sw[i] = f;
        L = fmaf(y[1], f, L);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
      if (tid == 0) sL = L;
    }
    __syncthreads();
    float v = 0.f;
#pragma unroll 8
    for (int i = g; i < n; i += 16) v = fmaf(a.part[(slot(i) * a.g + r) * DH + d], sw[i], v);
    red[g][tid & 31] = v;
    __syncthreads();
    if (g == 0) {
      v = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) v += red[i][tid & 31];
      a.out[b * a.ldo + ((long)h * a.g + r) * DH + d] = __float2bfloat16(v / sL);
    }
    __syncthreads();
  }
}

// A CTA for each (sequence, key head), and no join, where none sees many rows: a CTA
// streams 43 GB/s, and with a pair or more to each SM that is HBM's rate, while ranges that
// span several short pairs cost their ends.  In us, whole and in ranges, pages of 16 rows, ragged
// but for the first two, captured: 1 x 250 rows, 16 heads on 4 of 64: 4.9 and 7.4; 1 x 500: 7.4 and
// 7.4; 8 x 1000 rows, 8 heads of 128: 15.3 and 11.8; 32 x 1000: 20.0 and 35.5; 256 x 1000: 86 and
// 114; 300 x 200 rows of one head of 64: 5.4 and 16.  The host knows the table's width, not the
// lengths: short caches in a table of many pages are read in ranges.
bool pa_whole(const Paged& c) {
  constexpr long FEW = 384, MANY = 2048, SMS = 152;
  long rows = (long)c.max_pages * c.page;
  if (c.window > 0) rows = std::min(rows, (long)c.window + c.sinks + 2 * PA_TILE);
  return rows <= ((long)c.B * c.KV < SMS ? FEW : MANY);
}

// CTAs: two an SM, or a unit each.
int pa_grid(const Paged& c) {
  const long rows = std::min<long>((long)c.max_pages * c.page, 0x7fffffffL);
  const long units = (rows + PA_UNIT - 1) / PA_UNIT * c.B * c.KV;
  return (int)std::min<long>(PA_CTAS, units);
}

template <int DH>
cudaError_t pa_launch(const PaArgs& a, bool split, cudaStream_t st) {
  static KernelOnce once;
  cudaError_t e = once(reinterpret_cast<const void*>(paged_attn_kernel<DH>), PaCfg<DH>::SMEM);
  if (e != cudaSuccess) return e;
  const double rows = (double)a.B * a.KV * std::min<long>((long)a.max_pages * a.page, 0x7fffffffL);
  {
    // work: upper bound (every cache full)
    LaunchTimer lt("paged_attn", st, 4.0 * rows * a.g * DH, 4.0 * rows * DH);
    e = launch_kernel(paged_attn_kernel<DH>, a.G, PA_THREADS, PaCfg<DH>::SMEM, st, a);
    if (e != cudaSuccess || !split) return e;
  }
  LaunchTimer lt("paged_join", st, 0.0, 8.0 * a.G * a.g * (DH + 2));
  // about 1200 CTAs, or as many as there are columns for
  const long pairs = (long)a.B * a.KV;
  const int x = (int)std::min<long>(pairs, a.G), y = std::min(a.g * (DH / 32), (8 * 152 + x - 1) / x);
  return launch_kernel(paged_join_kernel<DH>, dim3(x, y), PJ_THREADS, 0, st, a);
}

}  // namespace

static_assert(PA_MAX_B == PF_PAGED_MAX_BATCH && PA_TILE == PF_PAGED_ROWS, "limits of the entry points");

size_t paged_attn_ws_bytes(const Paged& c) {
  return 2 * (size_t)pa_grid(c) * (c.H / c.KV) * (c.dh + 2) * sizeof(float);
}

cudaError_t paged_attn(const Paged& c, const bf16* q, long ldq, bf16* out, long ldo, float* ws,
                       cudaStream_t st) {
  launched.mark();
  PaArgs a{};
  a.q = q;
  a.ldq = ldq;
  a.K = c.K; a.V = c.V;
  a.table = c.table; a.len = c.len;
  a.out = out;
  a.ldo = ldo;
  a.part = ws;
  a.B = c.B; a.KV = c.KV; a.g = c.H / c.KV; a.page = c.page; a.max_pages = c.max_pages;
  a.window = c.window; a.sinks = c.sinks;
  a.n_pages = c.n_pages;
  a.whole = pa_whole(c);
  a.G = a.whole ? c.B * c.KV : pa_grid(c);
  a.sl2 = 1.4426950408889634f / sqrtf((float)c.dh);
  const bool split = !a.whole && (long)c.max_pages * c.page > PA_UNIT;  // else no pair has two units
  return c.dh == 128 ? pa_launch<128>(a, split, st) : pa_launch<64>(a, split, st);
}

}  // namespace pf

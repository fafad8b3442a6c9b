// Rows of a paged cache read back: the last start[b + 1] - start[b] rows of every sequence b as
// matrices of keys and values [rows, KV * dh] in bf16, in the order of the call's rows.  A
// quantised row's values x 2^e (paged_q8.cuh) are bf16 numbers, so that nothing is rounded.
//
// A copy: HBM traffic bounds it.  A CTA takes a few rows: a thread to each looks up where it
// lies, then all of them copy, 16 bytes of the pool a piece.
#include <algorithm>

#include "local.h"
#include "paged_q8.cuh"

namespace pf {

static Launched launched;
int take_dev_error_paged_read() { return launched.take(take_dev_error_tu); }
int set_wait_limit_paged_read(unsigned long long ns) { return set_wait_limit_tu(ns); }

namespace {

constexpr int PR_THREADS = 256;
constexpr int PR_ROWS = 32;  // of a CTA at most

struct PrArgs {
  const void *K, *V;
  const signed char *Ke, *Ve;
  const int *table, *len, *start;
  bf16 *k, *v;
  long ldk, ldv, rows, n_pages;
  int B, KV, page, max_pages, per;  // per: rows of a CTA
};

template <int DH, bool Q8>
__global__ void __launch_bounds__(PR_THREADS) paged_read_kernel(PrArgs a) {
  __shared__ long at[PR_ROWS];  // a row's place in the pool (of its first head); -1: zeros; -2: no sequence's
  pdl_enter();
  const long r0 = (long)blockIdx.x * a.per;
  const int n = (int)min((long)a.per, a.rows - r0), tid = threadIdx.x;
  if (tid < n) {
    const long i = r0 + tid;
    int b = (int)min(i, (long)a.B - 1);
    long p = -2;
    if (a.start) {  // the last sequence that begins at or before it (of those that begin there, the last)
      int hi = a.B;
      b = 0;
      while (hi - b > 1) {
        const int m = (b + hi) >> 1;
        if (a.start[m] <= i) b = m; else hi = m;
      }
    }
    const int t0 = a.start ? a.start[b] : (int)i, t1 = a.start ? a.start[b + 1] : (int)i + 1;
    if (i < a.B || a.start) {
      if (t0 <= i && i < t1) {
        const int len = a.len[b];
        const long r = len - (t1 - i);
        p = -1;
        if (r >= 0 && len <= (long)a.max_pages * a.page) {
          const int pg = a.table[(long)b * a.max_pages + r / a.page];
          if (pg >= 0 && pg < a.n_pages) p = (long)pg * a.KV * a.page + r % a.page;
        }
        if (p < 0) set_dev_error(DEVERR_CAPACITY);
      }
    }
    at[tid] = p;
  }
  __syncthreads();
  constexpr int PIECES = DH / (Q8 ? 16 : 8), U = 4;  // 16-byte pieces of a row and head; pieces in flight
  const int per = a.KV * PIECES, all = n * per;
#pragma unroll 1
  for (int e0 = tid; e0 < all; e0 += U * PR_THREADS) {
    uint4 u[2][U];
    float f[2][U];
    long p[U];
    int r[U], c[U], h[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int e = e0 + i * PR_THREADS;
      r[i] = e / per;
      const int x = e - r[i] * per;
      h[i] = x / PIECES;
      c[i] = x % PIECES;
      p[i] = e < all ? at[r[i]] : -2;
      u[0][i] = u[1][i] = make_uint4(0, 0, 0, 0);
      f[0][i] = f[1][i] = 0.f;
      if (p[i] >= 0) {
        const long q = p[i] + (long)h[i] * a.page;
        u[0][i] = static_cast<const uint4*>(a.K)[q * PIECES + c[i]];
        u[1][i] = static_cast<const uint4*>(a.V)[q * PIECES + c[i]];
        if (Q8) {
          f[0][i] = pq_scale(a.Ke[q]);
          f[1][i] = pq_scale(a.Ve[q]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (p[i] == -2) continue;
      bf16* const ko = a.k + (r0 + r[i]) * a.ldk + h[i] * DH + c[i] * (DH / PIECES);
      bf16* const vo = a.v + (r0 + r[i]) * a.ldv + h[i] * DH + c[i] * (DH / PIECES);
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        uint4* const o = reinterpret_cast<uint4*>(kv ? vo : ko);
        const uint4 x = u[kv][i];
        if (Q8) {
          const float s = pq_shift(f[kv][i]);
          const float2 ff = make_float2(f[kv][i], f[kv][i]), ss = make_float2(s, s);
          const uint2 v0 = pq_values(x.x, ff, ss), v1 = pq_values(x.y, ff, ss), v2 = pq_values(x.z, ff, ss),
                      v3 = pq_values(x.w, ff, ss);
          o[0] = make_uint4(v0.x, v0.y, v1.x, v1.y);
          o[1] = make_uint4(v2.x, v2.y, v3.x, v3.y);
        } else {
          o[0] = x;
        }
      }
    }
  }
}

}  // namespace

cudaError_t paged_read(const Paged& c, long rows, const int* start, bf16* k, long ldk, bf16* v, long ldv,
                       cudaStream_t st) {
  launched.mark();
  PrArgs a{};
  a.K = c.K; a.V = c.V; a.Ke = c.Ke; a.Ve = c.Ve;
  a.table = c.table; a.len = c.len; a.start = start;
  a.k = k; a.v = v;
  a.ldk = ldk; a.ldv = ldv;
  a.rows = rows;
  a.n_pages = c.n_pages;
  a.B = c.B; a.KV = c.KV; a.page = c.page; a.max_pages = c.max_pages;
  const long pieces = (long)c.KV * c.dh / (c.Ke ? 16 : 8);
  a.per = (int)std::min<long>(PR_ROWS, std::max<long>(1, 4 * PR_THREADS / pieces));
  LaunchTimer lt("paged_read", st, 0.0, (double)rows * c.KV * c.dh * (c.Ke ? 6.0 : 8.0));
  const int grid = (int)((rows + a.per - 1) / a.per);
  auto kern = c.Ke ? (c.dh == 64 ? paged_read_kernel<64, true> : paged_read_kernel<128, true>)
                   : (c.dh == 64 ? paged_read_kernel<64, false> : paged_read_kernel<128, false>);
  return launch_kernel(kern, grid, PR_THREADS, 0, st, a);
}

}  // namespace pf

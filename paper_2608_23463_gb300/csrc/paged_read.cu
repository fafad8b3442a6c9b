// Rows of a paged cache read back: the last start[b + 1] - start[b] rows of every sequence b as
// matrices of keys and values [rows, KV * dh] in bf16, in the order of the call's rows.  A
// quantised row's values x 2^e (paged_q8.cuh) are bf16 numbers, so that nothing is rounded.
//
// A copy: HBM traffic bounds it.  A CTA takes a few rows: a thread to each looks up where it
// lies, then all of them copy, 8 values of K and of V a turn.  Few registers and many warps carry
// it: 76925 rows of 16 quantised heads of 128, 154 us (6.2 TB/s) so, with two pieces in flight a
// thread 171, with four 193, with eight 299.
#include <algorithm>

#include "local.h"
#include "paged_q8.cuh"

namespace pf {

static Launched launched;
int take_dev_error_paged_read() { return launched.take(take_dev_error_tu); }
int set_wait_limit_paged_read(unsigned long long ns) { return set_wait_limit_tu(ns); }

namespace {

constexpr int PR_THREADS = 256;
constexpr int PR_TURNS = 8;  // pieces of a thread, about
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
  constexpr int PIECES = DH / 8;  // pieces of 8 values of a row and head
  const int per = a.KV * PIECES, all = n * per;
#pragma unroll 1
  for (int e = tid; e < all; e += PR_THREADS) {
    const int r = e / per, c = e - r * per;
    const long p = at[r];
    if (p == -2) continue;
    uint4 u[2];
    u[0] = u[1] = make_uint4(0, 0, 0, 0);
    if (p >= 0) {
      const long q = p + (long)(c / PIECES) * a.page, x = q * PIECES + c % PIECES;
      if (Q8) {
        const uint2 k = static_cast<const uint2*>(a.K)[x], v = static_cast<const uint2*>(a.V)[x];
        const float f[2] = {pq_scale(a.Ke[q]), pq_scale(a.Ve[q])};
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const float2 ff = make_float2(f[kv], f[kv]), ss = make_float2(pq_shift(f[kv]), pq_shift(f[kv]));
          const uint2 lo = pq_values(kv ? v.x : k.x, ff, ss), hi = pq_values(kv ? v.y : k.y, ff, ss);
          u[kv] = make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
      } else {
        u[0] = static_cast<const uint4*>(a.K)[x];
        u[1] = static_cast<const uint4*>(a.V)[x];
      }
    }
    *reinterpret_cast<uint4*>(a.k + (r0 + r) * a.ldk + c * 8) = u[0];
    *reinterpret_cast<uint4*>(a.v + (r0 + r) * a.ldv + c * 8) = u[1];
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
  const long pieces = (long)c.KV * c.dh / 8;
  // few rows: of less than PR_TURNS, down to one, so that they reach more SMs (one row of each of 8 sequences,
  // 16 quantised heads of 128: 2.1 us, 4.6 in one CTA)
  const long turns = std::min<long>(PR_TURNS, std::max<long>(1, rows * pieces / (2 * 152 * PR_THREADS)));
  a.per = (int)std::min<long>(PR_ROWS, std::max<long>(1, turns * PR_THREADS / pieces));
  LaunchTimer lt("paged_read", st, 0.0, (double)rows * c.KV * c.dh * (c.Ke ? 6.0 : 8.0));
  const int grid = (int)((rows + a.per - 1) / a.per);
  auto kern = c.Ke ? (c.dh == 64 ? paged_read_kernel<64, true> : paged_read_kernel<128, true>)
                   : (c.dh == 64 ? paged_read_kernel<64, false> : paged_read_kernel<128, false>);
  return launch_kernel(kern, grid, PR_THREADS, 0, st, a);
}

}  // namespace pf

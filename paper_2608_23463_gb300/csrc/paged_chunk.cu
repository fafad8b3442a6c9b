// Attention of the newest tokens of every sequence, any number of each, over a paged cache of
// keys and values on the 5th-generation tensor cores: tcgen05.mma with TMEM accumulators, TMA
// tiles, grouped heads, head width 64 or 128, cache in bf16 or quantised (paged_q8.cuh).
//
//   o_h = sum_j softmax_j(q_h . K_j / sqrt(dh)) V_j  over the rows j <= i of the sequence,
//   i the token's own row, with a window W also j > i - W or j < S (the sinks)
//
// paged_items.cuh cuts the work into items and deals their steps to the CTAs, one per SM.  A
// step is 128 rows of the cache against both query tiles of an item, 128 rows each of tokens
// times the query heads of one key head.
//   warp 0     TMA producer: an item's query tiles, and rings of K and V tiles; a tile is
//              fetched in boxes of the largest power of two of rows that divides a page, each
//              by the lane that looked its page up; blocks that no token of the item sees are
//              asked past the pool's end, which reads as zero
//   warp 1     MMA issuer of both tiles' scores: S = Q K^T (M=128, N=128)
//   warps 2-3  MMA issuers of tile A's and tile B's O += P V (M=128, N=dh, K=128), P from TMEM
//   warps 4-7  softmax of tile A, warps 8-11 of tile B: one row per thread (TMEM lane); the
//              running maximum moves by more than 2^8 only, which then scales O
//   warps 12-15 (quantised caches) fetch nothing: they turn the producer's raw tiles of bytes
//              into the bf16 tiles that the MMAs read
// TMEM holds both tiles' S and O; with dh = 128 P takes the place of S, from which it came.
// An item that one CTA holds whole is written; pieces leave (O, maximum, sum) and
// paged_chunk_join_kernel joins them in the order of the CTAs: results repeat bit for bit.
// P is rounded to bf16 (2^-9) for its product, its sum taken before that.
#include <algorithm>
#include <type_traits>

#include "local.h"
#include "paged_items.cuh"
#include "paged_q8.cuh"

namespace pf {

static Launched launched;
int take_dev_error_paged_chunk() { return launched.take(take_dev_error_tu); }
int set_wait_limit_paged_chunk(unsigned long long ns) { return set_wait_limit_tu(ns); }

namespace {

constexpr int PC_CTAS = 152;  // one an SM, whatever the device has: splits keep their places
constexpr int PC_MAX_B = 2048;
constexpr long PC_LONGEST = 0x7fffff00;  // rows of a sequence: indices of their tiles fit 32 bits
constexpr float PC_RESCALE = 8.f;

template <int DH, bool Q8>
struct PcCfg {
  static constexpr int THREADS = Q8 ? 512 : 384;
  // registers of a control (and converting) and of a softmax thread, of the pool at launch
  static constexpr int REGS_CTRL = Q8 ? 56 : 88, REGS_ROWS = Q8 ? 200 : 208;
  static constexpr int POOL = REGS_CTRL * (THREADS - 256) + REGS_ROWS * 256;
  static_assert(POOL <= (65536 / THREADS / 8 * 8) * THREADS, "register split");
  static constexpr int HALVES = DH / 64;
  static constexpr uint32_t HALF = PC_T * 128;  // 64 columns of a tile
  static constexpr uint32_t TILE = HALVES * HALF;
  static constexpr int NK = DH == 64 ? 4 : 2, NV = DH == 64 ? 4 : (Q8 ? 2 : 3);  // stages
  static constexpr uint32_t RAW = PC_T * DH;  // a tile of bytes
  static constexpr int NR = Q8 ? (DH == 64 ? 4 : 2) : 0;  // stages of them
  static constexpr uint32_t OFF_K = 2 * TILE, OFF_V = OFF_K + NK * TILE, OFF_RAW = OFF_V + NV * TILE;
  static constexpr uint32_t OFF_EXP = OFF_RAW + NR * RAW, OFF_BAR = OFF_EXP + NR * PC_T;
  static constexpr uint32_t SMEM = OFF_BAR + 512 + 1024;
  static_assert(SMEM <= 227 * 1024, "shared memory");
  static_assert((PC_MAX_B + 1) * 8 <= (NK + NV) * TILE, "the sequences' totals lie in the rings at first");
  // TMEM columns of tile w: S at 128 w, O and P
  static constexpr bool ALIAS = DH == 128;
  __host__ __device__ static constexpr uint32_t tm_o(int w) { return 256 + DH * w; }
  __host__ __device__ static constexpr uint32_t tm_p(int w) { return ALIAS ? 128 * w : 384 + 64 * w; }
};

struct PcArgs {
  PcGeo geo;
  const int *start, *len, *table;
  long rows;
  int page, max_pages, box;  // box: rows of a TMA box
  long n_pages;
  int G;           // CTAs
  int whole, few;  // items to a CTA from which none is cut (whole: none ever); steps' weight to a CTA at least
  float sl2;       // log2(e) / sqrt(dh)
  const bf16* q;
  bf16* out;
  long ldq, ldo;
  const void *K, *V;
  const signed char *Ke, *Ve;
  // pieces: where each CTA begins [G + 1], (maximum, sum) and O of the rows [2 G][rows of an item]
  PcAt* at;
  float2* ml;
  float* part;
  int piece_rows;
};

__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// mbar_wait_warp with the common case, a phase that has completed, up front.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity) {
  if (__all_sync(0xffffffffu, mbar_test_wait(bar, parity))) return true;
  return mbar_wait_warp(bar, parity);
}

// Sequence b: no tokens where its part of the call or its length cannot be.
__device__ __forceinline__ PcSeq pc_seq(const PcArgs& a, int b, bool* bad = nullptr) {
  PcSeq s;
  s.t0 = a.start[b];
  const int t1 = a.start[b + 1];
  s.n = t1 - s.t0;
  s.len = a.len[b];
  const bool rows = s.t0 >= 0 && t1 >= s.t0 && t1 <= a.rows;
  const bool ok = rows && s.len >= s.n && s.len <= min((long)a.max_pages * a.page, PC_LONGEST);
  if (bad) *bad = !ok;
  if (!ok) s.n = rows && bad ? s.n : 0;  // (asked for: rows to be zeroed)
  return s;
}

// The items from one place in the line to another.
struct PcWalk {
  PcAt at, end;
  PcSeq q;
  int pairs;
  __device__ __forceinline__ PcWalk(const PcArgs& a, const PcAt* ends) : at(ends[0]), end(ends[1]) {
    if (at.b < a.geo.B) load(a);
  }
  __device__ __forceinline__ void load(const PcArgs& a) {
    q = pc_seq(a, at.b);
    pairs = pc_pairs(a.geo, q);
  }
  __device__ __forceinline__ bool same() const { return at.b == end.b && at.h == end.h && at.u == end.u; }
  __device__ __forceinline__ bool more(const PcArgs& a) const {
    return at.b < a.geo.B && (!same() || at.s < end.s);
  }
  __device__ __forceinline__ void next(const PcArgs& a) {
    at.s = 0;
    if (same()) at.s = end.s;  // (a piece that ends there)
    else if (++at.u == pairs) {
      at.u = 0;
      if (++at.h == a.geo.KV) {
        at.h = 0;
        do {
          if (++at.b >= a.geo.B) return;
          load(a);
        } while (q.n == 0);
      }
    }
  }
};

// A piece of an item: its steps [s0, s1).
struct PcItem {
  PcSpan sp;
  int h, t0, toks, s0, s1;
  bool two, whole;  // with a tile B; all of its steps
  __device__ __forceinline__ PcItem(const PcArgs& a, const PcWalk& w) {
    sp = pc_span(a.geo, w.q, w.at.u);
    h = w.at.h;
    const int R = 2 * a.geo.tpt;
    t0 = w.q.t0 + w.at.u * R;
    toks = min(w.q.n - w.at.u * R, R);
    two = toks > a.geo.tpt;
    s0 = w.at.s;
    s1 = w.same() ? w.end.s : sp.steps;
    whole = s0 == 0 && s1 == sp.steps;
  }
};

// Page of row r of a sequence, or -1.
__device__ __forceinline__ long pc_page(const PcArgs& a, int b, int r) {
  const int pg = a.table[(long)b * a.max_pages + r / a.page];
  if (pg >= 0 && pg < a.n_pages) return pg;
  set_dev_error(DEVERR_CAPACITY);
  return -1;
}

// N values of row r (of the pool) from column c on.
template <int DH, bool Q8, int N>
__device__ __forceinline__ void pc_load(const void* pool, const signed char* ex, long r, int c, float* v) {
  if (Q8) {
    const float f = pq_scale(ex[r]), sh = pq_shift(f);
    const signed char* p = static_cast<const signed char*>(pool) + r * DH + c;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = fmaf((float)(p[i] + 128) + 8388608.f, f, sh);
  } else {
    const bf16* p = static_cast<const bf16*>(pool) + r * DH + c;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 x = unpack_bf16(*reinterpret_cast<const uint32_t*>(p + i));
      v[i] = x.x;
      v[i + 1] = x.y;
    }
  }
}

// Whether one of the rows [r0, r1) of V of a head holds a value that is not finite.  For a
// converged warp.
template <int DH, bool Q8>
__device__ __forceinline__ bool pc_not_finite(const PcArgs& a, int b, int h, int r0, int r1) {
  const int lane = threadIdx.x & 31;
  bool bad = false;
  for (int r = r0 + lane; r < r1; r += 32) {
    const long pg = pc_page(a, b, r);
    if (pg < 0) continue;
    const long at = (pg * a.geo.KV + h) * a.page + r % a.page;
    if (Q8) {
      bad |= a.Ve[at] == PQ_NAN;
    } else {
      const uint4* p = reinterpret_cast<const uint4*>(static_cast<const bf16*>(a.V) + at * DH);
#pragma unroll 1
      for (int i = 0; i < DH / 8; ++i) {
        const uint4 u = p[i];
        for (uint32_t w : {u.x, u.y, u.z, u.w}) bad |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
      }
    }
  }
  return __any_sync(0xffffffffu, bad);
}

// A row whose sums are not finite, though what spoilt them may be values that it does not see: in
// the MMA P = 0 met them.  Token t of the call (row i of sequence b), query head hq of key head h:
// where the blocks fetched for it (of the item with positions [pf, pl]) hold hidden rows of V that
// are not finite, it is worked out again from the rows that it sees.  For a converged warp: a
// key to a lane for the scores, columns for the sums.  Out of line: calls without such rows have
// none of its registers.
template <int DH, bool Q8>
__device__ __noinline__ void pc_repair(const PcArgs& a, int b, int h, int hq, int t, int i, int pf, int pl) {
  const int lane = threadIdx.x & 31, W = a.geo.W, bx = a.box;
  const int lo = W > 0 && i >= W ? i - W + 1 : 0, S = min(a.geo.S, lo);
  const int first = W > 0 && pf >= W ? (pf - W + 1) / bx * bx : 0;
  const int held = (int)min(min(((long)a.geo.S + bx - 1) / bx * bx, (long)lo), (long)(pf - pf % bx));
  if (!pc_not_finite<DH, Q8>(a, b, h, i + 1, (pl / bx + 1) * bx) &&
      !(W > 0 && (pc_not_finite<DH, Q8>(a, b, h, max(first, S), lo) || pc_not_finite<DH, Q8>(a, b, h, S, held))))
    return;
  constexpr int C = DH / 32;  // columns of a lane
  const bf16* q = a.q + t * a.ldq + (long)hq * DH;
  float acc[C] = {}, m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {  // the sinks before the window, the window
    const int end = part ? i + 1 : S;
#pragma unroll 1
    for (int j = part ? lo : 0; j < end; j += 32) {
      const bool in = j + lane < end;
      const long pg = in ? pc_page(a, b, j + lane) : -1;
      const long at = pg < 0 ? -1 : (pg * a.geo.KV + h) * a.page + (j + lane) % a.page;
      float s = 0.f;  // (a page out of range reads as zero)
      if (at >= 0) {
#pragma unroll 1
        for (int c = 0; c < DH; c += 8) {
          float x[8], y[8];
          load8_bf16(q + c, x);
          pc_load<DH, Q8, 8>(a.K, a.Ke, at, c, y);
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
        }
      }
      if (!in) s = -INFINITY;
      float mx = s;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float next = fmaxf(m, mx * a.sl2), ref = next == -INFINITY ? 0.f : next;
      const float corr = m == -INFINITY ? 1.f : ex2_approx(m - ref);
      m = next;
      const float p = in ? ex2_approx(fmaf(s, a.sl2, -ref)) : 0.f;
      float sum = p;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      l = fmaf(l, corr, sum);
      bool nan = true;
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c] *= corr;
#pragma unroll 1
      for (int k = 0; k < min(32, end - j); ++k) {
        const float pk = __shfl_sync(0xffffffffu, p, k);
        const long ak = __shfl_sync(0xffffffffu, at, k);
        if (ak < 0) continue;
        float y[C];
        pc_load<DH, Q8, C>(a.V, a.Ve, ak, C * lane, y);
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] = fmaf(pk, y[c], acc[c]);
      }
#pragma unroll
      for (int c = 0; c < C; ++c) nan &= acc[c] != acc[c];
      if (__all_sync(0xffffffffu, nan)) part = 2;  // for good, whatever follows
      if (part == 2) break;
    }
  }
  bf16* o = a.out + t * a.ldo + (long)hq * DH + C * lane;
#pragma unroll
  for (int c = 0; c < C; c += 2)
    *reinterpret_cast<uint32_t*>(o + c) = pack_bf16(acc[c] / l, acc[c + 1] / l);
}

// The CTA's part of the line, ends[0] to ends[1], and its share in the pieces' index.  pre: room
// for B + 1 totals.  Whole CTAs call it.
template <int THREADS>
__device__ __forceinline__ void pc_share_out(const PcArgs& a, long long* pre, PcAt* ends) {
  __shared__ long long wsum[THREADS / 32], total;
  __shared__ unsigned long long items;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) items = 0;
  __syncthreads();
  long long base = 0;
  for (int b0 = 0; b0 < a.geo.B; b0 += THREADS) {
    const int b = b0 + tid;
    long long u = 0;
    if (b < a.geo.B) {
      bool bad;
      PcSeq q = pc_seq(a, b, &bad);
      if (bad) {
        set_dev_error(DEVERR_CAPACITY);
      } else if (q.n > 0) {
        const int P = pc_pairs(a.geo, q);
        u = a.geo.KV * pc_cum(a.geo, q, P);
        atomicAdd(&items, (unsigned long long)P * a.geo.KV);
      }
    }
    long long v = u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long t = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += t;
    }
    if (lane == 31) wsum[warp] = v;
    __syncthreads();
    long long before = 0, all = 0;
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) before += wsum[w];
      all += wsum[w];
    }
    if (b < a.geo.B) pre[b] = base + before + v - u;
    base += all;
    __syncthreads();
  }
  if (tid == 0) {
    pre[a.geo.B] = base;
    total = base;
  }
  __syncthreads();
  if (warp < 2 && lane == 0) {
    const long long T = total;
    const bool whole = a.whole == 0 || items >= (unsigned long long)a.whole * a.G;
    const int n = whole ? a.G : (int)max(1ll, min((long long)a.G, T / a.few));
    const int c = min((int)blockIdx.x + warp, n);
    PcAt r{a.geo.B, 0, 0, 0};
    const long long x = pc_share(T, n, c);
    if (x < T) {
      int b = 0, hi = a.geo.B;
      while (hi - b > 1) {
        const int m = (b + hi) >> 1;
        if (pre[m] <= x) b = m; else hi = m;
      }
      // (the last of those that begin at x: it has tokens)
      const PcSeq q = pc_seq(a, b);
      const int P = pc_pairs(a.geo, q);
      const long long per = pc_cum(a.geo, q, P), y = x - pre[b];
      r.b = b;
      r.h = (int)(y / per);
      pc_find(a.geo, q, y % per, whole, &r.u, &r.s);
      if (r.s >= pc_span(a.geo, q, r.u).steps) {  // the next item's beginning
        r.s = 0;
        if (++r.u == P) {
          r.u = 0;
          if (++r.h == a.geo.KV) {
            r.h = 0;
            do ++r.b;
            while (r.b < a.geo.B && pre[r.b + 1] == pre[r.b]);
          }
        }
      }
    }
    ends[warp] = r;
    if (a.at && (warp == 0 || c == a.G)) a.at[c] = r;
    // (n < G: the CTAs from n on write the line's end, each its own)
    if (a.at && warp == 0 && (int)blockIdx.x > n) a.at[blockIdx.x] = r;
    if (a.at && warp == 1 && (int)blockIdx.x + 1 == a.G) a.at[a.G] = r;
  }
  __syncthreads();
}

template <int DH, bool Q8>
__global__ void __launch_bounds__(PcCfg<DH, Q8>::THREADS, 1)
    paged_chunk_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PcArgs a) {
  using C = PcCfg<DH, Q8>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ PcAt ends[2];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  const uint32_t sbase = smem_u32(smem), b0 = sbase + C::OFF_BAR;
  const uint32_t q_full = b0, q_empty = b0 + 8, done = b0 + 16, grp0 = b0 + 24, ring0 = grp0 + 2 * 48;
  auto s_full = [&](int w) { return grp0 + 48 * w; };
  auto s_free = [&](int w) { return grp0 + 48 * w + 8; };
  auto p_full = [&](int w) { return grp0 + 48 * w + 16; };
  auto p_free = [&](int w) { return grp0 + 48 * w + 24; };
  auto o_full = [&](int w) { return grp0 + 48 * w + 32; };
  auto o_free = [&](int w) { return grp0 + 48 * w + 40; };
  auto k_full = [&](int i) { return ring0 + 8 * i; };
  auto k_empty = [&](int i) { return ring0 + 8 * (C::NK + i); };
  auto v_full = [&](int i) { return ring0 + 8 * (2 * C::NK + i); };
  auto v_empty = [&](int i) { return ring0 + 8 * (2 * C::NK + C::NV + i); };
  auto r_full = [&](int i) { return ring0 + 8 * (2 * C::NK + 2 * C::NV + i); };
  auto r_empty = [&](int i) { return ring0 + 8 * (2 * C::NK + 2 * C::NV + C::NR + i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_BAR + 504);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    mbar_init(q_full, 1);
    mbar_init(q_empty, 8);  // one arrival per softmax warp
    mbar_init(done, 3);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full(i), 1);
      mbar_init(s_free(i), 4);
      mbar_init(p_full(i), 4);
      mbar_init(p_free(i), 1);
      mbar_init(o_full(i), 1);
      mbar_init(o_free(i), 4);
    }
    for (int i = 0; i < C::NK; ++i) {
      mbar_init(k_full(i), Q8 ? 4 : 1);  // (converting warps)
      mbar_init(k_empty(i), 1);
    }
    for (int i = 0; i < C::NV; ++i) {
      mbar_init(v_full(i), Q8 ? 4 : 1);
      mbar_init(v_empty(i), 2);  // one arrival per tile
    }
    for (int i = 0; i < C::NR; ++i) {
      mbar_init(r_full(i), 1);
      mbar_init(r_empty(i), 4);
    }
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_enter();  // the setup above overlaps the kernel before this one
  pc_share_out<C::THREADS>(a, reinterpret_cast<long long*>(smem + C::OFF_K), ends);
  // rows of sequences whose length cannot be
  for (int b = blockIdx.x; b < a.geo.B; b += gridDim.x) {
    bool bad;
    const PcSeq q = pc_seq(a, b, &bad);
    const int per = a.geo.KV * a.geo.g * (DH / 8);
    if (bad)
      for (long i = threadIdx.x; i < (long)q.n * per; i += C::THREADS)
        *reinterpret_cast<uint4*>(a.out + (q.t0 + i / per) * a.ldo + i % per * 8) = make_uint4(0, 0, 0, 0);
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the totals lay where the rings are
  __syncthreads();
  uint32_t k_issued = 0, v_issued = 0, r_issued = 0, q_issued = 0;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_CTRL));
    if (warp == 0) {
      // ------------------------------------------------------------ producer (all lanes)
      if (lane == 0) {
        prefetch_tmap(&tmQ);
        prefetch_tmap(&tmK);
        prefetch_tmap(&tmV);
      }
      const int nb = PC_T / a.box, H = Q8 ? 1 : C::HALVES;
      // lane: block of rows and half of their columns, or (Q8) the blocks' exponents
      const int blk = lane / H % nb, half = lane % H;
      const bool data = lane < nb * H, exps = Q8 && lane >= nb && lane < 2 * nb;
      const uint32_t qbytes = (uint32_t)(a.geo.tpt * a.geo.g * 128 * C::HALVES);
      bool ok = true;
      for (PcWalk w(a, ends); w.more(a) && ok; w.next(a)) {
        const PcItem m(a, w);
        auto page_of = [&](int s) -> int {  // the pool's page of the lane's block in step s
          if (s >= m.s1 || !(data || exps)) return 0;
          const int r = m.sp.tile(s) * PC_T + blk * a.box;
          const bool seen = r <= m.sp.pl && (a.geo.W == 0 || r + a.box - 1 > m.sp.pf - a.geo.W || r < a.geo.S);
          const long pg = seen ? pc_page(a, w.at.b, r) : -1;
          return (int)(pg < 0 ? a.n_pages : pg);  // (past the end: zeros)
        };
        if (!wait_warp(q_empty, (q_issued & 1) ^ 1)) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(q_full, m.two ? 2 * qbytes : qbytes);
          for (int t = 0; t < (m.two ? 2 : 1); ++t)
            for (int c = 0; c < C::HALVES; ++c)
              tma_load_3d(sbase + t * C::TILE + c * C::HALF, &tmQ, q_full, 64 * c, m.h * a.geo.g,
                          m.t0 + t * a.geo.tpt);
        }
        __syncwarp();
        ++q_issued;
        int pg_next = page_of(m.s0);
        for (int s = m.s0; s < m.s1; ++s) {
          const int pg = pg_next, row = (m.sp.tile(s) * PC_T + blk * a.box) % a.page;
          pg_next = page_of(s + 1);
          if (Q8) {
            for (int kv = 0; kv < 2; ++kv) {
              const uint32_t st = r_issued % (C::NR ? C::NR : 1);
              if (!wait_warp(r_empty(st), ((r_issued / (C::NR ? C::NR : 1)) & 1) ^ 1)) {
                ok = false;
                break;
              }
              // (exponents of blocks that no token sees, and of pages out of range: zeros)
              const bool in = exps && pg < a.n_pages;
              const uint32_t edst = sbase + C::OFF_EXP + st * PC_T + blk * a.box;
              if (exps && !in)
                for (int i = 0; i < a.box; i += 16)
                  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(edst + i), "r"(0) : "memory");
              const uint32_t ebytes = a.box * __popc(__ballot_sync(0xffffffffu, in));
              if (lane == 0) mbar_arrive_expect_tx(r_full(st), C::RAW + ebytes);
              __syncwarp();
              if (data)
                tma_load_4d(sbase + C::OFF_RAW + st * C::RAW + blk * a.box * DH, kv ? &tmV : &tmK, r_full(st), 0, row,
                            m.h, pg);
              else if (in)
                bulk_load(edst, (kv ? a.Ve : a.Ke) + ((long)pg * a.geo.KV + m.h) * a.page + row, a.box, r_full(st));
              __syncwarp();
              ++r_issued;
            }
            if (!ok) break;
          } else {
            const uint32_t sk = k_issued % C::NK, sv = v_issued % C::NV;
            const uint32_t off = half * C::HALF + blk * a.box * 128;
            if (!wait_warp(k_empty(sk), ((k_issued / C::NK) & 1) ^ 1)) {
              ok = false;
              break;
            }
            if (lane == 0) mbar_arrive_expect_tx(k_full(sk), C::TILE);
            __syncwarp();
            if (data) tma_load_4d(sbase + C::OFF_K + sk * C::TILE + off, &tmK, k_full(sk), 64 * half, row, m.h, pg);
            __syncwarp();
            ++k_issued;
            if (!wait_warp(v_empty(sv), ((v_issued / C::NV) & 1) ^ 1)) {
              ok = false;
              break;
            }
            if (lane == 0) mbar_arrive_expect_tx(v_full(sv), C::TILE);
            __syncwarp();
            if (data) tma_load_4d(sbase + C::OFF_V + sv * C::TILE + off, &tmV, v_full(sv), 64 * half, row, m.h, pg);
            __syncwarp();
            ++v_issued;
          }
        }
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------ MMA issuer: scores
      // The whole warp runs the loop; one elected lane issues and commits.
      constexpr uint32_t idesc = idesc_bf16_f32(PC_T, PC_T, 0, 0);
      const uint64_t dq0 = smem_desc_sw128(sbase, 16, 1024), dk0 = smem_desc_sw128(sbase + C::OFF_K, 16, 1024);
      uint32_t G = 0, gs[2] = {0, 0}, it = 0;  // steps, products of the tiles, items so far
      for (PcWalk wk(a, ends); wk.more(a); wk.next(a), ++it) {
        const PcItem m(a, wk);
        if (!wait_warp(q_full, it & 1)) break;
        int s = m.s0;
        for (; s < m.s1; ++s, ++G) {
          const uint32_t st = G % C::NK;
          if (!wait_warp(k_full(st), (G / C::NK) & 1)) break;
          bool ok = true;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            if (!ok || (w == 1 && !m.two)) continue;
            // S's place: read into registers, or (ALIAS) P in it taken up by its product
            if (gs[w] > 0 && !wait_warp(C::ALIAS ? p_free(w) : s_free(w), (gs[w] - 1) & 1)) {
              ok = false;
              continue;
            }
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int kk = 0; kk < DH / 16; ++kk) {
                const uint64_t o = (uint64_t)(kk / 4) * (C::HALF >> 4) + kk % 4 * 2;
                tc_mma_f16(tmem + 128 * w, dq0 + w * (C::TILE >> 4) + o, dk0 + st * (C::TILE >> 4) + o, idesc,
                           kk ? 1u : 0u);
              }
              tc_commit(s_full(w));
            }
            __syncwarp();
            ++gs[w];
          }
          if (!ok) break;
          if (elect_one()) tc_commit(k_empty(st));
          __syncwarp();
        }
        if (s < m.s1) break;  // a wait ran out
      }
      if (elect_one()) tc_commit(done);
      __syncwarp();
    } else {
      // ------------------------------------------------------------ MMA issuers: O of tiles A, B
      const int w = warp - 2;
      constexpr uint32_t idesc = idesc_bf16_f32(PC_T, DH, 0, 1);
      const uint32_t tO = tmem + C::tm_o(w), tP = tmem + C::tm_p(w);
      const uint64_t dv0 = smem_desc_sw128(sbase + C::OFF_V, C::HALF, 1024);
      uint32_t G = 0, gp = 0, io = 0;  // steps, products, items so far
      for (PcWalk wk(a, ends); wk.more(a); wk.next(a)) {
        const PcItem m(a, wk);
        const bool mine = w == 0 || m.two;
        int s = m.s0;
        for (; s < m.s1; ++s, ++G) {
          const uint32_t st = G % C::NV;
          if (!wait_warp(v_full(st), (G / C::NV) & 1)) break;
          if (!mine) {  // (after the wait: else it could pass the ring's round)
            if (elect_one()) mbar_arrive(v_empty(st));
            __syncwarp();
            continue;
          }
          if (!wait_warp(p_full(w), gp & 1)) break;
          if (s == m.s0 && io > 0 && !wait_warp(o_free(w), (io - 1) & 1)) break;
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < PC_T / 16; ++kk)
              tc_mma_f16_ts(tO, tP + kk * 8, dv0 + st * (C::TILE >> 4) + kk * (2048 >> 4), idesc,
                            (s > m.s0 || kk > 0) ? 1u : 0u);
            tc_commit(p_free(w));
            tc_commit(v_empty(st));
            if (s == m.s1 - 1) tc_commit(o_full(w));
          }
          __syncwarp();
          ++gp;
        }
        if (s < m.s1) break;  // a wait ran out
        if (mine) ++io;
      }
      if (elect_one()) tc_commit(done);
      __syncwarp();
    }
  } else if (warp < 12) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::REGS_ROWS));
    // ------------------------------------------------------------ softmax
    const int w = (warp - 4) >> 2;  // tile A (0) or B (1)
    const int q4 = warp & 3;        // TMEM lane quarter
    const int r = q4 * 32 + lane;   // row in the tile = TMEM lane
    const int tok = r / a.geo.g;    // its token in the tile (past the last: a row of its own that goes nowhere)
    const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16);
    const uint32_t ts = tl + 128 * w, to = tl + C::tm_o(w), tp = tl + C::tm_p(w);
    const float2 sl = make_float2(a.sl2, a.sl2);
    bool ok = true, late = false;  // late: a row was not finite
    uint32_t g = 0, io = 0, it = 0;
    for (PcWalk wk(a, ends); wk.more(a); wk.next(a), ++it) {
      const PcItem m(a, wk);
      if (w == 1 && !m.two) {
        if (!wait_warp(q_full, it & 1)) break;  // (else it could pass the other warps by a round)
        mbar_arrive_warp(q_empty);
        continue;
      }
      const int pos = m.sp.pf + w * a.geo.tpt + tok;  // row of the token in its sequence
      // tiles with keys hidden from some row of this tile: past the first one's diagonal, or
      // before the last one's window
      const int diag = m.sp.pf + w * a.geo.tpt;
      const int edge = a.geo.W > 0 ? diag + a.geo.tpt - a.geo.W : -0x7fffffff;
      float mref = -INFINITY, l = 0.f;
      auto step = [&](auto masked, int kt) -> bool {
        constexpr bool MASKED = decltype(masked)::value;
        if (!wait_warp(s_full(w), g & 1)) return false;
        tc_fence_after();
        // the scores into registers, the first half's maxima while the second comes
        uint32_t sc[PC_T];
        float mx[8];
        auto maxima = [&](int c0) {
#pragma unroll
          for (int c = c0; c < c0 + PC_T / 2; c += 16)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              mx[e] = c == 0 ? fmaxf(__uint_as_float(sc[2 * e]), __uint_as_float(sc[2 * e + 1]))
                             : max3f(mx[e], __uint_as_float(sc[c + 2 * e]), __uint_as_float(sc[c + 2 * e + 1]));
        };
        if (!MASKED) {
          tmem_ld32_async(ts, sc);
          tmem_ld32_async(ts + 32, sc + 32);
          tmem_wait_ld(sc);
          tmem_wait_ld(sc + 32);
          tmem_ld32_async(ts + 64, sc + 64);
          tmem_ld32_async(ts + 96, sc + 96);
          maxima(0);
#pragma unroll
          for (int e = 0; e < 8; ++e) asm volatile("" : "+f"(mx[e]));
          tmem_wait_ld(sc + 64);
          tmem_wait_ld(sc + 96);
        } else {
#pragma unroll
          for (int c = 0; c < PC_T; c += 32) tmem_ld32_async(ts + c, sc + c);
#pragma unroll
          for (int c = 0; c < PC_T; c += 32) tmem_wait_ld(sc + c);
        }
        if (!C::ALIAS) {  // the next scores may replace them
          tc_fence_before();
          mbar_arrive_warp(s_free(w));
        }
        if (MASKED) {
          // seen keys: (pos - W, pos], and the sinks; bit c of a word: its column c
          auto low = [](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };
#pragma unroll
          for (int c0 = 0; c0 < PC_T; c0 += 32) {
            const int b0 = kt * PC_T + c0;
            uint32_t vis = low(pos + 1 - b0);
            if (a.geo.W > 0) vis &= ~low(pos - a.geo.W + 1 - b0) | low(a.geo.S - b0);
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!(vis >> c & 1)) sc[c0 + c] = 0xff800000u;  // -inf
          }
          maxima(0);
        }
        maxima(PC_T / 2);
        const float mt =
            max3f(max3f(mx[0], mx[1], mx[2]), max3f(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * a.sl2;
        // the first keys set the reference; later ones raise it only by more than
        // PC_RESCALE, scaling O and the running sum
        if (__any_sync(0xffffffffu, mt > mref + PC_RESCALE)) {
          float corr = 1.f;
          if (mt > mref + PC_RESCALE) {
            if (mref != -INFINITY) corr = ex2_approx(mref - mt);
            mref = mt;
          }
          if (__any_sync(0xffffffffu, corr != 1.f)) {  // this warp's rows of O
            if (!wait_warp(p_free(w), (g - 1) & 1)) return false;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < DH; c += 16) {
              uint32_t ov[16];
              tmem_ld16(to + c, ov);
#pragma unroll
              for (int e = 0; e < 16; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * corr);
              tmem_st16(to + c, ov);
            }
            l *= corr;
          }
        }
        // P = 2^(s * sl2 - m) as bf16 pairs (key 2c, 2c + 1 in column c) and the row
        // sum, with packed fp32x2 arithmetic
        const float ref = mref == -INFINITY ? 0.f : mref;
        const float2 nm = make_float2(-ref, -ref);
        float2 ps[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        uint32_t pk[PC_T / 2];
#pragma unroll
        for (int hh = 0; hh < PC_T / 32; ++hh) {
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float2 z = __ffma2_rn(make_float2(__uint_as_float(sc[32 * hh + 2 * c]),
                                                    __uint_as_float(sc[32 * hh + 2 * c + 1])),
                                        sl, nm);
            const float2 pp = make_float2(ex2_approx(z.x), ex2_approx(z.y));
            ps[c & 1] = __fadd2_rn(ps[c & 1], pp);
            pk[16 * hh + c] = pack_bf16(pp.x, pp.y);
          }
          if (hh == 2 && !C::ALIAS) {  // the last tile's P has been consumed (ALIAS: before its S came)
            if (g > 0 && !wait_warp(p_free(w), (g - 1) & 1)) return false;
            tc_fence_after();
          }
          if (hh >= 2)
#pragma unroll
            for (int c = hh == 2 ? 0 : 16 * hh; c <= 16 * hh; c += 16) tmem_st16(tp + c, pk + c);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive_warp(p_full(w));
        l += (ps[0].x + ps[0].y) + (ps[1].x + ps[1].y);
        ++g;
        return true;
      };
#pragma unroll 1
      for (int s = m.s0; ok && s < m.s1; ++s) {
        const int kt = m.sp.tile(s);
        ok = kt * PC_T + PC_T - 1 > diag || kt * PC_T < edge ? step(std::true_type{}, kt) : step(std::false_type{}, kt);
      }
      if (!ok) break;
      // the item's O: after its last P V
      if (!wait_warp(o_full(w), io & 1)) break;
      ++io;
      tc_fence_after();
      const int toks = w ? m.toks - a.geo.tpt : min(m.toks, a.geo.tpt);
      if (m.whole) {
        // the warp's rows through the query tile's own, which no MMA reads any more, and out row by row
        const float inv = 1.f / l;  // (a row sees itself: 0 where its scores are all -inf, and 0 / 0 is NaN)
        float2 fin = make_float2(0.f, 0.f);  // zero, but for sums that are not finite
#pragma unroll
        for (int c = 0; c < DH; c += 32) {
          uint32_t ov[32];
          tmem_ld32_async(to + c, ov);
          tmem_wait_ld(ov);
          uint8_t* stg = smem + w * C::TILE + c / 64 * C::HALF + r * 128;
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            uint32_t pk[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 o = __fmul2_rn(make_float2(__uint_as_float(ov[i + 2 * e]), __uint_as_float(ov[i + 2 * e + 1])),
                                          make_float2(inv, inv));
              fin = __ffma2_rn(o, make_float2(0.f, 0.f), fin);
              pk[e] = pack_bf16(o.x, o.y);
            }
            *reinterpret_cast<uint4*>(stg + ((((c % 64 + i) / 8) ^ (r & 7)) << 4)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
          }
        }
        late |= fin.x + fin.y != 0.f && tok < toks;
        tc_fence_before();
        mbar_arrive_warp(o_free(w));
        bf16* const row = tok < toks ? a.out + (long)(m.t0 + w * a.geo.tpt + tok) * a.ldo +
                                           ((long)m.h * a.geo.g + r % a.geo.g) * DH
                                     : nullptr;
        constexpr int CH = DH / 8;  // 16-byte pieces of a row
#pragma unroll 4
        for (int i = 0; i < CH; ++i) {
          const int e = i * 32 + lane, rr = e / CH, c = e % CH;
          bf16* const dst = reinterpret_cast<bf16*>(__shfl_sync(0xffffffffu, (unsigned long long)row, rr));
          const uint4 u = *reinterpret_cast<const uint4*>(smem + w * C::TILE + c / 8 * C::HALF + (q4 * 32 + rr) * 128 +
                                                          (((c % 8) ^ (rr & 7)) << 4));
          if (dst) *reinterpret_cast<uint4*>(dst + c * 8) = u;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      } else {
        const long slot = (2l * blockIdx.x + (wk.at.b == ends[0].b && wk.at.h == ends[0].h && wk.at.u == ends[0].u ? 0 : 1)) *
                              a.piece_rows + w * PC_T + r;
        if (tok < toks) a.ml[slot] = make_float2(mref, l);
#pragma unroll 1
        for (int c = 0; c < DH; c += 32) {
          uint32_t ov[32];
          tmem_ld32_async(to + c, ov);
          tmem_wait_ld(ov);
          if (tok < toks)
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              *reinterpret_cast<uint4*>(a.part + slot * DH + c + i) = make_uint4(ov[i], ov[i + 1], ov[i + 2], ov[i + 3]);
        }
        tc_fence_before();
        mbar_arrive_warp(o_free(w));
      }
      mbar_arrive_warp(q_empty);
    }
    if (__any_sync(0xffffffffu, late)) {
      __syncwarp();
      for (PcWalk wk(a, ends); wk.more(a); wk.next(a)) {
        const PcItem m(a, wk);
        const int toks = w ? m.toks - a.geo.tpt : min(m.toks, a.geo.tpt);
        if (!m.whole) continue;
        bool bad = false;
        const int t = m.t0 + w * a.geo.tpt + tok, hq = m.h * a.geo.g + r % a.geo.g;
        if (tok < toks) {
          float sum = 0.f;
          for (int c = 0; c < DH; c += 8) {
            const uint4 u = __ldcg(reinterpret_cast<const uint4*>(a.out + t * a.ldo + (long)hq * DH + c));
            for (uint32_t x : {u.x, u.y, u.z, u.w}) sum = fmaf(unpack_bf16(x).x, 0.f, fmaf(unpack_bf16(x).y, 0.f, sum));
          }
          bad = sum != 0.f;
        }
        for (uint32_t again = __ballot_sync(0xffffffffu, bad); again; again &= again - 1) {
          const int src = __ffs(again) - 1;
          pc_repair<DH, Q8>(a, wk.at.b, m.h, __shfl_sync(0xffffffffu, hq, src), __shfl_sync(0xffffffffu, t, src),
                            __shfl_sync(0xffffffffu, m.sp.pf + w * a.geo.tpt + tok, src), m.sp.pf, m.sp.pl);
        }
      }
    }
  } else if (Q8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_CTRL));
    // ------------------------------------------------------------ bytes to bf16
    constexpr int LPR = DH / 16, RPW = 32 / LPR;  // lanes of a row, rows of a warp's load
    constexpr int NR = C::NR ? C::NR : 1;
    const int c = lane % LPR, sub = lane / LPR;
    bool ok = true;
    uint32_t R = 0, G = 0;  // raw tiles, steps so far
    for (PcWalk wk(a, ends); wk.more(a) && ok; wk.next(a)) {
      const PcItem m(a, wk);
      for (int s = m.s0; s < m.s1 && ok; ++s, ++G) {
#pragma unroll 1
        for (int kv = 0; kv < 2 && ok; ++kv, ++R) {
          const uint32_t st = R % NR, n = kv ? C::NV : C::NK, dst = G % n;
          const uint32_t full = kv ? v_full(dst) : k_full(dst), empty = kv ? v_empty(dst) : k_empty(dst);
          ok = wait_warp(empty, ((G / n) & 1) ^ 1) && wait_warp(r_full(st), (R / NR) & 1);
          if (!ok) break;
          const uint8_t* raw = smem + C::OFF_RAW + st * C::RAW;
          const signed char* ex = reinterpret_cast<const signed char*>(smem + C::OFF_EXP + st * PC_T);
          uint8_t* tile = smem + (kv ? C::OFF_V : C::OFF_K) + dst * C::TILE;
#pragma unroll 2
          for (int i = 0; i < PC_T / (4 * RPW); ++i) {
            const int row = (i * 4 + warp - 12) * RPW + sub;
            const uint4 u = *reinterpret_cast<const uint4*>(raw + row * DH + c * 16);
            const float f = pq_scale(ex[row]), sh = pq_shift(f);
            const float2 ff = make_float2(f, f), bb = make_float2(sh, sh);
            const uint2 v0 = pq_values(u.x, ff, bb), v1 = pq_values(u.y, ff, bb), v2 = pq_values(u.z, ff, bb),
                        v3 = pq_values(u.w, ff, bb);
            const uint4 lo = make_uint4(v0.x, v0.y, v1.x, v1.y), hi = make_uint4(v2.x, v2.y, v3.x, v3.y);
            uint8_t* o = tile + (c / 4) * C::HALF + row * 128;
            const int p = c % 4 * 2, flip = c / 4;  // (lanes of the second half write their pieces the other way round)
            *reinterpret_cast<uint4*>(o + (((p + flip) ^ (row & 7)) << 4)) = flip ? hi : lo;
            *reinterpret_cast<uint4*>(o + (((p + 1 - flip) ^ (row & 7)) << 4)) = flip ? lo : hi;
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_arrive_warp(r_empty(st));
          mbar_arrive_warp(full);
        }
      }
    }
  }
  tc_fence_before();
  if (__syncthreads_or(*(volatile int*)&g_dev_error == DEVERR_TIMEOUT)) {
    // error path: let this CTA's copies and MMAs land before smem / TMEM go
    if (warp == 0 && lane == 0) {
      for (uint32_t i = k_issued > C::NK ? k_issued - C::NK : 0; i < k_issued; ++i)
        mbar_wait_drain(k_full(i % C::NK), (i / C::NK) & 1);
      for (uint32_t i = v_issued > C::NV ? v_issued - C::NV : 0; i < v_issued; ++i)
        mbar_wait_drain(v_full(i % C::NV), (i / C::NV) & 1);
      if (Q8)
        for (uint32_t i = r_issued > C::NR ? r_issued - C::NR : 0; i < r_issued; ++i)
          mbar_wait_drain(r_full(i % (C::NR ? C::NR : 1)), (i / (C::NR ? C::NR : 1)) & 1);
      if (q_issued > 0) mbar_wait_drain(q_full, (q_issued - 1) & 1);
    }
    if (warp == 1 && lane == 0) mbar_wait_drain(done, 0);
  } else if (warp == 1 && lane == 0) {
    mbar_wait(done, 0);
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Items that lie on several CTAs: the pieces joined in the order of the CTAs.  CTA x takes the item
// that begins on CTA x and ends on a later one; CTAs y share its rows, a warp to a row.
constexpr int PJ_WARPS = 8;
template <int DH, bool Q8>
__global__ void __launch_bounds__(32 * PJ_WARPS) paged_chunk_join_kernel(const __grid_constant__ PcArgs a) {
  __shared__ PcAt at[PC_CTAS + 1];
  pdl_enter();
  for (int i = threadIdx.x; i <= a.G; i += 32 * PJ_WARPS) at[i] = a.at[i];
  __syncthreads();
  const int x = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const PcAt m = at[x + 1];
  auto same = [&](const PcAt& p) { return p.b == m.b && p.h == m.h && p.u == m.u; };
  if (m.s == 0 || (same(at[x]) && at[x].s > 0)) return;
  int n = 2;  // CTAs that begin inside the item, and this one (at[G] is the line's end)
  while (same(at[x + n]) && at[x + n].s > 0) ++n;
  // whether CTA x + k holds a piece of it: it may begin where the next one does
  auto holds = [&](int k) { return k < n && !(k > 0 && same(at[x + k + 1]) && at[x + k + 1].s == at[x + k].s); };
  const PcSeq q = pc_seq(a, m.b);
  const PcSpan sp = pc_span(a.geo, q, m.u);
  const int R = 2 * a.geo.tpt, toks = min(q.n - m.u * R, R), g = a.geo.g;
  const int first = same(at[x]) ? 0 : 1;  // piece 0 is the last of its CTA's, the others the first
  constexpr int C = DH / 32;
  for (int i = blockIdx.y * PJ_WARPS + warp; i < toks * g; i += gridDim.y * PJ_WARPS) {
    const int tok = i / g, hg = i % g, w = tok / a.geo.tpt, rr = w * PC_T + (tok - w * a.geo.tpt) * g + hg;
    auto slot = [&](int k) { return (2l * (x + k) + (k == 0 ? first : 0)) * a.piece_rows + rr; };
    float M = -INFINITY, L = 0.f, acc[C] = {};
    for (int k = lane; k < n; k += 32)
      if (holds(k)) M = fmaxf(M, a.ml[slot(k)].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    for (int k0 = 0; k0 < n; k0 += 32) {
      float f = 0.f;
      const bool in = holds(k0 + lane);
      if (in) {
        const float2 y = a.ml[slot(k0 + lane)];
        f = M == -INFINITY ? 0.f : ex2_approx(y.x - M);
        L = fmaf(y.y, f, L);
      }
      const uint32_t held = __ballot_sync(0xffffffffu, in);
#pragma unroll 8
      for (int k = 0; k < min(32, n - k0); ++k) {
        const float fk = __shfl_sync(0xffffffffu, f, k);
        if (!(held >> k & 1)) continue;
        const float* p = a.part + slot(k0 + k) * DH + C * lane;
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] = fmaf(p[c], fk, acc[c]);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
    const int t = q.t0 + m.u * R + tok, hq = m.h * g + hg;
    bf16* o = a.out + t * a.ldo + (long)hq * DH + C * lane;
    bool bad = false;
#pragma unroll
    for (int c = 0; c < C; c += 2) {
      const float2 v = make_float2(acc[c] / L, acc[c + 1] / L);
      bad |= fmaf(v.x, 0.f, v.y * 0.f) != 0.f;
      *reinterpret_cast<uint32_t*>(o + c) = pack_bf16(v.x, v.y);
    }
    if (__any_sync(0xffffffffu, bad)) pc_repair<DH, Q8>(a, m.b, m.h, hq, t, sp.pf + tok, sp.pf, sp.pl);
  }
}

struct PcPlan {
  int tpt, G, piece_rows;
  bool split;
  size_t at, ml, bytes;
};
PcPlan pc_plan(const Paged& c, long rows) {
  PcPlan p;
  const int g = c.H / c.KV;
  p.tpt = PC_T / g;
  long keys = std::min<long>((long)c.max_pages * c.page, 0x7fffffffL);
  if (c.window > 0) keys = std::min<long>(keys, (long)c.window + c.sinks + 2 * p.tpt + 2 * PC_T);
  const long steps = (keys + PC_T - 1) / PC_T, R = 2 * p.tpt;
  // items at most: a pair of each sequence that is not full, and the full ones
  const long items = (std::min<long>(c.B, rows) + rows / R) * c.KV;
  p.split = steps > 1;
  p.G = (int)std::min<long>(PC_CTAS, p.split ? (items > PC_CTAS ? PC_CTAS : items * std::min<long>(steps, PC_CTAS)) : items);
  p.G = std::max(p.G, 1);
  p.piece_rows = rows > p.tpt ? 2 * PC_T : PC_T;
  auto up = [](size_t n) { return (n + 255) & ~size_t(255); };
  p.at = 0;
  p.ml = up((p.G + 1) * sizeof(PcAt));
  const size_t slots = 2 * (size_t)p.G * p.piece_rows;
  p.bytes = p.ml + up(slots * sizeof(float2)) + slots * c.dh * sizeof(float);
  if (!p.split) p.bytes = 0;
  return p;
}

template <int DH, bool Q8>
cudaError_t pc_launch(const Paged& c, const PcArgs& a, const PcPlan& p, cudaStream_t st) {
  using C = PcCfg<DH, Q8>;
  CUtensorMap tq, tk, tv;
  if (!tmap_bf16_heads(&tq, a.q, DH, c.H, a.rows, a.ldq, a.geo.g, a.geo.tpt) ||
      !tmap_pages(&tk, c.K, Q8, DH, c.page, c.KV, c.n_pages, a.box) ||
      !tmap_pages(&tv, c.V, Q8, DH, c.page, c.KV, c.n_pages, a.box))
    return cudaErrorInvalidValue;
  static KernelOnce once;
  cudaError_t e = once(reinterpret_cast<const void*>(paged_chunk_kernel<DH, Q8>), C::SMEM, C::THREADS, C::POOL);
  if (e != cudaSuccess) return e;
  // work: upper bound (every cache full, all rows of the longest)
  const double keys = (double)std::min<long>((long)c.max_pages * c.page, 0x7fffffffL);
  {
    LaunchTimer lt("paged_chunk", st, 4.0 * a.rows * c.H * DH * keys,
                   (double)c.B * c.KV * keys * DH * (Q8 ? 2.0 : 4.0) + 4.0 * a.rows * c.H * DH);
    e = launch_kernel(paged_chunk_kernel<DH, Q8>, a.G, C::THREADS, C::SMEM, st, tq, tk, tv, a);
    if (e != cudaSuccess || !p.split) return e;
  }
  LaunchTimer lt("paged_chunk_join", st, 0.0, 8.0 * a.G * p.piece_rows * DH);
  return launch_kernel(paged_chunk_join_kernel<DH, Q8>, dim3(a.G, 8), 32 * PJ_WARPS, 0, st, a);
}

}  // namespace

static_assert(PC_MAX_B == PF_PAGED_MAX_BATCH, "limit of the entry points");

size_t paged_chunk_ws_bytes(const Paged& c, long rows) { return rows > 0 ? pc_plan(c, rows).bytes : 0; }

cudaError_t paged_chunk(const Paged& c, long rows, const bf16* q, long ldq, const int* start, bf16* out, long ldo,
                        void* ws, cudaStream_t st) {
  launched.mark();
  const PcPlan p = pc_plan(c, rows);
  PcArgs a{};
  a.geo = {c.B, c.KV, c.H / c.KV, p.tpt, c.window, c.sinks};
  a.start = start; a.len = c.len; a.table = c.table;
  a.rows = rows;
  a.page = c.page; a.max_pages = c.max_pages;
  a.n_pages = c.n_pages;
  a.box = std::min(PC_T, c.page & -c.page);
  a.G = p.G;
  a.whole = p.split ? 8 : 0;
  a.few = 3 * PC_T;
  a.sl2 = 1.4426950408889634f / sqrtf((float)c.dh);
  a.q = q; a.ldq = ldq;
  a.out = out; a.ldo = ldo;
  a.K = c.K; a.V = c.V; a.Ke = c.Ke; a.Ve = c.Ve;
  if (p.split) {
    char* w = static_cast<char*>(ws);
    a.at = reinterpret_cast<PcAt*>(w + p.at);
    a.ml = reinterpret_cast<float2*>(w + p.ml);
    a.part = reinterpret_cast<float*>(w + p.bytes) - 2 * (size_t)p.G * p.piece_rows * c.dh;
  }
  a.piece_rows = p.piece_rows;
  if (c.Ke) return c.dh == 128 ? pc_launch<128, true>(c, a, p, st) : pc_launch<64, true>(c, a, p, st);
  return c.dh == 128 ? pc_launch<128, false>(c, a, p, st) : pc_launch<64, false>(c, a, p, st);
}

}  // namespace pf

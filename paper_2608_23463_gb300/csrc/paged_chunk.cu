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
//   warps 2-3  MMA issuers of tile A's and tile B's O += P V (M=128, N=dh, K=128), P from TMEM; rows of V
//              behind an item's last token become zeros before its last product (quantised: finite, by the
//              warps that convert them)
//   warps 4-7  softmax of tile A, warps 8-11 of tile B: one row per thread (TMEM lane); the
//              running maximum moves by more than 2^8 only, which then scales O
//   warps 12-19 (quantised caches) turn the producer's raw tiles of bytes into the bf16 tiles
//              that the MMAs read, 2^-7 of the values
// An item of one query tile shares its steps out between the two tiles' places, the even to A's
// and the odd to B's, so that two steps are in flight as with two tiles.
// TMEM holds both tiles' S and O; with dh = 128 P takes the place of S, from which it came.
// An item that one CTA holds whole is written; pieces leave (O, maximum, sum) and
// paged_chunk_join_kernel joins them in the order of the CTAs: results repeat bit for bit.
// P is rounded to bf16 (half a step, 2^-8) for its product, its sum taken before that.
//
// Few tokens on long caches are bound by HBM (up to 8 tokens of each of 8 sequences over 77K rows of
// 16 heads of 128, 107 us: 5.9 TB/s), a long prompt's chunk by a tile's chain of scores, softmax and sum
// (2048 tokens on 30000 rows, 16 heads on 2: 338 to 364 us by what ran before it, 1.43 to 1.54 PFLOP/s,
// tensor pipe 67 %), quantised caches by the conversion beside the softmax (up to 5 tokens of each of 32
// sequences of 16 heads on 2, 58 us; from bf16 pages 54), short calls by instructions that come from L2 (12000 cycles before the first sum).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "local.h"
#include "paged_items.cuh"
#include "paged_q8.cuh"

namespace pf {

static Launched launched;
int take_dev_error_paged_chunk() { return launched.take(take_dev_error_tu); }
int set_wait_limit_paged_chunk(unsigned long long ns) { return set_wait_limit_tu(ns); }
static std::atomic<int> stop_after{-1};
void set_debug_chunk_steps(int steps) { stop_after.store(steps); }

namespace {

constexpr int PC_CTAS = 152;  // one an SM, whatever the device has: splits keep their places
constexpr int PC_MAX_B = 2048;
constexpr long PC_LONGEST = 0x7fffff00;  // rows of a sequence: indices of their tiles fit 32 bits
constexpr float PC_RESCALE = 8.f;

template <int DH, bool Q8>
struct PcCfg {
  static constexpr int CONV = Q8 ? 8 : 0;  // converting warps
  static constexpr int THREADS = 384 + 32 * CONV;
  // registers of a control (and converting) and of a softmax thread, of the pool at launch
  static constexpr int REGS_CTRL = Q8 ? 72 : 88, REGS_ROWS = Q8 ? 128 : 208;
  static constexpr int POOL = REGS_CTRL * (THREADS - 256) + REGS_ROWS * 256;
  static_assert(POOL <= (65536 / THREADS / 8 * 8) * THREADS, "register split");
  static constexpr int HALVES = DH / 64;
  static constexpr uint32_t HALF = PC_T * 128;  // 64 columns of a tile
  static constexpr uint32_t TILE = HALVES * HALF;
  static constexpr int NK = DH == 64 ? 4 : 2, NV = DH == 64 ? 4 : (Q8 ? 2 : 3);  // stages
  static constexpr uint32_t RAW = PC_T * DH;  // a tile of bytes
  static constexpr int NR = Q8 ? (DH == 64 ? 4 : 2) : 0;  // stages of them, half for K, half for V
  static constexpr int NQ = DH == 64 ? 2 : 1;  // items whose query tiles are held
  static constexpr int AHEAD = NK < NV ? NK : NV;  // steps of an item that can be loaded before its queries
  static constexpr uint32_t OFF_K = NQ * 2 * TILE, OFF_V = OFF_K + NK * TILE, OFF_RAW = OFF_V + NV * TILE;
  static constexpr uint32_t OFF_EXP = OFF_RAW + NR * RAW, OFF_BAR = OFF_EXP + NR * PC_T;
  static constexpr uint32_t SMEM = OFF_BAR + 512 + 1024;
  static_assert(SMEM <= 227 * 1024, "shared memory");
  static_assert((PC_MAX_B + 1) * 8 + PC_MAX_B * 20 <= (NK + NV) * TILE, "the totals lie in the rings at first");
  // TMEM columns of tile w: S at 128 w, O and P
  static constexpr bool ALIAS = DH == 128;
  static constexpr float SCALE = Q8 ? 1 << PQ_DOWN : 1;  // the tiles hold so much less than the values
  __host__ __device__ static constexpr uint32_t tm_o(int w) { return 256 + DH * w; }
  __host__ __device__ static constexpr uint32_t tm_p(int w) { return ALIAS ? 128 * w : 384 + 64 * w; }
};

struct PcArgs {
  PcGeo geo;
  const int *start, *len, *table;
  long rows;
  int page, max_pages, box, box_log;  // box: rows of a TMA box, 2^box_log
  int step_pages, step_rows;          // that a step of PC_T rows is
  long n_pages;
  int G;           // CTAs
  int few;         // weight to a CTA at least
  int long_item;   // steps from which an item's unmasked ones take the long form
  int stop;        // steps that a CTA's producer loads, for a test
  float sl2;       // log2(e) / sqrt(dh), of the tiles' keys
  const bf16* q;
  bf16* out;
  long ldq, ldo;
  const void *K, *V;
  const signed char *Ke, *Ve;
  // pieces: where each CTA begins [G + 1], (maximum, sum) [2 G][rows of an item], O [2 G][dh / 4][rows]
  PcAt* at;
  float2* ml;
  float4* part;
  int piece_rows;
};

__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16 bytes, or as many zeros, and the arrival of a thread's copies at a barrier that counts it.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool full) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(full ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
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

// A CTA's part of the line, and the sequence that it begins in.
struct PcEnds {
  PcAt at[2];
  PcSeq q;
};

// A piece of an item: its steps [s0, s1).  s1 = 0: there are no more.
struct PcItem {
  PcSpan sp;
  int b, h, t0, toks, s0, s1, place;  // place: of the piece among those of all CTAs
  int two, duo, whole;  // with a tile B; tile A's steps shared with tile B's place; all of its steps
};

// The items from one place in the line to another.
struct PcWalk {
  PcAt at, end;
  PcSeq q;
  int pairs, n;  // n: items so far
  __device__ __forceinline__ PcWalk(const PcArgs& a, const PcEnds& e) : at(e.at[0]), end(e.at[1]), q(e.q), n(0) {
    pairs = pc_pairs(a.geo, q);
  }
  __device__ __forceinline__ void next(const PcArgs& a, PcItem& m) {
    const bool last = at.b == end.b && at.h == end.h && at.u == end.u;
    m.s1 = 0;
    if (at.b >= a.geo.B || (last && at.s >= end.s)) return;
    m.sp = pc_span(a.geo, q, at.u);
    m.b = at.b;
    m.h = at.h;
    const int R = 2 * a.geo.tpt;
    m.t0 = q.t0 + at.u * R;
    m.toks = min(q.n - at.u * R, R);
    m.s0 = at.s;
    m.s1 = last ? end.s : m.sp.steps;
    m.two = m.toks > a.geo.tpt;
    m.duo = !m.two && m.s1 - m.s0 > 1;
    m.whole = m.s0 == 0 && m.s1 == m.sp.steps;
    m.place = 2 * blockIdx.x + (n++ ? 1 : 0);
    at.s = 0;
    if (last) {
      at.s = end.s;
    } else if (++at.u == pairs) {
      at.u = 0;
      if (++at.h == a.geo.KV) {
        at.h = 0;
        do {
          if (++at.b >= a.geo.B) return;
          q = pc_seq(a, at.b);
        } while (q.n == 0);
        pairs = pc_pairs(a.geo, q);
      }
    }
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
// are not finite and that another of the item's tokens sees, or that lie before those in a block of
// the window's first or the sinks' last, it is worked out again from the rows that it sees, the newest first: of a
// sequence that has turned to NaN those are NaN themselves, and the end of it.  For a converged warp: a
// key to a lane for the scores, columns for the sums, of which those from c0 to c1 are written.  Out of
// line: calls without such rows have none of its registers.
template <int DH, bool Q8>
__device__ __noinline__ void pc_repair(const PcArgs& a, int b, int h, int hq, int t, int i, int pf, int pl, int c0 = 0,
                                       int c1 = DH) {
  const int lane = threadIdx.x & 31, W = a.geo.W, bx = a.box;
  const int lo = W > 0 && i >= W ? i - W + 1 : 0, S = min(a.geo.S, lo);
  const int first = W > 0 && pf >= W ? (pf - W + 1) / bx * bx : 0;
  const int held = (int)min(min(((long)a.geo.S + bx - 1) / bx * bx, (long)lo), (long)(pf - pf % bx));
  if (!pc_not_finite<DH, Q8>(a, b, h, i + 1, pl + 1) &&
      !(W > 0 && (pc_not_finite<DH, Q8>(a, b, h, max(first, S), lo) || pc_not_finite<DH, Q8>(a, b, h, S, held))))
    return;
  constexpr int C = DH / 32;  // columns of a lane
  const bf16* q = a.q + t * a.ldq + (long)hq * DH;
  const float sl2 = a.sl2 / PcCfg<DH, Q8>::SCALE;
  float acc[C] = {}, m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {  // the window, the sinks before it, newest keys first
    const int begin = part ? 0 : lo;
#pragma unroll 1
    for (int j = part ? S : i + 1; j > begin; j -= 32) {
      const int key = j - 1 - lane;
      const bool in = key >= begin;
      const long pg = in ? pc_page(a, b, key) : -1;
      const long at = pg < 0 ? -1 : (pg * a.geo.KV + h) * a.page + key % a.page;
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
      const float next = fmaxf(m, mx * sl2), ref = next == -INFINITY ? 0.f : next;
      const float corr = m == -INFINITY ? 1.f : ex2_approx(m - ref);
      m = next;
      const float p = in ? ex2_approx(fmaf(s, sl2, -ref)) : 0.f;
      float sum = p;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      l = fmaf(l, corr, sum);
      bool nan = true;
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c] *= corr;
#pragma unroll 1
      for (int k = 0; k < min(32, j - begin); ++k) {
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
  if (C * lane < c0 || C * lane >= c1) return;
#pragma unroll
  for (int c = 0; c < C; c += 2)
    *reinterpret_cast<uint32_t*>(o + c) = pack_bf16(acc[c] / l, acc[c + 1] / l);
}

// Weight of a head of a sequence's; any_bad becomes 1 if it cannot be.
struct PcLoad {
  PcSeq q;
  long long weight;
  __device__ __forceinline__ PcLoad(const PcArgs& a, int b, int* any_bad) {
    bool bad;
    q = pc_seq(a, b, &bad);
    if (bad) {
      set_dev_error(DEVERR_CAPACITY);
      *any_bad = 1;
      q.n = 0;
    }
    const int P = pc_pairs(a.geo, q);
    weight = P > 0 ? pc_cum(a.geo, q, P, P) : 0;
  }
};

__device__ __forceinline__ long long warp_scan(long long v) {  // sums up to and with the lane
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long t = __shfl_up_sync(0xffffffffu, v, o);
    if ((int)(threadIdx.x & 31) >= o) v += t;
  }
  return v;
}

// The CTA's part of the line, and its entry in the pieces' index.  room: for B + 1 totals, B
// heads' weights and sequences.  (Each CTA works it out for itself: a kernel before this one would cost a launch.)
// pc_totals: more than PC_FEW sequences, by all of a CTA's threads.  pc_share_out: warp 0 the CTA's
// beginning, warp 1 the next one's.  Both are on the way to a call's first load, where every
// instruction comes from L2, to all SMs at once: 12000 cycles in their first form, by one thread.
struct PcRoom {
  long long* pre;  // pre[b]: weight of the sequences before b
  long long* head;  // of a head of each
  PcSeq* seq;
  __device__ __forceinline__ PcRoom(void* room, int B)
      : pre(static_cast<long long*>(room)), head(pre + B + 1), seq(reinterpret_cast<PcSeq*>(head + B)) {}
};
constexpr int PC_FEW = 128;
static_assert((PC_FEW + 1) * 8 + PC_FEW * 20 <= 4096, "a room for each");
template <int THREADS>
__device__ __noinline__ void pc_totals(const PcArgs& a, void* room, int* any_bad) {
  __shared__ long long wsum[THREADS / 32];
  const PcRoom m(room, a.geo.B);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = a.geo.B;
  long long T = 0;
  for (int b0 = 0; b0 < B; b0 += THREADS) {
    const int b = b0 + tid;
    long long u = 0;
    if (b < B) {
      const PcLoad x(a, b, any_bad);
      m.seq[b] = x.q;
      m.head[b] = x.weight;
      u = a.geo.KV * x.weight;
    }
    const long long v = warp_scan(u);
    if (lane == 31) wsum[warp] = v;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll 1
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) before += wsum[w];
      all += wsum[w];
    }
    if (b < B) m.pre[b] = T + before + v - u;
    T += all;
    __syncthreads();
  }
  if (tid == 0) m.pre[B] = T;
  __syncthreads();
}

__device__ __forceinline__ void pc_share_out(const PcArgs& a, void* room, int warp, PcEnds& ends, int* any_bad) {
  // (few sequences: each of the two warps in a room of its own)
  const PcRoom m(static_cast<char*>(room) + (a.geo.B <= PC_FEW ? warp * 4096 : 0), a.geo.B);
  const int lane = threadIdx.x & 31, B = a.geo.B;
  // the last of [0, hi) that does not begin behind the place, with all lanes
  auto find = [&](int hi, auto before) {
    int lo = 0;
#pragma unroll 1
    while (hi - lo > 1) {
      const int d = (unsigned)(hi - lo + 31) / 32, i = lo + (lane + 1) * d;
      const int k = __popc(__ballot_sync(0xffffffffu, i < hi && before(i)));
      hi = min(hi, lo + (k + 1) * d);
      lo += k * d;
    }
    return lo;
  };
  if (B <= PC_FEW) {
    const int per = (B + 31) / 32;
    long long u = 0;
#pragma unroll 1
    for (int i = 0; i < per; ++i) {
      const int b = lane * per + i;
      if (b >= B) break;
      const PcLoad x(a, b, any_bad);
      m.seq[b] = x.q;
      m.head[b] = x.weight;
      m.pre[b] = u;
      u += a.geo.KV * x.weight;
    }
    const long long v = warp_scan(u) - u;
#pragma unroll 1
    for (int b = lane * per; b < min(B, (lane + 1) * per); ++b) m.pre[b] += v;
    if (lane == 31) m.pre[B] = v + u;
    __syncwarp();
  }
  PcSeq q{0, 0, 0};
  const long long T = m.pre[B];
  int n = a.G;
  if (T < (long long)a.few * n) n = max(1, (int)T / a.few);
  const int c = min((int)blockIdx.x + warp, n);
  PcAt r{B, 0, 0, 0};
  long long y = pc_share(T, n, c);
  if (y < T) {
    r.b = find(B, [&](int i) { return m.pre[i] <= y; });  // (the last of those that begin there: it has tokens)
    y -= m.pre[r.b];
    q = m.seq[r.b];
    const int P = pc_pairs(a.geo, q);
    r.h = pc_head(m.head[r.b], y);
    r.u = find(P, [&](int i) { return pc_cum(a.geo, q, i, P) <= y; });
    // (pc_cum's copies are fetched one by one: lane 0 the weight before the pair, lane 1 with it)
    const long long w = pc_cum(a.geo, q, r.u + (lane & 1), P), w0 = __shfl_sync(0xffffffffu, w, 0);
    r.s = pc_step(pc_span(a.geo, q, r.u).steps, y - w0, __shfl_sync(0xffffffffu, w, 1) - w0);
  }
  if (lane == 0) {
    ends.at[warp] = r;
    if (warp == 0) ends.q = q;
    // (CTAs without a part write the line's end, each its own place)
    if (a.at && warp == 0) a.at[blockIdx.x] = r;
    if (a.at && warp == 1 && (int)blockIdx.x + 1 == a.G) a.at[a.G] = r;
  }
}

// CUT: for a test of the waits, the producer loads a.stop steps and no more (a kernel of its own: as a branch of the
// one that serves it cost 0.3 to 1 us of 78)
template <int DH, bool Q8, bool CUT>
__global__ void __launch_bounds__(PcCfg<DH, Q8>::THREADS, 1)
    paged_chunk_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PcArgs a) {
  using C = PcCfg<DH, Q8>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ PcEnds ends;
  __shared__ PcItem slot[2];
  __shared__ int any_bad;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  const uint32_t sbase = smem_u32(smem), b0 = sbase + C::OFF_BAR;
  const uint32_t done = b0, x_full = b0 + 8, x_free = b0 + 16, shared = b0 + 24, grp0 = b0 + 96, ring0 = grp0 + 2 * 56;
  auto q_full = [&](int i) { return b0 + 32 + 8 * i; };
  auto q_empty = [&](int i) { return b0 + 48 + 8 * i; };
  auto i_full = [&](int i) { return b0 + 64 + 8 * i; };
  auto i_empty = [&](int i) { return b0 + 80 + 8 * i; };
  auto s_full = [&](int w) { return grp0 + 56 * w; };
  auto s_free = [&](int w) { return grp0 + 56 * w + 8; };
  auto p_full = [&](int w) { return grp0 + 56 * w + 16; };
  auto p_free = [&](int w) { return grp0 + 56 * w + 24; };
  auto o_full = [&](int w) { return grp0 + 56 * w + 32; };
  auto o_free = [&](int w) { return grp0 + 56 * w + 40; };
  auto p_half = [&](int w) { return grp0 + 56 * w + 48; };
  auto k_full = [&](int i) { return ring0 + 8 * i; };
  auto k_empty = [&](int i) { return ring0 + 8 * (C::NK + i); };
  auto v_full = [&](int i) { return ring0 + 8 * (2 * C::NK + i); };
  auto v_empty = [&](int i) { return ring0 + 8 * (2 * C::NK + C::NV + i); };
  auto r_full = [&](int i) { return ring0 + 8 * (2 * C::NK + 2 * C::NV + i); };
  auto r_empty = [&](int i) { return ring0 + 8 * (2 * C::NK + 2 * C::NV + C::NR + i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_BAR + 504);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    any_bad = 0;
    mbar_init(done, 3);
    mbar_init(x_full, 4);
    mbar_init(x_free, 4);
    mbar_init(shared, 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full(i), 1);
      mbar_init(q_empty(i), 8);  // one arrival per softmax warp
      mbar_init(i_full(i), 1);
      mbar_init(i_empty(i), C::THREADS / 32 - 1);  // every warp but the producer's
      mbar_init(s_full(i), 1);
      mbar_init(s_free(i), 4);
      mbar_init(p_full(i), 4);
      mbar_init(p_half(i), 4);
      mbar_init(p_free(i), 1);
      mbar_init(o_full(i), 1);
      mbar_init(o_free(i), 4);
    }
    for (int i = 0; i < C::NK; ++i) {
      mbar_init(k_full(i), Q8 ? C::CONV : 1);  // (converting warps)
      mbar_init(k_empty(i), 1);
    }
    for (int i = 0; i < C::NV; ++i) {
      mbar_init(v_full(i), Q8 ? C::CONV : 1);
      mbar_init(v_empty(i), 2);  // one arrival per tile
    }
    for (int i = 0; i < C::NR; ++i) {
      mbar_init(r_full(i), 1 + 32);  // (the copies of the exponents)
      mbar_init(r_empty(i), C::CONV);
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
  // the join's launch may begin: it waits for this grid to end, and all of its CTAs are running
  if (a.at) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  void* const room = smem + C::OFF_K;
  if (a.geo.B > PC_FEW) pc_totals<C::THREADS>(a, room, &any_bad);
  uint32_t k_issued = 0, v_issued = 0, r_issued = 0, q_issued = 0;
  // Warp 0 walks the items and writes them down, two ahead at most, for the other warps.
  // item n: bounded, false where it does not come; a copy of it is kept, its place is free again
  auto take = [&](uint32_t n, PcItem& m) {
    const uint32_t i = n & 1;
    if (!wait_warp(i_full(i), (n >> 1) & 1)) return false;
    m = slot[i];
    mbar_arrive_warp(i_empty(i));
    return m.s1 > 0;
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_CTRL));
    if (warp < 2) {
      pc_share_out(a, room, warp, ends, &any_bad);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the totals lie where the rings will be
      mbar_arrive_warp(shared);
    }
    if (warp == 0) {
      // ------------------------------------------------------------ producer (all lanes)
      const int nb = PC_T >> a.box_log, H = Q8 ? 1 : C::HALVES;
      // lane, of 16 for K and 16 for V: a block of rows and half of its columns; Q8: 16 rows, of whose block
      // the first of its lanes has the data copied, and each 16 exponents
      const int sub = lane & 15, blk = Q8 ? (sub & 7) * 16 >> a.box_log : sub / H & (nb - 1), half = sub % H;
      const bool exps = Q8 && sub < 8, data = Q8 ? exps && (sub * 16 & (a.box - 1)) == 0 : sub < nb * H;
      const uint32_t qbytes = (uint32_t)(a.geo.tpt * a.geo.g * 128 * C::HALVES);
      bool ok = wait_warp(shared, 0);
      int left = a.stop;
      PcWalk walk(a, ends);
      while (ok) {
        PcItem m;
        walk.next(a, m);
        {
          const uint32_t i = q_issued & 1;  // (items so far)
          if (!wait_warp(i_empty(i), ((q_issued >> 1) & 1) ^ 1)) break;
          if (lane == 0) slot[i] = m;
          mbar_arrive_warp(i_full(i));
        }
        if (m.s1 == 0) break;
        if (CUT) m.s1 = min(m.s1, m.s0 + left);
        // The lane's block in a step: its row, the row's place in the table, and what stands there, which is
        // looked up a step ahead and not looked at before its turn.  (With divisions, and looked at once, a
        // step took the producer 2200 cycles and all else waited for it: 64 mixed sequences 89 us, 81 so.)
        int r, at, row, entry = 0;
        bool seen;
        const int* const table = a.table + (long)m.b * a.max_pages;
        auto place = [&](int s) {
          r = m.sp.tile(s) * PC_T + blk * a.box;
          at = (int)((unsigned)r / (unsigned)a.page);
          row = r - at * a.page;
        };
        auto look = [&] {
          seen = (data || exps) && r <= m.sp.pl && (a.geo.W == 0 || r + a.box - 1 > m.sp.pf - a.geo.W || r < a.geo.S);
          if (seen) entry = table[at];
        };
        place(m.s0);
        look();
        // the item's queries, as soon as those before them are done with and before a step's place is waited
        // for that only this item's steps free
        bool queries = false;
#pragma unroll 1
        for (int s = m.s0; s < m.s1; ++s) {
          const uint32_t qb = q_issued % C::NQ, par = ((q_issued / C::NQ) & 1) ^ 1;
          const bool must = s - m.s0 == C::AHEAD - 1 || s == m.s1 - 1;
          if (!queries && (must || __all_sync(0xffffffffu, mbar_test_wait(q_empty(qb), par)))) {
            ok = wait_warp(q_empty(qb), par);
            if (!ok) break;
            if (lane == 0) mbar_arrive_expect_tx(q_full(qb), m.two ? 2 * qbytes : qbytes);
            __syncwarp();
            if (lane < C::HALVES * (m.two ? 2 : 1)) {
              const int t = lane / C::HALVES, c = lane % C::HALVES;
              tma_load_3d(sbase + (2 * qb + t) * C::TILE + c * C::HALF, &tmQ, q_full(qb), 64 * c, m.h * a.geo.g,
                          m.t0 + t * a.geo.tpt);
            }
            __syncwarp();
            queries = true;
          }
          int pg = entry;
          const int from = row;
          if (!seen || pg < 0 || pg >= a.n_pages) {
            if (seen) set_dev_error(DEVERR_CAPACITY);
            pg = (int)a.n_pages;  // (past the end: zeros)
          }
          if (s + 1 < m.s1) {
            if (s + 1 == m.sp.ns) {
              place(s + 1);
            } else {
              r += PC_T;
              at += a.step_pages;
              row += a.step_rows;
              if (row >= a.page) {
                row -= a.page;
                ++at;
              }
            }
            look();
          }
          if constexpr (Q8) {
            // K's and V's bytes and exponents; at dh = 64 both at once, which at dh = 128, with a stage each,
            // would keep K's waiting for V's to be converted
            constexpr int N = C::NR / 2;
            constexpr bool BOTH = N > 1;
#pragma unroll 1
            for (int kv = 0; kv < (BOTH ? 1 : 2); ++kv) {
              const uint32_t ring = r_issued / 2 % N, par = ((r_issued / 2 / N) & 1) ^ 1;
              ok = wait_warp(r_empty(kv * N + ring), par) && (!BOTH || wait_warp(r_empty(N + ring), par));
              if (!ok) break;
              const int own = BOTH ? lane >> 4 : kv;
              const uint32_t st = own * N + ring;
              if (lane == 0 || (BOTH && lane == 16)) mbar_arrive_expect_tx(r_full(st), C::RAW);
              __syncwarp();
              if (data && own == lane >> 4)
                tma_load_4d(sbase + C::OFF_RAW + st * C::RAW + blk * a.box * DH, own ? &tmV : &tmK, r_full(st), 0, from, m.h,
                            pg);
              // one instruction for all of a tile's exponents (a bulk copy to a block took 130 cycles, as its data's
              // does); those of blocks that no token sees, and of pages out of range: zeros
              if (exps && own == lane >> 4) {
                const bool in = pg < a.n_pages;
                const signed char* e = own ? a.Ve : a.Ke;
                cp_async16(sbase + C::OFF_EXP + st * PC_T + sub * 16,
                           in ? e + ((long)pg * a.geo.KV + m.h) * a.page + from + (sub * 16 & (a.box - 1)) : e, in);
              }
              cp_async_arrive(r_full(kv * N + ring));
              if (BOTH) cp_async_arrive(r_full(N + ring));
              __syncwarp();
              r_issued += BOTH ? 2 : 1;
            }
          } else {
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
              uint32_t& n = kv ? v_issued : k_issued;
              const uint32_t ring = kv ? C::NV : C::NK, st = n % ring, full = kv ? v_full(st) : k_full(st);
              ok = wait_warp(kv ? v_empty(st) : k_empty(st), ((n / ring) & 1) ^ 1);
              if (!ok) break;
              if (lane == 0) mbar_arrive_expect_tx(full, C::TILE);
              __syncwarp();
              if (data && lane >> 4 == kv)
                tma_load_4d(sbase + (kv ? C::OFF_V : C::OFF_K) + st * C::TILE + half * C::HALF + blk * a.box * 128,
                            kv ? &tmV : &tmK, full, 64 * half, from, m.h, pg);
              __syncwarp();
              ++n;
            }
          }
          if (!ok) break;
        }
        if (queries) ++q_issued;
        if (CUT && (left -= m.s1 - m.s0) == 0) break;
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------ MMA issuer: scores
      // The whole warp runs the loop; one elected lane issues and commits.
      constexpr uint32_t idesc = idesc_bf16_f32(PC_T, PC_T, 0, 0);
      const uint64_t dq0 = smem_desc_sw128(sbase, 16, 1024), dk0 = smem_desc_sw128(sbase + C::OFF_K, 16, 1024);
      uint32_t G = 0, g0 = 0, g1 = 0;  // steps, products of the tiles so far
      PcItem m;
      for (uint32_t it = 0; take(it, m); ++it) {
        const uint32_t qb = it % C::NQ;
        if (!wait_warp(q_full(qb), (it / C::NQ) & 1)) break;
        int s = m.s0;
#pragma unroll 1
        for (; s < m.s1; ++s, ++G) {
          const uint32_t st = G % C::NK;
          if (!wait_warp(k_full(st), (G / C::NK) & 1)) break;
          bool ok = true;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            if (!ok || (m.duo ? ((s - m.s0) & 1) != w : w > m.two)) continue;
            // S's place: read into registers, or (ALIAS) P in it taken up by its product
            uint32_t& gs = w ? g1 : g0;
            ok = gs == 0 || wait_warp(C::ALIAS ? p_free(w) : s_free(w), (gs - 1) & 1);
            if (!ok) continue;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int kk = 0; kk < DH / 16; ++kk) {
                const uint64_t o = (uint64_t)(kk / 4) * (C::HALF >> 4) + kk % 4 * 2;
                tc_mma_f16(tmem + 128 * w, dq0 + (2 * qb + (m.two ? w : 0)) * (C::TILE >> 4) + o, dk0 + st * (C::TILE >> 4) + o,
                           idesc, kk ? 1u : 0u);
              }
              tc_commit(s_full(w));
            }
            __syncwarp();
            ++gs;
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
      PcItem m;
      for (uint32_t it = 0; take(it, m); ++it) {
        const bool mine = w == 0 || m.two || m.duo;
        // (its first and last step)
        const int first = m.duo ? m.s0 + w : m.s0, last = m.duo && ((m.s1 - 1 - first) & 1) ? m.s1 - 2 : m.s1 - 1;
        int s = m.s0;
#pragma unroll 1
        for (; s < m.s1; ++s, ++G) {
          const uint32_t st = G % C::NV;
          if (!wait_warp(v_full(st), (G / C::NV) & 1)) break;
          if (!mine || (m.duo && ((s - first) & 1))) {  // (after the wait: else it could pass the ring's round)
            if (elect_one()) mbar_arrive(v_empty(st));
            __syncwarp();
            continue;
          }
          if (s == first && io > 0 && !wait_warp(o_free(w), (io - 1) & 1)) break;
          if constexpr (!Q8) {
            // The item's last step: rows of V behind its last token, which may hold anything, become zeros (P = 0
            // times what is not finite is NaN), beside the softmax.  Tile B's warp writes the same zeros again,
            // maybe while tile A's product reads them: neither can see anything else.
            if (s == m.sp.steps - 1) {
              const int end = m.sp.pl % PC_T + 1, to = (end + a.box - 1) & -a.box;  // (blocks from there on: zeros)
#pragma unroll 1
              for (int i = end * 8 + lane; i < to * 8; i += 32)
#pragma unroll
                for (int hf = 0; hf < C::HALVES; ++hf)
                  *reinterpret_cast<uint4*>(smem + C::OFF_V + st * C::TILE + hf * C::HALF + i * 16) = make_uint4(0, 0, 0, 0);
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
            }
          }
          constexpr int PARTS = C::ALIAS ? 2 : 1;  // (the first half of the keys while the second half's P is made)
          bool ok = true;
#pragma unroll
          for (int part = 0; part < PARTS; ++part) {
            const bool end = part == PARTS - 1;
            ok = ok && wait_warp(end ? p_full(w) : p_half(w), gp & 1);
            if (!ok) continue;
            tc_fence_after();
            if (elect_one()) {
              constexpr int N = PC_T / 16 / PARTS;
              const uint32_t p = tP + part * (N * 8);
              const uint64_t v = dv0 + st * (C::TILE >> 4) + part * (N * (2048 >> 4));
#pragma unroll
              for (int kk = 0; kk < N; ++kk)
                tc_mma_f16_ts(tO, p + kk * 8, v + kk * (2048 >> 4), idesc, (s > first || part > 0 || kk > 0) ? 1u : 0u);
              if (end) {
                tc_commit(p_free(w));
                tc_commit(v_empty(st));
                if (s == last) tc_commit(o_full(w));
              }
            }
            __syncwarp();
          }
          if (!ok) break;
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
    uint32_t g = 0, io = 0, ix = 0;
    PcItem m;
    for (uint32_t it = 0; take(it, m); ++it) {
      if (w == 1 && !m.two && !m.duo) {
        // (else it could pass the other warps by a round)
        if (!wait_warp(q_full(it % C::NQ), (it / C::NQ) & 1)) break;
        mbar_arrive_warp(q_empty(it % C::NQ));
        continue;
      }
      const int mate = m.two ? w * a.geo.tpt : 0;  // the tile's first token in the item
      const int pos = m.sp.pf + mate + tok;        // row of the token in its sequence
      // tiles with keys hidden from some row of this tile: past the first one's diagonal, or
      // before the last one's window
      const int diag = m.sp.pf + mate;
      const int edge = a.geo.W > 0 ? diag + a.geo.tpt - a.geo.W : -0x7fffffff;
      float mref = -INFINITY, l = 0.f;
      // a warp without a row of the item's hands its steps on as they are: its rows of P and O go nowhere
      const int toks = m.two && w ? m.toks - a.geo.tpt : min(m.toks, a.geo.tpt);
      const bool idle = q4 * 32 >= toks * a.geo.g;
      // The maximum mt of a step's scores (log2 units) against the reference: the first keys set it,
      // later ones raise it only by more than PC_RESCALE, scaling O and the running sum.
      auto raise = [&](float mt) -> bool {
        if (!__any_sync(0xffffffffu, mt > mref + PC_RESCALE)) return true;
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
        return true;
      };
      // P = 2^(s * sl2 - m) of 32 keys as bf16 pairs (key 2c, 2c + 1 in column c), and their sums, with
      // packed fp32x2 arithmetic
      auto probabilities = [&](const uint32_t* sc, float2 nm, float2* ps, uint32_t* pk) {
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          const float2 z =
              __ffma2_rn(make_float2(__uint_as_float(sc[2 * c]), __uint_as_float(sc[2 * c + 1])), sl, nm);
          const float2 pp = make_float2(ex2_approx(z.x), ex2_approx(z.y));
          ps[c & 1] = __fadd2_rn(ps[c & 1], pp);
          pk[c] = pack_bf16(pp.x, pp.y);
        }
      };
      // a step whose keys every row sees: the scores in registers
      auto step = [&]() -> bool {
        if (!wait_warp(s_full(w), g & 1)) return false;
        tc_fence_after();
        // the first half's maxima while the second half comes
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
        if (!C::ALIAS) {  // the next scores may replace them
          tc_fence_before();
          mbar_arrive_warp(s_free(w));
        }
        maxima(PC_T / 2);
        if (!raise(max3f(max3f(mx[0], mx[1], mx[2]), max3f(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * a.sl2))
          return false;
        const float ref = mref == -INFINITY ? 0.f : mref;
        const float2 nm = make_float2(-ref, -ref);
        float2 ps[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        uint32_t pk[PC_T / 2];
#pragma unroll
        for (int hh = 0; hh < PC_T / 32; ++hh) {
          probabilities(sc + 32 * hh, nm, ps, pk + 16 * hh);
          if (C::ALIAS) {
            tmem_st16(tp + 16 * hh, pk + 16 * hh);
            if (hh == 1) {
              tmem_wait_st();
              tc_fence_before();
              mbar_arrive_warp(p_half(w));
            }
          } else if (hh >= 2) {
            if (hh == 2) {  // the last tile's P has been consumed (ALIAS: before its S came)
              if (g > 0 && !wait_warp(p_free(w), (g - 1) & 1)) return false;
              tc_fence_after();
            }
#pragma unroll
            for (int c = hh == 2 ? 0 : 16 * hh; c <= 16 * hh; c += 16) tmem_st16(tp + c, pk + c);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive_warp(p_full(w));
        l += (ps[0].x + ps[0].y) + (ps[1].x + ps[1].y);
        ++g;
        return true;
      };
      // any step, 32 keys at a time, from TMEM twice: a quarter of the instructions, all of which a
      // kernel's first steps wait for (they come from L2 at some 15 cycles each).  (The next 32 fetched
      // ahead of their turn: quantised prompts 194 us where 169 were.)
      auto step_short = [&](int kt) -> bool {
        if (!wait_warp(s_full(w), g & 1)) return false;
        tc_fence_after();
        const bool masked = kt * PC_T + PC_T - 1 > diag || kt * PC_T < edge;
        uint32_t sc[32];
        auto scores = [&](int c0) {
          tmem_ld32_async(ts + c0, sc);
          tmem_wait_ld(sc);
          if (masked) {
            // seen keys: (pos - W, pos], and the sinks; bit c of a word: its column c
            auto low = [](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };
            const int b0 = kt * PC_T + c0;
            uint32_t vis = low(pos + 1 - b0);
            if (a.geo.W > 0) vis &= ~low(pos - a.geo.W + 1 - b0) | low(a.geo.S - b0);
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!(vis >> c & 1)) sc[c] = 0xff800000u;  // -inf
          }
        };
        float mt = -INFINITY;
#pragma unroll 1
        for (int c0 = 0; c0 < PC_T; c0 += 32) {
          scores(c0);
          float mx[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            mx[e] = max3f(__uint_as_float(sc[8 * e]), __uint_as_float(sc[8 * e + 1]), __uint_as_float(sc[8 * e + 2]));
#pragma unroll
            for (int c = 3; c < 7; c += 2)
              mx[e] = max3f(mx[e], __uint_as_float(sc[8 * e + c]), __uint_as_float(sc[8 * e + c + 1]));
            mx[e] = fmaxf(mx[e], __uint_as_float(sc[8 * e + 7]));
          }
          mt = max3f(mt, max3f(mx[0], mx[1], mx[2]), mx[3]);
        }
        if (!raise(mt * a.sl2)) return false;
        if (!C::ALIAS && g > 0 && !wait_warp(p_free(w), (g - 1) & 1)) return false;
        tc_fence_after();
        const float ref = mref == -INFINITY ? 0.f : mref;
        const float2 nm = make_float2(-ref, -ref);
        float2 ps[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
        for (int c0 = 0; c0 < PC_T; c0 += 32) {
          scores(c0);
          uint32_t pk[16];
          probabilities(sc, nm, ps, pk);
          tmem_st16(tp + c0 / 2, pk);
          if (C::ALIAS && c0 == 32) {
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive_warp(p_half(w));
          }
        }
        tmem_wait_st();
        tc_fence_before();
        if (!C::ALIAS) mbar_arrive_warp(s_free(w));
        mbar_arrive_warp(p_full(w));
        l += (ps[0].x + ps[0].y) + (ps[1].x + ps[1].y);
        ++g;
        return true;
      };
      const int by = m.duo ? 2 : 1;
#pragma unroll 1
      for (int s = m.duo ? m.s0 + w : m.s0; ok && s < m.s1; s += by) {
        if (idle) {
          // (not ALIAS: the next scores may come before the last P has, which must be all four warps' first)
          ok = wait_warp(s_full(w), g & 1) && (C::ALIAS || g == 0 || wait_warp(p_free(w), (g - 1) & 1));
          if (!ok) break;
          ++g;
          mbar_arrive_warp(C::ALIAS ? p_half(w) : s_free(w));
          mbar_arrive_warp(p_full(w));
          continue;
        }
        const int kt = m.sp.tile(s);
        if constexpr (Q8)
          ok = step_short(kt);
        else
          ok = !m.two || m.s1 - m.s0 < a.long_item || kt * PC_T + PC_T - 1 > diag || kt * PC_T < edge ? step_short(kt) : step();
      }
      if (!ok) break;
      // the item's O: after its last P V
      if (!wait_warp(o_full(w), io & 1)) break;
      ++io;
      tc_fence_after();
      // shared steps: tile B's place hands its (maximum, sum) and its O, in two halves, to A's
      // through the second query tile's memory, which such an item does not use
      constexpr int XC = DH / 2;  // columns of a half: so many rows of 128 float4s
      const uint32_t qb = it % C::NQ;
      float4* const xch = reinterpret_cast<float4*>(smem + (2 * qb + 1) * C::TILE);
      if (m.duo && w == 1) {
        ok = wait_warp(x_free, (ix & 1) ^ 1);
        if (!ok) break;
        if (!idle) xch[r] = make_float4(mref, l, 0.f, 0.f);
        mbar_arrive_warp(x_full);
        ++ix;
#pragma unroll 1
        for (int c0 = 0; ok && c0 < DH; c0 += XC, ++ix) {
          ok = wait_warp(x_free, (ix & 1) ^ 1);
          if (!ok) break;
#pragma unroll 1
          for (int c = 0; c < XC && !idle; c += 32) {
            uint32_t ov[32];
            tmem_ld32_async(to + c0 + c, ov);
            tmem_wait_ld(ov);
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              xch[(c + i) / 4 * PC_T + r] = make_float4(__uint_as_float(ov[i]), __uint_as_float(ov[i + 1]),
                                                        __uint_as_float(ov[i + 2]), __uint_as_float(ov[i + 3]));
          }
          mbar_arrive_warp(x_full);
        }
        if (!ok) break;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        mbar_arrive_warp(o_free(w));
        mbar_arrive_warp(q_empty(qb));
        continue;
      }
      float fa = 1.f, fb = 0.f;  // factors of A's own and of B's
      if (m.duo) {
        ok = wait_warp(x_full, ix & 1);
        if (!ok) break;
        const float4 y = xch[r];
        mbar_arrive_warp(x_free);
        ++ix;
        const float M = fmaxf(mref, y.x);
        fa = mref == M ? 1.f : ex2_approx(mref - M);
        fb = y.x == M ? 1.f : ex2_approx(y.x - M);
        l = fmaf(l, fa, y.y * fb);
        mref = M;
      }
      const bool row_in = tok < toks;
      const float inv = m.whole ? C::SCALE / l : 1.f;  // (a row sees itself: 0 where its scores are all -inf, and 0 / 0 is NaN)
      const long place = m.place;
      float4* const part = a.part + (place * (DH / 4)) * a.piece_rows + w * PC_T + r;
      float2 fin = make_float2(0.f, 0.f);  // zero, but for sums that are not finite
#pragma unroll 1
      for (int c = 0; c < DH; c += 32) {
        if (idle) {
          if (m.duo && c % XC == 0) {
            ok = wait_warp(x_full, ix & 1);
            if (!ok) break;
            mbar_arrive_warp(x_free);
            ++ix;
          }
          continue;
        }
        uint32_t ov[32];
        tmem_ld32_async(to + c, ov);
        tmem_wait_ld(ov);
        if (m.duo) {
          if (c % XC == 0) ok = wait_warp(x_full, ix & 1);
          if (!ok) break;
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 y = xch[(c % XC + i) / 4 * PC_T + r];
            ov[i] = __float_as_uint(fmaf(__uint_as_float(ov[i]), fa, y.x * fb));
            ov[i + 1] = __float_as_uint(fmaf(__uint_as_float(ov[i + 1]), fa, y.y * fb));
            ov[i + 2] = __float_as_uint(fmaf(__uint_as_float(ov[i + 2]), fa, y.z * fb));
            ov[i + 3] = __float_as_uint(fmaf(__uint_as_float(ov[i + 3]), fa, y.w * fb));
          }
          if (c % XC == XC - 32) {
            mbar_arrive_warp(x_free);
            ++ix;
          }
        }
        if (m.whole) {
          // the warp's rows through the query tile's own, which no MMA reads any more
          uint8_t* stg = smem + (2 * qb + w) * C::TILE + c / 64 * C::HALF + r * 128;
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
        } else if (row_in) {
          // (four columns of a row, row by row: a lane to a row writes lines, not a piece of 32 of them)
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            part[(c + i) / 4 * a.piece_rows] = make_float4(__uint_as_float(ov[i]), __uint_as_float(ov[i + 1]),
                                                           __uint_as_float(ov[i + 2]), __uint_as_float(ov[i + 3]));
        }
      }
      if (!ok) break;
      tc_fence_before();
      mbar_arrive_warp(o_free(w));
      if (m.whole && !idle) {
        late |= fin.x + fin.y != 0.f && row_in;
        bf16* const row = row_in ? a.out + (long)(m.t0 + w * a.geo.tpt + tok) * a.ldo +
                                       ((long)m.h * a.geo.g + r % a.geo.g) * DH
                                 : nullptr;
        constexpr int CH = DH / 8;  // 16-byte pieces of a row
#pragma unroll 4
        for (int i = 0; i < CH; ++i) {
          const int e = i * 32 + lane, rr = e / CH, c = e % CH;
          bf16* const dst = reinterpret_cast<bf16*>(__shfl_sync(0xffffffffu, (unsigned long long)row, rr));
          const uint4 u = *reinterpret_cast<const uint4*>(smem + (2 * qb + w) * C::TILE + c / 8 * C::HALF + (q4 * 32 + rr) * 128 +
                                                          (((c % 8) ^ (rr & 7)) << 4));
          if (dst) *reinterpret_cast<uint4*>(dst + c * 8) = u;
        }
      } else if (row_in) {
        a.ml[place * a.piece_rows + w * PC_T + r] = make_float2(mref, l);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive_warp(q_empty(qb));
    }
    if (__any_sync(0xffffffffu, late)) {
      __syncwarp();
      PcWalk walk(a, ends);
      for (;;) {
        walk.next(a, m);
        if (m.s1 == 0) break;
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
          pc_repair<DH, Q8>(a, m.b, m.h, __shfl_sync(0xffffffffu, hq, src), __shfl_sync(0xffffffffu, t, src),
                            __shfl_sync(0xffffffffu, m.sp.pf + w * a.geo.tpt + tok, src), m.sp.pf, m.sp.pl);
        }
      }
    }
  } else if constexpr (Q8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_CTRL));
    // ------------------------------------------------------------ bytes to bf16
    constexpr int LPR = DH / 16, RPW = 32 / LPR;  // lanes of a row, rows of a warp's load
    constexpr int NR = C::NR ? C::NR / 2 : 1;
    const int c = lane % LPR, sub = lane / LPR;
    bool ok = true;
    uint32_t G = 0;  // steps so far
    PcItem m;
    for (uint32_t it = 0; ok && take(it, m); ++it) {
#pragma unroll 1
      for (int s = m.s0; s < m.s1 && ok; ++s, ++G) {
        const int end = s == m.sp.steps - 1 ? m.sp.pl % PC_T + 1 : PC_T;  // rows behind the last token: any finite ones
#pragma unroll 1
        for (int kv = 0; kv < 2; ++kv) {
          const uint32_t n = kv ? C::NV : C::NK, st = kv * NR + G % NR, dst = G % n;
          const uint32_t full = kv ? v_full(dst) : k_full(dst), empty = kv ? v_empty(dst) : k_empty(dst);
          const bool e = mbar_test_wait(empty, ((G / n) & 1) ^ 1), f = mbar_test_wait(r_full(st), (G / NR) & 1);
          if (!__all_sync(0xffffffffu, e && f))  // (mostly both have)
            ok = mbar_wait_warp(empty, ((G / n) & 1) ^ 1) && mbar_wait_warp(r_full(st), (G / NR) & 1);
          if (!ok) break;
          const uint8_t* raw = smem + C::OFF_RAW + st * C::RAW;
          const signed char* ex = reinterpret_cast<const signed char*>(smem + C::OFF_EXP + st * PC_T);
          uint8_t* tile = smem + (kv ? C::OFF_V : C::OFF_K) + dst * C::TILE;
          constexpr int TURNS = PC_T / (C::CONV * RPW), U = 2;  // rows of a lane; at a time (all four: 60.4 us where two take 58)
          static_assert(TURNS * C::CONV * RPW == PC_T && TURNS % U == 0, "each row once");
          uint8_t* const o0 = tile + (c / 4) * C::HALF;
          const int p = c % 4 * 2, flip = c / 4;  // (lanes of the second half write their pieces the other way round)
#pragma unroll 1
          for (int i = 0; i < TURNS; i += U) {
            uint4 u[U];
            int e[U];
            bool small = true;
#pragma unroll
            for (int k = 0; k < U; ++k) {
              const int row = ((i + k) * C::CONV + warp - 12) * RPW + sub;
              u[k] = *reinterpret_cast<const uint4*>(raw + row * DH + c * 16);
              e[k] = row < end ? ex[row] : 0;
              small &= pq_small(e[k]);
            }
            auto put = [&](int k, uint2 v0, uint2 v1, uint2 v2, uint2 v3) {
              const int row = ((i + k) * C::CONV + warp - 12) * RPW + sub;
              const uint4 lo = make_uint4(v0.x, v0.y, v1.x, v1.y), hi = make_uint4(v2.x, v2.y, v3.x, v3.y);
              uint8_t* const o = o0 + row * 128;
              *reinterpret_cast<uint4*>(o + (((p + flip) ^ (row & 7)) << 4)) = flip ? hi : lo;
              *reinterpret_cast<uint4*>(o + (((p + 1 - flip) ^ (row & 7)) << 4)) = flip ? lo : hi;
            };
            if (__all_sync(0xffffffffu, small)) {
#pragma unroll
              for (int k = 0; k < U; ++k) {
                const uint32_t f = pq_factor(e[k]), b = pq_offset(e[k]);
                put(k, pq_down(u[k].x, f, b), pq_down(u[k].y, f, b), pq_down(u[k].z, f, b), pq_down(u[k].w, f, b));
              }
            } else {
#pragma unroll
              for (int k = 0; k < U; ++k) {
                // (of the least exponents 2^(e - PQ_DOWN) is no fp32 number: in two factors.  Rows that hold
                // nothing yet may have exponents past the largest, whose shift is an infinity: what no token
                // sees must be finite, or P = 0 makes NaN of it)
                const int x = min(e[k], PQ_TOP);
                const float f = pq_scale(x == PQ_NAN ? x : max(x - PQ_DOWN, PQ_LOW)), b = pq_shift(f);
                const uint32_t g = pq_twice(min(x - PQ_DOWN - PQ_LOW, 0));
                const float2 ff = make_float2(f, f), bb = make_float2(b, b);
                put(k, pq_times(pq_values(u[k].x, ff, bb), g), pq_times(pq_values(u[k].y, ff, bb), g),
                    pq_times(pq_values(u[k].z, ff, bb), g), pq_times(pq_values(u[k].w, ff, bb), g));
              }
            }
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
        for (uint32_t i = r_issued > C::NR ? r_issued - C::NR : 0; i < r_issued; ++i) {
          constexpr int N = C::NR ? C::NR / 2 : 1;
          mbar_wait_drain(r_full((i & 1) * N + i / 2 % N), (i / 2 / N) & 1);
        }
      for (uint32_t i = q_issued > C::NQ ? q_issued - C::NQ : 0; i < q_issued; ++i)
        mbar_wait_drain(q_full(i % C::NQ), (i / C::NQ) & 1);
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
  // rows of sequences whose length cannot be
  for (int b = any_bad ? blockIdx.x : a.geo.B; b < a.geo.B; b += gridDim.x) {
    bool bad;
    const PcSeq q = pc_seq(a, b, &bad);
    const int per = a.geo.KV * a.geo.g * (DH / 8);
    if (bad)
      for (long i = threadIdx.x; i < (long)q.n * per; i += C::THREADS)
        *reinterpret_cast<uint4*>(a.out + (q.t0 + i / per) * a.ldo + i % per * 8) = make_uint4(0, 0, 0, 0);
  }
}

// Items that lie on several CTAs: the pieces joined in the order of the CTAs.  CTA x takes the item
// that begins on CTA x and ends on a later one; CTAs y take 32 of its rows each, a lane to a row and
// the columns four by four to the warps, U such groups each, N pieces at a time.
// FEW: a call of few items, each of eight pieces or more: CTA x takes the x-th such item, and CTAs z share
// its columns out.  (8 tokens on 30000 rows, 16 heads on 2 of 128: 32 us so, 37 otherwise; three short
// sequences 12.0 and 12.8; 8 x 4 tokens on 2000 rows, 4 heads of 64, more items: 19.2 and 17.1.)
constexpr int PJ_WARPS = 8;
template <int DH, bool Q8, bool FEW>
__global__ void __launch_bounds__(32 * PJ_WARPS) paged_chunk_join_kernel(const __grid_constant__ PcArgs a) {
  constexpr int C4 = DH / 4;  // groups of four columns
  constexpr int U = FEW ? 1 : C4 / PJ_WARPS, N = FEW ? 8 : 2;
  __shared__ uint32_t again;
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = FEW ? blockIdx.z : 0,
            c4 = (part * PJ_WARPS + warp) * U;
  auto same = [](const PcAt& p, const PcAt& m) { return p.b == m.b && p.h == m.h && p.u == m.u; };
  // whether an item begins on CTA k and ends on a later one
  auto cut = [&](const PcAt& begin, const PcAt& next) { return next.s > 0 && !(same(begin, next) && begin.s > 0); };
  int x = blockIdx.x;
  if (FEW) {
    int left = x;
    uint32_t in = 0;
    int k = -32;
    do {
      left -= __popc(in);
      k += 32;
      if (k >= a.G) return;
      in = __ballot_sync(0xffffffffu, k + lane < a.G && cut(a.at[min(k + lane, a.G)], a.at[min(k + lane + 1, a.G)]));
    } while (left >= __popc(in));
    for (; left > 0; --left) in &= in - 1;
    x = k + __ffs(in) - 1;
  }
  const PcAt m = a.at[x + 1], begin = a.at[x];
  if (!cut(begin, m)) return;
  const PcSeq q = pc_seq(a, m.b);
  const PcSpan sp = pc_span(a.geo, q, m.u);
  const int R = 2 * a.geo.tpt, toks = min(q.n - m.u * R, R), g = a.geo.g;
  const int rr = blockIdx.y * 32 + lane, w = rr / PC_T, tok = w * a.geo.tpt + rr % PC_T / g;
  const bool row_in = rr % PC_T < a.geo.tpt * g && tok < toks;
  if (!__any_sync(0xffffffffu, row_in)) return;  // (the same for all warps)
  if (threadIdx.x == 0) again = 0;
  __syncthreads();
  int n = 1;  // this CTA and those that begin inside the item (a.at[a.G] is the line's end)
  for (uint32_t in = ~0u; in == ~0u; n += __popc(in)) {
    const int k = x + n + lane;
    bool is = k <= a.G;
    if (is) {
      const PcAt p = a.at[k];
      is = same(p, m) && p.s > 0;
    }
    in = __ballot_sync(0xffffffffu, is);
  }
  const int first = same(begin, m) ? 0 : 1;  // piece 0 is the last of its CTA's, the others the first
  float4 acc[U] = {};
  float M = -INFINITY, L = 0.f;
#pragma unroll 1
  for (int k0 = 0; k0 < n; k0 += 32) {
    // the CTAs x + k that hold a piece: one may begin where the next one does
    const int kl = k0 + lane;
    const bool holds = kl < n && (kl == 0 || kl == n - 1 || a.at[x + kl + 1].s != a.at[x + kl].s);
    uint32_t pieces = __ballot_sync(0xffffffffu, holds);
    if (!row_in) continue;
    // what is summed so far is brought down to the largest maximum
#pragma unroll 1
    while (pieces) {
      float2 y[N];
      float4 v[N][U];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int k = k0 + __ffs(pieces) - 1;
        y[e] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) v[e][u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (pieces) {
          const long place = 2l * (x + k) + (k == 0 ? first : 0);
          const float4* p = a.part + (place * C4 + c4) * a.piece_rows + rr;
          y[e] = a.ml[place * a.piece_rows + rr];
#pragma unroll
          for (int u = 0; u < U; ++u) v[e][u] = p[u * a.piece_rows];
          pieces &= pieces - 1;
        }
      }
      float next = M;
#pragma unroll
      for (int e = 0; e < N; ++e) next = fmaxf(next, y[e].x);
      auto factor = [&](float m) { return m == next ? 1.f : ex2_approx(m - next); };  // (-inf, no keys at all: 1 of nothing)
      const float f = factor(M);
      M = next;
      float fe[N];
#pragma unroll
      for (int e = 0; e < N; ++e) fe[e] = factor(y[e].x);
      auto sum = [&](auto of, float before) {  // the last first
        float t = of(N - 1) * fe[N - 1];
#pragma unroll
        for (int e = N - 2; e >= 0; --e) t = fmaf(of(e), fe[e], t);
        return fmaf(before, f, t);
      };
      L = sum([&](int e) { return y[e].y; }, L);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        acc[u].x = sum([&](int e) { return v[e][u].x; }, acc[u].x);
        acc[u].y = sum([&](int e) { return v[e][u].y; }, acc[u].y);
        acc[u].z = sum([&](int e) { return v[e][u].z; }, acc[u].z);
        acc[u].w = sum([&](int e) { return v[e][u].w; }, acc[u].w);
      }
    }
  }
  const int t = q.t0 + m.u * R + tok, hq = m.h * g + rr % PC_T % g;
  if (row_in) {
    const float inv = PcCfg<DH, Q8>::SCALE / L;
    bf16* o = a.out + t * a.ldo + (long)hq * DH + c4 * 4;
    float fin = 0.f;  // zero, but for sums that are not finite
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float4 v = make_float4(acc[u].x * inv, acc[u].y * inv, acc[u].z * inv, acc[u].w * inv);
      fin = fmaf(v.x, 0.f, fmaf(v.y, 0.f, fmaf(v.z, 0.f, fmaf(v.w, 0.f, fin))));
      *reinterpret_cast<uint2*>(o + 4 * u) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    }
    if (fin != 0.f) atomicOr(&again, 1u << lane);
  }
  __syncthreads();
  uint32_t mask = again;
  constexpr int COLS = 4 * PJ_WARPS * U;  // of the CTA
  for (int i = 0; mask; ++i, mask &= mask - 1) {
    if (i % PJ_WARPS != warp) continue;
    const int src = __ffs(mask) - 1;
    pc_repair<DH, Q8>(a, m.b, m.h, __shfl_sync(0xffffffffu, hq, src), __shfl_sync(0xffffffffu, t, src),
                      __shfl_sync(0xffffffffu, sp.pf + tok, src), sp.pf, sp.pl, part * COLS, (part + 1) * COLS);
  }
}

struct PcPlan {
  int tpt, G, piece_rows;
  bool split;
  long items;  // at most
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
  p.items = items;
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
  static KernelOnce once[2];
  const auto kern = a.stop < 0 ? paged_chunk_kernel<DH, Q8, false> : paged_chunk_kernel<DH, Q8, true>;
  cudaError_t e = once[a.stop >= 0](reinterpret_cast<const void*>(kern), C::SMEM, C::THREADS, C::POOL);
  if (e != cudaSuccess) return e;
  // work: upper bound (every cache full, all rows of the longest)
  const double keys = (double)std::min<long>((long)c.max_pages * c.page, 0x7fffffffL);
  {
    LaunchTimer lt("paged_chunk", st, 4.0 * a.rows * c.H * DH * keys,
                   (double)c.B * c.KV * keys * DH * (Q8 ? 2.0 : 4.0) + 4.0 * a.rows * c.H * DH);
    e = launch_kernel(kern, a.G, C::THREADS, C::SMEM, st, tq, tk, tv, a);
    if (e != cudaSuccess || !p.split) return e;
  }
  LaunchTimer lt("paged_chunk_join", st, 0.0, 8.0 * a.G * p.piece_rows * DH);
  const int y = p.piece_rows / 32, z = DH / 4 / PJ_WARPS;
  if (8 * p.items <= PC_CTAS && p.items * y * z <= 3 * PC_CTAS)
    return launch_kernel(paged_chunk_join_kernel<DH, Q8, true>, dim3(p.items, y, z), 32 * PJ_WARPS, 0, st, a);
  return launch_kernel(paged_chunk_join_kernel<DH, Q8, false>, dim3(a.G, y), 32 * PJ_WARPS, 0, st, a);
}

}  // namespace

static_assert(PC_MAX_B == PF_PAGED_MAX_BATCH, "limit of the entry points");

size_t paged_chunk_ws_bytes(const Paged& c, long rows) { return rows > 0 ? pc_plan(c, rows).bytes : 0; }

cudaError_t paged_chunk(const Paged& c, long rows, const bf16* q, long ldq, const int* start, bf16* out, long ldo,
                        void* ws, cudaStream_t st) {
  launched.mark();
  const PcPlan p = pc_plan(c, rows);
  PcArgs a{};
  // (no sequence is as long as the widest windows: none, and sums with it stay within an int)
  a.geo = {c.B, c.KV, c.H / c.KV, p.tpt, c.window < PC_LONGEST ? c.window : 0, c.sinks};
  a.start = start; a.len = c.len; a.table = c.table;
  a.rows = rows;
  a.page = c.page; a.max_pages = c.max_pages;
  a.n_pages = c.n_pages;
  a.box = std::min(PC_T, c.page & -c.page);
  while (1 << a.box_log < a.box) ++a.box_log;
  a.step_pages = PC_T / c.page;
  a.step_rows = PC_T % c.page;
  a.G = p.G;
  // About a step and a half (three short sequences, up to 7 tokens on 1000 rows: 12.9 us so, 13.2 at 150, 16.2
  // at 1000).  Steps in the long form: 2048 tokens on 30000 rows 339 us so, 400 in the short one; sixteen prompts
  // of up to 1000 tokens, 16 heads on 8 of 64, 55.5 us so, 57.2 with all items' in the long one.
  a.few = 400;
  a.long_item = 8;
  a.stop = stop_after.load(std::memory_order_relaxed);
  a.sl2 = (c.Ke ? 1 << PQ_DOWN : 1) * 1.4426950408889634f / sqrtf((float)c.dh);
  a.q = q; a.ldq = ldq;
  a.out = out; a.ldo = ldo;
  a.K = c.K; a.V = c.V; a.Ke = c.Ke; a.Ve = c.Ve;
  if (p.split) {
    char* w = static_cast<char*>(ws);
    a.at = reinterpret_cast<PcAt*>(w + p.at);
    a.ml = reinterpret_cast<float2*>(w + p.ml);
    a.part = reinterpret_cast<float4*>(w + p.bytes) - 2 * (size_t)p.G * p.piece_rows * (c.dh / 4);
  }
  a.piece_rows = p.piece_rows;
  if (c.Ke) return c.dh == 128 ? pc_launch<128, true>(c, a, p, st) : pc_launch<64, true>(c, a, p, st);
  return c.dh == 128 ? pc_launch<128, false>(c, a, p, st) : pc_launch<64, false>(c, a, p, st);
}

}  // namespace pf

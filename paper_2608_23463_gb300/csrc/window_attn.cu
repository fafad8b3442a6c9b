// Causal attention in a sliding window with sinks, forward, on the
// 5th-generation tensor cores: tcgen05.mma with TMEM accumulators, TMA tiles,
// head width 64, grouped heads.
//
//   o_i = sum_j softmax_j(q_i . k_j / 8) v_j  over the keys
//   j <= i with i - j < W or j < S   (W: window, S: sinks)
//
// Work item = (two consecutive 128-query tiles A and B, query head, sequence);
// one persistent CTA per SM walks the items.  An item's key tiles are the
// sinks' [0, ns) and the window's [lo, hi], without those in between: its work
// is that of the window, whatever the length.  A tile takes no part in key
// tiles of its neighbour's that it does not see.
//   warp 0    TMA producer: the item's two Q tiles (double-buffered across
//             items) and a WA_STAGES-deep ring of (K, V) 128-key tiles, shared
//             by both query tiles; rows past the end of a sequence read as zero
//   warp 1    MMA issuer of both tiles' scores: S = Q K_j^T (M=128, N=128, K=64)
//             into the tile's TMEM score buffer as soon as its last scores are
//             in registers
//   warps 2-3 MMA issuers of tile A's and tile B's O += P V_j (M=128, N=64,
//             K=128), P from TMEM
//   warps 4-7 softmax of tile A, warps 8-11 of tile B: one query row per thread
//             (TMEM lane), its 128 scores in registers; P goes back to TMEM
// What bounds it: the chain of one softmax warp through a tile (about 430
// instructions, two such warps on each scheduler), beside 1024 cycles of MMAs
// and as many of exponentials for a pair of tiles.  262144 tokens of 16 heads on
// 4, window 4096: 3.98 ms (1.11 PFLOP/s).  What shortened the chain: maxima of
// the first half of the scores while the second comes from TMEM, P stored from
// its half on, and a loop of its own for tiles without masked keys (4.50
// without the three; 4.39 with the loop alone, 4.34 with it and either).
// As it was at 4.50, with parts left out: 2.74 with no arithmetic, 4.07 without
// the maxima, 3.55 without the exponentials.  Tried then: one MMA issuer for both
// tiles, which makes each wait for the other's softmax, and key tiles tested one
// by one: 5.06; two threads to a row (sixteen softmax warps): 5.27; chunks of 64
// keys in two buffers a tile that P shares with the scores: 5.50; O read out in
// the next item's first step: 5.03.
// A sinks' tile before the window that holds WT_FEW sinks at most is worked off
// as a tile of so many keys: 65536 tokens of 16 heads, window 1024, 4 sinks 448
// us without, 422 with it; 411 with each tile's scores and O issued by one warp,
// 399 so; 366 with the rows out by TMA, for which an item's end took a fifth of it.
// Code counts, its fetches more than its instructions: masks by the bits of a word in
// place of two compares of a column (4.17 to 3.95 ms where a tile in seventeen has one; 3.98 with
// the test for rows that are not finite).
// One body for tiles with masks and tiles without them spills: 4.59.
// A row's probabilities are taken against a reference m, the maximum of the
// first tile in which the row sees a key, raised only when a later tile's
// maximum exceeds it by more than WA_RESCALE (log2 units); then O and the sum
// are scaled.  P <= 2^WA_RESCALE is rounded to bf16 for its product (relative
// 2^-8, as any value), the sums take it unrounded.  A tile may hide all of its
// keys from a row (the window's first tile, seen by the tile's first rows
// only): such a row keeps no reference and adds zeros.
// Masked scores are set to -inf after the product, so a masked K may hold
// anything.  P = 0 meets its V in the MMA: an infinity or a NaN there reaches rows
// of its 128-row tile that do not see it.  A warp remembers that a row of its own
// was not finite, and goes through its items again at the end (wa_repair).
#include <algorithm>
#include <type_traits>

#include "local.h"
#include "window_tiles.cuh"

namespace pf {

static Launched launched;
int take_dev_error_window_attn() { return launched.take(take_dev_error_tu); }
int set_wait_limit_window_attn(unsigned long long ns) { return set_wait_limit_tu(ns); }

namespace {

constexpr int WA_D = 64;  // head width
constexpr int WA_STAGES = 4;
constexpr int WA_THREADS = 384;  // producer, three MMA issuers, two groups of four
// A softmax thread holds a row's 128 scores: the control warps give registers up, of the
// 168 that each thread has at launch.
constexpr int WA_REGS_CTRL = 88, WA_REGS_ROWS = 208;
static_assert(WA_REGS_CTRL * 128 + WA_REGS_ROWS * 256 == 168 * WA_THREADS, "register split");
constexpr float WA_RESCALE = 8.f;
constexpr uint32_t WA_T_BYTES = WT * WA_D * 2;  // 16 KB: a Q, K or V tile
constexpr uint32_t WA_OFF_KV = 4 * WA_T_BYTES;  // Q: [2 items][tiles A, B]
constexpr uint32_t WA_OFF_STG = WA_OFF_KV + WA_STAGES * 2 * WA_T_BYTES;  // a softmax warp's 32 output rows
constexpr uint32_t WA_OFF_BAR = WA_OFF_STG + 8 * 32 * WA_D * 2;
constexpr uint32_t WA_SMEM = WA_OFF_BAR + 512 + 1024;
static_assert(WA_SMEM <= 227 * 1024, "shared memory");
// TMEM columns of tile w: scores S at 128 w (fp32), O at 256 + 64 w (fp32), P at
// 384 + 64 w (bf16 pairs: key 2c in the low half of column c)
constexpr uint32_t WA_TMEM_COLS = 512;
constexpr uint32_t WA_TM_O = 256, WA_TM_P = 384;

struct WaArgs {
  float* lse;  // [B, H, L] in log2 units, or null
  int B, H, g;  // g: query heads to a key head
  WinTiles w;
  int n_st, n_items;  // tile pairs
  float sl2;          // log2(e) / sqrt(64)
  // as wa_repair reads and writes them
  const bf16 *q, *k, *v;
  bf16 *out, *rest;
  long ldq, ldk, ldv, ldo;
};

// Items are ranked from the last tile pair on (the first ones see the fewest
// keys); CTA c takes rank c of round 0, rank G-1-c of round 1, and so on.
__device__ __forceinline__ int wa_rank(int c, int round) {
  return round * (int)gridDim.x + ((round & 1) ? (int)gridDim.x - 1 - c : c);
}

// Item k: tile pair, head, sequence and the key tiles of both query tiles
// together: step j's is j < ns ? j : lo + j - ns; n of them.
struct WaItem {
  int u, h, b, ns, lo, n;
  __device__ __forceinline__ WaItem(const WaArgs& a, int k) {
    const int per = a.H * a.B;
    u = a.n_st - 1 - k / per;
    const int r = k % per;
    h = r % a.H;
    b = r / a.H;
    lo = a.w.lo(2 * u);
    ns = min(a.w.sT, lo);
    n = ns + min(2 * u + 1, a.w.n_t - 1) - lo + 1;
  }
  __device__ __forceinline__ int tile(int j) const { return j < ns ? j : lo + j - ns; }
};

// The steps of an item that query tile t takes part in: [0, a0) and [a1, a2).  Tile B
// may have left key tiles behind that A's window still holds, and A does not reach
// B's diagonal.
struct WaSteps {
  int a0, a1, a2;
  int few;  // the step of the few sinks' tile, or -1
  __device__ __forceinline__ WaSteps(const WaArgs& a, const WaItem& m, int t) {
    const int gap = max(m.lo, a.w.sT);  // first tile that only the window can show
    a1 = m.ns + max(a.w.lo(t) - m.lo, 0);
    a0 = min(m.ns + gap - m.lo, a1);
    a2 = t < a.w.n_t ? m.ns + t - m.lo + 1 : 0;
    if (t >= a.w.n_t) a0 = a1 = 0;
    few = a.w.few >= a.w.lo(t) ? -1 : a.w.few < m.ns ? a.w.few : m.ns + a.w.few - m.lo;
  }
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

// Whether one of the rows [r0, r1) of v (a head of a sequence) holds a value that is not
// finite.  For a converged warp.
__device__ __forceinline__ bool wa_not_finite(const bf16* v, long ldv, int r0, int r1) {
  const int lane = threadIdx.x & 31;
  bool bad = false;
  for (int r = r0 + (lane >> 3); r < r1; r += 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(v + r * ldv + (lane & 7) * 8);
    for (uint32_t w : {u.x, u.y, u.z, u.w}) bad |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
  }
  return __any_sync(0xffffffffu, bad);
}

// Columns 2 lane, 2 lane + 1 of row i's output, from the keys that it sees and no others.
// q: the row; k, v: its head and sequence.  For a converged warp: a key to a lane for the
// scores, two columns to a lane for the sums.
__device__ __forceinline__ float2 wa_row(const WaArgs& a, const bf16* q, const bf16* k, const bf16* v, int i) {
  const int lane = threadIdx.x & 31, lo = max(0, i - a.w.W + 1);
  float2 acc = make_float2(0.f, 0.f);
  float m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {  // the sinks before the window, the window
    const int end = part ? i + 1 : min(a.w.S, lo);
#pragma unroll 1
    for (int j = part ? lo : 0; j < end; j += 32) {
      const bool in = j + lane < end;
      float s = -INFINITY;
      if (in) {
        s = 0.f;
#pragma unroll 2
        for (int c = 0; c < WA_D; c += 8) {
          float x[8], y[8];
          load8_bf16(q + c, x);
          load8_bf16(k + (j + lane) * a.ldk + c, y);
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
        }
      }
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
      acc.x *= corr;
      acc.y *= corr;
#pragma unroll 8
      for (int t = 0; t < min(32, end - j); ++t) {
        const float pt = __shfl_sync(0xffffffffu, p, t);
        const float2 y = unpack_bf16(*reinterpret_cast<const uint32_t*>(v + (j + t) * a.ldv + 2 * lane));
        acc.x = fmaf(pt, y.x, acc.x);
        acc.y = fmaf(pt, y.y, acc.y);
      }
      // NaN for good, whatever follows
      if (__all_sync(0xffffffffu, acc.x != acc.x && acc.y != acc.y)) return acc;
    }
  }
  return make_float2(acc.x / l, acc.y / l);
}

// Rows that came out other than finite beside hidden rows of v that are not: in the MMA P = 0
// met them.  The softmax warp goes through its items' rows in memory again and works such
// rows out from the keys that they see.  Out of line and after the loop over the items: calls
// without such rows pay 0.1 of 9.7 us (3 x 1021 tokens, window 256) and 50 of 3930 (262144
// tokens, window 4096); from inside the loop 0.4 and 140.  With them (65536 tokens of 16 heads, the
// last 100 rows NaN): 3.6 ms in place of 0.36 at window 1024, 226 in place of 7 without a window.
// The loads of more keys at once halve that, but their registers cost every call as much again.
__device__ __noinline__ void wa_repair(WaArgs a, int warp) {
  const int lane = threadIdx.x & 31, w = (warp - 4) >> 2, q4 = warp & 3;
  asm volatile("fence.proxy.async;" ::: "memory");  // the rows went out by TMA
  __syncwarp();
#pragma unroll 1
  for (int rd = 0, k = wa_rank(blockIdx.x, 0); k < a.n_items; k = wa_rank(blockIdx.x, ++rd)) {
    const WaItem m(a, k);
    const int t = 2 * m.u + w, q0 = t * WT + q4 * 32;
    const long row0 = (long)m.b * a.w.L, kc = (long)(m.h / a.g) * WA_D;
    bf16* const out = a.out + row0 * a.ldo + m.h * WA_D;
    bool bad = false;
    if (q0 + lane < a.w.L) {
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < WA_D; c += 8) {
        const uint4 u = __ldcg(reinterpret_cast<const uint4*>(out + (q0 + lane) * a.ldo + c));
        for (uint32_t x : {u.x, u.y, u.z, u.w}) sum = fmaf(unpack_bf16(x).x, 0.f, fmaf(unpack_bf16(x).y, 0.f, sum));
      }
      bad = sum != 0.f;
    }
    uint32_t again = __ballot_sync(0xffffffffu, bad);
    if (!again) continue;
    // rows of v that its tiles hold and some of the warp's rows do not see: past the diagonal,
    // before the window, beside the sinks
    const bf16 *kp = a.k + row0 * a.ldk + kc, *vp = a.v + row0 * a.ldv + kc;
    const int lo = a.w.lo(t), ns = min(a.w.sT, lo);
    const int held = ns < a.w.sT ? 0 : a.w.few >= 0 ? a.w.few * WT + WT_FEW : ns * WT;
    if (!wa_not_finite(vp, a.ldv, q0 + 1, min(t * WT + WT, a.w.L)) &&
        !wa_not_finite(vp, a.ldv, max(lo * WT, a.w.S), min(q0 + 32 - a.w.W, a.w.L)) &&
        !wa_not_finite(vp, a.ldv, a.w.S, min(held, a.w.L)))
      continue;
#pragma unroll 1
    for (; again; again &= again - 1) {
      const int i = q0 + __ffs(again) - 1;
      const float2 o = wa_row(a, a.q + (row0 + i) * a.ldq + m.h * WA_D, kp, vp, i);
      const uint32_t x = pack_bf16(o.x, o.y);
      *reinterpret_cast<uint32_t*>(out + i * a.ldo + 2 * lane) = x;
      if (a.rest) {
        const float2 y = unpack_bf16(x);
        *reinterpret_cast<uint32_t*>(a.rest + ((row0 + i) * a.H + m.h) * WA_D + 2 * lane) =
            pack_bf16(o.x - y.x, o.y - y.y);
      }
    }
  }
}

__global__ void __launch_bounds__(WA_THREADS, 1)
    window_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                      const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmO,
                      const __grid_constant__ CUtensorMap tmR, WaArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  // q_full[2] q_empty[2] kv_full[S] kv_empty[S], per tile w: s_full s_free p_full
  // p_free o_full o_free, done
  const uint32_t b0 = smem_u32(smem + WA_OFF_BAR);
  const uint32_t q_full = b0, q_empty = b0 + 16, kv_full = b0 + 32,
                 kv_empty = kv_full + 8 * WA_STAGES, grp0 = kv_empty + 8 * WA_STAGES,
                 done = grp0 + 2 * 48;
  auto s_full = [&](int w) { return grp0 + 48 * w; };
  auto s_free = [&](int w) { return grp0 + 48 * w + 8; };
  auto p_full = [&](int w) { return grp0 + 48 * w + 16; };
  auto p_free = [&](int w) { return grp0 + 48 * w + 24; };
  auto o_full = [&](int w) { return grp0 + 48 * w + 32; };
  auto o_free = [&](int w) { return grp0 + 48 * w + 40; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + WA_OFF_BAR + 448);
  const uint32_t sbase = smem_u32(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full + 8 * i, 1);
      mbar_init(q_empty + 8 * i, 1);
      mbar_init(s_full(i), 1);
      mbar_init(s_free(i), 4);  // one arrival per softmax warp of the tile
      mbar_init(p_full(i), 4);
      mbar_init(p_free(i), 1);
      mbar_init(o_full(i), 1);
      mbar_init(o_free(i), 4);
    }
    for (int i = 0; i < WA_STAGES; ++i) {
      mbar_init(kv_full + 8 * i, 1);
      mbar_init(kv_empty + 8 * i, 2);  // one arrival per tile
    }
    mbar_init(done, 3);
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), WA_TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_enter();  // the setup above overlaps the kernel before this one
  uint32_t kv_issued = 0, q_issued = 0;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(WA_REGS_CTRL));
    if (warp == 0 && lane == 0) {
      // ------------------------------------------------------------ producer
      prefetch_tmap(&tmQ);
      prefetch_tmap(&tmK);
      prefetch_tmap(&tmV);
      bool ok = true;
      uint32_t it = 0;
      for (int rd = 0, k = wa_rank(blockIdx.x, 0); k < a.n_items && ok;
           k = wa_rank(blockIdx.x, ++rd), ++it) {
        const WaItem m(a, k);
        const int kc = m.h / a.g * WA_D;
        const uint32_t qb = it & 1;
        const bool two = 2 * m.u + 1 < a.w.n_t;
        if (!mbar_wait(q_empty + 8 * qb, ((it >> 1) & 1) ^ 1)) break;
        mbar_arrive_expect_tx(q_full + 8 * qb, two ? 2 * WA_T_BYTES : WA_T_BYTES);
        for (int w = 0; w < (two ? 2 : 1); ++w)
          tma_load_3d(sbase + (2 * qb + w) * WA_T_BYTES, &tmQ, q_full + 8 * qb, m.h * WA_D,
                      (2 * m.u + w) * WT, m.b);
        q_issued = it + 1;
        for (int j = 0; j < m.n; ++j) {
          const uint32_t g = kv_issued, st = g % WA_STAGES;
          if (!mbar_wait(kv_empty + 8 * st, ((g / WA_STAGES) & 1) ^ 1)) {
            ok = false;
            break;
          }
          const uint32_t kdst = sbase + WA_OFF_KV + st * 2 * WA_T_BYTES;
          const int row = m.tile(j) * WT;
          mbar_arrive_expect_tx(kv_full + 8 * st, 2 * WA_T_BYTES);
          tma_load_3d(kdst, &tmK, kv_full + 8 * st, kc, row, m.b);
          tma_load_3d(kdst + WA_T_BYTES, &tmV, kv_full + 8 * st, kc, row, m.b);
          kv_issued = g + 1;
        }
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------ MMA issuer: scores
      // The whole warp runs the loop; one elected lane issues and commits.
      constexpr uint32_t idesc_s = idesc_bf16_f32(WT, WT, 0, 0), idesc_few = idesc_bf16_f32(WT, WT_FEW, 0, 0);
      const uint64_t dq0 = smem_desc_sw128(sbase, 16, 1024);
      const uint64_t dk0 = smem_desc_sw128(sbase + WA_OFF_KV, 16, 1024);
      constexpr uint64_t STEP = 2 * WA_T_BYTES >> 4;  // a stage, in a descriptor's units
      uint32_t G = 0;         // stages so far
      uint32_t gs0 = 0, gs1 = 0;  // score products of the tiles so far
      // tile w's scores of step j, if it takes part in it
      auto scores = [&](int w, const WaSteps& sp, int j, uint64_t dq, uint64_t dk, uint32_t& gs) -> bool {
        if (j >= sp.a2 || (j >= sp.a0 && j < sp.a1)) return true;
        if (gs > 0 && !wait_warp(s_free(w), (gs - 1) & 1)) return false;
        tc_fence_after();
        const uint32_t idesc = j == sp.few ? idesc_few : idesc_s, tS = tmem + 128 * w;
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < WA_D / 16; ++kk)
            tc_mma_f16(tS, dq + kk * 2, dk + kk * 2, idesc, kk ? 1u : 0u);
          tc_commit(s_full(w));
        }
        __syncwarp();
        ++gs;
        return true;
      };
      uint32_t it = 0;
      for (int rd = 0, k = wa_rank(blockIdx.x, 0); k < a.n_items; k = wa_rank(blockIdx.x, ++rd), ++it) {
        const WaItem m(a, k);
        const WaSteps sa(a, m, 2 * m.u), sb(a, m, 2 * m.u + 1);
        const uint32_t qb = it & 1;
        if (!wait_warp(q_full + 8 * qb, (it >> 1) & 1)) break;
        const uint64_t dqa = dq0 + qb * (2 * WA_T_BYTES >> 4), dqb = dqa + (WA_T_BYTES >> 4);
        int j = 0;
        for (; j < m.n; ++j) {
          const uint32_t st = (G + j) % WA_STAGES;
          if (!wait_warp(kv_full + 8 * st, ((G + j) / WA_STAGES) & 1)) break;
          const uint64_t dk = dk0 + st * STEP;
          if (!scores(0, sa, j, dqa, dk, gs0) || !scores(1, sb, j, dqb, dk, gs1)) break;
        }
        if (j < m.n) break;  // a wait ran out
        if (elect_one()) tc_commit(q_empty + 8 * qb);
        __syncwarp();
        G += m.n;
      }
      if (elect_one()) tc_commit(done);
      __syncwarp();
    } else if (warp >= 2) {
      // ------------------------------------------------------------ MMA issuers: O of tiles A, B
      const int w = warp - 2;
      constexpr uint32_t idesc_o = idesc_bf16_f32(WT, WA_D, 0, 1);
      const uint32_t tO = tmem + WA_TM_O + 64 * w, tP = tmem + WA_TM_P + 64 * w;
      const uint64_t dv0 = smem_desc_sw128(sbase + WA_OFF_KV + WA_T_BYTES, 8192, 1024);
      constexpr uint64_t STEP = 2 * WA_T_BYTES >> 4;
      uint32_t G = 0, gp = 0;  // stages, products so far
      uint32_t io = 0;         // items so far
      for (int rd = 0, k = wa_rank(blockIdx.x, 0); k < a.n_items; k = wa_rank(blockIdx.x, ++rd)) {
        const WaItem m(a, k);
        const WaSteps sp(a, m, 2 * m.u + w);
        bool first = true;
        int j = 0;
        for (; j < m.n; ++j) {
          const uint32_t st = (G + j) % WA_STAGES;
          if (!wait_warp(kv_full + 8 * st, ((G + j) / WA_STAGES) & 1)) break;
          if (j >= sp.a2 || (j >= sp.a0 && j < sp.a1)) {
            // not this tile's (after the wait: else it could pass the ring's round)
            if (elect_one()) mbar_arrive(kv_empty + 8 * st);
            __syncwarp();
            continue;
          }
          if (!wait_warp(p_full(w), gp & 1)) break;
          if (first && io > 0 && !wait_warp(o_free(w), (io - 1) & 1)) break;
          tc_fence_after();
          const uint64_t dv = dv0 + st * STEP;
          const bool few = j == sp.few;
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < WT / 16; ++kk)
              if (kk < WT_FEW / 16 || !few)
                tc_mma_f16_ts(tO, tP + kk * 8, dv + kk * (2048 >> 4), idesc_o, (!first || kk > 0) ? 1u : 0u);
            tc_commit(p_free(w));
            tc_commit(kv_empty + 8 * st);
            if (j == sp.a2 - 1) tc_commit(o_full(w));
          }
          __syncwarp();
          first = false;
          ++gp;
        }
        if (j < m.n) break;  // a wait ran out
        if (!first) ++io;
        G += m.n;
      }
      if (elect_one()) tc_commit(done);
      __syncwarp();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(WA_REGS_ROWS));
    // ------------------------------------------------------------ softmax
    const int w = (warp - 4) >> 2;  // query tile A (0) or B (1)
    const int q4 = warp & 3;         // TMEM lane quarter
    const int r = q4 * 32 + lane;    // query row in the tile = TMEM lane
    const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16);
    const uint32_t ts = tl + 128 * w, to = tl + WA_TM_O + 64 * w, tp = tl + WA_TM_P + 64 * w;
    const float2 sl = make_float2(a.sl2, a.sl2);
    bool ok = true, late = false;  // late: a row was not finite
    uint32_t g = 0, io = 0;
    int k = wa_rank(blockIdx.x, 0);
    WaItem next(a, k);  // worked out while the item before it waits for its O
    for (int rd = 1; k < a.n_items; ++rd) {
      const WaItem m = next;
      const int t = 2 * m.u + w;
      if (t >= a.w.n_t) {
        k = wa_rank(blockIdx.x, rd);
        next = WaItem(a, k);
        continue;
      }
      const int q = t * WT + r;  // query index in the sequence
      // its key tiles: the sinks' [0, ns) and the window's [lo, t]; those before `clear`
      // and the diagonal's, t, hide keys from some row
      const int lo = a.w.lo(t), ns = min(a.w.sT, lo);
      const int past = t * WT + WT - 1 - a.w.W, clear = past >= 0 ? past / WT + 1 : 0;
      const int few = a.w.few < lo ? a.w.few : -1;  // the few sinks' tile
      float mref = -INFINITY, l = 0.f;
      // tile kt, of which the rows see none but its first NC keys
      auto step = [&](auto cols, auto masked, int kt) -> bool {
        constexpr int NC = decltype(cols)::value;
        if (!wait_warp(s_full(w), g & 1)) return false;
        tc_fence_after();
        // the scores into registers, the first half's maxima while the second comes; then the
        // next may replace them
        uint32_t sc[NC];
        float mx[8];
        auto maxima = [&](int c0) {
#pragma unroll
          for (int c = c0; c < c0 + NC / 2; c += 16)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              mx[e] = c == 0 ? fmaxf(__uint_as_float(sc[2 * e]), __uint_as_float(sc[2 * e + 1]))
                             : max3f(mx[e], __uint_as_float(sc[c + 2 * e]), __uint_as_float(sc[c + 2 * e + 1]));
        };
        constexpr bool HALVES = !decltype(masked)::value;  // (with masks too: 4.39 ms)
        if (HALVES) {
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
          for (int c = 0; c < NC; c += 32) tmem_ld32_async(ts + c, sc + c);
#pragma unroll
          for (int c = 0; c < NC; c += 32) tmem_wait_ld(sc + c);
        }
        tc_fence_before();
        mbar_arrive_warp(s_free(w));
        if (NC < WT) {
#pragma unroll
          for (int c = 0; c < NC; ++c)
            if (c >= a.w.S - kt * WT) sc[c] = 0xff800000u;  // -inf
        } else if (decltype(masked)::value) {
          // seen keys: (q - W, q], and the sinks; bit c of a word: its column c
          auto low = [](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };
#pragma unroll
          for (int c0 = 0; c0 < NC; c0 += 32) {
            const int b0 = kt * WT + c0;
            const uint32_t vis = low(q + 1 - b0) & (~low(q - a.w.W + 1 - b0) | low(a.w.S - b0));
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!(vis >> c & 1)) sc[c0 + c] = 0xff800000u;  // -inf
          }
        }
        // the maximum (log2 units), three-input maxima
        if (!HALVES) maxima(0);
        maxima(NC / 2);
        const float mt =
            max3f(max3f(mx[0], mx[1], mx[2]), max3f(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * a.sl2;
        // the first keys set the reference; later ones raise it only by more than
        // WA_RESCALE, scaling O and the running sum
        if (__any_sync(0xffffffffu, mt > mref + WA_RESCALE)) {
          float corr = 1.f;
          if (mt > mref + WA_RESCALE) {
            if (mref != -INFINITY) corr = ex2_approx(mref - mt);
            mref = mt;
          }
          if (__any_sync(0xffffffffu, corr != 1.f)) {  // this warp's rows of O
            if (!wait_warp(p_free(w), (g - 1) & 1)) return false;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 64; c += 16) {
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
        uint32_t pk[NC / 2];
        constexpr int OUT = NC < WT ? 0 : 2;  // P goes out from this quarter on (from 1: 4.28 ms, from 3: 4.35)
#pragma unroll
        for (int hh = 0; hh < NC / 32; ++hh) {
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float2 z = __ffma2_rn(make_float2(__uint_as_float(sc[32 * hh + 2 * c]),
                                                    __uint_as_float(sc[32 * hh + 2 * c + 1])),
                                        sl, nm);
            const float2 pp = make_float2(ex2_approx(z.x), ex2_approx(z.y));
            ps[c & 1] = __fadd2_rn(ps[c & 1], pp);
            pk[16 * hh + c] = pack_bf16(pp.x, pp.y);
          }
          if (hh == OUT) {  // the last tile's P has been consumed
            if (g > 0 && !wait_warp(p_free(w), (g - 1) & 1)) return false;
            tc_fence_after();
          }
          if (hh >= OUT)
#pragma unroll
            for (int c = hh == OUT ? 0 : 16 * hh; c <= 16 * hh; c += 16) tmem_st16(tp + c, pk + c);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive_warp(p_full(w));
        l += (ps[0].x + ps[0].y) + (ps[1].x + ps[1].y);
        ++g;
        return true;
      };
      // (one place each for tiles with and without masks: two of the first, and smaller cases
      // wait for instructions, 1 us of 33 for 2 x 1000 tokens)
      const std::integral_constant<int, WT> all{};
      int kt = ns > 0 ? 0 : lo;
#pragma unroll 1
      for (;;) {
#pragma unroll 1
        for (; ok && (kt < clear || kt == t); kt = kt + 1 == ns ? lo : kt + 1)
          ok = kt == few ? step(std::integral_constant<int, WT_FEW>{}, std::true_type{}, kt)
                         : step(all, std::true_type{}, kt);
        if (!ok || kt > t) break;
#pragma unroll 1
        for (; ok && kt < t; ++kt) ok = step(all, std::false_type{}, kt);
      }
      if (!ok) break;
      k = wa_rank(blockIdx.x, rd);
      next = WaItem(a, k);
      // the item's O: after its last P.V
      if (!wait_warp(o_full(w), io & 1)) break;
      ++io;
      tc_fence_after();
      uint32_t ov[64];
      tmem_ld32_async(to, ov);
      tmem_ld32_async(to + 32, ov + 32);
      tmem_wait_ld(ov);
      tmem_wait_ld(ov + 32);
      tc_fence_before();
      mbar_arrive_warp(o_free(w));
      float2 fin[4] = {};  // zero, but for sums that are not finite
#pragma unroll
      for (int i = 0; i < WA_D / 2; ++i)
        fin[i % 4] = __ffma2_rn(make_float2(__uint_as_float(ov[2 * i]), __uint_as_float(ov[2 * i + 1])),
                                make_float2(0.f, 0.f), fin[i % 4]);
      fin[0] = __fadd2_rn(__fadd2_rn(fin[0], fin[1]), __fadd2_rn(fin[2], fin[3]));
      late |= fin[0].x + fin[0].y != 0.f;
      // the warp's 32 rows go out by TMA from its own stage (128-byte swizzle; rows past the end
      // of the sequence are left out)
      const float inv = 1.f / l;  // (a row sees itself: 0 where its scores are all -inf, and 0 / 0 is NaN)
      uint8_t* const stg = smem + WA_OFF_STG + (warp - 4) * 4096;
      auto put = [&](const CUtensorMap* map, const uint32_t* v) {  // v: the row, bf16 pairs
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the store before
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<uint4*>(stg + lane * 128 + ((i ^ (lane & 7)) << 4)) =
              make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          if (t * WT + q4 * 32 < a.w.L)
            tma_store_3d(map, smem_u32(stg), m.h * WA_D, t * WT + q4 * 32, m.b);
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
      };
      uint32_t pk[WA_D / 2];
#pragma unroll
      for (int i = 0; i < WA_D / 2; ++i) {
        const float2 o = __fmul2_rn(make_float2(__uint_as_float(ov[2 * i]), __uint_as_float(ov[2 * i + 1])),
                                    make_float2(inv, inv));
        pk[i] = pack_bf16(o.x, o.y);
        ov[2 * i] = __float_as_uint(o.x);
        ov[2 * i + 1] = __float_as_uint(o.y);
      }
      put(&tmO, pk);
      if (a.lse) {  // the backward's Di = dO . O cancels against dP: it wants more than bf16's O
#pragma unroll
        for (int i = 0; i < WA_D / 2; ++i) {
          const float2 b = unpack_bf16(pk[i]);
          pk[i] = pack_bf16(__uint_as_float(ov[2 * i]) - b.x, __uint_as_float(ov[2 * i + 1]) - b.y);
        }
        put(&tmR, pk);
        if (q < a.w.L)
          a.lse[((long)m.b * a.H + m.h) * a.w.L + q] = mref + log2f(l);  // log2 units
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
    if (__any_sync(0xffffffffu, late)) wa_repair(a, warp);
  }
  tc_fence_before();
  if (__syncthreads_or(*(volatile int*)&g_dev_error != 0)) {
    // error path: let this CTA's copies and MMAs land before smem / TMEM go
    if (warp == 0 && lane == 0) {
      for (uint32_t G = kv_issued > WA_STAGES ? kv_issued - WA_STAGES : 0; G < kv_issued; ++G)
        mbar_wait_drain(kv_full + 8 * (G % WA_STAGES), (G / WA_STAGES) & 1);
      for (uint32_t t = q_issued > 2 ? q_issued - 2 : 0; t < q_issued; ++t)
        mbar_wait_drain(q_full + 8 * (t & 1), (t >> 1) & 1);
    }
    if (warp == 1 && lane == 0) mbar_wait_drain(done, 0);
  } else if (warp == 1 && lane == 0) {
    mbar_wait(done, 0);
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, WA_TMEM_COLS);
  }
}

}  // namespace

double window_pairs(const Window& c) {
  const double L = c.L, W = c.window > 0 ? std::min(c.window, c.L) : c.L;
  const double S = std::min<double>(c.sinks, L - W);
  // the window's triangle and band, and the sinks that lie below it, coming into sight one by one
  return W * (W + 1) / 2 + (L - W) * W + S * (S + 1) / 2 + (L - W - S) * S;
}

WindowSaved window_saved(const Window& c, void* p) {
  const size_t rows = (size_t)c.B * c.L, lse = (rows * c.H * sizeof(float) + 255) & ~size_t(255);
  return {static_cast<float*>(p), reinterpret_cast<bf16*>(static_cast<char*>(p) + lse),
          lse + rows * c.H * WA_D * sizeof(bf16)};
}

cudaError_t window_fwd(const Window& c, const QkvPtr& x, bf16* out, long ldo, const WindowSaved& v,
                       cudaStream_t st) {
  launched.mark();
  CUtensorMap tq, tk, tv, to, tr;
  if (!tmap_bf16_seq(&tq, x.q, (uint64_t)c.H * WA_D, c.L, c.B, x.ldq, WA_D, WT) ||
      !tmap_bf16_seq(&tk, x.k, (uint64_t)c.KV * WA_D, c.L, c.B, x.ldk, WA_D, WT) ||
      !tmap_bf16_seq(&tv, x.v, (uint64_t)c.KV * WA_D, c.L, c.B, x.ldv, WA_D, WT) ||
      !tmap_bf16_seq(&to, out, (uint64_t)c.H * WA_D, c.L, c.B, ldo, WA_D, 32) ||
      !tmap_bf16_seq(&tr, v.rest ? v.rest : out, (uint64_t)c.H * WA_D, c.L, c.B,
                     v.rest ? (uint64_t)c.H * WA_D : ldo, WA_D, 32))
    return cudaErrorInvalidValue;
  WaArgs a{};
  a.lse = v.lse;
  a.B = c.B;
  a.H = c.H;
  a.g = c.H / c.KV;
  a.w = WinTiles(c);
  a.n_st = (a.w.n_t + 1) / 2;
  const long items = (long)a.n_st * c.H * c.B;
  if (items > 0x3fffffff) return cudaErrorInvalidValue;
  a.n_items = (int)items;
  a.sl2 = 1.4426950408889634f / sqrtf((float)WA_D);
  a.q = static_cast<const bf16*>(x.q);
  a.k = static_cast<const bf16*>(x.k);
  a.v = static_cast<const bf16*>(x.v);
  a.out = out;
  a.rest = v.rest;
  a.ldq = x.ldq;
  a.ldk = x.ldk;
  a.ldv = x.ldv;
  a.ldo = ldo;
  static KernelOnce once;
  const cudaError_t e = once(reinterpret_cast<const void*>(window_fwd_kernel), WA_SMEM, WA_THREADS,
                             WA_REGS_CTRL * 128 + WA_REGS_ROWS * 256);
  if (e != cudaSuccess) return e;
  const double pairs = (double)c.B * c.H * window_pairs(c);
  LaunchTimer lt("window_fwd", st, 4.0 * WA_D * pairs,
                 2.0 * c.B * c.L * WA_D * ((v.lse ? 3.0 : 2.0) * c.H + 2.0 * c.KV) +
                     (v.lse ? 4.0 * c.B * c.H * c.L : 0.0));
  const int grid = std::min(a.n_items, num_sms());
  return launch_kernel(window_fwd_kernel, grid, WA_THREADS, WA_SMEM, st, tq, tk, tv, to, tr, a);
}

}  // namespace pf

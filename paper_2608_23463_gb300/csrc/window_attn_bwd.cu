// Backward of the windowed attention with sinks on the tcgen05 tensor cores,
// head width 64, grouped heads.  With P = softmax(q k / 8) recomputed from the
// saved LSE and Di = rowsum(dO * O), with O to 2^-17 (dS is a difference of the two: with
// O as rounded to bf16, rows of few keys lose dQ and dK to it):
//   dP = dO V^T,   dS = P * (dP - Di),   dV = P^T dO,   dK = dS^T Q / 8,
//   dQ = dS K / 8,   dK and dV summed over the query heads of a key head.
// Two kernels share one skeleton (no atomics, deterministic):
//   DKDV: stationary X1 = K, X2 = V of a 128-key tile; streamed Y1 = Q_j, Y2 =
//         dO_j of the query tiles that see it, one query head of the group
//         after the other, into the same accumulators
//           T1 = X1 Y1^T - 8 LSE / log2(e),  T2 = X2 Y2^T - Di  (TMEM, M=128 N=128)
//           E1 = P^T, E2 = dS^T  (bf16, written to TMEM by the row warps)
//           dV += E1 Y2,  dK += E2 Y1    (A from TMEM; TMEM accumulators)
//   DQ:   stationary X1 = Q, X2 = dO of a 128-query tile and head; streamed
//         Y1 = K_j, Y2 = V_j of the sinks' and the window's tiles
//           T1 = S,  T2 = dP,  E2 = dS,  dQ += E2 Y1
// DKDV's rows are keys, so that LSE and Di run along the columns, the same for every
// row: they come in as one more MMA (K=16) of ones with each query's LSE and Di, split
// in three bf16 each (24 bits).  From shared memory every thread read both for each of
// its columns, 128 KB a step at 128 bytes a cycle, and a producer warp staged them: 520
// us for 16384 causal tokens of 8 heads, of which 106 for the reads alone.  DQ's rows
// take theirs from the same array, loaded with X (from global memory at an item's start,
// each row waited 1000 cycles for them: dQ 424 us for 65536 tokens of 16 heads, 406 so).
// Roles: warp 0 TMA producer, warp 1 MMA issuer of T, warp 2 MMA issuer of the sums, warp 3
// their TMA stores, warps 4-19 the row warps: four per TMEM lane quarter, each thread one
// row (TMEM lane) and one quarter of the 128 streamed columns.  (One issuer for both took
// 700 cycles for T and 900 to 1200 for the sums of a step, more than their MMAs: it shares
// its scheduler with four row warps.  65536 tokens of 16 heads, window 1024: dK and dV 601
// us with it, 493 so; dQ 453 and 444.)
// The sinks are seen by every later query: their key tiles' steps are cut into
// pieces (wb_cut), as are all tiles' where there are few.  The pieces of a cut
// tile leave fp32 sums, those past its window of the sinks' rows alone;
// window_join_kernel adds them in order.  Items go round the CTAs, so that those
// at work at one time share their streamed tiles in L2.  (The steps of all tiles
// dealt to the CTAs in equal ranges instead: 65536 tokens of 16 heads on 4 key
// heads, window 1024: 800 us, 664 so; a range's tiles are too far apart.)
// An item's sums are read out in the next item's first step, when that step's E waits
// for them anyway: no warp waits for the end of an item's products.  They go out by TMA
// from where the item's X was (a row's 32 bytes a thread, stored directly, held the first
// step up by 1000 to 2000 cycles: dK and dV 493 us and dQ 444 so, 446 and 424 by TMA).
// The producer alone works out the items; the others read them from shared memory and
// count their steps up: what each step costs a warp beside its products and its 32
// columns is on the chain of every step.
// What bounds it: the chain of T's products (operands from shared memory at its 128 bytes a
// cycle, beside 34 KB of TMA writes a step), their commit and the row warps' reads of T, 1500
// to 1600 cycles a step, of which the MMAs take 1152 (DKDV, 73 % of the tensor pipe's time)
// and 768 (DQ).  65536 tokens of 16 heads, window 1024, 4 sinks: dK and dV 452 us, dQ 406.  Not faster: T in halves of 64
// columns or T1 and T2 handed over apart, so that the row warps' phases overlap; X in TMEM
// for DQ; Di into DQ's T by an MMA; Di worked out by a warp of DQ; waits that probe.
// Every mbarrier wait is bounded.  Masked columns have P = 0, and rows past the
// end of a sequence read as zero.
#include <algorithm>
#include <type_traits>

#include "local.h"
#include "window_tiles.cuh"

namespace pf {

static Launched launched;
int take_dev_error_window_attn_bwd() { return launched.take(take_dev_error_tu); }
int set_wait_limit_window_attn_bwd(unsigned long long ns) { return set_wait_limit_tu(ns); }

namespace {

constexpr int WB_D = 64;   // head width
constexpr int WB_EXT = 16;  // bf16 of a query's LSE and Di: three each, the rest zero
constexpr int WB_STAGES = 4;
constexpr int WB_ROW_THREADS = 512;  // warps 4-19
constexpr int WB_THREADS = 128 + WB_ROW_THREADS;
// A row thread holds 64 values of a step: the control warps give registers up, of the 96
// that each thread has at launch.
constexpr int WB_REGS_CTRL = 64, WB_REGS_ROWS = 104;
static_assert(WB_REGS_CTRL * 128 + WB_REGS_ROWS * 512 <= 96 * WB_THREADS, "register split");
constexpr uint32_t WB_T_BYTES = WT * WB_D * 2;  // 16 KB per tile
constexpr uint32_t WB_OFF_Y = 2 * 2 * WB_T_BYTES;                     // X: [2 bufs][X1, X2]
constexpr uint32_t WB_OFF_E = WB_OFF_Y + WB_STAGES * 2 * WB_T_BYTES;  // Y: [stage][Y1, Y2]
constexpr uint32_t WB_E_BYTES = WT * WB_EXT * 2;                       // LSE, Di: [stage][128][16]
constexpr uint32_t WB_OFF_ONE = WB_OFF_E + WB_STAGES * WB_E_BYTES;     // the ones for T1, for T2
constexpr uint32_t WB_OFF_BAR = WB_OFF_ONE + 2 * WB_E_BYTES;
constexpr uint32_t WB_OFF_ITEM = WB_OFF_BAR + 256;  // four items
constexpr uint32_t WB_SMEM = WB_OFF_ITEM + 4 * 48 + 1024;
// TMEM columns: T1 at 0, T2 at 128 (fp32), accumulators at 256 (dV or dQ) and 320
// (dK), E1 at 384, E2 at 448 (bf16 pairs: streamed column c in 32-bit column c / 2)
constexpr uint32_t WB_TMEM_COLS = 512;
constexpr uint32_t WB_TM_E = 384;
constexpr int WB_ACC = 2 * WB_D;  // dV | dK of a key

struct WbArgs {
  bf16 *out_u, *out_w;  // window_join_kernel: dV, dK.  Head h at column 64 h
  long ld_u, ld_w;
  int B, H, KV, g;
  WinTiles w;
  // DKDV: steps of a piece, pieces of a sink tile and of another tile, and the
  // pieces' sums [piece][128][dV | dK], fp32
  int C, np_s, np_w;
  float* part;
  int n_items;
  float sl2, scale;
};

__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Snake order over the CTAs of items ranked heaviest first.
__device__ __forceinline__ int wb_rank(int c, int round) {
  return round * (int)gridDim.x + ((round & 1) ? (int)gridDim.x - 1 - c : c);
}

// Query tiles that see key tile t: [t, t + wb_queries(t)).
__host__ __device__ __forceinline__ int wb_queries(const WinTiles& w, int t) {
  return (t < w.sT ? w.n_t - 1 : w.last_q(t)) - t + 1;
}
// Rows of key tile t that the steps [s0, s0 + n) of its list add to: all, or the sinks
// alone where every query tile is past its window.
__device__ __forceinline__ int wb_rows(const WinTiles& w, int t, int m, int s0, int n) {
  const int i = s0 % m;
  return t < w.sT && i + n <= m && t + i > w.last_q(t) ? min(WT, w.S - t * WT) : WT;
}

// A work item: stationary tile t of sequence b, head h (DKDV: the key head; DQ: the query
// head) and its n steps.  They stream
//   DKDV: query tiles t .. t + m - 1 of the group's heads in turn, from query tile
//         `tile` of head `head` on
//   DQ:   the sinks' key tiles [0, m) and the window's [lo, t], lo in `head`
struct __align__(16) WbItem {
  int t, h, b, n;
  int tile, head, m, piece;  // piece < 0: all of the tile's steps
  int rows, pad[3];          // DKDV: rows that a piece adds to
};

// DKDV: item k: the pieces of the sinks' tiles, then those of the others; n may be 0.
__device__ __forceinline__ WbItem wb_key_item(const WbArgs& a, int k) {
  WbItem i;
  const int per = a.KV * a.B, sinks = a.w.sT * a.np_s * per;
  const bool sink = k < sinks;
  const int kk = (sink ? k : k - sinks) / per, np = sink ? a.np_s : a.np_w, p = kk % np;
  const int hb = (sink ? k : k - sinks) - kk * per;
  i.t = (sink ? 0 : a.w.sT) + kk / np;
  i.b = hb / a.KV;
  i.h = hb - i.b * a.KV;
  i.m = wb_queries(a.w, i.t);
  const int s0 = p * a.C;
  i.n = max(0, min(i.m * a.g - s0, a.C));
  i.tile = i.t + s0 % i.m;
  i.head = i.h * a.g + s0 / i.m;
  i.piece = np == 1 ? -1 : k;
  i.rows = wb_rows(a.w, i.t, i.m, s0, i.n);
  return i;
}
// DQ: item k, from the last query tile on.
__device__ __forceinline__ WbItem wb_query_item(const WbArgs& a, int k) {
  WbItem i;
  const int per = a.H * a.B;
  i.t = a.w.n_t - 1 - k / per;
  i.h = k % per % a.H;
  i.b = k % per / a.H;
  i.head = a.w.lo(i.t);
  i.m = min(a.w.sT, i.head);
  i.n = i.m + i.t - i.head + 1;
  i.tile = i.m > 0 ? 0 : i.head;
  i.piece = -1;
  return i;
}

// The streamed tile of an item's steps, one after the other.
template <bool DKDV>
struct WbStep {
  int tile, head;  // head (DKDV): of the streamed queries
  __device__ __forceinline__ explicit WbStep(const WbItem& i) : tile(i.tile), head(i.head) {}
  __device__ __forceinline__ void next(const WbItem& i) {
    ++tile;
    if (DKDV) {
      if (tile == i.t + i.m) {
        tile = i.t;
        ++head;
      }
    } else if (tile == i.m) {
      tile = i.head;
    }
  }
};

// Shared-memory matrix descriptor of a K-major tile with rows of 32 bytes, 32-byte swizzle.
__device__ __forceinline__ uint64_t smem_desc_sw32(uint32_t saddr) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) | 1ull << 16 | (uint64_t)(256 >> 4) << 32 | 1ull << 46 |
         6ull << 61;
}

// A wait of a converged warp, the common case of a completed phase up front.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity) {
  if (__all_sync(0xffffffffu, mbar_test_wait(bar, parity))) return true;
  return mbar_wait_warp(bar, parity);
}

template <bool DKDV>
__global__ void __launch_bounds__(WB_THREADS, 1)
    window_bwd_kernel(const __grid_constant__ CUtensorMap tmX1, const __grid_constant__ CUtensorMap tmX2,
                      const __grid_constant__ CUtensorMap tmY1, const __grid_constant__ CUtensorMap tmY2,
                      const __grid_constant__ CUtensorMap tmE, const __grid_constant__ CUtensorMap tmU,
                      const __grid_constant__ CUtensorMap tmW, WbArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  const uint32_t b0 = smem_u32(smem + WB_OFF_BAR);
  // x_full[2] x_empty[2] y_full[S] y_empty[S] t_full t_free e_full e_free done o_full
  const uint32_t x_full = b0, x_empty = b0 + 16, y_full = b0 + 32,
                 y_empty = y_full + 8 * WB_STAGES, t_full = y_empty + 8 * WB_STAGES,
                 t_free = t_full + 8, e_full = t_free + 8, e_free = e_full + 8, done = e_free + 8,
                 o_full = done + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + WB_OFF_BAR + 240);
  const uint32_t sbase = smem_u32(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(x_full + 8 * i, 1);
      mbar_init(x_empty + 8 * i, 3);  // both issuers, the sums' store
    }
    mbar_init(t_full, 1);
    mbar_init(t_free, WB_ROW_THREADS / 32);  // one arrival per row warp
    mbar_init(e_full, WB_ROW_THREADS / 32);
    mbar_init(e_free, 1);
    for (int i = 0; i < WB_STAGES; ++i) {
      mbar_init(y_full + 8 * i, 1);
      mbar_init(y_empty + 8 * i, 1);
    }
    mbar_init(done, 2);
    mbar_init(o_full, WB_ROW_THREADS / 32);
    fence_barrier_init();
  }
  if (DKDV) {
    // rows of ones for LSE's three parts (T1) and Di's (T2), twice a row: the swizzle may put
    // either half first, and the other half meets zeros
    for (int i = threadIdx.x; i < 2 * WT * WB_EXT; i += WB_THREADS) {
      const int k = i % 8;
      reinterpret_cast<bf16*>(smem + WB_OFF_ONE)[i] =
          __float2bfloat16((i < WT * WB_EXT ? k < 3 : k >= 3 && k < 6) ? 1.f : 0.f);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the MMAs read them
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), WB_TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_enter();  // the setup above overlaps the kernel before this one
  uint32_t y_issued = 0, x_issued = 0;

  if (warp < 4) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(WB_REGS_CTRL));
  if (warp == 0) {
    // ------------------------------------------------------------ producer
    if (lane == 0) {
      prefetch_tmap(&tmX1);
      prefetch_tmap(&tmX2);
      prefetch_tmap(&tmY1);
      prefetch_tmap(&tmY2);
      prefetch_tmap(&tmE);
    }
    WbItem* const ring = reinterpret_cast<WbItem*>(smem + WB_OFF_ITEM);
    int rd = 0;
    auto next_item = [&]() -> WbItem {  // the next one with steps; n < 0 at the end
      for (int k; (k = wb_rank(blockIdx.x, rd)) < a.n_items; ++rd) {
        const WbItem i = DKDV ? wb_key_item(a, k) : wb_query_item(a, k);
        if (i.n > 0) {
          ++rd;
          return i;
        }
      }
      WbItem i{};
      i.n = -1;
      return i;
    };
    WbItem m = next_item();
    bool ok = true;
    for (uint32_t it = 0; ok; ++it) {
      const uint32_t xb = it & 1;
      // (item it - 2's sums have left this buffer: all have begun the item after it, no phase of
      // x_full is passed over, and its slot is read no more)
      if (!wait_warp(x_empty + 8 * xb, ((it >> 1) & 1) ^ 1)) break;
      if (lane == 0) {
        ring[it & 3] = m;
        if (m.n > 0) {
          const uint32_t xdst = sbase + xb * 2 * WB_T_BYTES;
          mbar_arrive_expect_tx(x_full + 8 * xb, 2 * WB_T_BYTES + (DKDV ? 0u : WB_E_BYTES));
          if (!DKDV)
            tma_load_3d(sbase + WB_OFF_E + xb * WB_E_BYTES, &tmE, x_full + 8 * xb, 0, m.t * WT,
                        m.b * a.H + m.h);
          tma_load_3d(xdst, &tmX1, x_full + 8 * xb, m.h * WB_D, m.t * WT, m.b);
          tma_load_3d(xdst + WB_T_BYTES, &tmX2, x_full + 8 * xb, m.h * WB_D, m.t * WT, m.b);
        } else {
          mbar_arrive(x_full + 8 * xb);
        }
      }
      if (m.n < 0) break;
      x_issued = it + 1;
      const WbItem m2 = next_item();
      WbStep<DKDV> sp(m);
      const int kv = m.h / a.g;  // DQ: the key head
      for (int j = 0; j < m.n; ++j) {
        const uint32_t G = y_issued, st = G % WB_STAGES;
        if (!wait_warp(y_empty + 8 * st, ((G / WB_STAGES) & 1) ^ 1)) {
          ok = false;
          break;
        }
        if (lane == 0) {
          const uint32_t ydst = sbase + WB_OFF_Y + st * 2 * WB_T_BYTES;
          const int yrow = sp.tile * WT, ycol = (DKDV ? sp.head : kv) * WB_D;
          mbar_arrive_expect_tx(y_full + 8 * st, 2 * WB_T_BYTES + (DKDV ? WB_E_BYTES : 0u));
          if (DKDV)
            tma_load_3d(sbase + WB_OFF_E + st * WB_E_BYTES, &tmE, y_full + 8 * st, 0, yrow,
                        m.b * a.H + sp.head);
          tma_load_3d(ydst, &tmY1, y_full + 8 * st, ycol, yrow, m.b);
          tma_load_3d(ydst + WB_T_BYTES, &tmY2, y_full + 8 * st, ycol, yrow, m.b);
        }
        y_issued = G + 1;
        sp.next(m);
      }
      m = m2;
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer: T
    // The whole warp runs the loop; one elected lane issues and commits.
    constexpr uint32_t idesc = idesc_bf16_f32(WT, WT, 0, 0);
    const WbItem* const ring = reinterpret_cast<const WbItem*>(smem + WB_OFF_ITEM);
    const uint64_t dx0 = smem_desc_sw128(sbase, 16, 1024);
    const uint64_t dy0 = smem_desc_sw128(sbase + WB_OFF_Y, 16, 1024);
    const uint64_t de0 = smem_desc_sw32(sbase + WB_OFF_E), one = smem_desc_sw32(sbase + WB_OFF_ONE);
    constexpr uint64_t TILE = WB_T_BYTES >> 4;  // in a descriptor's units
    bool ok = true;
    uint32_t G = 0;
    for (uint32_t it = 0; ok; ++it) {
      const uint32_t xb = it & 1;
      if (!wait_warp(x_full + 8 * xb, (it >> 1) & 1)) break;
      const int n = ring[it & 3].n;
      if (n < 0) break;
      const uint64_t d1 = dx0 + xb * 2 * TILE, d2 = d1 + TILE;
      for (int j = 0; j < n; ++j, ++G) {
        const uint32_t st = G % WB_STAGES;
        if (!wait_warp(y_full + 8 * st, (G / WB_STAGES) & 1) || !wait_warp(t_free, (G & 1) ^ 1)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint64_t y1 = dy0 + st * 2 * TILE, y2 = y1 + TILE, ye = de0 + st * (WB_E_BYTES >> 4);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < WB_D / 16; ++kk) {
            tc_mma_f16(tmem, d1 + kk * 2, y1 + kk * 2, idesc, kk ? 1u : 0u);
            tc_mma_f16(tmem + WT, d2 + kk * 2, y2 + kk * 2, idesc, kk ? 1u : 0u);
          }
          if (DKDV) {
            tc_mma_f16(tmem, one, ye, idesc, 1u);
            tc_mma_f16(tmem + WT, one + (WB_E_BYTES >> 4), ye, idesc, 1u);
          }
          tc_commit(t_full);
          if (j == n - 1) tc_commit(x_empty + 8 * xb);
        }
        __syncwarp();
      }
    }
    if (elect_one()) tc_commit(done);
    __syncwarp();
  } else if (warp == 2) {
    // ------------------------------------------------------------ MMA issuer: sums
    constexpr uint32_t idesc = idesc_bf16_f32(WT, WB_D, 0, 1);
    const WbItem* const ring = reinterpret_cast<const WbItem*>(smem + WB_OFF_ITEM);
    const uint64_t da0 = smem_desc_sw128(sbase + WB_OFF_Y, 8192, 1024);
    constexpr uint64_t TILE = WB_T_BYTES >> 4;
    const uint32_t e1 = tmem + WB_TM_E, e2 = e1 + WT / 2;
    bool ok = true;
    uint32_t G = 0;
    for (uint32_t it = 0; ok; ++it) {
      const uint32_t xb = it & 1;
      if (!wait_warp(x_full + 8 * xb, (it >> 1) & 1)) break;
      const int n = ring[it & 3].n;
      mbar_arrive_warp(x_empty + 8 * xb);
      if (n < 0) break;
      for (int j = 0; j < n; ++j, ++G) {
        const uint32_t st = G % WB_STAGES;
        // (the row warps have E from T, and T's products Y: the wait for Y is for this warp's sake)
        if (!wait_warp(y_full + 8 * st, (G / WB_STAGES) & 1) || !wait_warp(e_full, G & 1)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint64_t d1 = da0 + st * 2 * TILE, d2 = d1 + TILE;
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < WT / 16; ++kk) {
            const uint32_t acc = (j > 0 || kk > 0) ? 1u : 0u;
            if (DKDV) {
              tc_mma_f16_ts(tmem + 256, e1 + kk * 8, d2 + kk * (2048 >> 4), idesc, acc);  // dV += P^T dO
              tc_mma_f16_ts(tmem + 320, e2 + kk * 8, d1 + kk * (2048 >> 4), idesc, acc);  // dK += dS^T Q
            } else {
              tc_mma_f16_ts(tmem + 256, e2 + kk * 8, d1 + kk * (2048 >> 4), idesc, acc);  // dQ += dS K
            }
          }
          tc_commit(e_free);
          tc_commit(y_empty + 8 * st);
        }
        __syncwarp();
      }
    }
    if (elect_one()) tc_commit(done);
    __syncwarp();
  } else {
    // ------------------------------------------------------------ store of the sums
    // The row warps leave an item's dK and dV, or dQ, in the shared memory of its X, whose
    // products are done.
    const WbItem* const ring = reinterpret_cast<const WbItem*>(smem + WB_OFF_ITEM);
    for (uint32_t it = 0;; ++it) {
      const uint32_t xb = it & 1;
      if (!wait_warp(x_full + 8 * xb, (it >> 1) & 1)) break;
      if (ring[it & 3].n < 0 || !wait_warp(o_full, it & 1)) break;
      if (lane == 0) {
        const WbItem m = ring[it & 3];
        if (m.piece < 0) {
          const uint32_t src = sbase + xb * 2 * WB_T_BYTES;
          tma_store_3d(&tmU, src, m.h * WB_D, m.t * WT, m.b);
          if (DKDV) tma_store_3d(&tmW, src + WB_T_BYTES, m.h * WB_D, m.t * WT, m.b);
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        }
        mbar_arrive(x_empty + 8 * xb);
      }
      __syncwarp();
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(WB_REGS_ROWS));
    // ------------------------------------------------------------ row warps
    const int q4 = warp & 3;
    const int r = q4 * 32 + lane;  // stationary row in the tile = TMEM lane
    const int ch = (warp - 4) >> 2;   // quarter of the streamed columns: [32 ch, 32 ch + 32)
    const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16);
    const WbItem* const ring = reinterpret_cast<const WbItem*>(smem + WB_OFF_ITEM);
    struct Sums {
      uint32_t u[16], w[16];  // 16 columns of an item's dV / dQ and of its dK
    };
    auto load_sums = [&](Sums& v) {
      tmem_ld16(tl + 256 + 16 * ch, v.u);
      if (DKDV) tmem_ld16(tl + 320 + 16 * ch, v.w);
    };
    // item n's dV and dK (DKDV) or dQ to where warp 3 stores them from, or a piece's sums
    auto store_sums = [&](uint32_t n, const Sums& sum) {
      const WbItem& m = ring[n & 3];
      const uint32_t *u0 = sum.u, *w0 = sum.w;
      if (DKDV && m.piece >= 0) {  // sums of a cut tile
        if (r < m.rows && m.t * WT + r < a.w.L) {
          float* o = a.part + ((long)m.piece * WT + r) * WB_ACC + 16 * ch;
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            *reinterpret_cast<uint4*>(o + i) = make_uint4(u0[i], u0[i + 1], u0[i + 2], u0[i + 3]);
            *reinterpret_cast<uint4*>(o + WB_D + i) = make_uint4(w0[i], w0[i + 1], w0[i + 2], w0[i + 3]);
          }
        }
      } else {
        uint8_t* const dst = smem + (n & 1) * 2 * WB_T_BYTES + r * 128;
        auto put = [&](uint8_t* o, const uint32_t* v, float sc) {  // 128-byte swizzle
#pragma unroll
          for (int i = 0; i < 16; i += 8)
            *reinterpret_cast<uint4*>(o + (((2 * ch + i / 8) ^ (r & 7)) << 4)) = make_uint4(
                pack_bf16(__uint_as_float(v[i]) * sc, __uint_as_float(v[i + 1]) * sc),
                pack_bf16(__uint_as_float(v[i + 2]) * sc, __uint_as_float(v[i + 3]) * sc),
                pack_bf16(__uint_as_float(v[i + 4]) * sc, __uint_as_float(v[i + 5]) * sc),
                pack_bf16(__uint_as_float(v[i + 6]) * sc, __uint_as_float(v[i + 7]) * sc));
        };
        put(dst, u0, DKDV ? 1.f : a.scale);
        if (DKDV) put(dst + WB_T_BYTES, w0, a.scale);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // a TMA store reads them
      }
      mbar_arrive_warp(o_full);
    };
    bool ok = true;
    uint32_t G = 0;
    for (uint32_t it = 0; ok; ++it) {
      if (!wait_warp(x_full + 8 * (it & 1), (it >> 1) & 1)) break;
      const WbItem m = ring[it & 3];
      if (m.n < 0) {  // the last item's sums
        if (it > 0 && wait_warp(e_free, (G & 1) ^ 1)) {
          tc_fence_after();
          Sums v;
          load_sums(v);
          tc_fence_before();
          store_sums(it - 1, v);
        }
        break;
      }
      const int row = m.t * WT + r;  // key (DKDV) or query (DQ) index in the sequence
      float lse_r = 0.f, di_r = 0.f;  // DQ: the row's, negative
      if (!DKDV) {
        // (in one half of the 32 bytes, as the swizzle has it; the other is zeros)
        const uint4* e = reinterpret_cast<const uint4*>(smem + WB_OFF_E + (it & 1) * WB_E_BYTES + r * 32);
        float x[8], y[8];
        load8_bf16(reinterpret_cast<const bf16*>(e), x);
        load8_bf16(reinterpret_cast<const bf16*>(e + 1), y);
        lse_r = (((x[2] + y[2]) + (x[1] + y[1])) + (x[0] + y[0])) * a.sl2;
        di_r = ((x[5] + y[5]) + (x[4] + y[4])) + (x[3] + y[3]);
      }
      // streamed tiles in which some pair of a row is hidden: the diagonal's, DKDV those from
      // `edge` on, past some key's window or the sequence's end, DQ those before it that are
      // not all sinks
      const int past = DKDV ? 0 : m.t * WT + WT - 1 - a.w.W;
      const int edge = DKDV ? min(m.t * WT + WT <= a.w.S ? a.w.n_t : m.t + a.w.W / WT, a.w.L / WT)
                            : past >= 0 ? past / WT + 1 : 0;
      const int whole = a.w.S / WT;
      WbStep<DKDV> sp(m);
      for (int j = 0; j < m.n; ++j, ++G) {
        const uint32_t Gj = G;
        const int yt = sp.tile, c0 = yt * WT;  // first streamed index of this step
        sp.next(m);
        const bool hidden = yt == m.t || (DKDV ? yt >= edge : yt < edge && yt >= whole);
        if (!wait_warp(t_full, Gj & 1)) {
          ok = false;
          break;
        }
        tc_fence_after();
        uint32_t sa[32], pa[32];  // this thread's 32 columns of T1 and T2
        tmem_ld32_async(tl + 32 * ch, sa);
        tmem_ld32_async(tl + WT + 32 * ch, pa);
        tmem_wait_ld(sa);
        tmem_wait_ld(pa);
        tc_fence_before();
        mbar_arrive_warp(t_free);
        // P and dS of the thread's 32 columns from kb on, as bf16 pairs
        auto emit = [&](auto masked, int kb, uint32_t* pk, uint32_t* dk) {
          if (decltype(masked)::value) {
            // visible streamed columns: [lo, hi), and (DQ) the sinks below sk; bit c of `vis`:
            // column kb + c
            auto low = [](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };
            const int b0 = c0 + kb;  // the first column's index
            const uint32_t vis =
                DKDV ? low((row < a.w.S ? a.w.L : min(a.w.L, row + a.w.W)) - b0) & ~low(row - b0)
                     : low(row + 1 - b0) & (~low(row - a.w.W + 1 - b0) | low(a.w.S - b0));
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!(vis >> c & 1)) sa[c] = 0xff800000u;  // -inf: P = 0, and dS with it
          }
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const uint32_t* sv = sa + g * 8;
            const uint32_t* dv = pa + g * 8;
            // packed fp32x2 arithmetic (each lane an IEEE fp32 operation)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 sl = make_float2(a.sl2, a.sl2);
              const float2 sv2 =
                  make_float2(__uint_as_float(sv[2 * e]), __uint_as_float(sv[2 * e + 1]));
              const float2 dv2 =
                  make_float2(__uint_as_float(dv[2 * e]), __uint_as_float(dv[2 * e + 1]));
              const float2 z = DKDV ? __fmul2_rn(sv2, sl)
                                    : __ffma2_rn(sv2, sl, make_float2(lse_r, lse_r));
              const float2 p = make_float2(ex2_approx(z.x), ex2_approx(z.y));
              const float2 ds =
                  __fmul2_rn(p, DKDV ? dv2 : __fadd2_rn(dv2, make_float2(di_r, di_r)));
              pk[4 * g + e] = pack_bf16(p.x, p.y);
              dk[4 * g + e] = pack_bf16(ds.x, ds.y);
            }
          }
        };
        uint32_t pk[16], dk[16];  // this thread's 32 columns of E1 and E2
        const int kb = 32 * ch;
        if (hidden)
          emit(std::true_type{}, kb, pk, dk);
        else
          emit(std::false_type{}, kb, pk, dk);
        if (!wait_warp(e_free, (Gj & 1) ^ 1)) {  // the previous step's E has been read
          ok = false;
          break;
        }
        tc_fence_after();
        // the last item's sums are complete too, and nothing adds to them before this step's E
        // is there
        auto put_e = [&]() {
          const uint32_t te = tl + WB_TM_E + 16 * ch;
          if (DKDV) tmem_st16(te, pk);
          tmem_st16(te + WT / 2, dk);
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive_warp(e_full);
        };
        if (j == 0 && it > 0) {
          Sums v;
          load_sums(v);
          put_e();
          store_sums(it - 1, v);
        } else {
          put_e();
        }
      }
    }
  }
  tc_fence_before();
  if (__syncthreads_or(*(volatile int*)&g_dev_error != 0)) {
    // error path: let this CTA's copies and MMAs land before smem / TMEM go
    if (warp == 0 && lane == 0) {
      for (uint32_t Gd = y_issued > WB_STAGES ? y_issued - WB_STAGES : 0; Gd < y_issued; ++Gd)
        mbar_wait_drain(y_full + 8 * (Gd % WB_STAGES), (Gd / WB_STAGES) & 1);
      for (uint32_t t = x_issued > 2 ? x_issued - 2 : 0; t < x_issued; ++t)
        mbar_wait_drain(x_full + 8 * (t & 1), (t >> 1) & 1);
    }
    if (warp == 1 && lane == 0) mbar_wait_drain(done, 0);
  } else if (warp == 1 && lane == 0) {
    mbar_wait(done, 0);
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, WB_TMEM_COLS);
  }
}

// Sums of a cut key tile's pieces, in order.  CTA (16 rows, key head and
// sequence, tile): 8 threads to a row, 16 columns of dV | dK each.
__global__ void __launch_bounds__(128) window_join_kernel(WbArgs a) {
  pdl_enter();
  const int per = a.KV * a.B, hb = blockIdx.y, h = hb % a.KV, b = hb / a.KV;
  const int t = (a.np_s > 1 ? 0 : a.w.sT) + blockIdx.z;  // cut tiles: the sinks', or all, or the others
  const bool sink = t < a.w.sT;
  const int np = sink ? a.np_s : a.np_w;
  const int first = (sink ? t * np : a.w.sT * a.np_s + (t - a.w.sT) * np) * per + hb;
  const int r = blockIdx.x * 16 + threadIdx.x / 8, col = threadIdx.x % 8 * 16, row = t * WT + r;
  if (row >= a.w.L) return;
  const int m = wb_queries(a.w, t), all = m * a.g;
  float v[16] = {};
  for (int s0 = 0, i = 0; s0 < all; s0 += a.C, ++i) {
    if (r >= wb_rows(a.w, t, m, s0, min(a.C, all - s0))) continue;
    const float4* p = reinterpret_cast<const float4*>(a.part + ((long)(first + i * per) * WT + r) * WB_ACC +
                                                      col);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float4 x = p[e];
      v[4 * e] += x.x; v[4 * e + 1] += x.y; v[4 * e + 2] += x.z; v[4 * e + 3] += x.w;
    }
  }
  const long srow = (long)b * a.w.L + row;
  bf16* o = col < WB_D ? a.out_u + srow * a.ld_u + h * WB_D + col
                       : a.out_w + srow * a.ld_w + h * WB_D + col - WB_D;
  if (col >= WB_D)
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= a.scale;
  store8_bf16(o, v);
  store8_bf16(o + 8, v + 8);
}

// Di = rowsum(dO * O) per (sequence, head, query) beside LSE, in three bf16 each (24 bits) as an MMA
// of DKDV takes them: eight lanes per (row, head), each eight of the head's 64 columns, of WB_DOT_U (row, head)s 32 apart, whose loads go out at once.
// (One to a lane, and 64-bit divisions to find it: 86 us for 65536 tokens of 16 heads, 72 so; four to a lane 76.)
constexpr int WB_DOT_U = 2;
__global__ void __launch_bounds__(256) window_dot_kernel(const bf16* dO, long lddo,
                                                         const bf16* O, long ldo,
                                                         const bf16* rest,
                                                         const float* lse,
                                                         bf16* ext,
                                                         long items, int L, int H) {
  pdl_enter();
  const long it0 = (long)blockIdx.x * (32 * WB_DOT_U);
  const int row0 = (int)(it0 / H), h0 = (int)(it0 - (long)row0 * H);  // the CTA's first
  const int sub = threadIdx.x & 7, i0 = threadIdx.x >> 3;
  uint4 x[WB_DOT_U], y[WB_DOT_U], z[WB_DOT_U];
  float l[WB_DOT_U];
  long at[WB_DOT_U];
#pragma unroll
  for (int u = 0; u < WB_DOT_U; ++u) {
    const long it = min(it0 + i0 + 32 * u, items - 1);
    const unsigned hh = h0 + (int)(it - it0), r = hh / (unsigned)H;
    const int row = row0 + (int)r, h = (int)(hh - r * H), b = row / L;
    x[u] = *reinterpret_cast<const uint4*>(dO + row * lddo + h * WB_D + sub * 8);
    y[u] = *reinterpret_cast<const uint4*>(O + row * ldo + h * WB_D + sub * 8);
    z[u] = *reinterpret_cast<const uint4*>(rest + it * WB_D + sub * 8);
    at[u] = ((long)b * H + h) * L + (row - b * L);
    l[u] = lse[at[u]];
  }
#pragma unroll
  for (int u = 0; u < WB_DOT_U; ++u) {
    float a[8], b[8], c[8], v = 0.f;
    load8_bf16(reinterpret_cast<const bf16*>(&x[u]), a);
    load8_bf16(reinterpret_cast<const bf16*>(&y[u]), b);
    load8_bf16(reinterpret_cast<const bf16*>(&z[u]), c);
#pragma unroll
    for (int k = 0; k < 8; ++k) v = fmaf(a[k], b[k] + c[k], v);
#pragma unroll
    for (int s = 4; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    if (it0 + i0 + 32 * u < items && sub < 2) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (sub == 0) {
        // three bf16 that add up to x
        auto split = [](float x, bf16* p) {
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            p[i] = __float2bfloat16(x);
            x -= __bfloat162float(p[i]);
          }
        };
        __align__(16) bf16 e[8] = {};
        split(l[u] * (-8.f * 0.6931471805599453f), e);  // 8 / log2(e): T1 is multiplied by its inverse
        split(-v, e + 3);
        w = *reinterpret_cast<const uint4*>(e);
      }
      *reinterpret_cast<uint4*>(ext + at[u] * WB_EXT + 8 * sub) = w;
    }
  }
}

// How the key tiles' steps are cut.  A key tile of the window takes g (W / 128 + 1)
// steps, one of the sinks g n_t.  With fewer tiles than SMs all are cut, into pieces of
// half an SM's share of the steps (at least two: a piece costs 64 KB, written and read);
// else only the sinks', into pieces of a sixteenth of it, or of a window's tile.
struct Cut {
  int C, np_s, np_w;
  long items;
};
Cut wb_cut(const Window& c) {
  constexpr long SMS = 152;  // whatever the device has: the sums keep their order
  const WinTiles w(c);
  const long g = c.H / c.KV, heads = (long)c.KV * c.B;
  long steps = 0, longest = 0;  // of a key head; of its longest tile that is not the sinks'
  for (int t = 0; t < w.n_t; ++t) {
    const long n = wb_queries(w, t) * g;
    steps += n;
    if (t >= w.sT) longest = std::max(longest, n);
  }
  Cut r;
  r.C = (int)(w.n_t * heads < SMS ? std::max(2L, steps * heads / (2 * SMS))
                                  : std::max(longest, steps * heads / (16 * SMS)));
  const long sink = w.sT > 0 ? wb_queries(w, 0) * g : 1;
  r.np_s = (int)((sink + r.C - 1) / r.C);
  r.np_w = (int)std::max(1L, (longest + r.C - 1) / r.C);
  r.items = heads * ((long)w.sT * r.np_s + (long)(w.n_t - w.sT) * r.np_w);
  return r;
}

struct WbWs {
  float* part;
  bf16* ext;  // [B, H, L][16]
  size_t bytes;
};
WbWs wb_carve(void* ws, const Window& c) {
  auto up = [](size_t n) { return (n + 255) & ~size_t(255); };
  const WinTiles w(c);
  const Cut k = wb_cut(c);
  WbWs r;
  const size_t ext = up((size_t)c.B * c.H * c.L * WB_EXT * sizeof(bf16));
  r.ext = static_cast<bf16*>(ws);
  r.part = reinterpret_cast<float*>(static_cast<char*>(ws) + ext);
  // pieces are numbered as the items, the sinks' first
  const long pieces = k.np_w > 1 ? k.items : k.np_s > 1 ? (long)c.KV * c.B * w.sT * k.np_s : 0;
  r.bytes = ext + (size_t)pieces * WT * WB_ACC * sizeof(float) + 256;
  return r;
}

template <bool DKDV>
cudaError_t wb_launch(const CUtensorMap& x1, const CUtensorMap& x2, const CUtensorMap& y1,
                      const CUtensorMap& y2, const CUtensorMap& te, const CUtensorMap& u,
                      const CUtensorMap& w, const WbArgs& a, const char* label, double flops, double bytes,
                      cudaStream_t st) {
  auto kern = window_bwd_kernel<DKDV>;
  static KernelOnce once;
  const cudaError_t e = once(reinterpret_cast<const void*>(kern), WB_SMEM, WB_THREADS,
                             WB_REGS_CTRL * 128 + WB_REGS_ROWS * 512);
  if (e != cudaSuccess) return e;
  LaunchTimer lt(label, st, flops, bytes);
  const int grid = std::min(a.n_items, num_sms());
  return launch_kernel(kern, grid, WB_THREADS, WB_SMEM, st, x1, x2, y1, y2, te, u, w, a);
}

}  // namespace

size_t window_bwd_ws_bytes(const Window& c) { return wb_carve(nullptr, c).bytes; }

cudaError_t window_bwd(const Window& c, const QkvPtr& x, const bf16* out, long ldo,
                       const WindowSaved& v, const bf16* dout, long lddo, const QkvPtr& dx, void* ws,
                       cudaStream_t st) {
  launched.mark();
  CUtensorMap tq, tk, tv, td, te, gq, gk, gv;
  if (!tmap_bf16_seq(&tq, x.q, (uint64_t)c.H * WB_D, c.L, c.B, x.ldq, WB_D, WT) ||
      !tmap_bf16_seq(&tk, x.k, (uint64_t)c.KV * WB_D, c.L, c.B, x.ldk, WB_D, WT) ||
      !tmap_bf16_seq(&tv, x.v, (uint64_t)c.KV * WB_D, c.L, c.B, x.ldv, WB_D, WT) ||
      !tmap_bf16_seq(&td, dout, (uint64_t)c.H * WB_D, c.L, c.B, lddo, WB_D, WT) ||
      !tmap_bf16_seq(&gq, dx.q, (uint64_t)c.H * WB_D, c.L, c.B, dx.ldq, WB_D, WT) ||
      !tmap_bf16_seq(&gk, dx.k, (uint64_t)c.KV * WB_D, c.L, c.B, dx.ldk, WB_D, WT) ||
      !tmap_bf16_seq(&gv, dx.v, (uint64_t)c.KV * WB_D, c.L, c.B, dx.ldv, WB_D, WT))
    return cudaErrorInvalidValue;
  const WbWs wk = wb_carve(ws, c);
  if (!tmap_bf16_rows32(&te, wk.ext, c.L, (uint64_t)c.B * c.H, WT)) return cudaErrorInvalidValue;
  WbArgs a{};
  a.part = wk.part;
  a.B = c.B; a.H = c.H; a.KV = c.KV; a.g = c.H / c.KV;
  a.w = WinTiles(c);
  const Cut k = wb_cut(c);
  a.C = k.C; a.np_s = k.np_s; a.np_w = k.np_w;
  a.scale = 1.0f / sqrtf((float)WB_D);
  a.sl2 = a.scale * 1.4426950408889634f;
  const long q_items = (long)a.w.n_t * c.H * c.B;
  if (k.items > 0x3fffffff || q_items > 0x3fffffff) return cudaErrorInvalidValue;
  const double rows = (double)c.B * c.L, pairs = (double)c.B * c.H * window_pairs(c);
  cudaError_t e;
  {
    LaunchTimer lt("window_bwd_dot", st, 2.0 * rows * c.H * WB_D, rows * c.H * (6.0 * WB_D + 4.0 + 2.0 * WB_EXT));
    const long n = (long)c.B * c.L * c.H;
    e = launch_kernel(window_dot_kernel, (unsigned)((n + 32 * WB_DOT_U - 1) / (32 * WB_DOT_U)), 256, 0, st,
                      dout, lddo, out, ldo, v.rest, v.lse, wk.ext, n, c.L, c.H);
    if (e != cudaSuccess) return e;
  }
  a.out_u = static_cast<bf16*>(dx.v);
  a.ld_u = dx.ldv;
  a.out_w = static_cast<bf16*>(dx.k);
  a.ld_w = dx.ldk;
  a.n_items = (int)k.items;
  e = wb_launch<true>(tk, tv, tq, td, te, gv, gk, a, "window_bwd_dkdv", 8.0 * WB_D * pairs,
                      2.0 * rows * WB_D * (2.0 * c.H + 4.0 * c.KV), st);
  if (e != cudaSuccess) return e;
  const int cut = (k.np_s > 1 ? a.w.sT : 0) + (k.np_w > 1 ? a.w.n_t - a.w.sT : 0);
  if (cut > 0) {
    LaunchTimer lt("window_bwd_join", st, 0.0, 0.0);
    e = launch_kernel(window_join_kernel, dim3(WT / 16, c.KV * c.B, cut), 128, 0, st, a);
    if (e != cudaSuccess) return e;
  }
  a.n_items = (int)q_items;
  return wb_launch<false>(tq, td, tk, tv, te, gq, gq, a, "window_bwd_dq", 6.0 * WB_D * pairs,
                          2.0 * rows * WB_D * (3.0 * c.H + 2.0 * c.KV), st);
}

}  // namespace pf

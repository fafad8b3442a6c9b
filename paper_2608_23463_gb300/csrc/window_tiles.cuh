// Which 128-row tiles of keys the 128-row tiles of queries see, for causal
// attention in a sliding window with sinks (window_attn.cu, window_attn_bwd.cu).
#pragma once

#include "local.h"

namespace pf {

constexpr int WT = 128;  // rows of a tile
constexpr int WT_FEW = 32;  // so few sinks of a tile before the window are a narrower tile

struct WinTiles {
  int L, W, S;  // length; window (L: no limit); sinks below the window
  int n_t, sT;  // tiles of the sequence, and those that hold sinks
  int few;      // the last of those if it holds WT_FEW sinks at most, else -1
  WinTiles() = default;
  explicit WinTiles(const Window& c) {
    L = c.L;
    W = c.window > 0 && c.window < c.L ? c.window : c.L;
    S = W < L ? (c.sinks < L ? c.sinks : L) : 0;  // a window of everything holds the sinks
    n_t = (L + WT - 1) / WT;
    sT = (S + WT - 1) / WT;
    few = sT > 0 && S - (sT - 1) * WT <= WT_FEW ? sT - 1 : -1;
  }
  // first tile of the window of query tile t
  __host__ __device__ __forceinline__ int lo(int t) const {
    const int k = t * WT - W + 1;
    return k > 0 ? k / WT : 0;
  }
  // last query tile with key tile t in its window
  __host__ __device__ __forceinline__ int last_q(int t) const {
    const long q = ((long)t * WT + WT - 1 + W - 1) / WT;
    return q < n_t - 1 ? (int)q : n_t - 1;
  }
};

// A tile of the map's rows from shared memory, 128-byte swizzle (rows past the end of the
// sequence are left out).
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t saddr, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                   map),
               "r"(x), "r"(y), "r"(z), "r"(saddr)
               : "memory");
}

}  // namespace pf

// How the attention of many new tokens over a paged cache is cut into work (paged_chunk.cu).
//
// An item is (sequence, key head, two query tiles): a tile holds tpt = 128 / g tokens with
// the g query heads of the key head, g rows to a token, so that a row of K and V serves all
// of them.  Its steps are the 128-row tiles of the cache that its tokens see: the sinks' [0,
// ns) and the window's [lo, ...], without those in between.
// The items of all sequences stand in one line, (sequence, head, pair), each as long as its
// weight, and the CTAs share the line out evenly: one may begin and end inside an item.
// Weights within a sequence have a closed sum, so that a CTA finds its part from the
// sequences' totals alone.
#pragma once

#include <stdint.h>

namespace pf {

constexpr int PC_T = 128;  // rows of a query tile, keys of a step

struct PcGeo {
  int B, KV, g, tpt;
  int W, S;  // window (0: none), sinks
};

// A sequence: its new tokens are [t0, t0 + n) of the call's, the last n of its len rows.
struct PcSeq {
  int t0, n, len;
};

// A place in the line: step s of an item; b = B: its end.
struct PcAt {
  int b, h, u, s;
};

struct PcSpan {
  int pf, pl;  // positions of the first and the last token
  int ns, lo, steps;
  __host__ __device__ __forceinline__ int tile(int s) const { return s < ns ? s : lo + s - ns; }
};

__host__ __device__ __forceinline__ int pc_tiles(int rows) { return rows / PC_T + (rows % PC_T != 0); }
__host__ __device__ __forceinline__ int pc_pairs(const PcGeo& g, const PcSeq& q) {
  const unsigned R = 2 * g.tpt;
  return (int)((q.n + (R - 1)) / R);  // (0 <= n: unsigned, which takes fewer instructions)
}

__host__ __device__ __forceinline__ PcSpan pc_span(const PcGeo& g, const PcSeq& q, int u) {
  const int R = 2 * g.tpt, a = u * R, p0 = q.len - q.n;
  PcSpan s;
  s.pf = p0 + a;
  s.pl = p0 + (q.n - a < R ? q.n : a + R) - 1;
  s.lo = g.W > 0 && s.pf >= g.W ? (s.pf - g.W + 1) / PC_T : 0;
  const int sT = g.W > 0 ? pc_tiles(g.S) : 0;
  s.ns = sT < s.lo ? sT : s.lo;
  s.steps = s.ns + s.pl / PC_T - s.lo + 1;
  return s;
}

// What an item weighs, about in 8 cycles: a key (that its last token sees, of those that a full pair
// there would) 3, with one tile 2, half a step more for the last one's rest, and its beginning and end,
// some 8000 cycles.  (ITEM at 700, 1000 and 2000: three short sequences 15.5, 12.9 and 13.1 us, four
// quantised prompts 166.7, 166.8 and 175.2; a single tile's key at 1.5, 2 and 2.5: 64 mixed sequences
// 81.6, 80.0 and 89.4.)  The sum over the pairs before u, of P.
__host__ __device__ __forceinline__ long long pc_cum(const PcGeo& g, const PcSeq& q, int u, int P) {
  constexpr int ITEM = 1000, REST = 64;
  const int R = 2 * g.tpt, p0 = q.len - q.n;
  const long long cap = (long long)g.W + g.S + R;
  auto sum = [&](int n) {  // of keys
    int k = n;  // pairs that see no more than cap
    if (g.W > 0 && p0 + (long long)R * n > cap) k = cap > p0 ? (int)((unsigned)(cap - p0) / (unsigned)R) : 0;
    return (long long)k * p0 + R * ((long long)k * (k + 1) / 2) + (n - k) * cap + (long long)n * REST;
  };
  const bool single = u == P && q.n - (P - 1) * R <= g.tpt;
  const long long keys = sum(u);
  return 3 * keys - (single ? keys - sum(u - 1) : 0) + (long long)u * ITEM;
}

__host__ __device__ __forceinline__ float pc_quotient(float a, float b) {
#ifdef __CUDA_ARCH__
  return __fdividef(a, b);
#else
  return a / b;
#endif
}

// The step at weight y of a pair that weighs so much.  Neither this nor pc_share has to be exact, only
// the same for whoever asks, and to grow with y or c: a division of 64-bit numbers, cold, took 1000
// cycles of a call's first 20000.
__host__ __device__ __forceinline__ int pc_step(int steps, long long y, long long weight) {
  if (y <= 0) return 0;
  const int s = (int)(pc_quotient((float)y, (float)weight) * (float)steps);
  return s < steps ? s : steps - 1;
}

// The head of weight y, of `per` each; y becomes what is left.
__host__ __device__ __forceinline__ int pc_head(long long per, long long& y) {
  int h = (int)pc_quotient((float)y, (float)per);
  while (h > 0 && h * per > y) --h;  // (off by one at most)
  while ((h + 1) * per <= y) ++h;
  y -= h * per;
  return h;
}

// Where CTA c of n begins on a line of length T.
__host__ __device__ __forceinline__ long long pc_share(long long T, int n, int c) {
  if (c >= n) return T;
  const unsigned f = (unsigned)(pc_quotient((float)c, (float)n) * 4294967296.f);  // c <= 151, n <= 152: below 2^32
  return (long long)(((unsigned long long)T >> 32) * f + ((((unsigned long long)T & 0xffffffffu) * f) >> 32));
}

}  // namespace pf

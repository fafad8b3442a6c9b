// Internal launch interface of the local stream's attention operators
// (local_api.cu checks the arguments, the kernels are in local_rope.cu,
// paged_attn.cu, window_attn.cu and window_attn_bwd.cu).
#pragma once

#include <atomic>

#include "kernels.h"

namespace pf {

// What a kernel needs of the device before its first launch there: its shared memory, and
// (pool > 0) that its threads, `threads` of them, bring the `pool` registers that its warps
// share out among themselves (setmaxnreg): with fewer they would wait for ever.  Asked
// once per device and kernel: asked on every call, it took 2 of a small call's 14 us.
struct KernelOnce {
  std::atomic<unsigned long long> done{0};  // a bit per device
  cudaError_t operator()(const void* kern, int smem, int threads = 0, int pool = 0) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    if (pool > 0) {
      cudaFuncAttributes at;
      if ((e = cudaFuncGetAttributes(&at, kern)) != cudaSuccess) return e;
      if (at.numRegs * threads < pool) return cudaErrorInvalidConfiguration;
    }
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
  }
};

// Whether a file's kernels were ever launched, or recorded in a graph: pf_sync_check reads the
// error word of those that were (about 9 us each; 12 files take 108 us, the 8 without these 72).
struct Launched {
  std::atomic<bool> any{false};
  void mark() {
    if (!any.load(std::memory_order_relaxed)) any.store(true, std::memory_order_relaxed);
  }
  int take(int (*read)()) const { return any.load(std::memory_order_relaxed) ? read() : 0; }
};

// Rows of three matrices, leading dimensions in elements (of bf16 or fp32).
struct QkvPtr {
  void *q, *k, *v;
  long ldq, ldk, ldv;
};

struct QkRope {
  int H, KV, dh, f32, n_axes, pairs[3];
  double theta, eps;
};

struct Paged {
  int B, H, KV, dh, page, max_pages;
  long n_pages;
  int window, sinks;
  bf16 *K, *V;  // [n_pages, KV, page, dh]
  const int *table, *len;
};

// Windowed attention of B sequences of L rows: H query and KV key heads of 64.
struct Window {
  int B, L, H, KV, window, sinks;  // window 0: no limit
};
double window_pairs(const Window& c);  // visible (query, key) pairs of a head and sequence
// What the forward keeps for the backward: the rows' log-sums [B, H, L] in log2 units,
// and the output's rest [B * L, H * 64], out + rest being the output to 2^-17.
struct WindowSaved {
  float* lse;
  bf16* rest;
  size_t bytes;
};
WindowSaved window_saved(const Window& c, void* p);
// v.lse null: nothing is kept
cudaError_t window_fwd(const Window& c, const QkvPtr& x, bf16* out, long ldo, const WindowSaved& v,
                       cudaStream_t st);
size_t window_bwd_ws_bytes(const Window& c);
cudaError_t window_bwd(const Window& c, const QkvPtr& x, const bf16* out, long ldo,
                       const WindowSaved& v, const bf16* dout, long lddo, const QkvPtr& dx, void* ws,
                       cudaStream_t st);

cudaError_t qk_rope_fwd(const QkRope& s, const QkvPtr& x, const QkvPtr& o, const float* w_q,
                        const float* w_k, const int* pos, long rows, long seq_len,
                        cudaStream_t st);
// part: qk_rope_part_bytes(dh), read and written only with dw_q or dw_k.
size_t qk_rope_part_bytes(int dh);
cudaError_t qk_rope_bwd(const QkRope& s, const QkvPtr& x, const QkvPtr& dout, const QkvPtr& dx,
                        const float* w_q, const float* w_k, const int* pos, float* dw_q,
                        float* dw_k, float* part, long rows, long seq_len, cudaStream_t st);
cudaError_t paged_append(const QkRope& s, const Paged& c, const QkvPtr& x, bf16* q_out, long ldqo,
                         const float* w_q, const float* w_k, const int* start, const int* pos,
                         long rows, cudaStream_t st);
cudaError_t paged_advance(const Paged& c, const int* start, int* len, cudaStream_t st);

#define PF_PAGED_MAX_BATCH 2048  // sequences of a call
#define PF_PAGED_ROWS 16         // a page holds a multiple of so many rows
size_t paged_attn_ws_bytes(const Paged& c);
cudaError_t paged_attn(const Paged& c, const bf16* q, long ldq, bf16* out, long ldo, float* ws,
                       cudaStream_t st);

int take_dev_error_local_rope();
int take_dev_error_paged_attn();
int take_dev_error_window_attn();
int take_dev_error_window_attn_bwd();
int set_wait_limit_local_rope(unsigned long long ns);
int set_wait_limit_paged_attn(unsigned long long ns);
int set_wait_limit_window_attn(unsigned long long ns);
int set_wait_limit_window_attn_bwd(unsigned long long ns);

}  // namespace pf

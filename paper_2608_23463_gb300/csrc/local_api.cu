// C ABI of the local stream's attention operators (include/proxyformer.h):
// argument validation and the launches.
#include <stdarg.h>
#include <stdio.h>

#include "local.h"
#include "proxyformer.h"

using namespace pf;

pf_status pf_set_error(pf_status s, const char* msg);

namespace {

pf_status fail(pf_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return pf_set_error(s, buf);
}

#define PF_CUDA(call)                                                                 \
  do {                                                                                \
    cudaError_t e_ = (call);                                                          \
    if (e_ != cudaSuccess) return fail(PF_ERR_CUDA, "%s: %s", #call, cudaGetErrorString(e_)); \
  } while (0)

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Rows of a matrix: present, aligned, wide enough.
pf_status check_rows(const char* name, const void* p, int64_t ld, int64_t width, int size) {
  if (!p || !aligned16(p)) return fail(PF_ERR_INVALID_ARG, "%s is required, 16-byte aligned", name);
  if (ld < width || ld * size % 16 != 0 || ld > (int64_t(1) << 31))
    return fail(PF_ERR_INVALID_ARG, "%s: leading dimension %lld, needs at least %lld and whole 16 bytes",
                name, (long long)ld, (long long)width);
  return PF_OK;
}

// A matrix in memory, in bytes.
struct Area {
  const char* name;
  const void* p;
  int64_t rows, width, ld;
};

// Whether two matrices share a byte.  Columns of one wide matrix do not meet.
bool meet(const Area& a, const Area& b) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  if (pa >= pb + (b.rows - 1) * b.ld + b.width || pb >= pa + (a.rows - 1) * a.ld + a.width) return false;
  if (a.ld == b.ld) {
    // b's rows begin at column r of a's rows j, j + 1, ..., and may reach into the rows after those
    const int64_t d = static_cast<int64_t>(pb - pa);
    const int64_t j = d >= 0 ? d / a.ld : -((a.ld - 1 - d) / a.ld), r = d - j * a.ld;
    auto rows = [&](int64_t first) { return first < a.rows && -first < b.rows; };
    return (r < a.width && rows(j)) || (r + b.width > a.ld && rows(j + 1));
  }
  const bool swap = b.rows < a.rows;  // the rows of the one with fewer, among the other's
  const Area &x = swap ? b : a, &y = swap ? a : b;
  const uintptr_t px = swap ? pb : pa, py = swap ? pa : pb;
  for (int64_t i = 0; i < x.rows; ++i) {
    const int64_t at = static_cast<int64_t>(px - py) + i * x.ld;  // from y's first byte
    const int64_t k = at < y.width ? 0 : (at - y.width) / y.ld + 1;  // y's first row that ends after it
    if (k < y.rows && k * y.ld < at + x.width) return true;
  }
  return false;
}

// A result must lie apart from what is read or written beside it.
pf_status check_apart(const Area& out, const Area& other) {
  if (!meet(out, other)) return PF_OK;
  return fail(PF_ERR_INVALID_ARG, "%s overlaps %s", out.name, other.name);
}

#define PF_TRY(call)                     \
  do {                                   \
    pf_status s_ = (call);               \
    if (s_ != PF_OK) return s_;          \
  } while (0)

pf_status check_heads(int32_t H, int32_t KV, int32_t dh) {
  if (H < 1 || KV < 1 || H % KV != 0)
    return fail(PF_ERR_INVALID_ARG, "n_heads must be a positive multiple of n_kv");
  if (H > 4096) return fail(PF_ERR_UNSUPPORTED, "at most 4096 heads");
  if (dh != 64 && dh != 128) return fail(PF_ERR_UNSUPPORTED, "head width must be 64 or 128");
  return PF_OK;
}

pf_status check_qk(const pf_qk_desc* s) {
  if (!s) return fail(PF_ERR_INVALID_ARG, "qk descriptor is NULL");
  PF_TRY(check_heads(s->n_heads, s->n_kv, s->dh));
  if (s->dtype != PF_BF16 && s->dtype != PF_F32)
    return fail(PF_ERR_INVALID_ARG, "dtype must be PF_BF16 or PF_F32");
  if (s->n_axes < 0 || s->n_axes > 3) return fail(PF_ERR_INVALID_ARG, "n_axes must be in [0, 3]");
  int64_t p = 0;
  for (int i = 0; i < s->n_axes; ++i) {
    if (s->pairs[i] < 0) return fail(PF_ERR_INVALID_ARG, "pairs must not be negative");
    p += s->pairs[i];
  }
  if (p > s->dh / 2) return fail(PF_ERR_INVALID_ARG, "more pairs than the head holds");
  if (!(s->theta >= 1e-300) || !(s->eps > 0) || s->theta > 1e300)
    return fail(PF_ERR_INVALID_ARG, "theta must be in [1e-300, 1e300] and eps positive");
  return PF_OK;
}

QkRope rope_of(const pf_qk_desc& s) {
  QkRope r{s.n_heads, s.n_kv, s.dh, s.dtype == PF_F32, s.n_axes, {0, 0, 0}, s.theta, s.eps};
  for (int i = 0; i < s.n_axes; ++i) r.pairs[i] = s.pairs[i];
  return r;
}

QkvPtr ptr_of(const pf_qkv& x) {
  return {x.q, x.k, x.v, (long)x.ld_q, (long)x.ld_k, (long)x.ld_v};
}

pf_status check_qk_rows(const char* what, const pf_qkv* x, const pf_qk_desc& s) {
  if (!x) return fail(PF_ERR_INVALID_ARG, "%s is NULL", what);
  const int size = s.dtype == PF_F32 ? 4 : 2;
  PF_TRY(check_rows("q", x->q, x->ld_q, (int64_t)s.n_heads * s.dh, size));
  return check_rows("k", x->k, x->ld_k, (int64_t)s.n_kv * s.dh, size);
}

Area head_area(const char* name, const void* p, int64_t rows, int64_t ld, int32_t heads, int32_t dh, int size) {
  return {name, p, rows, (int64_t)heads * dh * size, ld * size};
}

// A result that may lie over the input that it comes from, value for value.
pf_status check_over(const Area& out, const Area& from) {
  if (out.p == from.p && (out.ld == from.ld || out.rows == 1)) return PF_OK;
  return check_apart(out, from);
}

// Results of queries and keys: each may lie over its own input, and apart from all else
// that is read (read_q, read_k: of `in`, what is).
pf_status check_qk_results(const pf_qk_desc& s, int64_t rows, const pf_qkv& out, const pf_qkv& in, bool read_q,
                           bool read_k) {
  const int size = s.dtype == PF_F32 ? 4 : 2;
  const Area oq = head_area("the result q", out.q, rows, out.ld_q, s.n_heads, s.dh, size),
             ok = head_area("the result k", out.k, rows, out.ld_k, s.n_kv, s.dh, size),
             q = head_area("q", in.q, rows, in.ld_q, s.n_heads, s.dh, size),
             k = head_area("k", in.k, rows, in.ld_k, s.n_kv, s.dh, size);
  if (read_q) {
    PF_TRY(check_over(oq, q));
    PF_TRY(check_apart(ok, q));
  }
  if (read_k) {
    PF_TRY(check_over(ok, k));
    PF_TRY(check_apart(oq, k));
  }
  return check_apart(oq, ok);
}

pf_status check_count(int64_t rows, int64_t seq_len, const int32_t* pos, int n_axes) {
  if (rows < 0 || rows > 0x7fffffff) return fail(PF_ERR_INVALID_ARG, "rows must be in [0, 2^31)");
  if (!pos && n_axes > 1) return fail(PF_ERR_INVALID_ARG, "several axes need positions");
  if (!pos && (seq_len < 1 || seq_len > 0x7fffffff))
    return fail(PF_ERR_INVALID_ARG, "seq_len must be in [1, 2^31)");
  return PF_OK;
}

pf_status check_window(const pf_window_desc* s) {
  if (!s) return fail(PF_ERR_INVALID_ARG, "window descriptor is NULL");
  if (s->batch < 1 || s->L < 1) return fail(PF_ERR_INVALID_ARG, "batch and L must be >= 1");
  if (s->L >= 1 << 30 || (int64_t)s->batch * s->L >= int64_t(1) << 31)
    return fail(PF_ERR_UNSUPPORTED, "L must be below 2^30 and batch * L below 2^31");
  PF_TRY(check_heads(s->n_heads, s->n_kv, s->dh));
  if (s->dh != 64) return fail(PF_ERR_UNSUPPORTED, "windowed attention: head width must be 64");
  if ((int64_t)s->batch * s->n_heads * ((s->L + 127) / 128) >= 1 << 28)
    return fail(PF_ERR_UNSUPPORTED, "too many query tiles");
  if (s->window < 0 || s->n_sink < 0)
    return fail(PF_ERR_INVALID_ARG, "window and n_sink must not be negative");
  return PF_OK;
}

Window window_of(const pf_window_desc& s) {
  return {s.batch, s.L, s.n_heads, s.n_kv, s.window, s.n_sink};
}

pf_status check_window_rows(const char* what, const pf_qkv* x, const pf_window_desc& s) {
  if (!x) return fail(PF_ERR_INVALID_ARG, "%s is NULL", what);
  const int64_t nq = (int64_t)s.n_heads * s.dh, nk = (int64_t)s.n_kv * s.dh;
  PF_TRY(check_rows("q", x->q, x->ld_q, nq, 2));
  PF_TRY(check_rows("k", x->k, x->ld_k, nk, 2));
  return check_rows("v", x->v, x->ld_v, nk, 2);
}

// The matrices of bf16 heads of a windowed call.
Area window_area(const pf_window_desc& s, const char* name, const void* p, int64_t ld, int32_t heads) {
  return head_area(name, p, (int64_t)s.batch * s.L, ld, heads, s.dh, 2);
}

pf_status check_paged(const pf_paged_desc* s) {
  if (!s) return fail(PF_ERR_INVALID_ARG, "paged descriptor is NULL");
  if (s->batch < 1) return fail(PF_ERR_INVALID_ARG, "batch must be >= 1");
  if (s->batch > PF_PAGED_MAX_BATCH)
    return fail(PF_ERR_UNSUPPORTED, "at most %d sequences", PF_PAGED_MAX_BATCH);
  PF_TRY(check_heads(s->n_heads, s->n_kv, s->dh));
  if (s->n_heads / s->n_kv > 16)
    return fail(PF_ERR_UNSUPPORTED, "at most 16 query heads to a key head");
  if (s->page < PF_PAGED_ROWS || s->page % PF_PAGED_ROWS != 0)
    return fail(PF_ERR_INVALID_ARG, "page must be a multiple of %d", PF_PAGED_ROWS);
  if (s->max_pages < 1 || s->n_pages < 1 || s->n_pages > 0x7fffffff)
    return fail(PF_ERR_INVALID_ARG, "max_pages and n_pages must be positive");
  if (s->window < 0 || s->n_sink < 0)
    return fail(PF_ERR_INVALID_ARG, "window and n_sink must not be negative");
  return PF_OK;
}

pf_status check_cache(const pf_paged_cache* c) {
  if (!c || !c->K || !c->V || !c->table || !c->len || !aligned16(c->K) || !aligned16(c->V))
    return fail(PF_ERR_INVALID_ARG, "K, V (16-byte aligned), table and len are required");
  return PF_OK;
}

// Of a quantised cache; e NULL: none is.
pf_status check_exp(const pf_paged_exp* e) {
  if (e && (!e->K || !e->V || !aligned16(e->K) || !aligned16(e->V)))
    return fail(PF_ERR_INVALID_ARG, "the exponents of K and V are required, 16-byte aligned");
  return PF_OK;
}

Paged paged_of(const pf_paged_desc& s, const pf_paged_cache* c, const pf_paged_exp* e = nullptr) {
  Paged p{s.batch, s.n_heads, s.n_kv, s.dh, s.page, s.max_pages, (long)s.n_pages, s.window, s.n_sink,
          nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
  if (e) {
    p.Ke = reinterpret_cast<signed char*>(e->K);
    p.Ve = reinterpret_cast<signed char*>(e->V);
  }
  if (c) {
    p.K = static_cast<bf16*>(c->K);
    p.V = static_cast<bf16*>(c->V);
    p.table = c->table;
    p.len = c->len;
  }
  return p;
}

pf_status append(const pf_paged_desc* desc, const pf_qk_desc* qk, int64_t rows, const pf_qkv* x, const float* w_q,
                 const float* w_k, const int32_t* start, const int32_t* pos, const pf_paged_cache* cache,
                 const pf_paged_exp* exp, void* q_out, int64_t ld_q_out, void* stream) {
  PF_TRY(check_paged(desc));
  PF_TRY(check_qk(qk));
  if (qk->n_heads != desc->n_heads || qk->n_kv != desc->n_kv || qk->dh != desc->dh)
    return fail(PF_ERR_INVALID_ARG, "the two descriptors' heads differ");
  if (qk->dtype != PF_BF16) return fail(PF_ERR_UNSUPPORTED, "the paged cache takes bf16");
  PF_TRY(check_count(rows, 1, pos, qk->n_axes));
  if (!start && rows != desc->batch)
    return fail(PF_ERR_INVALID_ARG, "without start every sequence has one token: rows must be batch");
  PF_TRY(check_cache(cache));
  PF_TRY(check_exp(exp));
  if (rows == 0) return PF_OK;
  if (!x) return fail(PF_ERR_INVALID_ARG, "x is NULL");
  if ((x->q == nullptr) != (q_out == nullptr))
    return fail(PF_ERR_INVALID_ARG, "x->q and q_out go together");
  if (q_out) {
    PF_TRY(check_rows("q", x->q, x->ld_q, (int64_t)desc->n_heads * desc->dh, 2));
    PF_TRY(check_rows("q_out", q_out, ld_q_out, (int64_t)desc->n_heads * desc->dh, 2));
  }
  PF_TRY(check_rows("k", x->k, x->ld_k, (int64_t)desc->n_kv * desc->dh, 2));
  PF_TRY(check_rows("v", x->v, x->ld_v, (int64_t)desc->n_kv * desc->dh, 2));
  if (q_out) {
    const Area o = head_area("q_out", q_out, rows, ld_q_out, desc->n_heads, desc->dh, 2);
    PF_TRY(check_over(o, head_area("q", x->q, rows, x->ld_q, desc->n_heads, desc->dh, 2)));
    PF_TRY(check_apart(o, head_area("k", x->k, rows, x->ld_k, desc->n_kv, desc->dh, 2)));
    PF_TRY(check_apart(o, head_area("v", x->v, rows, x->ld_v, desc->n_kv, desc->dh, 2)));
  }
  QkRope r = rope_of(*qk);
  if (!q_out) r.H = 0;
  PF_CUDA(paged_append(r, paged_of(*desc, cache, exp), ptr_of(*x), static_cast<bf16*>(q_out), (long)ld_q_out,
                       w_q, w_k, start, pos, rows, static_cast<cudaStream_t>(stream)));
  return PF_OK;
}

pf_status attn(const pf_paged_desc* desc, const void* q, int64_t ld_q, const pf_paged_cache* cache,
               const pf_paged_exp* exp, void* out, int64_t ld_out, void* ws, size_t ws_bytes, void* stream) {
  PF_TRY(check_paged(desc));
  PF_TRY(check_rows("q", q, ld_q, (int64_t)desc->n_heads * desc->dh, 2));
  PF_TRY(check_rows("out", out, ld_out, (int64_t)desc->n_heads * desc->dh, 2));
  PF_TRY(check_cache(cache));
  PF_TRY(check_exp(exp));
  const Paged p = paged_of(*desc, cache, exp);
  const size_t need = paged_attn_ws_bytes(p, exp != nullptr);
  if (!ws || !aligned16(ws) || ws_bytes < need)
    return fail(PF_ERR_WORKSPACE, "workspace too small: need %zu bytes, got %zu", need,
                ws ? ws_bytes : 0);
  // (a head's query is read before its row is written)
  PF_TRY(check_over(head_area("out", out, desc->batch, ld_out, desc->n_heads, desc->dh, 2),
                    head_area("q", q, desc->batch, ld_q, desc->n_heads, desc->dh, 2)));
  PF_CUDA(paged_attn(p, static_cast<const bf16*>(q), (long)ld_q, static_cast<bf16*>(out), (long)ld_out,
                     static_cast<float*>(ws), static_cast<cudaStream_t>(stream)));
  return PF_OK;
}

}  // namespace

extern "C" {

pf_status pf_qk_rope_fwd(const pf_qk_desc* desc, int64_t rows, int64_t seq_len, const pf_qkv* x,
                         const float* w_q, const float* w_k, const int32_t* pos,
                         const pf_qkv* out, void* stream) {
  PF_TRY(check_qk(desc));
  PF_TRY(check_count(rows, seq_len, pos, desc->n_axes));
  if (rows == 0) return PF_OK;
  PF_TRY(check_qk_rows("x", x, *desc));
  PF_TRY(check_qk_rows("out", out, *desc));
  PF_TRY(check_qk_results(*desc, rows, *out, *x, true, true));
  PF_CUDA(qk_rope_fwd(rope_of(*desc), ptr_of(*x), ptr_of(*out), w_q, w_k, pos, rows, seq_len,
                      static_cast<cudaStream_t>(stream)));
  return PF_OK;
}

size_t pf_qk_rope_workspace_size(const pf_qk_desc* desc) {
  return check_qk(desc) == PF_OK ? qk_rope_part_bytes(desc->dh) : 0;
}

pf_status pf_qk_rope_bwd(const pf_qk_desc* desc, int64_t rows, int64_t seq_len, const pf_qkv* x,
                         const float* w_q, const float* w_k, const int32_t* pos,
                         const pf_qkv* dout, const pf_qkv* dx, float* dw_q, float* dw_k, void* ws,
                         size_t ws_bytes, void* stream) {
  PF_TRY(check_qk(desc));
  PF_TRY(check_count(rows, seq_len, pos, desc->n_axes));
  if ((dw_q && !w_q) || (dw_k && !w_k))
    return fail(PF_ERR_INVALID_ARG, "a weight that is NULL has no gradient");
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    for (float* g : {dw_q, dw_k})
      if (g) PF_CUDA(cudaMemsetAsync(g, 0, desc->dh * sizeof(float), cs));
    return PF_OK;
  }
  PF_TRY(check_qk_rows("x", x, *desc));
  PF_TRY(check_qk_rows("dout", dout, *desc));
  PF_TRY(check_qk_rows("dx", dx, *desc));
  const bool dw = dw_q || dw_k;
  if (dw && (!ws || !aligned16(ws) || ws_bytes < qk_rope_part_bytes(desc->dh)))
    return fail(PF_ERR_WORKSPACE, "workspace too small: need %zu bytes, got %zu",
                qk_rope_part_bytes(desc->dh), ws ? ws_bytes : 0);
  PF_TRY(check_qk_results(*desc, rows, *dx, *dout, true, true));
  PF_TRY(check_qk_results(*desc, rows, *dx, *x, w_q != nullptr, w_k != nullptr));
  PF_CUDA(qk_rope_bwd(rope_of(*desc), ptr_of(*x), ptr_of(*dout), ptr_of(*dx), w_q, w_k, pos, dw_q,
                      dw_k, static_cast<float*>(ws), rows, seq_len, cs));
  return PF_OK;
}

pf_status pf_window_attn_fwd(const pf_window_desc* desc, const pf_qkv* x, void* out,
                             int64_t ld_out, void* saved, void* stream) {
  PF_TRY(check_window(desc));
  PF_TRY(check_window_rows("x", x, *desc));
  PF_TRY(check_rows("out", out, ld_out, (int64_t)desc->n_heads * desc->dh, 2));
  if (!aligned16(saved)) return fail(PF_ERR_INVALID_ARG, "saved must be 16-byte aligned");
  const Area o = window_area(*desc, "out", out, ld_out, desc->n_heads);
  PF_TRY(check_apart(o, window_area(*desc, "q", x->q, x->ld_q, desc->n_heads)));
  PF_TRY(check_apart(o, window_area(*desc, "k", x->k, x->ld_k, desc->n_kv)));
  PF_TRY(check_apart(o, window_area(*desc, "v", x->v, x->ld_v, desc->n_kv)));
  const Window c = window_of(*desc);
  PF_CUDA(window_fwd(c, ptr_of(*x), static_cast<bf16*>(out), (long)ld_out,
                     saved ? window_saved(c, saved) : WindowSaved{}, static_cast<cudaStream_t>(stream)));
  return PF_OK;
}

size_t pf_window_attn_saved_size(const pf_window_desc* desc) {
  return check_window(desc) == PF_OK ? window_saved(window_of(*desc), nullptr).bytes : 0;
}

size_t pf_window_attn_workspace_size(const pf_window_desc* desc) {
  return check_window(desc) == PF_OK ? window_bwd_ws_bytes(window_of(*desc)) : 0;
}

pf_status pf_window_attn_bwd(const pf_window_desc* desc, const pf_qkv* x, const void* out,
                             int64_t ld_out, const void* saved, const void* dout,
                             int64_t ld_dout, const pf_qkv* dx, void* ws, size_t ws_bytes,
                             void* stream) {
  PF_TRY(check_window(desc));
  PF_TRY(check_window_rows("x", x, *desc));
  PF_TRY(check_window_rows("dx", dx, *desc));
  PF_TRY(check_rows("out", out, ld_out, (int64_t)desc->n_heads * desc->dh, 2));
  PF_TRY(check_rows("dout", dout, ld_dout, (int64_t)desc->n_heads * desc->dh, 2));
  if (!saved || !aligned16(saved))
    return fail(PF_ERR_INVALID_ARG, "saved is required, 16-byte aligned");
  const Window c = window_of(*desc);
  const size_t need = window_bwd_ws_bytes(c);
  if (!ws || !aligned16(ws) || ws_bytes < need)
    return fail(PF_ERR_WORKSPACE, "workspace too small: need %zu bytes, got %zu", need,
                ws ? ws_bytes : 0);
  const int32_t H = desc->n_heads, KV = desc->n_kv;
  const Area grads[] = {window_area(*desc, "dq", dx->q, dx->ld_q, H), window_area(*desc, "dk", dx->k, dx->ld_k, KV),
                        window_area(*desc, "dv", dx->v, dx->ld_v, KV)};
  const Area read[] = {window_area(*desc, "q", x->q, x->ld_q, H), window_area(*desc, "k", x->k, x->ld_k, KV),
                       window_area(*desc, "v", x->v, x->ld_v, KV), window_area(*desc, "out", out, ld_out, H),
                       window_area(*desc, "dout", dout, ld_dout, H)};
  for (int i = 0; i < 3; ++i) {
    for (const Area& r : read) PF_TRY(check_apart(grads[i], r));
    for (int j = 0; j < i; ++j) PF_TRY(check_apart(grads[i], grads[j]));
  }
  PF_CUDA(window_bwd(c, ptr_of(*x), static_cast<const bf16*>(out), (long)ld_out,
                     window_saved(c, const_cast<void*>(saved)), static_cast<const bf16*>(dout), (long)ld_dout, ptr_of(*dx), ws,
                     static_cast<cudaStream_t>(stream)));
  return PF_OK;
}

pf_status pf_paged_advance(const pf_paged_desc* desc, const int32_t* start, pf_paged_cache* cache,
                           void* stream) {
  PF_TRY(check_paged(desc));
  if (!cache || !cache->len) return fail(PF_ERR_INVALID_ARG, "len is required");
  PF_CUDA(paged_advance(paged_of(*desc, cache), start, cache->len,
                        static_cast<cudaStream_t>(stream)));
  return PF_OK;
}

pf_status pf_paged_append(const pf_paged_desc* desc, const pf_qk_desc* qk, int64_t rows,
                          const pf_qkv* x, const float* w_q, const float* w_k,
                          const int32_t* start, const int32_t* pos, pf_paged_cache* cache,
                          void* q_out, int64_t ld_q_out, void* stream) {
  return append(desc, qk, rows, x, w_q, w_k, start, pos, cache, nullptr, q_out, ld_q_out, stream);
}

pf_status pf_paged_append_q8(const pf_paged_desc* desc, const pf_qk_desc* qk, int64_t rows, const pf_qkv* x,
                             const float* w_q, const float* w_k, const int32_t* start, const int32_t* pos,
                             pf_paged_cache* cache, const pf_paged_exp* exp, void* q_out, int64_t ld_q_out,
                             void* stream) {
  if (!exp) return fail(PF_ERR_INVALID_ARG, "exp is NULL");
  return append(desc, qk, rows, x, w_q, w_k, start, pos, cache, exp, q_out, ld_q_out, stream);
}

size_t pf_paged_attn_workspace_size(const pf_paged_desc* desc) {
  return check_paged(desc) == PF_OK ? paged_attn_ws_bytes(paged_of(*desc, nullptr), false) : 0;
}

size_t pf_paged_attn_q8_workspace_size(const pf_paged_desc* desc) {
  return check_paged(desc) == PF_OK ? paged_attn_ws_bytes(paged_of(*desc, nullptr), true) : 0;
}

pf_status pf_paged_attn(const pf_paged_desc* desc, const void* q, int64_t ld_q,
                        const pf_paged_cache* cache, void* out, int64_t ld_out, void* ws,
                        size_t ws_bytes, void* stream) {
  return attn(desc, q, ld_q, cache, nullptr, out, ld_out, ws, ws_bytes, stream);
}

pf_status pf_paged_attn_q8(const pf_paged_desc* desc, const void* q, int64_t ld_q, const pf_paged_cache* cache,
                           const pf_paged_exp* exp, void* out, int64_t ld_out, void* ws, size_t ws_bytes,
                           void* stream) {
  if (!exp) return fail(PF_ERR_INVALID_ARG, "exp is NULL");
  return attn(desc, q, ld_q, cache, exp, out, ld_out, ws, ws_bytes, stream);
}

size_t pf_paged_chunk_workspace_size(const pf_paged_desc* desc, int64_t rows) {
  if (check_paged(desc) != PF_OK || check_count(rows, 1, nullptr, 0) != PF_OK) return 0;
  return paged_chunk_ws_bytes(paged_of(*desc, nullptr), rows);
}

pf_status pf_paged_chunk_attn(const pf_paged_desc* desc, int64_t rows, const void* q, int64_t ld_q,
                              const int32_t* start, const pf_paged_cache* cache, const pf_paged_exp* exp, void* out,
                              int64_t ld_out, void* ws, size_t ws_bytes, void* stream) {
  PF_TRY(check_paged(desc));
  PF_TRY(check_count(rows, 1, nullptr, 0));
  if (!start) return fail(PF_ERR_INVALID_ARG, "start is required");
  PF_TRY(check_cache(cache));
  PF_TRY(check_exp(exp));
  if (rows == 0) return PF_OK;
  PF_TRY(check_rows("q", q, ld_q, (int64_t)desc->n_heads * desc->dh, 2));
  PF_TRY(check_rows("out", out, ld_out, (int64_t)desc->n_heads * desc->dh, 2));
  const Paged p = paged_of(*desc, cache, exp);
  const size_t need = paged_chunk_ws_bytes(p, rows);
  if (need > 0 && (!ws || !aligned16(ws) || ws_bytes < need))
    return fail(PF_ERR_WORKSPACE, "workspace too small: need %zu bytes, got %zu", need, ws ? ws_bytes : 0);
  PF_TRY(check_apart(head_area("out", out, rows, ld_out, desc->n_heads, desc->dh, 2),
                     head_area("q", q, rows, ld_q, desc->n_heads, desc->dh, 2)));
  PF_CUDA(paged_chunk(p, rows, static_cast<const bf16*>(q), (long)ld_q, start, static_cast<bf16*>(out), (long)ld_out,
                      ws, static_cast<cudaStream_t>(stream)));
  return PF_OK;
}

pf_status pf_paged_read(const pf_paged_desc* desc, int64_t rows, const int32_t* start, const pf_paged_cache* cache,
                        const pf_paged_exp* exp, void* k, int64_t ld_k, void* v, int64_t ld_v, void* stream) {
  PF_TRY(check_paged(desc));
  PF_TRY(check_count(rows, 1, nullptr, 0));
  if (!start && rows != desc->batch)
    return fail(PF_ERR_INVALID_ARG, "without start every sequence has one row: rows must be batch");
  PF_TRY(check_cache(cache));
  PF_TRY(check_exp(exp));
  if (rows == 0) return PF_OK;
  PF_TRY(check_rows("k", k, ld_k, (int64_t)desc->n_kv * desc->dh, 2));
  PF_TRY(check_rows("v", v, ld_v, (int64_t)desc->n_kv * desc->dh, 2));
  PF_TRY(check_apart(head_area("k", k, rows, ld_k, desc->n_kv, desc->dh, 2),
                     head_area("v", v, rows, ld_v, desc->n_kv, desc->dh, 2)));
  PF_CUDA(paged_read(paged_of(*desc, cache, exp), rows, start, static_cast<bf16*>(k), (long)ld_k,
                     static_cast<bf16*>(v), (long)ld_v, static_cast<cudaStream_t>(stream)));
  return PF_OK;
}

}  // extern "C"

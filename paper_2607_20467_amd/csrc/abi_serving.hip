// C-ABI entry points beside the denoising step: the paged cache and attention over it, attention over packed prompts,
// drawing tokens. Argument checks and launches only; every check happens on the host before anything is launched.
#include <math.h>

#include "dcl_internal.h"

using namespace dcl;

namespace {

bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Rows [T, heads, dh] of bfloat16 with a row stride.
dcl_status check_rows(const char* name, const void* p, int64_t stride, int32_t T, int32_t heads, int32_t dh) {
  if (T == 0) return DCL_OK;
  if (!p) return fail(DCL_E_ARG, "%s is NULL", name);
  if (misaligned(p, 16)) return fail(DCL_E_ARG, "%s must be 16-byte aligned", name);
  if (stride % 8 != 0 || stride < (int64_t)heads * dh || stride > ((int64_t)1 << 31))
    return fail(DCL_E_ARG, "%s: row stride %lld must be a multiple of 8 and at least %lld", name, (long long)stride,
                (long long)heads * dh);
  return DCL_OK;
}

dcl_status check_batch(const int32_t* cu, int32_t B, int32_t T, int32_t longest, const char* longest_name) {
  if (!cu) return fail(DCL_E_ARG, "cu is NULL");
  if (B < 1 || B > (1 << 16)) return fail(DCL_E_ARG, "B=%d outside [1, 2^16]", B);
  if (T < 0 || T > (1 << 22)) return fail(DCL_E_ARG, "T=%d outside [0, 2^22]", T);
  if (longest < 0 || longest > (1 << 22)) return fail(DCL_E_ARG, "%s=%d outside [0, 2^22]", longest_name, longest);
  return DCL_OK;
}

dcl_status check_head_dim(int32_t dh) {
  if (dh != 64 && dh != 128) return fail(DCL_E_UNSUPPORTED, "head_dim %d: kernels exist for 64 and 128", dh);
  return DCL_OK;
}

// Shapes of a pool and a batch's table, without its pointers.
dcl_status check_pool(const dcl_pages* g, int32_t max_pages) {
  if (!g) return fail(DCL_E_ARG, "pages is NULL");
  if (g->dtype != DCL_DTYPE_BF16 && g->dtype != DCL_DTYPE_E4M3)
    return fail(DCL_E_UNSUPPORTED, "pages dtype %d: bfloat16 or e4m3", g->dtype);
  dcl_status st = check_head_dim(g->head_dim);
  if (st != DCL_OK) return st;
  if (g->n_kv_heads < 1 || g->n_kv_heads > 1024) return fail(DCL_E_ARG, "n_kv_heads %d outside [1, 1024]", g->n_kv_heads);
  if (g->page_len < 16 || g->page_len > 1024 || (g->page_len & (g->page_len - 1)) != 0)
    return fail(DCL_E_ARG, "page_len %d must be a power of two in [16, 1024]", g->page_len);
  if (g->n_pages < 1) return fail(DCL_E_ARG, "n_pages %d must be >= 1", g->n_pages);
  if (max_pages < 1 || (int64_t)max_pages * g->page_len > (1 << 28))
    return fail(DCL_E_ARG, "max_pages %d: a sequence holds 1 page to 2^28 positions", max_pages);
  return DCL_OK;
}

dcl_status check_pages(const dcl_pages* g, const int32_t* table, int32_t max_pages, const int32_t* len,
                       const int32_t* cu, int32_t B, int32_t T, int32_t max_new) {
  dcl_status st = check_pool(g, max_pages);
  if (st == DCL_OK) st = check_batch(cu, B, T, max_new, "max_new");
  if (st != DCL_OK) return st;
  if (!g->k || !g->v) return fail(DCL_E_ARG, "pages: k / v is NULL");
  if (misaligned(g->k, 16) || misaligned(g->v, 16)) return fail(DCL_E_ARG, "pages: k / v must be 16-byte aligned");
  if (g->dtype == DCL_DTYPE_E4M3) {
    if (!g->k_scale || !g->v_scale) return fail(DCL_E_ARG, "pages: e4m3 needs k_scale and v_scale");
    if (misaligned(g->k_scale, 16) || misaligned(g->v_scale, 16))
      return fail(DCL_E_ARG, "pages: k_scale / v_scale must be 16-byte aligned");
  }
  if (!table || !len) return fail(DCL_E_ARG, "table / len is NULL");
  return DCL_OK;
}

Pages view(const dcl_pages* g, const int32_t* table, int32_t max_pages, const int32_t* len, const int32_t* cu, int32_t B,
           int32_t T, int32_t max_new) {
  Pages p;
  p.k = static_cast<uint8_t*>(g->k);
  p.v = static_cast<uint8_t*>(g->v);
  p.ks = g->k_scale;
  p.vs = g->v_scale;
  p.table = table;
  p.len = len;
  p.cu = cu;
  p.n_pages = g->n_pages;
  p.shift = __builtin_ctz((unsigned)g->page_len);
  p.max_pages = max_pages;
  p.Hkv = g->n_kv_heads;
  p.dh = g->head_dim;
  p.e4m3 = g->dtype == DCL_DTYPE_E4M3;
  p.B = B;
  p.T = T;
  p.max_new = max_new;
  return p;
}

dcl_status check_pages_copy(const dcl_pages* g, const int32_t* table, int32_t max_pages, const int32_t* len,
                            const int32_t* cu, int32_t B, int32_t T, int32_t max_new, const void* k, int64_t k_stride,
                            const void* v, int64_t v_stride) {
  dcl_status st = check_pages(g, table, max_pages, len, cu, B, T, max_new);
  if (st == DCL_OK) st = check_rows("k", k, k_stride, T, g->n_kv_heads, g->head_dim);
  if (st == DCL_OK) st = check_rows("v", v, v_stride, T, g->n_kv_heads, g->head_dim);
  if (st != DCL_OK) return st;
  if (((int64_t)max_new / 64 + 2) * g->n_kv_heads * B >= (1LL << 31))
    return fail(DCL_E_UNSUPPORTED, "B=%d sequences of %d new tokens: too many for one call", B, max_new);
  return DCL_OK;
}

dcl_status check_heads(int32_t n_heads, int32_t n_kv_heads) {
  if (n_kv_heads < 1 || n_heads < 1 || n_heads % n_kv_heads != 0 || n_heads > (1 << 16))
    return fail(DCL_E_UNSUPPORTED, "n_heads %d must be a positive multiple of n_kv_heads %d", n_heads, n_kv_heads);
  return DCL_OK;
}

// Workspace of an attention call over pages: the parts' outputs and their (reference, sum).
struct PartLayout {
  int nsplit;
  size_t ml, total;
};
PartLayout part_layout(const dcl_pages* g, int32_t n_heads, int32_t B, int32_t T, int32_t max_new, int32_t max_pages) {
  PartLayout L;
  L.nsplit = pages_attention_splits(g->n_kv_heads, n_heads / g->n_kv_heads, B, max_new, max_pages * g->page_len);
  const size_t rows = (size_t)L.nsplit * T * n_heads;
  L.ml = L.nsplit > 1 ? rows * g->head_dim * 4 : 0;
  L.total = L.nsplit > 1 ? L.ml + rows * 8 : 256;
  return L;
}

dcl_status check_attention_size(const dcl_pages* g, int32_t n_heads, int32_t B, int32_t max_new) {
  const int64_t tiles = ((int64_t)(n_heads / g->n_kv_heads) * max_new + 15) / 16;
  if (tiles * g->n_kv_heads * B * 64 >= (1LL << 31) || (int64_t)max_new * B * (n_heads + 8) >= (1LL << 31))
    return fail(DCL_E_UNSUPPORTED, "B=%d sequences of %d new tokens x %d heads: too many for one call", B, max_new, n_heads);
  return DCL_OK;
}

}  // namespace

extern "C" {

dcl_status dcl_pages_write(const dcl_pages* pages, const int32_t* table, int32_t max_pages, const int32_t* len,
                           const int32_t* cu, int32_t B, int32_t T, int32_t max_new, const void* k, int64_t k_stride,
                           const void* v, int64_t v_stride, hipStream_t stream) {
  dcl_status st = check_pages_copy(pages, table, max_pages, len, cu, B, T, max_new, k, k_stride, v, v_stride);
  if (st != DCL_OK) return st;
  (void)hipGetLastError();
  launch_pages_write(view(pages, table, max_pages, len, cu, B, T, max_new), static_cast<const bf16_t*>(k), (long)k_stride,
                     static_cast<const bf16_t*>(v), (long)v_stride, stream);
  return hip_check(hipGetLastError(), "pages_write launch");
}

dcl_status dcl_pages_read(const dcl_pages* pages, const int32_t* table, int32_t max_pages, const int32_t* len,
                          const int32_t* cu, int32_t B, int32_t T, int32_t max_new, void* k, int64_t k_stride, void* v,
                          int64_t v_stride, hipStream_t stream) {
  dcl_status st = check_pages_copy(pages, table, max_pages, len, cu, B, T, max_new, k, k_stride, v, v_stride);
  if (st != DCL_OK) return st;
  (void)hipGetLastError();
  launch_pages_read(view(pages, table, max_pages, len, cu, B, T, max_new), static_cast<bf16_t*>(k), (long)k_stride,
                    static_cast<bf16_t*>(v), (long)v_stride, stream);
  return hip_check(hipGetLastError(), "pages_read launch");
}

size_t dcl_pages_attention_workspace_bytes(const dcl_pages* pages, int32_t n_heads, int32_t B, int32_t T,
                                           int32_t max_new, int32_t max_pages) {
  if (check_pool(pages, max_pages) != DCL_OK || check_heads(n_heads, pages->n_kv_heads) != DCL_OK || B < 1 ||
      B > (1 << 16) || T < 0 || T > (1 << 22) || max_new < 0 || max_new > (1 << 22) ||
      check_attention_size(pages, n_heads, B, max_new) != DCL_OK)
    return 0;
  return part_layout(pages, n_heads, B, T, max_new, max_pages).total;
}

dcl_status dcl_pages_attention(const dcl_pages* pages, const int32_t* table, int32_t max_pages, const int32_t* len,
                               const int32_t* cu, int32_t B, int32_t T, int32_t max_new, const void* q,
                               int64_t q_stride, int32_t n_heads, float scale, int32_t causal, void* out, float* lse,
                               void* ws, size_t ws_bytes, hipStream_t stream) {
  dcl_status st = check_pages(pages, table, max_pages, len, cu, B, T, max_new);
  if (st == DCL_OK) st = check_heads(n_heads, pages->n_kv_heads);
  if (st == DCL_OK) st = check_rows("q", q, q_stride, T, n_heads, pages->head_dim);
  if (st == DCL_OK) st = check_rows("out", out, (int64_t)n_heads * pages->head_dim, T, n_heads, pages->head_dim);
  if (st == DCL_OK) st = check_attention_size(pages, n_heads, B, max_new);
  if (st != DCL_OK) return st;
  if (!isfinite(scale)) return fail(DCL_E_ARG, "scale must be finite");
  if (causal != 0 && causal != 1) return fail(DCL_E_ARG, "causal must be 0 or 1");
  const PartLayout L = part_layout(pages, n_heads, B, T, max_new, max_pages);
  if (!ws) return fail(DCL_E_ARG, "workspace is NULL");
  if (misaligned(ws, 256)) return fail(DCL_E_ARG, "workspace must be 256-byte aligned");
  if (ws_bytes < L.total) return fail(DCL_E_WORKSPACE, "workspace %zu bytes < required %zu", ws_bytes, L.total);
  PagesAttn a;
  a.p = view(pages, table, max_pages, len, cu, B, T, max_new);
  a.q = static_cast<const bf16_t*>(q);
  a.q_stride = (long)q_stride;
  a.out = static_cast<bf16_t*>(out);
  a.lse = lse;
  a.po = static_cast<float*>(ws);
  a.pml = reinterpret_cast<float2*>(static_cast<char*>(ws) + L.ml);
  a.H = n_heads;
  a.g = n_heads / pages->n_kv_heads;
  a.causal = causal;
  a.nsplit = L.nsplit;
  a.row_tiles = 0;
  a.scale_log2 = (float)(1.4426950408889634 * (double)scale);
  (void)hipGetLastError();
  launch_pages_attention(a, stream);
  return hip_check(hipGetLastError(), "pages_attention launch");
}

dcl_status dcl_prompt_attention(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                int64_t v_stride, const int32_t* cu, int32_t B, int32_t T, int32_t max_len,
                                int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale, int32_t causal,
                                void* out, float* lse, hipStream_t stream) {
  dcl_status st = check_batch(cu, B, T, max_len, "max_len");
  if (st == DCL_OK) st = check_head_dim(head_dim);
  if (st == DCL_OK) st = check_heads(n_heads, n_kv_heads);
  if (st == DCL_OK) st = check_rows("q", q, q_stride, T, n_heads, head_dim);
  if (st == DCL_OK) st = check_rows("k", k, k_stride, T, n_kv_heads, head_dim);
  if (st == DCL_OK) st = check_rows("v", v, v_stride, T, n_kv_heads, head_dim);
  if (st == DCL_OK) st = check_rows("out", out, (int64_t)n_heads * head_dim, T, n_heads, head_dim);
  if (st != DCL_OK) return st;
  if (!isfinite(scale)) return fail(DCL_E_ARG, "scale must be finite");
  if (causal != 0 && causal != 1) return fail(DCL_E_ARG, "causal must be 0 or 1");
  if (((int64_t)B * n_heads + 8) * (max_len / 64 + 1) >= (1LL << 31))
    return fail(DCL_E_UNSUPPORTED, "B=%d sequences of %d rows x %d heads: too many for one call", B, max_len, n_heads);
  PromptAttn a;
  a.q = static_cast<const bf16_t*>(q);
  a.k = static_cast<const bf16_t*>(k);
  a.v = static_cast<const bf16_t*>(v);
  a.q_stride = (long)q_stride;
  a.k_stride = (long)k_stride;
  a.v_stride = (long)v_stride;
  a.out = static_cast<bf16_t*>(out);
  a.lse = lse;
  a.cu = cu;
  a.B = B;
  a.T = T;
  a.max_len = max_len;
  a.H = n_heads;
  a.Hkv = n_kv_heads;
  a.dh = head_dim;
  a.causal = causal;
  a.q_tiles = 0;
  a.scale_log2 = (float)(1.4426950408889634 * (double)scale);
  (void)hipGetLastError();
  launch_prompt_attention(a, stream);
  return hip_check(hipGetLastError(), "prompt_attention launch");
}

}  // extern "C"

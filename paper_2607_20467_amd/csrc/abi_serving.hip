// C-ABI entry points beside the denoising step: the paged cache and attention over it, attention over packed prompts,
// drawing tokens. Argument checks and launches only; every check happens on the host before anything is launched.
#include <math.h>

#include "dcl_internal.h"

using namespace dcl;

namespace {

// |scale| log2(e), at least the least normal number: a masked score -inf times it stays -inf, and a scale of 0 gives
// every finite score (below 2^100) the exponent 0 to within 2^-26.
float scale_log2(float scale) {
  const double s = 1.4426950408889634 * fabs((double)scale);
  return s < 1.1754943508222875e-38 ? 1.1754943508222875e-38f : (float)s;
}

bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// A launch has fewer than 2^32 threads, and these kernels' workgroups have 256.
bool too_many(int64_t workgroups) { return workgroups >= (1 << 24); }

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
  if (g->dtype != DCL_DTYPE_BF16 && g->dtype != DCL_DTYPE_E4M3 && g->dtype != DCL_DTYPE_E2M1)
    return fail(DCL_E_UNSUPPORTED, "pages dtype %d: bfloat16, e4m3 or e2m1", g->dtype);
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
  if (g->dtype != DCL_DTYPE_BF16) {
    if (!g->k_scale || !g->v_scale) return fail(DCL_E_ARG, "pages: e4m3 and e2m1 need k_scale and v_scale");
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
  p.e2m1 = g->dtype == DCL_DTYPE_E2M1;
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
  if (too_many(((int64_t)max_new / 64 + 2) * g->n_kv_heads * B))
    return fail(DCL_E_UNSUPPORTED, "B=%d sequences of %d new tokens: too many for one call", B, max_new);
  return DCL_OK;
}

dcl_status check_heads(int32_t n_heads, int32_t n_kv_heads) {
  if (n_kv_heads < 1 || n_heads < 1 || n_heads % n_kv_heads != 0 || n_heads > (1 << 16))
    return fail(DCL_E_UNSUPPORTED, "n_heads %d must be a positive multiple of n_kv_heads %d", n_heads, n_kv_heads);
  return DCL_OK;
}

dcl_status check_attention_size(const dcl_pages* g, int32_t n_heads, int32_t B, int32_t max_new, int nsplit) {
  const int64_t rows = (int64_t)(n_heads / g->n_kv_heads) * max_new, tiles = rows <= 16 ? 1 : (rows + 31) / 32;
  const int64_t joined = nsplit > 16 ? n_heads : n_heads / 8 + 1;
  if (too_many(((int64_t)nsplit * B * g->n_kv_heads + 8) * tiles) || (nsplit > 1 && too_many(joined * max_new * B)))
    return fail(DCL_E_UNSUPPORTED, "B=%d sequences of %d new tokens x %d heads: too many for one call", B, max_new, n_heads);
  return DCL_OK;
}

// Sequences of a turn and the pool's shape.
dcl_status check_turn(const dcl_pages* g, const int32_t* table, int32_t max_pages, const int32_t* len, int32_t B,
                      const int32_t* free_pages, const int32_t* n_free, const void* ws, size_t ws_bytes) {
  dcl_status st = check_pool(g, max_pages);
  if (st != DCL_OK) return st;
  if (g->n_pages > (1 << 30)) return fail(DCL_E_UNSUPPORTED, "n_pages %d: at most 2^30 are handed out", g->n_pages);
  if (B < 1 || B > (1 << 16)) return fail(DCL_E_ARG, "B=%d outside [1, 2^16]", B);
  if ((int64_t)B * max_pages >= ((int64_t)1 << 31)) return fail(DCL_E_UNSUPPORTED, "B=%d rows of %d pages: a table of 2^31 entries", B, max_pages);
  if (!table || !len) return fail(DCL_E_ARG, "table / len is NULL");
  if (!free_pages || !n_free) return fail(DCL_E_ARG, "free_pages / n_free is NULL");
  if (!ws) return fail(DCL_E_ARG, "workspace is NULL");
  if (misaligned(ws, 256)) return fail(DCL_E_ARG, "workspace must be 256-byte aligned");
  const size_t need = dcl_pages_turn_workspace_bytes(B);
  if (ws_bytes < need) return fail(DCL_E_WORKSPACE, "workspace %zu bytes < required %zu", ws_bytes, need);
  return DCL_OK;
}

PagesTurn turn_args(const dcl_pages* g, int32_t* table, int32_t max_pages, int32_t* len, const int32_t* ask, int32_t B,
                    int32_t* free_pages, int32_t* n_free, void* ws) {
  PagesTurn a = {};
  a.table = table;
  a.len = len;
  a.ask = ask;
  a.free_pages = free_pages;
  a.n_free = n_free;
  a.ws = static_cast<int32_t*>(ws);
  a.B = B;
  a.n_pages = g->n_pages;
  a.shift = __builtin_ctz((unsigned)g->page_len);
  a.max_pages = max_pages;
  return a;
}

// Workspace of an attention call over pages: the parts' outputs and their (reference, sum). A call without rows has one
// part.
struct PartLayout {
  int nsplit, span, run;
  size_t ml, total;
};
dcl_status part_layout(const dcl_pages* g, int32_t n_heads, int32_t B, int32_t T, int32_t max_new, int32_t max_pages,
                       PartLayout* L) {
  const int capacity = max_pages * g->page_len;
  L->nsplit = 1;
  L->span = capacity;
  L->run = 0;
  if (T > 0 && max_new > 0) {
    // in one part first: what passes keeps the partition's products in 64 bits
    dcl_status st = check_attention_size(g, n_heads, B, max_new, 1);
    if (st != DCL_OK) return st;
    const int group = n_heads / g->n_kv_heads;
    if (g->dtype == DCL_DTYPE_E2M1) {
      pages4_attention_parts(g->n_kv_heads, group, B, max_new, capacity, &L->nsplit, &L->run);
    } else {
      L->span = pages_attention_span(g->n_kv_heads, group, B, max_new, capacity, g->dtype == DCL_DTYPE_E4M3);
      L->nsplit = (capacity + L->span - 1) / L->span;
    }
    st = check_attention_size(g, n_heads, B, max_new, L->nsplit);
    if (st != DCL_OK) return st;
  }
  const size_t rows = (size_t)L->nsplit * T * n_heads;
  L->ml = L->nsplit > 1 ? rows * g->head_dim * 4 : 0;
  L->total = L->nsplit > 1 ? L->ml + rows * 8 : 256;
  return DCL_OK;
}

// Most vocabulary ids of a sampled row: with 2^20 of them weights still have 42 bits.
constexpr int kSampleVocab = 1 << 20;

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

size_t sample_workspace(int32_t n, int32_t V) { return align256(n > 0 ? sample_ws_bytes(n, V) : 1); }

dcl_status check_sample(int32_t n, int32_t V, const dcl_sampling* how, const int32_t* token) {
  if (n < 0 || n > (1 << 22)) return fail(DCL_E_ARG, "n=%d outside [0, 2^22]", n);
  if (V < 1 || V > kSampleVocab) return fail(DCL_E_ARG, "vocab=%d outside [1, 2^20]", V);
  if (!how) return fail(DCL_E_ARG, "how is NULL");
  if (n > 0 && !how->uniform) return fail(DCL_E_ARG, "how.uniform is NULL");
  if (n > 0 && !token) return fail(DCL_E_ARG, "token is NULL");
  return DCL_OK;
}

dcl_status check_sample_workspace(const void* ws, size_t ws_bytes, size_t need) {
  if (!ws) return fail(DCL_E_ARG, "workspace is NULL");
  if (misaligned(ws, 256)) return fail(DCL_E_ARG, "workspace must be 256-byte aligned");
  if (ws_bytes < need) return fail(DCL_E_WORKSPACE, "workspace %zu bytes < required %zu", ws_bytes, need);
  return DCL_OK;
}

SampleArgs sample_args(const void* logits, int64_t stride, int bf16, int32_t n, int32_t V, const dcl_sampling& how,
                       int32_t* token, float* conf, int32_t* kept, void* ws) {
  SampleArgs a;
  a.logits = logits;
  a.stride = (long)stride;
  a.n = n;
  a.V = V;
  a.bf16 = bf16;
  int bits = 0;  // V <= 2^bits: the weights' sum stays below 2^62, a weight below 2^46
  while ((1 << bits) < V) ++bits;
  a.shift = bits < 17 ? 45 : 62 - bits;
  a.temperature = how.temperature;
  a.top_k = how.top_k;
  a.top_p = how.top_p;
  a.min_p = how.min_p;
  a.uniform = how.uniform;
  a.token = token;
  a.conf = conf;
  a.kept = kept;
  a.ws = ws;
  return a;
}

}  // namespace

extern "C" {

dcl_status dcl_pages_write(const dcl_pages* pages, const int32_t* table, int32_t max_pages, const int32_t* len,
                           const int32_t* cu, int32_t B, int32_t T, int32_t max_new, const void* k, int64_t k_stride,
                           const void* v, int64_t v_stride, hipStream_t stream) {
  dcl_status st = check_pages_copy(pages, table, max_pages, len, cu, B, T, max_new, k, k_stride, v, v_stride);
  if (st != DCL_OK) return st;
  (void)hipGetLastError();
  (pages->dtype == DCL_DTYPE_E2M1 ? launch_pages4_write : launch_pages_write)(
      view(pages, table, max_pages, len, cu, B, T, max_new), static_cast<const bf16_t*>(k), (long)k_stride,
      static_cast<const bf16_t*>(v), (long)v_stride, stream);
  return hip_check(hipGetLastError(), "pages_write launch");
}

dcl_status dcl_pages_read(const dcl_pages* pages, const int32_t* table, int32_t max_pages, const int32_t* len,
                          const int32_t* cu, int32_t B, int32_t T, int32_t max_new, void* k, int64_t k_stride, void* v,
                          int64_t v_stride, hipStream_t stream) {
  dcl_status st = check_pages_copy(pages, table, max_pages, len, cu, B, T, max_new, k, k_stride, v, v_stride);
  if (st != DCL_OK) return st;
  (void)hipGetLastError();
  (pages->dtype == DCL_DTYPE_E2M1 ? launch_pages4_read : launch_pages_read)(
      view(pages, table, max_pages, len, cu, B, T, max_new), static_cast<bf16_t*>(k), (long)k_stride,
      static_cast<bf16_t*>(v), (long)v_stride, stream);
  return hip_check(hipGetLastError(), "pages_read launch");
}

size_t dcl_pages_turn_workspace_bytes(int32_t B) {
  return B < 1 || B > (1 << 16) ? 0 : align256(pages_turn_ws_ints(B) * 4);
}

dcl_status dcl_pages_extend(const dcl_pages* pages, int32_t* table, int32_t max_pages, int32_t* len, const int32_t* count,
                            int32_t B, int32_t T, const int32_t* free_pages, int32_t* n_free, int32_t* cu, int32_t* pos,
                            int64_t* slot, void* ws, size_t ws_bytes, hipStream_t stream) {
  dcl_status st = check_turn(pages, table, max_pages, len, B, free_pages, n_free, ws, ws_bytes);
  if (st != DCL_OK) return st;
  if (T < 0 || T > (1 << 22)) return fail(DCL_E_ARG, "T=%d outside [0, 2^22]", T);
  if (!cu) return fail(DCL_E_ARG, "cu is NULL");
  PagesTurn a = turn_args(pages, table, max_pages, len, count, B, const_cast<int32_t*>(free_pages), n_free, ws);
  a.T = T;
  a.cu = cu;
  a.pos = pos;
  a.slot = slot;
  (void)hipGetLastError();
  launch_pages_extend(a, stream);
  return hip_check(hipGetLastError(), "pages_extend launch");
}

dcl_status dcl_pages_shrink(const dcl_pages* pages, int32_t* table, int32_t max_pages, int32_t* len, const int32_t* keep,
                            int32_t B, int32_t* free_pages, int32_t* n_free, void* ws, size_t ws_bytes,
                            hipStream_t stream) {
  dcl_status st = check_turn(pages, table, max_pages, len, B, free_pages, n_free, ws, ws_bytes);
  if (st != DCL_OK) return st;
  if (!keep) return fail(DCL_E_ARG, "keep is NULL");
  (void)hipGetLastError();
  launch_pages_shrink(turn_args(pages, table, max_pages, len, keep, B, free_pages, n_free, ws), stream);
  return hip_check(hipGetLastError(), "pages_shrink launch");
}

dcl_status dcl_heads_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const int32_t* pos,
                               int32_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, const float* g_q,
                               const float* g_k, float eps, float rope_base, int32_t rot_dim, void* q_out,
                               int64_t q_out_stride, void* k_out, int64_t k_out_stride, hipStream_t stream) {
  if (T < 0 || T > (1 << 22)) return fail(DCL_E_ARG, "T=%d outside [0, 2^22]", T);
  dcl_status st = check_head_dim(head_dim);
  if (st != DCL_OK) return st;
  if (n_heads < 0 || n_kv_heads < 0 || n_heads > (1 << 16) || n_kv_heads > (1 << 16) || n_heads + n_kv_heads < 1)
    return fail(DCL_E_ARG, "n_heads %d, n_kv_heads %d: each in [0, 2^16], not both 0", n_heads, n_kv_heads);
  if (n_heads > 0) st = check_rows("q", q, q_stride, T, n_heads, head_dim);
  if (st == DCL_OK && n_heads > 0) st = check_rows("q_out", q_out, q_out_stride, T, n_heads, head_dim);
  if (st == DCL_OK && n_kv_heads > 0) st = check_rows("k", k, k_stride, T, n_kv_heads, head_dim);
  if (st == DCL_OK && n_kv_heads > 0) st = check_rows("k_out", k_out, k_out_stride, T, n_kv_heads, head_dim);
  if (st != DCL_OK) return st;
  if (T > 0 && !pos) return fail(DCL_E_ARG, "pos is NULL");
  if (T > 1 && ((n_heads > 0 && q_out == q && q_out_stride != q_stride) || (n_kv_heads > 0 && k_out == k && k_out_stride != k_stride)))
    return fail(DCL_E_ARG, "an output over its input needs the input's row stride");
  if (misaligned(g_q, 16) || misaligned(g_k, 16)) return fail(DCL_E_ARG, "g_q / g_k must be 16-byte aligned");
  if (!(eps >= 0.f) || !isfinite(eps)) return fail(DCL_E_ARG, "eps must be >= 0");
  if (!(rope_base > 1.f) || !isfinite(rope_base)) return fail(DCL_E_ARG, "rope_base must be > 1");
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 16 != 0)
    return fail(DCL_E_ARG, "rot_dim %d must be a multiple of 16 in [0, head_dim]", rot_dim);
  if (T == 0) return DCL_OK;
  HeadsArgs a = {};
  a.q = static_cast<const bf16_t*>(q);
  a.k = static_cast<const bf16_t*>(k);
  a.q_out = static_cast<bf16_t*>(q_out);
  a.k_out = static_cast<bf16_t*>(k_out);
  a.q_stride = (long)q_stride;
  a.k_stride = (long)k_stride;
  a.q_out_stride = (long)q_out_stride;
  a.k_out_stride = (long)k_out_stride;
  a.pos = pos;
  a.g_q = g_q;
  a.g_k = g_k;
  a.T = T;
  a.H = n_heads;
  a.Hkv = n_kv_heads;
  a.dh = head_dim;
  a.rot = rot_dim;
  a.eps = eps;
  // powers in turn in 64 fraction bits: the last of 64 is off by less than 2^-56 of itself
  if (rot_dim > 0) {
    const long double step = powl((long double)rope_base, -2.0L / rot_dim);
    long double f = 0.15915494309189533576888376337251436L;  // 1 / (2 pi)
    for (int i = 0; i < rot_dim / 2; ++i, f *= step) a.turns[i] = (double)f;
  }
  (void)hipGetLastError();
  launch_heads_norm_rope(a, stream);
  return hip_check(hipGetLastError(), "heads_norm_rope launch");
}

size_t dcl_pages_attention_workspace_bytes(const dcl_pages* pages, int32_t n_heads, int32_t B, int32_t T,
                                           int32_t max_new, int32_t max_pages) {
  if (check_pool(pages, max_pages) != DCL_OK || check_heads(n_heads, pages->n_kv_heads) != DCL_OK || B < 1 ||
      B > (1 << 16) || T < 0 || T > (1 << 22) || max_new < 0 || max_new > (1 << 22))
    return 0;
  PartLayout L;
  return part_layout(pages, n_heads, B, T, max_new, max_pages, &L) == DCL_OK ? L.total : 0;
}

dcl_status dcl_pages_attention(const dcl_pages* pages, const int32_t* table, int32_t max_pages, const int32_t* len,
                               const int32_t* cu, int32_t B, int32_t T, int32_t max_new, const void* q,
                               int64_t q_stride, int32_t n_heads, float scale, int32_t causal, void* out, float* lse,
                               void* ws, size_t ws_bytes, hipStream_t stream) {
  dcl_status st = check_pages(pages, table, max_pages, len, cu, B, T, max_new);
  if (st == DCL_OK) st = check_heads(n_heads, pages->n_kv_heads);
  if (st == DCL_OK) st = check_rows("q", q, q_stride, T, n_heads, pages->head_dim);
  if (st == DCL_OK) st = check_rows("out", out, (int64_t)n_heads * pages->head_dim, T, n_heads, pages->head_dim);
  if (st != DCL_OK) return st;
  if (!isfinite(scale)) return fail(DCL_E_ARG, "scale must be finite");
  if (causal != 0 && causal != 1) return fail(DCL_E_ARG, "causal must be 0 or 1");
  PartLayout L;
  st = part_layout(pages, n_heads, B, T, max_new, max_pages, &L);
  if (st != DCL_OK) return st;
  if (!ws) return fail(DCL_E_ARG, "workspace is NULL");
  if (misaligned(ws, 256)) return fail(DCL_E_ARG, "workspace must be 256-byte aligned");
  if (ws_bytes < L.total) return fail(DCL_E_WORKSPACE, "workspace %zu bytes < required %zu", ws_bytes, L.total);
  if (T == 0 || max_new == 0) return DCL_OK;
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
  a.span = L.span;
  a.run = L.run;
  a.row_tiles = 0;
  a.q_sign = scale < 0.f ? 0x80008000u : 0u;
  a.scale_log2 = scale_log2(scale);
  (void)hipGetLastError();
  (pages->dtype == DCL_DTYPE_E2M1 ? launch_pages4_attention : launch_pages_attention)(a, stream);
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
  if (too_many(((int64_t)B * n_heads + 8) * ((max_len < T ? max_len : T) / 128 + 1)))
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
  a.q_sign = scale < 0.f ? 0x80008000u : 0u;
  a.scale_log2 = scale_log2(scale);
  (void)hipGetLastError();
  launch_prompt_attention(a, stream);
  return hip_check(hipGetLastError(), "prompt_attention launch");
}

size_t dcl_sample_workspace_bytes(int32_t n, int32_t vocab) {
  if (n < 0 || n > (1 << 22) || vocab < 1 || vocab > kSampleVocab) return 0;
  return sample_workspace(n, vocab);
}

dcl_status dcl_sample_tokens(const void* logits, int32_t dtype, int64_t row_stride, int32_t n, int32_t vocab,
                             const dcl_sampling* how, int32_t* token, float* conf, int32_t* kept, void* ws,
                             size_t ws_bytes, hipStream_t stream) {
  dcl_status st = check_sample(n, vocab, how, token);
  if (st != DCL_OK) return st;
  if (dtype != DCL_DTYPE_F32 && dtype != DCL_DTYPE_BF16) return fail(DCL_E_UNSUPPORTED, "logits dtype %d: float32 or bfloat16", dtype);
  if (n > 0 && !logits) return fail(DCL_E_ARG, "logits is NULL");
  if (misaligned(logits, dtype == DCL_DTYPE_F32 ? 4 : 2)) return fail(DCL_E_ARG, "logits must be aligned to its elements");
  if (row_stride < vocab || row_stride > ((int64_t)1 << 40)) return fail(DCL_E_ARG, "row stride %lld < vocab %d", (long long)row_stride, vocab);
  st = check_sample_workspace(ws, ws_bytes, sample_workspace(n, vocab));
  if (st != DCL_OK) return st;
  (void)hipGetLastError();
  launch_sample(sample_args(logits, row_stride, dtype == DCL_DTYPE_BF16, n, vocab, *how, token, conf, kept, ws), stream);
  return hip_check(hipGetLastError(), "sample_tokens launch");
}

size_t dcl_sample_hidden_workspace_bytes(dcl_model_t model, int32_t n) {
  const Model* m = reinterpret_cast<const Model*>(model);
  if (!m || n < 0 || n > (1 << 22) || m->cfg.vocab > kSampleVocab || (int64_t)n * m->cfg.vocab >= (1LL << 31)) return 0;
  return align256((size_t)n * m->cfg.vocab * 4) + sample_workspace(n, m->cfg.vocab);
}

dcl_status dcl_sample_hidden(dcl_model_t model, const void* hidden, int32_t n, const dcl_sampling* how, int32_t* token,
                             float* conf, int32_t* kept, void* ws, size_t ws_bytes, hipStream_t stream) {
  const Model* m = reinterpret_cast<const Model*>(model);
  if (!m) return fail(DCL_E_ARG, "model is NULL");
  const int32_t V = m->cfg.vocab;
  dcl_status st = check_sample(n, V, how, token);
  if (st != DCL_OK) return st;
  if ((int64_t)n * V >= (1LL << 31) || (int64_t)n * m->cfg.d_model >= (1LL << 31))
    return fail(DCL_E_UNSUPPORTED, "n=%d rows: the head addresses fewer than 2^31 elements", n);
  if (!m->loaded) return fail(DCL_E_STATE, "weights not loaded");
  if (n > 0 && !hidden) return fail(DCL_E_ARG, "hidden is NULL");
  if (misaligned(hidden, 16)) return fail(DCL_E_ARG, "hidden must be 16-byte aligned");
  st = check_sample_workspace(ws, ws_bytes, dcl_sample_hidden_workspace_bytes(model, n));
  if (st != DCL_OK) return st;
  if (n == 0) return DCL_OK;
  (void)hipGetLastError();
  float* logits = static_cast<float*>(ws);
  void* rest = static_cast<char*>(ws) + align256((size_t)n * V * 4);
  gemm_store_f32(reinterpret_cast<const bf16_t*>(static_cast<const char*>(m->wbuf) + m->lay.lm),
                 static_cast<const bf16_t*>(hidden), V, n, m->cfg.d_model, logits, stream);
  launch_sample(sample_args(logits, V, 0, n, V, *how, token, conf, kept, rest), stream);
  return hip_check(hipGetLastError(), "sample_hidden launch");
}

}  // extern "C"

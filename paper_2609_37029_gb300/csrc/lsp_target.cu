// C ABI of the target side of a round: host-side validation of the paged-cache,
// attention and verification calls (declarations and contracts: include/lsp.h).
#include <cuda_runtime.h>

#include <cmath>

#include "lsp_internal.h"

using namespace lsp;

namespace {

inline int esize(int dtype) { return dtype == LSP_DTYPE_BF16 ? 2 : 4; }
inline cudaStream_t S(lsp_stream_t s) { return static_cast<cudaStream_t>(s); }
inline bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// Lists of 32-bit words (or none): a kernel that read one at another address would fault.
template <typename... P>
inline bool words(P... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & 3) == 0; }

int num_sms(int* sms) {
  int dev = 0;
  return cudaGetDevice(&dev) == cudaSuccess &&
                 cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess
             ? LSP_OK
             : LSP_ERR_CUDA;
}

// Sizes, type and strides (no pointers).
int check_shape(const lsp_kv_cache* c) {
  if (!c) return LSP_ERR_ARG;
  if (c->dtype != LSP_DTYPE_BF16 && c->dtype != LSP_DTYPE_F32) return LSP_ERR_ARG;
  if (c->layers < 1 || c->pages < 1 || c->pages > (1 << 20) || c->nkv < 1 || c->nkv > 65535 || c->seqs < 1 ||
      c->max_pages < 1 || (int64_t)c->seqs * c->max_pages > (1 << 30))
    return LSP_ERR_SHAPE;
  if (c->page < 16 || c->page > 256 || (c->page & (c->page - 1)) || (c->d != 64 && c->d != 128)) return LSP_ERR_SHAPE;
  if ((int64_t)c->max_pages * c->page > (1 << 30)) return LSP_ERR_SHAPE;
  const int64_t stride[4] = {c->s_layer, c->s_page, c->s_head, c->s_slot};
  const int extent[4] = {c->layers, c->pages, c->nkv, c->page};
  for (int i = 0; i < 4; ++i)
    if (extent[i] > 1 && (stride[i] < c->d || stride[i] * esize(c->dtype) % 16 ||
                          stride[i] * esize(c->dtype) >= ((int64_t)1 << 40)))
      return LSP_ERR_SHAPE;
  return LSP_OK;
}

int view(const lsp_kv_cache* c, KvCache* out) {
  const int rc = check_shape(c);
  if (rc != LSP_OK) return rc;
  if (!c->k || !c->v || !c->table || !c->len || !c->refs || !aligned(c->k, 16) || !aligned(c->v, 16) ||
      !words(c->table, c->len, c->refs))
    return LSP_ERR_ARG;
  out->k = static_cast<char*>(c->k);
  out->v = static_cast<char*>(c->v);
  out->table = c->table;
  out->len = c->len;
  out->refs = c->refs;
  // a stride along an axis of one is never used: any valid one will do
  out->s_layer = c->layers > 1 ? c->s_layer : c->d;
  out->s_page = c->pages > 1 ? c->s_page : c->d;
  out->s_head = c->nkv > 1 ? c->s_head : c->d;
  out->s_slot = c->s_slot;
  out->layers = c->layers; out->pages = c->pages; out->page = c->page; out->nkv = c->nkv; out->d = c->d;
  out->seqs = c->seqs; out->max_pages = c->max_pages;
  return LSP_OK;
}

int entries(const int32_t* a, const int32_t* b, int n, const uint32_t* dev_error) {
  if (n < 0 || (n > 0 && (!a || !b)) || !words(a, b, dev_error)) return LSP_ERR_ARG;
  return n > kPagesMaxSeqs ? LSP_ERR_SHAPE : LSP_OK;
}

// The sizes of an attention call that its plan depends on.
int attn_shape(const lsp_kv_cache* c, int nq, int n, int total, PrefixAttnParams* p) {
  if (nq < 1 || n < 1 || total < 0) return LSP_ERR_ARG;
  if (nq % c->nkv || nq / c->nkv > kPrefixMaxRep || n > kPrefixMaxSeqs || (int64_t)total * nq > (1 << 30)) return LSP_ERR_SHAPE;
  p->nq = nq; p->nkv = c->nkv; p->rep = nq / c->nkv; p->d = c->d;
  p->n = n; p->total = total;
  return LSP_OK;
}

}  // namespace

extern "C" {

size_t lsp_pages_workspace_bytes(const lsp_kv_cache* cache) {
  return check_shape(cache) == LSP_OK ? pages_ws_bytes(cache->pages) : 0;
}

int lsp_pages_fork(const lsp_kv_cache* cache, const int32_t* src, const int32_t* dst, int n, uint32_t* dev_error,
                   lsp_stream_t stream) {
  KvCache c;
  int rc = view(cache, &c);
  if (rc == LSP_OK) rc = entries(src, dst, n, dev_error);
  if (rc != LSP_OK || n == 0) return rc;
  return launch_pages_fork(c, src, dst, n, dev_error, S(stream));
}

int lsp_pages_trim(const lsp_kv_cache* cache, const int32_t* seqs, const int32_t* new_len, int n, uint32_t* dev_error,
                   lsp_stream_t stream) {
  KvCache c;
  int rc = view(cache, &c);
  if (rc == LSP_OK) rc = entries(seqs, new_len, n, dev_error);
  if (rc != LSP_OK || n == 0) return rc;
  return launch_pages_trim(c, seqs, new_len, n, dev_error, S(stream));
}

int lsp_pages_reserve(const lsp_kv_cache* cache, const int32_t* seqs, const int32_t* add, int n, void* workspace,
                      size_t workspace_bytes, uint32_t* dev_error, lsp_stream_t stream) {
  KvCache c;
  int rc = view(cache, &c), sms = 0;
  if (rc == LSP_OK) rc = entries(seqs, add, n, dev_error);
  if (rc != LSP_OK || n == 0) return rc;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < pages_ws_bytes(c.pages)) return LSP_ERR_ARG;
  if ((rc = num_sms(&sms)) != LSP_OK) return rc;
  return launch_pages_reserve(c, seqs, add, n, workspace, esize(cache->dtype), sms, dev_error, S(stream));
}

int lsp_pages_compact(const lsp_kv_cache* cache, int32_t* live, void* workspace, size_t workspace_bytes,
                      lsp_stream_t stream) {
  KvCache c;
  int rc = view(cache, &c), sms = 0;
  if (rc != LSP_OK) return rc;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < pages_ws_bytes(c.pages) || !words(live)) return LSP_ERR_ARG;
  if ((rc = num_sms(&sms)) != LSP_OK) return rc;
  return launch_pages_compact(c, live, workspace, esize(cache->dtype), sms, S(stream));
}

int lsp_pages_write(const lsp_kv_cache* cache, int layer, const int32_t* seqs, const int32_t* start, int n,
                    const void* k_new, const void* v_new, int64_t row_stride, int total, uint32_t* dev_error,
                    lsp_stream_t stream) {
  KvCache c;
  const int rc = view(cache, &c);
  if (rc != LSP_OK) return rc;
  if (layer < 0 || layer >= c.layers || n < 0 || total < 0) return LSP_ERR_ARG;
  if (n == 0 || total == 0) return LSP_OK;
  if (!seqs || !start || !words(seqs, start, dev_error)) return LSP_ERR_ARG;
  const int es = esize(cache->dtype);
  if (!k_new || !v_new || !aligned(k_new, 16) || !aligned(v_new, 16)) return LSP_ERR_ARG;
  if (total > (1 << 28) || (total > 1 && (row_stride < (int64_t)c.nkv * c.d || row_stride * es % 16))) return LSP_ERR_SHAPE;
  c.k += (int64_t)layer * c.s_layer * es;
  c.v += (int64_t)layer * c.s_layer * es;
  return launch_pages_write(c, seqs, start, n, k_new, v_new, row_stride * es, total, es, dev_error, S(stream));
}

size_t lsp_prefix_attention_workspace_bytes(const lsp_kv_cache* cache, int nq, int n, int total) {
  PrefixAttnParams p = {};
  int sms = 0;
  if (check_shape(cache) != LSP_OK || attn_shape(cache, nq, n, total, &p) != LSP_OK || num_sms(&sms) != LSP_OK) return 0;
  return total == 0 ? 0 : prefix_attn_plan(&p, cache->dtype, sms);
}

int lsp_prefix_attention(const lsp_kv_cache* cache, int layer, const void* q, int64_t q_stride, int nq,
                         const int32_t* seqs, const int32_t* start, int n, int total, int shared_len, float scale,
                         void* out, float* lse, void* workspace, size_t workspace_bytes, uint32_t* dev_error,
                         lsp_stream_t stream) {
  KvCache c;
  PrefixAttnParams p = {};
  int rc = view(cache, &c), sms = 0;
  if (rc == LSP_OK) rc = attn_shape(cache, nq, n, total, &p);
  if (rc != LSP_OK) return rc;
  if (layer < 0 || layer >= c.layers || shared_len < 0 || !(scale > 0.f) || !std::isfinite(scale) || !seqs || !start ||
      !words(seqs, start, lse, dev_error))
    return LSP_ERR_ARG;
  if (total == 0) return LSP_OK;
  const int es = esize(cache->dtype);
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !workspace || !aligned(workspace, 256)) return LSP_ERR_ARG;
  if (total > 1 && (q_stride < (int64_t)nq * c.d || q_stride * es % 16 || q_stride * es >= ((int64_t)1 << 40)))
    return LSP_ERR_SHAPE;
  if ((rc = num_sms(&sms)) != LSP_OK) return rc;
  p.k = c.k + (int64_t)layer * c.s_layer * es;
  p.v = c.v + (int64_t)layer * c.s_layer * es;
  p.q = q; p.out = out; p.lse = lse;
  p.table = c.table; p.len = c.len; p.seqs = seqs; p.start = start;
  p.q_stride = total > 1 ? q_stride : (int64_t)nq * c.d;
  p.s_page = c.s_page; p.s_head = c.s_head; p.s_slot = c.s_slot;
  p.page = c.page; p.pages = c.pages; p.max_pages = c.max_pages; p.n_seqs = c.seqs;
  p.shared_len = shared_len < c.max_pages * c.page ? shared_len : c.max_pages * c.page;
  p.scale = scale; p.err = dev_error;
  if (workspace_bytes < prefix_attn_plan(&p, cache->dtype, sms)) return LSP_ERR_ARG;
  return launch_prefix_attention(p, cache->dtype, workspace, S(stream));
}

int lsp_verify_probs(const void* target_probs, const void* draft_probs, int dtype, const int32_t* draft_tokens,
                     const int32_t* n_draft, const float* u, const float* e, int C, int B, int V, int64_t ld_target,
                     int64_t ld_draft, int32_t* accepted_len, int32_t* next_token, int32_t* out_tokens,
                     uint32_t* dev_error, lsp_stream_t stream) {
  if (dtype != LSP_DTYPE_BF16 && dtype != LSP_DTYPE_F32) return LSP_ERR_ARG;
  if (!target_probs || !e || !accepted_len || !next_token || (B > 0 && (!draft_tokens || !u))) return LSP_ERR_ARG;
  if (C < 1 || C > (1 << 20) || B < 0 || B > 1024 || V < 1 || V > (1 << 30)) return LSP_ERR_SHAPE;
  if (ld_target < V || (draft_probs && B > 0 && ld_draft < V)) return LSP_ERR_SHAPE;
  const size_t es = esize(dtype);
  if (!aligned(target_probs, es) || !aligned(draft_probs, es) ||
      !words(draft_tokens, n_draft, u, e, accepted_len, next_token, out_tokens, dev_error))
    return LSP_ERR_ARG;
  VerifyProbsParams p;
  p.pt = target_probs; p.pq = B > 0 ? draft_probs : nullptr; p.y = draft_tokens; p.n = n_draft; p.u = u; p.e = e;
  p.accepted = accepted_len; p.next_token = next_token; p.out_tokens = out_tokens; p.err = dev_error;
  p.C = C; p.B = B; p.V = V; p.ld_t = ld_target; p.ld_q = ld_draft;
  int sms = 0;
  const int rc = num_sms(&sms);
  return rc == LSP_OK ? launch_verify_probs(p, dtype, sms, S(stream)) : rc;
}

}  // extern "C"

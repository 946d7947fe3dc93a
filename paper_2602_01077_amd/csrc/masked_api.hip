// C-ABI entry points of masked and paged attention: argument validation and dispatch.  Validation runs before any device call.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "common.h"
#include "masked.h"
#include "paged.h"

namespace pisa {
namespace {

bool misaligned(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (reinterpret_cast<uintptr_t>(p) & 15u) return true;
  return false;
}

int32_t launch_failed(const char* what, hipError_t e) {
  return fail(PISA_HIP_ERROR, "%s: %s (%d)", what, hipGetErrorName(e), (int)e);
}

size_t size_of(int dtype) { return dtype == PISA_BF16 ? 2 : 4; }

struct Extent {
  long long batch, heads, len;
};

// Strides in elements of a tensor [batch, heads, len, d] -> bytes.  Dimensions of one element have stride 0 afterwards.
int32_t resolve_strides(const char* name, const pisa_strides& s, const Extent& n, int d, int dtype, bool output, Strides* out) {
  pisa_strides t = s;
  if (t.batch == 0 && t.head == 0 && t.token == 0) t = pisa_strides{n.heads * n.len * d, n.len * d, d};
  if (n.batch <= 1) t.batch = 0;
  if (n.heads <= 1) t.head = 0;
  if (n.len <= 1) t.token = 0;
  const long long size = (long long)size_of(dtype);
  struct Dim {
    long long stride, n;
  } dims[3] = {{t.batch, n.batch}, {t.head, n.heads}, {t.token, n.len}};
  for (const Dim& x : dims) {
    if (x.stride > 0 && x.n > (1LL << 56) / x.stride) return fail(PISA_UNSUPPORTED, "%s: stride of %lld elements", name, x.stride);
    if (x.stride < 0) return fail(PISA_INVALID_ARG, "%s: strides must not be negative", name);
    if (x.stride >= (1LL << 40)) return fail(PISA_UNSUPPORTED, "%s: stride of %lld elements", name, x.stride);
    if (x.stride * size % 16 != 0)
      return fail(PISA_INVALID_ARG, "%s: strides must be multiples of 16 bytes (got %lld elements)", name, x.stride);
  }
  if (n.len > 1 && t.token < d) return fail(PISA_INVALID_ARG, "%s: token stride %lld is below head_dim", name, (long long)t.token);
  if (t.token * size * 64 >= (1LL << 31))
    return fail(PISA_UNSUPPORTED, "%s: 64 tokens must lie within 2 GiB (token stride %lld elements)", name, (long long)t.token);
  if (output) {
    std::sort(dims, dims + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
    long long extent = d;
    for (const Dim& x : dims) {
      if (x.n <= 1) continue;
      if (x.stride < extent) return fail(PISA_INVALID_ARG, "%s: elements overlap", name);
      extent += x.stride * (x.n - 1);
    }
  }
  *out = Strides{t.batch * size, t.head * size, t.token * size};
  return PISA_OK;
}

int32_t check_scores(float scale, float softcap, int head_dim, float* resolved) {
  if (!(scale == scale) || std::isinf(scale)) return fail(PISA_INVALID_ARG, "scale is not finite");
  if (!(softcap >= 0.f) || std::isinf(softcap)) return fail(PISA_INVALID_ARG, "softcap must be finite and >= 0");
  *resolved = scale > 0.f ? scale : 1.0f / std::sqrt((float)head_dim);
  // scores are divided by the cap before it is known how small they are: neither factor may leave the normal range
  if (softcap > 0.f && !(softcap >= 0x1p-64f && softcap <= 0x1p64f && *resolved / softcap >= 0x1p-96f && *resolved / softcap <= 0x1p96f))
    return fail(PISA_UNSUPPORTED, "softcap must be 0 or within 2^-64 .. 2^64, and scale / softcap within 2^-96 .. 2^96");
  return PISA_OK;
}
int32_t check_type(int dtype, int head_dim) {
  if (dtype != PISA_FP32 && dtype != PISA_BF16)
    return fail(PISA_INVALID_ARG, "dtype must be PISA_FP32 (0) or PISA_BF16 (1), got %d", dtype);
  if (head_dim != 64 && head_dim != 128) return fail(PISA_INVALID_ARG, "head_dim must be 64 or 128, got %d", head_dim);
  return PISA_OK;
}
int32_t check_heads(int heads, int kv_heads) {
  if (heads < 1 || kv_heads < 1 || heads % kv_heads != 0)
    return fail(PISA_INVALID_ARG, "heads (%d) must be a multiple of kv_heads (%d), both >= 1", heads, kv_heads);
  return PISA_OK;
}

int32_t resolve_masked(const pisa_masked_shape* s, Masked* m) {
  *m = Masked{};
  if (!s) return fail(PISA_INVALID_ARG, "shape is NULL");
  if (s->batch < 1 || s->q_len < 1 || s->kv_len < 0)
    return fail(PISA_INVALID_ARG, "batch and q_len must be >= 1, kv_len >= 0 (got %d, %d, %d)", s->batch, s->q_len, s->kv_len);
  int32_t rc = check_heads(s->heads, s->kv_heads);
  if (rc == PISA_OK) rc = check_type(s->dtype, s->head_dim);
  if (rc == PISA_OK) rc = check_scores(s->scale, s->softcap, s->head_dim, &m->scale);
  if (rc != PISA_OK) return rc;
  if (s->causal != 0 && s->causal != 1) return fail(PISA_INVALID_ARG, "causal must be 0 or 1, got %d", s->causal);
  if (s->num_docs < 0 || s->num_docs == 0x7fffffff) return fail(PISA_INVALID_ARG, "num_docs = %d", s->num_docs);
  constexpr int kLongest = 1 << 24;
  if (s->q_len > kLongest || s->kv_len > kLongest)
    return fail(PISA_UNSUPPORTED, "at most %d rows and keys are supported (got %d, %d)", kLongest, s->q_len, s->kv_len);
  if ((long long)s->batch * s->heads > 65535)
    return fail(PISA_UNSUPPORTED, "batch * heads = %lld exceeds 65535", (long long)s->batch * s->heads);
  const long long tiles = std::max(((long long)s->q_len + 127) / 128, ((long long)s->kv_len + 127) / 128);
  // a launch has below 2^32 threads
  if ((long long)s->batch * s->heads * tiles >= (1LL << 24) - 8) return fail(PISA_UNSUPPORTED, "tensor too large");
  m->batch = s->batch;
  m->heads = s->heads;
  m->kv_heads = s->kv_heads;
  m->group = s->heads / s->kv_heads;
  m->q_len = s->q_len;
  m->kv_len = s->kv_len;
  m->d = s->head_dim;
  m->dtype = s->dtype;
  m->causal = s->causal;
  m->n_docs = s->num_docs;
  m->cap = s->softcap;
  const Extent nq{s->batch, s->heads, s->q_len}, nk{s->batch, s->kv_heads, s->kv_len};
  rc = resolve_strides("q", s->q, nq, m->d, m->dtype, false, &m->sq);
  if (rc == PISA_OK) rc = resolve_strides("k", s->k, nk, m->d, m->dtype, false, &m->sk);
  if (rc == PISA_OK) rc = resolve_strides("v", s->v, nk, m->d, m->dtype, false, &m->sv);
  if (rc == PISA_OK) rc = resolve_strides("out", s->out, nq, m->d, m->dtype, true, &m->so);
  return rc;
}

int32_t check_mask(const Masked& m, const int32_t* doc_offsets, const int32_t* prefix) {
  if ((m.n_docs > 0) != (doc_offsets != nullptr))
    return fail(PISA_INVALID_ARG, "doc_offsets must be given if and only if num_docs > 0 (num_docs = %d)", m.n_docs);
  if (prefix && !m.causal) return fail(PISA_INVALID_ARG, "prefix needs causal (without it every row sees its whole document)");
  return PISA_OK;
}

int32_t resolve_paged(const pisa_paged_shape* s, Paged* p) {
  *p = Paged{};
  if (!s) return fail(PISA_INVALID_ARG, "shape is NULL");
  if (s->seqs < 1 || s->num_pages < 1 || s->max_pages < 1)
    return fail(PISA_INVALID_ARG, "seqs, num_pages and max_pages must be >= 1 (got %d, %d, %d)", s->seqs, s->num_pages, s->max_pages);
  if (s->page_size < 1 || s->page_size > 65536) return fail(PISA_INVALID_ARG, "page_size = %d outside [1, 65536]", s->page_size);
  int32_t rc = check_heads(s->heads, s->kv_heads);
  if (rc == PISA_OK) rc = check_type(s->dtype, s->head_dim);
  if (rc == PISA_OK) rc = check_scores(s->scale, s->softcap, s->head_dim, &p->scale);
  if (rc != PISA_OK) return rc;
  if ((long long)s->max_pages * s->page_size > (1LL << 30))
    return fail(PISA_UNSUPPORTED, "a row of the page table may hold at most 2^30 tokens (got %lld)", (long long)s->max_pages * s->page_size);
  if ((long long)s->seqs * s->heads >= (1LL << 24))        // a launch has below 2^32 threads
    return fail(PISA_UNSUPPORTED, "seqs * heads = %lld is not below 2^24", (long long)s->seqs * s->heads);
  p->seqs = s->seqs;
  p->heads = s->heads;
  p->kv_heads = s->kv_heads;
  p->group = s->heads / s->kv_heads;
  p->d = s->head_dim;
  p->dtype = s->dtype;
  p->page_size = s->page_size;
  p->num_pages = s->num_pages;
  p->max_pages = s->max_pages;
  p->cap = s->softcap;
  // all strides 0: [num_pages, page_size, kv_heads, d]
  const pisa_strides dense{(int64_t)s->page_size * s->kv_heads * s->head_dim, s->head_dim, (int64_t)s->kv_heads * s->head_dim};
  auto given = [&](const pisa_strides& t) { return t.batch == 0 && t.head == 0 && t.token == 0 ? dense : t; };
  const Extent n{s->num_pages, s->kv_heads, s->page_size};
  rc = resolve_strides("k_pages", given(s->k_pages), n, p->d, p->dtype, true, &p->sk);
  if (rc == PISA_OK) rc = resolve_strides("v_pages", given(s->v_pages), n, p->d, p->dtype, true, &p->sv);
  return rc;
}

}  // namespace
}  // namespace pisa

using namespace pisa;

#define PISA_CHECK_ALIGN(...)                                                                   \
  if (misaligned({__VA_ARGS__})) return fail(PISA_INVALID_ARG, "tensor and workspace pointers must be 16-byte aligned")
#define PISA_CHECK_WORKSPACE(need)                                                                                          \
  do {                                                                                                                      \
    if ((need) > 0 && !workspace) return fail(PISA_INVALID_ARG, "workspace is NULL (need %zu bytes)", (size_t)(need));      \
    if (workspace_bytes < (need))                                                                                           \
      return fail(PISA_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, need %zu", workspace_bytes, (size_t)(need));          \
  } while (0)

extern "C" {

size_t pisa_masked_attention_workspace_bytes(const pisa_masked_shape* shape) {
  Masked m;
  return resolve_masked(shape, &m) == PISA_OK ? masked_workspace_bytes(m) : 0;
}

int32_t pisa_masked_attention(const pisa_masked_shape* shape, const void* q, const void* k, const void* v,
                              const int32_t* doc_offsets, const int32_t* prefix, const float* slopes,
                              void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  Masked m;
  int32_t rc = resolve_masked(shape, &m);
  if (rc == PISA_OK) rc = check_mask(m, doc_offsets, prefix);
  if (rc != PISA_OK) return rc;
  if (!q || !out || (m.kv_len > 0 && (!k || !v))) return fail(PISA_INVALID_ARG, "q, k, v, out must not be NULL");
  PISA_CHECK_ALIGN(q, k, v, doc_offsets, prefix, slopes, out, lse, workspace);
  PISA_CHECK_WORKSPACE(masked_workspace_bytes(m));
  m.q = static_cast<const unsigned char*>(q);
  m.k = static_cast<const unsigned char*>(k);
  m.v = static_cast<const unsigned char*>(v);
  m.out = static_cast<unsigned char*>(out);
  m.lse = lse;
  m.docs = doc_offsets;
  m.prefix = prefix;
  m.slopes = slopes;
  m.workspace = workspace;
  const hipError_t e = launch_masked_attention(m, (hipStream_t)stream);
  return e == hipSuccess ? PISA_OK : launch_failed("pisa_masked_attention", e);
}

size_t pisa_masked_attention_backward_workspace_bytes(const pisa_masked_shape* shape) {
  Masked m;
  return resolve_masked(shape, &m) == PISA_OK ? masked_backward_workspace_bytes(m) : 0;
}

int32_t pisa_masked_attention_backward(const pisa_masked_shape* shape, const pisa_grad_strides* strides,
                                       const void* q, const void* k, const void* v, const void* out, const float* lse,
                                       const void* dout, const int32_t* doc_offsets, const int32_t* prefix,
                                       const float* slopes, void* dq, void* dk, void* dv,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  Masked m;
  int32_t rc = resolve_masked(shape, &m);
  if (rc == PISA_OK) rc = check_mask(m, doc_offsets, prefix);
  if (rc != PISA_OK) return rc;
  if (!q || !out || !lse || !dout || !dq) return fail(PISA_INVALID_ARG, "q, out, lse, dout, dq must not be NULL");
  if (m.kv_len > 0 && (!k || !v || !dk || !dv)) return fail(PISA_INVALID_ARG, "k, v, dk, dv must not be NULL");
  const Extent nq{m.batch, m.heads, m.q_len}, nk{m.batch, m.kv_heads, m.kv_len};
  rc = resolve_strides("dout", strides ? strides->dout : shape->out, nq, m.d, m.dtype, false, &m.sdo);
  if (rc == PISA_OK) rc = resolve_strides("dq", strides ? strides->dq : shape->q, nq, m.d, m.dtype, true, &m.sdq);
  if (rc == PISA_OK) rc = resolve_strides("dk", strides ? strides->dk : shape->k, nk, m.d, m.dtype, true, &m.sdk);
  if (rc == PISA_OK) rc = resolve_strides("dv", strides ? strides->dv : shape->v, nk, m.d, m.dtype, true, &m.sdv);
  if (rc != PISA_OK) return rc;
  if ((long long)m.group * ((m.q_len + 63) / 64) >= (1LL << 30)) return fail(PISA_UNSUPPORTED, "tensor too large");
  PISA_CHECK_ALIGN(q, k, v, out, lse, dout, doc_offsets, prefix, slopes, dq, dk, dv, workspace);
  PISA_CHECK_WORKSPACE(masked_backward_workspace_bytes(m));
  m.q = static_cast<const unsigned char*>(q);
  m.k = static_cast<const unsigned char*>(k);
  m.v = static_cast<const unsigned char*>(v);
  m.o = static_cast<const unsigned char*>(out);
  m.dout = static_cast<const unsigned char*>(dout);
  m.lse = const_cast<float*>(lse);
  m.dq = static_cast<unsigned char*>(dq);
  m.dk = static_cast<unsigned char*>(dk);
  m.dv = static_cast<unsigned char*>(dv);
  m.docs = doc_offsets;
  m.prefix = prefix;
  m.slopes = slopes;
  m.workspace = workspace;
  const hipError_t e = launch_masked_backward(m, (hipStream_t)stream);
  return e == hipSuccess ? PISA_OK : launch_failed("pisa_masked_attention_backward", e);
}

int32_t pisa_paged_append(const pisa_paged_shape* shape, const void* k, const void* v, int32_t tokens,
                          const int32_t* offsets, void* k_pages, void* v_pages,
                          const int32_t* page_table, const int32_t* lengths, void* stream) {
  Paged p;
  const int32_t rc = resolve_paged(shape, &p);
  if (rc != PISA_OK) return rc;
  if (tokens < 0) return fail(PISA_INVALID_ARG, "tokens = %d", tokens);
  if ((tokens > 0 && (!k || !v)) || !offsets || !k_pages || !v_pages || !page_table || !lengths)
    return fail(PISA_INVALID_ARG, "k, v, offsets, k_pages, v_pages, page_table, lengths must not be NULL");
  PISA_CHECK_ALIGN(k, v, offsets, k_pages, v_pages, page_table, lengths);
  if ((long long)tokens * p.kv_heads * p.d >= (1LL << 32)) return fail(PISA_UNSUPPORTED, "k and v must have below 2^32 elements");
  p.k = static_cast<unsigned char*>(k_pages);
  p.v = static_cast<unsigned char*>(v_pages);
  p.table = page_table;
  p.lengths = lengths;
  const hipError_t e = launch_paged_append(p, k, v, tokens, offsets, (hipStream_t)stream);
  return e == hipSuccess ? PISA_OK : launch_failed("pisa_paged_append", e);
}

size_t pisa_paged_attention_workspace_bytes(const pisa_paged_shape* shape) {
  Paged p;
  return resolve_paged(shape, &p) == PISA_OK ? paged_workspace_bytes(p) : 0;
}

int32_t pisa_paged_attention(const pisa_paged_shape* shape, const void* q, const void* k_pages, const void* v_pages,
                             const int32_t* page_table, const int32_t* lengths, const float* slopes,
                             void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  Paged p;
  const int32_t rc = resolve_paged(shape, &p);
  if (rc != PISA_OK) return rc;
  if (!q || !k_pages || !v_pages || !page_table || !lengths || !out)
    return fail(PISA_INVALID_ARG, "q, k_pages, v_pages, page_table, lengths, out must not be NULL");
  PISA_CHECK_ALIGN(q, k_pages, v_pages, page_table, lengths, slopes, out, lse, workspace);
  PISA_CHECK_WORKSPACE(paged_workspace_bytes(p));
  p.q = static_cast<const unsigned char*>(q);
  p.k = static_cast<unsigned char*>(const_cast<void*>(k_pages));
  p.v = static_cast<unsigned char*>(const_cast<void*>(v_pages));
  p.table = page_table;
  p.lengths = lengths;
  p.slopes = slopes;
  p.out = static_cast<unsigned char*>(out);
  p.lse = lse;
  p.workspace = workspace;
  const hipError_t e = launch_paged_attention(p, (hipStream_t)stream);
  return e == hipSuccess ? PISA_OK : launch_failed("pisa_paged_attention", e);
}

}  // extern "C"

// Masked attention: problem description shared by its host code and kernels, and the intervals that its masks are.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "pisa.h"

namespace pisa {

struct Strides {           // in bytes
  long long batch, head, token;
};

// A resolved call.  Pointers that a kernel does not use stay null.
struct Masked {
  const unsigned char *q, *k, *v, *o, *dout;
  unsigned char *out, *dq, *dk, *dv;
  float* lse;              // [batch][heads][q_len]
  const int32_t* docs;     // [batch][n_docs + 1], null if n_docs == 0
  const int32_t* prefix;   // [batch][max(n_docs, 1)], may be null
  const float* slopes;     // [heads], may be null
  Strides sq, sk, sv, so, sdo, sdq, sdk, sdv;
  int batch, heads, kv_heads, group, q_len, kv_len, d, dtype, causal, n_docs;
  float scale, cap;
  void* workspace;
};

size_t masked_workspace_bytes(const Masked& m);
hipError_t launch_masked_attention(const Masked& m, hipStream_t stream);
size_t masked_backward_workspace_bytes(const Masked& m);
hipError_t launch_masked_backward(const Masked& m, hipStream_t stream);

// Keys (of a row) or rows (of a key): lo <= x < hi; empty where lo >= hi.
struct Interval {
  int lo, hi;
};

// The document of position pos in batch element b: its first position and its end, clamped to the sequence; false: padding.
__device__ inline bool document_of(const Masked& m, int b, int pos, int* first, int* end, int* doc) {
  if (m.n_docs == 0) {
    *first = 0;
    *end = m.kv_len;
    *doc = 0;
    return true;
  }
  const int32_t* offs = m.docs + (long long)b * (m.n_docs + 1);
  int lo = 0, hi = m.n_docs + 1;                  // the last offset <= pos is number lo - 1
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (offs[mid] <= pos) lo = mid + 1;
    else hi = mid;
  }
  if (pos < 0 || lo == 0 || lo > m.n_docs) return false;
  *doc = lo - 1;
  *first = max(offs[lo - 1], 0);
  *end = min(offs[lo], m.kv_len);
  return true;
}
__device__ inline int prefix_end(const Masked& m, int b, int doc, int first) {
  if (!m.prefix) return first;
  const int p = m.prefix[(long long)b * max(m.n_docs, 1) + doc];
  return first + min(max(p, 0), m.kv_len);
}

// The keys that query row `row` (< q_len) sees.
__device__ inline Interval keys_of_row(const Masked& m, int b, int row) {
  const int pos = row + m.kv_len - m.q_len;
  int first, end, doc;
  if (!document_of(m, b, pos, &first, &end, &doc)) return {0, 0};
  if (m.causal) end = min(end, max(pos + 1, prefix_end(m, b, doc, first)));
  return first < end ? Interval{first, end} : Interval{0, 0};
}

// The query rows that see key `key` (< kv_len): the same relation from the other side.
__device__ inline Interval rows_of_key(const Masked& m, int b, int key) {
  const int shift = m.kv_len - m.q_len;
  int first, end, doc;
  if (!document_of(m, b, key, &first, &end, &doc)) return {0, 0};
  int lo = m.n_docs ? max(first - shift, 0) : 0;   // without documents rows before position 0 see the prefix as well
  if (m.causal && key >= prefix_end(m, b, doc, first)) lo = max(key - shift, 0);
  const int hi = min(end - shift, m.q_len);
  return lo < hi ? Interval{lo, hi} : Interval{0, 0};
}

// What a wave's (or workgroup's) intervals have in common, over the ones that are not empty: all lie in [lo, hi), all hold
// [full_lo, full_hi).  No interval at all: lo >= hi.
struct Span {
  int lo, hi, full_lo, full_hi;
};
__device__ inline Span span_of(const Interval& iv) {
  if (iv.lo >= iv.hi) return {0x7fffffff, 0, 0, 0x7fffffff};
  return {iv.lo, iv.hi, iv.lo, iv.hi};
}
__device__ inline Span join(const Span& a, const Span& b) {
  return {min(a.lo, b.lo), max(a.hi, b.hi), max(a.full_lo, b.full_lo), min(a.full_hi, b.full_hi)};
}
// over the 32 lanes of each half (the halves hold the same), the result uniform
__device__ inline Span span_of_wave(const Interval& iv) {
  Span s = span_of(iv);
#pragma unroll
  for (int x = 1; x < 32; x <<= 1)
    s = join(s, Span{__shfl_xor(s.lo, x), __shfl_xor(s.hi, x), __shfl_xor(s.full_lo, x), __shfl_xor(s.full_hi, x)});
  return {__builtin_amdgcn_readfirstlane(s.lo), __builtin_amdgcn_readfirstlane(s.hi), __builtin_amdgcn_readfirstlane(s.full_lo),
          __builtin_amdgcn_readfirstlane(s.full_hi)};
}
__device__ inline bool touches(const Span& s, int x0, int n) { return s.lo < x0 + n && s.hi > x0; }
__device__ inline bool covers(const Span& s, int x0, int n) { return s.full_lo <= x0 && s.full_hi >= x0 + n; }

// Workgroup ids are dealt round-robin to the 8 XCDs: each takes a contiguous range of items, so that one L2 serves a head.
__device__ inline int item_of_xcd(int per_xcd) { return (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8); }

}  // namespace pisa

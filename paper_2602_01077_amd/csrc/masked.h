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
hipError_t launch_masked_attention_f32(const Masked& m, hipStream_t stream);
hipError_t launch_masked_backward_f32(const Masked& m, hipStream_t stream);

// Keys (of a row) or rows (of a key): lo <= x < hi; empty where lo >= hi.
struct Interval {
  int lo, hi;
};

constexpr int kDocsInLds = 512;           // documents up to which a workgroup copies its borders to LDS
constexpr int kRankedTiles = 256;         // tiles of a head up to which masks with documents are taken by their size

// The document of position pos: its first position and its end, clamped to the sequence; false: padding.  offs: the borders.
__device__ inline bool document_of(const Masked& m, const int32_t* offs, int pos, int* first, int* end, int* doc) {
  if (m.n_docs == 0) {
    *first = 0;
    *end = m.kv_len;
    *doc = 0;
    return true;
  }
  int lo = 0, hi = m.n_docs + 1;                  // the last offset <= pos is number lo - 1
  while (lo < hi) {
    const int mid = (int)(((unsigned)lo + (unsigned)hi) >> 1);      // the sum passes 31 bits from 2^30 documents on
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
__device__ inline Interval keys_of_row(const Masked& m, const int32_t* offs, int b, int row) {
  const int pos = row + m.kv_len - m.q_len;
  int first, end, doc;
  if (!document_of(m, offs, pos, &first, &end, &doc)) return {0, 0};
  if (m.causal) end = min(end, max(pos + 1, prefix_end(m, b, doc, first)));
  return first < end ? Interval{first, end} : Interval{0, 0};
}

// The query rows that see key `key` (< kv_len): the same relation from the other side.
__device__ inline Interval rows_of_key(const Masked& m, const int32_t* offs, int b, int key) {
  const int shift = m.kv_len - m.q_len;
  int first, end, doc;
  if (!document_of(m, offs, key, &first, &end, &doc)) return {0, 0};
  int lo = m.n_docs ? max(first - shift, 0) : 0;   // without documents rows before position 0 see the prefix as well
  if (m.causal && key >= prefix_end(m, b, doc, first)) lo = max(key - shift, 0);
  const int hi = min(end - shift, m.q_len);
  return lo < hi ? Interval{lo, hi} : Interval{0, 0};
}

// The borders of batch element b, from LDS where they fit.  A barrier inside.
__device__ inline const int32_t* borders_of(const Masked& m, int b, int32_t* lds /* kDocsInLds + 1 */) {
  const int32_t* offs = m.docs + (long long)b * (m.n_docs + 1);
  if (m.n_docs == 0 || m.n_docs > kDocsInLds) return offs;
  for (int i = threadIdx.x; i <= m.n_docs; i += 256) lds[i] = offs[i];
  __syncthreads();
  return lds;
}

// Workgroup ids are dealt round-robin to the 8 XCDs.  An XCD gets whole heads, so that one L2 serves a head, as far as they go
// round, and its share of the tiles of the heads left over; a head's tiles, its own first, are numbered by rank, the ones with
// most work first, so that what is begun last is short.  Heads of an XCD are taken one after the other where there are many
// rounds of workgroups, and side by side where there are few.
struct Deal {
  int n_tiles, n_parts;    // of a head; workgroups that share a tile
  int whole, left;         // heads of an XCD; heads left over
  int side_by_side;
  int per_xcd;             // workgroups
};
inline Deal deal_of(int heads, int n_tiles, int n_parts, int slots /* of an XCD */) {
  Deal d{n_tiles, n_parts, heads / 8, heads % 8, 0, 0};
  d.per_xcd = (int)(((long long)d.whole * n_tiles + ((long long)d.left * n_tiles + 7) / 8) * n_parts);
  d.side_by_side = d.per_xcd < 4 * slots;
  return d;
}
struct Share {
  int head, rank, part;    // head < 0: none
};
__device__ inline Share share_of(const Deal& d) {
  const int xcd = blockIdx.x % 8, nth = blockIdx.x / 8;
  const int part = nth % d.n_parts;
  int m = nth / d.n_parts;
  const int left = d.left * d.n_tiles > xcd ? (d.left * d.n_tiles - xcd + 7) / 8 : 0;
  if (m < left) {
    const int u = 8 * m + xcd;
    return {8 * d.whole + u % d.left, u / d.left, part};
  }
  m -= left;
  if (m >= d.whole * d.n_tiles) return {-1, 0, 0};
  return d.side_by_side ? Share{xcd * d.whole + m % d.whole, m / d.whole, part}
                        : Share{xcd * d.whole + m / d.n_tiles, m % d.n_tiles, part};
}

// Which tile of 128 rows (or keys) has that rank: by hand where the mask is the same for all tiles or grows with them, else by
// the number of keys (rows) that its first and last row (key) see.  Barriers inside.
template <bool KEYS>
__device__ inline int tile_of_rank(const Masked& m, const int32_t* offs, int b, int rank, int n_tiles, int* size_s /* kRankedTiles + 1 */) {
  if (m.n_docs == 0 || n_tiles > kRankedTiles) return !KEYS && m.causal ? n_tiles - 1 - rank : rank;
  const int t = threadIdx.x, len = KEYS ? m.kv_len : m.q_len;
  int size = 0;
  if (t < n_tiles) {
    const int x0 = t * 128, x1 = min(x0 + 127, len - 1);
    const Interval a = KEYS ? rows_of_key(m, offs, b, x0) : keys_of_row(m, offs, b, x0);
    const Interval z = KEYS ? rows_of_key(m, offs, b, x1) : keys_of_row(m, offs, b, x1);
    if (a.lo < a.hi && z.lo < z.hi) size = max(a.hi, z.hi) - min(a.lo, z.lo);
    else size = max(a.hi - a.lo, z.hi - z.lo);
    size_s[t] = size;
  }
  __syncthreads();
  if (t < n_tiles) {
    int before = 0;
    for (int u = 0; u < n_tiles; ++u) before += size_s[u] > size || (size_s[u] == size && u < t);
    if (before == rank) size_s[kRankedTiles] = t;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(size_s[kRankedTiles]);
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

}  // namespace pisa

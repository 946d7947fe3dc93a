// Masked attention, backward: dq from a walk over the keys of 128 rows, dk and dv from a walk over the rows of 128 keys.
//
// Both walks make the scores again from q and k and the weights from the log-sum-exp that the forward pass left, so nothing
// of size q_len x kv_len is stored; seven products instead of five, and in exchange every sum is made by one workgroup in a
// fixed order, without atomics.  As in the forward pass all products are transposed:
//     dq walk (a lane holds one query row):  S^T = K Q^T,  dP^T = V dO^T,  dQ^T += K^T dS^T
//     dk, dv walk (a lane holds one key):    S = Q K^T,    dP = dO V^T,    dV^T += dO^T P,  dK^T += Q^T dS
// so that P and dS leave the first products in the lanes in which the second ones take them.  The dk, dv walk goes over the
// rows of all query heads that share the key head.
//
// Bound as the forward pass is, by products and plain operations that wait for each other: 12 heads of 8 192, causal, dq 345 us,
// dk and dv 412 (matrix cores 60 and 56 % busy, LDS 30 and 36 %); 24 heads of 4 608 without a mask 880-920 us together by card,
// 1 000-1 040 TFLOP/s over the seven products.  At 64 channels with capped and biased scores, 2 x 12 heads of 2 777, 103 and 97 us
// (matrix cores 20 and 27 %: vector instructions).
#include <algorithm>

#include "masked.h"
#include "tile.h"

namespace pisa {

using namespace tile;

namespace {

constexpr int kOwn = 128;                // rows (keys) of a workgroup, 32 to a wave
constexpr int CAP = 1, BIAS = 2;         // bits of MOD
constexpr float kHeavy = 0.1f;           // see masked_dq_kernel
constexpr int kMostHeavy = 10;           // weights of a row that can be as large

struct Plan {
  Deal deal;           // of tiles of 128 rows (dq), or keys (dk, dv) and the parts of their rows
  float* stat;         // [-lse, delta][batch][heads][q_len], the first in the domain of the scores
  float* part;         // parts > 1: [head][tile][part][dk, dv][128][d]; dq: [head][tile][part][128][d]
};

// Nothing is moved across, where registers are short.
template <bool TIGHT> __device__ __forceinline__ void phase() {
  if (TIGHT) __builtin_amdgcn_sched_barrier(0);
}

// A score and what its gradient is multiplied by.
template <typename T, int MOD> struct Scorer {
  float c, to_cap, slope;
  __device__ __forceinline__ Scorer(const Masked& p, int head) {
    const float u = sizeof(T) == 2 ? kLog2e : 1.f;
    c = (MOD & CAP ? p.cap : p.scale) * u;
    to_cap = MOD & CAP ? p.scale / p.cap : 0.f;
    slope = MOD & BIAS ? p.slopes[head] * u : 0.f;
  }
  // raw products to what weight() takes: capped ones to their tanh
  __device__ __forceinline__ void prepare(f32x16& s) const {
    if (MOD & CAP) cap_scores<T>(s, to_cap, 1.f);
  }
  // the weight exp(z - lse); `far` = pos - key; *gain = dz/ds
  __device__ __forceinline__ float weight(float s, float minus_lse, float far, float* gain) const {
    *gain = MOD & CAP ? __builtin_amdgcn_fmed3f(fmaf(-s, s, 1.f), 0.f, 1.f) : 1.f;       // within [0, 1] for s = -inf as well
    return exp_diff<T>(s, c, MOD & BIAS ? fmaf(-slope, fabsf(far), minus_lse) : minus_lse);
  }
};
template <typename T> __device__ __forceinline__ float in_domain(float lse) { return sizeof(T) == 2 ? lse * kLog2e : lse; }

__device__ __forceinline__ Span span_of_group(const Span& ws, int (*span_s)[4], int wave, int lane) {
  if (lane == 0) {
    span_s[wave][0] = ws.lo;
    span_s[wave][1] = ws.hi;
    span_s[wave][2] = ws.full_lo;
    span_s[wave][3] = ws.full_hi;
  }
  __syncthreads();
  Span gs{span_s[0][0], span_s[0][1], span_s[0][2], span_s[0][3]};
#pragma unroll
  for (int w = 1; w < 4; ++w) gs = join(gs, Span{span_s[w][0], span_s[w][1], span_s[w][2], span_s[w][3]});
  return Span{__builtin_amdgcn_readfirstlane(gs.lo), __builtin_amdgcn_readfirstlane(gs.hi), __builtin_amdgcn_readfirstlane(gs.full_lo),
              __builtin_amdgcn_readfirstlane(gs.full_hi)};
}

template <typename T> __device__ __forceinline__ float dot16(u32x4 a, u32x4 b) {      // of 16 bytes each
  float d = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (sizeof(T) == 2) {
      d = fmaf(__uint_as_float(a[e] << 16), __uint_as_float(b[e] << 16), d);
      d = fmaf(__uint_as_float(a[e] & 0xffff0000u), __uint_as_float(b[e] & 0xffff0000u), d);
    } else {
      d = fmaf(__uint_as_float(a[e]), __uint_as_float(b[e]), d);
    }
  }
  return d;
}

template <typename T> __device__ __forceinline__ f32x4 four_of(const unsigned char* src) {      // elements that lie together
  if constexpr (sizeof(T) == 4) return *reinterpret_cast<const f32x4*>(src);
  const u32x2 x = *reinterpret_cast<const u32x2*>(src);
  return f32x4{__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u)};
}

// The lane's row of sums, times f; zeros unless `some` (the sums of a row that has none can hold anything).
template <typename T, int D>
__device__ __forceinline__ void store_row(unsigned char* dst, const f32x16 (&acc)[Geo<T, D>::NDT], float f, bool some, int h) {
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int ch = 32 * dt + 8 * g + 4 * h;
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = some ? acc[dt][4 * g + e] * f : 0.f;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<u32x2*>(dst + 2 * ch) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
      else
        *reinterpret_cast<f32x4*>(dst + 4 * ch) = x;
    }
}

template <typename T, int D, int MOD>
__global__ __launch_bounds__(256, sizeof(T) == 2 || D == 64 ? 2 : 1) void masked_dq_kernel(Masked p, Plan plan) {
  using G = Geo<T, D>;
  constexpr int TILEB = G::TILEB, NDT = G::NDT;
  __shared__ __attribute__((aligned(1024))) unsigned char stage[4 * TILEB];      // K0 | V0 | K1 | V1
  constexpr bool MENDS = sizeof(T) == 2;
  __shared__ int span_s[4][4];
  __shared__ unsigned bad[2];
  // by thread: of its row, keys with its h; weight times dz/ds in 255ths (it multiplies a correction), above a key below 2^24
  __shared__ unsigned heavy[MENDS ? kMostHeavy : 1][MENDS ? 256 : 1];

  __shared__ int32_t docs_s[kDocsInLds + 1];
  __shared__ int size_s[kRankedTiles + 1];

  const Share share = share_of(plan.deal);
  if (share.head < 0) return;
  const int bh = share.head, b = bh / p.heads, head = bh % p.heads;
  const int32_t* offs = borders_of(p, b, docs_s);
  const int qt = tile_of_rank<false>(p, offs, b, share.rank, plan.deal.n_tiles, size_s);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lam = lane & 31, h = lane >> 5;
  const int row = qt * kOwn + 32 * wave + lam;
  Interval iv{0, 0};
  if (row < p.q_len) iv = keys_of_row(p, offs, b, row);
  const bool sees = iv.lo < iv.hi;
  const Span ws = span_of_wave(iv);
  if (tid < 2) bad[tid] = 0u;
  const Span gs = span_of_group(ws, span_s, wave, lane);

  const unsigned char* kg = p.k + b * p.sk.batch + (head / p.group) * p.sk.head;
  const unsigned char* vg = p.v + b * p.sv.batch + (head / p.group) * p.sv.head;
  const unsigned lds = (unsigned)(unsigned long long)(LDS_PTR(unsigned char)) & stage[0];
  Loader<T, D, sizeof(T) == 4> lk, lv;
  lk.init(wave, lane, (unsigned)p.sk.token);
  lv.init(wave, lane, (unsigned)p.sv.token);
  Reader<T, D> rd;
  rd.init(lane, lds);
  auto load = [&](int t, int par) INLINE {
    lk.load(wave, lane, kg + (long long)t * kRows * p.sk.token, p.kv_len - t * kRows, lds + 2 * par * TILEB);
    lv.load(wave, lane, vg + (long long)t * kRows * p.sv.token, p.kv_len - t * kRows, lds + (2 * par + 1) * TILEB);
  };
  int t_begin = 0, t_end = 0;
  if (gs.lo < gs.hi) {
    t_begin = gs.lo / kRows;
    t_end = (gs.hi + kRows - 1) / kRows;
  }
  if (!MENDS && plan.deal.n_parts > 1) {
    const int n = t_end - t_begin, first = t_begin;
    t_begin = first + (int)((long long)n * share.part / plan.deal.n_parts);
    t_end = first + (int)((long long)n * (share.part + 1) / plan.deal.n_parts);
  }
  if (t_begin < t_end) load(t_begin, 0);

  u32x4 q[G::STEPS], g[G::STEPS];                // the lane's rows of q and dout; zeros where the row sees nothing
  // Rows without a score above -inf have weights of 0, also those past the last: weights of 1, as rows of zeros would have, make
  // their wave look for heavy keys in every tile (8 heads of 130 rows on 2 000 keys, backward 118 us, 76 so).
  float delta = 0.f, minus_lse = -INFINITY;
  {
    const unsigned char* qs = p.q + b * p.sq.batch + head * p.sq.head + (long long)row * p.sq.token;
    const unsigned char* gsrc = p.dout + b * p.sdo.batch + head * p.sdo.head + (long long)row * p.sdo.token;
    const unsigned char* os = p.o + b * p.so.batch + head * p.so.head + (long long)row * p.so.token;
#pragma unroll
    for (int s = 0; s < G::STEPS; ++s) {
      q[s] = g[s] = u32x4{0, 0, 0, 0};
      if (sees) {
        q[s] = *reinterpret_cast<const u32x4*>(qs + 32 * s + 16 * h);
        g[s] = *reinterpret_cast<const u32x4*>(gsrc + 32 * s + 16 * h);
        delta += dot16<T>(g[s], *reinterpret_cast<const u32x4*>(os + 32 * s + 16 * h));
      }
    }
    delta += __shfl_xor(delta, 32);
    const float lse = sees ? p.lse[(size_t)bh * p.q_len + row] : -INFINITY;
    if (lse != -INFINITY) minus_lse = -in_domain<T>(lse);
  }
  const bool some = minus_lse != -INFINITY;
  const Scorer<T, MOD> sc(p, head);
  const int pos = row + p.kv_len - p.q_len;

  f32x16 acc[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) acc[dt] = (f32x16){0};
  // bf16: delta from a rounded out is off by e = -sum_j dz_ij (the sum is 0 otherwise), and dq by -e sum_j p_ij k_j, which is
  // as much as the other roundings together where few keys have most of a row's weight.  e is known when the walk is done; the
  // part of that sum that weights of kHeavy and more have, of which a row has few, is taken out then.  (The others' does not
  // matter: the sum falls with the number of keys that share the weight, and so does e.)  The two sums a score and the search for
  // such weights cost 1 % of the backward pass of long calls (24 heads of 4 608 913 -> 921 us; 64 channels 520 -> 540), 17 % of
  // short ones (8 heads of 1 024 62.8 -> 73.7; 69.6 with weights from 0.1875 on).
  float off = 0.f;
  int n_heavy = 0;

  auto trip = [&](int t, auto parity) INLINE {
    const int par = parity;
    const unsigned k_off = 2 * par * TILEB, v_off = k_off + TILEB;
    wait_loads();
    __syncthreads();
    if (t + 1 < t_end) load(t + 1, par ^ 1);
    if (!covers(gs, t * kRows, kRows)) {         // the product with K contracts over keys that not every row sees
      clean_tile<T, D>((LDS_PTR(unsigned char))&stage[0] + k_off, (LDS_PTR(unsigned))&bad[0], tid);
      __syncthreads();
    }
    if (!touches(ws, t * kRows, kRows)) return;
    const bool part = !covers(ws, t * kRows, kRows);
    auto half = [&](auto row0_tag) INLINE {
      constexpr int ROW0 = decltype(row0_tag)::value;
      f32x16 s = rows_times<T, D, ROW0>(rd, k_off, q);
      sc.prepare(s);
      f32x16 dp = rows_times<T, D, ROW0>(rd, v_off, g);
      Weights<T> w;
      const int key0 = t * kRows + ROW0 + 4 * h;
      if (part) {                                // masked keys: score -inf, nothing of v
        asm volatile("");                        // a branch: selects for every tile took a quarter of the walk's plain operations
        const unsigned n = (unsigned)(iv.hi - iv.lo);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if ((unsigned)(key0 + (r / 4) * 8 + r % 4 - iv.lo) >= n) {
            s[r] = -INFINITY;
            dp[r] = 0.f;
          }
      }
      const float ahead = (float)(pos - key0);
      float top = 0.f;
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        float x[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float gain;
          const float wt = sc.weight(s[r + u], minus_lse, ahead - (float)(((r + u) / 4) * 8 + (r + u) % 4), &gain);
          x[u] = wt * (dp[r + u] - delta);
          if (MENDS) {
            off += x[u];
            top = fmaxf(top, wt);
          }
          if (MOD & CAP) x[u] *= gain;
        }
        w.set(r, x[0], x[1]);
      }
      if (MENDS && __builtin_expect(__any(top >= kHeavy), 0)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = key0 + (r / 4) * 8 + r % 4;
          float gain;
          const float wt = sc.weight(s[r], minus_lse, ahead - (float)((r / 4) * 8 + r % 4), &gain);
          if (wt >= kHeavy && (unsigned)(key - iv.lo) < (unsigned)(iv.hi - iv.lo) && n_heavy < kMostHeavy) {
            heavy[n_heavy][tid] = (unsigned)fminf(fmaf(wt * gain, 255.f, 0.5f), 255.f) << 24 | (unsigned)key;
            ++n_heavy;
          }
        }
      }
      cols_times<T, D, ROW0>(rd, k_off, w, acc);
    };
    half(std::integral_constant<int, 0>{});
    half(std::integral_constant<int, 32>{});
  };
  walk_stages<T>(t_begin, t_end, trip);
  // Keys of inf or NaN in the tiles that were cleaned of them: their channels are NaN for the rows that see them.  The walk only
  // remembers that there were any.
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(bad[0] | bad[1]) != 0u, 0))
    for (int t = t_begin; t < t_end; ++t) {
      if (covers(gs, t * kRows, kRows)) continue;
      __syncthreads();
      if (tid < 2) bad[tid] = 0u;
      __syncthreads();
      mark_rows<T, D>(kg + (long long)t * kRows * p.sk.token, p.sk.token, p.kv_len - t * kRows, (LDS_PTR(unsigned))&bad[0], tid);
      __syncthreads();
#pragma unroll 1
      for (int r = 0; r < kRows; ++r) {
        if (!((__builtin_amdgcn_readfirstlane(bad[r >> 5]) >> (r & 31)) & 1u)) continue;
        const int key = t * kRows + r;
        const T* src = reinterpret_cast<const T*>(kg + (long long)key * p.sk.token);
        const bool mine = key >= iv.lo && key < iv.hi;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = (float)src[32 * dt + (e / 4) * 8 + 4 * h + e % 4];
            acc[dt][e] = fmaf(mine ? x : 0.f, 0.f, acc[dt][e]);
          }
      }
    }
  if constexpr (MENDS) {
    off += __shfl_xor(off, 32);
    delta += off;
    const int others = __shfl_xor(n_heavy, 32);
    const int counts[2] = {h ? others : n_heavy, h ? n_heavy : others};
#pragma unroll
    for (int half = 0; half < 2; ++half)         // the row's keys of h = 0, then of h = 1, by either lane for its channels
      for (int e = 0; __any(e < counts[half]); ++e)
        if (e < counts[half]) {
          const int of = (tid & ~32) + 32 * half;
          const unsigned entry = heavy[e][of];
          const T* src = reinterpret_cast<const T*>(kg + (long long)(entry & 0xffffffu) * p.sk.token);
          const float f = -off * ((float)(entry >> 24) * (1.f / 255.f));
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const u32x2 x = *reinterpret_cast<const u32x2*>(src + 32 * dt + 8 * g + 4 * h);
              acc[dt][4 * g] = fmaf(f, __uint_as_float(x.x << 16), acc[dt][4 * g]);
              acc[dt][4 * g + 1] = fmaf(f, __uint_as_float(x.x & 0xffff0000u), acc[dt][4 * g + 1]);
              acc[dt][4 * g + 2] = fmaf(f, __uint_as_float(x.y << 16), acc[dt][4 * g + 2]);
              acc[dt][4 * g + 3] = fmaf(f, __uint_as_float(x.y & 0xffff0000u), acc[dt][4 * g + 3]);
            }
        }
  }
  if (row < p.q_len && h == 0 && share.part == 0) {
    float* st = plan.stat + (size_t)bh * p.q_len + row;
    st[0] = minus_lse;
    st[(size_t)p.batch * p.heads * p.q_len] = some ? delta : 0.f;
  }
  if (!MENDS && plan.deal.n_parts > 1) {
    const size_t item = ((size_t)bh * plan.deal.n_tiles + qt) * plan.deal.n_parts + share.part;
    store_row<float, D>(reinterpret_cast<unsigned char*>(plan.part + (item * kOwn + 32 * wave + lam) * D), acc, p.scale, some, h);
    return;
  }
  if (row < p.q_len)
    store_row<T, D>(p.dq + b * p.sdq.batch + head * p.sdq.head + (long long)row * p.sdq.token, acc, p.scale, some, h);
}

template <typename T, int D, int MOD>
__global__ __launch_bounds__(256, sizeof(T) == 2 || D == 64 ? 2 : 1) void masked_dkv_kernel(Masked p, Plan plan) {
  using G = Geo<T, D>;
  constexpr int TILEB = G::TILEB, NDT = G::NDT;
  constexpr bool TIGHT = sizeof(T) == 2 && D == 128, ANEW = TIGHT || sizeof(T) == 4;
  __shared__ __attribute__((aligned(1024))) unsigned char stage[4 * TILEB];      // Q0 | dO0 | Q1 | dO1
  __shared__ __attribute__((aligned(16))) float stat[2][2][kRows];               // [parity][-lse, delta][row]
  __shared__ Interval seen_s[kOwn];              // for the tiles that need it: no registers for it in the walk
  __shared__ int span_s[4][4];
  __shared__ unsigned bad[2];

  __shared__ int32_t docs_s[kDocsInLds + 1];
  __shared__ int size_s[kRankedTiles + 1];

  const Share share = share_of(plan.deal);
  if (share.head < 0) return;
  const int bk = share.head, b = bk / p.kv_heads, kv_head = bk % p.kv_heads;
  const int32_t* offs = borders_of(p, b, docs_s);
  const int kt = tile_of_rank<true>(p, offs, b, share.rank, plan.deal.n_tiles, size_s);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lam = lane & 31, h = lane >> 5;
  const int key = kt * kOwn + 32 * wave + lam;
  Interval iv{0, 0};
  if (key < p.kv_len) iv = rows_of_key(p, offs, b, key);
  const bool seen = iv.lo < iv.hi;
  seen_s[32 * wave + lam] = iv;
  const Span ws = span_of_wave(iv);
  if (tid < 2) bad[tid] = 0u;
  const Span gs = span_of_group(ws, span_s, wave, lane);

  const unsigned lds = (unsigned)(unsigned long long)(LDS_PTR(unsigned char)) & stage[0];
  const unsigned lds_stat = (unsigned)(unsigned long long)(LDS_PTR(float)) & stat[0][0][0];
  Loader<T, D, ANEW> lq, lg;
  lq.init(wave, lane, (unsigned)p.sq.token);
  lg.init(wave, lane, (unsigned)p.sdo.token);
  Reader<T, D> rd;
  rd.init(lane, lds);

  // The walk: tiles t_begin .. of rows, for one query head of the group after the other; this workgroup's part of it.
  int t_begin = 0, n = 0;
  if (gs.lo < gs.hi) {
    t_begin = gs.lo / kRows;
    n = (gs.hi + kRows - 1) / kRows - t_begin;
  }
  const long long steps = (long long)n * p.group;
  const int i_begin = (int)(steps * share.part / plan.deal.n_parts), i_end = (int)(steps * (share.part + 1) / plan.deal.n_parts);
  int head = kv_head * p.group, t = t_begin;     // of the tile that is loaded next
  if (n > 0) {
    head += i_begin / n;
    t += i_begin % n;
  }
  const size_t all_rows = (size_t)p.batch * p.heads * p.q_len;
  auto load = [&](int par) INLINE {
    const int avail = p.q_len - t * kRows;
    if (wave < 2) {
      const float* st = plan.stat + wave * all_rows + ((size_t)b * p.heads + head) * p.q_len + t * kRows;
      dma_words(lds_stat + (par * 2 + wave) * (kRows * 4), (unsigned)(min(TIGHT ? lane_anew() : lane, avail - 1) * 4), st);
    }
    lq.load(wave, lane, p.q + b * p.sq.batch + head * p.sq.head + (long long)t * kRows * p.sq.token, avail, lds + 2 * par * TILEB);
    lg.load(wave, lane, p.dout + b * p.sdo.batch + head * p.sdo.head + (long long)t * kRows * p.sdo.token, avail,
            lds + (2 * par + 1) * TILEB);
  };

  u32x4 k[G::STEPS], v[G::STEPS];
  {
    const unsigned char* ks = p.k + b * p.sk.batch + kv_head * p.sk.head + (long long)key * p.sk.token;
    const unsigned char* vs = p.v + b * p.sv.batch + kv_head * p.sv.head + (long long)key * p.sv.token;
#pragma unroll
    for (int s = 0; s < G::STEPS; ++s) {
      k[s] = v[s] = u32x4{0, 0, 0, 0};
      if (seen) {
        k[s] = *reinterpret_cast<const u32x4*>(ks + 32 * s + 16 * h);
        v[s] = *reinterpret_cast<const u32x4*>(vs + 32 * s + 16 * h);
      }
    }
  }
  f32x16 dk[NDT], dv[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) dk[dt] = dv[dt] = (f32x16){0};

  if (i_begin < i_end) load(0);
  const int shift = p.kv_len - p.q_len;
  auto trip = [&](int i, auto parity) INLINE {
    const int par = parity;
    const unsigned q_off = 2 * par * TILEB, g_off = q_off + TILEB;
    const int x0 = t * kRows, head_now = head;
    wait_loads();
    __syncthreads();
    if (i + 1 < i_end) {
      if (++t == t_begin + n) {
        t = t_begin;
        ++head;
      }
      load(par ^ 1);
    }
    if (!covers(gs, x0, kRows)) {         // both second products contract over rows that do not all see every key
      const int thread = TIGHT ? 64 * wave + lane_anew() : tid;
      clean_tile<T, D>((LDS_PTR(unsigned char))&stage[0] + q_off, (LDS_PTR(unsigned))&bad[0], thread);
      clean_tile<T, D>((LDS_PTR(unsigned char))&stage[0] + g_off, (LDS_PTR(unsigned))&bad[0], thread);
      __syncthreads();
    }
    if (!touches(ws, x0, kRows)) return;
    const bool part = !covers(ws, x0, kRows);
    const Scorer<T, MOD> sc(p, head_now);
    auto half = [&](auto row0_tag) INLINE {
      constexpr int ROW0 = decltype(row0_tag)::value;
      // 192 of 256 registers hold k, v, dk and dv: addresses and row numbers are made anew where they are wanted, and the
      // products are kept apart from what follows, or the scheduler spills to feed them early
      if (TIGHT) asm volatile("" : "+v"(rd.rows), "+v"(rd.cols));
      f32x16 s = rows_times<T, D, ROW0>(rd, q_off, k);
      sc.prepare(s);
      f32x16 dp = rows_times<T, D, ROW0>(rd, g_off, v);
      phase<TIGHT>();
      Weights<T> wp, wd;
      const int ln = TIGHT ? lane_anew() : lane, h = ln >> 5, own = 32 * wave + (ln & 31);   // own: this lane's key of the tile
      const int row0 = x0 + ROW0 + 4 * h;
      const float ahead = (float)(row0 + shift - (kt * kOwn + own));
      auto stat4 = [&](int which, int e) INLINE {
        return *reinterpret_cast<LDS_PTR(const f32x4)>((LDS_PTR(const float))&stat[par][which][ROW0 + 8 * e + 4 * h]);
      };
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 ml = stat4(0, e), de = stat4(1, e);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int r = 4 * e + u;
          float gain;
          s[r] = sc.weight(s[r], ml[u], ahead + (float)(8 * e + u), &gain);
          dp[r] = s[r] * (dp[r] - de[u]);
          if (MOD & CAP) dp[r] *= gain;
        }
      }
      if (part) {
        asm volatile("");                        // a branch, as in masked_dq_kernel
        const int lo = seen_s[own].lo;
        const unsigned count = (unsigned)(seen_s[own].hi - lo);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if ((unsigned)(row0 + (r / 4) * 8 + r % 4 - lo) >= count) s[r] = dp[r] = 0.f;
      }
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        wp.set(r, s[r], s[r + 1]);
        wd.set(r, dp[r], dp[r + 1]);
      }
      phase<TIGHT>();
      cols_times<T, D, ROW0>(rd, g_off, wp, dv);
      cols_times<T, D, ROW0>(rd, q_off, wd, dk);
    };
    half(std::integral_constant<int, 0>{});
    phase<TIGHT>();
    half(std::integral_constant<int, 32>{});
  };
  walk_stages<T>(i_begin, i_end, trip);
  // Rows of inf or NaN in the tiles that were cleaned of them, for the keys that see them: dv takes dout's as they are (a weight is
  // positive), dk is NaN where q's are (0 * inf: such a score is one of -inf, or capped, or NaN), and delta, made of dout as it is,
  // has already reached all of dk.  The walk only remembers that there were any.
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(bad[0] | bad[1]) != 0u, 0))
    for (int i = 0; i < n * p.group; ++i) {      // all steps, those of other parts as well: either way the sums are not finite
      const int ln = lane_anew(), thread = 64 * wave + ln, h = ln >> 5;
      const int x0 = (t_begin + i % n) * kRows, head_now = kv_head * p.group + i / n;
      if (covers(gs, x0, kRows)) continue;
      const unsigned char* qs = p.q + b * p.sq.batch + head_now * p.sq.head + (long long)x0 * p.sq.token;
      const unsigned char* ds = p.dout + b * p.sdo.batch + head_now * p.sdo.head + (long long)x0 * p.sdo.token;
      __syncthreads();
      if (thread < 2) bad[thread] = 0u;
      __syncthreads();
      mark_rows<T, D>(qs, p.sq.token, p.q_len - x0, (LDS_PTR(unsigned))&bad[0], thread);
      mark_rows<T, D>(ds, p.sdo.token, p.q_len - x0, (LDS_PTR(unsigned))&bad[0], thread);
      __syncthreads();
#pragma unroll 1
      for (int r = 0; r < kRows; ++r) {
        if (!((__builtin_amdgcn_readfirstlane(bad[r >> 5]) >> (r & 31)) & 1u)) continue;
        const unsigned char *qr = qs + r * p.sq.token + 4 * h * sizeof(T), *dr = ds + r * p.sdo.token + 4 * h * sizeof(T);
        const Interval rows = seen_s[32 * wave + (ln & 31)];
        const bool mine = x0 + r >= rows.lo && x0 + r < rows.hi;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            phase<true>();
            const f32x4 x = four_of<T>(dr + (32 * dt + 2 * e) * sizeof(T)), y = four_of<T>(qr + (32 * dt + 2 * e) * sizeof(T));
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              dv[dt][e + u] += mine && !(fabsf(x[u]) < INFINITY) ? x[u] : 0.f;
              dk[dt][e + u] = fmaf(mine ? y[u] : 0.f, 0.f, dk[dt][e + u]);
            }
          }
      }
    }

  if (plan.deal.n_parts > 1) {
    const size_t item = ((size_t)bk * plan.deal.n_tiles + kt) * plan.deal.n_parts + share.part;
    unsigned char* dst = reinterpret_cast<unsigned char*>(plan.part + (item * 2 * kOwn + 32 * wave + lam) * D);
    store_row<float, D>(dst, dk, p.scale, seen, h);
    store_row<float, D>(dst + (size_t)kOwn * D * sizeof(float), dv, 1.f, seen, h);
    return;
  }
  if (key < p.kv_len) {
    store_row<T, D>(p.dk + b * p.sdk.batch + kv_head * p.sdk.head + (long long)key * p.sdk.token, dk, p.scale, seen, h);
    store_row<T, D>(p.dv + b * p.sdv.batch + kv_head * p.sdv.head + (long long)key * p.sdv.token, dv, 1.f, seen, h);
  }
}

// Adds the parts of 128 rows: a thread has four channels of one.  blockIdx.z: which of the tensors that lie side by side.
struct JoinTo {
  unsigned char* at[2];
  Strides stride[2];
  int heads, len, count;       // count: of those tensors
};
template <typename T, int D> __global__ __launch_bounds__(256) void masked_sum_kernel(Plan plan, JoinTo to) {
  constexpr int PER_ROW = D / 4, ROWS = 256 / PER_ROW;
  const int unit = blockIdx.y, tid = threadIdx.x, which = blockIdx.z, n_parts = plan.deal.n_parts;
  const int bh = unit / plan.deal.n_tiles, b = bh / to.heads, head = bh % to.heads;
  const int r = blockIdx.x * ROWS + tid / PER_ROW, ch = 4 * (tid % PER_ROW), row = unit % plan.deal.n_tiles * kOwn + r;
  if (row >= to.len) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  const float* src = plan.part + (((size_t)unit * n_parts * to.count + which) * kOwn + r) * D + ch;
  for (int i0 = 0; i0 < n_parts; i0 += 8) {      // eight parts under way at a time
    f32x4 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i0 + u < n_parts) x[u] = *reinterpret_cast<const f32x4*>(src + (size_t)(i0 + u) * to.count * kOwn * D);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i0 + u < n_parts) sum += x[u];
  }
  const Strides& sd = to.stride[which];
  unsigned char* dst = to.at[which] + b * sd.batch + head * sd.head + (long long)row * sd.token;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<u32x2*>(dst + 2 * ch) = u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
  else
    *reinterpret_cast<f32x4*>(dst + 4 * ch) = sum;
}

int tiles_of(int n) { return (n + kOwn - 1) / kOwn; }
// Two tiles or more to a part; one where all parts still find a compute unit each (2 heads of 300 126 -> 67 us; 4 of 1 000, where
// they do not, 116 -> 144).
long long f32_parts(const Masked& m, long long units, long long tiles) {
  const long long most = ((m.d == 64 ? 512 : 768) + units - 1) / units;
  return std::max(std::min(most, tiles / 2), std::min(256 / units, tiles));
}
int at_least_one(long long parts) { return parts < 1 ? 1 : (int)parts; }
Plan plan_q(const Masked& m) {
  Plan pl{};
  const long long units = (long long)m.batch * m.heads * tiles_of(m.q_len);
  const bool f32 = m.dtype == PISA_FP32;
  // fp32 products take so long that the keys of a tile are shared out until every compute unit has three workgroups to do (two
  // at 64 channels).  bf16 walks are not: what mends delta needs a row's whole sum.
  const long long tiles = (m.kv_len + kRows - 1) / kRows;
  const long long parts = f32 ? f32_parts(m, units, tiles) : 1;
  pl.deal = deal_of(m.batch * m.heads, tiles_of(m.q_len), at_least_one(parts), f32 ? 32 : 64);
  return pl;
}
Plan plan_kv(const Masked& m) {
  Plan pl{};
  const long long units = (long long)m.batch * m.kv_heads * tiles_of(m.kv_len);
  if (units == 0) return pl;
  // A key tile's rows are shared out where the tiles alone do not fill two rounds of the 512 places on the card (backward pass,
  // us, whole / shared out: 2 x 4 key heads of 2 777, 64 channels, 583 / 259; 13 heads of 6 000, causal, 988 / 845).  Causal
  // tiles differ in size and leave places idle for longer: up to 800 (12 of 8 192 1 112 / 1 018), the others up to 640 (24 of
  // 4 000 in documents, 768 tiles, 323 / 352).
  const bool f32 = m.dtype == PISA_FP32;
  const long long steps = (long long)m.group * ((m.q_len + kRows - 1) / kRows);
  const long long parts = f32 ? f32_parts(m, units, steps)
                              : (units >= (m.causal ? 800 : 640) ? 1 : std::min((1024 + units - 1) / units, steps / 4));
  pl.deal = deal_of(m.batch * m.kv_heads, tiles_of(m.kv_len), at_least_one(parts), f32 ? 32 : 64);
  return pl;
}
// Floats of the parts' sums: dq's are added up before the dk, dv walk writes its own.
size_t part_floats(const Masked& m, const Plan& pq, const Plan& pk) {
  const size_t q = pq.deal.n_parts > 1 ? (size_t)m.batch * m.heads * pq.deal.n_tiles * pq.deal.n_parts * kOwn * m.d : 0;
  const size_t k = pk.deal.n_parts > 1 ? (size_t)m.batch * m.kv_heads * pk.deal.n_tiles * pk.deal.n_parts * 2 * kOwn * m.d : 0;
  return std::max(q, k);
}

template <typename T, int D, int MOD> hipError_t launch_mod(const Masked& m, const Plan& pq, const Plan& pk, hipStream_t stream) {
  const dim3 block(256);
  const int slices = kOwn / (256 / (D / 4));
  hipLaunchKernelGGL((masked_dq_kernel<T, D, MOD>), dim3(8 * pq.deal.per_xcd), block, 0, stream, m, pq);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (pq.deal.n_parts > 1) {
    const JoinTo to{{m.dq, nullptr}, {m.sdq, {}}, m.heads, m.q_len, 1};
    hipLaunchKernelGGL((masked_sum_kernel<T, D>), dim3(slices, m.batch * m.heads * pq.deal.n_tiles, 1), block, 0, stream, pq, to);
    e = hipGetLastError();
  }
  if (e != hipSuccess || m.kv_len == 0) return e;
  hipLaunchKernelGGL((masked_dkv_kernel<T, D, MOD>), dim3(8 * pk.deal.per_xcd), block, 0, stream, m, pk);
  e = hipGetLastError();
  if (e != hipSuccess || pk.deal.n_parts == 1) return e;
  const JoinTo to{{m.dk, m.dv}, {m.sdk, m.sdv}, m.kv_heads, m.kv_len, 2};
  hipLaunchKernelGGL((masked_sum_kernel<T, D>), dim3(slices, m.batch * m.kv_heads * pk.deal.n_tiles, 2), block, 0, stream, pk, to);
  return hipGetLastError();
}
template <typename T, int D> hipError_t launch_td(const Masked& m, const Plan& pq, const Plan& pk, hipStream_t stream) {
  switch ((m.cap > 0.f ? CAP : 0) | (m.slopes ? BIAS : 0)) {
    case 0: return launch_mod<T, D, 0>(m, pq, pk, stream);
    case CAP: return launch_mod<T, D, CAP>(m, pq, pk, stream);
    case BIAS: return launch_mod<T, D, BIAS>(m, pq, pk, stream);
    default: return launch_mod<T, D, CAP | BIAS>(m, pq, pk, stream);
  }
}

size_t stat_bytes(const Masked& m) { return (2 * (size_t)m.batch * m.heads * m.q_len * sizeof(float) + 255) & ~(size_t)255; }

void places_in(const Masked& m, Plan* pq, Plan* pk) {          // the plans, with their places in the workspace
  *pq = plan_q(m);
  *pk = plan_kv(m);
  pq->stat = pk->stat = static_cast<float*>(m.workspace);
  pq->part = pk->part = reinterpret_cast<float*>(static_cast<unsigned char*>(m.workspace) + stat_bytes(m));
}

}  // namespace

// The fp32 kernels are compiled by themselves, from this file with PISA_MASKED_F32 set (build.py).
#ifdef PISA_MASKED_F32
hipError_t launch_masked_backward_f32(const Masked& m, hipStream_t stream) {
  Plan pq, pk;
  places_in(m, &pq, &pk);
  return m.d == 64 ? launch_td<float, 64>(m, pq, pk, stream) : launch_td<float, 128>(m, pq, pk, stream);
}
#else
size_t masked_backward_workspace_bytes(const Masked& m) {
  return stat_bytes(m) + part_floats(m, plan_q(m), plan_kv(m)) * sizeof(float);
}

hipError_t launch_masked_backward(const Masked& m, hipStream_t stream) {
  if (m.dtype == PISA_FP32) return launch_masked_backward_f32(m, stream);
  Plan pq, pk;
  places_in(m, &pq, &pk);
  return m.d == 64 ? launch_td<__bf16, 64>(m, pq, pk, stream) : launch_td<__bf16, 128>(m, pq, pk, stream);
}
#endif

}  // namespace pisa

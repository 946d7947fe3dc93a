// Masked attention, forward: one pass over the keys that a row sees, with a running maximum and sum.
//
// A workgroup has 128 query rows, a wave 32 of them; all products are transposed, so a lane holds one query row:
//     S^T (keys x rows) = K (keys x channels) Q^T,    O^T (channels x rows) += V^T (channels x keys) P^T
// and a row's mask, an interval of keys, is two registers of its lane.  Key tiles of 64 rows go through LDS by DMA, two stages
// each for K and V, one barrier a tile: behind it the loads of K(t+2) and V(t+1) go out, then the softmax of tile t,
// O^T += V(t)^T P(t)^T and S^T(t+1).  The walk goes over the tiles that some row of the workgroup sees; a wave leaves out
// those that none of its rows sees, and compares key numbers only in those that some of them see in part.
//
// Bound (bf16, 128 channels) by the turns that products, softmax and barriers take: no unit is full.  Causal, 12 heads of 8 192,
// 225 us: matrix cores 59 % busy, LDS 30 % (each matrix instruction takes a 1 KB operand from there); 24 heads of 4 608 tokens
// without a mask 250-263 us by card, 1 000-1 040 TFLOP/s.  32 rows a wave leave room for two waves on a SIMD, of which one is in its softmax while
// the other multiplies.  64 channels with capped and biased scores are bound by vector instructions (2 x 12 heads of 2 777, 70 us:
// matrix cores 18 %), fp32 by its matrix instruction (8 heads of 4 500, causal, 420 us, 72 % busy).
#include <algorithm>

#include "masked.h"
#include "tile.h"

namespace pisa {

using namespace tile;

namespace {

constexpr int kQRows = 128;
constexpr int CAP = 1, BIAS = 2;         // bits of MOD: scores capped, biased by distance

struct Plan {
  Deal deal;           // of tiles of 128 rows; parts: workgroups that share a tile's keys
  float* part_o;       // parts > 1: [head][tile][part][128][d] sums of weighted values, before division
  float* part_ml;      // [head][tile][part][2][128] maximum and sum of weights
};

template <typename T, int D> struct Row {        // what a lane holds of its query row
  f32x16 o[Geo<T, D>::NDT];
  float m, l;          // running maximum; this lane's share of the sum (keys with its h)
};

// The maximum takes in t (this lane's largest score); l and o are rescaled if some lane's moved.
template <typename T, int D> __device__ __forceinline__ void raise_max(Row<T, D>& st, float t) {
  t = fmaxf(t, __shfl_xor(t, 32));
  const float m = fmaxf(st.m, t);
  if (__any(m != st.m)) {
    const float f = st.m == -INFINITY ? 0.f : exp_of<T>(st.m - m);
    st.l *= f;
#pragma unroll
    for (int dt = 0; dt < Geo<T, D>::NDT; ++dt) st.o[dt] *= f;
    st.m = m;
  }
}

// What a wave's scores are made of: raw products times c, or their capped form, less slope times the distance.  The log2 domain
// in bf16.
template <typename T, int MOD> struct Score {
  float c, to_cap, cap, slope, near_limit;
  bool direct;
  Near near;             // in raw products, if direct
  __device__ __forceinline__ Score(const Masked& p, int head) : near(0.f) {
    const float unit = sizeof(T) == 2 ? kLog2e : 1.f;
    c = MOD & CAP ? 1.f : p.scale * unit;
    to_cap = MOD & CAP ? p.scale / p.cap : 0.f;
    cap = p.cap * unit;
    slope = MOD & BIAS ? p.slopes[head] * unit : 0.f;
    direct = (MOD & CAP) && Near::all_direct(cap, to_cap);
    near_limit = MOD & CAP ? (kNear / to_cap) * (kNear / to_cap) : 0.f;
    if (direct) {
      near = Near(cap);
      near.rescale(to_cap);
    }
  }
};

// Weights of 32 keys against the maximum as it stands, and their sum.  ahead: the row's position, counted from this lane's
// first key.  NEAR: s holds raw products, taken to be below the cap: the last step of their polynomial takes off the maximum,
// and their largest square, by which the caller sees whether they were, goes to top.
template <typename T, int MOD, bool NEAR>
__device__ __forceinline__ float weigh(const Score<T, MOD>& sc, const f32x16& s, float c, float slope, float minus_m, float ahead,
                                       Weights<T>& w, float& top) {
  float a = 0.f, b = 0.f;
#pragma unroll
  for (int r = 0; r < 16; r += 2) {
    float x[2], u[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int key = ((r + e) / 4) * 8 + (r + e) % 4;
      const float m = MOD & BIAS ? fmaf(-slope, fabsf(ahead - (float)key), minus_m) : minus_m;
      u[e] = s[r + e] * s[r + e];
      x[e] = exp_diff<T>(s[r + e], NEAR ? sc.near.of(u[e]) : c, m);
    }
    if (NEAR) top = fmaxf(fmaxf(u[0], u[1]), top);
    w.set(r, x[0], x[1]);
    if (r & 2) b += x[0] + x[1];
    else a += x[0] + x[1];
  }
  return a + b;
}

// The maximum is taken anew only where a lane's sum of weights against the old one reaches this (and on a wave's first tile, whose
// old maximum is -inf): fp32 and bf16 share their exponents, so a stale maximum costs no digits.  What it costs is range: weighted
// values are summed up to twice this factor (a row has two lanes), so values of 2^102 and less are safe whatever the scores.
constexpr float kStaleLimit = 0x1p24f;

template <typename T, int D, int MOD>
__global__ __launch_bounds__(256, sizeof(T) == 2 || D == 64 ? 2 : 1) void masked_fwd_kernel(Masked p, Plan plan) {
  using G = Geo<T, D>;
  constexpr int TILEB = G::TILEB, NDT = G::NDT;
  __shared__ __attribute__((aligned(1024))) unsigned char stage[4 * TILEB];      // K0 | K1 | V0 | V1
  __shared__ int span_s[4][4];
  __shared__ unsigned bad[2];

  __shared__ int32_t docs_s[kDocsInLds + 1];
  __shared__ int size_s[kRankedTiles + 1];

  const Share share = share_of(plan.deal);
  if (share.head < 0) return;
  const int bh = share.head, b = bh / p.heads, head = bh % p.heads;
  const int32_t* offs = borders_of(p, b, docs_s);
  const int qt = tile_of_rank<false>(p, offs, b, share.rank, plan.deal.n_tiles, size_s);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lam = lane & 31, h = lane >> 5;

  const int row = qt * kQRows + 32 * wave + lam;
  Interval iv{0, 0};
  if (row < p.q_len) iv = keys_of_row(p, offs, b, row);
  const bool sees = iv.lo < iv.hi;
  const Span ws = span_of_wave(iv);
  if (lane == 0) {
    span_s[wave][0] = ws.lo;
    span_s[wave][1] = ws.hi;
    span_s[wave][2] = ws.full_lo;
    span_s[wave][3] = ws.full_hi;
  }
  if (tid < 2) bad[tid] = 0u;

  const unsigned char* kg = p.k + b * p.sk.batch + (head / p.group) * p.sk.head;
  const unsigned char* vg = p.v + b * p.sv.batch + (head / p.group) * p.sv.head;
  const unsigned lds = (unsigned)(unsigned long long)(LDS_PTR(unsigned char)) & stage[0];
  Loader<T, D> lk, lv;
  lk.init(wave, lane, (unsigned)p.sk.token);
  lv.init(wave, lane, (unsigned)p.sv.token);
  Reader<T, D> rd;
  rd.init(lane, lds);

  u32x4 q[G::STEPS];                             // rows that see nothing take part as rows of zeros
  {
    const unsigned char* src = p.q + b * p.sq.batch + head * p.sq.head + (long long)row * p.sq.token;
#pragma unroll
    for (int s = 0; s < G::STEPS; ++s) {
      q[s] = u32x4{0, 0, 0, 0};
      if (sees) q[s] = *reinterpret_cast<const u32x4*>(src + 32 * s + 16 * h);
    }
  }
  const Score<T, MOD> sc(p, head);
  const int pos = row + p.kv_len - p.q_len;

  Row<T, D> st;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) st.o[dt] = (f32x16){0};
  st.m = -INFINITY;
  st.l = 0.f;

  __syncthreads();
  Span gs{span_s[0][0], span_s[0][1], span_s[0][2], span_s[0][3]};
#pragma unroll
  for (int w = 1; w < 4; ++w) gs = join(gs, Span{span_s[w][0], span_s[w][1], span_s[w][2], span_s[w][3]});
  gs = Span{__builtin_amdgcn_readfirstlane(gs.lo), __builtin_amdgcn_readfirstlane(gs.hi), __builtin_amdgcn_readfirstlane(gs.full_lo),
            __builtin_amdgcn_readfirstlane(gs.full_hi)};
  int t_begin = 0, t_end = 0;
  if (gs.lo < gs.hi) {
    t_begin = gs.lo / kRows;
    t_end = (gs.hi + kRows - 1) / kRows;
  }
  if (plan.deal.n_parts > 1) {
    const int n = t_end - t_begin, first = t_begin;
    t_begin = first + (int)((long long)n * share.part / plan.deal.n_parts);
    t_end = first + (int)((long long)n * (share.part + 1) / plan.deal.n_parts);
  }

  // The walk: ascending; where scores fall with the distance, from the rows' own tile down and then up from it, so that the
  // running maximum is met at once (a rising one is taken anew all the time: 24 / 8 heads of 500 rows, 9 001 keys, 110 us).
  const int n_tiles = t_end - t_begin;
  int start = t_begin, down = 0;
  if ((MOD & BIAS) && n_tiles > 0) {
    start = min(max((min(qt * kQRows + kQRows, p.q_len) - 1 + p.kv_len - p.q_len) / kRows, t_begin), t_end - 1);
    down = start - t_begin + 1;
  }
  auto tile_at = [&](int i) INLINE { return !(MOD & BIAS) ? t_begin + i : i < down ? start - i : t_begin + i; };

  auto load_k = [&](int t, int stage_at) INLINE {
    lk.load(wave, lane, kg + (long long)t * kRows * p.sk.token, p.kv_len - t * kRows, lds + stage_at * TILEB);
  };
  auto load_v = [&](int t, int stage_at) INLINE {
    lv.load(wave, lane, vg + (long long)t * kRows * p.sv.token, p.kv_len - t * kRows, lds + (2 + stage_at) * TILEB);
  };
  f32x16 s0, s1;                                 // S^T of the tile at hand: keys 0..31, 32..63
  auto scores = [&](int t, unsigned off) INLINE {
    if (!touches(ws, t * kRows, kRows)) return;
    s0 = rows_times<T, D, 0>(rd, off, q);
    s1 = rows_times<T, D, 32>(rd, off, q);
  };

  if (n_tiles > 0) {
    load_k(tile_at(0), 0);
    wait_loads();
    __syncthreads();
    if (n_tiles > 1) load_k(tile_at(1), 1);
    load_v(tile_at(0), 0);
    scores(tile_at(0), 0);
  }
  auto trip = [&](int i, auto parity) INLINE {
    const int par = parity, t = tile_at(i);
    const unsigned v_off = (2 + par) * TILEB;
    wait_loads();
    __syncthreads();
    if (i + 2 < n_tiles) load_k(tile_at(i + 2), par);
    if (i + 1 < n_tiles) load_v(tile_at(i + 1), par ^ 1);
    unsigned bad0 = 0u, bad1 = 0u;
    if (!covers(gs, t * kRows, kRows)) {         // seen in part by some row of the workgroup
      clean_tile<T, D>((LDS_PTR(unsigned char))&stage[0] + v_off, (LDS_PTR(unsigned))&bad[0], tid);
      __syncthreads();
      bad0 = __builtin_amdgcn_readfirstlane(bad[0]);
      bad1 = __builtin_amdgcn_readfirstlane(bad[1]);
      if (bad0 | bad1) {
        __syncthreads();
        if (tid < 2) bad[tid] = 0u;
      }
    }
    if (touches(ws, t * kRows, kRows)) {
      const float ahead = MOD & BIAS ? (float)(pos - t * kRows - 4 * h) : 0.f;
      const bool whole = covers(ws, t * kRows, kRows);
      const bool near = sizeof(T) == 2 && (MOD & CAP) && whole && sc.direct && i > 0;
      bool far = true;                           // this lane's scores are to be capped as they stand
      Weights<T> w0, w1;
      float sum = INFINITY, top = 0.f;           // the first tile has no maximum to be weighed against
      if (near) {
        sum = weigh<T, MOD, true>(sc, s0, 1.f, sc.slope, -st.m, ahead, w0, top);
        sum += weigh<T, MOD, true>(sc, s1, 1.f, sc.slope, -st.m, ahead - 32.f, w1, top);
        far = !(top <= sc.near_limit);
      }
      // Lane by lane, so that what a row gives does not hang on what its neighbours hold.  (The hint keeps this out of the way of
      // capped tiles: 24 heads of 4 608 tokens, capped and biased, 350 us without it, 324 with.)
      if (__builtin_expect(far, !(MOD & CAP))) {
        if (MOD & CAP) {
          cap_scores<T>(s0, sc.to_cap, sc.cap);
          cap_scores<T>(s1, sc.to_cap, sc.cap);
        }
        if (!whole) {
          const unsigned n = (unsigned)(iv.hi - iv.lo);
          const int at = t * kRows + 4 * h - iv.lo;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = (r / 4) * 8 + r % 4;
            if ((unsigned)(at + key) >= n) s0[r] = -INFINITY;
            if ((unsigned)(at + key + 32) >= n) s1[r] = -INFINITY;
          }
        }
        if (i > 0) {
          sum = weigh<T, MOD, false>(sc, s0, sc.c, sc.slope, -st.m, ahead, w0, top);
          sum += weigh<T, MOD, false>(sc, s1, sc.c, sc.slope, -st.m, ahead - 32.f, w1, top);
        }
      }
      if (__builtin_expect(__any(!(st.l + sum < kStaleLimit)), 0)) {
        // Row by row.  The scores are rounded as the maximum is taken of them: the largest key has weight 1, whatever its
        // size.  Where the sum was made by earlier tiles, it is what the maximum is raised by.
        bool again = !(st.l + sum < kStaleLimit);
        again |= (bool)__shfl_xor((int)again, 32);
        float peak = -INFINITY;
        if (again) {
          if (!far) {
            cap_scores<T>(s0, sc.to_cap, sc.cap);
            cap_scores<T>(s1, sc.to_cap, sc.cap);
          }
          {
#pragma clang fp contract(off)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float key = (float)((r / 4) * 8 + r % 4);
              s0[r] *= sc.c;
              s1[r] *= sc.c;
              if (MOD & BIAS) {
                s0[r] -= sc.slope * fabsf(ahead - key);
                s1[r] -= sc.slope * fabsf(ahead - 32.f - key);
              }
            }
          }
          peak = fmaxf(fmaxf(max_of(s0), max_of(s1)), st.m + log_of<T>(st.l));
        }
        raise_max<T, D>(st, peak);
        if (again) {
          const float nm = st.m == -INFINITY ? 0.f : -st.m;
          sum = weigh<T, MOD, false>(sc, s0, 1.f, 0.f, nm, ahead, w0, top);
          sum += weigh<T, MOD, false>(sc, s1, 1.f, 0.f, nm, ahead - 32.f, w1, top);
        }
      }
      st.l += sum;
      cols_times<T, D, 0>(rd, v_off, w0, st.o);
      cols_times<T, D, 32>(rd, v_off, w1, st.o);
      while (__builtin_expect((bad0 | bad1) != 0u, 0)) {      // values of inf or NaN, for the rows that see them
        const int r = bad0 ? __builtin_ctz(bad0) : 32 + __builtin_ctz(bad1);
        if (bad0) bad0 &= bad0 - 1u;
        else bad1 &= bad1 - 1u;
        const int key = t * kRows + r;
        if (key >= p.kv_len) break;
        const T* src = reinterpret_cast<const T*>(vg + (long long)key * p.sv.token);
        const bool mine = key >= iv.lo && key < iv.hi;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = (float)src[32 * dt + (e / 4) * 8 + 4 * h + e % 4];
            if (mine && !(fabsf(x) < INFINITY)) st.o[dt][e] += x;
          }
      }
    }
    if (i + 1 < n_tiles) scores(tile_at(i + 1), (par ^ 1) * TILEB);
  };
  walk_stages<T>(0, n_tiles, trip);

  st.l += __shfl_xor(st.l, 32);
  if (plan.deal.n_parts > 1) {
    const size_t item = ((size_t)bh * plan.deal.n_tiles + qt) * plan.deal.n_parts + share.part;
    float* po = plan.part_o + ((size_t)item * kQRows + 32 * wave + lam) * D;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 w = {st.o[dt][4 * g], st.o[dt][4 * g + 1], st.o[dt][4 * g + 2], st.o[dt][4 * g + 3]};
        *reinterpret_cast<f32x4*>(po + 32 * dt + 8 * g + 4 * h) = w;
      }
    if (h == 0) {
      plan.part_ml[((size_t)item * 2 + 0) * kQRows + 32 * wave + lam] = st.m;
      plan.part_ml[((size_t)item * 2 + 1) * kQRows + 32 * wave + lam] = sees ? st.l : 0.f;
    }
    return;
  }
  if (row < p.q_len) {
    const bool some = sees && st.l != 0.f;       // false: no key, or none with a score above -inf
    const float inv = 1.f / st.l;
    unsigned char* dst = p.out + b * p.so.batch + head * p.so.head + (long long)row * p.so.token;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = some ? st.o[dt][4 * g + e] * inv : 0.f;
        const int ch = 32 * dt + 8 * g + 4 * h;
        if constexpr (sizeof(T) == 2)
          *reinterpret_cast<u32x2*>(dst + 2 * ch) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
        else
          *reinterpret_cast<f32x4*>(dst + 4 * ch) = x;
      }
    if (p.lse && h == 0) p.lse[(size_t)bh * p.q_len + row] = some ? log_sum<T>(st.m, st.l) : -INFINITY;
  }
}

// Joins the parts of 128 rows: a thread has four channels of a row.  Workgroup: (batch, head, tile) x slices of its rows.
template <typename T, int D> __global__ __launch_bounds__(256) void masked_join_kernel(Masked p, Plan plan) {
  constexpr int PER_ROW = D / 4, ROWS = 256 / PER_ROW;
  const int unit = blockIdx.y, tid = threadIdx.x, n_parts = plan.deal.n_parts;
  const int bh = unit / plan.deal.n_tiles, b = bh / p.heads, head = bh % p.heads, qt = unit % plan.deal.n_tiles;
  const int r = blockIdx.x * ROWS + tid / PER_ROW, ch = 4 * (tid % PER_ROW), row = qt * kQRows + r;
  if (row >= p.q_len) return;
  const size_t item = (size_t)unit * n_parts;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < n_parts; i0 += 8) {      // eight parts under way at a time
    float mi[8], li[8];
    f32x4 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i0 + u < n_parts) {
        mi[u] = plan.part_ml[((item + i0 + u) * 2) * kQRows + r];
        li[u] = plan.part_ml[((item + i0 + u) * 2 + 1) * kQRows + r];
        x[u] = *reinterpret_cast<const f32x4*>(plan.part_o + ((item + i0 + u) * kQRows + r) * D + ch);
      }
    float top = m;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i0 + u < n_parts) top = fmaxf(top, mi[u] + log_of<T>(li[u]));      // a maximum can be stale by as much as its sum has grown
    if (l != 0.f) {
      const float f = exp_of<T>(m - top);
      l *= f;
      o *= f;
    }
    m = top;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i0 + u < n_parts && li[u] != 0.f) {    // 0: no key of the row in this part
        const float f = exp_of<T>(mi[u] - m);
        l += li[u] * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += x[u][e] * f;
      }
  }
  const bool sees = l != 0.f;
  const float inv = sees ? 1.f / l : 0.f;
  unsigned char* dst = p.out + b * p.so.batch + head * p.so.head + (long long)row * p.so.token;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<u32x2*>(dst + 2 * ch) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
  else
    *reinterpret_cast<f32x4*>(dst + 4 * ch) = f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  if (p.lse && ch == 0) p.lse[(size_t)bh * p.q_len + row] = sees ? log_sum<T>(m, l) : -INFINITY;
}

// Workgroups that share a tile's keys, where the tiles alone leave places on the card idle (64 an XCD in bf16, 32 in fp32) and
// there are keys enough to share.
int parts_of(const Masked& m) {
  const long long units = (long long)m.batch * m.heads * ((m.q_len + kQRows - 1) / kQRows), u = (units + 7) / 8;
  const long long tiles = (m.kv_len + kRows - 1) / kRows;
  const bool triangle = m.causal && 2LL * m.q_len > m.kv_len;        // tiles of very different size
  long long parts = 1;
  if (m.dtype == PISA_BF16) {
    // Equal tiles: one round of workgroups, never a few more (24 heads of 500 rows, 9 001 keys, five parts 99 us, six 134).
    // Those of a triangle are half as long on average and fill places as they end (12 heads of 2 048 two parts 48, three 42,
    // six 53; 24 of 2 000 one 63, two 56; 13 of 6 000 one 174, two 164).
    parts = triangle ? (256 + 3 * u - 1) / (3 * u) : 64 / u;
    parts = std::min(parts, tiles / 4);
  } else if (triangle) {
    // fp32 products take so long that three workgroups a compute unit pay (8 heads of 4 500: one part 850, two 574, three
    // 561, six 586), two at 64 channels.
    // Two tiles or more to a part; one where all parts still find a compute unit each (2 heads of 300 40 -> 25).
    parts = std::max(std::min(((m.d == 64 ? 64 : 96) + u - 1) / u, tiles / 2), std::min(32 / u, tiles));
  } else {
    // whole rounds of the 32 compute units of an XCD, and about a tile's time for a part's own sums and its part in the joining;
    // 512 parts an XCD at most, past which what a last round leaves idle is little
    long long best = 1LL << 60;
    for (long long n = 1; n <= 16 && (n == 1 || (n <= tiles / 2 && n * u <= 512)); ++n) {
      const long long rounds = (u * n + 31) / 32, cost = rounds * (tiles * 64 / n + 64);
      if (cost < best) {
        best = cost;
        parts = n;
      }
    }
  }
  return parts < 1 ? 1 : (int)parts;
}
size_t items_of(const Plan& pl, const Masked& m) { return (size_t)m.batch * m.heads * pl.deal.n_tiles * pl.deal.n_parts; }
Plan plan_of(const Masked& m) {
  Plan pl{};
  pl.deal = deal_of(m.batch * m.heads, (m.q_len + kQRows - 1) / kQRows, parts_of(m), m.dtype == PISA_BF16 ? 64 : 32);
  return pl;
}
Plan plan_in(const Masked& m) {                  // with its places in the workspace
  Plan pl = plan_of(m);
  if (pl.deal.n_parts > 1) {
    pl.part_o = static_cast<float*>(m.workspace);
    pl.part_ml = pl.part_o + items_of(pl, m) * kQRows * m.d;
  }
  return pl;
}

template <typename T, int D> hipError_t launch_td(const Masked& m, const Plan& pl, hipStream_t stream) {
  const dim3 grid(8 * pl.deal.per_xcd), block(256);
  switch ((m.cap > 0.f ? CAP : 0) | (m.slopes ? BIAS : 0)) {
    case 0: hipLaunchKernelGGL((masked_fwd_kernel<T, D, 0>), grid, block, 0, stream, m, pl); break;
    case CAP: hipLaunchKernelGGL((masked_fwd_kernel<T, D, CAP>), grid, block, 0, stream, m, pl); break;
    case BIAS: hipLaunchKernelGGL((masked_fwd_kernel<T, D, BIAS>), grid, block, 0, stream, m, pl); break;
    default: hipLaunchKernelGGL((masked_fwd_kernel<T, D, CAP | BIAS>), grid, block, 0, stream, m, pl); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || pl.deal.n_parts == 1) return e;
  hipLaunchKernelGGL((masked_join_kernel<T, D>), dim3(kQRows / (256 / (D / 4)), m.batch * m.heads * pl.deal.n_tiles), block, 0, stream, m, pl);
  return hipGetLastError();
}

}  // namespace

// The fp32 kernels are compiled by themselves, from this file with PISA_MASKED_F32 set (build.py).
#ifdef PISA_MASKED_F32
hipError_t launch_masked_attention_f32(const Masked& m, hipStream_t stream) {
  const Plan pl = plan_in(m);
  return m.d == 64 ? launch_td<float, 64>(m, pl, stream) : launch_td<float, 128>(m, pl, stream);
}
#else
size_t masked_workspace_bytes(const Masked& m) {
  const Plan pl = plan_of(m);
  return pl.deal.n_parts == 1 ? 0 : items_of(pl, m) * kQRows * (m.d + 2) * sizeof(float);
}

hipError_t launch_masked_attention(const Masked& m, hipStream_t stream) {
  if (m.dtype == PISA_FP32) return launch_masked_attention_f32(m, stream);
  const Plan pl = plan_in(m);
  return m.d == 64 ? launch_td<__bf16, 64>(m, pl, stream) : launch_td<__bf16, 128>(m, pl, stream);
}
#endif

}  // namespace pisa

// Masked attention, backward: dq from a walk over the keys of 128 rows, dk and dv from a walk over the rows of 128 keys.
//
// Both walks make the scores again from q and k and the weights from the log-sum-exp that the forward pass left, so nothing
// of size q_len x kv_len is stored; seven products instead of five, and in exchange every sum is made by one workgroup in a
// fixed order, without atomics.  As in the forward pass all products are transposed:
//     dq walk (a lane holds one query row):  S^T = K Q^T,  dP^T = V dO^T,  dQ^T += K^T dS^T
//     dk, dv walk (a lane holds one key):    S = Q K^T,    dP = dO V^T,    dV^T += dO^T P,  dK^T += Q^T dS
// so that P and dS leave the first products in the lanes in which the second ones take them.  The dk, dv walk goes over the
// rows of all query heads that share the key head.
#include "masked.h"
#include "tile.h"

namespace pisa {

using namespace tile;

namespace {

constexpr int kOwn = 128;                // rows (keys) of a workgroup, 32 to a wave
constexpr int CAP = 1, BIAS = 2;         // bits of MOD

struct Plan {
  int n_tiles;         // tiles of 128 rows (dq) or keys (dk, dv) to a head
  int n_parts;         // dk, dv: workgroups that share the rows of a key tile
  int total, per_xcd;
  float* delta;        // [batch][heads][q_len]
  float* part;         // n_parts > 1: [item][dk, dv][128][d]
};

// A score and what its gradient is multiplied by.
template <typename T, int MOD> struct Scorer {
  float c, to_cap, cap, slope;
  __device__ inline Scorer(const Masked& p, int head) {
    const float u = sizeof(T) == 2 ? kLog2e : 1.f;
    c = MOD ? 1.f : p.scale * u;
    to_cap = MOD & CAP ? p.scale / p.cap : p.scale * u;
    cap = p.cap * u;
    slope = MOD & BIAS ? p.slopes[head] * u : 0.f;
  }
  // the weight exp(z - lse) of the raw product s; `far` = |pos - key|; *gain = dz/ds
  __device__ inline float weight(float s, float minus_lse, float far, float* gain) const {
    *gain = 1.f;
    if (!MOD) return exp_diff<T>(s, c, minus_lse);
    float z = s * to_cap;
    if (MOD & CAP) {
      const float t = tanh_of<T>(z);
      *gain = (1.f - t) * (1.f + t);
      z = cap * t;
    }
    if (MOD & BIAS) z = fmaf(-slope, far, z);
    return exp_diff<T>(z, 1.f, minus_lse);
  }
};
template <typename T> __device__ inline float in_domain(float lse) { return sizeof(T) == 2 ? lse * kLog2e : lse; }

__device__ inline Span span_of_group(const Span& ws, int (*span_s)[4], int wave, int lane) {
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

template <typename T> __device__ inline float dot16(u32x4 a, u32x4 b) {      // of 16 bytes each
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

// The lane's row of sums, times f; zeros unless `some` (the sums of a row that has none can hold anything).
template <typename T, int D>
__device__ inline void store_row(unsigned char* dst, const f32x16 (&acc)[Geo<T, D>::NDT], float f, bool some, int h) {
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
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void masked_dq_kernel(Masked p, Plan plan) {
  using G = Geo<T, D>;
  constexpr int TILEB = G::TILEB, NDT = G::NDT;
  __shared__ __attribute__((aligned(1024))) unsigned char stage[4 * TILEB];      // K0 | V0 | K1 | V1
  __shared__ int span_s[4][4];
  __shared__ unsigned bad[2];

  const int item = item_of_xcd(plan.per_xcd);
  if ((int)(blockIdx.x / 8) >= plan.per_xcd || item >= plan.total) return;
  const int bh = item / plan.n_tiles, b = bh / p.heads, head = bh % p.heads;
  const int qt = p.causal ? plan.n_tiles - 1 - item % plan.n_tiles : item % plan.n_tiles;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lam = lane & 31, h = lane >> 5;
  const int row = qt * kOwn + 32 * wave + lam;
  Interval iv{0, 0};
  if (row < p.q_len) iv = keys_of_row(p, b, row);
  const bool sees = iv.lo < iv.hi;
  const Span ws = span_of_wave(iv);
  if (tid < 2) bad[tid] = 0u;
  const Span gs = span_of_group(ws, span_s, wave, lane);

  const unsigned char* kg = p.k + b * p.sk.batch + (head / p.group) * p.sk.head;
  const unsigned char* vg = p.v + b * p.sv.batch + (head / p.group) * p.sv.head;
  const unsigned lds = (unsigned)(unsigned long long)(LDS_PTR(unsigned char)) & stage[0];
  Loader<T, D> lk, lv;
  lk.init(wave, lane, (unsigned)p.sk.token);
  lv.init(wave, lane, (unsigned)p.sv.token);
  Reader<T, D> rd;
  rd.init(lane, lds);
  auto load = [&](int t, int par) {
    lk.load(wave, lane, kg + (long long)t * kRows * p.sk.token, p.kv_len - t * kRows, lds + 2 * par * TILEB);
    lv.load(wave, lane, vg + (long long)t * kRows * p.sv.token, p.kv_len - t * kRows, lds + (2 * par + 1) * TILEB);
  };
  int t_begin = 0, t_end = 0;
  if (gs.lo < gs.hi) {
    t_begin = gs.lo / kRows;
    t_end = (gs.hi + kRows - 1) / kRows;
    load(t_begin, 0);
  }

  u32x4 q[G::STEPS], g[G::STEPS];                // the lane's rows of q and dout; zeros where the row sees nothing
  float delta = 0.f, minus_lse = 0.f;
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
    if (sees) minus_lse = -in_domain<T>(p.lse[(size_t)bh * p.q_len + row]);
    if (row < p.q_len && h == 0) plan.delta[(size_t)bh * p.q_len + row] = delta;
  }
  const Scorer<T, MOD> sc(p, head);
  const int pos = row + p.kv_len - p.q_len;

  f32x16 acc[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) acc[dt] = (f32x16){0};

  for (int t = t_begin; t < t_end; ++t) {
    const int par = (t - t_begin) & 1;
    const unsigned k_off = 2 * par * TILEB, v_off = k_off + TILEB;
    wait_loads();
    __syncthreads();
    if (t + 1 < t_end) load(t + 1, par ^ 1);
    if (!covers(gs, t * kRows, kRows)) {         // the product with K contracts over keys that not every row sees
      clean_tile<T, D>((LDS_PTR(unsigned char))&stage[0] + k_off, (LDS_PTR(unsigned))&bad[0], tid);
      __syncthreads();
    }
    if (!touches(ws, t * kRows, kRows)) continue;
    const bool part = !covers(ws, t * kRows, kRows);
    auto half = [&](auto row0_tag) {
      constexpr int ROW0 = decltype(row0_tag)::value;
      const f32x16 s = rows_times<T, D, ROW0>(rd, k_off, q);
      const f32x16 dp = rows_times<T, D, ROW0>(rd, v_off, g);
      Weights<T> w;
      const unsigned n = (unsigned)(iv.hi - iv.lo);
      const int key0 = t * kRows + ROW0 + 4 * h;
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        float x[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int key = key0 + ((r + u) / 4) * 8 + (r + u) % 4;
          float gain;
          const float wt = sc.weight(s[r + u], minus_lse, fabsf((float)(pos - key)), &gain);
          x[u] = wt * (dp[r + u] - delta);
          if (MOD & CAP) x[u] *= gain;
          if (part && (unsigned)(key - iv.lo) >= n) x[u] = 0.f;
        }
        w.set(r, x[0], x[1]);
      }
      cols_times<T, D, ROW0>(rd, k_off, w, acc);
    };
    half(std::integral_constant<int, 0>{});
    half(std::integral_constant<int, 32>{});
  }
  if (row < p.q_len)
    store_row<T, D>(p.dq + b * p.sdq.batch + head * p.sdq.head + (long long)row * p.sdq.token, acc, p.scale, sees, h);
}

template <typename T, int D, int MOD>
__global__ __launch_bounds__(256, 1) void masked_dkv_kernel(Masked p, Plan plan) {
  using G = Geo<T, D>;
  constexpr int TILEB = G::TILEB, NDT = G::NDT;
  __shared__ __attribute__((aligned(1024))) unsigned char stage[4 * TILEB];      // Q0 | dO0 | Q1 | dO1
  __shared__ __attribute__((aligned(16))) float stat[2][2][kRows];               // [parity][-lse, delta][row]
  __shared__ int span_s[4][4];
  __shared__ unsigned bad[2];

  const int item = item_of_xcd(plan.per_xcd);
  if ((int)(blockIdx.x / 8) >= plan.per_xcd || item >= plan.total) return;
  const int part_no = item % plan.n_parts, unit = item / plan.n_parts;
  const int bk = unit / plan.n_tiles, b = bk / p.kv_heads, kv_head = bk % p.kv_heads;
  const int kt = unit % plan.n_tiles;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lam = lane & 31, h = lane >> 5;
  const int key = kt * kOwn + 32 * wave + lam;
  Interval iv{0, 0};
  if (key < p.kv_len) iv = rows_of_key(p, b, key);
  const bool seen = iv.lo < iv.hi;
  const Span ws = span_of_wave(iv);
  if (tid < 2) bad[tid] = 0u;
  const Span gs = span_of_group(ws, span_s, wave, lane);

  const unsigned lds = (unsigned)(unsigned long long)(LDS_PTR(unsigned char)) & stage[0];
  Loader<T, D> lq, lg;
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
  const int i_begin = (int)(steps * part_no / plan.n_parts), i_end = (int)(steps * (part_no + 1) / plan.n_parts);
  auto load = [&](int i, int par) {
    const int head = kv_head * p.group + i / n, t = t_begin + i % n;
    const int avail = p.q_len - t * kRows;
    lq.load(wave, lane, p.q + b * p.sq.batch + head * p.sq.head + (long long)t * kRows * p.sq.token, avail, lds + 2 * par * TILEB);
    lg.load(wave, lane, p.dout + b * p.sdo.batch + head * p.sdo.head + (long long)t * kRows * p.sdo.token, avail,
            lds + (2 * par + 1) * TILEB);
  };
  auto fetch_stat = [&](int i) -> float {        // threads 0..63: -lse, 64..127: delta
    const int head = kv_head * p.group + i / n, t = t_begin + i % n;
    const size_t at = ((size_t)b * p.heads + head) * p.q_len + min(t * kRows + (tid & 63), p.q_len - 1);
    return wave == 0 ? -in_domain<T>(p.lse[at]) : plan.delta[at];
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

  if (i_begin < i_end) {
    if (wave < 2) stat[0][wave][lane] = fetch_stat(i_begin);
    load(i_begin, 0);
  }
  const int shift = p.kv_len - p.q_len;
  for (int i = i_begin; i < i_end; ++i) {
    const int par = (i - i_begin) & 1;
    const unsigned q_off = 2 * par * TILEB, g_off = q_off + TILEB;
    const int t = t_begin + i % n;
    wait_loads();
    __syncthreads();
    if (i + 1 < i_end) {
      load(i + 1, par ^ 1);
      if (wave < 2) stat[par ^ 1][wave][lane] = fetch_stat(i + 1);
    }
    if (!covers(gs, t * kRows, kRows)) {         // both second products contract over rows that do not all see every key
      clean_tile<T, D>((LDS_PTR(unsigned char))&stage[0] + q_off, (LDS_PTR(unsigned))&bad[0], tid);
      clean_tile<T, D>((LDS_PTR(unsigned char))&stage[0] + g_off, (LDS_PTR(unsigned))&bad[0], tid);
      __syncthreads();
    }
    if (!touches(ws, t * kRows, kRows)) continue;
    const bool part = !covers(ws, t * kRows, kRows);
    const Scorer<T, MOD> sc(p, kv_head * p.group + i / n);
    auto half = [&](auto row0_tag) {
      constexpr int ROW0 = decltype(row0_tag)::value;
      const f32x16 s = rows_times<T, D, ROW0>(rd, q_off, k);
      const f32x16 dp = rows_times<T, D, ROW0>(rd, g_off, v);
      Weights<T> wp, wd;
      const unsigned count = (unsigned)(iv.hi - iv.lo);
      const int row0 = t * kRows + ROW0 + 4 * h;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 ml = *reinterpret_cast<LDS_PTR(const f32x4)>((LDS_PTR(const float))&stat[par][0][ROW0 + 8 * e + 4 * h]);
        const f32x4 de = *reinterpret_cast<LDS_PTR(const f32x4)>((LDS_PTR(const float))&stat[par][1][ROW0 + 8 * e + 4 * h]);
        float x[4], y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int r = 4 * e + u, row = row0 + 8 * e + u;
          float gain;
          x[u] = sc.weight(s[r], ml[u], fabsf((float)(row + shift - key)), &gain);
          y[u] = x[u] * (dp[r] - de[u]);
          if (MOD & CAP) y[u] *= gain;
          if (part) {
            x[u] = fmaf(0.f, de[u], x[u]);       // a row of dout that was cleaned of inf or NaN has a delta of NaN
            if ((unsigned)(row - iv.lo) >= count) x[u] = y[u] = 0.f;
          }
        }
        wp.set(4 * e, x[0], x[1]);
        wp.set(4 * e + 2, x[2], x[3]);
        wd.set(4 * e, y[0], y[1]);
        wd.set(4 * e + 2, y[2], y[3]);
      }
      cols_times<T, D, ROW0>(rd, g_off, wp, dv);
      cols_times<T, D, ROW0>(rd, q_off, wd, dk);
    };
    half(std::integral_constant<int, 0>{});
    half(std::integral_constant<int, 32>{});
  }

  if (plan.n_parts > 1) {
    unsigned char* dst = reinterpret_cast<unsigned char*>(plan.part + ((size_t)item * 2 * kOwn + 32 * wave + lam) * D);
    store_row<float, D>(dst, dk, p.scale, seen, h);
    store_row<float, D>(dst + (size_t)kOwn * D * sizeof(float), dv, 1.f, seen, h);
    return;
  }
  if (key < p.kv_len) {
    store_row<T, D>(p.dk + b * p.sdk.batch + kv_head * p.sdk.head + (long long)key * p.sdk.token, dk, p.scale, seen, h);
    store_row<T, D>(p.dv + b * p.sdv.batch + kv_head * p.sdv.head + (long long)key * p.sdv.token, dv, 1.f, seen, h);
  }
}

// Adds the parts of a key tile's dk and dv: a thread has four channels of one row of either.
template <typename T, int D> __global__ __launch_bounds__(256) void masked_dkv_join_kernel(Masked p, Plan plan) {
  constexpr int PER_ROW = D / 4, ROWS = 256 / PER_ROW;
  const int unit = blockIdx.y, tid = threadIdx.x, which = blockIdx.z;
  const int bk = unit / plan.n_tiles, b = bk / p.kv_heads, kv_head = bk % p.kv_heads;
  const int r = blockIdx.x * ROWS + tid / PER_ROW, ch = 4 * (tid % PER_ROW), key = unit % plan.n_tiles * kOwn + r;
  if (key >= p.kv_len) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < plan.n_parts; ++i)
    sum += *reinterpret_cast<const f32x4*>(plan.part + ((((size_t)unit * plan.n_parts + i) * 2 + which) * kOwn + r) * D + ch);
  const Strides& sd = which ? p.sdv : p.sdk;
  unsigned char* dst = (which ? p.dv : p.dk) + b * sd.batch + kv_head * sd.head + (long long)key * sd.token;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<u32x2*>(dst + 2 * ch) = u32x2{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
  else
    *reinterpret_cast<f32x4*>(dst + 4 * ch) = sum;
}

Plan plan_q(const Masked& m) {
  Plan pl{};
  pl.n_tiles = (m.q_len + kOwn - 1) / kOwn;
  pl.n_parts = 1;
  pl.total = m.batch * m.heads * pl.n_tiles;
  pl.per_xcd = (pl.total + 7) / 8;
  return pl;
}
Plan plan_kv(const Masked& m) {
  Plan pl{};
  pl.n_tiles = (m.kv_len + kOwn - 1) / kOwn;
  const long long units = (long long)m.batch * m.kv_heads * pl.n_tiles;
  if (units == 0) return pl;
  // Rows are shared out where the key tiles alone leave compute units idle.
  const long long steps = (long long)m.group * ((m.q_len + kRows - 1) / kRows);
  long long parts = units >= 256 ? 1 : 256 / units;
  parts = parts < steps / 4 ? parts : steps / 4;
  pl.n_parts = parts < 1 ? 1 : (int)parts;
  pl.total = (int)(units * pl.n_parts);
  pl.per_xcd = (pl.total + 7) / 8;
  return pl;
}

template <typename T, int D, int MOD> hipError_t launch_mod(const Masked& m, const Plan& pq, const Plan& pk, hipStream_t stream) {
  hipLaunchKernelGGL((masked_dq_kernel<T, D, MOD>), dim3(8 * pq.per_xcd), dim3(256), 0, stream, m, pq);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || pk.total == 0) return e;
  hipLaunchKernelGGL((masked_dkv_kernel<T, D, MOD>), dim3(8 * pk.per_xcd), dim3(256), 0, stream, m, pk);
  e = hipGetLastError();
  if (e != hipSuccess || pk.n_parts == 1) return e;
  hipLaunchKernelGGL((masked_dkv_join_kernel<T, D>), dim3(kOwn / (256 / (D / 4)), pk.total / pk.n_parts, 2), dim3(256), 0, stream, m, pk);
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

size_t delta_bytes(const Masked& m) { return ((size_t)m.batch * m.heads * m.q_len * sizeof(float) + 255) & ~(size_t)255; }

}  // namespace

size_t masked_backward_workspace_bytes(const Masked& m) {
  const Plan pk = plan_kv(m);
  return delta_bytes(m) + (pk.n_parts > 1 ? (size_t)pk.total * 2 * kOwn * m.d * sizeof(float) : 0);
}

hipError_t launch_masked_backward(const Masked& m, hipStream_t stream) {
  Plan pq = plan_q(m), pk = plan_kv(m);
  pq.delta = pk.delta = static_cast<float*>(m.workspace);
  pk.part = reinterpret_cast<float*>(static_cast<unsigned char*>(m.workspace) + delta_bytes(m));
  if (m.dtype == PISA_BF16) return m.d == 64 ? launch_td<__bf16, 64>(m, pq, pk, stream) : launch_td<__bf16, 128>(m, pq, pk, stream);
  return m.d == 64 ? launch_td<float, 64>(m, pq, pk, stream) : launch_td<float, 128>(m, pq, pk, stream);
}

}  // namespace pisa

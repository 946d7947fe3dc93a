// Attention of one new token per sequence over a paged cache, and the append that fills it.
//
// Bound by reading the cache (once for every 16 query heads that share a key head), so the work is cut by cached tokens,
// whatever sequence they belong to: the tiles of all (sequence, key head) units, laid one behind the other, are shared out
// evenly among a fixed number of workgroups, which find their range from the lengths on the device.  A workgroup walks its
// range unit by unit; units that it has not to itself leave (maximum, sum, weighted values) in the workspace, and a second
// launch joins them.
//
// A wave takes KT keys of a tile: K and V rows go to its own part of LDS by DMA, two stages, and it waits for its own loads
// alone (no barriers in the walk).  With v_mfma_f32_16x16x32_bf16 (fp32: 16x16x4) 16 query heads that share the key head are
// the columns of S^T = K Q^T and O^T = V^T P^T; register r of lane (j, g) holds key 4 g + r and column j, and that order of
// the keys serves the second product as it stands.
//
// Measured: 2 sequences of 200 000 tokens, 40 / 8 heads, 255 us (6.0 TB/s); 48 of up to 8 000, 32 / 8 heads, 164 us (5.2 TB/s: here a
// workgroup walks two or three units and fills its pipeline anew for each).
#include "paged.h"
#include "tile.h"

namespace pisa {

using namespace tile;

namespace {

constexpr int CAP = 1, BIAS = 2;
constexpr int kCols = 16;                        // query heads of a unit

template <typename T, int D> struct PGeo {
  static constexpr int KT = sizeof(T) == 2 ? 32 : 16;       // keys of a wave and tile
  static constexpr int ROWB = D * (int)sizeof(T);
  static constexpr int BYTES = KT * ROWB;                   // staged K (or V) of a wave
  static constexpr int NLD = BYTES / 1024;                  // loads of 1 KB
  static constexpr int CPR = ROWB / 16, RPL = 64 / CPR;
  static constexpr int NDT = D / 16;                        // 16-channel tiles
  static constexpr int WAVES = 4;
  static constexpr int THREADS = 64 * WAVES;
  static constexpr int TILE = WAVES * KT;                   // keys of a tile
  // workgroups: one or two fit a compute unit's LDS (two of two waves at 8 KB: 171 against 169 us for 48 sequences of up to 8 000)
  static constexpr int GROUPS = BYTES == 8192 ? 256 : 512;
  static constexpr int PER = THREADS / kCols;               // threads to a row where the waves' sums are joined
};

struct PPlan {
  int units;           // of a sequence: key heads x blocks of 16 query heads
  int blocks;          // of 16 query heads to a key head
  int solo;            // a workgroup to a (sequence, unit), nothing to join
  float* part_o;       // [workgroup][2][16][d] weighted values: of its first unit, of its last
  float* part_ml;      // [workgroup][2][2][16] maximum and sum
  int32_t* owners;     // [seq][unit][2] first and last workgroup; the first's slot is its second if the last has bit 30 set
};
constexpr int kSecondSlot = 1 << 30;

// What rows of masked keys are read from: weight 0 times a row of a foreign or unwritten page could be NaN.
__device__ const u32x4 zero_row[32] = {};

__device__ inline int length_of(const Paged& p, int s) {
  const long long most = (long long)p.max_pages * p.page_size;
  return (int)min((long long)max(p.lengths[s], 0), most);
}

// First tile of workgroup w's range: total * w / n (n workgroups take part).
__device__ inline long long first_tile(long long total, int n, int w) { return total * w / n; }

template <typename T> __device__ inline f32x4 mma16_step(u32x4 a, u32x4 b, f32x4 acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], acc, 0, 0, 0);
    return acc;
  }
}

// The waits of the walk, which the compiler cannot see: at most N of this wave's loads are still under way.
template <int N> __device__ inline void wait_all_but() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }
__device__ inline void dma_rows(unsigned lds, const unsigned char* src) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(src) : "memory", "m0");
}
__device__ inline void dma_word(unsigned lds, const int32_t* src) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds), "v"(src) : "memory", "m0");
}
__device__ inline const unsigned char* shfl_ptr(const unsigned char* p, int from) {
  const unsigned long long x = (unsigned long long)p;
  const unsigned lo = __shfl((int)(unsigned)x, from), hi = __shfl((int)(unsigned)(x >> 32), from);
  return (const unsigned char*)(((unsigned long long)hi << 32) | lo);
}

template <typename T, int D, int MOD>
__global__ __launch_bounds__(256, (PGeo<T, D>::GROUPS / 256)) void paged_kernel(Paged p, PPlan plan) {
  using P = PGeo<T, D>;
  constexpr int KT = P::KT, NKV = 2 * P::NLD;
  __shared__ __attribute__((aligned(1024))) unsigned char stage[P::WAVES][2][2][P::BYTES];    // [wave][parity][K, V]
  __shared__ __attribute__((aligned(16))) int32_t pages[P::WAVES][2][64];
  __shared__ long long scratch[P::WAVES];
  __shared__ float ml_s[P::WAVES][2][kCols];
  __shared__ long long found_s[2];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 15, g = lane >> 4;

  // ---- this workgroup's range of tiles, and the sequence it starts in ----
  // tiles up to and with sequence s0 + tid, from s0; *all: of the next THREADS sequences
  auto scan = [&](int s0, long long* all) {
    const int s = s0 + tid;
    long long incl = s < p.seqs ? (length_of(p, s) + P::TILE - 1) / P::TILE : 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const long long up = __shfl_up(incl, o);
      if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == 63) scratch[wave] = incl;
    __syncthreads();
    for (int w = 0; w < wave; ++w) incl += scratch[w];
    *all = 0;
#pragma unroll
    for (int w = 0; w < P::WAVES; ++w) *all += scratch[w];
    return incl;
  };
  long long x_begin = 0, x_end = 0, total = 0, seq_x = 0;
  int seq = 0, n_groups = 1;
  if (plan.solo) {
    seq = blockIdx.x / plan.units;
    const int unit = blockIdx.x % plan.units, tiles = (length_of(p, seq) + P::TILE - 1) / P::TILE;
    x_begin = (long long)unit * tiles;
    x_end = x_begin + tiles;
    if (tiles == 0) {
      const int kv_head = unit / plan.blocks, row = unit % plan.blocks * kCols + tid / P::PER;
      if (row >= p.group) return;
      const size_t head = (size_t)seq * p.heads + kv_head * p.group + row;
      for (int i = tid % P::PER; i < P::CPR; i += P::PER) *reinterpret_cast<u32x4*>(p.out + head * P::ROWB + 16 * i) = u32x4{0, 0, 0, 0};
      if (p.lse && tid % P::PER == 0) p.lse[head] = -INFINITY;
      return;
    }
  } else {
  long long here = 0, incl = scan(0, &here);
  total = here;
  for (int s0 = P::THREADS; s0 < p.seqs; s0 += P::THREADS) {
    long long more;
    scan(s0, &more);
    total += more;
  }
  total *= plan.units;
  n_groups = (int)min((long long)P::GROUPS, total);
  if ((int)blockIdx.x >= n_groups) return;
  x_begin = first_tile(total, n_groups, blockIdx.x);
  x_end = first_tile(total, n_groups, blockIdx.x + 1);
  {
    long long base = 0;                          // tiles of the sequences before s0
    for (int s0 = 0;;) {
      const int s = s0 + tid;
      const long long t = s < p.seqs ? (length_of(p, s) + P::TILE - 1) / P::TILE : 0;
      const long long lo = (base + incl - t) * plan.units, hi = (base + incl) * plan.units;
      if (lo <= x_begin && x_begin < hi) {
        found_s[0] = s;
        found_s[1] = lo;
      }
      base += here;
      s0 += P::THREADS;
      if (base * plan.units > x_begin || s0 >= p.seqs) break;      // uniform
      incl = scan(s0, &here);
    }
    __syncthreads();
  }
  seq = __builtin_amdgcn_readfirstlane((int)found_s[0]);
  seq_x = found_s[1];
  }

  const unsigned lds_stage = (unsigned)(unsigned long long)(LDS_PTR(unsigned char)) & stage[wave][0][0][0];
  const unsigned lds_pages = (unsigned)(unsigned long long)(LDS_PTR(int32_t)) & pages[wave][0][0];
  const float unit_scale = sizeof(T) == 2 ? kLog2e : 1.f;
  const float to_cap = MOD & CAP ? p.scale / p.cap : p.scale * unit_scale, cap = p.cap * unit_scale;
  const Near near(cap);

  for (long long x = x_begin; x < x_end;) {
    const int length = __builtin_amdgcn_readfirstlane(length_of(p, seq));
    const int tiles = (length + P::TILE - 1) / P::TILE;
    if (x >= seq_x + (long long)tiles * plan.units) {
      seq_x += (long long)tiles * plan.units;
      ++seq;
      continue;
    }
    const int unit = __builtin_amdgcn_readfirstlane((int)((x - seq_x) / tiles)), t0 = __builtin_amdgcn_readfirstlane((int)((x - seq_x) % tiles));
    const int t1 = __builtin_amdgcn_readfirstlane((int)min((long long)tiles, t0 + (x_end - x)));
    const int kv_head = unit / plan.blocks, block = unit % plan.blocks;
    const int row = block * kCols + j;           // of the group
    const bool real = row < p.group;
    const size_t head = (size_t)seq * p.heads + kv_head * p.group + row;
    const unsigned char* kg = p.k + kv_head * p.sk.head;
    const unsigned char* vg = p.v + kv_head * p.sv.head;
    const int32_t* table = p.table + (size_t)seq * p.max_pages;

    u32x4 q[P::ROWB / 64];
#pragma unroll
    for (int s = 0; s < P::ROWB / 64; ++s) {
      q[s] = u32x4{0, 0, 0, 0};
      if (real) q[s] = *reinterpret_cast<const u32x4*>(p.q + head * P::ROWB + 64 * s + 16 * g);
    }
    float slope = MOD & BIAS && real ? p.slopes[kv_head * p.group + row] * unit_scale : 0.f;
    f32x4 o[P::NDT];
#pragma unroll
    for (int dt = 0; dt < P::NDT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    // the loads above are complete before the walk, in which the compiler is to wait for nothing
#pragma unroll
    for (int s = 0; s < P::ROWB / 64; ++s) asm volatile("" : "+v"(q[s]));
    asm volatile("" : "+v"(slope));

    const int n = t1 - t0;
    const int key0 = t0 * P::TILE + wave * KT;   // this wave's first key of tile i: key0 + i TILE
    auto load_page = [&](int i) {
      const int key = min(key0 + i * P::TILE + lane % KT, length - 1);
      dma_word(lds_pages + (i & 1) * 256, table + key / p.page_size);
    };
    unsigned seen[2] = {0u, 0u};                 // bit k: key k of this wave's tile counts, by parity
    auto load_rows = [&](int i) {
      const int key = key0 + i * P::TILE + lane % KT;
      const int page = lds_read<int>(lds_pages + (i & 1) * 256 + 4 * (lane % KT));
      const bool ok = key < length && (unsigned)page < (unsigned)p.num_pages;
      const int slot = key % p.page_size;
      const unsigned char* none = reinterpret_cast<const unsigned char*>(&zero_row[0]);
      const unsigned char* kr = ok ? kg + (long long)page * p.sk.batch + (long long)slot * p.sk.token : none;
      const unsigned char* vr = ok ? vg + (long long)page * p.sv.batch + (long long)slot * p.sv.token : none;
      seen[i & 1] = (unsigned)__ballot(ok);
      const unsigned at = __builtin_amdgcn_readfirstlane(lds_stage + (i & 1) * 2 * P::BYTES);
#pragma unroll
      for (int u = 0; u < P::NLD; ++u) {
        const int r = P::RPL * u + lane / P::CPR;
        const unsigned chunk = (unsigned)(((lane % P::CPR) ^ swz<T, D>(r)) << 4);
        dma_rows(at + u * 1024, shfl_ptr(kr, r) + chunk);
      }
#pragma unroll
      for (int u = 0; u < P::NLD; ++u) {
        const int r = P::RPL * u + lane / P::CPR;
        const unsigned chunk = (unsigned)(((lane % P::CPR) ^ swz<T, D>(r)) << 4);
        dma_rows(at + P::BYTES + u * 1024, shfl_ptr(vr, r) + chunk);
      }
    };

    wait_all_but<0>();
    load_page(0);
    if (n > 1) {
      load_page(1);
      wait_all_but<1>();
    } else {
      wait_all_but<0>();
    }
    load_rows(0);
    for (int i = 0; i < n; ++i) {
      // under way: page numbers of tile i + 1, rows of tile i
      if (i + 1 < n) {
        wait_all_but<NKV>();                     // page numbers of tile i + 1
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");     // the stage that the next rows go to has been read
        if (i + 2 < n) {
          load_page(i + 2);
          load_rows(i + 1);
          wait_all_but<NKV + 1>();
        } else {
          load_rows(i + 1);
          wait_all_but<NKV>();
        }
      } else {
        wait_all_but<0>();
      }
      const unsigned k_at = lds_stage + (i & 1) * 2 * P::BYTES, v_at = k_at + P::BYTES;
      const unsigned bits = seen[i & 1];
      float z[KT / 4];
      float top = -INFINITY;
#pragma unroll
      for (int sub = 0; sub < KT / 16; ++sub) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < P::ROWB / 64; ++c)
          s = mma16_step<T>(lds_read<u32x4>(k_at + (16 * sub + j) * P::ROWB + (((4 * c + g) ^ swz<T, D>(16 * sub + j)) << 4)), q[c], s);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float y = s[r] * to_cap;
          if (MOD & CAP) y = tanh_times<T>(y, near, cap);
          if (MOD & BIAS) y = fmaf(-slope, (float)(length - 1 - (key0 + i * P::TILE + 16 * sub + 4 * g + r)), y);
          if (!((bits >> (16 * sub + 4 * g + r)) & 1u)) y = -INFINITY;
          z[4 * sub + r] = y;
          top = fmaxf(top, y);
        }
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m, top);
      if (__any(m_new != m)) {
        const float f = m == -INFINITY ? 0.f : exp_of<T>(m - m_new);
        l *= f;
#pragma unroll
        for (int dt = 0; dt < P::NDT; ++dt) o[dt] *= f;
        m = m_new;
      }
      const float minus_m = m == -INFINITY ? 0.f : -m;
#pragma unroll
      for (int e = 0; e < KT / 4; ++e) {
        z[e] = exp_of<T>(z[e] + minus_m);
        l += z[e];
      }
      if constexpr (sizeof(T) == 2) {
        const u32x4 w = {pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]), pack_bf16(z[4], z[5]), pack_bf16(z[6], z[7])};
#pragma unroll
        for (int dt = 0; dt < P::NDT; ++dt) {
          s16x4 a[2];
#pragma unroll
          for (int sub = 0; sub < 2; ++sub) {
            const int r = 16 * sub + 4 * g + (j >> 2);
            const unsigned at = v_at + r * P::ROWB + (((2 * dt + ((j & 3) >> 1)) ^ swz<T, D>(r)) << 4) + 8 * (j & 1);
            a[sub] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_PTR(s16x4)>((LDS_PTR(unsigned char))(unsigned long long)at));
          }
          const u32x2 l2 = __builtin_bit_cast(u32x2, a[0]), h2 = __builtin_bit_cast(u32x2, a[1]);
          o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, (u32x4{l2.x, l2.y, h2.x, h2.y})),
                                                          __builtin_bit_cast(bf16x8, w), o[dt], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int dt = 0; dt < P::NDT; ++dt) {
            const int k = 4 * g + r;
            const float a = lds_read<float>(v_at + k * P::ROWB + (((4 * dt + (j >> 2)) ^ swz<T, D>(k)) << 4) + 4 * (j & 3));
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, z[r], o[dt], 0, 0, 0);
          }
      }
    }

    // ---- join the four waves: each leaves its sums in its own stage ----
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    {
      LDS_PTR(float) dst = reinterpret_cast<LDS_PTR(float)>((LDS_PTR(unsigned char))&stage[wave][0][0][0]);
#pragma unroll
      for (int dt = 0; dt < P::NDT; ++dt) *reinterpret_cast<LDS_PTR(f32x4)>(dst + j * D + 16 * dt + 4 * g) = o[dt];
      if (g == 0) {
        ml_s[wave][0][j] = m;
        ml_s[wave][1][j] = l;
      }
    }
    __syncthreads();
    {
      constexpr int CH = D / P::PER;             // channels of a thread
      const int c = tid / P::PER, ch0 = (tid % P::PER) * CH, r = block * kCols + c;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < P::WAVES; ++w) top = fmaxf(top, ml_s[w][0][c]);
      float f[P::WAVES], sum = 0.f;
#pragma unroll
      for (int w = 0; w < P::WAVES; ++w) {
        f[w] = ml_s[w][0][c] == -INFINITY ? 0.f : exp_of<T>(ml_s[w][0][c] - top);
        sum += ml_s[w][1][c] * f[w];
      }
      const bool whole = t0 == 0 && t1 == tiles;
      const float norm = whole ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f;
      const size_t slot = (size_t)blockIdx.x * 2 + (x == x_begin ? 0 : 1);
      const size_t hd = (size_t)seq * p.heads + kv_head * p.group + r;
#pragma unroll
      for (int e = 0; e < CH; e += 4) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < P::WAVES; ++w)
          acc += *reinterpret_cast<LDS_PTR(const f32x4)>(reinterpret_cast<LDS_PTR(const float)>((LDS_PTR(unsigned char))&stage[w][0][0][0]) +
                                                         c * D + ch0 + e) * f[w];
        acc *= norm;
        if (!whole) {
          *reinterpret_cast<f32x4*>(plan.part_o + (slot * kCols + c) * D + ch0 + e) = acc;
        } else if (r < p.group) {
          if constexpr (sizeof(T) == 2)
            *reinterpret_cast<u32x2*>(p.out + (hd * D + ch0 + e) * 2) = u32x2{pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3])};
          else
            *reinterpret_cast<f32x4*>(p.out + (hd * D + ch0 + e) * 4) = acc;
        }
      }
      if (!plan.solo && t0 == 0 && tid == 0) {   // who has this unit, for the launch that joins
        const long long x1 = x + tiles - 1;
        int32_t* own = plan.owners + ((size_t)seq * plan.units + unit) * 2;
        own[0] = (int)blockIdx.x | (x == x_begin ? 0 : kSecondSlot);
        own[1] = (int)(((x1 + 1) * n_groups - 1) / total);       // the last workgroup whose range starts at or before x1
      }
      if (tid % P::PER == 0) {
        if (!whole) {
          plan.part_ml[(slot * 2 + 0) * kCols + c] = top;
          plan.part_ml[(slot * 2 + 1) * kCols + c] = sum;
        } else if (r < p.group && p.lse) {
          p.lse[hd] = sum == 0.f ? -INFINITY : log_sum<T>(top, sum);
        }
      }
    }
    __syncthreads();
    x += n;
  }
}

// A workgroup to a (sequence, unit): nothing to do where one workgroup had all of it.  A thread has D / 16 channels of a row.
template <typename T, int D> __global__ __launch_bounds__(256) void paged_join_kernel(Paged p, PPlan plan) {
  const int seq = blockIdx.x / plan.units, unit = blockIdx.x % plan.units, tid = threadIdx.x;
  const int kv_head = unit / plan.blocks, c = tid / 16, j = tid % 16, ch0 = j * (D / 16), r = unit % plan.blocks * kCols + c;
  const bool empty = length_of(p, seq) == 0;
  const int2 own = *reinterpret_cast<const int2*>(plan.owners + (size_t)blockIdx.x * 2);
  const int w0 = own.x & (kSecondSlot - 1), w1 = own.y;
  if ((!empty && w0 == w1) || r >= p.group) return;
  const size_t hd = (size_t)seq * p.heads + kv_head * p.group + r;

  float top = -INFINITY, sum = 0.f;
  f32x4 acc[D / 64];
#pragma unroll
  for (int e = 0; e < D / 64; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (!empty) {
    // parts 16 at a time, one to each of a row's 16 threads for the maximum and the factor
    auto slot_of = [&](int w) { return (size_t)w * 2 + (w == w0 && (own.x & kSecondSlot) ? 1 : 0); };
    for (int w = w0; w <= w1; w += 16) {
      float m = -INFINITY, l = 0.f;
      if (w + j <= w1) {
        m = plan.part_ml[slot_of(w + j) * 2 * kCols + c];
        l = plan.part_ml[(slot_of(w + j) * 2 + 1) * kCols + c];
      }
      float t = m;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) t = fmaxf(t, __shfl_xor(t, o, 16));
      const float m_new = fmaxf(top, t);
      const float old = top == -INFINITY ? 0.f : exp_of<T>(top - m_new);
      const float f = l == 0.f ? 0.f : exp_of<T>(m - m_new);
      top = m_new;
      float part = l * f;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) part += __shfl_xor(part, o, 16);
      sum = sum * old + part;
#pragma unroll
      for (int e = 0; e < D / 64; ++e) acc[e] *= old;
      const int n = min(16, w1 - w + 1);
      for (int i = 0; i < n; i += 4) {
        f32x4 x[4][D / 64];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < D / 64; ++e)
            x[u][e] = *reinterpret_cast<const f32x4*>(plan.part_o + (slot_of(w + min(i + u, n - 1)) * kCols + c) * D + ch0 + 4 * e);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float g = __shfl(f, min(i + u, 15), 16);         // 0 past the last part
          if (i + u < n && g != 0.f)
#pragma unroll
            for (int e = 0; e < D / 64; ++e) acc[e] += x[u][e] * g;
        }
      }
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int e = 0; e < D / 64; ++e) {
    const f32x4 y = acc[e] * inv;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<u32x2*>(p.out + (hd * D + ch0 + 4 * e) * 2) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
    else
      *reinterpret_cast<f32x4*>(p.out + (hd * D + ch0 + 4 * e) * 4) = y;
  }
  if (p.lse && j == 0) p.lse[hd] = sum == 0.f ? -INFINITY : log_sum<T>(top, sum);
}

// A thread moves 16 bytes of one token's key or value row of one head.
__global__ __launch_bounds__(256) void paged_append_kernel(Paged p, const unsigned char* k, const unsigned char* v, int tokens,
                                                           const int32_t* offsets, int chunks /* of 16 bytes in a row */) {
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long row = at / chunks;             // token, head, key or value
  const int chunk = (int)(at % chunks);
  const int which = (int)(row & 1);
  const long long th = row >> 1;
  const int head = (int)(th % p.kv_heads);
  if (th / p.kv_heads >= tokens) return;
  const int token = (int)(th / p.kv_heads);
  int lo = 0, hi = p.seqs + 1;                   // the last offset <= token is number lo - 1
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= token) lo = mid + 1;
    else hi = mid;
  }
  if (lo == 0 || lo > p.seqs) return;
  const int seq = lo - 1;
  const long long pos = (long long)p.lengths[seq] - ((long long)offsets[lo] - token);
  if (pos < 0 || pos >= (long long)p.max_pages * p.page_size) return;
  const int page = p.table[(size_t)seq * p.max_pages + pos / p.page_size];
  if ((unsigned)page >= (unsigned)p.num_pages) return;
  const Strides& st = which ? p.sv : p.sk;
  const u32x4 x = *reinterpret_cast<const u32x4*>((which ? v : k) + (th * chunks + chunk) * 16);
  *reinterpret_cast<u32x4*>((which ? p.v : p.k) + page * st.batch + head * st.head + (pos % p.page_size) * st.token + 16 * chunk) = x;
}

PPlan plan_of(const Paged& p) {
  PPlan pl{};
  pl.blocks = (p.group + kCols - 1) / kCols;
  pl.units = p.kv_heads * pl.blocks;
  // A table of two tiles at most: one workgroup walks them in less time than a second launch takes (8 / 2 heads, tables of 256
  // tokens 10.1 -> 7.8 us, of 512 10.1 -> 11.2).
  pl.solo = (long long)p.max_pages * p.page_size <= (p.dtype == PISA_BF16 ? 256 : 128);
  return pl;
}
int groups_of(const Paged& p) {
  if (p.dtype == PISA_BF16) return p.d == 64 ? PGeo<__bf16, 64>::GROUPS : PGeo<__bf16, 128>::GROUPS;
  return p.d == 64 ? PGeo<float, 64>::GROUPS : PGeo<float, 128>::GROUPS;
}

template <typename T, int D> hipError_t launch_td(const Paged& p, const PPlan& pl, hipStream_t stream) {
  const dim3 grid(pl.solo ? p.seqs * pl.units : PGeo<T, D>::GROUPS), block(256);
  switch ((p.cap > 0.f ? CAP : 0) | (p.slopes ? BIAS : 0)) {
    case 0: hipLaunchKernelGGL((paged_kernel<T, D, 0>), grid, block, 0, stream, p, pl); break;
    case CAP: hipLaunchKernelGGL((paged_kernel<T, D, CAP>), grid, block, 0, stream, p, pl); break;
    case BIAS: hipLaunchKernelGGL((paged_kernel<T, D, BIAS>), grid, block, 0, stream, p, pl); break;
    default: hipLaunchKernelGGL((paged_kernel<T, D, CAP | BIAS>), grid, block, 0, stream, p, pl); break;
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || pl.solo) return e;
  hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3(p.seqs * pl.units), block, 0, stream, p, pl);
  return hipGetLastError();
}

}  // namespace

size_t paged_workspace_bytes(const Paged& p) {
  return (size_t)groups_of(p) * 2 * kCols * (p.d + 2) * sizeof(float) + (size_t)p.seqs * plan_of(p).units * 2 * sizeof(int32_t);
}

hipError_t launch_paged_attention(const Paged& p, hipStream_t stream) {
  PPlan pl = plan_of(p);
  pl.part_o = static_cast<float*>(p.workspace);
  pl.part_ml = pl.part_o + (size_t)groups_of(p) * 2 * kCols * p.d;
  pl.owners = reinterpret_cast<int32_t*>(pl.part_ml + (size_t)groups_of(p) * 2 * 2 * kCols);
  if (p.dtype == PISA_BF16) return p.d == 64 ? launch_td<__bf16, 64>(p, pl, stream) : launch_td<__bf16, 128>(p, pl, stream);
  return p.d == 64 ? launch_td<float, 64>(p, pl, stream) : launch_td<float, 128>(p, pl, stream);
}

hipError_t launch_paged_append(const Paged& p, const void* k, const void* v, int tokens, const int32_t* offsets, hipStream_t stream) {
  if (tokens == 0) return hipSuccess;
  const int chunks = p.d * (p.dtype == PISA_BF16 ? 2 : 4) / 16;
  const long long threads = 2LL * tokens * p.kv_heads * chunks;
  hipLaunchKernelGGL(paged_append_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, p,
                     static_cast<const unsigned char*>(k), static_cast<const unsigned char*>(v), tokens, offsets, chunks);
  return hipGetLastError();
}

}  // namespace pisa

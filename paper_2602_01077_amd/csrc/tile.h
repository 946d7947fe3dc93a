// Device helpers of the masked attention kernels: 64-row tiles staged in LDS, and the products taken from them.
//
// Everything is a template over the element type T (__bf16 or float) and the head dimension D.  A tile is 64 rows of
// ROWB = D * sizeof(T) bytes.  Both kinds of operand are taken from one staged copy:
//   rows      the matrix instruction's A operand is 32 rows, contracted over channels (ds_read_b128: lane lam of each half h
//             reads 16 bytes of row lam, so a contraction step takes 32 bytes of every row)
//   columns   its A operand is 32 channels, contracted over rows (bf16: ds_read_b64_tr_b16; fp32: one value per lane)
// and the B operand is in registers: a lane's own row, or the probabilities as the first product left them.
// With v_mfma_f32_32x32x16_bf16 and v_mfma_f32_32x32x2_f32 alike, register r of lane (lam, h) of a product holds row
// (r / 4) * 8 + 4 h + r % 4 and column lam; a later contraction over those rows takes them in that order on both sides.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace pisa {
namespace tile {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// Lambdas and functions that take a wave's registers by reference: called out of line, those would lie in memory.
#define INLINE __attribute__((always_inline))
#define LDS_PTR(T) __attribute__((address_space(3))) T*

constexpr int kRows = 64;                        // rows of a staged tile
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// The lane number, made anew where it stands: for loops that have no register to keep it in.
__device__ __forceinline__ int lane_anew() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
  return lane;
}

template <typename T, int D> struct Geo {
  static constexpr int ROWB = D * (int)sizeof(T);
  static constexpr int TILEB = kRows * ROWB;
  static constexpr int STEPS = ROWB / 32;        // contraction steps over the channels (16 in bf16, 8 in fp32)
  static constexpr int NDT = D / 32;             // 32-channel tiles
  static constexpr int CPR = ROWB / 16;          // 16-byte chunks of a row
  static constexpr int RPL = 64 / CPR;           // rows that one wave-load of 1 KB covers
  static constexpr int NLD = TILEB / 4096;       // wave-loads per wave and tile, four waves
};

// The 16-byte chunks of staged row r lie at chunk index XOR swz(r).  Both kinds of read are free of bank conflicts with it: a
// ds_read_b128 of one chunk takes 16 rows on 16 different 16-byte columns of the 64 banks, and the two 16-lane groups of a
// half-wave that read 32 bytes each of four consecutive rows get eight different 32-byte columns.  fp32: rows r and r + 4,
// which the two halves read together, lie in different halves of the banks.
template <typename T, int D> __host__ __device__ constexpr int swz(int r) {
  if (sizeof(T) == 4) return (((r >> 2) & 1) << 3) | ((r & 3) << 1) | ((r >> 3) & 1);
  if (D == 128) return ((((r & 3) << 1) | ((r >> 2) & 1)) << 1) | ((r >> 3) & 1);
  return (((r >> 1) & 1) << 2) | (((r >> 2) & 1) << 1) | ((r >> 3) & 1);       // two rows share the 64 banks
}

// LDS-DMA of 1 KB: lane l's 16 bytes go to lds + 16 l.  In inline asm, so that the compiler puts no wait on it in front of
// reads of another stage; wait_loads() and a barrier come before the tile is read.  A scalar write of M0 needs one wait
// state before the load reads it.
__device__ __forceinline__ void dma_1kb(unsigned lds, unsigned voff, const unsigned char* base /* both uniform */) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}
// The same for one 4-byte word a lane.
__device__ __forceinline__ void dma_words(unsigned lds, unsigned voff, const void* base /* uniform, as lds */) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }     // vmcnt(0), the other counters left alone

// A wave's part in loading tiles of a tensor with `stride` bytes from row to row: rows 16 wave .. + 15, piece i of them rows
// RPL i .. + RPL - 1.  Rows past `avail` (>= 1) are replaced by the last valid one; the caller masks them.
// ANEW: every address is made anew for every tile, from the lane number alone.  The dk, dv walk has no registers for offsets:
// spilled, their reloads waited between the loads (24 heads of 4 608, backward 1 200 us, so 990).  Elsewhere they are worth
// a register for each piece (forward 275 us made anew, 257 so).
template <typename T, int D, bool ANEW = false> struct Loader {
  using G = Geo<T, D>;
  static_assert(G::RPL * G::NLD == 16, "a wave loads 16 rows, the swizzle's period");
  unsigned stride;
  unsigned off[ANEW ? 1 : G::NLD];               // byte offset from the tile's first row, piece by piece
  __device__ __forceinline__ static int row(int wave, int lane, int i) { return G::RPL * (G::NLD * wave + i) + lane / G::CPR; }
  __device__ __forceinline__ static unsigned chunk(int lane, int r) { return (unsigned)(((lane % G::CPR) ^ swz<T, D>(r)) << 4); }
  __device__ __forceinline__ void init(int wave, int lane, unsigned stride_) {
    stride = stride_;
#pragma unroll
    for (int i = 0; i < (ANEW ? 0 : G::NLD); ++i) off[i] = (unsigned)row(wave, lane, i) * stride + chunk(lane, row(wave, lane, i));
  }
  __device__ __forceinline__ void load(int wave, int lane, const unsigned char* base, int avail, unsigned lds) const {
    const unsigned at = __builtin_amdgcn_readfirstlane(lds + wave * (G::NLD * 1024));
    if constexpr (ANEW) {
      lane = lane_anew();
      const int l = lane / G::CPR;
      const unsigned chunk0 = chunk(lane, l);
#pragma unroll
      for (int i = 0; i < G::NLD; ++i) {
        // the swizzle only moves bits of the row: that of a row is that of its place in the piece XOR that of the piece
        const int r0 = 16 * wave + G::RPL * i;
        const unsigned c = chunk0 ^ (unsigned)(swz<T, D>(G::RPL * i) << 4);
        if (avail >= kRows) dma_1kb(at + i * 1024, (unsigned)l * stride + c, base + (unsigned)r0 * (unsigned long long)stride);
        else dma_1kb(at + i * 1024, (unsigned)min(r0 + l, avail - 1) * stride + c, base);
      }
    } else if (avail >= kRows) {
#pragma unroll
      for (int i = 0; i < G::NLD; ++i) dma_1kb(at + i * 1024, off[i], base);
    } else {
#pragma unroll
      for (int i = 0; i < G::NLD; ++i) {
        const int r = row(wave, lane, i);
        dma_1kb(at + i * 1024, (unsigned)min(r, avail - 1) * stride + chunk(lane, r), base);
      }
    }
  }
};

// This lane's addresses in a staged tile that starts at `tile` (a multiple of 1 KB).
template <typename T, int D> struct Reader {
  using G = Geo<T, D>;
  unsigned rows;                                 // 16 bytes of row lam, contraction step 0
  unsigned cols;                                 // columns: bf16, rows 0..7 of a contraction step of 16 (8..15: bit 4 flips)
  __device__ __forceinline__ void init(int lane, unsigned tile) {
    const int lam = lane & 31, h = lane >> 5;
    rows = tile + lam * G::ROWB + ((h ^ swz<T, D>(lam)) << 4);
    if (sizeof(T) == 2) {
      // lane j of a 16-lane group points at 4 channels of row j / 4 and receives channel j of the group's four rows
      const int j = lane & 15, kq = 4 * h + (j >> 2), lhalf = (lane >> 4) & 1;
      static_assert(sizeof(T) == 4 || swz<T, D>(8) == 1, "row r + 8 lies at row r's chunk XOR 1");
      cols = tile + kq * G::ROWB + (((2 * lhalf + ((j & 3) >> 1)) ^ swz<T, D>(kq)) << 4) + 8 * (j & 1);
    } else {
      // swz(row + 4 h) is swz(row) ^ (h << 3) for the rows that this lane starts from, and XOR of chunks is XOR of addresses
      cols = tile + 4 * h * G::ROWB + (lam & 3) * 4 + (((lam >> 2) ^ (h << 3)) << 4);
    }
  }
};

template <typename V> __device__ __forceinline__ V lds_read(unsigned at) {
  return *reinterpret_cast<LDS_PTR(const V)>((LDS_PTR(const unsigned char))(unsigned long long)at);
}

// One contraction step over channels (32 bytes of each row): acc += A B.
template <typename T> __device__ __forceinline__ f32x16 mma_step(u32x4 a, u32x4 b, f32x16 acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
    return acc;
  }
}

// What later steps take from LDS is under way before this one's products: three steps in bf16, one in fp32 (four instructions of
// twice the time).  Left to itself the scheduler moves reads to their use and waits for each (24 heads of 4 608, backward 915 us,
// so 888; fp32, 8 of 4 500, forward 895, so 776).  At 64 channels, where registers are left, plain operations may pass (24 of
// 4 608 forward 171 where they may not, 159 so; at 128 channels 253 and 258).
constexpr int kAhead = 3;
template <typename T, int D> __device__ __forceinline__ void read_ahead() {
  constexpr int kVector = 0x2, kScalar = 0x4, kTranscendental = 0x400;
  __builtin_amdgcn_sched_barrier(sizeof(T) == 2 && D == 64 ? kVector | kScalar | kTranscendental : 0);
}

// acc = (32 rows of the tile, from row ROW0) * (the lane's own row, all channels).  OFF: byte offset of the tile.
template <typename T, int D, int ROW0>
__device__ __forceinline__ f32x16 rows_times(const Reader<T, D>& rd, unsigned off, const u32x4 (&b)[Geo<T, D>::STEPS]) {
  f32x16 acc = (f32x16){0};
  if constexpr (sizeof(T) == 2) {
    constexpr int STEPS = Geo<T, D>::STEPS;
    u32x4 a[STEPS];
#pragma unroll
    for (int s = -kAhead; s < STEPS; ++s) {
      if (s + kAhead < STEPS) a[s + kAhead] = lds_read<u32x4>((rd.rows ^ ((s + kAhead) << 5)) + off + ROW0 * Geo<T, D>::ROWB);
      if (s < 0) continue;
      read_ahead<T, D>();
      acc = mma_step<T>(a[s], b[s], acc);
    }
  } else {
    unsigned at = rd.rows + off;                 // opaque: addresses kept for the walk would take the registers of what is read ahead
    asm volatile("" : "+v"(at));
    u32x4 a[2] = {lds_read<u32x4>(at + ROW0 * Geo<T, D>::ROWB)};
#pragma unroll
    for (int s = 0; s < Geo<T, D>::STEPS; ++s) {
      if (s + 1 < Geo<T, D>::STEPS) a[(s + 1) & 1] = lds_read<u32x4>((at ^ ((s + 1) << 5)) + ROW0 * Geo<T, D>::ROWB);
      read_ahead<T, D>();
      acc = mma_step<T>(a[s & 1], b[s], acc);
    }
  }
  return acc;
}

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  f32x2 f = {lo, hi};
  bf16x2 b = __builtin_convertvector(f, bf16x2);
  return __builtin_bit_cast(unsigned, b);
}

// 32 rows' worth of a lane's values as the B operand of the product that contracts over those rows.
template <typename T> struct Weights;
template <> struct Weights<__bf16> {
  u32x4 w[2];
  __device__ __forceinline__ void set(int r, float a, float b) { w[r >> 3][(r & 7) >> 1] = pack_bf16(a, b); }    // rows r, r + 1 (r even)
};
template <> struct Weights<float> {
  f32x16 w;
  __device__ __forceinline__ void set(int r, float a, float b) {
    w[r] = a;
    w[r + 1] = b;
  }
};

// acc[dt] += (32 rows of the tile, from row ROW0)^T (channels x rows) * weights (rows x the lane's column).
template <typename T, int D, int ROW0>
__device__ __forceinline__ void cols_times(const Reader<T, D>& rd, unsigned off, const Weights<T>& p, f32x16 (&acc)[Geo<T, D>::NDT]) {
  constexpr int ROWB = Geo<T, D>::ROWB;
  if constexpr (sizeof(T) == 2) {
    constexpr int NDT = Geo<T, D>::NDT, N = 2 * NDT;
    u32x4 a[N];
#pragma unroll
    for (int i = -kAhead; i < N; ++i) {
      if (i + kAhead < N) {
        const int s = (i + kAhead) / NDT, dt = (i + kAhead) % NDT;
        const unsigned at = off + (ROW0 + 16 * s) * ROWB;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            reinterpret_cast<LDS_PTR(s16x4)>((LDS_PTR(unsigned char))(unsigned long long)((rd.cols ^ (dt << 6)) + at)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            reinterpret_cast<LDS_PTR(s16x4)>((LDS_PTR(unsigned char))(unsigned long long)((rd.cols ^ (dt << 6) ^ 16) + at + 8 * ROWB)));
        const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
        a[i + kAhead] = u32x4{l2.x, l2.y, h2.x, h2.y};
      }
      if (i < 0) continue;
      read_ahead<T, D>();
      acc[i % NDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, p.w[i / NDT]),
                                                             acc[i % NDT], 0, 0, 0);
    }
  } else {
    constexpr int N = Geo<T, D>::NDT;
    unsigned at = rd.cols + off;
    asm volatile("" : "+v"(at));
    float a[2][N];
    auto read = [&](int r) INLINE {
      const int base = (r / 4) * 8 + r % 4;      // this lane reads row base + 4 h
#pragma unroll
      for (int dt = 0; dt < N; ++dt) a[r & 1][dt] = lds_read<float>((at ^ (unsigned)(((8 * (dt & 1)) ^ swz<T, D>(base)) << 4)) + 256 * (dt >> 1) + (ROW0 + base) * ROWB);
    };
    read(0);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if (r + 1 < 16) read(r + 1);
      read_ahead<T, D>();
#pragma unroll
      for (int dt = 0; dt < N; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[r & 1][dt], p.w[r], acc[dt], 0, 0, 0);
    }
  }
}

// exp of a difference of scores.  Scores are kept in the log2 domain in bf16 (the exponent is one fused operation) and in the
// natural one in fp32, where the rounded constant would cost the last digits: z - m is one fused operation on the raw
// product, small where the weight is not, and only then multiplied.
template <typename T> __device__ __forceinline__ float exp_diff(float s, float c, float minus_m) {
  if (sizeof(T) == 2) return __builtin_amdgcn_exp2f(fmaf(s, c, minus_m));
  return __builtin_amdgcn_exp2f(fmaf(s, c, minus_m) * kLog2e);
}
template <typename T> __device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(sizeof(T) == 2 ? x : x * kLog2e); }
template <typename T> __device__ __forceinline__ float log_of(float x) { return sizeof(T) == 2 ? __builtin_amdgcn_logf(x) : logf(x); }
// log of a sum of weights in that domain, and its way to the natural one
template <typename T> __device__ __forceinline__ float log_sum(float m, float l) {
  return sizeof(T) == 2 ? (m + log_of<T>(l)) * kLn2 : m + log_of<T>(l);
}

__device__ __forceinline__ float max_of(const f32x16& s) {
  float t = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) t = fmaxf(t, s[r]);
  return t;
}

// tanh of capped scores.  bf16: they mostly stay far below the cap, where an odd polynomial of degree 7 (fitted here to a
// relative 1e-7 for |x| <= 0.4) takes six plain operations; beyond, one exponential and one reciprocal, a quarter of the rate
// each, absolute error 1e-7.
constexpr float kNear = 0.4f;
struct Near {                                    // mult tanh(x) = x of(x^2)
  float c0, c1, c2, c3;
  // the same in s = x / to_cap, mult tanh(to_cap s) = s of(s^2), where no power of it leaves the range of fp32 (all_direct)
  __device__ __forceinline__ void rescale(float to_cap) {
    const float u = to_cap * to_cap;
    c0 *= to_cap;
    c1 *= to_cap * u;
    c2 *= to_cap * u * u;
    c3 *= to_cap * u * u * u;
  }
  __device__ __forceinline__ static bool all_direct(float mult, float to_cap) {
    return to_cap >= 0x1p-16f && to_cap <= 16.f && mult >= 0x1p-8f && mult <= 0x1p20f;
  }
  __device__ __forceinline__ Near(float mult) : c0(mult * 9.999999019e-01f), c1(mult * -3.333136246e-01f), c2(mult * 1.327097675e-01f), c3(mult * -4.755360305e-02f) {}
  __device__ __forceinline__ float of(float u) const { return fmaf(fmaf(fmaf(c3, u, c2), u, c1), u, c0); }
};
// mult tanh(x) of one value, as cap_scores has it.
template <typename T> __device__ __forceinline__ float tanh_times(float x, const Near& near, float mult) {
  if (sizeof(T) == 4) return mult * tanhf(x);
  const float far = fmaf(-2.f * mult, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * (2.f * kLog2e)) + 1.f), mult);
  return x * x <= kNear * kNear ? x * near.of(x * x) : far;          // the line that cap_scores draws
}
// s = mult tanh(to_cap s), to_cap > 0, for 32 rows' worth of scores.
template <typename T> __device__ __forceinline__ void cap_scores(f32x16& s, float to_cap, float mult) {
  if (sizeof(T) == 4) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = mult * tanhf(s[r] * to_cap);
    return;
  }
  const Near near(mult);
  float top = 0.f;
#pragma unroll
  for (int r = 0; r < 16; r += 2) {
    s[r] *= to_cap;
    s[r + 1] *= to_cap;
    top = fmaxf(fmaxf(s[r] * s[r], s[r + 1] * s[r + 1]), top);
  }
  if (__builtin_expect(!__any(!(top <= kNear * kNear)), 1)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] *= near.of(s[r] * s[r]);
  } else {                                       // score by score, so that what a row gives does not hang on its neighbours
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = tanh_times<T>(s[r], near, mult);
  }
}
// An element that is not finite, as its bits: infinity becomes the largest number, whose score is as far off and which a weight
// of 0 takes away, NaN becomes 0.
template <typename T> __device__ __forceinline__ unsigned tamed(unsigned w) {
  if (sizeof(T) == 2) return (w & 0x7fu) ? 0u : (w & 0x8000u) | 0x7f7fu;
  return (w & 0x7fffffu) ? 0u : (w & 0x80000000u) | 0x7f7fffffu;
}
// Whether some element of these 16 bytes is infinite or NaN: its exponent is all ones.
template <typename T> __device__ __forceinline__ bool unlike_finite(u32x4 w) {
  unsigned top = 0u;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    top = max(top, w[e] & 0x7f800000u);
    if (sizeof(T) == 2) top = max(top, (w[e] & 0x7f80u) << 16);
  }
  return top == 0x7f800000u;
}
// Non-finite elements of a staged tile are tamed, and the rows they were in marked in bad[0..1] (64 bits, zero before).  A
// product contracts over all rows of a tile, also where the weight is 0, and 0 * inf is NaN: tiles that are masked in part are
// cleaned first.  All 256 threads; a barrier before and after is the caller's.
template <typename T, int D> __device__ __forceinline__ void clean_tile(LDS_PTR(unsigned char) stage, LDS_PTR(unsigned) bad, int tid) {
  using G = Geo<T, D>;
#pragma unroll
  for (int i = 0; i < G::TILEB / 4096; ++i) {
    const int at = (i * 256 + tid) * 16;
    LDS_PTR(u32x4) p = reinterpret_cast<LDS_PTR(u32x4)>(stage + at);
    u32x4 w = *p;
    if (unlike_finite<T>(w)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (sizeof(T) == 2) {
          if ((w[e] & 0x7f80u) == 0x7f80u) w[e] = (w[e] & 0xffff0000u) | tamed<T>(w[e] & 0xffffu);
          if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] = (w[e] & 0xffffu) | tamed<T>(w[e] >> 16) << 16;
        } else if ((w[e] & 0x7f800000u) == 0x7f800000u) {
          w[e] = tamed<T>(w[e]);
        }
      }
      *p = w;
      const int r = at / G::ROWB;
      atomicOr((unsigned*)(bad + (r >> 5)), 1u << (r & 31));
    }
  }
}

// The same marks for 64 rows in memory, the first `avail` of them there.
template <typename T, int D> __device__ __forceinline__ void mark_rows(const unsigned char* rows, long long stride, int avail,
                                                                       LDS_PTR(unsigned) bad, int tid) {
  using G = Geo<T, D>;
  for (int i = 0; i < G::TILEB / 4096; ++i) {
    const int at = (i * 256 + tid) * 16, r = at / G::ROWB;
    if (r >= avail) continue;
    const u32x4 w = *reinterpret_cast<const u32x4*>(rows + r * stride + at % G::ROWB);
    if (unlike_finite<T>(w)) atomicOr((unsigned*)(bad + (r >> 5)), 1u << (r & 31));
  }
}

// A walk over double-buffered tiles, trip(i, parity).  In bf16 two at a time, so that the stages lie at offsets known when
// compiled, which every read from LDS then has in its instruction (24 heads of 4 608, forward 290 -> 272 us, backward 1 280 ->
// 1 212).  In fp32, which waits for its products, the copy only costs registers (8 heads of 4 500, causal, 561 -> 994).
template <typename T, typename Trip> __device__ __forceinline__ void walk_stages(int begin, int end, const Trip& trip) {
  if constexpr (sizeof(T) == 2) {
    for (int i = begin; i < end; i += 2) {
      trip(i, std::integral_constant<int, 0>{});
      if (i + 1 >= end) break;
      trip(i + 1, std::integral_constant<int, 1>{});
    }
  } else {
    for (int i = begin; i < end; ++i) trip(i, (i - begin) & 1);
  }
}

}  // namespace tile
}  // namespace pisa

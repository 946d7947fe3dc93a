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

#define LDS_PTR(T) __attribute__((address_space(3))) T*

constexpr int kRows = 64;                        // rows of a staged tile
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

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
template <typename T, int D> __device__ inline int swz(int r) {
  if (sizeof(T) == 4) return (((r >> 2) & 1) << 3) | ((r & 3) << 1) | ((r >> 3) & 1);
  if (D == 128) return ((((r & 3) << 1) | ((r >> 2) & 1)) << 1) | ((r >> 3) & 1);
  return (((r >> 1) & 1) << 2) | (((r >> 2) & 1) << 1) | ((r >> 3) & 1);       // two rows share the 64 banks
}

// LDS-DMA of 1 KB: lane l's 16 bytes go to lds + 16 l.  In inline asm, so that the compiler puts no wait on it in front of
// reads of another stage; wait_loads() and a barrier come before the tile is read.  A scalar write of M0 needs one wait
// state before the load reads it.
__device__ inline void dma_1kb(unsigned lds, unsigned voff, const unsigned char* base /* both uniform */) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}
// The same for one 4-byte word a lane.
__device__ inline void dma_words(unsigned lds, unsigned voff, const void* base /* uniform, as lds */) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}
__device__ inline void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }     // vmcnt(0), the other counters left alone

// This lane's part in loading tiles of a tensor with `stride` bytes from row to row.
template <typename T, int D> struct Loader {
  using G = Geo<T, D>;
  unsigned off[G::NLD];                          // byte offset from the tile's first row, piece by piece
  unsigned stride;
  __device__ inline static int row(int wave, int lane, int i) { return G::RPL * (G::NLD * wave + i) + lane / G::CPR; }
  __device__ inline static unsigned chunk(int lane, int r) { return (unsigned)(((lane % G::CPR) ^ swz<T, D>(r)) << 4); }
  __device__ inline void init(int wave, int lane, unsigned stride_) {
    stride = stride_;
#pragma unroll
    for (int i = 0; i < G::NLD; ++i) {
      const int r = row(wave, lane, i);
      off[i] = (unsigned)r * stride + chunk(lane, r);
    }
  }
  // Rows past `avail` (>= 1) are replaced by the last valid one; the caller masks them.
  __device__ inline void load(int wave, int lane, const unsigned char* base, int avail, unsigned lds) const {
    const unsigned at = __builtin_amdgcn_readfirstlane(lds + wave * (G::NLD * 1024));
    if (avail >= kRows) {
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
  unsigned cols[2];                              // bf16: columns, rows 0-7 and 8-15 of a contraction step of 16; fp32: rows e and e + 8
  __device__ inline void init(int lane, unsigned tile) {
    const int lam = lane & 31, h = lane >> 5;
    rows = tile + lam * G::ROWB + ((h ^ swz<T, D>(lam)) << 4);
    if (sizeof(T) == 2) {
      // lane j of a 16-lane group points at 4 channels of row j / 4 and receives channel j of the group's four rows
      const int j = lane & 15, kq = 4 * h + (j >> 2), lhalf = (lane >> 4) & 1;
#pragma unroll
      for (int u = 0; u < 2; ++u)
        cols[u] = tile + (kq + 8 * u) * G::ROWB + (((2 * lhalf + ((j & 3) >> 1)) ^ swz<T, D>(kq + 8 * u)) << 4) + 8 * (j & 1);
    } else {
      cols[0] = tile + 4 * h * G::ROWB + (lam & 3) * 4;
      cols[1] = (unsigned)(lam >> 2);
    }
  }
};

template <typename V> __device__ inline V lds_read(unsigned at) {
  return *reinterpret_cast<LDS_PTR(const V)>((LDS_PTR(const unsigned char))(unsigned long long)at);
}

// One contraction step over channels (32 bytes of each row): acc += A B.
template <typename T> __device__ inline f32x16 mma_step(u32x4 a, u32x4 b, f32x16 acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
    return acc;
  }
}

// acc = (32 rows of the tile, from row ROW0) * (the lane's own row, all channels).  OFF: byte offset of the tile.
template <typename T, int D, int ROW0>
__device__ inline f32x16 rows_times(const Reader<T, D>& rd, unsigned off, const u32x4 (&b)[Geo<T, D>::STEPS]) {
  f32x16 acc = (f32x16){0};
#pragma unroll
  for (int s = 0; s < Geo<T, D>::STEPS; ++s)
    acc = mma_step<T>(lds_read<u32x4>((rd.rows ^ (s << 5)) + off + ROW0 * Geo<T, D>::ROWB), b[s], acc);
  return acc;
}

__device__ inline unsigned pack_bf16(float lo, float hi) {
  f32x2 f = {lo, hi};
  bf16x2 b = __builtin_convertvector(f, bf16x2);
  return __builtin_bit_cast(unsigned, b);
}

// 32 rows' worth of a lane's values as the B operand of the product that contracts over those rows.
template <typename T> struct Weights;
template <> struct Weights<__bf16> {
  u32x4 w[2];
  __device__ inline void set(int r, float a, float b) { w[r >> 3][(r & 7) >> 1] = pack_bf16(a, b); }    // rows r, r + 1 (r even)
};
template <> struct Weights<float> {
  f32x16 w;
  __device__ inline void set(int r, float a, float b) {
    w[r] = a;
    w[r + 1] = b;
  }
};

// acc[dt] += (32 rows of the tile, from row ROW0)^T (channels x rows) * weights (rows x the lane's column).
template <typename T, int D, int ROW0>
__device__ inline void cols_times(const Reader<T, D>& rd, unsigned off, const Weights<T>& p, f32x16 (&acc)[Geo<T, D>::NDT]) {
  constexpr int ROWB = Geo<T, D>::ROWB;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int dt = 0; dt < Geo<T, D>::NDT; ++dt) {
        const unsigned at = off + (ROW0 + 16 * s) * ROWB;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            reinterpret_cast<LDS_PTR(s16x4)>((LDS_PTR(unsigned char))(unsigned long long)((rd.cols[0] ^ (dt << 6)) + at)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            reinterpret_cast<LDS_PTR(s16x4)>((LDS_PTR(unsigned char))(unsigned long long)((rd.cols[1] ^ (dt << 6)) + at)));
        const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
        const u32x4 a = {l2.x, l2.y, h2.x, h2.y};
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, p.w[s]), acc[dt],
                                                          0, 0, 0);
      }
  } else {
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int base = (r / 4) * 8 + r % 4;      // this lane reads row base + 4 h
      const unsigned z = (unsigned)(swz<T, D>(base) ^ (h << 3));       // swz(base + 4 h): bit 2 of the row is bit 3 of the swizzle
#pragma unroll
      for (int dt = 0; dt < Geo<T, D>::NDT; ++dt) {
        const float a = lds_read<float>(rd.cols[0] + off + (ROW0 + base) * ROWB + (((8 * dt + rd.cols[1]) ^ z) << 4));
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p.w[r], acc[dt], 0, 0, 0);
      }
    }
  }
}

// exp of a difference of scores.  Scores are kept in the log2 domain in bf16 (the exponent is one fused operation) and in the
// natural one in fp32, where the rounded constant would cost the last digits: z - m is one fused operation on the raw
// product, small where the weight is not, and only then multiplied.
template <typename T> __device__ inline float exp_diff(float s, float c, float minus_m) {
  if (sizeof(T) == 2) return __builtin_amdgcn_exp2f(fmaf(s, c, minus_m));
  return __builtin_amdgcn_exp2f(fmaf(s, c, minus_m) * kLog2e);
}
template <typename T> __device__ inline float exp_of(float x) { return __builtin_amdgcn_exp2f(sizeof(T) == 2 ? x : x * kLog2e); }
// log of a sum of weights in that domain, and its way to the natural one
template <typename T> __device__ inline float log_sum(float m, float l) {
  return sizeof(T) == 2 ? (m + __builtin_amdgcn_logf(l)) * kLn2 : m + logf(l);
}

__device__ inline float max_of(const f32x16& s) {
  float t = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) t = fmaxf(t, s[r]);
  return t;
}

// tanh.  bf16 paths: from one exponential and one reciprocal, absolute error about 1e-7.
template <typename T> __device__ inline float tanh_of(float x) {
  if (sizeof(T) == 4) return tanhf(x);
  return fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * (2.f * kLog2e)) + 1.f), 1.f);
}

// Non-finite elements of a staged tile are set to 0, and the rows they were in marked in bad[0..1] (64 bits, zero before).  A
// product contracts over all rows of a tile, also where the weight is 0, and 0 * inf is NaN: tiles that are masked in part are
// cleaned first.  All 256 threads; a barrier before and after is the caller's.
template <typename T, int D> __device__ inline void clean_tile(LDS_PTR(unsigned char) stage, LDS_PTR(unsigned) bad, int tid) {
  using G = Geo<T, D>;
#pragma unroll
  for (int i = 0; i < G::TILEB / 4096; ++i) {
    const int at = (i * 256 + tid) * 16;
    LDS_PTR(u32x4) p = reinterpret_cast<LDS_PTR(u32x4)>(stage + at);
    u32x4 w = *p;
    unsigned found = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (sizeof(T) == 2) {
        if ((w[e] & 0x7f80u) == 0x7f80u) {
          w[e] &= 0xffff0000u;
          found = 1;
        }
        if ((w[e] & 0x7f800000u) == 0x7f800000u) {
          w[e] &= 0xffffu;
          found = 1;
        }
      } else if ((w[e] & 0x7f800000u) == 0x7f800000u) {
        w[e] = 0u;
        found = 1;
      }
    }
    if (found) {
      *p = w;
      const int r = at / G::ROWB;
      atomicOr((unsigned*)(bad + (r >> 5)), 1u << (r & 31));
    }
  }
}

}  // namespace tile
}  // namespace pisa

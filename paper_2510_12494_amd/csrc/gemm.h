// The matrix-product core of the class head and of products in 8 bits on
// gfx950: C = A B^T of two operands whose rows are contiguous along the sum.
//
// A workgroup of WR x WC wavefronts owns a BM x BN tile.  The sum runs in steps
// of KB bytes of every row: a step's (BM + BN) * KB bytes are copied from
// global memory straight into one of NST buffers in LDS (16 bytes a lane), NST - 1
// steps ahead, with one barrier a step.  What a step holds depends on the type
// alone (128 bytes: 128 e4m3 values, 64 bf16 or 32 float32), so all types share
// the tile, its copies and its reads.
//
// A fragment is 16 rows of an operand; lane l holds 16-byte chunks l / 16 and
// l / 16 + 4 of row l % 16.  The sum may be taken in any order as long as A and
// B agree, so a chunk's elements go to one MFMA (bf16: 16x16x32), to four
// (float32: 16x16x4, an element each), or both chunks to one (e4m3: 16x16x128
// with a power of two for each block of 128).  That instruction adds consecutive
// products by eights, cut off 13 bits below the power of two of the largest one, and
// these sums to each other and the result as float32: off by 7 2^-13 of the magnitudes'
// sum at most, where a large product cancels beside small ones, and 1.5e-5 of the norm
// over ordinary ones whatever the length of the sum (256 and 4096 squared, 128 to 8192
// long), 1 / 100 of what rounding them to bf16 adds.  kE4m3Wide makes bf16 of the values,
// powers and all, and takes the bf16 instruction at half the rate, whose sums are float32
// ones; what lies past either end of bf16 goes by parts (EndsPart).
//
// LDS holds a fragment's rows together, chunk c of its row i at place
// c ^ swizzle(i): 16 lanes read 256 consecutive bytes in some order, without bank
// conflicts, while a copy writes lane after lane.  Which rows of the tile make
// up a fragment is free: columns are dealt to groups of DN = 4 fragments (fewer
// where a wavefront has fewer) in turn (fragment f, row i: DN i + f), so a lane's
// results of a group are DN consecutive columns and are stored at once; rows
// likewise (kDealt), or in blocks of 4 DM with four consecutive ones from each
// fragment (kBlocks), so that a lane has 4 DM consecutive rows of a column and can
// also store the transpose.
#pragma once
#include <utility>

#include "device.h"

namespace vfl {
namespace gemm {

using namespace dev;

enum Type { kE4m3, kE4m3Wide, kBf16, kF32 };
__host__ __device__ constexpr bool is_e4m3(Type t) { return t == kE4m3 || t == kE4m3Wide; }
enum Rows { kDealt, kBlocks };

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((address_space(3))) void lds_t;

// wait until at most n of this wavefront's vector-memory operations and none
// of its LDS operations are outstanding
template <int N>
__device__ __forceinline__ void wait_copies() {
  static_assert(N >= 0 && N < 64);
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

// wait until none of this wavefront's LDS operations is outstanding
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt((15) | (3 << 14) | (7 << 4)); }

// Sixteen e4m3 values times their power of two, whose exponent is s's low byte, as bf16:
// the conversion takes the power as a float32, whose exponent lies 23 bits up.
__device__ __forceinline__ void widen_e4m3(const u32x4& v, uint32_t s, bf16x8 (&out)[2]) {
  const float power = __uint_as_float((s & 255u) << 23);
  u32x4 w[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i / 2][2 * (i % 2)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], power, false));
    w[i / 2][2 * (i % 2) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], power, true));
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) out[t] = __builtin_bit_cast(bf16x8, w[t]);
}

// bf16 has every e4m3 value times the power of a byte from 3 (whose smallest magnitude is
// 2^-9 2^-124) to 246 (448 2^119 the largest).  A block of another power has its values
// moved by 2^64 towards 1 and those that they meet by as much the other way, one part of
// the rows and columns after the other, each pair in one part:
//   rows, columns:  between, between 0;  low, all +64;  high, all -64;  between, low -64;
//                   between, high +64
// What then leaves the bytes 0 to 246 is held there: its products are below 2^-149 or past
// float32 either way.
constexpr uint32_t kLowByte = 3, kHighByte = 246;
__device__ __forceinline__ bool at_an_end(uint32_t byte) { return byte - kLowByte > kHighByte - kLowByte; }
// whether one of four bytes may be such a one: those from 64 to 191, whose two highest
// bits differ, are not
__device__ __forceinline__ bool maybe_at_an_end(uint32_t four) {
  return ((four ^ (four << 1)) & 0x80808080u) != 0x80808080u;
}
// bits of sixteen values whose power is such a one; none of kMagnitudes: zeros
constexpr uint32_t kMagnitudes = 0x7f7f7f7fu;
__device__ __forceinline__ uint32_t bits_at_an_end(const u32x4& v, uint32_t byte) {
  return (v[0] | v[1] | v[2] | v[3]) & (at_an_end(byte) ? ~0u : 0u);
}
constexpr int kEndsParts = 5;
struct EndsPart {
  enum Take { kBetween, kLow, kHigh, kAll };
  int rows, columns, by;
  __device__ explicit EndsPart(int i)
      : rows(i == 1 ? kLow : i == 2 ? kHigh : kBetween),
        columns(i == 0 ? kBetween : i == 3 ? kLow : i == 4 ? kHigh : kAll),
        by(i == 0 ? 0 : i == 1 || i == 4 ? 64 : -64) {}
  __device__ static __forceinline__ void widen(const u32x4& v, uint32_t byte, int take, int by, bf16x8 (&out)[2]) {
    const int is = byte < kLowByte ? kLow : byte > kHighByte ? kHigh : kBetween;
    const bool in = take == kAll || take == is;
    widen_e4m3(in ? v : u32x4{0u, 0u, 0u, 0u}, (uint32_t)min(max((int)byte + by, 0), (int)kHighByte), out);
  }
};

// An operand: rows of ld bytes, `last` the last row's index; rows past it are
// read as that row (their results are not kept).  8-bit operands: the exponent
// bytes of step s at scale + s * scale_ld + row, in dwords of four rows.
struct Operand {
  const char* p;
  int64_t ld;
  int64_t last;
  const uint8_t* scale;
  int64_t scale_ld;
};

template <Type TY, int BM_, int BN_, int WR, int WC, int KB_, int NST_, Rows ROWS = kDealt>
struct Tile {
  static constexpr int BM = BM_, BN = BN_, KB = KB_, NST = NST_;
  static constexpr int kWaves = WR * WC, kThreads = 64 * kWaves;
  static constexpr int WM = BM / WR, WN = BN / WC, MF = WM / 16, NF = WN / 16;
  static constexpr int kStage = (BM + BN) * KB, kLds = NST * kStage;
  static constexpr int kRowsPerCopy = 1024 / KB, kChunks = KB / 16;
  static constexpr int kCopies = kStage / 1024 / kWaves;      // a wavefront's copies of a step
  static constexpr int kHalves = KB / 64;                     // 16-byte chunks a lane reads of a row
  static constexpr int kScales = is_e4m3(TY) ? (MF + NF) / 4 : 0;
  static constexpr int kBytes = is_e4m3(TY) ? 1 : TY == kBf16 ? 2 : 4, kElements = KB / kBytes;
  static_assert(KB == 64 || KB == 128);
  static_assert(!is_e4m3(TY) || KB == 128, "a step of e4m3 is one block of its scales");
  static_assert(kStage % (1024 * kWaves) == 0 && BM * KB % 1024 == 0);
  static constexpr int DM = MF < 4 ? MF : 4, DN = NF < 4 ? NF : 4;      // fragments of a group
  static_assert(MF % DM == 0 && NF % DN == 0);
  static_assert(!is_e4m3(TY) || (DM == 4 && DN == 4), "a dword of exponents is four rows");
  static_assert((NST - 2) * (kCopies + kScales) < 64);

  typedef f32x4 Acc[MF][NF];

  // the row within its group of row i of the group's fragment f
  __device__ static int row_of(int f, int i) {
    return ROWS == kDealt ? DM * i + f : 4 * DM * (i >> 2) + 4 * f + (i & 3);
  }
  __device__ static int col_of(int f, int i) { return DN * i + f; }

  // where in the tile this wavefront's results lie
  int lane, wm, wn;
  __device__ Tile() {
    lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wm = wave / WC * WM;
    wn = wave % WC * WN;
  }
  // tile row of result r (0..3) of row fragment f; first of the DN tile columns of
  // column fragments DN q .. DN q + DN - 1
  __device__ int row(int f, int r) const {
    return wm + 16 * DM * (f / DM) + row_of(f % DM, 4 * (lane >> 4) + r);
  }
  __device__ int col(int q) const { return wn + 16 * DN * q + DN * (lane & 15); }

  // acc += the sum over steps [s0, s1) of A's rows from m0 and B's from n0; s0 < s1
  __device__ void run(const Operand& A, const Operand& B, int64_t m0, int64_t n0, int s0, int s1, char* lds,
                      Acc& acc) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // this lane's source of each of the wavefront's copies: the offset from
    // the tile's first row, or the row that stands for those past the end
    static_assert(BM <= 256 && BN <= 256, "offsets are below 2^32: ld is below 2^24");
    const VFL_GLOBAL char* a0 = glb(A.p) + min(m0, A.last) * A.ld + (int64_t)s0 * KB;
    const VFL_GLOBAL char* b0 = glb(B.p) + min(n0, B.last) * B.ld + (int64_t)s0 * KB;
    uint32_t off[kCopies];
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      const int R = (wave + c * kWaves) * kRowsPerCopy + lane / kChunks;      // its LDS row
      const bool of_a = (wave + c * kWaves) * kRowsPerCopy < BM;              // uniform
      const int rr = of_a ? R : R - BM;
      const int f = rr >> 4, i = rr & 15;
      const int row = of_a ? f / DM * (16 * DM) + row_of(f % DM, i) : f / DN * (16 * DN) + col_of(f % DN, i);
      const int64_t top = of_a ? A.last - min(m0, A.last) : B.last - min(n0, B.last);
      const int swz = KB == 128 ? (i >> 1) & 7 : (i >> 2) & 3;
      off[c] = (uint32_t)(min((int64_t)row, top) * (of_a ? A.ld : B.ld)) + (uint32_t)(((lane % kChunks) ^ swz) * 16);
    }
    auto copy = [&](int s) {                         // step s0 + s
      char* dst = lds + (NST == 2 ? s & 1 : s % NST) * kStage;
#pragma unroll
      for (int c = 0; c < kCopies; ++c) {
        const int blk = wave + c * kWaves;
        const VFL_GLOBAL char* src = (blk * kRowsPerCopy < BM ? a0 : b0) + (int64_t)s * KB;
        __builtin_amdgcn_global_load_lds((VFL_GLOBAL void*)(src + off[c]), (lds_t*)(dst + blk * 1024), 16, 0, 0);
      }
    };
    // e4m3: the exponents of this lane's rows, a dword for four fragments
    uint32_t sa[kScales ? MF / 4 : 1], sb[kScales ? NF / 4 : 1], na[kScales ? MF / 4 : 1], nb[kScales ? NF / 4 : 1];
    const VFL_GLOBAL uint8_t *sa0 = nullptr, *sb0 = nullptr;
    uint32_t soa[kScales ? MF / 4 : 1], sob[kScales ? NF / 4 : 1];
    // the bits of such a dword that are rows' (past the last row lies anything)
    uint32_t ka[kScales ? MF / 4 : 1], kb[kScales ? NF / 4 : 1];
    if constexpr (is_e4m3(TY)) {
      static_assert(ROWS == kDealt, "a dword of exponents is four consecutive rows");
      sa0 = glb(A.scale);
      sb0 = glb(B.scale);
#pragma unroll
      for (int q = 0; q < MF / 4; ++q)
        soa[q] = (uint32_t)min(m0 + wm + 64 * q + 4 * (lane & 15), A.last & ~(int64_t)3);
#pragma unroll
      for (int q = 0; q < NF / 4; ++q)
        sob[q] = (uint32_t)min(n0 + wn + 64 * q + 4 * (lane & 15), B.last & ~(int64_t)3);
      auto rows = [](int64_t last, uint32_t at) { return 0xffffffffu >> (8 * (3 - (int)min(last - at, (int64_t)3))); };
#pragma unroll
      for (int q = 0; q < MF / 4; ++q) ka[q] = rows(A.last, soa[q]);
#pragma unroll
      for (int q = 0; q < NF / 4; ++q) kb[q] = rows(B.last, sob[q]);
    }
    auto scales = [&](int s, uint32_t* da, uint32_t* db) {
      const VFL_GLOBAL uint8_t* pa = sa0 + (int64_t)(s0 + s) * A.scale_ld;
      const VFL_GLOBAL uint8_t* pb = sb0 + (int64_t)(s0 + s) * B.scale_ld;
#pragma unroll
      for (int q = 0; q < MF / 4; ++q) da[q] = *(const VFL_GLOBAL uint32_t*)(pa + soa[q]);
#pragma unroll
      for (int q = 0; q < NF / 4; ++q) db[q] = *(const VFL_GLOBAL uint32_t*)(pb + sob[q]);
    };

    const int n = s1 - s0;
    const int fi = lane & 15, g = lane >> 4;
    const int swz = KB == 128 ? (fi >> 1) & 7 : (fi >> 2) & 3;
    int place[kHalves];
#pragma unroll
    for (int h = 0; h < kHalves; ++h) place[h] = fi * KB + ((g + 4 * h) ^ swz) * 16;

#pragma unroll
    for (int s = 0; s < NST - 1; ++s)
      if (s < n) copy(s);
    if constexpr (is_e4m3(TY)) scales(0, na, nb);
    bool ends = false;
    for (int s = 0; s < n; ++s) {
      // this wavefront's copies of step s have landed, and after the barrier
      // everyone's; everyone has also read step s - 1, whose buffer is next
      if (NST > 2 && s + NST - 2 < n) wait_copies<(NST - 2) * kCopies>();
      else wait_copies<0>();
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (is_e4m3(TY)) {
#pragma unroll
        for (int q = 0; q < MF / 4; ++q) sa[q] = TY == kE4m3Wide ? rows_alone(na[q], ka[q]) : na[q];
#pragma unroll
        for (int q = 0; q < NF / 4; ++q) sb[q] = TY == kE4m3Wide ? rows_alone(nb[q], kb[q]) : nb[q];
        if (s + 1 < n) scales(s + 1, na, nb);
      }
      if (s + NST - 1 < n) copy(s + NST - 1);
      __builtin_amdgcn_sched_barrier(0);
      const char* S = lds + (NST == 2 ? s & 1 : s % NST) * kStage;
      const char* SA = S + wm * KB;
      const char* SB = S + (BM + wn) * KB;
      if constexpr (TY == kE4m3) {
        u32x4 b[NF][2];
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int h = 0; h < 2; ++h) b[f][h] = *(const u32x4*)(SB + f * 16 * KB + place[h]);
#pragma unroll
        for (int f = 0; f < MF; ++f) {
          u32x4 a[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) a[h] = *(const u32x4*)(SA + f * 16 * KB + place[h]);
          mma8(a, b, sa[f / 4], sb, f & 3, acc[f], std::make_integer_sequence<int, NF>{});
        }
      } else if constexpr (TY == kE4m3Wide) {
        ends |= powers_at_an_end(SA, SB, place, sa, sb);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 b[NF][2];
#pragma unroll
          for (int f = 0; f < NF; ++f) widen_e4m3(*(const u32x4*)(SB + f * 16 * KB + place[h]), sb[f / 4] >> (8 * (f & 3)), b[f]);
#pragma unroll
          for (int f = 0; f < MF; ++f) {
            bf16x8 a[2];
            widen_e4m3(*(const u32x4*)(SA + f * 16 * KB + place[h]), sa[f / 4] >> (8 * (f & 3)), a);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int c = 0; c < NF; ++c)
                acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], b[c][t], acc[f][c], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) {
          u32x4 b[NF];
#pragma unroll
          for (int f = 0; f < NF; ++f) b[f] = *(const u32x4*)(SB + f * 16 * KB + place[h]);
#pragma unroll
          for (int f = 0; f < MF; ++f) {
            const u32x4 a = *(const u32x4*)(SA + f * 16 * KB + place[h]);
            if constexpr (TY == kBf16) {
#pragma unroll
              for (int c = 0; c < NF; ++c)
                acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                                    __builtin_bit_cast(bf16x8, b[c]), acc[f][c], 0, 0, 0);
            } else {
#pragma unroll
              for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int c = 0; c < NF; ++c)
                  acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[t]), __uint_as_float(b[c][t]),
                                                                   acc[f][c], 0, 0, 0);
            }
          }
        }
      }
    }
    if constexpr (TY == kE4m3Wide) {
      // values past an end of bf16 in this tile: the sum again, such steps by parts.  Beside
      // the other steps' products these took registers that every sum paid for (4096 cubed:
      // 129 us without parts, 133 so, 246 beside them).
      __syncthreads();
      if (threadIdx.x % 64 == 0) ((uint32_t*)lds)[wave] = ends;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWaves; ++w) ends |= ((const uint32_t*)lds)[w] != 0;
      if (!__any(ends)) return;
#pragma unroll
      for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int c = 0; c < NF; ++c) acc[f][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int s = 0; s < n; ++s) {
        __syncthreads();
        copy(s);
        scales(s, sa, sb);
#pragma unroll
        for (int q = 0; q < MF / 4; ++q) sa[q] = rows_alone(sa[q], ka[q]);
#pragma unroll
        for (int q = 0; q < NF / 4; ++q) sb[q] = rows_alone(sb[q], kb[q]);
        wait_copies<0>();
        __syncthreads();
        const char* S = lds + (NST == 2 ? s & 1 : s % NST) * kStage;
        mma_in_parts(S + wm * KB, S + (BM + wn) * KB, place, sa, sb, acc);
      }
    }
  }

  static constexpr uint32_t kOnes = 127 * 0x01010101u;        // powers of 1
  __device__ static __forceinline__ uint32_t rows_alone(uint32_t four, uint32_t keep) {
    return (four & keep) | (kOnes & ~keep);
  }
  // kE4m3Wide: whether a step has values whose powers take them past an end of bf16 (blocks
  // of zeros, whose power is the smallest one, have none); the same in every lane
  __device__ static __forceinline__ bool powers_at_an_end(const char* SA, const char* SB, const int (&place)[kHalves],
                                                          const uint32_t* sa, const uint32_t* sb) {
    bool maybe = false;
#pragma unroll
    for (int q = 0; q < MF / 4; ++q) maybe |= maybe_at_an_end(sa[q]);
#pragma unroll
    for (int q = 0; q < NF / 4; ++q) maybe |= maybe_at_an_end(sb[q]);
    if (!__any(maybe)) return false;
    asm volatile("" ::: "memory");                   // what is read here is not kept for the products
    uint32_t is = 0;
    auto look = [&](const char* S, uint32_t byte) {
#pragma unroll
      for (int h = 0; h < kHalves; ++h) is |= bits_at_an_end(*(const u32x4*)(S + place[h]), byte);
    };
#pragma unroll
    for (int f = 0; f < MF; ++f) look(SA + f * 16 * KB, (sa[f / 4] >> (8 * (f & 3))) & 255u);
#pragma unroll
    for (int f = 0; f < NF; ++f) look(SB + f * 16 * KB, (sb[f / 4] >> (8 * (f & 3))) & 255u);
    asm volatile("" ::: "memory");
    return __any((is & kMagnitudes) != 0);
  }
  __device__ static __forceinline__ void mma_in_parts(const char* SA, const char* SB, const int (&place)[kHalves],
                                                      const uint32_t* sa, const uint32_t* sb, Acc& acc) {
    const int parts = powers_at_an_end(SA, SB, place, sa, sb) ? kEndsParts : 1;
#pragma unroll 1
    for (int i = 0; i < parts; ++i) {
      const EndsPart part(i);
      asm volatile("" ::: "memory");                 // a part reads for itself
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        bf16x8 b[NF][2];
#pragma unroll
        for (int f = 0; f < NF; ++f)
          EndsPart::widen(*(const u32x4*)(SB + f * 16 * KB + place[h]), (sb[f / 4] >> (8 * (f & 3))) & 255u, part.columns,
                          -part.by, b[f]);
#pragma unroll
        for (int f = 0; f < MF; ++f) {
          bf16x8 a[2];
          EndsPart::widen(*(const u32x4*)(SA + f * 16 * KB + place[h]), (sa[f / 4] >> (8 * (f & 3))) & 255u, part.rows,
                          part.by, a);
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < NF; ++c)
              acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[t], b[c][t], acc[f][c], 0, 0, 0);
        }
      }
    }
  }

  // one row fragment of e4m3 times every column fragment; the exponent byte of a
  // fragment is its number's within four (an immediate of the instruction)
  template <int... C>
  __device__ static __forceinline__ void mma8(const u32x4 (&a)[2], const u32x4 (&b)[NF][2], uint32_t sa,
                                              const uint32_t* sb, int fa, f32x4 (&acc)[NF],
                                              std::integer_sequence<int, C...>) {
    struct Pair { u32x4 x, y; };
    const i32x8 va = __builtin_bit_cast(i32x8, (Pair{a[0], a[1]}));
    switch (fa) {
#define VFL_ROW_FRAGMENT(F)                                                                                   \
  case F:                                                                                                     \
    ((acc[C] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(                                              \
          va, __builtin_bit_cast(i32x8, (Pair{b[C][0], b[C][1]})), acc[C], 0, 0, F, (int)sa, C & 3,           \
          (int)sb[C / 4])),                                                                                   \
     ...);                                                                                                    \
    break
      VFL_ROW_FRAGMENT(0);
      VFL_ROW_FRAGMENT(1);
      VFL_ROW_FRAGMENT(2);
      VFL_ROW_FRAGMENT(3);
#undef VFL_ROW_FRAGMENT
    }
  }
};

// A matrix [sum x columns] whose rows are single terms of the sum: `chunks` 16-byte
// chunks a row, `last` the last row; what lies past either is read as the last one.
struct SumMajor {
  const char* p;
  int64_t ld;
  int64_t last;
  int chunks;
};

// C^T = A^T B (BOTH) or A^T B^T over the sum: A [sum x m], B [sum x n] or, as
// an Operand, [n x sum].  LDS holds what it is given, 16-byte chunk c of row k at
// place c ^ swizzle(k).  bf16 fragments of a sum-major operand come from transposing
// reads (ds_read_b64_tr_b16: 16 lanes give the addresses of four columns of
// four rows each, and lane i gets column i of the four rows), two for the eight
// terms that a lane of the MFMA holds; float32 ones are read element by element.
// Columns are dealt to D fragments by fours (fragment f, lane i: 4 D (i / 4) + 4 f +
// i % 4), which is what those reads can gather, and leaves a lane 4 D consecutive
// columns of A for each column of B: they are stored at once.
template <Type TY, int BM_, int BN_, int WR, int WC, int KB_, int NST_, bool BOTH>
struct SumTile {
  static constexpr int BM = BM_, BN = BN_, KB = KB_, NST = NST_;
  static constexpr int kWaves = WR * WC, kThreads = 64 * kWaves;
  static constexpr int WM = BM / WR, WN = BN / WC, MF = WM / 16, NF = WN / 16;
  static constexpr int kStage = (BM + BN) * KB, kLds = NST * kStage;
  static constexpr int kBytes = TY == kBf16 ? 2 : 4, kElements = KB / kBytes;   // terms of a step
  static constexpr int kCopies = kStage / 1024 / kWaves, kCopiesA = BM * KB / 1024;
  static constexpr int kHalves = KB / 64;
  static constexpr int D = MF < 4 ? MF : 4, DN = NF < 4 ? NF : 4;
  static_assert(TY == kBf16 || TY == kF32);
  static_assert(D >= 2 && DN >= 2, "the swizzles below");
  static_assert(MF % D == 0 && NF % DN == 0 && kStage % (1024 * kWaves) == 0 && BM * KB % 1024 == 0);
  static_assert(BM * kBytes >= 128 && BN * kBytes >= 128);
  static_assert((NST - 2) * kCopies < 64);
  typedef f32x4 Acc[MF][NF];

  int lane, wm, wn;
  __device__ SumTile() {
    lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wm = wave / WC * WM;
    wn = wave % WC * WN;
  }
  // the first of the 4 D consecutive columns of A that a lane's fragments D q .. hold
  __device__ int a_col(int q) const { return wm + 16 * D * q + 4 * D * (lane >> 4); }
  // the column of B of its fragment f
  __device__ int b_col(int f) const {
    return wn + 16 * DN * (f / DN) + 4 * DN * ((lane & 15) >> 2) + 4 * (f % DN) + (lane & 3);
  }

  // Four rows that are read at once (bf16: consecutive; float32: four apart) lie in
  // different banks: within what a fragment's reads leave free of a row, then in the
  // other half of 256 bytes (a row of 128 has none: two rows meet).  `per`: a row's chunks.
  __device__ static int swizzle(int k, int deal, int per) {
    const int lo = TY == kBf16 ? k & 1 : k >> 2 & 1, hi = TY == kBf16 ? k >> 1 & 1 : k >> 3 & 1;
    if (TY == kF32 && deal == 4) return lo | hi << 1;
    const int at = TY == kBf16 && deal == 2 ? 2 : 0;  // the chunks that eight bytes of each lie in
    return lo << at | (per >= 16 ? hi << 3 : 0);
  }

  __device__ void run(const SumMajor& A, const SumMajor& Bs, const Operand& B, int64_t m0, int64_t n0, int s0, int s1,
                      char* lds, Acc& acc) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // a copy's lane: row `row[c]` of the step (of a sum-major operand) at byte col[c]
    // of it, or the offset of its chunk from the tile's first row
    int row[kCopies];
    int64_t at[kCopies];
    const int64_t b_first = BOTH ? 0 : min(n0, B.last);
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      const int blk = wave + c * kWaves;
      const bool of_a = blk < kCopiesA;                                  // uniform
      if (of_a || BOTH) {
        const int per = (of_a ? BM : BN) * kBytes / 16;                  // chunks of a row
        const int u = (of_a ? blk : blk - kCopiesA) * 64 + lane;         // chunk of the operand's step
        const int k = u / per;
        const int ch = (u % per) ^ swizzle(k, of_a ? D : DN, per);
        const SumMajor& o = of_a ? A : Bs;
        const int64_t chunk = min((of_a ? m0 : n0) * kBytes / 16 + ch, (int64_t)o.chunks - 1);
        row[c] = k;
        at[c] = chunk * 16;
      } else {
        const int R = (blk - kCopiesA) * (1024 / KB) + lane / (KB / 16);
        const int f = R >> 4, i = R & 15;
        const int r = f / DN * (16 * DN) + 4 * DN * (i >> 2) + 4 * (f % DN) + (i & 3);
        const int swz = KB == 128 ? (i >> 1) & 7 : (i >> 2) & 3;
        row[c] = 0;
        at[c] = min((int64_t)r, B.last - b_first) * B.ld + ((lane % (KB / 16)) ^ swz) * 16;
      }
    }
    const VFL_GLOBAL char* const b0 = BOTH ? nullptr : glb(B.p) + b_first * B.ld;
    auto copy = [&](int s) {
      char* dst = lds + (NST == 2 ? s & 1 : s % NST) * kStage;
#pragma unroll
      for (int c = 0; c < kCopies; ++c) {
        const int blk = wave + c * kWaves;
        const bool of_a = blk < kCopiesA;
        const VFL_GLOBAL char* src;
        if (of_a || BOTH) {
          const SumMajor& o = of_a ? A : Bs;
          src = glb(o.p) + min((int64_t)(s0 + s) * kElements + row[c], o.last) * o.ld + at[c];
        } else {
          src = b0 + (int64_t)(s0 + s) * KB + at[c];
        }
        __builtin_amdgcn_global_load_lds((VFL_GLOBAL void*)src, (lds_t*)(dst + blk * 1024), 16, 0, 0);
      }
    };
    const int n = s1 - s0, i = lane & 15, g = lane >> 4;

    // this lane's byte in the sum-major operand of WIDTH columns: fragment f of the
    // wavefront's columns from w; bf16: rows k .. k + 3 by transposing reads
    auto transposed = [&](const char* S, int width, int deal, int w, int f, int k) {
      typedef __attribute__((ext_vector_type(4))) short s16x4;
      const int kk = k + (i >> 2);
      const int col = w + 16 * deal * (f / deal) + 4 * deal * (i & 3) + 4 * (f % deal);
      const int ch = (col / 8) ^ swizzle(kk, deal, width / 8);
      const char* p = S + kk * width * 2 + ch * 16 + (col % 8) * 2;
      return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                           (__attribute__((address_space(3))) s16x4*)p));
    };
    auto element = [&](const char* S, int width, int deal, int w, int f, int k) {
      const int col = w + 16 * deal * (f / deal) + 4 * deal * (i >> 2) + 4 * (f % deal) + (i & 3);
      const int ch = (col / 4) ^ swizzle(k, deal, width / 4);
      return *(const float*)(S + k * width * 4 + ch * 16 + (col % 4) * 4);
    };
    // the 16 bytes of the sum that lane (i, g) holds of a fragment: terms 8 (g + 4 h)
    // of bf16, 4 (g + 4 h) of float32
    auto fragment = [&](const char* S, int width, int deal, int w, int f, int h) {
      u32x4 v;
      if constexpr (TY == kBf16) {
        const u32x2 lo = transposed(S, width, deal, w, f, 8 * (g + 4 * h));
        const u32x2 hi = transposed(S, width, deal, w, f, 8 * (g + 4 * h) + 4);
        v = u32x4{lo[0], lo[1], hi[0], hi[1]};
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = __float_as_uint(element(S, width, deal, w, f, 4 * (g + 4 * h) + t));
      }
      return v;
    };

#pragma unroll
    for (int s = 0; s < NST - 1; ++s)
      if (s < n) copy(s);
    for (int s = 0; s < n; ++s) {
      if (NST > 2 && s + NST - 2 < n) wait_copies<(NST - 2) * kCopies>();
      else wait_copies<0>();
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      if (s + NST - 1 < n) copy(s + NST - 1);
      __builtin_amdgcn_sched_barrier(0);
      const char* S = lds + (NST == 2 ? s & 1 : s % NST) * kStage;
      const char* SB = S + BM * KB;
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        u32x4 b[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          if constexpr (BOTH) b[f] = fragment(SB, BN, DN, wn, f, h);
          else b[f] = *(const u32x4*)(SB + (wn + 16 * f + i) * KB + ((g + 4 * h) ^ (KB == 128 ? (i >> 1) & 7 : (i >> 2) & 3)) * 16);
        }
#pragma unroll
        for (int f = 0; f < MF; ++f) {
          const u32x4 a = fragment(S, BM, D, wm, f, h);
          if constexpr (TY == kBf16) {
#pragma unroll
            for (int c = 0; c < NF; ++c)
              acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                                  __builtin_bit_cast(bf16x8, b[c]), acc[f][c], 0, 0, 0);
          } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int c = 0; c < NF; ++c)
                acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[t]), __uint_as_float(b[c][t]),
                                                                 acc[f][c], 0, 0, 0);
          }
        }
      }
    }
  }
};

// What workgroup `block` of tm x tn tiles and `parts` parts of the sum takes.
// Workgroups are dealt to the eight XCDs in turn, so each XCD takes a contiguous
// range of an order that goes part by part and, in a part, walks bands of eight tile
// rows column by column: what a range reads of both operands meets in one L2
// (1024 x 500 x 32768 in 16 parts: 38 us with the tiles of a part on all XCDs).
struct Place { uint32_t m, n, part; };
__device__ __forceinline__ Place place_of(uint32_t block, uint32_t tm, uint32_t tn, uint32_t parts) {
  const uint32_t tiles = tm * tn, total = tiles * parts, per = total / 8, more = total % 8;
  const uint32_t x = block % 8;
  uint32_t t = x * per + min(x, more) + block / 8;
  Place p;
  p.part = t / tiles;
  t -= p.part * tiles;
  const uint32_t band = t / (8 * tn), in = t - band * 8 * tn, rows = min(8u, tm - 8 * band);
  p.m = 8 * band + in % rows;
  p.n = in / rows;
  return p;
}

}  // namespace gemm
}  // namespace vfl

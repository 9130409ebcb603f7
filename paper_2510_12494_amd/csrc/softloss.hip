// The softmax cross-entropy of a linear head over many classes on gfx950, with its
// gradients, without the logits in memory.
//
//   z = x w^T + bias, lse = log(sum_c exp z), loss = lse - z[label]
//   G = dloss (exp(z - lse) - onehot(label)), dx = G w, dw = G^T x, dbias = sum_r G
//
// Forward: a workgroup makes a tile of logits in registers (gemm.h) and leaves each
// row's largest value and sum of exponentials over the tile's classes; a second
// launch joins the tiles' pairs.  Backward: the classes go in pieces; a tile of
// logits is made again, turned into G in registers and stored once, in the operands'
// type, and two products read it, one along its rows and one along its columns.
//
// Exponentials and sums are taken to base 2 (z log2 e is one multiplication-addition
// with the bias, and the hardware's exponential is to base 2); one below 2^-126 is 0.
// A class whose bias is -inf, and a column past the last class, is out of every sum
// whatever its weights hold; a row without a label has a gradient of 0 whatever its
// input holds.
//
// Of 8192 x 256 bf16 rows over 100000 classes (three products of 2 x 8192 x 256 x 100000
// operations, 0.99 ms at a library product's rate, and the logits once more) a step
// takes 2.27 ms: copies of the operands 18 us, k_strip 442, its pairs joined 5, G 2 x 336,
// both products 2 x 560, what is summed 22 (a run once the clock has settled; within the
// first 20 ms of such load they take up to a quarter more).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ops8.h"
#include "product.h"

namespace vfl {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// what undoes the multiplication by kLog2e as float32 has it, in two parts
constexpr double kUnit = 1.0 / (double)kLog2e;
constexpr float kUnitHigh = (float)kUnit, kUnitLow = (float)(kUnit - (double)kUnitHigh);
constexpr int kThreads = 256;

template <typename T> constexpr int kRow = 128 / (int)sizeof(T);    // elements that operands' rows are padded to

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

// ------------------------------------------------------------------ operands
struct CopyArgs {
  Mat src;
  void* dst;
  int64_t dst_ld, rows;                // elements from row to row
  int64_t wrap;                        // rows of the copy, `rows` and zeros, that it holds twice (0: once, no zeros)
  const int32_t* labels;               // rows without a label are 0 (null: all are kept)
  const float* bias;                   // rows whose bias is -inf are 0
  int64_t classes;
  int cols;
};

// Rows padded with zeros to whole steps of a product, those that must not reach it
// as zeros: eight columns a thread, both matrices in one launch (1537 and 5003 rows of
// 333 float32: 7.3 us, of which the launch is 3; HBM bounds larger ones).
constexpr int kPadGrid = 16384;
template <typename T, Form F>
__device__ __forceinline__ void pad(const CopyArgs& j, uint32_t block) {
  const Cols k(j.cols, j.rows);
  const int per = (int)(j.dst_ld / 8);
  const int64_t chunks = (j.wrap ? 2 * j.wrap : j.rows) * per;
  for (int64_t at = (int64_t)block * kThreads + threadIdx.x; at < chunks; at += (int64_t)kPadGrid * kThreads) {
    const int64_t to = at / per, from = j.wrap && to >= j.wrap ? to - j.wrap : to, r = min(from, j.rows - 1);
    const int q = (int)(at - to * per);
    const bool edge = r >= k.edge;
    float v[8];
    chunk_values<F>(load_chunk<F>(row_of<T>(j.src, r), q, k, edge), q, k, edge, v);
    const bool keep = from < j.rows && (!j.labels || (j.labels[r] >= 0 && j.labels[r] < j.classes)) &&
                      (!j.bias || !(j.bias[r] == -__builtin_inff()));
    if (!keep) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    store8<false>((T*)j.dst + to * j.dst_ld + 8 * q, v);
  }
}
// two matrices of as many columns: the first `split` workgroups take the first one
template <typename T, Form F>
__global__ __launch_bounds__(kThreads) void k_pad(CopyArgs a, CopyArgs b, uint32_t split) {
  if (blockIdx.x < split) pad<T, F>(a, blockIdx.x);
  else pad<T, F>(b, blockIdx.x - split);
}

// -------------------------------------------------------------------- logits
struct LogitArgs {
  Operand w, x;                        // w: from the piece's first class
  const float* bias;                   // [classes] of the piece
  int steps;
  uint32_t tm, tn;                     // tiles of classes and of rows
  int64_t rows, classes;               // classes: left from the piece's first
  const int32_t* labels;
  // forward: [tm][rows] of (largest, sum), and [rows] of the label's logit (null: not kept),
  // to base 2
  f32x2* part;
  float* label_z;
  // backward
  const float *lse, *dloss;
  float scale;
  int64_t rest;                        // rows of G to that of what its rounding leaves (0: none)
  float* label_rest;                   // [rows]: or what the label's rounding leaves (null: not kept)
  int64_t first, all_classes;          // the piece's first class
  void* g;
  int64_t g_ld;
  float* part_bias;                    // [tn][bias_ld], from the piece's first class
  int64_t bias_ld;
};

// Over the four lanes of a wavefront that share lane % 16, in each of them.
__device__ __forceinline__ float quarters_sum(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ __forceinline__ float quarters_top(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// old + sum_t 2^(z_t - from).  A class that is out of every sum (bias -inf) has z =
// -inf, or NaN where its weights are no numbers; a maximum passes over the NaN, and
// a sum that is one is taken again without such classes, instead of a comparison and
// a selection for every logit (8192 x 256 rows, 100000 classes: 540 us with those).
template <int N>
__device__ __forceinline__ float sum_of(const float (&z)[N], const float (&bias)[N], float from, float old) {
  float s = old;
#pragma unroll
  for (int t = 0; t < N; ++t) s += exp2_of(z[t] - from);
  if (__any(s != s)) {
    s = old;
#pragma unroll
    for (int t = 0; t < N; ++t) s += bias[t] == -__builtin_inff() ? 0.f : exp2_of(z[t] - from);
  }
  return s;
}

// The logit of class `hit` of the lane's, where it has that.
template <int N>
__device__ __forceinline__ void keep_label(const float (&z)[N], const float (&bias)[N], uint32_t hit, float* to) {
  if (hit >= (uint32_t)N) return;
  float at = 0.f;
#pragma unroll
  for (int t = 0; t < N; ++t) at = hit == (uint32_t)t ? (bias[t] == -__builtin_inff() ? bias[t] : z[t]) : at;
  *to = at;
}

// LDS of a tile: the copies, then the biases of its classes and three words a row, each in
// whole wavefronts' copies.
template <class TL>
constexpr int row_words() { return TL::BN < 64 ? 64 : TL::BN; }
template <class TL>
constexpr int logits_lds() { return TL::kLds + 4 * TL::BM + 12 * row_words<TL>(); }

// A tile of classes x rows: with the classes as the MFMA's rows a lane holds 16
// consecutive classes (4 DM in general) of each of its batch rows, so a row's
// largest value and sum are mostly over a lane's own registers, what G needs of a
// row is loaded once a lane, and G is stored 16 bytes at a time.  The matrix cores and
// then the vector units bound it, which overlap only between workgroups: two a CU and
// tiles of 256 x 128 where rows are short (G of 8192 x 256 rows and 50176 classes: 360
// us, 585 TFLOP/s with an exponential a logit and 0.8 GB of G written), one of 256 x
// 256 where they are long (8192 x 1024 rows over 16000 classes, forward: 1.11 PFLOP/s).  float32:
// 1537 x 333 rows over 5003 classes 60 us, 85 TFLOP/s of 154; a library's product
// alone takes 62 there.
template <class TL, typename T, bool GRAD>
__global__ __launch_bounds__(TL::kThreads) void k_logits(LogitArgs j) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int WC = TL::BN / TL::WN, WR = TL::BM / TL::WM, RUN = 4 * TL::DM;
  static_assert(TL::MF == TL::DM, "a lane's classes are one run");
  static_assert(WR * TL::BN * 8 <= TL::kLds && WC * TL::BM * 4 <= TL::kLds);
  const Place at = place_of(blockIdx.x, j.tm, j.tn, 1);
  const uint32_t tm = at.m, tn = at.n;
  const TL tile;
  const int64_t c0 = (int64_t)tm * TL::BM, r0 = (int64_t)tn * TL::BN;
  const int64_t mine = c0 + tile.row(0, 0);

  // What the end of the tile needs is copied into LDS beside its first operands: to
  // load it after the products would add two latencies to every tile, to keep it in
  // registers would take workgroups off the CU.
  float* const e_bias = (float*)(smem + TL::kLds);   // [BM]
  constexpr int WORDS = row_words<TL>();
  int* const e_label = (int*)(e_bias + TL::BM);      // [BN], and lse, dloss
  float *const e_lse = (float*)(e_label + WORDS), *const e_d = e_lse + WORDS;
  {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    auto fetch = [&](const void* src, int64_t at, int64_t last, void* dst) {
      __builtin_amdgcn_global_load_lds((VFL_GLOBAL void*)(glb((const float*)src) + min(at, last)), (lds_t*)dst, 4, 0, 0);
    };
    constexpr int NB = TL::BM / 64, NR = WORDS / 64, KINDS = GRAD ? 3 : 1;
#pragma unroll
    for (int n = 0; n < (NB + KINDS * NR + TL::kWaves - 1) / TL::kWaves; ++n) {
      const int i = wave + n * TL::kWaves;
      if (i < NB) {
        if (j.bias) fetch(j.bias, c0 + 64 * i + tile.lane, j.classes - 1, e_bias + 64 * i);
      } else if (i < NB + KINDS * NR) {
        const int k = 64 * ((i - NB) % NR);
        const int64_t row = r0 + k + tile.lane;
        if (i < NB + NR) {
          if (GRAD || j.label_z) fetch(j.labels, row, j.rows - 1, e_label + k);
        } else if (i < NB + 2 * NR) fetch(j.lse, row, j.rows - 1, e_lse + k);
        else if (j.dloss) fetch(j.dloss, row, j.rows - 1, e_d + k);
      }
    }
  }

  typename TL::Acc acc;
#pragma unroll
  for (int f = 0; f < TL::MF; ++f)
#pragma unroll
    for (int c = 0; c < TL::NF; ++c) acc[f][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  tile.run(j.w, j.x, c0, r0, 0, j.steps, smem, acc);
  __syncthreads();                                   // the copies' buffers are free

  // the biases of the lane's classes to base 2; -inf: out of every sum
  float bias[RUN];
#pragma unroll
  for (int t = 0; t < RUN; t += 4) {
    const f32x4 b = j.bias ? *(const f32x4*)(e_bias + (int)(mine - c0) + t) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bias[t + i] = mine + t + i < j.classes ? b[i] * kLog2e : -__builtin_inff();
    }
  }

  if constexpr (!GRAD) {
    f32x2* const stat = (f32x2*)smem;                // [WR][BN]
#pragma unroll
    for (int c = 0; c < TL::NF; ++c) {
      float z[RUN], top = -__builtin_inff();
#pragma unroll
      for (int t = 0; t < RUN; ++t) z[t] = fmaf(acc[t / 4][c][t % 4], kLog2e, bias[t]);
#pragma unroll
      for (int t = 0; t < RUN; ++t) top = fmaxf(top, z[t]);
      top = quarters_top(top);
      const float from = top == -__builtin_inff() ? 0.f : top;
      const float sum = quarters_sum(sum_of(z, bias, from, 0.f));
      if (j.label_z) {
        const int in = tile.col(c / TL::DN) + c % TL::DN;
        if (r0 + in < j.rows) keep_label(z, bias, (uint32_t)e_label[in] - (uint32_t)mine, j.label_z + r0 + in);
      }
      if (tile.lane < 16) stat[tile.wm / TL::WM * TL::BN + tile.col(c / TL::DN) + c % TL::DN] = f32x2{top, sum};
    }
    __syncthreads();
    for (int i = threadIdx.x; i < TL::BN; i += TL::kThreads) {
      if (r0 + i >= j.rows) continue;
      f32x2 s = stat[i];
#pragma unroll
      for (int w = 1; w < WR; ++w) {
        const f32x2 o = stat[w * TL::BN + i];
        const float top = fmaxf(s[0], o[0]), from = top == -__builtin_inff() ? 0.f : top;
        s = f32x2{top, s[1] * exp2_of(s[0] - from) + o[1] * exp2_of(o[0] - from)};
      }
      j.part[(int64_t)tm * j.rows + r0 + i] = s;
    }
  } else {
    float total[RUN];
#pragma unroll
    for (int t = 0; t < RUN; ++t) total[t] = 0.f;
#pragma unroll
    for (int c = 0; c < TL::NF; ++c) {
      const int in = tile.col(c / TL::DN) + c % TL::DN;
      const int64_t row = r0 + in;
      // a row without a label, past the last row, or without any class: every
      // exponential is 0; hit: the label among the lane's classes
      const int label = e_label[in];
      const float lse = e_lse[in];
      const bool has = row < j.rows && label >= 0 && label < j.all_classes;
      const float lse2 = has && !(lse == -__builtin_inff()) ? lse * kLog2e : __builtin_inff();
      const float d = has ? (j.dloss ? e_d[in] : j.scale) : 0.f;
      // what rounding lse2 loses, as a factor of the row's exponentials
      const float low = fabsf(lse2) < __builtin_inff() ? fmaf(lse, kLog2e, -lse2) : 0.f, dp = fmaf(-low * kLn2, d, d);
      const int hit = has ? label - (int)(j.first + mine) : -1;
      float g[RUN];
#pragma unroll
      for (int t = 0; t < RUN; ++t) g[t] = 0.f;
      if (has) {                                     // whatever the weights hold
#pragma unroll
        for (int t = 0; t < RUN; ++t) g[t] = dp * exp2_of(fmaf(acc[t / 4][c][t % 4], kLog2e, bias[t]) - lse2);
      }
      if ((unsigned)hit < (unsigned)RUN) {
#pragma unroll
        for (int t = 0; t < RUN; ++t) g[t] -= hit == t && !(bias[t] == -__builtin_inff()) ? d : 0.f;
        if constexpr (sizeof(T) == 2) {
          if (j.label_rest) {
            float at = 0.f;
#pragma unroll
            for (int t = 0; t < RUN; ++t) at = hit == t ? g[t] : at;
            j.label_rest[row] = at - __uint_as_float(pack_bf16(at, 0.f) << 16);
          }
        }
      }
#pragma unroll
      for (int t = 0; t < RUN; ++t) total[t] += g[t];
      T* const to = (T*)j.g + row * j.g_ld + mine;
      if (sizeof(T) == 2 && j.rest && row >= j.rest) continue;   // where a second term lies
#pragma unroll
      for (int t = 0; t < RUN; t += 8) {
        if constexpr (RUN == 4) {
          store4(to, g);
          break;
        }
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = g[(t + i) % RUN];
        store8<false>(to + t, v);
        if constexpr (sizeof(T) == 2) {
          if (j.rest) {
            float w[8];
            Raw<uint16_t> stored;
            stored.a = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
            unpack(stored, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = v[i] - w[i];
            store8<false>(to + j.rest * j.g_ld + t, w);
          }
        }
      }
    }
    if (j.part_bias) {
      float* const sums = (float*)smem;              // [WC][BM]
#pragma unroll
      for (int t = 0; t < RUN; ++t) total[t] = group_sum<16>(total[t]);
      if ((tile.lane & 15) == 0) {
#pragma unroll
        for (int t = 0; t < RUN; ++t) sums[tile.wn / TL::WN * TL::BM + tile.row(0, 0) + t] = total[t];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < TL::BM; i += TL::kThreads) {
        float t = sums[i];
#pragma unroll
        for (int w = 1; w < WC; ++w) t += sums[w * TL::BM + i];
        j.part_bias[(int64_t)tn * j.bias_ld + c0 + i] = t;
      }
    }
  }
}

// The forward of rows of up to 256 columns in bf16 (KP panels of 64) over many classes: a
// workgroup keeps the fragments of 256 rows in registers and walks a strip of tiles of
// 128 classes, whose weights alone go through LDS.  Two groups of four wavefronts, one of
// each on a SIMD, take the halves of a tile half a turn apart: one group's products
// run in the matrix cores while the other's exponentials run in the vector units.
// A barrier ends each phase; a tile's weights are copied two phases ahead.  A lane
// carries the largest value and the sum of its own classes from tile to tile, so
// nothing crosses lanes before the strip's end.  8192 x 256 rows, 100000 classes: 449
// us, 600 in tiles (a matrix and a vector instruction do not quite overlap: halves of
// the wavefronts doing one each take 0.77 of the sum of the times); 16384 classes, 16
// tiles a workgroup, 92 and 93.
struct StripArgs {
  Operand w, x;
  const float* bias;
  int64_t rows, classes;
  f32x2* part;                         // [2 strips][rows] of (largest, sum), to base 2
  int tiles, strips;
};
constexpr int kStripRows = 256, kStripClasses = 128;
template <int KP>
constexpr int strip_lds() { return 2 * KP * 16384 + 4 * kStripClasses * 4; }

template <int KP>
__global__ __launch_bounds__(512) void k_strip(StripArgs j) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  float* const e_bias = (float*)(smem + 2 * KP * 16384);            // [4 tiles][128]
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave >> 2, rw = wave & 3;
  const uint32_t strip = blockIdx.x % (uint32_t)j.strips, block = blockIdx.x / (uint32_t)j.strips;
  const int t0 = (int)((int64_t)j.tiles * strip / j.strips), n = (int)((int64_t)j.tiles * (strip + 1) / j.strips) - t0;
  const int64_t row0 = (int64_t)block * kStripRows + 64 * rw + 4 * i;   // the lane's rows: row0 .. row0 + 3

  // a copy's lane: class `at` of the tile's half, byte `byte` of its panel (the
  // layout of gemm.h: rows in blocks, places swizzled)
  const int R = 8 * wave + (lane >> 3), ri = R & 15;
  const int at = 16 * (ri >> 2) + 4 * (R >> 4) + (ri & 3);
  const int byte = ((lane & 7) ^ ((ri >> 1) & 7)) * 16;
  auto copy = [&](int t) {                           // tile t0 + t
    const int64_t c0 = (int64_t)(t0 + t) * kStripClasses;
    char* const dst = smem + (t & 1) * (KP * 16384) + wave * 1024;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const VFL_GLOBAL char* src = glb(j.w.p) + min(c0 + 64 * h + at, j.w.last) * j.w.ld + byte;
#pragma unroll
      for (int p = 0; p < KP; ++p)
        __builtin_amdgcn_global_load_lds((VFL_GLOBAL void*)(src + 128 * p), (lds_t*)(dst + p * 16384 + h * 8192), 16, 0, 0);
    }
    if (j.bias && rw < 2 && group == 0)
      __builtin_amdgcn_global_load_lds(
          (VFL_GLOBAL void*)(glb(j.bias) + min(c0 + 64 * rw + lane, j.classes - 1)),
          (lds_t*)(e_bias + (t & 3) * kStripClasses + 64 * rw), 4, 0, 0);
  };
  copy(0);

  bf16x8 x[2 * KP][4];
  float top[4], sum[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const VFL_GLOBAL char* const src = glb(j.x.p) + min(row0 + c, j.x.last) * j.x.ld + 16 * g;
#pragma unroll
    for (int k = 0; k < 2 * KP; ++k) x[k][c] = __builtin_bit_cast(bf16x8, *(const VFL_GLOBAL u32x4*)(src + 64 * k));
    top[c] = -__builtin_inff();
    sum[c] = 0.f;
  }

  // Group 0 is in its products of tile t in phase 2 t and in its exponentials in phase
  // 2 t + 1, group 1 a phase later.  Tile t + 1's buffer was last read in phase 2 t - 1:
  // each group copies its share at the start of phase 2 t and waits for it at the
  // end of phase 2 t + 1.
  const int mine_at = (64 * group + i) * 128, swz = (i >> 1) & 7;
  wait_copies<0>();
  __builtin_amdgcn_s_barrier();
  if (group == 1) {
    if (n > 1) copy(1);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
  }
  for (int t = 0; t < n; ++t) {
    if (group == 0 && t + 1 < n) copy(t + 1);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 acc[4][4];
    const char* const S = smem + (t & 1) * (KP * 16384) + mine_at;
    // fragments of the weights are read a step ahead of their products: one
    // wavefront a SIMD is in this phase, and nothing else would hide the reads
    bf16x8 a[2][4];
    auto read = [&](int k) {
#pragma unroll
      for (int f = 0; f < 4; ++f)
        a[k & 1][f] = *(const bf16x8*)(S + (k >> 1) * 16384 + f * 2048 + ((g + 4 * (k & 1)) ^ swz) * 16);
    };
    read(0);
#pragma unroll
    for (int k = 0; k < 2 * KP; ++k) {
      if (k + 1 < 2 * KP) read(k + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          acc[f][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[k & 1][f], x[k][c], k ? acc[f][c] : f32x4{0.f, 0.f, 0.f, 0.f},
                                                              0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (group == 1) wait_copies<0>();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (group == 1 && t + 2 < n) copy(t + 2);
    __builtin_amdgcn_sched_barrier(0);

    const int mine = 64 * group + 16 * g;            // the lane's 16 classes
    const int64_t c0 = (int64_t)(t0 + t) * kStripClasses + mine;
    float bias[16];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 b = *(const f32x4*)(e_bias + (t & 3) * kStripClasses + mine + 4 * q);
#pragma unroll
      for (int u = 0; u < 4; ++u) bias[4 * q + u] = j.bias ? b[u] * kLog2e : 0.f;
    }
    if (c0 + 16 > j.classes) {
#pragma unroll
      for (int u = 0; u < 16; ++u) bias[u] = c0 + u < j.classes ? bias[u] : -__builtin_inff();
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float z[16], now = top[c];
#pragma unroll
      for (int u = 0; u < 16; ++u) z[u] = fmaf(acc[u / 4][c][u % 4], kLog2e, bias[u]);
#pragma unroll
      for (int u = 0; u < 16; ++u) now = fmaxf(now, z[u]);
      const float from = now == -__builtin_inff() ? 0.f : now, old = sum[c] * exp2_of(top[c] - from);
      sum[c] = sum_of(z, bias, from, old);
      top[c] = now;
    }
    __builtin_amdgcn_sched_barrier(0);
    if (group == 0) wait_copies<0>();
    else wait_lds();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  }
  if (group == 0) __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float all = quarters_top(top[c]), from = all == -__builtin_inff() ? 0.f : all;
    const float s = quarters_sum(sum[c] * exp2_of(top[c] - from));
    if (g == 0 && row0 + c < j.rows) j.part[(int64_t)(2 * strip + group) * j.rows + row0 + c] = f32x2{all, s};
  }
}

// ---------------------------------------------------------------------- join
struct FinishArgs {
  const f32x2* part;
  const float* label_z;
  Operand x, w;                        // after strips, and the biases
  const float* bias;
  const int32_t* labels;
  float *loss, *lse;
  int64_t rows, classes, tiles;
};

// A row a group of 16 lanes: the tiles' pairs joined, and the loss as the sum of two
// differences of what the tiles saw, both 0 or more: where the label has the largest
// logit the first is 0, whatever the logits' own rounding.  After strips (KP panels of
// 64 columns), whose registers have no room for labels, a wavefront makes the labels'
// logits of the 16 rows again, by the same instructions in the same order: the same bits.
// Latency bounds it: 3 to 5 us.
template <int KP>
__global__ __launch_bounds__(kThreads) void k_loss(FinishArgs j) {
  constexpr int kRows = kThreads / 16;
  const int lane = threadIdx.x & 15, in = threadIdx.x >> 4;
  const int64_t row = (int64_t)blockIdx.x * kRows + in;
  __shared__ float logits[kRows];
  if constexpr (KP > 0) {
    if (threadIdx.x < 64 && j.loss) {
      const int64_t r = min((int64_t)blockIdx.x * kRows + lane, j.rows - 1);
      const int label = j.labels[r];
      const int64_t c = label >= 0 && label < j.classes ? label : 0;
      const VFL_GLOBAL char* const x = glb(j.x.p) + r * j.x.ld + 16 * in;
      const VFL_GLOBAL char* const w = glb(j.w.p) + c * j.w.ld + 16 * in;
      const float b = j.bias ? j.bias[c] : 0.f;
      bf16x8 wf[2 * KP], xf[2 * KP];
#pragma unroll
      for (int k = 0; k < 2 * KP; ++k) {
        wf[k] = __builtin_bit_cast(bf16x8, *(const VFL_GLOBAL u32x4*)(w + 64 * k));
        xf[k] = __builtin_bit_cast(bf16x8, *(const VFL_GLOBAL u32x4*)(x + 64 * k));
      }
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 2 * KP; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[k], xf[k], acc, 0, 0, 0);
      // a lane has classes 4 in .. 4 in + 3 of row `lane`: its own is among them in one
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (lane == 4 * in + t) logits[lane] = b == -__builtin_inff() ? b : fmaf(acc[t], kLog2e, b * kLog2e);
    }
    __syncthreads();
  }
  if (row >= j.rows) return;
  const int label = j.loss ? j.labels[row] : -1;
  const bool has = label >= 0 && label < j.classes;
  const float z = !has ? 0.f : KP > 0 ? logits[in] : j.label_z[row];
  float top = -__builtin_inff(), sum = 0.f;
#pragma unroll 4
  for (int64_t t = lane; t < j.tiles; t += 16) {
    const f32x2 o = j.part[t * j.rows + row];
    const float now = fmaxf(top, o[0]), from = now == -__builtin_inff() ? 0.f : now;
    sum = sum * exp2_of(top - from) + o[1] * exp2_of(o[0] - from);
    top = now;
  }
  float all = top;
  all = fmaxf(all, dpp<0xB1>(all));
  all = fmaxf(all, dpp<0x4E>(all));
  all = fmaxf(all, dpp<0x141>(all));
  all = fmaxf(all, dpp<0x140>(all));
  const float from = all == -__builtin_inff() ? 0.f : all;
  sum = group_sum<16>(sum * exp2_of(top - from));
  if (lane > 0) return;
  const float log = __builtin_amdgcn_logf(sum);
  // no class at all (a sum that is no number is a row of no numbers)
  const bool none = all == -__builtin_inff() && sum == 0.f;
  if (j.lse) j.lse[row] = none ? all : fmaf(all, kUnitHigh, fmaf(all, kUnitLow, log * kUnitHigh));
  if (j.loss) j.loss[row] = !has ? 0.f : z == -__builtin_inff() ? __builtin_inff() : (all - z + log) * kUnitHigh;
}

// the gradients of no rows
template <typename T>
__global__ __launch_bounds__(kThreads) void k_zero(CopyArgs j) {
  for (int64_t r = blockIdx.x; r < j.rows; r += kPadGrid)
    for (int c = threadIdx.x; c < j.cols; c += kThreads) ((T*)j.dst)[r * j.dst_ld + c] = (T)0;
}

// What is summed at a backward pass's end, in one launch: the parts of dx, the parts
// of dw, and dbias over the tiles' rows, as many workgroups as each has (three launches
// of 2 to 5 us each for small sizes; HBM bounds large ones: 8 parts of 8192 x 256 and 64
// of dbias over 100000 classes 20 us).
struct BiasArgs { const float* part; float* dbias; int64_t ld, n; int parts; float factor; };
__device__ __forceinline__ void bias_block(const BiasArgs& j, uint32_t block) {
  const int64_t c = (int64_t)block * kThreads + threadIdx.x;
  if (c >= j.n) return;
  float t = 0.f;
#pragma unroll 8
  for (int i = 0; i < j.parts; ++i) t += j.part[i * j.ld + c];
  j.dbias[c] = t * j.factor;
}
struct EndArgs {
  JoinArgs x, w;
  BiasArgs b;
  uint32_t nx, nw;                     // workgroups of x and of w
  int x_slices, w_slices;
};
template <typename T>
__global__ __launch_bounds__(kThreads) void k_loss_end(EndArgs j) {
  static_assert(kThreads == kJoinThreads);
  const uint32_t b = blockIdx.x;
  if (b < j.nx) {
    if (j.x_slices) join_block<T, 16>(j.x, b);
    else join_block<T, 1>(j.x, b);
  } else if (b < j.nx + j.nw) {
    if (j.w_slices) join_block<T, 16>(j.w, b - j.nx);
    else join_block<T, 1>(j.w, b - j.nx);
  } else {
    bias_block(j.b, b - j.nx - j.nw);
  }
}

// ---------------------------------------------------------------------- plan
int64_t round_up(int64_t v, int64_t by) { return (v + by - 1) / by * by; }

// The tiles of the logits (classes x rows) and of the products (columns x rows of
// the result), by what the sizes fill.  float32 64 x 64: two
// steps of 128 bytes, 32 KB of LDS, let four workgroups on a CU (2048 rows x 512 over 2048 classes:
// 177 us, 197 in three steps; steps of 64 bytes 180).
template <typename T> struct Tiles;
template <> struct Tiles<uint16_t> {
  typedef Tile<kBf16, 256, 256, 4, 4, 128, 2, kBlocks> Long;    // many columns of x
  typedef Tile<kBf16, 256, 128, 4, 2, 64, 3, kBlocks> Short;   // few: two workgroups a CU
  typedef Tile<kBf16, 256, 64, 4, 1, 64, 4, kBlocks> Few;       // few rows
  typedef Tile<kBf16, 64, 64, 2, 2, 128, 3, kBlocks> Tiny;      // few tiles of these
  template <bool BOTH> using Large = SumTile<kBf16, 256, 256, 4, 4, 128, 2, BOTH>;
  template <bool BOTH> using Small = SumTile<kBf16, 128, 128, 2, 2, 128, 2, BOTH>;
  template <bool BOTH> using Least = SumTile<kBf16, 64, 64, 2, 2, 128, 3, BOTH>;
};
template <> struct Tiles<float> {
  typedef Tile<kF32, 128, 128, 2, 2, 64, 2, kBlocks> Long;
  typedef Tile<kF32, 128, 128, 2, 2, 64, 2, kBlocks> Short;
  typedef Tile<kF32, 64, 32, 4, 1, 128, 3, kBlocks> Few;        // few tiles of the next
  typedef Tile<kF32, 64, 64, 2, 2, 128, 2, kBlocks> Tiny;
  template <bool BOTH> using Large = SumTile<kF32, 128, 128, 2, 2, 64, 2, BOTH>;
  template <bool BOTH> using Small = SumTile<kF32, 64, 64, 2, 2, 128, 2, BOTH>;
  template <bool BOTH> using Least = Small<BOTH>;
};

enum Kind { kLong, kShort, kFew, kTiny };
// calls f(tile) with the kind's tile
template <typename T, typename F>
auto with_tile(Kind k, F f) {
  typedef Tiles<T> TS;
  return k == kLong    ? f((typename TS::Long*)nullptr)
         : k == kShort ? f((typename TS::Short*)nullptr)
         : k == kFew   ? f((typename TS::Few*)nullptr)
                       : f((typename TS::Tiny*)nullptr);
}

// The logits' tile: the largest that fills the CUs (bf16, a step in the tiles of the
// rule and in the next larger ones, us: 1000 rows x 1000 over 1000 classes 51, 94; 90 x
// 90 over 450 26, 37).  float32 tiles of 64 x 64 until those of 128 x 128 fill the CUs four
// times: a last round of these that is not full costs more (1537 rows over 5003 classes:
// 60 us, 87), and of 64 x 32 where not every CU has one of those: a step of a tile is then
// what a CU takes to make it (64 x 64 and 64 x 32, a step of the loss, us: 200 rows x 1000
// over 300 classes 71, 58; 4 x 1000 over 500 63, 49; 16 x 32 over 100 20, 23).
template <typename T>
Kind kind_of(int64_t rows, int dim, int64_t classes) {
  if (sizeof(T) == 4) {
    if (tiles_of(rows, 64) * tiles_of(classes, 64) <= 256) return kFew;
    return tiles_of(rows, 128) * tiles_of(classes, 128) < 1024 ? kTiny : kLong;
  }
  if (rows <= 64) return tiles_of(classes, 256) >= 192 ? kFew : kTiny;
  if (dim > 256 && tiles_of(rows, 256) * tiles_of(classes, 256) >= 192) return kLong;
  return tiles_of(rows, 128) * tiles_of(classes, 256) >= 192 ? kShort : kTiny;
}

// A product of m columns and n rows over `depth` terms, in the tiles that should take
// less time.  Steps timed over 8192 cubed (bf16) and 4096 cubed (float32).
enum Size { kLargeSum, kSmallSum, kLeastSum };
struct Pass : Cut { Size size; };
template <typename T>
Pass pass(int64_t m, int64_t n, int64_t depth) {
  typedef typename Tiles<T>::template Large<true> L;
  typedef typename Tiles<T>::template Small<true> S;
  typedef typename Tiles<T>::template Least<true> E;
  constexpr bool bf16 = sizeof(T) == 2;
  auto cut = [&](int bm, int bn, int elements, const StepTime& t) {
    return cut_up(m, n, bm, bn, (int)tiles_of(depth, elements), t);
  };
  Pass p{cut(L::BM, L::BN, L::kElements, bf16 ? StepTime{2.05, 2.05, 1} : StepTime{1.07, 1.3, 3}), kLargeSum};
  const Cut s = cut(S::BM, S::BN, S::kElements, bf16 ? StepTime{0.67, 0.8, 2} : StepTime{0.58, 0.8, 4});
  if (s.us < p.us) p = {s, kSmallSum};
  if (bf16) {
    const Cut e = cut(E::BM, E::BN, E::kElements, StepTime{0.22, 0.5, 3});
    if (e.us < p.us) p = {e, kLeastSum};
  }
  return p;
}
// columns of B of a tile
template <typename T>
int rows_of(Size s) {
  typedef Tiles<T> TS;
  return s == kLargeSum   ? TS::template Large<true>::BN
         : s == kSmallSum ? TS::template Small<true>::BN
                          : TS::template Least<true>::BN;
}

// Bytes of G.  A piece's products cut their sums into parts where it has few classes, and
// what the parts cost is paid for each piece (8192 x 256 rows, 100000 classes: 2.58 ms in
// pieces of 256 MB, 2.51 of 512, 2.40 of 1 GB, 2.31 where those are of a size).
constexpr int64_t kPiece = 1 << 30;

// bf16 gradients of at most so many rows take G as the sum of two terms, the second ones in
// rows of their own: a longer sum of dw, more rows of dx's sums.  What is lost where a
// row's largest term is rounded is the same for the whole row, and only over many rows
// does it average to what the result's own rounding loses.  In the norm, one term: dw is
// off by 1.7 times the latter (2 rows), 1.4 to 1.5 (100 to 500), 1.2 to 1.44 (more), with
// two by 1.0; dx is as far off as dw without LabelTerm, and with it, which costs nothing,
// by 1.0 to 1.35 of more rows than a few.  One term, two for dw, two for both, us: 512 x
// 256 rows over 100000 classes 222, 291, 315; 256 rows 156, 175, 198; 400 x 1000 over
// 10000 117, 131; 64 x 256 over 100000 97, 113, 113.
constexpr int64_t kTwoTerms = 512, kTwoTermsOfX = 256;

// Where things lie in the workspace, and how the classes are cut up.
struct Plan {
  Kind kind;
  int bm, bn;                                        // of the logits' tile
  int64_t dim_pad, rows_pad, all, piece, pieces;     // all, piece: classes in whole tiles
  int64_t rest;                                      // rows of G to its second terms' (0: none)
  bool x_terms;                                      // dx takes them too
  bool dx_sums, dw_sums;                             // float32 sums that are not the result yet
  int64_t g_rows;
  int64_t strips, parts;                             // k_strip's strips (0: tiles); the forward's pairs of a row
  size_t x, w, part, label_z, g, bias, dx, dw, label, bytes;
  Pass to_x, to_w;
};

template <typename T>
Plan plan(int64_t rows, int dim, int64_t classes) {
  Plan p{};
  size_t at = 0;
  auto take = [&](int64_t elements, size_t size) {
    const size_t here = at;
    at += ((size_t)elements * size + 255) & ~(size_t)255;
    return here;
  };
  p.kind = kind_of<T>(rows, dim, classes);
  with_tile<T>(p.kind, [&](auto* tile) {
    p.bm = std::remove_pointer_t<decltype(tile)>::BM;
    p.bn = std::remove_pointer_t<decltype(tile)>::BN;
  });
  p.dim_pad = round_up(dim, kRow<T>);
  p.rows_pad = round_up(rows, p.bn);
  p.all = round_up(classes, p.bm);                   // a step of every product divides a tile's classes
  p.rest = sizeof(T) == 4 || rows > kTwoTerms ? 0 : 2 * rows <= p.rows_pad ? p.rows_pad / 2 : p.rows_pad;
  p.g_rows = std::max(p.rows_pad, 2 * p.rest);
  p.x_terms = p.rest && rows <= kTwoTermsOfX;
  const int64_t most = kPiece / ((int64_t)sizeof(T) * p.g_rows) / p.bm * p.bm;
  p.piece = std::min<int64_t>(p.all, std::max<int64_t>(p.bm, most));
  p.pieces = (p.all + p.piece - 1) / p.piece;
  p.piece = round_up((p.all + p.pieces - 1) / p.pieces, p.bm);
  p.pieces = (p.all + p.piece - 1) / p.piece;
  const int64_t terms = p.rest ? p.g_rows : rows, x_rows = p.x_terms ? p.g_rows : rows;
  p.to_x = pass<T>(dim, x_rows, p.piece);
  p.to_w = pass<T>(dim, p.piece, terms);
  p.x = take(terms * p.dim_pad, sizeof(T));
  p.w = take(classes * p.dim_pad, sizeof(T));
  const size_t both = at;
  p.parts = p.all / p.bm;
  if (sizeof(T) == 2 && p.dim_pad <= 256) {
    const int64_t blocks = tiles_of(rows, kStripRows), tiles = tiles_of(classes, kStripClasses);
    const int64_t strips = std::max<int64_t>(1, 256 / blocks);
    if (rows > 128 && tiles >= 16 * strips) {
      p.strips = strips;
      p.parts = 2 * strips;
    }
  }
  p.part = take(p.parts * rows, sizeof(f32x2));
  p.label_z = take(rows, sizeof(float));
  const size_t forward = at;
  at = both;
  p.g = take(p.g_rows * p.piece, sizeof(T));
  p.bias = take(p.rows_pad / p.bn * p.all, sizeof(float));
  p.dx_sums = p.pieces > 1 || p.to_x.parts > 1 || p.x_terms;
  p.dw_sums = p.to_w.parts > 1;
  p.dx = take(p.dx_sums ? p.to_x.parts * x_rows * part_ld(dim) : 0, sizeof(float));
  p.dw = take(p.dw_sums ? p.to_w.parts * p.piece * part_ld(dim) : 0, sizeof(float));
  p.label = take(sizeof(T) == 2 && !p.x_terms ? rows : 0, sizeof(float));
  p.bytes = std::max(at, forward);
  return p;
}

// Operands of whole steps whose rows can be copied 16 bytes at a time: the matrices
// themselves where they are that and all their rows may be read, else copies.
template <typename T>
bool needs_copy(const Mat& m, int dim, int64_t dim_pad) {
  const int64_t ld = m.ld * (int64_t)sizeof(T);
  return dim != dim_pad || (uintptr_t)m.p % 16 != 0 || ld % 16 != 0 || ld >= (int64_t)1 << 24;
}
// labels: rows of x without one are zeros, bias: rows of w with -inf (null: as they are);
// wrap: x twice, with zeros from its rows to `wrap`
template <typename T>
hipError_t operands(const LossJob& j, int64_t dim_pad, const int32_t* labels, const float* bias, int64_t wrap, char* x_copy,
                    char* w_copy, Operand* x, Operand* w, hipStream_t st) {
  *x = {(const char*)j.x.p, j.x.ld * (int64_t)sizeof(T), j.rows - 1, nullptr, 0};
  *w = {(const char*)j.w.p, j.w.ld * (int64_t)sizeof(T), j.classes - 1, nullptr, 0};
  auto blocks = [&](int64_t rows) {
    return (uint32_t)std::min<int64_t>((rows * dim_pad / 8 + kThreads - 1) / kThreads, kPadGrid);
  };
  uint32_t nx = 0, nw = 0;
  if (labels || needs_copy<T>(j.x, j.dim, dim_pad)) {
    nx = blocks(wrap ? 2 * wrap : j.rows);
    x->p = x_copy;
    x->ld = dim_pad * (int64_t)sizeof(T);
  }
  if (bias || needs_copy<T>(j.w, j.dim, dim_pad)) {
    nw = blocks(j.classes);
    w->p = w_copy;
    w->ld = dim_pad * (int64_t)sizeof(T);
  }
  if (nx + nw == 0) return hipSuccess;
  const CopyArgs a{j.x, x_copy, dim_pad, j.rows, wrap, labels, nullptr, j.classes, j.dim};
  const CopyArgs b{j.w, w_copy, dim_pad, j.classes, 0, nullptr, bias, 0, j.dim};
  return enqueue(j.dim == dim_pad ? k_pad<T, kExact> : j.dim >= 8 ? k_pad<T, kRagged> : k_pad<T, kSmall>,
                 dim3(nx + nw), dim3(kThreads), 0, st, a, b, nx);
}

SumMajor terms(const Operand& o, int64_t row_bytes) { return {o.p, o.ld, o.last, (int)(row_bytes / 16)}; }

template <typename T, bool GRAD>
hipError_t logits(LogitArgs& a, const Plan& p, int64_t classes, hipStream_t st) {
  return with_tile<T>(p.kind, [&](auto* tile) {
    typedef std::remove_pointer_t<decltype(tile)> TL;
    a.steps = (int)(p.dim_pad / TL::kElements);
    a.tm = (uint32_t)tiles_of(classes, TL::BM);
    a.tn = (uint32_t)(p.rows_pad / TL::BN);
    return enqueue(k_logits<TL, T, GRAD>, dim3(a.tm * a.tn), dim3(TL::kThreads), logits_lds<TL>(), st, a);
  });
}

SumArgs& cut_as(SumArgs& a, const Cut& c) {
  a.steps = c.steps;
  a.per = c.per;
  a.tm = (uint32_t)c.tm;
  a.tn = (uint32_t)c.tn;
  a.parts = (uint32_t)c.parts;
  return a;
}

// dx's product, dw's, or both (tm 0: absent), in one launch where their tiles are of a size
template <typename T, template <bool> class TL>
hipError_t products_of(const SumArgs& x, const SumArgs& w, hipStream_t st) {
  if (!w.tm) return x.tm ? sum_product<TL<false>, T>(x, st) : hipSuccess;
  if (!x.tm) return sum_product<TL<true>, T>(w, st);
  const uint32_t nx = x.tm * x.tn * x.parts, nw = w.tm * w.tn * w.parts;
  return enqueue(k_sum_pair<TL<false>, TL<true>, T>, dim3(nx + nw), dim3(TL<false>::kThreads), TL<false>::kLds, st, x, w, nx);
}
template <typename T>
hipError_t products_in(Size s, const SumArgs& x, const SumArgs& w, hipStream_t st) {
  typedef Tiles<T> TS;
  return s == kLargeSum   ? products_of<T, TS::template Large>(x, w, st)
         : s == kSmallSum ? products_of<T, TS::template Small>(x, w, st)
                          : products_of<T, TS::template Least>(x, w, st);
}
template <typename T>
hipError_t products(const SumArgs& x, Size xs, const SumArgs& w, Size ws, hipStream_t st) {
  if (xs == ws || !w.tm) return products_in<T>(xs, x, w, st);
  const hipError_t e = products_in<T>(xs, x, SumArgs{}, st);
  return e != hipSuccess ? e : products_in<T>(ws, SumArgs{}, w, st);
}

template <typename T>
hipError_t forward(const LossJob& j, hipStream_t st) {
  const Plan p = plan<T>(j.rows, j.dim, j.classes);
  LogitArgs a{};
  hipError_t e = operands<T>(j, p.dim_pad, nullptr, nullptr, 0, j.workspace + p.x, j.workspace + p.w, &a.x, &a.w, st);
  if (e != hipSuccess) return e;
  f32x2* const part = (f32x2*)(j.workspace + p.part);
  float* const label_z = j.loss ? (float*)(j.workspace + p.label_z) : nullptr;
  if (p.strips) {
    const StripArgs s{a.w, a.x, j.bias, j.rows, j.classes, part, (int)tiles_of(j.classes, kStripClasses), (int)p.strips};
    auto run = [&](auto kernel, int lds) {
      return enqueue(kernel, dim3((unsigned)(tiles_of(j.rows, kStripRows) * p.strips)), dim3(512), lds, st, s);
    };
    e = p.dim_pad == 64    ? run(k_strip<1>, strip_lds<1>())
        : p.dim_pad == 128 ? run(k_strip<2>, strip_lds<2>())
        : p.dim_pad == 192 ? run(k_strip<3>, strip_lds<3>())
                           : run(k_strip<4>, strip_lds<4>());
  } else {
    a.bias = j.bias;
    a.rows = j.rows;
    a.classes = j.classes;
    a.part = part;
    a.labels = j.labels;
    a.label_z = label_z;
    e = logits<T, false>(a, p, j.classes, st);
  }
  if (e != hipSuccess) return e;
  const int64_t parts = p.strips ? p.parts : a.tm;
  const FinishArgs f{part, label_z, a.x, a.w, j.bias, j.labels, j.loss, j.lse, j.rows, j.classes, parts};
  const int64_t panels = p.strips ? p.dim_pad / 64 : 0;
  return enqueue(panels == 0   ? k_loss<0>
                 : panels == 1 ? k_loss<1>
                 : panels == 2 ? k_loss<2>
                 : panels == 3 ? k_loss<3>
                               : k_loss<4>,
                 dim3((unsigned)tiles_of(j.rows, kThreads / 16)), dim3(kThreads), 0, st, f);
}

template <typename T>
hipError_t zero(void* p, int64_t rows, int cols, int64_t ld, hipStream_t st) {
  if (!p) return hipSuccess;
  CopyArgs a{};
  a.dst = p;
  a.dst_ld = ld;
  a.rows = rows;
  a.cols = cols;
  return enqueue(k_zero<T>, dim3((unsigned)std::min<int64_t>(rows, kPadGrid)), dim3(kThreads), 0, st, a);
}

template <typename T>
hipError_t backward(const LossJob& j, hipStream_t st) {
  if (j.rows == 0) {
    const hipError_t e = zero<T>(j.dw.p, j.classes, j.dim, j.dw.ld, st);
    return e == hipSuccess ? zero<float>(j.dbias, 1, (int)j.classes, j.classes, st) : e;
  }
  const Plan p = plan<T>(j.rows, j.dim, j.classes);
  constexpr int64_t E = sizeof(T);
  char* const ws = j.workspace;
  LogitArgs a{};
  Operand w;
  // rows without a label and classes taken out may hold anything: they are zeros here
  hipError_t e = operands<T>(j, p.dim_pad, j.labels, j.bias, p.rest, ws + p.x, ws + p.w, &a.x, &w, st);
  a.rows = j.rows;
  a.lse = j.lse;
  a.dloss = j.dloss;
  a.labels = j.labels;
  // one factor for all rows is left to the sums, so that no term is rounded for it
  const bool factor = !j.dloss && std::isfinite(j.scale);
  a.scale = factor ? 1.f : j.scale;
  a.rest = p.rest;
  if (sizeof(T) == 2 && j.dx.p && !p.x_terms) a.label_rest = (float*)(ws + p.label);
  a.all_classes = j.classes;
  a.g = ws + p.g;
  a.g_ld = p.piece;
  a.bias_ld = p.all;
  const LabelTerm label{a.label_rest, j.labels, (const uint16_t*)w.p, w.ld / E, j.classes, factor ? j.scale : 1.f};
  for (int64_t i = 0; e == hipSuccess && i < p.pieces; ++i) {
    const int64_t first = i * p.piece, left = j.classes - first, mine = std::min(left, p.piece);
    const int64_t wide = round_up(mine, p.bm);       // columns of G that are written
    a.w = w;
    a.w.p = w.p + first * w.ld;
    a.w.last = left - 1;
    a.bias = j.bias ? j.bias + first : nullptr;
    a.classes = left;
    a.first = first;
    a.part_bias = j.dbias ? (float*)(ws + p.bias) + first : nullptr;
    e = logits<T, true>(a, p, wide, st);
    if (e != hipSuccess) return e;
    SumArgs x{}, w{};
    x.factor = w.factor = factor ? j.scale : 1.f;
    if (j.dx.p) {
      x.a = terms(a.w, p.dim_pad * E);
      x.b = {ws + p.g, p.piece * E, p.g_rows - 1, nullptr, 0};
      x.c = p.dx_sums ? (void*)(ws + p.dx) : j.dx.p;
      x.ldc = p.dx_sums ? part_ld(j.dim) : j.dx.ld;
      x.wide = p.dx_sums;
      x.m = j.dim;
      x.n = p.x_terms ? p.g_rows : j.rows;
      x.add = i > 0;
      if (!p.dx_sums) x.label = label;
      Pass t = p.to_x;
      // the last piece may have fewer steps than parts: all parts hold sums by then
      t.steps = (int)(wide / (p.piece / t.steps));
      t.per = (int)tiles_of(t.steps, t.parts);
      if (i > 0) t.parts = (int)tiles_of(t.steps, t.per);
      cut_as(x, t);
    }
    if (j.dw.p) {
      w.a = terms(a.x, p.dim_pad * E);
      if (p.rest) w.a.last = p.g_rows - 1;
      w.bs = {ws + p.g, p.piece * E, p.g_rows - 1, (int)(p.piece * E / 16)};
      w.m = j.dim;
      w.n = mine;
      w.c = p.dw_sums ? (void*)(ws + p.dw) : (T*)j.dw.p + first * j.dw.ld;
      w.ldc = p.dw_sums ? part_ld(j.dim) : j.dw.ld;
      w.wide = p.dw_sums;
      Pass t = p.to_w;
      t.tn = tiles_of(mine, rows_of<T>(t.size));
      cut_as(w, t);
    }
    e = products<T>(x, p.to_x.size, w, p.to_w.size, st);
    if (e != hipSuccess) return e;
    const bool last = i + 1 == p.pieces;
    EndArgs end{};
    uint32_t nb = 0;
    if (j.dw.p && p.dw_sums) {
      const Mat out = {(T*)j.dw.p + first * j.dw.ld, j.dw.ld};
      end.w = join_args((const float*)(ws + p.dw), p.to_w.parts, mine, j.dim, nullptr, 0, out);
      end.nw = (uint32_t)join_blocks(end.w);
      end.w_slices = joins_in_slices(end.w);
    }
    if (last && j.dx.p && p.dx_sums) {
      end.x = join_args((const float*)(ws + p.dx), p.to_x.parts, j.rows, j.dim, nullptr, 0, j.dx);
      if (p.x_terms) {                               // the second terms' rows are parts too
        end.x.parts = 2 * p.to_x.parts;
        end.x.m = p.rest;
      }
      end.x.label = label;
      end.nx = (uint32_t)join_blocks(end.x);
      end.x_slices = joins_in_slices(end.x);
    }
    if (last && j.dbias) {
      end.b = {(const float*)(ws + p.bias), j.dbias, p.all, j.classes, (int)(p.rows_pad / p.bn),
               factor ? j.scale : 1.f};
      nb = (uint32_t)tiles_of(j.classes, kThreads);
    }
    if (end.nx + end.nw + nb) e = enqueue(k_loss_end<T>, dim3(end.nx + end.nw + nb), dim3(kThreads), 0, st, end);
  }
  return e;
}

}  // namespace

size_t loss_workspace(Elt e, int64_t rows, int dim, int64_t classes) {
  return e == BF16 ? plan<uint16_t>(rows, dim, classes).bytes : plan<float>(rows, dim, classes).bytes;
}

hipError_t launch_loss_forward(Elt e, const LossJob& j, hipStream_t st) {
  return e == BF16 ? forward<uint16_t>(j, st) : forward<float>(j, st);
}

hipError_t launch_loss_backward(Elt e, const LossJob& j, hipStream_t st) {
  return e == BF16 ? backward<uint16_t>(j, st) : backward<float>(j, st);
}

}  // namespace vfl

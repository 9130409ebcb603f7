// The softmax cross-entropy of a linear head over many classes on gfx950, with its
// gradients, without the logits in memory.
//
//   z = x w^T + bias, lse = log(sum_c exp z), loss = lse - z[label]
//   G = dloss (exp(z - lse) - onehot(label)), dx = G w, dw = G^T x, dbias = sum_r G
//
// Forward: a workgroup makes a tile of logits in registers (gemm.h) and leaves each
// row's largest value and sum of exponentials over the tile's columns; a second
// launch joins the tiles' pairs.  Backward: the classes go in pieces; a tile of
// logits is made again, turned into G in registers and stored as it lies and
// transposed, in the operands' type, and two products read it.
//
// Exponentials and sums are taken to base 2 (z log2 e is one multiplication-addition
// with the bias, and the hardware's exponential is to base 2); one below 2^-126 is 0.  A class whose bias
// is -inf, and a column past the last class, is out of every sum whatever its
// weights hold; a row without a label has a gradient of 0 whatever its input holds.
#include <algorithm>

#include "ops8.h"
#include "product.h"

namespace vfl {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kThreads = 256;

template <typename T> constexpr Type type_of = sizeof(T) == 2 ? kBf16 : kF32;
template <typename T> constexpr int kStep = 128 / (int)sizeof(T);   // elements of a step of a product

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

// ------------------------------------------------------------------ operands
struct CopyArgs {
  const void* src;
  void* dst;
  int64_t ld, dst_ld, rows;            // elements from row to row
  const int32_t* labels;               // rows without a label are 0 (null: all are kept)
  const float* bias;                   // rows whose bias is -inf are 0
  int64_t classes;
  int cols;
};

// Rows padded with zeros to whole steps: of operands that are not so already.
constexpr int kPadGrid = 16384;
template <typename T>
__global__ __launch_bounds__(kThreads) void k_pad(CopyArgs j) {
  for (int64_t r = blockIdx.x; r < j.rows; r += kPadGrid)
    for (int c = threadIdx.x; c < j.dst_ld; c += kThreads)
      ((T*)j.dst)[r * j.dst_ld + c] = c < j.cols ? ((const T*)j.src)[r * j.ld + c] : (T)0;
}

// The transpose of [rows x cols], its rows padded with zeros to dst_ld: 64 x 64 a
// workgroup, through LDS.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_transpose(CopyArgs j) {
  __shared__ T tile[64][64 + 4 / sizeof(T) + 1];
  const int64_t r0 = (int64_t)blockIdx.x * 64;
  const int c0 = blockIdx.y * 64, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 4
  for (int i = wave; i < 64; i += 4) {
    const int64_t r = r0 + i;
    T v = (T)0;
    if (r < j.rows && c0 + lane < j.cols) {
      const bool keep = (!j.labels || (j.labels[r] >= 0 && j.labels[r] < j.classes)) && (!j.bias || j.bias[r] > -__builtin_inff());
      if (keep) v = ((const T*)j.src)[r * j.ld + c0 + lane];
    }
    tile[i][lane] = v;
  }
  __syncthreads();
#pragma unroll 4
  for (int i = wave; i < 64; i += 4)
    if (c0 + i < j.cols && r0 + lane < j.dst_ld) ((T*)j.dst)[(int64_t)(c0 + i) * j.dst_ld + r0 + lane] = tile[lane][i];
}

// -------------------------------------------------------------------- logits
struct LogitArgs {
  Operand x, w;                        // w: from the piece's first class
  const float* bias;                   // [classes] of the piece
  int steps;
  uint32_t tm, tn;
  int64_t rows, classes;               // classes: left from the piece's first
  f32x2* part;                         // forward: [tn][rows] of (largest, sum), to base 2
  // backward
  const float *lse, *dloss;
  const int32_t* labels;
  float scale;
  int64_t first, all_classes;          // the piece's first class
  void *g, *gt;
  int64_t g_ld, gt_ld;
  float* part_bias;                    // [tm][g_ld]
};

struct RowInfo { float lse2, d; int label, pad; };

template <class TL, typename T, bool GRAD>
__global__ __launch_bounds__(TL::kThreads) void k_logits(LogitArgs j) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int WC = TL::BN / TL::WN, WR = TL::BM / TL::WM, NQ = TL::NF / TL::DN;
  // the statistics of a tile's rows and columns fit the copies' buffers
  static_assert(TL::BM * 16 + WR * TL::BN * 4 <= TL::kLds && WC * TL::BM * 8 <= TL::kLds);
  uint32_t tm, tn;
  tile_of(blockIdx.x, j.tm, j.tn, &tm, &tn);
  const TL tile;
  typename TL::Acc acc;
#pragma unroll
  for (int f = 0; f < TL::MF; ++f)
#pragma unroll
    for (int c = 0; c < TL::NF; ++c) acc[f][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t m0 = (int64_t)tm * TL::BM, n0 = (int64_t)tn * TL::BN;
  tile.run(j.x, j.w, m0, n0, 0, j.steps, smem, acc);
  __syncthreads();                                   // the copies' buffers are free

  // the columns' biases to base 2, and their numbers (-2: out of every sum)
  float bias[TL::NF];
  int number[TL::NF];
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int c = 0; c < TL::DN; ++c) {
      const int64_t col = n0 + tile.col(q) + c;
      float b = -__builtin_inff();
      if (col < j.classes) b = j.bias ? j.bias[col] : 0.f;
      bias[q * TL::DN + c] = b * kLog2e;
      number[q * TL::DN + c] = b == -__builtin_inff() ? -2 : (int)(j.first + col);
    }
  auto logit = [&](int f, int c, int r) {
    const float z = fmaf(acc[f][c][r], kLog2e, bias[c]);
    return number[c] == -2 ? -__builtin_inff() : z;
  };

  if constexpr (!GRAD) {
    f32x2* const stat = (f32x2*)smem;                // [WC][BM]
#pragma unroll
    for (int f = 0; f < TL::MF; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float z[TL::NF], top = -__builtin_inff();
#pragma unroll
        for (int c = 0; c < TL::NF; ++c) {
          z[c] = logit(f, c, r);
          top = fmaxf(top, z[c]);
        }
        top = fmaxf(top, dpp<0xB1>(top));
        top = fmaxf(top, dpp<0x4E>(top));
        top = fmaxf(top, dpp<0x141>(top));
        top = fmaxf(top, dpp<0x140>(top));
        const float from = top == -__builtin_inff() ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < TL::NF; ++c) sum += exp2_of(z[c] - from);
        sum = group_sum<16>(sum);
        if ((tile.lane & 15) == 0) stat[tile.wn / TL::WN * TL::BM + tile.row(f, r)] = f32x2{top, sum};
      }
    __syncthreads();
    for (int i = threadIdx.x; i < TL::BM; i += TL::kThreads) {
      if (m0 + i >= j.rows) continue;
      f32x2 s = stat[i];
#pragma unroll
      for (int w = 1; w < WC; ++w) {
        const f32x2 o = stat[w * TL::BM + i];
        const float top = fmaxf(s[0], o[0]), from = top == -__builtin_inff() ? 0.f : top;
        s = f32x2{top, s[1] * exp2_of(s[0] - from) + o[1] * exp2_of(o[0] - from)};
      }
      j.part[(int64_t)tn * j.rows + m0 + i] = s;
    }
  } else {
    RowInfo* const info = (RowInfo*)smem;            // [BM]
    float* const sums = (float*)(smem + TL::BM * sizeof(RowInfo));   // [WR][BN]
    for (int i = threadIdx.x; i < TL::BM; i += TL::kThreads) {
      RowInfo v = {0.f, 0.f, -1, 0};
      const int64_t row = m0 + i;
      if (row < j.rows) {
        const int label = j.labels[row];
        if (label >= 0 && label < j.all_classes) {
          const float lse = j.lse[row];
          // no class at all: every exponential is 0
          v.lse2 = lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e;
          v.d = j.dloss ? j.dloss[row] : j.scale;
          v.label = label;
        }
      }
      info[i] = v;
    }
    __syncthreads();
    float total[TL::NF];
#pragma unroll
    for (int c = 0; c < TL::NF; ++c) total[c] = 0.f;
#pragma unroll
    for (int fb = 0; fb < TL::MF / TL::DM; ++fb)
#pragma unroll
      for (int fd = 0; fd < TL::DM; ++fd) {
        const int f = fb * TL::DM + fd;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = tile.row(f, r);
          const RowInfo v = info[row];
#pragma unroll
          for (int c = 0; c < TL::NF; ++c) {
            const float p = exp2_of(logit(f, c, r) - v.lse2);
            const float g = v.label < 0 ? 0.f : v.d * (p - (number[c] == v.label ? 1.f : 0.f));
            total[c] += g;
            acc[f][c][r] = g;
          }
          T* const out = (T*)j.g + (m0 + row) * j.g_ld + n0;
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            f32x4 w = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < TL::DN; ++c) w[c] = acc[f][q * TL::DN + c][r];
            store_to<TL::DN>(out + tile.col(q), w, TL::DN);
          }
        }
      }
    // 4 DM consecutive rows of each of the lane's columns
    if (j.gt) {
#pragma unroll
      for (int fb = 0; fb < TL::MF / TL::DM; ++fb)
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int c = 0; c < TL::DN; ++c) {
            T* const out = (T*)j.gt + (n0 + tile.col(q) + c) * j.gt_ld + m0 + tile.row(fb * TL::DM, 0);
#pragma unroll
            for (int fd = 0; fd < TL::DM; ++fd) store_to<4>(out + 4 * fd, acc[fb * TL::DM + fd][q * TL::DN + c], 4);
          }
    }
    if (j.part_bias) {
#pragma unroll
      for (int c = 0; c < TL::NF; ++c) total[c] = stride_sum<16>(total[c]);
      if (tile.lane < 16) {
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int c = 0; c < TL::DN; ++c) sums[tile.wm / TL::WM * TL::BN + tile.col(q) + c] = total[q * TL::DN + c];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < TL::BN; i += TL::kThreads) {
        float t = sums[i];
#pragma unroll
        for (int w = 1; w < WR; ++w) t += sums[w * TL::BN + i];
        j.part_bias[(int64_t)tm * j.g_ld + n0 + i] = t;
      }
    }
  }
}

// ---------------------------------------------------------------------- join
struct FinishArgs {
  const f32x2* part;
  Mat x, w;
  const float* bias;
  const int32_t* labels;
  float *loss, *lse;
  int64_t rows, classes, tiles;
  int dim;
};

// A row a group of 16 lanes: the tiles' pairs joined, and the label's logit.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_loss(FinishArgs j) {
  const int lane = threadIdx.x & 15;
  const int64_t row = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
  if (row >= j.rows) return;
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
  const float lse = (all + __builtin_amdgcn_logf(sum)) * kLn2;
  if (j.lse && lane == 0) j.lse[row] = lse;
  if (!j.loss) return;
  const int label = j.labels[row];
  float loss = 0.f;
  if (label >= 0 && label < j.classes) {
    const T* const x = row_of<T>(j.x, row);
    const T* const w = row_of<T>(j.w, label);
    float z = 0.f;
    for (int c = lane; c < j.dim; c += 16) z = fmaf(ld1<T>(x + c), ld1<T>(w + c), z);
    z = group_sum<16>(z);
    const float b = j.bias ? j.bias[label] : 0.f;
    loss = b == -__builtin_inff() ? __builtin_inff() : lse - (z + b);
  }
  if (lane == 0) j.loss[row] = loss;
}

// the gradients of no rows
template <typename T>
__global__ __launch_bounds__(kThreads) void k_zero(CopyArgs j) {
  for (int64_t r = blockIdx.x; r < j.rows; r += kPadGrid)
    for (int c = threadIdx.x; c < j.cols; c += kThreads) ((T*)j.dst)[r * j.dst_ld + c] = (T)0;
}

struct BiasArgs { const float* part; float* dbias; int64_t ld, n; int parts; };
__global__ __launch_bounds__(kThreads) void k_bias(BiasArgs j) {
  const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (c >= j.n) return;
  float t = 0.f;
#pragma unroll 8
  for (int i = 0; i < j.parts; ++i) t += j.part[i * j.ld + c];
  j.dbias[c] = t;
}

// ---------------------------------------------------------------------- plan
int64_t round_up(int64_t v, int64_t by) { return (v + by - 1) / by * by; }

template <typename T> struct Tiles;
template <> struct Tiles<uint16_t> {
  typedef Tile<kBf16, 256, 256, 2, 4, 128, 2, kBlocks> Large;
  typedef Tile<kBf16, 128, 128, 2, 2, 128, 2, kBlocks> Small;
};
template <> struct Tiles<float> {
  typedef Tile<kF32, 128, 128, 2, 2, 128, 2, kBlocks> Large;
  typedef Tile<kF32, 64, 64, 2, 2, 128, 2, kBlocks> Small;
};

struct Pass {
  bool large;
  int64_t tm, tn;
  int steps, parts, per;
};

// a product of m x n results over `depth` elements
template <typename T>
Pass pass(int64_t m, int64_t n, int64_t depth, bool split) {
  typedef Tiles<T> TS;
  Pass p;
  p.steps = (int)((depth + kStep<T> - 1) / kStep<T>);
  p.large = tiles_of(m, TS::Large::BM) * tiles_of(n, TS::Large::BN) >= 128;
  const int by = p.large ? TS::Large::BM : TS::Small::BM;
  p.tm = tiles_of(m, by);
  p.tn = tiles_of(n, by);
  int64_t parts = 1;
  if (split && p.tm * p.tn < 256) parts = std::max<int64_t>(1, std::min<int64_t>(512 / (p.tm * p.tn), p.steps / 8));
  p.per = (int)((p.steps + parts - 1) / parts);
  p.parts = (p.steps + p.per - 1) / p.per;
  return p;
}

constexpr int kPad = 256;              // rows of G, classes of a piece: whole tiles of any kind
constexpr int64_t kPiece = 64 << 20;   // bytes of G

// Where things lie in the workspace, and how the classes are cut up.
struct Plan {
  int64_t dim_pad, rows_pad, piece, pieces;          // piece: classes of one, in whole tiles
  size_t x, w, part, xt, wt, g, gt, bias, dx, dw, bytes;
  Pass forward, grad, to_x, to_w;
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
  p.dim_pad = round_up(dim, kStep<T>);
  p.rows_pad = round_up(rows, kPad);
  p.forward = pass<T>(rows, classes, dim, false);
  const int64_t all = round_up(classes, kPad);
  p.piece = std::min<int64_t>(all, std::max<int64_t>(kPad, kPiece / ((int64_t)sizeof(T) * p.rows_pad) / kPad * kPad));
  p.pieces = (all + p.piece - 1) / p.piece;
  p.grad = pass<T>(p.rows_pad, p.piece, dim, false);
  p.to_x = pass<T>(rows, dim, p.piece, true);
  p.to_w = pass<T>(p.piece, dim, p.rows_pad, true);
  p.x = take(rows * p.dim_pad, sizeof(T));
  p.w = take(classes * p.dim_pad, sizeof(T));
  const size_t both = at;
  p.part = take(p.forward.tn * rows, sizeof(f32x2));
  const size_t forward = at;
  at = both;
  p.xt = take(dim * p.rows_pad, sizeof(T));
  p.wt = take(dim * all, sizeof(T));
  p.g = take(p.rows_pad * p.piece, sizeof(T));
  p.gt = take(p.rows_pad * p.piece, sizeof(T));
  p.bias = take(p.grad.tm * p.piece, sizeof(float));
  p.dx = take(p.to_x.parts * rows * part_ld(dim), sizeof(float));
  p.dw = take(p.to_w.parts * p.piece * part_ld(dim), sizeof(float));
  p.bytes = std::max(at, forward);
  return p;
}

// an operand of whole steps: the matrix itself where it is one, else a padded copy
template <typename T>
hipError_t operand(const Mat& m, int64_t rows, int dim, int64_t dim_pad, char* copy, Operand* out, hipStream_t st) {
  *out = {(const char*)m.p, m.ld * (int64_t)sizeof(T), rows - 1, nullptr, 0};
  if (dim == dim_pad && (uintptr_t)m.p % 16 == 0 && out->ld % 16 == 0 && out->ld < (int64_t)1 << 24) return hipSuccess;
  out->p = copy;
  out->ld = dim_pad * (int64_t)sizeof(T);
  CopyArgs a{};
  a.src = m.p;
  a.dst = copy;
  a.ld = m.ld;
  a.dst_ld = dim_pad;
  a.rows = rows;
  a.cols = dim;
  return enqueue(k_pad<T>, dim3((unsigned)std::min<int64_t>(rows, kPadGrid)), dim3(kThreads), 0, st, a);
}

template <typename T>
hipError_t transpose(const Mat& m, int64_t rows, int dim, int64_t ld, const int32_t* labels, int64_t classes,
                     const float* bias, char* to, hipStream_t st) {
  CopyArgs a{};
  a.src = m.p;
  a.dst = to;
  a.ld = m.ld;
  a.dst_ld = ld;
  a.rows = rows;
  a.labels = labels;
  a.bias = bias;
  a.classes = classes;
  a.cols = dim;
  return enqueue(k_transpose<T>, dim3((unsigned)tiles_of(ld, 64), (unsigned)tiles_of(dim, 64)), dim3(kThreads), 0, st, a);
}

template <typename T, bool GRAD>
hipError_t logits(LogitArgs& a, const Pass& p, hipStream_t st) {
  typedef Tiles<T> TS;
  a.steps = p.steps;
  a.tm = (uint32_t)p.tm;
  a.tn = (uint32_t)p.tn;
  auto run = [&](auto kernel, int threads, int lds) { return enqueue(kernel, dim3(a.tm * a.tn), dim3(threads), lds, st, a); };
  return p.large ? run(k_logits<typename TS::Large, T, GRAD>, TS::Large::kThreads, TS::Large::kLds)
                 : run(k_logits<typename TS::Small, T, GRAD>, TS::Small::kThreads, TS::Small::kLds);
}

template <typename T, typename O>
hipError_t times(ProductArgs& a, const Pass& p, hipStream_t st) {
  typedef Tiles<T> TS;
  a.steps = p.steps;
  a.per = p.per;
  a.tm = (uint32_t)p.tm;
  a.tn = (uint32_t)p.tn;
  return p.large ? product<typename TS::Large, O>(a, p.parts, st) : product<typename TS::Small, O>(a, p.parts, st);
}

template <typename T>
hipError_t forward(const LossJob& j, hipStream_t st) {
  const Plan p = plan<T>(j.rows, j.dim, j.classes);
  LogitArgs a{};
  hipError_t e = operand<T>(j.x, j.rows, j.dim, p.dim_pad, j.workspace + p.x, &a.x, st);
  if (e == hipSuccess) e = operand<T>(j.w, j.classes, j.dim, p.dim_pad, j.workspace + p.w, &a.w, st);
  if (e != hipSuccess) return e;
  a.bias = j.bias;
  a.rows = j.rows;
  a.classes = j.classes;
  a.part = (f32x2*)(j.workspace + p.part);
  e = logits<T, false>(a, p.forward, st);
  if (e != hipSuccess) return e;
  const FinishArgs f{a.part, j.x, j.w, j.bias, j.labels, j.loss, j.lse, j.rows, j.classes, p.forward.tn, j.dim};
  return enqueue(k_loss<T>, dim3((unsigned)tiles_of(j.rows, kThreads / 16)), dim3(kThreads), 0, st, f);
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
  char* const ws = j.workspace;
  LogitArgs a{};
  Operand w;
  hipError_t e = operand<T>(j.x, j.rows, j.dim, p.dim_pad, ws + p.x, &a.x, st);
  if (e == hipSuccess) e = operand<T>(j.w, j.classes, j.dim, p.dim_pad, ws + p.w, &w, st);
  const int64_t all = round_up(j.classes, kPad);
  if (e == hipSuccess && j.dw.p) e = transpose<T>(j.x, j.rows, j.dim, p.rows_pad, j.labels, j.classes, nullptr, ws + p.xt, st);
  if (e == hipSuccess && j.dx.p) e = transpose<T>(j.w, j.classes, j.dim, all, nullptr, 0, j.bias, ws + p.wt, st);
  for (int64_t i = 0; e == hipSuccess && i < p.pieces; ++i) {
    const int64_t first = i * p.piece, left = j.classes - first, mine = std::min(left, p.piece);
    const int64_t wide = round_up(mine, kPad);       // columns of G that are written
    a.w = w;
    a.w.p = w.p + first * w.ld;
    a.w.last = left - 1;
    a.bias = j.bias ? j.bias + first : nullptr;
    a.rows = j.rows;
    a.classes = left;
    a.lse = j.lse;
    a.dloss = j.dloss;
    a.labels = j.labels;
    a.scale = j.scale;
    a.first = first;
    a.all_classes = j.classes;
    a.g = ws + p.g;
    a.gt = j.dw.p ? ws + p.gt : nullptr;
    a.g_ld = p.piece;
    a.gt_ld = p.rows_pad;
    a.part_bias = j.dbias ? (float*)(ws + p.bias) : nullptr;
    Pass grad = p.grad;
    grad.tn = tiles_of(wide, grad.large ? Tiles<T>::Large::BN : Tiles<T>::Small::BN);
    e = logits<T, true>(a, grad, st);
    if (e != hipSuccess) return e;
    if (j.dx.p) {
      ProductArgs b{};
      b.a = {ws + p.g, p.piece * (int64_t)sizeof(T), p.rows_pad - 1, nullptr, 0};
      b.b = {ws + p.wt + first * (int64_t)sizeof(T), all * (int64_t)sizeof(T), j.dim - 1, nullptr, 0};
      b.c = ws + p.dx;
      b.ldc = part_ld(j.dim);
      b.m = j.rows;
      b.n = j.dim;
      b.add = i > 0;
      Pass t = p.to_x;
      t.steps = (int)(wide / kStep<T>);
      // the last piece may have fewer steps than parts: every part of the sums
      // has been written by then
      t.per = (t.steps + t.parts - 1) / t.parts;
      if (i > 0) t.parts = (t.steps + t.per - 1) / t.per;
      e = times<T, float>(b, t, st);
      if (e != hipSuccess) return e;
    }
    if (j.dw.p) {
      ProductArgs b{};
      b.a = {ws + p.gt, p.rows_pad * (int64_t)sizeof(T), wide - 1, nullptr, 0};
      b.b = {ws + p.xt, p.rows_pad * (int64_t)sizeof(T), j.dim - 1, nullptr, 0};
      b.m = mine;
      b.n = j.dim;
      Pass t = p.to_w;
      t.tm = tiles_of(mine, t.large ? Tiles<T>::Large::BM : Tiles<T>::Small::BM);
      const Mat out = {(T*)j.dw.p + first * j.dw.ld, j.dw.ld};
      if (t.parts == 1) {
        b.c = out.p;
        b.ldc = out.ld;
        e = times<T, T>(b, t, st);
      } else {
        b.c = ws + p.dw;
        b.ldc = part_ld(j.dim);
        e = times<T, float>(b, t, st);
        if (e == hipSuccess) e = join<T>((const float*)(ws + p.dw), t.parts, mine, j.dim, nullptr, 0, out, st);
      }
      if (e != hipSuccess) return e;
    }
    if (j.dbias) {
      const BiasArgs b{(const float*)(ws + p.bias), j.dbias + first, p.piece, mine, (int)grad.tm};
      e = enqueue(k_bias, dim3((unsigned)tiles_of(mine, kThreads)), dim3(kThreads), 0, st, b);
    }
  }
  if (e == hipSuccess && j.dx.p)
    e = join<T>((const float*)(ws + p.dx), p.to_x.parts, j.rows, j.dim, nullptr, 0, j.dx, st);
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

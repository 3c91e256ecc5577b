// Orthogonalised matrices by Newton-Schulz products, and the update step that takes them.
//
// A list of matrices goes through the same launches together: sizes, two for each matrix's norm and its parts of 16 bits, and
// three products a step.  Matrices with more rows than columns are transposed when they are split and when the result
// leaves, so that every X is m x n, m <= n.
//
// Numbers of 32 bits are held as two of f16, the second what the first leaves, of which matrix instructions take the first
// (or, exact, first by first, first by second and second by first).  f16 and not bf16: three more bits at the same rate.  Why two
// parts where products are of the first alone: an update's small singular values grow by a each step, 485 times over five, and
// so does what rounding X leaves in their directions, unless a X is taken of the whole X; the rounding of a product's operands
// stays within the directions that the product has.  Worked out against 64 bits (a matrix of 8 large directions and a hundredth
// of noise, 384 x 1,024): 3.7e-2 with X in one part, 1.2e-3 with two.
#include "train_tiles.h"

#include <float.h>
#include <math.h>

#include <vector>

namespace fbx {
namespace train {
namespace {

typedef _Float16 f16;
constexpr uint32_t kMatrices = 32;        // of a launch
constexpr uint32_t kDepth = kStepBytes / sizeof(f16);
constexpr uint32_t kMostPartials = 256;   // of a matrix's sum of squares
constexpr int kX = 14;                    // X is held times 2^14, but for the first
constexpr float kSecond = 2048.f;         // second parts are held times this, so that they keep their 11 bits beside first parts near f16's end

// One matrix of a launch: what it is made of, where its result goes, and its scratch.
struct Matrix {
  const void* u;                          // the matrix, or a gradient
  float* m;                               // a gradient's momentum, or null
  void *out, *copy;                       // the result, or the weights
  uint64_t ld_u, ld_out;
  char* scratch;
  float step;                             // the result's factor (lr times the matrix's, or 1)
  uint32_t rows, columns;                 // of what is given
  uint32_t tall, m_side, n_side, wide_m, wide_n;  // of X: m x n; rows of either side made up to whole steps of depth
  uint32_t chunk, partials;               // elements whose squares a workgroup adds up; workgroups
  uint32_t exact;                         // products of both parts
  uint32_t at_norm, at_x, at_a;           // places in scratch, in units of 256 bytes (a, then b)

  __device__ f16* x(uint32_t turn, uint32_t part) const { return (f16*)(scratch + (uint64_t)at_x * 256u) + (uint64_t)(turn * 2u + part) * m_side * wide_n; }
  __device__ f16* a(uint32_t part) const { return (f16*)(scratch + (uint64_t)at_a * 256u) + (uint64_t)part * m_side * wide_m; }
  __device__ f16* b(uint32_t part) const { return a(2u + part); }
  __device__ double* squares() const { return (double*)(scratch + (uint64_t)at_norm * 256u); }
  __device__ float* factor() const { return (float*)(squares() + kMostPartials); }   // X = what is held first, times this
};

struct List {
  Matrix of[kMatrices];
  uint32_t first[kMatrices + 1];          // the first workgroup (or tile) of each
  uint32_t n;

  // The matrix that a workgroup is of: all of `first` is looked at at once, a lane each.  (A search among them waits for the arguments'
  // memory once a step, microseconds in all.)
  __device__ uint32_t find(uint32_t block) const {
    const uint32_t lane = threadIdx.x % 64u, begins = lane < n ? first[lane] : 0xffffffffu;
    return (uint32_t)__popcll(__ballot(begins <= block)) - 1u;
  }
};

// What is made of a gradient, and of a norm.
struct Given {
  uint32_t nesterov;
  float momentum, grad_scale;
  double eps;
};
struct PrepareArgs {
  List list;
  Given given;
};

// How results leave.
struct Leaving {
  uint32_t out, copy, weights;            // types; results go into weights
  float decay;                            // of them: 1 - lr weight_decay
};

// Eight adjacent elements from i on, of which the first n exist (more exist behind them where n is 8), wherever they begin.
template <class X>
__device__ __forceinline__ void fetch(float (&to)[8], const X* from, uint32_t n) {
  Pack<X, 8> p = {};
  if (n >= 8u) {
    __builtin_memcpy(&p, from, sizeof p);
  } else {
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e)
      if (e < n) p.v[e] = from[e];
  }
#pragma unroll
  for (uint32_t e = 0; e < 8u; ++e) to[e] = (float)p.v[e];
}

// Sum over a workgroup of 256 lanes, in all of them.
__device__ __forceinline__ double sum_of(double v, double* shared) {
#pragma unroll
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d, 64);
  if (threadIdx.x % 64u == 0u) shared[threadIdx.x / 64u] = v;
  __syncthreads();
  return (shared[0] + shared[1]) + (shared[2] + shared[3]);
}

// The power of two that brings a norm into [2^13, 2^14), and the factor that then makes X of a matrix: 1 / (norm + eps).  A matrix of zeros
// stays one, one that is not finite becomes NaN.
__device__ __forceinline__ int power_of(double norm) {
  if (!(norm > 0 && norm <= DBL_MAX)) return 0;
  int e;
  (void)frexp(norm, &e);   // norm in [2^(e - 1), 2^e)
  return kX - e;
}
__device__ __forceinline__ float factor_of(double norm, int k2, double eps) {
  return norm == 0 ? 0.f : norm <= DBL_MAX ? (float)(1.0 / ldexp(norm + eps, k2)) : __builtin_nanf("");
}

// Sums of squares, in 64 bits so that they stay within range whatever the gradient's size; momentum is brought up to date.
// A workgroup adds up `chunk` elements.  Three matrices of 10.7 M elements with momentum, 10 bytes each: 73 us, 4.4 TB/s.
template <class G, bool kGiven>
__global__ __launch_bounds__(256) void k_measure(PrepareArgs) {
#pragma clang fp contract(off)
  const PrepareArgs& p = launch_args<PrepareArgs>();
  const uint32_t which = same(p.list.find(blockIdx.x));
  const Matrix& t = p.list.of[which];
  const uint32_t part = blockIdx.x - p.list.first[which];
  const uint64_t all = (uint64_t)t.rows * t.columns, from = (uint64_t)part * t.chunk, to = from + t.chunk < all ? from + t.chunk : all;
  double sum = 0;
  if (kGiven || t.ld_u == t.columns) {
    for (uint64_t i = from + threadIdx.x * 8u; i < to; i += 2048u) {
      const uint32_t n = to - i < 8u ? (uint32_t)(to - i) : 8u;
      float u[8];
      fetch(u, (const G*)t.u + i, n);
      if (kGiven) {
        float m[8];
        fetch(m, t.m + i, n);
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e) {
          const float g = u[e] * p.given.grad_scale;
          m[e] = m[e] * p.given.momentum + g;
          u[e] = p.given.nesterov ? g + m[e] * p.given.momentum : m[e];
        }
        if (n == 8u) {
          __builtin_memcpy(t.m + i, m, sizeof m);
        } else {
#pragma unroll
          for (uint32_t e = 0; e < 8u; ++e)
            if (e < n) t.m[i + e] = m[e];
        }
      }
#pragma unroll
      for (uint32_t e = 0; e < 8u; ++e) sum += (double)u[e] * u[e];   // (zeros behind the last)
    }
  } else {
    for (uint64_t i = from + threadIdx.x; i < to; i += 256u) {
      const float u = (float)((const G*)t.u)[i / t.columns * t.ld_u + i % t.columns];
      sum += (double)u * u;
    }
  }
  __shared__ double sums[4];
  sum = sum_of(sum, sums);
  if (threadIdx.x == 0u) t.squares()[part] = sum;
}

// The matrix's parts of 16 bits, times the power of two that brings its norm into [2^13, 2^14): one times 2^14 for the
// steps that follow, and the factor that makes X of it.  A workgroup takes 64 x 64 elements of X (zeros beyond them).  The
// same three matrices: 54 us, 5.9 TB/s (part of it out of the last-level cache).
constexpr uint32_t kSquare = 64;
template <class G, bool kGiven>
__global__ __launch_bounds__(256) void k_split(PrepareArgs) {
#pragma clang fp contract(off)
  const PrepareArgs& p = launch_args<PrepareArgs>();
  const uint32_t which = same(p.list.find(blockIdx.x));
  const Matrix& t = p.list.of[which];
  const uint32_t tile = blockIdx.x - p.list.first[which], across = t.wide_n / kSquare, r0 = tile / across * kSquare, c0 = tile % across * kSquare;
  __shared__ double sums[4];
  __shared__ float turned[kSquare][kSquare + 1];
  const double square = threadIdx.x < t.partials ? t.squares()[threadIdx.x] : 0.0;
  const uint32_t line = threadIdx.x / 8u, place = threadIdx.x % 8u * 8u;   // lines `line` and `line` + 32 of the tile, eight elements of each
  // a tile of what is given has the rows of X, or its columns, for rows
  const uint32_t row0 = (t.tall ? c0 : r0) + line, column = (t.tall ? r0 : c0) + place;
  float u[2][8];
#pragma unroll
  for (uint32_t k = 0; k < 2u; ++k) {
    const uint32_t row = row0 + 32u * k, n = row >= t.rows || column >= t.columns ? 0u : t.columns - column < 8u ? t.columns - column : 8u;
    const uint64_t i = (uint64_t)(row < t.rows ? row : 0u) * t.ld_u + column;
    fetch(u[k], (const G*)t.u + i, n);
    if (kGiven) {
      float m[8];
      fetch(m, t.m + i, n);
#pragma unroll
      for (uint32_t e = 0; e < 8u; ++e) u[k][e] = p.given.nesterov ? u[k][e] * p.given.grad_scale + m[e] * p.given.momentum : m[e];
    }
  }
  const double norm = sqrt(sum_of(square, sums));
  const int k2 = power_of(norm);
  if (tile == 0u && threadIdx.x == 0u) *t.factor() = factor_of(norm, k2, p.given.eps);
  if (t.tall) {
#pragma unroll
    for (uint32_t k = 0; k < 2u; ++k)
#pragma unroll
      for (uint32_t e = 0; e < 8u; ++e) turned[line + 32u * k][place + e] = u[k][e];
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < 2u; ++k)
#pragma unroll
      for (uint32_t e = 0; e < 8u; ++e) u[k][e] = turned[place + e][line + 32u * k];
  }
#pragma unroll
  for (uint32_t k = 0; k < 2u; ++k) {
    const uint32_t r = r0 + line + 32u * k;
    if (r >= t.m_side) continue;
    const uint64_t at = (uint64_t)r * t.wide_n + c0 + place;
    Pack<f16, 8> high, low;
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e) {
      const float v = ldexpf(u[k][e], k2);
      high.v[e] = (f16)v;
      low.v[e] = (f16)((v - (float)high.v[e]) * kSecond);
    }
    *(Pack<f16, 8>*)(t.x(0, 0) + at) = high;
    *(Pack<f16, 8>*)(t.x(0, 1) + at) = low;
  }
}

// One launch's products, of every matrix of the list:
//   kGram     A = X X^T
//   kPolynom  B = a I + b A + c A A (A is its own transpose)
//   kNext     X = B X, into the other of two places
//   kLast     the same, and it leaves as the result, or goes into the weights
// The a X of a step is part of the product so that X need not be read again behind it (8 bytes an element in place of 4 are more than a
// tenth of a large product's time); where products are of first parts only a times X's second part is added.
enum Form { kGram, kPolynom, kNext, kLast };
struct ProductArgs {
  List list;
  uint32_t turn;                          // which X is read
  uint32_t begins;                        // X is what k_split left
  float keep, sum, diagonal;              // C = keep (what is there) + sum (the product) + diagonal I, but for the scale of the first X
  Leaving last;
};

typedef f16 f16x4 __attribute__((ext_vector_type(4)));
struct Halves {
  f16x4 high, low;
  __device__ explicit Halves(f32x4 v, float second = kSecond) {
    // (what v was made of may not be rounded to f16 at once where the first part is stored, and by way of 32 bits where it is taken off: now
    // and then the two are a unit apart, and the second part is then that much wrong)
    asm("" : "+v"(v));
    high = __builtin_convertvector(v, f16x4);
    low = __builtin_convertvector((v - __builtin_convertvector(high, f32x4)) * second, f16x4);
  }
};

// The result's elements of row r of X at four columns from c0 on, and from every 16th further on: as they are, or into the weights.
template <class P, int kNF>
__device__ __forceinline__ void leave(const Leaving& p, const Matrix& t, uint32_t r, uint32_t c0, const f32x4 (&v)[kNF]) {
  if (r >= t.m_side) return;
  float old[kNF][4] = {};
  const bool tall = t.tall != 0u;
  const uint64_t step = tall ? t.ld_out : 1u, base = tall ? r : r * t.ld_out;   // from column to column of X
  P* to = (P*)t.out + base;
  if (p.weights)
#pragma unroll
    for (int j = 0; j < kNF; ++j)
#pragma unroll
      for (uint32_t e = 0; e < 4u; ++e) {
        const uint32_t c = c0 + j * 16 + e;
        old[j][e] = (float)to[(c < t.n_side ? c : 0u) * step];
      }
#pragma unroll
  for (int j = 0; j < kNF; ++j) {
    const uint32_t c = c0 + j * 16;
    float o[4];
#pragma unroll
    for (uint32_t e = 0; e < 4u; ++e) {
      o[e] = v[j][e] * t.step;
      if (p.weights) o[e] = old[j][e] * p.decay - o[e];
    }
    if (!tall && c + 4u <= t.n_side) {
      const Pack<P, 4> w = {{(P)o[0], (P)o[1], (P)o[2], (P)o[3]}};
      __builtin_memcpy(to + c, &w, sizeof w);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 4u; ++e)
        if (c + e < t.n_side) to[(c + e) * step] = (P)o[e];
    }
    if (!t.copy) continue;
    auto copy = [&](auto like) __attribute__((always_inline)) {
      typedef decltype(like) C;
      C* there = (C*)t.copy + base;
#pragma unroll
      for (uint32_t e = 0; e < 4u; ++e)
        if (c + e < t.n_side) there[(c + e) * step] = (C)o[e];
    };
    if (p.copy == FBX_F16) copy((f16)0.f);
    else copy((__bf16)0.f);
  }
}

// BM x BN of C a workgroup, its WM x WN wavefronts side by side.  C's rows come from A; its columns from B, which is the first side
// of the matrix instructions, so that a lane holds four adjacent columns of a row.  Of a symmetric C tiles on and below the
// diagonal are worked out, and stored on either side of it.  kStages: steps whose tiles are in LDS or on their way there.
// Two of 2,624 x 4,096, products of first parts: A 70 to 76 us, B 53 to 57, X 150 to 163: 0.77, 0.66 and 0.72 PFLOP/s of what is needed; a library's
// product takes 59 us for each X, without a X and without storing two parts (0.95 PFLOP/s).  Of both parts: A 163 to 192, B 129 to 134, X 336 to 370.  In tiles of 128 two workgroups on a
// compute unit take 0.9 us for a step, of which reading and filling LDS is 0.73; 2 to 3 us before the first step and 6 to 8 behind the last (when all
// of them store at once) come on top, and the last of 2.6 rounds leaves units idle.  Measured and not faster: tiles of 256 x 128 by eight wavefronts
// with three steps in LDS (157 to 166), wavefronts that have a SIMD to themselves and read a quarter to a half less from LDS
// (128 x 64: 190 and 212; 128 x 128: spills), rows of X a line of memory further apart (the same), five steps in LDS for small tiles (the
// same), a transposed result by way of LDS (the same: kLast waits for the weights' memory).
template <Form kForm, int BM, int BN, int WM, int WN, int kStages, bool kExact>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_product(ProductArgs) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr bool kBoth = kExact && BM == 64;   // both parts of a step are brought into LDS together
  constexpr bool kTwin = kForm == kGram || kForm == kPolynom;
  constexpr int kWaves = WM * WN, kRows = BM / WM, kCols = BN / WN, kMF = kRows / 16, kNF = kCols / 16;
  typedef Tile<f16, BM, kWaves, false> TileA;
  typedef Tile<f16, BN, kWaves, !kTwin> TileB;
  __shared__ alignas(1024) char a0[BM * kStepBytes], b0[BN * kStepBytes], a1[BM * kStepBytes], b1[BN * kStepBytes];
  __shared__ alignas(1024) char a2[kStages > 2 ? BM * kStepBytes : 16], b2[kStages > 2 ? BN * kStepBytes : 16];
  __shared__ alignas(1024) char a3[kStages > 2 ? BM * kStepBytes : 16], b3[kStages > 2 ? BN * kStepBytes : 16];
  // kBoth: second parts
  __shared__ alignas(1024) char c0[kBoth ? BM * kStepBytes : 16], d0[kBoth ? BN * kStepBytes : 16], c1[kBoth ? BM * kStepBytes : 16], d1[kBoth ? BN * kStepBytes : 16];
  static_assert(!kBoth || kStages == 2, "");
  const ProductArgs& p = launch_args<ProductArgs>();
  const uint32_t lane = threadIdx.x % 64u, wave = same(threadIdx.x / 64u), wm = wave % WM, wn = wave / WM;
  uint32_t at;
  {  // workgroups go to the eight dies in turn: each die takes a stretch of the tiles
    const uint32_t n = gridDim.x, each = n / 8u, more = n % 8u, die = blockIdx.x % 8u;
    at = die * each + (die < more ? die : more) + blockIdx.x / 8u;
  }
  const uint32_t which = same(p.list.find(at));
  const Matrix& t = p.list.of[which];
  at -= p.list.first[which];
  uint32_t row0, col0;
  if (kTwin) {  // the i-th row of tiles has i + 1
    uint32_t i = (uint32_t)((__builtin_sqrtf(8.f * (float)at + 1.f) - 1.f) * 0.5f);
    while (i * (i + 1u) / 2u > at) --i;
    while ((i + 1u) * (i + 2u) / 2u <= at) ++i;
    row0 = same(i * BM);
    col0 = same((at - i * (i + 1u) / 2u) * BN);
  } else {      // eight row tiles wide, down the columns
    const uint32_t row_tiles = (t.m_side + BM - 1u) / BM, column_tiles = (t.n_side + BN - 1u) / BN;
    const uint32_t band = at / (8u * column_tiles), in_band = at - band * 8u * column_tiles, high = row_tiles - band * 8u < 8u ? row_tiles - band * 8u : 8u;
    row0 = same((band * 8u + in_band % high) * BM);
    col0 = same(in_band / high * BN);
  }
  const uint32_t m_side = same(t.m_side), wide_a = same(kForm == kGram ? t.wide_n : t.wide_m), wide_b = same(kForm == kPolynom ? t.wide_m : t.wide_n);
  const uint64_t ld_a = wide_a * 2u, ld_b = wide_b * 2u;
  const uint32_t each = wide_a / kDepth, end = kExact && !kBoth ? 3u * each : each;   // steps: of one product of parts, of all
  const char* of_a = (const char*)(kForm == kGram ? t.x(p.turn, 0) : kForm == kPolynom ? t.a(0) : t.b(0));
  const char* of_b = (const char*)(kForm == kPolynom ? t.a(0) : t.x(p.turn, 0));
  const uint64_t part_a = (uint64_t)m_side * ld_a, part_b = (uint64_t)m_side * ld_b;
  of_a += (uint64_t)row0 * ld_a;
  of_b += kTwin ? (uint64_t)col0 * ld_b : (uint64_t)col0 * 2u;
  TileA ta;
  TileB tb;
  ta.begin(wave, lane, ld_a, 0);
  tb.begin(wave, lane, ld_b, wide_b - col0);
  // (behind the last step: of nothing, so that every step's loads are as many)
  auto load_part = [&](char* to_a, char* to_b, uint32_t s, uint32_t k, bool second_a, bool second_b) __attribute__((always_inline)) {
    const bool none = s >= end;
    const char *a = of_a + (second_a ? part_a : 0u), *b = of_b + (second_b ? part_b : 0u);
    const uint32_t left = wide_a - k * kDepth;
    ta.load((lds_char*)to_a, a + (uint64_t)k * kStepBytes, ld_a, none ? 0u : m_side - row0, left, left * 2u, wave);
    if (kTwin) tb.load((lds_char*)to_b, b + (uint64_t)k * kStepBytes, ld_b, none ? 0u : m_side - col0, left, left * 2u, wave);
    else tb.load((lds_char*)to_b, b + (uint64_t)k * kDepth * ld_b, ld_b, none || m_side <= k * kDepth ? 0u : m_side - k * kDepth, 0, (wide_b - col0) * 2u, wave);
  };

  auto load = [&](char* to_a, char* to_b, uint32_t s) __attribute__((always_inline)) {
    const uint32_t pair = kBoth || !kExact ? 0u : s < each ? 2u : s < 2u * each ? 1u : 0u;  // second by first, first by second, first by first
    load_part(to_a, to_b, s, kBoth || !kExact ? s : s - (2u - pair) * each, pair == 2u, pair == 1u);
    if constexpr (kBoth) load_part(to_a == a0 ? c0 : c1, to_b == b0 ? d0 : d1, s, s, true, true);
  };

  // Two halves of a step's depth in turn: while one is multiplied out of registers the other's rows are read from LDS.
  // A step's barrier lies between the halves: behind it the next step's tile is there and nobody reads this step's any more, so
  // the loads of the step kStages later go there.
  f32x4 sum[kMF][kNF] = {}, second[kBoth ? kMF : 1][kBoth ? kNF : 1] = {};
  constexpr int kParts = kBoth ? 2 : 1;
  typename Frag<f16>::type fa[2][kParts][kMF], fb[2][kParts][kNF];
  auto read = [&](int part, const char* in_a, const char* in_b) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
      const char *from_a = q ? (in_a == a0 ? c0 : c1) : in_a, *from_b = q ? (in_b == b0 ? d0 : d1) : in_b;
#pragma unroll
      for (int i = 0; i < kMF; ++i) fa[part][q][i] = TileA::read((const lds_char*)from_a, wm * kRows + i * 16, part, lane);
#pragma unroll
      for (int j = 0; j < kNF; ++j) fb[part][q][j] = TileB::read((const lds_char*)from_b, wn * kCols + j * 16, part, lane);
    }
  };
  auto multiply = [&](int part) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kNF; ++j)
#pragma unroll
      for (int i = 0; i < kMF; ++i) {
        sum[i][j] = mma(fb[part][0][j], fa[part][0][i], sum[i][j]);
        if constexpr (kBoth) {
          second[i][j] = mma(fb[part][1][j], fa[part][0][i], second[i][j]);
          second[i][j] = mma(fb[part][0][j], fa[part][1][i], second[i][j]);
        }
      }
  };
  auto arrived = [](auto steps) {
    constexpr int n = decltype(steps)::value * (TileA::kLoads + TileB::kLoads) * kParts;
    static_assert(n < 64, "");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((n & 15) | (n >> 4) << 14 | 0x0070);  // (vmcnt n, lgkmcnt 0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](char* at_a, char* at_b, const char* next_a, const char* next_b, uint32_t s) __attribute__((always_inline)) {
    read(1, at_a, at_b);
    multiply(0);
    arrived(Kind<kStages - 2>());
    load(at_a, at_b, s + kStages);
    __builtin_amdgcn_sched_barrier(0);
    read(0, next_a, next_b);  // (behind the last step: what is there, unused)
    multiply(1);
    __builtin_amdgcn_sched_barrier(0);
  };
  load(a0, b0, 0);
  load(a1, b1, 1);
  if constexpr (kStages == 4) {
    load(a2, b2, 2);
    load(a3, b3, 3);
  }
  arrived(Kind<kStages - 1>());
  read(0, a0, b0);
  if constexpr (kStages == 4) {
    for (uint32_t s = 0;; s += 4) {
      step(a0, b0, a1, b1, s);
      if (s + 1 >= end) break;
      step(a1, b1, a2, b2, s + 1);
      if (s + 2 >= end) break;
      step(a2, b2, a3, b3, s + 2);
      if (s + 3 >= end) break;
      step(a3, b3, a0, b0, s + 3);
      if (s + 4 >= end) break;
    }
  } else {
    auto steps = [&](uint32_t from, uint32_t to) __attribute__((always_inline)) {
      for (uint32_t s = from; s < to; s += 2) {
        step(a0, b0, a1, b1, s);
        if (s + 1 < to) step(a1, b1, a0, b0, s + 1);
      }
    };
    if constexpr (kExact && !kBoth) {  // (the products of second parts first, an even number of steps)
      steps(0, 2u * each);
#pragma unroll
      for (int i = 0; i < kMF; ++i)
#pragma unroll
        for (int j = 0; j < kNF; ++j) sum[i][j] *= 1.f / kSecond;
      steps(2u * each, end);
    } else {
      steps(0, end);
    }
  }
  if constexpr (kBoth)
#pragma unroll
    for (int i = 0; i < kMF; ++i)
#pragma unroll
      for (int j = 0; j < kNF; ++j) sum[i][j] += second[i][j] * (1.f / kSecond);
  arrived(Kind<0>());  // (nothing is to land in LDS that may be another workgroup's by then)

  // The first X is held times 1 / f, every other one times 2^14.
  const float f = p.begins ? *t.factor() : 1.f;
  const float keep = p.keep * (kForm == kPolynom ? 1.f : f), product = p.sum * (kForm == kGram ? f * f : kForm == kPolynom ? 1.f : f);
  constexpr int kAtOnce = 16 / kNF < kMF ? 16 / kNF : kMF;   // 16 rows each, whose other operand is asked for together
  const uint32_t r_first = row0 + wm * kRows + lane % 16u, c_first = col0 + wn * kCols + lane / 16u * 4u;
  if constexpr (kTwin) {
    f16 *high = kForm == kGram ? t.a(0) : t.b(0), *low = kForm == kGram ? t.a(1) : t.b(1);
    const uint32_t wide = t.wide_m;
#pragma unroll
    for (int i0 = 0; i0 < kMF; i0 += kAtOnce) {
      Pack<f16, 4> there[kAtOnce][kNF][2] = {};
      if (kForm == kPolynom)
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
          for (int j = 0; j < kNF; ++j) {
            const uint32_t r = r_first + (i0 + i) * 16, c = c_first + j * 16;
            const uint64_t from = (uint64_t)(r < m_side ? r : m_side - 1u) * wide + (c < wide ? c : 0u);
            there[i][j][0] = *(const Pack<f16, 4>*)(t.a(0) + from);
            if (kExact) there[i][j][1] = *(const Pack<f16, 4>*)(t.a(1) + from);
          }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
        for (int j = 0; j < kNF; ++j) {
          const uint32_t r = r_first + (i0 + i) * 16, c = c_first + j * 16;
          f32x4 v = sum[i0 + i][j] * product;
          if (kForm == kPolynom)
#pragma unroll
            for (uint32_t e = 0; e < 4u; ++e) v[e] += ((float)there[i][j][0].v[e] + (float)there[i][j][1].v[e] * (1.f / kSecond)) * keep + (r == c + e && r < m_side ? p.diagonal : 0.f);
          const Halves w(v);
          const uint64_t to = (uint64_t)r * wide + c;
          if (r < m_side && c < wide) {
            *(f16x4*)(high + to) = w.high;
            if (kExact) *(f16x4*)(low + to) = w.low;
          }
          if (row0 != col0 && r < wide) {   // (columns are before the diagonal's tile, so within the rows; rows beyond the last are zeros)
#pragma unroll
            for (uint32_t e = 0; e < 4u; ++e) {
              high[(uint64_t)(c + e) * wide + r] = r < m_side ? w.high[e] : (f16)0.f;
              if (kExact) low[(uint64_t)(c + e) * wide + r] = r < m_side ? w.low[e] : (f16)0.f;
            }
          }
        }
    }
  } else {
    const f16* second = t.x(p.turn, 1);
    const uint32_t wide = t.wide_n;
    auto finish = [&](auto use) __attribute__((always_inline)) {
#pragma unroll
      for (int i0 = 0; i0 < kMF; i0 += kAtOnce) {
        Pack<f16, 4> there[kAtOnce][kNF] = {};
        if (!kExact)
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
            for (int j = 0; j < kNF; ++j) {
              const uint32_t r = r_first + (i0 + i) * 16, c = c_first + j * 16;
              there[i][j] = *(const Pack<f16, 4>*)(second + (uint64_t)(r < m_side ? r : m_side - 1u) * wide + (c < wide ? c : 0u));
            }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
          for (int j = 0; j < kNF; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[i0 + i][j][e] = sum[i0 + i][j][e] * product + (float)there[i][j].v[e] * keep;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) use(i0 + i, sum[i0 + i]);
      }
    };
    if constexpr (kForm == kNext) {
      f16 *high = t.x(p.turn ^ 1u, 0), *low = t.x(p.turn ^ 1u, 1);
      finish([&](int i, const f32x4 (&v)[kNF]) __attribute__((always_inline)) {
        const uint32_t r = r_first + i * 16;
#pragma unroll
        for (int j = 0; j < kNF; ++j) {
          const uint32_t c = c_first + j * 16;
          if (r >= m_side || c >= wide) continue;
          const Halves w(v[j]);
          const uint64_t to = (uint64_t)r * wide + c;
          *(f16x4*)(high + to) = w.high;
          *(f16x4*)(low + to) = w.low;
        }
      });
    } else {
      if (p.last.out == FBX_F32) finish([&](int i, const f32x4 (&v)[kNF]) __attribute__((always_inline)) { leave<float, kNF>(p.last, t, r_first + i * 16, c_first, v); });
      else if (p.last.out == FBX_F16) finish([&](int i, const f32x4 (&v)[kNF]) __attribute__((always_inline)) { leave<f16, kNF>(p.last, t, r_first + i * 16, c_first, v); });
      else finish([&](int i, const f32x4 (&v)[kNF]) __attribute__((always_inline)) { leave<__bf16, kNF>(p.last, t, r_first + i * 16, c_first, v); });
    }
  }
#endif
}

// A matrix that one workgroup's LDS holds: everything in one launch, a matrix a workgroup, where every product of its own would take
// the others' launches and ways through memory.  Products are of both parts.  X and A (and B in its place) lie in LDS as two
// parts each, rows 16 bytes longer than they need be so that those a read takes lie in different banks; a wavefront takes 32 x 32 of
// a product at a time, up to kBlocks of them, and what it worked out replaces an operand when all are done with it.
// All four products of the parts are added up, the smallest first: second by second too, which costs 3 us, as the second parts are not held
// larger here and a small matrix's errors average out least (five steps from
// 64 bits: 16 x 16 7.7e-7 -> 5.5e-7, 128 x 96 1.3e-6 -> 1.1e-6; products in 32 bits: 6.6e-7, 1.2e-6).
// One of 128 x 96, five steps: 41 us, where 17 launches took 98.  A step is 8 us: three products of which
// LDS's reads are 3, and as much for splitting and storing what they give, sixteen wavefronts sharing four SIMDs.
constexpr uint32_t kSmallLanes = 1024, kRoom = 158 * 1024;
constexpr int kBlocks = 2;
struct StepNumbers {
  float gram, keep, square, diagonal, next;
};
struct SmallArgs {
  List list;
  Given given;
  Leaving last;
  uint32_t steps;
  StepNumbers of[64];
};
__host__ __device__ inline uint32_t small_side(uint32_t n) { return (n + 31u) / 32u * 32u; }
__host__ __device__ inline uint32_t small_line(uint32_t n) { return 2u * n + 16u; }   // bytes of a row

template <class G>
__global__ __launch_bounds__(kSmallLanes) void k_small(SmallArgs) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef Frag<f16>::type F;
  __shared__ alignas(1024) char lds[kRoom];
  __shared__ double sums[kSmallLanes / 64];
  const SmallArgs& p = launch_args<SmallArgs>();
  const Matrix& t = p.list.of[blockIdx.x];
  const uint32_t lane = threadIdx.x % 64u, wave = same(threadIdx.x / 64u);
  uint32_t i = lane % 16u, g = lane / 16u;
  const uint32_t m_side = same(t.m_side), n_side = same(t.n_side), rows = small_side(m_side), columns = small_side(n_side);
  const uint32_t line_x = small_line(columns), line_a = small_line(rows), part_x = rows * line_x, part_a = rows * line_a;
  lds_char *x = (lds_char*)lds, *a = x + 2u * part_x;

  for (uint32_t at = threadIdx.x * 16u; at < 2u * (part_x + part_a); at += kSmallLanes * 16u) *(__attribute__((address_space(3))) f32x4*)(x + at) = f32x4{0.f, 0.f, 0.f, 0.f};
  __syncthreads();
  // An element's 32 bits wait for the norm in the two places of its parts.
  typedef __attribute__((address_space(3))) uint16_t Half;
  const uint32_t all = t.rows * t.columns, most = t.columns;
  const uint32_t further_r = kSmallLanes / most, further_c = kSmallLanes % most;
  auto place = [&](uint32_t r, uint32_t c) { return x + (t.tall ? c : r) * line_x + (t.tall ? r : c) * 2u; };
  double square = 0;
  {
#pragma clang fp contract(off)
    constexpr uint32_t kAtOnce = 4;
    uint32_t r[kAtOnce], c[kAtOnce];
    r[0] = threadIdx.x / most;
    c[0] = threadIdx.x % most;
    for (uint32_t at = threadIdx.x; at < all; at += kAtOnce * kSmallLanes) {
      float u[kAtOnce], m[kAtOnce];
#pragma unroll
      for (uint32_t e = 0; e < kAtOnce; ++e) {
        if (e) {
          r[e] = r[e - 1] + further_r;
          c[e] = c[e - 1] + further_c;
          if (c[e] >= most) {
            c[e] -= most;
            ++r[e];
          }
        }
        const uint32_t there = r[e] < t.rows ? r[e] : 0u;   // (beyond the last element: one that is there)
        u[e] = (float)((const G*)t.u)[there * t.ld_u + c[e]];
        if (t.m) m[e] = t.m[there * most + c[e]];
      }
#pragma unroll
      for (uint32_t e = 0; e < kAtOnce; ++e) {
        if (at + e * kSmallLanes >= all) continue;
        float v = u[e];
        if (t.m) {
          const float grad = v * p.given.grad_scale, now = m[e] * p.given.momentum + grad;
          t.m[r[e] * most + c[e]] = now;
          v = p.given.nesterov ? grad + now * p.given.momentum : now;
        }
        square += (double)v * v;
        lds_char* to = place(r[e], c[e]);
        *(Half*)to = (uint16_t)(__float_as_uint(v) >> 16);
        *(Half*)(to + part_x) = (uint16_t)__float_as_uint(v);
      }
      r[0] = r[kAtOnce - 1] + further_r;
      c[0] = c[kAtOnce - 1] + further_c;
      if (c[0] >= most) {
        c[0] -= most;
        ++r[0];
      }
    }
  }
#pragma unroll
  for (int d = 32; d; d /= 2) square += __shfl_xor(square, d, 64);
  if (lane == 0u) sums[wave] = square;
  __syncthreads();
  square = 0;
#pragma unroll
  for (uint32_t w = 0; w < kSmallLanes / 64u; ++w) square += sums[w];
  const double norm = sqrt(square);
  const int k2 = power_of(norm);
  const float f = factor_of(norm, k2, p.given.eps);
  for (uint32_t at = threadIdx.x * 2u; at < part_x; at += kSmallLanes * 2u) {   // (zeros stay zeros)
    lds_char* to = x + at;
    const float v = ldexpf(__uint_as_float((uint32_t)*(Half*)to << 16 | *(Half*)(to + part_x)), k2);
    const f16 high = (f16)v;
    *(__attribute__((address_space(3))) f16*)to = high;
    *(__attribute__((address_space(3))) f16*)(to + part_x) = (f16)(v - (float)high);
  }
  __syncthreads();

  // 16 rows from `first` on over 32 of depth from k on: along rows, or across them (a transposing read).
  auto along = [&](const lds_char* from, uint32_t line, uint32_t first, uint32_t k) { return *(const __attribute__((address_space(3))) F*)(from + (first + i) * line + k * 2u + g * 16u); };
  auto across = [&](const lds_char* from, uint32_t line, uint32_t first, uint32_t k) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    s16x4 h[2];
#pragma unroll
    for (uint32_t q = 0; q < 2u; ++q)
      h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(from + (k + 8u * g + 4u * q + i / 4u) * line + first * 2u + (i % 4u) * 8u));
    return __builtin_bit_cast(F, (s16x8)__builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  f32x4 sum[kBlocks][2][2];
  // where this wavefront's blocks begin in a product of `rows` x `rows`, and of `rows` x `columns`; none: beyond the rows
  uint32_t block_r[2][kBlocks], block_c[2][kBlocks];
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      const uint32_t over = (w ? columns : rows) / 32u, block = wave + n * (kSmallLanes / 64u);
      block_r[w][n] = same(block / over * 32u);
      block_c[w][n] = same(block % over * 32u);
    }
  // Places are worked out anew for every product and every store: kept from step to step they would not all fit the registers.
  auto anew = [&] { asm volatile("" : "+v"(i), "+v"(g)); };
  // This wavefront's blocks of a product: rows of `left` over `depth`, by rows of `right` (or across them).
  auto multiply = [&](const lds_char* left, uint32_t line_l, uint32_t part_l, const lds_char* right, uint32_t line_r, uint32_t part_r, uint32_t depth, auto is_across) __attribute__((always_inline)) {
    constexpr int w = decltype(is_across)::value;
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      anew();
      const uint32_t r0 = block_r[w][n], c0 = block_c[w][n];
      if (r0 >= rows) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[n][e / 2][e % 2] = f32x4{0.f, 0.f, 0.f, 0.f};
      for (uint32_t k = 0; k < depth; k += 32u) {
        F l[2][2], r[2][2];   // of 16 rows each, first and second parts
#pragma unroll
        for (uint32_t h = 0; h < 2u; ++h)
#pragma unroll
          for (uint32_t q = 0; q < 2u; ++q) {
            l[h][q] = along(left + q * part_l, line_l, r0 + 16u * h, k);
            if constexpr (decltype(is_across)::value) r[h][q] = across(right + q * part_r, line_r, c0 + 16u * h, k);
            else r[h][q] = along(right + q * part_r, line_r, c0 + 16u * h, k);
          }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int pair = 3; pair >= 0; --pair)   // (the smallest first)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j) sum[n][h][j] = mma(r[j][pair & 1], l[h][pair >> 1], sum[n][h][j]);
      }
    }
  };
  // f(row, first of four columns, sums) of every place that this wavefront has worked out.
  auto every = [&](auto which, auto f) __attribute__((always_inline)) {
    constexpr int w = decltype(which)::value;
#pragma unroll
    for (int n = 0; n < kBlocks; ++n) {
      anew();
      if (block_r[w][n] >= rows) continue;
#pragma unroll
      for (uint32_t h = 0; h < 2u; ++h)
#pragma unroll
        for (uint32_t j = 0; j < 2u; ++j) f(block_r[w][n] + 16u * h + i, block_c[w][n] + 16u * j + 4u * g, sum[n][h][j]);
    }
  };
  typedef __attribute__((address_space(3))) f16x4 Four;
  auto put = [&](lds_char* to, uint32_t part, f32x4 v) {
    const Halves w(v, 1.f);
    *(Four*)to = w.high;
    *(Four*)(to + part) = w.low;
  };
  for (uint32_t s = 0; s < p.steps; ++s) {
    const StepNumbers by = p.of[s];
    const float first = s ? 1.f : f;
    multiply(x, line_x, part_x, x, line_x, part_x, columns, Kind<0>());
    every(Kind<0>(), [&](uint32_t r, uint32_t c, f32x4& v) { put(a + r * line_a + c * 2u, part_a, v * (by.gram * first * first)); });
    __syncthreads();
    multiply(a, line_a, part_a, a, line_a, part_a, rows, Kind<0>());
    every(Kind<0>(), [&](uint32_t r, uint32_t c, f32x4& v) {
      const lds_char* at = a + r * line_a + c * 2u;
      const f16x4 high = *(const Four*)at, low = *(const Four*)(at + part_a);
#pragma unroll
      for (uint32_t e = 0; e < 4u; ++e) v[e] = v[e] * by.square + ((float)high[e] + (float)low[e]) * by.keep + (r == c + e && r < m_side ? by.diagonal : 0.f);
    });
    __syncthreads();
    every(Kind<0>(), [&](uint32_t r, uint32_t c, f32x4& v) { put(a + r * line_a + c * 2u, part_a, v); });
    __syncthreads();
    multiply(a, line_a, part_a, x, line_x, part_x, rows, Kind<1>());
    if (s + 1u == p.steps) break;
    __syncthreads();
    every(Kind<1>(), [&](uint32_t r, uint32_t c, f32x4& v) { put(x + r * line_x + c * 2u, part_x, v * (by.next * first)); });
    __syncthreads();
  }
  const float scale = p.of[p.steps - 1u].next * (p.steps == 1u ? f : 1.f);
  every(Kind<1>(), [&](uint32_t r, uint32_t c, f32x4& v) {
    const f32x4 one[1] = {v * scale};
    if (p.last.out == FBX_F32) leave<float, 1>(p.last, t, r, c, one);
    else if (p.last.out == FBX_F16) leave<f16, 1>(p.last, t, r, c, one);
    else leave<__bf16, 1>(p.last, t, r, c, one);
  });
#endif
}
bool is_small(uint32_t rows, uint32_t columns) {
  const uint32_t m = small_side(rows < columns ? rows : columns);
  const uint64_t n = small_side(rows < columns ? columns : rows), blocks = m / 32u * (n / 32u);
  return blocks <= (uint64_t)kBlocks * (kSmallLanes / 64) && m / 32u * (m / 32u) <= (uint64_t)kBlocks * (kSmallLanes / 64) &&
         2ull * m * (small_line((uint32_t)n) + small_line(m)) <= kRoom;
}

// The steps' scales: A is held times 2^a, B times 2^b, so that no first part reaches f16's end (65,504).
struct Step {
  double a, b, c;
  int at_a, at_b;
};
constexpr double kFull = 57344;   // (with an eighth to spare for what rounding adds)
// Bounds of the singular values before each step, from 1 on; how far they can go follows from the coefficients.
const char* plan(const fbx_ortho* h, std::vector<Step>* steps) {
  double most = 1;
  for (uint32_t i = 0; i < h->steps; ++i) {
    Step s{};
    s.a = h->coefficients[3 * i];
    s.b = h->coefficients[3 * i + 1];
    s.c = h->coefficients[3 * i + 2];
    if (!isfinite(s.a) || !isfinite(s.b) || !isfinite(s.c)) return "coefficients must be finite";
    double next = 0, polynom = 0;
    constexpr int kPlaces = 2048;
    for (int k = 0; k <= kPlaces; ++k) {
      const double v = most * k / kPlaces, q = s.a + v * v * (s.b + s.c * v * v);
      next = fmax(next, fabs(v * q));
      polynom = fmax(polynom, fabs(q));
    }
    // (between two places a polynomial of the fifth degree moves by less than this)
    const double slack = (fabs(s.a) + 3 * fabs(s.b) * most * most + 5 * fabs(s.c) * most * most * most * most) * most / kPlaces;
    next += slack;
    polynom += 2 * slack;
    auto scale = [](double top) {
      int e = kX;
      while (e > -kX && ldexp(top, e) > kFull) --e;
      return e;
    };
    s.at_a = scale(most * most);
    s.at_b = scale(fmax(polynom, 1e-3));
    if (polynom > 256 || (i + 1 < h->steps && next > 3)) return "coefficients: a step takes singular values beyond 3, or its polynomial beyond 256";
    most = fmax(next * 1.01, 0.25);
    steps->push_back(s);
  }
  return nullptr;
}

// A list of matrices as both calls see it.
struct Whole {
  const fbx_ortho* h;
  fbx_dtype in, out, copy;
  bool weights, nesterov;
  float momentum, grad_scale, decay;
  std::vector<Matrix> all;
};

// Tiles of 256 x 256 read least from LDS, smaller ones begin sooner, end sooner and leave fewer compute units idle.  What they were
// measured to take (2,624 x 4,096, 384 x 1,024; microseconds): `begin` before the first step and behind the last, a step alone on a compute unit,
// and among as many as fit one; kNext's results are twice what the others store.
// Where both parts are multiplied small tiles bring them into LDS together, once for three products (18 of 384 x 1,024: A 26 -> 18.6 us, B 15.7 -> 13.1); for tiles of 128 two workgroups would not fit a compute unit.
struct Size { uint32_t side, at_once; double begin[2], lone, full; };
constexpr Size kSizes[4] = {{256, 1, {14, 24}, 1.45, 1.8}, {128, 2, {9, 10.5}, 0.78, 0.9}, {64, 2, {7, 7}, 0.35, 0.43}, {64, 2, {6.5, 6.5}, 0.17, 0.25}};
uint64_t tiles_of(const Matrix& t, Form form, uint32_t side) {
  const uint64_t rows = ceil_div(t.m_side, side);
  return form == kGram || form == kPolynom ? rows * (rows + 1) / 2 : rows * ceil_div(t.n_side, side);
}
uint32_t choose(const Matrix* t, uint32_t n, Form form) {
  uint32_t best = 2;
  double least = 0;
  for (uint32_t i = 0; i < 3; ++i) {
    const Size& s = kSizes[i == 2 && t[0].exact ? 3 : i];   // (a launch's matrices are of one kind)
    const double begin = s.begin[form == kNext || form == kLast], slots = 256.0 * s.at_once;
    double tiles = 0, steps = 0, longest = 0;
    for (uint32_t k = 0; k < n; ++k) {
      const double count = (double)tiles_of(t[k], form, s.side), depth = (double)(form == kGram ? t[k].wide_n : t[k].wide_m) / kDepth * (t[k].exact ? 3 : 1);
      tiles += count;
      steps += count * depth;
      longest = fmax(longest, depth);
    }
    if (tiles >= most_blocks(512)) continue;
    const double rounds = floor(tiles / slots), rest = tiles - rounds * slots, mean = steps / tiles;
    const double takes = rounds * (begin + mean * s.full) + (rest > 0 ? begin + (rounds > 0 ? mean : longest) * (rest > 256.0 ? s.full : s.lone) : 0);
    if (!least || takes < least) {
      least = takes;
      best = i;
    }
  }
  return best;
}

template <Form kForm>
void multiply(ProductArgs& p, hipStream_t stream) {
  const uint32_t size = choose(p.list.of, p.list.n, kForm), side = kSizes[size].side;
  for (uint32_t i = 0; i < p.list.n; ++i) p.list.first[i + 1] = p.list.first[i] + (uint32_t)tiles_of(p.list.of[i], kForm, side);
  const dim3 grid(p.list.first[p.list.n]);
  auto launch = [&](auto exact) {
    constexpr bool e = decltype(exact)::value;
    if (size == 0) launch_on(stream, k_product<kForm, 256, 256, 2, 4, 2, e>, grid, dim3(512), 0, p);
    else if (size == 1) launch_on(stream, k_product<kForm, 128, 128, 2, 2, 2, e>, grid, dim3(256), 0, p);
    else launch_on(stream, k_product<kForm, 64, 64, 2, 2, e ? 2 : 4, e>, grid, dim3(256), 0, p);
  };
  if (p.list.of[0].exact) launch(std::true_type());
  else launch(std::false_type());
}

// Left to this (for weights; a result that is handed out is of both parts unless the caller says otherwise), products are of both parts where
// weights keep more than bf16 does, and for small matrices: their products take little beside their launches.  Weights in bf16 end up
// as near 64 bits either way (2,624 x 4,096: 1.66e-3, their own rounding), in 2.05 and 5.25 ms for three.  A result in bf16 would not: products of first
// parts leave it off by 1.76e-3 in place of 1.66e-3 (a decaying spectrum, 2,624 x 4,096), 2.27e-3 (normally distributed, 300 x 400), 9e-3 (a unit matrix of 319).
constexpr uint32_t kSmall = 256;
uint32_t is_exact(const Matrix& t, uint32_t asked, fbx_dtype out) {
  return asked != FBX_EXACT_BY_SIZE ? asked : out != FBX_BF16 || (t.rows < t.columns ? t.rows : t.columns) <= kSmall;
}

// Where a matrix's parts lie in its scratch; its size.
uint64_t lay_out(Matrix& t, uint32_t rows, uint32_t columns) {
  t.rows = rows;
  t.columns = columns;
  t.tall = rows > columns;
  t.m_side = t.tall ? columns : rows;
  t.n_side = t.tall ? rows : columns;
  t.wide_m = (uint32_t)round_up(t.m_side, kDepth);
  t.wide_n = (uint32_t)round_up(t.n_side, kDepth);
  const uint64_t all = (uint64_t)rows * columns;
  t.chunk = (uint32_t)round_up(ceil_div(all, kMostPartials), 2048);
  t.partials = (uint32_t)ceil_div(all, t.chunk);
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t was = at;
    at = round_up(at + bytes, 256);
    return (uint32_t)(was / 256);
  };
  t.at_norm = take(kMostPartials * 8 + 8);
  t.at_x = take(4ull * t.m_side * t.wide_n * sizeof(f16));
  t.at_a = take(4ull * t.m_side * t.wide_m * sizeof(f16));
  return at;
}

// The numbers of a step, for a first X held as k_split leaves it and others held times 2^14.
StepNumbers numbers_of(const std::vector<Step>& steps, size_t i) {
  const Step& s = steps[i];
  const double x = i ? ldexp(1, kX) : 1, a = ldexp(1, s.at_a), b = ldexp(1, s.at_b), next = i + 1 < steps.size() ? ldexp(1, kX) : 1;
  return StepNumbers{(float)(a / (x * x)), (float)(s.b * b / a), (float)(s.c * b / (a * a)), (float)(s.a * b), (float)(next / (b * x))};
}

// Matrices of a kind go together until there are kMatrices of them or their scratch is more than this: by then they fill the card.
constexpr uint64_t kTogether = 1ull << 30;
struct Batch {
  std::vector<uint32_t> of;
  uint64_t bytes;
  bool small;
};
std::vector<Batch> batches(std::vector<Matrix>& all) {
  std::vector<Batch> b;
  int open[3] = {-1, -1, -1};   // the last batch of matrices of each kind: small, of both parts, of first parts
  for (uint32_t i = 0; i < all.size(); ++i) {
    const bool small = is_small(all[i].rows, all[i].columns);
    const uint64_t bytes = lay_out(all[i], all[i].rows, all[i].columns) * !small;
    int& at = open[small ? 0 : all[i].exact ? 1 : 2];
    if (at < 0 || b[at].of.size() == kMatrices || b[at].bytes + bytes > kTogether) {
      at = (int)b.size();
      b.push_back(Batch{{}, 0, small});
    }
    b[at].of.push_back(i);
    b[at].bytes += bytes;
  }
  return b;
}
uint64_t scratch_of(std::vector<Matrix>& all) {
  uint64_t most = 0;
  for (const Batch& b : batches(all)) most = b.bytes > most ? b.bytes : most;
  return most;
}

template <class G, bool kGiven>
void prepare_as(const PrepareArgs& q, bool measure, hipStream_t stream) {
  launch_on(stream, measure ? k_measure<G, kGiven> : k_split<G, kGiven>, dim3(q.list.first[q.list.n]), dim3(256), 0, q);
}
void prepare(const PrepareArgs& q, bool measure, const Whole& w, hipStream_t stream) {
  const bool given = q.list.of[0].m != nullptr;
  if (w.in == FBX_F32) given ? prepare_as<float, true>(q, measure, stream) : prepare_as<float, false>(q, measure, stream);
  else if (w.in == FBX_F16) given ? prepare_as<f16, true>(q, measure, stream) : prepare_as<f16, false>(q, measure, stream);
  else given ? prepare_as<__bf16, true>(q, measure, stream) : prepare_as<__bf16, false>(q, measure, stream);
}

void run(Whole& w, const std::vector<Step>& steps, char* scratch, hipStream_t stream) {
  const Given given{w.nesterov, w.momentum, w.grad_scale, w.h->eps};
  const Leaving last{(uint32_t)w.out, (uint32_t)w.copy, w.weights, w.decay};
  for (const Batch& b : batches(w.all)) {
    const uint32_t n = (uint32_t)b.of.size();
    if (b.small) {
      SmallArgs p{};
      p.list.n = n;
      for (uint32_t i = 0; i < n; ++i) p.list.of[i] = w.all[b.of[i]];
      p.given = given;
      p.last = last;
      p.steps = (uint32_t)steps.size();
      for (size_t i = 0; i < steps.size(); ++i) p.of[i] = numbers_of(steps, i);
      if (w.in == FBX_F32) launch_on(stream, k_small<float>, dim3(n), dim3(kSmallLanes), 0, p);
      else if (w.in == FBX_F16) launch_on(stream, k_small<f16>, dim3(n), dim3(kSmallLanes), 0, p);
      else launch_on(stream, k_small<__bf16>, dim3(n), dim3(kSmallLanes), 0, p);
      continue;
    }
    PrepareArgs q{};
    ProductArgs p{};
    q.given = given;
    p.last = last;
    q.list.n = p.list.n = n;
    char* at = scratch;
    for (uint32_t i = 0; i < n; ++i) {
      Matrix& t = q.list.of[i] = w.all[b.of[i]];
      t.scratch = at;
      at += lay_out(t, t.rows, t.columns);
      p.list.of[i] = t;
    }
    for (uint32_t i = 0; i < n; ++i) q.list.first[i + 1] = q.list.first[i] + q.list.of[i].partials;
    prepare(q, true, w, stream);
    for (uint32_t i = 0; i < n; ++i) q.list.first[i + 1] = q.list.first[i] + (uint32_t)(ceil_div(q.list.of[i].m_side, kSquare) * (q.list.of[i].wide_n / kSquare));
    prepare(q, false, w, stream);
    for (size_t i = 0; i < steps.size(); ++i) {
      const StepNumbers s = numbers_of(steps, i);
      p.turn = i & 1u;
      p.begins = i == 0;
      p.keep = 0;
      p.sum = s.gram;
      multiply<kGram>(p, stream);
      p.keep = s.keep;
      p.sum = s.square;
      p.diagonal = s.diagonal;
      multiply<kPolynom>(p, stream);
      p.keep = (float)(steps[i].a * (i + 1 < steps.size() ? ldexp(1, kX) : 1) / (i ? ldexp(1, kX) : 1)) / kSecond;   // (of second parts)
      p.sum = s.next;
      if (i + 1 < steps.size()) multiply<kNext>(p, stream);
      else multiply<kLast>(p, stream);
    }
  }
}

fbx_status check(const fbx_ortho* h, std::vector<Step>* steps) {
  if (!h->steps || h->steps > 64) return refuse(FBX_E_ARG, "steps must be 1 .. 64");
  if (h->exact > FBX_EXACT_BY_SIZE) return refuse(FBX_E_ARG, "exact must be 0, 1 or FBX_EXACT_BY_SIZE");
  if (!h->coefficients) return refuse(FBX_E_ARG, "coefficients is NULL");
  if (!(h->eps >= 1e-30 && h->eps <= 1e30)) return refuse(FBX_E_ARG, "eps must be 1e-30 .. 1e30");
  const char* why = plan(h, steps);
  return why ? refuse(FBX_E_ARG, why) : FBX_OK;
}
fbx_status check_sides(uint32_t rows, uint32_t columns) {
  return !rows || !columns || rows > FBX_ORTHO_MOST || columns > FBX_ORTHO_MOST ? refuse(FBX_E_ARG, "rows and columns must be 1 .. FBX_ORTHO_MOST") : FBX_OK;
}
fbx_status check_scratch(const void* d_scratch, uint64_t bytes, uint64_t need) {
  if (need && (!d_scratch || (uintptr_t)d_scratch % 256u)) return refuse(FBX_E_ARG, "d_scratch is NULL or not 256-byte aligned");
  return bytes < need ? refuse(FBX_E_NOMEM, "scratch too small: the scratch function gives its size") : FBX_OK;
}
// What batches go by, for a call and for the size of its scratch alike: the matrices' sides, and the kind of their products.
template <class M>
fbx_status sides(const M* matrices, uint32_t n, uint32_t exact, fbx_dtype out, std::vector<Matrix>* all) {
  if (!matrices && n) return refuse(FBX_E_ARG, "matrices is NULL");
  for (uint32_t i = 0; i < n; ++i) {
    const fbx_status st = check_sides(matrices[i].rows, matrices[i].columns);
    if (st != FBX_OK) return st;
    Matrix t{};
    t.rows = matrices[i].rows;
    t.columns = matrices[i].columns;
    t.exact = is_exact(t, exact, out);
    all->push_back(t);
  }
  return FBX_OK;
}
// All that a step refuses but for its scratch, and what it is made of.
fbx_status check(const fbx_muon* h, const fbx_muon_matrix* matrices, uint32_t n, Whole* w, std::vector<Step>* steps) {
  if (!h) return refuse(FBX_E_ARG, "h is NULL");
  if (!known(h->param_dtype) || !known(h->grad_dtype)) return refuse(FBX_E_ARG, "unknown dtype");
  if (!(h->momentum >= 0 && h->momentum < 1)) return refuse(FBX_E_ARG, "momentum must be in [0, 1)");
  if (!isfinite((float)h->lr) || !isfinite((float)h->weight_decay) || !isfinite((float)h->grad_scale)) return refuse(FBX_E_ARG, "lr, weight_decay and grad_scale must be finite");
  fbx_status st = check(&h->ortho, steps);
  if (st == FBX_OK) st = sides(matrices, n, h->ortho.exact, h->param_dtype, &w->all);
  if (st != FBX_OK) return st;
  bool copy = false;
  for (uint32_t i = 0; i < n; ++i) copy |= matrices[i].d_copy != nullptr;
  for (uint32_t i = 0; i < n; ++i) {
    const fbx_muon_matrix& m = matrices[i];
    Matrix& t = w->all[i];
    if (!m.d_param || !m.d_grad || !m.d_m) return refuse(FBX_E_ARG, "a matrix lacks its weights, gradient or momentum");
    if ((uintptr_t)m.d_param % size_of(h->param_dtype) || (uintptr_t)m.d_grad % size_of(h->grad_dtype) || (uintptr_t)m.d_m % 4u) return refuse(FBX_E_ARG, "a matrix is not aligned to its elements");
    if (m.d_copy && (h->copy_dtype == FBX_F32 || !known(h->copy_dtype) || h->param_dtype != FBX_F32 || (uintptr_t)m.d_copy % 2u))
      return refuse(FBX_E_ARG, "a copy is in f16 or bf16, of weights in f32");
    if (copy && !m.d_copy) return refuse(FBX_E_ARG, "either all matrices have a copy or none");
    if (!isfinite((float)(h->lr * m.factor))) return refuse(FBX_E_ARG, "factor must be finite");
    t.u = m.d_grad;
    t.m = (float*)m.d_m;
    t.out = m.d_param;
    t.copy = m.d_copy;
    t.ld_u = t.ld_out = m.columns;
    t.step = (float)(h->lr * m.factor);
  }
  w->h = &h->ortho;
  w->in = h->grad_dtype;
  w->out = h->param_dtype;
  w->copy = h->copy_dtype;
  w->weights = true;
  w->nesterov = h->nesterov != 0;
  w->momentum = (float)h->momentum;
  w->grad_scale = (float)h->grad_scale;
  w->decay = (float)(1.0 - h->lr * h->weight_decay);
  return FBX_OK;
}
// (no exception may leave a call)
template <class F>
fbx_status guarded(F f) {
  try {
    return f();
  } catch (...) {
    return refuse(FBX_E_NOMEM, "out of host memory");
  }
}

}  // namespace
}  // namespace train
}  // namespace fbx

using namespace fbx::train;

extern "C" fbx_status fbx_ortho_scratch(const fbx_ortho* h, const fbx_ortho_matrix* matrices, uint32_t n, uint64_t* bytes) {
  return guarded([&] {
    if (!h || !bytes) return refuse(FBX_E_ARG, "h or bytes is NULL");
    std::vector<Matrix> all;
    const fbx_status st = sides(matrices, n, h->exact, h->out, &all);
    if (st == FBX_OK) *bytes = scratch_of(all);
    return st;
  });
}

extern "C" fbx_status fbx_orthogonalise(const fbx_ortho* h, const fbx_ortho_matrix* matrices, uint32_t n, void* d_scratch, uint64_t scratch_bytes, void* hip_stream) {
  return guarded([&] {
    if (!h) return refuse(FBX_E_ARG, "h is NULL");
    Whole w{};
    std::vector<Step> steps;
    if (!known(h->in) || !known(h->out)) return refuse(FBX_E_ARG, "unknown dtype");
    fbx_status st = check(h, &steps);
    if (st == FBX_OK) st = sides(matrices, n, h->exact, h->out, &w.all);
    if (st != FBX_OK) return st;
    for (uint32_t i = 0; i < n; ++i) {
      const fbx_ortho_matrix& m = matrices[i];
      Matrix& t = w.all[i];
      if (!m.d_u || !m.d_out) return refuse(FBX_E_ARG, "a matrix or its result is NULL");
      if ((uintptr_t)m.d_u % size_of(h->in) || (uintptr_t)m.d_out % size_of(h->out)) return refuse(FBX_E_ARG, "a matrix is not aligned to its elements");
      if (m.ld_u < m.columns || m.ld_out < m.columns || (m.ld_u | m.ld_out) >> 40) return refuse(FBX_E_ARG, "a stride is smaller than columns, or 2^40 or more");
      t.u = m.d_u;
      t.ld_u = m.ld_u;
      t.out = m.d_out;
      t.ld_out = m.ld_out;
      t.step = 1.f;
    }
    st = check_scratch(d_scratch, scratch_bytes, scratch_of(w.all));
    if (st != FBX_OK || !n) return st;
    w.h = h;
    w.in = h->in;
    w.out = h->out;
    run(w, steps, (char*)d_scratch, (hipStream_t)hip_stream);
    return launched();
  });
}

extern "C" fbx_status fbx_muon_scratch(const fbx_muon* h, const fbx_muon_matrix* matrices, uint32_t n, uint64_t* bytes) {
  return guarded([&] {
    if (!h || !bytes) return refuse(FBX_E_ARG, "h or bytes is NULL");
    std::vector<Matrix> all;
    const fbx_status st = sides(matrices, n, h->ortho.exact, h->param_dtype, &all);
    if (st == FBX_OK) *bytes = scratch_of(all);
    return st;
  });
}

extern "C" fbx_status fbx_muon_check(const fbx_muon* h, const fbx_muon_matrix* matrices, uint32_t n) {
  return guarded([&] {
    Whole w{};
    std::vector<Step> steps;
    return check(h, matrices, n, &w, &steps);
  });
}

extern "C" fbx_status fbx_muon_step(const fbx_muon* h, const fbx_muon_matrix* matrices, uint32_t n, void* d_scratch, uint64_t scratch_bytes, void* hip_stream) {
  return guarded([&] {
    Whole w{};
    std::vector<Step> steps;
    fbx_status st = check(h, matrices, n, &w, &steps);
    if (st == FBX_OK) st = check_scratch(d_scratch, scratch_bytes, scratch_of(w.all));
    if (st != FBX_OK || !n) return st;
    run(w, steps, (char*)d_scratch, (hipStream_t)hip_stream);
    return launched();
  });
}

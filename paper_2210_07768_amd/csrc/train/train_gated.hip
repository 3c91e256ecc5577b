// The gated feed-forward block h = act(x Wg^T) * (x Wu^T) and its gradient.
#include "train_common.h"

#include <math.h>

namespace fbx {
namespace train {
namespace {

// e^a and 1 / a by the hardware's approximations (one unit in the last place each, and |a| units for what a log2 e is rounded
// by): the exact division and exponential of 64 elements a lane were an eighth of a large product's time.
__device__ __forceinline__ float exponential(float a) { return __builtin_amdgcn_exp2f(a * 1.4426950408889634f); }
__device__ __forceinline__ float logistic(float a) { return __builtin_amdgcn_rcpf(1.f + exponential(-a)); }
__device__ __forceinline__ float bell_below(float a) { return 0.5f * (1.f + erff(a * 0.70710678118654752f)); }

template <int kAct>
__device__ __forceinline__ float act(float a) {
  if (kAct == FBX_ACT_SILU) return a * logistic(a);
  if (kAct == FBX_ACT_GELU) return a * bell_below(a);
  if (kAct == FBX_ACT_RELU) return a > 0.f || a != a ? a : 0.f;
  return logistic(a);
}
template <int kAct>
__device__ __forceinline__ float slope(float a) {
  if (kAct == FBX_ACT_SILU) {
    const float s = logistic(a);
    return s * (1.f + a * (1.f - s));
  }
  if (kAct == FBX_ACT_GELU) return bell_below(a) + a * exponential(-0.5f * a * a) * 0.39894228040143268f;
  if (kAct == FBX_ACT_RELU) return a > 0.f ? 1.f : 0.f;
  const float s = logistic(a);
  return s * (1.f - s);
}

typedef float f32x4 __attribute__((ext_vector_type(4)));

// One launch's product: C (rows x columns) = A B^T over depth, A and B in one of two orders.
//   kForward  A = x, B = the two weights side by side;  c: h
//   kSlopes   the same product;  c: a row of da, then of du, each `half` elements wide (zeros beyond columns)
//   kInputs   A = the rows kSlopes wrote, B = the weights, read along their rows;  c: dx
//   kWeights  A = those rows and B = x, both read along their rows (depth: the records);  c, c2: dWg, dWu
// da and du are rounded to the block's type on their way: they are operands of the next two products, and matrix instructions of
// 32-bit operands have a ninth of the rate of those of 16 (154 of 1,370 TFLOP/s).  The gradients' relative error against 64 bits is 1.4 times that of
// one rounding at the end: 2.9e-4 to 2.1e-4 in f16 (1,000 x 411 by 2 x 773), 2.3e-3 to 1.7e-3 in bf16 (16,384 x 2,624 by 2 x 4,096).
enum Form { kForward, kSlopes, kInputs, kWeights };

struct MmArgs {
  const void *a, *b, *b2;
  uint64_t ld_a, ld_b, ld_b2;  // in bytes
  const void* dh;
  void *c, *c2;
  uint64_t ld_dh, ld_c, ld_c2;  // in elements
  uint32_t rows, columns;      // of c (kForward, kSlopes: columns of each half; kWeights: rows of both weights, `half` apart)
  uint32_t depth, half;        // half: width of a half of what kSlopes writes, whole steps of depth
  uint32_t b_columns;          // kInputs, kWeights: elements in a row of B (a multiple of a load's)
  uint32_t act, wide;          // wide: c (and dh) can be moved four elements at a time
  uint32_t row_tiles, column_tiles, steps;  // steps: of depth, of a tile
  uint32_t whole, shares;      // tiles that are one workgroup's; workgroups that share the steps of each further tile
  f32x4* parts;                // of those: a share's sums, a tile's registers
};

constexpr uint32_t kOutside = 0xfffffff0u;  // an offset beyond every buffer
constexpr int kStepBytes = 128;  // of depth that are staged at a time: 64 elements of 16 bits, 32 of 32

template <class T>
struct Frag {
  typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
};
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) char lds_char;

// 16 x 16 of C += 16 of one side's rows x 16 of the other's over a load's depth (16 bytes a lane): lane l holds row l % 16
// of either side and the depth's (l / 16)-th part; of C, column l % 16 and rows 4 (l / 16) .. + 3.
__device__ __forceinline__ f32x4 mma(Frag<__bf16>::type a, Frag<__bf16>::type b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(Frag<_Float16>::type a, Frag<_Float16>::type b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(Frag<float>::type a, Frag<float>::type b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ uint32_t same(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }  // (in all lanes)

// A tile of one operand in LDS: kStepBytes of depth for R rows, R * 128 bytes, filled by loads that go past the
// registers: lane l's 16 bytes land at 16 l behind the wavefront's place, so the layout is made by which 16 bytes a lane asks for.
//   along depth (kAcross = false): a row's 128 bytes are eight chunks, chunk c of row r at place c ^ (r % 8), so that the 16
//     rows a read takes the same chunk of lie in different banks;
//   across (kAcross = true): for every element of depth a line of R elements, sixteen to a unit, unit u of line k at
//     place u ^ turn(k), so that the lines a transposing read takes the same unit of lie in different banks.
// What lies outside the operand is asked for beyond the buffer's end, which gives zeros.
template <class T, int R, int kWaves, bool kAcross>
struct Tile {
  static constexpr int kSize = sizeof(T), kDepth = kStepBytes / kSize, kLoads = R * kStepBytes / 1024 / kWaves, kUnits = R / 16;
  static_assert(kLoads >= 1, "");

  __device__ static uint32_t turn(uint32_t k) {
    if (kSize == 4) return (k >> 2) & 3u;
    if (R == 64) return ((k >> 1) & 1u) | ((k >> 3) & 1u) << 1;
    return (k & 3u) | ((k >> 3) & 1u) << 2;
  }

  uint32_t offset[kLoads];  // bytes from the tile's first element
  uint32_t deep;            // along depth: the first element of depth that this lane's loads take

  // wave: of kWaves; columns_left (across): elements from the tile's first to the operand's last
  __device__ void begin(uint32_t wave, uint32_t lane, uint64_t ld, uint32_t columns_left) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const uint32_t piece = wave * kLoads + j;  // 1024 bytes of the tile
      if (!kAcross) {
        const uint32_t chunk = (lane % 8u) ^ (lane / 8u);
        deep = chunk * (16 / kSize);
        offset[j] = (piece * 8u + lane / 8u) * (uint32_t)ld + chunk * 16u;
      } else {
        constexpr uint32_t chunks = R * kSize / 16;  // of a line
        const uint32_t at = piece * 64u + lane, k = at / chunks, c = at % chunks;
        const uint32_t column = (((c / kSize) ^ turn(k)) * kSize + c % kSize) * (16 / kSize);
        offset[j] = column < columns_left ? k * (uint32_t)ld + column * kSize : kOutside;
      }
    }
  }
  // from: the tile's first element at this step; lines: rows (along) or elements of depth (across) there are from it on;
  // depth_left (along): elements of depth from this step on
  __device__ void load(lds_char* to, const char* from, uint64_t ld, uint32_t lines, uint32_t depth_left, uint32_t line_bytes, uint32_t wave) const {
    const uint32_t most = kAcross ? (uint32_t)kDepth : (uint32_t)R, n = lines < most ? lines : most;
    // The buffer's descriptor (address, bytes, raw data): one for the wavefront, and said so, lest the compiler loop over
    // its lanes.  The load is written out because the compiler, where it knows of loads into LDS, waits for all of them
    // before a transposing read, whichever array that reads.  It has no result register; `arrived` waits for it.
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 r = {same((uint32_t)(uintptr_t)from), same((uint32_t)((uintptr_t)from >> 32) & 0xffffu), same(n ? (n - 1u) * (uint32_t)ld + line_bytes : 0u), 0x00020000u};
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const uint32_t at = same((uint32_t)(uintptr_t)to + (wave * kLoads + j) * 1024u);
      const uint32_t o = kAcross || deep < depth_left ? offset[j] : kOutside;
      // (five wait states between a vector instruction's write of a scalar register, the descriptor's, and its use here)
      if (j == 0) asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(o), "s"(r) : "memory", "m0");
      else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(o), "s"(r) : "memory", "m0");
    }
  }

  // Rows first .. first + 15 of the operand, part `part` (0, 1) of the step's depth.
  __device__ static typename Frag<T>::type read(const lds_char* tile, uint32_t first, int part, uint32_t lane) {
    typedef typename Frag<T>::type F;
    const uint32_t i = lane % 16u, g = lane / 16u;
    if constexpr (!kAcross) {
      return *(const __attribute__((address_space(3))) F*)(tile + (first + i) * kStepBytes + (((4u * part + g) ^ (i & 7u)) * 16u));
    } else if constexpr (kSize == 4) {
      F f;
#pragma unroll
      for (uint32_t j = 0; j < 4u; ++j)
        f[j] = *(const __attribute__((address_space(3))) float*)(tile + (part * 16u + 4u * g + j) * (R * 4u) + ((first / 16u) ^ g) * 64u + i * 4u);
      return f;
    } else {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      s16x4 h[2];
#pragma unroll
      for (uint32_t q = 0; q < 2u; ++q) {
        const uint32_t k = part * 32u + 8u * g + 4u * q + i / 4u;
        h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tile + k * (R * 2u) + ((first / 16u) ^ turn(k)) * 32u + (i % 4u) * 8u));
      }
      return __builtin_bit_cast(F, (s16x8)__builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

template <int kValue>
struct Kind {
  static constexpr int value = kValue;
};

// Four adjacent elements, of which the first n exist.
template <class T>
__device__ __forceinline__ void put(T* to, f32x4 v, uint32_t n, bool wide) {
  if (wide && n >= 4u) {
    *(Pack<T, 4>*)to = Pack<T, 4>{{(T)v[0], (T)v[1], (T)v[2], (T)v[3]}};
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 4u; ++j)
      if (j < n) to[j] = (T)v[j];
  }
}

// Eight row tiles wide, down the columns: tiles that are worked on at one time share rows of both sides in a die's cache.
template <int BM, int BN>
__device__ __forceinline__ void place(const MmArgs& p, uint32_t t, uint32_t& row0, uint32_t& col0) {
  const uint32_t band = t / (8u * p.column_tiles), in_band = t - band * 8u * p.column_tiles;
  const uint32_t high = p.row_tiles - band * 8u < 8u ? p.row_tiles - band * 8u : 8u;
  row0 = (band * 8u + in_band % high) * BM;
  col0 = in_band / high * BN;
}

// kSlopes: dh at four columns from c on, and from every 16th further on, of row r; zeros beyond it.
template <class T, int kN>
__device__ __forceinline__ void fetch_dh(const MmArgs& p, uint32_t r, uint32_t c0, Pack<T, 4> (&dh)[kN]) {
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    const uint32_t c = c0 + j * 16;
    const T* from = (const T*)p.dh + (uint64_t)r * p.ld_dh + c;
    dh[j] = Pack<T, 4>{};
    if (r >= p.rows) continue;
    if (p.wide && c + 4u <= p.columns) {
      dh[j] = *(const Pack<T, 4>*)from;
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 4u; ++e)
        if (c + e < p.columns) dh[j].v[e] = from[e];
    }
  }
}

// What becomes of 16 rows of a wavefront's sums (r: this lane's row; c0: its first column): they are rounded and stored.
// dh: kSlopes, of the same places.
template <class T, Form kForm, int kNF, int kAct>
__device__ __forceinline__ void finish_rows(const MmArgs& p, uint32_t r, uint32_t c0, const f32x4 (&sum)[kNF], const Pack<T, 4> (&dh)[kNF / 2]) {
  if constexpr (kForm == kForward || kForm == kSlopes) {
    if (r >= p.rows) return;
#pragma unroll
    for (int j = 0; j < kNF / 2; ++j) {
      const uint32_t c = c0 + j * 16;
      const f32x4 g = sum[j], u = sum[j + kNF / 2];
      if (kForm == kForward) {
        f32x4 h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = act<kAct>(g[e]) * u[e];
        put((T*)p.c + (uint64_t)r * p.ld_c + c, h, c < p.columns ? p.columns - c : 0u, p.wide);
      } else if (c < p.half) {
        f32x4 da, du;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          da[e] = (float)dh[j].v[e] * u[e] * slope<kAct>(g[e]);
          du[e] = (float)dh[j].v[e] * act<kAct>(g[e]);
        }
        put((T*)p.c + (uint64_t)r * p.ld_c + c, da, 4u, true);
        put((T*)p.c + (uint64_t)r * p.ld_c + p.half + c, du, 4u, true);
      }
    }
  } else {
    const uint32_t second = kForm == kWeights && r >= p.half ? 1u : 0u, row = r - second * p.half;
    if (row >= p.rows) return;
    T* to = second ? (T*)p.c2 + (uint64_t)row * p.ld_c2 : (T*)p.c + (uint64_t)row * p.ld_c;
#pragma unroll
    for (int j = 0; j < kNF; ++j) {
      const uint32_t c = c0 + j * 16;
      put(to + c, sum[j], c < p.columns ? p.columns - c : 0u, p.wide);
    }
  }
}

template <class T, Form kForm, int BM, int BN, int WM, int WN>
struct Split {
  static constexpr bool kTwo = kForm == kForward || kForm == kSlopes;
  static constexpr int kRows = BM / WM, kCols = BN / WN, kMF = kRows / 16, kNF = kCols / 16, kLanes = WM * WN * 64;
  // first row and column of C that a lane of wavefront (wm, wn) holds in its i-th 16 rows
  __device__ static uint32_t row(uint32_t row0, uint32_t wm, uint32_t lane, int i) { return row0 + wm * kRows + i * 16 + lane % 16u; }
  __device__ static uint32_t column(uint32_t col0, uint32_t wn, uint32_t lane) { return (kTwo ? col0 / 2u + wn * (kCols / 2) : col0 + wn * kCols) + lane / 16u * 4u; }

  // (all of dh is asked for before any is needed: asked for while the products are formed it does not fit the registers)
  template <int kN>
  __device__ __forceinline__ static void finish(const MmArgs& p, uint32_t row0, uint32_t col0, uint32_t wm, uint32_t wn, uint32_t lane, int i0, const f32x4 (&sum)[kN][kNF]) {
    const uint32_t c = column(col0, wn, lane);
    Pack<T, 4> dh[kN][kNF / 2];
#pragma unroll
    for (int i = 0; i < kN; ++i)
      if (kForm == kSlopes) fetch_dh(p, row(row0, wm, lane, i0 + i), c, dh[i]);
    auto all = [&](auto kind) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        finish_rows<T, kForm, kNF, decltype(kind)::value>(p, row(row0, wm, lane, i0 + i), c, sum[i], dh[i]);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (!kTwo || p.act == FBX_ACT_SILU) all(Kind<FBX_ACT_SILU>());
    else if (p.act == FBX_ACT_GELU) all(Kind<FBX_ACT_GELU>());
    else if (p.act == FBX_ACT_RELU) all(Kind<FBX_ACT_RELU>());
    else all(Kind<FBX_ACT_SIGMOID>());
  }
};

// BM x BN of C a workgroup at a time, its WM x WN wavefronts side by side (kForward, kSlopes: BN / 2 columns of either
// product).  C's rows come from A; its columns from B, which is the first side of the matrix instructions, so that a lane holds
// four adjacent columns of a row.
// kStages: steps whose tiles are in LDS or on their way there.
// Bound by the matrix units where the product is large: 65,536 x 2,624 by 2 x 4,096 in bf16 takes 2.25 to 2.42 ms from card to card,
// 1.16 to 1.25 PFLOP/s; they are busy 60 % of the cycles, at a clock that the power they draw keeps at 1.8 of 2.4 GHz, and reads from
// LDS meet no bank conflict.  A library's product of the same two matrices, without the activation, reaches 1.37.  The three products
// of a gradient of 16,384 records take 1.9 to 2.0 ms, 1.05 to 1.11 PFLOP/s, dh and both slopes moved in the first one's epilogue.  In 32 bits
// 4,096 x 384 by 2 x 1,024 and back is 175 us, 110 of 154 TFLOP/s.  Measured and slower: 32 x 32 x 16 instructions (8 %),
// workgroups that stay and take tile after tile (6 %), four wavefronts of 128 x 128, which read a third less from LDS (compiled,
// their sums are moved from register to register; with the instructions written out and loads spread among them the
// forward product takes 2 % less time and the gradient 5 % more: an epilogue has half the wavefronts).
template <class T, Form kForm, int BM, int BN, int WM, int WN, int kStages>
__global__ __launch_bounds__(WM * WN * 64) void k_mm(MmArgs p) {
#ifdef __HIP_DEVICE_COMPILE__  // (the host's pass, which makes the launch stub of it, does not know the buffer's type)
  typedef Split<T, kForm, BM, BN, WM, WN> S;
  constexpr bool kTwo = S::kTwo;
  constexpr int kWaves = WM * WN, kMF = S::kMF, kNF = S::kNF, kDepth = kStepBytes / sizeof(T);
  typedef Tile<T, BM, kWaves, kForm == kWeights> TileA;
  typedef Tile<T, BN, kWaves, !kTwo> TileB;
  // (arrays of their own, so that the compiler knows which of them a load goes to)
  __shared__ alignas(1024) char a0[BM * kStepBytes], b0[BN * kStepBytes], a1[BM * kStepBytes], b1[BN * kStepBytes];
  __shared__ alignas(1024) char a2[kStages > 2 ? BM * kStepBytes : 16], b2[kStages > 2 ? BN * kStepBytes : 16];
  __shared__ alignas(1024) char a3[kStages > 2 ? BM * kStepBytes : 16], b3[kStages > 2 ? BN * kStepBytes : 16];
  const uint32_t lane = threadIdx.x % 64u, wave = same(threadIdx.x / 64u), wm = wave % WM, wn = wave / WM;
  // Workgroups go to the eight dies in turn: each die takes a stretch of the whole tiles, then one of the shares.
  uint32_t t, first = 0, end = p.steps, part = 0;
  {
    const bool whole = blockIdx.x < p.whole;
    const uint32_t n = whole ? p.whole : gridDim.x - p.whole, i = whole ? blockIdx.x : blockIdx.x - p.whole, each = n / 8u, more = n % 8u, die = i % 8u;
    t = die * each + (die < more ? die : more) + i / 8u;
    if (!whole) {
      part = t;
      const uint32_t share = t % p.shares, steps = p.steps / p.shares, longer = p.steps % p.shares;
      first = share * steps + (share < longer ? share : longer);
      end = first + steps + (share < longer ? 1u : 0u);
      t = p.whole + t / p.shares;
    }
  }
  uint32_t row0, col0;
  place<BM, BN>(p, t, row0, col0);
  row0 = same(row0);  // (quotients are worked out in vector registers)
  col0 = same(col0);
  first = same(first);
  end = same(end);

  TileA ta;
  TileB tb;
  const bool up = kTwo && wave >= kWaves / 2;  // this wavefront loads of Wu
  const uint32_t turn = kForm == kInputs ? p.half / kDepth : 0u;  // kInputs: the first step whose lines are Wu's
  const char *a = (const char*)p.a, *b = (const char*)(up || (kForm == kInputs && first >= turn) ? p.b2 : p.b);
  const uint64_t ld_b = up || (kForm == kInputs && first >= turn) ? p.ld_b2 : p.ld_b;
  const uint32_t b_lines = kTwo && col0 / 2u < p.columns ? same(p.columns - col0 / 2u) : 0u;
  if (kForm == kWeights) {
    a += (uint64_t)row0 * sizeof(T);
    ta.begin(wave, lane, p.ld_a, 2 * p.half - row0);
  } else {
    a += (uint64_t)row0 * p.ld_a;
    ta.begin(wave, lane, p.ld_a, 0);
  }
  if (kTwo) {
    b += (uint64_t)(col0 / 2u) * ld_b;
    tb.begin(up ? wave - kWaves / 2 : wave, lane, ld_b, 0);
  } else {
    b += (uint64_t)col0 * sizeof(T);
    tb.begin(wave, lane, ld_b, p.b_columns - col0);
  }
  // (behind the last step: of nothing, so that every step's loads are as many)
  auto load = [&](char* to_a, char* to_b, uint32_t s) {
    const bool none = s >= end;
    if (kForm == kWeights) {
      const uint32_t left = none ? 0u : p.depth - s * kDepth;
      ta.load((lds_char*)to_a, a + (uint64_t)s * kDepth * p.ld_a, p.ld_a, left, 0, (2 * p.half - row0) * sizeof(T), wave);
      tb.load((lds_char*)to_b, b + (uint64_t)s * kDepth * p.ld_b, p.ld_b, left, 0, (p.b_columns - col0) * sizeof(T), wave);
    } else {
      const uint32_t left = (kTwo ? p.depth : 2 * p.half) - s * kDepth;
      ta.load((lds_char*)to_a, a + s * kStepBytes, p.ld_a, none ? 0u : p.rows - row0, left, left * sizeof(T), wave);
      if (kTwo) {
        tb.load((lds_char*)to_b, b + s * kStepBytes, ld_b, none ? 0u : b_lines, left, left * sizeof(T), wave);
      } else {  // (the weights one below the other, each made up to `half` lines: a step's lines are of one of them)
        if (s == turn) {
          b = (const char*)p.b2 + (uint64_t)col0 * sizeof(T);
          tb.begin(wave, lane, p.ld_b2, p.b_columns - col0);
        }
        const uint32_t line = (s >= turn ? s - turn : s) * kDepth;
        const uint64_t ld = s >= turn ? p.ld_b2 : p.ld_b;
        tb.load((lds_char*)to_b, b + line * ld, ld, none ? 0u : p.depth - line, 0, (p.b_columns - col0) * sizeof(T), wave);
      }
    }
  };

  // Two halves of a step's depth in turn: while one is multiplied out of registers the other's rows are read from LDS.
  // A step's barrier lies between the halves: behind it the next step's tile is there (its loads had kStages - 1 steps) and
  // nobody reads this step's any more, so the loads of the step kStages later go there.
  f32x4 sum[kMF][kNF] = {};
  typename Frag<T>::type fa[2][kMF], fb[2][kNF];
  auto read = [&](int part, const char* in_a, const char* in_b) {
#pragma unroll
    for (int i = 0; i < kMF; ++i) fa[part][i] = TileA::read((const lds_char*)in_a, wm * S::kRows + i * 16, part, lane);
#pragma unroll
    for (int j = 0; j < kNF; ++j) {
      const uint32_t first = !kTwo ? wn * S::kCols + j * 16 : wn * (S::kCols / 2) + j % (kNF / 2) * 16 + j / (kNF / 2) * (BN / 2);
      fb[part][j] = TileB::read((const lds_char*)in_b, first, part, lane);
    }
  };
  auto multiply = [&](int part) {
#pragma unroll
    for (int j = 0; j < kNF; ++j)
#pragma unroll
      for (int i = 0; i < kMF; ++i) sum[i][j] = mma(fb[part][j], fa[part][i], sum[i][j]);
  };
  // All but the last `steps` steps' loads are done, in every wavefront, and so are its reads.  (Loads that go past the
  // registers are not among what a barrier waits for, and it is not to wait for more of them than this.)
  auto arrived = [](auto steps) {
    constexpr int n = decltype(steps)::value * (TileA::kLoads + TileB::kLoads);
    static_assert(n < 64, "");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt((n & 15) | (n >> 4) << 14 | 0x0070);  // (vmcnt n, lgkmcnt 0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](char* at_a, char* at_b, const char* next_a, const char* next_b, uint32_t s) {
    read(1, at_a, at_b);
    multiply(0);
    arrived(Kind<kStages - 2>());
    load(at_a, at_b, s + kStages);
    __builtin_amdgcn_sched_barrier(0);
    read(0, next_a, next_b);  // (behind the last step: what is there, unused)
    multiply(1);
    __builtin_amdgcn_sched_barrier(0);
  };
  load(a0, b0, first);
  load(a1, b1, first + 1);
  if constexpr (kStages == 4) {
    load(a2, b2, first + 2);
    load(a3, b3, first + 3);
  }
  arrived(Kind<kStages - 1>());
  read(0, a0, b0);
  if constexpr (kStages == 4) {  // (left from within: on a way round that skips steps the compiler would wait for their loads)
    for (uint32_t s = first;; s += 4) {
      step(a0, b0, a1, b1, s);
      if (s + 1 >= end) break;
      step(a1, b1, a2, b2, s + 1);
      if (s + 2 >= end) break;
      step(a2, b2, a3, b3, s + 2);
      if (s + 3 >= end) break;
      step(a3, b3, a0, b0, s + 3);
      if (s + 4 >= end) break;
    }
  } else {  // (not left from within: that costs a copy of the sums, which large tiles have no registers for)
    for (uint32_t s = first; s < end; s += 2) {
      step(a0, b0, a1, b1, s);
      if (s + 1 < end) step(a1, b1, a0, b0, s + 1);
    }
  }
  arrived(Kind<0>());  // (nothing is to land in LDS that may be another workgroup's by then)

  if (blockIdx.x < p.whole) {
    S::template finish<kMF>(p, row0, col0, wm, wn, lane, 0, sum);
  } else {
    f32x4* to = p.parts + (uint64_t)part * (BM * BN / 4) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kMF; ++i)
#pragma unroll
      for (int j = 0; j < kNF; ++j) to[(i * kNF + j) * S::kLanes] = sum[i][j];
  }
#else
  (void)p;
#endif
}

// Adds up the shares of a tile, in the order of their steps, and finishes it.  A workgroup takes 16 rows of each
// wavefront's part of it.
template <class T, Form kForm, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void k_join(MmArgs p) {
  typedef Split<T, kForm, BM, BN, WM, WN> S;
  f32x4 sum[1][S::kNF] = {};
  const f32x4* in = p.parts + (uint64_t)blockIdx.x * p.shares * (BM * BN / 4) + (blockIdx.y * S::kNF) * S::kLanes + threadIdx.x;
  for (uint32_t n = 0; n < p.shares; ++n, in += BM * BN / 4)
#pragma unroll
    for (int j = 0; j < S::kNF; ++j) sum[0][j] += in[j * S::kLanes];
  uint32_t row0, col0;
  place<BM, BN>(p, p.whole + blockIdx.x, row0, col0);
  const uint32_t wave = threadIdx.x / 64u;
  S::template finish<1>(p, row0, col0, wave % WM, wave / WM, threadIdx.x % 64u, (int)blockIdx.y, sum);
}

// Up to 16 records: the weights are read once, straight into the matrix units' registers, and bound it.  A workgroup takes
// 16 columns of either product, its wavefronts a share of the depth each; their sums meet in LDS and are added in order.
// kWhole: rows begin at, and are, whole 16-byte loads; else they are read element by element, which for so few records
// costs less than a copy of the weights.  One record, 2 x 4,096 x 1,536 in bf16: 5.6 us, 25 MB at 4.5 TB/s.
constexpr int kFewWaves = 8;
template <class T, bool kWhole>
__global__ __launch_bounds__(kFewWaves * 64) void k_few(MmArgs p) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef typename Frag<T>::type F;
  constexpr uint32_t kLanes = 16 / sizeof(T), kStep = 4 * kLanes, kAhead = 4;
  __shared__ f32x4 sums[kFewWaves][2][64];
  const uint32_t lane = threadIdx.x % 64u, wave = threadIdx.x / 64u, i = lane % 16u, g = lane / 16u;
  const uint32_t n = blockIdx.x * 16u + i;
  const T* rows[3] = {(const T*)((const char*)p.b + n * p.ld_b), (const T*)((const char*)p.b2 + n * p.ld_b2), (const T*)((const char*)p.a + i * p.ld_a)};
  const bool in[3] = {n < p.columns, n < p.columns, i < p.rows};
  auto load = [&](int which, uint32_t k) {
    F f = {};
    if (in[which]) {
      if (kWhole) {
        if (k < p.depth) f = *(const F*)(rows[which] + k);
      } else {
#pragma unroll
        for (uint32_t e = 0; e < kLanes; ++e)
          if (k + e < p.depth) f[e] = rows[which][k + e];
      }
    }
    return f;
  };
  f32x4 sum[2] = {};
  for (uint32_t k0 = wave * kStep + g * kLanes; k0 - g * kLanes < p.depth; k0 += kFewWaves * kStep * kAhead) {
    F f[kAhead][3];
#pragma unroll
    for (uint32_t u = 0; u < kAhead; ++u)
#pragma unroll
      for (int which = 0; which < 3; ++which) f[u][which] = load(which, k0 + u * kFewWaves * kStep);
#pragma unroll
    for (uint32_t u = 0; u < kAhead; ++u) {
      sum[0] = mma(f[u][0], f[u][2], sum[0]);
      sum[1] = mma(f[u][1], f[u][2], sum[1]);
    }
  }
  sums[wave][0][lane] = sum[0];
  sums[wave][1][lane] = sum[1];
  __syncthreads();
  if (wave) return;
  f32x4 both[2] = {};
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    both[0] += sums[w][0][lane];
    both[1] += sums[w][1][lane];
  }
  const uint32_t c = blockIdx.x * 16u + g * 4u;
  const Pack<T, 4> none[1] = {};
  if (p.act == FBX_ACT_SILU) finish_rows<T, kForward, 2, FBX_ACT_SILU>(p, i, c, both, none);
  else if (p.act == FBX_ACT_GELU) finish_rows<T, kForward, 2, FBX_ACT_GELU>(p, i, c, both, none);
  else if (p.act == FBX_ACT_RELU) finish_rows<T, kForward, 2, FBX_ACT_RELU>(p, i, c, both, none);
  else finish_rows<T, kForward, 2, FBX_ACT_SIGMOID>(p, i, c, both, none);
#else
  (void)p;
#endif
}

// Copies of up to three matrices (blockIdx.y) whose rows of n elements are made `wide` long, whole 16-byte stores, with zeros
// behind.  2^lanes_log2 lanes a row, or all of a workgroup's; no quotient is taken (65,536 x 411 by 2 x 773 in bf16: the forward call
// 212 us, against 244 with an element a lane and its row by division).
struct PadArgs {
  const void* from[3];
  void* to[3];
  uint64_t ld[3], rows[3];
  uint32_t n, wide, lanes_log2;
};
template <class T>
__global__ __launch_bounds__(256) void k_pad_rows(PadArgs a) {
  constexpr uint32_t kEach = 16 / sizeof(T);
  const T* from = (const T*)a.from[blockIdx.y];
  T* to = (T*)a.to[blockIdx.y];
  const uint64_t ld = a.ld[blockIdx.y], rows = a.rows[blockIdx.y];
  const uint32_t lanes = 1u << a.lanes_log2, mine = threadIdx.x & (lanes - 1u), at_once = 256u >> a.lanes_log2;
  for (uint64_t r = (uint64_t)blockIdx.x * at_once + (threadIdx.x >> a.lanes_log2); r < rows; r += (uint64_t)gridDim.x * at_once)
    for (uint32_t c = mine * kEach; c < a.wide; c += lanes * kEach) {
      Pack<T, kEach> p;
#pragma unroll
      for (uint32_t e = 0; e < kEach; ++e) p.v[e] = c + e < a.n ? from[r * ld + c + e] : (T)0.f;
      *(Pack<T, kEach>*)(to + r * a.wide + c) = p;
    }
}

// How a product is cut: tiles of C, of which the last `shared` are shared out by steps of depth.
struct Cut {
  uint32_t size;  // 0: tiles of 256 x 256, 1: 128 x 128, 2: 64 x 64
  uint32_t row_tiles, column_tiles, steps, shared, shares;
  uint64_t parts_bytes() const { return shared ? (uint64_t)shared * shares * kSide[size] * kSide[size] * 4 : 0; }
  static constexpr uint32_t lanes(uint32_t size) { return size ? 256 : 512; }  // of a workgroup
  static constexpr uint32_t kSide[3] = {256, 128, 64};
};
constexpr uint32_t Cut::kSide[3];

// The cut that takes the least time, by what was measured (forward product, microseconds).  A workgroup takes `begin` and
// its steps; `lone`: a step of one that has a compute unit to itself, `full`: of one among the `at_once` that fit one.
// Large tiles read less from LDS for a product of 16-bit numbers (1.6 us for 256 x 256 a step and compute unit, against 1.9
// in tiles of 128 and 2.4 in tiles of 64), small ones begin sooner and leave fewer compute units idle; products of 32-bit numbers are bound by the matrix
// units at every size.  Tiles that do not fill the card another time can be shared out by steps, which
// costs a launch and their sums' way through memory: a write and a read at 5 TB/s.
// size kNoCut: more tiles of any size than a launch has workgroups.
constexpr uint32_t kNoCut = 3;
Cut cut(uint64_t rows, uint64_t columns, uint64_t steps, bool single) {
  struct Cost { uint32_t at_once; double begin, lone, full; };
  constexpr Cost kCost[2][3] = {{{1, 8, 1.4, 1.6}, {2, 5.5, 0.5, 0.95}, {2, 3.5, 0.22, 0.3}}, {{1, 10, 7.0, 7.0}, {2, 6, 1.95, 3.9}, {4, 3, 0.55, 2.15}}};
  constexpr uint32_t kUnits = 256;  // compute units
  constexpr double kJoin = 3.5, kBytes = 2 / 5e6;
  Cut best{};
  best.size = kNoCut;
  double least = 0;
  if (!steps) steps = 1;
  for (uint32_t size = 0; size < 3; ++size) {
    const Cost& c = kCost[single][size];
    const uint64_t side = Cut::kSide[size], row_tiles = ceil_div(rows, side), column_tiles = ceil_div(columns, side), tiles = row_tiles * column_tiles;
    const uint64_t slots = kUnits * c.at_once, rest = tiles % slots;
    if (tiles + 16 * slots > most_blocks(Cut::lanes(size))) continue;
    for (uint32_t n = 1; n <= 16 && (n == 1 || (rest && 4 * n <= steps)); ++n) {
      const uint64_t groups = rest * n, busy = ceil_div(groups < slots ? groups : slots, kUnits);
      const double step = c.full * busy / c.at_once;
      double takes = (double)(tiles / slots) * (c.begin + steps * c.full) + (double)ceil_div(groups, slots) * (c.begin + (double)ceil_div(steps, n) * (step > c.lone ? step : c.lone));
      if (n > 1) takes += kJoin + (double)groups * side * side * 4 * kBytes;
      if (!least || takes < least) {
        least = takes;
        best = Cut{size, (uint32_t)row_tiles, (uint32_t)column_tiles, (uint32_t)steps, n > 1 ? (uint32_t)rest : 0u, n > 1 ? n : 0u};
      }
    }
  }
  return best;
}

template <class T, Form kForm, int BM, int BN, int WM, int WN, int kStages>
void launch(const MmArgs& p, uint32_t shared, hipStream_t stream) {
  launch_on(stream, k_mm<T, kForm, BM, BN, WM, WN, kStages>, dim3(p.whole + shared * p.shares), dim3(WM * WN * 64), 0, p);
  if (shared) launch_on(stream, k_join<T, kForm, BM, BN, WM, WN>, dim3(shared, BM / WM / 16), dim3(WM * WN * 64), 0, p);
}
template <class T, Form kForm>
void launch_by_size(const MmArgs& p, const Cut& c, hipStream_t stream) {
  if (c.size == 0) launch<T, kForm, 256, 256, 2, 4, 2>(p, c.shared, stream);
  else if (c.size == 1) launch<T, kForm, 128, 128, 2, 2, 2>(p, c.shared, stream);
  else launch<T, kForm, 64, 64, 2, 2, sizeof(T) == 2 ? 4 : 2>(p, c.shared, stream);
}
template <Form kForm>
void launch_by_type(MmArgs& p, const Cut& c, fbx_dtype t, char* parts, hipStream_t stream) {
  p.row_tiles = c.row_tiles;
  p.column_tiles = c.column_tiles;
  p.steps = c.steps;
  p.whole = c.row_tiles * c.column_tiles - c.shared;
  p.shares = c.shares;
  p.parts = (f32x4*)parts;
  if (t == FBX_F32) launch_by_size<float, kForm>(p, c, stream);
  else if (t == FBX_F16) launch_by_size<_Float16, kForm>(p, c, stream);
  else launch_by_size<__bf16, kForm>(p, c, stream);
}

template <class T>
void launch_few(const MmArgs& p, bool whole, hipStream_t stream) {
  const dim3 grid((uint32_t)ceil_div(p.columns, 16));
  if (whole) launch_on(stream, k_few<T, true>, grid, dim3(kFewWaves * 64), 0, p);
  else launch_on(stream, k_few<T, false>, grid, dim3(kFewWaves * 64), 0, p);
}
void launch_few_by_type(const MmArgs& p, fbx_dtype t, bool whole, hipStream_t stream) {
  if (t == FBX_F32) launch_few<float>(p, whole, stream);
  else if (t == FBX_F16) launch_few<_Float16>(p, whole, stream);
  else launch_few<__bf16>(p, whole, stream);
}

fbx_status check(const fbx_gated* g) {
  if (!g) return refuse(FBX_E_ARG, "g is NULL");
  if (!known(g->dtype)) return refuse(FBX_E_ARG, "unknown dtype");
  if (g->act < FBX_ACT_SILU || g->act > FBX_ACT_SIGMOID) return refuse(FBX_E_ARG, "unknown act");
  if (g->records >> 31) return refuse(FBX_E_ARG, "records must be below 2^31");
  if (!g->inputs || g->inputs > 1u << 20 || !g->hidden || g->hidden > 1u << 20) return refuse(FBX_E_ARG, "inputs and hidden must be 1 .. 2^20");
  if (g->ld_x < g->inputs || g->ld_w_gate < g->inputs || g->ld_w_up < g->inputs) return refuse(FBX_E_ARG, "a stride is smaller than inputs");
  if ((g->ld_x | g->ld_w_gate | g->ld_w_up) >> 22) return refuse(FBX_E_ARG, "strides must be below 2^22");
  return FBX_OK;
}
fbx_status check_pointers(const fbx_gated* g, uintptr_t others) {
  if (!g->d_w_gate || !g->d_w_up || (g->records && !g->d_x)) return refuse(FBX_E_ARG, "d_x, d_w_gate or d_w_up is NULL");
  if (((uintptr_t)g->d_x | (uintptr_t)g->d_w_gate | (uintptr_t)g->d_w_up | others) % size_of(g->dtype)) return refuse(FBX_E_ARG, "a matrix is not aligned to its elements");
  return FBX_OK;
}
// What a call keeps in its scratch, and what the kernels read: a matrix whose rows are not whole 16-byte loads (its
// address, its stride or its width) is first copied to one whose are.
constexpr uint32_t kFewRecords = 16;
struct Shape {
  uint32_t size, lanes;        // bytes of an element; elements of a load
  uint32_t wide;               // inputs, rounded up to whole loads
  uint32_t half;               // hidden, rounded up to a step of depth
  bool few;                    // so few records that the weights are read as they are
  bool pad[3];                 // x, w_gate, w_up
  uint64_t at[3], slopes, parts, bytes;
  Cut forward, inputs, weights;
  bool fits() const { return forward.size != kNoCut && inputs.size != kNoCut && weights.size != kNoCut; }
};

Shape shape_of(const fbx_gated* g, bool backward) {
  Shape s{};
  s.size = size_of(g->dtype);
  s.lanes = 16u / s.size;
  s.wide = (uint32_t)round_up(g->inputs, s.lanes);
  s.half = (uint32_t)round_up(g->hidden, kStepBytes / s.size);
  s.few = !backward && g->records <= kFewRecords;
  const void* from[3] = {g->d_x, g->d_w_gate, g->d_w_up};
  const uint64_t ld[3] = {g->ld_x, g->ld_w_gate, g->ld_w_up};
  auto take = [&](uint64_t bytes) {
    const uint64_t was = s.bytes;
    s.bytes = round_up(s.bytes + bytes, 256);
    return was;
  };
  for (int i = 0; i < 3; ++i) {
    s.pad[i] = g->inputs % s.lanes || ld[i] % s.lanes || (uintptr_t)from[i] % 16u;
    s.at[i] = take(s.pad[i] && !s.few ? (i ? g->hidden : g->records) * (uint64_t)s.wide * s.size : 0);
  }
  const uint64_t depth = kStepBytes / s.size;
  s.forward = cut(g->records, 2ull * (backward ? s.half : g->hidden), ceil_div(s.wide, depth), s.size == 4);
  uint64_t parts = s.few ? 0 : s.forward.parts_bytes();
  if (backward) {
    s.slopes = take(g->records * 2ull * s.half * s.size);
    s.inputs = cut(g->records, g->inputs, 2ull * s.half / depth, s.size == 4);
    s.weights = cut(2ull * s.half, g->inputs, ceil_div(g->records, depth), s.size == 4);
    for (uint64_t b : {s.inputs.parts_bytes(), s.weights.parts_bytes()}) parts = b > parts ? b : parts;
  }
  s.parts = take(parts);
  return s;
}

// Fills in where the kernels read x and the weights, copying those that need it.
void operands(const fbx_gated* g, const Shape& s, char* scratch, const void* (&from)[3], uint64_t (&ld)[3], hipStream_t stream) {
  from[0] = g->d_x;
  from[1] = g->d_w_gate;
  from[2] = g->d_w_up;
  ld[0] = g->ld_x;
  ld[1] = g->ld_w_gate;
  ld[2] = g->ld_w_up;
  PadArgs a{};
  a.n = g->inputs;
  a.wide = s.wide;
  uint32_t n = 0;
  uint64_t most = 0;
  for (int i = 0; i < 3; ++i) {
    const uint64_t rows = i ? g->hidden : g->records;
    if (s.pad[i] && !s.few && rows) {
      a.from[n] = from[i];
      a.ld[n] = ld[i];
      a.to[n] = scratch + s.at[i];
      a.rows[n++] = rows;
      most = rows > most ? rows : most;
    }
    if (s.pad[i] && !s.few) {
      from[i] = scratch + s.at[i];
      ld[i] = s.wide;
    }
    ld[i] *= s.size;
  }
  if (!n) return;
  while (a.lanes_log2 < 8u && (s.lanes << a.lanes_log2) < s.wide) ++a.lanes_log2;
  const uint64_t blocks = ceil_div(most, 256u >> a.lanes_log2);
  const dim3 grid((uint32_t)(blocks < 65536 ? blocks : 65536), n);
  if (s.size == 4u) launch_on(stream, k_pad_rows<float>, grid, dim3(256), 0, a);
  else launch_on(stream, k_pad_rows<_Float16>, grid, dim3(256), 0, a);
}

bool four_at_a_time(const void* p, uint64_t ld, uint32_t size) { return (uintptr_t)p % (4 * size) == 0 && ld % 4 == 0; }

fbx_status check_scratch(const fbx_gated* g, int backward, const void* d_scratch, uint64_t scratch_bytes) {
  uint64_t need = 0;
  fbx_gated_scratch(g, backward, &need);
  if (need && (!d_scratch || (uintptr_t)d_scratch % 256u)) return refuse(FBX_E_ARG, "d_scratch is NULL or not 256-byte aligned");
  return scratch_bytes < need ? refuse(FBX_E_NOMEM, "scratch too small: fbx_gated_scratch gives its size") : FBX_OK;
}

}  // namespace
}  // namespace train
}  // namespace fbx

using namespace fbx::train;

extern "C" fbx_status fbx_gated_scratch(const fbx_gated* g, int backward, uint64_t* bytes) {
  const fbx_status st = check(g);
  if (st != FBX_OK) return st;
  if (!bytes) return refuse(FBX_E_ARG, "bytes is NULL");
  *bytes = shape_of(g, backward != 0).bytes;
  return FBX_OK;
}

extern "C" fbx_status fbx_gated_forward(const fbx_gated* g, void* d_h, uint64_t ld_h, void* d_scratch, uint64_t scratch_bytes, void* hip_stream) {
  fbx_status st = check(g);
  if (st == FBX_OK) st = check_pointers(g, (uintptr_t)d_h);
  if (st == FBX_OK) st = check_scratch(g, 0, d_scratch, scratch_bytes);
  if (st != FBX_OK) return st;
  if (ld_h < g->hidden || ld_h >> 22) return refuse(FBX_E_ARG, "ld_h is smaller than hidden, or 2^22 or more");
  if (!g->records) return FBX_OK;
  if (!d_h) return refuse(FBX_E_ARG, "d_h is NULL");
  const hipStream_t stream = (hipStream_t)hip_stream;
  const Shape s = shape_of(g, false);
  if (!s.fits()) return refuse(FBX_E_ARG, "records x hidden is too large for one call");
  const void* from[3];
  uint64_t ld[3];
  operands(g, s, (char*)d_scratch, from, ld, stream);
  MmArgs p{};
  p.a = from[0];
  p.b = from[1];
  p.b2 = from[2];
  p.ld_a = ld[0];
  p.ld_b = ld[1];
  p.ld_b2 = ld[2];
  p.c = d_h;
  p.ld_c = ld_h;
  p.rows = (uint32_t)g->records;
  p.columns = g->hidden;
  p.depth = s.few ? g->inputs : s.wide;
  p.act = g->act;
  p.wide = four_at_a_time(d_h, ld_h, s.size);
  if (s.few) {
    launch_few_by_type(p, g->dtype, !(s.pad[0] || s.pad[1] || s.pad[2]), stream);
    return launched();
  }
  launch_by_type<kForward>(p, s.forward, g->dtype, (char*)d_scratch + s.parts, stream);
  return launched();
}

extern "C" fbx_status fbx_gated_backward(const fbx_gated* g, const void* d_dh, uint64_t ld_dh, void* d_dx, uint64_t ld_dx, void* d_dw_gate,
                                         uint64_t ld_dw_gate, void* d_dw_up, uint64_t ld_dw_up, void* d_scratch, uint64_t scratch_bytes,
                                         void* hip_stream) {
  fbx_status st = check(g);
  if (st == FBX_OK) st = check_pointers(g, (uintptr_t)d_dh | (uintptr_t)d_dx | (uintptr_t)d_dw_gate | (uintptr_t)d_dw_up);
  if (st != FBX_OK) return st;
  if (ld_dh < g->hidden || ld_dh >> 22) return refuse(FBX_E_ARG, "ld_dh is smaller than hidden, or 2^22 or more");
  if (!d_dw_gate != !d_dw_up) return refuse(FBX_E_ARG, "d_dw_gate and d_dw_up are given together or not at all");
  if ((d_dx && (ld_dx < g->inputs || ld_dx >> 22)) || (d_dw_gate && (ld_dw_gate < g->inputs || ld_dw_up < g->inputs || (ld_dw_gate | ld_dw_up) >> 22)))
    return refuse(FBX_E_ARG, "a stride of a gradient is smaller than inputs, or 2^22 or more");
  if (g->records && !d_dh) return refuse(FBX_E_ARG, "d_dh is NULL");
  st = check_scratch(g, 1, d_scratch, scratch_bytes);
  if (st != FBX_OK) return st;
  if (!d_dx && !d_dw_gate) return FBX_OK;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const Shape s = shape_of(g, true);
  if (!s.fits()) return refuse(FBX_E_ARG, "records x hidden is too large for one call");
  char* scratch = (char*)d_scratch;
  const void* from[3];
  uint64_t ld[3];
  operands(g, s, scratch, from, ld, stream);
  char* parts = scratch + s.parts;
  if (g->records) {
    MmArgs p{};
    p.a = from[0];
    p.b = from[1];
    p.b2 = from[2];
    p.ld_a = ld[0];
    p.ld_b = ld[1];
    p.ld_b2 = ld[2];
    p.dh = d_dh;
    p.ld_dh = ld_dh;
    p.c = scratch + s.slopes;
    p.ld_c = 2ull * s.half;
    p.rows = (uint32_t)g->records;
    p.columns = g->hidden;
    p.half = s.half;
    p.depth = s.wide;
    p.act = g->act;
    p.wide = four_at_a_time(d_dh, ld_dh, s.size);
    launch_by_type<kSlopes>(p, s.forward, g->dtype, parts, stream);
  }
  if (g->records && d_dx) {
    MmArgs p{};
    p.a = scratch + s.slopes;
    p.ld_a = 2ull * s.half * s.size;
    p.b = from[1];
    p.b2 = from[2];
    p.ld_b = ld[1];
    p.ld_b2 = ld[2];
    p.c = d_dx;
    p.ld_c = ld_dx;
    p.rows = (uint32_t)g->records;
    p.columns = g->inputs;
    p.depth = g->hidden;
    p.half = s.half;
    p.b_columns = s.wide;
    p.wide = four_at_a_time(d_dx, ld_dx, s.size);
    launch_by_type<kInputs>(p, s.inputs, g->dtype, parts, stream);
  }
  if (d_dw_gate) {
    MmArgs p{};
    p.a = scratch + s.slopes;
    p.ld_a = 2ull * s.half * s.size;
    p.b = from[0];
    p.ld_b = ld[0];
    p.c = d_dw_gate;
    p.ld_c = ld_dw_gate;
    p.c2 = d_dw_up;
    p.ld_c2 = ld_dw_up;
    p.rows = g->hidden;
    p.columns = g->inputs;
    p.depth = (uint32_t)g->records;
    p.half = s.half;
    p.b_columns = s.wide;
    p.wide = four_at_a_time(d_dw_gate, ld_dw_gate, s.size) && four_at_a_time(d_dw_up, ld_dw_up, s.size);
    launch_by_type<kWeights>(p, s.weights, g->dtype, parts, stream);
  }
  return launched();
}

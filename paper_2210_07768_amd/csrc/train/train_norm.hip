// The norm of rows before a block (`norm`), what joins a block's result to the residual stream, with the next block's norm
// (`join`), and their gradients.
#include "train_common.h"

#include <float.h>
#include <math.h>

namespace fbx {
namespace train {
namespace {

constexpr uint32_t kPack = 8;                 // adjacent elements of a lane
constexpr uint32_t kMostLanes = 512;          // of a row, and of a workgroup
constexpr int kMostPacks = 4;                 // of a lane
static_assert(FBX_NORM_MOST == kMostPacks * kMostLanes * kPack, "a row is held by a workgroup's registers");

// Eight adjacent elements, in whole loads and stores wherever they begin: a row that is aligned to its elements only is moved
// sixteen bytes a lane like any other (the hardware takes such addresses), so odd widths and strides need no form of their own.
template <class X>
struct Raw {
  X v[kPack];
};

// How a row lies in lanes: fewer than 8 elements in one lane, up to 64 packs in less than a wavefront, more in whole wavefronts, 1, 2 or 4 to
// a lane.
enum Shape { kTiny1, kNarrow1, kWide1, kWide2, kWide4 };
constexpr int packs_of(Shape s) { return s == kWide4 ? 4 : s == kWide2 ? 2 : 1; }

// A workgroup's lanes: `slots` rows at a time, `lanes` to a row: a power of two below 64, or whole wavefronts (kWide).
template <bool kWide>
struct Group {
  uint32_t lanes, slot, mine, waves;
  float* shared;   // two times what a reduction leaves there, in turn
  uint32_t turn;

  __device__ Group(uint32_t lanes_, float* shared_) : lanes(lanes_), slot(threadIdx.x / lanes_), mine(threadIdx.x % lanes_), waves(lanes_ / 64u), shared(shared_), turn(0) {}

  // Sums over a row's lanes, in all of them.  Every lane of the workgroup takes part.
  template <int kN>
  __device__ __forceinline__ void sum(float (&v)[kN]) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      v[i] = sixteen(v[i], kWide ? 64u : lanes);
      if (kWide || lanes > 16u) {  // (both give each lane the sums of both halves)
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
        const uint32_t one = p[0], other = p[1];
        v[i] = __uint_as_float(one) + __uint_as_float(other);
      }
      if (kWide || lanes > 32u) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
        const uint32_t one = p[0], other = p[1];
        v[i] = __uint_as_float(one) + __uint_as_float(other);
      }
    }
#endif
    if (!kWide || waves == 1u) return;
    // (a wavefront that writes here for the next reduction but one has met all others at the next one's barrier, behind their reads)
    float* at = shared + turn * kWaves * kMostSums;
    turn ^= 1u;
    const uint32_t wave = threadIdx.x / 64u, lane = threadIdx.x % 64u;
    if (lane == 0u)
#pragma unroll
      for (int i = 0; i < kN; ++i) at[i * kWaves + wave] = v[i];
    __syncthreads();
    // the row's wavefronts' sums, one a lane of eight
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = lane % kWaves < waves ? at[i * kWaves + slot * waves + lane % kWaves] : 0.f;
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = sixteen(v[i], kWaves);
  }
  // Sums over 2, 4, 8 or 16 neighbouring lanes, as many as `n` reaches.
  __device__ __forceinline__ static float sixteen(float v, uint32_t n) {
#ifdef __HIP_DEVICE_COMPILE__
    auto moved = [](float x, auto control) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(control)::value, 15, 15, true)); };
    if (n > 1u) v += moved(v, std::integral_constant<int, 0xb1>());    // lane ^ 1
    if (n > 2u) v += moved(v, std::integral_constant<int, 0x4e>());    // lane ^ 2
    if (n > 4u) v += moved(v, std::integral_constant<int, 0x141>());   // 7 - lane, of eight: the other four
    if (n > 8u) v += moved(v, std::integral_constant<int, 0x140>());   // 15 - lane, of sixteen: the other eight
#endif
    return v;
  }
  static constexpr uint32_t kMostSums = 3, kWaves = kMostLanes / 64;
  static constexpr uint32_t kShared = 2 * kWaves * kMostSums;
};

// A row's packs of this lane.  Pack j begins at column (j * lanes + mine) * 8, or, where it would reach beyond the row, as much
// earlier as makes it end there: its first `skip` elements are another pack's, which it works out and stores like that one, but leaves out
// of sums.  A pack behind the row is all another's (skip = 8).  So no lane's loads depend on a condition: where they did, the compiler
// waited for them at once, and none were on their way while a row was worked on.  Rows of fewer than 8 elements (kTiny) are moved one by
// one, behind `skip` places that hold nothing.
template <int kN, bool kTiny>
struct Columns {
  int32_t c[kN];
  uint32_t skip[kN];
  bool ragged;   // the row is no whole number of packs
  template <class G>
  __device__ Columns(const G& g, uint32_t dim) {
    ragged = dim % kPack != 0u;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const uint32_t from = (j * g.lanes + g.mine) * kPack, over = from + kPack > dim ? from + kPack - dim : 0u;
      c[j] = (int32_t)(from - over);
      skip[j] = over < kPack ? over : kPack;
    }
  }
  __device__ bool owns(int j) const { return skip[j] < kPack; }
  // The sum of f(j, e) over this lane's elements.
  template <class F>
  __device__ __forceinline__ float sum(F f) const {
    float s = 0.f;
    if (!ragged) {
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        float t = 0.f;
#pragma unroll
        for (uint32_t e = 0; e < kPack; ++e) t += f(j, e);
        s += owns(j) ? t : 0.f;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kN; ++j)
#pragma unroll
        for (uint32_t e = 0; e < kPack; ++e) s += e >= skip[j] ? f(j, e) : 0.f;
    }
    return s;
  }
};
template <int kN>
using Row = float[kN][kPack];
template <int kN, class F>
__device__ __forceinline__ void each(F f) {
#pragma unroll
  for (int j = 0; j < kN; ++j)
#pragma unroll
    for (uint32_t e = 0; e < kPack; ++e) f(j, e);
}

template <class X, int kN, bool kTiny>
__device__ __forceinline__ void fetch_row(Raw<X> (&to)[kN], const X* row, const Columns<kN, kTiny>& at) {
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    if (!kTiny) {
      __builtin_memcpy(&to[j], row + at.c[j], sizeof to[j]);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < kPack; ++e) to[j].v[e] = e >= at.skip[j] ? row[at.c[j] + (int32_t)e] : (X)0.f;
    }
  }
}
template <class X, int kN, bool kTiny>
__device__ __forceinline__ void put_row(X* row, const Row<kN>& from, const Columns<kN, kTiny>& at, bool in) {
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    if (!in || !at.owns(j)) continue;
    Raw<X> r;
#pragma unroll
    for (uint32_t e = 0; e < kPack; ++e) r.v[e] = (X)from[j][e];
    if (!kTiny) {
      __builtin_memcpy(row + at.c[j], &r, sizeof r);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < kPack; ++e)
        if (e >= at.skip[j]) row[at.c[j] + (int32_t)e] = r.v[e];
    }
  }
}
template <class X, int kN>
__device__ __forceinline__ void widen(Row<kN>& to, const Raw<X> (&from)[kN]) {
  each<kN>([&](int j, uint32_t e) { to[j][e] = (float)from[j].v[e]; });
}
// A vector of weights, in the block's type or 32 bits; `none` where there is none.
template <class T, int kN, bool kTiny>
__device__ __forceinline__ void fetch_vector(Row<kN>& to, const void* from, bool single, const Columns<kN, kTiny>& at, float none) {
  if (!from) {
    each<kN>([&](int j, uint32_t e) { to[j][e] = none; });
  } else if (single) {
    Raw<float> r[kN];
    fetch_row(r, (const float*)from, at);
    widen(to, r);
  } else {
    Raw<T> r[kN];
    fetch_row(r, (const T*)from, at);
    widen(to, r);
  }
}

// v becomes (v - mean) / sqrt(variance + eps), or v / sqrt(mean square + eps); returns 1 / sqrt.  Squares are taken behind the mean:
// sums of squares less a squared mean would lose what a large mean hides.  What rounding left of the mean is found beside them
// and taken off too, so that a row of one large number is one of zeros.
struct Scale {
  float dim, one_dim, eps;   // one_dim: 1 / dim
};
template <int kN, bool kTiny, class G>
__device__ __forceinline__ float normalise(Row<kN>& v, G& g, const Columns<kN, kTiny>& at, bool layer, Scale by) {
  float square, rest = 0.f;
  if (layer) {
    float all[1] = {at.sum([&](int j, uint32_t e) { return v[j][e]; })};
    g.sum(all);
    const float mean = all[0] / by.dim;   // (the quotient, so that the mean of equal numbers is theirs if their sum is exact)
    each<kN>([&](int j, uint32_t e) { v[j][e] -= mean; });
    float s[2] = {at.sum([&](int j, uint32_t e) { return v[j][e] * v[j][e]; }), at.sum([&](int j, uint32_t e) { return v[j][e]; })};
    g.sum(s);
    rest = s[1] * by.one_dim;
    square = s[0] * by.one_dim - rest * rest;
    if (square < 0.f) square = 0.f;
  } else {
    float s[1] = {at.sum([&](int j, uint32_t e) { return v[j][e] * v[j][e]; })};
    g.sum(s);
    square = s[0] * by.one_dim;
  }
  const float inverse = __builtin_amdgcn_rsqf(square + by.eps);   // (a unit in the last place; eps is a normal number)
  if (layer) {
    rest *= inverse;
    each<kN>([&](int j, uint32_t e) { v[j][e] = v[j][e] * inverse - rest; });
  } else {
    each<kN>([&](int j, uint32_t e) { v[j][e] *= inverse; });
  }
  return inverse;
}

// p, the gradient of normalised rows, becomes that of what they were made from: inverse (p - mean p - unit mean(p unit)), the
// first mean for a layer's norm only.  more: another sum over the row, where it is wanted too.
template <int kN, bool kTiny, class G>
__device__ __forceinline__ void denormalise(Row<kN>& p, const Row<kN>& unit, float inverse, G& g, const Columns<kN, kTiny>& at, bool layer, Scale by, bool wanted, float& more) {
  float along = at.sum([&](int j, uint32_t e) { return p[j][e] * unit[j][e]; }), mean = 0.f;
  if (layer && wanted) {
    float s[3] = {along, at.sum([&](int j, uint32_t e) { return p[j][e]; }), more};
    g.sum(s);
    along = s[0];
    mean = s[1] * by.one_dim * inverse;
    more = s[2];
  } else if (layer || wanted) {
    float s[2] = {along, layer ? at.sum([&](int j, uint32_t e) { return p[j][e]; }) : more};
    g.sum(s);
    along = s[0];
    if (layer) mean = s[1] * by.one_dim * inverse;
    else more = s[1];
  } else {
    float s[1] = {along};
    g.sum(s);
    along = s[0];
  }
  along *= inverse * by.one_dim;
  each<kN>([&](int j, uint32_t e) { p[j][e] = p[j][e] * inverse - mean - unit[j][e] * along; });
}

// Every sum of columns of a workgroup, its rows in a fixed order: those of a wavefront by halves, then wavefront by wavefront
// (or row by row, where a row has more than one).  shared: a line of `wide` floats for each sum and wavefront (or row).
template <int kSums, int kN, bool kWide, bool kTiny>
__device__ __forceinline__ void leave_sums(Row<kN> (&sums)[kSums], float* to, uint32_t wide, const Group<kWide>& g, const Columns<kN, kTiny>& at, uint32_t slots, float* shared) {
  if (!kWide)
    for (uint32_t d = g.lanes; d < 64u; d *= 2u)
#pragma unroll
      for (int i = 0; i < kSums; ++i)
#pragma unroll
        for (int j = 0; j < kN; ++j)
#pragma unroll
          for (uint32_t e = 0; e < kPack; ++e) sums[i][j][e] += __shfl_xor(sums[i][j][e], d, 64);
  const uint32_t lines = kWide ? slots : blockDim.x / 64u, line = kWide ? g.slot : threadIdx.x / 64u;
  const bool first = kWide || threadIdx.x % 64u < g.lanes;   // (of the lanes that hold the same sums now)
  // (LDS and memory are written apart, and no pointer is made that lies before either: `c` may be below 0)
  auto leave = [&](float* into, uint32_t base) {
#pragma unroll
    for (int i = 0; i < kSums; ++i)
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        if (!at.owns(j) || !first) continue;
        if (at.skip[j] == 0u) {
          Pack<float, kPack> v;
#pragma unroll
          for (uint32_t e = 0; e < kPack; ++e) v.v[e] = sums[i][j][e];
          *(Pack<float, kPack>*)(into + base + i * wide + (uint32_t)at.c[j]) = v;
        } else {
#pragma unroll
          for (uint32_t e = 0; e < kPack; ++e)
            if (e >= at.skip[j]) into[base + i * wide + (uint32_t)(at.c[j] + (int32_t)e)] = sums[i][j][e];
        }
      }
  };
  if (lines == 1u) {
    leave(to, 0u);
    return;
  }
  leave(shared, line * wide * kSums);
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < wide * kSums; c += blockDim.x) {
    float v = shared[c];
    for (uint32_t l = 1; l < lines; ++l) v += shared[l * wide * kSums + c];
    to[c] = v;
  }
}

struct NormArgs {
  const void *x, *weight, *dy;
  void *out, *dx;
  float* sums;                      // of a gradient: a row of `wide` floats a workgroup
  uint64_t ld_x, ld_out, ld_dy, ld_dx, rows;
  uint32_t dim, wide, lanes, slots;
  uint32_t layer, single;           // single: vectors are in 32 bits
  Scale by;
};

// R: of the residual stream; T: of the result.  A row's loads are on their way while the one before it is worked on, but for rows that
// leave no registers for it (kAhead).
// Bound by memory: 65,536 x 2,624 in bf16, 0.69 GB, takes 118 us, 5.8 TB/s (a copy of 1 GiB: 5.0).  One row: 2.0 us, the call 4.3 to 5.
template <int kN>
constexpr bool kAhead = kN == 1;

template <class R, class T, Shape kShape>
__global__ __launch_bounds__(kMostLanes) void k_norm(NormArgs p) {
  constexpr int kN = packs_of(kShape);
  constexpr bool kWide = kShape >= kWide1, kTiny = kShape == kTiny1;
  __shared__ float shared[Group<kWide>::kShared];
  Group<kWide> g(p.lanes, shared);
  const Columns<kN, kTiny> at(g, p.dim);

  Row<kN> weight;
  fetch_vector<T>(weight, p.weight, p.single, at, 1.f);
  const uint64_t stride = (uint64_t)gridDim.x * p.slots, last = p.rows - 1u;
  uint64_t r = (uint64_t)blockIdx.x * p.slots + g.slot;
  Raw<R> raw[kN];
  auto get = [&](uint64_t r) { fetch_row(raw, (const R*)p.x + (r < last ? r : last) * p.ld_x, at); };
  get(r);
  for (uint64_t r0 = (uint64_t)blockIdx.x * p.slots; r0 < p.rows; r0 += stride, r += stride) {
    Row<kN> v;
    widen(v, raw);
    if (kAhead<kN>) get(r + stride);
    normalise(v, g, at, p.layer, p.by);
    each<kN>([&](int j, uint32_t e) { v[j][e] *= weight[j][e]; });
    put_row((T*)p.out + r * p.ld_out, v, at, r < p.rows);
    if (!kAhead<kN>) get(r + stride);
  }
}

// dx, and a workgroup's sums of dy times the unit rows.  16,384 x 411 in f16, a layer's norm, rows 414 apart: 13.4 us of the call's 14.8, 40 MB at
// 3.0 TB/s; 300 vector instructions a row of 64 lanes are 8 us of it.  4,096 x 384 in f32: 6.5 of 9.5 us.
template <class R, class T, Shape kShape>
__global__ __launch_bounds__(kMostLanes) void k_norm_grad(NormArgs p) {
  constexpr int kN = packs_of(kShape);
  constexpr bool kWide = kShape >= kWide1, kTiny = kShape == kTiny1;
  __shared__ float shared[Group<kWide>::kShared];
  extern __shared__ __attribute__((aligned(32))) float columns[];
  Group<kWide> g(p.lanes, shared);
  const Columns<kN, kTiny> at(g, p.dim);

  Row<kN> weight, sums[1] = {};
  fetch_vector<T>(weight, p.weight, p.single, at, 1.f);
  const uint64_t stride = (uint64_t)gridDim.x * p.slots, last = p.rows - 1u;
  uint64_t r = (uint64_t)blockIdx.x * p.slots + g.slot;
  Raw<R> raw_x[kN];
  Raw<T> raw_dy[kN];
  auto get = [&](uint64_t r) {
    const uint64_t there = r < last ? r : last;
    fetch_row(raw_x, (const R*)p.x + there * p.ld_x, at);
    fetch_row(raw_dy, (const T*)p.dy + there * p.ld_dy, at);
  };
  get(r);
  for (uint64_t r0 = (uint64_t)blockIdx.x * p.slots; r0 < p.rows; r0 += stride, r += stride) {
    Row<kN> unit, d;
    widen(unit, raw_x);
    widen(d, raw_dy);
    if (kAhead<kN>) get(r + stride);
    const float inverse = normalise(unit, g, at, p.layer, p.by);
    if (r < p.rows) each<kN>([&](int j, uint32_t e) { sums[0][j][e] += d[j][e] * unit[j][e]; });
    if (p.dx) {
      float none = 0.f;
      each<kN>([&](int j, uint32_t e) { d[j][e] *= weight[j][e]; });
      denormalise(d, unit, inverse, g, at, p.layer, p.by, false, none);
      put_row((R*)p.dx + r * p.ld_dx, d, at, r < p.rows);
    }
    if (!kAhead<kN>) get(r + stride);
  }
  if (p.sums) leave_sums(sums, p.sums + (uint64_t)blockIdx.x * p.wide, p.wide, g, at, p.slots, columns);
}

struct JoinArgs {
  const void *x, *y, *gate, *weight, *scale, *next_weight, *dout, *dnext;
  void *out, *next, *dx, *dy, *dgate;
  float* sums;                      // of a gradient: two rows of `wide` floats a workgroup
  uint64_t ld_x, ld_y, ld_gate, ld_out, ld_next, ld_dout, ld_dnext, ld_dx, ld_dy, ld_dgate, rows;
  uint32_t dim, wide, lanes, slots;
  uint32_t layer, single, post, then, each, sigmoid;  // each: a gate for each element, not one a row
  Scale by;
  float number;                     // the scale, where it is no vector
};

// e^-a by the hardware's exponential and reciprocal (one unit in the last place each).
__device__ __forceinline__ float logistic(float a) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * -1.4426950408889634f)); }

// act(gate) of a row's elements, from their own gates or its only one.
template <class T, int kN>
__device__ __forceinline__ void open(Row<kN>& to, const Raw<T> (&gate)[kN], T only, const JoinArgs& p) {
  if (!p.gate) {
    each<kN>([&](int j, uint32_t e) { to[j][e] = 1.f; });
  } else if (!p.each) {
    const float a = p.sigmoid ? logistic((float)only) : (float)only;
    each<kN>([&](int j, uint32_t e) { to[j][e] = a; });
  } else if (p.sigmoid) {
    each<kN>([&](int j, uint32_t e) { to[j][e] = logistic((float)gate[j].v[e]); });
  } else {
    widen(to, gate);
  }
}

// A row's operands as they are in memory.
template <class R, class T, int kN>
struct Operands {
  Raw<R> x[kN], dout[kN];
  Raw<T> y[kN], gate[kN], dnext[kN];
  T only;   // a row's only gate
};

template <class T, int kN, bool kTiny>
__device__ __forceinline__ void fetch_vectors(Row<kN>& weight, Row<kN>& next_weight, const JoinArgs& p, const Columns<kN, kTiny>& at) {
  Row<kN> scale;
  fetch_vector<T>(weight, p.weight, p.single, at, 1.f);
  fetch_vector<T>(scale, p.scale, p.single, at, p.number);
  if (p.then) fetch_vector<T>(next_weight, p.next_weight, p.single, at, 1.f);
  each<kN>([&](int j, uint32_t e) { weight[j][e] *= scale[j][e]; });
}

// Bound by memory: 65,536 x 2,624, a stream in f32, the block's side in bf16, a gate for each element, the next norm: 2.4 GB in 440 us,
// 5.5 TB/s.  One row of 1,536: 3.0 us, the call 5.4 to 6.  Above 8,192 columns (kWide4) a lane's 32 elements of each do not fit the registers,
// 45 to 111 of which go by way of scratch memory: 2,048 x 16,384 of the same types 184 us, 2.6 TB/s.
template <class R, class T, Shape kShape>
__global__ __launch_bounds__(kMostLanes) void k_join(JoinArgs p) {
  constexpr int kN = packs_of(kShape);
  constexpr bool kWide = kShape >= kWide1, kTiny = kShape == kTiny1;
  __shared__ float shared[Group<kWide>::kShared];
  Group<kWide> g(p.lanes, shared);
  const Columns<kN, kTiny> at(g, p.dim);

  Row<kN> weight, next_weight;
  if (kAhead<kN>) fetch_vectors<T>(weight, next_weight, p, at);
  const uint64_t stride = (uint64_t)gridDim.x * p.slots, last = p.rows - 1u;
  uint64_t r = (uint64_t)blockIdx.x * p.slots + g.slot;
  Operands<R, T, kN> now{};
  auto get = [&](uint64_t r) {
    const uint64_t there = r < last ? r : last;
    fetch_row(now.y, (const T*)p.y + there * p.ld_y, at);
    if (p.gate && p.each) fetch_row(now.gate, (const T*)p.gate + there * p.ld_gate, at);
    if (p.gate && !p.each) now.only = ((const T*)p.gate)[there * p.ld_gate];
    fetch_row(now.x, (const R*)p.x + there * p.ld_x, at);
  };
  get(r);
  for (uint64_t r0 = (uint64_t)blockIdx.x * p.slots; r0 < p.rows; r0 += stride, r += stride) {
    if (!kAhead<kN>) fetch_vectors<T>(weight, next_weight, p, at);
    Row<kN> v, gate, x;
    widen(v, now.y);
    open(gate, now.gate, now.only, p);
    widen(x, now.x);
    if (kAhead<kN>) get(r + stride);
    if (p.post) normalise(v, g, at, p.layer, p.by);
    each<kN>([&](int j, uint32_t e) { v[j][e] = x[j][e] + gate[j][e] * weight[j][e] * v[j][e]; });
    put_row((R*)p.out + r * p.ld_out, v, at, r < p.rows);
    if (p.then) {
      normalise(v, g, at, p.layer, p.by);
      each<kN>([&](int j, uint32_t e) { v[j][e] *= next_weight[j][e]; });
      put_row((T*)p.next + r * p.ld_next, v, at, r < p.rows);
    }
    if (!kAhead<kN>) get(r + stride);
  }
}

// The stream is worked out again from x, y and the gate: to keep it would cost the forward pass a write of what is read here anyway.
// 16,384 x 2,624 in bf16 with a gate for each element and the next norm: 0.69 GB in 165 to 176 us, 3.9 to 4.2 TB/s.  141 registers let twelve
// wavefronts be on a compute unit; 463 vector instructions and 16 exponentials and reciprocals a row and wavefront are 0.1 ms of it, hidden in
// part.  With loads that depended on conditions, waited for at once, it took 346.  1,000 x 411: 8.5 of the call's 14 us, of which
// one row takes 6.8: instructions come from memory once a launch.  Scratch memory holds what the registers do not: above 4,096 columns 9 to 21
// registers (4,096 x 8,192, a stream in f32: 177 us, 4.2 TB/s), above 8,192 about 700 (2,048 x 16,384: 690 us, 1.1 TB/s).
template <class R, class T, Shape kShape>
__global__ __launch_bounds__(kMostLanes) void k_join_grad(JoinArgs p) {
  constexpr int kN = packs_of(kShape);
  constexpr bool kWide = kShape >= kWide1, kTiny = kShape == kTiny1;
  __shared__ float shared[Group<kWide>::kShared];
  extern __shared__ __attribute__((aligned(32))) float columns[];
  Group<kWide> g(p.lanes, shared);
  const Columns<kN, kTiny> at(g, p.dim);

  Row<kN> weight, next_weight, sums[2] = {};
  if (kAhead<kN>) fetch_vectors<T>(weight, next_weight, p, at);
  const uint64_t stride = (uint64_t)gridDim.x * p.slots, last = p.rows - 1u;
  uint64_t r = (uint64_t)blockIdx.x * p.slots + g.slot;
  Operands<R, T, kN> now{};
  auto get = [&](uint64_t r) {
    const uint64_t there = r < last ? r : last;
    fetch_row(now.y, (const T*)p.y + there * p.ld_y, at);
    if (p.gate && p.each) fetch_row(now.gate, (const T*)p.gate + there * p.ld_gate, at);
    if (p.gate && !p.each) now.only = ((const T*)p.gate)[there * p.ld_gate];
    if (p.then) {
      fetch_row(now.x, (const R*)p.x + there * p.ld_x, at);
      fetch_row(now.dnext, (const T*)p.dnext + there * p.ld_dnext, at);
    }
    if (p.dout) fetch_row(now.dout, (const R*)p.dout + there * p.ld_dout, at);
  };
  get(r);
  for (uint64_t r0 = (uint64_t)blockIdx.x * p.slots; r0 < p.rows; r0 += stride, r += stride) {
    const bool in = r < p.rows;
    if (!kAhead<kN>) fetch_vectors<T>(weight, next_weight, p, at);
    const Operands<R, T, kN> it = now;
    if (kAhead<kN>) get(r + stride);
    Row<kN> unit, gate, by, d;   // by: gate times weight and scale
    widen(unit, it.y);
    float inverse = 1.f;
    if (p.post) inverse = normalise(unit, g, at, p.layer, p.by);
    open(gate, it.gate, it.only, p);
    each<kN>([&](int j, uint32_t e) { by[j][e] = gate[j][e] * weight[j][e]; });
    if (p.dout) widen(d, it.dout);
    else each<kN>([&](int j, uint32_t e) { d[j][e] = 0.f; });
    if (p.then) {
      Row<kN> after, q;
      each<kN>([&](int j, uint32_t e) { after[j][e] = (float)it.x[j].v[e] + by[j][e] * unit[j][e]; });
      const float after_inverse = normalise(after, g, at, p.layer, p.by);
      widen(q, it.dnext);
      if (in) each<kN>([&](int j, uint32_t e) { sums[1][j][e] += q[j][e] * after[j][e]; });
      each<kN>([&](int j, uint32_t e) { q[j][e] *= next_weight[j][e]; });
      float none = 0.f;
      denormalise(q, after, after_inverse, g, at, p.layer, p.by, false, none);
      each<kN>([&](int j, uint32_t e) { d[j][e] += q[j][e]; });
    }
    if (p.dx) put_row((R*)p.dx + r * p.ld_dx, d, at, in);
    // from here on: the gradient of what was added to x, through the gate, the scale and the weight
    const bool one = p.dgate && !p.each;
    float all = 0.f;
    {
      Row<kN> through;
      each<kN>([&](int j, uint32_t e) { through[j][e] = d[j][e] * unit[j][e]; });
      if (in) each<kN>([&](int j, uint32_t e) { sums[0][j][e] += through[j][e] * gate[j][e]; });
      if (one) {
        all = at.sum([&](int j, uint32_t e) { return through[j][e] * weight[j][e]; });
      } else if (p.dgate) {
        if (p.sigmoid) each<kN>([&](int j, uint32_t e) { through[j][e] *= by[j][e] * (1.f - gate[j][e]); });
        else each<kN>([&](int j, uint32_t e) { through[j][e] *= weight[j][e]; });
        put_row((T*)p.dgate + r * p.ld_dgate, through, at, in);
      }
    }
    each<kN>([&](int j, uint32_t e) { d[j][e] *= by[j][e]; });
    if (p.post) {
      denormalise(d, unit, inverse, g, at, p.layer, p.by, one, all);
    } else if (one) {
      float s[1] = {all};
      g.sum(s);
      all = s[0];
    }
    if (p.dy) put_row((T*)p.dy + r * p.ld_dy, d, at, in);
    if (one && in && g.mine == 0u) ((T*)p.dgate)[r * p.ld_dgate] = (T)(p.sigmoid ? all * gate[0][kPack - 1] * (1.f - gate[0][kPack - 1]) : all);
    if (!kAhead<kN>) get(r + stride);
  }
  if (p.sums) leave_sums(sums, p.sums + (uint64_t)blockIdx.x * 2u * p.wide, p.wide, g, at, p.slots, columns);
}

// Adds up the workgroups' sums of columns, in their order, and makes gradients of them: of the first, times the scale, the
// weight's; times the weight, the scale's; of the second the next weight's.  3 to 5 us.
struct SumArgs {
  const float* sums;
  const void *weight, *scale;
  void *first, *second, *third;
  uint32_t dim, wide, rows, n_sums;
  uint32_t single, half;            // half: vectors that are not in 32 bits are in f16, not bf16
  float number;
};
constexpr uint32_t kStrips = 32, kAtOnce = 32;   // workgroups' sums that are read side by side, columns
__global__ __launch_bounds__(kAtOnce * kStrips) void k_sum_columns(SumArgs p) {
  __shared__ float shared[kStrips][kAtOnce];
  const uint32_t lane = threadIdx.x % kAtOnce, strip = threadIdx.x / kAtOnce, c = blockIdx.x * kAtOnce + lane, which = blockIdx.y;
  const uint32_t each = (p.rows + kStrips - 1u) / kStrips, from = strip * each, to = from + each < p.rows ? from + each : p.rows;
  float s = 0.f;
  if (c < p.dim) {
    const float* in = p.sums + which * p.wide + c;
    const uint64_t step = (uint64_t)p.n_sums * p.wide;
#pragma unroll 16
    for (uint32_t r = from; r < to; ++r) s += in[r * step];
  }
  shared[strip][lane] = s;
  __syncthreads();
  if (strip || c >= p.dim) return;
  s = 0.f;
#pragma unroll
  for (uint32_t i = 0; i < kStrips; ++i) s += shared[i][lane];
  auto get = [&](const void* v, float none) { return !v ? none : p.single ? ((const float*)v)[c] : p.half ? (float)((const _Float16*)v)[c] : (float)((const __bf16*)v)[c]; };
  auto set = [&](void* v, float x) {
    if (!v) return;
    if (p.single) ((float*)v)[c] = x;
    else if (p.half) ((_Float16*)v)[c] = (_Float16)x;
    else ((__bf16*)v)[c] = (__bf16)x;
  };
  if (which) {
    set(p.third, s);
  } else {
    set(p.first, s * get(p.scale, p.number));
    set(p.second, s * get(p.weight, 1.f));
  }
}

// How rows go to lanes: `packs` of a lane, lanes of a row, rows a workgroup holds at a time, workgroups.
constexpr uint64_t kMostBlocks = 1u << 20;   // (a launch's lanes are counted in 32 bits)
struct Layout {
  uint32_t packs, lanes, slots, blocks;
  uint32_t threads() const { return lanes * slots; }
};
Layout lay_out(uint64_t rows, uint32_t dim, bool backward) {
  Layout l;
  const uint32_t packs = (uint32_t)ceil_div(dim, kPack);
  l.packs = 1;
  while (packs > l.packs * kMostLanes) l.packs *= 2u;
  const uint32_t need = (uint32_t)ceil_div(packs, l.packs);
  l.lanes = 1;
  while (l.lanes < need && l.lanes < 64u) l.lanes *= 2u;
  if (need > 64u) l.lanes = (uint32_t)round_up(need, 64);
  const uint32_t target = backward ? 512 : 256;
  l.slots = l.lanes < target ? target / l.lanes : 1u;
  // A gradient's workgroups leave sums of columns behind, so there are few; the others take a row four times, in which the weights that
  // a lane holds serve again (65,536 x 2,624 in bf16, norm and join: 2,048 workgroups 135 and 483 us, 8,192 122 and 448, 16,384 118 and
  // 437, 65,536 140 and 541), or less often where that leaves fewer than 2,048.
  const uint64_t groups = ceil_div(rows, l.slots), fours = ceil_div(groups, 4), least = backward ? 512 : fours > 2048 ? fours : 2048;
  l.blocks = (uint32_t)(groups < least ? groups : least < kMostBlocks ? least : kMostBlocks);
  return l;
}

uint32_t wide_of(uint32_t dim) { return (uint32_t)round_up(dim, kPack); }

fbx_status check_types(fbx_dtype stream, fbx_dtype block, fbx_dtype vectors) {
  if (!known(stream) || !known(block) || !known(vectors)) return refuse(FBX_E_ARG, "unknown dtype");
  if (stream != block && stream != FBX_F32) return refuse(FBX_E_ARG, "the stream is of the block's type or f32");
  if (vectors != block && vectors != FBX_F32) return refuse(FBX_E_ARG, "vectors are of the block's type or f32");
  return FBX_OK;
}
fbx_status check_sizes(uint64_t records, uint32_t dim, fbx_norm_kind kind, double eps) {
  if (records >> 40) return refuse(FBX_E_ARG, "records must be below 2^40");
  if (!dim || dim > FBX_NORM_MOST) return refuse(FBX_E_ARG, "dim must be 1 .. FBX_NORM_MOST");
  if (kind != FBX_NORM_RMS && kind != FBX_NORM_LAYER) return refuse(FBX_E_ARG, "unknown kind");
  if (!((float)eps >= FLT_MIN && (float)eps <= FLT_MAX)) return refuse(FBX_E_ARG, "eps must be a positive number of 32 bits");
  return FBX_OK;
}
// A matrix of `columns` elements a row.
fbx_status check_matrix(const void* p, uint64_t ld, uint64_t columns, fbx_dtype t, uint64_t records, const char* null, const char* why) {
  if (!p && records) return refuse(FBX_E_ARG, null);
  if ((uintptr_t)p % size_of(t)) return refuse(FBX_E_ARG, "a matrix is not aligned to its elements");
  if (ld < columns || ld >> 40) return refuse(FBX_E_ARG, why);
  return FBX_OK;
}
fbx_status check_vectors(fbx_dtype t, uintptr_t all) {
  return all % size_of(t) ? refuse(FBX_E_ARG, "a vector is not aligned to its elements") : FBX_OK;
}
fbx_status check_scratch(const void* d_scratch, uint64_t bytes, uint64_t need) {
  if (need && (!d_scratch || (uintptr_t)d_scratch % 256u)) return refuse(FBX_E_ARG, "d_scratch is NULL or not 256-byte aligned");
  return bytes < need ? refuse(FBX_E_NOMEM, "scratch too small: the scratch function gives its size") : FBX_OK;
}

fbx_status check(const fbx_norm* h) {
  if (!h) return refuse(FBX_E_ARG, "h is NULL");
  fbx_status st = check_types(h->stream, h->block, h->vectors);
  if (st == FBX_OK) st = check_sizes(h->records, h->dim, h->kind, h->eps);
  return st;
}
fbx_status check(const fbx_join* h) {
  if (!h) return refuse(FBX_E_ARG, "h is NULL");
  fbx_status st = check_types(h->stream, h->block, h->vectors);
  if (st == FBX_OK) st = check_sizes(h->records, h->dim, h->kind, h->eps);
  if (st != FBX_OK) return st;
  if (h->gate_act != FBX_GATE_NONE && h->gate_act != FBX_GATE_SIGMOID) return refuse(FBX_E_ARG, "unknown gate_act");
  if (h->d_gate && h->gate_columns != 1 && h->gate_columns != h->dim) return refuse(FBX_E_ARG, "gate_columns must be 1 or dim");
  if (!h->post && h->d_weight) return refuse(FBX_E_ARG, "a weight is the norm's: none without post");
  if (!isfinite((float)h->scale)) return refuse(FBX_E_ARG, "scale must be a finite number of 32 bits");
  return FBX_OK;
}

template <template <class, class, Shape> class K, class A>
void launch(const A& p, const Layout& l, fbx_dtype stream, fbx_dtype block, uint32_t lds, hipStream_t on) {
  const dim3 grid(l.blocks), threads(l.threads());
  auto go = [&](auto shape) {
    constexpr Shape s = decltype(shape)::value;
    if (stream == FBX_F32 && block == FBX_F32) launch_on(on, K<float, float, s>::kernel, grid, threads, lds, p);
    else if (stream == FBX_F32 && block == FBX_F16) launch_on(on, K<float, _Float16, s>::kernel, grid, threads, lds, p);
    else if (stream == FBX_F32) launch_on(on, K<float, __bf16, s>::kernel, grid, threads, lds, p);
    else if (stream == FBX_F16) launch_on(on, K<_Float16, _Float16, s>::kernel, grid, threads, lds, p);
    else launch_on(on, K<__bf16, __bf16, s>::kernel, grid, threads, lds, p);
  };
  if (p.dim < kPack) go(std::integral_constant<Shape, kTiny1>());
  else if (l.lanes < 64u) go(std::integral_constant<Shape, kNarrow1>());
  else if (l.packs == 1u) go(std::integral_constant<Shape, kWide1>());
  else if (l.packs == 2u) go(std::integral_constant<Shape, kWide2>());
  else go(std::integral_constant<Shape, kWide4>());
}
template <class R, class T, Shape kShape> struct Norm { static constexpr auto kernel = k_norm<R, T, kShape>; };
template <class R, class T, Shape kShape> struct NormGrad { static constexpr auto kernel = k_norm_grad<R, T, kShape>; };
template <class R, class T, Shape kShape> struct Join { static constexpr auto kernel = k_join<R, T, kShape>; };
template <class R, class T, Shape kShape> struct JoinGrad { static constexpr auto kernel = k_join_grad<R, T, kShape>; };

void sum_columns(SumArgs& s, uint32_t dim, uint32_t blocks, uint32_t n_sums, fbx_dtype vectors, hipStream_t stream) {
  s.dim = dim;
  s.wide = wide_of(dim);
  s.rows = blocks;
  s.n_sums = n_sums;
  s.single = vectors == FBX_F32;
  s.half = vectors == FBX_F16;
  launch_on(stream, k_sum_columns, dim3((uint32_t)ceil_div(dim, kAtOnce), n_sums), dim3(kAtOnce * kStrips), 0, s);
}

NormArgs args_of(const fbx_norm* h, const Layout& l) {
  NormArgs p{};
  p.x = h->d_x;
  p.ld_x = h->ld_x;
  p.weight = h->d_weight;
  p.rows = h->records;
  p.dim = h->dim;
  p.wide = wide_of(h->dim);
  p.lanes = l.lanes;
  p.slots = l.slots;
  p.layer = h->kind == FBX_NORM_LAYER;
  p.single = h->vectors == FBX_F32;
  p.by = Scale{(float)h->dim, (float)(1.0 / h->dim), (float)h->eps};
  return p;
}
JoinArgs args_of(const fbx_join* h, const Layout& l) {
  JoinArgs p{};
  p.x = h->d_x;
  p.ld_x = h->ld_x;
  p.y = h->d_y;
  p.ld_y = h->ld_y;
  p.gate = h->d_gate;
  p.ld_gate = h->ld_gate;
  p.weight = h->d_weight;
  p.scale = h->d_scale;
  p.next_weight = h->d_next_weight;
  p.rows = h->records;
  p.dim = h->dim;
  p.wide = wide_of(h->dim);
  p.lanes = l.lanes;
  p.slots = l.slots;
  p.layer = h->kind == FBX_NORM_LAYER;
  p.single = h->vectors == FBX_F32;
  p.post = h->post != 0;
  p.each = h->gate_columns != 1;
  p.sigmoid = h->gate_act == FBX_GATE_SIGMOID;
  p.by = Scale{(float)h->dim, (float)(1.0 / h->dim), (float)h->eps};
  p.number = (float)h->scale;
  return p;
}
uint32_t lds_of(const Layout& l, uint32_t dim, uint32_t sums) {
  const uint32_t lines = l.lanes < 64u ? l.threads() / 64u : l.slots;
  return lines > 1u ? lines * wide_of(dim) * sums * 4u : 0u;
}
uint64_t sums_bytes(uint64_t records, uint32_t dim, uint32_t sums) { return round_up((uint64_t)lay_out(records, dim, true).blocks * wide_of(dim) * sums * 4u, 256); }

}  // namespace
}  // namespace train
}  // namespace fbx

using namespace fbx::train;

extern "C" fbx_status fbx_norm_forward(const fbx_norm* h, void* d_out, uint64_t ld_out, void* hip_stream) {
  fbx_status st = check(h);
  if (st == FBX_OK) st = check_matrix(h->d_x, h->ld_x, h->dim, h->stream, h->records, "d_x is NULL", "ld_x is smaller than dim, or 2^40 or more");
  if (st == FBX_OK) st = check_matrix(d_out, ld_out, h->dim, h->block, h->records, "d_out is NULL", "ld_out is smaller than dim, or 2^40 or more");
  if (st == FBX_OK) st = check_vectors(h->vectors, (uintptr_t)h->d_weight);
  if (st != FBX_OK || !h->records) return st;
  const Layout l = lay_out(h->records, h->dim, false);
  NormArgs p = args_of(h, l);
  p.out = d_out;
  p.ld_out = ld_out;
  launch<Norm>(p, l, h->stream, h->block, 0, (hipStream_t)hip_stream);
  return launched();
}

extern "C" fbx_status fbx_norm_scratch(const fbx_norm* h, uint64_t* bytes) {
  const fbx_status st = check(h);
  if (st != FBX_OK) return st;
  if (!bytes) return refuse(FBX_E_ARG, "bytes is NULL");
  *bytes = sums_bytes(h->records, h->dim, 1);
  return FBX_OK;
}

extern "C" fbx_status fbx_norm_backward(const fbx_norm* h, const void* d_dy, uint64_t ld_dy, void* d_dx, uint64_t ld_dx, void* d_dweight, void* d_scratch,
                                        uint64_t scratch_bytes, void* hip_stream) {
  fbx_status st = check(h);
  if (st == FBX_OK) st = check_matrix(h->d_x, h->ld_x, h->dim, h->stream, h->records, "d_x is NULL", "ld_x is smaller than dim, or 2^40 or more");
  if (st == FBX_OK) st = check_matrix(d_dy, ld_dy, h->dim, h->block, h->records, "d_dy is NULL", "ld_dy is smaller than dim, or 2^40 or more");
  if (st == FBX_OK && d_dx) st = check_matrix(d_dx, ld_dx, h->dim, h->stream, h->records, "", "ld_dx is smaller than dim, or 2^40 or more");
  if (st == FBX_OK) st = check_vectors(h->vectors, (uintptr_t)h->d_weight | (uintptr_t)d_dweight);
  if (st == FBX_OK && d_dweight) st = check_scratch(d_scratch, scratch_bytes, sums_bytes(h->records, h->dim, 1));
  if (st != FBX_OK) return st;
  if (!d_dx && !d_dweight) return FBX_OK;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const Layout l = lay_out(h->records, h->dim, true);
  if (h->records) {
    NormArgs p = args_of(h, l);
    p.dy = d_dy;
    p.ld_dy = ld_dy;
    p.dx = d_dx;
    p.ld_dx = ld_dx;
    p.sums = d_dweight ? (float*)d_scratch : nullptr;
    launch<NormGrad>(p, l, h->stream, h->block, lds_of(l, h->dim, 1), stream);
  }
  if (d_dweight) {
    SumArgs s{};
    s.sums = (const float*)d_scratch;
    s.first = d_dweight;
    s.number = 1.f;
    sum_columns(s, h->dim, l.blocks, 1, h->vectors, stream);
  }
  return launched();
}

extern "C" fbx_status fbx_join_forward(const fbx_join* h, void* d_out, uint64_t ld_out, void* d_next, uint64_t ld_next, void* hip_stream) {
  fbx_status st = check(h);
  if (st == FBX_OK) st = check_matrix(h->d_x, h->ld_x, h->dim, h->stream, h->records, "d_x is NULL", "ld_x is smaller than dim, or 2^40 or more");
  if (st == FBX_OK) st = check_matrix(h->d_y, h->ld_y, h->dim, h->block, h->records, "d_y is NULL", "ld_y is smaller than dim, or 2^40 or more");
  if (st == FBX_OK && h->d_gate) st = check_matrix(h->d_gate, h->ld_gate, h->gate_columns, h->block, h->records, "", "ld_gate is smaller than gate_columns, or 2^40 or more");
  if (st == FBX_OK) st = check_matrix(d_out, ld_out, h->dim, h->stream, h->records, "d_out is NULL", "ld_out is smaller than dim, or 2^40 or more");
  if (st == FBX_OK && d_next) st = check_matrix(d_next, ld_next, h->dim, h->block, h->records, "", "ld_next is smaller than dim, or 2^40 or more");
  if (st == FBX_OK) st = check_vectors(h->vectors, (uintptr_t)h->d_weight | (uintptr_t)h->d_scale | (uintptr_t)h->d_next_weight);
  if (st != FBX_OK || !h->records) return st;
  const Layout l = lay_out(h->records, h->dim, false);
  JoinArgs p = args_of(h, l);
  p.out = d_out;
  p.ld_out = ld_out;
  p.next = d_next;
  p.ld_next = ld_next;
  p.then = d_next != nullptr;
  launch<Join>(p, l, h->stream, h->block, 0, (hipStream_t)hip_stream);
  return launched();
}

extern "C" fbx_status fbx_join_scratch(const fbx_join* h, uint64_t* bytes) {
  const fbx_status st = check(h);
  if (st != FBX_OK) return st;
  if (!bytes) return refuse(FBX_E_ARG, "bytes is NULL");
  *bytes = sums_bytes(h->records, h->dim, 2);
  return FBX_OK;
}

extern "C" fbx_status fbx_join_backward(const fbx_join* h, const fbx_join_gradients* g, void* d_scratch, uint64_t scratch_bytes, void* hip_stream) {
  fbx_status st = check(h);
  if (st != FBX_OK) return st;
  if (!g) return refuse(FBX_E_ARG, "g is NULL");
  const uint64_t n = h->records;
  if (!g->d_dout && !g->d_dnext && n) return refuse(FBX_E_ARG, "d_dout and d_dnext are both NULL");
  const bool then = g->d_dnext != nullptr, sums = g->d_dweight || g->d_dscale || g->d_dnext_weight;
  st = check_matrix(h->d_y, h->ld_y, h->dim, h->block, n, "d_y is NULL", "ld_y is smaller than dim, or 2^40 or more");
  if (st == FBX_OK && then) st = check_matrix(h->d_x, h->ld_x, h->dim, h->stream, n, "d_x is NULL", "ld_x is smaller than dim, or 2^40 or more");
  if (st == FBX_OK && h->d_gate) st = check_matrix(h->d_gate, h->ld_gate, h->gate_columns, h->block, n, "", "ld_gate is smaller than gate_columns, or 2^40 or more");
  if (st == FBX_OK && g->d_dout) st = check_matrix(g->d_dout, g->ld_dout, h->dim, h->stream, n, "", "ld_dout is smaller than dim, or 2^40 or more");
  if (st == FBX_OK && then) st = check_matrix(g->d_dnext, g->ld_dnext, h->dim, h->block, n, "", "ld_dnext is smaller than dim, or 2^40 or more");
  if (st == FBX_OK && g->d_dx) st = check_matrix(g->d_dx, g->ld_dx, h->dim, h->stream, n, "", "ld_dx is smaller than dim, or 2^40 or more");
  if (st == FBX_OK && g->d_dy) st = check_matrix(g->d_dy, g->ld_dy, h->dim, h->block, n, "", "ld_dy is smaller than dim, or 2^40 or more");
  if (st == FBX_OK && g->d_dgate) {
    if (!h->d_gate) return refuse(FBX_E_ARG, "a gate's gradient without a gate");
    st = check_matrix(g->d_dgate, g->ld_dgate, h->gate_columns, h->block, n, "", "ld_dgate is smaller than gate_columns, or 2^40 or more");
  }
  if (st == FBX_OK)
    st = check_vectors(h->vectors, (uintptr_t)h->d_weight | (uintptr_t)h->d_scale | (uintptr_t)h->d_next_weight | (uintptr_t)g->d_dweight | (uintptr_t)g->d_dscale | (uintptr_t)g->d_dnext_weight);
  if (st == FBX_OK && sums) st = check_scratch(d_scratch, scratch_bytes, sums_bytes(n, h->dim, 2));
  if (st != FBX_OK) return st;
  if (!g->d_dx && !g->d_dy && !g->d_dgate && !sums) return FBX_OK;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const Layout l = lay_out(n, h->dim, true);
  if (n) {
    JoinArgs p = args_of(h, l);
    p.dout = g->d_dout;
    p.ld_dout = g->ld_dout;
    p.dnext = g->d_dnext;
    p.ld_dnext = g->ld_dnext;
    p.dx = g->d_dx;
    p.ld_dx = g->ld_dx;
    p.dy = g->d_dy;
    p.ld_dy = g->ld_dy;
    p.dgate = g->d_dgate;
    p.ld_dgate = g->ld_dgate;
    p.then = then;
    p.sums = sums ? (float*)d_scratch : nullptr;
    launch<JoinGrad>(p, l, h->stream, h->block, lds_of(l, h->dim, 2), stream);
  }
  if (sums) {
    SumArgs s{};
    s.sums = (const float*)d_scratch;
    s.weight = h->d_weight;
    s.scale = h->d_scale;
    s.number = (float)h->scale;
    s.first = g->d_dweight;
    s.second = g->d_dscale;
    s.third = g->d_dnext_weight;
    sum_columns(s, h->dim, l.blocks, 2, h->vectors, stream);
  }
  return launched();
}

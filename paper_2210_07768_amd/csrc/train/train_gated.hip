// The gated feed-forward block h = act(x Wg^T) * (x Wu^T) and its gradient.
#include "train_common.h"

namespace fbx {
namespace train {
namespace {

__device__ __forceinline__ float logistic(float a) { return 1.f / (1.f + expf(-a)); }
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
  if (kAct == FBX_ACT_GELU) return bell_below(a) + a * expf(-0.5f * a * a) * 0.39894228040143268f;
  if (kAct == FBX_ACT_RELU) return a > 0.f ? 1.f : 0.f;
  const float s = logistic(a);
  return s * (1.f - s);
}

enum Form { kForward, kSlopes, kPlain };

// A rows x depth times the transpose of B columns x depth, element (i, k) of A at a[i * a_row + k * a_step].
struct MmArgs {
  const void *a, *b, *b2;    // kForward, kSlopes: b, b2 the two weights; kPlain: b2 the matrix that depth goes on with
  uint64_t a_row, a_step, b_row, b_step, b2_row, b2_step;
  const void* dh;            // kSlopes
  void *c, *c2;              // kForward: h; kSlopes: da, du; kPlain: rows below split, and from it on
  uint64_t ld_dh, ld_c, ld_c2;
  uint64_t rows, columns, depth, depth2;  // (depth2: of b2)
  uint64_t split;
};

constexpr int kTile = 64, kDeep = 16;

template <class T, Form kForm, int kAct>
__global__ __launch_bounds__(256) void k_mm(MmArgs p) {
  constexpr int kCols = kForm == kPlain ? kTile : kTile / 2;
  __shared__ float a_lds[kDeep][kTile + 4], b_lds[kDeep][kTile + 4];
  const uint64_t i0 = (uint64_t)blockIdx.x * kTile, j0 = (uint64_t)blockIdx.y * kCols;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float sum[4][4] = {};
  const uint64_t depth = p.depth + p.depth2;
  for (uint64_t k0 = 0; k0 < depth; k0 += kDeep) {
    for (int e = threadIdx.x; e < kTile * kDeep; e += 256) {
      const int i = e / kDeep, k = e % kDeep;
      const uint64_t kk = k0 + k;
      float v = 0.f;
      if (i0 + i < p.rows && kk < depth) v = (float)((const T*)p.a)[(i0 + i) * p.a_row + kk * p.a_step];
      a_lds[k][i] = v;
      v = 0.f;
      if (kForm == kPlain) {
        if (j0 + i < p.columns && kk < depth)
          v = kk < p.depth ? (float)((const T*)p.b)[(j0 + i) * p.b_row + kk * p.b_step] : (float)((const T*)p.b2)[(j0 + i) * p.b2_row + (kk - p.depth) * p.b2_step];
      } else if (kk < depth && j0 + i % kCols < p.columns) {
        v = i < kCols ? (float)((const T*)p.b)[(j0 + i) * p.b_row + kk] : (float)((const T*)p.b2)[(j0 + i - kCols) * p.b2_row + kk];
      }
      b_lds[k][i] = v;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDeep; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)  // (columns tx, tx + 16 of each half)
          sum[i][j] += a_lds[k][ty * 4 + i] * b_lds[k][tx + 16 * j];
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i) {
    const uint64_t r = i0 + ty * 4 + i;
    if (r >= p.rows) break;
    if (kForm == kPlain) {
      T* c = r < p.split ? (T*)p.c + r * p.ld_c : (T*)p.c2 + (r - p.split) * p.ld_c2;
      for (int j = 0; j < 4; ++j)
        if (j0 + tx + 16 * j < p.columns) c[j0 + tx + 16 * j] = (T)sum[i][j];
    } else {
      for (int j = 0; j < 2; ++j) {
        const uint64_t at = j0 + tx + 16 * j;
        if (at >= p.columns) continue;
        const float g = sum[i][j], u = sum[i][j + 2];
        if (kForm == kForward) {
          ((T*)p.c)[r * p.ld_c + at] = (T)(act<kAct>(g) * u);
        } else {
          const float dh = (float)((const T*)p.dh)[r * p.ld_dh + at];
          ((T*)p.c)[r * p.ld_c + at] = (T)(dh * u * slope<kAct>(g));
          ((T*)p.c2)[r * p.ld_c2 + at] = (T)(dh * act<kAct>(g));
        }
      }
    }
  }
}

template <class T, Form kForm>
void launch(const MmArgs& p, fbx_act act, hipStream_t stream) {
  const dim3 grid((uint32_t)ceil_div(p.rows, kTile), (uint32_t)ceil_div(p.columns, kForm == kPlain ? kTile : kTile / 2));
  if (kForm == kPlain || act == FBX_ACT_SILU) hipLaunchKernelGGL((k_mm<T, kForm, FBX_ACT_SILU>), grid, dim3(256), 0, stream, p);
  else if (act == FBX_ACT_GELU) hipLaunchKernelGGL((k_mm<T, kForm, FBX_ACT_GELU>), grid, dim3(256), 0, stream, p);
  else if (act == FBX_ACT_RELU) hipLaunchKernelGGL((k_mm<T, kForm, FBX_ACT_RELU>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((k_mm<T, kForm, FBX_ACT_SIGMOID>), grid, dim3(256), 0, stream, p);
}

template <Form kForm>
void launch_by_type(const MmArgs& p, fbx_dtype t, fbx_act act, hipStream_t stream) {
  if (t == FBX_F32) launch<float, kForm>(p, act, stream);
  else if (t == FBX_F16) launch<_Float16, kForm>(p, act, stream);
  else launch<__bf16, kForm>(p, act, stream);
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
  *bytes = backward ? round_up(2ull * g->records * g->hidden * size_of(g->dtype), 256) : 0;
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
  MmArgs p{};
  p.a = g->d_x;
  p.a_row = g->ld_x;
  p.a_step = 1;
  p.b = g->d_w_gate;
  p.b_row = g->ld_w_gate;
  p.b2 = g->d_w_up;
  p.b2_row = g->ld_w_up;
  p.c = d_h;
  p.ld_c = ld_h;
  p.rows = g->records;
  p.columns = g->hidden;
  p.depth = g->inputs;
  launch_by_type<kForward>(p, g->dtype, g->act, (hipStream_t)hip_stream);
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
  const hipStream_t stream = (hipStream_t)hip_stream;
  const uint64_t n = g->hidden, wide = 2 * n;
  char* slopes = (char*)d_scratch;  // a row: da, then du
  MmArgs p{};
  p.a = g->d_x;
  p.a_row = g->ld_x;
  p.a_step = 1;
  p.b = g->d_w_gate;
  p.b_row = g->ld_w_gate;
  p.b2 = g->d_w_up;
  p.b2_row = g->ld_w_up;
  p.dh = d_dh;
  p.ld_dh = ld_dh;
  p.c = slopes;
  p.c2 = slopes + n * size_of(g->dtype);
  p.ld_c = p.ld_c2 = wide;
  p.rows = g->records;
  p.columns = n;
  p.depth = g->inputs;
  if (g->records && (d_dx || d_dw_gate)) launch_by_type<kSlopes>(p, g->dtype, g->act, stream);
  if (g->records && d_dx) {
    MmArgs q{};
    q.a = slopes;
    q.a_row = wide;
    q.a_step = 1;
    q.b = g->d_w_gate;
    q.b_row = 1;
    q.b_step = g->ld_w_gate;
    q.b2 = g->d_w_up;
    q.b2_row = 1;
    q.b2_step = g->ld_w_up;
    q.c = d_dx;
    q.ld_c = ld_dx;
    q.rows = q.split = g->records;
    q.columns = g->inputs;
    q.depth = q.depth2 = n;
    launch_by_type<kPlain>(q, g->dtype, g->act, stream);
  }
  if (d_dw_gate) {
    MmArgs q{};
    q.a = slopes;
    q.a_row = 1;
    q.a_step = wide;
    q.b = g->d_x;
    q.b_row = 1;
    q.b_step = g->ld_x;
    q.c = d_dw_gate;
    q.ld_c = ld_dw_gate;
    q.c2 = d_dw_up;
    q.ld_c2 = ld_dw_up;
    q.rows = wide;
    q.split = n;
    q.columns = g->inputs;
    q.depth = g->records;
    launch_by_type<kPlain>(q, g->dtype, g->act, stream);
  }
  return launched();
}

// An AdamW step over many tensors at once, states in 32 or in 8 bits.
#include "train_common.h"

#include <math.h>

namespace fbx {
namespace train {
namespace {

constexpr uint32_t kTensorsPerLaunch = 128;  // (10 KB of arguments)
constexpr uint32_t kEach = 8;                 // elements of a lane
constexpr uint32_t kBlock = 256 * kEach;      // elements of a workgroup
static_assert(FBX_ADAMW_MOST == most_blocks(256) * kBlock, "a tensor is within one launch");

struct AdamwArgs {
  fbx_adamw_tensor t[kTensorsPerLaunch];
  uint64_t key[kTensorsPerLaunch];            // of the tensor's random bits
  uint32_t first_block[kTensorsPerLaunch + 1];
  uint32_t n, least_root;                     // least_root: the least code of a sqrt(v) above 0
  float keep, step_size, beta1, beta2, one_beta1, one_beta2, root_scale, eps, grad_scale;
};

template <class T>
__device__ __forceinline__ void load(float (&to)[kEach], const T* from, uint32_t n, bool wide) {
  if (wide) {
    const Pack<T, 16 / sizeof(T)>* p = (const Pack<T, 16 / sizeof(T)>*)from;
    Pack<T, 16 / sizeof(T)> v[kEach * sizeof(T) / 16];
#pragma unroll
    for (uint32_t i = 0; i < kEach * sizeof(T) / 16; ++i) v[i] = p[i];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) to[i] = (float)v[i / (16 / sizeof(T))].v[i % (16 / sizeof(T))];
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) to[i] = i < n ? (float)from[i] : 0.f;
  }
}

template <class T>
__device__ __forceinline__ void store(T* to, const float (&from)[kEach], uint32_t n, bool wide) {
  if (wide) {
    Pack<T, 16 / sizeof(T)>* p = (Pack<T, 16 / sizeof(T)>*)to;
#pragma unroll
    for (uint32_t i = 0; i < kEach * sizeof(T) / 16; ++i) {
      Pack<T, 16 / sizeof(T)> v;
#pragma unroll
      for (uint32_t j = 0; j < 16 / sizeof(T); ++j) v.v[j] = (T)from[i * (16 / sizeof(T)) + j];
      p[i] = v;
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i)
      if (i < n) to[i] = (T)from[i];
  }
}

// Eight codes times their block's scale.
__device__ __forceinline__ void decode(float (&to)[kEach], const uint8_t* codes, uint8_t scale, uint32_t n, bool wide) {
  uint32_t w[2] = {0u, 0u};
  if (wide) {
    const Pack<uint32_t, 2> p = *(const Pack<uint32_t, 2>*)codes;
    w[0] = p.v[0];
    w[1] = p.v[1];
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i)
      if (i < n) w[i / 4] |= (uint32_t)codes[i] << (8 * (i % 4));
  }
  // 2^(scale - 127); 0 stands for 2^-127, 255 for NaN
  const float s = __uint_as_float(scale == 255u ? 0x7fc00000u : scale ? (uint32_t)scale << 23 : 0x00400000u);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
    to[4 * i] = lo[0] * s;
    to[4 * i + 1] = lo[1] * s;
    to[4 * i + 2] = hi[0] * s;
    to[4 * i + 3] = hi[1] * s;
  }
}

// Eight codes of a block of 32, which four neighbouring lanes hold, and its scale.  random16(i): 16 random bits; least: the
// code, 0 or 1, of what is above 0 and would be rounded to 0 (1 for sqrt(v): rounded independently of m, it could become 0
// beside an m that does not, and the next update be m / eps).
template <class Random>
__device__ __forceinline__ void encode(uint8_t* codes, uint8_t* scale, const float (&x)[kEach], uint32_t n, bool wide, uint32_t least, Random random16) {
  uint32_t top = 0u;  // (magnitudes compare as integers, NaN above infinity above the rest)
#pragma unroll
  for (uint32_t i = 0; i < kEach; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    if (i < n && b > top) top = b;
  }
#pragma unroll
  for (int d = 1; d < 4; d <<= 1) {
    const uint32_t other = __shfl_xor(top, d, 64);
    top = other > top ? other : top;
  }
  const uint32_t e = top >> 23;
  const uint32_t b = e == 255u ? 255u : e > 8u ? e - 7u : 1u;
  const float inverse = __uint_as_float((254u - (b > 247u ? 247u : b)) << 23);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (uint32_t i = 0; i < kEach; ++i) {
    const float y = x[i] * inverse, a = fabsf(y);
    const int ee0 = (int)(__float_as_uint(a) >> 23) - 127, ee = ee0 < -6 ? -6 : ee0;
    const float t = a * __uint_as_float((uint32_t)(130 - ee) << 23);  // in units of the code's last place
    const uint32_t q = (uint32_t)floorf(t + (float)random16(i) * (1.f / 65536.f));
    const uint32_t code = b == 255u ? 127u : q + ((uint32_t)(ee + 6) << 3) + (y < 0.f ? 128u : 0u);
    w[i / 4] |= (code == 0u && x[i] > 0.f ? least : code) << (8 * (i % 4));
  }
  if (wide) {
    *(Pack<uint32_t, 2>*)codes = Pack<uint32_t, 2>{{w[0], w[1]}};
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i)
      if (i < n) codes[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
  if (n && threadIdx.x % 4u == 0u) *scale = (uint8_t)b;
}

// A workgroup takes 2,048 elements of one tensor, a lane eight adjacent ones (so that four lanes hold a block of
// 8-bit states).  P, G, C: types of weights, gradients, copies; kEight: states in 8 bits.
// Bound by memory: 175 M weights in 32 bits with gradients and copies in 16 and states in 8 take 567 to 579 us, 16.1 bytes each at
// 4.87 to 4.97 TB/s, what a copy reaches; 48 tensors of 0.53 M elements in all, in 32 bits,
// 8 to 9.3 us, of which the kernel takes 6.5.
template <class P, class G, class C, bool kEight, bool kCopy>
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs) {
#pragma clang fp contract(off)
  const AdamwArgs& a = launch_args<AdamwArgs>();
  uint32_t lo = 0u, hi = a.n;  // the tensor whose blocks hold this one
  while (hi - lo > 1u) {
    const uint32_t mid = (lo + hi) / 2u;
    if (a.first_block[mid] <= blockIdx.x) lo = mid;
    else hi = mid;
  }
  const fbx_adamw_tensor& t = a.t[lo];
  const uint64_t at = (uint64_t)(blockIdx.x - a.first_block[lo]) * kBlock + threadIdx.x * kEach;
  const uint32_t n = at >= t.n ? 0u : t.n - at < kEach ? (uint32_t)(t.n - at) : kEach;
  if (!kEight && !n) return;
  const uintptr_t all = (uintptr_t)t.d_param | (uintptr_t)t.d_grad | (kEight ? 0u : (uintptr_t)t.d_m | (uintptr_t)t.d_v) | (kCopy ? (uintptr_t)t.d_copy : 0u);
  const bool wide = n == kEach && all % 16u == 0u && (!kEight || ((uintptr_t)t.d_m | (uintptr_t)t.d_v) % 8u == 0u);
  float p[kEach], g[kEach], m[kEach], v[kEach];
  load(p, (const P*)t.d_param + at, n, wide);
  load(g, (const G*)t.d_grad + at, n, wide);
  if (kEight) {
    decode(m, (const uint8_t*)t.d_m + at, n ? t.d_m_scale[at / 32u] : 0u, n, wide);
    decode(v, (const uint8_t*)t.d_v + at, n ? t.d_v_scale[at / 32u] : 0u, n, wide);
  } else {
    load(m, (const float*)t.d_m + at, n, wide);
    load(v, (const float*)t.d_v + at, n, wide);
  }
  float root[kEach];
#pragma unroll
  for (uint32_t i = 0; i < kEach; ++i) {
    const float gi = g[i] * a.grad_scale, vi = kEight ? v[i] * v[i] : v[i];
    m[i] = m[i] * a.beta1 + gi * a.one_beta1;
    v[i] = vi * a.beta2 + (gi * gi) * a.one_beta2;
    root[i] = __builtin_sqrtf(v[i]);
    p[i] = p[i] * a.keep - (m[i] / (root[i] * a.root_scale + a.eps)) * a.step_size;
  }
  store((P*)t.d_param + at, p, n, wide);
  if (kCopy) store((C*)t.d_copy + at, p, n, wide);
  if (kEight) {
    uint64_t bits[kEach / 2];
#pragma unroll
    for (uint32_t i = 0; i < kEach / 2; ++i) bits[i] = mix64(a.key[lo] + at / 2u + i);
    encode((uint8_t*)t.d_m + at, t.d_m_scale + at / 32u, m, n, wide, 0u, [&](uint32_t i) { return (uint32_t)(bits[i / 2] >> (32 * (i % 2))) & 0xffffu; });
    encode((uint8_t*)t.d_v + at, t.d_v_scale + at / 32u, root, n, wide, a.least_root, [&](uint32_t i) { return (uint32_t)(bits[i / 2] >> (32 * (i % 2) + 16)) & 0xffffu; });
  } else {
    store((float*)t.d_m + at, m, n, wide);
    store((float*)t.d_v + at, v, n, wide);
  }
}

template <class P, class G, class C, bool kCopy>
void launch(const AdamwArgs& a, bool eight, hipStream_t stream) {
  const dim3 grid(a.first_block[a.n]);
  if (eight) launch_on(stream, k_adamw<P, G, C, true, kCopy>, grid, dim3(256), 0, a);
  else launch_on(stream, k_adamw<P, G, C, false, kCopy>, grid, dim3(256), 0, a);
}

template <class P, class G>
void launch_by_copy(const AdamwArgs& a, const fbx_adamw& h, bool copy, hipStream_t stream) {
  if (!copy) launch<P, G, float, false>(a, h.state_bits != 32u, stream);
  else if (h.copy_dtype == FBX_F16) launch<P, G, _Float16, true>(a, h.state_bits != 32u, stream);
  else launch<P, G, __bf16, true>(a, h.state_bits != 32u, stream);
}

template <class P>
void launch_by_grad(const AdamwArgs& a, const fbx_adamw& h, bool copy, hipStream_t stream) {
  if (h.grad_dtype == FBX_F32) launch_by_copy<P, float>(a, h, copy, stream);
  else if (h.grad_dtype == FBX_F16) launch_by_copy<P, _Float16>(a, h, copy, stream);
  else launch_by_copy<P, __bf16>(a, h, copy, stream);
}

}  // namespace
}  // namespace train
}  // namespace fbx

using namespace fbx::train;

extern "C" fbx_status fbx_adamw_step(const fbx_adamw* h, const fbx_adamw_tensor* tensors, uint32_t n_tensors, void* hip_stream) {
  if (!h || (!tensors && n_tensors)) return refuse(FBX_E_ARG, "h or tensors is NULL");
  if (!known(h->param_dtype) || !known(h->grad_dtype)) return refuse(FBX_E_ARG, "unknown dtype");
  if (h->state_bits != 8u && h->state_bits != 32u && h->state_bits != (8u | FBX_ADAMW_KEEP_ROOTS))
    return refuse(FBX_E_ARG, "state_bits must be 8 (also with FBX_ADAMW_KEEP_ROOTS) or 32");
  if (!h->step) return refuse(FBX_E_ARG, "step counts from 1");
  if (!(h->beta1 >= 0 && h->beta1 < 1 && h->beta2 >= 0 && h->beta2 < 1)) return refuse(FBX_E_ARG, "beta1 and beta2 must be in [0, 1)");
  if (!(h->eps >= 0) || !isfinite(h->lr) || !isfinite(h->weight_decay) || isnan(h->grad_scale)) return refuse(FBX_E_ARG, "lr, eps, weight_decay or grad_scale is not a number that makes sense");
  const bool eight = h->state_bits != 32u;
  const uint32_t ps = size_of(h->param_dtype), gs = size_of(h->grad_dtype);
  bool copy = false, any = false;
  for (uint32_t i = 0; i < n_tensors; ++i) {
    const fbx_adamw_tensor& t = tensors[i];
    if (!t.n) continue;
    if (!t.d_param || !t.d_grad || !t.d_m || !t.d_v || (eight && (!t.d_m_scale || !t.d_v_scale))) return refuse(FBX_E_ARG, "a tensor lacks its weights, gradient or state");
    if (t.n > FBX_ADAMW_MOST) return refuse(FBX_E_ARG, "a tensor has more than 2^35 - 2048 elements");
    if ((uintptr_t)t.d_param % ps || (uintptr_t)t.d_grad % gs || (!eight && ((uintptr_t)t.d_m | (uintptr_t)t.d_v) % 4u)) return refuse(FBX_E_ARG, "a tensor is not aligned to its elements");
    if (t.d_copy && (h->copy_dtype == FBX_F32 || !known(h->copy_dtype) || h->param_dtype != FBX_F32 || (uintptr_t)t.d_copy % 2u))
      return refuse(FBX_E_ARG, "a copy is in f16 or bf16, of weights in f32");
    copy |= t.d_copy != nullptr;
    any = true;
  }
  if (!any) return FBX_OK;
  for (uint32_t i = 0; copy && i < n_tensors; ++i)
    if (tensors[i].n && !tensors[i].d_copy) return refuse(FBX_E_ARG, "either all tensors have a copy or none");
  AdamwArgs a{};
  a.least_root = h->state_bits & FBX_ADAMW_KEEP_ROOTS ? 1u : 0u;
  a.keep = (float)(1.0 - h->lr * h->weight_decay);
  a.step_size = (float)(h->lr / (1.0 - pow(h->beta1, (double)h->step)));
  a.beta1 = (float)h->beta1;
  a.beta2 = (float)h->beta2;
  a.one_beta1 = (float)(1.0 - h->beta1);
  a.one_beta2 = (float)(1.0 - h->beta2);
  a.root_scale = (float)(1.0 / sqrt(1.0 - pow(h->beta2, (double)h->step)));
  a.eps = (float)h->eps;
  a.grad_scale = (float)h->grad_scale;
  const uint64_t key = mix64(h->seed + h->step);
  const hipStream_t stream = (hipStream_t)hip_stream;
  auto flush = [&]() {
    if (!a.n) return;
    if (h->param_dtype == FBX_F32) launch_by_grad<float>(a, *h, copy, stream);
    else if (h->param_dtype == FBX_F16) launch_by_grad<_Float16>(a, *h, false, stream);
    else launch_by_grad<__bf16>(a, *h, false, stream);
    a.n = 0;
  };
  for (uint32_t i = 0; i < n_tensors; ++i) {
    if (!tensors[i].n) continue;
    const uint64_t blocks = ceil_div(tensors[i].n, kBlock);
    if (a.n == kTensorsPerLaunch || (a.n && a.first_block[a.n] + blocks > most_blocks(256))) flush();
    a.t[a.n] = tensors[i];
    a.key[a.n] = mix64(key + i);
    a.first_block[a.n + 1] = a.first_block[a.n] + (uint32_t)blocks;
    ++a.n;
  }
  flush();
  return launched();
}

// Tiles of a product's operands in LDS, and the matrix instructions that read them: what the products of the gated block and
// of the orthogonalised updates share.
#pragma once

#include "train_common.h"

namespace fbx {
namespace train {

typedef float f32x4 __attribute__((ext_vector_type(4)));

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

}  // namespace train
}  // namespace fbx

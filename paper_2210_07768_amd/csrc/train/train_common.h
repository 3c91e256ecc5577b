// What the trainer's operators share: element types, packs of adjacent elements, slots as kernels see
// them, and the thread's error text.  Nothing here is part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "fbx_train.h"

namespace fbx {
namespace train {

// Notes why a call fails and returns `s`.
fbx_status refuse(fbx_status s, const char* why);
// A call's launches: each by `launch_on`, which notes the thread's first that fails; then `launched` gives FBX_OK, or FBX_E_HIP
// with the text of that one's error.  Errors that others left with the runtime stay there for them.
void note(hipError_t e);
fbx_status launched();
template <class... P>
void launch_on(hipStream_t stream, void (*kernel)(P...), dim3 grid, dim3 block, uint32_t lds, const std::enable_if_t<true, P>&... args) {
  void* at[] = {const_cast<void*>(static_cast<const void*>(&args))...};
  note(hipLaunchKernel((const void*)kernel, grid, block, at, lds, stream));
}

inline uint32_t size_of(fbx_dtype t) { return t == FBX_F32 ? 4u : 2u; }
inline bool known(fbx_dtype t) { return t == FBX_F32 || t == FBX_F16 || t == FBX_BF16; }
inline uint64_t round_up(uint64_t x, uint64_t to) { return (x + to - 1) / to * to; }
inline uint64_t ceil_div(uint64_t x, uint64_t by) { return (x + by - 1) / by; }

// The most workgroups a launch can have along x: it counts their lanes in 32 bits.
constexpr uint64_t most_blocks(uint32_t lanes) { return 0xffffffffu / lanes; }

// N adjacent elements, moved by one load or store.
template <class T, int N>
struct alignas(sizeof(T) * N) Pack {
  T v[N];
};

// The mixer of the extraction path (SplitMix64's output function).
__host__ __device__ __forceinline__ uint64_t mix64(uint64_t x) {
  x = (x ^ (x >> 30)) * 0xbf58476d1ce4e5b9ull;
  x = (x ^ (x >> 27)) * 0x94d049bb133111ebull;
  return x ^ (x >> 31);
}

// floor(mix64(sign) * rows / 2^64), rows < 2^31
__device__ __forceinline__ uint32_t row_of(uint64_t sign, uint32_t rows) {
  const uint64_t x = mix64(sign);
  return (uint32_t)(((x >> 32) * rows + (((x & 0xffffffffull) * rows) >> 32)) >> 32);
}

// A launch's arguments where the launch left them: indexing them by lane makes no copy.  For kernels with one
// argument, a struct.
template <class A>
__device__ __forceinline__ const A& launch_args() {
  return *(const A*)__builtin_amdgcn_kernarg_segment_ptr();
}

// One slot of signs.
struct SlotRef {
  const uint64_t* values;
  const uint64_t* offsets;    // null: arity signs a record
  const uint64_t* tile_ends;  // null: record order
  uint64_t n_values;
  uint32_t arity;
  uint32_t base;              // gradient: signs of the slots before
};
constexpr uint32_t kSlotsPerLaunch = 192;  // (9 KB of arguments; a launch fewer saves more than their way costs)

// Where record r's signs lie: [begin, begin + count), never outside the slot's values.
__device__ __forceinline__ void signs_of(const SlotRef& s, uint64_t r, uint64_t n_records, uint32_t tile, uint64_t& begin, uint32_t& count) {
  uint64_t end;
  if (!s.offsets) {
    begin = r * s.arity;
    end = begin + s.arity;
  } else {
    begin = s.offsets[r];
    end = s.tile_ends && (r + 1) % tile == 0 && r + 1 != n_records ? s.tile_ends[r / tile] : s.offsets[r + 1];
  }
  if (end > s.n_values) end = s.n_values;
  count = end > begin ? (uint32_t)(end - begin) : 0u;
}

// Checks a list of slots; total: signs in all.
fbx_status check_slots(const fbx_slot_view* slots, uint32_t n_slots, uint64_t n_records, uint32_t tile, uint64_t* total);
SlotRef slot_ref(const fbx_slot_view& v, uint32_t base);

}  // namespace train
}  // namespace fbx

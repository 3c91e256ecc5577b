// Rows of a table pooled per (record, slot): the first step of a model that is fed with signs.
#include "train_common.h"

#include <stdio.h>

namespace fbx {
namespace train {

namespace {
thread_local char g_error[256];
thread_local hipError_t g_launch = hipSuccess;
}

fbx_status refuse(fbx_status s, const char* why) {
  snprintf(g_error, sizeof g_error, "%s", why);
  return s;
}

void note(hipError_t e) {
  if (e != hipSuccess && g_launch == hipSuccess) g_launch = e;
}

fbx_status launched() {
  const hipError_t e = g_launch;
  if (e == hipSuccess) return FBX_OK;
  g_launch = hipSuccess;
  (void)hipGetLastError();  // (it is reported here)
  return refuse(FBX_E_HIP, hipGetErrorString(e));
}

fbx_status check_slots(const fbx_slot_view* slots, uint32_t n_slots, uint64_t n_records, uint32_t tile, uint64_t* total) {
  if (!slots && n_slots) return refuse(FBX_E_ARG, "slots is NULL");
  if (n_records >> 32) return refuse(FBX_E_ARG, "n_records must be below 2^32");
  uint64_t sum = 0;
  for (uint32_t i = 0; i < n_slots; ++i) {
    const fbx_slot_view& s = slots[i];
    if (s.n_values && !s.values) return refuse(FBX_E_ARG, "a slot has n_values but no values");
    if (s.n_values >> 32) return refuse(FBX_E_ARG, "a slot has 2^32 values or more");
    if (s.fixed_arity ? s.n_values != n_records * s.fixed_arity : !s.offsets)
      return refuse(FBX_E_ARG, s.fixed_arity ? "a slot of fixed arity must have fixed_arity * n_records values" : "a slot without fixed arity needs offsets");
    if (!s.fixed_arity && s.tile_ends && !tile) return refuse(FBX_E_ARG, "a slot has tile_ends: arrival_tile_records is needed");
    if (!s.fixed_arity && !s.tile_ends && tile) return refuse(FBX_E_ARG, "arrival_tile_records is given: every list slot needs tile_ends");
    sum += s.n_values;
  }
  if (total) *total = sum;
  return FBX_OK;
}

SlotRef slot_ref(const fbx_slot_view& v, uint32_t base) {
  return SlotRef{v.values, v.fixed_arity ? nullptr : v.offsets, v.fixed_arity ? nullptr : v.tile_ends, v.n_values, v.fixed_arity, base};
}

namespace {

constexpr uint32_t kTileRecords = 16, kTileSlots = 64;  // of a workgroup

struct EmbedArgs {
  SlotRef slots[kSlotsPerLaunch];
  const void* table;
  void* out;                 // of the launch's first slot
  uint64_t first_record, n_records, table_stride, record_stride;  // first_record: of the launch; n_records: in all
  uint32_t n_slots, each, rows, dim, tile, lanes_log2, mean;  // each: slots of a workgroup
};

// A workgroup takes 16 records of up to 64 slots (fewer slots where there are few records: `each`, blockIdx.y).  Its lanes first find, records side by side (slot-major signs
// are read whole lines at a time), where each (record, slot)'s signs lie and the first one's row; then 2^lanes_log2
// lanes a (record, slot), slots side by side (a record's pooled rows are written whole lines at a time, past the caches,
// which the table needs), each lane N adjacent columns, add the rows up in the order of the signs, four of
// those behind the first on their way at once.
// What bounds it is lines of 128 bytes fetched for shorter rows, whatever the loads' cache policy: 65,536 records of 164 slots,
// rows of 32 bytes in a table of 320 MB: 296 us for 1.42 GB of such lines and 0.34 GB of results, 6.0 TB/s (a kernel that does
// nothing but fetch lines at random reaches 6.4).  In two launches, which took 317, other shapes took: 32 records a workgroup
// 403 us (fewer workgroups at a time for the second stage to overlap the first's waits), two (record, slot)s in hand 365, both
// 409; one sign behind the first at a time costs lists a third more.
constexpr uint32_t kSigns = 4;
template <class T, int N>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs) {
  const EmbedArgs& a = launch_args<EmbedArgs>();
  __shared__ uint64_t begin[kTileSlots * (kTileRecords + 1)];
  __shared__ uint32_t count[kTileSlots * (kTileRecords + 1)], first[kTileSlots * (kTileRecords + 1)];
  const uint64_t r0 = a.first_record + (uint64_t)blockIdx.x * kTileRecords;
  const uint32_t s0 = blockIdx.y * a.each, n_slots = a.n_slots - s0 < a.each ? a.n_slots - s0 : a.each;
  const SlotRef* slots = a.slots + s0;
  const uint32_t n = (uint32_t)(a.n_records - r0 < kTileRecords ? a.n_records - r0 : kTileRecords);
  for (uint32_t i = threadIdx.x; i < n_slots * kTileRecords; i += 256u) {
    const uint32_t s = i / kTileRecords, r = i % kTileRecords;
    if (r >= n) continue;
    uint64_t b;
    uint32_t c;
    signs_of(slots[s], r0 + r, a.n_records, a.tile, b, c);
    const uint32_t at = s * (kTileRecords + 1) + r;
    begin[at] = b;
    count[at] = c;
    first[at] = c ? row_of(slots[s].values[b], a.rows) : 0u;
  }
  __syncthreads();
  typedef Pack<T, N> P;
  const uint32_t lanes = 1u << a.lanes_log2, mine = threadIdx.x & (lanes - 1u), groups = 256u >> a.lanes_log2;
  const T* table = (const T*)a.table;
  T* out = (T*)a.out + r0 * a.record_stride + (uint64_t)s0 * a.dim;
  for (uint32_t i = threadIdx.x >> a.lanes_log2; i < n * n_slots; i += groups) {
    const uint32_t r = i / n_slots, s = i - r * n_slots, at = s * (kTileRecords + 1) + r, c = count[at];
    const uint64_t* signs = slots[s].values + begin[at];
    for (uint32_t col = mine * N; col < a.dim; col += lanes * N) {
      P p = {};
      if (c) p = *(const P*)(table + first[at] * a.table_stride + col);
      float sum[N];
#pragma unroll
      for (int j = 0; j < N; ++j) sum[j] = (float)p.v[j];
      for (uint32_t k = 1; k < c; k += kSigns) {
        uint64_t sign[kSigns];
#pragma unroll
        for (uint32_t e = 0; e < kSigns; ++e) sign[e] = k + e < c ? signs[k + e] : 0ull;
        P q[kSigns] = {};
#pragma unroll
        for (uint32_t e = 0; e < kSigns; ++e)
          if (k + e < c) q[e] = *(const P*)(table + row_of(sign[e], a.rows) * a.table_stride + col);
#pragma unroll
        for (uint32_t e = 0; e < kSigns; ++e)
          if (k + e < c)
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] += (float)q[e].v[j];
      }
      P o;
#pragma unroll
      for (int j = 0; j < N; ++j) o.v[j] = (T)(a.mean && c > 1u ? sum[j] / (float)c : sum[j]);
      P* to = (P*)(out + r * a.record_stride + (uint64_t)s * a.dim + col);
      if constexpr (sizeof(P) >= 4) {
        typedef uint32_t Words __attribute__((ext_vector_type(sizeof(P) / 4)));
        __builtin_nontemporal_store(__builtin_bit_cast(Words, o), (Words*)to);
      } else {
        *to = o;
      }
    }
  }
}

template <class T, int N>
void launch(const EmbedArgs& a, hipStream_t stream) {
  const uint64_t blocks = ceil_div(a.n_records - a.first_record, kTileRecords), most = most_blocks(256);
  launch_on(stream, k_embed<T, N>, dim3((uint32_t)(blocks < most ? blocks : most), (uint32_t)ceil_div(a.n_slots, a.each)), dim3(256), 0, a);
}

template <class T>
void launch_by_width(const EmbedArgs& a, uint32_t n, hipStream_t stream) {
  if (n == 8) {
    if constexpr (sizeof(T) == 2) launch<T, 8>(a, stream);
  } else if (n == 4) {
    launch<T, 4>(a, stream);
  } else if (n == 2) {
    launch<T, 2>(a, stream);
  } else {
    launch<T, 1>(a, stream);
  }
}

}  // namespace
}  // namespace train
}  // namespace fbx

using namespace fbx::train;

extern "C" const char* fbx_train_last_error(void) { return g_error; }

extern "C" fbx_status fbx_embed_forward(const fbx_slot_view* slots, uint32_t n_slots, uint64_t n_records, uint32_t arrival_tile_records,
                                        const void* d_table, uint64_t rows, uint32_t dim, uint64_t table_stride, fbx_dtype dtype, int mean,
                                        void* d_out, uint64_t record_stride, void* hip_stream) {
  if (!known(dtype)) return refuse(FBX_E_ARG, "unknown dtype");
  if (!rows || rows >> 31) return refuse(FBX_E_ARG, "rows must be 1 .. 2^31 - 1");
  if (!dim || dim > 65536u || table_stride < dim || table_stride >> 32) return refuse(FBX_E_ARG, "dim must be 1 .. 65536 and table_stride at least dim");
  if (record_stride < (uint64_t)n_slots * dim || record_stride >> 40) return refuse(FBX_E_ARG, "record_stride must be at least n_slots * dim");
  const fbx_status st = check_slots(slots, n_slots, n_records, arrival_tile_records, nullptr);
  if (st != FBX_OK) return st;
  if (!n_slots || !n_records) return FBX_OK;
  if (!d_table || !d_out) return refuse(FBX_E_ARG, "d_table or d_out is NULL");
  const uint32_t e = size_of(dtype);
  if (((uintptr_t)d_table | (uintptr_t)d_out) % e) return refuse(FBX_E_ARG, "d_table and d_out must be aligned to their elements");
  // the widest pack, up to 16 bytes, that every row on either side is a multiple of
  const uint64_t all = (uintptr_t)d_table | (uintptr_t)d_out | dim * e | table_stride * e | record_stride * e;
  uint32_t n = 16u / e;
  while (n > 1u && all % (n * e)) n /= 2u;
  EmbedArgs a{};
  a.table = d_table;
  a.n_records = n_records;
  a.table_stride = table_stride;
  a.record_stride = record_stride;
  a.rows = (uint32_t)rows;
  a.dim = dim;
  a.tile = arrival_tile_records;
  a.mean = mean != 0;
  while ((1u << a.lanes_log2) * n < dim && a.lanes_log2 < 6u) ++a.lanes_log2;
  for (uint32_t s0 = 0; s0 < n_slots; s0 += kSlotsPerLaunch) {
    a.n_slots = n_slots - s0 < kSlotsPerLaunch ? n_slots - s0 : kSlotsPerLaunch;
    // (two workgroups a compute unit, as long as each has four slots: 5 records of 137 slots 46 us with 64 slots each, 12 with four)
    a.each = kTileSlots;
    while (a.each > 4u && ceil_div(n_records, kTileRecords) * ceil_div(a.n_slots, a.each) < 512u) a.each /= 2u;
    for (uint32_t i = 0; i < a.n_slots; ++i) a.slots[i] = slot_ref(slots[s0 + i], 0u);
    a.out = (char*)d_out + (uint64_t)s0 * dim * e;
    const hipStream_t stream = (hipStream_t)hip_stream;
    for (a.first_record = 0; a.first_record < n_records; a.first_record += most_blocks(256) * kTileRecords) {
      if (dtype == FBX_F32) launch_by_width<float>(a, n, stream);
      else if (dtype == FBX_F16) launch_by_width<_Float16>(a, n, stream);
      else launch_by_width<__bf16>(a, n, stream);
    }
  }
  return launched();
}

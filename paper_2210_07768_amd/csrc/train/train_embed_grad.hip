// The gradient of pooled rows with respect to their table, without atomics on it: (row, where it came from) pairs
// are sorted by row, stably, and a row's terms are then neighbours.
#include "train_common.h"

namespace fbx {
namespace train {
namespace {

// Pairs of a lane when sorting; a workgroup has 256 lanes.  Sixteen put more pairs of one digit next to each other; four
// make a pass shorter where there are too few pairs to fill the card (98,000 pairs: 10.8 us a pass and 6.4).
constexpr uint32_t kManyItems = 16, kFewItems = 4, kFewPairs = 1u << 18;
constexpr uint32_t kRun = 8;  // sorted terms a group of lanes adds up, all on their way at once
constexpr uint32_t kNone = 0xffffffffu;

struct PairArgs {
  SlotRef slots[kSlotsPerLaunch];
  uint32_t* keys;
  uint32_t* from;   // record * all slots + slot
  float* share;     // 1 / signs of (record, slot), by the same number; null for sums
  uint64_t n_records;
  uint32_t n_slots, first_slot, all_slots, rows, tile;
};

// A workgroup 256 records of a slot: their signs' rows, and where each came from, at the signs' own positions.  A lane takes
// a record's signs where there is one a record, or where records need not follow each other (arrival order); else lanes
// take neighbouring signs and look up whose they are.  13.1 M signs: 56 us, their bytes and the pairs' at 3.8 TB/s.
// Signs that no record's list holds (before the first one's, behind the last one's) have their place among the pairs too: as
// terms from nowhere, which add zeros to the last row, so that sorting needs no key beyond the rows.
__global__ __launch_bounds__(256) void k_pairs(PairArgs) {
  const PairArgs& a = launch_args<PairArgs>();
  __shared__ uint32_t ends[256];  // of the records' signs, from the first record's first on
  const SlotRef& s = a.slots[blockIdx.y];
  const uint64_t r0 = (uint64_t)blockIdx.x * 256u, r = r0 + threadIdx.x;
  const uint32_t n = r0 >= a.n_records ? 0u : (uint32_t)(a.n_records - r0 < 256u ? a.n_records - r0 : 256u);
  const uint32_t first = (uint32_t)r0 * a.all_slots + a.first_slot + blockIdx.y;  // of the first record
  uint64_t b = 0;
  uint32_t c = 0;
  if (threadIdx.x < n) {
    signs_of(s, r, a.n_records, a.tile, b, c);
    if (a.share) a.share[first + threadIdx.x * a.all_slots] = c > 1u ? 1.f / (float)c : 1.f;
  }
  if (!s.offsets || s.tile_ends) {
    const uint32_t from = first + threadIdx.x * a.all_slots;
    for (uint32_t i = 0; i < c; ++i) {
      a.keys[s.base + b + i] = row_of(s.values[b + i], a.rows);
      a.from[s.base + b + i] = from;
    }
    return;
  }
  const uint64_t held = s.offsets[0] < s.n_values ? s.offsets[0] : s.n_values, held_end = s.offsets[a.n_records] < s.n_values ? s.offsets[a.n_records] : s.n_values;
  for (uint64_t i = r0 + threadIdx.x; i < held + (s.n_values - held_end); i += gridDim.x * 256ull) {
    const uint64_t at = s.base + (i < held ? i : held_end + (i - held));
    a.keys[at] = a.rows - 1u;
    a.from[at] = kNone;
  }
  if (!n) return;
  const uint64_t begin = s.offsets[r0];
  if (threadIdx.x < n) ends[threadIdx.x] = (uint32_t)(b + c - begin);
  __syncthreads();
  const uint32_t all = begin < s.n_values ? ends[n - 1u] : 0u;
  const uint64_t room = begin < s.n_values ? s.n_values - begin : 0u;
  for (uint32_t i = threadIdx.x; i < all && i < room; i += 256u) {
    uint32_t lo = 0, hi = n;  // the first record that ends behind sign i
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2u;
      if (ends[mid] > i) hi = mid;
      else lo = mid + 1u;
    }
    a.keys[s.base + begin + i] = row_of(s.values[begin + i], a.rows);
    a.from[s.base + begin + i] = first + lo * a.all_slots;
  }
}

// Workgroups go to the eight dies in turn; this gives each die a stretch of neighbouring tiles.
__device__ __forceinline__ uint32_t tile_here() {
  const uint32_t each = gridDim.x / 8u, more = gridDim.x % 8u, die = blockIdx.x % 8u;
  return die * each + (die < more ? die : more) + blockIdx.x / 8u;
}

// Per tile of pairs, how many have each value of the digit; counts lie digit by digit.  (A wavefront has counters of its
// own, and its lanes that have the first one's digit are counted at once: the most frequent rows are next to each other after
// the first pass.  13.1 M pairs, signs as frequent as 1 / rank: 16 us in every pass, against
// 25 and 29 in the second and third.)
template <uint32_t kBits, uint32_t kItems>
__global__ __launch_bounds__(256) void k_digit_counts(const uint32_t* keys, uint32_t n, uint32_t shift, uint32_t n_tiles, uint32_t* counts) {
  constexpr uint32_t kBins = 1u << kBits;
  __shared__ uint32_t h[4][kBins];
  for (uint32_t i = threadIdx.x; i < 4u * kBins; i += 256u) h[i / kBins][i % kBins] = 0u;
  __syncthreads();
  const uint32_t tile = tile_here();
  const uint64_t at = (uint64_t)tile * (256u * kItems);
  uint32_t k[kItems];
#pragma unroll
  for (uint32_t i = 0; i < kItems; ++i) k[i] = at + i * 256u + threadIdx.x < n ? keys[at + i * 256u + threadIdx.x] : 0u;
#pragma unroll
  for (uint32_t i = 0; i < kItems; ++i) {
    if (at + i * 256u + threadIdx.x >= n) break;
    const uint32_t d = (k[i] >> shift) % kBins, d0 = __builtin_amdgcn_readfirstlane(d);
    const uint64_t same = __ballot(d == d0);
    if (d != d0) atomicAdd(&h[threadIdx.x / 64u][d], 1u);
    else if (__popcll(same & ((1ull << (threadIdx.x % 64u)) - 1ull)) == 0) atomicAdd(&h[threadIdx.x / 64u][d], (uint32_t)__popcll(same));
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < kBins; d += 256u) counts[d * (uint64_t)n_tiles + tile] = h[0][d] + h[1][d] + h[2][d] + h[3][d];
}

// Inclusive sums over the workgroup's 256 lanes.
__device__ __forceinline__ uint32_t sums_256(uint32_t v, uint32_t* four) {
  for (uint32_t d = 1; d < 64u; d <<= 1) {
    const uint32_t t = __shfl_up(v, d, 64);
    if (threadIdx.x % 64u >= d) v += t;
  }
  __syncthreads();
  if (threadIdx.x % 64u == 63u) four[threadIdx.x / 64u] = v;
  __syncthreads();
  for (uint32_t w = 0; w < threadIdx.x / 64u; ++w) v += four[w];
  return v;
}

// A workgroup a digit: counts of its tiles become how many pairs of earlier tiles have the digit.
__global__ __launch_bounds__(256) void k_digit_sums(uint32_t* counts, uint32_t n_tiles, uint32_t* totals) {
  constexpr uint32_t kEach = 8;
  __shared__ uint32_t four[4];
  __shared__ uint32_t all;
  uint32_t* c = counts + blockIdx.x * (uint64_t)n_tiles;
  uint32_t before = 0u;
  for (uint32_t i0 = 0; i0 < n_tiles; i0 += 256u * kEach) {
    const uint32_t i = i0 + threadIdx.x * kEach;
    uint32_t v[kEach], mine = 0u;
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) v[e] = i + e < n_tiles ? c[i + e] : 0u;
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) mine += v[e];
    const uint32_t sum = sums_256(mine, four);
    uint32_t at = before + sum - mine;
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) {
      if (i + e < n_tiles) c[i + e] = at;
      at += v[e];
    }
    if (threadIdx.x == 255u) all = sum;
    __syncthreads();
    before += all;
  }
  if (threadIdx.x == 0u) totals[blockIdx.x] = before;
}

// Moves a tile's pairs to where their digit's pairs go, in order: ranks inside a wavefront by comparing digits over
// its lanes, then over wavefronts and digits by sums; the tile is put in order in LDS, so that pairs of one digit are
// written next to each other.  Neighbouring tiles, whose pairs of a digit are neighbours too, are one die's: its cache joins
// their parts of a line.  13.1 M pairs: 53 us, 4.0 TB/s of pairs read and written (62 with tiles dealt to the dies in turn; tiles of
// 8,192 pairs are no faster, nor is one array in LDS for keys and then for the others, which leaves room for more workgroups).
template <uint32_t kBits, uint32_t kItems>
__global__ __launch_bounds__(256) void k_move_pairs(const uint32_t* keys, const uint32_t* from, uint32_t n, uint32_t shift, uint32_t n_tiles,
                                                    const uint32_t* counts, const uint32_t* totals, uint32_t* keys_out, uint32_t* from_out) {
  constexpr uint32_t kBins = 1u << kBits, kMine = kBins / 256u;  // a lane's digits: kMine neighbours
  __shared__ uint32_t seen[4][kBins], to[kBins], begin[kBins], four[4];
  __shared__ uint32_t k_lds[(256u * kItems)], f_lds[(256u * kItems)];
  const uint32_t lane = threadIdx.x % 64u, wave = threadIdx.x / 64u;
  for (uint32_t i = threadIdx.x; i < 4u * kBins; i += 256u) seen[i / kBins][i % kBins] = 0u;
  __syncthreads();
  const uint32_t tile = tile_here();
  const uint64_t at = (uint64_t)tile * (256u * kItems) + wave * (kItems * 64u) + lane;
  uint32_t k[kItems], f[kItems], rank[kItems];
#pragma unroll
  for (uint32_t i = 0; i < kItems; ++i) {
    const bool in = at + i * 64u < n;
    k[i] = in ? keys[at + i * 64u] : 0u;
    f[i] = in ? from[at + i * 64u] : 0u;
  }
  const uint64_t below = (1ull << lane) - 1ull;
#pragma unroll
  for (uint32_t i = 0; i < kItems; ++i) {
    const bool in = at + i * 64u < n;
    const uint32_t d = (k[i] >> shift) % kBins;
    uint64_t same = __ballot(in);
#pragma unroll
    for (uint32_t b = 0; b < kBits; ++b) {
      const uint64_t set = __ballot((d >> b) & 1u);
      same &= (d >> b) & 1u ? set : ~set;
    }
    const uint32_t before = in ? seen[wave][d] : 0u;
    rank[i] = before + __popcll(same & below);
    if (in && (same & below) == 0ull) seen[wave][d] = before + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  uint32_t mine[kMine], total[kMine], sum = 0u, sum_all = 0u;
#pragma unroll
  for (uint32_t e = 0; e < kMine; ++e) {
    const uint32_t d = threadIdx.x * kMine + e;
    mine[e] = 0u;
    for (uint32_t w = 0; w < 4u; ++w) {
      const uint32_t c = seen[w][d];
      seen[w][d] = mine[e];
      mine[e] += c;
    }
    total[e] = totals[d];
    sum += mine[e];
    sum_all += total[e];
  }
  uint32_t first = sums_256(sum, four) - sum, first_all = sums_256(sum_all, four) - sum_all;
#pragma unroll
  for (uint32_t e = 0; e < kMine; ++e) {
    const uint32_t d = threadIdx.x * kMine + e;
    begin[d] = first;
    to[d] = first_all + counts[d * (uint64_t)n_tiles + tile];
    first += mine[e];
    first_all += total[e];
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < kItems; ++i)
    if (at + i * 64u < n) {
      const uint32_t d = (k[i] >> shift) % kBins, p = begin[d] + seen[wave][d] + rank[i];
      k_lds[p] = k[i];
      f_lds[p] = f[i];
    }
  __syncthreads();
  const uint64_t first_pair = (uint64_t)tile * (256u * kItems);
  const uint32_t here = n - first_pair < (256u * kItems) ? (uint32_t)(n - first_pair) : (256u * kItems);
  for (uint32_t i = threadIdx.x; i < here; i += 256u) {
    const uint32_t d = (k_lds[i] >> shift) % kBins, p = to[d] + i - begin[d];
    keys_out[p] = k_lds[i];
    from_out[p] = f_lds[i];
  }
}

// A few pairs in one launch: a wavefront, which holds all keys in its registers, counts for each of four pairs the keys below
// its own, and equal ones before it, and writes it to that place.  (4,096 pairs of 17 bits: 11 us against 21 us for two
// passes.)
constexpr uint32_t kRankPairs = 4096, kRankEach = 4;
__global__ __launch_bounds__(256) void k_rank_pairs(const uint32_t* keys, const uint32_t* from, uint32_t n, uint32_t* keys_out, uint32_t* from_out) {
  constexpr uint32_t kPacks = kRankPairs / 256u;  // of four keys, of a lane
  const uint32_t lane = threadIdx.x % 64u, i0 = (blockIdx.x * 4u + threadIdx.x / 64u) * kRankEach;
  uint32_t all[kPacks][4];
#pragma unroll
  for (uint32_t j = 0; j < kPacks; ++j) {
    const uint32_t at = (j * 64u + lane) * 4u;
    if (at + 4u <= n) {
      const Pack<uint32_t, 4> q = *(const Pack<uint32_t, 4>*)(keys + at);
#pragma unroll
      for (uint32_t e = 0; e < 4u; ++e) all[j][e] = q.v[e];
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 4u; ++e) all[j][e] = at + e < n ? keys[at + e] : kNone;  // (no key is as large)
    }
  }
#pragma unroll
  for (uint32_t h = 0; h < kRankEach; ++h) {
    const uint32_t i = i0 + h;
    if (i >= n) return;
    const uint32_t k = keys[i];
    uint32_t rank = 0u;
#pragma unroll
    for (uint32_t j = 0; j < kPacks; ++j)
#pragma unroll
      for (uint32_t e = 0; e < 4u; ++e) rank += all[j][e] < k || (all[j][e] == k && (j * 64u + lane) * 4u + e < i) ? 1u : 0u;
#pragma unroll
    for (uint32_t d = 1; d < 64u; d <<= 1) rank += __shfl_xor(rank, d, 64);
    if (lane == 0u) {
      keys_out[rank] = k;
      from_out[rank] = from[i];
    }
  }
}

template <uint32_t kBits, uint32_t kItems>
void sort_pass(uint32_t* const (&keys)[2], uint32_t* const (&from)[2], int side, uint32_t n, uint32_t shift, uint32_t n_tiles, uint32_t* counts, uint32_t* totals,
               hipStream_t stream) {
  launch_on(stream, k_digit_counts<kBits, kItems>, dim3(n_tiles), dim3(256), 0, keys[side], n, shift, n_tiles, counts);
  launch_on(stream, k_digit_sums, dim3(1u << kBits), dim3(256), 0, counts, n_tiles, totals);
  launch_on(stream, k_move_pairs<kBits, kItems>, dim3(n_tiles), dim3(256), 0, keys[side], from[side], n, shift, n_tiles, counts, totals, keys[side ^ 1], from[side ^ 1]);
}

// Rows of the table up to the one of sorted term at - 1: the first row that belongs to what begins at term `at`.
__device__ __forceinline__ uint32_t rows_before(const uint32_t* keys, uint32_t n, uint32_t rows, uint64_t at) {
  if (!at) return 0u;
  if (at >= n) return rows;
  const uint32_t k = keys[at - 1u];
  return k < rows ? k + 1u : rows;
}

struct SumArgs {
  const uint32_t* keys;       // ascending; kNone: no term
  const uint32_t* from;       // terms are rows of dout ...
  const float* share;
  const float* terms;         // ... or, later, sums of stretches
  const void* dout;
  void* dtable;
  uint32_t* part_keys;        // two a workgroup: a row that began before it, a row that goes on after it
  float* parts;
  uint64_t record_stride, table_stride;
  uint32_t n, n_from, all_slots, rows, dim, lanes_log2, first_block, dense;  // first_block: of the launch; dense: a record's rows of dout directly follow the last one's
  uint32_t near;              // a workgroup zeroes its stretch of the table if that is no longer; 0: all zeroed before
};

// The sorted terms of a workgroup: kRun for every group of 2^lanes_log2 lanes, each lane N adjacent columns (blockIdx.y: which
// stretch of them).  A group adds its terms up one after the other.  A row that begins and ends in a group is written to the
// table; one that goes on is taken up by the group it begins in, which adds the next groups' shares of it; what
// began before the workgroup or goes on after it is left to the next launch, which adds such sums up the same way (at most two a
// workgroup, so three launches do for 10^8 terms).  kFirst: terms are rows of dout.
// Bound by the rows of dout, which are fetched in lines of 128 bytes in the order of the keys: 13.1 M terms of 32 bytes are 13.7 M
// lines, 1.76 GB, of which a kernel that does nothing else fetches 6.4 TB/s, and their sums' rows: 349 us in all, whether four or six
// workgroups are on a compute unit, and whether a group has 8 or 16 terms (98,000 terms of 64 bytes: 41 us the whole gradient with 8,
// 43.5 with 16, 44 with 4).  Whatever the loads' cache policy, a line is fetched whole; passing the caches by costs 60 us.
template <class T, int N, bool kFirst>
__global__ __launch_bounds__(256) void k_sum_rows(SumArgs a) {
  constexpr uint32_t kPad = kRun + 1;  // (a group's terms begin in another bank than the next one's)
  extern __shared__ uint32_t lds[];
  const uint32_t lanes = 1u << a.lanes_log2, groups = 256u >> a.lanes_log2, mine = threadIdx.x & (lanes - 1u), group = threadIdx.x >> a.lanes_log2;
  const uint32_t columns = lanes * N;
  uint32_t* key_of = lds;                                        // groups * kPad, then the one before and the one after
  uint32_t* from_of = lds + groups * kPad + 2u;                  // groups * kPad
  uint32_t* open = from_of + (kFirst ? groups * kPad : 0u);      // a group's flags: 1 began before it, 2 goes on after it, 4 all of it is one row's
  float* heads = (float*)(open + groups);                        // groups x columns
  const uint32_t block = a.first_block + blockIdx.x;
  const uint64_t b0 = (uint64_t)block * groups * kRun;
  const uint32_t here = a.n - b0 < groups * kRun ? (uint32_t)(a.n - b0) : groups * kRun;
  for (uint32_t i = threadIdx.x; i < groups * kRun; i += 256u) {
    const uint32_t at = i / kRun * kPad + i % kRun;
    key_of[at] = i < here ? a.keys[b0 + i] : kNone;
    if (kFirst) from_of[at] = i < here ? a.from[b0 + i] : 0u;
  }
  const uint32_t begin = kFirst && a.near ? rows_before(a.keys, a.n, a.rows, b0) : 0u;
  const uint32_t end = kFirst && a.near ? rows_before(a.keys, a.n, a.rows, b0 + groups * kRun) : 0u;
  uint32_t* ends = key_of + groups * kPad;
  if (threadIdx.x == 0u) {
    ends[0] = b0 ? a.keys[b0 - 1u] : kNone;
    ends[1] = b0 + here < a.n ? a.keys[b0 + here] : kNone;
  }
  __syncthreads();
  const uint32_t* keys = key_of + group * kPad;
  const uint32_t before = group ? key_of[(group - 1u) * kPad + kRun - 1u] : ends[0], last = keys[kRun - 1u];
  const uint32_t after = group + 1u < groups ? key_of[(group + 1u) * kPad] : ends[1];
  const uint32_t col = blockIdx.y * columns + mine * N;
  const bool in = col < a.dim;
  float* head = heads + group * columns + mine * N;
  auto write = [&](uint32_t row, const float (&sum)[N]) {
    if (row >= a.rows || !in) return;
    Pack<T, N> p;
#pragma unroll
    for (int j = 0; j < N; ++j) p.v[j] = (T)sum[j];
    *(Pack<T, N>*)((T*)a.dtable + row * a.table_stride + col) = p;
  };

  float sum[N] = {};
  uint32_t key = keys[0];
  bool began = key == before && key != kNone;  // the row at hand began before this group
  const bool goes_on = last == after && last != kNone;
  Pack<T, N> p[kRun] = {};
  Pack<float, N> q[kRun] = {};
  float w[kRun] = {};
#pragma unroll
  for (uint32_t e = 0; e < kRun; ++e) {
    if (!in || keys[e] == kNone) continue;
    if (kFirst) {
      const uint32_t from = from_of[group * kPad + e];
      if (from >= a.n_from) continue;
      uint64_t at = (uint64_t)from * a.dim;
      if (!a.dense) {
        const uint32_t r = from / a.all_slots;
        at = r * a.record_stride + (uint64_t)(from - r * a.all_slots) * a.dim;
      }
      p[e] = *(const Pack<T, N>*)((const T*)a.dout + at + col);
      w[e] = a.share ? a.share[from] : 1.f;
    } else {
      q[e] = *(const Pack<float, N>*)(a.terms + (b0 + group * kRun + e) * a.dim + col);
    }
  }
  if (kFirst && a.near) {  // (the terms asked for just now are awaited here too)
    const Pack<T, N> zero{};
    if (end > begin && end - begin <= a.near && in)
      for (uint32_t row = begin + group; row < end; row += groups) *(Pack<T, N>*)((T*)a.dtable + row * a.table_stride + col) = zero;
    __syncthreads();
  }
#pragma unroll
  for (uint32_t e = 0; e < kRun; ++e) {
    const uint32_t k = keys[e];
    if (k != key) {
      if (began) {
#pragma unroll
        for (int j = 0; j < N; ++j) head[j] = sum[j];
      } else {
        write(key, sum);  // (kNone is no row)
      }
      began = false;
      key = k;
#pragma unroll
      for (int j = 0; j < N; ++j) sum[j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) sum[j] += kFirst ? (a.share ? (float)p[e].v[j] * w[e] : (float)p[e].v[j]) : q[e].v[j];
  }
  const bool whole = began && goes_on;
  if (began) {
#pragma unroll
    for (int j = 0; j < N; ++j) head[j] = sum[j];
  } else if (!goes_on) {
    write(key, sum);
  }
  if (mine == 0u) open[group] = (keys[0] == before && keys[0] != kNone ? 1u : 0u) | (goes_on ? 2u : 0u) | (whole ? 4u : 0u);
  __syncthreads();

  // Adds the heads from group g on to sum, up to the row's end; true: the row goes on after the workgroup.
  auto follow = [&](uint32_t g, float (&total)[N]) {
    for (; g < groups; ++g) {
      const float* more = heads + g * columns + mine * N;
#pragma unroll
      for (int j = 0; j < N; ++j) total[j] += more[j];
      if (!(open[g] & 4u)) return false;
    }
    return true;
  };
  auto leave = [&](uint32_t which, uint32_t row, const float (&total)[N]) {
    if (mine == 0u && blockIdx.y == 0u) a.part_keys[2u * block + which] = row;
    if (in)
#pragma unroll
      for (int j = 0; j < N; ++j) a.parts[(2ull * block + which) * a.dim + col + j] = total[j];
  };
  const float none[N] = {};
  if (group == 0u && a.part_keys) {
    if (open[0] & 1u) {  // (all of the workgroup one row's: a second sum, of nothing, keeps the row's sums neighbours)
      float total[N] = {};
      const uint32_t row = key_of[0];
      if (follow(0u, total)) leave(1u, row, none);
      leave(0u, row, total);
    } else if (mine == 0u && blockIdx.y == 0u) {
      a.part_keys[2u * block] = kNone;
    }
    if (!(open[groups - 1u] & 2u) && mine == 0u && blockIdx.y == 0u) a.part_keys[2u * block + 1u] = kNone;
  }
  if (goes_on && !whole) {
    if (follow(group + 1u, sum)) leave(1u, last, sum);
    else write(last, sum);
  }
}

template <class T, int N>
__global__ __launch_bounds__(256) void k_clear_rows(void* to, uint64_t rows, uint32_t dim, uint64_t stride) {
  const uint32_t packs = dim / N;
  const uint64_t all = rows * packs;
  const Pack<T, N> zero{};
  for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < all; i += (uint64_t)gridDim.x * 256u)
    *(Pack<T, N>*)((T*)to + i / packs * stride + i % packs * N) = zero;
}

// Zeroes what the workgroups of k_sum_rows leave: stretches of the table, between the last rows of two of them, of more
// than `near` rows.  All workgroups take a part of each.
template <class T, int N>
__global__ __launch_bounds__(1024) void k_clear_far(SumArgs a, uint32_t each) {  // each: terms of a workgroup there
  constexpr uint32_t kMine = 16;  // a lane's, which are looked at one by one only if they are far together
  __shared__ uint32_t far[1024 * kMine], n_far;
  const uint32_t packs = a.dim / N, blocks = (uint32_t)(((uint64_t)a.n + each - 1u) / each);
  const Pack<T, N> zero{};
  for (uint32_t b0 = 0; b0 < blocks; b0 += 1024u * kMine) {
    if (threadIdx.x == 0u) n_far = 0u;
    __syncthreads();
    const uint32_t b = b0 + threadIdx.x * kMine;
    const uint32_t first = rows_before(a.keys, a.n, a.rows, (uint64_t)b * each), last = rows_before(a.keys, a.n, a.rows, (uint64_t)(b + kMine) * each);
    if (b < blocks && last > first && last - first > a.near) {
      uint32_t begin = first;
      for (uint32_t e = 0; e < kMine && b + e < blocks; ++e) {
        const uint32_t end = rows_before(a.keys, a.n, a.rows, (uint64_t)(b + e + 1u) * each);
        if (end > begin && end - begin > a.near) far[atomicAdd(&n_far, 1u)] = b + e;
        begin = end;
      }
    }
    __syncthreads();
    for (uint32_t f = 0; f < n_far; ++f) {
      const uint32_t begin = rows_before(a.keys, a.n, a.rows, (uint64_t)far[f] * each), end = rows_before(a.keys, a.n, a.rows, (far[f] + 1ull) * each);
      const uint64_t all = (uint64_t)(end - begin) * packs;
      for (uint64_t i = (uint64_t)blockIdx.x * 1024u + threadIdx.x; i < all; i += (uint64_t)gridDim.x * 1024u)
        *(Pack<T, N>*)((T*)a.dtable + (begin + i / packs) * a.table_stride + i % packs * N) = zero;
    }
    __syncthreads();
  }
}

// Where things lie in the scratch.
struct Layout {
  uint64_t keys[2], from[2], counts, totals, share, part_keys[2], parts[2], bytes;
  uint32_t n, n_tiles, passes, bits, items;  // bits: of a pass's digit; items: pairs of a lane
};

// Lanes (a power of two) for a row's columns: as many as rows of whole 16 bytes take, whatever they are: in what order sums are
// formed is not to follow from where a tensor lies.
uint32_t lanes_of(uint32_t dim, uint32_t size) {
  uint32_t log2 = 0;
  while ((1u << log2) * (16u / size) < dim && log2 < 6u) ++log2;
  return log2;
}

bool lay_out(Layout& l, uint64_t total, uint64_t n_records, uint32_t n_slots, uint64_t rows, uint32_t dim, bool mean) {
  if (total >> 32 || n_records * n_slots > most_blocks(256) * 256) return false;  // (k_pairs has a lane for a record)
  l.n = (uint32_t)total;
  l.items = total <= kFewPairs ? kFewItems : kManyItems;
  l.n_tiles = (uint32_t)ceil_div(total, 256u * l.items);
  uint32_t bits = 1;
  while ((rows - 1) >> bits) ++bits;
  l.passes = (bits + 8u) / 9u;  // (digits of nine bits where they save a pass)
  l.bits = (bits + l.passes - 1u) / l.passes > 8u ? 9u : 8u;
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    const uint64_t was = at;
    at = round_up(at + bytes, 256);
    return was;
  };
  for (int i = 0; i < 2; ++i) l.keys[i] = take(4 * total);
  for (int i = 0; i < 2; ++i) l.from[i] = take(4 * total);
  l.counts = take(4ull * l.n_tiles << l.bits);
  l.totals = take(4ull << l.bits);
  l.share = take(mean ? 4 * n_records * n_slots : 0);
  // (as many workgroups as there are where each has the fewest terms: elements of 32 bits)
  const uint32_t groups = 256u >> lanes_of(dim, 4);
  uint64_t blocks = ceil_div(total, groups * kRun);
  for (int i = 0; i < 2; ++i) {
    l.part_keys[i] = take(4 * 2 * blocks);
    l.parts[i] = take(4ull * 2 * blocks * dim);
    blocks = ceil_div(2 * blocks, groups * kRun);
  }
  l.bytes = at;
  return true;
}

template <class T, int N>
void sum_rows(SumArgs a, const Layout& l, char* scratch, uint64_t rows, hipStream_t stream) {
  const uint32_t groups = 256u >> a.lanes_log2, columns = N << a.lanes_log2;
  // Rows without terms.  Where most rows have some, a workgroup zeroes its own stretch just before it writes its sums into it, while
  // its first terms are on their way (13.1 M terms, 10 M rows of 32 bytes: 640 us the whole gradient, against 700 with all rows
  // zeroed first; zeroed before the terms are asked for, the stretch's lines have left the cache when the sums come, which costs 20);
  // where few have, stretches are long and unlike, and where there are few pairs it makes no difference.
  if (a.n > kFewPairs && rows <= 2ull * a.n) {
    a.near = 32u * groups * kRun;
    // (each of its workgroups looks at the ends of all 16 stretches)
    launch_on(stream, k_clear_far<T, N>, dim3(64), dim3(1024), 0, a, groups * kRun);
  } else {
    const uint64_t packs = rows * (a.dim / N);
    const uint32_t clear = (uint32_t)(ceil_div(packs, 256) < 16384 ? ceil_div(packs, 256) : 16384);
    launch_on(stream, k_clear_rows<T, N>, dim3(clear), dim3(256), 0, a.dtable, rows, a.dim, a.table_stride);
  }
  int side = 0;
  for (bool first = true; a.n; first = false) {
    const uint64_t blocks = ceil_div(a.n, groups * kRun);
    const bool last = blocks == 1;
    a.part_keys = last ? nullptr : (uint32_t*)(scratch + l.part_keys[side]);
    a.parts = last ? nullptr : (float*)(scratch + l.parts[side]);
    const uint32_t lds = 4u * ((first ? 2u : 1u) * groups * (kRun + 1u) + 2u + groups + groups * columns);
    for (uint64_t b = 0; b < blocks; b += most_blocks(256)) {
      const dim3 grid((uint32_t)(blocks - b < most_blocks(256) ? blocks - b : most_blocks(256)), (uint32_t)ceil_div(a.dim, columns));
      a.first_block = (uint32_t)b;
      if (first) launch_on(stream, k_sum_rows<T, N, true>, grid, dim3(256), lds, a);
      else launch_on(stream, k_sum_rows<T, N, false>, grid, dim3(256), lds, a);
    }
    if (last) break;
    a.keys = a.part_keys;
    a.terms = a.parts;
    a.n = (uint32_t)(2 * blocks);
    side ^= 1;
  }
}

template <class T>
void sum_rows_by_width(const SumArgs& a, uint32_t n, const Layout& l, char* scratch, uint64_t rows, hipStream_t stream) {
  if (n == 8) {
    if constexpr (sizeof(T) == 2) sum_rows<T, 8>(a, l, scratch, rows, stream);
  } else if (n == 4) {
    sum_rows<T, 4>(a, l, scratch, rows, stream);
  } else if (n == 2) {
    sum_rows<T, 2>(a, l, scratch, rows, stream);
  } else {
    sum_rows<T, 1>(a, l, scratch, rows, stream);
  }
}

}  // namespace
}  // namespace train
}  // namespace fbx

using namespace fbx::train;

extern "C" fbx_status fbx_embed_backward_scratch(const fbx_slot_view* slots, uint32_t n_slots, uint64_t n_records, uint64_t rows, uint32_t dim,
                                                 int mean, uint64_t* bytes) {
  if (!bytes) return refuse(FBX_E_ARG, "bytes is NULL");
  if (!rows || rows >> 31 || !dim || dim > 65536u) return refuse(FBX_E_ARG, "rows must be 1 .. 2^31 - 1, dim 1 .. 65536");
  if ((!slots && n_slots) || n_records >> 32) return refuse(FBX_E_ARG, "slots is NULL, or n_records is 2^32 or more");
  uint64_t total = 0;
  for (uint32_t i = 0; i < n_slots; ++i) {
    if (slots[i].n_values >> 32) return refuse(FBX_E_ARG, "2^32 signs or more");
    total += slots[i].n_values;
  }
  Layout l;
  if (!lay_out(l, total, n_records, n_slots, rows, dim, mean != 0)) return refuse(FBX_E_ARG, "2^32 signs or more, or records * slots above 2^32 - 256");
  *bytes = l.bytes;
  return FBX_OK;
}

extern "C" fbx_status fbx_embed_backward(const fbx_slot_view* slots, uint32_t n_slots, uint64_t n_records, uint32_t arrival_tile_records,
                                         const void* d_dout, uint64_t record_stride, uint64_t rows, uint32_t dim, uint64_t table_stride,
                                         fbx_dtype dtype, int mean, void* d_dtable, void* d_scratch, uint64_t scratch_bytes, void* hip_stream) {
  if (!known(dtype)) return refuse(FBX_E_ARG, "unknown dtype");
  if (!rows || rows >> 31) return refuse(FBX_E_ARG, "rows must be 1 .. 2^31 - 1");
  if (!dim || dim > 65536u || table_stride < dim || table_stride >> 32) return refuse(FBX_E_ARG, "dim must be 1 .. 65536 and table_stride at least dim");
  if (record_stride < (uint64_t)n_slots * dim || record_stride >> 40) return refuse(FBX_E_ARG, "record_stride must be at least n_slots * dim");
  uint64_t total = 0;
  const fbx_status st = check_slots(slots, n_slots, n_records, arrival_tile_records, &total);
  if (st != FBX_OK) return st;
  Layout l;
  if (!lay_out(l, total, n_records, n_slots, rows, dim, mean != 0)) return refuse(FBX_E_ARG, "2^32 signs or more, or records * slots above 2^32 - 256");
  if (!d_dtable || (!d_dout && total && n_records)) return refuse(FBX_E_ARG, "d_dtable or d_dout is NULL");
  const uint32_t e = size_of(dtype);
  if (((uintptr_t)d_dtable | (uintptr_t)d_dout) % e) return refuse(FBX_E_ARG, "d_dtable and d_dout must be aligned to their elements");
  if (l.bytes && (!d_scratch || (uintptr_t)d_scratch % 256u)) return refuse(FBX_E_ARG, "d_scratch is NULL or not 256-byte aligned");
  if (scratch_bytes < l.bytes) return refuse(FBX_E_NOMEM, "scratch too small: fbx_embed_backward_scratch gives its size");
  const hipStream_t stream = (hipStream_t)hip_stream;
  char* scratch = (char*)d_scratch;
  uint32_t* keys[2] = {(uint32_t*)(scratch + l.keys[0]), (uint32_t*)(scratch + l.keys[1])};
  uint32_t* from[2] = {(uint32_t*)(scratch + l.from[0]), (uint32_t*)(scratch + l.from[1])};
  uint32_t* counts = (uint32_t*)(scratch + l.counts);
  uint32_t* totals = (uint32_t*)(scratch + l.totals);
  float* share = mean ? (float*)(scratch + l.share) : nullptr;
  int side = 0;
  if (l.n) {
    PairArgs p{};
    p.keys = keys[0];
    p.from = from[0];
    p.share = share;
    p.n_records = n_records;
    p.all_slots = n_slots;
    p.rows = (uint32_t)rows;
    p.tile = arrival_tile_records;
    uint64_t longest = 0;  // list
    for (uint32_t i = 0; i < n_slots; ++i)
      if (!slots[i].fixed_arity && slots[i].n_values > longest) longest = slots[i].n_values;
    // (workgroups beyond those the records need, for signs that no record holds: none where a record has 16 signs or fewer)
    const uint64_t blocks = ceil_div(n_records, 256), more = ceil_div(longest, 4096) < 1024 ? ceil_div(longest, 4096) : 1024;
    uint32_t base = 0;
    for (uint32_t s0 = 0; s0 < n_slots; s0 += kSlotsPerLaunch) {
      p.first_slot = s0;
      p.n_slots = n_slots - s0 < kSlotsPerLaunch ? n_slots - s0 : kSlotsPerLaunch;
      for (uint32_t i = 0; i < p.n_slots; ++i) {
        p.slots[i] = slot_ref(slots[s0 + i], base);
        base += (uint32_t)slots[s0 + i].n_values;
      }
      launch_on(stream, k_pairs, dim3((uint32_t)(blocks > more ? blocks : more), p.n_slots), dim3(256), 0, p);
    }
    if (l.n <= kRankPairs) {
      launch_on(stream, k_rank_pairs, dim3((uint32_t)ceil_div(l.n, 4 * kRankEach)), dim3(256), 0, keys[0], from[0], l.n, keys[1], from[1]);
      side = 1;
    }
    for (uint32_t pass = 0; l.n > kRankPairs && pass < l.passes; ++pass, side ^= 1) {
      const auto sort = l.bits == 9u ? (l.items == kFewItems ? sort_pass<9, kFewItems> : sort_pass<9, kManyItems>)
                                     : (l.items == kFewItems ? sort_pass<8, kFewItems> : sort_pass<8, kManyItems>);
      sort(keys, from, side, l.n, l.bits * pass, l.n_tiles, counts, totals, stream);
    }
  }
  const uint64_t all = (uintptr_t)d_dout | (uintptr_t)d_dtable | dim * e | table_stride * e | record_stride * e;
  uint32_t n = 16u / e;
  while (n > 1u && all % (n * e)) n /= 2u;
  SumArgs a{};
  a.keys = keys[side];
  a.from = from[side];
  a.share = share;
  a.dout = d_dout;
  a.dtable = d_dtable;
  a.record_stride = record_stride;
  a.table_stride = table_stride;
  a.n = l.n;
  a.n_from = (uint32_t)(n_records * n_slots);
  a.dense = record_stride == (uint64_t)n_slots * dim;
  a.all_slots = n_slots;
  a.rows = (uint32_t)rows;
  a.dim = dim;
  a.lanes_log2 = lanes_of(dim, e);
  if (dtype == FBX_F32) sum_rows_by_width<float>(a, n, l, scratch, rows, stream);
  else if (dtype == FBX_F16) sum_rows_by_width<_Float16>(a, n, l, scratch, rows, stream);
  else sum_rows_by_width<__bf16>(a, n, l, scratch, rows, stream);
  return launched();
}

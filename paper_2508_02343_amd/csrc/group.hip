// Rows (slots) ordered by expert: a stable counting sort on the device, so that
// routing never waits for the host.
//
// c_e = number of slots of expert e; its rows start at 32 * sum over e' < e of
// ceil(c_e' / 32), in ascending slot order.  Latency-bound: 4 bytes in and about
// 4 out per slot.  Every wavefront takes a run of consecutive slots, 64 at a
// time.  A lane's rank among the 64 is the number of lower lanes with its expert:
// one ballot per bit of the expert number gives every lane the mask of its equals,
// so the order never depends on timing (atomics only add up counts).  The
// counts per wavefront and expert sit in LDS; their sums over the wavefronts in
// front and the padded starts give every wavefront its first row of each expert.
// More than kGroupChunk slots: a first launch leaves each workgroup's counts, the
// second places.
//
// Measured (us, as graph replays): 16 slots of 8 experts 5.5, 65536 of 128 9.8 (two
// launches; 0.06 TB/s of ids and rows).  What it takes is its chain of steps: the
// ids' load, a ballot per bit, four barriers, the stores.  With 4096 slots per
// workgroup and the ids read twice instead of kept with their ranks, 21.5 (then 11.7).
#include "grouped.hpp"

namespace mm {
namespace {

constexpr int kThreads = kGroupThreads, kWaves = kThreads / 64;

// Lanes whose key (below 2^bits) equals this lane's.
__device__ __forceinline__ uint64_t equals(int key, int bits) {
  uint64_t m = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const bool set = (key >> b) & 1;
    const uint64_t v = __ballot(set);
    m &= set ? v : ~v;
  }
  return m;
}

// An id as a key: ids outside [0, experts) become `experts`.
__device__ __forceinline__ int key_of(const GroupArgs& a, int64_t slot) {
  const int id = slot < a.rows ? a.ids[slot] : -1;
  return (unsigned)id < (unsigned)a.experts ? id : a.experts;
}

// Turns of a wavefront that fit in registers.
constexpr int kTurns = (int)(kGroupChunk / kThreads);

// Inclusive sum over the workgroup's threads of each of N values.
template <int N>
__device__ __forceinline__ void scan(int (&v)[N], int (*part)[N], int lane, int wave) {
#pragma unroll
  for (int k = 0; k < N; ++k)
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(v[k], d);
      if (lane >= d) v[k] += o;
    }
  if (lane == 63)
#pragma unroll
    for (int k = 0; k < N; ++k) part[wave][k] = v[k];
  __syncthreads();
  for (int w = 0; w < wave; ++w)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += part[w][k];
}

}  // namespace

// Each workgroup's slots per expert.
__global__ __launch_bounds__(kThreads) void group_count_kernel(GroupArgs a) {
  extern __shared__ uint32_t lds[];  // [experts]
  const int E = a.experts;
  if ((int)threadIdx.x < E) lds[threadIdx.x] = 0;
  __syncthreads();
  const int64_t s0 = (int64_t)blockIdx.x * kThreads * a.turns + threadIdx.x;
  for (int t = 0; t < a.turns; ++t) {
    const int key = key_of(a, s0 + (int64_t)t * kThreads);
    if (key < E) atomicAdd(&lds[key], 1u);  // (a count: the order does not matter)
  }
  __syncthreads();
  if ((int)threadIdx.x < E) a.counts[(int64_t)blockIdx.x * E + threadIdx.x] = (int32_t)lds[threadIdx.x];
}

// Places the slots; the rows, owners and tiles that no slot fills are shared out
// over the workgroups.
__global__ __launch_bounds__(kThreads) void group_place_kernel(GroupArgs a, int bits) {
  extern __shared__ uint32_t lds[];
  const int E = a.experts;
  uint32_t* const next = lds;                            // [kWaves][E]
  int* const total = (int*)(lds + kWaves * E);           // [E] slots of each expert
  int* const front = total + E;                          // [E] those of the workgroups in front
  int* const start = front + E;                          // [E] first row group
  int* const tile0 = start + E;                          // [2][E] first tile of 128 and of 256 rows
  int (*const part)[kTileLists] = (int (*)[kTileLists])(tile0 + 2 * E);  // [kWaves]
  __shared__ int ends[kTileLists];  // tiles in all
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t run = ((int64_t)blockIdx.x * kWaves + wave) * 64 * a.turns;
  int key[kTurns], rank[kTurns];
  const bool kept = a.turns <= kTurns;
  if (kept)
#pragma unroll
    for (int t = 0; t < kTurns; ++t) key[t] = t < a.turns ? key_of(a, run + 64 * t + lane) : E;
  for (int i = threadIdx.x; i < (kWaves + 2) * E; i += kThreads) next[i] = 0;  // (total and front with them)
  __syncthreads();
  uint32_t* const mine = next + wave * E;
  if (a.blocks > 1) {
    // every workgroup's counts, in slices of workgroups, several threads to an expert
    const int slices = kThreads / E, e = threadIdx.x % E, j = threadIdx.x / E;
    if (j < slices) {
      int before = 0, all = 0;
#pragma unroll 8
      for (int b = j; b < a.blocks; b += slices) {
        const int n = a.counts[(int64_t)b * E + e];
        before += b < (int)blockIdx.x ? n : 0;
        all += n;
      }
      atomicAdd(&total[e], all);
      atomicAdd(&front[e], before);
    }
  }
  // this wavefront's slots of each expert, and a slot's rank among them
  if (kept) {
#pragma unroll
    for (int t = 0; t < kTurns; ++t)
      if (t < a.turns) {  // uniform
        const uint64_t m = equals(key[t], bits);
        const int lower = __popcll(m & ((1ull << lane) - 1));
        rank[t] = key[t] < E ? (int)mine[key[t]] + lower : 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (key[t] < E && lower == 0) mine[key[t]] += (uint32_t)__popcll(m);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
  } else {
    for (int t = 0; t < a.turns; ++t) {
      const int k = key_of(a, run + 64 * (int64_t)t + lane);
      if (k < E) atomicAdd(&mine[k], 1u);
    }
  }
  __syncthreads();
  const int e = threadIdx.x;  // kThreads >= kMaxExperts
  int here = 0, before = 0, all = 0;
  if (e < E) {
    for (int w = 0; w < kWaves; ++w) {
      const int n = (int)next[w * E + e];
      next[w * E + e] = (uint32_t)here;
      here += n;
    }
    before = front[e];
    all = a.blocks > 1 ? total[e] : here;
  }
  int v[kTileLists];
#pragma unroll
  for (int k = 0; k < kTileLists; ++k) v[k] = (all + kTileRows[k] - 1) / kTileRows[k];
  const int own[kTileLists] = {v[0], v[1], v[2]};
  scan<kTileLists>(v, part, lane, wave);
  if (threadIdx.x == kThreads - 1)
#pragma unroll
    for (int k = 0; k < kTileLists; ++k) ends[k] = v[k];
  if (e < E) {
    const int s = v[0] - own[0];
    start[e] = s;
    total[e] = all;
#pragma unroll
    for (int k = 1; k < kTileLists; ++k) tile0[(k - 1) * E + e] = v[k] - own[k];
    if (blockIdx.x == 0) a.starts[e] = s * kRowGroup;
    for (int w = 0; w < kWaves; ++w) next[w * E + e] += (uint32_t)(s * kRowGroup + before);
  }
  __syncthreads();
  const int used = ends[0];  // row groups
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.starts[E] = used * kRowGroup;
#pragma unroll
    for (int k = 0; k < kTileLists; ++k) a.tile_counts[k] = ends[k];
  }
  // the slots, in their order
  if (kept) {
#pragma unroll
    for (int t = 0; t < kTurns; ++t)
      if (key[t] < E) a.slots[mine[key[t]] + rank[t]] = (int32_t)(run + 64 * t + lane);
  } else {
    for (int t = 0; t < a.turns; ++t) {
      const int64_t slot = run + 64 * (int64_t)t + lane;
      const int k = key_of(a, slot);
      const uint64_t m = equals(k, bits);
      const int lower = __popcll(m & ((1ull << lane) - 1));
      if (k < E) a.slots[mine[k] + lower] = (int32_t)slot;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (k < E && lower == 0) mine[k] += (uint32_t)__popcll(m);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
  // the row groups: owner, rows without a slot, tiles
  const int at = blockIdx.x * kThreads + threadIdx.x, stride = a.blocks * kThreads;
  for (int q = at; q < a.groups; q += stride) {
    int owner = -1, filled = 0;
    if (q < used) {
      int lo = 0, hi = E;  // the last expert whose first group is at or below q (later ones there have no rows)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= q) lo = mid;
        else hi = mid;
      }
      owner = lo;
      const int rel = q - start[lo], rest = total[lo] - rel * kRowGroup;
      filled = rest < kRowGroup ? rest : kRowGroup;
#pragma unroll
      for (int k = 0; k < kTileLists; ++k) {
        const int rows = kTileRows[k], per = rows / kRowGroup;
        if (rel % per == 0)
          a.tiles[k][k == 0 ? q : tile0[(k - 1) * E + lo] + rel / per] =
              RowTile{q, (uint32_t)owner | (uint32_t)(rest < rows ? rest : rows) << 16};
      }
    }
    a.owners[q] = owner;
    for (int r = filled; r < kRowGroup; ++r) a.slots[(int64_t)q * kRowGroup + r] = -1;
  }
  // places behind the last tile
#pragma unroll
  for (int k = 0; k < kTileLists; ++k)
    for (int i = ends[k] + at; i < a.ntiles[k]; i += stride) a.tiles[k][i] = RowTile{-1, 0};
}

hipError_t launch_group_rows(const GroupArgs& a, const Device& dev, hipStream_t stream) {
  int bits = 1;
  while ((1 << bits) <= a.experts) ++bits;  // keys 0 .. experts
  const int E = a.experts;
  auto place_lds = [](int n) { return ((kWaves + 5) * n + kWaves * kTileLists) * 4; };
  static DeviceOnce once;
  hipError_t e = allow_lds(once, dev, reinterpret_cast<const void*>(group_place_kernel), place_lds(kMaxExperts));
  if (e != hipSuccess) return e;
  if (a.blocks > 1) {
    hipLaunchKernelGGL(group_count_kernel, dim3(a.blocks), dim3(kThreads), E * 4, stream, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(group_place_kernel, dim3(a.blocks), dim3(kThreads), place_lds(E), stream, a, bits);
  return hipGetLastError();
}

}  // namespace mm

// Rows (slots) ordered by expert: a stable counting sort on the device, so that
// routing never waits for the host.
//
// c_e = number of slots of expert e; its rows start at 32 * sum over e' < e of
// ceil(c_e' / 32), in ascending slot order.  Latency-bound: 4 bytes in and about
// 4 out per slot.  Every wavefront takes a run of consecutive slots, 64 at a
// time.  A lane's rank among the 64 is the number of lower lanes with its expert:
// one ballot per bit of the expert number gives every lane the mask of its equals,
// so there are no atomics and the order never depends on timing.  The counts
// per wavefront and expert sit in LDS; their sums over the wavefronts in front
// and the padded starts make them the next free row of that wavefront and
// expert.  More than kGroupChunk slots: a first launch leaves each workgroup's
// counts, the second places.
#include "grouped.hpp"

namespace mm {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

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

// Adds the slots of each expert in this wavefront's run to n[expert].
__device__ __forceinline__ void count_run(const GroupArgs& a, int64_t first, int bits, uint32_t* n, int lane) {
  for (int t = 0; t < a.turns; ++t) {
    const int64_t s0 = first + 64 * (int64_t)t;
    if (s0 >= a.rows) break;
    const int key = key_of(a, s0 + lane);
    const uint64_t m = equals(key, bits);
    if (key < a.experts && (m & ((1ull << lane) - 1)) == 0) n[key] += (uint32_t)__popcll(m);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

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
__global__ __launch_bounds__(kThreads) void group_count_kernel(GroupArgs a, int bits) {
  extern __shared__ uint32_t lds[];  // [kWaves][experts]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int E = a.experts;
  for (int i = threadIdx.x; i < kWaves * E; i += kThreads) lds[i] = 0;
  __syncthreads();
  const int64_t run = ((int64_t)blockIdx.x * kWaves + wave) * 64 * a.turns;
  count_run(a, run, bits, lds + wave * E, lane);
  __syncthreads();
  const int e = threadIdx.x;
  if (e < E) {
    uint32_t n = 0;
    for (int w = 0; w < kWaves; ++w) n += lds[w * E + e];
    a.counts[(int64_t)blockIdx.x * E + e] = (int32_t)n;
  }
}

// Places the slots; the rows, owners and tiles that no slot fills are shared out
// over the workgroups.
__global__ __launch_bounds__(kThreads) void group_place_kernel(GroupArgs a, int bits) {
  extern __shared__ uint32_t lds[];
  const int E = a.experts;
  uint32_t* const next = lds;                            // [kWaves][E]
  int* const total = (int*)(lds + kWaves * E);           // [E] slots of each expert
  int* const start = total + E;                          // [E + 1] first row group
  int* const tile0 = start + E + 1;                      // [3][E] first tile of 2, 4, 8 row groups
  int (*const part)[kTileLists] = (int (*)[kTileLists])(tile0 + 3 * E);  // [kWaves]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < kWaves * E; i += kThreads) next[i] = 0;
  __syncthreads();
  const int64_t run = ((int64_t)blockIdx.x * kWaves + wave) * 64 * a.turns;
  count_run(a, run, bits, next + wave * E, lane);
  __syncthreads();
  const int e = threadIdx.x;  // kThreads >= kMaxExperts
  int here = 0, before = 0, all = 0;
  if (e < E) {
    for (int w = 0; w < kWaves; ++w) {
      const int n = (int)next[w * E + e];
      next[w * E + e] = (uint32_t)here;
      here += n;
    }
    all = here;
    if (a.blocks > 1) {
      all = 0;
      for (int b = 0; b < a.blocks; ++b) {
        const int n = a.counts[(int64_t)b * E + e];
        before += b < (int)blockIdx.x ? n : 0;
        all += n;
      }
    }
  }
  const int g = (all + kRowGroup - 1) / kRowGroup;
  int v[kTileLists] = {g, (g + 1) / 2, (g + 3) / 4, (g + 7) / 8};
  const int own[kTileLists] = {v[0], v[1], v[2], v[3]};
  scan<kTileLists>(v, part, lane, wave);
  if (e < E) {
    const int s = v[0] - own[0];
    start[e] = s;
    total[e] = all;
#pragma unroll
    for (int k = 1; k < kTileLists; ++k) tile0[(k - 1) * E + e] = v[k] - own[k];
    if (e == E - 1) {
      start[E] = v[0];
      if (blockIdx.x == 0) a.starts[E] = v[0] * kRowGroup;
    }
    if (blockIdx.x == 0) a.starts[e] = s * kRowGroup;
    for (int w = 0; w < kWaves; ++w) next[w * E + e] += (uint32_t)(s * kRowGroup + before);
  }
  __syncthreads();
  // the slots, in their order
  for (int t = 0; t < a.turns; ++t) {
    const int64_t s0 = run + 64 * (int64_t)t;
    if (s0 >= a.rows) break;
    const int key = key_of(a, s0 + lane);
    const uint64_t m = equals(key, bits);
    const int rank = __popcll(m & ((1ull << lane) - 1));
    if (key < E) a.slots[next[wave * E + key] + rank] = (int32_t)(s0 + lane);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (key < E && rank == 0) next[wave * E + key] += (uint32_t)__popcll(m);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  // the row groups: owner, rows without a slot, tiles
  const int used = start[E];
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
      const int rel = q - start[lo], left = total[lo] - rel * kRowGroup;
      filled = left < kRowGroup ? left : kRowGroup;
      const uint32_t o = (uint32_t)owner;
      a.tiles[0][q] = RowTile{q, o | (uint32_t)filled << 16};
#pragma unroll
      for (int k = 1; k < kTileLists; ++k)
        if ((rel & ((1 << k) - 1)) == 0) {
          const int most = kRowGroup << k;
          a.tiles[k][tile0[(k - 1) * E + lo] + (rel >> k)] = RowTile{q, o | (uint32_t)(left < most ? left : most) << 16};
        }
    } else {
      a.tiles[0][q] = RowTile{-1, 0};
    }
    a.owners[q] = owner;
    for (int r = filled; r < kRowGroup; ++r) a.slots[(int64_t)q * kRowGroup + r] = -1;
  }
  // tiles behind the last
#pragma unroll
  for (int k = 1; k < kTileLists; ++k) {
    int n = E > 0 ? tile0[(k - 1) * E + E - 1] + ((start[E] - start[E - 1] + (1 << k) - 1) >> k) : 0;
    for (int i = n + at; i < a.ntiles[k]; i += stride) a.tiles[k][i] = RowTile{-1, 0};
  }
}

hipError_t launch_group_rows(const GroupArgs& a, const Device& dev, hipStream_t stream) {
  int bits = 1;
  while ((1 << bits) <= a.experts) ++bits;  // keys 0 .. experts
  const int E = a.experts;
  const int count_lds = kWaves * E * 4;
  const int place_lds = (kWaves * E + 5 * E + 1) * 4 + kWaves * kTileLists * 4;
  constexpr int kMost = (int)((kWaves + 5) * kMaxExperts + 1 + kWaves * kTileLists) * 4;
  static DeviceOnce once_count, once_place;
  hipError_t e = allow_lds(once_place, dev, reinterpret_cast<const void*>(group_place_kernel), kMost);
  if (e != hipSuccess) return e;
  if (a.blocks > 1) {
    e = allow_lds(once_count, dev, reinterpret_cast<const void*>(group_count_kernel), kMost);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(group_count_kernel, dim3(a.blocks), dim3(kThreads), count_lds, stream, a, bits);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(group_place_kernel, dim3(a.blocks), dim3(kThreads), place_lds, stream, a, bits);
  return hipGetLastError();
}

}  // namespace mm

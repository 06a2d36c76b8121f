// Beam search: the states of a group's beams brought in line with the parents that its
// selection chose.
#include <algorithm>

#include "common.h"
#include "ops.h"

namespace tcl {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(1)));  // states of any size start anywhere

// Bytes that one workgroup copies of each state: 64 groups of 8 beams with 130 segments of 16 KB take 83.9 us, of 8 KB 80.9,
// of 4 KB 82.9.
constexpr int kSegment = 8 * 1024;
constexpr int kThreads = 256;

struct Pools {
  int n;
  int first[kPoolsPerLaunch + 1];  // a pool's first segment
  BeamPool p[kPoolsPerLaunch];
};

// Of a group's beams on one wavefront, beam b in lane b: its parent's lane (-1: none), the
// place of its state, and whether the state has to be copied there. The first child of a parent
// stays where the parent's state is; the others, in their order, go to the places of the parents
// without a child, in theirs. What is copied from is a place that is kept, and what is copied to is not, so the
// copies of a group neither wait for nor disturb each other, whatever the parents are.
struct Place {
  int from, to;  // of the pool; -1: nothing to copy
  int slot;      // the beam's place
};
__device__ __forceinline__ Place place_of(const int* __restrict__ parent, const int* __restrict__ slots, int W, int g,
                                          int n_slots) {
  const int lane = threadIdx.x & 63;
  const bool beam = lane < W;
  const int64_t row = (int64_t)g * W + lane;
  int p = -1, slot = -1;
  if (beam) {
    const int64_t q = parent[row] - (int64_t)g * W;
    p = q >= 0 && q < W ? (int)q : -1;
    slot = slots[row];
  }
  bool first = p >= 0;
  uint64_t kept = 0;
  for (int j = 0; j < W; ++j) {
    const int o = __shfl(p, j, 64);
    if (o >= 0) kept |= 1ull << o;
    if (j < lane && o == p) first = false;
  }
  const uint64_t all = W == 64 ? ~0ull : (1ull << W) - 1, others = __ballot(beam && !first);
  uint64_t free = all & ~kept;
  for (int k = __popcll(others & ((1ull << lane) - 1)); k > 0; --k) free &= free - 1;
  const int at = first ? p : free ? __ffsll((unsigned long long)free) - 1 : 0;
  const int mine = __shfl(slot, at, 64), theirs = __shfl(slot, p < 0 ? 0 : p, 64);
  const bool copy = beam && p >= 0 && !first && mine >= 0 && mine < n_slots && theirs >= 0 && theirs < n_slots;
  return {copy ? theirs : -1, copy ? mine : -1, mine};
}

// One segment of the states, of every beam of a group that moves. Bound by HBM: each moved
// state read and written once (230 MB moved in 79 us: children of one parent find it in the cache); the plan is formed
// again by every workgroup (about a microsecond).
__global__ __launch_bounds__(kThreads) void beam_reorder_kernel(int W, const int* __restrict__ parent,
                                                                const int* __restrict__ slots, int n_slots,
                                                                int* __restrict__ slots_out, int groups, Pools pools) {
  __shared__ int from[64], to[64];
  const int tid = threadIdx.x;
  int q = 0;
  while (q < pools.n && (int)blockIdx.x >= pools.first[q + 1]) ++q;
  const bool pool = q < pools.n;
  const int64_t bytes = pool ? pools.p[q].bytes : 0, o = pool ? (int64_t)(blockIdx.x - pools.first[q]) * kSegment : 0;
  const int len = (int)min((int64_t)kSegment, bytes - o), vecs = len / 16;
  for (int g = blockIdx.y; g < groups; g += gridDim.y) {
    __syncthreads();  // (the plan of the group before is read)
    if (tid < 64) {
      const Place pl = place_of(parent, slots, W, g, n_slots);
      from[tid] = pl.from;
      to[tid] = pl.to;
      if (slots_out && blockIdx.x == 0 && tid < W) slots_out[(int64_t)g * W + tid] = pl.slot;
    }
    __syncthreads();
    if (!pool) continue;
    for (int b = 0; b < W; ++b) {
      if (from[b] < 0) continue;
      const char* src = static_cast<const char*>(pools.p[q].data) + from[b] * bytes + o;
      char* dst = static_cast<char*>(pools.p[q].data) + to[b] * bytes + o;
      u32x4 v[kSegment / 16 / kThreads];
#pragma unroll
      for (int k = 0; k < kSegment / 16 / kThreads; ++k)
        if (tid + k * kThreads < vecs) v[k] = *reinterpret_cast<const u32x4_any*>(src + 16 * (tid + k * kThreads));
#pragma unroll
      for (int k = 0; k < kSegment / 16 / kThreads; ++k)
        if (tid + k * kThreads < vecs) *reinterpret_cast<u32x4_any*>(dst + 16 * (tid + k * kThreads)) = v[k];
      if (tid < len - 16 * vecs) dst[16 * vecs + tid] = src[16 * vecs + tid];
    }
  }
}

}  // namespace

hipError_t launch_beam_reorder(int groups, int W, const int* parent, const int* slots, int n_slots, int* slots_out,
                               int n_pools, const BeamPool* pools, hipStream_t s) {
  // fewer than 2^32 threads in a launch: what 63 of the largest pools take, and many groups of large states share workgroups
  constexpr int kMaxGroups = (1 << 24) - 1;
  int k = 0;
  do {
    Pools p = {};
    for (; k + p.n < n_pools && p.n < kPoolsPerLaunch; ++p.n) {
      const int segs = (int)((pools[k + p.n].bytes + kSegment - 1) / kSegment);
      if (segs > kMaxGroups - p.first[p.n]) break;
      p.p[p.n] = pools[k + p.n];
      p.first[p.n + 1] = p.first[p.n] + segs;
    }
    const int segs = std::max(p.first[p.n], 1);
    const dim3 grid(segs, std::min({groups, 65535, kMaxGroups / segs}));
    beam_reorder_kernel<<<grid, kThreads, 0, s>>>(W, parent, slots, n_slots, k == 0 ? slots_out : nullptr, groups, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k += p.n;
  } while (k < n_pools);
  return hipSuccess;
}

}  // namespace tcl

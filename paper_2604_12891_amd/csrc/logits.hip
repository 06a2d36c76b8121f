// Operators on rows of logits: log probabilities of given entries with the
// row's entropy and top alternatives, and distillation from a teacher's top
// logits (loss and gradient).
//
// A row is read in aligned 16-byte vectors whatever its own alignment: vector v
// covers entries v VE - h .. v VE - h + VE - 1, h the entries between the
// aligned address and the row's start, and only the first and the last vector of a
// row are read entry by entry. (A beam search's rows are read otherwise, see Row.)
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "ops.h"

namespace tcl {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int kTB = 256;  // threads of the streaming kernels

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// 16 bytes at the alignment of one entry.
template <typename T> struct Loose;
template <> struct Loose<float> { typedef u32x4 type __attribute__((aligned(4))); };
template <> struct Loose<uint16_t> { typedef u32x4 type __attribute__((aligned(2))); };

// A row's entries (or a part of it): VE to a vector. START: vectors count from the row's first entry (h is 0) and are read
// unaligned, so that rows of the same entries give the same sums, bit for bit, wherever they start.
template <typename T, bool START = false>
struct Row {
  static constexpr int VE = 16 / sizeof(T);
  const T* p;   // the first entry
  int cnt;      // entries
  int first;    // index of the first one as the caller counts
  int h;        // entries in front of p in its aligned vector
  int nvec;

  __device__ __forceinline__ Row(const LogitRows& a, int r) {
    const int64_t o = a.offs ? a.offs[r] : (int64_t)r * a.ld;
    p = static_cast<const T*>(a.x) + o;
    cnt = !a.offs ? a.V : a.x ? max(a.offs[r + 1] - a.offs[r], 0) : 0;
    first = a.offs ? a.offs[r] : 0;
    h = START ? 0 : (int)((reinterpret_cast<uintptr_t>(p) / sizeof(T)) % VE);
    nvec = cnt > 0 ? (cnt + h + VE - 1) / VE : 0;
  }
  __device__ __forceinline__ bool whole(int v) const { return v * VE >= h && v * VE - h + VE <= cnt; }
  // raw vector v; entries outside the row are -inf
  __device__ __forceinline__ u32x4 load(int v) const {
    if (whole(v)) {
      if constexpr (START) return *reinterpret_cast<const typename Loose<T>::type*>(p + (v * VE - h));
      else return *reinterpret_cast<const u32x4*>(p + (v * VE - h));
    }
    u32x4 x;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        const int i = v * VE - h + k;
        x[k] = i >= 0 && i < cnt ? __float_as_uint(p[i]) : 0xFF800000u;
      } else {
        const int i = v * VE - h + 2 * k;
        const uint32_t lo = i >= 0 && i < cnt ? p[i] : 0xFF80u, hi = i + 1 >= 0 && i + 1 < cnt ? p[i + 1] : 0xFF80u;
        x[k] = lo | hi << 16;
      }
    }
    return x;
  }
  static __device__ __forceinline__ float get(u32x4 x, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(x[i]);
    else return __uint_as_float(i & 1 ? x[i >> 1] & 0xFFFF0000u : x[i >> 1] << 16);
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return p[i];
    else return bf16_to_f32(p[i]);
  }
};

// ---------------------------------------------------------------- order of entries
// One number per entry that orders as the top list does: by value, NaN after
// every number, equal values by lower index. The value's bits as an unsigned number that
// rises with it (16 of them for bf16), from bit 32 up; below 2^b - index, 2^b > the row's
// entries. 0: no entry.
template <typename T>
__device__ __forceinline__ uint32_t ord_of(float x) {
  uint32_t u = __float_as_uint(x + 0.0f);  // -0 as 0
  u = u & 0x80000000u ? ~u : u | 0x80000000u;
  if (!(x == x)) u = 0;
  return sizeof(T) == 2 ? u >> 16 : u;
}
template <typename T>
__device__ __forceinline__ float ord_value(uint32_t u) {  // -inf for NaN
  if (sizeof(T) == 2) u = u << 16 | (u & 0x8000u ? 0 : 0xFFFFu);
  if (u <= 0x007FFFFFu) return -INFINITY;
  return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ int index_bits(int cnt) { return 32 - __clz(cnt); }

// ---------------------------------------------------------------- sums of a softmax
// m = max x, s = sum e, t = sum (x - m) e, e = exp((x - m) / temperature); zc = log2(e) / temperature.
struct Stats {
  float m, s, t;
};
__device__ __forceinline__ Stats merge(Stats a, Stats b, float zc) {
  const float m = fmaxf(a.m, b.m);
  Stats r = {m, 0.f, 0.f};
  // (a part whose maximum is a type's lowest value may have d s beyond fp32, and f 0)
  if (a.m > -INFINITY) {
    const float d = a.m == m ? 0.f : a.m - m, f = __builtin_amdgcn_exp2f(d * zc);
    r.s = f * a.s;
    r.t = f > 0.f ? f * fmaf(d, a.s, a.t) : 0.f;
  }
  if (b.m > -INFINITY) {
    const float d = b.m == m ? 0.f : b.m - m, f = __builtin_amdgcn_exp2f(d * zc);
    r.s = fmaf(f, b.s, r.s);
    if (f > 0.f) r.t = fmaf(f, fmaf(d, b.s, b.t), r.t);
  }
  return r;
}
__device__ __forceinline__ Stats wave_merge(Stats a, float zc) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const Stats b = {__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.t, o, 64)};
    a = merge(a, b, zc);
  }
  return a;
}

// ---------------------------------------------------------------- the K highest
// Finding the K highest costs one comparison per vector while the row streams by:
// every thread keeps its own highest entry, and in LDS the highest value of each of up
// to kGroups stretches of its entries. Of the threads' keys the K-th highest is a bound tau that
// at least K entries reach, and an entry that reaches it lies in a stretch, of one of the K threads
// whose highest does, whose highest value does: some K stretches, read again out of the caches. What
// is >= tau there goes to a list in LDS, K to some 2 K entries, and each entry of the list
// counts the ones above it for its rank. A list that overflows (rows made of many
// near-copies of one stretch) takes the exact K-th key by bisection over its bits instead.
constexpr int kMaxTop = 64;
constexpr int kGroups = 16;

template <int TB>
struct TopShared {
  static constexpr int kCap = 4 * TB;
  union {
    u64 cand[kCap];
    uint16_t high[kGroups][TB];  // bits 16..31 (of bf16 all) of a stretch's ord_of
  };
  u64 key[TB];
  u64 best[kMaxTop];
  uint16_t list[kMaxTop * kGroups];  // stretches to read again: group * TB + thread
  int n, nlist;
  u64 tau;
};

// On one wavefront: the K-th highest of n > K distinct keys (Q to a lane, 0: none), or a bound that exactly K
// reach, bit by bit, counting by ballot (comparing every key with every other takes 30 times the
// instructions at 256 keys). Value bits 32 .. top + 31, index bits 0 .. b.
template <int Q>
__device__ __forceinline__ u64 kth_key(const u64* k, int K, int top, int b) {
  u64 lo = 0;
  for (int bit = 31 + top; bit >= 0; --bit) {
    if (bit == 31) bit = b;
    const u64 trial = lo | 1ull << bit;
    int c = 0;
#pragma unroll
    for (int j = 0; j < Q; ++j) c += __popcll(__ballot(k[j] >= trial));
    if (c >= K) lo = trial;
    if (c == K) break;
  }
  return lo;
}

// From every thread's highest key (0: none) the bound tau.
template <int TB>
__device__ __forceinline__ void top_bound(TopShared<TB>& sh, u64 key, int K, int top, int b) {
  const int tid = threadIdx.x;
  sh.key[tid] = key;
  for (int i = tid; i < K; i += TB) sh.best[i] = 0;
  __syncthreads();
  if (tid < 64) {
    constexpr int Q = TB / 64;
    u64 k[Q];
    int have = 0;
#pragma unroll
    for (int j = 0; j < Q; ++j) {
      k[j] = sh.key[j * 64 + tid];
      have += __popcll(__ballot(k[j] != 0));
    }
    const u64 tau = have > K ? kth_key<Q>(k, K, top, b) : 1;  // too few: all entries
    if (tid == 0) {
      sh.n = 0;
      sh.nlist = 0;
      sh.tau = tau;
    }
  }
  __syncthreads();
}

// The K highest of the keys that each(f) hands to f on all threads together, into
// sh.best, highest first; at least K reach sh.tau (or all that there are). sh.n starts at 0.
template <int TB, typename Each>
__device__ __forceinline__ void top_collect(TopShared<TB>& sh, int K, int top, int b, Each each) {
  constexpr int kCap = TopShared<TB>::kCap;
  const int tid = threadIdx.x;
  auto gather = [&](u64 tau) {
    each([&](u64 k) {
      if (k >= tau) {
        const int p = atomicAdd(&sh.n, 1);
        if (p < kCap) sh.cand[p] = k;
      }
    });
    __syncthreads();
  };
  gather(sh.tau);
  int n = sh.n;
  if (n > kCap) {
    u64 lo = 0;  // at least K keys reach lo
    for (int bit = 31 + top; bit >= 0; --bit) {
      if (bit == 31) bit = b;
      const u64 trial = lo | 1ull << bit;
      int c = 0;
      each([&](u64 k) { c += k >= trial; });
      __syncthreads();
      if (tid == 0) sh.n = 0;
      __syncthreads();
      if (c) atomicAdd(&sh.n, c);
      __syncthreads();
      if (sh.n >= K) lo = trial;
    }
    __syncthreads();
    if (tid == 0) sh.n = 0;
    __syncthreads();
    gather(lo);
    n = min(sh.n, kCap);
  }
  if (n > K + K / 2 + 8) {
    // only the K highest of the list are ranked
    if (tid < 64) {
      constexpr int Q = kCap / 64;
      u64 k[Q];
#pragma unroll
      for (int j = 0; j < Q; ++j) k[j] = j * 64 + tid < n ? sh.cand[j * 64 + tid] : 0;
      const u64 lo = kth_key<Q>(k, K, top, b);
      int at = 0;
#pragma unroll
      for (int j = 0; j < Q; ++j) {
        const bool in = k[j] >= lo && k[j] != 0;
        const u64 m = __ballot(in);
        if (in) sh.cand[at + __popcll(m & ((1ull << tid) - 1))] = k[j];
        at += __popcll(m);
      }
    }
    n = K;
    __syncthreads();
  }
  for (int i = tid; i < n; i += TB) {
    const u64 k = sh.cand[i];
    int above = 0;
    for (int j = 0; j < n; ++j) above += sh.cand[j] > k;
    if (above < K) sh.best[above] = k;
  }
  __syncthreads();
}

// What leaves for one row.
struct LogprobOut {
  const int* tokens;
  float *logp, *entropy;
  int* top;
  float* top_logp;
};
// Rows that are a search's beams: whether beam r goes on (neither dead nor ended).
struct Beams {
  const float* score;
  const int* ended;  // or null
  __device__ __forceinline__ bool open(int r) const { return score[r] > -INFINITY && !(ended && ended[r] >= 0); }
};

template <typename T, int TB>
__device__ __forceinline__ void finish_row(const LogitRows& a, const Row<T>& row, int r, Stats st,
                                           const TopShared<TB>& sh, int K, const LogprobOut& o) {
  const float ls = logf(st.s);  // -inf for a row with nothing left
  const bool none = !(st.m > -INFINITY);
  auto logp = [&](float x) { return none || !(x > -INFINITY) ? -INFINITY : fmaf(x - st.m, a.inv_temp, -ls); };
  if (threadIdx.x == 0) {
    if (o.logp) {
      const int64_t i = (int64_t)o.tokens[r] - row.first;
      o.logp[r] = i >= 0 && i < row.cnt ? logp(row.at((int)i)) : NAN;
    }
    if (o.entropy) o.entropy[r] = none ? 0.f : fmaf(-a.inv_temp, st.t / st.s, ls);
  }
  for (int i = threadIdx.x; i < K; i += TB) {
    const u64 k = sh.best[i];
    const int64_t j = (int64_t)r * K + i;
    o.top[j] = k ? (int)((1u << index_bits(row.cnt)) - (uint32_t)k) + row.first : -1;
    if (o.top_logp) o.top_logp[j] = k ? logp(ord_value<T>((uint32_t)(k >> 32))) : -INFINITY;
  }
}

// A split's results in the workspace: the K highest keys, then the sums.
__device__ __forceinline__ int64_t split_stride(int K) { return (int64_t)K * 8 + 16; }

// One pass over a row (or the part of it that blockIdx.y names): running maximum with
// the sums rescaled when it rises, once per vector at most. Bound by HBM from a
// few thousand entries on: 4,096 rows of 32,768 bf16 entries in 66 us with 20 top entries, 53 without
// (58 at the rate of a copy, which also writes). A workgroup that went on to a next row whose first vectors were
// loaded ahead took 89. gridDim.y == 1: the row's results leave from here. BEAM: they go to the workspace, as
// those of splits do, and rows of beams that do not go on are not read.
template <typename T, int TB, bool BEAM = false>
__global__ __launch_bounds__(TB) void logprobs_kernel(LogitRows a, int K, LogprobOut o, char* __restrict__ ws,
                                                      Beams beams = {}) {
  if (BEAM && !beams.open(blockIdx.x)) return;
  constexpr int VE = Row<T>::VE;
  __shared__ __attribute__((aligned(16))) TopShared<TB> sh;
  __shared__ Stats part[TB / 64];
  const int r = blockIdx.x, tid = threadIdx.x;
  const Row<T, BEAM> row(a, r);
  const int per = (row.nvec + gridDim.y - 1) / gridDim.y;
  const int v0 = min((int)blockIdx.y * per, row.nvec), v1 = min(v0 + per, row.nvec);
  const float zc = a.inv_temp * kLog2e;
  Stats st = {-INFINITY, 0.f, 0.f};
  float best = -INFINITY;
  int bv = -1;
  u32x4 bx = {0, 0, 0, 0};  // the vector that holds it
  constexpr int U = 4;
  // trips of U vectors to a stretch
  const int trips = (v1 - v0 + U * TB - 1) / (U * TB), span = (trips + kGroups - 1) / kGroups;
  float high = -INFINITY;
  int trip = 0;
  for (int vb = v0 + tid; vb < v1; vb += U * TB, ++trip) {
    u32x4 x[U];
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (vb + k * TB < v1) x[k] = row.load(vb + k * TB);
    if (trip % span == 0) high = -INFINITY;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (vb + k * TB >= v1) break;
      float f[VE], vm = -INFINITY;
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        f[i] = Row<T>::get(x[k], i);
        vm = fmaxf(vm, f[i]);
      }
      high = fmaxf(high, vm);
      if (vm > best) {
        best = vm;
        bv = vb + k * TB;
        bx = x[k];
        // the sums move to the new maximum
        if (st.m > -INFINITY) {
          const float d = st.m - vm, g = __builtin_amdgcn_exp2f(d * zc);
          st.t = g > 0.f ? g * fmaf(d, st.s, st.t) : 0.f;
          st.s *= g;
        }
        st.m = vm;
      }
      if (st.m > -INFINITY) {
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          const float d = fmaxf(f[i] - st.m, -3.0e38f);  // -inf and NaN: no probability
          const float e = __builtin_amdgcn_exp2f(d * zc);
          st.s += e;
          st.t = fmaf(d, e, st.t);
        }
      }
    }
    if (K > 0) sh.high[trip / span][tid] = (uint16_t)(ord_of<T>(high) >> (8 * sizeof(T) - 16));
  }
  st = wave_merge(st, zc);
  if ((tid & 63) == 0) part[tid >> 6] = st;
  __syncthreads();
  st = part[0];
#pragma unroll
  for (int k = 1; k < TB / 64; ++k) st = merge(st, part[k], zc);

  if (K > 0) {
    const int b = index_bits(row.cnt);
    auto vec_keys = [&](int v, u32x4 y, auto f) {
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const int j = v * VE - row.h + i;
        if (j >= 0 && j < row.cnt) f((u64)ord_of<T>(Row<T>::get(y, i)) << 32 | ((1u << b) - (uint32_t)j));
      }
    };
    u64 key = 0;
    if (bv >= 0) {
      vec_keys(bv, bx, [&](u64 k) { key = max(key, k); });
    } else {  // nothing above -inf: the order among -inf and NaN
      for (int v = v0 + tid; v < v1; v += TB) vec_keys(v, row.load(v), [&](u64 k) { key = max(key, k); });
    }
    top_bound(sh, key, K, 8 * sizeof(T), b);
    const uint32_t need = (uint32_t)(sh.tau >> 32);
    if (key && key >= sh.tau) {
      const int mine = v0 + tid < v1 ? ((v1 - v0 - tid - 1) / (U * TB)) / span + 1 : 0;
      for (int g = 0; g < mine; ++g)
        if (sh.high[g][tid] >= need >> (8 * sizeof(T) - 16)) sh.list[atomicAdd(&sh.nlist, 1)] = (uint16_t)(g * TB + tid);
    }
    __syncthreads();
    // the vectors of those stretches, shared out over all threads
    const int each_n = U * span, units = sh.nlist * each_n;
    const float floor = ord_value<T>(need);
    top_collect(sh, K, 8 * sizeof(T), b, [&](auto f) {
      for (int q = tid; q < units; q += TB) {
        const int l = sh.list[q / each_n], v = v0 + l % TB + (l / TB * each_n + q % each_n) * TB;
        if (v >= v1) continue;
        const u32x4 y = row.load(v);
        float vm = -INFINITY;
#pragma unroll
        for (int i = 0; i < VE; ++i) vm = fmaxf(vm, Row<T>::get(y, i));
        if (vm >= floor) vec_keys(v, y, f);
      }
    });
  }
  if constexpr (!BEAM) {
    if (gridDim.y == 1) {
      finish_row(a, row, r, st, sh, K, o);
      return;
    }
  }
  char* w = ws + ((int64_t)r * gridDim.y + blockIdx.y) * split_stride(K);
  for (int i = tid; i < K; i += TB) reinterpret_cast<u64*>(w)[i] = sh.best[i];
  if (tid == 0) *reinterpret_cast<Stats*>(w + (int64_t)K * 8) = st;
}

// The splits of a row joined: one workgroup per row.
template <typename T>
__global__ __launch_bounds__(kTB) void logprobs_join_kernel(LogitRows a, int K, int splits, LogprobOut o,
                                                            const char* __restrict__ ws) {
  __shared__ __attribute__((aligned(16))) TopShared<kTB> sh;
  __shared__ Stats part[kTB / 64];
  const int r = blockIdx.x, tid = threadIdx.x;
  const Row<T> row(a, r);
  const float zc = a.inv_temp * kLog2e;
  const char* w = ws + (int64_t)r * splits * split_stride(K);
  Stats st = {-INFINITY, 0.f, 0.f};
  for (int k = tid; k < splits; k += kTB)
    st = merge(st, *reinterpret_cast<const Stats*>(w + k * split_stride(K) + (int64_t)K * 8), zc);
  st = wave_merge(st, zc);
  if ((tid & 63) == 0) part[tid >> 6] = st;
  __syncthreads();
  st = part[0];
#pragma unroll
  for (int k = 1; k < kTB / 64; ++k) st = merge(st, part[k], zc);
  if (K > 0) {
    auto each = [&](auto f) {
      for (int q = tid; q < splits * K; q += kTB) {
        const u64 k = reinterpret_cast<const u64*>(w + q / K * split_stride(K))[q % K];
        if (k) f(k);
      }
    };
    u64 key = 0;
    each([&](u64 k) { key = max(key, k); });
    const int b = index_bits(row.cnt);
    top_bound(sh, key, K, 8 * sizeof(T), b);
    top_collect(sh, K, 8 * sizeof(T), b, each);
  }
  finish_row(a, row, r, st, sh, K, o);
}

// ---------------------------------------------------------------- beam search: selection
// A group's K best candidates (b, v) by score_b + log p_b(v), out of its rows' lists of K: each list is
// sorted, so every round takes the best of the lists' heads. Scores are compared in 64 bits: fp32 would make
// neighbours equal that a long search's sum of log probabilities (-100: steps of 8e-6) cannot tell
// apart. (The sums of exponentials in them are fp32: against 64 bits their logarithms were off by up to 4e-7 for 77
// to 131,073 entries, 8e-7 for 1,000,003. Rows of the same entries have the same: lists come from rows read from
// their start, 512 of 131,073 bf16 entries in 52.5 us a call, 4 of 50,001 in fp32 in 16.4; by aligned vectors 48.8
// and 15.7.) Equal scores (a temperature or a score beyond which the logits' differences count nothing): the lower
// row, and in a row the order that its list has, by the logits. All scores are formed at once, as numbers that rise
// with them (0: none); then a wavefront runs the rounds, each the largest of its lanes' heads (the high halves as a
// rule tell) and one lane's step on, out of LDS where the lists fit: some 0.3 us. A chain of latencies: 5.7 us for 4
// beams and K = 4, 9.8 to 10.8 for 64 groups of 8 and K = 16 (the rows' lists, 512 rows of 131,072 bf16 entries, 37
// at the rate of 3.6 TB/s); counting how many candidates beat each instead of rounds took 12 to 26.
constexpr int kBeamLists = 1024;  // W x splits
constexpr int kBeamKeys = 4096;   // candidates held in LDS

__device__ __forceinline__ u64 order_of(double s) {  // 0 for -inf and NaN
  if (!(s > -(double)INFINITY)) return 0;
  const u64 u = __builtin_bit_cast(u64, s + 0.0);  // (-0 as 0)
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double score_of(u64 k) {
  return k == 0 ? -(double)INFINITY : __builtin_bit_cast(double, k >> 63 ? k & ~(1ull << 63) : ~k);
}
// The largest over a wavefront.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  auto turn = [](uint32_t x, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, false);
  };
  v = max(v, turn(v, std::integral_constant<int, 0x128>()));  // rows of 16 lanes, turned by 8, 4, 2, 1
  v = max(v, turn(v, std::integral_constant<int, 0x124>()));
  v = max(v, turn(v, std::integral_constant<int, 0x122>()));
  v = max(v, turn(v, std::integral_constant<int, 0x121>()));
  auto of = [&](int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
  return max(max(of(0), of(16)), max(of(32), of(48)));
}

template <typename T>
__global__ __launch_bounds__(kTB) void beam_join_kernel(LogitRows a, int W, int K, int splits, Beams beams,
                                                        int* __restrict__ parent, int* __restrict__ token,
                                                        float* __restrict__ out_score, const char* __restrict__ ws) {
  __shared__ u64 keys[kBeamKeys], order[kBeamKeys];
  __shared__ u64 head[kBeamLists];      // a list's best score that is left
  __shared__ uint16_t at[kBeamLists];   // and its place
  __shared__ Stats part[kBeamLists];
  __shared__ double base[64], top[64];  // score - log of the sum; the maximum
  __shared__ float own_score[64];
  __shared__ int alone[64];             // -1: an open beam; else it has ended with this token (-2: dead)
  __shared__ int from[kMaxTop];         // the candidates taken: list * K + place
  __shared__ u64 taken[kMaxTop];
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, lists = W * splits, N = lists * K;
  const float zc = a.inv_temp * kLog2e;
  const double it = a.inv_temp;
  const char* w = ws + (int64_t)g * lists * split_stride(K);
  const bool held = N <= kBeamKeys;
  auto key_of = [&](int l, int i) {
    return held ? keys[l * K + i] : reinterpret_cast<const u64*>(w + (int64_t)l * split_stride(K))[i];
  };
  // all that is read from memory at once (of rows that were not read whatever is there, for nothing)
  if (held)
    for (int q = tid; q < N; q += kTB) keys[q] = reinterpret_cast<const u64*>(w + (int64_t)(q / K) * split_stride(K))[q % K];
  for (int l = tid; l < lists; l += kTB) part[l] = *reinterpret_cast<const Stats*>(w + (int64_t)l * split_stride(K) + (int64_t)K * 8);
  if (tid < W) {
    const float score = beams.score[g * W + tid];
    const int ended = beams.ended ? beams.ended[g * W + tid] : -1;
    own_score[tid] = score;
    alone[tid] = !(score > -INFINITY) ? -2 : ended >= 0 ? ended : -1;
  }
  __syncthreads();
  for (int b = tid >> 6; b < W; b += kTB / 64) {
    Stats st = {-INFINITY, 0.f, 0.f};
    for (int k = lane; k < splits; k += 64) st = merge(st, part[b * splits + k], zc);
    if (splits > 1) st = wave_merge(st, zc);
    if (lane == 0) {
      base[b] = alone[b] == -1 ? (double)own_score[b] - log((double)st.s) : (double)own_score[b];
      top[b] = st.m;
    }
  }
  __syncthreads();
  auto make = [&](int l, int i) {
    const int b = l / splits;
    if (alone[b] != -1) return i == 0 && l % splits == 0 && alone[b] >= 0 ? order_of(base[b]) : 0;  // itself, once
    const u64 k = key_of(l, i);
    return k ? order_of(base[b] + ((double)ord_value<T>((uint32_t)(k >> 32)) - top[b]) * it) : 0;
  };
  if (held)
    for (int q = tid; q < N; q += kTB) order[q] = make(q / K, q % K);
  __syncthreads();
  auto next_of = [&](int l, int i) { return i >= K ? 0 : held ? order[l * K + i] : make(l, i); };
  for (int l = tid; l < lists; l += kTB) {
    head[l] = next_of(l, 0);
    at[l] = 0;
  }
  if (tid < kMaxTop) {
    from[tid] = -1;
    taken[tid] = 0;
  }
  __syncthreads();
  if (tid >= 64) return;
  // the best of the lane's lists (of equal ones the lowest), as a rule the one that it has
  u64 key = 0;
  int mine = lane;
  auto own = [&]() {
    key = 0;
    for (int l = lane; l < lists; l += 64)
      if (head[l] > key) {
        key = head[l];
        mine = l;
      }
  };
  own();
  for (int i = 0; i < K; ++i) {
    const uint32_t hi = (uint32_t)(key >> 32), lo = (uint32_t)key;
    u64 best = __ballot(hi == wave_max(hi));
    if (best & (best - 1)) {  // more than one: by the low halves, then by the list
      const bool in = best >> lane & 1;
      best &= __ballot(lo == wave_max(in ? lo : 0u));
      if (best & (best - 1)) {  // equal scores: the lowest row, then of its parts the highest logit and lowest token
        const uint32_t row = (uint32_t)~(mine / splits);
        best &= __ballot(row == wave_max(best >> lane & 1 ? row : 0u));
        if (best & (best - 1)) {
          const u64 k = best >> lane & 1 && key ? key_of(mine, at[mine]) : 0;
          const uint32_t khi = (uint32_t)(k >> 32), klo = (uint32_t)k;
          best &= __ballot(khi == wave_max(khi));
          best &= __ballot(klo == wave_max(best >> lane & 1 ? klo : 0u));
        }
      }
    }
    if (lane == __ffsll(best) - 1 && key) {
      const int p = at[mine];
      from[i] = mine * K + p;
      taken[i] = key;
      at[mine] = (uint16_t)(p + 1);
      const u64 k = next_of(mine, p + 1);
      head[mine] = k;
      key = k;
      if (lists > 64) own();
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  const int bits = index_bits(a.V);
  if (lane < K) {  // (K <= kMaxTop, a wavefront's lanes)
    const int64_t j = (int64_t)g * K + lane;
    const int q = from[lane], l = q / K, b = l / splits;
    parent[j] = q < 0 ? -1 : g * W + b;
    token[j] = q < 0 ? -1 : alone[b] == -1 ? (int)((1u << bits) - (uint32_t)key_of(l, q % K)) : alone[b];
    out_score[j] = (float)score_of(taken[lane]);
  }
}

// ---------------------------------------------------------------- distillation from top logits
// q = softmax of the teacher's K logits, p = softmax of the student's row, both at 1 / inv_temp:
//   loss = sum_k q_k (log q_k - log p_(i_k)),  dloss/dx_v = inv_temp (p_v - sum_k [i_k = v] q_k).
// Entries without a place in the row (index outside it) do not count. A row without any
// teacher's entry, or whose own entries are all -inf, has loss 0 and gradient 0.
// exp(d / temperature) for a difference d of logits. One product with log2(e) / temperature and the
// hardware's exp2 are off by |d / temperature| units of rounding, which a bf16 gradient does not show;
// for fp32 logits what the product and the constant round away is put back, down to exp2(-200), a zero:
// past it the product would overflow at low temperatures and a mask's -inf not count at high ones.
template <typename T>
struct ScaledExp {
  float hi, lo, least;
  __device__ __forceinline__ explicit ScaledExp(float inv_temp) {
    hi = inv_temp * kLog2e;
    lo = fmaf(inv_temp, 1.925963e-8f, fmaf(inv_temp, kLog2e, -hi));  // log2(e) is kLog2e + 1.925963e-8
    least = -200.f / hi;
  }
  __device__ __forceinline__ float operator()(float d) const {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(d * hi);
    d = d < least ? least : d;  // (a NaN stays one)
    const float t = d * hi, e = __builtin_amdgcn_exp2f(t);
    return fmaf(e, fmaf(d, lo, fmaf(d, hi, -t)) * kLn2, e);
  }
};
struct TeacherArgs {
  int K;
  const int* top;
  const float* val;
  const float* weight;
  float* loss;
  void* grad;
  int64_t ldg;
};

// Two values over a workgroup's wavefronts at once, the larger or the sum of each. `red` is
// used once, so one barrier is enough.
template <int NW, bool MAX>
__device__ __forceinline__ void block_reduce(float& a, float& b, float* red) {
  a = MAX ? wave_max(a) : wave_sum(a);
  b = MAX ? wave_max(b) : wave_sum(b);
  if ((threadIdx.x & 63) == 0) {
    red[threadIdx.x >> 6] = a;
    red[16 + (threadIdx.x >> 6)] = b;
  }
  __syncthreads();
  a = red[0];
  b = red[16];
#pragma unroll
  for (int k = 1; k < NW; ++k) {
    a = MAX ? fmaxf(a, red[k]) : a + red[k];
    b = MAX ? fmaxf(b, red[16 + k]) : b + red[16 + k];
  }
}

struct TeacherShared {  // three arrays of K in dynamic LDS
  float* x;              // the student's logit at the entry
  float* q;              // the teacher's logit, then its probability
  int* at;               // its place in the row, -1: none
  __device__ __forceinline__ TeacherShared(float* mem, int K)
      : x(mem), q(mem + K), at(reinterpret_cast<int*>(mem + 2 * K)) {}
};

// The teacher's entries of a row, and the student's logits there (read here, before
// a gradient may replace them). The thread's part of the maximum; +inf where one is NaN or +inf.
template <typename T, int NW>
__device__ __forceinline__ float teacher_entries(const TeacherShared& sh, const Row<T>& row, const TeacherArgs& t, int r,
                                                 const float* sx) {
  float m = -INFINITY;
  for (int k = threadIdx.x; k < t.K; k += 64 * NW) {
    const int i = t.top[(int64_t)r * t.K + k];
    const float v = t.val[(int64_t)r * t.K + k];
    const int64_t j = (int64_t)i - row.first;
    const bool have = i >= 0 && j >= 0 && j < row.cnt;
    sh.at[k] = have ? (int)j : -1;
    sh.q[k] = have ? v : -INFINITY;
    sh.x[k] = sx ? sx[k] : have ? row.at((int)j) : -INFINITY;
    m = fmaxf(m, sh.q[k]);
    if (have && !(v < INFINITY)) m = INFINITY;
  }
  return m;
}
// The thread's part of the teacher's sum of exponentials, m its maximum.
template <int NW>
__device__ __forceinline__ float teacher_sum(const TeacherShared& sh, int K, float m, float inv_temp) {
  float s = 0.f;
  const ScaledExp<float> ex(inv_temp);
  for (int k = threadIdx.x; k < K; k += 64 * NW) s += m > -INFINITY ? ex(sh.q[k] - m) : 0.f;
  return s;
}
// The thread's part of the loss; sh.q becomes q. mt, qs: the teacher's maximum and its sum of
// exponentials (mt = +inf makes all that follows NaN); ms, ls: the student's maximum and its sum's log.
template <int NW>
__device__ __forceinline__ float teacher_loss(const TeacherShared& sh, int K, float mt, float qs, float ms, float ls,
                                              float inv_temp) {
  float loss = 0.f;
  const ScaledExp<float> ex(inv_temp);
  const float lt = logf(qs);
  for (int k = threadIdx.x; k < K; k += 64 * NW) {
    const float d = sh.q[k] - mt, lq = fmaf(d, inv_temp, -lt), q = sh.at[k] >= 0 ? ex(d) / qs : 0.f;
    sh.q[k] = q;
    // (q first: log p of a mask of the type's lowest value may be beyond fp32 where q log p is not)
    if (q != 0.f) loss += fmaf(q * (sh.x[k] - ms), -inv_temp, q * (lq + ls));
  }
  return loss;
}

// Whether an entry of the list stands at another one's place, as far as this thread looks: the pairs
// are shared out over the workgroup.
template <int TB>
__device__ __forceinline__ bool teacher_twice(const TeacherShared& sh, int K) {
  const int slices = max(TB / K, 1), s = (int)threadIdx.x / K;
  bool twice = false;
  if (s < slices)
    for (int k = threadIdx.x - s * K; k < K; k += TB) {
      const int at = sh.at[k];
      for (int j = s; j < k; j += slices) twice |= at >= 0 && sh.at[j] == at;
    }
  return twice;
}
// Entry k of the list, if it is the first of its place: all the teacher's
// probability there. `twice`: there are entries at the place of others.
__device__ __forceinline__ bool teacher_place(const TeacherShared& sh, int K, int k, bool twice, float& q) {
  const int at = sh.at[k];
  bool first = at >= 0;
  q = sh.q[k];
  if (!twice) return first;
  q = 0.f;
  for (int j = 0; j < K; ++j) {
    const bool same = sh.at[j] == at;
    if (same) q += sh.q[j];
    first = first && !(same && j < k);
  }
  return first;
}

__device__ __forceinline__ void st_grad(float* p, float v) { *p = v; }
__device__ __forceinline__ void st_grad(uint16_t* p, float v) { *p = f32_to_bf16(v); }

// Gradient vector v of a row out of its raw logits, f(x) each.
template <typename T, typename F>
__device__ __forceinline__ void grad_vec(const Row<T>& row, T* g, bool same, int v, u32x4 x, F f) {
  constexpr int VE = Row<T>::VE;
  if (same && row.whole(v)) {
    u32x4 o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __float_as_uint(f(__uint_as_float(x[i])));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = f32x2_to_bf16x2(f(Row<T>::get(x, 2 * i)), f(Row<T>::get(x, 2 * i + 1)));
    }
    *reinterpret_cast<u32x4*>(g + (v * VE - row.h)) = o;
    return;
  }
#pragma unroll
  for (int i = 0; i < VE; ++i) {
    const int j = v * VE - row.h + i;
    if (j >= 0 && j < row.cnt) st_grad(g + j, f(Row<T>::get(x, i)));
  }
}

template <typename T>
__device__ __forceinline__ T* grad_row(const LogitRows& a, const TeacherArgs& t, int r) {
  return static_cast<T*>(t.grad) + (a.offs ? (int64_t)a.offs[r] : (int64_t)r * t.ldg);
}
template <typename T>
__device__ __forceinline__ bool same_phase(const Row<T>& row, const T* g) {
  return (int)((reinterpret_cast<uintptr_t>(g) / sizeof(T)) % Row<T>::VE) == row.h;
}

// One workgroup per row, the row's NV x 64 NW vectors held in registers from the one
// time they are read until the gradient leaves; of longer rows the rest is read
// again for each of the three passes. Bound by HBM: each entry read and written once; 2,048 rows of
// 131,072 bf16 entries in 251 us, 230 at the rate of a copy; 1,024 of 131,072 fp32 ones, half of which the
// registers hold, in 338.
template <typename T, int NW, int NV>
__global__ __launch_bounds__(64 * NW) void distill_row_kernel(LogitRows a, TeacherArgs t) {
  constexpr int VE = Row<T>::VE, TB = 64 * NW;
  extern __shared__ __attribute__((aligned(16))) float teacher_mem[];
  __shared__ float red[3][32];
  __shared__ int twice;
  TeacherShared sh(teacher_mem, t.K);
  if (threadIdx.x == 0) twice = 0;
  const int r = blockIdx.x, tid = threadIdx.x;
  const Row<T> row(a, r);
  const ScaledExp<T> ex(a.inv_temp);
  u32x4 x[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) x[k] = tid + k * TB < row.nvec ? row.load(tid + k * TB) : u32x4{0, 0, 0, 0};
  float mt = teacher_entries<T, NW>(sh, row, t, r, nullptr);
  float m = -INFINITY;
  auto vmax = [&](u32x4 v) {
#pragma unroll
    for (int i = 0; i < VE; ++i) m = fmaxf(m, Row<T>::get(v, i));
  };
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (tid + k * TB < row.nvec) vmax(x[k]);
  for (int v = tid + NV * TB; v < row.nvec; v += TB) vmax(row.load(v));
  // Between the passes the logits are opaque: else the compiler holds what one pass made of them (widened
  // values, differences, exponentials) for the next, beside them, up to 1 KB of spills per lane.
  auto hold = [&]() {
#pragma unroll
    for (int k = 0; k < NV; ++k) asm volatile("" : "+v"(x[k]));
  };
  block_reduce<NW, true>(m, mt, red[0]);
  if (NW < 16) hold();  // (at 1,024 threads, 128 registers, one (bf16) and four (fp32) are spilled so, six and three with it)
  if (t.grad && teacher_twice<TB>(sh, t.K)) twice = 1;
  if (!(m > -INFINITY)) m = 0.f;  // nothing but -inf (a sum of 0) or NaN (a sum of NaN)
  float s = 0.f, qs = teacher_sum<NW>(sh, t.K, mt, a.inv_temp);
  auto vsum = [&](u32x4 v) {
#pragma unroll
    for (int i = 0; i < VE; ++i) s += ex(Row<T>::get(v, i) - m);
  };
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (tid + k * TB < row.nvec) vsum(x[k]);
  for (int v = tid + NV * TB; v < row.nvec; v += TB) vsum(row.load(v));
  block_reduce<NW, false>(s, qs, red[1]);
  const bool live = mt > -INFINITY && s != 0.f;
  hold();
  float loss = teacher_loss<NW>(sh, t.K, mt, qs, m, logf(s), a.inv_temp), none = 0.f;
  block_reduce<NW, false>(loss, none, red[2]);
  if (tid == 0) t.loss[r] = live ? loss : 0.f;
  if (!t.grad) return;
  T* g = grad_row<T>(a, t, r);
  const bool same = same_phase(row, g);
  const float w = live ? (t.weight ? t.weight[r] : 1.f) * a.inv_temp : 0.f, ws = w / s;
  auto f = [&](float v) { return live ? ex(v - m) * ws : 0.f; };
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (tid + k * TB < row.nvec) grad_vec(row, g, same, tid + k * TB, x[k], f);
  for (int v = tid + NV * TB; v < row.nvec; v += TB) grad_vec(row, g, same, v, row.load(v), f);
  if (!live) return;
  __syncthreads();  // the entries below are written after the ones above
  for (int k = tid; k < t.K; k += TB) {
    float q;
    if (teacher_place(sh, t.K, k, twice != 0, q)) st_grad(g + sh.at[k], f(sh.x[k]) - w * q);
  }
}

// Few long rows: each is split over gridDim.y workgroups, once for the sums, and
// once more (out of the caches) for the gradient. The student's logits at the teacher's
// entries wait in the workspace meanwhile, as the gradient may replace them.
template <typename T>
__global__ __launch_bounds__(kTB) void distill_sums_kernel(LogitRows a, TeacherArgs t, Stats* __restrict__ part,
                                                           float* __restrict__ sx) {
  constexpr int VE = Row<T>::VE;
  __shared__ float red[2][32];
  const int r = blockIdx.x, tid = threadIdx.x;
  const Row<T> row(a, r);
  const int per = (row.nvec + gridDim.y - 1) / gridDim.y;
  const int v0 = min((int)blockIdx.y * per, row.nvec), v1 = min(v0 + per, row.nvec);
  const ScaledExp<T> ex(a.inv_temp);
  float m = -INFINITY, s = 0.f;
  constexpr int U = 4;
  for (int vb = v0 + tid; vb < v1; vb += U * kTB) {
    u32x4 x[U];
#pragma unroll
    for (int k = 0; k < U; ++k)
      if (vb + k * kTB < v1) x[k] = row.load(vb + k * kTB);
    float nm = m;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (vb + k * kTB >= v1) break;
#pragma unroll
      for (int i = 0; i < VE; ++i) nm = fmaxf(nm, Row<T>::get(x[k], i));
    }
    if (nm > m) {
      s = m > -INFINITY ? s * ex(m - nm) : s;
      m = nm;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (vb + k * kTB >= v1) break;
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        s += ex(Row<T>::get(x[k], i) - (m > -INFINITY ? m : 0.f));
      }
    }
  }
  float bm = m, none = 0.f;
  block_reduce<kTB / 64, true>(bm, none, red[0]);
  s = m > -INFINITY ? s * ex(m - bm) : s;
  block_reduce<kTB / 64, false>(s, none, red[1]);
  if (tid == 0) part[(int64_t)r * gridDim.y + blockIdx.y] = Stats{bm, s, 0.f};
  if (blockIdx.y == 0)
    for (int k = tid; k < t.K; k += kTB) {
      const int i = t.top[(int64_t)r * t.K + k];
      const int64_t j = (int64_t)i - row.first;
      sx[(int64_t)r * t.K + k] = i >= 0 && j >= 0 && j < row.cnt ? row.at((int)j) : -INFINITY;
    }
}

template <typename T>
__global__ __launch_bounds__(kTB) void distill_grad_kernel(LogitRows a, TeacherArgs t,
                                                           const Stats* __restrict__ part,
                                                           const float* __restrict__ sx) {
  constexpr int VE = Row<T>::VE, NW = kTB / 64;
  extern __shared__ __attribute__((aligned(16))) float teacher_mem[];
  __shared__ float red[3][32];
  __shared__ int twice;
  TeacherShared sh(teacher_mem, t.K);
  if (threadIdx.x == 0) twice = 0;
  const int r = blockIdx.x, tid = threadIdx.x, S = gridDim.y;
  const Row<T> row(a, r);
  const int per = (row.nvec + S - 1) / S;
  const int v0 = min((int)blockIdx.y * per, row.nvec), v1 = min(v0 + per, row.nvec);
  const ScaledExp<T> ex(a.inv_temp);
  float mt = teacher_entries<T, NW>(sh, row, t, r, sx + (int64_t)r * t.K);
  float m = -INFINITY, s = 0.f, none = 0.f;
  for (int k = 0; k < S; ++k) m = fmaxf(m, part[(int64_t)r * S + k].m);
  for (int k = 0; k < S; ++k) {
    const Stats p = part[(int64_t)r * S + k];
    s += p.m > -INFINITY ? p.s * ex(p.m - m) : p.s;
  }
  if (!(m > -INFINITY)) m = 0.f;
  block_reduce<NW, true>(mt, none, red[0]);
  if (t.grad && teacher_twice<kTB>(sh, t.K)) twice = 1;
  const bool live = mt > -INFINITY && s != 0.f;
  float qs = teacher_sum<NW>(sh, t.K, mt, a.inv_temp);
  block_reduce<NW, false>(qs, none, red[1]);
  float loss = teacher_loss<NW>(sh, t.K, mt, qs, m, logf(s), a.inv_temp);
  block_reduce<NW, false>(loss, none, red[2]);
  if (blockIdx.y == 0 && tid == 0) t.loss[r] = live ? loss : 0.f;
  if (!t.grad) return;
  T* g = grad_row<T>(a, t, r);
  const bool same = same_phase(row, g);
  const float w = live ? (t.weight ? t.weight[r] : 1.f) * a.inv_temp : 0.f, ws = w / s;
  auto f = [&](float v) { return live ? ex(v - m) * ws : 0.f; };
  for (int v = v0 + tid; v < v1; v += kTB) grad_vec(row, g, same, v, row.load(v), f);
  if (!live) return;
  __syncthreads();
  const int lo = v0 * VE - row.h, hi = v1 * VE - row.h;  // the entries of this part
  for (int k = tid; k < t.K; k += kTB) {
    float q;
    if (sh.at[k] >= lo && sh.at[k] < hi && teacher_place(sh, t.K, k, twice != 0, q))
      st_grad(g + sh.at[k], f(sh.x[k]) - w * q);
  }
}

// Parts of a row: one while the rows alone give every CU four workgroups, else
// enough for that, of 512 vectors (two per thread) at least. 4 rows of 50,001 fp32 logits:
// 24 parts and their join 14 us, one workgroup of 1,024 threads a row 18.
int row_splits(int n, int V) {
  const int vecs = V / 4 + 1;
  const int want = std::max(1, 1024 / std::max(n, 1));
  return std::max(1, std::min({want, vecs / 512, 64}));
}
// Distillation takes two passes over a split row instead of one in registers, so a row
// is split from where the registers of a workgroup do not hold it. 16 rows of 4,096 fp32
// logits: 11 us whole, 18 in two parts. (Of bf16 the registers hold twice as many; one rule, as a
// workspace's size does not depend on the type.)
int distill_splits(int n, int V) { return V / 4 + 1 <= 16 * 1024 ? 1 : row_splits(n, V); }

template <typename T>
hipError_t logprobs(const LogitRows& a, int K, const LogprobOut& o, char* ws, hipStream_t s) {
  // Up to 16 vectors per thread a row is not worth the second launch: 64 of 12,000 fp32 logits, K 20,
  // 12 us whole, 16 split; 8 of 30,000 in bf16, K 5, 13 and 15, in fp32 (30 vectors) 14 and 14.
  const int S = a.V / Row<T>::VE < 16 * kTB ? 1 : row_splits(a.n, a.V);
  // Many short rows: one wavefront each, or two for more top entries than half its lanes. 65,536 bf16 rows of
  // 2,048, K 20: 137 us, with kTB threads 308; 8,192 of 16,384 72 with one wavefront, 76 with kTB.
  if (S == 1 && a.n >= 256 && a.V <= 8192 && K <= 32) logprobs_kernel<T, 64><<<dim3(a.n), 64, 0, s>>>(a, K, o, ws);
  else if (S == 1 && a.n >= 256 && a.V <= 8192) logprobs_kernel<T, 128><<<dim3(a.n), 128, 0, s>>>(a, K, o, ws);
  else logprobs_kernel<T, kTB><<<dim3(a.n, S), kTB, 0, s>>>(a, K, o, ws);
  if (S > 1) logprobs_join_kernel<T><<<dim3(a.n), kTB, 0, s>>>(a, K, S, o, ws);
  return hipGetLastError();
}

// The rows' lists as logprobs() has them, then one workgroup per group, which joins few lists faster: a row is split
// from where one workgroup does not read all of it at once (256 rows of 16,000 bf16 entries 18.4 us a call, split in
// two 19.8; for 4 to 32 rows the host's part of a call hides either). A wavefront per row as in logprobs() pays from
// 2,048 rows: 4,096 rows of 4,096 29 us against 37, 1,024 rows of 8,192 18.1 against 17.4, 256 rows 19.8 against 17.2.
int beam_splits(int n, int W, int V) { return std::min(V / 4 + 1 <= 16 * kTB ? 1 : row_splits(n, V), kBeamLists / W); }

template <typename T>
hipError_t beam_select(const LogitRows& a, int W, int K, const Beams& beams, int* parent, int* token, float* out_score,
                       char* ws, hipStream_t s) {
  const int S = beam_splits(a.n, W, a.V);
  const LogprobOut o = {};
  if (S == 1 && a.n >= 2048 && a.V <= 8192 && K <= 32)
    logprobs_kernel<T, 64, true><<<dim3(a.n), 64, 0, s>>>(a, K, o, ws, beams);
  else
    logprobs_kernel<T, kTB, true><<<dim3(a.n, S), kTB, 0, s>>>(a, K, o, ws, beams);
  beam_join_kernel<T><<<dim3(a.n / W), kTB, 0, s>>>(a, W, K, S, beams, parent, token, out_score, ws);
  return hipGetLastError();
}

template <typename T>
hipError_t distill(const LogitRows& a, const TeacherArgs& t, char* ws, hipStream_t s) {
  const int S = distill_splits(a.n, a.V);
  if (S > 1) {
    Stats* part = reinterpret_cast<Stats*>(ws);
    float* sx = reinterpret_cast<float*>(ws + (size_t)a.n * S * sizeof(Stats));
    distill_sums_kernel<T><<<dim3(a.n, S), kTB, 0, s>>>(a, t, part, sx);
    distill_grad_kernel<T><<<dim3(a.n, S), kTB, 12 * t.K, s>>>(a, t, part, sx);
    return hipGetLastError();
  }
  const int vecs = a.V / Row<T>::VE + (a.V % Row<T>::VE != 0);
  if (vecs <= 64 * 4) distill_row_kernel<T, 1, 4><<<dim3(a.n), 64, 12 * t.K, s>>>(a, t);
  else if (vecs <= 256 * 4) distill_row_kernel<T, 4, 4><<<dim3(a.n), 256, 12 * t.K, s>>>(a, t);
  else if (vecs <= 512 * 8) distill_row_kernel<T, 8, 8><<<dim3(a.n), 512, 12 * t.K, s>>>(a, t);
  else if (vecs <= 512 * 16) distill_row_kernel<T, 8, 16><<<dim3(a.n), 512, 12 * t.K, s>>>(a, t);
  else distill_row_kernel<T, 16, 16><<<dim3(a.n), 1024, 12 * t.K, s>>>(a, t);
  return hipGetLastError();
}

}  // namespace

size_t logits_workspace_bytes(int n, int V, int K) {
  const int S = row_splits(n, V), D = distill_splits(n, V);
  const size_t lp = S > 1 ? (size_t)n * S * (K * 8 + 16) : 0;
  const size_t di = D > 1 ? (size_t)n * D * sizeof(Stats) + (size_t)n * K * sizeof(float) : 0;
  return std::max(lp, di);
}

hipError_t launch_logprobs(const LogitRows& a, const int* tokens, int K, float* logp, float* entropy, int* top,
                           float* top_logp, void* ws, hipStream_t s) {
  const LogprobOut o = {tokens, logp, entropy, top, top_logp};
  return a.bf16 ? logprobs<uint16_t>(a, K, o, static_cast<char*>(ws), s)
                : logprobs<float>(a, K, o, static_cast<char*>(ws), s);
}

hipError_t launch_distill_topk(const LogitRows& a, int K, const int* top, const float* teacher, const float* weight,
                               float* loss, void* grad, int64_t ldg, void* ws, hipStream_t s) {
  const TeacherArgs t = {K, top, teacher, weight, loss, grad, ldg};
  return a.bf16 ? distill<uint16_t>(a, t, static_cast<char*>(ws), s) : distill<float>(a, t, static_cast<char*>(ws), s);
}

size_t beam_select_workspace_bytes(int groups, int W, int V, int K) {
  const int n = groups * W;
  return (size_t)n * beam_splits(n, W, V) * (K * 8 + 16);
}

hipError_t launch_beam_select(const LogitRows& a, int W, int K, const float* score, const int* ended, int* parent,
                              int* token, float* out_score, void* ws, hipStream_t s) {
  const Beams b = {score, ended};
  return a.bf16 ? beam_select<uint16_t>(a, W, K, b, parent, token, out_score, static_cast<char*>(ws), s)
                : beam_select<float>(a, W, K, b, parent, token, out_score, static_cast<char*>(ws), s);
}

}  // namespace tcl

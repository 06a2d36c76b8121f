// The causal convolution and the selective scan as operators of their own,
// with states carried over: prompts (packed sequences), single tokens, and
// their gradients.
// Work along the rows is cut into tiles of R rows (packing.h).
#include <algorithm>

#include "common.h"
#include "ops.h"
#include "packing.h"

namespace tcl {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void st1(float* p, float v) { *p = v; }
__device__ __forceinline__ void st1(uint16_t* p, float v) { *p = f32_to_bf16(v); }

// Element of a wave-uniform row at a lane's byte offset, addressed as scalar base
// plus 32-bit lane offset. Left to itself the compiler adds the lane's part to the matrix's
// base once and the row's part per access, which costs a 64-bit vector sum and a
// register pair each (100 registers of the gradient kernel); readfirstlane keeps the row's
// address a scalar value of its own.
typedef __attribute__((address_space(1))) char gchar;
template <typename T>
__device__ __forceinline__ gchar* scalar_row(const T* row) {
  const uint64_t p = reinterpret_cast<uint64_t>(row);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32));
  return (gchar*)((uint64_t)hi << 32 | lo);
}
// (and the lane's part a 32-bit value at each access)
__device__ __forceinline__ uint32_t lane_part(uint32_t bytes) {
  asm("" : "+v"(bytes));
  return bytes;
}
template <typename T>
__device__ __forceinline__ T ld_at(const T* row, uint32_t bytes) {
  return *(const __attribute__((address_space(1))) T*)(scalar_row(row) + lane_part(bytes));
}
__device__ __forceinline__ void st_at(float* row, uint32_t bytes, float v) {
  *(__attribute__((address_space(1))) float*)(scalar_row(row) + lane_part(bytes)) = v;
}
__device__ __forceinline__ void st_at(uint16_t* row, uint32_t bytes, float v) {
  *(__attribute__((address_space(1))) uint16_t*)(scalar_row(row) + lane_part(bytes)) = f32_to_bf16(v);
}
// N consecutive floats there, N a multiple of 4.
template <int N>
__device__ __forceinline__ void ld_vec(const float* row, uint32_t bytes, float* v) {
#pragma unroll
  for (int n = 0; n < N; n += 4) {
    const floatx4 x = *reinterpret_cast<const floatx4*>(reinterpret_cast<const char*>(row) + bytes + 4 * n);
    v[n] = x.x; v[n + 1] = x.y; v[n + 2] = x.z; v[n + 3] = x.w;
  }
}
template <int N>
__device__ __forceinline__ void st_vec(float* row, uint32_t bytes, const float* v) {
#pragma unroll
  for (int n = 0; n < N; n += 4)
    *reinterpret_cast<floatx4*>(reinterpret_cast<char*>(row) + bytes + 4 * n) = floatx4{v[n], v[n + 1], v[n + 2], v[n + 3]};
}

// CH adjacent channels of a row; the storage type's raw bits, widened at use.
template <typename T, int CH> struct Pack { T v[CH]; };
template <> struct Pack<float, 4> { floatx4 v; };
template <> struct Pack<uint16_t, 4> { u32x2 v; };

template <typename T, int CH>
__device__ __forceinline__ Pack<T, CH> pk_load(const T* p) {
  return *reinterpret_cast<const Pack<T, CH>*>(p);
}
template <typename T, int CH>
__device__ __forceinline__ float pk_get(const Pack<T, CH>& p, int i) {
  if constexpr (CH == 1 || sizeof(T) == 4)
    return to_f32(p.v[i]);
  else
    return __uint_as_float(i & 1 ? p.v[i >> 1] & 0xFFFF0000u : p.v[i >> 1] << 16);
}
template <typename T, int CH>
__device__ __forceinline__ void pk_store(T* p, const float* v) {
  if constexpr (CH == 1) {
    st1(p, v[0]);
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<floatx4*>(p) = floatx4{v[0], v[1], v[2], v[3]};
  } else {
    Pack<T, CH> o;
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) o.v[i] = f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<Pack<T, CH>*>(p) = o;
  }
}

// ---------------------------------------------------------------- causal conv + SiLU
// u_t = SiLU(b + sum_k w_k x_{t-K+1+k}). A thread takes CH adjacent channels
// (four: 16 bytes in fp32; 8 in bf16, where eight would halve the wavefronts in
// flight) of one tile and keeps the last K rows in registers; rows in front of
// the tile are read again (K - 1 of R), those in front of the sequence come
// from its state. The thread of the first tile is also the one that writes
// the new state, after it has read the old one, so both may be the same
// memory. Bound by HBM: each x read once, each u written once; 20,415 rows of 4,096
// bf16 channels in 68 us (4.9 TB/s, a part out of the cache; 72 at the rate of a copy; a fifth more with
// eight channels a thread), one token of 256 sequences in 7.2 (3.6 at the rate of a copy: a thread's weights
// are as many bytes as its rows and states).
template <typename T, int K, int CH>
__global__ __launch_bounds__(256) void ssm_conv_kernel(const int* __restrict__ offs, int n_seq, int rows, int E,
                                                       int R, int64_t n_work, const T* __restrict__ x, int64_t ldx,
                                                       const float* __restrict__ w, const float* __restrict__ b,
                                                       const T* state, const int* __restrict__ slots, int n_slots,
                                                       T* state_out, T* __restrict__ u, int64_t ldu) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= n_work) return;
  const int CG = E / CH;
  const int e = (int)(id % CG) * CH;
  const Tile tl = find_tile(offs, n_seq, rows, R, (int)(id / CG));
  if (tl.seq < 0) return;
  const T* xs = x + (int64_t)tl.base * ldx + e;
  const int t0 = tl.j * R, t1 = min(t0 + R, tl.len);

  float wk[K][CH], bias[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    bias[c] = b ? b[e + c] : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) wk[k][c] = w[(int64_t)(e + c) * K + k];
  }
  // win[k] = x_{t-K+1+k}; the slot K - 1 is the token's own
  float win[K][CH];
  if constexpr (K > 1) {
    if (tl.j == 0) {
      const int sl = slot_of(slots, n_slots, tl.seq);
      const int64_t so = (int64_t)sl * (K - 1) * E + e;
#pragma unroll
      for (int k = 0; k < K - 1; ++k) {
#pragma unroll
        for (int c = 0; c < CH; ++c) win[k][c] = 0.f;
        if (state && sl >= 0) {
          const Pack<T, CH> p = pk_load<T, CH>(state + so + (int64_t)k * E);
#pragma unroll
          for (int c = 0; c < CH; ++c) win[k][c] = pk_get(p, c);
        }
      }
      if (state_out && sl >= 0) {
        // the last K - 1 rows of (old state, tokens)
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
          const int t = tl.len - (K - 1) + k;
          float v[CH];
          if (t >= 0) {
            const Pack<T, CH> p = pk_load<T, CH>(xs + (int64_t)t * ldx);
#pragma unroll
            for (int c = 0; c < CH; ++c) v[c] = pk_get(p, c);
          } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) v[c] = 0.f;
#pragma unroll
            for (int i = 0; i < K - 1; ++i)
              if (i == K - 1 + t)
#pragma unroll
                for (int c = 0; c < CH; ++c) v[c] = win[i][c];
          }
          pk_store<T, CH>(state_out + so + (int64_t)k * E, v);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < K - 1; ++k) {  // R >= K - 1: these rows are the sequence's
        const Pack<T, CH> p = pk_load<T, CH>(xs + (int64_t)(t0 - (K - 1) + k) * ldx);
#pragma unroll
        for (int c = 0; c < CH; ++c) win[k][c] = pk_get(p, c);
      }
    }
  }
  T* us = u + (int64_t)tl.base * ldu + e;
  constexpr int U = 4;  // rows whose loads are in flight together
  Pack<T, CH> nx[U];
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (t0 < t1) nx[i] = pk_load<T, CH>(xs + (int64_t)min(t0 + i, t1 - 1) * ldx);
  for (int t = t0; t < t1; t += U) {
    Pack<T, CH> cur[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      cur[i] = nx[i];
      if (t + U < t1) nx[i] = pk_load<T, CH>(xs + (int64_t)min(t + U + i, t1 - 1) * ldx);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (t + i >= t1) break;
      float o[CH];
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        win[K - 1][c] = pk_get(cur[i], c);
        float v = bias[c];
#pragma unroll
        for (int k = 0; k < K; ++k) v = fmaf(wk[k][c], win[k][c], v);
        o[c] = silu(v);
#pragma unroll
        for (int k = 0; k < K - 1; ++k) win[k][c] = win[k + 1][c];
      }
      pk_store<T, CH>(us + (int64_t)(t + i) * ldu, o);
    }
  }
}

// SiLU'(x) = sg (1 + x (1 - sg)), sg = sigmoid(x).
__device__ __forceinline__ float silu_grad(float x) {
  const float sg = rcp_fast(1.0f + exp_fast(-x));
  return sg * fmaf(x, 1.0f - sg, 1.0f);
}

// Gradients of the convolution. With g_t = du_t SiLU'(pre_t):
//   dx_t = sum_k w_k g_{t+K-1-k},  dw_k = sum_t g_t x_{t-K+1+k},  db = sum_t g_t
// and the state's rows are the x_t of t < 0. A thread takes CH channels of
// `per` tiles in a row; in each it walks forward over the tile's rows and the
// K - 1 behind it, forming pre and g again there, so that dx leaves complete and
// nothing passes between threads. dw and db stay in registers over its tiles
// and go out once, as part `p` of the partial sums. 20,415 rows of 4,096 bf16 channels in 120 us, 108 at
// the rate of a copy; 44 issue slots per 64 entries (by the counters) are 94 us by themselves. (Two channels a
// thread: 13% longer.) With K = 4 an fp32 thread holds 134 registers, three wavefronts to a SIMD, a bf16 one 122, four.
template <typename T, int K, int CH>
__global__ __launch_bounds__(256) void ssm_conv_bwd_kernel(
    const int* __restrict__ offs, int n_seq, int rows, int E, int R, int per, int parts, const T* __restrict__ x,
    int64_t ldx, const float* __restrict__ w, const float* __restrict__ b, const T* __restrict__ state,
    const T* __restrict__ du, int64_t lddu, const T* __restrict__ dstate_out, T* __restrict__ dx, int64_t lddx,
    T* __restrict__ dstate, float* __restrict__ part) {
  const int CG = E / CH;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= (int64_t)parts * CG) return;
  const int p = (int)(id / CG), e = (int)(id % CG) * CH;
  float wk[K][CH], bias[CH], dw[K][CH], db[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    bias[c] = b ? b[e + c] : 0.f;
    db[c] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      wk[k][c] = w[(int64_t)(e + c) * K + k];
      dw[k][c] = 0.f;
    }
  }
  for (int q = 0; q < per; ++q) {
    const Tile tl = find_tile(offs, n_seq, rows, R, p * per + q);
    if (tl.seq < 0) continue;
    const int t0 = tl.j * R, t1 = min(t0 + R, tl.len);
    const T* xs = x + (int64_t)tl.base * ldx + e;
    const T* dus = du + (int64_t)tl.base * lddu + e;
    T* dxs = dx + (int64_t)tl.base * lddx + e;
    const int64_t so = (int64_t)tl.seq * (K - 1) * E + e;
    float win[K][CH], g[K][CH];  // x_{t-K+1+k}; g[k] = g_{t-K+1+k}
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        win[k][c] = 0.f;
        g[k][c] = 0.f;
      }
      if (k < K - 1) {
        const T* src = nullptr;
        if (tl.j > 0) src = xs + (int64_t)(t0 - (K - 1) + k) * ldx;
        else if (state) src = state + so + (int64_t)k * E;
        if (src) {
          const Pack<T, CH> v = pk_load<T, CH>(src);
#pragma unroll
          for (int c = 0; c < CH; ++c) win[k][c] = pk_get(v, c);
        }
      }
    }
    // rows t0 .. t1 + K - 2; those past the sequence have g = 0
    const int tend = t1 + K - 1;
    constexpr int U = 2;
    Pack<T, CH> nx[U], nd[U];
    auto load = [&](int t) {
      if (tl.len == 0) return;
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = min(t + i, tl.len - 1);
        nx[i] = pk_load<T, CH>(xs + (int64_t)r * ldx);
        nd[i] = pk_load<T, CH>(dus + (int64_t)r * lddu);
      }
    };
    load(t0);
    for (int tb = t0; tb < tend; tb += U) {
      Pack<T, CH> cx[U], cd[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        cx[i] = nx[i];
        cd[i] = nd[i];
      }
      if (tb + U < tend) load(tb + U);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int t = tb + i;
        if (t >= tend) break;
        const bool in = t < tl.len, mine = t < t1;
        const int td = t - (K - 1);  // the row whose dx is complete with this one
        const bool out = td >= t0 || (tl.j == 0 && td < 0);
        float o[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          win[K - 1][c] = in ? pk_get(cx[i], c) : 0.f;
          float v = bias[c];
#pragma unroll
          for (int k = 0; k < K; ++k) v = fmaf(wk[k][c], win[k][c], v);
          const float gt = in ? pk_get(cd[i], c) * silu_grad(v) : 0.f;
          g[K - 1][c] = gt;
          if (mine) {
            db[c] += gt;
#pragma unroll
            for (int k = 0; k < K; ++k) dw[k][c] = fmaf(gt, win[k][c], dw[k][c]);
          }
          float d = 0.f;
#pragma unroll
          for (int k = 0; k < K; ++k) d = fmaf(wk[k][c], g[K - 1 - k][c], d);
          o[c] = d;
#pragma unroll
          for (int k = 0; k < K - 1; ++k) {
            win[k][c] = win[k + 1][c];
            g[k][c] = g[k + 1][c];
          }
        }
        if (!out) continue;
        const int k = td - (tl.len - (K - 1));  // the row of the new state that td is
        if (dstate_out && k >= 0) {
          const Pack<T, CH> v = pk_load<T, CH>(dstate_out + so + (int64_t)k * E);
#pragma unroll
          for (int c = 0; c < CH; ++c) o[c] += pk_get(v, c);
        }
        if (td >= 0) pk_store<T, CH>(dxs + (int64_t)td * lddx, o);
        else if (dstate) pk_store<T, CH>(dstate + so + (int64_t)(K - 1 + td) * E, o);
      }
    }
  }
  float* o = part + (int64_t)p * (K + 1) * E + e;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int k = 0; k < K; ++k) o[(int64_t)k * E + c] = dw[k][c];
    o[(int64_t)K * E + c] = db[c];
  }
}

// Sums of `parts` partial vectors part[p][M + extra][E] in a fixed order, laid out as
// the parameters are: o0[e, m] for m < M, then o1[e], o2[e] (null: not wanted).
constexpr int kSumLanes = 16;
template <int U>  // loads in flight: a trip is one latency
__global__ __launch_bounds__(64 * kSumLanes) void sum_parts_kernel(const float* __restrict__ part, int parts, int M,
                                                                   int total, int E, float* __restrict__ o0,
                                                                   float* __restrict__ o1, float* __restrict__ o2) {
  __shared__ float red[kSumLanes][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int64_t i = (int64_t)blockIdx.x * 64 + lane, stride = (int64_t)total * E;
  float acc = 0.f;
  if (i < stride) {
    const float* src = part + i;
    for (int p = g; p < parts; p += U * kSumLanes) {
      float v[U];
#pragma unroll
      for (int k = 0; k < U; ++k) v[k] = src[min(p + k * kSumLanes, parts - 1) * stride];
#pragma unroll
      for (int k = 0; k < U; ++k) acc += p + k * kSumLanes < parts ? v[k] : 0.f;
    }
  }
  red[g][lane] = acc;
  __syncthreads();
  if (g || i >= stride) return;
  acc = 0.f;
#pragma unroll
  for (int k = 0; k < kSumLanes; ++k) acc += red[k][lane];
  const int m = (int)(i / E), e = (int)(i % E);
  if (m < M) o0[(int64_t)e * M + m] = acc;
  else if (m == M) { if (o1) o1[e] = acc; }
  else if (o2) o2[e] = acc;
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}

// ---------------------------------------------------------------- selective scan, prompts
// s_t = exp(d_t A) s_{t-1} + d_t u_t B_t,  y_t = (C_t . s_t + D u_t) SiLU(z_t),
// d = softplus(dt + b_dt), A = -exp(A_log).
// One lane per channel holds its N states and decay rates (in base-2 units);
// a workgroup is one wavefront, so nothing waits for another. B and C rows
// go through LDS kTC tokens at a time (widened once, read as broadcasts), loaded and
// waited for in front of each kTC tokens; u, dt and z come two tokens at a time, the next two
// on their way meanwhile. Per token and wavefront 6 N issue slots for the states and
// some 35 for softplus, gate and output (146 in all by the counters, on a prompt), against 4 x 64
// elements of traffic: the vector unit is what bounds it: 4,096 programs of up to 25 tokens, E 512, fp32, in 142
// us, where their traffic takes 110 and their issue slots 124 (by the counters; a sixth of them is spent once per
// sequence); a prompt of 8,032 tokens, E 4,096, bf16 in chunks 113 + 12 + 150, the last of them 122 of issue.
//
// A sequence is cut into chunks of CL tokens when there are far too few of them to
// fill the GPU (scan_chunk). s -> P s + s_loc with P = exp(A sum d) is what a chunk does to a
// state, so LOCAL runs every chunk but a sequence's last from zero for (s_loc,
// sum d), ssm_combine_kernel composes them into every chunk's start state,
// and the plain form runs the chunks from there. Twice the exponentials.
constexpr int kTC = 32;

struct ScanIn {
  const int* offs;
  int n_seq, rows, E, CL, ntile;
  int64_t ldu, lddt, ldB, ldC, ldz;
  const float *A_log, *D, *b_dt, *state;
  const int* slots;
  int n_slots;
};

// blockIdx.x -> (tile, channel group): the channel groups of a tile follow each
// other on one XCD (workgroups go to the 8 XCDs in turn), whose L2 then holds
// the tile's B and C rows.
__device__ __forceinline__ bool tile_of_block(int ntile, int CG, int& w, int& cg) {
  const int xcd = blockIdx.x & 7, j = blockIdx.x >> 3;
  w = (j / CG) * 8 + xcd;
  cg = j % CG;
  return w < ntile;
}
inline unsigned tile_blocks(int ntile, int CG) { return (unsigned)((ntile + 7) / 8 * 8) * CG; }

__device__ __forceinline__ float decay_rate(float a_log) {  // A log2(e)
  return -__builtin_amdgcn_exp2f(a_log * kLog2e) * kLog2e;
}

template <typename T, int N, bool LOCAL>
__global__ __launch_bounds__(64, 4) void ssm_scan_kernel(ScanIn a, const T* __restrict__ u, const T* __restrict__ dt,
                                                         const T* __restrict__ B, const T* __restrict__ C,
                                                         const T* __restrict__ z, float* state_out,
                                                         T* __restrict__ y, int64_t ldy, float* cst, float* csum) {
  __shared__ __attribute__((aligned(16))) float sBC[kTC * 2 * N];
  int w, cg;
  if (!tile_of_block(a.ntile, (a.E + 63) / 64, w, cg)) return;
  const Tile tl = find_tile(a.offs, a.n_seq, a.rows, a.CL, w);
  if (tl.seq < 0) return;
  const int t0 = tl.j * a.CL, t1 = min(tl.len, t0 + a.CL);
  if (LOCAL && t1 == tl.len) return;  // nobody follows
  const int lane = threadIdx.x, E = a.E;
  const int e = cg * 64 + lane;
  const bool active = e < E;
  const int ec = active ? e : E - 1;

  const uint32_t le = ec * sizeof(T), lf = ec * 4, ln = ec * N * 4;  // a lane's place in a row
  float a2[N], s[N];
  ld_vec<N>(a.A_log, ln, a2);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    a2[n] = decay_rate(a2[n]);
    s[n] = 0.f;
  }
  const int sl = slot_of(a.slots, a.n_slots, tl.seq);
  if (!LOCAL) {
    if (cst) {
#pragma unroll
      for (int n = 0; n < N; ++n) s[n] = ld_at(cst + ((int64_t)w * N + n) * E, lf);
    } else if (a.state && sl >= 0) {
      ld_vec<N>(a.state + (int64_t)sl * E * N, ln, s);
    }
  }
  const float bias = a.b_dt ? a.b_dt[ec] : 0.f, Dv = !LOCAL && a.D ? a.D[ec] : 0.f;

  if (t0 < t1) {
    const int64_t r0 = tl.base;
    const T *us = u + r0 * a.ldu, *ds = dt + r0 * a.lddt, *zs = z ? z + r0 * a.ldz : nullptr;
    const T *Bs = B + r0 * a.ldB, *Cs = LOCAL ? nullptr : C + r0 * a.ldC;
    T* ys = LOCAL ? nullptr : y + r0 * ldy;
    // A stage: lane l takes column l % W (B's, then C's; LOCAL: B's only) of every
    // RW-th row from l / W on. Rows past the end read the last one again.
    constexpr int W = LOCAL ? N : 2 * N, RW = 64 / W, PER = kTC / RW;
    const int col = lane % W;
    const bool isB = LOCAL || col < N;
    const int64_t ldS = isB ? a.ldB : a.ldC;
    const T* src = isB ? Bs + col : Cs + (col - N);
    const T* last = src + (int64_t)(t1 - 1) * ldS;
    constexpr int U = 2;
    T nu[U], nd[U], nz[U];
    auto load = [&](int t) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = min(t + i, t1 - 1);
        nu[i] = ld_at(us + r * a.ldu, le);
        nd[i] = ld_at(ds + r * a.lddt, le);
        if (!LOCAL && z) nz[i] = ld_at(zs + r * a.ldz, le);
      }
    };
    float sum = 0.f;
    load(t0);
    for (int tc = t0; tc < t1; tc += kTC) {
      T st[PER];
      const T* q = src + (tc + lane / W) * ldS;
      if (tc + kTC <= t1) {
#pragma unroll
        for (int i = 0; i < PER; ++i, q += RW * ldS) st[i] = *q;
      } else {
#pragma unroll
        for (int i = 0; i < PER; ++i, q += RW * ldS) st[i] = tc + lane / W + i * RW < t1 ? *q : *last;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PER; ++i) sBC[i * 64 + lane] = to_f32(st[i]);
      __syncthreads();
      const int te = min(t1, tc + kTC);
      for (int tg = tc; tg < te; tg += U) {
        T cu[U], cd[U], cz[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          cu[i] = nu[i];
          cd[i] = nd[i];
          if (!LOCAL && z) cz[i] = nz[i];
        }
        if (tg + U < t1) load(tg + U);
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int t = tg + i;
          if (t >= te) break;
          const float* x = &sBC[(t - tc) * W];
          const float uv = to_f32(cu[i]), d = softplus(to_f32(cd[i]) + bias), du = d * uv;
          if (LOCAL) sum += d;
          float acc = 0.f;
#pragma unroll
          for (int n = 0; n < N; ++n) {
            s[n] = fmaf(__builtin_amdgcn_exp2f(d * a2[n]), s[n], du * x[n]);
            if (!LOCAL) acc = fmaf(s[n], x[N + n], acc);
          }
          if (!LOCAL) {
            acc = fmaf(Dv, uv, acc);
            if (z) acc *= silu(to_f32(cz[i]));
            if (active) st_at(ys + t * ldy, le, acc);
          }
        }
      }
    }
    if (LOCAL && active) st_at(csum + (int64_t)w * E, lf, sum);
  }
  if (!active) return;
  if (LOCAL) {
#pragma unroll
    for (int n = 0; n < N; ++n) st_at(cst + ((int64_t)w * N + n) * E, lf, s[n]);
  } else if (state_out && sl >= 0 && t1 == tl.len) {
    st_vec<N>(state_out + (int64_t)sl * E * N, ln, s);
  }
}

// The same, for batches too small to give a SIMD two wavefronts of one lane per channel but large
// enough that cutting the sequences (twice the exponentials) would not pay: Q = N / 4 lanes per channel
// hold four states each, and a token costs a wavefront a quarter. What a token needs once
// per channel (softplus, gate, output) is done by one lane for each of Q tokens and passed round by
// DPP, so it is not done Q times: 150 issue slots per token and 64 channels against 140. Tokens past the
// end have d = 0, which leaves the states as they are.
constexpr int kQuadThreads = 256;
template <typename T, int N>
__global__ __launch_bounds__(kQuadThreads) void ssm_scan_quad_kernel(
    ScanIn a, const T* __restrict__ u, const T* __restrict__ dt, const T* __restrict__ B, const T* __restrict__ C,
    const T* __restrict__ z, float* state_out, T* __restrict__ y, int64_t ldy) {
  constexpr int Q = N / 4, W = 2 * N, CH = kQuadThreads / Q, PER = kTC * W / kQuadThreads;
  __shared__ __attribute__((aligned(16))) float sBC[kTC * W];
  int w, cg;
  if (!tile_of_block(a.ntile, (a.E + CH - 1) / CH, w, cg)) return;
  const Tile tl = find_tile(a.offs, a.n_seq, a.rows, a.CL, w);
  if (tl.seq < 0) return;
  const int E = a.E, q = threadIdx.x % Q, n0 = 4 * q;
  const int e = cg * CH + threadIdx.x / Q;
  const bool active = e < E;
  const int ec = active ? e : E - 1;
  float a2[4], s[4] = {0.f, 0.f, 0.f, 0.f};
  ld_vec<4>(a.A_log, (uint32_t)(ec * N + n0) * 4, a2);
#pragma unroll
  for (int n = 0; n < 4; ++n) a2[n] = decay_rate(a2[n]);
  const int sl = slot_of(a.slots, a.n_slots, tl.seq);
  if (a.state && sl >= 0) ld_vec<4>(a.state + (int64_t)sl * E * N, (uint32_t)(ec * N + n0) * 4, s);
  const float bias = a.b_dt ? a.b_dt[ec] : 0.f, Dv = a.D ? a.D[ec] : 0.f;
  const int len = tl.len;
  const int64_t r0 = tl.base;
  const T *us = u + r0 * a.ldu + ec, *ds = dt + r0 * a.lddt + ec, *zs = z ? z + r0 * a.ldz + ec : nullptr;
  T* ys = y + r0 * ldy + ec;
  // staging: a thread takes one column of every RW-th row
  constexpr int RW = kQuadThreads / W;
  const int col = threadIdx.x % W, row0 = threadIdx.x / W;
  const int64_t ldS = col < N ? a.ldB : a.ldC;
  const T* src = col < N ? B + r0 * a.ldB + col : C + r0 * a.ldC + (col - N);
  T st[PER], nu, nd, nz;
  auto stage = [&](int t) {
#pragma unroll
    for (int i = 0; i < PER; ++i) st[i] = src[min(t + row0 + i * RW, len - 1) * ldS];
  };
  auto load = [&](int t) {  // the lane's token of the next Q
    const int64_t r = min(t + q, len - 1);
    nu = us[r * a.ldu];
    nd = ds[r * a.lddt];
    if (z) nz = zs[r * a.ldz];
  };
  if (len > 0) {
    stage(0);
    load(0);
  }
  for (int tc = 0; tc < len; tc += kTC) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) sBC[i * kQuadThreads + threadIdx.x] = to_f32(st[i]);
    __syncthreads();
    if (tc + kTC < len) stage(tc + kTC);
    const int te = min(len, tc + kTC);
    for (int tg = tc; tg < te; tg += Q) {
      const int t = tg + q;
      const float uv = to_f32(nu), d = t < len ? softplus(to_f32(nd) + bias) : 0.f, du = d * uv;
      const float gate = z ? silu(to_f32(nz)) : 1.f;
      if (tg + Q < len) load(tg + Q);
      float mine = 0.f;
      auto token = [&](int i, float di, float dui) {
        const float* x = &sBC[(tg - tc + i) * W + n0];
        float xb[4], xc[4], acc = 0.f;
        ld_vec<4>(x, 0, xb);
        ld_vec<4>(x + N, 0, xc);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          s[n] = fmaf(__builtin_amdgcn_exp2f(di * a2[n]), s[n], dui * xb[n]);
          acc = fmaf(s[n], xc[n], acc);
        }
        acc += dpp<0xB1>(acc);                 // quad_perm: lane ^ 1
        if (Q == 4) acc += dpp<0x4E>(acc);     // lane ^ 2
        if (q == i) mine = acc;
      };
      if constexpr (Q == 4) {  // quad_perm: lane i's value to all four
        token(0, dpp<0x00>(d), dpp<0x00>(du));
        token(1, dpp<0x55>(d), dpp<0x55>(du));
        token(2, dpp<0xAA>(d), dpp<0xAA>(du));
        token(3, dpp<0xFF>(d), dpp<0xFF>(du));
      } else {  // the even (odd) lane's value to its pair
        token(0, dpp<0xA0>(d), dpp<0xA0>(du));
        token(1, dpp<0xF5>(d), dpp<0xF5>(du));
      }
      if (active && t < len) st1(ys + t * ldy, fmaf(Dv, uv, mine) * gate);
    }
  }
  if (active && state_out && sl >= 0) st_vec<4>(state_out + (int64_t)sl * E * N, (uint32_t)(ec * N + n0) * 4, s);
}

// Every chunk's start state out of the chunks' (s_loc, sum d), in place of
// s_loc; and (blockIdx.y = 1) the adjoint that reaches every chunk's end out of the
// chunks' own adjoints of their start, in place of those. One thread per
// (channel, state, sequence), the chunks one after the other, kCombine of them loaded together
// (a trip also waits for the stores of the one before: few long trips).
constexpr int kCombine = 32;
template <int N>
__global__ __launch_bounds__(256) void ssm_combine_kernel(ScanIn a, float* __restrict__ cst,
                                                          const float* __restrict__ csum, float* __restrict__ G,
                                                          const float* __restrict__ dstate_out, int64_t first) {
  const int64_t id = first + (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int E = a.E;
  const int e = (int)(id % E), n = (int)(id / E % N);
  const int64_t seq = id / E / N;
  if (seq >= a.n_seq) return;
  const int o0 = min(max(a.offs[seq], 0), a.rows), o1 = min(max(a.offs[seq + 1], o0), a.rows);
  const int nch = max(1, (o1 - o0 + a.CL - 1) / a.CL);
  const int64_t w0 = o0 / a.CL + seq;
  const float a2 = decay_rate(a.A_log[(int64_t)e * N + n]);
  const bool back = blockIdx.y != 0;
  float* st = (back ? G : cst) + (w0 * N + n) * E + e;
  const float* sm = csum + w0 * E + e;
  const int64_t step = (int64_t)N * E;
  float s = 0.f;
  if (back) {
    if (dstate_out) s = dstate_out[(seq * E + e) * N + n];
  } else {
    const int sl = slot_of(a.slots, a.n_slots, (int)seq);
    if (a.state && sl >= 0) s = a.state[((int64_t)sl * E + e) * N + n];
  }
  // the chunk that comes last gives its place and takes part in nothing
  const int dir = back ? -1 : 1;
  if (back) {
    st += (nch - 1) * step;
    sm += (int64_t)(nch - 1) * E;
  }
  const int last = nch - 2;  // the last one to take part
  for (int c = 0; c <= last; c += kCombine) {
    float v[kCombine], d[kCombine];
#pragma unroll
    for (int i = 0; i < kCombine; ++i) {
      const int k = min(c + i, last) * dir;
      v[i] = st[k * step];
      d[i] = sm[(int64_t)k * E];
    }
#pragma unroll
    for (int i = 0; i < kCombine; ++i) {
      const bool in = c + i <= last;
      if (in) st[(c + i) * dir * step] = s;
      const float f = __builtin_amdgcn_exp2f(a2 * d[i]);
      s = in ? fmaf(f, s, v[i]) : s;
    }
  }
  st[(nch - 1) * dir * step] = s;
}


// ---------------------------------------------------------------- selective scan, single tokens
// N / 4 lanes per channel hold four states each: a wavefront reads and writes
// 1 KB of states in one access, and y is summed over the lanes of a channel
// by DPP. A workgroup takes 1,024 / N channels of SB sequences, whose loads are all in
// flight together and share the decay rates. Bound by the states' bytes: 256 sequences of 4,096 bf16
// channels (143 MB) in 22 us when the cache still holds some of them, 32 when it does not, a copy's rate.
template <typename T, int N, int SB>
__global__ __launch_bounds__(256) void ssm_scan_token_kernel(ScanIn a, const T* __restrict__ u,
                                                             const T* __restrict__ dt, const T* __restrict__ B,
                                                             const T* __restrict__ C, const T* __restrict__ z,
                                                             float* state_out, T* __restrict__ y, int64_t ldy) {
  constexpr int Q = N / 4;
  const int E = a.E, groups = (E + 256 / Q - 1) / (256 / Q), first = blockIdx.x / groups * SB;
  const int e = blockIdx.x % groups * (256 / Q) + threadIdx.x / Q, n0 = (threadIdx.x % Q) * 4;
  const bool active = e < E;
  const int ec = active ? e : E - 1;
  const floatx4 al = *reinterpret_cast<const floatx4*>(a.A_log + (int64_t)ec * N + n0);
  const float bias = a.b_dt ? a.b_dt[ec] : 0.f, Dv = a.D ? a.D[ec] : 0.f;
  floatx4 s[SB];
  T ur[SB], dr[SB], zr[SB], br[SB][4], cr[SB][4];
  int sl[SB];
#pragma unroll
  for (int i = 0; i < SB; ++i) {
    const int q = min(first + i, a.n_seq - 1);
    sl[i] = slot_of(a.slots, a.n_slots, q);
    s[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (a.state && sl[i] >= 0)
      s[i] = *reinterpret_cast<const floatx4*>(a.state + ((int64_t)sl[i] * E + ec) * N + n0);
    ur[i] = u[q * a.ldu + ec];
    dr[i] = dt[q * a.lddt + ec];
    if (z) zr[i] = z[q * a.ldz + ec];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      br[i][n] = B[q * a.ldB + n0 + n];
      cr[i][n] = C[q * a.ldC + n0 + n];
    }
  }
  float a2[4];
#pragma unroll
  for (int n = 0; n < 4; ++n) a2[n] = decay_rate(al[n]);
#pragma unroll
  for (int i = 0; i < SB; ++i) {
    const int q = first + i;
    const float uv = to_f32(ur[i]), d = softplus(to_f32(dr[i]) + bias), du = d * uv;
    float acc = 0.f;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      s[i][n] = fmaf(__builtin_amdgcn_exp2f(d * a2[n]), s[i][n], du * to_f32(br[i][n]));
      acc = fmaf(s[i][n], to_f32(cr[i][n]), acc);
    }
    acc += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(acc), 0xB1, 0xF, 0xF, false));  // xor 1
    if (Q == 4)
      acc += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(acc), 0x4E, 0xF, 0xF, false));  // xor 2
    acc = fmaf(Dv, uv, acc);
    if (z) acc *= silu(to_f32(zr[i]));
    if (!active || q >= a.n_seq) continue;
    if (state_out && sl[i] >= 0)
      *reinterpret_cast<floatx4*>(state_out + ((int64_t)sl[i] * E + e) * N + n0) = s[i];
    if (n0 == 0) st1(y + q * ldy + e, acc);
  }
}

// ---------------------------------------------------------------- selective scan, gradients
// Adjoints run backwards: g_t = q_t C_t + h_t, h_{t-1} = exp(d_t A) g_t, with q = dy SiLU(z)
// and h after the last token the gradient of the end state. Then
//   dB_t = sum_e g d u,  dC_t = sum_e q s_t,  dd = sum_n g (A a s_{t-1} + u B),
//   du = D q + d sum_n g B,  dz = dy (C . s_t + D u) SiLU'(z),  ddt = dd sigmoid(dt + b_dt),
//   dA_log = A sum_t g d a s_{t-1},  dD = sum_t q u,  db_dt = sum_t ddt.
// Sequences are cut into chunks of kBCL tokens, which the adjoints need as the
// states do: ssm_bwd_local_kernel forms a chunk's (s_loc, sum d) and, in the same
// forward walk, its adjoint of the start state, sum_t (prod a) C_t q_t;
// ssm_combine_kernel joins them. Sequences of one chunk skip both.
constexpr int kBCL = 30;  // tokens per chunk
constexpr int kSub = 6;   // tokens whose states are held in registers together

// nt rows of B | C, widened, into LDS by n threads (a multiple of 2N).
template <typename T, int N>
__device__ __forceinline__ void stage_bc(float* s, const T* B, int64_t ldB, const T* C, int64_t ldC, int nt, int tid,
                                         int n) {
  const int col = tid % (2 * N), step = n / (2 * N);
  const int64_t ld = col < N ? ldB : ldC;
  int row = tid / (2 * N);
  const T* q = (col < N ? B + col : C + (col - N)) + row * ld;
  for (; row < nt; row += step, q += step * ld) s[row * 2 * N + col] = to_f32(*q);
}

template <typename T, int N>
__global__ __launch_bounds__(64, 4) void ssm_bwd_local_kernel(ScanIn a, const T* __restrict__ u,
                                                              const T* __restrict__ dt, const T* __restrict__ B,
                                                              const T* __restrict__ C, const T* __restrict__ z,
                                                              const T* __restrict__ dy, int64_t lddy,
                                                              float* __restrict__ cst, float* __restrict__ csum,
                                                              float* __restrict__ G) {
  __shared__ __attribute__((aligned(16))) float sBC[kBCL * 2 * N];
  int w, cg;
  if (!tile_of_block(a.ntile, (a.E + 63) / 64, w, cg)) return;
  const Tile tl = find_tile(a.offs, a.n_seq, a.rows, kBCL, w);
  if (tl.seq < 0) return;
  const int t0 = tl.j * kBCL, t1 = min(tl.len, t0 + kBCL);
  const int lane = threadIdx.x, E = a.E;
  const int e = cg * 64 + lane;
  const bool active = e < E;
  const int ec = active ? e : E - 1;
  const int64_t r0 = tl.base;
  const uint32_t le = ec * sizeof(T), lf = ec * 4;
  float a2[N], s[N], p[N], g[N];
  ld_vec<N>(a.A_log, ec * N * 4, a2);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    a2[n] = decay_rate(a2[n]);
    s[n] = 0.f;
    p[n] = 1.f;
    g[n] = 0.f;
  }
  const float bias = a.b_dt ? a.b_dt[ec] : 0.f;
  float sum = 0.f;
  stage_bc<T, N>(sBC, B + (r0 + t0) * a.ldB, a.ldB, C + (r0 + t0) * a.ldC, a.ldC, t1 - t0, lane, 64);
  __syncthreads();
  if (t0 < t1) {
    constexpr int U = 2;
    T nu[U], nd[U], nz[U], ng[U];
    auto load = [&](int t) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int64_t r = r0 + min(t + i, t1 - 1);
        nu[i] = ld_at(u + r * a.ldu, le);
        nd[i] = ld_at(dt + r * a.lddt, le);
        ng[i] = ld_at(dy + r * lddy, le);
        if (z) nz[i] = ld_at(z + r * a.ldz, le);
      }
    };
    load(t0);
    for (int tg = t0; tg < t1; tg += U) {
      T cu[U], cd[U], cz[U], cg_[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        cu[i] = nu[i];
        cd[i] = nd[i];
        cg_[i] = ng[i];
        if (z) cz[i] = nz[i];
      }
      if (tg + U < t1) load(tg + U);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int t = tg + i;
        if (t >= t1) break;
        const float* x = &sBC[(t - t0) * 2 * N];
        const float d = softplus(to_f32(cd[i]) + bias), du = d * to_f32(cu[i]);
        const float q = z ? to_f32(cg_[i]) * silu(to_f32(cz[i])) : to_f32(cg_[i]);
        sum += d;
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const float an = __builtin_amdgcn_exp2f(d * a2[n]);
          s[n] = fmaf(an, s[n], du * x[n]);
          p[n] *= an;
          g[n] = fmaf(p[n], q * x[N + n], g[n]);
        }
      }
    }
  }
  if (!active) return;
  st_at(csum + (int64_t)w * E, lf, sum);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    st_at(cst + ((int64_t)w * N + n) * E, lf, s[n]);
    st_at(G + ((int64_t)w * N + n) * E, lf, g[n]);
  }
}

// Sums of many values over the 64 lanes, scattered over the lanes: halves of the
// values go to halves of the lanes step by step, half-wave and row swaps routing a pair at
// once, then within rows of 16 by DPP (rotation by 8, mirrors of 8, quad
// permutations). Some 2 M operations for M values instead of 12 M.
__device__ __forceinline__ float swap_add32(float a, float b) {  // lanes 0-31: a's sums, 32-63: b's
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float swap_add16(float a, float b) {  // rows 0, 2 of 16: a's sums, 1, 3: b's
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// M = 8 or 4 values over rows of 16 lanes: lane l of a row ends with value l M / 16's total.
template <int M>
__device__ __forceinline__ float reduce_rows(const float* v, int lane) {
  const bool b3 = (lane & 8) != 0, b2 = (lane & 4) != 0, b1 = (lane & 2) != 0;
  float x[M / 2], y[M / 4];
#pragma unroll
  for (int i = 0; i < M / 2; ++i) {  // row_ror:8
    const float mine = b3 ? v[M / 2 + i] : v[i], other = b3 ? v[i] : v[M / 2 + i];
    x[i] = mine + dpp<0x128>(other);
  }
#pragma unroll
  for (int i = 0; i < M / 4; ++i) {  // row_half_mirror: lane ^ 7
    const float mine = b2 ? x[M / 4 + i] : x[i], other = b2 ? x[i] : x[M / 4 + i];
    y[i] = mine + dpp<0x141>(other);
  }
  float s;
  if constexpr (M == 8) {
    const float mine = b1 ? y[1] : y[0], other = b1 ? y[0] : y[1];
    s = mine + dpp<0x4E>(other);  // quad_perm: lane ^ 2
  } else {
    s = y[0] + dpp<0x4E>(y[0]);
  }
  return s + dpp<0xB1>(s);  // lane ^ 1
}

// Sequences by falling length, lengths past kBCL as equals, by a count per length; equals in
// no fixed order, which nothing depends on (results lie where the sequence's do). One workgroup.
__global__ __launch_bounds__(1024) void ssm_order_kernel(const int* __restrict__ offs, int n_seq, int rows,
                                                         int* __restrict__ ord) {
  __shared__ int count[kBCL + 2];
  const int tid = threadIdx.x;
  auto bin = [&](int i) {  // 0: the longest
    const int o0 = min(max(offs[i], 0), rows), o1 = min(max(offs[i + 1], o0), rows);
    return kBCL + 1 - min(o1 - o0, kBCL + 1);
  };
  if (tid < kBCL + 2) count[tid] = 0;
  __syncthreads();
  for (int i = tid; i < n_seq; i += 1024) atomicAdd(&count[bin(i)], 1);
  __syncthreads();
  int before = 0;
  if (tid < kBCL + 2)
    for (int j = 0; j < tid; ++j) before += count[j];
  __syncthreads();
  if (tid < kBCL + 2) count[tid] = before;
  __syncthreads();
  for (int i = tid; i < n_seq; i += 1024) ord[atomicAdd(&count[bin(i)], 1)] = i;
}

// A workgroup takes `per` chunks of 64 nw channels one after the other, a lane per channel. The chunk's
// start state is walked forward once to leave the state in front of every
// kSub tokens (but the first) in LDS; then, from the last kSub tokens to the first, the states
// in front of each token are formed again into registers and the tokens walked
// backwards. dB and dC of a token are sums over channels: over a wavefront by
// swaps and DPP, over the workgroup's wavefronts through LDS, over
// workgroups (more than 64 nw channels) by ssm_sum_bc_kernel, all in a fixed order.
// dA_log, dD and db_dt leave as partial sums, one set per workgroup. 22 N slots per token and
// wavefront for the states, 70 for the two sums over channels, the rest for what is per channel: 462 instructions
// (515 slots) by the counters. Four sequences of 7,127 tokens together, E 2,048, bf16, in 276 us at best, of which issue
// takes 192 (the vector unit 75% busy, two wavefronts to a SIMD by 249 registers); chunks of 32 tokens in eights, 25
// registers spilled, took 16% longer. With N = 16 the loop of several chunks (MULTI) spills 9 to 10 registers.
template <typename T, int N, bool MULTI>
__global__ __launch_bounds__(256, 2) void ssm_bwd_kernel(
    ScanIn a, const T* __restrict__ u, const T* __restrict__ dt, const T* __restrict__ B, const T* __restrict__ C,
    const T* __restrict__ z, const T* __restrict__ dy, int64_t lddy, const float* __restrict__ cst,
    const float* __restrict__ H, const float* __restrict__ dstate_out, T* __restrict__ du_o, int64_t lddu,
    T* __restrict__ ddt_o, int64_t ldddt, T* __restrict__ dz_o, int64_t lddz, T* __restrict__ dB_o, int64_t lddB,
    T* __restrict__ dC_o, int64_t lddC, float* __restrict__ dstate, float* __restrict__ part, int parts, int per,
    const int* __restrict__ ord, float* __restrict__ bc_part) {
  constexpr int W = 2 * N, NSUB = kBCL / kSub;
  extern __shared__ __attribute__((aligned(16))) float smem[];
  const int nw = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, E = a.E;
  float* sBC = smem;                                       // [kBCL][2N]
  float* sRed = smem + kBCL * W;                           // [kSub][nw][2N]
  float* sCk = sRed + kSub * nw * W + wave * (NSUB - 1) * N * 64 + lane;  // [NSUB - 1][N][64] per wavefront
  int p, cg;
  const int CG = (E + blockDim.x - 1) / blockDim.x;
  if (!tile_of_block(parts, CG, p, cg)) return;
  if (!MULTI && ord) p = __builtin_amdgcn_readfirstlane(ord[p]);
  const int e = cg * blockDim.x + threadIdx.x;
  const bool active = e < E;
  const int ec = active ? e : E - 1;
  const uint32_t le = ec * sizeof(T), lf = ec * 4, ln = ec * N * 4;
  float a2[N], s[N], h[N], dA[N];
  ld_vec<N>(a.A_log, ln, a2);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    a2[n] = decay_rate(a2[n]);
    dA[n] = 0.f;
  }
  const float bias = a.b_dt ? a.b_dt[ec] : 0.f, Dv = a.D ? a.D[ec] : 0.f;
  float dD = 0.f, dbias = 0.f;
  // what the lane holds of a token's 2N sums: dB or dC by its half, the state's parity by its
  // row, the pair of states within the row
  const int place = lane / 32 * N + lane % 16 / (32 / N) * 2 + lane / 16 % 2;
  auto chunk = [&](int w) {
    const Tile tl = find_tile(a.offs, a.n_seq, a.rows, a.CL, w);
    if (tl.seq < 0) return;
    const int t0 = tl.j * kBCL, nt = max(0, min(tl.len - t0, kBCL));
    const int64_t r0 = (int64_t)tl.base + t0;
    // (the chunk before has left the shared memory behind a barrier)
    stage_bc<T, N>(sBC, B + r0 * a.ldB, a.ldB, C + r0 * a.ldC, a.ldC, nt, threadIdx.x, blockDim.x);
    auto start = [&]() {  // the state in front of the chunk
      if (cst) {
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] = ld_at(cst + ((int64_t)w * N + n) * E, lf);
      } else if (a.state) {
        ld_vec<N>(a.state + (int64_t)tl.seq * E * N, ln, s);
      } else {
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] = 0.f;
      }
    };
    start();
    if (cst) {
#pragma unroll
      for (int n = 0; n < N; ++n) h[n] = ld_at(H + ((int64_t)w * N + n) * E, lf);
    } else if (dstate_out) {
      ld_vec<N>(dstate_out + (int64_t)tl.seq * E * N, ln, h);
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n) h[n] = 0.f;
    }
    __syncthreads();
    const int nsub = (nt + kSub - 1) / kSub;
    const T *us = u + r0 * a.ldu, *ds = dt + r0 * a.lddt, *zs = z ? z + r0 * a.ldz : nullptr, *gs = dy + r0 * lddy;
    auto park = [&](int b) {  // s in front of the kSub tokens b; the first ones' place is the second ones'
      float* ck = sCk + max(b - 1, 0) * N * 64;
#pragma unroll
      for (int n = 0; n < N; ++n) ck[n * 64] = s[n];
    };
    for (int b = 0; b < nsub - 1; ++b) {
      if (b > 0) park(b);
      T ru[kSub], rd[kSub];
#pragma unroll
      for (int i = 0; i < kSub; ++i) {  // all of these tokens exist
        ru[i] = ld_at(us + (b * kSub + i) * a.ldu, le);
        rd[i] = ld_at(ds + (b * kSub + i) * a.lddt, le);
      }
#pragma unroll
      for (int i = 0; i < kSub; ++i) {
        const float d = softplus(to_f32(rd[i]) + bias), du = d * to_f32(ru[i]);
        const float* x = &sBC[(b * kSub + i) * W];
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] = fmaf(__builtin_amdgcn_exp2f(d * a2[n]), s[n], du * x[n]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (nsub > 0) park(nsub - 1);
    T cu, cd, cz, cg_;  // the token's inputs, one token ahead
    auto load = [&](int t) {
      const int64_t r = max(t, 0);
      cu = ld_at(us + r * a.ldu, le);
      cd = ld_at(ds + r * a.lddt, le);
      cg_ = ld_at(gs + r * lddy, le);
      if (z) cz = ld_at(zs + r * a.ldz, le);
    };
    if (nt > 0) load(nt - 1);
    for (int b = nsub - 1; b >= 0; --b) {
      if (b == 0 && nsub > 1) {
        start();
        park(0);
      }
      const float* ck = sCk + max(b - 1, 0) * N * 64;
      // the states behind each of the tokens but the last, and the tokens' steps
      float hist[kSub - 1][N], step[kSub];
      {
        T ru[kSub - 1], rd[kSub];
#pragma unroll
        for (int i = 0; i < kSub; ++i) {
          const int64_t t = min(b * kSub + i, nt - 1);
          if (i + 1 < kSub) ru[i] = ld_at(us + t * a.ldu, le);
          rd[i] = ld_at(ds + t * a.lddt, le);
        }
#pragma unroll
        for (int i = 0; i < kSub; ++i) {
          if (b * kSub + i < nt) {
            step[i] = softplus(to_f32(rd[i]) + bias);
            if (i + 1 < kSub) {
              const float du = step[i] * to_f32(ru[i]);
              const float* x = &sBC[(b * kSub + i) * W];
#pragma unroll
              for (int n = 0; n < N; ++n)
                hist[i][n] = fmaf(__builtin_amdgcn_exp2f(step[i] * a2[n]), i ? hist[i - 1][n] : ck[n * 64], du * x[n]);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int i = kSub - 1; i >= 0; --i) {
        const int t = b * kSub + i;
        if (t >= nt) continue;  // the same for the whole workgroup
        const float* x = &sBC[t * W];
        const float uv = active ? to_f32(cu) : 0.f, v = to_f32(cd) + bias, gy = active ? to_f32(cg_) : 0.f;
        const float zv = z ? to_f32(cz) : 0.f;
        load(t - 1);
        const float d = step[i], du = d * uv;
        float gate = 1.f, dgate = 0.f;
        if (z) {
          const float sg = rcp_fast(1.f + exp_fast(-zv));
          gate = zv * sg;
          dgate = sg * fmaf(zv, 1.f - sg, 1.f);
        }
        const float q = gy * gate;
        float yv = 0.f, gB = 0.f, dd = 0.f, red[N / 2], half[2];
        // A state's terms of dB and dC go through the first step of their sums at once, a pair
        // of states' through the second: N / 2 values stay of the 2 N. Four states at a time
        // (the barriers keep the scheduler from holding all of a token's B, C and terms).
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const float an = __builtin_amdgcn_exp2f(d * a2[n]);
          const float as = an * (i ? hist[i - 1][n] : ck[n * 64]);
          const float st = i + 1 < kSub ? hist[i][n] : fmaf(du, x[n], as);
          const float g = fmaf(q, x[N + n], h[n]);
          yv = fmaf(st, x[N + n], yv);
          gB = fmaf(g, x[n], gB);
          const float ga = g * as;
          dd = fmaf(ga, a2[n], dd);  // in units of 1 / ln 2
          dA[n] = fmaf(ga, d, dA[n]);
          h[n] = an * g;
          half[n % 2] = swap_add32(g * du, q * st);  // lanes 0-31: dB, 32-63: dC
          if (n % 2) red[n / 2] = swap_add16(half[0], half[1]);
          if (n % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
        yv = fmaf(Dv, uv, yv);
        const float ddt = fmaf(dd, kLn2, uv * gB) * rcp_fast(1.f + exp_fast(-v));
        dD = fmaf(q, uv, dD);
        dbias += ddt;
        if (active) {
          const int64_t r = r0 + t;
          st_at(du_o + r * lddu, le, fmaf(Dv, q, d * gB));
          st_at(ddt_o + r * ldddt, le, ddt);
          if (z) st_at(dz_o + r * lddz, le, gy * yv * dgate);
        }
        const float tot = reduce_rows<N / 2>(red, lane);
        if (lane % (64 / W) == 0) sRed[(i * nw + wave) * W + place] = tot;
        __builtin_amdgcn_sched_barrier(0);
      }
      __syncthreads();
      for (int i = threadIdx.x; i < min(kSub, nt - b * kSub) * W; i += blockDim.x) {
        const int k = i / W, col = i % W;
        float acc = 0.f;
        for (int j = 0; j < nw; ++j) acc += sRed[(k * nw + j) * W + col];
        const int64_t r = r0 + b * kSub + k;
        if (bc_part) bc_part[((int64_t)cg * a.rows + r) * W + col] = acc;
        else if (col < N) st1(dB_o + r * lddB + col, acc);
        else st1(dC_o + r * lddC + col - N, acc);
      }
      __syncthreads();
    }
    if (active && dstate && tl.j == 0) st_vec<N>(dstate + (int64_t)tl.seq * E * N, ln, h);
  };
  if constexpr (MULTI) {
    for (int w = p * per; w < min((p + 1) * per, a.ntile); ++w) chunk(w);
  } else {
    chunk(p);
  }
  if (!active) return;
  float* po = part + (int64_t)p * (N + 2) * E;
#pragma unroll
  for (int n = 0; n < N; ++n) st_at(po + (int64_t)n * E, lf, dA[n] * (a2[n] * kLn2));
  st_at(po + (int64_t)N * E, lf, dD);
  st_at(po + (int64_t)(N + 1) * E, lf, dbias);
}

// dB and dC over the channel groups. Rows that no sequence owns have no
// partial sums and are left as they are.
template <typename T, int N>
__global__ __launch_bounds__(256) void ssm_sum_bc_kernel(const int* __restrict__ offs, int n_seq, int rows, int CG,
                                                         const float* __restrict__ bc_part, T* __restrict__ dB,
                                                         int64_t lddB, T* __restrict__ dC, int64_t lddC) {
  constexpr int W = 2 * N;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / W;
  const int r0 = offs ? offs[0] : 0, r1 = offs ? min(offs[n_seq], rows) : n_seq;
  if (row < r0 || row >= r1) return;
  const int col = (int)(i % W);
  float acc = 0.f;
  for (int c = 0; c < CG; ++c) acc += bc_part[((int64_t)c * rows + row) * W + col];
  if (col < N) st1(dB + row * lddB + col, acc);
  else st1(dC + row * lddC + col - N, acc);
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

constexpr int kCUs = 256;

// ---- convolution plans
// Forward tiles: 32 rows reread 3 of 32 rows; with few rows, shorter tiles
// give the GPU more wavefronts to have in flight.
int conv_rows(int rows, int CG) {
  for (int R = 32; R > 8; R /= 2)
    if ((int64_t)rows / R * CG >= (int64_t)kCUs * 8 * 64) return R;
  return 8;
}
// Gradients: as many threads as four wavefronts to a SIMD are, at most 1,024 parts; a thread takes one
// tile, of as many rows as that leaves it, or several of kConvBwdRows where the sequences alone are more than
// that. Where they are nearly as many, what that leaves is far more than an even share, and a long sequence
// among short ones would be one thread's (20,000 tokens and 254 of one, 4,096 bf16 channels: 11.1 ms, now 0.49): a
// tile has at most kConvBwdShares times the even share, or kConvBwdMost rows, for an eighth more parts.
// (Twice the share: 0.24 ms there, but 255 sequences of 1,000 tokens 1.32 to 1.72.)
constexpr int kConvBwdRows = 32, kConvBwdMost = 256, kConvBwdShares = 8;
struct ConvParts {
  int R, per, parts;
};
ConvParts conv_parts(int n_seq, int rows, int E) {
  const int CG = (E + 3) / 4, want = std::max(1, std::min(1024, kCUs * 16 * 64 / CG));
  ConvParts p;
  p.R = kConvBwdRows;
  p.per = 1;
  if (want > n_seq) {
    const int64_t left = ((int64_t)rows + want - n_seq - 1) / (want - n_seq);
    p.R = std::max(p.R, (int)std::min(left, std::max<int64_t>(kConvBwdMost, kConvBwdShares * ((int64_t)rows / want + 1))));
  }
  const int tiles = rows / p.R + n_seq;
  if (want <= n_seq) p.per = (tiles + want - 1) / want;
  p.parts = (tiles + p.per - 1) / p.per;
  return p;
}

}  // namespace

// One trip up to 512 parts, by halves.
void sum_parts(const float* part, int parts, int M, int total, int E, float* o0, float* o1, float* o2, hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)total * E + 63) / 64));
  if (parts > 16 * kSumLanes) sum_parts_kernel<32><<<grid, 64 * kSumLanes, 0, s>>>(part, parts, M, total, E, o0, o1, o2);
  else sum_parts_kernel<16><<<grid, 64 * kSumLanes, 0, s>>>(part, parts, M, total, E, o0, o1, o2);
}

namespace {

template <typename T, int K, int CH>
hipError_t conv_fwd(const ConvOp& a, void* state_out, void* u, int64_t ldu, hipStream_t s) {
  const int CG = a.E / CH, R = a.offs ? conv_rows(a.rows, CG) : 8;
  const int64_t tiles = a.offs ? (int64_t)a.rows / R + a.n_seq : a.n_seq, work = tiles * CG;
  ssm_conv_kernel<T, K, CH><<<dim3((unsigned)((work + 255) / 256)), 256, 0, s>>>(
      a.offs, a.n_seq, a.rows, a.E, R, work, static_cast<const T*>(a.x), a.ldx, a.w, a.b,
      static_cast<const T*>(a.state), a.slots, a.n_slots, static_cast<T*>(state_out), static_cast<T*>(u), ldu);
  return hipGetLastError();
}

template <typename T, int K, int CH>
hipError_t conv_bwd(const ConvOp& a, const void* du, int64_t lddu, const void* dstate_out, void* dx, int64_t lddx,
                    float* dw, float* db, void* dstate, float* ws, hipStream_t s) {
  const int CG = a.E / CH;
  const ConvParts p = conv_parts(a.n_seq, a.rows, a.E);
  const int64_t work = (int64_t)p.parts * CG;
  ssm_conv_bwd_kernel<T, K, CH><<<dim3((unsigned)((work + 255) / 256)), 256, 0, s>>>(
      a.offs, a.n_seq, a.rows, a.E, p.R, p.per, p.parts, static_cast<const T*>(a.x), a.ldx, a.w, a.b,
      static_cast<const T*>(a.state), static_cast<const T*>(du), lddu, static_cast<const T*>(dstate_out),
      static_cast<T*>(dx), lddx, static_cast<T*>(dstate), ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  sum_parts(ws, p.parts, K, K + 1, a.E, dw, db, nullptr, s);
  return hipGetLastError();
}

// ---- scan plans
// How the forward scan runs, by the wavefronts that one lane per channel would give it. From 2,048 on
// (two to a SIMD) sequences run whole, a lane per channel; below, whole with N / 4 lanes per channel;
// below 256, longer than two stages, in chunks. E 4,096, bf16 (us: chunks / lane per channel / N / 4 lanes):
// 32 sequences of 1,024 tokens (2,048 wavefronts) 971 / 665 / 648, 16 544 / 547 / 395, 8 294 / 462 / 243;
// 4 of 256 (256) 60 / 121 / 61, one (64) 39 / 111 / 57; E 512: 16 of 512 (128) 57 / 220 / 83, 512 of 100
// at E 256 (2,048) 180 / 70 / 68, 64 of 128 at E 4,096 (4,096) - / 131 / 151.
int64_t scan_waves(int n_seq, int E) { return (int64_t)n_seq * ((E + 63) / 64); }
bool scan_quad(int n_seq, int E) { return scan_waves(n_seq, E) < 2048; }
// Tokens per chunk, 0 for whole sequences: enough chunks for four wavefronts to every SIMD, were all
// sequences L long.
int scan_chunk(int n_seq, int E, int L) {
  const int64_t waves = scan_waves(n_seq, E), fill = (int64_t)kCUs * 4 * 4;
  if (L <= 2 * kTC || waves >= 256) return 0;
  const int64_t chunks = fill / std::max<int64_t>(waves, 1);
  int64_t CL = (L + chunks - 1) / chunks;
  CL = std::max<int64_t>((CL + kTC - 1) / kTC * kTC, kTC);
  return CL < L ? (int)CL : 0;
}

ScanIn scan_in(const ScanOp& a, int CL) {
  ScanIn in;
  in.offs = a.offs; in.n_seq = a.n_seq; in.rows = a.rows; in.E = a.E; in.CL = CL;
  in.ntile = a.offs ? a.rows / CL + a.n_seq : a.n_seq;
  in.ldu = a.ldu; in.lddt = a.lddt; in.ldB = a.ldB; in.ldC = a.ldC; in.ldz = a.ldz;
  in.A_log = a.A_log; in.D = a.D; in.b_dt = a.b_dt; in.state = a.state;
  in.slots = a.slots; in.n_slots = a.n_slots;
  return in;
}

// The states and, with G, the adjoints. 2^30 threads to a launch (one has fewer than 2^32).
template <int N>
void combine(const ScanIn& in, float* cst, const float* csum, float* G, const float* dstate_out, hipStream_t s) {
  const int64_t n = (int64_t)in.n_seq * N * in.E;
  for (int64_t first = 0; first < n; first += (int64_t)1 << 30) {
    const int64_t k = std::min(n - first, (int64_t)1 << 30);
    ssm_combine_kernel<N><<<dim3((unsigned)((k + 255) / 256), G ? 2 : 1), 256, 0, s>>>(in, cst, csum, G, dstate_out,
                                                                                       first);
  }
}

template <typename T, int N>
hipError_t scan_fwd(const ScanOp& a, float* state_out, void* y_, int64_t ldy, float* ws, hipStream_t s) {
  const T *u = static_cast<const T*>(a.u), *dt = static_cast<const T*>(a.dt), *B = static_cast<const T*>(a.B),
          *C = static_cast<const T*>(a.C), *z = static_cast<const T*>(a.z);
  T* y = static_cast<T*>(y_);
  if (!a.offs) {
    const ScanIn in = scan_in(a, 1);
    const unsigned gx = (a.E + 1024 / N - 1) / (1024 / N);
    constexpr int SB = 4;
    if ((int64_t)gx * a.n_seq >= (int64_t)kCUs * 4 * SB)
      ssm_scan_token_kernel<T, N, SB><<<dim3(gx * ((a.n_seq + SB - 1) / SB)), 256, 0, s>>>(in, u, dt, B, C, z,
                                                                                          state_out, y, ldy);
    else
      ssm_scan_token_kernel<T, N, 1><<<dim3(gx * a.n_seq), 256, 0, s>>>(in, u, dt, B, C, z, state_out, y, ldy);
    return hipGetLastError();
  }
  const int CG = (a.E + 63) / 64, CL = scan_chunk(a.n_seq, a.E, a.L);
  if (!CL) {
    const ScanIn in = scan_in(a, a.rows + 1);  // one tile per sequence
    if (scan_quad(a.n_seq, a.E)) {
      constexpr int CH = kQuadThreads / (N / 4);
      ssm_scan_quad_kernel<T, N><<<dim3(tile_blocks(in.ntile, (a.E + CH - 1) / CH)), kQuadThreads, 0, s>>>(
          in, u, dt, B, C, z, state_out, y, ldy);
      return hipGetLastError();
    }
    ssm_scan_kernel<T, N, false><<<dim3(tile_blocks(in.ntile, CG)), 64, 0, s>>>(in, u, dt, B, C, z, state_out, y, ldy,
                                                                               nullptr, nullptr);
    return hipGetLastError();
  }
  const ScanIn in = scan_in(a, CL);
  float *cst = ws, *csum = ws + (int64_t)in.ntile * N * a.E;
  ssm_scan_kernel<T, N, true><<<dim3(tile_blocks(in.ntile, CG)), 64, 0, s>>>(in, u, dt, B, nullptr, nullptr, nullptr,
                                                                            nullptr, 0, cst, csum);
  combine<N>(in, cst, csum, nullptr, nullptr, s);
  ssm_scan_kernel<T, N, false><<<dim3(tile_blocks(in.ntile, CG)), 64, 0, s>>>(in, u, dt, B, C, z, state_out, y, ldy,
                                                                             cst, nullptr);
  return hipGetLastError();
}

struct BwdPlan {
  int nw, CG, ntile, per, parts;
  bool chunks;
  bool order;
  size_t cst, csum, G, part, bc, ord, total;  // in floats
};
BwdPlan bwd_plan(bool packed, int n_seq, int rows, int E, int N, int L) {
  BwdPlan p;
  p.nw = std::min(4, (E + 63) / 64);
  p.CG = (E + 64 * p.nw - 1) / (64 * p.nw);
  p.chunks = packed && L > kBCL;
  p.ntile = p.chunks ? rows / kBCL + n_seq : n_seq;
  // Short sequences, a chunk each, are handed out longest first, so that the workgroups (two on a CU at a time)
  // end together: 1,024 of 1 to 25 tokens, E 256, fp32, 118 to 83 us, 4,096 of them 387 to 288. With more
  // than 32 rounds of workgroups, or 16 of sequences with too few tokens to pay for partial sums as large
  // as two tokens, they go several to a workgroup in their order: 30,000 of 1 to 15, E 256, fp32, 1,326 us
  // against 1,459, 9,000 of 1 to 7 267 against 286 (of 1 to 15 459 against 437). Not chunks of long ones, which lose
  // 5% to the registers that the loop takes (with N = 16 it spills 9 to 10).
  const int64_t groups = (int64_t)p.ntile * p.CG, round = kCUs * 2;
  p.order = packed && !p.chunks && groups > round && groups <= 32 * round &&
            (groups < 16 * round || rows >= 6 * (int64_t)n_seq);
  p.per = p.chunks || p.order ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(16, groups / (8 * round)));
  p.parts = (p.ntile + p.per - 1) / p.per;
  size_t o = 0;
  const size_t st = p.chunks ? (size_t)p.ntile * N * E : 0;
  p.cst = o; o += st;
  p.G = o; o += st;
  p.csum = o; o += p.chunks ? (size_t)p.ntile * E : 0;
  p.part = o; o += (size_t)p.parts * (N + 2) * E;
  p.bc = o; o += p.CG > 1 ? (size_t)p.CG * rows * 2 * N : 0;
  p.ord = o; o += p.order ? n_seq : 0;
  p.total = o;
  return p;
}

template <typename T, int N>
hipError_t scan_bwd(const ScanOp& a, const void* dy_, int64_t lddy, const float* dstate_out, const ScanGrads& g,
                    float* ws, hipStream_t s) {
  const T *u = static_cast<const T*>(a.u), *dt = static_cast<const T*>(a.dt), *B = static_cast<const T*>(a.B),
          *C = static_cast<const T*>(a.C), *z = static_cast<const T*>(a.z), *dy = static_cast<const T*>(dy_);
  const BwdPlan p = bwd_plan(a.offs != nullptr, a.n_seq, a.rows, a.E, N, a.L);
  const ScanIn in = scan_in(a, p.chunks || !a.offs ? kBCL : a.rows + 1);  // (+ 1: a tile per sequence)
  float *cst = p.chunks ? ws + p.cst : nullptr, *G = p.chunks ? ws + p.G : nullptr, *part = ws + p.part,
        *bc = p.CG > 1 ? ws + p.bc : nullptr;
  if (p.chunks) {
    ssm_bwd_local_kernel<T, N><<<dim3(tile_blocks(in.ntile, (a.E + 63) / 64)), 64, 0, s>>>(
        in, u, dt, B, C, z, dy, lddy, cst, ws + p.csum, G);
    combine<N>(in, cst, ws + p.csum, G, dstate_out, s);
  }
  int* ord = p.order ? reinterpret_cast<int*>(ws + p.ord) : nullptr;
  if (ord) ssm_order_kernel<<<dim3(1), 1024, 0, s>>>(a.offs, a.n_seq, a.rows, ord);
  const size_t lds = sizeof(float) * (2 * N * (kBCL + kSub * p.nw) + (size_t)p.nw * (kBCL / kSub - 1) * N * 64);
  auto kernel = p.per > 1 ? &ssm_bwd_kernel<T, N, true> : &ssm_bwd_kernel<T, N, false>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  kernel<<<dim3(tile_blocks(p.parts, p.CG)), 64 * p.nw, lds, s>>>(
      in, u, dt, B, C, z, dy, lddy, cst, G, dstate_out, static_cast<T*>(g.du), g.lddu, static_cast<T*>(g.ddt),
      g.ldddt, static_cast<T*>(g.dz), g.lddz, static_cast<T*>(g.dB), g.lddB, static_cast<T*>(g.dC), g.lddC, g.dstate,
      part, p.parts, p.per, ord, bc);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (bc && a.rows > 0) {
    const int64_t n = (int64_t)a.rows * 2 * N;
    ssm_sum_bc_kernel<T, N><<<dim3((unsigned)((n + 255) / 256)), 256, 0, s>>>(
        a.offs, a.n_seq, a.rows, p.CG, bc, static_cast<T*>(g.dB), g.lddB, static_cast<T*>(g.dC), g.lddC);
  }
  sum_parts(part, p.parts, N, N + 2, a.E, g.dA_log, g.dD, g.db_dt, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_ssm_conv(const ConvOp& a, void* state_out, void* u, int64_t ldu, hipStream_t s) {
  const bool vec = a.E % 4 == 0 && a.ldx % 4 == 0 && ldu % 4 == 0 && aligned16(a.x) && aligned16(u) &&
                   aligned16(a.state) && aligned16(state_out);
#define TCL_CONV(KK)                                                                                       \
  case KK:                                                                                                 \
    if (a.bf16) return vec ? conv_fwd<uint16_t, KK, 4>(a, state_out, u, ldu, s)                            \
                           : conv_fwd<uint16_t, KK, 1>(a, state_out, u, ldu, s);                           \
    return vec ? conv_fwd<float, KK, 4>(a, state_out, u, ldu, s) : conv_fwd<float, KK, 1>(a, state_out, u, ldu, s);
  switch (a.K) {
    TCL_CONV(1)
    TCL_CONV(2)
    TCL_CONV(3)
    TCL_CONV(4)
  }
#undef TCL_CONV
  return hipErrorInvalidValue;
}

size_t ssm_conv_workspace_bytes(int n_seq, int rows, int E, int K) {
  return (size_t)conv_parts(n_seq, rows, E).parts * (K + 1) * E * sizeof(float);
}

hipError_t launch_ssm_conv_bwd(const ConvOp& a, const void* du, int64_t lddu, const void* dstate_out, void* dx,
                               int64_t lddx, float* dw, float* db, void* dstate, float* ws, hipStream_t s) {
  const bool vec = a.E % 4 == 0 && a.ldx % 4 == 0 && lddu % 4 == 0 && lddx % 4 == 0 && aligned16(a.x) &&
                   aligned16(du) && aligned16(dx) && aligned16(a.state) && aligned16(dstate_out) && aligned16(dstate);
#define TCL_CONV(KK)                                                                                          \
  case KK:                                                                                                    \
    if (a.bf16)                                                                                               \
      return vec ? conv_bwd<uint16_t, KK, 4>(a, du, lddu, dstate_out, dx, lddx, dw, db, dstate, ws, s)        \
                 : conv_bwd<uint16_t, KK, 1>(a, du, lddu, dstate_out, dx, lddx, dw, db, dstate, ws, s);       \
    return vec ? conv_bwd<float, KK, 4>(a, du, lddu, dstate_out, dx, lddx, dw, db, dstate, ws, s)             \
               : conv_bwd<float, KK, 1>(a, du, lddu, dstate_out, dx, lddx, dw, db, dstate, ws, s);
  switch (a.K) {
    TCL_CONV(1)
    TCL_CONV(2)
    TCL_CONV(3)
    TCL_CONV(4)
  }
#undef TCL_CONV
  return hipErrorInvalidValue;
}

size_t ssm_scan_workspace_bytes(int n_seq, int rows, int E, int N, int L) {
  const int CL = scan_chunk(n_seq, E, L);
  return CL ? ((size_t)rows / CL + n_seq) * (N + 1) * E * sizeof(float) : 0;
}

hipError_t launch_ssm_scan(const ScanOp& a, float* state_out, void* y, int64_t ldy, float* ws, hipStream_t s) {
  if (a.bf16)
    return a.N == 16 ? scan_fwd<uint16_t, 16>(a, state_out, y, ldy, ws, s)
                     : scan_fwd<uint16_t, 8>(a, state_out, y, ldy, ws, s);
  return a.N == 16 ? scan_fwd<float, 16>(a, state_out, y, ldy, ws, s) : scan_fwd<float, 8>(a, state_out, y, ldy, ws, s);
}

size_t ssm_scan_bwd_workspace_bytes(int n_seq, int rows, int E, int N, int L) {
  // (as many rows as sequences may also be single tokens without offsets, with a plan of their own)
  const size_t packed = bwd_plan(true, n_seq, rows, E, N, L).total;
  return (rows == n_seq ? std::max(packed, bwd_plan(false, n_seq, rows, E, N, 1).total) : packed) * sizeof(float);
}

hipError_t launch_ssm_scan_bwd(const ScanOp& a, const void* dy, int64_t lddy, const float* dstate_out,
                               const ScanGrads& g, float* ws, hipStream_t s) {
  if (a.bf16)
    return a.N == 16 ? scan_bwd<uint16_t, 16>(a, dy, lddy, dstate_out, g, ws, s)
                     : scan_bwd<uint16_t, 8>(a, dy, lddy, dstate_out, g, ws, s);
  return a.N == 16 ? scan_bwd<float, 16>(a, dy, lddy, dstate_out, g, ws, s)
                   : scan_bwd<float, 8>(a, dy, lddy, dstate_out, g, ws, s);
}

}  // namespace tcl

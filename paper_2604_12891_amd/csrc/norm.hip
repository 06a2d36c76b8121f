// Layer norm over the columns of a row matrix, and its gradients:
//   m = mean x, r = (mean (x - m)^2 + eps)^-1/2, h = (x - m) r, y = h w + b,
//   dx = r (g - mean g - h mean(g h)), g = dy w,  dw = sum over rows dy h,  db = sum over rows dy.
// Nothing is kept from the forward call: the gradients read x anyway, and a row's statistics
// are two reductions of what is then in registers. Both passes are bound by HBM, 2 and 3 arrays: 16,384 x 5,120 bf16 in
// 69 and 113 us, where a large copy's rate (4.8 TB/s) would take 70 and 106.
#include <algorithm>

#include "common.h"
#include "ops.h"

namespace tcl {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Rows of odd widths start anywhere: 16 bytes at the alignment of one element.
template <typename T> struct Loose;
template <> struct Loose<float> { typedef u32x4 type __attribute__((aligned(4))); };
template <> struct Loose<uint16_t> { typedef u32x4 type __attribute__((aligned(2))); };

__device__ __forceinline__ uint32_t raw1(const float* p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t raw1(const uint16_t* p) { return *p; }

// A thread's NV vectors of VE elements: vector j is number j * stride + t of the row.
template <typename T, int NV>
struct Cols {
  static constexpr int VE = 16 / sizeof(T);
  int C, t, stride;

  __device__ __forceinline__ int col(int j) const { return (j * stride + t) * VE; }
  __device__ __forceinline__ int have(int j) const { return min(max(C - col(j), 0), VE); }
  // f(j, i) for the entries that the row has: whole vectors without a test of each
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (col(j) + VE <= C) {
#pragma unroll
        for (int i = 0; i < VE; ++i) f(j, i);
      } else if (col(j) < C) {
#pragma unroll
        for (int i = 0; i < VE - 1; ++i)
          if (col(j) + i < C) f(j, i);
      }
    }
  }
  // the raw vectors, zeros past the row's end
  __device__ __forceinline__ void load(const T* row, u32x4* x) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = col(j);
      if (c + VE <= C) {
        x[j] = *reinterpret_cast<const typename Loose<T>::type*>(row + c);
      } else {
        x[j] = u32x4{0, 0, 0, 0};
        if (c < C) {
#pragma unroll
          for (int i = 0; i < VE - 1; ++i)
            if (c + i < C) {
              if constexpr (sizeof(T) == 4) x[j][i] = raw1(row + c + i);
              else x[j][i >> 1] |= raw1(row + c + i) << (16 * (i & 1));
            }
        }
      }
    }
  }
  static __device__ __forceinline__ float get(u32x4 x, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(x[i]);
    else return __uint_as_float(i & 1 ? x[i >> 1] & 0xFFFF0000u : x[i >> 1] << 16);
  }
  // vector j of results, rounded to T once
  __device__ __forceinline__ void store(T* row, int j, const float* v) const {
    const int c = col(j);
    if (c >= C) return;
    u32x4 o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
    }
    if (c + VE <= C) {
      *reinterpret_cast<typename Loose<T>::type*>(row + c) = o;
    } else {
#pragma unroll
      for (int i = 0; i < VE - 1; ++i)
        if (c + i < C) {
          if constexpr (sizeof(T) == 4) row[c + i] = v[i];
          else row[c + i] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
        }
    }
  }
  // NV vectors of parameters in fp32; `other` where there are none
  __device__ __forceinline__ void params(const float* p, float other, float (*w)[VE]) const {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VE; ++i) w[j][i] = p && col(j) + i < C ? p[col(j) + i] : other;
  }
};

// A barrier behind which LDS is seen; loads from memory stay under way.
__device__ __forceinline__ void sync_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}

__device__ __forceinline__ float sum16(float x) {
  x += dpp<0xB1>(x);          // xor 1
  x += dpp<0x4E>(x);          // xor 2
  x += dpp<0x141>(x);         // the other four of eight
  return x + dpp<0x140>(x);   // the other eight of sixteen
}

// N sums over a row: its LPR lanes, or (LPR == 0) the whole workgroup, whose wavefronts leave theirs in
// `red` (zeros where there is no wavefront). Every lane receives them.
constexpr int kWaves = 16;
template <int N>
struct Sums {
  float v[N];
};
template <int LPR, int N>
__device__ __forceinline__ Sums<N> reduce(Sums<N> a, Sums<N>* red) {
  constexpr int W = LPR ? LPR : 64;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float& x = a.v[i];
    x = sum16(x);
    if (W > 16) x += __shfl_xor(x, 16, 64);
    if (W > 32) x += __shfl_xor(x, 32, 64);
  }
  if constexpr (LPR == 0) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
    sync_lds();
    a = red[threadIdx.x & (kWaves - 1)];
#pragma unroll
    for (int i = 0; i < N; ++i) a.v[i] = sum16(a.v[i]);
  }
  return a;
}
// The places of wavefronts that a workgroup does not have.
template <int N>
__device__ __forceinline__ void clear_rest(Sums<N>* red) {
  const int k = (int)blockDim.x / 64 + threadIdx.x;
  if (k < kWaves)
#pragma unroll
    for (int i = 0; i < N; ++i) red[k].v[i] = 0.f;
}

// LPR lanes per row, 256 / LPR rows at a time (LPR == 0: the workgroup's threads, one row); workgroups
// stride over the rows with their parameters in registers, the next row on its way meanwhile. The
// variance is a second sum, of deviations: a sum of squares would lose the digits that a large mean takes. The
// deviations' own sum, which only the mean's rounding leaves, corrects both.
template <typename T, int NV, int LPR>
__global__ __launch_bounds__(LPR ? 256 : 1024) void norm_kernel(const T* __restrict__ x, int64_t ldx, int rows, int C,
                                                                const float* __restrict__ w,
                                                                const float* __restrict__ b, float eps,
                                                                T* __restrict__ y, int64_t ldy) {
  typedef Cols<T, NV> CL;
  constexpr int VE = CL::VE, RB = 256 / (LPR ? LPR : 256);
  __shared__ __attribute__((aligned(16))) Sums<1> red[2][kWaves];
  __shared__ __attribute__((aligned(16))) Sums<2> red2[2][kWaves];
  const int tid = threadIdx.x;
  const CL c = {C, LPR ? tid % (LPR ? LPR : 1) : tid, LPR ? LPR : (int)blockDim.x};
  float wv[NV][VE], bv[NV][VE];
  c.params(w, 1.f, wv);
  c.params(b, 0.f, bv);
  const float inv_C = 1.0f / (float)C;
  const int64_t own = LPR ? tid / (LPR ? LPR : 1) : 0, step = (int64_t)gridDim.x * RB;
  u32x4 next[NV];
  c.load(x + min((int64_t)blockIdx.x * RB + own, (int64_t)rows - 1) * ldx, next);
  if constexpr (LPR == 0)
    for (int k = 0; k < 2; ++k) {
      clear_rest(red[k]);
      clear_rest(red2[k]);
    }
  int phase = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * RB; r0 < rows; r0 += step, phase ^= 1) {
    const int64_t row = r0 + own;
    u32x4 xv[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) xv[j] = next[j];
    if (r0 + step < rows) c.load(x + min(row + step, (int64_t)rows - 1) * ldx, next);
    Sums<1> s = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VE; ++i) s.v[0] += CL::get(xv[j], i);  // (zeros past the end)
    const float m = reduce<LPR>(s, red[phase]).v[0] / (float)C;
    Sums<2> q = {0.f, 0.f};
    c.each([&](int j, int i) {
      const float d = CL::get(xv[j], i) - m;
      q.v[0] = fmaf(d, d, q.v[0]);
      q.v[1] += d;
    });
    q = reduce<LPR>(q, red2[phase]);
    const float more = q.v[1] * inv_C, r = 1.0f / sqrtf(fmaf(fmaf(-more, q.v[1], q.v[0]), inv_C, eps));
    if (row >= rows) continue;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float o[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) o[i] = fmaf(((CL::get(xv[j], i) - m) - more) * r, wv[j][i], bv[j][i]);
      c.store(y + row * ldy, j, o);
    }
  }
}

// The same rows backwards; sum g (x - m) comes with the variance, so there are two reductions here as well. Every
// thread keeps its columns' sums for dw and db over the rows that its workgroup takes; they leave as one partial
// vector per workgroup (part[block][2][C]).
template <typename T, int NV, int LPR>
__global__ __launch_bounds__(LPR ? 256 : 1024) void norm_bwd_kernel(const T* __restrict__ x, int64_t ldx, int rows,
                                                                    int C, const float* __restrict__ w, float eps,
                                                                    const T* __restrict__ dy, int64_t lddy,
                                                                    T* __restrict__ dx, int64_t lddx,
                                                                    float* __restrict__ part) {
  typedef Cols<T, NV> CL;
  constexpr int VE = CL::VE, RB = 256 / (LPR ? LPR : 256);
  __shared__ __attribute__((aligned(16))) Sums<2> red[2][kWaves];
  __shared__ __attribute__((aligned(16))) Sums<3> red2[2][kWaves];
  const int tid = threadIdx.x;
  const CL c = {C, LPR ? tid % (LPR ? LPR : 1) : tid, LPR ? LPR : (int)blockDim.x};
  float wv[NV][VE], dw[NV][VE], db[NV][VE];
  c.params(w, 1.f, wv);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VE; ++i) dw[j][i] = db[j][i] = 0.f;
  const float inv_C = 1.0f / (float)C;
  const int64_t own = LPR ? tid / (LPR ? LPR : 1) : 0, step = (int64_t)gridDim.x * RB;
  const int64_t first = min((int64_t)blockIdx.x * RB + own, (int64_t)rows - 1);
  u32x4 xn[NV], gn[NV];
  if constexpr (NV < 4) {
    c.load(x + first * ldx, xn);
    c.load(dy + first * lddy, gn);
  }
  if constexpr (LPR == 0)
    for (int k = 0; k < 2; ++k) {
      clear_rest(red[k]);
      clear_rest(red2[k]);
    }
  int phase = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * RB; r0 < rows; r0 += step, phase ^= 1) {
    const int64_t row = r0 + own;
    u32x4 xv[NV], gv[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      xv[j] = xn[j];
      gv[j] = gn[j];
    }
    if constexpr (NV == 4) {  // (no registers for the next row: 12,288 fp32 columns took 278 us, with spills, not 166)
      c.load(x + min(row, (int64_t)rows - 1) * ldx, xv);
      c.load(dy + min(row, (int64_t)rows - 1) * lddy, gv);
    } else if (r0 + step < rows) {
      const int64_t after = min(row + step, (int64_t)rows - 1);
      c.load(x + after * ldx, xn);
      c.load(dy + after * lddy, gn);
    }
    Sums<2> s = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        s.v[0] += CL::get(xv[j], i);  // (both are zero past the row's end)
        s.v[1] = fmaf(CL::get(gv[j], i), wv[j][i], s.v[1]);
      }
    s = reduce<LPR>(s, red[phase]);
    const float m = s.v[0] / (float)C, mg = s.v[1] * inv_C;
    Sums<3> q = {0.f, 0.f, 0.f};
    c.each([&](int j, int i) {
      const float d = CL::get(xv[j], i) - m;
      q.v[0] = fmaf(d, d, q.v[0]);
      q.v[1] += d;
      q.v[2] = fmaf(CL::get(gv[j], i) * wv[j][i], d, q.v[2]);
    });
    q = reduce<LPR>(q, red2[phase]);
    const float more = q.v[1] * inv_C, r = 1.0f / sqrtf(fmaf(fmaf(-more, q.v[1], q.v[0]), inv_C, eps));
    const float mgh = fmaf(-more, s.v[1], q.v[2]) * inv_C * r * r;  // (times r)
    if (row >= rows) continue;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float o[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float d = CL::get(gv[j], i), h = ((CL::get(xv[j], i) - m) - more) * r;
        o[i] = fmaf(r, fmaf(d, wv[j][i], -mg), -h * mgh);
        dw[j][i] = fmaf(d, h, dw[j][i]);
        db[j][i] += d;
      }
      c.store(dx + row * lddx, j, o);
    }
  }
  float* p = part + (int64_t)blockIdx.x * 2 * C;
  if constexpr (LPR) {
    // the rows' places of the workgroup together: lanes of a wavefront, then wavefronts
    __shared__ float sum[3][2][NV * VE][LPR];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VE; ++i)
#pragma unroll
        for (int o = LPR; o < 64; o *= 2) {
          dw[j][i] += __shfl_xor(dw[j][i], o, 64);
          db[j][i] += __shfl_xor(db[j][i], o, 64);
        }
    const int lane = tid & 63, wave = tid >> 6;
    if (wave > 0 && lane < LPR)
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          sum[wave - 1][0][j * VE + i][lane] = dw[j][i];
          sum[wave - 1][1][j * VE + i][lane] = db[j][i];
        }
    __syncthreads();
    if (wave > 0 || lane >= LPR) return;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VE; ++i)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          dw[j][i] += sum[k][0][j * VE + i][lane];
          db[j][i] += sum[k][1][j * VE + i][lane];
        }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VE; ++i)
      if (i < c.have(j)) {
        p[c.col(j) + i] = dw[j][i];
        p[C + c.col(j) + i] = db[j][i];
      }
}

// A row's vectors over the fewest lanes that hold it in one vector each, from 16 of them to a wavefront (two
// vectors up to 128); wider rows take a workgroup, of up to 1,024 threads, with a second vector a thread from 513
// on and four from 2,049. 2^26 entries, forward / backward in us: bf16 rows of 128 columns 55 / 85 on 16 lanes, 141 / 291
// on 64; of 4,096 (512 vectors) 53 / 92 with one vector a thread, 54 / 98 with two, which halve what the reductions
// cost but leave fewer wavefronts; of 5,120 55 / 93 with two, 72 / 119 with one; of 12,288 58 / 95 with two on 768
// threads, 95 / 120 with four on 384.
struct Shape {
  int nv, lpr;   // vectors per thread; lanes per row, 0: the workgroup
  int threads;
  int rows;      // at a time
};
Shape shape_of(bool bf16, int C) {
  const int v = (C + (bf16 ? 8 : 4) - 1) / (bf16 ? 8 : 4);
  if (v <= 16) return {1, 16, 256, 16};
  if (v <= 32) return {1, 32, 256, 8};
  if (v <= 64) return {1, 64, 256, 4};
  if (v <= 128) return {2, 64, 256, 4};
  const int nv = v <= 512 ? 1 : v <= 2048 ? 2 : 4;
  return {nv, 0, ((v + nv - 1) / nv + 63) / 64 * 64, 1};
}

// Workgroups: as many as are on a CU at once and no more (16,384 x 5,120 bf16: forward 69 us with 4 a CU, 80 with 6). For
// the gradients, whose every workgroup leaves a partial vector, still fewer: 113 us with 2 a CU, 131 with 3, and half the
// sums; with one vector a thread, whose rows need the most wavefronts, 3 (26,214 x 2,560 96, with 2 109).
int fwd_parts(const Shape& s, int rows) {
  return std::min((rows + s.rows - 1) / s.rows, 256 * std::max(1, (s.nv == 1 ? 2048 : 1280) / s.threads));
}
int bwd_parts(const Shape& s, int rows) {
  return std::min((rows + s.rows - 1) / s.rows, 256 * std::max(1, (s.lpr || s.nv > 1 ? 768 : 1024) / s.threads));
}

template <typename T, int NV, int LPR>
hipError_t fwd(const NormOp& a, const Shape& sh, void* y, int64_t ldy, hipStream_t s) {
  norm_kernel<T, NV, LPR><<<fwd_parts(sh, a.rows), sh.threads, 0, s>>>(static_cast<const T*>(a.x), a.ldx, a.rows, a.C, a.w, a.b, a.eps,
                                                      static_cast<T*>(y), ldy);
  return hipGetLastError();
}

template <typename T, int NV, int LPR>
hipError_t bwd(const NormOp& a, const Shape& sh, const void* dy, int64_t lddy, void* dx, int64_t lddx, float* part,
               hipStream_t s) {
  norm_bwd_kernel<T, NV, LPR><<<bwd_parts(sh, a.rows), sh.threads, 0, s>>>(
      static_cast<const T*>(a.x), a.ldx, a.rows, a.C, a.w, a.eps, static_cast<const T*>(dy), lddy, static_cast<T*>(dx),
      lddx, part);
  return hipGetLastError();
}

template <typename F>
hipError_t dispatch(const Shape& s, F f) {
  typedef std::integral_constant<int, 0> I0;
  typedef std::integral_constant<int, 1> I1;
  typedef std::integral_constant<int, 2> I2;
  typedef std::integral_constant<int, 4> I4;
  if (s.lpr == 16) return f(I1(), std::integral_constant<int, 16>());
  if (s.lpr == 32) return f(I1(), std::integral_constant<int, 32>());
  if (s.lpr == 64 && s.nv == 1) return f(I1(), std::integral_constant<int, 64>());
  if (s.lpr == 64) return f(I2(), std::integral_constant<int, 64>());
  if (s.nv == 1) return f(I1(), I0());
  if (s.nv == 2) return f(I2(), I0());
  return f(I4(), I0());
}

}  // namespace

hipError_t launch_layer_norm(const NormOp& a, void* y, int64_t ldy, hipStream_t s) {
  const Shape sh = shape_of(a.bf16, a.C);
  return dispatch(sh, [&](auto nv, auto lpr) {
    constexpr int NB = std::min(nv.value, 2);  // (bf16 rows have 2,048 vectors at most)
    return a.bf16 ? fwd<uint16_t, NB, lpr.value>(a, sh, y, ldy, s) : fwd<float, nv.value, lpr.value>(a, sh, y, ldy, s);
  });
}

size_t layer_norm_workspace_bytes(bool bf16, int rows, int C) {
  return (size_t)bwd_parts(shape_of(bf16, C), rows) * 2 * C * sizeof(float);
}

hipError_t launch_layer_norm_bwd(const NormOp& a, const void* dy, int64_t lddy, void* dx, int64_t lddx, float* dw,
                                 float* db, float* ws, hipStream_t s) {
  const Shape sh = shape_of(a.bf16, a.C);
  if (a.rows > 0) {
    const hipError_t e = dispatch(sh, [&](auto nv, auto lpr) {
      constexpr int NB = std::min(nv.value, 2);
      return a.bf16 ? bwd<uint16_t, NB, lpr.value>(a, sh, dy, lddy, dx, lddx, ws, s)
                    : bwd<float, nv.value, lpr.value>(a, sh, dy, lddy, dx, lddx, ws, s);
    });
    if (e != hipSuccess) return e;
  }
  sum_parts(ws, a.rows > 0 ? bwd_parts(sh, a.rows) : 0, 1, 2, a.C, dw, db, nullptr, s);
  return hipGetLastError();
}

}  // namespace tcl

// Layer norm over the columns of a row matrix, and its gradients:
//   m = mean x, r = (mean (x - m)^2 + eps)^-1/2, h = (x - m) r, y = h w + b,
//   dx = r (g - mean g - h mean(g h)), g = dy w,  dw = sum over rows dy h,  db = sum over rows dy.
// Nothing is kept from the forward call: the gradients read x anyway, and a row's statistics
// are one reduction of what is then in registers.
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

// Mean and sum of squared deviations of n values, and of two such sets together: no sum of
// squares is formed whose difference to the mean's square would lose digits.
struct Moments {
  float n, m, q;
};
__device__ __forceinline__ Moments join(Moments a, Moments b) {
  const float n = a.n + b.n, f = n > 0.f ? b.n / n : 0.f, d = b.m - a.m;
  return {n, fmaf(d, f, a.m), a.q + b.q + d * d * a.n * f};
}
__device__ __forceinline__ Moments shifted(Moments a, int o) {
  return {__shfl_xor(a.n, o, 64), __shfl_xor(a.m, o, 64), __shfl_xor(a.q, o, 64)};
}

// A row's reductions over LPR lanes of a wavefront, or (LPR == 0) the whole workgroup. `red` has
// room for the wavefronts' values twice over: rows alternate, so a row's readers and the
// next row's writers are one barrier apart.
template <int LPR>
__device__ __forceinline__ Moments reduce(Moments a, Moments* red) {
  constexpr int W = LPR ? LPR : 64;
  if constexpr (LPR == 0) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) a = join(a, shifted(a, o));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
    __syncthreads();
    a = red[0];
    for (int k = 1; k < (int)blockDim.x / 64; ++k) a = join(a, red[k]);
  } else {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) a = join(a, shifted(a, o));
  }
  return a;
}
template <int LPR>
__device__ __forceinline__ float2 reduce(float2 a, float2* red) {
  constexpr int W = LPR ? LPR : 64;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) {
    a.x += __shfl_xor(a.x, o, 64);
    a.y += __shfl_xor(a.y, o, 64);
  }
  if constexpr (LPR == 0) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
    __syncthreads();
    a = red[0];
    for (int k = 1; k < (int)blockDim.x / 64; ++k) a = {a.x + red[k].x, a.y + red[k].y};
  }
  return a;
}

template <typename T, int NV>
__device__ __forceinline__ Moments moments_of(const Cols<T, NV>& c, const u32x4* x) {
  constexpr int VE = Cols<T, NV>::VE;
  float n = 0.f, s = 0.f, q = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    n += (float)c.have(j);
#pragma unroll
    for (int i = 0; i < VE; ++i) s += Cols<T, NV>::get(x[j], i);  // (zeros past the end)
  }
  const float m = n > 0.f ? s / n : 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      const float d = i < c.have(j) ? Cols<T, NV>::get(x[j], i) - m : 0.f;
      q = fmaf(d, d, q);
    }
  return {n, m, q};
}

__device__ __forceinline__ float rstd_of(Moments a, float eps) { return 1.0f / sqrtf(a.q / a.n + eps); }

// LPR lanes per row, 256 / LPR rows at a time (LPR == 0: the workgroup's threads, one row); workgroups
// stride over the rows with their parameters in registers.
template <typename T, int NV, int LPR>
__global__ __launch_bounds__(LPR ? 256 : 1024) void norm_kernel(const T* __restrict__ x, int64_t ldx, int rows, int C,
                                                                const float* __restrict__ w,
                                                                const float* __restrict__ b, float eps,
                                                                T* __restrict__ y, int64_t ldy) {
  typedef Cols<T, NV> CL;
  constexpr int VE = CL::VE, RB = LPR ? 256 / LPR : 1;
  __shared__ Moments red[2][16];
  const int tid = threadIdx.x;
  const CL c = {C, LPR ? tid % (LPR ? LPR : 1) : tid, LPR ? LPR : (int)blockDim.x};
  float wv[NV][VE], bv[NV][VE];
  c.params(w, 1.f, wv);
  c.params(b, 0.f, bv);
  int phase = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * RB; r0 < rows; r0 += (int64_t)gridDim.x * RB, phase ^= 1) {
    const int64_t row = r0 + (LPR ? tid / (LPR ? LPR : 1) : 0);
    const bool live = row < rows;
    u32x4 xv[NV];
    c.load(x + (live ? row : r0) * ldx, xv);
    const Moments st = reduce<LPR>(moments_of(c, xv), red[phase]);
    const float r = rstd_of(st, eps);
    if (!live) continue;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float o[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) o[i] = fmaf((CL::get(xv[j], i) - st.m) * r, wv[j][i], bv[j][i]);
      c.store(y + row * ldy, j, o);
    }
  }
}

// The same rows backwards. Every thread keeps its columns' sums for dw and db over the rows
// that its workgroup takes; they leave as one partial vector per workgroup (part[block][2][C]).
template <typename T, int NV, int LPR>
__global__ __launch_bounds__(LPR ? 256 : 1024) void norm_bwd_kernel(const T* __restrict__ x, int64_t ldx, int rows,
                                                                    int C, const float* __restrict__ w, float eps,
                                                                    const T* __restrict__ dy, int64_t lddy,
                                                                    T* __restrict__ dx, int64_t lddx,
                                                                    float* __restrict__ part) {
  typedef Cols<T, NV> CL;
  constexpr int VE = CL::VE, RB = LPR ? 256 / LPR : 1;
  __shared__ Moments red[2][16];
  __shared__ float2 red2[2][16];
  const int tid = threadIdx.x;
  const CL c = {C, LPR ? tid % (LPR ? LPR : 1) : tid, LPR ? LPR : (int)blockDim.x};
  float wv[NV][VE], dw[NV][VE], db[NV][VE];
  c.params(w, 1.f, wv);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < VE; ++i) dw[j][i] = db[j][i] = 0.f;
  const float inv_C = 1.0f / (float)C;
  int phase = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * RB; r0 < rows; r0 += (int64_t)gridDim.x * RB, phase ^= 1) {
    const int64_t row = r0 + (LPR ? tid / (LPR ? LPR : 1) : 0);
    const bool live = row < rows;
    u32x4 xv[NV], gv[NV];
    c.load(x + (live ? row : r0) * ldx, xv);
    c.load(dy + (live ? row : r0) * lddy, gv);
    const Moments st = reduce<LPR>(moments_of(c, xv), red[phase]);
    const float r = rstd_of(st, eps);
    float2 s = {0.f, 0.f};  // sums of g and g h (dy is zero past the row's end)
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float g = CL::get(gv[j], i) * wv[j][i];
        s.x += g;
        s.y = fmaf(g, (CL::get(xv[j], i) - st.m) * r, s.y);
      }
    s = reduce<LPR>(s, red2[phase]);
    if (!live) continue;
    const float mg = s.x * inv_C, mgh = s.y * inv_C;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float o[VE];
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float d = CL::get(gv[j], i), h = (CL::get(xv[j], i) - st.m) * r;
        o[i] = r * (fmaf(d, wv[j][i], -mg) - h * mgh);
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

// A row's vectors over the fewest lanes that hold it in one vector each, from 16 of them to a
// wavefront; wider rows take a workgroup.
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
  const int nv = v <= 1024 ? 1 : v <= 2048 ? 2 : 4;
  return {nv, 0, ((v + nv - 1) / nv + 63) / 64 * 64, 1};
}

// Workgroups of the gradients: each leaves a partial vector, so no more than fill the GPU twice over.
int bwd_parts(const Shape& s, int rows) {
  const int fill = 256 * std::max(1, 2048 / s.threads);
  return std::min((rows + s.rows - 1) / s.rows, fill);
}

template <typename T, int NV, int LPR>
hipError_t fwd(const NormOp& a, const Shape& sh, void* y, int64_t ldy, hipStream_t s) {
  const int grid = std::min((a.rows + sh.rows - 1) / sh.rows, 256 * 8);
  norm_kernel<T, NV, LPR><<<grid, sh.threads, 0, s>>>(static_cast<const T*>(a.x), a.ldx, a.rows, a.C, a.w, a.b, a.eps,
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
    return a.bf16 ? fwd<uint16_t, nv.value, lpr.value>(a, sh, y, ldy, s) : fwd<float, nv.value, lpr.value>(a, sh, y, ldy, s);
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
      return a.bf16 ? bwd<uint16_t, nv.value, lpr.value>(a, sh, dy, lddy, dx, lddx, ws, s)
                    : bwd<float, nv.value, lpr.value>(a, sh, dy, lddy, dx, lddx, ws, s);
    });
    if (e != hipSuccess) return e;
  }
  sum_parts(ws, a.rows > 0 ? bwd_parts(sh, a.rows) : 0, 1, 2, a.C, dw, db, nullptr, s);
  return hipGetLastError();
}

}  // namespace tcl

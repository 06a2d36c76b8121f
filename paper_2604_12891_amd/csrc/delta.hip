// The gated delta rule with carried states: prompts, single tokens, gradients.
//
// Per value head, with a state S [Dk, Dv], each token does
//   S <- e^g S,  u = beta (v - S^T k),  S <- S + k u^T,  o = scale S^T q.
// A chunk of kC tokens with the state S0 in front of it, G_i = g_1 + .. + g_i, D_ij = e^(G_i - G_j) and
//   A_ij = beta_i D_ij k_i.k_j (j < i),  T = (I + A)^-1,  P_ij = scale D_ij q_i.k_j (j <= i)
// does the same as
//   R = beta (V - e^G K S0),  U = T R,  O = scale e^G Q S0 + P U,  S1 = e^G_C S0 + K^T (w U),  w_j = e^(G_C - G_j).
// T, P and the factors need no state: delta_prep_kernel forms them for all chunks at once, and what walks
// the chunks in order is left with matrix products. States do not mix their columns (Dv), so the walk is also
// spread over slices of them.
//
// G is summed and subtracted in 64 bits and its exponentials are taken of the differences: with g down to
// -inf, e^G_i / e^G_j would be 0 / 0 where D_ij is 1. A decay below e^-10000 counts as that.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "ops.h"
#include "packing.h"

namespace tcl {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kC = 64;        // tokens of a chunk
constexpr int kMat = kC * kC;        // entries of T or P
constexpr int kTParts = kMat / 2 * 3;  // floats that a matrix's three bf16 parts take
// Floats of a chunk's matrices in parts: T and P, or for the gradients T, T^T and P^T.
template <bool GRADS>
constexpr int kMats = (GRADS ? 3 : 2) * kTParts;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void st1(float* p, float v) { *p = v; }
__device__ __forceinline__ void st1(uint16_t* p, float v) { *p = f32_to_bf16(v); }

// Four neighbours of a row, widened, and back; rows start at any element.
typedef floatx4 floatx4_any __attribute__((aligned(4)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
__device__ __forceinline__ floatx4 ld4(const float* p) { return *reinterpret_cast<const floatx4_any*>(p); }
__device__ __forceinline__ floatx4 ld4(const uint16_t* p) {
  const u32x2 x = *reinterpret_cast<const u32x2_any*>(p);
  return floatx4{__uint_as_float(x[0] << 16), __uint_as_float(x[0] & 0xFFFF0000u), __uint_as_float(x[1] << 16),
                 __uint_as_float(x[1] & 0xFFFF0000u)};
}
__device__ __forceinline__ void st4(float* p, floatx4 v) { *reinterpret_cast<floatx4_any*>(p) = v; }
__device__ __forceinline__ void st4(uint16_t* p, floatx4 v) {
  *reinterpret_cast<u32x2_any*>(p) = u32x2{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
}

// e^x of a sum of logarithms in 64 bits, to an fp32 rounding or two.
__device__ __forceinline__ float exp_of(double x) {
  const double t = x * 1.4426950408889634;
  const double n = __builtin_rint(t);
  return ldexpf(__builtin_amdgcn_exp2f((float)(t - n)), n < -1000.0 ? -1000 : n > 1000.0 ? 1000 : (int)n);
}
__device__ __forceinline__ double log_decay(float g) { return g < -1e4f ? -1e4 : (double)g; }

// What lane `lane` of a wavefront has of an array at a wave-uniform address: a scalar base and a 32-bit offset (left
// to itself the compiler adds them up in vector registers); entries may start anywhere that their parts allow.
typedef __attribute__((address_space(1))) char gchar;
template <typename P>
__device__ __forceinline__ gchar* uniform(const P* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (gchar*)((uint64_t)hi << 32 | lo);
}
template <typename V, typename P>
__device__ __forceinline__ V at_lane(const P* p, int lane) {
  return *(const __attribute__((address_space(1))) V*)(uniform(p) + (uint32_t)(lane * (int)sizeof(V)));
}
template <typename V, typename P>
__device__ __forceinline__ V at_bytes(const P* p, uint32_t bytes) {
  return {*(const __attribute__((address_space(1))) typename V::loose*)(uniform(p) + bytes)};
}

struct DeltaIn {
  const int* offs;
  int n_seq, rows, Hk, H, Dk, Dv;
  int64_t ldq, ldk, ldv, ldg, ldb;
  const float *g, *beta;
  float scale;
  const float* state;
  const int* slots;
  int n_slots;
};

// ---------------------------------------------------------------- token by token
// A wavefront holds 32 columns of a head's state: lane l columns 4 (l / 8) .. + 3 of rows RK (l % 8) .. + RK - 1, so
// that sums over the rows are lanes' neighbours (DPP) and a state's lines are read whole. With
// p = S^T k and r = S^T q of the state before the token,
//   u = beta (v - a p),  o = scale (a r + (k.q) u),  S <- a S + k u^T:
// one reduction per token. Single tokens are bound by the states' bytes (192 x 32 heads of 128 x 128: 172 us for 805 MB,
// the rate of a large copy); sequences by the chain of a token's products, reduction and update (1.1 us a token, 0.5 for
// 64 x 64).
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float sum8(float v) {
  v += dpp<0xB1>(v);   // xor 1
  v += dpp<0x4E>(v);   // xor 2
  return v + dpp<0x141>(v);  // the other four of eight
}

template <typename T, int RK>
__global__ __launch_bounds__(64) void delta_walk_kernel(DeltaIn a, const T* __restrict__ q, const T* __restrict__ k,
                                                        const T* __restrict__ v, float* state_out, T* __restrict__ o,
                                                        int64_t ldo) {
  const int lane = threadIdx.x, kg = lane & 7, parts = (a.Dv + 31) / 32;
  const int h = (int)(blockIdx.x / parts % a.H), seq = (int)(blockIdx.x / parts / a.H);
  const int c = (int)(blockIdx.x % parts) * 32 + (lane >> 3) * 4, r0 = kg * RK;
  const bool live = c < a.Dv;
  int base = seq, len = 1;
  if (a.offs) {
    base = min(max(a.offs[seq], 0), a.rows);
    len = min(max(a.offs[seq + 1], base), a.rows) - base;
  }
  const int slot = slot_of(a.slots, a.n_slots, seq);
  const int64_t at = (((int64_t)slot * a.H + h) * a.Dk + r0) * a.Dv + c;
  floatx4 s[RK];
#pragma unroll
  for (int i = 0; i < RK; ++i) {
    s[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (a.state && slot >= 0 && live && r0 + i < a.Dk)
      s[i] = *reinterpret_cast<const floatx4*>(a.state + at + (int64_t)i * a.Dv);
  }
  const int hk = h / (a.H / a.Hk);
  const T* kp = k + base * a.ldk + (int64_t)hk * a.Dk + r0;
  const T* qp = q + base * a.ldq + (int64_t)hk * a.Dk + r0;
  const T* vp = v + base * a.ldv + (int64_t)h * a.Dv + c;
  const float* gp = a.g + base * a.ldg + h;
  const float* bp = a.beta + base * a.ldb + h;
  T* op = o + base * ldo + (int64_t)h * a.Dv + c;
  floatx4 kn[RK / 4], qn[RK / 4], vn = {0.f, 0.f, 0.f, 0.f};
  float gn = 0.f, bn = 0.f;
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < RK / 4; ++i) {
      kn[i] = qn[i] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (r0 + 4 * i < a.Dk) {
        kn[i] = ld4(kp + t * a.ldk + 4 * i);
        qn[i] = ld4(qp + t * a.ldq + 4 * i);
      }
    }
    if (live) vn = ld4(vp + t * a.ldv);
    gn = gp[t * a.ldg];
    bn = bp[t * a.ldb];
  };
  if (len > 0) fetch(0);
  for (int t = 0; t < len; ++t) {
    floatx4 kv[RK / 4], qv[RK / 4];
    const floatx4 vv = vn;
    const float dec = exp_of(log_decay(gn)), beta = bn;
#pragma unroll
    for (int i = 0; i < RK / 4; ++i) {
      kv[i] = kn[i];
      qv[i] = qn[i];
    }
    if (t + 1 < len) fetch(t + 1);
    floatx4 p = {0.f, 0.f, 0.f, 0.f}, r = p;
    float kq = 0.f;
#pragma unroll
    for (int i = 0; i < RK; ++i) {
      const float ki = kv[i / 4][i % 4], qi = qv[i / 4][i % 4];
      kq = fmaf(ki, qi, kq);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        p[j] = fmaf(s[i][j], ki, p[j]);
        r[j] = fmaf(s[i][j], qi, r[j]);
      }
    }
    kq = sum8(kq);
    floatx4 u, out;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u[j] = beta * fmaf(-dec, sum8(p[j]), vv[j]);
      out[j] = a.scale * fmaf(kq, u[j], dec * sum8(r[j]));
    }
#pragma unroll
    for (int i = 0; i < RK; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i][j] = fmaf(kv[i / 4][i % 4], u[j], dec * s[i][j]);
    if (kg == 0 && live) st4(op + t * ldo, out);
  }
  if (state_out && slot >= 0 && live)
#pragma unroll
    for (int i = 0; i < RK; ++i)
      if (r0 + i < a.Dk) *reinterpret_cast<floatx4*>(state_out + at + (int64_t)i * a.Dv) = s[i];
}

// A barrier behind which what the workgroup has written to LDS is seen; loads from memory stay under way.
__device__ __forceinline__ void sync_lds() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The same for a wavefront with itself: its lanes' writes in front of its lanes' reads.
__device__ __forceinline__ void sync_wave() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// ---------------------------------------------------------------- matrix products
// v_mfma_f32_16x16x4_f32: lane l holds A[l % 16][l / 16], B[l / 16][l % 16] and D[4 (l / 16) + r][l % 16]. The
// order of the k's is free, so four steps share one 16-byte read where k runs along memory: a
// fragment of 16 k's is, in lane l, the four entries k = 4 (l / 16) .. + 3 of its row.
__device__ __forceinline__ floatx4 mma16(floatx4 a, floatx4 b, floatx4 c) {
#pragma unroll
  for (int m = 0; m < 4; ++m) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[m], b[m], c, 0, 0, 0);
  return c;
}
// Fragment s of the 16 rows at p (leading dimension ld, in LDS): k along memory, or (frag_t) along the rows.
__device__ __forceinline__ floatx4 frag(const float* p, int ld, int s) {
  const int l = threadIdx.x & 63;
  return *reinterpret_cast<const floatx4*>(p + (l & 15) * ld + 16 * s + 4 * (l >> 4));
}
__device__ __forceinline__ floatx4 frag_t(const float* p, int ld, int s) {
  const int l = threadIdx.x & 63;
  const float* q = p + (16 * s + 4 * (l >> 4)) * ld + (l & 15);
  return floatx4{q[0], q[ld], q[2 * ld], q[3 * ld]};
}
// fp32-level products on the bf16 matrix cores: a value is a sum of three bf16 parts, each 2^-8 of the one in
// front (split3_pair), and of two values' nine products of parts the six down to 2^-16 count. What is bf16 in memory
// is one part; what is computed has three behind bf16 results too, whose terms may cancel (two, to 2^-16, behind answers, dQ
// and dK: a prompt of 8,032 tokens 308 us instead of 326, gradients 411 instead of 415). v_mfma_f32_16x16x32_bf16: lane l holds A[l % 16] and B[..][l % 16] at eight k's (which eight of the
// 32 is free, the same for both) and D[4 (l / 16) + r][l % 16]. Against v_mfma_f32_16x16x4_f32 a product takes an
// eighth of the cycles with one exact operand (three products), a third to a half with six.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
template <int N>
struct Parts {
  bf16x8 p[N];
};
__device__ __forceinline__ bf16x8 pack8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
template <int N>
__device__ __forceinline__ Parts<N> split8(floatx4 a, floatx4 b) {
  u32x4 h, m, l;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t x, y, z;
    split3_pair(a[2 * i], a[2 * i + 1], x, y, z);
    h[i] = x; m[i] = y; l[i] = z;
    split3_pair(b[2 * i], b[2 * i + 1], x, y, z);
    h[2 + i] = x; m[2 + i] = y; l[2 + i] = z;
  }
  Parts<N> r;
  r.p[0] = pack8(h);
  if constexpr (N > 1) r.p[1] = pack8(m);
  if constexpr (N > 2) r.p[2] = pack8(l);
  return r;
}
// Four neighbours' parts into LDS, part p at base + p * stride (bf16 entries).
template <int N>
__device__ __forceinline__ void put_parts(uint16_t* base, int stride, floatx4 v) {
  u32x2 w[3];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t x, y, z;
    split3_pair(v[2 * i], v[2 * i + 1], x, y, z);
    w[0][i] = x; w[1][i] = y; w[2][i] = z;
  }
#pragma unroll
  for (int p = 0; p < N; ++p) *reinterpret_cast<u32x2*>(base + p * stride) = w[p];
}
template <int N>
__device__ __forceinline__ Parts<N> get_parts(const uint16_t* base, int stride) {
  Parts<N> r;
#pragma unroll
  for (int p = 0; p < N; ++p) r.p[p] = pack8(*reinterpret_cast<const u32x4*>(base + p * stride));
  return r;
}
// Sums by the products' order, the smaller ones apart (and three chains of dependent instructions, not one).
struct Acc {
  floatx4 v[3];
  __device__ __forceinline__ void clear() { v[0] = v[1] = v[2] = floatx4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ floatx4 sum() const { return v[0] + (v[1] + v[2]); }
};
template <int NA, int NB>
__device__ __forceinline__ void mma32(const Parts<NA>& a, const Parts<NB>& b, Acc& c) {
#pragma unroll
  for (int i = 0; i < NA; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (i + j <= 2) c.v[i + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[j], c.v[i + j], 0, 0, 0);
}
// The same into one accumulator, where registers are short.
template <int NA, int NB>
__device__ __forceinline__ void mma32(const Parts<NA>& a, const Parts<NB>& b, floatx4& c) {
#pragma unroll
  for (int o = 2; o >= 0; --o)
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (o - i >= 0 && o - i < NB) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[o - i], c, 0, 0, 0);
}
// Four values' parts, each for itself.
template <int N>
struct Parts4 {
  u32x2 w[N];
  __device__ __forceinline__ uint16_t get(int part, int i) const { return (uint16_t)(w[part][i >> 1] >> (16 * (i & 1))); }
};
template <int N>
__device__ __forceinline__ Parts4<N> split4(floatx4 v) {
  Parts4<N> r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t x, y, z;
    split3_pair(v[2 * i], v[2 * i + 1], x, y, z);
    r.w[0][i] = x;
    if constexpr (N > 1) r.w[1][i] = y;
    if constexpr (N > 2) r.w[2][i] = z;
  }
  return r;
}
// Eight neighbours of a row as they are in memory.
template <typename T> struct Raw8;
template <> struct Raw8<uint16_t> {
  u32x4 v;
  typedef u32x4 any __attribute__((aligned(2)));
  __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const any*>(p); }
  // what lane `lane` has of an operand, eight entries each
  __device__ __forceinline__ void load_lane(const uint16_t* p, int lane) { v = at_lane<u32x4>(p, lane); }
  __device__ __forceinline__ void clear() { v = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ Parts<1> parts() const { return {{pack8(v)}}; }
};
template <> struct Raw8<float> {
  floatx4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = ld4(p); b = ld4(p + 4); }
  __device__ __forceinline__ void load_lane(const float* p, int lane) {
    a = at_lane<floatx4>(p, 2 * lane);
    b = at_lane<floatx4>(p, 2 * lane + 1);
  }
  __device__ __forceinline__ void clear() { a = b = floatx4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ Parts<3> parts() const { return split8<3>(a, b); }
};
// Four neighbours of a row as they are in memory.
template <typename T> struct Raw4;
template <> struct Raw4<uint16_t> {
  u32x2 v;
  typedef u32x2_any loose;
  __device__ __forceinline__ void load(const uint16_t* p) { v = *reinterpret_cast<const u32x2_any*>(p); }
  __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<u32x2_any*>(p) = v; }
};
template <> struct Raw4<float> {
  floatx4 v;
  typedef floatx4_any loose;
  __device__ __forceinline__ void load(const float* p) { v = ld4(p); }
  __device__ __forceinline__ void store(float* p) const { st4(p, v); }
};
__device__ __forceinline__ floatx4 widen(Raw4<float> x) { return x.v; }
__device__ __forceinline__ floatx4 widen(Raw4<uint16_t> x) {
  return floatx4{__uint_as_float(x.v[0] << 16), __uint_as_float(x.v[0] & 0xFFFF0000u), __uint_as_float(x.v[1] << 16),
                 __uint_as_float(x.v[1] & 0xFFFF0000u)};
}
// In products over tokens, the eight of lane group kq of the 32 from 32 s on: 32 s + 16 a + 4 kq + m at
// place 4 a + m. So the four tokens of a lane's results are neighbours in LDS, and two fragments (frag) of a
// matrix are one operand. Where token t = 16 w + 4 lk stands:
__device__ __forceinline__ int token_place(int w, int lk) { return 32 * (w >> 1) + 8 * lk + 4 * (w & 1); }
// A triangular matrix [kC, kC] as operands over tokens in N parts: of the 16 rows 16 w .., tokens 32 s ... (What is
// zero is not read, but an address is given for it too: a branch would hide from the compiler how many loads are
// under way, and it would wait for all.)
template <int N>
__device__ __forceinline__ Parts<N> mat_parts(const uint16_t* m, int w, int s) {
  Parts<N> r;
#pragma unroll
  for (int p = 0; p < N; ++p)
    r.p[p] = pack8(*reinterpret_cast<const u32x4*>(m + (((w * 2 + s) * N + p) * 64 + (threadIdx.x & 63)) * 8));
  return r;
}
template <int N>
__device__ __forceinline__ void put_mat(uint16_t* m, int w, int s, floatx4 a, floatx4 b) {
  const Parts<N> v = split8<N>(a, b);
#pragma unroll
  for (int p = 0; p < N; ++p)
    *reinterpret_cast<u32x4*>(m + (((w * 2 + s) * N + p) * 64 + (threadIdx.x & 63)) * 8) =
        __builtin_bit_cast(u32x4, v.p[p]);
}

// A chunk of a sequence: its first row and how many tokens it has.
struct Chunk {
  int row, n;
};

// Of a head's rows in a chunk the 16 tokens 16 w .. as operands of 32 k's, as they are in memory, D wide (a multiple of
// 8), zeros elsewhere.
template <typename T, int NS>
__device__ __forceinline__ void row_raw(const T* p, int64_t ld, Chunk c, int w, int D, Raw8<T>* f) {
  const int l = threadIdx.x & 63, t = 16 * w + (l & 15), k0 = 8 * (l >> 4);
  const T* q = p + (c.row + min(t, c.n - 1)) * ld + k0;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    f[s].clear();
    if (t < c.n && 32 * s + k0 < D) f[s].load(q + 32 * s);
  }
}

// ---------------------------------------------------------------- what needs no state
// T and P (or, for the gradients, T, T^T and P^T) as fragments and beta, e^G and w of every chunk, a
// workgroup per chunk and key head, which goes through the value heads that share it (or, where chunks are few, `parts`
// workgroups that share them out). Each of four
// wavefronts has 16 rows. T: the diagonal blocks of 16 by substitution, a column per lane, then blocks of
// 32 and 64 by products, T21 = -T22 A21 T11. Bound by what it writes, the matrices in parts above all: 126 chunks of 32
// heads (16 key heads) in bf16, 251 MB, 81 to 85 us; a chain of ten barriers a head hides only under the other workgroups of
// a CU (with room for fewer, 105).
constexpr int kLdM = kC + 4;

template <typename T, int DKP, bool GRADS>
__global__ __launch_bounds__(256, (sizeof(T) == 4 && DKP == 128 ? 2 : 4)) void delta_prep_kernel(DeltaIn a, const T* __restrict__ q, const T* __restrict__ k,
                                                         float* __restrict__ mats, float* __restrict__ coef,
                                                         T* __restrict__ ops, float* __restrict__ prods, int parts) {
  __shared__ __attribute__((aligned(16))) float sA[kC * kLdM], sT[kC * kLdM], sX[32 * 36];
  __shared__ double sG[kC];
  __shared__ float sB[kC];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = blockIdx.x % parts, tile = blockIdx.x / parts / a.Hk, hk = blockIdx.x / parts % a.Hk;
  const Tile tl = find_tile(a.offs, a.n_seq, a.rows, kC, tile);
  if (tl.seq < 0 || tl.len == 0) return;
  const Chunk c = {tl.base + tl.j * kC, min(kC, tl.len - tl.j * kC)};
  constexpr int NS = DKP / 32;
  const T* kp = k + (int64_t)hk * a.Dk;
  // products of rows: lane's entries, of row 16 w + li with key 16 t + 4 lk + r
  floatx4 kk[4], qk[4];
  Raw8<T> kf[NS], qf[NS];
  row_raw<T, NS>(kp, a.ldk, c, w, a.Dk, kf);
  row_raw<T, NS>(q + (int64_t)hk * a.Dk, a.ldq, c, w, a.Dk, qf);
  {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      kk[t] = qk[t] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (t > w || 16 * t >= c.n) continue;
      Raw8<T> bf[NS];
      row_raw<T, NS>(kp, a.ldk, c, t, a.Dk, bf);
      Acc x, y;
      x.clear();
      y.clear();
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const auto b = bf[s].parts();
        mma32(b, kf[s].parts(), x);
        mma32(b, qf[s].parts(), y);
      }
      kk[t] = x.sum();
      qk[t] = y.sum();
    }
  }
  const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
  if (GRADS && part == 0) {  // they are wanted again: forming them anew takes 22 us, writing them 2
    floatx4* out = reinterpret_cast<floatx4*>(prods) + ((int64_t)tile * a.Hk + hk) * (2 * kMat / 4);
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (t <= w) {
        out[(w * 4 + t) * 64 + lane] = qk[t];
        out[kMat / 4 + (w * 4 + t) * 64 + lane] = kk[t];
      }
  }
  // K, Q (for the gradients Q^T) and K^T as operands: a chunk's rows are a model's width apart, and every slice of every head that
  // reads them so would ask one channel of the cache for all of them
  if (part == 0) {
    T* out = ops + ((int64_t)tile * a.Hk + hk) * 3 * DKP * kC;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      *reinterpret_cast<Raw8<T>*>(out + ((w * NS + s) * 64 + lane) * 8) = kf[s];
      if constexpr (!GRADS) *reinterpret_cast<Raw8<T>*>(out + DKP * kC + ((w * NS + s) * 64 + lane) * 8) = qf[s];
    }
    auto across = [&](const T* m, int64_t ld, T* to) {  // a chunk's rows as operands over tokens
#pragma unroll
      for (int f = w; f < DKP / 16 * 2; f += 4) {
        const int col = 16 * (f >> 1) + li;
        alignas(16) T v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = 32 * (f & 1) + 16 * (i >> 2) + 4 * lk + (i & 3);
          v[i] = t < c.n && col < a.Dk ? m[(c.row + t) * ld + col] : T(0);
        }
        Raw8<T> x;
        x.load(v);
        *reinterpret_cast<Raw8<T>*>(to + (f * 64 + lane) * 8) = x;
      }
    };
    across(kp, a.ldk, out + 2 * DKP * kC);
    if constexpr (GRADS) across(q + (int64_t)hk * a.Dk, a.ldq, out + DKP * kC);
  }
  const int share = a.H / a.Hk;
  for (int hv = part; hv < share; hv += parts) {
    const int h = hk * share + hv;
    float* out = mats + ((int64_t)tile * a.H + h) * kMats<GRADS>;
    float* co = coef + ((int64_t)tile * a.H + h) * 3 * kC;
    // (as if it were another thread for every head: addresses formed once for all heads would not fit the registers)
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, li = lane & 15, lk = lane >> 4;
    __syncthreads();
    if (tid < kC) {
      // past the chunk's end nothing decays and nothing is written
      double G = tid < c.n ? log_decay(a.g[(c.row + tid) * a.ldg + h]) : 0.0;
      const float beta = tid < c.n ? a.beta[(c.row + tid) * a.ldb + h] : 0.f;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double up = __shfl_up(G, o, 64);
        if (tid >= o) G += up;
      }
      sG[tid] = G;
      sB[tid] = beta;
      const double end = __shfl(G, kC - 1, 64);
      co[tid] = beta;
      co[kC + tid] = exp_of(G);
      co[2 * kC + tid] = exp_of(end - G);
    }
    for (int i = tid; i < kC * kLdM; i += 256) sT[i] = 0.f;
    __syncthreads();
    floatx4 pm[4];
    {
      const int i = 16 * w + li;
      const double Gi = sG[i];
      const float bi = sB[i];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        floatx4 am;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = 16 * t + 4 * lk + r;
          const float d = j <= i ? exp_of(Gi - sG[j]) : 0.f;
          am[r] = j < i ? bi * d * kk[t][r] : 0.f;
          pm[t][r] = j <= i ? a.scale * d * qk[t][r] : 0.f;
        }
        *reinterpret_cast<floatx4*>(sA + i * kLdM + 16 * t + 4 * lk) = am;
      }
    }
    __syncthreads();
    {  // diagonal block w, column li (four lanes do the same)
      const float* A = sA + 16 * w * kLdM + 16 * w;
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float v = i == li ? 1.f : 0.f;
#pragma unroll
        for (int j = 0; j < i; ++j) v = fmaf(-A[i * kLdM + j], x[j], v);
        x[i] = v;
      }
      if (lk == 0)
#pragma unroll
        for (int i = 0; i < 16; ++i) sT[(16 * w + i) * kLdM + 16 * w + li] = x[i];
    }
    __syncthreads();
    const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
    if (w < 2) {  // blocks of 32, a wavefront each
      const int b = 32 * w;
      const floatx4 x = mma16(frag(sA + (b + 16) * kLdM + b, kLdM, 0), frag_t(sT + b * kLdM + b, kLdM, 0), zero);
#pragma unroll
      for (int r = 0; r < 4; ++r) sX[(16 * w + 4 * lk + r) * 36 + li] = x[r];
    }
    __syncthreads();
    if (w < 2) {
      const int b = 32 * w;
      const floatx4 x = mma16(frag(sT + (b + 16) * kLdM + b + 16, kLdM, 0), frag_t(sX + 16 * w * 36, 36, 0), zero);
#pragma unroll
      for (int r = 0; r < 4; ++r) sT[(b + 16 + 4 * lk + r) * kLdM + b + li] = -x[r];
    }
    __syncthreads();
    const int bi = 16 * (w >> 1), bj = 16 * (w & 1);  // the block of 32, a tile per wavefront
    {
      floatx4 x = zero;
#pragma unroll
      for (int s = 0; s < 2; ++s)
        x = mma16(frag(sA + (32 + bi) * kLdM, kLdM, s), frag_t(sT + bj, kLdM, s), x);
#pragma unroll
      for (int r = 0; r < 4; ++r) sX[(bi + 4 * lk + r) * 36 + bj + li] = x[r];
    }
    __syncthreads();
    {
      floatx4 x = zero;
#pragma unroll
      for (int s = 0; s < 2; ++s)
        x = mma16(frag(sT + (32 + bi) * kLdM + 32, kLdM, s), frag_t(sX + bj, 36, s), x);
#pragma unroll
      for (int r = 0; r < 4; ++r) sT[(32 + bi + 4 * lk + r) * kLdM + bj + li] = -x[r];
    }
    __syncthreads();  // P to where A was
#pragma unroll
    for (int t = 0; t < 4; ++t) *reinterpret_cast<floatx4*>(sA + (16 * w + li) * kLdM + 16 * t + 4 * lk) = pm[t];
    __syncthreads();
    uint16_t* tp = reinterpret_cast<uint16_t*>(out);
    if constexpr (GRADS) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s < w >> 1) continue;  // (zeros)
        put_mat<3>(tp + 2 * kTParts, w, s, frag_t(sT + 16 * w, kLdM, 2 * s), frag_t(sT + 16 * w, kLdM, 2 * s + 1));
        put_mat<3>(tp + 4 * kTParts, w, s, frag_t(sA + 16 * w, kLdM, 2 * s), frag_t(sA + 16 * w, kLdM, 2 * s + 1));
      }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (2 * s > w) continue;
      put_mat<3>(tp, w, s, frag(sT + 16 * w * kLdM, kLdM, 2 * s), frag(sT + 16 * w * kLdM, kLdM, 2 * s + 1));
      if constexpr (!GRADS)
        put_mat<3>(tp + 2 * kTParts, w, s, frag(sA + 16 * w * kLdM, kLdM, 2 * s),
                   frag(sA + 16 * w * kLdM, kLdM, 2 * s + 1));
    }
  }
}

// ---------------------------------------------------------------- the walk over chunks
// Workgroup b of n heads (of sequences) x parts: neighbours in b go to the eight XCDs in turn, and the slices of a
// head, which read the same keys and matrices, stay on one.
__device__ __forceinline__ void head_and_part(int b, int heads, int parts, int& head, int& part) {
  const int whole = heads / 8 * 8 * parts;
  if (b < whole) {
    head = b / (8 * parts) * 8 + b % 8;
    part = b / 8 % parts;
  } else {
    head = (b - whole) / parts + heads / 8 * 8;
    part = (b - whole) % parts;
  }
}

// Where entry k of row r (of 16) is in an array of D to a row: the eights of a row change places with the row, so that a
// column of eights is in different banks (rows 8 entries longer instead: conflicts in 18% of the walk's cycles, not 6%).
template <int D>
__device__ __forceinline__ int swap8(int r, int k) {
  return r * D + ((((k >> 3) ^ (D == 128 ? r : r >> 1)) & (D / 8 - 1)) << 3) + (k & 7);
}

// A workgroup per sequence, value head and slice of 16 columns. The parts of the state in LDS, [column][row],
// feed the products; the state itself stays in registers, tiles of 16 rows to a wavefront. Three barriers a chunk
// make three phases. Four wavefronts of 16 tokens each form R (K S0), then U (T R); four more the answers of
// the chunk before (P U), then Q S0, then the new state. So each SIMD has two to issue from, and LDS, whose 128
// bytes a cycle every product's operands share, is asked evenly. What
// the next chunk reads from memory is asked for as soon as its registers are free. SAVE (for the gradients): the states in
// front of the chunks and U are kept, no answers are formed, by the first four alone. Bound by the chain of a chunk's three
// phases: 126 chunks of 32 heads of 128 x 128 (one workgroup a CU) in 253 to 266 us, 2.0 a chunk, the matrix cores 19% busy,
// the vector units 25%. (With two parts behind bf16 answers, 237: then out of registers alone, without a load, 172, and with
// all the work on four wavefronts 336.)
template <typename T, int DKP, bool SAVE>
__global__ __launch_bounds__(SAVE ? 256 : 512) void delta_chunk_kernel(
    DeltaIn a, const T* __restrict__ v, const float* __restrict__ mats, const float* __restrict__ coef,
    const T* __restrict__ ops, float* state_out, T* __restrict__ o, int64_t ldo,
    float* __restrict__ s0, float* __restrict__ us) {
  constexpr int NW = SAVE ? 4 : 8, NT = DKP / 64;
  constexpr int NS = DKP / 32;
  __shared__ __attribute__((aligned(16))) uint16_t sS[3 * 16 * DKP], sR[3 * 16 * kC], sW[3 * 16 * kC], sU[3 * 16 * kC];
  // a wavefront's tokens' values and answers, on their way between rows in memory and columns in registers
  constexpr int LV = 20;
  __shared__ __attribute__((aligned(16))) T sV[NW][16 * LV];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), w = wv & 3;
  const bool answers = wv >= 4, tiles = SAVE || answers;  // what the wavefront is for
  const int parts = (a.Dv + 15) / 16;
  int head, part;
  head_and_part(blockIdx.x, a.n_seq * a.H, parts, head, part);
  const int c0 = part * 16, h = head % a.H, seq = head / a.H, hk = h / (a.H / a.Hk);
  const int base = min(max(a.offs ? a.offs[seq] : seq, 0), a.rows),
            len = a.offs ? min(max(a.offs[seq + 1], base), a.rows) - base : 1;
  const int key = !a.offs || kC > a.rows ? seq : base / kC + seq;
  const int slot = slot_of(a.slots, a.n_slots, seq);
  const bool col = c0 + li < a.Dv;  // the lane's column
  const int64_t size = (int64_t)a.Dk * a.Dv;
  const int place = token_place(w, lk);
  // state entries [16 (NT w + n) + 4 lk + r][c0 + li]
  floatx4 st[NT];
  auto at = [&](int n) { return (int64_t)(16 * (NT * w + n) + 4 * lk) * a.Dv + c0 + li; };
  auto in = [&](int n) { return tiles && 16 * (NT * w + n) + 4 * lk < a.Dk && col; };
  auto keep = [&](float* p, int n) {
    if (in(n))
#pragma unroll
      for (int r = 0; r < 4; ++r) p[at(n) + (int64_t)r * a.Dv] = st[n][r];
  };
  auto share = [&]() {
#pragma unroll
    for (int n = 0; n < NT; ++n) put_parts<3>(sS + swap8<DKP>(li, 16 * (NT * w + n) + 4 * lk), 16 * DKP, st[n]);
  };
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    st[n] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (a.state && slot >= 0 && in(n))
#pragma unroll
      for (int r = 0; r < 4; ++r) st[n][r] = a.state[((int64_t)slot * a.H + h) * size + at(n) + (int64_t)r * a.Dv];
  }
  if (tiles) share();
  const int chunks = (len + kC - 1) / kC;
  auto chunk = [&](int ch) { return Chunk{base + ch * kC, min(kC, len - ch * kC)}; };
  auto mat = [&](int ch) {
    return reinterpret_cast<const uint16_t*>(mats + ((int64_t)(key + ch) * a.H + h) * kMats<SAVE>);
  };
  Raw8<T> rf[NS], ktf[NT][2];
  Parts<3> tf[2];
  Parts<3> pf[2];
  floatx4 beta, e, wj;
  Raw4<T> vv;
  const int ldv = (int)a.ldv, cv = c0 + 4 * (lane & 3), tv = 16 * w + lane / 4;
  auto op = [&](int ch, int i) { return ops + (((int64_t)(key + ch) * a.Hk + hk) * 3 + i) * DKP * kC; };
  auto load_rows = [&](int ch) {
    const T* r = op(ch, answers ? 1 : 0);
#pragma unroll
    for (int s = 0; s < NS; ++s) rf[s] = *reinterpret_cast<const Raw8<T>*>(r + (uint32_t)(((w * NS + s) * 64 + lane) * 8));
  };
  // (rows past a chunk's end, and columns past a row's, are read as the last ones: the first meet a beta of zero, the
  // others' results are not kept)
  auto load_v = [&](int ch) {
    const Chunk c = chunk(ch);
    const T* vr = v + c.row * a.ldv + (int64_t)h * a.Dv;
    vv.load(vr + (uint32_t)(min(tv, c.n - 1) * ldv + min(cv, a.Dv - 4)));
  };
  auto factor = [&](int ch, int i) {
    return *reinterpret_cast<const floatx4*>(coef + ((int64_t)(key + ch) * a.H + h) * 3 * kC + i * kC + 16 * w + 4 * lk);
  };
  const int s1 = w >> 1;  // the last 32 tokens that the wavefront's rows of T and P reach
  auto load_t = [&](int ch) {
    tf[0] = mat_parts<3>(mat(ch), w, 0);
    tf[1] = mat_parts<3>(mat(ch), w, s1);
  };
  auto load_p = [&](int ch) {
    pf[0] = mat_parts<3>(mat(ch) + 2 * kTParts, w, 0);
    pf[1] = mat_parts<3>(mat(ch) + 2 * kTParts, w, s1);
  };
  auto load_kt = [&](int ch) {
    const T* p = op(ch, 2);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int s = 0; s < 2; ++s)
        ktf[n][s] = *reinterpret_cast<const Raw8<T>*>(p + (uint32_t)(((2 * (NT * w + n) + s) * 64 + lane) * 8));
  };
  // One loop for each kind of wavefront, with the same barriers: where both shared one, the compiler could not tell
  // which loads are under way and waited for all of them (as many us again).
  auto walk = [&](auto kind) {
    constexpr bool A = decltype(kind)::value;  // answers and (always where there are no others) the state
    constexpr bool B = !A;
    // (in the order of their first use, here and below: loads come back in order)
    load_rows(0);
    if constexpr (B) {
      load_v(0);
      beta = factor(0, 0);
      e = factor(0, 1);
      load_t(0);
      wj = factor(0, 2);
    }
    if constexpr (A || SAVE) load_kt(0);
    if constexpr (A) {
      load_p(0);
      e = factor(0, 1);
    }
    sync_lds();
    T* mine = sV[wv];
    Acc acc;
    floatx4 out;
    // the answers of chunk ch, from Q S0 (out) and U; asks for P and e of chunk `next`
    auto answer = [&](int ch, int next) {
      const Chunk c = chunk(ch);
      acc.clear();
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (s <= s1) mma32(pf[s], get_parts<3>(sU + swap8<kC>(li, 32 * s + 8 * lk), 16 * kC), acc);
      load_p(next);
      const floatx4 x = acc.sum();
#pragma unroll
      for (int r = 0; r < 4; ++r) st1(mine + (4 * lk + r) * LV + li, fmaf(a.scale * e[r], out[r], x[r]));
      sync_wave();
      e = factor(next, 1);
      T* orow = o + c.row * ldo + (int64_t)h * a.Dv;
      if (tv < c.n && cv < a.Dv)
        reinterpret_cast<const Raw4<T>*>(mine + lane / 4 * LV + 4 * (lane & 3))->store(orow + (uint32_t)(tv * (int)ldo + cv));
    };
    for (int ch = 0; ch < chunks; ++ch) {
      const Chunk c = chunk(ch);
      const int next = min(ch + 1, chunks - 1);  // (the last chunk's are read again: see mat_parts)
      if constexpr (B) {
        *reinterpret_cast<Raw4<T>*>(mine + lane / 4 * LV + 4 * (lane & 3)) = vv;
        sync_wave();
        acc.clear();
#pragma unroll
        for (int s = 0; s < NS; ++s)
          mma32(rf[s].parts(), get_parts<3>(sS + swap8<DKP>(li, 32 * s + 8 * lk), 16 * DKP), acc);
        load_rows(next);
        out = acc.sum();
#pragma unroll
        for (int r = 0; r < 4; ++r) out[r] = beta[r] * fmaf(-e[r], out[r], to_f32(mine[(4 * lk + r) * LV + li]));
        put_parts<3>(sR + swap8<kC>(li, place), 16 * kC, out);
        sync_wave();  // (the values are read)
        load_v(next);
        beta = factor(next, 0);
        e = factor(next, 1);
      } else if (ch > 0) {
        answer(ch - 1, ch);
      }
      if constexpr (SAVE)
#pragma unroll
        for (int n = 0; n < NT; ++n) keep(s0 + ((int64_t)(key + ch) * a.H + h) * size, n);
      sync_lds();
      if constexpr (B) {
        acc.clear();
#pragma unroll
        for (int s = 0; s < 2; ++s)
          if (s <= s1) mma32(tf[s], get_parts<3>(sR + swap8<kC>(li, 32 * s + 8 * lk), 16 * kC), acc);
        load_t(next);
        const floatx4 u = acc.sum();
        put_parts<3>(sW + swap8<kC>(li, place), 16 * kC, u * wj);
        wj = factor(next, 2);
        if constexpr (!SAVE) put_parts<3>(sU + swap8<kC>(li, place), 16 * kC, u);
        if (SAVE && col)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = 16 * w + 4 * lk + r;
            if (t < c.n) us[(((int64_t)(key + ch) * a.H + h) * kC + t) * a.Dv + c0 + li] = u[r];
          }
      } else {
        acc.clear();
#pragma unroll
        for (int s = 0; s < NS; ++s)
          mma32(rf[s].parts(), get_parts<3>(sS + swap8<DKP>(li, 32 * s + 8 * lk), 16 * DKP), acc);
        load_rows(next);
        out = acc.sum();
      }
      sync_lds();
      if constexpr (A || SAVE) {
        const float eC = coef[((int64_t)(key + ch) * a.H + h) * 3 * kC + 2 * kC - 1];
        Parts<3> wf[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) wf[s] = get_parts<3>(sW + swap8<kC>(li, 32 * s + 8 * lk), 16 * kC);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          acc.clear();
#pragma unroll
          for (int s = 0; s < 2; ++s) mma32(ktf[n][s].parts(), wf[s], acc);
          st[n] = st[n] * eC + acc.sum();
        }
        share();
        load_kt(next);
      }
      sync_lds();
    }
    if constexpr (A) answer(chunks - 1, chunks - 1);
  };
  if (chunks > 0) {
    if (answers) walk(std::true_type());
    else walk(std::false_type());
  }
  if (!SAVE && state_out && slot >= 0)
#pragma unroll
    for (int n = 0; n < NT; ++n) keep(state_out + ((int64_t)slot * a.H + h) * size, n);
}

// ---------------------------------------------------------------- gradients
// From dO and the adjoint dS1 of a chunk's end state:
//   dU = P^T dO + w K dS1,  dR = T^T dU,  dV = beta dR,
//   dS0 = e^G_C dS1 + scale Q^T (e^G dO) - K^T (beta e^G dR),
// which walks the chunks backwards as the forward pass walks them, keeping dS1 and dR; then, with
//   dA = -dR U^T (j < i),  dP = dO U^T (j <= i),  M1 = scale D dP,  M2 = beta D dA,
//   dQ = scale e^G dO S0^T + M1 K,
//   dK = -(beta e^G dR) S0^T + w U dS1^T + M1^T Q + (M2 + M2^T) K,
//   dbeta_i = dR_i . V_i - e^G_i k_i . (dR S0^T)_i + sum_j dA_ij D_ij k_i.k_j,
//   dg_t = sum_(i >= t > j) (dP_ij P_ij + dA_ij A_ij) + sum_(i >= t) (scale e^G q.(dO S0^T) - beta e^G k.(dR S0^T))_i
//          + sum_(j < t) (w k.(U dS1^T))_j + e^G_C <S0, dS1>
// all chunks at once. (dg_t is what passes over token t; as sums of such terms alone, without differences of
// the chunk's totals, it keeps its digits where a token forgets nearly all.)
// Two kinds of wavefronts as in the forward walk: four of 16 tokens each form dU and dR, and put what dO gives into
// LDS for the next chunk; four more the state's adjoint, Q^T (e dO) while dU and dR come about. Bound as that walk is:
// four sequences of up to 2,048 tokens, 16 heads of 128 x 128 in bf16, 125 us (the states' walk forwards 80).
template <typename T, int DKP>
__global__ __launch_bounds__(512) void delta_back_kernel(DeltaIn a, const T* __restrict__ d_o, int64_t lddo,
                                                         const float* __restrict__ mats, const float* __restrict__ coef,
                                                         const T* __restrict__ ops,
                                                         const float* __restrict__ dstate_out, float* __restrict__ dstate,
                                                         T* __restrict__ dv, int64_t lddv, float* __restrict__ ds1,
                                                         float* __restrict__ drs) {
  constexpr int NS = DKP / 32, NT = DKP / 64, KP = sizeof(T) == 2 ? 1 : 3, LV = 20;
  __shared__ __attribute__((aligned(16))) uint16_t sS[3 * 16 * DKP], sO[KP * 16 * kC], sE[3 * 16 * kC], sU[3 * 16 * kC],
      sW[3 * 16 * kC];
  __shared__ __attribute__((aligned(16))) float sV[4][16 * LV];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), w = wv & 3;
  const int parts = (a.Dv + 15) / 16;
  int head, part;
  head_and_part(blockIdx.x, a.n_seq * a.H, parts, head, part);
  const int c0 = part * 16, h = head % a.H, seq = head / a.H, hk = h / (a.H / a.Hk);
  const int base = min(max(a.offs ? a.offs[seq] : seq, 0), a.rows),
            len = a.offs ? min(max(a.offs[seq + 1], base), a.rows) - base : 1;
  const int key = !a.offs || kC > a.rows ? seq : base / kC + seq;
  const bool col = c0 + li < a.Dv;
  const int64_t size = (int64_t)a.Dk * a.Dv;
  const int place = token_place(w, lk);
  floatx4 st[NT];  // entries [16 (NT w + n) + 4 lk + r][c0 + li], of the last four wavefronts
  auto at = [&](int n) { return (int64_t)(16 * (NT * w + n) + 4 * lk) * a.Dv + c0 + li; };
  auto in = [&](int n) { return 16 * (NT * w + n) + 4 * lk < a.Dk && col; };
  auto keep = [&](float* p, int n) {
    if (in(n))
#pragma unroll
      for (int r = 0; r < 4; ++r) p[at(n) + (int64_t)r * a.Dv] = st[n][r];
  };
  auto share = [&]() {
#pragma unroll
    for (int n = 0; n < NT; ++n) put_parts<3>(sS + swap8<DKP>(li, 16 * (NT * w + n) + 4 * lk), 16 * DKP, st[n]);
  };
  const int chunks = (len + kC - 1) / kC;
  auto chunk = [&](int ch) { return Chunk{base + ch * kC, min(kC, len - ch * kC)}; };
  auto mat = [&](int ch, int i) {
    return reinterpret_cast<const uint16_t*>(mats + ((int64_t)(key + ch) * a.H + h) * kMats<true> + i * kTParts);
  };
  auto op = [&](int ch, int i) { return ops + (((int64_t)(key + ch) * a.Hk + hk) * 3 + i) * DKP * kC; };
  auto factor = [&](int ch, int i) {
    return at_lane<floatx4>(coef + ((int64_t)(key + ch) * a.H + h) * 3 * kC + i * kC + 16 * w, lk);
  };
  auto load_tiles = [&](Raw8<T> (*f)[2], const T* p) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int s = 0; s < 2; ++s) f[n][s].load_lane(p + (2 * (NT * w + n) + s) * 512, lane);
  };
  if (wv < 4) {
    const int cv = c0 + 4 * (lane & 3), tv = 16 * w + lane / 4, s0 = w >> 1;  // the first 32 tokens that T^T's rows reach
    float* mine = sV[wv];
    floatx4* rows = reinterpret_cast<floatx4*>(mine + lane / 4 * LV + 4 * (lane & 3));
    Raw8<T> rf[NS];
    Raw4<T> ov;
    Parts<3> pf[2], tf[2];
    floatx4 beta, e, wj;
    auto load_rows = [&](int ch) {
#pragma unroll
      for (int s = 0; s < NS; ++s) rf[s].load_lane(op(ch, 0) + (w * NS + s) * 512, lane);
    };
    auto load_mat = [&](Parts<3>* f, const uint16_t* m) {
      f[0] = mat_parts<3>(m, w, s0);
      f[1] = mat_parts<3>(m, w, 1);
    };
    auto load_o = [&](int ch) {
      const Chunk c = chunk(ch);
      ov = at_bytes<Raw4<T>>(d_o + c.row * lddo + (int64_t)h * a.Dv,
                             (uint32_t)(min(tv, c.n - 1) * (int)lddo + min(cv, a.Dv - 4)) * (uint32_t)sizeof(T));
    };
    // dO and scale e^G dO, zeros past the chunk's end, as columns into LDS
    auto put_o = [&](int ch) {
      const Chunk c = chunk(ch);
      *rows = widen(ov);
      sync_wave();
      floatx4 x;
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = 16 * w + 4 * lk + r < c.n ? mine[(4 * lk + r) * LV + li] : 0.f;
      put_parts<KP>(sO + swap8<kC>(li, place), 16 * kC, x);
      put_parts<3>(sE + swap8<kC>(li, place), 16 * kC, x * e * a.scale);
      sync_wave();
    };
    if (chunks > 0) {
      const int ch = chunks - 1;
      load_o(ch);
      e = factor(ch, 1);
      load_rows(ch);
      wj = factor(ch, 2);
      load_mat(pf, mat(ch, 2));
      load_mat(tf, mat(ch, 1));
      beta = factor(ch, 0);
      put_o(ch);
    }
    sync_lds();
    for (int ch = chunks - 1; ch >= 0; --ch) {
      const Chunk c = chunk(ch);
      const int next = max(ch - 1, 0);
      // ---- dU
      Acc acc;
      acc.clear();
#pragma unroll
      for (int s = 0; s < NS; ++s)
        mma32(rf[s].parts(), get_parts<3>(sS + swap8<DKP>(li, 32 * s + 8 * lk), 16 * DKP), acc);
      load_o(next);
      load_rows(next);
      const floatx4 y = acc.sum();
      acc.clear();
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (s >= s0) mma32(pf[s], get_parts<KP>(sO + swap8<kC>(li, 32 * s + 8 * lk), 16 * kC), acc);
      load_mat(pf, mat(next, 2));
      floatx4 x = acc.sum() + y * wj;
      put_parts<3>(sU + swap8<kC>(li, place), 16 * kC, x);
      wj = factor(next, 2);
      sync_lds();
      // ---- dR
      acc.clear();
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (s >= s0) mma32(tf[s], get_parts<3>(sU + swap8<kC>(li, 32 * s + 8 * lk), 16 * kC), acc);
      load_mat(tf, mat(next, 1));
      const floatx4 dr = acc.sum();
      put_parts<3>(sW + swap8<kC>(li, place), 16 * kC, -(dr * beta * e));
      sync_lds();
      // ---- what leaves, and the next chunk's dO
#pragma unroll
      for (int r = 0; r < 4; ++r) mine[(4 * lk + r) * LV + li] = dr[r];
      sync_wave();
      const floatx4 row = *rows;
      sync_wave();
#pragma unroll
      for (int r = 0; r < 4; ++r) mine[(4 * lk + r) * LV + li] = dr[r] * beta[r];
      sync_wave();
      const floatx4 rowb = *rows;
      sync_wave();
      beta = factor(next, 0);
      e = factor(next, 1);
      if (ch > 0) put_o(next);
      if (tv < c.n && cv < a.Dv) {
        *reinterpret_cast<floatx4*>(drs + (((int64_t)(key + ch) * a.H + h) * kC + tv) * a.Dv + cv) = row;
        st4(dv + (c.row + tv) * lddv + (int64_t)h * a.Dv + cv, rowb);
      }
      sync_lds();
    }
    return;
  }
  Raw8<T> qt[NT][2], kt[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    st[n] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (dstate_out && in(n))
#pragma unroll
      for (int r = 0; r < 4; ++r) st[n][r] = dstate_out[((int64_t)seq * a.H + h) * size + at(n) + (int64_t)r * a.Dv];
  }
  share();
  float eC = 0.f;
  if (chunks > 0) {
    load_tiles(qt, op(chunks - 1, 1));
    load_tiles(kt, op(chunks - 1, 2));
    eC = at_lane<float>(coef + ((int64_t)(key + chunks - 1) * a.H + h) * 3 * kC + 2 * kC - 1, 0);
  }
  sync_lds();
  for (int ch = chunks - 1; ch >= 0; --ch) {
    const int next = max(ch - 1, 0);
#pragma unroll
    for (int n = 0; n < NT; ++n) keep(ds1 + ((int64_t)(key + ch) * a.H + h) * size, n);
    Acc acc[NT];
    {
      Parts<3> ef[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) ef[s] = get_parts<3>(sE + swap8<kC>(li, 32 * s + 8 * lk), 16 * kC);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        acc[n].clear();
#pragma unroll
        for (int s = 0; s < 2; ++s) mma32(qt[n][s].parts(), ef[s], acc[n]);
      }
    }
    load_tiles(qt, op(next, 1));
    sync_lds();
    sync_lds();
    Parts<3> wf[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) wf[s] = get_parts<3>(sW + swap8<kC>(li, 32 * s + 8 * lk), 16 * kC);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int s = 0; s < 2; ++s) mma32(kt[n][s].parts(), wf[s], acc[n]);
      st[n] = st[n] * eC + acc[n].sum();
    }
    share();
    load_tiles(kt, op(next, 2));
    eC = at_lane<float>(coef + ((int64_t)(key + next) * a.H + h) * 3 * kC + 2 * kC - 1, 0);
    sync_lds();
  }
  if (dstate)
#pragma unroll
    for (int n = 0; n < NT; ++n) keep(dstate + ((int64_t)seq * a.H + h) * size, n);
}

// Over the 16 lanes that share l / 16.
__device__ __forceinline__ float sum16(float v) {
  v = sum8(v);
  return v + dpp<0x140>(v);
}
// The compiler asks for all operands of unrolled products at once, and spills others for them: not across this.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }
// Sum over the four lane groups l / 16; every lane receives it.
__device__ __forceinline__ float sum4(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

// What the chunks give once their states and adjoints are known, a workgroup per chunk and key head, which
// sums dQ and dK over the value heads that share it. Two sets of four wavefronts have 16 tokens each and
// half of the rows of dQ^T and dK^T each; the first also forms dP and M1, the second dA and M2. The states, their
// adjoints and U go through LDS in parts, 32 columns at a time; then M1 and M2 do, both ways round. 146 KB of LDS
// and 256 registers leave one workgroup to a CU, whose phases (a slice into LDS, its products, the matrices, their sums)
// follow each other: 87 chunks of 16 heads of 128 x 128 in bf16 164 to 168 us in 2.7 rounds of the CUs (over 20 more with
// the products of keys formed here again). 80 to 107 scalar registers are spilled to lanes of vector ones, and one vector
// register in fp32 at 128.
constexpr int kSl = 32, kLdSl = kSl + 8, kLdZ = kC + 8, kLdF = kC + 1;

template <typename T, int DKP>
__global__ __launch_bounds__(512) void delta_grads_kernel(DeltaIn a, const T* __restrict__ q, const T* __restrict__ k,
                                                          const T* __restrict__ v, const T* __restrict__ d_o,
                                                          int64_t lddo, const float* __restrict__ coef,
                                                          const T* __restrict__ ops, const float* __restrict__ prods,
                                                          const float* __restrict__ s0,
                                                          const float* __restrict__ ds1, const float* __restrict__ us,
                                                          const float* __restrict__ drs, T* __restrict__ dq,
                                                          int64_t lddq, T* __restrict__ dk, int64_t lddk,
                                                          float* __restrict__ dg, int64_t lddg,
                                                          float* __restrict__ dbeta, int64_t lddb) {
  constexpr int NT = DKP / 32;  // NT: tiles of 16 rows to a wavefront
  constexpr int kState = DKP * kLdSl, kU = kC * kLdSl, kZ = kC * kLdZ;  // bf16 entries of one part
  constexpr int KP = sizeof(T) == 2 ? 1 : 3;  // parts of an activation
  constexpr int kSlices = 6 * kState + (6 + KP) * kU, kProducts = 4 * 3 * kZ + 2 * 2 * kC * kLdF;
  __shared__ __attribute__((aligned(16))) uint16_t pool[kSlices > kProducts ? kSlices : kProducts];
  __shared__ double sG[kC];
  __shared__ float sQ1[2][kC], sK2[2][kC], sK3[2][kC], sRow[kC], sCol[kC], sSum[2][kC], sSeg[8][kC], sDot[8];
  uint16_t* sS0 = pool;
  uint16_t* sD1 = pool + 3 * kState;
  uint16_t* sUs = pool + 6 * kState;
  uint16_t* sDr = sUs + 3 * kU;
  uint16_t* sDo = sDr + 3 * kU;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wv & 3, set = wv >> 2;
  const int tile = blockIdx.x / a.Hk, hk = blockIdx.x % a.Hk;
  const Tile tl = find_tile(a.offs, a.n_seq, a.rows, kC, tile);
  if (tl.seq < 0 || tl.len == 0) return;
  const Chunk c = {tl.base + tl.j * kC, min(kC, tl.len - tl.j * kC)};
  const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
  const T* kp = k + (int64_t)hk * a.Dk;
  const T* qp = q + (int64_t)hk * a.Dk;
  const T* op = ops + ((int64_t)tile * a.Hk + hk) * 3 * DKP * kC;  // K, Q^T, K^T
  floatx4 dqa[NT], dka[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) dqa[n] = dka[n] = zero;
  const int share = a.H / a.Hk;
  const int64_t head = (int64_t)a.Dk * a.Dv;
  for (int hv = 0; hv < share; ++hv) {
    const int h = hk * share + hv;
    const int64_t th = (int64_t)tile * a.H + h;
    const float* co = coef + th * 3 * kC;
    // (as if it were another thread for every head: addresses formed once for all heads would not fit the registers)
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, li = lane & 15, lk = lane >> 4;
    const int t = 16 * w + li, t_in = min(t, c.n - 1);
    const int d0 = set * NT * 16 + 4 * lk;  // the lane's rows of tile n: d0 + 16 n + r
    sync_lds();
    if (tid < kC) {
      double G = tid < c.n ? log_decay(a.g[(c.row + tid) * a.ldg + h]) : 0.0;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const double up = __shfl_up(G, o, 64);
        if (tid >= o) G += up;
      }
      sG[tid] = G;
    }
    // a slice's share of this thread
    constexpr int NL = DKP * (kSl / 4) / 512;
    const int ut = tid / (kSl / 4), uc = 4 * (tid % (kSl / 4));
    floatx4 sv[NL], dvv[NL], uv, rr;
    Raw4<T> ov, vv;
    auto load = [&](int c0) {
      const float* sp = s0 + th * head + c0;
      const float* dp = ds1 + th * head + c0;
#pragma unroll
      for (int m = 0; m < NL; ++m) {
        const int r = ut + 64 * m;
        sv[m] = dvv[m] = zero;
        if (r < a.Dk && c0 + uc < a.Dv) {
          sv[m] = at_bytes<Raw4<float>>(sp, (uint32_t)(r * a.Dv + uc) * 4).v;
          dvv[m] = at_bytes<Raw4<float>>(dp, (uint32_t)(r * a.Dv + uc) * 4).v;
        }
      }
      uv = rr = zero;
      ov.v = vv.v = {};
      if (ut < c.n && c0 + uc < a.Dv) {
        const uint32_t at = (uint32_t)(ut * a.Dv + uc) * 4;
        uv = at_bytes<Raw4<float>>(us + th * kC * a.Dv + c0, at).v;
        rr = at_bytes<Raw4<float>>(drs + th * kC * a.Dv + c0, at).v;
        ov = at_bytes<Raw4<T>>(d_o + c.row * lddo + (int64_t)h * a.Dv + c0, (uint32_t)(ut * (int)lddo + uc) * (uint32_t)sizeof(T));
        vv = at_bytes<Raw4<T>>(v + c.row * a.ldv + (int64_t)h * a.Dv + c0, (uint32_t)(ut * (int)a.ldv + uc) * (uint32_t)sizeof(T));
      }
    };
    load(0);
    floatx4 dz[4], x1[NT], x2[NT], x3[NT];  // dP or dA (but for its sign), transposed; S0 dO^T, S0 dR^T, dS1 U^T
#pragma unroll
    for (int b = 0; b < 4; ++b) dz[b] = zero;
#pragma unroll
    for (int n = 0; n < NT; ++n) x1[n] = x2[n] = x3[n] = zero;
    float rv = 0.f, dot = 0.f;
    for (int c0 = 0; c0 < a.Dv; c0 += kSl) {
      sync_lds();  // (the slice before is read)
#pragma unroll
      for (int m = 0; m < NL; ++m) {
        put_parts<3>(sS0 + (ut + 64 * m) * kLdSl + uc, kState, sv[m]);
        put_parts<3>(sD1 + (ut + 64 * m) * kLdSl + uc, kState, dvv[m]);
#pragma unroll
        for (int e = 0; e < 4; ++e) dot = fmaf(sv[m][e], dvv[m][e], dot);
      }
      put_parts<3>(sUs + ut * kLdSl + uc, kU, uv);
      put_parts<3>(sDr + ut * kLdSl + uc, kU, rr);
      put_parts<KP>(sDo + ut * kLdSl + uc, kU, widen(ov));
      const floatx4 vw = widen(vv);
#pragma unroll
      for (int e = 0; e < 4; ++e) rv = fmaf(rr[e], vw[e], rv);
      if (c0 + kSl < a.Dv) load(c0 + kSl);
      sync_lds();
      const int own = t * kLdSl + 8 * lk;
      const Parts<3> rb = get_parts<3>(sDr + own, kU);
      const Parts<KP> ob = get_parts<KP>(sDo + own, kU);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (b > w) continue;
        const Parts<3> ub = get_parts<3>(sUs + (16 * b + li) * kLdSl + 8 * lk, kU);
        if (set) mma32(ub, rb, dz[b]);
        else mma32(ub, ob, dz[b]);
        keep_order();
      }
      const Parts<3> ub = get_parts<3>(sUs + own, kU);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int r = ((set * NT + n) * 16 + li) * kLdSl + 8 * lk;
        const Parts<3> x = get_parts<3>(sS0 + r, kState), y = get_parts<3>(sD1 + r, kState);
        mma32(x, ob, x1[n]);
        mma32(x, rb, x2[n]);
        mma32(y, ub, x3[n]);
        keep_order();
      }
    }
    // products of keys j with the set's rows (queries or keys) i: [16 b + 4 lk + r][t], as the preparation left them
    floatx4 zz[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      zz[b] = zero;
      if (b <= w) zz[b] = at_lane<floatx4>(prods + (((int64_t)tile * a.Hk + hk) * 2 + set) * kMat + (w * 4 + b) * 256, lane);
    }
    rv = sum8(rv);
    if ((tid & 7) == 0) sSum[1][ut] = rv;
    const float beta = co[t], e = co[kC + t], wj = co[2 * kC + t], eC = co[2 * kC - 1];
    // q.(dO S0^T), k.(dR S0^T), k.(U dS1^T) of the lane's token (the set's half of the rows), and dQ, dK's terms
    float q1 = 0.f, k2 = 0.f, k3 = 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      floatx4 qv = zero, kv = zero;
      if (d0 + 16 * n < a.Dk) {
        qv = widen(at_bytes<Raw4<T>>(qp + c.row * a.ldq + 16 * n, (uint32_t)(t_in * (int)a.ldq + d0) * (uint32_t)sizeof(T)));
        kv = widen(at_bytes<Raw4<T>>(kp + c.row * a.ldk + 16 * n, (uint32_t)(t_in * (int)a.ldk + d0) * (uint32_t)sizeof(T)));
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        q1 = fmaf(qv[r], x1[n][r], q1);
        k2 = fmaf(kv[r], x2[n][r], k2);
        k3 = fmaf(kv[r], x3[n][r], k3);
        dqa[n][r] = fmaf(a.scale * e, x1[n][r], dqa[n][r]);
        dka[n][r] = fmaf(wj, x3[n][r], fmaf(-beta * e, x2[n][r], dka[n][r]));
      }
    }
    q1 = sum4(q1); k2 = sum4(k2); k3 = sum4(k3);
    dot = sum4(sum16(dot));
    if (lk == 0) {
      sQ1[set][t] = q1;
      sK2[set][t] = k2;
      sK3[set][t] = k3;
    }
    if (lane == 0) sDot[wv] = dot;
    sync_lds();  // the slices are read
    // the set's matrix, M1 or M2 (below the diagonal), as rows and as columns over tokens in place
    uint16_t* sZ = pool + set * 2 * 3 * kZ;
    uint16_t* sZT = sZ + 3 * kZ;
    float* sF = reinterpret_cast<float*>(pool + 4 * 3 * kZ) + set * kC * kLdF;  // dP P or dA A
    float rowsum = 0.f;  // of dA D kk, of the lane's token
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      if (b > (w | 1)) continue;  // (the block behind the diagonal's too where they share 32 tokens: zeros)
      floatx4 z = zero, f = zero;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 16 * b + 4 * lk + r;
        if (j <= t) {
          const float d = exp_of(sG[t] - sG[j]);
          if (set) {
            const float ga = j < t ? -dz[b][r] * d : 0.f;
            z[r] = beta * ga;
            rowsum = fmaf(ga, zz[b][r], rowsum);
          } else {
            z[r] = a.scale * d * dz[b][r];
          }
          f[r] = j < t ? z[r] * zz[b][r] : 0.f;
        }
      }
      put_parts<3>(sZ + t * kLdZ + token_place(b, lk), kZ, z);
      const Parts4<3> p = split4<3>(z);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 16 * b + 4 * lk + r, at = token_place(w, li >> 2) + (li & 3);
#pragma unroll
        for (int i = 0; i < 3; ++i) sZT[i * kZ + j * kLdZ + at] = p.get(i, r);
        if (j <= t) sF[t * kLdF + j] = f[r];
      }
      keep_order();
    }
    rowsum = sum4(rowsum);
    if (set && lk == 0) sSum[0][t] = rowsum;
    sync_lds();
    {
      const uint16_t* m1 = pool;
      const uint16_t* m1t = pool + 3 * kZ;
      const uint16_t* m2 = pool + 2 * 3 * kZ;
      const uint16_t* m2t = pool + 3 * 3 * kZ;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int at = t * kLdZ + 32 * s + 8 * lk;
        const bool lo = s <= w >> 1, hi = s >= w >> 1;
        Parts<3> b1, b1t, b2, b2t;
        if (lo) {
          b1 = get_parts<3>(m1 + at, kZ);
          b2 = get_parts<3>(m2 + at, kZ);
        }
        if (hi) {
          b1t = get_parts<3>(m1t + at, kZ);
          b2t = get_parts<3>(m2t + at, kZ);
        }
        Raw8<T> kt[NT], qt[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          kt[n].load_lane(op + 2 * DKP * kC + (2 * (set * NT + n) + s) * 512, lane);
          qt[n].load_lane(op + DKP * kC + (2 * (set * NT + n) + s) * 512, lane);  // (always: a branch spilled 58 registers)
        }
        keep_order();
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const auto ka = kt[n].parts();
          if (lo) {
            mma32(ka, b1, dqa[n]);
            mma32(ka, b2, dka[n]);
          }
          if (hi) {
            mma32(qt[n].parts(), b1t, dka[n]);
            mma32(ka, b2t, dka[n]);
          }
          keep_order();
        }
      }
    }
    if (tid < kC && tid < c.n) {
      const float b = co[tid], ee = co[kC + tid];
      const float kr = sK2[0][tid] + sK2[1][tid];
      dbeta[(c.row + tid) * lddb + h] = sSum[1][tid] - ee * kr + sSum[0][tid];
      sRow[tid] = a.scale * ee * (sQ1[0][tid] + sQ1[1][tid]) - b * ee * kr;
      sCol[tid] = co[2 * kC + tid] * (sK3[0][tid] + sK3[1][tid]);
    } else if (tid < kC) {
      sRow[tid] = sCol[tid] = 0.f;
    }
    // column `lane` of the set's matrix, rows 16 w .. + 15: sums from each row to the last
    float z[16], z_all = 0.f;
#pragma unroll
    for (int i = 15; i >= 0; --i) {
      if (lane <= 16 * w + i) z_all += sF[(16 * w + i) * kLdF + lane];
      z[i] = z_all;
    }
    sSeg[wv][lane] = z_all;
    sync_lds();
    float below = 0.f;
    for (int x = w + 1; x < 4; ++x) below += sSeg[4 * set + x][lane];
    // entry [row, j]: what the pairs (i >= row, j) add to token row's sum
#pragma unroll
    for (int i = 0; i < 16; ++i) sF[(16 * w + i) * kLdF + lane] = z[i] + below;
    sync_lds();
    {
      const int row = tid >> 3, p = tid & 7;  // eight lanes to a token
      const float* f0 = reinterpret_cast<const float*>(pool + 4 * 3 * kZ);
      float sum = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int j = 8 * x + p;
        sum += j >= row ? sRow[j] : sCol[j] + f0[row * kLdF + j] + f0[(kC + row) * kLdF + j];
      }
      sum = sum8(sum);
      float all = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) all += sDot[x];
      if (p == 0 && row < c.n) dg[(c.row + row) * lddg + h] = fmaf(eC, all, sum);
    }
  }
  const int t = 16 * w + (threadIdx.x & 15), d0 = set * NT * 16 + 4 * (threadIdx.x >> 4 & 3);
  if (t < c.n)
#pragma unroll
    for (int n = 0; n < NT; ++n)
      if (d0 + 16 * n < a.Dk) {
        st4(dq + (c.row + t) * lddq + (int64_t)hk * a.Dk + d0 + 16 * n, dqa[n]);
        st4(dk + (c.row + t) * lddk + (int64_t)hk * a.Dk + d0 + 16 * n, dka[n]);
      }
}

// ---------------------------------------------------------------- launches

// From how many tokens a sequence, on average, chunks of kC pay. With few heads of sequences the walk's latency
// counts (some 0.5 to 1.1 us a token against 20 us for a first chunk and 4 to 6 for each after), with a full card what
// each has to do, of which chunks of fp32 values do the more. Walk / chunks in us, at tokens a sequence:
//   bf16, Dk = Dv = 128   16 heads     16: 22 / 18    24: 32 / 18     64: 78 / 18
//                         128          16: 23 / 26    24: 33 / 27     64: 82 / 29
//                         512          32: 66 / 76    40: 84 / 76     128: 254 / 105
//                         4,096        40: 488 / 517  48: 584 / 527   128: 1,744 / 889
//   fp32, 64              128          32: 20 / 22    48: 28 / 23
//                         512          64: 37 / 58    128: 69 / 81    192: 101 / 111
//                         1,024        64: 56 / 106   192: 165 / 256
//   fp32, 128             256          64: 56 / 71    96: 83 / 96     192: 161 / 131
//                         1,024        64: 181 / 257  192: 473 / 580
bool chunked(bool bf16, int n_seq, int rows, int H) {
  const int64_t heads = (int64_t)n_seq * H;
  const int64_t from = bf16 ? heads > 128 ? 40 : 24 : std::clamp<int64_t>(heads / 4, 32, 256);
  return rows >= from * n_seq;
}
constexpr int kPrepFill = 256;  // CUs
int64_t tiles_of(int n_seq, int rows) { return (int64_t)rows / kC + n_seq; }

DeltaIn in_of(const DeltaOp& a) {
  return {a.offs, a.n_seq, a.rows, a.Hk, a.H, a.Dk, a.Dv, a.ldq, a.ldk, a.ldv, a.ldg, a.ldb, a.g, a.beta, a.scale,
          a.state, a.slots, a.n_slots};
}

template <typename T>
hipError_t walk(const DeltaOp& a, float* state_out, void* o, int64_t ldo, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.n_seq * a.H * ((a.Dv + 31) / 32)));
  const T *q = static_cast<const T*>(a.q), *k = static_cast<const T*>(a.k), *v = static_cast<const T*>(a.v);
  if (a.Dk <= 64) delta_walk_kernel<T, 8><<<grid, 64, 0, s>>>(in_of(a), q, k, v, state_out, static_cast<T*>(o), ldo);
  else delta_walk_kernel<T, 16><<<grid, 64, 0, s>>>(in_of(a), q, k, v, state_out, static_cast<T*>(o), ldo);
  return hipGetLastError();
}

// Workgroups of the preparation for a chunk and key head: one for each value head where one for all leaves CUs idle (a
// prompt of 1,000 bf16 tokens, one key head, 2 value heads 46 -> 40 us a call, 16 of them 124 -> 42). They form the keys'
// products each for itself, so from a chunk and key head for every CU on it is one for all (4 sequences of 1,500 tokens each,
// 4 key heads, 12 value heads, fp32 heads of 128 x 128: 169 us, else 180; measured at this one size on that side).
int prep_parts(const DeltaOp& a, int64_t tiles) { return tiles * a.Hk < kPrepFill ? a.H / a.Hk : 1; }

template <typename T, int DKP>
hipError_t chunks(const DeltaOp& a, float* state_out, void* o, int64_t ldo, float* ws, hipStream_t s) {
  const int64_t tiles = tiles_of(a.n_seq, a.rows);
  float* coef = ws;
  float* mats = ws + tiles * a.H * 3 * kC;
  const T *q = static_cast<const T*>(a.q), *k = static_cast<const T*>(a.k), *v = static_cast<const T*>(a.v);
  T* ops = reinterpret_cast<T*>(mats + tiles * a.H * kMats<false>);
  const int parts = prep_parts(a, tiles);
  delta_prep_kernel<T, DKP, false><<<dim3((unsigned)(tiles * a.Hk * parts)), 256, 0, s>>>(in_of(a), q, k, mats, coef, ops,
                                                                                          nullptr, parts);
  delta_chunk_kernel<T, DKP, false><<<dim3((unsigned)((int64_t)a.n_seq * a.H * ((a.Dv + 15) / 16))), 512, 0, s>>>(
      in_of(a), v, mats, coef, ops, state_out, static_cast<T*>(o), ldo, nullptr, nullptr);
  return hipGetLastError();
}

// K, Q and K^T of every chunk and key head, in floats.
int64_t op_floats(bool bf16, int n_seq, int rows, int Hk, int Dk) {
  return tiles_of(n_seq, rows) * Hk * 3 * (Dk <= 64 ? 64 : 128) * kC / (bf16 ? 2 : 1);
}

// The parts of the gradients' workspace, in floats.
struct BackSpace {
  int64_t coef, mats, prods, s0, ds1, us, drs, ops, end;
  BackSpace(bool bf16, int n_seq, int rows, int Hk, int H, int Dk, int Dv) {
    const int64_t th = tiles_of(n_seq, rows) * H, head = (int64_t)Dk * Dv, act = th * kC * Dv;
    coef = 0;
    mats = coef + th * 3 * kC;
    prods = mats + th * kMats<true>;
    s0 = prods + tiles_of(n_seq, rows) * Hk * 2 * kMat;
    ds1 = s0 + th * head;
    us = ds1 + th * head;
    drs = us + act;
    ops = drs + act;
    end = ops + op_floats(bf16, n_seq, rows, Hk, Dk);
  }
};

template <typename T, int DKP>
hipError_t grads(const DeltaOp& a, const void* d_o_, int64_t lddo, const float* dstate_out, const DeltaGrads& g,
                 float* ws, hipStream_t s) {
  const int64_t tiles = tiles_of(a.n_seq, a.rows);
  const BackSpace b(a.bf16, a.n_seq, a.rows, a.Hk, a.H, a.Dk, a.Dv);
  T* ops = reinterpret_cast<T*>(ws + b.ops);
  const T *q = static_cast<const T*>(a.q), *k = static_cast<const T*>(a.k), *v = static_cast<const T*>(a.v);
  const T* d_o = static_cast<const T*>(d_o_);
  const DeltaIn in = in_of(a);
  const dim3 flat((unsigned)(tiles * a.Hk)), slices((unsigned)((int64_t)a.n_seq * a.H * ((a.Dv + 15) / 16)));
  const int parts = prep_parts(a, tiles);
  delta_prep_kernel<T, DKP, true><<<dim3(flat.x * parts), 256, 0, s>>>(in, q, k, ws + b.mats, ws + b.coef, ops,
                                                                       ws + b.prods, parts);
  delta_chunk_kernel<T, DKP, true><<<slices, 256, 0, s>>>(in, v, ws + b.mats, ws + b.coef, ops, nullptr, nullptr, 0,
                                                          ws + b.s0, ws + b.us);
  delta_back_kernel<T, DKP><<<slices, 512, 0, s>>>(in, d_o, lddo, ws + b.mats, ws + b.coef, ops, dstate_out, g.dstate,
                                                   static_cast<T*>(g.dv), g.lddv, ws + b.ds1, ws + b.drs);
  delta_grads_kernel<T, DKP><<<flat, 512, 0, s>>>(in, q, k, v, d_o, lddo, ws + b.coef, ops, ws + b.prods, ws + b.s0, ws + b.ds1,
                                                  ws + b.us, ws + b.drs, static_cast<T*>(g.dq), g.lddq, static_cast<T*>(g.dk),
                                                  g.lddk, g.dg, g.lddg, g.dbeta, g.lddb);
  return hipGetLastError();
}

}  // namespace

size_t delta_rule_workspace_bytes(bool bf16, int n_seq, int rows, int Hk, int H, int Dk, int Dv) {
  (void)Dv;
  if (!chunked(bf16, n_seq, rows, H)) return 0;
  return (size_t)(tiles_of(n_seq, rows) * H * (3 * kC + kMats<false>) + op_floats(bf16, n_seq, rows, Hk, Dk)) * sizeof(float);
}

hipError_t launch_delta_rule(const DeltaOp& a, float* state_out, void* o, int64_t ldo, float* ws, hipStream_t s) {
  if (!a.offs || !chunked(a.bf16, a.n_seq, a.rows, a.H))
    return a.bf16 ? walk<uint16_t>(a, state_out, o, ldo, s) : walk<float>(a, state_out, o, ldo, s);
  if (a.Dk <= 64)
    return a.bf16 ? chunks<uint16_t, 64>(a, state_out, o, ldo, ws, s) : chunks<float, 64>(a, state_out, o, ldo, ws, s);
  return a.bf16 ? chunks<uint16_t, 128>(a, state_out, o, ldo, ws, s) : chunks<float, 128>(a, state_out, o, ldo, ws, s);
}

size_t delta_rule_bwd_workspace_bytes(bool bf16, int n_seq, int rows, int Hk, int H, int Dk, int Dv) {
  return (size_t)BackSpace(bf16, n_seq, rows, Hk, H, Dk, Dv).end * sizeof(float);
}

hipError_t launch_delta_rule_bwd(const DeltaOp& a, const void* d_o, int64_t lddo, const float* dstate_out,
                                 const DeltaGrads& g, float* ws, hipStream_t s) {
  if (a.Dk <= 64)
    return a.bf16 ? grads<uint16_t, 64>(a, d_o, lddo, dstate_out, g, ws, s) : grads<float, 64>(a, d_o, lddo, dstate_out, g, ws, s);
  return a.bf16 ? grads<uint16_t, 128>(a, d_o, lddo, dstate_out, g, ws, s) : grads<float, 128>(a, d_o, lddo, dstate_out, g, ws, s);
}

}  // namespace tcl

// Shared by the kernels of the dense layers (networks that make the rule scores): types, activations, operand description.
#ifndef SPCFG_DENSE_H
#define SPCFG_DENSE_H

#include "gemm_nt_common.h"

namespace spcfg {
namespace dense {

using nt::bf16x8;
using nt::floatx16;
using nt::Split3;
using nt::uintx4;

// the element types of the boundary: float, or bf16 as raw 16 bits
template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<uint16_t>(uint16_t v) { return __uint_as_float((unsigned)v << 16); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t from_float<uint16_t>(float v) {
  return (uint16_t)(Split3::pack_rne(v, 0.0f) & 0xffffu);
}

// y = act(z) and its slope, in 32 bits, written for epilogues where dozens of values a lane wait for them: one exponential and one
// reciprocal of the hardware (1 ulp each) and products.
//   e^x as 2^(x log2 e), off by 1.5 2^-24 |x| of itself, which is all that the tails of silu and gelu lose: 4e-6 of silu at z = -80,
//   7e-7 and 1e-5 of gelu at z = -2 and -10 (x = -z^2 / 2, and the square's own roundings).
//   silu: z s, s = 1 / (1 + e^-z), slope s (1 + z (1 - s)).
//   gelu: with a = |z| / sqrt 2, erfc(a) = e^(-a^2) q(t), t = 1 / (1 + 0.49 a), q a polynomial without constant term, fitted here to
//   erfc(a) e^(a^2) on [0, 11] for the smallest largest relative error (2.7e-8; 3.5e-7 as q is evaluated in 32 bits).
//   y = max(z, 0) - |z| erfc(a) / 2; slope = (1 - erfc(a) / 2 or erfc(a) / 2) + z e^(-a^2) / sqrt(2 pi).
// Beyond |z| = 14.5 erfc is below what 32 bits hold.
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(1.44269504f * x); }
__device__ __forceinline__ float half_erfc(float z, float& e) {
  const float a = 0.70710678f * fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(0.49f, a, 1.0f));
  float q = -0.0567733148f;
  q = fmaf(q, t, 0.287798226f);
  q = fmaf(q, t, -0.529266789f);
  q = fmaf(q, t, 0.35331664f);
  q = fmaf(q, t, -0.0635568761f);
  q = fmaf(q, t, 0.218641415f);
  q = fmaf(q, t, 0.236318527f);
  q = fmaf(q, t, 0.277094389f);
  q = fmaf(q, t, 0.276427788f);
  e = exp_fast(-a * a);
  return 0.5f * e * (q * t);
}
__device__ __forceinline__ float relu_value(float z) { return z > 0.0f ? z : (z != z ? z : 0.0f); }
__device__ __forceinline__ float gelu_value(float z) {
  float e;
  const float h = half_erfc(z, e), r = fabsf(z) > 14.5f ? 0.0f : fabsf(z) * h;
  return z > 0.0f ? z - r : -r;
}
__device__ __forceinline__ float silu_value(float z) {
  const float r = z * __builtin_amdgcn_rcpf(1.0f + exp_fast(-z));
  return z == -INFINITY ? 0.0f : r;
}
__device__ __forceinline__ float relu_slope(float z) { return z > 0.0f ? 1.0f : (z != z ? z : 0.0f); }
__device__ __forceinline__ float gelu_slope(float z) {
  float e;
  const float h = half_erfc(z, e), s = (z > 0.0f ? 1.0f - h : h) + 0.39894228f * z * e;
  return fabsf(z) > 14.5f ? (z > 0.0f ? 1.0f : 0.0f) : s;
}
__device__ __forceinline__ float silu_slope(float z) {
  const float s = __builtin_amdgcn_rcpf(1.0f + exp_fast(-z)), r = s * fmaf(z, 1.0f - s, 1.0f);
  return fabsf(z) == INFINITY ? (z > 0.0f ? 1.0f : 0.0f) : r;
}
__device__ __forceinline__ float act_value(int act, float z) {
  if (act == SPCFG_ACT_RELU) return relu_value(z);
  if (act == SPCFG_ACT_GELU) return gelu_value(z);
  if (act == SPCFG_ACT_SILU) return silu_value(z);
  return z;
}
// N values at a time: one look at which activation it is
template <int N> __device__ __forceinline__ void act_values(int act, float (&v)[N]) {
  if (act == SPCFG_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = relu_value(v[i]);
  } else if (act == SPCFG_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = gelu_value(v[i]);
  } else if (act == SPCFG_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = silu_value(v[i]);
  }
}
// d[i] *= act'(z[i])
template <int N> __device__ __forceinline__ void times_slopes(int act, const float (&z)[N], float (&d)[N]) {
  if (act == SPCFG_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] *= relu_slope(z[i]);
  } else if (act == SPCFG_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] *= gelu_slope(z[i]);
  } else if (act == SPCFG_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] *= silu_slope(z[i]);
  }
}

// dz = grad_y * act'(z) beside bf16 operands is a 32-bit product: rounded to one bf16 value, 2^-8, it would put as much error into
// the gradients as their own rounding does (2.3e-3 in relative L2 where that alone makes 1.7e-3).  So it is multiplied as two pieces,
// hi = bf16(d) and lo = bf16(d - hi), good to 2^-17; in a second product, which matrix cores that wait for operands have room for.
struct Split2 {
  uintx4 hi, lo;
  __device__ __forceinline__ void cut(const float (&d)[8], bool two) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      hi[i] = Split3::pack_rne(d[2 * i], d[2 * i + 1]);
      if (two) {  // (beside an infinite piece the other is nothing, not inf - inf)
        const float h0 = __uint_as_float(hi[i] << 16), h1 = __uint_as_float(hi[i] & 0xffff0000u);
        lo[i] = Split3::pack_rne(fabsf(h0) == INFINITY ? 0.0f : d[2 * i] - h0, fabsf(h1) == INFINITY ? 0.0f : d[2 * i + 1] - h1);
      }
    }
  }
};
// how many: one where grad_y is bf16 and its slope 0 or 1, since dz is then a bf16 value itself
template <typename TI, typename TO> __host__ __device__ constexpr int dz_pieces(int act) {
  return sizeof(TI) == 4 ? 3 : sizeof(TO) == 2 && (act == SPCFG_ACT_NONE || act == SPCFG_ACT_RELU) ? 1 : 2;
}

// Everything a layer's kernels take.  R rows, I inputs, O outputs; matrices dense and row-major.
struct Args {
  int64_t R, I, O;
  int act, accumulate;
  const void *x, *W, *bias, *residual, *grad_y, *grad_x_add;
  const void* preact_in;
  void *y, *preact, *grad_x, *grad_W, *grad_bias;
};

// The three products of a layer: z = x W^T, dx = dz W, dW = dz^T x.
enum { FWD = 0, DX = 1, DW = 2 };

// N values of T as one access of N * sizeof(T) bytes, wherever they lie: global memory takes any alignment, and rows of odd
// lengths read and write 16 bytes at a time (4096 x 1023 x 1021 fp32 backward 129 us, element by element 158; bf16 49 and 72)
template <typename T, int N> __device__ __forceinline__ void get(const T* p, float (&v)[N]) {
  typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  T x[N];
  const V w = *reinterpret_cast<const V*>(p);
  __builtin_memcpy(x, &w, sizeof(x));
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = to_float<T>(x[i]);
}
template <typename T, int N> __device__ __forceinline__ void put(T* p, const float (&v)[N]) {
  typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  T x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = from_float<T>(v[i]);
  V w;
  __builtin_memcpy(&w, x, sizeof(x));
  *reinterpret_cast<V*>(p) = w;
}

template <typename T> __device__ __forceinline__ void get8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    get<T, 8>(p, v);
  } else {
    float a[4], b[4];
    get<T, 4>(p, a);
    get<T, 4>(p + 4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[i + 4] = b[i]; }
  }
}
template <typename T> __device__ __forceinline__ void put8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    put<T, 8>(p, v);
  } else {
    put<T, 4>(p, {v[0], v[1], v[2], v[3]});
    put<T, 4>(p + 4, {v[4], v[5], v[6], v[7]});
  }
}

// What becomes of a product's sums, one by one or eight adjacent ones of a row.
template <typename TI, typename TO, int FORM> struct Epilogue {
  int act, accumulate;
  const TI *bias, *add;
  const TO* residual;
  TO *y, *preact;
  TI* o;
  __device__ __forceinline__ explicit Epilogue(const Args& g)
      : act(g.act), accumulate(g.accumulate), bias(static_cast<const TI*>(g.bias)), add(static_cast<const TI*>(g.grad_x_add)),
        residual(static_cast<const TO*>(g.residual)), y(static_cast<TO*>(g.y)), preact(static_cast<TO*>(g.preact)),
        o(static_cast<TI*>(FORM == DX ? g.grad_x : g.grad_W)) {}
  __device__ __forceinline__ float bias_of(int64_t n, int64_t N) const {
    return FORM == FWD && bias && n < N ? to_float<TI>(bias[n]) : 0.0f;
  }
  __device__ __forceinline__ void one(int64_t at, float s, float b) const {
    if constexpr (FORM == FWD) {
      s += b;
      if (preact) preact[at] = from_float<TO>(s);
      s = act_value(act, s);
      if (residual) s += to_float<TO>(residual[at]);
      y[at] = from_float<TO>(s);
    } else if constexpr (FORM == DX) {
      if (add) s += to_float<TI>(add[at]);
      o[at] = from_float<TI>(s);
    } else {
      if (accumulate) s += to_float<TI>(o[at]);
      o[at] = from_float<TI>(s);
    }
  }
  __device__ __forceinline__ void eight(int64_t at, float (&s)[8], const float (&b)[8], int64_t left) const {
    if (left < 8) {
      for (int u = 0; u < 8; ++u)
        if (u < left) one(at + u, s[u], b[u]);
      return;
    }
    float r[8];
    if constexpr (FORM == FWD) {
#pragma unroll
      for (int u = 0; u < 8; ++u) s[u] += b[u];
      if (preact) put8<TO>(preact + at, s);
      act_values<8>(act, s);
      if (residual) {
        get8<TO>(residual + at, r);
#pragma unroll
        for (int u = 0; u < 8; ++u) s[u] += r[u];
      }
      put8<TO>(y + at, s);
    } else {
      if (FORM == DX ? add != nullptr : accumulate != 0) {
        get8<TI>(FORM == DX ? add + at : o + at, r);
#pragma unroll
        for (int u = 0; u < 8; ++u) s[u] += r[u];
      }
      put8<TI>(o + at, s);
    }
  }
};
template <typename TI>
__device__ __forceinline__ void store_bias(const Args& g, int64_t m, float s) {
  TI* o = static_cast<TI*>(g.grad_bias) + m;
  if (g.accumulate) s += to_float<TI>(*o);
  *o = from_float<TI>(s);
}

constexpr unsigned kMostWorkgroups = 1u << 22;  // of a launch, of up to 512 threads each

inline bool on16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// what a call computes: FORWARD, or of the backward pass dx, dW or both
enum { FORWARD = 0, BACK_X = 1, BACK_W = 2, BACK = 3 };

// Products in registers (dense_direct.hip), for any sizes, types and alignments; an estimate of what they take
double direct_us(int64_t R, int64_t I, int64_t O, int in_type, int act, int what);
void launch_direct_forward(const Args& a, int in_type, int out_type, hipStream_t st);
void launch_direct_backward(const Args& a, int in_type, int out_type, hipStream_t st);

// Tiled products (dense_tile.hip): workspace of a layer, 0 where it never takes them
size_t tiled_workspace(int64_t R, int64_t I, int64_t O, int in_type, int out_type, int act);
// whether these take the call: where they are estimated to be faster than products in registers
bool tiled_forward(const Args& a, int in_type, int out_type, void* ws, hipStream_t st);
bool tiled_backward(const Args& a, int in_type, int out_type, void* ws, hipStream_t st);

}  // namespace dense
}  // namespace spcfg
#endif

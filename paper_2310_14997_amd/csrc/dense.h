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

// y = act(z) and its slope, in 32 bits.  silu: z s(z) with slope s (1 + z (1 - s)); s = 1 / (1 + exp(-z)) is 0 where the exponential
// overflows, and z s is then -inf * 0 only for z = -inf itself, whose limit 0 is written out.
__device__ __forceinline__ float act_value(int act, float z) {
  if (act == SPCFG_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
  if (act == SPCFG_ACT_GELU) return z == -INFINITY ? 0.0f : 0.5f * z * erfcf(-0.70710678118654752f * z);
  if (act == SPCFG_ACT_SILU) return z == -INFINITY ? 0.0f : z / (1.0f + expf(-z));
  return z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
  if (act == SPCFG_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
  if (act == SPCFG_ACT_GELU) {
    if (fabsf(z) == INFINITY) return z > 0.0f ? 1.0f : 0.0f;
    return 0.5f * erfcf(-0.70710678118654752f * z) + z * 0.39894228040143268f * expf(-0.5f * z * z);
  }
  if (act == SPCFG_ACT_SILU) {
    if (fabsf(z) == INFINITY) return z > 0.0f ? 1.0f : 0.0f;
    const float s = 1.0f / (1.0f + expf(-z));
    return s * (1.0f + z * (1.0f - s));
  }
  return 1.0f;
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

// Epilogue of one element (m, n) of a product, whose sum is s.
template <typename TI, typename TO, int FORM>
__device__ __forceinline__ void store_one(const Args& g, int64_t m, int64_t n, float s) {
  const int64_t at = m * (FORM == FWD ? g.O : g.I) + n;
  if constexpr (FORM == FWD) {
    if (g.bias) s += to_float<TI>(static_cast<const TI*>(g.bias)[n]);
    if (g.preact) static_cast<TO*>(g.preact)[at] = from_float<TO>(s);
    s = act_value(g.act, s);
    if (g.residual) s += to_float<TO>(static_cast<const TO*>(g.residual)[at]);
    static_cast<TO*>(g.y)[at] = from_float<TO>(s);
  } else if constexpr (FORM == DX) {
    if (g.grad_x_add) s += to_float<TI>(static_cast<const TI*>(g.grad_x_add)[at]);
    static_cast<TI*>(g.grad_x)[at] = from_float<TI>(s);
  } else {
    TI* o = static_cast<TI*>(g.grad_W) + at;
    if (g.accumulate) s += to_float<TI>(*o);
    *o = from_float<TI>(s);
  }
}
template <typename TI>
__device__ __forceinline__ void store_bias(const Args& g, int64_t m, float s) {
  TI* o = static_cast<TI*>(g.grad_bias) + m;
  if (g.accumulate) s += to_float<TI>(*o);
  *o = from_float<TI>(s);
}

inline bool on16(const void* p) { return ((uintptr_t)p & 15) == 0; }

void launch_direct_forward(const Args& a, int in_type, int out_type, hipStream_t st);
void launch_direct_backward(const Args& a, int in_type, int out_type, hipStream_t st);

// Tiled products (dense_tile.hip): workspace of a layer, 0 where none of its products takes them
size_t tiled_workspace(int64_t R, int64_t I, int64_t O, int in_type, int out_type, int act);
// whether these take the call: sizes, and alignment of what is read as it lies
bool tiled_forward(const Args& a, int in_type, int out_type, void* ws, hipStream_t st);
bool tiled_backward(const Args& a, int in_type, int out_type, void* ws, hipStream_t st);

}  // namespace dense
}  // namespace spcfg
#endif

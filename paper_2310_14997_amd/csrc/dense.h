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

void launch_direct_forward(const Args& a, int in_type, int out_type, hipStream_t st);
void launch_direct_backward(const Args& a, int in_type, int out_type, hipStream_t st);

}  // namespace dense
}  // namespace spcfg
#endif

// Preference loss on pairs of sentences, by their log Z (a sentence and a corrupted copy, or any better and worse one), and
// its gradient, in the form that the reverse pass of the inside algorithm takes:
//   margin = (logZ_c - ref_c) - (logZ_r - ref_r),   x = beta margin
//   loss   = (1 - eps) softplus(-x) + eps softplus(x)
//   d loss / d margin = beta (eps s(x) - (1 - eps) s(-x)),  s(x) = 1 / (1 + exp(-x)); + at c, - at r
// One launch: workgroups of the first kind take the pairs, those of the second kind four sentences each.  These look through
// all pairs, a segment of 1024 per wavefront at a time with every load in flight, list the ones that their sentences are part
// of in LDS (in order), and then take the list 64 pairs at a time: what it takes to work a pair out, and its latency, is spent
// on the few pairs that matter.  No atomics: a sentence in many pairs has its sum in a fixed order (lane by lane, across
// lanes, across wavefronts), in 64 bits, as are the differences of log Z, which are small beside log Z itself.  Bound by
// latency at the sizes of a batch: 32 pairs of 64 sentences 4.2 us, 8192 of 960 7.2 us (58 us where every wavefront worked
// each pair out as it came to it).  Beyond, by the pairs that every four sentences look through: 2^17 of 960 71 us, 2^20 of 960
// 0.6 ms, 2^20 of 65536 5.4 ms.
#include <cmath>

#include "spcfg_internal.h"

namespace spcfg {
namespace {

constexpr int kOwn = 4;        // sentences of a workgroup
constexpr int kSeg = 16;       // pairs a lane looks through at a time
constexpr int kMostPairs = 1 << 20, kMostSentences = 1 << 16;

struct Args {
  int B, n;
  const float *logZ, *ref;
  const int32_t *chosen, *rejected;
  float beta, eps;
  const float* grad_loss;
  float *loss, *margin, *grad;
};

// margin of pair (i, j): out of range NaN; both sides infinite alike (two sentences that cannot be derived) 0 with *out set, as
// for an absent pair
__device__ __forceinline__ float margin_of(const Args& g, int i, int j, bool* out) {
  *out = i < 0 || j < 0;
  if (*out) return 0.0f;
  if (i >= g.B || j >= g.B) return NAN;
  const float a = g.logZ[i], b = g.logZ[j];
  const float ra = g.ref ? g.ref[i] : 0.0f, rb = g.ref ? g.ref[j] : 0.0f;
  const double d = ((double)a - ra) - ((double)b - rb);
  if (d != d && a == a && b == b && ra == ra && rb == rb) {
    *out = true;
    return 0.0f;
  }
  return (float)d;
}

__device__ __forceinline__ float weight_of(const Args& g, float margin) {
  const float x = g.beta * margin;
  return g.beta * (g.eps / (1.0f + expf(-x)) - (1.0f - g.eps) / (1.0f + expf(x)));
}

__global__ void __launch_bounds__(256) k_preference(Args g, int pair_blocks) {
  __shared__ int list[4][kSeg * 64];
  __shared__ double red[4][kOwn];
  if ((int)blockIdx.x < pair_blocks) {
    const int p = blockIdx.x * 256 + threadIdx.x;
    if (p >= g.n) return;
    bool out;
    const float m = margin_of(g, g.chosen[p], g.rejected[p], &out);
    const float x = g.beta * m, tail = log1pf(expf(-fabsf(x)));
    // (an infinite margin times a smoothing of 0 would be NaN)
    const float lo = fmaxf(-x, 0.0f) + tail, hi = fmaxf(x, 0.0f) + tail;
    const float l = (g.eps < 1.0f ? (1.0f - g.eps) * lo : 0.0f) + (g.eps > 0.0f ? g.eps * hi : 0.0f);
    g.loss[p] = out ? 0.0f : m != m ? m : l;
    g.margin[p] = m;
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int s0 = ((int)blockIdx.x - pair_blocks) * kOwn;
  double acc[kOwn] = {};
  for (int seg = wave * kSeg * 64; seg < g.n; seg += 4 * kSeg * 64) {
    int i[kSeg], j[kSeg], found = 0;
#pragma unroll
    for (int u = 0; u < kSeg; ++u) {
      const int p = seg + u * 64 + lane;
      i[u] = p < g.n ? g.chosen[p] : -1;
      j[u] = p < g.n ? g.rejected[p] : -1;
    }
#pragma unroll
    for (int u = 0; u < kSeg; ++u) {
      const bool mine = (unsigned)i[u] - (unsigned)s0 < (unsigned)kOwn || (unsigned)j[u] - (unsigned)s0 < (unsigned)kOwn;
      const unsigned long long m = __ballot(mine);
      if (mine) list[wave][found + __popcll(m & ((1ull << lane) - 1))] = seg + u * 64 + lane;
      found += __popcll(m);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (a wavefront reads only what it listed itself)
    for (int h = lane; h < found; h += 64) {
      const int p = list[wave][h], c = g.chosen[p], r = g.rejected[p];
      bool out;
      const float m = margin_of(g, c, r, &out);
      if (out || (c == r && m == m)) continue;  // (a sentence against itself adds and takes away the same)
      const double w = (double)weight_of(g, m) * (g.grad_loss ? g.grad_loss[p] : 1.0f);
#pragma unroll
      for (int u = 0; u < kOwn; ++u) {
        if (c == s0 + u) acc[u] += w;
        if (r == s0 + u) acc[u] -= w;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
#pragma unroll
  for (int u = 0; u < kOwn; ++u) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) acc[u] += __shfl_xor(acc[u], o, 64);
    if (lane == 0) red[wave][u] = acc[u];
  }
  __syncthreads();
  const int u = threadIdx.x;
  if (u < kOwn && s0 + u < g.B) g.grad[s0 + u] = (float)(((red[0][u] + red[1][u]) + red[2][u]) + red[3][u]);
}

int run(int32_t B, int32_t n, const float* logZ, const float* ref, const int32_t* chosen, const int32_t* rejected, float beta,
        float eps, const float* grad_loss, float* loss, float* margin, float* grad, bool forward, bool backward, hipStream_t st) {
  if (B < 1 || B > kMostSentences || n < 0 || n > kMostPairs) return SPCFG_ERR_SHAPE;
  if (!(beta > 0.0f) || !(beta < INFINITY) || !(eps >= 0.0f) || !(eps <= 1.0f)) return SPCFG_ERR_ARG;
  if (!logZ || (n > 0 && (!chosen || !rejected)) || (n > 0 && forward && (!loss || !margin)) || (backward && !grad))
    return SPCFG_ERR_ARG;
  // outputs are written while other workgroups read the inputs: none may share memory with anything else
  const Memory all[] = {{forward ? loss : nullptr, 4ll * n}, {forward ? margin : nullptr, 4ll * n}, {backward ? grad : nullptr, 4ll * B},
                        {logZ, 4ll * B}, {ref, 4ll * B}, {chosen, 4ll * n}, {rejected, 4ll * n}, {grad_loss, 4ll * n}};
  if (clash(all, 3, 8)) return SPCFG_ERR_ARG;
  for (const Memory& m : all)
    if ((uintptr_t)m.p & 3) return SPCFG_ERR_ARG;
  const int pb = forward ? (n + 255) / 256 : 0, sb = backward ? (B + kOwn - 1) / kOwn : 0;
  if (pb + sb == 0) return SPCFG_OK;
  const Args a{B, n, logZ, ref, chosen, rejected, beta, eps, grad_loss, loss, margin, grad};
  hipLaunchKernelGGL(k_preference, dim3(pb + sb), dim3(256), 0, st, a, pb);
  return launch_status();
}

}  // namespace
}  // namespace spcfg

using namespace spcfg;

extern "C" {

int spcfg_preference_forward(int32_t B, int32_t pairs, const float* logZ, const float* ref_logZ, const int32_t* chosen,
                             const int32_t* rejected, float beta, float smoothing, float* loss, float* margin,
                             void* hip_stream) {
  return run(B, pairs, logZ, ref_logZ, chosen, rejected, beta, smoothing, nullptr, loss, margin, nullptr, true, false,
             (hipStream_t)hip_stream);
}

int spcfg_preference_backward(int32_t B, int32_t pairs, const float* logZ, const float* ref_logZ, const int32_t* chosen,
                              const int32_t* rejected, float beta, float smoothing, const float* grad_loss,
                              float* grad_logZ, void* hip_stream) {
  return run(B, pairs, logZ, ref_logZ, chosen, rejected, beta, smoothing, grad_loss, nullptr, nullptr, grad_logZ, false, true,
             (hipStream_t)hip_stream);
}

int spcfg_preference_forward_backward(int32_t B, int32_t pairs, const float* logZ, const float* ref_logZ,
                                      const int32_t* chosen, const int32_t* rejected, float beta, float smoothing,
                                      const float* grad_loss, float* loss, float* margin, float* grad_logZ,
                                      void* hip_stream) {
  return run(B, pairs, logZ, ref_logZ, chosen, rejected, beta, smoothing, grad_loss, loss, margin, grad_logZ, true, true,
             (hipStream_t)hip_stream);
}

}  // extern "C"

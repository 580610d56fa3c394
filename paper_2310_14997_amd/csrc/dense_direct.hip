// Dense layers, small products: C[m][n] = sum_k A[m][k] B[n][k] with matrix operands loaded from global memory straight into
// the registers of the matrix instructions, whatever their order, alignment and size:
//   forward       z = x W^T              A = x  (k = inputs),       B = W    (both run along k)
//   d x           dz W, dz = gy act'(z)  A = dz (k = outputs),      B = W^T  (W runs along n)
//   d W           dz^T x                 A = dz^T (k = rows),       B = x^T  (both run across k), with db = row sums of A
// One output tile of 32 MT x 32 NT per workgroup; its eight wavefronts take 16-value chunks of K in turn, each with
// everything of its chunk in flight, and meet once, in LDS, where the epilogue runs on whole rows of the tile.  Small
// products are bound by latency: one load latency, a few matrix instructions and one exchange.  fp32 operands are cut
// exactly into three bf16 pieces in registers and multiplied as six piece products (nt::Split3), dz is formed on the way.
#include <type_traits>

#include "dense.h"

namespace spcfg {
namespace dense {

namespace {

constexpr int kWaves = 8;

// pieces of eight K values of one row, ready for the matrix instruction
template <typename T> struct Pieces;
template <> struct Pieces<float> {
  Split3 s;
  __device__ __forceinline__ void set(const float (&v)[8]) {
    s.cut(make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7]));
  }
  __device__ __forceinline__ void raw(const float (&v)[8]) { set(v); }
};
template <> struct Pieces<uint16_t> {
  uintx4 h;
  __device__ __forceinline__ void set(const float (&v)[8]) {  // dz is rounded to the operands' type, as W and x are
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = Split3::pack_rne(v[2 * i], v[2 * i + 1]);
  }
  __device__ __forceinline__ void raw(const uint16_t (&v)[8]) { __builtin_memcpy(&h, v, 16); }
};
__device__ __forceinline__ floatx16 mma(uintx4 a, uintx4 b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ void product(const Pieces<float>& a, const Pieces<float>& b, floatx16& c) {
  c = mma(a.s.lo, b.s.hi, c);
  c = mma(a.s.hi, b.s.lo, c);
  c = mma(a.s.mid, b.s.mid, c);
  c = mma(a.s.mid, b.s.hi, c);
  c = mma(a.s.hi, b.s.mid, c);
  c = mma(a.s.hi, b.s.hi, c);
}
__device__ __forceinline__ void product(const Pieces<uint16_t>& a, const Pieces<uint16_t>& b, floatx16& c) {
  c = mma(a.h, b.h, c);
}

// v[i] = element (row, k + i), i = 0 .. 7, of an operand that runs along k; zero from K on.  VEC: base and rows lie on 16 bytes
// and K is a multiple of 8.
template <typename T, bool VEC>
__device__ __forceinline__ void along(const T* __restrict__ row, int64_t k, int64_t K, T (&v)[8]) {
  if (VEC) {
    uintx4 w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      w[i] = k < K ? reinterpret_cast<const uintx4*>(row + k)[i] : uintx4{0, 0, 0, 0};
    __builtin_memcpy(v, w, sizeof(v));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < K ? row[k + i] : T(0);
  }
}
// the same of an operand that runs across k: column `col` of rows k .. k + 7
template <typename T>
__device__ __forceinline__ void across(const T* __restrict__ p, int64_t ld, int64_t col, int64_t k, int64_t K, T (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = k + i < K ? p[(k + i) * ld + col] : T(0);
}

template <typename TI, typename TO, int FORM, bool VEC, int MT, int NT>
__device__ __forceinline__ void tile_product(const Args& g, int64_t tm, int64_t tn, float* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int fr = lane & 31, fh = lane >> 5;
  const int64_t M = FORM == DW ? g.O : g.R, N = FORM == FWD ? g.O : g.I;
  const int64_t K = FORM == FWD ? g.I : FORM == DX ? g.O : g.R;
  const int64_t m0 = tm * (32 * MT), n0 = tn * (32 * NT);
  const TI* x = static_cast<const TI*>(g.x);
  const TI* W = static_cast<const TI*>(g.W);
  const TO* gy = static_cast<const TO*>(g.grad_y);
  const TO* z = static_cast<const TO*>(g.preact_in);
  const bool slope = g.act != SPCFG_ACT_NONE;

  floatx16 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
  float bsum[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) bsum[i] = 0.0f;

  // rows and columns past the end repeat the last one: their results are not stored
  int64_t ra[MT], rb[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) ra[i] = min(m0 + 32 * i + fr, M - 1);
#pragma unroll
  for (int j = 0; j < NT; ++j) rb[j] = min(n0 + 32 * j + fr, N - 1);

  // U chunks at a time: everything of theirs is asked for before any of it is used
  using T1 = typename std::conditional<FORM == FWD, TI, TO>::type;
  constexpr int U = FORM == FWD ? 4 : 2;
  const int64_t chunks = (K + 15) / 16;
  for (int64_t c0 = wave; c0 < chunks; c0 += kWaves * U) {
    T1 va[U][MT][8], vz[U][MT][8];
    TI vb[U][NT][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = (c0 + kWaves * u) * 16 + fh * 8;  // (from K on everything is zero)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if constexpr (FORM == FWD) {
          along<TI, VEC>(x + ra[i] * g.I, k, K, va[u][i]);
        } else if constexpr (FORM == DX) {
          along<TO, VEC>(gy + ra[i] * g.O, k, K, va[u][i]);
          if (slope) along<TO, VEC>(z + ra[i] * g.O, k, K, vz[u][i]);
        } else {
          across<TO>(gy, g.O, ra[i], k, K, va[u][i]);
          if (slope) across<TO>(z, g.O, ra[i], k, K, vz[u][i]);
        }
      }
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if constexpr (FORM == FWD) along<TI, VEC>(W + rb[j] * g.I, k, K, vb[u][j]);
        else across<TI>(FORM == DX ? W : x, g.I, rb[j], k, K, vb[u][j]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (c0 + kWaves * u >= chunks) break;
      Pieces<TI> A[MT], B[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if constexpr (FORM == FWD) {
          A[i].raw(va[u][i]);
        } else {
          float d[8], zz[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = to_float<TO>(va[u][i][e]);
          if (slope) {
#pragma unroll
            for (int e = 0; e < 8; ++e) zz[e] = to_float<TO>(vz[u][i][e]);
            times_slopes<8>(g.act, zz, d);
          }
          if (FORM == DW) {
#pragma unroll
            for (int e = 0; e < 8; ++e) bsum[i] += d[e];
          }
          A[i].set(d);
        }
      }
#pragma unroll
      for (int j = 0; j < NT; ++j) B[j].raw(vb[u][j]);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) product(A[i], B[j], acc[i][j]);
    }
  }

  // the eight partial tiles, summed in the order of the wavefronts; thread t then owns whole columns of rows
  constexpr int kTile = 32 * MT * 32 * NT;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int r = 32 * i + (v >> 2) * 8 + fh * 4 + (v & 3), cc = 32 * j + fr;
        lds[wave * kTile + r * (32 * NT) + cc] = acc[i][j][v];
      }
  float* bl = lds + kWaves * kTile;  // [wave][MT][64]
  if (FORM == DW) {
#pragma unroll
    for (int i = 0; i < MT; ++i) bl[(wave * MT + i) * 64 + lane] = bsum[i];
  }
  __syncthreads();
  const Epilogue<TI, TO, FORM> ep(g, N);
  for (int e = threadIdx.x; e < kTile; e += 64 * kWaves) {
    const int64_t m = m0 + e / (32 * NT), n = n0 + e % (32 * NT);
    if (m >= M || n >= N) continue;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += lds[w * kTile + e];
    ep.one(m * N + n, s, ep.bias_of(n, N));
  }
  if (FORM == DW && g.grad_bias && tn == 0 && threadIdx.x < 32 * MT) {
    const int64_t m = m0 + threadIdx.x;
    if (m < M) {
      const int i = threadIdx.x >> 5, l = threadIdx.x & 31;
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) s += bl[(w * MT + i) * 64 + l] + bl[(w * MT + i) * 64 + 32 + l];
      store_bias<TI>(g, m, s);
    }
  }
}

template <int MT, int NT> constexpr int lds_floats() { return kWaves * 32 * MT * 32 * NT + kWaves * MT * 64; }

template <typename TI, typename TO, bool VEC, int MT, int NT>
__global__ void __launch_bounds__(64 * kWaves) k_dense_forward(Args g, unsigned tiles_n) {
  __shared__ float lds[lds_floats<MT, NT>()];
  tile_product<TI, TO, FWD, VEC, MT, NT>(g, blockIdx.x / tiles_n, blockIdx.x % tiles_n, lds);
}

// both products of the backward pass in one launch: the tiles of dx first, then those of dW (either may be absent)
template <typename TI, typename TO, bool VEC, int MT, int NT>
__global__ void __launch_bounds__(64 * kWaves) k_dense_backward(Args g, unsigned tiles_x, unsigned tiles_i) {
  __shared__ float lds[lds_floats<MT, NT>()];
  const unsigned b = blockIdx.x;
  if (b < tiles_x) tile_product<TI, TO, DX, VEC, MT, NT>(g, b / tiles_i, b % tiles_i, lds);
  else tile_product<TI, TO, DW, VEC, MT, NT>(g, (b - tiles_x) / tiles_i, (b - tiles_x) % tiles_i, lds);
}

unsigned tiles(int64_t n, int t) { return (unsigned)((n + t - 1) / t); }

template <typename TI, typename TO>
void forward(const Args& a, hipStream_t st) {
  const bool vec = on16(a.x) && on16(a.W) && a.I % 8 == 0;
  const unsigned tn = tiles(a.O, 32), grid = tiles(a.R, 32) * tn;
  if (vec) hipLaunchKernelGGL((k_dense_forward<TI, TO, true, 1, 1>), dim3(grid), dim3(64 * kWaves), 0, st, a, tn);
  else hipLaunchKernelGGL((k_dense_forward<TI, TO, false, 1, 1>), dim3(grid), dim3(64 * kWaves), 0, st, a, tn);
}
template <typename TI, typename TO>
void backward(const Args& a, hipStream_t st) {
  const bool vec = on16(a.grad_y) && on16(a.preact_in) && a.O % 8 == 0;
  const unsigned ti = tiles(a.I, 32), tx = a.grad_x ? tiles(a.R, 32) * ti : 0, tw = a.grad_W ? tiles(a.O, 32) * ti : 0;
  if (vec) hipLaunchKernelGGL((k_dense_backward<TI, TO, true, 1, 1>), dim3(tx + tw), dim3(64 * kWaves), 0, st, a, tx, ti);
  else hipLaunchKernelGGL((k_dense_backward<TI, TO, false, 1, 1>), dim3(tx + tw), dim3(64 * kWaves), 0, st, a, tx, ti);
}

}  // namespace

// 3 us to start and end; then whichever is longer, the trips of one wavefront through k (128 values of a workgroup a trip) or those
// of all tiles on the whole chip.  Measured (us for this kernel / on tiles): forward fp32 512^3 7.8 / 14, 2048 x 512 x 512 21 / 18,
// 300 x 2000 x 300 19 / 23, bf16 5.1 / 6.9, 11.5 / 7.4, 10.8 / 17; backward fp32 512 x 256 x 256 9.3 / 15.5, 512^3 18 / 18.5,
// 8000 x 100 x 100 110 / 48, bf16 10.8 / 10.4, 17 / 11, 210 / 43.
double direct_us(int64_t R, int64_t I, int64_t O, int in_type, int what) {
  const bool fp32 = in_type == SPCFG_TYPE_F32;
  auto n = [](int64_t M, int64_t N) { return (double)tiles(M, 32) * tiles(N, 32); };
  auto trips = [](int64_t K) { return (double)((K + 127) / 128); };
  double longest = 0, all = 0;
  if (what == FORWARD) {
    longest = (fp32 ? 1.0 : 0.5) * trips(I);
    all = (fp32 ? 0.0045 : 0.002) * (I % 8 ? 2 : 1) * n(R, O) * trips(I);
  }
  if (what & BACK_X) {
    longest = (fp32 ? 1.5 : 1.0) * trips(O);
    all += (fp32 ? 0.007 : 0.0085) * n(R, I) * trips(O);
  }
  if (what & BACK_W) {
    const double w = (fp32 ? 1.6 : 3.0) * trips(R);
    longest = longest > w ? longest : w;
    all += (fp32 ? 0.007 : 0.0085) * n(O, I) * trips(R);
  }
  return 3 + (longest > all ? longest : all);
}

void launch_direct_forward(const Args& a, int in_type, int out_type, hipStream_t st) {
  if (in_type == SPCFG_TYPE_F32) forward<float, float>(a, st);
  else if (out_type == SPCFG_TYPE_F32) forward<uint16_t, float>(a, st);
  else forward<uint16_t, uint16_t>(a, st);
}
void launch_direct_backward(const Args& a, int in_type, int out_type, hipStream_t st) {
  if (in_type == SPCFG_TYPE_F32) backward<float, float>(a, st);
  else if (out_type == SPCFG_TYPE_F32) backward<uint16_t, float>(a, st);
  else backward<uint16_t, uint16_t>(a, st);
}

}  // namespace dense
}  // namespace spcfg

// Dense layers, small products: C[m][n] = sum_k A[m][k] B[n][k] with matrix operands loaded from global memory straight into
// the registers of the matrix instructions, whatever their order, alignment and size:
//   forward       z = x W^T              A = x  (k = inputs),       B = W    (both run along k)
//   d x           dz W, dz = gy act'(z)  A = dz (k = outputs),      B = W^T  (W runs along n)
//   d W           dz^T x                 A = dz^T (k = rows),       B = x^T  (both run across k), with db = row sums of A
// One output tile of T x T per workgroup (T = 16 or 32, the size of a matrix instruction); its eight wavefronts take chunks of
// K in turn, several at a time with everything of theirs in flight, and meet once, in LDS, where the epilogue runs on whole
// rows of the tile.  Small products are bound by latency: a few trips to memory, a few matrix instructions and one exchange.
// fp32 operands are cut exactly into three bf16 pieces in registers and multiplied as six piece products (nt::Split3), dz is
// formed on the way, beside bf16 operands as two bf16 pieces (Split2).
#include <type_traits>

#include "dense.h"

namespace spcfg {
namespace dense {

namespace {

constexpr int kWaves = 8;
// Chunks of K whose products are added up one behind the other, 256 a wavefront; the sums of such runs are added up in LDS.  A single
// running sum of 2^18 equal terms is off by 0.25 %.
constexpr int kRun = kWaves * 256;

typedef float floatx4 __attribute__((ext_vector_type(4)));

// pieces of eight K values of one row, ready for the matrix instruction
template <typename T> struct Pieces;
template <> struct Pieces<float> {
  Split3 s;
  __device__ __forceinline__ void set(const float (&v)[8]) {
    s.cut(make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7]));
  }
  __device__ __forceinline__ void raw(const float (&v)[8]) { set(v); }
  template <bool TWO> __device__ __forceinline__ void dz(const float (&v)[8]) { set(v); }
};
template <> struct Pieces<uint16_t> {
  Split2 s;
  __device__ __forceinline__ void raw(const uint16_t (&v)[8]) { __builtin_memcpy(&s.hi, v, 16); }
  template <bool TWO> __device__ __forceinline__ void dz(const float (&v)[8]) { s.cut(v, TWO); }
};

// the matrix instruction of T x T: 16 k, resp. 32; lane l holds row l % T of an operand, k = 8 (l / T) .. + 7
template <int T> struct Mma;
template <> struct Mma<32> {
  typedef floatx16 Acc;
  static constexpr int V = 16;
  static __device__ __forceinline__ int row(int v, int lane) { return (v >> 2) * 8 + (lane >> 5) * 4 + (v & 3); }
  static __device__ __forceinline__ Acc mul(uintx4 a, uintx4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct Mma<16> {
  typedef floatx4 Acc;
  static constexpr int V = 4;
  static __device__ __forceinline__ int row(int v, int lane) { return (lane >> 4) * 4 + v; }
  static __device__ __forceinline__ Acc mul(uintx4 a, uintx4 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <typename M, bool TWO>
__device__ __forceinline__ void product(const Pieces<float>& a, const Pieces<float>& b, typename M::Acc& c) {
  c = M::mul(a.s.lo, b.s.hi, c);
  c = M::mul(a.s.hi, b.s.lo, c);
  c = M::mul(a.s.mid, b.s.mid, c);
  c = M::mul(a.s.mid, b.s.hi, c);
  c = M::mul(a.s.hi, b.s.mid, c);
  c = M::mul(a.s.hi, b.s.hi, c);
}
template <typename M, bool TWO>
__device__ __forceinline__ void product(const Pieces<uint16_t>& a, const Pieces<uint16_t>& b, typename M::Acc& c) {
  if (TWO) c = M::mul(a.s.lo, b.s.hi, c);
  c = M::mul(a.s.hi, b.s.hi, c);
}

// v[i] = element (row, k + i), i = 0 .. 7, of an operand that runs along k; zero from K on (what is loaded there is the row's last,
// so that no load hangs on a branch).  VEC: base and rows lie on 16 bytes and K is a multiple of 8; otherwise whole chunks are
// read 16 bytes at a time as well, wherever they lie, and only a row's last chunk value by value (fp32 333 x 141 x 474 forward and
// backward 4.6 and 9.1 us, value by value throughout 6.2 and 11.7).
template <typename T, bool VEC>
__device__ __forceinline__ void along(const T* __restrict__ row, int64_t k, int64_t K, bool whole, T (&v)[8]) {
  if (VEC) {
    const uintx4* p = reinterpret_cast<const uintx4*>(row + min(k, K - 8));
    uintx4 w[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = p[i];
    __builtin_memcpy(v, w, sizeof(v));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k < K ? v[i] : T(0);
  } else if (whole) {
    __builtin_memcpy(v, row + k, sizeof(v));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = row[min(k + i, K - 1)];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < K ? v[i] : T(0);
  }
}
// the same of an operand that runs across k: column `col` of rows k .. k + 7
template <typename T>
__device__ __forceinline__ void across(const T* __restrict__ p, int64_t ld, int64_t col, int64_t k, int64_t K, T (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = p[min(k + i, K - 1) * ld + col];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = k + i < K ? v[i] : T(0);
}

template <int T> constexpr int lds_floats() { return kWaves * T * T + kWaves * 64; }

// TWO: dz in two pieces (beside bf16 operands).  LONG: K may have more than one run (a kernel of its own: the branch that is never
// taken costs bf16 1024 x 256 x 256 backward 15.7 us instead of 13.4).
template <typename TI, typename TO, int FORM, bool VEC, int T, bool LONG, bool TWO = false>
__device__ __forceinline__ void tile_product(const Args& g, int64_t tm, int64_t tn, float* lds) {
  using M = Mma<T>;
  constexpr int KC = 512 / T;  // k of a chunk
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int fr = lane & (T - 1), fh = lane / T;
  const int64_t rows = FORM == DW ? g.O : g.R, N = FORM == FWD ? g.O : g.I;
  const int64_t K = FORM == FWD ? g.I : FORM == DX ? g.O : g.R;
  const int64_t m0 = tm * T, n0 = tn * T;
  const TI* x = static_cast<const TI*>(g.x);
  const TI* W = static_cast<const TI*>(g.W);
  const TO* gy = static_cast<const TO*>(g.grad_y);
  const TO* z = static_cast<const TO*>(g.preact_in);
  const bool slope = g.act != SPCFG_ACT_NONE;

  float* bl = lds + kWaves * T * T;  // [wave][64]
  // rows and columns past the end repeat the last one: their results are not stored
  const int64_t ra = min(m0 + fr, rows - 1), rb = min(n0 + fr, N - 1);

  // U chunks at a time: everything of theirs is asked for before any of it is used
  using T1 = typename std::conditional<FORM == FWD, TI, TO>::type;
  constexpr int U = FORM == FWD ? 4 : 2;
  const int64_t chunks = (K + KC - 1) / KC;
  typename M::Acc acc;
  float bsum = 0.0f;
#pragma unroll
  for (int v = 0; v < M::V; ++v) acc[v] = 0.0f;
  // the run's sums to those of the runs before it, each thread its own
  int64_t run = kRun;  // where the run ends
  auto add_run = [&]() {
#pragma unroll
    for (int v = 0; v < M::V; ++v) {
      float* at = lds + wave * T * T + M::row(v, lane) * T + fr;
      *at = LONG && run > kRun ? *at + acc[v] : acc[v];
      acc[v] = 0.0f;
    }
    if (FORM == DW) bl[wave * 64 + lane] = LONG && run > kRun ? bl[wave * 64 + lane] + bsum : bsum;
    bsum = 0.0f;
    run += kRun;
  };
  for (int64_t c0 = wave; c0 < chunks; c0 += kWaves * U) {
    if (LONG && c0 >= run) add_run();
    T1 va[U][8], vz[U][8];
    TI vb[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u > 0 && c0 + kWaves * u >= chunks) break;
      const int64_t k = (c0 + kWaves * u) * KC + fh * 8;
      const bool whole = (c0 + kWaves * u + 1) * KC <= K;
      if constexpr (FORM == FWD) {
        along<TI, VEC>(x + ra * g.I, k, K, whole, va[u]);
        along<TI, VEC>(W + rb * g.I, k, K, whole, vb[u]);
      } else {
        if constexpr (FORM == DX) {
          along<TO, VEC>(gy + ra * g.O, k, K, whole, va[u]);
          if (slope) along<TO, VEC>(z + ra * g.O, k, K, whole, vz[u]);
        } else {
          across<TO>(gy, g.O, ra, k, K, va[u]);
          if (slope) across<TO>(z, g.O, ra, k, K, vz[u]);
        }
        across<TI>(FORM == DX ? W : x, g.I, rb, k, K, vb[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u > 0 && c0 + kWaves * u >= chunks) break;
      Pieces<TI> A, B;
      if constexpr (FORM == FWD) {
        A.raw(va[u]);
      } else {
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = to_float<TO>(va[u][e]);
        if (slope) {
          float zz[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) zz[e] = to_float<TO>(vz[u][e]);
          times_slopes<8>(g.act, zz, d);
        }
        if (FORM == DW) bsum += ((d[0] + d[1]) + (d[2] + d[3])) + ((d[4] + d[5]) + (d[6] + d[7]));
        A.template dz<TWO>(d);
      }
      B.raw(vb[u]);
      product<M, TWO>(A, B, acc);
    }
  }

  add_run();
  __syncthreads();

  // the eight partial tiles, summed in the order of the wavefronts; a thread then owns whole columns of rows
  const Epilogue<TI, TO, FORM> ep(g);
  for (int e = threadIdx.x; e < T * T; e += 64 * kWaves) {
    const int64_t m = m0 + e / T, n = n0 + e % T;
    if (m >= rows || n >= N) continue;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += lds[w * T * T + e];
    ep.one(m * N + n, s, ep.bias_of(n, N));
  }
  if (FORM == DW && g.grad_bias && tn == 0 && threadIdx.x < T) {
    const int64_t m = m0 + threadIdx.x;
    if (m < rows) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int h = 0; h < 64 / T; ++h) s += bl[w * 64 + h * T + threadIdx.x];
      store_bias<TI>(g, m, s);
    }
  }
}

template <typename TI, typename TO, bool VEC, int T, bool LONG>
__global__ void __launch_bounds__(64 * kWaves) k_dense_forward(Args g, unsigned tiles_n, unsigned first) {
  __shared__ float lds[lds_floats<T>()];
  const unsigned b = first + blockIdx.x;
  tile_product<TI, TO, FWD, VEC, T, LONG>(g, b / tiles_n, b % tiles_n, lds);
}

// both products of the backward pass in one launch: the tiles of dx first, then those of dW (either may be absent)
template <typename TI, typename TO, bool VEC, int T, bool LONG, bool TWO>
__global__ void __launch_bounds__(64 * kWaves) k_dense_backward(Args g, unsigned tiles_x, unsigned tiles_i, unsigned first) {
  __shared__ float lds[lds_floats<T>()];
  const unsigned b = first + blockIdx.x;
  if (b < tiles_x) tile_product<TI, TO, DX, VEC, T, LONG, TWO>(g, b / tiles_i, b % tiles_i, lds);
  else tile_product<TI, TO, DW, VEC, T, LONG, TWO>(g, (b - tiles_x) / tiles_i, (b - tiles_x) % tiles_i, lds);
}

unsigned tiles(int64_t n, int t) { return (unsigned)((n + t - 1) / t); }

// Tiles of 16 where there are few of 32, or no more than 16 rows (us on 16 / 32: fp32 30 x 512 x 512 4.8 / 7.7,
// 333 x 141 x 474 5.7 / 4.6, backward 8.7 / 9.9, 200 x 512 x 512 backward 15.7 / 11, 1 x 512 x 10000 8.9 / 10.5).
constexpr int kFew = 160;

// n workgroups in as many launches as it takes: a launch has less than 2^32 threads
template <typename F>
void in_launches(unsigned n, F launch) {
  for (unsigned first = 0; first < n; first += kMostWorkgroups) launch(n - first < kMostWorkgroups ? n - first : kMostWorkgroups, first);
}

template <typename TI, typename TO, int T, bool LONG>
void forward(const Args& a, hipStream_t st) {
  const bool vec = on16(a.x) && on16(a.W) && a.I % 8 == 0;
  const unsigned tn = tiles(a.O, T);
  in_launches(tiles(a.R, T) * tn, [&](unsigned n, unsigned first) {
    if (vec) hipLaunchKernelGGL((k_dense_forward<TI, TO, true, T, LONG>), dim3(n), dim3(64 * kWaves), 0, st, a, tn, first);
    else hipLaunchKernelGGL((k_dense_forward<TI, TO, false, T, LONG>), dim3(n), dim3(64 * kWaves), 0, st, a, tn, first);
  });
}
template <typename TI, typename TO, int T, bool LONG, bool TWO>
void backward(const Args& a, hipStream_t st) {
  const bool vec = on16(a.grad_y) && on16(a.preact_in) && a.O % 8 == 0;
  const unsigned ti = tiles(a.I, T), tx = a.grad_x ? tiles(a.R, T) * ti : 0, tw = a.grad_W ? tiles(a.O, T) * ti : 0;
  in_launches(tx + tw, [&](unsigned n, unsigned first) {
    if (vec) hipLaunchKernelGGL((k_dense_backward<TI, TO, true, T, LONG, TWO>), dim3(n), dim3(64 * kWaves), 0, st, a, tx, ti, first);
    else hipLaunchKernelGGL((k_dense_backward<TI, TO, false, T, LONG, TWO>), dim3(n), dim3(64 * kWaves), 0, st, a, tx, ti, first);
  });
}
template <int T> bool is_long(int64_t K) { return K > (int64_t)kRun * (512 / T); }

template <typename TI, typename TO, int T>
void forward(const Args& a, hipStream_t st) {
  if (is_long<T>(a.I)) forward<TI, TO, T, true>(a, st);
  else forward<TI, TO, T, false>(a, st);
}
template <typename TI, typename TO, int T, bool TWO>
void backward(const Args& a, hipStream_t st) {
  if (is_long<T>(a.O > a.R ? a.O : a.R)) backward<TI, TO, T, true, TWO>(a, st);
  else backward<TI, TO, T, false, TWO>(a, st);
}
template <typename TI, typename TO>
void forward(const Args& a, hipStream_t st) {
  if (a.R <= 16 || tiles(a.R, 32) * tiles(a.O, 32) < kFew) forward<TI, TO, 16>(a, st);
  else forward<TI, TO, 32>(a, st);
}
template <typename TI, typename TO, bool TWO>
void backward(const Args& a, hipStream_t st) {
  const unsigned ti = tiles(a.I, 32), n = (a.grad_x ? tiles(a.R, 32) * ti : 0) + (a.grad_W ? tiles(a.O, 32) * ti : 0);
  if (n < kFew) backward<TI, TO, 16, TWO>(a, st);
  else backward<TI, TO, 32, TWO>(a, st);
}

}  // namespace

// 3 us to start and end; then whichever is longer, the trips of one wavefront through k (counted in 128 values of a workgroup) or
// those of all tiles on the whole chip, both fitted on tiles of 16 and 32; backward more where the slope reads z.  Measured (us for
// this kernel / on tiles in LDS): forward fp32 512^3 8.3 / 14, 2048 x 512 x 512 22 / 18, bf16 700^3 8.7 / 13, 8192 x 64 x 64 4.0 / 4.8,
// 5108 x 355 x 355 30 / 14; backward fp32 512^3 18 / 19, 2048 x 128 x 128 32 / 18, 300 x 2000 x 300 27 / 22; bf16 to fp32
// 4811 x 30 x 30 20 / 24, 512^3 9.6 / 12, 2048 x 128 x 128 17 / 14, 10 x 3692 x 3142 48 / 38.
double direct_us(int64_t R, int64_t I, int64_t O, int in_type, int act, int what) {
  const bool fp32 = in_type == SPCFG_TYPE_F32;
  auto n = [](int64_t M, int64_t N) { return (double)tiles(M, 32) * tiles(N, 32); };
  auto trips = [](int64_t K) { return (double)((K + 127) / 128); };
  double longest = 0, all = 0, count = 0;
  if (what == FORWARD) {
    count = n(R, O);
    const bool small = R <= 16 || count < kFew;
    longest = (fp32 ? (small ? 0.5 : 0.65) : small ? 0.25 : 0.68) * trips(I);
    all = (fp32 ? (small ? 0.0048 : 0.0041) : (small ? 0.0018 : 0.0019) * (I % 8 ? 1.48 : 1)) * count * trips(I);
  } else {
    double work = 0, k = 0;
    if (what & BACK_X) {
      count += n(R, I);
      work += n(R, I) * trips(O);
      k = trips(O);
    }
    if (what & BACK_W) {
      count += n(O, I);
      work += n(O, I) * trips(R);
      k = trips(R) > k ? trips(R) : k;
    }
    const bool small = count < kFew;
    const double slope = act == SPCFG_ACT_NONE ? 1 : fp32 ? 1.58 : 1.42;
    longest = (small ? 0.45 : fp32 ? 1.05 : 0.95) * k * slope;
    all = (fp32 ? (small ? 0.0095 : 0.0046) : small ? 0.0055 : 0.003) * work * slope;
  }
  return 3 + (longest > all ? longest : all);
}

void launch_direct_forward(const Args& a, int in_type, int out_type, hipStream_t st) {
  if (in_type == SPCFG_TYPE_F32) forward<float, float>(a, st);
  else if (out_type == SPCFG_TYPE_F32) forward<uint16_t, float>(a, st);
  else forward<uint16_t, uint16_t>(a, st);
}
void launch_direct_backward(const Args& a, int in_type, int out_type, hipStream_t st) {
  if (in_type == SPCFG_TYPE_F32) backward<float, float, false>(a, st);
  else if (out_type == SPCFG_TYPE_F32) backward<uint16_t, float, true>(a, st);
  else if (dz_pieces<uint16_t, uint16_t>(a.act) == 2) backward<uint16_t, uint16_t, true>(a, st);
  else backward<uint16_t, uint16_t, false>(a, st);
}

}  // namespace dense
}  // namespace spcfg

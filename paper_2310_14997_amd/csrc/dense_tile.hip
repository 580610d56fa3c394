// Dense layers, large products: C[m][n] = sum_k A(m,k) B(n,k) on tiles in LDS, operands as planes of 16-bit values.
//
//  * bf16 operands are one plane, read where they lie.
//  * fp32 operands of the forward product are two fp16 planes: a row is scaled by a power of two so that its largest value lies
//    in [2^14, 2^15), hi = fp16(v), lo = fp16(2^11 (v - hi)), and C = sum hi hi + 2^-11 sum (hi lo + lo hi), the two sums in
//    fp32 accumulators of their own.  hi + 2^-11 lo is v to 2^-23 (for values down to 2^-29 of their row's largest; below that to
//    2^-51 of it) and the dropped lo lo is at most 2^-22 of a term: 2^-21 of each term in all, with either sign, whatever a row's scale,
//    where the next form has 2^-23, for half its matrix work (2048 x 512 x 10000: 1.7e-7 off in relative L2, a sum of fp32 products
//    4.1e-7).  Without the 2^11 lo would lose bits from 2^-16 of the largest value on.
//  * fp32 operands of the backward products are cut exactly into three bf16 planes (nt::Split3: hi, mid, lo) and multiplied as
//    six piece products: these run across rows, whose scales could not be taken out of the sum.
//  * dz = grad_y * act'(z) is written as planes by the kernel that cuts, which adds up the bias's gradient on the way: three of
//    fp32 operands, as above; with bf16 operands two, hi = bf16(dz) and lo = bf16(dz - hi), dz to 2^-17, multiplied as two piece
//    products with the other operand's one; one where grad_y is bf16 and its slope 0 or 1, and dz is a bf16 value (none is needed
//    without an activation: dz is grad_y).
//  * Each operand runs along k (rows of x and W in the forward product, rows of dz in dx) or across it (W in dx, dz and x in
//    dW): nothing is transposed in memory.  Tiles go from global memory straight to LDS (16 bytes a lane), a step being
//    32 or 64 values of k: rows of 64 or 128 bytes along k, with the 16-byte piece XORed with bits 2..3, resp. 1..3 of the
//    row; across k rows of 128 or 64 columns, with the 64-byte piece XORed with the row mod 4, resp. bit 1 of it.  Operands
//    come out of LDS with ds_read_b128, resp. with the transposing ds_read_b64_tr_b16.
//  * The order of a step is written out: products of 16 k while the next 16 are read; behind the first products of the last 16
//    the barrier - each wavefront's loads of the next step have landed, nobody needs this step's tiles any more - then the
//    next step's first operands are read and this step's place is filled with the tiles of step + NS.
//  * Few tiles: k is split over workgroups, which leave fp32 partial tiles; a second launch adds them in order.
// No workgroup waits for another; sums run in an order fixed by the sizes.
// Bound by the matrix cores on wide layers (bf16 8192^3 1250 TFLOP/s, 8192 x 4096 x 4096 with gelu 241 to 250 us = 1100 to 1140;
// a library product of that size 1297), by LDS reads on tiles of 128 (700 to 800 TFLOP/s), by latency below some 2e9 products.
// Backward 2048 x 512 x 10000 from fp32 gradients of bf16 layers: 130 us, of them two planes of dz 29, tiles 88 (two piece
// products each, 950 TFLOP/s of them), joining parts 5.
#include <type_traits>
#include <utility>

#include "dense.h"

namespace spcfg {
namespace dense {

namespace {

using nt::dma16;
using nt::lds_address;
using nt::static_for;

typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

// What lies beyond the end of k reads as zero.
__device__ uintx4 g_zeros;

struct Product {
  const uint16_t *A, *B;
  int64_t lda, ldb, plane_a, plane_b;  // in elements
  int64_t M, N, K;                     // K: rows, resp. columns that may be read along k
  int steps, steps_per_split, splits;
  unsigned tiles_m, tiles_n, wgs;
  float* partial;                      // [splits][M][N] where splits > 1
  const int *exp_a, *exp_b;            // fp16 planes: powers of two that the rows of A and B are scaled by
};

// One operand of one plane: eight k of a row or column per lane.
struct Frag { uintx2 lo, hi; };
__device__ __forceinline__ bf16x8 operand(const Frag& f) {
  return __builtin_bit_cast(bf16x8, uintx4{f.lo[0], f.lo[1], f.hi[0], f.hi[1]});
}
__device__ __forceinline__ bf16x8 operand(const uintx4& f) { return __builtin_bit_cast(bf16x8, f); }
__device__ __forceinline__ void tie(Frag& f) { asm volatile("" : "+v"(f.lo), "+v"(f.hi)); }
__device__ __forceinline__ void tie(uintx4& f) { asm volatile("" : "+v"(f)); }

// PA and PB planes of A and B; a tile of BM x BN by WM x WN wavefronts; BK values of k a step; NS steps in LDS.  Two fp16 planes of
// either (HALVES) lie side by side, 32 values of one and the same 32 of the other, so that a step is a whole line of 128 bytes of
// each row: to loads they are one plane (MA = MB = 1) of ME = 64 values a step.
template <int PA_, int PB_, int BM_, int BN_, int WM_, int WN_, int BK_, int NS_> struct Shape {
  static constexpr int PA = PA_, PB = PB_, BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, NS = NS_;
  static constexpr bool HALVES = PA == 2 && PB == 2;
  static constexpr int NW = WM * WN, MI = BM / (32 * WM), NI = BN / (32 * WN);
  static constexpr int MA = HALVES ? 1 : PA, MB = HALVES ? 1 : PB, ME = HALVES ? 2 * BK : BK;
  static constexpr int RB = 2 * ME;                   // bytes of a row along k
  static constexpr int PTA = BM * RB, PTB = BN * RB;  // bytes of one plane's tile
  static constexpr int TILE_B = MA * PTA, STAGE = TILE_B + MB * PTB;  // where B's tiles begin, and a step's bytes
  static constexpr int LA = PTA / 1024, LB = PTB / 1024;  // 1 KB loads of a plane's tile
  static constexpr int NDA = MA * LA / NW, ND = NDA + MB * LB / NW;  // of a wavefront and step, the first NDA of A
  static constexpr int CH = BK / 16;                  // chunks of 16 k in a step
  static constexpr int PP = HALVES ? 3 : PA == 3 ? 6 : PA;  // piece products
  static constexpr int NM = PP * MI * NI;             // matrix instructions of a chunk
  static constexpr int NA = HALVES ? 2 : 1;           // sums: fp16 planes keep the small products apart
  static constexpr int kLds = NS * STAGE;
  static_assert(PA == PB ? PA <= 3 : PA == 2 && PB == 1, "one, two or three planes of both, or two of A and one of B");
  static_assert(LA % NW == 0 && LB % NW == 0, "loads of a plane's tile are dealt evenly");
  static_assert((BM < 128) == (BN < 128), "panels across k are as wide for both operands");
  static_assert((ME == 32 || ME == 64) && (!HALVES || BK == 32) && CH % 2 == 0 && NS >= 2 && ND * (NS - 1) < 64, "");
};

#define SPCFG_SB __builtin_amdgcn_sched_barrier(0);

// eight floats of a row of which `left` are there
__device__ __forceinline__ void put_floats(float* p, const float (&s)[8], int64_t left) {
  if (left >= 8) {
    put<float, 4>(p, {s[0], s[1], s[2], s[3]});
    put<float, 4>(p + 4, {s[4], s[5], s[6], s[7]});
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (u < left) p[u] = s[u];
  }
}
__device__ __forceinline__ void add_floats(const float* p, float (&s)[8], int64_t left) {
  if (left >= 8) {
    float a[4], b[4];
    get<float, 4>(p, a);
    get<float, 4>(p + 4, b);
#pragma unroll
    for (int u = 0; u < 4; ++u) { s[u] += a[u]; s[u + 4] += b[u]; }
  } else {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (u < left) s[u] += p[u];
  }
}

// One tile of one product: workgroup `b` of `all`, both counted from a multiple of 8.
template <typename S, typename TI, typename TO, int FORM>
__device__ __forceinline__ void tile_product(const Args& g, const Product& p, unsigned b, unsigned all, unsigned char* lds) {
  constexpr bool TA = FORM == DW, TB = FORM != FWD;
  constexpr int PA = S::PA, PB = S::PB, MI = S::MI, NI = S::NI, ND = S::ND, NM = S::NM, NS = S::NS, CH = S::CH, ME = S::ME;
  constexpr bool HALVES = S::HALVES;
  static_assert(!HALVES || FORM == FWD, "fp16 planes run along k");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % S::WM, wn = wave / S::WM;

  // which tile: each XCD takes a run of consecutive ones, which form blocks of up to 8 row tiles
  const unsigned xcd = b & 7;
  unsigned t = xcd * (all >> 3) + min(xcd, all & 7) + (b >> 3);
  const unsigned per_split = p.tiles_m * p.tiles_n;
  const int split = __builtin_amdgcn_readfirstlane(t / per_split);
  t -= split * per_split;
  const unsigned band = t / (8 * p.tiles_n), rows_here = min(8u, p.tiles_m - band * 8), in_band = t - band * 8 * p.tiles_n;
  // (divisions are done in vector registers: back to scalar ones, where everything that depends on the tile alone stays)
  const int tile_m = __builtin_amdgcn_readfirstlane(band * 8 + in_band % rows_here);
  const int tile_n = __builtin_amdgcn_readfirstlane(in_band / rows_here);
  const int64_t m0 = (int64_t)tile_m * S::BM, n0 = (int64_t)tile_n * S::BN;
  const int k0 = split * p.steps_per_split, k1 = min(p.steps, k0 + p.steps_per_split);

  // this wavefront's loads: entry e of [A planes | B planes], 1 KB each.  Along k: 16 rows of 64 or 8 of 128 bytes; across: 4
  // of 256 (8 of 128 in tiles of 64), ME rows of one panel of 128 (64) columns after those of the other.
  // Addresses are a base per operand and plane, the same for all lanes, plus 32 bits (the host checks that these do).
  const unsigned lds0 = lds_address(lds);
  unsigned e_off[ND], e_lds[ND];
  constexpr int RL = 1024 / S::RB;                               // rows of a load along k
  // across: columns of a panel, rows of a load, loads of a panel
  constexpr int PW = S::BM < 128 ? 64 : 128, RP = 512 / PW, QA = ME / RP;
  // row of those, and piece: XOR with bits of the row (the loads of a plane are RL rows apart, a multiple of 8)
  const int r_al = lane / (64 / RL), c_al = (lane & (64 / RL - 1)) ^ (ME == 32 ? (r_al >> 2) & 3 : 0);
  const int r_ac = lane / (64 / RP), key_ac = PW == 128 ? r_ac & 3 : (r_ac >> 1) & 1;
  const int c_ac = ((lane % (64 / RP) >> 2) ^ key_ac) * 32 + (lane & 3) * 8;
  static_for<0, ND>([&](auto j) {
    constexpr int jv = decltype(j)::value;
    constexpr bool isA = jv < S::NDA;
    constexpr int per = isA ? S::LA : S::LB, e0 = S::NW * (isA ? jv : jv - S::NDA), plane = e0 / per;
    const int q = wave + e0 % per;
    e_lds[jv] = (unsigned)((isA ? plane * S::PTA : S::TILE_B + plane * S::PTB) + q * 1024);
    const int64_t ld = isA ? p.lda : p.ldb, len = isA ? p.M : p.N, o0 = isA ? m0 : n0;
    if constexpr (isA ? TA : TB) {
      const int64_t col = min(o0 + q / QA * PW + c_ac, (len + 7) / 8 * 8 - 8) - o0;  // (never before the tile: o0 < len)
      e_off[jv] = (unsigned)(2 * ((RP * (q % QA) + r_ac) * ld + col));
    } else {
      const int piece = ME == 32 ? c_al : c_al ^ (((RL * q + r_al) >> 1) & 7);
      e_off[jv] = (unsigned)(2 * (min(o0 + RL * q + r_al, len - 1) - o0) * ld + 16 * piece);
    }
  });
  const int64_t step_a = TA ? 2 * ME * p.lda : 2 * ME, step_b = TB ? 2 * ME * p.ldb : 2 * ME;  // bytes a step
  const unsigned char* base[S::MA + S::MB];  // of the step that is loaded next; A's planes, then B's
  static_for<0, S::MA + S::MB>([&](auto pl) {
    constexpr int v = decltype(pl)::value;
    if constexpr (v < S::MA)
      base[v] = reinterpret_cast<const unsigned char*>(p.A + v * p.plane_a + (TA ? m0 : m0 * p.lda)) + k0 * step_a;
    else
      base[v] = reinterpret_cast<const unsigned char*>(p.B + (v - S::MA) * p.plane_b + (TB ? n0 : n0 * p.ldb)) + k0 * step_b;
    // (opaque: otherwise they are computed anew from kernel arguments inside the loop, and waiting for those waits for
    // operand reads as well)
    asm volatile("" : "+s"(base[v]));
  });
  int64_t by_a = step_a, by_b = step_b;
  asm volatile("" : "+s"(by_a), "+s"(by_b));
  auto load_one = [&](auto j, unsigned stage) {
    constexpr int jv = decltype(j)::value;
    constexpr bool isA = jv < S::NDA;
    constexpr int plane = S::NW * (isA ? jv : jv - S::NDA) / (isA ? S::LA : S::LB);
    dma16(base[isA ? plane : S::MA + plane] + e_off[jv], lds0 + stage + e_lds[jv]);
  };
  auto advance = [&]() {
#pragma unroll
    for (int v = 0; v < S::MA + S::MB; ++v) base[v] += v < S::MA ? by_a : by_b;
  };
  // the last step of all where k ends inside it: what lies beyond reads as zero
  const int last_left = (int)(p.K - (int64_t)(p.steps - 1) * ME);  // values of the last step, 1 .. ME
  const int whole = last_left < ME ? p.steps - 1 : p.steps;        // steps that are whole
  auto load_last = [&](unsigned stage) {
    static_for<0, ND>([&](auto j) {
      constexpr int jv = decltype(j)::value;
      constexpr bool isA = jv < S::NDA;
      constexpr int per = isA ? S::LA : S::LB, e0 = S::NW * (isA ? jv : jv - S::NDA), plane = e0 / per;
      const int q = wave + e0 % per;
      const int k = (isA ? TA : TB) ? RP * (q % QA) + r_ac : 8 * (ME == 32 ? c_al : c_al ^ (((RL * q + r_al) >> 1) & 7));
      const unsigned char* at = base[isA ? plane : S::MA + plane] + e_off[jv];
      dma16(k < last_left ? at : reinterpret_cast<const unsigned char*>(&g_zeros), lds0 + stage + e_lds[jv]);
    });
  };

  // operand reads: byte offsets inside a stage of the fragments of the first 16 k of plane 0
  unsigned fa[TA ? MI : 1], fb[TB ? NI : 1];
  {
    const int fr = lane & 31, fh = lane >> 5;
    const unsigned al = (unsigned)(fr * S::RB + (fh ^ (ME == 32 ? (fr >> 2) & 3 : (fr >> 1) & 7)) * 16);
    const int li = lane & 15, lq = lane >> 4;
    const unsigned ac = (unsigned)((8 * (lq >> 1) + (li >> 2)) * (2 * PW) + 32 * (lq & 1) + 8 * (li & 3));
    const int key = PW == 128 ? li >> 2 : (li >> 3) & 1;
    constexpr int PB = PW / 32;  // blocks of 32 columns of a panel
    if constexpr (TA) {
#pragma unroll
      for (int f = 0; f < MI; ++f) {
        const int blk = wm * MI + f;
        fa[f] = ac + (unsigned)(blk / PB * (ME * 2 * PW) + ((blk % PB) ^ key) * 64);
      }
    } else {
      fa[0] = al + (unsigned)(wm * MI * 32 * S::RB);
    }
    if constexpr (TB) {
#pragma unroll
      for (int f = 0; f < NI; ++f) {
        const int blk = wn * NI + f;
        fb[f] = S::TILE_B + ac + (unsigned)(blk / PB * (ME * 2 * PW) + ((blk % PB) ^ key) * 64);
      }
    } else {
      fb[0] = S::TILE_B + al + (unsigned)(wn * NI * 32 * S::RB);
    }
  }
  using FA = typename std::conditional<TA, Frag, uintx4>::type;
  using FB = typename std::conditional<TB, Frag, uintx4>::type;
  struct Chunk { FA a[PA][MI]; FB b[PB][NI]; };
  Chunk X, Y;
  // fragment r of a chunk: planes of A, then of B
  constexpr int NF = PA * MI + PB * NI;
  auto read_one = [&](Chunk& F, auto r, unsigned stage, auto chunk) {
    constexpr int rv = decltype(r)::value, cv = decltype(chunk)::value;
    if constexpr (rv < PA * MI) {
      constexpr int pl = rv / MI, f = rv % MI;
      if constexpr (TA) {
        const unsigned at = lds0 + stage + fa[f];
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(F.a[pl][f].lo) : "v"(at), "n"(pl * S::PTA + cv * 32 * PW));
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(F.a[pl][f].hi) : "v"(at), "n"(pl * S::PTA + cv * 32 * PW + 8 * PW));
      } else {
        const unsigned at = lds0 + stage + (fa[0] ^ (cv * 32u + (HALVES ? pl * 64u : 0u)));
        asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(F.a[pl][f]) : "v"(at), "n"((HALVES ? 0 : pl * S::PTA) + f * 32 * S::RB));
      }
    } else {
      constexpr int pl = (rv - PA * MI) / NI, f = (rv - PA * MI) % NI;
      if constexpr (TB) {
        const unsigned at = lds0 + stage + fb[f];
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(F.b[pl][f].lo) : "v"(at), "n"(pl * S::PTB + cv * 32 * PW));
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(F.b[pl][f].hi) : "v"(at), "n"(pl * S::PTB + cv * 32 * PW + 8 * PW));
      } else {
        const unsigned at = lds0 + stage + (fb[0] ^ (cv * 32u + (HALVES ? pl * 64u : 0u)));
        asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(F.b[pl][f]) : "v"(at), "n"((HALVES ? 0 : pl * S::PTB) + f * 32 * S::RB));
      }
    }
  };
  auto wait_reads = [&](Chunk& F) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int f = 0; f < PA * MI; ++f) tie(F.a[f / MI][f % MI]);
#pragma unroll
    for (int f = 0; f < PB * NI; ++f) tie(F.b[f / NI][f % NI]);
  };
  floatx16 acc[S::NA][MI][NI];
#pragma unroll
  for (int a = 0; a < S::NA; ++a)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[a][i][j][v] = 0.0f;
  auto mfma_one = [&](Chunk& F, auto i) {
    constexpr int pp = decltype(i)::value / (MI * NI), rem = decltype(i)::value % (MI * NI), mi = rem / NI, ni = rem % NI;
    if constexpr (HALVES) {  // lo*hi and hi*lo into the second sum, hi*hi into the first (0 hi, 1 lo)
      constexpr int pa = pp == 0 ? 1 : 0, pb = pp == 1 ? 1 : 0, a = pp == 2 ? 0 : 1;
      acc[a][mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, F.a[pa][mi]),
                                                              __builtin_bit_cast(halfx8, F.b[pb][ni]), acc[a][mi][ni], 0, 0, 0);
    } else {  // three planes: lo*hi, hi*lo, mid*mid, mid*hi, hi*mid, hi*hi (0 hi, 1 mid, 2 lo); two of A: lo*B, hi*B (0 hi, 1 lo)
      constexpr int pa = PA < 3 ? PA - 1 - pp : pp == 0 ? 2 : (pp == 2 || pp == 3 ? 1 : 0);
      constexpr int pb = PA < 3 ? 0 : pp == 1 ? 2 : (pp == 2 || pp == 4 ? 1 : 0);
      acc[0][mi][ni] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(F.a[pa][mi]), operand(F.b[pb][ni]), acc[0][mi][ni], 0, 0, 0);
    }
  };

  const int n = k1 - k0;
  static_for<0, NS>([&](auto s) {
    constexpr int sv = decltype(s)::value;
    if (sv < n) {
      if (k0 + sv < whole) static_for<0, ND>([&](auto j) { load_one(j, sv * S::STAGE); });
      else load_last(sv * S::STAGE);
      advance();
    }
  });
  if (n >= NS) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND * (NS - 1)) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  SPCFG_SB
  if (n > 0) static_for<0, NF>([&](auto r) { read_one(X, r, 0u, std::integral_constant<int, 0>{}); });
  unsigned cur = 0;
  constexpr int RPF = (NF + NM - 1) / NM;                          // reads behind each product of the first half
  constexpr int NB = NM >= 8 ? 2 : 1, RS = NM - NB;                // products ahead of the barrier, and behind it
  constexpr int RPS = RS > 0 ? (NF + RS - 1) / RS : NF;
  for (int i = 0; i < n; ++i) {
    const unsigned nxt = cur + S::STAGE == NS * S::STAGE ? 0 : cur + S::STAGE;
    static_for<0, CH - 1>([&](auto c) {
      constexpr int cv = decltype(c)::value;
      Chunk &F = cv % 2 ? Y : X, &G = cv % 2 ? X : Y;
      SPCFG_SB
      wait_reads(F);
      SPCFG_SB
      static_for<0, NM>([&](auto m) {
        constexpr int mv = decltype(m)::value;
        mfma_one(F, m);
        SPCFG_SB
        static_for<0, RPF>([&](auto q) {
          constexpr int r = mv * RPF + decltype(q)::value;
          if constexpr (r < NF) read_one(G, std::integral_constant<int, r>{}, cur, std::integral_constant<int, cv + 1>{});
        });
        SPCFG_SB
      });
    });
    SPCFG_SB
    wait_reads(Y);
    SPCFG_SB
    static_for<0, NB>([&](auto m) { mfma_one(Y, m); });
    SPCFG_SB
    if (i + NS <= n) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ND * (NS - 2)) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    SPCFG_SB
    const bool more = i + NS < n && k0 + i + NS < whole;
    if (i + NS < n && k0 + i + NS >= whole) load_last(cur);
    SPCFG_SB
    if constexpr (RS == 0) {  // (a single product a chunk: nothing to put them between)
      static_for<0, NF>([&](auto r) { read_one(X, r, nxt, std::integral_constant<int, 0>{}); });
      if (more) static_for<0, ND>([&](auto j) { load_one(j, cur); });
    }
    static_for<NB, NM>([&](auto m) {
      constexpr int s = decltype(m)::value - NB;
      mfma_one(Y, m);
      SPCFG_SB
      static_for<0, RPS>([&](auto q) {
        constexpr int r = s * RPS + decltype(q)::value;
        if constexpr (r < NF) read_one(X, std::integral_constant<int, r>{}, nxt, std::integral_constant<int, 0>{});
      });
      if (more) {
        static_for<0, ND>([&](auto j) {
          if constexpr ((decltype(j)::value * RS) / ND == s) load_one(j, cur);
        });
      }
      SPCFG_SB
    });
    advance();
    cur = nxt;
  }
  wait_reads(X);  // (the last step read ahead into a place without new data: nothing of it is used)

  // Epilogue: 32 rows of a wavefront at a time go through its own part of LDS, from the accumulators' order (32 x 32 tile: column
  // lane % 32, row 8 (v / 4) + 4 (lane / 32) + v % 4) to eight adjacent columns a lane.  Rows there are 32 NI + 8 floats
  // apart: the two halves of a wavefront write rows four apart, in different banks; groups of four columns change places in
  // odd rows, so that the reads of adjacent rows are in different banks too.
  constexpr int LR = 32 * NI + 8, PER_ROW = 4 * NI, ROWS = 64 / PER_ROW;  // lanes of a row, rows at a time
  static_assert(S::NW * 32 * LR * 4 <= S::kLds, "the epilogue's rows fit");
  __syncthreads();  // (nobody reads operands any more)
  float* out = reinterpret_cast<float*>(lds) + wave * 32 * LR;
  const int odd = lane / PER_ROW % 2 * 4;
  const int64_t mw = m0 + wm * MI * 32 + lane / PER_ROW, c = n0 + wn * NI * 32 + lane % PER_ROW * 8;
  const Epilogue<TI, TO, FORM> ep(g);
  float* part = p.splits > 1 ? p.partial + (int64_t)split * p.M * p.N : nullptr;
  float bias[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) bias[u] = ep.bias_of(c + u, p.N);
  auto total = [&](int mi, int ni, int v) {
    return S::NA == 2 ? fmaf(acc[S::NA - 1][mi][ni][v], 0x1p-11f, acc[0][mi][ni][v]) : acc[0][mi][ni][v];
  };
  int down[8];
  if (HALVES) {
#pragma unroll
    for (int u = 0; u < 8; ++u) down[u] = p.exp_b[min(c + u, p.N - 1)];
  }
  static_for<0, MI>([&](auto i) {
    constexpr int mi = decltype(i)::value;
    static_for<0, 16 * NI>([&](auto w) {
      constexpr int v = decltype(w)::value / NI, ni = decltype(w)::value % NI;
      out[(8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * LR + ((ni * 32 + (lane & 31)) ^ ((v & 1) * 4))] = total(mi, ni, v);
    });
    // (a wavefront's own accesses to LDS are in order; the fences keep the compiler's)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int r = 0; r < 32; r += ROWS) {
      const int64_t m = mw + mi * 32 + r;
      const float* from = out + (r + lane / PER_ROW) * LR + lane % PER_ROW * 8;
      float s[8];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        s[u] = from[odd + u];
        s[u + 4] = from[4 - odd + u];
      }
      if (m >= p.M || c >= p.N) continue;
      if (HALVES) {
        const int e = p.exp_a[m];
#pragma unroll
        for (int u = 0; u < 8; ++u) s[u] = __builtin_amdgcn_ldexpf(s[u], -(e + down[u]));
      }
      if (part) put_floats(part + m * p.N + c, s, p.N - c);
      else ep.eight(m * p.N + c, s, bias, p.N - c);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  });
}

// The bias's gradient: 64 columns a workgroup, the parts of the rows dealt to the wavefronts, joined in their order.
template <int NW, typename TI>
__device__ __forceinline__ void bias_sums(const Args& g, const float* __restrict__ part, int parts, unsigned block, float* red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (int64_t)block * 64 + lane;
  constexpr int U = 8;  // sums of a thread: as many loads in flight, and shorter runs
  float f[U] = {};
  if (c < g.O) {
    for (int q = wave; q < parts; q += U * NW) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = part[(int64_t)min(q + u * NW, parts - 1) * g.O + c];
#pragma unroll
      for (int u = 0; u < U; ++u) f[u] += q + u * NW < parts ? v[u] : 0.0f;
    }
  }
  float s = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
  red[wave * 64 + lane] = s;
  __syncthreads();
  if (wave == 0 && c < g.O) {
#pragma unroll
    for (int w = 1; w < NW; ++w) s += red[w * 64 + lane];
    store_bias<TI>(g, c, s);
  }
}

// 2 wavefronts per SIMD or more; two workgroups per CU where LDS has room for them
template <typename S> constexpr int waves_per_simd() { return S::kLds <= 80 * 1024 ? 2 * S::NW / 4 : S::NW / 4; }

template <typename S, typename TI, typename TO>
__global__ void __launch_bounds__(64 * S::NW, waves_per_simd<S>()) k_dense_forward_tiles(Args g, Product p) {
  __shared__ __align__(1024) unsigned char lds[S::kLds];
  tile_product<S, TI, TO, FWD>(g, p, blockIdx.x, p.wgs, lds);
}

// Both products of the backward pass and the bias's gradient in one launch: the CUs that one leaves idle are the other's.  Each
// part's workgroups start at a multiple of 8, so that the XCD is the same function of either index.
template <typename S, typename TI, typename TO>
__global__ void __launch_bounds__(64 * S::NW, waves_per_simd<S>())
    k_dense_backward_tiles(Args g, Product px, Product pw, const float* sums, int parts) {
  __shared__ __align__(1024) unsigned char lds[S::kLds];
  unsigned b = blockIdx.x;
  const unsigned room_x = (px.wgs + 7) / 8 * 8, room_w = (pw.wgs + 7) / 8 * 8;
  if (b < room_x) {
    if (b < px.wgs) tile_product<S, TI, TO, DX>(g, px, b, px.wgs, lds);
  } else if ((b -= room_x) < room_w) {
    if (b < pw.wgs) tile_product<S, TI, TO, DW>(g, pw, b, pw.wgs, lds);
  } else {
    bias_sums<S::NW, TI>(g, sums, parts, b - room_w, reinterpret_cast<float*>(lds));
  }
}

// Partial tiles added up in the order of their k, eight columns a thread.
template <typename TI, typename TO, int FORM>
__device__ __forceinline__ void join(const Args& g, const Product& p, unsigned block, unsigned blocks) {
  const int64_t per_row = (p.N + 7) / 8, n = p.M * per_row, all = p.M * p.N;
  const Epilogue<TI, TO, FORM> ep(g);
  for (int64_t e = (int64_t)block * 256 + threadIdx.x; e < n; e += (int64_t)blocks * 256) {
    const int64_t m = e / per_row, c = (e - m * per_row) * 8;
    float s[8] = {}, bias[8];
#pragma unroll 4
    for (int q = 0; q < p.splits; ++q) add_floats(p.partial + q * all + m * p.N + c, s, p.N - c);
#pragma unroll
    for (int u = 0; u < 8; ++u) bias[u] = ep.bias_of(c + u, p.N);
    ep.eight(m * p.N + c, s, bias, p.N - c);
  }
}

template <typename TI, typename TO>
__global__ void __launch_bounds__(256) k_dense_forward_join(Args g, Product p) {
  join<TI, TO, FWD>(g, p, blockIdx.x, gridDim.x);
}
template <typename TI, typename TO>
__global__ void __launch_bounds__(256) k_dense_backward_join(Args g, Product px, Product pw, unsigned blocks_x) {
  if (blockIdx.x < blocks_x) join<TI, TO, DX>(g, px, blockIdx.x, blocks_x);
  else join<TI, TO, DW>(g, pw, blockIdx.x - blocks_x, gridDim.x - blocks_x);
}

// ---- planes --------------------------------------------------------------------------------------------------------------
// Rows and columns of a matrix in planes are rounded up to a step's 32, with zeros, so that products may run along either.
int64_t up32(int64_t n) { return (n + 31) / 32 * 32; }

__device__ __forceinline__ void put_planes(uint16_t* dst, int64_t plane, const float (&v)[8], float) {
  Split3 s;
  s.cut(make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7]));
  *reinterpret_cast<uintx4*>(dst) = s.hi;
  *reinterpret_cast<uintx4*>(dst + plane) = s.mid;
  *reinterpret_cast<uintx4*>(dst + 2 * plane) = s.lo;
}
__device__ __forceinline__ void put_planes(uint16_t* dst, int64_t, const float (&v)[8], uint16_t) {
  Split2 s;
  s.cut(v, false);
  *reinterpret_cast<uintx4*>(dst) = s.hi;
}
// dz as planes of the operands' type
__device__ __forceinline__ void put_dz(uint16_t* dst, int64_t plane, const float (&v)[8], bool, float) {
  put_planes(dst, plane, v, 0.0f);
}
__device__ __forceinline__ void put_dz(uint16_t* dst, int64_t plane, const float (&v)[8], bool two, uint16_t) {
  Split2 s;
  s.cut(v, two);
  *reinterpret_cast<uintx4*>(dst) = s.hi;
  if (two) *reinterpret_cast<uintx4*>(dst + plane) = s.lo;
}

// eight values of a row from column c on, zero outside the matrix (where the nearest ones inside are loaded: no load hangs on a
// branch of its own).  The eight that hold a row's end are its last, moved down.
template <typename T>
__device__ __forceinline__ void eight(const T* __restrict__ src, int64_t rows, int64_t cols, int64_t r, int64_t c, float (&v)[8]) {
  T x[8];
  const T* row = src + min(r, rows - 1) * cols;
  if (cols >= 8) {
    __builtin_memcpy(x, row + min(c, cols - 8), sizeof(x));
    if (cols & 7) {
      const int by = (int)min(c - min(c, cols - 8), (int64_t)7);
#pragma unroll
      for (int d = 4; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < 8 - d; ++i) x[i] = by & d ? x[i + d] : x[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = row[min(c + i, cols - 1)];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = r < rows && c + i < cols ? to_float<T>(x[i]) : 0.0f;
}

// Planes of one matrix, eight values a thread at a time, by `blocks` workgroups.
template <typename T>
__device__ __forceinline__ void cut(const T* __restrict__ src, uint16_t* __restrict__ dst, int64_t rows, int64_t cols, unsigned block,
                                    unsigned blocks) {
  const int64_t ld = (cols + 31) / 32 * 32, rows32 = (rows + 31) / 32 * 32;
  for (int64_t e = ((int64_t)block * 256 + threadIdx.x) * 8; e < rows32 * ld; e += (int64_t)blocks * (256 * 8)) {
    int64_t r, c;
    if (e < ((int64_t)1 << 31)) {  // (a division in 32 bits is far cheaper)
      r = (unsigned)e / (unsigned)ld;
      c = (unsigned)e - (unsigned)r * (unsigned)ld;
    } else {
      r = e / ld;
      c = e - r * ld;
    }
    float v[8];
    eight<T>(src, rows, cols, r, c, v);
    put_planes(dst + e, rows32 * ld, v, T());
  }
}

// dz = grad_y * act'(z) in planes (where dst is given) and, part by part of the rows, its sums over them (where sums is): 512
// columns and `span` rows a workgroup, a row per wavefront at a time.
template <typename TI, typename TO>
__device__ __forceinline__ void make_dz(const Args& g, uint16_t* __restrict__ dst, float* __restrict__ sums, int span,
                                        unsigned col_blocks, unsigned block, float (*red)[512]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (int64_t)(block % col_blocks) * 512 + lane * 8;
  const unsigned part = block / col_blocks;
  const int64_t ld = (g.O + 31) / 32 * 32, rows32 = (g.R + 31) / 32 * 32;
  const int64_t r1 = min(rows32, (int64_t)(part + 1) * span);
  const TO* gy = static_cast<const TO*>(g.grad_y);
  const TO* z = static_cast<const TO*>(g.preact_in);
  const bool two = dz_pieces<TI, TO>(g.act) == 2;
  float s[8] = {};
  if (c < ld) {
    // (four rows' loads in flight)
    for (int64_t r0 = (int64_t)part * span + wave; r0 < r1; r0 += 16) {
      float d[4][8], y[4][8];
#pragma unroll
      for (int u = 0; u < 4; ++u) eight<TO>(gy, g.R, g.O, r0 + 4 * u, c, d[u]);
      if (g.act != SPCFG_ACT_NONE) {
#pragma unroll
        for (int u = 0; u < 4; ++u) eight<TO>(z, g.R, g.O, r0 + 4 * u, c, y[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u) times_slopes<8>(g.act, y[u], d[u]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (dst && r0 + 4 * u < r1) put_dz(dst + (r0 + 4 * u) * ld + c, rows32 * ld, d[u], two, TI());
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += (d[0][i] + d[1][i]) + (d[2][i] + d[3][i]);
    }
  }
  if (!sums) return;
  if (wave) {
#pragma unroll
    for (int i = 0; i < 8; ++i) red[wave - 1][lane * 8 + i] = s[i];
  }
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < g.O)
        sums[(int64_t)part * g.O + c + i] = ((s[i] + red[0][lane * 8 + i]) + red[1][lane * 8 + i]) + red[2][lane * 8 + i];
  }
}

// What a product reads that is not there yet, in one launch: dz and the sums for the bias's gradient, planes of x, planes of W.
// Bound by HBM: 10 bytes a value of fp32 operands.
struct Prepare {
  uint16_t *dz, *x, *W;
  float* sums;
  int span;
  unsigned col_blocks, blocks_z, blocks_x, blocks_W;  // workgroups of each
};
template <typename TI, typename TO>
__global__ void __launch_bounds__(256) k_dense_prepare(Args g, Prepare q) {
  __shared__ float red[3][512];
  unsigned b = blockIdx.x;
  if (b < q.blocks_z) make_dz<TI, TO>(g, q.dz, q.sums, q.span, q.col_blocks, b, red);
  else if ((b -= q.blocks_z) < q.blocks_x) cut<TI>(static_cast<const TI*>(g.x), q.x, g.R, g.I, b, q.blocks_x);
  else cut<TI>(static_cast<const TI*>(g.W), q.W, g.O, g.I, b - q.blocks_x, q.blocks_W);
}

// fp16 planes of the rows of x and W and the powers of two that they are scaled by.  A group of `group` lanes (a power of two, eight
// values a lane at a time) takes a row: its largest magnitude, then the pieces.  Up to 32 values a lane stay in registers
// in between, longer rows are read again.  A row of zeros, or with an infinity in it, keeps its scale.
struct Halves {
  const float* src[2];
  _Float16* dst[2];
  int* exps[2];
  int64_t rows[2], cols;
  unsigned blocks0;  // workgroups of the first matrix
  int group;
};
__global__ void __launch_bounds__(256) k_dense_halves(Halves h) {
  const int w = blockIdx.x >= h.blocks0;
  const int G = h.group, gl = threadIdx.x & (G - 1);
  const int64_t r = (int64_t)(blockIdx.x - (w ? h.blocks0 : 0)) * (256 / G) + threadIdx.x / G;
  if (r >= h.rows[w]) return;  // (whole groups at a time)
  const float* src = h.src[w];
  const int64_t cols = h.cols, ld = (cols + 31) / 32 * 32;
  constexpr int E = 4;
  float v[E][8];
  float m = 0.0f;
  const bool kept = ld <= (int64_t)G * 8 * E;
  if (kept) {
#pragma unroll
    for (int e = 0; e < E; ++e) eight<float>(src, h.rows[w], cols, r, ((int64_t)e * G + gl) * 8, v[e]);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[e][i]));
  } else {
    for (int64_t c = gl * 8; c < ld; c += G * 8) {
      eight<float>(src, h.rows[w], cols, r, c, v[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[0][i]));
    }
  }
  for (int o = 1; o < G; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const int e = m > 0.0f && m < INFINITY ? 14 - __builtin_amdgcn_frexp_expf(m) + 1 : 0;  // (m = f 2^x with f in [1/2, 1))
  if (gl == 0) h.exps[w][r] = e;
  auto put = [&](int64_t c, const float (&x)[8]) {
    if (c >= ld) return;
    halfx8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float s = __builtin_amdgcn_ldexpf(x[i], e);
      hi[i] = (_Float16)s;
      lo[i] = (_Float16)((s - (float)hi[i]) * 0x1p11f);
    }
    _Float16* d = h.dst[w] + 2 * r * ld + c / 32 * 64 + c % 32;
    *reinterpret_cast<halfx8*>(d) = hi;
    *reinterpret_cast<halfx8*>(d + 32) = lo;
  };
  if (kept) {
#pragma unroll
    for (int e2 = 0; e2 < E; ++e2) put(((int64_t)e2 * G + gl) * 8, v[e2]);
  } else {
    for (int64_t c = gl * 8; c < ld; c += G * 8) {
      eight<float>(src, h.rows[w], cols, r, c, v[0]);
      put(c, v[0]);
    }
  }
}

// ---- which form, and what it needs -----------------------------------------------------------------------------------------
int64_t tiles(int64_t n, int t) { return (n + t - 1) / t; }
// workgroups that cut a matrix of `n` values
unsigned cut_blocks(int64_t n) {
  const int64_t b = tiles(n / 8, 256);
  return b < (int64_t)kMostWorkgroups ? (unsigned)b : kMostWorkgroups;
}
// The most of k that one sum runs over, 2^12 matrix instructions one behind the other: longer ones are split whatever that costs.
constexpr int kLongestSum = 1 << 16;

// A product as tiles that go through all of k: `n` of them, of `steps` steps.
struct Work { int64_t n, steps; };

// Tiles of t x t: `room` workgroups at a time on the chip, `start` us to start and end one, `wait` us a step of bk that it takes
// alone (latency), `busy` us a step of one per CU at full rate, shares of `least` steps or more.
struct Tiling { int t, bk, room, least; double start, wait, busy; };
struct Choice { int t, sa, sb; double us; };

// Into how many workgroups each tile's steps are cut, for two products of one launch (or one, the other of no size), with one
// tiling.  A step takes what it takes alone or its share of the CU, whichever is longer; the launch is estimated as the longest
// workgroup where all run at once, as their mean with half the longest on top where they do not; splitting costs a launch
// more (6 us) and partial tiles written and read again at 4 TB/s.  Of the lengths that cut the longer product into 1, 2, 3, ... shares the best is taken.
// Measured (us): 4096 x 512 x 512 in fp32 (128 tiles of 128 x 128, 16 steps) in two 37, in one 30, on 64 x 64 24;
// bf16 8192 x 4096 x 4096 on 256 x 256 241, on 128 x 128 320; 2048 x 512 x 10000 61, 43; 512^3 on 128 x 128 9.7, on 64 x 64 6.9;
// backward with dz in two pieces, on 256, 128 and 64: 8192 x 2048 x 2048 289, 326, 411; 2048 x 512 x 10000 148, 133, 170;
// 512^3 30, 15.5, 12.
void consider(const Tiling& g, const int64_t (&a)[3], const int64_t (&b)[3], Choice* best) {
  auto work = [&](const int64_t (&d)[3]) {
    return Work{d[2] ? tiles(d[0], g.t) * tiles(d[1], g.t) : 0, tiles(d[2], g.bk)};
  };
  const Work wa = work(a), wb = work(b);
  const int64_t longer = wb.steps > wa.steps ? wb.steps : wa.steps;
  for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256}) {
    if (s > 1 && longer < (int64_t)s * g.least) break;
    if (s > 32 && tiles(longer, 32) <= kLongestSum / g.bk) break;
    if (tiles(longer, s) > kLongestSum / g.bk) continue;
    const int64_t len = tiles(longer, s), pa = wa.n ? tiles(wa.steps, (int)len) : 0;
    const int64_t pb = wb.n ? tiles(wb.steps, (int)len) : 0;
    const double wgs = (double)(wa.n * pa + wb.n * pb);
    if (wgs > kMostWorkgroups) continue;
    const double here = (wgs < g.room ? wgs : g.room) / 256;
    const double step = here * g.busy > g.wait ? here * g.busy : g.wait;
    const double ta = pa ? g.start + step * tiles(wa.steps, (int)pa) : 0;
    const double tb = pb ? g.start + step * tiles(wb.steps, (int)pb) : 0;
    const double most = ta > tb ? ta : tb, mean = (wa.n * pa * ta + wb.n * pb * tb) / g.room;
    double us = wgs <= g.room ? most : mean + 0.5 * most;
    if (us < most) us = most;
    const int64_t parts = (pa > 1 ? wa.n * pa : 0) + (pb > 1 ? wb.n * pb : 0);
    if (parts) us += 6 + 2e-6 * parts * g.t * g.t;
    if (us < best->us) *best = Choice{g.t, (int)(pa ? pa : 1), (int)(pb ? pb : 1), us};
  }
}

// What a call does and where it keeps it.
struct Plan {
  bool on;                 // whether the layer takes tiled products at all
  bool cut;                // x and W as planes (fp32, or rows that do not all lie on 16 bytes)
  int dz;                  // planes of dz that are written; 0: dz is grad_y
  int64_t x, w, z;         // elements of one plane of x, W, dz
  int span, parts;         // rows of a part of the bias's gradient
  Choice c;
  size_t off_x, off_w, off_e, off_z, off_sums, off_pa, off_pb, bytes;
};

// laid: whether x, W and (backward) grad_y lie on 16 bytes; where they do not, they are laid out in planes as rows of odd lengths are
// (bf16 8192 x 4096 x 4096 with GELU, all two bytes off: forward 310 us, 267 where they lie on 16 bytes, in registers 7068).
// known: the tiling, where it was chosen before.
Plan plan_of(int64_t R, int64_t I, int64_t O, int in_type, int out_type, int act, int what, bool laid,
             const Choice* known = nullptr) {
  Plan p{};
  const int64_t most = 1 << 22;  // rows that long have offsets inside a tile (256 rows, or 64 across k) of more than 32 bits
  if (R < 1 || I >= most || O >= most) return p;
  const bool fp32 = in_type == SPCFG_TYPE_F32;
  const int pl = fp32 ? 3 : 1;
  p.cut = fp32 || I % 8 != 0 || !laid;
  const int pz = fp32 ? 3 : out_type == SPCFG_TYPE_F32 ? dz_pieces<uint16_t, float>(act) : dz_pieces<uint16_t, uint16_t>(act);
  p.dz = what != FORWARD && (pz > 1 || act != SPCFG_ACT_NONE || O % 8 != 0 || !laid) ? pz : 0;
  p.x = up32(R) * up32(I);
  p.w = up32(O) * up32(I);
  p.z = up32(R) * up32(O);
  const int64_t cb = tiles(up32(O), 512);
  int64_t span = (up32(R) * cb / 1024 + 15) / 16 * 16;  // about 1024 workgroups, 16 rows at a time
  if (span < 16) span = 16;
  if (span > 2048) span = 2048;  // (128 additions one behind the other)
  p.span = (int)span;
  p.parts = (int)tiles(up32(R), p.span);
  const int64_t none[3] = {0, 0, 0}, f[3] = {R, O, I}, x[3] = {R, I, O}, w[3] = {O, I, R};
  const int64_t(&da)[3] = what == FORWARD ? f : what & BACK_X ? x : none;
  const int64_t(&db)[3] = what & BACK_W ? w : none;
  p.c.us = 1e30;
  if (known) {
    p.c = *known;
  } else if (fp32 && what == FORWARD) {
    consider(Tiling{64, 32, 512, 8, 5, 0.31, 0.29}, da, db, &p.c);
    consider(Tiling{128, 32, 512, 6, 5, 0.95, 0.8}, da, db, &p.c);
  } else if (fp32) {
    consider(Tiling{64, 32, 512, 8, 5, 0.45, 0.39}, da, db, &p.c);
    consider(Tiling{128, 32, 256, 6, 5, 1.2, 1.25}, da, db, &p.c);
  } else if (what != FORWARD && pz == 2) {  // two piece products
    consider(Tiling{64, 64, 512, 4, 5, 0.4, 0.3}, da, db, &p.c);
    consider(Tiling{128, 64, 512, 4, 5, 0.9, 0.8}, da, db, &p.c);
    consider(Tiling{256, 64, 256, 10, 15, 2, 2.5}, da, db, &p.c);
  } else {
    consider(Tiling{64, 64, 512, 4, 5, 0.3, what == FORWARD ? 0.3 : 0.25}, da, db, &p.c);
    consider(Tiling{128, 64, 512, 3, 5, 0.75, 0.67}, da, db, &p.c);
    consider(Tiling{256, 64, 256, 3, 15, 1.5, 1.75}, da, db, &p.c);
  }
  // beside the products: a launch for planes and dz, 3 us (backward, with two kinds of workgroups in both launches, 5) and its bytes at
  // 4 TB/s
  const double si = fp32 ? 4 : 2, so = out_type == SPCFG_TYPE_F32 ? 4 : 2;
  double bytes = 0;
  const double a_value = fp32 && what == FORWARD ? 8 : si * 2.5;
  if (p.cut) bytes += a_value * ((what != BACK_X ? (double)R * I : 0) + (what != BACK_W ? (double)O * I : 0));
  if (what != FORWARD) bytes += (double)R * O * ((act ? 2 : 1) * so + 2 * p.dz);
  const double us = p.c.us + (what == FORWARD ? 0.5 : 2) + (bytes > 0 ? 3 + bytes / 4e6 : 0);
  p.on = us < direct_us(R, I, O, in_type, act, what);
  if (!p.on) return p;
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at += (n + 255) / 256 * 256; return o; };
  p.off_x = take(p.cut ? (size_t)p.x * 2 * pl : 0);
  p.off_w = take(p.cut ? (size_t)p.w * 2 * pl : 0);
  p.off_e = take(fp32 && what == FORWARD ? (size_t)(R + O) * 4 : 0);
  p.off_z = take((size_t)p.z * 2 * p.dz);
  p.off_sums = take(what != FORWARD ? (size_t)p.parts * O * 4 : 0);
  p.off_pa = take(p.c.sa > 1 ? (size_t)p.c.sa * da[0] * da[1] * 4 : 0);
  p.off_pb = take(p.c.sb > 1 ? (size_t)p.c.sb * db[0] * db[1] * 4 : 0);
  p.bytes = at;
  return p;
}

// Grid and steps follow from the shape that is launched, so that the two cannot disagree; splits only go down from the plan's.
template <typename S> void shape_up(Product* p, int splits) {
  p->tiles_m = (unsigned)tiles(p->M, S::BM);
  p->tiles_n = (unsigned)tiles(p->N, S::BN);
  p->steps = (int)tiles(p->K, S::ME);
  p->steps_per_split = (int)tiles(p->steps, splits);
  p->splits = (int)tiles(p->steps, p->steps_per_split);
  p->wgs = p->tiles_m * p->tiles_n * p->splits;
}
unsigned join_blocks(const Product& p) {
  const int64_t n = p.splits > 1 ? tiles(p.M * tiles(p.N, 8), 256) : 0;
  return (unsigned)(n < 4096 ? n : 4096);
}

template <typename S, typename TI, typename TO>
void launch_forward(const Args& a, Product p, int splits, hipStream_t st) {
  shape_up<S>(&p, splits);
  hipLaunchKernelGGL((k_dense_forward_tiles<S, TI, TO>), dim3(p.wgs), dim3(64 * S::NW), 0, st, a, p);
  if (p.splits > 1) hipLaunchKernelGGL((k_dense_forward_join<TI, TO>), dim3(join_blocks(p)), dim3(256), 0, st, a, p);
}
template <typename S, typename TI, typename TO>
void launch_backward(const Args& a, Product x, Product w, int sx, int sw, const float* sums, int parts, hipStream_t st) {
  if (a.grad_x) shape_up<S>(&x, sx);
  if (a.grad_W) shape_up<S>(&w, sw);
  const unsigned n = (x.wgs + 7) / 8 * 8 + (w.wgs + 7) / 8 * 8 + (sums ? (unsigned)tiles(a.O, 64) : 0);
  hipLaunchKernelGGL((k_dense_backward_tiles<S, TI, TO>), dim3(n), dim3(64 * S::NW), 0, st, a, x, w, sums, parts);
  const unsigned jx = join_blocks(x), jw = join_blocks(w);
  if (jx + jw) hipLaunchKernelGGL((k_dense_backward_join<TI, TO>), dim3(jx + jw), dim3(256), 0, st, a, x, w, jx);
}

// The shapes of the products, by the planes of their operands: tiles of 64, 128 and (bf16) 256; at 128 and 256 two wavefronts per
// SIMD and workgroup, one issuing while the other waits
template <int PA, int PB> struct Shapes;
template <> struct Shapes<1, 1> {
  using T64 = Shape<1, 1, 64, 64, 2, 2, 64, 4>;
  using T128 = Shape<1, 1, 128, 128, 2, 4, 64, 2>;
  using T256 = Shape<1, 1, 256, 256, 2, 4, 64, 2>;
};
template <> struct Shapes<2, 1> {
  using T64 = Shape<2, 1, 64, 64, 2, 2, 64, 3>;
  using T128 = Shape<2, 1, 128, 128, 2, 4, 32, 3>;  // (2048 x 512 x 10000 133 us, with two steps of 64 151, two of 32 148)
  using T256 = Shape<2, 1, 256, 256, 2, 4, 32, 3>;
};
template <> struct Shapes<2, 2> {
  using T64 = Shape<2, 2, 64, 64, 2, 2, 32, 4>;
  using T128 = Shape<2, 2, 128, 128, 2, 4, 32, 2>;
};
template <> struct Shapes<3, 3> {
  using T64 = Shape<3, 3, 64, 64, 2, 2, 32, 3>;
  using T128 = Shape<3, 3, 128, 128, 2, 4, 32, 3>;
};

template <typename TI, typename TO>
void forward(const Args& a, const Plan& p, char* ws, hipStream_t st) {
  Product q{};
  q.M = a.R;
  q.N = a.O;
  q.partial = reinterpret_cast<float*>(ws + p.off_pa);
  if constexpr (std::is_same<TI, float>::value) {
    Halves h{};
    h.src[0] = static_cast<const float*>(a.x); h.src[1] = static_cast<const float*>(a.W);
    h.dst[0] = reinterpret_cast<_Float16*>(ws + p.off_x); h.dst[1] = reinterpret_cast<_Float16*>(ws + p.off_w);
    h.exps[0] = reinterpret_cast<int*>(ws + p.off_e); h.exps[1] = h.exps[0] + a.R;
    h.rows[0] = a.R; h.rows[1] = a.O;
    h.cols = a.I;
    h.group = 8;
    while (h.group < 64 && h.group * 8 < a.I) h.group *= 2;
    h.blocks0 = (unsigned)tiles(a.R, 256 / h.group);
    hipLaunchKernelGGL(k_dense_halves, dim3(h.blocks0 + (unsigned)tiles(a.O, 256 / h.group)), dim3(256), 0, st, h);
    q.A = reinterpret_cast<const uint16_t*>(h.dst[0]); q.B = reinterpret_cast<const uint16_t*>(h.dst[1]);
    q.exp_a = h.exps[0]; q.exp_b = h.exps[1];
    q.lda = q.ldb = q.K = 2 * up32(a.I);
  } else if (p.cut) {
    Prepare r{};
    r.x = reinterpret_cast<uint16_t*>(ws + p.off_x);
    r.W = reinterpret_cast<uint16_t*>(ws + p.off_w);
    r.blocks_x = cut_blocks(p.x);
    r.blocks_W = cut_blocks(p.w);
    hipLaunchKernelGGL((k_dense_prepare<TI, TO>), dim3(r.blocks_x + r.blocks_W), dim3(256), 0, st, a, r);
    q.A = r.x; q.B = r.W;
    q.lda = q.ldb = q.K = up32(a.I);
  } else {
    q.A = static_cast<const uint16_t*>(a.x); q.B = static_cast<const uint16_t*>(a.W);
    q.lda = q.ldb = q.K = a.I;
  }
  using S = typename std::conditional<std::is_same<TI, float>::value, Shapes<2, 2>, Shapes<1, 1>>::type;
  if (p.c.t == 64) return launch_forward<typename S::T64, TI, TO>(a, q, p.c.sa, st);
  if constexpr (!std::is_same<TI, float>::value) {
    if (p.c.t == 256) return launch_forward<typename S::T256, TI, TO>(a, q, p.c.sa, st);
  }
  launch_forward<typename S::T128, TI, TO>(a, q, p.c.sa, st);
}

template <typename S, typename TI, typename TO>
void backward(const Args& a, const Plan& p, char* ws, hipStream_t st) {
  const uint16_t *x = static_cast<const uint16_t*>(a.x), *W = static_cast<const uint16_t*>(a.W);
  const uint16_t* z = static_cast<const uint16_t*>(a.grad_y);
  int64_t ldi = a.I, ldo = a.O;
  Prepare r{};
  if (p.cut) {
    r.x = reinterpret_cast<uint16_t*>(ws + p.off_x);
    r.W = reinterpret_cast<uint16_t*>(ws + p.off_w);
    if (a.grad_W) r.blocks_x = cut_blocks(p.x);
    if (a.grad_x) r.blocks_W = cut_blocks(p.w);
    x = r.x; W = r.W; ldi = up32(a.I);
  }
  if (a.grad_bias) r.sums = reinterpret_cast<float*>(ws + p.off_sums);
  if (p.dz) { r.dz = reinterpret_cast<uint16_t*>(ws + p.off_z); z = r.dz; ldo = up32(a.O); }
  if (r.dz || r.sums) {
    r.span = p.span;
    r.col_blocks = (unsigned)tiles(up32(a.O), 512);
    r.blocks_z = r.col_blocks * p.parts;
  }
  const unsigned n = r.blocks_z + r.blocks_x + r.blocks_W;
  if (n) hipLaunchKernelGGL((k_dense_prepare<TI, TO>), dim3(n), dim3(256), 0, st, a, r);
  const bool padded = p.cut && p.dz;  // whether the rows of both operands go on, as zeros, to a multiple of 32
  Product dx{}, dw{};
  dx.A = z; dx.lda = ldo; dx.plane_a = p.z;
  dx.B = W; dx.ldb = ldi; dx.plane_b = p.w;
  dx.M = a.R; dx.N = a.I;
  dx.K = padded ? up32(a.O) : a.O;
  dx.partial = reinterpret_cast<float*>(ws + p.off_pa);
  dw.A = z; dw.lda = ldo; dw.plane_a = p.z;
  dw.B = x; dw.ldb = ldi; dw.plane_b = p.x;
  dw.M = a.O; dw.N = a.I;
  dw.K = padded ? up32(a.R) : a.R;
  dw.partial = reinterpret_cast<float*>(ws + p.off_pb);
  if (p.c.t == 64) return launch_backward<typename S::T64, TI, TO>(a, dx, dw, p.c.sa, p.c.sb, r.sums, p.parts, st);
  if constexpr (!std::is_same<TI, float>::value) {
    if (p.c.t == 256) return launch_backward<typename S::T256, TI, TO>(a, dx, dw, p.c.sa, p.c.sb, r.sums, p.parts, st);
  }
  launch_backward<typename S::T128, TI, TO>(a, dx, dw, p.c.sa, p.c.sb, r.sums, p.parts, st);
}

}  // namespace

size_t tiled_workspace(int64_t R, int64_t I, int64_t O, int in_type, int out_type, int act) {
  size_t most = 0;
  for (int what : {FORWARD, BACK_X, BACK_W, BACK}) {
    const Plan p = plan_of(R, I, O, in_type, out_type, act, what, true);
    const size_t off16 = p.on ? plan_of(R, I, O, in_type, out_type, act, what, false, &p.c).bytes : 0;
    most = p.bytes > most ? p.bytes : most;
    most = off16 > most ? off16 : most;
  }
  return most;
}

bool tiled_forward(const Args& a, int in_type, int out_type, void* ws, hipStream_t st) {
  const Plan p = plan_of(a.R, a.I, a.O, in_type, out_type, a.act, FORWARD, on16(a.x) && on16(a.W));
  if (!p.on) return false;
  char* w = static_cast<char*>(ws);
  if (in_type == SPCFG_TYPE_F32) forward<float, float>(a, p, w, st);
  else if (out_type == SPCFG_TYPE_F32) forward<uint16_t, float>(a, p, w, st);
  else forward<uint16_t, uint16_t>(a, p, w, st);
  return true;
}

bool tiled_backward(const Args& a, int in_type, int out_type, void* ws, hipStream_t st) {
  const Plan p = plan_of(a.R, a.I, a.O, in_type, out_type, a.act, (a.grad_x ? BACK_X : 0) | (a.grad_W ? BACK_W : 0),
                         on16(a.x) && on16(a.W) && on16(a.grad_y));
  if (!p.on) return false;
  char* w = static_cast<char*>(ws);
  if (in_type == SPCFG_TYPE_F32) backward<Shapes<3, 3>, float, float>(a, p, w, st);
  else if (out_type == SPCFG_TYPE_F32) backward<Shapes<2, 1>, uint16_t, float>(a, p, w, st);
  else if (p.dz == 2) backward<Shapes<2, 1>, uint16_t, uint16_t>(a, p, w, st);
  else backward<Shapes<1, 1>, uint16_t, uint16_t>(a, p, w, st);
  return true;
}

}  // namespace dense
}  // namespace spcfg

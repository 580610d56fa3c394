// Distillation of rows of scores from a teacher's top entries, and its gradient.  Per row, with student scores s over V
// entries, teacher scores t at the entries id, temperature tau:
//   p = softmax(t / tau) over the entries that are there,   q = softmax(s / tau) over the row,   lse = log sum exp(s / tau)
//   loss = tau^2 sum_e p_e (log p_e - log q_id(e)),         d loss / d s_j = tau (q_j - sum_{e: id(e) = j} p_e)
// Bound by HBM: the row is read once and its gradient written once.  A row that a workgroup can hold in registers is one
// pass; longer rows are split over workgroups along V: one launch leaves each part's maximum and sum of exponentials (and, once
// a row, the teacher's part), a second one joins them and writes the gradient.  Maxima, sums and p are in 32 bits; logarithms
// and the sum over the teacher's entries, whose terms cancel where q is near p, in 64, and so is the sum of p of equal ids.
// 2048 rows of 10000 floats, k = 64, forward and backward: 32.6 us (5.0 TB/s; a copy of that size 30).  8 rows of 131071 bf16,
// k = 128: 9.3 us, two launches one behind the other.
#include <cmath>
#include <type_traits>

#include "spcfg_internal.h"

namespace spcfg {
namespace {

constexpr double kLog2e = 1.4426950408889634;
constexpr int kMostEntries = 1024;  // of the teacher's, a row: they are kept in LDS, 10 bytes each

typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<uint16_t>(uint16_t v) { return __uint_as_float((unsigned)v << 16); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t from_float<uint16_t>(float v) {
  return __builtin_bit_cast(uint16_t, (__bf16)v);
}

struct Args {
  int64_t R, V;
  int k, parts;         // parts of a row along V, `span` vectors of 16 bytes each
  int64_t span;
  float tau, by_two;    // by_two: log2(e) / tau
  const void *logits, *teacher;
  const int32_t* ids;
  const float* grad_loss;
  float *loss, *lse;
  const float* lse_in;
  void* grad;
  struct RowTeacher* rec;  // [R] what the first launch of a split call leaves for the second
  float2* stat;            // [R][parts]: maximum, sum of exp((s - maximum) / tau)
};
struct RowTeacher {
  float top, inv;       // p = exp((t - top) / tau) * inv
  int some, bad;
  double terms, sum;    // sum of p (log p - s / tau), sum of p
};

// exp(d / tau), d <= 0: three roundings of the exponent, as many as exp of d * (1 / tau) has, and a unit of the power; below 2^-126
// 0.  (With expf, which splits its argument, 4096 rows of 8000 bf16 scores take 38.8 us instead of 34.0.)
__device__ __forceinline__ float power(const Args& g, float d) { return __builtin_amdgcn_exp2f(d * g.by_two); }

// What a row's scores are taken from: their maximum, where that is -inf 0.  The sum is 0 then, lse = -inf, and loss and gradient are
// NaN, as 0 / 0 has it.
__device__ __forceinline__ float from_top(float m) { return m == -INFINITY ? 0.0f : m; }

// ---- sums and maxima over a workgroup of NT threads, N values at a time, in a fixed order --------------------------------
// (one barrier: a kernel gives each call 48 floats of its own)
template <typename F, typename X> __device__ __forceinline__ X across_wave(X v, F f) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, 64));
  return v;
}
template <int NT, int N, typename F>
__device__ __forceinline__ void all(float (&v)[N], float* red, F f) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = across_wave(v[i], f);
  if (NT == 64) return;
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) red[i * 16 + (threadIdx.x >> 6)] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = red[i * 16];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v[i] = f(v[i], red[i * 16 + w]);
  }
}
struct Add { template <typename X> __device__ __forceinline__ X operator()(X a, X b) const { return a + b; } };
struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// ---- a row in vectors of 16 bytes -------------------------------------------------------------------------------------
// Vector i holds the elements i * W - off .. + W - 1 of the row, off the row's offset from 16 bytes: whatever V and the
// base are, all but the row's ends are whole aligned vectors; the ends go element by element.
template <typename T> struct Row {
  static constexpr int W = 16 / (int)sizeof(T);
  const T* p;
  int64_t V;
  int off;
  __device__ __forceinline__ Row(const void* base, int64_t row, int64_t V_)
      : p(static_cast<const T*>(base) + row * V_), V(V_), off((int)(((uintptr_t)p & 15) / sizeof(T))) {}
  __device__ __forceinline__ int64_t vectors() const { return (V + off + W - 1) / W; }
  __device__ __forceinline__ bool whole(int64_t i) const { return i * W >= off && i * W - off + W <= V; }
  __device__ __forceinline__ void load(int64_t i, float (&x)[W]) const {  // -inf outside the row
    T v[W];
    if (whole(i)) {
      const uintx4 u = *reinterpret_cast<const uintx4*>(p + (i * W - off));
      __builtin_memcpy(v, &u, 16);
#pragma unroll
      for (int e = 0; e < W; ++e) x[e] = to_float<T>(v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const int64_t c = i * W - off + e;
        x[e] = c >= 0 && c < V ? to_float<T>(p[c]) : -INFINITY;
      }
    }
  }
  // o: the row's gradient, `same` where it has the row's offset from 16 bytes
  __device__ __forceinline__ void store(T* __restrict__ o, bool same, int64_t i, const float (&x)[W]) const {
    T v[W];
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] = from_float<T>(x[e]);
    if (same && whole(i)) {
      uintx4 u;
      __builtin_memcpy(&u, v, 16);
      *reinterpret_cast<uintx4*>(o + (i * W - off)) = u;
    } else {
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const int64_t c = i * W - off + e;
        if (c >= 0 && c < V) o[c] = v[e];
      }
    }
  }
};

// ---- the teacher's entries ---------------------------------------------------------------------------------------------
// in LDS, of k entries: a workgroup of one wavefront takes little of it, so that many fit a CU
struct Entries {
  int* id;         // -1 where absent
  float* w;        // the score, then exp((score - top) / tau)
  uint16_t* next;  // in a vector's chain
  __device__ __forceinline__ Entries(int* lds, int k)
      : id(lds), w(reinterpret_cast<float*>(lds + k)), next(reinterpret_cast<uint16_t*>(lds + 2 * k)) {}
};
unsigned entries_bytes(int k) { return (unsigned)(k * 10 + 15) / 16 * 16; }
struct Teacher {
  float top, inv;       // p = w * inv
  bool some, bad;       // whether any entry is there; whether an id is out of range or a score NaN or +inf
};

// Fills E with the row's ids and scores; an entry with a negative id or a score of -inf is absent, whatever else it holds.  This
// thread's share of the largest score, and of whether something is wrong.
template <typename T, int NT>
__device__ __forceinline__ void load_entries(const Args& g, int64_t row, Entries& E, float* top, float* wrong) {
  const T* t = static_cast<const T*>(g.teacher) + row * g.k;
  const int32_t* ids = g.ids + row * g.k;
  *top = -INFINITY;
  *wrong = 0.0f;
  for (int e = threadIdx.x; e < g.k; e += NT) {
    int id = ids[e];
    const float a = to_float<T>(t[e]);
    if (id >= 0 && a != -INFINITY && (id >= g.V || !(a < INFINITY))) *wrong = 1.0f;
    if (id >= g.V || a == -INFINITY) id = -1;
    E.id[e] = id < 0 ? -1 : id;
    E.w[e] = a;
    if (id >= 0) *top = fmaxf(*top, a);
  }
}
// E.w from scores to exponentials (each thread its own), and their sum over this thread's
template <int NT>
__device__ __forceinline__ float weigh_entries(const Args& g, Entries& E, float top) {
  float total = 0.0f;
  for (int e = threadIdx.x; e < g.k; e += NT) {
    const float w = E.id[e] >= 0 ? power(g, E.w[e] - top) : 0.0f;
    E.w[e] = w;
    total += w;
  }
  return total;
}
__device__ __forceinline__ Teacher teacher_of(float top, float wrong, float total) {
  Teacher t;
  t.top = top;
  t.bad = wrong != 0.0f;
  t.some = total > 0.0f || t.bad;
  t.inv = 1.0f / total;
  return t;
}
// between(): what else comes between the barrier that the ids are behind and the last one
template <typename T, int NT, typename F>
__device__ __forceinline__ Teacher teacher_row(const Args& g, int64_t row, Entries& E, float* red, F between) {
  float v[2];
  load_entries<T, NT>(g, row, E, &v[0], &v[1]);
  all<NT, 2>(v, red, Max());
  between();
  float total[1] = {weigh_entries<NT>(g, E, v[0])};
  all<NT, 1>(total, red + 48, Add());
  return teacher_of(v[0], v[1], total[0]);
}

// One wavefront: sum of p (log p - s / tau) and of p over the row's entries, in 64 bits.  E is complete (behind a barrier).
template <typename T>
__device__ __forceinline__ void loss_terms(const Args& g, int64_t row, const Entries& E, const Teacher& tr, double* terms,
                                           double* sum) {
  const T* t = static_cast<const T*>(g.teacher) + row * g.k;
  const T* s = static_cast<const T*>(g.logits) + row * g.V;
  const double inv_tau = 1.0 / g.tau, top = tr.top * inv_tau, log_inv = log((double)tr.inv);
  double a = 0.0, b = 0.0;
  for (int e = threadIdx.x & 63; e < g.k; e += 64) {
    const int id = E.id[e];
    const double p = id >= 0 ? (double)(E.w[e] * tr.inv) : 0.0;
    if (p > 0.0) {
      a += p * (to_float<T>(t[e]) * inv_tau - top + log_inv - to_float<T>(s[id]) * inv_tau);
      b += p;
    }
  }
  *terms = across_wave(a, Add());
  *sum = across_wave(b, Add());
}
__device__ __forceinline__ float loss_of(const Args& g, bool some, bool bad, double terms, double sum, double lse) {
  return bad ? NAN : some ? (float)((double)g.tau * g.tau * (terms + sum * lse)) : 0.0f;
}

// The gradient of a span of the row, E vectors a thread.  The entries that fall into a vector hang from its head as a chain
// (entry + 1, 0: none), so the thread that has the vector subtracts them before it stores it: no second look at the row, no wait
// for its stores.  hang comes when the heads are empty and the ids there, each behind a barrier, write behind another.  The
// chain's order is left open: equal ids are added up in the order of the list.
template <typename T, int NT, int N>
__device__ __forceinline__ void empty(int (&head)[N]) {
#pragma unroll
  for (int e = 0; e < N / NT; ++e) head[e * NT + threadIdx.x] = 0;
}
template <typename T, int NT, int N>
__device__ __forceinline__ void hang(const Args& g, const Entries& E, const Row<T>& s, int64_t first, int64_t last,
                                     int (&head)[N]) {
  for (int e = threadIdx.x; e < g.k; e += NT) {
    const int64_t id = E.id[e], i = (id + s.off) / Row<T>::W;
    if (id >= 0 && i >= first && i < last) E.next[e] = (uint16_t)atomicExch(&head[i - first], e + 1);
  }
}
// x: exp((s - m) / tau), by = scale * inv; p_of(e): p of entry e
template <typename T, int NT, int E, int N, typename P>
__device__ __forceinline__ void write(const Args& g, const Entries& ent, const Row<T>& s, int64_t row, int64_t first, int64_t last,
                                      const int (&head)[N], const float (&x)[E][Row<T>::W], float scale, float inv, P p_of) {
  constexpr int W = Row<T>::W;
  static_assert(N >= NT * E && E <= 32, "a head a vector");
  T* o = static_cast<T*>(g.grad) + row * g.V;
  const bool same = (((uintptr_t)o ^ (uintptr_t)s.p) & 15) == 0;
  const float by = scale * inv;
  unsigned held = 0;  // vectors with entries: one at a time, by code that is there once
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int64_t i = first + (int64_t)e * NT + threadIdx.x;
    if (i >= last) continue;
    if (head[e * NT + threadIdx.x] != 0 && scale != 0.0f) {
      held |= 1u << e;
      continue;
    }
    float v[W];
#pragma unroll
    for (int u = 0; u < W; ++u) v[u] = scale == 0.0f ? 0.0f : x[e][u] * by;
    s.store(o, same, i, v);
  }
  while (held) {
    const int at = __builtin_ctz(held);
    held &= held - 1;
    const int64_t i = first + (int64_t)at * NT + threadIdx.x;
    float q[W], v[W];
#pragma unroll
    for (int u = 0; u < W; ++u) {
      q[u] = x[0][u];
#pragma unroll
      for (int e = 1; e < E; ++e) q[u] = e == at ? x[e][u] : q[u];
      q[u] *= inv;
      v[u] = scale * q[u];
    }
    unsigned seen = 0, again = 0;
    const auto put = [&](int w, float p) {
#pragma unroll
      for (int u = 0; u < W; ++u) v[u] = u == w ? scale * (q[u] - p) : v[u];
    };
    for (int n = head[at * NT + threadIdx.x]; n != 0; n = ent.next[n - 1]) {
      const int w = (int)((ent.id[n - 1] + s.off) % W);
      again |= seen & (1u << w);
      seen |= 1u << w;
      put(w, p_of(n - 1));
    }
    while (again) {
      const int w = __builtin_ctz(again);
      again &= again - 1;
      const int id = (int)(i * W - s.off + w);
      double p = 0.0;  // of up to kMostEntries terms
      for (int e = 0; e < g.k; ++e)
        if (ent.id[e] == id) p += p_of(e);
      put(w, (float)p);
    }
    s.store(o, same, i, v);
  }
}

// what the row's loss counts, and what its gradient is scaled by; 0: the row is all zeros
__device__ __forceinline__ float row_weight(const Args& g, int64_t row) { return g.grad_loss ? g.grad_loss[row] : 1.0f; }
__device__ __forceinline__ float row_scale(const Args& g, float weight, bool some, bool bad) {
  if (weight == 0.0f || !some) return 0.0f;
  return bad ? NAN : weight * g.tau;
}

// ---- a row per workgroup, in registers ----------------------------------------------------------------------------------
// The gradient alone (no place for the loss) takes the row's sum again: an lse in 32 bits is good to 2^-24 of itself only, and q would
// be off by that much times |lse| (2.4e-5 at 400, scores of +-4 at a temperature of 0.01), all of a row to the same side.
template <typename T, int NT, int E, bool GRAD>
__global__ void __launch_bounds__(NT) k_distill_rows(Args g) {
  constexpr int W = Row<T>::W;
  __shared__ float red[96];
  extern __shared__ __attribute__((aligned(16))) int lds[];
  Entries ent(lds, g.k);
  __shared__ int head[GRAD ? NT * E : 1];
  const int64_t row = blockIdx.x;
  const Row<T> s(g.logits, row, g.V);
  const int64_t nv = s.vectors();
  const float weight = GRAD ? row_weight(g, row) : 0.0f;
  float x[E][W];
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e * NT < nv) s.load((int64_t)e * NT + threadIdx.x, x[e]);
  // maxima of the row and of the teacher's scores together, then both sums of exponentials
  float v[3] = {-INFINITY, 0.0f, 0.0f};
  load_entries<T, NT>(g, row, ent, &v[1], &v[2]);
  if constexpr (GRAD) empty<T, NT>(head);
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e * NT < nv) {
#pragma unroll
      for (int u = 0; u < W; ++u) v[0] = fmaxf(v[0], x[e][u]);
    }
  all<NT, 3>(v, red, Max());  // (behind it every entry's id is in LDS)
  if (NT == 64) __syncthreads();
  if constexpr (GRAD) hang<T, NT>(g, ent, s, 0, nv, head);
  const float m = from_top(v[0]);
  float sums[2] = {0.0f, weigh_entries<NT>(g, ent, v[1])};
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e * NT < nv) {
#pragma unroll
      for (int u = 0; u < W; ++u) {
        x[e][u] = power(g, x[e][u] - m);
        sums[0] += x[e][u];
      }
    }
  all<NT, 2>(sums, red + 48, Add());
  if (NT == 64) __syncthreads();
  const Teacher tr = teacher_of(v[1], v[2], sums[1]);
  const float inv = 1.0f / sums[0];
  if constexpr (GRAD) {
    const float scale = row_scale(g, weight, tr.some, tr.bad);
    write<T, NT, E>(g, ent, s, row, 0, nv, head, x, scale, inv, [&](int e) { return ent.w[e] * tr.inv; });
  }
  if (threadIdx.x < 64 && (!GRAD || g.loss)) {
    double terms, sum;
    loss_terms<T>(g, row, ent, tr, &terms, &sum);
    if (threadIdx.x == 0) {
      const double lse = (double)m / g.tau + log((double)sums[0]);
      g.loss[row] = loss_of(g, tr.some, tr.bad, terms, sum, lse);
      g.lse[row] = (float)lse;
    }
  }
}

// ---- rows split along V ---------------------------------------------------------------------------------------------------
constexpr int kPartThreads = 256;

// E: vectors of a thread
template <typename T, int E>
__global__ void __launch_bounds__(kPartThreads) k_distill_stats(Args g) {
  constexpr int W = Row<T>::W, NT = kPartThreads;
  __shared__ float red[96];
  extern __shared__ __attribute__((aligned(16))) int lds[];
  Entries ent(lds, g.k);
  const int64_t row = blockIdx.x / (g.parts + 1);
  const int part = (int)(blockIdx.x % (g.parts + 1));
  if (part == g.parts) {  // the row's teacher: what the second launch needs of it
    const Teacher tr = teacher_row<T, NT>(g, row, ent, red, [] {});
    if (threadIdx.x < 64) {
      double terms, all_p;
      loss_terms<T>(g, row, ent, tr, &terms, &all_p);
      if (threadIdx.x == 0) g.rec[row] = RowTeacher{tr.top, tr.inv, tr.some, tr.bad, terms, all_p};
    }
    return;
  }
  const Row<T> s(g.logits, row, g.V);
  const int64_t first = part * g.span, last = min(s.vectors(), first + g.span);
  float x[E][W];
  float m = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int64_t i = first + (int64_t)e * NT + threadIdx.x;
#pragma unroll
    for (int u = 0; u < W; ++u) x[e][u] = -INFINITY;
    if (i < last) s.load(i, x[e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int u = 0; u < W; ++u) m = fmaxf(m, x[e][u]);
  float top[1] = {m};
  all<NT, 1>(top, red, Max());
  m = top[0];
  float sum[1] = {0.0f};
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int u = 0; u < W; ++u) sum[0] += x[e][u] == -INFINITY ? 0.0f : power(g, x[e][u] - m);
  all<NT, 1>(sum, red + 48, Add());
  if (threadIdx.x == 0) g.stat[row * g.parts + part] = make_float2(m, sum[0]);
}

// JOIN: from the parts' maxima and sums and the row's record, part 0 writing loss and lse; otherwise from the lse that the caller
// kept, with the exponents s / tau - lse in 64 bits, so that the rounding of lse is all that q loses.  Where lse is not finite (it
// may not fit 32 bits at a tiny temperature) the gradient is NaN.
template <typename T, int E, bool JOIN, bool GRAD>
__global__ void __launch_bounds__(kPartThreads) k_distill_finish(Args g, int parts_here) {
  constexpr int W = Row<T>::W, NT = kPartThreads;
  __shared__ float red[96];
  extern __shared__ __attribute__((aligned(16))) int lds[];
  Entries ent(lds, g.k);
  __shared__ int head[GRAD ? NT * E : 1];
  const int64_t row = blockIdx.x / parts_here;
  const int part = (int)(blockIdx.x % parts_here), lane = threadIdx.x & 63;
  const Row<T> s(g.logits, row, g.V);
  const int64_t first = part * g.span, last = min(s.vectors(), first + g.span);
  float x[E][W];
  if constexpr (GRAD) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int64_t i = first + (int64_t)e * NT + threadIdx.x;
      if (i < last) s.load(i, x[e]);
    }
  }
  const float weight = GRAD ? row_weight(g, row) : 0.0f;
  if constexpr (GRAD) empty<T, NT>(head);
  Teacher tr;
  float m, inv;
  double by_two = 0.0, from = 0.0;
  if (JOIN) {
    // (every wavefront joins the parts for itself: no barrier to wait at)
    const RowTeacher rec = g.rec[row];
    tr.top = rec.top; tr.inv = rec.inv; tr.some = rec.some; tr.bad = rec.bad;
    if constexpr (GRAD) {
      float a, b;
      load_entries<T, NT>(g, row, ent, &a, &b);
      __syncthreads();
      hang<T, NT>(g, ent, s, first, last, head);
      __syncthreads();
    }
    m = -INFINITY;
    for (int c = lane; c < g.parts; c += 64) m = fmaxf(m, g.stat[row * g.parts + c].x);
    m = from_top(across_wave(m, Max()));
    float sum = 0.0f;
    for (int c = lane; c < g.parts; c += 64) {
      const float2 v = g.stat[row * g.parts + c];
      sum += v.y * power(g, v.x - m);  // (a part of nothing but -inf adds 0)
    }
    sum = across_wave(sum, Add());
    inv = 1.0f / sum;
    if (part == 0 && threadIdx.x == 0) {
      const double lse = (double)m / g.tau + log((double)sum);
      g.loss[row] = loss_of(g, tr.some, tr.bad, rec.terms, rec.sum, lse);
      g.lse[row] = (float)lse;
    }
  } else {
    tr = teacher_row<T, NT>(g, row, ent, red, [&] { hang<T, NT>(g, ent, s, first, last, head); });
    const float lse = g.lse_in[row];
    m = 0.0f;
    inv = fabsf(lse) < INFINITY ? 1.0f : NAN;
    by_two = kLog2e / g.tau;
    from = lse * kLog2e;
  }
  if constexpr (GRAD) {
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int u = 0; u < W; ++u)
        x[e][u] = JOIN ? power(g, x[e][u] - m) : __builtin_amdgcn_exp2f((float)(x[e][u] * by_two - from));
    write<T, NT, E>(g, ent, s, row, first, last, head, x, row_scale(g, weight, tr.some, tr.bad), inv,
                    [&](int e) { return (JOIN ? power(g, ent.w[e] - tr.top) : ent.w[e]) * tr.inv; });
  }
}

// ---- which form a call takes ---------------------------------------------------------------------------------------------
// A long row whole: 512 threads, so that a row is on its way at once and the registers allow two or more rows a CU, or 256 where
// that leaves fewer threads idle (forward and backward, threads x vectors: 2048 rows of 10000 bf16 scores, 1251 vectors: 256 x 6
// 28.6 us, 512 x 3 31.6, 256 x 16 46.6, but 64 rows 9.8 and 8.0; 64 rows of 10000 floats, 2500 vectors: 512 x 5 8.0, 256 x 10 10.7,
// 2048 rows 34.2 and 33.4; 4096 rows of 30000 bf16 scores: 512 x 8 145, 256 x 16 205).
// A part of a row is at most kPartThreads * each vectors: one a thread while that makes no more than kFewParts parts, the shortest
// way from the scores to the gradient (8 rows of 131071 bf16 scores, forward and backward: 9.3 us, with eight a thread 14.1), more as
// there are more rows, since each part reads the teacher's entries and the row's other parts' sums (100 rows of 131072 25.8 us, with
// one a thread 31.4).
constexpr int kMostEach = 8, kFewParts = 1024, kFewRows = 512;
struct Split { int parts, each; int64_t span; };
int64_t row_vectors(int64_t V, int W) { return (V + W - 1 + W - 1) / W; }  // at the worst offset
Split split_of(int64_t R, int64_t V, int W) {
  const int64_t nv = row_vectors(V, W);
  int each = 1;
  int64_t parts;
  for (;; each *= 2) {
    parts = (nv + kPartThreads * each - 1) / (kPartThreads * each);
    if (each == kMostEach || parts == 1 || R * parts <= kFewParts) break;
  }
  const int64_t span = (nv + parts - 1) / parts;
  return Split{(int)((nv + span - 1) / span), each, span};
}
bool in_registers(int64_t V, int W) { return row_vectors(V, W) <= 256 * 16; }

template <typename F>
void each(int n, F launch) {
  if (n == 1) launch(std::integral_constant<int, 1>());
  else if (n == 2) launch(std::integral_constant<int, 2>());
  else if (n == 4) launch(std::integral_constant<int, 4>());
  else launch(std::integral_constant<int, kMostEach>());
}

// rows that a workgroup holds
template <typename T, bool GRAD>
void launch_rows(const Args& a, hipStream_t st) {
  const int64_t nv = row_vectors(a.V, Row<T>::W);
  const unsigned lds = entries_bytes(a.k);
  const dim3 grid((unsigned)a.R);
  if (nv <= 64 * 2) hipLaunchKernelGGL((k_distill_rows<T, 64, 2, GRAD>), grid, dim3(64), lds, st, a);
  else if (nv <= 64 * 4) hipLaunchKernelGGL((k_distill_rows<T, 64, 4, GRAD>), grid, dim3(64), lds, st, a);
  else if (nv <= 256 * 4) hipLaunchKernelGGL((k_distill_rows<T, 256, 4, GRAD>), grid, dim3(256), lds, st, a);
  else if (a.R <= kFewRows && nv <= 512 * 3) hipLaunchKernelGGL((k_distill_rows<T, 512, 3, GRAD>), grid, dim3(512), lds, st, a);
  else if (nv <= 256 * 6) hipLaunchKernelGGL((k_distill_rows<T, 256, 6, GRAD>), grid, dim3(256), lds, st, a);
  else if (nv <= 512 * 5) hipLaunchKernelGGL((k_distill_rows<T, 512, 5, GRAD>), grid, dim3(512), lds, st, a);
  else hipLaunchKernelGGL((k_distill_rows<T, 512, 8, GRAD>), grid, dim3(512), lds, st, a);
}
template <typename T, bool GRAD>
void launch_forward(Args a, hipStream_t st) {
  constexpr int W = Row<T>::W;
  if (in_registers(a.V, W)) return launch_rows<T, GRAD>(a, st);
  const unsigned lds = entries_bytes(a.k);
  const Split sp = split_of(a.R, a.V, W);
  a.parts = sp.parts;
  a.span = sp.span;
  const int here = GRAD ? sp.parts : 1;
  each(sp.each, [&](auto e) {
    constexpr int E = decltype(e)::value;
    hipLaunchKernelGGL((k_distill_stats<T, E>), dim3((unsigned)(a.R * (sp.parts + 1))), dim3(kPartThreads), lds, st, a);
    hipLaunchKernelGGL((k_distill_finish<T, GRAD ? E : 1, true, GRAD>), dim3((unsigned)(a.R * here)), dim3(kPartThreads), lds, st, a,
                       here);
  });
}
template <typename T>
void launch_backward(Args a, hipStream_t st) {
  if (in_registers(a.V, Row<T>::W)) return launch_rows<T, true>(a, st);
  const Split sp = split_of(a.R, a.V, Row<T>::W);
  a.parts = sp.parts;
  a.span = sp.span;
  each(sp.each, [&](auto e) {
    hipLaunchKernelGGL((k_distill_finish<T, decltype(e)::value, false, true>), dim3((unsigned)(a.R * sp.parts)), dim3(kPartThreads),
                       entries_bytes(a.k), st, a, sp.parts);
  });
}

size_t need(int64_t R, int64_t V) {
  size_t most = 0;
  for (int W : {4, 8})
    if (!in_registers(V, W)) {
      const size_t n = (size_t)R * (sizeof(RowTeacher) + split_of(R, V, W).parts * sizeof(float2));
      if (n > most) most = n;
    }
  return (most + 255) / 256 * 256;
}

int check_sizes(int32_t R, int32_t V) {
  return R < 0 || V < 1 || R > (1 << 20) || V > (1 << 24) || (int64_t)R * V > ((int64_t)1 << 36) ? SPCFG_ERR_SHAPE : SPCFG_OK;
}

// checks what all three calls share and fills their arguments
int check(int32_t type, int32_t rows, int32_t V, int32_t k, const void* logits, const void* teacher, const int32_t* ids,
          float tau, Args* a) {
  if (type != SPCFG_TYPE_F32 && type != SPCFG_TYPE_BF16) return SPCFG_ERR_UNSUPPORTED;
  const int rc = check_sizes(rows, V);
  if (rc) return rc;
  if (k < 1 || k > kMostEntries) return SPCFG_ERR_SHAPE;
  const double by_two = kLog2e / tau;
  if (!(tau > 0.0f) || !(tau < INFINITY) || !((float)by_two < INFINITY)) return SPCFG_ERR_ARG;
  if (rows > 0 && (!logits || !teacher || !ids)) return SPCFG_ERR_ARG;
  const uintptr_t mask = type == SPCFG_TYPE_F32 ? 3 : 1;
  if (((uintptr_t)logits & mask) || ((uintptr_t)teacher & mask) || ((uintptr_t)ids & 3)) return SPCFG_ERR_ARG;
  *a = Args{};
  a->R = rows; a->V = V; a->k = k; a->tau = tau; a->by_two = (float)by_two;
  a->logits = logits; a->teacher = teacher; a->ids = ids;
  return SPCFG_OK;
}
int check_grad(int32_t type, const Args& a) {
  if (a.R > 0 && !a.grad) return SPCFG_ERR_ARG;
  return ((uintptr_t)a.grad & (type == SPCFG_TYPE_F32 ? 3 : 1)) != 0 ? SPCFG_ERR_ARG : SPCFG_OK;
}
// outputs are written while other workgroups read: nothing shares their memory
int check_memory(int32_t type, const Args& a, const void* ws) {
  for (const float* p : {(const float*)a.loss, (const float*)a.lse, a.grad_loss, a.lse_in})
    if ((uintptr_t)p & 3) return SPCFG_ERR_ARG;
  const int64_t size = type == SPCFG_TYPE_F32 ? 4 : 2, n = a.R * a.V * size;
  const Memory all[] = {{a.loss, a.R * 4}, {a.lse, a.R * 4}, {a.grad, n}, {ws, ws ? (int64_t)need(a.R, a.V) : 0}, {a.logits, n},
                        {a.teacher, a.R * a.k * size}, {a.ids, a.R * a.k * 4}, {a.grad_loss, a.R * 4}, {a.lse_in, a.R * 4}};
  return clash(all, 4, 9) ? SPCFG_ERR_ARG : SPCFG_OK;
}
int check_workspace(int64_t R, int64_t V, const void* ws, size_t bytes) {
  const size_t n = need(R, V);
  if (n == 0) return SPCFG_OK;
  if (!ws) return SPCFG_ERR_ARG;
  return ((uintptr_t)ws & 255) != 0 || bytes < n ? SPCFG_ERR_WORKSPACE : SPCFG_OK;
}

}  // namespace
}  // namespace spcfg

using namespace spcfg;

extern "C" {

int spcfg_distill_workspace_bytes(int32_t rows, int32_t V, size_t* out_bytes) {
  const int rc = check_sizes(rows, V);
  if (rc) return rc;
  if (!out_bytes) return SPCFG_ERR_ARG;
  *out_bytes = rows == 0 ? 0 : need(rows, V);
  return SPCFG_OK;
}

int spcfg_distill_forward(int32_t type, int32_t rows, int32_t V, int32_t k, const void* logits, const void* teacher_logits,
                          const int32_t* teacher_ids, float temperature, float* loss, float* lse, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  Args a;
  int rc = check(type, rows, V, k, logits, teacher_logits, teacher_ids, temperature, &a);
  if (rc) return rc;
  if (rows == 0) return SPCFG_OK;
  if (!loss || !lse) return SPCFG_ERR_ARG;
  a.loss = loss; a.lse = lse;
  if ((rc = check_memory(type, a, workspace))) return rc;
  if ((rc = check_workspace(rows, V, workspace, workspace_bytes))) return rc;
  a.rec = static_cast<RowTeacher*>(workspace); a.stat = reinterpret_cast<float2*>(a.rec + rows);
  if (type == SPCFG_TYPE_F32) launch_forward<float, false>(a, (hipStream_t)hip_stream);
  else launch_forward<uint16_t, false>(a, (hipStream_t)hip_stream);
  return launch_status();
}

int spcfg_distill_backward(int32_t type, int32_t rows, int32_t V, int32_t k, const void* logits, const void* teacher_logits,
                           const int32_t* teacher_ids, float temperature, const float* lse, const float* grad_loss,
                           void* grad_logits, void* hip_stream) {
  Args a;
  int rc = check(type, rows, V, k, logits, teacher_logits, teacher_ids, temperature, &a);
  if (rc) return rc;
  if (rows == 0) return SPCFG_OK;
  if (!lse) return SPCFG_ERR_ARG;
  a.lse_in = lse; a.grad_loss = grad_loss; a.grad = grad_logits;
  if ((rc = check_grad(type, a)) || (rc = check_memory(type, a, nullptr))) return rc;
  if (type == SPCFG_TYPE_F32) launch_backward<float>(a, (hipStream_t)hip_stream);
  else launch_backward<uint16_t>(a, (hipStream_t)hip_stream);
  return launch_status();
}

int spcfg_distill_forward_backward(int32_t type, int32_t rows, int32_t V, int32_t k, const void* logits,
                                   const void* teacher_logits, const int32_t* teacher_ids, float temperature,
                                   const float* grad_loss, float* loss, float* lse, void* grad_logits, void* workspace,
                                   size_t workspace_bytes, void* hip_stream) {
  Args a;
  int rc = check(type, rows, V, k, logits, teacher_logits, teacher_ids, temperature, &a);
  if (rc) return rc;
  if (rows == 0) return SPCFG_OK;
  if (!loss || !lse) return SPCFG_ERR_ARG;
  a.grad_loss = grad_loss; a.grad = grad_logits; a.loss = loss; a.lse = lse;
  if ((rc = check_grad(type, a)) || (rc = check_memory(type, a, workspace))) return rc;
  if ((rc = check_workspace(rows, V, workspace, workspace_bytes))) return rc;
  a.rec = static_cast<RowTeacher*>(workspace); a.stat = reinterpret_cast<float2*>(a.rec + rows);
  if (type == SPCFG_TYPE_F32) launch_forward<float, true>(a, (hipStream_t)hip_stream);
  else launch_forward<uint16_t, true>(a, (hipStream_t)hip_stream);
  return launch_status();
}

}  // extern "C"

// Distillation of rows of scores from a teacher's top entries, and its gradient.  Per row, with student scores s over V
// entries, teacher scores t at the entries id, temperature tau:
//   p = softmax(t / tau) over the entries that are there,   q = softmax(s / tau) over the row,   lse = log sum exp(s / tau)
//   loss = tau^2 sum_e p_e (log p_e - log q_id(e)),         d loss / d s_j = tau (q_j - sum_{e: id(e) = j} p_e)
// Bound by HBM: the row is read once and its gradient written once.  A row that a workgroup can hold in registers is one
// pass; longer rows, and few rows, are split over workgroups along V: one launch leaves each part's maximum and sum of
// exponentials, a second one joins them and writes the gradient.  Maxima, sums and p are in 32 bits; logarithms and the
// sum over the teacher's entries, whose terms cancel where q is near p, in 64.
#include <cmath>

#include "spcfg_internal.h"

namespace spcfg {
namespace {

constexpr int kMostEntries = 1024;  // of the teacher's, a row: they are kept in LDS

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
  float tau, inv_tau;
  const void *logits, *teacher;
  const int32_t* ids;
  const float* grad_loss;
  float *loss, *lse;
  const float* lse_in;
  void* grad;
  float2* stat;         // [R][parts]: maximum, sum of exp((s - maximum) / tau)
};

// ---- sums and maxima over a workgroup of NT threads, in a fixed order ------------------------------------------------
template <int NT, typename F, typename X>
__device__ __forceinline__ X all(X v, X* red, F f) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, 64));
  if (NT == 64) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) v = f(v, red[i]);
  return v;
}
template <int NT, typename X> __device__ __forceinline__ X all_sum(X v, X* red) {
  return all<NT>(v, red, [](X a, X b) { return a + b; });
}
template <int NT> __device__ __forceinline__ float all_max(float v, float* red) {
  return all<NT>(v, red, [](float a, float b) { return fmaxf(a, b); });
}

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
struct Entries {
  alignas(16) int id[kMostEntries];  // -1 where absent, and up to the next multiple of 4
  float p[kMostEntries];
};
struct Teacher {
  bool some, bad;           // whether any entry is there; whether an id is out of range or a score NaN
  double top, log_total;    // log p = t / tau - top - log_total
};

// Fills E with the row's ids and p; an entry with a negative id or a score of -inf is absent.
template <typename T, int NT>
__device__ Teacher teacher_row(const Args& g, int64_t row, Entries& E, float* red) {
  const T* t = static_cast<const T*>(g.teacher) + row * g.k;
  const int32_t* ids = g.ids + row * g.k;
  float top = -INFINITY, wrong = 0.0f;
  for (int e = threadIdx.x; e < g.k; e += NT) {
    int id = ids[e];
    const float a = to_float<T>(t[e]);
    if (id >= 0 && (id >= g.V || a != a)) wrong = 1.0f;
    if (id >= g.V || a == -INFINITY) id = -1;
    E.id[e] = id < 0 ? -1 : id;
    E.p[e] = a;
    if (id >= 0) top = fmaxf(top, a);
  }
  if (threadIdx.x < 3 && g.k + threadIdx.x < (unsigned)((g.k + 3) / 4 * 4)) E.id[g.k + threadIdx.x] = -1;
  top = all_max<NT>(top, red);
  wrong = all_max<NT>(wrong, red);
  float total = 0.0f;
  for (int e = threadIdx.x; e < g.k; e += NT) {
    const float w = E.id[e] >= 0 ? expf((E.p[e] - top) * g.inv_tau) : 0.0f;
    E.p[e] = w;
    total += w;
  }
  total = all_sum<NT>(total, red);
  Teacher r;
  r.bad = wrong != 0.0f || !(total < INFINITY);
  r.some = total > 0.0f || r.bad;
  const float inv = 1.0f / total;
  for (int e = threadIdx.x; e < g.k; e += NT) E.p[e] *= inv;
  __syncthreads();
  r.top = (double)top / g.tau;
  r.log_total = log((double)total);
  return r;
}

// loss of the row on every thread: entries' terms summed in 64 bits
template <typename T, int NT>
__device__ float row_loss(const Args& g, int64_t row, const Entries& E, const Teacher& tr, double lse, double* red) {
  const T* t = static_cast<const T*>(g.teacher) + row * g.k;
  const T* s = static_cast<const T*>(g.logits) + row * g.V;
  double sum = 0.0;
  for (int e = threadIdx.x; e < g.k; e += NT) {
    const int id = E.id[e];
    const double p = E.p[e];
    if (id >= 0 && p > 0.0) {
      const double log_p = (double)to_float<T>(t[e]) / g.tau - tr.top - tr.log_total;
      sum += p * (log_p - ((double)to_float<T>(s[id]) / g.tau - lse));
    }
  }
  sum = all_sum<NT>(sum, red);
  if (tr.bad) return NAN;
  return tr.some ? (float)((double)g.tau * g.tau * sum) : 0.0f;
}

// Gradient entries that the teacher has, for ids in [lo, hi): the first of equal ids writes what all of them add up to, in
// their order.  The caller's other entries have been written before a barrier.
template <typename T, int NT, typename Q>
__device__ void write_entries(const Args& g, int64_t row, const Entries& E, float scale, int64_t lo, int64_t hi, Q q_of) {
  T* o = static_cast<T*>(g.grad) + row * g.V;
  for (int e = threadIdx.x; e < g.k; e += NT) {
    const int id = E.id[e];
    const bool mine = id >= 0 && id >= lo && id < hi;
    if (!__any(mine)) continue;
    const float q = mine ? q_of(id) : 0.0f;
    // equal ids: any before this one, any behind it (four at a time; from k on there is no id)
    bool before = false, behind = false;
#pragma unroll 4
    for (int f = 0; f < g.k; f += 4) {
      const int4 at = *reinterpret_cast<const int4*>(&E.id[f]);
      const int v[4] = {at.x, at.y, at.z, at.w};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        before |= v[u] == id && f + u < e;
        behind |= v[u] == id && f + u > e;
      }
    }
    if (!mine || before) continue;
    float p = E.p[e];
    if (behind) {
      for (int f = e + 1; f < g.k; ++f)
        if (E.id[f] == id) p += E.p[f];
    }
    o[id] = from_float<T>(scale * (q - p));
  }
}

// what the gradient of a row is scaled by; 0: the row is all zeros
__device__ __forceinline__ float row_scale(const Args& g, int64_t row, const Teacher& tr) {
  const float w = g.grad_loss ? g.grad_loss[row] : 1.0f;
  if (w == 0.0f || !tr.some) return 0.0f;
  return tr.bad ? NAN : w * g.tau;
}

// ---- a row per workgroup, in registers ----------------------------------------------------------------------------------
template <typename T, int NT, int E, bool GRAD>
__global__ void __launch_bounds__(NT) k_distill_rows(Args g) {
  constexpr int W = Row<T>::W;
  __shared__ float red[16];
  __shared__ double redd[16];
  __shared__ Entries ent;
  const int64_t row = blockIdx.x;
  const Row<T> s(g.logits, row, g.V);
  const int64_t nv = s.vectors();
  float x[E][W];
  float m = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (e * NT < nv) {
      s.load((int64_t)e * NT + threadIdx.x, x[e]);
    }
  }
  const Teacher tr = teacher_row<T, NT>(g, row, ent, red);
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e * NT < nv) {
#pragma unroll
      for (int u = 0; u < W; ++u) m = fmaxf(m, x[e][u]);
    }
  m = all_max<NT>(m, red);
  float sum = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e * NT < nv) {
#pragma unroll
      for (int u = 0; u < W; ++u) {
        // outside the row -inf gives 0, unless the whole row is -inf: NaN, as the definition has it
        x[e][u] = expf((x[e][u] - m) * g.inv_tau);
        sum += x[e][u];
      }
    }
  sum = all_sum<NT>(sum, red);
  const double lse = (double)m / g.tau + log((double)sum);
  const float loss = row_loss<T, NT>(g, row, ent, tr, lse, redd);
  if (threadIdx.x == 0) {
    g.loss[row] = loss;
    g.lse[row] = (float)lse;
  }
  if (!GRAD) return;
  const float scale = row_scale(g, row, tr);
  T* o = static_cast<T*>(g.grad) + row * g.V;
  const bool same = (((uintptr_t)o ^ (uintptr_t)s.p) & 15) == 0;
  const float inv = 1.0f / sum, by = scale * inv;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e * NT < nv) {
#pragma unroll
      for (int u = 0; u < W; ++u) x[e][u] = scale == 0.0f ? 0.0f : x[e][u] * by;
      s.store(o, same, (int64_t)e * NT + threadIdx.x, x[e]);
    }
  if (scale == 0.0f) return;
  __syncthreads();
  write_entries<T, NT>(g, row, ent, scale, 0, g.V, [&](int id) {
    return expf((to_float<T>(s.p[id]) - m) * g.inv_tau) * inv;
  });
}

// ---- rows split along V ---------------------------------------------------------------------------------------------------
constexpr int kPartThreads = 256, kPartE = 8;

template <typename T>
__global__ void __launch_bounds__(kPartThreads) k_distill_stats(Args g) {
  constexpr int W = Row<T>::W, NT = kPartThreads;
  __shared__ float red[16];
  const int64_t row = blockIdx.x / g.parts;
  const int part = (int)(blockIdx.x % g.parts);
  const Row<T> s(g.logits, row, g.V);
  const int64_t first = part * g.span, last = min(s.vectors(), first + g.span);
  float x[kPartE][W];
  float m = -INFINITY;
#pragma unroll
  for (int e = 0; e < kPartE; ++e) {
    const int64_t i = first + (int64_t)e * NT + threadIdx.x;
#pragma unroll
    for (int u = 0; u < W; ++u) x[e][u] = -INFINITY;
    if (i < last) s.load(i, x[e]);
  }
#pragma unroll
  for (int e = 0; e < kPartE; ++e)
#pragma unroll
    for (int u = 0; u < W; ++u) m = fmaxf(m, x[e][u]);
  m = all_max<NT>(m, red);
  float sum = 0.0f;
#pragma unroll
  for (int e = 0; e < kPartE; ++e)
#pragma unroll
    for (int u = 0; u < W; ++u) sum += x[e][u] == -INFINITY ? 0.0f : expf((x[e][u] - m) * g.inv_tau);
  sum = all_sum<NT>(sum, red);
  if (threadIdx.x == 0) g.stat[row * g.parts + part] = make_float2(m, sum);
}

// JOIN: from the parts' maxima and sums, part 0 writing loss and lse; otherwise from the lse that the caller kept
template <typename T, bool JOIN, bool GRAD>
__global__ void __launch_bounds__(kPartThreads) k_distill_finish(Args g, int parts_here) {
  constexpr int W = Row<T>::W, NT = kPartThreads;
  __shared__ float red[16];
  __shared__ double redd[16];
  __shared__ Entries ent;
  const int64_t row = blockIdx.x / parts_here;
  const int part = (int)(blockIdx.x % parts_here);
  const Row<T> s(g.logits, row, g.V);
  const int64_t first = part * g.span, last = min(s.vectors(), first + g.span);
  float x[kPartE][W];
  if (GRAD) {
#pragma unroll
    for (int e = 0; e < kPartE; ++e) {
      const int64_t i = first + (int64_t)e * NT + threadIdx.x;
      if (i < last) s.load(i, x[e]);
    }
  }
  const Teacher tr = teacher_row<T, NT>(g, row, ent, red);
  float m, inv;
  if (JOIN) {
    m = -INFINITY;
    for (int c = threadIdx.x; c < g.parts; c += NT) m = fmaxf(m, g.stat[row * g.parts + c].x);
    m = all_max<NT>(m, red);
    float sum = 0.0f;
    for (int c = threadIdx.x; c < g.parts; c += NT) {
      const float2 v = g.stat[row * g.parts + c];
      sum += v.y * expf((v.x - m) * g.inv_tau);  // a part of nothing but -inf adds 0, a row of nothing else gives NaN
    }
    sum = all_sum<NT>(sum, red);
    inv = 1.0f / sum;
    if (part == 0) {
      const double lse = (double)m / g.tau + log((double)sum);
      const float loss = row_loss<T, NT>(g, row, ent, tr, lse, redd);
      if (threadIdx.x == 0) {
        g.loss[row] = loss;
        g.lse[row] = (float)lse;
      }
    }
  } else {
    m = g.lse_in[row] * g.tau;  // exp((s - tau lse) / tau) is q itself
    inv = 1.0f;
  }
  if (!GRAD) return;
  const float scale = row_scale(g, row, tr), by = scale * inv;
  T* o = static_cast<T*>(g.grad) + row * g.V;
  const bool same = (((uintptr_t)o ^ (uintptr_t)s.p) & 15) == 0;
#pragma unroll
  for (int e = 0; e < kPartE; ++e) {
    const int64_t i = first + (int64_t)e * NT + threadIdx.x;
    if (i < last) {
#pragma unroll
      for (int u = 0; u < W; ++u) x[e][u] = scale == 0.0f ? 0.0f : expf((x[e][u] - m) * g.inv_tau) * by;
      s.store(o, same, i, x[e]);
    }
  }
  if (scale == 0.0f) return;
  __syncthreads();
  write_entries<T, NT>(g, row, ent, scale, first * W - s.off, last * W - s.off, [&](int id) {
    return expf((to_float<T>(s.p[id]) - m) * g.inv_tau) * inv;
  });
}

// ---- which form a call takes ---------------------------------------------------------------------------------------------
// A part of a row: at most kPartThreads * kPartE vectors.
struct Split { int parts; int64_t span; };
int64_t row_vectors(int64_t V, int W) { return (V + W - 1 + W - 1) / W; }  // at the worst offset
Split split_of(int64_t R, int64_t V, int W) {
  const int64_t nv = row_vectors(V, W), most = kPartThreads * kPartE;
  int64_t parts = (nv + most - 1) / most;
  // few rows: enough parts for 512 workgroups, of at least one vector a thread
  const int64_t want = (512 + R - 1) / R, fit = (nv + kPartThreads - 1) / kPartThreads;
  const int64_t more = want < fit ? want : fit;
  if (parts < more) parts = more;
  const int64_t span = (nv + parts - 1) / parts;
  return Split{(int)((nv + span - 1) / span), span};
}
bool in_registers(int64_t R, int64_t V, int W) {
  (void)R;
  return row_vectors(V, W) <= 256 * 16;
}

template <typename T, bool GRAD>
void launch_forward(Args a, hipStream_t st) {
  constexpr int W = Row<T>::W;
  const int64_t nv = row_vectors(a.V, W);
  if (in_registers(a.R, a.V, W)) {
    const dim3 grid((unsigned)a.R);
    if (nv <= 64 * 4) hipLaunchKernelGGL((k_distill_rows<T, 64, 4, GRAD>), grid, dim3(64), 0, st, a);
    else if (nv <= 256 * 4) hipLaunchKernelGGL((k_distill_rows<T, 256, 4, GRAD>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_distill_rows<T, 256, 16, GRAD>), grid, dim3(256), 0, st, a);
    return;
  }
  const Split sp = split_of(a.R, a.V, W);
  a.parts = sp.parts;
  a.span = sp.span;
  hipLaunchKernelGGL((k_distill_stats<T>), dim3((unsigned)(a.R * sp.parts)), dim3(kPartThreads), 0, st, a);
  const int here = GRAD ? sp.parts : 1;
  hipLaunchKernelGGL((k_distill_finish<T, true, GRAD>), dim3((unsigned)(a.R * here)), dim3(kPartThreads), 0, st, a, here);
}
template <typename T>
void launch_backward(Args a, hipStream_t st) {
  const Split sp = split_of(a.R, a.V, Row<T>::W);
  a.parts = sp.parts;
  a.span = sp.span;
  hipLaunchKernelGGL((k_distill_finish<T, false, true>), dim3((unsigned)(a.R * sp.parts)), dim3(kPartThreads), 0, st, a, sp.parts);
}

size_t need(int64_t R, int64_t V) {
  size_t most = 0;
  for (int W : {4, 8})
    if (!in_registers(R, V, W)) {
      const size_t n = (size_t)R * split_of(R, V, W).parts * sizeof(float2);
      if (n > most) most = n;
    }
  return (most + 255) / 256 * 256;
}

int check_sizes(int32_t R, int32_t V) {
  return R < 0 || V < 1 || R > (1 << 20) || V > (1 << 24) || (int64_t)R * V > ((int64_t)1 << 36) ? SPCFG_ERR_SHAPE : SPCFG_OK;
}

bool overlap(const void* p, int64_t pb, const void* q, int64_t qb) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return p && q && a < b + (uintptr_t)qb && b < a + (uintptr_t)pb;
}

// checks what all three calls share and fills their arguments
int check(int32_t type, int32_t rows, int32_t V, int32_t k, const void* logits, const void* teacher, const int32_t* ids,
          float tau, Args* a) {
  if (type != SPCFG_TYPE_F32 && type != SPCFG_TYPE_BF16) return SPCFG_ERR_UNSUPPORTED;
  const int rc = check_sizes(rows, V);
  if (rc) return rc;
  if (k < 1 || k > kMostEntries) return SPCFG_ERR_SHAPE;
  if (!(tau > 0.0f) || !(tau < INFINITY) || !(1.0f / tau < INFINITY)) return SPCFG_ERR_ARG;
  if (rows > 0 && (!logits || !teacher || !ids)) return SPCFG_ERR_ARG;
  const uintptr_t mask = type == SPCFG_TYPE_F32 ? 3 : 1;
  if (((uintptr_t)logits & mask) || ((uintptr_t)teacher & mask) || ((uintptr_t)ids & 3)) return SPCFG_ERR_ARG;
  *a = Args{};
  a->R = rows; a->V = V; a->k = k; a->tau = tau; a->inv_tau = 1.0f / tau;
  a->logits = logits; a->teacher = teacher; a->ids = ids;
  return SPCFG_OK;
}
int check_grad(int32_t type, const Args& a, const void* grad) {
  const int64_t size = type == SPCFG_TYPE_F32 ? 4 : 2, n = a.R * a.V * size;
  if (a.R > 0 && !grad) return SPCFG_ERR_ARG;
  if ((uintptr_t)grad & (size - 1)) return SPCFG_ERR_ARG;
  if (overlap(grad, n, a.logits, n) || overlap(grad, n, a.teacher, a.R * a.k * size) || overlap(grad, n, a.ids, a.R * a.k * 4) ||
      overlap(grad, n, a.grad_loss, a.R * 4) || overlap(grad, n, a.lse_in, a.R * 4))
    return SPCFG_ERR_ARG;
  return SPCFG_OK;
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
  if ((rc = check_workspace(rows, V, workspace, workspace_bytes))) return rc;
  a.loss = loss; a.lse = lse; a.stat = static_cast<float2*>(workspace);
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
  if ((rc = check_grad(type, a, grad_logits))) return rc;
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
  a.grad_loss = grad_loss; a.grad = grad_logits;
  if ((rc = check_grad(type, a, grad_logits))) return rc;
  if ((rc = check_workspace(rows, V, workspace, workspace_bytes))) return rc;
  a.loss = loss; a.lse = lse; a.stat = static_cast<float2*>(workspace);
  if (type == SPCFG_TYPE_F32) launch_forward<float, true>(a, (hipStream_t)hip_stream);
  else launch_forward<uint16_t, true>(a, (hipStream_t)hip_stream);
  return launch_status();
}

}  // extern "C"

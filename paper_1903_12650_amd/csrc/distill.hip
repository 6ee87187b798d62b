// Distillation from a teacher's largest logits: their selection (topk_rows) and the loss and gradient of student logits against
// them (distill_fwd_bwd).
//
// Sums of exponentials run with their maximum: (m, s) stands for s * exp(m / T).  m starts at the lowest finite float, so that
// nothing is ever subtracted from an infinity of its own sign: a logit of -infinity adds exp(-infinity) = 0, a row of nothing else
// leaves s = 0, a logit of +infinity or NaN makes s NaN.
#include <float.h>

#include <algorithm>

#include "common.h"

namespace rn50 {

constexpr int kTopMax = 256;  // entries of a row, at most
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}
// exp(x) for x <= 0 with the hardware's exponential; `scale` = log2(e) / T.
__device__ __forceinline__ float exp_scaled(float x, float scale) { return __builtin_amdgcn_exp2f(x * scale); }

// ------------------------------------------------------------- largest logits
// The order of the logits as unsigned integers: -0 and +0 are one, a NaN is above everything.
__device__ __forceinline__ uint32_t order_key(float x) {
  uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  if (u == 0x80000000u) u = 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One workgroup per row.  The key of the k-th largest logit is found digit by digit (four of 8 bits, a histogram each over the
// logits that share the digits in front); logits above it are taken as they come, those equal to it in the order of their classes;
// a rank by counting puts them in order.  The row is read six times: right for every row, fast for none.
template <typename T>
__global__ __launch_bounds__(256) void topk_rows_kernel(const T* __restrict__ logits, int64_t ld, int N, int C, int k, float temperature,
                                                        float* __restrict__ values, int32_t* __restrict__ indices, float* __restrict__ tail) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t found[4];
  __shared__ uint32_t sel_key[kTopMax];
  __shared__ int sel_at[kTopMax];
  __shared__ int taken[5];
  __shared__ float red_m[4], red_s[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int n = blockIdx.x; n < N; n += gridDim.x) {
    const T* row = logits + n * ld;
    const int kk = min(k, C);
    uint32_t prefix = 0;
    int need = kk;  // how many are still to be taken among the logits that share the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
      hist[tid] = 0;
      __syncthreads();
      for (int i = tid; i < C; i += 256) {
        const uint32_t key = order_key(Elem<T>::load(row + i));
        if (shift == 24 || key >> (shift + 8) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        int above = 0, d = 255;
        while (d > 0 && above + static_cast<int>(hist[d]) < need) above += hist[d--];
        found[0] = d;
        found[1] = above;
      }
      __syncthreads();
      prefix = prefix << 8 | found[0];
      need -= found[1];
      __syncthreads();
    }
    if (tid == 0) taken[4] = 0;
    __syncthreads();
    // above the k-th key: kk - need of them, in any order; equal to it: the first `need` classes, counted chunk by chunk
    int equal = 0, last = -1;
    for (int base = 0; base < C; base += 256) {
      const int i = base + tid;
      const uint32_t key = i < C ? order_key(Elem<T>::load(row + i)) : 0;
      if (i < C && key > prefix) {
        const int at = atomicAdd(&taken[4], 1);
        sel_key[at] = key;
        sel_at[at] = i;
      }
      const bool eq = i < C && key == prefix;
      const uint64_t votes = __ballot(eq);
      if (lane == 0) taken[wave] = __popcll(votes);
      __syncthreads();
      int before = equal;
      for (int w = 0; w < wave; ++w) before += taken[w];
      const int pos = before + __popcll(votes & ((1ull << lane) - 1));
      if (eq && pos < need) {
        sel_key[kk - need + pos] = key;
        sel_at[kk - need + pos] = i;
        if (pos == need - 1) found[2] = i;
      }
      equal += taken[0] + taken[1] + taken[2] + taken[3];
      __syncthreads();
    }
    last = found[2];  // the last class that was taken among the equal ones
    if (tid < kk) {
      const uint32_t key = sel_key[tid];
      const int at = sel_at[tid];
      int rank = 0;
      for (int j = 0; j < kk; ++j) rank += sel_key[j] > key || (sel_key[j] == key && sel_at[j] < at);
      values[static_cast<int64_t>(n) * k + rank] = Elem<T>::load(row + at);
      indices[static_cast<int64_t>(n) * k + rank] = at;
    } else if (tid < k) {
      values[static_cast<int64_t>(n) * k + tid] = -INFINITY;
      indices[static_cast<int64_t>(n) * k + tid] = -1;
    }
    if (tail) {
      const float scale = kLog2e / temperature;
      float m = -FLT_MAX, s = 0.f;
      for (int i = tid; i < C; i += 256) {
        const float x = Elem<T>::load(row + i);
        const uint32_t key = order_key(x);
        if (key > prefix || (key == prefix && i <= last)) continue;
        const float top = fmaxf(m, x);
        s = s * exp_scaled(m - top, scale) + exp_scaled(x - top, scale);
        m = top;
      }
      const float wm = wave_max(m);
      const float wsum = wave_sum(s * exp_scaled(m - wm, scale));
      if (lane == 0) red_m[wave] = wm, red_s[wave] = wsum;
      __syncthreads();
      if (tid == 0) {
        const float top = fmaxf(fmaxf(red_m[0], red_m[1]), fmaxf(red_m[2], red_m[3]));
        float sum = 0.f;
        for (int w = 0; w < 4; ++w) sum += red_s[w] * exp_scaled(red_m[w] - top, scale);
        tail[n] = sum == 0.f ? -INFINITY : static_cast<float>(static_cast<double>(top) / temperature + log(static_cast<double>(sum)));
      }
    }
    __syncthreads();
  }
}

// --------------------------------------------------------- distillation loss
struct DistillArgs {
  const void* logits;
  void* grad;  // (or null)
  const float* t_values;
  const int32_t* t_indices;
  const float *t_tail, *row_weight;
  const int32_t* labels;
  float* row_loss;
  int64_t ld, grad_ld;
  int N, C, k;
  float temperature, alpha, smoothing, grad_scale;
};

// What a row's kernel has to know of the sums' exponentials.  The loss needs those of (z - m) / T and, with labels, of z - m.
// EXPS = 1: one of the two (T = 1, or alpha = 0 or 1); 2, 4: T = 2 or 4, whose second exponential is a power of the first (a
// multiplication or two in place of an exponential's four issue slots); 0: both.
struct Scales {
  float t, one;  // log2(e) / T and log2(e) (EXPS = 1: the one that is needed, twice)
  float slack;   // the reference stays while logits pass it by less than this: 2^20 in either sum
};
__device__ __forceinline__ Scales scales_of(const DistillArgs& a, int exps) {
  Scales s;
  s.t = exps == 1 && a.alpha == 0.f ? kLog2e : kLog2e / a.temperature;
  s.one = exps == 1 ? s.t : kLog2e;
  s.slack = 20.f / fmaxf(s.t, s.one);
  return s;
}

// A running sum of exponentials.  Its reference is a logit that has been seen, not the largest one: the sums lose nothing by a
// reference that is too low by less than `slack`, and moving it with every new maximum would cost two exponentials a vector.
template <int EXPS>
struct Sums {
  float ref = -FLT_MAX, lim = -FLT_MAX, st = 0.f, s1 = 0.f;
  __device__ __forceinline__ void one(float x, const Scales& sc) {
    const float d = x - ref, y = __builtin_amdgcn_exp2f(d * sc.t);
    st += y;
    if constexpr (EXPS == 2) s1 = fmaf(y, y, s1);
    if constexpr (EXPS == 4) {
      const float y2 = y * y;
      s1 = fmaf(y2, y2, s1);
    }
    if constexpr (EXPS == 0) s1 += __builtin_amdgcn_exp2f(d * sc.one);
  }
  template <int V>
  __device__ __forceinline__ void add(const float* x, const Scales& sc) {
    float top = x[0];
#pragma unroll
    for (int j = 1; j < V; ++j) top = fmaxf(top, x[j]);
    if (top > lim) {
      const float f = __builtin_amdgcn_exp2f((ref - top) * sc.t);
      st *= f;
      if constexpr (EXPS == 0) s1 *= __builtin_amdgcn_exp2f((ref - top) * sc.one);
      if constexpr (EXPS == 2) s1 *= f * f;
      if constexpr (EXPS == 4) s1 *= (f * f) * (f * f);
      ref = top;
      lim = top + sc.slack;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) one(x[j], sc);
  }
};

// The sums of a row (or of a slice of one), complete: s_t * exp((.) / T) and s_1 * exp(.) about `ref`, and the sum of the logits.
struct RowSums {
  float ref, st, s1;
  double sz;
};
// Sums of a workgroup's threads, in a fixed order; complete in every thread.  `red`: a RowSums for each wave.
template <int EXPS, int NT>
__device__ __forceinline__ RowSums block_sums(const Sums<EXPS>& a, double sz, bool want_sz, const Scales& sc, RowSums* red) {
  const int wave = threadIdx.x >> 6;
  RowSums r;
  r.ref = wave_max(a.ref);
  const float f = __builtin_amdgcn_exp2f((a.ref - r.ref) * sc.t);
  r.st = wave_sum(a.st * f);
  if constexpr (EXPS == 1) r.s1 = r.st;
  if constexpr (EXPS == 2) r.s1 = wave_sum(a.s1 * (f * f));
  if constexpr (EXPS == 4) r.s1 = wave_sum(a.s1 * ((f * f) * (f * f)));
  if constexpr (EXPS == 0) r.s1 = wave_sum(a.s1 * __builtin_amdgcn_exp2f((a.ref - r.ref) * sc.one));
  r.sz = want_sz ? wave_sum(sz) : 0.0;
  if constexpr (NT == 64) return r;
  if ((threadIdx.x & 63) == 0) red[wave] = r;
  __syncthreads();
  RowSums t = red[0];
  for (int w = 1; w < NT / 64; ++w) t.ref = fmaxf(t.ref, red[w].ref);
  t.st = t.s1 = 0.f;
  t.sz = 0.0;
  for (int w = 0; w < NT / 64; ++w) {
    const float d = red[w].ref - t.ref;
    t.st += red[w].st * __builtin_amdgcn_exp2f(d * sc.t);
    t.s1 += red[w].s1 * __builtin_amdgcn_exp2f(d * sc.one);
    t.sz += red[w].sz;
  }
  return t;
}

// What the gradient pass needs of its row: d = coef_t * exp((z - ref) / T) + coef_1 * exp(z - ref) - offset (EXPS = 1: both
// coefficients in coef_t) for every class; the classes at[0..special) get value[] instead.
struct RowGrad {
  float ref, coef_t, coef_1, offset;
};
struct RowShared {
  int at[kTopMax + 1];      // classes of the entries (-1: absent), then the label's if it is none of theirs
  float z[kTopMax + 1];     // their logits; z[kTopMax]: the label's
  float value[kTopMax + 1];
  RowGrad g;
};

// A row's loss and the coefficients of its gradient, by one wave.  Everything is relative to the largest logit and the largest
// cell, in double: the logarithms are those of sums of exponentials, and differences of them are small beside the logits.
// (Loops that are not unrolled: this is done once a row, and its registers are the kernel's.)
template <int EXPS>
__device__ __forceinline__ void row_finish(const DistillArgs& a, const Scales& sc, const RowSums& r, int n, float w, int label, RowShared& sh) {
  const int lane = threadIdx.x & 63;
  const bool kl_on = a.alpha > 0.f, ce_on = label >= 0;
  const int k = kl_on ? a.k : 0;
  const double t_inv = 1.0 / static_cast<double>(a.temperature), log2e = static_cast<double>(kLog2e);
  const float* tv = a.t_values + static_cast<int64_t>(n) * a.k;
  float M = r.ref;
  float vt = -INFINITY;  // (of the teacher's logits; its largest cell follows)
#pragma unroll 1
  for (int j = lane; j < k; j += 64)
    if (sh.at[j] >= 0) {
      M = fmaxf(M, sh.z[j]);
      vt = fmaxf(vt, tv[j]);
    }
  M = wave_max(M);
  vt = wave_max(vt);
  const float tail = kl_on && a.t_tail ? a.t_tail[n] : -INFINITY;
  const double Mt = fmax(static_cast<double>(tail), vt * t_inv);
  const bool empty = Mt == -INFINITY;
  const double tau = empty ? -INFINITY : static_cast<double>(tail) - Mt;
  // sums: the student's at T and at 1, the teacher's
  float eT = 0.f, e1 = 0.f, eS = 0.f;
#pragma unroll 1
  for (int j = lane; j < k; j += 64)
    if (sh.at[j] >= 0) {
      const float d = sh.z[j] - M, e = __builtin_amdgcn_exp2f(d * sc.t);
      eT += e;
      e1 += EXPS == 1 ? e : __builtin_amdgcn_exp2f(d * sc.one);
      eS += empty ? 0.f : __builtin_amdgcn_exp2f(static_cast<float>((tv[j] * t_inv - Mt) * log2e));
    }
  const float down = r.ref - M, pt = empty ? 0.f : __builtin_amdgcn_exp2f(static_cast<float>(tau * log2e));
  const double AT = static_cast<double>(wave_sum(eT)) + static_cast<double>(r.st) * __builtin_amdgcn_exp2f(down * sc.t);
  const double A1 = static_cast<double>(wave_sum(e1)) + static_cast<double>(r.s1) * __builtin_amdgcn_exp2f(down * sc.one);
  const double S = static_cast<double>(wave_sum(eS)) + pt;
  const bool none = AT == 0;  // every logit is -infinity
  // four logarithms at once (log 0 = -infinity)
  const double lg = log(lane == 0 ? AT : lane == 1 ? A1 : lane == 2 ? S : static_cast<double>(r.st));
  const double Z = __shfl(lg, 0, 64), Z1 = __shfl(lg, 1, 64), L = __shfl(lg, 2, 64);
  const double to_t = static_cast<double>(sc.t) / log2e, to_1 = static_cast<double>(sc.one) / log2e;  // the scales as the exponentials have them
  const double lam = static_cast<double>(down) * to_t + __shfl(lg, 3, 64);
  const double pr = pt / S, qr = static_cast<double>(r.st) * __builtin_amdgcn_exp2f(down * sc.t) / AT;
  const double g = none ? 0.0 : static_cast<double>(a.grad_scale) * w;
  const double gt = empty ? 0.0 : g * a.alpha * a.temperature, g1 = ce_on ? g * (1.0 - a.alpha) : 0.0;
  RowGrad c;
  c.ref = r.ref;
  c.coef_t = r.st == 0.f || gt == 0 ? 0.f : static_cast<float>(gt * (qr - pr) / r.st);
  c.coef_1 = g1 == 0 ? 0.f : static_cast<float>(g1 * __builtin_amdgcn_exp2f(down * sc.one) / A1);
  c.offset = static_cast<float>(g1 * a.smoothing / a.C);
  if constexpr (EXPS == 1) c.coef_t += c.coef_1;  // (the same exponential)
  double kl = 0;
  bool label_is_entry = false;
#pragma unroll 1
  for (int j = lane; j < k; j += 64)
    if (sh.at[j] >= 0) {
      const float d = sh.z[j] - M;
      float p = 0.f;
      if (!empty) {
        const double logp = tv[j] * t_inv - Mt - L;
        p = __builtin_amdgcn_exp2f(static_cast<float>(logp * log2e));
        if (p != 0.f) kl += p * (logp - ((static_cast<double>(sh.z[j]) - M) * to_t - Z));
      }
      double v = -static_cast<double>(c.offset);
      const float e = __builtin_amdgcn_exp2f(d * sc.t);
      if (gt != 0) v += gt * (e / AT - p);
      if (g1 != 0) v += g1 * (EXPS == 1 ? e : __builtin_amdgcn_exp2f(d * sc.one)) / A1;
      if (ce_on && sh.at[j] == label) v -= g1 * (1.0 - a.smoothing), label_is_entry = true;
      sh.value[j] = static_cast<float>(v);
    }
  kl = wave_sum(kl);
  if (pr != 0) kl += pr * ((tau - L) - (lam - Z));
  const float z_label = ce_on ? sh.z[kTopMax] : 0.f;
  const bool known = __any(label_is_entry);
  if (lane == 0) {
    double loss = 0;
    if (!none) {
      if (!empty) loss += static_cast<double>(a.alpha) * a.temperature * a.temperature * kl;
      if (ce_on) {
        double ce = -(1.0 - a.smoothing) * ((static_cast<double>(z_label) - M) * to_1 - Z1);
        if (a.smoothing > 0.f) ce -= static_cast<double>(a.smoothing) / a.C * ((r.sz - static_cast<double>(a.C) * M) - a.C * Z1);
        loss += (1.0 - a.alpha) * ce;
      }
    }
    a.row_loss[n] = static_cast<float>(loss);
    sh.at[kTopMax] = ce_on && !known ? label : -1;
    if (ce_on && !known) {
      const float d = z_label - c.ref, y = __builtin_amdgcn_exp2f(d * sc.t);
      float v = fmaf(c.coef_t, y, -c.offset);
      if constexpr (EXPS != 1) v += c.coef_1 * __builtin_amdgcn_exp2f(d * sc.one);
      sh.value[kTopMax] = v - static_cast<float>(g1 * (1.0 - a.smoothing));
    }
    sh.g = c;
  }
}

template <typename T>
struct RowOf {  // a row as vectors of V elements: whole ones, then what is left of the last, the rest of it -infinity
  static constexpr int V = Elem<T>::VEC;
  const T* p;
  int C;
  __device__ __forceinline__ Vec16 load(int v) const {
    const int i = v * V;
    Vec16 x;
    if (i + V <= C) {
      x = load16_any(p + i);
    } else {
      float f[V];
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = i + j < C ? Elem<T>::load(p + i + j) : -INFINITY;
      Elem<T>::pack(f, x);
    }
    return x;
  }
};
template <typename T>
__device__ __forceinline__ void store_vector(T* p, int C, int v, const float* f) {
  constexpr int V = Elem<T>::VEC;
  const int i = v * V;
  if (i + V <= C) {
    Vec16 x;
    Elem<T>::pack(f, x);
    store16_any(p + i, x);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (i + j < C) Elem<T>::store(p + i + j, f[j]);
  }
}
template <typename T, int EXPS>
__device__ __forceinline__ void gradient_of(const Vec16& x, const RowGrad& g, const Scales& sc, float* d) {
  constexpr int V = Elem<T>::VEC;
  float z[V];
  Elem<T>::unpack(x, z);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float u = z[j] - g.ref, y = __builtin_amdgcn_exp2f(u * sc.t);
    d[j] = fmaf(g.coef_t, y, -g.offset);
    if constexpr (EXPS == 2) d[j] = fmaf(g.coef_1, y * y, d[j]);
    if constexpr (EXPS == 4) {
      const float y2 = y * y;
      d[j] = fmaf(g.coef_1, y2 * y2, d[j]);
    }
    if constexpr (EXPS == 0) d[j] = fmaf(g.coef_1, __builtin_amdgcn_exp2f(u * sc.one), d[j]);
  }
}

// Reads a row's entries, those of classes that exist and appear for the first time: sh.at, sh.z.  Every thread of the workgroup calls it.
// (Which of two equal classes comes first is found by comparison with those in front, but only where the bits say that there are two.)
template <typename T, int NT>
__device__ __forceinline__ void read_entries(const DistillArgs& a, const T* row, int n, int k, int label, RowShared& sh) {
  const int tid = threadIdx.x;
  static_assert(NT >= 64, "waves");
  for (int j = tid; j < k; j += NT) {
    const int c = a.t_indices[static_cast<int64_t>(n) * a.k + j];
    sh.at[j] = c >= 0 && c < a.C ? c : -1;
  }
  if (tid == 0 && label >= 0) sh.z[kTopMax] = Elem<T>::load(row + label);
  __syncthreads();
}
template <typename T, int NT>
__device__ __forceinline__ void drop_repeated(const T* row, int k, bool repeated, RowShared& sh) {
  const int tid = threadIdx.x;
  if (__syncthreads_or(repeated)) {
    bool drop[(kTopMax + NT - 1) / NT];
#pragma unroll
    for (int i = 0; i < (kTopMax + NT - 1) / NT; ++i) {
      const int j = tid + NT * i, c = j < k ? sh.at[j] : -1;
      drop[i] = false;
      for (int h = 0; h < j && c >= 0; ++h) drop[i] |= sh.at[h] == c;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < (kTopMax + NT - 1) / NT; ++i)
      if (drop[i]) sh.at[tid + NT * i] = -1;
  }
  for (int j = tid; j < k; j += NT)  // (each thread its own entries)
    if (sh.at[j] >= 0) sh.z[j] = Elem<T>::load(row + sh.at[j]);
  __syncthreads();
}

// One workgroup per row, NT threads.
// U > 0: the row is U vectors a thread at most and stays in registers between the sums and the gradient: it is read once.  U = 0: it is
// read twice, in chunks of classes whose membership bits fit LDS.
template <typename T, int EXPS, int NT, int U>
__global__ __launch_bounds__(NT) void distill_rows_kernel(const DistillArgs a) {
  constexpr int V = Elem<T>::VEC;
  constexpr int CHUNK = U > 0 ? U * NT * V : 65536;  // classes whose membership bits are in LDS at a time
  __shared__ uint32_t member[CHUNK / 32];
  __shared__ RowShared sh;
  __shared__ RowSums red[NT / 64];
  const int tid = threadIdx.x;
  const Scales sc = scales_of(a, EXPS);
  const int k = a.alpha > 0.f ? a.k : 0;
  // (a grid of rows, not a loop over them: what the end of a row needs in constants would stay in registers through its sums)
  const int n = blockIdx.y * gridDim.x + blockIdx.x;
  if (n >= a.N) return;
  {
    const RowOf<T> row{static_cast<const T*>(a.logits) + n * a.ld, a.C};
    T* grad = a.grad ? static_cast<T*>(a.grad) + n * a.grad_ld : nullptr;
    const int vecs = (a.C + V - 1) / V;
    const float w = a.row_weight ? a.row_weight[n] : 1.f / static_cast<float>(a.N);
    if (w == 0.f) {
      float zero[V] = {};
      for (int v = tid; grad && v < vecs; v += NT) store_vector(grad, a.C, v, zero);
      if (tid == 0) a.row_loss[n] = 0.f;
      return;
    }
    int label = a.labels && a.alpha < 1.f ? a.labels[n] : -1;
    if (label >= a.C) label = -1;
    const bool want_sz = label >= 0 && a.smoothing > 0.f;
    Vec16 held[U > 0 ? U : 1];
    if constexpr (U > 0) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u * NT + tid < vecs) held[u] = row.load(u * NT + tid);
    }
    read_entries<T, NT>(a, row.p, n, k, label, sh);
    Sums<EXPS> sums;
    double sz = 0;  // (in double: beside classes masked with the lowest float it still holds what the others add)
    auto add = [&](const Vec16& x, int v, int first) __attribute__((always_inline)) {
      float z[V];
      Elem<T>::unpack(x, z);
      if (want_sz) {
#pragma unroll
        for (int j = 0; j < V; ++j) sz += v * V + j < a.C ? static_cast<double>(z[j]) : 0.0;
      }
      const int at = (v - first) * V;
      const uint32_t bits = member[at >> 5] >> (at & 31) & ((1u << V) - 1);
      if (bits) {
#pragma unroll
        for (int j = 0; j < V; ++j) z[j] = bits >> j & 1 ? -INFINITY : z[j];
      }
      sums.template add<V>(z, sc);
    };
    bool repeated = false;
    for (int c0 = 0; c0 < a.C; c0 += CHUNK) {
      const int chunk = min(a.C - c0, CHUNK);
      if (c0) __syncthreads();
      for (int i = tid; i < (chunk + 31) / 32; i += NT) member[i] = 0;
      __syncthreads();
      for (int j = tid; j < k; j += NT) {
        const int at = sh.at[j] - c0;
        if (sh.at[j] >= c0 && at < chunk) repeated |= atomicOr(&member[at >> 5], 1u << (at & 31)) >> (at & 31) & 1;
      }
      __syncthreads();
      if constexpr (U > 0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u * NT + tid < vecs) {
            add(held[u], u * NT + tid, 0);
            // the gradient unpacks them again: floats kept from here would be twice the registers
            asm volatile("" : "+v"(held[u].u.x), "+v"(held[u].u.y), "+v"(held[u].u.z), "+v"(held[u].u.w));
            __builtin_amdgcn_sched_barrier(0);
          }
      } else {
        const int first = c0 / V, last = (c0 + chunk + V - 1) / V;
        for (int v = first + tid; v < last; v += NT) add(row.load(v), v, first);
      }
    }
    drop_repeated<T, NT>(row.p, k, repeated, sh);
    const RowSums r = block_sums<EXPS, NT>(sums, sz, want_sz, sc, red);
    if (tid < 64) row_finish<EXPS>(a, sc, r, n, w, label, sh);
    __syncthreads();
    if (grad) {
      const RowGrad g = sh.g;
      float d[V];
      if constexpr (U > 0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u * NT + tid < vecs) {
            gradient_of<T, EXPS>(held[u], g, sc, d);
            store_vector(grad, a.C, u * NT + tid, d);
            __builtin_amdgcn_sched_barrier(0);
          }
      } else {
        for (int v = tid; v < vecs; v += NT) {
          gradient_of<T, EXPS>(row.load(v), g, sc, d);
          store_vector(grad, a.C, v, d);
        }
      }
      __syncthreads();
      // the entries' classes and the label's: written once more (behind the barrier: the same memory)
      for (int j = tid; j < k; j += NT)
        if (sh.at[j] >= 0) Elem<T>::store(grad + sh.at[j], sh.value[j]);
      if (tid == 0 && sh.at[kTopMax] >= 0) Elem<T>::store(grad + sh.at[kTopMax], sh.value[kTopMax]);
    }
  }
}

// loss = sum_n w_n row_loss_n, in double, in a fixed order.
__global__ __launch_bounds__(256) void distill_loss_kernel(const float* __restrict__ row_loss, const float* __restrict__ row_weight, int N,
                                                           float* __restrict__ loss) {
  __shared__ double red[256];
  double s = 0;
  for (int n = threadIdx.x; n < N; n += 256) {
    if (row_weight == nullptr) s += row_loss[n];
    else if (row_weight[n] != 0.f) s += static_cast<double>(row_weight[n]) * row_loss[n];
  }
  red[threadIdx.x] = s;
  __syncthreads();
  for (int step = 128; step > 0; step >>= 1) {
    if (threadIdx.x < step) red[threadIdx.x] += red[threadIdx.x + step];
    __syncthreads();
  }
  if (threadIdx.x == 0) loss[0] = static_cast<float>(row_weight ? red[0] : red[0] / N);
}

static int check_rows(const char* who, int N, int C, int dtype, const void* logits, int64_t ld) {
  RN50_REQUIRE(dtype == RN50_F32 || dtype == RN50_BF16, RN50_ERR_INVALID, "%s: dtype %d", who, dtype);
  RN50_REQUIRE(N > 0 && C > 0, RN50_ERR_INVALID, "%s: non-positive size", who);
  RN50_REQUIRE(C <= (1 << 30), RN50_ERR_UNSUPPORTED, "%s: C=%d", who, C);
  RN50_REQUIRE(logits, RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(ld >= C, RN50_ERR_INVALID, "%s: rows of %d elements %lld apart", who, C, static_cast<long long>(ld));
  RN50_REQUIRE(aligned_to(logits, dtype == RN50_BF16 ? 2 : 4), RN50_ERR_ALIGN, "%s: pointer not aligned to an element", who);
  return RN50_OK;
}
template <typename T, int EXPS>
static void distill_rows(const DistillArgs& a, dim3 grid, hipStream_t s) {
  constexpr int V = Elem<T>::VEC;
  const int64_t vecs = ceil_div(a.C, V);
  if (vecs <= 256) RN50_LAUNCH("distill", (distill_rows_kernel<T, EXPS, 256, 1>), grid, dim3(256), 0, s, a);
  else if (vecs <= 256 * 4) RN50_LAUNCH("distill", (distill_rows_kernel<T, EXPS, 256, 4>), grid, dim3(256), 0, s, a);
  else if (vecs <= 512 * 8) RN50_LAUNCH("distill", (distill_rows_kernel<T, EXPS, 512, 8>), grid, dim3(512), 0, s, a);
  else if (vecs <= 1024 * 8) RN50_LAUNCH("distill", (distill_rows_kernel<T, EXPS, 1024, 8>), grid, dim3(1024), 0, s, a);
  else if (vecs <= 1024 * 16) RN50_LAUNCH("distill", (distill_rows_kernel<T, EXPS, 1024, 16>), grid, dim3(1024), 0, s, a);
  else RN50_LAUNCH("distill", (distill_rows_kernel<T, EXPS, 256, 0>), grid, dim3(256), 0, s, a);
}
template <typename T>
static void distill_run(const DistillArgs& a, dim3 grid, hipStream_t s) {
  const bool both = a.alpha > 0.f && a.alpha < 1.f && a.labels;
  if (!both || a.temperature == 1.f) distill_rows<T, 1>(a, grid, s);
  else if (a.temperature == 2.f) distill_rows<T, 2>(a, grid, s);
  else if (a.temperature == 4.f) distill_rows<T, 4>(a, grid, s);
  else distill_rows<T, 0>(a, grid, s);
}
constexpr int kRowGrid = 1 << 20;  // workgroups of a launch over rows, at most: they take the rows in turn

}  // namespace rn50

using namespace rn50;

extern "C" size_t topk_rows_workspace_bytes(int N, int C, int k) {
  (void)N; (void)C; (void)k;
  return 0;
}

extern "C" int topk_rows(int N, int C, int k, int dtype, const void* logits, int64_t ld, float temperature, float* values, int32_t* indices,
                         float* tail_lse, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  if (int rc = check_rows("topk_rows", N, C, dtype, logits, ld)) return rc;
  RN50_REQUIRE(k >= 1 && k <= kTopMax, RN50_ERR_UNSUPPORTED, "topk_rows: k=%d outside [1, %d]", k, kTopMax);
  RN50_REQUIRE(temperature > 0.f && temperature <= FLT_MAX, RN50_ERR_INVALID, "topk_rows: temperature %g", temperature);
  RN50_REQUIRE(values && indices, RN50_ERR_INVALID, "topk_rows: null pointer");
  RN50_REQUIRE(aligned_to(values, 4) && aligned_to(indices, 4) && aligned_to(tail_lse, 4), RN50_ERR_ALIGN, "topk_rows: pointer not aligned to an element");
  RN50_REQUIRE(aligned16(workspace), RN50_ERR_ALIGN, "topk_rows: workspace not 16-byte aligned");
  const size_t need = topk_rows_workspace_bytes(N, C, k);
  RN50_REQUIRE(workspace_bytes >= need && (need == 0 || workspace), RN50_ERR_WORKSPACE, "topk_rows: workspace %zu < %zu bytes", workspace_bytes, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid(std::min(N, kRowGrid));
  if (dtype == RN50_BF16)
    RN50_LAUNCH("topk_rows", topk_rows_kernel<uint16_t>, grid, dim3(256), 0, s, static_cast<const uint16_t*>(logits), ld, N, C, k, temperature, values, indices, tail_lse);
  else
    RN50_LAUNCH("topk_rows", topk_rows_kernel<float>, grid, dim3(256), 0, s, static_cast<const float*>(logits), ld, N, C, k, temperature, values, indices, tail_lse);
  return launch_status("topk_rows");
}

extern "C" size_t distill_workspace_bytes(const rn50_distill_desc* d) {
  (void)d;
  return 0;
}

extern "C" int distill_fwd_bwd(const rn50_distill_desc* d, const void* logits, const float* t_values, const int32_t* t_indices, const float* t_tail,
                               const int32_t* labels, const float* row_weight, float* loss_out, float* row_loss_out, void* dlogits,
                               void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const char* who = "distill_fwd_bwd";
  RN50_REQUIRE(d, RN50_ERR_INVALID, "%s: null descriptor", who);
  if (int rc = check_rows(who, d->N, d->C, d->dtype, logits, d->ld)) return rc;
  RN50_REQUIRE(d->k >= 0 && d->k <= kTopMax, RN50_ERR_UNSUPPORTED, "%s: k=%d outside [0, %d]", who, d->k, kTopMax);
  RN50_REQUIRE(d->temperature > 0.f && d->temperature <= FLT_MAX, RN50_ERR_INVALID, "%s: temperature %g", who, d->temperature);
  RN50_REQUIRE(d->alpha >= 0.f && d->alpha <= 1.f, RN50_ERR_INVALID, "%s: alpha %g", who, d->alpha);
  RN50_REQUIRE(d->label_smoothing >= 0.f && d->label_smoothing <= 1.f, RN50_ERR_INVALID, "%s: label_smoothing %g", who, d->label_smoothing);
  RN50_REQUIRE(d->k == 0 || (t_values && t_indices), RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(loss_out && row_loss_out, RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(!dlogits || d->grad_ld >= d->C, RN50_ERR_INVALID, "%s: gradient rows of %d elements %lld apart", who, d->C,
               static_cast<long long>(d->grad_ld));
  RN50_REQUIRE(dlogits != logits || d->grad_ld == d->ld, RN50_ERR_INVALID, "%s: a gradient in the logits' place with rows of its own", who);
  RN50_REQUIRE(aligned_to(t_values, 4) && aligned_to(t_indices, 4) && aligned_to(t_tail, 4) && aligned_to(labels, 4) && aligned_to(row_weight, 4) &&
                   aligned_to(loss_out, 4) && aligned_to(row_loss_out, 4) && aligned_to(dlogits, d->dtype == RN50_BF16 ? 2 : 4),
               RN50_ERR_ALIGN, "%s: pointer not aligned to an element", who);
  RN50_REQUIRE(aligned16(workspace), RN50_ERR_ALIGN, "%s: workspace not 16-byte aligned", who);
  const size_t need = distill_workspace_bytes(d);
  RN50_REQUIRE(workspace_bytes >= need && (need == 0 || workspace), RN50_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, workspace_bytes, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  DistillArgs a{logits, dlogits, t_values, t_indices, t_tail, row_weight, labels, row_loss_out, d->ld, d->grad_ld, d->N, d->C, d->k,
                d->temperature, d->alpha, d->label_smoothing, d->grad_scale};
  const dim3 grid(std::min(d->N, kRowGrid));
  if (d->dtype == RN50_BF16) distill_run<uint16_t>(a, grid, s);
  else distill_run<float>(a, grid, s);
  RN50_LAUNCH("distill_loss", distill_loss_kernel, dim3(1), dim3(256), 0, s, row_loss_out, row_weight, d->N, loss_out);
  return launch_status(who);
}

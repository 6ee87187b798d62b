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

constexpr int kChunk = 65536;  // classes whose membership bits are in LDS at a time

// The row's numbers that the gradient pass needs.
struct RowGrad {
  float m;       // reference of the exponentials
  float coef_t;  // of exp((z - m) / T): alpha T w (q_r - p_r) / s
  float coef_1;  // of exp(z - m): (1 - alpha) w / S
  float offset;  // (1 - alpha) w ls / C
};

// One workgroup per row.
template <typename T>
__global__ __launch_bounds__(256) void distill_rows_kernel(const DistillArgs a) {
  __shared__ uint32_t member[kChunk / 32];
  __shared__ int at_s[kTopMax];
  __shared__ float z_s[kTopMax];
  __shared__ double v_s[kTopMax];
  __shared__ float red[4][4];
  __shared__ double red_z[4];
  __shared__ double shared_d[8];
  __shared__ RowGrad rg_s;
  __shared__ int state_s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float scale = kLog2e / a.temperature;
  const double beta = 1.0 / static_cast<double>(a.temperature);
  const bool kl_on = a.alpha > 0.f;
  for (int n = blockIdx.x; n < a.N; n += gridDim.x) {
    const T* row = static_cast<const T*>(a.logits) + n * a.ld;
    T* grad = a.grad ? static_cast<T*>(a.grad) + n * a.grad_ld : nullptr;
    const float w = a.row_weight ? a.row_weight[n] : 1.f / static_cast<float>(a.N);
    if (w == 0.f) {
      for (int i = tid; grad && i < a.C; i += 256) Elem<T>::store(grad + i, 0.f);
      if (tid == 0) a.row_loss[n] = 0.f;
      continue;
    }
    const int label = a.labels && a.alpha < 1.f ? a.labels[n] : -1;
    const bool ce_on = label >= 0 && label < a.C;
    // entries: absent ones have class -1
    const int k = kl_on ? a.k : 0;
    if (tid < k) at_s[tid] = a.t_indices[static_cast<int64_t>(n) * a.k + tid];
    __syncthreads();
    int at = -1;
    if (tid < k) {
      at = at_s[tid];
      if (at < 0 || at >= a.C) at = -1;
      for (int j = 0; j < tid && at >= 0; ++j)
        if (at_s[j] == at) at = -1;
    }
    __syncthreads();
    if (tid < k) {
      at_s[tid] = at;
      z_s[tid] = at >= 0 ? Elem<T>::load(row + at) : -INFINITY;
      v_s[tid] = at >= 0 ? a.t_values[static_cast<int64_t>(n) * a.k + tid] * beta : -INFINITY;
    }
    const float z_label = ce_on ? Elem<T>::load(row + label) : 0.f;
    // the classes that are no entry: maximum, sum at T, sum at 1, sum of the logits
    float m = -FLT_MAX, st = 0.f, s1 = 0.f;
    double sz = 0;  // (in double: of masked classes at the lowest float it still leaves what the others add)
    for (int c0 = 0; c0 < a.C; c0 += kChunk) {
      __syncthreads();
      for (int i = tid; i < kChunk / 32; i += 256) member[i] = 0;
      __syncthreads();
      if (tid < k && at >= c0 && at - c0 < kChunk) atomicOr(&member[(at - c0) >> 5], 1u << ((at - c0) & 31));
      __syncthreads();
      for (int i = c0 + tid; i < min(a.C, c0 + kChunk); i += 256) {
        const float z = Elem<T>::load(row + i);
        if (a.smoothing > 0.f) sz += z;
        if ((member[(i - c0) >> 5] >> ((i - c0) & 31)) & 1) continue;
        const float top = fmaxf(m, z);
        st = st * exp_scaled(m - top, scale) + exp_scaled(z - top, scale);
        s1 = s1 * exp_scaled(m - top, kLog2e) + exp_scaled(z - top, kLog2e);
        m = top;
      }
    }
    {
      const float wm = wave_max(m);
      const float wt = wave_sum(st * exp_scaled(m - wm, scale)), w1 = wave_sum(s1 * exp_scaled(m - wm, kLog2e));
      const double wz = wave_sum(sz);
      if (lane == 0) red[wave][0] = wm, red[wave][1] = wt, red[wave][2] = w1, red_z[wave] = wz;
    }
    __syncthreads();
    if (tid == 0) {  // (first form: one thread)
      float top = -FLT_MAX;
      for (int i = 0; i < 4; ++i) top = fmaxf(top, red[i][0]);
      double ST = 0, S1 = 0, SZ = 0;
      for (int i = 0; i < 4; ++i) {
        ST += red[i][1] * exp_scaled(red[i][0] - top, scale);
        S1 += red[i][2] * exp_scaled(red[i][0] - top, kLog2e);
        SZ += red_z[i];
      }
      const double rest = ST;
      float M = top;
      for (int j = 0; j < k; ++j) M = fmaxf(M, z_s[j]);
      double AT = rest * exp_scaled(top - M, scale), A1 = S1 * exp_scaled(top - M, kLog2e);
      for (int j = 0; j < k; ++j) {
        AT += exp_scaled(z_s[j] - M, scale);
        A1 += exp_scaled(z_s[j] - M, kLog2e);
      }
      const bool none = AT == 0;  // every logit is -infinity
      // relative to M and Mt, so that nothing is lost beside large ones: log sums of exponentials (log 0 = -infinity)
      const double Z = log(AT), Z1 = log(A1), lam = (static_cast<double>(top) - M) * beta + log(rest);
      const double tau = kl_on && a.t_tail ? static_cast<double>(a.t_tail[n]) : -INFINITY;
      double Mt = tau, kl = 0, pr = 0, L = 0;
      for (int j = 0; j < k; ++j) Mt = fmax(Mt, v_s[j]);
      const bool empty = Mt == -INFINITY;
      if (!empty) {
        double S = exp(tau - Mt);
        for (int j = 0; j < k; ++j) S += exp(v_s[j] - Mt);
        L = log(S);
        for (int j = 0; j < k; ++j) {
          const double p = exp(v_s[j] - Mt - L);
          if (p != 0) kl += p * ((v_s[j] - Mt - L) - ((static_cast<double>(z_s[j]) - M) * beta - Z));
        }
        pr = exp(tau - Mt - L);
        if (pr != 0) kl += pr * ((tau - Mt - L) - (lam - Z));
      }
      double loss = 0;
      if (!none) {
        if (!empty) loss += static_cast<double>(a.alpha) * a.temperature * a.temperature * kl;
        if (ce_on) {
          double ce = -(1.0 - a.smoothing) * (static_cast<double>(z_label) - M - Z1);
          if (a.smoothing > 0.f) ce -= static_cast<double>(a.smoothing) / a.C * ((SZ - static_cast<double>(a.C) * M) - a.C * Z1);
          loss += (1.0 - a.alpha) * ce;
        }
      }
      a.row_loss[n] = static_cast<float>(loss);
      const double g = none ? 0.0 : static_cast<double>(a.grad_scale) * w;
      const double gt = empty ? 0.0 : g * a.alpha * a.temperature, g1 = ce_on ? g * (1.0 - a.alpha) : 0.0;
      RowGrad r;
      r.m = top;
      r.coef_t = rest == 0 || gt == 0 ? 0.f : static_cast<float>(gt * (exp(lam - Z) - pr) / rest);
      r.coef_1 = g1 == 0 ? 0.f : static_cast<float>(g1 * exp_scaled(top - M, kLog2e) / A1);
      r.offset = static_cast<float>(g1 * a.smoothing / a.C);
      rg_s = r;
      state_s = none;
      shared_d[0] = Z; shared_d[1] = L; shared_d[2] = gt; shared_d[3] = g1; shared_d[4] = Z1; shared_d[5] = M; shared_d[6] = Mt;
    }
    __syncthreads();
    if (grad) {
      const RowGrad r = rg_s;
      const double Z = shared_d[0], L = shared_d[1], gt = shared_d[2], g1 = shared_d[3], Z1 = shared_d[4], M = shared_d[5], Mt = shared_d[6];
      const bool none = state_s;
      for (int i = tid; i < a.C; i += 256) {
        const float z = Elem<T>::load(row + i);
        float d = none ? 0.f : -r.offset;
        if (r.coef_t != 0.f) d += r.coef_t * exp_scaled(z - r.m, scale);
        if (r.coef_1 != 0.f) d += r.coef_1 * exp_scaled(z - r.m, kLog2e);
        Elem<T>::store(grad + i, d);
      }
      __syncthreads();
      // the entries' classes and the label's: written once more, whole
      if (!none) {
        const double off = g1 * a.smoothing / a.C;
        bool label_is_entry = false;
        for (int j = 0; j < k; ++j) label_is_entry |= at_s[j] == label;
        if (tid < k && at >= 0) {
          double d = -off;
          if (gt != 0) d += gt * (exp((z_s[tid] - M) * beta - Z) - exp(v_s[tid] - Mt - L));
          if (g1 != 0) d += g1 * exp(z_s[tid] - M - Z1);
          if (at == label) d -= g1 * (1.0 - a.smoothing);
          Elem<T>::store(grad + at, static_cast<float>(d));
        }
        if (tid == 0 && ce_on && !label_is_entry) {
          float d = -r.offset + r.coef_t * exp_scaled(z_label - r.m, scale) + r.coef_1 * exp_scaled(z_label - r.m, kLog2e);
          d -= static_cast<float>(g1 * (1.0 - a.smoothing));
          Elem<T>::store(grad + label, d);
        }
      }
    }
    __syncthreads();
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
  if (d->dtype == RN50_BF16) RN50_LAUNCH("distill", distill_rows_kernel<uint16_t>, grid, dim3(256), 0, s, a);
  else RN50_LAUNCH("distill", distill_rows_kernel<float>, grid, dim3(256), 0, s, a);
  RN50_LAUNCH("distill_loss", distill_loss_kernel, dim3(1), dim3(256), 0, s, row_loss_out, row_weight, d->N, loss_out);
  return launch_status(who);
}

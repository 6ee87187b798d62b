// Distillation from a teacher's largest logits: their selection (topk_rows) and the loss and gradient of student logits against
// them (distill_fwd_bwd).
//
// Sums of exponentials run with their maximum: (m, s) stands for s * exp(m / T).  m starts at the lowest finite float, so that
// nothing is ever subtracted from an infinity of its own sign: a logit of -infinity adds exp(-infinity) = 0, a row of nothing else
// leaves s = 0, a NaN makes s NaN.  A logit of +infinity does so too, except among the classes that topk_rows did not take (Sums::infinite).
#include <float.h>
#include <stdlib.h>

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
// Sum and maximum of a wave's floats, the same in every lane: four exchanges inside rows of 16 lanes (moves between lanes in the ALU; through
// LDS, as wave_sum has them, each is some hundred cycles that a row's end waits for), then the four rows' values from scalar registers.
template <int CTRL>
__device__ __forceinline__ float lane_move(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float from_lane(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }
__device__ __forceinline__ float quick_sum(float x) {
  x += lane_move<0xB1>(x);   // lanes 1 apart
  x += lane_move<0x4E>(x);   // 2 apart
  x += lane_move<0x141>(x);  // the other half of 8, mirrored
  x += lane_move<0x140>(x);  // the other half of 16, mirrored
  return (from_lane(x, 0) + from_lane(x, 16)) + (from_lane(x, 32) + from_lane(x, 48));
}
__device__ __forceinline__ float quick_max(float x) {
  x = fmaxf(x, lane_move<0xB1>(x));
  x = fmaxf(x, lane_move<0x4E>(x));
  x = fmaxf(x, lane_move<0x141>(x));
  x = fmaxf(x, lane_move<0x140>(x));
  return fmaxf(fmaxf(from_lane(x, 0), from_lane(x, 16)), fmaxf(from_lane(x, 32), from_lane(x, 48)));
}

// Rows start at any element; their vectors start where 16 bytes do (vectors across that boundary took 228 us for loss and gradient of
// 4096 x 50001 bf16, 98 for its largest logits; 50000 classes 184 and 89).  A row's classes count from the first vector on: place 0 is class
// `head`, and the `head` classes in front of it follow the last class.
struct Places {
  int head, classes;
  template <typename T>
  __device__ __forceinline__ Places(const T* row, int C)
      : head(min(C, static_cast<int>((0u - static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row))) % 16u / sizeof(T)))), classes(C) {}
  __device__ __forceinline__ int class_at(int place) const { return place + head < classes ? place + head : place + head - classes; }
  __device__ __forceinline__ int of(int c) const { return c >= head ? c - head : c + classes - head; }  // (0 <= c < classes)
};

// A workgroup for each of N rows, row blockIdx.y * gridDim.x + blockIdx.x.
static dim3 row_grid(int N) { return N <= 65536 ? dim3(N) : dim3(65536, static_cast<unsigned>(ceil_div(N, 65536))); }

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
// multiplication or two in place of an exponential's four issue slots); 0: both.  T = 2 -> 3, bf16: the loss of 4096 x 50001 93 -> 100 us, loss
// and gradient of 8192 x 8192 69.5 -> 75.5; of longer and of short rows the same.
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
  __device__ __forceinline__ void move(float to, const Scales& sc) {
    const float f = __builtin_amdgcn_exp2f((ref - to) * sc.t);
    st *= f;
    if constexpr (EXPS == 0) s1 *= __builtin_amdgcn_exp2f((ref - to) * sc.one);
    if constexpr (EXPS == 2) s1 *= f * f;
    if constexpr (EXPS == 4) s1 *= (f * f) * (f * f);
    ref = to;
    lim = to + sc.slack;
  }
  __device__ __forceinline__ void join(Sums other, const Scales& sc) {
    const float to = fmaxf(ref, other.ref);
    move(to, sc);
    other.move(to, sc);
    st += other.st;
    s1 += other.s1;
  }
  // A logit of +infinity makes the sum infinite and leaves the reference finite: nothing is subtracted from an infinity, here or where sums
  // are joined (this one's reference is the largest there), and a NaN stays.
  __device__ __forceinline__ void infinite(const Scales& sc) {
    move(FLT_MAX, sc);
    st += INFINITY;
  }
  template <int V>
  __device__ __forceinline__ void add(const float* x, const Scales& sc) {
    float top = x[0];
#pragma unroll
    for (int j = 1; j < V; ++j) top = fmaxf(top, x[j]);
    if (__any(top > lim)) {  // (one branch for the wave: without it the move is computed for every vector and selected)
      if (top > lim) move(top, sc);
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
// The sums of `n` parts, in their order.
__device__ __forceinline__ RowSums joined(const RowSums* part, int n, const Scales& sc) {
  RowSums t = part[0];
  for (int w = 1; w < n; ++w) t.ref = fmaxf(t.ref, part[w].ref);
  t.st = t.s1 = 0.f;
  t.sz = 0.0;
  for (int w = 0; w < n; ++w) {
    const float d = part[w].ref - t.ref;
    t.st += part[w].st * __builtin_amdgcn_exp2f(d * sc.t);
    t.s1 += part[w].s1 * __builtin_amdgcn_exp2f(d * sc.one);
    t.sz += part[w].sz;
  }
  return t;
}
// Sums of a workgroup's threads, in a fixed order; complete in every thread.  `red`: a RowSums for each wave.
template <int EXPS, int NT>
__device__ __forceinline__ RowSums block_sums(const Sums<EXPS>& a, double sz, bool want_sz, const Scales& sc, RowSums* red) {
  const int wave = threadIdx.x >> 6;
  RowSums r;
  r.ref = quick_max(a.ref);
  const float f = __builtin_amdgcn_exp2f((a.ref - r.ref) * sc.t);
  r.st = quick_sum(a.st * f);
  if constexpr (EXPS == 1) r.s1 = r.st;
  if constexpr (EXPS == 2) r.s1 = quick_sum(a.s1 * (f * f));
  if constexpr (EXPS == 4) r.s1 = quick_sum(a.s1 * ((f * f) * (f * f)));
  if constexpr (EXPS == 0) r.s1 = quick_sum(a.s1 * __builtin_amdgcn_exp2f((a.ref - r.ref) * sc.one));
  r.sz = want_sz ? wave_sum(sz) : 0.0;
  if constexpr (NT == 64) return r;
  if ((threadIdx.x & 63) == 0) red[wave] = r;
  __syncthreads();
  return joined(red, NT / 64, sc);
}

// ------------------------------------------------------------- largest logits
// The order of the logits as unsigned integers: -0 and +0 are one, a NaN is above everything (and below the last integer).
__device__ __forceinline__ uint32_t order_key(float x) {
  uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xfffffffeu;
  if (u == 0x80000000u) u = 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// The least logit whose key reaches `key` (no NaN's).
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
constexpr uint32_t kKeyOfNothing = 0x007fffffu;   // order_key(-infinity)
constexpr uint32_t kKeyOfInfinity = 0xff800000u;  // order_key(+infinity)

struct TopkArgs {
  const void* logits;
  int64_t ld;
  int N, C, k;
  float temperature;
  float* values;
  int32_t* indices;
  float* tail;  // (or null)
  // slices of rows: each one's largest logits, their classes, and the sum of its others
  int slices, width;
  float* part_values;
  int32_t* part_at;
  RowSums* part_sums;
};
enum { kTopkRows, kTopkSlices, kTopkJoin };  // whole rows; slices of rows; the slices' largest logits
constexpr int kTopkThreads = 256, kTopkCand = 768, kTopkStreams = 4, kTopkOwners = 512;  // threads of a row, candidates, streams of a thread, those read again (find_bound: 400)

struct TopkShared {
  __align__(16) unsigned long long cand[kTopkCand];  // (key, ~class) of the logits that may be among the largest: larger is in front
  float value[kTopkCand], spare[kTopkCand];
  int owner[kTopkOwners];
  __align__(16) int count[2][4 * 16];
  int taken;
  int last;
  uint32_t hist[256], found[2];
  int first[256];             // candidates of every bin of keys, as lists
  int16_t next[kTopkCand];
  RowSums red[kTopkThreads / 64];
};

// Where a row's results go.
template <int MODE>
struct TopkOut {
  const TopkArgs& a;
  int n, slice;
  __device__ __forceinline__ void put(int rank, float x, int at) const {
    if (MODE == kTopkSlices) {
      const int64_t i = (static_cast<int64_t>(n) * a.slices + slice) * a.k + rank;
      a.part_values[i] = x;
      a.part_at[i] = at < 0 ? at : at + slice * a.width;
    } else {
      const int64_t i = static_cast<int64_t>(n) * a.k + rank;
      a.values[i] = x;
      a.indices[i] = MODE == kTopkJoin ? a.part_at[static_cast<int64_t>(n) * a.slices * a.k + at] : at;
    }
  }
  __device__ __forceinline__ float value(int rank) const {
    return MODE == kTopkSlices ? a.part_values[(static_cast<int64_t>(n) * a.slices + slice) * a.k + rank] : a.values[static_cast<int64_t>(n) * a.k + rank];
  }
  __device__ __forceinline__ int at(int rank) const {
    return MODE == kTopkSlices ? a.part_at[(static_cast<int64_t>(n) * a.slices + slice) * a.k + rank] - slice * a.width
                               : a.indices[static_cast<int64_t>(n) * a.k + rank];
  }
};

// Of 256 bins, one a thread, with `mine` in this thread's: how many are in this and all higher ones.  Behind it the waves are past a barrier.
__device__ __forceinline__ int sum_from_here(int mine, TopkShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int from = __shfl_down(sum, off, 64);
    sum += lane + off < 64 ? from : 0;
  }
  if (lane == 0) sh.count[0][wave] = sum;
  __syncthreads();
  for (int w = wave + 1; w < 4; ++w) sum += sh.count[0][w];
  return sum;
}
// Bins of keys, 256 from lo to top.  Keys go by exponents: between a logit below zero and one above lie more than a hundred powers of two in
// which no logit is, and bins of equal width would put all logits into a few.  So magnitudes below 2^-8 of the larger end's count as one
// there: of(.) leaves the order as it is, and a key reaches at(b) where its bin is b or a higher one.  (An end beyond 2^64 is a mask or no
// number: the other end decides.)  4096 x 4000 bf16, 64 entries on
// both sides of zero, 99 -> 39 us.
struct KeyBins {
  int flat, first, last, shift;
  uint32_t end;
  __device__ __forceinline__ KeyBins(uint32_t lo, uint32_t top) : end(top + 1u) {
    const int a = static_cast<int>(lo ^ 0x80000000u), b = static_cast<int>(top ^ 0x80000000u);
    const int below = ~a > 0x5f800000 ? 0 : ~a, above = b > 0x5f800000 ? 0 : b;
    flat = a < 0 && b > 0 ? max(0, max(below, above) - (8 << 23)) : 0;
    first = fold(a);
    last = fold(b);
    shift = max(0, 24 - __clz(static_cast<int>(static_cast<uint32_t>(last) - static_cast<uint32_t>(first))));
  }
  __device__ __forceinline__ int fold(int x) const { return x - min(max(x, -flat), flat); }
  __device__ __forceinline__ uint32_t of(uint32_t key) const {
    return (static_cast<uint32_t>(fold(static_cast<int>(key ^ 0x80000000u))) - static_cast<uint32_t>(first)) >> shift;
  }
  __device__ __forceinline__ uint32_t at(uint32_t bin) const {  // (bin 256: behind the last key)
    const uint32_t step = bin << shift;
    if (step > static_cast<uint32_t>(last) - static_cast<uint32_t>(first) || bin > 255) return end;
    return unfold(static_cast<int>(static_cast<uint32_t>(first) + step));
  }
  __device__ __forceinline__ uint32_t unfold(int x) const { return static_cast<uint32_t>(x > 0 ? x + flat : x - flat) ^ 0x80000000u; }
};
// A key that at least kk of the workgroup's keys reach, hardly more if possible; where that takes a key that many have (`tie`), fewer than
// kk reach the one after it.  At least kk keys reach lo, none passes top.  The keys' bins (256 from lo to top) mostly hold few enough
// where the kk-th lies; otherwise its bin is halved until they do.  Every thread calls it, behind a barrier, with `hist` zero, as it
// leaves it.
template <int G>
__device__ __forceinline__ uint32_t find_bound(const uint32_t* key, uint32_t lo, uint32_t top, int kk, bool* tie, TopkShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int enough = kk + kk / 2 + 16;
  const KeyBins bins(lo, top);
#pragma unroll
  for (int g = 0; g < G; ++g)
    if (key[g] >= lo) atomicAdd(&sh.hist[bins.of(key[g])], 1u);
  __syncthreads();
  const int mine = static_cast<int>(sh.hist[tid]);
  sh.hist[tid] = 0;
  const int from_here = sum_from_here(mine, sh);
  if (from_here >= kk && from_here - mine < kk) {
    sh.found[0] = tid;
    sh.found[1] = from_here;
  }
  __syncthreads();
  int reach = static_cast<int>(sh.found[1]);
  lo = max(lo, bins.at(sh.found[0]));
  *tie = false;
  if (reach <= enough) return lo;
  uint32_t hi = bins.at(sh.found[0] + 1);
  for (int turn = 0; hi - lo > 1 && reach > enough; turn ^= 1) {
    const uint32_t mid = lo + ((hi - lo) >> 1);
    int c = 0;
#pragma unroll
    for (int g = 0; g < G; ++g) c += __popcll(__ballot(key[g] >= mid));
    if (lane == 0) sh.count[turn][8 + wave] = c;
    __syncthreads();
    c = (sh.count[turn][8] + sh.count[turn][9]) + (sh.count[turn][10] + sh.count[turn][11]);
    if (c >= kk) lo = mid, reach = c;
    else hi = mid;
  }
  *tie = reach > enough;
  return lo;
}
// Candidates in order: the first kk to the output, the others' values to `spare`.  Their keys, lo to hi, fall into 256 bins; a candidate comes
// behind those of higher bins, and behind the larger ones of its own, which it looks through.  (Looking through all of them took 4 us
// for 147 candidates, 13 for 365.)  Every thread calls it, behind a barrier; `hist` is zero and `first` -1 then.
static_assert(kTopkThreads == 256, "a bin a thread");
template <int MODE>
__device__ __forceinline__ void put_ranked(int cands, int kk, uint32_t lo, uint32_t hi, const TopkOut<MODE>& out, TopkShared& sh) {
  const int tid = threadIdx.x;
  const KeyBins bins(lo, hi);
  for (int c = tid; c < cands; c += kTopkThreads) {
    const uint32_t bin = bins.of(static_cast<uint32_t>(sh.cand[c] >> 32));
    atomicAdd(&sh.hist[bin], 1u);
    sh.next[c] = static_cast<int16_t>(atomicExch(&sh.first[bin], c));
  }
  __syncthreads();
  // of every bin, how many are in higher ones
  const int mine = static_cast<int>(sh.hist[tid]), sum = sum_from_here(mine, sh);
  sh.hist[tid] = static_cast<uint32_t>(sum - mine);
  __syncthreads();
  for (int c = tid; c < cands; c += kTopkThreads) {
    const unsigned long long me = sh.cand[c];
    const uint32_t bin = bins.of(static_cast<uint32_t>(me >> 32));
    int rank = static_cast<int>(sh.hist[bin]);
    for (int j = sh.first[bin]; j >= 0; j = sh.next[j]) rank += sh.cand[j] > me;
    if (rank < kk) out.put(rank, sh.value[c], static_cast<int>(~static_cast<uint32_t>(me)));
    else sh.spare[rank - kk] = sh.value[c];
  }
  __syncthreads();
}

// The `need` first classes whose key is `key`, in their order, to the ranks from `rank` on; returns the last of them.  Every thread calls it.
template <typename T, int MODE>
__device__ __forceinline__ int take_equal(const T* row, int C, uint32_t key, int need, int rank, const TopkOut<MODE>& out, TopkShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int before = 0;
#pragma unroll 1
  for (int base = 0; base < C && before < need; base += kTopkThreads) {
    const int i = base + tid;
    const float x = i < C ? Elem<T>::load(row + i) : 0.f;
    const bool eq = i < C && order_key(x) == key;
    const uint64_t votes = __ballot(eq);
    __syncthreads();
    if (lane == 0) sh.count[0][wave] = __popcll(votes);
    __syncthreads();
    int pos = before + __popcll(votes & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) pos += sh.count[0][w];
    if (eq && pos < need) {
      out.put(rank + pos, x, i);
      if (pos == need - 1) sh.last = i;
    }
    before += sh.count[0][0] + sh.count[0][1] + sh.count[0][2] + sh.count[0][3];
  }
  __syncthreads();
  return sh.last;
}
// The sum over the classes that were not taken: keys below `key`, and equal to it behind class `last`.  INF: +infinity may be among them,
// of which there are more than places then (looked for everywhere it costs rows of equal logits 4 %).
template <bool INF, typename T>
__device__ __forceinline__ void add_rest(const T* row, int C, uint32_t key, int last, const Scales& sc, Sums<1>& rest) {
#pragma unroll 1
  for (int i = threadIdx.x; i < C; i += kTopkThreads) {
    const float x = Elem<T>::load(row + i);
    const uint32_t o = order_key(x);
    if (o < key || (o == key && i > last)) {
      if (INF && x == INFINITY) rest.infinite(sc);
      else rest.template add<1>(&x, sc);
    }
  }
}

__device__ __forceinline__ float tail_of(const RowSums& sum, float temperature) {
  return sum.st == 0.f ? -INFINITY : static_cast<float>(static_cast<double>(sum.ref) / temperature + log(static_cast<double>(sum.st)));
}

// Any row, NaN and infinities among it: the key of the k-th largest logit digit by digit (four of 8 bits, a histogram each over the logits
// that share the digits in front).  The row is read seven times; only rows that the way below cannot take come here.
template <typename T, int MODE>
__device__ __forceinline__ void topk_any(const T* row, int C, int kk, const Scales& sc, const TopkOut<MODE>& out, TopkShared& sh, Sums<1>& rest) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0;
  int need = kk;  // how many are still to be taken among the logits that share the prefix
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    sh.hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < C; i += kTopkThreads) {
      const uint32_t key = order_key(Elem<T>::load(row + i));
      if (shift == 24 || key >> (shift + 8) == prefix) atomicAdd(&sh.hist[(key >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      int above = 0, d = 255;
      while (d > 0 && above + static_cast<int>(sh.hist[d]) < need) above += sh.hist[d--];
      sh.found[0] = d;
      sh.found[1] = above;
    }
    __syncthreads();
    prefix = prefix << 8 | sh.found[0];
    need -= sh.found[1];
  }
  __syncthreads();
  if (tid == 0) sh.taken = 0;
  __syncthreads();
  for (int i = tid; i < C; i += kTopkThreads) {  // (kk - need of them)
    const float x = Elem<T>::load(row + i);
    const uint32_t key = order_key(x);
    if (key > prefix) {
      const int at = atomicAdd(&sh.taken, 1);
      sh.cand[at] = static_cast<unsigned long long>(key) << 32 | ~static_cast<uint32_t>(i);
      sh.value[at] = x;
    }
  }
  __syncthreads();
  const int above = kk - need;
  if (tid < above) {
    const unsigned long long mine = sh.cand[tid];
    int rank = 0;
    for (int j = 0; j < above; ++j) rank += sh.cand[j] > mine;
    out.put(rank, sh.value[tid], static_cast<int>(~static_cast<uint32_t>(mine)));
  }
  const int last = take_equal<T, MODE>(row, C, prefix, need, above, out, sh);
  rest = Sums<1>();
  if (prefix >= kKeyOfInfinity) add_rest<true>(row, C, prefix, last, sc, rest);
  else add_rest<false>(row, C, prefix, last, sc, rest);
}

// One workgroup per row (or slice of one).  The row goes by once in 1024 streams of vectors, four a thread, each with its two largest
// vector maxima, the sum of exponentials of the vector that has the largest, and that of the others.  A bound below which no logit of the
// row's k largest can lie is the k-th largest of the streams' maxima, or a little less: of streams whose maximum reaches it (little
// more than k) that vector is read again, of the few whose second does all vectors, for the logits that reach it (little more than k
// again), and these are put in order by counting.  The sums of what is read again are taken anew without them: nothing is subtracted.
// 4096 x 50001 bf16, 100 entries 88 us, 4.7 TB/s; bound by instructions: 39.7 million of a wave's, 3.2 million of them exponentials of four
// issue slots, keep the vector ALUs busy in nine of ten cycles.  (With whole streams read again, 2048 x 131072 float, 16 vectors a stream, 256 us.)
// Where many maxima are equal (masks, ties), the logits above their value are the candidates and the rest of the k is taken from the
// equal ones in the order of the classes.
template <typename T, int MODE>
__global__ __launch_bounds__(kTopkThreads, 8) void topk_rows_kernel(const TopkArgs a) {
  constexpr int V = Elem<T>::VEC, NT = kTopkThreads, G = kTopkStreams;
  __shared__ TopkShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int slice = MODE == kTopkSlices ? blockIdx.x : 0, n = MODE == kTopkSlices ? blockIdx.y : blockIdx.y * gridDim.x + blockIdx.x;
  if (n >= a.N) return;
  const int C = MODE == kTopkSlices ? min(a.width, a.C - slice * a.width) : a.C;
  const T* row = static_cast<const T*>(a.logits) + n * a.ld + static_cast<int64_t>(slice) * a.width;
  const Places places(row, C);
  const T* vecs = row + places.head;
  const int kk = min(a.k, C), whole = (C - places.head) / V, left = C - whole * V;
  const TopkOut<MODE> out{a, n, slice};
  Scales sc;
  sc.t = sc.one = kLog2e / a.temperature;
  sc.slack = 20.f / sc.t;
  float m[G], second[G], best[G], st[G], ref = -FLT_MAX, lim = -FLT_MAX;  // (one reference for a thread's streams, as in Sums)
  int round[G];                                                           // where a stream's largest is
#pragma unroll
  for (int g = 0; g < G; ++g) m[g] = second[g] = -INFINITY, best[g] = st[g] = 0.f, round[g] = 0;
  auto take = [&](const Vec16& x, int g, int r) __attribute__((always_inline)) {
    float z[V];
    Elem<T>::unpack(x, z);
    float top = z[0];
#pragma unroll
    for (int j = 1; j < V; ++j) top = fmaxf(top, z[j]);
    if (__any(top > lim)) {
      if (top > lim) {
        const float f = __builtin_amdgcn_exp2f((ref - top) * sc.t);
#pragma unroll
        for (int i = 0; i < G; ++i) st[i] *= f, best[i] *= f;
        ref = top;
        lim = top + sc.slack;
      }
    }
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) sum += __builtin_amdgcn_exp2f((z[j] - ref) * sc.t);
    const bool up = top > m[g];
    st[g] += up ? best[g] : sum;
    best[g] = up ? sum : best[g];
    second[g] = up ? m[g] : fmaxf(second[g], top);
    m[g] = up ? top : m[g];
    round[g] = up ? r : round[g];
  };
  int v = tid, r = 0;
  for (; v + (G - 1) * NT < whole; v += G * NT, ++r) {
    Vec16 x[G];
#pragma unroll
    for (int g = 0; g < G; ++g) x[g] = load16(vecs + (v + g * NT) * V);
#pragma unroll
    for (int g = 0; g < G; ++g) take(x[g], g, r);
  }
  {
    Vec16 x[G];
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (v + g * NT < whole) x[g] = load16(vecs + (v + g * NT) * V);
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (v + g * NT < whole) take(x[g], g, r);
  }
  const int c_left = places.class_at(whole * V + tid);
  const float z_left = tid < left ? Elem<T>::load(row + c_left) : -INFINITY;  // (the classes of no vector)
  if (tid == 0) sh.taken = 0;
  sh.hist[tid] = 0;
  sh.first[tid] = -1;
  uint32_t key[G];
  float all = 0.f, tm = m[0];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    key[g] = order_key(m[g]);
    all += st[g] + best[g];
    tm = fmaxf(tm, m[g]);
  }
  {
    const float most = quick_max(tm), least = -quick_max(tid < kk ? -tm : -INFINITY);
    // (a sum is NaN where a logit is NaN or +infinity: maxima say nothing then)
    const uint64_t odd = __ballot(!(all == all) || !(z_left <= FLT_MAX));
    if (lane == 0) sh.count[1][wave] = __float_as_int(most), sh.count[1][4 + wave] = __float_as_int(least), sh.count[1][12 + wave] = odd != 0;
  }
  __syncthreads();
  const bool odd = (sh.count[1][12] | sh.count[1][13]) | (sh.count[1][14] | sh.count[1][15]);
  Sums<1> rest;
  if (!odd) {
    float most = -INFINITY, least = INFINITY;
    for (int w = 0; w < 4; ++w) {
      most = fmaxf(most, __int_as_float(sh.count[1][w]));
      least = fminf(least, __int_as_float(sh.count[1][4 + w]));
    }
    bool tie;
    uint32_t lo = find_bound<G>(key, order_key(least), order_key(most), kk, &tie, sh);  // (the first kk threads' maxima reach `least`)
    uint32_t bound = tie ? lo + 1 : lo;
    float from = logit_of(bound);
    // what is read again, listed in a fixed order: single vectors from the front, streams from the end; the sums of everything else stay
    rest.ref = ref;
    rest.lim = lim;
    uint64_t one[G], more[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      one[g] = __ballot(m[g] >= from && second[g] < from);
      more[g] = __ballot(m[g] >= from && second[g] >= from);
      if (lane == 0) sh.count[0][16 + g * 4 + wave] = __popcll(one[g]) | __popcll(more[g]) << 16;
    }
    __syncthreads();
    int counts = 0;  // (single vectors, streams)
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int4 c = *reinterpret_cast<const int4*>(&sh.count[0][16 + g * 4]);
      const int at = counts + (wave > 0 ? c.x : 0) + (wave > 1 ? c.y : 0) + (wave > 2 ? c.z : 0);
      counts += (c.x + c.y) + (c.z + c.w);
      const uint64_t below = (1ull << lane) - 1;
      if (m[g] >= from) {
        const bool single = second[g] < from;
        if (single) sh.owner[(at & 0xffff) + __popcll(one[g] & below)] = tid + (round[g] * G + g) * NT;
        else sh.owner[kTopkOwners - 1 - (at >> 16) - __popcll(more[g] & below)] = tid + g * NT;
        rest.st += single ? st[g] : 0.f;
      } else {
        rest.st += st[g] + best[g];
      }
    }
    const int singles = counts & 0xffff, streams = counts >> 16;
    sh.spare[tid] = rest.st;  // (a second look starts from it)
    auto candidate = [&](float x, int i) __attribute__((always_inline)) {
      const int at = atomicAdd(&sh.taken, 1);
      if (at < kTopkCand) {
        sh.cand[at] = static_cast<unsigned long long>(order_key(x)) << 32 | ~static_cast<uint32_t>(i);
        sh.value[at] = x;
      }
    };
    __syncthreads();
    // (vector of item i: a listed one, or one of a listed stream's)
    const int rounds = max(1, (whole + G * NT - 1) / (G * NT)), items = singles + streams * rounds;
    auto vector_of = [&](int i) __attribute__((always_inline)) {
      if (i < singles) return sh.owner[i];
      if (i >= items) return whole;
      const int o = (i - singles) / rounds;
      return sh.owner[kTopkOwners - 1 - o] + (i - singles - o * rounds) * (G * NT);
    };
    // (the candidates' largest key: of the streams' or of the classes of no vector)
    uint32_t top = order_key(most);
    for (int i = 0; i < left; ++i) top = max(top, order_key(Elem<T>::load(row + places.class_at(whole * V + i))));
    int cands;
#pragma unroll 1
    for (;;) {
      if (tid < left) {
        if (z_left >= from) candidate(z_left, c_left);
        else rest.template add<1>(&z_left, sc);
      }
      constexpr int AHEAD = 2;  // vectors whose loads go out together
      for (int i0 = tid; i0 < items; i0 += AHEAD * NT) {
        Vec16 x[AHEAD];
        int vec[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          vec[u] = vector_of(i0 + u * NT);
          if (vec[u] < whole) x[u] = load16(vecs + vec[u] * V);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          if (vec[u] >= whole) continue;
          float z[V];
          Elem<T>::unpack(x[u], z);
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (z[j] >= from) {
              candidate(z[j], places.head + vec[u] * V + j);
              z[j] = -INFINITY;
            }
          rest.template add<V>(z, sc);
        }
      }
      __syncthreads();
      cands = sh.taken;
      if (cands <= kTopkCand) break;
      // Too many: large logits lie side by side (rows in the order of their classes' frequency).  A higher bound from bins of what is read
      // again, the k-th largest's bin in bins of its own while it has too many: 4096 x 50001 bf16 in descending order 99 us (digit by digit,
      // as topk_any does, 1490).
      uint32_t hi = top;
      int above = 0;
      lo = bound;
#pragma unroll 1
      for (;;) {
        const int shift = max(0, 24 - __clz(static_cast<int>(hi - lo)));
        auto count = [&](float x) __attribute__((always_inline)) {
          const uint32_t at = order_key(x);
          if (at >= lo && at <= hi) atomicAdd(&sh.hist[(at - lo) >> shift], 1u);
        };
        if (tid < left) count(z_left);
#pragma unroll 1
        for (int i = tid; i < items; i += NT) {
          const int vec = vector_of(i);
          if (vec >= whole) continue;
          float z[V];
          Elem<T>::unpack(load16(vecs + vec * V), z);
#pragma unroll
          for (int j = 0; j < V; ++j) count(z[j]);
        }
        __syncthreads();
        const int here = static_cast<int>(sh.hist[tid]), sum = above + sum_from_here(here, sh);
        if (sum >= kk && sum - here < kk) {
          sh.found[0] = tid;
          sh.found[1] = sum;
          sh.last = here;
        }
        sh.hist[tid] = 0;
        if (tid == 0) sh.taken = 0;
        __syncthreads();
        const int reach = static_cast<int>(sh.found[1]);
        lo += sh.found[0] << shift;
        tie = shift == 0 && reach > kTopkCand;
        if (tie || reach <= kTopkCand) break;
        hi = min(hi, lo + ((1u << shift) - 1));
        above = reach - sh.last;
      }
      bound = tie ? lo + 1 : lo;
      from = logit_of(bound);
      rest.ref = ref;
      rest.lim = lim;
      rest.st = sh.spare[tid];
    }
    put_ranked(cands, kk, bound, top, out, sh);
    for (int c = tid; c < cands - kk; c += NT) rest.template add<1>(&sh.spare[c], sc);
    if (cands < kk) {  // (many equal maxima)
      const int last = take_equal<T, MODE>(row, C, lo, kk - cands, cands, out, sh);
      if (lo != kKeyOfNothing) {  // (the sums have all of the equal ones, and nothing is subtracted)
        rest = Sums<1>();
        add_rest<false>(row, C, lo, last, sc, rest);
      }
    }
  } else {
    topk_any<T, MODE>(row, C, kk, sc, out, sh, rest);
  }
  for (int r = kk + tid; r < a.k; r += NT) {
    if (MODE == kTopkSlices) {
      out.put(r, -INFINITY, -1);
    } else {
      a.values[static_cast<int64_t>(n) * a.k + r] = -INFINITY;
      a.indices[static_cast<int64_t>(n) * a.k + r] = -1;
    }
  }
  if (MODE == kTopkRows && a.tail == nullptr) return;
  __syncthreads();
  RowSums sum = block_sums<1, NT>(rest, 0.0, false, sc, sh.red);
  // The sums' references are those of all logits.  Where the others lie so far below the largest that terms may have been lost (each less than
  // 2^-126 of a sum about it, fewer than 2^30 of them), they are taken anew.
  if (sum.st < 0x1p-60f && kk < C && out.value(kk - 1) != -INFINITY) {
    __syncthreads();
    rest = Sums<1>();
    add_rest<false>(row, C, order_key(out.value(kk - 1)), out.at(kk - 1), sc, rest);  // (+infinity among them would have made it infinite)
    sum = block_sums<1, NT>(rest, 0.0, false, sc, sh.red);
  }
  if (tid != 0) return;
  if (sum.st == 0.f) sum.ref = -FLT_MAX;  // (a slice of nothing: its sum is joined with others)
  if (MODE == kTopkSlices) a.part_sums[static_cast<int64_t>(n) * a.slices + slice] = sum;
  else a.tail[n] = tail_of(sum, a.temperature);
}

// A row whose logits are PER a thread at most, in registers; they are their own streams, and nothing is read again.  The rows are short
// ones, or the largest logits of a row's slices (slices in their order, each in its own: equal logits lie in the order of their classes).
// One workgroup per row.  Bound by the chain from loads over bins and order to the output: 40 x 1000, 8 entries 6.1 us, of which a launch that does
// nothing takes 2 to 4; the joining of 1 x 131072, 64 entries 6.6 behind the slices' 9.3.
constexpr int kJoin = 16;
template <typename T, int MODE, int PER>
__global__ __launch_bounds__(kTopkThreads) void topk_short_kernel(const TopkArgs a) {
  constexpr int NT = kTopkThreads;
  constexpr bool JOIN = MODE == kTopkJoin;
  __shared__ TopkShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = blockIdx.y * gridDim.x + blockIdx.x;
  if (n >= a.N) return;
  const int total = JOIN ? a.slices * a.k : a.C;  // (JOIN: at least k of them logits, every slice but the last has k)
  const int kk = min(a.k, total);
  const T* list = JOIN ? reinterpret_cast<const T*>(a.part_values) + static_cast<int64_t>(n) * total : static_cast<const T*>(a.logits) + n * a.ld;
  const TopkOut<MODE> out{a, n, 0};
  Scales sc;
  sc.t = sc.one = kLog2e / a.temperature;
  sc.slack = 20.f / sc.t;
  float z[PER];
  uint32_t key[PER], most = 0, least = 0xffffffffu;
#pragma unroll
  for (int g = 0; g < PER; ++g) {
    const int i = g * NT + tid;
    z[g] = i < total ? Elem<T>::load(list + i) : -INFINITY;
  }
#pragma unroll
  for (int g = 0; g < PER; ++g) {
    const bool in = g * NT + tid < total;
    key[g] = in ? order_key(z[g]) : 0;
    most = max(most, key[g]);
    least = min(least, in ? key[g] : least);
  }
  if (tid == 0) sh.taken = 0;
  sh.hist[tid] = 0;
  sh.first[tid] = -1;
  if (JOIN) least = order_key(Elem<T>::load(list + a.k - 1));  // of the first slice's k logits the last is one that k reach
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), off, 64)));
    if (!JOIN) least = min(least, static_cast<uint32_t>(__shfl_xor(static_cast<int>(least), off, 64)));
  }
  if (lane == 0) sh.count[1][wave] = static_cast<int>(most), sh.count[1][4 + wave] = static_cast<int>(least);
  __syncthreads();
  for (int w = 0; w < 4; ++w) {
    most = max(most, static_cast<uint32_t>(sh.count[1][w]));
    least = min(least, static_cast<uint32_t>(sh.count[1][4 + w]));
  }
  // (a row of masked logits and a few others: its bins are those of the others)
  if (!JOIN && least == kKeyOfNothing) {
    uint32_t above = most;
    int c = 0;
#pragma unroll
    for (int g = 0; g < PER; ++g)
      if (key[g] > kKeyOfNothing) {
        above = min(above, key[g]);
        ++c;
      }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      above = min(above, static_cast<uint32_t>(__shfl_xor(static_cast<int>(above), off, 64)));
      c += __shfl_xor(c, off, 64);
    }
    __syncthreads();
    if (lane == 0) sh.count[1][wave] = static_cast<int>(above), sh.count[1][4 + wave] = c;
    __syncthreads();
    c = 0;
    for (int w = 0; w < 4; ++w) {
      above = min(above, static_cast<uint32_t>(sh.count[1][w]));
      c += sh.count[1][4 + w];
    }
    if (c >= kk) least = above;
  }
  bool tie;
  const uint32_t lo = find_bound<PER>(key, least, most, kk, &tie, sh);
  const uint32_t bound = tie ? lo + 1 : lo;
#pragma unroll
  for (int g = 0; g < PER; ++g)
    if (key[g] >= bound) {
      const int at = atomicAdd(&sh.taken, 1);
      if (at < kTopkCand) {
        sh.cand[at] = static_cast<unsigned long long>(key[g]) << 32 | ~static_cast<uint32_t>(g * NT + tid);
        sh.value[at] = z[g];
      }
      z[g] = -INFINITY;
    }
  __syncthreads();
  const int cands = min(sh.taken, kTopkCand);  // (find_bound lets at most 400 through)
  put_ranked(cands, kk, bound, most, out, sh);
  if (cands < kk) {  // the rest from the equal ones, in their order
    const int need = kk - cands;
    uint64_t votes[PER];
#pragma unroll
    for (int g = 0; g < PER; ++g) {
      votes[g] = __ballot(key[g] == lo);
      if (lane == 0) sh.count[0][g * 4 + wave] = __popcll(votes[g]);
    }
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int g = 0; g < PER; ++g) {
      int pos = before + __popcll(votes[g] & ((1ull << lane) - 1));
      for (int w = 0; w < 4; ++w) {
        const int c = sh.count[0][g * 4 + w];
        pos += w < wave ? c : 0;
        before += c;
      }
      if (key[g] == lo && pos < need) {
        out.put(cands + pos, z[g], g * NT + tid);
        z[g] = -INFINITY;
      }
    }
  }
  for (int r = kk + tid; r < a.k; r += NT) {
    a.values[static_cast<int64_t>(n) * a.k + r] = -INFINITY;
    a.indices[static_cast<int64_t>(n) * a.k + r] = -1;
  }
  if (a.tail == nullptr) return;
  Sums<1> rest;
  if (most >= kKeyOfInfinity) {
    bool left = false;  // of more infinities than places
#pragma unroll
    for (int g = 0; g < PER; ++g) {
      left |= z[g] == INFINITY;
      z[g] = z[g] == INFINITY ? -INFINITY : z[g];
    }
    for (int c = tid; c < cands - kk; c += NT)
      if (sh.spare[c] == INFINITY) left = true, sh.spare[c] = -INFINITY;
    if (left) rest.infinite(sc);
  }
  rest.template add<PER>(z, sc);
  for (int c = tid; c < cands - kk; c += NT) rest.template add<1>(&sh.spare[c], sc);
  if (JOIN && tid < a.slices) {
    const RowSums part = a.part_sums[static_cast<int64_t>(n) * a.slices + tid];
    Sums<1> p;
    p.ref = part.ref;
    p.st = part.st;
    rest.join(p, sc);
  }
  const RowSums sum = block_sums<1, NT>(rest, 0.0, false, sc, sh.red);
  if (tid == 0) a.tail[n] = tail_of(sum, a.temperature);
}

// What the gradient pass needs of its row: d = coef_t * exp((z - ref) / T) + coef_1 * exp(z - ref) - offset (EXPS = 1: both
// coefficients in coef_t) for every class; the classes at[0..k] get value[] instead.
struct RowGrad {
  float ref, coef_t, coef_1, offset;
};
struct RowShared {
  int at[kTopMax + 1];      // classes of the entries (-1: absent), then the label's if it is none of theirs
  float z[kTopMax + 1];     // their logits; z[kTopMax]: the label's
  float t[kTopMax];         // the teacher's
  float value[kTopMax + 1];
  int first[1024], next[kTopMax + 1];  // the entries of every thread, as lists
  RowGrad g;
};
// Hands entry j, of class c, to the thread that writes class c's gradient: of whole vectors of V classes in turn, of the classes of no
// vector one each.  (c: from the first class of the workgroup's slice; a class outside is nobody's here.)
template <int V, int NT>
__device__ __forceinline__ void hand_over(RowShared& sh, const Places& places, int j, int c) {
  if (c < 0 || c >= places.classes) return;
  const int whole = (places.classes - places.head) / V * V, at = places.of(c);
  sh.next[j] = atomicExch(&sh.first[at < whole ? at / V % NT : at - whole], j);
}

// A row's gradient coefficients and loss, by one wave.  Everything is relative to the largest logit and the largest cell; the logarithms
// are those of sums of exponentials, and differences of them are small beside the logits: in double.  The coefficients first (the
// other waves wait for them), the loss when they are gone.  (Loops that are not unrolled: their registers are the kernel's.)
template <int EXPS, int V, int NT>
struct RowEnd {
  const DistillArgs& a;
  const Scales& sc;
  const RowSums& r;
  RowShared& sh;
  int label, k, first;  // (the first class of the workgroup's slice of the row)
  const Places& places;
  float M, tau, AT, A1, S, pt;
  double Mt;
  bool empty, none;

  __device__ __forceinline__ RowEnd(const DistillArgs& a_, const Scales& sc_, const RowSums& r_, RowShared& sh_, int label_, int k_, int first_, const Places& places_)
      : a(a_), sc(sc_), r(r_), sh(sh_), label(label_), k(k_), first(first_), places(places_) {}
  __device__ __forceinline__ float cell(double over) const { return __builtin_amdgcn_exp2f(static_cast<float>(over * static_cast<double>(kLog2e))); }
  __device__ __forceinline__ double teacher(int j) const { return sh.t[j] * (1.0 / static_cast<double>(a.temperature)) - Mt; }

  __device__ __forceinline__ void gradient(float w, float tail) {
    const int lane = threadIdx.x & 63;
    M = r.ref;
    float vt = -INFINITY;
#pragma unroll 1
    for (int j = lane; j < k; j += 64)
      if (sh.at[j] >= 0) {
        M = fmaxf(M, sh.z[j]);
        vt = fmaxf(vt, sh.t[j]);
      }
    M = quick_max(M);
    vt = quick_max(vt);
    Mt = fmax(static_cast<double>(tail), vt * (1.0 / static_cast<double>(a.temperature)));
    empty = Mt == -INFINITY;
    tau = empty ? -INFINITY : static_cast<float>(tail - Mt);
    // sums: the student's at T and at 1, the teacher's
    float eT = 0.f, e1 = 0.f, eS = 0.f;
#pragma unroll 1
    for (int j = lane; j < k; j += 64)
      if (sh.at[j] >= 0) {
        const float d = sh.z[j] - M, e = __builtin_amdgcn_exp2f(d * sc.t);
        eT += e;
        if constexpr (EXPS != 1) e1 += __builtin_amdgcn_exp2f(d * sc.one);
        if (!empty) eS += cell(teacher(j));
      }
    const float down = r.ref - M, rest = r.st * __builtin_amdgcn_exp2f(down * sc.t), from_1 = __builtin_amdgcn_exp2f(down * sc.one);
    pt = empty ? 0.f : __builtin_amdgcn_exp2f(tau * kLog2e);
    AT = quick_sum(eT) + rest;
    A1 = EXPS == 1 ? AT : fmaf(r.s1, from_1, quick_sum(e1));
    S = quick_sum(eS) + pt;
    none = AT == 0.f;  // every logit is -infinity
    if (!a.grad) return;
    const bool ce_on = label >= 0;
    const float g = none ? 0.f : a.grad_scale * w;
    const float gt = empty ? 0.f : g * a.alpha * a.temperature, g1 = ce_on ? g * (1.f - a.alpha) : 0.f;
    const float by_t = 1.f / AT, by_1 = EXPS == 1 ? by_t : 1.f / A1, by_s = empty ? 0.f : 1.f / S;
    RowGrad c;
    c.ref = r.ref;
    c.coef_t = r.st == 0.f || gt == 0.f ? 0.f : gt * (rest * by_t - pt * by_s) / r.st;
    c.coef_1 = g1 == 0.f ? 0.f : g1 * from_1 * by_1;
    c.offset = g1 * a.smoothing / static_cast<float>(a.C);
    if constexpr (EXPS == 1) c.coef_t += c.coef_1;  // (the same exponential)
    bool label_is_entry = false;
#pragma unroll 1
    for (int j = lane; j < k; j += 64)
      if (sh.at[j] >= 0) {
        const float d = sh.z[j] - M, e = __builtin_amdgcn_exp2f(d * sc.t);
        float v = -c.offset;
        if (gt != 0.f) v += gt * (e * by_t - cell(teacher(j)) * by_s);
        if (g1 != 0.f) v += g1 * (EXPS == 1 ? e : __builtin_amdgcn_exp2f(d * sc.one)) * by_1;
        if (ce_on && sh.at[j] == label) v -= g1 * (1.f - a.smoothing), label_is_entry = true;
        sh.value[j] = v;
      }
    const bool known = __any(label_is_entry);
    if (lane == 0) {
      sh.at[kTopMax] = label;
      if (ce_on && !known) {
        const float d = sh.z[kTopMax] - c.ref, y = __builtin_amdgcn_exp2f(d * sc.t);
        float v = fmaf(c.coef_t, y, -c.offset);
        if constexpr (EXPS != 1) v += c.coef_1 * __builtin_amdgcn_exp2f(d * sc.one);
        sh.value[kTopMax] = v - g1 * (1.f - a.smoothing);
        hand_over<V, NT>(sh, places, kTopMax, label - first);
      }
      sh.g = c;
    }
  }

  __device__ __forceinline__ float loss() const {  // (valid in lane 0)
    const int lane = threadIdx.x & 63;
    // four logarithms at once (log 0 = -infinity)
    const double lg = log(static_cast<double>(lane == 0 ? AT : lane == 1 ? A1 : lane == 2 ? S : r.st));
    const double Z = __shfl(lg, 0, 64), Z1 = __shfl(lg, 1, 64), L = __shfl(lg, 2, 64);
    const double ln2 = 0.69314718055994530942;
    const double to_t = static_cast<double>(sc.t) * ln2, to_1 = static_cast<double>(sc.one) * ln2;  // the scales as the exponentials have them
    const double lam = (static_cast<double>(r.ref) - M) * to_t + __shfl(lg, 3, 64);
    double kl = 0;
#pragma unroll 1
    for (int j = lane; j < k; j += 64)
      if (sh.at[j] >= 0 && !empty) {
        const double logp = teacher(j) - L;
        const float p = cell(logp);
        if (p != 0.f) kl += p * (logp - ((static_cast<double>(sh.z[j]) - M) * to_t - Z));
      }
    kl = wave_sum(kl);
    if (pt != 0.f) kl += cell(tau - L) * ((tau - L) - (lam - Z));
    double loss = 0;
    if (!none) {
      if (!empty) loss += static_cast<double>(a.alpha) * a.temperature * a.temperature * kl;
      if (label >= 0) {
        double ce = 0;  // (a term of weight 0 is none, also where the label's logit is -infinity)
        if (a.smoothing < 1.f) ce = -(1.0 - a.smoothing) * ((static_cast<double>(sh.z[kTopMax]) - M) * to_1 - Z1);
        if (a.smoothing > 0.f) ce -= static_cast<double>(a.smoothing) / a.C * ((r.sz - static_cast<double>(a.C) * M) - a.C * Z1);
        loss += (1.0 - a.alpha) * ce;
      }
    }
    return static_cast<float>(loss);
  }
};

template <int EXPS>
__device__ __forceinline__ float gradient_of(float z, const RowGrad& g, const Scales& sc) {
  const float u = z - g.ref, y = __builtin_amdgcn_exp2f(u * sc.t);
  float d = fmaf(g.coef_t, y, -g.offset);
  if constexpr (EXPS == 2) d = fmaf(g.coef_1, y * y, d);
  if constexpr (EXPS == 4) {
    const float y2 = y * y;
    d = fmaf(g.coef_1, y2 * y2, d);
  }
  if constexpr (EXPS == 0) d = fmaf(g.coef_1, __builtin_amdgcn_exp2f(u * sc.one), d);
  return d;
}
template <typename T, int EXPS, bool STREAM>
__device__ __forceinline__ void store_gradient(T* to, const Vec16& x, const RowGrad& g, const Scales& sc) {
  constexpr int V = Elem<T>::VEC;
  float z[V];
  Elem<T>::unpack(x, z);
#pragma unroll
  for (int j = 0; j < V; ++j) z[j] = gradient_of<EXPS>(z[j], g, sc);
  Vec16 d;
  Elem<T>::pack(z, d);
  if constexpr (STREAM) store16_any_stream(to, d);
  else store16_any(to, d);
}

// One workgroup per row, NT threads, at least as many as a row has entries: a thread has one at most.  Whole vectors of V classes go round the
// threads, the classes of no vector (in front of the first, behind the last) are one thread's each.
// U > 0: the row is U vectors a thread at most and stays in registers between the sums and the gradient: it is read once.  U = 0: it is
// read for the sums and again for the gradient (from its end), in chunks of classes whose membership bits fit LDS; the gradient is stored past the
// caches, which keep the rows for their second reading (2048 x 131072 bf16 272 -> 246 us, float 500 -> 476).  A thread adds the same vectors in
// the same order in both.  Bound: the loss of 4096 x 50001 bf16, 87 us, by instructions (41.5 million of a wave's, one exponential a logit: the vector ALUs are never idle);
// loss and gradient of 2048 x 131072, 250 us, by memory: one reading from it, one from the last-level cache and one writing, 6.4 TB/s together.
template <typename T, int EXPS, int NT, int U>
__global__ __launch_bounds__(NT) void distill_rows_kernel(const DistillArgs a) {
  constexpr int V = Elem<T>::VEC;
  constexpr int CHUNK = U > 0 ? U * NT * V + 32 : 65536;  // classes whose membership bits are in LDS at a time
  constexpr int G = sizeof(T) == 2 ? 2 : 4, GG = 4;       // vectors whose loads go out together, for the sums and the gradient (U = 0)
  __shared__ uint32_t member[CHUNK / 32];
  __shared__ RowShared sh;
  __shared__ RowSums red[NT / 64];
  const int tid = threadIdx.x;
  // (a grid of rows, not a loop over them: what the end of a row needs in constants would stay in registers through its sums)
  const int n = blockIdx.y * gridDim.x + blockIdx.x;
  if (n >= a.N) return;
  const Scales sc = scales_of(a, EXPS);
  const T* row = static_cast<const T*>(a.logits) + n * a.ld;
  T* grad = a.grad ? static_cast<T*>(a.grad) + n * a.grad_ld : nullptr;
  const Places places(row, a.C);
  const T* vecs = row + places.head;
  const int k = a.alpha > 0.f ? a.k : 0, whole = (a.C - places.head) / V, left = a.C - whole * V;
  // what the row's end needs goes out first: it is a chain of loads (entry, its logit)
  int at = -1;
  if (tid < k) {
    at = a.t_indices[static_cast<int64_t>(n) * a.k + tid];
    sh.t[tid] = a.t_values[static_cast<int64_t>(n) * a.k + tid];
  }
  const float w = a.row_weight ? a.row_weight[n] : 1.f / static_cast<float>(a.N);
  const float tail = a.alpha > 0.f && a.t_tail ? a.t_tail[n] : -INFINITY;
  int label = a.labels && a.alpha < 1.f ? a.labels[n] : -1;
  if (label >= a.C) label = -1;
  Vec16 held[U > 0 ? U : 1];
  if constexpr (U > 0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * NT + tid < whole) held[u] = load16(vecs + (u * NT + tid) * V);
  }
  const int mine = whole * V + tid, c_left = places.class_at(mine);  // (tid < left)
  const float z_left = tid < left ? Elem<T>::load(row + c_left) : -INFINITY;
  if (w == 0.f) {  // (behind the loads: the weight is a load as well)
    for (int i = tid; grad && i < a.C; i += NT) Elem<T>::store(grad + i, 0.f);
    if (tid == 0) a.row_loss[n] = 0.f;
    return;
  }
  if (at >= a.C || at < 0) at = -1;
  const float z_at = at >= 0 ? Elem<T>::load(row + at) : -INFINITY;
  if (tid == 0 && label >= 0) sh.z[kTopMax] = Elem<T>::load(row + label);
  const int place = at >= 0 ? places.of(at) : -1;

  const bool want_sz = label >= 0 && a.smoothing > 0.f;
  Sums<EXPS> sums;
  double sz = 0;  // (in double: beside classes masked with the lowest float it still holds what the others add)
  auto members = [&](int e) __attribute__((always_inline)) {  // e: a vector's first place, from the chunk's first
    return member[static_cast<uint32_t>(e) >> 5] >> (e & 31) & ((1u << V) - 1);
  };
  auto add = [&](const Vec16& x, uint32_t bits) __attribute__((always_inline)) {
    float z[V];
    Elem<T>::unpack(x, z);
    if (want_sz) {
#pragma unroll
      for (int j = 0; j < V; ++j) sz += static_cast<double>(z[j]);
    }
    if (__any(bits)) {
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
    if (place >= c0 && place - c0 < chunk) repeated = atomicOr(&member[(place - c0) >> 5], 1u << ((place - c0) & 31)) >> ((place - c0) & 31) & 1;
    __syncthreads();
    if constexpr (U > 0) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (u * NT + tid < whole) {
          add(held[u], members((u * NT + tid) * V));
          // the gradient unpacks them again: floats kept from here would be twice the registers
          asm volatile("" : "+v"(held[u].u.x), "+v"(held[u].u.y), "+v"(held[u].u.z), "+v"(held[u].u.w));
          __builtin_amdgcn_sched_barrier(0);
        }
    } else {
      const T* from = vecs + c0;
      const int last = min(whole - c0 / V, CHUNK / V);
      int v = tid;
      for (; v + (G - 1) * NT < last; v += G * NT) {
        Vec16 x[G];
#pragma unroll
        for (int g = 0; g < G; ++g) x[g] = load16(from + (v + g * NT) * V);
        uint32_t bits[G];
#pragma unroll
        for (int g = 0; g < G; ++g) bits[g] = members((v + g * NT) * V);
#pragma unroll
        for (int g = 0; g < G; ++g) add(x[g], bits[g]);
      }
      for (; v < last; v += NT) add(load16(from + v * V), members(v * V));
    }
    if (tid < left && mine >= c0 && mine - c0 < chunk) {
      if (want_sz) sz += static_cast<double>(z_left);
      if (!(member[(mine - c0) >> 5] >> ((mine - c0) & 31) & 1)) sums.template add<1>(&z_left, sc);
    }
  }
  if (tid < k) {
    sh.at[tid] = at;
    sh.z[tid] = z_at;
  }
  sh.first[tid] = -1;
  if (__syncthreads_or(repeated)) {  // of entries with the same class the first stands
    bool drop = false;
    for (int h = 0; h < tid && at >= 0 && tid < k; ++h) drop |= sh.at[h] == at;
    __syncthreads();
    if (drop) sh.at[tid] = at = -1;
  }
  if (at >= 0) hand_over<V, NT>(sh, places, tid, at);
  const RowSums r = block_sums<EXPS, NT>(sums, sz, want_sz, sc, red);
  RowEnd<EXPS, V, NT> end(a, sc, r, sh, label, k, 0, places);
  if (tid < 64) end.gradient(w, tail);
  __syncthreads();
  if (tid < 64) {
    const float loss = end.loss();
    if (tid == 0) a.row_loss[n] = loss;
  }
  if (!grad) return;
  const RowGrad g = sh.g;
  T* to = grad + places.head;
  if constexpr (U > 0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * NT + tid < whole) {
        store_gradient<T, EXPS, false>(to + (u * NT + tid) * V, held[u], g, sc);
        __builtin_amdgcn_sched_barrier(0);
      }
  } else {
    // from the end, where the caches still have the row
    int v = (whole - 1 - tid) / NT * NT + tid;  // (whole <= tid: below tid)
    if (whole <= tid) v = -1;
    for (; v >= (GG - 1) * NT; v -= GG * NT) {
      Vec16 x[GG];
#pragma unroll
      for (int i = 0; i < GG; ++i) x[i] = load16(vecs + (v - i * NT) * V);
#pragma unroll
      for (int i = 0; i < GG; ++i) store_gradient<T, EXPS, true>(to + (v - i * NT) * V, x[i], g, sc);
    }
    for (; v >= 0; v -= NT) store_gradient<T, EXPS, true>(to + v * V, load16(vecs + v * V), g, sc);
  }
  if (tid < left) Elem<T>::store(grad + c_left, gradient_of<EXPS>(z_left, g, sc));
  // The entries' classes and the label's: written once more, each by the thread that wrote it first (whose stores to one address stay in
  // order: no barrier, which would wait for every store of the row).
  for (int j = sh.first[tid]; j >= 0; j = sh.next[j]) Elem<T>::store(grad + sh.at[j], sh.value[j]);
}

// Few rows: slices of a row by workgroups of their own, in two launches.  The first leaves the sums of every slice and, from the slice that
// has it, every entry's class and logit (a gradient in the logits' place overwrites them in the second); the second joins the
// sums, every slice for itself, and writes the slice's gradient.  Bound by their chains: 7 x 131072 bf16, 32 entries 4.5 and 5.6 us and 3.4 for the loss,
// of which a launch that does nothing takes 2 to 4 each.
struct SliceArgs {
  RowSums* sums;  // [N][slices]
  int* at;        // [N][kTopMax]
  float* z;       // [N][kTopMax + 1], the last the label's
  float* loss;
  int slices, width;  // (width: a multiple of 32 classes)
};
constexpr int kSliceThreads = 256;
template <typename T, int EXPS>
__global__ __launch_bounds__(kSliceThreads) void distill_slice_sums_kernel(const DistillArgs a, const SliceArgs p) {
  constexpr int V = Elem<T>::VEC, NT = kSliceThreads, CHUNK = 16384, G = 2;
  __shared__ uint32_t member[CHUNK / 32];
  __shared__ RowSums red[NT / 64];
  __shared__ int at_s[kTopMax];
  const int tid = threadIdx.x, slice = blockIdx.x, n = blockIdx.y;
  const int first = slice * p.width, classes = min(p.width, a.C - first);
  const Scales sc = scales_of(a, EXPS);
  const int k = a.alpha > 0.f ? a.k : 0;
  const T* row = static_cast<const T*>(a.logits) + n * a.ld + first;
  const Places places(row, classes);
  const T* vecs = row + places.head;
  const int whole = (classes - places.head) / V, left = classes - whole * V, c_left = places.class_at(whole * V + tid);  // (tid < left)
  int at = tid < k ? a.t_indices[static_cast<int64_t>(n) * a.k + tid] : -1;
  if (a.row_weight && a.row_weight[n] == 0.f) return;
  int label = a.labels && a.alpha < 1.f ? a.labels[n] : -1;
  if (label >= a.C) label = -1;
  if (at >= a.C || at < 0) at = -1;
  const bool mine = at >= first && at - first < classes;
  const int place = mine ? places.of(at - first) : -1;
  const float z_at = mine ? Elem<T>::load(row + (at - first)) : -INFINITY;
  if (tid == 0 && label >= first && label - first < classes) p.z[static_cast<int64_t>(n) * (kTopMax + 1) + kTopMax] = Elem<T>::load(row + (label - first));
  if (tid < k) at_s[tid] = at;
  const bool want_sz = label >= 0 && a.smoothing > 0.f;
  Sums<EXPS> sums;
  double sz = 0;
  auto members = [&](int e) __attribute__((always_inline)) { return member[static_cast<uint32_t>(e) >> 5] >> (e & 31) & ((1u << V) - 1); };
  auto add = [&](const Vec16& x, uint32_t bits) __attribute__((always_inline)) {
    float z[V];
    Elem<T>::unpack(x, z);
    if (want_sz) {
#pragma unroll
      for (int j = 0; j < V; ++j) sz += static_cast<double>(z[j]);
    }
    if (__any(bits)) {
#pragma unroll
      for (int j = 0; j < V; ++j) z[j] = bits >> j & 1 ? -INFINITY : z[j];
    }
    sums.template add<V>(z, sc);
  };
  bool repeated = false;
  for (int c0 = 0; c0 < classes; c0 += CHUNK) {
    const int chunk = min(classes - c0, CHUNK), last = min(whole - c0 / V, CHUNK / V), e_at = place - c0;
    if (c0) __syncthreads();
    for (int i = tid; i < (chunk + 31) / 32; i += NT) member[i] = 0;
    __syncthreads();
    if (mine && e_at >= 0 && e_at < chunk) repeated = atomicOr(&member[e_at >> 5], 1u << (e_at & 31)) >> (e_at & 31) & 1;
    __syncthreads();
    const T* from = vecs + c0;
    int v = tid;
    for (; v + (G - 1) * NT < last; v += G * NT) {
      Vec16 x[G];
#pragma unroll
      for (int g = 0; g < G; ++g) x[g] = load16(from + (v + g * NT) * V);
      uint32_t bits[G];
#pragma unroll
      for (int g = 0; g < G; ++g) bits[g] = members((v + g * NT) * V);
#pragma unroll
      for (int g = 0; g < G; ++g) add(x[g], bits[g]);
    }
    for (; v < last; v += NT) add(load16(from + v * V), members(v * V));
    const int e = whole * V + tid - c0;
    if (tid < left && e >= 0 && e < chunk) {
      const float z = Elem<T>::load(row + c_left);
      if (want_sz) sz += static_cast<double>(z);
      if (!(member[e >> 5] >> (e & 31) & 1)) sums.template add<1>(&z, sc);
    }
  }
  if (__syncthreads_or(repeated)) {  // of entries with the same class, all of them in this slice, the first stands
    bool drop = false;
    for (int h = 0; h < tid && mine; ++h) drop |= at_s[h] == at;
    if (drop) at = -1;
  }
  if (mine || (tid < k && at < 0 && slice == 0)) {  // (an entry of no class: the first slice's)
    p.at[static_cast<int64_t>(n) * kTopMax + tid] = at;
    p.z[static_cast<int64_t>(n) * (kTopMax + 1) + tid] = z_at;
  }
  const RowSums r = block_sums<EXPS, NT>(sums, sz, want_sz, sc, red);
  if (tid == 0) p.sums[static_cast<int64_t>(n) * p.slices + slice] = r;
}
template <typename T, int EXPS>
__global__ __launch_bounds__(kSliceThreads) void distill_slice_end_kernel(const DistillArgs a, const SliceArgs p) {
  constexpr int V = Elem<T>::VEC, NT = kSliceThreads, G = 2;
  __shared__ RowShared sh;
  __shared__ RowSums red[NT / 64];
  const int tid = threadIdx.x, slice = blockIdx.x, n = blockIdx.y;
  const int first = slice * p.width, classes = min(p.width, a.C - first);
  const Scales sc = scales_of(a, EXPS);
  const int k = a.alpha > 0.f ? a.k : 0;
  const float w = a.row_weight ? a.row_weight[n] : 1.f / static_cast<float>(a.N);
  const T* row = static_cast<const T*>(a.logits) + n * a.ld + first;
  T* grad = a.grad ? static_cast<T*>(a.grad) + n * a.grad_ld + first : nullptr;
  const Places places(row, classes);
  const T* vecs = row + places.head;
  const int whole = (classes - places.head) / V, left = classes - whole * V, c_left = places.class_at(whole * V + tid);  // (tid < left)
  if (w != 0.f) {
    const float tail = a.alpha > 0.f && a.t_tail ? a.t_tail[n] : -INFINITY;
    int label = a.labels && a.alpha < 1.f ? a.labels[n] : -1;
    if (label >= a.C) label = -1;
    int at = -1;
    if (tid < k) {
      at = p.at[static_cast<int64_t>(n) * kTopMax + tid];
      sh.at[tid] = at;
      sh.z[tid] = p.z[static_cast<int64_t>(n) * (kTopMax + 1) + tid];
      sh.t[tid] = a.t_values[static_cast<int64_t>(n) * a.k + tid];
    }
    if (tid == 0 && label >= 0) sh.z[kTopMax] = p.z[static_cast<int64_t>(n) * (kTopMax + 1) + kTopMax];
    sh.first[tid] = -1;
    Sums<EXPS> sums;  // a slice's a thread
    double sz = 0;
    if (tid < p.slices) {
      const RowSums part = p.sums[static_cast<int64_t>(n) * p.slices + tid];
      sums.ref = part.ref; sums.st = part.st; sums.s1 = part.s1;
      sz = part.sz;
    }
    __syncthreads();
    if (at >= 0) hand_over<V, NT>(sh, places, tid, at - first);
    const RowSums r = block_sums<EXPS, NT>(sums, sz, label >= 0 && a.smoothing > 0.f, sc, red);
    RowEnd<EXPS, V, NT> end(a, sc, r, sh, label, k, first, places);
    if (tid < 64) end.gradient(w, tail);
    __syncthreads();
    if (slice == 0 && tid < 64) {
      const float loss = end.loss();
      if (tid == 0) a.row_loss[n] = loss;
      if (tid == 0 && a.N == 1) *p.loss = w * loss;
    }
    if (grad) {
      const RowGrad g = sh.g;
      T* to = grad + places.head;
      int v = tid;
      for (; v + (G - 1) * NT < whole; v += G * NT) {
        Vec16 x[G];
#pragma unroll
        for (int i = 0; i < G; ++i) x[i] = load16(vecs + (v + i * NT) * V);
#pragma unroll
        for (int i = 0; i < G; ++i) store_gradient<T, EXPS, false>(to + (v + i * NT) * V, x[i], g, sc);
      }
      for (; v < whole; v += NT) store_gradient<T, EXPS, false>(to + v * V, load16(vecs + v * V), g, sc);
      if (tid < left) Elem<T>::store(grad + c_left, gradient_of<EXPS>(Elem<T>::load(row + c_left), g, sc));
      for (int j = sh.first[tid]; j >= 0; j = sh.next[j]) Elem<T>::store(grad + (sh.at[j] - first), sh.value[j]);
    }
  } else {
    for (int i = tid; grad && i < classes; i += NT) Elem<T>::store(grad + i, 0.f);
    if (slice == 0 && tid == 0) a.row_loss[n] = 0.f;
    if (slice == 0 && tid == 0 && a.N == 1) *p.loss = 0.f;
  }
}

// loss = sum_n w_n row_loss_n, in double, in a fixed order.  One workgroup: a few kilobytes, eight of each thread's loads at a time
// (one at a time 32768 rows took 77 us).
__global__ __launch_bounds__(1024) void distill_loss_kernel(const float* __restrict__ row_loss, const float* __restrict__ row_weight, int N,
                                                            float* __restrict__ loss) {
  __shared__ double red[16];
  constexpr int U = 8;
  double s = 0;
  for (int64_t n0 = threadIdx.x; n0 < N; n0 += U * 1024) {
    float l[U], w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t n = n0 + u * 1024;
      l[u] = n < N ? row_loss[n] : 0.f;
      w[u] = n < N && row_weight ? row_weight[n] : 1.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) s += w[u] != 0.f ? static_cast<double>(w[u]) * l[u] : 0.0;
  }
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) s += red[i];
    loss[0] = static_cast<float>(row_weight ? s : s / N);
  }
}

// Slices of a row where rows are few (1: a workgroup does the row), every one of at least k classes but the last, and the parts of the
// workspace that they need.  A workgroup a row -> slices: 1 x 131072, 64 entries 18.0 -> 16.2 us (of 2048 classes 20.1), 256 entries float
// 32.7 -> 23.5, 32 x 131072 19.7 -> 18.0, 200 x 131072 float 43.0 -> 32.6; 1 x 65536 float 14.8 -> 14.8, 1 x 32768 10.0 -> 14.7.
static void topk_slicing(int N, int C, int k, TopkArgs* a, void* workspace, size_t* bytes) {
  int least = 80000, target = 512, most_rows = 240, narrow = 8192;
#ifdef RN50_TUNING  // tuning builds only: RN50_TOPK_SLICES=least classes of a row,workgroups,rows,least classes of a slice
  if (const char* e = getenv("RN50_TOPK_SLICES")) sscanf(e, "%d,%d,%d,%d", &least, &target, &most_rows, &narrow);
#endif
  *bytes = 0;
  if (N > most_rows || C < least) return;
  const int64_t want = std::min<int64_t>({ceil_div(target, N), ceil_div(C, narrow), kTopkThreads, kJoin * kTopkThreads / k});
  if (want < 2) return;
  const int width = static_cast<int>(align_up(static_cast<size_t>(ceil_div(C, want)), 32)), slices = static_cast<int>(ceil_div(C, width));
  const size_t list = align_up(static_cast<size_t>(N) * slices * k * 4, 256);
  *bytes = 2 * list + sizeof(RowSums) * N * slices;
  if (!a) return;
  unsigned char* p = static_cast<unsigned char*>(workspace);
  a->slices = slices;
  a->width = width;
  a->part_values = reinterpret_cast<float*>(p);
  a->part_at = reinterpret_cast<int32_t*>(p + list);
  a->part_sums = reinterpret_cast<RowSums*>(p + 2 * list);
}
template <typename T>
static void topk_run(TopkArgs a, hipStream_t s) {
  if (a.slices < 2) {
    // Short rows in registers (us, streams -> registers): 40 x 1000, 8 entries 6.6 -> 5.9, 64 x 1000, 256 entries float 51 -> 7.0 (fewer vectors than
    // entries: no bound from their maxima), 86 x 306, 75 entries bf16 26 -> 6.0; with 16 logits a thread 64 x 2000, 200 entries bf16 28 -> 10.4, but
    // 100 entries 8.2 -> 9.2, 64 x 4000, 256 entries 13.2 -> 14.2, 4096 x 2048, 16 entries 21 -> 42.
    if (a.C <= kTopkThreads * 4)
      RN50_LAUNCH("topk_rows", (topk_short_kernel<T, kTopkRows, 4>), row_grid(a.N), dim3(kTopkThreads), 0, s, a);
    else if (a.C <= kTopkThreads * kJoin && a.C / Elem<T>::VEC * 2 < a.k * 3)
      RN50_LAUNCH("topk_rows", (topk_short_kernel<T, kTopkRows, kJoin>), row_grid(a.N), dim3(kTopkThreads), 0, s, a);
    else
      RN50_LAUNCH("topk_rows", (topk_rows_kernel<T, kTopkRows>), row_grid(a.N), dim3(kTopkThreads), 0, s, a);
    return;
  }
  RN50_LAUNCH("topk_rows", (topk_rows_kernel<T, kTopkSlices>), dim3(a.slices, a.N), dim3(kTopkThreads), 0, s, a);
  RN50_LAUNCH("topk_rows", (topk_short_kernel<float, kTopkJoin, kJoin>), row_grid(a.N), dim3(kTopkThreads), 0, s, a);
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
  // Rows that are read twice are read from the last-level cache (256 MB) the second time while all that are in flight fit it: with four
  // workgroups of rows of 256 KB on a compute unit they do not, so LDS that nobody uses keeps the fourth away (2048 x 131072 bf16 256 -> 250 us,
  // 2048 x 180000 392 -> 369).
  const int64_t fit = (int64_t{224} << 20) / (256 * static_cast<int64_t>(a.C) * static_cast<int64_t>(sizeof(T)));
  const int pad = !a.grad || fit > 3 ? 0 : fit == 3 ? 24 * 1024 : 37 * 1024;
#define ROWS(NT, U) RN50_LAUNCH("distill", (distill_rows_kernel<T, EXPS, NT, U>), grid, dim3(NT), U == 0 && NT == 512 ? pad : 0, s, a)
#ifdef RN50_TUNING  // tuning builds only: RN50_DISTILL=threads,vectors held by a thread
  if constexpr (EXPS == 2) {
    int nt, u;
    if (const char* e = getenv("RN50_DISTILL"); e && sscanf(e, "%d,%d", &nt, &u) == 2) {
#define FORCED(NT, U) if (nt == NT && u == U) { ROWS(NT, U); return; }
      FORCED(64, 4) FORCED(64, 8) FORCED(128, 2) FORCED(128, 4) FORCED(256, 0) FORCED(512, 0) FORCED(1024, 0) FORCED(256, 1) FORCED(256, 2) FORCED(256, 4) FORCED(256, 8) FORCED(512, 4) FORCED(512, 8) FORCED(512, 16) FORCED(1024, 8)
#undef FORCED
    }
  }
#endif
  // Small workgroups for short rows: a row is mostly its own end, which few waves share and barriers of few waves part (bf16, 256 threads -> 128:
  // 32768 x 1000 121 -> 90 us, 32768 x 4096 183 -> 161; 64 threads 82, but 40 x 1000 8.9 -> 9.5).  From 1024 vectors on the row is
  // streamed: held in registers it leaves too few workgroups to cover one another (held, streamed: 16384 x 8192 150, 158, 16384 x 16384 262, 250,
  // by 512 threads 4096 x 50001 342, 200).  256 threads against 512: 8192 x 20000 165, 186; 8192 x 24576 191, 187; 8192 x 32768 253, 240;
  // 4096 x 50001 219, 200; 2048 x 131072 279, 253.  512 against 1024: 1024 x 262144 264, 274; float 2048 x 131072 492, 493, 2048 x 180000 771,
  // 703 (fewer rows in flight for the last-level cache), 1024 x 262144 544, 511.
  const bool few = a.k <= 128;  // (an entry a thread)
  if (vecs <= 256) {
    if (few) ROWS(128, 2);
    else ROWS(256, 1);
  } else if (vecs <= 512) {
    if (few) ROWS(128, 4);
    else ROWS(256, 2);
  } else if (vecs <= 1024) {
    ROWS(256, 4);
  } else if (vecs <= 3072) {
    ROWS(256, 0);
  } else if (vecs <= 32768) {
    ROWS(512, 0);
  } else {
    ROWS(1024, 0);
  }
#undef ROWS
}
template <typename T, int EXPS>
static void distill_slices(const DistillArgs& a, const SliceArgs& p, hipStream_t s) {
  RN50_LAUNCH("distill", (distill_slice_sums_kernel<T, EXPS>), dim3(p.slices, a.N), dim3(kSliceThreads), 0, s, a, p);
  RN50_LAUNCH("distill", (distill_slice_end_kernel<T, EXPS>), dim3(a.grad ? p.slices : 1, a.N), dim3(kSliceThreads), 0, s, a, p);
}
template <typename T, int EXPS>
static void distill_exps(const DistillArgs& a, const SliceArgs& p, hipStream_t s) {
  if (p.slices > 1) distill_slices<T, EXPS>(a, p, s);
  else distill_rows<T, EXPS>(a, row_grid(a.N), s);
  if (p.slices == 1 || a.N > 1) {  // (the slices of a single row leave its loss)
    RN50_LAUNCH("distill_loss", distill_loss_kernel, dim3(1), dim3(1024), 0, s, a.row_loss, a.row_weight, a.N, p.loss);
  }
}
template <typename T>
static void distill_run(const DistillArgs& a, const SliceArgs& p, hipStream_t s) {
  const bool both = a.alpha > 0.f && a.alpha < 1.f && a.labels;
  if (!both || a.temperature == 1.f) distill_exps<T, 1>(a, p, s);
  else if (a.temperature == 2.f) distill_exps<T, 2>(a, p, s);
  else if (a.temperature == 4.f) distill_exps<T, 4>(a, p, s);
  else distill_exps<T, 0>(a, p, s);
}

// Slices of a row (1: a workgroup does the row) and their width.  Loss and gradient, 64 entries, a workgroup a row -> slices: 1 x 131072 bf16
// 27.1 -> 9.8 us, 7 x 131072 27.6 -> 11.7, 64 x 32768 15.3 -> 13.4, 128 x 131072 29.2 -> 24.9; 200 x 131072 32.2 -> 35.7, 7 x 20000 float 11.5 -> 12.1,
// 16 x 8192 float 10.2 -> 11.9: up to 128 rows of 4096 vectors and more.
static int distill_slicing(int N, int C, int dtype, int* width) {
  const int V = dtype == RN50_BF16 ? 8 : 4;
  *width = C;
  int least = 4096 * V, target = 1024, most_rows = 128;
#ifdef RN50_TUNING  // tuning builds only: RN50_DISTILL_SLICES=least vectors of a row,workgroups,rows
  if (const char* e = getenv("RN50_DISTILL_SLICES")) {
    sscanf(e, "%d,%d,%d", &least, &target, &most_rows);
    least *= V;
  }
#endif
  if (N > most_rows || C < least) return 1;
  const int64_t want = std::min<int64_t>({ceil_div(target, N), ceil_div(C, kSliceThreads * V), kSliceThreads});
  if (want < 2) return 1;
  *width = static_cast<int>(align_up(static_cast<size_t>(ceil_div(C, want)), 32));
  return static_cast<int>(ceil_div(C, *width));
}
static SliceArgs slice_args(int N, int C, int dtype, void* workspace, size_t* bytes) {
  SliceArgs p{};
  p.slices = distill_slicing(N, C, dtype, &p.width);
  size_t at = 0;
  auto part = [&](size_t size) {
    unsigned char* b = static_cast<unsigned char*>(workspace) + at;
    at += align_up(size, 256);
    return workspace ? b : nullptr;
  };
  if (p.slices > 1) {
    p.sums = reinterpret_cast<RowSums*>(part(sizeof(RowSums) * N * p.slices));
    p.at = reinterpret_cast<int*>(part(sizeof(int) * N * kTopMax));
    p.z = reinterpret_cast<float*>(part(sizeof(float) * N * (kTopMax + 1)));
  }
  *bytes = at;
  return p;
}

}  // namespace rn50

using namespace rn50;

extern "C" size_t topk_rows_workspace_bytes(int N, int C, int k) {
  size_t bytes = 0;
  if (N > 0 && C > 0 && k > 0 && k <= kTopMax) topk_slicing(N, C, k, nullptr, nullptr, &bytes);
  return bytes;
}

extern "C" int topk_rows(int N, int C, int k, int dtype, const void* logits, int64_t ld, float temperature, float* values, int32_t* indices,
                         float* tail_lse, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  if (int rc = check_rows("topk_rows", N, C, dtype, logits, ld)) return rc;
  RN50_REQUIRE(k >= 1 && k <= kTopMax, RN50_ERR_UNSUPPORTED, "topk_rows: k=%d outside [1, %d]", k, kTopMax);
  RN50_REQUIRE(temperature >= FLT_MIN && temperature <= FLT_MAX, RN50_ERR_INVALID, "topk_rows: temperature %g", temperature);
  RN50_REQUIRE(values && indices, RN50_ERR_INVALID, "topk_rows: null pointer");
  RN50_REQUIRE(aligned_to(values, 4) && aligned_to(indices, 4) && aligned_to(tail_lse, 4), RN50_ERR_ALIGN, "topk_rows: pointer not aligned to an element");
  RN50_REQUIRE(aligned16(workspace), RN50_ERR_ALIGN, "topk_rows: workspace not 16-byte aligned");
  const size_t need = topk_rows_workspace_bytes(N, C, k);
  RN50_REQUIRE(workspace_bytes >= need && (need == 0 || workspace), RN50_ERR_WORKSPACE, "topk_rows: workspace %zu < %zu bytes", workspace_bytes, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  TopkArgs a{logits, ld, N, C, k, temperature, values, indices, tail_lse, 1, 0, nullptr, nullptr, nullptr};
  size_t bytes;
  topk_slicing(N, C, k, &a, workspace, &bytes);
  if (dtype == RN50_BF16) topk_run<uint16_t>(a, s);
  else topk_run<float>(a, s);
  return launch_status("topk_rows");
}

extern "C" size_t distill_workspace_bytes(const rn50_distill_desc* d) {
  size_t bytes = 0;
  if (d && d->N > 0 && d->C > 0) slice_args(d->N, d->C, d->dtype, nullptr, &bytes);
  return bytes;
}

extern "C" int distill_fwd_bwd(const rn50_distill_desc* d, const void* logits, const float* t_values, const int32_t* t_indices, const float* t_tail,
                               const int32_t* labels, const float* row_weight, float* loss_out, float* row_loss_out, void* dlogits,
                               void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const char* who = "distill_fwd_bwd";
  RN50_REQUIRE(d, RN50_ERR_INVALID, "%s: null descriptor", who);
  if (int rc = check_rows(who, d->N, d->C, d->dtype, logits, d->ld)) return rc;
  RN50_REQUIRE(d->k >= 0 && d->k <= kTopMax, RN50_ERR_UNSUPPORTED, "%s: k=%d outside [0, %d]", who, d->k, kTopMax);
  RN50_REQUIRE(d->temperature >= FLT_MIN && d->temperature <= FLT_MAX, RN50_ERR_INVALID, "%s: temperature %g", who, d->temperature);
  RN50_REQUIRE(d->alpha >= 0.f && d->alpha <= 1.f, RN50_ERR_INVALID, "%s: alpha %g", who, d->alpha);
  RN50_REQUIRE(d->label_smoothing >= 0.f && d->label_smoothing <= 1.f, RN50_ERR_INVALID, "%s: label_smoothing %g", who, d->label_smoothing);
  RN50_REQUIRE(d->k == 0 || (t_values && t_indices), RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(loss_out && row_loss_out, RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(!dlogits || d->grad_ld >= d->C, RN50_ERR_INVALID, "%s: gradient rows of %d elements %lld apart", who, d->C,
               static_cast<long long>(d->grad_ld));
  RN50_REQUIRE(dlogits != logits || d->grad_ld == d->ld || d->N == 1, RN50_ERR_INVALID, "%s: a gradient in the logits' place with rows of its own", who);
  RN50_REQUIRE(aligned_to(t_values, 4) && aligned_to(t_indices, 4) && aligned_to(t_tail, 4) && aligned_to(labels, 4) && aligned_to(row_weight, 4) &&
                   aligned_to(loss_out, 4) && aligned_to(row_loss_out, 4) && aligned_to(dlogits, d->dtype == RN50_BF16 ? 2 : 4),
               RN50_ERR_ALIGN, "%s: pointer not aligned to an element", who);
  RN50_REQUIRE(aligned16(workspace), RN50_ERR_ALIGN, "%s: workspace not 16-byte aligned", who);
  const size_t need = distill_workspace_bytes(d);
  RN50_REQUIRE(workspace_bytes >= need && (need == 0 || workspace), RN50_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, workspace_bytes, need);
  hipStream_t s = static_cast<hipStream_t>(stream);
  DistillArgs a{logits, dlogits, t_values, t_indices, t_tail, row_weight, labels, row_loss_out, d->ld, d->grad_ld, d->N, d->C, d->k,
                d->temperature, d->alpha, d->label_smoothing, d->grad_scale};
  size_t bytes;
  SliceArgs p = slice_args(d->N, d->C, d->dtype, workspace, &bytes);
  p.loss = loss_out;
  if (d->dtype == RN50_BF16) distill_run<uint16_t>(a, p, s);
  else distill_run<float>(a, p, s);
  return launch_status(who);
}

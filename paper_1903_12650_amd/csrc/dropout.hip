// Dropout: y = kept ? x / (share kept) : 0, the mask drawn anew from a counter wherever it is needed and never stored.
#include <math.h>

#include <algorithm>

#include "dropout.h"

namespace rn50 {

int check_dropout(const char* who, const rn50_dropout* d) {
  if (!d) return RN50_OK;
  RN50_REQUIRE(d->p >= 0.f && d->p <= 1.f, RN50_ERR_INVALID, "%s: dropout probability %g", who, static_cast<double>(d->p));
  RN50_REQUIRE(aligned_to(d->step, 8), RN50_ERR_ALIGN, "%s: the step's counter is not 8-byte aligned", who);
  return RN50_OK;
}
DropArgs drop_args(const rn50_dropout* d) {
  if (!d) return DropArgs{0, 0, 0, 1.f, 0, nullptr};
  const uint32_t t = static_cast<uint32_t>(rint(static_cast<double>(d->p) * 65536.0));
  return DropArgs{static_cast<uint32_t>(d->seed), static_cast<uint32_t>(d->seed >> 32), t,
                  t < 65536 ? static_cast<float>(65536.0 / (65536.0 - t)) : 0.f, d->call, d->step};
}

constexpr int64_t kPastBytes = 32 << 20;  // outputs that the L2s would not hold for the next kernel are stored past them

// A workgroup takes `rows` whole rows at a time, or a part of one row (rows == 1: grid.y parts); item l of them is block l % per_row of row l / per_row:
// eight elements, the 128 bits of one Philox call.  Bound by memory, Philox's multiplications beside it: 50176 x 1024 bf16 with residual 54 us (308 MB, 5.7 TB/s),
// without 36 (206 MB).
struct DropoutArgs {
  DropArgs d;
  const void *x, *residual;
  void* y;
  int64_t ldx, ldr, ldy;
  int M, K, per_row, rows;
  FastDiv by_row;
};
template <typename T, bool RESIDUAL, bool PAST>
__global__ __launch_bounds__(256) void dropout_kernel(const DropoutArgs a) {
  constexpr int V = Elem<T>::VEC;
  const uint64_t call = drop_call(a.d);
  for (int64_t m0 = static_cast<int64_t>(blockIdx.x) * a.rows; m0 < a.M; m0 += static_cast<int64_t>(gridDim.x) * a.rows) {
    const int rows = static_cast<int>(min(static_cast<int64_t>(a.rows), a.M - m0));
    const uint32_t items = static_cast<uint32_t>(rows) * static_cast<uint32_t>(a.per_row), part = 256u * gridDim.y;
    for (uint32_t l = blockIdx.y * 256u + threadIdx.x; l < items; l += part) {
      const uint32_t r = fdiv(l, a.by_row), c = l - r * a.per_row;
      const int64_t m = m0 + r;
      const int k = static_cast<int>(c) * 8, n = min(8, a.K - k);
      const T* x = static_cast<const T*>(a.x) + m * a.ldx + k;
      const T* res = RESIDUAL ? static_cast<const T*>(a.residual) + m * a.ldr + k : nullptr;
      T* y = static_cast<T*>(a.y) + m * a.ldy + k;
      float f[8], g[8];
      if (n == 8) {
#pragma unroll
        for (int j = 0; j < 8; j += V) Elem<T>::unpack(load16_any(x + j), f + j);
        if constexpr (RESIDUAL) {
#pragma unroll
          for (int j = 0; j < 8; j += V) Elem<T>::unpack(load16_any(res + j), g + j);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f[j] = j < n ? Elem<T>::load(x + j) : 0.f;
          if constexpr (RESIDUAL) g[j] = j < n ? Elem<T>::load(res + j) : 0.f;
        }
      }
      const DropBits bits = drop_bits(a.d, call, static_cast<uint64_t>(m) * static_cast<uint32_t>(a.per_row) + c);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool keep = drop_keeps(a.d, bits, j);
        if constexpr (RESIDUAL) f[j] = keep ? fmaf(f[j], a.d.factor, g[j]) : g[j];
        else f[j] = keep ? f[j] * a.d.factor : 0.f;
      }
      if (n == 8) {
#pragma unroll
        for (int j = 0; j < 8; j += V) {
          Vec16 o;
          Elem<T>::pack(f + j, o);
          if constexpr (PAST) store16_any_stream(y + j, o);
          else store16_any(y + j, o);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < n) Elem<T>::store(y + j, f[j]);
      }
    }
  }
}

static int dropout_run(const char* who, const rn50_dropout* d, int M, int K, int dtype, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                       void* y, int64_t ldy, void* stream) {
  clear_error();
  RN50_REQUIRE(dtype == RN50_F32 || dtype == RN50_BF16, RN50_ERR_INVALID, "%s: dtype %d", who, dtype);
  RN50_REQUIRE(M > 0 && K > 0, RN50_ERR_INVALID, "%s: non-positive size", who);
  RN50_REQUIRE(d && x && y, RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(ldx >= K && ldy >= K && (!residual || ldr >= K), RN50_ERR_INVALID, "%s: rows of %d elements closer together than that", who, K);
  const uintptr_t size = dtype == RN50_BF16 ? 2 : 4;
  RN50_REQUIRE(aligned_to(x, size) && aligned_to(residual, size) && aligned_to(y, size), RN50_ERR_ALIGN, "%s: pointer not aligned to an element", who);
  RN50_REQUIRE(M == 1 || ((y != x || ldy == ldx) && (y != residual || ldy == ldr)), RN50_ERR_INVALID,
               "%s: the output in an input's place with rows of another distance", who);
  if (int rc = check_dropout(who, d)) return rc;
  DropoutArgs a{drop_args(d), x, residual, y, ldx, ldr, ldy, M, K, static_cast<int>(ceil_div(K, 8)), 1, {}};
  a.by_row = make_fastdiv(static_cast<uint32_t>(a.per_row));
  // As many rows a workgroup as make whole rounds of its threads, as long as there are eight workgroups a compute unit: 50000 rows of 100 blocks two at
  // a time 33 us, five 28 (otherwise one item a thread: 50176 x 1024 with a residual 55 us, four 58).
  const int64_t one = a.per_row;
  auto idle = [&](int64_t rows) { return static_cast<double>(align_up(static_cast<size_t>(rows * one), 256)) / static_cast<double>(rows * one); };
  int64_t rows = std::max<int64_t>(1, 256 / one), most = std::min<int64_t>(8 * rows, M / 2048);
  for (int64_t r = rows + 1; r <= most && one < 4096; ++r)
    if (idle(r) < idle(rows) - 0.03) rows = r;
  constexpr int64_t kMostGroups = 1 << 20;  // (the rest of the rows by the same workgroups)
  const int64_t parts = rows > 1 ? 1 : std::min<int64_t>(ceil_div(one, 256), 16);
  a.rows = static_cast<int>(rows);
  const dim3 grid(static_cast<unsigned>(std::min(ceil_div(M, rows), kMostGroups)), static_cast<unsigned>(parts));
  hipStream_t s = static_cast<hipStream_t>(stream);
  // (float: a lane's two stores are every other 16 bytes, half lines, which past the caches cost more: 50176 x 1024 72 -> 84 us)
  const bool past = dtype == RN50_BF16 && static_cast<int64_t>(M) * K * 2 >= kPastBytes;
#define DROPOUT(T, RESIDUAL)                                                                                           \
  do {                                                                                                                 \
    if (past) RN50_LAUNCH("dropout", (dropout_kernel<T, RESIDUAL, true>), grid, dim3(256), 0, s, a);                   \
    else RN50_LAUNCH("dropout", (dropout_kernel<T, RESIDUAL, false>), grid, dim3(256), 0, s, a);                       \
  } while (0)
  if (dtype == RN50_BF16 && residual) DROPOUT(uint16_t, true);
  else if (dtype == RN50_BF16) DROPOUT(uint16_t, false);
  else if (residual) DROPOUT(float, true);
  else DROPOUT(float, false);
#undef DROPOUT
  return launch_status(who);
}

}  // namespace rn50

using namespace rn50;

extern "C" int dropout_fwd(const rn50_dropout* d, int M, int K, int dtype, const void* x, int64_t ldx, const void* residual, int64_t ld_residual,
                           void* y, int64_t ldy, void* stream) {
  return dropout_run("dropout_fwd", d, M, K, dtype, x, ldx, residual, ld_residual, y, ldy, stream);
}

extern "C" int dropout_bwd(const rn50_dropout* d, int M, int K, int dtype, const void* dy, int64_t ld_dy, void* dx, int64_t ld_dx, void* stream) {
  return dropout_run("dropout_bwd", d, M, K, dtype, dy, ld_dy, nullptr, 0, dx, ld_dx, stream);
}

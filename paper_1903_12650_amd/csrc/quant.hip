// Products in 8-bit integers: rows quantized with one scale each, and y = (sum_k q w) * q_scale * w_scale + bias on the
// integer matrix cores (v_mfma_i32_32x32x32_i8).
#include "common.h"
#include <algorithm>

namespace rn50 {

constexpr int kI8MaxK = 131071;       // 128 * 128 * K stays below 2^31
constexpr float kI8Floor = 0x1p-100f;  // smaller rows are quantized as if their largest magnitude were this: 127 / a stays finite
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// scale and 127 / a of a row from the bits of its largest magnitude (an infinity's or a NaN's are above every number's).
__device__ __forceinline__ float i8_scale(uint32_t amax_bits, float* inv) {
  const float a = fmaxf(__uint_as_float(amax_bits), kI8Floor);
  const bool finite = amax_bits < 0x7f800000u;
  *inv = finite ? 127.f / a : 0.f;
  return finite ? a / 127.f : __uint_as_float(0x7fc00000u);
}
// rint(x * inv) as the low byte.  Two roundings, as the definition has them: 1.5 * 2^23 added to a number of magnitude 127 leaves its
// nearest integer (ties to even) in the low bits, and a fused multiply-add would round once.
__device__ __forceinline__ uint32_t i8_of(float x, float inv) {
#pragma clang fp contract(off)
  const float t = x * inv;
  return __float_as_uint(t + 12582912.f) & 255u;
}

// One workgroup per row, which is read twice.
template <typename T>
__global__ __launch_bounds__(256) void quant_rows_kernel(const T* __restrict__ x, int64_t ldx, int M, int K, int Kp, int8_t* __restrict__ q,
                                                         float* __restrict__ scale) {
  __shared__ uint32_t red[4];
  for (int m = blockIdx.x; m < M; m += gridDim.x) {
    const T* row = x + m * ldx;
    uint32_t top = 0;
    for (int k = threadIdx.x; k < K; k += 256) top = max(top, __float_as_uint(Elem<T>::load(row + k)) & 0x7fffffffu);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), off, 64)));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(red[0], red[1]), max(red[2], red[3]));
    float inv;
    const float s = i8_scale(top, &inv);
    const bool finite = top < 0x7f800000u;
    int8_t* out = q + static_cast<int64_t>(m) * Kp;
    for (int k = threadIdx.x; k < Kp; k += 256)
      out[k] = k < K && finite ? static_cast<int8_t>(i8_of(Elem<T>::load(row + k), inv)) : static_cast<int8_t>(0);
    if (threadIdx.x == 0) scale[m] = s;
  }
}

// 64x64 outputs per workgroup, 32x32 per wave, operands from memory.  Lane l supplies row l % 32, bytes 16 * (l / 32)..+15 of a k step
// of 32; it receives column l % 32 (of the second operand), rows (v / 4) * 8 + (l / 32) * 4 + v % 4.
template <typename T>
__global__ __launch_bounds__(256) void matmul_i8_kernel(const int8_t* __restrict__ q, const float* __restrict__ qs, const int8_t* __restrict__ w,
                                                        const float* __restrict__ ws, const float* __restrict__ bias, T* __restrict__ y,
                                                        int64_t ldy, int M, int N, int Kp) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int m0 = blockIdx.y * 64 + (wave & 1) * 32, n0 = blockIdx.x * 64 + (wave >> 1) * 32;
  const int8_t* pa = q + static_cast<int64_t>(min(m0 + (lane & 31), M - 1)) * Kp + 16 * (lane >> 5);
  const int8_t* pb = w + static_cast<int64_t>(min(n0 + (lane & 31), N - 1)) * Kp + 16 * (lane >> 5);
  i32x16 acc;
#pragma unroll
  for (int v = 0; v < 16; ++v) acc[v] = 0;
  for (int k = 0; k < Kp; k += 32)
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const i32x4*>(pa + k), *reinterpret_cast<const i32x4*>(pb + k), acc, 0, 0, 0);
  const int n = n0 + (lane & 31);
  if (n >= N) return;
  const float t = ws[n], b = bias ? bias[n] : 0.f;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int m = m0 + (v >> 2) * 8 + (lane >> 5) * 4 + (v & 3);
    if (m < M) Elem<T>::store(y + m * ldy + n, fmaf(static_cast<float>(acc[v]) * qs[m], t, b));
  }
}

static int check_quant(const char* who, int M, int K, int dtype, const void* x, int64_t ldx) {
  RN50_REQUIRE(dtype == RN50_F32 || dtype == RN50_BF16, RN50_ERR_INVALID, "%s: dtype %d", who, dtype);
  RN50_REQUIRE(M > 0 && K > 0, RN50_ERR_INVALID, "%s: non-positive size", who);
  RN50_REQUIRE(K <= kI8MaxK, RN50_ERR_UNSUPPORTED, "%s: K=%d beyond %d, what a 32-bit sum holds", who, K, kI8MaxK);
  RN50_REQUIRE(x, RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(ldx >= K, RN50_ERR_INVALID, "%s: rows of %d elements %lld apart", who, K, static_cast<long long>(ldx));
  RN50_REQUIRE(aligned_to(x, dtype == RN50_BF16 ? 2 : 4), RN50_ERR_ALIGN, "%s: pointer not aligned to an element", who);
  return RN50_OK;
}
static int check_product(const char* who, int M, int N, int K, const void* w, const float* w_scale, const float* bias, int y_dtype, const void* y,
                         int64_t ldy) {
  RN50_REQUIRE(y_dtype == RN50_F32 || y_dtype == RN50_BF16, RN50_ERR_INVALID, "%s: dtype %d", who, y_dtype);
  RN50_REQUIRE(M > 0 && N > 0 && K > 0, RN50_ERR_INVALID, "%s: non-positive size", who);
  RN50_REQUIRE(K <= kI8MaxK, RN50_ERR_UNSUPPORTED, "%s: K=%d beyond %d, what a 32-bit sum holds", who, K, kI8MaxK);
  RN50_REQUIRE(ceil_div(M, 64) <= 65535 && N <= (1 << 28), RN50_ERR_UNSUPPORTED, "%s: M=%d or N=%d beyond the launch grid", who, M, N);
  RN50_REQUIRE(w && w_scale && y, RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(ldy >= N, RN50_ERR_INVALID, "%s: rows of %d elements %lld apart", who, N, static_cast<long long>(ldy));
  RN50_REQUIRE(aligned16(w), RN50_ERR_ALIGN, "%s: 8-bit rows not 16-byte aligned", who);
  RN50_REQUIRE(aligned_to(w_scale, 4) && aligned_to(bias, 4) && aligned_to(y, y_dtype == RN50_BF16 ? 2 : 4), RN50_ERR_ALIGN,
               "%s: pointer not aligned to an element", who);
  return RN50_OK;
}

static void quant_run(int M, int K, int dtype, const void* x, int64_t ldx, int8_t* q, float* scale, hipStream_t s) {
  const int Kp = static_cast<int>(quant_i8_row_bytes(K));
  const dim3 grid(std::min(M, 1 << 20));
  if (dtype == RN50_BF16)
    RN50_LAUNCH("quant_rows_i8", quant_rows_kernel<uint16_t>, grid, dim3(256), 0, s, static_cast<const uint16_t*>(x), ldx, M, K, Kp, q, scale);
  else
    RN50_LAUNCH("quant_rows_i8", quant_rows_kernel<float>, grid, dim3(256), 0, s, static_cast<const float*>(x), ldx, M, K, Kp, q, scale);
}
static void product_run(int M, int N, int K, const int8_t* q, const float* qs, const int8_t* w, const float* ws, const float* bias, int y_dtype,
                        void* y, int64_t ldy, hipStream_t s) {
  const int Kp = static_cast<int>(quant_i8_row_bytes(K));
  const dim3 grid(ceil_div(N, 64), ceil_div(M, 64));
  if (y_dtype == RN50_BF16)
    RN50_LAUNCH("matmul_i8", matmul_i8_kernel<uint16_t>, grid, dim3(256), 0, s, q, qs, w, ws, bias, static_cast<uint16_t*>(y), ldy, M, N, Kp);
  else
    RN50_LAUNCH("matmul_i8", matmul_i8_kernel<float>, grid, dim3(256), 0, s, q, qs, w, ws, bias, static_cast<float*>(y), ldy, M, N, Kp);
}

}  // namespace rn50

using namespace rn50;

extern "C" size_t quant_i8_row_bytes(int K) { return K < 1 || K > kI8MaxK ? 0 : align_up(static_cast<size_t>(K), 64); }

extern "C" int quant_rows_i8(int M, int K, int dtype, const void* x, int64_t ldx, int8_t* q, float* scale, void* stream) {
  clear_error();
  if (int rc = check_quant("quant_rows_i8", M, K, dtype, x, ldx)) return rc;
  RN50_REQUIRE(q && scale, RN50_ERR_INVALID, "quant_rows_i8: null pointer");
  RN50_REQUIRE(aligned16(q) && aligned_to(scale, 4), RN50_ERR_ALIGN, "quant_rows_i8: 8-bit rows not 16-byte aligned");
  quant_run(M, K, dtype, x, ldx, q, scale, static_cast<hipStream_t>(stream));
  return launch_status("quant_rows_i8");
}

extern "C" int matmul_i8(int M, int N, int K, const int8_t* q, const float* q_scale, const int8_t* w, const float* w_scale, const float* bias,
                         int y_dtype, void* y, int64_t ldy, void* stream) {
  clear_error();
  if (int rc = check_product("matmul_i8", M, N, K, w, w_scale, bias, y_dtype, y, ldy)) return rc;
  RN50_REQUIRE(q && q_scale, RN50_ERR_INVALID, "matmul_i8: null pointer");
  RN50_REQUIRE(aligned16(q) && aligned_to(q_scale, 4), RN50_ERR_ALIGN, "matmul_i8: 8-bit rows not 16-byte aligned");
  product_run(M, N, K, q, q_scale, w, w_scale, bias, y_dtype, y, ldy, static_cast<hipStream_t>(stream));
  return launch_status("matmul_i8");
}

extern "C" size_t fc_i8_workspace_bytes(int M, int K) {
  const size_t row = quant_i8_row_bytes(K);
  return M < 1 || row == 0 ? 0 : align_up(static_cast<size_t>(M) * row, 256) + align_up(static_cast<size_t>(M) * 4, 256);
}

extern "C" int fc_i8_fwd(int M, int N, int K, int x_dtype, const void* x, int64_t ldx, const int8_t* w, const float* w_scale, const float* bias,
                         int y_dtype, void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  if (int rc = check_quant("fc_i8_fwd", M, K, x_dtype, x, ldx)) return rc;
  if (int rc = check_product("fc_i8_fwd", M, N, K, w, w_scale, bias, y_dtype, y, ldy)) return rc;
  const size_t need = fc_i8_workspace_bytes(M, K);
  RN50_REQUIRE(workspace && workspace_bytes >= need, RN50_ERR_WORKSPACE, "fc_i8_fwd: workspace %zu < %zu bytes", workspace_bytes, need);
  RN50_REQUIRE(aligned16(workspace), RN50_ERR_ALIGN, "fc_i8_fwd: pointer not 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  int8_t* q = static_cast<int8_t*>(workspace);
  float* qs = reinterpret_cast<float*>(q + align_up(static_cast<size_t>(M) * quant_i8_row_bytes(K), 256));
  quant_run(M, K, x_dtype, x, ldx, q, qs, s);
  product_run(M, N, K, q, qs, w, w_scale, bias, y_dtype, y, ldy, s);
  return launch_status("fc_i8_fwd");
}

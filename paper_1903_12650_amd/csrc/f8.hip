// Products in 8-bit floating point with a power of two for every 128 numbers of the axis that is summed: matrices quantized along
// their rows and, transposed, along their columns; the products; a linear layer's forward and backward pass.
#include <stdlib.h>

#include <algorithm>
#include <type_traits>

#include "conv_internal.h"
#include "dropout.h"

namespace rn50 {

constexpr int kF8MaxK = 1 << 22;        // 256 rows of it stay inside a buffer descriptor's 32 bits
constexpr uint32_t kF8Floor = 27u << 23;  // the bits of 2^-100: blocks below are quantized as if this were their largest magnitude
constexpr int kFloatBlocks = 128;         // blocks of 128 numbers that one float of an exact sum takes: its roundings
constexpr int64_t kPastBytes = 32 << 20;  // outputs that the L2s would not hold for the next kernel are stored past the caches
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// Scale byte (e + 127) of a block from the bits of its largest magnitude, and 2^-e: with a = 1.m 2^(E - 127), the least e with
// a <= 1.75 * 2^8 (e4m3; 2^15 e5m2) * 2^e.  An infinity's and a NaN's bits are above every number's: byte 127, `finite` false.
template <bool E5>
__device__ __forceinline__ uint32_t f8_scale(uint32_t amax_bits, float* inv, bool* finite) {
  const uint32_t a = max(amax_bits, kF8Floor);
  *finite = a < 0x7f800000u;
  const uint32_t byte = *finite ? (a >> 23) - (E5 ? 15u : 8u) + ((a & 0x7fffffu) > 0x600000u ? 1u : 0u) : 127u;
  *inv = __uint_as_float((254u - byte) << 23);
  return byte;
}
// Four numbers as 8-bit ones, the first in the low byte.
template <bool E5>
__device__ __forceinline__ uint32_t f8_four(float a, float b, float c, float d, bool finite) {
  int w;
  if constexpr (E5) w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false), true);
  else w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
  return finite ? static_cast<uint32_t>(w) : 0x7f7f7f7fu;
}
// Largest of a row of 16 lanes, in all of them.
__device__ __forceinline__ uint32_t max_of_16_lanes(uint32_t v) {
  constexpr int ROR = 0x120;  // row_ror:n
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), ROR + 8, 0xf, 0xf, false)));
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), ROR + 4, 0xf, 0xf, false)));
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), ROR + 2, 0xf, 0xf, false)));
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), ROR + 1, 0xf, 0xf, false)));
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// ------------------------------------------------------------- quantization
struct QuantArgs {
  const void* x;
  int64_t ldx;
  int M, K, tiles_k;
  uint8_t *q, *scale, *qt, *scale_t;
  int Kp, Mp;
  double* sums;  // [row tiles][K]: the columns' sums of each tile of x as it is; or NULL
  DropArgs drop;
};
// A tile of 16 * R rows by 128 columns in registers: thread t holds rows R * (t / 16) .. + R - 1 of the eight columns at 8 * (t % 16), the
// elements of one Philox call a row.  A block along a row is 16 lanes' (DPP), a block along a column the workgroup's (LDS, R = 8).  x is read once for
// both, and for the columns' sums; bound by memory: 8192 x 8192 bf16 both ways 55 us (268 MB, 4.9 TB/s), behind a dropout as much arithmetic as memory
// (8192 x 4096 32 to 37 us, Philox's multiplications 15 of them).
template <typename T, bool E5, int R, bool COLS, bool DROP, bool PAST>
__device__ __forceinline__ void quant_tile(const QuantArgs& a, int tile) {
  constexpr int V = Elem<T>::VEC;
  static_assert(!COLS || R == 8, "a block of 128 rows");
  const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4;
  const int tm = tile / a.tiles_k, tk = tile - tm * a.tiles_k;
  const int m0 = tm * 16 * R + rg * R, k0 = tk * 128 + cg * 8, cols = a.K - k0;
  float f[R][8];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const T* row = static_cast<const T*>(a.x) + static_cast<int64_t>(m0 + i) * a.ldx + k0;
    if (m0 + i < a.M && cols >= 8) {
#pragma unroll
      for (int j = 0; j < 8; j += V) Elem<T>::unpack(load16_any(row + j), f[i] + j);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = m0 + i < a.M && j < cols ? Elem<T>::load(row + j) : 0.f;
    }
  }
  __shared__ uint32_t red[COLS ? 16 : 1][COLS ? 128 : 1];
  __shared__ uint32_t col_scale[COLS ? 128 : 1];
  __shared__ uint4 turned[COLS ? 1024 : 1];
  if (COLS && a.sums) {
    // two columns' sums of a row group are 16 bytes, pair p of thread cg's four in place p ^ (cg / 4): 16 lanes' stores touch all banks
    double2 (*part)[64] = reinterpret_cast<double2 (*)[64]>(turned);
    static_assert(!COLS || sizeof(turned) >= 16 * 64 * sizeof(double2), "the row groups' sums fit");
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      double2 s = make_double2(f[0][2 * p], f[0][2 * p + 1]);
#pragma unroll
      for (int i = 1; i < R; ++i) {
        s.x += f[i][2 * p];
        s.y += f[i][2 * p + 1];
      }
      part[rg][cg * 4 + (p ^ (cg >> 2))] = s;
    }
    __syncthreads();
    if (tid < 128 && tk * 128 + tid < a.K) {
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < 16; ++i) s += reinterpret_cast<const double*>(part[i])[(tid >> 1 ^ tid >> 5) * 2 + (tid & 1)];
      a.sums[static_cast<int64_t>(tm) * a.K + tk * 128 + tid] = s;
    }
    __syncthreads();
  }
  if constexpr (DROP) {
    const uint64_t call = drop_call(a.drop), per_row = static_cast<uint64_t>((a.K + 7) >> 3);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const DropBits bits = drop_bits(a.drop, call, static_cast<uint64_t>(m0 + i) * per_row + static_cast<uint32_t>(k0 >> 3));
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = drop_keeps(a.drop, bits, j) ? f[i][j] * a.drop.factor : 0.f;
    }
  }
  if (a.q) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, magnitude(f[i][j]));
      float inv;
      bool finite;
      const uint32_t byte = f8_scale<E5>(max_of_16_lanes(top), &inv, &finite);
      if (m0 + i >= a.M) continue;  // (a row's 16 lanes together)
      uint2 o = make_uint2(f8_four<E5>(f[i][0] * inv, f[i][1] * inv, f[i][2] * inv, f[i][3] * inv, finite),
                           f8_four<E5>(f[i][4] * inv, f[i][5] * inv, f[i][6] * inv, f[i][7] * inv, finite));
      if (cols < 8) {  // zeros past the last column, in NaN blocks too
        const uint64_t keep = cols <= 0 ? 0 : (1ull << (8 * cols)) - 1;
        o.x &= static_cast<uint32_t>(keep);
        o.y &= static_cast<uint32_t>(keep >> 32);
      }
      uint64_t* to = reinterpret_cast<uint64_t*>(a.q + static_cast<int64_t>(m0 + i) * a.Kp + k0);
      if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(uint64_t, o), to);
      else *to = __builtin_bit_cast(uint64_t, o);
      if (cg == 0) {
        uint8_t* s = a.scale + (static_cast<int64_t>(tk >> 2) * a.M + m0 + i) * 4;
        s[tk & 3] = static_cast<uint8_t>(byte);
        if (tk == a.tiles_k - 1)
          for (int j = (tk & 3) + 1; j < 4; ++j) s[j] = 0;
      }
    }
  }
  if constexpr (COLS) {
    if (!a.qt) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) top = max(top, magnitude(f[i][j]));
      red[rg][cg * 8 + j] = top;
    }
    __syncthreads();
    if (tid < 128) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = max(top, red[i][tid]);
      float inv;
      bool finite;
      const uint32_t byte = f8_scale<E5>(top, &inv, &finite);
      col_scale[tid] = byte | (finite ? 0u : 256u);
      const int k = tk * 128 + tid;
      if (k < a.K) {
        uint8_t* s = a.scale_t + (static_cast<int64_t>(tm >> 2) * a.K + k) * 4;
        s[tm & 3] = static_cast<uint8_t>(byte);
        if (tm == (a.Mp >> 7) - 1)
          for (int j = (tm & 3) + 1; j < 4; ++j) s[j] = 0;
      }
    }
    __syncthreads();
    // Turned through LDS: column c has 16 pieces of 8 bytes, piece r of eight rows in place r ^ (c / 8), so that both sides touch all banks.
    const int rows = a.M - m0;
    const uint64_t keep = rows >= 8 ? ~0ull : rows <= 0 ? 0ull : (1ull << (8 * rows)) - 1;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t s = col_scale[cg * 8 + j];
      const float inv = __uint_as_float((254u - (s & 255u)) << 23);
      const bool finite = s < 256u;
      uint2 o = make_uint2(f8_four<E5>(f[0][j] * inv, f[1][j] * inv, f[2][j] * inv, f[3][j] * inv, finite),
                           f8_four<E5>(f[4][j] * inv, f[5][j] * inv, f[6][j] * inv, f[7][j] * inv, finite));
      o.x &= static_cast<uint32_t>(keep);
      o.y &= static_cast<uint32_t>(keep >> 32);
      reinterpret_cast<uint2*>(turned)[(cg * 8 + j) * 16 + (rg ^ cg)] = o;
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int c = p * 32 + (tid >> 3), piece = tid & 7, g = c >> 3, k = tk * 128 + c;
      Vec16 o;
      o.u = turned[c * 8 + (piece ^ (g >> 1))];
      if (g & 1) o.u = make_uint4(o.u.z, o.u.w, o.u.x, o.u.y);
      uint8_t* to = a.qt + static_cast<int64_t>(k) * a.Mp + tm * 128 + piece * 16;
      if (k < a.K) {
        if constexpr (PAST) store16_any_stream(to, o);
        else store16(to, o);
      }
    }
  }
}

template <typename T, bool E5, int R, bool COLS, bool DROP, bool PAST>
__global__ __launch_bounds__(256) void quant_blocks_kernel(const QuantArgs a) {
  quant_tile<T, E5, R, COLS, DROP, PAST>(a, blockIdx.x);
}
// The columns' part of a tile alone, 32 columns of it: thread t holds rows 2 * (t / 4), + 1 of the eight columns at 8 * (t % 4).
template <typename T, bool E5, bool DROP>
__device__ __forceinline__ void quant_columns(const QuantArgs& a, int tile) {
  constexpr int V = Elem<T>::VEC;
  const int tiles = (a.K + 31) >> 5, tid = threadIdx.x, cg = tid & 3, rg = tid >> 2;
  const int tm = tile / tiles, tk = tile - tm * tiles;
  const int m0 = tm * 128 + rg * 2, k0 = tk * 32 + cg * 8, cols = a.K - k0;
  float f[2][8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const T* row = static_cast<const T*>(a.x) + static_cast<int64_t>(m0 + i) * a.ldx + k0;
    if (m0 + i < a.M && cols >= 8) {
#pragma unroll
      for (int j = 0; j < 8; j += V) Elem<T>::unpack(load16_any(row + j), f[i] + j);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = m0 + i < a.M && j < cols ? Elem<T>::load(row + j) : 0.f;
    }
  }
  __shared__ uint32_t red[64][33];
  __shared__ __align__(16) double part[64][33];
  __shared__ uint32_t col_scale[32];
  uint4* turned = reinterpret_cast<uint4*>(part);  // (behind the sums)
  if (a.sums) {
#pragma unroll
    for (int j = 0; j < 8; ++j) part[rg][cg * 8 + j] = static_cast<double>(f[0][j]) + f[1][j];
  }
  if constexpr (DROP) {
    const uint64_t call = drop_call(a.drop), per_row = static_cast<uint64_t>((a.K + 7) >> 3);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const DropBits bits = drop_bits(a.drop, call, static_cast<uint64_t>(m0 + i) * per_row + static_cast<uint32_t>(k0 >> 3));
#pragma unroll
      for (int j = 0; j < 8; ++j) f[i][j] = drop_keeps(a.drop, bits, j) ? f[i][j] * a.drop.factor : 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) red[rg][cg * 8 + j] = max(magnitude(f[0][j]), magnitude(f[1][j]));
  __syncthreads();
  if ((tid & 63) < 32 && tid < 128) {  // half a wave the largest magnitudes, half of another the sums
    const int c = tid & 31, k = tk * 32 + c;
    if (tid < 32) {
      uint32_t top = 0;
#pragma unroll 16
      for (int i = 0; i < 64; ++i) top = max(top, red[i][c]);
      float inv;
      bool finite;
      const uint32_t byte = f8_scale<E5>(top, &inv, &finite);
      col_scale[c] = byte | (finite ? 0u : 256u);
      if (a.qt && k < a.K) {
        uint8_t* s = a.scale_t + (static_cast<int64_t>(tm >> 2) * a.K + k) * 4;
        s[tm & 3] = static_cast<uint8_t>(byte);
        if (tm == (a.Mp >> 7) - 1)
          for (int j = (tm & 3) + 1; j < 4; ++j) s[j] = 0;
      }
    } else if (a.sums && k < a.K) {
      double s = 0.0;
#pragma unroll 16
      for (int i = 0; i < 64; ++i) s += part[i][c];
      a.sums[static_cast<int64_t>(tm) * a.K + k] = s;
    }
  }
  if (!a.qt) return;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t s = col_scale[cg * 8 + j];
    const float inv = __uint_as_float((254u - (s & 255u)) << 23);
    uint32_t two = f8_four<E5>(f[0][j] * inv, f[1][j] * inv, 0.f, 0.f, s < 256u);
    if (m0 + 1 >= a.M) two &= m0 < a.M ? 0xffu : 0u;  // zeros past the last row, in NaN blocks too
    reinterpret_cast<uint16_t*>(turned)[(cg * 8 + j) * 64 + rg] = static_cast<uint16_t>(two);
  }
  __syncthreads();
  const int k = tk * 32 + (tid >> 3);
  if (k < a.K) *reinterpret_cast<uint4*>(a.qt + static_cast<int64_t>(k) * a.Mp + tm * 128 + (tid & 7) * 16) = turned[tid];
}
// Few tiles: rows and columns by workgroups of their own, 32 rows and 32 columns each, which read x twice but fill the card.
template <typename T, bool E5, bool DROP>
__global__ __launch_bounds__(256) void quant_small_kernel(const QuantArgs a, int row_tiles) {
  if (static_cast<int>(blockIdx.x) < row_tiles) quant_tile<T, E5, 2, false, DROP, false>(a, blockIdx.x);
  else quant_columns<T, E5, DROP>(a, blockIdx.x - row_tiles);
}

// db[n] = the sum of the row tiles' sums, all of it in 64 bits: a gradient's columns all but cancel, and floats over a tile's 128 rows cost three times the
// error (backward pass of 50176 x 1024 -> 256 85.4 -> 86.3 us, of 8192 x 4096 -> 4096 329.6 -> 331.2).  Four threads a column, each every fourth tile in
// order, then the four; the same order whichever kernel has it along (a launch of its own for these few bytes costs 4 us, and with one thread a column 90 us
// at 392 tiles of 256 columns).
struct SumArgs {
  const double* sums;
  int tiles, N;
  float* db;
};
constexpr int kSumColumns = 64;
__device__ __forceinline__ void f8_column_sums(const SumArgs& a, int group) {
  extern __shared__ __align__(16) unsigned char smem[];
  double* red = reinterpret_cast<double*>(smem);
  const int tid = threadIdx.x, part = tid >> 6, n = group * kSumColumns + (tid & 63);
  if (tid < 256) {
    double s = 0.0;
    if (n < a.N) {
#pragma unroll 8
      for (int t = part; t < a.tiles; t += 4) s += a.sums[static_cast<int64_t>(t) * a.N + n];
    }
    red[tid] = s;
  }
  __syncthreads();
  if (tid < 64 && n < a.N) a.db[n] = static_cast<float>((red[tid] + red[64 + tid]) + (red[128 + tid] + red[192 + tid]));
}
__global__ __launch_bounds__(256) void f8_column_sums_kernel(const SumArgs a) { f8_column_sums(a, blockIdx.x); }

// ------------------------------------------------------------------ products
// 16 numbers of a row as bfloat16, times a power of two: exact.
template <bool E5>
__device__ __forceinline__ void f8_to_bf16(i32x4 v, float scale, bf16x8* out) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x2 two;
      if constexpr (E5) two = h ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[i], scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[i], scale, false);
      else two = h ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], scale, false);
      const int at = 4 * i + 2 * h;
      out[at >> 3][at & 7] = two[0];
      out[at >> 3][(at & 7) + 1] = two[1];
    }
}
// Half of a block's power: at the end of float's range q 2^e may be 2^128, past bfloat16's.  Sums of products of both halves are a quarter: kBack puts them right.
__device__ __forceinline__ float half_scale(uint32_t byte) { return __uint_as_float(byte << 23) * 0.5f; }
constexpr float kBack = 4.f;

struct F8Args {
  const uint8_t *a, *w;
  const uint32_t *as, *ws;  // dword [g][row]: four blocks' bytes
  const float* bias;
  void* y;
  int64_t ldy;
  int M, N, Kp, tiles_m, tiles_n;
  int part;       // blocks of the sum a workgroup takes (a multiple of 4; all of them: one part)
  float* partial; // more than one part: float [part][M][N], summed by f8_join_kernel, which has bias, drop and y
  DropArgs drop;  // of y's elements; threshold 0: none
  int groups;     // workgroups of the product; those behind them add up `sum`
  SumArgs sum;
};

// V consecutive columns of row m, from column n (a multiple of V; V divides 8).
template <int V>
__device__ __forceinline__ void drop_columns(const F8Args& a, uint64_t call, int m, int n, float* f) {
  const DropBits bits = drop_bits(a.drop, call, static_cast<uint64_t>(m) * static_cast<uint32_t>((a.N + 7) >> 3) + static_cast<uint32_t>(n >> 3));
#pragma unroll
  for (int j = 0; j < V; ++j) {
    bool keep = drop_keeps(a.drop, bits, j);
    if (V == 4 && (n & 4)) keep = drop_keeps(a.drop, bits, j + 4);
    f[j] = keep ? f[j] * a.drop.factor : 0.f;
  }
}

// A tile of the product by WM x WN waves, each of 32x32 blocks of it.  FAST (bfloat16 results): two 8-bit fragments and their rows' scale bytes go into
// v_mfma_scale_f32_32x32x64_f8f6f4 as they are, the scaling costs nothing.  Of every eight products these matrix cores drop what lies below 2^-13 of the
// largest, 1.2e-5 to 1.6e-5 of a sum's usual size, a hundredth of its rounding to bfloat16: one result in 45 to 80 is rounded to the other side (2.7e-4 of y's
// size between the two), the error against 64 bits is 1.6593e-3 instead of 1.6592e-3 with float sums, which take twice as long (8192^3).  EXACT (float
// results): fragments become bfloat16, times their power of two (exact: 4 of its 8 bits), for v_mfma_f32_32x32x16_bf16, since the 8-bit matrix cores drop bits
// that a float result has.
// Operands go from memory into LDS past the registers, RING stages of 128 numbers a row, a row's 16-byte pieces exchanged so that a fragment's reads touch all
// banks.  What bounds it: large tiles' matrix cores, at the clock that their power leaves (8192^3 bfloat16 397 to 447 us, 2460 to 2770 TFLOP/s, of
// zeros 317; 8192 x 4096 x 4096 into floats 195 to 223, 1230 to 1410); middle ones' conversions and LDS reads beside the matrix cores (1001 x 2047 ->
// 4099 into floats 27 to 29 us, matrix cores busy 35 %); with short sums starts and ends (50176 x 256 -> 1024 bfloat16 37 us: 25 without the sum, 32 without
// the stores).  Four waves of 128x128 421 us where eight of 128x64 take 397; stages of 64 numbers, half lines of memory, 569.
// Tiles go to the XCDs in runs, columns after columns of GROUP row tiles, so that an XCD's L2 sees both operands several times (GROUP 8: 495 us
// to 492 at the time of its trial).
// What a stage's loads are asked for: past the last stage nothing, from the beginning.  A lane's offset is checked against the length less the scalar
// offset, a difference that must not go below 0 (no length behind an offset would leave the answer to how the hardware subtracts).
struct StageRange {
  uint32_t bytes, offset;
};
__host__ __device__ constexpr StageRange stage_range(uint32_t bytes, int st, int stages) {
  return st < stages ? StageRange{bytes, static_cast<uint32_t>(st) * 128u} : StageRange{0, 0};
}
// Lanes ask for `at` of a row, 112 at most, of as many stages as a single row has.
constexpr bool stages_stay_inside(int stages) {
  for (int st = 0; st < stages + 8; ++st) {
    const StageRange r = stage_range(static_cast<uint32_t>(stages) * 128u, st, stages);
    if (r.offset > r.bytes) return false;
    if ((112u + 16u <= r.bytes - r.offset) != (st < stages)) return false;
  }
  return true;
}
static_assert(stages_stay_inside(1) && stages_stay_inside(2) && stages_stay_inside(5) && stages_stay_inside(64), "stages past the sum ask for nothing");

// LDS: RING stages and two groups' scales, where the output is staged afterwards.
template <int BM, int BN, int WM, int WN, int RING>
constexpr int f8_tile_lds() {
  constexpr int loop = RING * (BM + BN) * 128 + 2 * (BM + BN) * 4, output = WM * WN * 32 * (BN / WN + 4) * 4;
  return loop > output ? loop : output;
}
template <typename T, bool E5, bool EXACT, int BM, int BN, int WM, int WN, int RING>
__device__ __forceinline__ void f8_tile_product(const F8Args& a, int group) {
  constexpr int CB = 128, PPR = CB / 16, NT = 64 * WM * WN, RPL = NT / PPR, RA = BM / RPL, RB = BN / RPL, TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr int STAGE = (BM + BN) * CB, SCALES = (BM + BN) * 4;
  static_assert(RA * RPL == BM && RB * RPL == BN && TM >= 1 && TN >= 1 && (RING & (RING - 1)) == 0, "whole passes, whole blocks");
  extern __shared__ __align__(16) unsigned char smem[];  // RING stages, two groups' scales
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int wm = wave % WM, wn = wave / WM;
  constexpr int GROUP = 4;
  const int tiles = a.tiles_m * a.tiles_n, number = xcd_remap(group, a.groups), share = number / tiles, id = number - share * tiles;
  const int per = GROUP * a.tiles_n, g = id / per, r = id - g * per, high = min(GROUP, a.tiles_m - g * GROUP);
  const int m0 = (g * GROUP + r % high) * BM, n0 = r / high * BN;
  const int rows = min(BM, a.M - m0), cols = min(BN, a.N - n0);
  const int first = share * a.part, blocks = min(a.part, (a.Kp >> 7) - first), stages = blocks * (128 / CB);
  const uint32_t first_byte = static_cast<uint32_t>(first) * 128u;
  const rsrc_words rsA = make_rsrc_words(a.a + static_cast<int64_t>(m0) * a.Kp + first_byte, static_cast<uint32_t>(rows) * a.Kp - first_byte);
  const rsrc_words rsB = make_rsrc_words(a.w + static_cast<int64_t>(n0) * a.Kp + first_byte, static_cast<uint32_t>(cols) * a.Kp - first_byte);
  const int slot = tid % PPR, lrow = tid / PPR, piece = slot ^ ((lrow >> 1) & (PPR - 1));
  uint32_t at_a[RA], at_b[RB];
#pragma unroll
  for (int i = 0; i < RA; ++i) at_a[i] = lrow + RPL * i < rows ? static_cast<uint32_t>(lrow + RPL * i) * a.Kp + piece * 16 : kOob;
#pragma unroll
  for (int i = 0; i < RB; ++i) at_b[i] = lrow + RPL * i < cols ? static_cast<uint32_t>(lrow + RPL * i) * a.Kp + piece * 16 : kOob;
  typedef __attribute__((address_space(3))) unsigned char* lds_byte_ptr;
  const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_byte_ptr)smem));
  const uint32_t dst = __builtin_amdgcn_readfirstlane(base + static_cast<uint32_t>(wave) * 1024u);
  constexpr int NL = RA + RB;
  auto load_one = [&](int st, int l) __attribute__((always_inline)) {  // (l known when compiling)
    const uint32_t to = dst + static_cast<uint32_t>(st & (RING - 1)) * STAGE;
    rsrc_words r = l < RA ? rsA : rsB;
    const uint32_t at = l < RA ? at_a[l < RA ? l : 0] : at_b[l < RA ? 0 : l - RA], by = l < RA ? l * (RPL * CB) : BM * CB + (l - RA) * (RPL * CB);
    if constexpr (RING == 2) {  // (nothing past the last stage: the waits are for all loads)
      const uint32_t so = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(st) * CB);
      buffer_load16_to_lds_if(__builtin_amdgcn_readfirstlane(st < stages ? 1 : 0), r, to + by, at, so);
    } else {  // (past the last stage zeros, so that the waits' counts hold)
      const StageRange range = stage_range(static_cast<uint32_t>(r.z), st, stages);
      r.z = static_cast<int>(range.bytes);
      buffer_load16_to_lds(r, to + by, at, __builtin_amdgcn_readfirstlane(range.offset));
    }
  };
  // The scales of a group of four blocks are a dword a row, brought into LDS like the operands: 64 rows of the tile or of its columns a wave,
  // a group ahead, again with every block (branches here would let the compiler move a step's products behind the next barrier).
  constexpr int PARTS = (BM + BN) / 64;
  auto load_scales = [&](int four) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < (PARTS + WM * WN - 1) / (WM * WN); ++i) {
      const int part = __builtin_amdgcn_readfirstlane((i * WM * WN + wave) % PARTS);
      const bool of_a = part < BM / 64;
      const uint32_t* from = of_a ? a.as + static_cast<int64_t>((first >> 2) + four) * a.M + m0 : a.ws + static_cast<int64_t>((first >> 2) + four) * a.N + n0;
      const int there = four * 4 < blocks ? of_a ? rows : cols : 0;
      buffer_load4_to_lds(make_rsrc_words(from, static_cast<uint32_t>(there) * 4u), base + RING * STAGE + static_cast<uint32_t>(four & 1) * SCALES + part * 256,
                          static_cast<uint32_t>((of_a ? part : part - BM / 64) * 64 + lane) * 4u);
    }
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  int frag[CB / 32];
#pragma unroll
  for (int u = 0; u < CB / 32; ++u) frag[u] = (lane & 31) * CB + (((2 * u + (lane >> 5)) ^ ((lane >> 1) & (PPR - 1))) << 4);
  // Fragments a step ahead (FAST: a stage, EXACT: half of one), across stages as well: the last step of a stage is multiplied behind the barrier that frees
  // the stage's buffer, while the next stage's fragments and the loads of the one RING stages on are on their way.
  constexpr bool PIPED = EXACT && TM * TN <= 4;
  constexpr int READS = EXACT ? 1 : 2;
  i32x4 fa[2][READS][TM], fb[2][READS][TN];
  uint32_t sa[TM], sb[TN], next_a[TM], next_b[TN];
  constexpr int SB = 32 * READS, STEPS = 128 / SB;  // bytes of a row a step; steps a block
  constexpr int READ = READS * (TM + TN);
  auto read_one = [&](int block, int step, int n) __attribute__((always_inline)) {  // fragment n of a step, into set step & 1
    const int st = block * (128 / CB) + step * SB / CB, u = n / (TM + TN), f = n % (TM + TN), at = frag[step * SB % CB / 32 + u];
    const unsigned char* t = smem + (st & (RING - 1)) * STAGE + at;
    if (f < TN) fb[step & 1][u][f] = *reinterpret_cast<const i32x4*>(t + (BM + wn * (BN / WN) + f * 32) * CB);
    else fa[step & 1][u][f - TN] = *reinterpret_cast<const i32x4*>(t + (wm * (BM / WM) + (f - TN) * 32) * CB);
  };
  auto read = [&](int block, int step) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < READ; ++n) read_one(block, step, n);
  };
  auto read_scales = [&](int block) __attribute__((always_inline)) {
    const unsigned char* t = smem + RING * STAGE + (block >> 2 & 1) * SCALES + (lane & 31) * 4;
#pragma unroll
    for (int i = 0; i < TM; ++i) next_a[i] = *reinterpret_cast<const uint32_t*>(t + (wm * (BM / WM) + i * 32) * 4);
#pragma unroll
    for (int j = 0; j < TN; ++j) next_b[j] = *reinterpret_cast<const uint32_t*>(t + (BM + wn * (BN / WN) + j * 32) * 4);
  };
  // A step's products; between them, one after the other, the next step's fragments are read and a stage's loads requested: in a bunch
  // they hold the products up, four waves' 16 loads for as long as they take to go out.
  auto multiply = [&](int set, int next_block, int next_step, bool loads, int st) __attribute__((always_inline)) {
    constexpr int SLOTS = (EXACT ? 2 : 1) * TM * TN;
    bf16x8 xa[EXACT ? TM : 1][2], xb[EXACT ? TN : 1][2];
    if constexpr (EXACT) {
#pragma unroll
      for (int j = 0; j < TN; ++j) f8_to_bf16<false>(fb[set][0][j], half_scale(sb[j] & 255u), xb[j]);
#pragma unroll
      for (int i = 0; i < TM; ++i) f8_to_bf16<E5>(fa[set][0][i], half_scale(sa[i] & 255u), xa[i]);
    }
#pragma unroll
    for (int n = 0; n < SLOTS; ++n) {
      const int i = n % (TM * TN) / TN, j = n % TN;
      if constexpr (EXACT) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb[j][n / (TM * TN)], xa[i][n / (TM * TN)], acc[i][j], 0, 0, 0);
      } else {
        const i32x8 va = __builtin_shufflevector(fa[set][0][i], fa[set][READS - 1][i], 0, 1, 2, 3, 4, 5, 6, 7);
        const i32x8 vb = __builtin_shufflevector(fb[set][0][j], fb[set][READS - 1][j], 0, 1, 2, 3, 4, 5, 6, 7);
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(vb, va, acc[i][j], 0, E5 ? 1 : 0, 0, static_cast<int>(sb[j]), 0, static_cast<int>(sa[i]));
      }
#pragma unroll
      for (int r = n * READ / SLOTS; r < (n + 1) * READ / SLOTS; ++r) read_one(next_block, next_step, r);
      if (loads) {
#pragma unroll
        for (int l = n * NL / SLOTS; l < (n + 1) * NL / SLOTS; ++l) load_one(st, l);
      }
    }
    // (the compiler would move every read to where its product waits for it)
#pragma unroll
    for (int n = 0; n < SLOTS; ++n) {
      __builtin_amdgcn_sched_group_barrier(8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(256, (READ + SLOTS - 1) / SLOTS, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  load_scales(0);
  load_scales(1);
#pragma unroll
  for (int st = 0; st < RING; ++st)
#pragma unroll
    for (int l = 0; l < NL; ++l) load_one(st, l);
  if (RING == 2 && stages == 1) wait_loads_then_barrier<0>();  // (there is no second stage whose loads may be on their way)
  else wait_loads_then_barrier<(RING - 1) * NL>();
  if (wm * (BM / WM) >= rows || wn * (BN / WN) >= cols) {  // a wave without rows or columns of its own loads and waits as the others do
    for (int block = 0; block < blocks; ++block) {
      wait_loads_then_barrier<(RING - 2) * NL>();
      load_scales(((block + 1) >> 2) + 1);
#pragma unroll
      for (int l = 0; l < NL; ++l) load_one(block + RING, l);
    }
    wait_loads_then_barrier<0>();
    return;
  }
  read_scales(0);
  read(0, 0);
  if constexpr (PIPED) {
    // Step t: its products, between them the conversion of step t + 1's fragments and the reads of step t + 2's.
    bf16x8 xa[2][TM][2], xb[2][TN][2];
    float fa_scale[TM], fb_scale[TN];
    auto take_scales = [&](int block) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < TM; ++i) fa_scale[i] = half_scale(next_a[i] >> ((block & 3) * 8) & 255u);
#pragma unroll
      for (int j = 0; j < TN; ++j) fb_scale[j] = half_scale(next_b[j] >> ((block & 3) * 8) & 255u);
    };
    auto convert = [&](int set) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < TN; ++j) f8_to_bf16<false>(fb[set][0][j], fb_scale[j], xb[set][j]);
#pragma unroll
      for (int i = 0; i < TM; ++i) f8_to_bf16<E5>(fa[set][0][i], fa_scale[i], xa[set][i]);
    };
    read(0, 1);
    take_scales(0);
    convert(0);
    for (int block = 0; block < blocks; ++block) {
#pragma unroll
      for (int step = 0; step < 4; ++step) {
        if (step == 2) {  // the next stage is there, and everyone has read this one
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          wait_loads_then_barrier<(RING - 2) * NL>();
          read_scales(block + 1);
          load_scales(((block + 1) >> 2) + 1);
        }
        if (step == 3) take_scales(block + 1);
        __builtin_amdgcn_sched_barrier(0);
        constexpr int SLOTS = 2 * TM * TN;
#pragma unroll
        for (int n = 0; n < SLOTS; ++n) {
          const int i = n % (TM * TN) / TN, j = n % TN, h = n / (TM * TN);
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb[step & 1][j][h], xa[step & 1][i][h], acc[i][j], 0, 0, 0);
#pragma unroll
          for (int r = n * READ / SLOTS; r < (n + 1) * READ / SLOTS; ++r) read_one(step < 2 ? block : block + 1, (step + 2) & 3, r);
          if (step == 2) {
#pragma unroll
            for (int l = n * NL / SLOTS; l < (n + 1) * NL / SLOTS; ++l) load_one(block + RING, l);
          }
        }
        convert((step + 1) & 1);
#pragma unroll
        for (int n = 0; n < SLOTS; ++n) {
          __builtin_amdgcn_sched_group_barrier(8, 1, 0);
          __builtin_amdgcn_sched_group_barrier(256, (READ + SLOTS - 1) / SLOTS, 0);
          __builtin_amdgcn_sched_group_barrier(2, 8 * READ / SLOTS, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  } else {
    for (int block = 0; block < blocks; ++block) {
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = next_a[i] >> ((block & 3) * 8);
#pragma unroll
      for (int j = 0; j < TN; ++j) sb[j] = next_b[j] >> ((block & 3) * 8);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int step = 0; step < STEPS; ++step) {
        const int done = (step + 1) * SB;  // bytes of this block whose fragments have been read
        const int next = done < 128 ? block : block + 1, st = block * (128 / CB) + done / CB - 1;
        if (done % CB == 0) {  // the next stage: it is there, and everyone has read this one, whose buffer is loaded anew
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          wait_loads_then_barrier<(RING - 2) * NL>();
          if (done == 128) {
            read_scales(block + 1);
            load_scales(((block + 1) >> 2) + 1);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        multiply(step & 1, next, (step + 1) % STEPS, done % CB == 0, st + RING);  // (behind the last stage: zeros, not used)
      }
    }
  }
  // Output: a wave's 32 rows at a time through LDS (its own part of it), whole rows of the wave's columns from there.
  constexpr int WC = BN / WN, PITCH = WC + 4;  // floats (rows 16 bytes further along the banks)
  static_assert(WM * WN * 32 * PITCH * 4 <= f8_tile_lds<BM, BN, WM, WN, RING>(), "the output stage fits");
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  wait_loads_then_barrier<0>();
  float* mine = reinterpret_cast<float*>(smem) + wave * 32 * PITCH;
  constexpr int V = Elem<T>::VEC, LPR = WC / V, RPP = 64 / LPR;  // lanes a row, rows a pass
  const int col = n0 + wn * WC + lane % LPR * V;
  T* const y = static_cast<T*>(a.y) + (a.partial ? static_cast<int64_t>(share) * a.M * a.N : 0);
  const uint64_t call = a.drop.threshold ? drop_call(a.drop) : 0;
  float b[V];
#pragma unroll
  for (int j = 0; j < V; ++j) b[j] = a.bias && col + j < a.N ? a.bias[col + j] : 0.f;
  auto output = [&](auto past) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          *reinterpret_cast<float4*>(mine + (lane & 31) * PITCH + j * 32 + v * 8 + (lane >> 5) * 4) =
              make_float4(acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]);
      __builtin_amdgcn_wave_barrier();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int p = 0; p < 32 / RPP; ++p) {
        const int row = p * RPP + lane / LPR, m = m0 + wm * (BM / WM) + i * 32 + row;
        if (m < a.M && col < a.N) {
          float f[V];
#pragma unroll
          for (int j = 0; j < V; ++j) f[j] = fmaf(mine[row * PITCH + lane % LPR * V + j], EXACT ? kBack : 1.f, b[j]);
          if (a.drop.threshold) drop_columns<V>(a, call, m, col, f);
          T* to = y + m * a.ldy + col;
          if (col + V <= a.N) {
            Vec16 o;
            Elem<T>::pack(f, o);
            if constexpr (decltype(past)::value) store16_any_stream(to, o);
            else store16_any(to, o);
          } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
              if (col + j < a.N) Elem<T>::store(to + j, f[j]);
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  };
  // (two whole copies: a choice at each store would be merged into one ordinary store)
  if (!a.partial && static_cast<int64_t>(a.M) * a.N * static_cast<int64_t>(sizeof(T)) >= kPastBytes) output(std::true_type{});
  else output(std::false_type{});
}

template <typename T, bool E5, bool EXACT, int BM, int BN, int WM, int WN, int RING>
__global__ __launch_bounds__(64 * WM * WN) void matmul_f8_kernel(const F8Args a) {
  if (static_cast<int>(blockIdx.x) < a.groups) f8_tile_product<T, E5, EXACT, BM, BN, WM, WN, RING>(a, blockIdx.x);
  else f8_column_sums(a.sum, blockIdx.x - a.groups);
}

// Few rows (M <= 16 * MB): the weights go by once, bound by memory; a workgroup owns 16 * CB columns, its waves a part of K each.  A wave's lane has column
// lane % 16 and 32 numbers at 32 * (lane / 16) of a block of 128, straight from memory, U blocks' loads in flight; they meet the rows' (the second operand) in
// v_mfma_scale_f32_16x16x128_f8f6f4, or (EXACT) as bfloat16, times their power of two, in v_mfma_f32_16x16x32_bf16.  The waves' sums are added through LDS, in
// order.  (bfloat16 results from float sums: 64 x 4096 -> 7000 23.4 -> 25.2 us, 8 x 1024 -> 16384 with the quantization 6.2 -> 7.7.)  1 x 2048 -> 1000 with the
// quantization 5.4 us, 40 x 2048 -> 1000 5.9, of them 2 to 3 the launch; 1 x 8192 -> 8192 18, 3.7 TB/s.
// X: the rows are float or bfloat16 and quantized here, block by block as they are needed (a block's 128 numbers are four lanes'): no second launch.
// (The rows' loads beside the weights', U blocks ahead, change nothing: 40 x 2048 -> 1000 6.0 -> 6.4 us, 40 x 8192 -> 8192 34.0 -> 33.5.)
// FOLD (EXACT, sums of which a wave has more than kFloatBlocks blocks): a register takes that many before it is added to the others, in registers that the
// other kernels do without (32 rows' ones have 127 of the 128 that leave a unit two workgroups; with the sums kept in LDS and 128 registers 24 x 4096 -> 7000
// took 14.4 us instead of 14.1).
constexpr int kFewThreads = 512, kFewWaves = kFewThreads / 64;
constexpr int kFewLong = kFewWaves * kFloatBlocks * 128;
struct F8FewArgs {
  F8Args p;
  const void* x;
  int64_t ldx;
  int K;
};
__device__ __forceinline__ uint32_t scale_byte(const uint32_t* scales, int rows, int row, int block) {
  return reinterpret_cast<const uint8_t*>(scales)[(static_cast<int64_t>(block >> 2) * rows + row) * 4 + (block & 3)];
}
template <typename T, bool E5, bool EXACT, int MB, int CB, typename X, bool FOLD = false>
__device__ __forceinline__ void f8_few_product(const F8FewArgs& a, int group) {
  constexpr bool FUSED = !std::is_void<X>::value;
  constexpr int U = FUSED || CB > 1 ? 2 : 4;
  __shared__ float red[kFewWaves][MB][256];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, sub = lane >> 4;
  const int n0 = group * (16 * CB), M = a.p.M, N = a.p.N, Kp = a.p.Kp;
  const int blocks = Kp >> 7, from = blocks * wave / kFewWaves, to = blocks * (wave + 1) / kFewWaves;
  int col[CB];
  i32x4 fw[U][CB][2];
  uint32_t sw[U][CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) col[c] = min(n0 + c * 16 + (lane & 15), N - 1);
  auto load_w = [&](int u, int k) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      const uint8_t* w = a.p.w + static_cast<int64_t>(col[c]) * Kp + static_cast<int64_t>(k) * 128 + 32 * sub;
      fw[u][c][0] = *reinterpret_cast<const i32x4*>(w);
      fw[u][c][1] = *reinterpret_cast<const i32x4*>(w + 16);
      sw[u][c] = scale_byte(a.p.ws, N, col[c], k);
    }
  };
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (from + u < to) load_w(u, from + u);
  int row[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) row[b] = min(b * 16 + (lane & 15), M - 1);
  f32x4 acc[CB][MB];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[c][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  f32x4 folded[FOLD ? CB : 1][MB];
  if constexpr (FOLD) {
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int b = 0; b < MB; ++b) folded[c][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto fold = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        folded[c][b] += acc[c][b];
        acc[c][b] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
  };
  for (int s = from; s < to; s += U) {
    if constexpr (FOLD) {
      if (((s - from) & (kFloatBlocks - 1)) == 0) fold();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = s + u;
      if (k >= to) break;
      bf16x8 w[EXACT ? CB : 1][4];
      i32x8 w8[EXACT ? 1 : CB];
      uint32_t scale_w[CB];
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        scale_w[c] = sw[u][c];
        if constexpr (EXACT) {
          f8_to_bf16<false>(fw[u][c][0], half_scale(sw[u][c]), w[c]);
          f8_to_bf16<false>(fw[u][c][1], half_scale(sw[u][c]), w[c] + 2);
        } else {
          w8[c] = __builtin_shufflevector(fw[u][c][0], fw[u][c][1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
      }
      if (k + U < to) load_w(u, k + U);
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        i32x4 q[2];
        uint32_t byte;
        if constexpr (FUSED) {
          constexpr int V = Elem<X>::VEC;
          float f[32];
          const int at = k * 128 + 32 * sub;
          const X* x = static_cast<const X*>(a.x) + row[b] * a.ldx + at;
          if (at + 32 <= a.K) {
#pragma unroll
            for (int j = 0; j < 32; j += V) Elem<X>::unpack(load16_any(x + j), f + j);
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) f[j] = at + j < a.K ? Elem<X>::load(x + j) : 0.f;
          }
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < 32; ++j) top = max(top, magnitude(f[j]));
          top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 16, 64)));
          top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32, 64)));
          float inv;
          bool finite;
          byte = f8_scale<E5>(top, &inv, &finite);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            q[j >> 2][j & 3] = static_cast<int>(f8_four<E5>(f[4 * j] * inv, f[4 * j + 1] * inv, f[4 * j + 2] * inv, f[4 * j + 3] * inv, finite));
        } else {
          const uint8_t* x = a.p.a + static_cast<int64_t>(row[b]) * Kp + static_cast<int64_t>(k) * 128 + 32 * sub;
          q[0] = *reinterpret_cast<const i32x4*>(x);
          q[1] = *reinterpret_cast<const i32x4*>(x + 16);
          byte = scale_byte(a.p.as, M, row[b], k);
        }
        if constexpr (EXACT) {
          bf16x8 v[4];
          f8_to_bf16<E5>(q[0], half_scale(byte), v);
          f8_to_bf16<E5>(q[1], half_scale(byte), v + 2);
#pragma unroll
          for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int h = 0; h < 4; ++h) acc[c][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[c][h], v[h], acc[c][b], 0, 0, 0);
        } else {
          const i32x8 v = __builtin_shufflevector(q[0], q[1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
          for (int c = 0; c < CB; ++c)
            acc[c][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8[c], v, acc[c][b], 0, E5 ? 1 : 0, 0, static_cast<int>(scale_w[c]), 0, static_cast<int>(byte));
        }
      }
    }
  }
  if constexpr (FOLD) {
    fold();
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
      for (int b = 0; b < MB; ++b) acc[c][b] = folded[c][b];
  }
  const uint64_t call = a.p.drop.threshold ? drop_call(a.p.drop) : 0;
  // column 4 * (lane / 16) + i of the 16, row lane % 16
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    if (c) __syncthreads();  // (`red` has been read)
#pragma unroll
    for (int b = 0; b < MB; ++b) *reinterpret_cast<f32x4*>(&red[wave][b][(lane & 15) * 16 + 4 * sub]) = acc[c][b];
    __syncthreads();
    for (int e = tid; e < MB * 256; e += kFewThreads) {
      const int b = e >> 8, m = b * 16 + ((e >> 4) & 15), n = n0 + c * 16 + (e & 15);
      if (m < M && n < N) {
        float y = a.p.bias ? a.p.bias[n] : 0.f, sum = 0.f;
#pragma unroll
        for (int v = 0; v < kFewWaves; ++v) sum += red[v][b][e & 255];
        y = fmaf(sum, EXACT ? kBack : 1.f, y);
        if (a.p.drop.threshold) {
          const DropBits bits = drop_bits(a.p.drop, call, static_cast<uint64_t>(m) * static_cast<uint32_t>((N + 7) >> 3) + static_cast<uint32_t>(n >> 3));
          y = drop_keeps_at(a.p.drop, bits, n & 7) ? y * a.p.drop.factor : 0.f;
        }
        Elem<T>::store(static_cast<T*>(a.p.y) + m * a.p.ldy + n, y);
      }
    }
  }
}

template <typename T, bool E5, int MB, int CB, typename X, bool FOLD>
__global__ __launch_bounds__(kFewThreads) void matmul_f8_few_kernel(const F8FewArgs a) {
  f8_few_product<T, E5, sizeof(T) == 4, MB, CB, X, FOLD>(a, blockIdx.x);
}
// The two products of a backward pass of few rows in one launch: the input's gradient by the first workgroups, the weights' (a sum of one
// block) by tiles, and the bias's behind them.
template <typename T, bool E5, int MB>
__global__ __launch_bounds__(kFewThreads) void f8_few_backward_kernel(const F8FewArgs x, const F8Args w) {
  const int group = static_cast<int>(blockIdx.x) - x.p.groups;
  if (group < 0) f8_few_product<T, E5, sizeof(T) == 4, MB, 1, void>(x, blockIdx.x);
  else if (group < w.groups) f8_tile_product<float, E5, true, 128, 128, 4, 2, 2>(w, group);
  else f8_column_sums(w.sum, group - w.groups);
}

// The parts of sums that were split, in order, with what the products' output stage has: read once from the caches, 4.5 us for 14 parts of 256 x 1024.
template <typename T>
__global__ __launch_bounds__(256) void f8_join_kernel(const F8Args a, int parts) {
  constexpr int V = Elem<T>::VEC;
  const uint64_t call = a.drop.threshold ? drop_call(a.drop) : 0;
  const int per_row = (a.N + V - 1) / V;
  const int64_t items = static_cast<int64_t>(a.M) * per_row, plane = static_cast<int64_t>(a.M) * a.N;
  for (int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; e < items; e += static_cast<int64_t>(gridDim.x) * 256) {
    const int m = static_cast<int>(e / per_row), n = static_cast<int>(e - static_cast<int64_t>(m) * per_row) * V;
    const float* p = a.partial + static_cast<int64_t>(m) * a.N + n;
    float f[V];
    T* to = static_cast<T*>(a.y) + m * a.ldy + n;
    if (n + V <= a.N) {
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = 0.f;
#pragma unroll 4
      for (int s = 0; s < parts; ++s) {
        float g[V];
#pragma unroll
        for (int j = 0; j < V; j += 4) Elem<float>::unpack(load16_any(p + s * plane + j), g + j);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] += g[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        f[j] = 0.f;
        for (int s = 0; s < parts && n + j < a.N; ++s) f[j] += p[s * plane + j];
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] += a.bias && n + j < a.N ? a.bias[n + j] : 0.f;
    if (a.drop.threshold) drop_columns<V>(a, call, m, n, f);
    if (n + V <= a.N) {
      Vec16 o;
      Elem<T>::pack(f, o);
      store16_any(to, o);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (n + j < a.N) Elem<T>::store(to + j, f[j]);
    }
  }
}

// ------------------------------------------------------------------- launches
static int sum_groups(const SumArgs& a) { return a.db ? static_cast<int>(ceil_div(a.N, kSumColumns)) : 0; }
static void sum_columns(const SumArgs& a, hipStream_t s) {
  if (a.db) RN50_LAUNCH("quant_blocks_f8", f8_column_sums_kernel, dim3(static_cast<unsigned>(sum_groups(a))), dim3(256), 256 * sizeof(double), s, a);
}
template <typename T, bool E5, bool EXACT, int BM, int BN, int WM, int WN, int RING>
static void f8_tile(F8Args a, int parts, hipStream_t s) {
  constexpr int lds = f8_tile_lds<BM, BN, WM, WN, RING>();
  a.tiles_m = static_cast<int>(ceil_div(a.M, BM));
  a.tiles_n = static_cast<int>(ceil_div(a.N, BN));
  const auto kernel = matmul_f8_kernel<T, E5, EXACT, BM, BN, WM, WN, RING>;
  allow_big_lds(kernel, lds);
  a.groups = a.tiles_m * a.tiles_n * parts;
  RN50_LAUNCH("matmul_f8", kernel, dim3(static_cast<unsigned>(a.groups + sum_groups(a.sum))), dim3(64 * WM * WN), lds, s, a);
}
// How a sum of K numbers is split over workgroups: `count` parts of `part` blocks each (the last may have fewer).
struct F8Parts {
  int count, part;
};
constexpr int kFewRows = 64;
static F8Parts f8_parts(int M, int N, int K, bool exact) {
  const int blocks = static_cast<int>(ceil_div(K, 128));
  const int64_t tiles = ceil_div(M, 128) * ceil_div(N, 128);
  int64_t n = 1;
  if (M > kFewRows) {
    // Where tiles are few and sums long, so that both cover the card; the parts cost a second launch (parts, one 64x64 or 128x64 tile a sum; us by sums of 2048,
    // 4096, 6200, 8192, 11000): float 300 -> 500 (12 tiles) 11.4, 11.9, 13.9, 15.4, 17.8 and 11.1, 18.4, 26.0, 32.7, 42.6, 500 -> 1000 (32) 13.0, 17.0,
    // 22.6, 23.8, 26.1 and 11.3, 18.6, 26.2, 33.0, 42.8, 1000 -> 1000 (64) 17.2, 24.0, 28.8, 28.4, 34.5 and 11.7, 18.9, 27.0, 33.3, 43.3, 1024 -> 2000
    // (128) 25.1, 29.6, 39.3, 43.1, 53.1 and 15.9, 25.6, 35.8, 44.9, 58.6; bfloat16 12 tiles 11.2, 12.0, 13.7, 16.0, 17.0 and 8.2, 12.5, 17.3, 21.3, 27.3,
    // 32 11.7, 14.9, 19.7, 21.3, 22.3 and 8.3, 12.5, 17.2, 21.3, 27.2, 128 21.5, 23.2, 26.9, 29.1, 34.6 and 10.6, 16.4, 22.1, 27.7, 34.9.
    const int least = exact ? (tiles <= 32 ? 32 : 64) : (tiles <= 16 ? 32 : 80);
    if (tiles <= 128 && blocks >= least) n = std::min<int64_t>(256 / tiles, blocks / 8);
    // (for the floats' roundings; up to 16 parts, since each is a matrix of its own)
    if (exact) n = std::max(n, std::min<int64_t>(16, ceil_div(blocks, kFloatBlocks)));
    if (tiles * n > (1 << 20)) n = 1;
  }
  const int part = static_cast<int>(align_up(static_cast<size_t>(ceil_div(blocks, n)), 4));
  return F8Parts{static_cast<int>(ceil_div(blocks, part)), part};
}
static size_t f8_partial_bytes(int M, int N, int K, int y_dtype) {  // (float results: as many parts as others or more, whatever the tiles)
  const F8Parts p = f8_parts(M, N, K, y_dtype != RN50_BF16);
  return p.count > 1 ? align_up(static_cast<size_t>(p.count) * M * N * 4, 256) : 0;
}
template <typename T, bool E5, bool EXACT>
static void f8_tiles(const F8Args& a, int parts, hipStream_t s) {
#ifdef RN50_TUNING  // tuning builds only: RN50_F8_TILE=tile
  if (const char* e = getenv("RN50_F8_TILE")) {
    switch (atoi(e)) {
      case 256: return f8_tile<T, E5, EXACT, 256, 256, 2, 4, 2>(a, parts, s);
      case 1288: return f8_tile<T, E5, EXACT, 128, 128, 4, 2, 2>(a, parts, s);
      case 1284: return f8_tile<T, E5, EXACT, 128, 128, 2, 2, 4>(a, parts, s);
      case 128644: return f8_tile<T, E5, EXACT, 128, 64, 2, 2, 4>(a, parts, s);
      case 128642: return f8_tile<T, E5, EXACT, 128, 64, 2, 2, 2>(a, parts, s);
      case 642: return f8_tile<T, E5, EXACT, 64, 64, 2, 2, 2>(a, parts, s);
      case 644: return f8_tile<T, E5, EXACT, 64, 64, 2, 2, 4>(a, parts, s);
    }
  }
#endif
  // The largest tile of which there are enough for the 256 compute units, us (256x256, 128x128 by eight waves, by four with four buffers, 128x64, 64x64 with four;
  // bfloat16 / float): 4096^3 59, 70, -, -, - / 105, 124, 135, 181, 189; 1001 x 2047 -> 4099 (68, 264, 264, 520, 1040 tiles) 26, 19, 25, 27, 24 /
  // 48, 31, 38, 41, 34; 4096 x 4096 -> 1024 (64, 256, 256, 512, 1024) 42, 25, 22, 30, 33 / 84, 37, 38, 47, 51; 512 x 4096 -> 4096 (32, 128, 128, 256, 512)
  // 42, 24, 19, 16.5, 18 / 83, 32, 32, 25, 26; 1000 x 2048 -> 1000 (16, 64, 64, 128, 256) 25, 14, 12, 10, 8 / 46, 18, 20, 14, 12.
  // The 256x256 one leaves a unit a single workgroup, so only where its last round is full enough, with short sums fuller (256x256, 128x128): 50176 ->
  // 1024 by 784 tiles, sums of 256 39.5, 37.3 / 63, 55, of 768 60, 64 / 104, 98; 20000 -> 2000 by 632, 256 41, 37 / 52, 45.5, 1024 63, 64 / 95, 95;
  // 8192 -> 4096 by 512, 256 21, 26 / 36, 37; 8192 -> 8192 by 1024, 128 - / 74, 47.
  // With more than one and up to one and a half 128x128 tiles a unit units that have two end last: 128x64 ones with two buffers, three a unit, all in one round
  // (128x128, 128x64; bfloat16 / float): 1001 x 2047 -> 4099 by 264, 520 20.2, 18.8 / 31.9, 29.0, x 512 10.3, 9.1 / 14.5, 13.0, x 8192 60, 57 / 103, 93;
  // 2048 -> 2816 by 352, 704, x 512 10.5, 9.5 / 15.2, 14.2, x 8192 61.6, 62.1 / 109, 104; 2000 -> 4000 by 512, 1008, x 1000 15.9, 18.5 / 23.9, 26.0.
  // Four buffers pay with long sums a workgroup only.  256 tiles, 128x128 by eight waves and two buffers, by four and four, sums of 256, 1024, 4096, 8192:
  // 6.6, 10.7, 26.6, 47.7 and 7.7, 10.7, 22.3, 37.3 / 9.2, 15.2, 37.1, 67 and 10.7, 16.1, 36.9, 64.  1024 -> 2000 by 512 64x64 with two buffers, by 256
  // 128x64 with four, sums of 256, 512, 1024: 5.3, 6.0, 8.1 and 5.8, 6.5, 7.9 / 6.7, 7.9, 10.7 and 7.5, 8.4, 10.9; 300 -> 500 64x64, two and
  // four: 4.4, 4.8, 6.1 and 4.6, 5.0, 6.2 / 4.9, 5.8, 7.7 and 5.0, 5.9, 7.7.
  auto tiles = [&](int bm, int bn) { return ceil_div(a.M, bm) * ceil_div(a.N, bn) * parts; };
  const int64_t large = tiles(256, 256), places = ceil_div(large, 256) * 256;
  if (large > 128 && !(EXACT && a.Kp <= 256) && (large <= 256 || large * 10 >= places * (a.Kp <= 1024 ? 9 : 8))) f8_tile<T, E5, EXACT, 256, 256, 2, 4, 2>(a, parts, s);
  else if (tiles(128, 128) > 256 && tiles(128, 64) <= 768) f8_tile<T, E5, EXACT, 128, 64, 2, 2, 2>(a, parts, s);
  else if (tiles(128, 128) > 256) f8_tile<T, E5, EXACT, 128, 128, 4, 2, 2>(a, parts, s);
  else if (tiles(128, 128) > 128 && a.part <= (EXACT ? 32 : 8)) f8_tile<T, E5, EXACT, 128, 128, 4, 2, 2>(a, parts, s);
  else if (tiles(128, 128) > 128) f8_tile<T, E5, EXACT, 128, 128, 2, 2, 4>(a, parts, s);
  else if (a.part <= 4) f8_tile<T, E5, EXACT, 64, 64, 2, 2, 2>(a, parts, s);
  else if (tiles(128, 64) > 128) f8_tile<T, E5, EXACT, 128, 64, 2, 2, 4>(a, parts, s);
  else f8_tile<T, E5, EXACT, 64, 64, 2, 2, 4>(a, parts, s);
}
template <typename T, bool E5, int MB, int CB, typename X>
static void f8_few_columns(const F8FewArgs& a, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(ceil_div(a.p.N, 16 * CB)));
  if (sizeof(T) == 4 && a.p.Kp > kFewLong) RN50_LAUNCH("matmul_f8", (matmul_f8_few_kernel<T, E5, MB, CB, X, sizeof(T) == 4>), grid, dim3(kFewThreads), 0, s, a);
  else RN50_LAUNCH("matmul_f8", (matmul_f8_few_kernel<T, E5, MB, CB, X, false>), grid, dim3(kFewThreads), 0, s, a);
}
template <typename T, bool E5, int MB, typename X>
static void f8_few(const F8FewArgs& a, hipStream_t s) {
  // 32 columns a workgroup, which read and convert (or quantize) the rows half as often, where enough workgroups are left: 64 x 8192 -> 8192 44 -> 29 us,
  // 64 x 1024 -> 16384 17 -> 12, 16 x 8192 -> 8192 with quantization 27 -> 21, 1 x 8192 -> 8192 20 -> 18; 40 x 4096 -> 4096 10.7 -> 13.
  if (a.p.N >= 8192) f8_few_columns<T, E5, MB, 2, X>(a, s);
  else f8_few_columns<T, E5, MB, 1, X>(a, s);
}
template <typename T, bool E5, bool EXACT>
static void f8_product(F8Args a, int K, void* partial, hipStream_t s) {
#ifdef RN50_TUNING
  const bool few = a.M <= kFewRows && !getenv("RN50_F8_TILE");
#else
  const bool few = a.M <= kFewRows;
#endif
  if (few) {
    const F8FewArgs f{a, nullptr, 0, 0};
    if (a.M <= 16) f8_few<T, E5, 1, void>(f, s);
    else if (a.M <= 32) f8_few<T, E5, 2, void>(f, s);
    else if (a.M <= 48) f8_few<T, E5, 3, void>(f, s);
    else f8_few<T, E5, 4, void>(f, s);
    return sum_columns(a.sum, s);
  }
  F8Parts parts = f8_parts(a.M, a.N, K, EXACT);
#ifdef RN50_TUNING
  if (getenv("RN50_F8_TILE")) parts = F8Parts{1, a.Kp >> 7};
#endif
  if (parts.count == 1) {
    a.part = a.Kp >> 7;
    return f8_tiles<T, E5, EXACT>(a, 1, s);
  }
  F8Args p = a;  // the parts' sums, then all of them with the output stage's work
  p.part = parts.part;
  p.partial = static_cast<float*>(partial);
  p.y = partial;
  p.ldy = a.N;
  p.bias = nullptr;
  p.drop = drop_args(nullptr);
  f8_tiles<float, E5, EXACT>(p, parts.count, s);
  a.partial = p.partial;
  const int64_t items = static_cast<int64_t>(a.M) * ceil_div(a.N, Elem<T>::VEC);
  RN50_LAUNCH("matmul_f8", f8_join_kernel<T>, dim3(static_cast<unsigned>(std::min<int64_t>(ceil_div(items, 256), 1 << 16))), dim3(256), 0, s, a, parts.count);
}
static void f8_run(int a_format, int y_dtype, const F8Args& a, int K, void* partial, hipStream_t s) {
  if (y_dtype == RN50_BF16 && a_format == RN50_E5M2) f8_product<uint16_t, true, false>(a, K, partial, s);
  else if (y_dtype == RN50_BF16) f8_product<uint16_t, false, false>(a, K, partial, s);
  else if (a_format == RN50_E5M2) f8_product<float, true, true>(a, K, partial, s);
  else f8_product<float, false, true>(a, K, partial, s);
}

// Both products of a backward pass in one launch: few rows (whose sum into the weights is one block), more outputs than the few rows' kernel would take, and
// an input's gradient that leaves room on the card beside the weights'.  One launch, two (M x K -> N, us): 40 x 2048 -> 1000 12.3, 15.8, 40 x 2048 ->
// 2048 17.5, 21.0, 64 x 1024 -> 16384 48, 63, 8 x 4096 -> 8192 42, 45; 40 x 4096 -> 2048 22.9, 20.4, 40 x 4096 -> 4096 38, 31, 40 x 8192 -> 8192 122, 81.
static bool f8_few_backward_fits(int M, int N, int K) { return M <= kFewRows && N > kFewRows && N <= kFewLong && (M <= 16 || K <= 2048); }
template <typename T, bool E5>
static void f8_few_backward(F8Args x, F8Args w, hipStream_t s) {
  constexpr int lds = f8_tile_lds<128, 128, 4, 2, 2>();
  x.groups = static_cast<int>(ceil_div(x.N, 16));
  w.tiles_m = static_cast<int>(ceil_div(w.M, 128));
  w.tiles_n = static_cast<int>(ceil_div(w.N, 128));
  w.groups = w.tiles_m * w.tiles_n;
  w.part = w.Kp >> 7;
  const F8FewArgs f{x, nullptr, 0, 0};
  const dim3 grid(static_cast<unsigned>(x.groups + w.groups + sum_groups(w.sum)));
#define FEW_BACKWARD(MB)                                                                                                  \
  do {                                                                                                                    \
    allow_big_lds(f8_few_backward_kernel<T, E5, MB>, lds);                                                                \
    RN50_LAUNCH("matmul_f8", (f8_few_backward_kernel<T, E5, MB>), grid, dim3(kFewThreads), lds, s, f, w);                 \
  } while (0)
  if (x.M <= 16) FEW_BACKWARD(1);
  else if (x.M <= 48) FEW_BACKWARD(3);
  else FEW_BACKWARD(4);
#undef FEW_BACKWARD
}
// Whether fc_f8_fwd takes its rows as they are.  Two launches -> one: 1 x 2048 -> 1000 7.8 -> 5.0 us, 8 x 4096 -> 4096 10.4 -> 8.2, 16 x 8192 -> 8192 20.6 -> 20.6
// (every workgroup quantizes the rows).
static bool f8_fused(int M) { return M <= 16; }

template <typename T, bool E5, bool DROP>
static void quant_launch(QuantArgs a, bool past, hipStream_t s) {
  const bool cols = a.qt || a.sums;
  // (us, by tiles and by rows and columns apart: 40 x 1000 float 6.8, 4.5, 1001 x 2047 float 7.0, 5.0, 2048 x 2048 bf16 7.1, 5.9, 4096 x 2048 9.5, 12.8)
  if (cols && ceil_div(a.M, 128) * a.tiles_k <= 256) {
    const int row_tiles = a.q ? static_cast<int>(ceil_div(a.M, 32) * a.tiles_k) : 0;
    const unsigned small = static_cast<unsigned>(row_tiles + ceil_div(a.M, 128) * ceil_div(a.K, 32));
    RN50_LAUNCH("quant_blocks_f8", (quant_small_kernel<T, E5, DROP>), dim3(small), dim3(256), 0, s, a, row_tiles);
    return;
  }
  // Stored past the caches where no product follows at once: both ways of 8192 x 8192 bf16 62 -> 58 us, of 8192 x 4096 31 -> 24, 8192 x 8192 alone 37 -> 35; in front of a
  // product they cost more than they save (50176 x 1024 -> 256 backward 89 -> 103).
  const unsigned grid = static_cast<unsigned>(ceil_div(a.M, cols ? 128 : 32) * a.tiles_k);
#define QUANT(R, COLS, PAST) RN50_LAUNCH("quant_blocks_f8", (quant_blocks_kernel<T, E5, R, COLS, DROP, PAST>), dim3(grid), dim3(256), 0, s, a)
  if (cols && past) QUANT(8, true, true);
  else if (cols) QUANT(8, true, false);
  else if (past) QUANT(2, false, true);
  else QUANT(2, false, false);
#undef QUANT
}
template <typename T>
static void quant_typed(const QuantArgs& a, int format, bool past, hipStream_t s) {
  if (format == RN50_E5M2) {
    if (a.drop.threshold) quant_launch<T, true, true>(a, past, s);
    else quant_launch<T, true, false>(a, past, s);
  } else {
    if (a.drop.threshold) quant_launch<T, false, true>(a, past, s);
    else quant_launch<T, false, false>(a, past, s);
  }
}
static void quant_run(int M, int K, int dtype, const void* x, int64_t ldx, const rn50_dropout* drop, int format, uint8_t* q, uint8_t* scale,
                      uint8_t* qt, uint8_t* scale_t, double* sums, bool past, hipStream_t s) {
  const QuantArgs a{x, ldx, M, K, static_cast<int>(ceil_div(K, 128)), q, scale, qt, scale_t, static_cast<int>(quant_f8_row_bytes(K)),
                    static_cast<int>(quant_f8_row_bytes(M)), sums, drop_args(drop)};
  if (dtype == RN50_BF16) quant_typed<uint16_t>(a, format, past, s);
  else quant_typed<float>(a, format, past, s);
}

// --------------------------------------------------------------------- checks
static int check_matrix(const char* who, int M, int K, int dtype, const void* x, int64_t ldx) {
  RN50_REQUIRE(dtype == RN50_F32 || dtype == RN50_BF16, RN50_ERR_INVALID, "%s: dtype %d", who, dtype);
  RN50_REQUIRE(M > 0 && K > 0, RN50_ERR_INVALID, "%s: non-positive size", who);
  RN50_REQUIRE(x, RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(ldx >= K, RN50_ERR_INVALID, "%s: rows of %d elements %lld apart", who, K, static_cast<long long>(ldx));
  RN50_REQUIRE(aligned_to(x, dtype == RN50_BF16 ? 2 : 4), RN50_ERR_ALIGN, "%s: pointer not aligned to an element", who);
  return RN50_OK;
}
static int check_quantized(const char* who, const void* q, const void* scale) {
  RN50_REQUIRE(q && scale, RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(aligned16(q) && aligned16(scale), RN50_ERR_ALIGN, "%s: 8-bit matrix or its scales not 16-byte aligned", who);
  return RN50_OK;
}
static int check_format(const char* who, int format) {
  RN50_REQUIRE(format == RN50_E4M3 || format == RN50_E5M2, RN50_ERR_INVALID, "%s: format %d", who, format);
  return RN50_OK;
}
static int check_sum(const char* who, int K) {
  RN50_REQUIRE(K <= kF8MaxK, RN50_ERR_UNSUPPORTED, "%s: sums of %d numbers, more than %d", who, K, kF8MaxK);
  return RN50_OK;
}
static int check_tiles(const char* who, int M, int N, int rows, int cols) {
  RN50_REQUIRE(ceil_div(M, rows) * ceil_div(N, cols) <= (1 << 22), RN50_ERR_UNSUPPORTED, "%s: %d by %d beyond the launch grid", who, M, N);
  return RN50_OK;
}
static int check_product_size(const char* who, int M, int N) {
  if (int rc = check_tiles(who, M, N, 64, 64)) return rc;
  RN50_REQUIRE(N <= (1 << 26), RN50_ERR_UNSUPPORTED, "%s: %d columns beyond the launch grid", who, N);
  return RN50_OK;
}
static int check_workspace(const char* who, const void* workspace, size_t bytes, size_t need) {
  if (need == 0) return RN50_OK;
  RN50_REQUIRE(workspace && bytes >= need, RN50_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, bytes, need);
  RN50_REQUIRE(aligned16(workspace), RN50_ERR_ALIGN, "%s: pointer not 16-byte aligned", who);
  return RN50_OK;
}

// A workspace's parts, one behind the other.
struct Parts {
  uint8_t* p;
  size_t used = 0;
  template <typename T = uint8_t>
  T* take(size_t bytes) {
    uint8_t* at = p ? p + used : nullptr;
    used += align_up(bytes, 256);
    return reinterpret_cast<T*>(at);
  }
};
static const uint32_t* words(const uint8_t* scale) { return reinterpret_cast<const uint32_t*>(scale); }
static F8Args product_args(int M, int N, int K, const uint8_t* a, const uint8_t* as, const uint8_t* w, const uint8_t* ws, const float* bias, void* y,
                           int64_t ldy, const rn50_dropout* drop) {
  return F8Args{a, w, words(as), words(ws), bias, y, ldy, M, N, static_cast<int>(quant_f8_row_bytes(K)), 0, 0, 0, nullptr, drop_args(drop), 0, {}};
}

}  // namespace rn50

using namespace rn50;

extern "C" size_t quant_f8_row_bytes(int K) { return K < 1 || K > kF8MaxK ? 0 : align_up(static_cast<size_t>(K), 128); }
extern "C" size_t quant_f8_scale_bytes(int rows, int K) {
  return rows < 1 || K < 1 || K > kF8MaxK ? 0 : static_cast<size_t>(ceil_div(K, 512)) * static_cast<size_t>(rows) * 4;
}

extern "C" int quant_blocks_f8(int M, int K, int dtype, const void* x, int64_t ldx, const rn50_dropout* dropout, int format, uint8_t* q,
                               uint8_t* scale, uint8_t* qt, uint8_t* scale_t, void* stream) {
  const char* who = "quant_blocks_f8";
  clear_error();
  if (int rc = check_matrix(who, M, K, dtype, x, ldx)) return rc;
  if (int rc = check_format(who, format)) return rc;
  if (int rc = check_dropout(who, dropout)) return rc;
  RN50_REQUIRE(q || qt, RN50_ERR_INVALID, "%s: null pointer", who);
  if (q || scale)
    if (int rc = check_quantized(who, q, scale)) return rc;
  if (qt || scale_t)
    if (int rc = check_quantized(who, qt, scale_t)) return rc;
  if (q)
    if (int rc = check_sum(who, K)) return rc;
  if (qt)
    if (int rc = check_sum(who, M)) return rc;
  if (int rc = check_tiles(who, M, K, qt ? 128 : 32, 128)) return rc;
  quant_run(M, K, dtype, x, ldx, dropout, format, q, scale, qt, scale_t, nullptr, static_cast<int64_t>(M) * K >= kPastBytes, static_cast<hipStream_t>(stream));
  return launch_status(who);
}

extern "C" size_t matmul_f8_workspace_bytes_for(int M, int N, int K, int y_dtype) {
  return M < 1 || N < 1 || quant_f8_row_bytes(K) == 0 ? 0 : f8_partial_bytes(M, N, K, y_dtype);
}
extern "C" size_t matmul_f8_workspace_bytes(int M, int N, int K) { return matmul_f8_workspace_bytes_for(M, N, K, RN50_F32); }

extern "C" int matmul_f8(int M, int N, int K, int a_format, const uint8_t* a, const uint8_t* a_scale, const uint8_t* w, const uint8_t* w_scale,
                         const float* bias, int y_dtype, void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "matmul_f8";
  clear_error();
  RN50_REQUIRE(M > 0 && N > 0 && K > 0, RN50_ERR_INVALID, "%s: non-positive size", who);
  if (int rc = check_format(who, a_format)) return rc;
  if (int rc = check_sum(who, K)) return rc;
  if (int rc = check_quantized(who, a, a_scale)) return rc;
  if (int rc = check_quantized(who, w, w_scale)) return rc;
  if (int rc = check_matrix(who, M, N, y_dtype, y, ldy)) return rc;
  RN50_REQUIRE(aligned_to(bias, 4), RN50_ERR_ALIGN, "%s: pointer not aligned to an element", who);
  if (int rc = check_product_size(who, M, N)) return rc;
  if (int rc = check_workspace(who, workspace, workspace_bytes, matmul_f8_workspace_bytes_for(M, N, K, y_dtype))) return rc;
  f8_run(a_format, y_dtype, product_args(M, N, K, a, a_scale, w, w_scale, bias, y, ldy, nullptr), K, workspace, static_cast<hipStream_t>(stream));
  return launch_status(who);
}

extern "C" size_t fc_f8_fwd_workspace_bytes_for(int M, int N, int K, int y_dtype) {
  if (M < 1 || N < 1 || quant_f8_row_bytes(K) == 0) return 0;
  Parts parts{nullptr};
  parts.take(static_cast<size_t>(M) * quant_f8_row_bytes(K));
  parts.take(quant_f8_scale_bytes(M, K));
  return parts.used + matmul_f8_workspace_bytes_for(M, N, K, y_dtype);
}
extern "C" size_t fc_f8_fwd_workspace_bytes(int M, int N, int K) { return fc_f8_fwd_workspace_bytes_for(M, N, K, RN50_F32); }

extern "C" int fc_f8_fwd(int M, int N, int K, int x_dtype, const void* x, int64_t ldx, const rn50_dropout* dropout, const uint8_t* w,
                         const uint8_t* w_scale, const float* bias, int y_dtype, void* y, int64_t ldy, uint8_t* xt, uint8_t* xt_scale,
                         void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "fc_f8_fwd";
  clear_error();
  if (int rc = check_matrix(who, M, K, x_dtype, x, ldx)) return rc;
  RN50_REQUIRE(N > 0, RN50_ERR_INVALID, "%s: non-positive size", who);
  if (int rc = check_dropout(who, dropout)) return rc;
  if (int rc = check_sum(who, K)) return rc;
  if (int rc = check_quantized(who, w, w_scale)) return rc;
  if (int rc = check_matrix(who, M, N, y_dtype, y, ldy)) return rc;
  RN50_REQUIRE(aligned_to(bias, 4), RN50_ERR_ALIGN, "%s: pointer not aligned to an element", who);
  if (xt || xt_scale) {
    if (int rc = check_quantized(who, xt, xt_scale)) return rc;
    if (int rc = check_sum(who, M)) return rc;
  }
  if (int rc = check_product_size(who, M, N)) return rc;
  if (int rc = check_tiles(who, M, K, xt ? 128 : 32, 128)) return rc;
  if (int rc = check_workspace(who, workspace, workspace_bytes, fc_f8_fwd_workspace_bytes_for(M, N, K, y_dtype))) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Parts parts{static_cast<uint8_t*>(workspace)};
  uint8_t* q = parts.take(static_cast<size_t>(M) * quant_f8_row_bytes(K));
  uint8_t* qs = parts.take(quant_f8_scale_bytes(M, K));
  if (f8_fused(M) && !xt && !dropout) {
    const F8FewArgs a{product_args(M, N, K, nullptr, nullptr, w, w_scale, bias, y, ldy, nullptr), x, ldx, K};
    if (x_dtype == RN50_BF16 && y_dtype == RN50_BF16) f8_few<uint16_t, false, 1, uint16_t>(a, s);
    else if (x_dtype == RN50_BF16) f8_few<float, false, 1, uint16_t>(a, s);
    else if (y_dtype == RN50_BF16) f8_few<uint16_t, false, 1, float>(a, s);
    else f8_few<float, false, 1, float>(a, s);
    return launch_status(who);
  }
  quant_run(M, K, x_dtype, x, ldx, dropout, RN50_E4M3, q, qs, xt, xt_scale, nullptr, false, s);
  f8_run(RN50_E4M3, y_dtype, product_args(M, N, K, q, qs, w, w_scale, bias, y, ldy, nullptr), K, parts.take(0), s);
  return launch_status(who);
}

// The parts of a backward pass's workspace: what is not asked for has none.
struct BackwardParts {
  uint8_t *q, *qs, *qt, *qts;
  double* sums;
  void* partial;
  size_t bytes;
};
static BackwardParts backward_parts(void* workspace, int M, int N, int K, int dx_dtype, bool dx, bool dW, bool db) {
  Parts parts{static_cast<uint8_t*>(workspace)};
  BackwardParts b;
  b.q = parts.take(dx ? static_cast<size_t>(M) * quant_f8_row_bytes(N) : 0);
  b.qs = parts.take(dx ? quant_f8_scale_bytes(M, N) : 0);
  b.qt = parts.take(dW ? static_cast<size_t>(N) * quant_f8_row_bytes(M) : 0);
  b.qts = parts.take(dW ? quant_f8_scale_bytes(N, M) : 0);
  b.sums = parts.take<double>(db ? static_cast<size_t>(ceil_div(M, 128)) * N * sizeof(double) : 0);
  b.partial = parts.take(0);
  b.bytes = parts.used + std::max(dx ? f8_partial_bytes(M, K, N, dx_dtype) : 0, dW ? f8_partial_bytes(N, K, M, RN50_F32) : 0);
  return b;
}

extern "C" size_t fc_f8_bwd_workspace_bytes_for(int M, int N, int K, int dx_dtype, int dx, int dW, int db) {
  if (quant_f8_row_bytes(M) == 0 || quant_f8_row_bytes(N) == 0 || K < 1) return 0;
  return backward_parts(nullptr, M, N, K, dx_dtype, dx != 0, dW != 0, db != 0).bytes;
}
extern "C" size_t fc_f8_bwd_workspace_bytes(int M, int N, int K) { return fc_f8_bwd_workspace_bytes_for(M, N, K, RN50_F32, 1, 1, 1); }

extern "C" int fc_f8_bwd(int M, int N, int K, int dy_dtype, const void* dy, int64_t ld_dy, int format, const uint8_t* wt, const uint8_t* wt_scale,
                         const uint8_t* xt, const uint8_t* xt_scale, const rn50_dropout* dropout, int dx_dtype, void* dx, int64_t ld_dx,
                         float* dW, float* db, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "fc_f8_bwd";
  clear_error();
  if (int rc = check_matrix(who, M, N, dy_dtype, dy, ld_dy)) return rc;
  RN50_REQUIRE(K > 0, RN50_ERR_INVALID, "%s: non-positive size", who);
  if (int rc = check_format(who, format)) return rc;
  if (int rc = check_dropout(who, dropout)) return rc;
  if (int rc = check_sum(who, M)) return rc;
  if (int rc = check_sum(who, N)) return rc;
  RN50_REQUIRE(dx || dW || db, RN50_ERR_INVALID, "%s: null pointer", who);
  if (dx) {
    if (int rc = check_quantized(who, wt, wt_scale)) return rc;
    if (int rc = check_matrix(who, M, K, dx_dtype, dx, ld_dx)) return rc;
  }
  if (dW)
    if (int rc = check_quantized(who, xt, xt_scale)) return rc;
  RN50_REQUIRE(aligned_to(dW, 4) && aligned_to(db, 4), RN50_ERR_ALIGN, "%s: pointer not aligned to an element", who);
  if (int rc = check_tiles(who, M, N, 32, 128)) return rc;
  if (int rc = check_product_size(who, M, K)) return rc;
  if (int rc = check_product_size(who, N, K)) return rc;
  const BackwardParts at = backward_parts(workspace, M, N, K, dx_dtype, dx, dW, db);
  if (int rc = check_workspace(who, workspace, workspace_bytes, at.bytes)) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  quant_run(M, N, dy_dtype, dy, ld_dy, nullptr, format, dx ? at.q : nullptr, at.qs, dW ? at.qt : nullptr, at.qts, db ? at.sums : nullptr, false, s);
  const SumArgs sum{at.sums, static_cast<int>(ceil_div(M, 128)), N, db};
  F8Args px = product_args(M, K, N, at.q, at.qs, wt, wt_scale, nullptr, dx, ld_dx, dropout), pw = product_args(N, K, M, at.qt, at.qts, xt, xt_scale, nullptr, dW, K, nullptr);
  if (dW) pw.sum = sum;
  if (dx && dW && f8_few_backward_fits(M, N, K)) {
    if (dx_dtype == RN50_BF16 && format == RN50_E5M2) f8_few_backward<uint16_t, true>(px, pw, s);
    else if (dx_dtype == RN50_BF16) f8_few_backward<uint16_t, false>(px, pw, s);
    else if (format == RN50_E5M2) f8_few_backward<float, true>(px, pw, s);
    else f8_few_backward<float, false>(px, pw, s);
    return launch_status(who);
  }
  if (dx) f8_run(format, dx_dtype, px, N, at.partial, s);
  if (dW) f8_run(format, RN50_F32, pw, M, at.partial, s);
  else sum_columns(sum, s);
  return launch_status(who);
}

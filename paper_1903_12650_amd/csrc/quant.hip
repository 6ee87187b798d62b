// Products in 8-bit integers: rows quantized with one scale each, and y = (sum_k q w) * q_scale * w_scale + bias on the
// integer matrix cores (v_mfma_i32_32x32x32_i8).
#include <stdlib.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "conv_internal.h"

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

// Largest magnitude of a 16-byte vector, as bits: magnitudes order like unsigned integers, an infinity and NaN above every number.
template <typename T>
__device__ __forceinline__ uint32_t top_of(uint32_t top, const Vec16& x) {
  if constexpr (sizeof(T) == 4) {
    return max(max(max(top, x.u.x & 0x7fffffffu), max(x.u.y & 0x7fffffffu, x.u.z & 0x7fffffffu)), x.u.w & 0x7fffffffu);
  } else {  // two halves side by side, each its own maximum
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    auto half = [](uint32_t v) { return __builtin_bit_cast(u16x2, v & 0x7fff7fffu); };
    const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(half(x.u.x), half(x.u.y)), __builtin_elementwise_max(half(x.u.z), half(x.u.w)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), m));
  }
}
template <typename T>
__device__ __forceinline__ uint32_t top_float_bits(uint32_t top) {  // as a float's
  return sizeof(T) == 4 ? top : max(top & 0xffffu, top >> 16) << 16;
}
// Four quantized numbers, the first in the low byte (0 where the row is not finite: inv is 0 then, and the bytes are cleared).
__device__ __forceinline__ uint32_t i8_four(const float* x, float inv) {
  const uint32_t a = i8_of(x[0], inv), b = i8_of(x[1], inv), c = i8_of(x[2], inv), d = i8_of(x[3], inv);
  return (a | b << 8) | (c << 16 | d << 24);
}
template <typename T>
__device__ __forceinline__ void store_quantized(int8_t* to, const Vec16& x, float inv) {  // (to: aligned to the vector's bytes)
  float f[Elem<T>::VEC];
  Elem<T>::unpack(x, f);
  if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(to) = inv != 0.f ? i8_four(f, inv) : 0u;
  else *reinterpret_cast<uint2*>(to) = inv != 0.f ? make_uint2(i8_four(f, inv), i8_four(f + 4, inv)) : make_uint2(0u, 0u);
}

// NT threads per row (a wave, or the workgroup), the row U vectors a thread at most: it is read once.  U = 0: it is read twice.  Bound by memory:
// 8192 x 8192 bf16 (134 MB read, 67 written) 36 us, 50176 x 1024 27, 5.7 TB/s.
template <typename T, int NT, int U>
__global__ __launch_bounds__(256) void quant_rows_kernel(const T* __restrict__ x, int64_t ldx, int M, int K, int Kp, int8_t* __restrict__ q,
                                                         float* __restrict__ scale) {
  constexpr int V = Elem<T>::VEC;
  static_assert(NT == 64 || NT == 256, "a wave or a workgroup");
  __shared__ uint32_t red[4];
  const int64_t m = (static_cast<int64_t>(blockIdx.y) * gridDim.x + blockIdx.x) * (256 / NT) + threadIdx.x / NT;
  if (m >= M) return;  // (a whole wave, or all of them)
  const int t = threadIdx.x % NT, whole = K / V, left = K - whole * V;
  const T* row = x + m * ldx;
  int8_t* out = q + m * Kp;
  uint32_t top = 0;
  Vec16 held[U > 0 ? U : 1];
  const float z_left = t < left ? Elem<T>::load(row + whole * V + t) : 0.f;
  if constexpr (U > 0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      held[u].u = make_uint4(0, 0, 0, 0);
      if (u * NT + t < whole) held[u] = load16_any(row + (u * NT + t) * V);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) top = top_of<T>(top, held[u]);
  } else {
#pragma unroll 4
    for (int v = t; v < whole; v += NT) top = top_of<T>(top, load16_any(row + v * V));
  }
  top = max(top_float_bits<T>(top), __float_as_uint(z_left) & 0x7fffffffu);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), off, 64)));
  if constexpr (NT == 256) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(red[0], red[1]), max(red[2], red[3]));
  }
  float inv;
  const float s = i8_scale(top, &inv);
  if constexpr (U > 0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * NT + t < whole) store_quantized<T>(out + (u * NT + t) * V, held[u], inv);
  } else {
#pragma unroll 4
    for (int v = t; v < whole; v += NT) store_quantized<T>(out + v * V, load16_any(row + v * V), inv);
  }
  // the numbers behind the last whole vector, and the zeros behind them
  const int rest = Kp - whole * V;
  for (int i = t; i < rest; i += NT) out[whole * V + i] = static_cast<int8_t>(i < left && inv != 0.f ? i8_of(z_left, inv) : 0u);
  if (t == 0) scale[m] = s;
}

// ------------------------------------------------------------------- product
struct ProductArgs {
  const int8_t *q, *w;
  const float *qs, *ws, *bias;
  void* y;
  int64_t ldy;
  int M, N, Kp, tiles_m, tiles_n;
};

// Tile BM x BN, WM x WN waves of 32x32 blocks (v_mfma_i32_32x32x32_i8).  A chunk is 128 bytes of every row of both operands, brought
// straight into LDS (16 bytes a lane) into one of RING buffers while another is multiplied: one barrier a chunk.  Piece p (16 bytes) of
// row r lies in slot p ^ ((r >> 1) & 7), which spreads the fragment reads (32 rows of one piece) over all banks.  Rows past the last and
// the second half of a last chunk of 64 bytes are zeros.  The weights are the first operand, so that a lane has 4 consecutive columns of one row.
// What bounds it: large products the power that the matrix cores may draw beside LDS (8192^3 437 to 490 us, 2.2 to 2.5 POP/s; of zeros
// 326), middle ones a workgroup's own chain: some 4 us of start, first loads and output stage around 0.6 (128x128) to 1.7 us (256x256)
// a chunk, of which the matrix cores need 0.2 to 0.85.  Fragments are requested a step ahead (by the compiler's own order, where they are
// needed: 8192^3 466 us, by 128x128 540 -> 513, 4096 x 1024 -> 4096 29.6 -> 25.4).
template <typename T, int BM, int BN, int WM, int WN, int RING>
__global__ __launch_bounds__(64 * WM * WN) void matmul_i8_kernel(const ProductArgs a) {
  constexpr int NT = 64 * WM * WN, RPL = NT / 8, RA = BM / RPL, RB = BN / RPL, TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr int STAGE = (BM + BN) * 128;
  // Requests of the next chunk: between the first steps where nothing else runs on the compute unit meanwhile (256x256: 8192^3 459 -> 437 us,
  // 300 x 8192 -> 8192 88 -> 78), all at the front elsewhere (128x128: 8192^3 513, 532 spread).
  constexpr bool SPREAD = NT == 512;
  static_assert(RA * RPL == BM && RB * RPL == BN && TM >= 1 && TN >= 1, "whole passes, whole blocks");
  extern __shared__ __align__(16) unsigned char smem[];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int wm = wave % WM, wn = wave / WM;
  // Neighbouring tiles run on one XCD: they go down GROUP row tiles before the next column tile, so that the tiles of an XCD's 32 compute
  // units share rows of both operands in its L2.
  constexpr int GROUP = 4;
  const int id = xcd_remap(blockIdx.x, gridDim.x);
  const int per = GROUP * a.tiles_n, g = id / per, r = id - g * per, high = min(GROUP, a.tiles_m - g * GROUP);
  const int m0 = (g * GROUP + r % high) * BM, n0 = r / high * BN;
  const int rows = min(BM, a.M - m0), cols = min(BN, a.N - n0);
  const rsrc_words rsA = make_rsrc_words(a.q + static_cast<int64_t>(m0) * a.Kp, static_cast<uint32_t>(rows) * a.Kp);
  const rsrc_words rsB = make_rsrc_words(a.w + static_cast<int64_t>(n0) * a.Kp, static_cast<uint32_t>(cols) * a.Kp);
  const int slot = tid & 7, lrow = tid >> 3, piece = slot ^ ((lrow >> 1) & 7);
  uint32_t at_a[RA], at_b[RB];
#pragma unroll
  for (int i = 0; i < RA; ++i) at_a[i] = lrow + RPL * i < rows ? static_cast<uint32_t>(lrow + RPL * i) * a.Kp + piece * 16 : kOob;
#pragma unroll
  for (int i = 0; i < RB; ++i) at_b[i] = lrow + RPL * i < cols ? static_cast<uint32_t>(lrow + RPL * i) * a.Kp + piece * 16 : kOob;
  typedef __attribute__((address_space(3))) unsigned char* lds_byte_ptr;
  const uint32_t dst = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_byte_ptr)smem)) + static_cast<uint32_t>(wave) * 1024u);
  const int chunks = (a.Kp + 127) >> 7;
  enum { ROWS = 1, COLUMNS = 2 };
  auto load = [&](int c, int buffer, int what) __attribute__((always_inline)) {
    const uint32_t so = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(c) * 128u), to = dst + static_cast<uint32_t>(buffer) * STAGE;
    const bool in = c * 128 + piece * 16 < a.Kp;
#pragma unroll
    for (int i = 0; i < RA; ++i)
      if (what & ROWS) buffer_load16_to_lds(rsA, to + i * (RPL * 128), in ? at_a[i] : kOob, so);
#pragma unroll
    for (int i = 0; i < RB; ++i)
      if (what & COLUMNS) buffer_load16_to_lds(rsB, to + BM * 128 + i * (RPL * 128), in ? at_b[i] : kOob, so);
  };
  i32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
  int frag[4];
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) frag[kk] = (lane & 31) * 128 + (((2 * kk + (lane >> 5)) ^ ((lane >> 1) & 7)) << 4);
#pragma unroll
  for (int c = 0; c < RING - 1; ++c)
    if (c < chunks) load(c, c, ROWS | COLUMNS);
  int now = 0, next = RING - 1;  // buffers of this chunk and of the one that is requested
  for (int c = 0; c < chunks; ++c) {
    ring_wait<RING, RA + RB>(chunks - 1 - c);  // this chunk is there, and the buffer of the one before it has been read
    const int ahead = c + RING - 1, into = next;
    if (!SPREAD && ahead < chunks) load(ahead, into, ROWS | COLUMNS);
    const unsigned char* ta = smem + now * STAGE + wm * (BM / WM) * 128;
    const unsigned char* tb = smem + now * STAGE + BM * 128 + wn * (BN / WN) * 128;
    now = now + 1 == RING ? 0 : now + 1;
    next = next + 1 == RING ? 0 : next + 1;
    i32x4 fa[2][TM], fb[2][TN];
    auto read = [&](int kk) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < TM; ++i) fa[kk & 1][i] = *reinterpret_cast<const i32x4*>(ta + i * 32 * 128 + frag[kk]);
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[kk & 1][j] = *reinterpret_cast<const i32x4*>(tb + j * 32 * 128 + frag[kk]);
    };
    read(0);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      if (kk < 3) read(kk + 1);
      if (SPREAD && kk < 2 && ahead < chunks) load(ahead, into, kk == 0 ? ROWS : COLUMNS);
      __builtin_amdgcn_sched_barrier(0);  // (the compiler would move every read to where its product waits for it)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[kk & 1][j], fa[kk & 1][i], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // Output: a wave's 32 rows at a time through LDS (its own part of it), whole rows of the wave's columns from there.
  constexpr int WC = BN / WN, PITCH = WC + 4;  // floats (rows 16 bytes further along the banks)
  static_assert(WM * WN * 32 * PITCH * 4 <= RING * STAGE, "the output stage fits the ring");
  lds_reads_then_barrier();
  float* mine = reinterpret_cast<float*>(smem) + wave * 32 * PITCH;
  constexpr int V = Elem<T>::VEC, LPR = WC / V, RPP = 64 / LPR;  // lanes a row, rows a pass
  const int col = n0 + wn * WC + lane % LPR * V;
  float t[V], b[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    t[j] = col + j < a.N ? a.ws[col + j] : 0.f;
    b[j] = a.bias && col + j < a.N ? a.bias[col + j] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float4 f = make_float4(acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]);
        *reinterpret_cast<float4*>(mine + (lane & 31) * PITCH + j * 32 + v * 8 + (lane >> 5) * 4) = f;
      }
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int p = 0; p < 32 / RPP; ++p) {
      const int row = p * RPP + lane / LPR, m = m0 + wm * (BM / WM) + i * 32 + row;
      if (m < a.M && col < a.N) {
        const float s = a.qs[m];
        float f[V];
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = fmaf(mine[row * PITCH + lane % LPR * V + j] * s, t[j], b[j]);
        T* to = static_cast<T*>(a.y) + m * a.ldy + col;
        if (col + V <= a.N) {
          Vec16 o;
          Elem<T>::pack(f, o);
          store16_any(to, o);
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
}

// Few rows (M <= 16 * MB): the weights go by once, bound by memory; a workgroup owns 16 * CB columns, its waves a part of K each.  A wave's lane reads
// 16 bytes of column lane % 16 at 16 * (lane / 16) of a step of 64, straight into the matrix cores (v_mfma_i32_16x16x64_i8), U steps'
// loads in flight; the rows of activations are the second operand.  The waves' integer sums are added through LDS.  1 x 8192 -> 8192 14.4 us with
// the quantization (67 MB at 4.7 TB/s; a launch's start and end take some 4), 64 x 8192 -> 8192 31 (every workgroup reads the rows from its L2).
// X: the activations are float or bfloat16 and quantized here (up to 16 rows, into LDS: all threads each row, more than kFusedRows a wave a
// row), while the first weights are on their way: no second launch; every workgroup does so for itself.
constexpr int kFewThreads = 512, kFewWaves = kFewThreads / 64, kFusedRows = 4;
struct FewArgs {
  ProductArgs p;
  const void* x;
  int64_t ldx;
  int K;
};
template <typename T, int MB, int CB, typename X>
__global__ __launch_bounds__(kFewThreads) void matmul_i8_few_kernel(const FewArgs a) {
  constexpr bool FUSED = !std::is_void<X>::value;
  constexpr int U = MB >= 4 ? 2 : 8 / CB;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int red[kFewWaves][MB][256];
  __shared__ float scale_s[16 * MB];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int n0 = blockIdx.x * (16 * CB), M = a.p.M, N = a.p.N, Kp = a.p.Kp;
  const int steps = Kp >> 6, from = steps * wave / kFewWaves, to = steps * (wave + 1) / kFewWaves;
  const int8_t* wp[CB];
  i32x4 fw[U][CB];
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    wp[c] = a.p.w + static_cast<int64_t>(min(n0 + c * 16 + (lane & 15), N - 1)) * Kp + 16 * (lane >> 4);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (from + u < to) fw[u][c] = *reinterpret_cast<const i32x4*>(wp[c] + (from + u) * 64);
  }
  const int8_t* xq[MB];  // this lane's rows
  if constexpr (FUSED) {
    constexpr int V = Elem<X>::VEC;
    const int whole = a.K / V, left = a.K - whole * V;
    if (M > kFusedRows) {  // a wave a row
      for (int m = wave; m < M; m += kFewWaves) {
        const X* row = static_cast<const X*>(a.x) + m * a.ldx;
        uint32_t top = 0;
        for (int v = lane; v < whole; v += 64) top = top_of<X>(top, load16_any(row + v * V));
        const float z_left = lane < left ? Elem<X>::load(row + whole * V + lane) : 0.f;
        top = max(top_float_bits<X>(top), __float_as_uint(z_left) & 0x7fffffffu);
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), off, 64)));
        float inv;
        const float s = i8_scale(top, &inv);
        int8_t* out = reinterpret_cast<int8_t*>(smem) + m * Kp;
        for (int v = lane; v < whole; v += 64) store_quantized<X>(out + v * V, load16_any(row + v * V), inv);
        for (int i = lane; i < Kp - whole * V; i += 64) out[whole * V + i] = static_cast<int8_t>(i < left && inv != 0.f ? i8_of(z_left, inv) : 0u);
        if (lane == 0) scale_s[m] = s;
      }
    } else {  // all threads each of them
      uint32_t top[kFusedRows];
      float z_left[kFusedRows];
#pragma unroll
      for (int m = 0; m < kFusedRows; ++m) {
        top[m] = 0;
        z_left[m] = 0.f;
        if (m < M) {
          const X* row = static_cast<const X*>(a.x) + m * a.ldx;
          for (int v = tid; v < whole; v += kFewThreads) top[m] = top_of<X>(top[m], load16_any(row + v * V));
          if (tid < left) z_left[m] = Elem<X>::load(row + whole * V + tid);
        }
      }
#pragma unroll
      for (int m = 0; m < kFusedRows; ++m)
        if (m < M) {
          uint32_t t = max(top_float_bits<X>(top[m]), __float_as_uint(z_left[m]) & 0x7fffffffu);
#pragma unroll
          for (int off = 32; off > 0; off >>= 1) t = max(t, static_cast<uint32_t>(__shfl_xor(static_cast<int>(t), off, 64)));
          if (lane == 0) red[wave][0][m] = static_cast<int>(t);
        }
      __syncthreads();
#pragma unroll
      for (int m = 0; m < kFusedRows; ++m)
        if (m < M) {
          uint32_t t = 0;
#pragma unroll
          for (int w = 0; w < kFewWaves; ++w) t = max(t, static_cast<uint32_t>(red[w][0][m]));
          float inv;
          const float s = i8_scale(t, &inv);
          const X* row = static_cast<const X*>(a.x) + m * a.ldx;
          int8_t* out = reinterpret_cast<int8_t*>(smem) + m * Kp;
          for (int v = tid; v < whole; v += kFewThreads) store_quantized<X>(out + v * V, load16_any(row + v * V), inv);
          if (tid < Kp - whole * V) out[whole * V + tid] = static_cast<int8_t>(tid < left && inv != 0.f ? i8_of(z_left[m], inv) : 0u);
          if (tid == 0) scale_s[m] = s;
        }
    }
    __syncthreads();
  }
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    const int m = min(b * 16 + (lane & 15), M - 1);
    xq[b] = (FUSED ? reinterpret_cast<const int8_t*>(smem) : a.p.q) + static_cast<int64_t>(m) * Kp + 16 * (lane >> 4);
  }
  i32x4 acc[CB][MB];
#pragma unroll
  for (int c = 0; c < CB; ++c)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[c][b] = i32x4{0, 0, 0, 0};
  int s = from;
  // Where a step has four loads of rows: whole groups without a test per step, behind which these loads would stay (64 x 8192 -> 8192 35.5 ->
  // 30.9 us; with one or two the compiler holds more in registers than there are).
  for (; MB >= 4 && s + U <= to; s += U) {
    i32x4 w[U][CB], x[U][MB];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int b = 0; b < MB; ++b) x[u][b] = *reinterpret_cast<const i32x4*>(xq[b] + (s + u) * 64);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        w[u][c] = fw[u][c];
        if (s + U + u < to) fw[u][c] = *reinterpret_cast<const i32x4*>(wp[c] + (s + U + u) * 64);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int c = 0; c < CB; ++c) acc[c][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][c], x[u][b], acc[c][b], 0, 0, 0);
  }
  for (; s < to; s += U) {
    i32x4 w[U][CB];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < CB; ++c) {
        w[u][c] = fw[u][c];
        if (s + U + u < to) fw[u][c] = *reinterpret_cast<const i32x4*>(wp[c] + (s + U + u) * 64);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < to) {
#pragma unroll
        for (int b = 0; b < MB; ++b) {
          const i32x4 x = *reinterpret_cast<const i32x4*>(xq[b] + (s + u) * 64);
#pragma unroll
          for (int c = 0; c < CB; ++c) acc[c][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][c], x, acc[c][b], 0, 0, 0);
        }
      }
  }
  // column 4 * (lane / 16) + i of the 16, row lane % 16
#pragma unroll
  for (int c = 0; c < CB; ++c) {
    if (FUSED || c) __syncthreads();  // (`red` has been read)
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[wave][b][(lane & 15) * 16 + 4 * (lane >> 4) + i] = acc[c][b][i];
    __syncthreads();
#pragma unroll
    for (int e = tid; e < MB * 256; e += kFewThreads) {
      const int b = e >> 8, m = b * 16 + ((e >> 4) & 15), n = n0 + c * 16 + (e & 15);
      if (m < M && n < N) {
        int sum = 0;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) sum += red[w][b][e & 255];
        const float s = FUSED ? scale_s[m] : a.p.qs[m];
        Elem<T>::store(static_cast<T*>(a.p.y) + m * a.p.ldy + n, fmaf(static_cast<float>(sum) * s, a.p.ws[n], a.p.bias ? a.p.bias[n] : 0.f));
      }
    }
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
  RN50_REQUIRE(ceil_div(M, 64) * ceil_div(N, 64) <= (1 << 22) && N <= (1 << 26), RN50_ERR_UNSUPPORTED, "%s: M=%d by N=%d beyond the launch grid", who, M, N);
  RN50_REQUIRE(w && w_scale && y, RN50_ERR_INVALID, "%s: null pointer", who);
  RN50_REQUIRE(ldy >= N, RN50_ERR_INVALID, "%s: rows of %d elements %lld apart", who, N, static_cast<long long>(ldy));
  RN50_REQUIRE(aligned16(w), RN50_ERR_ALIGN, "%s: 8-bit rows not 16-byte aligned", who);
  RN50_REQUIRE(aligned_to(w_scale, 4) && aligned_to(bias, 4) && aligned_to(y, y_dtype == RN50_BF16 ? 2 : 4), RN50_ERR_ALIGN,
               "%s: pointer not aligned to an element", who);
  return RN50_OK;
}

template <typename T>
static void quant_typed(int M, int K, const T* x, int64_t ldx, int8_t* q, float* scale, hipStream_t s) {
  const int Kp = static_cast<int>(quant_i8_row_bytes(K));
  const int64_t vecs = K / Elem<T>::VEC;
  const auto grid = [M](int rows) {  // of workgroups of so many rows
    const int64_t n = ceil_div(M, rows);
    return n <= 65536 ? dim3(static_cast<unsigned>(n)) : dim3(65536, static_cast<unsigned>(ceil_div(n, 65536)));
  };
#define QUANT(NT, U) RN50_LAUNCH("quant_rows_i8", (quant_rows_kernel<T, NT, U>), grid(256 / NT), dim3(256), 0, s, x, ldx, M, K, Kp, q, scale)
  if (vecs <= 64) QUANT(64, 1);
  else if (vecs <= 64 * 2) QUANT(64, 2);
  else if (vecs <= 64 * 4) QUANT(64, 4);
  else if (vecs <= 64 * 8) QUANT(64, 8);
  else if (vecs <= 256 * 4) QUANT(256, 4);
  else if (vecs <= 256 * 8) QUANT(256, 8);
  else QUANT(256, 0);
#undef QUANT
}
static void quant_run(int M, int K, int dtype, const void* x, int64_t ldx, int8_t* q, float* scale, hipStream_t s) {
  if (dtype == RN50_BF16) quant_typed(M, K, static_cast<const uint16_t*>(x), ldx, q, scale, s);
  else quant_typed(M, K, static_cast<const float*>(x), ldx, q, scale, s);
}
template <typename T, int BM, int BN, int WM, int WN, int RING>
static void product_tile(ProductArgs a, hipStream_t s) {
  constexpr int lds = RING * (BM + BN) * 128;
  a.tiles_m = static_cast<int>(ceil_div(a.M, BM));
  a.tiles_n = static_cast<int>(ceil_div(a.N, BN));
  const auto kernel = matmul_i8_kernel<T, BM, BN, WM, WN, RING>;
  allow_big_lds(kernel, lds);
  RN50_LAUNCH("matmul_i8", kernel, dim3(static_cast<unsigned>(a.tiles_m) * a.tiles_n), dim3(64 * WM * WN), lds, s, a);
}
template <typename T, int MB, int CB, typename X>
static void few_rows(const FewArgs& a, hipStream_t s) {
  const auto kernel = matmul_i8_few_kernel<T, MB, CB, X>;
  const int lds = std::is_void<X>::value ? 0 : static_cast<int>(align_up(static_cast<size_t>(a.p.M) * a.p.Kp, 16));
  if (lds) allow_big_lds(kernel, lds);
  RN50_LAUNCH("matmul_i8", kernel, dim3(static_cast<unsigned>(ceil_div(a.p.N, 16 * CB))), dim3(kFewThreads), lds, s, a);
}
template <typename T>
static void few_rows_quantized(const ProductArgs& p, hipStream_t s) {
  const FewArgs a{p, nullptr, 0, 0};
  // 32 columns a workgroup, which reads the rows half as often, where enough workgroups are left: 64 x 8192 -> 8192 46 -> 36 us, 20 x 4096 -> 8192
  // 17.3 -> 14.7, 48 x 2048 -> 16384 24.7 -> 18.2; 33 x 4096 -> 4096 13.6 -> 16.0, 64 x 8192 -> 2048 23 -> 28; with 16 rows 8192 -> 8192 23.8 -> 24.2.
  const bool wide = p.N >= 8192;
  if (p.M <= 16) {
    few_rows<T, 1, 1, void>(a, s);
  } else if (p.M <= 32) {
    if (wide) few_rows<T, 2, 2, void>(a, s);
    else few_rows<T, 2, 1, void>(a, s);
  } else {
    if (wide) few_rows<T, 4, 2, void>(a, s);
    else few_rows<T, 4, 1, void>(a, s);
  }
}
constexpr int kFewRows = 64;
// Whether fc_i8_fwd takes its rows as they are.  Two launches -> one: 1 x 2048 -> 1000 7.6 -> 5.2 us, 1 x 8192 -> 8192 19 -> 16, 16 x 1024 -> 1000 8.3 -> 5.8;
// 3 x 8192 -> 16384 34 -> 36 (every workgroup quantizes all rows), 64 x 256 -> 1000 8.3 -> 9.9 (eight rows a wave).
static bool few_fused(int M, int K) {
  int64_t most = 16384;
#ifdef RN50_TUNING  // tuning builds only: RN50_I8_FUSED=numbers
  if (const char* e = getenv("RN50_I8_FUSED")) most = atoi(e);
#endif
  return M <= 16 && static_cast<int64_t>(M) * static_cast<int64_t>(quant_i8_row_bytes(K)) <= most;
}
template <typename T>
static void product_typed(const ProductArgs& a, hipStream_t s) {
#ifdef RN50_TUNING  // tuning builds only: RN50_I8_TILE=rows
  if (const char* e = getenv("RN50_I8_TILE")) {
    switch (atoi(e)) {
      case 256: return product_tile<T, 256, 256, 2, 4, 2>(a, s);
      case 128: return product_tile<T, 128, 128, 2, 2, 2>(a, s);
      case 12864: return product_tile<T, 128, 64, 2, 2, 3>(a, s);
      case 64: return product_tile<T, 64, 64, 2, 2, 2>(a, s);
      case 1: return few_rows_quantized<T>(a, s);
    }
  }
#endif
  if (a.M <= kFewRows) return few_rows_quantized<T>(a, s);
  // The largest tile of which there are enough for the 256 compute units (256x256, 128x128, 128x64, 64x64 in us): 4096^3 61, 72, 92, 109;
  // 5000 x 5000 -> 1000 (80, 320, 640, 1264 tiles) 64, 42, 52, 58; 300 x 8192 -> 8192 (64, 192, 384, 640) 79, 42, 36, 40; 512 x 4096 -> 4096
  // (32, 128, 256, 512) 44, 23, 16, 18; 1000 x 2048 -> 1000 (16, 64, 128, 256) 26, 13, 9.7, 7.6.  The 256x256 one leaves a unit a single
  // workgroup, so only where its last round is full enough, 256x256 and 128x128: 1024 -> 256 by 130 tiles of 256 rows 21.7, 22.6, by 196 23.1, 24.6,
  // by 240 25.0, 27.0, by 300 38.6, 35.5, by 380 43.6, 41.5, by 420 44.5, 47.5; 4096 -> 2048 by 136 tiles 51, 56, by 200 53, 60, by 264 100, 87,
  // by 384 107, 106, by 424 110, 123.  Three or four buffers instead of two cost the workgroups that share a unit (4096^3 by 128x128 a quarter).
  auto tiles = [&](int bm, int bn) { return ceil_div(a.M, bm) * ceil_div(a.N, bn); };
  const int64_t large = tiles(256, 256);
  if (large > 128 && (large <= 256 || large * 5 >= ceil_div(large, 256) * 256 * 4)) product_tile<T, 256, 256, 2, 4, 2>(a, s);
  else if (tiles(128, 128) >= 256) product_tile<T, 128, 128, 2, 2, 2>(a, s);
  else if (tiles(128, 64) >= 256) product_tile<T, 128, 64, 2, 2, 3>(a, s);
  else product_tile<T, 64, 64, 2, 2, 2>(a, s);
}
static void product_run(int M, int N, int K, const int8_t* q, const float* qs, const int8_t* w, const float* ws, const float* bias, int y_dtype,
                        void* y, int64_t ldy, hipStream_t s) {
  const ProductArgs a{q, w, qs, ws, bias, y, ldy, M, N, static_cast<int>(quant_i8_row_bytes(K)), 0, 0};
  if (y_dtype == RN50_BF16) product_typed<uint16_t>(a, s);
  else product_typed<float>(a, s);
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
  if (few_fused(M, K)) {
    const FewArgs a{{nullptr, w, nullptr, w_scale, bias, y, ldy, M, N, static_cast<int>(quant_i8_row_bytes(K)), 0, 0}, x, ldx, K};
    if (x_dtype == RN50_BF16 && y_dtype == RN50_BF16) few_rows<uint16_t, 1, 1, uint16_t>(a, s);
    else if (x_dtype == RN50_BF16) few_rows<float, 1, 1, uint16_t>(a, s);
    else if (y_dtype == RN50_BF16) few_rows<uint16_t, 1, 1, float>(a, s);
    else few_rows<float, 1, 1, float>(a, s);
    return launch_status("fc_i8_fwd");
  }
  quant_run(M, K, x_dtype, x, ldx, q, qs, s);
  product_run(M, N, K, q, qs, w, w_scale, bias, y_dtype, y, ldy, s);
  return launch_status("fc_i8_fwd");
}

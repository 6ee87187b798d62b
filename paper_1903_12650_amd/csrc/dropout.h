// A dropout's mask as a function of (seed, call, place), for the kernels that drop elements as they read or write them.
#pragma once
#include "common.h"

namespace rn50 {

struct DropArgs {
  uint32_t key0, key1;
  uint32_t threshold;  // an element is kept where its 16 bits reach this (65536: nothing is kept)
  float factor;        // 1 / the share that is kept
  uint64_t call;
  const uint64_t* step;
};
// Whether the arguments are refused, and what the kernels take (d NULL: everything is kept).
int check_dropout(const char* who, const rn50_dropout* d);
DropArgs drop_args(const rn50_dropout* d);

// This call's number: fixed, or moved on by a counter in device memory (read when the kernel runs).
__device__ __forceinline__ uint64_t drop_call(const DropArgs& d) { return d.call + (d.step ? *d.step : 0); }

// Philox4x32-10 (Salmon et al., SC'11) of counter (b low, b high | 2^31, call low, call high): 16 bits for each of the eight
// elements of a row's block b, element j the half j % 2 of word j / 2.  (Bit 63 keeps these counters apart from those of
// resnet_init_params, whose second word is an element index of at most 2^31.)
struct DropBits {
  uint32_t w[4];
};
__device__ __forceinline__ DropBits drop_bits(const DropArgs& d, uint64_t call, uint64_t b) {
  uint32_t c0 = static_cast<uint32_t>(b), c1 = static_cast<uint32_t>(b >> 32) | 0x80000000u, c2 = static_cast<uint32_t>(call),
           c3 = static_cast<uint32_t>(call >> 32), k0 = d.key0, k1 = d.key1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = static_cast<uint64_t>(0xD2511F53u) * c0, p1 = static_cast<uint64_t>(0xCD9E8D57u) * c2;
    c0 = static_cast<uint32_t>(p1 >> 32) ^ c1 ^ k0;
    c1 = static_cast<uint32_t>(p1);
    c2 = static_cast<uint32_t>(p0 >> 32) ^ c3 ^ k1;
    c3 = static_cast<uint32_t>(p0);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return DropBits{{c0, c1, c2, c3}};
}
__device__ __forceinline__ bool drop_keeps(const DropArgs& d, const DropBits& r, int j) {  // (j known when compiling)
  return (j & 1 ? r.w[j >> 1] >> 16 : r.w[j >> 1] & 0xffffu) >= d.threshold;
}
// The same for any j.
__device__ __forceinline__ bool drop_keeps_at(const DropArgs& d, const DropBits& r, int j) {
  const uint32_t lo = j & 2 ? r.w[1] : r.w[0], hi = j & 2 ? r.w[3] : r.w[2], w = j & 4 ? hi : lo;
  return (j & 1 ? w >> 16 : w & 0xffffu) >= d.threshold;
}

}  // namespace rn50

// The paged 4-bit cache: its format on the device, and what the kernels that read and write it share.
#pragma once

#include <type_traits>

#include "common.cuh"

namespace seqtree {

constexpr int kGranule = SEQ_KV4_GRANULE;             // tokens
constexpr int kGranuleBytes = SEQ_KV4_GRANULE_BYTES;  // K codes, V codes, K params, V params
constexpr int kCodeBytes = 64;                        // a row's codes
constexpr int kGranuleV = kGranule * kCodeBytes;      // where V's codes start
constexpr int kGranuleParams = 2 * kGranuleV;         // where K's (scale, mid) start; V's 64 bytes behind them

__host__ __device__ inline bool kv4_page_size_ok(int page_size) { return page_size == 16 || page_size == 32 || page_size == 64 || page_size == 128; }

// Four bits -> half precision, exactly.  `w` holds nibbles 0..3 of one row in its low half and of another in its high half (or
// nibbles 0..3 and 4..7 of one row); out[k] is the pair (nibble k of the low half, nibble k of the high half), each less 8.  A nibble in bits 0..3
// of 0x6400 is 1024 + x, one in bits 4..7 of 0x5400 is 64 + x: two nibbles come out without a shift.
__device__ __forceinline__ uint32_t hsub2_bits(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t hfma2_bits(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t hmul2_bits(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <int kMask, int kOr>
__device__ __forceinline__ uint32_t and_or(uint32_t w) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(w), "n"(kMask), "n"(kOr));
  return d;
}
__device__ __forceinline__ void unpack4(uint32_t w, uint32_t* out) {
  const uint32_t v = w >> 8;
  out[0] = hsub2_bits(and_or<0x000f000f, 0x64006400>(w), 0x64086408u);
  out[1] = hsub2_bits(and_or<0x00f000f0, 0x54005400>(w), 0x54805480u);
  out[2] = hsub2_bits(and_or<0x000f000f, 0x64006400>(v), 0x64086408u);
  out[3] = hsub2_bits(and_or<0x00f000f0, 0x54005400>(v), 0x54805480u);
}

}  // namespace seqtree

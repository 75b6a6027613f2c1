// Rows of 4 bits: format (see hack.h) and what its kernels share.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "hack_internal.h"

namespace hack {
namespace kv4 {

constexpr int kBlock = 16;                       // elements that share a scale
// (1 + m/8) 2^(e-20) as bf16: the byte's eight bits in place of the last exponent and first mantissa bits
constexpr uint32_t kScaleBias = (127 - 20) << 7;

// The planes as a kernel sees them.
struct Planes {
  unsigned char *k_codes, *v_codes, *k_scales, *v_scales;
  const int64_t* row_off;
  long long rows;
  int cap;
};

#if defined(__CUDACC__)
__device__ __forceinline__ long long first_row(const Planes& p, int head) {
  return p.row_off ? (long long)p.row_off[head] : (long long)head * p.cap;
}
// Whether a head's rows are in the planes
__device__ __forceinline__ bool inside(const Planes& p, long long first) { return first >= 0 && first <= p.rows - p.cap; }
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(((byte << 4) + kScaleBias) << 16); }
__device__ __forceinline__ uint32_t bf162_mul(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t bf162_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
// A pair of scales as bf16x2 from two bytes (in bits 0-7 and 16-23), and -136 times it.  Code c + 8 in the low bits of 0x4300 is
// the bf16 number 136 + c, and (136 + c) s - 136 s = c s: every term and the result are exact (136 has five
// significant bits, s four).
struct Scale2 { uint32_t s, off; };
__device__ __forceinline__ Scale2 scale2(uint32_t bytes) {
  Scale2 r;
  r.s = bytes * 16 + (kScaleBias | kScaleBias << 16);
  r.off = bf162_mul(r.s, 0xc308c308u);           // -136, twice
  return r;
}
// Codes in bits 0-3 and 16-19 of w >> shift: two values
__device__ __forceinline__ uint32_t values2(uint32_t w, int shift, const Scale2& s) {
  uint32_t x;
  asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(x) : "r"(w >> shift));   // (w & mask) | magic
  return bf162_fma(x, s.s, s.off);
}
// x += the low, y += the high bf16 number of w
__device__ __forceinline__ void add_bf162(float& x, float& y, uint32_t w) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.bf16 %0, l, %0;\n\tadd.rn.f32.bf16 %1, h, %1;\n\t}" : "+f"(x), "+f"(y) : "r"(w));
}
#endif

}  // namespace kv4

hack_status_t kv4_check(const hack_kv4_t* kv);          // HACK_OK, or the error with its text
kv4::Planes kv4_planes(const hack_kv4_t* kv);
// The rows that a layer holds (a: its lengths and planes) behind the lens rows of the 4-bit cache; launches: counts on.
hack_status_t launch_store_kv4(const StepArgs& a, int dtype, const hack_kv4_t* kv, const int32_t* lens, uint64_t& launches, cudaStream_t st);

}  // namespace hack

// Device helpers of the 8-bit cache's kernels.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace epara {

constexpr float KV8_TINY_SCALE = 1.17549435e-38f;     // 2^-126
constexpr float KV8_MOST_V = 1.7014118e38f;           // 2^127: of a V scale times that factor
constexpr float KV8_NONE = -3.4028234e38f;            // the maximum of a row that has seen no score
constexpr int KV8_MOST_UP = 120;                      // weights -- probability x V scale -- are multiplied by at most 2^120 to make fp16 of them

// two fp32 -> two e4m3 codes (lo in the low byte), nearest even, NaN to NaN
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// two codes (the low 16 bits) -> two fp16, exact
__device__ __forceinline__ uint32_t to_f16x2(uint32_t two_codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two_codes));
  return r;
}
__device__ __forceinline__ float2 to_float2(uint32_t two_codes) {
  const uint32_t h = to_f16x2(two_codes);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// A request's new rows [row, row + n), from the prefix sums `q_rows` (or one row each); what they say is clamped to the T rows.
__device__ __forceinline__ void new_rows(const int32_t* q_rows, int b, int T, int& row, int& n) {
  if (q_rows == nullptr) { row = b; n = b < T ? 1 : 0; return; }
  row = min(max(q_rows[b], 0), T);
  n = min(max(q_rows[b + 1], row), T) - row;
}

// The request of row t, by a converged warp: how many requests end at or before it (B: none has it).  32 looks at a time.
__device__ __forceinline__ int request_of(const int32_t* q_rows, int B, int t) {
  int lo = 0, hi = B;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, c = __popc(__ballot_sync(0xffffffffu, q_rows[min(lo + ((int)(threadIdx.x & 31) + 1) * step, hi)] <= t));
    hi = c == 32 ? hi : min(lo + (c + 1) * step, hi) - 1;
    lo = c == 32 ? hi : lo + c * step;
  }
  return lo;
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
// ... zeros instead when `valid` is false (the source is not read then)
__device__ __forceinline__ void cp16_zfill(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// A query row with the largest magnitude `top` is multiplied by `up`, a power of two that brings it to [2^14, 2^15), before it becomes
// fp16: what is 2^-28 of the largest is still a normal number.  Returns the factor that turns the row's scores into log2 units.
template <int HD>
__device__ __forceinline__ float row_factor(float top, float& up) {
  const int ex = min(max((int)(__float_as_uint(top) >> 23), 15), 254);       // biased exponent
  up = __uint_as_float((uint32_t)min(254 + 14 - ex, 254) << 23);
  return 1.4426950408889634f * rsqrtf((float)HD) / up;
}

}  // namespace epara

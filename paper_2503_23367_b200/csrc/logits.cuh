// What the kernels on rows of logits share: exponentials, sums of them against a maximum, and how such sums are put together.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cfloat>
#include <cstdint>

namespace fv {
namespace logits_detail {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// set() once for every device that is current in a call.
template <typename F> inline cudaError_t once_per_device(std::atomic<uint64_t>& done, F set) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1))) return e;
  e = set();
  if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
  return e;
}

// ---- small pieces -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float exp2_fast(float x) {   // 2^x within 2^-22 of its value, 0 at -inf, NaN at NaN
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float warp_max(float v) {   // (no NaN comes here)
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
__device__ __forceinline__ void put_status(int32_t* status, int code) {
  if (status) atomicCAS(status, 0, code);
}

// ---- exponents ---------------------------------------------------------------------------------------------------------------
// e = 2^d, d = (x - m) c, c = log2(e) / tau.  Near 0 (|m c| < 2^21) d is taken as x c - R in one operation, rounded once, R = m c in fp32 (or that of an earlier maximum): all of a row's
// exponents are off by the one number m c - R, by which the sums are put right (delta).  That saves half an instruction per logit.  For the maximum that R was taken from, delta is the
// rounding of m c alone: the largest logit then adds 1 to s and next to nothing to t, and an entropy of almost 0 keeps its digits.  (With the whole number next to m c, t held up to half of s, and the
// difference of the two was off by 2^-25.)  Far from 0, where x c has no fraction left (masks of -1e9, of the type's lowest value), the difference is taken first.
constexpr float kFar = 2097152.f;      // 2^21
__device__ __forceinline__ float safe_max(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ bool is_near(float m, float c) { return fabsf(m * c) < kFar; }
__device__ __forceinline__ float reference(float m, float c) { return fmaxf(m * c, -2.f * kFar); }   // a thread far below the row's maximum adds nothing
__device__ __forceinline__ float delta(float m, float c, float R) { return fmaf(-m, c, R); }   // d from m less d from R
template <bool NEAR> struct Expo {
  uint64_t a, b;
  __device__ __forceinline__ Expo(float ref, float c) : a(pack2(c, c)), b(pack2(-ref, -ref)) {}   // ref: R near, m far
  __device__ __forceinline__ uint64_t operator()(uint64_t x) const { return NEAR ? fma2(x, a, b) : mul2(add2(x, b), a); }
};
__device__ __forceinline__ uint64_t exp2_pair(uint64_t d) {
  float a, b;
  unpack2(d, a, b);
  return pack2(exp2_fast(a), exp2_fast(b));
}
__device__ __forceinline__ float sum_pair(uint64_t v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}
// What the parts of a row know of it, and what the whole row comes to.
struct Part { float m, s, t; };
struct Stat { float m, L, H, s; };
// Sums whose exponents were too small by delta, against m.
template <typename S> __device__ __forceinline__ Part part_of(float m, const S& sums, float delta) {
  const float s = sum_pair(add2(sums.s[0], sums.s[1])), t = sum_pair(add2(sums.t[0], sums.t[1]));
  if (s == 0.f) return {m, 0.f, 0.f};
  const float f = exp2_fast(delta);
  return {m, s * f, fmaf(delta, s, t) * f};
}
template <bool ENT> __device__ __forceinline__ Stat stat_of(float m, float s, float t) {
  if (s > 0.f && s < 1.f) s = 1.f;      // rounding: the largest logit alone adds 1, and no log probability is above 0
  Stat r{m, logf(s), 0.f, s};
  if (ENT && s != 0.f) {
    r.H = r.L - kLn2 * (t / s);
    if (r.H < 0.f) r.H = 0.f;
  }
  return r;
}
// Two sets of elements, each with its sums against its own maximum, against a common one.  s = 0: nothing but -inf, its maximum means nothing.
template <bool ENT> __device__ __forceinline__ Part against(const Part& p, float m, float c) {
  const float up = (safe_max(p.m) - safe_max(m)) * c, f = p.s == 0.f ? 0.f : exp2_fast(up);
  return {m, p.s * f, ENT && f != 0.f ? fmaf(p.s, up, p.t) * f : 0.f};
}
// The union of a warp's sets, in every lane.
template <bool ENT> __device__ __forceinline__ Part warp_union(const Part& mine, float c) {
  Part r = against<ENT>(mine, warp_max(mine.m), c);
  r.s = warp_sum(r.s);
  if (ENT) r.t = warp_sum(r.t);
  return r;
}

}  // namespace logits_detail
}  // namespace fv

// Pieces of a row of bf16 or fp32 values on their way between memory and fp32 registers, two values in a register pair.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace {

template <int BYTES> struct Word;
template <> struct Word<16> { using type = uint4; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<4> { using type = unsigned; };
template <> struct Word<2> { using type = unsigned short; };
template <class T, int CH> using Chunk = typename Word<sizeof(T) * CH>::type;

// Two fp32 values in one 64-bit register: the arithmetic below takes an instruction for both.
using F2 = float2;
__device__ __forceinline__ F2 two(float lo, float hi) { return make_float2(lo, hi); }
__device__ __forceinline__ float low(F2 v) { return v.x; }
__device__ __forceinline__ float high(F2 v) { return v.y; }
__device__ __forceinline__ F2 mul(F2 a, F2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) { return __ffma2_rn(a, b, c); }

// A chunk as pairs of neighbouring channels (CH = 1: one value and a zero).
__host__ __device__ constexpr int pairs_of(int ch) { return (ch + 1) / 2; }
template <class T, int CH>
__device__ __forceinline__ void unpack(const Chunk<T, CH>& c, F2 (&v)[pairs_of(CH)]) {
  if constexpr (sizeof(T) == 4) {
    const float* f = reinterpret_cast<const float*>(&c);
#pragma unroll
    for (int i = 0; i < pairs_of(CH); ++i) v[i] = two(f[2 * i], CH > 1 ? f[2 * i + 1] : 0.f);
  } else if constexpr (CH == 1) {
    v[0] = two(__uint_as_float((unsigned)c << 16), 0.f);
  } else {
    const unsigned* h = reinterpret_cast<const unsigned*>(&c);
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) v[i] = two(__uint_as_float(h[i] << 16), __uint_as_float(h[i] & 0xffff0000u));
  }
}
// (the one rounding of the operators with bf16 tensors)
template <class T, int CH>
__device__ __forceinline__ Chunk<T, CH> pack(const F2 (&v)[pairs_of(CH)]) {
  Chunk<T, CH> c;
  if constexpr (sizeof(T) == 4) {
    float* f = reinterpret_cast<float*>(&c);
#pragma unroll
    for (int i = 0; i < CH; ++i) f[i] = i & 1 ? high(v[i / 2]) : low(v[i / 2]);
  } else if constexpr (CH == 1) {
    const __nv_bfloat16 h = __float2bfloat16_rn(low(v[0]));
    c = *reinterpret_cast<const unsigned short*>(&h);
  } else {
    unsigned* h = reinterpret_cast<unsigned*>(&c);
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {
      const __nv_bfloat162 w = __floats2bfloat162_rn(low(v[i]), high(v[i]));
      h[i] = *reinterpret_cast<const unsigned*>(&w);
    }
  }
  return c;
}

// A thread's own piece of memory into its own place in shared memory, asynchronously (`on` false: zeros).
template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from, bool on) {
  const unsigned at = (unsigned)__cvta_generic_to_shared(to), n = on ? BYTES : 0;
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(from), "r"(n) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(at), "l"(from), "r"(n), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

}  // namespace

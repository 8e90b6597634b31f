// What the row kernels of the attentions over the 8-bit and the 4-bit cache share: segments of cut work, ring waits, query rows.
#pragma once

#include "quant_common.cuh"

namespace echokv {

struct QaDesc {                                   // an item cut at the end of CTA g's share
  int n_parts;                                    // CTAs that hold parts of it (0: none starts here)
  int b, tile, h;
};

struct QaSeg {
  unsigned long long item;                        // first unit of the item
  unsigned long long item_end;
  int b, tile, h;
  int valid, starts, ends;
};

__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
// bounded wait of a whole warp on a copy's barrier
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long start = clock64();
  while (clock64() - start < kWaitLimitCycles) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
  }
  return false;
}

// n / d, mostly of numbers that fit 32 bits (a 64-bit division is long)
__device__ __forceinline__ unsigned long long quotient(unsigned long long n, unsigned long long d) {
  return ((n | d) >> 32) == 0 ? (unsigned long long)((uint32_t)n / (uint32_t)d) : n / d;
}

// four consecutive elements of a row in the storage type
template <typename T>
struct Quad;
template <>
struct Quad<__nv_bfloat16> {
  uint2 w;
  static constexpr int kPerLoad = 2;               // quads of one 16-byte load
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void zero() { w = make_uint2(0u, 0u); }
  __device__ __forceinline__ static void load16(const __nv_bfloat16* p, Quad* q) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    q[0].w = make_uint2(v.x, v.y);
    q[1].w = make_uint2(v.z, v.w);
  }
  __device__ __forceinline__ static void zero16(Quad* q) {
    q[0].zero();
    q[1].zero();
  }
  __device__ __forceinline__ float get(int e) const {
    const uint32_t x = e < 2 ? w.x : w.y;
    return __uint_as_float(e & 1 ? x & 0xffff0000u : x << 16);
  }
  // magnitudes compare as integers, infinities and NaN above everything finite (a pair of them at once here)
  __device__ __forceinline__ uint32_t top(uint32_t t) const {
    return __vmaxu2(t, __vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu));
  }
  __device__ __forceinline__ static uint32_t top_bits(uint32_t t) { return max(t & 0xffff0000u, t << 16); }
};
template <>
struct Quad<float> {
  uint4 w;
  static constexpr int kPerLoad = 1;
  __device__ __forceinline__ void load(const float* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { w = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ static void load16(const float* p, Quad* q) { q->load(p); }
  __device__ __forceinline__ static void zero16(Quad* q) { q->zero(); }
  __device__ __forceinline__ float get(int e) const { return __uint_as_float(e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w); }
  __device__ __forceinline__ uint32_t top(uint32_t t) const {
    return max(max(t, w.x & 0x7fffffffu), max(w.y & 0x7fffffffu, max(w.z & 0x7fffffffu, w.w & 0x7fffffffu)));
  }
  __device__ __forceinline__ static uint32_t top_bits(uint32_t t) { return t; }
};
// fp16 operands of a pair: the rounded one and what it leaves, times low_up (a power of two)
struct HalfPair {
  uint32_t hi, lo;
};
template <bool LOW>
__device__ __forceinline__ HalfPair split_pair(float x0, float x1, float low_up = 1.f) {
  HalfPair p;
  p.hi = h2(x0, x1);
  p.lo = 0u;
  if (LOW) {
    const float2 w = h2_float(p.hi);
    p.lo = h2((x0 - w.x) * low_up, (x1 - w.y) * low_up);
  }
  return p;
}

// transposes an 8 x 8 matrix of 16-bit elements held as matrix fragments
__device__ __forceinline__ uint32_t movm(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16(x); }

}  // namespace echokv

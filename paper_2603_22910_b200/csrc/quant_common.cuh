// What the kernels over the 8-bit cache share: the sequences of a call, codes to fp16, the score transforms.
#pragma once

#include <cuda_fp16.h>

#include "ptx_sm100.cuh"
#include "serving.h"

namespace echokv {

// One sequence of a call.  error != 0: nothing is attended; rows [first, first + n) of out are zeroed where n > 0.
struct QuantSeq {
  int slot, len, first, n, error;
};

__device__ __forceinline__ QuantSeq quant_seq(const QuantAttnArgs& a, int b) {
  // (everything that is read is asked for at once)
  const int c0 = a.cu ? a.cu[b] : b, c1 = a.cu ? a.cu[b + 1] : b + 1, slot = a.slots ? a.slots[b] : b, len = a.lens[b];
  QuantSeq s;
  s.slot = slot;
  s.len = len;
  s.error = 0;
  if (c0 < 0 || c1 < c0 || c1 > a.n_tokens) {
    s.error = ECHOKV_EBADLENGTH;
    s.first = 0;
    s.n = 0;
    return s;
  }
  s.first = c0;
  s.n = c1 - c0;
  if (s.n > 0) {
    if (slot < 0 || slot >= a.g.max_batch) s.error = ECHOKV_EBADPAGE;
    else if (len < s.n || len > a.g.max_pages * a.g.page_tokens || s.n > a.max_new) s.error = ECHOKV_EBADLENGTH;
  }
  return s;
}

// Which of the two attention kernels takes the sequences of many query rows (chunk_rows of them per KV head and more)?  Both cut
// the work of all sequences into equal shares: the row kernel in units of 16 keys x 8 query rows, the chunk kernel in tiles of
// 128 keys of items of 256 query rows, with a cost of 4 tiles to an item.  Measured (32 / 8 heads of 128, int8): by rows 15 us + 92
// ns for every unit of an SM; by chunks 28 us (two more launches, longer start) + 0.30 us for every 16 keys of an item on an
// SM.  (One sequence over 8192 keys: 16 tokens 38 us by rows, 40 by chunks, 32 tokens 57 and 40, 128 tokens 172 and 49; over
// 1024 keys, 64 tokens 30 and 30; 8 sequences over 32768 keys, 64 tokens: 2560 and 322.)  Both kernels compute the answer from
// the lengths, every thread of a block the same one.
constexpr int kCkItemCost = 4;                     // in tiles of 128 keys: queries, first tile, result
__device__ __forceinline__ bool many_rows(const QuantAttnArgs& a, const QuantSeq& s) {
  return a.chunk_rows > 0 && !s.error && (long long)s.n * a.group >= a.chunk_rows;
}
__device__ __forceinline__ bool take_chunks(const QuantAttnArgs& a, int sm_count) {
  if (a.chunk_rows == 0) return false;
  __shared__ unsigned long long sums[32][2];       // a warp's units by rows, by chunks
  unsigned long long by_rows = 0, by_chunks = 0;
  for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
    const QuantSeq s = quant_seq(a, b);
    if (!many_rows(a, s)) continue;
    const unsigned long long rows = (unsigned long long)s.n * a.group, blocks = (s.len + kQuantBlock - 1) / kQuantBlock;
    by_rows += (rows + 7) / 8 * blocks * a.g.n_kv_heads;
    by_chunks += (rows + 255) / 256 * (blocks + 8 * kCkItemCost) * a.g.n_kv_heads;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    by_rows += __shfl_xor_sync(0xffffffffu, by_rows, o);
    by_chunks += __shfl_xor_sync(0xffffffffu, by_chunks, o);
  }
  if ((threadIdx.x & 31) == 0) {
    sums[threadIdx.x >> 5][0] = by_rows;
    sums[threadIdx.x >> 5][1] = by_chunks;
  }
  __syncthreads();
  by_rows = by_chunks = 0;
#pragma unroll 1
  for (unsigned w = 0; w < blockDim.x / 32; ++w) {
    by_rows += sums[w][0];
    by_chunks += sums[w][1];
  }
  return 10 * by_rows > 1400ull * sm_count + 33 * by_chunks;
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// tanh to ~3e-7 of its value: away from 0 by 1 - 2 / (e^{2y} + 1), near 0 (where that form cancels) by the Taylor series
// y - y^3/3 + 2 y^5/15 - 17 y^7/315 + 62 y^9/2835, whose next term is 1.5e-8 of y at 0.25
__device__ __forceinline__ float tanh_f32(float y) {
  const float y2 = y * y;
  float s = 62.f / 2835.f;
  s = fmaf(s, y2, -17.f / 315.f);
  s = fmaf(s, y2, 2.f / 15.f);
  s = fmaf(s, y2, -1.f / 3.f);
  s = fmaf(s * y2, y, y);
  const float e = exp2_approx(fabsf(y) * (2.f * kLog2e));      // +inf for large |y|: the quotient is 0
  const float t = copysignf(fmaf(-2.f, rcp_approx(e + 1.f), 1.f), y);
  return y2 < 0.0625f ? s : t;
}

// fp16 pair
__device__ __forceinline__ uint32_t h2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 h2_float(uint32_t w) {
  const __half2 v = *reinterpret_cast<const __half2*>(&w);
  return __half22float2(v);
}

// Codes -> fp16, exactly.  int8: 1024 + (c + 128) has the byte c ^ 0x80 as the low bits of its fp16 pattern 0x6400 | u; subtracting
// 1152 leaves c.  e4m3: the conversion instruction.
template <int FMT>
__device__ __forceinline__ uint32_t codes_bias(uint32_t w) { return FMT == ECHOKV_INT8 ? w ^ 0x80808080u : w; }
// bytes (lo, hi) = (0, 1) or (2, 3) of a word that went through codes_bias
template <int FMT, int HALF>
__device__ __forceinline__ uint32_t codes_pair(uint32_t w) {
  uint32_t r;
  if (FMT == ECHOKV_INT8) {
    const uint32_t x = __byte_perm(w, 0x64646464u, HALF ? 0x4342 : 0x4140);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0x64806480u));
  } else {
    const uint16_t x = (uint16_t)(HALF ? w >> 16 : w & 0xffffu);
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(x));
  }
  return r;
}

__device__ __forceinline__ void mma_m16n8k16_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                 uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Operands in the storage type are scaled by a power of two that takes their largest magnitude m to [2^14, 2^15): a bf16
// then is an fp16 exactly down to 2^-31 of the largest.  Returns that power for m in fp32's normal range (else 1: zero, or an
// infinity or NaN that the products carry on) and its inverse.
__device__ __forceinline__ float scale_up_to_half(float m, float* inverse) {
  const int e = (int)(__float_as_uint(m) >> 23) & 0xff;
  int k = 127 + 14 - e;                        // 2^k * m in [2^14, 2^15)
  if (e == 0 || e == 255) k = 0;
  k = k > 126 ? 126 : k < -126 ? -126 : k;
  *inverse = __uint_as_float((uint32_t)(127 - k) << 23);
  return __uint_as_float((uint32_t)(127 + k) << 23);
}

}  // namespace echokv

// What the kernels over the 4-bit cache share: codes and scales to fp16 and back.
#pragma once

#include "quant_common.cuh"

namespace echokv {

// byte 0 of w (two e2m1 codes) -> fp16 pair, low half first; exact
__device__ __forceinline__ uint32_t e2m1_pair(uint32_t w) {
  uint32_t r;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
// all four bytes
__device__ __forceinline__ void e2m1_bytes(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\tcvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// two e4m3 scales (low 16 bits) -> fp16 pair; exact
__device__ __forceinline__ uint32_t e4m3_scales(uint32_t w) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
  return r;
}
// the low halves of a's bytes and of b's << 4 (b given shifted), or the high halves of a's (given shifted) and of b's
__device__ __forceinline__ uint32_t fp4_zip(uint32_t low, uint32_t high) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xe4;" : "=r"(r) : "r"(low), "r"(high), "r"(0x0f0f0f0fu));      // low & m | high & ~m
  return r;
}
__device__ __forceinline__ uint32_t fp4_mul(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// two fp32 -> a byte of two e2m1 codes (to nearest even, at most 6), lo in its low half
__device__ __forceinline__ uint32_t e2m1_byte(float lo, float hi) {
  uint32_t r;
  asm("{\n\t.reg .b8 b;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n\tcvt.u32.u8 %0, b;\n\t}" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// fp32 >= 0 -> e4m3 (to nearest even, at most 448)
__device__ __forceinline__ uint32_t e4m3_code(float x) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
  return r & 0xffu;
}
constexpr uint32_t kE4m3Nan = 0x7fu;

// A kernel whose blocks may be there before the one before it on the stream has ended.  It begins with after_the_one_before(), behind which
// everything that was written before is seen; where it lets its own successor come early, it does so after that.  (A call's second kernel
// may read the call's inputs sooner: the first one has waited for them before it let the second one come.)
template <typename... P, typename... A>
inline cudaError_t launch_early(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
__device__ __forceinline__ void after_the_one_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_the_next_one_come() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace echokv

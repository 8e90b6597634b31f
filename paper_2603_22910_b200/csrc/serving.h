// Host-side launchers of the serving-step kernels (internal to the library): plan, rotation, 8-bit append, 8-bit attention.
#pragma once

#include <atomic>

#include "common.cuh"

namespace echokv {

constexpr int kPlanMaxBatch = 8192;                 // sequences of one plan: 20 bytes of shared memory each
constexpr int kQuantBlock = ECHOKV_QUANT_BLOCK_TOKENS;
constexpr int kMaxAxes = 4;

__device__ __forceinline__ void report_opt(int32_t* status, int code) {
  if (status != nullptr) atomicCAS(status, 0, code);
}

// 16 bytes of elements from fp32
template <typename T>
__device__ __forceinline__ void store16(T* p, const float* v);
template <>
__device__ __forceinline__ void store16<float>(float* p, const float* v) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
template <>
__device__ __forceinline__ void store16<__nv_bfloat16>(__nv_bfloat16* p, const float* v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// The shared memory that `kernel` may ask for at a launch on the current device: set once per device and kernel (one `done` each).
template <typename K>
inline cudaError_t allow_smem(K* kernel, size_t bytes, std::atomic<unsigned long long>* done) {
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (device & 63);
  if (done->load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) done->fetch_or(bit, std::memory_order_relaxed);
  return e;
}

struct PlanArgs {
  int32_t* table;
  const int32_t* slots;        // [B] or null
  const int32_t* lens;
  const int32_t* new_lens;
  const int32_t* free_pages;
  const int32_t* free_count;
  int B, n_tokens;
  int page_tokens, page_shift, max_pages, max_batch;
  long long n_pages;
  echokv_step_plan out;
  int32_t* status;
};
cudaError_t launch_plan(const PlanArgs& a, cudaStream_t stream);

struct ReleaseArgs {
  const int32_t* table;
  const int32_t* slots;
  const int32_t* lens;
  int32_t* free_pages;
  int32_t* free_count;
  int B, page_tokens, page_shift, max_pages, max_batch;
  long long n_pages;
  int32_t* status;
};
cudaError_t launch_release(const ReleaseArgs& a, cudaStream_t stream);

struct RotateArgs {
  const void* in[2];           // q, k (null: nothing to do)
  void* out[2];
  long long in_stride[2], out_stride[2];   // elements
  int heads[2];
  int head_dim, rot_dim, n_tokens, dtype;
  bool in_place[2];
  const int32_t* pos;          // [n_axes][n_tokens]
  float sign;
  unsigned char axis[64];      // axis of every frequency index
  double turns[64];            // theta^(-2 j / rot) / (2 pi)
};
cudaError_t launch_rotate(const RotateArgs& a, int sm_count, cudaStream_t stream);

// Geometry of one layer's 8-bit (or 4-bit) cache, by value into kernels.
struct QuantGeom {
  unsigned char* blocks;       // 4 bits: [n_pages][H][P / 16] blocks of 18 d bytes (the next three are not used then)
  unsigned char* codes[2];     // K, V: [n_pages][H][P][d]
  float* scales[2];            // [n_pages][H][P / 16]
  void* tail[2];               // [max_batch][H][16][d]
  int n_kv_heads, head_dim, page_tokens, page_shift, max_pages, max_batch;
  long long n_pages;
};

struct QuantAppendArgs {
  QuantGeom g;
  const void* x[2];            // new K, V rows
  long long stride[2];         // elements
  const int64_t* slot_map;
  const int32_t* token_seqs;
  const int32_t* cu;
  const int32_t* slots;        // or null
  int B, n_tokens, dtype, format;
  int32_t* status;
};
cudaError_t launch_quant_append(const QuantAppendArgs& a, int sm_count, cudaStream_t stream);

struct QuantAttnArgs {
  QuantGeom g;
  const void* q;
  long long q_stride;          // elements
  void* out;
  const int32_t* table;
  const int32_t* slots;        // or null
  const int32_t* lens;
  const int32_t* cu;           // or null: one token per sequence
  const float* slopes;         // or null
  const int32_t* prefix;       // or null
  int B, n_tokens, max_new;
  int n_q_heads, group, group_shift, dtype, format;
  int chunk_rows;              // sequences with at least this many query rows per KV head (new tokens x group) can be the
                               // chunk kernel's; 0: there is none (see take_chunks)
  int sm_count;
  float scale, softcap;
  float out_scale;             // 4 bits: what the output is multiplied by
  unsigned char* ws;
  int32_t* status;
};
uint64_t quant_attn_workspace_bytes(int head_dim);
cudaError_t launch_quant_attn(const QuantAttnArgs& a, int sm_count, cudaStream_t stream);
// the sequences with chunk_rows query rows and more (bf16)
uint64_t quant_chunk_workspace_bytes(int head_dim);
cudaError_t launch_quant_chunk(const QuantAttnArgs& a, int sm_count, cudaStream_t stream);

// ---- the cache held in 4 bits -------------------------------------------------------------------------------------
constexpr int kFp4 = 2;                             // QuantAttnArgs.format of it (beside ECHOKV_INT8, ECHOKV_E4M3)
constexpr int kFp4Group = ECHOKV_FOURBIT_GROUP;
__host__ __device__ constexpr int fp4_block_bytes(int d) { return 18 * d; }
// byte offsets in a block: K codes, V codes, K scales, V scales
__host__ __device__ constexpr int fp4_k_at(int d, int tok, int f) { return tok * (d / 2) + f / 2; }
__host__ __device__ constexpr int fp4_v_at(int d, int tok, int f) {
  return 8 * d + (((tok / 8 * 8 + f / (d / 8)) * 4 + tok / 2 % 4) * 2 + tok % 2) * (d / 16) + f % (d / 8) / 2;
}
__host__ __device__ constexpr int fp4_ks_at(int d, int tok, int f) { return 16 * d + tok * (d / 16) + f / 16; }
__host__ __device__ constexpr int fp4_vs_at(int d, int tok, int f) { return 17 * d + f / 16 * 16 + tok; }

struct Fp4Geom {
  unsigned char* blocks;
  int8_t* bounds;              // or null
  float* bound_scales;
  int n_kv_heads, head_dim, page_tokens, page_shift, max_pages, max_batch;
  long long n_pages;
};

struct Fp4AppendArgs {
  Fp4Geom g;
  const void* q;               // or null
  void* q_out;
  const void* x[2];            // new K, V rows
  long long q_stride, q_out_stride, stride[2];   // elements
  const int32_t* pos;          // [n_axes][n_tokens], or null: no rotation
  const int64_t* slot_map;
  int n_q_heads, n_tokens, dtype, rot_dim;
  float unit6[2], inv_unit[2]; // 1 / (6 unit), 1 / unit
  int32_t* status;
  unsigned char axis[64];      // axis of every frequency index
  double turns[64];            // theta^(-2 j / rot) / (2 pi)
};
cudaError_t launch_fp4_append(const Fp4AppendArgs& a, int sm_count, cudaStream_t stream);

struct Fp4ReadArgs {
  Fp4Geom g;
  const int64_t* slot_map;
  void* out[2];                // or null
  long long stride[2];         // elements
  float unit[2];
  int n_tokens, dtype;
  int32_t* status;
};
cudaError_t launch_fp4_read(const Fp4ReadArgs& a, cudaStream_t stream);

// Tokens as queries of their own: sequence and position of each.
struct Fp4Tokens {
  const int32_t* seqs;         // [n_tokens]
  const int32_t* positions;
  const int32_t* pages;        // [n_tokens][H][n_select]
  int n_select;
};

struct Fp4SelectArgs {
  Fp4Geom g;
  const void* q;
  long long q_stride;
  const int32_t* table;
  const int32_t* slots;        // or null
  Fp4Tokens t;
  int32_t* out;
  int B, n_tokens, n_first, n_recent, n_q_heads, group, group_shift, dtype;
  unsigned char* ws;
  int32_t* status;
};
uint64_t fp4_select_workspace_bytes();
cudaError_t launch_fp4_select(const Fp4SelectArgs& a, int sm_count, cudaStream_t stream);

struct Fp4AttnArgs : QuantAttnArgs {
  Fp4Tokens t;                 // t.seqs null: the whole cache, by sequences
};
uint64_t fp4_attn_workspace_bytes(int head_dim);
cudaError_t launch_fp4_attn(const Fp4AttnArgs& a, int sm_count, cudaStream_t stream);

}  // namespace echokv

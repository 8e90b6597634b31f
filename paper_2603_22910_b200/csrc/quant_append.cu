// Append to a cache held in 8 bits: a scale for each block of 16 tokens and KV head.
//
// The work is bytes: every new row is read once, every completed block written once in half (a quarter) of the bytes.  One warp
// takes one (block, head, K or V): a lane holds head_dim / 32 elements of each of the 16 rows, all 16 loads in
// flight at once, the largest magnitude by one warp reduction, the codes go back 128 contiguous bytes a row.
// A CTA looks at 16 consecutive new tokens of the step; the tokens in it that end a block (the last row of a block, or the last
// token of its sequence) are the work, times the heads, times K and V, spread over the CTA's warps (and over the
// grid's second axis when the step has few tokens).
//
// The tail.  Rows of an open block wait in the storage type.  If a sequence's new tokens complete its open block AND leave
// a new one open, the old tail rows must be read before the new ones overwrite them: both blocks are then done by the
// same warp, that of the last token, in this order.  No other pair of work items touches the same tail rows.
#include "serving.h"

namespace echokv {

namespace {

constexpr int kAppendWarps = 8;

// N consecutive elements of a row held by one lane, as fp32
template <typename T, int N>
struct Piece;
template <>
struct Piece<__nv_bfloat16, 4> {
  __device__ static void load(const __nv_bfloat16* p, float* v) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
    v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
  }
};
template <>
struct Piece<__nv_bfloat16, 2> {
  __device__ static void load(const __nv_bfloat16* p, float* v) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
    v[0] = __uint_as_float(w << 16); v[1] = __uint_as_float(w & 0xffff0000u);
  }
};
template <>
struct Piece<float, 4> {
  __device__ static void load(const float* p, float* v) {
    const float4 w = *reinterpret_cast<const float4*>(p);
    v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
  }
};
template <>
struct Piece<float, 2> {
  __device__ static void load(const float* p, float* v) {
    const float2 w = *reinterpret_cast<const float2*>(p);
    v[0] = w.x; v[1] = w.y;
  }
};

// two fp32 values -> two e4m3 codes, round to nearest even, in range by construction
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int FMT, int N>
__device__ __forceinline__ uint32_t encode(const float* v, float inv) {
  uint32_t w = 0;
  if (FMT == ECHOKV_INT8) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int c = max(-127, min(127, __float2int_rn(v[e] * inv)));
      w |= (uint32_t)(c & 0xff) << (8 * e);
    }
  } else {
    float y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = v[e] * inv;
#pragma unroll
    for (int e = 0; e < N; e += 2) w |= e4m3_pair(y[e], y[e + 1]) << (8 * e);
  }
  return w;
}

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(kAppendWarps * 32) quant_append_kernel(const __grid_constant__ QuantAppendArgs a) {
  constexpr int N = D / 32;                 // elements of a row per lane
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const QuantGeom& g = a.g;
  const int w0 = blockIdx.x * kQuantBlock;  // first token of the CTA's window
  const long long n_rows = g.n_pages * g.page_tokens;

  // lane i < 16 describes token w0 + i
  const int t = w0 + lane;
  long long row = -1;
  int seq = -1, slot = -1, c0 = 0, c1 = 0;
  bool end = false;
  if (lane < kQuantBlock && t < a.n_tokens) {
    row = a.slot_map[t];
    if (row != -1) {
      seq = a.token_seqs[t];
      bool ok = row >= 0 && row < n_rows && seq >= 0 && seq < a.B;
      if (ok) {
        slot = a.slots ? a.slots[seq] : seq;
        c0 = a.cu[seq];
        c1 = a.cu[seq + 1];
        ok = slot >= 0 && slot < g.max_batch && c0 >= 0 && c0 <= t && c1 > t && c1 <= a.n_tokens;
      }
      if (!ok) {
        report_opt(a.status, ECHOKV_EBADPAGE);
        row = -1;
      }
      end = ok && ((row & (kQuantBlock - 1)) == kQuantBlock - 1 || t == c1 - 1);
    }
  }
  const uint32_t ends = __ballot_sync(0xffffffffu, end);
  if (ends == 0) return;
  const int per_end = 2 * g.n_kv_heads, n_items = __popc(ends) * per_end;

  for (int item = blockIdx.y * kAppendWarps + warp; item < n_items; item += gridDim.y * kAppendWarps) {
    const int which_end = item / per_end, hk = item - which_end * per_end, kv = hk & 1, h = hk >> 1;
    uint32_t left = ends;
    for (int i = 0; i < which_end; ++i) left &= left - 1;
    const int src = __ffs(left) - 1;
    const int te = w0 + src;
    const long long re = __shfl_sync(0xffffffffu, row, src);
    const int first = __shfl_sync(0xffffffffu, c0, src), last = __shfl_sync(0xffffffffu, c1, src) - 1;
    const int my_slot = __shfl_sync(0xffffffffu, slot, src);
    const int r0 = (int)(re & (kQuantBlock - 1));
    // new tokens of this block: the run of consecutive rows that ends here
    const auto run_length = [&](int t_end, long long r_end) {
      const int inside = (int)(r_end & (kQuantBlock - 1));
      bool same = false;
      if (lane <= inside && t_end - lane >= first) same = a.slot_map[t_end - lane] == r_end - lane;
      const uint32_t m = ~__ballot_sync(0xffffffffu, same);
      return m == 0 ? 32 : __ffs(m) - 1;
    };
    const T* x = static_cast<const T*>(a.x[kv]);
    T* tail = static_cast<T*>(g.tail[kv]) + ((long long)my_slot * g.n_kv_heads + h) * kQuantBlock * D;

    // quantise the block whose last row is r_end, the new token t_end; its first 16 - n rows come from the tail
    const auto quantise = [&](int t_end, long long r_end, int n) {
      float v[kQuantBlock][N];
#pragma unroll
      for (int j = 0; j < kQuantBlock; ++j) {
        const T* p = j >= kQuantBlock - n ? x + (long long)(t_end - (kQuantBlock - 1) + j) * a.stride[kv] + h * D : tail + j * D;
        Piece<T, N>::load(p + lane * N, v[j]);
      }
      // magnitudes compare as integers, infinities and NaN above everything finite
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < kQuantBlock; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(v[j][e]) & 0x7fffffffu);
      top = __reduce_max_sync(0xffffffffu, top);
      const bool finite = top < 0x7f800000u;
      // the scale is part of what the cache stores: its roundings are the ones the interface states (one product, one
      // division to nearest), whatever the compiler's fast-math setting
      const float scale = finite ? fmaxf(__fmul_rn(__uint_as_float(top), FMT == ECHOKV_INT8 ? 1.0f / 127.0f : 1.0f / 448.0f),
                                         7.8886090522101181e-31f)
                                 : __uint_as_float(0x7fc00000u);
      const float inv = __fdiv_rn(1.0f, scale);
      const long long page = r_end >> g.page_shift;
      const int inside = (int)(r_end & (g.page_tokens - 1)) - (kQuantBlock - 1);
      unsigned char* codes = g.codes[kv] + ((page * g.n_kv_heads + h) * g.page_tokens + inside) * D + lane * N;
#pragma unroll
      for (int j = 0; j < kQuantBlock; ++j) {
        const uint32_t w = finite ? encode<FMT, N>(v[j], inv) : 0u;
        if (N == 4) *reinterpret_cast<uint32_t*>(codes + j * D) = w;
        else *reinterpret_cast<uint16_t*>(codes + j * D) = (uint16_t)w;
      }
      if (lane == 0) g.scales[kv][(page * g.n_kv_heads + h) * (g.page_tokens / kQuantBlock) + inside / kQuantBlock] = scale;
    };

    const int n = run_length(te, re);
    // the sequence's first block of this step: does it start in the tail, and where does it end
    const long long rf = a.slot_map[first], rl = a.slot_map[last];
    const int off = (int)(rf & (kQuantBlock - 1)), t_first_end = first + (kQuantBlock - 1) - off;
    const bool leaves_open = rl >= 0 && (rl & (kQuantBlock - 1)) != kQuantBlock - 1;
    if (r0 == kQuantBlock - 1) {
      // (a first block that starts in the tail is left to the warp of the last token if that one writes the tail)
      const bool deferred = rf >= 0 && off > 0 && te == t_first_end && leaves_open;
      if (!deferred) quantise(te, re, n);
    } else {
      // (te is the sequence's last token)
      if (rf >= 0 && off > 0 && t_first_end < te) {
        const long long r_end = a.slot_map[t_first_end];
        if (r_end == rf + (kQuantBlock - 1) - off) {
          quantise(t_first_end, r_end, run_length(t_first_end, r_end));
          __syncwarp();
        }
      }
      for (int j = r0 - n + 1; j <= r0; ++j) {
        const T* p = x + (long long)(te - r0 + j) * a.stride[kv] + h * D;
        if (N * sizeof(T) == 16) *reinterpret_cast<uint4*>(tail + j * D + lane * N) = *reinterpret_cast<const uint4*>(p + lane * N);
        else if (N * sizeof(T) == 8) *reinterpret_cast<uint2*>(tail + j * D + lane * N) = *reinterpret_cast<const uint2*>(p + lane * N);
        else *reinterpret_cast<uint32_t*>(tail + j * D + lane * N) = *reinterpret_cast<const uint32_t*>(p + lane * N);
      }
    }
  }
}

template <typename T, int FMT, int D>
cudaError_t launch(const QuantAppendArgs& a, int sm_count, cudaStream_t stream) {
  const int windows = (a.n_tokens + kQuantBlock - 1) / kQuantBlock;
  // enough warps to fill the machine with one item each where the step is small: a window of a decode step holds up
  // to 16 ends x 2 H items
  int gy = (4 * sm_count + windows - 1) / windows;
  const int most = (kQuantBlock * 2 * a.g.n_kv_heads + kAppendWarps - 1) / kAppendWarps;
  gy = gy < 1 ? 1 : gy > most ? most : gy;
  quant_append_kernel<T, FMT, D><<<dim3((unsigned)windows, (unsigned)gy), kAppendWarps * 32, 0, stream>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_t(const QuantAppendArgs& a, int sm_count, cudaStream_t stream) {
  const bool i8 = a.format == ECHOKV_INT8;
  if (a.g.head_dim == 128) return i8 ? launch<T, ECHOKV_INT8, 128>(a, sm_count, stream) : launch<T, ECHOKV_E4M3, 128>(a, sm_count, stream);
  return i8 ? launch<T, ECHOKV_INT8, 64>(a, sm_count, stream) : launch<T, ECHOKV_E4M3, 64>(a, sm_count, stream);
}

}  // namespace

cudaError_t launch_quant_append(const QuantAppendArgs& a, int sm_count, cudaStream_t stream) {
  return a.dtype == ECHOKV_BF16 ? launch_t<__nv_bfloat16>(a, sm_count, stream) : launch_t<float>(a, sm_count, stream);
}

}  // namespace echokv

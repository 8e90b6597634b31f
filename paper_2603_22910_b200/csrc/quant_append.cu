// Append to a cache held in 8 bits: a scale for each block of 16 tokens and KV head.
//
// The work is bytes: every new row is read once, every completed block written once in half (a quarter) of the bytes.  One warp
// takes one (block, head, K or V): a lane holds head_dim / 32 elements of each of the 16 rows, all 16 loads in flight at once,
// the largest magnitude by one warp reduction, the codes go back 128 contiguous bytes a row.  (K and V by one warp, 32 loads in
// flight at half the warps: 46 against 44 us for 33 thousand tokens, 5.6 against 4.3 us for a decode step.)
// Measured: 33 thousand tokens of 8 bf16 heads of 128 in 43 us (198 MB, 4.6 TB/s), a decode step of 64 tokens in 4.4 us.  What
// keeps it from the memory's rate: a warp's 16 loads are all it has in flight until its block is reduced and written.
// (2, 4 and 16 warps per CTA: 79, 54 and 43.4 us; 3 CTAs per SM instead of 4: 46.6.)
// A CTA looks at 16 consecutive new tokens of the step; the tokens in it that end a block (the last row of a block, or the last
// token of its sequence) are the work, times the heads, times K and V, spread over the CTA's warps (and over the grid's
// second axis when the step has few tokens).
//
// The tail.  Rows of an open block wait in the storage type.  If a sequence's new tokens complete its open block AND leave
// a new one open, the old tail rows must be read before the new ones overwrite them: both blocks are then done by the
// same warp, that of the last token, in this order.  No other pair of work items touches the same tail rows.
#include "serving.h"

namespace echokv {

namespace {

constexpr int kAppendWarps = 8;

// N consecutive elements of a row held by one lane, in W words
template <typename T, int N>
struct Piece {
  static constexpr int W = N * sizeof(T) / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (W == 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (W == 2) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x; w[1] = v.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (W == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (W == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(p) = w[0];
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
  // magnitudes compare as integers, infinities and NaN above everything finite (bf16: two of them at once)
  __device__ __forceinline__ uint32_t top(uint32_t t) const {
#pragma unroll
    for (int i = 0; i < W; ++i) t = sizeof(T) == 4 ? max(t, w[i] & 0x7fffffffu) : __vmaxu2(t, w[i] & 0x7fff7fffu);
    return t;
  }
  __device__ __forceinline__ static uint32_t top_bits(uint32_t t) { return sizeof(T) == 4 ? t : max(t & 0xffff0000u, t << 16); }
};

// two fp32 values -> two e4m3 codes, round to nearest even, in range by construction
__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// (No clamp: with inv the rounded inverse of a rounded amax / Q, |v| inv <= Q (1 + 2^-21), which rounds to Q.)
template <int FMT, int N>
__device__ __forceinline__ uint32_t encode(const float (&v)[N], float inv) {
  float y[N];
#pragma unroll
  for (int e = 0; e < N; e += 2) unpack_f2(mul_f2(pack_f2(v[e], v[e + 1]), pack_f2(inv, inv)), y[e], y[e + 1]);
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    if (FMT == ECHOKV_INT8) w |= (__byte_perm((uint32_t)__float2int_rn(y[e]), (uint32_t)__float2int_rn(y[e + 1]), 0x0040) & 0xffffu) << (8 * e);
    else w |= e4m3_pair(y[e], y[e + 1]) << (8 * e);
  }
  return w;
}

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(kAppendWarps * 32, sizeof(T) == 2 ? 4 : 2) quant_append_kernel(const __grid_constant__ QuantAppendArgs a) {
  constexpr int N = D / 32;                 // elements of a row per lane
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const QuantGeom& g = a.g;
  const int w0 = blockIdx.x * kQuantBlock;  // first token of the CTA's window
  const long long n_rows = g.n_pages * g.page_tokens;

  // lane 16 + i describes token w0 + i of the window, lane i the token 16 before it (whose row tells where a block's new
  // tokens begin).  Everything that is looked up is looked up here, for all the window's tokens at once.
  const int t = w0 - kQuantBlock + lane;
  const bool mine = lane >= kQuantBlock && t < a.n_tokens;
  const long long row = t >= 0 && t < a.n_tokens ? a.slot_map[t] : -1;
  int slot = -1, c0 = 0, c1 = 0;
  bool end = false;
  long long rf = -1, rl = -1;                  // rows of the sequence's first and last new token
  if (mine && row != -1) {
    const int seq = a.token_seqs[t];
    bool ok = row >= 0 && row < n_rows && seq >= 0 && seq < a.B;
    if (ok) {
      slot = a.slots ? a.slots[seq] : seq;
      c0 = a.cu[seq];
      c1 = a.cu[seq + 1];
      ok = slot >= 0 && slot < g.max_batch && c0 >= 0 && c0 <= t && c1 > t && c1 <= a.n_tokens;
    }
    if (!ok) report_opt(a.status, ECHOKV_EBADPAGE);
    end = ok && ((row & (kQuantBlock - 1)) == kQuantBlock - 1 || t == c1 - 1);
    if (end) {
      rf = a.slot_map[c0];
      rl = a.slot_map[c1 - 1];
      if (rf >= n_rows) rf = -1;               // (that token's own window reports it)
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
    const int te = w0 - kQuantBlock + src;
    const long long re = __shfl_sync(0xffffffffu, row, src);
    const int first = __shfl_sync(0xffffffffu, c0, src);
    const int my_slot = __shfl_sync(0xffffffffu, slot, src);
    const int r0 = (int)(re & (kQuantBlock - 1));
    const long long tail_at = ((long long)my_slot * g.n_kv_heads + h) * kQuantBlock * D + lane * N;
    // this lane's elements of a new token, and of a row of the tail
    const long long stride = a.stride[kv];
    const T* x = static_cast<const T*>(a.x[kv]) + h * D + lane * N;
    T* tail = static_cast<T*>(g.tail[kv]) + tail_at;

    // quantise the block whose last row is r_end, the new token t_end; its first 16 - n rows come from the tail
    const auto quantise = [&](int t_end, long long r_end, int n) {
      Piece<T, N> v[kQuantBlock];
      const T* fresh = x + (t_end - (kQuantBlock - 1)) * stride;
      if (n == kQuantBlock) {
#pragma unroll
        for (int j = 0; j < kQuantBlock; ++j, fresh += stride) v[j].load(fresh);
      } else {
#pragma unroll
        for (int j = 0; j < kQuantBlock; ++j, fresh += stride) v[j].load(j >= kQuantBlock - n ? fresh : tail + j * D);
      }
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < kQuantBlock; ++j) top = v[j].top(top);
      top = __reduce_max_sync(0xffffffffu, Piece<T, N>::top_bits(top));
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
        float y[N];
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = v[j].get(e);
        const uint32_t w = finite ? encode<FMT, N>(y, inv) : 0u;
        if (N == 4) *reinterpret_cast<uint32_t*>(codes + j * D) = w;
        else *reinterpret_cast<uint16_t*>(codes + j * D) = (uint16_t)w;
      }
      if (lane == 0) g.scales[kv][(page * g.n_kv_heads + h) * (g.page_tokens / kQuantBlock) + inside / kQuantBlock] = scale;
    };

    // new tokens of this block: the run of consecutive rows that ends here
    const bool same = lane <= src && lane > src - kQuantBlock && src - lane <= r0 && te - (src - lane) >= first && row == re - (src - lane);
    const int n = __clz(~(__ballot_sync(0xffffffffu, same) << (31 - src)));
    // the sequence's first block of this step: does it start in the tail, and where does it end
    const long long first_row = __shfl_sync(0xffffffffu, rf, src), last_row = __shfl_sync(0xffffffffu, rl, src);
    const int off = (int)(first_row & (kQuantBlock - 1)), t_first_end = first + (kQuantBlock - 1) - off;
    const bool leaves_open = last_row >= 0 && (last_row & (kQuantBlock - 1)) != kQuantBlock - 1;
    if (r0 == kQuantBlock - 1) {
      // (a first block that starts in the tail is left to the warp of the last token if that one writes the tail)
      const bool deferred = first_row >= 0 && off > 0 && te == t_first_end && leaves_open;
      if (!deferred) quantise(te, re, n);
    } else {
      // (te is the sequence's last token)
      if (first_row >= 0 && off > 0 && t_first_end < te - r0) {
        // its new tokens: 16 - off of them, if the rows follow one another as they should
        const long long r_end = a.slot_map[t_first_end];
        if (r_end == first_row + (kQuantBlock - 1) - off) {
          quantise(t_first_end, r_end, kQuantBlock - off);
          __syncwarp();
        }
      }
      for (int j = r0 - n + 1; j <= r0; ++j) {
        Piece<T, N> v;
        v.load(x + (te - r0 + j) * stride);
        v.store(tail + j * D);
      }
    }
  }
}

template <typename T, int FMT, int D>
cudaError_t launch(const QuantAppendArgs& a, int sm_count, cudaStream_t stream) {
  const int windows = (a.n_tokens + kQuantBlock - 1) / kQuantBlock;
  // enough warps to fill the machine with one item each where the step is small: a window of a decode step holds up
  // to 16 ends x 2 H items; two CTAs to a window at least (33 thousand tokens: 44.0 us with one, 43.0 with two, 50 with four)
  int gy = (4 * sm_count + windows - 1) / windows;
  const int most = (kQuantBlock * 2 * a.g.n_kv_heads + kAppendWarps - 1) / kAppendWarps;
  gy = gy < 2 ? 2 : gy;
  gy = gy > most ? most : gy;
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

// Append to a cache held in 8 bits: a scale for each block of 16 tokens and KV head.
//
// The work is bytes: every new row is read once, every completed block written once in half (a quarter) of the bytes.  One warp
// takes one (block, head, K or V): a lane holds head_dim / 32 elements of each of the 16 rows, all 16 loads in flight at once,
// the largest magnitude by one warp reduction, the codes go back 128 contiguous bytes a row.  (K and V by one warp, 32 loads in
// flight at half the warps: 46 against 44 us for 33 thousand tokens, 5.6 against 4.3 us for a decode step.)
// Measured: 33 thousand tokens of 8 bf16 heads of 128 in 42 us (198 MB, 4.7 TB/s), a decode step of 128 tokens in 4.3 us.  What
// keeps it from the memory's rate: a warp's 16 loads are all it has in flight until its block is reduced and written.
// (2, 4 and 16 warps per CTA: 79, 54 and 43.4 us; 3 CTAs per SM instead of 4: 46.6.)
// A CTA looks at 16 consecutive new tokens of the step; the tokens in it that end a block (the last row of a block, or the last
// token of its sequence that has a row) are the work, times the heads, times K and V, spread over the CTA's warps (and over the
// grid's second axis when the step has few tokens).  Tokens without a row may lie anywhere among a sequence's: where one is met, the
// block's others are looked for around it.
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

// What is looked for where tokens without a row (skipped, bad) lie among a sequence's; functions of their own, so that the common
// way's registers and instructions are its own.  All for a whole warp.
struct Tokens {
  const int64_t* slot_map;
  const int32_t* token_seqs;
  long long n_rows;
  // row of new token u, -1 if it has none of sequence q
  __device__ __forceinline__ long long row_of(int u, int q) const {
    const long long r = slot_map[u];
    return r >= 0 && r < n_rows && token_seqs[u] == q ? r : -1;
  }
};
struct Placed {
  int u;
  long long row;
};
// the first token in [u, until) of sequence q that has a row (until, -1: none)
__device__ __noinline__ Placed first_placed(const Tokens s, int u, int until, int q) {
  const int lane = threadIdx.x & 31;
  for (; u < until; u += 32) {
    const long long r = u + lane < until ? s.row_of(u + lane, q) : -1;
    const uint32_t have = __ballot_sync(0xffffffffu, r >= 0);
    if (have) {
      const int k = __ffs(have) - 1;
      return Placed{u + k, __shfl_sync(0xffffffffu, r, k)};
    }
  }
  return Placed{until, -1};
}
// the last one in (before, u]; before, -1: none
__device__ __noinline__ Placed last_placed(const Tokens s, int before, int u, int q) {
  const int lane = threadIdx.x & 31;
  for (; u > before; u -= 32) {
    const long long r = u - lane > before ? s.row_of(u - lane, q) : -1;
    const uint32_t have = __ballot_sync(0xffffffffu, r >= 0);
    if (have) {
      const int k = __ffs(have) - 1;
      return Placed{u - k, __shfl_sync(0xffffffffu, r, k)};
    }
  }
  return Placed{before, -1};
}
// lane j: the new token of row j of the block whose row r is token u's (so far n rows of a run that ends there), looking back to
// token `first`; -1 up to the last row that is not new.  row0: the block's first row.
__device__ __noinline__ int tokens_back(const Tokens s, int u, int r, int n, long long row0, int first, int q) {
  const int lane = threadIdx.x & 31;
  int tok = lane <= r && lane > r - n ? u - (r - lane) : -1;
  int want = r - n;
  for (u -= n; want >= 0 && u >= first; u -= 32) {
    const long long at = u - lane >= first ? s.row_of(u - lane, q) : -1;
    for (uint32_t have = __ballot_sync(0xffffffffu, at >= 0); have && want >= 0; have &= have - 1, --want) {
      const int k = __ffs(have) - 1;
      if (__shfl_sync(0xffffffffu, at, k) != row0 + want) want = -1;       // (rows that do not follow one another: the rest is the tail's)
      if (lane == want) tok = u - k;
    }
  }
  return tok;
}

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(kAppendWarps * 32, sizeof(T) == 2 ? 4 : 2) quant_append_kernel(const __grid_constant__ QuantAppendArgs a) {
  constexpr int N = D / 32;                 // elements of a row per lane
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const QuantGeom& g = a.g;
  const int w0 = blockIdx.x * kQuantBlock;  // first token of the CTA's window
  const long long n_rows = g.n_pages * g.page_tokens;

  const Tokens tokens = {a.slot_map, a.token_seqs, n_rows};
  // lanes 15 to 30 describe the window's tokens, the ones before them the 15 tokens that a block of theirs may begin with, lane
  // 31 the token behind.  What every token needs is looked up here, for all of them at once.
  const int t = w0 - (kQuantBlock - 1) + lane;
  long long row = -1;
  int seq = -1;
  if (t >= 0 && t < a.n_tokens) {
    row = a.slot_map[t];
    seq = a.token_seqs[t];
  }
  const bool placed = row >= 0 && row < n_rows;
  int slot = -1, c0 = 0, c1 = 0;
  bool ok = false;
  if (lane >= kQuantBlock - 1 && lane < 31 && row != -1) {
    ok = placed && seq >= 0 && seq < a.B;
    if (ok) {
      slot = a.slots ? a.slots[seq] : seq;
      c0 = a.cu[seq];
      c1 = a.cu[seq + 1];
      ok = slot >= 0 && slot < g.max_batch && c0 >= 0 && c0 <= t && c1 > t && c1 <= a.n_tokens;
    }
    if (!ok) report_opt(a.status, ECHOKV_EBADPAGE);
  }
  // The work: the last token of every block, and the last token of every sequence that has a row (a token of the same sequence
  // is right behind most others; where none is, one is looked for)
  const bool next = __shfl_down_sync(0xffffffffu, placed ? seq : -1, 1) == seq;
  const bool full = ok && (row & (kQuantBlock - 1)) == kQuantBlock - 1;
  bool last = ok && !full && (t + 1 >= c1 || !next);
  for (uint32_t ask = __ballot_sync(0xffffffffu, last && t + 1 < c1); ask; ask &= ask - 1) {
    const int src = __ffs(ask) - 1;
    const int until = __shfl_sync(0xffffffffu, c1, src);
    if (first_placed(tokens, __shfl_sync(0xffffffffu, t, src) + 2, until, __shfl_sync(0xffffffffu, seq, src)).u < until && lane == src) last = false;
  }
  const uint32_t ends = __ballot_sync(0xffffffffu, full || last);
  if (ends == 0) return;
  const int per_end = 2 * g.n_kv_heads, n_items = __popc(ends) * per_end;

  for (int item = blockIdx.y * kAppendWarps + warp; item < n_items; item += gridDim.y * kAppendWarps) {
    const int which_end = item / per_end, hk = item - which_end * per_end, kv = hk & 1, h = hk >> 1;
    uint32_t left = ends;
    for (int i = 0; i < which_end; ++i) left &= left - 1;
    const int src = __ffs(left) - 1;
    const int te = w0 - (kQuantBlock - 1) + src;
    const long long re = __shfl_sync(0xffffffffu, row, src);
    const int first = __shfl_sync(0xffffffffu, c0, src), until = __shfl_sync(0xffffffffu, c1, src);
    const int my_slot = __shfl_sync(0xffffffffu, slot, src), my_seq = __shfl_sync(0xffffffffu, seq, src);
    const int r0 = (int)(re & (kQuantBlock - 1));
    const long long tail_at = ((long long)my_slot * g.n_kv_heads + h) * kQuantBlock * D + lane * N;
    // this lane's elements of a new token, and of a row of the tail
    const long long stride = a.stride[kv];
    const T* x = static_cast<const T*>(a.x[kv]) + h * D + lane * N;
    T* tail = static_cast<T*>(g.tail[kv]) + tail_at;

    // new tokens of this block: the run of consecutive rows that ends here (n of them), and those before it if tokens without a row
    // cut it
    const bool own = placed && seq == my_seq;
    const bool same = own && lane <= src && lane > src - kQuantBlock && src - lane <= r0 && te - (src - lane) >= first && row == re - (src - lane);
    const int n = __clz(~(__ballot_sync(0xffffffffu, same) << (31 - src)));
    const bool cut = n <= r0 && te - n >= first && !__shfl_sync(0xffffffffu, own, src - n);
    const int tok = cut ? tokens_back(tokens, te, r0, n, re - r0, first, my_seq) : lane <= r0 && lane > r0 - n ? te - (r0 - lane) : -1;
    // The block to quantise, if any: its last row and the token there, its new tokens as above
    bool has_block = true, q_cut = cut;
    long long q_end = re;
    int q_te = te, q_n = n, q_tok = tok;
    if (r0 == kQuantBlock - 1) {
      // (a first block that starts in the tail is left to the warp of the last token if that one writes the tail)
      if (te + 1 < until && __shfl_sync(0xffffffffu, tok, 0) < 0) {
        const long long first_row = first_placed(tokens, first, until, my_seq).row, last_row = last_placed(tokens, te, until - 1, my_seq).row;
        has_block = (first_row ^ re) >= kQuantBlock || last_row < 0 || (last_row & (kQuantBlock - 1)) == kQuantBlock - 1;
      }
    } else {
      // te is the sequence's last token with a row: the sequence's first block of this step, if it starts in the tail and is another
      has_block = false;
      if (te > first) {
        const Placed f = first_placed(tokens, first, until, my_seq);
        const int off = (int)(f.row & (kQuantBlock - 1));
        if (off > 0 && (f.row ^ re) >= kQuantBlock) {
          // the token that ends that block: where it is if no token between is without a row, or looked for
          q_end = f.row - off + kQuantBlock - 1;
          q_n = kQuantBlock - off;
          q_te = f.u + q_n - 1;
          has_block = q_te < te && tokens.row_of(q_te, my_seq) == q_end;
          q_cut = !has_block;
          if (q_cut) {
            Placed p = f;
            while (p.row != q_end && p.u < te) p = first_placed(tokens, p.u + 1, te, my_seq);
            q_te = p.u;
            has_block = p.row == q_end;
            if (has_block) q_tok = tokens_back(tokens, q_te, kQuantBlock - 1, 1, f.row - off, first, my_seq);
          }
        }
      }
    }
    if (has_block) {
      // quantise it; rows that are not new come from the tail
      Piece<T, N> v[kQuantBlock];
      if (!q_cut) {
        const T* fresh = x + (q_te - (kQuantBlock - 1)) * stride;
        if (q_n == kQuantBlock) {
#pragma unroll
          for (int j = 0; j < kQuantBlock; ++j, fresh += stride) v[j].load(fresh);
        } else {
#pragma unroll
          for (int j = 0; j < kQuantBlock; ++j, fresh += stride) v[j].load(j >= kQuantBlock - q_n ? fresh : tail + j * D);
        }
      } else {
#pragma unroll
        for (int j = 0; j < kQuantBlock; ++j) {
          const int u = __shfl_sync(0xffffffffu, q_tok, j);
          v[j].load(u >= 0 ? x + u * stride : tail + j * D);
        }
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
      const long long page = q_end >> g.page_shift;
      const int inside = (int)(q_end & (g.page_tokens - 1)) - (kQuantBlock - 1);
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
    }
    if (r0 != kQuantBlock - 1) {
      __syncwarp();
      for (uint32_t rows = __ballot_sync(0xffffffffu, tok >= 0); rows; rows &= rows - 1) {
        const int j = __ffs(rows) - 1, u = __shfl_sync(0xffffffffu, tok, j);
        Piece<T, N> v;
        v.load(x + u * stride);
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

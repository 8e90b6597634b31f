// Append to a cache held in 4 bits with the rotation on the way, the bounds of the pages that it touches, and rows read back.
//
//   y = R(position) x,   s = e4m3(max |y| / (6 unit)),   code = e2m1(y / (s unit))        for every 16 features of a token
//
// Bytes bound it: every row is read once, queries written once, keys and values in 9/32 of their bytes.  A block takes a few tokens.  Its
// threads first form the (cos, sin) of the tokens' rot / 2 angles in shared memory, once for all heads of q and k: in fp64, rounded to
// fp32 once, so that the codes are those of the exact angle but for the last bit of a cosine.  A unit of q is 8 features of the first
// half of a rotation and their partners of the second.  A unit of k and v is a group of 16 features of both: the thread reads its
// key group and that group's partners (which another thread of the warp has as its own, so they come from the first level cache), turns
// it, and has all it needs for the scale without asking other threads.  A token that is not finite is told by a vote.
// The format has no rows that wait: a token is written where it belongs and no other token matters.
// Measured: 34.5 thousand tokens of 32 / 8 bf16 heads of 128 (747 MB) 130 us, 5.7 TB/s; keys and values alone 67 us, of which the
// rotation takes 25; a decode step of 128 tokens 4.1 us.  (Three blocks to an SM 209 us with the bounds and the rows back, five 199, four 192;
// keys read as pairs of partners, whose threads share a group's scale: 137 against 134.)
#include "fp4_common.cuh"

namespace echokv {

namespace {

constexpr int kFaThreads = 256;
constexpr int kFaTokens = 8;                       // tokens per block (prompts: 2 217, 4 192, 8 190 us)

// 8 elements in the storage type as they are in memory
template <typename T>
struct Eight {
  static constexpr int W = sizeof(T) * 8 / 16;
  uint4 w[W];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < W; ++i) reinterpret_cast<uint4*>(p)[i] = w[i];
  }
  // as pairs of fp32; flip: sign bits that are turned over on the way
  __device__ __forceinline__ void get(uint64_t (&v)[4], uint32_t flip = 0u) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t x[4] = {w[0].x ^ flip, w[0].y ^ flip, w[0].z ^ flip, w[0].w ^ flip};
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = pack_u2(x[e] << 16, x[e] & 0xffff0000u);
    } else {
      flip &= 0x80000000u;
      v[0] = pack_u2(w[0].x ^ flip, w[0].y ^ flip);
      v[1] = pack_u2(w[0].z ^ flip, w[0].w ^ flip);
      v[2] = pack_u2(w[W - 1].x ^ flip, w[W - 1].y ^ flip);
      v[3] = pack_u2(w[W - 1].z ^ flip, w[W - 1].w ^ flip);
    }
  }
};
constexpr uint32_t kFlip = 0x80008000u;
template <typename T>
__device__ __forceinline__ void store8(T* p, const uint64_t (&x)[4]) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) unpack_f2(x[e], v[2 * e], v[2 * e + 1]);
#pragma unroll
  for (int i = 0; i < 8; i += Vec16<T>::N) store16<T>(p + i, v + i);
}

// Cosines and sines of a token: those of two neighbouring frequency indices as (cos, cos, sin, sin), the first pairs of all pieces of 8
// side by side, then the second ones: what lanes of neighbouring pieces read together is contiguous.
__device__ __forceinline__ int turn_at(int j, int pieces) { return (((j & 7) >> 1) * pieces + (j >> 3)) * 4 + (j & 1); }
// 8 features of one half of a rotation and their partners (those of the second half with their signs turned over) -> turned, every step
// rounded
__device__ __forceinline__ void turn8(uint64_t (&x)[4], const uint64_t (&partner)[4], const float* cs, int piece, int pieces) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float4 w = *reinterpret_cast<const float4*>(cs + (e * pieces + piece) * 4);
    // (a packed product and a packed sum would become one rounding)
    float a0, a1, b0, b1;
    unpack_f2(mul_f2(x[e], pack_f2(w.x, w.y)), a0, a1);
    unpack_f2(mul_f2(partner[e], pack_f2(w.z, w.w)), b0, b1);
    x[e] = pack_f2(__fadd_rn(a0, b0), __fadd_rn(a1, b1));
  }
}

// 16 values -> their scale's code and 8 bytes of codes
struct Group {
  uint32_t scale;
  uint2 codes;
};
__device__ __forceinline__ uint32_t largest(const uint64_t (&x)[2][4]) {
  uint32_t top = 0;                                // (magnitudes compare as integers, infinities and NaN above everything finite)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t lo, hi;
    unpack_u2(x[i >> 2][i & 3], lo, hi);
    top = max(max(top, lo & 0x7fffffffu), hi & 0x7fffffffu);
  }
  return top;
}
__device__ __forceinline__ Group encode(const uint64_t (&x)[2][4], uint32_t a, float unit6, float inv_unit) {
  Group r;
  r.scale = e4m3_code(__fmul_rn(__uint_as_float(a), unit6));
  const float s = h2_float(e4m3_scales(r.scale)).x;
  const float m = s > 0.f ? __fdiv_rn(inv_unit, s) : 0.f;
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float lo, hi;
    unpack_f2(mul_f2(x[i >> 2][i & 3], pack_f2(m, m)), lo, hi);
    w[i >> 2] |= e2m1_byte(lo, hi) << (8 * (i & 3));
  }
  r.codes = make_uint2(w[0], w[1]);
  return r;
}

template <typename T, int D>
__global__ void __launch_bounds__(kFaThreads, 4) fp4_append_kernel(const __grid_constant__ Fp4AppendArgs a, int tokens_per_block) {
  constexpr int G = D / kFp4Group;                 // groups of a head (4 or 8 lanes side by side)
  __shared__ __align__(16) float cs[kFaTokens][128];
  const int half = a.rot_dim >> 1, pieces = half >> 3, tid = threadIdx.x, lane = tid & 31;
  after_the_one_before();
  let_the_next_one_come();
  const int t0 = blockIdx.x * tokens_per_block, nt = min(tokens_per_block, a.n_tokens - t0);
  const Fp4Geom& g = a.g;
  const int H = g.n_kv_heads;
  for (int i = tid; i < nt * half; i += kFaThreads) {
    const int t = i / half, j = i - t * half;
    const double turns = (double)a.pos[(long long)a.axis[j] * a.n_tokens + t0 + t] * a.turns[j];
    double s, c;
    sincospi(2.0 * (turns - rint(turns)), &s, &c);
    cs[t][turn_at(j, pieces)] = (float)c;
    cs[t][turn_at(j, pieces) + 2] = (float)s;
  }
  __syncthreads();

  // ---- keys and values
  const int items = nt * H * G, steps = (items + kFaThreads - 1) / kFaThreads;
#pragma unroll 1
  for (int step = 0; step < steps; ++step) {
    const int i = step * kFaThreads + tid;
    const bool live = i < items;                   // (a head's G lanes are all live or none is)
    // (a block's tokens side by side: what they write of a block's rows, four tokens a sector, is then written together)
    const int u = live ? i / G : 0, grp = i % G, h = u / nt, t = u - h * nt;
    const long long row = live ? a.slot_map[t0 + t] : -1;
    const bool in_pool = row >= 0 && (row >> g.page_shift) < g.n_pages;
    if (live && row != -1 && !in_pool) report_opt(a.status, ECHOKV_EBADPAGE);
    Eight<T> k[2], p[2], v[2];
    uint64_t x[2][4], y[2][4];
    if (in_pool) {
      const T* kp = static_cast<const T*>(a.x[0]) + (long long)(t0 + t) * a.stride[0] + h * D;
      const T* vp = static_cast<const T*>(a.x[1]) + (long long)(t0 + t) * a.stride[1] + h * D + grp * kFp4Group;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int f = grp * kFp4Group + 8 * e;
        k[e].load(kp + f);
        p[e].load(kp + (f < half ? f + half : f < a.rot_dim ? f - half : f));
        v[e].load(vp + 8 * e);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int f = grp * kFp4Group + 8 * e;
        k[e].get(x[e]);
        if (f < a.rot_dim) {
          uint64_t w[4];
          p[e].get(w, f < half ? kFlip : 0u);
          turn8(x[e], w, cs[t], (f < half ? f : f - half) >> 3, pieces);
        }
        v[e].get(y[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e >> 2][e & 3] = y[e >> 2][e & 3] = 0ull;
    }
    const uint32_t ka = largest(x), va = largest(y);
    const uint32_t vote = __ballot_sync(0xffffffffu, max(ka, va) >= 0x7f800000u);
    if (!in_pool) continue;
    Group kg = encode(x, ka, a.unit6[0], a.inv_unit[0]), vg = encode(y, va, a.unit6[1], a.inv_unit[1]);
    if (vote >> (lane & ~(G - 1)) & ((1u << G) - 1)) {
      kg.scale = kE4m3Nan;
      vg.scale = 0u;
      kg.codes = vg.codes = make_uint2(0u, 0u);
    }
    const int inside = (int)(row & (g.page_tokens - 1)), r = inside & 15, f = grp * kFp4Group;
    unsigned char* blk = g.blocks + (((row >> g.page_shift) * H + h) * (g.page_tokens / 16) + (inside >> 4)) * fp4_block_bytes(D);
    *reinterpret_cast<uint2*>(blk + fp4_k_at(D, r, f)) = kg.codes;
    if (D == 128) {
      *reinterpret_cast<uint2*>(blk + fp4_v_at(D, r, f)) = vg.codes;
    } else {
      *reinterpret_cast<uint32_t*>(blk + fp4_v_at(D, r, f)) = vg.codes.x;
      *reinterpret_cast<uint32_t*>(blk + fp4_v_at(D, r, f + 8)) = vg.codes.y;
    }
    blk[fp4_ks_at(D, r, f)] = (unsigned char)kg.scale;
    blk[fp4_vs_at(D, r, f)] = (unsigned char)vg.scale;
  }

  // ---- queries: 8 features and their partners, or two pieces of what is only copied
  if (a.q == nullptr) return;
  constexpr int U = D / 16, kStep = kFaThreads / U, kBatch = sizeof(T) == 2 ? 2 : 1;
  const int c = tid % U;
  const bool turn = c < pieces;
  const int e0 = turn ? c * 8 : a.rot_dim + 2 * (c - pieces) * 8, e1 = turn ? half + c * 8 : e0 + 8;
  if (!turn && a.q == a.q_out) return;
  const int n = nt * a.n_q_heads;
#pragma unroll 1
  for (int u = tid / U; u < n; u += kBatch * kStep) {
    Eight<T> x[kBatch][2];
    T* dst[kBatch];
    int tok[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int at = u + b * kStep;
      tok[b] = at / a.n_q_heads;
      dst[b] = nullptr;
      if (at < n) {
        const int head = at - tok[b] * a.n_q_heads;
        const T* src = static_cast<const T*>(a.q) + (long long)(t0 + tok[b]) * a.q_stride + head * D;
        dst[b] = static_cast<T*>(a.q_out) + (long long)(t0 + tok[b]) * a.q_out_stride + head * D;
        x[b][0].load(src + e0);
        x[b][1].load(src + e1);
      }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (dst[b] == nullptr) continue;
      if (turn) {
        uint64_t y0[4], y1[4], n1[4], z[4];
        x[b][0].get(y0);
        x[b][1].get(y1);
        x[b][1].get(n1, kFlip);
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = y0[e];
        turn8(y0, n1, cs[tok[b]], c, pieces);
        turn8(y1, z, cs[tok[b]], c, pieces);
        store8<T>(dst[b] + e0, y0);
        store8<T>(dst[b] + e1, y1);
      } else {
        x[b][0].store(dst[b] + e0);
        x[b][1].store(dst[b] + e1);
      }
    }
  }
}

// Bounds of the pages that the call touched: a block looks at `chunk` tokens (31; 1 of a decode step) for the last ones of their pages; a warp
// takes such a page for one head.  It brings the keys of 64 tokens to shared memory at a time, all on their way at once (what the first kernel
// wrote comes from the second level cache), then goes through them in a short loop, a lane with 8 features of every second
// (fourth) token, so that little is left to join at the end.  (A kernel like this one runs its code once: what is unrolled is fetched
// for nothing.  Loads to registers, which the compiler put next to their uses: 20 to 36 us after 34.5 thousand tokens, now 15 behind the
// kernel before it; 16.5 by itself.)
constexpr int kFbWarps = 8;
constexpr int kFbBlocks = 4;                       // of 16 tokens, at a time

// The row of the first token from i on that has one (-1: none), by a whole warp: there may be many without one (a padded step), so 256
// are looked at at once.
__device__ __noinline__ long long next_row(const int64_t* slot_map, long long i, int n_tokens, int page_shift, long long n_pages) {
  const int lane = threadIdx.x & 31;
  for (; i < n_tokens; i += 256) {
    long long row[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) row[e] = i + 32 * e + lane < n_tokens ? slot_map[i + 32 * e + lane] : -1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t placed = __ballot_sync(0xffffffffu, row[e] >= 0 && (row[e] >> page_shift) < n_pages);
      if (placed) return __shfl_sync(0xffffffffu, row[e], __ffs(placed) - 1);
    }
  }
  return -1;
}

template <int D>
__global__ void __launch_bounds__(kFbWarps * 32) fp4_bounds_kernel(const __grid_constant__ Fp4AppendArgs a, int chunk) {
  constexpr int L = D / 8, R = 32 / L;             // lanes of a token, tokens that the warp looks at at once
  constexpr int BB = fp4_block_bytes(D), kKeys = 9 * D;               // bytes of a block, of its keys' codes and scales
  __shared__ __align__(16) unsigned char keys[kFbWarps][kFbBlocks * kKeys];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane / L, f = lane % L * 8;
  const Fp4Geom& g = a.g;
  const int H = g.n_kv_heads, worker = blockIdx.y * kFbWarps + warp, workers = gridDim.y * kFbWarps;
  const uint32_t mine_at = smem_u32(keys[warp]);
  after_the_one_before();
  const auto row_of = [&](long long i) {
    const long long row = i < a.n_tokens ? a.slot_map[i] : -1;
    return row >= 0 && (row >> g.page_shift) < g.n_pages ? row : -1;
  };
  // (a block of one token looks at those behind it with its other lanes)
  const long long i = (long long)blockIdx.x * chunk + lane, mine = row_of(i);
  // the next token that has a row: one of the next lanes', and for the last of those looked for behind them (where its page has room)
  const uint32_t placed = __ballot_sync(0xffffffffu, mine >= 0), later = placed & ~(1u << lane | ((1u << lane) - 1));
  long long next = __shfl_sync(0xffffffffu, mine, later ? __ffs(later) - 1 : lane);
  if (!later) next = -1;
  const int end = 31 - __clz(placed);
  if (placed != 0 && end < chunk && (long long)blockIdx.x * chunk + 32 < a.n_tokens) {
    const long long row = __shfl_sync(0xffffffffu, mine, end);
    if ((row & (g.page_tokens - 1)) != g.page_tokens - 1) {
      const long long n = next_row(a.slot_map, (long long)blockIdx.x * chunk + 32, a.n_tokens, g.page_shift, g.n_pages);
      if (lane == end) next = n;
    }
  }
  const bool last = mine >= 0 && lane < chunk && (next < 0 || (next >> g.page_shift) != (mine >> g.page_shift));
  // (page, head) pairs in turn: `off` is this warp's next one, from the present page's first head on
  int off = worker;
  for (uint32_t pages = __ballot_sync(0xffffffffu, last); pages; pages &= pages - 1, off -= H) {
    if (off >= H) continue;
    const long long row = __shfl_sync(0xffffffffu, mine, __ffs(pages) - 1);
    const long long page = row >> g.page_shift;
    const int n = (int)(row & (g.page_tokens - 1)) + 1;
    for (; off < H; off += workers) {
      const int h = off;
      const unsigned char* blk = g.blocks + (page * H + h) * (g.page_tokens / 16) * fp4_block_bytes(D);
      __half2 top[4], low[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        top[e] = __half2half2(__ushort_as_half(0xfc00));        // -inf
        low[e] = __half2half2(__ushort_as_half(0x7c00));
      }
      bool nan = false;
#pragma unroll 1
      for (int base = 0; base < n; base += 16 * kFbBlocks) {
        const int n_here = min(n - base, 16 * kFbBlocks);
        const unsigned char* src = blk + (base >> 4) * BB;
#pragma unroll 1
        for (int k = 0; 16 * k < n_here; ++k, src += BB) {
#pragma unroll
          for (int x = 0; x < D / 64; ++x)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine_at + k * kKeys + (x * 32 + lane) * 16), "l"(src + (x * 32 + lane) * 16) : "memory");
          if (lane < D / 16)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine_at + k * kKeys + 8 * D + lane * 16), "l"(src + 16 * D + lane * 16) : "memory");
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
#pragma unroll 2
        for (int t = r; t < n_here; t += R) {
          const unsigned char* b = keys[warp] + (t >> 4) * kKeys;
          const uint32_t code = b[8 * D + (t & 15) * (D / 16) + f / 16];
          nan |= (code & 0x7fu) == kE4m3Nan;
          const uint32_t s = e4m3_scales(code | code << 8);
          uint32_t x[4];
          e2m1_bytes(*reinterpret_cast<const uint32_t*>(b + (t & 15) * (D / 2) + f / 2), x);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[e] = fp4_mul(x[e], s);
            const __half2 z = *reinterpret_cast<const __half2*>(&x[e]);
            top[e] = __hmax2(top[e], z);
            low[e] = __hmin2(low[e], z);
          }
        }
        __syncwarp();                              // (the next tokens go to the same place)
      }
      float most = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
#pragma unroll
        for (int o = L; o < 32; o <<= 1) {
          top[e] = __hmax2(top[e], __shfl_xor_sync(0xffffffffu, top[e], o));
          low[e] = __hmin2(low[e], __shfl_xor_sync(0xffffffffu, low[e], o));
        }
        const float2 x = __half22float2(top[e]), y = __half22float2(low[e]);
        most = fmaxf(most, fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(y.x), fabsf(y.y))));
      }
      most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));      // (magnitudes: their bits are in their order)
      nan = __any_sync(0xffffffffu, nan);
      const float scale = fmaxf(__fmul_rn(most, 1.f / 127.f), 0x1p-60f), inv = __frcp_rn(scale);
      if (r == 0) {
        uint32_t out[2][2] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 x = __half22float2(top[e >> 1]), y = __half22float2(low[e >> 1]);
          const auto code = [&](float v) { return (uint32_t)(nan ? 0 : min(127, max(-127, __float2int_rn(__fmul_rn(v, inv))))) & 0xffu; };
          out[0][e >> 2] |= code(e & 1 ? x.y : x.x) << (8 * (e & 3));
          out[1][e >> 2] |= code(e & 1 ? y.y : y.x) << (8 * (e & 3));
        }
        int8_t* dst = g.bounds + (page * H + h) * 2 * D + f;
        *reinterpret_cast<uint2*>(dst) = make_uint2(out[0][0], out[0][1]);
        *reinterpret_cast<uint2*>(dst + D) = make_uint2(out[1][0], out[1][1]);
      }
      if (lane == 0) g.bound_scales[page * H + h] = nan ? __uint_as_float(0x7fc00000u) : scale;
    }
  }
}

// Rows back: a thread per group of 16 features of a token and head, key and value.
template <typename T, int D>
__global__ void __launch_bounds__(kFaThreads) fp4_read_kernel(const __grid_constant__ Fp4ReadArgs a) {
  constexpr int G = D / kFp4Group;
  after_the_one_before();
  const Fp4Geom& g = a.g;
  const int H = g.n_kv_heads;
  const long long i = (long long)blockIdx.x * kFaThreads + threadIdx.x;
  // (four tokens of a head side by side: their values share the cache's sectors)
  const int grp = (int)(i % G), f = grp * kFp4Group;
  const long long u = i / (4 * G);
  const int t = (int)(u / H) * 4 + (int)(i / G) % 4, h = (int)(u % H);
  if (t >= a.n_tokens) return;
  const long long row = a.slot_map[t];
  const bool in_pool = row >= 0 && (row >> g.page_shift) < g.n_pages;
  if (row != -1 && !in_pool) report_opt(a.status, ECHOKV_EBADPAGE);
  uint32_t w[2][2] = {}, s[2] = {};
  if (in_pool) {
    const int inside = (int)(row & (g.page_tokens - 1)), r = inside & 15;
    const unsigned char* blk = g.blocks + (((row >> g.page_shift) * H + h) * (g.page_tokens / 16) + (inside >> 4)) * fp4_block_bytes(D);
    const uint2 k = *reinterpret_cast<const uint2*>(blk + fp4_k_at(D, r, f));
    w[0][0] = k.x; w[0][1] = k.y;
    w[1][0] = *reinterpret_cast<const uint32_t*>(blk + fp4_v_at(D, r, f));
    w[1][1] = *reinterpret_cast<const uint32_t*>(blk + fp4_v_at(D, r, f + 8));
    s[0] = blk[fp4_ks_at(D, r, f)];
    s[1] = blk[fp4_vs_at(D, r, f)];
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (a.out[k] == nullptr) continue;
    const uint32_t s2 = e4m3_scales(s[k] | s[k] << 8);
    T* dst = static_cast<T*>(a.out[k]) + (long long)t * a.stride[k] + h * D + f;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      uint64_t v[4];
      uint32_t pairs[4];
      e2m1_bytes(w[k][p], pairs);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 x = h2_float(fp4_mul(pairs[e], s2));
        v[e] = mul_f2(pack_f2(x.x, x.y), pack_f2(a.unit[k], a.unit[k]));
      }
      store8<T>(dst + 8 * p, v);
    }
  }
}

template <typename T, int D>
cudaError_t launch_append(const Fp4AppendArgs& a, int sm_count, cudaStream_t stream) {
  // few tokens: one per block, so that a decode step's rows spread over the SMs
  const int per_block = a.n_tokens <= 4 * sm_count ? 1 : kFaTokens;
  cudaError_t e = launch_early(fp4_append_kernel<T, D>, dim3((unsigned)((a.n_tokens + per_block - 1) / per_block)), kFaThreads, 0, stream, a, per_block);
  if (e != cudaSuccess || a.g.bounds == nullptr) return e;
  // (many tokens: 31 to a block, whose lanes then see the one behind them, most of which are not the last ones of their pages, and the
  // heads over several blocks if these are few; a decode step: a block for each token)
  const int chunk = a.n_tokens <= 4 * sm_count ? 1 : 31, blocks = (a.n_tokens + chunk - 1) / chunk;
  const int y = chunk == 1 || blocks >= sm_count ? 1 : min((31 * a.g.n_kv_heads + kFbWarps - 1) / kFbWarps, (2 * sm_count + blocks - 1) / blocks);
  return launch_early(fp4_bounds_kernel<D>, dim3(blocks, y), kFbWarps * 32, 0, stream, a, chunk);
}

}  // namespace

cudaError_t launch_fp4_append(const Fp4AppendArgs& a, int sm_count, cudaStream_t stream) {
  if (a.dtype == ECHOKV_BF16) return a.g.head_dim == 128 ? launch_append<__nv_bfloat16, 128>(a, sm_count, stream) : launch_append<__nv_bfloat16, 64>(a, sm_count, stream);
  return a.g.head_dim == 128 ? launch_append<float, 128>(a, sm_count, stream) : launch_append<float, 64>(a, sm_count, stream);
}

cudaError_t launch_fp4_read(const Fp4ReadArgs& a, cudaStream_t stream) {
  const long long n = (a.n_tokens + 3ll) / 4 * 4 * a.g.n_kv_heads * (a.g.head_dim / kFp4Group);
  const unsigned grid = (unsigned)((n + kFaThreads - 1) / kFaThreads);
  const bool wide = a.g.head_dim == 128;
  if (a.dtype == ECHOKV_BF16)
    return wide ? launch_early(fp4_read_kernel<__nv_bfloat16, 128>, dim3(grid), kFaThreads, 0, stream, a)
                : launch_early(fp4_read_kernel<__nv_bfloat16, 64>, dim3(grid), kFaThreads, 0, stream, a);
  return wide ? launch_early(fp4_read_kernel<float, 128>, dim3(grid), kFaThreads, 0, stream, a)
              : launch_early(fp4_read_kernel<float, 64>, dim3(grid), kFaThreads, 0, stream, a);
}

}  // namespace echokv

// Attention over a cache held in 8 bits, one or a few queries per sequence (decode steps, drafts to verify).
//
//   x_t = scale q . k_t  [capped by softcap tanh(x / softcap)] [- slope |p - t|],   o = sum_t 2^(x_t log2e - m) v_t / sum_t 2^(...)
//
// The codes are read once from HBM and that is the bound; everything else has to fit beside the stream (23 bytes per
// clock and SM).  The design:
//
//   work     A unit is one 16-token block (one scale) of one KV head for one tile of 8 query rows (the query heads that share
//            the KV head, times a sequence's new tokens).  The units of all sequences are laid end to end and cut into
//            equal shares, one per CTA and within it one per warp, computed on the device from the lengths: ragged
//            batches, one long request and a thousand short ones all balance.  A share cuts at most two (sequence, head)
//            items; their partial results (running maximum, sum, output) are combined inside the CTA through shared
//            memory and between CTAs by a second small kernel.
//   copies   A warp fills a ring of its own by TMA, one box of 16 token rows for K and one for V per block, in the 128-byte
//            swizzle: every operand read is then free of bank conflicts.  No barrier between warps.
//   products mma.sync m16n8k16 in fp16 with the tokens (then the head's features) on the M rows and the 8 query rows on N:
//            S^T = K q^T, O^T = V^T P^T, 8 instructions each per block and no padding of the queries to 16 rows.  S^T
//            becomes the operand P^T by one 8 x 8 transposition per 8 tokens in registers.  Codes convert to fp16 exactly; fp32
//            queries, and the probabilities beside them, take a second product with their low-order halves (22 bits).
//            (tcgen05's 128 rows would be padding here, and the tensor pipe is not what bounds.)
//   softmax  The running maximum is a reference that moves only when a score is 2^8 above it: the common path compares and votes,
//            without a reduction over the tokens.
//   scales   The K scale multiplies the score, the V scale the probability.  fp16's range is kept by references that are powers of
//            two: two per query row, one of them for the V scales that the row sees, which moves with the maximum's.
//   tail     The open block is in the storage type: bf16 rows are operands of the bf16 product as they are, fp32 rows become pairs of
//            fp16, each token's around its own power of two.  It is attended first, while the first copies are on their way.
// Measured: 16 sequences over 32768 keys (1.07 GB of codes) 177 us, 6.1 TB/s; 32 ragged ones with capped scores, e4m3, 168 us,
// 6.0 TB/s; one token over 777 keys 12.6 us, all latency (this kernel 7.5, the second one 3, launches).
// (Rings filled by cp.async: 4.4 TB/s.  Warps x stages, first case: 12 x 3 177 us, 10 x 4 193, 8 x 4 192, 16 x 2 225.)
#include "quant_common.cuh"
#include "recon_tc.h"

namespace echokv {

namespace {

constexpr int kQaWarps = 12;
constexpr int kQaThreads = kQaWarps * 32;
constexpr int kQaRows = 8;                        // query rows per tile
constexpr int kQaStages = 3;
constexpr int kQaMergeThreads = kQaRows * 32;
constexpr int kQaMaxCtas = 512;
constexpr int kQaItemCost = 6;                     // what an item costs beside its blocks (queries, first copies, result), in
                                                  // blocks: units are dealt out as if an item began with that many more
constexpr int kQaMinShare = 2 * kQaWarps;         // units per CTA at least
constexpr float kQaGrow = 8.f;                    // the references move when a score is 2^8 above them
constexpr float kQaPScale = 32.f;                 // P <= 2^8 times a scale ratio <= 1 times 2^5: 2^13 at most
constexpr int kQaLeastExp = 27;                   // references of V scales are 2^-100 or more, as the scales are

struct QaDesc {                                   // an item cut at the end of CTA g's share
  int n_parts;                                    // CTAs that hold parts of it (0: none starts here)
  int b, tile, h;
};

__host__ __device__ constexpr int qa_stage_bytes(int D) { return 2 * kQuantBlock * D; }      // K codes, V codes
// byte offset of 16-byte piece x of token row `tok`: rows of 128 bytes (one token of 128 features, two of 64), swizzled
template <int D>
__device__ __forceinline__ uint32_t qa_off(int tok, int x) {
  if (D == 128) return tok * 128 + ((x ^ (tok & 7)) << 4);
  return (tok >> 1) * 128 + ((((tok & 1) * 4 + x) ^ ((tok >> 1) & 7)) << 4);
}

struct QaSeg {
  unsigned long long item;                        // first unit of the item
  unsigned long long item_end;
  int b, tile, h;
  int valid, starts, ends;
};

template <int D>
struct QaSmem {
  // a warp's segment that goes on from the warp before it, and (over the warp's ring, once that is at rest) the one
  // that goes on in the next warp
  float o_first[kQaWarps][kQaRows][D];
  QaSeg seg[2 * kQaWarps];
  float m[2 * kQaWarps][kQaRows], l[2 * kQaWarps][kQaRows];
  unsigned long long pre[kQaThreads + 1];
  unsigned long long warp_sums[kQaWarps];
  unsigned long long full[kQaWarps][kQaStages];
  int4 info[kQaThreads];                          // slot, length, first token, tokens (0: nothing to do) of a small batch
};
template <int D>
__host__ __device__ constexpr size_t qa_ring_bytes() { return (size_t)kQaWarps * kQaStages * qa_stage_bytes(D); }

// workspace: [ctas] QaDesc | [ctas][2][8] (m, l) | [ctas][2][8][D] o
template <int D>
struct QaWork {
  QaDesc* desc;
  float2* ml;
  float* o;
  __host__ __device__ explicit QaWork(unsigned char* ws) {
    desc = reinterpret_cast<QaDesc*>(ws);
    ml = reinterpret_cast<float2*>(ws + kQaMaxCtas * sizeof(QaDesc));
    o = reinterpret_cast<float*>(ws + kQaMaxCtas * (sizeof(QaDesc) + 2 * kQaRows * sizeof(float2)));
  }
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

// What the kernel needs of a sequence: w = 0 tokens where nothing is attended here.
// (without: the sequences of many rows are the chunk kernel's)
__device__ __forceinline__ int4 seq_info(const QuantAttnArgs& a, int b, bool tell, bool without) {
  const QuantSeq s = quant_seq(a, b);
  if (s.error && tell) report_opt(a.status, s.error);
  return make_int4(s.slot, s.len, s.first, s.error || (without && many_rows(a, s)) ? 0 : s.n);
}
__device__ __forceinline__ int row_tiles(const QuantAttnArgs& a, int n) { return (n * a.group + kQaRows - 1) / kQaRows; }
__device__ __forceinline__ unsigned long long units_of(const QuantAttnArgs& a, const int4& s) {
  return (unsigned long long)row_tiles(a, s.w) * a.g.n_kv_heads * ((s.y + kQuantBlock - 1) / kQuantBlock + kQaItemCost);
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
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// c + 0 * a of two bf16 each: a magnitude of 0 as long as every a was finite (and NaN from then on)
__device__ __forceinline__ uint32_t zero_fma_bf16x2(uint32_t a, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(0u), "r"(c));
  return d;
}
// fp16 operands of x * up: the rounded pair and what it leaves
struct HalfPair {
  uint32_t hi, lo;
};
template <bool LOW>
__device__ __forceinline__ HalfPair split_pair(float x0, float x1) {
  HalfPair p;
  p.hi = h2(x0, x1);
  p.lo = 0u;
  if (LOW) {
    const float2 w = h2_float(p.hi);
    p.lo = h2(x0 - w.x, x1 - w.y);
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

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(kQaThreads, 1) quant_attn_kernel(const __grid_constant__ CUtensorMap tm_k,
                                                                   const __grid_constant__ CUtensorMap tm_v,
                                                                   const __grid_constant__ QuantAttnArgs a) {
  constexpr int KC = D / 64;                      // 16-byte pieces of a key row per lane
  constexpr int KS = D / 16;                      // k-steps of q . k
  constexpr int NT = D / 8;                       // V bytes per token and lane (features NT r .. NT r + NT - 1)
  constexpr int MT = D / 16;                      // output tiles of 16 features: features NT r + 2 j and NT r + 2 j + 1
  constexpr bool kF32 = sizeof(T) == 4;
  extern __shared__ __align__(1024) unsigned char qa_raw[];
  QaSmem<D>& sm = *reinterpret_cast<QaSmem<D>*>(qa_raw + qa_ring_bytes<D>());
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;
  const uint32_t ring = smem_u32(qa_raw) + warp * kQaStages * qa_stage_bytes(D);
  const QuantGeom& g = a.g;
  const int H = g.n_kv_heads;
  // output rows [8][D] of segment `at`
  const auto seg_rows = [&](int at) -> float* {
    return at & 1 ? reinterpret_cast<float*>(qa_raw + (size_t)(at >> 1) * kQaStages * qa_stage_bytes(D)) : &sm.o_first[at >> 1][0][0];
  };

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_v) : "memory");
  }
  // ---- the units of the call, and this CTA's and warp's share of them
  const bool without = take_chunks(a, a.sm_count);
  const int per = (a.B + kQaThreads - 1) / kQaThreads;
  {
    unsigned long long n = 0;
#pragma unroll 1
    for (int b = tid * per; b < min(a.B, (tid + 1) * per); ++b) {
      const int4 s = seq_info(a, b, blockIdx.x == 0, without);
      if (per == 1) sm.info[b] = s;
      n += units_of(a, s);
    }
    unsigned long long x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) sm.warp_sums[warp] = x;
    if (tid < 2 * kQaWarps) sm.seg[tid].valid = 0;
    if (lane == 0) {
      for (int i = 0; i < kQaStages; ++i) mbar_init(smem_u32(&sm.full[warp][i]), 1);
      mbar_fence_init();
    }
    __syncthreads();
    unsigned long long before = 0;
    for (int w = 0; w < warp; ++w) before += sm.warp_sums[w];
    sm.pre[tid + 1] = before + x;
    if (tid == 0) sm.pre[0] = 0;
    __syncthreads();
  }
  const unsigned long long total = sm.pre[kQaThreads];
  unsigned long long share = quotient(total + gridDim.x - 1, gridDim.x);
  if (share < kQaMinShare) share = kQaMinShare;
  const unsigned long long cta0 = min(total, share * blockIdx.x), cta1 = min(total, cta0 + share);
  const unsigned long long wshare = quotient(cta1 - cta0 + kQaWarps - 1, kQaWarps);
  unsigned long long u = min(cta1, cta0 + wshare * warp);
  const unsigned long long u_end = min(cta1, u + wshare);

  // the sequence of unit u: the last thread whose prefix is not above it, in two votes
  int b = 0;
  unsigned long long base = 0;                    // first unit of sequence b
  if (u < u_end) {
    static_assert(kQaWarps <= 32, "a lane per run of 32 prefixes");
    const int run = __popc(__ballot_sync(0xffffffffu, lane < kQaWarps && sm.pre[lane * 32] <= u)) - 1;
    const int at = run * 32 + __popc(__ballot_sync(0xffffffffu, sm.pre[run * 32 + lane] <= u)) - 1;
    b = at * per;
    base = sm.pre[at];
  }
  const bool plain = !(a.softcap > 0.f) && a.slopes == nullptr;
  const float cap_in = a.softcap > 0.f ? 1.f / a.softcap : 0.f, cap_out = a.softcap * kLog2e;

  uint32_t filled = 0, used = 0;                  // blocks this warp has asked for and taken from its ring
  bool dead = false;                              // a copy did not arrive (reported); the warp gives up
  while (u < u_end && !dead) {
    int4 info = per == 1 ? sm.info[b] : seq_info(a, b, false, without);
    unsigned long long n_units = units_of(a, info);
    while (base + n_units <= u) {
      base += n_units;
      ++b;
      info = per == 1 ? sm.info[b] : seq_info(a, b, false, without);
      n_units = units_of(a, info);
    }
    const int slot = info.x, len = info.y, first_token = info.z, n_new = info.w;
    const int n_blk = (len + kQuantBlock - 1) / kQuantBlock, tiles = row_tiles(a, n_new);
    const unsigned long long rem = u - base;
    const int ht = (int)quotient(rem, n_blk + kQaItemCost), at0 = (int)(rem - (unsigned long long)ht * (n_blk + kQaItemCost));
    const int h = tiles == 1 ? ht : ht / tiles, tile = ht - h * tiles;
    const unsigned long long item = u - at0, item_end = item + n_blk + kQaItemCost;
    const unsigned long long seg_end = min(item_end, u_end);
    // blocks [blk0, blk0 + nb) of the item
    const int blk0 = max(0, at0 - kQaItemCost), nb = max(0, (int)(seg_end - item) - kQaItemCost) - blk0;
    if (nb == 0) {
      u = seg_end;
      continue;
    }
    const int n_full = len / kQuantBlock;       // blocks held as codes; block n_full is the open one

    // ---- the blocks held as codes: copies
    const int n_codes = max(0, min(nb, n_full - blk0));
    const int32_t* pages = a.table + (long long)slot * g.max_pages;
    // lane l keeps pages and scales of blocks 32 n + l of the segment: of the current 32, and fetched ahead of the next 32
    int page_cur, page_next;
    float ks_cur, vs_cur, ks_next = 0.f, vs_next = 0.f;
    const auto load_pages = [&](int group) {
      const int j = 32 * group + lane;
      int id = j < n_codes ? pages[(blk0 + j) * kQuantBlock >> g.page_shift] : 0;
      if (id < 0 || id >= g.n_pages) {
        report_opt(a.status, ECHOKV_EBADPAGE);
        id = 0;
      }
      return id;
    };
    const auto load_scales = [&](int group, int page, float* ks, float* vs) {
      const int j = 32 * group + lane;
      if (j < n_codes) {
        const int inside = (blk0 + j) * kQuantBlock & (g.page_tokens - 1);
        const long long at = ((long long)page * H + h) * (g.page_tokens / kQuantBlock) + inside / kQuantBlock;
        *ks = g.scales[0][at];
        *vs = g.scales[1][at];
      }
    };
    page_cur = load_pages(0);
    // ---- the query rows: this lane loads a quarter of row r as operand; its scores are of rows 2 c and 2 c + 1
    const int n_rows = n_new * a.group;
    uint32_t qh[KS][2], ql[kF32 ? KS : 1][2];
    float c_row[2];
    const int qrow_r = tile * kQaRows + r;
    const bool ok = qrow_r < n_rows;
    const T* qp = static_cast<const T*>(a.q) + (long long)(first_token + (ok ? qrow_r >> a.group_shift : 0)) * a.q_stride +
                  (long long)(h * a.group + (qrow_r & (a.group - 1))) * D;
    Quad<T> qv[KS];
#pragma unroll
    for (int x = 0; x < KS; x += Quad<T>::kPerLoad)
      if (ok) Quad<T>::load16(qp + KC * 16 * c + 4 * x, &qv[x]);
      else Quad<T>::zero16(&qv[x]);
    page_next = load_pages(1);
    ks_cur = vs_cur = 0.f;
    load_scales(0, page_cur, &ks_cur, &vs_cur);
    int group = 0;
    const auto issue = [&](int j) {
      const int page = __shfl_sync(0xffffffffu, (j >> 5) == group ? page_cur : page_next, j & 31);
      const int row = (page * H + h) * (g.page_tokens * D / 128) + ((blk0 + j) * kQuantBlock & (g.page_tokens - 1)) * D / 128;
      if (lane == 0) {
        const int st = filled % kQaStages;
        const uint32_t bar = smem_u32(&sm.full[warp][st]), dst = ring + st * qa_stage_bytes(D);
        mbar_arrive_expect_tx(bar, qa_stage_bytes(D));
        tma_load_2d(dst, &tm_k, 0, row, bar);
        tma_load_2d(dst + kQuantBlock * D, &tm_v, 0, row, bar);
      }
      ++filled;
    };
    for (int j = 0; j < min(kQaStages, n_codes); ++j) issue(j);

    {
      // (magnitudes compare as integers; an infinity or NaN gives the factor 1 and goes on through the products)
      uint32_t bits = 0;
#pragma unroll
      for (int x = 0; x < KS; ++x) bits = qv[x].top(bits);
      bits = Quad<T>::top_bits(bits);
      bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 1));
      bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 2));
      const float top = __uint_as_float(bits);
      float back;
      const float up = scale_up_to_half(top, &back);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        c_row[e] = __shfl_sync(0xffffffffu, back, 4 * (2 * c + e)) * a.scale * (a.softcap > 0.f ? 1.f : kLog2e);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const HalfPair p = split_pair<kF32>(qv[ks].get(2 * f) * up, qv[ks].get(2 * f + 1) * up);
          qh[ks][f] = p.hi;
          if (kF32) ql[ks][f] = p.lo;
        }
    }
    const int prefix = a.prefix ? a.prefix[b] : 0;
    int pos[2];
    float slope2[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int qrow = tile * kQaRows + 2 * c + e;
      pos[e] = len - n_new + (qrow < n_rows ? qrow >> a.group_shift : 0);
      slope2[e] = a.slopes ? a.slopes[h * a.group + (qrow & (a.group - 1))] * kLog2e : 0.f;
    }

    float o[MT][4];                               // rows: feature NT r + 2 j (0, 1) and + 1 (2, 3); columns: query rows 2 c, 2 c + 1
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int f = 0; f < 4; ++f) o[j][f] = 0.f;
    // Per query row: the reference of its maximum (0 until it has seen a key, which the first one seen moves), and how far
    // above the reference a score may be before that moves.
    float m_ref[2] = {0.f, 0.f}, grow[2] = {-3.0e38f, -3.0e38f}, l_run[2] = {0.f, 0.f};
    // the reference of the V scales that the row sees (negative: none yet, and the output in units of 1), kQaPScale / it; the smaller
    // one of the two rows
    float v_ref[2] = {-kQaPScale, -kQaPScale}, v_inv[2] = {0.f, 0.f}, v_low = -kQaPScale;
    const int pos_first = len - n_new + (tile * kQaRows >> a.group_shift);     // the tile's first query: blocks up to it are seen whole

    // a scaled product q . k of token tok and query row 2 c + e -> the score in base-2 units
    const auto score = [&](float y, int e, int tok) {
      if (a.softcap > 0.f) y = cap_out * tanh_f32(y * cap_in);
      if (a.slopes) y -= slope2[e] * fabsf((float)(pos[e] - tok));
      return y;
    };
    // Scores of two blocks (sc[n][2 t + e]: token r + 8 t of block n, query row 2 c + e; the first token is tok0) -> probabilities as
    // operands (ph[n][t]: query row r, tokens 8 t + 2 c, + 1), references moved if needed.  masked: some token may be unseen,
    // those from tok_end on all are.
    constexpr int NB = 2;
    const auto softmax_blocks = [&](bool masked, int tok0, int tok_end, float (&sc)[NB][4], const float (&k_scale)[NB], const float (&v_scale)[NB],
                                    uint32_t (&ph)[NB][2], uint32_t (&pl)[NB][2]) {
      bool above = false;
      // the V scale where the row sees some of the block
      const auto seen_scale = [&](int n, int e) {
        const int tok = tok0 + n * kQuantBlock;
        return !masked || (tok < tok_end && (tok <= pos[e] || tok < prefix)) ? v_scale[n] : -INFINITY;
      };
      // x - m_ref, in base-2 units
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const float f0 = c_row[0] * k_scale[n], f1 = c_row[1] * k_scale[n];
        if (plain) {
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[n][i] = fmaf(sc[n][i], i & 1 ? f1 : f0, -m_ref[i & 1]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            sc[n][i] = score(sc[n][i] * (i & 1 ? f1 : f0), i & 1, tok0 + n * kQuantBlock + 8 * (i >> 1) + r) - m_ref[i & 1];
        }
        if (masked) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int tok = tok0 + n * kQuantBlock + 8 * (i >> 1) + r;
            if (!(tok < tok_end && (tok <= pos[i & 1] || tok < prefix))) sc[n][i] = -INFINITY;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) above |= sc[n][i] > grow[i & 1];
        above |= v_scale[n] > v_low;
      }
      if (__any_sync(0xffffffffu, above)) {
        float alpha[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = -INFINITY;
#pragma unroll
          for (int n = 0; n < NB; ++n) mx = fmaxf(mx, fmaxf(sc[n][e], sc[n][2 + e]));
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
          const bool first = grow[e] != kQaGrow;         // nothing seen so far: sum and output are still 0
          alpha[e] = 1.f;
          if (mx > (first ? -INFINITY : 0.f)) {
            if (!first) alpha[e] = exp2_approx(-mx);
            grow[e] = kQaGrow;
            m_ref[e] += mx;
            l_run[e] *= alpha[e];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
              sc[n][e] -= mx;
              sc[n][2 + e] -= mx;
            }
          }
        }
        // (the open block's output is in units of 1: a first reference far below it would take it out of fp32's range)
        int least[2] = {kQaLeastExp, kQaLeastExp};
        if (!kF32 && n_codes < nb && __any_sync(0xffffffffu, v_low < 0.f)) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < MT; ++j) top = max(top, max(__float_as_uint(o[j][e]) & 0x7fffffffu, __float_as_uint(o[j][2 + e]) & 0x7fffffffu));
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, w));
            if (v_ref[e] < 0.f) least[e] = max(kQaLeastExp, (int)(top >> 23) - 95);      // 2^100 of the reference's units at most
          }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float v_top = fmaxf(seen_scale(0, e), seen_scale(1, e));
          if (v_top > v_ref[e]) {
            // the power of two above the scale
            const int ex = max((int)(__float_as_uint(v_top) >> 23) + 1, least[e]);
            const float old = fabsf(v_ref[e]) * (1.f / kQaPScale);
            v_ref[e] = __uint_as_float(ex << 23);
            v_inv[e] = kQaPScale * __uint_as_float((254 - ex) << 23);
            alpha[e] *= old * v_inv[e];
          }
        }
        v_low = fminf(v_ref[0], v_ref[1]);
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
          for (int f = 0; f < 4; ++f) o[j][f] *= alpha[f & 1];
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const float pv[2] = {v_scale[n] * v_inv[0], v_scale[n] * v_inv[1]};
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = exp2_approx(sc[n][i]);
          l_run[i & 1] += p[i];
          p[i] *= pv[i & 1];
          if (masked && sc[n][i] == -INFINITY) p[i] = 0.f;       // (0 times a scale that is NaN)
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const HalfPair w = split_pair<kF32>(p[2 * t], p[2 * t + 1]);
          ph[n][t] = movm(w.hi);
          if (kF32) pl[n][t] = movm(w.lo);
        }
      }
    };
    const auto mma_pv = [&](float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&ph)[2], const uint32_t (&pl)[2]) {
      mma_m16n8k16_f16(d, a0, a1, a2, a3, ph[0], ph[1]);
      if (kF32) mma_m16n8k16_f16(d, a0, a1, a2, a3, pl[0], pl[1]);
    };

    // ---- the open block, in the storage type, while the first copies are on their way
    if (n_codes < nb) {
      const int n_open = len - n_full * kQuantBlock;
      const long long open_at = ((long long)slot * H + h) * kQuantBlock * D;
      const T* kt = static_cast<const T*>(g.tail[0]) + open_at;
      const T* vt = static_cast<const T*>(g.tail[1]) + open_at;
      Quad<T> kq[2][KS], vq[4][NT / 4];              // key rows r, r + 8; value rows 2 c, 2 c + 1, 2 c + 8, 2 c + 9, this lane's features
      // (fp32: the queries' order of features.  bf16: one of their own in which four lanes read 64 bytes side by side.)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int x = 0; x < KS; x += Quad<T>::kPerLoad)
          if (r + 8 * t < n_open) Quad<T>::load16(kt + (r + 8 * t) * D + (kF32 ? KC * 16 * c + 4 * x : 16 * x + 8 * c), &kq[t][x]);
          else Quad<T>::zero16(&kq[t][x]);
      const auto load_values = [&]() {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int tok = 2 * c + (t & 1) + (t >> 1) * 8;
#pragma unroll
          for (int x = 0; x < NT / 4; x += Quad<T>::kPerLoad)
            if (tok < n_open) Quad<T>::load16(vt + tok * D + NT * r + 4 * x, &vq[t][x]);
            else Quad<T>::zero16(&vq[t][x]);
        }
      };
      if (!kF32) load_values();                      // (fp32 rows take twice the registers: the values after the scores)
      // A block with an infinity or NaN acts as a block of codes does: its scale is NaN and its values are 0, so that a query
      // that sees none of it is left alone.
      float sc[4] = {0.f, 0.f, 0.f, 0.f}, v_mul = 1.f;
      float f_row[2], f_tok[2] = {1.f, 1.f};         // what the products of query row 2 c + e and token r + 8 t are multiplied by
      float v_up[4], v_tok[2];                       // fp32: the powers of two of this lane's value rows; 1 / that of tokens r, r + 8
      if constexpr (kF32) {
        // fp16 pairs, each token's around its own power of two: what a query does not see has no part in what it does
        uint32_t bad = 0;
        float k_up[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          uint32_t top = 0;
#pragma unroll
          for (int x = 0; x < KS; ++x) top = kq[t][x].top(top);
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          k_up[t] = scale_up_to_half(__uint_as_float(top), &f_tok[t]);
          bad |= top >= 0x7f800000u;
        }
        const bool k_ok = !__any_sync(0xffffffffu, bad);
#pragma unroll
        for (int x = 0; x < KS; ++x) {
          HalfPair p[4];                             // tokens r, r + 8; elements 0, 1 and 2, 3
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!k_ok) kq[t][x].zero();
#pragma unroll
            for (int f = 0; f < 2; ++f) p[2 * f + t] = split_pair<true>(kq[t][x].get(2 * f) * k_up[t], kq[t][x].get(2 * f + 1) * k_up[t]);
          }
          mma_m16n8k16_f16(sc, p[0].hi, p[1].hi, p[2].hi, p[3].hi, qh[x][0], qh[x][1]);
          mma_m16n8k16_f16(sc, p[0].hi, p[1].hi, p[2].hi, p[3].hi, ql[x][0], ql[x][1]);
          mma_m16n8k16_f16(sc, p[0].lo, p[1].lo, p[2].lo, p[3].lo, qh[x][0], qh[x][1]);
        }
        f_row[0] = k_ok ? c_row[0] : __uint_as_float(0x7fc00000u);
        f_row[1] = k_ok ? c_row[1] : __uint_as_float(0x7fc00000u);
        load_values();
        bad = 0;
        float back[4];                               // (0 for a row of zeros)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uint32_t top = 0;
#pragma unroll
          for (int x = 0; x < NT / 4; ++x) top = vq[t][x].top(top);
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, w));
          v_up[t] = scale_up_to_half(__uint_as_float(top), &back[t]);
          if (top < 0x00800000u) back[t] = 0.f;
          bad |= top >= 0x7f800000u;
        }
        if (__any_sync(0xffffffffu, bad)) v_mul = __uint_as_float(0x7fc00000u);
        // token r is value row r & 1 of lanes r / 2, r + 8 the row two on
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float even = __shfl_sync(0xffffffffu, back[2 * t], r >> 1), odd = __shfl_sync(0xffffffffu, back[2 * t + 1], r >> 1);
          v_tok[t] = r & 1 ? odd : even;
        }
      } else {
        // bf16 rows are operands as they are.  Zero times an element tells whether it is finite.
        uint32_t k_bad = 0, v_bad = 0;
        Quad<T> qt[KS];
#pragma unroll
        for (int x = 0; x < KS; x += 2)
          if (ok) Quad<T>::load16(qp + 16 * x + 8 * c, &qt[x]);
          else Quad<T>::zero16(&qt[x]);
#pragma unroll
        for (int x = 0; x < KS; ++x) {
          mma_m16n8k16_bf16(sc, kq[0][x].w.x, kq[1][x].w.x, kq[0][x].w.y, kq[1][x].w.y, qt[x].w.x, qt[x].w.y);
#pragma unroll
          for (int t = 0; t < 2; ++t) k_bad = zero_fma_bf16x2(kq[t][x].w.x, zero_fma_bf16x2(kq[t][x].w.y, k_bad));
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int x = 0; x < NT / 4; ++x) v_bad = zero_fma_bf16x2(vq[t][x].w.x, zero_fma_bf16x2(vq[t][x].w.y, v_bad));
        f_row[0] = f_row[1] = __any_sync(0xffffffffu, (k_bad & 0x7fff7fffu) != 0) ? __uint_as_float(0x7fc00000u) : a.scale * (a.softcap > 0.f ? 1.f : kLog2e);
        if (__any_sync(0xffffffffu, (v_bad & 0x7fff7fffu) != 0)) v_mul = __uint_as_float(0x7fc00000u);
      }
      if (v_mul != v_mul) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int x = 0; x < NT / 4; ++x) vq[t][x].zero();
      }
      // (the first block of the segment: the references are what it says, and there is nothing to scale)
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int tok = n_full * kQuantBlock + 8 * (i >> 1) + r;
        x[i] = tok < len && (tok <= pos[i & 1] || tok < prefix) ? score(sc[i] * (f_row[i & 1] * f_tok[i >> 1]), i & 1, tok) : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float mx = fmaxf(x[e], x[2 + e]);
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        if (mx > -INFINITY) {
          m_ref[e] = mx;
          grow[e] = kQaGrow;
        }
      }
      uint32_t ph[2], pl[2];
      float p[4];
      if constexpr (kF32) {
        // a row's reference: the largest 1 / power of two of the values that it sees
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = fmaxf(x[e] == -INFINITY ? 0.f : v_tok[0], x[2 + e] == -INFINITY ? 0.f : v_tok[1]);
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
          if (top > 0.f) {
            v_ref[e] = fmaxf(top, __uint_as_float(kQaLeastExp << 23));
            v_inv[e] = kQaPScale * __uint_as_float((254u << 23) - __float_as_uint(v_ref[e]));
          }
        }
        v_low = fminf(v_ref[0], v_ref[1]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = exp2_approx(x[i] - m_ref[i & 1]);
        l_run[i & 1] += p[i];
        float m = v_mul;
        if (kF32) m *= v_tok[i >> 1] * v_inv[i & 1];
        p[i] = x[i] == -INFINITY ? 0.f : p[i] * m;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if constexpr (kF32) {
          const HalfPair w = split_pair<true>(p[2 * t], p[2 * t + 1]);
          ph[t] = movm(w.hi);
          pl[t] = movm(w.lo);
        } else {
          // bf16 has the values' range, a pair of them 16 bits
          const uint32_t w = pack_bf16x2(p[2 * t], p[2 * t + 1]);
          ph[t] = movm(w);
          pl[t] = movm(pack_bf16x2(p[2 * t] - __uint_as_float(w << 16), p[2 * t + 1] - __uint_as_float(w & 0xffff0000u)));
        }
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {                 // features 2 m, 2 m + 1; tokens 0, 1 and 2, 3
        if constexpr (kF32) {
          HalfPair w[4];
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int f = 0; f < 2; ++f)
              w[2 * f + e] = split_pair<true>(vq[2 * f][m / 2].get(2 * (m & 1) + e) * v_up[2 * f], vq[2 * f + 1][m / 2].get(2 * (m & 1) + e) * v_up[2 * f + 1]);
          mma_pv(o[m], w[0].hi, w[1].hi, w[2].hi, w[3].hi, ph, pl);
          mma_m16n8k16_f16(o[m], w[0].lo, w[1].lo, w[2].lo, w[3].lo, ph[0], ph[1]);
        } else {
          uint32_t w[4];
#pragma unroll
          for (int f = 0; f < 2; ++f) {
            const uint32_t t0 = m & 1 ? vq[2 * f][m / 2].w.y : vq[2 * f][m / 2].w.x, t1 = m & 1 ? vq[2 * f + 1][m / 2].w.y : vq[2 * f + 1][m / 2].w.x;
            w[2 * f] = __byte_perm(t0, t1, 0x5410);
            w[2 * f + 1] = __byte_perm(t0, t1, 0x7632);
          }
          mma_m16n8k16_bf16(o[m], w[0], w[1], w[2], w[3], ph[0], ph[1]);
          mma_m16n8k16_bf16(o[m], w[0], w[1], w[2], w[3], pl[0], pl[1]);
        }
      }
    }

    // ---- the blocks held as codes, two per step
#pragma unroll 1
    for (int j = 0; j < n_codes; j += 2) {
      const bool two = j + 1 < n_codes;
      float sc[2][4], ks[2], vs[2];
      uint32_t src[2];
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int f = 0; f < 4; ++f) sc[n][f] = 0.f;
      if ((j & 31) == 0 && j > 0) {
        ++group;
        page_cur = page_next;
        ks_cur = ks_next;
        vs_cur = vs_next;
        page_next = load_pages(group + 1);
      }
      if ((j & 31) == 16) load_scales(group + 1, page_next, &ks_next, &vs_next);
      bool arrived = true;
      const uint32_t used_before = used;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        if (n == 0 || two) {
          const int st = used % kQaStages;
          arrived &= warp_wait(smem_u32(&sm.full[warp][st]), (used / kQaStages) & 1);
          src[n] = ring + st * qa_stage_bytes(D);
          ++used;
        } else {
          src[n] = src[0];                         // (an odd last block stands in for its partner, which is masked)
        }
        ks[n] = __shfl_sync(0xffffffffu, ks_cur, (j + (two ? n : 0)) & 31);
        vs[n] = __shfl_sync(0xffffffffu, vs_cur, (j + (two ? n : 0)) & 31);
      }
      if (!__all_sync(0xffffffffu, arrived)) {
        dead = true;
        used = used_before;
        break;
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        float sb[4] = {0.f, 0.f, 0.f, 0.f};        // two chains of products
#pragma unroll
        for (int i = 0; i < KC; ++i) {
          const uint4 k0 = lds16(src[n] + qa_off<D>(r, KC * c + i)), k1 = lds16(src[n] + qa_off<D>(r + 8, KC * c + i));
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t x0 = codes_bias<FMT>(w == 0 ? k0.x : w == 1 ? k0.y : w == 2 ? k0.z : k0.w);
            const uint32_t x1 = codes_bias<FMT>(w == 0 ? k1.x : w == 1 ? k1.y : w == 2 ? k1.z : k1.w);
            const int x = 4 * i + w;
            const uint32_t a0 = codes_pair<FMT, 0>(x0), a1 = codes_pair<FMT, 0>(x1), a2 = codes_pair<FMT, 1>(x0), a3 = codes_pair<FMT, 1>(x1);
            mma_m16n8k16_f16(w & 1 ? sb : sc[n], a0, a1, a2, a3, qh[x][0], qh[x][1]);
            if (kF32) mma_m16n8k16_f16(w & 1 ? sc[n] : sb, a0, a1, a2, a3, ql[x][0], ql[x][1]);
          }
        }
#pragma unroll
        for (int f = 0; f < 4; ++f) sc[n][f] += sb[f];
      }
      const int tok0 = (blk0 + j) * kQuantBlock;
      uint32_t ph[2][2], pl[2][2];
      softmax_blocks(!two || tok0 + 2 * kQuantBlock - 1 > pos_first, tok0, two ? 0x7fffffff : tok0 + kQuantBlock, sc, ks, vs, ph, pl);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        uint32_t vw[4][NT / 4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t at = src[n] + kQuantBlock * D + qa_off<D>(2 * c + (t & 1) + (t >> 1) * 8, r * NT / 16) + (NT == 16 ? 0 : (r & 1) * 8);
          if (NT == 16) {
            const uint4 w = lds16(at);
            vw[t][0] = w.x; vw[t][1] = w.y; vw[t][NT / 4 - 2] = w.z; vw[t][NT / 4 - 1] = w.w;
          } else {
            const uint2 w = lds8(at);
            vw[t][0] = w.x; vw[t][1] = w.y;
          }
        }
#pragma unroll
        for (int w = 0; w < NT / 4; ++w) {
          const uint32_t t0 = codes_bias<FMT>(vw[0][w]), t1 = codes_bias<FMT>(vw[1][w]), t2 = codes_bias<FMT>(vw[2][w]),
                         t3 = codes_bias<FMT>(vw[3][w]);
          // features 4 w, 4 w + 1 (lo) and 4 w + 2, 4 w + 3 (hi) of token pairs
          const uint32_t lo01 = __byte_perm(t0, t1, 0x5140), hi01 = __byte_perm(t0, t1, 0x7362);
          const uint32_t lo23 = __byte_perm(t2, t3, 0x5140), hi23 = __byte_perm(t2, t3, 0x7362);
          mma_pv(o[2 * w], codes_pair<FMT, 0>(lo01), codes_pair<FMT, 1>(lo01), codes_pair<FMT, 0>(lo23), codes_pair<FMT, 1>(lo23), ph[n], pl[n]);
          mma_pv(o[2 * w + 1], codes_pair<FMT, 0>(hi01), codes_pair<FMT, 1>(hi01), codes_pair<FMT, 0>(hi23), codes_pair<FMT, 1>(hi23), ph[n], pl[n]);
        }
      }
      __syncwarp();                                // (all lanes have read the blocks: they may be overwritten)
#pragma unroll
      for (int n = 0; n < 2; ++n)
        if (j + kQaStages + n < n_codes) issue(j + kQaStages + n);
    }
    if (dead) {
      // let every copy that was asked for land, as far as it does, before the shared memory is given back
      if (lane == 0) {
        report_opt(a.status, ECHOKV_ETIMEOUT);
        for (; used < filled; ++used) mbar_drain(smem_u32(&sm.full[warp][used % kQaStages]), (used / kQaStages) & 1);
      }
      break;
    }

    // ---- the segment's result
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) l_run[e] += __shfl_xor_sync(0xffffffffu, l_run[e], w);
    const float o_scale[2] = {fabsf(v_ref[0]) * (1.f / kQaPScale), fabsf(v_ref[1]) * (1.f / kQaPScale)};
    const bool starts = blk0 == 0, ends = seg_end == item_end;
    if (starts && ends) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int qrow = tile * kQaRows + 2 * c + e;
        if (qrow < n_rows) {
          const float inv = l_run[e] == 0.f ? 0.f : o_scale[e] / l_run[e];
          float v[NT];
#pragma unroll
          for (int j = 0; j < MT; ++j) {
            v[2 * j] = o[j][e] * inv;
            v[2 * j + 1] = o[j][2 + e] * inv;
          }
          T* dst = static_cast<T*>(a.out) +
                   ((long long)(first_token + (qrow >> a.group_shift)) * a.n_q_heads + h * a.group + (qrow & (a.group - 1))) * D + NT * r;
#pragma unroll
          for (int f = 0; f < NT; f += Vec16<T>::N) store16<T>(dst + f, v + f);
        }
      }
    } else {
      const int at = 2 * warp + (starts ? 1 : 0);
      if (lane == 0) {
        QaSeg& q = sm.seg[at];
        q.item = item; q.item_end = item_end;
        q.b = b; q.tile = tile; q.h = h;
        q.starts = starts; q.ends = ends;
        q.valid = 1;
      }
      float* dst = seg_rows(at);
      if (r == 0) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          sm.m[at][2 * c + e] = l_run[e] == 0.f ? -INFINITY : m_ref[e];
          sm.l[at][2 * c + e] = l_run[e];
        }
      }
      __syncwarp();                               // (the rows of the second kind lie over the ring)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int j = 0; j < MT; ++j)
          *reinterpret_cast<float2*>(dst + (2 * c + e) * D + NT * r + 2 * j) = make_float2(o[j][e] * o_scale[e], o[j][2 + e] * o_scale[e]);
    }
    u = seg_end;
  }

  // ---- segments of one item side by side in this CTA: combine them; what is still cut goes to the workspace.  A warp per query
  //      row; lane k looks at segment k.
  __syncthreads();
  if (warp >= kQaRows) return;
  const QaWork<D> ws(a.ws);
  constexpr int E = D / 32;
  static_assert(2 * kQaWarps <= 32, "a lane per segment");
  const bool is_seg = lane < 2 * kQaWarps && sm.seg[lane < 2 * kQaWarps ? lane : 0].valid;
  const unsigned long long my_item = is_seg ? sm.seg[lane].item : ~0ull;
  const float my_m = is_seg ? sm.m[lane][warp] : -INFINITY, my_l = is_seg ? sm.l[lane][warp] : 0.f;
  uint32_t todo = __ballot_sync(0xffffffffu, is_seg);
  QaDesc desc = {0, 0, 0, 0};
  while (todo) {
    const int i = __ffs(todo) - 1;
    const uint32_t mine = __ballot_sync(0xffffffffu, my_item == __shfl_sync(0xffffffffu, my_item, i)) & todo;
    todo &= ~mine;
    const QaSeg& first = sm.seg[i];
    const bool starts = first.starts, ends = sm.seg[31 - __clz(mine)].ends;
    const bool in = (mine >> lane) & 1;
    const float m = warp_max(in ? my_m : -INFINITY);
    // (a row that has seen nothing has the sum 0 -- or NaN)
    const float w = !in || my_l == 0.f ? 0.f : exp2_approx(my_m - m);
    const float l = warp_sum(in ? w * my_l : 0.f);
    float acc[E] = {};
    for (uint32_t left = mine; left; left &= left - 1) {
      const int k = __ffs(left) - 1;
      const float wk = __shfl_sync(0xffffffffu, w, k);
      const float* o = seg_rows(k) + warp * D + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += wk * o[e];
    }
    if (starts && ends) {
      const int4 s = per == 1 ? sm.info[first.b] : seq_info(a, first.b, false, without);
      const int qrow = first.tile * kQaRows + warp;
      if (qrow < s.w * a.group) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* dst = static_cast<T*>(a.out) +
                 ((long long)(s.z + (qrow >> a.group_shift)) * a.n_q_heads + first.h * a.group + (qrow & (a.group - 1))) * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) dst[e] = from_f32<T>(acc[e] * inv);
      }
    } else {
      const long long p = ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * kQaRows + warp;
      if (lane == 0) ws.ml[p] = make_float2(m, l);
#pragma unroll
      for (int e = 0; e < E; ++e) ws.o[p * D + lane * E + e] = acc[e];
      if (starts) desc = QaDesc{(int)(quotient(first.item_end - 1, share) - blockIdx.x) + 1, first.b, first.tile, first.h};
    }
  }
  if (tid == 0) ws.desc[blockIdx.x] = desc;
}

// Joins the items that shares cut: block g the one that begins in CTA g and goes on in the next ones.  Also zeroes the rows of
// unusable sequences.  Launched while the first kernel runs, it waits for that one's end.
template <typename T, int D>
__global__ void __launch_bounds__(kQaMergeThreads) quant_merge_kernel(const __grid_constant__ QuantAttnArgs a) {
  constexpr int E = D / 32;
  const int tid = threadIdx.x, lane = tid & 31, row = tid >> 5;
  const QaWork<D> ws(a.ws);
  asm volatile("griddepcontrol.wait;" ::: "memory");
#pragma unroll 1
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    const QuantSeq s = quant_seq(a, b);
    if (s.error && s.n > 0) {
      T* dst = static_cast<T*>(a.out) + (long long)s.first * a.n_q_heads * D;
      const long long n = (long long)s.n * a.n_q_heads * D;
      for (long long i = tid; i < n; i += kQaMergeThreads) dst[i] = from_f32<T>(0.f);
    }
  }
  const QaDesc d = ws.desc[blockIdx.x];
  if (d.n_parts == 0) return;
  const auto part = [&](int p) -> long long { return ((long long)(blockIdx.x + p) * 2 + (p == 0 ? 1 : 0)) * kQaRows + row; };
  const int4 s = seq_info(a, d.b, false, false);
  float m = -INFINITY;
  for (int p = lane; p < d.n_parts; p += 32) m = fmaxf(m, ws.ml[part(p)].x);
  m = warp_max(m);
  float l = 0.f, acc[E] = {};
#pragma unroll 4
  for (int p = 0; p < d.n_parts; ++p) {
    const float2 ml = ws.ml[part(p)];
    const float w = ml.y == 0.f ? 0.f : exp2_approx(ml.x - m);
    l += w * ml.y;
    const float* o = ws.o + part(p) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] += w * o[e];
  }
  const int qrow = d.tile * kQaRows + row;
  if (qrow >= s.w * a.group) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* dst = static_cast<T*>(a.out) +
           ((long long)(s.z + (qrow >> a.group_shift)) * a.n_q_heads + d.h * a.group + (qrow & (a.group - 1))) * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = from_f32<T>(acc[e] * inv);
}

template <typename T, int FMT, int D>
cudaError_t launch(const QuantAttnArgs& a, int sm_count, cudaStream_t stream) {
  constexpr size_t smem = qa_ring_bytes<D>() + sizeof(QaSmem<D>);
  static_assert(kQaStages * qa_stage_bytes(D) >= kQaRows * D * 4, "a segment's rows fit over a warp's ring");
  static_assert(smem <= 227 * 1024, "shared memory of one CTA");
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_smem(quant_attn_kernel<T, FMT, D>, smem, &done);
  if (e != cudaSuccess) return e;
  // the codes as rows of 128 bytes (64 two-byte elements to TMA), boxes of one block
  CUtensorMap maps[2];
  for (int i = 0; i < 2; ++i) {
    const uint64_t dims[2] = {64, (uint64_t)a.g.n_pages * a.g.n_kv_heads * a.g.page_tokens * D / 128}, strides[1] = {128};
    const uint32_t box[2] = {64, kQuantBlock * D / 128};
    if ((e = encode_tiled_bf16(&maps[i], a.g.codes[i], 2, dims, strides, box)) != cudaSuccess) return e;
  }
  const int grid = sm_count < kQaMaxCtas ? sm_count : kQaMaxCtas;
  quant_attn_kernel<T, FMT, D><<<grid, kQaThreads, smem, stream>>>(maps[0], maps[1], a);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kQaMergeThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, quant_merge_kernel<T, D>, a);
}

template <typename T>
cudaError_t launch_t(const QuantAttnArgs& a, int sm_count, cudaStream_t stream) {
  const bool i8 = a.format == ECHOKV_INT8;
  if (a.g.head_dim == 128) return i8 ? launch<T, ECHOKV_INT8, 128>(a, sm_count, stream) : launch<T, ECHOKV_E4M3, 128>(a, sm_count, stream);
  return i8 ? launch<T, ECHOKV_INT8, 64>(a, sm_count, stream) : launch<T, ECHOKV_E4M3, 64>(a, sm_count, stream);
}

}  // namespace

uint64_t quant_attn_workspace_bytes(int head_dim) {
  const uint64_t n = (uint64_t)kQaMaxCtas * (sizeof(QaDesc) + 2ull * kQaRows * (sizeof(float2) + (uint64_t)head_dim * sizeof(float)));
  return (n + 255) / 256 * 256;
}

cudaError_t launch_quant_attn(const QuantAttnArgs& a, int sm_count, cudaStream_t stream) {
  return a.dtype == ECHOKV_BF16 ? launch_t<__nv_bfloat16>(a, sm_count, stream) : launch_t<float>(a, sm_count, stream);
}

}  // namespace echokv

// Attention over a cache held in 8 bits for chunks of bf16 queries, on the 5th-generation tensor cores.
//
//   O = softmax(score(Q K^T)) V over 128 keys at a time, 256 query rows of one KV head per work item (the query heads that
//   share it, times the new tokens), as two tiles of 128 rows that share every key / value tile, so that one tile's products
//   run while the other's softmax does.
//
// The codes become fp16 operand tiles in shared memory (exactly, for K; rounded to fp16 with their scale, for V) on the way to the
// products: nothing dequantised is written to memory, and a tile is converted once for 256 query rows.  Roles of a CTA (one per SM):
//   warps 0-3 / 4-7  softmax of tile 0 / 1, a thread per query row, 32 keys at a time.  Probabilities are taken against a reference per
//                    row, 2^(s - ref), a whole number that moves only when 32 probabilities could leave fp16's range: the
//                    common piece is done in one pass without looking for its maximum.  When it moves, what the row has so far --
//                    its sum, its output, the probabilities of this tile already stored -- is scaled by a power of two.
//                    (Two threads per row: 436 against 383 us when the whole took that; asking for the next 32 scores before
//                    the present ones are done: 481 against 435.)
//   warps 8-14       conversion: codes of the next tile are on their way in registers while the present one is turned into fp16 and
//                    stored in the 128-byte swizzle (key tiles K-major, value tiles as stored, N-major).  Eight lanes of a
//                    warp keep the pages and scales of the tile's eight blocks.
//   warp 15          issues the products, by one elected thread: S_x = Q_x K^T from shared memory, O_x += P_x V with P_x in tensor memory
//                    over the first half of S_x.
// Tensor memory: S_0 | S_1 | O_0 | O_1.  The K scale multiplies the score beside the row's own factor (one value per 16 columns).
// A V scale is split at the power of two above it: the rest of it times 64 multiplies the codes on their way to fp16 (below 2^15), the
// power, in units of the item's largest, the probabilities, whose reference is per row: values that a row does not see have no
// part in its range.  (With the whole scale on the codes, in units of the largest: 300 against 305 us plain, 397 both capped, but a
// value 2^40 times the others took the rows before it to a hundred times their tolerance.)
// Work: the key tiles of all items, with a cost of 4 tiles to each item, are laid end to end and cut into equal shares, one per CTA.
// A share cuts at most two items; the parts of an item -- o / l, reference, l -- go to the workspace and a second kernel
// joins them in the order of their keys.  (2 x 1024 tokens over 8192 keys, 256 items for 148 SMs: 433 -> 393 us; one sequence of 64
// tokens over 32768 keys, 8 items: 630 -> 87 us.)  Every wait is bounded.
// Bound: 128 exponentials per row and tile at 16 per clock and SM take twice the products' time.  Measured (2 x 1024 tokens over
// 8192 keys, 32 / 8 heads, e4m3): 305 us = 845 TFLOP/s without a cap, 397 us = 649 with one; a tile of 128 keys takes both halves 2.4 us
// where its products take 1.1 and its exponentials 1.1: each half's scores -> probabilities (1.45 us) -> products (1.0 us) chain is
// longer than what the other half covers.  Tensor pipe 38 / 29 %, exponentials' pipe 38 / 30 %, issue slots 45 / 48 % busy.
// (Scores in pieces of 64 keys, so that the next 64's products run while the softmax works on these: half as wide and
// half again as many products, 400 us against 293 then.)
// A cache in 4 bits takes the same way: its values, code times scale, are fp16 exactly, for K and V both, so there are no scales beside the
// score or the probability.  (The same chunks 296 us, capped 391.)
#include <type_traits>

#include "fp4_common.cuh"

namespace echokv {

namespace {

constexpr int kCkTile = 128;                       // query rows per tile, keys per tile
constexpr int kCkRows = 2 * kCkTile;
constexpr int kCkSoftmaxThreads = 256, kCkConvThreads = 224;
constexpr int kCkThreads = kCkSoftmaxThreads + kCkConvThreads + 32;
constexpr int kCkChunkBytes = kCkTile * 128;       // [128 rows x 64 features] fp16, 128-byte swizzle
constexpr int kCkRing = 4;                         // scales and V references: see where they are written
// A reference that moves goes 2^r below the largest score the row has seen, so that its largest probability is above 2^(r - 1).  What
// is less than 2^-25 is 0 as fp16, while the sum (fp32) keeps it: over n keys up to n 2^-(24 + r) of the largest one's mass.  r =
// log2 n - 13 holds that to 2^-11, what rounding a probability to fp16 does (up to r = 8, 2 million keys); r is 0 at least, which leaves
// room for a sum 2^11 to 2^16 as large before the reference moves again.  Measured (2 x 1024 tokens over 8192 keys, scores of spread
// 2.5): 299 us, 416 with r = 6, 343 if the first reference comes from 32 keys instead of 128 (V scales whole on the codes, as they were
// then).  (References 2^8 ABOVE the scores never move here, 293 us, but with 0.9 of the mass on the first of 8192 keys the output is 6 % off, of 32768 keys half.)
__device__ __forceinline__ float ck_below(int n_keys) { return (float)min(8, max(0, 32 - __clz(n_keys - 1) - 13)); }
constexpr float kCkSumLimit = 65504.f;             // a row's 32 probabilities sum to less: each fits fp16
constexpr float kCkVScale = 64.f;
constexpr int kCkVSpan = 90;                      // V scales below 2^-90 of the item's largest share its unit (a sum of 2^-e times 2^11 pieces fits fp32)
constexpr int kCkMaxCtas = 160;                    // (of the workspace's layout)
constexpr int kCkMinShare = 3;                     // units per CTA at least
constexpr int kCkMergeCols = 16;                   // features per thread of the merge

struct CkDesc {                                    // an item cut at the end of CTA g's share
  int n_parts;                                     // CTAs that hold parts of it (0: none starts here)
  int first, n_rows, h, row0;
  int pad[3];
};
// workspace: [ctas] CkDesc | [ctas][2][256] (m, l) | [ctas][2][D / 4][256] four features of o / l
template <int D>
struct CkWork {
  CkDesc* desc;
  float2* ml;
  float4* o;
  __host__ __device__ explicit CkWork(unsigned char* ws) {
    desc = reinterpret_cast<CkDesc*>(ws);
    ml = reinterpret_cast<float2*>(ws + kCkMaxCtas * sizeof(CkDesc));
    o = reinterpret_cast<float4*>(ws + kCkMaxCtas * (sizeof(CkDesc) + 2 * kCkRows * sizeof(float2)));
  }
};

__device__ __forceinline__ uint64_t ck_desc(uint32_t smem_addr, uint32_t lead_bytes) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((smem_addr & 0x3ffffu) >> 4);
  d |= static_cast<uint64_t>(lead_bytes >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
// fp16 x fp16 -> fp32, M = 128: S with both operands K-major, O with an N-major B operand
constexpr uint32_t kCkIdescS = (1u << 4) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
template <int D>
__host__ __device__ constexpr uint32_t ck_idesc_pv() { return (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((128u >> 4) << 24); }

// byte offset of 16-byte piece `piece` (8 features) of row `row` in an operand tile of D features
__device__ __forceinline__ uint32_t ck_off(int row, int piece) {
  return (piece >> 3) * kCkChunkBytes + row * 128 + (((piece & 7) ^ (row & 7)) << 4);
}
__device__ __forceinline__ void sts16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ bool ck_wait(unsigned long long* bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  const uint32_t b = smem_u32(bar);
  if (mbar_try_wait(b, parity)) return true;
  const long long start = clock64();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(b, parity)) return true;
    if (*abort_flag) return false;
    if (clock64() - start > kWaitLimitCycles) {
      *abort_flag = 1;
      report_opt(status, ECHOKV_ETIMEOUT);
      return false;
    }
  }
}
// the same for a whole warp, with one answer
__device__ __forceinline__ bool ck_wait_warp(unsigned long long* bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  return __all_sync(0xffffffffu, ck_wait(bar, parity, abort_flag, status)) != 0;
}
// one arrival for a warp whose lanes are all done
__device__ __forceinline__ void warp_arrive(unsigned long long* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(bar));
}

// 16 consecutive columns of this thread's lane, into the first half of r (valid after tmem_ld_wait)
__device__ __forceinline__ void tmem_ld16_issue(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_st16_regs(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// x -> tanh(g x) for 32 of them (g[0] for the first 16), two at a time: y times a polynomial in z = y^2, the nearest one in the largest
// relative error (found by iteratively reweighted least squares on Chebyshev points) -- of degree 3 for z <= 1/4 (5.5e-7) or
// of degree 5 for z <= 1 (6e-7).  Returns the largest z (a NaN is smaller than anything here and stays one).
template <bool SMALL>
__device__ __forceinline__ float tanh_pieces(uint32_t (&x)[32], float g0, float g1) {
  constexpr float c0 = SMALL ? 0.999999463558197f : 0.9999994039535522f, c1 = SMALL ? -0.33326318860054016f : -0.3332904279232025f,
                  c2 = SMALL ? 0.13190296292304993f : 0.13281434774398804f, c3 = SMALL ? -0.04440222680568695f : -0.05160567909479141f;
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const float g = j < 8 ? g0 : g1;
    const uint64_t y = mul_f2(pack_u2(x[2 * j], x[2 * j + 1]), pack_f2(g, g)), z = mul_f2(y, y);
    float z0, z1;
    unpack_f2(z, z0, z1);
    top = max3(top, z0, z1);
    uint64_t s;
    if (SMALL) {
      s = pack_f2(c3, c3);
    } else {
      s = fma_f2(pack_f2(-0.003067061770707369f, -0.003067061770707369f), z, pack_f2(0.016743119806051254f, 0.016743119806051254f));
      s = fma_f2(s, z, pack_f2(c3, c3));
    }
    s = fma_f2(s, z, pack_f2(c2, c2));
    s = fma_f2(s, z, pack_f2(c1, c1));
    s = fma_f2(s, z, pack_f2(c0, c0));
    unpack_u2(mul_f2(y, s), x[2 * j], x[2 * j + 1]);
  }
  return top;
}

// Issued by one elected thread of a warp whose lanes are together, so that descriptors stay in uniform registers (from a branch of lane 0
// alone each operand is moved there anew: 70-90 cycles per product instead of the 32-64 it takes)
__device__ __forceinline__ void ck_mma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void ck_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void ck_commit(unsigned long long* bar) {
  asm volatile(
      "{\n\t.reg .pred e;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
      ::"r"(smem_u32(bar))
      : "memory");
}

// What the softmax of a row needs beside its scores.
struct CkRow {
  uint32_t s_addr, o_addr;                         // tensor memory: scores (and probabilities) of the tile, output so far
  float c_row, cap_in, cap_out, slope2, below;
  int capped, biased;
  int pos;
};
// 32 keys of a row (columns 32 c .. of the tile, keys key0 ..) the careful way: any score transform, masks (the first n_vis keys of the tile
// are seen), and the reference moved where the probabilities need it -- then what the row has so far (its sum, the
// probabilities of this tile already stored, its output if there is one) is scaled by a power of two.  m: the reference, a
// whole number, -inf until the row has seen a key.  Returns (m, l).  A function of its own, so that the common way's registers
// and instructions are its own too.
template <int D>
__device__ __noinline__ float2 careful_piece(const CkRow w, const int c, const int key0, const int n_vis, const bool has_output, float f0,
                                             float f1, const float4 v_exp, float m_ref, float l_run) {
  uint32_t sr[32], pk[16];
  tmem_st_wait();
  tmem_ld32_issue(w.s_addr + 32 * c, sr);
  tmem_ld_wait();
#pragma unroll
  for (int j = 0; j < 32; ++j) sr[j] = __float_as_uint(__uint_as_float(sr[j]) * (j < 16 ? f0 : f1));
  // (a loop for each transform: branches inside one loop cost 2 us a piece)
  if (w.capped) {
#pragma unroll
    for (int j = 0; j < 32; ++j) sr[j] = __float_as_uint(w.cap_out * tanh_f32(__uint_as_float(sr[j]) * w.cap_in));
  }
  if (w.biased) {
    const float d = (float)(w.pos - key0);         // (exact up to 2^24 keys, as the distances themselves)
#pragma unroll
    for (int j = 0; j < 32; ++j) sr[j] = __float_as_uint(__uint_as_float(sr[j]) - w.slope2 * fabsf(d - j));
  }
  const int vis_c = n_vis - 32 * c;
  if (__any_sync(0xffffffffu, vis_c < 32)) {
#pragma unroll
    for (int j = 0; j < 32; ++j) sr[j] = j < vis_c ? sr[j] : 0xff800000u;
  }
  // (with the V scale's part, as the common way has it)
#pragma unroll
  for (int j = 0; j < 32; ++j) sr[j] = __float_as_uint(__uint_as_float(sr[j]) + (j < 16 ? v_exp.x : v_exp.z));
  float sum = 0.f;
#pragma unroll 1
  for (int attempt = 0;; ++attempt) {
    const float m = m_ref == -INFINITY ? 0.f : m_ref;
    float sums[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float p0 = exp2_approx(__uint_as_float(sr[2 * j]) - m), p1 = exp2_approx(__uint_as_float(sr[2 * j + 1]) - m);
      sums[j >> 3] += p0 + p1;
      pk[j] = h2(p0, p1);
    }
    sum = fmaf(sums[0], v_exp.y, sums[1] * v_exp.w);
    const bool move = !(sums[0] + sums[1] < kCkSumLimit) || m_ref == -INFINITY;
    if (attempt > 0 || !__any_sync(0xffffffffu, move)) break;
    float alpha = 1.f;
    if (move) {
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 32; ++j) mx = fmaxf(mx, __uint_as_float(sr[j]));
      if (mx > m_ref + w.below) {
        const float m_new = ceilf(mx) - w.below;
        if (m_ref > -INFINITY) alpha = exp2_approx(m_ref - m_new);
        m_ref = m_new;
      }
      l_run *= alpha;
    }
    // (through fp32: probabilities near fp16's largest times a power of two below its smallest)
#pragma unroll 1
    for (int cc = 0; cc < c; ++cc) {
      uint32_t old[32];
      tmem_ld16_issue(w.s_addr + 16 * cc, old);
      tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float2 p = h2_float(old[j]);
        old[j] = h2(p.x * alpha, p.y * alpha);
      }
      tmem_st16(w.s_addr + 16 * cc, old);
    }
    if (has_output) {
      // O is at rest (the product that wrote these scores came after every earlier one)
#pragma unroll 1
      for (int cc = 0; cc < D / 16; ++cc) {
        uint32_t old[32];
        tmem_ld16_issue(w.o_addr + 16 * cc, old);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j) old[j] = __float_as_uint(__uint_as_float(old[j]) * alpha);
        tmem_st16(w.o_addr + 16 * cc, old);
      }
    }
    tmem_st_wait();
  }
  tmem_st16_regs(w.s_addr + 16 * c, pk);
  return make_float2(m_ref, l_run + sum);
}

// The row blocks of a sequence: block j holds tokens [j per, (j + 1) per) times the group and sees kv_end(j) keys.  Everything is a
// power of two but the lengths, so that the tiles of the first j blocks have a closed form.
struct CkSeq {
  int slot, len, first, n;                         // (n = 0: not a sequence of this kernel)
  int prefix, blocks, per_shift;                   // 2^per_shift tokens per block
  __device__ __forceinline__ int kv_end(int j) const {
    const long long last = min((long long)n, (long long)(j + 1) << per_shift);
    return (int)max((long long)(len - n) + last, (long long)prefix);
  }
  // sum over i < m of floor(i / 2^shift)
  __device__ __forceinline__ static unsigned long long floors(unsigned long long m, int shift) {
    const unsigned long long q = m >> shift, r = m & ((1ull << shift) - 1);
    return (q == 0 ? 0ull : (q * (q - 1) / 2) << shift) + q * r;
  }
  // tiles of blocks [0, j): those that see no more than the prefix, those with all their tokens, the last
  __device__ __forceinline__ unsigned long long tiles(int j) const {
    const int full = min(j, blocks - 1), base = len - n;
    const int flat = prefix > base ? min(full, (prefix - base) >> per_shift) : 0;
    unsigned long long t = (unsigned long long)flat * ((prefix + kCkTile - 1) / kCkTile);
    // floor((base + 127 + i per) / 128) for i in (flat, full]
    if (per_shift <= 7) {
      const unsigned long long at = (unsigned long long)(base + kCkTile - 1) >> per_shift;
      t += floors(at + full + 1, 7 - per_shift) - floors(at + flat + 1, 7 - per_shift);
    } else {
      t += (unsigned long long)(full - flat) * ((base + kCkTile - 1) / kCkTile) +
           ((unsigned long long)full * (full + 1) - (unsigned long long)flat * (flat + 1));
    }
    return j == blocks ? t + (len + kCkTile - 1) / kCkTile : t;
  }
  __device__ __forceinline__ unsigned long long units(int j) const { return tiles(j) + (unsigned long long)j * kCkItemCost; }
};
struct CkItem {
  CkSeq s;
  int b, j, h;                                     // row block j of (sequence b, KV head h):
  int row0, n_rows, act;                           // rows [row0, row0 + 256) of n_rows; act: tiles of rows that hold one
  int kv_end, n_tiles;
  int t0, t1;                                      // tiles of keys that are this CTA's (none: t1 <= t0)
  unsigned long long end;                          // unit behind the item
};
__device__ __forceinline__ CkSeq ck_seq(const QuantAttnArgs& a, int b) {
  const QuantSeq s = quant_seq(a, b);
  CkSeq c;
  c.slot = s.slot; c.len = s.len; c.first = s.first;
  c.n = many_rows(a, s) ? s.n : 0;
  c.prefix = a.prefix && c.n > 0 ? min(a.prefix[b], s.len) : 0;
  c.blocks = (int)(((long long)c.n * a.group + kCkRows - 1) / kCkRows);
  c.per_shift = 8 - a.group_shift;
  return c;
}
__device__ __forceinline__ unsigned long long ck_ctas(unsigned long long total) {
  return min((unsigned long long)gridDim.x, total / kCkMinShare + 1);
}
__device__ __forceinline__ unsigned long long ck_units(const QuantAttnArgs& a, const CkSeq& s) {
  return s.n > 0 ? s.units(s.blocks) * a.g.n_kv_heads : 0;
}

struct CkTail {
  unsigned long long q_full[2], s_full[2], p_ready[2], o_done[2];
  unsigned long long k_full[2], k_empty[2], v_full[2], v_empty[2], drain;
  unsigned long long pre[kCkThreads + 1];
  unsigned long long warp_sums[32];
  float k_scale[kCkRing][8];                       // [tile][16-key block]
  alignas(16) float2 v_exp[kCkRing][8];                        // [tile][16-key block] how far the block's V scale is below the item's, (e, 2^-e), e <= 0
  float v_ref[kCkRing];                            // [item]
  unsigned long long share[2];                     // this CTA's units
  CkItem item[kCkThreads / 32];                    // every warp's present item (in registers it would spill)
  float red[3][kCkConvThreads / 32];
  uint32_t tmem_base;
  int abort_flag;
};
template <int D>
__host__ __device__ constexpr size_t ck_smem_bytes() { return 1024 + (size_t)(D / 64) * kCkChunkBytes * (2 + 2 + 2) + sizeof(CkTail); }

// Finding items is code of its own that all roles share: a step through it costs less than fetching copies of it.
// (sequence, row block, head) -> the rest; the item begins at unit `start`
__device__ __forceinline__ void ck_complete(const QuantAttnArgs& a, const CkTail& t, CkItem& it, unsigned long long start) {
  it.row0 = it.j * kCkRows;
  it.n_rows = it.s.n * a.group;
  it.act = it.n_rows - it.row0 > kCkTile ? 2 : 1;
  it.kv_end = it.s.kv_end(it.j);
  it.n_tiles = (it.kv_end + kCkTile - 1) / kCkTile;
  it.end = start + it.n_tiles + kCkItemCost;
  it.t0 = start >= t.share[0] ? 0 : max(0, (int)(t.share[0] - start) - kCkItemCost);
  it.t1 = (int)(min(t.share[1], it.end) - start) - kCkItemCost;
}
// the warp's item becomes the one that unit u is of (every lane writes the same)
__device__ __noinline__ void ck_find(const QuantAttnArgs& a, CkTail& t, unsigned long long u) {
  const int per = (a.B + kCkThreads - 1) / kCkThreads, H = a.g.n_kv_heads;
  int lo = 0, hi = kCkThreads;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.pre[mid] <= u) lo = mid; else hi = mid;
  }
  CkItem it;
  it.b = lo * per;
  unsigned long long base = t.pre[lo];
  it.s = ck_seq(a, it.b);
  if (per > 1) {
    for (unsigned long long n = ck_units(a, it.s); base + n <= u; n = ck_units(a, it.s)) {
      base += n;
      it.s = ck_seq(a, ++it.b);
    }
  }
  const unsigned long long rem = u - base;
  int j = 0, j_hi = it.s.blocks;                   // the row block: the last one whose units begin at or before u
#pragma unroll 1
  while (j_hi - j > 1) {
    const int mid = (j + j_hi) >> 1;
    if (it.s.units(mid) * H <= rem) j = mid; else j_hi = mid;
  }
  it.j = j;
  const uint32_t in_block = (uint32_t)(rem - it.s.units(j) * H), n = (it.s.kv_end(j) + kCkTile - 1) / kCkTile + kCkItemCost;
  it.h = (int)(in_block / n);
  ck_complete(a, t, it, u - (in_block - it.h * n));
  t.item[threadIdx.x >> 5] = it;
  __syncwarp();
}
// the one after it, if that begins in this CTA's share; true if it has tiles there (only the first and the last can be without)
__device__ __noinline__ bool ck_next(const QuantAttnArgs& a, CkTail& t) {
  CkItem it = t.item[threadIdx.x >> 5];
  if (it.end >= t.share[1]) return false;
  if (++it.h == a.g.n_kv_heads) {
    it.h = 0;
    if (++it.j == it.s.blocks) {
      it.j = 0;
      do it.s = ck_seq(a, ++it.b); while (it.s.n == 0);
    }
  }
  ck_complete(a, t, it, it.end);
  __syncwarp();
  t.item[threadIdx.x >> 5] = it;
  __syncwarp();
  return it.t1 > it.t0;
}
// the first that has tiles in the share, if any
__device__ __forceinline__ bool ck_first(const QuantAttnArgs& a, CkTail& t) {
  if (t.share[1] <= t.share[0]) return false;
  ck_find(a, t, t.share[0]);
  const CkItem& it = t.item[threadIdx.x >> 5];
  return it.t1 > it.t0 || ck_next(a, t);
}

template <int FMT, int D>
__global__ void __launch_bounds__(kCkThreads, 1) quant_chunk_kernel(const __grid_constant__ QuantAttnArgs a) {
  constexpr int NC = D / 64;
  constexpr int kTileBytes = NC * kCkChunkBytes;
  constexpr int kPieces = D / 16;                  // 16-code pieces of a row
  constexpr int kRowStep = kCkConvThreads / kPieces;          // rows that the conversion threads take at once,
  constexpr int NP = (kCkTile + kRowStep - 1) / kRowStep;     // one piece each, in this many goes
  extern __shared__ unsigned char ck_raw[];
  const uint32_t smem0 = (smem_u32(ck_raw) + 1023u) & ~1023u;
  const uint32_t q_addr = smem0, k_addr = q_addr + 2 * kTileBytes, v_addr = k_addr + 2 * kTileBytes;
  CkTail& t = *reinterpret_cast<CkTail*>(ck_raw + (smem0 - smem_u32(ck_raw)) + 6 * kTileBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const QuantGeom& g = a.g;
  const int H = g.n_kv_heads;
  volatile int* abort_flag = &t.abort_flag;

  const CkWork<D> ws(a.ws);
  if (!take_chunks(a, a.sm_count)) {               // (the same answer in every thread)
    if (tid == 0) ws.desc[blockIdx.x].n_parts = 0;
    return;
  }

  // ---- barriers, tensor memory, and the items of the call
  const int per = (a.B + kCkThreads - 1) / kCkThreads;
  if (tid == 0) {
    t.abort_flag = 0;
    for (int x = 0; x < 2; ++x) {
      mbar_init(smem_u32(&t.q_full[x]), kCkTile / 32);
      mbar_init(smem_u32(&t.s_full[x]), 1);
      mbar_init(smem_u32(&t.p_ready[x]), kCkTile / 32);
      mbar_init(smem_u32(&t.o_done[x]), 1);
      mbar_init(smem_u32(&t.k_full[x]), kCkConvThreads / 32);
      mbar_init(smem_u32(&t.k_empty[x]), 1);
      mbar_init(smem_u32(&t.v_full[x]), kCkConvThreads / 32);
      mbar_init(smem_u32(&t.v_empty[x]), 1);
    }
    mbar_init(smem_u32(&t.drain), 1);
    mbar_fence_init();
  }
  {
    unsigned long long n = 0;
#pragma unroll 1
    for (int b = tid * per; b < min(a.B, (tid + 1) * per); ++b) n += ck_units(a, ck_seq(a, b));
    unsigned long long x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) t.warp_sums[warp] = x;
    __syncthreads();
    unsigned long long before = 0;
    for (int w = 0; w < warp; ++w) before += t.warp_sums[w];
    t.pre[tid + 1] = before + x;
    if (tid == 0) t.pre[0] = 0;
    if (tid == kCkThreads - 1) {
      const unsigned long long total = before + x, ctas = ck_ctas(total);
      t.share[0] = blockIdx.x < ctas ? total * blockIdx.x / ctas : total;
      t.share[1] = blockIdx.x < ctas ? total * (blockIdx.x + 1) / ctas : total;
    }
  }
  if (warp == kCkThreads / 32 - 1) {
    tmem_alloc(smem_u32(&t.tmem_base), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = t.tmem_base;

  if (warp == kCkThreads / 32 - 1) {
    // =============================== products ===================================================
    {
      // an item that begins in this share and goes on behind it, for the merge
      CkDesc d = {};
      const unsigned long long u0 = t.share[0], u1 = t.share[1], total = t.pre[kCkThreads], ctas = ck_ctas(total);
      if (u1 > u0 && u1 < total) {
        ck_find(a, t, u1 - 1);
        const CkItem last = t.item[warp];
        __syncwarp();
        const unsigned long long start = last.end - last.n_tiles - kCkItemCost;
        const int done = (int)(u1 - start) - kCkItemCost;      // its tiles up to the share's end
        if (start + kCkItemCost >= u0 && done > 0 && done < last.n_tiles) {
          d.n_parts = (int)((last.end * ctas - 1) / total) - (int)blockIdx.x + 1;
          d.first = last.s.first; d.n_rows = last.n_rows; d.h = last.h; d.row0 = last.row0;
        }
      }
      if (lane == 0) ws.desc[blockIdx.x] = d;
    }
    {
      bool alive = true;
      uint32_t T = 0, n_item = 0, n_p[2] = {0, 0}; // tiles and items so far; tiles of either half
      // operand descriptors: the low words hold the address (in units of 16 bytes, far from a carry), the high words stay
      uint32_t q_lo0, k_lo0, v_lo0, kmajor_hi, v_hi;
      unpack_u2(ck_desc(q_addr, 16), q_lo0, kmajor_hi);
      unpack_u2(ck_desc(k_addr, 16), k_lo0, kmajor_hi);
      unpack_u2(ck_desc(v_addr, kCkChunkBytes), v_lo0, v_hi);
      const CkItem& it = t.item[warp];
      for (bool more = ck_first(a, t); more && alive; more = ck_next(a, t), ++n_item) {
        const auto issue_s = [&](int x, uint32_t tile) {
          const uint32_t q_lo = q_lo0 + x * (kTileBytes >> 4), k_lo = k_lo0 + (tile & 1) * (kTileBytes >> 4);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            constexpr uint32_t kStep = kCkChunkBytes >> 4;
            ck_mma_ss(tmem + x * 128, pack_u2(q_lo + (kk >> 2) * kStep + 2 * (kk & 3), kmajor_hi),
                        pack_u2(k_lo + (kk >> 2) * kStep + 2 * (kk & 3), kmajor_hi), kCkIdescS, kk > 0 ? 1u : 0u);
          }
          ck_commit(&t.s_full[x]);
          if (x == it.act - 1) ck_commit(&t.k_empty[tile & 1]);
        };
        // (of both tiles, at work or not: this thread is then never two items ahead of either's softmax warps)
        for (int x = 0; x < 2 && alive; ++x) alive = ck_wait_warp(&t.q_full[x], n_item & 1, abort_flag, a.status);
        if (alive) alive = ck_wait_warp(&t.k_full[T & 1], (T >> 1) & 1, abort_flag, a.status);
        if (!alive) break;
        tc_fence_after();
        for (int x = 0; x < it.act; ++x) issue_s(x, T);
        for (int tile = it.t0; tile < it.t1 && alive; ++tile, ++T) {
          if (!ck_wait_warp(&t.v_full[T & 1], (T >> 1) & 1, abort_flag, a.status)) { alive = false; break; }
          const uint32_t v_lo = v_lo0 + (T & 1) * (kTileBytes >> 4);
          for (int x = 0; x < it.act && alive; ++x) {
            if (!ck_wait_warp(&t.p_ready[x], n_p[x] & 1, abort_flag, a.status)) { alive = false; break; }
            ++n_p[x];
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)         // 16 keys: 8 columns of packed probabilities, 2048 bytes of value rows
              ck_mma_ts(tmem + 256 + x * D, tmem + x * 128 + 8 * kk, pack_u2(v_lo + 128 * kk, v_hi), ck_idesc_pv<D>(),
                                 (tile > it.t0 || kk > 0) ? 1u : 0u);
            if (tile + 1 == it.t1) ck_commit(&t.o_done[x]);
            if (x == it.act - 1) ck_commit(&t.v_empty[T & 1]);
            if (tile + 1 < it.t1) {
              if (x == 0) {
                if (!ck_wait_warp(&t.k_full[(T + 1) & 1], ((T + 1) >> 1) & 1, abort_flag, a.status)) { alive = false; break; }
                tc_fence_after();
              }
              issue_s(x, T + 1);
            }
          }
        }
        // (an idle second half waits for this too: its warps must not run items ahead of the barriers' phases)
        if (alive && it.act == 1) ck_commit(&t.o_done[1]);
      }
      if (!alive) {
        // every product issued so far retires before the tensor memory is given back
        ck_commit(&t.drain);
        mbar_drain(smem_u32(&t.drain), 0);
      }
    }
  } else if (warp >= kCkSoftmaxThreads / 32) {
    // =============================== conversion =================================================
    const int ct = tid - kCkSoftmaxThreads;
    bool alive = true;
    uint32_t T = 0, n_item = 0;
    const auto conv_all = [&](bool ok) {           // barrier of the conversion threads, ANDing a flag
      uint32_t r;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\t"
          "setp.ne.b32 q, %1, 0;\n\t"
          "bar.red.and.pred p, 1, 224, q;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(r)
          : "r"(ok ? 1u : 0u)
          : "memory");
      return r != 0;
    };
    // this thread's pieces: piece my_piece of rows my_row + kRowStep p.  Eight lanes that store together take four pieces of
    // an even row and of the next one: eight different banks in the swizzle.
    const int my_row = D == 128 ? (ct >> 5) * 4 + (lane >> 4) * 2 + ((lane >> 2) & 1) : ct / kPieces;
    const int my_piece = D == 128 ? ((lane >> 3) & 1) * 4 + (lane & 3) : ct % kPieces;
    // its two 16-byte halves in an operand tile; kRowStep rows on, the swizzle turns by kRowStep mod 8 (0 or 4)
    const uint32_t at0 = ck_off(my_row, 2 * my_piece), at1 = ck_off(my_row, 2 * my_piece + 1);
    const auto store_piece = [&](uint32_t dst, int p, const uint32_t (&w)[8]) {
      const uint32_t turn = (p & 1) ? (kRowStep & 4) << 4 : 0;
      sts16(dst + (at0 ^ turn) + p * kRowStep * 128, w[0], w[1], w[2], w[3]);
      sts16(dst + (at1 ^ turn) + p * kRowStep * 128, w[4], w[5], w[6], w[7]);
    };
    const CkItem& it = t.item[warp];
    if constexpr (FMT == kFp4) {
      // a piece is a group of 16 features of a token: 8 bytes of codes and their scale, exact in fp16
      constexpr int BB = fp4_block_bytes(D);
      struct Piece4 {
        uint2 codes;
        uint32_t scale;
      };
      const auto convert = [&](const Piece4& x, bool there, uint32_t (&w)[8]) {
        const uint32_t s2 = e4m3_scales(x.scale | x.scale << 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = there ? fp4_mul(e2m1_pair(x.codes.x >> (8 * e)), s2) : 0u;
          w[4 + e] = there ? fp4_mul(e2m1_pair(x.codes.y >> (8 * e)), s2) : 0u;
        }
      };
      for (bool more = ck_first(a, t); more && alive; more = ck_next(a, t)) {
        const int32_t* pages = a.table + (long long)it.s.slot * g.max_pages;
        // lane l < 8 looks up block l of a tile, one tile ahead (blocks behind the end: block 0 of the pool, not looked at)
        const auto ask_page = [&](int tile) {
          const int tok = (tile * 8 + lane) * kQuantBlock;
          return lane < 8 && tok < it.s.len ? pages[tok >> g.page_shift] : 0;
        };
        const auto checked = [&](int id) {
          if (id < 0 || id >= g.n_pages) {
            report_opt(a.status, ECHOKV_EBADPAGE);
            id = 0;
          }
          return id;
        };
        const unsigned char* blk[NP];
        Piece4 kc[NP], vc[NP];
        const auto fetch_k = [&](int tile, int page8) {
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const int row = min(my_row + kRowStep * p, kCkTile - 1);
            const int page = __shfl_sync(0xffffffffu, page8, row >> 4);
            const int inside = (tile * 8 + (row >> 4)) & ((g.page_tokens >> 4) - 1);
            blk[p] = g.blocks + (((long long)page * H + it.h) * (g.page_tokens >> 4) + inside) * BB;
          }
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const int r = min(my_row + kRowStep * p, kCkTile - 1) & 15, f = 16 * my_piece;
            kc[p].codes = *reinterpret_cast<const uint2*>(blk[p] + fp4_k_at(D, r, f));
            kc[p].scale = blk[p][fp4_ks_at(D, r, f)];
          }
        };
        const auto fetch_v = [&] {
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const int r = min(my_row + kRowStep * p, kCkTile - 1) & 15, f = 16 * my_piece;
            if constexpr (D == 128) {
              vc[p].codes = *reinterpret_cast<const uint2*>(blk[p] + fp4_v_at(D, r, f));
            } else {
              vc[p].codes.x = *reinterpret_cast<const uint32_t*>(blk[p] + fp4_v_at(D, r, f));
              vc[p].codes.y = *reinterpret_cast<const uint32_t*>(blk[p] + fp4_v_at(D, r, f + 8));
            }
            vc[p].scale = blk[p][fp4_vs_at(D, r, f)];
          }
        };
        int page_next = ask_page(it.t0 + 1);
        fetch_k(it.t0, checked(ask_page(it.t0)));
        fetch_v();
        for (int tile = it.t0; tile < it.t1; ++tile, ++T) {
          const int st = T & 1;
          const uint32_t parity = ((T >> 1) & 1) ^ 1;
          alive = __all_sync(0xffffffffu, ck_wait(&t.k_empty[st], parity, abort_flag, a.status));
          if (!alive) break;
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const int row = my_row + kRowStep * p;
            if (row >= kCkTile) break;
            uint32_t w[8];
            convert(kc[p], tile * kCkTile + row < it.s.len, w);
            store_piece(k_addr + st * kTileBytes, p, w);
          }
          fence_proxy_async_smem();
          warp_arrive(&t.k_full[st]);
          if (tile + 1 < it.t1) {
            // (the values of this tile are in registers: their places are not needed any more)
            fetch_k(tile + 1, checked(page_next));
            page_next = ask_page(tile + 2);
          }
          alive = __all_sync(0xffffffffu, ck_wait(&t.v_empty[st], parity, abort_flag, a.status));
          if (!alive) break;
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            const int row = my_row + kRowStep * p;
            if (row >= kCkTile) break;
            uint32_t w[8];
            convert(vc[p], tile * kCkTile + row < it.s.len, w);
            store_piece(v_addr + st * kTileBytes, p, w);
          }
          fence_proxy_async_smem();
          warp_arrive(&t.v_full[st]);
          if (tile + 1 < it.t1) fetch_v();
        }
      }
    } else
    for (bool more = ck_first(a, t); more; more = ck_next(a, t), ++n_item) {
      if (!conv_all(alive)) break;                 // (a wait that ran out: all leave together)
      const int32_t* pages = a.table + (long long)it.s.slot * g.max_pages;
      const int n_full = it.s.len / kQuantBlock, n_codes = min(n_full, (it.kv_end + kQuantBlock - 1) / kQuantBlock);   // blocks of codes seen
      // the open block is seen, and in one of these tiles
      const bool open = it.kv_end > n_full * kQuantBlock && n_full / 8 >= it.t0 && n_full / 8 < it.t1;
      const long long open_at = ((long long)it.s.slot * H + it.h) * kQuantBlock * D;
      const auto page_of = [&](int tok) {          // page of a token that exists
        int id = pages[tok >> g.page_shift];
        if (id < 0 || id >= g.n_pages) {
          report_opt(a.status, ECHOKV_EBADPAGE);
          id = 0;
        }
        return id;
      };
      const auto scale_at = [&](int blk, int page) {
        return ((long long)page * H + it.h) * (g.page_tokens / kQuantBlock) + ((blk * kQuantBlock & (g.page_tokens - 1)) / kQuantBlock);
      };
      // lane l < 8 keeps page and scales of block l of a tile, asked for two tiles (pages) and one (scales) ahead and looked at
      // only when they are needed
      const auto ask_page = [&](int tile) {
        const int blk = tile * 8 + lane;
        return lane < 8 && blk < n_codes ? pages[blk * kQuantBlock >> g.page_shift] : 0;
      };
      const auto checked = [&](int id) {
        if (id < 0 || id >= g.n_pages) {
          report_opt(a.status, ECHOKV_EBADPAGE);
          id = 0;
        }
        return id;
      };
      float ks_next = 0.f, vs_next = 0.f, vs_cur;
      const auto load_scales = [&](int tile, int page) {
        const int blk = tile * 8 + lane;
        ks_next = vs_next = 0.f;
        if (lane < 8 && blk < n_codes) {
          const long long at = scale_at(blk, page);
          vs_next = g.scales[1][at];
          ks_next = g.scales[0][at];
        }
      };
      // codes of this thread's pieces, fetched one tile ahead: K's when the present tile's K has been converted, so that they are on
      // their way while V is, and the other way round (rows behind the last block of codes: page 0's, not looked at)
      uint4 kc[NP], vc[NP];
      uint32_t at[NP];
      const unsigned char* k_base = g.codes[0] + 16 * my_piece;
      const unsigned char* v_base = g.codes[1] + 16 * my_piece;
      const auto fetch_k = [&](int tile, int page8) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const int row = min(my_row + kRowStep * p, kCkTile - 1);
          const int page = __shfl_sync(0xffffffffu, page8, row >> 4);
          at[p] = (uint32_t)((page * H + it.h) * g.page_tokens + ((tile * kCkTile + row) & (g.page_tokens - 1)));
        }
#pragma unroll
        for (int p = 0; p < NP; ++p) kc[p] = *reinterpret_cast<const uint4*>(k_base + (size_t)at[p] * D);
      };
      const auto fetch_v = [&] {
#pragma unroll
        for (int p = 0; p < NP; ++p) vc[p] = *reinterpret_cast<const uint4*>(v_base + (size_t)at[p] * D);
      };
      // 16 features of a row of the open block as fp16 pairs, or zeros
      const auto open_row = [&](int which, int row, float up, uint32_t (&w)[8]) {
        const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(g.tail[which]) + open_at + (long long)row * D + 16 * my_piece;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const uint4 x = *reinterpret_cast<const uint4*>(p + 8 * q);
          const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) w[4 * q + e] = h2(__uint_as_float(y[e] << 16) * up, __uint_as_float(y[e] & 0xffff0000u) * up);
        }
      };
      int page8 = checked(ask_page(it.t0)), page8_next = ask_page(it.t0 + 1);
      load_scales(it.t0, page8);
      fetch_k(it.t0, page8);
      fetch_v();
      // the largest V scale in these tiles, and the largest magnitudes of the open block
      float v_top = 0.f;
      for (int blk = 8 * it.t0 + ct; blk < min(n_codes, 8 * it.t1); blk += kCkConvThreads) v_top = fmaxf(v_top, g.scales[1][scale_at(blk, page_of(blk * kQuantBlock))]);
      uint32_t open_k = 0, open_v = 0;
      if (open) {
        const int n_open = it.s.len - n_full * kQuantBlock;
        const uint32_t* kt = reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(g.tail[0]) + open_at);
        const uint32_t* vt = reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(g.tail[1]) + open_at);
        for (int w = ct; w < n_open * D / 2; w += kCkConvThreads) {
          open_k = __vmaxu2(open_k, kt[w] & 0x7fff7fffu);
          open_v = __vmaxu2(open_v, vt[w] & 0x7fff7fffu);
        }
      }
      open_k = __reduce_max_sync(0xffffffffu, max(open_k & 0xffff0000u, open_k << 16));
      open_v = __reduce_max_sync(0xffffffffu, max(open_v & 0xffff0000u, open_v << 16));
      v_top = warp_max(v_top);
      if (lane == 0) {
        t.red[0][ct >> 5] = v_top;
        t.red[1][ct >> 5] = __uint_as_float(open_k);
        t.red[2][ct >> 5] = __uint_as_float(open_v);
      }
      conv_all(true);
#pragma unroll
      for (int w = 0; w < kCkConvThreads / 32; ++w) {
        v_top = fmaxf(v_top, t.red[0][w]);
        open_k = max(open_k, __float_as_uint(t.red[1][w]));
        open_v = max(open_v, __float_as_uint(t.red[2][w]));
      }
      // A block with an infinity or NaN: its K scale (that of the scores) is NaN, its rows are 0, so that a query that sees
      // none of it is left alone.
      float open_back = 1.f;
      const bool open_bad = open_k >= 0x7f800000u || open_v >= 0x7f800000u;
      const float open_up = scale_up_to_half(__uint_as_float(open_k), &open_back);
      const float open_scale = open_bad ? 0.f : __uint_as_float(open_v) * (1.f / 448.f);
      v_top = fmaxf(v_top, open_scale);
      // the power of two above it
      const uint32_t ve = v_top > 0.f ? (__float_as_uint(v_top) >> 23) + 1 : 127u;
      const float v_ref = __uint_as_float(ve << 23);
      // a block's values are held in units of the power of two above its own scale, the rest is its probabilities'
      const auto v_exponent = [&](float scale) { return min(max((__float_as_uint(scale) >> 23) + 1, (uint32_t)max(1, (int)ve - kCkVSpan)), ve); };
      const auto v_unit = [&](float scale) { return kCkVScale * __uint_as_float((254 - v_exponent(scale)) << 23); };
      // (the ring: item n + 4's value overwrites item n's when the tiles of items n + 1 to n + 3 have been written, two of
      // which the products have to have read, the first of them after the softmax warps took item n's result)
      if (ct == 0) t.v_ref[n_item % kCkRing] = v_ref * (1.f / kCkVScale);

      for (int tile = it.t0; tile < it.t1; ++tile, ++T) {
        const int st = T & 1;
        const uint32_t parity = ((T >> 1) & 1) ^ 1;
        alive = __all_sync(0xffffffffu, ck_wait(&t.k_empty[st], parity, abort_flag, a.status));
        if (!alive) break;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const int row = my_row + kRowStep * p, tok = tile * kCkTile + row, blk = tok / kQuantBlock;
          if (row >= kCkTile) break;
          uint32_t w[8];
          if (blk < n_codes) {
            const uint32_t c4[4] = {kc[p].x, kc[p].y, kc[p].z, kc[p].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t x = codes_bias<FMT>(c4[e]);
              w[2 * e] = codes_pair<FMT, 0>(x);
              w[2 * e + 1] = codes_pair<FMT, 1>(x);
            }
          } else if (open && !open_bad && tok < it.s.len) {
            open_row(0, tok - n_full * kQuantBlock, open_up, w);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = 0u;
          }
          store_piece(k_addr + st * kTileBytes, p, w);
        }
        // (the ring: tile T + 4's scales are written when S(T + 2) is complete, so after softmax(T + 1) was)
        vs_cur = vs_next;
        if (ct < 8) {
          if (open && tile * 8 + ct == n_full) ks_next = open_bad ? __uint_as_float(0x7fc00000u) : open_back;
          t.k_scale[T % kCkRing][ct] = vs_cur == vs_cur ? ks_next : vs_cur;
          const uint32_t below = ve - v_exponent(open && tile * 8 + ct == n_full ? open_scale : vs_cur);
          t.v_exp[T % kCkRing][ct] = make_float2(-(float)below, __uint_as_float((127u + below) << 23));
        }
        fence_proxy_async_smem();
        warp_arrive(&t.k_full[st]);
        if (tile + 1 < it.t1) {
          page8 = checked(page8_next);
          page8_next = ask_page(tile + 2);
          load_scales(tile + 1, page8);
          fetch_k(tile + 1, page8);
        }

        // what the values of this lane's block are multiplied by
        const float ratio = vs_cur * v_unit(vs_cur);
        const uint32_t r2_mine = h2(ratio, ratio);
        alive = __all_sync(0xffffffffu, ck_wait(&t.v_empty[st], parity, abort_flag, a.status));
        if (!alive) break;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const int row = my_row + kRowStep * p, tok = tile * kCkTile + row, blk = tok / kQuantBlock;
          const uint32_t r2 = __shfl_sync(0xffffffffu, r2_mine, (row >> 4) & 7);
          if (row >= kCkTile) break;
          uint32_t w[8];
          if (blk < n_codes && (r2 & 0x7fffu) <= 0x7c00u) {          // (not NaN)
            const uint32_t c4[4] = {vc[p].x, vc[p].y, vc[p].z, vc[p].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t x = codes_bias<FMT>(c4[e]);
              w[2 * e] = fp4_mul(codes_pair<FMT, 0>(x), r2);
              w[2 * e + 1] = fp4_mul(codes_pair<FMT, 1>(x), r2);
            }
          } else if (blk >= n_codes && open && !open_bad && tok < it.s.len) {
            open_row(1, tok - n_full * kQuantBlock, v_unit(open_scale), w);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = 0u;
          }
          store_piece(v_addr + st * kTileBytes, p, w);
        }
        fence_proxy_async_smem();
        warp_arrive(&t.v_full[st]);
        if (tile + 1 < it.t1) fetch_v();
      }
    }
  } else {
    // =============================== softmax ====================================================
    const int x = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_base = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_addr = lane_base + x * 128, o_addr = lane_base + 256 + x * D;
    const float cap_in = a.softcap > 0.f ? 1.f / a.softcap : 0.f, cap_out = a.softcap * kLog2e;
    uint32_t T = 0, n_item = 0, n_mine = 0, n_done = 0;   // (of this half: tiles and results, whose barriers move with them)
    const auto load_q = [&](const CkItem& it) {
      // the warp's 32 query rows, fetched into their places with 16 (8) lanes side by side on a row, all on their way at once
      // (rows of none of the queries: zeros), ...
      {
        constexpr int kLanes = D / 8, kPerGo = 32 / kLanes;
        const int my = lane / kLanes, p = lane % kLanes;
        const int r_warp = it.row0 + x * kCkTile + (warp & 3) * 32;
        const __nv_bfloat16* qb = static_cast<const __nv_bfloat16*>(a.q) + (long long)it.s.first * a.q_stride + (long long)it.h * a.group * D + 8 * p;
#pragma unroll 1
        for (int go = 0; go < kLanes; ++go) {
          const int rr = go * kPerGo + my, rq = r_warp + rr;           // row of the warp, of the sequence
          const bool ok = rq < it.n_rows;
          const void* src = ok ? qb + (long long)(rq >> a.group_shift) * a.q_stride + (rq & (a.group - 1)) * D : a.q;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(q_addr + x * kTileBytes + ck_off((warp & 3) * 32 + rr, p)), "l"(src),
                       "r"(ok ? 16 : 0)
                       : "memory");
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
      }
      // ... then made fp16 around its power of two by the row's own thread (the swizzle keeps the lanes on different banks)
      const uint32_t q_row = q_addr + x * kTileBytes + row * 128;
      const auto q_at = [&](int p) { return q_row + (p >> 3) * kCkChunkBytes + (((p & 7) ^ (row & 7)) << 4); };
      const auto read4 = [&](int p, uint4 (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w) : "r"(q_at(p + i)) : "memory");
      };
      uint32_t top = 0;
#pragma unroll 1
      for (int p = 0; p < D / 8; p += 4) {
        uint4 v[4];
        read4(p, v);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          top = __vmaxu2(__vmaxu2(top, __vmaxu2(v[i].x & 0x7fff7fffu, v[i].y & 0x7fff7fffu)), __vmaxu2(v[i].z & 0x7fff7fffu, v[i].w & 0x7fff7fffu));
      }
      float c_row;
      const float up = query_scale(__uint_as_float(max(top & 0xffff0000u, top << 16)), a.softcap > 0.f, &c_row);
#pragma unroll 1
      for (int p = 0; p < D / 8; p += 4) {
        uint4 v[4];
        read4(p, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t y[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
          uint32_t z[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] = h2(__uint_as_float(y[e] << 16) * up, __uint_as_float(y[e] & 0xffff0000u) * up);
          sts16(q_at(p + i), z[0], z[1], z[2], z[3]);
        }
      }
      c_row *= a.scale * (a.softcap > 0.f ? 1.f : kLog2e);
      fence_proxy_async_smem();
      warp_arrive(&t.q_full[x]);
      return c_row;
    };
    const CkItem& it = t.item[warp];
    bool more = ck_first(a, t);
    float c_row = more ? load_q(it) : 0.f;
    while (more) {
      if (x >= it.act) {
        T += it.t1 - it.t0;
        if (!__all_sync(0xffffffffu, ck_wait(&t.o_done[x], n_done & 1, abort_flag, a.status))) break;
        ++n_done;
        ++n_item;
        more = ck_next(a, t);
        if (more) c_row = load_q(it);
        continue;
      }
      const int r = it.row0 + x * kCkTile + row;
      const bool row_ok = r < it.n_rows;
      const int qi = row_ok ? r >> a.group_shift : 0, head = it.h * a.group + (r & (a.group - 1));
      const int pos = it.s.len - it.s.n + qi;
      // keys [0, vis) are seen; a row of none of the queries sees everything (its scores are 0) and goes nowhere
      const int vis = row_ok ? max(pos + 1, it.s.prefix) : 0x7fffffff;
      const float slope2 = a.slopes && row_ok ? a.slopes[head] * kLog2e : 0.f;
      CkRow w;
      w.s_addr = s_addr; w.o_addr = o_addr;
      w.c_row = c_row; w.cap_in = cap_in; w.cap_out = cap_out; w.slope2 = slope2;
      w.below = ck_below(it.kv_end);
      w.capped = a.softcap > 0.f; w.biased = a.slopes != nullptr;
      w.pos = pos;
      // the reference (-inf until the row has seen a key) and the sum of the row's probabilities
      float m_ref = -INFINITY, l_run = 0.f;
      bool alive = true, wide = false;             // wide: the capped scores need the longer polynomial (as the last tile's did)
      for (int tile = it.t0; tile < it.t1; ++tile, ++T, ++n_mine) {
        alive = __all_sync(0xffffffffu, ck_wait(&t.s_full[x], n_mine & 1, abort_flag, a.status));
        if (!alive) break;
        tc_fence_after();
        const int n_vis = max(0, min(kCkTile, vis - tile * kCkTile));
        // (the values of the 4-bit cache are whole in their operands)
        const auto k_scale = [&](int i) { return FMT == kFp4 ? 1.f : t.k_scale[T % kCkRing][i]; };
        const auto v_exp2 = [&](int c) {
          return FMT == kFp4 ? make_float4(0.f, 1.f, 0.f, 1.f) : *reinterpret_cast<const float4*>(&t.v_exp[T % kCkRing][2 * c]);
        };
        // the common way: the reference where it is
        float top = 0.f;
        const auto piece = [&](auto mode_tag, auto masked_tag, uint32_t (&sr)[32], int c) {
          constexpr int kMode = decltype(mode_tag)::value;               // 0: scores as they are, 1 / 2: capped, short / long polynomial
          constexpr bool kMasked = decltype(masked_tag)::value;          // some key of the tile is not seen
          const int vis_c = max(0, min(32, n_vis - 32 * c));
          const uint32_t seen = kMasked ? (uint32_t)((1ull << vis_c) - 1) : 0xffffffffu;
          float f0 = c_row * k_scale(2 * c), f1 = c_row * k_scale(2 * c + 1);      // (16 keys each)
          bool bad = false;
          if (kMode > 0) {
            const float z = tanh_pieces<kMode == 1>(sr, f0 * cap_in, f1 * cap_in);
            top = fmaxf(top, z);
            bad = !(z <= (kMode == 1 ? 0.25f : 1.f)) && (!kMasked || vis_c > 0);
            f0 = f1 = cap_out;
          }
          // p times 2^e of its block's V scale: what a row does not see has no part in its products' range
          const float4 ve = v_exp2(c);
          uint32_t pk[16];
          uint64_t sum2[2] = {0ull, 0ull};           // of the first 16 keys, of the others
          const uint64_t nm0 = pack_f2(ve.x - m_ref, ve.x - m_ref), nm1 = pack_f2(ve.z - m_ref, ve.z - m_ref);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float f = j < 8 ? f0 : f1;
            float y0, y1;
            unpack_f2(fma_f2(pack_u2(sr[2 * j], sr[2 * j + 1]), pack_f2(f, f), j < 8 ? nm0 : nm1), y0, y1);
            if (kMasked && !(seen >> (2 * j) & 1)) y0 = -INFINITY;
            if (kMasked && !(seen >> (2 * j + 1) & 1)) y1 = -INFINITY;
            const float p0 = exp2_approx(y0), p1 = exp2_approx(y1);
            sum2[j >> 3] = add_f2(sum2[j >> 3], pack_f2(p0, p1));
            pk[j] = h2(p0, p1);
          }
          float a0, a1, b0, b1;
          unpack_f2(sum2[0], a0, a1);
          unpack_f2(sum2[1], b0, b1);
          a0 += a1;
          b0 += b1;
          bad |= !(a0 + b0 < kCkSumLimit);
          if (__any_sync(0xffffffffu, bad)) return false;
          l_run += fmaf(a0, ve.y, b0 * ve.w);
          // over scores that have been read: columns 16 c .. of the tile's 128
          tmem_st16_regs(s_addr + 16 * c, pk);
          return true;
        };
        // pieces from c on done the common way; the rest of the tile, from the first one that it does not do for, the careful way
        const auto pieces_of = [&](auto mode_tag, auto masked_tag, int c) {
#pragma unroll 1
          for (; c < 4; ++c) {
            uint32_t sr[32];
            tmem_ld32_issue(s_addr + 32 * c, sr);
            tmem_ld_wait();
            if (!piece(mode_tag, masked_tag, sr, c)) break;
          }
          return c;
        };
        const auto careful = [&](int c) {
          const float2 r = careful_piece<D>(w, c, tile * kCkTile + 32 * c, n_vis, tile > it.t0, c_row * k_scale(2 * c), c_row * k_scale(2 * c + 1),
                                            v_exp2(c), m_ref, l_run);
          m_ref = r.x;
          l_run = r.y;
        };
        const bool full = __all_sync(0xffffffffu, n_vis == kCkTile);
        if (!w.biased && full && tile == it.t0) {
          // the first reference: what the tile's 128 keys ask for (the capped scores' largest is the largest score's)
          float mx = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            uint32_t sr[32];
            tmem_ld32_issue(s_addr + 32 * c, sr);
            tmem_ld_wait();
            float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              mx0 = fmaxf(mx0, __uint_as_float(sr[j]));
              mx1 = fmaxf(mx1, __uint_as_float(sr[16 + j]));
            }
            mx0 *= c_row * k_scale(2 * c);
            mx1 *= c_row * k_scale(2 * c + 1);
            if (w.capped) {
              mx0 = cap_out * tanh_f32(mx0 * cap_in);
              mx1 = cap_out * tanh_f32(mx1 * cap_in);
            }
            mx = fmaxf(mx, fmaxf(mx0 + v_exp2(c).x, mx1 + v_exp2(c).z));
          }
          if (mx > -INFINITY) m_ref = ceilf(mx) - w.below;
        }
        int done = 0;
        if (!w.biased) {
          // (a row that sees none of these keys needs no reference)
          if (!__all_sync(0xffffffffu, m_ref > -INFINITY || n_vis == 0)) careful(done++);
          if (__all_sync(0xffffffffu, m_ref > -INFINITY || n_vis == 0)) {
            const auto go = [&](auto mode_tag) {
              done = full ? pieces_of(mode_tag, std::false_type(), done) : pieces_of(mode_tag, std::true_type(), done);
            };
            if (!w.capped) {
              go(std::integral_constant<int, 0>());
            } else {
              if (wide) go(std::integral_constant<int, 2>()); else go(std::integral_constant<int, 1>());
              wide = __any_sync(0xffffffffu, top > 0.25f);
            }
          }
        }
#pragma unroll 1
        for (; done < 4; ++done) careful(done);
        tmem_st_wait();
        tc_fence_before();
        warp_arrive(&t.p_ready[x]);
      }
      if (!alive) break;
      // ---- the row's result.  The next item's queries come first: its scores are then under way meanwhile.  (This
      // item's scores are complete; its V reference stays in the ring until the products have seen the next queries.)
      const float inv = l_run == 0.f ? 0.f : (FMT == kFp4 ? a.out_scale : t.v_ref[n_item % kCkRing]) / l_run;
      const bool whole = it.t1 - it.t0 == it.n_tiles;
      // (a part: o / l beside the reference and l, in the slot of an item that goes on from the CTA before or in the next)
      const long long slot = (long long)blockIdx.x * 2 + (it.t0 == 0);
      if (!whole) ws.ml[slot * kCkRows + x * kCkTile + row] = make_float2(m_ref, l_run);
      float4* part = ws.o + slot * (D / 4) * kCkRows + x * kCkTile + row;
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.out) + ((long long)(it.s.first + qi) * a.n_q_heads + head) * D;
      ++n_item;
      more = ck_next(a, t);
      if (more) c_row = load_q(it);
      alive = __all_sync(0xffffffffu, ck_wait(&t.o_done[x], n_done & 1, abort_flag, a.status));
      if (!alive) break;
      ++n_done;
      tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t orow[32];
        tmem_ld32_issue(o_addr + 32 * c, orow);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(orow[j + e]) * inv;
          if (!whole) {
            part[(8 * c + j / 4) * kCkRows] = make_float4(v[0], v[1], v[2], v[3]);
            part[(8 * c + j / 4 + 1) * kCkRows] = make_float4(v[4], v[5], v[6], v[7]);
          } else if (row_ok) {
            store16<__nv_bfloat16>(dst + 32 * c + j, v);
          }
        }
      }
      tc_fence_before();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kCkThreads / 32 - 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// The items that were cut: a thread per row and 16 features, parts joined in the order of their keys.
template <int D>
__global__ void __launch_bounds__(kCkRows) quant_chunk_merge_kernel(const __grid_constant__ QuantAttnArgs a) {
  const CkWork<D> ws(a.ws);
  const int row = threadIdx.x, col = blockIdx.y * kCkMergeCols;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const CkDesc d = ws.desc[blockIdx.x];
  const int r = d.row0 + row;
  if (d.n_parts == 0 || r >= d.n_rows) return;
  const auto slot = [&](int p) -> long long { return (long long)(blockIdx.x + p) * 2 + (p == 0); };
  float m = -INFINITY;
  for (int p = 0; p < d.n_parts; ++p) m = fmaxf(m, ws.ml[slot(p) * kCkRows + row].x);
  float l = 0.f, acc[kCkMergeCols] = {};
#pragma unroll 2
  for (int p = 0; p < d.n_parts; ++p) {
    const float2 ml = ws.ml[slot(p) * kCkRows + row];
    const float w = ml.y == 0.f ? 0.f : exp2_approx(ml.x - m) * ml.y;
    l += w;
    const float4* o = ws.o + (slot(p) * (D / 4) + col / 4) * kCkRows + row;
#pragma unroll
    for (int e = 0; e < kCkMergeCols / 4; ++e) {
      const float4 v = o[e * kCkRows];
      acc[4 * e] += w * v.x; acc[4 * e + 1] += w * v.y; acc[4 * e + 2] += w * v.z; acc[4 * e + 3] += w * v.w;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < kCkMergeCols; ++e) acc[e] *= inv;
  __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(a.out) +
                       ((long long)(d.first + (r >> a.group_shift)) * a.n_q_heads + d.h * a.group + (r & (a.group - 1))) * D + col;
#pragma unroll
  for (int e = 0; e < kCkMergeCols; e += 8) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = acc[e + i];
    store16<__nv_bfloat16>(dst + e, v);
  }
}

template <int FMT, int D>
cudaError_t launch(const QuantAttnArgs& a, int sm_count, cudaStream_t stream) {
  constexpr size_t smem = ck_smem_bytes<D>();
  static_assert(smem <= 227 * 1024, "shared memory of one CTA");
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_smem(quant_chunk_kernel<FMT, D>, smem, &done);
  if (e != cudaSuccess) return e;
  const int grid = sm_count < kCkMaxCtas ? sm_count : kCkMaxCtas;
  quant_chunk_kernel<FMT, D><<<grid, kCkThreads, smem, stream>>>(a);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, D / kCkMergeCols);
  cfg.blockDim = dim3(kCkRows);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, quant_chunk_merge_kernel<D>, a);
}

}  // namespace

uint64_t quant_chunk_workspace_bytes(int head_dim) {
  const uint64_t n = (uint64_t)kCkMaxCtas * (sizeof(CkDesc) + 2ull * kCkRows * (sizeof(float2) + (uint64_t)head_dim * sizeof(float)));
  return (n + 255) / 256 * 256;
}

cudaError_t launch_quant_chunk(const QuantAttnArgs& a, int sm_count, cudaStream_t stream) {
  if (a.format == kFp4) return a.g.head_dim == 128 ? launch<kFp4, 128>(a, sm_count, stream) : launch<kFp4, 64>(a, sm_count, stream);
  const bool i8 = a.format == ECHOKV_INT8;
  if (a.g.head_dim == 128) return i8 ? launch<ECHOKV_INT8, 128>(a, sm_count, stream) : launch<ECHOKV_E4M3, 128>(a, sm_count, stream);
  return i8 ? launch<ECHOKV_INT8, 64>(a, sm_count, stream) : launch<ECHOKV_E4M3, 64>(a, sm_count, stream);
}

}  // namespace echokv

// Attention over a cache held in 4 bits, one or a few queries per sequence (decode steps, drafts to verify), over the whole cache or over
// pages that each token lists.
//
//   x_t = scale q . k_t  [capped by softcap tanh(x / softcap)] [- slope |p - t|],   o = sum_t 2^(x_t log2e - m) v_t / sum_t 2^(...)
//
// The blocks are read once from HBM and that is the bound; beside the stream every value has to be turned into fp16, 41 of them per
// clock and SM.  The design:
//
//   work     A unit is one 16-token block of one KV head for 8 or 16 query rows (the query heads that share the KV head, times a
//            sequence's new tokens).  The units of all sequences are laid end to end and cut into equal shares, one per CTA and
//            within it one per warp, computed on the device from the lengths.  A share cuts at most two (sequence, head) items;
//            their partial results (running maximum, sum, output) are combined inside the CTA through shared memory and between CTAs by a
//            second small kernel.  With lists an item is one token and head, its blocks those of its listed pages.
//   copies   A block is 18 d contiguous bytes (K and V codes and scales): one bulk copy into a ring of the warp's own, two blocks to a
//            stage.  The block's layout is the operands': what a lane reads lies side by side with what its neighbours read.
//   products mma.sync m16n8k16 in fp16 with the tokens (then the head's features) on the M rows and the 8 query rows on N.  A value
//            e2m1 x e4m3 has 6 bits and lies between 2^-10 and 2688: it is an fp16 exactly.  fp32 queries, and the
//            probabilities beside them, take a second product with their low-order halves (22 bits).
//   softmax  The running maximum is a reference that moves only when a score is 2^8 above it; probabilities are 2^5 times themselves, so
//            that fp16 holds them down to 2^-29 of the largest (with a second half, in fp32, to 2^-42).
// Measured (device time, both kernels): 16 requests over 32768 keys, 8 bf16 heads of 128 118 us, 5.1 TB/s (the copies alone 110; fp32
// queries 158); 32 ragged requests of 32 heads, pages of 16, 132 us, capped 147 (copies 122); one request of 777 keys 9.7; 8 drafts
// for each of 16 requests over 32768 keys 341 us (by items of 8 rows 434); 64 listed pages of 64 tokens for 16 tokens 27 us. The
// conversion to fp16 by the instruction and a byte select of its result: 118 us; by shifts 160, by whole-number arithmetic no better.
#include "fp4_common.cuh"
#include <type_traits>

#include "quant_rows.cuh"

namespace echokv {

namespace {

// Q tiles of 8 query rows make up an item: 1, or 2 where a call may have more rows than one tile has (their values are then converted once).
// (Heads of 128, one tile: 12 warps 119.5 us for 16 x 32768 keys, 14 134, 16 121; of 64, 16 x 8192 keys of 32 heads: 12 89, 16 79.
// A call's max_new decides for all of its rows: the single tokens of that batch take 118 us in a call of theirs, 138 to 140 where another
// sequence may have 3 tokens and more, 144 beside chunks.)
template <int D, int Q>
struct FqShape {
  static constexpr int kWarps = Q == 2 ? (D == 128 ? 8 : 12) : D == 128 ? 12 : 16, kThreads = kWarps * 32;
  static constexpr int kRows = 8 * Q;
};
constexpr int kFqTile = 8;                        // query rows per tile
constexpr int kFqStages = 3;                      // of two blocks each
constexpr int kFqMaxCtas = 512;
constexpr int kFqItemCost = 6;                    // what an item costs beside its blocks (queries, first copies, result), in blocks
constexpr float kFqBelow = 5.f;                   // the reference stands 2^5 below the largest score it was taken from,
constexpr float kFqGrow = 8.f + kFqBelow;         // and moves when a score is 2^13 above it (probabilities up to there fit fp16)
constexpr float kFqLowUp = 8192.f;                // (fp32) low-order halves of probabilities, 2^2 at most, are held 2^13 times themselves: down
                                                  // to 2^-42 of the largest, so that many small ones count beside a large one
constexpr int kFqNowhere = 0x40000000;            // the first token of a block that nobody sees

__host__ __device__ constexpr int fq_stage_bytes(int D) { return 2 * fp4_block_bytes(D); }

template <int THREADS>
struct FqPlanShared {
  unsigned long long pre[THREADS + 1];
  unsigned long long warp_sums[THREADS / 32];
  int4 info[THREADS];                             // slot, length, first token, tokens (0: nothing to do) of the owners
};

template <int D, int Q>
struct FqSmem {
  // a warp's segment that goes on from the warp before it, and (over the warp's ring, once that is at rest) the one
  // that goes on in the next warp
  static constexpr int kWarps = FqShape<D, Q>::kWarps, kRows = FqShape<D, Q>::kRows;
  float o_first[kWarps][kRows][D];
  QaSeg seg[2 * kWarps];
  float m[2 * kWarps][kRows], l[2 * kWarps][kRows];
  unsigned long long full[kWarps][kFqStages];
  FqPlanShared<FqShape<D, Q>::kThreads> plan;
  int2 tok[kWarps][kFqStages];                  // with lists: first tokens of a stage's blocks
};
template <int D, int Q>
__host__ __device__ constexpr size_t fq_ring_bytes() { return (size_t)FqShape<D, Q>::kWarps * kFqStages * fq_stage_bytes(D); }

// workspace: [ctas][2][rows] (m, l) | [ctas][2][rows][D] o
template <int ROWS>
struct FqWork {
  float2* ml;
  float* o;
  __host__ __device__ explicit FqWork(unsigned char* ws) {
    ml = reinterpret_cast<float2*>(ws);
    o = reinterpret_cast<float*>(ws + kFqMaxCtas * 2 * ROWS * sizeof(float2));
  }
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// Item owners: the sequences of the call, or with lists its tokens.
template <bool LIST>
__device__ __forceinline__ int owners(const Fp4AttnArgs& a) { return LIST ? a.n_tokens : a.B; }
template <bool LIST>
__device__ __forceinline__ QuantSeq owner(const Fp4AttnArgs& a, int b) {
  if (!LIST) return quant_seq(a, b);
  QuantSeq s;
  const int seq = a.t.seqs[b], pos = a.t.positions[b];
  s.first = b;
  s.n = seq < 0 ? 0 : 1;
  s.slot = 0;
  s.error = 0;
  s.len = pos + 1;
  if (seq < 0) return s;
  if (seq < a.B) s.slot = a.slots ? a.slots[seq] : seq;
  if (seq >= a.B || s.slot < 0 || s.slot >= a.g.max_batch) s.error = ECHOKV_EBADPAGE;
  else if (pos < 0 || pos >= a.g.max_pages * a.g.page_tokens) s.error = ECHOKV_EBADLENGTH;
  return s;
}
// What the kernel needs of an owner: w = 0 tokens where nothing is attended here.
// (without: the sequences of many rows are the chunk kernel's)
template <bool LIST>
__device__ __forceinline__ int4 owner_info(const Fp4AttnArgs& a, int b, bool tell, bool without) {
  const QuantSeq s = owner<LIST>(a, b);
  if (s.error && tell) report_opt(a.status, s.error);
  return make_int4(s.slot, s.len, s.first, s.error || (without && many_rows(a, s)) ? 0 : s.n);
}
template <int ROWS>
__device__ __forceinline__ int row_items(const QuantAttnArgs& a, int n) { return (n * a.group + ROWS - 1) / ROWS; }
template <bool LIST>
__device__ __forceinline__ int blocks_of(const Fp4AttnArgs& a, int len) {
  if (LIST) return min(a.t.n_select, ((len - 1) >> a.g.page_shift) + 1) << (a.g.page_shift - 4);
  return (len + kQuantBlock - 1) / kQuantBlock;
}
template <bool LIST, int ROWS>
__device__ __forceinline__ unsigned long long units_of(const Fp4AttnArgs& a, const int4& s) {
  return s.w == 0 ? 0 : (unsigned long long)row_items<ROWS>(a, s.w) * a.g.n_kv_heads * (blocks_of<LIST>(a, s.y) + kFqItemCost);
}

// How the work of a call is cut: every block of either kernel works it out from the lengths.  Up to 32 owners: a lane of every warp has
// one, and no thread waits for another; more: a thread has a run of them.
template <bool LIST, int THREADS, int ROWS>
struct FqPlan {
  const Fp4AttnArgs& a;
  FqPlanShared<THREADS>& sm;
  int n_own, per;
  bool few, without;
  int4 mine;                                      // (few) of this lane's owner
  unsigned long long mine_pre, total, share;
  // found: the owner of a unit, the first unit of it
  int b = -1;
  unsigned long long base;
  int4 info;

  __device__ __forceinline__ FqPlan(const Fp4AttnArgs& args, FqPlanShared<THREADS>& shared, int ctas, int min_share, bool tell) : a(args), sm(shared) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    without = !LIST && take_chunks(a, a.sm_count);
    n_own = owners<LIST>(a);
    few = n_own <= 32;
    per = (n_own + THREADS - 1) / THREADS;
    unsigned long long n = 0;
    if (few) {
      mine = make_int4(0, 0, 0, 0);
      if (lane < n_own) mine = owner_info<LIST>(a, lane, tell && warp == 0, without);
      n = units_of<LIST, ROWS>(a, mine);
    } else {
#pragma unroll 1
      for (int k = tid * per; k < min(n_own, (tid + 1) * per); ++k) {
        const int4 s = owner_info<LIST>(a, k, tell, without);
        if (per == 1) sm.info[k] = s;
        n += units_of<LIST, ROWS>(a, s);
      }
    }
    unsigned long long x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (few) {
      mine_pre = x - n;
      total = __shfl_sync(0xffffffffu, x, 31);
    } else {
      if (lane == 31) sm.warp_sums[warp] = x;
      __syncthreads();
      unsigned long long before = 0;
      for (int w = 0; w < warp; ++w) before += sm.warp_sums[w];
      sm.pre[tid + 1] = before + x;
      if (tid == 0) sm.pre[0] = 0;
      __syncthreads();
      total = sm.pre[THREADS];
    }
    share = quotient(total + ctas - 1, ctas);
    if (share < (unsigned long long)min_share) share = min_share;
  }
  __device__ __forceinline__ int4 info_of(int k) const {
    if (few) return make_int4(__shfl_sync(0xffffffffu, mine.x, k), __shfl_sync(0xffffffffu, mine.y, k), __shfl_sync(0xffffffffu, mine.z, k), __shfl_sync(0xffffffffu, mine.w, k));
    return per == 1 ? sm.info[k] : owner_info<LIST>(a, k, false, without);
  }
  // the owner of unit u < total, by a whole warp: the last one whose units begin at or before it (units are asked for in order)
  __device__ __forceinline__ void locate(unsigned long long u) {
    const int lane = threadIdx.x & 31;
    if (few) {
      b = __popc(__ballot_sync(0xffffffffu, lane < n_own && mine_pre <= u)) - 1;
      base = __shfl_sync(0xffffffffu, mine_pre, b);
      info = info_of(b);
      return;
    }
    static_assert(THREADS <= 1024, "a lane per run of 32 prefixes");
    // (with runs of owners: on from the last one found, whose units end where the next unit begins)
    if (per == 1 || b < 0) {
      const int run = __popc(__ballot_sync(0xffffffffu, lane < THREADS / 32 && sm.pre[lane * 32 < THREADS ? lane * 32 : 0] <= u)) - 1;
      const int at = run * 32 + __popc(__ballot_sync(0xffffffffu, sm.pre[run * 32 + lane] <= u)) - 1;
      b = at * per;
      base = sm.pre[at];
      info = info_of(b);
    }
    for (unsigned long long n = units_of<LIST, ROWS>(a, info); base + n <= u; n = units_of<LIST, ROWS>(a, info)) {
      base += n;
      info = info_of(++b);
    }
  }
};
// The item of a unit of the owner that the plan has found.
struct FqItem {
  int n_blk, h, tile;
  unsigned long long first, end;                  // its units: kFqItemCost, then one per block
};
template <bool LIST, int THREADS, int ROWS>
__device__ __forceinline__ FqItem item_of(const FqPlan<LIST, THREADS, ROWS>& p, unsigned long long u) {
  FqItem it;
  it.n_blk = blocks_of<LIST>(p.a, p.info.y);
  const int tiles = row_items<ROWS>(p.a, p.info.w), n = it.n_blk + kFqItemCost;
  const unsigned long long rem = u - p.base;
  const int ht = (int)quotient(rem, n);
  it.h = tiles == 1 ? ht : ht / tiles;
  it.tile = ht - it.h * tiles;
  it.first = p.base + (unsigned long long)ht * n;
  it.end = it.first + n;
  return it;
}

template <typename T, int D, bool LIST, int Q>
__global__ void __launch_bounds__(FqShape<D, Q>::kThreads, 1) fp4_attn_kernel(const __grid_constant__ Fp4AttnArgs a) {
  constexpr int kFqWarps = FqShape<D, Q>::kWarps, kFqThreads = FqShape<D, Q>::kThreads, kRows = FqShape<D, Q>::kRows;
  constexpr int kFqMinShare = 2 * kFqWarps;       // units of a CTA at least
  constexpr int KC = D / 64;                      // groups of a key row per lane
  constexpr int KS = D / 16;                      // k-steps of q . k
  constexpr int NT = D / 8;                       // features of the output per lane (NT r .. NT r + NT - 1)
  constexpr int MT = D / 16;                      // output tiles of 16 features: features NT r + 2 j and NT r + 2 j + 1
  constexpr int BB = fp4_block_bytes(D);
  constexpr int NB = 2;                           // blocks of a step
  constexpr bool kF32 = sizeof(T) == 4;
  extern __shared__ __align__(1024) unsigned char fq_raw[];
  FqSmem<D, Q>& sm = *reinterpret_cast<FqSmem<D, Q>*>(fq_raw + fq_ring_bytes<D, Q>());
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;
  const uint32_t ring = smem_u32(fq_raw) + warp * kFqStages * fq_stage_bytes(D);
  const QuantGeom& g = a.g;
  const int H = g.n_kv_heads;
  // output rows [rows][D] of segment `at`
  const auto seg_rows = [&](int at) -> float* {
    return at & 1 ? reinterpret_cast<float*>(fq_raw + (size_t)(at >> 1) * kFqStages * fq_stage_bytes(D)) : &sm.o_first[at >> 1][0][0];
  };

  if (lane == 0) {
    for (int i = 0; i < kFqStages; ++i) mbar_init(smem_u32(&sm.full[warp][i]), 1);
    mbar_fence_init();
  }
  if (lane < 2) sm.seg[2 * warp + lane].valid = 0;
  __syncwarp();
  after_the_one_before();
  let_the_next_one_come();                        // (the second kernel reads what this one does, and waits for its end)
  // ---- this CTA's and warp's share of the call's units
  FqPlan<LIST, kFqThreads, kRows> plan(a, sm.plan, gridDim.x, kFqMinShare, blockIdx.x == 0);
  const unsigned long long total = plan.total, share = plan.share;
  const unsigned long long cta0 = min(total, share * blockIdx.x), cta1 = min(total, cta0 + share);
  const unsigned long long wshare = quotient(cta1 - cta0 + kFqWarps - 1, kFqWarps);
  unsigned long long u = min(cta1, cta0 + wshare * warp);
  const unsigned long long u_end = min(cta1, u + wshare);
  const bool plain = !(a.softcap > 0.f) && a.slopes == nullptr;
  const float cap_in = a.softcap > 0.f ? 1.f / a.softcap : 0.f, cap_out = a.softcap * kLog2e;

  const float out_scale = a.out_scale;
  int fill = 0, take = 0;                         // the stages of this warp's ring that are filled and taken next,
  uint32_t phase = 0;                             // and the parity of the latter's barrier
  bool dead = false;                              // a copy did not arrive (reported); the warp gives up
  while (u < u_end && !dead) {
    plan.locate(u);
    const FqItem it = item_of(plan, u);
    const int slot = plan.info.x, len = plan.info.y, first_token = plan.info.z, n_new = plan.info.w, b = plan.b;
    const int h = it.h, tile = it.tile, at0 = (int)(u - it.first);
    const unsigned long long item = it.first, item_end = it.end;
    const unsigned long long seg_end = min(item_end, u_end);
    // blocks [blk0, blk0 + nb) of the item
    const int blk0 = max(0, at0 - kFqItemCost), nb = max(0, (int)(seg_end - item) - kFqItemCost) - blk0;
    if (nb == 0) {
      u = seg_end;
      continue;
    }

    // ---- copies
    const int32_t* pages = a.table + (long long)slot * g.max_pages;
    const int32_t* list = LIST ? a.t.pages + ((long long)first_token * H + h) * a.t.n_select : nullptr;
    // lane l keeps the place of block 32 n + l of the segment (block of the pool, and with lists its first token): of the 32 that are
    // being asked for, and looked up ahead of the next 32
    struct Place {
      int blk, tok;
    };
    const int in_page = g.page_shift - 4;          // log2 of a page's blocks
    const auto look_up = [&](int group) {
      Place p = {0, kFqNowhere};
      const int j = 32 * group + lane;
      if (j < nb) {
        int logical = (blk0 + j) >> in_page;
        if (LIST) {
          const int own = (len - 1) >> g.page_shift;
          const int e = list[logical];
          if (e > own) report_opt(a.status, ECHOKV_EBADPAGE);
          logical = e < 0 || e > own ? -1 : e;
        }
        if (logical >= 0) {
          int page = pages[logical];
          if (page < 0 || page >= g.n_pages) {
            report_opt(a.status, ECHOKV_EBADPAGE);
            page = 0;
          }
          const int inside = (blk0 + j) & ((1 << in_page) - 1);
          p.blk = ((page * H + h) << in_page) + inside;
          p.tok = (logical << g.page_shift) + inside * kQuantBlock;
        }
      }
      return p;
    };
    Place cur = look_up(0);
    // ---- the query rows: this lane loads a quarter of row r of every tile as operand; its scores are of rows 2 c and 2 c + 1
    const int n_rows = n_new * a.group, row0 = tile * kRows;
    // up to four rows stand in the even columns, so that a lane's second column is nobody's and costs nothing
    const bool spread = n_rows - row0 <= 4, two_tiles = Q == 2 && n_rows - row0 > kFqTile;
    uint32_t qh[Q][KS][2], ql[kF32 ? KS : 1][2];
    float c_row[Q][2];
    Quad<T> qv[Q][KS];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int qrow_r = row0 + q * kFqTile + (spread ? r >> 1 : r);
      const bool ok = qrow_r < n_rows && !(spread && (r & 1));
      const T* qp = static_cast<const T*>(a.q) + (long long)(first_token + (ok ? qrow_r >> a.group_shift : 0)) * a.q_stride +
                    (long long)(h * a.group + (qrow_r & (a.group - 1))) * D;
#pragma unroll
      for (int x = 0; x < KS; x += Quad<T>::kPerLoad)
        if (ok) Quad<T>::load16(qp + KC * 16 * c + 4 * x, &qv[q][x]);
        else Quad<T>::zero16(&qv[q][x]);
    }
    Place next = {0, kFqNowhere};
    const int n_steps = (nb + NB - 1) / NB;
    int left = 0;                                  // stages asked for and not yet taken
    int asked = 0;                                 // steps whose copies are under way or done
    const auto issue = [&]() {
      if ((asked & 15) == 0 && asked > 0) {
        cur = next;
        next = look_up((asked >> 4) + 1);
      }
      const int j = asked * NB;
      const int b0 = __shfl_sync(0xffffffffu, cur.blk, j & 31), b1 = __shfl_sync(0xffffffffu, cur.blk, (j + 1) & 31);
      int2 tok;
      if (LIST) {
        tok.x = __shfl_sync(0xffffffffu, cur.tok, j & 31);
        tok.y = __shfl_sync(0xffffffffu, cur.tok, (j + 1) & 31);
      }
      if (lane == 0) {
        const uint32_t bar = smem_u32(&sm.full[warp][fill]), dst = ring + fill * fq_stage_bytes(D);
        if (LIST) sm.tok[warp][fill] = tok;
        mbar_arrive_expect_tx(bar, j + 1 < nb ? 2 * BB : BB);
        bulk_load(dst, g.blocks + (long long)b0 * BB, BB, bar);
        if (j + 1 < nb) bulk_load(dst + BB, g.blocks + (long long)b1 * BB, BB, bar);
      }
      ++asked;
      ++left;
      fill = fill == kFqStages - 1 ? 0 : fill + 1;
    };
    while (asked < min(kFqStages, n_steps)) issue();
    next = look_up(1);                             // (not needed before the sixteenth step)

#pragma unroll
    for (int q = 0; q < Q; ++q) {
      // (magnitudes compare as integers, an infinity or NaN above everything finite)
      uint32_t bits = 0;
#pragma unroll
      for (int x = 0; x < KS; ++x) bits = qv[q][x].top(bits);
      bits = Quad<T>::top_bits(bits);
      bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 1));
      bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, 2));
      float back;
      const float up = query_scale(__uint_as_float(bits), a.softcap > 0.f, &back);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        c_row[q][e] = __shfl_sync(0xffffffffu, back, 4 * (2 * c + e)) * a.scale * (a.softcap > 0.f ? 1.f : kLog2e);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const HalfPair p = split_pair<kF32>(qv[q][ks].get(2 * f) * up, qv[q][ks].get(2 * f + 1) * up);
          qh[q][ks][f] = p.hi;
          if (kF32) ql[ks][f] = bits < 0x7f800000u ? p.lo : 0u;      // (an infinity less itself)
        }
    }
    const int prefix = !LIST && a.prefix ? min(a.prefix[b], len) : 0;          // (a prefix that comes in pieces is longer than what is there)
    int pos[Q][2], row_of[Q][2];                  // (row_of: -1 where the column is nobody's)
    float slope2[Q][2];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        row_of[q][e] = spread ? (q == 0 && e == 0 ? c : -1) : q * kFqTile + 2 * c + e;
        const int qrow = row0 + max(row_of[q][e], 0);
        pos[q][e] = len - n_new + (qrow < n_rows ? qrow >> a.group_shift : 0);
        slope2[q][e] = a.slopes ? a.slopes[h * a.group + (qrow & (a.group - 1))] * kLog2e : 0.f;
      }

    float o[Q][MT][4];                            // rows: feature NT r + 2 j (0, 1) and + 1 (2, 3); columns: query rows 2 c, 2 c + 1
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int f = 0; f < 4; ++f) o[q][j][f] = 0.f;
    // Per query row: the reference of its maximum (0 until it has seen a key, which the first one seen moves), and how far
    // above the reference a score may be before that moves.
    float m_ref[Q][2], grow[Q][2], l_run[Q][2];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m_ref[q][e] = l_run[q][e] = 0.f;
        grow[q][e] = -3.0e38f;
      }
    const int pos_first = len - n_new + (row0 >> a.group_shift);               // the item's first query: blocks up to it are seen whole

    // a scaled product q . k of token tok and a query row -> the score in base-2 units
    const auto score = [&](float y, int at, float slope, int tok) {
      if (a.softcap > 0.f) y = cap_out * tanh_f32(y * cap_in);
      if (a.slopes) y -= slope * fabsf((float)(at - tok));
      return y;
    };

    // One step: two blocks of the stage that has arrived.  MASKED: some of their tokens may be unseen, or the second block is not there.
    const auto attend = [&](auto masked_tag, auto spread_tag, auto tiles_tag, int step, uint32_t src) {
      constexpr bool MASKED = decltype(masked_tag)::value;
      constexpr int E = decltype(spread_tag)::value ? 1 : 2;      // columns of a lane that are anybody's
      constexpr int L = decltype(tiles_tag)::value;               // tiles that have a row
      int tok0[NB];
      if (LIST) {
        const int2 t = sm.tok[warp][take];
        tok0[0] = t.x;
        tok0[1] = t.y;
      } else {
        tok0[0] = (blk0 + step * NB) * kQuantBlock;
        tok0[1] = tok0[0] + kQuantBlock;
      }
      const bool two = !MASKED || step * NB + 1 < nb;
      if (!two) tok0[1] = kFqNowhere;              // (the first block stands in for it)
      const auto seen = [&](int tok, int at) { return tok <= at || (!LIST && tok < prefix); };
      const uint32_t part[NB] = {src, two ? src + BB : src};

      // ---- the values' codes and scales (used last: on their way while the scores are worked out)
      uint32_t vt[NB][2][2][D / 64], vs[NB][2];    // [tokens 2 c, + 1 | 8 on][which of the two]
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t at = part[n] + 8 * D + t * 4 * D + lane * 8 * KC;
          if constexpr (D == 128) {
            const uint4 v = lds16(at);
            vt[n][t][0][0] = v.x; vt[n][t][0][D / 64 - 1] = v.y; vt[n][t][1][0] = v.z; vt[n][t][1][D / 64 - 1] = v.w;
          } else {
            const uint2 v = lds8(at);
            vt[n][t][0][0] = v.x; vt[n][t][1][0] = v.y;
          }
          uint16_t w;
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(part[n] + 17 * D + (r * NT / 16) * 16 + 8 * t + 2 * c) : "memory");
          vs[n][t] = e4m3_scales(w);
        }

      // ---- scores
      float sc[L][NB][4];                         // [tile][n][2 t + e]: token r + 8 t of block n, query row 2 c + e
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        uint32_t kw[2][2 * KC], ks[2][KC];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t at = part[n] + t * 4 * D + lane * 8 * KC;
          if constexpr (D == 128) {
            const uint4 v = lds16(at);
            kw[t][0] = v.x; kw[t][1] = v.y; kw[t][2 * KC - 2] = v.z; kw[t][2 * KC - 1] = v.w;
            uint16_t w;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(part[n] + 16 * D + (r + 8 * t) * 8 + 2 * c) : "memory");
            const uint32_t s = e4m3_scales(w);
            ks[t][0] = __byte_perm(s, 0u, 0x1010);
            ks[t][KC - 1] = __byte_perm(s, 0u, 0x3232);
          } else {
            const uint2 v = lds8(at);
            kw[t][0] = v.x; kw[t][1] = v.y;
            uint16_t w;
            asm volatile("{\n\t.reg .u8 b;\n\tld.shared.u8 b, [%1];\n\tcvt.u16.u8 %0, b;\n\t}" : "=h"(w) : "r"(part[n] + 16 * D + (r + 8 * t) * 4 + c) : "memory");
            const uint32_t s = e4m3_scales(w);
            ks[t][0] = __byte_perm(s, 0u, 0x1010);
          }
        }
        // two chains of products.  (fp32: the tensor core cuts its sums off where it adds to them, 2^-23 of the sum each time and always
        // towards 0, so a word's products are summed by themselves and the low-order halves' apart.)
        float sb[L][4];
#pragma unroll
        for (int q = 0; q < L; ++q)
#pragma unroll
          for (int f = 0; f < 4; ++f) sb[q][f] = sc[q][n][f] = 0.f;
#pragma unroll
        for (int w = 0; w < 2 * KC; ++w) {
          uint32_t x[2][4];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            e2m1_bytes(kw[t][w], x[t]);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[t][i] = fp4_mul(x[t][i], ks[t][w / 2]);
          }
          if constexpr (kF32) {
            float hi[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              mma_m16n8k16_f16(hi, x[0][2 * s], x[1][2 * s], x[0][2 * s + 1], x[1][2 * s + 1], qh[0][2 * w + s][0], qh[0][2 * w + s][1]);
              mma_m16n8k16_f16(sb[0], x[0][2 * s], x[1][2 * s], x[0][2 * s + 1], x[1][2 * s + 1], ql[2 * w + s][0], ql[2 * w + s][1]);
            }
#pragma unroll
            for (int f = 0; f < 4; ++f) sc[0][n][f] += hi[f];
          } else {
#pragma unroll
            for (int q = 0; q < L; ++q) {
              mma_m16n8k16_f16(sc[q][n], x[0][0], x[1][0], x[0][1], x[1][1], qh[q][2 * w][0], qh[q][2 * w][1]);
              mma_m16n8k16_f16(sb[q], x[0][2], x[1][2], x[0][3], x[1][3], qh[q][2 * w + 1][0], qh[q][2 * w + 1][1]);
            }
          }
        }
#pragma unroll
        for (int q = 0; q < L; ++q)
#pragma unroll
          for (int f = 0; f < 4; ++f) sc[q][n][f] += sb[q][f];
      }

      // ---- probabilities as operands (ph[tile][n][t]: query row r, tokens 8 t + 2 c, + 1), the references moved if needed
      float most[L][2];
      bool above = false;
#pragma unroll
      for (int q = 0; q < L; ++q) {
        most[q][0] = most[q][1] = -INFINITY;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          if (plain) {
#pragma unroll
            for (int i = 0; i < 4; i += 3 - E) sc[q][n][i] = fmaf(sc[q][n][i], c_row[q][i & 1], -m_ref[q][i & 1]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; i += 3 - E)
              sc[q][n][i] = score(sc[q][n][i] * c_row[q][i & 1], pos[q][i & 1], slope2[q][i & 1], tok0[n] + 8 * (i >> 1) + r) - m_ref[q][i & 1];
          }
          if (MASKED) {
#pragma unroll
            for (int i = 0; i < 4; i += 3 - E)
              if (!seen(tok0[n] + 8 * (i >> 1) + r, pos[q][i & 1])) sc[q][n][i] = -INFINITY;
          }
#pragma unroll
          for (int e = 0; e < E; ++e) most[q][e] = fmaxf(most[q][e], fmaxf(sc[q][n][e], sc[q][n][2 + e]));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) above |= most[q][e] > grow[q][e];
      }
      if (__any_sync(0xffffffffu, above)) {
#pragma unroll
        for (int q = 0; q < L; ++q) {
          float alpha[2] = {1.f, 1.f};
#pragma unroll
          for (int e = 0; e < E; ++e) {
            float mx = most[q][e];
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
            mx -= kFqBelow;
            const bool first = grow[q][e] != kFqGrow;    // nothing seen so far: sum and output are still 0
            if (mx > (first ? -INFINITY : 0.f)) {
              if (!first) alpha[e] = exp2_approx(-mx);
              grow[q][e] = kFqGrow;
              m_ref[q][e] += mx;
              l_run[q][e] *= alpha[e];
#pragma unroll
              for (int n = 0; n < NB; ++n) {
                sc[q][n][e] -= mx;
                sc[q][n][2 + e] -= mx;
              }
            }
          }
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int f = 0; f < 4; f += 3 - E) o[q][m][f] *= alpha[f & 1];
        }
      }
      uint32_t ph[L][NB][2], pl[NB][2];
#pragma unroll
      for (int q = 0; q < L; ++q)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          float p[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 4; i += 3 - E) {
            p[i] = exp2_approx(sc[q][n][i]);
            l_run[q][i & 1] += p[i];
          }
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const HalfPair w = split_pair<kF32>(p[2 * t], p[2 * t + 1], kFqLowUp);
            ph[q][n][t] = movm(w.hi);
            if (kF32) pl[n][t] = movm(w.lo);
          }
        }

      // ---- output
      // (behind the sequence's end there may be anything: a NaN times a probability of 0)
      if (MASKED) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int tok = tok0[n] + 8 * t + 2 * c;
            if (tok >= len) vs[n][t] = 0u;
            else if (tok + 1 >= len) vs[n][t] &= 0xffffu;
          }
      }
      // word w of block n's codes -> operands: features 2 i and 2 i + 1, a byte for both tokens
      const auto values = [&](int n, int w, uint32_t (&x)[2][4], uint32_t (&y)[2][4]) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          e2m1_bytes(fp4_zip(vt[n][t][0][w], vt[n][t][1][w] << 4), x[t]);
          e2m1_bytes(fp4_zip(vt[n][t][0][w] >> 4, vt[n][t][1][w]), y[t]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            x[t][i] = fp4_mul(x[t][i], vs[n][t]);
            y[t][i] = fp4_mul(y[t][i], vs[n][t]);
          }
        }
      };
      if constexpr (kF32) {
        // (a step's products are summed by themselves, as above, those with the probabilities' low-order halves around their own power)
#pragma unroll
        for (int w = 0; w < D / 64; ++w) {
          uint32_t x[NB][2][4], y[NB][2][4];
#pragma unroll
          for (int n = 0; n < NB; ++n) values(n, w, x[n], y[n]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float hi[4] = {0.f, 0.f, 0.f, 0.f}, lo[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int n = 0; n < NB; ++n) {
              mma_m16n8k16_f16(hi, x[n][0][i], y[n][0][i], x[n][1][i], y[n][1][i], ph[0][n][0], ph[0][n][1]);
              mma_m16n8k16_f16(lo, x[n][0][i], y[n][0][i], x[n][1][i], y[n][1][i], pl[n][0], pl[n][1]);
            }
#pragma unroll
            for (int f = 0; f < 4; ++f) o[0][4 * w + i][f] += fmaf(lo[f], 1.f / kFqLowUp, hi[f]);
          }
        }
      } else {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int w = 0; w < D / 64; ++w) {
            uint32_t x[2][4], y[2][4];
            values(n, w, x, y);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int q = 0; q < L; ++q) mma_m16n8k16_f16(o[q][4 * w + i], x[0][i], y[0][i], x[1][i], y[1][i], ph[q][n][0], ph[q][n][1]);
          }
      }
    };
#pragma unroll 1
    for (int step = 0; step < n_steps; ++step) {
      if (!__all_sync(0xffffffffu, warp_wait(smem_u32(&sm.full[warp][take]), phase))) {
        dead = true;
        break;
      }
      bool masked;
      if (LIST) {
        const int2 t = sm.tok[warp][take];
        masked = max(t.x, t.y) + kQuantBlock - 1 > pos_first || step * NB + 1 >= nb;
      } else {
        masked = (blk0 + (step + 1) * NB) * kQuantBlock - 1 > pos_first || step * NB + 1 >= nb;
      }
      const uint32_t src = ring + take * fq_stage_bytes(D);
      const std::integral_constant<int, 1> one;
      if (spread) {
        if (masked) attend(std::true_type(), std::true_type(), one, step, src); else attend(std::false_type(), std::true_type(), one, step, src);
      } else if (!two_tiles) {
        if (masked) attend(std::true_type(), std::false_type(), one, step, src); else attend(std::false_type(), std::false_type(), one, step, src);
      } else if constexpr (Q == 2) {
        const std::integral_constant<int, 2> two;
        if (masked) attend(std::true_type(), std::false_type(), two, step, src); else attend(std::false_type(), std::false_type(), two, step, src);
      }
      __syncwarp();                                // (all lanes have read the stage: it may be overwritten)
      if (++take == kFqStages) {
        take = 0;
        phase ^= 1;
      }
      --left;
      if (asked < n_steps) issue();
    }
    if (dead) {
      // let every copy that was asked for land, as far as it does, before the shared memory is given back
      if (lane == 0) {
        report_opt(a.status, ECHOKV_ETIMEOUT);
        for (; left > 0; --left) {
          mbar_drain(smem_u32(&sm.full[warp][take]), phase);
          if (++take == kFqStages) {
            take = 0;
            phase ^= 1;
          }
        }
      }
      break;
    }

    // ---- the segment's result
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) l_run[q][e] += __shfl_xor_sync(0xffffffffu, l_run[q][e], w);
    const bool starts = blk0 == 0, ends = seg_end == item_end;
    if (starts && ends) {
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int qrow = row0 + row_of[q][e];
          if (row_of[q][e] >= 0 && qrow < n_rows) {
            const float inv = l_run[q][e] == 0.f ? 0.f : out_scale / l_run[q][e];
            float v[NT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              v[2 * m] = o[q][m][e] * inv;
              v[2 * m + 1] = o[q][m][2 + e] * inv;
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
        for (int q = 0; q < Q; ++q)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (row_of[q][e] < 0) continue;
            sm.m[at][row_of[q][e]] = l_run[q][e] == 0.f ? -INFINITY : m_ref[q][e];
            sm.l[at][row_of[q][e]] = l_run[q][e];
          }
      }
      __syncwarp();                               // (the rows of the second kind lie over the ring)
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (row_of[q][e] < 0) continue;
#pragma unroll
          for (int m = 0; m < MT; ++m) *reinterpret_cast<float2*>(dst + row_of[q][e] * D + NT * r + 2 * m) = make_float2(o[q][m][e], o[q][m][2 + e]);
        }
    }
    u = seg_end;
  }

  // ---- segments of one item side by side in this CTA: combine them; what is still cut goes to the workspace.  A warp per query
  //      row; lane k looks at segment k.
  __syncthreads();
  const FqWork<kRows> ws(a.ws);
  constexpr int E = D / 32;
  static_assert(2 * kFqWarps <= 32, "a lane per segment");
  const bool is_seg = lane < 2 * kFqWarps && sm.seg[lane < 2 * kFqWarps ? lane : 0].valid;
  const unsigned long long my_item = is_seg ? sm.seg[lane].item : ~0ull;
#pragma unroll 1
  for (int row = warp; row < kRows; row += kFqWarps) {
    const float my_m = is_seg ? sm.m[lane][row] : -INFINITY, my_l = is_seg ? sm.l[lane][row] : 0.f;
    uint32_t todo = __ballot_sync(0xffffffffu, is_seg);
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
        const float* o = seg_rows(k) + row * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += wk * o[e];
      }
      if (starts && ends) {
        const int4 s = plan.info_of(first.b);
        const int qrow = first.tile * kRows + row;
        if (qrow < s.w * a.group) {
          const float inv = l == 0.f ? 0.f : out_scale / l;
          T* dst = static_cast<T*>(a.out) +
                   ((long long)(s.z + (qrow >> a.group_shift)) * a.n_q_heads + first.h * a.group + (qrow & (a.group - 1))) * D + lane * E;
#pragma unroll
          for (int e = 0; e < E; ++e) dst[e] = from_f32<T>(acc[e] * inv);
        }
      } else {
        const long long p = ((long long)blockIdx.x * 2 + (starts ? 1 : 0)) * kRows + row;
        if (lane == 0) ws.ml[p] = make_float2(m, l);
#pragma unroll
        for (int e = 0; e < E; ++e) ws.o[p * D + lane * E + e] = acc[e];
      }
    }
  }
}

// Joins the items that shares cut: block g the one whose first block of keys is in CTA g and that goes on in the next ones.  Also zeroes
// the rows of unusable sequences (tokens).  Launched while the first kernel runs, it works out what it has to join and waits for that
// one's end.
template <typename T, int D, bool LIST, int Q>
__global__ void __launch_bounds__(FqShape<D, Q>::kRows * 32) fp4_merge_kernel(const __grid_constant__ Fp4AttnArgs a) {
  constexpr int E = D / 32;
  constexpr int kRows = FqShape<D, Q>::kRows, kThreads = kRows * 32;       // a warp per query row
  __shared__ FqPlanShared<kThreads> shared;
  const int tid = threadIdx.x, lane = tid & 31, row = tid >> 5;
  const FqWork<kRows> ws(a.ws);
  FqPlan<LIST, kThreads, kRows> plan(a, shared, gridDim.x, 2 * FqShape<D, Q>::kWarps, false);
  const unsigned long long from = plan.share * blockIdx.x, behind = from + plan.share;      // the units of CTA g
  int n_parts = 0;
  FqItem it = {};
  if (behind < plan.total) {
    plan.locate(behind);
    it = item_of(plan, behind);
    const unsigned long long first_block = it.first + kFqItemCost;
    if (first_block < behind && first_block >= from) n_parts = (int)quotient(it.end - 1, plan.share) - (int)blockIdx.x + 1;
  }
  after_the_one_before();
#pragma unroll 1
  for (int b = blockIdx.x; b < plan.n_own; b += gridDim.x) {
    const QuantSeq s = owner<LIST>(a, b);
    if (s.error && s.n > 0) {
      T* dst = static_cast<T*>(a.out) + (long long)s.first * a.n_q_heads * D;
      const long long n = (long long)s.n * a.n_q_heads * D;
      for (long long i = tid; i < n; i += kThreads) dst[i] = from_f32<T>(0.f);
    }
  }
  const float out_scale = a.out_scale;
  if (n_parts == 0) return;
  const auto part = [&](int p) -> long long { return ((long long)(blockIdx.x + p) * 2 + (p == 0 ? 1 : 0)) * kRows + row; };
  const int4 s = plan.info;
  float m = -INFINITY;
  for (int p = lane; p < n_parts; p += 32) m = fmaxf(m, ws.ml[part(p)].x);
  m = warp_max(m);
  float l = 0.f, acc[E] = {};
#pragma unroll 4
  for (int p = 0; p < n_parts; ++p) {
    const float2 ml = ws.ml[part(p)];
    const float w = ml.y == 0.f ? 0.f : exp2_approx(ml.x - m);
    l += w * ml.y;
    const float* o = ws.o + part(p) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] += w * o[e];
  }
  const int qrow = it.tile * kRows + row;
  if (qrow >= s.w * a.group) return;
  const float inv = l == 0.f ? 0.f : out_scale / l;
  T* dst = static_cast<T*>(a.out) +
           ((long long)(s.z + (qrow >> a.group_shift)) * a.n_q_heads + it.h * a.group + (qrow & (a.group - 1))) * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = from_f32<T>(acc[e] * inv);
}

template <typename T, int D, bool LIST, int Q>
cudaError_t launch(const Fp4AttnArgs& a, int sm_count, cudaStream_t stream) {
  constexpr size_t smem = fq_ring_bytes<D, Q>() + sizeof(FqSmem<D, Q>);
  static_assert(kFqStages * fq_stage_bytes(D) >= FqShape<D, Q>::kRows * D * 4, "a segment's rows fit over a warp's ring");
  static_assert(smem <= 227 * 1024, "shared memory of one CTA");
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_smem(fp4_attn_kernel<T, D, LIST, Q>, smem, &done);
  if (e != cudaSuccess) return e;
  const int grid = sm_count < kFqMaxCtas ? sm_count : kFqMaxCtas;
  if ((e = launch_early(fp4_attn_kernel<T, D, LIST, Q>, dim3(grid), FqShape<D, Q>::kThreads, smem, stream, a)) != cudaSuccess) return e;
  return launch_early(fp4_merge_kernel<T, D, LIST, Q>, dim3(grid), FqShape<D, Q>::kRows * 32, 0, stream, a);
}

template <typename T, int D>
cudaError_t launch_l(const Fp4AttnArgs& a, int sm_count, cudaStream_t stream) {
  if (a.t.seqs) return launch<T, D, true, 1>(a, sm_count, stream);
  // sequences may have more rows than a tile: items of two
  if constexpr (sizeof(T) == 2) {
    if (a.max_new > kFqTile >> a.group_shift) return launch<T, D, false, 2>(a, sm_count, stream);
  }
  return launch<T, D, false, 1>(a, sm_count, stream);
}

}  // namespace

uint64_t fp4_attn_workspace_bytes(int head_dim) {
  const uint64_t n = (uint64_t)kFqMaxCtas * 2 * 2 * kFqTile * (sizeof(float2) + (uint64_t)head_dim * sizeof(float));
  return (n + 255) / 256 * 256;
}

cudaError_t launch_fp4_attn(const Fp4AttnArgs& a, int sm_count, cudaStream_t stream) {
  if (a.dtype == ECHOKV_BF16) return a.g.head_dim == 128 ? launch_l<__nv_bfloat16, 128>(a, sm_count, stream) : launch_l<__nv_bfloat16, 64>(a, sm_count, stream);
  return a.g.head_dim == 128 ? launch_l<float, 128>(a, sm_count, stream) : launch_l<float, 64>(a, sm_count, stream);
}

}  // namespace echokv

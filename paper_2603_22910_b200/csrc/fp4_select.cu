// The pages that a query reads: those whose keys' bounds allow the largest scores.
//
//   score(q, page) = s_q s_page sum_c (code_c > 0 ? code_c top_c : code_c low_c),   the largest over the query heads of a KV head
//
// The sum is one product of whole numbers, [q+ | q-] . [top | low], of 2 d terms: mma.sync m16n8k32 on 8-bit integers with the
// pages on the M rows and the query rows on N, exact in 32 bits, so that equal pages are equal and the choice does not depend on
// the order of anything.  A block takes one KV head of one token, or of up to 8 neighbours of one sequence where there are tokens enough
// for all SMs (a page's bounds are then read once for them).  A warp takes 16 pages at a time, whose bounds its lanes have asked for
// two steps before, each the pieces that it will use itself, and writes their scores, as whole numbers in the order of the
// floats, in the pages' order to shared memory.  The n_select largest are then found by counting eight bits at a time from the
// top of what the keys differ in, and copied in order: what comes out is ascending, and of equal scores the first pages stay.
// When the buffer is full it is cut down to n_select in the same way, so that a sequence may have any number of pages.  Few tokens over
// long caches are split along the pages; a second kernel then chooses among what the parts chose.
// The bound is reading the bounds, 2 d + 4 bytes a page and head.  Measured (8 heads of 128): 64 of 1024 pages for 16 tokens 15.5
// us, about 5 each for start, reading with scores, and the choice; one token among 62500 pages, in 18 parts, 55 us; 64 decode tokens
// among 1875 pages each 71 us, 3.5 TB/s; 256 tokens of 4 requests among 3750 pages 194 us, 4096 of 4 prompts among 1250 pages 987.
#include "fp4_common.cuh"

namespace echokv {

namespace {

constexpr int kFsMaxWarps = 16;                    // of a block: 16, or 8 where two blocks share an SM or there is no room for more
constexpr int kFsDepth = 2;                        // steps under way
__host__ __device__ constexpr int fs_step(int warps) { return warps * 16; }        // pages that a block takes at once
constexpr int kFsEntries = 16384;                  // keys of a block, of all its tokens
constexpr int kFsMaxTokens = 8;                    // tokens of a block: each has room for 2048 keys, ECHOKV_FOURBIT_MAX_SELECT and a step
constexpr int kFsMaxParts = 320;                   // (token, head, part of the pages) with a place in the workspace
constexpr int kFsMinPages = 512;                   // pages of a part at least
constexpr size_t kFsRoom = 227 * 1024;             // shared memory of a CTA
constexpr uint32_t kFsAlways = 0xffffffffu;        // key of a page that is taken in any case (0: of one behind the token's own)

struct FsPart {
  uint32_t* keys;                                  // [kFsMaxParts][ECHOKV_FOURBIT_MAX_SELECT]
  uint32_t* pages;
  int* counts;                                     // [kFsMaxParts]
  __host__ __device__ explicit FsPart(unsigned char* ws) {
    keys = reinterpret_cast<uint32_t*>(ws);
    pages = keys + kFsMaxParts * ECHOKV_FOURBIT_MAX_SELECT;
    counts = reinterpret_cast<int*>(pages + kFsMaxParts * ECHOKV_FOURBIT_MAX_SELECT);
  }
};

// of the warps that choose for one token
struct FsGroup {
  uint32_t hist[256];
  uint32_t red[kFsMaxWarps][4], side[kFsMaxWarps][2];
  uint32_t bin, want, whole;
};

__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// floats in their order, as whole numbers above 0
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);     // (-0 is 0)
  return b >> 31 ? ~b : b | 0x80000000u;
}

// Which of n keys are the k largest (of equal ones the first; all that are not 0 if there are no more).  For a group of `warps` warps (warp:
// this one's number among them, bar: their barrier), after a barrier of theirs.
struct FsChoice {
  uint32_t lo, bin, want;                          // keys whose (key - lo) << up >> shift is above bin, and the first `want` of those that are bin
  int up, shift;
  bool all, none;
  // +1: taken in any case, 0: one of the last bin, -1: not taken
  __device__ __forceinline__ int side(uint32_t x) const {
    if (x == 0) return -1;
    if (x == kFsAlways || all) return 1;
    if (none) return -1;
    const uint32_t p = (x - lo) << up >> shift;
    return p > bin ? 1 : p == bin ? 0 : -1;
  }
};
__device__ __forceinline__ void group_sync(int bar, int warps) { asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(32 * warps) : "memory"); }

__device__ __noinline__ FsChoice choose(const uint32_t* key, int n, int k, FsGroup& sm, int warp, int warps, int bar) {
  const int lane = threadIdx.x & 31, tid = warp * 32 + lane, threads = 32 * warps;
  // what lies between 0 and always: how much, from where to where
  uint32_t always = 0, some = 0, lo = 0xffffffffu, hi = 0;
#pragma unroll 4
  for (int i = tid; i < n; i += threads) {
    const uint32_t x = key[i];
    const bool normal = x != 0 && x != kFsAlways;
    always += x == kFsAlways;
    some += normal;
    lo = min(lo, normal ? x : 0xffffffffu);
    hi = max(hi, normal ? x : 0u);
  }
  always = __reduce_add_sync(0xffffffffu, always);
  some = __reduce_add_sync(0xffffffffu, some);
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) {
    sm.red[warp][0] = always;
    sm.red[warp][1] = some;
    sm.red[warp][2] = lo;
    sm.red[warp][3] = hi;
  }
  for (int i = tid; i < 256; i += threads) sm.hist[i] = 0;
  group_sync(bar, warps);
  always = some = hi = 0;
  lo = 0xffffffffu;
  for (int w = 0; w < warps; ++w) {
    always += sm.red[w][0];
    some += sm.red[w][1];
    lo = min(lo, sm.red[w][2]);
    hi = max(hi, sm.red[w][3]);
  }
  FsChoice f;
  f.lo = lo;
  f.up = hi > lo ? __clz(hi - lo) : 0;             // the normal keys' place between lo and hi, from bit 31 down
  f.want = (uint32_t)k - min((uint32_t)k, always);
  f.bin = 0;
  f.shift = 32;
  f.all = some <= f.want;
  f.none = !f.all && f.want == 0;
  while (!f.all && !f.none && f.shift > 0) {
    f.shift -= 8;
#pragma unroll 4
    for (int i = tid; i < n; i += threads) {
      const uint32_t x = key[i];
      if (x == 0 || x == kFsAlways) continue;
      const uint32_t p = (x - lo) << f.up;
      if (f.shift == 24 || p >> (f.shift + 8) == f.bin) atomicAdd(&sm.hist[p >> f.shift & 255], 1u);
    }
    group_sync(bar, warps);
    if (warp == 0) {
      // eight bins to a lane, from the top
      uint32_t c[8], sum = 0;
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        c[b] = sm.hist[255 - 8 * lane - b];
        sm.hist[255 - 8 * lane - b] = 0;
        sum += c[b];
      }
      uint32_t before = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += y;
      }
      before -= sum;
      if (before < f.want && f.want <= before + sum) {
#pragma unroll
        for (int b = 0; b < 8; ++b) {
          if (before < f.want && f.want <= before + c[b]) {
            sm.bin = f.bin << 8 | (uint32_t)(255 - 8 * lane - b);
            sm.want = f.want - before;
            sm.whole = f.want - before == c[b];
          }
          before += c[b];
        }
      }
    }
    group_sync(bar, warps);
    f.bin = sm.bin;
    f.want = sm.want;
    if (sm.whole) break;                           // (the bin is taken as a whole: nothing below it matters)
  }
  return f;
}

// The chosen ones of n keys in their order: take(place, index) for each, by all warps of a group.  Returns how many (k at most).
template <typename F>
__device__ __forceinline__ int chosen(const FsChoice& f, const uint32_t* key, int n, int k, FsGroup& sm, int warp, int warps, int bar, const F& take) {
  const int lane = threadIdx.x & 31;
  // every warp has a run of the keys
  const int run = ((n + warps - 1) / warps + 31) & ~31, from = min(n, warp * run), until = min(n, from + run);
  uint32_t above = 0, equal = 0;
  for (int i = from + lane; i < until; i += 32) {
    const int s = f.side(key[i]);
    above += s > 0;
    equal += s == 0;
  }
  above = __reduce_add_sync(0xffffffffu, above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) {
    sm.side[warp][0] = above;
    sm.side[warp][1] = equal;
  }
  group_sync(bar, warps);
  uint32_t before_above = 0, before_equal = 0, all_above = 0, all_equal = 0;
  for (int w = 0; w < warps; ++w) {
    if (w < warp) {
      before_above += sm.side[w][0];
      before_equal += sm.side[w][1];
    }
    all_above += sm.side[w][0];
    all_equal += sm.side[w][1];
  }
  const uint32_t lower = (1u << lane) - 1;
#pragma unroll 1
  for (int i0 = from; i0 < until; i0 += 32) {
    const int i = i0 + lane, s = f.side(i < until ? key[i] : 0u);
    const uint32_t b_above = __ballot_sync(0xffffffffu, s > 0), b_equal = __ballot_sync(0xffffffffu, s == 0);
    const uint32_t rank_equal = before_equal + __popc(b_equal & lower), rank_above = before_above + __popc(b_above & lower);
    const uint32_t at = rank_above + min(rank_equal, f.want);
    if ((s > 0 || (s == 0 && rank_equal < f.want)) && at < (uint32_t)k) take((int)at, i);      // (k at most, whatever the keys)
    before_above += __popc(b_above);
    before_equal += __popc(b_equal);
  }
  return (int)min((uint32_t)k, all_above + min(all_equal, f.want));
}
// The pages of a buffer's keys: those of the first `kept` ones are listed, the others follow one another.
struct FsPages {
  uint32_t* list;
  int kept;
  uint32_t start;
  __device__ __forceinline__ uint32_t operator()(int i) const { return i < kept ? list[i] : start + (uint32_t)(i - kept); }
};
// The buffer cut down to the k chosen ones, listed, by the group's first warp alone (what it writes lies before what it still
// reads); where there are fewer, keys of 0 behind them.
__device__ __forceinline__ void cut_down(uint32_t* key, const FsPages& page, int n, int k, FsGroup& sm, int warp, int warps, int bar) {
  const FsChoice f = choose(key, n, k, sm, warp, warps, bar);
  if (warp == 0) {
    const int lane = threadIdx.x & 31;
    const uint32_t lower = (1u << lane) - 1;
    uint32_t above = 0, equal = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += 32) {
      const uint32_t x = i0 + lane < n ? key[i0 + lane] : 0u, y = i0 + lane < n ? page(i0 + lane) : 0u;
      const int s = f.side(x);
      const uint32_t b_above = __ballot_sync(0xffffffffu, s > 0), b_equal = __ballot_sync(0xffffffffu, s == 0);
      const uint32_t rank_equal = equal + __popc(b_equal & lower);
      const uint32_t at = above + __popc(b_above & lower) + min(rank_equal, f.want);
      __syncwarp();
      if ((s > 0 || (s == 0 && rank_equal < f.want)) && at < (uint32_t)k) {
        key[at] = x;
        page.list[at] = y;
      }
      above += __popc(b_above);
      equal += __popc(b_equal);
      __syncwarp();
    }
    for (uint32_t i = above + min(equal, f.want) + lane; i < (uint32_t)k; i += 32) key[i] = 0u;
  }
  group_sync(bar, warps);
}

// One token: its sequence's row of the block table and its own page (-1 with an error).
constexpr int kFsNotAsked = -1000;                 // (no error that is reported)
struct FsToken {
  int slot, own, error;
};
__device__ __forceinline__ FsToken token_of(const Fp4SelectArgs& a, int i) {
  const int seq = a.t.seqs[i], pos = a.t.positions[i];
  FsToken t = {0, -1, 0};
  if (seq < 0) t.error = kFsNotAsked;
  else if (seq >= a.B) t.error = ECHOKV_EBADPAGE;
  else {
    t.slot = a.slots ? a.slots[seq] : seq;
    if (t.slot < 0 || t.slot >= a.g.max_batch) t.error = ECHOKV_EBADPAGE;
    else if (pos < 0 || pos >= a.g.max_pages * a.g.page_tokens) t.error = ECHOKV_EBADLENGTH;
    else t.own = pos >> a.g.page_shift;
  }
  return t;
}
// all pages up to the own one and -1 behind them (none: own = -1)
__device__ __forceinline__ void write_all(const Fp4SelectArgs& a, int token, int h, int own, int tid, int threads) {
  int32_t* out = a.out + ((long long)token * a.g.n_kv_heads + h) * a.t.n_select;
  for (int j = tid; j < a.t.n_select; j += threads) out[j] = j <= own ? j : -1;
}

// bytes of a step's bounds for one warp: 16 pages, a lane's pieces [piece][lane] and scales [2][lane]
__host__ __device__ constexpr int fs_stage_bytes(int d) { return 16 * 2 * d + 2 * 32 * 4; }

template <typename T, int D, int kFsWarps>
__global__ void __launch_bounds__(kFsWarps * 32, kFsWarps == 8 ? 2 : 1) fp4_select_kernel(const __grid_constant__ Fp4SelectArgs a, int tile_tokens, int capacity) {
  constexpr int kFsThreads = kFsWarps * 32, kFsStep = fs_step(kFsWarps);
  constexpr int W = D / 64;                        // 16-byte pieces of a lane: features 64 i + 16 c and on
  extern __shared__ __align__(16) unsigned char fs_raw[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;
  const Fp4Geom& g = a.g;
  const int H = g.n_kv_heads, K = a.t.n_select;
  const int h = blockIdx.x % H, i0 = (int)(blockIdx.x / H);
  const int part = blockIdx.y, parts = gridDim.y;
  const uint32_t ring = smem_u32(fs_raw) + warp * kFsDepth * fs_stage_bytes(D);
  // [warps][depth] stages | [rows][2] query codes, q+ and q- | [rows] their scales | [tokens] groups | [tokens][capacity] keys | [tokens][K] lists
  const int rows8 = (tile_tokens * a.group + 7) & ~7;
  uint32_t (*q_code)[2][D / 4] = reinterpret_cast<uint32_t (*)[2][D / 4]>(fs_raw + kFsWarps * kFsDepth * fs_stage_bytes(D));
  float* q_scale = reinterpret_cast<float*>(q_code + rows8);
  FsGroup* sm = reinterpret_cast<FsGroup*>(q_scale + rows8);
  uint32_t* key_of = reinterpret_cast<uint32_t*>(sm + tile_tokens);
  uint32_t* list_of = key_of + tile_tokens * capacity;

  after_the_one_before();
  // the block's tokens: i0 and those behind it at the following positions of its sequence, up to the next multiple of
  // tile_tokens; a token that belongs to one before it has nothing to do
  const FsToken first = token_of(a, i0);
  const int pos0 = a.t.positions[i0];
  int n_tok = 1;
  {
    const int seq = a.t.seqs[i0];
    const auto follows = [&](int i) { return a.t.seqs[i] == seq && a.t.positions[i] - pos0 == i - i0; };
    if (first.error == 0) {
      if (i0 > 0 && pos0 % tile_tokens != 0 && follows(i0 - 1)) return;
      while (n_tok < tile_tokens && i0 + n_tok < a.n_tokens && (pos0 + n_tok) % tile_tokens != 0 && token_of(a, i0 + n_tok).error == 0 && follows(i0 + n_tok))
        ++n_tok;
    }
  }
  if (first.error != 0 && first.error != kFsNotAsked && tid == 0 && part == 0 && h == 0) report_opt(a.status, first.error);
  const int most = first.error == 0 ? (pos0 + n_tok - 1) >> g.page_shift : -1;      // the last page that one of them sees
  if (most < K) {
    if (parts == 1)
      for (int k = 0; k < n_tok; ++k) write_all(a, i0 + k, h, most < 0 ? -1 : (pos0 + k) >> g.page_shift, tid, kFsThreads);
    else if (tid == 0) FsPart(a.ws).counts[blockIdx.x * parts + part] = 0;
    return;
  }
  const int share = ((most + parts) / parts + kFsStep - 1) / kFsStep * kFsStep;
  const int p0 = min(most + 1, part * share), p1 = min(most + 1, p0 + share), n_steps = (p1 - p0 + kFsStep - 1) / kFsStep;
  const int32_t* table = a.table + (long long)first.slot * g.max_pages;
  // this lane's pages of a step (rows r and r + 8 of the warp's 16)
  struct Ids {
    int id[2];
  };
  const auto look_up = [&](int step) {
    Ids x;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int page = p0 + step * kFsStep + warp * 16 + r + 8 * t;
      x.id[t] = page < p1 ? table[page] : 0;
      if (x.id[t] < 0 || x.id[t] >= g.n_pages) {
        report_opt(a.status, ECHOKV_EBADPAGE);
        x.id[t] = 0;
      }
    }
    return x;
  };
  const auto ask = [&](int step, const Ids& x) {
    if (step < n_steps) {
      const uint32_t dst = ring + step % kFsDepth * fs_stage_bytes(D);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const long long line = (long long)x.id[t] * H + h;
        const int8_t* p = g.bounds + line * 2 * D + 16 * c;
#pragma unroll
        for (int i = 0; i < 2 * W; ++i)            // (the largest values' pieces, then the smallest ones')
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + ((t * 2 * W + i) * 32 + lane) * 16), "l"(p + 64 * i) : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + 16 * 2 * D + (t * 32 + lane) * 4), "l"(g.bound_scales + line) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  Ids ids;
  {
    Ids x[kFsDepth];
#pragma unroll
    for (int i = 0; i < kFsDepth; ++i) x[i] = look_up(i);
#pragma unroll
    for (int i = 0; i < kFsDepth; ++i) ask(i, x[i]);
    ids = look_up(kFsDepth);
  }

  {
    // ---- query rows as codes, a warp per row (a lane: D / 32 features)
    const int rows = n_tok << a.group_shift, groups = (rows + 7) >> 3;
    for (int row = warp; row < 8 * groups; row += kFsWarps) {
      constexpr int N = D / 32;
      float x[N] = {};
      if (row < rows) {
        const T* p = static_cast<const T*>(a.q) + (long long)(i0 + (row >> a.group_shift)) * a.q_stride +
                     (long long)(h * a.group + (row & (a.group - 1))) * D + N * lane;
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = to_f32(p[e]);
      }
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
      top = __reduce_max_sync(0xffffffffu, top);
      const bool fine = top < 0x7f800000u;
      const float s_q = fminf(fmaxf(__fmul_rn(fine ? __uint_as_float(top) : 0.f, 1.f / 127.f), 0x1p-60f), 0x1p100f), inv = __frcp_rn(s_q);
      unsigned char* up = reinterpret_cast<unsigned char*>(&q_code[row][0][0]) + N * lane;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int code = fine ? min(127, max(-127, __float2int_rn(__fmul_rn(x[e], inv)))) : 0;
        up[e] = (unsigned char)max(code, 0);
        up[D + e] = (unsigned char)min(code, 0);
      }
      if (lane == 0) q_scale[row] = s_q;
    }
    __syncthreads();

    // ---- the warps that choose for one token
    int warps = kFsWarps;
    while (warps * n_tok > kFsWarps) warps >>= 1;
    const int my_k = warp / warps, my_warp = warp - my_k * warps, bar = 1 + my_k;
    uint32_t* my_key = key_of + my_k * capacity;
    FsPages my_page = {list_of + my_k * K, 0, (uint32_t)p0};

    // ---- pages [p0, p1), 16 to a warp
    int n = 0;                                     // keys in the buffer, the same for all tokens
#pragma unroll 1
    for (int step = 0; step < n_steps; ++step) {
      const int base = p0 + step * kFsStep, at = base + warp * 16 + r;
      if (n + kFsStep > capacity) {
        __syncthreads();
        if (my_k < n_tok) cut_down(my_key, my_page, n, K, sm[my_k], my_warp, warps, bar);
        n = K;
        my_page.kept = K;
        my_page.start = (uint32_t)base;
        __syncthreads();
      }
      const Ids coming = ids;
      ids = look_up(step + kFsDepth + 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(kFsDepth - 1) : "memory");
      const uint32_t src = ring + step % kFsDepth * fs_stage_bytes(D);
      uint4 b[2][2 * W];                           // [page r, r + 8][the largest values' pieces, the smallest ones']
      float s_page[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < 2 * W; ++i)
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(b[t][i].x), "=r"(b[t][i].y), "=r"(b[t][i].z), "=r"(b[t][i].w)
                       : "r"(src + ((t * 2 * W + i) * 32 + lane) * 16) : "memory");
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(s_page[t]) : "r"(src + 16 * 2 * D + (t * 32 + lane) * 4) : "memory");
      }
#pragma unroll 1
      for (int grp = 0; grp < groups; ++grp) {
        int acc[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) {
          const uint4 q = *reinterpret_cast<const uint4*>(&q_code[8 * grp + r][i / W][16 * (i % W) + 4 * c]);
          mma_s8(acc, b[0][i].x, b[1][i].x, b[0][i].y, b[1][i].y, q.x, q.y);
          mma_s8(acc, b[0][i].z, b[1][i].z, b[0][i].w, b[1][i].w, q.z, q.w);
        }
        const float2 s_col = *reinterpret_cast<const float2*>(&q_scale[8 * grp + 2 * c]);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          // (a page whose scale is NaN: the largest finite score; then the largest over the columns of a token, in all of its lanes)
          float x[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            x[e] = __fmul_rn(__fmul_rn(e ? s_col.y : s_col.x, s_page[t]), (float)acc[2 * t + e]);
            if (x[e] != x[e]) x[e] = 3.402823466e38f;
          }
          if (a.group > 1) x[0] = fmaxf(x[0], x[1]);
          if (a.group > 2) x[0] = fmaxf(x[0], __shfl_xor_sync(0xffffffffu, x[0], 1));
          if (a.group > 4) x[0] = fmaxf(x[0], __shfl_xor_sync(0xffffffffu, x[0], 2));
          const int page = at + 8 * t;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            // (the column that writes for its token: the first of the token's)
            const int row = 8 * grp + 2 * c + e, tok = row >> a.group_shift;
            if (row >= rows || (row & (a.group - 1)) != 0 || page >= p1) continue;
            const int own = (pos0 + tok) >> g.page_shift;
            const bool always = page < a.n_first || page > own - a.n_recent;
            key_of[tok * capacity + n + page - base] = page > own ? 0u : always ? kFsAlways : ordered(x[e]);
          }
        }
      }
      ask(step + kFsDepth, coming);                // (over what this lane has read)
      n += min(kFsStep, p1 - base);
    }
    __syncthreads();

    // ---- the choice
    if (my_k < n_tok) {
      const int token = i0 + my_k, own = (pos0 + my_k) >> g.page_shift;
      if (parts == 1 && own < K) {
        write_all(a, token, h, own, my_warp * 32 + lane, 32 * warps);
      } else {
        const FsChoice f = choose(my_key, n, K, sm[my_k], my_warp, warps, bar);
        if (parts == 1) {
          int32_t* out = a.out + ((long long)token * H + h) * K;
          const int m = chosen(f, my_key, n, K, sm[my_k], my_warp, warps, bar, [&](int at, int i) { out[at] = (int32_t)my_page(i); });
          for (int j = m + my_warp * 32 + lane; j < K; j += 32 * warps) out[j] = -1;
        } else {
          const FsPart ws(a.ws);
          const int slot = blockIdx.x * parts + part;
          const int m = chosen(f, my_key, n, K, sm[my_k], my_warp, warps, bar, [&](int at, int i) {
            ws.keys[slot * ECHOKV_FOURBIT_MAX_SELECT + at] = my_key[i];
            ws.pages[slot * ECHOKV_FOURBIT_MAX_SELECT + at] = my_page(i);
          });
          if (tid == 0) ws.counts[slot] = m;
        }
      }
    }
  }
}

// Chooses among what the parts of one token and head chose (each of them ascending, and so all of them one after the other).
__global__ void __launch_bounds__(kFsMaxWarps * 32) fp4_select_merge_kernel(const __grid_constant__ Fp4SelectArgs a, int parts, int capacity) {
  constexpr int kThreads = kFsMaxWarps * 32;
  extern __shared__ __align__(16) unsigned char fs_raw[];
  __shared__ FsGroup sm;
  const int tid = threadIdx.x, warp = tid >> 5, H = a.g.n_kv_heads, K = a.t.n_select, token = blockIdx.x / H, h = blockIdx.x % H;
  uint32_t *key = reinterpret_cast<uint32_t*>(fs_raw), *page = key + capacity;
  const FsPages pages = {page, capacity, 0u};
  const FsPart ws(a.ws);
  const int own = token_of(a, token).own;
  after_the_one_before();
  if (own < K) {
    write_all(a, token, h, own, tid, kThreads);
    return;
  }
  int n = 0;
  for (int p = 0; p < parts; ++p) {
    const int slot = blockIdx.x * parts + p, m = ws.counts[slot];
    if (n + m > capacity) {
      __syncthreads();
      cut_down(key, pages, n, K, sm, warp, kFsMaxWarps, 1);
      n = K;
    }
    for (int j = tid; j < m; j += kThreads) {
      key[n + j] = ws.keys[slot * ECHOKV_FOURBIT_MAX_SELECT + j];
      page[n + j] = ws.pages[slot * ECHOKV_FOURBIT_MAX_SELECT + j];
    }
    n += m;
  }
  __syncthreads();
  const FsChoice f = choose(key, n, K, sm, warp, kFsMaxWarps, 1);
  int32_t* out = a.out + ((long long)token * H + h) * K;
  const int m = chosen(f, key, n, K, sm, warp, kFsMaxWarps, 1, [&](int at, int i) { out[at] = (int32_t)page[i]; });
  for (int j = m + tid; j < K; j += kThreads) out[j] = -1;
}

int capacity_of(int tokens, int K, int step, long long wanted) {
  long long c = wanted < kFsEntries / tokens ? wanted : kFsEntries / tokens;
  const long long least = K + step;                // (1280 at most: 8 tokens have 2048 entries each)
  return (int)((c > least ? c : least) + 31) / 32 * 32;
}

template <typename T, int D, int W>
cudaError_t launch_of(const Fp4SelectArgs& a, dim3 grid, size_t smem, int tile_tokens, int capacity, cudaStream_t stream) {
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = allow_smem(fp4_select_kernel<T, D, W>, kFsRoom, &done);
  return e != cudaSuccess ? e : launch_early(fp4_select_kernel<T, D, W>, grid, W * 32, smem, stream, a, tile_tokens, capacity);
}

template <typename T, int D>
cudaError_t launch(const Fp4SelectArgs& a, int sm_count, cudaStream_t stream) {
  const int K = a.t.n_select;
  const long long heads = (long long)a.n_tokens * a.g.n_kv_heads;
  int tile_tokens = 1, parts = 1;
  const auto capacity = [&](int warps) { return capacity_of(tile_tokens, K, fs_step(warps), (a.g.max_pages + parts - 1) / parts + 2 * fs_step(warps)); };
  const auto smem_of = [&](int warps) {
    const int rows = (tile_tokens * a.group + 7) & ~7;
    return (size_t)warps * kFsDepth * fs_stage_bytes(D) + (size_t)rows * (2 * D + 4) + tile_tokens * (sizeof(FsGroup) + 4ull * (capacity(warps) + K));
  };
  const auto two_fit = [&] { return smem_of(8) <= kFsRoom / 2 - 1024; };     // on an SM
  // Tokens of a block: up to how many a sequence has on average, if there are B of them (more than tokens: B is a bound that says nothing),
  // as many as leave a block for every SM; not 8 where two blocks of 4 fit on an SM and of 8 do not (4096 tokens of 1250 pages: 987 and
  // 1053 us; where neither do, 256 tokens of 3750 pages, 282 and 194).
  // With few tokens the pages of one may be in parts.
  while (tile_tokens < kFsMaxTokens && (a.B > a.n_tokens || (long long)tile_tokens * a.B < a.n_tokens) && heads >= 2ll * tile_tokens * sm_count) {
    const bool two = two_fit();
    tile_tokens *= 2;
    if (tile_tokens == kFsMaxTokens && two && !two_fit()) {
      tile_tokens /= 2;
      break;
    }
  }
  if (tile_tokens == 1) {
    const long long room = sm_count < kFsMaxParts ? sm_count : kFsMaxParts;
    const long long most = (a.g.max_pages + kFsMinPages - 1) / kFsMinPages;
    parts = (int)(room / heads < most ? room / heads : most);
    if (parts < 1) parts = 1;
  }
  static_assert(8 * kFsDepth * fs_stage_bytes(128) + kFsMaxTokens * 8 * 260 + kFsMaxTokens * sizeof(FsGroup) + kFsEntries * 4 +
                kFsMaxTokens * (32 + ECHOKV_FOURBIT_MAX_SELECT) * 4 <= kFsRoom, "shared memory of one CTA, however many tokens and pages");
  // 16 warps, or two blocks of 8 to an SM where there are blocks for it (128 blocks: 15.5 us with 16 warps, 17 with 8, of 192 32 and 32, of
  // 320 70 and 64, of 512 95 and 71; 18 parts of a million keys 55 and 71)
  const bool shared_sm = 4 * heads > 5ll * tile_tokens * sm_count && two_fit();
  const int warps = !shared_sm && smem_of(16) <= kFsRoom ? 16 : 8;
  const dim3 grid((unsigned)heads, parts);
  cudaError_t e = warps == 16 ? launch_of<T, D, 16>(a, grid, smem_of(16), tile_tokens, capacity(16), stream)
                              : launch_of<T, D, 8>(a, grid, smem_of(8), tile_tokens, capacity(8), stream);
  if (e != cudaSuccess || parts == 1) return e;
  const int merge_capacity = capacity_of(1, K, K, (long long)parts * K);
  static std::atomic<unsigned long long> done_merge{0};
  if ((e = allow_smem(fp4_select_merge_kernel, kFsEntries * 8 + 32 * 8, &done_merge)) != cudaSuccess) return e;
  return launch_early(fp4_select_merge_kernel, dim3((unsigned)heads), kFsMaxWarps * 32, (size_t)merge_capacity * 8, stream, a, parts, merge_capacity);
}

}  // namespace

uint64_t fp4_select_workspace_bytes() {
  const uint64_t n = (uint64_t)kFsMaxParts * (2 * ECHOKV_FOURBIT_MAX_SELECT + 1) * 4;
  return (n + 255) / 256 * 256;
}

cudaError_t launch_fp4_select(const Fp4SelectArgs& a, int sm_count, cudaStream_t stream) {
  if (a.dtype == ECHOKV_BF16) return a.g.head_dim == 128 ? launch<__nv_bfloat16, 128>(a, sm_count, stream) : launch<__nv_bfloat16, 64>(a, sm_count, stream);
  return a.g.head_dim == 128 ? launch<float, 128>(a, sm_count, stream) : launch<float, 64>(a, sm_count, stream);
}

}  // namespace echokv

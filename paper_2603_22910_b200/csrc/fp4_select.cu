// The pages that a query reads: those whose keys' bounds allow the largest scores.
//
//   score(q, page) = s_q s_page sum_c (code_c > 0 ? code_c top_c : code_c low_c),   the largest over the query heads of a KV head
//
// The sum is one product of whole numbers, [q+ | q-] . [top | low], of 2 d terms: mma.sync m16n8k32 on 8-bit integers with the
// pages on the M rows and up to 8 query rows on N, exact in 32 bits, so that equal pages are equal and the choice does not depend on
// the order of anything.  A block takes one KV head of one token (or of as many tokens as fill 8 query rows, where there are tokens
// enough for all SMs); its warps take 16 pages each and write the scores, as whole numbers in the order of the floats, in the pages' order
// to shared memory.  The n_select largest are then found by a search of their least one, two bits at a time, by counting, and
// those at and above it are copied in order: what comes out is ascending, and of equal scores the first pages stay.  When the
// buffer is full it is cut down to n_select in the same way, so that a sequence may have any number of pages.  Few tokens over long caches
// are split along the pages; a second kernel then chooses among what the parts chose.
// The bound is reading the bounds, 2 d + 4 bytes a page and head.
#include "fp4_common.cuh"

namespace echokv {

namespace {

constexpr int kFsWarps = 8;
constexpr int kFsThreads = kFsWarps * 32;
constexpr int kFsStep = kFsWarps * 16;             // pages that a block takes at once
constexpr int kFsEntries = 16384;                  // keys of a block, of all its tokens
constexpr int kFsMaxParts = 640;                   // (token, head, part of the pages) with a place in the workspace
constexpr int kFsMinPages = 512;                   // pages of a part at least
constexpr uint32_t kFsAlways = 0xffffffffu;        // key of a page that is taken in any case (0: of one behind the token's own)

struct FsPart {
  uint32_t* keys;                                  // [kFsMaxParts][ECHOKV_FP4_MAX_SELECT]
  uint32_t* pages;
  int* counts;                                     // [kFsMaxParts]
  __host__ __device__ explicit FsPart(unsigned char* ws) {
    keys = reinterpret_cast<uint32_t*>(ws);
    pages = keys + kFsMaxParts * ECHOKV_FP4_MAX_SELECT;
    counts = reinterpret_cast<int*>(pages + kFsMaxParts * ECHOKV_FP4_MAX_SELECT);
  }
};

struct FsSmem {
  uint32_t key[ECHOKV_FP4_MAX_SELECT], page[ECHOKV_FP4_MAX_SELECT];
  int counts[2][kFsWarps][3];
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

// The k largest of n keys (n > k; of equal ones the first) and their pages, in their order, to sm.key / sm.page.  For the whole block, after a
// barrier; ends with one.
__device__ void choose(const uint32_t* key, const uint32_t* page, int n, int k, FsSmem& sm) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // the k-th largest key, from its top bits down: the largest v with k keys or more at or above it
  uint32_t v = 0;
#pragma unroll 1
  for (int shift = 30; shift >= 0; shift -= 2) {
    uint32_t c1 = 0, c2 = 0, c3 = 0;
    const uint32_t t1 = v | 1u << shift, t2 = v | 2u << shift, t3 = v | 3u << shift;
#pragma unroll 4
    for (int i = tid; i < n; i += kFsThreads) {
      const uint32_t x = key[i];
      c1 += x >= t1;
      c2 += x >= t2;
      c3 += x >= t3;
    }
    c1 = __reduce_add_sync(0xffffffffu, c1);
    c2 = __reduce_add_sync(0xffffffffu, c2);
    c3 = __reduce_add_sync(0xffffffffu, c3);
    int (&out)[kFsWarps][3] = sm.counts[(shift >> 1) & 1];
    if (lane == 0) {
      out[warp][0] = (int)c1;
      out[warp][1] = (int)c2;
      out[warp][2] = (int)c3;
    }
    __syncthreads();
    int a1 = 0, a2 = 0, a3 = 0;
#pragma unroll
    for (int w = 0; w < kFsWarps; ++w) {
      a1 += out[w][0];
      a2 += out[w][1];
      a3 += out[w][2];
    }
    v = a3 >= k ? t3 : a2 >= k ? t2 : a1 >= k ? t1 : v;
  }
  // every warp has a run of the keys: how many of it are above v, how many are v
  const int run = ((n + kFsWarps - 1) / kFsWarps + 31) & ~31, from = warp * run, until = min(n, from + run);
  uint32_t above = 0, equal = 0;
  for (int i = from + lane; i < until; i += 32) {
    above += key[i] > v;
    equal += key[i] == v;
  }
  above = __reduce_add_sync(0xffffffffu, above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  __syncthreads();                                 // (the counts of the last search step have been read)
  if (lane == 0) {
    sm.counts[0][warp][0] = (int)above;
    sm.counts[0][warp][1] = (int)equal;
  }
  __syncthreads();
  int all_above = 0, before_above = 0, before_equal = 0;
#pragma unroll
  for (int w = 0; w < kFsWarps; ++w) {
    all_above += sm.counts[0][w][0];
    if (w < warp) {
      before_above += sm.counts[0][w][0];
      before_equal += sm.counts[0][w][1];
    }
  }
  const int room = k - all_above;                  // of the equal ones, the first so many
  const uint32_t lower = (1u << lane) - 1;
#pragma unroll 1
  for (int i0 = from; i0 < until; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t x = i < until ? key[i] : 0;
    const uint32_t b_above = __ballot_sync(0xffffffffu, i < until && x > v), b_equal = __ballot_sync(0xffffffffu, i < until && x == v);
    const int rank_equal = before_equal + __popc(b_equal & lower), rank_above = before_above + __popc(b_above & lower);
    const bool take = (b_above >> lane & 1) || ((b_equal >> lane & 1) && rank_equal < room);
    if (take) {
      const int at = rank_above + min(rank_equal, room);
      sm.key[at] = x;
      sm.page[at] = page[i];
    }
    before_above += __popc(b_above);
    before_equal += __popc(b_equal);
  }
  __syncthreads();
}

// One token: its sequence's row of the block table and its own page (error: none of them, -1: nothing is asked for).
struct FsToken {
  int slot, own, error;
};
__device__ __forceinline__ FsToken token_of(const Fp4SelectArgs& a, int i) {
  const int seq = a.t.seqs[i], pos = a.t.positions[i];
  FsToken t = {0, -1, 0};
  if (seq < 0) t.error = -1000;
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
__device__ __forceinline__ void write_all(const Fp4SelectArgs& a, int token, int h, int own) {
  int32_t* out = a.out + ((long long)token * a.g.n_kv_heads + h) * a.t.n_select;
  for (int j = threadIdx.x; j < a.t.n_select; j += kFsThreads) out[j] = j <= own ? j : -1;
}

template <typename T, int D>
__global__ void __launch_bounds__(kFsThreads) fp4_select_kernel(const __grid_constant__ Fp4SelectArgs a, int tile_tokens, int capacity) {
  constexpr int W = D / 64;                        // 16-byte pieces of a lane: features 64 i + 16 c and on
  extern __shared__ __align__(16) uint32_t fs_raw[];
  __shared__ FsSmem sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;
  const Fp4Geom& g = a.g;
  const int H = g.n_kv_heads, K = a.t.n_select;
  const int h = blockIdx.x % H, i0 = (int)(blockIdx.x / H) * tile_tokens, n_tok = min(tile_tokens, a.n_tokens - i0);
  const int part = blockIdx.y, parts = gridDim.y;
  uint32_t* key_of = fs_raw;                       // [tile_tokens][capacity]
  uint32_t* page_of = fs_raw + tile_tokens * capacity;

  // the tokens one sequence after the other
  for (int k0 = 0, k1; k0 < n_tok; k0 = k1) {
    const FsToken first = token_of(a, i0 + k0);
    k1 = k0 + 1;
    while (k1 < n_tok && first.error == 0 && a.t.seqs[i0 + k1] == a.t.seqs[i0 + k0]) ++k1;
    int most = -1;                                 // the last page that one of them sees
    for (int k = k0; k < k1; ++k) {
      const FsToken t = token_of(a, i0 + k);
      if (t.error != 0 && t.error != -1000 && tid == 0 && part == 0) report_opt(a.status, t.error);
      most = max(most, t.own);
    }
    if (most < K) {
      if (parts == 1)
        for (int k = k0; k < k1; ++k) write_all(a, i0 + k, h, token_of(a, i0 + k).own);
      else if (tid == 0) FsPart(a.ws).counts[blockIdx.x * parts + part] = 0;
      continue;
    }
    // ---- query rows as codes: this lane's pieces of row r
    uint32_t qp[W][4], qn[W][4];
    float s_q;
    {
      const int k = r >> a.group_shift;
      float x[W][16];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        if (k >= k0 && k < k1) {
          const T* p = static_cast<const T*>(a.q) + (long long)(i0 + k) * a.q_stride + (long long)(h * a.group + (r & (a.group - 1))) * D + 64 * i + 16 * c;
#pragma unroll
          for (int e = 0; e < 16; e += Vec16<T>::N) Vec16<T>::load(p + e, &x[i][e]);
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) x[i][e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(x[i][e]) & 0x7fffffffu);
      }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const bool fine = top < 0x7f800000u;
      s_q = fminf(fmaxf(__fmul_rn(fine ? __uint_as_float(top) : 0.f, 1.f / 127.f), 0x1p-60f), 0x1p100f);
      const float inv = fine ? __frcp_rn(s_q) : 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t up = 0, down = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int code = fine ? min(127, max(-127, __float2int_rn(__fmul_rn(x[i][4 * w + e], inv)))) : 0;
            up |= (uint32_t)max(code, 0) << (8 * e);
            down |= ((uint32_t)min(code, 0) & 0xffu) << (8 * e);
          }
          qp[i][w] = up;
          qn[i][w] = down;
        }
    }
    float s_col[2];
    int own[2], tok[2];
    bool mine[2];                                  // columns 2 c, 2 c + 1: their token (of the tile), and whether this lane writes for it
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int col = 2 * c + e;
      s_col[e] = __shfl_sync(0xffffffffu, s_q, 4 * col);
      tok[e] = col >> a.group_shift;
      const bool in = tok[e] >= k0 && tok[e] < k1;
      own[e] = in ? token_of(a, i0 + tok[e]).own : -1;
      mine[e] = in && (col & (a.group - 1)) == 0;
    }

    // ---- pages [p0, p1), 16 to a warp
    const int share = (((most + parts) / parts) + kFsStep - 1) / kFsStep * kFsStep;
    const int p0 = min(most + 1, part * share), p1 = min(most + 1, p0 + share);
    const int32_t* table = a.table + (long long)first.slot * g.max_pages;
    int n = 0;                                     // keys in the buffer, the same for all tokens
    for (int base = p0; base < p1; base += kFsStep) {
      if (n + kFsStep > capacity) {
        __syncthreads();
        for (int k = k0; k < k1; ++k) {
          choose(key_of + k * capacity, page_of + k * capacity, n, K, sm);
          for (int j = tid; j < K; j += kFsThreads) {
            key_of[k * capacity + j] = sm.key[j];
            page_of[k * capacity + j] = sm.page[j];
          }
          __syncthreads();
        }
        n = K;
      }
      const int at = base + warp * 16 + r;
      uint4 hi[2][W], lo[2][W];
      float s_page[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int page = at + 8 * t;
        int id = page < p1 ? table[page] : 0;
        if (id < 0 || id >= g.n_pages) {
          report_opt(a.status, ECHOKV_EBADPAGE);
          id = 0;
        }
        const long long line = (long long)id * H + h;
        const uint4* p = reinterpret_cast<const uint4*>(g.bounds + line * 2 * D) + c;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          hi[t][i] = p[4 * i];
          lo[t][i] = p[D / 16 + 4 * i];
        }
        s_page[t] = g.bound_scales[line];
      }
      int acc[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < W; ++i) {
        mma_s8(acc, hi[0][i].x, hi[1][i].x, hi[0][i].y, hi[1][i].y, qp[i][0], qp[i][1]);
        mma_s8(acc, hi[0][i].z, hi[1][i].z, hi[0][i].w, hi[1][i].w, qp[i][2], qp[i][3]);
        mma_s8(acc, lo[0][i].x, lo[1][i].x, lo[0][i].y, lo[1][i].y, qn[i][0], qn[i][1]);
        mma_s8(acc, lo[0][i].z, lo[1][i].z, lo[0][i].w, lo[1][i].w, qn[i][2], qn[i][3]);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        uint32_t k[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float x = __fmul_rn(__fmul_rn(s_col[e], s_page[t]), (float)acc[2 * t + e]);
          k[e] = ordered(x != x ? 3.402823466e38f : x);
        }
        if (a.group > 1) k[0] = k[1] = max(k[0], k[1]);
        if (a.group > 2) k[0] = max(k[0], __shfl_xor_sync(0xffffffffu, k[0], 1));
        if (a.group > 4) k[0] = max(k[0], __shfl_xor_sync(0xffffffffu, k[0], 2));
        const int page = at + 8 * t, to = n + page - base;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (!mine[e] || page >= p1) continue;
          const bool always = page < a.n_first || page > own[e] - a.n_recent;
          key_of[tok[e] * capacity + to] = page > own[e] ? 0u : always ? kFsAlways : k[e];
          page_of[tok[e] * capacity + to] = (uint32_t)page;
        }
      }
      n += min(kFsStep, p1 - base);
    }
    __syncthreads();

    // ---- the choice
    for (int k = k0; k < k1; ++k) {
      const uint32_t* key = key_of + k * capacity;
      const uint32_t* page = page_of + k * capacity;
      int m = n;
      if (parts == 1) {
        const int own_k = token_of(a, i0 + k).own;
        if (own_k < K) {
          write_all(a, i0 + k, h, own_k);
          continue;
        }
      }
      if (n > K) {
        choose(key, page, n, K, sm);
        key = sm.key;
        page = sm.page;
        m = K;
      }
      if (parts == 1) {
        int32_t* out = a.out + ((long long)(i0 + k) * H + h) * K;
        for (int j = tid; j < K; j += kFsThreads) out[j] = (int32_t)page[j];
      } else {
        const FsPart ws(a.ws);
        const int slot = blockIdx.x * parts + part;
        for (int j = tid; j < m; j += kFsThreads) {
          ws.keys[slot * ECHOKV_FP4_MAX_SELECT + j] = key[j];
          ws.pages[slot * ECHOKV_FP4_MAX_SELECT + j] = page[j];
        }
        if (tid == 0) ws.counts[slot] = m;
      }
      __syncthreads();                             // (sm and the buffer are used again)
    }
  }
}

// Chooses among what the parts of one token and head chose (each of them ascending, and so all of them one after the other).
__global__ void __launch_bounds__(kFsThreads) fp4_select_merge_kernel(const __grid_constant__ Fp4SelectArgs a, int parts, int capacity) {
  extern __shared__ __align__(16) uint32_t fs_raw[];
  __shared__ FsSmem sm;
  const int tid = threadIdx.x, H = a.g.n_kv_heads, K = a.t.n_select, token = blockIdx.x / H, h = blockIdx.x % H;
  uint32_t *key = fs_raw, *page = fs_raw + capacity;
  const FsPart ws(a.ws);
  const int own = token_of(a, token).own;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (own < K) {
    write_all(a, token, h, own);
    return;
  }
  int n = 0;
  for (int p = 0; p < parts; ++p) {
    const int slot = blockIdx.x * parts + p, m = ws.counts[slot];
    if (n + m > capacity) {
      __syncthreads();
      choose(key, page, n, K, sm);
      for (int j = tid; j < K; j += kFsThreads) {
        key[j] = sm.key[j];
        page[j] = sm.page[j];
      }
      __syncthreads();
      n = K;
    }
    for (int j = tid; j < m; j += kFsThreads) {
      key[n + j] = ws.keys[slot * ECHOKV_FP4_MAX_SELECT + j];
      page[n + j] = ws.pages[slot * ECHOKV_FP4_MAX_SELECT + j];
    }
    n += m;
  }
  __syncthreads();
  const uint32_t* from = page;
  if (n > K) {
    choose(key, page, n, K, sm);
    from = sm.page;
  }
  int32_t* out = a.out + ((long long)token * H + h) * K;
  for (int j = tid; j < K; j += kFsThreads) out[j] = j < n ? (int32_t)from[j] : -1;
}

template <typename T, int D>
cudaError_t launch(const Fp4SelectArgs& a, int sm_count, cudaStream_t stream) {
  const int H = a.g.n_kv_heads, K = a.t.n_select;
  const long long heads = (long long)a.n_tokens * H;
  // tokens enough for every SM: as many to a block as share the products' 8 columns; otherwise one, and its pages in parts
  const int tile_tokens = heads <= 2 * sm_count ? 1 : 8 >> a.group_shift;
  const long long tiles = (a.n_tokens + tile_tokens - 1) / tile_tokens;
  int parts = 1;
  if (tile_tokens == 1) {
    const long long room = 2 * sm_count < kFsMaxParts ? 2 * sm_count : kFsMaxParts;
    const long long most = (a.g.max_pages + kFsMinPages - 1) / kFsMinPages;
    parts = (int)(room / heads < most ? room / heads : most);
    if (parts < 1) parts = 1;
  }
  const auto capacity_of = [&](int tokens, long long wanted) {
    long long c = wanted < kFsEntries / tokens ? wanted : kFsEntries / tokens;
    const long long least = K + kFsStep;           // (1152 at most: 8 tokens have 2048 entries each)
    return (int)((c > least ? c : least) + 31) / 32 * 32;
  };
  const int capacity = capacity_of(tile_tokens, ((a.g.max_pages + parts - 1) / parts + 2 * kFsStep));
  const size_t smem = (size_t)tile_tokens * capacity * 8;
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_smem(fp4_select_kernel<T, D>, kFsEntries * 8 + 8 * 32 * 8, &done);
  if (e != cudaSuccess) return e;
  fp4_select_kernel<T, D><<<dim3((unsigned)(tiles * H), parts), kFsThreads, smem, stream>>>(a, tile_tokens, capacity);
  if ((e = cudaGetLastError()) != cudaSuccess || parts == 1) return e;
  const int merge_capacity = capacity_of(1, (long long)parts * K > 2 * K ? (long long)parts * K : 2 * K);
  static std::atomic<unsigned long long> done_merge{0};
  if ((e = allow_smem(fp4_select_merge_kernel, kFsEntries * 8 + 8 * 32 * 8, &done_merge)) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)heads);
  cfg.blockDim = dim3(kFsThreads);
  cfg.dynamicSmemBytes = (size_t)merge_capacity * 8;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, fp4_select_merge_kernel, a, parts, merge_capacity);
}

}  // namespace

uint64_t fp4_select_workspace_bytes() {
  const uint64_t n = (uint64_t)kFsMaxParts * (2 * ECHOKV_FP4_MAX_SELECT + 1) * 4;
  return (n + 255) / 256 * 256;
}

cudaError_t launch_fp4_select(const Fp4SelectArgs& a, int sm_count, cudaStream_t stream) {
  if (a.dtype == ECHOKV_BF16) return a.g.head_dim == 128 ? launch<__nv_bfloat16, 128>(a, sm_count, stream) : launch<__nv_bfloat16, 64>(a, sm_count, stream);
  return a.g.head_dim == 128 ? launch<float, 128>(a, sm_count, stream) : launch<float, 64>(a, sm_count, stream);
}

}  // namespace echokv

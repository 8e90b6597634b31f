// The plan of a serving step: block table rows, slot map and free list from the requests' lengths.
//
// Integer work of a few kilobytes, so latency is all there is: ONE launch of one thread-block cluster.  Every CTA of the cluster
// scans the whole batch by itself (two block-wide prefix sums over pages and tokens; the results stay in shared
// memory), a cluster barrier makes sure that all of them have read the lengths and the free count, and then
// each writes its share of the tokens and pages -- so the lengths and the count can be updated in place, without a second
// launch, an atomic or a workspace.  Eight CTAs write a megabyte of token entries in well under the launch time; small steps
// run as one CTA.  Measured: 256 decode tokens 5.0 us, 64 prompts with 33 thousand tokens 9.9 us (three dependent
// round trips to memory, two scans and the launch).
#include "serving.h"

#include "ptx_sm100.cuh"

namespace echokv {

namespace {

constexpr int kPlanThreads = 512;
constexpr int kPlanCluster = 8;
// Up to so many tokens one CTA, above it a cluster of eight (64 sequences; 256 tokens 5.0 us with one, 5.7 with eight; 1024 5.3 and
// 5.6; 2048 6.4 and 5.7; 4096 8.6 and 5.8)
constexpr int kPlanSmallTokens = 1024;

// exclusive prefix sum over the block's threads; *total = sum over all
__device__ __forceinline__ long long block_scan(long long v, long long* warp_sums, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    long long s = lane < kPlanThreads / 32 ? warp_sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    if (lane < kPlanThreads / 32) warp_sums[lane] = s;
  }
  __syncthreads();
  const long long before = warp > 0 ? warp_sums[warp - 1] : 0;
  *total = warp_sums[kPlanThreads / 32 - 1];
  __syncthreads();
  return before + x - v;
}

// largest i in [0, n) with a[i] <= v (a ascending, a[0] <= v)
__device__ __forceinline__ int find_last(const int* a, int n, int v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= v) lo = mid; else hi = mid;
  }
  return lo;
}

struct Seq {
  int slot, len, fresh, old_pages, need;
  int error;
};

__device__ __forceinline__ Seq load_seq(const PlanArgs& a, int b) {
  Seq s;
  s.slot = a.slots ? a.slots[b] : b;
  s.len = a.lens[b];
  s.fresh = a.new_lens[b];
  s.error = 0;
  const long long cap = (long long)a.max_pages * a.page_tokens;
  if (s.slot < 0 || s.slot >= a.max_batch) s.error = ECHOKV_EBADPAGE;
  else if (s.len < 0 || s.fresh < 0 || (long long)s.len + s.fresh > cap) s.error = ECHOKV_EBADLENGTH;
  if (s.error) s.fresh = 0;
  s.old_pages = s.error ? 0 : (s.len + a.page_tokens - 1) >> a.page_shift;
  s.need = s.error ? 0 : ((s.len + s.fresh + a.page_tokens - 1) >> a.page_shift) - s.old_pages;
  return s;
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(PlanArgs a) {
  extern __shared__ int plan_smem[];
  __shared__ long long warp_sums[kPlanThreads / 32];
  const int B = a.B, tid = threadIdx.x;
  // per sequence: first new token, tokens before the step, pages before it, pages taken before it, block table row
  int* cu = plan_smem;                // [B + 1]
  int* len_s = cu + B + 1;
  int* page0 = len_s + B;             // exclusive prefix of the pages needed, [B + 1] (clamped to what is there)
  int* old_s = page0 + B + 1;
  int* slot_s = old_s + B;
  const int rank = (int)(gridDim.x > 1 ? cluster_ctarank() : 0), n_cta = gridDim.x;

  long long count = a.free_count[0];
  count = count < 0 ? 0 : count > a.n_pages ? a.n_pages : count;
  const int per = (B + kPlanThreads - 1) / kPlanThreads;
  const int b0 = min(B, tid * per), b1 = min(B, b0 + per);
  // pages and tokens that the sequences ask for
  long long need = 0, toks = 0;
  for (int b = b0; b < b1; ++b) {
    const Seq s = load_seq(a, b);
    need += s.need;
    toks += s.fresh;
  }
  long long total;
  long long page_at = block_scan(need, warp_sums, &total);
  long long tok_at = block_scan(toks, warp_sums, &total);
  // who is served.  The served sequences that take pages are the first ones that need any, so what is taken from the
  // stack is contiguous.
  long long taken = 0, used = 0;
  for (int b = b0; b < b1; ++b) {
    const Seq s = load_seq(a, b);
    const bool fits = (s.need == 0 || page_at + s.need <= count) && tok_at + s.fresh <= a.n_tokens;
    if (rank == 0 && (s.error || !fits)) report_opt(a.status, s.error ? s.error : ECHOKV_ECAPACITY);
    page0[b] = (int)(page_at < count ? page_at : count);
    if (fits && s.need > 0) used = page_at + s.need;
    page_at += s.need;
    tok_at += s.fresh;
    len_s[b] = s.len;
    old_s[b] = s.old_pages;
    slot_s[b] = s.error ? -1 : s.slot;
    cu[b] = fits ? s.fresh : 0;
    taken += cu[b];
  }
  long long at = block_scan(taken, warp_sums, &total);
  for (int b = b0; b < b1; ++b) {
    const int n = cu[b];
    cu[b] = (int)at;
    at += n;
  }
  const int n_live = (int)total;
  if (tid == 0) cu[B] = n_live;
  // pages taken = largest end of a served sequence's pages
  {
    __syncthreads();
    long long u = used;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const long long v = __shfl_xor_sync(0xffffffffu, u, o);
      if (v > u) u = v;
    }
    if ((tid & 31) == 0) warp_sums[tid >> 5] = u;
    __syncthreads();
    u = 0;
    for (int i = 0; i < kPlanThreads / 32; ++i)
      if (warp_sums[i] > u) u = warp_sums[i];
    used = u;
  }
  if (tid == 0) page0[B] = (int)used;
  __syncthreads();
  if (n_cta > 1) cluster_sync_all();          // everyone has read the lengths and the count: they may change now

  if (rank == 0) {
    for (int b = tid; b < B; b += kPlanThreads) {
      a.out.cu_tokens[b] = cu[b];
      a.out.seq_lens[b] = len_s[b] + cu[b + 1] - cu[b];
    }
    if (tid == 0) {
      a.out.cu_tokens[B] = n_live;
      a.out.free_count[0] = (int32_t)(count - used);
    }
  }
  const int stride = n_cta * kPlanThreads, first = rank * kPlanThreads + tid;
  // pages taken -> block table
  for (int k = first; k < (int)used; k += stride) {
    const int b = find_last(page0, B, k);     // (equal entries: the last one, which is the one that needs pages)
    const int page = a.free_pages[count - 1 - k];
    if (page < 0 || page >= a.n_pages) report_opt(a.status, ECHOKV_EBADPAGE);
    a.table[(long long)slot_s[b] * a.max_pages + old_s[b] + k - page0[b]] = page;
  }
  // tokens, four of a thread's at a time so that their page look-ups overlap
  constexpr int kBatch = 4;
  for (int t0 = first; t0 < a.n_tokens; t0 += kBatch * stride) {
    int seq[kBatch], pos[kBatch], page[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + i * stride;
      seq[i] = pos[i] = page[i] = -1;
      if (t < n_live) {
        const int b = find_last(cu, B, t);
        seq[i] = b;
        pos[i] = len_s[b] + t - cu[b];
        const int pi = pos[i] >> a.page_shift;
        page[i] = pi < old_s[b] ? a.table[(long long)slot_s[b] * a.max_pages + pi] : a.free_pages[count - 1 - (page0[b] + pi - old_s[b])];
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + i * stride;
      if (t >= a.n_tokens) break;
      const bool ok = page[i] >= 0 && page[i] < a.n_pages;
      if (seq[i] >= 0 && !ok) report_opt(a.status, ECHOKV_EBADPAGE);
      a.out.positions[t] = pos[i];
      a.out.token_seqs[t] = seq[i];
      a.out.slot_map[t] = seq[i] >= 0 && ok ? (long long)page[i] * a.page_tokens + (pos[i] & (a.page_tokens - 1)) : -1;
    }
  }
}

__global__ void __launch_bounds__(kPlanThreads) release_kernel(ReleaseArgs a) {
  extern __shared__ int plan_smem[];
  __shared__ long long warp_sums[kPlanThreads / 32];
  int* page0 = plan_smem;             // [B]
  const int B = a.B, tid = threadIdx.x;
  const long long cap = (long long)a.max_pages * a.page_tokens;
  auto pages_of = [&](int b, bool tell) -> int {
    const int slot = a.slots ? a.slots[b] : b, len = a.lens[b];
    const int err = (slot < 0 || slot >= a.max_batch) ? ECHOKV_EBADPAGE : (len < 0 || len > cap) ? ECHOKV_EBADLENGTH : 0;
    if (err && tell) report_opt(a.status, err);
    return err ? 0 : (len + a.page_tokens - 1) >> a.page_shift;
  };
  long long count = a.free_count[0];
  count = count < 0 ? 0 : count > a.n_pages ? a.n_pages : count;
  const int per = (B + kPlanThreads - 1) / kPlanThreads;
  const int b0 = min(B, tid * per), b1 = min(B, b0 + per);
  // pages that can go back: those with a valid id (counted first, so that the list stays without holes)
  long long n = 0;
  for (int b = b0; b < b1; ++b) n += pages_of(b, true);
  long long total;
  long long at = block_scan(n, warp_sums, &total);
  for (int b = b0; b < b1; ++b) {
    page0[b] = (int)(at < 0x7fffffff ? at : 0x7fffffff);
    at += pages_of(b, false);
  }
  // (more pages than the pool has cannot all be somebody's)
  if (total > a.n_pages || total > 0x7ffffffe) {
    if (tid == 0) report_opt(a.status, ECHOKV_ECAPACITY);
    total = a.n_pages < 0x7ffffffe ? a.n_pages : 0x7ffffffe;
  }
  __syncthreads();
  // in rounds of one page per thread: a scan over the valid ones gives each its place
  long long done = count;
  for (long long base = 0; base < total; base += kPlanThreads) {
    const long long k = base + tid;
    int page = -1;
    if (k < total) {
      const int b = find_last(page0, B, (int)k);
      page = a.table[(long long)(a.slots ? a.slots[b] : b) * a.max_pages + (int)k - page0[b]];
      if (page < 0 || page >= a.n_pages) {
        report_opt(a.status, ECHOKV_EBADPAGE);
        page = -1;
      }
    }
    long long got;
    const long long place = done + block_scan(page >= 0 ? 1 : 0, warp_sums, &got);
    if (page >= 0) {
      if (place < a.n_pages) a.free_pages[place] = page;
      else report_opt(a.status, ECHOKV_ECAPACITY);
    }
    done += got;
  }
  if (tid == 0) a.free_count[0] = (int32_t)(done < a.n_pages ? done : a.n_pages);
}

}  // namespace

cudaError_t launch_plan(const PlanArgs& a, cudaStream_t stream) {
  const size_t smem = (size_t)(5 * a.B + 2) * sizeof(int);
  if (smem > 40 * 1024) {
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_smem(plan_kernel, (5 * kPlanMaxBatch + 2) * sizeof(int), &done);
    if (e != cudaSuccess) return e;
  }
  if (a.n_tokens <= kPlanSmallTokens) {
    plan_kernel<<<1, kPlanThreads, smem, stream>>>(a);
    return cudaGetLastError();
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kPlanCluster);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = cfg.gridDim.x;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, plan_kernel, a);
}

cudaError_t launch_release(const ReleaseArgs& a, cudaStream_t stream) {
  release_kernel<<<1, kPlanThreads, (size_t)a.B * sizeof(int), stream>>>(a);
  return cudaGetLastError();
}

}  // namespace echokv

// C-ABI of the serving step over an 8-bit cache: argument checking and kernel arguments.  No call allocates; the calling
// thread's current device is put back.
#include <cmath>
#include <cstring>
#include <mutex>

#include "serving.h"

using namespace echokv;

namespace {

constexpr int kMaxDevices = 64;
constexpr int kMaxRows = 1 << 27;   // new tokens of a call: times 8 query heads they still fit 31 bits
constexpr int kChunkRows = 64;      // query rows per KV head (new tokens x query heads that share it) from which a bf16 sequence can be the
                                    // chunk kernel's

int sm_count_of(int device, int* out) {
  static std::mutex mutex;
  static int known[kMaxDevices] = {};
  if (device < 0 || device >= kMaxDevices) return ECHOKV_EINVAL;
  std::lock_guard<std::mutex> lock(mutex);
  if (known[device] == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) return ECHOKV_ECUDA;
    known[device] = n;
  }
  *out = known[device];
  return ECHOKV_OK;
}

// Makes `device` current for the call and puts the caller's back.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    if (cudaGetDevice(&before_) != cudaSuccess) return;
    if (before_ != device) {
      if (cudaSetDevice(device) != cudaSuccess) return;
      switched_ = true;
    }
    ok_ = sm_count_of(device, &sm_count) == ECHOKV_OK;
  }
  ~OnDevice() {
    if (switched_) cudaSetDevice(before_);
  }
  bool ok() const { return ok_; }
  int sm_count = 0;

 private:
  int before_ = 0;
  bool switched_ = false, ok_ = false;
};

inline bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// arrays of int32 or fp32 (NULL where one is optional)
template <typename... P>
inline bool words(const P*... p) {
  return (aligned(p, 4) && ...);
}

int log2_of(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

int check_pages(const echokv_config* c) {
  if (c->max_batch < 1 || c->max_pages_per_seq < 1 || c->n_pages < 1 || c->device < 0 || c->device >= kMaxDevices) return ECHOKV_EINVAL;
  if (c->n_pages > 0x7fffffffll) return ECHOKV_EINVAL;                                  // (page ids are int32)
  if ((long long)c->max_pages_per_seq * c->page_tokens > (1ll << 30)) return ECHOKV_EINVAL;
  if (c->page_tokens != 16 && c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128) return ECHOKV_EUNSUPPORTED;
  return ECHOKV_OK;
}

int check_heads(const echokv_config* c) {
  if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads % c->n_kv_heads != 0) return ECHOKV_EINVAL;
  if (c->dtype != ECHOKV_BF16 && c->dtype != ECHOKV_FP32) return ECHOKV_EINVAL;
  if (c->device < 0 || c->device >= kMaxDevices) return ECHOKV_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return ECHOKV_EUNSUPPORTED;
  const int g = c->n_q_heads / c->n_kv_heads;
  if (g != 1 && g != 2 && g != 4 && g != 8) return ECHOKV_EUNSUPPORTED;
  return ECHOKV_OK;
}

int check_all(const echokv_config* c) {
  if (!c) return ECHOKV_EINVAL;
  int rc = check_heads(c);
  if (rc == ECHOKV_OK) rc = check_pages(c);
  // (the rows of the 8-bit pools are indexed in 32 bits: 2^31 rows of 64 bytes are 128 GB)
  if (rc == ECHOKV_OK && (long long)c->n_pages * c->n_kv_heads >= 0x7fffffffll / c->page_tokens) rc = ECHOKV_EINVAL;
  if (rc == ECHOKV_OK && (!(c->softmax_scale >= 0.f) || !std::isfinite(c->softmax_scale))) rc = ECHOKV_EINVAL;
  return rc;
}

// (the two attention kernels of a call use it one after the other)
uint64_t quant_workspace(const echokv_config* c) {
  const uint64_t rows = quant_attn_workspace_bytes(c->head_dim), chunks = quant_chunk_workspace_bytes(c->head_dim);
  return c->dtype == ECHOKV_BF16 && chunks > rows ? chunks : rows;
}

// rows of `width` elements, `stride` elements apart: 16-byte aligned, not overlapping
bool rows_ok(const void* p, long long stride, int width, int elem) {
  return p != nullptr && aligned(p, 16) && stride >= width && stride * elem % 16 == 0 && stride < (1ll << 40);
}

// does one of `n` rows (`width` bytes, `stride` bytes apart) have a byte of [other, other + size)?
bool rows_meet(const void* rows, long long stride, long long width, long long n, const void* other, long long size) {
  const long long from = (long long)(reinterpret_cast<uintptr_t>(other) - reinterpret_cast<uintptr_t>(rows));
  const long long i = from < width ? 0 : (from - width) / stride + 1;      // the first row that ends behind `other`
  return i < n && i * stride < from + size;
}

int quant_geom(const echokv_config* c, const echokv_quant_cache* q, QuantGeom* g) {
  if (!q || !q->k_codes || !q->v_codes || !q->k_scales || !q->v_scales || !q->k_tail || !q->v_tail) return ECHOKV_EINVAL;
  if (!aligned(q->k_codes, 16) || !aligned(q->v_codes, 16) || !aligned(q->k_scales, 16) || !aligned(q->v_scales, 16) ||
      !aligned(q->k_tail, 16) || !aligned(q->v_tail, 16))
    return ECHOKV_EINVAL;
  if (q->format != ECHOKV_INT8 && q->format != ECHOKV_E4M3) return ECHOKV_EINVAL;
  g->codes[0] = static_cast<unsigned char*>(q->k_codes); g->codes[1] = static_cast<unsigned char*>(q->v_codes);
  g->scales[0] = q->k_scales; g->scales[1] = q->v_scales;
  g->tail[0] = q->k_tail; g->tail[1] = q->v_tail;
  g->n_kv_heads = c->n_kv_heads; g->head_dim = c->head_dim;
  g->page_tokens = c->page_tokens; g->page_shift = log2_of(c->page_tokens);
  g->max_pages = c->max_pages_per_seq; g->max_batch = c->max_batch;
  g->n_pages = c->n_pages;
  return ECHOKV_OK;
}

}  // namespace

extern "C" {

int echokv_plan_tokens(const echokv_config* cfg, int32_t* dev_block_table, const int32_t* dev_seq_slots,
                       const int32_t* dev_seq_lens, const int32_t* dev_new_lens, const int32_t* dev_free_pages,
                       const int32_t* dev_free_count, int B, int n_tokens, const echokv_step_plan* plan,
                       int32_t* dev_status, void* stream) {
  if (!cfg || !dev_block_table || !dev_seq_lens || !dev_new_lens || !dev_free_pages || !dev_free_count || !plan) return ECHOKV_EINVAL;
  if (B < 1 || n_tokens < 0 || n_tokens > (1 << 30)) return ECHOKV_EINVAL;
  if (!plan->cu_tokens || !plan->seq_lens || !plan->free_count) return ECHOKV_EINVAL;
  if (n_tokens > 0 && (!plan->positions || !plan->token_seqs || !plan->slot_map)) return ECHOKV_EINVAL;
  if (!words(dev_block_table, dev_seq_slots, dev_seq_lens, dev_new_lens, dev_free_pages, dev_free_count, dev_status, plan->cu_tokens,
             plan->positions, plan->token_seqs, plan->seq_lens, plan->free_count) || !aligned(plan->slot_map, 8))
    return ECHOKV_EINVAL;
  const int rc = check_pages(cfg);
  if (rc != ECHOKV_OK) return rc;
  if (B > cfg->max_batch || B > kPlanMaxBatch) return ECHOKV_ECAPACITY;
  OnDevice dev(cfg->device);
  if (!dev.ok()) return ECHOKV_ECUDA;
  PlanArgs a;
  a.table = dev_block_table; a.slots = dev_seq_slots; a.lens = dev_seq_lens; a.new_lens = dev_new_lens;
  a.free_pages = dev_free_pages; a.free_count = dev_free_count;
  a.B = B; a.n_tokens = n_tokens;
  a.page_tokens = cfg->page_tokens; a.page_shift = log2_of(cfg->page_tokens);
  a.max_pages = cfg->max_pages_per_seq; a.max_batch = cfg->max_batch; a.n_pages = cfg->n_pages;
  a.out = *plan;
  a.status = dev_status;
  return launch_plan(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ECHOKV_OK : ECHOKV_ECUDA;
}

int echokv_release_pages(const echokv_config* cfg, const int32_t* dev_block_table, const int32_t* dev_seq_slots,
                         const int32_t* dev_seq_lens, int B, int32_t* dev_free_pages, int32_t* dev_free_count,
                         int32_t* dev_status, void* stream) {
  if (!cfg || !dev_block_table || !dev_seq_lens || !dev_free_pages || !dev_free_count || B < 1) return ECHOKV_EINVAL;
  if (!words(dev_block_table, dev_seq_slots, dev_seq_lens, dev_free_pages, dev_free_count, dev_status)) return ECHOKV_EINVAL;
  const int rc = check_pages(cfg);
  if (rc != ECHOKV_OK) return rc;
  if (B > cfg->max_batch || B > kPlanMaxBatch) return ECHOKV_ECAPACITY;
  OnDevice dev(cfg->device);
  if (!dev.ok()) return ECHOKV_ECUDA;
  ReleaseArgs a;
  a.table = dev_block_table; a.slots = dev_seq_slots; a.lens = dev_seq_lens;
  a.free_pages = dev_free_pages; a.free_count = dev_free_count;
  a.B = B;
  a.page_tokens = cfg->page_tokens; a.page_shift = log2_of(cfg->page_tokens);
  a.max_pages = cfg->max_pages_per_seq; a.max_batch = cfg->max_batch; a.n_pages = cfg->n_pages;
  a.status = dev_status;
  return launch_release(a, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ECHOKV_OK : ECHOKV_ECUDA;
}

int echokv_rotate(const echokv_config* cfg, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                  void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, const int32_t* dev_positions,
                  int n_axes, const int32_t* sections, int interleaved, int rot_dim, double theta, int inverse,
                  int n_tokens, void* stream) {
  if (!cfg || n_tokens < 0 || n_tokens > (1 << 30) || n_axes < 1 || n_axes > kMaxAxes) return ECHOKV_EINVAL;
  if (!(theta >= 1.0) || !std::isfinite(theta)) return ECHOKV_EINVAL;
  const int rc = check_heads(cfg);
  if (rc != ECHOKV_OK) return rc;
  const int elem = cfg->dtype == ECHOKV_BF16 ? 2 : 4, d = cfg->head_dim;
  if (rot_dim == 0) rot_dim = d;
  if (rot_dim < 0 || rot_dim > d || rot_dim % (32 / elem) != 0) return ECHOKV_EUNSUPPORTED;
  const int half = rot_dim / 2;
  RotateArgs a;
  if (sections) {
    int sum = 0;
    for (int i = 0; i < n_axes; ++i) {
      if (sections[i] < 0 || sections[i] > half) return ECHOKV_EINVAL;
      sum += sections[i];
    }
    if (sum != half) return ECHOKV_EINVAL;
  } else if (n_axes != 1) {
    return ECHOKV_EINVAL;
  }
  if (n_tokens == 0) return ECHOKV_OK;
  if (!dev_positions || !aligned(dev_positions, 4)) return ECHOKV_EINVAL;
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  const int64_t is[2] = {q_stride, k_stride}, os[2] = {q_out_stride, k_out_stride};
  const int heads[2] = {cfg->n_q_heads, cfg->n_kv_heads};
  for (int i = 0; i < 2; ++i) {
    if ((in[i] == nullptr) != (out[i] == nullptr)) return ECHOKV_EINVAL;
    a.in[i] = in[i]; a.out[i] = out[i];
    a.in_stride[i] = is[i]; a.out_stride[i] = os[i];
    a.heads[i] = heads[i];
    a.in_place[i] = in[i] == out[i];
    if (!in[i]) continue;
    if (!rows_ok(in[i], is[i], heads[i] * d, elem) || !rows_ok(out[i], os[i], heads[i] * d, elem)) return ECHOKV_EINVAL;
    if (a.in_place[i] && is[i] != os[i]) return ECHOKV_EINVAL;
  }
  if (!q && !k) return ECHOKV_EINVAL;
  a.head_dim = d; a.rot_dim = rot_dim; a.n_tokens = n_tokens; a.dtype = cfg->dtype;
  a.pos = dev_positions;
  a.sign = inverse ? -1.f : 1.f;
  int axis = 0, until = sections ? sections[0] : half;
  // theta^(-2 j / rot) as a running product: 64 factors, 64 roundings of 2^-53
  const double step = std::pow(theta, -2.0 / rot_dim);
  double freq = 1.0 / 6.283185307179586476925287;
  for (int j = 0; j < half; ++j) {
    if (interleaved && sections) {
      axis = j % n_axes;
      if (j / n_axes >= sections[axis]) axis = 0;
    } else {
      while (j >= until) until += sections[++axis];
    }
    a.axis[j] = (unsigned char)axis;
    a.turns[j] = freq;
    freq *= step;
  }
  OnDevice dev(cfg->device);
  if (!dev.ok()) return ECHOKV_ECUDA;
  return launch_rotate(a, dev.sm_count, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ECHOKV_OK : ECHOKV_ECUDA;
}

int echokv_query_quant_sizes(const echokv_config* cfg, echokv_quant_sizes* out) {
  if (!out) return ECHOKV_EINVAL;
  const int rc = check_all(cfg);
  if (rc != ECHOKV_OK) return rc;
  const uint64_t rows = (uint64_t)cfg->n_pages * cfg->page_tokens * cfg->n_kv_heads;
  out->codes_bytes = rows * cfg->head_dim;
  out->scales_bytes = rows / kQuantBlock * 4;
  out->tail_bytes = (uint64_t)cfg->max_batch * cfg->n_kv_heads * kQuantBlock * cfg->head_dim * (cfg->dtype == ECHOKV_BF16 ? 2 : 4);
  out->workspace_bytes = quant_workspace(cfg);
  return ECHOKV_OK;
}

int echokv_quant_append(const echokv_config* cfg, const echokv_quant_cache* cache, const void* k_new, int64_t k_stride,
                        const void* v_new, int64_t v_stride, const int64_t* dev_slot_map,
                        const int32_t* dev_token_seqs, const int32_t* dev_cu_tokens, const int32_t* dev_seq_slots, int B,
                        int n_tokens, int32_t* dev_status, void* stream) {
  int rc = check_all(cfg);
  if (rc != ECHOKV_OK) return rc;
  if (B < 1 || n_tokens < 0 || n_tokens > kMaxRows) return ECHOKV_EINVAL;
  QuantAppendArgs a;
  if ((rc = quant_geom(cfg, cache, &a.g)) != ECHOKV_OK) return rc;
  if (B > cfg->max_batch) return ECHOKV_ECAPACITY;
  if (n_tokens == 0) return ECHOKV_OK;
  const int elem = cfg->dtype == ECHOKV_BF16 ? 2 : 4, width = cfg->n_kv_heads * cfg->head_dim;
  if (!rows_ok(k_new, k_stride, width, elem) || !rows_ok(v_new, v_stride, width, elem)) return ECHOKV_EINVAL;
  if (!dev_slot_map || !dev_token_seqs || !dev_cu_tokens) return ECHOKV_EINVAL;
  if (!aligned(dev_slot_map, 8) || !words(dev_token_seqs, dev_cu_tokens, dev_seq_slots, dev_status)) return ECHOKV_EINVAL;
  a.x[0] = k_new; a.x[1] = v_new;
  a.stride[0] = k_stride; a.stride[1] = v_stride;
  a.slot_map = dev_slot_map; a.token_seqs = dev_token_seqs; a.cu = dev_cu_tokens; a.slots = dev_seq_slots;
  a.B = B; a.n_tokens = n_tokens; a.dtype = cfg->dtype; a.format = cache->format;
  a.status = dev_status;
  OnDevice dev(cfg->device);
  if (!dev.ok()) return ECHOKV_ECUDA;
  return launch_quant_append(a, dev.sm_count, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ECHOKV_OK : ECHOKV_ECUDA;
}

int echokv_quant_attention(const echokv_config* cfg, const echokv_quant_cache* cache, const echokv_score_options* options,
                           const void* q, int64_t q_stride, void* out, const int32_t* dev_block_table,
                           const int32_t* dev_seq_slots, const int32_t* dev_seq_lens, const int32_t* dev_cu_tokens, int B,
                           int n_tokens, int max_new, void* workspace, uint64_t workspace_bytes, int32_t* dev_status,
                           void* stream) {
  int rc = check_all(cfg);
  if (rc != ECHOKV_OK) return rc;
  if (B < 1 || n_tokens < 0 || n_tokens > kMaxRows || max_new < 1) return ECHOKV_EINVAL;
  if (!dev_cu_tokens && (n_tokens != B || max_new != 1)) return ECHOKV_EINVAL;
  QuantAttnArgs a;
  if ((rc = quant_geom(cfg, cache, &a.g)) != ECHOKV_OK) return rc;
  // (a cap so small that its inverse leaves fp32's range is no cap anybody means)
  if (options && (!(options->softcap == 0.f || options->softcap >= 1e-30f) || !std::isfinite(options->softcap))) return ECHOKV_EINVAL;
  if (B > cfg->max_batch) return ECHOKV_ECAPACITY;
  if (n_tokens == 0) return ECHOKV_OK;
  const int elem = cfg->dtype == ECHOKV_BF16 ? 2 : 4;
  if (!rows_ok(q, q_stride, cfg->n_q_heads * cfg->head_dim, elem)) return ECHOKV_EINVAL;
  if (!out || !aligned(out, 16) || !dev_block_table || !dev_seq_lens) return ECHOKV_EINVAL;
  // (the kernels read an item's queries before they write its rows, so in place is as good as apart)
  const long long row_bytes = (long long)cfg->n_q_heads * cfg->head_dim * elem;
  if (!(q == out && (n_tokens == 1 || q_stride * elem == row_bytes)) &&
      rows_meet(q, q_stride * elem, row_bytes, n_tokens, out, n_tokens * row_bytes))
    return ECHOKV_EINVAL;
  if (!words(dev_block_table, dev_seq_slots, dev_seq_lens, dev_cu_tokens, dev_status)) return ECHOKV_EINVAL;
  if (options && !words(options->alibi_slopes, options->prefix_lens)) return ECHOKV_EINVAL;
  if (!workspace || !aligned(workspace, 256)) return ECHOKV_EINVAL;
  if (workspace_bytes < quant_workspace(cfg)) return ECHOKV_ECAPACITY;
  a.q = q; a.q_stride = q_stride; a.out = out;
  a.table = dev_block_table; a.slots = dev_seq_slots; a.lens = dev_seq_lens; a.cu = dev_cu_tokens;
  a.softcap = options ? options->softcap : 0.f;
  a.slopes = options ? options->alibi_slopes : nullptr;
  a.prefix = options ? options->prefix_lens : nullptr;
  a.B = B; a.n_tokens = n_tokens; a.max_new = max_new;
  a.n_q_heads = cfg->n_q_heads; a.group = cfg->n_q_heads / cfg->n_kv_heads; a.group_shift = log2_of(a.group);
  a.dtype = cfg->dtype; a.format = cache->format;
  a.scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / std::sqrt((float)cfg->head_dim);
  a.chunk_rows = cfg->dtype == ECHOKV_BF16 && (long long)max_new * a.group >= kChunkRows ? kChunkRows : 0;
  a.ws = static_cast<unsigned char*>(workspace);
  a.status = dev_status;
  OnDevice dev(cfg->device);
  if (!dev.ok()) return ECHOKV_ECUDA;
  a.sm_count = dev.sm_count;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.chunk_rows > 0 && launch_quant_chunk(a, dev.sm_count, s) != cudaSuccess) return ECHOKV_ECUDA;
  return launch_quant_attn(a, dev.sm_count, s) == cudaSuccess ? ECHOKV_OK : ECHOKV_ECUDA;
}

}  // extern "C"

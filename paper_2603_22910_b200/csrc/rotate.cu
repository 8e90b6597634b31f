// Rotary position embedding of fresh queries and keys over several position axes.
//
// One pass over q and k (read once, written once); the work per element is three FLOP, so the kernel is HBM-bound for prompts and
// launch-bound for decode.  A block takes a few tokens: its threads first form the (cos, sin) of the tokens' rot/2
// angles in shared memory -- once per token, for all heads of q and k -- then stream the rows, each thread a 16-byte piece of the
// first and of the second half of a head.  Angles: position * theta^(-2j/rot) / 2 pi in fp64, reduced to the nearest
// whole turn there (positions of a million tokens lose nothing), the remainder turned into sin / cos in fp32 by
// sincospi.
#include "serving.h"

namespace echokv {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotTokens = 4;                   // tokens per block: 4 x 64 angles = one per thread

template <typename T>
__global__ void __launch_bounds__(kRotThreads) rotate_kernel(const __grid_constant__ RotateArgs a, int tokens_per_block) {
  constexpr int N = Vec16<T>::N;
  __shared__ float2 cs[kRotTokens][64];
  const int half = a.rot_dim >> 1, tid = threadIdx.x;
  const int t0 = blockIdx.x * tokens_per_block, nt = min(tokens_per_block, a.n_tokens - t0);
  for (int i = tid; i < nt * half; i += kRotThreads) {
    const int t = i / half, j = i - t * half;
    const double turns = (double)a.pos[(long long)a.axis[j] * a.n_tokens + t0 + t] * a.turns[j];
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    cs[t][j] = make_float2(c, s * a.sign);
  }
  __syncthreads();
  // pieces of a head: half / N rotated pairs, then the 16-byte pieces behind rot_dim (copied unless in place)
  const int pairs = half / N;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (a.in[which] == nullptr) continue;
    const int rest = a.in_place[which] ? 0 : (a.head_dim - a.rot_dim) / N;
    const int per_head = pairs + rest, per_token = per_head * a.heads[which];
    const T* in = static_cast<const T*>(a.in[which]);
    T* out = static_cast<T*>(a.out[which]);
    for (int i = tid; i < nt * per_token; i += kRotThreads) {
      const int t = i / per_token, r = i - t * per_token, h = r / per_head, c = r - h * per_head;
      const T* src = in + (long long)(t0 + t) * a.in_stride[which] + h * a.head_dim;
      T* dst = out + (long long)(t0 + t) * a.out_stride[which] + h * a.head_dim;
      if (c < pairs) {
        float x1[N], x2[N];
        Vec16<T>::load(src + c * N, x1);
        Vec16<T>::load(src + half + c * N, x2);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float2 w = cs[t][c * N + e];
          const float y1 = x1[e] * w.x - x2[e] * w.y, y2 = x2[e] * w.x + x1[e] * w.y;
          x1[e] = y1;
          x2[e] = y2;
        }
        store16<T>(dst + c * N, x1);
        store16<T>(dst + half + c * N, x2);
      } else {
        const int o = a.rot_dim + (c - pairs) * N;
        *reinterpret_cast<uint4*>(dst + o) = *reinterpret_cast<const uint4*>(src + o);
      }
    }
  }
}

}  // namespace

cudaError_t launch_rotate(const RotateArgs& a, int sm_count, cudaStream_t stream) {
  // few tokens: one per block, so that a decode step's rows spread over the SMs
  const int per_block = a.n_tokens <= 4 * sm_count ? 1 : kRotTokens;
  const unsigned grid = (unsigned)((a.n_tokens + per_block - 1) / per_block);
  if (a.dtype == ECHOKV_BF16) rotate_kernel<__nv_bfloat16><<<grid, kRotThreads, 0, stream>>>(a, per_block);
  else rotate_kernel<float><<<grid, kRotThreads, 0, stream>>>(a, per_block);
  return cudaGetLastError();
}

}  // namespace echokv

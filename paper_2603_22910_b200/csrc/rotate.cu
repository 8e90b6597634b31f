// Rotary position embedding of fresh queries and keys over several position axes.
//
// One pass over q and k (read once, written once); the work per element is three FLOP, so the kernel is HBM-bound for prompts and
// launch-bound for decode.  A block takes a few tokens: its threads first form the (cos, sin) of the tokens' rot/2
// angles in shared memory -- once per token, for all heads of q and k -- then stream the rows.  A unit of that is two 16-byte pieces
// of a head: a piece of the first half with its partner of the second, or two neighbours of what is only copied; a
// thread keeps its place in the head and goes from head to head, two units' loads in flight.  Angles: position *
// theta^(-2j/rot) / 2 pi in fp64, reduced to the nearest whole turn there (positions of a million tokens lose nothing), the
// remainder turned into sin / cos in fp32 by sincospi.  Measured: 16385 tokens of 40 bf16 heads of 128 in 57 us (336 MB, 5.9
// TB/s), 2049 of 64 fp32 heads, half of each rotated, in 22 us (6.1 TB/s), 64 tokens in 2.9 us.
#include "serving.h"

namespace echokv {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotTokens = 4;                   // tokens per block: 4 x 64 angles = one per thread

template <typename T, int D>
__global__ void __launch_bounds__(kRotThreads, 5) rotate_kernel(const __grid_constant__ RotateArgs a, int tokens_per_block) {
  constexpr int N = Vec16<T>::N;                 // elements of a piece
  constexpr int U = D / (2 * N);                 // units of a head
  constexpr int kBatch = 2;                      // units of a thread in flight (with 5 blocks per SM; 4 units and 3 blocks: 65
                                                 // against 57 us for 16385 tokens of 40 heads, 27 against 22 us in fp32)
  __shared__ __align__(16) float2 cs[kRotTokens][64];
  const int half = a.rot_dim >> 1, tid = threadIdx.x;
  const int t0 = blockIdx.x * tokens_per_block, nt = min(tokens_per_block, a.n_tokens - t0);
  for (int i = tid; i < nt * half; i += kRotThreads) {
    const int t = i / half, j = i - t * half;
    const double turns = (double)a.pos[(long long)a.axis[j] * a.n_tokens + t0 + t] * a.turns[j];
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    // (two neighbours of a piece side by side, pieces next: what eight lanes read together is contiguous)
    const int piece = j / N, e = j - piece * N;
    cs[t][((e >> 1) * (half / N) + piece) * 2 + (e & 1)] = make_float2(c, s * a.sign);
  }
  __syncthreads();
  const int pairs = half / N, c = tid % U;
  const bool turn = c < pairs;
  // the unit's two pieces within a head
  const int e0 = turn ? c * N : a.rot_dim + 2 * (c - pairs) * N, e1 = turn ? half + c * N : e0 + N;
  const int hq = a.in[0] ? a.heads[0] : 0, hall = hq + (a.in[1] ? a.heads[1] : 0);
  constexpr int kStep = kRotThreads / U;         // heads that the block takes at once
  // head `h` of token `t` (heads of q, then of k), taken kStep further each time
  int t = 0, h = tid / U;
  const auto settle = [&]() {
    while (h >= hall && t < nt) {
      h -= hall;
      ++t;
    }
  };
  settle();
  while (t < nt) {
    uint4 x[kBatch][2];
    T* dst[kBatch];
    int tok[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      dst[k] = nullptr;
      tok[k] = t;
      if (t < nt) {
        const int which = h < hq ? 0 : 1, head = h - (which ? hq : 0);
        if (turn || !a.in_place[which]) {
          const T* src = static_cast<const T*>(a.in[which]) + (long long)(t0 + t) * a.in_stride[which] + head * D;
          dst[k] = static_cast<T*>(a.out[which]) + (long long)(t0 + t) * a.out_stride[which] + head * D;
          x[k][0] = *reinterpret_cast<const uint4*>(src + e0);
          x[k][1] = *reinterpret_cast<const uint4*>(src + e1);
        }
        h += kStep;
        settle();
      }
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (dst[k] == nullptr) continue;
      if (turn) {
        float x1[N], x2[N];
        Vec16<T>::load(reinterpret_cast<const T*>(&x[k][0]), x1);
        Vec16<T>::load(reinterpret_cast<const T*>(&x[k][1]), x2);
        const float4* w4 = reinterpret_cast<const float4*>(&cs[tok[k]][c * 2]);
#pragma unroll
        for (int e = 0; e < N; e += 2) {
          const float4 w = w4[(e / 2) * pairs];
          const float y1 = x1[e] * w.x - x2[e] * w.y, y2 = x2[e] * w.x + x1[e] * w.y;
          const float z1 = x1[e + 1] * w.z - x2[e + 1] * w.w, z2 = x2[e + 1] * w.z + x1[e + 1] * w.w;
          x1[e] = y1; x2[e] = y2;
          x1[e + 1] = z1; x2[e + 1] = z2;
        }
        store16<T>(dst[k] + e0, x1);
        store16<T>(dst[k] + e1, x2);
      } else {
        *reinterpret_cast<uint4*>(dst[k] + e0) = x[k][0];
        *reinterpret_cast<uint4*>(dst[k] + e1) = x[k][1];
      }
    }
  }
}

template <typename T>
void launch(const RotateArgs& a, unsigned grid, int per_block, cudaStream_t stream) {
  if (a.head_dim == 128) rotate_kernel<T, 128><<<grid, kRotThreads, 0, stream>>>(a, per_block);
  else rotate_kernel<T, 64><<<grid, kRotThreads, 0, stream>>>(a, per_block);
}

}  // namespace

cudaError_t launch_rotate(const RotateArgs& a, int sm_count, cudaStream_t stream) {
  // few tokens: one per block, so that a decode step's rows spread over the SMs
  const int per_block = a.n_tokens <= 4 * sm_count ? 1 : kRotTokens;
  const unsigned grid = (unsigned)((a.n_tokens + per_block - 1) / per_block);
  if (a.dtype == ECHOKV_BF16) launch<__nv_bfloat16>(a, grid, per_block, stream);
  else launch<float>(a, grid, per_block, stream);
  return cudaGetLastError();
}

}  // namespace echokv

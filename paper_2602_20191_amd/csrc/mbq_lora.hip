// Low-rank adapters of many requests at once beside the shared projections, forward and backward.
#include "mbq_lora.h"

namespace mbq {

namespace {
__device__ __forceinline__ float bf16_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ int own_rank(const int32_t* ranks, int a, int r) {
  if (!ranks) return r;
  const int own = ranks[a];
  return own < 0 ? 0 : (own > r ? r : own);
}
}  // namespace

// Stable grouping by adapter: workgroup a counts the tokens of smaller adapters (where a's begin) and then ranks its own by
// ballots.  Workgroup n takes the tokens without one.  Every workgroup reads the whole assignment, which the caches hold.
constexpr int kSortThreads = 256;
__global__ __launch_bounds__(kSortThreads) void lora_sort_kernel(const int32_t* __restrict__ adapter, int T, int n,
                                                                 int32_t* __restrict__ perm,
                                                                 int32_t* __restrict__ offsets) {
  constexpr int kWaves = kSortThreads / 64;
  __shared__ int counts[2][kWaves];
  const int a = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const auto key = [&](int i) {
    const int id = adapter[i];
    return (unsigned)id < (unsigned)n ? id : n;
  };
  int less = 0;
  for (int i = tid; i < T; i += kSortThreads) less += key(i) < a;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) less += __shfl_xor(less, off, 64);
  if (lane == 0) counts[0][wave] = less;
  __syncthreads();
  int at = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) at += counts[0][w];
  if (tid == 0) offsets[a] = at;
  __syncthreads();
  for (int i0 = 0, turn = 0; i0 < T; i0 += kSortThreads, turn ^= 1) {
    const int i = i0 + tid;
    const bool mine = i < T && key(i) == a;
    const unsigned long long found = __ballot(mine);
    if (lane == 0) counts[turn][wave] = __popcll(found);
    __syncthreads();
    int before = at;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) before += counts[turn][w];
      at += counts[turn][w];
    }
    if (mine) perm[before + __popcll(found & ((1ull << lane) - 1))] = i;
  }
}

mbq_status launch_lora_sort(const int32_t* adapter, int64_t T, int64_t n, int32_t* perm, int32_t* offsets,
                            hipStream_t stream) {
  hipLaunchKernelGGL(lora_sort_kernel, dim3((unsigned)n + 1), dim3(kSortThreads), 0, stream, adapter, (int)T, (int)n, perm,
                     offsets);
  return hip_status(hipGetLastError(), "lora_sort_kernel launch");
}

// h[t][j] = (scale) sum over L columns of x[t][.] w[a][j][.], one workgroup per token.
template <typename In>
__global__ __launch_bounds__(256) void lora_shrink_kernel(const In* __restrict__ x, int64_t L, const uint16_t* __restrict__ w,
                                                          int n, int r, const int32_t* __restrict__ ranks,
                                                          const float* __restrict__ scale,
                                                          const int32_t* __restrict__ adapter, float* __restrict__ h) {
  __shared__ float part[4];
  const int64_t t = blockIdx.x;
  const int a = adapter[t], tid = threadIdx.x;
  const int own = (unsigned)a < (unsigned)n ? own_rank(ranks, a, r) : 0;
  for (int j = 0; j < r; ++j) {
    float sum = 0.f;
    if (j < own) {
      const uint16_t* row = w + ((int64_t)a * r + j) * L;
      for (int64_t k = tid; k < L; k += 256) {
        float v;
        if constexpr (sizeof(In) == 2) v = bf16_value(x[t * L + k]);
        else v = x[t * L + k];
        sum += v * bf16_value(row[k]);
      }
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
    __syncthreads();
    if ((tid & 63) == 0) part[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) {
      sum = part[0] + part[1] + part[2] + part[3];
      h[t * r + j] = j < own ? (scale ? scale[a] * sum : sum) : 0.f;
    }
  }
}

// y[t][c] = base[t][c] + (scale) sum_j h[t][j] w[a][j][c], one thread per output.
__global__ __launch_bounds__(256) void lora_expand_kernel(const float* __restrict__ h, int64_t T, int64_t L,
                                                          const uint16_t* __restrict__ w, int n, int r,
                                                          const int32_t* __restrict__ ranks, const float* __restrict__ scale,
                                                          const int32_t* __restrict__ adapter, const float* base, float* y) {
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (idx >= T * L) return;
  const int64_t t = idx / L, c = idx - t * L;
  const int a = adapter[t];
  float sum = 0.f;
  if ((unsigned)a < (unsigned)n) {
    const int own = own_rank(ranks, a, r);
    for (int j = 0; j < own; ++j) sum += h[t * r + j] * bf16_value(w[((int64_t)a * r + j) * L + c]);
    if (scale) sum *= scale[a];
  }
  y[idx] = (base ? base[idx] : 0.f) + sum;
}

// d[a][j][c] = (scale) sum over the tokens of a of h[t][j] x[t][c], one thread per value.
template <typename In>
__global__ __launch_bounds__(256) void lora_outer_kernel(const float* __restrict__ h, const In* __restrict__ x, int64_t L,
                                                         int r, const int32_t* __restrict__ ranks,
                                                         const float* __restrict__ scale, const int32_t* __restrict__ perm,
                                                         const int32_t* __restrict__ offsets, float* __restrict__ d) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int j = blockIdx.y, a = blockIdx.z;
  if (c >= L) return;
  float sum = 0.f;
  if (j < own_rank(ranks, a, r))
    for (int i = offsets[a]; i < offsets[a + 1]; ++i) {
      const int64_t t = perm[i];
      float v;
      if constexpr (sizeof(In) == 2) v = bf16_value(x[t * L + c]);
      else v = x[t * L + c];
      sum += h[t * r + j] * v;
    }
  d[((int64_t)a * r + j) * L + c] = scale ? sum * scale[a] : sum;
}

size_t lora_workspace_bytes(int64_t T, int64_t K, int n, int r) {
  (void)K;
  return (size_t)T * n * r * 4 + 256;
}

mbq_status launch_lora(const LoraCall& c, hipStream_t stream) {
  float* h = reinterpret_cast<float*>(c.ws);
  for (int p = 0; p < c.n; ++p) {
    float* hp = c.H[p] ? c.H[p] : h + (size_t)p * c.T * c.r;
    hipLaunchKernelGGL((lora_shrink_kernel<uint16_t>), dim3((unsigned)c.T), dim3(256), 0, stream, c.X, c.K, c.A[p],
                       (int)c.adapters, c.r, c.ranks, (const float*)nullptr, c.adapter, hp);
    hipLaunchKernelGGL(lora_expand_kernel, dim3((unsigned)((c.T * c.N[p] + 255) / 256)), dim3(256), 0, stream, hp, c.T,
                       c.N[p], c.B[p], (int)c.adapters, c.r, c.ranks, c.scale, c.adapter, c.base[p], c.Y[p]);
  }
  return hip_status(hipGetLastError(), "adapter kernels' launch");
}

size_t lora_backward_workspace_bytes(int64_t T, int64_t K, int n, const int64_t* N, int64_t adapters, int r) {
  (void)K, (void)N, (void)adapters;
  return (size_t)T * n * r * 4 + 256;
}

mbq_status launch_lora_backward(const LoraCall& c, hipStream_t stream) {
  float* const g = reinterpret_cast<float*>(c.ws);
  for (int p = 0; p < c.n; ++p) {
    if (c.T > 0) {
      hipLaunchKernelGGL((lora_shrink_kernel<float>), dim3((unsigned)c.T), dim3(256), 0, stream, c.dY[p], c.N[p], c.B[p],
                         (int)c.adapters, c.r, c.ranks, c.scale, c.adapter, g);
      if (c.dX)
        hipLaunchKernelGGL(lora_expand_kernel, dim3((unsigned)((c.T * c.K + 255) / 256)), dim3(256), 0, stream, g, c.T, c.K,
                           c.A[p], (int)c.adapters, c.r, c.ranks, (const float*)nullptr, c.adapter, p ? c.dX : c.dx_base,
                           c.dX);
    }
    if (c.dA[p])
      hipLaunchKernelGGL((lora_outer_kernel<uint16_t>), dim3((unsigned)((c.K + 255) / 256), c.r, (unsigned)c.adapters),
                         dim3(256), 0, stream, g, c.X, c.K, c.r, c.ranks, (const float*)nullptr, c.perm, c.offsets, c.dA[p]);
    if (c.dB[p])
      hipLaunchKernelGGL((lora_outer_kernel<float>), dim3((unsigned)((c.N[p] + 255) / 256), c.r, (unsigned)c.adapters),
                         dim3(256), 0, stream, c.Hin[p], c.dY[p], c.N[p], c.r, c.ranks, c.scale, c.perm, c.offsets, c.dB[p]);
  }
  return hip_status(hipGetLastError(), "adapter gradients' launch");
}

}  // namespace mbq

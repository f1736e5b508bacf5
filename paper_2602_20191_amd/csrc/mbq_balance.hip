// The routers' training beside a frozen blob: tokens per precision and the balance loss with its gradient for the logits,
// and the logits' gradient taken on to the routers' parameters and their input.
#include "mbq_lora.h"

namespace mbq {

namespace {
__device__ __forceinline__ float bf16_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
}  // namespace

// One workgroup per router: a pass for counts and probabilities, a pass for the gradient.
__global__ __launch_bounds__(256) void balance_kernel(const BalanceCall c) {
  __shared__ double part[256][MBQ_MAX_SLICES + 1];
  __shared__ int count[256][MBQ_MAX_SLICES];
  const int tid = threadIdx.x, P = c.P;
  const double* S = c.logits[blockIdx.x];
  double sum[MBQ_MAX_SLICES] = {};
  int seen[MBQ_MAX_SLICES] = {};
  const auto softmax = [&](int64_t t, double* p) {
    int best = 0;
    double m = S[t * P];
    for (int e = 1; e < P; ++e)
      if (S[t * P + e] > m) m = S[t * P + e], best = e;
    double total = 0.0;
    for (int e = 0; e < P; ++e) total += p[e] = exp(S[t * P + e] - m);
    for (int e = 0; e < P; ++e) p[e] /= total;
    return best;
  };
  for (int64_t t = tid; t < c.T; t += 256) {
    if (c.mask && !c.mask[t]) continue;
    double p[MBQ_MAX_SLICES];
    const int best = softmax(t, p);
    for (int e = 0; e < P; ++e) sum[e] += p[e], seen[e] += e == best;
  }
  for (int e = 0; e < P; ++e) part[tid][e] = sum[e], count[tid][e] = seen[e];
  __syncthreads();
  double prob[MBQ_MAX_SLICES] = {}, u[MBQ_MAX_SLICES] = {};
  long long tokens[MBQ_MAX_SLICES] = {}, n = 0;
  for (int e = 0; e < P; ++e) {
    for (int i = 0; i < 256; ++i) prob[e] += part[i][e], tokens[e] += count[i][e];
    n += tokens[e];
  }
  const double per = n ? 1.0 / (double)n : 0.0;
  double loss = 0.0;
  for (int e = 0; e < P; ++e) {
    u[e] = (double)tokens[e] * per * c.weight[e];
    loss += u[e] * prob[e] * per;
  }
  if (tid == 0) {
    for (int e = 0; e < P; ++e) c.counts[blockIdx.x][e] = (int)tokens[e];
    c.loss[blockIdx.x][0] = (float)(c.coef * loss);
  }
  float* d = c.dlogits[blockIdx.x];
  if (!d) return;
  for (int64_t t = tid; t < c.T; t += 256) {
    double p[MBQ_MAX_SLICES] = {}, mean = 0.0;
    if (!c.mask || c.mask[t]) softmax(t, p);
    for (int e = 0; e < P; ++e) mean += u[e] * p[e];
    for (int e = 0; e < P; ++e) d[t * P + e] = p[e] == 0.0 ? 0.f : (float)(c.coef * per * p[e] * (u[e] - mean));
  }
}

size_t balance_loss_workspace_bytes(int64_t T, int n) {
  (void)T, (void)n;
  return 256;
}

mbq_status launch_balance_loss(const BalanceCall& c, hipStream_t stream) {
  hipLaunchKernelGGL(balance_kernel, dim3((unsigned)c.n), dim3(256), 0, stream, c);
  return hip_status(hipGetLastError(), "balance_kernel launch");
}

__global__ __launch_bounds__(256) void route_dx_kernel(const RouteBackwardCall c) {
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (idx >= c.T * c.K) return;
  const int64_t t = idx / c.K, k = idx - t * c.K;
  float sum = 0.f;
  if (!c.mask || c.mask[t])
    for (int p = 0; p < c.n; ++p)
      for (int e = 0; e < c.P; ++e) sum += c.dlogits[p][t * c.P + e] * c.Wr[p][e * c.K + k];
  c.dX[idx] = (c.base ? c.base[idx] : 0.f) + sum;
}
__global__ __launch_bounds__(256) void route_dw_kernel(const RouteBackwardCall c) {
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int e = blockIdx.y, p = blockIdx.z;
  if (k > c.K) return;
  float sum = 0.f;
  for (int64_t t = 0; t < c.T; ++t)
    if (!c.mask || c.mask[t]) sum += c.dlogits[p][t * c.P + e] * (k < c.K ? bf16_value(c.X[t * c.K + k]) : 1.f);
  if (k < c.K) {
    if (c.dWr[p]) c.dWr[p][e * c.K + k] = sum;
  } else if (c.dbr[p]) {
    c.dbr[p][e] = sum;
  }
}

size_t route_backward_workspace_bytes(int64_t T, int64_t K, int n, int P) {
  (void)T, (void)K, (void)n, (void)P;
  return 256;
}

mbq_status launch_route_backward(const RouteBackwardCall& c, hipStream_t stream) {
  if (c.dX && c.T > 0)
    hipLaunchKernelGGL(route_dx_kernel, dim3((unsigned)((c.T * c.K + 255) / 256)), dim3(256), 0, stream, c);
  if (c.dWr[0] || c.dbr[0])
    hipLaunchKernelGGL(route_dw_kernel, dim3((unsigned)(c.K / 256 + 1), c.P, c.n), dim3(256), 0, stream, c);
  return hip_status(hipGetLastError(), "route gradients' launch");
}

}  // namespace mbq

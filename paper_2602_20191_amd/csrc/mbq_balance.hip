// The routers' training beside a frozen blob: tokens per precision and the balance loss with its gradient for the logits,
// and the logits' gradient taken on to the routers' parameters and their input.
#include "mbq_lora.h"

namespace mbq {

namespace {
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef floatx4 floatx4_any __attribute__((aligned(4)));  // base and dX begin at any float
__device__ __forceinline__ float low_bf16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high_bf16(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
}  // namespace

// ---- the loss ----------------------------------------------------------------------------------------------------
// Everything is fp64: the gradient is p (u_e - sum_j u_j p_j), a small difference where the mix is near its target.  The
// gradient needs every token's choice, so there are two passes over the logits, one launch for up to kBalanceSmall tokens (a
// workgroup per router that keeps its tokens' softmax in registers), two launches beyond, the second re-reading logits that the
// caches hold.  Bound by launches: 512 tokens 4.0 us; 32768 tokens and four routers, 6 MB, 4.8 and
// 5.5 us.
constexpr int kBalanceSmall = 1024, kSmallThreads = 512, kBalanceThreads = 256, kBalanceBlocks = 128;

struct BalanceSums {
  double p[MBQ_MAX_SLICES];
  int count[MBQ_MAX_SLICES];
};

template <int P>
struct Softmax {
  double p[P];
  int best;  // the first maximum
};
template <int P>
__device__ __forceinline__ Softmax<P> softmax(const double* __restrict__ S) {
  double v[P];
#pragma unroll
  for (int e = 0; e < P; ++e) v[e] = S[e];
  Softmax<P> r;
  r.best = 0;
  double m = v[0];
#pragma unroll
  for (int e = 1; e < P; ++e)
    if (v[e] > m) m = v[e], r.best = e;
  double total = 0.0;
#pragma unroll
  for (int e = 0; e < P; ++e) total += r.p[e] = exp(v[e] - m);
  const double inverse = 1.0 / total;
#pragma unroll
  for (int e = 0; e < P; ++e) r.p[e] *= inverse;
  return r;
}
// a token that is left out: no choice, no probability
template <int P>
__device__ __forceinline__ Softmax<P> token(const double* S, const uint8_t* mask, int64_t t, bool there) {
  Softmax<P> r = {};
  r.best = -1;
  if (there && (!mask || mask[t])) r = softmax<P>(S + t * P);
  return r;
}

// The sums of all threads, in a fixed order, to every thread of the workgroup.
template <int P, int kThreads>
__device__ __forceinline__ BalanceSums workgroup_sums(BalanceSums s, BalanceSums* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int e = 0; e < P; ++e)
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      s.p[e] += __shfl_xor(s.p[e], off, 64);
      s.count[e] += __shfl_xor(s.count[e], off, 64);
    }
  if (lane == 0) lds[wave] = s;
  __syncthreads();
  BalanceSums all = {};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w)
#pragma unroll
    for (int e = 0; e < P; ++e) all.p[e] += lds[w].p[e], all.count[e] += lds[w].count[e];
  return all;
}

template <int P>
struct Loss {
  double u[P], per, loss;  // per: 1 / tokens kept, 0 if none
};
template <int P>
__device__ __forceinline__ Loss<P> loss_of(const BalanceCall& c, const BalanceSums& s) {
  Loss<P> l;
  long long n = 0;
#pragma unroll
  for (int e = 0; e < P; ++e) n += s.count[e];
  l.per = n ? 1.0 / (double)n : 0.0;
  l.loss = 0.0;
#pragma unroll
  for (int e = 0; e < P; ++e) {
    l.u[e] = (double)s.count[e] * l.per * c.weight[e];
    l.loss += l.u[e] * s.p[e] * l.per;
  }
  return l;
}
template <int P>
__device__ __forceinline__ void write_loss(const BalanceCall& c, int router, const BalanceSums& s, const Loss<P>& l) {
#pragma unroll
  for (int e = 0; e < P; ++e) c.counts[router][e] = s.count[e];
  c.loss[router][0] = (float)(c.coef * l.loss);
}
template <int P>
__device__ __forceinline__ void write_gradient(const BalanceCall& c, int router, int64_t t, const Softmax<P>& r,
                                               const Loss<P>& l) {
  double mean = 0.0;
#pragma unroll
  for (int e = 0; e < P; ++e) mean += l.u[e] * r.p[e];
  float* d = c.dlogits[router] + t * P;
#pragma unroll
  for (int e = 0; e < P; ++e) d[e] = (float)(c.coef * l.per * r.p[e] * (l.u[e] - mean));
}

template <int P>
__global__ __launch_bounds__(kSmallThreads) void balance_small_kernel(const BalanceCall c) {
  constexpr int kEach = kBalanceSmall / kSmallThreads;  // tokens of a thread
  __shared__ BalanceSums lds[kSmallThreads / 64];
  const int router = blockIdx.x;
  Softmax<P> r[kEach];
  BalanceSums s = {};
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int t = k * kSmallThreads + threadIdx.x;
    r[k] = token<P>(c.logits[router], c.mask, t, t < c.T);
#pragma unroll
    for (int e = 0; e < P; ++e) s.p[e] += r[k].p[e], s.count[e] += r[k].best == e;
  }
  s = workgroup_sums<P, kSmallThreads>(s, lds);
  const Loss<P> l = loss_of<P>(c, s);
  if (threadIdx.x == 0) write_loss<P>(c, router, s, l);
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int t = k * kSmallThreads + threadIdx.x;
    if (c.dlogits[router] && t < c.T) write_gradient<P>(c, router, t, r[k], l);
  }
}

// grid (blocks, routers); a workgroup's sums go to ws[router][block]
template <int P>
__global__ __launch_bounds__(kBalanceThreads) void balance_sums_kernel(const BalanceCall c) {
  __shared__ BalanceSums lds[kBalanceThreads / 64];
  BalanceSums s = {};
  for (int64_t t = (int64_t)blockIdx.x * kBalanceThreads + threadIdx.x; t < c.T; t += (int64_t)gridDim.x * kBalanceThreads) {
    const Softmax<P> r = token<P>(c.logits[blockIdx.y], c.mask, t, true);
#pragma unroll
    for (int e = 0; e < P; ++e) s.p[e] += r.p[e], s.count[e] += r.best == e;
  }
  s = workgroup_sums<P, kBalanceThreads>(s, lds);
  if (threadIdx.x == 0) reinterpret_cast<BalanceSums*>(c.ws)[blockIdx.y * gridDim.x + blockIdx.x] = s;
}
// every workgroup adds the blocks' sums up again
template <int P>
__global__ __launch_bounds__(kBalanceThreads) void balance_gradient_kernel(const BalanceCall c, int blocks) {
  static_assert(kBalanceBlocks <= kBalanceThreads, "a thread per block");
  __shared__ BalanceSums lds[kBalanceThreads / 64];
  const int router = blockIdx.y;
  BalanceSums s = {};
  if ((int)threadIdx.x < blocks) s = reinterpret_cast<const BalanceSums*>(c.ws)[router * blocks + threadIdx.x];
  s = workgroup_sums<P, kBalanceThreads>(s, lds);
  const Loss<P> l = loss_of<P>(c, s);
  if (blockIdx.x == 0 && threadIdx.x == 0) write_loss<P>(c, router, s, l);
  if (!c.dlogits[router]) return;
  for (int64_t t = (int64_t)blockIdx.x * kBalanceThreads + threadIdx.x; t < c.T; t += (int64_t)gridDim.x * kBalanceThreads)
    write_gradient<P>(c, router, t, token<P>(c.logits[router], c.mask, t, true), l);
}

namespace {
int balance_blocks(int64_t T) {
  const int64_t blocks = (T + kBalanceThreads - 1) / kBalanceThreads;
  return (int)(blocks < kBalanceBlocks ? blocks : kBalanceBlocks);
}
template <int P>
void launch_balance(const BalanceCall& c, hipStream_t stream) {
  if (c.T <= kBalanceSmall) {
    hipLaunchKernelGGL(balance_small_kernel<P>, dim3(c.n), dim3(kSmallThreads), 0, stream, c);
    return;
  }
  const int blocks = balance_blocks(c.T);
  hipLaunchKernelGGL(balance_sums_kernel<P>, dim3(blocks, c.n), dim3(kBalanceThreads), 0, stream, c);
  const bool gradient = c.dlogits[0] != nullptr;
  hipLaunchKernelGGL(balance_gradient_kernel<P>, dim3(gradient ? (unsigned)((c.T + kBalanceThreads - 1) / kBalanceThreads) : 1, c.n),
                     dim3(kBalanceThreads), 0, stream, c, blocks);
}
}  // namespace

size_t balance_loss_workspace_bytes(int64_t T, int n) {
  return T <= kBalanceSmall ? 256 : (size_t)balance_blocks(T) * n * sizeof(BalanceSums) + 256;
}

mbq_status launch_balance_loss(const BalanceCall& c, hipStream_t stream) {
  switch (c.P) {
    case 1: launch_balance<1>(c, stream); break;
    case 2: launch_balance<2>(c, stream); break;
    case 3: launch_balance<3>(c, stream); break;
    default: launch_balance<4>(c, stream); break;
  }
  return hip_status(hipGetLastError(), "balance kernels' launch");
}

// ---- the routers' gradients ----------------------------------------------------------------------------------------
// One pass over X (and base) for all routers that read it: a lane owns four columns, holds their router weights and their
// sums of dWr, and walks over the tokens of its share, four at a time, whose dlogits come from LDS.  32 multiply-adds a column and token for
// four routers of four outputs, under half of what the vector units do in the time the memory needs, so it is bound by memory.
// A workgroup's four wavefronts share 256 columns and take tokens in turn; their sums meet in LDS, the chunks' in a second
// launch, in order.  4096 tokens of 8192 columns, three routers: 79 us, 336 MB at 4.3 TB/s, and 5 us for the join.
constexpr int kRouteColumns = 256, kRouteWaves = 4, kRouteAhead = 4, kRouteStage = 64;

struct RouteBackwardArgs {
  RouteBackwardCall c;
  int chunk;        // tokens of a workgroup
  float* partial;   // [chunk][n P][K], then [chunk][n P]; null: one chunk, results go to dWr and dbr
  float* partial_b;
};

// kRouters: routers of the call.
template <int kRouters, bool kStream>
__global__ __launch_bounds__(256) void route_backward_kernel(const RouteBackwardArgs s) {
  constexpr int kOut = kRouters * 4;
  __shared__ float red[kRouteWaves][4][4][64];
  __shared__ __align__(16) float ds[kRouteStage][kOut];  // dlogits of the tokens at hand, zero for those left out
  __shared__ uint32_t keeps[kRouteStage];                // all ones, or zero for a token left out
  const RouteBackwardCall& c = s.c;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), P = c.P;
  const int64_t K = c.K, c0 = (int64_t)blockIdx.x * kRouteColumns + 4 * lane;
  float w[kOut][4], sum[kOut][4];
#pragma unroll
  for (int o = 0; o < kOut; ++o)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[o][i] = 0.f;
      w[o][i] = 0.f;
      if ((o & 3) < P && c0 < K) w[o][i] = c.Wr[o >> 2][(int64_t)(o & 3) * K + c0 + i];  // (K is a multiple of 128)
    }
  const int64_t t0 = (int64_t)blockIdx.y * s.chunk, t1 = min(t0 + s.chunk, c.T);
  float bias = 0.f;  // thread o of the first workgroups: the sum of dlogits of output o

  struct Loads {
    uint2 x[kRouteAhead];
    floatx4 y[kRouteAhead];
  };
  const bool with_base = c.dX && c.base;
  const auto load = [&](Loads& l, int64_t t) {  // tokens t .. t + 3 (those that are not there repeat the last)
#pragma unroll
    for (int k = 0; k < kRouteAhead; ++k) {
      const int64_t row = min(t + k, t1 - 1) * K;
      l.x[k] = uint2{0, 0};
      l.y[k] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (c0 >= K) continue;
      l.x[k] = *reinterpret_cast<const uint2*>(c.X + row + c0);
      if (!with_base) continue;
      const floatx4_any* from = reinterpret_cast<const floatx4_any*>(c.base + row + c0);
      if constexpr (kStream)
        l.y[k] = __builtin_nontemporal_load(from);
      else
        l.y[k] = *from;
    }
  };
  const auto use = [&](const Loads& l, int64_t t, int at) {  // at: where the tokens' dlogits lie
#pragma unroll
    for (int k = 0; k < kRouteAhead; ++k) {
      if (t + k >= t1) break;
      const uint32_t keep = keeps[at + k];
      float d[kOut];
#pragma unroll
      for (int o = 0; o < kOut; o += 4) *reinterpret_cast<floatx4*>(d + o) = *reinterpret_cast<const floatx4*>(&ds[at + k][o]);
      const uint32_t xl = l.x[k].x & keep, xh = l.x[k].y & keep;
      const float xv[4] = {low_bf16(xl), high_bf16(xl), low_bf16(xh), high_bf16(xh)};
      floatx4 y = l.y[k];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float g = 0.f;
#pragma unroll
        for (int o = 0; o < kOut; ++o) {
          g += d[o] * w[o][i];
          sum[o][i] += d[o] * xv[i];
        }
        y[i] += __uint_as_float(__float_as_uint(g) & keep);
      }
      if (c.dX && c0 < K) {
        floatx4_any* to = reinterpret_cast<floatx4_any*>(c.dX + (t + k) * K + c0);
        if constexpr (kStream)
          __builtin_nontemporal_store(y, to);
        else
          *to = y;
      }
    }
  };
  for (int64_t stage = t0; stage < t1; stage += kRouteStage) {
    const int count = (int)min((int64_t)kRouteStage, t1 - stage);
    Loads now, next;
    if (stage + wave * kRouteAhead < t1) load(now, stage + wave * kRouteAhead);
    __syncthreads();
    for (int e = threadIdx.x; e < count * kOut; e += 256) {
      const int k = e / kOut, o = e - k * kOut;
      const int64_t token = stage + k;
      float v = 0.f;
      if ((o & 3) < P && (!c.mask || c.mask[token])) v = c.dlogits[o >> 2][token * P + (o & 3)];
      ds[k][o] = v;
    }
    for (int k = threadIdx.x; k < count; k += 256) keeps[k] = !c.mask || c.mask[stage + k] ? 0xFFFFFFFFu : 0u;
    __syncthreads();
    if (blockIdx.x == 0 && threadIdx.x < kOut)
      for (int k = 0; k < count; ++k) bias += ds[k][threadIdx.x];
    for (int k = wave * kRouteAhead; k < count; k += kRouteWaves * kRouteAhead) {
      const bool more = k + kRouteWaves * kRouteAhead < count;
      if (more) load(next, stage + k + kRouteWaves * kRouteAhead);
      use(now, stage + k, k);
      if (more) now = next;
    }
  }
  const int outputs = kRouters * P;
  if (c.dWr[0] || s.partial)
#pragma unroll
    for (int p = 0; p < kRouters; ++p) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave][e][i][lane] = sum[4 * p + e][i];
      __syncthreads();
      // wavefront e writes output e
      if (wave < P) {
        float* to = s.partial ? s.partial + ((int64_t)blockIdx.y * outputs + p * P + wave) * K : c.dWr[p] + (int64_t)wave * K;
        floatx4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[i] = (red[0][wave][i][lane] + red[1][wave][i][lane]) + (red[2][wave][i][lane] + red[3][wave][i][lane]);
        if (c0 < K) *reinterpret_cast<floatx4_any*>(to + c0) = v;
      }
    }
  if (blockIdx.x == 0 && threadIdx.x < kOut && (threadIdx.x & 3) < P && (c.dbr[0] || s.partial)) {
    const int o = threadIdx.x;
    if (s.partial)
      s.partial_b[(int64_t)blockIdx.y * outputs + (o >> 2) * P + (o & 3)] = bias;
    else
      c.dbr[o >> 2][o & 3] = bias;
  }
}

// The chunks' sums, in order.
__global__ __launch_bounds__(256) void route_join_kernel(const RouteBackwardArgs s, int chunks) {
  const RouteBackwardCall& c = s.c;
  const int64_t outputs = (int64_t)c.n * c.P, values = outputs * c.K, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const bool weight = i < values;
  if (i >= values + outputs) return;
  const float* from = weight ? s.partial + i : s.partial_b + (i - values);
  const int64_t next = weight ? values : outputs;
  float sum = 0.f;
  int k = 0;
  for (; k + 8 <= chunks; k += 8) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = from[(k + e) * next];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[e];
  }
  for (; k < chunks; ++k) sum += from[k * next];
  if (weight) {
    const int64_t o = i / c.K, p = o / c.P;
    if (c.dWr[p]) c.dWr[p][(o - p * c.P) * c.K + (i - o * c.K)] = sum;
  } else {
    const int64_t o = i - values, p = o / c.P;
    if (c.dbr[p]) c.dbr[p][o - p * c.P] = sum;
  }
}

namespace {
// Tokens of a workgroup: about 1024 workgroups, but at least 32 tokens each, so that the chunks' sums stay small beside X
// (333 tokens of 2176 columns 12.5 us at 64, 9.7 at 32 and at 16).
int route_chunk(int64_t T, int64_t K) {
  const int64_t blocks = (K + kRouteColumns - 1) / kRouteColumns;
  int64_t chunk = T * blocks / 1024;
  chunk = (chunk + 15) / 16 * 16;
  return (int)(chunk < 32 ? 32 : chunk);
}
int64_t route_chunks(int64_t T, int64_t K) { return (T + route_chunk(T, K) - 1) / route_chunk(T, K); }

template <int kRouters>
void route_backward(const RouteBackwardArgs& s, bool stream_past, dim3 grid, hipStream_t stream) {
  if (stream_past)
    hipLaunchKernelGGL((route_backward_kernel<kRouters, true>), grid, dim3(256), 0, stream, s);
  else
    hipLaunchKernelGGL((route_backward_kernel<kRouters, false>), grid, dim3(256), 0, stream, s);
}
}  // namespace

// No call of fewer tokens takes more: T / chunk is at most 33 / 32 of 1024 / blocks, as chunk is at least 32 and at least the
// whole part of T blocks / 1024.
size_t route_backward_workspace_bytes(int64_t T, int64_t K, int n, int P) {
  const int64_t blocks = (K + kRouteColumns - 1) / kRouteColumns;
  const int64_t by_length = (T + 31) / 32, by_split = (33 * 32 + blocks - 1) / blocks, chunks = by_length < by_split ? by_length : by_split;
  return chunks > 1 ? (size_t)(chunks * n * P * (K + 1) * 4) + 256 : 256;
}

mbq_status launch_route_backward(const RouteBackwardCall& c, hipStream_t stream) {
  if (c.T == 0) {  // no pointer but the sums' need be valid
    ZeroList zl[2] = {};
    for (int p = 0; p < c.n; ++p) {
      zl[0].p[p] = c.dWr[p];
      zl[0].n[p] = c.P * c.K;
      zl[1].p[p] = c.dbr[p];
      zl[1].n[p] = c.P;
    }
    const mbq_status st = c.dWr[0] ? launch_zero_outputs(zl[0], stream) : MBQ_OK;
    return st == MBQ_OK && c.dbr[0] ? launch_zero_outputs(zl[1], stream) : st;
  }
  if (!c.dX && !c.dWr[0] && !c.dbr[0]) return MBQ_OK;
  RouteBackwardArgs s = {};
  s.c = c;
  s.chunk = route_chunk(c.T, c.K);
  const int64_t chunks = route_chunks(c.T, c.K);
  if (chunks > 1 && (c.dWr[0] || c.dbr[0])) {
    s.partial = reinterpret_cast<float*>(c.ws);
    s.partial_b = s.partial + chunks * c.n * c.P * c.K;
  }
  const bool stream_past = c.T * c.K * 4 > (32 << 20);  // more than the L2 caches hold: see mbq_lora.hip
  const dim3 grid((unsigned)((c.K + kRouteColumns - 1) / kRouteColumns), (unsigned)chunks);
  switch (c.n) {
    case 1: route_backward<1>(s, stream_past, grid, stream); break;
    case 2: route_backward<2>(s, stream_past, grid, stream); break;
    case 3: route_backward<3>(s, stream_past, grid, stream); break;
    default: route_backward<4>(s, stream_past, grid, stream); break;
  }
  if (s.partial) {
    const int64_t values = (int64_t)c.n * c.P * (c.K + 1);
    hipLaunchKernelGGL(route_join_kernel, dim3((unsigned)((values + 255) / 256)), dim3(256), 0, stream, s, (int)chunks);
  }
  return hip_status(hipGetLastError(), "route gradients' launch");
}

}  // namespace mbq

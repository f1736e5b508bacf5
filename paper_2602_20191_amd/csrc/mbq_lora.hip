// Low-rank adapters of many requests at once beside the shared projections, forward and backward.
#include "mbq_bf16_codes.h"
#include "mbq_lora.h"

namespace mbq {

namespace {

__device__ __forceinline__ float bf16_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float low_bf16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high_bf16(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
__device__ __forceinline__ int own_rank(const int32_t* ranks, int a, int r) {
  if (!ranks) return r;
  const int own = ranks[a];
  return own < 0 ? 0 : (own > r ? r : own);
}

// fp32 operands of the matrix cores.  A value is cut into three bf16 pieces: the nearest bf16, the nearest to the rest, and
// what is left, which bf16 holds, as both subtractions are exact: x = hi + mid + lo to the last bit of fp32 (parts below
// 2^-133 are lost; an infinity comes out as NaN).  mid is at most 2^-8 and lo 2^-17 of the power of two below x, of either
// sign: cutting off instead leaves 2^-7 and 2^-15 of x's sign, and a product of two values without mid lo and lo mid is then
// up to 8 x 2^-24 too small, where this is at most 2^-24 off either way.  Values that would round to infinity start with the
// largest bf16 (and a mid of up to 2^-7).  Two values make a dword of each piece.
struct Pieces {
  uint4 hi, mid, lo;
};
__device__ __forceinline__ uint32_t high_halves(float a, float b) {  // a in the low half
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ uint32_t nearest_pair(float a, float b) {
  typedef float floatx2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, b}, bf16x2));
}
__device__ __forceinline__ void cut_pair(float a, float b, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  const float most = __uint_as_float(0x7F7F0000u);
  hi = nearest_pair(__builtin_amdgcn_fmed3f(a, -most, most), __builtin_amdgcn_fmed3f(b, -most, most));
  a -= low_bf16(hi);
  b -= high_bf16(hi);
  mid = nearest_pair(a, b);
  lo = high_halves(a - low_bf16(mid), b - high_bf16(mid));
}
__device__ __forceinline__ Pieces cut(const float v[8]) {
  Pieces p;
  cut_pair(v[0], v[1], p.hi.x, p.mid.x, p.lo.x);
  cut_pair(v[2], v[3], p.hi.y, p.mid.y, p.lo.y);
  cut_pair(v[4], v[5], p.hi.z, p.mid.z, p.lo.z);
  cut_pair(v[6], v[7], p.hi.w, p.mid.w, p.lo.w);
  return p;
}

// Tiles.  Tokens grouped by adapter are cut, adapter by adapter, into tiles of at most m; the tokens without one are class n.
// Class a gets the tiles from number offsets[a] / m + a on, which is enough for its tokens whatever the groups' sizes and
// leaves at most one tile per class empty, so tile -> class is a search among offsets (63 ways a step) and the number of
// tiles, T / m + n + 1, is known to the host.
struct Tile {
  int a;      // class
  int begin;  // tokens perm[begin .. begin + count - 1]
  int count;  // may be zero
  int first;  // number among the class's tiles
};
__device__ __forceinline__ int clamped(int v, int most) { return v < 0 ? 0 : (v > most ? most : v); }
__device__ __forceinline__ Tile find_tile(const int32_t* __restrict__ offsets, int n, int T, int tile, int m) {
  const int lane = threadIdx.x & 63;
  int lo = 0, span = n + 1;
  while (true) {
    // 63 ways: the lane behind the last class that is asked about has where that class ends
    const int step = (span + 62) / 63, a = lo + lane * step;
    const int off = a <= n ? clamped(offsets[a], T) : T;
    const int reached = max(1, (int)__popcll(__ballot(lane * step < span && off / m + a <= tile)));
    if (step == 1) {
      Tile t;
      t.a = lo + reached - 1;
      const int from = __builtin_amdgcn_readlane(off, reached - 1), end = __builtin_amdgcn_readlane(off, reached);
      t.first = tile - (from / m + t.a);
      t.begin = (int)min(from + (long long)t.first * m, (long long)T);
      t.count = clamped(end - t.begin, m);
      return t;
    }
    lo += (reached - 1) * step;
    span = min(step, span - (reached - 1) * step);
  }
}
__device__ __forceinline__ int token_at(const int32_t* __restrict__ perm, int T, int i) { return clamped(perm[i], T - 1); }
// Neighbouring work items on one XCD (blocks go round the eight of them), so that a pool is read into one L2.
__device__ __forceinline__ int xcd_item(int block, int items) {
  const int per = (items + 7) >> 3;
  return (block >> 3) < per ? (block & 7) * per + (block >> 3) : items;
}
unsigned xcd_blocks(int64_t items) { return (unsigned)((items + 7) / 8 * 8); }

bool wide(const void* p, int64_t columns, int per, int bytes) {
  return columns % per == 0 && (uintptr_t)p % (size_t)bytes == 0;
}
// Accesses of 16 bytes at the alignment of their elements, which the hardware takes (aligned ones cost the same).
typedef floatx4 floatx4_any __attribute__((aligned(4)));
typedef uint32_t uint32x4 __attribute__((ext_vector_type(4)));
typedef uint32x4 uint32x4_any __attribute__((aligned(2)));

}  // namespace

// Stable grouping by adapter: workgroup a counts the tokens of smaller adapters (where a's begin) and then ranks its own by
// ballots.  Workgroup n takes the tokens without one.  Every workgroup reads the whole assignment, which the caches hold
// (4096 tokens of 256 adapters 9 us, 96 of 2000 6.5: a launch, and two passes over the assignment).
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

// ---- up to 64 tokens: every token by itself, on the vector units -----------------------------------------------
// A decode batch reads each request's factors once (r (K + N) values), so it is bound by the latency of two dependent
// launches and then by memory; grouping tokens would save nothing where adapters differ and only cached reads where they do not.
// 64 tokens of 48 adapters, rank 32, 4096 to 2 x 14336: 6.3 and 14.9 us, 100 MB at 4.7 TB/s.
constexpr int64_t kDecodeTokens = 64;
constexpr int kDecodeColumns = 512;  // of a wavefront's pass: 16 bytes a lane

struct DecodeArgs {
  const uint16_t* X;
  const uint16_t *A[MBQ_MAX_GROUP], *B[MBQ_MAX_GROUP];
  const float* base[MBQ_MAX_GROUP];
  float *Y[MBQ_MAX_GROUP], *H[MBQ_MAX_GROUP];
  int64_t N[MBQ_MAX_GROUP];
  int64_t K;
  int T, n, r, parts, part_columns;
  const int32_t *adapter, *ranks;
  const float* scale;
  float* partial;  // [projection][token][part][r]
};

// Part of h[t][.]: grid (parts of K x 16 ranks, tokens, projections), four rows of A a wavefront.
__global__ __launch_bounds__(256) void lora_decode_shrink_kernel(const DecodeArgs d) {
  const int block = blockIdx.x / d.parts, part = blockIdx.x - block * d.parts, t = blockIdx.y, p = blockIdx.z, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int a = d.adapter[t];
  if ((unsigned)a >= (unsigned)d.n) return;
  const int own = own_rank(d.ranks, a, d.r);
  const int begin = part * d.part_columns, end = min((int64_t)begin + d.part_columns, d.K);
  const uint16_t* x = d.X + (int64_t)t * d.K;
  const uint16_t* w = d.A[p] + (int64_t)a * d.r * d.K;
  float* out = d.partial + ((int64_t)(p * d.T + t) * d.parts + part) * d.r;
  const int j0 = 16 * block + wave;
  if (j0 < own) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k = begin + lane * 8; k < end; k += kDecodeColumns) {
      const uint4 xv = *reinterpret_cast<const uint4*>(x + k);
      uint4 wv[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) wv[i] = *reinterpret_cast<const uint4*>(w + (int64_t)min(j0 + 4 * i, own - 1) * d.K + k);
      const uint32_t xs[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t ws[4] = {wv[i].x, wv[i].y, wv[i].z, wv[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[i] += low_bf16(xs[e]) * low_bf16(ws[e]);
          s[i] += high_bf16(xs[e]) * high_bf16(ws[e]);
        }
      }
    }
    // four sums over 64 lanes: two exchanges leave each row to 16 lanes
    const bool upper = lane & 32, odd = lane & 16;
    const float s01 = (upper ? s[1] : s[0]) + __shfl_xor(upper ? s[0] : s[1], 32, 64);
    const float s23 = (upper ? s[3] : s[2]) + __shfl_xor(upper ? s[2] : s[3], 32, 64);
    float sum = (odd ? s23 : s01) + __shfl_xor(odd ? s01 : s23, 16, 64);
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
    const int j = j0 + 4 * ((upper ? 1 : 0) + (odd ? 2 : 0));
    if ((lane & 15) == 0 && j < own) out[j] = sum;
  }
}

// y[t][.] = base + scale sum_j h[j] B[j][.] for 512 columns of a token: four wavefronts take rows of B in turn, up to 16 each
// on their way while h is put together, and are added in LDS.  kWide: eight neighbouring columns a lane; else columns 64
// apart, one value at a time.
template <bool kWide>
__global__ __launch_bounds__(256) void lora_decode_expand_kernel(const DecodeArgs d) {
  constexpr int kAhead = kWide ? 16 : 4, kRow = kDecodeColumns + 4;
  __shared__ float h[MBQ_LORA_MAX_RANK];
  __shared__ __align__(16) float sums[4][kRow];
  const int t = blockIdx.y, p = blockIdx.z, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t N = d.N[p], first = (int64_t)blockIdx.x * kDecodeColumns;
  if (first >= N) return;
  const int a = __builtin_amdgcn_readfirstlane(d.adapter[t]);
  // the two columns that the thread writes
  const int64_t c1 = first + 2 * tid;
  float y[2] = {0.f, 0.f};
  if (d.base[p]) {
    const float* base = d.base[p] + (int64_t)t * N;
    if constexpr (kWide) {
      if (c1 < N) {
        const float2 v = *reinterpret_cast<const float2*>(base + c1);
        y[0] = v.x, y[1] = v.y;
      }
    } else {
      if (c1 < N) y[0] = base[c1];
      if (c1 + 1 < N) y[1] = base[c1 + 1];
    }
  }
  const int own = (unsigned)a < (unsigned)d.n ? own_rank(d.ranks, a, d.r) : 0;
  const uint16_t* w = d.B[p] + (own ? (int64_t)a * d.r * N : 0);
  const int64_t c0 = first + (kWide ? lane * 8 : lane);
  uint4 wv[kAhead];
  const auto load = [&](int j0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (j0 + 4 * i >= own) break;
      const uint16_t* row = w + (int64_t)(j0 + 4 * i) * N;
      if constexpr (kWide) {
        wv[i] = *reinterpret_cast<const uint4*>(row + min(c0, N - 8));
      } else {
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = row[min(c0 + 64 * e, N - 1)];
        wv[i] = uint4{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
      }
    }
  };
  load(wave);
  const float* part = d.partial + (int64_t)(p * d.T + t) * d.parts * d.r;
  const float scale = own ? d.scale[a] : 0.f;
  for (int j = tid; j < d.r; j += 256) {
    float sum = 0.f;
    if (j < own)
      for (int s = 0; s < d.parts; s += 8) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = s + i < d.parts ? part[(s + i) * d.r + j] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[i];
      }
    if (d.H[p] && blockIdx.x == 0) d.H[p][(int64_t)t * d.r + j] = sum;
    h[j] = sum * scale;
  }
  __syncthreads();
  float acc[8] = {};
  for (int j0 = wave; j0 < own; j0 += 4 * kAhead) {
    if (j0 > wave) load(j0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (j0 + 4 * i >= own) break;
      const float hj = h[j0 + 4 * i];
      const uint32_t vs[4] = {wv[i].x, wv[i].y, wv[i].z, wv[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[2 * e] += hj * low_bf16(vs[e]), acc[2 * e + 1] += hj * high_bf16(vs[e]);
    }
  }
  if constexpr (kWide) {
    *reinterpret_cast<float4*>(&sums[wave][8 * lane]) = float4{acc[0], acc[1], acc[2], acc[3]};
    *reinterpret_cast<float4*>(&sums[wave][8 * lane + 4]) = float4{acc[4], acc[5], acc[6], acc[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][lane + 64 * e] = acc[e];
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 2; ++e) y[e] += (sums[0][2 * tid + e] + sums[1][2 * tid + e]) + (sums[2][2 * tid + e] + sums[3][2 * tid + e]);
  float* to = d.Y[p] + (int64_t)t * N;
  if constexpr (kWide) {
    if (c1 < N) *reinterpret_cast<float2*>(to + c1) = float2{y[0], y[1]};
  } else {
    if (c1 < N) to[c1] = y[0];
    if (c1 + 1 < N) to[c1 + 1] = y[1];
  }
}

// Both in one launch, where that costs few bytes: a workgroup forms all of a token's h and the columns of its own.  Every
// workgroup of a token reads its rows of A, the others' from the caches, but a dependent launch (about 4 us) is saved.
// One token at 2048 x 2048, rank 16: 5.3 us; 16 tokens of as many adapters on q, k, v of 4096: 7.2 us (14 MB).
constexpr int kFusedThreads = 512, kFusedColumns = 4 * kFusedThreads;
constexpr int kFusedPieces = 8, kFusedPass = kFusedPieces * kDecodeColumns;  // columns of K whose loads are under way together
template <bool kWide>
__global__ __launch_bounds__(kFusedThreads) void lora_decode_fused_kernel(const DecodeArgs d) {
  constexpr int kWaves = kFusedThreads / 64, kAhead = 16;
  __shared__ float h[MBQ_LORA_MAX_RANK];
  const int t = blockIdx.y, p = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t N = d.N[p];
  if ((int64_t)blockIdx.x * kFusedColumns >= N) return;
  const int64_t c0 = (int64_t)blockIdx.x * kFusedColumns + (kWide ? 4 * tid : tid);
  const auto column = [&](int c) { return c0 + (kWide ? c : kFusedThreads * c); };
  const int a = d.adapter[t];
  const uint16_t* x = d.X + (int64_t)t * d.K;
  uint4 xv[kFusedPieces];
  const auto load_x = [&](int64_t k0) {
#pragma unroll
    for (int i = 0; i < kFusedPieces; ++i) {
      const int64_t k = k0 + i * kDecodeColumns + lane * 8;
      xv[i] = uint4{0, 0, 0, 0};
      if (k < d.K) xv[i] = *reinterpret_cast<const uint4*>(x + k);
    }
  };
  load_x(0);
  floatx4 y = {0.f, 0.f, 0.f, 0.f};
  if (d.base[p]) {
    const float* base = d.base[p] + (int64_t)t * N;
    if constexpr (kWide) {
      if (c0 < N) y = *reinterpret_cast<const floatx4*>(base + c0);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (column(c) < N) y[c] = base[column(c)];
    }
  }
  const bool some = (unsigned)a < (unsigned)d.n;
  const int own = some ? own_rank(d.ranks, a, d.r) : 0;
  const float scale = some ? d.scale[a] : 0.f;
  const uint16_t* w = d.B[p] + (some ? (int64_t)a * d.r * N : 0);
  uint2 wv[kAhead];
  const auto load_w = [&](int j0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint16_t* row = w + (int64_t)min(j0 + i, own - 1) * N;
      if constexpr (kWide) {
        wv[i] = *reinterpret_cast<const uint2*>(row + min(c0, N - 4));
      } else {
        wv[i].x = row[min(column(0), N - 1)] | (uint32_t)row[min(column(1), N - 1)] << 16;
        wv[i].y = row[min(column(2), N - 1)] | (uint32_t)row[min(column(3), N - 1)] << 16;
      }
    }
  };
  if (own) load_w(0);
  if (own < d.r && d.H[p] && blockIdx.x == 0)
    for (int j = own + tid; j < d.r; j += kFusedThreads) d.H[p][(int64_t)t * d.r + j] = 0.f;
  for (int j0 = 2 * wave; j0 < own; j0 += 2 * kWaves) {
    const uint16_t* rows = d.A[p] + ((int64_t)a * d.r + j0) * d.K;
    const int64_t next = j0 + 1 < own ? d.K : 0;
    float s[2] = {0.f, 0.f};
    for (int64_t k0 = 0; k0 < d.K; k0 += kFusedPass) {
      if (d.K > kFusedPass) load_x(k0);
      uint4 r[2][kFusedPieces];
#pragma unroll
      for (int i = 0; i < kFusedPieces; ++i) {
        const int64_t k = min(k0 + i * kDecodeColumns + lane * 8, d.K - 8);  // (x is zero behind the last column)
        r[0][i] = *reinterpret_cast<const uint4*>(rows + k);
        r[1][i] = *reinterpret_cast<const uint4*>(rows + next + k);
      }
#pragma unroll
      for (int i = 0; i < kFusedPieces; ++i) {
        const bool there = k0 + i * kDecodeColumns + lane * 8 < d.K;
        const uint32_t xs[4] = {xv[i].x, xv[i].y, xv[i].z, xv[i].w};
#pragma unroll
        for (int o = 0; o < 2; ++o) {
          const uint32_t ws[4] = {r[o][i].x, r[o][i].y, r[o][i].z, r[o][i].w};
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sum += low_bf16(xs[e]) * low_bf16(ws[e]);
            sum += high_bf16(xs[e]) * high_bf16(ws[e]);
          }
          s[o] += there ? sum : 0.f;
        }
      }
    }
    const bool upper = lane & 32;
    float sum = (upper ? s[1] : s[0]) + __shfl_xor(upper ? s[0] : s[1], 32, 64);
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
    const int j = j0 + (upper ? 1 : 0);
    if ((lane & 31) == 0 && j < own) {
      if (d.H[p] && blockIdx.x == 0) d.H[p][(int64_t)t * d.r + j] = sum;
      h[j] = sum * scale;
    }
  }
  __syncthreads();
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < own; j0 += kAhead) {
    if (j0) load_w(j0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float hj = j0 + i < own ? h[j0 + i] : 0.f;
      acc[0] += hj * low_bf16(wv[i].x), acc[1] += hj * high_bf16(wv[i].x);
      acc[2] += hj * low_bf16(wv[i].y), acc[3] += hj * high_bf16(wv[i].y);
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) y[c] += acc[c];
  float* to = d.Y[p] + (int64_t)t * N;
  if constexpr (kWide) {
    if (c0 < N) *reinterpret_cast<floatx4*>(to + c0) = y;
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (column(c) < N) to[column(c)] = y[c];
  }
}

// ---- beyond: tiles of 32 tokens of one adapter, on the matrix cores ---------------------------------------------
constexpr int kTile = 32;
constexpr int kWaves = 4;

// What the kernels have in common: the assignment, and h as it lies between them: partial[part][unit][place][16], unit = 16
// ranks of a projection (projection-major), place = where perm has the token.
struct TileArgs {
  int T, n, r, rt, units, parts_log2, tiles;  // rt: units of a projection
  const int32_t *adapter, *perm, *offsets, *ranks;  // adapter: null unless tiles are numbered by places
  const float* scale;
  float* partial;
};
// In the forward pass, where the pool has more adapters than the call has tokens, the tiles are numbered by the places of
// their first tokens instead: T numbers, not T / 32 + n + 1 (96 tokens, 2048 x 2048, rank 16 of 2000 adapters: 46.5 -> 11.8 us; 512 tokens on q,
// k, v of 4096, 1000 adapters: 276 -> 199).
__device__ __forceinline__ Tile tile_of(const TileArgs& t, int tile) {
  if (!t.adapter) return find_tile(t.offsets, t.n, t.T, tile, kTile);
  const unsigned id = (unsigned)t.adapter[token_at(t.perm, t.T, tile)];
  Tile at;
  at.a = id < (unsigned)t.n ? (int)id : t.n;
  const int off = clamped(t.offsets[at.a], t.T), end = at.a < t.n ? clamped(t.offsets[at.a + 1], t.T) : t.T;
  at.begin = tile;
  at.first = (tile - off) / kTile;
  at.count = tile >= off && (tile - off) % kTile == 0 ? clamped(end - tile, kTile) : 0;
  return at;
}

// Between a wavefront's LDS stores and its reads of what other lanes stored, either way round.  The hardware takes a wavefront's
// LDS accesses in their order, so this is no instruction; it keeps the compiler, which sees one lane's addresses, from changing it.
__device__ __forceinline__ void wavefront_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

struct ShrinkArgs {
  TileArgs t;
  const void* x[MBQ_MAX_GROUP];  // one for all (forward) or one per projection
  const uint16_t* w[MBQ_MAX_GROUP];
  int64_t L[MBQ_MAX_GROUP];  // columns
  int share[MBQ_MAX_GROUP], extra[MBQ_MAX_GROUP];  // stages of a wavefront, one more for the first `extra` of them
  int rt_inverse;                                  // 2^16 / rt, rounded up: units are few
  bool shared;                                     // one x
};

// Part of h = x w^T for a tile: the tokens' rows are the one operand, 16 ranks of the adapter the other.  A wavefront stages 64
// columns of its rows through LDS of its own (no barrier), since the operands' lane order (a row a lane) would make every
// 16 bytes of a load a request of its own: reading x and w straight into the operands took 40 us for q, k, v of a 70B-shaped
// block at 4096 tokens.  The 16-byte pieces of a row lie in LDS at their number xor the row's, which spreads both accesses over the
// banks.  Four wavefronts and `parts` workgroups share the columns; x is read once for up to kUnits units (the projections
// that share it).  Bound by reading x: 4096 tokens of 8192 columns, 3 x 16 ranks 19 us, 3.6 TB/s; in fp32 (the gradient's g) 2048
// tokens of 3 x 4096 columns 24 us, 4.2 TB/s.
template <typename In, int kUnits>
__global__ __launch_bounds__(256) void lora_shrink_kernel(const ShrinkArgs s) {
  constexpr bool kExact = sizeof(In) == 2;
  constexpr int kPer = 16 / (int)sizeof(In);     // columns of a 16-byte piece of x
  constexpr int kCols = 64, kXPieces = kCols / kPer, kWPieces = kCols / 8;
  constexpr int kXRows = 64 / kXPieces, kWRows = 64 / kWPieces;  // rows of a load of the wavefront
  constexpr int kXLoads = kTile / kXRows, kWLoads = kUnits * 16 / kWRows;
  constexpr int kXBytes = kTile * kXPieces * 16, kWBytes = kUnits * 16 * kWPieces * 16;
  __shared__ __align__(16) char lds[kWaves * (kXBytes + kWBytes)];
  static_assert(sizeof(lds) >= kWaves * kUnits * 8 * 64 * 4, "the sums are joined in the same LDS");
  // the tiles of tokens without an adapter come last: where there are many tiles, the others are dealt out evenly
  const int bare = s.t.tiles < 64 ? 0 : clamped(s.t.offsets[s.t.n], s.t.T);
  const int tiles = s.t.tiles < 64 ? s.t.tiles : s.t.adapter ? bare : bare / kTile + s.t.n;
  const int item = xcd_item(blockIdx.x, tiles << s.t.parts_log2);
  const int tile = item >> s.t.parts_log2, part = item & ((1 << s.t.parts_log2) - 1);
  if (tile >= tiles) return;
  const int source = blockIdx.y, chunk = blockIdx.z;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4;
  const Tile at = tile_of(s.t, tile);
  if (at.a >= s.t.n || at.count == 0) return;
  const int own = own_rank(s.t.ranks, at.a, s.t.r);
  if (own == 0) return;
  const int most = s.shared ? s.t.units : s.t.rt;  // units of this source
  const int unit0 = chunk * kUnits;
  const int64_t L = s.L[source];
  char* const xs = lds + wave * (kXBytes + kWBytes);
  char* const ws = xs + kXBytes;
  const auto x_row = [&](int row) {
    return static_cast<const In*>(s.x[source]) + (int64_t)token_at(s.t.perm, s.t.T, at.begin + min(row, at.count - 1)) * L;
  };
  const auto w_row = [&](int row) {  // rows that are not there repeat others, whose sums are not used
    const int unit = min(unit0 + (row >> 4), most - 1), p = s.shared ? unit * s.rt_inverse >> 16 : source;
    return s.w[p] + ((int64_t)at.a * s.t.r + min(16 * (s.shared ? unit - p * s.t.rt : unit) + (row & 15), own - 1)) * L;
  };
  const auto x_at = [&](int row, int piece) { return xs + (row * kXPieces + (piece ^ (row & (kXPieces - 1)))) * 16; };
  const auto w_at = [&](int row, int piece) { return ws + (row * kWPieces + (piece ^ (row & (kWPieces - 1)))) * 16; };

  const int xc = lane % kXPieces * kPer, wc = lane % kWPieces * 8;  // the lane's columns of a stage
  const In* x[kXLoads];
  const uint16_t* w[kWLoads];
#pragma unroll
  for (int i = 0; i < kXLoads; ++i) x[i] = x_row(i * kXRows + lane / kXPieces) + xc;
#pragma unroll
  for (int i = 0; i < kWLoads; ++i) w[i] = w_row(i * kWRows + lane / kWPieces) + wc;
  uint4 xv[kXLoads], wv[kWLoads];
  const auto load = [&](int64_t k) {
    if (k + kCols <= L) {
#pragma unroll
      for (int i = 0; i < kXLoads; ++i) {
        if constexpr (kExact)
          xv[i] = *reinterpret_cast<const uint4*>(x[i] + k);
        else
          xv[i] = __builtin_bit_cast(uint4, *reinterpret_cast<const floatx4_any*>(x[i] + k));
      }
#pragma unroll
      for (int i = 0; i < kWLoads; ++i) {
        if constexpr (kExact)
          wv[i] = *reinterpret_cast<const uint4*>(w[i] + k);
        else
          wv[i] = __builtin_bit_cast(uint4, *reinterpret_cast<const uint32x4_any*>(w[i] + k));
      }
    } else {  // the last columns of an L that is no multiple of 64; the branch also keeps the loads ahead of the products: without it
              // (where the forward's L, a multiple of 128, needs none) they sank behind them and 18.6 us were 37
#pragma unroll
      for (int i = 0; i < kXLoads; ++i) {
        In v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[e] = k + xc + e < L ? x[i][k + e] : In(0);
        xv[i] = __builtin_bit_cast(uint4, v);
      }
#pragma unroll
      for (int i = 0; i < kWLoads; ++i) {
        uint16_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + wc + e < L ? w[i][k + e] : uint16_t(0);
        wv[i] = __builtin_bit_cast(uint4, v);
      }
    }
  };
  const auto store = [&]() {
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) *reinterpret_cast<uint4*>(x_at(i * kXRows + lane / kXPieces, lane % kXPieces)) = xv[i];
#pragma unroll
    for (int i = 0; i < kWLoads; ++i) *reinterpret_cast<uint4*>(w_at(i * kWRows + lane / kWPieces, lane % kWPieces)) = wv[i];
  };
  floatx4 acc[kUnits][2];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) acc[u][0] = acc[u][1] = floatx4{0.f, 0.f, 0.f, 0.f};
  const auto use = [&]() {
#pragma unroll
    for (int k = 0; k < kCols / 32; ++k) {
      uint4 wf[kUnits];
#pragma unroll
      for (int u = 0; u < kUnits; ++u) wf[u] = *reinterpret_cast<const uint4*>(w_at(16 * u + (lane & 15), 4 * k + q));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = 16 * h + (lane & 15);
        if constexpr (kExact) {
          const uint4 xf = *reinterpret_cast<const uint4*>(x_at(row, 4 * k + q));
#pragma unroll
          for (int u = 0; u < kUnits; ++u) acc[u][h] = bf::mfma(xf, wf[u], acc[u][h]);
        } else {
          const float4 a = *reinterpret_cast<const float4*>(x_at(row, 8 * k + 2 * q));
          const float4 b = *reinterpret_cast<const float4*>(x_at(row, 8 * k + 2 * q + 1));
          const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
          const Pieces pc = cut(v);
#pragma unroll
          for (int u = 0; u < kUnits; ++u) {
            acc[u][h] = bf::mfma(pc.lo, wf[u], acc[u][h]);
            acc[u][h] = bf::mfma(pc.mid, wf[u], acc[u][h]);
            acc[u][h] = bf::mfma(pc.hi, wf[u], acc[u][h]);
          }
        }
      }
    }
  };
  const int share = part * kWaves + wave, first = share * s.share[source] + min(share, s.extra[source]);
  const int64_t k0 = (int64_t)first * kCols, k1 = k0 + (s.share[source] + (share < s.extra[source] ? 1 : 0)) * kCols;
  if (k0 < k1) load(k0);
  for (int64_t k = k0; k < k1; k += kCols) {
    store();
    wavefront_order();
    if (k + kCols < k1) load(k + kCols);
    use();
    wavefront_order();
  }
  __syncthreads();
  float* const red = reinterpret_cast<float*>(lds);  // [wave][value][lane]
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[((wave * kUnits + u) * 8 + h * 4 + i) * 64 + lane] = acc[u][h][i];
  __syncthreads();
#pragma unroll
  for (int e = threadIdx.x; e < kUnits * 128; e += 256) {  // four ranks of a token
    const int u = e >> 7, token = (e >> 2) & 31, j = 4 * (e & 3);
    const int from = ((u * 8 + (token >> 4) * 4 + (token & 3)) * 64) + ((token >> 2) & 3) * 16 + j;
    if (unit0 + u >= most || token >= at.count) continue;
    float4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const float4 v = *reinterpret_cast<const float4*>(red + i * (kUnits * 512) + from);
      sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
    }
    const int unit = (s.shared ? 0 : source * s.t.rt) + unit0 + u;
    *reinterpret_cast<float4*>(s.t.partial + (((int64_t)part * s.t.units + unit) * s.t.T + at.begin + token) * 16 + j) = sum;
  }
}

// Four ranks from j on of the token at a place, summed over the parts (in order, four loads on their way at a time).
__device__ __forceinline__ float4 whole_h(const TileArgs& t, int p, int place, int j) {
  const float* at = t.partial + ((int64_t)(p * t.rt + (j >> 4)) * t.T + place) * 16 + (j & 15);
  const int64_t next = (int64_t)t.units * t.T * 16;
  const int parts = 1 << t.parts_log2;
  float4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < parts; s += 4) {
    float4 v[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (s + i < parts) v[i] = *reinterpret_cast<const float4*>(at + (s + i) * next);
#pragma unroll
    for (int i = 0; i < 4; ++i) sum.x += v[i].x, sum.y += v[i].y, sum.z += v[i].z, sum.w += v[i].w;
  }
  return sum;
}

// What is read and written once and is more than the L2 caches hold goes past them: the reads of the launches that follow
// do not then wait for dirty lines to leave (q, k, v of a 70B-shaped block at 4096 tokens 119 -> 106 us).
template <bool kStream>
__device__ __forceinline__ floatx4 load4(const float* p) {
  if constexpr (kStream) return __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(p));
  return *reinterpret_cast<const floatx4*>(p);
}
template <bool kStream>
__device__ __forceinline__ void store4(float* p, floatx4 v) {
  if constexpr (kStream)
    __builtin_nontemporal_store(v, reinterpret_cast<floatx4*>(p));
  else
    *reinterpret_cast<floatx4*>(p) = v;
}

// Four columns of eight rows, as loaded, into four operands of eight rows each.
__device__ __forceinline__ void turn(const uint2 v[8], uint4 w[4]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint32_t d[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t even = c < 2 ? v[2 * e].x : v[2 * e].y, odd = c < 2 ? v[2 * e + 1].x : v[2 * e + 1].y;
      d[e] = __builtin_amdgcn_perm(odd, even, c & 1 ? 0x07060302u : 0x05040100u);
    }
    w[c] = uint4{d[0], d[1], d[2], d[3]};
  }
}

constexpr int kExpandColumns = 256;  // of a workgroup
struct ExpandArgs {
  TileArgs t;
  const uint16_t* w[MBQ_MAX_GROUP];
  const float* base[MBQ_MAX_GROUP];
  float *y[MBQ_MAX_GROUP], *H[MBQ_MAX_GROUP];
  int64_t L[MBQ_MAX_GROUP];
  int outputs, first[MBQ_MAX_GROUP], blocks;  // blocks of columns: an output's first, of all of them
  bool wide[MBQ_MAX_GROUP];
};

// y = base + scale h w for a tile.  h goes 32 ranks at a time, cut into pieces, through LDS (lane: token, eight ranks); w is turned in registers: a lane loads four columns of eight ranks and pairs ranks up by one byte
// permutation a dword.  kWide: MFMA c of a set of four yields columns 4 (lane mod 16) + c, so that a lane's four results of
// one token are one 16-byte access to base and y; else columns 16 c + lane mod 16.  base, and the next step's h and w, are on
// their way while a step is multiplied.  Bound by reading base and writing y: 4096 tokens, 10240 columns, rank 16 62 us, 5.4 TB/s.
constexpr int kStep = 32, kStride = kStep + 8;
struct ExpandLds {
  uint16_t pieces[2][3][kTile][kStride];
};
__device__ __forceinline__ int expand_output(const ExpandArgs& s, int block_id) {
  const int item = xcd_item(block_id, s.t.tiles * s.blocks), block = item - item / s.blocks * s.blocks;
  int out = 0;
  while (out + 1 < s.outputs && block >= s.first[out + 1]) ++out;
  return out;
}
template <bool kWide, bool kStream>
__device__ __forceinline__ void expand_block(const ExpandArgs& s, int block_id, ExpandLds* lds) {
  const int item = xcd_item(block_id, s.t.tiles * s.blocks);
  if (item >= s.t.tiles * s.blocks) return;
  const int tile = item / s.blocks;
  int block = item - tile * s.blocks, out = 0;
  while (out + 1 < s.outputs && block >= s.first[out + 1]) ++out;
  block -= s.first[out];
  const int64_t L = s.L[out];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane >> 4;
  const Tile at = tile_of(s.t, tile);
  if (at.count == 0) return;
  const bool some = at.a < s.t.n;
  const int own = some ? own_rank(s.t.ranks, at.a, s.t.r) : 0;
  const float scale = some ? s.t.scale[at.a] : 0.f;
  const float* base = s.base[out];
  float* y = s.y[out];
  float* H = block == 0 ? s.H[out] : nullptr;
  const int64_t c0 = (int64_t)block * kExpandColumns + wave * 64 + (lane & 15) * (kWide ? 4 : 1);
  const auto column = [&](int c) { return c0 + (kWide ? c : 16 * c); };
  const int place = at.begin + min(tid >> 3, at.count - 1);  // of the thread's token of h

  int64_t to[2][4];  // a lane's four tokens of either half
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      to[h][i] = (int64_t)token_at(s.t.perm, s.t.T, at.begin + min(16 * h + 4 * q + i, at.count - 1)) * L;
  const auto there = [&](int h, int i) { return 16 * h + 4 * q + i < at.count; };
  floatx4 b[2][4];
  const bool copies = !(own == 0 && y == base);
  if (copies) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        b[h][i] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (!base || !there(h, i)) continue;
        if constexpr (kWide) {
          if (c0 < L) b[h][i] = load4<kStream>(base + to[h][i] + c0);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (column(c) < L) b[h][i][c] = base[to[h][i] + column(c)];
        }
      }
  }
  floatx4 acc[2][4];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[h][c] = floatx4{0.f, 0.f, 0.f, 0.f};

  const int steps = (own + kStep - 1) / kStep;
  float4 hv;
  uint2 wv[8];  // four columns of ranks 8 q ..
  const uint16_t* w = s.w[out] + (some ? (int64_t)at.a * s.t.r * L : 0);
  const auto load = [&](int j0) {
    const int j = j0 + 4 * (tid & 7);
    hv = float4{0.f, 0.f, 0.f, 0.f};
    if (j < own) hv = whole_h(s.t, out, place, j);
#pragma unroll
    for (int e = 0; e < 8; ++e) {  // ranks that are not there meet zeros
      const uint16_t* row = w + (int64_t)min(j0 + 8 * q + e, own - 1) * L;
      if constexpr (kWide) {
        wv[e] = *reinterpret_cast<const uint2*>(row + min(c0, L - 4));
      } else {
        wv[e].x = row[min(column(0), L - 1)] | (uint32_t)row[min(column(1), L - 1)] << 16;
        wv[e].y = row[min(column(2), L - 1)] | (uint32_t)row[min(column(3), L - 1)] << 16;
      }
    }
  };
  if (steps) load(0);
  for (int step = 0; step < steps; ++step) {
    {
      const int j = step * kStep + 4 * (tid & 7);
      float v[4] = {hv.x, hv.y, hv.z, hv.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (j + e >= own) v[e] = 0.f;
        if (H && j + e < s.t.r && (tid >> 3) < at.count)
          H[(int64_t)token_at(s.t.perm, s.t.T, place) * s.t.r + j + e] = v[e];
        v[e] *= scale;
      }
      uint2 pc[3];
      cut_pair(v[0], v[1], pc[2].x, pc[1].x, pc[0].x);
      cut_pair(v[2], v[3], pc[2].y, pc[1].y, pc[0].y);
#pragma unroll
      for (int i = 0; i < 3; ++i) *reinterpret_cast<uint2*>(&lds->pieces[step & 1][i][tid >> 3][4 * (tid & 7)]) = pc[i];
    }
    uint4 w4[4];
    turn(wv, w4);
    if (step + 1 < steps) load((step + 1) * kStep);
    __syncthreads();  // (the other buffer's readers passed the barrier before: two buffers do)
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 av = *reinterpret_cast<const uint4*>(&lds->pieces[step & 1][i][16 * h + (lane & 15)][8 * q]);
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[h][c] = bf::mfma(av, w4[c], acc[h][c]);
      }
  }
  if (H)  // ranks that are not there
    for (int e = tid; e < at.count * s.t.r; e += 256) {
      const int j = e % s.t.r;
      if (j >= steps * kStep) H[(int64_t)token_at(s.t.perm, s.t.T, at.begin + e / s.t.r) * s.t.r + j] = 0.f;
    }
  if (!copies) return;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!there(h, i)) continue;
#pragma unroll
      for (int c = 0; c < 4; ++c) b[h][i][c] += acc[h][c][i];
      if constexpr (kWide) {
        if (c0 < L) store4<kStream>(y + to[h][i] + c0, b[h][i]);
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (column(c) < L) y[to[h][i] + column(c)] = b[h][i][c];
      }
    }
}

template <bool kStream>
__global__ __launch_bounds__(256) void lora_expand_kernel(const ExpandArgs s) {
  __shared__ __align__(16) ExpandLds lds;
  expand_block<true, kStream>(s, blockIdx.x, &lds);
}
// where some output's rows are not 16-byte aligned
__global__ __launch_bounds__(256) void lora_expand_any_kernel(const ExpandArgs s) {
  __shared__ __align__(16) ExpandLds lds;
  if (s.wide[expand_output(s, blockIdx.x)])
    expand_block<true, false>(s, blockIdx.x, &lds);
  else
    expand_block<false, false>(s, blockIdx.x, &lds);
}

// The operands of the gradients' products, cut into pieces and scaled.  By ranks, for the products over tokens:
// fragments[projection][tile][unit][piece][lane] holds 16 bytes, rank 16 unit + lane mod 16 of tokens 8 (lane / 16) .. + 7 of
// the tile.  By tokens, for dX: by_token[tile][projection][32 ranks][piece][half][lane], token 16 half + lane mod 16, ranks
// 8 (lane / 16) .. + 7.  What is not there is zero.  One workgroup per (tile, projection, 32 ranks), of g (summed over its
// parts) and of h as the forward pass left it.  5 us for 2048 tokens, 3 x 16 ranks.
struct FragmentArgs {
  TileArgs t;
  int n, steps;  // projections; 32 ranks each
  const float* h[MBQ_MAX_GROUP];
  uint4 *g_fragments, *h_fragments, *by_token;  // null: not wanted
};
__global__ __launch_bounds__(256) void lora_fragment_kernel(const FragmentArgs s) {
  constexpr int kRow = 36;  // floats of a row in LDS: 16-byte aligned, spread over the banks
  constexpr int kEach = 4;  // tokens of a thread
  __shared__ __align__(16) float v[kTile][kRow];  // [token][rank]
  const int tile = blockIdx.x, p = blockIdx.y, step = blockIdx.z >> 1, tid = threadIdx.x, lane = tid & 63, q = lane >> 4;
  const bool of_h = blockIdx.z & 1;
  if (of_h ? !s.h_fragments : !s.g_fragments && !s.by_token) return;
  const Tile at = find_tile(s.t.offsets, s.t.n, s.t.T, tile, kTile);
  if (at.a >= s.t.n || at.count == 0) return;
  const int own = own_rank(s.t.ranks, at.a, s.t.r);
  const float scale = s.t.scale[at.a];
  const int j = 32 * step + (tid & 31), token0 = kEach * (tid >> 5);
  float sum[kEach] = {};
  if (j < own) {
    if (of_h) {
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        sum[e] = s.h[p][(int64_t)token_at(s.t.perm, s.t.T, at.begin + min(token0 + e, at.count - 1)) * s.t.r + j];
    } else {
      const float* from = s.t.partial + ((int64_t)(p * s.t.rt + (j >> 4)) * s.t.T + at.begin) * 16 + (j & 15);
      const int64_t next = (int64_t)s.t.units * s.t.T * 16;
      const int parts = 1 << s.t.parts_log2;
      for (int i = 0; i < parts; i += 4) {
        float part[4][kEach] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i + k < parts)
#pragma unroll
            for (int e = 0; e < kEach; ++e) part[k][e] = from[(i + k) * next + min(token0 + e, at.count - 1) * 16];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int e = 0; e < kEach; ++e) sum[e] += part[k][e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) v[token0 + e][tid & 31] = j < own && token0 + e < at.count ? sum[e] * scale : 0.f;
  __syncthreads();
  // wavefronts 0 and 1: the units, 2 and 3: the halves of the tokens
  uint4* const fragments = of_h ? s.h_fragments : s.g_fragments;
  const int w = tid >> 6, half = w & 1, unit = 2 * step + half;
  if (w < 2 ? !fragments || unit >= s.t.rt : of_h || !s.by_token) return;
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = w < 2 ? v[8 * q + e][16 * half + (lane & 15)] : v[16 * half + (lane & 15)][8 * q + e];
  const Pieces pc = cut(x);
  if (w < 2) {
    uint4* to = fragments + (((int64_t)p * s.t.tiles + tile) * s.t.rt + unit) * 192 + lane;
    to[0] = pc.hi;
    to[64] = pc.mid;
    to[128] = pc.lo;
  } else {
    uint4* to = s.by_token + (((int64_t)tile * s.n + p) * s.steps + step) * 384 + half * 64 + lane;
    to[0] = pc.lo;
    to[128] = pc.mid;
    to[256] = pc.hi;
  }
}

struct OuterArgs {
  TileArgs t;
  const void* x[MBQ_MAX_GROUP];
  int64_t L[MBQ_MAX_GROUP];
  const uint4* fragments;
  float* d[MBQ_MAX_GROUP];
  float* more[MBQ_MAX_GROUP];  // [chunk][r][L]: chunks of an adapter behind its first
  int chunk;                   // tokens of a chunk, a multiple of kTile * kWaves
  int chunks;                  // of all adapters
  int groups;                  // of kUnits units
  int blocks;                  // of columns, of the widest
  int round;                   // workgroups of a (projection, group)
};
struct OuterWork {
  Tile at;
  int p, unit0, units, block, tile0;  // tile0: the chunk's first tile among all
  int own;                            // the adapter's rank
  float* d;                           // an adapter's first chunk goes to the gradient itself
};
template <int kUnits, int kWidth>
__device__ __forceinline__ bool outer_work(const OuterArgs& s, int block_id, OuterWork& w) {
  const int of = block_id / s.round, item = xcd_item(block_id - of * s.round, s.chunks * s.blocks);
  if (item >= s.chunks * s.blocks) return false;
  // an XCD has a range of columns and all chunks, some of which are empty; a tile's h is small
  w.block = item / s.chunks;
  const int number = item - w.block * s.chunks;
  w.p = of / s.groups;
  w.unit0 = (of - w.p * s.groups) * kUnits;
  w.units = min(kUnits, s.t.rt - w.unit0);
  const int64_t L = s.L[w.p];
  if ((int64_t)w.block * kWidth >= L) return false;
  w.at = find_tile(s.t.offsets, s.t.n, s.t.T, number, s.chunk);
  if (w.at.a >= s.t.n || (w.at.count == 0 && w.at.first > 0)) return false;
  const int off = clamped(s.t.offsets[w.at.a], s.t.T);
  w.tile0 = off / kTile + w.at.a + w.at.first * (s.chunk / kTile);
  w.d = w.at.first == 0 ? s.d[w.p] + (int64_t)w.at.a * s.t.r * L
                        : s.more[w.p] + (int64_t)(off / s.chunk + w.at.first) * s.t.r * L;
  w.own = own_rank(s.t.ranks, w.at.a, s.t.r);
  if (w.own <= 16 * w.unit0) w.at.count = 0;  // zeros
  return true;
}
// A gradient without tokens: four columns a thread.
template <int kUnits, int kWidth>
__device__ __forceinline__ void outer_zeros(const OuterArgs& s, const OuterWork& w, int64_t L) {
  const int64_t c = (int64_t)w.block * kWidth + threadIdx.x % (kWidth / 4) * 4;
  const int end = min(16 * (w.unit0 + w.units), s.t.r);
  for (int j = 16 * w.unit0 + threadIdx.x / (kWidth / 4); j < end; j += 1024 / kWidth) {
    float* to = w.d + (int64_t)j * L + c;
    if (c + 4 <= L)
      *reinterpret_cast<floatx4_any*>(to) = floatx4{0.f, 0.f, 0.f, 0.f};
    else
      for (int e = 0; c + e < L; ++e) to[e] = 0.f;
  }
}
// The tokens of a lane's eight rows of a tile.
struct Rows {
  int token[8];
};
__device__ __forceinline__ Rows rows_of(const TileArgs& t, const Tile& at, int i) {
  Rows r;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    r.token[e] = token_at(t.perm, t.T, at.begin + min(i * kTile + 8 * ((int)(threadIdx.x & 63) >> 4) + e, at.count - 1));
  return r;
}

// dA[a] = g^T x over a chunk's tokens: ranks are the rows, x is turned in registers: a lane loads eight columns of eight tokens'
// rows, and one byte permutation a dword pairs two tokens of a column.  128 columns a workgroup; its four wavefronts take
// tiles in turn, the next tile's x under way, and are added in LDS.
constexpr int kWidthX = 128, kWidthY = 256;  // columns of a workgroup
struct OuterXLds {
  float red[kWaves][32][64];
};
template <int kUnits>
__device__ __forceinline__ void outer_x_block(const OuterArgs& s, int block_id, OuterXLds* lds) {
  constexpr int kWidth = kWidthX;
  auto& red = lds->red;
  OuterWork w;
  if (!outer_work<kUnits, kWidth>(s, block_id, w)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t L = s.L[w.p], c = (int64_t)w.block * kWidth + (lane & 15) * 8;  // (K is a multiple of 128)
  if (w.at.count == 0) {
    outer_zeros<kUnits, kWidth>(s, w, L);
    return;
  }
  const uint16_t* x = static_cast<const uint16_t*>(s.x[w.p]) + c;
  floatx4 acc[kUnits][8];
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[u][e] = floatx4{0.f, 0.f, 0.f, 0.f};
  uint4 v[8], h[kUnits][3];
  const auto load = [&](int i, const Rows& r) {
    const uint4* from = s.fragments + (((int64_t)w.p * s.t.tiles + w.tile0 + i) * s.t.rt + w.unit0) * 192 + lane;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const uint4*>(x + (int64_t)r.token[e] * L);
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int k = 0; k < 3; ++k) h[u][k] = from[(u < w.units ? u : 0) * 192 + k * 64];
  };
  const int tiles = (w.at.count + kTile - 1) / kTile;
  Rows r;
  if (wave < tiles) {
    r = rows_of(s.t, w.at, wave);
    load(wave, r);
    if (wave + kWaves < tiles) r = rows_of(s.t, w.at, wave + kWaves);
  }
  for (int i = wave; i < tiles; i += kWaves) {
    uint4 xv[8], hv[kUnits][3];
#pragma unroll
    for (int col = 0; col < 8; ++col) {
      const auto word = [&](int e) { return col < 2 ? v[e].x : col < 4 ? v[e].y : col < 6 ? v[e].z : v[e].w; };
      uint32_t d[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        d[e] = __builtin_amdgcn_perm(word(2 * e + 1), word(2 * e), col & 1 ? 0x07060302u : 0x05040100u);
      xv[col] = uint4{d[0], d[1], d[2], d[3]};
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int k = 0; k < 3; ++k) hv[u][k] = h[u][k];
    if (i + kWaves < tiles) {
      load(i + kWaves, r);
      if (i + 2 * kWaves < tiles) r = rows_of(s.t, w.at, i + 2 * kWaves);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int k = 2; k >= 0; --k)
#pragma unroll
        for (int col = 0; col < 8; ++col) acc[u][col] = bf::mfma(hv[u][k], xv[col], acc[u][col]);
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (u) __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[wave][e * 4 + i][lane] = acc[u][e][i];
    __syncthreads();
    for (int e = tid; e < 16 * kWidth; e += 256) {
      const int j = e / kWidth, col = e - j * kWidth, value = (col & 7) * 4 + (j & 3), l = (j >> 2) * 16 + (col >> 3);
      const int rank = 16 * (w.unit0 + u) + j;
      if (u < w.units && rank < s.t.r) {  // (beyond the adapter's rank a zero met x, whatever that is)
        const float sum = (red[0][value][l] + red[1][value][l]) + (red[2][value][l] + red[3][value][l]);
        w.d[(int64_t)rank * L + (int64_t)w.block * kWidth + col] = rank < w.own ? sum : 0.f;
      }
    }
  }
}

// dB[a] = h^T dy over a chunk's tokens, the same way: a lane loads four columns of eight tokens' rows, cuts the values into
// pieces as it pairs tokens up.  Of the nine products of pieces six are formed; mid lo, lo mid and lo lo, together at most 2^-24
// of the product and of either sign, half a step of fp32, are left out.  256 columns a workgroup, 64 a wavefront, tile after
// tile; a tile's h is shared through LDS, the next tile's h and dy are under way.
// kWide: columns 4 (lane mod 16) + c, 16-byte accesses; else 16 c + lane mod 16.
template <int kUnits>
struct OuterYLds {
  uint4 hs[2][kUnits * 192];
};
template <int kUnits, bool kWide>
__device__ __forceinline__ void outer_y_block(const OuterArgs& s, int block_id, OuterYLds<kUnits>* lds) {
  constexpr int kWidth = kWidthY, kLoads = (kUnits * 192 + 255) / 256;
  OuterWork w;
  if (!outer_work<kUnits, kWidth>(s, block_id, w)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane >> 4;
  const int64_t L = s.L[w.p], c0 = (int64_t)w.block * kWidth + wave * 64 + (lane & 15) * (kWide ? 4 : 1);
  const auto column = [&](int c) { return c0 + (kWide ? c : 16 * c); };
  if (w.at.count == 0) {
    outer_zeros<kUnits, kWidth>(s, w, L);
    return;
  }
  const float* x = static_cast<const float*>(s.x[w.p]);
  floatx4 acc[kUnits][4];
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[u][e] = floatx4{0.f, 0.f, 0.f, 0.f};
  struct Loads {
    floatx4 v[8];
    uint4 h[kLoads];
  };
  const int tiles = (w.at.count + kTile - 1) / kTile;
  const uint4* const fragments = s.fragments + (((int64_t)w.p * s.t.tiles + w.tile0) * s.t.rt + w.unit0) * 192;
  Rows r;
  // tile i, whose tokens are in r; then the tokens of the next
  const auto load = [&](Loads& l, int i) {
    if (i >= tiles) return;
    const uint4* from = fragments + (int64_t)i * s.t.rt * 192;
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const int e = tid + 256 * k;
      l.h[k] = from[e < w.units * 192 ? e : 0];  // (units that are not there are not written)
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float* row = x + (int64_t)r.token[e] * L;
      if constexpr (kWide) {
        l.v[e] = *reinterpret_cast<const floatx4*>(row + min(c0, L - 4));
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) l.v[e][c] = row[min(column(c), L - 1)];
      }
    }
    if (i + 1 < tiles) r = rows_of(s.t, w.at, i + 1);
  };
  const auto use = [&](Loads& l, int i) {
    auto& hs = lds->hs[i & 1];
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (tid + 256 * k < kUnits * 192) hs[tid + 256 * k] = l.h[k];
    Pieces pc[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float f[8] = {l.v[0][c], l.v[1][c], l.v[2][c], l.v[3][c], l.v[4][c], l.v[5][c], l.v[6][c], l.v[7][c]};
      pc[c] = cut(f);
    }
    load(l, i + 2);
    __syncthreads();  // (the other buffer's readers passed the barrier before: two buffers do)
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const uint4 hi = hs[u * 192 + lane], mid = hs[u * 192 + 64 + lane], lo = hs[u * 192 + 128 + lane];
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[u][c] = bf::mfma(lo, pc[c].hi, acc[u][c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[u][c] = bf::mfma(mid, pc[c].mid, acc[u][c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[u][c] = bf::mfma(hi, pc[c].lo, acc[u][c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[u][c] = bf::mfma(mid, pc[c].hi, acc[u][c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[u][c] = bf::mfma(hi, pc[c].mid, acc[u][c]);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[u][c] = bf::mfma(hi, pc[c].hi, acc[u][c]);
    }
  };
  Loads a, b;
  if (tiles) r = rows_of(s.t, w.at, 0);
  load(a, 0);
  load(b, 1);
  for (int i = 0; i < tiles; i += 2) {
    use(a, i);
    if (i + 1 < tiles) use(b, i + 1);
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (u >= w.units) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = 16 * (w.unit0 + u) + 4 * q + i;
      if (j >= s.t.r) continue;
      float* to = w.d + (int64_t)j * L;
      const bool used = j < w.own;  // (beyond the adapter's rank a zero met dy, whatever that is)
      const floatx4 value = {acc[u][0][i], acc[u][1][i], acc[u][2][i], acc[u][3][i]};
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (column(c) < L) to[column(c)] = used ? value[c] : 0.f;
    }
  }
}

// dX = base + sum over the projections of g A for a tile, 256 columns at a time for `span` of them: as lora_expand_kernel, but
// with g as lora_fragment_kernel left it and the projections' ranks one after the other in the same sums.  The next step's
// operands are under way across the blocks of columns.
struct DxArgs {
  TileArgs t;
  const uint16_t* w[MBQ_MAX_GROUP];
  const float* base;
  float* y;
  int64_t L;
  int blocks, span, n, steps;  // blocks of span * 256 columns; projections; steps of 32 ranks of a projection in by_token
  const uint4* by_token;
};
template <bool kWide, bool kStream>
__device__ __forceinline__ void dx_block(const DxArgs& s, int block_id) {
  const int item = xcd_item(block_id, s.t.tiles * s.blocks);
  if (item >= s.t.tiles * s.blocks) return;
  const int tile = item / s.blocks, block = item - tile * s.blocks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4;
  const Tile at = find_tile(s.t.offsets, s.t.n, s.t.T, tile, kTile);
  if (at.count == 0) return;
  const bool some = at.a < s.t.n;
  const int own = some ? own_rank(s.t.ranks, at.a, s.t.r) : 0;
  if (own == 0 && s.y == s.base) return;
  const int64_t L = s.L;
  int64_t to[2][4];  // a lane's four tokens of either half
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      to[h][i] = (int64_t)token_at(s.t.perm, s.t.T, at.begin + min(16 * h + 4 * q + i, at.count - 1)) * L;
  const auto there = [&](int h, int i) { return 16 * h + 4 * q + i < at.count; };
  int64_t c0 = (int64_t)block * s.span * kExpandColumns + wave * 64 + (lane & 15) * (kWide ? 4 : 1);  // of the next loads
  const auto column = [&](int64_t from, int c) { return from + (kWide ? c : 16 * c); };
  const int blocks = (int)min((int64_t)s.span, (L - (int64_t)block * s.span * kExpandColumns + kExpandColumns - 1) / kExpandColumns);
  const int per = (own + kStep - 1) / kStep, steps = per * s.n;
  floatx4 b[2][4], acc[2][4];
  uint4 hf[6];
  uint2 wv[8];
  const auto load_base = [&](int64_t c) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        b[h][i] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (!s.base || !there(h, i)) continue;
        if constexpr (kWide) {
          if (c < L) b[h][i] = load4<kStream>(s.base + to[h][i] + c);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (column(c, e) < L) b[h][i][e] = s.base[to[h][i] + column(c, e)];
        }
      }
  };
  const auto load = [&](int64_t c, int p, int j0) {
    const uint4* from = s.by_token + (((int64_t)tile * s.n + p) * s.steps + j0 / kStep) * 384 + lane;
#pragma unroll
    for (int i = 0; i < 6; ++i) hf[i] = from[64 * i];
    const uint16_t* w = s.w[p] + (int64_t)at.a * s.t.r * L;
#pragma unroll
    for (int e = 0; e < 8; ++e) {  // ranks that are not there meet zeros
      const uint16_t* row = w + (int64_t)min(j0 + 8 * q + e, own - 1) * L;
      if constexpr (kWide) {
        wv[e] = *reinterpret_cast<const uint2*>(row + min(c, L - 4));
      } else {
        wv[e].x = row[min(column(c, 0), L - 1)] | (uint32_t)row[min(column(c, 1), L - 1)] << 16;
        wv[e].y = row[min(column(c, 2), L - 1)] | (uint32_t)row[min(column(c, 3), L - 1)] << 16;
      }
    }
  };
  int64_t c = c0;  // of the sums
  load_base(c);
  if (steps) load(c0, 0, 0);
  int p = 0, j0 = 0;  // of the next loads
  for (int k = 0; k < blocks; ++k) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[h][e] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int step = 0; step < steps; ++step) {
      uint4 a[6], w4[4];
#pragma unroll
      for (int i = 0; i < 6; ++i) a[i] = hf[i];
      turn(wv, w4);
      j0 += kStep;
      if (j0 >= own) {
        j0 = 0;
        if (++p == s.n) p = 0, c0 += kExpandColumns;
      }
      if (step + 1 < steps || k + 1 < blocks) load(c0, p, j0);
#pragma unroll
      for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[h][e] = bf::mfma(a[2 * i + h], w4[e], acc[h][e]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!there(h, i)) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) b[h][i][e] += acc[h][e][i];
        if constexpr (kWide) {
          if (c < L) store4<kStream>(s.y + to[h][i] + c, b[h][i]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (column(c, e) < L) s.y[to[h][i] + column(c, e)] = b[h][i][e];
        }
      }
    c += kExpandColumns;
    if (k + 1 < blocks) load_base(c);
  }
}

// What comes after g and h are cut: dB, dA and dX in one launch, the longest first.  Each alone leaves much of the chip
// waiting for its own loads.  2048 tokens, 3 x 4096 of 4096, rank 16 45 us, 183 MB past the L2 caches; 4096 tokens, 2 x 11008,
// rank 64 146 us, 643 MB at 4.4 TB/s: dY, which g's launch has read already, and X once for each projection and 32 ranks of dA.
// The vector units are busy 41 % of that time and the matrix units 29 % (dB: six instructions a pair of operands, and cutting dY),
// and two wavefronts a SIMD do not hide all of it behind the loads.
struct GradientArgs {
  OuterArgs y, x;
  DxArgs dx;
  int y_blocks, x_blocks;  // workgroups of dB, of dA; the others do dX
};
template <int kUnits, bool kWideY, bool kWideX, bool kStream>
__global__ __launch_bounds__(256, 2) void lora_gradient_kernel(const GradientArgs s) {
  constexpr int kUnitsX = kUnits < 2 ? kUnits : 2;
  __shared__ __align__(16) union {
    OuterYLds<kUnits> y;
    OuterXLds x;
  } lds;
  const int block = blockIdx.x;
  if (block < s.y_blocks)
    outer_y_block<kUnits, kWideY>(s.y, block, &lds.y);
  else if (block < s.y_blocks + s.x_blocks)
    outer_x_block<kUnitsX>(s.x, block - s.y_blocks, &lds.x);
  else
    dx_block<kWideX, kStream>(s.dx, block - s.y_blocks - s.x_blocks);
}

// d[a] += the chunks behind an adapter's first, in order.  7.5 us for 8 adapters of 3 x (4096 + 4096) columns, rank 16.
struct JoinArgs {
  int T;
  int chunk[2 * MBQ_MAX_GROUP];
  const int32_t* offsets;
  float* d[2 * MBQ_MAX_GROUP];
  const float* more[2 * MBQ_MAX_GROUP];
  int64_t values[2 * MBQ_MAX_GROUP];  // r L
};
__global__ __launch_bounds__(256) void lora_join_kernel(const JoinArgs s) {
  const int a = blockIdx.x, k = blockIdx.z, chunk = s.chunk[k];
  const int off = clamped(s.offsets[a], s.T), end = clamped(s.offsets[a + 1], s.T);
  const int chunks = end > off ? (end - off - 1) / chunk : 0;  // behind the first
  if (chunks == 0) return;
  const int64_t values = s.values[k];
  float* d = s.d[k];
  const float* more = s.more[k] + (int64_t)(off / chunk) * values;
  for (int64_t i = (int64_t)blockIdx.y * 256 + threadIdx.x; i < values; i += (int64_t)gridDim.y * 256) {
    float sum = d[a * values + i];
    int c = 1;
    for (; c + 3 <= chunks; c += 4) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = more[(c + e) * values + i];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += v[e];
    }
    for (; c <= chunks; ++c) sum += more[c * values + i];
    d[a * values + i] = sum;
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------
namespace {

constexpr int64_t kCacheBytes = 32 << 20;  // the eight L2 caches
// Workgroups of 256 threads in a launch: fewer than 2^32 threads, some left for rounding up to the eight XCDs.
constexpr int64_t kMostBlocks = ((int64_t)1 << 24) - 1024;

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

TileArgs tile_args(const LoraCall& c) {
  TileArgs t = {};
  t.T = (int)c.T;
  t.n = (int)c.adapters;
  t.r = c.r;
  t.rt = (c.r + 15) / 16;
  t.units = t.rt * c.n;
  t.tiles = (int)(c.T / kTile + c.adapters + 1);
  t.perm = c.perm;
  t.offsets = c.offsets;
  t.ranks = c.ranks;
  t.scale = c.scale;
  return t;
}
// Parts along the columns (their log2): about two workgroups a compute unit at the tiles that hold tokens, and at least a
// stage of 64 columns per wavefront.
constexpr int kMostPartsLog2 = 4, kShrinkWorkgroups = 384;
int shrink_parts_log2(int64_t T, int64_t L) {
  const int64_t tiles = up(T, kTile) / kTile;
  int parts = 0;
  while (parts < kMostPartsLog2 && (tiles << parts) < kShrinkWorkgroups && (kWaves * 64 << (parts + 1)) <= L) ++parts;
  return parts;
}
void shrink_shares(ShrinkArgs* s, int source) {
  const int64_t stages = up(s->L[source], 64) / 64, shares = (int64_t)kWaves << s->t.parts_log2;
  s->share[source] = (int)(stages / shares);
  s->extra[source] = (int)(stages % shares);
}
size_t partial_bytes(int64_t T, int units, int parts_log2) { return ((size_t)T * units * 64) << parts_log2; }
// The most of calls of up to T tokens: fewer tokens may have more parts.
size_t most_partial_bytes(int64_t T, int64_t L, int units) {
  size_t most = partial_bytes(T, units, shrink_parts_log2(T, L));
  for (int parts = 1; parts <= kMostPartsLog2; ++parts) {
    const int64_t last = (int64_t)((kShrinkWorkgroups - 1) >> (parts - 1)) * kTile, t = last < T ? last : T;  // with that many
    const size_t bytes = partial_bytes(t, units, shrink_parts_log2(t, L));
    most = bytes > most ? bytes : most;
  }
  return most;
}
int decode_parts(int64_t K, int* columns) {
  const int64_t passes = up(K, kDecodeColumns) / kDecodeColumns, each = (passes + 15) / 16;
  *columns = (int)(each * kDecodeColumns);
  return (int)((passes + each - 1) / each);
}

// One launch instead of two where a token's rows of A are at most 128 KB (4096 columns at rank 16: 16 tokens on three
// projections 8.7 -> 7.5 us, one token 5.9 either way and one launch less for the host; 256 KB: 6.3 -> 7.9 us) and all
// workgroups together read at most 32 MB of them (25 MB: 10.2 -> 9.9 us; 50 MB: 15.4 -> 17.5).
bool decode_fuses(int64_t T, int64_t K, int n, int64_t widest, int r) {
  const int64_t bytes = K * r * 2;
  return bytes <= 128 << 10 && T * n * (up(widest, kFusedColumns) / kFusedColumns) * bytes <= 32 << 20;
}

template <typename In>
void shrink(const ShrinkArgs& s, int sources, hipStream_t stream) {
  const int units = s.shared ? s.t.units : s.t.rt;
  const dim3 grid(xcd_blocks((int64_t)s.t.tiles << s.t.parts_log2), sources, (units + 3) / 4);
  if (units == 1)
    hipLaunchKernelGGL((lora_shrink_kernel<In, 1>), grid, dim3(256), 0, stream, s);
  else if (units == 2)
    hipLaunchKernelGGL((lora_shrink_kernel<In, 2>), grid, dim3(256), 0, stream, s);
  else if (units == 3)
    hipLaunchKernelGGL((lora_shrink_kernel<In, 3>), grid, dim3(256), 0, stream, s);
  else
    hipLaunchKernelGGL((lora_shrink_kernel<In, 4>), grid, dim3(256), 0, stream, s);
}
// -> workgroups
int64_t expand_blocks(ExpandArgs* s, int outputs) {
  s->outputs = outputs;
  for (int i = 0; i < outputs; ++i) {
    s->first[i] = s->blocks;
    s->blocks += (int)(up(s->L[i], kExpandColumns) / kExpandColumns);
  }
  return xcd_blocks((int64_t)s->t.tiles * s->blocks);
}
bool streams_past(int64_t T, int64_t columns) { return T * columns * 4 > kCacheBytes; }

constexpr int kUnitsX = 2, kUnitsY = 4;  // of the kernels above at the largest ranks
template <int kUnits>
void gradients(const GradientArgs& g, bool wy, bool wx, bool streams, unsigned blocks, hipStream_t stream) {
  const dim3 grid(blocks), threads(256);
  if (wy && wx && streams)
    hipLaunchKernelGGL((lora_gradient_kernel<kUnits, true, true, true>), grid, threads, 0, stream, g);
  else if (wy && wx)
    hipLaunchKernelGGL((lora_gradient_kernel<kUnits, true, true, false>), grid, threads, 0, stream, g);
  else if (wy)
    hipLaunchKernelGGL((lora_gradient_kernel<kUnits, true, false, false>), grid, threads, 0, stream, g);
  else if (wx)
    hipLaunchKernelGGL((lora_gradient_kernel<kUnits, false, true, false>), grid, threads, 0, stream, g);
  else
    hipLaunchKernelGGL((lora_gradient_kernel<kUnits, false, false, false>), grid, threads, 0, stream, g);
}
int outer_groups(int rt, int units) { return (rt + units - 1) / units; }

// Tokens of a chunk of the gradients' products: about `wanted` workgroups, but chunks of at least 8 r tokens, whose arrays
// are then small beside what a chunk reads.  dB wants two workgroups a compute unit (one: 4096 tokens to 2 x 11008, rank 32,
// 204 -> 210 us); dA, which takes a third of its time, one up to rank 32 (q, k, v of 4096, 2048 tokens, rank 16: two 83.5
// -> one 78.9 us) and two beyond, where each has more to do (the same at rank 64: one 122, two 115 us).
struct OuterSplit {
  int64_t workgroups, wanted;  // of a chunk; in all
  int r;
};
int outer_chunk(int64_t T, const OuterSplit& s) {
  int64_t chunk = T * s.workgroups / s.wanted;
  if (chunk < 8 * s.r) chunk = 8 * s.r;
  if (chunk > T) chunk = T;
  return (int)up(chunk < 1 ? 1 : chunk, kTile * kWaves);
}
// The most arrays of chunks of a call of up to T tokens: T / chunk is at most 129 / 128 of wanted / workgroups, as chunk is at
// least 128 and at least the whole part of T workgroups / wanted.
int64_t most_chunks(int64_t T, const OuterSplit& s) {
  const int64_t least = up(8 * s.r, kTile * kWaves);
  if (T <= least) return 0;
  const int64_t by_length = up(T, least) / least, by_split = (129 * s.wanted + 128 * s.workgroups - 1) / (128 * s.workgroups);
  return by_length < by_split ? by_length : by_split;
}
int64_t blocks_of(int64_t L, int width) { return up(L, width) / width; }

// most: no call of fewer tokens takes more bytes.
struct BackwardPlan {
  int parts_log2, chunk_x, chunk_y;
  size_t partial, fragments, by_token, more_x, more_y[MBQ_MAX_GROUP];  // bytes; fragments: of g or of h
  size_t most;
};
BackwardPlan backward_plan(int64_t T, int64_t K, int n, const int64_t* N, int64_t adapters, int r) {
  BackwardPlan b = {};
  const int rt = (r + 15) / 16;
  int64_t most = 0, blocks = 0;
  for (int p = 0; p < n; ++p) {
    most = N[p] > most ? N[p] : most;
    blocks += blocks_of(N[p], kWidthY);
  }
  b.parts_log2 = shrink_parts_log2(T, most);
  const OuterSplit x = {blocks_of(K, kWidthX) * n * outer_groups(rt, kUnitsX), rt <= 2 ? 256 : 512, r};
  const OuterSplit y = {blocks * outer_groups(rt, kUnitsY), 512, r};
  b.chunk_x = outer_chunk(T, x);
  b.chunk_y = outer_chunk(T, y);
  const int64_t tiles = T / kTile + adapters + 1;
  b.partial = up((int64_t)partial_bytes(T, rt * n, b.parts_log2), 256);
  b.fragments = (size_t)n * tiles * rt * 192 * sizeof(uint4);
  b.by_token = (size_t)n * tiles * ((r + 31) / 32) * 384 * sizeof(uint4);
  b.more_x = up((int64_t)((T - 1) / b.chunk_x + 1) * r * K * 4, 256);
  b.most = up((int64_t)most_partial_bytes(T, most, rt * n), 256) + 2 * b.fragments + b.by_token;
  for (int p = 0; p < n; ++p) {
    b.more_y[p] = up((int64_t)((T - 1) / b.chunk_y + 1) * r * N[p] * 4, 256);
    b.most += up(most_chunks(T, x) * r * K * 4, 256) + up(most_chunks(T, y) * r * N[p] * 4, 256);
  }
  return b;
}

}  // namespace

bool lora_fits(const LoraCall& c) {
  if (c.T <= kDecodeTokens) return true;
  int64_t blocks = 0;
  for (int p = 0; p < c.n; ++p) blocks += blocks_of(c.N[p], kExpandColumns);
  const int64_t tiles = c.T / kTile + c.adapters + 1;
  return (c.T < tiles ? c.T : tiles) * blocks <= kMostBlocks;
}
bool lora_backward_fits(int64_t T, int64_t K, int n, const int64_t* N, int64_t adapters, int r) {
  if (T == 0) return true;
  const BackwardPlan b = backward_plan(T, K, n, N, adapters, r);
  const int rt = (r + 15) / 16;
  int64_t most = 0;
  for (int p = 0; p < n; ++p) most = N[p] > most ? N[p] : most;
  const int64_t y = (T / b.chunk_y + adapters + 1) * blocks_of(most, kWidthY) * outer_groups(rt, kUnitsY) * n;
  const int64_t x = (T / b.chunk_x + adapters + 1) * blocks_of(K, kWidthX) * outer_groups(rt, kUnitsX) * n;
  return y + x + (T / kTile + adapters + 1) * blocks_of(K, kExpandColumns) <= kMostBlocks;
}

size_t lora_workspace_bytes(int64_t T, int64_t K, int n, int r) {
  int columns;
  const size_t decode = (size_t)(T < kDecodeTokens ? T : kDecodeTokens) * n * r * decode_parts(K, &columns) * 4;
  const size_t tiles = T <= kDecodeTokens ? 0 : most_partial_bytes(T, K, (r + 15) / 16 * n);
  return (decode > tiles ? decode : tiles) + 256;
}

mbq_status launch_lora(const LoraCall& c, hipStream_t stream) {
  if (c.T <= kDecodeTokens) {
    DecodeArgs d = {};
    d.X = c.X;
    d.K = c.K;
    d.T = (int)c.T;
    d.n = (int)c.adapters;
    d.r = c.r;
    d.parts = decode_parts(c.K, &d.part_columns);
    d.adapter = c.adapter;
    d.ranks = c.ranks;
    d.scale = c.scale;
    d.partial = reinterpret_cast<float*>(c.ws);
    int64_t most = 0;
    bool w = true;
    for (int p = 0; p < c.n; ++p) {
      d.A[p] = c.A[p];
      d.B[p] = c.B[p];
      d.N[p] = c.N[p];
      d.base[p] = c.base[p];
      d.Y[p] = c.Y[p];
      d.H[p] = c.H[p];
      most = c.N[p] > most ? c.N[p] : most;
      w = w && wide(c.B[p], c.N[p], 8, 16) && wide(c.Y[p], c.N[p], 4, 16) && wide(c.base[p], c.N[p], 4, 16);
    }
    if (decode_fuses(c.T, c.K, c.n, most, c.r)) {
      const dim3 one((unsigned)(up(most, kFusedColumns) / kFusedColumns), d.T, c.n);
      if (w)
        hipLaunchKernelGGL(lora_decode_fused_kernel<true>, one, dim3(kFusedThreads), 0, stream, d);
      else
        hipLaunchKernelGGL(lora_decode_fused_kernel<false>, one, dim3(kFusedThreads), 0, stream, d);
      return hip_status(hipGetLastError(), "adapter kernel's launch");
    }
    hipLaunchKernelGGL(lora_decode_shrink_kernel, dim3(d.parts * ((c.r + 15) / 16), d.T, c.n), dim3(256), 0, stream, d);
    const dim3 grid((unsigned)(up(most, kDecodeColumns) / kDecodeColumns), d.T, c.n);
    if (w)
      hipLaunchKernelGGL(lora_decode_expand_kernel<true>, grid, dim3(256), 0, stream, d);
    else
      hipLaunchKernelGGL(lora_decode_expand_kernel<false>, grid, dim3(256), 0, stream, d);
    return hip_status(hipGetLastError(), "adapter kernels' launch");
  }
  ShrinkArgs s = {};
  s.t = tile_args(c);
  if (c.T < s.t.tiles) {
    s.t.tiles = (int)c.T;
    s.t.adapter = c.adapter;
  }
  s.t.partial = reinterpret_cast<float*>(c.ws);
  s.t.parts_log2 = shrink_parts_log2(c.T, c.K);
  s.shared = true;
  s.rt_inverse = (65535 + s.t.rt) / s.t.rt;
  s.x[0] = c.X;
  s.L[0] = c.K;
  shrink_shares(&s, 0);
  ExpandArgs e = {};
  bool w = true;
  for (int p = 0; p < c.n; ++p) {
    s.w[p] = c.A[p];
    e.w[p] = c.B[p];
    e.base[p] = c.base[p];
    e.y[p] = c.Y[p];
    e.H[p] = c.H[p];
    e.L[p] = c.N[p];
    e.wide[p] = wide(c.B[p], c.N[p], 4, 8) && wide(c.Y[p], c.N[p], 4, 16) && wide(c.base[p], c.N[p], 4, 16);
    w = w && e.wide[p];
  }
  shrink<uint16_t>(s, 1, stream);
  e.t = s.t;
  const dim3 grid((unsigned)expand_blocks(&e, c.n));
  int64_t columns = 0;
  for (int p = 0; p < c.n; ++p) columns += c.N[p];
  if (!w)
    hipLaunchKernelGGL(lora_expand_any_kernel, grid, dim3(256), 0, stream, e);
  else if (streams_past(c.T, columns))
    hipLaunchKernelGGL(lora_expand_kernel<true>, grid, dim3(256), 0, stream, e);
  else
    hipLaunchKernelGGL(lora_expand_kernel<false>, grid, dim3(256), 0, stream, e);
  return hip_status(hipGetLastError(), "adapter kernels' launch");
}

size_t lora_backward_workspace_bytes(int64_t T, int64_t K, int n, const int64_t* N, int64_t adapters, int r) {
  return T == 0 ? 256 : backward_plan(T, K, n, N, adapters, r).most + 256;
}

mbq_status launch_lora_backward(const LoraCall& c, hipStream_t stream) {
  if (c.T == 0) {
    ZeroList zl[2] = {};
    for (int p = 0; p < c.n; ++p) {
      zl[0].p[p] = c.dA[p];
      zl[0].n[p] = c.adapters * c.r * c.K;
      zl[1].p[p] = c.dB[p];
      zl[1].n[p] = c.adapters * c.r * c.N[p];
    }
    const mbq_status st = c.dA[0] ? launch_zero_outputs(zl[0], stream) : MBQ_OK;
    return st == MBQ_OK && c.dB[0] ? launch_zero_outputs(zl[1], stream) : st;
  }
  const BackwardPlan plan = backward_plan(c.T, c.K, c.n, c.N, c.adapters, c.r);
  ShrinkArgs s = {};
  s.t = tile_args(c);
  s.t.partial = reinterpret_cast<float*>(c.ws);
  s.t.parts_log2 = plan.parts_log2;
  bool wy = true;
  for (int p = 0; p < c.n; ++p) {
    s.x[p] = c.dY[p];
    s.w[p] = c.B[p];
    s.L[p] = c.N[p];
    shrink_shares(&s, p);
    wy = wy && wide(c.dY[p], c.N[p], 4, 16);
  }
  char* const ws = c.ws + plan.partial;
  FragmentArgs f = {};
  f.t = s.t;
  f.n = c.n;
  f.steps = (c.r + 31) / 32;
  f.g_fragments = c.dA[0] ? reinterpret_cast<uint4*>(ws) : nullptr;
  f.h_fragments = c.dB[0] ? reinterpret_cast<uint4*>(ws + plan.fragments) : nullptr;
  f.by_token = c.dX ? reinterpret_cast<uint4*>(ws + 2 * plan.fragments) : nullptr;
  for (int p = 0; p < c.n; ++p) f.h[p] = c.Hin[p];
  if (c.dX || c.dA[0]) shrink<float>(s, c.n, stream);
  if (c.dX || c.dA[0] || c.dB[0])
    hipLaunchKernelGGL(lora_fragment_kernel, dim3(s.t.tiles, c.n, 2 * f.steps), dim3(256), 0, stream, f);
  GradientArgs g = {};
  bool wx = true;
  int64_t dx_blocks = 0;
  if (c.dX) {
    DxArgs& e = g.dx;
    e.t = s.t;
    e.n = c.n;
    e.steps = f.steps;
    e.by_token = f.by_token;
    for (int p = 0; p < c.n; ++p) e.w[p] = c.A[p];
    e.base = c.dx_base;
    e.y = c.dX;
    e.L = c.K;
    // about two workgroups a compute unit at the tiles that hold tokens
    const int64_t span = up(c.T, kTile) / kTile * blocks_of(c.K, kExpandColumns) / 512;
    e.span = (int)(span < 1 ? 1 : span > 8 ? 8 : span);
    e.blocks = (int)blocks_of(c.K, e.span * kExpandColumns);
    dx_blocks = xcd_blocks((int64_t)e.t.tiles * e.blocks);
    wx = wide(c.dX, c.K, 4, 16) && wide(c.dx_base, c.K, 4, 16);
  }
  JoinArgs join = {};
  join.T = (int)c.T;
  join.offsets = c.offsets;
  int joins = 0;  // outputs that have chunks
  int64_t join_blocks = 1;
  char* more = ws + 2 * plan.fragments + plan.by_token;
  for (int side = 0; side < 2; ++side) {  // dA from g and X, dB from h and dY
    OuterArgs& o = side ? g.y : g.x;
    o.t = s.t;
    o.fragments = side ? f.h_fragments : f.g_fragments;
    o.chunk = side ? plan.chunk_y : plan.chunk_x;
    o.chunks = (int)(c.T / o.chunk + c.adapters + 1);
    o.groups = outer_groups(s.t.rt, side ? kUnitsY : kUnitsX);
    int64_t most = 0;
    for (int p = 0; p < c.n; ++p) {
      o.x[p] = side ? (const void*)c.dY[p] : c.X;
      o.L[p] = side ? c.N[p] : c.K;
      o.d[p] = side ? c.dB[p] : c.dA[p];
      most = o.L[p] > most ? o.L[p] : most;
      if (c.T > o.chunk) {
        o.more[p] = reinterpret_cast<float*>(more);
        more += side ? plan.more_y[p] : plan.more_x;
        if (!o.d[p]) continue;
        const int k = joins++;
        join.chunk[k] = o.chunk;
        join.d[k] = o.d[p];
        join.more[k] = o.more[p];
        join.values[k] = (int64_t)c.r * o.L[p];
        const int64_t blocks = up(join.values[k], 1024) / 1024;
        if (blocks > join_blocks) join_blocks = blocks < 4096 ? blocks : 4096;
      }
    }
    if (!o.d[0]) continue;
    o.blocks = (int)blocks_of(most, side ? kWidthY : kWidthX);
    o.round = (int)xcd_blocks((int64_t)o.chunks * o.blocks);
    (side ? g.y_blocks : g.x_blocks) = o.round * o.groups * c.n;
  }
  const unsigned blocks = (unsigned)(g.y_blocks + g.x_blocks + dx_blocks);
  if (blocks == 0) return MBQ_OK;
  if (s.t.rt == 1)
    gradients<1>(g, wy, wx, streams_past(c.T, c.K), blocks, stream);
  else if (s.t.rt == 2)
    gradients<2>(g, wy, wx, streams_past(c.T, c.K), blocks, stream);
  else
    gradients<4>(g, wy, wx, streams_past(c.T, c.K), blocks, stream);
  if (joins)
    hipLaunchKernelGGL(lora_join_kernel, dim3((unsigned)c.adapters, (unsigned)join_blocks, joins), dim3(256), 0, stream, join);
  return hip_status(hipGetLastError(), "adapter gradients' launch");
}

}  // namespace mbq

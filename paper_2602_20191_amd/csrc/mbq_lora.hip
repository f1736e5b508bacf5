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

// fp32 operands of the matrix cores.  A value is cut into three bf16 pieces of eight significant bits each, by cutting off
// and subtracting, both exact: x = hi + mid + lo to the last bit of fp32 (parts below 2^-133 are lost; an infinity comes out
// as NaN).  Two values make a dword of each piece.
struct Pieces {
  uint4 hi, mid, lo;
};
__device__ __forceinline__ uint32_t high_halves(float a, float b) {  // a in the low half
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ void cut_pair(float a, float b, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  const float ah = __uint_as_float(__float_as_uint(a) & 0xFFFF0000u), bh = __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
  hi = high_halves(ah, bh);
  a -= ah;
  b -= bh;
  const float am = __uint_as_float(__float_as_uint(a) & 0xFFFF0000u), bm = __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
  mid = high_halves(am, bm);
  lo = high_halves(a - am, b - bm);
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
// leaves at most one tile per class empty, so tile -> class is a search among offsets (64 ways a step) and the number of
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
  while (span > 1) {
    const int step = (span + 63) >> 6, a = lo + lane * step;
    const bool reached = lane * step < span && clamped(offsets[a], T) / m + a <= tile;
    const int k = __popcll(__ballot(reached));
    if (k > 1) lo += (k - 1) * step;
    span = min(step, span - (k > 1 ? (k - 1) * step : 0));
  }
  Tile t;
  t.a = lo;
  const int off = clamped(offsets[lo], T), end = lo < n ? clamped(offsets[lo + 1], T) : T;
  t.first = tile - (off / m + lo);
  const long long begin = off + (long long)t.first * m;
  t.begin = (int)min(begin, (long long)T);
  t.count = clamped((int)(end - t.begin), m);
  t.a = __builtin_amdgcn_readfirstlane(t.a);
  t.begin = __builtin_amdgcn_readfirstlane(t.begin);
  t.count = __builtin_amdgcn_readfirstlane(t.count);
  t.first = __builtin_amdgcn_readfirstlane(t.first);
  return t;
}
__device__ __forceinline__ int token_at(const int32_t* __restrict__ perm, int T, int i) { return clamped(perm[i], T - 1); }
// Neighbouring work items on one XCD (blocks go round the eight of them), so that a pool is read into one L2.
__device__ __forceinline__ int xcd_item(int items) {
  const int per = (items + 7) >> 3;
  return ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
}
unsigned xcd_blocks(int64_t items) { return (unsigned)((items + 7) / 8 * 8); }

bool wide(const void* p, int64_t columns, int per, int bytes) {
  return columns % per == 0 && (uintptr_t)p % (size_t)bytes == 0;
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

// ---- up to 64 tokens: every token by itself, on the vector units -----------------------------------------------
// A decode batch reads each request's factors once (r (K + N) values), so it is bound by the latency of two dependent
// launches and then by memory; grouping tokens would save nothing where adapters differ and only cached reads where they do not.
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

// Part of h[t][.]: grid (parts of K, tokens, projections), four rows of A at a time per wavefront.
__global__ __launch_bounds__(256) void lora_decode_shrink_kernel(const DecodeArgs d) {
  const int part = blockIdx.x, t = blockIdx.y, p = blockIdx.z, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int a = d.adapter[t];
  if ((unsigned)a >= (unsigned)d.n) return;
  const int own = own_rank(d.ranks, a, d.r);
  const int begin = part * d.part_columns, end = min((int64_t)begin + d.part_columns, d.K);
  const uint16_t* x = d.X + (int64_t)t * d.K;
  const uint16_t* w = d.A[p] + (int64_t)a * d.r * d.K;
  float* out = d.partial + ((int64_t)(p * d.T + t) * d.parts + part) * d.r;
  for (int j0 = wave; j0 < own; j0 += 16) {
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

// y[t][.] = base + scale sum_j h[j] B[j][.]: one wavefront per 512 columns of a token; 16 rows of B are on their way while h
// is put together.  kWide: eight neighbouring columns a lane; else columns 64 apart, one value at a time.
template <bool kWide>
__global__ __launch_bounds__(64) void lora_decode_expand_kernel(const DecodeArgs d) {
  constexpr int kAhead = 16;
  __shared__ float h[MBQ_LORA_MAX_RANK];
  const int t = blockIdx.y, p = blockIdx.z, lane = threadIdx.x;
  const int64_t N = d.N[p];
  const int64_t c0 = (int64_t)blockIdx.x * kDecodeColumns + (kWide ? lane * 8 : lane);
  if ((int64_t)blockIdx.x * kDecodeColumns >= N) return;
  const int a = d.adapter[t];
  const int own = (unsigned)a < (unsigned)d.n ? own_rank(d.ranks, a, d.r) : 0;
  const uint16_t* w = d.B[p] + (own ? (int64_t)a * d.r * N : 0);
  float w8[kAhead][8];
  const auto rows = [&](int j0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint16_t* row = w + (int64_t)min(j0 + i, own - 1) * N;
      if constexpr (kWide) {
        const uint4 v = *reinterpret_cast<const uint4*>(row + min(c0, N - 8));
        const uint32_t vs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) w8[i][2 * e] = low_bf16(vs[e]), w8[i][2 * e + 1] = high_bf16(vs[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) w8[i][e] = bf16_value(row[min(c0 + 64 * e, N - 1)]);
      }
    }
  };
  if (own) rows(0);
  const float* part = d.partial + (int64_t)(p * d.T + t) * d.parts * d.r;
  const float scale = own ? d.scale[a] : 0.f;
  for (int j = lane; j < d.r; j += 64) {
    float sum = 0.f;
    if (j < own)
      for (int s = 0; s < d.parts; ++s) sum += part[s * d.r + j];
    if (d.H[p] && blockIdx.x == 0) d.H[p][(int64_t)t * d.r + j] = sum;
    h[j] = sum * scale;
  }
  __syncthreads();
  float acc[8] = {};
  for (int j0 = 0; j0 < own; j0 += kAhead) {
    if (j0) rows(j0);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const float hj = j0 + i < own ? h[j0 + i] : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += hj * w8[i][e];
    }
  }
  const float* base = d.base[p] ? d.base[p] + (int64_t)t * N : nullptr;
  float* y = d.Y[p] + (int64_t)t * N;
  if constexpr (kWide) {
    if (c0 < N) {
      float4 v[2] = {};
      if (base) v[0] = *reinterpret_cast<const float4*>(base + c0), v[1] = *reinterpret_cast<const float4*>(base + c0 + 4);
      v[0].x += acc[0], v[0].y += acc[1], v[0].z += acc[2], v[0].w += acc[3];
      v[1].x += acc[4], v[1].y += acc[5], v[1].z += acc[6], v[1].w += acc[7];
      *reinterpret_cast<float4*>(y + c0) = v[0];
      *reinterpret_cast<float4*>(y + c0 + 4) = v[1];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c0 + 64 * e < N) y[c0 + 64 * e] = (base ? base[c0 + 64 * e] : 0.f) + acc[e];
  }
}

// ---- beyond: tiles of 32 tokens of one adapter, on the matrix cores ---------------------------------------------
constexpr int kTile = 32;
constexpr int kWaves = 4;

// What the kernels have in common: the assignment, and h as it lies between them: partial[part][unit][place][16], unit = 16
// ranks of a projection (projection-major), place = where perm has the token.
struct TileArgs {
  int T, n, r, rt, units, parts, tiles;  // rt: units of a projection
  const int32_t *perm, *offsets, *ranks;
  const float* scale;
  float* partial;
};

struct ShrinkArgs {
  TileArgs t;
  const void* x[MBQ_MAX_GROUP];  // one for all (forward) or one per projection
  const uint16_t* w[MBQ_MAX_GROUP];
  int64_t L[MBQ_MAX_GROUP];  // columns
  int chunks;                // grid.y = sources * chunks; a chunk is kUnits units
  bool shared;               // one x
};

// Part of h = x w^T for a tile: the tokens' rows are the one operand, as they lie in memory (lane: token, eight columns), 16
// ranks of the adapter the other.  Four wavefronts and `parts` workgroups share the columns; x is read once for up to kUnits
// units (the projections that share it).  Bound by reading x.
template <typename In, int kUnits, bool kWide>
__global__ __launch_bounds__(256) void lora_shrink_kernel(const ShrinkArgs s) {
  __shared__ float red[kWaves][kUnits * 8][64];
  const int item = xcd_item(s.t.tiles * s.t.parts);
  if (item >= s.t.tiles * s.t.parts) return;
  const int tile = item / s.t.parts, part = item - tile * s.t.parts;
  const int source = blockIdx.y / s.chunks, chunk = blockIdx.y - source * s.chunks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4;
  const Tile at = find_tile(s.t.offsets, s.t.n, s.t.T, tile, kTile);
  if (at.a >= s.t.n || at.count == 0) return;
  const int own = own_rank(s.t.ranks, at.a, s.t.r);
  if (own == 0) return;
  const int most = s.shared ? s.t.units : s.t.rt;  // units of this source
  const int unit0 = chunk * kUnits;
  const int64_t L = s.L[source];
  const In* x[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    x[h] = static_cast<const In*>(s.x[source]) +
           (int64_t)token_at(s.t.perm, s.t.T, at.begin + min(16 * h + (lane & 15), at.count - 1)) * L + 8 * q;
  const uint16_t* w[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int unit = min(unit0 + u, most - 1), p = s.shared ? unit / s.t.rt : source;
    const int j = min(16 * (s.shared ? unit - p * s.t.rt : unit) + (lane & 15), own - 1);
    w[u] = s.w[p] + ((int64_t)at.a * s.t.r + j) * L + 8 * q;
  }
  floatx4 acc[kUnits][2];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) acc[u][0] = acc[u][1] = floatx4{0.f, 0.f, 0.f, 0.f};

  // a step is 32 columns from column k on; left: columns of the lane's eight that exist (8 but in the last step)
  constexpr bool kExact = sizeof(In) == 2;
  constexpr int kAhead = kExact ? 4 : 2;  // steps whose loads are on their way together
  struct Step {
    uint4 w[kUnits];
    uint4 x[2][kExact ? 1 : 2];
  };
  const auto load = [&](Step& st, int64_t k, int left) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (kExact) {
        st.x[h][0] = *reinterpret_cast<const uint4*>(x[h] + k);
      } else if constexpr (kWide) {
        st.x[h][0] = st.x[h][1] = uint4{0, 0, 0, 0};
        if (left > 0) {
          st.x[h][0] = *reinterpret_cast<const uint4*>(x[h] + k);
          st.x[h][1] = *reinterpret_cast<const uint4*>(x[h] + k + 4);
        }
      } else {
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < left ? __float_as_uint(x[h][k + e]) : 0u;
        st.x[h][0] = uint4{v[0], v[1], v[2], v[3]};
        st.x[h][1] = uint4{v[4], v[5], v[6], v[7]};
      }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if constexpr (kWide) {
        st.w[u] = *reinterpret_cast<const uint4*>(w[u] + (left > 0 ? k : -8 * q));
      } else {
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = w[u][e < left ? k + e : -8 * q];
        st.w[u] = uint4{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
      }
    }
  };
  const auto use = [&](const Step& st) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if constexpr (kExact) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) acc[u][h] = bf::mfma(st.x[h][0], st.w[u], acc[u][h]);
      } else {
        const uint4 a = st.x[h][0], b = st.x[h][1];
        const float v[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                            __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
        const Pieces pc = cut(v);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
          acc[u][h] = bf::mfma(pc.lo, st.w[u], acc[u][h]);
          acc[u][h] = bf::mfma(pc.mid, st.w[u], acc[u][h]);
          acc[u][h] = bf::mfma(pc.hi, st.w[u], acc[u][h]);
        }
      }
    }
  };
  const int64_t steps = L >> 5, shares = (int64_t)s.t.parts * kWaves, share = (int64_t)part * kWaves + wave;
  int64_t k = (steps * share / shares) << 5;
  const int64_t k1 = (steps * (share + 1) / shares) << 5;
  for (; k + 32 * kAhead <= k1; k += 32 * kAhead) {
    Step st[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(st[i], k + 32 * i, 8);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) use(st[i]);
  }
  for (; k < k1; k += 32) {
    Step st;
    load(st, k, 8);
    use(st);
  }
  if constexpr (!kExact) {  // (K is a multiple of 128)
    if (share == shares - 1 && (L & 31)) {
      Step st;
      load(st, steps << 5, clamped((int)(L & 31) - 8 * q, 8));
      use(st);
    }
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[wave][(u * 2 + h) * 4 + i][lane] = acc[u][h][i];
  __syncthreads();
#pragma unroll
  for (int e = threadIdx.x; e < kUnits * 512; e += 256) {
    const int value = e >> 6, l = e & 63, u = value >> 3, h = (value >> 2) & 1, i = value & 3;
    if (unit0 + u >= most) continue;
    const float sum = (red[0][value][l] + red[1][value][l]) + (red[2][value][l] + red[3][value][l]);
    const int unit = s.shared ? unit0 + u : source * s.t.rt + unit0 + u;
    const int token = 16 * h + 4 * (l >> 4) + i;
    if (token < at.count)
      s.t.partial[(((int64_t)part * s.t.units + unit) * s.t.T + at.begin + token) * 16 + (l & 15)] = sum;
  }
}

// Eight ranks from j on of the token at a place, summed over the parts.
__device__ __forceinline__ void whole_h(const TileArgs& t, int p, int place, int j, float v[8]) {
  const float* at = t.partial + ((int64_t)(p * t.rt + (j >> 4)) * t.T + place) * 16 + (j & 15);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  for (int s = 0; s < t.parts; ++s) {
    const float4 a = *reinterpret_cast<const float4*>(at), b = *reinterpret_cast<const float4*>(at + 4);
    v[0] += a.x, v[1] += a.y, v[2] += a.z, v[3] += a.w, v[4] += b.x, v[5] += b.y, v[6] += b.z, v[7] += b.w;
    at += (int64_t)t.units * t.T * 16;
  }
}

struct ExpandArgs {
  TileArgs t;
  const uint16_t* w[MBQ_MAX_GROUP];
  const float* base[MBQ_MAX_GROUP];
  float *y[MBQ_MAX_GROUP], *H[MBQ_MAX_GROUP];
  int64_t L[MBQ_MAX_GROUP];
  int blocks;   // of columns, of the widest output
  int sources;  // projections that add to one output: 1 (forward: output blockIdx.y), or all (backward: output 0)
};

// y = base + sum over the sources of scale h w for a tile.  h, cut into pieces, goes through LDS (lane: token, eight ranks); w
// is turned in registers: a lane loads four neighbouring columns of eight ranks and pairs ranks up by one byte permutation a
// dword, so MFMA c of a set of four yields columns 4 (lane mod 16) + c, and a lane's four results of one token are one 16-byte
// access to base and y.  Bound by reading base and writing y.
template <int kSub, bool kWide>
__global__ __launch_bounds__(256) void lora_expand_kernel(const ExpandArgs s) {
  constexpr int kStage = 64, kStride = kStage + 8;  // ranks in LDS at a time
  __shared__ __align__(16) uint16_t pieces[3][kTile][kStride];
  __shared__ int rows[kTile];
  const int item = xcd_item(s.t.tiles * s.blocks);
  if (item >= s.t.tiles * s.blocks) return;
  const int tile = item / s.blocks, block = item - tile * s.blocks;
  const int out = s.sources == 1 ? blockIdx.y : 0;
  const int64_t L = s.L[out];
  if ((int64_t)block * (256 * kSub) >= L) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane >> 4;
  const Tile at = find_tile(s.t.offsets, s.t.n, s.t.T, tile, kTile);
  if (at.count == 0) return;
  const bool some = at.a < s.t.n;
  const int own = some ? own_rank(s.t.ranks, at.a, s.t.r) : 0;
  const float scale = some ? s.t.scale[at.a] : 0.f;
  const float* base = s.base[out];
  float* y = s.y[out];
  float* H = block == 0 ? s.H[out] : nullptr;
  if (tid < kTile) rows[tid] = token_at(s.t.perm, s.t.T, at.begin + min(tid, at.count - 1));
  const int64_t c0 = (int64_t)block * (256 * kSub) + wave * (64 * kSub) + 4 * (lane & 15);

  floatx4 acc[kSub][2][4];
#pragma unroll
  for (int b = 0; b < kSub; ++b)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[b][h][c] = floatx4{0.f, 0.f, 0.f, 0.f};

  __syncthreads();
  if (H && own == 0)
    for (int e = tid; e < at.count * s.t.r; e += 256) H[(int64_t)rows[e / s.t.r] * s.t.r + e % s.t.r] = 0.f;
  const int p0 = s.sources == 1 ? out : 0;
  for (int p = p0; p < p0 + s.sources; ++p) {
    const uint16_t* w = s.w[p] + (some ? (int64_t)at.a * s.t.r * L : 0);
    for (int j0 = 0; j0 < (H && own ? s.t.r : own); j0 += kStage) {
      {  // thread: token tid / 8, eight ranks
        const int token = tid >> 3, j = j0 + 8 * (tid & 7);
        float v[8] = {};
        if (j < own && token < at.count) whole_h(s.t, p, at.begin + token, j, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (j + e >= own) v[e] = 0.f;
          if (H && j + e < s.t.r && token < at.count) H[(int64_t)rows[token] * s.t.r + j + e] = v[e];
          v[e] *= scale;
        }
        const Pieces pc = cut(v);
        *reinterpret_cast<uint4*>(&pieces[0][token][8 * (tid & 7)]) = pc.lo;
        *reinterpret_cast<uint4*>(&pieces[1][token][8 * (tid & 7)]) = pc.mid;
        *reinterpret_cast<uint4*>(&pieces[2][token][8 * (tid & 7)]) = pc.hi;
      }
      __syncthreads();
      for (int k = 0; k < kStage && j0 + k < own; k += 32) {
        uint4 hv[3][2];
#pragma unroll
        for (int i = 0; i < 3; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) hv[i][h] = *reinterpret_cast<const uint4*>(&pieces[i][16 * h + (lane & 15)][k + 8 * q]);
#pragma unroll
        for (int b = 0; b < kSub; ++b) {
          const int64_t c = c0 + 64 * b;
          uint2 v[8];  // four columns of ranks j0 + k + 8 q ..; ranks that are not there meet zeros
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint16_t* row = w + (int64_t)min(j0 + k + 8 * q + e, own - 1) * L;
            if constexpr (kWide) {
              v[e] = *reinterpret_cast<const uint2*>(row + min(c, L - 4));
            } else {
              v[e].x = row[min(c, L - 1)] | (uint32_t)row[min(c + 1, L - 1)] << 16;
              v[e].y = row[min(c + 2, L - 1)] | (uint32_t)row[min(c + 3, L - 1)] << 16;
            }
          }
#pragma unroll
          for (int col = 0; col < 4; ++col) {
            uint32_t d[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t even = col < 2 ? v[2 * e].x : v[2 * e].y, odd = col < 2 ? v[2 * e + 1].x : v[2 * e + 1].y;
              d[e] = __builtin_amdgcn_perm(odd, even, col & 1 ? 0x07060302u : 0x05040100u);
            }
            const uint4 wv = {d[0], d[1], d[2], d[3]};
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int i = 0; i < 3; ++i) acc[b][h][col] = bf::mfma(hv[i][h], wv, acc[b][h][col]);
          }
        }
      }
      __syncthreads();
    }
  }
  if (own == 0 && y == base) return;
#pragma unroll
  for (int b = 0; b < kSub; ++b) {
    const int64_t c = c0 + 64 * b;
    if (c >= L) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int token = 16 * h + 4 * q + i;
        if (token >= at.count) continue;
        const int64_t to = (int64_t)rows[token] * L + c;
        if constexpr (kWide) {
          float4 v = base ? *reinterpret_cast<const float4*>(base + to) : float4{0.f, 0.f, 0.f, 0.f};
          v.x += acc[b][h][0][i], v.y += acc[b][h][1][i], v.z += acc[b][h][2][i], v.w += acc[b][h][3][i];
          *reinterpret_cast<float4*>(y + to) = v;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (c + e < L) y[to + e] = (base ? base[to + e] : 0.f) + acc[b][h][e][i];
        }
      }
  }
}

// The operands of the gradients' products over tokens: fragments[projection][tile][unit of the projection][piece][lane] holds
// 16 bytes, rank 16 unit + lane mod 16 of tokens 8 (lane / 16) .. + 7 of the tile; tokens that are not there are zero.  One
// wavefront per (tile, projection): of g (summed over its parts) or of h as the forward pass left it, times the scale.
struct FragmentArgs {
  TileArgs t;
  const float* h[MBQ_MAX_GROUP];  // null: g from t.partial
  uint4* fragments;
};
__global__ __launch_bounds__(64) void lora_fragment_kernel(const FragmentArgs s) {
  const int tile = blockIdx.x, p = blockIdx.y, lane = threadIdx.x, q = lane >> 4;
  const Tile at = find_tile(s.t.offsets, s.t.n, s.t.T, tile, kTile);
  if (at.a >= s.t.n || at.count == 0) return;
  const int own = own_rank(s.t.ranks, at.a, s.t.r);
  const float scale = s.t.scale[at.a];
  for (int unit = 0; unit < s.t.rt; ++unit) {
    const int j = 16 * unit + (lane & 15);
    float v[8] = {};
    if (j < own) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int token = 8 * q + e;
        if (token >= at.count) continue;
        if (s.h[p]) {
          v[e] = s.h[p][(int64_t)token_at(s.t.perm, s.t.T, at.begin + token) * s.t.r + j];
        } else {
          const float* from = s.t.partial + ((int64_t)(p * s.t.rt + unit) * s.t.T + at.begin + token) * 16 + (lane & 15);
          for (int i = 0; i < s.t.parts; ++i) v[e] += from[(int64_t)i * s.t.units * s.t.T * 16];
        }
        v[e] *= scale;
      }
    }
    const Pieces pc = cut(v);
    uint4* to = s.fragments + (((int64_t)p * s.t.tiles + tile) * s.t.rt + unit) * 192 + lane;
    to[0] = pc.hi;
    to[64] = pc.mid;
    to[128] = pc.lo;
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
  int groups;                  // of kUnits units; grid.y = groups * projections
  int blocks;                  // of columns, of the widest
};

// Chunk of d[a] = h^T x over the tokens of a chunk: ranks are the rows, x is turned in registers: a lane loads 16 bytes of
// eight tokens' rows, and a dword of MFMA c's operand pairs two tokens of column c (for bf16 one byte permutation; fp32 values
// are cut into pieces, and of the nine products of pieces the six above 2^-32 are formed).  Four wavefronts take tiles in
// turn and are added in LDS.  An adapter's first chunk goes to d itself.  Bound by reading x.
template <typename In, int kUnits, bool kWide>
__global__ __launch_bounds__(256) void lora_outer_kernel(const OuterArgs s) {
  constexpr int kCols = 16 / (int)sizeof(In), kWidth = 16 * kCols;  // columns of a lane, of the workgroup
  __shared__ float red[kWaves][kCols * 4][64];
  const int chunks = s.t.T / s.chunk + s.t.n + 1;
  const int item = xcd_item(chunks * s.blocks);
  if (item >= chunks * s.blocks) return;
  const int number = item / s.blocks, block = item - number * s.blocks;
  const int p = blockIdx.y / s.groups, unit0 = (blockIdx.y - p * s.groups) * kUnits;
  const int64_t L = s.L[p];
  if ((int64_t)block * kWidth >= L) return;
  const Tile at = find_tile(s.t.offsets, s.t.n, s.t.T, number, s.chunk);
  if (at.a >= s.t.n || (at.count == 0 && at.first > 0)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane >> 4;
  const int64_t c = (int64_t)block * kWidth + (lane & 15) * kCols;
  const In* x = static_cast<const In*>(s.x[p]);
  // the chunk's first tile among all tiles
  const int off = clamped(s.t.offsets[at.a], s.t.T), tile0 = off / kTile + at.a + at.first * (s.chunk / kTile);
  const int units = min(kUnits, s.t.rt - unit0);
  floatx4 acc[kUnits][kCols];
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int e = 0; e < kCols; ++e) acc[u][e] = floatx4{0.f, 0.f, 0.f, 0.f};

  if (own_rank(s.t.ranks, at.a, s.t.r) > 16 * unit0)
    for (int i = wave; i * kTile < at.count; i += kWaves) {
      const uint4* from = s.fragments + (((int64_t)p * s.t.tiles + tile0 + i) * s.t.rt + unit0) * 192 + lane;
      uint4 h[kUnits][3];
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int k = 0; k < 3; ++k) h[u][k] = from[(u < units ? u : 0) * 192 + k * 64];
      uint4 v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const In* row = x + (int64_t)token_at(s.t.perm, s.t.T, at.begin + min(i * kTile + 8 * q + e, at.count - 1)) * L;
        if constexpr (kWide) {
          v[e] = *reinterpret_cast<const uint4*>(row + min(c, L - kCols));
        } else if constexpr (sizeof(In) == 4) {
          const uint32_t* bits = reinterpret_cast<const uint32_t*>(row);
          v[e] = uint4{bits[min(c, L - 1)], bits[min(c + 1, L - 1)], bits[min(c + 2, L - 1)], bits[min(c + 3, L - 1)]};
        }
      }
#pragma unroll
      for (int col = 0; col < kCols; ++col) {
        const auto word = [&](int e) {
          const int k = sizeof(In) == 2 ? col >> 1 : col;
          return k == 0 ? v[e].x : k == 1 ? v[e].y : k == 2 ? v[e].z : v[e].w;
        };
        if constexpr (sizeof(In) == 2) {
          uint32_t d[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            d[e] = __builtin_amdgcn_perm(word(2 * e + 1), word(2 * e), col & 1 ? 0x07060302u : 0x05040100u);
          const uint4 xv = {d[0], d[1], d[2], d[3]};
#pragma unroll
          for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int k = 2; k >= 0; --k) acc[u][col] = bf::mfma(h[u][k], xv, acc[u][col]);
        } else {
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(word(e));
          const Pieces pc = cut(f);
#pragma unroll
          for (int u = 0; u < kUnits; ++u) {
            acc[u][col] = bf::mfma(h[u][2], pc.hi, acc[u][col]);
            acc[u][col] = bf::mfma(h[u][1], pc.mid, acc[u][col]);
            acc[u][col] = bf::mfma(h[u][0], pc.lo, acc[u][col]);
            acc[u][col] = bf::mfma(h[u][1], pc.hi, acc[u][col]);
            acc[u][col] = bf::mfma(h[u][0], pc.mid, acc[u][col]);
            acc[u][col] = bf::mfma(h[u][0], pc.hi, acc[u][col]);
          }
        }
      }
    }
  float* d = at.first == 0 ? s.d[p] + (int64_t)at.a * s.t.r * L
                           : s.more[p] + (int64_t)(off / s.chunk + at.first) * s.t.r * L;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (u) __syncthreads();
#pragma unroll
    for (int e = 0; e < kCols; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[wave][e * 4 + i][lane] = acc[u][e][i];
    __syncthreads();
    for (int e = tid; e < 16 * kWidth; e += 256) {
      const int j = e / kWidth, col = e - j * kWidth, value = (col % kCols) * 4 + (j & 3), l = (j >> 2) * 16 + col / kCols;
      const int64_t to = (int64_t)block * kWidth + col;
      if (u < units && 16 * (unit0 + u) + j < s.t.r && to < L)
        d[(int64_t)(16 * (unit0 + u) + j) * L + to] =
            (red[0][value][l] + red[1][value][l]) + (red[2][value][l] + red[3][value][l]);
    }
  }
}

// d[a] += the chunks behind an adapter's first, in order.
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
  if (chunk == 0) return;
  const int off = clamped(s.offsets[a], s.T), end = clamped(s.offsets[a + 1], s.T);
  const int chunks = end > off ? (end - off - 1) / chunk : 0;  // behind the first
  if (chunks == 0) return;
  const int64_t values = s.values[k];
  float* d = s.d[k];
  for (int64_t i = (int64_t)blockIdx.y * 256 + threadIdx.x; i < values; i += (int64_t)gridDim.y * 256) {
    float sum = d[a * values + i];
    for (int c = 1; c <= chunks; ++c) sum += s.more[k][(int64_t)(off / chunk + c) * values + i];
    d[a * values + i] = sum;
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------
namespace {

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
// Parts along the columns: enough workgroups for two a compute unit at the tiles that hold tokens, and at least two steps of
// 32 columns per wavefront.
int shrink_parts(int64_t T, int64_t L) {
  const int64_t tiles = up(T, kTile) / kTile;
  int64_t parts = (512 + tiles - 1) / tiles;
  parts = parts < L / (kWaves * 64) ? parts : L / (kWaves * 64);
  return (int)(parts < 1 ? 1 : parts > 16 ? 16 : parts);
}
size_t partial_bytes(int64_t T, int units, int parts) { return (size_t)T * units * parts * 64; }
int decode_parts(int64_t K, int* columns) {
  const int64_t passes = up(K, kDecodeColumns) / kDecodeColumns, each = (passes + 15) / 16;
  *columns = (int)(each * kDecodeColumns);
  return (int)((passes + each - 1) / each);
}

template <typename In, bool kWide>
void shrink(const ShrinkArgs& s, int sources, hipStream_t stream) {
  const dim3 grid(xcd_blocks((int64_t)s.t.tiles * s.t.parts), (unsigned)(sources * s.chunks));
  const int units = s.shared ? s.t.units : s.t.rt;
  if (units == 1)
    hipLaunchKernelGGL((lora_shrink_kernel<In, 1, kWide>), grid, dim3(256), 0, stream, s);
  else if (units == 2)
    hipLaunchKernelGGL((lora_shrink_kernel<In, 2, kWide>), grid, dim3(256), 0, stream, s);
  else if (units == 3)
    hipLaunchKernelGGL((lora_shrink_kernel<In, 3, kWide>), grid, dim3(256), 0, stream, s);
  else
    hipLaunchKernelGGL((lora_shrink_kernel<In, 4, kWide>), grid, dim3(256), 0, stream, s);
}
int shrink_chunks(int units) { return (units + 3) / 4; }

void expand(const ExpandArgs& s0, int outputs, bool w, hipStream_t stream) {
  ExpandArgs s = s0;
  int64_t most = 0;
  for (int i = 0; i < outputs; ++i) most = s.L[i] > most ? s.L[i] : most;
  const bool two = w && most * s.t.T >= (int64_t)512 * 512 * kTile;  // 512 columns a workgroup where that leaves two a compute unit
  s.blocks = (int)(up(most, two ? 512 : 256) / (two ? 512 : 256));
  const dim3 grid(xcd_blocks((int64_t)s.t.tiles * s.blocks), (unsigned)outputs);
  if (w && two)
    hipLaunchKernelGGL((lora_expand_kernel<2, true>), grid, dim3(256), 0, stream, s);
  else if (w)
    hipLaunchKernelGGL((lora_expand_kernel<1, true>), grid, dim3(256), 0, stream, s);
  else
    hipLaunchKernelGGL((lora_expand_kernel<1, false>), grid, dim3(256), 0, stream, s);
}

template <typename In, bool kWide>
void outer(const OuterArgs& s, int n, hipStream_t stream) {
  const dim3 grid(xcd_blocks((int64_t)(s.t.T / s.chunk + s.t.n + 1) * s.blocks), (unsigned)(n * s.groups));
  if (s.t.rt == 1)
    hipLaunchKernelGGL((lora_outer_kernel<In, 1, kWide>), grid, dim3(256), 0, stream, s);
  else if (s.t.rt == 2)
    hipLaunchKernelGGL((lora_outer_kernel<In, 2, kWide>), grid, dim3(256), 0, stream, s);
  else
    hipLaunchKernelGGL((lora_outer_kernel<In, 4, kWide>), grid, dim3(256), 0, stream, s);
}

// Tokens of a chunk of the gradients' products: about 1024 workgroups, but chunks of at least 8 r tokens, whose arrays are
// then small beside what a chunk reads.
int outer_chunk(int64_t T, int64_t workgroups, int r) {
  int64_t chunk = T * workgroups / 1024;
  if (chunk < 8 * r) chunk = 8 * r;
  return (int)up(chunk < 1 ? 1 : chunk, kTile * kWaves);
}
int64_t blocks_of(int64_t L, int width) { return up(L, width) / width; }
constexpr int kWidthX = 128, kWidthY = 64;  // columns of a workgroup of lora_outer_kernel: bf16, fp32

struct BackwardPlan {
  int parts, chunk_x, chunk_y;
  size_t partial, fragments, more_x, more_y[MBQ_MAX_GROUP];  // bytes; fragments: of g or of h
  size_t bytes;
};
BackwardPlan backward_plan(int64_t T, int64_t K, int n, const int64_t* N, int64_t adapters, int r) {
  BackwardPlan b = {};
  const int rt = (r + 15) / 16, groups = (rt + 3) / 4;
  int64_t most = 0, blocks = 0;
  for (int p = 0; p < n; ++p) {
    most = N[p] > most ? N[p] : most;
    blocks += blocks_of(N[p], kWidthY);
  }
  b.parts = shrink_parts(T, most);
  b.chunk_x = outer_chunk(T, blocks_of(K, kWidthX) * n * groups, r);
  b.chunk_y = outer_chunk(T, blocks * groups, r);
  b.partial = up((int64_t)partial_bytes(T, rt * n, b.parts), 256);
  b.fragments = (size_t)n * (T / kTile + adapters + 1) * rt * 3072;
  b.more_x = up((int64_t)((T - 1) / b.chunk_x + 1) * r * K * 4, 256);
  b.bytes = b.partial + 2 * b.fragments;
  for (int p = 0; p < n; ++p) {
    b.more_y[p] = up((int64_t)((T - 1) / b.chunk_y + 1) * r * N[p] * 4, 256);
    b.bytes += (T > b.chunk_x ? b.more_x : 0) + (T > b.chunk_y ? b.more_y[p] : 0);
  }
  return b;
}

}  // namespace

size_t lora_workspace_bytes(int64_t T, int64_t K, int n, int r) {
  int columns;
  if (T <= kDecodeTokens) return (size_t)T * n * r * decode_parts(K, &columns) * 4 + 256;
  return partial_bytes(T, (r + 15) / 16 * n, shrink_parts(T, K)) + 256;
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
    hipLaunchKernelGGL(lora_decode_shrink_kernel, dim3(d.parts, d.T, c.n), dim3(256), 0, stream, d);
    const dim3 grid((unsigned)(up(most, kDecodeColumns) / kDecodeColumns), d.T, c.n);
    if (w)
      hipLaunchKernelGGL(lora_decode_expand_kernel<true>, grid, dim3(64), 0, stream, d);
    else
      hipLaunchKernelGGL(lora_decode_expand_kernel<false>, grid, dim3(64), 0, stream, d);
    return hip_status(hipGetLastError(), "adapter kernels' launch");
  }
  ShrinkArgs s = {};
  s.t = tile_args(c);
  s.t.partial = reinterpret_cast<float*>(c.ws);
  s.t.parts = shrink_parts(c.T, c.K);
  s.shared = true;
  s.x[0] = c.X;
  s.L[0] = c.K;
  s.chunks = shrink_chunks(s.t.units);
  ExpandArgs e = {};
  bool w = true;
  for (int p = 0; p < c.n; ++p) {
    s.w[p] = c.A[p];
    e.w[p] = c.B[p];
    e.base[p] = c.base[p];
    e.y[p] = c.Y[p];
    e.H[p] = c.H[p];
    e.L[p] = c.N[p];
    w = w && wide(c.B[p], c.N[p], 4, 8) && wide(c.Y[p], c.N[p], 4, 16) && wide(c.base[p], c.N[p], 4, 16);
  }
  shrink<uint16_t, true>(s, 1, stream);
  e.t = s.t;
  e.sources = 1;
  expand(e, c.n, w, stream);
  return hip_status(hipGetLastError(), "adapter kernels' launch");
}

size_t lora_backward_workspace_bytes(int64_t T, int64_t K, int n, const int64_t* N, int64_t adapters, int r) {
  return T == 0 ? 256 : backward_plan(T, K, n, N, adapters, r).bytes + 256;
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
  s.t.parts = plan.parts;
  s.chunks = shrink_chunks(s.t.rt);
  bool w = true, wy = true;
  for (int p = 0; p < c.n; ++p) {
    s.x[p] = c.dY[p];
    s.w[p] = c.B[p];
    s.L[p] = c.N[p];
    wy = wy && wide(c.dY[p], c.N[p], 4, 16);
    w = w && wide(c.B[p], c.N[p], 8, 16);
  }
  if (c.dX || c.dA[0]) {
    if (w && wy)
      shrink<float, true>(s, c.n, stream);
    else
      shrink<float, false>(s, c.n, stream);
  }
  if (c.dX) {
    ExpandArgs e = {};
    e.t = s.t;
    e.sources = c.n;
    for (int p = 0; p < c.n; ++p) e.w[p] = c.A[p];
    e.base[0] = c.dx_base;
    e.y[0] = c.dX;
    e.L[0] = c.K;
    expand(e, 1, wide(c.dX, c.K, 4, 16) && wide(c.dx_base, c.K, 4, 16), stream);
  }
  char* ws = c.ws + plan.partial;
  JoinArgs join = {};
  join.T = (int)c.T;
  join.offsets = c.offsets;
  bool joins = false;
  for (int side = 0; side < 2; ++side) {  // dA from g and X, dB from h and dY
    char* const fragments = ws;
    ws += plan.fragments;
    if (!(side ? c.dB[0] : c.dA[0])) continue;
    FragmentArgs f = {};
    f.t = s.t;
    f.fragments = reinterpret_cast<uint4*>(fragments);
    for (int p = 0; p < c.n; ++p) f.h[p] = side ? c.Hin[p] : nullptr;
    hipLaunchKernelGGL(lora_fragment_kernel, dim3(s.t.tiles, c.n), dim3(64), 0, stream, f);
    OuterArgs o = {};
    o.t = s.t;
    o.fragments = f.fragments;
    o.chunk = side ? plan.chunk_y : plan.chunk_x;
    o.groups = (s.t.rt + 3) / 4;
    int64_t most = 0;
    for (int p = 0; p < c.n; ++p) {
      o.x[p] = side ? (const void*)c.dY[p] : c.X;
      o.L[p] = side ? c.N[p] : c.K;
      o.d[p] = side ? c.dB[p] : c.dA[p];
      most = o.L[p] > most ? o.L[p] : most;
      if (c.T > o.chunk) {
        char* const more = c.ws + plan.partial + 2 * plan.fragments + (side && c.T > plan.chunk_x ? c.n * plan.more_x : 0);
        size_t at = 0;
        for (int i = 0; i < p; ++i) at += side ? plan.more_y[i] : plan.more_x;
        o.more[p] = reinterpret_cast<float*>(more + at);
        const int k = side * MBQ_MAX_GROUP + p;
        join.chunk[k] = o.chunk;
        join.d[k] = o.d[p];
        join.more[k] = o.more[p];
        join.values[k] = (int64_t)c.r * o.L[p];
        joins = true;
      }
    }
    o.blocks = (int)blocks_of(most, side ? kWidthY : kWidthX);
    if (!side)
      outer<uint16_t, true>(o, c.n, stream);
    else if (wy)
      outer<float, true>(o, c.n, stream);
    else
      outer<float, false>(o, c.n, stream);
  }
  if (joins)
    hipLaunchKernelGGL(lora_join_kernel, dim3((unsigned)c.adapters, 64, 2 * MBQ_MAX_GROUP), dim3(256), 0, stream, join);
  return hip_status(hipGetLastError(), "adapter gradients' launch");
}

}  // namespace mbq

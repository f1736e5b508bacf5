// Entry points of what stands beside a frozen blob (include/mbq.h): adapters, the balance loss, the routers' gradients.
// Every check comes before the first launch.
#include <math.h>

#include "mbq_lora.h"

using namespace mbq;

namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
constexpr int64_t kMost = (int64_t)1 << 24;  // tokens, columns

mbq_status bad(mbq_status status, const char* who, const char* what) {
  set_error("%s: %s", who, what);
  return status;
}
mbq_status check_sizes(const char* who, int64_t T, int64_t K, int n) {
  if (n < 1 || n > MBQ_MAX_GROUP) {
    set_error("%s: n_proj=%d outside 1..%d", who, n, MBQ_MAX_GROUP);
    return MBQ_ERR_INVALID_ARG;
  }
  if (T < 0 || T > kMost || K <= 0 || K > kMost || K % kGroup != 0) {
    set_error("%s: bad sizes T=%lld K=%lld", who, (long long)T, (long long)K);
    return MBQ_ERR_BAD_SHAPE;
  }
  return MBQ_OK;
}
mbq_status check_workspace(const char* who, const void* ws, size_t have, size_t need) {
  if (ws && have >= need && aligned(ws, 256)) return MBQ_OK;
  set_error("%s: workspace null, too small or misaligned (%zu, needed %zu)", who, have, need);
  return MBQ_ERR_WORKSPACE;
}
// pools and assignment, the same for both directions
mbq_status lora_call(const char* who, const uint16_t* X, int64_t T, int64_t K, int n, const uint16_t* const* A,
                     const uint16_t* const* B, const int64_t* N, int64_t adapters, int r, const int32_t* ranks,
                     const float* scale, const int32_t* adapter, const int32_t* perm, const int32_t* offsets, LoraCall* c) {
  const mbq_status st = check_sizes(who, T, K, n);
  if (st != MBQ_OK) return st;
  if (r < 1 || r > MBQ_LORA_MAX_RANK || adapters < 1 || adapters > MBQ_LORA_MAX_ADAPTERS) {
    set_error("%s: rank %d outside 1..%d or %lld adapters outside 1..%d", who, r, MBQ_LORA_MAX_RANK, (long long)adapters,
              MBQ_LORA_MAX_ADAPTERS);
    return MBQ_ERR_BAD_SHAPE;
  }
  if (!A || !B || !N) return bad(MBQ_ERR_INVALID_ARG, who, "null pointer array");
  for (int p = 0; p < n; ++p)
    if (N[p] < 1 || N[p] > kMost) {
      set_error("%s: N=%lld of projection %d outside 1..2^24", who, (long long)N[p], p);
      return MBQ_ERR_BAD_SHAPE;
    }
  if (T > 0) {
    if (!X || !aligned(X, 16) || !scale || !adapter || !perm || !offsets || !aligned(scale, 4) || !aligned(ranks, 4) ||
        !aligned(adapter, 4) || !aligned(perm, 4) || !aligned(offsets, 4))
      return bad(MBQ_ERR_INVALID_ARG, who, "null or misaligned pointer (X needs 16-byte alignment)");
    for (int p = 0; p < n; ++p)
      if (!A[p] || !B[p] || !aligned(A[p], 16) || !aligned(B[p], 2)) {
        set_error("%s: null or misaligned pool of projection %d (A needs 16-byte alignment)", who, p);
        return MBQ_ERR_INVALID_ARG;
      }
  }
  *c = LoraCall{};
  c->X = X;
  c->T = T;
  c->K = K;
  c->n = n;
  for (int p = 0; p < n; ++p) {
    c->A[p] = A[p];
    c->B[p] = B[p];
    c->N[p] = N[p];
  }
  c->adapters = adapters;
  c->r = r;
  c->ranks = ranks;
  c->scale = scale;
  c->adapter = adapter;
  c->perm = perm;
  c->offsets = offsets;
  return MBQ_OK;
}

}  // namespace

extern "C" {

mbq_status mbq_lora_sort(const int32_t* adapter, int64_t T, int64_t n_adapters, int32_t* perm, int32_t* offsets,
                         void* stream) {
  ApiScope scope;
  if (T < 0 || T > kMost || n_adapters < 1 || n_adapters > MBQ_LORA_MAX_ADAPTERS) {
    set_error("mbq_lora_sort: bad sizes T=%lld n_adapters=%lld", (long long)T, (long long)n_adapters);
    return MBQ_ERR_BAD_SHAPE;
  }
  if (!offsets || (T > 0 && (!adapter || !perm)) || !aligned(adapter, 4) || !aligned(perm, 4) || !aligned(offsets, 4))
    return bad(MBQ_ERR_INVALID_ARG, "mbq_lora_sort", "null or misaligned pointer");
  return launch_lora_sort(adapter, T, n_adapters, perm, offsets, (hipStream_t)stream);
}

size_t mbq_lora_workspace_bytes(int64_t T, int64_t K, int n_proj, int r) {
  if (check_sizes("mbq_lora_workspace_bytes", T, K, n_proj) != MBQ_OK || r < 1 || r > MBQ_LORA_MAX_RANK) return 0;
  return lora_workspace_bytes(T, K, n_proj, r);
}

mbq_status mbq_lora_group(const uint16_t* X, int64_t T, int64_t K, int n_proj, const uint16_t* const* A_host,
                          const uint16_t* const* B_host, const int64_t* N_host, int64_t n_adapters, int r,
                          const int32_t* ranks, const float* scale, const int32_t* adapter, const int32_t* perm,
                          const int32_t* offsets, const float* const* base_host, float* const* Y_host,
                          float* const* H_host, void* ws, size_t ws_bytes, void* stream) {
  ApiScope scope;
  const char* who = "mbq_lora_group";
  LoraCall c;
  mbq_status st = lora_call(who, X, T, K, n_proj, A_host, B_host, N_host, n_adapters, r, ranks, scale, adapter, perm, offsets,
                            &c);
  if (st != MBQ_OK || T == 0) return st;
  if (!Y_host) return bad(MBQ_ERR_INVALID_ARG, who, "null pointer array");
  for (int p = 0; p < n_proj; ++p) {
    c.base[p] = base_host ? base_host[p] : nullptr;
    c.Y[p] = Y_host[p];
    c.H[p] = H_host ? H_host[p] : nullptr;
    if (!c.Y[p] || !aligned(c.Y[p], 4) || !aligned(c.base[p], 4) || (H_host && !c.H[p]) || !aligned(c.H[p], 4)) {
      set_error("%s: null or misaligned output or base of projection %d", who, p);
      return MBQ_ERR_INVALID_ARG;
    }
  }
  if (!lora_fits(c)) return bad(MBQ_ERR_BAD_SHAPE, who, "too many adapters for outputs this wide");
  st = check_workspace(who, ws, ws_bytes, lora_workspace_bytes(T, K, n_proj, r));
  if (st != MBQ_OK) return st;
  c.ws = (char*)ws;
  return launch_lora(c, (hipStream_t)stream);
}

size_t mbq_lora_backward_workspace_bytes(int64_t T, int64_t K, int n_proj, const int64_t* N_host, int64_t n_adapters,
                                         int r) {
  if (check_sizes("mbq_lora_backward_workspace_bytes", T, K, n_proj) != MBQ_OK || r < 1 || r > MBQ_LORA_MAX_RANK || !N_host ||
      n_adapters < 1 || n_adapters > MBQ_LORA_MAX_ADAPTERS)
    return 0;
  for (int p = 0; p < n_proj; ++p)
    if (N_host[p] < 1 || N_host[p] > kMost) return 0;
  if (!lora_backward_fits(T, K, n_proj, N_host, n_adapters, r)) return 0;
  return lora_backward_workspace_bytes(T, K, n_proj, N_host, n_adapters, r);
}

mbq_status mbq_lora_backward_group(const uint16_t* X, int64_t T, int64_t K, int n_proj, const uint16_t* const* A_host,
                                   const uint16_t* const* B_host, const int64_t* N_host, int64_t n_adapters, int r,
                                   const int32_t* ranks, const float* scale, const int32_t* adapter, const int32_t* perm,
                                   const int32_t* offsets, const float* const* dY_host, const float* const* H_host,
                                   const float* base, float* dX, float* const* dA_host, float* const* dB_host, void* ws,
                                   size_t ws_bytes, void* stream) {
  ApiScope scope;
  const char* who = "mbq_lora_backward_group";
  LoraCall c;
  mbq_status st = lora_call(who, X, T, K, n_proj, A_host, B_host, N_host, n_adapters, r, ranks, scale, adapter, perm, offsets,
                            &c);
  if (st != MBQ_OK) return st;
  if (T > 0 && (!dY_host || (dB_host && !H_host))) return bad(MBQ_ERR_INVALID_ARG, who, "null pointer array");
  for (int p = 0; p < n_proj; ++p) {
    c.dY[p] = T > 0 ? dY_host[p] : nullptr;
    c.Hin[p] = T > 0 && H_host ? H_host[p] : nullptr;
    c.dA[p] = dA_host ? dA_host[p] : nullptr;
    c.dB[p] = dB_host ? dB_host[p] : nullptr;
    if ((T > 0 && (!c.dY[p] || (dB_host && !c.Hin[p]))) || (dA_host && !c.dA[p]) || (dB_host && !c.dB[p]) ||
        !aligned(c.dY[p], 4) || !aligned(c.Hin[p], 4) || !aligned(c.dA[p], 4) || !aligned(c.dB[p], 4)) {
      set_error("%s: null or misaligned gradient or H of projection %d", who, p);
      return MBQ_ERR_INVALID_ARG;
    }
  }
  if (!aligned(base, 4) || !aligned(dX, 4)) return bad(MBQ_ERR_INVALID_ARG, who, "misaligned base or dX");
  if (!lora_backward_fits(T, K, n_proj, N_host, n_adapters, r))
    return bad(MBQ_ERR_BAD_SHAPE, who, "too many adapters for gradients this wide");
  st = check_workspace(who, ws, ws_bytes, lora_backward_workspace_bytes(T, K, n_proj, N_host, n_adapters, r));
  if (st != MBQ_OK) return st;
  c.dx_base = base;
  c.dX = T > 0 ? dX : nullptr;
  c.ws = (char*)ws;
  return launch_lora_backward(c, (hipStream_t)stream);
}

size_t mbq_balance_loss_workspace_bytes(int64_t T, int n_proj) {
  if (T < 0 || T > kMost || n_proj < 1 || n_proj > MBQ_MAX_GROUP) return 0;
  return balance_loss_workspace_bytes(T, n_proj);
}

mbq_status mbq_balance_loss_group(int n_proj, const double* const* logits_host, int64_t T, int P, const uint8_t* mask,
                                  const double* target_host, double coef, int32_t* const* counts_host,
                                  float* const* loss_host, float* const* dlogits_host, void* ws, size_t ws_bytes,
                                  void* stream) {
  ApiScope scope;
  const char* who = "mbq_balance_loss_group";
  mbq_status st = check_sizes(who, T, kGroup, n_proj);
  if (st != MBQ_OK) return st;
  if (P < 1 || P > MBQ_MAX_SLICES) {
    set_error("%s: P=%d outside 1..%d", who, P, MBQ_MAX_SLICES);
    return MBQ_ERR_BAD_SHAPE;
  }
  if (!counts_host || !loss_host || (T > 0 && !logits_host)) return bad(MBQ_ERR_INVALID_ARG, who, "null pointer array");
  if (!isfinite(coef)) return bad(MBQ_ERR_INVALID_ARG, who, "coef is not finite");
  BalanceCall c = {};
  c.n = n_proj;
  c.T = T;
  c.P = P;
  c.mask = mask;
  c.coef = coef;
  for (int e = 0; e < P; ++e) {
    c.weight[e] = target_host ? 1.0 / target_host[e] : (double)P;
    if (!isfinite(c.weight[e]) || !(c.weight[e] > 0.0)) {
      set_error("%s: target[%d] = %g must be finite and > 0", who, e, target_host[e]);
      return MBQ_ERR_INVALID_ARG;
    }
  }
  for (int p = 0; p < n_proj; ++p) {
    c.logits[p] = T > 0 ? logits_host[p] : nullptr;
    c.counts[p] = counts_host[p];
    c.loss[p] = loss_host[p];
    c.dlogits[p] = dlogits_host && T > 0 ? dlogits_host[p] : nullptr;
    if ((T > 0 && (!c.logits[p] || (dlogits_host && !c.dlogits[p]))) || !c.counts[p] || !c.loss[p] ||
        !aligned(c.logits[p], P % 2 ? 8 : 16) || !aligned(c.counts[p], 4) || !aligned(c.loss[p], 4) ||
        !aligned(c.dlogits[p], 4)) {
      set_error("%s: null or misaligned pointer of router %d", who, p);
      return MBQ_ERR_INVALID_ARG;
    }
  }
  st = check_workspace(who, ws, ws_bytes, balance_loss_workspace_bytes(T, n_proj));
  if (st != MBQ_OK) return st;
  c.ws = (char*)ws;
  return launch_balance_loss(c, (hipStream_t)stream);
}

size_t mbq_route_backward_workspace_bytes(int64_t T, int64_t K, int n_proj, int P) {
  if (check_sizes("mbq_route_backward_workspace_bytes", T, K, n_proj) != MBQ_OK || P < 1 || P > MBQ_MAX_SLICES) return 0;
  return route_backward_workspace_bytes(T, K, n_proj, P);
}

mbq_status mbq_route_backward_group(const uint16_t* X, int64_t T, int64_t K, int n_proj, const float* const* Wr_host, int P,
                                    const float* const* dlogits_host, const uint8_t* mask, const float* base, float* dX,
                                    float* const* dWr_host, float* const* dbr_host, void* ws, size_t ws_bytes,
                                    void* stream) {
  ApiScope scope;
  const char* who = "mbq_route_backward_group";
  mbq_status st = check_sizes(who, T, K, n_proj);
  if (st != MBQ_OK) return st;
  if (P < 1 || P > MBQ_MAX_SLICES) {
    set_error("%s: P=%d outside 1..%d", who, P, MBQ_MAX_SLICES);
    return MBQ_ERR_BAD_SHAPE;
  }
  if (T > 0 && (!X || !aligned(X, 16) || !Wr_host || !dlogits_host))
    return bad(MBQ_ERR_INVALID_ARG, who, "null pointer array or null/misaligned X");
  if (!aligned(base, 4) || !aligned(dX, 4)) return bad(MBQ_ERR_INVALID_ARG, who, "misaligned base or dX");
  RouteBackwardCall c = {};
  c.X = X;
  c.T = T;
  c.K = K;
  c.n = n_proj;
  c.P = P;
  c.mask = mask;
  c.base = base;
  c.dX = T > 0 ? dX : nullptr;
  for (int p = 0; p < n_proj; ++p) {
    c.Wr[p] = T > 0 ? Wr_host[p] : nullptr;
    c.dlogits[p] = T > 0 ? dlogits_host[p] : nullptr;
    c.dWr[p] = dWr_host ? dWr_host[p] : nullptr;
    c.dbr[p] = dbr_host ? dbr_host[p] : nullptr;
    if ((T > 0 && (!c.Wr[p] || !c.dlogits[p])) || (dWr_host && !c.dWr[p]) || (dbr_host && !c.dbr[p]) ||
        !aligned(c.Wr[p], 16) || !aligned(c.dlogits[p], 4) || !aligned(c.dWr[p], 4) || !aligned(c.dbr[p], 4)) {
      set_error("%s: null or misaligned pointer of router %d", who, p);
      return MBQ_ERR_INVALID_ARG;
    }
  }
  st = check_workspace(who, ws, ws_bytes, route_backward_workspace_bytes(T, K, n_proj, P));
  if (st != MBQ_OK) return st;
  c.ws = (char*)ws;
  return launch_route_backward(c, (hipStream_t)stream);
}

}  // extern "C"

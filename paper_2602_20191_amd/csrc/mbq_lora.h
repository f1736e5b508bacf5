// Low-rank adapters beside the shared projections: what the entry points hand to the launchers.
#pragma once

#include "mbq_common.h"

namespace mbq {

struct LoraCall {
  const uint16_t* X;
  int64_t T, K;
  int n;  // projections
  const uint16_t *A[MBQ_MAX_GROUP], *B[MBQ_MAX_GROUP];
  int64_t N[MBQ_MAX_GROUP];
  int64_t adapters;
  int r;
  const int32_t* ranks;
  const float* scale;
  const int32_t *adapter, *perm, *offsets;
  // forward
  const float* base[MBQ_MAX_GROUP];
  float *Y[MBQ_MAX_GROUP], *H[MBQ_MAX_GROUP];
  // backward
  const float *dY[MBQ_MAX_GROUP], *Hin[MBQ_MAX_GROUP];
  const float* dx_base;
  float* dX;
  float *dA[MBQ_MAX_GROUP], *dB[MBQ_MAX_GROUP];
  char* ws;
};

mbq_status launch_lora_sort(const int32_t* adapter, int64_t T, int64_t n, int32_t* perm, int32_t* offsets,
                            hipStream_t stream);
// whether the launches' grids can be that large
bool lora_fits(const LoraCall& c);
bool lora_backward_fits(int64_t T, int64_t K, int n, const int64_t* N, int64_t adapters, int r);
size_t lora_workspace_bytes(int64_t T, int64_t K, int n, int r);
mbq_status launch_lora(const LoraCall& c, hipStream_t stream);
size_t lora_backward_workspace_bytes(int64_t T, int64_t K, int n, const int64_t* N, int64_t adapters, int r);
mbq_status launch_lora_backward(const LoraCall& c, hipStream_t stream);

struct BalanceCall {
  int n;
  const double* logits[MBQ_MAX_GROUP];
  int64_t T;
  int P;
  const uint8_t* mask;
  double weight[MBQ_MAX_SLICES];  // 1 / target share
  double coef;
  int32_t* counts[MBQ_MAX_GROUP];
  float *loss[MBQ_MAX_GROUP], *dlogits[MBQ_MAX_GROUP];
  char* ws;
};
size_t balance_loss_workspace_bytes(int64_t T, int n);
mbq_status launch_balance_loss(const BalanceCall& c, hipStream_t stream);

struct RouteBackwardCall {
  const uint16_t* X;
  int64_t T, K;
  int n, P;
  const float *Wr[MBQ_MAX_GROUP], *dlogits[MBQ_MAX_GROUP];
  const uint8_t* mask;
  const float* base;
  float* dX;
  float *dWr[MBQ_MAX_GROUP], *dbr[MBQ_MAX_GROUP];
  char* ws;
};
size_t route_backward_workspace_bytes(int64_t T, int64_t K, int n, int P);
mbq_status launch_route_backward(const RouteBackwardCall& c, hipStream_t stream);

}  // namespace mbq

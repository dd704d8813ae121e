// Placement policies: the arguments that api checks pass to the kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "mlsim.h"

namespace mlsim {

constexpr float kLeastTemperature = 0x1p-126f;

// A policy's logits and settings (kernel argument; every field uniform).
struct PolicyArgs {
  const void *logits;       // [n_pol][n_ops][n_res] of `dtype`, strides ld_pol and ld_op in elements
  int64_t ld_pol, ld_op;
  int64_t block;            // consecutive scenarios sharing a policy
  int64_t phase;            // scen0 modulo the period
  int64_t period;           // block * n_pol, INT64_MAX where that overflows
  const float *settings;    // [n_pol][4] temperature, top_k, top_p, min_p, or null: the four below
  float temperature, top_k, top_p, min_p;
  int32_t dtype;
  int32_t n_pol, n_ops, n_res;
};

// Gradient rows: same shape and type as the logits, strides of their own.
struct PolicyOut {
  void *p;
  int64_t ld_pol, ld_op;
};

// A teacher's table: K resources and logits per op and policy.
struct PolicyTop {
  const uint16_t *res;
  const void *logits;       // of the policy's dtype
  int64_t ld_res_pol, ld_res_op, ld_log_pol, ld_log_op;
  int32_t top;
};

int64_t policy_work(const PolicyArgs &p, int64_t n_scen);  // scratch bytes of logp and grad
int launch_policy_sample(const PolicyArgs &p, int64_t n_scen, const float *u, int64_t ld_u, uint16_t *place,
                         int64_t ld_place, hipStream_t st);
int launch_policy_logp(const PolicyArgs &p, int64_t n_scen, const uint16_t *place, int64_t ld_place, float *logp,
                       void *work, hipStream_t st);
int launch_policy_grad(const PolicyArgs &p, int64_t n_scen, const uint16_t *place, int64_t ld_place,
                       const float *weight, const PolicyOut &grad, void *work, hipStream_t st);
int launch_policy_distill(const PolicyArgs &p, const PolicyTop &top, const float *weight, float *loss,
                          const PolicyOut &grad, hipStream_t st);

}  // namespace mlsim

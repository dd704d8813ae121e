// C ABI entry points of placement policies: argument checks and dispatch.
#include <algorithm>
#include <cmath>

#include "policy.hpp"
#include "sim.hpp"

using namespace mlsim;

namespace {

int elem_bytes(int32_t dtype) { return dtype == SIM_F32 ? 4 : 2; }

// Largest element offset + 1 of an array [n_pol][n_ops][n] with these strides,
// or -1 where it leaves the address range.
int64_t extent(int64_t n_pol, int64_t n_ops, int64_t n, int64_t ld_pol, int64_t ld_op) {
  const __int128 e = (__int128)(n_pol - 1) * ld_pol + (__int128)(n_ops - 1) * ld_op + n;
  return e > ((__int128)1 << 60) ? -1 : (int64_t)e;
}

bool aligned(const void *p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// The checks every call makes, and the kernels' view of the policy.
int make_policy(const sim_policy *p, int64_t n_scen, PolicyArgs &a) {
  if (!p || n_scen < 0) return SIM_E_INVAL;
  if (p->dtype != SIM_F32 && p->dtype != SIM_BF16 && p->dtype != SIM_F16) return SIM_E_INVAL;
  if (p->n_pol < 1 || p->n_ops < 0 || p->n_res < 1) return SIM_E_INVAL;
  if (p->n_ops > SIM_MAX_OPS || p->n_res > SIM_MAX_RES) return SIM_E_LIMIT;
  if (n_scen > SIM_MAX_POLICY_SCEN) return SIM_E_LIMIT;
  if (p->block < 1 || p->scen0 < 0 || n_scen > INT64_MAX - p->scen0) return SIM_E_INVAL;
  if (!p->settings) {
    if (p->temperature != 0 && !(p->temperature >= kLeastTemperature && std::isfinite(p->temperature))) return SIM_E_INVAL;
    if (p->top_k < 0 || !(p->top_p >= 0 && p->top_p <= 1) || !(p->min_p >= 0 && p->min_p <= 1)) return SIM_E_INVAL;
  } else if (!aligned(p->settings, 4)) {
    return SIM_E_INVAL;
  }
  if (p->ld_pol < 0 || p->ld_op < 0) return SIM_E_INVAL;
  if (p->n_ops > 0 && (!p->logits || !aligned(p->logits, elem_bytes(p->dtype)) ||
                       extent(p->n_pol, p->n_ops, p->n_res, p->ld_pol, p->ld_op) < 0))
    return SIM_E_INVAL;
  a = PolicyArgs{};
  a.logits = p->logits;
  a.ld_pol = p->ld_pol;
  a.ld_op = p->ld_op;
  a.block = p->n_pol == 1 ? INT64_MAX : p->block;
  a.period = a.block > INT64_MAX / p->n_pol ? INT64_MAX : a.block * p->n_pol;
  a.phase = p->n_pol == 1 ? 0 : p->scen0 % a.period;  // a saturated period is beyond scen0 + n_scen
  a.settings = p->settings;
  a.temperature = p->temperature;
  a.top_k = (float)std::min(p->top_k, SIM_MAX_RES);
  a.top_p = p->top_p;
  a.min_p = p->min_p;
  a.dtype = p->dtype;
  a.n_pol = p->n_pol;
  a.n_ops = p->n_ops;
  a.n_res = p->n_res;
  return SIM_OK;
}

// A gradient's strides: rows in one of the two orders, none over another.
int make_out(const PolicyArgs &a, void *grad, int64_t ld_pol, int64_t ld_op, PolicyOut &out) {
  if (!grad || !aligned(grad, elem_bytes(a.dtype)) || ld_pol < 0 || ld_op < 0) return SIM_E_INVAL;
  const int64_t ops = extent(1, a.n_ops, a.n_res, 0, ld_op), pols = extent(a.n_pol, 1, a.n_res, ld_pol, 0);
  if (ops < 0 || pols < 0 || extent(a.n_pol, a.n_ops, a.n_res, ld_pol, ld_op) < 0) return SIM_E_INVAL;
  const bool one_op = a.n_ops == 1, one_pol = a.n_pol == 1;
  const bool by_pol = (one_op || ld_op >= a.n_res) && (one_pol || ld_pol >= ops);
  const bool by_op = (one_pol || ld_pol >= a.n_res) && (one_op || ld_op >= pols);
  if (!by_pol && !by_op) return SIM_E_INVAL;
  out = PolicyOut{grad, ld_pol, ld_op};
  return SIM_OK;
}

bool bad_work(const PolicyArgs &a, int64_t n_scen, const void *work, int64_t work_bytes) {
  const int64_t need = policy_work(a, n_scen);
  return work_bytes < need || (need > 0 && (!work || !aligned(work, 8)));
}

}  // namespace

extern "C" int sim_policy_sample(const sim_policy *p, int64_t n_scen, const float *u, int64_t ld_u, uint16_t *place,
                                 int64_t ld_place, void *stream) {
  PolicyArgs a;
  if (int rc = make_policy(p, n_scen, a)) return rc;
  if (a.n_ops == 0 || n_scen == 0) return SIM_OK;
  if (!u || !place || !aligned(u, 4) || !aligned(place, 2) || ld_u < n_scen || ld_place < n_scen ||
      extent(1, a.n_ops, n_scen, 0, ld_u) < 0 || extent(1, a.n_ops, n_scen, 0, ld_place) < 0)
    return SIM_E_INVAL;
  return launch_policy_sample(a, n_scen, u, ld_u, place, ld_place, (hipStream_t)stream);
}

extern "C" int64_t sim_policy_work(const sim_policy *p, int64_t n_scen) {
  PolicyArgs a;
  if (int rc = make_policy(p, n_scen, a)) return rc;
  return a.n_ops == 0 || n_scen == 0 ? 0 : policy_work(a, n_scen);
}

extern "C" int sim_policy_logp(const sim_policy *p, int64_t n_scen, const uint16_t *place, int64_t ld_place,
                               float *logp, void *work, int64_t work_bytes, void *stream) {
  PolicyArgs a;
  if (int rc = make_policy(p, n_scen, a)) return rc;
  if (n_scen == 0) return SIM_OK;
  if (!logp || !aligned(logp, 4)) return SIM_E_INVAL;
  if (a.n_ops == 0)  // the empty sum
    return launch_zero((int32_t *)logp, n_scen, n_scen, 1, (hipStream_t)stream);
  if (!place || !aligned(place, 2) || ld_place < n_scen || extent(1, a.n_ops, n_scen, 0, ld_place) < 0)
    return SIM_E_INVAL;
  if (bad_work(a, n_scen, work, work_bytes)) return SIM_E_INVAL;
  return launch_policy_logp(a, n_scen, place, ld_place, logp, work, (hipStream_t)stream);
}

extern "C" int sim_policy_grad(const sim_policy *p, int64_t n_scen, const uint16_t *place, int64_t ld_place,
                               const float *weight, void *grad, int64_t ld_gpol, int64_t ld_gop, void *work,
                               int64_t work_bytes, void *stream) {
  PolicyArgs a;
  if (int rc = make_policy(p, n_scen, a)) return rc;
  if (a.n_ops == 0) return SIM_OK;
  PolicyOut out;
  if (int rc = make_out(a, grad, ld_gpol, ld_gop, out)) return rc;
  if (n_scen > 0 && (!place || !weight || !aligned(place, 2) || !aligned(weight, 4) || ld_place < n_scen ||
                     extent(1, a.n_ops, n_scen, 0, ld_place) < 0))
    return SIM_E_INVAL;
  if (n_scen > 0 && bad_work(a, n_scen, work, work_bytes)) return SIM_E_INVAL;
  return launch_policy_grad(a, n_scen, place, ld_place, weight, out, work, (hipStream_t)stream);
}

extern "C" int sim_policy_distill(const sim_policy *p, const uint16_t *top_res, int64_t ld_res_pol,
                                  int64_t ld_res_op, const void *top_logits, int64_t ld_log_pol, int64_t ld_log_op,
                                  int32_t top, const float *weight, float *loss, void *grad, int64_t ld_gpol,
                                  int64_t ld_gop, void *stream) {
  PolicyArgs a;
  if (int rc = make_policy(p, 0, a)) return rc;
  if (top < 1 || top > SIM_MAX_RES || ld_res_pol < 0 || ld_res_op < 0 || ld_log_pol < 0 || ld_log_op < 0)
    return SIM_E_INVAL;
  if (a.n_ops == 0) return SIM_OK;
  if (!top_res || !top_logits || !loss || !aligned(top_res, 2) || !aligned(top_logits, elem_bytes(a.dtype)) ||
      !aligned(loss, 4) || (weight && !aligned(weight, 4)) ||
      extent(a.n_pol, a.n_ops, top, ld_res_pol, ld_res_op) < 0 ||
      extent(a.n_pol, a.n_ops, top, ld_log_pol, ld_log_op) < 0)
    return SIM_E_INVAL;
  PolicyOut out{};
  if (grad)
    if (int rc = make_out(a, grad, ld_gpol, ld_gop, out)) return rc;
  const PolicyTop t{top_res, top_logits, ld_res_pol, ld_res_op, ld_log_pol, ld_log_op, top};
  return launch_policy_distill(a, t, weight, loss, out, (hipStream_t)stream);
}

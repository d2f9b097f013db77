// Draws from rows of scores, and their loss: the C entry points. Kernels: choice.hip.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <string>

#include "../../include/emr.h"
#include "choice.h"

namespace emr {
emr_status set_error(emr_status st, const std::string& msg);
}
extern "C" hipError_t emr_launch_choice(int kind, const void* args, hipStream_t s);

namespace {

emr_status failf(emr_status st, const char* fmt, ...) {
  char b[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(b, sizeof b, fmt, ap);
  va_end(ap);
  return emr::set_error(st, b);
}

static_assert(EMR_F32 == emr::kTypeF32 && EMR_BF16 == emr::kTypeBf16 && EMR_F16 == emr::kTypeF16, "");

int64_t type_size(int32_t type) { return type == EMR_F32 ? 4 : 2; }

emr_status check_scores(const char* who, const emr_scores* S) {
  if (!S) return failf(EMR_E_INVAL, "%s: scores is NULL", who);
  if (S->type != EMR_F32 && S->type != EMR_BF16 && S->type != EMR_F16)
    return failf(EMR_E_INVAL, "%s: score type %d", who, S->type);
  if (S->rows < 0 || S->n < 1)
    return failf(EMR_E_INVAL, "%s: %lld rows of %lld scores", who, (long long)S->rows,
                 (long long)S->n);
  if (S->rows > INT32_MAX || S->n > INT32_MAX)
    return failf(EMR_E_LIMIT, "%s: %lld rows of %lld scores (at most 2^31 - 1 each)", who,
                 (long long)S->rows, (long long)S->n);
  if (S->stride < 0 || S->stride > INT64_MAX / 4 / (S->rows > 0 ? S->rows : 1))
    return failf(EMR_E_INVAL, "%s: row stride %lld", who, (long long)S->stride);
  if (S->rows > 0 && (!S->x || (uintptr_t)S->x % (uintptr_t)type_size(S->type) != 0))
    return failf(EMR_E_INVAL, "%s: scores NULL or not aligned to their type", who);
  return EMR_OK;
}

// Whether groups of four entries of every row are aligned to their size.
int32_t aligned4(const void* p, int64_t stride, int32_t type) {
  return (uintptr_t)p % (uintptr_t)(4 * type_size(type)) == 0 && stride % 4 == 0;
}

}  // namespace

extern "C" {

emr_status emr_sample(const emr_scores* scores, const emr_sampling* rule, const float* u, int64_t draws,
                      int32_t* index, float* logp, void* stream) {
  const emr_status st = check_scores("sample", scores);
  if (st != EMR_OK) return st;
  if (!rule) return failf(EMR_E_INVAL, "sample: rule is NULL");
  if (!rule->row_temperature && !(rule->temperature >= 0.0f))
    return failf(EMR_E_INVAL, "sample: temperature %g is not at least 0", (double)rule->temperature);
  if (!rule->row_top_k && rule->top_k < 0)
    return failf(EMR_E_INVAL, "sample: top_k %d is negative", rule->top_k);
  if (!rule->row_top_p && !(rule->top_p > 0.0f && rule->top_p <= 1.0f))
    return failf(EMR_E_INVAL, "sample: top_p %g outside (0, 1]", (double)rule->top_p);
  if (!rule->row_min_p && !(rule->min_p >= 0.0f && rule->min_p <= 1.0f))
    return failf(EMR_E_INVAL, "sample: min_p %g outside [0, 1]", (double)rule->min_p);
  if (draws < 0 || draws > INT64_MAX / 8 / (scores->rows > 0 ? scores->rows : 1))
    return failf(EMR_E_INVAL, "sample: %lld draws", (long long)draws);
  if (scores->rows == 0 || draws == 0) return EMR_OK;
  if (!u || !index) return failf(EMR_E_INVAL, "sample: u or index is NULL");
  emr::SampleArgs a{};
  a.x = scores->x;
  a.stride = scores->stride;
  a.rows = scores->rows;
  a.n = (uint32_t)scores->n;
  a.type = scores->type;
  a.vec = aligned4(scores->x, scores->stride, scores->type);
  a.t = rule->temperature;
  a.p = rule->top_p;
  a.min_p = rule->min_p;
  a.k = rule->top_k;
  a.row_t = rule->row_temperature;
  a.row_k = rule->row_top_k;
  a.row_p = rule->row_top_p;
  a.row_min_p = rule->row_min_p;
  a.u = u;
  a.draws = draws;
  a.index = index;
  a.logp = logp;
  const uint32_t groups = (a.n + emr::kDrawPart - 1) / emr::kDrawPart;
  a.part = (groups + emr::kDrawSegs - 1) / emr::kDrawSegs * emr::kDrawPart;
  const hipError_t e = emr_launch_choice(0, &a, (hipStream_t)stream);
  if (e != hipSuccess) return failf(EMR_E_DEVICE, "sample: %s", hipGetErrorString(e));
  return EMR_OK;
}

emr_status emr_answer_loss(const emr_scores* scores, const int32_t* index, const float* scale,
                           float temperature, float* loss, void* grad, int64_t grad_stride,
                           void* stream) {
  const emr_status st = check_scores("loss", scores);
  if (st != EMR_OK) return st;
  if (!(temperature >= 1.17549435e-38f && std::isfinite(temperature)))
    return failf(EMR_E_INVAL, "loss: temperature %g is not a positive normal number",
                 (double)temperature);
  if (scores->rows == 0) return EMR_OK;
  if (!loss && !grad) return failf(EMR_E_INVAL, "loss: neither loss nor grad is asked for");
  if (grad && (grad_stride < scores->n || grad_stride > INT64_MAX / 4 / (scores->rows + 1)))
    return failf(EMR_E_INVAL, "loss: grad's row stride %lld is below %lld scores",
                 (long long)grad_stride, (long long)scores->n);
  if (grad && (uintptr_t)grad % (uintptr_t)type_size(scores->type) != 0)
    return failf(EMR_E_INVAL, "loss: grad is not aligned to its type");
  if (!index) return failf(EMR_E_INVAL, "loss: index is NULL");
  emr::LossArgs a{};
  a.x = scores->x;
  a.stride = scores->stride;
  a.rows = scores->rows;
  a.n = (uint32_t)scores->n;
  a.type = scores->type;
  a.vec = aligned4(scores->x, scores->stride, scores->type) &&
          (!grad || aligned4(grad, grad_stride, scores->type));
  a.inv_t = 1.0f / temperature;
  a.index = index;
  a.scale = scale;
  a.loss = loss;
  a.grad = grad;
  a.grad_stride = grad_stride;
  const hipError_t e = emr_launch_choice(1, &a, (hipStream_t)stream);
  if (e != hipSuccess) return failf(EMR_E_DEVICE, "loss: %s", hipGetErrorString(e));
  return EMR_OK;
}

}  // extern "C"

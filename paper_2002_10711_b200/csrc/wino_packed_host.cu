// Host side of the layers with 4-bit weights: argument checks and sizes.
#include <cmath>

#include "wino.h"
#include "wino_launch.h"

using namespace wino;

namespace {

constexpr int32_t kMaxSize = 1 << 24;          // K, C: sums of K * C / 2 bytes stay far below 2^63

bool size_ok(int32_t K, int32_t C) { return K >= 1 && C >= 1 && K <= kMaxSize && C <= kMaxSize; }
bool group_ok(int32_t group) { return group == 32 || group == 64 || (group >= 128 && group % 128 == 0); }
bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool real_type(int32_t t) { return t == WINO_FLOAT || t == WINO_BF16 || t == WINO_FP16; }
int bytes_of(int32_t t) { return t == WINO_INT8 ? 1 : t == WINO_FLOAT ? 4 : 2; }

int check_packed(const wino_packed_t& w) {
  if (!size_ok(w.K, w.C) || !group_ok(w.group)) return WINO_ERR_INVALID;
  if (w.scale_dtype != WINO_BF16 && w.scale_dtype != WINO_FP16) return WINO_ERR_INVALID;
  if (w.codes_dev == nullptr || w.scales_dev == nullptr) return WINO_ERR_INVALID;
  if (!aligned(w.codes_dev, 16) || !aligned(w.scales_dev, 16) || !aligned(w.zeros_dev, 16)) return WINO_ERR_ALIGNMENT;
  return WINO_OK;
}
bool quant_ok(const wino_quant_t& q) {
  return std::isfinite(q.scale) && q.scale > 0.0f && q.qmin <= q.qmax && q.qmin >= -128 && q.qmax <= 127 &&
         q.zero_point >= -128 && q.zero_point <= 127;
}
// rows of n elements, `stride` apart
bool stride_ok(int64_t rows, int64_t n, int64_t stride) {
  return rows <= 1 ? stride >= 0 : stride >= n && stride <= (int64_t)1 << 40;
}
int device_sms(int* sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return WINO_ERR_CUDA;
  // asked of the runtime once per device and thread
  static thread_local int known_dev = -1, known_sms = 0;
  if (dev != known_dev) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = kDefaultSms;
    known_dev = dev; known_sms = n;
  }
  *sms = known_sms;
  return WINO_OK;
}

}  // namespace

extern "C" {

size_t wino_packed_code_bytes(int32_t K, int32_t C) {
  return size_ok(K, C) ? (size_t)((K + 15) / 16) * ((C + 127) / 128) * 1024 : 0;
}

size_t wino_packed_scale_count(int32_t K, int32_t C, int32_t group) {
  return size_ok(K, C) && group_ok(group) ? (size_t)((K + 15) / 16) * (((size_t)C + group - 1) / group) * 16 : 0;
}

int wino_quantize_weights(const wino_packed_t* out, const void* w, int32_t w_dtype, int64_t w_stride,
                          void* values, void* stream) {
  if (out == nullptr || w == nullptr) return WINO_ERR_INVALID;
  const int rc = check_packed(*out);
  if (rc != WINO_OK) return rc;
  if (!real_type(w_dtype) || !stride_ok(out->K, out->C, w_stride)) return WINO_ERR_INVALID;
  if (!aligned(w, bytes_of(w_dtype)) || !aligned(values, bytes_of(w_dtype))) return WINO_ERR_ALIGNMENT;
  return launch_quantize(*out, w, w_dtype, w_stride, values, (cudaStream_t)stream);
}

int wino_linear_forward(const wino_linear_desc_t* d, const void* x, const float* bias, void* y, void* stream) {
  if (d == nullptr) return WINO_ERR_INVALID;
  int rc = check_packed(d->w);
  if (rc != WINO_OK) return rc;
  if (d->M < 0 || d->M > kMaxSize) return WINO_ERR_INVALID;
  if (d->x_dtype != WINO_INT8 && !real_type(d->x_dtype)) return WINO_ERR_INVALID;
  if (d->y_dtype != WINO_INT8 && !real_type(d->y_dtype)) return WINO_ERR_INVALID;
  if (!stride_ok(d->M, d->w.C, d->x_stride) || !stride_ok(d->M, d->w.K, d->y_stride)) return WINO_ERR_INVALID;
  if (d->x_dtype == WINO_INT8 && !quant_ok(d->q_x)) return WINO_ERR_INVALID;
  if (d->y_dtype == WINO_INT8 && !quant_ok(d->q_Y)) return WINO_ERR_INVALID;
  if (d->M == 0) return WINO_OK;
  if (x == nullptr || y == nullptr) return WINO_ERR_INVALID;
  if (!aligned(x, bytes_of(d->x_dtype)) || !aligned(y, bytes_of(d->y_dtype)) || !aligned(bias, 4))
    return WINO_ERR_ALIGNMENT;
  int sms = 0;
  if ((rc = device_sms(&sms)) != WINO_OK) return rc;
  // A grid's second dimension holds 65535 slices of 8 rows or more: more rows go in several launches.
  constexpr int32_t kMost = 1 << 18;
  wino_linear_desc_t part = *d;
  for (int32_t m = 0; m < d->M && rc == WINO_OK; m += kMost) {
    part.M = d->M - m < kMost ? d->M - m : kMost;
    rc = launch_linear(part, static_cast<const char*>(x) + m * d->x_stride * bytes_of(d->x_dtype), bias,
                       static_cast<char*>(y) + m * d->y_stride * bytes_of(d->y_dtype), sms, (cudaStream_t)stream);
  }
  return rc;
}

static int check_experts(const wino_experts_desc_t* d) {
  if (d == nullptr) return WINO_ERR_INVALID;
  if (d->T < 0 || d->T > kMaxSize || !size_ok(d->I, d->D) || !real_type(d->dtype)) return WINO_ERR_INVALID;
  if (d->E < 1 || d->top_k < 1 || d->top_k > d->E) return WINO_ERR_INVALID;
  if (d->normalize != 0 && d->normalize != 1) return WINO_ERR_INVALID;
  if (d->E > 512 || d->top_k > 16) return WINO_ERR_UNSUPPORTED;
  return WINO_OK;
}

size_t wino_experts_workspace_bytes(const wino_experts_desc_t* d) {
  return check_experts(d) == WINO_OK ? experts_workspace(d->T, d->I, d->top_k, d->dtype) : 0;
}

int wino_experts_forward(const wino_experts_desc_t* d, const void* x, const void* router, const float* router_bias,
                         void* y, int32_t* ids, float* weights, void* workspace, void* stream) {
  int rc = check_experts(d);
  if (rc != WINO_OK) return rc;
  const wino_packed_t* const part[3] = {&d->gate, &d->up, &d->down};
  for (const wino_packed_t* w : part)
    if ((rc = check_packed(*w)) != WINO_OK) return rc;
  if (d->gate.K != d->I || d->up.K != d->I || d->down.K != d->D || d->gate.C != d->D || d->up.C != d->D ||
      d->down.C != d->I || d->gate.group != d->up.group || d->gate.scale_dtype != d->up.scale_dtype ||
      (d->gate.zeros_dev == nullptr) != (d->up.zeros_dev == nullptr))
    return WINO_ERR_INVALID;
  if (!stride_ok(d->T, d->D, d->x_stride) || !stride_ok(d->T, d->D, d->y_stride)) return WINO_ERR_INVALID;
  if (d->T == 0) return WINO_OK;
  if (x == nullptr || router == nullptr || y == nullptr || ids == nullptr || weights == nullptr)
    return WINO_ERR_INVALID;
  if (workspace == nullptr) return WINO_ERR_WORKSPACE;
  const int size = bytes_of(d->dtype);
  if (!aligned(x, size) || !aligned(router, size) || !aligned(y, size) || !aligned(router_bias, 4) ||
      !aligned(ids, 4) || !aligned(weights, 4) || !aligned(workspace, 16))
    return WINO_ERR_ALIGNMENT;
  int sms = 0;
  if ((rc = device_sms(&sms)) != WINO_OK) return rc;
  return launch_experts(*d, x, router, router_bias, y, ids, weights, workspace, sms, (cudaStream_t)stream);
}

}  // extern "C"

// Operator-level entry points of the C ABI (declared in include/fdg_ops.h): group normalisation with an activation, and tensors
// held in 8 bits.
#include "../../include/fdg.h"
#include "../../include/fdg_ops.h"
#include "group_norm.cuh"

namespace fdg {
typedef __nv_bfloat16 bf16;

static bool precision_ok(int precision) { return precision == FDG_FP32_CUDACORE || precision == FDG_BF16_TC; }
static unsigned elem_bytes(int precision) { return precision == FDG_BF16_TC ? 2 : 4; }
static fdg_status status_of(cudaError_t e) { return e == cudaSuccess ? FDG_OK : FDG_ERR_CUDA; }

// Values whose bytes, blocks of 32 and shares can be counted in the widths that the kernels use.
static bool rows_ok(size_t rows, int C) { return C >= 1 && C <= 1 << 28 && rows >= 1 && rows <= ((size_t)1 << 36) / (size_t)C; }
static bool gn_shape_ok(int precision, const fdg_gn_shape* s) {
  return s && precision_ok(precision) && s->N >= 1 && s->N <= 1 << 30 && s->HW >= 1 && s->C >= 1 && s->groups >= 1 && s->C % s->groups == 0 &&
         s->C <= 1 << 16 && rows_ok((size_t)s->N * (size_t)s->HW, s->C);
}
static bool floats_ok(std::initializer_list<const float*> arrays) {
  for (const float* a : arrays)
    if (!aligned_to(a, sizeof(float))) return false;
  return true;
}
static size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// Scratch: the forward pass's rows of sums; the backward pass's per-image totals [N][2][C], where it forms them, and its rows of sums.
static size_t forward_need(const gn::Plan& pl) { return align256(gn::partial_floats(pl) * sizeof(float)); }
static size_t totals_bytes(const gn::Plan& pl) { return gn::merges_backward(pl.g) ? 0 : align256((size_t)pl.g.N * 2 * pl.g.C * sizeof(float)); }
static size_t backward_need(const gn::Plan& pl) { return totals_bytes(pl) + align256(gn::partial_floats(pl) * sizeof(float)); }

template <typename T>
static cudaError_t gn_forward_as(const gn::Plan& pl, const void* x, const float* gamma, const float* beta, const void* res, int act, float eps,
                                 void* y, float* stats, uint8_t* gate, int8_t* codes, uint8_t* scales, void* scratch, cudaStream_t st) {
  gn::Forward<T> p{};
  p.x = (const T*)x; p.gamma = gamma; p.beta = beta; p.res = (const T*)res; p.y = (T*)y; p.stats = stats; p.gate = gate;
  p.codes = codes; p.scales = scales; p.eps = eps; p.act = act;
  p.partial = static_cast<float*>(scratch);
  return gn::launch_forward<T>(st, pl, p);
}
template <typename T>
static cudaError_t gn_backward_as(const gn::Plan& pl, const void* dy, const void* x, const int8_t* codes, const uint8_t* scales,
                                  const float* stats, const float* gamma, const float* beta, int act, const void* mask, const uint8_t* gate,
                                  const void* res, void* dx, float* dgamma, float* dbeta, void* scratch, cudaStream_t st) {
  gn::Backward<T> p{};
  p.dy = (const T*)dy; p.x = (const T*)x; p.codes = codes; p.scales = scales; p.stats = stats; p.gamma = gamma; p.beta = beta;
  p.mask = (const T*)mask; p.gate = gate; p.res = (const T*)res; p.dx = (T*)dx;
  p.slope = act == FDG_ACT_SILU ? gn::SLOPE_SILU : mask ? gn::SLOPE_MASK : gate ? gn::SLOPE_BITS : gn::SLOPE_ONE;
  p.totals = static_cast<float*>(scratch);
  p.partial = reinterpret_cast<float*>(static_cast<char*>(scratch) + totals_bytes(pl));
  p.dgamma = dgamma; p.dbeta = dbeta;
  return gn::launch_backward<T>(st, pl, p);
}
}  // namespace fdg

using namespace fdg;

extern "C" {

fdg_status fdg_ckpt_encode(int precision, const void* x, size_t rows, int C, int8_t* codes, uint8_t* scales, fdg_stream stream) {
  if (!x || !codes || !scales || !precision_ok(precision) || !rows_ok(rows, C) || !aligned_to(x, elem_bytes(precision))) return FDG_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return status_of(precision == FDG_BF16_TC ? launch_ckpt_encode<bf16>(st, (const bf16*)x, rows, C, codes, scales)
                                            : launch_ckpt_encode<float>(st, (const float*)x, rows, C, codes, scales));
}

fdg_status fdg_ckpt_decode(int precision, const int8_t* codes, const uint8_t* scales, size_t rows, int C, void* x, fdg_stream stream) {
  if (!x || !codes || !scales || !precision_ok(precision) || !rows_ok(rows, C) || !aligned_to(x, elem_bytes(precision))) return FDG_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return status_of(precision == FDG_BF16_TC ? launch_ckpt_decode<bf16>(st, codes, scales, rows, C, (bf16*)x)
                                            : launch_ckpt_decode<float>(st, codes, scales, rows, C, (float*)x));
}

fdg_status fdg_gn_scratch_bytes(int precision, const fdg_gn_shape* s, int backward, size_t* bytes) {
  if (!bytes || !gn_shape_ok(precision, s)) return FDG_ERR_INVALID_ARG;
  const int b = (int)elem_bytes(precision);
  if (!backward) {
    const gn::Plan pl = gn::plan_forward(b, s->N, s->HW, s->C, s->groups);
    *bytes = forward_need(pl);
    return FDG_OK;
  }
  const gn::Plan pl = gn::plan_backward(b, s->N, s->HW, s->C, s->groups);
  *bytes = backward_need(pl);
  return FDG_OK;
}

fdg_status fdg_gn_forward(int precision, const fdg_gn_shape* s, const void* x, const float* gamma, const float* beta, const void* res, int act,
                          float eps, void* y, float* stats, uint8_t* gate, int8_t* codes, uint8_t* scales, void* scratch, size_t scratch_bytes,
                          fdg_stream stream) {
  if (!gn_shape_ok(precision, s) || !x || !gamma || !beta || !y || !stats || !(eps > 0.f)) return FDG_ERR_INVALID_ARG;
  if (act != FDG_ACT_NONE && act != FDG_ACT_RELU && act != FDG_ACT_SILU) return FDG_ERR_INVALID_ARG;
  if ((act == FDG_ACT_SILU && res) || (gate && act != FDG_ACT_RELU) || (codes != nullptr) != (scales != nullptr)) return FDG_ERR_INVALID_ARG;
  const unsigned b = elem_bytes(precision);
  if (!aligned_to(x, b) || !aligned_to(y, b) || !aligned_to(res, b) || !aligned_to(scratch, 256) || !floats_ok({gamma, beta, stats}))
    return FDG_ERR_INVALID_ARG;
  const gn::Plan pl = gn::plan_forward((int)b, s->N, s->HW, s->C, s->groups);
  const size_t need = forward_need(pl);
  if (need > 0 && (!scratch || scratch_bytes < need)) return FDG_ERR_WORKSPACE_TOO_SMALL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return status_of(precision == FDG_BF16_TC ? gn_forward_as<bf16>(pl, x, gamma, beta, res, act, eps, y, stats, gate, codes, scales, scratch, st)
                                            : gn_forward_as<float>(pl, x, gamma, beta, res, act, eps, y, stats, gate, codes, scales, scratch, st));
}

fdg_status fdg_gn_backward(int precision, const fdg_gn_shape* s, const void* dy, const void* x, const int8_t* codes, const uint8_t* scales,
                           const float* stats, const float* gamma, const float* beta, int act, const void* mask, const uint8_t* gate,
                           const void* res, void* dx, float* dgamma, float* dbeta, void* scratch, size_t scratch_bytes, fdg_stream stream) {
  if (!gn_shape_ok(precision, s) || !dy || !stats || !gamma || !dx || !dgamma || !dbeta) return FDG_ERR_INVALID_ARG;
  if (act != FDG_ACT_NONE && act != FDG_ACT_RELU && act != FDG_ACT_SILU) return FDG_ERR_INVALID_ARG;
  if ((codes != nullptr) != (scales != nullptr) || (x != nullptr) == (codes != nullptr)) return FDG_ERR_INVALID_ARG;
  if ((mask != nullptr) + (gate != nullptr) != (act == FDG_ACT_RELU ? 1 : 0) || (act == FDG_ACT_SILU && !beta)) return FDG_ERR_INVALID_ARG;
  const unsigned b = elem_bytes(precision);
  if (!aligned_to(dy, b) || !aligned_to(x, b) || !aligned_to(mask, b) || !aligned_to(res, b) || !aligned_to(dx, b) ||
      !aligned_to(scratch, 256) || !floats_ok({stats, gamma, beta, dgamma, dbeta}))
    return FDG_ERR_INVALID_ARG;
  const gn::Plan pl = gn::plan_backward((int)b, s->N, s->HW, s->C, s->groups);
  if (!scratch || scratch_bytes < backward_need(pl)) return FDG_ERR_WORKSPACE_TOO_SMALL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return status_of(precision == FDG_BF16_TC
                       ? gn_backward_as<bf16>(pl, dy, x, codes, scales, stats, gamma, beta, act, mask, gate, res, dx, dgamma, dbeta, scratch, st)
                       : gn_backward_as<float>(pl, dy, x, codes, scales, stats, gamma, beta, act, mask, gate, res, dx, dgamma, dbeta, scratch, st));
}

}  // extern "C"

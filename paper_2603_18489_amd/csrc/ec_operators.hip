// Entry points of the operators around a step: tokens drawn from rows of logits, matrices in microscaled 4-bit floating point.
#include <cmath>
#include <string>

#include "ec_internal.h"

using namespace ec;

namespace {

constexpr int kVocabMax = 163840;         // as ec_init
constexpr int kSampleRowsMax = 65535;
constexpr int kMxKMax = 131072;
constexpr int64_t kMxRowsMax = 1 << 24;   // to and from 4 bits
constexpr int64_t kMxLinearRowsMax = 1 << 19;
constexpr int kMxLinearColsMax = 1 << 20;

int op_fail(int code, const char* msg) {
  set_global_error(msg);
  return code;
}
// what the launches left behind
int op_done(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return EC_OK;
  try {
    set_global_error((std::string(what) + ": " + hipGetErrorString(e)).c_str());
  } catch (...) {
    set_global_error(what);
  }
  return EC_ERR_HIP;
}
bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }
bool plain_type(int32_t t) { return t == EC_T_F32 || t == EC_T_BF16; }
size_t type_bytes(int32_t t) { return t == EC_T_F32 ? 4 : 2; }

int check_mx(const uint8_t* codes, const uint8_t* scales, int32_t k) {
  if (!codes || !scales) return op_fail(EC_ERR_ARG, "codes and scales must not be NULL");
  if (!aligned(codes, 16)) return op_fail(EC_ERR_ARG, "codes must be 16-byte aligned");
  if (k < 32 || k > kMxKMax || k % 32) return op_fail(EC_ERR_ARG, "k must be a multiple of 32 in [32, 131072]");
  return EC_OK;
}

}  // namespace

extern "C" {

int ec_row_sample(const void* logits, int32_t type, int32_t rows, int32_t vocab, size_t ld, const float* uniforms,
                  const ec_sample_cfg* cfg, int32_t* tokens, float* stats, void* workspace, size_t workspace_bytes,
                  void* hip_stream) {
  if (!cfg) return op_fail(EC_ERR_ARG, "cfg must not be NULL");
  if (!plain_type(type)) return op_fail(EC_ERR_ARG, "logits must be EC_T_F32 or EC_T_BF16");
  if (rows < 0 || rows > kSampleRowsMax) return op_fail(EC_ERR_ARG, "rows must be in [0, 65535]");
  if (vocab < 2 || vocab > kVocabMax) return op_fail(EC_ERR_ARG, "vocab must be in [2, 163840]");
  if (!(cfg->temperature >= 0.f) || !std::isfinite(cfg->temperature))
    return op_fail(EC_ERR_ARG, "temperature must be finite and not negative");
  if (cfg->top_k < 0) return op_fail(EC_ERR_ARG, "top_k must not be negative");
  if (!(cfg->top_p > 0.f && cfg->top_p <= 1.f)) return op_fail(EC_ERR_ARG, "top_p must be in (0, 1]");
  if (!(cfg->min_p >= 0.f && cfg->min_p <= 1.f)) return op_fail(EC_ERR_ARG, "min_p must be in [0, 1]");
  if (rows == 0) return EC_OK;
  if (!logits || !uniforms || !tokens || !stats)
    return op_fail(EC_ERR_ARG, "logits, uniforms, tokens and stats must not be NULL");
  if (ld < (size_t)vocab) return op_fail(EC_ERR_ARG, "row stride smaller than vocab");
  if (!aligned(stats, 16)) return op_fail(EC_ERR_ARG, "stats must be 16-byte aligned");
  if (!aligned(logits, type_bytes(type)) || !aligned(uniforms, 4) || !aligned(tokens, 4))
    return op_fail(EC_ERR_ARG, "logits, uniforms and tokens must be aligned to their elements");
  if (const size_t need = ec_row_sample_workspace_bytes(rows, vocab)) {
    if (!workspace || !aligned(workspace, 256)) return op_fail(EC_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need) return op_fail(EC_ERR_WORKSPACE, "workspace smaller than ec_row_sample_workspace_bytes()");
  }
  const bool greedy = cfg->temperature == 0.f;
  SampleArgs a;
  a.scale = 1.4426950408889634 / (greedy ? 1.0 : (double)cfg->temperature);
  a.per_z = 16.0 / (greedy ? 1.0 : (double)cfg->temperature);
  a.top_k = greedy ? 1 : cfg->top_k < vocab ? cfg->top_k : 0;
  a.top_p = cfg->top_p;
  a.min_z = cfg->min_p > 0.f ? std::log((double)cfg->min_p) * (greedy ? 1.0 : (double)cfg->temperature) : -INFINITY;
  launch_sample_rows(logits, type == EC_T_BF16, rows, vocab, ld, uniforms, a, tokens, (float4*)stats, workspace,
                     (hipStream_t)hip_stream);
  return op_done("sampling kernels");
}

size_t ec_row_sample_workspace_bytes(int32_t rows, int32_t vocab) {
  if (rows < 0 || rows > kSampleRowsMax || vocab < 2 || vocab > kVocabMax) return 0;
  return sample_workspace(rows, vocab);
}

int ec_mx_quantize(const void* x, int32_t type, int64_t rows, int32_t k, size_t ld, uint8_t* codes, uint8_t* scales,
                   void* hip_stream) {
  if (!plain_type(type)) return op_fail(EC_ERR_ARG, "x must be EC_T_F32 or EC_T_BF16");
  if (rows < 0 || rows > kMxRowsMax) return op_fail(EC_ERR_ARG, "rows must be in [0, 16777216]");
  if (k < 32 || k > kMxKMax || k % 32) return op_fail(EC_ERR_ARG, "k must be a multiple of 32 in [32, 131072]");
  if (rows == 0) return EC_OK;
  const int rc = check_mx(codes, scales, k);
  if (rc != EC_OK) return rc;
  if (!x) return op_fail(EC_ERR_ARG, "x must not be NULL");
  if (ld < (size_t)k) return op_fail(EC_ERR_ARG, "row stride smaller than k");
  if (!aligned(x, type_bytes(type))) return op_fail(EC_ERR_ARG, "x must be aligned to its elements");
  launch_mx_quantize(x, type == EC_T_BF16, rows, k / 32, ld, codes, scales, (hipStream_t)hip_stream);
  return op_done("quantisation kernel");
}

int ec_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t k, void* out, int32_t type, size_t ld,
                     void* hip_stream) {
  if (!plain_type(type)) return op_fail(EC_ERR_ARG, "out must be EC_T_F32 or EC_T_BF16");
  if (rows < 0 || rows > kMxRowsMax) return op_fail(EC_ERR_ARG, "rows must be in [0, 16777216]");
  if (k < 32 || k > kMxKMax || k % 32) return op_fail(EC_ERR_ARG, "k must be a multiple of 32 in [32, 131072]");
  if (rows == 0) return EC_OK;
  const int rc = check_mx(codes, scales, k);
  if (rc != EC_OK) return rc;
  if (!out) return op_fail(EC_ERR_ARG, "out must not be NULL");
  if (ld < (size_t)k) return op_fail(EC_ERR_ARG, "row stride smaller than k");
  if (!aligned(out, type_bytes(type))) return op_fail(EC_ERR_ARG, "out must be aligned to its elements");
  launch_mx_dequantize(codes, scales, rows, k / 32, out, type == EC_T_BF16, ld, (hipStream_t)hip_stream);
  return op_done("dequantisation kernel");
}

size_t ec_mx_packed_bytes(int32_t n, int32_t k) {
  if (n < 1 || n > kMxLinearColsMax || k < 32 || k > kMxKMax || k % 32) return 0;
  return mx_packed_bytes(n, k / 32);
}

int ec_mx_pack(const uint8_t* codes, const uint8_t* scales, int32_t n, int32_t k, void* packed, size_t packed_bytes,
               void* hip_stream) {
  if (n < 1 || n > kMxLinearColsMax) return op_fail(EC_ERR_ARG, "n must be in [1, 1048576]");
  const int rc = check_mx(codes, scales, k);
  if (rc != EC_OK) return rc;
  if (!packed || !aligned(packed, 256)) return op_fail(EC_ERR_WORKSPACE, "packed is NULL or not 256-byte aligned");
  if (packed_bytes < ec_mx_packed_bytes(n, k))
    return op_fail(EC_ERR_WORKSPACE, "packed smaller than ec_mx_packed_bytes()");
  launch_mx_pack(codes, scales, n, k / 32, (uint8_t*)packed, (hipStream_t)hip_stream);
  return op_done("packing kernel");
}

size_t ec_mx_linear_workspace_bytes(int32_t x_type, int64_t rows, int32_t n, int32_t k) {
  if ((x_type != EC_T_BF16 && x_type != EC_T_MXFP4) || rows < 0 || rows > kMxLinearRowsMax || !ec_mx_packed_bytes(n, k)) return 0;
  return mx_linear_workspace(x_type == EC_T_MXFP4, rows, n, k / 32);
}

int ec_debug_mx_blocks(int32_t x_type, int64_t rows, int32_t n, int32_t k, int32_t shape[3]) {
  if (x_type != EC_T_BF16 && x_type != EC_T_MXFP4) return op_fail(EC_ERR_ARG, "x must be EC_T_BF16 or EC_T_MXFP4");
  if (rows < 1 || rows > kMxLinearRowsMax || !ec_mx_packed_bytes(n, k)) return op_fail(EC_ERR_ARG, "rows, n or k outside ec_mx_linear's limits");
  if (!shape) return op_fail(EC_ERR_ARG, "shape must not be NULL");
  mx_linear_blocks(x_type == EC_T_MXFP4, rows, n, k / 32, shape);
  return EC_OK;
}

int ec_mx_linear(const void* x, const uint8_t* x_scales, int32_t x_type, int64_t rows, size_t ld, const void* packed, int32_t n,
                 int32_t k, void* y, int32_t y_type, size_t ldy, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (x_type != EC_T_BF16 && x_type != EC_T_MXFP4) return op_fail(EC_ERR_ARG, "x must be EC_T_BF16 or EC_T_MXFP4");
  if (!plain_type(y_type)) return op_fail(EC_ERR_ARG, "y must be EC_T_F32 or EC_T_BF16");
  if (rows < 0 || rows > kMxLinearRowsMax) return op_fail(EC_ERR_ARG, "rows must be in [0, 524288]");
  if (n < 1 || n > kMxLinearColsMax) return op_fail(EC_ERR_ARG, "n must be in [1, 1048576]");
  if (k < 32 || k > kMxKMax || k % 32) return op_fail(EC_ERR_ARG, "k must be a multiple of 32 in [32, 131072]");
  if (rows == 0) return EC_OK;
  if (!x || !packed || !y) return op_fail(EC_ERR_ARG, "x, packed and y must not be NULL");
  if (!aligned(x, 16) || !aligned(packed, 256)) return op_fail(EC_ERR_ARG, "x must be 16-byte, packed 256-byte aligned");
  if (x_type == EC_T_MXFP4 && !x_scales) return op_fail(EC_ERR_ARG, "x_scales must not be NULL");
  if (x_type == EC_T_BF16 && (ld < (size_t)k || ld % 8))
    return op_fail(EC_ERR_ARG, "x's row stride must be a multiple of 8 elements, k or more");
  if (ldy < (size_t)n) return op_fail(EC_ERR_ARG, "y's row stride is smaller than n");
  if (!aligned(y, type_bytes(y_type))) return op_fail(EC_ERR_ARG, "y must be aligned to its elements");
  if (const size_t need = ec_mx_linear_workspace_bytes(x_type, rows, n, k)) {
    if (!workspace || !aligned(workspace, 256)) return op_fail(EC_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need) return op_fail(EC_ERR_WORKSPACE, "workspace smaller than ec_mx_linear_workspace_bytes()");
  }
  launch_mx_linear(x, x_type == EC_T_MXFP4 ? x_scales : nullptr, rows, ld, (const uint8_t*)packed, n, k / 32, y,
                   y_type == EC_T_BF16, ldy, workspace, (hipStream_t)hip_stream);
  return op_done("product kernel");
}

}  // extern "C"

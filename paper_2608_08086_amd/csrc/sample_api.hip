// Entry point of sampling (archer_ops.h): host-side checks, then the launch.
#include "archer_ops.h"
#include "errors.h"
#include "sample.h"

namespace {
bool known(int dtype) { return dtype == ARCHER_BF16 || dtype == ARCHER_FP32 || dtype == ARCHER_FP16; }
bool vocab_fits(int vocab) { return vocab >= 1 && vocab <= SAMPLE_MAX_VOCAB; }
}  // namespace

extern "C" size_t archer_op_sample_ws_bytes(int32_t dtype, int32_t rows, int32_t vocab) {
  return known(dtype) && rows >= 1 && vocab_fits(vocab) ? sample_ws_bytes(rows) : 0;
}

extern "C" archer_status archer_op_sample(int32_t dtype, int32_t rows, int32_t vocab, const void* logits, int64_t row_stride,
                                          int32_t exclude, const float* u, const float* temperature, const int32_t* top_k,
                                          const float* top_p, const float* min_p, int32_t* token, float* logp,
                                          void* workspace, size_t ws_bytes, void* hip_stream) {
  if (!known(dtype)) return archer_fail(ARCHER_E_ARG, "dtype must be ARCHER_BF16, ARCHER_FP32 or ARCHER_FP16");
  if (rows < 0) return archer_fail(ARCHER_E_SHAPE, "rows must not be negative");
  if (!vocab_fits(vocab)) return archer_fail(ARCHER_E_SHAPE, "vocab must be in [1, 524288]");
  if (exclude < -1 || exclude >= vocab) return archer_fail(ARCHER_E_ARG, "exclude must be a token or -1");
  if (rows == 0) return ARCHER_OK;
  if (!logits || !u || !token) return archer_fail(ARCHER_E_ARG, "null operand");
  if ((uintptr_t)logits & (dtype == ARCHER_FP32 ? 3 : 1)) return archer_fail(ARCHER_E_ARG, "logits must be aligned to their elements");
  if (!workspace || ((uintptr_t)workspace & 255) || ws_bytes < sample_ws_bytes(rows))
    return archer_fail(ARCHER_E_WORKSPACE, "workspace too small or misaligned");
  SampleArgs a;
  a.logits = logits; a.ld = row_stride; a.rows = rows; a.vocab = vocab; a.exclude = exclude;
  a.u = u; a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p;
  a.token = token; a.logp = logp;
  launch_sample(dtype, a, workspace, (hipStream_t)hip_stream);
  if (hipError_t e = hipGetLastError()) return archer_fail(ARCHER_E_HIP, std::string("archer_op_sample: ") + hipGetErrorString(e));
  return ARCHER_OK;
}

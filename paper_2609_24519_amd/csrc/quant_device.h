// Device helpers of the operators of quantised inference: element types and the sequences of a batch.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <mutex>
#include <set>
#include <string>

#include "awe_quant.h"

namespace awe {
namespace {

using bf16 = __bf16;
using f16 = _Float16;

// Rounds to nearest, ties to even.
__device__ __forceinline__ void store_real(void* p, int64_t i, awe_dtype t, float v) {
  if (t == AWE_F32)
    reinterpret_cast<float*>(p)[i] = v;
  else if (t == AWE_BF16)
    reinterpret_cast<bf16*>(p)[i] = (bf16)v;
  else
    reinterpret_cast<f16*>(p)[i] = (f16)v;
}

// Sequence b of a batch: its first row, rows and length.  What does not fit the host's bounds is refused
// here, before any index is formed from it (rows = 0, and the flag).
struct Seq {
  int32_t row0, rows, len;
};
__device__ __forceinline__ Seq sequence(const awe_batch& b, int32_t s, bool stored, int32_t* flag, bool report) {
  const int32_t r0 = b.starts[s], r1 = b.starts[s + 1], len = b.lengths[s];
  const bool ok = r0 >= 0 && r1 >= r0 && r1 <= b.rows && r1 - r0 <= b.max_rows && len >= 0 && len <= b.max_length &&
                  (!stored || r1 - r0 <= len);
  if (!ok && report && flag != nullptr) *flag = 1;
  return ok ? Seq{r0, r1 - r0, len} : Seq{0, 0, 0};
}

// Block holding position p of sequence s (p < len <= max_length <= ld_blocks * block), or -1 and the flag.
__device__ __forceinline__ int32_t block_of(const awe_cache& c, const awe_batch& b, int32_t s, int32_t p, int32_t* flag) {
  const int32_t id = b.blocks[s * b.ld_blocks + p / c.block];
  if (id >= 0 && id < c.num_blocks) return id;
  if (flag != nullptr) *flag = 1;
  return -1;
}

awe_status launched(const char* what) {
  const hipError_t err = hipGetLastError();
  if (err == hipSuccess) return AWE_OK;
  set_error(std::string(what) + ": " + hipGetErrorString(err));
  return AWE_ERR_HIP;
}

}  // namespace
}  // namespace awe

// Launch descriptions of the operators of quantised inference (awe_w4.hip, awe_cache.hip); the
// arguments are checked in awe_quant_api.cpp.
#pragma once

#include "awe_internal.h"

namespace awe {

struct W4Launch {
  int64_t M, N, K;
  const void* x;
  int64_t ldx;
  awe_dtype x_type;
  const float* x_scales;  // nullable
  const uint8_t* w;
  int64_t ldw;
  const void* scales;
  int64_t lds;
  awe_dtype s_type;
  const uint8_t* zeros;  // nullable: 8 everywhere
  int64_t ldz;
  int64_t group;  // a multiple of 32, or at least K
  void* y;
  int64_t ldy;
  awe_dtype y_type;
};
awe_status launch_w4(const W4Launch& g, hipStream_t stream);

// Rows of one tensor: element (i, h, d) at p[i*row + h*head + d].
struct Rows {
  void* p;
  int64_t row, head;
};

struct CacheLaunch {
  awe_cache c;
  awe_batch b;
  awe_dtype type;
  Rows k, v;
  int32_t* flag;
};
awe_status launch_cache_store(const CacheLaunch& g, hipStream_t stream);
awe_status launch_cache_load(const CacheLaunch& g, hipStream_t stream);

struct AttendLaunch {
  awe_cache c;
  awe_batch b;
  awe_dtype type;
  Rows q, o;
  int32_t q_heads;
  float scale;
  bool causal;
  void* ws;
  int32_t* flag;
};
awe_status launch_cache_attend(const AttendLaunch& g, hipStream_t stream);
// How a call is laid over workgroups, from its host-side sizes alone.
constexpr int kRowsColumns = 128;  // columns of a workgroup whose waves have columns of their own
struct AttendPlan {
  bool own_columns;  // a wave has columns of its own and sees all tokens; otherwise a workgroup's waves share
                     // 16 columns and split the tokens
  int32_t groups;    // workgroups along the columns
  int32_t splits;    // workgroups along the tokens
  int32_t chunk;     // tokens of each
  size_t workspace;
};
AttendPlan plan_attend(const awe_cache& c, const awe_batch& b, int32_t q_heads);

}  // namespace awe

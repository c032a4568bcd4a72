// An int8 cache of keys and values with a scale per block and head: awe_cache_store, awe_cache_load and
// awe_cache_attend.
#include "quant_device.h"

namespace awe {
namespace {

// Where dimension d of slot t lies within its block and head: keys by token, values by dimension.
__device__ __forceinline__ int64_t element(const awe_cache& c, bool values, int t, int d) {
  return values ? (int64_t)d * c.block + t : (int64_t)t * c.head_dim + d;
}

// One workgroup per touched block, head and tensor: workgroup (j, head, tensor + 2 * sequence) takes the
// sequence's j-th block that gets rows.
struct Tile {
  Seq s;
  int32_t id, first, t0, t1;  // block, position of its slot 0, slots that get rows
};
__device__ __forceinline__ Tile tile_of(const CacheLaunch& g, int32_t* flag) {
  Tile t;
  t.s = sequence(g.b, blockIdx.z >> 1, true, flag, threadIdx.x == 0);
  t.id = -1;
  const int32_t pos0 = t.s.len - t.s.rows;
  t.first = (pos0 / g.c.block + (int32_t)blockIdx.x) * g.c.block;
  if (t.s.rows == 0 || t.first >= t.s.len) return t;
  t.t0 = pos0 > t.first ? pos0 - t.first : 0;
  t.t1 = t.s.len - t.first < g.c.block ? t.s.len - t.first : g.c.block;
  t.id = block_of(g.c, g.b, blockIdx.z >> 1, t.first, threadIdx.x == 0 ? flag : nullptr);
  return t;
}

__global__ __launch_bounds__(256) void store_plain_kernel(CacheLaunch g) {
  const Tile t = tile_of(g, g.flag);
  if (t.id < 0) return;
  const bool values = blockIdx.z & 1;
  const int head = blockIdx.y, D = g.c.head_dim;
  const Rows& r = values ? g.v : g.k;
  const int64_t at = (int64_t)t.id * g.c.heads + head;
  int8_t* q = (values ? g.c.v : g.c.k) + at * g.c.block * D;
  float* scale = (values ? g.c.v_scales : g.c.k_scales) + at;
  const int64_t row0 = t.s.row0 + (t.first - (t.s.len - t.s.rows));  // row of slot 0
  float most = 0.f;
  bool bad = false;
  for (int e = threadIdx.x; e < (t.t1 - t.t0) * D; e += 256) {
    const float x = fabsf(load_real(r.p, (row0 + t.t0 + e / D) * r.row + head * r.head + e % D, g.type));
    if (x <= 3.402823466e38f)
      most = fmaxf(most, x);
    else
      bad = true;
  }
  if (bad && g.flag != nullptr) *g.flag = 1;
  __shared__ float part[256];
  part[threadIdx.x] = most;
  __syncthreads();
  for (int d = 128; d > 0; d >>= 1) {
    if (threadIdx.x < d) part[threadIdx.x] = fmaxf(part[threadIdx.x], part[threadIdx.x + d]);
    __syncthreads();
  }
  const float old = t.t0 > 0 ? *scale : 0.f;
  const float now = fmaxf(old, part[0] / 127.f);
  __syncthreads();  // every thread has read the old scale
  if (threadIdx.x == 0) *scale = now;
  if (now != old) {
    const float ratio = old / now;
    for (int e = threadIdx.x; e < t.t0 * D; e += 256) {
      int8_t* p = q + element(g.c, values, e / D, e % D);
      *p = (int8_t)fminf(fmaxf(rintf((float)*p * ratio), -127.f), 127.f);
    }
  }
  for (int e = threadIdx.x; e < (t.t1 - t.t0) * D; e += 256) {
    const float x = load_real(r.p, (row0 + t.t0 + e / D) * r.row + head * r.head + e % D, g.type);
    const float v = now > 0.f && fabsf(x) <= 3.402823466e38f ? fminf(fmaxf(rintf(x / now), -127.f), 127.f) : 0.f;
    q[element(g.c, values, t.t0 + e / D, e % D)] = (int8_t)v;
  }
}

__global__ __launch_bounds__(256) void load_plain_kernel(CacheLaunch g) {
  const Tile t = tile_of(g, g.flag);
  if (t.id < 0) return;
  const bool values = blockIdx.z & 1;
  const int head = blockIdx.y, D = g.c.head_dim;
  const Rows& r = values ? g.v : g.k;
  const int64_t at = (int64_t)t.id * g.c.heads + head;
  const int8_t* q = (values ? g.c.v : g.c.k) + at * g.c.block * D;
  const float scale = (values ? g.c.v_scales : g.c.k_scales)[at];
  const int64_t row0 = t.s.row0 + (t.first - (t.s.len - t.s.rows));
  for (int e = threadIdx.x; e < (t.t1 - t.t0) * D; e += 256)
    store_real(r.p, (row0 + t.t0 + e / D) * r.row + head * r.head + e % D, g.type,
               (float)q[element(g.c, values, t.t0 + e / D, e % D)] * scale);
}

// One wave per row and query head: 64 tokens at a time, one per lane, for the scores, and the
// dimensions over the lanes for the values; running maximum and sum.
__global__ __launch_bounds__(64) void attend_plain_kernel(AttendLaunch g) {
  const int lane = threadIdx.x, D = g.c.head_dim, qh = blockIdx.y, head = qh / (g.q_heads / g.c.heads);
  const Seq s = sequence(g.b, blockIdx.z, false, g.flag, lane == 0);
  __shared__ float qs[256], ps[64];
  for (int32_t i = blockIdx.x; i < s.rows; i += gridDim.x) {
    __syncthreads();
    for (int d = lane; d < D; d += 64)
      qs[d] = load_real(g.q.p, (int64_t)(s.row0 + i) * g.q.row + qh * g.q.head + d, g.type);
    __syncthreads();
    const int32_t keys = g.causal ? s.len - s.rows + i + 1 : s.len;
    float m = -INFINITY, l = 0.f, o[4] = {};
    for (int32_t j0 = 0; j0 < keys; j0 += 64) {
      const int32_t j = j0 + lane;
      const int32_t id = j < keys ? block_of(g.c, g.b, blockIdx.z, j, g.flag) : -1;
      const int64_t at = (int64_t)id * g.c.heads + head;
      float score = -INFINITY;
      if (id >= 0) {
        const int8_t* k = g.c.k + at * g.c.block * D + element(g.c, false, j % g.c.block, 0);
        float dot = 0.f;
        for (int d = 0; d < D; ++d) dot += qs[d] * (float)k[d];
        score = dot * g.c.k_scales[at] * g.scale;
      }
      float top = score;
      for (int d = 32; d > 0; d >>= 1) {
        const float other = __shfl_xor(top, d);
        top = other > top || other != other ? other : top;
      }
      if (top == -INFINITY) continue;
      const float now = top > m || top != top ? top : m, keep = m == -INFINITY ? 0.f : expf(m - now);
      const float p = score == -INFINITY ? 0.f : expf(score - now);
      m = now;
      float sum = p;
      for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
      l = l * keep + sum;
      ps[lane] = p;
      __syncthreads();
      for (int a = 0; a < D / 64; ++a) {
        o[a] *= keep;
        for (int t = 0; t < 64; ++t) {
          const int32_t id_t = __shfl(id, t);
          if (id_t < 0) continue;
          const int64_t at_t = (int64_t)id_t * g.c.heads + head;
          const float v = (float)g.c.v[at_t * g.c.block * D + element(g.c, true, (j0 + t) % g.c.block, a * 64 + lane)];
          o[a] += ps[t] * v * g.c.v_scales[at_t];
        }
      }
      __syncthreads();
    }
    for (int a = 0; a < D / 64; ++a)
      store_real(g.o.p, (int64_t)(s.row0 + i) * g.o.row + qh * g.o.head + a * 64 + lane, g.type, l == 0.f ? 0.f : o[a] / l);
  }
}

// Grid (blocks that can be touched, heads, 2 * sequences); sequences go over in parts of the grid's limit.
template <class K>
awe_status launch_tiles(K kernel, CacheLaunch g, const char* what, hipStream_t stream) {
  const unsigned x = (unsigned)((g.b.max_rows + g.c.block - 1) / g.c.block + 1);
  const int32_t all = g.b.sequences;
  for (int32_t s = 0; s < all; s += 32767) {
    CacheLaunch part = g;
    part.b.sequences = all - s < 32767 ? all - s : 32767;
    part.b.starts += s;
    part.b.lengths += s;
    part.b.blocks += s * g.b.ld_blocks;
    hipLaunchKernelGGL(kernel, dim3(x, (unsigned)g.c.heads, 2u * part.b.sequences), dim3(256), 0, stream, part);
    const awe_status st = launched(what);
    if (st != AWE_OK) return st;
  }
  return AWE_OK;
}

}  // namespace

awe_status launch_cache_store(const CacheLaunch& g, hipStream_t stream) {
  return launch_tiles(store_plain_kernel, g, "cache store launch", stream);
}

awe_status launch_cache_load(const CacheLaunch& g, hipStream_t stream) {
  return launch_tiles(load_plain_kernel, g, "cache load launch", stream);
}

awe_status launch_cache_attend(const AttendLaunch& g, hipStream_t stream) {
  const unsigned x = (unsigned)(g.b.max_rows < 4096 ? g.b.max_rows : 4096);
  for (int32_t s = 0; s < g.b.sequences; s += 65535) {
    AttendLaunch part = g;
    part.b.sequences = g.b.sequences - s < 65535 ? g.b.sequences - s : 65535;
    part.b.starts += s;
    part.b.lengths += s;
    part.b.blocks += s * g.b.ld_blocks;
    hipLaunchKernelGGL(attend_plain_kernel, dim3(x, (unsigned)g.q_heads, (unsigned)part.b.sequences), dim3(64), 0,
                       stream, part);
    const awe_status st = launched("attention launch");
    if (st != AWE_OK) return st;
  }
  return AWE_OK;
}

}  // namespace awe

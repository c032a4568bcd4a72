// An int8 cache of keys and values with a scale per block and head: awe_cache_store, awe_cache_load and
// awe_cache_attend.
#include "quant_device.h"

namespace awe {
namespace {

// ---- store and load -------------------------------------------------------------------------
// One workgroup per touched block, head and tensor: workgroup (j, head, tensor + 2 * sequence) takes the
// sequence's j-th block that gets rows.  Bound by the rows' and the cache's bytes, and by the chain of reads that
// leads to them (starts and lengths, table, rows, then the largest); for 4544 rows of 8 heads of 128 in
// BF16, storing takes 12 us (28 MB, 2.3 TB/s), loading 8 (28 MB, 3.5 TB/s).  A thread has up to kPatches
// patches of four adjacent tokens by eight dimensions; storing keeps them in registers between the search for
// the largest and the rounding, so rows are read once (reading them twice, and dividing by the scale: 18.6 us).
// Values, which are kept by dimension, are turned over in LDS, a word of four tokens at a time.
struct Tile {
  int32_t id, t0, t1;  // block (-1: nothing to do), slots that get rows
  int64_t row0;        // row of slot 0 (of slot t0 at the earliest)
};
__device__ __forceinline__ Tile tile_of(const CacheLaunch& g) {
  const bool one = threadIdx.x == 0;
  const Seq s = sequence(g.b, blockIdx.z >> 1, true, g.flag, one && blockIdx.x == 0);
  const int32_t pos0 = s.len - s.rows, first = (pos0 / g.c.block + (int32_t)blockIdx.x) * g.c.block;
  if (s.rows == 0 || first >= s.len) return Tile{-1, 0, 0, 0};
  const int32_t id = block_of(g.c, g.b, blockIdx.z >> 1, first, one ? g.flag : nullptr);
  return Tile{id, pos0 > first ? pos0 - first : 0, std::min(s.len - first, g.c.block), (int64_t)s.row0 + first - pos0};
}

// Eight elements of a row at any address, as words and as floats.
template <class E>
struct __attribute__((packed)) Any8Of {
  E v[8];
};
template <class E>
struct __attribute__((packed)) Words {
  static constexpr int kN = 2 * sizeof(E);
  uint32_t w[kN];

  __device__ __forceinline__ float value(int i) const {
    if constexpr (std::is_same<E, float>::value) return __builtin_bit_cast(float, w[i]);
    if constexpr (std::is_same<E, bf16>::value) return __builtin_bit_cast(float, i % 2 == 0 ? w[i / 2] << 16 : w[i / 2] & 0xffff0000u);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i / 2] >> (16 * (i % 2))));
  }
};
// The largest magnitudes of words of elements, as bits: whole numbers are ordered as the magnitudes are, and an
// infinity or a NaN is at least kBad.
template <class E>
struct Magnitude {
  typedef uint16_t u2 __attribute__((ext_vector_type(2)));
  static constexpr uint32_t kBad = std::is_same<E, float>::value ? 0x7f800000u : std::is_same<E, bf16>::value ? 0x7f80u : 0x7c00u;
  static __device__ __forceinline__ uint32_t larger(uint32_t most, uint32_t w) {
    if constexpr (sizeof(E) == 4) return std::max(most, w & 0x7fffffffu);
    const uint32_t m = w & 0x7fff7fffu;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u2, most), __builtin_bit_cast(u2, m)));
  }
  static __device__ __forceinline__ uint32_t top(uint32_t most) {  // of a word's elements
    return sizeof(E) == 4 ? most : std::max(most & 0xffffu, most >> 16);
  }
  static __device__ __forceinline__ uint32_t finite(uint32_t w) {  // 0 for the elements that are not
    if constexpr (sizeof(E) == 4) return (w & 0x7fffffffu) >= kBad ? 0u : w;
    return ((w & 0x7fffu) >= kBad ? 0u : w & 0xffffu) | (((w >> 16) & 0x7fffu) >= kBad ? 0u : w & 0xffff0000u);
  }
  static __device__ __forceinline__ float value(uint32_t top) {
    return Words<E>{{sizeof(E) == 4 ? top : top & 0xffffu}}.value(0);
  }
};

// rint(x / scale) within [-127, 127], its low byte the result's, for finite x and one scale > 0.  With
// both brought to a scale in [1, 2) (exactly, but for x far below half a step), q = x y for the rounded reciprocal
// y of the scale is within an ulp of the quotient, and one step with the exact remainder rounds it correctly; so this
// is the quotient of the formula in 3 instructions, not the 10 of a division.  Adding 1.5 2^23 rounds to
// a whole number, ties to even.
struct Quantiser {
  float unit, reciprocal;
  int power;
  __device__ __forceinline__ explicit Quantiser(float scale)
      : power(scale > 0.f ? 1 - __builtin_amdgcn_frexp_expf(scale) : 0) {
    unit = scale > 0.f ? ldexpf(scale, power) : 1.f;
    reciprocal = 1.f / unit;
  }
  __device__ __forceinline__ uint32_t operator()(float x) const {
    x = __builtin_amdgcn_ldexpf(x, power);
    float q = x * reciprocal;
    q = __builtin_fmaf(__builtin_fmaf(-q, unit, x), reciprocal, q);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(q, -127.f, 127.f) + 12582912.f);
  }
};
// The low bytes of four words.
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

// Dynamic LDS: a block of values by dimension, rows padded by a word.
extern __shared__ uint8_t turned[];
size_t turned_bytes(const awe_cache& c) { return (size_t)c.head_dim * (c.block + 4); }

// The patches of a block: the e-th covers slots slot .. slot + 3 (some of which may get no row) and
// dimensions d .. d + 7.
struct Patch {
  int32_t slot, d;
};
__device__ __forceinline__ int patches(const Tile& t, int D) { return ((t.t1 + 3) / 4 - t.t0 / 4) * (D / 8); }
__device__ __forceinline__ Patch patch(const Tile& t, int D, int e) {
  return Patch{4 * (t.t0 / 4 + e / (D / 8)), 8 * (e % (D / 8))};
}

template <class E, int kPatches>
__global__ __launch_bounds__(256) void store_kernel(CacheLaunch g) {
  const Tile t = tile_of(g);
  if (t.id < 0) return;
  const bool values = blockIdx.z & 1;
  const int head = blockIdx.y, D = g.c.head_dim, block = g.c.block, threads = blockDim.x;
  const Rows& r = values ? g.v : g.k;
  const int64_t at = (int64_t)t.id * g.c.heads + head;
  int8_t* q = (values ? g.c.v : g.c.k) + at * block * D;
  float* scale = (values ? g.c.v_scales : g.c.k_scales) + at;
  const E* rows = reinterpret_cast<const E*>(r.p) + t.row0 * r.row + head * r.head;
  const int n = patches(t, D);
  Words<E> x[kPatches][4] = {};
#pragma unroll
  for (int u = 0; u < kPatches; ++u) {
    const int e = threadIdx.x + u * threads;
    if (e >= n) break;
    const Patch at = patch(t, D, e);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (at.slot + k >= t.t0 && at.slot + k < t.t1)
        x[u][k] = *reinterpret_cast<const Words<E>*>(rows + (at.slot + k) * r.row + at.d);
  }
  const float old = t.t0 > 0 ? *scale : 0.f;
  using Size = Magnitude<E>;
  auto largest = [&] {
    uint32_t m = 0;
#pragma unroll
    for (int u = 0; u < kPatches; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int w = 0; w < Words<E>::kN; ++w) m = Size::larger(m, x[u][k].w[w]);
    return Size::top(m);
  };
  uint32_t top = largest();
  if (top >= Size::kBad) {
    if (g.flag != nullptr) *g.flag = 1;
#pragma unroll
    for (int u = 0; u < kPatches; ++u)
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int w = 0; w < Words<E>::kN; ++w) x[u][k].w[w] = Size::finite(x[u][k].w[w]);
    top = largest();
  }
  float most = Size::value(top);
  __shared__ float part[4];
  for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
  __syncthreads();  // (every thread has read the old scale)
  for (int w = 0; w < threads / 64; ++w) most = fmaxf(most, part[w]);
  const float now = fmaxf(old, most / 127.f);
  if (threadIdx.x == 0) *scale = now;
  if (now != old && t.t0 > 0) {
    // the older tokens on the new scale, 16 bytes at a time: keys' first t0 rows, values' first t0 columns
    const float ratio = old / now;
    const int chunks = values ? (t.t0 + 15) / 16 : D / 16, lines = values ? D : t.t0, line = values ? block : D;
    for (int e = threadIdx.x; e < lines * chunks; e += threads) {
      const int c = e % chunks;
      uint4* p = reinterpret_cast<uint4*>(q + (e / chunks) * line + 16 * c);
      const int keep = values ? t.t0 - 16 * c : 16;  // the bytes after these are not older tokens
      uint4 w = *p;
      int8_t* b = reinterpret_cast<int8_t*>(&w);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < keep) b[i] = (int8_t)fminf(fmaxf(rintf((float)b[i] * ratio), -127.f), 127.f);
      *p = w;
    }
    __syncthreads();  // the rows' bytes share words with these
  }
  const int stride = block + 4;
  const Quantiser byte_of(now);
#pragma unroll
  for (int u = 0; u < kPatches; ++u) {
    const int e = threadIdx.x + u * threads;
    if (e >= n) break;
    const Patch at = patch(t, D, e);
    uint32_t b[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) b[k][i] = now > 0.f ? byte_of(x[u][k].value(i)) : 0u;
    if (!values) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (at.slot + k >= t.t0 && at.slot + k < t.t1)
          *reinterpret_cast<uint2*>(q + (at.slot + k) * D + at.d) =
              uint2{low_bytes(b[k][0], b[k][1], b[k][2], b[k][3]), low_bytes(b[k][4], b[k][5], b[k][6], b[k][7])};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        *reinterpret_cast<uint32_t*>(turned + (at.d + i) * stride + at.slot) = low_bytes(b[0][i], b[1][i], b[2][i], b[3][i]);
    }
  }
  if (!values) return;
  __syncthreads();
  if (t.t0 == 0 && t.t1 == block) {
    for (int e = threadIdx.x; e < D * block / 16; e += threads) {
      const int d = e / (block / 16), c = e % (block / 16);
      const uint32_t* w = reinterpret_cast<const uint32_t*>(turned + d * stride + 16 * c);
      reinterpret_cast<uint4*>(q)[e] = uint4{w[0], w[1], w[2], w[3]};
    }
  } else {
    const int len = t.t1 - t.t0;
    for (int e = threadIdx.x; e < D * len; e += threads)
      q[e / len * block + t.t0 + e % len] = (int8_t)turned[e / len * stride + t.t0 + e % len];
  }
}

template <class E, int kPatches>
__global__ __launch_bounds__(256) void load_kernel(CacheLaunch g) {
  const Tile t = tile_of(g);
  if (t.id < 0) return;
  const bool values = blockIdx.z & 1;
  const int head = blockIdx.y, D = g.c.head_dim, block = g.c.block, stride = block + 4, threads = blockDim.x;
  const Rows& r = values ? g.v : g.k;
  const int64_t at = (int64_t)t.id * g.c.heads + head;
  const int8_t* q = (values ? g.c.v : g.c.k) + at * block * D;
  const float scale = (values ? g.c.v_scales : g.c.k_scales)[at];
  E* rows = reinterpret_cast<E*>(r.p) + t.row0 * r.row + head * r.head;
  const int n = patches(t, D);
  if (values) {
    const int c0 = t.t0 / 16, chunks = (t.t1 + 15) / 16 - c0;  // those that hold the slots
    for (int e = threadIdx.x; e < D * chunks; e += threads) {
      const int d = e / chunks, c = c0 + e % chunks;
      const uint4 w = *reinterpret_cast<const uint4*>(q + d * block + 16 * c);
      uint32_t* p = reinterpret_cast<uint32_t*>(turned + d * stride + 16 * c);
      p[0] = w.x, p[1] = w.y, p[2] = w.z, p[3] = w.w;
    }
    __syncthreads();
  }
  // the patches' rows, from byte(k, i): dimension i of the k-th token, sign-extended or with bytes above it
  auto write = [&](const Patch& at, auto byte) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (at.slot + k < t.t0 || at.slot + k >= t.t1) continue;
      Any8Of<E> v;
#pragma unroll
      for (int i = 0; i < 8; ++i) v.v[i] = (E)((float)(int8_t)byte(k, i) * scale);
      *reinterpret_cast<Any8Of<E>*>(rows + (at.slot + k) * r.row + at.d) = v;
    }
  };
#pragma unroll
  for (int u = 0; u < kPatches; ++u) {
    const int e = threadIdx.x + u * threads;
    if (e >= n) break;
    const Patch at = patch(t, D, e);
    if (values) {
      uint32_t w[8];  // four tokens each
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint32_t*>(turned + (at.d + i) * stride + at.slot);
      write(at, [&](int k, int i) { return w[i] >> (8 * k); });
    } else {
      uint2 w[4];  // (slots without a row: the first one that has a row again)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w[k] = *reinterpret_cast<const uint2*>(q + (at.slot + k >= t.t0 && at.slot + k < t.t1 ? at.slot + k : t.t0) * D + at.d);
      write(at, [&](int k, int i) { return (i < 4 ? w[k].x : w[k].y) >> (8 * (i % 4)); });
    }
  }
}

// ---- attention ------------------------------------------------------------------------------
// A wave works on 16-column tiles: column c of a sequence's cache head is row c / share with query head
// c % share of that head's group.  Tokens come 64 at a time, four chunks of 16 that each lie in one block:
//   S^T (tokens x columns) = K Q^T,  P = exp2(S - running maximum),  O^T (dimensions x columns) = V^T P^T,
// both on the 16x16x32 FP16 MFMA.  Lane 16 q + i holds, of the operands, row (token or dimension) i or
// column i at the reduction indices of quarter q, and of a result, column i at rows 4 q .. 4 q + 3.
// The order of tokens and dimensions along a reduction and of the rows of S^T is free, so it is taken such that nothing
// moves between lanes and every load is 16 bytes: row i of S^T's tile t is token 16 (i / 4) + 4 t + i % 4, so
// lane (q, i) gets the scores of tokens 16 q .. 16 q + 15, which are its part of P^T, and it loads the same
// 16 tokens of dimension i from V, 16 adjacent bytes as V is kept by dimension.
// int8 becomes FP16 exactly (a byte permute into 1024 + u, less 1152).  Queries become FP16 by a power
// of two per column that brings the largest below 2^15: what that loses lies 2^-40 below the largest.
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;     // per workgroup
constexpr int kTokens = 64;   // per step of a wave
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLargeScore = 1024.f;

union Halves {
  h8 v;
  h2 p[4];
  uint32_t w[4];
};

// Eight int8 (two words) as FP16.
__device__ __forceinline__ h8 widen(uint32_t a, uint32_t b) {
  Halves r;
  const h2 less = {(_Float16)-1152.f, (_Float16)-1152.f};
  a ^= 0x80808080u;
  b ^= 0x80808080u;
  r.w[0] = __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u);
  r.w[1] = __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u);
  r.w[2] = __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u);
  r.w[3] = __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u);
#pragma unroll
  for (int i = 0; i < 4; ++i) r.p[i] += less;
  return r.v;
}

// A product rounded by itself, never within a fused multiply-add.
__device__ __forceinline__ float product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// Largest over the four quarters of a column (NaN is passed over; it shows in the sum).
__device__ __forceinline__ float quarters_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

struct AttendArgs {
  AttendLaunch g;
  int32_t share, log2_block;
  int32_t chunk;       // tokens of a workgroup that splits them, a multiple of kWaves * kTokens
  int32_t splits;      // workgroups per sequence, head and column tile
  int32_t col_groups;  // column groups (workgroups along the columns) that max_rows asks for
  float* part;         // workspace: kPart(D) floats per column and split
};

// Partial results of column c (of sequence s, head h) and split x: maximum, sum, and D values.
__device__ __forceinline__ int64_t part_index(const AttendArgs& a, int s, int h, int64_t c, int x, int D) {
  const int64_t cols = (int64_t)a.g.b.max_rows * a.share;
  return ((((int64_t)s * a.g.c.heads + h) * cols + c) * a.splits + x) * (D + 4);
}

// A row's element type.
template <awe_dtype T>
struct RowType;
template <>
struct RowType<AWE_BF16> {
  using Elem = __bf16;
};
template <>
struct RowType<AWE_F16> {
  using Elem = _Float16;
};
// What a wave keeps of its 16 kQ columns: queries, running maximum, weights' sum and weighted values.
template <awe_dtype T, int D, int kQ>
struct Columns {
  using Elem = typename RowType<T>::Elem;
  int64_t col0, cols;  // the first one, and the sequence's
  int32_t last[kQ];    // tokens that a column sees
  float factor[kQ];    // of its scores, for powers of two
  h8 q[kQ][D / 32];
  f4 o[kQ][D / 16];
  float m[kQ], l[kQ];
  float e[kQ];  // log2 of the largest weight times its values' scale, as of the maximum's
  // Weights go into the second product as two FP16 numbers, the weight and what its rounding left, which hold
  // them to 2^-22 of a weight (and to 2^-40 of the column's largest).
  static constexpr int kParts = 2;

  __device__ __forceinline__ void begin(const AttendArgs& a, const Seq& s, int head, int64_t first) {
    const int q4 = (threadIdx.x & 63) >> 4, i16 = threadIdx.x & 15;
    col0 = first;
    cols = (int64_t)s.rows * a.share;
#pragma unroll
    for (int t = 0; t < kQ; ++t) {
      const int64_t col = col0 + 16 * t + i16;
      const bool ok = col < cols;
      const int32_t row = ok ? (int32_t)(col / a.share) : 0;
      last[t] = !ok ? 0 : a.g.causal ? s.len - s.rows + row + 1 : s.len;
      // (past the last column: the first one again, without any token)
      const Elem* p = reinterpret_cast<const Elem*>(a.g.q.p) + (int64_t)(s.row0 + row) * a.g.q.row +
                      (int64_t)(head * a.share + (ok ? col % a.share : 0)) * a.g.q.head;
      Any8Of<Elem> v[D / 32];
      float most = 0.f;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) v[j] = *reinterpret_cast<const Any8Of<Elem>*>(p + 64 * (j >> 1) + 16 * q4 + 8 * (j & 1));
#pragma unroll
      for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf((float)v[j].v[e]));
      most = quarters_max(most);
      const int ex = most > 0.f ? __builtin_amdgcn_frexp_expf(most) : 0;
#pragma unroll
      for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) q[t][j][e] = (_Float16)ldexpf(a.g.scale < 0.f ? -(float)v[j].v[e] : (float)v[j].v[e], 15 - ex);
      factor[t] = ldexpf(fabsf(a.g.scale) * kLog2e, ex - 15);
      m[t] = e[t] = -INFINITY;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) o[t][d] = f4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Softmax of the lane's 16 tokens (from token pv on) of its column, against the running maximum: scores to
  // weights.  They lie in one block, so the weights times its values' scale, on the power of two that makes the column's
  // largest 2^15, are exp2 of one linear function of the scores, and the weights' own sum is theirs by a factor.
  // FP16 keeps 11 bits of what is at least 2^-29 of the column's largest, and to 2^-40 of it of the rest; what
  // a column does not see, or gives no weight, takes no part in that.
  // The running maximum is a rounded product.  Beside a maximum of 2^10 that rounding, and the scales' logarithms'
  // in the sum with it, are up to 2^-14 each; from there on scores are first taken from the lane's largest, whose
  // product is rounded as the maximum is, so that no weight passes 2^15 however large the scores are.
  __device__ __forceinline__ void softmax(f4 (&sc)[kQ][4], h8 (&pf)[kParts][kQ][2], bool ok, float ks, float vs, int32_t pv) {
    const float log_vs = (float)__builtin_amdgcn_frexp_expf(vs) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(vs));
#pragma unroll
    for (int t = 0; t < kQ; ++t) {
      float f = factor[t] * ks;
      const int32_t see = ok ? last[t] - pv : 0;  // of the lane's tokens, the first so many
      if (__any(f == 0.f)) {  // (a masked score times 0 would be no number; one of a NaN or an infinity is none)
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[t][b][r] *= f == 0.f ? 0.f : 1.f;
        f = f == 0.f ? 1.f : f;
      }
      if (__any(see < 16)) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[t][b][r] = 4 * b + r < see ? sc[t][b][r] : -INFINITY;
      }
      float top = sc[t][0][0];
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, sc[t][b][r]);
      const float most = product(top, f), now = fmaxf(m[t], quarters_max(most));
      const float base = now == -INFINITY ? 0.f : now;
      const float reach = (most - base) + log_vs;  // log2 of the lane's largest weight times the scale
      const float held = e[t] + (m[t] - base);
      e[t] = fmaxf(held, quarters_max(reach));
      const float ref = e[t] == -INFINITY ? 0.f : e[t];
      const float drop = __builtin_amdgcn_exp2f(m[t] - base), keep = __builtin_amdgcn_exp2f(held - ref);
      const bool some = reach > ref - 40.f;  // (FP16 holds no smaller weight; but it counts in the sum)
      const float log_w = some ? (log_vs - ref) + 15.f : 0.f, per_w = some ? __builtin_amdgcn_exp2f(-log_w) : 1.f;
      float shift = log_w - base;
      const bool large = fabsf(base) > kLargeScore;
      if (__any(large)) {  // (what other columns of the wave need changes nothing in this one)
        const float least = large && top != -INFINITY ? top : 0.f;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[t][b][r] -= least;
        shift = large ? (product(least, f) - base) + log_w : shift;
      }
      m[t] = now;
      float sum = 0.f;
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const f2 p = {__builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][b][r], f, shift)),
                        __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][b][r + 1], f, shift))};
          sum += p[0] + p[1];
          const h2 high = __builtin_convertvector(p, h2);
          const f2 left = {__builtin_fmaf((float)high[0], -1.f, p[0]), __builtin_fmaf((float)high[1], -1.f, p[1])};
          const h2 low = __builtin_convertvector(left, h2);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            pf[0][t][b >> 1][4 * (b & 1) + r + i] = high[i];
            pf[1][t][b >> 1][4 * (b & 1) + r + i] = low[i];
          }
        }
      l[t] = l[t] * drop + sum * per_w;
      if (__any(!some)) {
#pragma unroll
        for (int u = 0; u < 2 * kParts; ++u)
          if (!some) pf[u >> 1][t][u & 1] = h8{};
      }
      if (__any(keep != 1.f)) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[t][d] *= keep;
      }
    }
  }

  // The sums of the quarters, and the values in their own scale.
  __device__ __forceinline__ void end() {
#pragma unroll
    for (int t = 0; t < kQ; ++t) {
      l[t] += __shfl_xor(l[t], 16);
      l[t] += __shfl_xor(l[t], 32);
      const float whole = e[t] == -INFINITY ? 0.f : ceilf(e[t]), part = e[t] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(e[t] - whole);
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[t][d][r] = ldexpf(o[t][d][r] * part, (int)whole - 15);
    }
  }
};

// Where a column's result goes.
template <class Elem>
__device__ __forceinline__ Elem* result(const AttendArgs& a, const Seq& s, int head, int64_t col) {
  return reinterpret_cast<Elem*>(a.g.o.p) + (int64_t)(s.row0 + col / a.share) * a.g.o.row +
         (head * a.share + col % a.share) * a.g.o.head;
}

// The cache as a lane sees it, 64 tokens a step: keys' row i of score tile t is token 16 (i / 4) + 4 t + i % 4,
// values' tokens are 16 q .. 16 q + 15.
template <int D>
struct Tokens {
  const awe_cache& c;
  const int32_t* table;
  int64_t tile;
  int32_t len, head, log2_block, key, value, k_lane, v_lane;

  __device__ __forceinline__ Tokens(const AttendArgs& a, int sid, int head_, int32_t len_)
      : c(a.g.c), table(a.g.b.blocks + (int64_t)sid * a.g.b.ld_blocks), tile((int64_t)a.g.c.block * D), len(len_), head(head_), log2_block(a.log2_block) {
    const int q4 = (threadIdx.x & 63) >> 4, i16 = threadIdx.x & 15;
    key = 16 * (i16 >> 2);
    value = 16 * q4;
    k_lane = (i16 & 3) * D + 16 * q4;
    v_lane = i16 * c.block;
  }
  // The block ids of a step's chunks: as they are in the table, -1 past the sequence's end.
  __device__ __forceinline__ void ids(int32_t t0, int32_t& k, int32_t& v) const {
    k = t0 + key < len ? table[(t0 + key) >> log2_block] : -1;
    v = t0 + value < len ? table[(t0 + value) >> log2_block] : -1;
  }
  __device__ __forceinline__ bool valid(int32_t id) const { return id >= 0 && id < c.num_blocks; }
  __device__ __forceinline__ int64_t at(int32_t id) const {  // (without a valid id block 0 is read, and has no weight)
    return (int64_t)(valid(id) ? id : 0) * c.heads + head;
  }
  __device__ __forceinline__ const int8_t* keys(int32_t t0, int32_t id) const {
    return c.k + at(id) * tile + ((t0 + key) & (c.block - 1)) * D + k_lane;  // + 4 t D + 64 d
  }
  __device__ __forceinline__ const int8_t* values(int32_t t0, int32_t id) const {
    return c.v + at(id) * tile + ((t0 + value) & (c.block - 1)) + v_lane;  // + 16 d block
  }
};

// Few columns: a workgroup has 16 of them and a chunk of the tokens, which its waves take 64 at a time in
// turn.  Bound by the cache's bytes: a wave has a step's keys and values in flight while it works on
// the step before.  Traced, 64 sequences of up to 8192 tokens, 8 heads of 128, take 119 us (549 MB, 4.6 TB/s; a copy
// reaches 5.2), one sequence of 65,536 28 us (134 MB, 4.8 TB/s).  It goes through all tokens, also those
// that a causal row does not see: rows are few here.
template <awe_dtype T, int D>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 1 : 2) void attend_split_kernel(AttendArgs a) {
  using Elem = typename RowType<T>::Elem;
  const awe_cache& c = a.g.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q4 = lane >> 4, i16 = lane & 15;
  const int sid = blockIdx.z, head = blockIdx.y;
  const int group = blockIdx.x / a.splits, split = blockIdx.x % a.splits;
  const Seq s = sequence(a.g.b, sid, false, a.g.flag, threadIdx.x == 0 && blockIdx.x == 0);
  const int64_t cols = (int64_t)s.rows * a.share, col0 = (int64_t)group * 16;
  if (col0 >= cols) return;
  // tokens of this workgroup; a sequence without any is one empty chunk
  const int32_t from = split * a.chunk;
  if (split > 0 && from >= s.len) return;
  int32_t to = s.len - from > a.chunk ? from + a.chunk : s.len;
  if (c.num_blocks == 0 && to > from) {  // every id is out of range
    to = from;
    if (a.g.flag != nullptr) *a.g.flag = 1;
  }
  Columns<T, D, 1> x;
  x.begin(a, s, head, col0);
  const Tokens<D> tokens(a, sid, head, s.len);

  constexpr int32_t step = kWaves * kTokens;
  u4 kr[4][D / 64], vr[D / 16];
  float ks = 0.f, vs = 0.f;
  auto fetch_keys = [&](int32_t t0, int32_t id) {
    const int8_t* p = tokens.keys(t0, id);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int d = 0; d < D / 64; ++d) kr[t][d] = *reinterpret_cast<const u4*>(p + 4 * t * D + 64 * d);
  };
  auto fetch_values = [&](int32_t t0, int32_t id) {
    const int8_t* p = tokens.values(t0, id);
#pragma unroll
    for (int d = 0; d < D / 16; ++d) vr[d] = *reinterpret_cast<const u4*>(p + 16 * d * c.block);
    ks = c.k_scales[tokens.at(id)];
    vs = c.v_scales[tokens.at(id)];
  };
  int32_t t0 = from + wave * kTokens;
  int32_t ik = -1, iv = -1, ik1 = -1, iv1 = -1;
  if (t0 < to) {
    tokens.ids(t0, ik, iv);
    fetch_keys(t0, ik);
    fetch_values(t0, iv);
    tokens.ids(t0 + step, ik1, iv1);
  }
  for (; t0 < to; t0 += step) {
    const bool ok = tokens.valid(iv);
    const int32_t pv = t0 + 16 * q4;
    if (!ok && pv < s.len && a.g.flag != nullptr) *a.g.flag = 1;
    f4 sc[1][4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      sc[0][b] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < D / 32; ++j)
        sc[0][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen(kr[b][j >> 1][2 * (j & 1)], kr[b][j >> 1][2 * (j & 1) + 1]), x.q[0][j], sc[0][b], 0, 0, 0);
    }
    const float ks0 = ok ? ks : 0.f, vs0 = ok ? vs : 0.f;
    if (t0 + step < to) fetch_keys(t0 + step, ik1);
    h8 pf[x.kParts][1][2];
    x.softmax(sc, pf, ok, ks0, vs0, pv);
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const h8 vf = widen(vr[d][2 * e], vr[d][2 * e + 1]);
#pragma unroll
        for (int u = 0; u < x.kParts; ++u) x.o[0][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[u][0][e], x.o[0][d], 0, 0, 0);
      }
    if (t0 + step < to) {
      fetch_values(t0 + step, iv1);
      iv = iv1;
      tokens.ids(t0 + 2 * step, ik1, iv1);
    }
  }
  x.end();

  // the waves' parts of each column, through LDS: 64 dimensions at a time
  constexpr int kDim = 64;
  __shared__ float ow[kWaves][16][kDim + 4], mw[kWaves][16], lw[kWaves][16];
  const bool whole = s.len <= a.chunk;
  const int cl = threadIdx.x >> 4, d = 4 * (threadIdx.x & 15);  // this thread's column and dimensions
  const int64_t col = col0 + cl;
#pragma unroll
  for (int d0 = 0; d0 < D; d0 += kDim) {
    __syncthreads();
    if (q4 == 0 && d0 == 0) {
      mw[wave][i16] = x.m[0];
      lw[wave][i16] = x.l[0];
    }
#pragma unroll
    for (int e = 0; e < kDim / 16; ++e) *reinterpret_cast<f4*>(&ow[wave][i16][16 * e + 4 * q4]) = x.o[0][d0 / 16 + e];
    __syncthreads();
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, mw[w][cl]);
    f4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(mw[w][cl] - (top == -INFINITY ? 0.f : top));
      sum += lw[w][cl] * f;
      v += *reinterpret_cast<const f4*>(&ow[w][cl][d]) * f;
    }
    if (col >= cols) continue;
    if (whole) {
      Elem* out = result<Elem>(a, s, head, col) + d0 + d;
#pragma unroll
      for (int r = 0; r < 4; ++r) out[r] = (Elem)(sum == 0.f ? 0.f : v[r] / sum);
    } else {
      float* p = a.part + part_index(a, sid, head, col, split, D);
      *reinterpret_cast<f4*>(p + 4 + d0 + d) = v;
      if (d0 == 0 && d == 0) {
        p[0] = top;
        p[1] = sum;
      }
    }
  }
}

// Asks for the order of a block of n reads from LDS with kQ products each: six reads ahead of the products.
template <int n, int kQ>
__device__ __forceinline__ void reads_ahead() {
  constexpr int kAhead = 6, kMfma = 0x8, kRead = 0x100;
  __builtin_amdgcn_sched_group_barrier(kRead, kAhead, 0);
#pragma unroll
  for (int i = 0; i < n - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(kMfma, kQ, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kMfma, kAhead * kQ, 0);
}

// Many columns: each of the kW waves has 16 kQ columns, and together they go through the tokens, 64 a step.
// A step's keys and values become FP16 once per workgroup: a wave fetches its share as it would for itself, and puts the
// operands into LDS lane by lane, where every wave reads them as they are (twice: a step's while the
// next one's are on their way).  Bound by vector instructions, softmax's most of all (61 % of a CU's busy cycles), and
// by products (36 %): calls back to back, prompts that take 164 GFLOP run 308-316 us (the FP16 MFMA alone: 131, and
// half as much again for the weights' second numbers; with weights of one number each: 265).  Workgroups of 256
// columns were slower (387 instead of 251, with one number).
template <awe_dtype T, int D, int kQ, int kW>
__global__ __launch_bounds__(64 * kW, D == 256 ? 1 : 2) void attend_rows_kernel(AttendArgs a) {
  using Elem = typename RowType<T>::Elem;
  constexpr int kKeys = 4 * D / 32, kValues = D / 16 * 2;  // operands of a step
  constexpr int kLoads = D / 16;                            // 16-byte loads of a lane: of keys, and of values
  const awe_cache& c = a.g.c;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q4 = lane >> 4, i16 = lane & 15;
  // The last columns see the most tokens: they go first.  Heads are next to each other, so that with
  // eight of them the workgroups of a head, which read the same tokens, are on one XCD (293 us instead of
  // 316 for prompts of up to 2048 tokens, as the kernel was then; all sequences' last columns first took 491).
  const uint32_t per_seq = (uint32_t)a.col_groups * a.g.c.heads, in = blockIdx.x % per_seq;
  const int head = in % a.g.c.heads, sid = blockIdx.x / per_seq, group = a.col_groups - 1 - (int)(in / a.g.c.heads);
  const Seq s = sequence(a.g.b, sid, false, a.g.flag, threadIdx.x == 0 && group == 0);
  const int64_t cols = (int64_t)s.rows * a.share, first = (int64_t)group * kW * 16 * kQ;
  if (first >= cols) return;
  int32_t to = s.len;
  if (a.g.causal) {  // the last column's row sees the most tokens
    const int64_t end = std::min<int64_t>(first + kW * 16 * kQ, cols);
    to = std::min(to, s.len - s.rows + (int32_t)((end - 1) / a.share) + 1);
  }
  if (c.num_blocks == 0 && to > 0) {  // every id is out of range
    to = 0;
    if (a.g.flag != nullptr) *a.g.flag = 1;
  }
  Columns<T, D, kQ> x;
  x.begin(a, s, head, first + wave * 16 * kQ);
  const Tokens<D> tokens(a, sid, head, s.len);

  extern __shared__ uint8_t attend_lds[];
  h8(*lds)[kKeys + kValues][64] = reinterpret_cast<h8(*)[kKeys + kValues][64]>(attend_lds);
  // this wave's share of a step: loads wave, wave + kW, ... of the 2 kLoads
  constexpr int kMine = 2 * kLoads / kW;
  static_assert(kMine * kW == 2 * kLoads, "the waves share the loads evenly");
  u4 raw[kMine];
  float ks = 0.f, vs = 0.f;
  auto fetch = [&](int32_t t0, int32_t ik, int32_t iv) {
    const int8_t* pk = tokens.keys(t0, ik);
    const int8_t* pv = tokens.values(t0, iv);
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const int load = wave + n * kW;
      const int8_t* p = load < kLoads ? pk + 4 * (load / (D / 64)) * D + 64 * (load % (D / 64)) : pv + 16 * (load - kLoads) * c.block;
      raw[n] = *reinterpret_cast<const u4*>(p);
    }
    ks = c.k_scales[tokens.at(iv)];
    vs = c.v_scales[tokens.at(iv)];
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const int load = wave + n * kW;
      lds[buf][2 * load][lane] = widen(raw[n][0], raw[n][1]);
      lds[buf][2 * load + 1][lane] = widen(raw[n][2], raw[n][3]);
    }
  };
  int32_t ik = -1, iv = -1, ik1 = -1, iv1 = -1;
  if (to > 0) {
    tokens.ids(0, ik, iv);
    fetch(0, ik, iv);
    tokens.ids(kTokens, ik1, iv1);
    put(0);
  }
  int buf = 0;
  for (int32_t t0 = 0; t0 < to; t0 += kTokens, buf ^= 1) {
    __syncthreads();  // the step's operands are there, and nobody reads the other half any more
    const bool ok = tokens.valid(iv), more = t0 + kTokens < to;
    const int32_t pv = t0 + 16 * q4;
    if (!ok && pv < s.len && a.g.flag != nullptr) *a.g.flag = 1;
    const float ks0 = ok ? ks : 0.f, vs0 = ok ? vs : 0.f;
    if (more) {
      fetch(t0 + kTokens, ik1, iv1);
      iv = iv1;
      tokens.ids(t0 + 2 * kTokens, ik1, iv1);
    }
    f4 sc[kQ][4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
#pragma unroll
      for (int t = 0; t < kQ; ++t) sc[t][b] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        const h8 kf = lds[buf][b * (D / 32) + j][lane];
#pragma unroll
        for (int t = 0; t < kQ; ++t) sc[t][b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, x.q[t][j], sc[t][b], 0, 0, 0);
      }
    }
    reads_ahead<kKeys, kQ>();
    h8 pf[x.kParts][kQ][2];
    x.softmax(sc, pf, ok, ks0, vs0, pv);
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const h8 vf = lds[buf][kKeys + 2 * d + e][lane];
#pragma unroll
        for (int t = 0; t < kQ; ++t)
#pragma unroll
          for (int u = 0; u < x.kParts; ++u) x.o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[u][t][e], x.o[t][d], 0, 0, 0);
      }
    reads_ahead<kValues, kQ * x.kParts>();
    if (more) put(buf ^ 1);
  }
  x.end();
#pragma unroll
  for (int t = 0; t < kQ; ++t) {
    const int64_t col = x.col0 + 16 * t + i16;
    if (col >= cols) continue;
    Elem* out = result<Elem>(a, s, head, col);
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) out[16 * d + 4 * q4 + r] = (Elem)(x.l[t] == 0.f ? 0.f : x.o[t][d][r] / x.l[t]);
  }
}

// Joins the splits of a column: out = sum_x 2^(m_x - m) v_x / sum_x 2^(m_x - m) l_x, m the largest m_x.  D / 64 dimensions
// per lane, eight splits at a time in flight: a wave per column, or where there are more splits than kJoinAlone
// the waves of a workgroup, in turn.  Bound by latency: 4.8 us for 64 splits of 32 columns.
constexpr int kJoinAlone = 16;
template <awe_dtype T, int D>
__global__ __launch_bounds__(64 * kWaves) void attend_join_kernel(AttendArgs a) {
  using Elem = typename RowType<T>::Elem;
  constexpr int kAtOnce = 8;
  const int sid = blockIdx.z, head = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Seq s = sequence(a.g.b, sid, false, nullptr, false);
  const bool alone = a.splits <= kJoinAlone;
  const int64_t col = alone ? (int64_t)blockIdx.x * kWaves + wave : blockIdx.x;
  if (s.len <= a.chunk || col >= (int64_t)s.rows * a.share) return;
  const int n = (s.len + a.chunk - 1) / a.chunk;
  const float* p = a.part + part_index(a, sid, head, col, 0, D);
  float top = -INFINITY;
  for (int x = lane; x < n; x += 64) top = fmaxf(top, p[(int64_t)x * (D + 4)]);
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f, v[D / 64] = {};
  const int in_turn = alone ? 1 : kWaves;
  for (int x0 = alone ? 0 : wave; x0 < n; x0 += in_turn * kAtOnce) {
    float m[kAtOnce], l[kAtOnce], o[kAtOnce][D / 64];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int x = x0 + u * in_turn;
      const float* px = p + (int64_t)(x < n ? x : x0) * (D + 4);
      m[u] = x < n ? px[0] : -INFINITY;
      l[u] = px[1];
#pragma unroll
      for (int d = 0; d < D / 64; ++d) o[u][d] = px[4 + 64 * d + lane];
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      if (x0 + u * in_turn >= n) break;
      const float f = __builtin_amdgcn_exp2f(m[u] - base);
      sum += l[u] * f;
#pragma unroll
      for (int d = 0; d < D / 64; ++d) v[d] += o[u][d] * f;
    }
  }
  Elem* out = result<Elem>(a, s, head, col);
  if (alone) {
#pragma unroll
    for (int d = 0; d < D / 64; ++d) out[64 * d + lane] = (Elem)(sum == 0.f ? 0.f : v[d] / sum);
    return;
  }
  __shared__ float parts[kWaves][D + 1];
#pragma unroll
  for (int d = 0; d < D / 64; ++d) parts[wave][64 * d + lane] = v[d];
  if (lane == 0) parts[wave][D] = sum;
  __syncthreads();
  for (int d = threadIdx.x; d < D; d += 64 * kWaves) {
    float t = 0.f, w = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      t += parts[k][D];
      w += parts[k][d];
    }
    out[d] = (Elem)(t == 0.f ? 0.f : w / t);
  }
}

// Grid (blocks that can be touched, heads, 2 * sequences); sequences go over in parts of the grid's limit.
template <class K>
awe_status launch_blocks(K kernel, CacheLaunch g, int threads, const char* what, hipStream_t stream) {
  // n rows touch at most 1 + ceil((n - 1) / block) blocks
  const unsigned x = (unsigned)((std::min(g.b.max_rows, g.b.rows) + g.c.block - 2) / g.c.block + 1);
  const int32_t all = g.b.sequences;
  for (int32_t s = 0; s < all; s += 32767) {
    CacheLaunch part = g;
    part.b.sequences = all - s < 32767 ? all - s : 32767;
    part.b.starts += s;
    part.b.lengths += s;
    part.b.blocks += s * g.b.ld_blocks;
    hipLaunchKernelGGL(kernel, dim3(x, (unsigned)g.c.heads, 2u * part.b.sequences), dim3(threads), turned_bytes(g.c), stream, part);
    const awe_status st = launched(what);
    if (st != AWE_OK) return st;
  }
  return AWE_OK;
}

template <class E>
awe_status launch_type(const CacheLaunch& g, bool load, hipStream_t stream) {
  const int patches = g.c.block / 4 * (g.c.head_dim / 8), threads = std::min(256, (patches + 63) / 64 * 64);
  const char* what = load ? "cache load launch" : "cache store launch";
  auto launch = [&](auto n) {
    constexpr int k = decltype(n)::value;
    return load ? launch_blocks(load_kernel<E, k>, g, threads, what, stream) : launch_blocks(store_kernel<E, k>, g, threads, what, stream);
  };
  return patches <= threads       ? launch(std::integral_constant<int, 1>{})
         : patches <= 2 * threads ? launch(std::integral_constant<int, 2>{})
                                  : launch(std::integral_constant<int, 4>{});  // 128 x 256 at most
}
awe_status launch_cache(const CacheLaunch& g, bool load, hipStream_t stream) {
  return g.type == AWE_F32    ? launch_type<float>(g, load, stream)
         : g.type == AWE_BF16 ? launch_type<bf16>(g, load, stream)
                              : launch_type<f16>(g, load, stream);
}

}  // namespace

awe_status launch_cache_store(const CacheLaunch& g, hipStream_t stream) { return launch_cache(g, false, stream); }
awe_status launch_cache_load(const CacheLaunch& g, hipStream_t stream) { return launch_cache(g, true, stream); }

namespace {
template <awe_dtype T, int D>
awe_status launch_attend(const AttendArgs& a, bool own_columns, hipStream_t stream) {
  const unsigned heads = (unsigned)a.g.c.heads, seqs = (unsigned)a.g.b.sequences;
  if (own_columns) {
    constexpr int kQ = D == 256 ? 1 : 2, kW = kRowsColumns / (16 * kQ), bytes = 2 * (4 * D / 32 + D / 16 * 2) * 1024;
    static std::mutex mu;
    static std::set<int> done;
    auto kernel = attend_rows_kernel<T, D, kQ, kW>;
    const awe_status st = set_lds_limit(reinterpret_cast<const void*>(kernel), bytes, mu, done);
    if (st != AWE_OK) return st;
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.col_groups * heads * seqs), dim3(64 * kW), bytes, stream, a);
    return launched("attention launch");
  }
  const dim3 block(64 * kWaves);
  hipLaunchKernelGGL((attend_split_kernel<T, D>), dim3((unsigned)(a.col_groups * a.splits), heads, seqs), block, 0, stream, a);
  awe_status st = launched("attention launch");
  if (st != AWE_OK || a.splits == 1) return st;
  const int64_t cols = a.g.b.max_rows * a.share;
  hipLaunchKernelGGL((attend_join_kernel<T, D>), dim3((unsigned)(a.splits <= kJoinAlone ? (cols + kWaves - 1) / kWaves : cols), heads, seqs), block, 0, stream, a);
  return launched("attention join launch");
}
}  // namespace

awe_status launch_cache_attend(const AttendLaunch& g, hipStream_t stream) {
  const AttendPlan plan = plan_attend(g.c, g.b, g.q_heads);
  // sequences go over in parts of the grid's limit
  int32_t most = 65535;
  if (plan.own_columns) {
    const int64_t each = (int64_t)plan.groups * g.c.heads;
    if (each > 0x7fffff) {
      set_error("too many rows and heads");
      return AWE_ERR_UNSUPPORTED;
    }
    most = (int32_t)(0x7fffff / each);
  }
  for (int32_t s = 0; s < g.b.sequences; s += most) {
    AttendArgs a{};
    a.g = g;
    a.g.b.sequences = std::min(most, g.b.sequences - s);
    a.g.b.starts += s;
    a.g.b.lengths += s;
    a.g.b.blocks += s * g.b.ld_blocks;
    if (a.g.b.max_rows > a.g.b.rows) a.g.b.max_rows = a.g.b.rows;
    a.share = g.q_heads / g.c.heads;
    a.log2_block = __builtin_ctz((unsigned)g.c.block);
    a.chunk = plan.chunk;
    a.splits = plan.splits;
    a.col_groups = plan.groups;
    a.part = reinterpret_cast<float*>(g.ws);
    auto launch = [&](auto type) {
      constexpr awe_dtype T = decltype(type)::value;
      return g.c.head_dim == 64    ? launch_attend<T, 64>(a, plan.own_columns, stream)
             : g.c.head_dim == 128 ? launch_attend<T, 128>(a, plan.own_columns, stream)
                                   : launch_attend<T, 256>(a, plan.own_columns, stream);
    };
    const awe_status st = g.type == AWE_BF16 ? launch(std::integral_constant<awe_dtype, AWE_BF16>{})
                                             : launch(std::integral_constant<awe_dtype, AWE_F16>{});
    if (st != AWE_OK) return st;
  }
  return AWE_OK;
}

}  // namespace awe

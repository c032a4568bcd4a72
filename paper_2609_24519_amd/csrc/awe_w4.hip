// Products with 4-bit weights in scaled groups (awe_gemm_w4):
//   Y[i,j] = sx[i] sum_g s[j,g] sum_{k in g} X[i,k] (u[j,k] - z[j,g]).
//
// A code becomes a number of X's type by being placed in the mantissa of 16: 16 + u, a shift and one
// and-or for two codes (exact in BF16 and FP16; for int8 X the codes are bytes as they are).  The matrix
// instruction sums x (16 + u) over a group in FP32 (int32 for int8), and
//   sum x (u - z) = sum x (16 + u) - (16 + z) sum x,
// with sum x from the same instruction on a column of ones.  The group's scale then multiplies the
// FP32 sum, so neither scales nor weights are ever rounded.
#include "quant_device.h"

namespace awe {
namespace {

typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// 16 and 8 bytes from any address.
struct __attribute__((packed)) Any16 {
  uint32_t w[4];
};
struct __attribute__((packed)) Any8 {
  uint32_t w[2];
};

// What depends on X's type: eight codes (a word) or eight elements of X as one lane's operand of a
// 16 x 16 x 32 product, in one order of the eight (0 4 1 5 2 6 3 7; for int8 the even ones, then the odd).
template <awe_dtype T>
struct Kind;

// The magic number in a vector register, where an and-or can take it beside a constant mask (from two
// constants the compiler makes two instructions).
__device__ __forceinline__ uint32_t in_vector(uint32_t x) {
  asm("" : "+v"(x));
  return x;
}

// Pairs (0, 4), (1, 5), (2, 6), (3, 7) of eight 16-bit elements.
__device__ __forceinline__ u4 paired(const u4& x) {
  return u4{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
            __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
}

template <>
struct Kind<AWE_BF16> {
  using Elem = uint16_t;
  using Raw = u4;  // eight elements
  using Op = u4;
  using Acc = f4;
  using Sum = float;
  static constexpr float kBias = 16.f;
  static __device__ __forceinline__ Sum add(const Op& x, Sum s) {  // the elements' sum
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t pair = x[w];  // (bit_cast of the element itself takes the first one)
      s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, pair), __builtin_bit_cast(b2, 0x3f803f80u), s, false);
    }
    return s;
  }
  static __device__ __forceinline__ uint32_t magic() { return in_vector(0x41804180u); }  // 16
  static __device__ __forceinline__ Op codes(uint32_t w, uint32_t magic) {
    constexpr uint32_t mask = 0x00780078u;  // a code's place in the mantissa of 16
    return u4{((w << 3) & mask) | magic, ((w >> 1) & mask) | magic, ((w >> 5) & mask) | magic, ((w >> 9) & mask) | magic};
  }
  static __device__ __forceinline__ Op elems(const Raw& x) { return paired(x); }
  static __device__ __forceinline__ Op ones() { return u4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}; }
  static __device__ __forceinline__ Acc zero() { return f4{0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ Acc mul(const Op& a, const Op& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  }
};

template <>
struct Kind<AWE_F16> {
  using Elem = uint16_t;
  using Raw = u4;
  using Op = u4;
  using Acc = f4;
  using Sum = float;
  static constexpr float kBias = 16.f;
  static __device__ __forceinline__ Sum add(const Op& x, Sum s) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t pair = x[w];
      s = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, pair), __builtin_bit_cast(h2, 0x3c003c00u), s, false);
    }
    return s;
  }
  static __device__ __forceinline__ uint32_t magic() { return in_vector(0x4c004c00u); }
  static __device__ __forceinline__ Op codes(uint32_t w, uint32_t magic) {
    constexpr uint32_t mask = 0x03c003c0u;
    return u4{((w << 6) & mask) | magic, ((w << 2) & mask) | magic, ((w >> 2) & mask) | magic, ((w >> 6) & mask) | magic};
  }
  static __device__ __forceinline__ Op elems(const Raw& x) { return paired(x); }
  static __device__ __forceinline__ Op ones() { return u4{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u}; }
  static __device__ __forceinline__ Acc zero() { return f4{0.f, 0.f, 0.f, 0.f}; }
  static __device__ __forceinline__ Acc mul(const Op& a, const Op& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
};

template <>
struct Kind<AWE_I8> {
  using Elem = uint8_t;
  using Raw = uint64_t;
  using Op = uint64_t;
  using Acc = i4;
  using Sum = int;
  static constexpr int kBias = 0;
  static __device__ __forceinline__ Sum add(Op x, Sum s) {
    s = __builtin_amdgcn_sdot4((int)x, 0x01010101, s, false);
    return __builtin_amdgcn_sdot4((int)(x >> 32), 0x01010101, s, false);
  }
  static __device__ __forceinline__ uint32_t magic() { return 0; }
  static __device__ __forceinline__ Op codes(uint32_t w, uint32_t) {
    return (uint64_t)(w & 0x0f0f0f0fu) | (uint64_t)((w >> 4) & 0x0f0f0f0fu) << 32;
  }
  static __device__ __forceinline__ Op elems(Raw x) {
    const uint32_t a = (uint32_t)x, b = (uint32_t)(x >> 32);
    return (uint64_t)__builtin_amdgcn_perm(b, a, 0x06040200u) | (uint64_t)__builtin_amdgcn_perm(b, a, 0x07050301u) << 32;
  }
  static __device__ __forceinline__ Op ones() { return 0x0101010101010101ull; }
  static __device__ __forceinline__ Acc zero() { return i4{0, 0, 0, 0}; }
  static __device__ __forceinline__ Acc mul(Op a, Op b, const Acc& c) {
    return __builtin_amdgcn_mfma_i32_16x16x32_i8((long)a, (long)b, c, 0, 0, 0);
  }
};

// Eight elements of X from any address.
template <awe_dtype T>
__device__ __forceinline__ typename Kind<T>::Raw load8(const typename Kind<T>::Elem* p) {
  if constexpr (T == AWE_I8) {
    const Any8 a = *reinterpret_cast<const Any8*>(p);
    return (uint64_t)a.w[0] | (uint64_t)a.w[1] << 32;
  } else {
    const Any16 a = *reinterpret_cast<const Any16*>(p);
    return u4{a.w[0], a.w[1], a.w[2], a.w[3]};
  }
}
// Words of the four quarters of a wave transposed: word j of quarter q becomes word q of quarter j.
__device__ __forceinline__ u4 across_quarters(u4 w) {
  auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
  auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  return u4{c[0], c[1], d[0], d[1]};
}

// The same, such that quarter q's words 2 c and 2 c + 1 are the ones at indices 64 c + 16 q .. + 15: sixteen
// adjacent elements per quarter.
__device__ __forceinline__ u4 across_quarters_by_16(u4 w) {
  auto a = __builtin_amdgcn_permlane16_swap(w[0], w[2], false, false);
  auto b = __builtin_amdgcn_permlane16_swap(w[1], w[3], false, false);
  auto c = __builtin_amdgcn_permlane32_swap(a[0], a[1], false, false);
  auto d = __builtin_amdgcn_permlane32_swap(b[0], b[1], false, false);
  return u4{c[0], d[0], c[1], d[1]};
}

// ---- results whose sums in FP32 leave its range ----------------------------------------------
// With an infinity, or elements so large that 16 and more times them pass FP32's range, sum x (16 + u) and
// (16 + z) sum x are infinite where the formula's sum need not be.  Such a result is not finite, as no infinity or NaN
// leaves a sum again, and is computed once more: in a row with a NaN it is NaN either way, in a row with infinities
// their terms decide, and otherwise a wave adds the formula's terms in 64 bits, which hold them all, a result at a time.
// Bound by the latency of loads: 512 rows against 8192 x 8192 (0.09 ms) take 0.14 ms with an infinity in one row, 1.9
// with one in each, 0.34 with a NaN in each, 0.8 with one row of elements near 2^122 and 40 with all of them such.
template <awe_dtype T>
struct Eight {
  typename Kind<T>::Elem v[8];

  // Elements k .. k + 7 of a row of K, 0 past its end.
  __device__ __forceinline__ Eight(const typename Kind<T>::Elem* row, uint32_t k, uint32_t K) {
    if (k + 8 <= K) {
      *this = __builtin_bit_cast(Eight, load8<T>(row + k));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = k + i < K ? row[k + i] : 0;
    }
  }
  // Of its elements: bit i if the i-th is an infinity, bit 8 if one is a NaN.
  __device__ __forceinline__ uint32_t special() const {
    constexpr uint32_t infinity = T == AWE_BF16 ? 0x7f80u : 0x7c00u;
    uint32_t r = 0;
    if constexpr (T != AWE_I8)
#pragma unroll
      for (int i = 0; i < 8; ++i) r |= (v[i] & 0x7fffu) == infinity ? 1u << i : (v[i] & 0x7fffu) > infinity ? 256u : 0u;
    return r;
  }
  __device__ __forceinline__ double value(int i) const {
    if constexpr (T == AWE_I8) return (double)(int8_t)v[i];
    if constexpr (T == AWE_BF16) return (double)__builtin_bit_cast(float, (uint32_t)v[i] << 16);
    return (double)__builtin_bit_cast(_Float16, (uint16_t)v[i]);
  }
};

// A scale and a zero point as the formula has them.
__device__ __forceinline__ float scale_at(const W4Launch& g, int64_t j, int64_t grp) {
  return g.s_type == AWE_F32    ? reinterpret_cast<const float*>(g.scales)[j * g.lds + grp]
         : g.s_type == AWE_BF16 ? (float)reinterpret_cast<const bf16*>(g.scales)[j * g.lds + grp]
                                : (float)reinterpret_cast<const f16*>(g.scales)[j * g.lds + grp];
}
__device__ __forceinline__ int zero_at(const W4Launch& g, int64_t j, int64_t grp) {
  return g.zeros != nullptr ? g.zeros[j * g.ldz + grp] : 8;
}

// Y[m,j] without its rounding, on every lane.
template <awe_dtype T>
__device__ __forceinline__ double by_definition(const W4Launch& g, int64_t m, int64_t j) {
  const auto* x = reinterpret_cast<const typename Kind<T>::Elem*>(g.x) + m * g.ldx;
  const uint8_t* w = g.w + j * g.ldw;
  const uint32_t K = (uint32_t)g.K, group = (uint32_t)g.group;
  double sum = 0.;
#pragma unroll 1
  for (uint32_t k = 8 * (threadIdx.x & 63); k < K; k += 512) {  // (eight indices lie in one group)
    const int64_t grp = k / group;
    const float s = scale_at(g, j, grp);
    const int z = zero_at(g, j, grp);
    const Eight<T> e(x, k, K);
    uint8_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = k + 2 * i < K ? w[k / 2 + i] : 0;
    double part = 0.;
#pragma unroll
    for (int i = 0; i < 8; ++i) part += e.value(i) * (double)((int)(c[i / 2] >> (4 * (i & 1)) & 15) - z);
    sum += (double)s * part;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  return g.x_scales != nullptr ? sum * (double)g.x_scales[m] : sum;
}

// Y[m,j] of the lanes with mine set, each with its j, for a row m with infinities: their terms alone, as the
// others' sum is finite.
template <awe_dtype T>
__device__ __forceinline__ float by_infinities(const W4Launch& g, bool mine, int64_t m, int64_t j) {
  const auto* x = reinterpret_cast<const typename Kind<T>::Elem*>(g.x) + m * g.ldx;
  const uint32_t K = (uint32_t)g.K, mine_at = 8 * (threadIdx.x & 63);
  float sum = 0.f;
#pragma unroll 1
  for (uint32_t k0 = 0; k0 < K; k0 += 512) {
    const uint32_t special = k0 + mine_at < K ? Eight<T>(x, k0 + mine_at, K).special() : 0;
#pragma unroll 1
    for (uint64_t lanes = __ballot(special != 0); lanes != 0; lanes &= lanes - 1) {
      const int from = __builtin_ctzll(lanes);
#pragma unroll 1
      for (uint32_t bits = __shfl(special, from); bits != 0; bits &= bits - 1) {
        const uint32_t k = k0 + 8 * from + __builtin_ctz(bits);
        if (mine) {
          const int64_t grp = k / (uint32_t)g.group;
          const int code = g.w[j * g.ldw + k / 2] >> (4 * (k & 1)) & 15;
          const float infinity = x[k] >> 15 ? -INFINITY : INFINITY;
          sum += scale_at(g, j, grp) * (infinity * (float)(code - zero_at(g, j, grp)));
        }
      }
      if (!__any(mine && sum == sum)) return sum;  // NaN in all of them, and it stays
    }
  }
  return sum;
}

// For the whole wave: what a lane's Y[m,j] with bad set takes.
enum class Again { kNothing, kDefinition, kInfinities };
template <awe_dtype T>
__device__ __forceinline__ Again again(const W4Launch& g, bool bad, int64_t m) {
  if constexpr (T == AWE_I8) return bad ? Again::kDefinition : Again::kNothing;
  uint64_t left = __ballot(bad), finite = 0, infinite = 0;
  while (left != 0) {
    const int64_t row = __shfl(m, __builtin_ctzll(left));
    const uint64_t of_row = __ballot(m == row) & left;
    left &= ~of_row;
    const auto* x = reinterpret_cast<const typename Kind<T>::Elem*>(g.x) + row * g.ldx;
    uint32_t special = 0;
#pragma unroll 4
    for (uint32_t k = 8 * (threadIdx.x & 63); k < (uint32_t)g.K; k += 512) special |= Eight<T>(x, k, (uint32_t)g.K).special();
    if (__any(special >= 256)) continue;  // a NaN
    (__any(special != 0) ? infinite : finite) |= of_row;
  }
  const uint64_t me = uint64_t(1) << (threadIdx.x & 63);
  return infinite & me ? Again::kInfinities : finite & me ? Again::kDefinition : Again::kNothing;
}

// For the whole wave: Y[m,j] again.
template <awe_dtype T>
__device__ __forceinline__ void store_again(const W4Launch& g, Again how, int64_t m, int64_t j) {
  if constexpr (T != AWE_I8) {
    uint64_t left = __ballot(how == Again::kInfinities);
#pragma unroll 1
    while (left != 0) {
      const int64_t row = __shfl(m, __builtin_ctzll(left));
      const bool mine = how == Again::kInfinities && m == row;
      left &= ~__ballot(mine);
      const float y = by_infinities<T>(g, mine, row, j);
      if (mine) store_real(g.y, m * g.ldy + j, g.y_type, y);
    }
  }
#pragma unroll 1
  for (uint64_t left = __ballot(how == Again::kDefinition); left != 0; left &= left - 1) {
    const int lane = __builtin_ctzll(left);
    const double y = by_definition<T>(g, __shfl(m, lane), __shfl(j, lane));
    if ((int)(threadIdx.x & 63) == lane) store_real(g.y, m * g.ldy + j, g.y_type, (float)y);
  }
}

constexpr int kChunk = 128;  // reduction indices of a wave's step: 16 bytes of codes per lane

struct W4Args {
  W4Launch g;
  int32_t units;  // group / 128, or group / 64 or / 32 where 128 does not divide it
};

// A lane loads row n of W at indices 32 q .. 32 q + 31 of the chunk (16 bytes); the words are then transposed over
// the quarters, so that step j covers indices 32 j .. 32 j + 31, 8 q .. 8 q + 7 of them in this lane: a step
// lies in one group (groups begin at multiples of 32 indices), and a load of X's operand reads 64 (int8: 32) adjacent bytes
// of each row.  kPairs (int8 with groups of whole 64s): steps 2 c and 2 c + 1 cover 64 c .. 64 c + 63 between
// them, 16 adjacent indices in this lane, one load of X.
template <bool kPairs>
__device__ __forceinline__ int step_offset(int q, int j) {
  return kPairs ? 64 * (j >> 1) + 16 * q + 8 * (j & 1) : 32 * j + 8 * q;
}

// 128 bits, the low word first, shifted right by n < 128.
__device__ __forceinline__ u4 shifted(u4 v, int n) {
  const uint64_t lo = (uint64_t)v[0] | (uint64_t)v[1] << 32, hi = (uint64_t)v[2] | (uint64_t)v[3] << 32;
  const uint64_t a = n >= 64 ? hi >> (n - 64) : n > 0 ? lo >> n | hi << (64 - n) : lo, b = n >= 64 ? 0 : hi >> n;
  return u4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
}
// 16 bytes at byte `at` of a row of `bytes` bytes, 0 past its end (nothing there is read): the row's last 16
// bytes, shifted into place.
__device__ __forceinline__ u4 row_end(const uint8_t* row, int64_t at, int64_t bytes) {
  if (at >= bytes) return u4{0, 0, 0, 0};
  if (bytes < 16) {
    u4 r = {0, 0, 0, 0};
    for (int b = 0; b < (int)(bytes - at); ++b) {
      const uint32_t v = (uint32_t)row[at + b] << (8 * (b & 3));
#pragma unroll
      for (int w = 0; w < 4; ++w) r[w] |= w == b >> 2 ? v : 0u;
    }
    return r;
  }
  const int64_t from = at + 16 <= bytes ? at : bytes - 16;
  const Any16 v = *reinterpret_cast<const Any16*>(row + from);
  return shifted(u4{v.w[0], v.w[1], v.w[2], v.w[3]}, 8 * (int)(at - from));
}
// Eight elements of a row of K at k, 0 past its end.
template <awe_dtype T>
__device__ __forceinline__ typename Kind<T>::Raw load8_end(const typename Kind<T>::Elem* row, int64_t k, int64_t K) {
  constexpr int kE = sizeof(typename Kind<T>::Elem);
  const u4 v = row_end(reinterpret_cast<const uint8_t*>(row), k * kE, K * kE);
  if constexpr (T == AWE_I8)
    return (uint64_t)v[0] | (uint64_t)v[1] << 32;
  else
    return v;
}

// A scale as it lies in memory, and its value.
template <awe_dtype S>
__device__ __forceinline__ uint32_t raw_scale(const uint8_t* p) {
  if constexpr (S == AWE_F32)
    return *reinterpret_cast<const uint32_t*>(p);
  else
    return *reinterpret_cast<const uint16_t*>(p);
}
template <awe_dtype S>
__device__ __forceinline__ float scale_value(uint32_t raw) {
  if constexpr (S == AWE_F32) return __builtin_bit_cast(float, raw);
  if constexpr (S == AWE_BF16) return __builtin_bit_cast(float, raw << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)raw);
}

// Bytes of a row as they are loaded.  kOdd: at any address, as the words that hold them (the last one may be one
// more), put together when they are used; the memory system takes about twice as long for wide loads at addresses
// that are not multiples of 4.  Up to three bytes on either side of the operand are read with its first and last
// word and not used: an aligned word that holds a byte of the operand lies in that byte's page.
template <int kBytes, bool kOdd>
struct Piece {
  static constexpr int kN = kBytes / 4;
  struct Aligned {
    uint32_t w[kN];
  };
  uint32_t w[kN + (kOdd ? 1 : 0)];

  __device__ __forceinline__ void load(const uint8_t* p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const Aligned a = *reinterpret_cast<const Aligned*>(kOdd ? at & ~uintptr_t(3) : at);
#pragma unroll
    for (int i = 0; i < kN; ++i) w[i] = a.w[i];
    if constexpr (kOdd) w[kN] = *reinterpret_cast<const uint32_t*>((at + kBytes - 1) & ~uintptr_t(3));
  }
  __device__ __forceinline__ uint32_t word(int i, uint32_t shift) const {  // shift: the address modulo 4
    if constexpr (kOdd) return __builtin_amdgcn_alignbyte(w[i + 1], w[i], shift);
    return w[i];
  }
};
__device__ __forceinline__ uint32_t in_word(const uint8_t* p) { return (uint32_t)reinterpret_cast<uintptr_t>(p) & 3; }

// Few rows, or few outputs: 16 kN outputs per workgroup, whose kW waves take the chunks of the reduction in turn, each
// with up to kM x 16 rows of X.  Operands go straight from memory to the matrix unit, and a wave's loop is one
// copy of the code for kD chunks, whose loads the compiler spreads over the products.  Bound by the weights' bytes
// and the loads' latency: calls back to back, one row at 8192 x 8192 takes 11.2 us (35 MB, 3.1 TB/s; traced by
// itself 11.9), 16 int8 rows 12.7 (12.6).  Unrolled further to fetch ahead, it spends more time on fetching
// instructions than it saves (13.2 us for one row; X staged in LDS: 13.2; 16 outputs per workgroup: 14.3).
constexpr int kW = 8;

// S: the scales' type, or kAnyScale for the one that the call says (one row at 8192 x 8192: 14.1 us instead of 11.2).
// kOddX, kOddW: rows of X or W that begin off 4-byte addresses.
constexpr awe_dtype kAnyScale = AWE_I32;

template <awe_dtype T, int kM, int kN, int kD, int kFold, awe_dtype S, bool kOddX, bool kOddW>
__global__ __launch_bounds__(64 * kW, 2) void w4_rows_kernel(W4Args a) {
  using X = Kind<T>;
  using Elem = typename X::Elem;
  constexpr int kUnits = 4 / kFold;  // of a chunk
  constexpr bool kPairs = T == AWE_I8 && kFold > 1;
  constexpr int kS = kFold < 4 ? kD : 1;
  constexpr int kE = sizeof(Elem), kLoads = kPairs ? 2 : 4, kLoad = 128 * kE / 4 / kLoads;  // of X, in a chunk: bytes each
  const W4Launch& g = a.g;
  const awe_dtype s_type = S == kAnyScale ? g.s_type : S;
  const int s_bytes = s_type == AWE_F32 ? 4 : 2;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
  const int64_t n0 = (int64_t)blockIdx.x * 16 * kN, m0 = (int64_t)blockIdx.y * 16 * kM;

  // Each operand: the tile's first row (a scalar address) and this lane's 32-bit offset in bytes.  Past
  // the last row or output, that one again: its result is not stored.
  const bool has_z = g.zeros != nullptr;
  const uint8_t* wb = g.w + n0 * g.ldw;
  const uint8_t* sb = reinterpret_cast<const uint8_t*>(g.scales) + n0 * g.lds * s_bytes;
  const uint8_t* zb = has_z ? g.zeros + n0 * g.ldz : g.w;  // (any byte, where there are none)
  const uint8_t* xb = reinterpret_cast<const uint8_t*>(g.x) + m0 * g.ldx * kE;
  uint32_t wo[kN], so[kN], zo[kN], xo[kM];
#pragma unroll
  for (int t = 0; t < kN; ++t) {
    const uint32_t n = (uint32_t)std::min<int64_t>(16 * t + i, g.N - 1 - n0);
    wo[t] = n * (uint32_t)g.ldw + 16 * q;
    so[t] = n * (uint32_t)g.lds * s_bytes;
    zo[t] = has_z ? n * (uint32_t)g.ldz : 0;
  }
#pragma unroll
  for (int t = 0; t < kM; ++t) xo[t] = ((uint32_t)std::min<int64_t>(16 * t + i, g.M - 1 - m0) * (uint32_t)g.ldx + step_offset<kPairs>(q, 0)) * kE;
  const uint32_t magic = X::magic();
  f4 acc[kN][kM];
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int u = 0; u < kM; ++u) acc[t][u] = f4{0.f, 0.f, 0.f, 0.f};

  // A chunk's products.  s, z: a lane's scale and zero point of output tile t, in the quarter that fetched
  // it: the step's, or `of` where a chunk lies in one group.
  auto chunk = [&](auto codes, auto row, const uint32_t (&s)[kN], const uint32_t (&z)[kN], int of) {
    u4 c[kN];
#pragma unroll
    for (int t = 0; t < kN; ++t) c[t] = kPairs ? across_quarters_by_16(codes(t)) : across_quarters(codes(t));
    typename X::Acc part[kN][kM], sum[kM];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool first = j % kFold == 0;
      typename X::Op e[kM];
#pragma unroll
      for (int u = 0; u < kM; ++u) {
        e[u] = X::elems(row(u, j));
        sum[u] = X::mul(e[u], X::ones(), first ? X::zero() : sum[u]);
      }
#pragma unroll
      for (int t = 0; t < kN; ++t) {
        const typename X::Op op = X::codes(c[t][j], magic);
#pragma unroll
        for (int u = 0; u < kM; ++u) part[t][u] = X::mul(e[u], op, first ? X::zero() : part[t][u]);
      }
      if (j % kFold != kFold - 1) continue;
      // a group's part: part - (bias + z) sum x, times the group's scale
#pragma unroll
      for (int t = 0; t < kN; ++t) {
        const int from = 16 * (kFold < 4 ? j : of) + i;
        const uint32_t raw = __shfl(s[t], from);
        const float sc = s_type == AWE_F32 ? scale_value<AWE_F32>(raw) : s_type == AWE_BF16 ? scale_value<AWE_BF16>(raw) : scale_value<AWE_F16>(raw);
        const float b = X::kBias + (has_z ? (float)__shfl(z[t], from) : 8.f);
#pragma unroll
        for (int u = 0; u < kM; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[t][u][r] += sc * ((float)part[t][u][r] - b * (float)sum[u][r]);
      }
    }
  };
  const int32_t full = (int32_t)(g.K / kChunk), last = (int32_t)((g.K - 1) / g.group);
  // this lane's scales in the group of a unit
  auto scales = [&](uint32_t unit, uint32_t (&s)[kN], uint32_t (&z)[kN]) {
    const int32_t grp = std::min((int32_t)(unit / (uint32_t)a.units), last);
#pragma unroll
    for (int t = 0; t < kN; ++t) {
      const uint8_t* p = sb + (so[t] + (uint32_t)grp * s_bytes);
      s[t] = s_type == AWE_F32 ? raw_scale<AWE_F32>(p) : raw_scale<AWE_F16>(p);
      z[t] = zb[zo[t] + (has_z ? (uint32_t)grp : 0)];
    }
  };

#pragma unroll 1
  for (int32_t c0 = wave; c0 < full; c0 += kW * kD) {  // chunks c0 + u kW
    Piece<16, kOddW> cw[kD][kN];
    Piece<kLoad, kOddX> xr[kD][kM][kLoads];
    uint32_t s[kS][kN], z[kS][kN];
#pragma unroll
    for (int u = 0; u < kD; ++u) {
      const int64_t c = std::min(c0 + u * kW, full - 1);  // (past the end: the last one again, unused)
#pragma unroll
      for (int t = 0; t < kN; ++t) cw[u][t].load(wb + c * (kChunk / 2) + wo[t]);
    }
    // quarter q fetches the scales of the q-th chunk (of step q of each, where it has several)
#pragma unroll
    for (int v = 0; v < kS; ++v) scales(kFold < 4 ? kUnits * (c0 + v * kW) + q / kFold : c0 + q * kW, s[v], z[v]);
#pragma unroll
    for (int u = 0; u < kD; ++u) {
      const int64_t c = std::min(c0 + u * kW, full - 1);
#pragma unroll
      for (int t = 0; t < kM; ++t)
#pragma unroll
        for (int j = 0; j < kLoads; ++j) xr[u][t][j].load(xb + (c * kChunk + step_offset<kPairs>(0, j * (4 / kLoads))) * kE + xo[t]);
    }
#pragma unroll
    for (int u = 0; u < kD; ++u) {
      if (c0 + u * kW >= full) break;
      auto codes = [&](int t) {
        const uint32_t shift = in_word(wb + wo[t]);
        const Piece<16, kOddW>& p = cw[u][t];
        return u4{p.word(0, shift), p.word(1, shift), p.word(2, shift), p.word(3, shift)};
      };
      auto row = [&](int t, int j) {
        const uint32_t shift = in_word(xb + xo[t]);
        const Piece<kLoad, kOddX>& p = xr[u][t][kPairs ? j / 2 : j];
        if constexpr (T == AWE_I8) {
          const int first = kPairs ? 2 * (j & 1) : 0;
          return (uint64_t)p.word(first, shift) | (uint64_t)p.word(first + 1, shift) << 32;
        } else {
          return u4{p.word(0, shift), p.word(1, shift), p.word(2, shift), p.word(3, shift)};
        }
      };
      chunk(codes, row, s[kFold < 4 ? u : 0], z[kFold < 4 ? u : 0], u);
    }
  }

  // the last, short chunk
  if ((int64_t)full * kChunk < g.K && full % kW == wave) {
    const int64_t k0 = (int64_t)full * kChunk;
    u4 cw[kN];
    typename X::Raw xr[kM][4];
    uint32_t s[kN], z[kN];
#pragma unroll
    for (int t = 0; t < kN; ++t) cw[t] = row_end(wb + (wo[t] - 16 * q), k0 / 2 + 16 * q, (g.K + 1) / 2);
#pragma unroll
    for (int t = 0; t < kM; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Elem* row = reinterpret_cast<const Elem*>(xb + (xo[t] - step_offset<kPairs>(q, 0) * kE));
        xr[t][j] = load8_end<T>(row, k0 + step_offset<kPairs>(q, j), g.K);
      }
    scales(kFold < 4 ? kUnits * full + q / kFold : full, s, z);
    chunk([&](int t) { return cw[t]; }, [&](int t, int j) { return xr[t][j]; }, s, z, 0);
  }

  __shared__ struct {
    float red[kW][16 * kM][16 * kN + 1];
  } lds;
  // the waves' sums, and Y
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int u = 0; u < kM; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) lds.red[wave][16 * u + 4 * q + r][16 * t + i] = acc[t][u][r];
  __syncthreads();
#pragma unroll 1
  for (int e = threadIdx.x; e < 256 * kM * kN; e += 64 * kW) {  // (a wave's lanes together)
    const int row = e / (16 * kN), col = e % (16 * kN);
    const int64_t m = m0 + row, j = n0 + col;
    const bool ok = m < g.M && j < g.N;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kW; ++k) v += lds.red[k][row][col];
    if (ok) store_real(g.y, m * g.ldy + j, g.y_type, g.x_scales != nullptr ? v * g.x_scales[m] : v);
    const bool bad = ok && !__builtin_isfinite(v);
    if (__any(bad)) store_again<T>(g, again<T>(g, bad, m), m, j);
  }
}

// Many rows: a workgroup has 16 kM rows and 64 kN outputs, 16 kN of them each of its four waves, and goes
// through the reduction chunk by chunk.  The rows of X lie in LDS, twice (one chunk is multiplied while the
// next one is put there in the order of the codes, and the one after that is on its way), together with what
// the codes' bias makes of each row, -(bias + 8) sum x over a group, which is where a group's sum starts; scales
// and zero points lie there too, as floats.  A wave's weights go from memory to its registers, and no other
// wave unpacks them.
// kG groups of four waves take the chunks in turn, each with X of its own in LDS, and add up at the end, so that
// a CU with one workgroup has two waves per SIMD, too.  Bound by vector instructions (58 % of a CU's busy cycles for
// 4096 rows with zero points, for the codes and the folding; MFMAs are busy for 34 %), at the two waves per SIMD that
// the registers allow: calls back to back, BF16 rows against 8192 x 8192 take 93 us for 512 (740 TFLOP/s; traced
// by itself 106) and 711-722 for 4096 (760-770; a plain product of BF16 numbers reaches 1250).
template <awe_dtype T, int kM, int kN, int kFold>
struct TileLds {  // of a group of waves
  using X = Kind<T>;
  static constexpr int kRows = 16 * kM, kCols = 64 * kN, kSub = 4 / kFold;
  alignas(16) uint8_t x[2][kRows * kChunk * sizeof(typename X::Elem)];
  alignas(16) typename X::Sum start[2][kSub][kRows], sum[2][kSub][kRows];
  float s[2][kSub][kCols], z[2][kSub][kCols];
};
template <awe_dtype T, int kM, int kN, int kG, int kFold>
constexpr int tile_lds_bytes() {
  const int groups = kG * (int)sizeof(TileLds<T, kM, kN, kFold>), sums = (kG - 1) * 256 * kM * kN * 16;
  return groups > sums ? groups : sums;
}

template <awe_dtype T, int kM, int kN, int kG, int kFold>
__global__ __launch_bounds__(256 * kG, 2) void w4_tile_kernel(W4Args a) {
  using X = Kind<T>;
  using Elem = typename X::Elem;
  using Raw = typename X::Raw;
  using Acc = typename X::Acc;
  using Sum = typename X::Sum;
  constexpr int kE = sizeof(Elem), kRows = 16 * kM, kCols = 64 * kN, kSub = 4 / kFold;
  constexpr int kPer = 256 / kRows;           // threads that fetch a row
  constexpr int kPieces = kChunk / 8 / kPer;  // pieces of 8 elements each of them has
  static_assert(kPieces == 4, "a thread's pieces make up a step of 32 indices");
  static_assert(kCols <= 256, "a thread per output fetches its scale");
  static_assert(4 * kM * kN <= 64, "a bit for each of a lane's results");
  const W4Launch& g = a.g;
  const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), tid = threadIdx.x & 255;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, q = lane >> 4, i = lane & 15;
  // Workgroups go round the eight XCDs; each takes a run of tiles, eight tiles high, so that the ones it
  // works on at a time share rows and weights in its L2.
  const int64_t tiles_m = (g.M + kRows - 1) / kRows, tiles_n = (g.N + kCols - 1) / kCols, tiles = tiles_m * tiles_n;
  const int64_t per_xcd = (tiles + 7) / 8, tile = (int64_t)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= per_xcd || tile >= tiles) return;
  const int64_t band = tile / (8 * tiles_n), high = std::min<int64_t>(8, tiles_m - 8 * band), in = tile - band * 8 * tiles_n;
  const int64_t m0 = (8 * band + in % high) * kRows, n0 = in / high * kCols;

  extern __shared__ uint8_t tile_lds[];
  TileLds<T, kM, kN, kFold>& lds = reinterpret_cast<TileLds<T, kM, kN, kFold>*>(tile_lds)[group];
  // where a row's piece of 8 elements lies: units of 16 bytes, permuted by the row, so that the same
  // piece of 16 rows lies in different banks
  auto place = [](int row, int piece) {
    return kE == 2 ? row * 256 + ((piece ^ (row & 15)) << 4) : row * 128 + (((piece >> 1) ^ (row & 7)) << 4) + 8 * (piece & 1);
  };

  // this thread's part of the fetching: pieces first .. first + kPieces - 1 of a row, and the scale of an output
  const int my_row = tid / kPer, first = tid % kPer * kPieces;
  const uint8_t* xb = reinterpret_cast<const uint8_t*>(g.x) + m0 * g.ldx * kE;
  const uint32_t xo = ((uint32_t)std::min<int64_t>(my_row, g.M - 1 - m0) * (uint32_t)g.ldx + 8 * first) * kE;
  const int32_t full = (int32_t)(g.K / kChunk), chunks = (int32_t)((g.K + kChunk - 1) / kChunk);
  const int32_t last = (int32_t)((g.K - 1) / g.group);
  const bool has_z = g.zeros != nullptr;
  const int s_shift = g.s_type == AWE_F32 ? 2 : 1;
  const uint32_t my_col = (uint32_t)std::min<int64_t>(tid, g.N - 1 - n0);
  const uint8_t* sb = reinterpret_cast<const uint8_t*>(g.scales) + ((n0 * g.lds) << s_shift);
  const uint8_t* zb = has_z ? g.zeros + n0 * g.ldz : g.w;  // (any byte, where there are none)
  const uint32_t so = (my_col * (uint32_t)g.lds) << s_shift, zo = has_z ? my_col * (uint32_t)g.ldz : 0;
  struct Fetched {
    Raw x[kPieces];
    uint32_t s[kSub], z[kSub];  // as they lie in memory: nothing may wait for them here
  };
  auto fetch = [&](Fetched& f, int32_t c, bool end) {
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      f.x[p] = end ? load8_end<T>(reinterpret_cast<const Elem*>(xb + (xo - 8 * first * kE)), (int64_t)c * kChunk + 8 * (first + p), g.K)
                   : load8<T>(reinterpret_cast<const Elem*>(xb + ((int64_t)c * kChunk + 8 * p) * kE + xo));
    }
#pragma unroll
    for (int j = 0; j < kSub; ++j) {
      const int32_t grp = std::min((int32_t)((uint32_t)(kSub * c + j) / (uint32_t)a.units), last);
      const uint8_t* s = sb + (so + ((uint32_t)grp << s_shift));
      f.s[j] = s_shift == 2 ? raw_scale<AWE_F32>(s) : raw_scale<AWE_F16>(s);
      f.z[j] = zb[zo + (has_z ? (uint32_t)grp : 0)];
    }
  };
  auto keep = [&](const Fetched& f, int buf) {
    Sum sum = 0;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
      const typename X::Op e = X::elems(f.x[p]);
      sum = X::add(e, sum);
      *reinterpret_cast<typename X::Op*>(lds.x[buf] + place(my_row, first + p)) = e;
    }
#pragma unroll
    for (int d = 1; d < kFold; d *= 2) sum += __shfl_xor(sum, d);
    const int step = first / 4;  // this thread's
    if (step % kFold == 0) {
      lds.start[buf][step / kFold][my_row] = sum * -(X::kBias + 8);
      lds.sum[buf][step / kFold][my_row] = sum;
    }
    if (tid >= kCols) return;
#pragma unroll
    for (int j = 0; j < kSub; ++j) {
      lds.s[buf][j][tid] = g.s_type == AWE_F32    ? scale_value<AWE_F32>(f.s[j])
                                   : g.s_type == AWE_BF16 ? scale_value<AWE_BF16>(f.s[j])
                                                          : scale_value<AWE_F16>(f.s[j]);
      lds.z[buf][j][tid] = has_z ? 8.f - (float)f.z[j] : 0.f;  // of sum x, beside what the sum starts from
    }
  };

  // this wave's weights
  const int64_t nw = n0 + 16 * kN * wave;
  const uint8_t* wb = g.w + std::min(nw, g.N - 1) * g.ldw;
  uint32_t wo[kN];
#pragma unroll
  for (int t = 0; t < kN; ++t)
    wo[t] = (uint32_t)std::max<int64_t>(0, std::min<int64_t>(16 * t + i, g.N - 1 - nw)) * (uint32_t)g.ldw + 16 * q;
  auto codes = [&](u4 (&w)[kN], int32_t c, bool end) {
#pragma unroll
    for (int t = 0; t < kN; ++t) {
      if (!end) {
        const Any16 v = *reinterpret_cast<const Any16*>(wb + (int64_t)c * (kChunk / 2) + wo[t]);
        w[t] = u4{v.w[0], v.w[1], v.w[2], v.w[3]};
      } else {
        w[t] = row_end(wb + (wo[t] - 16 * q), (int64_t)c * (kChunk / 2) + 16 * q, (g.K + 1) / 2);
      }
    }
  };

  const uint32_t magic = X::magic();
  f4 acc[kN][kM];
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int u = 0; u < kM; ++u) acc[t][u] = f4{0.f, 0.f, 0.f, 0.f};

  auto multiply = [&](u4 (&now)[kN], int buf) {
    Acc part[kN][kM];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int sub = j / kFold;
      const bool begin = j % kFold == 0;
      typename X::Op e[kM];
      Acc start[kM];
#pragma unroll
      for (int u = 0; u < kM; ++u) {
        e[u] = *reinterpret_cast<const typename X::Op*>(lds.x[buf] + place(16 * u + i, kFold < 4 ? 4 * j + q : 4 * q + j));
        if (begin) start[u] = *reinterpret_cast<const Acc*>(&lds.start[buf][sub][16 * u + 4 * q]);
      }
#pragma unroll
      for (int t = 0; t < kN; ++t) {
        if (kFold < 4 && j == 0) now[t] = across_quarters(now[t]);
        const typename X::Op op = X::codes(now[t][j], magic);
#pragma unroll
        for (int u = 0; u < kM; ++u) part[t][u] = X::mul(e[u], op, begin ? start[u] : part[t][u]);
      }
      if (j % kFold != kFold - 1) continue;
#pragma unroll
      for (int t = 0; t < kN; ++t) {
        const int col = 16 * (kN * wave + t) + i;
        const float sc = lds.s[buf][sub][col];
#pragma unroll
        for (int u = 0; u < kM; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[t][u][r] += sc * (float)part[t][u][r];
      }
      if (has_z) {
#pragma unroll
        for (int u = 0; u < kM; ++u) start[u] = *reinterpret_cast<const Acc*>(&lds.sum[buf][sub][16 * u + 4 * q]);
#pragma unroll
        for (int t = 0; t < kN; ++t) {
          const int col = 16 * (kN * wave + t) + i;
          const float zc = lds.s[buf][sub][col] * lds.z[buf][sub][col];
#pragma unroll
          for (int u = 0; u < kM; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[t][u][r] += zc * (float)start[u][r];
        }
      }
    }
  };

  const int32_t stages = (full + kG - 1) / kG;
  if (stages > 0) {
    Fetched f;
    u4 now[kN], ahead[kN];
    if (group < full) {
      codes(now, group, false);
      fetch(f, group, false);
      keep(f, 0);
      if (group + kG < full) fetch(f, group + kG, false);
    }
#pragma unroll 1
    for (int32_t st = 0; st < stages; ++st) {
      const int32_t c = kG * st + group;
      __syncthreads();  // chunk c is there, and nobody reads the other half any more
      if (c < full) {
        if (c + kG < full) {
          codes(ahead, c + kG, false);
          keep(f, (st & 1) ^ 1);
        }
        if (c + 2 * kG < full) fetch(f, c + 2 * kG, false);
        multiply(now, st & 1);
      }
#pragma unroll
      for (int t = 0; t < kN; ++t) now[t] = ahead[t];
    }
  }
  if (full < chunks) {  // the last, short chunk
    u4 now[kN];
    if (group == full % kG) {
      Fetched f;
      codes(now, full, true);
      fetch(f, full, true);
      keep(f, stages & 1);
    }
    __syncthreads();
    if (group == full % kG) multiply(now, stages & 1);
  }
  if (kG > 1) {
    float* part = reinterpret_cast<float*>(tile_lds);
    __syncthreads();
    if (group == 1)
#pragma unroll
      for (int t = 0; t < kN; ++t)
#pragma unroll
        for (int u = 0; u < kM; ++u)
#pragma unroll
          for (int r = 0; r < 4; ++r) part[((t * kM + u) * 4 + r) * 256 + tid] = acc[t][u][r];
    __syncthreads();
    if (group == 1) return;
#pragma unroll
    for (int t = 0; t < kN; ++t)
#pragma unroll
      for (int u = 0; u < kM; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[t][u][r] += part[((t * kM + u) * 4 + r) * 256 + tid];
  }

#pragma unroll
  for (int u = 0; u < kM; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t m = m0 + 16 * u + 4 * q + r;
      if (m >= g.M) continue;
      const float sx = g.x_scales != nullptr ? g.x_scales[m] : 1.f;
#pragma unroll
      for (int t = 0; t < kN; ++t)
        if (nw + 16 * t + i < g.N) store_real(g.y, m * g.ldy + nw + 16 * t + i, g.y_type, acc[t][u][r] * sx);
    }
  // (looked through by itself, 4096 rows of 8192 outputs take 713 us; within the stores above, 738)
  bool odd = false;
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int u = 0; u < kM; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) odd |= !__builtin_isfinite(acc[t][u][r]);
  if (!__any(odd)) return;
  uint64_t bad = 0;  // bit (4 u + r) kN + t
#pragma unroll
  for (int u = 0; u < kM; ++u)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < kN; ++t)
        if (m0 + 16 * u + 4 * q + r < g.M && nw + 16 * t + i < g.N)
          bad |= (uint64_t)!__builtin_isfinite(acc[t][u][r]) << ((4 * u + r) * kN + t);
#pragma unroll 1
  for (int e = 0; e < 4 * kM; ++e) {
    const uint32_t of_row = (uint32_t)(bad >> (e * kN)) & ((1u << kN) - 1);
    if (!__any(of_row != 0)) continue;
    const int64_t m = m0 + 16 * (e / 4) + 4 * q + e % 4;
    const Again how = again<T>(g, of_row != 0, m);
#pragma unroll 1
    for (int t = 0; t < kN; ++t) store_again<T>(g, of_row >> t & 1 ? how : Again::kNothing, m, nw + 16 * t + i);
  }
}

awe_status too_many() {
  set_error("too many outputs for one launch");
  return AWE_ERR_UNSUPPORTED;
}

template <awe_dtype T, int kFold, int kM, int kN, int kD>
awe_status launch_rows(const W4Args& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.g.N + 16 * kN - 1) / (16 * kN)), (unsigned)((a.g.M + 16 * kM - 1) / (16 * kM)));
  const dim3 block(64 * kW);
  if ((int64_t)grid.x * block.x >= int64_t(1) << 32) return too_many();
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
  // Rows off 4-byte addresses are loaded as words and put together (33 FP16 rows, 1537 outputs, K = 2049: 9 us
  // instead of 17; one row against odd rows of W, 8192 x 8192: 15 instead of 21); X's alone are not told apart from both.
  auto odd = [](const void* p, int64_t rows, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 4 != 0 || (rows > 1 && stride % 4 != 0);
  };
  if (odd(a.g.x, a.g.M, a.g.ldx * (int64_t)sizeof(typename Kind<T>::Elem)))
    launch(w4_rows_kernel<T, kM, kN, kD, kFold, kAnyScale, true, true>);
  else if (odd(a.g.w, a.g.N, a.g.ldw))
    launch(w4_rows_kernel<T, kM, kN, kD, kFold, kAnyScale, false, true>);
  else if (a.g.s_type == AWE_F32)
    launch(w4_rows_kernel<T, kM, kN, kD, kFold, AWE_F32, false, false>);
  else if (a.g.s_type == AWE_BF16)
    launch(w4_rows_kernel<T, kM, kN, kD, kFold, AWE_BF16, false, false>);
  else
    launch(w4_rows_kernel<T, kM, kN, kD, kFold, AWE_F16, false, false>);
  return launched("w4 launch");
}

template <awe_dtype T, int kM, int kN, int kG, int kFold>
awe_status launch_tile(const W4Args& a, int64_t tiles, hipStream_t stream) {
  static std::mutex mu;
  static std::set<int> done;
  constexpr int bytes = tile_lds_bytes<T, kM, kN, kG, kFold>();
  static_assert(kG <= 2 && bytes <= 160 * 1024 / (3 - kG), "the workgroups of a CU fit its LDS");
  auto kernel = w4_tile_kernel<T, kM, kN, kG, kFold>;
  if ((tiles + 7) / 8 * 8 * 256 * kG >= int64_t(1) << 32) return too_many();
  const awe_status st = set_lds_limit(reinterpret_cast<const void*>(kernel), bytes, mu, done);
  if (st != AWE_OK) return st;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(256 * kG), bytes, stream, a);
  return launched("w4 launch");
}

template <awe_dtype T, int kFold>
awe_status launch_tiles(const W4Args& a, hipStream_t stream) {
  auto tiles = [&](int cols) { return ((a.g.M + 63) / 64) * ((a.g.N + cols - 1) / cols); };
  // the widest tile that still gives each of the 256 CUs one; two workgroups per CU where there are enough (four
  // groups of waves on the narrowest tile: 47 us instead of 53 at 1024 x 1024 x 8192, but 90 instead of 77 at 1536 rows)
  if constexpr (kFold > 1) {  // (a fold at every step needs more registers than such a tile leaves)
    if (tiles(256) >= 512) return launch_tile<T, 4, 4, 1, kFold>(a, tiles(256), stream);
    if (tiles(256) >= 256) return launch_tile<T, 4, 4, 2, kFold>(a, tiles(256), stream);
  }
  if (tiles(128) >= 256) return launch_tile<T, 4, 2, 2, kFold>(a, tiles(128), stream);
  return launch_tile<T, 4, 1, 2, kFold>(a, tiles(64), stream);
}

template <awe_dtype T, int kFold>
awe_status launch_kind(const W4Args& a, hipStream_t stream) {
  // Up to 64 rows, and more while workgroups of 32 x 32 are at most two for each of the 256 CUs: these split the
  // reduction over eight waves, a tile over two groups.  In us, split / tile, of BF16 rows, int8 ones, BF16 with
  // groups of 32, and BF16 against rows of W off words:
  //   128 x  128 x 8192   19 / 43   12 / 35   20 / 73   20 / 55
  //   512 x 1024 x 8192   43 / 53   30 / 41   50 / 97   48 / 65
  //  1024 x 1024 x 8192   80 / 53   54 / 41   97 / 98   94 / 65
  //  1024 x 1024 x  512   13 / 10   10 /  9   19 / 12   17 / 10
  //    64 x 8192 x 8192   44 / 49   30 / 38   50 / 94   49 / 66
  if (a.g.M > 64 && ((a.g.N + 31) / 32) * ((a.g.M + 31) / 32) > 512) return launch_tiles<T, kFold>(a, stream);
  // 16 outputs a workgroup while that is at most one per CU (M = 1: 8.4 us instead of 10.4 at 4096 x 8192,
  // but 12.3 instead of 10.9 at 8192 x 8192); beyond, 32 halve what is read of X
  const int rows = a.g.M <= 16 ? 16 : 32;
  const bool narrow = ((a.g.N + 15) / 16) * ((a.g.M + rows - 1) / rows) <= 256;
  if (rows == 16) return narrow ? launch_rows<T, kFold, 1, 1, 4>(a, stream) : launch_rows<T, kFold, 1, 2, 4>(a, stream);
  return narrow ? launch_rows<T, kFold, 2, 1, 2>(a, stream) : launch_rows<T, kFold, 2, 2, 2>(a, stream);
}

template <int kFold>
awe_status launch_type(const W4Args& a, hipStream_t stream) {
  if (a.g.x_type == AWE_BF16) return launch_kind<AWE_BF16, kFold>(a, stream);
  if (a.g.x_type == AWE_F16) return launch_kind<AWE_F16, kFold>(a, stream);
  return launch_kind<AWE_I8, kFold>(a, stream);
}

}  // namespace

awe_status launch_w4(const W4Launch& g, hipStream_t stream) {
  W4Args a{};
  a.g = g;
  // one group of at least K indices counts as one of whole chunks
  if (g.group >= g.K) a.g.group = std::max<int64_t>(1, (g.K + kChunk - 1) / kChunk) * kChunk;
  // a sum is folded at least every 128 indices, and at every multiple of 32 or 64 where a group may end there
  const int fold = a.g.group % 128 == 0 ? 4 : a.g.group % 64 == 0 ? 2 : 1;
  a.units = (int32_t)(a.g.group / (32 * fold));
  return fold == 4 ? launch_type<4>(a, stream) : fold == 2 ? launch_type<2>(a, stream) : launch_type<1>(a, stream);
}

}  // namespace awe

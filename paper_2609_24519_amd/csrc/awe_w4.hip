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

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
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
  static constexpr float kBias = 16.f;
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
  static constexpr float kBias = 16.f;
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
  static constexpr float kBias = 0.f;
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

constexpr int kChunk = 128;  // reduction indices of a wave's step: 16 bytes of codes per lane

struct W4Args {
  W4Launch g;
  int32_t units;      // group / 128, or group / 32 where 128 does not divide it
};

// A lane loads row n of W at indices 32 q .. 32 q + 31 of the chunk (16 bytes); the words are then transposed over
// the quarters, so that step j covers indices 32 j .. 32 j + 31, 8 q .. 8 q + 7 of them in this lane: a step
// lies in one group (groups begin at multiples of 32 indices), and a load of X's operand reads 64 (int8: 32) adjacent bytes
// of each row.
__device__ __forceinline__ int step_offset(int q, int j) { return 32 * j + 8 * q; }

// 16 bytes at byte `at` of a row of `bytes` bytes, 0 past its end (nothing there is read).
__device__ u4 row_end(const uint8_t* row, int64_t at, int64_t bytes) {
  u4 r = {0, 0, 0, 0};
  const int n = (int)std::max<int64_t>(0, std::min<int64_t>(bytes - at, 16));
#pragma unroll
  for (int b = 0; b < 16; ++b) r[b >> 2] |= (b < n ? (uint32_t)row[at + b] : 0u) << (8 * (b & 3));
  return r;
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

// Few rows: 16 kN outputs per workgroup, whose kW waves take the chunks of the reduction in turn, each
// with up to kM x 16 rows of X.  Operands go straight from memory to the matrix unit, and a wave's loop is one
// copy of the code for kD chunks, whose loads the compiler spreads over the products: unrolled
// further to fetch ahead, it spent more time on fetching instructions than it saved (13.2 us instead of
// 10.6 for one row at 8192 x 8192; X staged in LDS: 13.2; 16 outputs per workgroup: 14.3).
constexpr int kW = 8;

template <awe_dtype T, int kM, int kN, int kD, bool kFine, awe_dtype S>
__global__ __launch_bounds__(64 * kW, 2) void w4_rows_kernel(W4Args a) {
  using X = Kind<T>;
  using Elem = typename X::Elem;
  constexpr int kS = kFine ? kD : 1;
  constexpr int kE = sizeof(Elem), kSE = S == AWE_F32 ? 4 : 2;
  const W4Launch& g = a.g;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
  const int64_t n0 = (int64_t)blockIdx.x * 16 * kN, m0 = (int64_t)blockIdx.y * 16 * kM;

  // Each operand: the tile's first row (a scalar address) and this lane's 32-bit offset in bytes.  Past
  // the last row or output, that one again: its result is not stored.
  const bool has_z = g.zeros != nullptr;
  const uint8_t* wb = g.w + n0 * g.ldw;
  const uint8_t* sb = reinterpret_cast<const uint8_t*>(g.scales) + n0 * g.lds * kSE;
  const uint8_t* zb = has_z ? g.zeros + n0 * g.ldz : g.w;  // (any byte, where there are none)
  const uint8_t* xb = reinterpret_cast<const uint8_t*>(g.x) + m0 * g.ldx * kE;
  uint32_t wo[kN], so[kN], zo[kN], xo[kM];
#pragma unroll
  for (int t = 0; t < kN; ++t) {
    const uint32_t n = (uint32_t)std::min<int64_t>(16 * t + i, g.N - 1 - n0);
    wo[t] = n * (uint32_t)g.ldw + 16 * q;
    so[t] = n * (uint32_t)g.lds * kSE;
    zo[t] = has_z ? n * (uint32_t)g.ldz : 0;
  }
#pragma unroll
  for (int t = 0; t < kM; ++t) xo[t] = ((uint32_t)std::min<int64_t>(16 * t + i, g.M - 1 - m0) * (uint32_t)g.ldx + 8 * q) * kE;
  const uint32_t magic = X::magic();
  f4 acc[kN][kM];
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int u = 0; u < kM; ++u) acc[t][u] = f4{0.f, 0.f, 0.f, 0.f};

  // A chunk's products.  s, z: a lane's scale and zero point of output tile t, in quarter `of` + step (kFine) or
  // in quarter `of`.
  auto chunk = [&](const u4 (&cw)[kN], const typename X::Raw (&xr)[kM][4], const uint32_t (&s)[kN], const uint32_t (&z)[kN],
                   int of) {
    u4 c[kN];
#pragma unroll
    for (int t = 0; t < kN; ++t) c[t] = across_quarters(cw[t]);
    typename X::Acc part[kN][kM], sum[kM];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool first = kFine || j == 0;
      typename X::Op e[kM];
#pragma unroll
      for (int u = 0; u < kM; ++u) {
        e[u] = X::elems(xr[u][j]);
        sum[u] = X::mul(e[u], X::ones(), first ? X::zero() : sum[u]);
      }
#pragma unroll
      for (int t = 0; t < kN; ++t) {
        const typename X::Op op = X::codes(c[t][j], magic);
#pragma unroll
        for (int u = 0; u < kM; ++u) part[t][u] = X::mul(e[u], op, first ? X::zero() : part[t][u]);
      }
      if (!kFine && j < 3) continue;
      // a group's part: part - (bias + z) sum x, times the group's scale
#pragma unroll
      for (int t = 0; t < kN; ++t) {
        const int from = 16 * (kFine ? j : of) + i;
        const float sc = scale_value<S>(__shfl(s[t], from)), b = X::kBias + (has_z ? (float)__shfl(z[t], from) : 8.f);
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
      s[t] = raw_scale<S>(sb + (so[t] + (uint32_t)grp * kSE));
      z[t] = zb[zo[t] + (has_z ? (uint32_t)grp : 0)];
    }
  };

#pragma unroll 1
  for (int32_t c0 = wave; c0 < full; c0 += kW * kD) {  // chunks c0 + u kW
    u4 cw[kD][kN];
    typename X::Raw xr[kD][kM][4];
    uint32_t s[kS][kN], z[kS][kN];
#pragma unroll
    for (int u = 0; u < kD; ++u) {
      const int64_t c = std::min(c0 + u * kW, full - 1);  // (past the end: the last one again, unused)
#pragma unroll
      for (int t = 0; t < kN; ++t) {
        const Any16 v = *reinterpret_cast<const Any16*>(wb + c * (kChunk / 2) + wo[t]);
        cw[u][t] = u4{v.w[0], v.w[1], v.w[2], v.w[3]};
      }
    }
    // quarter q fetches the scales of the q-th chunk (of step q of each, if fine)
#pragma unroll
    for (int v = 0; v < kS; ++v) scales(kFine ? 4 * (c0 + v * kW) + q : c0 + q * kW, s[v], z[v]);
#pragma unroll
    for (int u = 0; u < kD; ++u) {
      const int64_t c = std::min(c0 + u * kW, full - 1);
#pragma unroll
      for (int t = 0; t < kM; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) xr[u][t][j] = load8<T>(reinterpret_cast<const Elem*>(xb + (c * kChunk + 32 * j) * kE + xo[t]));
    }
#pragma unroll
    for (int u = 0; u < kD; ++u) {
      if (c0 + u * kW >= full) break;
      chunk(cw[u], xr[u], s[kFine ? u : 0], z[kFine ? u : 0], u);
    }
  }

  // the last, short chunk, X filled up with zeros in LDS
  __shared__ union {
    float red[kW][16 * kM][16 * kN + 1];
    alignas(16) Elem x[16 * kM][kChunk];
  } lds;
  if ((int64_t)full * kChunk < g.K) {
    const int64_t k0 = (int64_t)full * kChunk;
    for (int e = threadIdx.x; e < 16 * kM * kChunk; e += 64 * kW) {
      const int64_t row = m0 + e / kChunk, k = k0 + e % kChunk;
      lds.x[e / kChunk][e % kChunk] = row < g.M && k < g.K ? reinterpret_cast<const Elem*>(g.x)[row * g.ldx + k] : 0;
    }
    __syncthreads();
    if (full % kW == wave) {
      u4 cw[kN];
      typename X::Raw xr[kM][4];
      uint32_t s[kN], z[kN];
#pragma unroll
      for (int t = 0; t < kN; ++t) cw[t] = row_end(wb + (wo[t] - 16 * q), k0 / 2 + 16 * q, (g.K + 1) / 2);
#pragma unroll
      for (int t = 0; t < kM; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) xr[t][j] = *reinterpret_cast<const typename X::Raw*>(&lds.x[16 * t + i][step_offset(q, j)]);
      scales(kFine ? 4 * full + q : full, s, z);
      chunk(cw, xr, s, z, 0);
    }
    __syncthreads();
  }

  // the waves' sums, and Y
#pragma unroll
  for (int t = 0; t < kN; ++t)
#pragma unroll
    for (int u = 0; u < kM; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) lds.red[wave][16 * u + 4 * q + r][16 * t + i] = acc[t][u][r];
  __syncthreads();
  for (int e = threadIdx.x; e < 256 * kM * kN; e += 64 * kW) {
    const int row = e / (16 * kN), col = e % (16 * kN);
    const int64_t m = m0 + row, j = n0 + col;
    if (m >= g.M || j >= g.N) continue;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kW; ++k) v += lds.red[k][row][col];
    store_real(g.y, m * g.ldy + j, g.y_type, g.x_scales != nullptr ? v * g.x_scales[m] : v);
  }
}

template <awe_dtype T, int kM, int kN, int kD>
awe_status launch_rows(const W4Args& a, bool fine, hipStream_t stream) {
  const dim3 grid((unsigned)((a.g.N + 16 * kN - 1) / (16 * kN)), (unsigned)((a.g.M + 16 * kM - 1) / (16 * kM)));
  const dim3 block(64 * kW);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
  if (a.g.s_type == AWE_F32)
    fine ? launch(w4_rows_kernel<T, kM, kN, kD, true, AWE_F32>) : launch(w4_rows_kernel<T, kM, kN, kD, false, AWE_F32>);
  else if (a.g.s_type == AWE_BF16)
    fine ? launch(w4_rows_kernel<T, kM, kN, kD, true, AWE_BF16>) : launch(w4_rows_kernel<T, kM, kN, kD, false, AWE_BF16>);
  else
    fine ? launch(w4_rows_kernel<T, kM, kN, kD, true, AWE_F16>) : launch(w4_rows_kernel<T, kM, kN, kD, false, AWE_F16>);
  return launched("w4 launch");
}

template <awe_dtype T>
awe_status launch_kind(const W4Args& a, bool fine, hipStream_t stream) {
  if (a.g.M <= 16) {
    switch (getenv("TRYN") ? atoi(getenv("TRYN")) : 0) {
      case 1: return launch_rows<T, 1, 1, 4>(a, fine, stream);
      default: return launch_rows<T, 1, 2, 4>(a, fine, stream);
    }
  }
    switch (getenv("TRYN") ? atoi(getenv("TRYN")) : 0) {
      case 1: return launch_rows<T, 4, 1, 2>(a, fine, stream);
      default: return launch_rows<T, 2, 2, 2>(a, fine, stream);
    }
}

}  // namespace

awe_status launch_w4(const W4Launch& g, hipStream_t stream) {
  // one group of at least K indices counts as a long one
  const bool fine = g.group % kChunk != 0 && g.group < g.K;
  W4Args a{};
  a.g = g;
  if (g.group >= g.K) a.g.group = std::max<int64_t>(1, (g.K + kChunk - 1) / kChunk) * kChunk;
  a.units = (int32_t)(a.g.group / (fine ? 32 : kChunk));
  if (g.x_type == AWE_BF16) return launch_kind<AWE_BF16>(a, fine, stream);
  if (g.x_type == AWE_F16) return launch_kind<AWE_F16>(a, fine, stream);
  return launch_kind<AWE_I8>(a, fine, stream);
}

}  // namespace awe

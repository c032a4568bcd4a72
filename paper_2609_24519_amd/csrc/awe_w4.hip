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
// The first n of them (0 for the rest): a load each for the bits of n.
struct __attribute__((packed)) Any4 {
  uint32_t w;
};
struct __attribute__((packed)) Any2 {
  uint16_t w;
};
template <awe_dtype T>
__device__ __forceinline__ typename Kind<T>::Raw load8_short(const typename Kind<T>::Elem* p, int n) {
  if (n >= 8) return load8<T>(p);
  uint64_t lo = 0, hi = 0;
  const int at2 = n & 4, at1 = n & 6;  // where the pair and the last one lie
  if constexpr (T == AWE_I8) {
    if (n > 0) {
      if (n & 4) lo = reinterpret_cast<const Any4*>(p)->w;
      if (n & 2) lo |= (uint64_t)reinterpret_cast<const Any2*>(p + at2)->w << (8 * at2);
      if (n & 1) lo |= (uint64_t)p[at1] << (8 * at1);
    }
    return lo;
  } else {
    if (n > 0) {
      if (n & 4) {
        const Any8 v = *reinterpret_cast<const Any8*>(p);
        lo = (uint64_t)v.w[0] | (uint64_t)v.w[1] << 32;
      }
      if (n & 2) (at2 ? hi : lo) |= reinterpret_cast<const Any4*>(p + at2)->w;
      if (n & 1) (at1 & 4 ? hi : lo) |= (uint64_t)p[at1] << (16 * (at1 & 2));
    }
    return u4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
  }
}
template <awe_dtype T>
__device__ __forceinline__ typename Kind<T>::Raw none() {
  return typename Kind<T>::Raw{};
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
  int32_t units;  // group / 128, or group / 32 where 128 does not divide it
};

// The chunk of a lane: row n of W at indices 32 q .. 32 q + 31 of the chunk.  kFine: a group may begin at any
// multiple of 32 indices, so each product of 32 indices has to lie in one group: the words are
// transposed over the quarters, and step j covers indices 32 j .. 32 j + 31 (8 q .. 8 q + 7 of them in
// this lane); otherwise step j covers 8 j .. 8 j + 7 of every quarter's 32.
template <bool kFine>
__device__ __forceinline__ int step_offset(int q, int j) {
  return kFine ? 32 * j + 8 * q : 32 * q + 8 * j;
}

// Few rows: 16 outputs per workgroup, whose kW waves take the chunks of the reduction in turn, each
// with kM x 16 rows of X; operands go straight from memory to the matrix unit.  Bound by the
// weights' bytes: a wave has kU chunks of them in flight.
template <awe_dtype T, int kM, bool kFine>
__global__ __launch_bounds__(512) void w4_rows_kernel(W4Args a) {
  using X = Kind<T>;
  constexpr int kW = 8, kU = kM == 1 ? 4 : kM == 2 ? 2 : 1;
  const W4Launch& g = a.g;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * 16 * kM;
  const int64_t n = n0 + i < g.N ? n0 + i : g.N - 1;
  const uint8_t* w = g.w + n * g.ldw + 16 * q;
  const typename X::Elem* x[kM];
  bool ok[kM];
#pragma unroll
  for (int t = 0; t < kM; ++t) {
    ok[t] = m0 + 16 * t + i < g.M;
    x[t] = reinterpret_cast<const typename X::Elem*>(g.x) + (ok[t] ? m0 + 16 * t + i : 0) * g.ldx;
  }
  const uint32_t magic = X::magic();
  f4 acc[kM];
#pragma unroll
  for (int t = 0; t < kM; ++t) acc[t] = f4{0.f, 0.f, 0.f, 0.f};

  // adds a group's part: part - (bias + z) sum x, times the group's scale
  auto fold = [&](const typename X::Acc* part, const typename X::Acc* sum, float s, float z) {
    const float b = X::kBias + z;
#pragma unroll
    for (int t = 0; t < kM; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t][r] += s * ((float)part[t][r] - b * (float)sum[t][r]);
  };
  auto chunk = [&](u4 cw, const typename X::Raw (&xr)[kM][4], const float* s, const float* z) {
    typename X::Acc part[kM], sum[kM];
    if (kFine) cw = across_quarters(cw);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const typename X::Op c = X::codes(cw[j], magic);
      const bool first = kFine || j == 0;
#pragma unroll
      for (int t = 0; t < kM; ++t) {
        const typename X::Op e = X::elems(xr[t][j]);
        part[t] = X::mul(e, c, first ? X::zero() : part[t]);
        sum[t] = X::mul(e, X::ones(), first ? X::zero() : sum[t]);
      }
      if (kFine || j == 3) fold(part, sum, s[kFine ? j : 0], z[kFine ? j : 0]);
    }
  };
  // scale and zero point of lane's output in the group of unit u (128 or 32 indices)
  constexpr int kS = kFine ? 4 : 1;
  auto scales = [&](int32_t c, float* s, float* z, int units) {
#pragma unroll
    for (int j = 0; j < kS; ++j) {
      const int32_t grp = (uint32_t)(kFine ? 4 * c + (j < units ? j : 0) : c) / (uint32_t)a.units;
      s[j] = load_real(g.scales, n * g.lds + grp, g.s_type);
      z[j] = g.zeros != nullptr ? (float)g.zeros[n * g.ldz + grp] : 8.f;
    }
  };

  const int32_t full = (int32_t)(g.K / kChunk);
  for (int32_t c0 = wave; c0 < full; c0 += kW * kU) {
    u4 cw[kU];
    typename X::Raw xr[kU][kM][4];
    float s[kU][kS], z[kU][kS];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int32_t c = c0 + u * kW;
      if (c < full) {
        const Any16 v = *reinterpret_cast<const Any16*>(w + (int64_t)c * (kChunk / 2));
        cw[u] = u4{v.w[0], v.w[1], v.w[2], v.w[3]};
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int32_t c = c0 + u * kW;
      if (c < full) {
#pragma unroll
        for (int t = 0; t < kM; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            xr[u][t][j] = ok[t] ? load8<T>(x[t] + (int64_t)c * kChunk + step_offset<kFine>(q, j)) : none<T>();
        scales(c, s[u], z[u], 4);
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (c0 + u * kW < full) chunk(cw[u], xr[u], s[u], z[u]);
  }
  // the last, short chunk
  if ((int64_t)full * kChunk < g.K && full % kW == wave) {
    const int64_t k0 = (int64_t)full * kChunk;
    const int left = (int)(g.K - k0), bytes = (left + 1) / 2 - 16 * q;
    u4 cw = {0, 0, 0, 0};
    const uint8_t* p = w + k0 / 2;
#pragma unroll
    for (int b = 0; b < 16; ++b) cw[b >> 2] |= (b < bytes ? (uint32_t)p[b] : 0u) << (8 * (b & 3));
    typename X::Raw xr[kM][4];
#pragma unroll
    for (int t = 0; t < kM; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int off = step_offset<kFine>(q, j);
        xr[t][j] = load8_short<T>(x[t] + k0 + off, ok[t] ? left - off : 0);
      }
    float s[kS], z[kS];
    scales(full, s, z, (left + 31) / 32);
    chunk(cw, xr, s, z);
  }

  // the waves' sums, and Y
  __shared__ float red[kW][16 * kM][17];
#pragma unroll
  for (int t = 0; t < kM; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) red[wave][16 * t + 4 * q + r][i] = acc[t][r];
  __syncthreads();
  for (int e = threadIdx.x; e < 256 * kM; e += 512) {
    const int64_t m = m0 + (e >> 4), j = n0 + (e & 15);
    if (m >= g.M || j >= g.N) continue;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kW; ++k) v += red[k][e >> 4][e & 15];
    store_real(g.y, m * g.ldy + j, g.y_type, g.x_scales != nullptr ? v * g.x_scales[m] : v);
  }
}

template <awe_dtype T, int kM>
awe_status launch_rows(const W4Args& a, bool fine, hipStream_t stream) {
  const dim3 grid((unsigned)((a.g.N + 15) / 16), (unsigned)((a.g.M + 16 * kM - 1) / (16 * kM)));
  if (fine)
    hipLaunchKernelGGL((w4_rows_kernel<T, kM, true>), grid, dim3(512), 0, stream, a);
  else
    hipLaunchKernelGGL((w4_rows_kernel<T, kM, false>), grid, dim3(512), 0, stream, a);
  return launched("w4 launch");
}

template <awe_dtype T>
awe_status launch_kind(const W4Args& a, bool fine, hipStream_t stream) {
  if (a.g.M <= 16) return launch_rows<T, 1>(a, fine, stream);
  if (a.g.M <= 32) return launch_rows<T, 2>(a, fine, stream);
  return launch_rows<T, 4>(a, fine, stream);
}

}  // namespace

awe_status launch_w4(const W4Launch& g, hipStream_t stream) {
  // one group of at least K indices counts as a long one
  const bool fine = g.group % kChunk != 0 && g.group < g.K;
  const int64_t group = g.group < g.K ? g.group : (g.K + kChunk - 1) / kChunk * kChunk;
  W4Args a{g, (int32_t)std::max<int64_t>(1, group / (fine ? 32 : kChunk))};
  if (g.x_type == AWE_BF16) return launch_kind<AWE_BF16>(a, fine, stream);
  if (g.x_type == AWE_F16) return launch_kind<AWE_F16>(a, fine, stream);
  return launch_kind<AWE_I8>(a, fine, stream);
}

}  // namespace awe

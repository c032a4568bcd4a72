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
  int32_t units;           // group / 128, or group / 32 where 128 does not divide it
  int32_t step_g, step_u;  // 8 chunks are step_g groups and step_u units
};

// The chunk of a lane: row n of W at indices 32 q .. 32 q + 31 of the chunk.  kFine: a group may begin at any
// multiple of 32 indices, so each product of 32 indices has to lie in one group: the words are
// transposed over the quarters, and step j covers indices 32 j .. 32 j + 31 (8 q .. 8 q + 7 of them in
// this lane); otherwise step j covers 8 j .. 8 j + 7 of every quarter's 32.
template <bool kFine>
__device__ __forceinline__ int step_offset(int q, int j) {
  return kFine ? 32 * j + 8 * q : 32 * q + 8 * j;
}

// A scale as it lies in memory, and its value.
template <bool kS4>
__device__ __forceinline__ uint32_t raw_scale(const void* p, int64_t i) {
  if constexpr (kS4)
    return reinterpret_cast<const uint32_t*>(p)[i];
  else
    return reinterpret_cast<const uint16_t*>(p)[i];
}
template <bool kS4>
__device__ __forceinline__ float scale_value(uint32_t raw, bool is_bf16) {
  if constexpr (kS4) return __builtin_bit_cast(float, raw);
  const float h = (float)__builtin_bit_cast(_Float16, (uint16_t)raw);
  return is_bf16 ? __builtin_bit_cast(float, raw << 16) : h;
}

// Few rows: 16 outputs per workgroup, whose kW waves take the chunks of the reduction in turn, each
// with kM x 16 rows of X; operands go straight from memory to the matrix unit.  Bound by the
// weights' bytes: a wave has kD chunks of them in flight, and the rows of one chunk ahead.
constexpr int kW = 8;
template <awe_dtype T, int kM, bool kFine, bool kS4>
__global__ __launch_bounds__(64 * kW, kM == 1 ? 4 : 2) void w4_rows_kernel(W4Args a) {
  using X = Kind<T>;
  constexpr int kD = kFine ? 2 : (kM == 1 ? 8 : 4);   // chunks of W in flight
  constexpr int kX = kFine && kM == 4 ? 1 : 2;          // chunks of X (kD is a multiple)
  constexpr int kS = kFine ? 4 : 1;
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
  const bool is_bf16 = g.s_type == AWE_BF16, has_z = g.zeros != nullptr;
  const int64_t s0 = n * g.lds, z0 = n * g.ldz;
  const uint8_t* zp = has_z ? g.zeros : g.w;  // (any byte, where there are none)
  const uint32_t magic = X::magic();
  f4 acc[kM];
#pragma unroll
  for (int t = 0; t < kM; ++t) acc[t] = f4{0.f, 0.f, 0.f, 0.f};

  // adds a group's part: part - (bias + z) sum x, times the group's scale
  auto fold = [&](const typename X::Acc* part, const typename X::Acc* sum, uint32_t rs, uint32_t rz) {
    const float s = scale_value<kS4>(rs, is_bf16), b = X::kBias + (has_z ? (float)rz : 8.f);
#pragma unroll
    for (int t = 0; t < kM; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t][r] += s * ((float)part[t][r] - b * (float)sum[t][r]);
  };
  auto chunk = [&](u4 cw, const typename X::Raw (&xr)[kM][4], const uint32_t* s, const uint32_t* z) {
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
  // Scales and zero points of the lane's output in the groups of a chunk whose first unit is unit `u` of
  // group `grp`; groups past `last` are not touched.
  auto scales = [&](int32_t grp, int32_t u, int32_t last, uint32_t* s, uint32_t* z) {
#pragma unroll
    for (int j = 0; j < kS; ++j) {
      const int32_t at = grp < last ? grp : last;
      s[j] = raw_scale<kS4>(g.scales, s0 + at);
      z[j] = zp[has_z ? z0 + at : 0];
      if (++u == a.units) u = 0, ++grp;
    }
  };
  auto codes = [&](int32_t c) {
    const Any16 v = *reinterpret_cast<const Any16*>(w + (int64_t)c * (kChunk / 2));
    return u4{v.w[0], v.w[1], v.w[2], v.w[3]};
  };
  auto rows = [&](int32_t c, typename X::Raw (&xr)[kM][4]) {
#pragma unroll
    for (int t = 0; t < kM; ++t) {
      const typename X::Elem* p = x[t] + (int64_t)c * kChunk;
      if constexpr (T == AWE_I8 && !kFine) {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const u4 v = ok[t] ? load8<AWE_BF16>(reinterpret_cast<const uint16_t*>(p + step_offset<kFine>(q, j))) : u4{0, 0, 0, 0};
          xr[t][j] = (uint64_t)v[0] | (uint64_t)v[1] << 32;
          xr[t][j + 1] = (uint64_t)v[2] | (uint64_t)v[3] << 32;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) xr[t][j] = ok[t] ? load8<T>(p + step_offset<kFine>(q, j)) : none<T>();
      }
    }
  };

  // chunk wave + 8 t begins in unit `unit` of group `grp` (ahead: of the chunk that is fetched next)
  const int32_t full = (int32_t)(g.K / kChunk);
  const uint32_t first_unit = (uint32_t)wave * (kFine ? 4 : 1);
  int32_t grp = (int32_t)(first_unit / (uint32_t)a.units), unit = (int32_t)(first_unit % (uint32_t)a.units);
  auto next = [&] {
    grp += a.step_g;
    unit += a.step_u;
    if (unit >= a.units) unit -= a.units, ++grp;
  };
  const int32_t last = (int32_t)((g.K - 1) / g.group);
  if (wave < full) {
    u4 cw[kD];
    typename X::Raw xr[kX][kM][4];
    uint32_t s[kD][kS], z[kD][kS];
#pragma unroll
    for (int u = 0; u < kD; ++u) {  // (past the end: the last chunk again, unused)
      const int32_t c = wave + u * kW;
      cw[u] = codes(c < full ? c : full - 1);
      scales(grp, unit, last, s[u], z[u]);
      next();
    }
    if (kX == 2) rows(wave, xr[0]);
    for (int32_t c0 = wave; c0 < full; c0 += kW * kD) {
#pragma unroll
      for (int u = 0; u < kD; ++u) {
        const int32_t c = c0 + u * kW;
        if (c >= full) break;
        if (kX == 2)
          rows(c + kW < full ? c + kW : full - 1, xr[(u + 1) % kX]);
        else
          rows(c, xr[0]);
        chunk(cw[u], xr[u % kX], s[u], z[u]);
        const int32_t ahead = c + kW * kD;
        if (ahead < full) {
          cw[u] = codes(ahead);
          scales(grp, unit, last, s[u], z[u]);
          next();
        }
      }
    }
  }
  // the last, short chunk, filled up with zeros in LDS
  __shared__ union {
    float red[kW][16 * kM][17];
    struct {
      alignas(16) uint8_t w[16][kChunk / 2];
      alignas(16) typename X::Elem x[16 * kM][kChunk];
    } end;
  } lds;
  if ((int64_t)full * kChunk < g.K) {
    const int64_t k0 = (int64_t)full * kChunk;
    const int left = (int)(g.K - k0);
    for (int e = threadIdx.x; e < 16 * (kChunk / 2); e += 64 * kW) {
      const int64_t row = n0 + e / (kChunk / 2);
      const int b = e % (kChunk / 2);
      lds.end.w[e / (kChunk / 2)][b] = row < g.N && 2 * b < left ? g.w[row * g.ldw + k0 / 2 + b] : 0;
    }
    for (int e = threadIdx.x; e < 16 * kM * kChunk; e += 64 * kW) {
      const int64_t row = m0 + e / kChunk;
      const int k = e % kChunk;
      lds.end.x[e / kChunk][k] =
          row < g.M && k < left ? reinterpret_cast<const typename X::Elem*>(g.x)[row * g.ldx + k0 + k] : 0;
    }
    __syncthreads();
    if (full % kW == wave) {
      const u4 cw = *reinterpret_cast<const u4*>(&lds.end.w[i][16 * q]);
      typename X::Raw xr[kM][4];
#pragma unroll
      for (int t = 0; t < kM; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          xr[t][j] = *reinterpret_cast<const typename X::Raw*>(&lds.end.x[16 * t + i][step_offset<kFine>(q, j)]);
      uint32_t s[kS], z[kS];
      const uint32_t u0 = (uint32_t)full * (kFine ? 4 : 1);
      scales((int32_t)(u0 / (uint32_t)a.units), (int32_t)(u0 % (uint32_t)a.units), last, s, z);
      chunk(cw, xr, s, z);
    }
    __syncthreads();
  }

  // the waves' sums, and Y
#pragma unroll
  for (int t = 0; t < kM; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) lds.red[wave][16 * t + 4 * q + r][i] = acc[t][r];
  __syncthreads();
  for (int e = threadIdx.x; e < 256 * kM; e += 64 * kW) {
    const int64_t m = m0 + (e >> 4), j = n0 + (e & 15);
    if (m >= g.M || j >= g.N) continue;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kW; ++k) v += lds.red[k][e >> 4][e & 15];
    store_real(g.y, m * g.ldy + j, g.y_type, g.x_scales != nullptr ? v * g.x_scales[m] : v);
  }
}

template <awe_dtype T, int kM>
awe_status launch_rows(const W4Args& a, bool fine, hipStream_t stream) {
  const dim3 grid((unsigned)((a.g.N + 15) / 16), (unsigned)((a.g.M + 16 * kM - 1) / (16 * kM))), block(64 * kW);
  const bool s4 = a.g.s_type == AWE_F32;
  if (fine && s4)
    hipLaunchKernelGGL((w4_rows_kernel<T, kM, true, true>), grid, block, 0, stream, a);
  else if (fine)
    hipLaunchKernelGGL((w4_rows_kernel<T, kM, true, false>), grid, block, 0, stream, a);
  else if (s4)
    hipLaunchKernelGGL((w4_rows_kernel<T, kM, false, true>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((w4_rows_kernel<T, kM, false, false>), grid, block, 0, stream, a);
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
  W4Args a{g, 1, 0, 0};
  if (g.group >= g.K) a.g.group = std::max<int64_t>(1, (g.K + kChunk - 1) / kChunk) * kChunk;
  a.units = (int32_t)(a.g.group / (fine ? 32 : kChunk));
  const int32_t units = kW * (fine ? 4 : 1);  // of kW chunks
  a.step_g = units / a.units;
  a.step_u = units % a.units;
  if (g.x_type == AWE_BF16) return launch_kind<AWE_BF16>(a, fine, stream);
  if (g.x_type == AWE_F16) return launch_kind<AWE_F16>(a, fine, stream);
  return launch_kind<AWE_I8>(a, fine, stream);
}

}  // namespace awe

// paged_device.h -- what the kernels over the paged key/value cache share: element types, the
// row quantisation rule and where a token lies.
#pragma once

#include "tilemix_device.h"
#include "tilemix_internal.h"

#include <type_traits>

namespace tilemix {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// 16-bit element types by their tilemix_format.
template <int TYPE>
struct Elem;
template <>
struct Elem<TILEMIX_FP16> {
  typedef _Float16 t;
  static constexpr uint32_t kInf = 0x7c00;   // bits of infinity: finite magnitudes lie below
};
template <>
struct Elem<TILEMIX_BF16> {
  typedef __bf16 t;
  static constexpr uint32_t kInf = 0x7f80;
};

template <int TYPE>
__device__ __forceinline__ float bits_to_float(uint32_t low16) {
  if constexpr (TYPE == TILEMIX_BF16) return __builtin_bit_cast(float, low16 << 16);
  return half_bits_to_float((uint16_t)low16);
}

template <int TYPE>
__device__ __forceinline__ uint32_t float_to_bits(float x) {   // round to nearest even
  return __builtin_bit_cast(uint16_t, (typename Elem<TYPE>::t)x);
}

constexpr bool is_8bit(int format) { return format == TILEMIX_INT8 || format == TILEMIX_E4M3; }
template <int FORMAT>
constexpr int kElemBytes = is_8bit(FORMAT) ? 1 : 2;
template <int FORMAT>
constexpr float kTop = FORMAT == TILEMIX_INT8 ? 127.0f : 448.0f;

// Page and slot of token t of sequence b; page < 0: none (t outside the table, or no page there).
struct Slot {
  int page, slot;
};
__device__ __forceinline__ Slot find_slot(const PagedPool& p, int b, long long t) {
  const long long e = t >> p.page_shift;
  if (t < 0 || e >= p.max_pages) return {-1, 0};
  const int page = p.table[b * p.stride_table + e];
  return {page >= 0 && page < p.pages ? page : -1, (int)(t & ((1 << p.page_shift) - 1))};
}

// The rule that makes the codes of a row with a = max |x| > 0, finite: the exact quotient top x / a, rounded once.
// Both are scaled by one power of two, 2^e, so that nothing overflows and a loses no bits (subnormal rows
// included).  t = 2^e top x is then exact in FP32 (127, and 448 = 7 2^6: at most 18 bits), and so is the
// residual t - q0 a of an estimate q0, so that q = q0 + (t - q0 a) r with r within 2^-22 of 1 / a is the correctly
// rounded quotient: it errs by 2^-44 of it before it is rounded, and a quotient of 18 by 11 bits is no
// nearer than 2^-36 to the midpoint of two FP32 numbers.  Such a quotient that is no tie of the codes' grid is
// further from one than 2^-23 of itself, so rounding q again, to the code, gives the code of the exact
// quotient (checked for every pair of such numbers).
template <int FORMAT>
struct RowScale {
  float a, rcp;     // 2^e a and its reciprocal
  float m;          // 2^e top
  float scale;      // as stored
  bool plain;       // a > 0 and finite: otherwise all codes are 0
  // amax: bits of max |x| of a row of TYPE.
  template <int TYPE>
  __device__ __forceinline__ static RowScale of(uint32_t amax) {
    RowScale r;
    const float x = bits_to_float<TYPE>(amax);
    const bool finite = amax < Elem<TYPE>::kInf;
    r.plain = finite && amax > 0;
    // a / top, correctly rounded, by the same residual step (where the quotient is not subnormal).
    constexpr float kInv = 1.0f / kTop<FORMAT>;
    const float s0 = x * kInv;
    r.scale = fmaf(fmaf(-s0, kTop<FORMAT>, x), kInv, s0);
    if (x < 0x1p-100f) r.scale = x / kTop<FORMAT>;
    r.scale = finite ? r.scale : __builtin_nanf("");
    // 2^e a in [1, 2); for rows below 2^-118 (BF16) less, down to 2^-14, since 2^e top has to be finite.
    const int e = r.plain ? min(1 - __builtin_amdgcn_frexp_expf(x), 119) : 0;
    r.a = r.plain ? __builtin_amdgcn_ldexpf(x, e) : 1.0f;
    r.rcp = __builtin_amdgcn_rcpf(r.a);
    r.m = __builtin_amdgcn_ldexpf(kTop<FORMAT>, e);
    return r;
  }
  // top x / a.
  __device__ __forceinline__ float quot(float x) const {
    const float t = x * m, q0 = t * rcp;
    return fmaf(fmaf(-q0, a, t), rcp, q0);
  }
  // Codes of four values as bytes, the first lowest.
  __device__ __forceinline__ uint32_t codes(float x0, float x1, float x2, float x3) const {
    const float q0 = quot(x0), q1 = quot(x1), q2 = quot(x2), q3 = quot(x3);
    uint32_t w;
    if constexpr (FORMAT == TILEMIX_INT8) {
      auto word = [](float q) { return __builtin_bit_cast(uint32_t, q + 12582912.0f); };
      w = pack4(word(q0), word(q1), word(q2), word(q3));
    } else {
      // |q| <= 448 (1 + 2^-24), which rounds to 448: the conversion never saturates.
      w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q0, q1, 0, false);
      w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q2, q3, (int)w, true);
    }
    return plain ? w : 0u;
  }
};

// Four codes times the row's scale, each rounded to FP32 (the empty asm keeps the compiler from joining the
// product with a conversion to FP16 in one mixed-precision instruction, which rounds once only).
template <int FORMAT>
__device__ __forceinline__ void widen4(uint32_t w, float scale, float (&x)[4]) {
  if constexpr (FORMAT == TILEMIX_INT8) {
    // With the sign bit flipped a byte reads as code + 128.
    const uint32_t u = w ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = ((float)((u >> (8 * i)) & 0xffu) - 128.0f) * scale;
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0] * scale;
    x[1] = lo[1] * scale;
    x[2] = hi[0] * scale;
    x[3] = hi[1] * scale;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("" : "+v"(x[i]));
}

// f(D, TYPE, FORMAT) as integral constants.
template <typename F>
inline hipError_t for_paged_types(int d, int type, int format, F&& f) {
  using std::integral_constant;
  auto by_format = [&](auto D) -> hipError_t {
    using H = integral_constant<int, TILEMIX_FP16>;
    using B = integral_constant<int, TILEMIX_BF16>;
    using I = integral_constant<int, TILEMIX_INT8>;
    using E = integral_constant<int, TILEMIX_E4M3>;
    if (type == TILEMIX_FP16) {
      if (format == TILEMIX_FP16) return f(D, H{}, H{});
      if (format == TILEMIX_INT8) return f(D, H{}, I{});
      if (format == TILEMIX_E4M3) return f(D, H{}, E{});
    } else if (type == TILEMIX_BF16) {
      if (format == TILEMIX_BF16) return f(D, B{}, B{});
      if (format == TILEMIX_INT8) return f(D, B{}, I{});
      if (format == TILEMIX_E4M3) return f(D, B{}, E{});
    }
    return hipErrorInvalidValue;
  };
  if (d == 128) return by_format(integral_constant<int, 128>{});
  if (d == 64) return by_format(integral_constant<int, 64>{});
  return hipErrorInvalidValue;
}

}  // namespace tilemix

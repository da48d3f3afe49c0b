// Device helpers that several translation units share: values of the three float types in groups of eight, sums and maxima over a
// wavefront, e4m3 with power-of-two scales.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <utility>

namespace jenga {

// Compile-time loop: f(integral_constant<int, 0>) ... f(integral_constant<int, N - 1>).
template <typename F, int... Is>
__device__ __forceinline__ void each_impl(F&& f, std::integer_sequence<int, Is...>) {
  (f(std::integral_constant<int, Is>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each_impl(f, std::make_integer_sequence<int, N>{});
}

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// 16 bytes at any address that is a multiple of two (or four) bytes: ordinary loads and stores take any address.
struct __attribute__((packed, aligned(2))) Piece16 {
  uint32_t w[4];
};
struct __attribute__((packed, aligned(4))) Piece32 {
  uint32_t w[8];
};

// Eight values as they lie in memory, and in float32.  Rounding to 16 bits is to nearest even.
template <typename T>
struct Eight;
template <>
struct Eight<__bf16> {
  typedef Piece16 raw;
  static __device__ __forceinline__ f32x8 wide(const raw& r) {
    bf16x8 v;
    __builtin_memcpy(&v, &r, 16);
    return __builtin_convertvector(v, f32x8);
  }
  static __device__ __forceinline__ raw narrow(const f32x8& f) {
    const bf16x8 v = __builtin_convertvector(f, bf16x8);
    raw r;
    __builtin_memcpy(&r, &v, 16);
    return r;
  }
};
template <>
struct Eight<_Float16> {
  typedef Piece16 raw;
  static __device__ __forceinline__ f32x8 wide(const raw& r) {
    f16x8 v;
    __builtin_memcpy(&v, &r, 16);
    return __builtin_convertvector(v, f32x8);
  }
  static __device__ __forceinline__ raw narrow(const f32x8& f) {
    const f16x8 v = __builtin_convertvector(f, f16x8);
    raw r;
    __builtin_memcpy(&r, &v, 16);
    return r;
  }
};
template <>
struct Eight<float> {
  typedef Piece32 raw;
  static __device__ __forceinline__ f32x8 wide(const raw& r) {
    f32x8 v;
    __builtin_memcpy(&v, &r, 32);
    return v;
  }
  static __device__ __forceinline__ raw narrow(const f32x8& f) {
    raw r;
    __builtin_memcpy(&r, &f, 32);
    return r;
  }
};

// The first n of eight values (n may be more); what is behind them reads as +0.
template <typename T>
__device__ __forceinline__ typename Eight<T>::raw load_eight(const T* p, int64_t n) {
  typename Eight<T>::raw r;
  if (n >= 8) {
    r = *(const typename Eight<T>::raw*)p;
  } else {
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = (T)0.0f;
      if (i < n) v[i] = p[i];
    }
    __builtin_memcpy(&r, v, sizeof(r));
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void store_eight(T* p, const f32x8& f, int64_t n) {
  if (n >= 8) {
    *(typename Eight<T>::raw*)p = Eight<T>::narrow(f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (T)f[i];
  }
}

// Reductions in the vector ALU (DPP).  row_shr 1, 2, 4, 8 leave the result of each row of 16 lanes in its last lane, row_bcast
// 15 and 31 join the rows in lane 63; row_ror 8, 4, 2, 1 leave it in all 16 lanes.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_f32(float old, float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, x), CTRL, ROW_MASK,
                                                               0xF, false));
}
__device__ __forceinline__ float wave_sum_f32(float v) {
  v += dpp_f32<0x111, 0xF>(0.f, v);
  v += dpp_f32<0x112, 0xF>(0.f, v);
  v += dpp_f32<0x114, 0xF>(0.f, v);
  v += dpp_f32<0x118, 0xF>(0.f, v);
  v += dpp_f32<0x142, 0xA>(0.f, v);
  v += dpp_f32<0x143, 0xC>(0.f, v);
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float row_max_f32(float v) {   // over the 16 lanes of a DPP row
  v = fmaxf(v, dpp_f32<0x128, 0xF>(v, v));
  v = fmaxf(v, dpp_f32<0x124, 0xF>(v, v));
  v = fmaxf(v, dpp_f32<0x122, 0xF>(v, v));
  v = fmaxf(v, dpp_f32<0x121, 0xF>(v, v));
  return v;
}

// e4m3 with a power-of-two scale: values v of a block are kept as e4m3(v 2^-e), e the least whole number with
// max |v| <= 448 2^e over the block's finite values (0 where they are all zero), at least -127; the scale byte is e + 127.
// Multiplying by a power of two is exact, so the only rounding is the one to e4m3 (nearest even, v_cvt_pk_fp8_f32); what is
// not finite becomes NaN.
__device__ __forceinline__ float finite_magnitude(float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? a : 0.f;   // NaN compares false
}
__device__ __forceinline__ uint32_t scale_byte(float largest) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, largest);
  if (bits == 0) return 127;
  const int e = (int)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);   // 448 = 1.75 * 2^8
  return e < 0 ? 0u : (uint32_t)e;
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }
__device__ __forceinline__ uint2 to_e4m3(const f32x8& v, float inverse) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inverse, v[1] * inverse, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inverse, v[3] * inverse, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inverse, v[5] * inverse, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inverse, v[7] * inverse, hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}
__device__ __forceinline__ float largest_of(const f32x8& v) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));   // NaN loses
  if (m == __builtin_inff()) {
    m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_magnitude(v[i]));
  }
  return m;
}

// e2m1 with a power-of-two scale: values v of a block of 32 are kept as e2m1(v 2^-e), e the least whole number with max |v| <= 6 2^e
// (0 where they are all zero), at least -127; the scale byte is e + 127, and 255 where a value is not finite.  Multiplying by a
// power of two is exact, so the only rounding is the one to e2m1 (nearest, ties to even, v_cvt_scalef32_pk_fp4_f32).
__device__ __forceinline__ float magnitude_of(const f32x8& v) {   // NaN wins
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = v[i];   // a bit cast of an element in its place takes the first one (clang 22)
    m = max(m, __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu);
  }
  return __builtin_bit_cast(float, m);
}
__device__ __forceinline__ float quad_max(float v) {   // over four neighbouring lanes, of magnitudes; NaN wins
  auto bits = [](float f) { return __builtin_bit_cast(uint32_t, f); };
  uint32_t m = max(bits(v), bits(dpp_f32<0xB1, 0xF>(0.f, v)));
  m = max(m, bits(dpp_f32<0x4E, 0xF>(0.f, __builtin_bit_cast(float, m))));
  return __builtin_bit_cast(float, m);
}
__device__ __forceinline__ uint32_t mx_scale_byte(float largest) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, largest);
  if (bits == 0) return 127;
  if (bits >= 0x7F800000u) return 255;
  const int e = (int)(bits >> 23) - 2 + ((bits & 0x7FFFFFu) > 0x400000u ? 1 : 0);   // 6 = 1.5 * 2^2
  return e < 0 ? 0u : (uint32_t)e;
}
// Eight values, the first in the lowest four bits.
__device__ __forceinline__ uint32_t to_e2m1(const f32x8& v, uint32_t byte) {
  uint32_t r = 0;
#if defined(__HIP_DEVICE_COMPILE__)
  const float inverse = inverse_scale(min(byte, 254u));
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0] * inverse, v[1] * inverse, 1.0f, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2] * inverse, v[3] * inverse, 1.0f, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4] * inverse, v[5] * inverse, 1.0f, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6] * inverse, v[7] * inverse, 1.0f, 3);
  if (byte == 255u) r = 0;   // its scale says it all
#endif
  return r;
}

}  // namespace jenga

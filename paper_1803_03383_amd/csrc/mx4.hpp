// 4-bit microscaled values (MX4): device-side pieces shared by the quantizer, the products and the
// reader.  A block of 32 values has the scale 2^(s - 127), the smallest power of two (s >= 0) with
// max |x| <= 6 2^(s - 127); a value is a sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6.
#pragma once

#include <type_traits>

#include "halp_device.hpp"
#include "../../include/halp.h"

namespace halp {

using v2bf16 = __bf16 __attribute__((ext_vector_type(2)));
using v2f16 = _Float16 __attribute__((ext_vector_type(2)));
using v4f32 = float __attribute__((ext_vector_type(4)));
using v16f32 = float __attribute__((ext_vector_type(16)));
using v4i32 = int __attribute__((ext_vector_type(4)));
using v8i32 = int __attribute__((ext_vector_type(8)));

constexpr int kMxBlock = 32;   // values per scale
constexpr int kMxGroup = 128;  // values per stored group: 64 bytes of codes, 4 scales
constexpr int64_t kMxRowMost = 131072;  // columns of the row product: a row of x fits LDS

inline __host__ __device__ int64_t mx_groups(int64_t cols) { return (cols + kMxGroup - 1) / kMxGroup; }

struct MxView {  // a halp_mx4 as kernels take it
  uint8_t* codes;
  uint8_t* scales;
  int64_t ldc, lds, rows, cols;
};

inline MxView mx_view(const halp_mx4& q) {
  return MxView{static_cast<uint8_t*>(q.codes), q.scales, q.ldc, q.lds, q.rows, q.cols};
}

// scale byte of a block whose largest magnitude has these fp32 bits: max = 1.f 2^e needs 2^(e - 2),
// and 2^(e - 1) past 1.5 2^e = 6 2^(e - 2); 255 where it is not finite
__device__ __forceinline__ uint32_t mx_scale(uint32_t max_bits) {
  const int s = (int)(max_bits >> 23) - 2 + ((max_bits & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return max_bits >= 0x7F800000u ? 255u : (uint32_t)(s > 0 ? s : 0);
}

// 2^(127 - s) for s <= 254: what a value is multiplied by (exact); 0 for s = 255, so that its codes are 0
__device__ __forceinline__ float mx_inverse(uint32_t s) {
  return __builtin_bit_cast(float, s == 255u ? 0u : (254u - s) << 23);
}

// 2^(s - 127) (2^-127 is subnormal), NaN for s = 255
__device__ __forceinline__ float mx_scale_value(uint32_t s) {
  return __builtin_bit_cast(float, s == 255u ? 0x7FC00000u : (s ? s << 23 : 0x400000u));
}

// ---- 16 bytes of values in one lane: four floats, or eight of 16 bits ------------------------------
using v2f32 = float __attribute__((ext_vector_type(2)));
using v2u16 = unsigned short __attribute__((ext_vector_type(2)));

// the values from p on (any alignment of T), n of them, zeros behind
template <typename T>
__device__ __forceinline__ uint4 mx_load16(const T* p, int64_t n) {
  constexpr int kV = 16 / sizeof(T);
  struct __attribute__((packed, aligned(sizeof(T)))) Loose { uint32_t w[4]; };
  if (n >= kV) {
    const Loose l = *reinterpret_cast<const Loose*>(p);
    return uint4{l.w[0], l.w[1], l.w[2], l.w[3]};
  }
  uint32_t w[4] = {};
#pragma unroll
  for (int e = 0; e < kV; ++e)
    if (e < n) {
      if constexpr (sizeof(T) == 4) w[e] = __builtin_bit_cast(uint32_t, p[e]);
      else w[e / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, p[e]) << (16 * (e % 2));
    }
  return uint4{w[0], w[1], w[2], w[3]};
}

// Bits in T of the largest magnitude: those of magnitudes are ordered as whole numbers, NaN above infinity.
template <typename T>
__device__ __forceinline__ uint32_t mx_max16(uint4 v) {
  if constexpr (sizeof(T) == 4) {
    constexpr uint32_t k = 0x7FFFFFFFu;
    return max(max(v.x & k, v.y & k), max(v.z & k, v.w & k));
  } else {
    const auto pair = [](uint32_t w) { return __builtin_bit_cast(v2u16, w & 0x7FFF7FFFu); };
    const v2u16 m = __builtin_elementwise_max(__builtin_elementwise_max(pair(v.x), pair(v.y)), __builtin_elementwise_max(pair(v.z), pair(v.w)));
    return max((uint32_t)m.x, (uint32_t)m.y);
  }
}

// largest of 4 or 8 adjacent lanes
template <int LANES>
__device__ __forceinline__ uint32_t mx_max_of_lanes(uint32_t m) {
  m = max(m, dpp_quad_swap1(m));
  m = max(m, dpp_quad_swap2(m));
  if constexpr (LANES == 8) m = max(m, dpp_half_mirror(m));
  return m;
}

// fp32 bits of a magnitude from its bits in T
template <typename T>
__device__ __forceinline__ uint32_t mx_max_bits(uint32_t m) {
  if constexpr (std::is_same_v<T, float>) return m;
  else if constexpr (std::is_same_v<T, __bf16>) return m << 16;
  else return __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)m));
}

// Two values to the byte SEL of c, to the nearest with ties to the even code: v_cvt_scalef32_pk_fp4 divides by the
// scale's power of two and rounds so.  w: two 16-bit values, or the first of two floats.
template <typename T, int SEL>
__device__ __forceinline__ uint32_t mx_codes2(uint32_t c, uint32_t w, uint32_t w2, float scale) {
  if constexpr (std::is_same_v<T, float>)
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __builtin_bit_cast(float, w), __builtin_bit_cast(float, w2), scale, SEL);
  else if constexpr (std::is_same_v<T, __bf16>)
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2bf16, w), scale, SEL);
  else
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(v2f16, w), scale, SEL);
}

// the lane's four or eight codes
template <typename T>
__device__ __forceinline__ uint32_t mx_codes16(uint4 v, uint32_t s) {
  const float scale = __builtin_bit_cast(float, s << 23);
  uint32_t c = 0;
  if constexpr (sizeof(T) == 4) {
    c = mx_codes2<T, 0>(c, v.x, v.y, scale);
    c = mx_codes2<T, 1>(c, v.z, v.w, scale);
  } else {
    c = mx_codes2<T, 0>(c, v.x, 0, scale);
    c = mx_codes2<T, 1>(c, v.y, 0, scale);
    c = mx_codes2<T, 2>(c, v.z, 0, scale);
    c = mx_codes2<T, 3>(c, v.w, 0, scale);
  }
  return s == 255u ? 0u : c;
}

template <typename T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }

template <typename F>
int with_type(int32_t type, F&& f) {  // f(a value of the type); the caller has checked the number
  switch (type) {
    case HALP_TYPE_F32: return f(float{});
    case HALP_TYPE_BF16: return f(__bf16{});
    default: return f(_Float16{});
  }
}

inline int type_bytes(int32_t type) { return type == HALP_TYPE_F32 ? 4 : 2; }
inline bool type_known(int32_t type) { return type >= HALP_TYPE_F32 && type <= HALP_TYPE_F16; }

// launchers; arguments have been checked
int launch_mx4_quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ldx, const MxView* q,
                        const MxView* qt, int32_t rounding, uint64_t seed, uint32_t epoch, int cus, hipStream_t s);
int launch_mx4_dequantize(const MxView& q, void* out, int32_t type, int64_t ldo, hipStream_t s);
int launch_mx4_product(const MxView& a, const MxView& b, void* c, int32_t type, int64_t ldc, bool accumulate,
                       void* workspace, int64_t workspace_bytes, int cus, hipStream_t s);
int64_t mx4_product_workspace(int64_t M, int64_t N, int64_t K, int cus);
int launch_mx4_row_product(const void* x, int32_t xtype, int64_t M, int64_t ldx, const MxView& w, void* y,
                           int32_t ytype, int64_t ldy, int cus, hipStream_t s);

}  // namespace halp

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

// |x| 2^(127 - s) = t in [0, 6] to a code.  The step is 1/2, 1 or 2 for t below 2, 4 and 6.
__device__ __forceinline__ uint32_t mx_round_nearest(float t) {
  const int k = t >= 4.f ? 2 : (t >= 2.f ? 1 : 0);
  return (uint32_t)__builtin_rintf(ldexpf(t, 1 - k)) + 2u * k;  // half way: the even multiple is the even code
}

// the same, up where the fraction of t / step is at least (511 - 2 r) / 512, r in [0, 256): the
// comparison is one of integers, since only whole 512ths of the fraction matter
__device__ __forceinline__ uint32_t mx_round_stochastic(float t, uint32_t r) {
  const uint32_t z = (uint32_t)(t * 1024.f);
  const uint32_t k = z >= 4096u ? 2u : (z >= 2048u ? 1u : 0u);
  return (((z >> k) + 2u * r + 1u) >> 9) + 2u * k;
}

// value of a code without its scale
__device__ __forceinline__ float mx_code_value(uint32_t c) {
  const uint32_t m = c & 7u;
  // 0 and .5 by hand, the others: exponent m / 2 - 1, mantissa bit m % 2
  const uint32_t bits = m < 2u ? (m ? 0x3F000000u : 0u) : ((m >> 1) + 126u) << 23 | (m & 1u) << 22;
  return __builtin_bit_cast(float, bits | (c & 8u) << 28);
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
                        const MxView* qt, int32_t rounding, uint64_t seed, uint32_t epoch, hipStream_t s);
int launch_mx4_dequantize(const MxView& q, void* out, int32_t type, int64_t ldo, hipStream_t s);
int launch_mx4_product(const MxView& a, const MxView& b, void* c, int32_t type, int64_t ldc, bool accumulate,
                       void* workspace, int64_t workspace_bytes, int cus, hipStream_t s);
int64_t mx4_product_workspace(int64_t M, int64_t N, int64_t K, int cus);
int launch_mx4_row_product(const void* x, int32_t xtype, int64_t M, int64_t ldx, const MxView& w, void* y,
                           int32_t ytype, int64_t ldy, hipStream_t s);

}  // namespace halp

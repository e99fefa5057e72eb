// Products of MX4 matrices on the matrix cores: c = a b^T (+ c).
#include "halp_internal.hpp"
#include "mx4.hpp"

namespace halp {
namespace {

struct ProductArgs {
  MxView a, b;
  void* c;
  int64_t ldc;
  int accumulate;
};

// v_mfma_scale_f32_16x16x128_f8f6f4, both operands in 4 bits: lane l holds row l % 16 and the block of 32
// values l / 16 of a group of 128, with that block's scale in byte 0; the result's lane l holds
// column l % 16 of rows 4 (l / 16) .. + 3.
__device__ __forceinline__ v4f32 mfma4(uint4 a, uint4 b, v4f32 c, uint32_t sa, uint32_t sb) {
  const v8i32 x{(int)a.x, (int)a.y, (int)a.z, (int)a.w}, y{(int)b.x, (int)b.y, (int)b.z, (int)b.w};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)sa, 0, (int)sb);
}

// One wave per 16 x 16 piece of c, operands straight from memory.  Rows past the end repeat the last one.
template <typename T>
__global__ __launch_bounds__(64) void product_tiles(ProductArgs a) {
  const int lane = threadIdx.x, r = lane % 16, q = lane / 16;
  const int64_t tn = (a.b.rows + 15) / 16, m0 = blockIdx.x / tn * 16, n0 = blockIdx.x % tn * 16;
  const int64_t m = min(m0 + r, a.a.rows - 1), n = min(n0 + r, a.b.rows - 1);
  const uint8_t *ca = a.a.codes + m * a.a.ldc + q * 16, *cb = a.b.codes + n * a.b.ldc + q * 16;
  const uint8_t *sa = a.a.scales + m * a.a.lds + q, *sb = a.b.scales + n * a.b.lds + q;
  v4f32 acc{};
  for (int64_t g = 0; g < mx_groups(a.a.cols); ++g)
    acc = mfma4(*reinterpret_cast<const uint4*>(ca + 64 * g), *reinterpret_cast<const uint4*>(cb + 64 * g), acc,
                sa[4 * g], sb[4 * g]);
  if (n0 + r >= a.b.rows) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = m0 + 4 * q + i;
    if (row >= a.a.rows) break;
    T* c = static_cast<T*>(a.c) + row * a.ldc + n0 + r;
    *c = (T)(a.accumulate ? to_f32(*c) + acc[i] : acc[i]);
  }
}

struct RowArgs {
  const void* x;
  int64_t M, ldx;
  MxView w;
  void* y;
  int64_t ldy;
};

// One wave per 16 rows of w; a lane quantizes the block of x that it multiplies.
template <typename X, typename Y>
__global__ __launch_bounds__(64) void row_product(RowArgs a) {
  const int lane = threadIdx.x, r = lane % 16, q = lane / 16;
  const int64_t n0 = blockIdx.x * 16ll, n = min(n0 + r, a.w.rows - 1);
  const X* x = static_cast<const X*>(a.x) + min((int64_t)r, a.M - 1) * a.ldx;
  const uint8_t *cb = a.w.codes + n * a.w.ldc + q * 16, *sb = a.w.scales + n * a.w.lds + q;
  v4f32 acc{};
  for (int64_t g = 0; g < mx_groups(a.w.cols); ++g) {
    const int64_t k0 = g * kMxGroup + q * kMxBlock;
    float v[kMxBlock];
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < kMxBlock; ++e) {
      v[e] = k0 + e < a.w.cols ? to_f32(x[k0 + e]) : 0.f;
      most = max(most, __builtin_bit_cast(uint32_t, v[e]) & 0x7FFFFFFFu);
    }
    const uint32_t s = mx_scale(most);
    const float inv = mx_inverse(s);
    uint32_t out[4] = {};
#pragma unroll
    for (int e = 0; e < kMxBlock; ++e) {
      const uint32_t bits = __builtin_bit_cast(uint32_t, v[e]);
      const uint32_t c = mx_round_nearest(__builtin_bit_cast(float, bits & 0x7FFFFFFFu) * inv) | (bits >> 31) << 3;
      out[e / 8] |= (s == 255u ? 0u : c) << (4 * (e % 8));
    }
    acc = mfma4(uint4{out[0], out[1], out[2], out[3]}, *reinterpret_cast<const uint4*>(cb + 64 * g), acc, s, sb[4 * g]);
  }
  if (n0 + r >= a.w.rows) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = 4 * q + i;
    if (row < a.M) static_cast<Y*>(a.y)[row * a.ldy + n0 + r] = (Y)acc[i];
  }
}

}  // namespace

int64_t mx4_product_workspace(int64_t, int64_t, int64_t, int) { return 0; }

int launch_mx4_product(const MxView& a, const MxView& b, void* c, int32_t type, int64_t ldc, bool accumulate, void*,
                       int64_t, hipStream_t s) {
  const int64_t tiles = (a.rows + 15) / 16 * ((b.rows + 15) / 16);
  if (tiles >= int64_t(1) << 31) return HALP_ERR_UNSUPPORTED;
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(product_tiles<T>, dim3((unsigned)tiles), dim3(64), 0, s, ProductArgs{a, b, c, ldc, accumulate});
    return hip_ok(hipGetLastError());
  });
}

int launch_mx4_row_product(const void* x, int32_t xtype, int64_t M, int64_t ldx, const MxView& w, void* y,
                           int32_t ytype, int64_t ldy, hipStream_t s) {
  return with_type(xtype, [&](auto xt) {
    return with_type(ytype, [&](auto yt) {
      using X = decltype(xt);
      using Y = decltype(yt);
      hipLaunchKernelGGL((row_product<X, Y>), dim3((unsigned)((w.rows + 15) / 16)), dim3(64), 0, s,
                         RowArgs{x, M, ldx, w, y, ldy});
      return hip_ok(hipGetLastError());
    });
  });
}

}  // namespace halp

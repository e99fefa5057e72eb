// Matrices into MX4, along their rows and along their columns, and back.
#include "halp_internal.hpp"
#include "mx4.hpp"

namespace halp {
namespace {

struct QuantArgs {
  const void* x;
  int64_t rows, cols, ldx;
  MxView q;  // the form that is written
  uint64_t seed;
  uint32_t epoch;
};

// One thread per block of the form (row i, block j of 32 places): its values lie in a row of x, or,
// for the transposed form, in a column.
template <typename T, bool COLS, bool RANDOM>
__global__ __launch_bounds__(256) void quantize_blocks(QuantArgs a) {
  const int64_t per = 4 * mx_groups(a.q.cols), total = a.q.rows * per;
  for (int64_t b = blockIdx.x * 256ll + threadIdx.x; b < total; b += gridDim.x * 256ll) {
    const int64_t i = COLS ? b % a.q.rows : b / per, j = COLS ? b / a.q.rows : b % per;
    const T* x = static_cast<const T*>(a.x) + (COLS ? j * kMxBlock * a.ldx + i : i * a.ldx + j * kMxBlock);
    const int64_t left = a.q.cols - j * kMxBlock;
    float v[kMxBlock];
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < kMxBlock; ++e) {
      v[e] = e < left ? to_f32(x[COLS ? e * a.ldx : e]) : 0.f;
      most = max(most, __builtin_bit_cast(uint32_t, v[e]) & 0x7FFFFFFFu);
    }
    const uint32_t s = mx_scale(most);
    const float inv = mx_inverse(s);
    uint32_t out[4] = {};
    const int64_t per16 = (a.q.cols + 15) / 16;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      U4 r{};
      if (RANDOM) r = stream_block(a.seed, COLS ? kMx4Cols : kMx4Rows, a.epoch, (uint64_t)(i * per16 + 2 * j + h));
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t bits = __builtin_bit_cast(uint32_t, v[16 * h + e]);
        const float t = __builtin_bit_cast(float, bits & 0x7FFFFFFFu) * inv;
        const uint32_t c = RANDOM ? mx_round_stochastic(t, pick(r, e / 4) >> (8 * (e % 4)) & 255u) : mx_round_nearest(t);
        out[2 * h + e / 8] |= (s == 255u ? 0u : c | (bits >> 31) << 3) << (4 * (e % 8));
      }
    }
    *reinterpret_cast<uint4*>(a.q.codes + i * a.q.ldc + j * 16) = uint4{out[0], out[1], out[2], out[3]};
    a.q.scales[i * a.q.lds + j] = (uint8_t)s;
  }
}

struct ReadArgs {
  MxView q;
  void* out;
  int64_t ldo;
};

// eight values (four bytes of codes) per thread
template <typename T>
__global__ __launch_bounds__(256) void dequantize(ReadArgs a) {
  const int64_t per = (a.q.cols + 7) / 8, total = a.q.rows * per;
  for (int64_t b = blockIdx.x * 256ll + threadIdx.x; b < total; b += gridDim.x * 256ll) {
    const int64_t i = b / per, j = b % per;
    const uint32_t c = *reinterpret_cast<const uint32_t*>(a.q.codes + i * a.q.ldc + j * 4);
    const float s = mx_scale_value(a.q.scales[i * a.q.lds + j / 4]);
    T* out = static_cast<T*>(a.out) + i * a.ldo + j * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (j * 8 + e < a.q.cols) out[e] = (T)(mx_code_value(c >> (4 * e)) * s);
  }
}

unsigned blocks_for(int64_t threads) {
  const int64_t n = (threads + 255) / 256;
  return (unsigned)(n < 65536 ? n : 65536);
}

}  // namespace

int launch_mx4_quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ldx, const MxView* q,
                        const MxView* qt, int32_t rounding, uint64_t seed, uint32_t epoch, hipStream_t s) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    for (int form = 0; form < 2; ++form) {
      const MxView* v = form ? qt : q;
      if (!v || v->rows == 0 || v->cols == 0) continue;
      const QuantArgs a{x, rows, cols, ldx, *v, seed, epoch};
      const dim3 grid(blocks_for(v->rows * 4 * mx_groups(v->cols)));
      const bool random = rounding == HALP_ROUND_STOCHASTIC;
      if (form && random) hipLaunchKernelGGL((quantize_blocks<T, true, true>), grid, dim3(256), 0, s, a);
      else if (form) hipLaunchKernelGGL((quantize_blocks<T, true, false>), grid, dim3(256), 0, s, a);
      else if (random) hipLaunchKernelGGL((quantize_blocks<T, false, true>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((quantize_blocks<T, false, false>), grid, dim3(256), 0, s, a);
    }
    return hip_ok(hipGetLastError());
  });
}

int launch_mx4_dequantize(const MxView& q, void* out, int32_t type, int64_t ldo, hipStream_t s) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(dequantize<T>, dim3(blocks_for(q.rows * ((q.cols + 7) / 8))), dim3(256), 0, s, ReadArgs{q, out, ldo});
    return hip_ok(hipGetLastError());
  });
}

}  // namespace halp

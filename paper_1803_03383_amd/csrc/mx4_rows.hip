// Products of a few rows with an MX4 matrix: y = Q(x) w^T, the rows quantized on the way.
//
// Bound by trips to memory, one after another.  A workgroup quantizes the rows into LDS and then takes units of w, one
// after another: 16 rows for each `split` of its waves, which share K between them and join their sums in LDS in the order of
// the waves.  A wave reads w in chunks of four groups (512 values) of 16 rows, across the units' borders.  Its first two are asked for
// before the rows, and each further one before the products of the chunk two before it; but as this is compiled a
// chunk has arrived before the next load is asked for (its word of scales is masked as soon as it is there, and chunks
// change registers), so that what is on the way at a time is one chunk a wave: 13 rows times 11000 x 5000 take 12 us, 29 MB of w
// at the rate of a copy 6.  Within a chunk lane quarter q takes the four blocks of group q: its codes are 64 bytes in a row,
// its four scales one word, and v_mfma_scale_f32_16x16x128_f8f6f4 multiplies block j of the four groups.
#include "halp_internal.hpp"
#include "mx4.hpp"

namespace halp {
namespace {

constexpr int kWaves = 16;  // of a workgroup at most
constexpr int kMostLds = 160 * 1024;

// LDS bytes of a quantized row of x, whole chunks: codes and scales, each with what keeps 16 rows off each other's banks
__host__ __device__ inline int64_t code_row(int64_t chunks) { return 256 * chunks + 16; }
__host__ __device__ inline int64_t scale_row(int64_t chunks) { return 16 * chunks + 4; }

// sums of two units: one is read while the next is written
__host__ __device__ inline int sum_bytes(int waves) { return 2 * waves * 64 * (int)sizeof(v4f32); }

static_assert(kMostLds - 2 * kWaves * 64 * 16 >= (256 + 16) * (kMxRowMost / 512) + 20, "a row and the sums fit");

struct RowArgs {
  const void* x;
  int64_t M, ldx;
  MxView w;
  void* y;
  int64_t ldy;
  int split, tiles;  // waves that share 16 rows; such tiles of a workgroup's unit
};

// Lane l holds row l % 16 and block l / 16 of four of both operands, with that block's scale in byte SEL; the result's
// lane l holds column l % 16 (a row of y) and rows 4 (l / 16) .. + 3 (rows of x).
template <int SEL>
__device__ __forceinline__ v4f32 mfma4(uint4 x, uint4 y, v4f32 c, uint32_t sx, uint32_t sy) {
  const v4i32 xv = __builtin_bit_cast(v4i32, x), yv = __builtin_bit_cast(v4i32, y);
  const v8i32 p = __builtin_shufflevector(xv, xv, 0, 1, 2, 3, -1, -1, -1, -1), q = __builtin_shufflevector(yv, yv, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, q, c, 4, 4, SEL, (int)sx, SEL, (int)sy);
}

struct Chunk {
  uint4 w[4];
  uint32_t scales;
};

template <typename X, typename Y>
__global__ __launch_bounds__(64 * kWaves) void row_product(RowArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, q = lane / 16;
  const int groups = (int)mx_groups(a.w.cols), chunks = (groups + 3) / 4;
  const int part = wave % a.split, own = wave / a.split, tiles = a.tiles, waves = a.split * tiles;
  const int c0 = chunks * part / a.split, c1 = chunks * (part + 1) / a.split;
  const int64_t units = (a.w.rows + 16 * tiles - 1) / (16 * tiles);
  v4f32* sums = reinterpret_cast<v4f32*>(lds);
  uint8_t *codes = lds + sum_bytes(waves), *scales = codes + a.M * code_row(chunks);

  // the chunk c of the unit's rows; rows past the end repeat the last one, a group past the last has no scale
  const auto load = [&](int64_t unit, int c) {
    const int64_t n = min((unit * tiles + own) * 16 + r, a.w.rows - 1);
    const int g = min(4 * c + q, groups - 1);
    const uint8_t* at = a.w.codes + n * a.w.ldc + 64 * (int64_t)g;
    Chunk k;
#pragma unroll
    for (int j = 0; j < 4; ++j) k.w[j] = *reinterpret_cast<const uint4*>(at + 16 * j);
    const uint32_t s = *reinterpret_cast<const uint32_t*>(a.w.scales + n * a.w.lds + 4 * (int64_t)g);
    k.scales = 4 * c + q < groups ? s : 0;
    return k;
  };
  int64_t next_unit = blockIdx.x;
  int next_c = c0;
  const auto load_next = [&] {  // in the order in which they are multiplied
    Chunk k{};
    if (next_unit < units && c0 < c1) {
      k = load(next_unit, next_c);
      if (++next_c == c1) next_c = c0, next_unit += gridDim.x;
    }
    return k;
  };
  Chunk first = load_next(), second = load_next();

  // 16 bytes of x per lane, four or eight lanes to a block, several rows under way; what lies behind the last column is
  // zero
  constexpr int kV = 16 / sizeof(X), kLanes = kMxBlock / kV, kAhead = 4;
  const int pieces = 512 / kV * chunks, rows = (int)a.M;  // pieces: a multiple of 64, all lanes of a wave or none
  for (int p = threadIdx.x; p < pieces; p += 64 * waves) {
    const int64_t left = a.w.cols - kV * (int64_t)p;
    const X* x = static_cast<const X*>(a.x) + kV * (int64_t)p;
    const auto put = [&](int m, uint4 v) {
      const uint32_t s = mx_scale(mx_max_bits<X>(mx_max_of_lanes<kLanes>(mx_max16<X>(v)))), c = mx_codes16<X>(v, s);
      if constexpr (sizeof(X) == 4) *reinterpret_cast<uint16_t*>(codes + m * code_row(chunks) + 2 * p) = (uint16_t)c;
      else *reinterpret_cast<uint32_t*>(codes + m * code_row(chunks) + 4 * p) = c;
      if (p % kLanes == 0) scales[m * scale_row(chunks) + p / kLanes] = (uint8_t)s;
    };
    int m = 0;
    if (__all(left >= kV))
      for (; m + kAhead <= rows; m += kAhead) {
        uint4 v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u] = mx_load16(x + (m + u) * a.ldx, kV);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) put(m + u, v[u]);
      }
    // The wave in which the rows end: lanes beyond read the rows' last 16 bytes and move them to their place, with zeros
    // behind, several rows under way here too (value by value, row after row, 13 rows of 5000 took 1.4 us longer).
    else if (a.w.cols >= kV) {
      const int bytes = (int)(kV - min(max(left, (int64_t)0), (int64_t)kV)) * (int)sizeof(X);
      const X* from = static_cast<const X*>(a.x) + min(kV * (int64_t)p, a.w.cols - kV);
      for (; m + kAhead <= rows; m += kAhead) {
        uint4 v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u] = mx_load16(from + (m + u) * a.ldx, kV);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          uint4 w = v[u];
          if (sizeof(X) == 2 && bytes & 2)
            w = uint4{__builtin_amdgcn_alignbyte(w.y, w.x, 2), __builtin_amdgcn_alignbyte(w.z, w.y, 2), __builtin_amdgcn_alignbyte(w.w, w.z, 2), w.w >> 16};
          if (bytes & 4) w = uint4{w.y, w.z, w.w, 0};
          if (bytes & 8) w = uint4{w.z, w.w, 0, 0};
          if (bytes & 16) w = uint4{};
          put(m + u, w);
        }
      }
    }
#pragma unroll 1
    for (; m < rows; ++m) put(m, mx_load16(x + m * a.ldx, left));
  }
  __syncthreads();

  const int m = min(r, (int)a.M - 1);
  const uint8_t *xc = codes + m * code_row(chunks) + 64 * q, *xs = scales + m * scale_row(chunks) + 4 * q;
  int parity = 0;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x, parity ^= 1) {
    v4f32 acc{};
    for (int c = c0; c < c1; ++c) {
      const Chunk k = first;
      first = second;
      second = load_next();
      const uint4* x = reinterpret_cast<const uint4*>(xc + 256 * c);
      const uint32_t s = *reinterpret_cast<const uint32_t*>(xs + 16 * c);
      acc = mfma4<0>(k.w[0], x[0], acc, k.scales, s);
      acc = mfma4<1>(k.w[1], x[1], acc, k.scales, s);
      acc = mfma4<2>(k.w[2], x[2], acc, k.scales, s);
      acc = mfma4<3>(k.w[3], x[3], acc, k.scales, s);
    }
    if (a.split > 1) {
      v4f32* to = sums + parity * waves * 64;
      to[wave * 64 + lane] = acc;
      // the sums only: nothing in memory is waited for
      lds_barrier();
      if (part) continue;
      for (int k = 1; k < a.split; ++k) acc += to[(wave + k) * 64 + lane];
    }
    const int64_t n = (unit * tiles + own) * 16 + 4 * q;
    if (r < a.M) {
      Y* y = static_cast<Y*>(a.y) + r * a.ldy + n;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < a.w.rows) y[e] = (Y)acc[e];
    }
  }
}

}  // namespace

int launch_mx4_row_product(const void* x, int32_t xtype, int64_t M, int64_t ldx, const MxView& w, void* y,
                           int32_t ytype, int64_t ldy, int cus, hipStream_t s) {
  const int64_t chunks = (mx_groups(w.cols) + 3) / 4, row = code_row(chunks) + scale_row(chunks);
  // How K is shared: `turn` chunks per wave and unit, with the fewest chunks one after another over all of a CU's units,
  // half a chunk counted for a unit's own.  One row times 11000 x 5000 (688 tiles of ten chunks): 10.0 us with a
  // chunk a wave and unit (three units to a CU), 8.8 with two (one unit of 15 waves).
  const int64_t all = (w.rows + 15) / 16;
  int split = 1, tiles = 1;
  double least = 1e300;
  for (int64_t turn = (chunks + kWaves - 1) / kWaves; chunks && turn <= chunks; ++turn) {
    const int64_t parts = (chunks + turn - 1) / turn, fit = kWaves / parts, per_cu = (all + cus - 1) / cus;
    const int64_t t = per_cu < fit ? per_cu : fit, units = (all + t - 1) / t;
    const double length = (double)((units + cus - 1) / cus) * (turn + 0.5);
    if (length < least) least = length, split = (int)parts, tiles = (int)t;
  }
  const int waves = split * tiles;
  const int64_t units = (all + tiles - 1) / tiles, most = (kMostLds - sum_bytes(waves)) / row;
  return with_type(xtype, [&](auto xt) {
    return with_type(ytype, [&](auto yt) {
      using X = decltype(xt);
      using Y = decltype(yt);
      for (int64_t m = 0; m < M; m += most) {
        // LDS holds `most` rows of x: each as many take a launch
        const int64_t rows = M - m < most ? M - m : most, lds = sum_bytes(waves) + rows * row;
        const int64_t a_cu = kMostLds / lds < kWaves / waves ? kMostLds / lds : kWaves / waves, held = cus * a_cu;
        if (hip_fail(hipFuncSetAttribute(reinterpret_cast<const void*>(row_product<X, Y>),
                                         hipFuncAttributeMaxDynamicSharedMemorySize, kMostLds), "hipFuncSetAttribute"))
          return (int)HALP_ERR_HIP;
        hipLaunchKernelGGL((row_product<X, Y>), dim3((unsigned)(units < held ? units : held)), dim3(64 * waves), (size_t)lds, s,
                           RowArgs{static_cast<const X*>(x) + m * ldx, rows, ldx, w, static_cast<Y*>(y) + m * ldy, ldy, split, tiles});
      }
      return hip_ok(hipGetLastError());
    });
  });
}

}  // namespace halp

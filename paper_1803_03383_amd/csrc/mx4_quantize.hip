// Matrices into MX4, along their rows and along their columns, and back.
//
// Bound by memory: x is read once for both forms.  A wave holds a tile of R rows and 1 KB of each in registers, 16
// bytes of a row per lane (eight where tiles are few).  A block of a row then lies in four or eight adjacent
// lanes, a block of a column in one lane (R = 32), so that no values move between waves; four waves take the four blocks of
// a stored group of the transposed form, and their codes meet in LDS to leave 64 bytes at a time.
#include <utility>

#include "halp_internal.hpp"
#include "mx4.hpp"

namespace halp {
namespace {

struct QuantArgs {
  const void* x;
  int64_t rows, cols, ldx;
  MxView q, qt;
  uint64_t seed;
  uint32_t epoch;
  int64_t across, tiles;  // tiles of a workgroup side by side, and in all
};

// ---- stochastic rounding -------------------------------------------------------------------------

// 2 r + 1 of byte e of two words of random bytes, as a pair of 16 bits
__device__ __forceinline__ v2u16 odd_pair(uint32_t w0, uint32_t w1, int e) {
  const uint32_t r = __builtin_amdgcn_perm(w1, w0, 0x0C000C00u | (4u + e) << 16 | e);
  return __builtin_bit_cast(v2u16, r << 1 | 0x00010001u);
}

// Codes of N = 4 or 8 values in order, from the random bytes of w0 (the first four) and w1.  The bits of 2^-14 t in fp16, t =
// |x| / scale <= 6 and cut towards zero, are 512 times the code of the grid's value below t and the fraction in 512ths
// of the step (below 1 it is subnormal, which is the grid's step of 1/2), so that the fraction's comparison with
// (511 - 2 r) / 512 is the carry of adding 2 r + 1: 5 instructions a value.
template <int N>
__device__ __forceinline__ uint32_t codes_random(const float* v, uint32_t s, uint32_t w0, uint32_t w1) {
  const int down = 113 - (int)s;
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < N / 2; ++e) {  // values e and e + N / 2 end up in the low and the high half
    const v2u16 t = __builtin_bit_cast(v2u16, __builtin_amdgcn_cvt_pkrtz(ldexpf(v[e], down), ldexpf(v[e + N / 2], down)));
    const uint32_t p = __builtin_bit_cast(uint32_t, (v2u16)(t + (N == 8 ? odd_pair(w0, w1, e) : odd_pair(w0, w0 >> 16, e))));
    c |= ((e < 3 ? p >> (9 - 4 * e) : p << 3) & 0x00070007u << 4 * e) | (p >> (12 - 4 * e) & 0x00080008u << 4 * e);
  }
  if (N == 4) c = (c | c >> 8) & 0xFFFFu;
  return s == 255u ? 0u : c;
}

// V values of a lane as words
template <typename T, int V>
struct Piece {
  static constexpr int kWords = V * sizeof(T) / 4;
  uint32_t w[kWords];
};

// value e of a lane's
template <typename T, int V>
__device__ __forceinline__ float value_at(const Piece<T, V>& v, int e) {
  const uint32_t w = v.w[e * (int)sizeof(T) / 4];
  if constexpr (std::is_same_v<T, float>) return __builtin_bit_cast(float, w);
  else if constexpr (std::is_same_v<T, __bf16>) return __builtin_bit_cast(float, e % 2 ? w & 0xFFFF0000u : w << 16);
  else return (float)__builtin_bit_cast(_Float16, (uint16_t)(e % 2 ? w >> 16 : w));
}

// the same as mx_max16 and mx_codes16 take it: zeros behind
template <typename T, int V>
__device__ __forceinline__ uint4 whole(const Piece<T, V>& v) {
  if constexpr (Piece<T, V>::kWords == 4) return uint4{v.w[0], v.w[1], v.w[2], v.w[3]};
  else return uint4{v.w[0], v.w[1], 0, 0};
}

template <typename T, int V>
__device__ __forceinline__ uint32_t row_codes(const Piece<T, V>& v, uint32_t s) {
  if constexpr (Piece<T, V>::kWords == 4) {
    return mx_codes16<T>(whole(v), s);
  } else {
    const float scale = __builtin_bit_cast(float, s << 23);
    const uint32_t c = mx_codes2<T, 1>(mx_codes2<T, 0>(0, v.w[0], 0, scale), v.w[1], 0, scale);
    return s == 255u ? 0u : c;
  }
}

template <typename T, int V>
__device__ __forceinline__ uint32_t row_codes_random(const Piece<T, V>& v, uint32_t s, uint32_t w0, uint32_t w1) {
  float f[V];
#pragma unroll
  for (int e = 0; e < V; ++e) f[e] = value_at(v, e);
  return codes_random<V>(f, s, w0, w1);
}

// ---- a wave's tile -------------------------------------------------------------------------------

template <typename T, int R, int V>
struct Tile {
  static constexpr int kV = V, kWords = Piece<T, V>::kWords;
  Piece<T, V> v[R];

  // rows row0 .. and columns col .. col + kV - 1 of x, zeros outside.  All loads are made, those of rows and columns
  // outside from others, so that nothing stands between them.  A lane's piece may reach past the last
  // column, into what lies between the rows or into the next one, and is masked; rows so near the end that such a piece
  // would reach past the last element are read value by value.
  __device__ __forceinline__ void load(const QuantArgs& a, int64_t row0, int64_t col) {
    const int64_t left = a.cols - col;  // of this lane's columns
    const bool ragged = __any(left < kV);
    const int64_t near = ragged ? a.rows - 1 - (kV - 2) / a.ldx : a.rows;  // the first such row
    typedef uint32_t __attribute__((ext_vector_type(kWords))) Words;
    typedef Words __attribute__((aligned(sizeof(T)))) Loose;
    Words w[R] = {};
    if (near > 0) {
      const T* x = static_cast<const T*>(a.x) + (left > 0 ? col : 0) + min(row0, near - 1) * a.ldx;
      const int more = __builtin_amdgcn_readfirstlane((int)min((int64_t)R, near - 1 - row0));  // rows after the first
#pragma unroll
      for (int i = 0; i < R; ++i) {
        w[i] = *reinterpret_cast<const Loose*>(x);
        x += i < more ? a.ldx : 0;
      }
    }
    const int rows = (int)max(min((int64_t)R, a.rows - row0), (int64_t)0);
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int k = 0; k < kWords; ++k) v[i].w[k] = w[i][k];
    if (rows < R) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (i >= rows) v[i] = Piece<T, V>{};
    }
    if (!ragged) return;
    constexpr int kPer = kV / kWords;  // values of a word
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      const uint32_t mask = left >= (k + 1) * kPer ? ~0u : left > k * kPer ? 0xFFFFu : 0u;
#pragma unroll
      for (int i = 0; i < R; ++i) v[i].w[k] &= mask;
    }
#pragma unroll 1
    for (int64_t row = max(row0, near); row < row0 + rows; ++row) {
      const T* from = static_cast<const T*>(a.x) + row * a.ldx + col;
      uint32_t u[kWords] = {};
#pragma unroll
      for (int e = 0; e < kV; ++e)
        if (e < left) {
          if constexpr (sizeof(T) == 4) u[e] = __builtin_bit_cast(uint32_t, from[e]);
          else u[e / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, from[e]) << (16 * (e % 2));
        }
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int k = 0; k < kWords; ++k)
          if (i == (int)(row - row0)) v[i].w[k] = u[k];
    }
  }
};

// Random words of this lane's V values of row i of x: w0, w1 (eight) or w0 (four) of the block of 16 columns that two
// or four adjacent lanes share.  Each of them makes the block of another row, and they exchange words: rows are taken
// two or four at a time.
template <int V>
struct RowRandom {
  static constexpr int kRows = 16 / V;  // rows at a time, and lanes that share a block
  uint32_t w[kRows][2];

  __device__ __forceinline__ void make(const QuantArgs& a, int64_t row0, int64_t col) {
    const int k = threadIdx.x % kRows;
    const U4 r = stream_block(a.seed, kMx4Rows, a.epoch, (uint64_t)((row0 + k) * ((a.cols + 15) / 16) + col / 16));
    if constexpr (kRows == 2) {
      const uint32_t p = dpp_quad_swap1(k ? r.x : r.z), q = dpp_quad_swap1(k ? r.y : r.w);
      w[0][0] = k ? p : r.x;
      w[0][1] = k ? q : r.y;
      w[1][0] = k ? r.z : p;
      w[1][1] = k ? r.w : q;
    } else {  // word k of each lane's block: a 4 x 4 transpose over the quad
      const bool odd = k & 1, high = k & 2;
      const uint32_t a0 = dpp_quad_swap1(odd ? r.x : r.y), a1 = dpp_quad_swap1(odd ? r.z : r.w);
      const uint32_t x0 = odd ? a0 : r.x, x1 = odd ? r.y : a0, x2 = odd ? a1 : r.z, x3 = odd ? r.w : a1;
      const uint32_t b0 = dpp_quad_swap2(high ? x0 : x2), b1 = dpp_quad_swap2(high ? x1 : x3);
      w[0][0] = high ? b0 : x0;
      w[1][0] = high ? b1 : x1;
      w[2][0] = high ? x2 : b0;
      w[3][0] = high ? x3 : b1;
    }
  }
};

// f(0), f(1), ... each with its index as a type: a loop of so many instructions is not unrolled, and its rows would not
// stay in registers
template <typename F, int... I>
__device__ __forceinline__ void for_each_index(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

template <typename T, bool ROWS, bool COLS, bool RANDOM, int R, int V>
__global__ __launch_bounds__(256, 2) void quantize_tiles(QuantArgs a) {
  constexpr int kV = V, kLanes = kMxBlock / kV;
  static_assert(!COLS || R == kMxBlock, "");
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  // The column blocks of the four waves meet here: blocks by value, lane and wave, the wave's place permuted so that lanes
  // write to all banks (8192 x 8192 fp16 both ways 63 us without it and 54 with).  Not where they are rounded
  // stochastically: the arithmetic bounds that.  In us without and with it, 8192 x 8192 fp16 both ways 79 / 83 and columns alone
  // 52 / 46, 8192 x 4096 bf16 38 / 39 and 22 / 22, 4095 x 5000 fp32 40.1 / 40.5 and 21.1 / 21.4.
  constexpr bool kMeet = COLS && !RANDOM;
  __shared__ uint4 out[kMeet ? 64 * kV * 4 : 1];
  __shared__ __align__(4) uint8_t out_scales[kMeet ? 64 * kV * 4 : 4];
  const int forms = gridDim.y == 1 ? 3 : 1 << blockIdx.y;  // of a tile, by this workgroup
  for (int64_t t = blockIdx.x; t < a.tiles; t += gridDim.x) {
    const int64_t row0 = (t / a.across * 4 + wave) * R, col = (t % a.across * 64 + lane) * kV;
    Tile<T, R, V> x;
    x.load(a, row0, col);
    if (ROWS && forms & 1) {
      const bool stored = col < mx_groups(a.cols) * kMxGroup;
      uint8_t *codes = a.q.codes + row0 * a.q.ldc + col / 2, *scales = a.q.scales + row0 * a.q.lds + col / kMxBlock;
      const int there = (int)min((int64_t)R, a.rows - row0), rows = stored ? there : 0;
      RowRandom<V> random;
      uint32_t kept = 0;  // of the lanes of a block, one keeps the scale of each row
      const auto one = [&](auto index) {
        constexpr int i = decltype(index)::value;
        if (RANDOM && i >= there) return;
        // opaque, or the compiler would convert the values of all rows first, past the registers
        if constexpr (COLS && RANDOM && std::is_same_v<T, _Float16>) {
#pragma unroll
          for (int k = 0; k < x.kWords; ++k) asm volatile("" : "+v"(x.v[i].w[k]));
        }
        if (RANDOM && i % random.kRows == 0) random.make(a, row0 + i, col);
        const uint32_t s = mx_scale(mx_max_bits<T>(mx_max_of_lanes<kLanes>(mx_max16<T>(whole(x.v[i])))));
        const uint32_t c = RANDOM ? row_codes_random(x.v[i], s, random.w[i % random.kRows][0], random.w[i % random.kRows][1])
                                  : row_codes(x.v[i], s);
        if (i < rows) {
          if constexpr (V == 4) *reinterpret_cast<uint16_t*>(codes + i * a.q.ldc) = (uint16_t)c;
          else *reinterpret_cast<uint32_t*>(codes + i * a.q.ldc) = c;
        }
        if (lane % kLanes == i % kLanes) kept = s;
        if (i % kLanes == kLanes - 1 || i == (RANDOM ? there : R) - 1) {
          const int row = i / kLanes * kLanes + lane % kLanes;
          if (row <= i && row < rows) scales[row * a.q.lds] = (uint8_t)kept;
        }
      };
      for_each_index(one, std::make_integer_sequence<int, R>{});
    }
    if (COLS && forms & 2) {
      const int64_t block = t / a.across * 4 + wave;  // of a row of the transposed form
      const int64_t per16 = (a.rows + 15) / 16;
#pragma unroll
      for (int e = 0; e < kV; ++e) {
        const int k = e * (int)sizeof(T) / 4, part = e * (int)sizeof(T) % 4;  // word and byte of value e
        // opaque, or what was made of the values for the rows would be kept for here
#pragma unroll
        for (int i = 0; i < R; ++i) asm volatile("" : "+v"(x.v[i].w[k]));
        const auto word = [&](int i) { return x.v[i].w[k]; };
        // two rows' values of the column as a pair, for 16-bit types
        const auto pair = [&](int i) { return __builtin_amdgcn_perm(word(i + 1), word(i), part ? 0x07060302u : 0x05040100u); };
        uint32_t most = 0;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int i = 0; i < R; ++i) most = max(most, word(i) & 0x7FFFFFFFu);
        } else {
          v2u16 m{};
#pragma unroll
          for (int i = 0; i < R; i += 2) m = __builtin_elementwise_max(m, __builtin_bit_cast(v2u16, pair(i) & 0x7FFF7FFFu));
          most = max((uint32_t)m.x, (uint32_t)m.y);
        }
        const uint32_t s = mx_scale(mx_max_bits<T>(most));
        uint32_t c[4];
        if constexpr (RANDOM) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            c[2 * h] = c[2 * h + 1] = 0;
            if (row0 + 16 * h >= a.rows) continue;
            const U4 r = stream_block(a.seed, kMx4Cols, a.epoch, (uint64_t)((col + e) * per16 + 2 * block + h));
            float f[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] = value_at(x.v[16 * h + i], e);
            c[2 * h] = codes_random<8>(f, s, r.x, r.y);
            c[2 * h + 1] = codes_random<8>(f + 8, s, r.z, r.w);
          }
        } else {
          const float scale = __builtin_bit_cast(float, s << 23);
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            uint32_t d = 0;
            if constexpr (sizeof(T) == 4) {
              d = mx_codes2<T, 0>(d, word(8 * g), word(8 * g + 1), scale);
              d = mx_codes2<T, 1>(d, word(8 * g + 2), word(8 * g + 3), scale);
              d = mx_codes2<T, 2>(d, word(8 * g + 4), word(8 * g + 5), scale);
              d = mx_codes2<T, 3>(d, word(8 * g + 6), word(8 * g + 7), scale);
            } else {
              d = mx_codes2<T, 0>(d, pair(8 * g), 0, scale);
              d = mx_codes2<T, 1>(d, pair(8 * g + 2), 0, scale);
              d = mx_codes2<T, 2>(d, pair(8 * g + 4), 0, scale);
              d = mx_codes2<T, 3>(d, pair(8 * g + 6), 0, scale);
            }
            c[g] = s == 255u ? 0u : d;
          }
        }
        if constexpr (kMeet) {
          out[(e * 64 + lane) * 4 + (wave ^ (lane / 4 % 4))] = uint4{c[0], c[1], c[2], c[3]};
          out_scales[(e * 64 + lane) * 4 + wave] = (uint8_t)s;
        } else if (col + e < a.cols) {
          *reinterpret_cast<uint4*>(a.qt.codes + (col + e) * a.qt.ldc + 16 * block) = uint4{c[0], c[1], c[2], c[3]};
          a.qt.scales[(col + e) * a.qt.lds + block] = (uint8_t)s;
        }
      }
      if constexpr (!kMeet) continue;
      __syncthreads();
      // the four waves' blocks of a column leave together, 64 bytes and a word of scales
      const int64_t col0 = t % a.across * 64 * kV, group = t / a.across;
#pragma unroll
      for (int i = threadIdx.x; i < 64 * kV * 4; i += 256) {
        const int n = i / 4, l = n / kV, e = n % kV;  // column n of the tile: value e of lane l
        if (col0 + n < a.cols)
          *reinterpret_cast<uint4*>(a.qt.codes + (col0 + n) * a.qt.ldc + 64 * group + 16 * (i % 4)) = out[(e * 64 + l) * 4 + (i % 4 ^ (l / 4 % 4))];
      }
#pragma unroll
      for (int n = threadIdx.x; n < 64 * kV; n += 256)
        if (col0 + n < a.cols)
          *reinterpret_cast<uint32_t*>(a.qt.scales + (col0 + n) * a.qt.lds + 4 * group) =
              *reinterpret_cast<const uint32_t*>(out_scales + (n % kV * 64 + n / kV) * 4);
      __syncthreads();
    }
  }
}

struct ReadArgs {
  MxView q;
  void* out;
  int64_t ldo, across, tiles;
};

// values of the two codes of byte SEL, scaled
template <int SEL>
__device__ __forceinline__ void read_two(uint32_t c, float scale, float* f) {
  const v2f32 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, SEL);
  f[0] = v.x * scale;
  f[1] = v.y * scale;
}

// Eight rows per wave, 16 bytes of each per lane.
template <typename T>
__global__ __launch_bounds__(256) void dequantize(ReadArgs a) {
  constexpr int kV = 16 / sizeof(T), R = 8;
  struct __attribute__((packed, aligned(sizeof(T)))) Piece { T v[kV]; };
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  for (int64_t t = blockIdx.x; t < a.tiles; t += gridDim.x) {
    const int64_t row0 = (t / a.across * 4 + wave) * R, col = (t % a.across * 64 + lane) * kV, left = a.q.cols - col;
    const uint8_t *codes = a.q.codes + row0 * a.q.ldc + col / 2, *scales = a.q.scales + row0 * a.q.lds + col / kMxBlock;
    T* out = static_cast<T*>(a.out) + row0 * a.ldo + col;
    const auto run = [&](auto all) {  // all: every lane has its values of every row
      const int rows = all ? R : left > 0 ? (int)min((int64_t)R, a.q.rows - row0) : 0;
      uint32_t c[R], s[R];
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (i < rows) {
          if constexpr (kV == 8) c[i] = *reinterpret_cast<const uint32_t*>(codes + i * a.q.ldc);
          else c[i] = *reinterpret_cast<const uint16_t*>(codes + i * a.q.ldc);
          s[i] = scales[i * a.q.lds];
        }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (i >= rows) break;
        const float scale = mx_scale_value(s[i]);
        float f[8];
        read_two<0>(c[i], scale, f);
        read_two<1>(c[i], scale, f + 2);
        if constexpr (kV == 8) {
          read_two<2>(c[i], scale, f + 4);
          read_two<3>(c[i], scale, f + 6);
        }
        Piece o;
#pragma unroll
        for (int e = 0; e < kV; ++e) o.v[e] = (T)f[e];
        if (all || left >= kV) {
          *reinterpret_cast<Piece*>(out + i * a.ldo) = o;
        } else {
#pragma unroll
          for (int e = 0; e < kV; ++e)
            if (e < left) out[i * a.ldo + e] = o.v[e];
        }
      }
    };
    if (row0 + R <= a.q.rows && __all(left >= kV)) run(std::true_type{});
    else run(std::false_type{});
  }
}

// a launch holds fewer than 2^32 threads: 256 for each of these workgroups
unsigned grid_of(int64_t tiles) { return (unsigned)(tiles < (1 << 22) ? tiles : 1 << 22); }

}  // namespace

int launch_mx4_quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ldx, const MxView* q,
                        const MxView* qt, int32_t rounding, uint64_t seed, uint32_t epoch, int cus, hipStream_t s) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    const auto by_width = [&](auto values) {  // of a lane
      constexpr int V = decltype(values)::value;
      constexpr int64_t kWidth = 64 * V;  // columns of a tile
      QuantArgs a{x, rows, cols, ldx, q ? *q : MxView{}, qt ? *qt : MxView{}, seed, epoch, 0, 0};
      // the padding is written too: of the columns where rows are quantized, of the rows where columns are
      a.across = ((q ? mx_groups(cols) * kMxGroup : cols) + kWidth - 1) / kWidth;
      const bool random = rounding == HALP_ROUND_STOCHASTIC;
      // Rows alone: one row a wave where there are so few that the waves count, else eight.
      const int height = qt ? 32 : rows <= 1024 ? 1 : 8;
      a.tiles = a.across * ((rows + 4 * height - 1) / (4 * height));
      // Both forms of a tile by one workgroup, so that x is read once; by two, side by side, where that leaves no CU without
      // one (300 x 4096 in bf16 8.3 us instead of 10.9, stochastically 15.0 instead of 22.0, with eight values a lane)
      const dim3 grid(grid_of(a.tiles), q && qt && a.tiles <= cus ? 2 : 1);
      const auto launch = [&](auto with_rows, auto with_cols, auto is_random, auto tall) {
        hipLaunchKernelGGL((quantize_tiles<T, decltype(with_rows)::value, decltype(with_cols)::value, decltype(is_random)::value,
                                           decltype(tall)::value, V>), grid, dim3(256), 0, s, a);
      };
      const std::true_type yes{};
      const std::false_type no{};
      const auto by_form = [&](auto is_random) {
        if (q && qt) launch(yes, yes, is_random, std::integral_constant<int, 32>{});
        else if (qt) launch(no, yes, is_random, std::integral_constant<int, 32>{});
        else if constexpr (V == 16 / sizeof(T)) {
          if (height == 8) launch(yes, no, is_random, std::integral_constant<int, 8>{});
          else launch(yes, no, is_random, std::integral_constant<int, 1>{});
        }
      };
      if (random) by_form(yes);
      else by_form(no);
      return hip_ok(hipGetLastError());
    };
    // Four values of 16 bits a lane instead of eight, twice as many tiles, where tiles are few.  In bf16, us with eight and
    // four: columns of 300 x 4096 7.4 / 5.6, 4096 x 4096 13.3 / 13.0, 8192 x 4096 22.9 / 23.2; both forms of 300 x 4096
    // 8.6 / 8.1 and 2000 x 4096 11.6 / 12.1, stochastically 15.0 / 12.9 and 17.9 / 17.0, of 3000 x 4096 23.0 / 27.7.
    if constexpr (sizeof(T) == 2) {
      const int64_t tiles = ((rows + 127) / 128) * ((cols + 511) / 512);
      if (qt && tiles <= (!q ? cus : rounding == HALP_ROUND_STOCHASTIC ? cus / 2 : cus / 4)) return by_width(std::integral_constant<int, 4>{});
    }
    return by_width(std::integral_constant<int, 16 / sizeof(T)>{});
  });
}

int launch_mx4_dequantize(const MxView& q, void* out, int32_t type, int64_t ldo, hipStream_t s) {
  return with_type(type, [&](auto t) {
    using T = decltype(t);
    constexpr int64_t kWidth = 64 * 16 / sizeof(T);
    const int64_t across = (q.cols + kWidth - 1) / kWidth, tiles = across * ((q.rows + 31) / 32);
    hipLaunchKernelGGL(dequantize<T>, dim3(grid_of(tiles)), dim3(256), 0, s,
                       ReadArgs{q, out, ldo, across, tiles});
    return hip_ok(hipGetLastError());
  });
}

}  // namespace halp

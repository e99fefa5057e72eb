// Products of MX4 matrices on the matrix cores: c = a b^T (+ c).
//
// A workgroup makes a tile of c.  Stages of 256 values of K (128 bytes of codes and 8 scales a row) of both
// operands go to LDS by global_load_lds, in two or three buffers; a wave reads fragments of 32 rows and multiplies
// them with v_mfma_scale_f32_32x32x64_f8f6f4 in 4 bits (the 16x16x128 form sustains 5.1 - 5.9
// PFLOP/s on random codes, this one 6.8, where the power limit holds it).  The order of K within a stage
// is free as long as both operands have the same: lane half h takes the four blocks of group h of a row,
// so that its scales of the stage are one word and the instruction picks the byte.  16-byte pieces of
// a row are permuted in LDS (piece p of row r lies at p ^ r / 2 % 8), so that the 16 rows that are read at once
// cover every bank once; the permutation is made on the source address.
#include "halp_internal.hpp"
#include "mx4.hpp"
#include "mx4_plan.hpp"

namespace halp {
namespace {

constexpr int kStage = 128;  // bytes of a row per stage: two groups of 128 values

struct ProductArgs {
  MxView a, b;
  void* c;
  int64_t ldc;
  int accumulate;
  int vec;         // c's rows can be written 16 bytes at a time
  int tiles_m, tiles_n;
  int cuts;        // parts of K; more than one: part z goes to rows z M and up of c
};

// Lane l holds row l % 32 and block l / 32 of two of both operands, with that block's scale in byte SEL; the result's
// lane l holds column l % 32 (a row of y) and rows 8 (i / 4) + 4 (l / 32) + i % 4 (rows of x), i = 0 .. 15.
template <int SEL>
__device__ __forceinline__ v16f32 mfma4(uint4 x, uint4 y, v16f32 c, uint32_t sx, uint32_t sy) {
  // 4-bit operands are the first four registers
  const v4i32 xv = __builtin_bit_cast(v4i32, x), yv = __builtin_bit_cast(v4i32, y);
  const v8i32 p = __builtin_shufflevector(xv, xv, 0, 1, 2, 3, -1, -1, -1, -1), q = __builtin_shufflevector(yv, yv, 0, 1, 2, 3, -1, -1, -1, -1);
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(p, q, c, 4, 4, SEL, (int)sx, SEL, (int)sy);
}

using LPtr = __attribute__((address_space(3))) void*;

// 64 times 16 bytes from base + off (a lane's own, 32 bits) to LDS at `to` (bytes, a multiple of 1024 past the wave's
// start) and up, lane after lane.  Issued by hand: the compiler takes the builtin for a store to all of LDS
// and would have every later LDS read wait for it.  Complete after s_waitcnt vmcnt(0).  on: ~0 or 0, all lanes or none, so that
// a load can be left out without a branch, which would part the products around it.  All lanes are active.  m0 holds `to`.
__device__ __forceinline__ void to_lds(const uint8_t* base, uint32_t off, uint32_t to, uint32_t on) {
  asm volatile("s_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1"
               ::"{m0}"(to), "v"(off), "s"(base), "s"(on));
}

// the same of 64 times 4 bytes, 256 in all
__device__ __forceinline__ void word_to_lds(const uint8_t* base, uint32_t off, uint32_t to, uint32_t on) {
  asm volatile("s_mov_b32 exec_lo, %3\n\ts_mov_b32 exec_hi, %3\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b64 exec, -1"
               ::"{m0}"(to), "v"(off), "s"(base), "s"(on));
}

// a pointer that is the same in every lane, in scalar registers
__device__ __forceinline__ const uint8_t* scalar(const uint8_t* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return reinterpret_cast<const uint8_t*>((uint64_t)hi << 32 | lo);
}

// The codes of ROWS rows of one operand for a tile: where a lane loads from.  In LDS they lie row after row.
template <int ROWS, int THREADS>
struct Codes {
  static constexpr int kLoads = ROWS * 8 / THREADS;  // per lane and stage
  static_assert(kLoads * THREADS == ROWS * 8, "");
  const uint8_t* base;
  uint32_t off[kLoads];

  __device__ __forceinline__ void init(const MxView& m, int64_t row0, int64_t stage0) {
    base = scalar(m.codes + row0 * m.ldc + stage0 * kStage);
    // rows past the end repeat the last one; 256 rows of less than 2^23 bytes are within 32 bits
    const uint32_t last = (uint32_t)min((int64_t)ROWS - 1, m.rows - 1 - row0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t p = i * THREADS + threadIdx.x, r = p / 8;
      off[i] = min(r, last) * (uint32_t)m.ldc + 16 * ((p ^ r / 2) & 7);
      asm volatile("" : "+v"(off[i]));  // one register: the compiler would keep the 64-bit multiply-add's two
    }
  }
  // load i of stage s to LDS address c.  half: the stage has one group only, which is read in place of the other.
  __device__ __forceinline__ void fetch(int i, int64_t s, bool half, uint32_t c, uint32_t on) const {
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), p = i * THREADS + threadIdx.x;
    to_lds(scalar(base + s * kStage), off[i] - (half ? 16 * ((p ^ (p / 16)) & 4) : 0), c + i * THREADS * 16 + wave * 1024, on);
  }
};

// The scales of both operands' rows, 16 bytes of a row at a time, two stages: a load takes about two cycles of the CU for each
// line of memory that it touches, and the 8 bytes of a stage alone took 0.24 us beside the codes' 0.41 in
// tiles of 128.  (Four stages at a time are no faster: their words meet on fewer banks, or more loads are left out, which
// take their time too.)  In LDS they lie row after row, a's first.
template <int BM, int BN, int THREADS>
struct Scales {
  static constexpr int kLoads = (BM + BN) / THREADS, kPair = (BM + BN) * 16;
  static_assert(kLoads * THREADS == BM + BN && BM % 64 == 0, "a wave's load is of one operand");
  const uint8_t *a, *b;
  uint32_t off[kLoads], begin, last;  // begin: of the first stage in a row; last: where the last 16 bytes of a row begin

  __device__ static __forceinline__ uint32_t row_at(const MxView& ma, const MxView& mb, int64_t m0, int64_t n0, int row) {
    return row < BM ? (uint32_t)min((int64_t)row, ma.rows - 1 - m0) * (uint32_t)ma.lds
                    : (uint32_t)min((int64_t)row - BM, mb.rows - 1 - n0) * (uint32_t)mb.lds;
  }
  __device__ __forceinline__ void init(const MxView& ma, const MxView& mb, int64_t m0, int64_t n0, int64_t groups, int first) {
    a = scalar(ma.scales + m0 * ma.lds);
    b = scalar(mb.scales + n0 * mb.lds);
    begin = 8 * first;
    last = groups < 4 ? ~0u / 2 : (uint32_t)(4 * groups - 16);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      off[i] = row_at(ma, mb, m0, n0, i * THREADS + threadIdx.x);
      asm volatile("" : "+v"(off[i]));
    }
  }
  // Load i of the stages s and s + 1 (s even) to LDS address k.  What would reach past the row is read from its last 16 bytes
  // instead: see moved().
  __device__ __forceinline__ void fetch(int i, int s, uint32_t k, uint32_t on) const {
    const uint32_t p = i * THREADS + __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * 64;
    to_lds(scalar(p < BM ? a : b), off[i] + min(begin + 8 * s, last), k + p * 16, on);
  }
  // The first two stages of rows with fewer than four groups, which have no 16 bytes: word by word, the last one in place
  // of those that are not there.
  __device__ __forceinline__ void fetch_words(const MxView& ma, const MxView& mb, int64_t m0, int64_t n0, int64_t groups, uint32_t k) const {
#pragma unroll 1
    for (int i = 0; i < 4 * kLoads; ++i) {
      const uint32_t p = i * THREADS + __builtin_amdgcn_readfirstlane(threadIdx.x / 64) * 64;
      const uint32_t word = min(4 * (threadIdx.x % 4), (uint32_t)(4 * groups - 4));
      word_to_lds(scalar(p < 4 * BM ? a : b), row_at(ma, mb, m0, n0, (i * THREADS + threadIdx.x) / 4) + word, k + p * 4, ~0u);
    }
  }
  // how far stage s lies behind its place, since its 16 bytes were read from before
  __device__ __forceinline__ uint32_t moved(int s) const {
    const uint32_t at = begin + 8 * (s & ~1);
    return at > last ? at - last : 0;
  }
};

// Tiles of WM FM x WN FN fragments, one wave FM x FN of them.  A stage is four steps (block j of each group) of FM x FN
// products.  A step's fragments are read during the step before; the barrier that a stage has arrived for
// stands one step before its first product, when all of the stage before has been read, so that the
// matrix cores do not wait for it.  D buffers: D - 1 stages are on their way or in use.  Scales come in pairs of
// stages, each asked for when the pair before it begins, into two buffers of their own.
template <typename T, int WM, int WN, int FM, int FN, int D>
__global__ __launch_bounds__(WM * WN * 64) void product_tiles(ProductArgs a) {
  constexpr int kThreads = WM * WN * 64, BM = WM * FM * 32, BN = WN * FN * 32;
  constexpr int kBuffer = (BM + BN) * kStage;
  using S = Scales<BM, BN, kThreads>;
  static_assert(D <= 3, "a pair of scales has arrived D - 1 stages after it was asked for, and is read after two");
  __shared__ __align__(16) uint8_t lds[2 * S::kPair + D * kBuffer];

  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane % 32, h = lane / 32;
  const int wm = wave / WN, wn = wave % WN;
  // workgroups go to the XCDs in turn: each XCD takes a run of the cuts' tiles, in bands of eight tile rows, so that it
  // reads its cuts of K only
  const int tiles = a.tiles_m * a.tiles_n, total = tiles * a.cuts, at = blockIdx.y * tiles + blockIdx.x, x = at % 8;
  const int item = x * (total / 8) + min(x, total % 8) + at / 8, cut = item / tiles, tile = item % tiles;
  const int band = tile / (8 * a.tiles_n), rest = tile % (8 * a.tiles_n), height = min(8, a.tiles_m - 8 * band);
  const int64_t m0 = (int64_t)(8 * band + rest % height) * BM, n0 = (int64_t)(rest / height) * BN;

  Codes<BM, kThreads> ca;
  Codes<BN, kThreads> cb;
  S sc;
  const int64_t groups = mx_groups(a.a.cols), all = (groups + 1) / 2;
  const int first = (int)(all * cut / a.cuts), stages = (int)(all * (cut + 1) / a.cuts) - first;
  const bool odd = (groups & 1) && cut == a.cuts - 1;  // the last stage has one group
  ca.init(a.a, m0, first);
  cb.init(a.b, n0, first);
  sc.init(a.a, a.b, m0, n0, groups, first);

  const uint32_t lds0 = (uint32_t)(uintptr_t)(LPtr)lds;
  // every stage asks for as many, left out or not, so that they can be counted
  constexpr int kLoads = ca.kLoads + cb.kLoads + sc.kLoads;
  const auto fetch = [&](int i, int s, int buffer, int pair) {  // load i: codes of stage s; scales of stages pair, pair + 1
    const uint32_t at = lds0 + 2 * S::kPair + buffer * kBuffer;
    const bool half = odd && s == stages - 1;
    const uint32_t on = __builtin_amdgcn_readfirstlane(s < stages ? ~0u : 0u);
    if (i < ca.kLoads) ca.fetch(i, s, half, at, on);
    else if (i < ca.kLoads + cb.kLoads) cb.fetch(i - ca.kLoads, s, half, at + BM * kStage, on);
    else if (i < kLoads)
      sc.fetch(i - ca.kLoads - cb.kLoads, pair, lds0 + pair / 2 % 2 * S::kPair, __builtin_amdgcn_readfirstlane(pair % 2 == 0 && pair < stages ? ~0u : 0u));
  };

  v16f32 acc[FM][FN] = {};
  uint4 fx[2][FM] = {}, fy[2][FN] = {};  // fragments by step
  uint32_t sx[FM] = {}, sy[FN] = {};

  // row m of the products of step j
  const auto products = [&](auto step, int m) {
    constexpr int j = decltype(step)::value;
#pragma unroll
    for (int n = 0; n < FN; ++n) acc[m][n] = mfma4<j>(fy[j % 2][n], fx[j % 2][m], acc[m][n], sy[n], sx[m]);
  };

  if (stages && groups < 4) sc.fetch_words(a.a, a.b, m0, n0, groups, lds0);
#pragma unroll
  for (int s = 0; s < D - 1; ++s)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) fetch(i, s, s, s == 0 && groups >= 4 ? 0 : 1);
  int buffer = 0, free = D - 1;  // of this stage; of the next one that is asked for
  for (int s = 0; s < stages; ++s) {
    // this stage has arrived (the loads of those behind it may be under way), and every wave has read the one before
    static_assert((D - 2) * kLoads < 64, "");
    if (D > 2 && s + D - 2 < stages) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((D - 2) * kLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const uint8_t* codes = lds + 2 * S::kPair + buffer * kBuffer;
    // Row m of the products of a step, with a part of the next step's reads and of the next stage's loads before it.
    // The order is held: the compiler would put the reads behind the products, where they are waited for.
    const auto part = [&](auto step, int j, int m) {  // j: the step that is read
      const int piece = (((4 * h + j) ^ r / 2) & 7) * 16;
#pragma unroll
      for (int n = m * FN / FM; n < (m + 1) * FN / FM; ++n)
        fy[j % 2][n] = *reinterpret_cast<const uint4*>(codes + BM * kStage + ((wn * FN + n) * 32 + r) * kStage + piece);
      fx[j % 2][m] = *reinterpret_cast<const uint4*>(codes + ((wm * FM + m) * 32 + r) * kStage + piece);
      constexpr int kPer = (kLoads + 3 * FM - 1) / (3 * FM);  // all in the first three steps
#pragma unroll
      for (int n = 0; n < kPer; ++n) fetch((j * FM + m) * kPer + n, s + D - 1, free, s + 2);
      __builtin_amdgcn_sched_barrier(0);
      products(step, m);
      __builtin_amdgcn_sched_barrier(0);
    };
    uint32_t nx[FM], ny[FN];
    const uint8_t* scales = lds + s / 2 % 2 * S::kPair + 8 * (s % 2) + 4 * h + sc.moved(s);
#pragma unroll
    for (int m = 0; m < FM; ++m) nx[m] = *reinterpret_cast<const uint32_t*>(scales + 16 * ((wm * FM + m) * 32 + r));
#pragma unroll
    for (int n = 0; n < FN; ++n) ny[n] = *reinterpret_cast<const uint32_t*>(scales + 16 * (BM + (wn * FN + n) * 32 + r));
#pragma unroll
    for (int m = 0; m < FM; ++m) part(std::integral_constant<int, 3>{}, 0, m);
    // The group that an odd row's last stage lacks gets scales of 0 on both sides, 2^-254 together: what was read in
    // its place adds nothing.
    const bool none = s == stages - 1 && odd && h;
#pragma unroll
    for (int m = 0; m < FM; ++m) sx[m] = none ? 0 : nx[m];
#pragma unroll
    for (int n = 0; n < FN; ++n) sy[n] = none ? 0 : ny[n];
#pragma unroll
    for (int m = 0; m < FM; ++m) part(std::integral_constant<int, 0>{}, 1, m);
#pragma unroll
    for (int m = 0; m < FM; ++m) part(std::integral_constant<int, 1>{}, 2, m);
#pragma unroll
    for (int m = 0; m < FM; ++m) part(std::integral_constant<int, 2>{}, 3, m);
    free = buffer;
    buffer = buffer == D - 1 ? 0 : buffer + 1;
  }
#pragma unroll
  for (int m = 0; m < FM; ++m) products(std::integral_constant<int, 3>{}, m);

  // 32 rows at a time through LDS (each wave its own part), so that rows leave in 16-byte pieces, whole lines
  // together: straight from the accumulators a line would be written 8 bytes at a time.  The rows lie where the last stage's
  // codes were: every wave must have its fragments of them, not only have asked for them.  The last products may stand
  // behind the barrier, and the compiler waits for their fragments no earlier, so the barrier does.
  constexpr int kPer = 16 / sizeof(T), kRow = FN * 32 + kPer, kPieces = FN * 32 / kPer;  // elements, pieces a row
  static_assert(WM * WN * 32 * kRow * sizeof(T) <= sizeof lds, "");
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  T* own = reinterpret_cast<T*>(lds) + wave * 32 * kRow;
#pragma unroll
  for (int m = 0; m < FM; ++m) {
    struct alignas(4 * sizeof(T)) Four { T v[4]; };
    struct alignas(16) Piece { T v[kPer]; };
#pragma unroll
    for (int n = 0; n < FN; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        Four o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o.v[e] = (T)acc[m][n][4 * g + e];
        *reinterpret_cast<Four*>(own + r * kRow + n * 32 + 8 * g + 4 * h) = o;
      }
#pragma unroll
    for (int p = lane; p < 32 * kPieces; p += 64) {
      Piece o = *reinterpret_cast<const Piece*>(own + p / kPieces * kRow + p % kPieces * kPer);
      const int64_t row = m0 + (wm * FM + m) * 32 + p / kPieces, col = n0 + wn * FN * 32 + p % kPieces * kPer;
      if (row >= a.a.rows) continue;
      T* c = static_cast<T*>(a.c) + (cut * a.a.rows + row) * a.ldc + col;
      if (a.vec && col + kPer <= a.b.rows) {
        if (a.accumulate) {
          const Piece before = *reinterpret_cast<const Piece*>(c);
#pragma unroll
          for (int e = 0; e < kPer; ++e) o.v[e] = (T)(to_f32(before.v[e]) + to_f32(o.v[e]));
        }
        *reinterpret_cast<Piece*>(c) = o;
      } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          if (col + e < a.b.rows) c[e] = (T)(a.accumulate ? to_f32(c[e]) + to_f32(o.v[e]) : to_f32(o.v[e]));
      }
    }
  }
}

struct JoinArgs {
  const float* parts;  // [cuts][M][ldp]
  void* c;
  int64_t M, N, ldp, ldc;
  int cuts, accumulate;
};

// c = the parts' sum in their order (+ c): four columns per thread
template <typename T>
__global__ __launch_bounds__(256) void join_cuts(JoinArgs a) {
  const int64_t per = a.ldp / 4;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < a.M * per; i += gridDim.x * 256ll) {
    const int64_t row = i / per, col = i % per * 4;
    v4f32 sum = *reinterpret_cast<const v4f32*>(a.parts + row * a.ldp + col);
    for (int z = 1; z < a.cuts; ++z) sum += *reinterpret_cast<const v4f32*>(a.parts + (z * a.M + row) * a.ldp + col);
    T* c = static_cast<T*>(a.c) + row * a.ldc + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < a.N) c[e] = (T)(a.accumulate ? to_f32(c[e]) + sum[e] : sum[e]);
  }
}

}  // namespace

int64_t mx4_product_workspace(int64_t M, int64_t N, int64_t K, int cus) {
  return plan_workspace(M, N, product_plan(M, N, K, cus, kMostCuts));
}

int launch_mx4_product(const MxView& a, const MxView& b, void* c, int32_t type, int64_t ldc, bool accumulate,
                       void* workspace, int64_t workspace_bytes, int cus, hipStream_t s) {
  const ProductPlan p = product_plan_within(a.rows, b.rows, a.cols, cus, workspace_bytes);
  const int64_t t = p.tile, tm = (a.rows + t - 1) / t, tn = (b.rows + t - 1) / t;
  const auto tiles = [&](auto kind, void* out, int64_t ld, bool add) {
    using T = decltype(kind);
    const int vec = ld * sizeof(T) % 16 == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
    const ProductArgs args{a, b, out, ld, add, vec, (int)tm, (int)tn, p.cuts};
    const dim3 grid((unsigned)(tm * tn), (unsigned)p.cuts);
    if (p.tile == 256) hipLaunchKernelGGL((product_tiles<T, 2, 4, 4, 2, 2>), grid, dim3(512), 0, s, args);
    // 128: two buffers let two workgroups share a CU; where each has one to itself, a third hides the loads' latency
    // (1000 x 784 x 60000 in four parts 63 and 50 us, 4096 x 4096 x 4096 49 and 60)
    else if (p.tile == 128 && tm * tn * p.cuts > cus) hipLaunchKernelGGL((product_tiles<T, 2, 2, 2, 2, 2>), grid, dim3(256), 0, s, args);
    else if (p.tile == 128) hipLaunchKernelGGL((product_tiles<T, 2, 2, 2, 2, 3>), grid, dim3(256), 0, s, args);
    else hipLaunchKernelGGL((product_tiles<T, 1, 2, 2, 1, 3>), grid, dim3(128), 0, s, args);
    return hip_ok(hipGetLastError());
  };
  return with_type(type, [&](auto kind) {
    using T = decltype(kind);
    if (p.cuts == 1) return tiles(T{}, c, ldc, accumulate);
    const int64_t ldp = parts_stride(b.rows);
    if (const int rc = tiles(float{}, workspace, ldp, false)) return rc;
    const int64_t blocks = (a.rows * (ldp / 4) + 255) / 256;
    hipLaunchKernelGGL(join_cuts<T>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s,
                       JoinArgs{static_cast<const float*>(workspace), c, a.rows, b.rows, ldp, ldc, p.cuts, accumulate});
    return hip_ok(hipGetLastError());
  });
}

}  // namespace halp

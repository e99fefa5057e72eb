// AdamW over many tensors in one launch, states in 32 or in 8 bits, and the norm of all gradients.
#include <cmath>
#include <cstring>
#include <new>

#include "halp_internal.hpp"
#include "mx4.hpp"

namespace halp {
namespace {

constexpr int kThreads = 256;
constexpr int kParts = 4;         // groups of four elements that a lane takes at a time
constexpr int kChunk = 4 * kThreads * kParts;  // elements of one tensor that a workgroup takes at a time
constexpr int kNormParts = 2048;  // partial sums of the gradient norm at most

struct Tensor {
  halp_adamw_tensor t;
  int64_t first;  // chunks of the tensors before this one
  int64_t whole;  // 1 where every pointer is aligned to four elements
};

struct StepArgs {
  const Tensor* tensors;
  const int32_t* owner;  // of each chunk, its tensor
  int64_t chunks;
  double lr, beta1, beta2, decay;
  float eps;
  int64_t step;
  const int64_t* step_at;
  const float* lr_at;
  const float* grad_scale;
  uint64_t seed;
};

// beta^t by repeated squaring, in 64 bits
__device__ double power(double beta, uint64_t t) {
  double r = 1;
  for (; t; t >>= 1, beta *= beta)
    if (t & 1) r *= beta;
  return r;
}

// ---- states in 8 bits -------------------------------------------------------------------------
// The format of m (BIAS 7, largest 1.75 2^8) and of v (BIAS 15, largest 1.875 2^15): three mantissa bits.
template <int BIAS>
__device__ __forceinline__ uint32_t state_scale(uint32_t max_bits) {
  constexpr int kTop = BIAS == 7 ? 8 : 15;
  constexpr uint32_t kOver = BIAS == 7 ? 0x600000u : 0x700000u;
  const int s = (int)(max_bits >> 23) - kTop + ((max_bits & 0x7FFFFFu) > kOver ? 1 : 0);
  return max_bits >= 0x7F800000u ? 255u : (uint32_t)(s > 0 ? s : 0);
}

// a >= 0 times 2^(127 - s) in the format, rounded up or down by 16 random bits (u, shifted left by 4): what lies below
// the third mantissa bit carries into it with its own probability.  A number below the least normal one
// has a fixed step, that of the least binade, and is moved there by adding its first number.
template <int BIAS>
__device__ __forceinline__ uint32_t state_code(float a, float inv, uint32_t u) {
  constexpr float kLeast = BIAS == 7 ? 0x1p-6f : 0x1p-14f;
  constexpr uint32_t kZero = (127u - BIAS) << 23;  // bits of the format's exponent 0
  const float t = a * inv;
  const bool low = t < kLeast;
  const uint32_t bits = __builtin_bit_cast(uint32_t, low ? t + kLeast : t);
  return (bits + u - (low ? kZero + (1u << 23) - 8u : kZero - 8u)) >> 20;
}

// The values of four codes of m: an 8-bit format of the hardware.
__device__ __forceinline__ void read_m4(uint32_t c, uint32_t s, float* m) {
  const float scale = mx_scale_value(s);
  const v2f32 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  m[0] = a.x * scale;
  m[1] = a.y * scale;
  m[2] = b.x * scale;
  m[3] = b.y * scale;
}

// ... and of v: the upper bits of a 16-bit float without its sign
__device__ __forceinline__ void read_v4(uint32_t c, uint32_t s, float* v) {
  const float scale = mx_scale_value(s);
  const v2f16 a = __builtin_bit_cast(v2f16, __builtin_amdgcn_perm(0, c, 0x0C010C00u) << 7),
              b = __builtin_bit_cast(v2f16, __builtin_amdgcn_perm(0, c, 0x0C030C02u) << 7);
  v[0] = (float)a.x * scale;
  v[1] = (float)a.y * scale;
  v[2] = (float)b.x * scale;
  v[3] = (float)b.y * scale;
}

// largest of eight adjacent lanes
__device__ __forceinline__ uint32_t max_of_8(uint32_t v) {
  v = max(v, dpp_quad_swap1(v));
  v = max(v, dpp_quad_swap2(v));
  return max(v, dpp_half_mirror(v));
}

// ---- four elements ----------------------------------------------------------------------------
template <typename T>
struct alignas(4 * sizeof(T)) Four {
  T v[4];
};

// k of them from element e on; whole: all four, aligned
template <typename T>
__device__ __forceinline__ Four<T> load4(const void* p, int64_t e, int k, bool whole) {
  const T* at = static_cast<const T*>(p) + e;
  Four<T> r;
  if (whole) {
    r = *reinterpret_cast<const Four<T>*>(at);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = i < k ? at[i] : T(0);
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void store4(void* p, int64_t e, int k, bool whole, const Four<T>& r) {
  T* at = static_cast<T*>(p) + e;
  if (whole) {
    *reinterpret_cast<Four<T>*>(at) = r;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < k) at[i] = r.v[i];
}

// sqrt(v) within a step and a reciprocal within one: v_sqrt_f32 takes subnormal numbers for zero, so small ones are scaled
__device__ __forceinline__ float fast_sqrt(float v) {
  const bool small = v < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(small ? v * 0x1p96f : v);
  return small ? r * 0x1p-48f : r;
}

// Four consecutive elements per lane, eight lanes to a block of 8-bit states.  Bound by memory with 32-bit states: 240 M
// elements at 5.3 TB/s where steps follow each other, 5.0 behind the norm of the same gradients (a copy of 2 GB runs at
// 4.9).  With 8-bit states the random blocks and the conversions take about as long as the memory: 100 M at 4.3 TB/s in a row of
// steps, 4.7 among other work, and 5.1 with gradients in fp32 and a copy.  Those kernels are held to 128 registers, four waves
// a SIMD, and spill two to five of them; with three waves and nothing spilled the same steps take 324 us in place of 325
// and 360 in place of 355.
template <typename G, typename C, bool BITS8>
__global__ __launch_bounds__(kThreads, BITS8 ? 4 : 2) void adamw_step(StepArgs a) {
  const float scale = a.grad_scale ? *a.grad_scale : 1.f;
  if (!(fabsf(scale) < __builtin_inff())) return;
  const int64_t step = a.step_at ? *a.step_at : a.step;
  const float lr_at = a.lr_at ? *a.lr_at : 0.f;
  if (step < 1 || step >= (int64_t(1) << 32) || !(lr_at >= 0 && lr_at < __builtin_inff())) return;
  const double lr = a.lr_at ? (double)lr_at : a.lr;
  const float keep = (float)(1 - lr * a.decay), rate = (float)(lr / (1 - power(a.beta1, step))),
              root = (float)(1 / sqrt(1 - power(a.beta2, step))), b1 = (float)a.beta1, b2 = (float)a.beta2,
              n1 = (float)(1 - a.beta1), n2 = (float)(1 - a.beta2);
  for (int64_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const Tensor& d = a.tensors[a.owner[chunk]];
    const halp_adamw_tensor t = d.t;
    const uint64_t seed = a.seed + (uint64_t)(&d - a.tensors);
    const int64_t e0 = (chunk - d.first) * kChunk + 4 * threadIdx.x;
    const auto run = [&](auto all) {  // all: every lane has its four, aligned
      // everything is asked for before any of it is used
      Four<float> p[kParts], m[kParts], v[kParts];
      Four<G> g[kParts];
      uint32_t mc[kParts], vc[kParts], ms[kParts], vs[kParts];
      const auto elements = [&](int u) { return all ? 4 : (int)max((int64_t)0, min((int64_t)4, t.n - e0 - u * 4 * kThreads)); };
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        const int64_t e = e0 + u * 4 * kThreads;
        const int k = elements(u);
        const bool whole = all || (d.whole && k == 4);
        p[u] = load4<float>(t.p, e, k, whole);
        g[u] = load4<G>(t.g, e, k, whole);
        if constexpr (BITS8) {
          mc[u] = __builtin_bit_cast(uint32_t, load4<uint8_t>(t.m, e, k, whole));
          vc[u] = __builtin_bit_cast(uint32_t, load4<uint8_t>(t.v, e, k, whole));
          ms[u] = k ? t.m_scale[e / 32] : 0;
          vs[u] = k ? t.v_scale[e / 32] : 0;
        } else {
          m[u] = load4<float>(t.m, e, k, whole);
          v[u] = load4<float>(t.v, e, k, whole);
        }
      }
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        const int64_t e = e0 + u * 4 * kThreads;
        const int k = elements(u);
        const bool whole = all || (d.whole && k == 4);
        if (!all && e - 4 * threadIdx.x >= t.n) break;  // the same for all lanes
        if constexpr (BITS8) {
          read_m4(mc[u], ms[u], m[u].v);
          read_v4(vc[u], vs[u], v[u].v);
        }
        uint32_t mmax = 0, vmax = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float gs = (float)g[u].v[i] * scale;
          float &mi = m[u].v[i], &vi = v[u].v[i], &pi = p[u].v[i];
          mi = mi * b1 + gs * n1;
          vi = vi * b2 + (gs * gs) * n2;
          pi = pi * keep - rate * (mi * __builtin_amdgcn_rcpf(fast_sqrt(vi) * root + a.eps));
          if (BITS8 && (all || i < k)) {
            mmax = max(mmax, __builtin_bit_cast(uint32_t, mi) & 0x7FFFFFFFu);
            vmax = max(vmax, __builtin_bit_cast(uint32_t, vi) & 0x7FFFFFFFu);
          }
        }
        store4(t.p, e, k, whole, p[u]);
        if (t.copy) {
          Four<C> c;
#pragma unroll
          for (int i = 0; i < 4; ++i) c.v[i] = (C)p[u].v[i];
          store4(t.copy, e, k, whole, c);
        }
        if constexpr (BITS8) {
          const uint32_t sm = state_scale<7>(max_of_8(mmax)), sv = state_scale<15>(max_of_8(vmax));
          const float im = mx_inverse(sm), iv = mx_inverse(sv);
          const U4 r = stream_block(seed, kMoments, (uint32_t)step, (uint64_t)e / 4);
          uint32_t cm = 0, cv = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t w = pick(r, i);
            const float mi = m[u].v[i];
            const uint32_t sign = __builtin_bit_cast(uint32_t, mi) >> 31 << 7;
            cm |= ((state_code<7>(fabsf(mi), im, (w & 0xFFFFu) << 4) & 127u) | sign) << (8 * i);
            cv |= (state_code<15>(v[u].v[i], iv, w >> 16 << 4) & 255u) << (8 * i);
          }
          if (sm == 255u) cm = 0;
          if (sv == 255u) cv = 0;
          store4(t.m, e, k, whole, __builtin_bit_cast(Four<uint8_t>, cm));
          store4(t.v, e, k, whole, __builtin_bit_cast(Four<uint8_t>, cv));
          if (k && threadIdx.x % 8 == 0) {
            t.m_scale[e / 32] = (uint8_t)sm;
            t.v_scale[e / 32] = (uint8_t)sv;
          }
        } else {
          store4(t.m, e, k, whole, m[u]);
          store4(t.v, e, k, whole, v[u]);
        }
      }
    };
    if (d.whole && (chunk - d.first + 1) * kChunk <= t.n) run(std::true_type{});
    else run(std::false_type{});
  }
}

// ---- norm of all gradients --------------------------------------------------------------------
struct NormArgs {
  const Tensor* tensors;
  const int32_t* owner;
  int64_t chunks;
  double* parts;
  int used;
  double most;
  float* out;
};

__device__ __forceinline__ double block_sum(double v) {  // in thread 0
  __shared__ double waves[16];
  for (int w = 32; w; w >>= 1) v += __shfl_down(v, w);
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = v;
  __syncthreads();
  double r = 0;
  if (threadIdx.x == 0)
    for (unsigned w = 0; w < blockDim.x / 64; ++w) r += waves[w];
  return r;
}

template <typename G>
__global__ __launch_bounds__(kThreads) void norm_parts(NormArgs a) {
  double sums[4] = {};
  for (int64_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const Tensor& d = a.tensors[a.owner[chunk]];
    const int64_t e0 = (chunk - d.first) * kChunk + 4 * threadIdx.x;
    Four<G> g[kParts];
    if (d.whole && (chunk - d.first + 1) * kChunk <= d.t.n) {
#pragma unroll
      for (int u = 0; u < kParts; ++u) g[u] = load4<G>(d.t.g, e0 + u * 4 * kThreads, 4, true);
    } else {
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        const int64_t e = e0 + u * 4 * kThreads;
        g[u] = load4<G>(d.t.g, e, (int)max((int64_t)0, min((int64_t)4, d.t.n - e)), false);
      }
    }
#pragma unroll
    for (int u = 0; u < kParts; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double x = (double)(float)g[u].v[i];
        sums[i] = __builtin_fma(x, x, sums[i]);
      }
  }
  const double sum = block_sum((sums[0] + sums[1]) + (sums[2] + sums[3]));
  if (threadIdx.x == 0) a.parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kThreads) void norm_join(NormArgs a) {
  double sum = 0;
  for (int i = threadIdx.x; i < a.used; i += kThreads) sum += a.parts[i];
  sum = block_sum(sum);
  if (threadIdx.x) return;
  const double norm = sqrt(sum);
  a.out[0] = (float)norm;
  a.out[1] = !(norm < __builtin_inf()) ? __builtin_nanf("") : (norm > a.most ? (float)(a.most / norm) : 1.f);
}

struct ReadArgs {
  const uint8_t *m, *ms, *v, *vs;
  float *mo, *vo;
  int64_t n;
  bool whole;
};

__global__ __launch_bounds__(kThreads) void read_moments(ReadArgs a) {
  for (int64_t chunk = blockIdx.x; chunk * kChunk < a.n; chunk += gridDim.x) {
    const int64_t e0 = chunk * kChunk + 4 * threadIdx.x;
    const auto run = [&](auto all) {
      uint32_t mc[kParts], vc[kParts], ms[kParts], vs[kParts];
      const auto elements = [&](int u) { return all ? 4 : (int)max((int64_t)0, min((int64_t)4, a.n - e0 - u * 4 * kThreads)); };
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        const int64_t e = e0 + u * 4 * kThreads;
        const int k = elements(u);
        mc[u] = __builtin_bit_cast(uint32_t, load4<uint8_t>(a.m, e, k, all));
        vc[u] = __builtin_bit_cast(uint32_t, load4<uint8_t>(a.v, e, k, all));
        ms[u] = k ? a.ms[e / 32] : 0;
        vs[u] = k ? a.vs[e / 32] : 0;
      }
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        const int64_t e = e0 + u * 4 * kThreads;
        Four<float> m, v;
        read_m4(mc[u], ms[u], m.v);
        read_v4(vc[u], vs[u], v.v);
        store4(a.mo, e, elements(u), all, m);
        store4(a.vo, e, elements(u), all, v);
      }
    };
    if (a.whole && (chunk + 1) * kChunk <= a.n) run(std::true_type{});
    else run(std::false_type{});
  }
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int check_tensor(const halp_adamw_tensor& t, int bits, int32_t grad_type, int32_t copy_type) {
  if (t.n < 0 || t.n >= (int64_t(1) << 40)) return HALP_ERR_INVALID;
  if (t.n == 0) return HALP_OK;
  if (!t.p || !t.g || !t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale))) return HALP_ERR_NULL;
  if (!aligned(t.p, 4) || !aligned(t.g, type_bytes(grad_type)) || !aligned(t.copy, type_bytes(copy_type))) return HALP_ERR_ALIGN;
  if (bits == 32 && (!aligned(t.m, 4) || !aligned(t.v, 4))) return HALP_ERR_ALIGN;
  return HALP_OK;
}

unsigned grid_for(int64_t chunks, int64_t most) { return (unsigned)(chunks < most ? chunks : most); }

}  // namespace
}  // namespace halp

using namespace halp;

struct halp_adamw {
  void* workspace = nullptr;  // Tensor [count], the partial sums of the norm, the tensor of each chunk
  const Tensor* tensors = nullptr;
  double* parts = nullptr;
  const int32_t* owner = nullptr;
  int64_t chunks = 0;
  int bits = 32;
  int32_t grad_type = 0, copy_type = 0;
  uint64_t seed = 0;
};

extern "C" {

int halp_adamw_create(halp_adamw** out, const halp_adamw_tensor* tensors, int64_t count, int32_t state_bits,
                      int32_t grad_type, int32_t copy_type, uint64_t seed) {
  if (!out) return HALP_ERR_NULL;
  *out = nullptr;
  if (!tensors) return HALP_ERR_NULL;
  if (count < 1 || count >= (int64_t(1) << 24) || !type_known(grad_type) || !type_known(copy_type)) return HALP_ERR_INVALID;
  if (state_bits != 8 && state_bits != 32) return HALP_ERR_UNSUPPORTED;
  for (int64_t i = 0; i < count; ++i)
    if (const int rc = check_tensor(tensors[i], state_bits, grad_type, copy_type)) return rc;
  int64_t chunks = 0;
  for (int64_t i = 0; i < count; ++i) chunks += (tensors[i].n + kChunk - 1) / kChunk;
  const size_t list_bytes = sizeof(Tensor) * count, part_bytes = sizeof(double) * kNormParts, bytes = list_bytes + part_bytes + 4 * chunks;
  halp_adamw* h = new (std::nothrow) halp_adamw();
  char* host = new (std::nothrow) char[bytes];
  if (!h || !host) {
    delete h;
    delete[] host;
    return HALP_ERR_HIP;
  }
  h->chunks = chunks; h->bits = state_bits; h->grad_type = grad_type; h->copy_type = copy_type; h->seed = seed;
  const size_t state = state_bits == 8 ? 4 : 16;
  int32_t* owner = reinterpret_cast<int32_t*>(host + list_bytes + part_bytes);
  int64_t first = 0;
  for (int64_t i = 0; i < count; ++i) {
    const halp_adamw_tensor& t = tensors[i];
    const Tensor d{t, first, aligned(t.p, 16) && aligned(t.g, 4 * type_bytes(grad_type)) && aligned(t.m, state) &&
                                 aligned(t.v, state) && aligned(t.copy, 4 * type_bytes(copy_type))};
    std::memcpy(host + sizeof(Tensor) * i, &d, sizeof d);
    for (int64_t k = 0; k < (t.n + kChunk - 1) / kChunk; ++k) owner[first++] = (int32_t)i;
  }
  std::memset(host + list_bytes, 0, part_bytes);
  const bool bad = hip_fail(hipMalloc(&h->workspace, bytes), "hipMalloc(adamw)") ||
                   hip_fail(hipMemcpy(h->workspace, host, bytes, hipMemcpyHostToDevice), "hipMemcpy(adamw)");
  delete[] host;
  if (bad) {
    halp_adamw_destroy(h);
    return HALP_ERR_HIP;
  }
  char* base = static_cast<char*>(h->workspace);
  h->tensors = reinterpret_cast<const Tensor*>(base);
  h->parts = reinterpret_cast<double*>(base + list_bytes);
  h->owner = reinterpret_cast<const int32_t*>(base + list_bytes + part_bytes);
  *out = h;
  return HALP_OK;
}

int halp_adamw_destroy(halp_adamw* h) {
  if (!h) return HALP_ERR_NULL;
  if (h->workspace) (void)hipFree(h->workspace);
  delete h;
  return HALP_OK;
}

int halp_adamw_step(halp_adamw* h, const halp_adamw_args* p, void* stream) {
  if (!h || !p) return HALP_ERR_NULL;
  if (!(p->lr >= 0) || !std::isfinite(p->lr) || !(p->beta1 >= 0 && p->beta1 < 1) || !(p->beta2 >= 0 && p->beta2 < 1) ||
      !((float)p->eps >= 0x1p-126f && (float)p->eps < 0x1p126f) || !(p->weight_decay >= 0) || !std::isfinite(p->weight_decay))
    return HALP_ERR_INVALID;
  if (!p->step_at && (p->step < 1 || p->step >= (int64_t(1) << 32))) return HALP_ERR_INVALID;
  if (!aligned(p->step_at, 8) || !aligned(p->lr_at, 4) || !aligned(p->grad_scale, 4)) return HALP_ERR_ALIGN;
  if (h->chunks == 0) return HALP_OK;
  const StepArgs a{h->tensors, h->owner, h->chunks, p->lr, p->beta1, p->beta2,
                   p->weight_decay, (float)p->eps, p->step, p->step_at, p->lr_at, p->grad_scale, h->seed};
  const dim3 grid(grid_for(h->chunks, int64_t(1) << 20));
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return with_type(h->grad_type, [&](auto g) {
    return with_type(h->copy_type, [&](auto c) {
      using G = decltype(g);
      using C = decltype(c);
      if (h->bits == 8) hipLaunchKernelGGL((adamw_step<G, C, true>), grid, dim3(kThreads), 0, s, a);
      else hipLaunchKernelGGL((adamw_step<G, C, false>), grid, dim3(kThreads), 0, s, a);
      return hip_ok(hipGetLastError());
    });
  });
}

int halp_adamw_grad_norm(halp_adamw* h, double max_norm, float* out, void* stream) {
  if (!h || !out) return HALP_ERR_NULL;
  if (!(max_norm > 0)) return HALP_ERR_INVALID;
  if (!aligned(out, 4)) return HALP_ERR_ALIGN;
  NormArgs a{h->tensors, h->owner, h->chunks, h->parts, (int)grid_for(h->chunks, kNormParts),
             max_norm, out};
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return with_type(h->grad_type, [&](auto g) {
    using G = decltype(g);
    if (a.used) hipLaunchKernelGGL(norm_parts<G>, dim3(a.used), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(norm_join, dim3(1), dim3(kThreads), 0, s, a);
    return hip_ok(hipGetLastError());
  });
}

int halp_adamw_read_moments(const uint8_t* m, const uint8_t* m_scale, const uint8_t* v, const uint8_t* v_scale,
                            int64_t n, float* m_out, float* v_out, void* stream) {
  if (n < 0 || n >= (int64_t(1) << 40)) return HALP_ERR_INVALID;
  if (n == 0) return HALP_OK;
  if (!m || !m_scale || !v || !v_scale || !m_out || !v_out) return HALP_ERR_NULL;
  if (!aligned(m_out, 4) || !aligned(v_out, 4)) return HALP_ERR_ALIGN;
  const bool whole = aligned(m, 4) && aligned(v, 4) && aligned(m_out, 16) && aligned(v_out, 16);
  const dim3 grid(grid_for((n + kChunk - 1) / kChunk, int64_t(1) << 20));
  hipLaunchKernelGGL(read_moments, grid, dim3(kThreads), 0, reinterpret_cast<hipStream_t>(stream),
                     ReadArgs{m, m_scale, v, v_scale, m_out, v_out, n, whole});
  return hip_ok(hipGetLastError());
}

}  // extern "C"

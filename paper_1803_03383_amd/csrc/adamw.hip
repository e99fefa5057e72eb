// AdamW over many tensors in one launch, states in 32 or in 8 bits, and the norm of all gradients.
#include <cmath>
#include <cstring>
#include <new>

#include "halp_internal.hpp"
#include "mx4.hpp"

namespace halp {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;      // elements of one tensor that a workgroup takes at a time
constexpr int kNormParts = 2048;  // partial sums of the gradient norm at most

struct Tensor {
  halp_adamw_tensor t;
  int64_t first;  // chunks of the tensors before this one
  int64_t whole;  // 1 where every pointer is aligned to four elements
};

struct StepArgs {
  const Tensor* tensors;
  int64_t count, chunks;
  double lr, beta1, beta2, decay;
  float eps;
  int64_t step;
  const int64_t* step_at;
  const float* lr_at;
  const float* grad_scale;
  uint64_t seed;
};

__device__ __forceinline__ const Tensor& tensor_of(const Tensor* t, int64_t count, int64_t chunk) {
  int64_t lo = 0, hi = count;  // the last tensor whose first chunk is not past this one
  while (hi - lo > 1) {
    const int64_t mid = (lo + hi) / 2;
    if (t[mid].first <= chunk) lo = mid;
    else hi = mid;
  }
  return t[lo];
}

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

// a >= 0 times 2^(127 - s) in the format, rounded up or down by 16 random bits: what lies below the
// third mantissa bit carries into it with its own probability.  A number below the least normal one
// has a fixed step, that of the least binade, and is moved there by adding its first number.
template <int BIAS>
__device__ __forceinline__ uint32_t state_code(float a, float inv, uint32_t u) {
  constexpr float kLeast = BIAS == 7 ? 0x1p-6f : 0x1p-14f;
  const float t = a * inv;
  const bool low = t < kLeast;
  const uint32_t bits = __builtin_bit_cast(uint32_t, low ? t + kLeast : t);
  return ((bits + 16u * u + 8u) >> 20) - 8u * (127 - BIAS) - (low ? 8u : 0u);
}

__device__ __forceinline__ float read_m(uint32_t c, uint32_t s) {  // c: one byte
  const uint32_t f = c & 7u, e = c >> 3 & 15u;
  const float a = e ? __builtin_bit_cast(float, (e + 120u) << 23 | f << 20) : (float)f * 0x1p-9f;
  return s == 255u ? __builtin_nanf("") : ldexpf(c & 128u ? -a : a, (int)s - 127);
}

__device__ __forceinline__ float read_v(uint32_t c, uint32_t s) {
  const uint32_t f = c & 7u, e = c >> 3;
  const float a = e ? __builtin_bit_cast(float, (e + 112u) << 23 | f << 20) : (float)f * 0x1p-17f;
  return s == 255u ? __builtin_nanf("") : ldexpf(a, (int)s - 127);
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

template <typename T>
__device__ __forceinline__ Four<T> load4(const void* p, int64_t e, int k, bool whole) {
  const T* at = static_cast<const T*>(p) + e;
  Four<T> r{};
  if (whole) return *reinterpret_cast<const Four<T>*>(at);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < k) r.v[i] = at[i];
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

// Four consecutive elements per lane, eight lanes to a block of 8-bit states.
template <typename G, typename C, bool BITS8>
__global__ __launch_bounds__(kThreads) void adamw_step(StepArgs a) {
  const float scale = a.grad_scale ? *a.grad_scale : 1.f;
  if (!(fabsf(scale) < __builtin_inff())) return;
  const int64_t step = a.step_at ? *a.step_at : a.step;
  if (step < 1 || step >= (int64_t(1) << 32)) return;
  const double lr = a.lr_at ? (double)*a.lr_at : a.lr;
  const float keep = (float)(1 - lr * a.decay), rate = (float)(lr / (1 - power(a.beta1, step))),
              root = (float)(1 / sqrt(1 - power(a.beta2, step))), b1 = (float)a.beta1, b2 = (float)a.beta2,
              n1 = (float)(1 - a.beta1), n2 = (float)(1 - a.beta2);
  for (int64_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const Tensor& d = tensor_of(a.tensors, a.count, chunk);
    const halp_adamw_tensor t = d.t;
    const uint64_t seed = a.seed + (uint64_t)(&d - a.tensors);
    for (int part = 0; part < kChunk; part += 4 * kThreads) {
      const int64_t e = (chunk - d.first) * kChunk + part + 4 * threadIdx.x;
      if (e - 4 * threadIdx.x >= t.n) break;
      const int k = (int)(t.n - e < 4 ? (t.n - e > 0 ? t.n - e : 0) : 4);  // elements of this lane
      const bool whole = d.whole && k == 4;
      Four<float> p = load4<float>(t.p, e, k, whole), m, v;
      const Four<G> g = load4<G>(t.g, e, k, whole);
      if (BITS8) {
        const Four<uint8_t> mc = load4<uint8_t>(t.m, e, k, whole), vc = load4<uint8_t>(t.v, e, k, whole);
        const uint32_t ms = k ? t.m_scale[e / 32] : 0, vs = k ? t.v_scale[e / 32] : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          m.v[i] = read_m(mc.v[i], ms);
          v.v[i] = read_v(vc.v[i], vs);
        }
      } else {
        m = load4<float>(t.m, e, k, whole);
        v = load4<float>(t.v, e, k, whole);
      }
      uint32_t mmax = 0, vmax = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float gs = (float)g.v[i] * scale;
        m.v[i] = m.v[i] * b1 + gs * n1;
        v.v[i] = v.v[i] * b2 + (gs * gs) * n2;
        p.v[i] = p.v[i] * keep - rate * (m.v[i] / (sqrtf(v.v[i]) * root + a.eps));
        if (i < k) {
          mmax = max(mmax, __builtin_bit_cast(uint32_t, m.v[i]) & 0x7FFFFFFFu);
          vmax = max(vmax, __builtin_bit_cast(uint32_t, v.v[i]) & 0x7FFFFFFFu);
        }
      }
      store4(t.p, e, k, whole, p);
      if (t.copy) {
        Four<C> c;
#pragma unroll
        for (int i = 0; i < 4; ++i) c.v[i] = (C)p.v[i];
        store4(t.copy, e, k, whole, c);
      }
      if (BITS8) {
        const uint32_t ms = state_scale<7>(max_of_8(mmax)), vs = state_scale<15>(max_of_8(vmax));
        const float mi = mx_inverse(ms), vi = mx_inverse(vs);
        const U4 r = stream_block(seed, kMoments, (uint32_t)step, (uint64_t)e / 4);
        Four<uint8_t> mc, vc;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t u = pick(r, i), bits = __builtin_bit_cast(uint32_t, m.v[i]);
          const uint32_t cm = state_code<7>(__builtin_bit_cast(float, bits & 0x7FFFFFFFu), mi, u & 0xFFFFu) | (bits >> 24 & 128u);
          const uint32_t cv = state_code<15>(v.v[i], vi, u >> 16);
          mc.v[i] = (uint8_t)(ms == 255u ? 0u : cm);
          vc.v[i] = (uint8_t)(vs == 255u ? 0u : cv);
        }
        store4(t.m, e, k, whole, mc);
        store4(t.v, e, k, whole, vc);
        if (k && threadIdx.x % 8 == 0) {
          t.m_scale[e / 32] = (uint8_t)ms;
          t.v_scale[e / 32] = (uint8_t)vs;
        }
      } else {
        store4(t.m, e, k, whole, m);
        store4(t.v, e, k, whole, v);
      }
    }
  }
}

// ---- norm of all gradients --------------------------------------------------------------------
struct NormArgs {
  const Tensor* tensors;
  int64_t count, chunks;
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
  double sum = 0;
  for (int64_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const Tensor& d = tensor_of(a.tensors, a.count, chunk);
    for (int part = 0; part < kChunk; part += 4 * kThreads) {
      const int64_t e = (chunk - d.first) * kChunk + part + 4 * threadIdx.x;
      if (e >= d.t.n) break;
      const int k = (int)(d.t.n - e < 4 ? d.t.n - e : 4);
      const Four<G> g = load4<G>(d.t.g, e, k, d.whole && k == 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += (double)(float)g.v[i] * (double)(float)g.v[i];
    }
  }
  sum = block_sum(sum);
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
};

__global__ __launch_bounds__(kThreads) void read_moments(ReadArgs a) {
  for (int64_t e = blockIdx.x * (int64_t)kThreads + threadIdx.x; e < a.n; e += gridDim.x * (int64_t)kThreads) {
    a.mo[e] = read_m(a.m[e], a.ms[e / 32]);
    a.vo[e] = read_v(a.v[e], a.vs[e / 32]);
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
  void* device_list = nullptr;  // Tensor [count], then the partial sums of the norm
  double* parts = nullptr;
  int64_t count = 0, chunks = 0;
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
  halp_adamw* h = new (std::nothrow) halp_adamw();
  Tensor* list = new (std::nothrow) Tensor[count];
  if (!h || !list) {
    delete h;
    delete[] list;
    return HALP_ERR_HIP;
  }
  h->count = count; h->bits = state_bits; h->grad_type = grad_type; h->copy_type = copy_type; h->seed = seed;
  const size_t state = state_bits == 8 ? 4 : 16;
  for (int64_t i = 0; i < count; ++i) {
    const halp_adamw_tensor& t = tensors[i];
    list[i].t = t;
    list[i].first = h->chunks;
    list[i].whole = aligned(t.p, 16) && aligned(t.g, 4 * type_bytes(grad_type)) && aligned(t.m, state) &&
                    aligned(t.v, state) && aligned(t.copy, 4 * type_bytes(copy_type));
    h->chunks += (t.n + kChunk - 1) / kChunk;
  }
  const size_t bytes = sizeof(Tensor) * count;
  const bool bad = hip_fail(hipMalloc(&h->device_list, bytes + sizeof(double) * kNormParts), "hipMalloc(adamw)") ||
                   hip_fail(hipMemcpy(h->device_list, list, bytes, hipMemcpyHostToDevice), "hipMemcpy(adamw)");
  delete[] list;
  if (bad) {
    halp_adamw_destroy(h);
    return HALP_ERR_HIP;
  }
  h->parts = reinterpret_cast<double*>(static_cast<char*>(h->device_list) + bytes);
  *out = h;
  return HALP_OK;
}

int halp_adamw_destroy(halp_adamw* h) {
  if (!h) return HALP_ERR_NULL;
  if (h->device_list) (void)hipFree(h->device_list);
  delete h;
  return HALP_OK;
}

int halp_adamw_step(halp_adamw* h, const halp_adamw_args* p, void* stream) {
  if (!h || !p) return HALP_ERR_NULL;
  if (!(p->lr >= 0) || !std::isfinite(p->lr) || !(p->beta1 >= 0 && p->beta1 < 1) || !(p->beta2 >= 0 && p->beta2 < 1) ||
      !((float)p->eps > 0) || !std::isfinite((float)p->eps) || !(p->weight_decay >= 0) || !std::isfinite(p->weight_decay))
    return HALP_ERR_INVALID;
  if (!p->step_at && (p->step < 1 || p->step >= (int64_t(1) << 32))) return HALP_ERR_INVALID;
  if (!aligned(p->step_at, 8) || !aligned(p->lr_at, 4) || !aligned(p->grad_scale, 4)) return HALP_ERR_ALIGN;
  if (h->chunks == 0) return HALP_OK;
  const StepArgs a{static_cast<const Tensor*>(h->device_list), h->count, h->chunks, p->lr, p->beta1, p->beta2,
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
  NormArgs a{static_cast<const Tensor*>(h->device_list), h->count, h->chunks, h->parts, (int)grid_for(h->chunks, kNormParts),
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
  const dim3 grid(grid_for((n + kThreads - 1) / kThreads, 65536));
  hipLaunchKernelGGL(read_moments, grid, dim3(kThreads), 0, reinterpret_cast<hipStream_t>(stream),
                     ReadArgs{m, m_scale, v, v_scale, m_out, v_out, n});
  return hip_ok(hipGetLastError());
}

}  // extern "C"

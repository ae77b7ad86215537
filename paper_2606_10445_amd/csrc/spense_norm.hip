// Norms before and after a block, fused with its gate, the residual scale and the per-token
// fp8 quantisation that the next Spense GEMM takes.  Per token row:
//   t = y * rsqrt(mean(y^2) + eps) * w_post   (y itself without a post-norm),
//   r = alpha * x + g * t                     (x itself without a block output),
//   n = r * rsqrt(mean(r^2) + eps) * w_pre,
// r rounded to the stream's type, n to the activations' type and / or to e4m3fn codes with
// scale max|n| / 448.  Everything between the loads and those roundings is fp32, and n is
// formed from the fp32 r, not from the rounded one: a row is rounded once on each way out.
//
// Memory-bound: 12 fp32 operations per element against 2 to 14 bytes.  A row is read once
// and held in registers between its three reductions (sum of y^2, sum of r^2, max of |n|).
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "spense.h"
#include "spense_internal.h"

namespace spense {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

struct NormArgs {
  const uint8_t* x;
  int64_t ldx_b;
  const uint8_t* y;  // NULL: no block output
  int64_t ldy_b;
  const uint8_t* gate;  // NULL: 1
  int64_t ldg_b;        // 0: one row for all tokens
  const uint8_t* wpost;  // NULL: no post-norm
  const uint8_t* wpre;   // NULL: ones
  int32_t w_bf16;
  float alpha, eps;
  int64_t K;
  uint8_t* r;  // NULL: not written
  int64_t ldr_b;
  uint8_t* n;  // NULL: not written
  int64_t ldn_b;
  uint8_t* q;  // NULL: not written
  int64_t ldq;
  float* scales;
};

__device__ __forceinline__ float bf16_f32(uint32_t lo16) { return __uint_as_float(lo16 << 16); }
__device__ __forceinline__ uint32_t f32_bf16(float v) {
  __bf16 h = (__bf16)v;  // round to nearest even
  return (uint32_t)__builtin_bit_cast(uint16_t, h);
}

// E = 8: elements k .. k + 7, 16-byte aligned; E = 1: element k.
template <bool BF, int E>
__device__ __forceinline__ void load_vals(float (&v)[E], const uint8_t* row, int64_t k) {
  if constexpr (E == 1) {
    if constexpr (BF)
      v[0] = bf16_f32(reinterpret_cast<const uint16_t*>(row)[k]);
    else
      v[0] = reinterpret_cast<const float*>(row)[k];
  } else if constexpr (BF) {
    const v4i a = *reinterpret_cast<const v4i*>(row + 2 * k);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e & 1 ? __uint_as_float((uint32_t)a[e / 2] & 0xffff0000u) : bf16_f32((uint32_t)a[e / 2] & 0xffffu);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const v4i a = *reinterpret_cast<const v4i*>(row + 4 * k + 16 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * h + e] = __int_as_float(a[e]);
    }
  }
}

template <bool BF, int E>
__device__ __forceinline__ void store_vals(const float (&v)[E], uint8_t* row, int64_t k) {
  if constexpr (E == 1) {
    if constexpr (BF)
      reinterpret_cast<uint16_t*>(row)[k] = (uint16_t)f32_bf16(v[0]);
    else
      reinterpret_cast<float*>(row)[k] = v[0];
  } else if constexpr (BF) {
    v4i a;
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = (int)(f32_bf16(v[2 * e]) | (f32_bf16(v[2 * e + 1]) << 16));
    *reinterpret_cast<v4i*>(row + 2 * k) = a;
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<v4i*>(row + 4 * k + 16 * h) =
          (v4i){__float_as_int(v[4 * h]), __float_as_int(v[4 * h + 1]), __float_as_int(v[4 * h + 2]), __float_as_int(v[4 * h + 3])};
  }
}

template <int E>
__device__ __forceinline__ void load_weights(float (&v)[E], const uint8_t* w, int bf, int64_t k) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = 1.0f;
  } else if (bf) {
    load_vals<true, E>(v, w, k);
  } else {
    load_vals<false, E>(v, w, k);
  }
}

// Codes of v / s (a correctly rounded division; |v / s| rounds to at most 448).
template <int E>
__device__ __forceinline__ void store_codes(const float (&v)[E], float s, uint8_t* q, int64_t k) {
  if constexpr (E == 1) {
    q[k] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[0] / s, 0.0f, 0, false);
  } else {
    typedef int v2i __attribute__((ext_vector_type(2)));
    v2i w;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] / s, v[4 * h + 3] / s,
                                             __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] / s, v[4 * h + 1] / s, 0, false), true);
    *reinterpret_cast<v2i*>(q + k) = w;
  }
}

// Sum or maximum over the workgroup; `red` (16 floats) is used by one reduction only, so one
// barrier is enough.
template <bool MAX>
__device__ __forceinline__ float block_reduce(float v, float* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const float u = __shfl_xor(v, o, 64);
    v = MAX ? fmaxf(v, u) : v + u;
  }
  const int nw = blockDim.x >> 6;
  if (nw == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = red[0];
  for (int i = 1; i < nw; ++i) s = MAX ? fmaxf(s, red[i]) : s + red[i];
  return s;
}

// Rows of up to NJ * E * blockDim.x elements, in registers: thread t owns pieces t + j *
// blockDim.x of E elements.  K is a multiple of E.
template <bool XBF, bool YBF, int E, int NJ>
__global__ __launch_bounds__(1024) void block_norm_kernel(NormArgs a) {
  __shared__ float red[3][16];
  const int64_t m = blockIdx.x;
  const uint8_t* xr = a.x + m * a.ldx_b;
  const float invk = 1.0f / (float)a.K;
  float r[NJ][E], t[NJ][E], g[NJ][E];
  bool in[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int64_t k = (int64_t)E * (threadIdx.x + (int64_t)blockDim.x * j);
    in[j] = k < a.K;
    const int64_t ks = in[j] ? k : 0;  // pieces past the row read its first one and are masked
    load_vals<XBF, E>(r[j], xr, ks);
    if (a.y) load_vals<YBF, E>(t[j], a.y + m * a.ldy_b, ks);
    if (a.gate) load_vals<YBF, E>(g[j], a.gate + m * a.ldg_b, ks);
  }
  if (a.y) {
    if (a.wpost) {
      float ss = 0.0f;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) ss += in[j] ? t[j][e] * t[j][e] : 0.0f;
      const float inv = rsqrtf(block_reduce<false>(ss, red[0]) * invk + a.eps);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float w[E];
        load_weights<E>(w, a.wpost, a.w_bf16, in[j] ? (int64_t)E * (threadIdx.x + (int64_t)blockDim.x * j) : 0);
#pragma unroll
        for (int e = 0; e < E; ++e) t[j][e] = t[j][e] * inv * w[e];
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < E; ++e) r[j][e] = a.alpha * r[j][e] + (a.gate ? g[j][e] * t[j][e] : t[j][e]);
  }
  if (a.r) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (in[j]) store_vals<XBF, E>(r[j], a.r + m * a.ldr_b, (int64_t)E * (threadIdx.x + (int64_t)blockDim.x * j));
  }
  if (!a.n && !a.q) return;
  float ss = 0.0f;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < E; ++e) ss += in[j] ? r[j][e] * r[j][e] : 0.0f;
  const float inv = rsqrtf(block_reduce<false>(ss, red[1]) * invk + a.eps);
  float amax = 0.0f;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int64_t k = (int64_t)E * (threadIdx.x + (int64_t)blockDim.x * j);
    float w[E];
    load_weights<E>(w, a.wpre, a.w_bf16, in[j] ? k : 0);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      r[j][e] = r[j][e] * inv * w[e];
      if (in[j]) amax = fmaxf(amax, fabsf(r[j][e]));
    }
    if (a.n && in[j]) store_vals<YBF, E>(r[j], a.n + m * a.ldn_b, k);
  }
  if (!a.q) return;
  amax = block_reduce<true>(amax, red[2]);
  const float s = amax > 0.0f ? amax / 448.0f : 1.0f;
  if (threadIdx.x == 0) a.scales[m] = s;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
    if (in[j]) store_codes<E>(r[j], s, a.q + m * a.ldq, (int64_t)E * (threadIdx.x + (int64_t)blockDim.x * j));
}

// Rows of any length: four passes over the row (the later ones from L2), each forming the
// same values with the same instructions.  The outputs are written in the last pass only,
// element k by the thread that read it, so r may be x and n may be y.
template <bool XBF, bool YBF>
__global__ __launch_bounds__(1024) void block_norm_long_kernel(NormArgs a) {
  __shared__ float red[3][16];
  const int64_t m = blockIdx.x;
  const uint8_t* xr = a.x + m * a.ldx_b;
  const uint8_t* yr = a.y ? a.y + m * a.ldy_b : nullptr;
  const float invk = 1.0f / (float)a.K;
  float inv1 = 1.0f;
  if (yr && a.wpost) {
    float ss = 0.0f;
    for (int64_t k = threadIdx.x; k < a.K; k += blockDim.x) {
      float v[1];
      load_vals<YBF, 1>(v, yr, k);
      ss += v[0] * v[0];
    }
    inv1 = rsqrtf(block_reduce<false>(ss, red[0]) * invk + a.eps);
  }
  auto residual = [&](int64_t k) {
    float x[1];
    load_vals<XBF, 1>(x, xr, k);
    if (!yr) return x[0];
    float t[1], w[1], g[1] = {1.0f};
    load_vals<YBF, 1>(t, yr, k);
    if (a.wpost) {
      load_weights<1>(w, a.wpost, a.w_bf16, k);
      t[0] = t[0] * inv1 * w[0];
    }
    if (!a.gate) return a.alpha * x[0] + t[0];
    load_vals<YBF, 1>(g, a.gate + m * a.ldg_b, k);
    return a.alpha * x[0] + g[0] * t[0];
  };
  float inv = 1.0f, s = 1.0f;
  if (a.n || a.q) {
    float ss = 0.0f;
    for (int64_t k = threadIdx.x; k < a.K; k += blockDim.x) {
      const float r = residual(k);
      ss += r * r;
    }
    inv = rsqrtf(block_reduce<false>(ss, red[1]) * invk + a.eps);
  }
  auto normed = [&](float r, int64_t k) {
    float w[1];
    load_weights<1>(w, a.wpre, a.w_bf16, k);
    return r * inv * w[0];
  };
  if (a.q) {
    float amax = 0.0f;
    for (int64_t k = threadIdx.x; k < a.K; k += blockDim.x) amax = fmaxf(amax, fabsf(normed(residual(k), k)));
    amax = block_reduce<true>(amax, red[2]);
    s = amax > 0.0f ? amax / 448.0f : 1.0f;
    if (threadIdx.x == 0) a.scales[m] = s;
  }
  for (int64_t k = threadIdx.x; k < a.K; k += blockDim.x) {
    const float r[1] = {residual(k)};
    const float n[1] = {normed(r[0], k)};
    if (a.r) store_vals<XBF, 1>(r, a.r + m * a.ldr_b, k);
    if (a.n) store_vals<YBF, 1>(n, a.n + m * a.ldn_b, k);
    if (a.q) store_codes<1>(n, s, a.q + m * a.ldq, k);
  }
}

template <bool XBF, bool YBF>
hipError_t launch_norm(const NormArgs& a, int64_t M, bool vec, hipStream_t st) {
  const dim3 grid((unsigned)M);
  auto launch = [&](auto kernel, int64_t per_thread) {
    const int64_t threads = ((a.K + per_thread - 1) / per_thread + 63) / 64 * 64;
    hipLaunchKernelGGL(kernel, grid, dim3((unsigned)threads), 0, st, a);
    return hipGetLastError();
  };
  if (vec && a.K <= 8192) return launch(block_norm_kernel<XBF, YBF, 8, 1>, 8);
  if (vec && a.K <= 16384) return launch(block_norm_kernel<XBF, YBF, 8, 2>, 16);
  if (vec && a.K <= 32768) return launch(block_norm_kernel<XBF, YBF, 8, 4>, 32);
  if (a.K <= 4096) return launch(block_norm_kernel<XBF, YBF, 1, 4>, 4);
  if (a.K <= 16384) return launch(block_norm_kernel<XBF, YBF, 1, 16>, 16);
  hipLaunchKernelGGL((block_norm_long_kernel<XBF, YBF>), grid, dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace spense

using spense::api_fail;

extern "C" int spense_block_norm(const spense_block_norm_t* p, hipStream_t stream) {
  if (!p) return api_fail(SPENSE_ERR_ARG, "block_norm arguments are NULL");
  const spense_block_norm_t& b = *p;
  auto bad_type = [](int32_t t) { return t != SPENSE_BF16 && t != SPENSE_F32; };
  if (b.M < 0 || b.K < 0 || b.M > INT32_MAX || b.K > INT32_MAX)
    return api_fail(SPENSE_ERR_ARG, "bad M=%lld K=%lld", (long long)b.M, (long long)b.K);
  if (bad_type(b.x_type)) return api_fail(SPENSE_ERR_ARG, "x_type %d is not bf16 or f32", b.x_type);
  if (bad_type(b.y_type)) return api_fail(SPENSE_ERR_ARG, "y_type %d is not bf16 or f32", b.y_type);
  if (bad_type(b.w_type)) return api_fail(SPENSE_ERR_ARG, "w_type %d is not bf16 or f32", b.w_type);
  if (!(b.eps >= 0.0f) || !(b.eps < INFINITY)) return api_fail(SPENSE_ERR_ARG, "eps is negative or not finite");
  if (!b.y && (b.gate || b.post_weight)) return api_fail(SPENSE_ERR_ARG, "a gate or post_weight needs a block output y");
  if ((b.q != nullptr) != (b.scales != nullptr)) return api_fail(SPENSE_ERR_ARG, "q and scales go together");
  if (b.M == 0 || b.K == 0) return spense::api_ok();
  if (!b.x) return api_fail(SPENSE_ERR_ARG, "x is NULL");
  if (!b.residual && !b.normed && !b.q) return api_fail(SPENSE_ERR_ARG, "no output is asked for");
  if (b.ldx < b.K || (b.y && b.ldy < b.K) || (b.gate && b.ldg != 0 && b.ldg < b.K) || (b.residual && b.ldr < b.K) ||
      (b.normed && b.ldn < b.K) || (b.q && b.ldq < b.K))
    return api_fail(SPENSE_ERR_ARG, "leading dimension below K");
  const int64_t xs = b.x_type == SPENSE_BF16 ? 2 : 4, ys = b.y_type == SPENSE_BF16 ? 2 : 4,
                ws = b.w_type == SPENSE_BF16 ? 2 : 4;
  bool vec = b.K % 8 == 0, fits = true;
  auto view = [&](const void* ptr, int64_t ld, int64_t es, int64_t align) {  // an operand's alignment
    if (!ptr) return;
    fits = fits && reinterpret_cast<uintptr_t>(ptr) % es == 0;
    vec = vec && reinterpret_cast<uintptr_t>(ptr) % align == 0 && (ld * es) % align == 0;
  };
  view(b.x, b.ldx, xs, 16);
  view(b.y, b.ldy, ys, 16);
  view(b.gate, b.ldg, ys, 16);
  view(b.post_weight, 0, ws, 16);
  view(b.weight, 0, ws, 16);
  view(b.residual, b.ldr, xs, 16);
  view(b.normed, b.ldn, ys, 16);
  view(b.q, b.ldq, 1, 8);
  view(b.scales, 0, 4, 4);
  if (!fits) return api_fail(SPENSE_ERR_ALIGN, "an operand is not aligned to its elements");
  int rc = spense::api_check_device();
  if (rc) return rc;
  spense::NormArgs a;
  a.x = static_cast<const uint8_t*>(b.x), a.ldx_b = b.ldx * xs;
  a.y = static_cast<const uint8_t*>(b.y), a.ldy_b = b.ldy * ys;
  a.gate = static_cast<const uint8_t*>(b.gate), a.ldg_b = b.ldg * ys;
  a.wpost = static_cast<const uint8_t*>(b.post_weight), a.wpre = static_cast<const uint8_t*>(b.weight);
  a.w_bf16 = b.w_type == SPENSE_BF16;
  a.alpha = b.residual_scale, a.eps = b.eps, a.K = b.K;
  a.r = static_cast<uint8_t*>(b.residual), a.ldr_b = b.ldr * xs;
  a.n = static_cast<uint8_t*>(b.normed), a.ldn_b = b.ldn * ys;
  a.q = b.q, a.ldq = b.ldq, a.scales = b.scales;
  const bool xb = b.x_type == SPENSE_BF16, yb = b.y_type == SPENSE_BF16;
  const hipError_t e = xb ? (yb ? spense::launch_norm<true, true>(a, b.M, vec, stream)
                                : spense::launch_norm<true, false>(a, b.M, vec, stream))
                          : (yb ? spense::launch_norm<false, true>(a, b.M, vec, stream)
                                : spense::launch_norm<false, false>(a, b.M, vec, stream));
  if (e != hipSuccess) return api_fail(SPENSE_ERR_HIP, "block norm launch failed: %s", hipGetErrorString(e));
  return spense::api_ok();
}

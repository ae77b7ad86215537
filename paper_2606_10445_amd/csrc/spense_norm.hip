// Norms before and after a block, fused with its gate, the residual scale and the per-token
// fp8 quantisation that the next Spense GEMM takes.  Per token row:
//   t = y * rsqrt(mean(y^2) + eps) * w_post   (y itself without a post-norm),
//   r = alpha * x + g * t                     (x itself without a block output),
//   n = r * rsqrt(mean(r^2) + eps) * w_pre,
// r rounded to the stream's type, n to the activations' type and / or to e4m3fn codes with
// scale max|n| / 448.  Everything between the loads and those roundings is fp32, and n is
// formed from the fp32 r, not from the rounded one: a row is rounded once on each way out.
//
// Memory-bound by its bytes (12 operations an element against 2 to 29 bytes), but a row's three
// reductions (sum of y^2, sum of r^2, max of |n|) wait for each other with the row held in
// registers, so what counts is rows in flight: 8192 x 5120 bf16 with gate, residual, n and codes 94 us,
// 4.0 TB/s, fp32 5.5 TB/s where a copy reaches 5.1; four-pieces-a-thread rows and single waves a
// row hold fewer and took 128 and 170 us.
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
  int64_t M, K;
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

// Eight elements from column k of a row.  AL: 16-byte aligned (8 for codes) and K a multiple of 8;
// else the same wide accesses at the alignment of the elements.
template <int ALIGN>
struct Wide;
template <>
struct Wide<16> {
  typedef int type __attribute__((ext_vector_type(4), aligned(16)));
};
template <>
struct Wide<4> {
  typedef int type __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Wide<2> {
  typedef int type __attribute__((ext_vector_type(4), aligned(2)));
};
template <bool AL>
struct Codes {
  typedef int type __attribute__((ext_vector_type(2), aligned(8)));
};
template <>
struct Codes<false> {
  typedef int type __attribute__((ext_vector_type(2), aligned(1)));
};

template <bool BF, bool AL>
__device__ __forceinline__ void load8(float (&v)[8], const uint8_t* row, int64_t k) {
  typedef typename Wide<AL ? 16 : BF ? 2 : 4>::type W;
  if constexpr (BF) {
    const W a = *reinterpret_cast<const W*>(row + 2 * k);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e & 1 ? __uint_as_float((uint32_t)a[e / 2] & 0xffff0000u) : bf16_f32((uint32_t)a[e / 2] & 0xffffu);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const W a = *reinterpret_cast<const W*>(row + 4 * k + 16 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * h + e] = __int_as_float(a[e]);
    }
  }
}

template <bool BF>
__device__ __forceinline__ float load1(const uint8_t* row, int64_t k) {
  if constexpr (BF)
    return bf16_f32(reinterpret_cast<const uint16_t*>(row)[k]);
  else
    return reinterpret_cast<const float*>(row)[k];
}

template <bool BF>
__device__ __forceinline__ void store1(float v, uint8_t* row, int64_t k) {
  if constexpr (BF)
    reinterpret_cast<uint16_t*>(row)[k] = (uint16_t)f32_bf16(v);
  else
    reinterpret_cast<float*>(row)[k] = v;
}

// A piece's elements from column k (of eight) on to a row: all of them, or those from element
// `from` on.
template <bool BF, bool AL>
__device__ __forceinline__ void store8(const float (&v)[8], uint8_t* row, int64_t k, int from) {
  typedef typename Wide<AL ? 16 : BF ? 2 : 4>::type W;
  if (from == 0) {
    if constexpr (BF) {
      W a;
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = (int)(f32_bf16(v[2 * e]) | (f32_bf16(v[2 * e + 1]) << 16));
      *reinterpret_cast<W*>(row + 2 * k) = a;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<W*>(row + 4 * k + 16 * h) =
            (W){__float_as_int(v[4 * h]), __float_as_int(v[4 * h + 1]), __float_as_int(v[4 * h + 2]), __float_as_int(v[4 * h + 3])};
    }
  } else if constexpr (!AL) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= from) store1<BF>(v[e], row, k + e);
  }
}

template <bool AL>
__device__ __forceinline__ void weights8(float (&v)[8], const uint8_t* w, int bf, int64_t k) {
  if (!w) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 1.0f;
  } else if (bf) {
    load8<true, AL>(v, w, k);
  } else {
    load8<false, AL>(v, w, k);
  }
}

__device__ __forceinline__ float weight1(const uint8_t* w, int bf, int64_t k) {
  return !w ? 1.0f : bf ? load1<true>(w, k) : load1<false>(w, k);
}

// v / s for one s and many v, correctly rounded as the division that spense_quantize_fp8 takes, so
// that the codes are its codes: from y = 1 / s correctly rounded, two steps of Markstein's correction
// (q + y (v - q s) with exact remainders: the first quotient within an ulp, the second correct), five
// operations against the division's ten and a reciprocal.  Holds while no remainder underflows: scales
// outside [2^-60, 2^60] divide; a v below 2^-40 s may be off in its last bits and is a zero code
// either way, whose sign is v's.  FEW: a thread has too few elements for that to pay (one piece: M = 1,
// K = 5120 4.8 us against 5.1; two, M = 8192 95.8 against 93.6 with the correction).
template <bool FEW>
struct Divisor {
  float s, y;
  bool plain;
  __device__ __forceinline__ explicit Divisor(float s_)
      : s(s_), y(FEW ? 0.0f : 1.0f / s_), plain(FEW || !(s_ >= 0x1p-60f && s_ <= 0x1p60f)) {}
  __device__ __forceinline__ float of(float v) const {
    float q = v * y;
    q = __builtin_fmaf(__builtin_fmaf(-q, s, v), y, q);
    q = __builtin_fmaf(__builtin_fmaf(-q, s, v), y, q);
    return __builtin_copysignf(q, v);
  }
};

template <typename D>
__device__ __forceinline__ uint8_t code1(float v, const D& d) {
  return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(d.plain ? v / d.s : d.of(v), 0.0f, 0, false);
}

template <bool AL, typename D>
__device__ __forceinline__ void codes8(const float (&v)[8], const D& d, uint8_t* q, int64_t k, int from) {
  typedef typename Codes<AL>::type W;
  if (from == 0) {
    float t[8];
    if (d.plain) {
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = v[e] / d.s;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = d.of(v[e]);
    }
    W w;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(t[4 * h + 2], t[4 * h + 3],
                                             __builtin_amdgcn_cvt_pk_fp8_f32(t[4 * h], t[4 * h + 1], 0, false), true);
    *reinterpret_cast<W*>(q + k) = w;
  } else if constexpr (!AL) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= from) q[k + e] = code1(v[e], d);
  }
}

// Sum or maximum over L lanes (a power of two up to 64), or with L = 0 over the workgroup; `red`
// (16 floats) is used by one reduction only, so one barrier is enough.
template <bool MAX, int L = 0>
__device__ __forceinline__ float row_reduce(float v, float* red) {
#pragma unroll
  for (int o = (L ? L : 64) / 2; o >= 1; o >>= 1) {
    const float u = __shfl_xor(v, o, 64);
    v = MAX ? fmaxf(v, u) : v + u;
  }
  const int nw = blockDim.x >> 6;
  if (L || nw == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = red[0];
  for (int i = 1; i < nw; ++i) s = MAX ? fmaxf(s, red[i]) : s + red[i];
  return s;
}

// Rows of 8 to 8 * NJ * blockDim.x elements, in registers: thread t owns pieces t + j * blockDim.x
// of eight columns.  A ragged last piece is read as the row's last eight columns, its first `from`
// of them (the owner of the piece before has them) left out of the sums and stores; a piece past the
// row has from = 8.  So every load is one wide access and none sits behind a branch.
// L > 0: short rows, L lanes of a wave each, 256 / L rows a workgroup, no barrier.
template <bool XBF, bool YBF, bool AL, int NJ, int MAXT, int L>
__global__ __launch_bounds__(MAXT) void block_norm_kernel(NormArgs a) {
  __shared__ float red[3][16];
  const int64_t m = L ? (int64_t)blockIdx.x * (256 / (L ? L : 1)) + threadIdx.x / (L ? L : 1) : blockIdx.x;
  if (L && m >= a.M) return;
  const int tid = L ? threadIdx.x % (L ? L : 1) : threadIdx.x, nthr = L ? L : blockDim.x;
  const uint8_t* xr = a.x + m * a.ldx_b;
  const float invk = 1.0f / (float)a.K;
  float r[NJ][8], t[NJ][8], g[NJ][8];
  int col[NJ], from[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int k = 8 * (tid + nthr * j), last = (int)a.K - 8;
    col[j] = min(k, last);
    from[j] = AL ? (k < (int)a.K ? 0 : 8) : min(k - col[j], 8);  // AL: K is a multiple of 8
    load8<XBF, AL>(r[j], xr, col[j]);
    if (a.y) load8<YBF, AL>(t[j], a.y + m * a.ldy_b, col[j]);
    if (a.gate) load8<YBF, AL>(g[j], a.gate + m * a.ldg_b, col[j]);
  }
  auto squares = [&](const float (&v)[8], int f) {  // of the piece's own elements
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += AL || e >= f ? v[e] * v[e] : 0.0f;
    return AL && f ? 0.0f : ss;
  };
  if (a.y) {
    if (a.wpost) {
      float ss = 0.0f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) ss += squares(t[j], from[j]);
      const float inv = rsqrtf(row_reduce<false, L>(ss, red[0]) * invk + a.eps);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        float w[8];
        weights8<AL>(w, a.wpost, a.w_bf16, col[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[j][e] = t[j][e] * inv * w[e];
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) r[j][e] = a.alpha * r[j][e] + (a.gate ? g[j][e] * t[j][e] : t[j][e]);
  }
  if (a.r) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) store8<XBF, AL>(r[j], a.r + m * a.ldr_b, col[j], from[j]);
  }
  if (!a.n && !a.q) return;
  float ss = 0.0f;
#pragma unroll
  for (int j = 0; j < NJ; ++j) ss += squares(r[j], from[j]);
  const float inv = rsqrtf(row_reduce<false, L>(ss, red[1]) * invk + a.eps);
  float amax = 0.0f;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    float w[8];
    weights8<AL>(w, a.wpre, a.w_bf16, col[j]);
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      r[j][e] = r[j][e] * inv * w[e];
      if (AL || e >= from[j]) top = fmaxf(top, fabsf(r[j][e]));
    }
    if (!AL || !from[j]) amax = fmaxf(amax, top);
    if (a.n) store8<YBF, AL>(r[j], a.n + m * a.ldn_b, col[j], from[j]);
  }
  if (!a.q) return;
  amax = row_reduce<true, L>(amax, red[2]);
  const float s = amax > 0.0f ? amax / 448.0f : 1.0f;
  if (tid == 0) a.scales[m] = s;
  const Divisor<NJ == 1> d(s);
#pragma unroll
  for (int j = 0; j < NJ; ++j) codes8<AL>(r[j], d, a.q + m * a.ldq, col[j], from[j]);
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
      const float v = load1<YBF>(yr, k);
      ss += v * v;
    }
    inv1 = rsqrtf(row_reduce<false>(ss, red[0]) * invk + a.eps);
  }
  auto residual = [&](int64_t k) {
    const float x = load1<XBF>(xr, k);
    if (!yr) return x;
    float t = load1<YBF>(yr, k);
    if (a.wpost) t = t * inv1 * weight1(a.wpost, a.w_bf16, k);
    return a.alpha * x + (a.gate ? load1<YBF>(a.gate + m * a.ldg_b, k) * t : t);
  };
  float inv = 1.0f, s = 1.0f;
  if (a.n || a.q) {
    float ss = 0.0f;
    for (int64_t k = threadIdx.x; k < a.K; k += blockDim.x) {
      const float r = residual(k);
      ss += r * r;
    }
    inv = rsqrtf(row_reduce<false>(ss, red[1]) * invk + a.eps);
  }
  auto normed = [&](float r, int64_t k) { return r * inv * weight1(a.wpre, a.w_bf16, k); };
  if (a.q) {
    float amax = 0.0f;
    for (int64_t k = threadIdx.x; k < a.K; k += blockDim.x) amax = fmaxf(amax, fabsf(normed(residual(k), k)));
    amax = row_reduce<true>(amax, red[2]);
    s = amax > 0.0f ? amax / 448.0f : 1.0f;
    if (threadIdx.x == 0) a.scales[m] = s;
  }
  const Divisor<true> d(s);
  for (int64_t k = threadIdx.x; k < a.K; k += blockDim.x) {
    const float r = residual(k), n = normed(r, k);
    if (a.r) store1<XBF>(r, a.r + m * a.ldr_b, k);
    if (a.n) store1<YBF>(n, a.n + m * a.ldn_b, k);
    if (a.q) a.q[m * a.ldq + k] = code1(n, d);
  }
}

// From this many rows two pieces a thread instead of one: half the waves a row, so more rows in flight.
// us, one -> two: 600 x 5120 bf16 11.6 -> 8.5, 1024 17.2 -> 13.2, 8192 103 -> 94, 4096 x 8192 76 -> 59;
// below, one row a CU, one piece is faster (256 x 5120 5.7).
constexpr int64_t kManyRows = 512;

// Lanes of a row of up to 512 elements; the most threads a longer row's workgroup can have.
int64_t row_lanes(int64_t K) { return K < 8 ? 1024 : K <= 128 ? 16 : K <= 256 ? 32 : K <= 512 ? 64 : 1024; }

template <bool XBF, bool YBF, bool AL>
hipError_t launch_norm_rows(const NormArgs& a, int64_t M, hipStream_t st) {
  auto launch = [&](auto kernel, int64_t nj) {
    const int64_t threads = ((a.K + 8 * nj - 1) / (8 * nj) + 63) / 64 * 64;
    hipLaunchKernelGGL(kernel, dim3((unsigned)M), dim3((unsigned)threads), 0, st, a);
    return hipGetLastError();
  };
  auto launch_short = [&](auto kernel) {
    const int64_t rows = 256 / row_lanes(a.K);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((M + rows - 1) / rows)), dim3(256), 0, st, a);
    return hipGetLastError();
  };
  if (a.K <= 128) return launch_short(block_norm_kernel<XBF, YBF, AL, 1, 256, 16>);
  if (a.K <= 256) return launch_short(block_norm_kernel<XBF, YBF, AL, 1, 256, 32>);
  if (a.K <= 512) return launch_short(block_norm_kernel<XBF, YBF, AL, 1, 256, 64>);
  if (M >= kManyRows && a.K <= 8192) return launch(block_norm_kernel<XBF, YBF, AL, 2, 512, 0>, 2);
  if (a.K <= 8192) return launch(block_norm_kernel<XBF, YBF, AL, 1, 1024, 0>, 1);
  if (a.K <= 16384) return launch(block_norm_kernel<XBF, YBF, AL, 2, 1024, 0>, 2);
  return launch(block_norm_kernel<XBF, YBF, AL, 4, 1024, 0>, 4);
}

template <bool XBF, bool YBF>
hipError_t launch_norm(const NormArgs& a, int64_t M, bool aligned, hipStream_t st) {
  if (a.K < 8 || a.K > 32768) {
    hipLaunchKernelGGL((block_norm_long_kernel<XBF, YBF>), dim3((unsigned)M), dim3(1024), 0, st, a);
    return hipGetLastError();
  }
  return aligned ? launch_norm_rows<XBF, YBF, true>(a, M, st) : launch_norm_rows<XBF, YBF, false>(a, M, st);
}

}  // namespace
}  // namespace spense

using spense::api_fail;

extern "C" int spense_block_norm(const spense_block_norm_t* p, hipStream_t stream) {
  if (!p) return api_fail(SPENSE_ERR_ARG, "block_norm arguments are NULL");
  const spense_block_norm_t& b = *p;
  auto bad_type = [](int32_t t) { return t != SPENSE_BF16 && t != SPENSE_F32; };
  if (b.M < 0 || b.K < 1 || b.M > INT32_MAX || b.K > INT32_MAX)
    return api_fail(SPENSE_ERR_ARG, "bad M=%lld K=%lld", (long long)b.M, (long long)b.K);
  if (bad_type(b.x_type)) return api_fail(SPENSE_ERR_ARG, "x_type %d is not bf16 or f32", b.x_type);
  if (bad_type(b.y_type)) return api_fail(SPENSE_ERR_ARG, "y_type %d is not bf16 or f32", b.y_type);
  if (bad_type(b.w_type)) return api_fail(SPENSE_ERR_ARG, "w_type %d is not bf16 or f32", b.w_type);
  if (!(b.eps >= 0.0f) || !(b.eps < INFINITY)) return api_fail(SPENSE_ERR_ARG, "eps is negative or not finite");
  if (!b.y && (b.gate || b.post_weight)) return api_fail(SPENSE_ERR_ARG, "a gate or post_weight needs a block output y");
  if ((b.q != nullptr) != (b.scales != nullptr)) return api_fail(SPENSE_ERR_ARG, "q and scales go together");
  if (b.M == 0) return spense::api_ok();
  if (!b.x) return api_fail(SPENSE_ERR_ARG, "x is NULL");
  if (!b.residual && !b.normed && !b.q) return api_fail(SPENSE_ERR_ARG, "no output is asked for");
  if (b.ldx < b.K || (b.y && b.ldy < b.K) || (b.gate && b.ldg != 0 && b.ldg < b.K) || (b.residual && b.ldr < b.K) ||
      (b.normed && b.ldn < b.K) || (b.q && b.ldq < b.K))
    return api_fail(SPENSE_ERR_ARG, "leading dimension below K");
  if (b.residual && (b.residual == b.y || b.residual == b.normed))
    return api_fail(SPENSE_ERR_ARG, "the residual in the place of y or of normed");
  if (b.normed && b.normed == b.x) return api_fail(SPENSE_ERR_ARG, "normed in the place of x");
  // in place, each thread overwrites what it alone has read: with another pitch it would be another row's
  if (b.M > 1 && ((b.residual && b.residual == b.x && b.ldr != b.ldx) || (b.normed && b.normed == b.y && b.ldn != b.ldy)))
    return api_fail(SPENSE_ERR_ARG, "an output in the place of its input must have its leading dimension");
  if (!spense::grid_fits(b.M + 255, spense::row_lanes(b.K))) return api_fail(SPENSE_ERR_ARG, "M=%lld too large for the grid", (long long)b.M);
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
  a.alpha = b.residual_scale, a.eps = b.eps, a.M = b.M, a.K = b.K;
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

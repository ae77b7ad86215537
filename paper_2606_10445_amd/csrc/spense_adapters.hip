// Low-rank adapters of many requests beside a shared projection:
//   Y[m] = base[m] + s_a * B_a (A_a x_m),  a the adapter of token m (none: Y[m] = base[m]),
// A_a R x K and B_a N x R in bf16, tokens grouped by adapter (spense_group_rows).
//
// Two launches.  The first forms V = s_a x_scale (A_a x) for tiles of 16 or 64 tokens of one
// adapter on 16x16x32 bf16 matrix instructions, K cut over the four waves of a workgroup and
// over workgroups; each writes its fp32 partial sums.  The second adds the partials in a fixed
// order, forms B_a V for the tile and adds it to base on the way to Y.
//
// Roundings: fp8 codes and bf16 activations enter the matrix instructions exactly (every
// e4m3fn value is a bf16 value), sums are fp32.  V enters the second product as two bf16
// numbers, hi + lo, 2^-17 of V off at most; the matrix work that doubles is far from the
// bound.  Y is rounded once.
//
// Memory-bound: for prompts by base and Y (6 bytes an output against 2 R multiply-adds), for
// decoding by A and B of the adapters in the batch.
#include "spense_gemm_device.h"
#include "spense_rows_device.h"

namespace spense {
namespace {

struct AdapterArgs {
  const uint8_t* X;
  int64_t ldx_b;
  const float* xs;  // NULL: 1
  const int32_t* order;
  const int32_t* offsets;
  const uint8_t* A;
  const uint8_t* B;
  const float* scale;  // NULL: 1
  const uint8_t* base;
  int64_t ldb_b;
  uint8_t* Y;
  int64_t ldy_b;
  float* part;  // slices x M x R
  int32_t M, K, N, R, count, slices;
  uint32_t x_bytes;
  int32_t vec;       // base and Y rows in aligned pieces of eight
  int32_t in_place;  // base is Y: rows without an adapter are left alone
  int32_t nblocks;   // second launch: workgroups along N
};

typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// Sixteen e4m3fn codes as bf16, in two halves of eight (exact).
__device__ __forceinline__ void codes_to_bf16(v4i c, v4i (&out)[2]) {
  typedef float v2f __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8(c[2 * h + w], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c[2 * h + w], true);
      // the low half of an fp32 that is a bf16 value is zero
      out[h][2 * w] = (int)((__float_as_uint(a[0]) >> 16) | (__float_as_uint(a[1]) & 0xffff0000u));
      out[h][2 * w + 1] = (int)((__float_as_uint(b[0]) >> 16) | (__float_as_uint(b[1]) & 0xffff0000u));
    }
}

__device__ __forceinline__ v4f mma_bf16(v4i a, v4i b, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// V partials of one tile (CT * 16 tokens), RT * 16 ranks from 16 RT * blockIdx.z and one K
// slice.  A step is 64 columns: lane group q takes columns [16 q, 16 q + 16) of both operands
// (a permutation of K inside the step, the same on both sides), which makes a row's step one
// 128-byte line of A.
template <bool FP8, int RT, int CT>
__global__ __launch_bounds__(256) void adapter_shrink_kernel(AdapterArgs a) {
  RowTile t;
  if (!find_tile(a.offsets, a.count, a.M, false, 16 * CT, blockIdx.x, t)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, li = lane & 15, lq = lane >> 4;
  const int r0 = 16 * RT * blockIdx.z;
  const int steps = (a.K + 63) / 64;
  const int s0 = (int)((int64_t)steps * blockIdx.y / a.slices), s1 = (int)((int64_t)steps * (blockIdx.y + 1) / a.slices);
  const __amdgpu_buffer_rsrc_t rx = rsrc(a.X, a.x_bytes),
                               ra = rsrc(a.A + (int64_t)t.group * a.R * a.K * 2, (uint32_t)a.R * (uint32_t)a.K * 2u);
  constexpr int XS = FP8 ? 1 : 2;
  uint32_t xo[CT], ao[RT];
  int row[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int p = t.p0 + 16 * c + li;
    row[c] = p < t.p1 ? a.order[p] : -1;
    if (row[c] >= a.M) row[c] = -1;
    xo[c] = row[c] >= 0 ? (uint32_t)((int64_t)row[c] * a.ldx_b) + 16u * XS * lq : kOOB;
  }
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int i = r0 + 16 * r + li;
    ao[r] = i < a.R ? (uint32_t)i * (uint32_t)a.K * 2u + 32u * lq : kOOB;
  }
  v4f acc[RT][CT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[r][c] = (v4f){0.f, 0.f, 0.f, 0.f};
  for (int s = s0 + wave; s < s1; s += 4) {
    const bool in = 64 * s + 16 * lq < a.K;  // K is a multiple of 32
    v4i av[RT][2], xv[CT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h) av[r][h] = bl16<0>(ra, sel(in, ao[r] == kOOB ? kOOB : ao[r] + 16u * h), 128 * s);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if constexpr (FP8) {
        codes_to_bf16(bl16<0>(rx, sel(in, xo[c]), 64 * s), xv[c]);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) xv[c][h] = bl16<0>(rx, sel(in, xo[c] == kOOB ? kOOB : xo[c] + 16u * h), 128 * s);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[r][c] = mma_bf16(av[r][h], xv[c][h], acc[r][c]);
  }
  xdl_fence();
  // the four waves' sums in LDS, one token tile at a time; wave r' adds rank tile r'
  __shared__ v4f red[4 * RT * 64];
  const float sa = a.scale ? a.scale[t.group] : 1.0f;
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    if (c) __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r) red[(wave * RT + r) * 64 + lane] = acc[r][c];
    __syncthreads();
    if (wave < RT && row[c] >= 0) {
      v4f v = red[wave * 64 + lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) v += red[(w * RT + wave) * 64 + lane];
      const float f = a.xs ? a.xs[row[c]] : 1.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = v[e] * f * sa;
      const int r = r0 + 16 * wave + 4 * lq;
      if (r < a.R)
        *reinterpret_cast<v4f*>(a.part + ((int64_t)blockIdx.y * a.M + t.p0 + 16 * c + li) * a.R + r) = v;
    }
  }
}

template <bool BF>
__device__ __forceinline__ void load8(float (&v)[8], const uint8_t* row, int n) {
  if constexpr (BF) {
    const u4 d = *reinterpret_cast<const u4*>(row + 2 * (int64_t)n);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? d[e / 2] & 0xffff0000u : d[e / 2] << 16);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const v4f d = *reinterpret_cast<const v4f*>(row + 4 * (int64_t)n + 16 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * h + e] = d[e];
    }
  }
}

template <bool BF>
__device__ __forceinline__ void store8(const float (&v)[8], uint8_t* row, int n) {
  if constexpr (BF) {
    u4 d;
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = bf16_bits(v[2 * e]) | (bf16_bits(v[2 * e + 1]) << 16);
    *reinterpret_cast<u4*>(row + 2 * (int64_t)n) = d;
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<v4f*>(row + 4 * (int64_t)n + 16 * h) = (v4f){v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
  }
}

template <bool BF>
__device__ __forceinline__ float load1(const uint8_t* row, int n) {
  return BF ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[n] << 16)
            : reinterpret_cast<const float*>(row)[n];
}

template <bool BF>
__device__ __forceinline__ void store1(float v, uint8_t* row, int n) {
  if constexpr (BF)
    reinterpret_cast<uint16_t*>(row)[n] = (uint16_t)bf16_bits(v);
  else
    reinterpret_cast<float*>(row)[n] = v;
}

// Y for one tile and 32 * 4 * kExpandSteps output columns: wave w takes 32 columns at a time.
// The rows of the two 16-row matrix products of a step are dealt so that lane (token, q) ends
// with eight consecutive outputs, columns 8 q .. 8 q + 7 of the 32.  The product's k index runs
// over hi of all R ranks, then lo of all R; lane group q of instruction j holds ranks 8 (4 j +
// q) mod R on.
constexpr int kExpandSteps = 4;

template <bool BBF, bool YBF, int KS, int CT>
__global__ __launch_bounds__(256) void adapter_expand_kernel(AdapterArgs a) {
  RowTile t;
  if (!find_tile(a.offsets, a.count, a.M, true, 16 * CT, blockIdx.x / a.nblocks, t)) return;
  const bool none = t.group == a.count;
  if (none && a.in_place) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, li = lane & 15, lq = lane >> 4;
  __shared__ v4i vfrag[CT * KS * 64];
  const int rb = a.R / 8;
  if (!none) {
    for (int f = wave; f < CT * KS; f += 4) {
      const int c = f / KS, b = 4 * (f % KS) + lq;  // eight of the 2 R virtual ranks
      const int p = t.p0 + 16 * c + li;
      v4i w = {0, 0, 0, 0};
      if (b < 2 * rb && p < t.p1) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
        for (int s = 0; s < a.slices; ++s) {
          const float* pp = a.part + ((int64_t)s * a.M + p) * a.R + 8 * (b < rb ? b : b - rb);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const v4f d = *reinterpret_cast<const v4f*>(pp + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * h + e] += d[e];
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t hi = bf16_bits(v[e]);
          const float hf = __uint_as_float(hi << 16);
          // what hi leaves; nothing where hi is infinite or NaN
          const uint32_t bits = b < rb ? hi : (fabsf(hf) <= 3.3895314e38f ? bf16_bits(v[e] - hf) : 0u);
          w[e / 2] |= (int)(bits << (16 * (e & 1)));
        }
      }
      vfrag[f * 64 + lane] = w;
    }
    __syncthreads();
  }
  v4i vf[CT][KS];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int j = 0; j < KS; ++j) vf[c][j] = none ? (v4i){0, 0, 0, 0} : vfrag[(c * KS + j) * 64 + lane];
  int row[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int p = t.p0 + 16 * c + li;
    row[c] = p < t.p1 ? a.order[p] : -1;
    if (row[c] >= a.M) row[c] = -1;
  }
  const __amdgpu_buffer_rsrc_t rw =
      rsrc(a.B + (int64_t)(none ? 0 : t.group) * a.N * a.R * 2, none ? 0u : (uint32_t)a.N * (uint32_t)a.R * 2u);
  const int n_wg = (blockIdx.x % a.nblocks) * 128 * kExpandSteps;
#pragma unroll 2
  for (int s = 0; s < kExpandSteps; ++s) {
    const int n0 = n_wg + 32 * (4 * s + wave);
    if (n0 >= a.N) break;
    v4i bw[2][KS];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int n = n0 + 8 * (li >> 2) + 4 * i + (li & 3);
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const int b = 4 * j + lq;
        bw[i][j] = bl16<0>(rw, sel(n < a.N && b < 2 * rb, (uint32_t)n * (uint32_t)a.R * 2u + 16u * (uint32_t)(b < rb ? b : b - rb)));
      }
    }
    const int nq = n0 + 8 * lq;
    const bool whole = a.vec && nq + 8 <= a.N;
    float o[CT][8];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const uint8_t* br = a.base + (int64_t)(row[c] < 0 ? 0 : row[c]) * a.ldb_b;
      if (whole && row[c] >= 0) {
        load8<BBF>(o[c], br, nq);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[c][e] = row[c] >= 0 && nq + e < a.N ? load1<BBF>(br, nq + e) : 0.0f;
      }
    }
    v4f acc[CT][2];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        acc[c][i] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < KS; ++j) acc[c][i] = mma_bf16(bw[i][j], vf[c][j], acc[c][i]);
      }
    xdl_fence();
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if (row[c] < 0) continue;
      uint8_t* yr = a.Y + (int64_t)row[c] * a.ldy_b;
      if (!none) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[c][4 * i + e] += acc[c][i][e];
      }
      if (whole) {
        store8<YBF>(o[c], yr, nq);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (nq + e < a.N) store1<YBF>(o[c][e], yr, nq + e);
      }
    }
  }
}

// Tokens of a tile: 64 where the batch holds many tokens per adapter, so that A and B rows feed
// four matrix instructions a load; 16 where it does not (a tile holds one adapter's tokens).
int tile_tokens(int64_t M, int32_t count, int32_t R) { return R <= 64 && M >= 32 * (int64_t)count && M >= 128 ? 64 : 16; }

// K slices: workgroups for every CU, at least four steps a wave apart from the last.
int k_slices(int64_t M, int32_t count, int64_t K, int32_t R) {
  const int64_t T = tile_tokens(M, count, R), wg = most_tiles(M, count, false, T) * ((R + 63) / 64);
  int64_t s = (512 + wg - 1) / wg;
  const int64_t most = (K + 511) / 512;
  s = s < most ? s : most;
  return (int)(s < 1 ? 1 : s > 16 ? 16 : s);
}

template <bool FP8, int CT>
void launch_shrink(const AdapterArgs& a, int64_t tiles, hipStream_t st) {
  auto go = [&](auto kernel, int rt) {
    const dim3 grid((unsigned)tiles, (unsigned)a.slices, (unsigned)((a.R + 16 * rt - 1) / (16 * rt)));
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
  };
  if (a.R <= 16)
    go(adapter_shrink_kernel<FP8, 1, CT>, 1);
  else if (a.R <= 32)
    go(adapter_shrink_kernel<FP8, 2, CT>, 2);
  else
    go(adapter_shrink_kernel<FP8, 4, CT>, 4);
}

template <bool BBF, bool YBF>
void launch_expand(const AdapterArgs& a, int T, int64_t tiles, hipStream_t st) {
  const dim3 grid((unsigned)(tiles * a.nblocks));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  const int ks = (2 * a.R + 31) / 32;
  if (T == 64) {
    if (ks <= 1)
      go(adapter_expand_kernel<BBF, YBF, 1, 4>);
    else if (ks <= 2)
      go(adapter_expand_kernel<BBF, YBF, 2, 4>);
    else
      go(adapter_expand_kernel<BBF, YBF, 4, 4>);
  } else {
    if (ks <= 1)
      go(adapter_expand_kernel<BBF, YBF, 1, 1>);
    else if (ks <= 2)
      go(adapter_expand_kernel<BBF, YBF, 2, 1>);
    else if (ks <= 4)
      go(adapter_expand_kernel<BBF, YBF, 4, 1>);
    else
      go(adapter_expand_kernel<BBF, YBF, 8, 1>);
  }
}

bool bad_pool(const spense_adapters_t& p) {
  return p.count < 1 || p.count > SPENSE_MAX_GROUPS || p.R < 8 || p.R > 128 || p.R % 8 || p.K < 1 || p.N < 1 ||
         p.K > INT32_MAX || p.N > INT32_MAX || p.K % 32;
}

}  // namespace
}  // namespace spense

using spense::api_fail;

extern "C" {

size_t spense_adapters_workspace_size(int64_t M, const spense_adapters_t* pool) {
  if (!pool || M < 1 || M > INT32_MAX || spense::bad_pool(*pool)) return 0;
  return (size_t)spense::k_slices(M, pool->count, pool->K, pool->R) * (size_t)M * (size_t)pool->R * 4;
}

int spense_add_adapters(const void* X, int32_t x_type, int64_t M, int64_t ldx, const float* x_scale, const int32_t* order,
                        const int32_t* offsets, const spense_adapters_t* pool, const void* base, int32_t base_type,
                        int64_t ldb, void* Y, int64_t ldy, uint32_t out_flags, void* ws, size_t ws_bytes,
                        hipStream_t stream) {
  if (!pool) return api_fail(SPENSE_ERR_ARG, "the pool is NULL");
  const spense_adapters_t& P = *pool;
  if (P.count < 1 || P.count > SPENSE_MAX_GROUPS)
    return api_fail(SPENSE_ERR_ARG, "count=%d outside [1, %d]", P.count, SPENSE_MAX_GROUPS);
  if (P.R < 8 || P.R > 128 || P.R % 8) return api_fail(SPENSE_ERR_ARG, "R=%d is not a multiple of 8 in [8, 128]", P.R);
  if (P.K < 1 || P.N < 1 || P.K > INT32_MAX || P.N > INT32_MAX)
    return api_fail(SPENSE_ERR_ARG, "bad K=%lld N=%lld", (long long)P.K, (long long)P.N);
  if (P.K % 32) return api_fail(SPENSE_ERR_ALIGN, "K=%lld is not a multiple of 32", (long long)P.K);
  if (x_type != SPENSE_FP8_E4M3FN && x_type != SPENSE_BF16) return api_fail(SPENSE_ERR_ARG, "x_type %d is not fp8 or bf16", x_type);
  if (base_type != SPENSE_BF16 && base_type != SPENSE_F32)
    return api_fail(SPENSE_ERR_ARG, "base_type %d is not bf16 or f32", base_type);
  if (out_flags & ~1u) return api_fail(SPENSE_ERR_ARG, "unknown out_flags 0x%x", out_flags);
  if (M < 0 || M > INT32_MAX) return api_fail(SPENSE_ERR_ARG, "bad M");
  if (M == 0) return spense::api_ok();
  if (!X || !order || !offsets || !P.A || !P.B || !base || !Y) return api_fail(SPENSE_ERR_ARG, "NULL pointer");
  if (ldx < P.K || ldb < P.N || ldy < P.N) return api_fail(SPENSE_ERR_ARG, "leading dimension below the row length");
  const int64_t xs = x_type == SPENSE_BF16 ? 2 : 1, bs = base_type == SPENSE_BF16 ? 2 : 4,
                ys = (out_flags & SPENSE_OUT_F32) ? 4 : 2;
  auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if (at(X) % 16 || (ldx * xs) % 16) return api_fail(SPENSE_ERR_ALIGN, "X must be 16-byte aligned with a 16-byte multiple row pitch");
  if (at(P.A) % 16 || at(P.B) % 16) return api_fail(SPENSE_ERR_ALIGN, "A and B must be 16-byte aligned");
  if (at(base) % bs || at(Y) % ys) return api_fail(SPENSE_ERR_ALIGN, "base or Y misaligned");
  const bool same = base == Y;
  if (same && (bs != ys || ldb != ldy)) return api_fail(SPENSE_ERR_ARG, "base in the place of Y must have its type and ldy");
  const int64_t lim = (int64_t)1 << 31;
  const int64_t xb = ((M - 1) * ldx + P.K) * xs;
  if (xb >= lim) return api_fail(SPENSE_ERR_ARG, "X spans 2 GiB or more");
  if (P.K * P.R * 2 >= lim || P.N * P.R * 2 >= lim) return api_fail(SPENSE_ERR_ARG, "an adapter spans 2 GiB or more");
  const int T = spense::tile_tokens(M, P.count, P.R);
  const int64_t nblocks = (P.N + 128 * spense::kExpandSteps - 1) / (128 * spense::kExpandSteps);
  const int64_t tiles = spense::most_tiles(M, P.count, false, T), all_tiles = spense::most_tiles(M, P.count, true, T);
  if (all_tiles * nblocks > INT32_MAX) return api_fail(SPENSE_ERR_ARG, "M x N too large for the grid");
  const size_t need = spense_adapters_workspace_size(M, pool);
  if (!ws || ws_bytes < need) return api_fail(SPENSE_ERR_WS, "workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
  if (at(ws) % 16) return api_fail(SPENSE_ERR_ALIGN, "workspace must be 16-byte aligned");
  int rc = spense::api_check_device();
  if (rc) return rc;
  spense::AdapterArgs a;
  a.X = static_cast<const uint8_t*>(X), a.ldx_b = ldx * xs, a.xs = x_scale;
  a.order = order, a.offsets = offsets;
  a.A = static_cast<const uint8_t*>(P.A), a.B = static_cast<const uint8_t*>(P.B), a.scale = P.scale;
  a.base = static_cast<const uint8_t*>(base), a.ldb_b = ldb * bs;
  a.Y = static_cast<uint8_t*>(Y), a.ldy_b = ldy * ys;
  a.part = static_cast<float*>(ws);
  a.M = (int32_t)M, a.K = (int32_t)P.K, a.N = (int32_t)P.N, a.R = P.R, a.count = P.count;
  a.slices = spense::k_slices(M, P.count, P.K, P.R);
  a.x_bytes = (uint32_t)xb;
  a.vec = at(base) % 16 == 0 && a.ldb_b % 16 == 0 && at(Y) % 16 == 0 && a.ldy_b % 16 == 0;
  a.in_place = same;
  a.nblocks = (int32_t)nblocks;
  if (x_type == SPENSE_FP8_E4M3FN)
    T == 64 ? spense::launch_shrink<true, 4>(a, tiles, stream) : spense::launch_shrink<true, 1>(a, tiles, stream);
  else
    T == 64 ? spense::launch_shrink<false, 4>(a, tiles, stream) : spense::launch_shrink<false, 1>(a, tiles, stream);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    if (bs == 2)
      ys == 2 ? spense::launch_expand<true, true>(a, T, all_tiles, stream) : spense::launch_expand<true, false>(a, T, all_tiles, stream);
    else
      ys == 2 ? spense::launch_expand<false, true>(a, T, all_tiles, stream) : spense::launch_expand<false, false>(a, T, all_tiles, stream);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return api_fail(SPENSE_ERR_HIP, "adapter launch failed: %s", hipGetErrorString(e));
  return spense::api_ok();
}

}  // extern "C"

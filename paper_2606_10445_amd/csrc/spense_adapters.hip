// Low-rank adapters of many requests beside a shared projection:
//   Y[m] = base[m] + s_a * B_a (A_a x_m),  a the adapter of token m (none: Y[m] = base[m]),
// A_a R x K and B_a N x R in bf16, tokens grouped by adapter (spense_group_rows).
//
// Two launches.  The first forms V = s_a x_scale (A_a x) for tiles of 16 or 32 tokens of one
// adapter on 16x16x32 bf16 matrix instructions, K cut over the waves of a workgroup and
// over workgroups; each writes its fp32 partial sums.  The second adds the partials in a fixed
// order, forms B_a V for the tile and adds it to base on the way to Y.
//
// Roundings: fp8 codes and bf16 activations enter the matrix instructions exactly (every
// e4m3fn value is a bf16 value), sums are fp32.  V enters the second product as two bf16
// numbers, hi + lo, 2^-17 of V off at most; the matrix work that doubles is far from the
// bound.  (An infinite entry of B times lo, which may be zero or of the other sign, makes NaN of an
// infinite sum.)  Y is rounded once.
//
// Memory-bound: for prompts by base and Y (6 bytes an output against 2 R multiply-adds), for
// decoding by A and B of the adapters in the batch.
#include <cstdio>

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
  int32_t in_place;  // base is Y: rows without an adapter are left alone
  int32_t nblocks;   // second launch: workgroups along N
  int32_t steps;     // and steps of 128 columns each of them takes
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

// V partials of one tile (16 CT tokens), RT * 16 ranks from 16 RT * blockIdx.z and one K
// slice (1, 2, 4 or 8 of them; workgroups of XCD x = blockIdx.x % 8 all take slice x % slices, so
// that an XCD reads that part of the adapters and activations only).  A step is 64 columns: lane group q
// takes columns [16 q, 16 q + 16) of both operands (a permutation of K inside the step, the same on
// both sides), which makes a row's step one 128-byte line of A.
template <bool FP8, int RT, int CT, int NW>
__global__ __launch_bounds__(64 * NW) void adapter_shrink_kernel(AdapterArgs a) {
  RowTile t;
  const int x = blockIdx.x & 7, slice = x % a.slices;
  if (!find_tile(a.offsets, a.count, a.M, false, 16 * CT, (blockIdx.x >> 3) * (8 / a.slices) + x / a.slices, t)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, li = lane & 15, lq = lane >> 4;
  const int r0 = 16 * RT * blockIdx.z;
  const int steps = (a.K + 63) / 64;
  const int s0 = (int)((int64_t)steps * slice / a.slices), s1 = (int)((int64_t)steps * (slice + 1) / a.slices);
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
  for (int s = s0 + wave; s < s1; s += 2 * NW) {  // two steps' loads in flight
    v4i av[2][RT][2], xv[2][CT][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int su = s + u * NW;
      const bool in = su < s1 && 64 * su + 16 * lq < a.K;  // K is a multiple of 32
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        if constexpr (FP8) {
          xv[u][c][0] = bl16<0>(rx, sel(in, xo[c]), 64 * su);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h) xv[u][c][h] = bl16<0>(rx, sel(in, xo[c] == kOOB ? kOOB : xo[c] + 16u * h), 128 * su);
        }
      }
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) av[u][r][h] = bl16<0>(ra, sel(in, ao[r] == kOOB ? kOOB : ao[r] + 16u * h), 128 * su);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (FP8) {
#pragma unroll
        for (int c = 0; c < CT; ++c) codes_to_bf16(xv[u][c][0], xv[u][c]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int c = 0; c < CT; ++c) acc[r][c] = mma_bf16(av[u][r][h], xv[u][c][h], acc[r][c]);
    }
  }
  xdl_fence();
  // the waves' sums in LDS, one token tile at a time; wave r' adds rank tile r'
  __shared__ v4f red[NW * RT * 64];
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
      for (int w = 1; w < NW; ++w) v += red[(w * RT + wave) * 64 + lane];
      const float f = a.xs ? a.xs[row[c]] : 1.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = v[e] * f * sa;
      const int r = r0 + 16 * wave + 4 * lq;
      if (r < a.R)
        *reinterpret_cast<v4f*>(a.part + ((int64_t)slice * a.M + t.p0 + 16 * c + li) * a.R + r) = v;
    }
  }
}

// Eight consecutive bf16 or fp32 values as they lie in memory, and as fp32.  Wide accesses at the
// alignment of the elements: a row of base or Y may start anywhere.
template <bool BF>
struct Eight {
  v4i d[BF ? 1 : 2];
};

template <bool BF>
__device__ __forceinline__ Eight<BF> load8(const uint8_t* row, int n) {
  Eight<BF> v;
#pragma unroll
  for (int h = 0; h < (BF ? 1 : 2); ++h) v.d[h] = load16u<BF ? 2 : 4>(row + (BF ? 2 : 4) * (int64_t)n + 16 * h);
  return v;
}

template <bool BF>
__device__ __forceinline__ float value(const Eight<BF>& v, int e) {
  if constexpr (BF)
    return __uint_as_float(e & 1 ? (uint32_t)v.d[0][e / 2] & 0xffff0000u : (uint32_t)v.d[0][e / 2] << 16);
  else
    return __int_as_float(v.d[e / 4][e % 4]);
}

template <bool BF>
__device__ __forceinline__ void store8(const float (&v)[8], uint8_t* row, int n) {
  if constexpr (BF) {
    v4i d;
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = (int)(bf16_bits(v[2 * e]) | (bf16_bits(v[2 * e + 1]) << 16));
    store16u<2>(row + 2 * (int64_t)n, d);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      store16u<4>(row + 4 * (int64_t)n + 16 * h, __builtin_bit_cast(v4i, (v4f){v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]}));
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

// Y for one tile and 128 * a.steps output columns: wave w takes 32 columns at a time.
// The rows of the two 16-row matrix products of a step are dealt so that lane (token, q) ends
// with eight consecutive outputs, columns 8 q .. 8 q + 7 of the 32.  The product's k index runs
// over hi of all ranks, then lo: for R <= 16 both in one instruction (lane group q holds eight
// ranks, block q mod R / 8), else lo in the second half of the KS instructions, on the same
// fragments of B.  V's fragments stay in LDS, whose reads hide behind the loads.  A step's B and base are
// requested a step ahead, the first step's before V is there, without branches a lane takes by itself
// (base two steps ahead: no faster).
template <bool BBF, bool YBF, int KS, int CT>
__global__ __launch_bounds__(256) void adapter_expand_kernel(AdapterArgs a) {
  constexpr int KB = KS == 1 ? 1 : KS / 2;  // fragments of B
  RowTile t;
  if (!find_tile(a.offsets, a.count, a.M, true, 16 * CT, blockIdx.x / a.nblocks, t)) return;
  const bool none = t.group == a.count;
  if (none && a.in_place) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, li = lane & 15, lq = lane >> 4;
  __shared__ v4i vfrag[CT * KS * 64];
  const int rb = a.R / 8;
  const __amdgpu_buffer_rsrc_t rw =
      rsrc(a.B + (int64_t)(none ? 0 : t.group) * a.N * a.R * 2, none ? 0u : (uint32_t)a.N * (uint32_t)a.R * 2u);
  const int n_wg = (blockIdx.x % a.nblocks) * 128 * a.steps;
  int row[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int p = t.p0 + 16 * c + li;
    row[c] = p < t.p1 ? a.order[p] : -1;
    if (row[c] >= a.M) row[c] = -1;
  }
  v4i bw[2][KB];
  auto load_b = [&](int s) {
    const int n0 = n_wg + 32 * (4 * s + wave);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int n = n0 + 8 * (li >> 2) + 4 * i + (li & 3);
#pragma unroll
      for (int j = 0; j < KB; ++j) {
        const int b = KS == 1 && lq >= rb ? lq - rb : 4 * j + lq;  // eight ranks
        bw[i][j] = bl16<0>(rw, sel(n < a.N && b < rb, (uint32_t)n * (uint32_t)a.R * 2u + 16u * (uint32_t)b));
      }
    }
  };
  // base of token tile c in step s; tokens there are none of read row 0 and are not written
  auto load_base = [&](int s, int c) {
    return load8<BBF>(a.base + (int64_t)max(row[c], 0) * a.ldb_b, n_wg + 32 * (4 * s + wave) + 8 * lq);
  };
  // whole pieces of eight for every lane of the step (the same for all of the wave)
  auto whole = [&](int s) { return n_wg + 32 * (4 * s + wave) + 32 <= a.N; };
  Eight<BBF> ob[CT];
  load_b(0);
  if (whole(0)) {
#pragma unroll
    for (int c = 0; c < CT; ++c) ob[c] = load_base(0, c);
  }
  // V of the tile: the slices' sums in order, as fragments of hi and lo.  A wave makes fragment pairs u =
  // wave, wave + 4, ... (token tile u / KB, ranks of fragment u % KB), all of a slice's loads requested
  // together; where hi and lo share an instruction one fragment, of which lanes from rb on hold lo.
  {
    constexpr int PAIRS = CT * KB, PW = (PAIRS + 3) / 4;
    float v[PW][8];
    const float* pp[PW];
    bool in[PW];
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int u = wave + 4 * i, c = u / KB, b = KS == 1 && lq >= rb ? lq - rb : 4 * (u % KB) + lq, p = t.p0 + 16 * c + li;
      in[i] = !none && u < PAIRS && b < rb && p < t.p1;
      pp[i] = a.part + (in[i] ? (int64_t)p * a.R + 8 * b : 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
    }
    const int64_t slice = (int64_t)a.M * a.R;
    if (!none && wave < PAIRS) {
#pragma unroll(PW == 1 ? 8 : 2)
      for (int s = 0; s < a.slices; ++s) {
#pragma unroll
        for (int i = 0; i < PW; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const v4f d = *reinterpret_cast<const v4f*>(pp[i] + s * slice + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][4 * h + e] += d[e];
          }
      }
    }
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int u = wave + 4 * i, c = u / KB, j = u % KB;
      if (u >= PAIRS) break;
      v4i hi = {0, 0, 0, 0}, lo = {0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t h = bf16_bits(v[i][e]);
        const float hf = __uint_as_float(h << 16);
        // what hi leaves; nothing where hi is infinite or NaN
        const uint32_t l = fabsf(hf) <= 3.3895314e38f ? bf16_bits(v[i][e] - hf) : 0u;
        hi[e / 2] |= (int)(h << (16 * (e & 1)));
        lo[e / 2] |= (int)(l << (16 * (e & 1)));
      }
      if (!in[i]) hi = lo = (v4i){0, 0, 0, 0};
      if constexpr (KS == 1) {
        vfrag[c * 64 + lane] = lq >= rb ? lo : hi;
      } else {
        vfrag[(c * KS + j) * 64 + lane] = hi;
        vfrag[(c * KS + j + KB) * 64 + lane] = lo;
      }
    }
    __syncthreads();
  }
  for (int s = 0; s < a.steps; ++s) {
    const int n0 = n_wg + 32 * (4 * s + wave), nq = n0 + 8 * lq;
    if (n0 >= a.N) return;
    const bool full = whole(s);
    v4f acc[CT][2];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      acc[c][0] = acc[c][1] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const v4i vf = vfrag[(c * KS + j) * 64 + lane];
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[c][i] = mma_bf16(bw[i][j % KB], vf, acc[c][i]);
      }
    }
    xdl_fence();
    if (s + 1 < a.steps) load_b(s + 1);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      uint8_t* yr = a.Y + (int64_t)row[c] * a.ldy_b;
      if (full) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = none ? value<BBF>(ob[c], e) : value<BBF>(ob[c], e) + acc[c][e / 4][e % 4];
        if (row[c] >= 0) store8<YBF>(o, yr, nq);
      } else if (row[c] >= 0) {  // the ragged end of N
        const uint8_t* br = a.base + (int64_t)row[c] * a.ldb_b;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (nq + e >= a.N) continue;
          const float o = load1<BBF>(br, nq + e);
          store1<YBF>(none ? o : o + acc[c][e / 4][e % 4], yr, nq + e);
        }
      }
    }
    if (s + 1 < a.steps && whole(s + 1)) {
#pragma unroll
      for (int c = 0; c < CT; ++c) ob[c] = load_base(s + 1, c);
    }
  }
}

// Tokens of a tile: 32 where the batch holds many tokens per adapter, so that A and B rows feed several
// matrix instructions a load; 16 where it does not (a tile holds one adapter's tokens).  64 in the second
// launch: M = 2048 in runs of 150, R = 64 52.3 us against 52.6, M = 1000, R = 32, N = 16384 in runs of 100 43.4
// against 44.7, but M = 500, R = 64 in runs of 70 30.0 against 25.6.
int tile_tokens(int64_t M, int32_t count, int32_t R) { return R <= 64 && M >= 32 * (int64_t)count && M >= 128 ? 32 : 16; }

// K slices: a workgroup for every CU (two where tiles are of 16 tokens, each with two rounds of steps or
// more); but every slice is another M x R of partial sums, which each workgroup along N of the second
// launch reads again.  us (both launches and the grouping): M = 2048, R = 64, N = 8192, 80 tiles, 2 / 4
// slices 60.5 / 54.7; M = 4096, R = 64, 132 tiles, 2 / 4 39.0 / 44.5; M = 1000, R = 32, N = 16384, 40 tiles, 4 / 8
// 39.1 / 42.4; tiles of 16 at 8 / 16: M = 64, R = 16, N = 25600 16.8 / 17.3, M = 256, N = 8192 11.8 / 12.8.
int k_slices(int64_t M, int32_t count, int64_t K, int32_t R) {
  const int T = tile_tokens(M, count, R);
  const bool many = T == 32;
  const int64_t wg = most_tiles(M, count, false, T) * ((R + 63) / 64);
  int64_t s = ((many ? 256 : 512) + wg - 1) / wg;
  const int64_t cap = many ? 4 : 8, most = (K + 511) / 512;
  s = s < most ? s : most;
  s = s < cap ? s : cap;
  return s >= 8 ? 8 : s >= 4 ? 4 : s >= 2 ? 2 : 1;
}

template <bool FP8, int CT>
void launch_shrink(const AdapterArgs& a, int64_t tiles, hipStream_t st) {
  constexpr int NW = CT == 2 ? 8 : 4;
  auto go = [&](auto kernel, int rt) {
    const int64_t per = 8 / a.slices;  // tiles of eight workgroups
    const dim3 grid((unsigned)((tiles + per - 1) / per * 8), 1, (unsigned)((a.R + 16 * rt - 1) / (16 * rt)));
    hipLaunchKernelGGL(kernel, grid, dim3(64 * NW), 0, st, a);
  };
  if (a.R <= 16)
    go(adapter_shrink_kernel<FP8, 1, CT, NW>, 1);
  else if (a.R <= 32)
    go(adapter_shrink_kernel<FP8, 2, CT, NW>, 2);
  else
    go(adapter_shrink_kernel<FP8, 4, CT, NW>, 4);
}

template <bool BBF, bool YBF>
void launch_expand(const AdapterArgs& a, int T, int64_t tiles, hipStream_t st) {
  const dim3 grid((unsigned)(tiles * a.nblocks));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a); };
  if (T == 32) {
    if (a.R <= 16)
      go(adapter_expand_kernel<BBF, YBF, 1, 2>);
    else if (a.R <= 32)
      go(adapter_expand_kernel<BBF, YBF, 2, 2>);
    else
      go(adapter_expand_kernel<BBF, YBF, 4, 2>);
  } else {
    if (a.R <= 16)
      go(adapter_expand_kernel<BBF, YBF, 1, 1>);
    else if (a.R <= 32)
      go(adapter_expand_kernel<BBF, YBF, 2, 1>);
    else if (a.R <= 64)
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
  if (!pool || M < 1 || M > SPENSE_MAX_GROUP_ROWS || spense::bad_pool(*pool)) return 0;
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
  if (M < 0 || M > SPENSE_MAX_GROUP_ROWS)
    return api_fail(SPENSE_ERR_ARG, "M=%lld outside [0, %d]", (long long)M, SPENSE_MAX_GROUP_ROWS);
  if (M == 0) return spense::api_ok();
  if (!X || !order || !offsets || !P.A || !P.B || !base || !Y) return api_fail(SPENSE_ERR_ARG, "NULL pointer");
  if (ldx < P.K || ldb < P.N || ldy < P.N) return api_fail(SPENSE_ERR_ARG, "leading dimension below the row length");
  const int64_t xs = x_type == SPENSE_BF16 ? 2 : 1, bs = base_type == SPENSE_BF16 ? 2 : 4,
                ys = (out_flags & SPENSE_OUT_F32) ? 4 : 2;
  auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if (at(X) % 16 || (M > 1 && (ldx * xs) % 16))
    return api_fail(SPENSE_ERR_ALIGN, "X must be 16-byte aligned with a 16-byte multiple row pitch");
  if (at(P.A) % 16 || at(P.B) % 16) return api_fail(SPENSE_ERR_ALIGN, "A and B must be 16-byte aligned");
  if (at(base) % bs || at(Y) % ys) return api_fail(SPENSE_ERR_ALIGN, "base or Y misaligned");
  const bool same = base == Y;
  if (same && (bs != ys || ldb != ldy)) return api_fail(SPENSE_ERR_ARG, "base in the place of Y must have its type and ldy");
  const int64_t lim = (int64_t)1 << 31;
  const int64_t xb = ((M - 1) * ldx + P.K) * xs;
  if (xb >= lim) return api_fail(SPENSE_ERR_ARG, "X spans 2 GiB or more");
  if (P.K * P.R * 2 >= lim || P.N * P.R * 2 >= lim) return api_fail(SPENSE_ERR_ARG, "an adapter spans 2 GiB or more");
  const int T = spense::tile_tokens(M, P.count, P.R);
  const int64_t tiles = spense::most_tiles(M, P.count, false, T), all_tiles = spense::most_tiles(M, P.count, true, T);
  // columns a workgroup: as many of 1024 (512 with tiles of 32), 512 or 256 as leave workgroups enough,
  // their start (the tile, V) then paid less often.  us at 256 / 512 / 1024: M = 64 over 28 adapters, N = 25600
  // 18.9 / 17.3 / 15.4; M = 1 7.9 / 8.6 / 10.0, M = 128 over 8, N = 8192 9.6 / 10.3 / 12.6; M = 2048, N = 8192
  // with the grouping 53.8 / 52.6 / 54.7.
  const int64_t used = P.count < M ? P.count : M, tiles_used = T == 32 ? M / 32 + used / 2 : used;
  int steps = T == 32 ? 4 : 8;
  while (steps > 2 && tiles_used * ((P.N + 128 * steps - 1) / (128 * steps)) < 512) steps /= 2;
  const int64_t nblocks = (P.N + 128 * steps - 1) / (128 * steps);
  if (!spense::grid_fits(all_tiles * nblocks, 256)) return api_fail(SPENSE_ERR_ARG, "M x N too large for the grid");
  const size_t need = spense_adapters_workspace_size(M, pool);
  if (spense::api_log_level() >= 2)
    fprintf(stderr, "spense: adapters M=%lld count=%d R=%d K=%lld N=%lld -> tile_tokens=%d k_slices=%d steps=%d workspace=%zu\n",
            (long long)M, P.count, P.R, (long long)P.K, (long long)P.N, T, spense::k_slices(M, P.count, P.K, P.R), steps, need);
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
  a.in_place = same;
  a.nblocks = (int32_t)nblocks;
  a.steps = steps;
  if (x_type == SPENSE_FP8_E4M3FN)
    T == 32 ? spense::launch_shrink<true, 2>(a, tiles, stream) : spense::launch_shrink<true, 1>(a, tiles, stream);
  else
    T == 32 ? spense::launch_shrink<false, 2>(a, tiles, stream) : spense::launch_shrink<false, 1>(a, tiles, stream);
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

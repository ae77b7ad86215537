// Rows grouped by an index (expert or adapter), and the rows of a token's experts summed back.
//
// Grouping is a stable counting sort in one launch whose workgroups do not wait for each other: a
// workgroup places 1024 (256) consecutive entries, one a thread, and counts the keys of all n for itself
// (those before its entries and those after, with LDS additions: whole numbers, the same in any
// order).  Inside a wave a lane finds the lanes with its key by ballots over the key's bits; its
// rank is the number of lower ones.  The order is the index order, whatever the timing.
//
// Latency-bound at decode sizes (n = 64: 3.7 us); n = 16384 takes 8 us in a row of such launches, 11
// behind a copy of 1 GiB, which leaves idx in no cache, 13 in a pass behind a long product (one workgroup
// walking all entries with ballots 22, its CU's vector instructions the bound), 65536 18, 2^20 0.65 ms:
// the counting grows with n^2 / 1024, so that is the most a call takes.
#include <hip/hip_runtime.h>

#include "spense.h"
#include "spense_internal.h"

namespace spense {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

template <int kGroupThreads>
__global__ __launch_bounds__(kGroupThreads) void group_rows_kernel(const int32_t* __restrict__ idx, int64_t n, int groups,
                                                                   int bits, int32_t* __restrict__ order,
                                                                   int32_t* __restrict__ inverse,
                                                                   int32_t* __restrict__ offsets) {
  constexpr int kGroupWaves = kGroupThreads / 64;
  constexpr int kKeys = SPENSE_MAX_GROUPS + 1;  // the groups and one for entries outside them
  __shared__ int before[kKeys], after[kKeys];   // entries with each key before this workgroup's, and from there on
  __shared__ uint16_t cnt[kGroupWaves][kKeys];  // this workgroup's, by wave
  __shared__ int wsum[kGroupWaves], carry;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t mine = (int64_t)blockIdx.x * kGroupThreads + threadIdx.x, start = (int64_t)blockIdx.x * kGroupThreads;
  for (int g = threadIdx.x; g <= groups; g += kGroupThreads) {
    before[g] = after[g] = 0;
#pragma unroll
    for (int w = 0; w < kGroupWaves; ++w) cnt[w][g] = 0;
  }
  if (threadIdx.x == 0) carry = 0;
  auto key_of = [&](int64_t i) {
    const int v = idx[i];
    return v >= 0 && v < groups ? v : groups;
  };
  const bool in = mine < n;
  const int key = in ? key_of(mine) : groups;
  __syncthreads();
  constexpr int kBatch = 8;  // loads in flight
  for (int64_t i = threadIdx.x; i - threadIdx.x < n; i += kBatch * kGroupThreads) {
    int k[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) k[u] = i + u * kGroupThreads < n ? key_of(i + u * kGroupThreads) : -1;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      int* const part = i - lane + u * kGroupThreads < start ? before : after;  // a wave's entries are all on one side
      const int one = __builtin_amdgcn_readfirstlane(k[u]);
      if (__ballot(k[u] == one) == ~0ull) {  // one key in the whole wave: one addition
        if (one >= 0 && lane == 0) atomicAdd(&part[one], 64);
      } else if (k[u] >= 0) {
        atomicAdd(&part[k[u]], 1);
      }
    }
  }
  // lanes of this wave with this lane's key (its own included); all lanes take part
  uint64_t peers = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((key >> b) & 1);
    peers &= (key >> b) & 1 ? set : ~set;
  }
  const uint64_t lower = peers & ((1ull << lane) - 1);
  if (in && !lower) cnt[wave][key] = (uint16_t)__popcll(peers);
  __syncthreads();
  // before[g]: this workgroup's first position of key g; cnt: of each wave's first, from there
  for (int g0 = 0; g0 <= groups; g0 += kGroupThreads) {
    const int g = g0 + threadIdx.x;
    const int tot = g <= groups ? before[g] + after[g] : 0;
    int inc = tot;  // inclusive prefix over the keys
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(inc, o, 64);
      if (lane >= o) inc += u;
    }
    if (lane == 63) wsum[wave] = inc;
    __syncthreads();
    int base = carry + inc - tot;
    for (int w = 0; w < wave; ++w) base += wsum[w];
    __syncthreads();
    if (threadIdx.x == kGroupThreads - 1) carry = base + tot;
    if (g <= groups) {
      if (blockIdx.x == 0) offsets[g] = base;
      before[g] += base;
      int sum = 0;
#pragma unroll
      for (int w = 0; w < kGroupWaves; ++w) {
        const int c = cnt[w][g];
        cnt[w][g] = (uint16_t)sum;
        sum += c;
      }
    }
    __syncthreads();
  }
  if (in) {
    const int p = before[key] + cnt[wave][key] + __popcll(lower);
    order[p] = (int32_t)mine;
    if (inverse) inverse[mine] = key < groups ? p : -1;
  }
}

// Y[t] = sum_j w[t, j] * D[inverse[t * top + j]] in fp32, j ascending; entries without a row
// (-1, or outside [0, n)) add nothing.  A workgroup takes 256 * E columns of a token.
template <bool DBF, bool YBF, int E>
__global__ __launch_bounds__(256) void combine_rows_kernel(const uint8_t* __restrict__ D, int64_t ldd_b, int64_t n,
                                                           const int32_t* __restrict__ inverse, const float* __restrict__ w,
                                                           int top, int64_t N, uint8_t* __restrict__ Y, int64_t ldy_b,
                                                           int blocks) {
  const int64_t t = blockIdx.x / blocks;
  const int64_t c = ((int64_t)(blockIdx.x % blocks) * 256 + threadIdx.x) * E;
  if (c >= N) return;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
  for (int j = 0; j < top; ++j) {
    const int p = inverse[t * top + j];
    if (p < 0 || p >= n) continue;
    const float wj = w ? w[t * top + j] : 1.0f;
    const uint8_t* row = D + (int64_t)p * ldd_b;
    float v[E];
    if constexpr (E == 1) {
      v[0] = DBF ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[c] << 16)
                 : reinterpret_cast<const float*>(row)[c];
    } else if constexpr (DBF) {
      typedef uint32_t u2 __attribute__((ext_vector_type(2)));
      const u2 d = *reinterpret_cast<const u2*>(row + 2 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(e & 1 ? d[e / 2] & 0xffff0000u : d[e / 2] << 16);
    } else {
      const v4f d = *reinterpret_cast<const v4f*>(row + 4 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = d[e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = __builtin_fmaf(wj, v[e], acc[e]);
  }
  uint8_t* yr = Y + t * ldy_b;
  auto bf = [](float f) {
    __bf16 h = (__bf16)f;
    return (uint32_t)__builtin_bit_cast(uint16_t, h);
  };
  if constexpr (E == 1) {
    if constexpr (YBF)
      reinterpret_cast<uint16_t*>(yr)[c] = (uint16_t)bf(acc[0]);
    else
      reinterpret_cast<float*>(yr)[c] = acc[0];
  } else if constexpr (YBF) {
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    *reinterpret_cast<u2*>(yr + 2 * c) = (u2){bf(acc[0]) | (bf(acc[1]) << 16), bf(acc[2]) | (bf(acc[3]) << 16)};
  } else {
    *reinterpret_cast<v4f*>(yr + 4 * c) = (v4f){acc[0], acc[1], acc[2], acc[3]};
  }
}

template <bool DBF, bool YBF>
hipError_t launch_combine(const uint8_t* D, int64_t ldd_b, int64_t n, const int32_t* inverse, const float* w, int64_t T,
                          int top, int64_t N, uint8_t* Y, int64_t ldy_b, bool vec, hipStream_t st) {
  const int64_t per = vec ? 1024 : 256, blocks = (N + per - 1) / per;
  const dim3 grid((unsigned)(T * blocks));
  if (vec)
    hipLaunchKernelGGL((combine_rows_kernel<DBF, YBF, 4>), grid, dim3(256), 0, st, D, ldd_b, n, inverse, w, top, N, Y, ldy_b,
                       (int)blocks);
  else
    hipLaunchKernelGGL((combine_rows_kernel<DBF, YBF, 1>), grid, dim3(256), 0, st, D, ldd_b, n, inverse, w, top, N, Y, ldy_b,
                       (int)blocks);
  return hipGetLastError();
}

}  // namespace
}  // namespace spense

using spense::api_fail;

extern "C" {

int spense_group_rows(const int32_t* idx, int64_t n, int32_t groups, int32_t* order, int32_t* inverse, int32_t* offsets,
                      hipStream_t stream) {
  if (n < 0 || n > SPENSE_MAX_GROUP_ROWS)
    return api_fail(SPENSE_ERR_ARG, "n=%lld outside [0, %d]", (long long)n, SPENSE_MAX_GROUP_ROWS);
  if (groups < 1 || groups > SPENSE_MAX_GROUPS)
    return api_fail(SPENSE_ERR_ARG, "groups=%d outside [1, %d]", groups, SPENSE_MAX_GROUPS);
  if (!offsets || (n > 0 && (!idx || !order))) return api_fail(SPENSE_ERR_ARG, "NULL pointer");
  int rc = spense::api_check_device();
  if (rc) return rc;
  int bits = 1;
  while ((groups >> bits) != 0) ++bits;  // keys 0 .. groups
  if (n <= 256 && groups < 256)
    hipLaunchKernelGGL(spense::group_rows_kernel<256>, dim3(1), dim3(256), 0, stream, idx, n, groups, bits, order, inverse,
                       offsets);
  else
    hipLaunchKernelGGL(spense::group_rows_kernel<1024>, dim3((unsigned)(n > 0 ? (n + 1023) / 1024 : 1)), dim3(1024), 0, stream, idx, n,
                       groups, bits, order, inverse, offsets);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return api_fail(SPENSE_ERR_HIP, "group rows launch failed: %s", hipGetErrorString(e));
  return spense::api_ok();
}

int spense_combine_rows(const void* D, int32_t d_type, int64_t n, int64_t ldd, const int32_t* inverse,
                        const float* weights, int64_t T, int32_t top, int64_t N, void* Y, int64_t ldy, uint32_t out_flags,
                        hipStream_t stream) {
  if (d_type != SPENSE_BF16 && d_type != SPENSE_F32) return api_fail(SPENSE_ERR_ARG, "d_type %d is not bf16 or f32", d_type);
  if (n < 0 || T < 0 || N < 0 || top < 1 || n > SPENSE_MAX_GROUP_ROWS || T > SPENSE_MAX_GROUP_ROWS || N > INT32_MAX ||
      T * top > SPENSE_MAX_GROUP_ROWS)
    return api_fail(SPENSE_ERR_ARG, "bad n=%lld T=%lld top=%d N=%lld", (long long)n, (long long)T, top, (long long)N);
  if (out_flags & ~1u) return api_fail(SPENSE_ERR_ARG, "unknown out_flags 0x%x", out_flags);
  if (T == 0 || N == 0) return spense::api_ok();
  if ((n > 0 && !D) || !inverse || !Y) return api_fail(SPENSE_ERR_ARG, "NULL pointer");
  if ((n > 0 && ldd < N) || ldy < N) return api_fail(SPENSE_ERR_ARG, "leading dimension below N");
  const int64_t ds = d_type == SPENSE_BF16 ? 2 : 4, ys = (out_flags & SPENSE_OUT_F32) ? 4 : 2;
  const uintptr_t dp = reinterpret_cast<uintptr_t>(D), yp = reinterpret_cast<uintptr_t>(Y);
  if (dp % ds || yp % ys) return api_fail(SPENSE_ERR_ALIGN, "D or Y misaligned");
  if (D == Y) return api_fail(SPENSE_ERR_ARG, "Y in the place of D");
  if (!spense::grid_fits(T * ((N + 255) / 256), 256)) return api_fail(SPENSE_ERR_ARG, "T x N too large for the grid");
  int rc = spense::api_check_device();
  if (rc) return rc;
  // four columns a thread where D's and Y's quads are aligned
  const bool vec = N % 4 == 0 && dp % (4 * ds) == 0 && ldd % 4 == 0 && yp % (4 * ys) == 0 && ldy % 4 == 0;
  const uint8_t* d8 = static_cast<const uint8_t*>(D);
  uint8_t* y8 = static_cast<uint8_t*>(Y);
  const bool db = d_type == SPENSE_BF16, yb = ys == 2;
  auto go = [&](auto f) { return f(d8, ldd * ds, n, inverse, weights, T, top, N, y8, ldy * ys, vec, stream); };
  const hipError_t e = db ? (yb ? go(spense::launch_combine<true, true>) : go(spense::launch_combine<true, false>))
                          : (yb ? go(spense::launch_combine<false, true>) : go(spense::launch_combine<false, false>));
  if (e != hipSuccess) return api_fail(SPENSE_ERR_HIP, "combine launch failed: %s", hipGetErrorString(e));
  return spense::api_ok();
}

}  // extern "C"

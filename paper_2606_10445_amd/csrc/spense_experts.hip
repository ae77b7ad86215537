// Products grouped by expert on Spense weights: Y[p] = X[row(p)] W_e^T for the positions p of
// expert e (spense_group_rows), ragged groups of any size, one or two weights per expert (gate
// and up) in one launch.  Nothing of the grouping is read on the host.
//
// Few rows an expert (decoding): the weights of the experts that got rows are the traffic, 0.625
// byte a 2:4 entry and one a dense entry.  experts_rows_kernel streams them once per tile of 16 or
// 32 positions: a wave owns 16 weight rows over all of K and keeps three chunks of 512 columns in
// registers ahead of the one in its matrix instructions; the tile's activations, gathered row by row,
// go through LDS a chunk at a time, shared by the workgroup's waves.  64 experts of 1536 x 5120, gate
// and up, 256 rows that 56 of them get: 633 MB of weights in 95 us, 6.7 TB/s, where a plain read reaches
// 7.0.  experts_stream_kernel does the same for a short K, in tiles of up to 64 positions.  Both read whole
// chunks of 512 columns, padding included: 1.45 times the kept bytes where K = 1408 is 1056 2:4 and 352 dense.
// Many rows: the 128 x 128 and 256 x 256 kernels over tiles of positions (spense_gemm_mid.hip,
// spense_gemm_big2.hip).
#include <cstdio>
#include <cstring>

#include "spense_gemm_device.h"
#include "spense_rows_device.h"

namespace spense {
namespace {

// A region of one weight as the row-split kernel sees it: its 16-row tiles from `tile0` on.
struct ExpertRegion {
  int32_t tile0, row0, rows, mat;
  int32_t n_sp, n_de;  // chunks of 512 columns, 2:4 then dense
  int32_t wg0;         // experts_stream_kernel: its first workgroup
};

struct ExpertArgs {
  const uint8_t* X;
  int64_t ldx_b;
  uint32_t x_bytes;
  const float* sx;
  int32_t K, kbound;  // kbound: the first dense column of an input-split weight, 0 of an output-split one
  int32_t out_f32;
  int32_t tiles, wgs;  // 16-row tiles of all regions, workgroups of a tile of positions
  int32_t tiles_wave;  // experts_stream_kernel: row tiles of a wave
  int32_t nreg;
  ExpertRegion reg[4];
  MatDesc mat[2];
};

template <int CT, int WV>
__global__ __launch_bounds__(64 * WV) void experts_rows_kernel(ExpertArgs a, ExpertRows er) {
  typedef XTile<kFP8, CT> XT;
  constexpr int NS = 4, D = NS - 1, P = CT == 1 ? 4 : 1;
  constexpr int KC = XT::CHUNK_K, XI = XT::BYTES / 1024 / WV, NL = 9;  // loads a chunk: activations, weights
  static_assert(XI >= 1 && XI * 1024 * WV == XT::BYTES, "an activation chunk splits evenly over the waves");
  RowTile t;
  if (!find_tile(er.offsets, er.count, er.n, false, 16 * CT, blockIdx.x / a.wgs, t)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, li = lane & 15, lq = lane >> 4;
  const int tile = (blockIdx.x % a.wgs) * WV + wave;
  const bool active = tile < a.tiles;
  int ri = 0;
  for (int i = 1; i < a.nreg; ++i)
    if (tile >= a.reg[i].tile0) ri = i;
  const ExpertRegion& R = a.reg[ri];
  const MatDesc& MD = a.mat[R.mat];
  const int rt = tile - R.tile0, nbase = R.row0 + 16 * rt, rowend = R.row0 + R.rows;
  const int64_t e = t.group;
  __shared__ __attribute__((aligned(1024))) uint8_t xbuf[NS][XT::BYTES];
  const __amdgpu_buffer_rsrc_t rx = rsrc(a.X, a.x_bytes), rv = rsrc(MD.values + e * MD.v_bytes, MD.v_bytes),
                               rm = rsrc(reinterpret_cast<const uint8_t*>(MD.meta) + e * MD.m_bytes, MD.m_bytes),
                               rd = rsrc(MD.dense + e * MD.d_bytes, MD.d_bytes);
  // this lane's 16 bytes of each activation block it copies: tile row and column, swizzled as XTile says
  uint32_t xo[XI];
#pragma unroll
  for (int i = 0; i < XI; ++i) {
    const int byte = (wave * XI + i) * 1024 + 16 * lane, r = byte / XT::ROW_B, b = ((byte % XT::ROW_B) >> 4) ^ (r & 31);
    const int src = t.p0 + r < t.p1 ? source_row(er, t.p0 + r) : -1;
    xo[i] = src >= 0 ? (uint32_t)((int64_t)src * a.ldx_b) + 16u * b : kOOB;
  }
  // the output's scales, requested before any weight
  EpiScales<1, CT> es;
  if (active) {
    epi_scales(es, MD.sw ? MD.sw + e * er.N : nullptr, nullptr, er.n, nbase + 4 * lq, t.p0 + li, rowend);
    source_scales<CT>(es.x, er, a.sx, t.p0 + li, t.p1);
  }
  v4f acc[1][CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) acc[0][c] = (v4f){0.f, 0.f, 0.f, 0.f};

  // chunks of the workgroup: [0, kbound) then [kbound, K), 512 columns each; an output-split
  // region is of one kind over all of them
  const int nb = (a.kbound + KC - 1) / KC, chunks = nb + (a.K - a.kbound + KC - 1) / KC;
  const uint32_t vt = (uint32_t)rt * (uint32_t)R.n_sp * 4096u + 16u * lane, mt = (uint32_t)rt * (uint32_t)R.n_sp * 1024u + 16u * lane,
                 dt = (uint32_t)rt * (uint32_t)R.n_de * 8192u + 16u * lane;
  auto load = [&](WChunk& W, int c) {
    load_chunk_tiled(W, c < R.n_sp, c < chunks, c, max(c - R.n_sp, 0), vt, mt, dt, rv, rm, rd);
  };
  auto xload = [&](int buf, int c) {
    const int kc = c < nb ? c * KC : a.kbound + (c - nb) * KC, ke = c >= chunks ? -1 : c < nb ? a.kbound : a.K;
#pragma unroll
    for (int i = 0; i < XI; ++i) {
      const int byte = (wave * XI + i) * 1024 + 16 * lane, r = byte / XT::ROW_B, b = ((byte % XT::ROW_B) >> 4) ^ (r & 31);
      lds_load16<0>(rx, xbuf[buf] + (wave * XI + i) * 1024, kc + 16 * b < ke ? xo[i] : kOOB, max(kc, 0));
    }
  };
  // the pipeline of spense_gemm_rows_kernel: chunk c + D requested in step c, the barrier after
  // it waits for the activations of chunk c + 1 only
  auto run = [&](auto act_const) {
    constexpr bool ACT = decltype(act_const)::value;
    constexpr int AFTER = ACT ? NL + (D - 1) * (XI + NL) : (D - 1) * XI;
    WChunk slot[NS][1];
#pragma unroll
    for (int d = 0; d < D; ++d) {
      xload(d, d);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (ACT) load(slot[d][0], d);
      __builtin_amdgcn_sched_barrier(0);
    }
    barrier_vm<AFTER>();
    auto step = [&](auto s_const, int c) {
      constexpr int S = decltype(s_const)::value, SD = (S + D) % NS;
      xload(SD, c + D);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (ACT) {
        load(slot[SD][0], c + D);
        __builtin_amdgcn_sched_barrier(0);
        mma_chunk<kFP8, CT, 1, true, P>(acc, slot[S], c < R.n_sp, xbuf[S], li, lq);
        __builtin_amdgcn_sched_barrier(0);
      }
      barrier_vm<AFTER>();
    };
    int c = 0;
    for (; c + NS <= chunks; c += NS) static_for<NS>([&](auto s_const) { step(s_const, c + decltype(s_const)::value); });
    static_for<NS - 1>([&](auto s_const) {
      if (c + decltype(s_const)::value < chunks) step(s_const, c + decltype(s_const)::value);
    });
  };
  if (active)
    run(std::true_type());
  else
    run(std::false_type());
  if (!active) return;
  xdl_fence();
  GemmArgs o;
  o.out_f32 = a.out_f32;
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int p = t.p0 + 16 * c + li, n0 = nbase + 4 * lq;
    if (p < t.p1 && n0 < rowend) store4e(MD.Y, MD.ldy, MD.sw != nullptr, MD.vec_store, o, es, 0, c, acc[0][c], p, n0, rowend);
  }
}

// Where a tile's activations fit LDS whole (16 CT rows x K): copied once behind one barrier, after
// which each wave streams the weights of its row tiles (`tiles_wave` of them, WV apart) on its
// own, the next tile's first chunks requested while the last of this one are multiplied.  The start
// of a workgroup (finding its tile, the activations) is then paid once per WV times tiles_wave row
// tiles, and a short K does not drain the pipeline between them.  A workgroup's row tiles are of one
// region.  Tiles of 16 positions: workgroups of four waves, three of them a CU (8 experts of 5120 x 1536,
// 4 rows each: 11.8 us against 13.9 with eight waves of four register slots); wider tiles: one of eight.
constexpr int kStreamTiles = 8;  // most row tiles of a wave

template <int CT, int WV>
__global__ __launch_bounds__(64 * WV) void experts_stream_kernel(ExpertArgs a, ExpertRows er) {
  typedef XTile<kFP8, CT> XT;
  constexpr int NS = CT == 2 ? 4 : 3, D = NS - 1, P = 1;  // one token tile: three waves a SIMD
  constexpr int KC = XT::CHUNK_K, XI = XT::BYTES / 1024 / WV, NL = 9;
  RowTile t;
  if (!find_tile(er.offsets, er.count, er.n, false, 16 * CT, blockIdx.x / a.wgs, t)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, li = lane & 15, lq = lane >> 4;
  const int wg = blockIdx.x % a.wgs;
  int ri = 0;
  for (int i = 1; i < a.nreg; ++i)
    if (wg >= a.reg[i].wg0) ri = i;
  const ExpertRegion& R = a.reg[ri];
  const MatDesc& MD = a.mat[R.mat];
  const int64_t e = t.group;
  const int tiles = (R.rows + 15) / 16, first = (wg - R.wg0) * WV * a.tiles_wave + wave;  // the wave's row tiles: first, first + WV, ...
  const int mine = min(a.tiles_wave, (tiles - first + WV - 1) / WV);
  const int nb = (a.kbound + KC - 1) / KC, chunks = nb + (a.K - a.kbound + KC - 1) / KC;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  float* const lsw = reinterpret_cast<float*>(lds + chunks * XT::BYTES) + wave * (16 * kStreamTiles);  // scales of the wave's rows
  const __amdgpu_buffer_rsrc_t rx = rsrc(a.X, a.x_bytes), rv = rsrc(MD.values + e * MD.v_bytes, MD.v_bytes),
                               rm = rsrc(reinterpret_cast<const uint8_t*>(MD.meta) + e * MD.m_bytes, MD.m_bytes),
                               rd = rsrc(MD.dense + e * MD.d_bytes, MD.d_bytes),
                               rs = rsrc(MD.sw ? MD.sw + e * er.N : nullptr, MD.sw ? 4u * (uint32_t)er.N : 0u);
  uint32_t xo[XI];
  int col[XI];
#pragma unroll
  for (int i = 0; i < XI; ++i) {
    const int byte = (wave * XI + i) * 1024 + 16 * lane, r = byte / XT::ROW_B;
    col[i] = 16 * (((byte % XT::ROW_B) >> 4) ^ (r & 31));
    const int src = t.p0 + r < t.p1 ? source_row(er, t.p0 + r) : -1;
    xo[i] = src >= 0 ? (uint32_t)((int64_t)src * a.ldx_b) + (uint32_t)col[i] : kOOB;
  }
  float xs[CT];
  source_scales<CT>(xs, er, a.sx, t.p0 + li, t.p1);
  // scales, four row tiles a load: lane l row l % 16 of row tile l / 16
#pragma unroll
  for (int i = 0; i < kStreamTiles / 4; ++i) {
    const int srow = 16 * (first + WV * (4 * i + lq)) + li;
    lds_load4<0>(rs, reinterpret_cast<uint8_t*>(lsw + 64 * i), srow < R.rows ? 4u * (uint32_t)(R.row0 + srow) : kOOB, 0);
  }
  for (int c = 0; c < chunks; ++c) {
    const int kc = c < nb ? c * KC : a.kbound + (c - nb) * KC, ke = c < nb ? a.kbound : a.K;
#pragma unroll
    for (int i = 0; i < XI; ++i)
      lds_load16<0>(rx, lds + c * XT::BYTES + (wave * XI + i) * 1024, kc + col[i] < ke ? xo[i] : kOOB, kc);
  }
  auto run = [&](auto act_const) {
    constexpr bool ACT = decltype(act_const)::value;
    WChunk slot[NS][1];
    // the chunk to request next: chunk lc of the tile at vt, mt, dt
    int lc = 0, left = mine * chunks;
    uint32_t vt = (uint32_t)first * (uint32_t)R.n_sp * 4096u + 16u * lane, mt = (uint32_t)first * (uint32_t)R.n_sp * 1024u + 16u * lane,
             dt = (uint32_t)first * (uint32_t)R.n_de * 8192u + 16u * lane;
    auto load = [&](WChunk& W) {
      load_chunk_tiled(W, lc < R.n_sp, left > 0, lc, max(lc - R.n_sp, 0), vt, mt, dt, rv, rm, rd);
      --left;
      if (++lc == chunks) {
        lc = 0;
        vt += (uint32_t)WV * (uint32_t)R.n_sp * 4096u;
        mt += (uint32_t)WV * (uint32_t)R.n_sp * 1024u;
        dt += (uint32_t)WV * (uint32_t)R.n_de * 8192u;
      }
    };
    if constexpr (ACT) {
#pragma unroll
      for (int d = 0; d < D; ++d) {
        __builtin_amdgcn_sched_barrier(0);
        load(slot[d][0]);
      }
    }
    barrier_vm<ACT ? D * NL : 0>();  // every wave's activations and scales have landed
    if constexpr (ACT) {
      v4f acc[1][CT];
#pragma unroll
      for (int c = 0; c < CT; ++c) acc[0][c] = (v4f){0.f, 0.f, 0.f, 0.f};
      int cc = 0, r = 0;  // the chunk and tile to multiply
      auto step = [&](auto s_const) {
        constexpr int S = decltype(s_const)::value, SD = (S + D) % NS;
        load(slot[SD][0]);
        __builtin_amdgcn_sched_barrier(0);
        mma_chunk<kFP8, CT, 1, true, P>(acc, slot[S], cc < R.n_sp, lds + cc * XT::BYTES, li, lq);
        __builtin_amdgcn_sched_barrier(0);
        if (++cc == chunks) {
          xdl_fence();
          const int n0 = R.row0 + 16 * (first + WV * r) + 4 * lq, rowend = R.row0 + R.rows;
          const v4f w = MD.sw ? *reinterpret_cast<const v4f*>(lsw + 16 * r + 4 * lq) : (v4f){1.f, 1.f, 1.f, 1.f};
          GemmArgs o;
          o.out_f32 = a.out_f32;
#pragma unroll
          for (int c = 0; c < CT; ++c) {
            const int p = t.p0 + 16 * c + li;
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = acc[0][c][q] * w[q] * xs[c];
            if (p < t.p1 && n0 < rowend) put4(MD.Y, MD.ldy, MD.vec_store, o, v, p, n0, rowend);
            acc[0][c] = (v4f){0.f, 0.f, 0.f, 0.f};
          }
          cc = 0;
          ++r;
        }
      };
      int i = mine * chunks;
      for (; i >= NS; i -= NS) static_for<NS>([&](auto s_const) { step(s_const); });
      static_for<NS - 1>([&](auto s_const) {
        if (decltype(s_const)::value < i) step(s_const);
      });
    }
  };
  if (mine > 0)
    run(std::true_type());
  else
    run(std::false_type());
}

template <int CT, int WV>
hipError_t launch_rows(const ExpertArgs& a, const ExpertRows& er, int64_t grid, hipStream_t s) {
  hipLaunchKernelGGL((experts_rows_kernel<CT, WV>), dim3((unsigned)grid), dim3(64 * WV), 0, s, a, er);
  return hipGetLastError();
}

template <int CT, int WV>
hipError_t launch_stream(const ExpertArgs& a, const ExpertRows& er, int64_t grid, int lds, hipStream_t s) {
  const hipError_t e = set_big_lds(experts_stream_kernel<CT, WV>, 0, CT, 160 * 1024);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((experts_stream_kernel<CT, WV>), dim3((unsigned)grid), dim3(64 * WV), lds, s, a, er);
  return hipGetLastError();
}

}  // namespace
}  // namespace spense

using spense::api_fail;

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Kernels of the grouped products.
enum Kernel { kRows16, kRows32, kRows64, kMid, kBig };

// Chunks of 512 columns that experts_stream_kernel takes, beyond which waiting for all activations
// costs more than the pipeline's drains (2048 x 4096, 8 rows an expert: 15.1 us
// against 10.5; 4096 x 2560 22.3 against 23.9; 5120 x 1536 39 against 48).
constexpr int64_t kStreamChunks = 6;

int64_t stream_lds(int64_t chunks, int ct) { return chunks * ct * 8192 + 8 * 16 * spense::kStreamTiles * 4; }
bool streams(int64_t chunks, int ct) { return chunks <= kStreamChunks && stream_lds(chunks, ct) <= 160 * 1024; }

int64_t rows_per_expert(int64_t n, int64_t count) { return n / (count < n ? count : n); }

// Tiles of 256 x 256 rather than 128 x 128: for many rows an expert where the smaller tiles need a
// second round of the 256 CUs.  us at 64 / 96 / 112 / 128 / 256 / 512 rows an expert, 128 x 128 and 256 x
// 256: 32 experts of 1536 x 5120 50 / 54 / 58 / 81 / 117 / 205, 50 / 51 / 52 / 53 / 99 / 142; 32 of 5120 x
// 1536 60 / 67 / 76 / 97 / 157 / 279, 64 / 66 / 67 / 70 / 104 / 179; 10 of 2915 x 2176 (230 of the smaller
// tiles up to 128 rows) 16 / 17 / 18 / 30 / 44 / 72, 21 / 22 / 24 / 25 / 31 / 54.
bool big_tiles(int64_t n, int64_t count, int64_t N, int weights) {
  const int64_t avg = rows_per_expert(n, count), used = count < n ? count : n;
  return avg >= 96 && used * ceil_div(avg, 128) * ceil_div(N, 128) * weights > 256;
}

// The kernel for n rows in count groups: by the rows an expert gets on average where they spread
// evenly (the counts themselves are on the device).  A tile that an expert's rows do not fit costs its
// weights again, a wider one little, and less with the activations in LDS.  us at 8 / 12 / 20 / 32 /
// 40 rows an expert, tiles of 16, 32, 64: 32 experts of 5120 x 1536 39 / 58 / 61 / 81 / 102, 41 / 41
// / 43 / 67 / 71, 42 / 43 / 44 / 48 / 50 (128 x 128: 53 at 32, 55 at 48 against 51); 32 of 1536 x 5120 at
// 12 / 16 / 24 / 32 / 48 36 / - / - / - / -, 40 / 41 / 45 / 64 / 77, 43 / 44 / 47 / 48 / 51, 128 x 128 - /
// - / 45 / 46 / 46.
Kernel choose_kernel(int64_t n, int64_t count, int64_t N, int weights, int64_t chunks) {
  const int64_t avg = rows_per_expert(n, count);
  if (big_tiles(n, count, N, weights)) return kBig;
  if (avg <= (streams(chunks, 1) ? 8 : 12)) return kRows16;
  if (avg <= (streams(chunks, 2) ? 18 : 24)) return kRows32;
  return avg < 48 && streams(chunks, 4) ? kRows64 : kMid;
}

// One call's checked arguments.
struct Call {
  const uint8_t* X;
  int64_t ldx, xb;
  const float* x_scale;
  spense::ExpertRows er;
  int64_t N, K, db;
  bool in_split;
  int weights;
  spense::MatDesc mat[2];
  struct {
    int64_t row0, rows, kbound;
    int mat;
  } reg[4];
  int nreg;
  bool out_f32;
};

// Validates everything but the outputs and fills c (mat[i].Y and what depends on it excepted).
// c.er.n == 0: nothing to do.
int check_call(Call& c, const void* X, int64_t rows_x, int64_t ldx, const float* x_scale, const int32_t* order, int32_t top,
               const int32_t* offsets, int64_t n, int32_t count, int32_t weights, const spense_packed_t* const* packed,
               const float* const* w_scales) {
  if (weights < 1 || weights > 2) return api_fail(SPENSE_ERR_ARG, "weights=%d outside [1, 2]", weights);
  if (count < 1 || count > SPENSE_MAX_GROUPS)
    return api_fail(SPENSE_ERR_ARG, "count=%d outside [1, %d]", count, SPENSE_MAX_GROUPS);
  if (!packed) return api_fail(SPENSE_ERR_ARG, "NULL array");
  if (n < 0 || n > SPENSE_MAX_GROUP_ROWS || rows_x < 0 || rows_x > INT32_MAX)
    return api_fail(SPENSE_ERR_ARG, "bad n=%lld rows_x=%lld", (long long)n, (long long)rows_x);
  if (top < 1) return api_fail(SPENSE_ERR_ARG, "top=%d", top);
  for (int i = 0; i < weights; ++i) {
    if (!packed[i]) return api_fail(SPENSE_ERR_ARG, "packed[%d] is NULL", i);
    int rc = spense::api_check_packed(packed[i]);
    if (rc) return rc;
    const spense_packed_t& P = *packed[i];
    if (P.dtype != SPENSE_FP8_E4M3FN || P.layout != SPENSE_LAYOUT_TILED)
      return api_fail(SPENSE_ERR_ARG, "experts' weights must be fp8 in the tiled layout");
    if (P.N != packed[0]->N || P.K != packed[0]->K || P.split != packed[0]->split || P.dense_begin != packed[0]->dense_begin)
      return api_fail(SPENSE_ERR_ARG, "the two weights must have one geometry");
  }
  const spense_packed_t& P = *packed[0];
  memset(&c, 0, sizeof c);
  c.N = P.N, c.K = P.K, c.db = P.dense_begin, c.in_split = P.split == SPENSE_SPLIT_INPUT, c.weights = weights;
  if (n == 0 || c.N == 0) return SPENSE_OK;
  if (c.K < 1) return api_fail(SPENSE_ERR_ARG, "K=0");
  if (!X || !offsets) return api_fail(SPENSE_ERR_ARG, "X or offsets is NULL");
  if (ldx < c.K) return api_fail(SPENSE_ERR_ARG, "ldx=%lld < K=%lld", (long long)ldx, (long long)c.K);
  if (reinterpret_cast<uintptr_t>(X) % 16 || (rows_x > 1 && ldx % 16))
    return api_fail(SPENSE_ERR_ALIGN, "X must be 16-byte aligned with a 16-byte multiple row pitch");
  const int64_t lim = (int64_t)1 << 31;
  c.X = static_cast<const uint8_t*>(X), c.ldx = ldx, c.xb = rows_x > 0 ? (rows_x - 1) * ldx + c.K : 0, c.x_scale = x_scale;
  if (c.xb >= lim) return api_fail(SPENSE_ERR_ARG, "X spans 2 GiB or more");
  spense_tiled_layout_t T;
  int rc = spense_tiled_layout(c.N, c.K, P.dtype, P.split, P.dense_begin, &T);
  if (rc) return rc;
  if ((int64_t)T.values_bytes >= lim || (int64_t)T.meta_bytes >= lim || (int64_t)T.dense_bytes >= lim)
    return api_fail(SPENSE_ERR_ARG, "an expert's weight spans 2 GiB or more");
  // regions: the dense rows of every weight first (their workgroups carry more bytes), then the 2:4 rows
  for (int kind = 0; kind < (c.in_split ? 1 : 2); ++kind)
    for (int i = 0; i < weights; ++i) {
      if (c.in_split)
        c.reg[c.nreg++] = {0, c.N, c.db, i};
      else if (kind == 0 && c.N > c.db)
        c.reg[c.nreg++] = {c.db, c.N - c.db, 0, i};
      else if (kind == 1 && c.db > 0)
        c.reg[c.nreg++] = {0, c.db, c.K, i};
    }
  for (int i = 0; i < weights; ++i)
    c.mat[i] = spense::MatDesc{static_cast<const uint8_t*>(packed[i]->values), packed[i]->meta,
                               static_cast<const uint8_t*>(packed[i]->dense), (uint32_t)T.values_bytes,
                               (uint32_t)T.meta_bytes, (uint32_t)T.dense_bytes, nullptr, 0,
                               w_scales ? w_scales[i] : nullptr, 0};
  c.er.order = order, c.er.offsets = offsets, c.er.n = (int32_t)n, c.er.count = count, c.er.top = top;
  c.er.rows_x = (int32_t)rows_x, c.er.N = (int32_t)c.N;
  return SPENSE_OK;
}

void set_output(Call& c, int i, void* Y, int64_t ldy, bool f32) {
  c.out_f32 = f32;
  c.mat[i].Y = Y, c.mat[i].ldy = ldy;
  c.mat[i].vec_store = 1;  // at any alignment of the elements
}

// The dispatch log's line of a launch: positions of a tile, waves of a workgroup, row tiles of a wave, row blocks.
void log_launch(const Call& c, const char* kernel, int positions, int waves, int tiles_wave, int64_t blocks) {
  if (spense::api_log_level() < 2) return;
  fprintf(stderr,
          "spense: experts n=%d count=%d weights=%d N=%lld K=%lld split=%s dense_begin=%lld -> %s positions=%d waves=%d "
          "tiles_wave=%d row_blocks=%lld\n",
          c.er.n, c.er.count, c.weights, (long long)c.N, (long long)c.K, c.in_split ? "input" : "output", (long long)c.db, kernel,
          positions, waves, tiles_wave, (long long)blocks);
}

// A launch of the 128 x 128 or, with `big`, the 256 x 256 kernel; pmax: the gate / up pair, the
// fp32 H to mat[0].Y and its row maxima (pmax_ld of them a row) to pmax.
int launch_tiles(Call& c, bool big, float* pmax, int64_t pmax_ld, hipStream_t stream) {
  spense::GemmArgs g;
  memset(&g, 0, sizeof g);
  g.X = c.X, g.ldx_b = c.ldx, g.x_bytes = (uint32_t)c.xb, g.sx = c.x_scale;
  g.M = c.er.n, g.N = (int32_t)c.N, g.out_f32 = c.out_f32;
  g.tiled = 1, g.tblocks = 1, g.nmat = c.weights;
  g.mat[0] = c.mat[0], g.mat[1] = c.mat[1];
  g.hmax = pmax, g.hmax_ld = (int32_t)pmax_ld;
  const int64_t rows = pmax || !big ? 128 : 256;
  int64_t blocks = 0;
  for (int i = 0; i < c.nreg; ++i) {
    if (pmax && c.reg[i].mat) continue;  // a pair's regions are the gate's
    spense::Region& R = g.reg[g.nreg++];
    R.row0 = (int32_t)c.reg[i].row0, R.rows = (int32_t)c.reg[i].rows;
    R.kbound = (int32_t)c.reg[i].kbound, R.kend = (int32_t)c.K;
    R.dense_row_off = c.in_split ? 0 : (int32_t)c.db, R.dense_col_off = c.in_split ? (int32_t)c.db : 0;
    R.ksplit = 1, R.mat = c.reg[i].mat, R.wg0 = (int32_t)blocks, R.nrb = (int32_t)ceil_div(c.reg[i].rows, rows);
    blocks += R.nrb;
  }
  g.groups = (int32_t)blocks, g.hg0 = g.groups;
  if (!spense::grid_fits(spense::most_tiles(c.er.n, c.er.count, false, big ? 256 : 128) * blocks + 8, big ? 512 : 768))
    return api_fail(SPENSE_ERR_ARG, "n x N too large for the grid");
  log_launch(c, !big ? "128x128" : pmax ? "256x256, gate/up paired" : "256x256", big ? 256 : 128, big ? 8 : 12, 1, blocks);
  int rc = spense::api_check_device();
  if (rc) return rc;
  const hipError_t e = big ? spense::launch_experts_big2(g, c.er, stream) : spense::launch_experts_mid(g, c.er, stream);
  return e == hipSuccess ? SPENSE_OK : api_fail(SPENSE_ERR_HIP, "experts launch failed: %s", hipGetErrorString(e));
}

int launch_few(Call& c, int64_t chunks, int ct, hipStream_t stream) {
  spense::ExpertArgs a;
  memset(&a, 0, sizeof a);
  a.X = c.X, a.ldx_b = c.ldx, a.x_bytes = (uint32_t)c.xb, a.sx = c.x_scale;
  a.K = (int32_t)c.K, a.kbound = c.in_split ? (int32_t)c.db : 0, a.out_f32 = c.out_f32, a.nreg = c.nreg;
  a.mat[0] = c.mat[0], a.mat[1] = c.mat[1];
  int64_t tiles = 0;
  for (int i = 0; i < c.nreg; ++i) {
    a.reg[i] = {(int32_t)tiles, (int32_t)c.reg[i].row0, (int32_t)c.reg[i].rows, c.reg[i].mat,
                (int32_t)ceil_div(c.reg[i].kbound, 512), (int32_t)ceil_div(c.K - c.reg[i].kbound, 512), 0};
    tiles += ceil_div(c.reg[i].rows, 16);
  }
  a.tiles = (int32_t)tiles;
  const int64_t most = spense::most_tiles(c.er.n, c.er.count, false, 16 * ct);
  const int64_t lds = stream_lds(chunks, ct);
  const bool stream_kernel = streams(chunks, ct);
  const int64_t used = c.er.count < c.er.n ? c.er.count : c.er.n, tiles_even = used * ceil_div(c.er.n / used, 16 * ct);
  // Waves a workgroup: eight for wider tiles, four for tiles of 16, or two of them where the fullest CU, of up to
  // 12 waves, then gets fewer.  us at four / two, gate and up of one token's experts: 1 of 1536 x 5120 13.8 / 11.4, 2 14.5 /
  // 11.8, 6 22.4 / 20.1, 8 23.4 / 21.5; as many waves either way: 4 15.6 / 15.9, 10 25.0 / 25.4, 64 experts 99.9
  // / 103.3.
  auto fullest = [&](int64_t w) { return w * ceil_div(tiles_even * ceil_div(tiles, w), 256); };
  const int wv = ct > 1 ? 8 : !stream_kernel && fullest(4) <= 12 && fullest(2) < fullest(4) ? 2 : 4;
  if (stream_kernel) {
    auto wgs = [&](int64_t per) {
      int64_t w = 0;
      for (int i = 0; i < c.nreg; ++i) {
        a.reg[i].wg0 = (int32_t)w;
        w += ceil_div(ceil_div(c.reg[i].rows, 16), wv * per);
      }
      return w;
    };
    // row tiles of a wave: rounds of the workgroups that run at once (three of four waves or one of eight a
    // CU) times a workgroup's time, its start as long as 90 KB of a CU's weights; tiles as even groups give
    const int64_t at_once = 256 * (ct == 1 ? 3 : 1);
    const int64_t step = (ct == 1 ? 192 : 128) * c.K * 23 / 32;  // a CU's bytes for one row tile a wave, a quarter dense
    int64_t best = 0;
    for (int64_t per = 1; per <= spense::kStreamTiles; ++per) {
      const int64_t cost = ceil_div(tiles_even * wgs(per), at_once) * (90000 + per * step);
      if (per == 1 || cost < best) best = cost, a.tiles_wave = (int32_t)per;
    }
    a.wgs = (int32_t)wgs(a.tiles_wave);
  } else {
    a.wgs = (int32_t)ceil_div(tiles, wv);
  }
  const int64_t grid = most * a.wgs;
  if (!spense::grid_fits(grid, 64 * wv)) return api_fail(SPENSE_ERR_ARG, "n x N too large for the grid");
  log_launch(c, stream_kernel ? "stream" : "rows", 16 * ct, wv, stream_kernel ? a.tiles_wave : 1, a.wgs);
  int rc = spense::api_check_device();
  if (rc) return rc;
  const hipError_t e = stream_kernel ? (ct == 1   ? spense::launch_stream<1, 4>(a, c.er, grid, (int)lds, stream)
                                        : ct == 2 ? spense::launch_stream<2, 8>(a, c.er, grid, (int)lds, stream)
                                                  : spense::launch_stream<4, 8>(a, c.er, grid, (int)lds, stream))
                                     : (wv == 2   ? spense::launch_rows<1, 2>(a, c.er, grid, stream)
                                        : wv == 4 ? spense::launch_rows<1, 4>(a, c.er, grid, stream)
                                                  : spense::launch_rows<2, 8>(a, c.er, grid, stream));
  return e == hipSuccess ? SPENSE_OK : api_fail(SPENSE_ERR_HIP, "experts launch failed: %s", hipGetErrorString(e));
}

int launch_products(Call& c, hipStream_t stream) {
  const int64_t kbound = c.in_split ? c.db : 0, chunks = ceil_div(kbound, 512) + ceil_div(c.K - kbound, 512);
  const Kernel k = choose_kernel(c.er.n, c.er.count, c.N, c.weights, chunks);
  if (k >= kMid) return launch_tiles(c, k == kBig, nullptr, 0, stream);
  return launch_few(c, chunks, k == kRows16 ? 1 : k == kRows32 ? 2 : 4, stream);
}

// The workspace of the gate / up pair: H, or G then U, fp32 with rows padded to 64 elements, and
// behind H its row maxima (two per block of 128 weight rows and region).
int64_t glu_ld(int64_t N) { return ceil_div(N, 64) * 64; }
int64_t glu_maxima(int64_t N) { return 2 * (ceil_div(N, 128) + 1); }
int64_t glu_rows_bytes(int64_t n, int64_t N) { return ceil_div(n * glu_ld(N) * 4, 256) * 256; }

}  // namespace

extern "C" {

int spense_gemm_experts(const void* X, int64_t rows_x, int64_t ldx, const float* x_scale, const int32_t* order, int32_t top,
                        const int32_t* offsets, int64_t n, int32_t count, int32_t weights,
                        const spense_packed_t* const* packed, const float* const* w_scales, void* const* Y,
                        const int64_t* ldy, uint32_t out_flags, hipStream_t stream) {
  Call c;
  int rc = check_call(c, X, rows_x, ldx, x_scale, order, top, offsets, n, count, weights, packed, w_scales);
  if (rc) return rc;
  if (!Y || !ldy) return api_fail(SPENSE_ERR_ARG, "NULL array");
  if (out_flags & ~1u) return api_fail(SPENSE_ERR_ARG, "unknown out_flags 0x%x", out_flags);
  if (c.er.n == 0) return spense::api_ok();
  const bool f32 = (out_flags & SPENSE_OUT_F32) != 0;
  for (int i = 0; i < weights; ++i) {
    if (!Y[i] || (i && Y[i] == Y[0])) return api_fail(SPENSE_ERR_ARG, "Y[%d] is NULL or Y[0]", i);
    if (ldy[i] < c.N) return api_fail(SPENSE_ERR_ARG, "ldy[%d] < N", i);
    if (reinterpret_cast<uintptr_t>(Y[i]) % (f32 ? 4 : 2)) return api_fail(SPENSE_ERR_ALIGN, "Y[%d] misaligned", i);
    if (n * ldy[i] > (int64_t)1 << 40) return api_fail(SPENSE_ERR_ARG, "Y[%d] too large", i);
    set_output(c, i, Y[i], ldy[i], f32);
  }
  rc = launch_products(c, stream);
  return rc ? rc : spense::api_ok();
}

size_t spense_gemm_experts_glu_fp8_workspace_size(int64_t n, int32_t count, int64_t N) {
  if (n < 1 || n > SPENSE_MAX_GROUP_ROWS || N < 1 || N > INT32_MAX || count < 1 || count > SPENSE_MAX_GROUPS) return 0;
  if (big_tiles(n, count, N, 2)) return (size_t)(glu_rows_bytes(n, N) + n * glu_maxima(N) * 4);
  return (size_t)(2 * glu_rows_bytes(n, N));
}

int spense_gemm_experts_glu_fp8(const void* X, int64_t rows_x, int64_t ldx, const float* x_scale, const int32_t* order,
                                int32_t top, const int32_t* offsets, int64_t n, int32_t count, const spense_packed_t* gate,
                                const spense_packed_t* up, const float* w_scale_gate, const float* w_scale_up, uint8_t* q,
                                int64_t ldq, float* scales, void* ws, size_t ws_bytes, hipStream_t stream) {
  const spense_packed_t* const packed[2] = {gate, up};
  const float* const w_scales[2] = {w_scale_gate, w_scale_up};
  Call c;
  int rc = check_call(c, X, rows_x, ldx, x_scale, order, top, offsets, n, count, 2, packed, w_scales);
  if (rc) return rc;
  if (c.er.n == 0) return spense::api_ok();
  if (c.in_split) return api_fail(SPENSE_ERR_ARG, "gate and up must be output-split");
  if (!q || !scales) return api_fail(SPENSE_ERR_ARG, "q or scales is NULL");
  if (ldq < c.N) return api_fail(SPENSE_ERR_ARG, "ldq=%lld < N=%lld", (long long)ldq, (long long)c.N);
  const size_t need = spense_gemm_experts_glu_fp8_workspace_size(n, count, c.N);
  if (!ws || ws_bytes < need)
    return api_fail(SPENSE_ERR_WS, "workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : (size_t)0);
  if (reinterpret_cast<uintptr_t>(ws) % 256) return api_fail(SPENSE_ERR_ALIGN, "workspace must be 256-byte aligned");
  if (!spense::grid_fits(n * ceil_div(c.N, 2048), 256)) return api_fail(SPENSE_ERR_ARG, "n x N too large for the quantisation grid");
  const int64_t ld = glu_ld(c.N), half = glu_rows_bytes(n, c.N);
  float* const H = static_cast<float*>(ws);
  float* const second = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + half);
  hipError_t e;
  if (big_tiles(n, count, c.N, 2)) {
    int64_t blocks = 0;
    for (int i = 0; i < c.nreg; ++i)
      if (c.reg[i].mat == 0) blocks += ceil_div(c.reg[i].rows, 128);
    set_output(c, 0, H, ld, true);
    rc = launch_tiles(c, true, second, 2 * blocks, stream);
    if (rc) return rc;
    e = spense::launch_quantize_rowmax(H, ld, n, c.N, second, (int)(2 * blocks), q, ldq, scales, stream);
  } else {
    set_output(c, 0, H, ld, true);
    set_output(c, 1, second, ld, true);
    rc = launch_products(c, stream);
    if (rc) return rc;
    e = spense::launch_glu_quantize(SPENSE_F32, H, ld * 4, second, ld * 4, n, c.N, q, ldq, scales, stream);
  }
  if (e != hipSuccess) return api_fail(SPENSE_ERR_HIP, "experts quantise launch failed: %s", hipGetErrorString(e));
  return spense::api_ok();
}

}  // extern "C"

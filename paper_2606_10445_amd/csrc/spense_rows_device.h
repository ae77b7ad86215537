// Device helper of the kernels that work on rows grouped by an index (spense_group_rows).
#pragma once
#include "spense_internal.h"

namespace spense {
namespace {

// Sixteen bytes at any address that is a multiple of ALIGN (the element's size).
template <int ALIGN>
struct Unaligned16;
template <>
struct Unaligned16<2> {
  typedef int type __attribute__((ext_vector_type(4), aligned(2)));
};
template <>
struct Unaligned16<4> {
  typedef int type __attribute__((ext_vector_type(4), aligned(4)));
};
typedef int rows_v4i __attribute__((ext_vector_type(4)));

template <int ALIGN>
__device__ __forceinline__ rows_v4i load16u(const void* p) {
  return *reinterpret_cast<const typename Unaligned16<ALIGN>::type*>(p);
}
template <int ALIGN>
__device__ __forceinline__ void store16u(void* p, rows_v4i v) {
  *reinterpret_cast<typename Unaligned16<ALIGN>::type*>(p) = v;
}

struct RowTile {
  int group;   // count: the rows of no group
  int p0, p1;  // positions [p0, p1), at most T of them
};

// The tiles of T positions that the groups are cut into, group by group (with `rest`, then those of
// the positions in no group); a tile never spans two groups.  The whole wave makes it with the same
// arguments; each lane counts a contiguous share of the groups, so the search costs one load latency and
// a prefix over the lanes.  Offsets are clamped to [0, n] and to ascend, so a tile lies in [0, n)
// whatever they hold.
struct RowTiles {
  const int32_t* offsets;
  int count, n, groups, per, T;
  int a0, b0, sum, inc;  // the lane's first group, the tiles of its groups, those up to its last
  int total;             // all tiles

  __device__ __forceinline__ int tiles_of(int a, int b) const { return (b - a + T - 1) / T; }
  __device__ __forceinline__ void segment(int e, int& a, int& b) const {
    a = min(max(offsets[e], 0), n);
    b = e < count ? max(min(max(offsets[e + 1], 0), n), a) : n;
  }

  __device__ __forceinline__ RowTiles(const int32_t* offsets_, int count_, int n_, bool rest, int T_)
      : offsets(offsets_), count(count_), n(n_), groups(rest ? count_ + 1 : count_), per((groups + 63) >> 6), T(T_), a0(0), b0(0) {
    const int lane = threadIdx.x & 63;
    if (lane * per < groups) segment(lane * per, a0, b0);
    sum = tiles_of(a0, b0);
    for (int i = 1; i < per; ++i) {
      const int e = lane * per + i;
      if (e < groups) {
        int a, b;
        segment(e, a, b);
        sum += tiles_of(a, b);
      }
    }
    inc = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(inc, o, 64);
      if (lane >= o) inc += u;
    }
    total = __builtin_amdgcn_readlane(inc, 63);
  }

  // Tile g; false past the last one.
  __device__ __forceinline__ bool find(int g, RowTile& out) const {
    if (g >= total) return false;
    const int lane = threadIdx.x & 63;
    const uint64_t mine = __ballot(g >= inc - sum && g < inc);
    int at = g - (inc - sum), e = lane * per, p0 = a0 + at * T, p1 = min(b0, p0 + T);
    bool found = at < tiles_of(a0, b0);
    at -= tiles_of(a0, b0);
    for (int i = 1; i < per; ++i) {
      const int f = lane * per + i;
      if (f < groups && !found) {
        int a, b;
        segment(f, a, b);
        const int tiles = tiles_of(a, b);
        if (at < tiles) {
          e = f, p0 = a + at * T, p1 = min(b, p0 + T);
          found = true;
        }
        at -= tiles;
      }
    }
    const int src = __builtin_ctzll(mine);
    out.group = __builtin_amdgcn_readlane(e, src);
    out.p0 = __builtin_amdgcn_readlane(p0, src);
    out.p1 = __builtin_amdgcn_readlane(p1, src);
    return true;
  }
};

__device__ __forceinline__ bool find_tile(const int32_t* offsets, int count, int n, bool rest, int T, int g, RowTile& out) {
  return RowTiles(offsets, count, n, rest, T).find(g, out);
}

// Tile and row block of workgroup g of a grid of tiles x row blocks: the pairs, tile by tile, in eight
// equal runs, one an XCD (workgroup g is on XCD g % 8), so that a tile's activations and an expert's
// weights are read by one or two XCDs and each has the same number of pairs.  (Row blocks x, x + 8, ... of
// every tile on XCD x read the weights once too, but 10 row blocks left six XCDs half idle: 32 experts'
// gate / up of 1536 rows, 256 rows each, 200 us.)
__device__ __forceinline__ bool find_pair(const ExpertRows& er, int T, int blocks, RowTile& out, int& block) {
  const RowTiles tiles(er.offsets, er.count, er.n, false, T);
  const int64_t pairs = (int64_t)tiles.total * blocks, run = (pairs + 7) / 8;
  const int64_t l = blockIdx.x >> 3, g = (blockIdx.x & 7) * run + l;
  if (l >= run || g >= pairs) return false;
  block = (int)(g % blocks);
  return tiles.find((int)(g / blocks), out);
}

// The activation row of position p < n, -1 where order names none.
__device__ __forceinline__ int source_row(const ExpertRows& er, int p) {
  if (!er.order) return p < er.rows_x ? p : -1;
  const int i = er.order[p];
  const int r = (int)((unsigned)i / (unsigned)er.top);
  return i >= 0 && r < er.rows_x ? r : -1;
}

// The token scales of positions p, p + 16, ... below pend (1 elsewhere and without scales).
template <int CT>
__device__ __forceinline__ void source_scales(float (&x)[CT], const ExpertRows& er, const float* sx, int p, int pend) {
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int src = sx && p + 16 * c < pend ? source_row(er, p + 16 * c) : -1;
    x[c] = src >= 0 ? sx[src] : 1.0f;
  }
}

// The same two for tiles of many positions (p[c] >= 0; -1 from pend on): every entry of order is requested
// before the first is used, without branches around the loads.  Gate and up of 16 experts of 1536 x 5120, 256
// rows each 83.7 -> 79.6 us; where most of a tile is empty the branches that skip it are faster: 56 rows over
// 8 experts 29.4 us against 30.3.
template <int C>
__device__ __forceinline__ void source_rows(const ExpertRows& er, const int (&p)[C], int pend, int (&src)[C]) {
  int i[C];
  unsigned top = 1;
  if (er.order) {
    top = (unsigned)er.top;
#pragma unroll
    for (int c = 0; c < C; ++c) i[c] = er.order[min(p[c], er.n - 1)];
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) i[c] = p[c];
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int r = (int)((unsigned)i[c] / top);
    src[c] = (p[c] < pend) & (i[c] >= 0) & (r < er.rows_x) ? r : -1;
  }
}

template <int CT>
__device__ __forceinline__ void source_rows_scales(float (&x)[CT], const ExpertRows& er, const float* sx, int p, int pend) {
#pragma unroll
  for (int c = 0; c < CT; ++c) x[c] = 1.0f;
  if (!sx || er.rows_x == 0) return;
  int q[CT], src[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) q[c] = p + 16 * c;
  source_rows(er, q, pend, src);
#pragma unroll
  for (int c = 0; c < CT; ++c) x[c] = sx[max(src[c], 0)];
#pragma unroll
  for (int c = 0; c < CT; ++c) x[c] = src[c] >= 0 ? x[c] : 1.0f;
}

// Most tiles that find_tile can give (host).
inline int64_t most_tiles(int64_t n, int64_t count, bool rest, int64_t T) {
  const int64_t groups = count + (rest ? 1 : 0);
  return n / T + (groups < n ? groups : n);
}

}  // namespace
}  // namespace spense

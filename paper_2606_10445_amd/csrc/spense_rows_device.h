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

// Tile g of the tiles of T positions that the groups are cut into, group by group (with
// `rest`, then those of the positions in no group); false past the last one.  A tile never
// spans two groups.  The whole wave calls it with the same arguments; each lane counts a
// contiguous share of the groups, so the search costs one load latency and a prefix over the
// lanes.  Offsets are clamped to [0, n] and to ascend, so a tile lies in [0, n) whatever they hold.
__device__ __forceinline__ bool find_tile(const int32_t* __restrict__ offsets, int count, int n, bool rest, int T, int g,
                                          RowTile& out) {
  const int lane = threadIdx.x & 63;
  const int groups = rest ? count + 1 : count;
  const int per = (groups + 63) >> 6;
  auto segment = [&](int e, int& a, int& b) {
    a = min(max(offsets[e], 0), n);
    b = e < count ? max(min(max(offsets[e + 1], 0), n), a) : n;
  };
  int a0 = 0, b0 = 0, sum = 0;  // the lane's first group; its tiles
  if (lane * per < groups) segment(lane * per, a0, b0);
  sum = (b0 - a0 + T - 1) / T;
  const int first = sum;
  for (int i = 1; i < per; ++i) {
    const int e = lane * per + i;
    if (e < groups) {
      int a, b;
      segment(e, a, b);
      sum += (b - a + T - 1) / T;
    }
  }
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(inc, o, 64);
    if (lane >= o) inc += u;
  }
  const uint64_t mine = __ballot(g >= inc - sum && g < inc);
  if (!mine) return false;
  int at = g - (inc - sum), e = lane * per, p0 = a0 + at * T, p1 = min(b0, p0 + T);
  bool found = at < first;
  at -= first;
  for (int i = 1; i < per; ++i) {
    const int f = lane * per + i;
    if (f < groups && !found) {
      int a, b;
      segment(f, a, b);
      const int tiles = (b - a + T - 1) / T;
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

// Most tiles that find_tile can give (host).
inline int64_t most_tiles(int64_t n, int64_t count, bool rest, int64_t T) {
  const int64_t groups = count + (rest ? 1 : 0);
  return n / T + (groups < n ? groups : n);
}

}  // namespace
}  // namespace spense

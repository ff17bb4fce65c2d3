// Rotary positions and per-head norms of queries and keys (gfx950).
//
// A row holds heads of dh columns side by side.  The rotation turns pairs of a head's first rot
// columns by the angle pos table[i] of their row; the norm divides a head by its root mean square
// and scales it by a gain, before the rotation.
//
// All of this is bound by the rows' traffic (8 bytes a value forward, 12 backward).  An angle
// belongs to a row and a pair, not to a head: a workgroup takes a tile of rows, computes the tile's
// cosines and sines once into LDS and uses them for every head.  Rows whose heads, rotated width and
// length come in fours go in aligned 16-byte loads; of others, the norms take 16 bytes at any
// alignment, the rotation columns.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <initializer_list>

#include "kernels.h"

namespace ooc {

namespace {

constexpr int TPB = 256;

// m cos a and m sin a of a = pos f.  Positions far out need the angle in 64 bits: at a million
// positions an fp32 angle is off by 0.06.  The product is rounded to a double as in the definition,
// a multiple of pi / 2 (in two doubles) taken off, and the rest, within +-pi/4, goes through the
// Taylor series in fp32: the first term left out is below 2e-9.
__device__ inline float2 turn(int32_t pos, double f, float m) {
  const double a = (double)pos * f;
  const double n = rint(a * 0.63661977236758134308);
  double d = fma(n, -1.57079632679489661923, a);
  d = fma(n, -6.12323399573676603587e-17, d);
  const float r = (float)d, r2 = r * r;
  const float s = r + r * r2 * (-1.f / 6 + r2 * (1.f / 120 + r2 * (-1.f / 5040 + r2 * (1.f / 362880))));
  const float c = 1.f + r2 * (-0.5f + r2 * (1.f / 24 + r2 * (-1.f / 720 + r2 * (1.f / 40320 - r2 * (1.f / 3628800)))));
  const int q = (int)((long long)n & 3);
  const float cs = q & 1 ? s : c, sn = q & 1 ? c : s;
  return make_float2(m * (q == 1 || q == 2 ? -cs : cs), m * (q >= 2 ? -sn : sn));
}

// x / d for 0 <= x < 2^31 and an invariant d >= 1 by one multiply-high (Granlund and Montgomery,
// 1994): with l = ceil(log2 d) and m = floor(2^(31 + l) / d) + 1, floor(x m / 2^(31 + l)) is the
// quotient.  d = 1 has l = 0 and would need m = 2^31 + 1 at a shift of -1: it takes m = 2^32 - 1 and
// x + 1.
struct Divisor {
  uint32_t m = 0xffffffffu, shift = 0, add = 1;
  static Divisor of(int d) {
    Divisor r;
    if (d <= 1) return r;
    uint32_t l = 0;
    while ((1u << l) < (uint32_t)d) ++l;
    r.m = (uint32_t)((1ull << (31 + l)) / (uint32_t)d + 1);
    r.shift = l - 1;
    r.add = 0;
    return r;
  }
  __device__ int div(int x) const { return (int)(__umulhi((uint32_t)x + add, m) >> shift); }
};

// What a launch knows of its rows.
struct Rows {
  int64_t rows;
  int cols, dh, heads, used, half, layout;   // used = heads dh, half = rot / 2
  int h1;                                    // heads of the first gain
  int tile;                                  // rows a workgroup takes at once
  Divisor by_half, by_dh, by_heads, by_items, by_rest;
  int items;                                 // of a row: V columns each
  // The norms' squares are of down x, down a power of two with dh down^2 <= 1: their sum is at most
  // the largest square, where a sum of 1024 squares of 1e18 would pass fp32's range.  The factor is
  // exact; squares that vanish below 2^-126 are of no account beside 1e-5.
  float down;
};

// The pairs' (m cos, m sin) of rows r0 .. r0 + n into cs [n][half].
__device__ inline void turns(float2* cs, const int32_t* __restrict__ pos,
                             const double* __restrict__ table, int64_t r0, int n, const Rows& r) {
  const float m = (float)table[r.half];
  for (int t = threadIdx.x; t < n * r.half; t += TPB) {
    const int row = r.by_half.div(t);
    cs[t] = turn(pos[r0 + row], table[t - row * r.half], m);
  }
}

// four neighbouring values, aligned to 16 bytes, or to 4
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
struct Four {
  float v[4];
};
__device__ inline Four load(const float* p) {
  const float4 t = *reinterpret_cast<const float4*>(p);
  Four x;
  x.v[0] = t.x; x.v[1] = t.y; x.v[2] = t.z; x.v[3] = t.w;
  return x;
}
__device__ inline void store(float* p, const Four& x) {
  *reinterpret_cast<float4*>(p) = make_float4(x.v[0], x.v[1], x.v[2], x.v[3]);
}
// The same of a head of which `left` columns remain: four of them aligned to 16 bytes, or (ODD) as
// many as there are, at any alignment, and zeros.
template <bool ODD>
__device__ inline Four load(const float* p, int left) {
  if constexpr (!ODD) {
    return load(p);
  } else {
    Four x;
    if (left >= 4) {
      const float4u t = *reinterpret_cast<const float4u*>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.v[e] = t[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x.v[e] = e < left ? p[e] : 0.f;
    }
    return x;
  }
}
template <bool ODD>
__device__ inline void store(float* p, int left, const Four& x) {
  if constexpr (!ODD) {
    store(p, x);
  } else if (left >= 4) {
    *reinterpret_cast<float4u*>(p) = float4u{x.v[0], x.v[1], x.v[2], x.v[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[e] = x.v[e];
  }
}

// The other end of the pair of column d < 2 half.
__device__ inline int partner(int d, int half, int layout) {
  return !layout ? d ^ 1 : d < half ? d + half : d - half;
}
// Where the partners of columns d .. d + 3 of a head begin, for turned(): of neighbours and of columns
// that stay, at d.
__device__ inline int partners_at(int d, int half, int layout) {
  return layout && d < 2 * half ? partner(d, half, layout) : d;
}
// The four values at partners_at(d) of the head at p.  ODD: value by value where the columns are of
// both halves, or of the last and behind it.
template <bool ODD>
__device__ inline Four partners(const float* p, int d, int half) {
  if constexpr (!ODD) {
    return load(p + partner(d, half, 1));
  } else {
    if (d + 4 <= half || (d >= half && d + 4 <= 2 * half)) return load<true>(p + partner(d, half, 1), 4);
    Four x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x.v[e] = d + e < 2 * half ? p[partner(d + e, half, 1)] : 0.f;
    return x;
  }
}
// The columns d .. turned (the first of them is; ODD: those at and past 2 half are not): own their
// values, other their partners', cs the row's turns.
template <bool ODD>
__device__ inline Four turned(const Four& own, const Four& other, int d, const float2* cs, int half,
                              int layout, bool back) {
  Four y = own;
  const float to = back ? -1.f : 1.f;
  if (!layout) {
    float2 t[2];
    if constexpr (ODD) {
      t[0] = cs[d / 2];
      t[1] = d + 2 < 2 * half ? cs[d / 2 + 1] : make_float2(1.f, 0.f);
    } else {
      const float4 u = *reinterpret_cast<const float4*>(cs + d / 2);
      t[0] = make_float2(u.x, u.y);
      t[1] = make_float2(u.z, u.w);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if (ODD && d + 2 * j >= 2 * half) break;   // (1 x is x, but 0 x is not always 0)
      const float s = to * t[j].y;
      y.v[2 * j] = own.v[2 * j] * t[j].x - own.v[2 * j + 1] * s;
      y.v[2 * j + 1] = own.v[2 * j + 1] * t[j].x + own.v[2 * j] * s;
    }
    return y;
  }
  if constexpr (ODD) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (d + e >= 2 * half) break;
      const bool second = d + e >= half;
      const float2 t = cs[d + e - (second ? half : 0)];
      y.v[e] = own.v[e] * t.x + (second ? to : -to) * (other.v[e] * t.y);
    }
  } else {
    const bool second = d >= half;
    const int i = second ? d - half : d;
    const float sign = second ? to : -to;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 t = cs[i + e];
      y.v[e] = own.v[e] * t.x + sign * (other.v[e] * t.y);
    }
  }
  return y;
}

// ---------------------------------------------------------------- rotation
// A thread has kFlight items' loads in flight.
constexpr int kFlight = 4;

__global__ __launch_bounds__(TPB) void rope_kernel(const float* __restrict__ x,
                                                   const int32_t* __restrict__ pos,
                                                   const double* __restrict__ table,
                                                   float* __restrict__ y, Rows r, bool back) {
  extern __shared__ float4 lds[];
  float2* cs = reinterpret_cast<float2*>(lds);
  const int64_t r0 = (int64_t)blockIdx.x * r.tile;
  const int n = (int)min((int64_t)r.tile, r.rows - r0);
  turns(cs, pos, table, r0, n, r);
  __syncthreads();
  const float* xt = x + r0 * r.cols;
  float* yt = y + r0 * r.cols;
  const int total = n * r.items, step = TPB * gridDim.y;
  for (int i0 = blockIdx.y * TPB + threadIdx.x; i0 < total; i0 += kFlight * step) {
    Four own[kFlight], other[kFlight];
    int row[kFlight], c[kFlight], d[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      const int i = min(i0 + u * step, total - 1);
      row[u] = r.by_items.div(i);
      c[u] = (i - row[u] * r.items) * 4;
      d[u] = c[u] - r.by_dh.div(c[u]) * r.dh;
      if (c[u] >= r.used || d[u] >= 2 * r.half) d[u] = -1;   // copied
      const float* p = xt + (int64_t)row[u] * r.cols + c[u];
      own[u] = load(p);
      other[u] = own[u];
      if (d[u] >= 0 && r.layout) other[u] = load(p - d[u] + partner(d[u], r.half, r.layout));
    }
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      if (i0 + u * step >= total) break;
      if (d[u] >= 0)
        own[u] = turned<false>(own[u], other[u], d[u], cs + row[u] * r.half, r.half, r.layout, back);
      store(yt + (int64_t)row[u] * r.cols + c[u], own[u]);
    }
  }
}

// The same value by value: a thread owns columns, places each in its head once and turns it for all
// rows of the tile.  Value by value over the whole tile, with two divisions each, the vector
// instructions were the bound: 32771 rows of 26 heads of 85, 34 columns turned: 162 us, so 154 (3.8 TB/s).
constexpr int kMaxTile = 8;
__global__ __launch_bounds__(TPB) void rope_columns_kernel(const float* __restrict__ x,
                                                           const int32_t* __restrict__ pos,
                                                           const double* __restrict__ table,
                                                           float* __restrict__ y, Rows r, bool back) {
  extern __shared__ float4 lds[];
  float2* cs = reinterpret_cast<float2*>(lds);
  const int64_t r0 = (int64_t)blockIdx.x * r.tile;
  const int n = (int)min((int64_t)r.tile, r.rows - r0);
  turns(cs, pos, table, r0, n, r);
  __syncthreads();
  for (int c = blockIdx.y * TPB + threadIdx.x; c < r.cols; c += TPB * gridDim.y) {
    const int d = c - r.by_dh.div(c) * r.dh;
    const bool turned = c < r.used && d < 2 * r.half;
    const int to = turned ? partner(d, r.half, r.layout) - d : 0;
    const int i = turned ? (r.layout ? min(d, d + to) : d >> 1) : 0;
    const float sign = turned ? ((to < 0) != back ? 1.f : -1.f) : 0.f;
    const float* p = x + r0 * r.cols + c;
    float own[kMaxTile], other[kMaxTile];
#pragma unroll
    for (int k = 0; k < kMaxTile; ++k)
      if (k < n) {
        own[k] = p[(int64_t)k * r.cols];
        other[k] = p[(int64_t)k * r.cols + to];
      }
    float* o = y + r0 * r.cols + c;
#pragma unroll
    for (int k = 0; k < kMaxTile; ++k)
      if (k < n) {
        const float2 t = cs[k * r.half + i];
        o[(int64_t)k * r.cols] = turned ? own[k] * t.x + sign * (other[k] * t.y) : own[k];
      }
  }
}

// ---------------------------------------------------------------- per-head norms
// A group of G neighbouring lanes holds one head of one row, lane l of it the four columns from
// 4 (l + G k) on, k < K.
template <int G>
__device__ inline float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// The columns behind the heads of a tile's rows are copied, all rows' together: a row at a time, with
// most threads idle, 12288 rows of 20 heads of 64 and 256 columns took 3 us more forward, 2 backward (39).
template <bool ODD>
__device__ inline void copy_rest(const float* __restrict__ x, float* __restrict__ y, int64_t r0, int n,
                                 const Rows& r) {
  const int rest = r.cols - r.used, items = (rest + 3) / 4, total = n * items;
#pragma unroll 2
  for (int t = threadIdx.x; t < total; t += TPB) {
    const int row = r.by_rest.div(t), c = 4 * (t - row * items);
    const int64_t at = (r0 + row) * r.cols + r.used + c;
    store<ODD>(y + at, rest - c, load<ODD>(x + at, rest - c));
  }
}

template <bool ODD, int G, int K>
__global__ __launch_bounds__(TPB) void qknorm_fwd_kernel(const float* __restrict__ x,
                                                         const float* __restrict__ gain,
                                                         const int32_t* __restrict__ pos,
                                                         const double* __restrict__ table,
                                                         float* __restrict__ y, Rows r) {
  extern __shared__ float4 lds[];
  float2* cs = reinterpret_cast<float2*>(lds);
  const int64_t r0 = (int64_t)blockIdx.x * r.tile;
  const int n = (int)min((int64_t)r.tile, r.rows - r0);
  if (r.half) {
    turns(cs, pos, table, r0, n, r);
    __syncthreads();
  }
  const int lane = threadIdx.x % G, step = TPB / G * gridDim.y, total = n * r.heads;
  // With one four a lane, both rows' gains of it and of its partners stay in registers: 12288 rows of
  // 20 heads of 64 and 256 columns took 39 us with their loads for every head, so 34 (4.4 TB/s).
  Four kept[2] = {}, kept_partners[2] = {};
  if (K == 1 && 4 * lane < r.dh) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float* g = gain + (w && r.h1 < r.heads ? r.dh : 0);
      kept[w] = load<ODD>(g + 4 * lane, r.dh - 4 * lane);
      if (partners_at(4 * lane, r.half, r.layout) != 4 * lane)
        kept_partners[w] = partners<ODD>(g, 4 * lane, r.half);
    }
  }
  const auto of_head = [&](const Four (&both)[2], int h) {
    Four x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x.v[e] = h < r.h1 ? both[0].v[e] : both[1].v[e];
    return x;
  };
  for (int u = blockIdx.y * (TPB / G) + threadIdx.x / G; u < total; u += step) {
    const int row = r.by_heads.div(u), h = u - row * r.heads;
    const int64_t at = (r0 + row) * r.cols + h * r.dh;
    const float* g = gain + (h < r.h1 ? 0 : r.dh);
    Four own[K], other[K];
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int d = 4 * (lane + G * k);
      own[k] = {};
      if (d < r.dh) {
        own[k] = load<ODD>(x + at + d, r.dh - d);
        const bool at_hand = partners_at(d, r.half, r.layout) == d;
        other[k] = at_hand ? own[k] : partners<ODD>(x + at, d, r.half);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float t = r.down * own[k].v[e];
        q += t * t;
      }
    }
    const float rs = 1.f / sqrtf(group_sum<G>(q) / (r.down * r.down * (float)r.dh) + 1e-5f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int d = 4 * (lane + G * k);
      if (d >= r.dh) continue;
      const Four gd = K == 1 ? of_head(kept, h) : load<ODD>(g + d, r.dh - d);
#pragma unroll
      for (int e = 0; e < 4; ++e) own[k].v[e] = gd.v[e] * (own[k].v[e] * rs);
      if (d < 2 * r.half) {
        if (partners_at(d, r.half, r.layout) != d) {
          const Four gp = K == 1 ? of_head(kept_partners, h) : partners<ODD>(g, d, r.half);
#pragma unroll
          for (int e = 0; e < 4; ++e) other[k].v[e] = gp.v[e] * (other[k].v[e] * rs);
        }
        own[k] = turned<ODD>(own[k], other[k], d, cs + row * r.half, r.half, r.layout, false);
      }
      store<ODD>(y + at + d, r.dh - d, own[k]);
    }
  }
  if (blockIdx.y == 0) copy_rest<ODD>(x, y, r0, n, r);
}

// A workgroup per row slice; its groups' sums of dgain are added in their order.
template <bool ODD, int G, int K>
__global__ __launch_bounds__(TPB) void qknorm_bwd_kernel(
    const float* __restrict__ x, const float* __restrict__ gain, const int32_t* __restrict__ pos,
    const double* __restrict__ table, const float* __restrict__ dy, float* __restrict__ dx,
    float* __restrict__ part, Rows r, int64_t len) {
  extern __shared__ float4 lds[];
  float2* cs = reinterpret_cast<float2*>(lds);
  const int lane = threadIdx.x % G, group = threadIdx.x / G;
  float acc[2][K][4];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[0][k][e] = acc[1][k][e] = 0.f;
  const int64_t s0 = blockIdx.x * len, s1 = min(r.rows, s0 + len);
  for (int64_t r0 = s0; r0 < s1; r0 += r.tile) {
    const int n = (int)min((int64_t)r.tile, s1 - r0), total = n * r.heads;
    if (r.half) {
      __syncthreads();
      turns(cs, pos, table, r0, n, r);
      __syncthreads();
    }
    for (int u = group; u < total; u += TPB / G) {
      const int row = r.by_heads.div(u), h = u - row * r.heads;
      const int64_t at = (r0 + row) * r.cols + h * r.dh;
      const bool second = h >= r.h1;
      const float* g = gain + (second ? r.dh : 0);
      Four xv[K], z[K], gd[K];
      float q = 0.f, dot = 0.f;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int d = 4 * (lane + G * k);
        xv[k] = z[k] = gd[k] = {};
        if (d < r.dh) {
          xv[k] = load<ODD>(x + at + d, r.dh - d);
          z[k] = load<ODD>(dy + at + d, r.dh - d);
          gd[k] = load<ODD>(g + d, r.dh - d);
          if (d < 2 * r.half) {
            const bool at_hand = partners_at(d, r.half, r.layout) == d;
            const Four other = at_hand ? z[k] : partners<ODD>(dy + at, d, r.half);
            z[k] = turned<ODD>(z[k], other, d, cs + row * r.half, r.half, r.layout, true);
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float t = r.down * xv[k].v[e];
          q += t * t;
          dot += gd[k].v[e] * z[k].v[e] * t;
        }
      }
      q = group_sum<G>(q);
      dot = group_sum<G>(dot);
      const float rs = 1.f / sqrtf(q / (r.down * r.down * (float)r.dh) + 1e-5f);
      const float mean = dot * rs / (r.down * (float)r.dh);   // of gain z xhat
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int d = 4 * (lane + G * k);
        Four o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float xh = xv[k].v[e] * rs, zx = z[k].v[e] * xh;
          acc[0][k][e] += second ? 0.f : zx;
          acc[1][k][e] += second ? zx : 0.f;
          o.v[e] = rs * (gd[k].v[e] * z[k].v[e] - xh * mean);
        }
        if (d < r.dh) store<ODD>(dx + at + d, r.dh - d, o);
      }
    }
    copy_rest<ODD>(dy, dx, r0, n, r);
  }
  // [groups][2][4 G K] in the turns' place
  float* sums = reinterpret_cast<float*>(lds);
  constexpr int N = 4 * G * K;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = 4 * (lane + G * k) + e;
      sums[(group * 2) * N + d] = acc[0][k][e];
      sums[(group * 2 + 1) * N + d] = acc[1][k][e];
    }
  __syncthreads();
  const int rows = r.h1 < r.heads ? 2 : 1;
  for (int c = threadIdx.x; c < rows * r.dh; c += TPB) {
    const int w = c >= r.dh ? 1 : 0, d = c - w * r.dh;
    float s = 0.f;
#pragma unroll 4
    for (int k = 0; k < TPB / G; ++k) s += sums[(k * 2 + w) * N + d];
    part[(int64_t)blockIdx.x * rows * r.dh + c] = s;
  }
}

// dgain = the slices' partials: a workgroup owns 16 columns, its 64 rows of threads take the slices
// s = row mod 64 in increasing order, eight loads in flight, and one row adds the 64 results in order.
constexpr int kFinCols = 16, kFinRows = 64, kFlights = 8;
__global__ __launch_bounds__(kFinCols * kFinRows) void qknorm_finalize(const float* __restrict__ part,
                                                                       float* __restrict__ dgain,
                                                                       int n, int64_t slices) {
  __shared__ float sums[kFinRows][kFinCols];
  const int c = blockIdx.x * kFinCols + threadIdx.x % kFinCols, row = threadIdx.x / kFinCols;
  float s = 0.f;
  if (c < n)
    for (int64_t k0 = row; k0 < slices; k0 += kFlights * kFinRows) {
      float x[kFlights];
#pragma unroll
      for (int i = 0; i < kFlights; ++i) {
        const int64_t k = k0 + i * kFinRows;
        x[i] = part[min(k, slices - 1) * n + c];
        if (k >= slices) x[i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < kFlights; ++i) s += x[i];
    }
  sums[row][threadIdx.x % kFinCols] = s;
  __syncthreads();
  if (row || c >= n) return;
  float t = 0.f;
#pragma unroll 8
  for (int k = 0; k < kFinRows; ++k) t += sums[k][threadIdx.x];
  dgain[c] = t;
}

// ---------------------------------------------------------------- launches
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Aligned 16-byte items: every head, the rotated width (each half of it where pairs lie half apart)
// and every row a multiple of four columns.
bool in_fours(const RopeShape& s, std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (!aligned16(p)) return false;
  return s.dh % 4 == 0 && s.cols % 4 == 0 && s.rot % (s.layout ? 8 : 4) == 0;
}

Rows rows_of(const RopeShape& s, int64_t h1, int V, int64_t rows_a_group) {
  Rows r;
  r.rows = s.rows;
  r.cols = (int)s.cols;
  r.dh = (int)s.dh;
  r.heads = (int)s.heads;
  r.used = (int)(s.heads * s.dh);
  r.half = (int)s.rot / 2;
  r.layout = (int)s.layout;
  r.h1 = (int)h1;
  r.items = r.cols / V;
  for (r.down = 1.f; r.down * r.down * (float)s.dh > 1.f;) r.down *= 0.5f;
  // Rows a workgroup takes: their turns keep its threads busy at 8 rows of 64 rotated columns, and
  // a launch has at least 1024 workgroups where it has the rows for them.
  r.tile = (int)std::max<int64_t>(1, std::min<int64_t>(kMaxTile, rows_a_group));
  r.by_half = Divisor::of(r.half);
  r.by_dh = Divisor::of(r.dh);
  r.by_heads = Divisor::of(r.heads);
  r.by_items = Divisor::of(r.items);
  r.by_rest = Divisor::of((r.cols - r.used + 3) / 4);
  return r;
}
unsigned blocks(int64_t rows, int64_t tile) { return (unsigned)((rows + tile - 1) / tile); }
// Parts a tile's items or heads are cut into where there are few tiles: 512 workgroups in all, and
// `least` threads' worth of work in each.
unsigned parts(unsigned tiles, int64_t work, int64_t least) {
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, work / least));
}

// Lanes a head of q fours of columns takes and fours a lane: the fewest idle lanes, and of these the
// fewest fours.  Forward + backward, 20000 rows of 10 heads of 96 and 192 columns: 49 + 61 us so, 59 +
// 64 one four a lane (8 of 32 lanes idle).  Odd widths value by value instead: heads of 85, 32 columns
// turned, 90 + 76 us, so 47 + 69.
#define GROUPS(ODD, CALL)                              \
  if (q <= 8) CALL(ODD, 8, 1);                         \
  else if (q <= 16) CALL(ODD, 16, 1);                  \
  else if (q <= 24) CALL(ODD, 8, 3);                   \
  else if (q <= 32) CALL(ODD, 32, 1);                  \
  else if (q <= 48) CALL(ODD, 16, 3);                  \
  else if (q <= 64) CALL(ODD, 64, 1);                  \
  else if (q <= 96) CALL(ODD, 32, 3);                  \
  else if (q <= 128) CALL(ODD, 64, 2);                 \
  else if (q <= 192) CALL(ODD, 64, 3);                 \
  else CALL(ODD, 64, 4)
#define BY_WIDTH(CALL)                                 \
  const int q = (r.dh + 3) / 4;                        \
  if (in_fours(s, pointers)) {                         \
    GROUPS(false, CALL);                               \
  } else {                                             \
    GROUPS(true, CALL);                                \
  }

}  // namespace

hipError_t rope(bool back, const float* x, const int32_t* pos, const double* table, float* y,
                const RopeShape& s, hipStream_t st) {
  const bool four = in_fours(s, {x, y});
  const Rows r = rows_of(s, s.heads, four ? 4 : 1, s.rows / 1024);
  const unsigned nx = blocks(r.rows, r.tile);
  const dim3 grid(nx, parts(nx, (int64_t)r.tile * r.items, TPB));
  const unsigned lds = (unsigned)(r.tile * r.half * sizeof(float2));
  if (four)
    hipLaunchKernelGGL(rope_kernel, grid, dim3(TPB), lds, st, x, pos, table, y, r, back);
  else
    hipLaunchKernelGGL(rope_columns_kernel, grid, dim3(TPB), lds, st, x, pos, table, y, r, back);
  return hipGetLastError();
}

hipError_t qknorm_fwd(const float* x, const float* gain, const int32_t* pos, const double* table,
                      float* y, const RopeShape& s, int64_t h1, hipStream_t st) {
  const std::initializer_list<const void*> pointers = {x, gain, y};
  const Rows r = rows_of(s, h1, 4, s.rows / 1024);
  const unsigned nx = blocks(r.rows, r.tile);
  const unsigned lds = (unsigned)(r.tile * r.half * sizeof(float2));
#define FWD(ODD, G, K)                                                                                  \
  hipLaunchKernelGGL((qknorm_fwd_kernel<ODD, G, K>), dim3(nx, parts(nx, (int64_t)r.tile * r.heads, TPB / G)), \
                     dim3(TPB), lds, st, x, gain, pos, table, y, r)
  BY_WIDTH(FWD)
#undef FWD
  return hipGetLastError();
}

hipError_t qknorm_bwd(const float* x, const float* gain, const int32_t* pos, const double* table,
                      const float* dy, float* dx, float* dgain, float* part, const RopeShape& s,
                      int64_t h1, int64_t slices, hipStream_t st) {
  const int64_t len = (s.rows + slices - 1) / slices;
  const std::initializer_list<const void*> pointers = {x, gain, dy, dx};
  const Rows r = rows_of(s, h1, 4, len);
  const int n = (int)((h1 < s.heads ? 2 : 1) * s.dh);
#define BWD(ODD, G, K)                                                                                  \
  hipLaunchKernelGGL((qknorm_bwd_kernel<ODD, G, K>), dim3((unsigned)slices), dim3(TPB),             \
                     (unsigned)std::max<size_t>(r.tile * r.half * sizeof(float2),                 \
                                                TPB * 8 * K * sizeof(float)),                 \
                     st, x, gain, pos, table, dy, dx, part, r, len)
  BY_WIDTH(BWD)
#undef BWD
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(qknorm_finalize, dim3((unsigned)((n + kFinCols - 1) / kFinCols)),
                     dim3(kFinCols * kFinRows), 0, st, part, dgain, n, slices);
  return hipGetLastError();
}

}  // namespace ooc

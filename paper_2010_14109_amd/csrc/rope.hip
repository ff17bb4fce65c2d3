// Rotary positions and per-head norms of queries and keys (gfx950).
//
// A row holds heads of dh columns side by side.  The rotation turns pairs of a head's first rot
// columns by the angle pos table[i] of their row; the norm divides a head by its root mean square
// and scales it by a gain, before the rotation.
//
// All of this is bound by the rows' traffic.  An angle belongs to a row and a pair, not to a head:
// a workgroup takes a tile of rows, computes the tile's cosines and sines once into LDS and uses
// them for every head.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"

namespace ooc {

namespace {

constexpr int TPB = 256;

// m cos a and m sin a of a = pos f.  Positions far out need the angle in 64 bits: at a million
// positions an fp32 angle is off by 0.06.  The product is rounded to a double as in the definition,
// a multiple of pi / 2 (in two doubles) taken off exactly, and the rest, within +-pi/4, goes through
// the Taylor series in fp32: the first term left out is below 2e-9.
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

// Rows a workgroup takes at once.
constexpr int kMaxTile = 8;

// The pairs' (m cos, m sin) of rows r0 .. r0 + n into cs [n][half].
__device__ inline void turns(float2* cs, const int32_t* pos, const double* table, int64_t r0, int n,
                             int half) {
  const float m = (float)table[half];
  for (int t = threadIdx.x; t < n * half; t += TPB) cs[t] = turn(pos[r0 + t / half], table[t % half], m);
}

// What column d of a head becomes: own x[d] + sign x[partner].
struct Pair {
  int partner, i;
  float sign;
};
__device__ inline Pair pair_of(int d, int half, int layout, bool back) {
  const bool second = layout == 0 ? d & 1 : d >= half;
  Pair p;
  p.partner = layout == 0 ? d ^ 1 : second ? d - half : d + half;
  p.i = layout == 0 ? d >> 1 : second ? d - half : d;
  p.sign = second != back ? 1.f : -1.f;
  return p;
}

__global__ __launch_bounds__(TPB) void rope_kernel(const float* __restrict__ x,
                                                   const int32_t* __restrict__ pos,
                                                   const double* __restrict__ table,
                                                   float* __restrict__ y, RopeShape r, int tile,
                                                   bool back) {
  extern __shared__ float2 cs[];
  const int64_t r0 = (int64_t)blockIdx.x * tile;
  const int n = (int)min((int64_t)tile, r.rows - r0), half = (int)r.rot / 2;
  turns(cs, pos, table, r0, n, half);
  __syncthreads();
  const int cols = (int)r.cols, dh = (int)r.dh, used = (int)(r.heads * r.dh);
  for (int row = 0; row < n; ++row) {
    const float* xr = x + (r0 + row) * r.cols;
    float* yr = y + (r0 + row) * r.cols;
    for (int c = threadIdx.x; c < cols; c += TPB) {
      const int d = c % dh;
      float v = xr[c];
      if (c < used && d < (int)r.rot) {
        const Pair p = pair_of(d, half, (int)r.layout, back);
        const float2 w = cs[row * half + p.i];
        v = v * w.x + p.sign * xr[c - d + p.partner] * w.y;
      }
      yr[c] = v;
    }
  }
}

__device__ inline float wave_sum(float v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// One wave per (row, head), lane l owning the columns l, l + 64, ...
__global__ __launch_bounds__(TPB) void qknorm_fwd_kernel(const float* __restrict__ x,
                                                         const float* __restrict__ gain,
                                                         const int32_t* __restrict__ pos,
                                                         const double* __restrict__ table,
                                                         float* __restrict__ y, RopeShape r,
                                                         int h1, int tile) {
  extern __shared__ float2 cs[];
  const int64_t r0 = (int64_t)blockIdx.x * tile;
  const int n = (int)min((int64_t)tile, r.rows - r0), half = (int)r.rot / 2, dh = (int)r.dh;
  if (half) turns(cs, pos, table, r0, n, half);
  __syncthreads();
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, heads = (int)r.heads;
  for (int u = w; u < n * heads; u += TPB / 64) {
    const int row = u / heads, h = u % heads;
    const float* xr = x + (r0 + row) * r.cols + h * dh;
    float* yr = y + (r0 + row) * r.cols + h * dh;
    const float* g = gain + (h < h1 ? 0 : dh);
    float q = 0.f;
    for (int d = lane; d < dh; d += 64) q += xr[d] * xr[d];
    const float rs = 1.f / sqrtf(wave_sum(q) / (float)dh + 1e-5f);
    for (int d = lane; d < dh; d += 64) {
      float v = g[d] * (xr[d] * rs);
      if (d < 2 * half) {
        const Pair p = pair_of(d, half, (int)r.layout, false);
        const float2 t = cs[row * half + p.i];
        v = v * t.x + p.sign * (g[p.partner] * (xr[p.partner] * rs)) * t.y;
      }
      yr[d] = v;
    }
  }
  const int used = heads * dh, rest = (int)r.cols - used;
  for (int row = 0; row < n; ++row)
    for (int c = threadIdx.x; c < rest; c += TPB)
      y[(r0 + row) * r.cols + used + c] = x[(r0 + row) * r.cols + used + c];
}

// A workgroup per row slice; its waves' sums of dgain are added in wave order.
constexpr int kMaxJ = 16;   // columns a lane owns at dh = 1024
__global__ __launch_bounds__(TPB) void qknorm_bwd_kernel(
    const float* __restrict__ x, const float* __restrict__ gain, const int32_t* __restrict__ pos,
    const double* __restrict__ table, const float* __restrict__ dy, float* __restrict__ dx,
    float* __restrict__ part, RopeShape r, int h1, int64_t len, int tile) {
  extern __shared__ float2 cs[];
  const int half = (int)r.rot / 2, dh = (int)r.dh, heads = (int)r.heads;
  const int groups = h1 < heads ? 2 : 1;
  float* sums = reinterpret_cast<float*>(cs + tile * half);   // [groups][dh]
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float acc[2][kMaxJ];
#pragma unroll
  for (int j = 0; j < kMaxJ; ++j) acc[0][j] = acc[1][j] = 0.f;
  const int64_t s0 = blockIdx.x * len, s1 = min(r.rows, s0 + len);
  for (int64_t r0 = s0; r0 < s1; r0 += tile) {
    const int n = (int)min((int64_t)tile, s1 - r0);
    __syncthreads();
    if (half) turns(cs, pos, table, r0, n, half);
    __syncthreads();
    for (int u = w; u < n * heads; u += TPB / 64) {
      const int row = u / heads, h = u % heads;
      const int64_t at = (r0 + row) * r.cols + h * dh;
      const int second = h < h1 ? 0 : 1;
      const float* g = gain + second * dh;
      float q = 0.f, dot = 0.f, z[kMaxJ];
#pragma unroll
      for (int j = 0; j < kMaxJ; ++j) {
        const int d = lane + 64 * j;
        z[j] = 0.f;
        if (d < dh) {
          z[j] = dy[at + d];
          if (d < 2 * half) {
            const Pair p = pair_of(d, half, (int)r.layout, true);
            const float2 t = cs[row * half + p.i];
            z[j] = z[j] * t.x + p.sign * dy[at + p.partner] * t.y;
          }
          q += x[at + d] * x[at + d];
          dot += g[d] * z[j] * x[at + d];
        }
      }
      const float rs = 1.f / sqrtf(wave_sum(q) / (float)dh + 1e-5f);
      const float mean = wave_sum(dot) * rs / (float)dh;   // of gain z xhat
#pragma unroll
      for (int j = 0; j < kMaxJ; ++j) {
        const int d = lane + 64 * j;
        if (d < dh) {
          const float xh = x[at + d] * rs, zx = z[j] * xh;
          acc[0][j] += second ? 0.f : zx;
          acc[1][j] += second ? zx : 0.f;
          dx[at + d] = rs * (g[d] * z[j] - xh * mean);
        }
      }
    }
    const int used = heads * dh, rest = (int)r.cols - used;
    for (int row = 0; row < n; ++row)
      for (int c = threadIdx.x; c < rest; c += TPB)
        dx[(r0 + row) * r.cols + used + c] = dy[(r0 + row) * r.cols + used + c];
  }
  for (int k = 0; k < TPB / 64; ++k) {
    __syncthreads();
    if (w == k) {
#pragma unroll
      for (int j = 0; j < kMaxJ; ++j) {
        const int d = lane + 64 * j;
        if (d < dh) {
          sums[d] = (k ? sums[d] : 0.f) + acc[0][j];
          if (groups == 2) sums[dh + d] = (k ? sums[dh + d] : 0.f) + acc[1][j];
        }
      }
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < groups * dh; c += TPB) part[blockIdx.x * (int64_t)(groups * dh) + c] = sums[c];
}

// dgain = the slices' partials added in order
__global__ __launch_bounds__(TPB) void qknorm_finalize(const float* __restrict__ part,
                                                       float* __restrict__ dgain, int n,
                                                       int64_t slices) {
  const int c = blockIdx.x * TPB + threadIdx.x;
  if (c >= n) return;
  float s = 0.f;
  for (int64_t k = 0; k < slices; ++k) s += part[k * n + c];
  dgain[c] = s;
}

// Rows per workgroup: all of a launch's cosines fit kMaxTile rows, fewer where that would leave
// compute units without work.
int row_tile(const RopeShape& r) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(kMaxTile, r.rows / 1024));
}

unsigned blocks(int64_t rows, int64_t tile) { return (unsigned)((rows + tile - 1) / tile); }

}  // namespace

hipError_t rope(bool back, const float* x, const int32_t* pos, const double* table, float* y,
                const RopeShape& r, hipStream_t s) {
  const int tile = row_tile(r);
  hipLaunchKernelGGL(rope_kernel, dim3(blocks(r.rows, tile)), dim3(TPB),
                     (unsigned)(tile * r.rot / 2 * sizeof(float2)), s, x, pos, table, y, r, tile,
                     back);
  return hipGetLastError();
}

hipError_t qknorm_fwd(const float* x, const float* gain, const int32_t* pos, const double* table,
                      float* y, const RopeShape& r, int64_t h1, hipStream_t s) {
  const int tile = row_tile(r);
  hipLaunchKernelGGL(qknorm_fwd_kernel, dim3(blocks(r.rows, tile)), dim3(TPB),
                     (unsigned)(tile * r.rot / 2 * sizeof(float2)), s, x, gain, pos, table, y, r,
                     (int)h1, tile);
  return hipGetLastError();
}

hipError_t qknorm_bwd(const float* x, const float* gain, const int32_t* pos, const double* table,
                      const float* dy, float* dx, float* dgain, float* part, const RopeShape& r,
                      int64_t h1, int64_t slices, hipStream_t s) {
  const int64_t len = (r.rows + slices - 1) / slices;
  const int tile = (int)std::min<int64_t>(kMaxTile, len);
  const int n = (int)((h1 < r.heads ? 2 : 1) * r.dh);
  hipLaunchKernelGGL(qknorm_bwd_kernel, dim3((unsigned)slices), dim3(TPB),
                     (unsigned)(tile * r.rot / 2 * sizeof(float2) + n * sizeof(float)), s, x, gain,
                     pos, table, dy, dx, part, r, (int)h1, len, tile);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(qknorm_finalize, dim3((unsigned)((n + TPB - 1) / TPB)), dim3(TPB), 0, s, part,
                     dgain, n, slices);
  return hipGetLastError();
}

}  // namespace ooc

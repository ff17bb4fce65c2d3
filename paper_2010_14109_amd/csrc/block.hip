// Dropout whose mask is never stored, and the join of a block with its residual stream (gfx950):
// the norm behind the block, its gate, dropout, the residual sum and the norm before the next block
// in one pass.
//
// All of this is bound by memory traffic: dropout 8 bytes a value, the join 16 forward (two tensors
// read, two written) and 24 backward (four read, two written).  A row's values stay in registers
// between its sums, so nothing is read twice.  50 M values dropped: 70 us, 5.8 TB/s, the ten rounds of
// the generator taking a third of the vector instructions' time; 12288 x 1024 joined: 35 us forward (5.7
// TB/s), 59 backward (5.1) and 6 for the sums of the gains.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "kernels.h"

namespace ooc {

namespace {

constexpr int TPB = 256;
constexpr float kEps = 1e-5f;

typedef float floatx4u __attribute__((ext_vector_type(4), aligned(4)));   // at a 4-byte aligned address

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------- random words
// Philox 4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011): four random words from a counter of four words and a key of two, in ten rounds of two
// 32 x 32 -> 64 bit products.  Value i of a tensor takes word i % 4 of counter (i / 4, salt).
struct Words {
  uint32_t v[4];
};
__device__ inline Words philox(uint64_t counter, uint64_t salt, uint2 key) {
  uint32_t a = (uint32_t)counter, b = (uint32_t)(counter >> 32), c = (uint32_t)salt,
           d = (uint32_t)(salt >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p = (uint64_t)a * 0xD2511F53u, q = (uint64_t)c * 0xCD9E8D57u;
    a = (uint32_t)(q >> 32) ^ b ^ key.x;
    c = (uint32_t)(p >> 32) ^ d ^ key.y;
    b = (uint32_t)q;
    d = (uint32_t)p;
    key.x += 0x9E3779B9u;
    key.y += 0xBB67AE85u;
  }
  return {{a, b, c, d}};
}

// What is dropped, and what the kept are multiplied by, rounded to fp32.
struct Drop {
  uint32_t below;
  float keep;
  uint64_t salt;
  static Drop of(int64_t drop, int64_t salt) {
    return {(uint32_t)drop, (float)(4294967296.0 / (4294967296.0 - (double)drop)), (uint64_t)salt};
  }
  __device__ float apply(uint32_t word, float x) const { return word >= below ? x * keep : 0.f; }
};

// ---------------------------------------------------------------- dropout
template <bool DROP>
__global__ __launch_bounds__(TPB) void dropout_kernel(const float* __restrict__ x,
                                                      const uint32_t* __restrict__ seed,
                                                      float* __restrict__ y, int64_t n, Drop drop) {
  const uint2 key = DROP ? make_uint2(seed[0], seed[1]) : make_uint2(0, 0);
  const int64_t stride = (int64_t)gridDim.x * TPB, fours = n / 4;
  int64_t j = (int64_t)blockIdx.x * TPB + threadIdx.x;
  for (; j < fours; j += stride) {
    float4 v = reinterpret_cast<const float4*>(x)[j];
    if (DROP) {
      const Words w = philox((uint64_t)j, drop.salt, key);
      v = make_float4(drop.apply(w.v[0], v.x), drop.apply(w.v[1], v.y), drop.apply(w.v[2], v.z),
                      drop.apply(w.v[3], v.w));
    }
    reinterpret_cast<float4*>(y)[j] = v;
  }
  if (j == fours) {   // the one thread that comes to the values behind the last four
    const Words w = DROP ? philox((uint64_t)j, drop.salt, key) : Words{};
    for (int e = 0; e < (int)(n % 4); ++e)
      y[4 * j + e] = DROP ? drop.apply(w.v[e], x[4 * j + e]) : x[4 * j + e];
  }
}

// ---------------------------------------------------------------- join
// A row is held by W waves, E groups of four columns a lane.
template <int W, int E>
struct Row {
  static constexpr int kThreads = W > 4 ? 64 * W : TPB;
  static constexpr int kRows = kThreads / (64 * W);   // rows a workgroup works on at once
  static __device__ int sub() { return (int)threadIdx.x / (64 * W); }
  static __device__ int column(int k) { return 4 * ((int)threadIdx.x % (64 * W) + k * 64 * W); }
};

struct Four {
  float v[4];
};
__device__ inline Four load4(const float* p, int c, int d) {
  Four r;
  if (c + 4 <= d) {
    const floatx4u a = *reinterpret_cast<const floatx4u*>(p + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) r.v[e] = a[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) r.v[e] = c + e < d ? p[c + e] : 0.f;
  }
  return r;
}
__device__ inline void store4(float* p, int c, int d, const Four& x) {
  if (c + 4 <= d) {
    *reinterpret_cast<floatx4u*>(p + c) = floatx4u{x.v[0], x.v[1], x.v[2], x.v[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < d) p[c + e] = x.v[e];
  }
}

template <int CTRL>
__device__ inline float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL,
                                                               0xf, 0xf, true));
}
// the sum of a wave's values, in every lane
__device__ inline float wave_sum(float x) {
  x += dpp<0xb1>(x);    // quad_perm 1 0 3 2
  x += dpp<0x4e>(x);    // quad_perm 2 3 0 1
  x += dpp<0x141>(x);   // mirrored within 8
  x += dpp<0x140>(x);   // mirrored within 16
  uint32_t v = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const uint32_t a = r[0], b = r[1];
  x = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
  v = __builtin_bit_cast(uint32_t, x);
  const auto t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  const uint32_t c = t[0], d = t[1];
  return __builtin_bit_cast(float, c) + __builtin_bit_cast(float, d);
}
// The row's sum of x; `room` is kRows W floats of LDS, used once.
template <int W>
__device__ inline float row_sum(float x, float* room) {
  x = wave_sum(x);
  if constexpr (W > 1) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) room[w] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) x += room[w / W * W + k];
  }
  return x;
}

// Four values from index i on, dropped: KIND 0 none are, 1 indexes of a row's fours are multiples of
// four, 2 they are not, and take words of two counters.
template <int KIND>
__device__ inline Words words_at(uint64_t i, const Drop& drop, uint2 key) {
  if constexpr (KIND == 1) return philox(i / 4, drop.salt, key);
  const Words a = philox(i / 4, drop.salt, key), b = philox(i / 4 + 1, drop.salt, key);
  const int at = (int)(i % 4);
  Words r;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 7; ++k) w = at + e == k ? (k < 4 ? a.v[k] : b.v[k - 4]) : w;
    r.v[e] = w;
  }
  return r;
}
template <int KIND>
__device__ inline Four dropped(const Words& w, const Drop& drop, const Four& x) {
  if constexpr (KIND == 0) return x;
  Four r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r.v[e] = drop.apply(w.v[e], x.v[e]);
  return r;
}

struct Join4 {
  const float *post, *gate, *pre, *scale;
  const uint32_t* seed;
  int64_t rows, per;   // per: rows that share a gate
  int d;
  Drop drop;
};

template <int W, int E, int KIND>
__global__ __launch_bounds__((Row<W, E>::kThreads)) void join_fwd_kernel(
    const float* __restrict__ x, const float* __restrict__ f, Join4 j, float* __restrict__ h,
    float* __restrict__ n, float* __restrict__ stats) {
  using R = Row<W, E>;
  __shared__ float room[2][R::kThreads / 64];
  const int64_t row = (int64_t)blockIdx.x * R::kRows + R::sub();
  const bool live = row < j.rows;
  const int64_t at = (live ? row : 0) * j.d;
  const float* gate = j.gate + (live ? row / j.per : 0) * j.d;
  Four v[E], y[E];
  float ff = 0.f, hh = 0.f;
#pragma unroll
  for (int k = 0; k < E; ++k) {
    const int c = R::column(k);
    v[k] = load4(f + at, c, j.d);
    y[k] = load4(x + at, c, j.d);
#pragma unroll
    for (int e = 0; e < 4; ++e) ff = fmaf(v[k].v[e], v[k].v[e], ff);
  }
  const float rf = 1.f / sqrtf(row_sum<W>(ff, room[0]) / (float)j.d + kEps);
  const float rho = j.scale[0];
  const uint2 key = KIND ? make_uint2(j.seed[0], j.seed[1]) : make_uint2(0, 0);
#pragma unroll
  for (int k = 0; k < E; ++k) {
    const int c = R::column(k);
    const Four a = load4(j.post, c, j.d), g = load4(gate, c, j.d);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[k].v[e] *= rf * a.v[e];
    if constexpr (KIND) v[k] = dropped<KIND>(words_at<KIND>((uint64_t)(at + c), j.drop, key), j.drop, v[k]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[k].v[e] = fmaf(g.v[e], v[k].v[e], rho * y[k].v[e]);
      hh = fmaf(y[k].v[e], y[k].v[e], hh);
    }
    if (live) store4(h + at, c, j.d, y[k]);
  }
  const float rh = 1.f / sqrtf(row_sum<W>(hh, room[1]) / (float)j.d + kEps);
  if (!live) return;
#pragma unroll
  for (int k = 0; k < E; ++k) {
    const int c = R::column(k);
    const Four p = load4(j.pre, c, j.d);
    Four o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o.v[e] = p.v[e] * (y[k].v[e] * rh);
    store4(n + at, c, j.d, o);
  }
  if (threadIdx.x % (64 * W) == 0) {
    stats[2 * row] = rf;
    stats[2 * row + 1] = rh;
  }
}

// A workgroup takes the rows of one slice of a gate's rows and keeps their sums of dpost, dgate and
// dpre in registers; its rows' waves add theirs up at the end.
template <int W, int E, int KIND>
__global__ __launch_bounds__((Row<W, E>::kThreads), 2) void join_bwd_kernel(
    const float* __restrict__ f, const float* __restrict__ h, const float* __restrict__ stats,
    Join4 j, const float* __restrict__ dh, const float* __restrict__ dn, float* __restrict__ dx,
    float* __restrict__ df, float* __restrict__ part, int64_t slices, int64_t slice_rows) {
  using R = Row<W, E>;
  __shared__ float room[2][2][R::kThreads / 64];
  __shared__ float sums[R::kRows > 1 ? R::kRows - 1 : 1][R::kRows > 1 ? 256 * W * E : 1];
  const int64_t group = blockIdx.x / slices, slice = blockIdx.x % slices;
  const int64_t r0 = group * j.per + min(j.per, slice * slice_rows);
  const int64_t r1 = group * j.per + min(j.per, (slice + 1) * slice_rows);
  const float* gate = j.gate + group * j.d;
  const float rho = j.scale[0], inv = 1.f / (float)j.d;
  const uint2 key = KIND ? make_uint2(j.seed[0], j.seed[1]) : make_uint2(0, 0);
  Four acc[3][E] = {};   // dpost, dgate, dpre
  int turn = 0;
  for (int64_t r = r0; r < r1; r += R::kRows, turn ^= 1) {
    const int64_t row = r + R::sub();
    const bool live = row < r1;
    const int64_t at = (live ? row : r) * j.d;
    const float rf = stats[2 * (live ? row : r)], rh = stats[2 * (live ? row : r) + 1];
    Four v[E], t[E], g[E], m[E];
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const int c = R::column(k);
      v[k] = load4(f + at, c, j.d);
      t[k] = load4(h + at, c, j.d);
      m[k] = load4(dn + at, c, j.d);
      if (dh) g[k] = load4(dh + at, c, j.d);
      else g[k] = Four{};
    }
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const Four p = load4(j.pre, R::column(k), j.d);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[k].v[e] *= rf;
        t[k].v[e] *= rh;
        acc[2][k].v[e] += live ? m[k].v[e] * t[k].v[e] : 0.f;
        m[k].v[e] *= p.v[e];
        q = fmaf(m[k].v[e], t[k].v[e], q);
      }
    }
    q = row_sum<W>(q, room[turn][0]) * inv;
    float p = 0.f;
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const int c = R::column(k);
      const Four a = load4(j.post, c, j.d), b = load4(gate, c, j.d);
      Words w{};
      if constexpr (KIND) w = words_at<KIND>((uint64_t)(at + c), j.drop, key);
      Four u, o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g[k].v[e] = fmaf(rh, m[k].v[e] - t[k].v[e] * q, g[k].v[e]);   // all that h gets
        o.v[e] = rho * g[k].v[e];
        u.v[e] = a.v[e] * v[k].v[e];
      }
      if (live) store4(dx + at, c, j.d, o);
      u = dropped<KIND>(w, j.drop, u);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[1][k].v[e] += live ? g[k].v[e] * u.v[e] : 0.f;
        g[k].v[e] *= b.v[e];
      }
      g[k] = dropped<KIND>(w, j.drop, g[k]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[0][k].v[e] += live ? g[k].v[e] * v[k].v[e] : 0.f;
        g[k].v[e] *= a.v[e];
        p = fmaf(g[k].v[e], v[k].v[e], p);
      }
    }
    p = row_sum<W>(p, room[turn][1]) * inv;
    if (live)
#pragma unroll
      for (int k = 0; k < E; ++k) {
        Four o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o.v[e] = rf * (g[k].v[e] - v[k].v[e] * p);
        store4(df + at, R::column(k), j.d, o);
      }
  }
  float* out = part + (int64_t)blockIdx.x * 3 * j.d;
#pragma unroll
  for (int s = 0; s < 3; ++s) {
    if constexpr (R::kRows > 1) {
      if (R::sub() > 0)
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) sums[R::sub() - 1][R::column(k) + e] = acc[s][k].v[e];
      __syncthreads();
    }
    if (R::sub() == 0)
#pragma unroll
      for (int k = 0; k < E; ++k) {
        if constexpr (R::kRows > 1)
#pragma unroll
          for (int o = 0; o < R::kRows - 1; ++o)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[s][k].v[e] += sums[o][R::column(k) + e];
        store4(out + (int64_t)s * j.d, R::column(k), j.d, acc[s][k]);
      }
    if constexpr (R::kRows > 1) __syncthreads();
  }
}

// dpost, dpre and the gates' gradients from the slices' sums, 64 columns a workgroup, in a fixed
// order: a thread takes every 16th slice, then the 16 are added.
constexpr int kSumRows = 16;
__global__ __launch_bounds__(64 * kSumRows) void join_sum_kernel(const float* __restrict__ part,
                                                                 float* __restrict__ dpost,
                                                                 float* __restrict__ dgate,
                                                                 float* __restrict__ dpre, int d,
                                                                 int64_t groups, int64_t slices) {
  __shared__ float sums[kSumRows][64];
  const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  const int64_t what = blockIdx.y;   // 0: dpost, 1: dpre, 2 + g: gate g
  const int which = what == 0 ? 0 : what == 1 ? 2 : 1;
  const int64_t first = what < 2 ? 0 : (what - 2) * slices, last = what < 2 ? groups * slices : first + slices;
  float acc = 0.f;
  for (int64_t s = first + sub; s < last; s += 8 * kSumRows) {   // eight loads in flight
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t u = s + k * kSumRows;
      x[k] = u < last && c < d ? part[(u * 3 + which) * d + c] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) acc += x[k];
  }
  sums[sub][lane] = acc;
  __syncthreads();
  if (sub || c >= d) return;
  acc = 0.f;
#pragma unroll
  for (int k = 0; k < kSumRows; ++k) acc += sums[k][lane];
  (what == 0 ? dpost : what == 1 ? dpre : dgate + (what - 2) * d)[c] = acc;
}

Join4 of(const float* post, const float* gate, const float* pre, const float* scale,
         const uint32_t* seed, const JoinShape& a) {
  return {post, gate, pre, scale, seed, a.rows, a.rows / a.groups, (int)a.d, Drop::of(a.drop, a.salt)};
}

#define JOIN_KIND(W, E, LAUNCH)          \
  if (!a.drop) { LAUNCH(W, E, 0); }      \
  else if (a.d % 4 == 0) { LAUNCH(W, E, 1); } \
  else { LAUNCH(W, E, 2); }
#define JOIN_WIDTH(LAUNCH)                                 \
  if (a.d <= 256) { JOIN_KIND(1, 1, LAUNCH) }              \
  else if (a.d <= 512) { JOIN_KIND(1, 2, LAUNCH) }         \
  else if (a.d <= 1024) { JOIN_KIND(1, 4, LAUNCH) }        \
  else if (a.d <= 2048) { JOIN_KIND(2, 4, LAUNCH) }        \
  else if (a.d <= 4096) { JOIN_KIND(4, 4, LAUNCH) }        \
  else { JOIN_KIND(8, 4, LAUNCH) }

}  // namespace

hipError_t dropout(const float* x, const uint32_t* seed, float* y, int64_t n, int64_t drop,
                   int64_t salt, hipStream_t s) {
  const unsigned grid = (unsigned)std::min<int64_t>(n / 4 / TPB + 1, 16384);
  const Drop d = Drop::of(drop, salt);
  if (drop) hipLaunchKernelGGL(dropout_kernel<true>, dim3(grid), dim3(TPB), 0, s, x, seed, y, n, d);
  else hipLaunchKernelGGL(dropout_kernel<false>, dim3(grid), dim3(TPB), 0, s, x, seed, y, n, d);
  return hipGetLastError();
}

// Workgroups to fill the chip: three a CU where a wave holds a row, two where a row takes more waves
// (12288 x 1024 with gradients: 112 us with 512, 103 with 768, 109 with 1024; 9193 x 1365: 148 with 512, 169
// with 768).  A slice has eight rows or more, where there are as many, so that its three rows of sums are
// little beside them.
int64_t join_slices(int64_t rows, int64_t d, int64_t groups) {
  const int64_t want = d <= 1024 ? 768 : 512;
  return std::max<int64_t>(1, std::min(ceil_div(want, groups), ceil_div(rows / groups, 8)));
}

hipError_t join_fwd(const float* x, const float* f, const float* post, const float* gate,
                    const float* pre, const float* scale, const uint32_t* seed, float* h, float* n,
                    float* stats, const JoinShape& a, hipStream_t s) {
  const Join4 j = of(post, gate, pre, scale, seed, a);
#define FWD(W, E, KIND)                                                                             \
  hipLaunchKernelGGL((join_fwd_kernel<W, E, KIND>), dim3((unsigned)ceil_div(a.rows, Row<W, E>::kRows)), \
                     dim3(Row<W, E>::kThreads), 0, s, x, f, j, h, n, stats)
  JOIN_WIDTH(FWD)
#undef FWD
  return hipGetLastError();
}

hipError_t join_bwd(const float* f, const float* h, const float* stats, const float* post,
                    const float* gate, const float* pre, const float* scale, const uint32_t* seed,
                    const float* dh, const float* dn, float* dx, float* df, float* dpost,
                    float* dgate, float* dpre, float* part, const JoinShape& a, int64_t slices,
                    hipStream_t s) {
  const Join4 j = of(post, gate, pre, scale, seed, a);
  const int64_t len = ceil_div(a.rows / a.groups, slices);
#define BWD(W, E, KIND)                                                                            \
  hipLaunchKernelGGL((join_bwd_kernel<W, E, KIND>), dim3((unsigned)(a.groups * slices)),           \
                     dim3(Row<W, E>::kThreads), 0, s, f, h, stats, j, dh, dn, dx, df, part, slices, len)
  JOIN_WIDTH(BWD)
#undef BWD
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(join_sum_kernel, dim3((unsigned)ceil_div(a.d, 64), (unsigned)(2 + a.groups)),
                     dim3(64 * kSumRows), 0, s, part, dpost, dgate, dpre, (int)a.d, a.groups, slices);
  return hipGetLastError();
}

}  // namespace ooc

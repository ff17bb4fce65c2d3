// Cross attention: queries against the first klen states of their sequence (gfx950).
//
// One pass over the states with the running maximum and sum of the softmax; no matrix of scores is
// kept.  The backward recomputes the probabilities from the forward's row logarithms lse.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels.h"

namespace ooc {

namespace {

constexpr int TPB = 256;
constexpr int kJ = 4;   // columns a lane owns at dh = 256

__device__ inline float wave_sum(float v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

struct Row {
  float v[kJ];
};
__device__ inline Row load_row(const float* p, int dh) {
  Row r;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < kJ; ++j) r.v[j] = lane + 64 * j < dh ? p[lane + 64 * j] : 0.f;
  return r;
}
__device__ inline void store_row(float* p, const Row& r, int dh) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < kJ; ++j)
    if (lane + 64 * j < dh) p[lane + 64 * j] = r.v[j];
}
__device__ inline float dot(const Row& a, const Row& b) {
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < kJ; ++j) s += a.v[j] * b.v[j];
  return wave_sum(s);
}
__device__ inline void fma_row(Row& a, float s, const Row& b) {
#pragma unroll
  for (int j = 0; j < kJ; ++j) a.v[j] += s * b.v[j];
}

__device__ inline bool bad_length(int n, int Tk) { return n < 0 || n > Tk; }

// One wave per query row: (b, i, h) in the order of q's rows and heads.
__global__ __launch_bounds__(TPB) void fwd_kernel(const float* __restrict__ q,
                                                  const float* __restrict__ kv,
                                                  const int32_t* __restrict__ klen,
                                                  float* __restrict__ y, float* __restrict__ lse,
                                                  AttendShape a, float scale) {
  const int64_t u = (int64_t)blockIdx.x * (TPB / 64) + (threadIdx.x >> 6);
  if (u >= a.B * a.Tq * a.H) return;
  const int64_t h = u % a.H, i = u / a.H % a.Tq, b = u / a.H / a.Tq;
  const int n = klen[b], dh = (int)a.dh;
  const int64_t d2 = 2 * a.Hkv * a.dh;
  const float* k = kv + b * a.Tk * d2 + h / (a.H / a.Hkv) * a.dh;
  const Row qr = load_row(q + u * a.dh, dh);
  Row acc = {};
  float m = -INFINITY, sum = 0.f;
  for (int j = 0; j < n && !bad_length(n, (int)a.Tk); ++j) {
    const float s = dot(qr, load_row(k + j * d2, dh)) * scale;
    const float top = fmaxf(m, s), f = expf(m - top), p = expf(s - top);
#pragma unroll
    for (int e = 0; e < kJ; ++e) acc.v[e] *= f;
    sum = sum * f + p;
    fma_row(acc, p, load_row(k + j * d2 + a.Hkv * a.dh, dh));
    m = top;
  }
  const float inv = bad_length(n, (int)a.Tk) ? NAN : n ? 1.f / sum : 0.f;
#pragma unroll
  for (int e = 0; e < kJ; ++e) acc.v[e] *= inv;
  store_row(y + u * a.dh, acc, dh);
  if ((threadIdx.x & 63) == 0)
    lse[(b * a.H + h) * a.Tq + i] = bad_length(n, (int)a.Tk) ? NAN : m + logf(sum);
}

__global__ __launch_bounds__(TPB) void dq_kernel(const float* __restrict__ q,
                                                 const float* __restrict__ kv,
                                                 const int32_t* __restrict__ klen,
                                                 const float* __restrict__ y,
                                                 const float* __restrict__ lse,
                                                 const float* __restrict__ dy,
                                                 float* __restrict__ dq, float* __restrict__ delta,
                                                 AttendShape a, float scale) {
  const int64_t u = (int64_t)blockIdx.x * (TPB / 64) + (threadIdx.x >> 6);
  if (u >= a.B * a.Tq * a.H) return;
  const int64_t h = u % a.H, i = u / a.H % a.Tq, b = u / a.H / a.Tq;
  const int n = klen[b], dh = (int)a.dh;
  const int64_t d2 = 2 * a.Hkv * a.dh, at = (b * a.H + h) * a.Tq + i;
  const float* k = kv + b * a.Tk * d2 + h / (a.H / a.Hkv) * a.dh;
  const Row qr = load_row(q + u * a.dh, dh), g = load_row(dy + u * a.dh, dh);
  const float l = lse[at], dl = n ? dot(g, load_row(y + u * a.dh, dh)) : 0.f;
  Row acc = {};
  for (int j = 0; j < n && !bad_length(n, (int)a.Tk); ++j) {
    const Row kr = load_row(k + j * d2, dh);
    const float p = expf(dot(qr, kr) * scale - l);
    fma_row(acc, p * (dot(g, load_row(k + j * d2 + a.Hkv * a.dh, dh)) - dl) * scale, kr);
  }
  if (bad_length(n, (int)a.Tk))
    for (int e = 0; e < kJ; ++e) acc.v[e] = NAN;
  store_row(dq + u * a.dh, acc, dh);
  if ((threadIdx.x & 63) == 0) delta[at] = dl;
}

// One wave per state and key head, over the query rows of its heads.
__global__ __launch_bounds__(TPB) void dkv_kernel(const float* __restrict__ q,
                                                  const float* __restrict__ kv,
                                                  const int32_t* __restrict__ klen,
                                                  const float* __restrict__ lse,
                                                  const float* __restrict__ dy,
                                                  const float* __restrict__ delta,
                                                  float* __restrict__ dkv, AttendShape a,
                                                  float scale) {
  const int64_t u = (int64_t)blockIdx.x * (TPB / 64) + (threadIdx.x >> 6);
  if (u >= a.B * a.Tk * a.Hkv) return;
  const int64_t hk = u % a.Hkv, j = u / a.Hkv % a.Tk, b = u / a.Hkv / a.Tk, G = a.H / a.Hkv;
  const int n = klen[b], dh = (int)a.dh;
  const int64_t at = (b * a.Tk + j) * 2 * a.Hkv * a.dh + hk * a.dh, v = a.Hkv * a.dh;
  Row dk = {}, dv = {};
  if (bad_length(n, (int)a.Tk)) {
    for (int e = 0; e < kJ; ++e) dk.v[e] = dv.v[e] = NAN;
  } else if (j < n) {
    const Row kr = load_row(kv + at, dh), vr = load_row(kv + at + v, dh);
    for (int64_t h = hk * G; h < (hk + 1) * G; ++h)
      for (int64_t i = 0; i < a.Tq; ++i) {
        const int64_t row = ((b * a.Tq + i) * a.H + h) * a.dh, st = (b * a.H + h) * a.Tq + i;
        const Row qr = load_row(q + row, dh), g = load_row(dy + row, dh);
        const float p = expf(dot(qr, kr) * scale - lse[st]);
        fma_row(dv, p, g);
        fma_row(dk, p * (dot(g, vr) - delta[st]) * scale, qr);
      }
  }
  store_row(dkv + at, dk, dh);
  store_row(dkv + at + v, dv, dh);
}

unsigned waves(int64_t n) { return (unsigned)((n + TPB / 64 - 1) / (TPB / 64)); }

}  // namespace

int64_t attention_key_slices(const AttendShape&, bool) { return 1; }
int64_t attention_query_slices(const AttendShape&) { return 1; }

hipError_t cross_attention_fwd(const float* q, const float* kv, const int32_t* klen, float* y,
                               float* lse, float*, const AttendShape& a, int64_t, hipStream_t s) {
  hipLaunchKernelGGL(fwd_kernel, dim3(waves(a.B * a.Tq * a.H)), dim3(TPB), 0, s, q, kv, klen, y,
                     lse, a, 1.f / sqrtf((float)a.dh));
  return hipGetLastError();
}

hipError_t cross_attention_bwd(const float* q, const float* kv, const int32_t* klen,
                               const float* y, const float* lse, const float* dy, float* dq,
                               float* dkv, float* delta, float*, const AttendShape& a, int64_t,
                               int64_t, hipStream_t s) {
  const float scale = 1.f / sqrtf((float)a.dh);
  hipLaunchKernelGGL(dq_kernel, dim3(waves(a.B * a.Tq * a.H)), dim3(TPB), 0, s, q, kv, klen, y, lse,
                     dy, dq, delta, a, scale);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(dkv_kernel, dim3(waves(a.B * a.Tk * a.Hkv)), dim3(TPB), 0, s, q, kv, klen, lse,
                     dy, delta, dkv, a, scale);
  return hipGetLastError();
}

}  // namespace ooc

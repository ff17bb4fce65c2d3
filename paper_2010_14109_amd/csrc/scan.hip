// Gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) x_t with a = sigmoid(f), forward and
// backward, over sequences of any length (gfx950).
//
// Steps compose: a run of steps maps the state before it to A h + B, A the product of its gates, and
// runs join by (A2, B2) after (A1, B1) = (A1 A2, A2 B1 + B2).  The backward is the same recurrence
// from the last row to the first: with G_t = a_t (dh_t + G_(t+1)), the gradient of h_t is
// dh_t + G_(t+1).
//
// It is bound by memory traffic, 12 bytes a value forward (f, x read, h written) and 24 backward (f,
// x, h, dh read, df, dx written), if each value is read once.  So a workgroup keeps a stretch of rows
// in registers: a lane loads kSteps rows of its column, reduces them to (A, B), all runs of the
// stretch meet in LDS, each lane takes in the runs before its own and walks its rows with the state
// that it then knows.  Rows of the next stretch are on their way meanwhile.  Where the columns of all
// sequences do not fill the chip, time is cut into slices: a first pass reduces every slice to (A, B),
// and each workgroup of the second takes in the slices before its own.  24 x 512 x 1024: 30 us forward, 61
// backward, 5.0 TB/s; 1 x 32765 x 1365 in 47 slices: 140 and 267, behind first passes of 88 and 78.
//
// A gate of exactly zero (f far below) or a row that starts afresh cuts the state off, whatever it was, an
// infinity or a NaN too.  Such a run has a negative A, so that it is told from one whose product of gates is
// below fp32's range, which hands on what is not finite: which rows that reaches does not depend on
// how they are divided into runs.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "kernels.h"

namespace ooc {

namespace {


int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <int CL>
constexpr int kWaves = CL == 64 ? 8 : 16;   // of a workgroup, at most

constexpr uint32_t kXcds = 8;

struct Scan {
  int B, T, C, slices, slice_len;
  // Neighbours run on one die: where a row is no multiple of a cache line, they share lines.
  bool together;
};

// a = sigmoid(f) and 1 - a, each to a few units in its last place: with e = exp(-|f|), 1 / (1 + e) and
// e / (1 + e).  The exponent -|f| log2 e is split in a float and its remainder, whose part e takes in as 1 +
// x; the reciprocal is corrected once.  (The library's exponential and quotient, with more instructions:
// 24 x 512 x 1024 forward 33 us, 31 so.)
__device__ inline void gate_of(float f, float& a, float& rest) {
  constexpr float kLog2e = 1.44269504088896340736f, kLow = 1.92596299e-8f, kLn2 = 0.69314718055994530942f;
  const float x = -fabsf(f), t = x * kLog2e, low = fmaf(x, kLog2e, -t) + x * kLow;
  const float e0 = __builtin_amdgcn_exp2f(t), e = t < -126.f ? e0 : fmaf(e0 * low, kLn2, e0), d = 1.f + e;
  float r = __builtin_amdgcn_rcpf(d);
  r = fmaf(fmaf(-d, r, 1.f), r, r);
  const float er = e * r;
  a = f >= 0.f ? r : er;
  rest = f >= 0.f ? er : r;
}
// Whether a run cuts off what is before it, by the sign of A: its magnitude may fall to -0, and where A is a
// NaN, whatever its sign, B is one too.
__device__ inline bool cuts(float A) { return __builtin_bit_cast(int, A) < 0; }
// the state behind a run (A, B)
__device__ inline float after(float A, float B, float h) { return cuts(A) ? B : fmaf(A, h, B); }
// A of a run and what is before it
__device__ inline float gates(float A, float before) { return cuts(A) ? -1.f : A * before; }

// One lane's rows: column c, rows t0 .. of its sequence in the order of the pass (backward: from the
// last on), those at and past `end` being no rows (they change nothing).
template <bool BACK, int S>
struct Lane {
  float f[S], x[S], d[S], p[S];   // backward: d = dh, p = h of the row before
  int fresh[S];
  __device__ void load(const float* fx, const float* h0, const int32_t* fr, const float* h,
                       const float* dh, const Scan& s, int b, int c, int t0, int end, bool sum_only) {
    const int cc = min(c, s.C - 1);
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const int u = min(t0 + k, end - 1), t = BACK ? s.T - 1 - u : u;
      const int64_t row = (int64_t)b * s.T + t;
      const float* q = fx + row * 2 * s.C + cc;
      f[k] = q[0];
      if (!BACK || !sum_only) x[k] = q[s.C];
      fresh[k] = fr ? fr[row] : 0;
      if (BACK) {
        d[k] = dh[row * s.C + cc];
        if (!sum_only) {
          p[k] = 0.f;
          if (t > 0) p[k] = h[(row - 1) * s.C + cc];
          else if (h0) p[k] = h0[(int64_t)b * s.C + cc];
        }
      }
    }
  }
};

// SUM: only reduce the slice to (A, B), into part.
template <bool BACK, bool SUM, int S, int CL>
__global__ __launch_bounds__(64 * kWaves<CL>, 4) void scan_kernel(
    const float* __restrict__ fx, const float* __restrict__ h0, const int32_t* __restrict__ fr,
    const float* __restrict__ hin, const float* __restrict__ dh, float* __restrict__ out,
    float* __restrict__ dh0, float* __restrict__ part, Scan s) {
  constexpr int R = 64 / CL;   // runs of a wave
  __shared__ float2 runs[2][kWaves<CL>][CL];
  const int nw = blockDim.x >> 6, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, col = lane % CL, sub = lane / CL;
  const uint32_t blocks = (s.C + CL - 1) / CL, slices = SUM ? s.slices - 1 : s.slices;
  const uint32_t items = blocks * s.B * slices, id = blockIdx.x;
  const uint32_t item = s.together ? id % kXcds * (gridDim.x / kXcds) + id / kXcds : id;
  if (item >= items) return;
  const int b = item / blocks % s.B, c = (int)(item % blocks) * CL + col, slice = item / (blocks * s.B);
  const int begin = min(s.T, slice * s.slice_len), end = min(s.T, begin + s.slice_len);
  float state = 0.f, A_all = 1.f;
  if (!SUM) {
    if (!BACK && h0 && c < s.C) state = h0[(int64_t)b * s.C + c];
    if (c < s.C)
      for (int k = 0; k < slice; ++k) {
        const float* q = part + ((int64_t)b * s.slices + k) * 2 * s.C + c;
        state = after(q[0], q[s.C], state);
      }
  }
  Lane<BACK, S> next;
  if (begin < end) next.load(fx, h0, fr, hin, dh, s, b, c, begin + (w * R + sub) * S, end, SUM);
  int buf = 0;
  for (int r = begin; r < end; r += nw * R * S, buf ^= 1) {
    const int t0 = r + (w * R + sub) * S;
    float a[S], rest[S], al[S], B = 0.f, A = 1.f;
    const Lane<BACK, S> now = next;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      gate_of(now.f[k], a[k], rest[k]);
      al[k] = now.fresh[k] || a[k] == 0.f ? -1.f : a[k];
      if (t0 + k < end) {
        B = BACK ? (al[k] < 0.f ? 0.f : al[k] * (now.d[k] + B)) : after(al[k], rest[k] * now.x[k], B);
        A = gates(al[k], A);
      }
    }
    // the wave's runs up to a lane's own; the last one's are the wave's
    float A0 = 1.f, B0 = 0.f;
    if constexpr (R > 1) {
#pragma unroll
      for (int o = CL; o < 64; o *= 2) {
        const float a1 = __shfl_up(A, o, 64), b1 = __shfl_up(B, o, 64);
        if (lane >= o) {
          B = after(A, B, b1);
          A = gates(A, a1);
        }
      }
      A0 = __shfl_up(A, CL, 64);
      B0 = __shfl_up(B, CL, 64);
    }
    if (sub == R - 1) runs[buf][w][col] = make_float2(A, B);
    if (r + nw * R * S < end) next.load(fx, h0, fr, hin, dh, s, b, c, t0 + nw * R * S, end, SUM);
    __syncthreads();
    float mine = state;
    for (int k = 0; k < nw; ++k) {
      const float2 run = runs[buf][k][col];
      if (k == w) mine = state;
      state = after(run.x, run.y, state);
      A_all = gates(run.x, A_all);
    }
    if (R > 1 && sub) mine = after(A0, B0, mine);
    if (SUM || c >= s.C) continue;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      if (t0 + k >= end) break;
      const int t = BACK ? s.T - 1 - (t0 + k) : t0 + k;
      const int64_t row = (int64_t)b * s.T + t;
      if (!BACK) {
        mine = after(al[k], rest[k] * now.x[k], mine);
        out[row * s.C + c] = mine;
      } else {
        const float g = now.d[k] + mine, before = al[k] < 0.f ? 0.f : now.p[k];
        mine = al[k] < 0.f ? 0.f : al[k] * g;
        out[row * 2 * s.C + c] = g * (before - now.x[k]) * (a[k] * rest[k]);
        out[row * 2 * s.C + s.C + c] = rest[k] * g;
      }
    }
  }
  if (w || sub || c >= s.C) return;
  if (SUM) {
    float* q = part + ((int64_t)b * s.slices + slice) * 2 * s.C + c;
    q[0] = A_all;
    q[s.C] = state;
  } else if (BACK && dh0 && end == s.T && begin < s.T) {
    dh0[(int64_t)b * s.C + c] = state;
  }
}

// Rows of a lane, as many as leave a SIMD four waves with the next ones on their way; one where there
// is one.
constexpr int kSteps = 16, kBackSteps = 8;

// Columns of a workgroup: 64, a row's 256 bytes together; or 16, a wave holding four runs, where a
// sequence is over in two rounds of such workgroups and values are so few that launches count and not
// traffic (with gradients, 4 x 512 x 512: 24 us, 34 in slices of 64 columns; 16 x 512 x 512: 49 and 45; 2 x
// 2048 x 256: 51 and 34).
bool few(const ScanShape& a) { return a.T > 1 && a.T <= 1024 && a.B * a.T * a.C <= (1 << 21); }
// Rows of f and x that do not start with a cache line of 128 bytes.
bool odd_rows(const ScanShape& a) { return a.C % 32 != 0; }

template <bool BACK, int S, int CL>
hipError_t scan(const float* fx, const float* h0, const int32_t* fresh, const float* h, const float* dh,
                float* out, float* dh0, float* part, const ScanShape& a, int64_t slices,
                hipStream_t st) {
  const Scan s{(int)a.B, (int)a.T, (int)a.C, (int)slices, (int)ceil_div(a.T, slices), odd_rows(a)};
  const auto grid = [&](int64_t n) { return dim3((unsigned)(ceil_div(a.B * ceil_div(a.C, CL) * n, kXcds) * kXcds)); };
  const unsigned threads = 64 * (unsigned)std::min<int64_t>(kWaves<CL>, ceil_div(s.slice_len, S * 64 / CL));
  if (slices > 1) {
    hipLaunchKernelGGL((scan_kernel<BACK, true, S, CL>), grid(slices - 1), dim3(threads), 0, st,
                       fx, h0, fresh, h, dh, out, dh0, part, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((scan_kernel<BACK, false, S, CL>), grid(slices), dim3(threads), 0, st,
                     fx, h0, fresh, h, dh, out, dh0, part, s);
  return hipGetLastError();
}

}  // namespace

// Slices where the columns of all sequences are too few workgroups: some 512 of them, twice as many where
// neighbours share lines, and 128 rows or more in each.
int64_t scan_slices(const ScanShape& a) {
  const int64_t blocks = a.B * ceil_div(a.C, 64);
  if (few(a) || blocks >= 256) return 1;
  return std::max<int64_t>(1, std::min<int64_t>({ceil_div(odd_rows(a) ? 1024 : 512, blocks), a.T / 128,
                                                  kMaxScanSlices}));
}

hipError_t scan_fwd(const float* fx, const float* h0, const int32_t* fresh, float* h, float* part,
                    const ScanShape& a, int64_t slices, hipStream_t s) {
#define FWD(S, CL) scan<false, S, CL>(fx, h0, fresh, nullptr, nullptr, h, nullptr, part, a, slices, s)
  if (a.T == 1) return FWD(1, 64);
  return few(a) ? FWD(kSteps, 16) : FWD(kSteps, 64);
#undef FWD
}

hipError_t scan_bwd(const float* fx, const float* h0, const int32_t* fresh, const float* h,
                    const float* dh, float* dfx, float* dh0, float* part, const ScanShape& a,
                    int64_t slices, hipStream_t s) {
#define BWD(S, CL) scan<true, S, CL>(fx, h0, fresh, h, dh, dfx, dh0, part, a, slices, s)
  if (a.T == 1) return BWD(1, 64);
  return few(a) ? BWD(kBackSteps, 16) : BWD(kBackSteps, 64);
#undef BWD
}

}  // namespace ooc

// Cross attention: queries against the first klen states of their sequence (gfx950).
//
// One pass over the states with the running maximum and sum of the softmax; no matrix of scores is
// kept.  The backward recomputes the probabilities from the forward's row logarithms lse, in two
// passes, one over the states for dq and one over the queries for dk and dv, so that every sum has
// a fixed order and no two workgroups add to the same memory.
//
// Products.  All of it is fp32, and the fp32 matrix instructions run at a sixteenth of the fp16
// ones' rate.  A matrix (a column of the wave's own side, a tile of rows of the other) is scaled by
// a power of two that brings its largest value to 2^14 .. 2^15 and split into fp16 pieces, h =
// fp16(x), l = fp16(x - h); x y is the sum of h h, h l and l h, accumulated in fp32.  Three
// instructions where splitting into bfloat16 pieces takes six, two pieces to keep and move instead of
// three.  The scales are exact and multiply into factors that are applied anyway.  What is computed
// and multiplied again (probabilities, score gradients) is itself scaled by a running power of two
// per column: its values lie within 2^15, and sums are rescaled, as for the running maximum, in the
// rare tiles where one passes it.
//
// What that gives up against fp32, for the speed of three products instead of six: the pieces of a
// value are off by up to 2^-23 of it (fp32: 2^-24), and l l, up to 2^-22 of x y, is left out.  l has
// no bits below 2^-25, so a value 2^-16 and more below its matrix's largest is off by up to 2^-39 of
// that: of a column's own head columns, or of all head columns of a tile's 32 or 64 rows.  Likewise a
// probability or score gradient is off by up to 2^-35 of its column's largest (each times the power
// of two of the tile it meets; 2^-36 forward, see kTop): where a state that takes nearly all
// probability brings nothing itself, the others' part of y is off by 2^-36 / their probability.
//
// Tiles.  A wave owns 32 columns: of queries (forward, dq) or of states (dk, dv).  Their pieces stay
// in registers as the B operands of 32 x 32 x 16 products.  The other side passes through LDS in
// tiles of rows, split once for the four waves of a workgroup.  Products are formed transposed
// (rows of the tile x own columns), so a lane holds 16 rows of one column: the softmax's maximum
// and sum take one exchange between the two halves of a wave, and the probabilities are already
// the B operand of the next product, up to the order of its terms, in which the A operand (the same
// tile, read through the transposing LDS loads) follows.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "kernels.h"

namespace ooc {

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr uint32_t kNone = 0x80000000u;   // past the length of every descriptor
constexpr uint32_t kXcds = 8;

// A width of head columns, padded to DH: a piece's row is DH / 8 chunks of 16 bytes in kRow bytes.
// The odd number of chunks a row is long spreads the 16 rows of 256 bytes' worth of row reads over
// all banks, and the four rows of a transposing read too.
template <int DH>
struct Width {
  static constexpr int kSteps = DH / 16;                  // 16-wide products over the head columns
  static constexpr int kBlocks = DH / 32;                 // 32-row blocks of head columns
  static constexpr int kChunks = DH / 8;
  static constexpr int kLanes = DH == 32 ? 4 : DH == 64 ? 8 : DH <= 128 ? 16 : 32;   // that load a row
  static constexpr int kRow = (DH == 32 ? 7 : DH == 64 ? 9 : DH == 96 ? 13 : DH == 128 ? 19 : 35) * 16;
  // The forward: rows of a tile, waves that share columns, each with its part of the sums (where
  // registers hold no more), blocks it then sums.
  static constexpr int kTile = DH <= 64 ? 64 : 32;
  static constexpr int kParts = DH <= 128 ? 1 : 2;
  static constexpr int kSums = kBlocks / kParts;
  // The backward up to 64 head columns: rows of a tile, waves of a workgroup.
  static constexpr int kBackTile = 64, kBackWaves = 4;
  // The backward above, by pairs of waves: waves of a workgroup, tile buffers, waves a SIMD holds.
  static constexpr int kPairWaves = DH <= 128 ? 8 : 4;
  static constexpr int kBuffers = DH <= 128 ? 2 : 1;
  static constexpr int kOccupancy = DH <= 128 ? 2 : 1;
  static constexpr int kBackCols = DH <= 64 ? 32 * kBackWaves : 16 * kPairWaves;
  static constexpr int kBackRows = DH <= 64 ? kBackTile : 32;
};

// ---------------------------------------------------------------- exchange between lanes
// the values of the two lanes 32 apart, the lower one's first
__device__ inline floatx2 halves(float x) {
  const uint32_t v = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  const uint32_t lo = r[0], hi = r[1];   // a bit_cast of a vector's element takes its first
  return {__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi)};
}
__device__ inline float max_of_halves(float x) {
  const floatx2 r = halves(x);
  return fmaxf(r[0], r[1]);
}
__device__ inline float sum_of_halves(float x) {
  const floatx2 r = halves(x);
  return r[0] + r[1];
}
template <int CTRL>
__device__ inline float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL,
                                                               0xf, 0xf, true));
}
// largest of the wave's values (>= 0)
__device__ inline float wave_max(float x) {
  x = fmaxf(x, dpp<0xb1>(x));    // quad_perm 1 0 3 2
  x = fmaxf(x, dpp<0x4e>(x));    // quad_perm 2 3 0 1
  x = fmaxf(x, dpp<0x141>(x));   // mirrored within 8
  x = fmaxf(x, dpp<0x140>(x));   // mirrored within 16
  const uint32_t v = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const uint32_t a = r[0], b = r[1];
  return max_of_halves(fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
}

// ---------------------------------------------------------------- scaled pieces
__device__ inline float exp2_of(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }
// floor(log2 x) of x >= 0, at least -112 and at most 128: with it 2^(14 - e) and 2^(e - 14) are
// normal numbers
__device__ inline int exponent(float x) {
  return max((int)(__builtin_bit_cast(uint32_t, x) >> 23) - 127, -112);
}

struct Pieces {
  half8v h, l;
};
// x scale = h + l.  The remainders are single instructions (fma of fp32 and fp16 operands, rounded
// to fp16); as a literal, a factor of 1 would be folded into a conversion and a subtraction.
__device__ inline void split2(float x, float y, float scale, uint32_t& h, uint32_t& l) {
  const half2v hh = __builtin_convertvector((floatx2){x * scale, y * scale}, half2v);
  half2v ll;
  ll[0] = (_Float16)__builtin_fmaf(x, scale, -(float)hh[0]);
  ll[1] = (_Float16)__builtin_fmaf(y, scale, -(float)hh[1]);
  h = __builtin_bit_cast(uint32_t, hh);
  l = __builtin_bit_cast(uint32_t, ll);
}
__device__ inline Pieces split8(const float* v, float scale) {
  uint4 h, l;
  split2(v[0], v[1], scale, h.x, l.x);
  split2(v[2], v[3], scale, h.y, l.y);
  split2(v[4], v[5], scale, h.z, l.z);
  split2(v[6], v[7], scale, h.w, l.w);
  return {__builtin_bit_cast(half8v, h), __builtin_bit_cast(half8v, l)};
}
// the same of values in fp16's range
__device__ inline Pieces split8(const float* v) {
  float one = 1.f;
  asm("" : "+s"(one));
  uint4 h, l;
  uint32_t* hp[4] = {&h.x, &h.y, &h.z, &h.w};
  uint32_t* lp[4] = {&l.x, &l.y, &l.z, &l.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const half2v hh = __builtin_convertvector((floatx2){v[2 * i], v[2 * i + 1]}, half2v);
    half2v ll;
    ll[0] = (_Float16)__builtin_fmaf(v[2 * i], one, -(float)hh[0]);
    ll[1] = (_Float16)__builtin_fmaf(v[2 * i + 1], one, -(float)hh[1]);
    *hp[i] = __builtin_bit_cast(uint32_t, hh);
    *lp[i] = __builtin_bit_cast(uint32_t, ll);
  }
  return {__builtin_bit_cast(half8v, h), __builtin_bit_cast(half8v, l)};
}
__device__ inline float max_abs(const float* v, int n) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < n; ++e) m = fmaxf(m, fabsf(v[e]));
  return m;
}

__device__ inline floatx16 mma(half8v a, half8v b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ inline floatx16 mma(const Pieces& a, const Pieces& b, floatx16 c) {
  c = mma(a.l, b.h, c);
  c = mma(a.h, b.l, c);
  return mma(a.h, b.h, c);
}

// ---------------------------------------------------------------- rows of memory
__device__ inline __amdgpu_buffer_rsrc_t buffer(const float* p, int64_t values) {
  const int64_t n = values < 0 ? 0 : values > (int64_t(1) << 29) ? (int64_t(1) << 29) : values;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p), 0, (int)((uint32_t)n * 4u),
                                           0x00020000);
}
// eight values at a byte offset (of any 4-byte alignment); what lies past the length is zero.  (Both
// offsets are the lane's, which the length is compared with.)
__device__ inline void load8(__amdgpu_buffer_rsrc_t r, uint32_t off, float* v) {
  const float4 a = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0));
  const float4 b = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(off + 16u), 0, 0));
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
// four values at a 4-byte aligned address
typedef float floatx4u __attribute__((ext_vector_type(4), aligned(4)));

// columns at and past dh of the eight from d on are zero
template <bool EXACT>
__device__ inline void trim(float* v, int d, int dh) {
  if constexpr (!EXACT) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = d + e < dh ? v[e] : 0.f;
  }
}

// The query rows of a key head are numbered g Tq + i over its G heads and their positions.
struct Shape {
  int B, Tq, Tk, H, Hkv, G, dh;
  int R;                // G Tq
  int64_t ldq, ldk;     // H dh, 2 Hkv dh
  float scale;          // 1 / sqrt(dh)
};
__device__ inline int64_t query_row(const Shape& s, int b, int hk, int r) {
  const int g = r / s.Tq, i = r - g * s.Tq;
  return ((int64_t)b * s.Tq + i) * s.ldq + (int64_t)(hk * s.G + g) * s.dh;
}
__device__ inline int64_t key_row(const Shape& s, int b, int hk, int j) {
  return ((int64_t)b * s.Tk + j) * s.ldk + (int64_t)hk * s.dh;
}
__device__ inline int64_t stat_row(const Shape& s, int b, int hk) {
  return ((int64_t)b * s.H + (int64_t)hk * s.G) * s.Tq;
}

// head columns d .. d + 7 of the row at p, zero past the last
template <bool EXACT>
__device__ inline void load_eight(const float* p, int d, int dh, float* v) {
  if (EXACT || d + 8 <= dh) {
    const floatx4u a = *reinterpret_cast<const floatx4u*>(p + d), b = *reinterpret_cast<const floatx4u*>(p + d + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = a[e];
      v[4 + e] = b[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = d + e < dh ? p[d + e] : 0.f;
  }
}

// A wave's own columns: lane l holds column l mod 32, head columns 16 s + 8 (l / 32) .. + 8 of every
// step s.  p: the column's row (a column past the last takes the last one's; it is not stored).
template <int DH, bool EXACT>
__device__ inline void load_column(const float* p, int dh, float (&v)[DH / 2]) {
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int s = 0; s < DH / 16; ++s) load_eight<EXACT>(p, 16 * s + 8 * half, dh, v + 8 * s);
}
// Returns the inverse scale.
template <int DH>
__device__ inline float split_column(const float (&v)[DH / 2], Pieces (&o)[DH / 16]) {
  float m = max_abs(v, DH / 2);
  m = max_of_halves(m);
  const int e = exponent(m);
  const float scale = exp2_of(14 - e);
#pragma unroll
  for (int s = 0; s < DH / 16; ++s) o[s] = split8(v + 8 * s, scale);
  return exp2_of(e - 14);
}

// One matrix of a tile: T rows of pieces in LDS.
template <int DH, int T>
struct Rows {
  using Wd = Width<DH>;
  static constexpr int kPiece = T * Wd::kRow;
  static constexpr int kBytes = 2 * kPiece;
  static __device__ void store(char* lds, int row, int c, const Pieces& p) {
    *reinterpret_cast<half8v*>(lds + row * Wd::kRow + c * 16) = p.h;
    *reinterpret_cast<half8v*>(lds + kPiece + row * Wd::kRow + c * 16) = p.l;
  }
  // A operand, rows r0 .. r0 + 31 of the tile x step s of the head columns
  static __device__ Pieces by_row(const char* lds, int r0, int s) {
    const int l = threadIdx.x & 63;
    const char* p = lds + (r0 + (l & 31)) * Wd::kRow + (2 * s + (l >> 5)) * 16;
    return {*reinterpret_cast<const half8v*>(p), *reinterpret_cast<const half8v*>(p + kPiece)};
  }
  // A operand, head columns 32 block .. + 31 x the 16 rows r0 .. of the tile, in the order in which
  // a lane of a 32 x 32 result holds rows: half h of the wave has rows 4 h .. + 3 and 8 + 4 h .. + 3
  static __device__ half8v transposed(const char* lds, int r0, int block) {
    const int l = threadIdx.x & 63, t = l & 15;
    const char* p = lds + (r0 + 4 * (l >> 5) + (t >> 2)) * Wd::kRow +
                    (32 * block + 16 * ((l >> 4) & 1) + 4 * (t & 3)) * 2;
    typedef __attribute__((address_space(3))) short4v* Lds;
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p);
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 8 * Wd::kRow));
    const half4v x = __builtin_bit_cast(half4v, a), y = __builtin_bit_cast(half4v, b);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ Pieces by_column(const char* lds, int r0, int block) {
    return {transposed(lds, r0, block), transposed(lds + kPiece, r0, block)};
  }
  // the same for 16 x 16 x 32: head columns 16 block .. + 15 x all 32 rows, quarter g of the wave
  // having rows 4 g .. + 3 and 16 + 4 g .. + 3
  static __device__ half8v transposed16(const char* lds, int block) {
    const int l = threadIdx.x & 63, t = l & 15;
    const char* p = lds + (4 * (l >> 4) + (t >> 2)) * Wd::kRow + (16 * block + 4 * (t & 3)) * 2;
    typedef __attribute__((address_space(3))) short4v* Lds;
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p);
    const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 16 * Wd::kRow));
    const half4v x = __builtin_bit_cast(half4v, a), y = __builtin_bit_cast(half4v, b);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ Pieces by_column16(const char* lds, int block) {
    return {transposed16(lds, block), transposed16(lds + kPiece, block)};
  }
};

// The workgroup's place: pairs (b, key head), tiles of columns, slices of the other side.  The
// tiles of a pair run on one die, whose L2 then holds the pair's states (or queries).
struct Place {
  int b, hk, tile, slice;
  bool none;
};
__device__ inline Place place(const Shape& s, int tiles) {
  const uint32_t pairs = (uint32_t)s.B * s.Hkv, id = blockIdx.x;
  const uint32_t idx = id / kXcds, pair = idx / tiles * kXcds + id % kXcds;
  return {(int)(pair / s.Hkv), (int)(pair % s.Hkv), (int)(idx % tiles), (int)blockIdx.y, pair >= pairs};
}

// Sum t of a lane holds, in r, head column 32 (first + t) + 8 (r / 4) + 4 half + r % 4 of its column.
template <int N, bool EXACT, class F>
__device__ inline void store_column(float* p, int first, int dh, F value) {
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int d = 32 * (first + t) + 8 * q + 4 * half;
      if (EXACT || d + 4 <= dh) {
        *reinterpret_cast<floatx4u*>(p + d) =
            floatx4u{value(t, 4 * q), value(t, 4 * q + 1), value(t, 4 * q + 2), value(t, 4 * q + 3)};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (d + e < dh) p[d + e] = value(t, 4 * q + e);
      }
    }
}

__device__ inline float4 at4(const float* lds, int row) {
  return *reinterpret_cast<const float4*>(lds + row);
}
__device__ inline float pick(const float4& v, int e) {
  return e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w;
}

// What a masked row's score becomes, for the last tile of a sequence: rows at and past `left`.
__device__ inline void mask_rows(floatx16& a, int r0, int left) {
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int i = 0; i < 16; ++i) a[i] = r0 + 8 * (i / 4) + 4 * half + i % 4 < left ? a[i] : -INFINITY;
}

// The values of two matrices' next tile of T rows on their way from memory to LDS, W waves a
// workgroup: a thread holds units of 8 head columns, of the rows of the first matrix, then of the
// second.  The matrix of a unit is uniform over a wave, as T rows are whole waves' worth.
template <int DH, int W, int T>
struct Raw {
  using Wd = Width<DH>;
  static constexpr int kThreads = 64 * W;
  static constexpr int kLanes = Wd::kLanes;
  static constexpr int kUnits = (2 * T * kLanes + kThreads - 1) / kThreads;
  static_assert(T * kLanes % 64 == 0, "a wave's units are of one matrix");
  float v[kUnits][8];
  static __device__ int row(int u) { return ((int)threadIdx.x + u * kThreads) / kLanes; }
  static __device__ bool second(int u) { return __builtin_amdgcn_readfirstlane(row(u)) >= T; }
  static __device__ bool idle(int u) {
    return 2 * T * kLanes % kThreads && __builtin_amdgcn_readfirstlane(row(u)) >= 2 * T;
  }
  static __device__ int chunk() { return (int)threadIdx.x % kLanes; }
  // a, b: the matrices from the tile's first row on, ld values a row's distance, `rows` of them there
  template <bool EXACT>
  __device__ void load(const float* a, const float* b, int64_t ld, int rows, int dh) {
    const int64_t len = rows > 0 ? (int64_t)(min(rows, T) - 1) * ld + dh : 0;
    const auto ra = buffer(a, len), rb = buffer(b, len);
    const int c = chunk();
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int r = row(u) % T;
      uint32_t off = (uint32_t)(r * ld + 8 * c) * 4u;
      if (r >= rows || 8 * c >= dh || idle(u)) off = kNone;
      load8(second(u) ? rb : ra, off, v[u]);
      trim<EXACT>(v[u], 8 * c, dh);
    }
  }
  // rows i .. of the group's heads, numbered g Tq + position; a, b: position 0 of its first head
  template <bool EXACT>
  __device__ void load_packed(const float* a, const float* b, const Shape& s, int i, int rows) {
    const int64_t len = (int64_t)(s.Tq - 1) * s.ldq + (int64_t)s.G * s.dh;
    const auto ra = buffer(a, len), rb = buffer(b, len);
    const int c = chunk();
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int r = row(u) % T, g = (i + r) / s.Tq, k = i + r - g * s.Tq;
      uint32_t off = (uint32_t)(k * s.ldq + (int64_t)g * s.dh + 8 * c) * 4u;
      if (r >= rows || 8 * c >= s.dh || idle(u)) off = kNone;
      load8(second(u) ? rb : ra, off, v[u]);
      trim<EXACT>(v[u], 8 * c, s.dh);
    }
  }
  // The wave's largest finite values of the two matrices.  An infinity does not count: the other
  // values keep their pieces, and its remainder is a NaN that reaches whatever reads it.
  __device__ void publish(floatx2* tops) const {
    float ma = 0.f, mb = 0.f;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const float m = max_abs(v[u], 8);
      if (second(u)) mb = fmaxf(mb, m);
      else ma = fmaxf(ma, m);
    }
    if (__any(fmaxf(ma, mb) == INFINITY)) {
      ma = mb = 0.f;
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float x = fabsf(v[u][k]), m = x < INFINITY ? x : 0.f;
          if (second(u)) mb = fmaxf(mb, m);
          else ma = fmaxf(ma, m);
        }
    }
    ma = wave_max(ma);
    mb = wave_max(mb);
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = {ma, mb};
  }
  // The exponents of the tiles' largest values, from what every wave has published.
  static __device__ int2 exponents(const floatx2* tops) {
    float ma = 0.f, mb = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      ma = fmaxf(ma, tops[k][0]);
      mb = fmaxf(mb, tops[k][1]);
    }
    return {exponent(ma), exponent(mb)};
  }
  __device__ void store(char* a, char* b, int2 e) const {
    const float sa = exp2_of(14 - e.x), sb = exp2_of(14 - e.y);
    const int c = chunk();
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const Pieces p = split8(v[u], second(u) ? sb : sa);
      if ((kLanes == Wd::kChunks || c < Wd::kChunks) && !idle(u))
        Rows<DH, T>::store(second(u) ? b : a, row(u) % T, c, p);
    }
  }
};

// ---------------------------------------------------------------- forward
// The running softmax of a column, in powers of two and apart for the two sums it divides, as a
// tile's values bring an exponent of their own (ve of Raw::exponents, -112 for zeros).  ms is a whole
// number no more than kLag below the largest score, and the sum of probabilities is in units of 2^ms.
// d is a whole number, and ms + d no more than kRoom below the largest score + ve: a probability meets
// the values' pieces as p = 2^(score - ms - d + ve + kTop), so that p is at most 2^15 and the largest are
// above 2^11; of one below 2^-2 its pieces hold what is above 2^-25, 2^-36 of the largest or less.  Both are
// whole so that changing them is exact.  (More room, from 2^8 up, would rescale less often: 1 % of
// 24 x 512 x 512, nothing elsewhere, for four bits of small p.)
//
// Two rare cases take the terms apart: p too far below the units of the sum (d - ve past kFar: other
// tiles' values are far larger, or this one's are zero, and p may vanish while the probability counts),
// and scores from kLarge on: a score is a product a c, rounded where the largest is taken and exact in
// fma(a, c, ..), and the difference could take p out of its room, d and ve be lost beside ms.  There
// each score is rounded, ms taken off, and the probability computed for the sum alone.
constexpr float kTop = 12.f, kRoom = 3.f, kLag = 64.f, kFar = 64.f, kLarge = 0x1p22f;
__device__ inline bool outgrown(float top, float ve, float d, float ms) {
  const float t = top - ms;
  return t + ve > d + kRoom || t > kLag;
}
// d and ms for a tile with the largest score `top`; returns the factor of the sums with d
__device__ inline float raise(float top, float ve, float& d, float& ms, float& sum) {
  const float us = fmaxf(ms, ceilf(top)), by = ms == us ? 0.f : ms - us;
  const float now = d + by, up = fmaxf(now, ceilf(top - us + ve));
  sum *= exp2f(by);
  ms = us;
  d = up;
  return now == up ? 1.f : exp2f(now - up);
}
// a c, rounded: without the barrier the compiler makes one fma of the product and a subtraction behind it
__device__ inline float score(float a, float c) {
  float t = a * c;
  asm("" : "+v"(t));
  return t;
}
// What turns a column's sum of p times scaled values into its quotient by `total`, a factor, and log2
// of the sum of 2^score.  The factor is 2^(d - 26) / total, total's power of two taken into the
// exponent; where that is below the normal numbers' (values below 2^-94 times the states that share the
// weight), the sum takes kDown of it.
struct Quotient {
  static constexpr float kDown = 0x1p-60f;
  float factor, log;
  bool low;
  __device__ Quotient(float total, float d, float ms) {
    const float l = __builtin_amdgcn_logf(total), whole = rintf(l), e = d - (kTop + 14.f) - whole;
    low = e < -120.f;
    factor = __builtin_amdgcn_exp2f(low ? e + 60.f : e) / (total * __builtin_amdgcn_exp2f(-whole));
    log = ms + l;
  }
};

// A workgroup of wide() has 256 columns: up to 64 head columns two sets of 32 a wave, so that each
// A operand is read for both; above, eight waves, so that a tile is split once for all. Others have
// 128 (above 128 head columns, 64).
template <int DH, bool WIDE>
struct Forward {
  static constexpr int kWaves = WIDE && DH > 64 ? 8 : 4;
  static constexpr int kSets = WIDE && DH <= 64 ? 2 : 1;
  static constexpr int kCols = 32 * kWaves * kSets / Width<DH>::kParts;
};
template <int DH, bool EXACT, bool WIDE>
__global__ __launch_bounds__((64 * Forward<DH, WIDE>::kWaves), DH <= 128 ? 2 : 1) void fwd_kernel(
    const float* __restrict__ q, const float* __restrict__ kv, const int32_t* __restrict__ klen,
    float* __restrict__ y, float* __restrict__ lse, Shape s, int tiles, int slice_len,
    int64_t y_slice, int64_t lse_slice) {
  using Wd = Width<DH>;
  constexpr int T = Wd::kTile, W = Forward<DH, WIDE>::kWaves, C = Forward<DH, WIDE>::kSets;
  using Rw = Rows<DH, T>;
  __shared__ __attribute__((aligned(16))) char ks[Rw::kBytes];
  __shared__ __attribute__((aligned(16))) char vs[Rw::kBytes];
  __shared__ floatx2 tops[W];
  const Place at = place(s, tiles);
  if (at.none) return;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  const int col0 = at.tile * Forward<DH, WIDE>::kCols + w / Wd::kParts * 32 * C + (lane & 31);
  const int first = w % Wd::kParts * Wd::kSums;
  const int n = klen[at.b];
  const bool bad = n < 0 || n > s.Tk;
  const int k0 = bad ? 0 : min(n, at.slice * slice_len), k1 = bad ? 0 : min(n, k0 + slice_len);

  Pieces qp[C][Wd::kSteps];
  float qc[C];
#pragma unroll
  for (int x = 0; x < C; ++x) {
    float v[DH / 2];
    load_column<DH, EXACT>(q + query_row(s, at.b, at.hk, min(col0 + 32 * x, s.R - 1)), s.dh, v);
    qc[x] = split_column<DH>(v, qp[x]) * s.scale * kLog2e;
  }
  floatx16 o[C][Wd::kSums];
  float d[C], ms[C], sum[C];   // see kTop
#pragma unroll
  for (int x = 0; x < C; ++x) {
    d[x] = ms[x] = -INFINITY;
    sum[x] = 0.f;
#pragma unroll
    for (int t = 0; t < Wd::kSums; ++t) o[x][t] = floatx16{};
  }
  Raw<DH, W, T> raw;
  const auto fetch = [&](int j) {
    const int64_t r = key_row(s, at.b, at.hk, j);
    raw.template load<EXACT>(kv + r, kv + r + (int64_t)s.Hkv * s.dh, s.ldk, k1 - j, s.dh);
  };
  if (k0 < k1) fetch(k0);
  for (int j0 = k0; j0 < k1; j0 += T) {
    raw.publish(tops);
    __syncthreads();
    const int2 e = raw.exponents(tops);
    raw.store(ks, vs, e);
    __syncthreads();
    if (j0 + T < k1) fetch(j0 + T);
    const float ve = (float)e.y;
#pragma unroll 1
    for (int r0 = 0; r0 < T; r0 += 32) {
      if (r0 && j0 + r0 >= k1) break;
      floatx16 a[C];
#pragma unroll
      for (int x = 0; x < C; ++x) a[x] = floatx16{};
#pragma unroll
      for (int t = 0; t < Wd::kSteps; ++t) {
        const Pieces k = Rw::by_row(ks, r0, t);
#pragma unroll
        for (int x = 0; x < C; ++x) a[x] = mma(k, qp[x][t], a[x]);
      }
      if (j0 + r0 + 32 > k1)
#pragma unroll
        for (int x = 0; x < C; ++x) mask_rows(a[x], r0, k1 - j0);
      float c[C], top[C];
      bool past = false;
#pragma unroll
      for (int x = 0; x < C; ++x) {
        // (no smaller than the normal numbers: a masked score stays -inf)
        c[x] = fmaxf(qc[x] * exp2_of(e.x - 14), 0x1p-126f);
        top[x] = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) top[x] = fmaxf(top[x], a[x][i]);
        top[x] = score(max_of_halves(top[x]), c[x]);
        past |= outgrown(top[x], ve, d[x], ms[x]);
      }
      if (__builtin_expect(__any(past), 0))
#pragma unroll
        for (int x = 0; x < C; ++x) {
          const float f = raise(top[x], ve, d[x], ms[x], sum[x]);
#pragma unroll
          for (int t = 0; t < Wd::kSums; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[x][t][i] *= f;
        }
      Pieces pp[C][2];
#pragma unroll
      for (int x = 0; x < C; ++x) {
        const float far = d[x] - ve;
        const bool apart = __any(far > kFar || fabsf(ms[x]) > kLarge);
        float base = -ms[x], p[16], part = 0.f, alone = 0.f;
        if (__builtin_expect(apart, 0)) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            a[x][i] = score(a[x][i], c[x]) - ms[x];
            alone += __builtin_amdgcn_exp2f(a[x][i]);
          }
          c[x] = 1.f;
          base = 0.f;
        }
        const float off = base - (far - kTop);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          p[i] = __builtin_amdgcn_exp2f(fmaf(a[x][i], c[x], off));
          part += p[i];
        }
        sum[x] = apart ? sum[x] + alone : fmaf(part, __builtin_amdgcn_exp2f(far - kTop), sum[x]);
        pp[x][0] = split8(p);
        pp[x][1] = split8(p + 8);
      }
#pragma unroll
      for (int t = 0; t < Wd::kSums; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const Pieces v = Rw::by_column(vs, r0 + 16 * h, first + t);
#pragma unroll
          for (int x = 0; x < C; ++x) o[x][t] = mma(v, pp[x][h], o[x][t]);
        }
    }
  }
#pragma unroll
  for (int x = 0; x < C; ++x) {
    const float total = sum_of_halves(sum[x]);
    const int col = col0 + 32 * x;
    if (col >= s.R) continue;
    const float none = bad ? NAN : 0.f;
    const Quotient f(total, d[x], ms[x]);
    if (__any(f.low))
#pragma unroll
      for (int t = 0; t < Wd::kSums; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[x][t][i] *= f.low ? Quotient::kDown : 1.f;
    store_column<Wd::kSums, EXACT>(y + at.slice * y_slice + query_row(s, at.b, at.hk, col), first, s.dh,
                                   [&](int t, int i) { return k0 < k1 ? o[x][t][i] * f.factor : none; });
    if (half == 0 && first == 0)
      lse[at.slice * lse_slice + stat_row(s, at.b, at.hk) + col] =
          bad ? NAN : k0 < k1 ? f.log * kLn2 : -INFINITY;
  }
}

// ---------------------------------------------------------------- forward of a few queries
// A key head with at most 16 query rows (a token of each sequence and its group's heads) is bound by
// reading the states once.  Each wave takes tiles of 32 states of its own, without barriers: k goes
// from memory straight into the A operand, v through the wave's part of LDS.  A workgroup's waves
// and then the slices join their results.  Products are 16 x 16 x 32: 16 columns are all there is,
// and half the registers of 32 let a SIMD hold three waves, where there are as many.
// One token of 8 sequences of up to 4096 states, 16 heads of 64 on 4 key heads: 33.9 us with the
// kernel for many queries, 18 with this one (14, and 4 for the join; reading the 34 MB at the rate of
// a large copy takes 7).
constexpr int kFewWaves = 4, kFewRows = 16;
typedef float floatx4 __attribute__((ext_vector_type(4)));
__device__ inline floatx4 mma16(const Pieces& a, const Pieces& b, floatx4 c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.l, b.h, c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.l, c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.h, c, 0, 0, 0);
}
// over the four lanes 16 apart
__device__ inline float max_of_quarters(float x) {
  const uint32_t v = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const uint32_t a = r[0], b = r[1];
  return max_of_halves(fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
}
__device__ inline float sum_of_quarters(float x) {
  const uint32_t v = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  const uint32_t a = r[0], b = r[1];
  return sum_of_halves(__builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
}

template <int DH, bool EXACT>
__global__ __launch_bounds__(64 * kFewWaves, DH <= 64 ? 3 : 2) void few_kernel(
    const float* __restrict__ q, const float* __restrict__ kv, const int32_t* __restrict__ klen,
    float* __restrict__ y, float* __restrict__ lse, Shape s, int tiles, int slice_len,
    int64_t y_slice, int64_t lse_slice) {
  constexpr int T = 32, W = kFewWaves, kSteps = DH / 32, kBlocks = DH / 16;
  __shared__ __attribute__((aligned(16))) char mine[W][Rows<DH, T>::kBytes];
  __shared__ float ls[W][kFewRows];
  // a wave's results take its tile's place
  constexpr int kYs = DH + 4;
  static_assert(kFewRows * kYs * 4 <= Rows<DH, T>::kBytes, "room for the results");
  const auto ys = [&](int wave, int r, int d) -> float* {
    return reinterpret_cast<float*>(mine[wave]) + r * kYs + d;
  };
  const Place at = place(s, tiles);
  if (at.none) return;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, quarter = lane >> 4, l16 = lane & 15;
  const int n = klen[at.b];
  const bool bad = n < 0 || n > s.Tk;
  const int k0 = bad ? 0 : min(n, at.slice * slice_len), k1 = bad ? 0 : min(n, k0 + slice_len);

  // a lane's values of a tile: rows l mod 16 and 16 more, head columns 32 t + 8 (l / 16) .. + 8
  float k[DH / 2], v[DH / 2];
  const auto load_tile = [&](int j, int64_t to, float (&x)[DH / 2]) {
    const auto r = buffer(kv + key_row(s, at.b, at.hk, min(j, s.Tk - 1)) + to,
                          j < k1 ? (int64_t)(min(T, k1 - j) - 1) * s.ldk + s.dh : 0);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < kSteps; ++t) {
        const int d = 32 * t + 8 * quarter, row = 16 * h + l16;
        float* o = x + 8 * (h * kSteps + t);
        load8(r, row < k1 - j && d < s.dh ? (uint32_t)(row * s.ldk + d) * 4u : kNone, o);
        trim<EXACT>(o, d, s.dh);
      }
  };
  const int64_t to_v = (int64_t)s.Hkv * s.dh;
  char* vs = mine[w];
  const int j1 = k0 + w * T;
  load_tile(j1, 0, k);
  load_tile(j1, to_v, v);

  Pieces qp[kSteps];
  float qc;
  {
    const float* p = q + query_row(s, at.b, at.hk, min(l16, s.R - 1));
    float x[DH / 4];
#pragma unroll
    for (int t = 0; t < kSteps; ++t) load_eight<EXACT>(p, 32 * t + 8 * quarter, s.dh, x + 8 * t);
    const int e = exponent(max_of_quarters(max_abs(x, DH / 4)));
#pragma unroll
    for (int t = 0; t < kSteps; ++t) qp[t] = split8(x + 8 * t, exp2_of(14 - e));
    qc = exp2_of(e - 14) * s.scale * kLog2e;
  }
  floatx4 o[kBlocks];
#pragma unroll
  for (int t = 0; t < kBlocks; ++t) o[t] = floatx4{};
  float d = -INFINITY, ms = -INFINITY, sum = 0.f;   // see kTop
  const auto largest = [&](const float (&x)[DH / 2]) {
    float top = max_abs(x, DH / 2);
    if (__any(top == INFINITY)) {   // the largest finite one: see Raw::publish
      top = 0.f;
#pragma unroll
      for (int i = 0; i < DH / 2; ++i) top = fmaxf(top, fabsf(x[i]) < INFINITY ? fabsf(x[i]) : 0.f);
    }
    return exponent(wave_max(top));
  };
  for (int j0 = j1; j0 < k1; j0 += W * T) {
    const int ek = largest(k);
    floatx4 a[2] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < kSteps; ++t)
        a[h] = mma16(split8(k + 8 * (h * kSteps + t), exp2_of(14 - ek)), qp[t], a[h]);
    load_tile(j0 + W * T, 0, k);
    const int ev = largest(v);
    // (the wave's LDS accesses stay in order; the fences keep the compiler from moving them)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < kSteps; ++t)
        Rows<DH, T>::store(vs, 16 * h + l16, 4 * t + quarter, split8(v + 8 * (h * kSteps + t), exp2_of(14 - ev)));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    load_tile(j0 + W * T, to_v, v);
    float c = fmaxf(qc * exp2_of(ek - 14), 0x1p-126f);   // a masked score stays -inf
    const float ve = (float)ev;
    float p[8], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool there = 16 * (i / 4) + 4 * quarter + i % 4 < k1 - j0;
      p[i] = there ? a[i / 4][i % 4] : -INFINITY;
      top = fmaxf(top, p[i]);
    }
    top = score(max_of_quarters(top), c);
    if (__builtin_expect(__any(outgrown(top, ve, d, ms)), 0)) {
      const float f = raise(top, ve, d, ms, sum);
#pragma unroll
      for (int t = 0; t < kBlocks; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] *= f;
    }
    const float far = d - ve;
    const bool apart = __any(far > kFar || fabsf(ms) > kLarge);
    float base = -ms, part = 0.f, alone = 0.f;
    if (__builtin_expect(apart, 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = score(p[i], c) - ms;
        alone += __builtin_amdgcn_exp2f(p[i]);
      }
      c = 1.f;
      base = 0.f;
    }
    const float off = base - (far - kTop);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(p[i], c, off));
      part += p[i];
    }
    sum = apart ? sum + alone : fmaf(part, __builtin_amdgcn_exp2f(far - kTop), sum);
    const Pieces pp = split8(p);
#pragma unroll
    for (int t = 0; t < kBlocks; ++t) o[t] = mma16(Rows<DH, T>::by_column16(vs, t), pp, o[t]);
  }
  sum = sum_of_quarters(sum);
  const Quotient f(sum, d, ms);
  const bool none = sum == 0.f;   // a wave without states
  const float down = f.low ? Quotient::kDown : 1.f;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int t = 0; t < kBlocks; ++t)
    *reinterpret_cast<float4*>(ys(w, l16, 16 * t + 4 * quarter)) =
        none ? make_float4(0.f, 0.f, 0.f, 0.f)
             : make_float4(o[t][0] * down * f.factor, o[t][1] * down * f.factor,
                           o[t][2] * down * f.factor, o[t][3] * down * f.factor);
  if (quarter == 0) ls[w][l16] = bad ? NAN : none ? -INFINITY : f.log;
  __syncthreads();
  for (int u = threadIdx.x; u < s.R * DH; u += 64 * W) {
    const int r = u / DH, d = u % DH;
    float most = -INFINITY, total = 0.f, acc = 0.f;
#pragma unroll
    for (int x = 0; x < W; ++x) most = fmaxf(most, ls[x][r]);
#pragma unroll
    for (int x = 0; x < W; ++x) {
      const float l = ls[x][r];
      if (l == -INFINITY) continue;   // (a NaN goes on)
      const float g = exp2f(l - most);
      total += g;
      acc = fmaf(g, *ys(x, r, d), acc);
    }
    if (d < s.dh)
      y[at.slice * y_slice + query_row(s, at.b, at.hk, r) + d] = total == 0.f ? 0.f : acc / total;
    if (d == 0)
      lse[at.slice * lse_slice + stat_row(s, at.b, at.hk) + r] =
          total == 0.f ? -INFINITY : (most + log2f(total)) * kLn2;
  }
}

// y and lse of a row from its slices': the slices' outputs weighted by exp(lse_s - lse).  A wave a
// row, lane k holding slice k's weight.
constexpr int kJoinWaves = 4;
__global__ __launch_bounds__(64 * kJoinWaves) void join_kernel(const float* __restrict__ part,
                                                               float* __restrict__ y,
                                                               float* __restrict__ lse, Shape s,
                                                               int slices, int64_t y_size,
                                                               int64_t rows) {
  const float* pl = part + slices * y_size;
  const int lane = threadIdx.x & 63;
  const int64_t stride = (int64_t)gridDim.x * kJoinWaves;
  for (int64_t row = (int64_t)blockIdx.x * kJoinWaves + (threadIdx.x >> 6); row < rows; row += stride) {
    const int64_t h = row % s.H, bi = row / s.H, i = bi % s.Tq, b = bi / s.Tq;   // row (b, i, h)
    const int64_t st = (b * s.H + h) * s.Tq + i;
    const float l = lane < slices ? pl[lane * rows + st] : -INFINITY;
    float top = l;
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float f = l == -INFINITY ? 0.f : expf(l - top);   // a slice with a NaN makes the row one
    float sum = f;
    for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x, 64);
    const float g = sum == 0.f ? 0.f : f / sum;
    for (int d0 = 0; d0 < s.dh; d0 += 64) {
      const int d = d0 + lane;
      float acc = 0.f;
      for (int k0 = 0; k0 < slices; k0 += 4) {   // four loads in flight
        float x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          x[k] = part[min(k0 + k, slices - 1) * y_size + row * s.dh + min(d, s.dh - 1)];
#pragma unroll
        for (int k = 0; k < 4; ++k) acc = fmaf(__shfl(g, k0 + k, 64), x[k], acc);   // (0 past the last)
      }
      if (d < s.dh) y[row * s.dh + d] = acc;
    }
    if (lane == 0) lse[st] = sum == 0.f ? -INFINITY : top + logf(sum);
  }
}

// ---------------------------------------------------------------- backward
// The scale f of a column's values before they are split, which keeps them within 2^15, where a
// tile with the largest value `top` needs a smaller one; the sums follow.  It brings `top` to 2^10 ..
// 2^11: lower leaves the pieces of small values fewer bits, higher rescales more often (2^12: 24 x 512 x
// 512, 121 -> 124 us dk and dv, 89 -> 91 dq; 2^8 is no faster than 2^10).
constexpr int kFresh = 10;
__device__ inline bool passes(float top, float f) { return top * f > 0x1p15f; }
template <int N>
__device__ inline void rescale(float top, float& f, floatx16 (&acc)[N]) {
  const float g = passes(top, f) ? exp2_of(max(kFresh - exponent(top), -126)) : f, up = g / f;
  f = g;
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[t][i] *= up;
}
constexpr float kFirst = 0x1p126f;   // f before the first values
// A column's scale times a matrix's, finite: where the product is not, the values are zero or below
// 2^-111.
__device__ inline float both(float f, float g) { return fminf(f * g, 0x1p126f); }

// Loads the row tiles of the pass over the queries: rows i .. of the group's heads, numbered g Tq +
// position.  A tile stays within a head where a head fills one, else it packs the group's heads.
struct QueryTiles {
  const float *q, *dy, *lse, *delta;   // lse, delta: of the group's first head
  int b, hk, i1, T;
  __device__ bool packed(const Shape& s) const { return s.Tq < T; }
  __device__ int rows_at(const Shape& s, int i) const {
    return packed(s) ? min(T, i1 - i) : min(min(T, i1 - i), s.Tq - i % s.Tq);
  }
  // nl, dl: of row threadIdx.x, -lse in powers of two and delta; a row that is not there gets a
  // probability of 0
  template <bool EXACT, class R>
  __device__ void load(const Shape& s, int i, R& raw, float& nl, float& dl) const {
    const int rows = i < i1 ? rows_at(s, i) : 0;
    if (!packed(s)) {
      const int64_t r = query_row(s, b, hk, min(i, s.R - 1));
      raw.template load<EXACT>(q + r, dy + r, s.ldq, rows, s.dh);
    } else {
      const int64_t to = (int64_t)b * s.Tq * s.ldq + (int64_t)hk * s.G * s.dh;
      raw.template load_packed<EXACT>(q + to, dy + to, s, i, rows);
    }
    if ((int)threadIdx.x < T) {
      const bool there = (int)threadIdx.x < rows;
      nl = there ? -lse[i + threadIdx.x] * kLog2e : -INFINITY;
      dl = there ? delta[i + threadIdx.x] : 0.f;
    }
  }
};

// Up to 64 head columns a wave holds both matrices of its columns and all its sums: four waves a
// workgroup, two workgroups a CU.

// Over the states: dq.  Columns are queries.
template <int DH, bool EXACT>
__global__ __launch_bounds__(64 * Width<DH>::kBackWaves, 2) void dq_kernel(
    const float* __restrict__ q, const float* __restrict__ kv, const int32_t* __restrict__ klen,
    const float* __restrict__ y, const float* __restrict__ lse, const float* __restrict__ dy,
    float* __restrict__ dq, float* __restrict__ delta, Shape s, int tiles, int slice_len,
    int64_t dq_slice) {
  using Wd = Width<DH>;
  constexpr int T = Wd::kBackTile, W = Wd::kBackWaves;
  using Rw = Rows<DH, T>;
  __shared__ __attribute__((aligned(16))) char ks[Rw::kBytes];
  __shared__ __attribute__((aligned(16))) char vs[Rw::kBytes];
  __shared__ floatx2 tops[W];
  const Place at = place(s, tiles);
  if (at.none) return;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  const int col = (at.tile * W + w) * 32 + (lane & 31), here = min(col, s.R - 1);
  const int n = klen[at.b];
  const bool bad = n < 0 || n > s.Tk;
  const int k0 = bad ? 0 : min(n, at.slice * slice_len), k1 = bad ? 0 : min(n, k0 + slice_len);

  const int64_t qrow = query_row(s, at.b, at.hk, here), st = stat_row(s, at.b, at.hk) + here;
  Pieces qp[Wd::kSteps], gp[Wd::kSteps];
  float qc, gf, dl = 0.f;
  {
    float v[DH / 2], u[DH / 2];
    load_column<DH, EXACT>(q + qrow, s.dh, v);
    qc = split_column<DH>(v, qp) * s.scale * kLog2e;
    load_column<DH, EXACT>(dy + qrow, s.dh, v);
    gf = split_column<DH>(v, gp);
    load_column<DH, EXACT>(y + qrow, s.dh, u);
#pragma unroll
    for (int i = 0; i < DH / 2; ++i) dl = fmaf(v[i], u[i], dl);
    dl = sum_of_halves(dl);
  }
  if (col < s.R && half == 0 && at.slice == 0) delta[st] = dl;
  const float nl = -lse[st] * kLog2e;
  floatx16 acc[Wd::kBlocks];
#pragma unroll
  for (int t = 0; t < Wd::kBlocks; ++t) acc[t] = floatx16{};
  float f = kFirst;
  Raw<DH, W, T> raw;
  const auto fetch = [&](int j) {
    const int64_t r = key_row(s, at.b, at.hk, j);
    raw.template load<EXACT>(kv + r, kv + r + (int64_t)s.Hkv * s.dh, s.ldk, k1 - j, s.dh);
  };
  if (k0 < k1) fetch(k0);
  for (int j0 = k0; j0 < k1; j0 += T) {
    raw.publish(tops);
    __syncthreads();
    const int2 e = raw.exponents(tops);
    raw.store(ks, vs, e);
    __syncthreads();
    if (j0 + T < k1) fetch(j0 + T);
    // (no smaller than the normal numbers: a masked score stays -inf)
    const float kf = exp2_of(e.x - 14), c = fmaxf(qc * kf, 0x1p-126f), cv = gf * exp2_of(e.y - 14);
#pragma unroll 1
    for (int r0 = 0; r0 < T && j0 + r0 < k1; r0 += 32) {
      floatx16 a = {}, b = {};
#pragma unroll
      for (int t = 0; t < Wd::kSteps; ++t) a = mma(Rw::by_row(ks, r0, t), qp[t], a);
#pragma unroll
      for (int t = 0; t < Wd::kSteps; ++t) b = mma(Rw::by_row(vs, r0, t), gp[t], b);
      if (j0 + r0 + 32 > k1) mask_rows(a, r0, k1 - j0);
      float x[16], top = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[i] = __builtin_amdgcn_exp2f(fmaf(a[i], c, nl)) * fmaf(b[i], cv, -dl);
        top = fmaxf(top, fabsf(x[i]));
      }
      // dS 2^(e.x - 14) is what meets the pieces of k
      top = max_of_halves(top) * kf;
      if (__any(passes(top, f))) rescale(top, f, acc);
      const Pieces xp[2] = {split8(x, both(f, kf)), split8(x + 8, both(f, kf))};
#pragma unroll
      for (int t = 0; t < Wd::kBlocks; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) acc[t] = mma(Rw::by_column(ks, r0 + 16 * h, t), xp[h], acc[t]);
    }
  }
  if (col >= s.R) return;
  const float out = s.scale / f;
  store_column<Wd::kBlocks, EXACT>(dq + at.slice * dq_slice + qrow, 0, s.dh, [&](int t, int i) {
    return bad ? NAN : acc[t][i] * out;
  });
}

// Over the queries: dk and dv.  Columns are states.
template <int DH, bool EXACT>
__global__ __launch_bounds__(64 * Width<DH>::kBackWaves, 2) void dkv_kernel(
    const float* __restrict__ q, const float* __restrict__ kv, const int32_t* __restrict__ klen,
    const float* __restrict__ lse, const float* __restrict__ dy, const float* __restrict__ delta,
    float* __restrict__ dkv, Shape s, int tiles, int slice_len, int64_t dkv_slice) {
  using Wd = Width<DH>;
  constexpr int T = Wd::kBackTile, W = Wd::kBackWaves;
  using Rw = Rows<DH, T>;
  __shared__ __attribute__((aligned(16))) char qs[Rw::kBytes];
  __shared__ __attribute__((aligned(16))) char gs[Rw::kBytes];
  __shared__ __attribute__((aligned(16))) float nl[T], dl[T];
  __shared__ floatx2 tops[W];
  const Place at = place(s, tiles);
  if (at.none) return;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  const int j = (at.tile * W + w) * 32 + (lane & 31);
  const int n = klen[at.b];
  const bool bad = n < 0 || n > s.Tk;
  // rows of this slice; a workgroup without states has nothing to add
  const bool any = !bad && at.tile * W * 32 < n;
  const int i0 = any ? min(s.R, at.slice * slice_len) : 0, i1 = any ? min(s.R, i0 + slice_len) : 0;

  const int64_t krow = key_row(s, at.b, at.hk, min(j, s.Tk - 1)), to_v = (int64_t)s.Hkv * s.dh;
  Pieces kp[Wd::kSteps], vp[Wd::kSteps];
  float kc, vf;
  {
    float v[DH / 2];
    load_column<DH, EXACT>(kv + krow, s.dh, v);
    kc = split_column<DH>(v, kp) * s.scale * kLog2e;
    load_column<DH, EXACT>(kv + krow + to_v, s.dh, v);
    vf = split_column<DH>(v, vp);
  }
  floatx16 dk[Wd::kBlocks], dv[Wd::kBlocks];
#pragma unroll
  for (int t = 0; t < Wd::kBlocks; ++t) dk[t] = dv[t] = floatx16{};
  float fk = kFirst, fv = kFirst;
  const int64_t st = stat_row(s, at.b, at.hk);
  const QueryTiles rows{q, dy, lse + st, delta + st, at.b, at.hk, i1, T};
  Raw<DH, W, T> raw;
  float ll = 0.f, dd = 0.f;
  if (i0 < i1) rows.load<EXACT>(s, i0, raw, ll, dd);
  for (int i = i0; i < i1;) {
    raw.publish(tops);
    __syncthreads();
    const int2 e = raw.exponents(tops);
    raw.store(qs, gs, e);
    if ((int)threadIdx.x < T) {
      nl[threadIdx.x] = ll;
      dl[threadIdx.x] = dd;
    }
    __syncthreads();
    const int there = rows.rows_at(s, i);
    i += there;
    if (i < i1) rows.load<EXACT>(s, i, raw, ll, dd);
    const float qf = exp2_of(e.x - 14), gf = exp2_of(e.y - 14), c = kc * qf, cv = vf * gf;
#pragma unroll 1
    for (int r0 = 0; r0 < there; r0 += 32) {
      floatx16 a = {}, b = {};
#pragma unroll
      for (int t = 0; t < Wd::kSteps; ++t) a = mma(Rw::by_row(qs, r0, t), kp[t], a);
#pragma unroll
      for (int t = 0; t < Wd::kSteps; ++t) b = mma(Rw::by_row(gs, r0, t), vp[t], b);
      float p[16], x[16], ptop = 0.f, xtop = 0.f;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int row = r0 + 8 * g + 4 * half;
        const float4 l4 = at4(nl, row), d4 = at4(dl, row);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          p[4 * g + k] = __builtin_amdgcn_exp2f(fmaf(a[4 * g + k], c, pick(l4, k)));
          x[4 * g + k] = p[4 * g + k] * fmaf(b[4 * g + k], cv, -pick(d4, k));
          ptop = fmaxf(ptop, p[4 * g + k]);
          xtop = fmaxf(xtop, fabsf(x[4 * g + k]));
        }
      }
      ptop = max_of_halves(ptop) * gf;
      xtop = max_of_halves(xtop) * qf;
      if (__any(passes(ptop, fv) || passes(xtop, fk))) {
        rescale(ptop, fv, dv);
        rescale(xtop, fk, dk);
      }
      {
        const Pieces pp[2] = {split8(p, both(fv, gf)), split8(p + 8, both(fv, gf))};
#pragma unroll
        for (int t = 0; t < Wd::kBlocks; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h) dv[t] = mma(Rw::by_column(gs, r0 + 16 * h, t), pp[h], dv[t]);
      }
      const Pieces xp[2] = {split8(x, both(fk, qf)), split8(x + 8, both(fk, qf))};
#pragma unroll
      for (int t = 0; t < Wd::kBlocks; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) dk[t] = mma(Rw::by_column(qs, r0 + 16 * h, t), xp[h], dk[t]);
    }
  }
  if (j >= s.Tk) return;
  const float ok = s.scale / fk, ov = 1.f / fv;
  const bool live = j < n;
  float* out = dkv + at.slice * dkv_slice + krow;
  store_column<Wd::kBlocks, EXACT>(out, 0, s.dh, [&](int t, int k) {
    return bad ? NAN : live ? dk[t][k] * ok : 0.f;
  });
  store_column<Wd::kBlocks, EXACT>(out + to_v, 0, s.dh, [&](int t, int k) {
    return bad ? NAN : live ? dv[t][k] * ov : 0.f;
  });
}

// Above 64 head columns both matrices and all sums of a column set take more than the 256 registers
// of a lane with which a SIMD holds two waves.  A pair of waves shares 32 columns instead: role 0
// holds a first matrix and forms the scores and probabilities, role 1 a second and forms dP; they
// exchange values through LDS, and each then multiplies on.  The waves of a pair sit on one SIMD:
// while one computes exponentials or splits the next tiles, the other multiplies.  2 x 4096 x 4096,
// 16 heads of 128 on 4, on one card: dk and dv 3.24 -> 1.65 ms, dq 1.56 -> 1.34 (over several cards, as
// their clocks allow: 1.65 .. 1.79 and 1.34 .. 1.45).  At 64 columns, where one wave's
// registers suffice, pairs are slower (24 x 512 x 512: 0.22 against 0.20 ms and 0.19 against 0.15).

// Over the states: dq.  Columns are queries; role 0 holds q, role 1 dy; each multiplies half of the
// rows of dS and k.
template <int DH, bool EXACT>
__global__ __launch_bounds__(64 * Width<DH>::kPairWaves, Width<DH>::kOccupancy) void dq_pair_kernel(
    const float* __restrict__ q, const float* __restrict__ kv, const int32_t* __restrict__ klen,
    const float* __restrict__ y, const float* __restrict__ lse, const float* __restrict__ dy,
    float* __restrict__ dq, float* __restrict__ delta, Shape s, int tiles, int slice_len,
    int64_t dq_slice) {
  using Wd = Width<DH>;
  constexpr int T = 32, W = Wd::kPairWaves, kPairs = W / 2, NB = Wd::kBuffers;
  using Rw = Rows<DH, T>;
  __shared__ __attribute__((aligned(16))) char mats[NB][2][Rw::kBytes];   // tiles of k and v
  __shared__ float4 meet[kPairs][2][2][64];
  __shared__ floatx2 tops[W];
  const Place at = place(s, tiles);
  if (at.none) return;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  const int pair = w % kPairs, role = __builtin_amdgcn_readfirstlane(w / kPairs);
  const int col = (at.tile * kPairs + pair) * 32 + (lane & 31), here = min(col, s.R - 1);
  const int n = klen[at.b];
  const bool bad = n < 0 || n > s.Tk;
  const int k0 = bad ? 0 : min(n, at.slice * slice_len), k1 = bad ? 0 : min(n, k0 + slice_len);

  const int64_t qrow = query_row(s, at.b, at.hk, here), st = stat_row(s, at.b, at.hk) + here;
  Pieces own[Wd::kSteps];   // q, or dy
  float cf, row = 0.f;      // row: -lse in powers of two, or -delta
  {
    float v[DH / 2];
    load_column<DH, EXACT>((role ? dy : q) + qrow, s.dh, v);
    cf = split_column<DH>(v, own);
    if (role) {
      float u[DH / 2];
      load_column<DH, EXACT>(y + qrow, s.dh, u);
#pragma unroll
      for (int i = 0; i < DH / 2; ++i) row = fmaf(v[i], u[i], row);
      row = -sum_of_halves(row);
      if (col < s.R && half == 0 && at.slice == 0) delta[st] = -row;
    } else {
      cf *= s.scale * kLog2e;
      row = -lse[st] * kLog2e;
    }
  }
  floatx16 acc[Wd::kBlocks];
#pragma unroll
  for (int t = 0; t < Wd::kBlocks; ++t) acc[t] = floatx16{};
  float f = kFirst;
  Raw<DH, W, T> raw;
  const auto fetch = [&](int j) {
    const int64_t r = key_row(s, at.b, at.hk, min(j, s.Tk - 1));
    raw.template load<EXACT>(kv + r, kv + r + (int64_t)s.Hkv * s.dh, s.ldk, k1 - j, s.dh);
  };
  const auto stage = [&](int buf) -> int2 {
    const int2 e = raw.exponents(tops);
    raw.store(mats[buf][0], mats[buf][1], e);
    return e;
  };
  if (k0 < k1) {
    fetch(k0);
    raw.publish(tops);
    __syncthreads();
    int2 e = stage(0);
    int buf = 0;
    fetch(k0 + T);
    __syncthreads();
    for (int j0 = k0;; j0 += T) {
      const bool more = j0 + T < k1;
      floatx16 a = {};
      const char* z = mats[buf][role];
#pragma unroll
      for (int t = 0; t < Wd::kSteps; ++t) a = mma(Rw::by_row(z, 0, t), own[t], a);
      float c = cf * exp2_of((role ? e.y : e.x) - 14);
      if (!role) {
        c = fmaxf(c, 0x1p-126f);   // a masked score stays -inf
        if (j0 + T > k1) mask_rows(a, 0, k1 - j0);
#pragma unroll
        for (int i = 0; i < 16; ++i) a[i] = __builtin_amdgcn_exp2f(fmaf(a[i], c, row));
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) a[i] = fmaf(a[i], c, row);
      }
      // the half of the rows that the other wave multiplies
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const int i = 4 * g;
        meet[pair][role][g][lane] = role ? make_float4(a[i], a[i + 1], a[i + 2], a[i + 3])
                                         : make_float4(a[i + 8], a[i + 9], a[i + 10], a[i + 11]);
      }
      raw.publish(tops);
      __syncthreads();
      // dS 2^(e.x - 14) is what meets the pieces of k
      const float kf = exp2_of(e.x - 14);
      float p[8], top = 0.f;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float4 o = meet[pair][1 - role][g][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[4 * g + i] = pick(o, i) * (role ? a[8 + 4 * g + i] : a[4 * g + i]);
          top = fmaxf(top, fabsf(p[4 * g + i]));
        }
      }
      top = max_of_halves(top) * kf;
      if (__any(passes(top, f))) rescale(top, f, acc);
      const Pieces pp = split8(p, both(f, kf));
      const auto advance = [&] {
        e = stage(NB - 1 - buf);
        fetch(j0 + 2 * T);
      };
      if (NB == 2 && role && more) advance();
#pragma unroll
      for (int t = 0; t < Wd::kBlocks; ++t) acc[t] = mma(Rw::by_column(mats[buf][0], 16 * role, t), pp, acc[t]);
      if (!more) break;
      if (NB == 1) __syncthreads();
      if (NB == 1 || !role) advance();
      buf = NB - 1 - buf;
      __syncthreads();
    }
  }
  // the pair's halves together, through the tiles' memory
  float* join = reinterpret_cast<float*>(&mats[0][0][0]) + pair * (Wd::kBlocks * 16 * 64);
  static_assert(kPairs * Wd::kBlocks * 16 * 64 * 4 <= (int)sizeof(mats), "room to join");
  const float out = s.scale / f;
  __syncthreads();
  if (role)
#pragma unroll
    for (int t = 0; t < Wd::kBlocks; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) join[(t * 16 + i) * 64 + lane] = acc[t][i] * out;
  __syncthreads();
  if (role || col >= s.R) return;
  store_column<Wd::kBlocks, EXACT>(dq + at.slice * dq_slice + qrow, 0, s.dh, [&](int t, int i) {
    return bad ? NAN : fmaf(acc[t][i], out, join[(t * 16 + i) * 64 + lane]);
  });
}

// Over the queries: dk and dv.  Columns are states; role 0 holds k and sums dv, role 1 holds v and
// sums dk.
template <int DH, bool EXACT>
__global__ __launch_bounds__(64 * Width<DH>::kPairWaves, Width<DH>::kOccupancy) void dkv_pair_kernel(
    const float* __restrict__ q, const float* __restrict__ kv, const int32_t* __restrict__ klen,
    const float* __restrict__ lse, const float* __restrict__ dy, const float* __restrict__ delta,
    float* __restrict__ dkv, Shape s, int tiles, int slice_len, int64_t dkv_slice) {
  using Wd = Width<DH>;
  constexpr int T = 32, W = Wd::kPairWaves, kPairs = W / 2, NB = Wd::kBuffers;
  using Rw = Rows<DH, T>;
  __shared__ __attribute__((aligned(16))) char mats[NB][2][Rw::kBytes];   // tiles of q and dy
  __shared__ __attribute__((aligned(16))) float nl[NB][T], dl[NB][T];
  __shared__ float4 meet[kPairs][4][64];
  __shared__ floatx2 tops[W];
  const Place at = place(s, tiles);
  if (at.none) return;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  const int pair = w % kPairs, role = __builtin_amdgcn_readfirstlane(w / kPairs);
  const int j = (at.tile * kPairs + pair) * 32 + (lane & 31);
  const int n = klen[at.b];
  const bool bad = n < 0 || n > s.Tk;
  // rows of this slice; a workgroup without states has nothing to add
  const bool any = !bad && at.tile * kPairs * 32 < n;
  const int i0 = any ? min(s.R, at.slice * slice_len) : 0, i1 = any ? min(s.R, i0 + slice_len) : 0;

  const int64_t krow = key_row(s, at.b, at.hk, min(j, s.Tk - 1)), to_v = (int64_t)s.Hkv * s.dh;
  Pieces own[Wd::kSteps];   // k, or v
  float cf;
  {
    float v[DH / 2];
    load_column<DH, EXACT>(kv + krow + (role ? to_v : 0), s.dh, v);
    cf = split_column<DH>(v, own);
    if (!role) cf *= s.scale * kLog2e;
  }
  floatx16 acc[Wd::kBlocks];   // dv, or dk
#pragma unroll
  for (int t = 0; t < Wd::kBlocks; ++t) acc[t] = floatx16{};
  float f = kFirst;
  const int64_t st = stat_row(s, at.b, at.hk);
  const QueryTiles rows{q, dy, lse + st, delta + st, at.b, at.hk, i1, T};
  Raw<DH, W, T> raw;
  float ll = 0.f, dd = 0.f;
  const auto stage = [&](int buf) -> int2 {
    const int2 e = raw.exponents(tops);
    raw.store(mats[buf][0], mats[buf][1], e);
    if ((int)threadIdx.x < T) {
      nl[buf][threadIdx.x] = ll;
      dl[buf][threadIdx.x] = dd;
    }
    return e;
  };
  if (i0 < i1) {
    rows.load<EXACT>(s, i0, raw, ll, dd);
    raw.publish(tops);
    __syncthreads();
    int2 e = stage(0);
    int i = i0 + rows.rows_at(s, i0), buf = 0;
    rows.load<EXACT>(s, i, raw, ll, dd);
    __syncthreads();
    while (true) {
      const bool more = i < i1;
      floatx16 a = {};
      const char* z = mats[buf][role];
#pragma unroll
      for (int t = 0; t < Wd::kSteps; ++t) a = mma(Rw::by_row(z, 0, t), own[t], a);
      const float c = cf * exp2_of((role ? e.y : e.x) - 14);
      float v[16], top = 0.f;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 r4 = at4(role ? dl[buf] : nl[buf], 8 * g + 4 * half);
        if (!role) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            v[4 * g + k] = __builtin_amdgcn_exp2f(fmaf(a[4 * g + k], c, pick(r4, k)));
          meet[pair][g][lane] = make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[4 * g + k] = fmaf(a[4 * g + k], c, -pick(r4, k));
        }
      }
      raw.publish(tops);
      __syncthreads();
      if (role)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 p4 = meet[pair][g][lane];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[4 * g + k] *= pick(p4, k);
        }
#pragma unroll
      for (int k = 0; k < 16; ++k) top = fmaxf(top, fabsf(v[k]));
      // the values meet dy's pieces, or q's: times the scale of those
      const float other = exp2_of((role ? e.x : e.y) - 14);
      top = max_of_halves(top) * other;
      if (__any(passes(top, f))) rescale(top, f, acc);
      const Pieces pp[2] = {split8(v, both(f, other)), split8(v + 8, both(f, other))};
      const auto advance = [&] {
        e = stage(NB - 1 - buf);
        i += rows.rows_at(s, i);
        rows.load<EXACT>(s, i, raw, ll, dd);
      };
      if (NB == 2 && role && more) advance();
#pragma unroll
      for (int t = 0; t < Wd::kBlocks; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) acc[t] = mma(Rw::by_column(mats[buf][1 - role], 16 * h, t), pp[h], acc[t]);
      if (!more) break;
      if (NB == 1) __syncthreads();
      if (NB == 1 || !role) advance();
      buf = NB - 1 - buf;
      __syncthreads();
    }
  }
  if (j >= s.Tk) return;
  const float out = (role ? s.scale : 1.f) / f;   // dk goes where k is, dv where v is
  const bool live = j < n;
  store_column<Wd::kBlocks, EXACT>(
      dkv + at.slice * dkv_slice + krow + (role ? 0 : to_v), 0, s.dh,
      [&](int t, int k) { return bad ? NAN : live ? acc[t][k] * out : 0.f; });
}

// out = the slices' partial sums added in order
__global__ void sum_kernel(const float* __restrict__ part, float* __restrict__ out, int slices,
                           int64_t size) {
  const int64_t stride = (int64_t)gridDim.x * blockDim.x;
  for (int64_t u = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; u < size; u += stride) {
    float acc = 0.f;
    for (int k0 = 0; k0 < slices; k0 += 8) {   // eight loads in flight
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = k0 + k < slices ? part[(k0 + k) * size + u] : 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) acc += x[k];
    }
    out[u] = acc;
  }
}

// ---------------------------------------------------------------- launches
Shape shape_of(const AttendShape& a) {
  Shape s;
  s.B = (int)a.B; s.Tq = (int)a.Tq; s.Tk = (int)a.Tk; s.H = (int)a.H; s.Hkv = (int)a.Hkv;
  s.G = (int)(a.H / a.Hkv);
  s.dh = (int)a.dh;
  s.R = s.G * s.Tq;
  s.ldq = a.H * a.dh;
  s.ldk = 2 * a.Hkv * a.dh;
  s.scale = 1.f / sqrtf((float)a.dh);
  return s;
}

int tile_rows(int64_t dh) { return dh <= 64 ? Width<64>::kTile : 32; }
int back_columns(int64_t dh) {
  return dh <= 64 ? Width<64>::kBackCols : dh <= 128 ? Width<128>::kBackCols : Width<256>::kBackCols;
}
int back_rows(int64_t dh) { return dh <= 64 ? Width<64>::kBackRows : Width<128>::kBackRows; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
dim3 grid_of(const Shape& s, int tiles, int64_t slices) {
  return dim3((unsigned)(ceil_div((int64_t)s.B * s.Hkv, kXcds) * kXcds * tiles), (unsigned)slices);
}
// Whether the forward's workgroups have 256 columns, not 128: where that leaves less than a tenth
// more columns idle, which is what the wide ones gain (4096 x 4096: 0.86 against 0.96 ms at 2 x 16
// heads of 128, 0.89 against 0.98 at 4 x 16 heads of 64; 333 queries, 12 heads of 85: 81 us wide,
// 60 narrow), and there are two of them for each CU (77 states, 2 x 4096 queries, 8 heads of 64:
// 18.1 us wide, 16.8 narrow).
bool wide(const AttendShape& a) {
  const int64_t halves = ceil_div(a.Tq * (a.H / a.Hkv), 128);
  return a.dh <= 128 && (halves % 2 == 0 || halves >= 10) && a.B * a.Hkv * ceil_div(halves, 2) >= 512;
}
int fwd_columns(const AttendShape& a) { return wide(a) ? 256 : a.dh <= 128 ? 128 : 64; }
unsigned flat_grid(int64_t n) { return (unsigned)std::min<int64_t>(ceil_div(n, 256), 4096); }
int64_t slice_of(int64_t n, int64_t slices, int64_t tile) {
  return ceil_div(ceil_div(n, slices), tile) * tile;
}

// Workgroups to aim for, and the fewest tiles a slice is worth cutting off for.
constexpr int64_t kWant = 512, kFewWant = 256, kMinTiles = 2;
int64_t slices_for(int64_t groups, int64_t tiles, int64_t want = kWant, int64_t least = kMinTiles) {
  if (groups >= want) return 1;
  return std::max<int64_t>(1, std::min<int64_t>({ceil_div(want, groups), tiles / least,
                                                  kMaxAttentionSlices}));
}
bool few_rows(const AttendShape& a) { return a.Tq * (a.H / a.Hkv) <= kFewRows && a.dh <= 128; }

#define TO_64(CALL)                        \
  if (s.dh == 32) CALL(32, true);          \
  else if (s.dh < 32) CALL(32, false);     \
  else if (s.dh == 64) CALL(64, true);     \
  else CALL(64, false)
#define FROM_65_TO_128(CALL)               \
  if (s.dh == 96) CALL(96, true);          \
  else if (s.dh < 96) CALL(96, false);     \
  else if (s.dh == 128) CALL(128, true);   \
  else CALL(128, false)
#define TO_128(CALL)                       \
  if (s.dh <= 64) {                        \
    TO_64(CALL);                           \
  } else {                                 \
    FROM_65_TO_128(CALL);                  \
  }
#define ABOVE_128(CALL)                    \
  if (s.dh == 256) CALL(256, true);        \
  else CALL(256, false)
#define ABOVE_64(CALL)                     \
  if (s.dh > 128) {                        \
    ABOVE_128(CALL);                       \
  } else {                                 \
    FROM_65_TO_128(CALL);                  \
  }
#define LAUNCH(KERNEL, WAVES, TILES, SLICES, ...) \
  hipLaunchKernelGGL(KERNEL, grid_of(s, TILES, SLICES), dim3(64 * WAVES), 0, st, __VA_ARGS__)

}  // namespace

int64_t attention_key_slices(const AttendShape& a, bool fwd) {
  if (fwd && few_rows(a))
    return slices_for(a.B * a.Hkv, ceil_div(a.Tk, 32 * kFewWaves), kFewWant, 1);
  const int64_t tiles = ceil_div(a.Tq * (a.H / a.Hkv), fwd ? fwd_columns(a) : back_columns(a.dh));
  return slices_for(a.B * a.Hkv * tiles, ceil_div(a.Tk, fwd ? tile_rows(a.dh) : back_rows(a.dh)));
}
int64_t attention_query_slices(const AttendShape& a) {
  return slices_for(a.B * a.Hkv * ceil_div(a.Tk, back_columns(a.dh)), ceil_div(a.Tq * (a.H / a.Hkv), back_rows(a.dh)));
}

hipError_t cross_attention_fwd(const float* q, const float* kv, const int32_t* klen, float* y,
                               float* lse, float* part, const AttendShape& a, int64_t slices,
                               hipStream_t st) {
  const Shape s = shape_of(a);
  const bool few = few_rows(a);
  const int tiles = few ? 1 : (int)ceil_div(s.R, fwd_columns(a));
  const int len = (int)slice_of(s.Tk, slices, few ? 32 : tile_rows(s.dh));
  const int64_t size = a.B * a.Tq * s.ldq, rows = a.B * a.H * a.Tq;
  float* yo = slices > 1 ? part : y;
  float* lo = slices > 1 ? part + slices * size : lse;
#define ARGS q, kv, klen, yo, lo, s, tiles, len, size, rows
#define FEW(D, X) LAUNCH((few_kernel<D, X>), kFewWaves, tiles, slices, ARGS)
#define WIDE(D, X) LAUNCH((fwd_kernel<D, X, true>), (Forward<D, true>::kWaves), tiles, slices, ARGS)
#define FWD(D, X) LAUNCH((fwd_kernel<D, X, false>), (Forward<D, false>::kWaves), tiles, slices, ARGS)
  if (few) {
    TO_128(FEW);
  } else if (wide(a)) {
    TO_128(WIDE);
  } else if (s.dh <= 128) {
    TO_128(FWD);
  } else {
    ABOVE_128(FWD);
  }
#undef FWD
#undef WIDE
#undef FEW
#undef ARGS
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || slices == 1) return e;
  hipLaunchKernelGGL(join_kernel, dim3((unsigned)std::min<int64_t>(ceil_div(rows, kJoinWaves), 8192)),
                     dim3(64 * kJoinWaves), 0, st, part, y, lse, s, (int)slices, size, rows);
  return hipGetLastError();
}

hipError_t cross_attention_bwd(const float* q, const float* kv, const int32_t* klen,
                               const float* y, const float* lse, const float* dy, float* dq,
                               float* dkv, float* delta, float* part, const AttendShape& a,
                               int64_t q_slices, int64_t kv_slices, hipStream_t st) {
  const Shape s = shape_of(a);
  const int64_t q_size = a.B * a.Tq * s.ldq, kv_size = a.B * a.Tk * s.ldk;
  {
    const int tiles = (int)ceil_div(s.R, back_columns(s.dh));
    const int len = (int)slice_of(s.Tk, q_slices, back_rows(s.dh));
    float* out = q_slices > 1 ? part : dq;
#define ARGS q, kv, klen, y, lse, dy, out, delta, s, tiles, len, q_size
#define DQ(D, X) LAUNCH((dq_kernel<D, X>), Width<D>::kBackWaves, tiles, q_slices, ARGS)
#define DQ_PAIR(D, X) LAUNCH((dq_pair_kernel<D, X>), Width<D>::kPairWaves, tiles, q_slices, ARGS)
    if (s.dh <= 64) {
      TO_64(DQ);
    } else {
      ABOVE_64(DQ_PAIR);
    }
#undef DQ_PAIR
#undef DQ
#undef ARGS
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (q_slices > 1) {
      hipLaunchKernelGGL(sum_kernel, dim3(flat_grid(q_size)), dim3(256), 0, st, part, dq,
                         (int)q_slices, q_size);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  const int tiles = (int)ceil_div(s.Tk, back_columns(s.dh));
  const int len = (int)slice_of(s.R, kv_slices, back_rows(s.dh));
  float* out = kv_slices > 1 ? part : dkv;
#define ARGS q, kv, klen, lse, dy, delta, out, s, tiles, len, kv_size
#define DKV(D, X) LAUNCH((dkv_kernel<D, X>), Width<D>::kBackWaves, tiles, kv_slices, ARGS)
#define DKV_PAIR(D, X) LAUNCH((dkv_pair_kernel<D, X>), Width<D>::kPairWaves, tiles, kv_slices, ARGS)
  if (s.dh <= 64) {
    TO_64(DKV);
  } else {
    ABOVE_64(DKV_PAIR);
  }
#undef DKV_PAIR
#undef DKV
#undef ARGS
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || kv_slices == 1) return e;
  hipLaunchKernelGGL(sum_kernel, dim3(flat_grid(kv_size)), dim3(256), 0, st, part, dkv,
                     (int)kv_slices, kv_size);
  return hipGetLastError();
}

}  // namespace ooc

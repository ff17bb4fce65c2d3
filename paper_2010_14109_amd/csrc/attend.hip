// Cross attention: queries against the first klen states of their sequence (gfx950), and the rules by which
// all attention without a matrix of scores chooses its kernels.  The kernels, and what they are built on,
// are in attend_kernels.h.
#include "attend_kernels.h"

namespace ooc {

// Whether a key head's query rows are few enough for the kernel of few.
constexpr int64_t kFewRows = 16;
static_assert(kFewRows == kFewColumns, "the columns that kernel has");
bool attention_few(const AttendShape& a) { return a.Tq * (a.H / a.Hkv) <= kFewRows && a.dh <= 128; }

// Whether the forward's workgroups have 256 columns, not 128: where that leaves less than a tenth
// more columns idle, which is what the wide ones gain (4096 x 4096: 0.86 against 0.96 ms at 2 x 16
// heads of 128, 0.89 against 0.98 at 4 x 16 heads of 64; 333 queries, 12 heads of 85: 81 us wide,
// 60 narrow), and there are two of them for each CU (77 states, 2 x 4096 queries, 8 heads of 64:
// 18.1 us wide, 16.8 narrow).  Under spans, two sets of columns a wave spill up to 64 head columns (24 x 512
// in documents, 16 heads of 64, with gradients: 378 us wide, 306 narrow); above, neither is slower.
bool attention_wide(const AttendShape& a, bool spans) {
  if (spans && a.dh <= 64) return false;
  const int64_t halves = ceil_div(a.Tq * (a.H / a.Hkv), 128);
  return a.dh <= 128 && (halves % 2 == 0 || halves >= 10) && a.B * a.Hkv * ceil_div(halves, 2) >= 512;
}

int64_t attention_key_slices(const AttendShape& a, bool fwd, bool spans) {
  if (fwd && attention_few(a))
    return slices_for(a.B * a.Hkv, ceil_div(a.Tk, 32 * kFewWaves), kFewWant, 1);
  const int64_t tiles = ceil_div(a.Tq * (a.H / a.Hkv), fwd ? fwd_columns(a, spans) : back_columns(a.dh));
  return slices_for(a.B * a.Hkv * tiles, ceil_div(a.Tk, fwd ? tile_rows(a.dh) : back_rows(a.dh)),
                    spans && fwd && a.dh <= 64 ? kSpanWant : kWant);
}
int64_t attention_query_slices(const AttendShape& a) {
  return slices_for(a.B * a.Hkv * ceil_div(a.Tk, back_columns(a.dh)),
                    ceil_div(a.Tq * (a.H / a.Hkv), back_rows(a.dh)));
}

hipError_t cross_attention_fwd(const float* q, const float* kv, const int32_t* klen, float* y,
                               float* lse, float* part, const AttendShape& a, int64_t slices,
                               hipStream_t s) {
  return attend_fwd(q, kv, FirstStates{klen}, y, lse, part, a, slices, s);
}

hipError_t cross_attention_bwd(const float* q, const float* kv, const int32_t* klen,
                               const float* y, const float* lse, const float* dy, float* dq,
                               float* dkv, float* delta, float* part, const AttendShape& a,
                               int64_t q_slices, int64_t kv_slices, hipStream_t s) {
  return attend_bwd(q, kv, FirstStates{klen}, y, lse, dy, dq, dkv, delta, part, a, q_slices, kv_slices, s);
}

}  // namespace ooc

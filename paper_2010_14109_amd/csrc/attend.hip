// Cross attention: queries against the first klen states of their sequence (gfx950).  The kernels, and
// what they are built on, are in attend_kernels.h.
#include "attend_kernels.h"

namespace ooc {

int64_t attention_key_slices(const AttendShape& a, bool fwd, bool spans) {
  if (fwd && few_rows(a))
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

// Span attention: each query against a span of the states of its sequence (gfx950): causal, a sliding
// window, documents packed into a sequence, a prefix, a token behind a cache are all such spans.  The
// kernels are those of cross attention (attend_kernels.h) with another view of what is seen.
//
// Tiles of states that no query of a workgroup sees are not loaded, and only blocks of 32 x 32 that a span
// cuts compare states with spans.  Blocks that a wave does not see at all are not multiplied in the
// forward, nor in the backward up to 64 head columns; above, pairs of waves multiply every block of a tile.
// The pass for dk and dv finds the queries that see its states by the bounds of every 32 queries, which
// the pass for dq leaves.  It is bound by vector instructions (exponentials, splitting, cap and bias) where spans
// are long: 2 x 4096 in a window of 1024, 16 heads of 128 on 4, capped, 243 us forward, 393 dq, 548 dk and
// dv, 0.55 of what three fp16 products a product allow; by loads and stores where they are short: 24 x 512 in
// documents, 16 heads of 64, 56, 81 and 99.  Above 128 head columns a SIMD holds one wave and registers spill,
// the more at widths that are no 256: 4 x 2048 causal, 8 heads on 2, of 256 and capped, 598, 1024 and 1598 (190,
// 190 and 285 at the rate of the products needed), of 200 and biased, 851, 1095 and 2651 (149, 149 and 223).
#include "attend_kernels.h"

namespace ooc {

hipError_t span_attention_fwd(const float* q, const float* kv, const int32_t* span, const float* mod,
                              bool cap, bool bias, float* y, float* lse, float* part,
                              const AttendShape& a, int64_t slices, hipStream_t s) {
  const AllSpans v{span, mod, nullptr, bias};
  return cap ? attend_fwd(q, kv, Spans<true>{v}, y, lse, part, a, slices, s)
             : attend_fwd(q, kv, Spans<false>{v}, y, lse, part, a, slices, s);
}

hipError_t span_attention_bwd(const float* q, const float* kv, const int32_t* span, const float* mod,
                              bool cap, bool bias, const float* y, const float* lse, const float* dy,
                              float* dq, float* dkv, float* delta, int32_t* bounds, float* part,
                              const AttendShape& a, int64_t q_slices, int64_t kv_slices,
                              hipStream_t s) {
  const AllSpans v{span, mod, bounds, bias};
  return cap ? attend_bwd(q, kv, Spans<true>{v}, y, lse, dy, dq, dkv, delta, part, a, q_slices, kv_slices, s)
             : attend_bwd(q, kv, Spans<false>{v}, y, lse, dy, dq, dkv, delta, part, a, q_slices, kv_slices, s);
}

}  // namespace ooc

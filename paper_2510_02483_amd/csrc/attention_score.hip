// Launches of the attention kernels of attn_tile.h on packed sequences with capped scores and
// windows.
#include "attn_tile.h"

namespace ls {

namespace {

// f(a ModScore) for the cap (0: none) and the window (of at most `total` positions).
template <class F>
hipError_t with_score(const ScoreShape& c, F&& f) {
  if (c.cap > 0.f) return f(ModScore<true>{c.window, 2.0f * LOG2E * c.scale / c.cap, c.cap * LOG2E, c.rest});
  return f(ModScore<false>{c.window, 0.f, 0.f, c.rest});
}

}  // namespace

hipError_t packed_score_attn_fwd(const PackedShape& p, const ScoreShape& c, const void* plan, const bf16_t* qkv,
                                 bf16_t* o, float* lse, hipStream_t s) {
  const AttnShape sh = packed_shape(p);
  const PackedView v = packed_view(p, plan);
  return with_score(c, [&](auto sc) {
    using SC = decltype(sc);
    return p.d == 64 ? attn_fwd_t<64, true, SC>(sh, v, qkv, o, lse, s, sc, c.scale)
                     : attn_fwd_t<128, true, SC>(sh, v, qkv, o, lse, s, sc, c.scale);
  });
}

hipError_t packed_score_attn_bwd(const PackedShape& p, const ScoreShape& c, const void* plan, const bf16_t* qkv,
                                 const bf16_t* o, const float* lse, const bf16_t* dout, bf16_t* dqkv, void* ws,
                                 hipStream_t s) {
  const AttnShape sh = packed_shape(p);
  const PackedView v = packed_view(p, plan);
  return with_score(c, [&](auto sc) {
    using SC = decltype(sc);
    return p.d == 64 ? packed_attn_bwd_t<64, SC>(sh, v, qkv, o, lse, dout, dqkv, ws, s, sc, c.scale)
                     : packed_attn_bwd_t<128, SC>(sh, v, qkv, o, lse, dout, dqkv, ws, s, sc, c.scale);
  });
}

}  // namespace ls

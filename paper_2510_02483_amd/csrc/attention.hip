// Launches of the attention kernels of attn_tile.h on batches of equal lengths and on packed sequences.
#include "attn_tile.h"

namespace ls {

namespace {

// Split of each kv head's query-head group over workgroups of the dK/dV
// kernel: the smallest divisor of the group size that gives at least two
// workgroups per compute unit (256 CUs), or the whole group.
int dkdv_split(const AttnShape& sh) {
  const int G = sh.nq / sh.nkv;
  const int64_t g1 = (int64_t)((sh.seq + BWD_BKV - 1) / BWD_BKV) * sh.nkv * sh.batch;
  for (int h = 1; h < G; ++h)
    if (G % h == 0 && g1 * h >= 512) return h;
  return G;
}

template <int D>
hipError_t attn_bwd_t(const AttnShape& sh, const bf16_t* qkv, const bf16_t* o, const float* lse, const bf16_t* dout,
                      bf16_t* dqkv, const float* rope_cs, void* ws, hipStream_t s) {
  const int64_t T = (int64_t)sh.batch * sh.seq;
  float* Dv = (float*)ws;
  float* lse2 = Dv + T * sh.nq;
  hipLaunchKernelGGL((attn_bwd_pre_kernel<D, false>), dim3((unsigned)((T + 3) / 4)), dim3(256), 0, s, sh, o, dout, lse, Dv,
                     lse2, (const bf16_t*)nullptr, false, 0.f);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const float scale = 1.0f / sqrtf((float)(sh.d_scale > 0 ? sh.d_scale : D));
  const int hsplit = dkdv_split(sh);
  float* part = hsplit > 1 ? (float*)((char*)ws + bwd_ws_head(sh)) : nullptr;
  const unsigned gkv = (unsigned)((sh.seq + BWD_BKV - 1) / BWD_BKV) * sh.nkv * sh.batch * hsplit;
  const PackedView none;
  if (part)
    hipLaunchKernelGGL((attn_bwd_dkdv_kernel<D, true, false, PlainScore>), dim3(gkv), dim3(256), 0, s, sh, none, qkv, dout,
                       (const float*)lse2, (const float*)Dv, dqkv, rope_cs, scale, scale * LOG2E, hsplit, part, PlainScore{});
  else
    hipLaunchKernelGGL((attn_bwd_dkdv_kernel<D, false, false, PlainScore>), dim3(gkv), dim3(256), 0, s, sh, none, qkv, dout,
                       (const float*)lse2, (const float*)Dv, dqkv, rope_cs, scale, scale * LOG2E, 1, nullptr, PlainScore{});
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (part) {
    const int64_t rows = T * sh.nkv;  // one wave each, four per workgroup
    hipLaunchKernelGGL((attn_bwd_dkdv_reduce<D>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, sh, hsplit,
                       (const float*)part, dqkv, rope_cs, scale);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const unsigned gq = (unsigned)((sh.seq + BQ - 1) / BQ) * sh.nq * sh.batch;
  hipLaunchKernelGGL((attn_bwd_dq_kernel<D, false, PlainScore>), dim3(gq), dim3(256), 0, s, sh, none, qkv, dout,
                     (const float*)lse2, (const float*)Dv, dqkv, rope_cs, scale, scale * LOG2E, (const float*)nullptr,
                     PlainScore{});
  return hipGetLastError();
}

}  // namespace

hipError_t attn_fwd(const AttnShape& sh, const bf16_t* qkv, bf16_t* o, float* lse, hipStream_t s) {
  if (sh.d == 128) return attn_fwd_t<128, false>(sh, {}, qkv, o, lse, s);
  if (sh.d == 64) return attn_fwd_t<64, false>(sh, {}, qkv, o, lse, s);
  return hipErrorInvalidValue;
}

size_t attn_bwd_workspace(const AttnShape& sh) {
  // D and the base-2 log-sum-exp of every query, then (when the dK/dV group
  // is split) the fp32 partial dK | dV rows of every split
  const int hsplit = dkdv_split(sh);
  const int64_t part = hsplit > 1 ? (int64_t)hsplit * sh.batch * sh.seq * sh.nkv * 2 * sh.d * (int64_t)sizeof(float) : 0;
  return (size_t)(bwd_ws_head(sh) + part);
}

hipError_t attn_bwd(const AttnShape& sh, const bf16_t* qkv, const bf16_t* o, const float* lse, const bf16_t* dout,
                    bf16_t* dqkv, const float* rope_cs, void* ws, hipStream_t s) {
  if (sh.d == 128) return attn_bwd_t<128>(sh, qkv, o, lse, dout, dqkv, rope_cs, ws, s);
  if (sh.d == 64) return attn_bwd_t<64>(sh, qkv, o, lse, dout, dqkv, rope_cs, ws, s);
  return hipErrorInvalidValue;
}

hipError_t packed_attn_fwd(const PackedShape& p, const void* plan, const bf16_t* qkv, bf16_t* o, float* lse,
                           hipStream_t s) {
  const AttnShape sh = packed_shape(p);
  if (p.d == 64) return attn_fwd_t<64, true>(sh, packed_view(p, plan), qkv, o, lse, s);
  return attn_fwd_t<128, true>(sh, packed_view(p, plan), qkv, o, lse, s);
}

size_t packed_attn_bwd_workspace(const PackedShape& p) {
  // D and the base-2 log-sum-exp of every row and head, then the slots of partial dK | dV
  return (size_t)(bwd_ws_head(packed_shape(p)) + packed_layout(p).max_slots * p.nkv * PACKED_ROWS * 2 *
                                                   (p.d == 64 ? 64 : 128) * 4);
}

hipError_t packed_attn_bwd(const PackedShape& p, const void* plan, const bf16_t* qkv, const bf16_t* o, const float* lse,
                           const bf16_t* dout, bf16_t* dqkv, void* ws, hipStream_t s) {
  const AttnShape sh = packed_shape(p);
  if (p.d == 64) return packed_attn_bwd_t<64>(sh, packed_view(p, plan), qkv, o, lse, dout, dqkv, ws, s);
  return packed_attn_bwd_t<128>(sh, packed_view(p, plan), qkv, o, lse, dout, dqkv, ws, s);
}

}  // namespace ls

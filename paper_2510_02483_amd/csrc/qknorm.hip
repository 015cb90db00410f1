// Queries and keys normed per head and turned by their position, in one pass over a
// packed projection buffer, and its backward pass.
//
// For a head x of d features with gain g, at position p of its sequence:
//   r = (mean x^2 + eps)^-1/2,  n = r g x,  y = R_p n
// (R_p turns the pairs (i, i + d/2) by p theta^(-2i/d)).  Backward, for dy:
//   dn = R_p^T dy,  a = g dn,  dx = r (a - x r <a, x r> / d),  dg = sum over rows and heads of r dn x.
// r is formed again from x, which the backward pass reads anyhow: nothing is saved.
//
// A wave takes a row; G lanes (4, 8 or 16) take a head, lane c of them V pairs: features
// V c .. and d/2 + V c .., so that loads and stores are V bf16 wide, sums over a head
// stay in G neighbouring lanes (lane swaps of the vector unit) and 64 / G heads are
// worked on at once.  V = 8 where a head's half is a multiple of 8, else 4; lanes past a
// head's features, and past the last head, work on zeros.
//
// Bound by HBM bandwidth: every row is read and written once, all sums in fp32, one
// rounding to bf16.  8135 rows of 24/8 heads of 128: forward 29 us (5.7 TB/s), backward 43 + 5 us for the gains' sums
// (5.8 TB/s); 4099 rows of 64/64 heads of 104: 70 us (4.7 TB/s) and 97 + 6 us (5.1 TB/s).
#include <math.h>

#include <algorithm>

#include "packed.h"

namespace ls {

namespace {

constexpr int QKN_WAVES = 4;
constexpr int SUM_GROUPS = 16;   // threads that share a column of those

template <int CTRL>
LS_DEV float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// Sum over the G lanes of a head (all lanes active): within quads, across the halves of
// eight lanes, of sixteen (mirrored: after the steps before, the lanes there agree).
template <int G>
LS_DEV float head_sum(float v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  if constexpr (G >= 8) v += dpp<0x141>(v);
  if constexpr (G >= 16) v += dpp<0x140>(v);
  return v;
}

template <int G>
LS_DEV float head_max(float v) {  // (of values from 0 on)
  v = fmaxf(v, dpp<0xB1>(v));
  v = fmaxf(v, dpp<0x4E>(v));
  if constexpr (G >= 8) v = fmaxf(v, dpp<0x141>(v));
  if constexpr (G >= 16) v = fmaxf(v, dpp<0x140>(v));
  return v;
}

// V features of either half of a head, and the cos and sin of their angles.
template <int V>
struct Pairs {
  float a[V], b[V];
};
// The same as loaded: what is in flight takes half the registers.
template <int V>
struct RawPairs {
  typedef uint32_t words __attribute__((ext_vector_type(V / 2)));
  words u, w;
  LS_DEV void load(const bf16_t* p, int half, bool ok) {
    u = w = words{};
    if (ok) {
      u = *(const words*)p;
      w = *(const words*)(p + half);
    }
  }
  LS_DEV Pairs<V> pairs() const {
    Pairs<V> x;
#pragma unroll
    for (int e = 0; e < V / 2; ++e) {
      x.a[2 * e] = bf_lo(u[e]);
      x.a[2 * e + 1] = bf_hi(u[e]);
      x.b[2 * e] = bf_lo(w[e]);
      x.b[2 * e + 1] = bf_hi(w[e]);
    }
    return x;
  }
};
template <int V>
LS_DEV Pairs<V> load_pairs(const bf16_t* p, int half, bool ok) {
  RawPairs<V> r;
  r.load(p, half, ok);
  return r.pairs();
}
// Groups of 64 / G heads whose loads a wave issues together (src and dst may be one, so that the compiler keeps loads
// behind earlier stores), as the registers of four waves to a SIMD allow.
template <int V>
constexpr int batch_of() { return V == 4 ? 2 : 1; }
template <int V>
LS_DEV void store_pairs(bf16_t* p, int half, const Pairs<V>& x) {
  typedef uint32_t words __attribute__((ext_vector_type(V / 2)));
  words u, w;
#pragma unroll
  for (int e = 0; e < V / 2; ++e) {
    u[e] = pack_bf2(x.a[2 * e], x.a[2 * e + 1]);
    w[e] = pack_bf2(x.b[2 * e], x.b[2 * e + 1]);
  }
  *(words*)p = u;
  *(words*)(p + half) = w;
}
// A head's sum of squares.
template <int V, int G>
LS_DEV float squares(const Pairs<V>& x) {
  float ss = 0.f;
#pragma unroll
  for (int e = 0; e < V; ++e) ss += x.a[e] * x.a[e] + x.b[e] * x.b[e];
  return head_sum<G>(ss);
}
// r = (mean x^2 + eps)^-1/2 of a head.  bf16 reaches as far as fp32: squares of values beyond 2^64 leave its
// range, and those below 2^-63 lose bits, which counts where mean and eps are small.  Where a head of the wave is so
// (`ok`: the lane has one), its x is divided by 2^k, the size of the larger of max |x| and sqrt(eps), r is that of
// the divided head, and `far` is set; any other head has k = 0, so that nothing changes for it.  (r x is the same;
// what else r multiplies is to be divided by 2^k.)  Ordinary data pays a comparison and a ballot: 8135 rows of
// 24/8 heads of 128, both passes, 77.6 -> 77.9 us.
template <int V, int G>
LS_DEV float inverse_size(Pairs<V>& x, int d, float eps, bool ok, bool& far, int& k) {
  float ms = squares<V, G>(x) / (float)d + eps;
  far = __ballot(ok && !(ms >= 0x1p-96f && ms < INFINITY));
  k = 0;
  if (far) {
    float big = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) big = fmaxf(big, fmaxf(fabsf(x.a[e]), fabsf(x.b[e])));
    big = fmaxf(head_max<G>(big), sqrtf(eps));
    if (!(ms >= 0x1p-96f && ms < INFINITY) && big > 0.f && big < INFINITY) k = ilogbf(big);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      x.a[e] = ldexpf(x.a[e], -k);
      x.b[e] = ldexpf(x.b[e], -k);
    }
    ms = squares<V, G>(x) / (float)d + ldexpf(eps, -2 * k);
  }
  return 1.0f / sqrtf(ms);
}
// The row's angles, one per lane in fp64 as turns without their whole part (in fp32 the
// fraction of a far position's angle would be lost), then handed to the lanes of the pairs.
template <int V>
LS_DEV Pairs<V> row_turns(double turns, int pos, int c) {
  const double t = pos * turns;
  float sn, cs;
  sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
  Pairs<V> out;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    out.a[e] = __shfl(cs, V * c + e);
    out.b[e] = __shfl(sn, V * c + e);
  }
  return out;
}
LS_DEV double turns_of(int pair, int half, double log2_theta) {
  return exp2(-(double)(pair % half) / half * log2_theta) * 0.15915494309189533577;
}
// v of one row goes along where the result lies elsewhere.
LS_DEV void copy_v(const bf16_t* src, bf16_t* dst, int n, int lane, int seg, int segs) {
  constexpr int U = 4;
  for (int i = 64 * U * seg + lane; i < n / 8; i += 64 * U * segs) {
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + 64 * u < n / 8) x[u] = ((const u32x4*)src)[i + 64 * u];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + 64 * u < n / 8) ((u32x4*)dst)[i + 64 * u] = x[u];
  }
}

template <int V, int G>
__global__ __launch_bounds__(64 * QKN_WAVES, 4) void qk_norm_rope_kernel(
    int total, int seg_bits, int nq, int nkv, int d, float eps, double log2_theta, const int32_t* __restrict__ pos,
    const bf16_t* __restrict__ gq, const bf16_t* __restrict__ gk, const bf16_t* src, bf16_t* dst) {
  constexpr int HPW = 64 / G, U = batch_of<V>();
  const int lane = threadIdx.x & 63, half = d / 2, c = lane % G, h0 = lane / G;
  const bool in = V * c < half;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * d;
  const double turns = turns_of(lane, half, log2_theta);
  const Pairs<V> gains[2] = {load_pairs<V>(gq + V * c, half, in), load_pairs<V>(gk + V * c, half, in)};
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  for (int64_t unit = (int64_t)blockIdx.x * QKN_WAVES + wave; unit < (int64_t)total << seg_bits;
       unit += (int64_t)gridDim.x * QKN_WAVES) {
    const int64_t row = unit >> seg_bits;
    const int segs = 1 << seg_bits, seg = (int)unit & (segs - 1);
    const int p = pos[row];
    if (p < 0 || p > row) continue;
    const Pairs<V> cs = row_turns<V>(turns, p, c);
    auto heads = [&](int first, int n, const Pairs<V>& g) {
      for (int hu = seg * U * HPW; hu < n; hu += segs * U * HPW) {
        const int64_t at0 = row * ld + (int64_t)(first + hu + h0) * d + V * c;
        RawPairs<V> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u].load(src + at0 + u * HPW * d, half, in && hu + u * HPW + h0 < n);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (hu + u * HPW >= n) break;
          const bool ok = in && hu + u * HPW + h0 < n;
          const int64_t at = at0 + u * HPW * d;
          Pairs<V> x = raw[u].pairs();
          bool far;
          int k;
          const float r = inverse_size<V, G>(x, d, eps, ok, far, k);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float a = x.a[e] * r * g.a[e], b = x.b[e] * r * g.b[e];
            x.a[e] = a * cs.a[e] - b * cs.b[e];
            x.b[e] = a * cs.b[e] + b * cs.a[e];
          }
          if (ok) store_pairs<V>(dst + at, half, x);
        }
      }
    };
    heads(0, nq, gains[0]);
    heads(nq, nkv, gains[1]);
    const int64_t v = row * ld + (int64_t)(nq + nkv) * d;
    if (src != dst) copy_v(src + v, dst + v, nkv * d, lane, seg, segs);
  }
}

// A workgroup's sums for the gains' gradients, of the rows that its waves take, go to
// part[blockIdx.x][2d] (q's, then k's), which gain_sum_kernel adds.  Sums over a lane's rows
// and heads, then over the lanes of the same features, then over the waves: a fixed
// order.
template <int V, int G>
__global__ __launch_bounds__(64 * QKN_WAVES, V == 4 ? 4 : 3) void qk_norm_rope_bwd_kernel(
    int total, int seg_bits, int nq, int nkv, int d, float eps, double log2_theta, const int32_t* __restrict__ pos,
    const bf16_t* __restrict__ gq, const bf16_t* __restrict__ gk, const bf16_t* __restrict__ src, const bf16_t* dy,
    bf16_t* dx, float* __restrict__ part) {
  constexpr int HPW = 64 / G, U = batch_of<V>();
  __shared__ float red[QKN_WAVES][2][2 * V * G];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int half = d / 2, c = lane % G, h0 = lane / G;
  const bool in = V * c < half;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * d;
  const double turns = turns_of(lane, half, log2_theta);
  const Pairs<V> gains[2] = {load_pairs<V>(gq + V * c, half, in), load_pairs<V>(gk + V * c, half, in)};
  Pairs<V> sums[2] = {};
  for (int64_t unit = (int64_t)blockIdx.x * QKN_WAVES + wave; unit < (int64_t)total << seg_bits;
       unit += (int64_t)gridDim.x * QKN_WAVES) {
    const int64_t row = unit >> seg_bits;
    const int segs = 1 << seg_bits, seg = (int)unit & (segs - 1);
    const int p = pos[row];
    if (p < 0 || p > row) continue;
    const Pairs<V> cs = row_turns<V>(turns, p, c);
    auto heads = [&](int first, int n, const Pairs<V>& g, Pairs<V>& sum) {
      for (int hu = seg * U * HPW; hu < n; hu += segs * U * HPW) {
        const int64_t at0 = row * ld + (int64_t)(first + hu + h0) * d + V * c;
        RawPairs<V> xr[U], tr[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const bool ok = in && hu + u * HPW + h0 < n;
          xr[u].load(src + at0 + u * HPW * d, half, ok);
          tr[u].load(dy + at0 + u * HPW * d, half, ok);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (hu + u * HPW >= n) break;
          const bool ok = in && hu + u * HPW + h0 < n;
          const int64_t at = at0 + u * HPW * d;
          Pairs<V> x = xr[u].pairs();
          const Pairs<V> t = tr[u].pairs();
          bool far;
          int k;
          const float size = inverse_size<V, G>(x, d, eps, ok, far, k);
          const float r = ok ? size : 0.f;  // (a lane without a head adds nothing to the gains' sums, eps 0 too)
          Pairs<V> dn;
          float dot = 0.f;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            dn.a[e] = t.a[e] * cs.a[e] + t.b[e] * cs.b[e];
            dn.b[e] = t.b[e] * cs.a[e] - t.a[e] * cs.b[e];
            dot += g.a[e] * dn.a[e] * x.a[e] + g.b[e] * dn.b[e] * x.b[e];
          }
          // <a, x r> / d: with r inside, no power of it can leave the range
          const float coef = r * head_sum<G>(dot) / (float)d;
          Pairs<V> out;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float na = x.a[e] * r, nb = x.b[e] * r;
            sum.a[e] += dn.a[e] * na;
            sum.b[e] += dn.b[e] * nb;
            out.a[e] = r * (g.a[e] * dn.a[e] - na * coef);
            out.b[e] = r * (g.b[e] * dn.b[e] - nb * coef);
          }
          if (far) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              out.a[e] = ldexpf(out.a[e], -k);
              out.b[e] = ldexpf(out.b[e], -k);
            }
          }
          if (ok) store_pairs<V>(dx + at, half, out);
        }
      }
    };
    heads(0, nq, gains[0], sums[0]);
    heads(nq, nkv, gains[1], sums[1]);
    const int64_t v = row * ld + (int64_t)(nq + nkv) * d;
    if (dy != dx) copy_v(dy + v, dx + v, nkv * d, lane, seg, segs);
  }
  if (!part) return;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) {
      float v = e < V ? sums[k].a[e % V] : sums[k].b[e % V];
#pragma unroll
      for (int o = G; o < 64; o <<= 1) v += __shfl_xor(v, o);
      if (h0 == 0) red[wave][k][2 * V * c + e] = v;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * d; i += 64 * QKN_WAVES) {
    // feature f of a gain: lane (f mod d/2) / V of a head, value f mod V of its half
    const int k = i / d, f = i % d, u = f % half, e = 2 * V * (u / V) + u % V + (f < half ? 0 : V);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < QKN_WAVES; ++w) v += red[w][k][e];
    part[(int64_t)blockIdx.x * 2 * d + i] = v;
  }
}

// dg (+)= the sum of the parts, 64 columns to a workgroup, 16 threads to a column; in
// fp64 and a fixed order.
__global__ __launch_bounds__(64 * SUM_GROUPS) void gain_sum_kernel(int parts, int d, const float* __restrict__ part,
                                                                   float* __restrict__ dgq, float* __restrict__ dgk,
                                                                   int accumulate) {
  __shared__ double red[SUM_GROUPS][64];
  const int c = threadIdx.x & 63, g = threadIdx.x >> 6, i = blockIdx.x * 64 + c;
  double v = 0.0;
  if (i < 2 * d) {
#pragma unroll 8
    for (int p = g; p < parts; p += SUM_GROUPS) v += part[(int64_t)p * 2 * d + i];
  }
  red[g][c] = v;
  __syncthreads();
  if (g > 0 || i >= 2 * d) return;
  for (int k = 1; k < SUM_GROUPS; ++k) v += red[k][c];
  float* out = i < d ? dgq : dgk;
  if (!out) return;
  out += i % d;
  *out = (float)(accumulate ? v + *out : v);
}

// f(V, G) for a head size.
template <class F>
void by_head(int d, F&& f) {
  using std::integral_constant;
  if (d == 64) f(integral_constant<int, 8>{}, integral_constant<int, 4>{});
  else if (d % 16 == 0) f(integral_constant<int, 8>{}, integral_constant<int, 8>{});
  else f(integral_constant<int, 4>{}, integral_constant<int, 16>{});
}

// Waves that share a row: of a few thousand rows one wave each would leave the card's last round of workgroups nearly
// empty (4099 rows of 64/64 heads of 104, 1025 workgroups: backward 125 us, 98 with eight waves to a row), so a row is
// cut in equal parts while there are fewer than 32768 pieces; not unequally (24/8 heads of 128 in two: 50 -> 59 us).
int segment_bits(const PackedShape& p) {
  const int batch = p.d == 64 ? 16 : 8;  // heads
  int bits = 0;
  while (((int64_t)p.total << bits) < 32768 && p.nq % (batch << (bits + 1)) == 0) ++bits;
  return bits;
}
// Workgroups of the backward pass, and rows of partial gain gradients: its pieces in whole rounds of as many workgroups
// as run at once (four waves to a SIMD, three of the instances with V = 8): 8135 rows of 24/8 heads of 128 in
// 678 workgroups 43 us, in 1017, of which 768 run at once, 53.
int qkn_parts(const PackedShape& p) {
  const int64_t need = (((int64_t)p.total << segment_bits(p)) + QKN_WAVES - 1) / QKN_WAVES;
  const int64_t most = PACKED_CUS * (p.d % 16 == 0 ? 3 : 4), rounds = (need + most - 1) / most;
  return (int)((need + rounds - 1) / rounds);
}

}  // namespace

hipError_t packed_qk_norm_rope(const PackedShape& p, const void* plan, double theta, float eps, const bf16_t* gq,
                               const bf16_t* gk, const bf16_t* src, bf16_t* dst, hipStream_t s) {
  const int bits = segment_bits(p);
  const int64_t need = (((int64_t)p.total << bits) + QKN_WAVES - 1) / QKN_WAVES;
  const dim3 grid((unsigned)std::min<int64_t>(need, 8192)), block(64 * QKN_WAVES);
  by_head(p.d, [&](auto v, auto g) {
    hipLaunchKernelGGL((qk_norm_rope_kernel<decltype(v)::value, decltype(g)::value>), grid, block, 0, s, (int)p.total, bits,
                       p.nq, p.nkv, p.d, eps, log2(theta), packed_pos(p, plan), gq, gk, src, dst);
  });
  return hipGetLastError();
}

size_t packed_qk_norm_rope_bwd_workspace(const PackedShape& p) { return (size_t)qkn_parts(p) * 2 * p.d * 4; }

hipError_t packed_qk_norm_rope_bwd(const PackedShape& p, const void* plan, double theta, float eps, const bf16_t* gq,
                                   const bf16_t* gk, const bf16_t* src, const bf16_t* dy, bf16_t* dx, float* dgq,
                                   float* dgk, int accumulate, void* ws, hipStream_t s) {
  const int parts = qkn_parts(p);
  float* part = dgq || dgk ? (float*)ws : nullptr;
  by_head(p.d, [&](auto v, auto g) {
    hipLaunchKernelGGL((qk_norm_rope_bwd_kernel<decltype(v)::value, decltype(g)::value>), dim3((unsigned)parts),
                       dim3(64 * QKN_WAVES), 0, s, (int)p.total, segment_bits(p), p.nq, p.nkv, p.d, eps, log2(theta),
                       packed_pos(p, plan), gq, gk, src, dy, dx, part);
  });
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !part) return e;
  hipLaunchKernelGGL(gain_sum_kernel, dim3((unsigned)((2 * p.d + 63) / 64)), dim3(64 * SUM_GROUPS), 0, s, parts, p.d,
                     (const float*)part, dgq, dgk, accumulate);
  return hipGetLastError();
}

}  // namespace ls

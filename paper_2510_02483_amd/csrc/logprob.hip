// Log probabilities of given tokens, entropies and top alternatives of logits scale h E^T that
// are never kept: what follows the product (gemm_tile.h holds its epilogue).
//
// logprob_rows_kernel joins a row's column blocks (m, s, u), m the block's maximum in base 2, s
// the sum of 2^(z - m) and u that of (z - m) 2^(z - m):
//   M = max m,  S = sum s 2^(m - M),  U = sum 2^(m - M) (u + (m - M) s),
//   lse = (M + log2 S) ln 2,  entropy = (log2 S - U / S) ln 2.
//
// logprob_top_kernel finds the k largest logits of a row from the largest of every 16 columns:
// they lie in the k groups of 16 that come first by (maximum, lower group first): a logit
// outside these is beaten by the maximum of each of them, on a tie by its lower column.  The 16 k
// logits of those groups are formed again, by vector instructions, and the k first by (value,
// lower column first) are the result.  A value formed again differs from the product's
// by the order of its fp32 sum.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace ls {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int LP_THREADS = 1024;
constexpr int LP_WAVES = LP_THREADS / 64;
constexpr int LP_ROWS = 16;  // rows per workgroup of logprob_rows_kernel
constexpr int GROUP = 16;    // columns

struct RowStat {
  float m = -INFINITY, s = 0.f, u = 0.f;
  LS_DEV void join(float bm, float bs, float bu) {
    const float hi = fmaxf(m, bm), ref = hi == -INFINITY ? 0.f : hi;
    const float da = m - ref, db = bm - ref, a = __builtin_amdgcn_exp2f(da), b = __builtin_amdgcn_exp2f(db);
    // (-inf times a sum of 0 would be NaN)
    u = a * fmaf(fmaxf(da, -1000.0f), s, u) + b * fmaf(fmaxf(db, -1000.0f), bs, bu);
    s = a * s + b * bs;
    m = hi;
  }
};

// 16 rows per workgroup and 64 threads per row, each at every 64th column block; then wave 0
// joins the 64.  Bound by latency (few rows) and by reading 16 bytes per row and block.
__global__ __launch_bounds__(LP_THREADS) void logprob_rows_kernel(int64_t T, int V, int64_t blocks, float scale,
                                                                  const f32x4* __restrict__ stats,
                                                                  const float* __restrict__ zt,
                                                                  const int32_t* __restrict__ targets,
                                                                  float* __restrict__ logprob,
                                                                  float* __restrict__ entropy, float* __restrict__ lse) {
  constexpr int PER = LP_THREADS / LP_ROWS;  // threads per row
  __shared__ float pm[PER][LP_ROWS], ps[PER][LP_ROWS], pu[PER][LP_ROWS];
  const int lane = threadIdx.x & 63, r = threadIdx.x % LP_ROWS, k = threadIdx.x / LP_ROWS;
  const int64_t row = (int64_t)blockIdx.x * LP_ROWS + r;
  RowStat st;
  if (row < T) {
#pragma unroll 4
    for (int64_t b = k; b < blocks; b += PER) {
      const f32x4 x = stats[b * T + row];
      st.join(x[0], x[1], x[2]);
    }
  }
  pm[k][r] = st.m;
  ps[k][r] = st.s;
  pu[k][r] = st.u;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  for (int w = k + 64 / LP_ROWS; w < PER; w += 64 / LP_ROWS) st.join(pm[w][r], ps[w][r], pu[w][r]);
#pragma unroll
  for (int o = LP_ROWS; o < 64; o <<= 1) st.join(__shfl_xor(st.m, o), __shfl_xor(st.s, o), __shfl_xor(st.u, o));
  if (lane >= LP_ROWS || row >= T) return;
  const float ls = __log2f(st.s);
  const int t = targets[row];
  const bool ok = t >= 0 && t < V;
  lse[row] = (st.m + ls) * kLn2;
  logprob[row] = ok ? (fmaf(zt[row], scale * kLog2e, -st.m) - ls) * kLn2 : t == -1 ? 0.f : NAN;
  entropy[row] = ok ? (ls - st.u / st.s) * kLn2 : t == -1 ? 0.f : NAN;
}

// The first k by (value, lower index first) of what was offered, one to a lane, in order;
// -inf and no index where there are fewer.  NaN is never among them.
struct TopList {
  float v = -INFINITY;
  int i = INT32_MAX;
  static LS_DEV bool beats(float v, int i, float w, int j) { return v > w || (v == w && i < j); }
  // A value of every lane (index INT32_MAX: none); all lanes take part.
  LS_DEV void offer(float cv, int ci, int k, int lane) {
    for (;;) {
      const float lv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), k - 1));
      const int li = __builtin_amdgcn_readlane(i, k - 1);
      const unsigned long long in = __ballot(ci != INT32_MAX && beats(cv, ci, lv, li));
      if (!in) return;
      const int from = __builtin_ctzll(in);
      const float nv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(cv), from));
      const int ni = __builtin_amdgcn_readlane(ci, from);
      if (lane == from) ci = INT32_MAX;
      const bool ahead = beats(v, i, nv, ni);  // a prefix of the lanes
      const float uv = __shfl_up(v, 1);
      const int ui = __shfl_up(i, 1);
      const int place = __popcll(__ballot(ahead && lane < k));
      if (lane == place) {
        v = nv;
        i = ni;
      } else if (lane > place) {
        v = uv;
        i = ui;
      }
    }
  }
};

// The 16 logits of group `g` for the row's h, unscaled: lane c < 16 gets column 16 g + c (columns past
// the vocabulary are not read).  Every lane works on 8 features of all 16 columns at a time.
LS_DEV float group_logit(const bf16_t* __restrict__ h, const bf16_t* __restrict__ embed, int H, int V, int64_t g,
                         int lane) {
  float acc[GROUP];
#pragma unroll
  for (int c = 0; c < GROUP; ++c) acc[c] = 0.f;
  const bf16_t* e = embed + g * GROUP * H;
  const int last = (int)(V - g * GROUP < GROUP ? V - g * GROUP : GROUP) - 1;
  for (int f = 8 * lane; f < H; f += 512) {
    const u32x4 a = *(const u32x4*)(h + f);
    u32x4 b[GROUP];
#pragma unroll
    for (int c = 0; c < GROUP; ++c) b[c] = *(const u32x4*)(e + (int64_t)(c < last ? c : last) * H + f);
#pragma unroll
    for (int c = 0; c < GROUP; ++c)
#pragma unroll
      for (int w = 0; w < 4; ++w) acc[c] = fmaf(bf_lo(a[w]), bf_lo(b[c][w]), fmaf(bf_hi(a[w]), bf_hi(b[c][w]), acc[c]));
  }
  float out = 0.f;
#pragma unroll
  for (int c = 0; c < GROUP; ++c) {
    const float s = wave_sum(acc[c]);
    if (lane == c) out = s;
  }
  return out;
}

// ROWS 1: a workgroup's 16 waves share a row's groups of columns; their lists are joined
// before its logits are formed, k / 16 groups to a wave.  ROWS 16: a wave to a row; the
// workgroup reads 64 groups of its 16 rows at a time, whole lines, through LDS.
template <int ROWS>
__global__ __launch_bounds__(LP_THREADS) void logprob_top_kernel(int64_t T, int H, int V, int top, float scale,
                                                                 const bf16_t* __restrict__ h,
                                                                 const bf16_t* __restrict__ embed,
                                                                 const float* __restrict__ gmax,
                                                                 const float* __restrict__ lse,
                                                                 int32_t* __restrict__ ids,
                                                                 float* __restrict__ logprob) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int groups = (V + GROUP - 1) / GROUP;
  TopList best;
  int64_t row;
  if constexpr (ROWS == 1) {
    __shared__ float sv[LP_WAVES][LOGPROB_TOP];
    __shared__ int si[LP_WAVES][LOGPROB_TOP];
    row = blockIdx.x;
    for (int g0 = 64 * wave; g0 < groups; g0 += LP_THREADS) {
      const int g = g0 + lane;
      best.offer(g < groups ? gmax[(int64_t)g * T + row] : 0.f, g < groups ? g : INT32_MAX, top, lane);
    }
    sv[wave][lane] = best.v;
    si[wave][lane] = best.i;
    __syncthreads();
    best = TopList{};  // every wave joins all lists
    for (int w = 0; w < LP_WAVES; ++w) best.offer(sv[w][lane], lane < top ? si[w][lane] : INT32_MAX, top, lane);
    __syncthreads();
    TopList mine;  // this wave's groups
    for (int n = wave; n < top; n += LP_WAVES) {
      const int g = __builtin_amdgcn_readlane(best.i, n);
      if (g >= groups) continue;
      const float z = group_logit(h + row * H, embed, H, V, g, lane);
      mine.offer(z, lane < GROUP && g * GROUP + lane < V ? g * GROUP + lane : INT32_MAX, top, lane);
    }
    sv[wave][lane] = mine.v;
    si[wave][lane] = mine.i;
    __syncthreads();
    if (wave > 0) return;
    best = mine;
    for (int w = 1; w < LP_WAVES && w < top; ++w) best.offer(sv[w][lane], lane < top ? si[w][lane] : INT32_MAX, top, lane);
  } else {
    static_assert(ROWS == LP_WAVES, "a wave to a row");
    __shared__ float tile[2][ROWS][64 + 1];
    const int64_t row0 = (int64_t)blockIdx.x * ROWS;
    row = row0 + wave;
    const int r = threadIdx.x % ROWS, gg = threadIdx.x / ROWS;
    const bool in = row0 + r < T;
    auto load = [&](int g0) { return in && g0 + gg < groups ? gmax[(int64_t)(g0 + gg) * T + row0 + r] : 0.f; };
    float next = load(0);
    int at = 0;
    for (int g0 = 0; g0 < groups; g0 += 64, at ^= 1) {
      tile[at][r][gg] = next;
      if (g0 + 64 < groups) next = load(g0 + 64);
      __syncthreads();
      const int g = g0 + lane;
      best.offer(tile[at][wave][lane], g < groups ? g : INT32_MAX, top, lane);
    }
    if (row >= T) return;
    TopList mine;
    for (int n = 0; n < top; ++n) {
      const int g = __builtin_amdgcn_readlane(best.i, n);
      if (g >= groups) break;
      const float z = group_logit(h + row * H, embed, H, V, g, lane);
      mine.offer(z, lane < GROUP && g * GROUP + lane < V ? g * GROUP + lane : INT32_MAX, top, lane);
    }
    best = mine;
  }
  if (lane >= top) return;
  ids[row * top + lane] = best.i == INT32_MAX ? -1 : best.i;
  logprob[row * top + lane] = best.i == INT32_MAX ? -INFINITY : best.v * scale - lse[row];
}

}  // namespace

hipError_t logprob_rows(int64_t T, int V, int64_t blocks, float scale, const float* stats, const float* zt,
                        const int32_t* targets, float* logprob, float* entropy, float* lse, hipStream_t s) {
  hipLaunchKernelGGL(logprob_rows_kernel, dim3((unsigned)((T + LP_ROWS - 1) / LP_ROWS)), dim3(LP_THREADS), 0, s, T, V,
                     blocks, scale, (const f32x4*)stats, zt, targets, logprob, entropy, lse);
  return hipGetLastError();
}

hipError_t logprob_top(int64_t T, int H, int V, int top, float scale, const bf16_t* h, const bf16_t* embed,
                       const float* gmax, const float* lse, int32_t* ids, float* logprob, hipStream_t s) {
  if (T <= 1024)
    hipLaunchKernelGGL((logprob_top_kernel<1>), dim3((unsigned)T), dim3(LP_THREADS), 0, s, T, H, V, top, scale, h, embed,
                       gmax, lse, ids, logprob);
  else
    hipLaunchKernelGGL((logprob_top_kernel<16>), dim3((unsigned)((T + 15) / 16)), dim3(LP_THREADS), 0, s, T, H, V, top,
                       scale, h, embed, gmax, lse, ids, logprob);
  return hipGetLastError();
}

}  // namespace ls

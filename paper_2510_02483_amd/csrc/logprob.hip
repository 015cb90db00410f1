// Log probabilities of given tokens, entropies and top alternatives of logits scale h E^T that
// are never kept: what follows the product (gemm_tile.h holds its epilogue).
//
// logprob_rows_kernel joins a row's column blocks (m, s, u), m the block's maximum in base 2, s
// the sum of 2^(z - m) and u that of (z - m) 2^(z - m):
//   M = max m,  S = sum s 2^(m - M),  U = sum 2^(m - M) (u + (m - M) s),
//   lse = (M + log2 S) ln 2,  entropy = (log2 S - U / S) ln 2.
//
// The k largest logits of a row are found from the largest of every 8 columns: they lie in the
// k groups of 8 that come first by (maximum, lower group first): a logit
// outside these is beaten by the maximum of each of them, on a tie by its lower column.  The 8 k
// logits of those groups are formed again, by vector instructions, and the k first by (value,
// lower column first) are the result.  A value formed again differs from the product's
// by the order of its fp32 sum.  Groups of 8 balance the two: 4096 rows, hidden 2048, vocabulary 128256, five
// alternatives: 262 MB of maxima written and read and 0.7 GB of head weights read again, 187 us for both
// (groups of 16, 131 MB and 1.3 GB: 288 us with the maxima by group, rows next to each other).
#include <math.h>

#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace ls {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int LP_THREADS = 1024;
constexpr int LP_WAVES = LP_THREADS / 64;
constexpr int LP_ROWS = 16;  // rows per workgroup of logprob_rows_kernel
constexpr int GROUP = 8;     // columns

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

// A row's three results from its joined statistics.
LS_DEV void finish_row(const LogprobRows& x, int V, int64_t row, const RowStat& st, int t, float zt) {
  const float ls = __log2f(st.s);
  const bool ok = t >= 0 && t < V;
  x.lse[row] = (st.m + ls) * kLn2;
  x.logprob[row] = ok ? (fmaf(zt, x.scale * kLog2e, -st.m) - ls) * kLn2 : t == -1 ? 0.f : NAN;
  x.entropy[row] = ok ? (ls - st.u / st.s) * kLn2 : t == -1 ? 0.f : NAN;
}

// 16 rows per workgroup and 64 threads per row, each at every 64th column block; then wave 0
// joins the 64.  Bound by latency (few rows) and by reading 16 bytes per row and block.
__global__ __launch_bounds__(LP_THREADS) void logprob_rows_kernel(int64_t T, int V, LogprobRows x) {
  constexpr int PER = LP_THREADS / LP_ROWS;  // threads per row
  __shared__ float pm[PER][LP_ROWS], ps[PER][LP_ROWS], pu[PER][LP_ROWS];
  const int lane = threadIdx.x & 63, r = threadIdx.x % LP_ROWS, k = threadIdx.x / LP_ROWS;
  const int64_t row = (int64_t)blockIdx.x * LP_ROWS + r;
  RowStat st;
  if (row < T) {
#pragma unroll 4
    for (int64_t b = k; b < x.blocks; b += PER) {
      const f32x4 v = ((const f32x4*)x.stats)[b * T + row];
      st.join(v[0], v[1], v[2]);
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
  finish_row(x, V, row, st, x.targets[row], x.zt[row]);
}

// The first k by (value, lower index first) of what was offered, one to a lane, in order;
// -inf and no index where there are fewer.  NaN is never among them.
struct TopList {
  float v = -INFINITY;
  int i = INT32_MAX;
  static LS_DEV uint32_t lane_below(uint32_t x) {  // (DPP wave_shr:1)
    return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x138, 0xf, 0xf, false);
  }
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
      const float uv = __uint_as_float(lane_below(__float_as_uint(v)));
      const int ui = (int)lane_below((uint32_t)i);
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

// N (4 or 8) logits of columns c0 .. for the row's h, unscaled: a lane gets that of column c0 + lane % N (columns past the
// vocabulary are not read).  Every lane works on 8 features of all columns at a time; the sums of the
// lanes' shares are formed N to a wave at once, half the columns going to either half of the lanes.
template <int N, int UNROLL>
LS_DEV float logits(const bf16_t* __restrict__ h, const bf16_t* __restrict__ embed, int H, int V, int64_t c0, int lane) {
  float acc[N];
#pragma unroll
  for (int c = 0; c < N; ++c) acc[c] = 0.f;
  const bf16_t* e = embed + c0 * H;
  const int last = (int)(V - c0 < N ? V - c0 : N) - 1;
#pragma unroll UNROLL
  for (int f = 8 * lane; f < H; f += 512) {
    const u32x4 a = *(const u32x4*)(h + f);
    u32x4 b[N];
#pragma unroll
    for (int c = 0; c < N; ++c) b[c] = *(const u32x4*)(e + (int64_t)(c < last ? c : last) * H + f);
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
      for (int w = 0; w < 4; ++w) acc[c] = fmaf(bf_lo(a[w]), bf_lo(b[c][w]), fmaf(bf_hi(a[w]), bf_hi(b[c][w]), acc[c]));
  }
#pragma unroll
  for (int o = N / 2; o >= 1; o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int c = 0; c < o; ++c) {
      const float other = __shfl_xor(up ? acc[c] : acc[c + o], o);
      acc[c] = (up ? acc[c + o] : acc[c]) + other;
    }
  }
  float sum = acc[0];
#pragma unroll
  for (int o = N; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
  return sum;
}

// One row to a workgroup, for few rows: the time of the longest chain counts.  Of the largest group of each thread
// each wave takes its first (its second, .. with more than 16 alternatives): the `top` first of these bound the groups
// that can be among the first `top` from below, and the few that the bound does not beat are
// collected.  The place of each among all of them is counted by a thread each; the chosen groups' logits, 4 columns to a wave
// at a time, are placed the same way.  (Should values lie so that more than 1024 pass the bound, every wave
// keeps a list of its own instead.)  The row's statistics are joined here too, which saves a launch.
// Vocabulary 32000, hidden 2048, eight alternatives of one row: 14 us, of which 5 wait for the weights.
struct TopRows {
  float v[LP_WAVES * LOGPROB_TOP];  // groups, then logits of the chosen groups
  int i[LP_WAVES * LOGPROB_TOP];
  float bv[LP_WAVES];  // the waves' parts of the bound
  int bi[LP_WAVES], count;
  float ov[LOGPROB_TOP];  // chosen
  int oi[LOGPROB_TOP];
  float sm[LP_WAVES], ss[LP_WAVES], su[LP_WAVES];  // the waves' statistics of the row
  float lse;
};
__global__ __launch_bounds__(LP_THREADS) void logprob_top_one_kernel(int64_t T, int H, int V, int top, LogprobRows x,
                                                                     const bf16_t* __restrict__ h,
                                                                     const bf16_t* __restrict__ embed,
                                                                     GroupMax gmax,
                                                                     int32_t* __restrict__ ids,
                                                                     float* __restrict__ logprob) {
  __shared__ __attribute__((aligned(16))) TopRows sh;
  static_assert(GROUP * LOGPROB_TOP <= LP_WAVES * LOGPROB_TOP, "the chosen groups' logits fit");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t row = blockIdx.x;
  const int groups = (V + GROUP - 1) / GROUP;
  // the first `top` of n (a multiple of 4) entries of sh.v, sh.i, in order, to ov, oi; entries with no index never
  auto choose = [&](int n) {
    if (tid < LOGPROB_TOP) {
      sh.ov[tid] = -INFINITY;
      sh.oi[tid] = INT32_MAX;
    }
    __syncthreads();
    if (tid < n && sh.i[tid] != INT32_MAX) {
      const float v = sh.v[tid];
      const int i = sh.i[tid];
      int place = 0;
#pragma unroll 4
      for (int j = 0; j < n; j += 4) {
        const f32x4 w = *(const f32x4*)&sh.v[j];
        const i32x4 u = *(const i32x4*)&sh.i[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) place += TopList::beats(w[e], u[e], v, i);
      }
      if (place < top) {
        sh.ov[place] = v;
        sh.oi[place] = i;
      }
    }
    __syncthreads();
  };

  // (zt is written for a target in [0, V) only)
  const int target = tid == 0 ? x.targets[row] : 0;
  const float zt = tid == 0 ? x.zt[row] : 0.f;
  RowStat st;
  for (int64_t b = tid; b < x.blocks; b += LP_THREADS) {
    const f32x4 v = ((const f32x4*)x.stats)[b * T + row];
    st.join(v[0], v[1], v[2]);
  }
  // the thread's largest, then the wave's
  float v = -INFINITY;
  int i = INT32_MAX;
#pragma unroll 4
  for (int g = tid; g < groups; g += LP_THREADS) {
    const float u = gmax.v[gmax_at(gmax.groups, gmax.rows, row, g)];
    if (TopList::beats(u, g, v, i)) {
      v = u;
      i = g;
    }
  }
  for (int n = (top + LP_WAVES - 1) / LP_WAVES; n > 0; --n) {
    const float wv = wave_max(v);
    const unsigned long long in = __ballot(i != INT32_MAX && v == wv);
    // (lanes hold groups in no order: of equal ones the lowest)
    int wi = INT32_MAX;
    for (unsigned long long left = in; left; left &= left - 1)
      wi = min(wi, __builtin_amdgcn_readlane(i, __builtin_ctzll(left)));
    if (lane == 0) {
      sh.bv[wave] = wi == INT32_MAX ? -INFINITY : wv;
      sh.bi[wave] = wi;
    }
    if (i == wi) {
      v = -INFINITY;
      i = INT32_MAX;
    }
  }
  if (tid == 0) sh.count = 0;
  __syncthreads();
  float bv = -INFINITY;
  int bi = INT32_MAX;
  {
    const float mv = sh.bv[lane % LP_WAVES];
    const int mi = sh.bi[lane % LP_WAVES];
    int place = 0;
#pragma unroll
    for (int w = 0; w < LP_WAVES; ++w) place += TopList::beats(sh.bv[w], sh.bi[w], mv, mi);
    const unsigned long long in = __ballot(mi != INT32_MAX && place == min(top, LP_WAVES) - 1);
    if (in) {  // (else there are fewer groups than that: all pass)
      bv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mv), __builtin_ctzll(in)));
      bi = __builtin_amdgcn_readlane(mi, __builtin_ctzll(in));
    }
  }
#pragma unroll 4
  for (int g = tid; g < groups; g += LP_THREADS) {
    const float u = gmax.v[gmax_at(gmax.groups, gmax.rows, row, g)];
    if (!TopList::beats(bv, bi, u, g)) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < LP_THREADS) {
        sh.v[at] = u;
        sh.i[at] = g;
      }
    }
  }
  __syncthreads();
  int n = sh.count;
  if (n > LP_THREADS) {
    n = LP_WAVES * top;
    TopList best;
    for (int g0 = 64 * wave; g0 < groups; g0 += LP_THREADS) {
      const int g = g0 + lane;
      best.offer(g < groups ? gmax.v[gmax_at(gmax.groups, gmax.rows, row, g)] : 0.f, g < groups ? g : INT32_MAX, top, lane);
    }
    if (lane < top) {
      sh.v[wave * top + lane] = best.v;
      sh.i[wave * top + lane] = best.i;
    }
  } else if (tid < (-n & 3)) {
    sh.v[n + tid] = -INFINITY;
    sh.i[n + tid] = INT32_MAX;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) st.join(__shfl_xor(st.m, o), __shfl_xor(st.s, o), __shfl_xor(st.u, o));
  if (lane == 0) {
    sh.sm[wave] = st.m;
    sh.ss[wave] = st.s;
    sh.su[wave] = st.u;
  }
  choose((n + 3) & ~3);
  for (int q = wave; q < 2 * top; q += LP_WAVES) {
    const int g = __builtin_amdgcn_readfirstlane(sh.oi[q >> 1]);
    const int64_t c0 = (int64_t)g * GROUP + 4 * (q & 1);
    const bool any = g < groups && c0 < V;
    const float z = any ? logits<4, 4>(h + row * H, embed, H, V, c0, lane) : NAN;
    if (lane < 4) {  // a NaN is no alternative
      const bool ok = any && c0 + lane < V && z == z;
      sh.v[4 * q + lane] = ok ? z : -INFINITY;
      sh.i[4 * q + lane] = ok ? (int)c0 + lane : INT32_MAX;
    }
  }
  if (tid == 0) {
    for (int w = 1; w < LP_WAVES; ++w) st.join(sh.sm[w], sh.ss[w], sh.su[w]);
    finish_row(x, V, row, st, target, zt);
    sh.lse = (st.m + __log2f(st.s)) * kLn2;
  }
  __syncthreads();  // (the chosen groups have been read)
  choose(GROUP * top);
  if (tid >= top) return;
  i = sh.oi[tid];
  ids[row * top + tid] = i == INT32_MAX ? -1 : i;
  logprob[row * top + tid] = i == INT32_MAX ? -INFINITY : sh.ov[tid] * x.scale - sh.lse;
}

// A wave to a row, for many rows; the workgroup reads 1024 groups of its 16 (or 4) rows at a time through LDS, the next
// 1024 in flight meanwhile (with 256, which are 16 KB to a compute unit, memory's latency bounds it: 224 us at the size
// above).  Bound by reading the chosen groups' head weights again.
template <int ROWS>
__global__ __launch_bounds__(64 * ROWS) void logprob_top_kernel(int64_t T, int H, int V, int top, float scale,
                                                                 const bf16_t* __restrict__ h,
                                                                 const bf16_t* __restrict__ embed,
                                                                 GroupMax gmax,
                                                                 const float* __restrict__ lse,
                                                                 int32_t* __restrict__ ids,
                                                                 float* __restrict__ logprob) {
  constexpr int CHUNKS = 16;
  __shared__ float tile[2][ROWS][64 * CHUNKS + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int groups = (V + GROUP - 1) / GROUP;
  TopList best;
  const int64_t row0 = (int64_t)blockIdx.x * ROWS, row = row0 + wave;
  const int r = threadIdx.x % ROWS, gg = threadIdx.x / ROWS;
  const bool in = row0 + r < T;
  float next[CHUNKS];
  auto load = [&](int g0) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int g = g0 + 64 * c + gg;
      next[c] = in && g < groups ? gmax.v[gmax_at(gmax.groups, gmax.rows, row0 + r, g)] : -INFINITY;
    }
  };
  load(0);
  int at = 0;
  for (int g0 = 0; g0 < groups; g0 += 64 * CHUNKS, at ^= 1) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) tile[at][r][64 * c + gg] = next[c];
    load(g0 + 64 * CHUNKS);
    __syncthreads();
#pragma unroll 1
    for (int c0 = 0; c0 < CHUNKS; c0 += 4) {
      // (one look at four, as most are beaten by the list's last; an equal one comes later and is beaten too)
      float most = -INFINITY;
#pragma unroll
      for (int c = c0; c < c0 + 4; ++c) most = fmaxf(most, tile[at][wave][64 * c + lane]);
      const float lv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(best.v), top - 1));
      const int li = __builtin_amdgcn_readlane(best.i, top - 1);
      if (li != INT32_MAX && !__ballot(most > lv)) continue;
#pragma unroll 1
      for (int c = c0; c < c0 + 4; ++c) {
        const int g = g0 + 64 * c + lane;
        best.offer(tile[at][wave][64 * c + lane], g < groups ? g : INT32_MAX, top, lane);
      }
    }
  }
  if (row >= T) return;
  TopList mine;
  for (int n = 0; n < top; ++n) {
    const int g = __builtin_amdgcn_readlane(best.i, n);
    if (g >= groups) break;
    const float z = logits<GROUP, 2>(h + row * H, embed, H, V, (int64_t)g * GROUP, lane);
    mine.offer(z, lane < GROUP && g * GROUP + lane < V ? g * GROUP + lane : INT32_MAX, top, lane);
  }
  if (lane >= top) return;
  ids[row * top + lane] = mine.i == INT32_MAX ? -1 : mine.i;
  logprob[row * top + lane] = mine.i == INT32_MAX ? -INFINITY : mine.v * scale - lse[row];
}

}  // namespace

hipError_t logprob_rows(int64_t T, int V, const LogprobRows& x, hipStream_t s) {
  hipLaunchKernelGGL(logprob_rows_kernel, dim3((unsigned)((T + LP_ROWS - 1) / LP_ROWS)), dim3(LP_THREADS), 0, s, T, V, x);
  return hipGetLastError();
}

hipError_t logprob_top(int64_t T, int H, int V, int top, const LogprobRows& x, const bf16_t* h, const bf16_t* embed,
                       const GroupMax& gmax, int32_t* ids, float* logprob, hipStream_t s) {
  // us for all rows, one to a workgroup / 4 / 16 (hidden 2048): vocabulary 32000, five alternatives, 512 rows 41 / 52 / 72,
  // 1024 rows 77 / 55 / 73, 4096 rows 279 / 153 / 145; vocabulary 128256 96 / 83 / 108, 187 / 87 / 118 and 734 / 268 / 192;
  // 64 alternatives, 1024 rows 382 / 393 / 570 and 504 / 490 / 875, 2048 rows 722 / 783 / 764 and 968 / 855 / 944
  if (T <= (top > 16 ? 1024 : 512)) {
    hipLaunchKernelGGL(logprob_top_one_kernel, dim3((unsigned)T), dim3(LP_THREADS), 0, s, T, H, V, top, x, h, embed, gmax,
                       ids, logprob);
    return hipGetLastError();
  }
  const hipError_t e = logprob_rows(T, V, x, s);
  if (e != hipSuccess) return e;
  auto launch = [&](auto rows) {
    constexpr int ROWS = decltype(rows)::value;
    hipLaunchKernelGGL((logprob_top_kernel<ROWS>), dim3((unsigned)((T + ROWS - 1) / ROWS)), dim3(64 * ROWS), 0, s, T, H, V,
                       top, x.scale, h, embed, gmax, (const float*)x.lse, ids, logprob);
  };
  if (T <= 1024) launch(std::integral_constant<int, 4>{});
  else launch(std::integral_constant<int, 16>{});
  return hipGetLastError();
}

}  // namespace ls

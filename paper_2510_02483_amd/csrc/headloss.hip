// The cross-entropy of logits h E^T that are never kept: what follows and precedes
// the products (gemm_tile.h holds their epilogues).
//
// Forward: z = h E^T tile by tile; each wave leaves the maximum and the sum of
// exponentials of its 128 (or 64) columns per row, 8 bytes for 128 logits, and the
// target's logit.  head_rows_kernel joins a row's blocks:
//   lse = M + ln sum_b s_b exp(m_b - M),  M = max m_b.
// Backward: the n rows that have a target are gathered first, so that prompts and
// padding cost nothing and whatever their h holds (uninitialised memory, NaN) reaches
// no gradient; n stays on the device, where the products read it.  Then for each piece
// of the vocabulary: z again, dz = softmax(z) - onehot in bf16, dh += dz E_piece in
// fp32 and dE_piece = (dloss / N) dz^T h.  At the end dh goes back to its rows, times
// dloss / N, in bf16.
//
// The products are bound by the matrix cores (2 T V H operations forward, 6 n V H
// backward), the kernels here by memory and latency: 8 bytes per row and column
// block forward, a copy of h and of dh backward.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace ls {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int HL_THREADS = 1024;
constexpr int HL_WAVES = HL_THREADS / 64;
constexpr int HL_ROWS = 16;     // rows per workgroup of head_rows_kernel
constexpr int HL_GATHER = 512;  // threads of the gathering workgroups

LS_DEV bool has_target(int t, int V) { return t >= 0 && t < V; }

// Sums v and n over the workgroup in a fixed order (valid in thread 0).
LS_DEV void block_sums(double& v, int& n, double* vp, int* np) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    v += __shfl_xor(v, o);
    n += __shfl_xor(n, o);
  }
  if ((threadIdx.x & 63) == 0) {
    vp[threadIdx.x >> 6] = v;
    np[threadIdx.x >> 6] = n;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    v = 0.0;
    n = 0;
    for (int w = 0; w < HL_WAVES; ++w) {
      v += vp[w];
      n += np[w];
    }
  }
}

// A row's maximum and sum of exponentials, joined from its column blocks.  A block
// without finite logits (max -inf, sum 0) changes nothing.
struct RowStat {
  float m = -INFINITY, s = 0.f;
  LS_DEV void join(float bm, float bs) {
    const float hi = fmaxf(m, bm);
    const float ref = hi == -INFINITY ? 0.f : hi;
    s = s * __builtin_amdgcn_exp2f((m - ref) * kLog2e) + bs * __builtin_amdgcn_exp2f((bm - ref) * kLog2e);
    m = hi;
  }
  // Writes the row's results; returns its loss and whether it counts.
  LS_DEV float finish(int64_t row, int V, const float* zt, const int32_t* targets, float* lse, float* row_loss,
                      int& n) const {
    const float l = m + __log2f(s) * kLn2;
    const int t = targets[row];
    const float r = t == -1 ? 0.f : has_target(t, V) ? l - zt[row] : NAN;
    lse[row] = l;
    row_loss[row] = r;
    n = has_target(t, V);
    return r;
  }
};

// 16 rows per workgroup and 64 threads per row, each at every 64th column block (16
// neighbouring rows' 8 bytes are one 128-byte line); then wave 0 joins the 64.  A
// lone workgroup also forms the loss.  Bound by latency (few rows: the walk over
// the blocks) and by reading 8 bytes per row and block: with the mean's launch 11 to
// 14 us for 256 to 4096 rows of 1002 blocks; 64 rows per workgroup took 15 to 17.
__global__ __launch_bounds__(HL_THREADS) void head_rows_kernel(int64_t T, int V, int64_t blocks,
                                                               const float2* __restrict__ stats,
                                                               const float* __restrict__ zt,
                                                               const int32_t* __restrict__ targets,
                                                               float* __restrict__ lse, float* __restrict__ row_loss,
                                                               float* __restrict__ loss) {
  constexpr int PER = HL_THREADS / HL_ROWS;  // threads per row
  __shared__ float pm[PER][HL_ROWS], ps[PER][HL_ROWS];
  const int lane = threadIdx.x & 63, r = threadIdx.x % HL_ROWS, k = threadIdx.x / HL_ROWS;
  const int64_t row = (int64_t)blockIdx.x * HL_ROWS + r;
  RowStat st;
  if (row < T) {
#pragma unroll 4
    for (int64_t b = k; b < blocks; b += PER) {
      const float2 x = stats[b * T + row];
      st.join(x.x, x.y);
    }
  }
  pm[k][r] = st.m;
  ps[k][r] = st.s;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  for (int w = k + 64 / HL_ROWS; w < PER; w += 64 / HL_ROWS) st.join(pm[w][r], ps[w][r]);
#pragma unroll
  for (int o = HL_ROWS; o < 64; o <<= 1) st.join(__shfl_xor(st.m, o), __shfl_xor(st.s, o));
  int n = 0;
  float v = 0.f;
  if (lane < HL_ROWS && row < T) v = st.finish(row, V, zt, targets, lse, row_loss, n);
  if (gridDim.x > 1) return;
  double sum = (double)v;
#pragma unroll
  for (int o = 1; o < HL_ROWS; o <<= 1) {
    sum += __shfl_xor(sum, o);
    n += __shfl_xor(n, o);
  }
  if (lane == 0) loss[0] = (float)(sum / (double)max(n, 1));
}

// One workgroup: loss = sum of row losses over the rows that have a target, in fp64 in a fixed order.
__global__ __launch_bounds__(HL_THREADS) void head_mean_kernel(int64_t T, int V, const int32_t* __restrict__ targets,
                                                               const float* __restrict__ row_loss,
                                                               float* __restrict__ loss) {
  __shared__ double vp[HL_WAVES];
  __shared__ int np[HL_WAVES];
  double v = 0.0;
  int n = 0;
  for (int64_t t = threadIdx.x; t < T; t += HL_THREADS) {
    v += (double)row_loss[t];
    n += has_target(targets[t], V);
  }
  block_sums(v, n, vp, np);
  if (threadIdx.x == 0) loss[0] = (float)(v / (double)max(n, 1));
}

// The rows that have a target (any but -1), gathered in their order: every row's
// place among them (-1: none), their number, their targets, lse and h, and the
// factor of all gradients.  A workgroup takes `per` rows and counts the targets before
// them by itself (4 bytes a row, from the L2), so that one launch does it all; the
// last one sees every row and leaves the number and the factor.
// Bound by HBM bandwidth: h is read once and written once.
__global__ __launch_bounds__(HL_GATHER) void head_gather_kernel(int64_t T, int H, int V, int64_t per,
                                                                const int32_t* __restrict__ targets,
                                                                const float* __restrict__ dloss,
                                                                const bf16_t* __restrict__ h,
                                                                const float* __restrict__ lse,
                                                                int32_t* __restrict__ slot, int* __restrict__ rows,
                                                                float* __restrict__ coef, bf16_t* __restrict__ hc,
                                                                int32_t* __restrict__ tc, float* __restrict__ lc) {
  constexpr int WAVES = HL_GATHER / 64;
  __shared__ int part[2][WAVES], place[HL_GATHER];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r0 = (int64_t)blockIdx.x * per, r1 = r0 + per < T ? r0 + per : T;
  int before = 0, valid = 0;
  for (int64_t t = tid; t < r0; t += HL_GATHER) {
    const int g = targets[t];
    before += g != -1;
    valid += has_target(g, V);
  }
  auto sum = [&](int v, int* p) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
    if (lane == 0) p[wave] = v;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all += p[w];
    return all;
  };
  before = sum(before, part[0]);
  for (int64_t c0 = r0; c0 < r1; c0 += HL_GATHER) {
    const int64_t t = c0 + tid;
    const int g = t < r1 ? targets[t] : -1;
    valid += has_target(g, V);
    const unsigned long long in = __ballot(g != -1);
    if (lane == 0) part[1][wave] = __popcll(in);
    __syncthreads();
    int at = before + __popcll(in & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      at += w < wave ? part[1][w] : 0;
      before += part[1][w];
    }
    place[tid] = g == -1 ? -1 : at;
    if (t < r1) {
      slot[t] = place[tid];
      if (g != -1) {
        tc[at] = g;
        lc[at] = lse[t];
      }
    }
    __syncthreads();
    const int n = (int)(r1 - c0 < HL_GATHER ? r1 - c0 : HL_GATHER);
    for (int k = wave; k < n; k += WAVES) {
      const int to = place[k];
      if (to < 0) continue;
      const u32x4* src = (const u32x4*)(h + (c0 + k) * H);
      u32x4* dst = (u32x4*)(hc + (int64_t)to * H);
      for (int c = lane; c < H / 8; c += 64) dst[c] = src[c];
    }
    __syncthreads();
  }
  if (blockIdx.x + 1 < gridDim.x) return;
  valid = sum(valid, part[0]);
  if (tid == 0) {
    rows[0] = before;
    coef[0] = (dloss ? dloss[0] : 1.0f) / (float)max(valid, 1);
  }
}

// One wave per row; the only rounding of dh.
__global__ __launch_bounds__(256) void head_scatter_kernel(int64_t T, int H, const int32_t* __restrict__ slot,
                                                           const float* __restrict__ coef,
                                                           const float* __restrict__ dhc, bf16_t* __restrict__ dh) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= T) return;
  const int at = slot[t];
  u32x4* dst = (u32x4*)(dh + t * H);
  if (at < 0) {
    for (int c = lane; c < H / 8; c += 64) dst[c] = u32x4{0u, 0u, 0u, 0u};
    return;
  }
  const float k = coef[0];
  const f32x4* src = (const f32x4*)(dhc + (int64_t)at * H);
  for (int c = lane; c < H / 8; c += 64) {
    const f32x4 a = src[2 * c] * k, b = src[2 * c + 1] * k;
    dst[c] = u32x4{pack_bf2(a[0], a[1]), pack_bf2(a[2], a[3]), pack_bf2(b[0], b[1]), pack_bf2(b[2], b[3])};
  }
}

}  // namespace

hipError_t head_rows(int64_t T, int V, int64_t blocks, const float* stats, const float* zt, const int32_t* targets,
                     float* lse, float* row_loss, float* loss, hipStream_t s) {
  const unsigned grid = (unsigned)((T + HL_ROWS - 1) / HL_ROWS);
  hipLaunchKernelGGL(head_rows_kernel, dim3(grid), dim3(HL_THREADS), 0, s, T, V, blocks, (const float2*)stats, zt,
                     targets, lse, row_loss, loss);
  if (grid == 1) return hipGetLastError();
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(head_mean_kernel, dim3(1), dim3(HL_THREADS), 0, s, T, V, targets, row_loss, loss);
  return hipGetLastError();
}

hipError_t head_gather(int64_t T, int H, int V, const int32_t* targets, const float* dloss, const bf16_t* h,
                       const float* lse, int32_t* slot, int* rows, float* coef, bf16_t* hc, int32_t* tc, float* lc,
                       hipStream_t s) {
  // a row per wave, or as many as leave 512 workgroups
  int64_t per = (T + 511) / 512;
  if (per < HL_GATHER / 64) per = HL_GATHER / 64;
  hipLaunchKernelGGL(head_gather_kernel, dim3((unsigned)((T + per - 1) / per)), dim3(HL_GATHER), 0, s, T, H, V, per,
                     targets, dloss, h, lse, slot, rows, coef, hc, tc, lc);
  return hipGetLastError();
}

hipError_t head_scatter(int64_t T, int H, const int32_t* slot, const float* coef, const float* dhc, bf16_t* dh,
                        hipStream_t s) {
  hipLaunchKernelGGL(head_scatter_kernel, dim3((unsigned)((T + 3) / 4)), dim3(256), 0, s, T, H, slot, coef, dhc, dh);
  return hipGetLastError();
}

}  // namespace ls

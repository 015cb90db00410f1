// The norm of many gradient tensors together, and the tensors clipped by it.
//
//   norm = sqrt(sum over all tensors of g^2),  out = g min(1, max_norm / (norm + 1e-6)).
//
// Tensors are taken in chunks of GN_CHUNK elements, numbered through all tensors of a
// launch; the table of up to GN_TENSORS tensors is a kernel argument, so that nothing is copied to
// the device first and a captured launch holds it.  Workgroup b of a fixed number takes chunks
// b, b + GN_BLOCKS, ..: its sum of squares, in fp64 (the square of any finite value is), goes
// to partial[b], added to by the launches of further tensors; the order of all sums depends
// on the tensors' sizes only.
//
// Bound by HBM bandwidth: the norm reads every gradient once, clipping reads and
// writes each once.  5.3e8 fp32 elements: norm 370 us (5.7 TB/s), clipped into bf16 583 us (5.5 TB/s; from the last tensor
// on, which the norm read last, no less: the last-level cache keeps little of a stream).
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace ls {

namespace {

constexpr int GN_THREADS = 256;
constexpr int GN_BLOCKS = 2048;
constexpr int GN_CHUNK = 16384;  // elements: 16 loads of 16 bytes of fp32 to a thread

struct GradTable {
  const void* in[GN_TENSORS];
  void* out[GN_TENSORS];
  int64_t n[GN_TENSORS];
  uint32_t first[GN_TENSORS + 1];  // a tensor's first chunk
  uint32_t in_bf16[(GN_TENSORS + 31) / 32], out_bf16[(GN_TENSORS + 31) / 32];
  int tensors;
};
static_assert(sizeof(GradTable) < 3584, "a kernel's arguments hold 4 KB");

// Calls f(tensor, first element, elements) for each chunk of the workgroup.
template <class F>
LS_DEV void for_chunks(const GradTable& t, F&& f) {
  const uint32_t chunks = t.first[t.tensors];
  for (uint32_t k = blockIdx.x; k < chunks; k += gridDim.x) {
    int lo = 0, hi = t.tensors;  // the last tensor whose first chunk is k or before (empty ones have none)
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (t.first[mid] <= k) lo = mid;
      else hi = mid;
    }
    const int64_t at = (int64_t)(k - t.first[lo]) * GN_CHUNK;
    const int64_t left = t.n[lo] - at;
    f(lo, at, (int)(left < GN_CHUNK ? left : GN_CHUNK));
  }
}
LS_DEV bool bit(const uint32_t* w, int i) { return w[i / 32] >> (i % 32) & 1; }

__global__ __launch_bounds__(GN_THREADS) void grad_sumsq_kernel(GradTable t, double* __restrict__ partial, int add) {
  __shared__ double red[GN_THREADS / 64];
  const int tid = threadIdx.x;
  double acc = 0.0;
  for_chunks(t, [&](int i, int64_t at, int n) {
    if (bit(t.in_bf16, i)) {
      const bf16_t* p = (const bf16_t*)t.in[i] + at;
#pragma unroll 8
      for (int j = tid; j < n / 8; j += GN_THREADS) {
        const u32x4 x = ((const u32x4*)p)[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double a = bf_lo(x[e]), b = bf_hi(x[e]);
          acc += a * a;
          acc += b * b;
        }
      }
      for (int j = (n & ~7) + tid; j < n; j += GN_THREADS) {
        const double a = bf2f(p[j]);
        acc += a * a;
      }
    } else {
      const float* p = (const float*)t.in[i] + at;
#pragma unroll 8
      for (int j = tid; j < n / 4; j += GN_THREADS) {
        const f32x4 x = ((const f32x4*)p)[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc += (double)x[e] * x[e];
      }
      for (int j = (n & ~3) + tid; j < n; j += GN_THREADS) acc += (double)p[j] * p[j];
    }
  });
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) acc += __shfl_xor(acc, o);
  if ((tid & 63) == 0) red[tid >> 6] = acc;
  __syncthreads();
  if (tid == 0) {
    double s = add ? partial[blockIdx.x] : 0.0;
#pragma unroll
    for (int w = 0; w < GN_THREADS / 64; ++w) s += red[w];
    partial[blockIdx.x] = s;
  }
}

// One workgroup: norm = sqrt(sum partial).
__global__ __launch_bounds__(GN_THREADS) void grad_norm_kernel(int parts, const double* __restrict__ partial,
                                                               float* __restrict__ norm) {
  __shared__ double red[GN_THREADS / 64];
  double acc = 0.0;
#pragma unroll 8
  for (int i = threadIdx.x; i < parts; i += GN_THREADS) acc += partial[i];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) acc += __shfl_xor(acc, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < GN_THREADS / 64; ++w) s += red[w];
    norm[0] = (float)sqrt(s);
  }
}

// Where the factor is 1, tensors that are their own result are not touched.
__global__ __launch_bounds__(GN_THREADS) void grad_clip_kernel(GradTable t, const float* __restrict__ norm, float max_norm) {
  const int tid = threadIdx.x;
  const double c = (double)max_norm / ((double)norm[0] + 1e-6);
  const float f = c >= 1.0 ? 1.0f : (float)c;  // (a norm of NaN gives NaN, one of infinity 0)
  for_chunks(t, [&](int i, int64_t at, int n) {
    const bool ib = bit(t.in_bf16, i), ob = bit(t.out_bf16, i);
    if (t.in[i] == t.out[i] && f == 1.0f) return;
    auto one = [&](int j) {
      const float x = ib ? bf2f(((const bf16_t*)t.in[i])[at + j]) : ((const float*)t.in[i])[at + j];
      if (ob) ((bf16_t*)t.out[i])[at + j] = (bf16_t)f2bf(x * f);
      else ((float*)t.out[i])[at + j] = x * f;
    };
    auto eights = [&](auto in_bf16, auto out_bf16) {
#pragma unroll 4
      for (int j = tid; j < n / 8; j += GN_THREADS) {
        f32x4 a, b;
        if constexpr (decltype(in_bf16)::value) {
          const u32x4 x = ((const u32x4*)((const bf16_t*)t.in[i] + at))[j];
          a = f32x4{bf_lo(x[0]), bf_hi(x[0]), bf_lo(x[1]), bf_hi(x[1])};
          b = f32x4{bf_lo(x[2]), bf_hi(x[2]), bf_lo(x[3]), bf_hi(x[3])};
        } else {
          const f32x4* p = (const f32x4*)((const float*)t.in[i] + at);
          a = p[2 * j];
          b = p[2 * j + 1];
        }
        a *= f;
        b *= f;
        if constexpr (decltype(out_bf16)::value) {
          ((u32x4*)((bf16_t*)t.out[i] + at))[j] =
              u32x4{pack_bf2(a[0], a[1]), pack_bf2(a[2], a[3]), pack_bf2(b[0], b[1]), pack_bf2(b[2], b[3])};
        } else {
          f32x4* p = (f32x4*)((float*)t.out[i] + at);
          p[2 * j] = a;
          p[2 * j + 1] = b;
        }
      }
    };
    if (ib && ob) eights(std::true_type{}, std::true_type{});
    else if (ib) eights(std::true_type{}, std::false_type{});
    else if (ob) eights(std::false_type{}, std::true_type{});
    else eights(std::false_type{}, std::false_type{});
    for (int j = (n & ~7) + tid; j < n; j += GN_THREADS) one(j);
  });
}

// The next tensors that a launch takes, from `from` on: as many as the table and 2^31 chunks hold.
int fill(GradTable& t, int n, int from, const GradTensor* in, const GradTensor* out) {
  t = GradTable{};
  int64_t chunks = 0;
  int i = from;
  for (; i < n && t.tensors < GN_TENSORS; ++i) {
    const int k = t.tensors;
    if (in[i].n == 0) continue;
    const int64_t more = (in[i].n + GN_CHUNK - 1) / GN_CHUNK;
    if (chunks + more >= (int64_t)1 << 31) break;
    t.in[k] = in[i].p;
    t.out[k] = out ? out[i].p : nullptr;
    t.n[k] = in[i].n;
    t.first[k] = (uint32_t)chunks;
    if (in[i].bf16) t.in_bf16[k / 32] |= 1u << (k % 32);
    if (out && out[i].bf16) t.out_bf16[k / 32] |= 1u << (k % 32);
    chunks += more;
    t.first[++t.tensors] = (uint32_t)chunks;
  }
  return i;
}

}  // namespace

size_t grad_norm_workspace() { return GN_BLOCKS * sizeof(double); }

hipError_t grad_norm(int n, const GradTensor* g, float* norm, void* ws, hipStream_t s) {
  double* partial = (double*)ws;
  GradTable t;
  unsigned grid = 1;  // the first launch's, which writes the partial sums of all
  for (int i = 0; i < n || i == 0;) {
    const bool first = i == 0;
    int64_t all = 0;
    if (first) {
      for (int k = 0; k < n; ++k) all += (g[k].n + GN_CHUNK - 1) / GN_CHUNK;
      grid = (unsigned)std::max<int64_t>(std::min<int64_t>(all, GN_BLOCKS), 1);
    }
    i = fill(t, n, i, g, nullptr);
    hipLaunchKernelGGL(grad_sumsq_kernel, dim3(grid), dim3(GN_THREADS), 0, s, t, partial, first ? 0 : 1);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (i >= n) break;
  }
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(GN_THREADS), 0, s, (int)grid, (const double*)partial, norm);
  return hipGetLastError();
}

hipError_t grad_clip(int n, const GradTensor* g, const float* norm, float max_norm, const GradTensor* out, hipStream_t s) {
  GradTable t;
  for (int i = 0; i < n;) {
    i = fill(t, n, i, g, out);
    if (t.tensors == 0) continue;
    const unsigned grid = std::min<uint32_t>(t.first[t.tensors], GN_BLOCKS);
    hipLaunchKernelGGL(grad_clip_kernel, dim3(grid), dim3(GN_THREADS), 0, s, t, norm, max_norm);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ls

// Packed sequences: the plan that the packed operators share, and rotary
// position embedding with positions that restart at every sequence.
#include <math.h>

#include "packed.h"

namespace ls {

namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_WAVES = PLAN_THREADS / 64;
constexpr int LEVELS = 4 * PLAN_THREADS;  // classes of work that the list of tiles is ordered by
constexpr int FEW = 4;                    // tiles of a sequence that one thread enters by itself

// Inclusive prefix sum over the workgroup's threads.
LS_DEV int block_scan(int v, int* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  if (lane == 63) part[wave] = v;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before += part[w];
  __syncthreads();
  return v + before;
}

// Rows of sequence s, 0 for an empty one or one that does not lie inside the total.
LS_DEV int seq_len(const int32_t* cu, int s, int total, int& start) {
  const int a = cu[s], b = cu[s + 1];
  start = a;
  return a >= 0 && b > a && b <= total ? b - a : 0;
}

// Workgroup 0 lists the tiles and the short sequences, the others find the rows'
// positions.
//
// The list of tiles is a counting sort by rank (a tile's work), the highest first: ranks
// are counted with one range update per sequence in a difference array, whose
// prefix sum is the number of tiles per class of 2^shift ranks (the classes
// are single ranks up to 524288 rows).  Inside a class the order is that of
// the LDS atomics; it decides when a tile is computed, never what.
//
// Bound by latency: one pass over cu_seqlens, two scans, one more pass.
__global__ __launch_bounds__(PLAN_THREADS) void packed_plan_kernel(int total, int n, const int32_t* __restrict__ cu,
                                                                   PackedHead* __restrict__ head,
                                                                   PackedTile* __restrict__ tiles, int max_tiles,
                                                                   PackedTile* __restrict__ shorts, int max_shorts,
                                                                   int32_t* __restrict__ pos) {
  const int tid = threadIdx.x;
  if (blockIdx.x > 0) {
    const int row = ((int)blockIdx.x - 1) * PLAN_THREADS + tid;
    if (row >= total) return;
    // first entry of cu beyond the row (n + 1 entries): the sequence before it holds the row
    int lo = 0, hi = n + 1;
    while (lo < hi) {
      const int mid = lo + (hi - lo) / 2;
      if (cu[mid] > row) hi = mid;
      else lo = mid + 1;
    }
    const int start = lo >= 1 ? cu[lo - 1] : 0;
    pos[row] = lo >= 1 && lo <= n && start >= 0 && start <= row ? row - start : -1;
    return;
  }
  __shared__ int level[LEVELS + 1];
  __shared__ int part[PLAN_WAVES];
  __shared__ int nshort;
  const int max_rank = (total - 1) / PACKED_ROWS;
  int shift = 0;
  while (max_rank >> shift >= LEVELS) ++shift;
  for (int i = tid; i <= LEVELS; i += PLAN_THREADS) level[i] = 0;
  if (tid == 0) nshort = 0;
  __syncthreads();
  const int per = 1 << shift;
  for (int s = tid; s < n; s += PLAN_THREADS) {
    int start;
    const int len = seq_len(cu, s, total, start);
    if (len <= PACKED_SHORT) continue;
    // classes 0 .. top-1 get `per` ranks each, class `top` the rest
    const int m = (len - 1) / PACKED_ROWS + 1, top = (m - 1) >> shift, rest = m - (top << shift);
    atomicAdd(&level[0], per);
    atomicAdd(&level[top], rest - per);
    atomicAdd(&level[top + 1], -rest);
  }
  __syncthreads();
  // tiles per class, then the first slot of each class (the highest class first)
  int c[4], sum = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    sum += level[4 * tid + k];
    c[k] = sum;
  }
  int before = block_scan(sum, part) - sum, tiles_here = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    c[k] += before;
    tiles_here += c[k];
  }
  const int upto = block_scan(tiles_here, part);
  if (tid == PLAN_THREADS - 1) level[LEVELS] = upto;
  __syncthreads();
  const int all = level[LEVELS];
  int slot = all - upto + tiles_here;  // tiles of this thread's classes and all higher ones
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    slot -= c[k];
    level[4 * tid + k] = slot;
  }
  __syncthreads();
  auto enter = [&](int start, int len, int rank) {
    const int at = atomicAdd(&level[rank >> shift], 1);
    // (lengths that are out of order may give more tiles than the list has room for)
    if (at >= 0 && at < max_tiles) tiles[at] = PackedTile{start, len, rank, 0};
  };
  // a thread enters the first tiles of its sequence, the wave the rest of a long one
  for (int s0 = 0; s0 < n; s0 += PLAN_THREADS) {
    const int s = s0 + tid;
    int start = 0, len = 0;
    if (s < n) len = seq_len(cu, s, total, start);
    const unsigned long long few = __ballot(len > 0 && len <= PACKED_SHORT);
    if (few) {
      const int lane = tid & 63;
      int at = 0;
      if (lane == 0) at = atomicAdd(&nshort, __popcll(few));
      at = __shfl(at, 0) + __popcll(few & ((1ull << lane) - 1));
      if ((few >> lane & 1) && at < max_shorts) shorts[at] = PackedTile{start, len, 0, 0};
    }
    if (len <= PACKED_SHORT) len = 0;
    const int m = len > 0 ? (len - 1) / PACKED_ROWS + 1 : 0;
    for (int r = 0; r < m && r < FEW; ++r) enter(start, len, r);
    unsigned long long longer = __ballot(m > FEW);
    while (longer) {
      const int l = __builtin_ctzll(longer);
      longer &= longer - 1;
      const int wstart = __shfl(start, l), wlen = __shfl(len, l), wm = __shfl(m, l);
      for (int r = FEW + (tid & 63); r < wm; r += 64) enter(wstart, wlen, r);
    }
  }
  __syncthreads();
  if (tid == 0) *head = PackedHead{min(max(all, 0), max_tiles), min(nshort, max_shorts)};
}

// q and k of one row turned by its position: pairs (i, i + D/2) of every head,
// angle p theta^(-2i/D), backwards with inverse.  A wave takes a row; lane l
// works on 8 pairs (16 bytes of either half), pairs 8 (l % (D/16)) .. of the
// heads l / (D/16), + 64 / (D/16), ..., so that it needs 8 angles for all of them.
//
// Angles are formed in fp64, as turns whose whole part is dropped (in fp32 the
// fraction of a far position's angle would be lost), one per lane and row, and
// handed around by lane reads.  Rotation in fp32, one rounding to bf16.
//
// Bound by HBM bandwidth: each row is read and written once.
constexpr int ROPE_WAVES = 4;

template <int D>
__global__ __launch_bounds__(64 * ROPE_WAVES) void packed_rope_kernel(int total, int nq, int nkv, double log2_theta,
                                                                      int inverse, const int32_t* __restrict__ pos,
                                                                      const bf16_t* src, bf16_t* dst) {
  constexpr int HALF = D / 2, CH = HALF / 8, HPW = 64 / CH;  // 16-byte chunks per half; heads at a time
  const int lane = threadIdx.x & 63, c = lane % CH, h0 = lane / CH;
  const int turned = nq + nkv;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * D;
  // turns per position of pair lane % HALF
  const double turns = exp2(-(double)(lane % HALF) / HALF * log2_theta) * 0.15915494309189533577;
  for (int64_t row = (int64_t)blockIdx.x * ROPE_WAVES + (threadIdx.x >> 6); row < total;
       row += (int64_t)gridDim.x * ROPE_WAVES) {
    const int p = pos[row];
    if (p < 0 || p > row) continue;
    const double t = p * turns;
    float sn, cs;
    sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
    if (inverse) sn = -sn;
    float ce[8], se[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      ce[e] = __shfl(cs, 8 * c + e);
      se[e] = __shfl(sn, 8 * c + e);
    }
    const bf16_t* x = src + row * ld + 8 * c;
    bf16_t* y = dst + row * ld + 8 * c;
    for (int h = h0; h < turned; h += HPW) {
      const u32x4 a = *(const u32x4*)(x + h * D), b = *(const u32x4*)(x + h * D + HALF);
      u32x4 lo, hi;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a0 = bf_lo(a[e]), a1 = bf_hi(a[e]), b0 = bf_lo(b[e]), b1 = bf_hi(b[e]);
        lo[e] = pack_bf2(a0 * ce[2 * e] - b0 * se[2 * e], a1 * ce[2 * e + 1] - b1 * se[2 * e + 1]);
        hi[e] = pack_bf2(a0 * se[2 * e] + b0 * ce[2 * e], a1 * se[2 * e + 1] + b1 * ce[2 * e + 1]);
      }
      *(u32x4*)(y + h * D) = lo;
      *(u32x4*)(y + h * D + HALF) = hi;
    }
    if (src != dst) {  // out of place: v goes along
      const u32x4* v = (const u32x4*)(src + row * ld + (int64_t)turned * D);
      u32x4* w = (u32x4*)(dst + row * ld + (int64_t)turned * D);
      for (int i = lane; i < nkv * D / 8; i += 64) w[i] = v[i];
    }
  }
}

}  // namespace

size_t packed_plan_bytes(const PackedShape& p) { return packed_layout(p).total; }

hipError_t packed_plan(const PackedShape& p, const int32_t* cu, void* plan, hipStream_t s) {
  const unsigned grid = 1 + (unsigned)((p.total + PLAN_THREADS - 1) / PLAN_THREADS);
  const PackedLayout l = packed_layout(p);
  char* b = (char*)plan;
  hipLaunchKernelGGL(packed_plan_kernel, dim3(grid), dim3(PLAN_THREADS), 0, s, (int)p.total, p.n_seqs, cu,
                     (PackedHead*)b, (PackedTile*)(b + l.tiles), (int)l.max_tiles, (PackedTile*)(b + l.shorts),
                     (int)l.max_shorts, (int32_t*)(b + l.pos));
  return hipGetLastError();
}

hipError_t packed_rope(const PackedShape& p, const void* plan, double theta, int inverse, const bf16_t* src,
                       bf16_t* dst, hipStream_t s) {
  const int64_t need = (p.total + ROPE_WAVES - 1) / ROPE_WAVES;
  const dim3 grid((unsigned)(need < 8192 ? need : 8192)), block(64 * ROPE_WAVES);
  const int32_t* pos = packed_view(p, plan).pos;
  if (p.d == 128)
    hipLaunchKernelGGL((packed_rope_kernel<128>), grid, block, 0, s, (int)p.total, p.nq, p.nkv, log2(theta), inverse,
                       pos, src, dst);
  else if (p.d == 64)
    hipLaunchKernelGGL((packed_rope_kernel<64>), grid, block, 0, s, (int)p.total, p.nq, p.nkv, log2(theta), inverse,
                       pos, src, dst);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace ls

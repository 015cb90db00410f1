// Packed sequences: the plan that the packed operators share, and rotary
// position embedding with positions that restart at every sequence.
#include <math.h>

#include "packed.h"

namespace ls {

namespace {

constexpr int PLAN_THREADS = 512;
constexpr int PLAN_WAVES = PLAN_THREADS / 64;
constexpr int LEVELS = 4 * PLAN_THREADS;  // classes of work that the list of tiles is ordered by

// Inclusive prefix sums of N values over the workgroup's threads, and their totals.
// (`part` may be used again after a barrier.)
template <int N>
LS_DEV void block_scan(int (&v)[N], int (&all)[N], int (*part)[PLAN_WAVES]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int u = __shfl_up(v[k], o);
      if (lane >= o) v[k] += u;
    }
  if (lane == 63) {
#pragma unroll
    for (int k = 0; k < N; ++k) part[k][wave] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    all[k] = 0;
    int before = 0;
#pragma unroll
    for (int w = 0; w < PLAN_WAVES; ++w) {
      const int p = part[k][w];
      before += w < wave ? p : 0;
      all[k] += p;
    }
    v[k] += before;
  }
}

// Rows of sequence s, 0 for an empty one or one that does not lie inside the total.
LS_DEV int seq_len(const int32_t* cu, int s, int total, int& start) {
  const int a = cu[s], b = cu[s + 1];
  start = a;
  return a >= 0 && b > a && b <= total ? b - a : 0;
}

// Sums of two values over the workgroup (every thread gets them).
LS_DEV void block_sums(long long (&v)[2], long long (*part)[PLAN_WAVES]) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    v[0] += __shfl_xor(v[0], o);
    v[1] += __shfl_xor(v[1], o);
  }
  if ((threadIdx.x & 63) == 0) {
    part[0][threadIdx.x >> 6] = v[0];
    part[1][threadIdx.x >> 6] = v[1];
  }
  __syncthreads();
  v[0] = v[1] = 0;
#pragma unroll
  for (int w = 0; w < PLAN_WAVES; ++w) {
    v[0] += part[0][w];
    v[1] += part[1][w];
  }
}

// Workgroup 0 lists the tiles, the middle and short sequences and the pieces of
// dK/dV work, the others find the rows' positions.
//
// The list of tiles is a counting sort by rank (a tile's work), the highest first:
// ranks are counted with one range update per sequence in a difference array,
// whose prefix sum is the number of tiles per class of 2^shift ranks (the
// classes are single ranks up to 262144 rows).  Inside a class the order is that
// of the LDS atomics; it decides when a tile is computed, never what.  Tiles of a
// class are cut into the same number of parts, so that a tile's place among the
// pieces and its slots follow from its place in its class.
//
// Middle and short sequences are computed by a wave or two for all heads of a group, which
// takes long where the group is large; a few of them, too few to fill the card, are
// listed as tiles instead, whose heads are shared out by twos (the backward's main kernel
// on one sequence of 64 rows, heads of 128: 8/2 heads 29 us by one pair of waves, 19
// by two; 32/2: 103, 20; on one of 32 rows 15, 10 and 46, 11).
//
// Lengths that are out of order and add up to more than the total make a plan
// without sequences: the lists have no room for them, and entering them could take
// as many steps as there are sequences times tiles.
//
// Bound by latency, 5 to 8 us: one pass over cu_seqlens, two scans and a sum, one
// more pass.
__global__ __launch_bounds__(PLAN_THREADS) void packed_plan_kernel(int total, int n, int nkv, int group,
                                                                   const int32_t* __restrict__ cu, char* plan,
                                                                   PackedLayout lay) {
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
    ((int32_t*)(plan + lay.pos))[row] = lo >= 1 && lo <= n && start >= 0 && start <= row ? row - start : -1;
    return;
  }
  PackedTile* tiles = (PackedTile*)(plan + lay.tiles);
  PackedTile* mids = (PackedTile*)(plan + lay.mids);
  PackedTile* shorts = (PackedTile*)(plan + lay.shorts);
  PackedItem* items = (PackedItem*)(plan + lay.items);
  // per class: counts of ranks, then tiles entered so far; first tile; first piece; first slot
  __shared__ int level[LEVELS + 1], first[LEVELS], piece[LEVELS], slot[LEVELS];
  __shared__ int part[1][PLAN_WAVES], part3[3][PLAN_WAVES];
  __shared__ long long part64[2][PLAN_WAVES];
  __shared__ int counts[2][PLAN_WAVES];  // of a wave: tiles, middle and short sequences
  __shared__ int nmid, nshort, nsplit;
  const int max_rank = (total - 1) / PACKED_ROWS;
  int shift = 0;
  while (max_rank >> shift >= LEVELS) ++shift;
  for (int i = tid; i <= LEVELS; i += PLAN_THREADS) level[i] = 0;
  if (tid == 0) nmid = nshort = nsplit = 0;
  __syncthreads();
  const int per = 1 << shift;
  long long rows = 0;
  // (the latter of the whole wave, in its first lane, which is in every turn)
  int tiles_here = 0, few_here = 0;
  for (int s = tid; s < n; s += PLAN_THREADS) {
    int start;
    const int len = seq_len(cu, s, total, start);
    rows += len;
    few_here += __popcll(__ballot(len > 0 && len <= PACKED_MID));
    if (len <= PACKED_MID) continue;
    // classes 0 .. top-1 get `per` ranks each, class `top` the rest
    const int m = (len - 1) / PACKED_ROWS + 1, top = (m - 1) >> shift, rest = m - (top << shift);
    tiles_here += m;
    atomicAdd(&level[0], per);
    atomicAdd(&level[top], rest - per);
    atomicAdd(&level[top + 1], -rest);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) tiles_here += __shfl_xor(tiles_here, o);
  if ((tid & 63) == 0) {
    counts[0][tid >> 6] = tiles_here;
    counts[1][tid >> 6] = few_here;
  }
  __syncthreads();
  constexpr int PT = LEVELS / PLAN_THREADS;  // classes per thread
  int c[PT], sum[1] = {0}, unused[1];
#pragma unroll
  for (int k = 0; k < PT; ++k) {
    sum[0] += level[PT * tid + k];
    c[k] = sum[0];
  }
  const int mine = sum[0];
  block_scan(sum, unused, part);
  const int before = sum[0] - mine;
  // work of a class's last rank, in units of 128 queries of one head
  auto units = [&](int l) { return ((long long)(l + 1) << shift) * group; };
  long long sums[2] = {0, rows};
#pragma unroll
  for (int k = 0; k < PT; ++k) {
    c[k] += before;
    sums[0] += c[k] * units(PT * tid + k);
  }
  block_sums(sums, part64);
  if (sums[1] > total) {
    if (tid == 0) *(PackedHead*)plan = PackedHead{0, 0, 0, 0, 0};
    return;
  }
  int tiles_all = 0, few = 0;
#pragma unroll
  for (int w = 0; w < PLAN_WAVES; ++w) {
    tiles_all += counts[0][w];
    few += counts[1][w];
  }
  const bool as_tiles = group > PACKED_PART && few <= packed_few(nkv) && tiles_all + few <= lay.max_tiles;
  if (as_tiles) {
    if (tid == 0) c[0] += few;
    sums[0] += few * units(0);
  }
  // A part's work at most (PACKED_PART or more): half of a compute unit's share of the tiles' work in whole units of
  // the group (parts of fractions were slower by up to a quarter where there are enough of whole ones), or, where
  // there is little work for so many heads, a 64th of it and of the small sequences' (8/2 heads of 128, longest
  // document 183 rows: backward 32 -> 24 us; without the small sequences in it, 60 short documents: 40 -> 43).
  // In 32 bits, clamped: the plan's time is that of one thread's instructions.
  auto clamped = [](long long v) { return (unsigned)min(v, 1ll << 30); };
  auto share = [&](long long work, int n) { return max(clamped((work * nkv + n - 1) / n), (unsigned)PACKED_PART); };
  const unsigned half = (share(sums[0], 2 * PACKED_CUS) + (unsigned)group - 1) / (unsigned)group * (unsigned)group;
  const unsigned target = min(half, share(sums[0] + (as_tiles ? 0ll : (long long)few * group), 64));
  auto parts_of = [&](int l) { return (int)min((clamped(units(l)) + target - 1) / target, 1023u); };
  // the first tile, piece and slot of each class, the highest class first
  int own[3] = {0, 0, 0}, all[3];  // tiles, pieces, slots
#pragma unroll
  for (int k = 0; k < PT; ++k) {
    if (c[k] == 0) continue;
    const int p = parts_of(PT * tid + k);
    own[0] += c[k];
    own[1] += c[k] * p;
    own[2] += p > 1 ? c[k] * p : 0;
    if (p > 1) atomicAdd(&nsplit, c[k]);
  }
  int upto_here[3] = {own[0], own[1], own[2]};
  block_scan(upto_here, all, part3);
  int at_t = all[0] - upto_here[0] + own[0], at_p = all[1] - upto_here[1] + own[1],
      at_s = all[2] - upto_here[2] + own[2];
#pragma unroll
  for (int k = 0; k < PT; ++k) {
    const int l = PT * tid + k;
    level[l] = 0;
    if (c[k] == 0) continue;
    const int p = parts_of(l);
    first[l] = at_t -= c[k];
    piece[l] = at_p -= c[k] * p;
    slot[l] = at_s -= p > 1 ? c[k] * p : 0;
  }
  __syncthreads();
  auto enter = [&](int start, int len, int rank) {
    const int l = rank >> shift, p = parts_of(l);
    const int i = atomicAdd(&level[l], 1), at = first[l] + i, q = piece[l] + i * p;
    if (at < 0 || at >= lay.max_tiles || q < 0 || q + p > lay.max_items) return;  // (never)
    // a class of many ranks may cut its lowest into more parts than they have steps: their last pieces are empty
    const int first_key = ((len - 1) / PACKED_ROWS - rank) * PACKED_ROWS;
    const int mine = (int)min((long long)p, (long long)group * ((len - first_key + PACKED_STEP - 1) / PACKED_STEP));
    PackedTile t{start, len, rank, 1, 0};
    t.parts = (unsigned)mine;
    t.slot = p > 1 ? (unsigned)(slot[l] + i * p) : 0u;
    tiles[at] = t;
    for (int j = 0; j < p; ++j) items[q + j] = j < mine ? PackedItem{t, j, {0, 0, 0}} : PackedItem{};
  };
  // a wave takes 64 sequences at a time and enters 64 of their tiles at a time
  for (int s0 = 0; s0 < n; s0 += PLAN_THREADS) {
    const int s = s0 + tid;
    int start = 0, len = 0;
    if (s < n) len = seq_len(cu, s, total, start);
    auto enter_small = [&](bool in, int* count, PackedTile* list, int64_t room) {
      const unsigned long long few = __ballot(in);
      if (!few) return;
      const int lane = tid & 63;
      int at = 0;
      if (lane == 0) at = atomicAdd(count, __popcll(few));
      at = __shfl(at, 0) + __popcll(few & ((1ull << lane) - 1));
      if (in && at < room) list[at] = PackedTile{start, len, 0, 1, 0};
    };
    if (!as_tiles) {
      enter_small(len > PACKED_SHORT && len <= PACKED_MID, &nmid, mids, lay.max_mids);
      enter_small(len > 0 && len <= PACKED_SHORT, &nshort, shorts, lay.max_shorts);
      if (len <= PACKED_MID) len = 0;
    }
    const int m = len > 0 ? (len - 1) / PACKED_ROWS + 1 : 0;
    int upto = m;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(upto, o);
      if ((tid & 63) >= o) upto += u;
    }
    const int in_wave = __shfl(upto, 63);
    for (int f = tid & 63; f - (tid & 63) < in_wave; f += 64) {
      int l = 0;  // sequences of the wave whose tiles all come before the f-th
#pragma unroll
      for (int b = 32; b >= 1; b >>= 1)
        if (__shfl(upto, l + b - 1) <= f) l += b;
      const int lstart = __shfl(start, l), llen = __shfl(len, l), first_f = __shfl(upto - m, l);
      if (f < in_wave) enter(lstart, llen, f - first_f);
    }
  }
  __syncthreads();
  if (tid == 0) {
    auto upto = [](int v, int64_t most) { return (int)(v < 0 ? 0 : v > most ? most : v); };
    *(PackedHead*)plan = PackedHead{upto(all[0], lay.max_tiles), upto(nmid, lay.max_mids), upto(nshort, lay.max_shorts),
                                    upto(all[1], lay.max_items), upto(nsplit, lay.max_tiles)};
  }
}

// q and k of one row turned by its position: pairs (i, i + d/2) of every head,
// angle p theta^(-2i/d), backwards with inverse.  A wave takes a row; lane l
// works on V pairs (V consecutive features of either half), pairs V c .. of the
// heads h0, h0 + hpw, ... with c = l % CH, h0 = l / CH and CH = d / (2V) pieces of a
// half, so that it needs V angles for all of them.  V = 8 (16-byte loads) where a
// half is a multiple of 8, else 4.
//
// Angles are formed in fp64, as turns whose whole part is dropped (in fp32 the
// fraction of a far position's angle would be lost), one per lane and row, and
// handed around by lane reads.  Rotation in fp32, one rounding to bf16.
//
// Bound by HBM bandwidth: each row is read and written once.  8135 rows of 24 + 2 x 8
// heads of 128: 27 us, 6.2 TB/s of 167 MB that the last-level cache holds in part.
constexpr int ROPE_WAVES = 4;

template <int V>
__global__ __launch_bounds__(64 * ROPE_WAVES) void packed_rope_kernel(int total, int nq, int nkv, int d,
                                                                      double log2_theta, int inverse,
                                                                      const int32_t* __restrict__ pos,
                                                                      const bf16_t* src, bf16_t* dst) {
  typedef uint32_t words __attribute__((ext_vector_type(V / 2)));
  const int lane = threadIdx.x & 63, half = d / 2, ch = half / V, hpw = 64 / ch, c = lane % ch, h0 = lane / ch;
  const int turned = nq + nkv;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * d;
  // turns per position of pair `lane` (lanes past the last pair: of a pair again)
  const double turns = exp2(-(double)(lane % half) / half * log2_theta) * 0.15915494309189533577;
  for (int64_t row = (int64_t)blockIdx.x * ROPE_WAVES + (threadIdx.x >> 6); row < total;
       row += (int64_t)gridDim.x * ROPE_WAVES) {
    const int p = pos[row];
    if (p < 0 || p > row) continue;
    const double t = p * turns;
    float sn, cs;
    sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
    if (inverse) sn = -sn;
    float ce[V], se[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      ce[e] = __shfl(cs, V * c + e);
      se[e] = __shfl(sn, V * c + e);
    }
    const bf16_t* x = src + row * ld + V * c;
    bf16_t* y = dst + row * ld + V * c;
    if (h0 < hpw) {
      for (int h = h0; h < turned; h += hpw) {
        const words a = *(const words*)(x + h * d), b = *(const words*)(x + h * d + half);
        words lo, hi;
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
          const float a0 = bf_lo(a[e]), a1 = bf_hi(a[e]), b0 = bf_lo(b[e]), b1 = bf_hi(b[e]);
          lo[e] = pack_bf2(a0 * ce[2 * e] - b0 * se[2 * e], a1 * ce[2 * e + 1] - b1 * se[2 * e + 1]);
          hi[e] = pack_bf2(a0 * se[2 * e] + b0 * ce[2 * e], a1 * se[2 * e + 1] + b1 * ce[2 * e + 1]);
        }
        *(words*)(y + h * d) = lo;
        *(words*)(y + h * d + half) = hi;
      }
    }
    if (src != dst) {  // out of place: v goes along
      const u32x4* v = (const u32x4*)(src + row * ld + (int64_t)turned * d);
      u32x4* w = (u32x4*)(dst + row * ld + (int64_t)turned * d);
      for (int i = lane; i < nkv * d / 8; i += 64) w[i] = v[i];
    }
  }
}

}  // namespace

size_t packed_plan_bytes(const PackedShape& p) { return packed_layout(p).total; }

hipError_t packed_plan(const PackedShape& p, const int32_t* cu, void* plan, hipStream_t s) {
  const unsigned grid = 1 + (unsigned)((p.total + PLAN_THREADS - 1) / PLAN_THREADS);
  hipLaunchKernelGGL(packed_plan_kernel, dim3(grid), dim3(PLAN_THREADS), 0, s, (int)p.total, p.n_seqs, p.nkv,
                     p.nq / p.nkv, cu, (char*)plan, packed_layout(p));
  return hipGetLastError();
}

hipError_t packed_rope(const PackedShape& p, const void* plan, double theta, int inverse, const bf16_t* src,
                       bf16_t* dst, hipStream_t s) {
  const int64_t need = (p.total + ROPE_WAVES - 1) / ROPE_WAVES;
  const dim3 grid((unsigned)(need < 8192 ? need : 8192)), block(64 * ROPE_WAVES);
  const int32_t* pos = packed_pos(p, plan);
  if (p.d % 16 == 0)
    hipLaunchKernelGGL((packed_rope_kernel<8>), grid, block, 0, s, (int)p.total, p.nq, p.nkv, p.d, log2(theta), inverse,
                       pos, src, dst);
  else
    hipLaunchKernelGGL((packed_rope_kernel<4>), grid, block, 0, s, (int)p.total, p.nq, p.nkv, p.d, log2(theta), inverse,
                       pos, src, dst);
  return hipGetLastError();
}

}  // namespace ls

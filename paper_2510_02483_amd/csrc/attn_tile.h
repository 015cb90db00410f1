// Causal grouped-query attention on gfx950 matrix cores: forward with an
// online softmax over key tiles (log-sum-exp saved), backward that recomputes
// the probabilities from the log-sum-exp.
//
// Layouts: qkv is [batch*seq, (nq + 2*nkv)*d] bf16 (q heads, then k heads, then
// v heads of one token in one row), o and dout are [batch*seq, nq*d], lse and
// D are [batch, nq, seq] fp32.  Query head h reads kv head h / (nq/nkv).
//
// Every streamed operand (K and V tiles in the forward and dQ kernels, Q and
// dO tiles in the dK/dV kernel) goes from global memory to LDS with buffer
// loads that write LDS directly, double-buffered: the loads of tile t+1 are in
// flight while the matrix cores work on tile t, with one barrier per tile.
// Tiles stay row-major in LDS ([row][d], 16-byte chunks XOR-swizzled by the
// row).  An operand is read either along d (a 16-byte read per lane: keys or
// queries as MFMA rows) or transposed (two ds_read_b64_tr_b16 per lane: d as
// MFMA rows, 4 consecutive keys/queries per read), and the swizzle keeps both
// kinds of read free of bank conflicts.
//
// The probabilities of a 32x32 MFMA block sit in registers with a lane owning
// one query (forward, dQ) or one key (dK/dV) and holding, for each 16-row
// k-step, the rows 4lh+{0..3} and 8+4lh+{0..3} (lh = lane/32).  Used as the B
// operand of the next product they define a permuted k order, and the
// transposed reads of the A operand fetch their rows in that same order.
//
// Forward (one workgroup = 128 queries of one head, 4 waves x 32): S^T = K Q^T
// per 64-key tile with Q in registers, base-2 online softmax with 1/sqrt(d)
// folded into one multiplier, O^T += V^T P^T.
// Backward, two kernels and no atomics.  dK/dV (one workgroup = 128 keys of
// one kv head, 4 waves x 32 keys, K and V in registers) loops over the query
// heads of its group and over 64-query tiles from the diagonal on: S = Q K^T,
// dP = dO V^T, P and dS = P (dP - D) in registers, dV^T += dO^T P and
// dK^T += Q^T dS (the sum over the group's heads happens in the same
// registers).  dQ (one workgroup = 128 queries of one head) loops over key
// tiles like the forward: S^T, dP^T, dQ^T += K^T dS^T.  Both write their
// gradient already scaled and un-rotated (inverse RoPE) in bf16.
//
// Workgroups are numbered so that the longest (most causal tiles) start
// first, which balances the triangular work over the compute units.
//
// Packed sequences (template argument PACKED; packed.h) run the same kernels: a
// workgroup takes its tile from the plan's list, longest first, instead of from
// batch and seq, and everything it loads ends at its sequence.  What differs:
//  - sequences of up to 64 rows have code of their own (short_fwd, short_bwd,
//    mid_bwd), a wave or two per sequence and head instead of a tile of 128 rows;
//  - the dK/dV work of long key tiles is cut into parts, whose fp32 sums the dQ
//    launch adds (join_parts): lengths vary, and one sequence's first key tile may have
//    more queries than a compute unit's share of everything (8135 rows of which
//    4272 in one document, 24/8 heads of 128: dK/dV 413 -> 355 us);
//  - heads between 64 and 128 features are read as they lie, zeros past their width.
// Per query and key pair they are as fast as on equal lengths: 8135 rows in 12
// documents, 24/8 heads of 128, forward 156-164 us (780-815 TFLOP/s), backward 505-545 us by card.
// Heads of 72 to 120 run the products of 128: of 72, 0.78 of its time forward and 0.86 backward.
#pragma once
#include <math.h>

#include "packed.h"

namespace ls {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

constexpr int BQ = 128;       // queries per workgroup (forward, dQ)
constexpr int BKV = 64;       // keys per tile (forward, dQ)
constexpr int BWD_BKV = 128;  // keys per workgroup (dK/dV)
constexpr int BWD_BQ = 64;    // queries per tile (dK/dV)
constexpr int DKDV_STAGES = 3;  // their stages in LDS
static_assert(BQ == PACKED_ROWS && BWD_BKV == PACKED_ROWS && BWD_BQ == PACKED_STEP, "one plan of packed sequences for all kernels");

LS_DEV u32x4 load16(const bf16_t* p) { return *(const u32x4*)p; }
LS_DEV u32x4 pack_frag(const f32x16& v, int r0) {
  return u32x4{pack_bf2(v[r0], v[r0 + 1]), pack_bf2(v[r0 + 2], v[r0 + 3]), pack_bf2(v[r0 + 4], v[r0 + 5]),
               pack_bf2(v[r0 + 6], v[r0 + 7])};
}
LS_DEV float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
// s plus the two bf16 values of a word.
LS_DEV float add_bf2(uint32_t w, float s) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3f803f80u), s, false);
}

// What a score is, in the base-2 exponent of the softmax, and which keys a query sees.
// PlainScore: q.k times a scale, every key up to the query.
// ModScore: within the window, key > query - window, and (CAPPED) cap tanh(scale q.k / cap):
// with r = 1 / (1 + exp(2 scale q.k / cap)), tanh is 1 - 2r and its slope 4 r (1 - r), so
// that two transcendental instructions give both, without branches, for any argument (r = 0 and 1
// at its ends).  r carries 1.9 x 2^-23 from the instructions (exp2 and reciprocal good to
// 2^-23, the sum to 2^-24), the score 2 cap times that; the factor 4 of the slope goes into the
// scale of dq and dk.
// P, and in the backward pass dS, go into their products as bf16, which the matrix cores multiply sixteen times as fast as
// fp32: one rounding of each entry, while scores, softmax and sums are of 32 bits.  Of dqkv's norm 0.0024 are off in all
// (scores of a standard deviation of 4; 0.0017 is the rounding of dqkv itself).
struct PlainScore {
  static constexpr bool ON = false, CAPPED = false;
  static constexpr int window = 0;  // (unused, as c2)
  static constexpr float c2 = 0.f;
};
template <bool CAP>
struct ModScore {
  static constexpr bool ON = true, CAPPED = CAP;
  int window;  // positions that a query sees, itself included
  float in;    // capped: 2 log2(e) scale / cap, what q.k is multiplied with
  float c2;    // capped: cap log2(e), the largest score in base 2
  bf16_t* rest;  // null, or what the rounding of o left (written by the forward pass, read by the backward pass)
  // r of a raw score, and the base-2 score c2 tanh = c2 - 2 c2 r less `m`
  LS_DEV float half(float x) const { return __builtin_amdgcn_rcpf(1.0f + ex2(x * in)); }
  LS_DEV float less(float r, float m) const { return fmaf(r, -2.0f * c2, c2 - m); }
};
// Key `key` is seen by query `q` (positions in one sequence).
template <class SC>
LS_DEV bool hidden_key(const SC& sc, int key, int q) {
  if constexpr (SC::ON) return key > q || key <= q - sc.window;
  else return key > q;
}

// Row-major LDS tile [rows][D]: 16-byte chunk c of row r sits at slot
// c ^ tile_swz(r).  The LDS serves 16 lanes of a 16-byte read and 32 lanes of
// an 8-byte read per clock over 64 banks (a 256-byte window):
//  - a 16-byte read along d covers 16 consecutive rows at one chunk: the swizzle
//    is a bijection of r % 16 (D = 128, one row per window) or of (r/2) % 8 for
//    each parity of r (D = 64, two rows per window);
//  - a transposing read covers 4 consecutive rows (4-aligned) x 4 consecutive
//    chunks (4-aligned): the swizzle moves the rows' chunk groups apart
//    (bits 2..3 of the slot for D = 128, bit 2 plus the window half for D = 64)
//    while its low two bits only depend on r / 4.
template <int D>
LS_DEV int tile_swz(int r) {
  if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

// Loads of tiles: rows row0 .. row0+ROWS-1, columns col0 .. col0+D-1 of a
// row-major bf16 matrix (leading dimension ld elements, `rows` rows) into an
// LDS tile in the swizzled layout above; rows at or past `rows` read as zero.
// Each load fills 1 KB of the tile (64/(D/8) rows); wave w fills the
// consecutive blocks w*PER .. w*PER+PER-1 with one M0 write.  The per-lane
// byte offsets of the wave's share are computed once, for every tile of a
// loop; a tile only moves the scalar resource, whose base is the tile's first
// element and whose end is row `rows` (the tile's columns lie within a row:
// col0 + width <= ld).  Columns at or past `width`, a multiple of 8, read as zero.
template <int D, int ROWS>
struct TileLoader {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, PER = ROWS / RPI / 4;
  static_assert(PER == 2 || PER == 4, "loads split evenly over 4 waves in groups of 2 or 4");
  uint32_t off[PER];
  LS_DEV TileLoader(int64_t ld, int wave, int lane, int width = D) {
#pragma unroll
    for (int jj = 0; jj < PER; ++jj) {
      const int rr = (wave * PER + jj) * RPI + lane / CPR;
      const int c = (lane % CPR) ^ tile_swz<D>(rr);
      off[jj] = 8 * c < width ? ((uint32_t)rr * (uint32_t)ld + (uint32_t)(8 * c)) * 2u : LS_OOB;
    }
  }
  LS_DEV void operator()(const bf16_t* m, int64_t ld, int row0, int rows, int col0, bf16_t* t, int wave) const {
    const i32x4 r = rsrc(m + (int64_t)row0 * ld + col0, clamp_bytes((int64_t)(rows - row0) * ld * 2 - (int64_t)col0 * 2));
    DmaLoad l[PER];
#pragma unroll
    for (int jj = 0; jj < PER; ++jj) l[jj] = DmaLoad{r, off[jj]};
    dma16_group<PER>(l, t + wave * PER * 512);
  }
};

// 64 floats v[i0 .. i0+63] of a buffer of `n` floats (resource r; entries at or
// past n read as zero) into t[0..63]; t must hold 256 floats (lanes 16..63 of
// the instruction write zeros to t[64..255]).
LS_DEV void load_vec64(i32x4 r, int i0, int n, float* t, int lane) {
  const int i = i0 + 4 * lane;
  dma16(r, (lane < 16 && i < n) ? (uint32_t)(i * 4) : LS_OOB, t);
}

// MFMA operand from a tile, read along d: lane gets row `row`, d = 16s + 8lh .. +7.
template <int D>
LS_DEV u32x4 row_frag(const bf16_t* t, int row, int s, int lh) {
  return *(const u32x4*)(t + row * D + 8 * ((2 * s + lh) ^ tile_swz<D>(row)));
}

// MFMA A operand of the transposed tile: lane gets column (d) c32 + lane%32 and
// the 8 rows 16s + 4lh + {0..3} and 16s + 8 + 4lh + {0..3} (the permuted k
// order of probabilities held in registers), via two transposing reads.
template <int D>
LS_DEV u32x4 colt_frag(const bf16_t* t, int c32, int s, int lane) {
  const int g = lane >> 4, q = lane & 15;
  const int col = c32 + 16 * (g & 1) + 4 * (q & 3);
  u32x4 out;
#pragma unroll
  for (int hh = 0; hh < 2; ++hh) {
    const int kk = 16 * s + 4 * (g >> 1) + 8 * hh + (q >> 2);
    const bf16_t* p = t + kk * D + 8 * ((col >> 3) ^ tile_swz<D>(kk)) + (col & 7);
    const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)p);
    const u32x2 w = __builtin_bit_cast(u32x2, v);
    out[2 * hh] = w[0];
    out[2 * hh + 1] = w[1];
  }
  return out;
}

// The same two kinds of operand reads by LDS byte address: this lane's
// addresses relative to a tile at `base` take only D/16 values for row reads
// (row lr, d step s; the 32-row block adds a constant) and 2·D/32 for
// transposing reads (d block i, row group hh; the 16-row step adds a
// constant), so they are computed once and held in registers the compiler
// cannot rematerialise.  With the other tiles in the same layout at constant
// distances (stages, arrays), every read is then one LDS instruction with an
// immediate offset.
template <int D>
struct FragAddr {
  uint32_t row[D / 16], col[D / 32][2];
  LS_DEV FragAddr(uint32_t base, int lane) {
    const int lr = lane & 31, lh = lane >> 5, g = lane >> 4, q = lane & 15;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      row[s] = base + 2u * (uint32_t)(lr * D + 8 * ((2 * s + lh) ^ tile_swz<D>(lr)));
      asm volatile("" : "+v"(row[s]));
    }
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int kk = 4 * (g >> 1) + 8 * hh + (q >> 2), c = 32 * i + 16 * (g & 1) + 4 * (q & 3);
        col[i][hh] = base + 2u * (uint32_t)(kk * D + 8 * ((c >> 3) ^ tile_swz<D>(kk)) + (c & 7));
        asm volatile("" : "+v"(col[i][hh]));
      }
  }
  // row_frag(tile at base + off, 32-row block, s, lh) for off = block * 32 * D * 2 + ...
  LS_DEV u32x4 rows(int s, uint32_t off) const { return *(const LDS_AS u32x4*)(size_t)(row[s] + off); }
  // colt_frag(tile at base + off, 32 i, step, lane) for off = step * 16 * D * 2 + ...
  LS_DEV u32x4 cols(int i, uint32_t off) const {
    u32x4 out;
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const u32x2 w = __builtin_bit_cast(
          u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(size_t)(col[i][hh] + off)));
      out[2 * hh] = w[0];
      out[2 * hh + 1] = w[1];
    }
    return out;
  }
};

// The first tile of 64 keys that a tile of queries from q0 on sees any of.
template <class SC>
LS_DEV int first_key_tile(const SC& sc, int q0) {
  if constexpr (SC::ON) return max(q0 - sc.window + 1, 0) / BKV;
  else return 0;
}

// Query-tile workgroups (forward, dQ): the 1-D grid runs the longest tiles
// (highest query index, most keys) first.
//
// A tile belongs to one sequence: S rows from row row0 of the token-major
// matrices, whose values of head h (log-sum-exp, D) start at vec0 of a vector
// with one entry per token of a head.  Equal sequences (batch x seq) follow
// from the workgroup's number, packed ones from the plan's list of tiles, which
// is in order of falling work too (packed.h); S = 0: no tile.
struct QTile {
  int qt, h, S;
  int64_t row0, vec0;
};
LS_DEV QTile q_tile(const AttnShape& sh) {
  const int nqt = (sh.seq + BQ - 1) / BQ, per = sh.nq * sh.batch;
  const int x = (int)blockIdx.x, h = (x % per) % sh.nq, b = (x % per) / sh.nq;
  return QTile{nqt - 1 - x / per, h, sh.seq, (int64_t)b * sh.seq, ((int64_t)b * sh.nq + h) * sh.seq};
}
LS_DEV QTile q_tile(const AttnShape& sh, const PackedTile& t, int h) {
  return QTile{t.rank, h, t.len, t.start, (int64_t)h * sh.seq + t.start};
}

// Online softmax with a lagging reference maximum: the running reference m
// moves only when some query's scores exceed it by more than 2^LAG (base 2), so
// that most tiles skip the rescale of O and l.  P = 2^(s - m) then lies in
// (0, 2^LAG]: bf16 keeps its relative precision at any such magnitude, and O,
// l in fp32 stay far from overflow.  The result, O = sum P V / sum P and the
// log-sum-exp m + log2 l, does not depend on the reference point.
constexpr float LAG = 8.0f;

// Query head of the y-th workgroup of a packed tile or unit: the kv heads one after the
// other, so that where their number allows, all readers of one kv head's keys and
// values run on the same XCD (workgroups go to the 8 XCDs in turn) and find them
// in its L2 (24/8 heads of 128, 8135 rows: forward 166 -> 164 us, training pass 710 -> 703).
LS_DEV int packed_head(int y, int nq, int nkv) { return y % nkv * (nq / nkv) + y / nkv; }

// A wave's own 32-row tile in LDS, from the rows that its lanes hold as MFMA
// operands (lane: row lr, d = 16s + 8lh .. +7), for transposing reads.
template <int D>
LS_DEV void put_rows(bf16_t* t, const u32x4 (&f)[D / 16], int lr, int lh) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s) *(u32x4*)(t + lr * D + 8 * ((2 * s + lh) ^ tile_swz<D>(lr))) = f[s];
}
// A sequence's rows as a buffer (rows past the sequence read as zero), and the
// operands of 32 of them: `off` is the byte offset of the lane's row and first
// feature; features at or past `width` read as zero.  Without branches, so that the
// loads of all operands are in flight together.
LS_DEV __amdgpu_buffer_rsrc_t seq_rows(const bf16_t* m, const PackedTile& t, int64_t ld) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)(m + t.start * ld), 0, (int)(t.len * ld * 2), 0x00020000);
}
template <int D>
LS_DEV void get_rows(u32x4 (&f)[D / 16], __amdgpu_buffer_rsrc_t r, uint32_t off, int lh, int width) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
    f[s] = __builtin_amdgcn_raw_buffer_load_b128(r, 16 * s + 8 * lh < width ? off + 32 * s + 16 * lh : LS_OOB, 0, 0);
}
// Orders a wave's own LDS writes before its later reads (the LDS serves a wave's accesses in order).
LS_DEV void wave_lds_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// What rounding a lane's row of o (columns 32i + 8(r/4) + 4lh + r%4, times inv) to bf16 leaves, in bf16: with it the
// backward pass has <dO, O> to 2^-17 of its terms instead of 2^-8.  Where the softmax is peaked that error, which all
// of a row's dS share, is larger than the rounding of dS itself (600 rows, scores of a standard deviation of 4: dqkv
// 0.0032 of its norm off without, 0.0024 with it).
template <int D, class SC>
LS_DEV void store_rest(const SC& sc, int64_t at, const f32x16 (&oacc)[D / 32], float inv, int hd, int lh) {
  if (!sc.rest) return;
  bf16_t* row = sc.rest + at;
  auto left = [](float x) { return x - bf2f(f2bf(x)); };
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      const int d = 32 * i + 8 * rq + 4 * lh;
      if (d >= hd) continue;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = left(oacc[i][4 * rq + e] * inv);
      *(u32x2*)(row + d) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
    }
}

// Forward of one head of a packed sequence of up to 32 NB rows by one wave: every
// operand straight from global memory, V through the wave's own LDS tile `vt` for
// its transpose.  A workgroup's four waves work on four sequences, without
// barriers, where a 128-row tile would leave most of them idle and wait
// for one sequence's loads at a time: 301 sequences of 27 rows on average (191 at
// most), 16 heads of 128: forward 50 us in tiles, 33 so.
template <int D, int NB, class SC>
LS_DEV void short_fwd(const AttnShape& sh, const SC& sc, const PackedTile& t, int h, const bf16_t* __restrict__ qkv,
                      bf16_t* __restrict__ o, float* __restrict__ lse, float sl2, bf16_t* vt) {
  const int nq = sh.nq, nkv = sh.nkv, kvh = h / (nq / nkv), hd = sh.d;
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * hd;
  const __amdgpu_buffer_rsrc_t rows = seq_rows(qkv, t, ld);
  auto at = [&](int b, int head) { return (uint32_t)((32 * b + lr) * (int)ld + head * hd) * 2u; };
  u32x4 qf[D / 16], kf[NB][D / 16];
  get_rows<D>(qf, rows, at(0, h), lh, hd);
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    u32x4 vf[D / 16];
    get_rows<D>(kf[b], rows, at(b, nq + kvh), lh, hd);
    get_rows<D>(vf, rows, at(b, nq + nkv + kvh), lh, hd);
    put_rows<D>(vt + 32 * b * D, vf, lr, lh);
  }
  wave_lds_order();
#pragma unroll
  for (int qb = 0; qb < NB; ++qb) {
    if (qb > 0) get_rows<D>(qf, rows, at(qb, h), lh, hd);
    f32x16 s[NB];
    float mx = -INFINITY;
    // lane holds query 32qb + lr, keys 32b + 8(r/4) + 4lh + r%4
#pragma unroll
    for (int b = 0; b <= qb; ++b) {
      s[b] = f32x16{};
#pragma unroll
      for (int c = 0; c < D / 16; ++c) s[b] = mfma32(kf[b][c], qf[c], s[b]);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int k = 8 * (r >> 2) + 4 * lh + (r & 3);
        if constexpr (SC::CAPPED) s[b][r] = sc.less(sc.half(s[b][r]), 0.f);
        if (SC::ON ? hidden_key(sc, 32 * b + k, 32 * qb + lr) : b == qb && k > lr) s[b][r] = -INFINITY;
        mx = fmaxf(mx, s[b][r]);
      }
    }
    if constexpr (SC::CAPPED) sl2 = 1.0f;  // (scores in base 2 already)
    const float m = halves_max(mx) * sl2;
    float sum = 0.f, sumb = 0.f;  // (ON: also of the probabilities as rounded, as in attn_fwd_kernel)
    f32x16 oacc[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) oacc[i] = f32x16{};
#pragma unroll
    for (int b = 0; b <= qb; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = ex2(fmaf(s[b][r], sl2, -m));
        sum += s[b][r];
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const u32x4 pf = pack_frag(s[b], 8 * c);
        if constexpr (SC::ON) {
#pragma unroll
          for (int w = 0; w < 4; ++w) sumb = add_bf2(pf[w], sumb);
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) oacc[i] = mfma32(colt_frag<D>(vt + 32 * b * D, 32 * i, c, lane), pf, oacc[i]);
      }
    }
    const float l = halves_sum(sum), lb = SC::ON ? halves_sum(sumb) : l;
    if (32 * qb + lr >= t.len) continue;
    const float inv = 1.0f / lb;
    const int64_t at_row = (t.start + (int64_t)(32 * qb + lr)) * nq * hd + h * hd;
    bf16_t* orow = o + at_row;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq)
        if (32 * i + 8 * rq + 4 * lh < hd)
          *(u32x2*)(orow + 32 * i + 8 * rq + 4 * lh) = u32x2{pack_bf2(oacc[i][4 * rq] * inv, oacc[i][4 * rq + 1] * inv),
                                                             pack_bf2(oacc[i][4 * rq + 2] * inv, oacc[i][4 * rq + 3] * inv)};
    if constexpr (SC::ON) store_rest<D>(sc, at_row, oacc, inv, hd, lh);
    if (lh == 0) lse[(int64_t)h * sh.seq + t.start + 32 * qb + lr] = (m + log2f(l)) * LN2;
  }
}

template <int D, bool PACKED, class SC>
__global__ __launch_bounds__(256, PACKED && D == 64 ? (SC::ON ? 3 : 4) : 2) void attn_fwd_kernel(
    AttnShape sh, PackedView pk, const bf16_t* __restrict__ qkv, bf16_t* __restrict__ o, float* __restrict__ lse,
    float sl2, SC sc) {
  __shared__ __attribute__((aligned(1024))) bf16_t Ks[2][BKV * D];
  __shared__ __attribute__((aligned(1024))) bf16_t Vs[2][BKV * D];
  // the scale in a register before the loop: a scalar load still in flight
  // at the loop entry makes the first LDS wait of every tile a full wait
  asm volatile("" : "+s"(sl2));

  const int nq = sh.nq, nkv = sh.nkv;
  QTile qtile;
  if constexpr (PACKED) {
    static_assert(sizeof(Ks) >= 2 * PACKED_MID * D * sizeof(bf16_t), "a tile of V per wave");
    PackedTile t;
    const int x = packed_wg(), head = packed_head(x % nq, nq, nkv);
    const bool whole = packed_unit(pk, x / nq, sh.seq, t);
    if (t.len == 0) return;
    if (!whole) {
      const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
      bf16_t* vt = (w < 2 ? &Ks[0][0] : &Vs[0][0]) + (w & 1) * PACKED_MID * D;
      if (t.len <= PACKED_SHORT) short_fwd<D, 1>(sh, sc, t, head, qkv, o, lse, sl2, vt);
      else short_fwd<D, 2>(sh, sc, t, head, qkv, o, lse, sl2, vt);
      return;
    }
    qtile = q_tile(sh, t, head);
  } else {
    qtile = q_tile(sh);
  }
  const int S = qtile.S, h = qtile.h, kvh = h / (nq / nkv), hd = PACKED ? sh.d : D;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * hd;
  const bf16_t* base = qkv + qtile.row0 * ld;
  const int tid = threadIdx.x, lane = tid & 63, wave = SC::ON ? __builtin_amdgcn_readfirstlane(tid >> 6) : tid >> 6;
  const int lr = lane & 31, lh = lane >> 5;
  const int q0 = qtile.qt * BQ;
  const int qrow = q0 + 32 * wave + lr;
  const int wave_qmin = q0 + 32 * wave, wave_qmax = wave_qmin + 31;
  const int kcol = (nq + kvh) * hd, vcol = (nq + nkv + kvh) * hd;

  const int kv_end = min(S, q0 + BQ);
  const int nkt = (kv_end + BKV - 1) / BKV;
  const int kt0 = first_key_tile(sc, q0);

  const TileLoader<D, BKV> tl(ld, wave, lane, hd);
  auto load_kv = [&](int kv0, bf16_t* kt, bf16_t* vt) {
    tl(base, ld, kv0, S, kcol, kt, wave);
    tl(base, ld, kv0, S, vcol, vt, wave);
  };
  load_kv(SC::ON ? kt0 * BKV : 0, Ks[0], Vs[0]);

  u32x4 qf[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
    qf[s] = qrow < S && 16 * s + 8 * lh < hd ? load16(base + (int64_t)qrow * ld + h * hd + 16 * s + 8 * lh)
                                             : u32x4{0u, 0u, 0u, 0u};

  f32x16 oacc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
  // (a window may leave a query no key of a tile: its maximum stays finite then)
  float m = SC::ON ? -3.402823466e38f : -INFINITY, l = 0.f;
  // ON: the sum of the probabilities as rounded for their product with V.  O over it, not over l, has a rounding
  // in common above and below, and a query whose weight lies on one key gets that key's values: o + rest was 0.0011 of its
  // norm off over l with scores of a standard deviation of 4.  The log-sum-exp stays that of the unrounded.
  float lb = 0.f;
  // Capped: in the tile's registers r = (1 - tanh) / 2 stands for the score, which falls with it: its least value is
  // the largest score's, a hidden key's is +inf, and one more fma makes it the exponent.
  constexpr float HIDDEN = SC::CAPPED ? INFINITY : -INFINITY;

  // operand reads by per-lane LDS address (K rows, V^T columns); the stage,
  // the array, the 32-key block and the 16-key step add constants
  const FragAddr<D> fa(lds_offset(&Ks[0][0]), lane);
  constexpr uint32_t STAGE = BKV * D * 2;
  const uint32_t v_minus_k = lds_offset(&Vs[0][0]) - lds_offset(&Ks[0][0]);

  sync_lds();
  // one 64-key tile in stage CUR (a constant: the loop below runs two per pass)
  auto step = [&](auto cur_c, int kt) {
    constexpr int cur = decltype(cur_c)::value;
    const int kv0 = kt * BKV;
    if (kt + 1 < nkt) load_kv(kv0 + BKV, Ks[cur ^ 1], Vs[cur ^ 1]);
    bool seen = kv0 <= wave_qmax;  // else every key of the tile is in this wave's future
    bool edge = kv0 + BKV - 1 > wave_qmin;
    if constexpr (SC::ON) {
      seen = seen && kv0 + BKV - 1 > wave_qmin - sc.window;
      edge = edge || kv0 <= wave_qmax - sc.window;
    }
    if (seen) {
      f32x16 sacc[BKV / 32];
#pragma unroll
      for (int bb = 0; bb < BKV / 32; ++bb)
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[bb][r] = 0.f;
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
#pragma unroll
        for (int bb = 0; bb < BKV / 32; ++bb)
          sacc[bb] = mfma32(fa.rows(s, cur * STAGE + bb * 32 * D * 2), qf[s], sacc[bb]);
      // lane holds query qrow, keys kv0 + 32bb + 8(r/4) + 4lh + r%4
      if constexpr (SC::CAPPED) {
#pragma unroll
        for (int bb = 0; bb < BKV / 32; ++bb)
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[bb][r] = sc.half(sacc[bb][r]);
      }
      if (edge) {
        if constexpr (SC::ON) asm volatile("");  // keeps the block a branch rather than selects on every tile
#pragma unroll
        for (int bb = 0; bb < BKV / 32; ++bb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (hidden_key(sc, kv0 + 32 * bb + 8 * (r >> 2) + 4 * lh + (r & 3), qrow)) sacc[bb][r] = HIDDEN;
      }
      float mx = HIDDEN;
#pragma unroll
      for (int bb = 0; bb < BKV / 32; ++bb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = SC::CAPPED ? fminf(mx, sacc[bb][r]) : fmaxf(mx, sacc[bb][r]);
      // key 0 is visible to every query: finite from the first tile on
      const float mc = fmaxf(m, SC::CAPPED ? fmaf(halves_max(-mx), 2.0f * sc.c2, sc.c2) : halves_max(mx) * sl2);
      if (__builtin_amdgcn_ballot_w64(mc > m + LAG)) {
        const float alpha = ex2(m - mc);
        m = mc;
        l *= alpha;
        if constexpr (SC::ON) lb *= alpha;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) oacc[i] *= alpha;
      }
      float ls = 0.f;
      const float top = sc.c2 - m;
#pragma unroll
      for (int bb = 0; bb < BKV / 32; ++bb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = ex2(SC::CAPPED ? fmaf(sacc[bb][r], -2.0f * sc.c2, top) : fmaf(sacc[bb][r], sl2, -m));
          sacc[bb][r] = p;
          ls += p;
        }
      if constexpr (SC::ON) l += ls;  // (this lane's keys: the halves are added at the end)
      else l += halves_sum(ls);
#pragma unroll
      for (int s = 0; s < BKV / 16; ++s) {
        const u32x4 pf = pack_frag(sacc[s >> 1], 8 * (s & 1));
        if constexpr (SC::ON) {
#pragma unroll
          for (int w = 0; w < 4; ++w) lb = add_bf2(pf[w], lb);
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
          oacc[i] = mfma32(fa.cols(i, v_minus_k + cur * STAGE + s * 16 * D * 2), pf, oacc[i]);
      }
    }
    sync_lds();
  };
  for (int kt = SC::ON ? kt0 : 0; kt < nkt; kt += 2) {
    step(std::integral_constant<int, 0>{}, kt);
    if (kt + 1 < nkt) step(std::integral_constant<int, 1>{}, kt + 1);
  }

  if constexpr (SC::ON) {
    l = halves_sum(l);
    lb = halves_sum(lb);
  }
  if (qrow < S) {
    const float inv = 1.0f / (SC::ON ? lb : l);
    bf16_t* orow = o + (qtile.row0 + qrow) * nq * hd + h * hd;
    if constexpr (SC::ON) store_rest<D>(sc, (qtile.row0 + qrow) * nq * hd + h * hd, oacc, inv, hd, lh);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const int d = 32 * i + 8 * rq + 4 * lh;
        if (PACKED && d >= hd) continue;
        *(u32x2*)(orow + d) = u32x2{pack_bf2(oacc[i][4 * rq] * inv, oacc[i][4 * rq + 1] * inv),
                                    pack_bf2(oacc[i][4 * rq + 2] * inv, oacc[i][4 * rq + 3] * inv)};
      }
    if (lh == 0) lse[qtile.vec0 + qrow] = (m + log2f(l)) * LN2;
  }
}

// attn_bwd_pre_kernel for one row of packed sequences and heads of any width: D / 8 lanes a head.
template <int D, bool REST>
LS_DEV void bwd_pre_row(const AttnShape& sh, const bf16_t* __restrict__ orow, const bf16_t* __restrict__ drow,
                        const float* __restrict__ lse, float* __restrict__ Dv, float* __restrict__ lse2, int64_t t,
                        const bf16_t* __restrict__ rrow, bool neg, float less) {
  constexpr int CPH = D / 8;
  const int lane = threadIdx.x & 63, c = lane % CPH;
  for (int h = lane / CPH; h - lane / CPH < sh.nq; h += 64 / CPH) {
    float acc = 0.f;
    if (h < sh.nq && 8 * c < sh.d) {
      const u32x4 a = load16(orow + h * sh.d + 8 * c), g = load16(drow + h * sh.d + 8 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc += bf_lo(a[e]) * bf_lo(g[e]) + bf_hi(a[e]) * bf_hi(g[e]);
      if constexpr (REST) {
        const u32x4 r = load16(rrow + h * sh.d + 8 * c);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc += bf_lo(r[e]) * bf_lo(g[e]) + bf_hi(r[e]) * bf_hi(g[e]);
      }
    }
#pragma unroll
    for (int off = CPH / 2; off >= 1; off >>= 1) acc += __shfl_xor(acc, off);
    if (c == 0 && h < sh.nq) {
      const int64_t i = (int64_t)h * sh.seq + t;
      Dv[i] = neg ? -acc : acc;
      lse2[i] = lse[i] * LOG2E - less;
    }
  }
}

// D[b,h,s] = <dO, O> over the head's d columns (fp32), and the log-sum-exp in
// base 2 (lse * log2(e)), the form the backward kernels subtract.
// REST: O is o and the rest that its rounding left.  neg: -D, what dP starts from where scores are modified; less: c2 of a
// cap, which every exponent less the log-sum-exp holds (the difference, at most 2 c2, is rounded once: 2^-24 of it, below
// the 2^-21 cap that a capped score carries).
template <int D, bool PACKED, bool REST = false>
__global__ __launch_bounds__(256) void attn_bwd_pre_kernel(AttnShape sh, const bf16_t* __restrict__ o,
                                                           const bf16_t* __restrict__ dout,
                                                           const float* __restrict__ lse, float* __restrict__ Dv,
                                                           float* __restrict__ lse2, const bf16_t* __restrict__ rest,
                                                           bool neg, float less) {
  constexpr int CPH = D / 8;  // 16-byte chunks per head
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)(PACKED ? packed_wg() : (int)blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (t >= (int64_t)sh.batch * sh.seq) return;
  if constexpr (PACKED) {
    const int64_t at = t * sh.nq * sh.d;
    bwd_pre_row<D, REST>(sh, o + at, dout + at, lse, Dv, lse2, t, rest + at, neg, less);
    return;
  }
  const int b = (int)(t / sh.seq), s = (int)(t % sh.seq);
  const int chunks = sh.nq * CPH;
  const bf16_t* orow = o + t * sh.nq * D;
  const bf16_t* drow = dout + t * sh.nq * D;
  for (int c0 = 0; c0 < chunks; c0 += 64) {
    const int c = c0 + lane;
    float acc = 0.f;
    if (c < chunks) {
      const u32x4 a = load16(orow + c * 8), g = load16(drow + c * 8);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc += bf_lo(a[e]) * bf_lo(g[e]) + bf_hi(a[e]) * bf_hi(g[e]);
    }
#pragma unroll
    for (int off = CPH / 2; off >= 1; off >>= 1) acc += __shfl_xor(acc, off);
    if (c < chunks && (c % CPH) == 0) {
      const int64_t i = ((int64_t)b * sh.nq + c / CPH) * sh.seq + s;
      Dv[i] = acc;
      lse2[i] = lse[i] * LOG2E;
    }
  }
}

// Inverse rotation of a gradient held in MFMA layout: lane holds columns
// 32i + 8(r/4) + 4lh + r%4 of one row at position `pos`; the pair partner of
// column d < D/2 is d + D/2, in register block i + D/64 of the same lane.
// Without rotation (rope_cs null) only columns below `width` are stored.
template <int D>
LS_DEV void unrotate_store(const f32x16 (&acc)[D / 32], float scale, const float* rope_cs, int seq, int pos, int lh,
                           bf16_t* row, int width = D) {
  constexpr int HALF = D / 2, IP = HALF / 32;
  if (rope_cs == nullptr) {
    auto store = [&](bool whole) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
          const int d = 32 * i + 8 * rq + 4 * lh;
          if (!whole && d >= width) continue;
          *(u32x2*)(row + d) = u32x2{pack_bf2(acc[i][4 * rq] * scale, acc[i][4 * rq + 1] * scale),
                                     pack_bf2(acc[i][4 * rq + 2] * scale, acc[i][4 * rq + 3] * scale)};
        }
    };
    if (width == D) store(true);
    else store(false);
    return;
  }
  // cos and sin of the lane's angle indices (4 consecutive ones per 8-column
  // group, 16-byte loads), all in flight before the rotations use them; the
  // second half of the head uses the angles of the first
  const float* cb = rope_cs + (int64_t)pos * HALF;
  const float* sb = rope_cs + (int64_t)seq * HALF + (int64_t)pos * HALF;
  f32x4 c4[IP][4], s4[IP][4];
#pragma unroll
  for (int i = 0; i < IP; ++i)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      const int d = 32 * i + 8 * rq + 4 * lh;
      c4[i][rq] = *(const f32x4*)(cb + d);
      s4[i][rq] = *(const f32x4*)(sb + d);
    }
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      const int d = 32 * i + 8 * rq + 4 * lh;
      float out[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = acc[i][4 * rq + e] * scale;
        if (i < IP) {  // first half: x1' = x1 cos + x2 sin
          const float x2 = acc[i + IP][4 * rq + e] * scale;
          out[e] = x * c4[i][rq][e] + x2 * s4[i][rq][e];
        } else {  // second half: x2' = x2 cos - x1 sin
          const float x1 = acc[i - IP][4 * rq + e] * scale;
          out[e] = x * c4[i - IP][rq][e] - x1 * s4[i - IP][rq][e];
        }
      }
      *(u32x2*)(row + d) = u32x2{pack_bf2(out[0], out[1]), pack_bf2(out[2], out[3])};
    }
}

// A lane's key row [dK | dV] of partial sums: columns 32i + 8(r/4) + 4lh + r%4.
template <int D>
LS_DEV void store_sums(float* row, const f32x16 (&dk)[D / 32], const f32x16 (&dv)[D / 32], int lh) {
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      const int c = 32 * i + 8 * rq + 4 * lh;
      *(f32x4*)(row + c) = f32x4{dk[i][4 * rq], dk[i][4 * rq + 1], dk[i][4 * rq + 2], dk[i][4 * rq + 3]};
      *(f32x4*)(row + D + c) = f32x4{dv[i][4 * rq], dv[i][4 * rq + 1], dv[i][4 * rq + 2], dv[i][4 * rq + 3]};
    }
}

// The probability of a raw score, exp2 of the base-2 score less the log-sum-exp L (capped: c2 - 2 c2 r - (L + c2)), and
// (capped) w = r (1 - r), a quarter of the cap's slope.
template <class SC>
LS_DEV float prob_slope(const SC& sc, float s, float sl2, float L, float& w) {
  if constexpr (SC::CAPPED) {
    const float r = sc.half(s);
    w = fmaf(-r, r, r);
    return ex2(fmaf(r, -2.0f * sc.c2, -L));
  } else {
    return ex2(fmaf(s, sl2, -L));
  }
}

// Backward of one kv head of a packed sequence of up to 32 rows by one wave: dQ of
// its query heads g0 .. g1 - 1 of the group, and dK and dV summed over them (to
// `sums`, if given, as a part's fp32 sums).  D = sum P dP comes from the wave's own P and dP:
// of few keys it is as large as dP, and from the rounded o it would cost dS more
// than its own rounding does.
// Scores and dP are formed both ways round, with the lanes owning keys for dK and
// dV and owning queries for dQ: two more small products instead of transposing
// dS.  K, Q and dO go through the wave's own LDS tiles for their transposes.
template <int D>
constexpr int short_lds_bytes() {
  return 3 * PACKED_SHORT * D * 2 + 2 * PACKED_SHORT * 4;
}
template <int D, class SC>
LS_DEV void short_bwd(const AttnShape& sh, const SC& sc, const PackedTile& t, int kvh, const bf16_t* __restrict__ qkv,
                      const bf16_t* __restrict__ dout, const float* __restrict__ lse2,
                      bf16_t* __restrict__ dqkv, float scale, float sl2, char* lds, int g0, int g1, float* sums) {
  constexpr int NSD = D / 16, NI = D / 32;
  const int nq = sh.nq, nkv = sh.nkv, hq0 = kvh * (nq / nkv) + g0, hq1 = kvh * (nq / nkv) + g1, hd = sh.d;
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * hd, ldo = (int64_t)nq * hd;
  const bool ok = lr < t.len;
  const int64_t r0 = t.start + (int64_t)(ok ? lr : 0);
  bf16_t *kt = (bf16_t*)lds, *qt = kt + PACKED_SHORT * D, *ot = qt + PACKED_SHORT * D;
  float *lv = (float*)(ot + PACKED_SHORT * D), *dvv = lv + PACKED_SHORT;
  u32x4 kf[NSD], vf[NSD], qf[NSD], of[NSD];
  const __amdgpu_buffer_rsrc_t rows = seq_rows(qkv, t, ld), drows = seq_rows(dout, t, ldo);
  auto at = [&](int r, int64_t ldr, int head) { return (uint32_t)(r * (int)ldr + head * hd) * 2u; };
  get_rows<D>(kf, rows, at(lr, ld, nq + kvh), lh, hd);
  get_rows<D>(vf, rows, at(lr, ld, nq + nkv + kvh), lh, hd);
  f32x16 dk[NI], dv[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) dk[i] = dv[i] = f32x16{};
  for (int h = hq0; h < hq1; ++h) {
    get_rows<D>(qf, rows, at(lr, ld, h), lh, hd);
    get_rows<D>(of, drows, at(lr, ldo, h), lh, hd);
    const int64_t v0 = (int64_t)h * sh.seq + t.start;
    const float L = ok ? lse2[v0 + lr] : 0.f;
    if (h == hq0) put_rows<D>(kt, kf, lr, lh);
    put_rows<D>(qt, qf, lr, lh);
    put_rows<D>(ot, of, lr, lh);
    if (lh == 0) lv[lr] = L;
    wave_lds_order();
    {  // lanes own queries: element r is key 8(r/4) + 4lh + r%4
      f32x16 s{}, p{}, dq[NI];
      float Dr = 0.f;
#pragma unroll
      for (int c = 0; c < NSD; ++c) {
        s = mfma32(kf[c], qf[c], s);
        p = mfma32(vf[c], of[c], p);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float w;
        s[r] = prob_slope(sc, s[r], sl2, L, w);
        if (hidden_key(sc, 8 * (r >> 2) + 4 * lh + (r & 3), lr)) s[r] = p[r] = 0.f;
        Dr = fmaf(s[r], p[r], Dr);
        if constexpr (SC::CAPPED) s[r] *= w;
      }
      Dr = halves_sum(Dr);
      if (lh == 0) dvv[lr] = Dr;
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = s[r] * (p[r] - Dr);
#pragma unroll
      for (int i = 0; i < NI; ++i) dq[i] = f32x16{};
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const u32x4 sf = pack_frag(p, 8 * c);
#pragma unroll
        for (int i = 0; i < NI; ++i) dq[i] = mfma32(colt_frag<D>(kt, 32 * i, c, lane), sf, dq[i]);
      }
      if (ok) unrotate_store<D>(dq, scale, nullptr, 0, 0, lh, dqkv + r0 * ld + h * hd, hd);
    }
    wave_lds_order();
    {  // lanes own keys: element r is query 8(r/4) + 4lh + r%4
      f32x16 s{}, p{};
#pragma unroll
      for (int c = 0; c < NSD; ++c) {
        s = mfma32(qf[c], kf[c], s);
        p = mfma32(of[c], vf[c], p);
      }
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const f32x4 lq = *(const f32x4*)&lv[8 * rq + 4 * lh], dq4 = *(const f32x4*)&dvv[8 * rq + 4 * lh];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * rq + e;
          if constexpr (SC::ON) {
            float w;
            s[r] = prob_slope(sc, s[r], sl2, lq[e], w);
            if (hidden_key(sc, lr, 8 * rq + 4 * lh + e)) s[r] = 0.f;
            p[r] = (SC::CAPPED ? s[r] * w : s[r]) * (p[r] - dq4[e]);
          } else {
            if (8 * rq + 4 * lh + e < lr) s[r] = -INFINITY;
            s[r] = ex2(fmaf(s[r], sl2, -lq[e]));
            p[r] = s[r] * (p[r] - dq4[e]);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const u32x4 pf = pack_frag(s, 8 * c), sf = pack_frag(p, 8 * c);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          dv[i] = mfma32(colt_frag<D>(ot, 32 * i, c, lane), pf, dv[i]);
          dk[i] = mfma32(colt_frag<D>(qt, 32 * i, c, lane), sf, dk[i]);
        }
      }
    }
    wave_lds_order();
  }
  if (!ok) return;
  if (sums) {
    store_sums<D>(sums + lr * (2 * D), dk, dv, lh);
    return;
  }
  unrotate_store<D>(dk, scale, nullptr, 0, 0, lh, dqkv + r0 * ld + (nq + kvh) * hd, hd);
  unrotate_store<D>(dv, 1.0f, nullptr, 0, 0, lh, dqkv + r0 * ld + (nq + nkv + kvh) * hd, hd);
}

// The same for a middle sequence, of up to 64 rows, by a pair of waves: wave j of the
// pair owns keys and queries 32j .. 32j + 31, takes the other's Q, dO and K rows
// from the pair's LDS tiles, and (wave 1) V of the first rows from global memory.
// The barriers are the workgroup's, so both pairs go through all heads; a pair
// without a sequence (len 0) only waits.
template <int D>
constexpr int mid_lds_bytes() {
  return 3 * PACKED_MID * D * 2 + 2 * PACKED_MID * 4;
}
template <int D, class SC>
LS_DEV void mid_bwd(const AttnShape& sh, const SC& sc, const PackedTile& t, int kvh, const bf16_t* __restrict__ qkv,
                    const bf16_t* __restrict__ dout, const float* __restrict__ lse2,
                    bf16_t* __restrict__ dqkv, float scale, float sl2, char* lds, int g0, int g1, float* sums) {
  constexpr int NSD = D / 16, NI = D / 32;
  const int nq = sh.nq, nkv = sh.nkv, hq0 = kvh * (nq / nkv) + g0, hq1 = kvh * (nq / nkv) + g1, hd = sh.d;
  const int lane = threadIdx.x & 63, lr = lane & 31, lh = lane >> 5;
  const int j = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) & 1, row = 32 * j + lr;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * hd, ldo = (int64_t)nq * hd;
  const bool ok = row < t.len;
  const int64_t r0 = t.start + (int64_t)(ok ? row : 0);
  bf16_t *kt = (bf16_t*)lds, *qt = kt + PACKED_MID * D, *ot = qt + PACKED_MID * D;
  float *lv = (float*)(ot + PACKED_MID * D), *dvv = lv + PACKED_MID;
  u32x4 kf[NSD], vf[NSD], qf[NSD], of[NSD];
  const __amdgpu_buffer_rsrc_t rows = seq_rows(qkv, t, ld), drows = seq_rows(dout, t, ldo);
  auto at = [&](int r, int64_t ldr, int head) { return (uint32_t)(r * (int)ldr + head * hd) * 2u; };
  get_rows<D>(kf, rows, at(row, ld, nq + kvh), lh, hd);
  get_rows<D>(vf, rows, at(row, ld, nq + nkv + kvh), lh, hd);
  f32x16 dk[NI], dv[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) dk[i] = dv[i] = f32x16{};
  for (int h = hq0; h < hq1; ++h) {
    get_rows<D>(qf, rows, at(row, ld, h), lh, hd);
    get_rows<D>(of, drows, at(row, ldo, h), lh, hd);
    const int64_t v = (int64_t)h * sh.seq + t.start;
    const float L = ok ? lse2[v + row] : 0.f;
    if (h > hq0) sync_lds();  // the tiles of the head before are read
    if (h == hq0) put_rows<D>(kt + 32 * j * D, kf, lr, lh);
    put_rows<D>(qt + 32 * j * D, qf, lr, lh);
    put_rows<D>(ot + 32 * j * D, of, lr, lh);
    if (lh == 0) lv[row] = L;
    sync_lds();
    // the wave's queries, keys of block b: element r is key 32b + 8(r/4) + 4lh + r%4
    f32x16 dq[NI], s2[2], p2[2];
#pragma unroll
    for (int i = 0; i < NI; ++i) dq[i] = f32x16{};
    if (t.len > 0) {
      float Dr = 0.f;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        s2[b] = p2[b] = f32x16{};
        if (b > j) continue;
        if (b == j) {
#pragma unroll
          for (int c = 0; c < NSD; ++c) p2[b] = mfma32(vf[c], row_frag<D>(ot, row, c, lh), p2[b]);
        } else {  // (a middle sequence has all of its first 32 rows)
          u32x4 v0[NSD];
          get_rows<D>(v0, rows, at(lr, ld, nq + nkv + kvh), lh, hd);
#pragma unroll
          for (int c = 0; c < NSD; ++c) p2[b] = mfma32(v0[c], row_frag<D>(ot, row, c, lh), p2[b]);
        }
#pragma unroll
        for (int c = 0; c < NSD; ++c)
          s2[b] = mfma32(row_frag<D>(kt, 32 * b + lr, c, lh), row_frag<D>(qt, row, c, lh), s2[b]);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float w;
          s2[b][r] = prob_slope(sc, s2[b][r], sl2, L, w);
          if (hidden_key(sc, 32 * b + 8 * (r >> 2) + 4 * lh + (r & 3), row)) s2[b][r] = p2[b][r] = 0.f;
          Dr = fmaf(s2[b][r], p2[b][r], Dr);
          if constexpr (SC::CAPPED) s2[b][r] *= w;
        }
      }
      Dr = halves_sum(Dr);
      if (lh == 0) dvv[row] = Dr;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if (b > j) continue;
#pragma unroll
        for (int r = 0; r < 16; ++r) p2[b][r] = s2[b][r] * (p2[b][r] - Dr);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const u32x4 sf = pack_frag(p2[b], 8 * c);
#pragma unroll
          for (int i = 0; i < NI; ++i) dq[i] = mfma32(colt_frag<D>(kt + 32 * b * D, 32 * i, c, lane), sf, dq[i]);
        }
      }
    }
    sync_lds();  // the other wave's D
    if (t.len == 0) continue;
    // the wave's keys, queries of block b: element r is query 32b + 8(r/4) + 4lh + r%4
    for (int b = j; b < 2; ++b) {
      f32x16 s{}, p{};
#pragma unroll
      for (int c = 0; c < NSD; ++c) {
        s = mfma32(row_frag<D>(qt, 32 * b + lr, c, lh), kf[c], s);
        p = mfma32(row_frag<D>(ot, 32 * b + lr, c, lh), vf[c], p);
      }
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const int at = 32 * b + 8 * rq + 4 * lh;
        const f32x4 lq = *(const f32x4*)&lv[at], dq4 = *(const f32x4*)&dvv[at];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * rq + e;
          if constexpr (SC::ON) {
            float w;
            s[r] = prob_slope(sc, s[r], sl2, lq[e], w);
            if (hidden_key(sc, row, at + e)) s[r] = 0.f;
            p[r] = (SC::CAPPED ? s[r] * w : s[r]) * (p[r] - dq4[e]);
          } else {
            if (at + e < row) s[r] = -INFINITY;
            s[r] = ex2(fmaf(s[r], sl2, -lq[e]));
            p[r] = s[r] * (p[r] - dq4[e]);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const u32x4 pf = pack_frag(s, 8 * c), sf = pack_frag(p, 8 * c);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          dv[i] = mfma32(colt_frag<D>(ot + 32 * b * D, 32 * i, c, lane), pf, dv[i]);
          dk[i] = mfma32(colt_frag<D>(qt + 32 * b * D, 32 * i, c, lane), sf, dk[i]);
        }
      }
    }
    if (ok) unrotate_store<D>(dq, scale, nullptr, 0, 0, lh, dqkv + r0 * ld + h * hd, hd);
  }
  if (!ok) return;
  if (sums) {
    store_sums<D>(sums + row * (2 * D), dk, dv, lh);
    return;
  }
  unrotate_store<D>(dk, scale, nullptr, 0, 0, lh, dqkv + r0 * ld + (nq + kvh) * hd, hd);
  unrotate_store<D>(dv, 1.0f, nullptr, 0, 0, lh, dqkv + r0 * ld + (nq + nkv + kvh) * hd, hd);
}

// dK and dV for 128 keys of one kv head (4 waves x 32 keys), summed over the
// query heads of the group, no atomics.  The 1-D grid runs the key tiles with
// the most queries after them (lowest key index) first.  With few kv heads
// (and so few workgroups) the group's query heads are split over `hsplit`
// workgroups, each of which writes its fp32 partial sums to `part`
// ([hsplit][batch*seq][nkv][dK | dV]); attn_bwd_dkdv_reduce then adds the
// partials in a fixed order and stores dK and dV.
//
// A wave issues one MFMA per slot.  Each 32-query block of a 64-query tile
// takes four phases: S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS.
// The softmax work is spread between the MFMAs: P = exp2(S - LSE) (and its
// bf16 operands) during the dP phase, dS = P (dP - D) during the dV phase, so
// the vector ALU works while the matrix core does.  Every MFMA operand read
// from LDS is issued RA slots ahead into a ring of registers (across tile
// boundaries too), so no MFMA waits on an LDS read.  Three LDS stages: RA
// slots before the end of tile t each wave waits for its loads of tile t+1
// and for the other waves (whose reads of tile t-1 are then done), and the
// loads of tile t+2 go into tile t-1's stage.
//
// Packed sequences: a workgroup takes a piece of the plan's work on tiles (a key tile and kv
// head, or a part of its 64-query steps of all heads of the group, whose partial
// sums go to a slot of `part`), or past those four short sequences and a kv head.
// One stage: Q tile, dO tile, log-sum-exp (base 2) and D of its queries
// (every operand of a stage within the reach of an LDS instruction's offset).
template <int D>
struct DkdvStage {
  bf16_t q[BWD_BQ * D];
  bf16_t o[BWD_BQ * D];
  float l[256];
  float d[256];
};
template <int D, bool SPLIT, bool PACKED, class SC>
LS_DEV void dkdv_tile(const AttnShape& sh, const SC& sc, const PackedView& pk, const int x, DkdvStage<D> (&stg)[DKDV_STAGES],
                      const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ dout, const float* __restrict__ lse2,
                      const float* __restrict__ Dv, bf16_t* __restrict__ dqkv, const float* __restrict__ rope_cs,
                      float scale, float sl2, int hsplit_arg, float* __restrict__ part) {
  constexpr int NSD = D / 16, NI = D / 32;  // 16-wide d steps; 32-row d blocks
  constexpr int P1 = NSD, P2 = NSD, P3 = 2 * NI, P4 = 2 * NI;  // slots per phase
  constexpr int NB = P1 + P2 + P3 + P4;     // slots of a 32-query block
  constexpr int NSLOT = 2 * NB;
  constexpr int RING = 8, RA = RING - 1;    // operand ring; read-ahead in slots
  static_assert(NSLOT % RING == 0, "ring positions repeat every tile");
  static_assert(P1 >= 4 && P2 >= 4 && 16 % P2 == 0 && 16 % P3 == 0, "phase sizes");
  constexpr int BAR = NSLOT - RA;           // slot of the barrier
  const int hsplit = SPLIT ? hsplit_arg : 1;  // the unsplit instance folds every split term away
  const int nq = sh.nq, nkv = sh.nkv, G = nq / nkv, Gs = SPLIT ? G / hsplit : G;
  const int per = nkv * sh.batch * hsplit;
  const int hs = (x % per) % hsplit, kvh = ((x % per) / hsplit) % nkv, b = ((x % per) / hsplit) / nkv;
  int kvt = x / per, S = sh.seq;
  int64_t row0 = (int64_t)b * S, vec0 = (int64_t)b * nq * S;  // this sequence's first row; its entry of head 0's vectors
  int parts = 1, part_no = 0, slot = 0;
  if constexpr (PACKED) {
    static_assert(sizeof(stg) >= 4 * short_lds_bytes<D>() && sizeof(stg) >= 2 * mid_lds_bytes<D>(),
                  "the tiles of small sequences");
    PackedTile t;
    const PackedKind kind = packed_piece(pk, kvt, sh.seq, t, part_no);
    if (kind == PACKED_IS_MID) {
      const int pair = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 7);
      mid_bwd<D>(sh, sc, t, kvh, qkv, dout, lse2, dqkv, scale, sl2, (char*)&stg[0] + pair * mid_lds_bytes<D>(), 0, G,
                 nullptr);
      return;
    }
    if (t.len == 0) return;
    if (kind == PACKED_IS_SHORT) {
      const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
      short_bwd<D>(sh, sc, t, kvh, qkv, dout, lse2, dqkv, scale, sl2, (char*)&stg[0] + w * short_lds_bytes<D>(), 0, G,
                   nullptr);
      return;
    }
    parts = __builtin_amdgcn_readfirstlane((int)t.parts);
    slot = __builtin_amdgcn_readfirstlane((int)t.slot);
    if (t.len <= PACKED_MID) {  // few small sequences: the group's heads are what is cut
      const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
      const int g0 = G * part_no / parts, g1 = G * (part_no + 1) / parts;
      float* sums = parts > 1 ? part + (((int64_t)slot + part_no) * nkv + kvh) * (PACKED_ROWS * 2 * D) : nullptr;
      if (t.len <= PACKED_SHORT) {
        if (w == 0) short_bwd<D>(sh, sc, t, kvh, qkv, dout, lse2, dqkv, scale, sl2, (char*)&stg[0], g0, g1, sums);
      } else {
        if (w >= 2) t.len = 0;  // (the first pair's)
        mid_bwd<D>(sh, sc, t, kvh, qkv, dout, lse2, dqkv, scale, sl2, (char*)&stg[0] + (w >> 1) * mid_lds_bytes<D>(), g0,
                   g1, sums);
      }
      return;
    }
    kvt = (t.len + BWD_BKV - 1) / BWD_BKV - 1 - t.rank;  // the most work: the first keys
    S = t.len;
    row0 = vec0 = t.start;
  }
  const int hd = PACKED ? sh.d : D;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * hd;
  const int64_t ldo = (int64_t)nq * hd;
  const bf16_t* base = qkv + row0 * ld;
  const bf16_t* dbase = dout + row0 * ldo;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int kv0 = kvt * BWD_BKV;
  const int kvrow = kv0 + 32 * wave + lr;

  // tiles t = 0 .. Gs*nqt-1: query head kvh*G + hs*Gs + t/nqt, queries q_begin + (t%nqt)*BWD_BQ ..
  const int q_begin = kv0;  // earlier queries see none of these keys
  int q_end = S;
  if constexpr (SC::ON) q_end = min(S, kv0 + BWD_BKV - 1 + sc.window);  // nor do later ones
  const int nqt = (q_end - q_begin + BWD_BQ - 1) / BWD_BQ;
  int tbegin = 0, ntiles = Gs * nqt;  // (packed: this part's)
  if constexpr (PACKED && SC::ON) {
    // the plan's parts count all queries behind a key; a window may leave a part none, whose sums are 0
    const int all = ntiles;
    tbegin = (int)((int64_t)all * part_no / parts);
    ntiles = (int)((int64_t)all * (part_no + 1) / parts);
  } else if constexpr (PACKED) {
    if (parts > 1) {
      // (a plan has no more parts than steps; whatever it holds, a part has a step, within the sequence)
      const int all = ntiles;
      tbegin = min((int)((int64_t)all * part_no / parts), all - 1);
      ntiles = max((int)((int64_t)all * (part_no + 1) / parts), tbegin + 1);
    }
  }
  const TileLoader<D, BWD_BQ> tlq(ld, wave, lane, hd), tlo(ldo, wave, lane, hd);
  // modified scores: the head and the query tile of the next tile to load, and of the current one, are counted, as divisions
  // by nqt cost a tenth of the loop's scalar instructions (6007 rows of 12/4 heads of 64 through a window of 300, training
  // pass 86.5 -> 84.2 us; plain scores, whose loop hides them, 450 -> 461 with both changes of this kind)
  int next_h = 0, next_q = 0, tile_q = 0;
  if constexpr (SC::ON) {
    next_h = kvh * G + hs * Gs + tbegin / nqt;
    next_q = tile_q = tbegin % nqt;
  }
  auto issue = [&](int t, int st) {
    const int h = SC::ON ? next_h : kvh * G + hs * Gs + t / nqt, q0 = q_begin + (SC::ON ? next_q : t % nqt) * BWD_BQ;
    if constexpr (SC::ON) {
      if (++next_q == nqt) {
        next_q = 0;
        ++next_h;
      }
    }
    tlq(base, ld, q0, S, h * hd, stg[st].q, wave);
    tlo(dbase, ldo, q0, S, h * hd, stg[st].o, wave);
    const int64_t v0 = vec0 + (int64_t)h * sh.seq;
    if (wave == 0) load_vec64(rsrc(lse2 + v0, (uint32_t)S * 4), q0, S, stg[st].l, lane);
    if (wave == 1) load_vec64(rsrc(Dv + v0, (uint32_t)S * 4), q0, S, stg[st].d, lane);
  };
  if (!SC::ON || tbegin < ntiles) issue(tbegin, 0);
  if (tbegin + 1 < ntiles) issue(tbegin + 1, 1);

  u32x4 kf[NSD], vf[NSD];
#pragma unroll
  for (int s = 0; s < NSD; ++s) {
    const bool ok = kvrow < S && 16 * s + 8 * lh < hd;
    kf[s] = ok ? load16(base + (int64_t)kvrow * ld + (nq + kvh) * hd + 16 * s + 8 * lh) : u32x4{0u, 0u, 0u, 0u};
    vf[s] = ok ? load16(base + (int64_t)kvrow * ld + (nq + nkv + kvh) * hd + 16 * s + 8 * lh) : u32x4{0u, 0u, 0u, 0u};
  }

  f32x16 dk[NI], dv[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[i][r] = dv[i][r] = 0.f;

  // MFMA A operand of slot j of the tile in stage st.
  auto operand = [&](auto j_c, int st) -> u32x4 {
    constexpr int j = decltype(j_c)::value;
    constexpr int qb = j / NB, k = j % NB;
    if constexpr (k < P1) return row_frag<D>(stg[st].q, 32 * qb + lr, k, lh);
    else if constexpr (k < P1 + P2) return row_frag<D>(stg[st].o, 32 * qb + lr, k - P1, lh);
    else if constexpr (k < P1 + P2 + P3) {
      constexpr int c = k - P1 - P2;
      return colt_frag<D>(stg[st].o, 32 * (c % NI), 2 * qb + c / NI, lane);
    } else {
      constexpr int c = k - P1 - P2 - P3;
      return colt_frag<D>(stg[st].q, 32 * (c % NI), 2 * qb + c / NI, lane);
    }
  };

  u32x4 ring[RING];
  f32x16 sacc, pacc;
  f32x16 wacc;  // capped: P times a quarter of the cap's slope
  f32x4 Lq[2], Dq[2];  // base-2 log-sum-exp and D of the block's queries 8rq + 4lh + {0..3}, rq even / odd
  u32x4 pf[2], sf[2];

  // One tile in stage st; st1 and st2 are the stages of the next two tiles
  // (the three rotate from tile to tile).
  auto tile = [&](int t, int st, int st1, int st2) {
    const int q0 = q_begin + (SC::ON ? tile_q : t % nqt) * BWD_BQ;
    if constexpr (SC::ON) {
      if (++tile_q == nqt) tile_q = 0;
    }
    // causal mask, on the tiles at the diagonal only (some query of the tile
    // precedes some key of the wave): element r of block qb is query
    // q0 + 4lh + c with c = 32qb + 8(r/4) + r%4, kept when c >= lo, i.e.
    // q >= kvrow; a masked score becomes -inf, so its probability is
    // exp2(-inf) = 0.  Queries past the end of the sequence need no mask: their
    // Q, dO, LSE and D read as zero, so they add nothing to dK or dV.
    const int lo = kvrow - q0 - 4 * lh;
    bool diag = q0 < kv0 + 32 * wave + 31;
    if constexpr (SC::ON) diag = diag || q0 + BWD_BQ - 1 >= kv0 + 32 * wave + sc.window;
    static_for<NSLOT>([&](auto j_c) {
      constexpr int j = decltype(j_c)::value;
      constexpr int qb = j / NB, k = j % NB;
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (j == BAR) {
        LS_WAIT_VMCNT(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 2 < ntiles) issue(t + 2, st2);
      }
      const u32x4 a = ring[j % RING];
      if constexpr (k < P1) {  // S = Q K^T; read the block's log-sum-exp
        sacc = mfma32(a, kf[k], k == 0 ? f32x16{} : sacc);
        // (modified scores: -D of the block's queries, from which dP's sums start)
        if constexpr (SC::ON && k < 4) {
          const f32x4 d = *(const f32x4*)&stg[st].d[32 * qb + 8 * k + 4 * lh];
#pragma unroll
          for (int e = 0; e < 4; ++e) pacc[4 * k + e] = d[e];
        }
        if constexpr (k == P1 - 1) Lq[0] = *(const f32x4*)&stg[st].l[32 * qb + 4 * lh];
      } else if constexpr (k < P1 + P2) {  // dP = dO V^T, meanwhile P = exp2(S sl2 - LSE2)
        constexpr int c = k - P1, PER = 16 / P2;
        pacc = mfma32(a, vf[c], c == 0 && !SC::ON ? f32x16{} : pacc);
        if constexpr (c == 0 && !SC::CAPPED) {
          if (diag) {
            asm volatile("");  // keeps the block a branch rather than selects on every tile
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int q = 32 * qb + 8 * (r >> 2) + (r & 3);
              bool hide = q < lo;
              if constexpr (SC::ON) hide = hide || q - lo >= sc.window;
              if (hide) sacc[r] = -INFINITY;
            }
          }
        }
        static_for<PER>([&](auto u_c) {
          constexpr int r = c * PER + decltype(u_c)::value, rq = r >> 2, e = r & 3;
          // the next group's log-sum-exp, one group ahead
          if constexpr (e == 0 && rq < 3) Lq[(rq + 1) & 1] = *(const f32x4*)&stg[st].l[32 * qb + 8 * (rq + 1) + 4 * lh];
          if constexpr (!SC::ON && r == 12) Dq[0] = *(const f32x4*)&stg[st].d[32 * qb + 4 * lh];
          if constexpr (SC::CAPPED) {
            float w;
            sacc[r] = prob_slope(sc, sacc[r], sl2, Lq[rq & 1][e], w);
            wacc[r] = sacc[r] * w;
          } else {
            sacc[r] = ex2(fmaf(sacc[r], sl2, -Lq[rq & 1][e]));
          }
          if constexpr (SC::CAPPED && (r & 7) == 7) {  // a capped score is finite: masked afterwards
            if (diag) {
              asm volatile("");
#pragma unroll
              for (int u = r - 7; u <= r; ++u) {
                const int q = 32 * qb + 8 * (u >> 2) + (u & 3);
                if (q < lo || q - lo >= sc.window) sacc[u] = wacc[u] = 0.f;
              }
            }
          }
          if constexpr ((r & 7) == 7) pf[r >> 3] = pack_frag(sacc, r - 7);
        });
      } else if constexpr (k < P1 + P2 + P3) {  // dV^T += dO^T P, meanwhile dS = P (dP - D)
        constexpr int c = k - P1 - P2, PER = 16 / P3;
        dv[c % NI] = mfma32(a, pf[c / NI], dv[c % NI]);
        static_for<PER>([&](auto u_c) {
          constexpr int r = c * PER + decltype(u_c)::value, rq = r >> 2, e = r & 3;
          if constexpr (!SC::ON && e == 0 && rq < 3)
            Dq[(rq + 1) & 1] = *(const f32x4*)&stg[st].d[32 * qb + 8 * (rq + 1) + 4 * lh];
          if constexpr (SC::ON) pacc[r] *= SC::CAPPED ? wacc[r] : sacc[r];
          else pacc[r] = sacc[r] * (pacc[r] - Dq[rq & 1][e]);
          if constexpr ((r & 7) == 7) sf[r >> 3] = pack_frag(pacc, r - 7);
        });
      } else {  // dK^T += Q^T dS
        constexpr int c = k - P1 - P2 - P3;
        dk[c % NI] = mfma32(a, sf[c / NI], dk[c % NI]);
      }
      // operand of slot j + RA (of this tile or, past its end, of the next)
      if constexpr (j + RA < NSLOT) ring[(j + RA) % RING] = operand(std::integral_constant<int, j + RA>{}, st);
      else ring[(j + RA) % RING] = operand(std::integral_constant<int, j + RA - NSLOT>{}, st1);
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  LS_WAIT_VMCNT(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  static_for<RA>([&](auto j_c) { ring[decltype(j_c)::value] = operand(j_c, 0); });
  int st = 0, st1 = 1, st2 = 2;
  for (int t = tbegin; t < ntiles; ++t) {
    tile(t, st, st1, st2);
    const int tmp = st;
    st = st1;
    st1 = st2;
    st2 = tmp;
  }

  // dK = scale * dS^T Q (un-rotated), dV = P^T dO.  Lane holds key kvrow.
  if (kvrow >= S) return;
  if (SPLIT || (PACKED && parts > 1)) {  // this workgroup's partial sums; lane holds columns 32i + 8(r/4) + 4lh + r%4
    float* row = part;
    if constexpr (SPLIT) row += (((int64_t)hs * sh.batch * sh.seq + row0 + kvrow) * nkv + kvh) * (2 * D);
    else row += (((int64_t)slot + part_no) * nkv + kvh) * (PACKED_ROWS * 2 * D) + (32 * wave + lr) * (2 * D);
    store_sums<D>(row, dk, dv, lh);
  } else {
    unrotate_store<D>(dk, scale, rope_cs, S, kvrow, lh, dqkv + (row0 + kvrow) * ld + (nq + kvh) * hd, hd);
    unrotate_store<D>(dv, 1.0f, nullptr, S, kvrow, lh, dqkv + (row0 + kvrow) * ld + (nq + nkv + kvh) * hd, hd);
  }
}

template <int D, bool SPLIT, bool PACKED, class SC>
__global__ __launch_bounds__(256, PACKED && D == 64 ? 2 : 1) void attn_bwd_dkdv_kernel(AttnShape sh, PackedView pk,
                                                                const bf16_t* __restrict__ qkv,
                                                                const bf16_t* __restrict__ dout,
                                                                const float* __restrict__ lse2,
                                                                const float* __restrict__ Dv, bf16_t* __restrict__ dqkv,
                                                                const float* __restrict__ rope_cs, float scale,
                                                                float sl2, int hsplit, float* __restrict__ part, SC sc) {
  __shared__ __attribute__((aligned(1024))) DkdvStage<D> stg[DKDV_STAGES];
  dkdv_tile<D, SPLIT, PACKED>(sh, sc, pk, PACKED ? packed_wg() : (int)blockIdx.x, stg, qkv, dout, lse2, Dv, dqkv,
                              rope_cs, scale, sl2, hsplit, part);
}

// dK and dV of 32 rows of a packed key tile, if its work was cut into parts, and one kv
// head: the parts' sums added in their order, scaled and rounded.  Workgroup x of
// packed_joins takes quarter x % 4 of tile x / 4 / nkv, a wave 8 rows of it, a
// lane 2D / 64 columns of [dK | dV]; the loads of four parts are in flight together.
__host__ __device__ inline int packed_joins(const PackedView& pk, int nkv) { return packed_max_split(pk) * nkv * 4; }
template <int D>
LS_DEV void join_parts(const AttnShape& sh, const PackedView& pk, int x, const float* __restrict__ part,
                       bf16_t* __restrict__ dqkv, float scale) {
  constexpr int E = 2 * D / 64, ROWS = 8, AHEAD = 4;
  const int nkv = sh.nkv, kvh = (x >> 2) % nkv, tile = (x >> 2) / nkv;
  const PackedHead head = *pk.head;
  const PackedTile t = packed_checked(pk.tiles[tile], sh.seq);  // (one of max_tiles)
  if (tile >= min(packed_count(head.tiles, pk.max_tiles), packed_count(head.split, pk.max_tiles))) return;
  const int parts = __builtin_amdgcn_readfirstlane((int)t.parts), slot = __builtin_amdgcn_readfirstlane((int)t.slot);
  if (t.len == 0 || parts < 2 || slot + parts > pk.max_slots) return;
  const int kv0 = ((t.len - 1) / BWD_BKV - t.rank) * BWD_BKV;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c0 = E * lane;
  typedef float fE __attribute__((ext_vector_type(E)));
  const int hd = sh.d;
  const int64_t ld = (int64_t)(sh.nq + 2 * nkv) * hd, step = (int64_t)nkv * (PACKED_ROWS * 2 * D);
  const bool is_k = c0 < D;
  const int col = is_k ? c0 : c0 - D;
  const float c = is_k ? scale : 1.0f;
  const float* src = part + ((int64_t)slot * nkv + kvh) * (PACKED_ROWS * 2 * D) + c0;
  bf16_t* dst = dqkv + (t.start + (int64_t)kv0) * ld + (int64_t)(sh.nq + (is_k ? 0 : nkv) + kvh) * hd + col;
  const int r0 = 32 * (x & 3) + ROWS * wave;
  if (kv0 + r0 >= t.len) return;
  fE v[ROWS], u[AHEAD][ROWS];
#pragma unroll
  for (int k = 0; k < ROWS; ++k) v[k] = fE{};
  // (rows past the end of the sequence are in the slot, unwritten, and go nowhere)
  for (int p = 0; p < parts; p += AHEAD) {
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
#pragma unroll
      for (int k = 0; k < ROWS; ++k) u[a][k] = *(const fE*)(src + min(p + a, parts - 1) * step + (r0 + k) * (2 * D));
    __builtin_amdgcn_sched_barrier(0);  // all of them before the first is waited for
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
      if (p + a < parts) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) v[k] += u[a][k];
      }
  }
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    if (kv0 + r0 + k >= t.len || col >= hd) break;
    bf16_t* y = dst + (r0 + k) * ld;
    if constexpr (E == 4) *(u32x2*)y = u32x2{pack_bf2(v[k][0] * c, v[k][1] * c), pack_bf2(v[k][2] * c, v[k][3] * c)};
    else *(uint32_t*)y = pack_bf2(v[k][0] * c, v[k][1] * c);
  }
}

// Sum of the hsplit partial dK / dV rows of attn_bwd_dkdv_kernel, in split
// order, then scale and inverse RoPE for dK, bf16 stores into dqkv.  One wave
// per (token, kv head): lane l holds columns 4l .. 4l+3 of [dK | dV] (D = 128)
// or 2l .. 2l+1 (D = 64); the RoPE partner of dK column c < D/2 is c + D/2.
template <int D>
__global__ __launch_bounds__(256) void attn_bwd_dkdv_reduce(AttnShape sh, int hsplit, const float* __restrict__ part,
                                                            bf16_t* __restrict__ dqkv, const float* __restrict__ rope_cs,
                                                            float scale) {
  constexpr int E = 2 * D / 64;  // columns per lane
  constexpr int HALF = D / 2;
  const int lane = threadIdx.x & 63;
  const int64_t T = (int64_t)sh.batch * sh.seq;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);  // (token, kv head)
  if (w >= T * sh.nkv) return;
  const int64_t t = w / sh.nkv;
  const int kvh = (int)(w % sh.nkv), pos = (int)(t % sh.seq);
  const int c0 = E * lane;  // first of this lane's columns in [dK | dV]
  float v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = 0.f;
  for (int hs = 0; hs < hsplit; ++hs) {
    const float* src = part + ((int64_t)hs * T * sh.nkv + w) * (2 * D) + c0;
    if constexpr (E == 4) {
      const f32x4 a = *(const f32x4*)src;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += a[e];
    } else {
      const float2 a = *(const float2*)src;
      v[0] += a.x;
      v[1] += a.y;
    }
  }
  const bool is_k = c0 < D;
  // partner columns of dK (c0 +- D/2): lanes HALF/E apart
  float pv[E];
#pragma unroll
  for (int e = 0; e < E; ++e) pv[e] = __shfl_xor(v[e], HALF / E);
  const int64_t ld = (int64_t)(sh.nq + 2 * sh.nkv) * D;
  bf16_t* row = dqkv + t * ld + (int64_t)(sh.nq + (is_k ? 0 : sh.nkv) + kvh) * D;
  const int d0 = is_k ? c0 : c0 - D;
  float out[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (!is_k) {
      out[e] = v[e];
    } else if (!rope_cs) {
      out[e] = v[e] * scale;
    } else {
      const int d = d0 + e, i = d % HALF;
      const float cs = rope_cs[(int64_t)pos * HALF + i];
      const float sn = rope_cs[(int64_t)sh.seq * HALF + (int64_t)pos * HALF + i];
      // inverse rotation: x1' = x1 cos + x2 sin, x2' = x2 cos - x1 sin
      out[e] = d < HALF ? (v[e] * cs + pv[e] * sn) * scale : (v[e] * cs - pv[e] * sn) * scale;
    }
  }
  if constexpr (E == 4) *(u32x2*)(row + d0) = u32x2{pack_bf2(out[0], out[1]), pack_bf2(out[2], out[3])};
  else *(uint32_t*)(row + d0) = pack_bf2(out[0], out[1]);
}

// dQ for 128 queries of one head (4 waves x 32 queries): loops over the key
// tiles up to the diagonal, recomputes S^T and dP^T with keys as MFMA rows (a
// lane owns one query, as in the forward), forms dS^T in registers and
// accumulates dQ^T += K^T dS^T.
//
// Per 64-key tile a wave issues one MFMA per slot: S^T and dP^T of key block 0,
// then of key block 1, then dQ^T for block 0 and for block 1.  The softmax work
// of block 0 (P = exp2(S - LSE), dS = P (dP - D), bf16 operands) runs between
// the MFMAs of block 1's S^T and dP^T, that of block 1 between the MFMAs of
// block 0's dQ^T.  MFMA operands from LDS are read RA slots ahead into a ring
// of registers within the tile; two workgroups per compute unit keep the
// matrix cores busy across tile boundaries and while one wave waits.
template <int D, bool PACKED, class SC>
LS_DEV void dq_tile(const AttnShape& sh, const SC& sc, const QTile& qtile, bf16_t (&Ks)[2][BKV * D],
                    bf16_t (&Vs)[2][BKV * D], const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ dout,
                    const float* __restrict__ lse2, const float* __restrict__ Dv, bf16_t* __restrict__ dqkv,
                    const float* __restrict__ rope_cs, float scale, float sl2) {
  constexpr int NSD = D / 16, NI = D / 32;
  constexpr int PS = 2 * NSD;                // slots of one block's S^T and dP^T (interleaved)
  constexpr int PQ = 2 * NI;                 // slots of one block's dQ^T
  constexpr int NSLOT = 2 * PS + 2 * PQ;
  constexpr int RING = 2, RA = RING - 1;
  static_assert(NSLOT % RING == 0 && 16 % PS == 0 && 16 % PQ == 0, "slot counts");
  const int nq = sh.nq, nkv = sh.nkv;
  const int S = qtile.S, h = qtile.h, kvh = h / (nq / nkv), hd = PACKED ? sh.d : D;
  const int64_t ld = (int64_t)(nq + 2 * nkv) * hd;
  const int64_t ldo = (int64_t)nq * hd;
  const bf16_t* base = qkv + qtile.row0 * ld;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int q0 = qtile.qt * BQ;
  const int qrow = q0 + 32 * wave + lr;
  const bool qok = qrow < S;
  const int kcol = (nq + kvh) * hd, vcol = (nq + nkv + kvh) * hd;

  const int kv_end = min(S, q0 + BQ);
  const int nkt = (kv_end + BKV - 1) / BKV;
  const int kt0 = first_key_tile(sc, q0);
  const TileLoader<D, BKV> tl(ld, wave, lane, hd);
  tl(base, ld, SC::ON ? kt0 * BKV : 0, S, kcol, Ks[0], wave);
  tl(base, ld, SC::ON ? kt0 * BKV : 0, S, vcol, Vs[0], wave);

  u32x4 qf[NSD], df[NSD];
#pragma unroll
  for (int s = 0; s < NSD; ++s) {
    const bool ok = qok && 16 * s + 8 * lh < hd;
    qf[s] = ok ? load16(base + (int64_t)qrow * ld + h * hd + 16 * s + 8 * lh) : u32x4{0u, 0u, 0u, 0u};
    df[s] = ok ? load16(dout + (qtile.row0 + qrow) * ldo + h * hd + 16 * s + 8 * lh) : u32x4{0u, 0u, 0u, 0u};
  }
  const float L2 = qok ? lse2[qtile.vec0 + qrow] : 0.f;
  const float Dq = qok ? Dv[qtile.vec0 + qrow] : 0.f;  // (modified scores: -D)

  f32x16 dq[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[i][r] = 0.f;

  // operand reads by per-lane LDS address (K and V rows, K^T columns); the
  // stage, the array, the 32-key block and the 16-key step add constants
  const FragAddr<D> fa(lds_offset(&Ks[0][0]), lane);
  constexpr uint32_t STAGE = BKV * D * 2;
  const uint32_t v_minus_k = lds_offset(&Vs[0][0]) - lds_offset(&Ks[0][0]);

  // MFMA A operand of slot j of the tile in stage ST.
  auto operand = [&](auto j_c, auto st_c) -> u32x4 {
    constexpr int j = decltype(j_c)::value, st = decltype(st_c)::value;
    if constexpr (j < 2 * PS) {  // rows of K (k even) or V (k odd)
      constexpr int bb = j / PS, k = j % PS;
      return fa.rows(k >> 1, st * STAGE + bb * 32 * D * 2 + ((k & 1) ? v_minus_k : 0u));
    } else {  // K^T columns
      constexpr int bb = (j - 2 * PS) / PQ, c = (j - 2 * PS) % PQ;
      return fa.cols(c % NI, st * STAGE + (2 * bb + c / NI) * 16 * D * 2);
    }
  };

  u32x4 ring[RING];
  f32x16 sacc[2], pacc[2];
  u32x4 sf[2][2];
  // causal mask: element r of key block bb is key kv0 + 4lh + c with
  // c = 32bb + 8(r/4) + r%4, kept when c <= hi, i.e. key <= qrow.  Keys past the
  // end of the sequence need no mask beyond that: their K and V read as zero.
  // Modified scores, with a window's two borders, are masked on the tiles only that have a key which
  // some query of the wave does not see (`edge`): 8135 rows of 24/8 heads of 128, cap 30, dQ 264 -> 251 us; plain ones, one
  // comparison and select each, are no faster so.
  auto soft = [&](auto bb_c, auto r_c, int hi, bool edge) {
    constexpr int bb = decltype(bb_c)::value, r = decltype(r_c)::value;
    constexpr int c0 = 32 * bb + 8 * (r >> 2) + (r & 3);
    float w;
    float p = prob_slope(sc, sacc[bb][r], sl2, L2, w);
    if constexpr (SC::CAPPED) p *= w;
    if constexpr (!SC::ON) {
      if (c0 > hi) p = 0.f;
    }
    pacc[bb][r] = SC::ON ? p * (pacc[bb][r] + Dq) : p * (pacc[bb][r] - Dq);
    if constexpr ((r & 7) == 7) {
      if constexpr (SC::ON) {
        if (edge) {
          asm volatile("");  // keeps the block a branch rather than selects on every tile
#pragma unroll
          for (int u = r - 7; u <= r; ++u) {
            const int c = 32 * bb + 8 * (u >> 2) + (u & 3);
            if (c > hi || c <= hi - sc.window) pacc[bb][u] = 0.f;
          }
        }
      }
      sf[bb][r >> 3] = pack_frag(pacc[bb], r - 7);
    }
  };

  sync_lds();
  // one 64-key tile in stage CUR (a constant: the loop below runs two per pass)
  auto step = [&](auto cur_c, int kt) {
    constexpr int cur = decltype(cur_c)::value;
    const int kv0 = kt * BKV;
    if (kt + 1 < nkt) {
      tl(base, ld, kv0 + BKV, S, kcol, Ks[cur ^ 1], wave);
      tl(base, ld, kv0 + BKV, S, vcol, Vs[cur ^ 1], wave);
    }
    const int hi = qrow - kv0 - 4 * lh, wave_qmin = q0 + 32 * wave;
    bool edge = kv0 + BKV - 1 > wave_qmin;
    if constexpr (SC::ON) edge = edge || kv0 <= wave_qmin + 31 - sc.window;
    static_for<RA>([&](auto j_c) { ring[decltype(j_c)::value] = operand(j_c, cur_c); });
    static_for<NSLOT>([&](auto j_c) {
      constexpr int j = decltype(j_c)::value;
      __builtin_amdgcn_sched_barrier(0);
      const u32x4 a = ring[j % RING];
      if constexpr (j < 2 * PS) {
        constexpr int bb = j / PS, k = j % PS, s = k >> 1;
        if constexpr (k & 1) pacc[bb] = mfma32(a, df[s], s == 0 ? f32x16{} : pacc[bb]);
        else sacc[bb] = mfma32(a, qf[s], s == 0 ? f32x16{} : sacc[bb]);
        if constexpr (bb == 1) {  // softmax of block 0
          constexpr int PER = 16 / PS;
          static_for<PER>([&](auto u) {
            soft(std::integral_constant<int, 0>{}, std::integral_constant<int, k * PER + decltype(u)::value>{}, hi, edge);
          });
        }
      } else {
        constexpr int bb = (j - 2 * PS) / PQ, c = (j - 2 * PS) % PQ;
        dq[c % NI] = mfma32(a, sf[bb][c / NI], dq[c % NI]);
        if constexpr (bb == 0) {  // softmax of block 1
          constexpr int PER = 16 / PQ;
          static_for<PER>([&](auto u) {
            soft(std::integral_constant<int, 1>{}, std::integral_constant<int, c * PER + decltype(u)::value>{}, hi, edge);
          });
        }
      }
      if constexpr (j + RA < NSLOT) ring[(j + RA) % RING] = operand(std::integral_constant<int, j + RA>{}, cur_c);
      __builtin_amdgcn_sched_barrier(0);
    });
    sync_lds();
  };
  for (int kt = SC::ON ? kt0 : 0; kt < nkt; kt += 2) {
    step(std::integral_constant<int, 0>{}, kt);
    if (kt + 1 < nkt) step(std::integral_constant<int, 1>{}, kt + 1);
  }
  if (!qok) return;
  unrotate_store<D>(dq, scale, rope_cs, S, qrow, lh, dqkv + (qtile.row0 + qrow) * ld + h * hd, hd);
}

template <int D, bool PACKED, class SC>
__global__ __launch_bounds__(256, 2) void attn_bwd_dq_kernel(AttnShape sh, PackedView pk,
                                                              const bf16_t* __restrict__ qkv,
                                                              const bf16_t* __restrict__ dout,
                                                              const float* __restrict__ lse2,
                                                              const float* __restrict__ Dv, bf16_t* __restrict__ dqkv,
                                                              const float* __restrict__ rope_cs, float scale,
                                                              float sl2, const float* __restrict__ part, SC sc) {
  __shared__ __attribute__((aligned(1024))) bf16_t Ks[2][BKV * D];
  __shared__ __attribute__((aligned(1024))) bf16_t Vs[2][BKV * D];
  QTile qtile;
  if constexpr (PACKED) {
    // the last workgroups finish dK and dV; short sequences have their dQ already
    const int x = (int)blockIdx.x, joins = x - pk.max_tiles * sh.nq;
    if (joins >= 0) {
      join_parts<D>(sh, pk, joins, part, dqkv, scale);
      return;
    }
    PackedTile t;
    if (!packed_unit(pk, x / sh.nq, sh.seq, t) || t.len <= PACKED_MID) return;
    qtile = q_tile(sh, t, packed_head(x % sh.nq, sh.nq, sh.nkv));
  } else {
    qtile = q_tile(sh);
  }
  dq_tile<D, PACKED>(sh, sc, qtile, Ks, Vs, qkv, dout, lse2, Dv, dqkv, rope_cs, scale, sl2);
}

// dK/dV and dQ of packed sequences in one launch, for batches whose launches one after
// the other would each leave compute units idle behind their longest tiles
// (packed_one_launch).  The pieces of dK/dV come first, then the query tiles,
// both in order of falling work; the other way round was slower (6 documents on 3000
// rows, 12/4 heads of 64: backward 41 us, this way 39, two launches 47).
template <int D, class SC>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void packed_bwd_kernel(AttnShape sh, PackedView pk,
                                                             const bf16_t* __restrict__ qkv,
                                                             const bf16_t* __restrict__ dout,
                                                             const float* __restrict__ lse2,
                                                             const float* __restrict__ Dv, bf16_t* __restrict__ dqkv,
                                                             float scale, float sl2, float* __restrict__ part,
                                                             int pieces, SC sc) {
  union Lds {
    DkdvStage<D> stg[DKDV_STAGES];
    struct {
      bf16_t k[2][BKV * D], v[2][BKV * D];
    } dq;
  };
  __shared__ __attribute__((aligned(1024))) char lds[sizeof(Lds)];
  Lds& m = *(Lds*)lds;
  const int x = (int)blockIdx.x;
  if (x < pieces) {
    dkdv_tile<D, false, true>(sh, sc, pk, x, m.stg, qkv, dout, lse2, Dv, dqkv, nullptr, scale, sl2, 1, part);
    return;
  }
  PackedTile t;
  if (!packed_unit(pk, (x - pieces) / sh.nq, sh.seq, t) || t.len <= PACKED_MID) return;  // (small ones have their dQ)
  dq_tile<D, true>(sh, sc, q_tile(sh, t, packed_head((x - pieces) % sh.nq, sh.nq, sh.nkv)), m.dq.k, m.dq.v, qkv, dout, lse2,
                   Dv, dqkv, nullptr, scale, sl2);
}

template <int D>
__global__ __launch_bounds__(256) void packed_join_kernel(AttnShape sh, PackedView pk, bf16_t* __restrict__ dqkv,
                                                          float scale, const float* __restrict__ part) {
  join_parts<D>(sh, pk, (int)blockIdx.x, part, dqkv, scale);
}

template <int D, bool PACKED, class SC = PlainScore>
hipError_t attn_fwd_t(const AttnShape& sh, const PackedView& pk, const bf16_t* qkv, bf16_t* o, float* lse,
                      hipStream_t s, const SC& sc = {}, float own_scale = 0.f) {
  const dim3 grid = PACKED ? packed_grid((int64_t)pk.max_units * sh.nq)
                           : dim3((unsigned)((sh.seq + BQ - 1) / BQ) * sh.nq * sh.batch);
  const float sl2 = SC::ON ? LOG2E * own_scale
                           : LOG2E / sqrtf((float)(PACKED ? sh.d : sh.d_scale > 0 ? sh.d_scale : D));
  hipLaunchKernelGGL((attn_fwd_kernel<D, PACKED, SC>), grid, dim3(256), 0, s, sh, pk, qkv, o, lse, sl2, sc);
  return hipGetLastError();
}

// Bytes of the backward workspace before the partial sums: D, then the base-2 log-sum-exp.
// In whole 256 bytes: the sums are stored and read as 16-byte vectors.
int64_t bwd_ws_head(const AttnShape& sh) {
  return (2 * (int64_t)sh.batch * sh.seq * sh.nq * (int64_t)sizeof(float) + 255) & ~(int64_t)255;
}

// Whether dK/dV and dQ go into one launch (and the joining of parts into one behind it): up to
// four query tiles to a compute unit.  Backward, one launch against two, at query
// tiles times heads of (heads of 64) 348: 39 / 47 us, 704: 45 / 53, 1280: 91 / 93,
// short documents of 3040: 62 / 58; (of 128, where one launch leaves dQ one
// workgroup to a compute unit instead of two) 320: 71 / 82, 600: 209 / 227, 1824: 261 / 251.
bool packed_one_launch(const AttnShape& sh, const PackedView& pk) { return (int64_t)pk.max_tiles * sh.nq <= 4 * PACKED_CUS; }

// own_scale: of a ModScore, what q.k is multiplied with before the cap.
template <int D, class SC = PlainScore>
hipError_t packed_attn_bwd_t(const AttnShape& sh, const PackedView& pk, const bf16_t* qkv, const bf16_t* o,
                             const float* lse, const bf16_t* dout, bf16_t* dqkv, void* ws, hipStream_t s,
                             const SC& sc = {}, float own_scale = 0.f) {
  const int64_t T = sh.seq;
  float* Dv = (float*)ws;
  float* lse2 = Dv + T * sh.nq;
  float* part = (float*)((char*)ws + bwd_ws_head(sh));
  const bf16_t* rest = nullptr;
  if constexpr (SC::ON) rest = sc.rest;
  if (SC::ON && rest)
    hipLaunchKernelGGL((attn_bwd_pre_kernel<D, true, SC::ON>), packed_grid((T + 3) / 4), dim3(256), 0, s, sh, o, dout, lse,
                       Dv, lse2, rest, SC::ON, sc.c2);
  else
    hipLaunchKernelGGL((attn_bwd_pre_kernel<D, true>), packed_grid((T + 3) / 4), dim3(256), 0, s, sh, o, dout, lse, Dv,
                       lse2, rest, SC::ON, sc.c2);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const float qk = SC::ON ? own_scale : 1.0f / sqrtf((float)sh.d), sl2 = qk * LOG2E;
  const float scale = SC::CAPPED ? 4.0f * qk : qk;  // (dS holds a quarter of the cap's slope)
  const unsigned gkv = (unsigned)(pk.max_units + pk.max_items - pk.max_tiles) * sh.nkv;
  if (packed_one_launch(sh, pk)) {
    hipLaunchKernelGGL((packed_bwd_kernel<D, SC>), dim3(gkv + (unsigned)pk.max_tiles * sh.nq), dim3(256), 0, s, sh, pk,
                       qkv, dout, (const float*)lse2, (const float*)Dv, dqkv, scale, sl2, part, (int)gkv, sc);
    e = hipGetLastError();
    const int joins = packed_joins(pk, sh.nkv);  // 0 with more than 2 PACKED_CUS kv heads, which cut no tile
    if (e != hipSuccess || joins == 0) return e;
    hipLaunchKernelGGL((packed_join_kernel<D>), dim3((unsigned)joins), dim3(256), 0, s, sh, pk, dqkv, scale,
                       (const float*)part);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((attn_bwd_dkdv_kernel<D, false, true, SC>), packed_grid(gkv), dim3(256), 0, s, sh, pk, qkv, dout,
                     (const float*)lse2, (const float*)Dv, dqkv, (const float*)nullptr, scale, sl2, 1, part, sc);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (one dimension's worth of tiles has more rows than the card's memory holds)
  const unsigned gq = (unsigned)packed_joins(pk, sh.nkv) + (unsigned)pk.max_tiles * sh.nq;
  hipLaunchKernelGGL((attn_bwd_dq_kernel<D, true, SC>), dim3(gq), dim3(256), 0, s, sh, pk, qkv, dout,
                     (const float*)lse2, (const float*)Dv, dqkv, (const float*)nullptr, scale, sl2, (const float*)part,
                     sc);
  return hipGetLastError();
}

AttnShape packed_shape(const PackedShape& p) { return AttnShape{1, (int)p.total, p.nq, p.nkv, p.d}; }

}  // namespace

}  // namespace ls

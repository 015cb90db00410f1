// Internal launch interface between the C ABI layer and the HIP kernels.
// Every launcher enqueues work on `stream` and returns the launch status.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ls {

typedef uint16_t bf16_t;

// ---- matrix products --------------------------------------------------------
// C[m,n] = sum_k A(m,k) B(k,n), bf16 operands, fp32 accumulation.
// A: a_kcontig ? A[m*lda + k] : A[k*lda + m].
// B: b_kcontig ? row n of B (element k contiguous) : row k of B (element n contiguous).
//    The rows of B may come from up to three buffers: row index r (n if
//    b_kcontig, else k) reads seg[s] for the last s with start[s] <= r, at row
//    r - start[s] of that buffer.
// With glu set (b_kcontig only), virtual column n maps to gate row (n/128)*64 + n%64
// when (n/64) is even and to the up row with the same index when odd (seg[0] =
// gate, seg[1] = up, glu_rows = rows of each).
enum Epilogue {
  EPI_BF16 = 0,     // C (bf16) = acc
  EPI_RESID = 1,    // C (bf16) = acc + R
  EPI_ROPE = 2,     // C (bf16) = rotate(acc) on columns < rope_cols, acc elsewhere
  EPI_GLU_FWD = 3,  // gu[m][i] = g, gu[m][I+i] = u (C; skipped when null), act[m][i] = silu(g) u
  EPI_GLU_BWD = 4,  // C = dgu: dgu[m][i] = acc u silu'(g), dgu[m][I+i] = acc silu(g)
  EPI_F32 = 5,      // F (fp32, rows split over up to three buffers) (+)= acc
  EPI_PART = 6,     // kpart[slice] = acc: a slice of a split K (256 x 256 tiles; set by gemm())
  EPI_LSE = 7,      // acc are logits: maximum and sum of exponentials per row and column block, target logits
  EPI_DZ = 8,       // C (bf16) = softmax(acc) - onehot
  EPI_DH = 9,       // F (fp32) (+)= acc
  EPI_DE = 10,      // F (fp32) (+)= coef acc
  EPI_DE16 = 11,    // C (bf16) = coef acc
  EPI_STAT = 12,    // acc are logits: as EPI_LSE with what the entropy needs, and the largest of every 8 columns
  EPI_DLP = 13,     // C (bf16) = gradient of log probability and entropy for the scaled logits, over a common factor
};

struct GemmArgs {
  int M = 0, N = 0, K = 0;
  const bf16_t* A = nullptr;
  int64_t lda = 0;
  bool a_kcontig = true;
  const bf16_t* B[3] = {nullptr, nullptr, nullptr};
  int b_start[3] = {0, 1 << 30, 1 << 30};
  int64_t ldb = 0;
  bool b_kcontig = true;
  bool glu = false;
  int glu_rows = 0;
  int epi = EPI_BF16;
  bf16_t* C = nullptr;
  int64_t ldc = 0;
  const bf16_t* R = nullptr;      // EPI_RESID, leading dimension ldc
  const float* rope_cs = nullptr; // EPI_ROPE: [seq][head_dim/2] cos then [seq][head_dim/2] sin
  int seq = 1, head_dim = 128, rope_cols = 0;
  bf16_t* act = nullptr;          // EPI_GLU_FWD: [M][I]
  const bf16_t* gu_in = nullptr;  // EPI_GLU_BWD: saved [M][2I]
  int glu_I = 0;
  float* F[3] = {nullptr, nullptr, nullptr};  // EPI_F32; EPI_DH, EPI_DE: F[0]
  int f_start[3] = {0, 1 << 30, 1 << 30};
  int64_t ldf = 0;
  int accumulate = 0;
  // EPI_LSE and EPI_DZ: columns are entries col0 .. col0 + N - 1 of a vocabulary, row m has target[m] (-1: none)
  int col0 = 0, vocab = 0;
  const int32_t* target = nullptr;
  // EPI_LSE: [column block][M] (max, sum of exp(z - max)); two blocks per tile column.  EPI_STAT: [column block][M]
  // (m = max of the scaled logits in base 2, sum of 2^(z - m), sum of (z - m) 2^(z - m), 0)
  float* stats = nullptr;
  float* zt = nullptr;          // EPI_LSE: [M], the logit of a row's target where this product has it
  const float* lse = nullptr;   // EPI_DZ: [M]
  const float* coef = nullptr;  // EPI_DE, EPI_DE16: one factor of the results (on the device)
  // The token rows that count, on the device, at most as many as the host says: rows of C (M) of EPI_DZ and
  // EPI_DH, the depth K of EPI_DE and EPI_DE16.
  const int* rows = nullptr;
  // fp32 workspace for splitting K over workgroups when the output tiles alone
  // would leave compute units idle (slices * M * N floats, one slice fewer for
  // EPI_F32, see gemm_kpart_floats); null or smaller means fewer slices or none.
  float* kpart = nullptr;
  int64_t kpart_floats = 0;
  int ksplit = 1;   // slices of K (set by gemm())
  int fill = 0;     // EPI_DH: workgroups that its slices may fill when the rows are few (set by gemm())
  int group_m = 8;  // tile rows per group of the launch order (set by the launch)
  // EPI_STAT and EPI_DLP: what a logit is multiplied with, times log2(e)
  float scale2 = 0.f;
  float* gmax = nullptr;  // EPI_STAT: null, or the largest logit of every 8 columns of the vocabulary, at gmax_at
  int gmax_groups = 0, gmax_rows = 0;
  // EPI_DLP: the rows' gradients of log probability and entropy, the entropy [M], and the common factor (one)
  const float* dlogp = nullptr;
  const float* dent = nullptr;
  const float* ent = nullptr;
  const float* cmax = nullptr;
};

// The workgroup tile and the slices of K of a launch.
struct GemmPlan {
  int bm = 256, bn = 256, ks = 1;
  bool deep = true;  // 128 x 128: four LDS stages, one workgroup per CU; else two and two
  int stages() const { return bn != 128 ? 2 : bm == 256 ? 3 : deep ? 4 : 2; }
};
// What gemm() chooses with kpart_floats of scratch (and the forced shape, if any).
GemmPlan gemm_plan(const GemmArgs& a, int64_t kpart_floats);
// The same without scratch and whatever shape is forced; a forced one has no narrower columns.
GemmPlan gemm_plan_free(const GemmArgs& a);
// `used`, if given, gets the choice.
hipError_t gemm(const GemmArgs& a, hipStream_t s, GemmPlan* used = nullptr);
// Floats of GemmArgs::kpart with which a product of this shape and epilogue
// runs with its full split of K (0: it is not split).
int64_t gemm_kpart_floats(const GemmArgs& a);
// The launches behind gemm(), one per operand layout: a tile shape the epilogue
// has, with a.ksplit and a.group_m set.  TILE_256x128: three LDS stages;
// TILE_128_DEEP: four, one workgroup per CU; TILE_128: two stages, two
// workgroups per CU.
enum GemmTile { TILE_256, TILE_256x192, TILE_192x256, TILE_192, TILE_256x128, TILE_128, TILE_128_DEEP };
hipError_t gemm_nt(const GemmArgs& a, GemmTile t, hipStream_t s);
hipError_t gemm_nn(const GemmArgs& a, GemmTile t, hipStream_t s);
hipError_t gemm_tn(const GemmArgs& a, GemmTile t, hipStream_t s);
hipError_t gemm_head(const GemmArgs& a, GemmTile t, hipStream_t s);  // the instances that only the head loss uses
hipError_t gemm_logprob(const GemmArgs& a, GemmTile t, hipStream_t s);  // EPI_STAT, EPI_DLP
// Force the tile shape of later gemm launches (bm, bn in {256, 192}; 0, 0 =
// automatic).  Variants that only exist as 256 x 256 ignore it.  -1 on bad sizes.
int gemm_tile_override(int bm, int bn);

// ---- RMSNorm ------------------------------------------------------------------
hipError_t rmsnorm_fwd(int64_t rows, int hidden, float eps, const bf16_t* x, const bf16_t* gamma,
                       bf16_t* h, float* r, hipStream_t s);
// Partial buffer of rmsnorm_bwd: rmsnorm_bwd_parts(rows, hidden) x hidden floats.
int rmsnorm_bwd_parts(int64_t rows, int hidden);
hipError_t rmsnorm_bwd(int64_t rows, int hidden, const bf16_t* x, const bf16_t* gamma, const float* r,
                       const bf16_t* dh, const bf16_t* dres, bf16_t* dx, float* dgamma, int accumulate,
                       float* partial, hipStream_t s);

// ---- RoPE table -------------------------------------------------------------
// cs[p][i] = cos(p theta^(-2i/d)), cs[seq*t/2 + p*t/2 + i] = sin(...), computed in
// fp64, for a table of t/2 entries per position (t = table_dim, 0 = head_dim);
// entries i >= head_dim/2 of a wider table are cos 1, sin 0.
hipError_t rope_table(int seq, int head_dim, double theta, float* cs, hipStream_t s, int table_dim = 0);

// ---- attention ----------------------------------------------------------------
struct AttnShape {
  int batch, seq, nq, nkv, d;
  int d_scale = 0;  // features per head behind the softmax scale 1/sqrt(d_scale) (0: d)
};
hipError_t attn_fwd(const AttnShape& sh, const bf16_t* qkv, bf16_t* o, float* lse, hipStream_t s);
// Workspace for attn_bwd: D and the base-2 log-sum-exp, [batch*nq*seq] fp32 each.
size_t attn_bwd_workspace(const AttnShape& sh);
// rope_cs may be null (no inverse rotation of dq and dk).
hipError_t attn_bwd(const AttnShape& sh, const bf16_t* qkv, const bf16_t* o, const float* lse,
                    const bf16_t* dout, bf16_t* dqkv, const float* rope_cs, void* ws, hipStream_t s);

// ---- packed sequences -------------------------------------------------------------
// `total` rows hold n_seqs sequences end to end; see packed.h for the plan.
constexpr int PACKED_ROWS = 128;  // rows of a tile of the plan (query and key tiles of the attention kernels)
constexpr int PACKED_SHORT = 32;  // sequences of up to so many rows are one wave's work each
struct PackedShape {
  int64_t total;
  int n_seqs, nq, nkv, d;
};
size_t packed_plan_bytes(const PackedShape& p);
hipError_t packed_plan(const PackedShape& p, const int32_t* cu, void* plan, hipStream_t s);
// dst = q and k of src turned (v copied unless dst == src); rows of no sequence are left alone.
hipError_t packed_rope(const PackedShape& p, const void* plan, double theta, int inverse, const bf16_t* src,
                       bf16_t* dst, hipStream_t s);
// dst = q and k of src normed per head (gains gq, gk of d features) and turned (v copied unless dst == src).
hipError_t packed_qk_norm_rope(const PackedShape& p, const void* plan, double theta, float eps, const bf16_t* gq,
                               const bf16_t* gk, const bf16_t* src, bf16_t* dst, hipStream_t s);
// dx = its gradient for src, from dy (may be dx); dgq and dgk (either may be null) (+)= those of the gains.
size_t packed_qk_norm_rope_bwd_workspace(const PackedShape& p);
hipError_t packed_qk_norm_rope_bwd(const PackedShape& p, const void* plan, double theta, float eps, const bf16_t* gq,
                                   const bf16_t* gk, const bf16_t* src, const bf16_t* dy, bf16_t* dx, float* dgq,
                                   float* dgk, int accumulate, void* ws, hipStream_t s);
hipError_t packed_attn_fwd(const PackedShape& p, const void* plan, const bf16_t* qkv, bf16_t* o, float* lse,
                           hipStream_t s);
size_t packed_attn_bwd_workspace(const PackedShape& p);
hipError_t packed_attn_bwd(const PackedShape& p, const void* plan, const bf16_t* qkv, const bf16_t* o, const float* lse,
                           const bf16_t* dout, bf16_t* dqkv, void* ws, hipStream_t s);

// The same attention with scores cap tanh(scale q.k / cap) (cap 0: scale q.k) over the last `window` positions
// (1 .. total); workspace: packed_attn_bwd_workspace.
// rest: null, or what rounding o to bf16 left, in bf16 (an output of the forward call).
struct ScoreShape {
  float scale, cap;
  int window;
  bf16_t* rest = nullptr;
};
hipError_t packed_score_attn_fwd(const PackedShape& p, const ScoreShape& c, const void* plan, const bf16_t* qkv,
                                 bf16_t* o, float* lse, hipStream_t s);
hipError_t packed_score_attn_bwd(const PackedShape& p, const ScoreShape& c, const void* plan, const bf16_t* qkv,
                                 const bf16_t* o, const float* lse, const bf16_t* dout, bf16_t* dqkv, void* ws,
                                 hipStream_t s);

// ---- padded head layout (64 < d < 128 held in 128-wide slots) -------------------
// Feature s of a head sits at slot s (s < d/2) or dp/2 + s - d/2; other slots are zero.
hipError_t pad_head_rows(const bf16_t* src, bf16_t* dst, int heads, int d, int dp, int cols, hipStream_t s);
hipError_t pad_head_cols(const bf16_t* src, bf16_t* dst, int rows, int heads, int d, int dp, hipStream_t s);
hipError_t unpad_head_rows(const float* src, float* dst, int heads, int d, int dp, int cols, int accumulate,
                           hipStream_t s);
hipError_t unpad_head_cols(const float* src, float* dst, int rows, int heads, int d, int dp, int accumulate,
                           hipStream_t s);

// ---- token embedding and cross-entropy ------------------------------------------
// x[t] = E[ids[t]] ([T, H] bf16); an id outside [0, V) gives a NaN row.
hipError_t embed_fwd(int64_t T, int H, int V, const int32_t* ids, const bf16_t* E, bf16_t* x, hipStream_t s);
// dE[ids[t]] += dx[t], repeated ids summed in token order (deterministic; ids
// outside [0, V) skipped).  H a multiple of 8, at most 8192.
hipError_t embed_bwd(int64_t T, int H, int V, const int32_t* ids, const bf16_t* dx, float* dE, hipStream_t s);
// tg[t] = targets[t], or (targets null) ids[t+1] within a sequence of S tokens
// and -1 at its last position; counts[0] = rows with a target in [0, V).
hipError_t ce_targets(int64_t T, int S, int V, const int32_t* ids, const int32_t* targets, int32_t* tg, int* counts,
                      hipStream_t s);
// Per row of z [rows, V] bf16: row_loss = lse - z[tg]; z <- (softmax - onehot) / max(counts[0], 1).
hipError_t ce_rows(int64_t rows, int V, bf16_t* z, const int32_t* tg, const int* counts, float* row_loss,
                   hipStream_t s);
// loss = sum(row_loss[0 .. T)) / max(counts[0], 1).
hipError_t ce_loss(int64_t T, const float* row_loss, const int* counts, float* loss, hipStream_t s);

// ---- head loss (cross-entropy of h E^T whose logits are not kept) ------------------
// Per row from EPI_LSE's statistics (`blocks` column blocks): lse, row_loss (0 without a target, NaN for one
// outside [-1, V)), and loss = sum(row_loss) / max(rows with a target in [0, V), 1).
hipError_t head_rows(int64_t T, int V, int64_t blocks, const float* stats, const float* zt, const int32_t* targets,
                     float* lse, float* row_loss, float* loss, hipStream_t s);
// The rows that have a target (any but -1), gathered in their order: slot[t] = row t's place among them or -1,
// rows[0] = how many, coef[0] = dloss[0] (null: 1) / max(rows with a target in [0, V), 1), and their h, targets, lse.
hipError_t head_gather(int64_t T, int H, int V, const int32_t* targets, const float* dloss, const bf16_t* h,
                       const float* lse, int32_t* slot, int* rows, float* coef, bf16_t* hc, int32_t* tc, float* lc,
                       hipStream_t s);
// The same with the rows' gradients of log probability and entropy (null: 0) and the entropy, gathered to gc, ec and
// nc; coef[0] = scale c, coef[1] = c, the largest finite |g| or |e| of a row with a target in [0, V).
struct LogprobGrads {
  const float *g, *e, *ent;
  float *gc, *ec, *nc;
  float scale;
};
hipError_t logprob_gather(int64_t T, int H, int V, const int32_t* targets, const LogprobGrads& x, const bf16_t* h,
                          const float* lse, int32_t* slot, int* rows, float* coef, bf16_t* hc, int32_t* tc, float* lc,
                          hipStream_t s);
// dh[t] = coef dhc[slot[t]] rounded to bf16, 0 for a row without a target.
hipError_t head_scatter(int64_t T, int H, const int32_t* slot, const float* coef, const float* dhc, bf16_t* dh,
                        hipStream_t s);

// ---- log probabilities of given tokens -------------------------------------------------
// Per row from EPI_STAT's statistics: lse of the scaled logits; logprob and entropy (both 0 without a target, NaN for
// one outside [-1, V)).
struct LogprobRows {
  int64_t blocks;  // column blocks
  const float *stats, *zt;
  const int32_t* targets;
  float *logprob, *entropy, *lse;
  float scale;
};
hipError_t logprob_rows(int64_t T, int V, const LogprobRows& x, hipStream_t s);
// The same, and the `top` (1 .. 64) largest logits of every row, ties to the lower column, from the largest of every 8
// columns (gmax): ids (-1 past the vocabulary) and scaled logit - lse.
constexpr int LOGPROB_TOP = 64;
// Where a row's maximum of group g lies: blocks of 2^rows rows (16, or as many as there are), in each group by group,
// so that a workgroup that takes 16 rows reads one piece of memory.
__host__ __device__ inline int64_t gmax_at(int groups, int rows, int64_t m, int g) {
  return ((((m >> rows) * groups) + g) << rows) + (m & ((1 << rows) - 1));
}
struct GroupMax {
  const float* v;
  int groups, rows;
};
hipError_t logprob_top(int64_t T, int H, int V, int top, const LogprobRows& x, const bf16_t* h, const bf16_t* embed,
                       const GroupMax& gmax, int32_t* ids, float* logprob, hipStream_t s);

// ---- gradients of many tensors ------------------------------------------------------
constexpr int GN_TENSORS = 96;  // tensors that one launch takes
struct GradTensor {
  void* p;
  int64_t n;
  bool bf16;
};
// norm = the L2 norm of all n tensors together; ws: grad_norm_workspace() bytes.
size_t grad_norm_workspace();
hipError_t grad_norm(int n, const GradTensor* g, float* norm, void* ws, hipStream_t s);
// out[i] = g[i] min(1, max_norm / (norm + 1e-6)), out[i] of as many elements as g[i], or g[i] itself.
hipError_t grad_clip(int n, const GradTensor* g, const float* norm, float max_norm, const GradTensor* out, hipStream_t s);

// ---- optimizer ------------------------------------------------------------------
struct AdamwHyper {
  float lr, beta1, beta2, eps, weight_decay, max_norm;  // max_norm <= 0: no clipping
  int step;                                            // t >= 1
};
// Workspace bytes of adamw_step (independent of n).
size_t adamw_workspace();
// Global-norm clip + AdamW over n fp32 parameters (decay on the first n_decay);
// param (bf16 copy) and grad_norm may be null.
hipError_t adamw_step(int64_t n, int64_t n_decay, const AdamwHyper& hp, float* master, bf16_t* param,
                      const float* grad, float* m, float* v, float* grad_norm, void* ws, hipStream_t s);

}  // namespace ls

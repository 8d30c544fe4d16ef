// tokens_internal.h -- limits, workspaces and launchers shared by the HIP
// translation units of the operators on token tables (include/flashtokens.h).
#pragma once

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "fkm_internal.h"

namespace fkm {

constexpr int64_t TOK_MAX_M = 1 << 24, TOK_MAX_V = 1 << 20, TOK_MAX_D = 8192;
constexpr int TOK_MAX_K = 32;
// Of the gradients of log probabilities: the products' offsets within 256 rows of M fp16
// values are 32 bits wide.
constexpr int64_t TOK_MAX_GRAD_M = (1 << 23) - 64;

// api.hip
int check_device();
int check_ptrs(std::initializer_list<const void*> ps);
int hip_status(hipError_t e);

// Positions sorted by token: a stable radix sort of (token, position), in as many
// passes of at most 8 bits as the tokens take (update.hip).  keys / vals: [B, M]
// each, the sorted ones in keys[0] / vals[0]; total[b] the number of positions
// with a token.
struct TokenSort {
  int32_t *keys[2], *vals[2];
  int32_t *hist, *bins;  // [B, 256, chunks], [B, 256]
  int32_t* total;        // [B]
};
hipError_t launch_token_sort(const int32_t* idx, int64_t B, int64_t M, int64_t V,
                             const TokenSort& t, hipStream_t s);

hipError_t launch_embed(const void* W, int dt, const int32_t* idx, int64_t B, int64_t M, int64_t V,
                        int64_t D, float scale, void* out, hipStream_t s);

// Copies of 16-bit rows of D elements, X's and W's, in rows of the next multiple of 8.
hipError_t launch_pad_both(const void* X, int64_t xrows, void* xpad, const void* W, int64_t wrows,
                           void* wpad, int64_t D, hipStream_t s);

struct EmbedGradWs {
  TokenSort sort;
  float* carry;  // [B, slices, 2, D] sums of runs cut by slice ends
  size_t total;
};
EmbedGradWs embed_grad_carve(void* base, int64_t B, int64_t M, int64_t V, int64_t D);
hipError_t launch_embed_grad(const void* G, int gdt, const int32_t* idx, int64_t B, int64_t M,
                             int64_t V, int64_t D, float scale, bool accumulate, void* dW, int wdt,
                             const EmbedGradWs& w, hipStream_t s);

// ---- scores against a table (logprobs.h) ----------------------------------------
// Products are tiled 256 positions x 256 (or 128) table rows; contractions are cut
// in stages of 64 elements.
constexpr int LP_BB = 256, LP_DC = 64;
// A scored row's columns come in groups of 64, whose best scores lead to the k best.
constexpr int LP_GROUP = 64;

// tokens_logprobs.  Rows are taken in blocks whose stored scores (k > 0 only) stay
// within LP_SCORE_BYTES; column blocks of 256 are shared out over `splits`
// workgroups a row block, whose softmax statistics are merged.
constexpr int64_t LP_SCORE_BYTES = (int64_t)1 << 30;
//
// Workgroup ids go round-robin over the 8 XCDs.  Blocks of A by blocks of B (and
// instances) are walked in super-tiles of ga x gb workgroups, each on one XCD, so
// that the 32 resident there share both operands' stages through its L2: per stage
// ga + gb blocks come from beyond it instead of up to 33.
struct Raster {
  int na, nb, ga, gb;  // blocks of A and B, and of a super-tile
  int64_t supers;      // of all instances
  int64_t blocks() const { return (supers + 7) / 8 * 8 * ga * gb; }  // of the grid
};
// 4 x 8 where there are as many, then smaller until the XCDs' loads differ by at
// most an eighth.
inline Raster make_raster(int64_t na, int64_t nb, int64_t inst) {
  Raster r{(int)na, (int)nb, (int)(na < 4 ? na : 4), 0, 0};
  r.gb = (int)(nb < 32 / r.ga ? nb : 32 / r.ga);
  if (r.gb < 8) r.ga = (int)(na < 32 / r.gb ? na : 32 / r.gb);
  for (;;) {
    r.supers = (na + r.ga - 1) / r.ga * ((nb + r.gb - 1) / r.gb) * inst;
    if (r.ga * r.gb == 1 || r.blocks() * 8 <= na * nb * inst * 9) return r;
    if (r.ga > r.gb) r.ga = (r.ga + 1) / 2;
    else r.gb = (r.gb + 1) / 2;
  }
}
// At most this many workgroups come of sharing out the column blocks.
constexpr int64_t SCORE_WGS = 1024;
// Shares of the column blocks: the number with the least rounds of 256 workgroups
// times what one takes, its blocks and about three stages of filling and emptying.
inline int score_splits(int64_t nmb, int64_t B, int64_t nvb, int64_t stages) {
  const int64_t most = std::min(nvb, std::max<int64_t>(1, SCORE_WGS / (nmb * B)));
  int best = 1;
  double least = HUGE_VAL;
  for (int64_t s = 1; s <= most; s += s < 8 ? 1 : s < 64 ? 8 : s / 8 / 8 * 8) {
    const double us = (double)((make_raster(s, nmb, B).blocks() + 255) / 256) *
                      ((double)((nvb + s - 1) / s * stages) + 3);
    if (us < least) least = us, best = (int)s;
  }
  return best;
}
// Few rows, or few of both: workgroups of 64 columns by 64 rows, two to a CU, instead of
// tiles.  Always up to 64 rows; else where the estimates, in us, say so: a workgroup's
// fixed part and its quarter of the contraction in units of 64 elements, against a tile's
// column blocks.
constexpr int64_t LP_FEW_M = 64, LP_FEW_WGS = 2048;
inline bool score_few(int64_t B, int64_t M, int64_t V, int64_t Dk) {
  if (M <= LP_FEW_M) return true;
  const int64_t units = (Dk + 63) / 64, wgs = (M + 63) / 64 * ((V + 63) / 64) * B;
  if (wgs > LP_FEW_WGS) return false;
  const int64_t nmb = (M + LP_BB - 1) / LP_BB, nvb = (V + 255) / 256;
  const int s = score_splits(nmb, B, nvb, units);
  const double few = (double)((wgs + 511) / 512) * (5 + 0.9 * (double)((units + 3) / 4));
  const double tile = (double)((make_raster(s, nmb, B).blocks() + 255) / 256) *
                      (3 + (double)((nvb + s - 1) / s) * (1.4 * (double)units + 4));
  return few < tile;
}
struct LogprobsPlan {
  int64_t rows;    // rows of a block (all of M for k = 0)
  bool few;        // a workgroup for every 64 columns and up to 64 rows
  // k > 0 and many scores: the first `head` column blocks in a launch of their own, whose
  // scores bound the k best from below; of the others only what exceeds that is stored
  int head, head_splits;
  int splits;      // shares of the (other) columns, a workgroup each
};
struct LogprobsWs {
  void *xpad, *wpad;  // rows of Dk elements, where D is no multiple of 8
  float4* part;       // [B, splits, rows] max, sum, weighted sum of each share
  float* zt;          // [B, rows] score of the target
  float* gmax;        // [B, rows, groups] best score of each group (k > 0)
  float* z;           // [B, rows, ldz] scores (k > 0)
  float* bound;       // [B, rows] (k > 0)
  int64_t Dk, ldz, groups;
  LogprobsPlan plan;
  size_t total;
};

struct LogprobsArgs {
  const void *X, *W;
  const float* bias;
  const int32_t* target;
  int64_t B, M, V, D;
  float scale;
  int k;
  float *logprob, *entropy, *lse;
  int32_t* top_idx;
  float* top_logprob;
};

// tokens_logprobs_grad.  dz of a block of table rows (Vc of them; all, where it
// fits LP_DZ_BYTES with its transpose) and instances (all or one) is stored in fp16,
// and both products read it and transposed fp16 copies of X and W.
constexpr int64_t LP_DZ_BYTES = (int64_t)1 << 30;
constexpr int64_t LP_ACC_BYTES = (int64_t)1 << 30;
constexpr int64_t LP_NARROW = 256, LP_NARROW_SCORES = 1 << 25;
constexpr int64_t LP_EXACT = 64;     // fp16 positions up to which a target's dz is exact
constexpr int64_t STATS_WGS = 1024;  // most workgroups of an instance's statistics
// One position.  p = 2^l of a score z: without offsets l = z log2 e - lse, lse in units of
// log 2, one fma of the accumulator; offsets (one may be the type's lowest value) need
// l + more = (z - lse) log2 e, lse in natural units and `more` 0 but for far rows.  dz =
// 2^(l + more) (c0 + c1 (l + more)), and g more at the target.
struct RowGrad {
  float g;        // gradient of the log probability over `gs` (>= 0 without gradients of
                  // entropies), DZ_UP times that
  float c0, c1;   // -(h entropy + g) and -h ln 2 (`more` in them), h the entropy's gradient
  float lse;
  int target;     // -1: none
  int active;     // takes part at all
  float gs;       // what g, h and so dz of this row are divided by
  float part;     // what dW takes of gs over the largest into dz (faint_part): g, c0 and c1
                  // are times this
};
// Elements from row to row of dz and the copies: 128 bytes past a multiple of 1 KiB, so
// that a stage's 64 bytes of each of 512 rows do not all lie in one L2 channel.
inline int64_t grad_ld(int64_t n) { return n % 512 == 0 ? n + 64 : n; }
struct GradWs {
  void *xpad, *wpad;
  RowGrad* rows;    // [B, M]
  float4* stats;    // [B, workgroups] largest gs and magnitudes of X and W
  float4* scales;   // [B] the largest gs, the factors of X and W
  void *dz, *dzt;   // [nb, M, grad_ld(Vp)], [nb, Vp, grad_ld(Mp)]
  void *xt, *wt;    // [nb, D, grad_ld(Mp)], [nb, D, grad_ld(Vp)]
  float* accx;      // dX over the blocks of table rows, where there are several: [M, Dk],
                    // or all their shares
  float* part;      // [nb, splits, rows, D] shares of a contraction
  int64_t Dk, Mp, Vp, Vc;
  bool narrow;      // short rows: dz is not stored (logprobs_narrow.h)
  int nb;           // instances at a time (B or 1)
  int sx, sw;       // shares of dX's and dW's contractions
  size_t total;
};

struct GradArgs {
  const void *X, *W;
  const float* bias;
  const int32_t* target;
  const float *lse, *entropy, *g, *h;
  int64_t B, M, V, D;
  float scale;
  void *dX, *dW;
};
hipError_t launch_logprobs_bf16(const LogprobsArgs& a, const LogprobsWs& w, hipStream_t s);
hipError_t launch_logprobs_f16(const LogprobsArgs& a, const LogprobsWs& w, hipStream_t s);
hipError_t launch_logprobs_grad_bf16(const GradArgs& a, const GradWs& w, hipStream_t s);
hipError_t launch_logprobs_grad_f16(const GradArgs& a, const GradWs& w, hipStream_t s);

}  // namespace fkm

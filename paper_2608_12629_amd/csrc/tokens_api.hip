// tokens_api.hip -- the C ABI of the operators on token tables (declared in
// include/flashtokens.h): argument validation on the host before anything touches
// the GPU, workspace carving and the choice of shares.
#include <algorithm>
#include <cmath>

#include "../../include/flashtokens.h"
#include "tokens_internal.h"

namespace fkm {

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

int check_tokens(int64_t B, int64_t M, int64_t V, int64_t D, int dt) {
  if (B < 1 || M < 1 || V < 1 || D < 1) return FKM_ERR_INVALID_ARG;
  if (dt != DT_F32 && dt != DT_BF16 && dt != DT_F16) return FKM_ERR_INVALID_ARG;
  if (B > 65535 || M > TOK_MAX_M || V > TOK_MAX_V || D > TOK_MAX_D) return FKM_ERR_UNSUPPORTED;
  return FKM_OK;
}
int check_scores(int64_t B, int64_t M, int64_t V, int64_t D, int64_t k, int dt) {
  const int rc = check_tokens(B, M, V, D, dt);
  if (rc) return rc;
  if (k < 0 || k > V) return FKM_ERR_INVALID_ARG;
  if (dt == DT_F32 || k > TOK_MAX_K) return FKM_ERR_UNSUPPORTED;
  return FKM_OK;
}
int check_grads(int64_t B, int64_t M, int64_t V, int64_t D, int dt) {
  const int rc = check_scores(B, M, V, D, 0, dt);
  return rc ? rc : M > TOK_MAX_GRAD_M ? FKM_ERR_UNSUPPORTED : FKM_OK;
}
// Arrays of one 4-byte element a position or token, which the kernels read and write one at a
// time, may start at any: ids + t of a sequence.
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }
int check_elements(std::initializer_list<const void*> needed,
                   std::initializer_list<const void*> optional = {}) {
  for (const void* p : needed)
    if (!p || !aligned4(p)) return FKM_ERR_INVALID_ARG;
  for (const void* p : optional)
    if (!aligned4(p)) return FKM_ERR_INVALID_ARG;
  return FKM_OK;
}

struct Taker {
  char* p;
  size_t o = 0;
  template <typename T>
  void operator()(T*& out, size_t bytes) {
    out = (T*)(p ? p + o : nullptr);
    o = (o + bytes + 255) & ~size_t(255);
  }
};
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// At most this many workgroups come of sharing out a contraction: two rounds on 256 CUs.
constexpr int64_t OUT_WGS = 512;
constexpr int64_t HEAD_SCORES = 1 << 24;  // scores from which alternatives take a head

LogprobsWs logprobs_carve(void* base, int64_t B, int64_t M, int64_t V, int64_t D, int k) {
  LogprobsWs w{};
  Taker take{(char*)base};
  w.Dk = up(D, 8);
  w.ldz = up(V, 256);
  w.groups = cdiv(V, LP_GROUP);
  w.plan.rows = M;
  if (k) w.plan.rows = std::min(M, std::max<int64_t>(LP_SCORE_BYTES / (B * w.ldz * 4) / 256, 1) * 256);
  const int64_t nmb = cdiv(w.plan.rows, LP_BB), wgs = nmb * B;
  w.plan.few = w.plan.rows == M && score_few(B, M, V, w.Dk);
  const int64_t nvb = w.ldz / 256, stages = cdiv(w.Dk, LP_DC);
  // A head of an eighth of the columns (of 8 groups for each of the k best at the least)
  // where storing every score would cost more than two launches: 4,096 x 65,536 x
  // 1,024, k = 20: 1,014 -> 588 us.
  if (k && !w.plan.few && B * w.plan.rows * w.ldz >= HEAD_SCORES) {
    const int64_t head = std::max(nvb / 8, cdiv(8 * k, 4));
    if (head <= nvb / 4) w.plan.head = (int)head;
  }
  if (w.plan.head) w.plan.head_splits = score_splits(nmb, B, w.plan.head, stages);
  w.plan.splits = w.plan.few ? (int)cdiv(V, 64) : score_splits(nmb, B, nvb - w.plan.head, stages);
  take(w.xpad, w.Dk != D ? (size_t)(B * M * w.Dk) * 2 : 0);
  take(w.wpad, w.Dk != D ? (size_t)(B * V * w.Dk) * 2 : 0);
  // B x splits x rows, for any number of shares that these or fewer rows would get
  take(w.part, (size_t)std::max(2 * std::max(SCORE_WGS, wgs) * LP_BB,
                                B * std::min(M, LP_FEW_M) * cdiv(V, 64)) * sizeof(float4));
  take(w.zt, (size_t)(B * w.plan.rows) * 4);
  take(w.gmax, k ? (size_t)(B * w.plan.rows * w.groups) * 4 : 0);
  take(w.z, k ? (size_t)(B * w.plan.rows * w.ldz) * 4 : 0);
  take(w.bound, k ? (size_t)(B * w.plan.rows) * 4 : 0);
  w.total = take.o;
  return w;
}

// Shares of a contraction of `stages` stages over `tiles` output tiles: enough to
// fill the chip, of at least 8 stages.
int out_splits(int64_t tiles, int64_t stages) {
  return (int)std::max<int64_t>(1, std::min(OUT_WGS / tiles, stages / 8));
}

// Shares of the streamed side over `blocks` workgroups: up to narrow_wgs of a side in all
// (both sides' fill the CUs once), of at least 4 stages.
int64_t narrow_wgs(int64_t D) { return D <= 64 ? 512 : 256; }
int narrow_splits(int64_t blocks, int64_t stages, int64_t D) {
  return (int)std::max<int64_t>(1, std::min(narrow_wgs(D) / blocks, stages / 4));
}

GradWs grad_carve(void* base, int64_t B, int64_t M, int64_t V, int64_t D) {
  GradWs w{};
  Taker take{(char*)base};
  w.Dk = up(D, 8);
  w.Mp = up(M, 64);
  const int64_t Vall = up(V, 64), one = w.Mp * Vall * 4;
  // dz is not stored for rows of up to 128 elements (us, stored / not, 64 x 64 x 64 23 /
  // 16, 10,007 x 1,003 x 128 52 / 46, 16,384 x 4,096 x 128 240 / 104).  From there to 256
  // the four products take longer than storing as long as dz stays in the caches: not
  // stored where the calls are short or the two copies of dz (4 bytes a score) pass 128
  // MiB (1,000 x 1,000 x 256 48 / 38, 10,007 x 1,003 x 200 65 / 74, 4,096 x 4,096 x 256
  // 79 / 87, 8,192 x 8,192 x 256 328 / 202).
  const int64_t scores = B * w.Mp * Vall;
  w.narrow = D <= 128 || (D <= LP_NARROW && (scores <= 1 << 22 || scores >= LP_NARROW_SCORES));
  w.nb = w.narrow || B * one <= LP_DZ_BYTES ? (int)B : 1;
  w.Vc = w.narrow || w.nb * one <= LP_DZ_BYTES || V <= 256
             ? V : std::min(V, std::max<int64_t>(LP_DZ_BYTES / (4 * w.Mp) / 256, 1) * 256);
  w.Vp = up(w.Vc, 64);
  const int64_t dt = cdiv(D, 256);
  if (w.narrow) {
    w.sx = narrow_splits(B * cdiv(M, 128), Vall / 64, D);
    w.sw = narrow_splits(B * cdiv(V, 128), w.Mp / 64, D);
  } else {
    w.sx = out_splits(w.nb * cdiv(M, LP_BB) * dt, w.Vp / LP_DC);
    w.sw = out_splits(w.nb * cdiv(w.Vc, LP_BB) * dt, w.Mp / LP_DC);
    // shares of every block of table rows are kept until the last (4,096 x 131,072 x 512
    // in two blocks: 4,357 us with one share of each, 2,194 so)
    if (w.Vc < V)
      w.sx = (int)std::min<int64_t>(w.sx, std::max<int64_t>(1, LP_ACC_BYTES / (cdiv(V, w.Vc) * M * w.Dk * 4)));
  }
  take(w.xpad, w.Dk != D ? (size_t)(B * M * w.Dk) * 2 : 0);
  take(w.wpad, w.Dk != D ? (size_t)(B * V * w.Dk) * 2 : 0);
  take(w.rows, (size_t)(B * M) * sizeof(RowGrad));
  take(w.stats, (size_t)(B * std::min(STATS_WGS, M + V)) * sizeof(float4));
  take(w.scales, (size_t)B * sizeof(float4));
  // sizes that never shrink as M grows, whatever the plan then is
  // (and 64 more elements a row: grad_ld)
  const size_t dz = (size_t)(std::max(std::min(B * one, LP_DZ_BYTES) / 2, w.Mp * 256 * 2) +
                             B * std::max(w.Mp, Vall) * 64 * 2);
  const size_t held = D <= 128 ? 0 : D > LP_NARROW ? dz :
      (size_t)(std::min(scores, LP_NARROW_SCORES) + B * std::max(w.Mp, Vall) * 64) * 2;
  take(w.dz, held);
  take(w.dzt, held);
  take(w.xt, (size_t)(B * D * (w.Mp + 64)) * 2);
  take(w.wt, (size_t)(B * D * (Vall + 64)) * 2);
  take(w.accx, w.Vc < V ? (size_t)std::max(M * w.Dk * 4, LP_ACC_BYTES) : 0);
  const double cap = (double)OUT_WGS * LP_BB * 256;  // elements of all shared-out tiles
  const double px = Vall / 512 < 2 ? 0 : std::min((double)B * M * w.Dk * (Vall / 512), cap);
  const double pw = w.Mp / 512 < 2 ? 0 : std::min((double)B * V * w.Dk * (w.Mp / 512), cap);
  // narrow: at most narrow_wgs x 128 rows of a side in shares
  const double ncap = (double)narrow_wgs(D) * 128 * (double)w.Dk;
  const double nx = std::min((double)B * M * w.Dk * std::max<int64_t>(1, Vall / 256), ncap);
  const double nw = std::min((double)B * V * w.Dk * std::max<int64_t>(1, w.Mp / 256), ncap);
  take(w.part, (size_t)(D <= 128 ? nx + nw : D <= LP_NARROW ? std::max(nx + nw, px + pw) : px + pw) * 4);
  w.total = take.o;
  return w;
}

}  // namespace

}  // namespace fkm

using namespace fkm;

extern "C" {

int tokens_embed(const void* W, int dtype, const int32_t* idx, int64_t B, int64_t M, int64_t V,
                 int64_t D, float scale, void* out, void* stream) {
  int rc;
  if ((rc = check_ptrs({W, out})) || (rc = check_elements({idx}))) return rc;
  if ((rc = check_tokens(B, M, V, D, dtype))) return rc;
  if ((rc = check_device())) return rc;
  return hip_status(launch_embed(W, dtype, idx, B, M, V, D, scale, out, (hipStream_t)stream));
}

size_t tokens_embed_grad_workspace_bytes(int64_t B, int64_t M, int64_t V, int64_t D, int gdtype) {
  if (check_tokens(B, M, V, D, gdtype) != FKM_OK) return 0;
  return embed_grad_carve(nullptr, B, M, V, D).total;
}

int tokens_embed_grad(const void* G, int gdtype, const int32_t* idx, int64_t B, int64_t M,
                      int64_t V, int64_t D, float scale, int accumulate, void* dW, int wdtype,
                      void* ws, size_t ws_bytes, void* stream) {
  int rc;
  if ((rc = check_ptrs({G, dW})) || (rc = check_elements({idx}))) return rc;
  if ((rc = check_tokens(B, M, V, D, gdtype))) return rc;
  if (wdtype != gdtype && wdtype != DT_F32) return FKM_ERR_INVALID_ARG;
  const EmbedGradWs w = embed_grad_carve(ws, B, M, V, D);
  if (!ws || !aligned16(ws) || ws_bytes < w.total) return FKM_ERR_WORKSPACE;
  if ((rc = check_device())) return rc;
  return hip_status(launch_embed_grad(G, gdtype, idx, B, M, V, D, scale, accumulate != 0, dW, wdtype,
                                      w, (hipStream_t)stream));
}

size_t tokens_logprobs_workspace_bytes(int64_t B, int64_t M, int64_t V, int64_t D, int k,
                                       int xdtype) {
  if (check_scores(B, M, V, D, k, xdtype) != FKM_OK) return 0;
  return logprobs_carve(nullptr, B, M, V, D, k).total;
}

int tokens_logprobs(const void* X, const void* W, int xdtype, const float* bias,
                    const int32_t* target, int64_t B, int64_t M, int64_t V, int64_t D, float scale,
                    int k, float* logprob, float* entropy, float* lse, int32_t* top_idx,
                    float* top_logprob, void* ws, size_t ws_bytes, void* stream) {
  int rc;
  if ((rc = check_ptrs({X, W}))) return rc;
  if ((rc = check_elements({lse}, {bias, target, logprob, entropy, top_idx, top_logprob}))) return rc;
  if (target && !logprob) return FKM_ERR_INVALID_ARG;
  if (k > 0 && (!top_idx || !top_logprob)) return FKM_ERR_INVALID_ARG;
  if (!std::isfinite(scale)) return FKM_ERR_INVALID_ARG;
  if ((rc = check_scores(B, M, V, D, k, xdtype))) return rc;
  const LogprobsWs w = logprobs_carve(ws, B, M, V, D, k);
  if (!ws || !aligned16(ws) || ws_bytes < w.total) return FKM_ERR_WORKSPACE;
  if ((rc = check_device())) return rc;
  const LogprobsArgs a{X, W, bias, target, B, M, V, D, scale, k, logprob, entropy, lse, top_idx,
                       top_logprob};
  return hip_status((xdtype == DT_BF16 ? launch_logprobs_bf16 : launch_logprobs_f16)(
      a, w, (hipStream_t)stream));
}

size_t tokens_logprobs_grad_workspace_bytes(int64_t B, int64_t M, int64_t V, int64_t D,
                                            int xdtype) {
  if (check_grads(B, M, V, D, xdtype) != FKM_OK) return 0;
  return grad_carve(nullptr, B, M, V, D).total;
}

int tokens_logprobs_grad(const void* X, const void* W, int xdtype, const float* bias,
                         const int32_t* target, const float* lse, const float* entropy,
                         const float* grad_logprob, const float* grad_entropy, int64_t B, int64_t M,
                         int64_t V, int64_t D, float scale, void* dX, void* dW, void* ws,
                         size_t ws_bytes, void* stream) {
  int rc;
  if ((rc = check_ptrs({X, W, dX, dW}))) return rc;
  if ((rc = check_elements({target, lse, grad_logprob}, {bias, entropy, grad_entropy}))) return rc;
  if (grad_entropy && !entropy) return FKM_ERR_INVALID_ARG;
  if (!std::isfinite(scale)) return FKM_ERR_INVALID_ARG;
  if ((rc = check_grads(B, M, V, D, xdtype))) return rc;
  const GradWs w = grad_carve(ws, B, M, V, D);
  if (!ws || !aligned16(ws) || ws_bytes < w.total) return FKM_ERR_WORKSPACE;
  if ((rc = check_device())) return rc;
  const GradArgs a{X, W, bias, target, lse, entropy, grad_logprob, grad_entropy, B, M, V, D, scale,
                   dX, dW};
  return hip_status((xdtype == DT_BF16 ? launch_logprobs_grad_bf16 : launch_logprobs_grad_f16)(
      a, w, (hipStream_t)stream));
}

}  // extern "C"

// C-ABI entry points of the token operators: dropout, node states from a token
// table and its gradient, the cross entropy over a vocabulary, distillation from
// a teacher's lists.  Arguments are checked on the host, then the kernels are
// launched on the caller's stream.
#include <hip/hip_runtime.h>

#include <cmath>

#include "common.h"
#include "kernels.h"

using namespace ggnn;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

ggnn_status device_status(hipError_t err, const char* what) {
  if (err == hipSuccess) return GGNN_OK;
  return fail(GGNN_ERR_DEVICE, "%s: %s", what, hipGetErrorString(err));
}

#define CHECK_PTR(p, name)                                                  \
  do {                                                                      \
    GGNN_CHECK_ARG((p) != nullptr, "%s is NULL", name);                     \
    GGNN_CHECK_ARG(aligned16(p), "%s is not 16-byte aligned", name);        \
  } while (0)
#define CHECK_OPT_PTR(p, name)                                              \
  do {                                                                      \
    if ((p) != nullptr) GGNN_CHECK_ARG(aligned16(p), "%s is not 16-byte aligned", name); \
  } while (0)

inline hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

// Whether the byte ranges [p, p + pb) and [q, q + qb) share no byte.
bool disjoint(const void* p, size_t pb, const void* q, size_t qb) {
  const char *a = static_cast<const char*>(p), *c = static_cast<const char*>(q);
  return a + pb <= c || c + qb <= a;
}

// Element numbers of one call (a lane's number of eight must fit 32 bits).
constexpr int64_t kMaxElements = (int64_t)1 << 34;
constexpr int32_t kMaxTokens = 1 << 30;   // listed tokens of a call
constexpr int32_t kMaxRows = 1 << 24;     // chosen nodes of a call

ggnn_status make_dropout(float p, uint64_t seed, uint64_t offset, Dropout* d) {
  GGNN_CHECK_ARG(p >= 0.f && p < 1.f, "p=%g must be in [0, 1)", (double)p);   // NaN fails too
  const long cut = std::lround((double)p * 65536.0);
  d->cut = (uint32_t)(cut < 65535 ? cut : 65535);
  d->scale = 65536.f / (float)(65536 - d->cut);
  d->seed_lo = (uint32_t)seed;
  d->seed_hi = (uint32_t)(seed >> 32);
  d->offset_lo = (uint32_t)offset;
  d->offset_hi = (uint32_t)(offset >> 32);
  return GGNN_OK;
}

ggnn_status check_embed(int32_t n, int32_t H, int32_t V, const int32_t* tok_ptr, const int32_t* tok, int32_t n_tok,
                        float scale) {
  GGNN_CHECK_ARG(n >= 0, "n=%d must not be negative", n);
  GGNN_CHECK_ARG(supported_H(H), "H=%d must be one of 32, 64, 128, 256", H);
  GGNN_CHECK_ARG((int64_t)n * H <= kMaxElements, "n*H exceeds 2^34 elements");
  GGNN_CHECK_ARG(V >= 1, "V=%d must be at least 1", V);
  GGNN_CHECK_ARG(n_tok >= 0 && n_tok <= kMaxTokens, "n_tok=%d must be in [0, 2^30]", n_tok);
  GGNN_CHECK_ARG(tok_ptr != nullptr || n_tok <= n, "n_tok=%d exceeds n=%d, with one token per node", n_tok, n);
  GGNN_CHECK_ARG(std::isfinite(scale), "scale must be finite");
  CHECK_OPT_PTR(tok_ptr, "tok_ptr");
  if (n_tok > 0) CHECK_PTR(tok, "tok");
  return GGNN_OK;
}

ggnn_status check_rows(int32_t dt, int32_t n_nodes, int32_t H, int32_t n_rows, int32_t V, const void* X,
                       const void* W, const float* bias, const int32_t* node) {
  GGNN_CHECK_ARG(supported_dtype(dt), "unknown dtype %d", dt);
  GGNN_CHECK_ARG(n_nodes >= 1, "n_nodes=%d must be at least 1", n_nodes);
  GGNN_CHECK_ARG(supported_H(H), "H=%d must be one of 32, 64, 128, 256", H);
  GGNN_CHECK_ARG((int64_t)n_nodes * H <= kMaxElements, "n_nodes*H exceeds 2^34 elements");
  GGNN_CHECK_ARG(n_rows >= 0 && n_rows <= kMaxRows, "n_rows=%d must be in [0, 2^24]", n_rows);
  GGNN_CHECK_ARG(node != nullptr || n_rows <= n_nodes, "n_rows=%d exceeds n_nodes=%d, with no node list", n_rows,
                 n_nodes);
  GGNN_CHECK_ARG(V >= 1 && (int64_t)V * H < ((int64_t)1 << 31), "V=%d must be at least 1, and V*H below 2^31", V);
  CHECK_PTR(X, "X");
  CHECK_PTR(W, "W");
  CHECK_OPT_PTR(bias, "bias");
  CHECK_OPT_PTR(node, "node");
  return GGNN_OK;
}

ggnn_status check_vocab(int32_t dt, int32_t n_nodes, int32_t H, int32_t n_rows, int32_t V, const void* X,
                        const void* W, const float* bias, const int32_t* node, const int32_t* target,
                        const float* lse) {
  const ggnn_status st = check_rows(dt, n_nodes, H, n_rows, V, X, W, bias, node);
  if (st != GGNN_OK) return st;
  CHECK_OPT_PTR(target, "target");
  if (n_rows > 0) CHECK_PTR(lse, "lse");
  return GGNN_OK;
}

// What the losses over a vocabulary share of their arguments.
VocabArgs vocab_args(int32_t n_nodes, int32_t n_rows, int32_t V, const void* X, const void* W, const float* bias,
                     const int32_t* node, float* loss, float* lse, void* workspace) {
  VocabArgs c{};
  c.n_nodes = n_nodes; c.R = n_rows; c.V = V;
  c.X = X; c.W = W; c.bias = bias; c.node = node;
  c.scale = 1.f;
  c.loss = loss; c.lse = lse;
  c.ws = workspace;
  return c;
}

ggnn_status check_gradients(int32_t dt, int32_t n_nodes, int32_t H, int32_t V, const void* X, const void* W,
                            const float* weight, float scale, const float* dX, const float* dW, const float* dbias) {
  GGNN_CHECK_ARG(std::isfinite(scale), "scale must be finite");
  CHECK_PTR(dX, "dX");
  CHECK_PTR(dW, "dW");
  CHECK_OPT_PTR(dbias, "dbias");
  CHECK_OPT_PTR(weight, "weight");
  const size_t es = dtype_bytes(dt), nx = (size_t)n_nodes * H, nw = (size_t)V * H;
  GGNN_CHECK_ARG(disjoint(dX, nx * 4, X, nx * es) && disjoint(dX, nx * 4, W, nw * es), "dX overlaps X or W");
  GGNN_CHECK_ARG(disjoint(dW, nw * 4, W, nw * es) && disjoint(dW, nw * 4, X, nx * es) &&
                     disjoint(dW, nw * 4, dX, nx * 4),
                 "dW overlaps W, X or dX");
  return GGNN_OK;
}

constexpr int32_t kMaxList = 64;                              // entries of a row's list
constexpr float kMinTemperature = 1e-3f, kMaxTemperature = 1e3f;

ggnn_status check_temperature(float t) {
  GGNN_CHECK_ARG(t >= kMinTemperature && t <= kMaxTemperature, "temperature=%g must be in [0.001, 1000]", (double)t);
  return GGNN_OK;
}

bool distill_sizes(int32_t dt, int32_t H, int32_t n_rows, int32_t V, int32_t K) {
  return supported_dtype(dt) && supported_H(H) && n_rows > 0 && n_rows <= kMaxRows && V >= 1 &&
         (int64_t)V * H < ((int64_t)1 << 31) && K >= 1 && K <= kMaxList && (int64_t)n_rows * K <= kMaxTokens;
}

ggnn_status check_distill(int32_t n_rows, int32_t K, const int32_t* t_id, const float* t_logit, const float* t_lse,
                          float temperature, const float* loss) {
  GGNN_CHECK_ARG(K >= 1 && K <= kMaxList, "K=%d must be in [1, %d]", K, kMaxList);
  GGNN_CHECK_ARG((int64_t)n_rows * K <= kMaxTokens, "n_rows*K exceeds 2^30 listings");
  const ggnn_status st = check_temperature(temperature);
  if (st != GGNN_OK) return st;
  if (n_rows > 0) {
    CHECK_PTR(t_id, "teacher_id");
    CHECK_PTR(t_logit, "teacher_logit");
    CHECK_PTR(loss, "loss");
  }
  CHECK_OPT_PTR(t_lse, "teacher_lse");
  return GGNN_OK;
}

bool top_sizes(int32_t dt, int32_t H, int32_t n_rows, int32_t V, int32_t K, int64_t n_listed) {
  return supported_dtype(dt) && supported_H(H) && n_rows > 0 && n_rows <= kMaxRows && V >= 1 &&
         (int64_t)V * H < ((int64_t)1 << 31) && K >= 1 && K <= kMaxList && n_listed >= 0 && n_listed <= kMaxTokens;
}

ggnn_status check_rules(int32_t V, const ggnn_token_rules* u) {
  if (u == nullptr) return GGNN_OK;
  GGNN_CHECK_ARG(u->n_masks >= 0, "n_masks=%d must not be negative", u->n_masks);
  if (u->n_masks > 0) {
    CHECK_PTR(u->mask, "mask");
    GGNN_CHECK_ARG(u->mask_words >= (V + 31) / 32, "mask_words=%d must be at least %d for V=%d", u->mask_words,
                   (V + 31) / 32, V);
    CHECK_OPT_PTR(u->mask_of, "mask_of");
  }
  GGNN_CHECK_ARG(u->n_seen >= 0 && u->n_add >= 0 && (int64_t)u->n_seen + u->n_add <= kMaxTokens,
                 "n_seen=%d and n_add=%d must not be negative, nor exceed 2^30 together", u->n_seen, u->n_add);
  if (u->n_seen > 0) {
    CHECK_PTR(u->seen_ptr, "seen_ptr");
    CHECK_PTR(u->seen, "seen");
    GGNN_CHECK_ARG(std::isfinite(u->repetition) && u->repetition > 0.f, "repetition=%g must be finite and positive",
                   (double)u->repetition);
    GGNN_CHECK_ARG(std::isfinite(u->presence) && std::isfinite(u->frequency), "presence and frequency must be finite");
  }
  if (u->n_add > 0) {
    CHECK_PTR(u->add_ptr, "add_ptr");
    CHECK_PTR(u->add, "add");
    CHECK_PTR(u->value, "value");
  }
  return GGNN_OK;
}

}  // namespace

extern "C" {

ggnn_status ggnn_dropout(ggnn_dtype dt, int64_t count, const void* X, float p, uint64_t seed, uint64_t offset,
                         void* Y, void* stream) {
  clear_error();
  GGNN_CHECK_ARG(supported_dtype(dt), "unknown dtype %d", dt);
  GGNN_CHECK_ARG(count >= 0 && count <= kMaxElements, "count=%lld must be in [0, 2^34]", (long long)count);
  Dropout d;
  const ggnn_status st = make_dropout(p, seed, offset, &d);
  if (st != GGNN_OK) return st;
  if (count == 0) return GGNN_OK;
  CHECK_PTR(X, "X");
  CHECK_PTR(Y, "Y");
  const size_t bytes = (size_t)count * dtype_bytes(dt);
  GGNN_CHECK_ARG(X == Y || disjoint(X, bytes, Y, bytes), "X and Y overlap without being one buffer");
  return device_status(launch_dropout(dt, count, X, Y, d, as_stream(stream)), "dropout");
}

ggnn_status ggnn_embed(ggnn_dtype dt, int32_t n, int32_t H, int32_t V, const void* table, const int32_t* tok_ptr,
                       const int32_t* tok, int32_t n_tok, float scale, int32_t mean, float p, uint64_t seed,
                       uint64_t offset, void* X, void* stream) {
  clear_error();
  GGNN_CHECK_ARG(supported_dtype(dt), "unknown dtype %d", dt);
  ggnn_status st = check_embed(n, H, V, tok_ptr, tok, n_tok, scale);
  if (st != GGNN_OK) return st;
  Dropout d;
  st = make_dropout(p, seed, offset, &d);
  if (st != GGNN_OK) return st;
  if (n == 0) return GGNN_OK;
  CHECK_PTR(table, "table");
  CHECK_PTR(X, "X");
  const size_t es = dtype_bytes(dt);
  GGNN_CHECK_ARG(disjoint(table, (size_t)V * H * es, X, (size_t)n * H * es), "X overlaps the table");
  return device_status(launch_embed(dt, n, H, V, table, tok_ptr, tok, n_tok, scale, mean != 0, d, X,
                                    as_stream(stream)),
                       "embed");
}

size_t ggnn_embed_bwd_workspace_bytes(int32_t n, int32_t H, int32_t V, int32_t n_tok) {
  if (n <= 0 || !supported_H(H) || V < 1 || n_tok <= 0 || n_tok > kMaxTokens) return 0;
  return embed_bwd_workspace(H, n_tok);
}

ggnn_status ggnn_embed_bwd(int32_t n, int32_t H, int32_t V, const int32_t* tok_ptr, const int32_t* tok,
                           int32_t n_tok, float scale, int32_t mean, float p, uint64_t seed, uint64_t offset,
                           const float* dX, float* dtable, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  ggnn_status st = check_embed(n, H, V, tok_ptr, tok, n_tok, scale);
  if (st != GGNN_OK) return st;
  Dropout d;
  st = make_dropout(p, seed, offset, &d);
  if (st != GGNN_OK) return st;
  if (n == 0 || n_tok == 0) return GGNN_OK;
  CHECK_PTR(dX, "dX");
  CHECK_PTR(dtable, "dtable");
  GGNN_CHECK_ARG(disjoint(dX, (size_t)n * H * 4, dtable, (size_t)V * H * 4), "dtable overlaps dX");
  const size_t need = embed_bwd_workspace(H, n_tok);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))
    return fail(GGNN_ERR_WORKSPACE, "embed_bwd needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
                workspace ? workspace_bytes : (size_t)0);
  return device_status(launch_embed_bwd(n, H, V, tok_ptr, tok, n_tok, scale, mean != 0, d, dX, dtable, workspace,
                                        as_stream(stream)),
                       "embed_bwd");
}

size_t ggnn_vocab_workspace_bytes(ggnn_dtype dt, int32_t H, int32_t n_rows, int32_t V, int32_t grad) {
  if (!supported_dtype(dt) || !supported_H(H) || n_rows <= 0 || n_rows > kMaxRows || V < 1 ||
      (int64_t)V * H >= ((int64_t)1 << 31))
    return 0;
  return vocab_workspace(dt, H, n_rows, V, grad != 0);
}

ggnn_status ggnn_vocab_loss(ggnn_dtype dt, int32_t n_nodes, int32_t H, int32_t n_rows, int32_t V, const void* X,
                            const void* W, const float* bias, const int32_t* node, const int32_t* target,
                            float* loss, float* lse, int32_t* best, void* workspace, size_t workspace_bytes,
                            void* stream) {
  clear_error();
  const ggnn_status st = check_vocab(dt, n_nodes, H, n_rows, V, X, W, bias, node, target, lse);
  if (st != GGNN_OK) return st;
  if (n_rows == 0) return GGNN_OK;
  if (target != nullptr) CHECK_PTR(loss, "loss");
  CHECK_OPT_PTR(loss, "loss");
  CHECK_OPT_PTR(best, "best");
  const size_t need = vocab_workspace(dt, H, n_rows, V, false);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))
    return fail(GGNN_ERR_WORKSPACE, "vocab_loss needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
                workspace ? workspace_bytes : (size_t)0);
  VocabArgs c{};
  c.n_nodes = n_nodes; c.R = n_rows; c.V = V;
  c.X = X; c.W = W; c.bias = bias; c.node = node; c.target = target;
  c.scale = 1.f;
  c.loss = loss; c.lse = lse; c.best = best;
  c.ws = workspace;
  return device_status(launch_vocab(dt, H, c, false, as_stream(stream)), "vocab_loss");
}

ggnn_status ggnn_vocab_loss_grad(ggnn_dtype dt, int32_t n_nodes, int32_t H, int32_t n_rows, int32_t V, const void* X,
                                 const void* W, const float* bias, const int32_t* node, const int32_t* target,
                                 const float* weight, float scale, float* loss, float* lse, float* dX, float* dW,
                                 float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const ggnn_status st = check_vocab(dt, n_nodes, H, n_rows, V, X, W, bias, node, target, lse);
  if (st != GGNN_OK) return st;
  GGNN_CHECK_ARG(std::isfinite(scale), "scale must be finite");
  CHECK_PTR(dX, "dX");
  CHECK_PTR(dW, "dW");
  CHECK_OPT_PTR(dbias, "dbias");
  CHECK_OPT_PTR(weight, "weight");
  if (n_rows == 0) return device_status(launch_fill_zero(dX, (size_t)n_nodes * H, as_stream(stream)), "vocab_loss_grad");
  CHECK_PTR(target, "target");
  CHECK_PTR(loss, "loss");
  const size_t need = vocab_workspace(dt, H, n_rows, V, true);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))
    return fail(GGNN_ERR_WORKSPACE, "vocab_loss_grad needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
                workspace ? workspace_bytes : (size_t)0);
  const size_t es = dtype_bytes(dt);
  GGNN_CHECK_ARG(disjoint(dX, (size_t)n_nodes * H * 4, X, (size_t)n_nodes * H * es) &&
                     disjoint(dX, (size_t)n_nodes * H * 4, W, (size_t)V * H * es),
                 "dX overlaps X or W");
  GGNN_CHECK_ARG(disjoint(dW, (size_t)V * H * 4, W, (size_t)V * H * es) &&
                     disjoint(dW, (size_t)V * H * 4, X, (size_t)n_nodes * H * es) &&
                     disjoint(dW, (size_t)V * H * 4, dX, (size_t)n_nodes * H * 4),
                 "dW overlaps W, X or dX");
  VocabArgs c{};
  c.n_nodes = n_nodes; c.R = n_rows; c.V = V;
  c.X = X; c.W = W; c.bias = bias; c.node = node; c.target = target;
  c.weight = weight; c.scale = scale;
  c.loss = loss; c.lse = lse;
  c.dX = dX; c.dW = dW; c.dbias = dbias;
  c.ws = workspace;
  return device_status(launch_vocab(dt, H, c, true, as_stream(stream)), "vocab_loss_grad");
}

size_t ggnn_vocab_distill_workspace_bytes(ggnn_dtype dt, int32_t H, int32_t n_rows, int32_t V, int32_t K,
                                          int32_t grad) {
  if (!distill_sizes(dt, H, n_rows, V, K)) return 0;
  return vocab_workspace(dt, H, n_rows, V, grad != 0, K);
}

ggnn_status ggnn_vocab_distill(ggnn_dtype dt, int32_t n_nodes, int32_t H, int32_t n_rows, int32_t V, const void* X,
                               const void* W, const float* bias, const int32_t* node, int32_t K,
                               const int32_t* teacher_id, const float* teacher_logit, const float* teacher_lse,
                               float temperature, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                               void* stream) {
  clear_error();
  ggnn_status st = check_vocab(dt, n_nodes, H, n_rows, V, X, W, bias, node, nullptr, lse);
  if (st == GGNN_OK) st = check_distill(n_rows, K, teacher_id, teacher_logit, teacher_lse, temperature, loss);
  if (st != GGNN_OK) return st;
  if (n_rows == 0) return GGNN_OK;
  const size_t need = vocab_workspace(dt, H, n_rows, V, false, K);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))
    return fail(GGNN_ERR_WORKSPACE, "vocab_distill needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
                workspace ? workspace_bytes : (size_t)0);
  VocabArgs c = vocab_args(n_nodes, n_rows, V, X, W, bias, node, loss, lse, workspace);
  c.temper = make_temper(temperature);
  c.K = K; c.t_id = teacher_id; c.t_logit = teacher_logit; c.t_lse = teacher_lse;
  return device_status(launch_vocab(dt, H, c, false, as_stream(stream)), "vocab_distill");
}

ggnn_status ggnn_vocab_distill_grad(ggnn_dtype dt, int32_t n_nodes, int32_t H, int32_t n_rows, int32_t V,
                                    const void* X, const void* W, const float* bias, const int32_t* node, int32_t K,
                                    const int32_t* teacher_id, const float* teacher_logit, const float* teacher_lse,
                                    float temperature, const float* weight, float scale, int32_t add, float* loss,
                                    float* lse, float* dX, float* dW, float* dbias, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  clear_error();
  ggnn_status st = check_vocab(dt, n_nodes, H, n_rows, V, X, W, bias, node, nullptr, lse);
  if (st == GGNN_OK) st = check_distill(n_rows, K, teacher_id, teacher_logit, teacher_lse, temperature, loss);
  if (st == GGNN_OK) st = check_gradients(dt, n_nodes, H, V, X, W, weight, scale, dX, dW, dbias);
  if (st != GGNN_OK) return st;
  if (n_rows == 0)
    return add != 0 ? GGNN_OK
                    : device_status(launch_fill_zero(dX, (size_t)n_nodes * H, as_stream(stream)), "vocab_distill_grad");
  const size_t need = vocab_workspace(dt, H, n_rows, V, true, K);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))
    return fail(GGNN_ERR_WORKSPACE, "vocab_distill_grad needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
                workspace ? workspace_bytes : (size_t)0);
  VocabArgs c = vocab_args(n_nodes, n_rows, V, X, W, bias, node, loss, lse, workspace);
  c.temper = make_temper(temperature);
  c.K = K; c.t_id = teacher_id; c.t_logit = teacher_logit; c.t_lse = teacher_lse;
  c.weight = weight; c.scale = scale; c.add = add != 0;
  c.dX = dX; c.dW = dW; c.dbias = dbias;
  return device_status(launch_vocab(dt, H, c, true, as_stream(stream)), "vocab_distill_grad");
}

size_t ggnn_vocab_top_workspace_bytes(ggnn_dtype dt, int32_t H, int32_t n_rows, int32_t V, int32_t K,
                                      int64_t n_listed) {
  if (!top_sizes(dt, H, n_rows, V, K, n_listed)) return 0;
  return top_workspace(dt, H, n_rows, V, K, (int)n_listed);
}

ggnn_status ggnn_vocab_top(ggnn_dtype dt, int32_t n_nodes, int32_t H, int32_t n_rows, int32_t V, const void* X,
                           const void* W, const float* bias, const int32_t* node, const ggnn_token_rules* rules,
                           float temperature, int32_t K, int32_t* top, float* logit, float* lse, void* workspace,
                           size_t workspace_bytes, void* stream) {
  clear_error();
  ggnn_status st = check_rows(dt, n_nodes, H, n_rows, V, X, W, bias, node);
  if (st != GGNN_OK) return st;
  GGNN_CHECK_ARG(K >= 1 && K <= kMaxList, "K=%d must be in [1, %d]", K, kMaxList);
  st = check_temperature(temperature);
  if (st == GGNN_OK) st = check_rules(V, rules);
  if (st != GGNN_OK) return st;
  if (n_rows == 0) return GGNN_OK;
  CHECK_PTR(top, "top");
  CHECK_PTR(logit, "logit");
  CHECK_OPT_PTR(lse, "lse");
  TopArgs a{};
  a.n_nodes = n_nodes; a.R = n_rows; a.V = V; a.K = K;
  a.X = X; a.W = W; a.bias = bias; a.node = node;
  a.temper = make_temper(temperature);
  a.top = top; a.logit = logit; a.lse = lse;
  a.repetition = 1.f;
  if (rules != nullptr) {
    if (rules->n_masks > 0) {
      a.mask = rules->mask; a.mask_of = rules->mask_of;
      a.n_masks = rules->n_masks; a.mask_words = rules->mask_words;
    }
    if (rules->n_seen > 0) {
      a.seen_ptr = rules->seen_ptr; a.seen = rules->seen; a.n_seen = rules->n_seen;
      a.repetition = rules->repetition; a.presence = rules->presence; a.frequency = rules->frequency;
    }
    if (rules->n_add > 0) {
      a.add_ptr = rules->add_ptr; a.add = rules->add; a.value = rules->value; a.n_add = rules->n_add;
    }
  }
  const size_t need = top_workspace(dt, H, n_rows, V, K, a.n_seen + a.n_add);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))
    return fail(GGNN_ERR_WORKSPACE, "vocab_top needs a 16-byte aligned workspace of %zu bytes (got %zu)", need,
                workspace ? workspace_bytes : (size_t)0);
  a.ws = workspace;
  return device_status(launch_top(dt, H, a, as_stream(stream)), "vocab_top");
}

}  // extern "C"

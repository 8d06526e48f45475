// C-ABI entry points of the token operators: dropout, node states from a token
// table and its gradient, the cross entropy over a vocabulary.  Arguments are
// checked on the host, then the kernels are launched on the caller's stream.
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

ggnn_status check_vocab(int32_t dt, int32_t n_nodes, int32_t H, int32_t n_rows, int32_t V, const void* X,
                        const void* W, const float* bias, const int32_t* node, const int32_t* target,
                        const float* lse) {
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
  CHECK_OPT_PTR(target, "target");
  if (n_rows > 0) CHECK_PTR(lse, "lse");
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

}  // extern "C"

// C ABI of the language model operators: argument checks and launches.
#include <math.h>

#include "zeno_guard.h"
#include "zeno_operators.h"

using zeno::DeviceGuard;
using zeno::Range;
using zeno::Rows;

namespace {

constexpr int64_t kMaxRows = 0x7fffffff, kMaxCols = (int64_t)1 << 30, kMaxWeights = (int64_t)1 << 20, kMaxStride = (int64_t)1 << 44, kMaxVocab = (int64_t)1 << 24;
constexpr int kMaxGroups = 65535;

bool type_ok(int32_t type) { return type == ZENO_F32 || type == ZENO_BF16; }

// Sizes that every call shares: m groups of n rows of cols entries.
zeno_status check_sizes(int32_t m, int64_t n, int64_t cols) {
    if (m < 0 || n < 0 || cols < 1) return ZENO_ERR_INVALID_ARG;
    if (m > kMaxGroups || n > kMaxRows || (int64_t)m * n > kMaxRows || cols > kMaxCols) return ZENO_ERR_UNSUPPORTED;
    return ZENO_OK;
}

int size_of(int32_t type) { return type == ZENO_BF16 ? 2 : 4; }

bool placed(const void *p, int size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }

// Rows of `cols` elements of `size` bytes that do not overlap (with no rows, anything goes).  Inputs may be one group for all (a stride of 0).
bool rows_ok(const zeno_rows *v, int size, int32_t m, int64_t n, int64_t cols, bool input = true) {
    if (!v) return false;
    if (m == 0 || n == 0) return true;
    if (!v->data || !placed(v->data, size)) return false;
    if (n > 1 && (v->row < cols || v->row > kMaxStride)) return false;
    if (m == 1 || (input && v->group == 0)) return true;
    if (v->group < cols || v->group > kMaxStride) return false;
    return v->group >= (n - 1) * (n > 1 ? v->row : 0) + cols || v->row >= (m - 1) * v->group + cols;      // groups, or rows, behind one another
}

Rows rows_of(const zeno_rows *v, int64_t n) {
    Rows r = {};
    if (v) r = Rows{v->data, v->row, v->group, n > 0 ? n : 1};
    return r;
}

bool workspace_ok(const void *p, int64_t bytes, int64_t need) {
    return need == 0 || (p && bytes >= need && reinterpret_cast<uintptr_t>(p) % 16 == 0);
}

int64_t blocks_of(int64_t cols) { return (cols + ZENO_SAVED_BLOCK - 1) / ZENO_SAVED_BLOCK; }

// Runs a launcher on a device; whatever error an earlier call of the caller's left behind is none of this one's.
template <typename F>
zeno_status on_device(int32_t device, F launch) {
    DeviceGuard guard(device);
    if (guard.err != cudaSuccess) return ZENO_ERR_CUDA;
    return launch() == cudaSuccess ? ZENO_OK : ZENO_ERR_CUDA;
}

}  // namespace

extern "C" {

zeno_status zeno_layer_norm(int32_t device, int32_t type, int32_t param_type, const zeno_rows *x, int32_t m, int64_t n,
                            int64_t cols, const void *w, const void *b, int64_t ldw, float eps, const zeno_rows *y,
                            float *mean, float *rstd, void *stream) {
    Range range("zeno_layer_norm");
    if (!type_ok(type) || !type_ok(param_type) || !isfinite(eps) || eps < 0.f) return ZENO_ERR_INVALID_ARG;
    const zeno_status st = check_sizes(m, n, cols);
    if (st != ZENO_OK) return st;
    const int size = size_of(type), wsize = size_of(param_type);
    if (!rows_ok(x, size, m, n, cols) || !rows_ok(y, size, m, n, cols, false) || !w || (ldw != 0 && ldw < cols)) return ZENO_ERR_INVALID_ARG;
    if (!placed(w, wsize) || !placed(b, wsize) || !placed(mean, 4) || !placed(rstd, 4)) return ZENO_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return ZENO_OK;
    zeno::NormArgs a = {rows_of(x, n), rows_of(y, n), m, n, cols, w, b, ldw, eps, mean, rstd};
    return on_device(device, [&] { return zeno::launch_layer_norm(type, param_type, a, static_cast<cudaStream_t>(stream)); });
}

int64_t zeno_layer_norm_gradient_workspace(int32_t m, int64_t n, int64_t cols) {
    return check_sizes(m, n, cols) == ZENO_OK && cols <= kMaxWeights ? zeno::norm_gradient_workspace(m, n, cols) : 0;
}

zeno_status zeno_layer_norm_gradient(int32_t device, int32_t type, int32_t param_type, const zeno_rows *dy, const zeno_rows *x,
                                     const zeno_rows *codes, const zeno_rows *scales, int32_t m, int64_t n, int64_t cols,
                                     const void *w, int64_t ldw, const float *mean, const float *rstd, const zeno_rows *dx,
                                     void *dw, void *db, int64_t ldg, void *workspace, int64_t workspace_bytes, void *stream) {
    Range range("zeno_layer_norm_gradient");
    if (!type_ok(type) || !type_ok(param_type)) return ZENO_ERR_INVALID_ARG;
    const zeno_status st = check_sizes(m, n, cols);
    if (st != ZENO_OK) return st;
    const bool rows = m > 0 && n > 0;
    if (cols > kMaxWeights && (dw || db)) return ZENO_ERR_UNSUPPORTED;
    const int size = size_of(type), wsize = size_of(param_type);
    if (!rows_ok(dy, size, m, n, cols) || (x ? !rows_ok(x, size, m, n, cols) : !rows_ok(codes, 1, m, n, cols) || !rows_ok(scales, 4, m, n, blocks_of(cols))))
        return ZENO_ERR_INVALID_ARG;
    if (!placed(w, wsize) || !placed(dw, wsize) || !placed(db, wsize) || !placed(mean, 4) || !placed(rstd, 4)) return ZENO_ERR_INVALID_ARG;
    if ((rows && (!mean || !rstd)) || (dx && (!rows_ok(dx, size, m, n, cols, false) || !w || (ldw != 0 && ldw < cols)))) return ZENO_ERR_INVALID_ARG;
    if ((dw || db) && m > 1 && ldg < cols) return ZENO_ERR_INVALID_ARG;
    if (!workspace_ok(workspace, workspace_bytes, zeno_layer_norm_gradient_workspace(m, n, cols))) return ZENO_ERR_INVALID_ARG;
    if (m == 0) return ZENO_OK;
    zeno::NormGradArgs a = {rows_of(dy, n), rows_of(x, n), rows_of(x ? nullptr : codes, n), rows_of(x ? nullptr : scales, n), rows_of(dx, n),
                            m, n, cols, w, ldw, mean, rstd, dw, db, ldg, static_cast<float *>(workspace)};
    return on_device(device, [&] { return zeno::launch_layer_norm_gradient(type, param_type, a, static_cast<cudaStream_t>(stream)); });
}

zeno_status zeno_pack_activations(int32_t device, int32_t type, const zeno_rows *x, int32_t m, int64_t n, int64_t cols,
                                  const zeno_rows *codes, const zeno_rows *scales, void *stream) {
    Range range("zeno_pack_activations");
    if (!type_ok(type)) return ZENO_ERR_INVALID_ARG;
    const zeno_status st = check_sizes(m, n, cols);
    if (st != ZENO_OK) return st;
    if (!rows_ok(x, size_of(type), m, n, cols) || !rows_ok(codes, 1, m, n, cols, false) || !rows_ok(scales, 4, m, n, blocks_of(cols), false)) return ZENO_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return ZENO_OK;
    zeno::PackArgs a = {rows_of(x, n), rows_of(codes, n), rows_of(scales, n), m, n, cols};
    return on_device(device, [&] { return zeno::launch_pack(type, a, static_cast<cudaStream_t>(stream)); });
}

// The checks of zeno_dense_gradient that the size of its workspace depends on; fills in everything but the outputs.
static zeno_status check_dense(int32_t type, const zeno_rows *dy, const zeno_rows *codes, const zeno_rows *scales, int32_t m, int64_t n, int64_t inputs,
                               int64_t outputs, zeno::DenseGradArgs *a) {
    if (!type_ok(type)) return ZENO_ERR_INVALID_ARG;
    zeno_status st = check_sizes(m, n, inputs);
    if (st == ZENO_OK) st = check_sizes(m, n, outputs);
    if (st != ZENO_OK) return st;
    if (inputs > kMaxWeights || outputs > kMaxWeights) return ZENO_ERR_UNSUPPORTED;
    if (!rows_ok(dy, size_of(type), m, n, outputs) || !rows_ok(codes, 1, m, n, inputs)) return ZENO_ERR_INVALID_ARG;
    *a = {rows_of(dy, n), rows_of(codes, n), rows_of(scales, n), m, n, inputs, outputs, nullptr, nullptr, 0, 0, nullptr};
    return ZENO_OK;
}

int64_t zeno_dense_gradient_workspace(int32_t type, const zeno_rows *dy, const zeno_rows *codes, int32_t m, int64_t n, int64_t inputs, int64_t outputs) {
    zeno::DenseGradArgs a;
    return check_dense(type, dy, codes, nullptr, m, n, inputs, outputs, &a) == ZENO_OK && m > 0 ? zeno::dense_gradient_workspace(type, a) : 0;
}

zeno_status zeno_dense_gradient(int32_t device, int32_t type, int32_t param_type, const zeno_rows *dy, const zeno_rows *codes,
                                const zeno_rows *scales, int32_t m, int64_t n, int64_t inputs, int64_t outputs, void *dw,
                                int64_t ldw, void *db, int64_t ldb, void *workspace, int64_t workspace_bytes, void *stream) {
    Range range("zeno_dense_gradient");
    if (!type_ok(param_type)) return ZENO_ERR_INVALID_ARG;
    zeno::DenseGradArgs a;
    const zeno_status st = check_dense(type, dy, codes, scales, m, n, inputs, outputs, &a);
    if (st != ZENO_OK) return st;
    if (!rows_ok(scales, 4, m, n, blocks_of(inputs)) || !placed(dw, size_of(param_type)) || !placed(db, size_of(param_type))) return ZENO_ERR_INVALID_ARG;
    if (m == 0) return ZENO_OK;
    if (!dw || (m > 1 && (ldw < inputs * outputs || (db && ldb < outputs)))) return ZENO_ERR_INVALID_ARG;
    if (!workspace_ok(workspace, workspace_bytes, zeno::dense_gradient_workspace(type, a))) return ZENO_ERR_INVALID_ARG;
    a.dw = dw;
    a.db = db;
    a.ldw = ldw;
    a.ldb = ldb;
    a.workspace = static_cast<float *>(workspace);
    return on_device(device, [&] { return zeno::launch_dense_gradient(type, param_type, a, static_cast<cudaStream_t>(stream)); });
}

zeno_status zeno_operator_status(int32_t device, void *stream) {
    DeviceGuard guard(device);
    int status = 0;
    if (guard.err != cudaSuccess || zeno::read_operator_status(device, static_cast<cudaStream_t>(stream), &status) != cudaSuccess) return ZENO_ERR_CUDA;
    return status ? ZENO_ERR_TIMEOUT : ZENO_OK;
}

zeno_status zeno_debug_set_operator_wait_limit(uint32_t polls) {
    zeno::set_operator_wait_limit(polls);
    return ZENO_OK;
}

zeno_status zeno_token_logprobs(int32_t device, int32_t type, const zeno_rows *logits, int32_t m, int64_t n, int64_t vocab,
                                const int32_t *targets, int32_t top, float *logprobs, float *entropy, float *lse,
                                int32_t *top_idx, float *top_logprobs, void *stream) {
    Range range("zeno_token_logprobs");
    if (!type_ok(type) || top < 0 || top > vocab) return ZENO_ERR_INVALID_ARG;
    if (top > ZENO_MAX_TOP) return ZENO_ERR_UNSUPPORTED;
    const zeno_status st = check_sizes(m, n, vocab);
    if (st != ZENO_OK) return st;
    if (!rows_ok(logits, size_of(type), m, n, vocab)) return ZENO_ERR_INVALID_ARG;
    if (!placed(targets, 4) || !placed(logprobs, 4) || !placed(entropy, 4) || !placed(lse, 4) || !placed(top_idx, 4) || !placed(top_logprobs, 4)) return ZENO_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return ZENO_OK;
    if (logprobs && !targets) return ZENO_ERR_INVALID_ARG;
    if (!top_idx && !top_logprobs) top = 0;
    zeno::LogprobArgs a = {rows_of(logits, n), m, n, vocab, targets, top, logprobs, entropy, lse, top_idx, top_logprobs};
    return on_device(device, [&] { return zeno::launch_token_logprobs(type, a, static_cast<cudaStream_t>(stream)); });
}

zeno_status zeno_token_gradient(int32_t device, int32_t type, const zeno_rows *logits, int32_t m, int64_t n, int64_t vocab,
                                const int32_t *targets, const float *lse, const float *entropy, const float *g_logprob,
                                const float *g_entropy, const zeno_rows *grad, void *stream) {
    Range range("zeno_token_gradient");
    if (!type_ok(type)) return ZENO_ERR_INVALID_ARG;
    const zeno_status st = check_sizes(m, n, vocab);
    if (st != ZENO_OK) return st;
    if (!rows_ok(logits, size_of(type), m, n, vocab) || !rows_ok(grad, size_of(type), m, n, vocab, false)) return ZENO_ERR_INVALID_ARG;
    if (!placed(targets, 4) || !placed(lse, 4) || !placed(entropy, 4) || !placed(g_logprob, 4) || !placed(g_entropy, 4)) return ZENO_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return ZENO_OK;
    if (!targets || !lse || !g_logprob || (g_entropy && !entropy)) return ZENO_ERR_INVALID_ARG;
    zeno::TokenGradArgs a = {rows_of(logits, n), rows_of(grad, n), m, n, vocab, targets, lse, entropy, g_logprob, g_entropy};
    return on_device(device, [&] { return zeno::launch_token_gradient(type, a, static_cast<cudaStream_t>(stream)); });
}

// Rows of a table or of output weights, one after the other: a group's begin `ld` entries after the previous group's (0: one matrix for all of them).
static zeno_status check_table(const void *w, int64_t ld, int size, int32_t m, int64_t vocab, int64_t cols, bool shared) {
    if ((!w && m > 0) || !placed(w, size)) return ZENO_ERR_INVALID_ARG;
    if (m > 1 && !(shared && ld == 0) && ld < vocab * cols) return ZENO_ERR_INVALID_ARG;
    return ZENO_OK;
}

static zeno_status check_vocab(int32_t m, int64_t n, int64_t vocab, int64_t cols) {
    if (vocab < 1) return ZENO_ERR_INVALID_ARG;
    const zeno_status st = check_sizes(m, n, cols);
    if (st != ZENO_OK) return st;
    return vocab > kMaxVocab || cols > kMaxWeights ? ZENO_ERR_UNSUPPORTED : ZENO_OK;
}

zeno_status zeno_embed(int32_t device, int32_t type, int32_t param_type, const int32_t *tokens, int32_t m, int64_t n, int64_t vocab, int64_t cols,
                       const void *table, int64_t ldt, float scale, const zeno_rows *y, void *stream) {
    Range range("zeno_embed");
    if (!type_ok(type) || !type_ok(param_type) || !isfinite(scale)) return ZENO_ERR_INVALID_ARG;
    zeno_status st = check_vocab(m, n, vocab, cols);
    if (st == ZENO_OK) st = check_table(table, ldt, size_of(param_type), m, vocab, cols, true);
    if (st != ZENO_OK) return st;
    if (!rows_ok(y, size_of(type), m, n, cols, false) || !placed(tokens, 4)) return ZENO_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return ZENO_OK;
    if (!tokens) return ZENO_ERR_INVALID_ARG;
    zeno::EmbedArgs a = {tokens, m, n, vocab, cols, table, m > 1 ? ldt : 0, scale, rows_of(y, n)};
    return on_device(device, [&] { return zeno::launch_embed(type, param_type, a, static_cast<cudaStream_t>(stream)); });
}

int64_t zeno_embed_gradient_workspace(int32_t m, int64_t n, int64_t vocab, int64_t cols) {
    return check_vocab(m, n, vocab, cols) == ZENO_OK && m > 0 ? zeno::embed_gradient_workspace(m, n, vocab, cols) : 0;
}

zeno_status zeno_embed_gradient(int32_t device, int32_t type, int32_t param_type, const int32_t *tokens, const zeno_rows *dy, int32_t m, int64_t n,
                                int64_t vocab, int64_t cols, float scale, int32_t add, void *dtable, int64_t ldt, void *workspace, int64_t workspace_bytes,
                                void *stream) {
    Range range("zeno_embed_gradient");
    if (!type_ok(type) || !type_ok(param_type) || !isfinite(scale)) return ZENO_ERR_INVALID_ARG;
    zeno_status st = check_vocab(m, n, vocab, cols);
    if (st != ZENO_OK) return st;
    if (!rows_ok(dy, size_of(type), m, n, cols) || !placed(tokens, 4) || (m > 0 && n > 0 && !tokens)) return ZENO_ERR_INVALID_ARG;
    if (m == 0) return ZENO_OK;
    st = check_table(dtable, ldt, size_of(param_type), m, vocab, cols, false);
    if (st != ZENO_OK) return st;
    if (!workspace_ok(workspace, workspace_bytes, zeno::embed_gradient_workspace(m, n, vocab, cols))) return ZENO_ERR_INVALID_ARG;
    if (!zeno::embed_gradient_fits(n, vocab, cols)) return ZENO_ERR_UNSUPPORTED;
    zeno::EmbedGradArgs a = {tokens, rows_of(dy, n), m, n, vocab, cols, scale, add != 0, dtable, ldt, workspace};
    return on_device(device, [&] { return zeno::launch_embed_gradient(type, param_type, a, static_cast<cudaStream_t>(stream)); });
}

// The checks of the log probabilities from hidden states that the size of the workspace depends on; fills in what it goes by.
static zeno_status check_head(int32_t type, int32_t param_type, int32_t m, int64_t n, int64_t cols, int64_t vocab, const void *w, int64_t ldw,
                              zeno::HeadArgs *a) {
    if (!type_ok(type) || !type_ok(param_type)) return ZENO_ERR_INVALID_ARG;
    zeno_status st = check_vocab(m, n, vocab, cols);
    if (st == ZENO_OK) st = check_table(w, ldw, size_of(param_type), m, vocab, cols, true);
    if (st != ZENO_OK) return st;
    if ((int64_t)m * ((n + 255) / 256 * 256) > kMaxRows - 256) return ZENO_ERR_UNSUPPORTED;
    *a = {};
    a->m = m;
    a->n = n;
    a->cols = cols;
    a->vocab = vocab;
    a->w = w;
    a->ldw = m > 1 ? ldw : 0;
    return ZENO_OK;
}

int64_t zeno_linear_logprobs_workspace(int32_t type, int32_t param_type, int32_t m, int64_t n, int64_t cols, int64_t vocab, const void *w, int64_t ldw) {
    zeno::HeadArgs a;
    return check_head(type, param_type, m, n, cols, vocab, w, ldw, &a) == ZENO_OK ? zeno::head_workspace(type, param_type, false, a) : 0;
}

zeno_status zeno_linear_logprobs(int32_t device, int32_t type, int32_t param_type, const zeno_rows *x, int32_t m, int64_t n, int64_t cols, int64_t vocab,
                                 const void *w, int64_t ldw, const int32_t *targets, float scale, float *logprobs, float *lse, void *workspace,
                                 int64_t workspace_bytes, void *stream) {
    Range range("zeno_linear_logprobs");
    if (!isfinite(scale)) return ZENO_ERR_INVALID_ARG;
    zeno::HeadArgs a;
    const zeno_status st = check_head(type, param_type, m, n, cols, vocab, w, ldw, &a);
    if (st != ZENO_OK) return st;
    if (!rows_ok(x, size_of(type), m, n, cols) || !placed(targets, 4) || !placed(logprobs, 4) || !placed(lse, 4)) return ZENO_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return ZENO_OK;
    if (!targets || !workspace_ok(workspace, workspace_bytes, zeno::head_workspace(type, param_type, false, a))) return ZENO_ERR_INVALID_ARG;
    a.x = rows_of(x, n);
    a.targets = targets;
    a.scale = scale;
    a.logprobs = logprobs;
    a.lse = lse;
    a.workspace = workspace;
    return on_device(device, [&] { return zeno::launch_head_logprobs(type, param_type, a, static_cast<cudaStream_t>(stream)); });
}

int64_t zeno_linear_logprobs_gradient_workspace(int32_t type, int32_t param_type, int32_t m, int64_t n, int64_t cols, int64_t vocab, const void *w,
                                                int64_t ldw, int32_t want_dx) {
    zeno::HeadArgs a;
    if (check_head(type, param_type, m, n, cols, vocab, w, ldw, &a) != ZENO_OK) return 0;
    a.dx.data = want_dx ? &a : nullptr;
    return zeno::head_workspace(type, param_type, true, a);
}

zeno_status zeno_linear_logprobs_gradient(int32_t device, int32_t type, int32_t param_type, const zeno_rows *x, int32_t m, int64_t n, int64_t cols,
                                          int64_t vocab, const void *w, int64_t ldw, const int32_t *targets, float scale, const float *lse,
                                          const float *g_logprob, const zeno_rows *dx, void *dw, int64_t lddw, void *workspace, int64_t workspace_bytes,
                                          void *stream) {
    Range range("zeno_linear_logprobs_gradient");
    if (!isfinite(scale)) return ZENO_ERR_INVALID_ARG;
    zeno::HeadArgs a;
    zeno_status st = check_head(type, param_type, m, n, cols, vocab, w, ldw, &a);
    if (st != ZENO_OK) return st;
    if (!rows_ok(x, size_of(type), m, n, cols) || (dx && !rows_ok(dx, size_of(type), m, n, cols, false))) return ZENO_ERR_INVALID_ARG;
    if (!placed(targets, 4) || !placed(lse, 4) || !placed(g_logprob, 4)) return ZENO_ERR_INVALID_ARG;
    if (m > 0 && n > 0 && (!targets || !lse || !g_logprob)) return ZENO_ERR_INVALID_ARG;
    if (m == 0) return ZENO_OK;
    if (dw) {
        st = check_table(dw, lddw, size_of(param_type), m, vocab, cols, false);
        if (st != ZENO_OK) return st;
    }
    a.dx.data = dx && n > 0 ? &a : nullptr;
    if (!workspace_ok(workspace, workspace_bytes, zeno::head_workspace(type, param_type, true, a))) return ZENO_ERR_INVALID_ARG;
    if (!dw && (!dx || n == 0)) return ZENO_OK;
    a.x = rows_of(x, n);
    a.dx = rows_of(dx, n);
    a.targets = targets;
    a.scale = scale;
    a.lse_in = lse;
    a.g = g_logprob;
    a.dw = dw;
    a.lddw = lddw;
    a.workspace = workspace;
    return on_device(device, [&] { return zeno::launch_head_gradient(type, param_type, a, static_cast<cudaStream_t>(stream)); });
}

}  // extern "C"

// echo_ops_host.cpp -- C entry points of the training-step operators (echo_ops.h): argument checks,
// the device guard and the launches.  Nothing here allocates device memory or waits.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "echo.h"
#include "echo_internal.h"
#include "echo_ops.h"
#include "echo_ops_internal.h"

using namespace echo;

namespace {

constexpr int64_t kMaxRows = INT32_MAX;
constexpr int64_t kMaxCols = int64_t(1) << 24;
constexpr int64_t kMaxElements = int64_t(1) << 38; // grids stay below 2^32 work-items
constexpr int64_t kMaxSorted = int64_t(1) << 26;   // rows of a table whose gradient's tokens are sorted
// Tokens of a table's gradient: a wavefront sums at least 32 of them over at least 256 columns, so at most 1.5 * 2^25
// wavefronts (of rows * cols <= 2^38) and those that write zeros stay below 2^32 work-items.
constexpr int64_t kMaxTokens = int64_t(1) << 29;
// Every sorting workgroup, one for 64 rows of the table, reads every id twice: 2^20 tokens and 2^18 rows take 5.4 ms, and a
// launch at this bound some tenths of a second.  Sizes allowed one by one would take minutes.
constexpr int64_t kMaxSortWork = int64_t(1) << 42;
constexpr int64_t kMaxStride = int64_t(1) << 28;   // 2^31 rows of 4-byte elements stay below 2^62 bytes

int64_t elem(int32_t type) { return type == ECHO_F32 ? 4 : 2; }
bool is_type(int32_t t) { return t == ECHO_F32 || t == ECHO_F16 || t == ECHO_BF16; }

// The bytes of an argument: rows of `width` bytes, `pitch` apart.  `same`: an output that may be exactly an input of
// the same layout; such pairs carry the same nonzero number.
struct Span {
    const char *name;
    const void *p;
    int64_t rows, width, pitch;
    int same;
    int64_t bytes() const { return rows > 0 && width > 0 ? (rows - 1) * pitch + width : 0; }
};
Span matrix(const char *name, const void *p, int64_t rows, int64_t cols, int64_t stride, int64_t e, int same = 0) {
    return {name, p, rows, cols * e, stride * e, same};
}
Span vector(const char *name, const void *p, int64_t n, int64_t e) { return {name, p, 1, n * e, 0, 0}; }
// Whether two arguments share a byte.  Rows of one pitch may lie in each other's gaps; of two pitches that are not the same
// the whole spans have to be apart.
bool meet(const Span &a, const Span &b) {
    const int64_t m = a.bytes(), n = b.bytes();
    if (!a.p || !b.p || m <= 0 || n <= 0) return false;
    const uintptr_t p = (uintptr_t)a.p, q = (uintptr_t)b.p;
    if (p >= q + (uintptr_t)n || q >= p + (uintptr_t)m) return false;
    const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch;
    if (pitch <= 0 || (b.rows > 1 && b.pitch != pitch)) return true;
    // how far into a's rows b's begin
    const int64_t by = p <= q ? (int64_t)(q - p) % pitch : (pitch - (int64_t)(p - q) % pitch) % pitch;
    return by < a.width || by + b.width > pitch;
}
// Every output against every input and every other output.
int check_spans(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
    for (const Span *o = outs.begin(); o != outs.end(); ++o) {
        for (const Span *q = outs.begin(); q != o; ++q)
            if (meet(*o, *q)) return set_error(ECHO_ERR_ARG, "%s and %s overlap", o->name, q->name);
        for (const Span &i : ins)
            if (meet(*o, i) && !(o->same && (o->same & i.same) && o->p == i.p && o->bytes() == i.bytes()))
                return set_error(ECHO_ERR_ARG, "%s overlaps %s", o->name, i.name);
    }
    return ECHO_OK;
}

int check_matrix(const char *name, const void *p, int64_t rows, int64_t stride, int64_t e) {
    if (rows && !p) return set_error(ECHO_ERR_ARG, "%s is null", name);
    if (stride < 0 || stride > kMaxStride)
        return set_error(ECHO_ERR_ARG, "%s: row stride %lld outside [0, 2^28]", name, (long long)stride);
    if ((uintptr_t)p % (uintptr_t)e) return set_error(ECHO_ERR_ARG, "%s is not aligned to its elements", name);
    return ECHO_OK;
}
int check_vector(const char *name, const void *p, int64_t e, bool required) {
    if (required && !p) return set_error(ECHO_ERR_ARG, "%s is null", name);
    if ((uintptr_t)p % (uintptr_t)e) return set_error(ECHO_ERR_ARG, "%s is not aligned to its elements", name);
    return ECHO_OK;
}
int check_sizes(int64_t rows, int64_t cols) {
    if (rows < 0 || rows > kMaxRows) return set_error(ECHO_ERR_ARG, "rows = %lld outside [0, 2^31)", (long long)rows);
    if (cols < 1 || cols > kMaxCols) return set_error(ECHO_ERR_ARG, "cols = %lld outside [1, 2^24]", (long long)cols);
    if (rows * cols > kMaxElements)
        return set_error(ECHO_ERR_RANGE, "%lld rows of %lld pass 2^38 elements", (long long)rows, (long long)cols);
    return ECHO_OK;
}
int check_types(int32_t type, int32_t other, const char *what) {
    if (!is_type(type)) return set_error(ECHO_ERR_ARG, "unknown element type %d", type);
    if (other != type && other != ECHO_F32)
        return set_error(ECHO_ERR_ARG, "%s must be the activations' type or 32 bits (got %d)", what, other);
    return ECHO_OK;
}
int check_index(int32_t index_type) {
    if (index_type != ECHO_I32 && index_type != ECHO_I64)
        return set_error(ECHO_ERR_ARG, "unknown index type %d", index_type);
    return ECHO_OK;
}
int check_shard(int64_t start, int64_t n) {
    if (start < 0 || n < 0 || n > kMaxRows || start > INT64_MAX - n)
        return set_error(ECHO_ERR_ARG, "vocabulary shard [%lld, +%lld) out of range", (long long)start, (long long)n);
    return ECHO_OK;
}
int check_shard_of(int64_t start, int64_t n, int64_t whole) {
    const int rc = check_shard(start, n);
    if (rc == ECHO_OK && start + n > whole)
        return set_error(ECHO_ERR_ARG, "vocabulary shard [%lld, +%lld) passes the vocabulary of %lld",
                         (long long)start, (long long)n, (long long)whole);
    return rc;
}
int check_workspace(const void *p, int64_t bytes, int64_t need) {
    if (need && (!p || bytes < need))
        return set_error(ECHO_ERR_ARG, "workspace holds %lld bytes, needs %lld", (long long)(p ? bytes : 0),
                         (long long)need);
    if ((uintptr_t)p % 16) return set_error(ECHO_ERR_ARG, "workspace is not aligned to 16 bytes");
    return ECHO_OK;
}

constexpr int64_t kMaxTop = 1024;
constexpr int64_t kMaxHeadRows = int64_t(1) << 24, kMaxHidden = int64_t(1) << 20;

int check_teacher(const void *ids, int32_t index_type, const void *teacher, int32_t teacher_type, int32_t type, int64_t rows,
                  int64_t top, float temperature) {
    if (teacher_type != type && teacher_type != ECHO_F32)
        return set_error(ECHO_ERR_ARG, "teacher_type must be the activations' type or 32 bits (got %d)", teacher_type);
    if (top < 1 || top > kMaxTop) return set_error(ECHO_ERR_ARG, "top = %lld outside [1, 1024]", (long long)top);
    if (!(temperature >= 1e-6f && temperature <= 1e6f))
        return set_error(ECHO_ERR_ARG, "temperature %g outside [1e-6, 1e6]", (double)temperature);
    const int rc = check_vector("ids", ids, index_type == ECHO_I64 ? 8 : 4, rows > 0);
    return rc != ECHO_OK ? rc : check_vector("teacher", teacher, elem(teacher_type), rows > 0);
}
int check_head_sizes(int64_t rows, int64_t cols, int64_t vocab) {
    if (rows < 0 || rows > kMaxHeadRows) return set_error(ECHO_ERR_ARG, "rows = %lld outside [0, 2^24]", (long long)rows);
    if (cols < 1 || cols > kMaxHidden) return set_error(ECHO_ERR_ARG, "cols = %lld outside [1, 2^20]", (long long)cols);
    if (vocab < 1 || vocab > kMaxHeadRows) return set_error(ECHO_ERR_ARG, "vocab = %lld outside [1, 2^24]", (long long)vocab);
    if (rows * cols > kMaxElements || rows * vocab > kMaxElements || vocab * cols > kMaxElements)
        return set_error(ECHO_ERR_RANGE, "%lld rows of %lld over %lld ids: a product passes 2^38", (long long)rows, (long long)cols,
                         (long long)vocab);
    return ECHO_OK;
}

// Runs f on GPU `device` and leaves the thread's current device as it was.
template <class F>
int on_device(int device, const char *what, F f) {
    int before = -1;
    hipError_t e = hipGetDevice(&before);
    if (e != hipSuccess) return set_error(ECHO_ERR_HIP, "hipGetDevice: %s", hipGetErrorString(e));
    if (before != device && (e = hipSetDevice(device)) != hipSuccess)
        return set_error(ECHO_ERR_HIP, "hipSetDevice(%d): %s", device, hipGetErrorString(e));
    e = f();
    if (before != device) (void)hipSetDevice(before);
    if (e != hipSuccess) return set_error(ECHO_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return ECHO_OK;
}

#define ECHO_TRY(call)                 \
    do {                               \
        const int rc_ = (call);        \
        if (rc_ != ECHO_OK) return rc_; \
    } while (0)

}  // namespace

extern "C" {

int echo_layer_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                    const void *weight, const void *bias, int32_t type, int32_t weight_type, int64_t rows,
                    int64_t cols, float eps, void *y, void *sum, float *mean, float *rstd, int hip_device,
                    void *hip_stream) {
    clear_error();
    ECHO_TRY(check_types(type, weight_type, "weight_type"));
    ECHO_TRY(check_sizes(rows, cols));
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return set_error(ECHO_ERR_ARG, "eps must be finite and >= 0");
    const int64_t e = elem(type), we = elem(weight_type);
    const int64_t live = residual ? rows : 0;
    ECHO_TRY(check_matrix("x", x, rows, x_stride, e));
    ECHO_TRY(check_matrix("residual", residual, live, residual ? residual_stride : 0, e));
    ECHO_TRY(check_vector("weight", weight, we, rows > 0));
    ECHO_TRY(check_vector("bias", bias, we, false));
    ECHO_TRY(check_matrix("y", y, rows, cols, e));
    if (rows && !residual != !sum) return set_error(ECHO_ERR_ARG, "sum is given exactly when residual is");
    ECHO_TRY(check_matrix("sum", sum, live, cols, e));
    ECHO_TRY(check_vector("mean", mean, 4, rows > 0));
    ECHO_TRY(check_vector("rstd", rstd, 4, rows > 0));
    ECHO_TRY(check_spans({matrix("y", y, rows, cols, cols, e), matrix("sum", sum, live, cols, cols, e, 1), vector("mean", mean, rows, 4),
                          vector("rstd", rstd, rows, 4)},
                         {matrix("x", x, rows, cols, x_stride, e, rows < 2 || x_stride == cols),
                          matrix("residual", residual, live, cols, residual_stride, e, rows < 2 || residual_stride == cols),
                          vector("weight", weight, cols, we), vector("bias", bias, cols, we)}));
    if (!rows) return ECHO_OK;
    const NormArgs a{x, residual, weight, bias, x_stride, residual_stride, rows, (int)cols, eps, y, sum, mean, rstd};
    return on_device(hip_device, "layer norm", [&] {
        return launch_norm(a, type, weight_type, static_cast<hipStream_t>(hip_stream));
    });
}

int64_t echo_layer_norm_grad_workspace(int64_t rows, int64_t cols) {
    if (rows < 0 || rows > kMaxRows || cols < 1 || cols > kMaxCols) return 0;
    return (int64_t)norm_grad_parts(rows, cols) * 2 * cols * 4;
}

int echo_layer_norm_grad(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *weight,
                         const float *mean, const float *rstd, const void *grad_residual,
                         int64_t grad_residual_stride, int32_t type, int32_t weight_type, int64_t rows, int64_t cols,
                         void *dx, void *dweight, void *dbias, int32_t grad_type, int32_t accumulate,
                         void *workspace, int64_t workspace_bytes, int hip_device, void *hip_stream) {
    clear_error();
    ECHO_TRY(check_types(type, weight_type, "weight_type"));
    if (grad_type != weight_type && grad_type != ECHO_F32)
        return set_error(ECHO_ERR_ARG, "grad_type must be the weight's type or 32 bits (got %d)", grad_type);
    ECHO_TRY(check_sizes(rows, cols));
    const int64_t e = elem(type), we = elem(weight_type), ge = elem(grad_type);
    const int64_t live = grad_residual ? rows : 0;
    ECHO_TRY(check_matrix("dy", dy, rows, dy_stride, e));
    ECHO_TRY(check_matrix("x", x, rows, x_stride, e));
    ECHO_TRY(check_matrix("grad_residual", grad_residual, live, grad_residual ? grad_residual_stride : 0, e));
    ECHO_TRY(check_vector("weight", weight, we, rows > 0));
    ECHO_TRY(check_vector("mean", mean, 4, rows > 0));
    ECHO_TRY(check_vector("rstd", rstd, 4, rows > 0));
    ECHO_TRY(check_matrix("dx", dx, rows, cols, e));
    ECHO_TRY(check_vector("dweight", dweight, ge, true));
    ECHO_TRY(check_vector("dbias", dbias, ge, false));
    const int64_t need = echo_layer_norm_grad_workspace(rows, cols);
    ECHO_TRY(check_workspace(workspace, workspace_bytes, need));
    ECHO_TRY(check_spans({matrix("dx", dx, rows, cols, cols, e, 1), vector("dweight", dweight, cols, ge),
                          vector("dbias", dbias, cols, ge), vector("workspace", workspace, need, 1)},
                         {matrix("dy", dy, rows, cols, dy_stride, e, rows < 2 || dy_stride == cols),
                          matrix("x", x, rows, cols, x_stride, e),
                          matrix("grad_residual", grad_residual, live, cols, grad_residual_stride, e, rows < 2 || grad_residual_stride == cols),
                          vector("weight", weight, cols, we), vector("mean", mean, rows, 4), vector("rstd", rstd, rows, 4)}));
    const NormGradArgs a{dy, x, weight, grad_residual, mean, rstd, dy_stride, x_stride, grad_residual_stride, rows,
                         (int)cols, dx, dweight, dbias, static_cast<float *>(workspace), norm_grad_parts(rows, cols),
                         accumulate != 0};
    return on_device(hip_device, "layer norm gradient", [&] {
        return launch_norm_grad(a, type, weight_type, grad_type, static_cast<hipStream_t>(hip_stream));
    });
}

int echo_embedding(const void *ids, int32_t index_type, const void *weight, int64_t weight_stride, int32_t type,
                   int64_t rows, int64_t cols, int64_t vocab_start, int64_t vocab, float scale, void *out,
                   int hip_device, void *hip_stream) {
    clear_error();
    ECHO_TRY(check_types(type, type, "type"));
    ECHO_TRY(check_index(index_type));
    ECHO_TRY(check_sizes(rows, cols));
    ECHO_TRY(check_shard(vocab_start, vocab));
    const int64_t e = elem(type), ie = index_type == ECHO_I64 ? 8 : 4;
    ECHO_TRY(check_vector("ids", ids, ie, rows > 0));
    ECHO_TRY(check_matrix("weight", weight, rows ? vocab : 0, weight_stride, e));
    ECHO_TRY(check_matrix("out", out, rows, cols, e));
    ECHO_TRY(check_spans({matrix("out", out, rows, cols, cols, e)},
                         {vector("ids", ids, rows, ie), matrix("weight", weight, vocab, cols, weight_stride, e)}));
    if (!rows) return ECHO_OK;
    const EmbedArgs a{ids, weight, weight_stride, rows, vocab_start, (int)cols, (int)vocab, scale, out};
    return on_device(hip_device, "embedding", [&] {
        return launch_embed(a, type, index_type, static_cast<hipStream_t>(hip_stream));
    });
}

int64_t echo_embedding_grad_workspace(int64_t rows, int64_t cols, int64_t vocab) {
    if (rows < 0 || rows > kMaxRows || cols < 1 || cols > kMaxCols || vocab < 0 || vocab > kMaxSorted) return 0;
    return embed_grad_bytes(rows, cols, vocab);
}

int echo_embedding_grad(const void *ids, int32_t index_type, const void *dy, int64_t dy_stride, int32_t type,
                        int64_t rows, int64_t cols, int64_t vocab_start, int64_t vocab, float scale, void *dweight,
                        int32_t grad_type, int32_t accumulate, void *workspace, int64_t workspace_bytes,
                        int hip_device, void *hip_stream) {
    clear_error();
    ECHO_TRY(check_types(type, grad_type, "grad_type"));
    ECHO_TRY(check_index(index_type));
    ECHO_TRY(check_sizes(rows, cols));
    ECHO_TRY(check_shard(vocab_start, vocab));
    const int64_t e = elem(type), ge = elem(grad_type), ie = index_type == ECHO_I64 ? 8 : 4;
    ECHO_TRY(check_vector("ids", ids, ie, rows > 0));
    ECHO_TRY(check_matrix("dy", dy, rows, dy_stride, e));
    ECHO_TRY(check_matrix("dweight", dweight, vocab, cols, ge));
    if (vocab > kMaxSorted) return set_error(ECHO_ERR_RANGE, "vocab = %lld passes 2^26", (long long)vocab);
    if (rows > kMaxTokens) return set_error(ECHO_ERR_RANGE, "rows = %lld pass 2^29", (long long)rows);
    if (rows * vocab > kMaxSortWork)
        return set_error(ECHO_ERR_RANGE, "%lld tokens times %lld rows pass 2^42", (long long)rows, (long long)vocab);
    const int64_t need = echo_embedding_grad_workspace(rows, cols, vocab);
    ECHO_TRY(check_workspace(workspace, workspace_bytes, need));
    ECHO_TRY(check_spans({vector("dweight", dweight, vocab * cols, ge), vector("workspace", workspace, need, 1)},
                         {vector("ids", ids, rows, ie), matrix("dy", dy, rows, cols, dy_stride, e)}));
    if (!vocab || (!rows && accumulate)) return ECHO_OK;
    const EmbedGradArgs a{ids, dy, dy_stride, rows, vocab_start, (int)cols, (int)vocab, scale, dweight,
                          accumulate != 0, workspace};
    return on_device(hip_device, "embedding gradient", [&] {
        return launch_embed_grad(a, type, index_type, grad_type, static_cast<hipStream_t>(hip_stream));
    });
}

int echo_cross_entropy(const void *logits, int64_t logits_stride, int32_t type, const void *targets,
                       int32_t index_type, int64_t rows, int64_t cols, int64_t vocab_start, int64_t vocab_size,
                       float *lse, float *target, float *loss, const float *grad_loss, void *grad,
                       int64_t grad_stride, int hip_device, void *hip_stream) {
    clear_error();
    ECHO_TRY(check_types(type, type, "type"));
    ECHO_TRY(check_index(index_type));
    ECHO_TRY(check_sizes(rows, cols));
    ECHO_TRY(check_shard_of(vocab_start, cols, vocab_size));
    const bool whole = vocab_start == 0 && vocab_size == cols;
    if (!whole && (loss || grad))
        return set_error(ECHO_ERR_ARG, "loss and grad need the whole vocabulary; a shard gives lse and target");
    if (rows && !lse && !target && !loss && !grad) return set_error(ECHO_ERR_ARG, "no output is asked for");
    if (rows && !grad != !grad_loss) return set_error(ECHO_ERR_ARG, "grad_loss is given exactly when grad is");
    const int64_t e = elem(type), ie = index_type == ECHO_I64 ? 8 : 4, live = grad ? rows : 0;
    ECHO_TRY(check_matrix("logits", logits, rows, logits_stride, e));
    ECHO_TRY(check_vector("targets", targets, ie, rows > 0));
    ECHO_TRY(check_vector("lse", lse, 4, false));
    ECHO_TRY(check_vector("target", target, 4, false));
    ECHO_TRY(check_vector("loss", loss, 4, false));
    ECHO_TRY(check_vector("grad_loss", grad_loss, 4, false));
    ECHO_TRY(check_matrix("grad", grad, live, grad ? grad_stride : 0, e));
    if (live > 1 && grad_stride < cols) return set_error(ECHO_ERR_ARG, "rows of grad overlap");
    const bool dense = rows < 2 || logits_stride == grad_stride;
    ECHO_TRY(check_spans({matrix("grad", grad, live, cols, grad_stride, e, 1), vector("lse", lse, rows, 4),
                          vector("target", target, rows, 4), vector("loss", loss, rows, 4)},
                         {matrix("logits", logits, rows, cols, logits_stride, e, dense),
                          vector("targets", targets, rows, ie), vector("grad_loss", grad_loss, rows, 4)}));
    if (!rows) return ECHO_OK;
    const LossArgs a{logits, targets, logits_stride, rows, vocab_start, vocab_size, (int)cols, lse, target, loss,
                     nullptr, grad_loss, grad, grad_stride};
    return on_device(hip_device, "cross entropy", [&] {
        return launch_loss(a, type, index_type, static_cast<hipStream_t>(hip_stream));
    });
}

int echo_cross_entropy_grad(const void *logits, int64_t logits_stride, int32_t type, const void *targets,
                            int32_t index_type, int64_t rows, int64_t cols, int64_t vocab_start, int64_t vocab_size,
                            const float *lse, const float *grad_loss, void *grad, int64_t grad_stride,
                            int hip_device, void *hip_stream) {
    clear_error();
    ECHO_TRY(check_types(type, type, "type"));
    ECHO_TRY(check_index(index_type));
    ECHO_TRY(check_sizes(rows, cols));
    ECHO_TRY(check_shard_of(vocab_start, cols, vocab_size));
    const int64_t e = elem(type), ie = index_type == ECHO_I64 ? 8 : 4;
    ECHO_TRY(check_matrix("logits", logits, rows, logits_stride, e));
    ECHO_TRY(check_vector("targets", targets, ie, rows > 0));
    ECHO_TRY(check_vector("lse", lse, 4, rows > 0));
    ECHO_TRY(check_vector("grad_loss", grad_loss, 4, rows > 0));
    ECHO_TRY(check_matrix("grad", grad, rows, grad_stride, e));
    if (rows > 1 && grad_stride < cols) return set_error(ECHO_ERR_ARG, "rows of grad overlap");
    const bool dense = rows < 2 || logits_stride == grad_stride;
    ECHO_TRY(check_spans({matrix("grad", grad, rows, cols, grad_stride, e, 1)},
                         {matrix("logits", logits, rows, cols, logits_stride, e, dense),
                          vector("targets", targets, rows, ie), vector("lse", lse, rows, 4),
                          vector("grad_loss", grad_loss, rows, 4)}));
    if (!rows) return ECHO_OK;
    const LossArgs a{logits, targets, logits_stride, rows, vocab_start, vocab_size, (int)cols, nullptr, nullptr,
                     nullptr, lse, grad_loss, grad, grad_stride};
    return on_device(hip_device, "cross entropy gradient", [&] {
        return launch_loss_grad(a, type, index_type, static_cast<hipStream_t>(hip_stream));
    });
}

}  // extern "C"

namespace {

// Loss (lse_in null) and gradient of distillation.
int distill(DistillArgs a, int32_t type, int32_t index_type, int32_t teacher_type, int64_t cols, int64_t top, bool grads,
            int hip_device, void *hip_stream, const char *what) {
    ECHO_TRY(check_types(type, type, "type"));
    ECHO_TRY(check_index(index_type));
    ECHO_TRY(check_sizes(a.rows, cols));
    ECHO_TRY(check_teacher(a.ids, index_type, a.teacher, teacher_type, type, a.rows, top, a.temperature));
    ECHO_TRY(check_shard_of(a.vocab_start, cols, a.vocab_size));
    const bool whole = a.vocab_start == 0 && a.vocab_size == cols, only_grad = grads;
    if (!only_grad) {
        if (!whole && (a.loss || a.grad))
            return set_error(ECHO_ERR_ARG, "loss and grad need the whole vocabulary; a shard gives lse, target and entropy");
        if (a.rows && !a.lse && !a.target && !a.entropy && !a.loss && !a.grad)
            return set_error(ECHO_ERR_ARG, "no output is asked for");
        if (a.rows && !a.grad != !a.grad_loss) return set_error(ECHO_ERR_ARG, "grad_loss is given exactly when grad is");
    }
    const int64_t e = elem(type), ie = index_type == ECHO_I64 ? 8 : 4, live = only_grad || a.grad ? a.rows : 0;
    ECHO_TRY(check_matrix("logits", a.logits, a.rows, a.logits_stride, e));
    ECHO_TRY(check_vector("lse", only_grad ? a.lse_in : a.lse, 4, only_grad && a.rows > 0));
    ECHO_TRY(check_vector("target", a.target, 4, false));
    ECHO_TRY(check_vector("entropy", a.entropy, 4, false));
    ECHO_TRY(check_vector("loss", a.loss, 4, false));
    ECHO_TRY(check_vector("grad_loss", a.grad_loss, 4, live > 0));
    ECHO_TRY(check_matrix("grad", a.grad, live, live ? a.grad_stride : 0, e));
    if (live > 1 && a.grad_stride < cols) return set_error(ECHO_ERR_ARG, "rows of grad overlap");
    const bool dense = a.rows < 2 || a.logits_stride == a.grad_stride;
    ECHO_TRY(check_spans({matrix("grad", a.grad, live, cols, a.grad_stride, e, 1), vector("lse", a.lse, a.rows, 4),
                          vector("target", a.target, a.rows, 4), vector("entropy", a.entropy, a.rows, 4),
                          vector("loss", a.loss, a.rows, 4)},
                         {matrix("logits", a.logits, a.rows, cols, a.logits_stride, e, dense),
                          vector("ids", a.ids, a.rows * top, ie), vector("teacher", a.teacher, a.rows * top, elem(teacher_type)),
                          vector("lse", a.lse_in, a.rows, 4), vector("grad_loss", a.grad_loss, a.rows, 4)}));
    if (!a.rows) return ECHO_OK;
    a.cols = (int)cols;
    a.top = (int)top;
    a.inv_t = 1.0f / a.temperature;
    a.k2 = a.inv_t * 1.44269504088896341f;
    return on_device(hip_device, what, [&] {
        return launch_distill(a, type, static_cast<hipStream_t>(hip_stream));
    });
}

// The head's four calls; top is 0 with one target a row.
int linear(LinearArgs a, int64_t cols, int64_t vocab, int64_t top, int64_t workspace_bytes, int hip_device, void *hip_stream,
           const char *what) {
    const bool teacher = top != 0;
    ECHO_TRY(check_types(a.type, a.type, "type"));
    ECHO_TRY(check_index(a.index_type));
    ECHO_TRY(check_head_sizes(a.rows, cols, vocab));
    if (teacher)
        ECHO_TRY(check_teacher(a.targets, a.index_type, a.teacher, a.teacher_type, a.type, a.rows, top, a.temperature));
    else
        ECHO_TRY(check_vector("targets", a.targets, a.index_type == ECHO_I64 ? 8 : 4, a.rows > 0));
    ECHO_TRY(check_shard_of(a.vocab_start, vocab, a.vocab_size));
    a.cols = (int)cols;
    a.vocab = (int)vocab;
    a.top = (int)top;
    const bool whole = a.vocab_start == 0 && a.vocab_size == vocab;
    if (a.forward) {
        if (!whole && (a.loss || a.dhidden || a.dweight))
            return set_error(ECHO_ERR_ARG, "loss and gradients need the whole vocabulary; a shard gives its statistics");
        if (a.rows && !a.lse && !a.target && !a.entropy && !a.loss && !a.dweight)
            return set_error(ECHO_ERR_ARG, "no output is asked for");
        a.grads = a.dweight != nullptr;
        if (a.rows && (!a.dhidden != !a.dweight || !a.grad_loss != !a.dweight))
            return set_error(ECHO_ERR_ARG, "grad_loss, dhidden and dweight are given together");
        if (a.rows && a.grads && !a.lse) return set_error(ECHO_ERR_ARG, "gradients need lse");
    }
    const int64_t e = elem(a.type), ie = a.index_type == ECHO_I64 ? 8 : 4, live = a.grads ? a.rows : 0;
    if (a.grads && a.grad_type != a.type && a.grad_type != ECHO_F32)
        return set_error(ECHO_ERR_ARG, "grad_type must be the activations' type or 32 bits (got %d)", a.grad_type);
    const int64_t ge = elem(a.grad_type);
    ECHO_TRY(check_matrix("hidden", a.hidden, a.rows, a.hidden_stride, e));
    ECHO_TRY(check_matrix("weight", a.weight, a.rows ? vocab : 0, a.weight_stride, e));
    ECHO_TRY(check_vector("lse", a.forward ? a.lse : a.lse_in, 4, !a.forward && a.rows > 0));
    ECHO_TRY(check_vector("target", a.target, 4, false));
    ECHO_TRY(check_vector("entropy", a.entropy, 4, false));
    ECHO_TRY(check_vector("loss", a.loss, 4, false));
    ECHO_TRY(check_vector("grad_loss", a.grad_loss, 4, live > 0));
    ECHO_TRY(check_matrix("dhidden", a.dhidden, live, a.cols, e));
    ECHO_TRY(check_vector("dweight", a.dweight, ge, a.grads));
    const int64_t need = a.rows ? linear_bytes(a) : 0;
    ECHO_TRY(check_workspace(a.workspace, workspace_bytes, need));
    ECHO_TRY(check_spans({matrix("dhidden", a.dhidden, live, cols, cols, e), vector("dweight", a.grads ? a.dweight : nullptr, vocab * cols, ge),
                          vector("lse", a.lse, a.rows, 4), vector("target", a.target, a.rows, 4),
                          vector("entropy", a.entropy, a.rows, 4), vector("loss", a.loss, a.rows, 4),
                          vector("workspace", a.workspace, need, 1)},
                         {matrix("hidden", a.hidden, a.rows, cols, a.hidden_stride, e),
                          matrix("weight", a.weight, vocab, cols, a.weight_stride, e),
                          vector(teacher ? "ids" : "targets", a.targets, a.rows * (teacher ? top : 1), ie),
                          vector("teacher", a.teacher, a.rows * top, teacher ? elem(a.teacher_type) : 4),
                          vector("lse", a.lse_in, a.rows, 4), vector("grad_loss", a.grad_loss, a.rows, 4)}));
    if (!a.rows && (!a.grads || a.accumulate)) return ECHO_OK;
    return on_device(hip_device, what, [&] { return launch_linear(a, static_cast<hipStream_t>(hip_stream)); });
}

}  // namespace

extern "C" {

int echo_distillation(const void *logits, int64_t logits_stride, int32_t type, const void *ids, int32_t index_type,
                      const void *teacher, int32_t teacher_type, int64_t rows, int64_t cols, int64_t top,
                      int64_t vocab_start, int64_t vocab_size, float temperature, float *lse, float *target,
                      float *entropy, float *loss, const float *grad_loss, void *grad, int64_t grad_stride,
                      int hip_device, void *hip_stream) {
    clear_error();
    const DistillArgs a{logits, ids, teacher, logits_stride, rows, vocab_start, vocab_size, 0, 0, index_type, teacher_type,
                        temperature, lse, target, entropy, loss, nullptr, grad_loss, grad, grad_stride};
    return distill(a, type, index_type, teacher_type, cols, top, false, hip_device, hip_stream, "distillation");
}

int echo_distillation_grad(const void *logits, int64_t logits_stride, int32_t type, const void *ids, int32_t index_type,
                           const void *teacher, int32_t teacher_type, int64_t rows, int64_t cols, int64_t top,
                           int64_t vocab_start, int64_t vocab_size, float temperature, const float *lse,
                           const float *grad_loss, void *grad, int64_t grad_stride, int hip_device, void *hip_stream) {
    clear_error();
    const DistillArgs a{logits, ids, teacher, logits_stride, rows, vocab_start, vocab_size, 0, 0, index_type, teacher_type,
                        temperature, nullptr, nullptr, nullptr, nullptr, lse, grad_loss, grad, grad_stride};
    return distill(a, type, index_type, teacher_type, cols, top, true, hip_device, hip_stream, "distillation gradient");
}

int64_t echo_linear_workspace(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                              int32_t type, int64_t rows, int64_t cols, int64_t vocab, int64_t top, int32_t loss,
                              int32_t grads) {
    if (!is_type(type) || rows < 1 || rows > kMaxHeadRows || cols < 1 || cols > kMaxHidden || vocab < 1 || vocab > kMaxHeadRows ||
        top < 0 || top > kMaxTop || rows * cols > kMaxElements || rows * vocab > kMaxElements || vocab * cols > kMaxElements)
        return 0;
    LinearArgs a{};
    a.hidden = hidden;
    a.weight = weight;
    a.hidden_stride = hidden_stride;
    a.weight_stride = weight_stride;
    a.rows = rows;
    a.type = type;
    a.cols = (int)cols;
    a.vocab = (int)vocab;
    a.top = (int)top;
    a.forward = loss != 0;
    a.grads = grads != 0;
    return linear_bytes(a);
}

int echo_linear_cross_entropy(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                              int32_t type, const void *targets, int32_t index_type, int64_t rows, int64_t cols,
                              int64_t vocab, int64_t vocab_start, int64_t vocab_size, float *lse, float *target,
                              float *loss, const float *grad_loss, void *dhidden, void *dweight, int32_t grad_type,
                              int32_t accumulate, void *workspace, int64_t workspace_bytes, int hip_device,
                              void *hip_stream) {
    clear_error();
    const LinearArgs a{hidden, weight, hidden_stride, weight_stride, rows, type, 0, 0, targets, nullptr, index_type, ECHO_F32, 0,
                       1.0f, vocab_start, vocab_size, true, false, lse, target, nullptr, loss, nullptr, grad_loss, dhidden,
                       dweight, grad_type, accumulate != 0, workspace};
    return linear(a, cols, vocab, 0, workspace_bytes, hip_device, hip_stream, "linear cross entropy");
}

int echo_linear_cross_entropy_grad(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                                   int32_t type, const void *targets, int32_t index_type, int64_t rows, int64_t cols,
                                   int64_t vocab, int64_t vocab_start, int64_t vocab_size, const float *lse,
                                   const float *grad_loss, void *dhidden, void *dweight, int32_t grad_type,
                                   int32_t accumulate, void *workspace, int64_t workspace_bytes, int hip_device,
                                   void *hip_stream) {
    clear_error();
    const LinearArgs a{hidden, weight, hidden_stride, weight_stride, rows, type, 0, 0, targets, nullptr, index_type, ECHO_F32, 0,
                       1.0f, vocab_start, vocab_size, false, true, nullptr, nullptr, nullptr, nullptr, lse, grad_loss, dhidden,
                       dweight, grad_type, accumulate != 0, workspace};
    return linear(a, cols, vocab, 0, workspace_bytes, hip_device, hip_stream, "linear cross entropy gradient");
}

int echo_linear_distillation(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                             int32_t type, const void *ids, int32_t index_type, const void *teacher,
                             int32_t teacher_type, int64_t rows, int64_t cols, int64_t vocab, int64_t top,
                             int64_t vocab_start, int64_t vocab_size, float temperature, float *lse, float *target,
                             float *entropy, float *loss, const float *grad_loss, void *dhidden, void *dweight,
                             int32_t grad_type, int32_t accumulate, void *workspace, int64_t workspace_bytes,
                             int hip_device, void *hip_stream) {
    clear_error();
    if (top < 1) return set_error(ECHO_ERR_ARG, "top = %lld outside [1, 1024]", (long long)top);
    const LinearArgs a{hidden, weight, hidden_stride, weight_stride, rows, type, 0, 0, ids, teacher, index_type, teacher_type, 0,
                       temperature, vocab_start, vocab_size, true, false, lse, target, entropy, loss, nullptr, grad_loss,
                       dhidden, dweight, grad_type, accumulate != 0, workspace};
    return linear(a, cols, vocab, top, workspace_bytes, hip_device, hip_stream, "linear distillation");
}

int echo_linear_distillation_grad(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                                  int32_t type, const void *ids, int32_t index_type, const void *teacher,
                                  int32_t teacher_type, int64_t rows, int64_t cols, int64_t vocab, int64_t top,
                                  int64_t vocab_start, int64_t vocab_size, float temperature, const float *lse,
                                  const float *grad_loss, void *dhidden, void *dweight, int32_t grad_type,
                                  int32_t accumulate, void *workspace, int64_t workspace_bytes, int hip_device,
                                  void *hip_stream) {
    clear_error();
    if (top < 1) return set_error(ECHO_ERR_ARG, "top = %lld outside [1, 1024]", (long long)top);
    const LinearArgs a{hidden, weight, hidden_stride, weight_stride, rows, type, 0, 0, ids, teacher, index_type, teacher_type, 0,
                       temperature, vocab_start, vocab_size, false, true, nullptr, nullptr, nullptr, nullptr, lse, grad_loss,
                       dhidden, dweight, grad_type, accumulate != 0, workspace};
    return linear(a, cols, vocab, top, workspace_bytes, hip_device, hip_stream, "linear distillation gradient");
}

}  // extern "C"

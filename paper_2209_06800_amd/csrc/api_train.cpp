// Argument checking of the entry points for training: lookup, grouped Update, distillation loss.
#include "mgg_internal.h"

namespace mgg {

static inline bool dtype_ok(mgg_dtype_t t) { return t == MGG_F32 || t == MGG_BF16; }
static inline bool index_ok(mgg_index_t t) { return t == MGG_I32 || t == MGG_I64; }
static inline size_t size_of(mgg_dtype_t t) { return t == MGG_BF16 ? 2 : 4; }
static inline size_t size_of(mgg_index_t t) { return t == MGG_I64 ? 8 : 4; }
static inline bool misaligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

static mgg_status_t check_workspace(const void *workspace, size_t have, size_t need)
{
    if (!workspace || misaligned(workspace, 256)) return fail(MGG_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (have < need) return fail(MGG_ERR_INVALID_ARG, "workspace too small: %zu < %zu", have, need);
    return MGG_OK;
}

static mgg_status_t check_lookup(int64_t n, mgg_index_t id_type, const void *ids, int64_t table_rows, mgg_dtype_t table_dtype, const void *table,
                                 int32_t dim, int64_t ld_table, mgg_dtype_t row_dtype, const void *rows, int64_t ld_rows)
{
    if (n < 0 || table_rows < 0 || dim < 1 || ld_table < dim || ld_rows < dim)
        return fail(MGG_ERR_INVALID_ARG, "n %lld, table_rows %lld, dim %d, leading dimensions %lld (table) and %lld", (long long)n, (long long)table_rows, dim,
                    (long long)ld_table, (long long)ld_rows);
    if (!index_ok(id_type) || !dtype_ok(table_dtype) || !dtype_ok(row_dtype)) return fail(MGG_ERR_INVALID_ARG, "unknown dtype");
    if (table_rows > INT32_MAX - 1) return fail(MGG_ERR_UNSUPPORTED, "%lld table rows", (long long)table_rows);
    if ((n > 0 && (!ids || !rows)) || (table_rows > 0 && !table)) return fail(MGG_ERR_INVALID_ARG, "NULL pointer");
    if (misaligned(ids, size_of(id_type)) || misaligned(table, size_of(table_dtype)) || misaligned(rows, size_of(row_dtype)))
        return fail(MGG_ERR_INVALID_ARG, "pointer not aligned to its element size");
    return MGG_OK;
}

static bool grouped_sizes_ok(int64_t n_rows, int32_t n_groups, int32_t d_in, int32_t d_out)
{
    return n_rows >= 0 && n_groups >= 0 && d_in >= 1 && d_out >= 1;
}

static mgg_status_t check_grouped(int64_t n_rows, int32_t n_groups, const int64_t *group_ptr, int32_t d_in, int32_t d_out, mgg_act_t act)
{
    if (!grouped_sizes_ok(n_rows, n_groups, d_in, d_out)) return fail(MGG_ERR_INVALID_ARG, "n_rows %lld, n_groups %d, d_in %d, d_out %d", (long long)n_rows, n_groups, d_in, d_out);
    if (act == MGG_ACT_SOFTMAX) return fail(MGG_ERR_UNSUPPORTED, "the grouped Update has no softmax");
    if (act != MGG_ACT_NONE && act != MGG_ACT_RELU) return fail(MGG_ERR_INVALID_ARG, "unknown activation");
    if (n_rows > INT32_MAX || n_groups > 65535 || d_in > (1 << 22) || d_out > (1 << 22))
        return fail(MGG_ERR_UNSUPPORTED, "n_rows %lld, n_groups %d, d_in %d, d_out %d", (long long)n_rows, n_groups, d_in, d_out);
    if (!group_ptr || misaligned(group_ptr, 8)) return fail(MGG_ERR_INVALID_ARG, "group_ptr is NULL or not aligned");
    return MGG_OK;
}

// a matrix of the grouped calls: rows [n x d], NULL allowed where nothing of it is used
static mgg_status_t check_matrix(const char *name, bool used, const void *p, mgg_dtype_t dtype, int64_t ld, int32_t d)
{
    if (!used) return MGG_OK;
    if (!p) return fail(MGG_ERR_INVALID_ARG, "%s is NULL", name);
    if (ld < d) return fail(MGG_ERR_INVALID_ARG, "leading dimension %lld of %s is less than its %d columns", (long long)ld, name, d);
    if (ld > (1 << 22)) return fail(MGG_ERR_UNSUPPORTED, "leading dimension %lld of %s", (long long)ld, name);
    if (misaligned(p, size_of(dtype))) return fail(MGG_ERR_INVALID_ARG, "%s is not aligned to its element size", name);
    return MGG_OK;
}

static mgg_status_t check_distill(const Distill &q, int64_t ld_grad)
{
    if (q.n_rows < 0 || q.n_classes < 1 || q.k < 1 || q.ld_logits < q.n_classes || q.ld_ids < q.k || q.ld_top < q.k || (q.grad && ld_grad < q.n_classes))
        return fail(MGG_ERR_INVALID_ARG, "n_rows %lld, n_classes %d, k %d, leading dimensions %lld (logits), %lld (ids), %lld (teacher), %lld (gradient)",
                    (long long)q.n_rows, q.n_classes, q.k, (long long)q.ld_logits, (long long)q.ld_ids, (long long)q.ld_top, (long long)ld_grad);
    if (!dtype_ok(q.logits_dtype) || !dtype_ok(q.top_dtype) || !index_ok(q.id_type) || (q.grad && !dtype_ok(q.grad_dtype))) return fail(MGG_ERR_INVALID_ARG, "unknown dtype");
    if (!(q.temperature >= 1e-6f && q.temperature <= 1e6f)) return fail(MGG_ERR_INVALID_ARG, "temperature %g", static_cast<double>(q.temperature));
    if (q.k > 1024 || q.n_rows > INT32_MAX - 1 || q.n_classes > INT32_MAX - 1) return fail(MGG_ERR_UNSUPPORTED, "n_rows %lld, n_classes %d, k %d", (long long)q.n_rows, q.n_classes, q.k);
    if (q.n_rows > 0 && (!q.logits || !q.top_ids || !q.top_logits || !q.loss)) return fail(MGG_ERR_INVALID_ARG, "NULL pointer");
    if (misaligned(q.logits, size_of(q.logits_dtype)) || misaligned(q.top_logits, size_of(q.top_dtype)) || misaligned(q.top_ids, size_of(q.id_type)) ||
        misaligned(q.row_weight, 4) || misaligned(q.loss, 4) || (q.grad && misaligned(q.grad, size_of(q.grad_dtype))))
        return fail(MGG_ERR_INVALID_ARG, "pointer not aligned to its element size");
    if (q.grad == q.logits && q.grad && (q.grad_dtype != q.logits_dtype || ld_grad != q.ld_logits))
        return fail(MGG_ERR_INVALID_ARG, "a gradient in place of the logits needs their dtype and leading dimension");
    return MGG_OK;
}

}  // namespace mgg

using namespace mgg;

extern "C" {

mgg_status_t mgg_embed(int64_t n, mgg_index_t id_type, const void *ids, int64_t table_rows, mgg_dtype_t table_dtype, const void *table, int32_t dim,
                       int64_t ld_table, float scale, mgg_dtype_t out_dtype, void *out, int64_t ld_out, void *stream)
{
    mgg_status_t s = check_lookup(n, id_type, ids, table_rows, table_dtype, table, dim, ld_table, out_dtype, out, ld_out);
    if (s != MGG_OK || n == 0) return s;
    return launch_embed(n, id_type, ids, table_rows, table_dtype, table, dim, ld_table, scale, out_dtype, out, ld_out, static_cast<hipStream_t>(stream));
}

size_t mgg_embed_grad_workspace_bytes(int64_t n, int64_t table_rows, int32_t dim)
{
    if (n < 0 || table_rows < 0 || dim < 1 || table_rows > INT32_MAX - 1 || n > (1 << 30)) return 0;
    return embed_grad_workspace(n, table_rows, dim);
}

mgg_status_t mgg_embed_grad(int64_t n, mgg_index_t id_type, const void *ids, int64_t table_rows, mgg_dtype_t grad_dtype, const void *grad_out, int32_t dim,
                            int64_t ld_grad, float scale, int32_t accumulate, mgg_dtype_t out_dtype, void *grad_table, int64_t ld_table, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    mgg_status_t s = check_lookup(n, id_type, ids, table_rows, out_dtype, grad_table, dim, ld_table, grad_dtype, grad_out, ld_grad);
    if (s == MGG_OK && accumulate != 0 && accumulate != 1) s = fail(MGG_ERR_INVALID_ARG, "accumulate must be 0 or 1");
    if (s == MGG_OK && n > (1 << 30)) s = fail(MGG_ERR_UNSUPPORTED, "%lld ids", (long long)n);
    if (s == MGG_OK) s = check_workspace(workspace, workspace_bytes, embed_grad_workspace(n, table_rows, dim));
    if (s != MGG_OK || table_rows == 0) return s;
    return launch_embed_grad(n, id_type, ids, table_rows, grad_dtype, grad_out, dim, ld_grad, scale, accumulate != 0, out_dtype, grad_table, ld_table, workspace,
                             static_cast<hipStream_t>(stream));
}

mgg_status_t mgg_update_grouped(int64_t n_rows, int32_t n_groups, const int64_t *group_ptr, mgg_dtype_t a_dtype, const void *a, int64_t ld_a, int32_t d_in,
                                mgg_dtype_t w_dtype, const void *w, const float *bias, int32_t d_out, mgg_act_t act, mgg_dtype_t out_dtype, void *out,
                                int64_t ld_out, void *stream)
{
    mgg_status_t s = check_grouped(n_rows, n_groups, group_ptr, d_in, d_out, act);
    if (s != MGG_OK) return s;
    if (!dtype_ok(a_dtype) || !dtype_ok(w_dtype) || !dtype_ok(out_dtype)) return fail(MGG_ERR_INVALID_ARG, "unknown dtype");
    if (a_dtype != w_dtype) return fail(MGG_ERR_UNSUPPORTED, "the grouped Update takes rows and weights of one dtype");
    const bool work = n_rows > 0 && n_groups > 0;
    s = check_matrix("a", work, a, a_dtype, ld_a, d_in);
    if (s == MGG_OK) s = check_matrix("w", work, w, w_dtype, d_out, d_out);
    if (s == MGG_OK) s = check_matrix("out", work, out, out_dtype, ld_out, d_out);
    if (s == MGG_OK && misaligned(bias, 4)) s = fail(MGG_ERR_INVALID_ARG, "bias is not aligned to its element size");
    if (s != MGG_OK || !work) return s;
    return launch_update_grouped(n_rows, n_groups, group_ptr, a_dtype, a, ld_a, d_in, w, bias, d_out, act == MGG_ACT_RELU, out_dtype, out, ld_out,
                                 static_cast<hipStream_t>(stream));
}

size_t mgg_update_grouped_grad_workspace_bytes(int64_t n_rows, int32_t n_groups, int32_t d_in, int32_t d_out, mgg_dtype_t dtype, mgg_act_t act)
{
    if (!grouped_sizes_ok(n_rows, n_groups, d_in, d_out) || !dtype_ok(dtype) || (act != MGG_ACT_NONE && act != MGG_ACT_RELU) || n_rows > INT32_MAX ||
        n_groups > 65535 || d_in > (1 << 22) || d_out > (1 << 22))
        return 0;
    return grouped_grad_workspace(n_rows, n_groups, d_in, d_out, dtype, act == MGG_ACT_RELU);
}

mgg_status_t mgg_update_grouped_grad(int64_t n_rows, int32_t n_groups, const int64_t *group_ptr, mgg_dtype_t dtype, const void *grad_out, int64_t ld_grad,
                                     mgg_act_t act, mgg_dtype_t out_dtype, const void *out, int64_t ld_out, const void *a, int64_t ld_a, int32_t d_in,
                                     const void *w, int32_t d_out, mgg_dtype_t grad_a_dtype, void *grad_a, int64_t ld_grad_a, mgg_dtype_t grad_w_dtype,
                                     void *grad_w, float *grad_bias, int32_t accumulate, void *workspace, size_t workspace_bytes, void *stream)
{
    mgg_status_t s = check_grouped(n_rows, n_groups, group_ptr, d_in, d_out, act);
    if (s != MGG_OK) return s;
    if (!dtype_ok(dtype) || !dtype_ok(out_dtype) || !dtype_ok(grad_a_dtype) || !dtype_ok(grad_w_dtype)) return fail(MGG_ERR_INVALID_ARG, "unknown dtype");
    if (accumulate & ~(MGG_ACC_W | MGG_ACC_BIAS)) return fail(MGG_ERR_INVALID_ARG, "unknown bits in accumulate");
    const bool relu = act == MGG_ACT_RELU, rows = n_rows > 0 && n_groups > 0;
    s = check_matrix("grad_out", rows && (grad_a || grad_w || grad_bias), grad_out, dtype, ld_grad, d_out);
    if (s == MGG_OK) s = check_matrix("out", rows && relu && (grad_a || grad_w || grad_bias), out, out_dtype, ld_out, d_out);
    if (s == MGG_OK) s = check_matrix("a", rows && grad_w, a, dtype, ld_a, d_in);
    if (s == MGG_OK) s = check_matrix("w", rows && grad_a, w, dtype, d_out, d_out);
    if (s == MGG_OK) s = check_matrix("grad_a", rows && grad_a, grad_a, grad_a_dtype, ld_grad_a, d_in);
    if (s == MGG_OK) s = check_matrix("grad_w", grad_w, grad_w, grad_w_dtype, d_out, d_out);
    if (s == MGG_OK && misaligned(grad_bias, 4)) s = fail(MGG_ERR_INVALID_ARG, "grad_bias is not aligned to its element size");
    if (s == MGG_OK) s = check_workspace(workspace, workspace_bytes, grouped_grad_workspace(n_rows, n_groups, d_in, d_out, dtype, relu));
    if (s != MGG_OK || n_groups == 0) return s;
    GroupedGrad q{};
    q.n_rows = n_rows; q.n_groups = n_groups; q.d_in = d_in; q.d_out = d_out; q.group_ptr = group_ptr;
    q.dtype = dtype; q.out_dtype = out_dtype; q.grad_a_dtype = grad_a_dtype; q.grad_w_dtype = grad_w_dtype;
    q.grad_out = grad_out; q.out = out; q.a = a; q.w = w;
    q.ld_grad = ld_grad; q.ld_out = ld_out; q.ld_a = ld_a; q.ld_grad_a = ld_grad_a;
    q.relu = relu; q.add_w = accumulate & MGG_ACC_W; q.add_bias = accumulate & MGG_ACC_BIAS;
    q.grad_a = rows ? grad_a : nullptr; q.grad_w = grad_w; q.grad_bias = grad_bias;
    return launch_update_grouped_grad(q, workspace, static_cast<hipStream_t>(stream));
}

size_t mgg_distill_workspace_bytes(int64_t n_rows, int32_t n_classes)
{
    if (n_rows < 0 || n_classes < 1 || n_rows > INT32_MAX - 1 || n_classes > INT32_MAX - 1) return 0;
    return distill_workspace(n_rows, n_classes);
}

mgg_status_t mgg_distill_loss(int64_t n_rows, int32_t n_classes, mgg_dtype_t logits_dtype, const void *logits, int64_t ld_logits, int32_t k,
                              mgg_index_t id_type, const void *top_ids, int64_t ld_ids, mgg_dtype_t top_dtype, const void *top_logits, int64_t ld_top,
                              float temperature, const float *row_weight, float *loss, mgg_dtype_t grad_dtype, void *grad_logits, int64_t ld_grad,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    Distill q{};
    q.n_rows = n_rows; q.n_classes = n_classes; q.k = k;
    q.ld_logits = ld_logits; q.ld_ids = ld_ids; q.ld_top = ld_top; q.ld_grad = ld_grad;
    q.logits_dtype = logits_dtype; q.top_dtype = top_dtype; q.grad_dtype = grad_dtype; q.id_type = id_type;
    q.logits = logits; q.top_ids = top_ids; q.top_logits = top_logits; q.row_weight = row_weight;
    q.temperature = temperature; q.loss = loss; q.grad = grad_logits;
    mgg_status_t s = check_distill(q, ld_grad);
    if (s == MGG_OK) s = check_workspace(workspace, workspace_bytes, distill_workspace(n_rows, n_classes));
    if (s != MGG_OK || n_rows == 0) return s;
    return launch_distill(q, workspace, static_cast<hipStream_t>(stream));
}

}  // extern "C"

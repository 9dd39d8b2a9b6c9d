// xred_layer.hip -- the C ABI of the calls around a reduced activation:
// argument checks and dispatch to the launchers (xred_norm.hip, xred_route.hip,
// xred_experts.hip).  As elsewhere, everything is checked before anything is enqueued.
#include "xred_layer.hpp"

namespace xred {
namespace {

bool row_type(xred_dtype d)
{
    return d == XRED_FLOAT32 || d == XRED_BFLOAT16 || d == XRED_FLOAT16;
}

// A matrix of the call: where its rows lie, in bytes.
struct Matrix {
    const void *data;
    uint64_t stride, width, rows;   // bytes between rows, bytes of a row
    uint64_t span() const { return (rows - 1) * stride + width; }
};

// m (present, at least one row of at least one element) as a Matrix.
xred_status check_rows(const xred_rows &m, uint64_t rows, uint64_t columns, uint64_t es,
                       const char *name, Matrix *out)
{
    if (m.stride < columns)
        return fail(XRED_INVALID_ARGUMENT, "%s: row distance %llu is below the row's %llu elements",
                    name, (unsigned long long)m.stride, (unsigned long long)columns);
    uint64_t bytes;
    if (__builtin_mul_overflow(m.stride, es, &bytes) || mul_overflows(bytes, rows))
        return fail(XRED_INVALID_ARGUMENT, "%s: size overflows", name);
    *out = Matrix{m.data, bytes, columns * es, rows};
    return check_buf(m.data, out->span(), es, name, 0);
}

// Whether rows of a and b share a byte, other than being the same rows when
// `exact_ok`.  Matrices at one row distance may interleave (column ranges of
// one larger matrix); at different distances their whole spans count.
bool rows_overlap(const Matrix &a, const Matrix &b, bool exact_ok)
{
    if (a.data == b.data && a.stride == b.stride && a.width == b.width && exact_ok) return false;
    if (!bad_overlap(a.data, a.span(), b.data, b.span(), false)) return false;
    if (a.stride != b.stride) return true;
    const uintptr_t x = (uintptr_t)a.data, y = (uintptr_t)b.data;
    const uint64_t s = a.stride, d = y >= x ? (y - x) % s : (s - (x - y) % s) % s;
    return d < a.width || s - d < b.width;
}

xred_status check_weight(const void *w, xred_dtype wt, xred_dtype dtype, uint64_t hidden,
                         Matrix *out)
{
    if (wt != dtype && wt != XRED_FLOAT32)
        return fail(XRED_UNSUPPORTED, "weight_dtype %d with dtype %d", (int)wt, (int)dtype);
    return check_rows(xred_rows{(void *)w, hidden}, 1, hidden, elem_size(wt), "weight", out);
}

// No output shares bytes with another matrix of the call.  may[i]: the output
// out[i] may be exactly one of the first n[i] inputs.
xred_status check_apart(const Matrix *out, const char *const *names, int nout, const Matrix *in,
                        int nin, const int *may)
{
    for (int i = 0; i < nout; ++i) {
        for (int j = 0; j < nin; ++j)
            if (rows_overlap(out[i], in[j], j < may[i]))
                return fail(XRED_ALIAS, "%s overlaps an input", names[i]);
        for (int j = 0; j < i; ++j)
            if (rows_overlap(out[i], out[j], false))
                return fail(XRED_ALIAS, "%s overlaps %s", names[i], names[j]);
    }
    return XRED_SUCCESS;
}

// What xred_route and its gradient share.
xred_status check_route(xred_dtype dtype, xred_score score, uint32_t flags, uint32_t experts,
                        uint32_t topk, uint64_t tokens)
{
    if (!row_type(dtype)) return fail(XRED_UNSUPPORTED, "dtype %d", (int)dtype);
    if (score != XRED_SCORE_SOFTMAX && score != XRED_SCORE_SIGMOID)
        return fail(XRED_INVALID_ARGUMENT, "unknown score %d", (int)score);
    if (flags & ~(unsigned)XRED_ROUTE_RENORM)
        return fail(XRED_INVALID_ARGUMENT, "unknown flag bits 0x%x", flags);
    if (experts < 1 || experts > XRED_MAX_EXPERTS)
        return fail(XRED_UNSUPPORTED, "experts = %u outside 1..%d", experts, XRED_MAX_EXPERTS);
    if (topk < 1 || topk > experts || topk > XRED_MAX_TOPK)
        return fail(topk >= 1 && topk <= experts ? XRED_UNSUPPORTED : XRED_INVALID_ARGUMENT,
                    "topk = %u outside 1..min(experts = %u, %d)", topk, experts, XRED_MAX_TOPK);
    if (tokens > (uint64_t)INT64_MAX / (4 * XRED_MAX_TOPK))
        return fail(XRED_INVALID_ARGUMENT, "tokens * topk overflows");
    return XRED_SUCCESS;
}

// What the calls on dispatched rows share: topk, the row length, and the slots
// (pos, and the binary32 values beside it) of at least one token.
xred_status check_slots(uint64_t tokens, uint32_t topk, uint64_t hidden, uint64_t es)
{
    if (topk < 1 || topk > XRED_MAX_TOPK)
        return fail(XRED_UNSUPPORTED, "topk = %u outside 1..%d", topk, XRED_MAX_TOPK);
    if (hidden < 1 || hidden > (1u << 30) / es)
        return fail(XRED_UNSUPPORTED, "hidden = %llu: rows of 1 element to 1 GiB are supported",
                    (unsigned long long)hidden);
    if (tokens > (uint64_t)INT64_MAX / (4 * XRED_MAX_TOPK))
        return fail(XRED_INVALID_ARGUMENT, "tokens * topk overflows");
    return XRED_SUCCESS;
}

xred_status check_words(const void *p, uint64_t tokens, uint64_t topk, const char *name, Matrix *out)
{
    return check_rows(xred_rows{(void *)p, topk}, tokens, topk, 4, name, out);
}

}  // namespace
}  // namespace xred

using namespace xred;

#define TRY(call)                                    \
    do {                                             \
        const xred_status st_ = (call);              \
        if (st_ != XRED_SUCCESS) return st_;         \
    } while (0)

extern "C" {

XRED_API xred_status xred_fold_norm(const xred_fold_norm_args *args, void *hip_stream)
{
    if (args == nullptr) return fail(XRED_INVALID_ARGUMENT, "args is NULL");
    const xred_fold_norm_args &a = *args;
    if (trace_enabled())
        trace_printf("xred_fold_norm nsrc=%u rows=%llu hidden=%llu dtype=%d group=%u stream=%p",
                     a.nsrc, (unsigned long long)a.rows, (unsigned long long)a.hidden,
                     (int)a.dtype, a.group, hip_stream);
    if (a.nsrc < 1 || a.nsrc > XRED_MAX_SRC)
        return fail(XRED_INVALID_ARGUMENT, "nsrc = %u outside 1..%d", a.nsrc, XRED_MAX_SRC);
    if (!row_type(a.dtype)) return fail(XRED_UNSUPPORTED, "dtype %d", (int)a.dtype);
    if (a.hidden < 1 || a.hidden > XRED_MAX_HIDDEN)
        return fail(XRED_UNSUPPORTED, "hidden = %llu outside 1..%d", (unsigned long long)a.hidden,
                    XRED_MAX_HIDDEN);
    if (!(a.eps >= 0.0f)) return fail(XRED_INVALID_ARGUMENT, "eps is negative or a NaN");
    if (a.group != 0 && (a.group < 32 || a.group > 512 || (a.group & (a.group - 1))))
        return fail(XRED_INVALID_ARGUMENT, "group = %u is not 0, 32, 64, 128, 256 or 512", a.group);
    if (a.rows == 0) return XRED_SUCCESS;   // buffers of no rows may be NULL
    if (!a.out.data && !a.out8.data)
        return fail(XRED_INVALID_ARGUMENT, "neither out nor out8 is given");
    if ((a.out8.data == nullptr) != (a.scale.data == nullptr))
        return fail(XRED_INVALID_ARGUMENT, "out8 and scale go together");
    if (a.srcs == nullptr) return fail(XRED_INVALID_ARGUMENT, "srcs is NULL");
    const uint64_t es = elem_size(a.dtype);
    Matrix in[XRED_MAX_SRC + 2], out[5];
    const char *names[5];
    int nin = 0, nout = 0, may[5];
    for (uint32_t p = 0; p < a.nsrc; ++p)
        TRY(check_rows(xred_rows{(void *)a.srcs[p], a.src_stride}, a.rows, a.hidden, es, "srcs",
                       &in[nin++]));
    if (a.residual.data)
        TRY(check_rows(a.residual, a.rows, a.hidden, es, "residual", &in[nin++]));
    const int same = nin;
    if (a.weight) TRY(check_weight(a.weight, a.weight_dtype, a.dtype, a.hidden, &in[nin++]));
    auto output = [&](const xred_rows &m, uint64_t columns, uint64_t size, const char *name,
                      int in_place) {
        names[nout] = name;
        may[nout] = in_place;
        return m.data ? check_rows(m, a.rows, columns, size, name, &out[nout++]) : XRED_SUCCESS;
    };
    TRY(output(a.sum, a.hidden, es, "sum", same));
    TRY(output(a.out, a.hidden, es, "out", same));
    TRY(output(a.out8, a.hidden, 1, "out8", 0));
    TRY(output(a.scale, a.group ? (a.hidden + a.group - 1) / a.group : 1, 4, "scale", 0));
    TRY(output(xred_rows{a.rstd, 1}, 1, 4, "rstd", 0));
    TRY(check_apart(out, names, nout, in, nin, may));
    const hipError_t e = launch_fold_norm(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? XRED_SUCCESS : hip_fail(e, "fold_norm launch");
}

XRED_API size_t xred_fold_norm_grad_workspace(uint64_t rows, uint64_t hidden)
{
    if (hidden > XRED_MAX_HIDDEN) return 0;
    const uint32_t a = norm_grad_slices(rows, hidden, 2), b = norm_grad_slices(rows, hidden, 4);
    return (size_t)(a > b ? a : b) * hidden * 4;
}

XRED_API xred_status xred_fold_norm_grad(const xred_fold_norm_grad_args *args, void *hip_stream)
{
    if (args == nullptr) return fail(XRED_INVALID_ARGUMENT, "args is NULL");
    const xred_fold_norm_grad_args &a = *args;
    if (trace_enabled())
        trace_printf("xred_fold_norm_grad rows=%llu hidden=%llu dtype=%d stream=%p",
                     (unsigned long long)a.rows, (unsigned long long)a.hidden, (int)a.dtype,
                     hip_stream);
    if (!row_type(a.dtype)) return fail(XRED_UNSUPPORTED, "dtype %d", (int)a.dtype);
    if (a.hidden < 1 || a.hidden > XRED_MAX_HIDDEN)
        return fail(XRED_UNSUPPORTED, "hidden = %llu outside 1..%d", (unsigned long long)a.hidden,
                    XRED_MAX_HIDDEN);
    if (a.rows == 0 && !a.dweight) return XRED_SUCCESS;
    const uint64_t es = elem_size(a.dtype);
    Matrix in[5], out[3];
    const char *names[3];
    int nin = 0, nout = 0, may[3] = {0, 0, 0};
    if (a.rows) {
        TRY(check_rows(a.dout, a.rows, a.hidden, es, "dout", &in[nin++]));
        if (a.dsum.data) TRY(check_rows(a.dsum, a.rows, a.hidden, es, "dsum", &in[nin++]));
        may[0] = nin;
        TRY(check_rows(a.sum, a.rows, a.hidden, es, "sum", &in[nin++]));
        TRY(check_rows(xred_rows{(void *)a.rstd, 1}, a.rows, 1, 4, "rstd", &in[nin++]));
        if (a.weight) TRY(check_weight(a.weight, a.weight_dtype, a.dtype, a.hidden, &in[nin++]));
        names[nout] = "dx";
        TRY(check_rows(a.dx, a.rows, a.hidden, es, "dx", &out[nout++]));
    }
    if (a.dweight) {
        names[nout] = "dweight";
        TRY(check_rows(xred_rows{a.dweight, a.hidden}, 1, a.hidden, 4, "dweight", &out[nout++]));
        const uint64_t need = xred_fold_norm_grad_workspace(a.rows, a.hidden);
        if (a.workspace_bytes < need)
            return fail(XRED_INVALID_ARGUMENT, "workspace of %llu bytes, %llu are needed",
                        (unsigned long long)a.workspace_bytes, (unsigned long long)need);
        if (need) {
            TRY(check_buf(a.workspace, need, 16, "workspace", 0));
            names[nout] = "workspace";
            out[nout++] = Matrix{a.workspace, need, need, 1};
        }
    }
    TRY(check_apart(out, names, nout, in, nin, may));
    const hipError_t e = launch_fold_norm_grad(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? XRED_SUCCESS : hip_fail(e, "fold_norm_grad launch");
}

XRED_API xred_status xred_route(const xred_route_args *args, void *hip_stream)
{
    if (args == nullptr) return fail(XRED_INVALID_ARGUMENT, "args is NULL");
    const xred_route_args &a = *args;
    if (trace_enabled())
        trace_printf("xred_route tokens=%llu experts=%u topk=%u groups=%u score=%d dtype=%d "
                     "stream=%p", (unsigned long long)a.tokens, a.experts, a.topk, a.groups,
                     (int)a.score, (int)a.dtype, hip_stream);
    TRY(check_route(a.dtype, a.score, a.flags, a.experts, a.topk, a.tokens));
    if (a.groups < 1 || a.groups > XRED_MAX_EXPERT_GROUPS || a.experts % a.groups != 0)
        return fail(XRED_INVALID_ARGUMENT, "groups = %u: not a divisor of %u experts up to %d",
                    a.groups, a.experts, XRED_MAX_EXPERT_GROUPS);
    if (a.groups > 1 && (a.group_topk < 1 || a.group_topk > a.groups))
        return fail(XRED_INVALID_ARGUMENT, "group_topk = %u outside 1..%u", a.group_topk, a.groups);
    if (a.groups > 1 && a.group_score != 1 && a.group_score != 2)
        return fail(XRED_INVALID_ARGUMENT, "group_score = %u is neither 1 nor 2", a.group_score);
    if (a.tokens == 0) return XRED_SUCCESS;
    Matrix in[2], out[2];
    const char *const names[2] = {"ids", "weights"};
    const int may[2] = {0, 0};
    int nin = 0;
    TRY(check_rows(a.logits, a.tokens, a.experts, elem_size(a.dtype), "logits", &in[nin++]));
    if (a.bias)
        TRY(check_rows(xred_rows{(void *)a.bias, a.experts}, 1, a.experts, 4, "bias", &in[nin++]));
    TRY(check_rows(xred_rows{a.ids, a.topk}, a.tokens, a.topk, 4, "ids", &out[0]));
    TRY(check_rows(xred_rows{a.weights, a.topk}, a.tokens, a.topk, 4, "weights", &out[1]));
    TRY(check_apart(out, names, 2, in, nin, may));
    const hipError_t e = launch_route(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? XRED_SUCCESS : hip_fail(e, "route launch");
}

XRED_API xred_status xred_route_grad(const xred_route_grad_args *args, void *hip_stream)
{
    if (args == nullptr) return fail(XRED_INVALID_ARGUMENT, "args is NULL");
    const xred_route_grad_args &a = *args;
    if (trace_enabled())
        trace_printf("xred_route_grad tokens=%llu experts=%u topk=%u score=%d dtype=%d stream=%p",
                     (unsigned long long)a.tokens, a.experts, a.topk, (int)a.score, (int)a.dtype,
                     hip_stream);
    TRY(check_route(a.dtype, a.score, a.flags, a.experts, a.topk, a.tokens));
    if (a.tokens == 0) return XRED_SUCCESS;
    const uint64_t es = elem_size(a.dtype);
    Matrix in[3], out[1];
    const char *const names[1] = {"dlogits"};
    const int may[1] = {0};
    TRY(check_rows(a.logits, a.tokens, a.experts, es, "logits", &in[0]));
    TRY(check_rows(xred_rows{(void *)a.ids, a.topk}, a.tokens, a.topk, 4, "ids", &in[1]));
    TRY(check_rows(xred_rows{(void *)a.dweights, a.topk}, a.tokens, a.topk, 4, "dweights", &in[2]));
    TRY(check_rows(a.dlogits, a.tokens, a.experts, es, "dlogits", &out[0]));
    TRY(check_apart(out, names, 1, in, 3, may));
    const hipError_t e = launch_route_grad(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? XRED_SUCCESS : hip_fail(e, "route_grad launch");
}

XRED_API size_t xred_dispatch_plan_workspace(uint64_t slots, uint32_t experts)
{
    return experts > XRED_MAX_EXPERTS ? 0 : (size_t)dispatch_plan_bytes(slots, experts);
}

XRED_API xred_status xred_dispatch_plan(const xred_dispatch_plan_args *args, void *hip_stream)
{
    if (args == nullptr) return fail(XRED_INVALID_ARGUMENT, "args is NULL");
    const xred_dispatch_plan_args &a = *args;
    if (trace_enabled())
        trace_printf("xred_dispatch_plan tokens=%llu topk=%u experts=%u stream=%p",
                     (unsigned long long)a.tokens, a.topk, a.experts, hip_stream);
    if (a.experts < 1 || a.experts > XRED_MAX_EXPERTS)
        return fail(XRED_UNSUPPORTED, "experts = %u outside 1..%d", a.experts, XRED_MAX_EXPERTS);
    TRY(check_slots(a.tokens, a.topk, 1, 1));
    const uint64_t n = a.tokens * a.topk;
    if (n > INT32_MAX)
        return fail(XRED_UNSUPPORTED, "%llu slots, at most 2^31 - 1 are supported",
                    (unsigned long long)n);
    Matrix in[1], out[5];
    const char *names[5];
    int nin = 0, nout = 0;
    const int may[5] = {0, 0, 0, 0, 0};
    auto output = [&](void *p, uint64_t words, const char *name) {
        names[nout] = name;
        return check_words(p, 1, words, name, &out[nout++]);
    };
    TRY(output(a.counts, a.experts, "counts"));
    TRY(output(a.offsets, a.experts + 1, "offsets"));
    if (n) {
        TRY(check_words(a.ids, 1, n, "ids", &in[nin++]));
        TRY(output(a.pos, n, "pos"));
        if (a.slots) TRY(output(a.slots, n, "slots"));
    }
    const uint64_t need = dispatch_plan_bytes(n, a.experts);
    if (a.workspace_bytes < need)
        return fail(XRED_INVALID_ARGUMENT, "workspace of %llu bytes, %llu are needed",
                    (unsigned long long)a.workspace_bytes, (unsigned long long)need);
    if (need) {
        TRY(check_buf(a.workspace, need, 16, "workspace", 0));
        names[nout] = "workspace";
        out[nout++] = Matrix{a.workspace, need, need, 1};
    }
    TRY(check_apart(out, names, nout, in, nin, may));
    const hipError_t e = launch_dispatch_plan(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? XRED_SUCCESS : hip_fail(e, "dispatch_plan launch");
}

XRED_API xred_status xred_dispatch(const xred_dispatch_args *args, void *hip_stream)
{
    if (args == nullptr) return fail(XRED_INVALID_ARGUMENT, "args is NULL");
    const xred_dispatch_args &a = *args;
    if (trace_enabled())
        trace_printf("xred_dispatch tokens=%llu topk=%u hidden=%llu out_rows=%llu dtype=%d "
                     "stream=%p", (unsigned long long)a.tokens, a.topk,
                     (unsigned long long)a.hidden, (unsigned long long)a.out_rows, (int)a.dtype,
                     hip_stream);
    const uint64_t es = elem_size(a.dtype);
    if (es == 0) return fail(XRED_INVALID_ARGUMENT, "unknown dtype %d", (int)a.dtype);
    TRY(check_slots(a.tokens, a.topk, a.hidden, es));
    if ((a.scale.data == nullptr) != (a.out_scale.data == nullptr) && a.tokens && a.out_rows)
        return fail(XRED_INVALID_ARGUMENT, "scale and out_scale go together");
    if (a.scale.data) TRY(check_slots(a.tokens, a.topk, a.scale_columns, 4));
    if (a.tokens == 0 || a.out_rows == 0) return XRED_SUCCESS;
    Matrix in[3], out[2];
    const char *const names[2] = {"out", "out_scale"};
    const int may[2] = {0, 0};
    TRY(check_rows(a.x, a.tokens, a.hidden, es, "x", &in[0]));
    TRY(check_words(a.pos, a.tokens, a.topk, "pos", &in[1]));
    TRY(check_rows(a.out, a.out_rows, a.hidden, es, "out", &out[0]));
    if (a.scale.data) {
        TRY(check_rows(a.scale, a.tokens, a.scale_columns, 4, "scale", &in[2]));
        TRY(check_rows(a.out_scale, a.out_rows, a.scale_columns, 4, "out_scale", &out[1]));
    }
    const int more = a.scale.data ? 1 : 0;
    TRY(check_apart(out, names, 1 + more, in, 2 + more, may));
    const hipError_t e = launch_dispatch(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? XRED_SUCCESS : hip_fail(e, "dispatch launch");
}

XRED_API xred_status xred_combine(const xred_combine_args *args, void *hip_stream)
{
    if (args == nullptr) return fail(XRED_INVALID_ARGUMENT, "args is NULL");
    const xred_combine_args &a = *args;
    if (trace_enabled())
        trace_printf("xred_combine tokens=%llu topk=%u hidden=%llu y_rows=%llu dtype=%d stream=%p",
                     (unsigned long long)a.tokens, a.topk, (unsigned long long)a.hidden,
                     (unsigned long long)a.y_rows, (int)a.dtype, hip_stream);
    if (!row_type(a.dtype)) return fail(XRED_UNSUPPORTED, "dtype %d", (int)a.dtype);
    const uint64_t es = elem_size(a.dtype);
    TRY(check_slots(a.tokens, a.topk, a.hidden, es));
    if (a.tokens == 0) return XRED_SUCCESS;
    Matrix in[4], out[1];
    const char *const names[1] = {"out"};
    int nin = 0, may[1] = {0};
    if (a.base.data) {
        TRY(check_rows(a.base, a.tokens, a.hidden, es, "base", &in[nin++]));
        may[0] = nin;
    }
    if (a.y_rows) TRY(check_rows(a.y, a.y_rows, a.hidden, es, "y", &in[nin++]));
    TRY(check_words(a.pos, a.tokens, a.topk, "pos", &in[nin++]));
    if (a.weights) TRY(check_words(a.weights, a.tokens, a.topk, "weights", &in[nin++]));
    TRY(check_rows(a.out, a.tokens, a.hidden, es, "out", &out[0]));
    TRY(check_apart(out, names, 1, in, nin, may));
    const hipError_t e = launch_combine(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? XRED_SUCCESS : hip_fail(e, "combine launch");
}

XRED_API xred_status xred_combine_grad(const xred_combine_grad_args *args, void *hip_stream)
{
    if (args == nullptr) return fail(XRED_INVALID_ARGUMENT, "args is NULL");
    const xred_combine_grad_args &a = *args;
    if (trace_enabled())
        trace_printf("xred_combine_grad tokens=%llu topk=%u hidden=%llu y_rows=%llu dtype=%d "
                     "stream=%p", (unsigned long long)a.tokens, a.topk,
                     (unsigned long long)a.hidden, (unsigned long long)a.y_rows, (int)a.dtype,
                     hip_stream);
    if (!row_type(a.dtype)) return fail(XRED_UNSUPPORTED, "dtype %d", (int)a.dtype);
    const uint64_t es = elem_size(a.dtype);
    TRY(check_slots(a.tokens, a.topk, a.hidden, es));
    if (a.tokens == 0) return XRED_SUCCESS;
    Matrix in[4], out[2];
    const char *names[2];
    int nin = 0, nout = 0, may[2] = {0, 0};
    if (a.y_rows) {
        if (a.dweights) {
            TRY(check_rows(a.y, a.y_rows, a.hidden, es, "y", &in[nin++]));
            may[0] = nin;
        }
        names[nout] = "dy";
        TRY(check_rows(a.dy, a.y_rows, a.hidden, es, "dy", &out[nout++]));
    }
    TRY(check_rows(a.dout, a.tokens, a.hidden, es, "dout", &in[nin++]));
    TRY(check_words(a.pos, a.tokens, a.topk, "pos", &in[nin++]));
    TRY(check_words(a.weights, a.tokens, a.topk, "weights", &in[nin++]));
    if (a.dweights) {
        names[nout] = "dweights";
        TRY(check_words(a.dweights, a.tokens, a.topk, "dweights", &out[nout++]));
    }
    if (nout == 0) return XRED_SUCCESS;
    TRY(check_apart(out, names, nout, in, nin, may));
    const hipError_t e = launch_combine_grad(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? XRED_SUCCESS : hip_fail(e, "combine_grad launch");
}

}  // extern "C"

// C ABI of the routed layer and its training step: checks of arguments, then the launches.
#include "dense_checks.h"

#include <cstdlib>

using namespace seer;

namespace {

// Memory that a call reads, or writes.
struct Span {
    Extent at;
    bool written;
};

// True: nothing that is written is anything else's, too.  Looked through in the order of the addresses, which lists often come in.
bool written_apart(Span *spans, size_t n)
{
    const auto before = [](const Span &a, const Span &b) { return a.at.begin < b.at.begin; };
    if (!std::is_sorted(spans, spans + n, before)) std::sort(spans, spans + n, before);
    uintptr_t any = 0, written = 0;             // where what came so far ends
    for (size_t i = 0; i < n; ++i) {
        const Span &s = spans[i];
        if (s.at.begin < (s.written ? any : written)) return false;
        any = std::max(any, s.at.end);
        if (s.written) written = std::max(written, s.at.end);
    }
    return true;
}

// Clipped or not: every tensor is there, has a type and room in the address space, and lies apart from the norm and the workspace.
int check_grads(const seer_grad *tensors, int32_t count, const float *norm, bool clip, void *workspace, size_t workspace_bytes)
{
    if (count < 0 || (count > 0 && !tensors) || bad_pointer(norm, 4)) return SEER_EINVAL;
    const Extent at_norm = extent(norm, 4), at_ws = extent(workspace, workspace ? std::min(workspace_bytes, grad_workspace_bytes()) : 0);
    const auto apart_from_both = [&](const void *p, size_t bytes) {
        const Extent e = extent(p, bytes);
        return !overlap(e, at_norm) && !overlap(e, at_ws);
    };
    if (overlap(at_norm, at_ws)) return SEER_EINVAL;
    size_t spans = 0;
    for (int32_t i = 0; i < count; ++i) {
        const seer_grad &t = tensors[i];
        if (t.n < 0 || t.n > INT64_MAX / 8 || !is_float(t.type)) return SEER_EINVAL;
        if (t.n == 0) continue;
        const size_t size = size_of(t.type);
        if (bad_pointer(t.grad, size) || !apart_from_both(t.grad, (size_t)t.n * size)) return SEER_EINVAL;
        if (!clip) continue;
        if (bad_pointer(t.out, size) || !apart_from_both(t.out, (size_t)t.n * size)) return SEER_EINVAL;
        spans += t.out == t.grad ? 1 : 2;
    }
    if (spans < 2) return SEER_OK;
    // what is clipped lies apart from every other gradient and from what else is clipped
    Span few[128], *list = spans <= sizeof few / sizeof *few ? few : static_cast<Span *>(std::malloc(spans * sizeof(Span)));
    if (!list) return SEER_EINVAL;
    size_t n = 0;
    for (int32_t i = 0; i < count; ++i) {
        const seer_grad &t = tensors[i];
        if (t.n == 0) continue;
        const size_t bytes = (size_t)t.n * size_of(t.type);
        list[n++] = Span{extent(t.out, bytes), true};
        if (t.out != t.grad) list[n++] = Span{extent(t.grad, bytes), false};
    }
    const bool apart = written_apart(list, n);
    if (list != few) std::free(list);
    return apart ? SEER_OK : SEER_EINVAL;
}

} // namespace

extern "C" {

size_t seer_route_workspace_bytes(int32_t tokens, int32_t choices, int32_t experts)
{
    if (tokens < 0 || choices < 1 || experts < 1 || experts > SEER_MAX_EXPERTS || (int64_t)tokens * choices > INT32_MAX) return 0;
    return route_workspace_bytes((uint32_t)tokens * (uint32_t)choices, (uint32_t)experts);
}

int seer_route(const void *expert, int32_t index_type, const seer_routing *r, void *workspace, size_t workspace_bytes,
               void *stream)
{
    const int rc = check_routing(r, true);
    if (rc != SEER_OK) return rc;
    if (index_type != SEER_I32 && index_type != SEER_I64) return SEER_EINVAL;
    const uint32_t count = (uint32_t)r->tokens * (uint32_t)r->choices;
    if (bad_pointer(r->expert_ptr, 4)) return SEER_EINVAL;
    if (count && (bad_pointer(r->slot_choice, 4) || bad_pointer(expert, index_type == SEER_I64 ? 8 : 4))) return SEER_EINVAL;
    const Extent in = extent(expert, (size_t)count * (index_type == SEER_I64 ? 8 : 4));
    const Extent ptr = extent(r->expert_ptr, ((size_t)r->experts + 1) * 4), order = extent(r->slot_choice, (size_t)count * 4),
                 slots = extent(r->choice_slot, (size_t)count * 4);
    if (overlap(in, ptr) || overlap(in, order) || overlap(in, slots) || overlap(ptr, order) || overlap(ptr, slots) || overlap(order, slots))
        return SEER_EINVAL;
    const size_t need = route_workspace_bytes(count, (uint32_t)r->experts);
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return SEER_EWORKSPACE;
    const Extent ws = extent(workspace, need);
    if (overlap(ws, in) || overlap(ws, ptr) || overlap(ws, order) || overlap(ws, slots)) return SEER_EINVAL;
    launch_route(expert, index_type == SEER_I64, count, (uint32_t)r->experts, r->expert_ptr, r->slot_choice, r->choice_slot,
                 workspace, on(stream));
    return done();
}

int seer_route_gather(const seer_routing *r, const seer_dense *x, const float *weight, const seer_dense *out, void *stream)
{
    int rc = check_routing(r, true);
    if (rc != SEER_OK) return rc;
    if (!x || !out) return SEER_EINVAL;
    const int64_t count = (int64_t)r->tokens * r->choices;
    if ((rc = check_dense(x, r->tokens, x->cols, -1)) != SEER_OK || (rc = check_dense(out, count, x->cols, x->type)) != SEER_OK) return rc;
    if (weight && bad_pointer(weight, 4)) return SEER_EINVAL;
    if (count == 0 || x->cols == 0) return SEER_OK;
    if (overlap(extent(out), extent(x)) || overlap(extent(out), extent(weight, weight ? (size_t)count * 4 : 0)) ||
        overlap(extent(out), extent(r->choice_slot, (size_t)count * 4)))
        return SEER_EINVAL;
    launch_route_gather(rows_of(r, x->cols), weight, *x, *out, on(stream));
    return done();
}

int seer_route_combine(const seer_routing *r, const seer_dense *z, const float *weight, const seer_dense *y, void *stream)
{
    int rc = check_routing(r, true);
    if (rc != SEER_OK) return rc;
    if (!z || !y) return SEER_EINVAL;
    const int64_t count = (int64_t)r->tokens * r->choices;
    if ((rc = check_dense(z, count, z->cols, -1)) != SEER_OK || (rc = check_dense(y, r->tokens, z->cols, z->type)) != SEER_OK) return rc;
    if (weight && bad_pointer(weight, 4)) return SEER_EINVAL;
    if (count == 0 || z->cols == 0) return SEER_OK;
    if (overlap(extent(y), extent(z)) || overlap(extent(y), extent(weight, weight ? (size_t)count * 4 : 0)) ||
        overlap(extent(y), extent(r->choice_slot, (size_t)count * 4)))
        return SEER_EINVAL;
    launch_route_combine(rows_of(r, z->cols), weight, *z, *y, on(stream));
    return done();
}

int seer_route_grad(const seer_routing *r, const seer_dense *dy, const seer_dense *z, const float *weight, const seer_dense *dz,
                    float *dweight, void *stream)
{
    int rc = check_routing(r, true);
    if (rc != SEER_OK) return rc;
    if (!dy || (!z && dweight)) return SEER_EINVAL;
    const int64_t count = (int64_t)r->tokens * r->choices;
    if ((rc = check_dense(dy, r->tokens, dy->cols, -1)) != SEER_OK) return rc;
    if (z && (rc = check_dense(z, count, dy->cols, dy->type)) != SEER_OK) return rc;
    if (dz && (rc = check_dense(dz, count, dy->cols, dy->type)) != SEER_OK) return rc;
    if ((weight && bad_pointer(weight, 4)) || (dweight && bad_pointer(dweight, 4))) return SEER_EINVAL;
    if (count == 0 || (!dz && !dweight)) return SEER_OK;
    const Extent ins[] = {extent(dy), z ? extent(z) : Extent{0, 0}, extent(weight, weight ? (size_t)count * 4 : 0),
                          extent(r->choice_slot, (size_t)count * 4)};
    const Extent rows = dz ? extent(dz) : Extent{0, 0}, dots = extent(dweight, dweight ? (size_t)count * 4 : 0);
    if (overlap(rows, dots)) return SEER_EINVAL;
    for (const Extent &in : ins)
        if (overlap(in, rows) || overlap(in, dots)) return SEER_EINVAL;
    launch_route_grad(rows_of(r, dy->cols), weight, *dy, z, dz, dweight, on(stream));
    return done();
}

// What a quantisation writes to q: the columns that are set to zero belong to it, too, also behind its last row.
static Extent quantised_extent(const seer_dense *q)
{
    if (q->rows == 0) return {0, 0};
    return extent(q->data, (size_t)((q->rows - 1) * q->ld + std::min<int64_t>(q->ld, (q->cols + 15) & ~(int64_t)15)));
}

// q and scale of `rows` rows, and their input.
static int check_quantized(const seer_dense *x, const seer_dense *q, const float *scale, int64_t rows)
{
    if (!q || q->type != SEER_I8) return SEER_EINVAL;
    const int rc = check_dense(q, rows, x->cols, SEER_I8);
    if (rc != SEER_OK) return rc;
    if (rows > 0 && bad_pointer(scale, 4)) return SEER_EINVAL;
    const Extent qe = quantised_extent(q), se = extent(scale, (size_t)rows * 4);
    if (overlap(qe, se) || overlap(qe, extent(x)) || overlap(se, extent(x))) return SEER_EINVAL;
    return SEER_OK;
}

int seer_i8_quantize(const seer_dense *x, const seer_dense *q, float *scale, void *stream)
{
    if (!x) return SEER_EINVAL;
    int rc = check_dense(x, x->rows, x->cols, -1);
    if (rc != SEER_OK || (rc = check_quantized(x, q, scale, x->rows)) != SEER_OK) return rc;
    if (x->rows == 0) return SEER_OK;
    launch_quantize(RouteRows{nullptr, (uint32_t)x->rows, 1, (uint32_t)x->cols}, *x, *q, scale, on(stream));
    return done();
}

int seer_route_gather_i8(const seer_routing *r, const seer_dense *x, const seer_dense *q, float *scale, void *stream)
{
    int rc = check_routing(r, true);
    if (rc != SEER_OK) return rc;
    if (!x) return SEER_EINVAL;
    const int64_t count = (int64_t)r->tokens * r->choices;
    if ((rc = check_dense(x, r->tokens, x->cols, -1)) != SEER_OK || (rc = check_quantized(x, q, scale, count)) != SEER_OK) return rc;
    if (count == 0) return SEER_OK;
    const Extent slots = extent(r->choice_slot, (size_t)count * 4);
    if (overlap(slots, quantised_extent(q)) || overlap(slots, extent(scale, (size_t)count * 4))) return SEER_EINVAL;
    launch_quantize(rows_of(r, x->cols), *x, *q, scale, on(stream));
    return done();
}

size_t seer_i8_product_workspace_bytes(int64_t rows, int64_t channels, int64_t columns, int32_t groups)
{
    if (rows < 0 || channels < 0 || columns < 0 || groups < 1 || rows > INT32_MAX || channels > INT32_MAX || columns > SEER_I8_MAX_K) return 0;
    return i8_workspace_bytes((uint32_t)rows, (uint32_t)channels, (uint32_t)columns, (uint32_t)groups);
}

int seer_i8_product(const seer_dense *a, const float *a_scale, const seer_dense *b, const float *b_scale, const int32_t *group_ptr,
                    int32_t groups, const seer_dense *out, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!a || !b || !out || groups < 1 || (!group_ptr && groups != 1)) return SEER_EINVAL;
    int rc;
    if ((rc = check_dense(a, a->rows, a->cols, SEER_I8)) != SEER_OK || (rc = check_dense(out, a->rows, out->cols, -1)) != SEER_OK) return rc;
    if (out->cols > INT32_MAX / groups) return SEER_EINVAL;
    if ((rc = check_dense(b, (int64_t)groups * out->cols, a->cols, SEER_I8)) != SEER_OK) return rc;
    if (a->cols > SEER_I8_MAX_K) return SEER_ELIMIT;
    if (a->rows == 0 || out->cols == 0) return SEER_OK;
    if (bad_pointer(a_scale, 4) || bad_pointer(b_scale, 4) || (group_ptr && bad_pointer(group_ptr, 4))) return SEER_EINVAL;
    const Extent to = extent(out), ins[] = {extent(a), extent(b), extent(a_scale, (size_t)a->rows * 4), extent(b_scale, (size_t)b->rows * 4),
                                            extent(group_ptr, group_ptr ? ((size_t)groups + 1) * 4 : 0)};
    for (const Extent &in : ins)
        if (overlap(to, in)) return SEER_EINVAL;
    I8Args p{static_cast<const int8_t *>(a->data), static_cast<const int8_t *>(b->data), a_scale, b_scale, group_ptr, out->data,
             a->ld, b->ld, out->ld, (uint32_t)a->rows, (uint32_t)out->cols, (uint32_t)a->cols, (uint32_t)groups, out->type};
    if (!i8_product_fits(p)) return SEER_ELIMIT;
    const I8Plan plan = i8_plan(p);
    const size_t need = plan.kernel == SEER_I8_SHARED ? i8_workspace_bytes(p.rows, p.channels, p.columns, p.groups) : 0;
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return SEER_EWORKSPACE;
    const Extent ws = extent(workspace, need);
    if (overlap(ws, to)) return SEER_EINVAL;
    for (const Extent &in : ins)
        if (overlap(ws, in)) return SEER_EINVAL;
    launch_i8_product(p, plan, workspace, on(stream));
    return done();
}

int seer_i8_product_kernel(const seer_dense *a, const seer_dense *b, const int32_t *group_ptr, int32_t groups)
{
    if (!a || !b || groups < 1 || (!group_ptr && groups != 1)) return SEER_EINVAL;
    int rc;
    if ((rc = check_dense(a, a->rows, a->cols, SEER_I8)) != SEER_OK || (rc = check_dense(b, b->rows, a->cols, SEER_I8)) != SEER_OK) return rc;
    if (b->rows % groups != 0) return SEER_EINVAL;
    if (a->cols > SEER_I8_MAX_K) return SEER_ELIMIT;
    I8Args p{static_cast<const int8_t *>(a->data), static_cast<const int8_t *>(b->data), nullptr, nullptr, group_ptr, nullptr, a->ld, b->ld, 0,
             (uint32_t)a->rows, (uint32_t)(b->rows / groups), (uint32_t)a->cols, (uint32_t)groups, SEER_F32};
    if (!i8_product_fits(p)) return SEER_ELIMIT;
    return p.rows == 0 || p.channels == 0 ? SEER_I8_NONE : i8_plan(p).kernel;
}

// Rows of 4-bit values: their blocks are whole and lie at multiples of 16 bytes.
static int check_mx4(const seer_mx4 *m, int64_t rows, int64_t cols)
{
    if (!m || m->rows != rows || m->cols != cols || rows < 0 || cols < 0 || rows > INT32_MAX || cols > INT32_MAX) return SEER_EINVAL;
    const int64_t blocks = (cols + 31) / 32;
    if (m->ld < 16 * blocks || (rows > 1 && cols > 0 && m->ld % 16 != 0) || m->scale_ld < blocks) return SEER_EINVAL;
    if (rows > 0 && (m->ld > (INT64_MAX / 8) / rows || m->scale_ld > (INT64_MAX / 8) / rows)) return SEER_EINVAL;
    if (rows > 0 && cols > 0 && (bad_pointer(m->data, 16) || !m->scale)) return SEER_EINVAL;
    return SEER_OK;
}
static Extent codes_extent(const seer_mx4 *m)
{
    if (m->rows == 0 || m->cols == 0) return {0, 0};
    return extent(m->data, (size_t)((m->rows - 1) * m->ld + (m->cols + 31) / 32 * 16));
}
static Extent scales_extent(const seer_mx4 *m)
{
    if (m->rows == 0 || m->cols == 0) return {0, 0};
    return extent(m->scale, (size_t)((m->rows - 1) * m->scale_ld + (m->cols + 31) / 32));
}

static int quantize_mx4(const RouteRows &r, const seer_dense *x, const seer_mx4 *q, int64_t rows, Extent slots, void *stream)
{
    int rc;
    if ((rc = check_dense(x, r.tokens, x->cols, -1)) != SEER_OK || (rc = check_mx4(q, rows, x->cols)) != SEER_OK) return rc;
    if (rows == 0 || x->cols == 0) return SEER_OK;
    const Extent codes = codes_extent(q), scales = scales_extent(q), in = extent(x);
    if (overlap(codes, scales) || overlap(codes, in) || overlap(scales, in) || overlap(codes, slots) || overlap(scales, slots)) return SEER_EINVAL;
    launch_mx4_quantize(r, *x, *q, on(stream));
    return done();
}

int seer_mx4_quantize(const seer_dense *x, const seer_mx4 *q, void *stream)
{
    if (!x || x->rows < 0 || x->rows > INT32_MAX) return SEER_EINVAL;
    return quantize_mx4(RouteRows{nullptr, (uint32_t)x->rows, 1, (uint32_t)x->cols}, x, q, x->rows, Extent{0, 0}, stream);
}

int seer_route_gather_mx4(const seer_routing *r, const seer_dense *x, const seer_mx4 *q, void *stream)
{
    const int rc = check_routing(r, true);
    if (rc != SEER_OK) return rc;
    if (!x) return SEER_EINVAL;
    const int64_t count = (int64_t)r->tokens * r->choices;
    return quantize_mx4(rows_of(r, x->cols), x, q, count, extent(r->choice_slot, (size_t)count * 4), stream);
}

size_t seer_mx4_product_workspace_bytes(int64_t rows, int64_t channels, int64_t columns, int32_t groups)
{
    if (rows < 0 || channels < 0 || columns < 0 || groups < 1 || rows > INT32_MAX || channels > INT32_MAX || columns > INT32_MAX) return 0;
    return mx4_workspace_bytes((uint32_t)rows, (uint32_t)channels, (uint32_t)((columns + 31) / 32), (uint32_t)groups);
}

int seer_mx4_product(const seer_mx4 *a, const seer_mx4 *b, const int32_t *group_ptr, int32_t groups, const seer_dense *out, void *workspace,
                     size_t workspace_bytes, void *stream)
{
    if (!a || !b || !out || groups < 1 || (!group_ptr && groups != 1)) return SEER_EINVAL;
    int rc;
    if ((rc = check_mx4(a, a->rows, a->cols)) != SEER_OK || (rc = check_dense(out, a->rows, out->cols, -1)) != SEER_OK) return rc;
    if (out->cols > INT32_MAX / groups) return SEER_EINVAL;
    if ((rc = check_mx4(b, (int64_t)groups * out->cols, a->cols)) != SEER_OK) return rc;
    if (groups > SEER_MAX_EXPERTS) return SEER_ELIMIT;
    if (a->rows == 0 || out->cols == 0) return SEER_OK;
    if (group_ptr && bad_pointer(group_ptr, 4)) return SEER_EINVAL;
    const Extent to = extent(out), ins[] = {codes_extent(a), codes_extent(b), scales_extent(a), scales_extent(b),
                                            extent(group_ptr, group_ptr ? ((size_t)groups + 1) * 4 : 0)};
    for (const Extent &in : ins)
        if (overlap(to, in)) return SEER_EINVAL;
    const auto bytes = [](const void *p) { return static_cast<const uint8_t *>(p); };
    const Mx4Args p{bytes(a->data), bytes(b->data), bytes(a->scale), bytes(b->scale), group_ptr, out->data, a->ld, b->ld, a->scale_ld, b->scale_ld, out->ld,
                    (uint32_t)a->rows, (uint32_t)out->cols, (uint32_t)((a->cols + 31) / 32), (uint32_t)groups, out->type};
    if (!mx4_product_fits(p)) return SEER_ELIMIT;
    const Mx4Plan plan = mx4_plan(p);
    const size_t need = plan.kernel == SEER_MX4_SHARED ? mx4_workspace_bytes(p.rows, p.channels, p.blocks, p.groups) : 0;
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return SEER_EWORKSPACE;
    const Extent ws = extent(workspace, need);
    if (overlap(ws, to)) return SEER_EINVAL;
    for (const Extent &in : ins)
        if (overlap(ws, in)) return SEER_EINVAL;
    launch_mx4_product(p, plan, workspace, on(stream));
    return done();
}

int seer_mx4_product_plan(const seer_mx4 *a, const seer_mx4 *b, const int32_t *group_ptr, int32_t groups, int32_t *tokens, int32_t *shares)
{
    if (!a || !b || groups < 1 || (!group_ptr && groups != 1)) return SEER_EINVAL;
    int rc;
    if ((rc = check_mx4(a, a->rows, a->cols)) != SEER_OK || (rc = check_mx4(b, b->rows, a->cols)) != SEER_OK) return rc;
    if (b->rows % groups != 0) return SEER_EINVAL;
    const Mx4Args p{nullptr, nullptr, nullptr, nullptr, group_ptr, nullptr, a->ld, b->ld, a->scale_ld, b->scale_ld, 0,
                    (uint32_t)a->rows, (uint32_t)(b->rows / groups), (uint32_t)((a->cols + 31) / 32), (uint32_t)groups, SEER_F32};
    if (!mx4_product_fits(p)) return SEER_ELIMIT;
    const Mx4Plan plan = p.rows == 0 || p.channels == 0 ? Mx4Plan{SEER_MX4_NONE, 0, 1} : mx4_plan(p);
    if (tokens) *tokens = (int32_t)plan.tokens;
    if (shares) *shares = (int32_t)plan.shares;
    return plan.kernel;
}

int seer_mx4_product_kernel(const seer_mx4 *a, const seer_mx4 *b, const int32_t *group_ptr, int32_t groups)
{
    return seer_mx4_product_plan(a, b, group_ptr, groups, nullptr, nullptr);
}

size_t seer_grad_workspace_bytes(void) { return grad_workspace_bytes(); }

int seer_grad_norm(const seer_grad *tensors, int32_t count, float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = check_grads(tensors, count, norm, false, workspace, workspace_bytes);
    if (rc != SEER_OK) return rc;
    if (!workspace || !aligned16(workspace) || workspace_bytes < grad_workspace_bytes()) return SEER_EWORKSPACE;
    launch_grad_norm(tensors, count, norm, workspace, on(stream));
    return done();
}

int seer_grad_clip(const seer_grad *tensors, int32_t count, float max_norm, float *norm, void *workspace, size_t workspace_bytes,
                   void *stream)
{
    const int rc = check_grads(tensors, count, norm, true, workspace, workspace_bytes);
    if (rc != SEER_OK) return rc;
    if (!(max_norm >= 0.0f)) return SEER_EINVAL;
    if (!workspace || !aligned16(workspace) || workspace_bytes < grad_workspace_bytes()) return SEER_EWORKSPACE;
    launch_grad_clip(tensors, count, max_norm, norm, workspace, on(stream));
    return done();
}

} // extern "C"

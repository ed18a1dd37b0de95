// C ABI of what a routed layer is fed by: the router's choice and the embedding of tokens.  Checks of arguments, then the launches.
#include "dense_checks.h"

#include <cmath>

using namespace seer;

namespace {

int check_choice(const seer_dense *logits, const seer_choice *how)
{
    if (!logits || !how) return SEER_EINVAL;
    const int rc = check_dense(logits, logits->rows, logits->cols, -1);
    if (rc != SEER_OK) return rc;
    if (logits->cols < 1 || how->choices < 1 || how->groups < 1 || how->best_groups < 1 || how->best_groups > how->groups) return SEER_EINVAL;
    if (logits->cols > SEER_MAX_EXPERTS || how->choices > SEER_MAX_CHOICES || how->groups > SEER_MAX_EXPERT_GROUPS) return SEER_ELIMIT;
    if (logits->cols % how->groups != 0 || how->choices > logits->cols / how->groups * how->best_groups) return SEER_EINVAL;
    if ((how->score != SEER_SOFTMAX && how->score != SEER_SIGMOID) || (how->group_best != 1 && how->group_best != 2) || !std::isfinite(how->factor))
        return SEER_EINVAL;
    if (logits->rows * how->choices > INT32_MAX) return SEER_EINVAL;
    return SEER_OK;
}

int check_tokens(const void *token, int32_t index_type, int64_t tokens)
{
    if (index_type != SEER_I32 && index_type != SEER_I64) return SEER_EINVAL;
    return tokens > 0 && bad_pointer(token, index_type == SEER_I64 ? 8 : 4) ? SEER_EINVAL : SEER_OK;
}
Extent token_extent(const void *token, int32_t index_type, int64_t tokens) { return extent(token, (size_t)tokens * (index_type == SEER_I64 ? 8 : 4)); }

} // namespace

extern "C" {

int seer_route_choose(const seer_dense *logits, const float *bias, const seer_choice *how, int32_t *expert, float *weight, void *stream)
{
    const int rc = check_choice(logits, how);
    if (rc != SEER_OK) return rc;
    if (bias && bad_pointer(bias, 4)) return SEER_EINVAL;
    if (logits->rows == 0) return SEER_OK;
    if (bad_pointer(expert, 4) || bad_pointer(weight, 4)) return SEER_EINVAL;
    const size_t bytes = (size_t)logits->rows * how->choices * 4;
    const Extent e = extent(expert, bytes), w = extent(weight, bytes), x = extent(logits), b = extent(bias, bias ? (size_t)logits->cols * 4 : 0);
    if (overlap(e, w) || overlap(e, x) || overlap(e, b) || overlap(w, x) || overlap(w, b)) return SEER_EINVAL;
    launch_choose(*logits, bias, *how, expert, weight, on(stream));
    return done();
}

int seer_route_choose_grad(const seer_dense *logits, const seer_choice *how, const int32_t *expert, const float *dweight,
                           const seer_dense *dlogits, void *stream)
{
    int rc = check_choice(logits, how);
    if (rc != SEER_OK) return rc;
    if (!dlogits) return SEER_EINVAL;
    if ((rc = check_dense(dlogits, logits->rows, logits->cols, logits->type)) != SEER_OK) return rc;
    if (logits->rows == 0) return SEER_OK;
    if (bad_pointer(expert, 4) || bad_pointer(dweight, 4)) return SEER_EINVAL;
    const size_t bytes = (size_t)logits->rows * how->choices * 4;
    const Extent to = extent(dlogits);
    if (overlap(to, extent(logits)) || overlap(to, extent(expert, bytes)) || overlap(to, extent(dweight, bytes))) return SEER_EINVAL;
    launch_choose_grad(*logits, *how, expert, dweight, *dlogits, on(stream));
    return done();
}

int seer_embed(const void *token, int32_t index_type, const seer_dense *table, float scale, const seer_dense *out, void *stream)
{
    if (!table || !out) return SEER_EINVAL;
    int rc;
    if ((rc = check_dense(table, table->rows, table->cols, -1)) != SEER_OK ||
        (rc = check_dense(out, out->rows, table->cols, table->type)) != SEER_OK || (rc = check_tokens(token, index_type, out->rows)) != SEER_OK)
        return rc;
    if (out->rows == 0 || out->cols == 0) return SEER_OK;
    const Extent to = extent(out);
    if (overlap(to, extent(table)) || overlap(to, token_extent(token, index_type, out->rows))) return SEER_EINVAL;
    launch_embed(token, index_type == SEER_I64, (uint32_t)out->rows, *table, scale, *out, on(stream));
    return done();
}

size_t seer_embed_grad_workspace_bytes(int64_t tokens, int64_t rows, int64_t columns)
{
    if (tokens < 0 || rows < 0 || columns < 0 || tokens > INT32_MAX || rows > INT32_MAX || columns > INT32_MAX) return 0;
    return embed_grad_workspace_bytes((uint32_t)tokens, (uint32_t)rows, (uint32_t)columns);
}

int seer_embed_grad(const void *token, int32_t index_type, const seer_dense *dy, float scale, int32_t accumulate, const seer_dense *dtable,
                    void *workspace, size_t workspace_bytes, void *stream)
{
    if (!dy || !dtable) return SEER_EINVAL;
    int rc;
    if ((rc = check_dense(dy, dy->rows, dy->cols, -1)) != SEER_OK || (rc = check_dense(dtable, dtable->rows, dy->cols, -1)) != SEER_OK ||
        (rc = check_tokens(token, index_type, dy->rows)) != SEER_OK)
        return rc;
    if (dtable->type != dy->type && dtable->type != SEER_F32) return SEER_EINVAL;
    if (dtable->rows == 0 || dy->cols == 0 || (accumulate && dy->rows == 0)) return SEER_OK;
    const Extent to = extent(dtable), y = extent(dy), ids = token_extent(token, index_type, dy->rows);
    if (overlap(to, y) || overlap(to, ids)) return SEER_EINVAL;
    const size_t need = embed_grad_workspace_bytes((uint32_t)dy->rows, (uint32_t)dtable->rows, (uint32_t)dy->cols);
    if (need && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return SEER_EWORKSPACE;
    const Extent ws = extent(workspace, need);
    if (overlap(ws, to) || overlap(ws, y) || overlap(ws, ids)) return SEER_EINVAL;
    launch_embed_grad(token, index_type == SEER_I64, *dy, scale, accumulate != 0, *dtable, workspace, on(stream));
    return done();
}

} // extern "C"

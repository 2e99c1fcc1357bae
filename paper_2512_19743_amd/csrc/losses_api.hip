// Host side of the losses on features and on routed experts: argument checks,
// workspace sizes, launches. No call allocates, synchronises or reads device
// memory, so every one can be captured into a graph.
#include <cmath>
#include <cstdio>

#include "../../include/apml.h"
#include "balance.h"
#include "errors.h"
#include "linear_ce.h"

using namespace apml;

namespace {

apml_status bad(const char *msg) { return fail_with(APML_ERR_INVALID_ARG, msg); }

apml_status short_workspace(const char *call, size_t need, size_t have)
{
    char text[160];
    std::snprintf(text, sizeof(text), "%s needs a workspace of %zu bytes, got %zu", call, need, have);
    return fail_with(APML_ERR_INVALID_ARG, text);
}

apml_status launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? APML_OK : fail_with(APML_ERR_DEVICE, hipGetErrorString(e));
}

bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

apml_status check_desc(const apml_linear_ce_desc *d)
{
    if (!d)
        return bad("desc must be non-NULL");
    if (d->struct_size < sizeof(apml_linear_ce_desc))
        return bad("apml_linear_ce_desc.struct_size is smaller than this library's struct");
    if (d->dtype < APML_F32 || d->dtype > APML_F16)
        return bad("dtype must be APML_F32, APML_BF16 or APML_F16");
    if (d->target_type != APML_I64 && d->target_type != APML_I32)
        return bad("target_type must be APML_I64 or APML_I32");
    if (d->reduction < APML_REDUCE_NONE || d->reduction > APML_REDUCE_MEAN)
        return bad("reduction must be APML_REDUCE_NONE, _SUM or _MEAN");
    if (d->samples < 1 || d->rows < 1 || d->classes < 1 || d->dim < 1)
        return bad("need samples >= 1, rows >= 1, classes >= 1 and dim >= 1");
    if (!std::isfinite(d->scale) || !std::isfinite(d->z_weight))
        return bad("scale and z_weight must be finite");
    if (!std::isfinite(d->scale * kLog2E)) // what the logits are multiplied by
        return bad("scale must lie within +-2.35e38");
    // a launch's workgroups and the offsets within a tile are 32-bit
    if (d->dim > (1 << 20) || d->classes > (1 << 26) || (int64_t)d->samples * d->rows > (1 << 26))
        return fail_with(APML_ERR_UNSUPPORTED, "dim beyond 2^20, classes beyond 2^26 or samples * rows beyond 2^26");
    if ((((int64_t)d->classes + 127) / 128) * (((int64_t)d->dim + 127) / 128) * d->samples > ((int64_t)1 << 24))
        return fail_with(APML_ERR_UNSUPPORTED, "too many classes and features for one launch");
    return APML_OK;
}

apml_status check_launches(const CeProblem &p)
{
    return ce_launches_fit(p) ? APML_OK : fail_with(APML_ERR_UNSUPPORTED, "too many rows, classes or features for one launch");
}

CeProblem problem_of(const apml_linear_ce_desc &d, const void *x, const void *w, const void *target)
{
    CeProblem p{};
    p.type = (ElemType)d.dtype;
    p.target32 = d.target_type == APML_I32;
    p.samples = d.samples;
    p.rows = d.rows;
    p.classes = d.classes;
    p.dim = d.dim;
    p.scale = d.scale;
    p.z_weight = d.z_weight;
    p.ignore_index = d.ignore_index;
    p.reduction = d.reduction;
    p.x = x;
    p.w = w;
    p.target = target;
    return p;
}

apml_status check_inputs(const apml_linear_ce_desc &d, const void *x, const void *w, const void *target,
                         const void *workspace)
{
    if (!x || !w || !target || !workspace)
        return bad("x, w, target and workspace must be non-NULL device pointers");
    const size_t size = elem_size((ElemType)d.dtype);
    if (!aligned(x, size) || !aligned(w, size) || !aligned(target, d.target_type == APML_I32 ? 4 : 8))
        return bad("x, w and target must be aligned to their elements");
    if (!aligned(workspace, 256))
        return bad("workspace must be aligned to 256 bytes");
    return APML_OK;
}

// What a pointer that is not known yet may need: copies of both operands.
const void *const kUnaligned = (const void *)1;

apml_status check_balance(const apml_balance_desc *d)
{
    if (!d)
        return bad("desc must be non-NULL");
    if (d->struct_size < sizeof(apml_balance_desc))
        return bad("apml_balance_desc.struct_size is smaller than this library's struct");
    if (d->dtype < APML_F32 || d->dtype > APML_F16)
        return bad("dtype must be APML_F32, APML_BF16 or APML_F16");
    if (d->index_type != APML_I64 && d->index_type != APML_I32)
        return bad("index_type must be APML_I64 or APML_I32");
    if (d->reduction < APML_REDUCE_NONE || d->reduction > APML_REDUCE_MEAN)
        return bad("reduction must be APML_REDUCE_NONE, _SUM or _MEAN");
    if (d->samples < 1 || d->tokens < 1 || d->experts < 1 || d->chosen < 1)
        return bad("need samples >= 1, tokens >= 1, experts >= 1 and chosen >= 1");
    if (!std::isfinite(d->z_weight))
        return bad("z_weight must be finite");
    if (d->experts > kMaxExperts)
        return fail_with(APML_ERR_UNSUPPORTED, "more than 1024 experts");
    if (d->samples > (1 << 20) || (int64_t)d->samples * d->tokens > (1 << 30) ||
        (int64_t)d->tokens * d->chosen > (1 << 30))
        return fail_with(APML_ERR_UNSUPPORTED,
                         "samples beyond 2^20, samples * tokens beyond 2^30 or tokens * chosen beyond 2^30");
    return APML_OK;
}

BalanceProblem problem_of(const apml_balance_desc &d, const void *logits, const void *index, const uint8_t *valid)
{
    BalanceProblem p{};
    p.type = (ElemType)d.dtype;
    p.index32 = d.index_type == APML_I32;
    p.samples = d.samples;
    p.tokens = d.tokens;
    p.experts = d.experts;
    p.chosen = d.chosen;
    p.reduction = d.reduction;
    p.z_weight = d.z_weight;
    p.logits = logits;
    p.index = index;
    p.valid = valid;
    return p;
}

} // namespace

extern "C" {

void apml_linear_ce_desc_default(apml_linear_ce_desc *d)
{
    *d = apml_linear_ce_desc{};
    d->struct_size = sizeof(*d);
    d->samples = 1;
    d->scale = 1.0f;
    d->ignore_index = -100;
    d->reduction = APML_REDUCE_MEAN;
}

apml_status apml_linear_ce_workspace(const apml_linear_ce_desc *desc, const void *x, const void *w,
                                     size_t *forward_bytes, size_t *backward_bytes)
{
    clear_error();
    if (const apml_status st = check_desc(desc))
        return st;
    if (!forward_bytes && !backward_bytes)
        return bad("forward_bytes or backward_bytes must be non-NULL");
    const CeProblem p = problem_of(*desc, x ? x : kUnaligned, w ? w : kUnaligned, nullptr);
    if (const apml_status st = check_launches(p))
        return st;
    if (forward_bytes)
        *forward_bytes = ce_plan_forward(p).bytes;
    if (backward_bytes)
        *backward_bytes = ce_plan_backward(p, true, true).bytes;
    return APML_OK;
}

apml_status apml_linear_ce_forward(const apml_linear_ce_desc *desc, const void *x, const void *w, const void *target,
                                   float *loss, float *state, void *workspace, size_t workspace_bytes,
                                   apml_stream stream)
{
    clear_error();
    if (const apml_status st = check_desc(desc))
        return st;
    if (!loss)
        return bad("loss must be a non-NULL device pointer");
    if (const apml_status st = check_inputs(*desc, x, w, target, workspace))
        return st;
    if (!aligned(loss, 4) || !aligned(state, 16))
        return bad("loss must be aligned to 4 bytes, state to 16");
    const CeProblem p = problem_of(*desc, x, w, target);
    if (const apml_status st = check_launches(p))
        return st;
    const CeForwardPlan plan = ce_plan_forward(p);
    if (workspace_bytes < plan.bytes)
        return short_workspace("apml_linear_ce_forward", plan.bytes, workspace_bytes);
    auto *rows = (CeRow *)state;
    float *total = state ? state + 4 * (int64_t)p.samples * p.rows : nullptr;
    ce_forward(p, plan, (uint8_t *)workspace, loss, rows, total, (hipStream_t)stream);
    return launched();
}

apml_status apml_linear_ce_backward(const apml_linear_ce_desc *desc, const void *x, const void *w, const void *target,
                                    const float *state, const float *grad_loss, void *grad_x, void *grad_w,
                                    void *workspace, size_t workspace_bytes, apml_stream stream)
{
    clear_error();
    if (const apml_status st = check_desc(desc))
        return st;
    if (!state || !grad_loss || (!grad_x && !grad_w))
        return bad("state, grad_loss and one of grad_x and grad_w must be non-NULL device pointers");
    if (const apml_status st = check_inputs(*desc, x, w, target, workspace))
        return st;
    const size_t size = elem_size((ElemType)desc->dtype);
    if (!aligned(state, 16) || !aligned(grad_x, size) || !aligned(grad_w, size) || !aligned(grad_loss, 4))
        return bad("state must be aligned to 16 bytes, the gradients to their elements");
    const CeProblem p = problem_of(*desc, x, w, target);
    if (const apml_status st = check_launches(p))
        return st;
    const CeBackwardPlan plan = ce_plan_backward(p, grad_x, grad_w);
    if (workspace_bytes < plan.bytes)
        return short_workspace("apml_linear_ce_backward", plan.bytes, workspace_bytes);
    ce_backward(p, plan, (uint8_t *)workspace, (const CeRow *)state, state + 4 * (int64_t)p.samples * p.rows, grad_loss,
                grad_x, grad_w, (hipStream_t)stream);
    return launched();
}

void apml_balance_desc_default(apml_balance_desc *d)
{
    *d = apml_balance_desc{};
    d->struct_size = sizeof(*d);
    d->samples = 1;
    d->chosen = 1;
    d->reduction = APML_REDUCE_MEAN;
}

apml_status apml_balance_workspace(const apml_balance_desc *desc, size_t *bytes)
{
    clear_error();
    if (const apml_status st = check_balance(desc))
        return st;
    if (!bytes)
        return bad("bytes must be non-NULL");
    *bytes = balance_plan(problem_of(*desc, nullptr, nullptr, nullptr)).bytes;
    return APML_OK;
}

apml_status apml_balance_forward(const apml_balance_desc *desc, const void *logits, const void *index,
                                 const uint8_t *valid, int64_t *counts, float *loss, float *state, void *workspace,
                                 size_t workspace_bytes, apml_stream stream)
{
    clear_error();
    if (const apml_status st = check_balance(desc))
        return st;
    if (!logits || !counts || !loss || !workspace)
        return bad("logits, counts, loss and workspace must be non-NULL device pointers");
    if (!aligned(logits, elem_size((ElemType)desc->dtype)) || !aligned(index, desc->index_type == APML_I32 ? 4 : 8))
        return bad("logits and index must be aligned to their elements");
    if (!aligned(counts, 8) || !aligned(loss, 4) || !aligned(state, 4))
        return bad("counts, loss and state must be aligned to their elements");
    if (!aligned(workspace, 256))
        return bad("workspace must be aligned to 256 bytes");
    const BalanceProblem p = problem_of(*desc, logits, index, valid);
    const BalancePlan plan = balance_plan(p);
    if (workspace_bytes < plan.bytes)
        return short_workspace("apml_balance_forward", plan.bytes, workspace_bytes);
    balance_forward(p, plan, (uint8_t *)workspace, counts, loss, state, (hipStream_t)stream);
    return launched();
}

apml_status apml_balance_backward(const apml_balance_desc *desc, const void *logits, const uint8_t *valid,
                                  const float *state, const float *grad_loss, void *grad_logits, apml_stream stream)
{
    clear_error();
    if (const apml_status st = check_balance(desc))
        return st;
    if (!logits || !state || !grad_loss || !grad_logits)
        return bad("logits, state, grad_loss and grad_logits must be non-NULL device pointers");
    const size_t size = elem_size((ElemType)desc->dtype);
    if (!aligned(logits, size) || !aligned(grad_logits, size) || !aligned(state, 4) || !aligned(grad_loss, 4))
        return bad("logits, grad_logits, state and grad_loss must be aligned to their elements");
    balance_backward(problem_of(*desc, logits, nullptr, valid), state, grad_loss, grad_logits, (hipStream_t)stream);
    return launched();
}

apml_status apml_expert_counts(const void *index, int32_t index_type, const uint8_t *valid, int32_t samples,
                               int32_t tokens, int32_t chosen, int32_t experts, int64_t *counts, apml_stream stream)
{
    clear_error();
    apml_balance_desc d;
    apml_balance_desc_default(&d);
    d.index_type = index_type;
    d.samples = samples;
    d.tokens = tokens;
    d.chosen = chosen;
    d.experts = experts;
    if (const apml_status st = check_balance(&d))
        return st;
    if (!index || !counts)
        return bad("index and counts must be non-NULL device pointers");
    if (!aligned(index, index_type == APML_I32 ? 4 : 8) || !aligned(counts, 8))
        return bad("index and counts must be aligned to their elements");
    expert_counts(problem_of(d, nullptr, index, valid), counts, (hipStream_t)stream);
    return launched();
}

} // extern "C"

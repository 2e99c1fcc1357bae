// The balance loss of routed experts and the tokens per expert: what the host
// side (losses_api.hip) and the kernels (balance.hip) share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "linear_ce.h"

namespace apml {

constexpr int kMaxExperts = 1024;

struct BalanceProblem {
    ElemType type;
    bool index32;                          // expert indices are int32 (else int64)
    int samples, tokens, experts, chosen;  // per sample
    int reduction;                         // 0 none, 1 sum, 2 mean
    float z_weight;
    const void *logits;                    // [samples][tokens][experts]
    const void *index;                     // [samples][tokens][chosen], or NULL
    const uint8_t *valid;                  // [samples][tokens], or NULL: all
};

struct BalancePlan {
    int chunks, tokens; // chunks of tokens a sample, tokens of a chunk
    size_t p, count, z, loss, ticket, bytes;
};
BalancePlan balance_plan(const BalanceProblem &p);
// state: [samples][experts + 1] floats (E (f_e - min f), then 1 / valid tokens), or NULL.
// counts: written where index is given, else read.
void balance_forward(const BalanceProblem &p, const BalancePlan &plan, uint8_t *ws, int64_t *counts, float *loss,
                     float *state, hipStream_t s);
void balance_backward(const BalanceProblem &p, const float *state, const float *grad_loss, void *grad, hipStream_t s);
void expert_counts(const BalanceProblem &p, int64_t *counts, hipStream_t s);

} // namespace apml

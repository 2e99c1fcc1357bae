// Softmax cross entropy of rows x against classes w: what its host side
// (losses_api.hip) and its kernels (linear_ce.hip) share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace apml {

// The element types of features, logits and their gradients (apml_dtype).
enum class ElemType : int { f32 = 0, bf16 = 1, f16 = 2 };
inline size_t elem_size(ElemType t) { return t == ElemType::f32 ? 4 : 2; }

constexpr int kCeStep = 64; // elements of the summed axis that one step of a product takes
constexpr float kLog2E = 1.44269504088896340736f;

// What the forward pass keeps of a row: its largest logit in units of log 2,
// 1 / sum exp(z - top), the part of its softmax that is not the target's, and its
// log-sum-exp. The loss and the target's gradient come from `miss`, a sum without
// the target's term: where the target's probability is next to 1, lse - z_target
// and p - 1 would be differences of nearly equal numbers.
struct CeRow {
    float top, inv_total, miss, lse;
};

struct CeProblem {
    ElemType type;
    bool target32;                   // targets are int32 (else int64)
    int samples, rows, classes, dim; // `samples` problems, each with its own x, w and targets
    float scale, z_weight;
    int64_t ignore_index;
    int reduction;                   // 0 none, 1 sum, 2 mean
    const void *x, *w, *target;
};

// Byte offsets of the temporaries in the workspace, from the sizes and the
// pointers' alignment alone.
struct CeForwardPlan {
    bool pack_x, pack_w;         // copied: rows of dim_pad elements, in planes for float32
    bool whole_f32;              // float32 multiplied as it is
    int dim_pad;                 // dim up to a multiple of kCeStep
    int parts;                   // groups of classes with a maximum and a sum of their own
    size_t x, w, part, picked, sums, ticket, bytes;
};
CeForwardPlan ce_plan_forward(const CeProblem &p);
// Whether every launch of the two passes has fewer than 2^32 threads, which is
// what a dispatch counts them in.
bool ce_launches_fit(const CeProblem &p);
// loss: [samples * rows] (reduction none) or [1]; rows: the state or NULL;
// total: two floats (sum of the losses, rows that count) or NULL.
void ce_forward(const CeProblem &p, const CeForwardPlan &plan, uint8_t *ws, float *loss, CeRow *rows, float *total,
                hipStream_t s);

struct CeBackwardPlan {
    bool pack_x, pack_w;
    int dim_pad, rows_pad;       // rows up to a multiple of kCeStep
    int piece_samples, piece_rows, piece_classes; // the part of the logits' gradient that exists at a time
    int g_rows;                  // piece_rows up to a multiple of kCeStep
    int ld_g;                    // elements of a row of it, a multiple of kCeStep
    int split_x, split_w;        // parts of the sum over the classes (grad_x) and over the rows (grad_w)
    bool whole_g;                // it holds float32 values as they are, else planes or 16-bit values
    bool sum_x, sum_w;           // the gradient is summed in float32 over several pieces or parts
    int tops;                    // workgroups of the pass over the upstream gradients (0: all rows have the same)
    int size_lanes;              // lanes a row with which that pass reads x as well (0: it does not)
    size_t x, w, coef, block_top, top, xs, g, part_x, part_w, bytes;
};
CeBackwardPlan ce_plan_backward(const CeProblem &p, bool want_x, bool want_w);
void ce_backward(const CeProblem &p, const CeBackwardPlan &plan, uint8_t *ws, const CeRow *rows, const float *total,
                 const float *grad_loss, void *grad_x, void *grad_w, hipStream_t s);

} // namespace apml

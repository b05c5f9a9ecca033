// Softmax cross entropy of small problems without packing (xent_direct.hip).
#pragma once

#include "rfsf_internal.h"

namespace rfsf {

struct DirectGradient {
    void *out;                  // null: not asked for
    int64_t ld;
    float *parts;               // [cuts][rows][K] of a sum in several parts
    int64_t per_cut;            // summed indices of a part (of up to 16 rows or classes: rows of the many for a workgroup, in both)
    uint32_t cuts;
};
struct XentDirect {
    const void *Phi, *W;
    const int64_t *labels;
    const float *weight;        // null: the mean
    float *loss;
    int64_t N, K, C, ld_phi, ld_w;
    int32_t gradients;
    bool one_pass;              // all in one launch, the sum over the parts of dW left out
    bool fused;                 // scores and softmax in one launch. Otherwise:
    float *scores;              // [column_cuts][N][ld_scores]
    int64_t ld_scores, columns_per_cut;
    uint32_t column_cuts;
    float2 *partial;            // maximum and sum of exponentials of every 16 classes, [..][N]; null: few classes
    float *G;                   // G without the mean's scale: [N][ld_g], in the scores' place, or by_class [C][ld_g]
    int64_t ld_g;               // (a multiple of four)
    bool by_class;              // there are at most 16 rows, and fewer than classes
    uint32_t *counts;           // rows that count, of every 16, or in count_tiles numbers altogether
    int32_t count_tiles;
    bool count_here;            // one_pass_kernel: counts all rows before it starts
    DirectGradient dphi, dw;
    unsigned blocks_phi;        // workgroups of dPhi, those of dW follow
};

bool xent_direct(const rfsf_xent_shape &shape);                 // this way is taken: a function of the shape alone
size_t xent_direct_bytes(const rfsf_xent_shape &shape);
hipError_t launch_xent_direct(const rfsf_xent_shape &shape, const void *Phi, const void *W, const int64_t *labels, const float *weight, float *loss,
                              void *dPhi, void *dW, void *workspace, hipStream_t stream);

}  // namespace rfsf

// What the entry points (api_block.hip) ask of the residual block's kernels: plans (host only) and launches.
#pragma once
#include "dropout.h"
#include "train_ends.h"

namespace cac {

// ---- dropout.hip
struct DropGeom {
    long rows, cols, ld_x, ld_r; // ld: elements
    int dtype;
    float alpha;
};
hipError_t launch_dropout(const DropGeom &g, const Drop &d, const void *X, const void *R, void *Y, hipStream_t st);

// ---- block_norm.hip
struct NormGeom {
    long T, D, ld_f, ld_r;
    int dtype, post, pre; // cac_norm
    long gate_rows;       // rows that share one of the gate's; 0: no gate
    float eps_post, eps_pre, alpha;
};
struct NormSplit { // which rows a workgroup has
    bool own_groups;                      // backward: a slot has groups of the gate to itself
    long per_group;                       // backward: workgroups that share a group
    long blocks, rows_per_block;
};
struct NormPlan {
    int lanes, waves, chunks;             // to a row; groups of eight to a lane
    int slots;                            // rows that a workgroup has in hand at once
    long groups;                          // of rows with one gate (1 where there is none)
    NormSplit split, sums;                // sums: of the backward pass' sums over rows
    bool two;                             // ... which have a launch of their own
    size_t o_known, bytes;
};
struct NormParams { const float *gate, *w_post, *b_post, *w_pre, *b_pre; };
struct NormGrads { float *gate, *w_post, *b_post, *w_pre, *b_pre; };
void plan_norm(const NormGeom &g, bool backward, NormPlan *p);
hipError_t launch_norm_fwd(const NormGeom &g, const NormPlan &p, const Drop &d, const void *F, const void *R, const NormParams &w, void *S, void *H,
                           hipStream_t st);
hipError_t launch_norm_bwd(const NormGeom &g, const NormPlan &p, const Drop &d, const void *F, const void *S, const NormParams &w, const void *dH,
                           const void *dS, void *dR, void *dF, const NormGrads &o, void *ws, hipStream_t st);

// ---- linear.hip
struct LinearGeom {
    long T, D, N, ld_x, ld_w, ld_r; // ld: elements
    int dtype, act;                 // cac_act
    bool bias;
    float alpha;
    bool drops;
};
struct LinearPlan {
    bool few;                // few rows: W is read as it lies, by workgroups that have all rows of some features
    bool pack_x, pack_w;     // rows that are not whole numbers of 16 bytes go through the workspace
    bool again;              // backward: the pre-activation is formed again
    bool grad;               // backward: the pre-activation's gradient is a matrix of its own (else it is dY)
    long ld_x, ld_w, ld_u;   // elements from a row of the operands, as they are multiplied, to the next
    TileChoice y, dx, dw;
    bool together;           // backward: dX, dW and db in one launch, where both are asked for
    long parts;              // of the rows, that db is summed in (0: in one)
    size_t o_x, o_w, o_u, o_db, o_sum, o_sum2, bytes;
};
bool plan_linear(const LinearGeom &g, bool backward, LinearPlan *p); // false: a product too large for one grid
hipError_t launch_linear_fwd(const LinearGeom &g, const LinearPlan &p, const Drop &d, const void *X, const void *W, const void *b, const void *R,
                             void *Y, void *ws, hipStream_t st);
hipError_t launch_linear_bwd(const LinearGeom &g, const LinearPlan &p, const Drop &d, const void *X, const void *W, const void *b, const void *dY,
                             void *dX, void *dW, void *db, void *ws, hipStream_t st);

} // namespace cac

// What the entry points (api_train.hip) ask of the loss' and the update's kernels: plans (host only) and launches.
#pragma once
#include "common.h"

namespace cac {

struct TileChoice { int shape, slices; }; // of a product (mm_core.h)

// ---- loss.hip: softmax cross entropy of a linear classifier
struct LossGeom {
    long T, D, V;
    long ld_h, ld_w; // elements
    int dtype;
    bool bias;
    long ignore;
};
struct LossPlan {
    bool few;         // few rows, short forward passes: row m of the products is row m of H, zeros where it does not count
    bool direct;      // ... and all is read where it lies
    bool odd;         // ... which does not all start on 16 bytes
    bool split, raw;  // float: operands as two halves, or (few rows) as they lie
    bool rests;       // G's rounding errors are kept as rows of their own
    bool pack_w;      // the weights go through the workspace, piece by piece
    bool pair;        // backward: dW, dH and db in one launch
    long dp;          // features, in whole chunks of 8
    long row_bytes;   // of a packed row
    long piece;       // classes in one piece
    int pieces;
    TileChoice z, w, h; // the logits' product, dW's, dH's
    long parts;       // forward: maximum and sum, this many for every row
    size_t o_meta, o_h, o_w, o_part, o_z, o_g, o_peak, o_again, o_acc, bytes;
};
void plan_loss(const LossGeom &g, bool backward, LossPlan *p);
hipError_t launch_loss_fwd(const LossGeom &g, const LossPlan &p, const void *H, const void *W, const void *b, const int64_t *labels,
                           float *loss, float *lse, void *ws, hipStream_t st);
hipError_t launch_loss_bwd(const LossGeom &g, const LossPlan &p, const void *H, const void *W, const void *b, const int64_t *labels,
                           const float *lse, const float *gloss, void *dH, void *dW, void *db, void *ws, hipStream_t st);

// ---- muon.hip: Newton-Schulz products and the update made of them
struct MuonGeom {
    long rows, cols;
    int batch, steps, dtype, grad_dtype;
    bool nesterov;
};
struct MuonNarrowPlan { // muon_narrow.hip: a shorter side of at most 64
    int width, slices;  // columns to a workgroup, workgroups to a matrix
    size_t o_x, o_part, o_exps, bytes;
};
bool plan_muon_narrow(const MuonGeom &g, MuonNarrowPlan *p);
hipError_t launch_muon_narrow(const MuonGeom &g, const MuonNarrowPlan &p, const void *G, float *M, void *W, void *O, float momentum, float keep,
                              float lr, void *ws, hipStream_t st);
struct MuonPlan {
    bool narrow;
    MuonNarrowPlan np;
    bool tall;          // more rows than columns: X^T X in the place of X X^T
    long r;             // the shorter side
    long ld_x, ld_a;    // bytes of a row
    TileChoice gram, poly, apply;
    bool fits;          // every launch's grid is one that there is
    int sum_blocks;     // partial sums of squares of one matrix
    size_t o_sum, o_lift, o_x[2], o_a, o_b, o_part, bytes;
};
void plan_muon(const MuonGeom &g, MuonPlan *p);
// M, W: null where only O is asked for; O: null where the weights are updated
hipError_t launch_muon(const MuonGeom &g, const MuonPlan &p, const void *G, float *M, void *W, void *O, float momentum, float keep,
                       float lr, void *ws, hipStream_t st);

} // namespace cac

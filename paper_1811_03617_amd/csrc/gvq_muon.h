// Newton-Schulz orthogonalisation and the Muon step: launchers (host side).
#pragma once
#include "gvq_internal.h"
#include "gvq_muon_plan.h"

struct MuonMatrix {
    int64_t batch, rows, cols;
};

struct MuonPlan {   // where things lie in a workspace, in bytes
    int64_t m, n;                 // shorter and longer side: X is kept as m rows of n numbers
    int64_t ldn, ldm;             // padded row lengths in numbers
    int64_t x[2], gram, poly;     // of one matrix: two planes each
    int64_t per;                  // bytes of one matrix's planes
    int64_t sums, parts_at;       // partial sums of squares; partial products
    int64_t factors;              // of every step, GVQ_MAX_STEPS a matrix
    int64_t bytes;                // of the whole workspace
    int parts;                    // partial sums of squares of a matrix
    NsChoice gram_by, poly_by, step_by;
};
// false: the sizes are out of range.
bool gvq_muon_plan(const MuonMatrix& x, MuonPlan* p);

struct MuonArgs {
    MuonMatrix x;
    const void* grad;
    gvq_dtype_t grad_dtype;
    int64_t ld_grad, stride_grad;    // elements
    float* momentum;                 // null: orthogonalise the gradient itself
    int64_t ld_momentum;
    float beta;
    int nesterov;
    const double* coef;              // host [steps][3], null: the default
    int steps;
    double eps;
    void* out;                       // the result, or the weight that it updates
    gvq_dtype_t out_dtype;
    int64_t ld_out, stride_out;
    int update;                      // 0: out = X, 1: out = keep * out - rate * X
    float keep, rate;
    char* workspace;
};
int gvq_launch_muon(const MuonArgs& a, hipStream_t st);

// The gradient and momentum as kernels see them.
struct MuonPrep {
    const void* grad;
    int64_t ld_grad, stride_grad;
    float* momentum;
    int64_t ld_momentum;
    float beta;
    int nesterov;
    int64_t rows, cols;
    int parts;           // partial sums of squares of a matrix
    double eps;
    int turn;            // more rows than columns: X is the transpose
};
MuonPrep gvq_muon_prep(const MuonArgs& a);
// The coefficients, and the steps' factors of a matrix whose norm is far above eps.
struct MuonCoef {
    float v[GVQ_MAX_STEPS][3];
    NsFactors whole[GVQ_MAX_STEPS];
    int steps;
};
MuonCoef gvq_muon_coef(const MuonArgs& a);
int gvq_muon_parts(const MuonMatrix& x);
// M <- beta M + G and the sums of squares of U, `p.parts` per matrix.
int gvq_launch_muon_norm(const MuonArgs& a, const MuonPrep& p, double* sums, hipStream_t st);

// Matrices with at most 64 rows or columns (gvq_muon_small.hip).
struct MuonSmallPlan {
    int64_t m, n, ldn, run, groups, per, x, grams[2], sums, factors, bytes;
    int parts;
    bool one;            // in one work-group, which does not look at its workspace (256 bytes all the same)
};
bool gvq_muon_small_takes(const MuonMatrix& x);
int64_t gvq_muon_small_plan(const MuonMatrix& x, MuonSmallPlan* p);   // bytes of the workspace
int gvq_launch_muon_small(const MuonArgs& a, hipStream_t st);

// A teacher's top logits against a student's softmax: arguments and the launcher's declaration.
#pragma once
#include "gvq_device.h"

struct DistillArgs {
    const void* logits;       // [rows][vocab]
    int64_t rows, ld;
    int vocab;
    const void* top;          // [rows][n_top]
    int top_bf16;
    int64_t ld_top;
    const int64_t* index;     // [rows][n_top]; outside [0, vocab): the entry is absent
    int64_t ld_index;
    int n_top;
    const float* weight;      // [rows] or null: ones
    double t64;               // temperature t,
    float t, per_t, log2_t;   // t, 1 / t, log2(e) / t
    float* loss;              // [rows]
    void* grad;               // [rows][vocab] or null
    int64_t ld_grad;
};

// Pieces that a row is cut into: few rows of many logits.  workspace: two floats for each, or half as many pieces of two doubles.
int gvq_distill_parts(int64_t rows, int64_t vocab);
int gvq_launch_distill(const DistillArgs& a, gvq_dtype_t dtype, void* workspace, hipStream_t st);

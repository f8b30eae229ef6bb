// Softmax cross entropy of a few float32 rows (internal; xent_few.cu).
#pragma once

#include "head_gemm.h"

namespace pvs {
namespace head {

constexpr int kFewRows = 16;      // at most
constexpr int kFewDim = 1024;     // the widest row

struct FewArgs {
    const float* x;               // [rows, dim], rows <= kFewRows
    int64_t ldx;
    int rows;
    const float* w;               // [items, dim], of the whole vocabulary from item0 on
    int64_t ldw, items, item0;
    int dim;
    float k2;                     // scale log2(e)
    const float* bias;            // of the same items, or null
    const int64_t* targets;       // forward: left out of their rows' statistics (null: none)
    int64_t ignore_index;
    // the forward pass: a block's (m, s) of row t at part[block * part_rows + t]
    float2* part;
    int64_t part_rows;
    // the backward pass
    const GradRow* row;
    const float4* stats;          // of the forward pass, for rows without targets
    float* g;                     // [items][few_rows_padded(rows)]
    float* slots;                 // sums of dx, [block][rows, ldslot], or null
    int64_t slot_stride, ldslot;
    bool accumulate;              // added to what slots hold
    float* dw;                    // or null
    int64_t lddw;
    float scale;
};

// Blocks of a launch, each of which leaves its share of the sums.
int few_blocks(int64_t items, const Device& dev);
// The rows that a launch works on.
int few_rows_padded(int64_t rows);
cudaError_t launch_few_stats(const FewArgs& a, int blocks, cudaStream_t st);
// The backward pass in two launches: G, then the gradients from it.
cudaError_t launch_few_softmax(const FewArgs& a, int blocks, cudaStream_t st);
cudaError_t launch_few_columns(const FewArgs& a, int blocks, cudaStream_t st);

}  // namespace head
}  // namespace pvs

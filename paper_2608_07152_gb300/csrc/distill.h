// What distillation adds to the softmax cross entropy (internal; distill.cu).
#pragma once

#include "../../include/head.h"
#include "head_gemm.h"

namespace pvs {
namespace head {

constexpr int kMaxTop = 1024;            // items to a list
// What the forward pass keeps of a slot that is not in its row's list.
constexpr float kNoHit = 2.0f;

// A block of rows of a call.
struct TopRows {
    pvs_xent_args a;                     // the block's
    const int64_t* ids;                  // [rows][top]
    const void* logits;                  // [rows][top] of `dtype`
    int top, dtype;
    float teacher_scale;
};

// Each row's items in ascending order, INT_MAX for what is none, the slots that they were in,
// and where each tile of items begins among them (tiles 0: nowhere).
struct TopLists {
    TopRows r;
    int* list;                           // [rows][top]
    uint16_t* slot;                      // [rows][top]
    uint16_t* first;                     // [tiles][rows]
    int tiles, piece_tiles;              // tile q starts at item q / piece_tiles * piece + ...
    int64_t piece;
    int tile;                            // ... q % piece_tiles * tile
};

// The student's logits of the listed items, in powers of two: float32 products.
struct TopDots {
    TopRows r;
    const int* list;
    float k2;
    bool wide;                           // 16-bit rows of whole, aligned eights
    float* dots;                         // [rows][top]
};
// Both, in one launch or two.
cudaError_t launch_top_lists(const TopLists& a, const TopDots& dots, cudaStream_t st);

// A row's loss and what the backward pass wants, from its tiles' statistics: of every item, or
// (apart) of those that are not listed.
struct TopJoin {
    TopRows r;
    const int* list;
    const uint16_t* slot;
    const float* dots;
    const float2* part;                  // [n][rows]
    int64_t n;
    bool apart;
    float* loss;
    float4* stats;
    float* hits;                         // [rows][top]
};
cudaError_t launch_top_join(const TopJoin& a, const Device& dev, cudaStream_t st);

// G of the listed items of a piece, over what the product wrote there.
struct TopScatter {
    const int64_t* ids;
    const float* hits;                   // [rows][top]
    const float* grad;                   // [rows]
    const float* up;                     // f16: the power of two of every gradient, or null
    int64_t rows, v0, n;
    int top;
    uint16_t* g;                         // [parts][rows][ldg], or null
    int64_t ldg, g_part;
    int parts, f16;
    float* few;                          // else [n][few_rows]
    int few_rows;
};
cudaError_t launch_top_scatter(const TopScatter& a, cudaStream_t st);

}  // namespace head
}  // namespace pvs

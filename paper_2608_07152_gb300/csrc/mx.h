// Microscaled 4-bit rows (internal; mx_pack.cu, mx_gemm.cu).
#pragma once

#include "head_gemm.h"

namespace pvs {
namespace head {

// Columns as they are kept: whole blocks of 128.
inline int mx_padded(int cols) { return (cols + 127) / 128 * 128; }

// Bytes of the scales of `rows` rows.
inline int64_t mx_scale_bytes(int64_t rows, int kp, int group) {
    return (rows + 127) / 128 * (kp / (4 * group)) * 512;
}

// Whether packed rows' pointers can be read.
inline bool mx_operand(const void* codes, const void* scales, const void* row_scales, int group) {
    return codes && scales && on_elements(codes, 16) && on_elements(scales, 16) &&
           (group == 32 || (row_scales && on_elements(row_scales, 4)));
}

cudaError_t launch_mx_pack(const void* x, int64_t ldx, int64_t rows, int cols, int dtype, int group,
                           uint8_t* codes, uint8_t* scales, float* row_scales, cudaStream_t st);

}  // namespace head
}  // namespace pvs

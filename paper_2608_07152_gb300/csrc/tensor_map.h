// TMA tensor maps, encoded by the driver on the host.
#pragma once

#include <cstdint>

#include <cuda.h>

namespace pvs {

// Row-major matrix of `elem`-byte elements, boxes of box_cols x box_rows, 128-byte
// swizzle, elements past the matrix read as zero; false when the driver refuses it.
bool tensor_map_2d(CUtensorMap* m, CUtensorMapDataType type, int elem, const void* base,
                   uint64_t rows, uint64_t cols, uint32_t box_cols, uint32_t box_rows);

// The same for `parts` matrices with leading dimension ld, part_stride elements
// apart, a box within one of them.
bool tensor_map_3d(CUtensorMap* m, CUtensorMapDataType type, int elem, const void* base,
                   uint64_t parts, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t part_stride,
                   uint32_t box_cols, uint32_t box_rows);

// Blocks of 512 bytes [rows][cols] without gaps, boxes of `box` neighbours in a row, no swizzle,
// blocks past the matrix read as zeros.
bool tensor_map_blocks(CUtensorMap* m, const void* base, uint64_t rows, uint64_t cols, uint32_t box);

}  // namespace pvs

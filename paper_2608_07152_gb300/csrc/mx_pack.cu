// Rows in microscaled 4-bit floating point (head.h): packing and unpacking.
//
// Bound by memory: a row is read once (groups of 16: its largest element first; up to 1,024
// elements of it stay in registers) and leaves half a byte an element and a byte a group.  A
// warp takes a row, a lane eight neighbours at a time, so that a group of 16 is two lanes and
// one of 32 four.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>

#include "../../include/head.h"
#include "kernels.h"
#include "mx.h"
#include "pvs_common.cuh"

namespace pvs {
namespace head {
namespace {

constexpr int kPackThreads = 256;
constexpr int kPackWarps = kPackThreads / 32;
constexpr int kHeld = 4;             // steps of 256 elements that stay in registers

__device__ __forceinline__ float mx_element(const void* p, int dtype, int64_t i) {
    if (dtype == PVS_F32) return static_cast<const float*>(p)[i];
    if (dtype == PVS_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

// Eight elements of a row from column c, zeros past it.
template <bool WIDE>
__device__ __forceinline__ void load_eight(const void* x, int dtype, int64_t row, int c, int cols,
                                           float (&v)[8]) {
    uint32_t u[4];
    if (WIDE && c + 8 <= cols && dtype == PVS_F32) {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(x) + row + c);
        const float4 a = __ldg(q), b = __ldg(q + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
        v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        return;
    }
    if (c + 8 > cols || dtype == PVS_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? mx_element(x, dtype, row + c + i) : 0.0f;
        return;
    }
    const uint16_t* p = static_cast<const uint16_t*>(x) + row + c;
    if (WIDE) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
        u[0] = a.x, u[1] = a.y, u[2] = a.z, u[3] = a.w;
    } else {
        load_eight_halves(p, u);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (dtype == PVS_BF16) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
}

// The largest magnitude's bits; an infinity's or more where one is not finite.
__device__ __forceinline__ uint32_t top_bits(const float (&v)[8]) {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(v[i]) & 0x7fffffffu);
    return t;
}

// Eight values in units of their scale to e2m1, ties to the even code, beyond 6 to 6.
__device__ __forceinline__ uint32_t e2m1_of(const float (&q)[8]) {
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    return r;
}

struct PackArgs {
    const void* x;
    int64_t ldx, rows, padded_rows;
    int cols, dtype, kp;
    uint8_t* codes;
    uint8_t* scales;
    float* row_scales;               // groups of 16
};

// The four bytes of a block's four groups of kLanes lanes, in the first of its lanes.
template <int kLanes>
__device__ __forceinline__ uint32_t four_of(uint32_t byte) {
    const int first = (threadIdx.x & 31) & ~(4 * kLanes - 1);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= __shfl_sync(0xffffffffu, byte, first + i * kLanes) << (8 * i);
    return w;
}

template <bool kSixteen, bool WIDE>
__global__ void __launch_bounds__(kPackThreads) mx_pack_kernel(const PackArgs a) {
    constexpr int kLanes = kSixteen ? 2 : 4;           // of a group
    next_early();
    wait_before();
    const int lane = threadIdx.x & 31;
    const int blocks = a.kp / (kLanes * 32);
    for (int64_t row = (int64_t)blockIdx.x * kPackWarps + (threadIdx.x >> 5); row < a.padded_rows;
         row += (int64_t)gridDim.x * kPackWarps) {
        uint8_t* to = a.scales + row / 128 * blocks * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4;
        if (row >= a.rows) {
            for (int b = lane; b < blocks; b += 32) *reinterpret_cast<uint32_t*>(to + (int64_t)b * 512) = 0;
            continue;
        }
        const int64_t at = row * a.ldx;
        float v[kHeld][8];
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            load_eight<WIDE>(a.x, a.dtype, at, 256 * i + 8 * lane, a.cols, v[i]);
        float row_up = 1.0f;                           // 1 / the row's scale
        bool bad_row = false;
        if (kSixteen) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < kHeld; ++i) top = max(top, top_bits(v[i]));
            for (int c = 256 * kHeld; c < a.cols; c += 256) {
                float w[8];
                load_eight<WIDE>(a.x, a.dtype, at, c + 8 * lane, a.cols, w);
                top = max(top, top_bits(w));
            }
            top = __reduce_max_sync(0xffffffffu, top);
            bad_row = top >= 0x7f800000u;
            // 2^(floor(log2 top) - 10): the scales of groups then reach 171 to 352 of 448
            const int e = top == 0 ? 127 : max((int)(top >> 23) - 10, 1);
            row_up = __uint_as_float((uint32_t)(254 - e) << 23);
            if (lane == 0)
                a.row_scales[row] = bad_row ? __int_as_float(0x7fffffff) : __uint_as_float((uint32_t)e << 23);
        }
#pragma unroll 1
        for (int c = 0; c < a.kp; c += 256) {
            float w[8];
            if (c < 256 * kHeld) {
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (c == 256 * i) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k] = v[i][k];
                    }
            } else {
                load_eight<WIDE>(a.x, a.dtype, at, c + 8 * lane, a.cols, w);
            }
            uint32_t top = top_bits(w);
#pragma unroll
            for (int o = 1; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            uint32_t byte, word;
            if (!kSixteen) {
                // 2^(floor(log2 top) - 2), its exponent with bias 127: multiplying is exact
                byte = (uint32_t)max((int)(top >> 23) - 2, 0);
                const float up = __uint_as_float((254u - byte) << 23);
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] *= up;
                word = e2m1_of(w);
                if (top >= 0x7f800000u) byte = 255, word = 0;
            } else {
                const __nv_fp8_storage_t s8 =
                    __nv_cvt_float_to_fp8(__uint_as_float(top) * (1.0f / 6.0f) * row_up, __NV_SATFINITE, __NV_E4M3);
                byte = s8;
                const float s = __half2float(__half(__nv_cvt_fp8_to_halfraw(s8, __NV_E4M3)));
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float x = w[k] * row_up;     // (exact but for what is far below a code)
                    float q = x / s;
                    // a quotient that was rounded to a border between codes (three bits, zeros
                    // behind them) goes a last bit towards what the division left over
                    const float left = fmaf(-q, s, x);
                    const uint32_t u = __float_as_uint(q);
                    if (left != 0.0f && q != 0.0f && (u & 0x1fffffu) == 0)
                        q = __uint_as_float((left > 0.0f) == (q > 0.0f) ? u + 1u : u - 1u);
                    w[k] = q;
                }
                word = e2m1_of(w);
                if (bad_row || byte == 0) word = 0;
                if (bad_row) byte = 0;
            }
            if (c + 8 * lane < a.kp)
                *reinterpret_cast<uint32_t*>(a.codes + row * (a.kp / 2) + (c + 8 * lane) / 2) = word;
            const uint32_t four = four_of<kLanes>(byte);
            const int b = (c + 8 * lane) / (32 * kLanes);
            if ((lane & (4 * kLanes - 1)) == 0 && b < blocks)
                *reinterpret_cast<uint32_t*>(to + (int64_t)b * 512) = four;
        }
    }
}

// What codes stand for, eight a thread.
template <bool kSixteen, bool WIDE>
__global__ void __launch_bounds__(kPackThreads) mx_unpack_kernel(const uint8_t* __restrict__ codes,
                                                                 const uint8_t* __restrict__ scales,
                                                                 const float* __restrict__ row_scales,
                                                                 int64_t rows, int cols, int kp, void* out,
                                                                 int64_t ldout, int dtype) {
    next_early();
    wait_before();
    constexpr int kGroup = kSixteen ? 16 : 32;
    const int pieces = (cols + 7) / 8, blocks = kp / (4 * kGroup);
    const int64_t total = rows * pieces, step = (int64_t)gridDim.x * kPackThreads;
    for (int64_t i = (int64_t)blockIdx.x * kPackThreads + threadIdx.x; i < total; i += step) {
        const int64_t row = i / pieces;
        const int c = (int)(i - row * pieces) * 8;
        const uint32_t word = __ldg(reinterpret_cast<const uint32_t*>(codes + row * (kp / 2) + c / 2));
        const uint8_t byte = __ldg(scales + (row / 128 * blocks + c / (4 * kGroup)) * 512 + (row & 31) * 16 +
                                   ((row >> 5) & 3) * 4 + c / kGroup % 4);
        float unit;
        if (kSixteen)
            unit = __half2float(__half(__nv_cvt_fp8_to_halfraw(byte, __NV_E4M3))) * __ldg(row_scales + row);
        else
            unit = byte == 255 ? __int_as_float(0x7fffffff)
                   : byte == 0 ? 0x1p-127f : __uint_as_float((uint32_t)byte << 23);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t n = word >> (4 * k) & 15u;
            // 0, 1/2, 1, 3/2, 2, 3, 4, 6
            const uint32_t e = n >> 1 & 3u, m = n & 1u;
            const float f = e == 0 ? 0.5f * (float)m : __uint_as_float((126u + e) << 23 | m << 22);
            v[k] = (n & 8u ? -f : f) * unit;
        }
        const int64_t at = row * ldout + c;
        if (dtype == PVS_F32) {
            float* o = static_cast<float*>(out) + at;
            if (WIDE && c + 8 <= cols) {
                *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < cols) o[k] = v[k];
            }
        } else {
            uint16_t h[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                h[k] = dtype == PVS_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v[k]))
                                         : __half_as_ushort(__float2half_rn(v[k]));
            uint16_t* o = static_cast<uint16_t*>(out) + at;
            if (WIDE && c + 8 <= cols) {
                *reinterpret_cast<uint4*>(o) =
                    make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16,
                               h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < cols) o[k] = h[k];
            }
        }
    }
}

bool mx_wide(const void* p, int64_t ld, int dtype) {
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % (dtype == PVS_F32 ? 4 : 8) == 0;
}
bool mx_shape(int64_t rows, int32_t cols, int32_t group, int32_t dtype) {
    return rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= 32767 && (group == 16 || group == 32) &&
           dtype >= PVS_BF16 && dtype <= PVS_F32;
}
pvs_status mx_queued(cudaError_t e) {
    if (e == cudaSuccess) return PVS_OK;
    cudaGetLastError();
    return PVS_ERR_CUDA;
}

}  // namespace

cudaError_t launch_mx_pack(const void* x, int64_t ldx, int64_t rows, int cols, int dtype, int group,
                           uint8_t* codes, uint8_t* scales, float* row_scales, cudaStream_t st) {
    const PackArgs a{x, ldx, rows, round_up(rows, 128), cols, dtype, mx_padded(cols), codes, scales, row_scales};
    const int64_t grid = std::min<int64_t>((a.padded_rows + kPackWarps - 1) / kPackWarps, 1 << 20);
    const bool w = mx_wide(x, ldx, dtype);
    count_launches(1);
    return launch_early(group == 16 ? (w ? mx_pack_kernel<true, true> : mx_pack_kernel<true, false>)
                                    : (w ? mx_pack_kernel<false, true> : mx_pack_kernel<false, false>),
                        grid, kPackThreads, 0, st, a);
}

}  // namespace head
}  // namespace pvs

using namespace pvs;
using namespace pvs::head;

extern "C" pvs_status pvs_mx_pack(const void* x, int64_t ldx, int64_t rows, int32_t cols, int32_t dtype,
                                  int32_t group, uint8_t* codes, uint8_t* scales, float* row_scales,
                                  void* cuda_stream) {
    if (!mx_shape(rows, cols, group, dtype) || ldx < cols) return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!x || !on_elements(x, element_bytes(dtype)) || !mx_operand(codes, scales, row_scales, group))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    return mx_queued(launch_mx_pack(x, ldx, rows, cols, dtype, group, codes, scales, row_scales,
                                    static_cast<cudaStream_t>(cuda_stream)));
}

extern "C" pvs_status pvs_mx_unpack(const uint8_t* codes, const uint8_t* scales, const float* row_scales,
                                    int64_t rows, int32_t cols, int32_t group, void* out, int64_t ldout,
                                    int32_t dtype, void* cuda_stream) {
    if (!mx_shape(rows, cols, group, dtype) || ldout < cols) return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!out || !on_elements(out, element_bytes(dtype)) || !mx_operand(codes, scales, row_scales, group))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    const int64_t pieces = rows * ((cols + 7) / 8);
    const int64_t grid = std::min<int64_t>((pieces + kPackThreads - 1) / kPackThreads, 1 << 20);
    const bool w = mx_wide(out, ldout, dtype);
    count_launches(1);
    return mx_queued(launch_early(
        group == 16 ? (w ? mx_unpack_kernel<true, true> : mx_unpack_kernel<true, false>)
                    : (w ? mx_unpack_kernel<false, true> : mx_unpack_kernel<false, false>),
        grid, kPackThreads, 0, static_cast<cudaStream_t>(cuda_stream), codes, scales, row_scales, rows, cols,
        mx_padded(cols), out, ldout, dtype));
}

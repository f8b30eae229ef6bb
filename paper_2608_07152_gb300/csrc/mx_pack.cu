// Rows in microscaled 4-bit floating point (head.h): packing and unpacking.
//
// A row is read once (groups of 16: its largest element first; up to 4,096 elements of it stay in
// the registers of one to four warps) and leaves half a byte an element and a byte a group.  A lane
// takes eight neighbours, so that a group of 16 is two lanes and one of 32 four.
//
// 200,000 rows of 1,000 in f16, groups of 32: 76 us (6.6 TB/s; issue 80%), in bf16 and groups of 16 94
// (5.3: issue bounds it, in float32 150, 6.0); to float32 again 137 (6.6 TB/s).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include <algorithm>

#include "../../include/head.h"
#include "f32x2.cuh"
#include "kernels.h"
#include "mx.h"
#include "pvs_common.cuh"

namespace pvs {
namespace head {
namespace {

constexpr int kPackThreads = 256;
constexpr int kPackWarps = kPackThreads / 32;
constexpr int kHeld = 4;             // steps of 256 elements that stay in registers

// Eight neighbours of a row as they lie: four words of 16-bit elements, or eight float32.
template <int DT>
struct Eight {
    uint32_t u[DT == PVS_F32 ? 8 : 4];

    // From column c of the row at element `row`, zeros past it.
    template <bool WIDE>
    __device__ __forceinline__ void load(const void* x, int64_t row, int c, int cols) {
        if constexpr (DT == PVS_F32) {
            const float* p = static_cast<const float*>(x) + row + c;
            if (WIDE && c + 8 <= cols) {
                const uint4* q = reinterpret_cast<const uint4*>(p);
                const uint4 f = __ldg(q), g = __ldg(q + 1);
                u[0] = f.x, u[1] = f.y, u[2] = f.z, u[3] = f.w;
                u[4] = g.x, u[5] = g.y, u[6] = g.z, u[7] = g.w;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = c + i < cols ? __float_as_uint(__ldg(p + i)) : 0u;
            }
        } else {
            const uint16_t* p = static_cast<const uint16_t*>(x) + row + c;
            if (c + 8 > cols) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    u[i] = (c + 2 * i < cols ? (uint32_t)__ldg(p + 2 * i) : 0u) |
                           (c + 2 * i + 1 < cols ? (uint32_t)__ldg(p + 2 * i + 1) : 0u) << 16;
            } else if (WIDE) {
                const uint4 f = __ldg(reinterpret_cast<const uint4*>(p));
                u[0] = f.x, u[1] = f.y, u[2] = f.z, u[3] = f.w;
            } else {
                load_eight_halves(p, u);
            }
        }
    }
    // The largest magnitude's bits as a float32; an infinity's or more where one is not finite.
    __device__ __forceinline__ uint32_t top() const {
        if constexpr (DT == PVS_F32) {
            uint32_t t = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) t = max(t, u[i] & 0x7fffffffu);
            return t;
        } else {
            const uint32_t m = 0x7fff7fffu;
            const uint32_t t = __vmaxu2(__vmaxu2(u[0] & m, u[1] & m), __vmaxu2(u[2] & m, u[3] & m));
            const uint32_t h = max(t >> 16, t & 0xffffu);
            if (DT == PVS_BF16) return h << 16;
            return __float_as_uint(__half2float(__ushort_as_half((uint16_t)h)));
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == PVS_F32) {
                v[2 * i] = __uint_as_float(u[2 * i]);
                v[2 * i + 1] = __uint_as_float(u[2 * i + 1]);
            } else if constexpr (DT == PVS_BF16) {
                v[2 * i] = __uint_as_float(u[i] << 16);
                v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
                v[2 * i] = f.x;
                v[2 * i + 1] = f.y;
            }
        }
    }
};

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
    int cols, kp;
    uint8_t* codes;
    uint8_t* scales;
    float* row_scales;               // groups of 16
};

// The code of x / unit from q = x times about 1 / unit, off by 2^-22 of itself at most.  A border
// between codes (1/4 to 5) has three bits and its product with a unit seven.  An element of 16-bit
// type has 11 at most: x is a border's product, or an 11th bit of that product away from it,
// which is 2^-13 or more in q.  So q to a multiple of 2^-13 is the border, or on its side of it:
// one FMA and one addition, two elements an instruction.  A float32 may be nearer: there the
// border's product decides, exactly.
__device__ __forceinline__ void by_grid(float (&w)[8], float up) {
    constexpr float kGrid = 1536.0f;                   // 3/2 2^10: float32 steps of 2^-13 around it
    const uint64_t f = f2_pack(up, up), plus = f2_pack(kGrid, kGrid), minus = f2_pack(-kGrid, -kGrid);
#pragma unroll
    for (int k = 0; k < 8; k += 2)
        f2_unpack(f2_add(f2_fma(f2_pack(w[k], w[k + 1]), f, plus), minus), w[k], w[k + 1]);
}
__device__ __forceinline__ float beside_border(float q, float x, float unit) {
    const uint32_t u = (__float_as_uint(q) + 0x40u) & ~0x7fu;
    if ((u & 0x1fffffu) != 0) return q;
    const float left = fmaf(-__uint_as_float(u), unit, x);
    const bool more = (left > 0.0f) == (x > 0.0f);
    return __uint_as_float(left == 0.0f ? u : more ? u + 1u : u - 1u);
}
__device__ __forceinline__ float about_inverse(float s) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    return r;
}
__device__ __forceinline__ void times(float (&w)[8], float f) {
    const uint64_t ff = f2_pack(f, f);
#pragma unroll
    for (int k = 0; k < 8; k += 2) f2_unpack(f2_mul(f2_pack(w[k], w[k + 1]), ff), w[k], w[k + 1]);
}

// A row of groups of 16: its scale r and 1 / r.
struct RowScale {
    float r, up;
    bool bad;
};

// A lane's eight elements to `code`, and the scale of the group that they are in to `scale`.
template <bool kSixteen, int DT>
__device__ __forceinline__ void pack_eight(const Eight<DT>& in, bool here, uint32_t* code, uint8_t* scale,
                                           const RowScale& row) {
    constexpr int kLanes = kSixteen ? 2 : 4;           // of a group
    uint32_t top = in.top();
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    uint32_t byte, word;
    float w[8];
    in.values(w);
    if (!kSixteen) {
        // 2^(floor(log2 top) - 2), its exponent with bias 127: multiplying is exact
        byte = (uint32_t)max((int)(top >> 23) - 2, 0);
        times(w, __uint_as_float((254u - byte) << 23));
        word = e2m1_of(w);
        if (top >= 0x7f800000u) byte = 255, word = 0;
    } else {
        const __nv_fp8_storage_t s8 =
            __nv_cvt_float_to_fp8(__uint_as_float(top) * (1.0f / 6.0f) * row.up, __NV_SATFINITE, __NV_E4M3);
        byte = s8;
        const float s = __half2float(__half(__nv_cvt_fp8_to_halfraw(s8, __NV_E4M3)));
        float unit = s * row.r, up = about_inverse(s) * row.up;
        if (row.up > 0x1p100f) {
            // (a row so small that 1 / unit may be no float32)
            times(w, row.up);
            unit = s;
            up = about_inverse(s);
        }
        if (DT != PVS_F32) {
            by_grid(w, up);
            word = e2m1_of(w);
        } else {
            float q[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) q[k] = w[k];
            times(q, up);
#pragma unroll
            for (int k = 0; k < 8; ++k) q[k] = beside_border(q[k], w[k], unit);
            word = e2m1_of(q);
        }
        if (row.bad || byte == 0) word = 0;
        if (row.bad) byte = 0;
    }
    if (!here) return;
    *code = word;
    if ((threadIdx.x & (kLanes - 1)) == 0) *scale = (uint8_t)byte;
}

// Blocks to an SM, which set how many loads are in flight: 16,384 rows of 4,096 in bf16, in groups
// of 16, took 55 us with the registers that the compiler takes by itself, 36 with four blocks, 42
// with six; in groups of 32 30, 30 and 28; in float32 and groups of 16 72 with two, 51 with four.
constexpr int pack_blocks(bool sixteen, int dtype) { return dtype == PVS_F32 || sixteen ? 4 : 6; }

// A block takes kPackWarps / kWarps rows at a time, kWarps warps to a row, each 1,024 columns in
// registers (again from memory where a row is longer than all of them hold).
template <bool kSixteen, int DT, bool WIDE, int kWarps>
__global__ void __launch_bounds__(kPackThreads, pack_blocks(kSixteen, DT)) mx_pack_kernel(const PackArgs a) {
    constexpr int kRows = kPackWarps / kWarps, kCols = 256 * kHeld;
    __shared__ uint32_t tops[2][kPackWarps];
    [[maybe_unused]] int turn = 0;
    next_early();
    wait_before();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, in_row = warp % kWarps;
    const int blocks = a.kp / (kSixteen ? 64 : 128);
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.padded_rows; row0 += (int64_t)gridDim.x * kRows) {
        const int64_t row = row0 + warp / kWarps;
        const bool here = row < a.rows;
        uint8_t* to = a.scales + row / 128 * blocks * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4;
        // a lane's codes and scale of a step of 256 columns; a step on, 32 words and kStep bytes
        constexpr int kGroups = kSixteen ? 16 : 8, kStep = kGroups * 128, kLanes = 32 / kGroups;
        uint32_t* code = reinterpret_cast<uint32_t*>(a.codes + row * (a.kp / 2)) + lane;
        uint8_t* scale = to + lane / kLanes / 4 * 512 + lane / kLanes % 4;
        const int64_t at = row * a.ldx;
        Eight<DT> v[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            v[i].template load<WIDE>(a.x, at, in_row * kCols + 256 * i + 8 * lane, here ? a.cols : 0);
        RowScale rs{1.0f, 1.0f, false};
        if (kSixteen) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < kHeld; ++i) top = max(top, v[i].top());
            for (int c0 = (in_row + kWarps) * kCols; here && c0 < a.cols; c0 += kWarps * kCols) {
                for (int c = c0; c < min(c0 + kCols, a.cols); c += 256) {
                    Eight<DT> w;
                    w.template load<WIDE>(a.x, at, c + 8 * lane, a.cols);
                    top = max(top, w.top());
                }
            }
            top = __reduce_max_sync(0xffffffffu, top);
            if (kWarps > 1) {
                // (a barrier of the row's warps; the next row's tops go to the other half)
                uint32_t* t = tops[turn & 1] + warp / kWarps * kWarps;
                if (lane == 0) t[in_row] = top;
                asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / kWarps), "n"(kWarps * 32) : "memory");
#pragma unroll
                for (int i = 0; i < kWarps; ++i) top = max(top, t[i]);
                ++turn;
            }
            rs.bad = top >= 0x7f800000u;
            // 2^(floor(log2 top) - 10): the largest scale of its groups is 176 to 352, of 448
            const int e = top == 0 ? 127 : max((int)(top >> 23) - 10, 1);
            rs.r = __uint_as_float((uint32_t)e << 23);
            rs.up = __uint_as_float((uint32_t)(254 - e) << 23);
            if (lane == 0 && in_row == 0 && here)
                a.row_scales[row] = rs.bad ? __int_as_float(0x7fffffff) : rs.r;
        }
        if (!here) {
            if (row < a.padded_rows)
                for (int b = in_row * 32 + lane; b < blocks; b += kWarps * 32)
                    *reinterpret_cast<uint32_t*>(to + (int64_t)b * 512) = 0;
            continue;
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int n = in_row * kHeld + i;
            if (256 * n < a.kp)
                pack_eight<kSixteen, DT>(v[i], 256 * n + 8 * lane < a.kp, code + 32 * n, scale + kStep * n, rs);
        }
        for (int n0 = (in_row + kWarps) * kHeld; 256 * n0 < a.kp; n0 += kWarps * kHeld) {
            for (int n = n0; n < n0 + kHeld && 256 * n < a.kp; ++n) {
                Eight<DT> w;
                w.template load<WIDE>(a.x, at, 256 * n + 8 * lane, a.cols);
                pack_eight<kSixteen, DT>(w, 256 * n + 8 * lane < a.kp, code + 32 * n, scale + kStep * n, rs);
            }
        }
    }
}

using PackKernel = void (*)(const PackArgs);
template <bool kSixteen, int DT>
PackKernel pack_of(bool wide, int warps) {
    return warps == 1   ? (wide ? mx_pack_kernel<kSixteen, DT, true, 1> : mx_pack_kernel<kSixteen, DT, false, 1>)
           : warps == 2 ? (wide ? mx_pack_kernel<kSixteen, DT, true, 2> : mx_pack_kernel<kSixteen, DT, false, 2>)
                        : (wide ? mx_pack_kernel<kSixteen, DT, true, 4> : mx_pack_kernel<kSixteen, DT, false, 4>);
}
template <bool kSixteen>
PackKernel pack_of(int dtype, bool wide, int warps) {
    return dtype == PVS_F32   ? pack_of<kSixteen, PVS_F32>(wide, warps)
           : dtype == PVS_F16 ? pack_of<kSixteen, PVS_F16>(wide, warps)
                              : pack_of<kSixteen, PVS_BF16>(wide, warps);
}

// A code's value: 0, 1/2, 1, 3/2, 2, 3, 4, 6, and bit 3 the sign.
__device__ __forceinline__ float value_of(uint32_t n) {
    const uint32_t e = n >> 1 & 3u, m = n & 1u;
    const uint32_t f = e == 0 ? m * 0x3f000000u : (126u + e) << 23 | m << 22;
    return __uint_as_float(f | (n & 8u) << 28);
}
template <bool kSixteen>
__device__ __forceinline__ float unit_of(uint32_t byte) {
    if (kSixteen) return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3)));
    return byte == 255 ? __int_as_float(0x7fffffff) : byte == 0 ? 0x1p-127f : __uint_as_float(byte << 23);
}
__device__ __forceinline__ uint16_t mx_narrow(float v, int dtype) {
    return dtype == PVS_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}

// What codes stand for: eight a thread where rows of `out` are aligned, else one, so that
// neighbours write neighbours.  A code's value times its group's scale is exact, so that the product
// with the row's is the only one that rounds (both scales together may be infinite, or no whole
// number of the smallest float32).
constexpr int kUnpack = 4;
template <bool kSixteen, bool WIDE>
__global__ void __launch_bounds__(kPackThreads) mx_unpack_kernel(const uint8_t* __restrict__ codes,
                                                                 const uint8_t* __restrict__ scales,
                                                                 const float* __restrict__ row_scales,
                                                                 int64_t rows, int cols, int kp, void* out,
                                                                 int64_t ldout, int dtype) {
    next_early();
    wait_before();
    constexpr int kGroup = kSixteen ? 16 : 32;
    const int blocks = kp / (4 * kGroup);
    auto scale_at = [&](int64_t row, int c) {
        return __ldg(scales + (row / 128 * blocks + c / (4 * kGroup)) * 512 + (row & 31) * 16 +
                     ((row >> 5) & 3) * 4 + c / kGroup % 4);
    };
    if (!WIDE) {
        for (int64_t row = (int64_t)blockIdx.x * kPackWarps + (threadIdx.x >> 5); row < rows;
             row += (int64_t)gridDim.x * kPackWarps) {
            const float rs = kSixteen ? __ldg(row_scales + row) : 1.0f;
#pragma unroll 4
            for (int c = threadIdx.x & 31; c < cols; c += 32) {
                const uint32_t n = __ldg(codes + row * (kp / 2) + c / 2) >> (4 * (c & 1)) & 15u;
                const float v = value_of(n) * unit_of<kSixteen>(scale_at(row, c)) * rs;
                if (dtype == PVS_F32)
                    static_cast<float*>(out)[row * ldout + c] = v;
                else
                    static_cast<uint16_t*>(out)[row * ldout + c] = mx_narrow(v, dtype);
            }
        }
        return;
    }
    // a warp takes neighbouring pieces of 256 columns
    const int lane = threadIdx.x & 31, slabs = (cols + 255) / 256;
    const int64_t total = rows * slabs, p0 = ((int64_t)blockIdx.x * kPackWarps + (threadIdx.x >> 5)) * kUnpack;
    int64_t row = quotient_of(p0, slabs);
    int c = (int)(p0 - row * slabs) * 256 + 8 * lane;
#pragma unroll
    for (int i = 0; i < kUnpack; ++i, c += 256) {
        if (p0 + i >= total) return;
        if (c - 8 * lane >= cols) {
            ++row;
            c = 8 * lane;
        }
        if (c >= cols) continue;
        const uint32_t word = __ldg(reinterpret_cast<const uint32_t*>(codes + row * (kp / 2) + c / 2));
        const float unit = unit_of<kSixteen>(scale_at(row, c)), rs = kSixteen ? __ldg(row_scales + row) : 1.0f;
        float v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(word >> (8 * k)), __NV_E2M1);
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
            v[2 * k] = f.x;
            v[2 * k + 1] = f.y;
        }
        times(v, unit);
        if (kSixteen) times(v, rs);
        const int64_t at = row * ldout + c;
        if (dtype == PVS_F32) {
            float* o = static_cast<float*>(out) + at;
            if (c + 8 <= cols && (reinterpret_cast<uintptr_t>(o) & 31u) == 0) {
                asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(o), "f"(v[0]), "f"(v[1]),
                             "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                             : "memory");
            } else if (c + 8 <= cols) {
                *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < cols) o[k] = v[k];
            }
        } else {
            uint32_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                h[k] = mx_narrow(v[2 * k], dtype) | (uint32_t)mx_narrow(v[2 * k + 1], dtype) << 16;
            uint16_t* o = static_cast<uint16_t*>(out) + at;
            if (c + 8 <= cols) {
                *reinterpret_cast<uint4*>(o) = make_uint4(h[0], h[1], h[2], h[3]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < cols) o[k] = (uint16_t)(h[k >> 1] >> (16 * (k & 1)));
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
    const PackArgs a{x, ldx, rows, round_up(rows, 128), cols, mx_padded(cols), codes, scales, row_scales};
    const int warps = a.kp > 512 * kHeld ? 4 : a.kp > 256 * kHeld ? 2 : 1;
    const int64_t per_block = kPackWarps / warps;
    const int64_t grid = std::min<int64_t>((a.padded_rows + per_block - 1) / per_block, 1 << 20);
    const bool w = mx_wide(x, ldx, dtype);
    count_launches(1);
    return launch_early(group == 16 ? pack_of<true>(dtype, w, warps) : pack_of<false>(dtype, w, warps), grid,
                        kPackThreads, 0, st, a);
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
    const bool w = mx_wide(out, ldout, dtype);
    const int64_t per_block = kPackWarps * (w ? kUnpack : 1);
    const int64_t blocks = (rows * (w ? (cols + 255) / 256 : 1) + per_block - 1) / per_block;
    if (blocks > 0x7fffffff) return PVS_ERR_INVALID;
    count_launches(1);
    return mx_queued(launch_early(
        group == 16 ? (w ? mx_unpack_kernel<true, true> : mx_unpack_kernel<true, false>)
                    : (w ? mx_unpack_kernel<false, true> : mx_unpack_kernel<false, false>),
        blocks, kPackThreads, 0, static_cast<cudaStream_t>(cuda_stream), codes, scales, row_scales, rows, cols,
        mx_padded(cols), out, ldout, dtype));
}

// Products of a few rows with weights kept in 4 bits (head.h).
//
// Bound by the weights' bytes (half a byte each, and the scales).  A warp takes 16
// rows of weights by 128 of k at a time: each lane 16 bytes (32 codes) of two
// rows, which the layout orders so that one 32-bit word of the four lanes of a row
// is one group of 32.  A code's nibble u under the exponent of 16 is the bf16
// 16 + u / 8 (exact); 17 less is an eighth of the code, and pairs of them are the
// A operand of mma.sync m16n8k16 as they stand.  The B operand's 8 columns are
// the rows of x in one (bf16), two (f16) or three (float32) exact bf16 parts.
// A group's product starts from zero and joins the float32 sums times its scale.
// k is split over the warps of a block where there are few rows of weights.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "../../include/head.h"
#include "head_gemm.h"
#include "kernels.h"
#include "pvs_common.cuh"

namespace pvs {
namespace head {
namespace {

constexpr int kWqThreads = 256;
constexpr int kWqWarps = kWqThreads / 32;
constexpr int kWqBlockBytes = 2048;      // x fragments of 128 of k and 8 columns
constexpr int kWqSmem = 96 * 1024;       // of x fragments, at most

__device__ __forceinline__ float load_x(const void* p, int dtype, int64_t i) {
    if (dtype == PVS_F32) return static_cast<const float*>(p)[i];
    if (dtype == PVS_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_y(void* p, int dtype, int64_t i, float v) {
    if (dtype == PVS_F32)
        static_cast<float*>(p)[i] = v;
    else if (dtype == PVS_BF16)
        static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else
        static_cast<__half*>(p)[i] = __float2half_rn(v);
}

// The bits of one bf16 part of x: parts 0, 1, .. are its leading 8 bits, the
// next 8, ..; cut, not rounded, so that they add up to x.
__device__ __forceinline__ uint32_t part_bits(float x, int part) {
    uint32_t h = __float_as_uint(x) & 0xffff0000u;
    for (int i = 0; i < part; ++i) {
        x = isfinite(x) ? x - __uint_as_float(h) : 0.0f;
        h = __float_as_uint(x) & 0xffff0000u;
    }
    // a NaN whose payload is in the low bits stays one
    if (x != x) h |= 0x00400000u;
    return h >> 16;
}

// Pair `m` of a word's nibbles, m and m + 4, as two bf16 codes in eighths: no
// product with x is larger than x then, and only a result that is too large for
// float32 overflows.
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int m) {
    const uint32_t u = ((w >> (4 * m)) & 0x000f000fu) | 0x41804180u;   // 16 + u / 8
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(u), "r"(0x41884188u));   // - 17
    return r;
}

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct WqArgs {
    const void* x;
    int64_t ldx;
    int batch, parts, dtype;
    const uint8_t* codes;
    const uint16_t* scales;
    int64_t rows;
    int cols, blocks;        // blocks of 128 of k
    void* y;
    int64_t ldy;
    int kw;                  // warps that share rows, each with blocks of its own
    int chunk;               // blocks whose x fragments are in shared memory at once
};

// NT: 8 columns (parts of rows of x) each; GROUP: weights per scale.
template <int NT, int GROUP>
__global__ void __launch_bounds__(kWqThreads) wq_matvec_kernel(const WqArgs a) {
    extern __shared__ uint4 xf[];                     // [block][word][NT][lane]
    __shared__ float out[kWqWarps][16][NT * 8 + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int team = warp / a.kw, share = warp % a.kw;
    const int teams = kWqWarps / a.kw;
    constexpr int kScales = 128 / GROUP;              // a block
    const int64_t code_row = (int64_t)a.blocks * 64, scale_row = (int64_t)a.blocks * kScales;
    const int64_t tiles = (a.rows + 15) / 16;
    const bool reload = a.chunk < a.blocks;
    bool loaded = false;
    for (int64_t t0 = (int64_t)blockIdx.x * teams; t0 < tiles; t0 += (int64_t)gridDim.x * teams) {
        const int64_t tile = t0 + team;
        const int64_t r0 = min(tile * 16 + g, a.rows - 1), r1 = min(tile * 16 + g + 8, a.rows - 1);
        float acc[NT][4] = {};
        for (int c0 = 0; c0 < a.blocks; c0 += a.chunk) {
            const int c1 = min(c0 + a.chunk, a.blocks);
            if (reload || !loaded) {
                __syncthreads();
                for (int i = threadIdx.x; i < (c1 - c0) * 4 * NT * 32; i += kWqThreads) {
                    const int l = i & 31, nt = (i >> 5) % NT, word = (i / (32 * NT)) & 3;
                    const int blk = c0 + i / (128 * NT);
                    const int col = nt * 8 + (l >> 2), b = col / a.parts, part = col % a.parts;
                    const int k = blk * 128 + word * 32 + (l & 3) * 8;
                    uint32_t h[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        h[j] = b < a.batch && k + j < a.cols
                                   ? part_bits(load_x(a.x, a.dtype, b * a.ldx + k + j), part)
                                   : 0u;
                    xf[i] = make_uint4(h[0] | (h[4] << 16), h[1] | (h[5] << 16),
                                       h[2] | (h[6] << 16), h[3] | (h[7] << 16));
                }
                __syncthreads();
                loaded = true;
            }
            if (tile < tiles) {
                for (int blk = c0 + share; blk < c1; blk += a.kw) {
                    const uint4 w0 = __ldg(reinterpret_cast<const uint4*>(
                        a.codes + r0 * code_row + (int64_t)blk * 64 + t * 16));
                    const uint4 w1 = __ldg(reinterpret_cast<const uint4*>(
                        a.codes + r1 * code_row + (int64_t)blk * 64 + t * 16));
                    const uint32_t a0[4] = {w0.x, w0.y, w0.z, w0.w};
                    const uint32_t a1[4] = {w1.x, w1.y, w1.z, w1.w};
                    float s0[kScales], s1[kScales];
#pragma unroll
                    for (int i = 0; i < kScales; ++i) {
                        s0[i] = __uint_as_float(
                            (uint32_t)__ldg(a.scales + r0 * scale_row + blk * kScales + i) << 16);
                        s1[i] = __uint_as_float(
                            (uint32_t)__ldg(a.scales + r1 * scale_row + blk * kScales + i) << 16);
                    }
                    const uint4* xb = xf + (blk - c0) * 4 * NT * 32 + lane;
                    float part[NT][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (i % (GROUP / 32) == 0) {
#pragma unroll
                            for (int n = 0; n < NT; ++n)
                                part[n][0] = part[n][1] = part[n][2] = part[n][3] = 0.0f;
                        }
                        uint32_t p0[4], p1[4];
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            p0[m] = code_pair(a0[i], m);
                            p1[m] = code_pair(a1[i], m);
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint4 x = xb[(i * NT + n) * 32];
                            mma_16816(part[n], p0[0], p1[0], p0[1], p1[1], x.x, x.y);
                            mma_16816(part[n], p0[2], p1[2], p0[3], p1[3], x.z, x.w);
                        }
                        if (i % (GROUP / 32) == GROUP / 32 - 1) {
                            const float f0 = s0[i / (GROUP / 32)], f1 = s1[i / (GROUP / 32)];
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                acc[n][0] = fmaf(f0, part[n][0], acc[n][0]);
                                acc[n][1] = fmaf(f0, part[n][1], acc[n][1]);
                                acc[n][2] = fmaf(f1, part[n][2], acc[n][2]);
                                acc[n][3] = fmaf(f1, part[n][3], acc[n][3]);
                            }
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            out[warp][g][n * 8 + 2 * t] = acc[n][0];
            out[warp][g][n * 8 + 2 * t + 1] = acc[n][1];
            out[warp][g + 8][n * 8 + 2 * t] = acc[n][2];
            out[warp][g + 8][n * 8 + 2 * t + 1] = acc[n][3];
        }
        __syncthreads();
        // a row of y takes the sums of a team's warps, smallest parts first
        for (int i = threadIdx.x; i < teams * 16 * a.batch; i += kWqThreads) {
            const int r = i % (teams * 16), b = i / (teams * 16);
            const int64_t row = t0 * 16 + r;
            if (row >= a.rows) continue;
            float v = 0.0f;
            for (int p = a.parts - 1; p >= 0; --p)
                for (int s = 0; s < a.kw; ++s)
                    v += out[(r >> 4) * a.kw + s][r & 15][b * a.parts + p];
            store_y(a.y, a.dtype, b * a.ldy + row, 8.0f * v);
        }
        __syncthreads();
    }
}

template <int NT>
cudaError_t launch_matvec(const WqArgs& a, int group, int grid, cudaStream_t st) {
    const size_t smem = (size_t)a.chunk * NT * kWqBlockBytes;
    const void* fn = group == 32   ? (const void*)wq_matvec_kernel<NT, 32>
                     : group == 64 ? (const void*)wq_matvec_kernel<NT, 64>
                                   : (const void*)wq_matvec_kernel<NT, 128>;
    cudaError_t e = raise_smem_limit(fn, smem);
    if (e != cudaSuccess) return e;
    count_launches(1);
    if (group == 32)
        wq_matvec_kernel<NT, 32><<<grid, kWqThreads, smem, st>>>(a);
    else if (group == 64)
        wq_matvec_kernel<NT, 64><<<grid, kWqThreads, smem, st>>>(a);
    else
        wq_matvec_kernel<NT, 128><<<grid, kWqThreads, smem, st>>>(a);
    return cudaGetLastError();
}

// A warp per block of 128 weights, four to a lane.
__global__ void __launch_bounds__(256) wq_pack_kernel(const void* w, int64_t ldw, int64_t rows,
                                                      int cols, int dtype, int group, int blocks,
                                                      uint8_t* codes, uint16_t* scales) {
    const int lane = threadIdx.x & 31;
    const int64_t total = rows * blocks;
    const int64_t step = (int64_t)gridDim.x * 8;
    for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < total; i += step) {
        const int64_t row = i / blocks;
        const int blk = (int)(i - row * blocks);
        const int k = blk * 128 + lane * 4;
        float v[4], top = 0.0f;
        bool finite = true;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = k + j < cols ? load_x(w, dtype, row * ldw + k + j) : 0.0f;
            finite &= isfinite(v[j]);
            top = fmaxf(top, fabsf(v[j]));
        }
        const int lanes = group / 4;
        for (int o = lanes / 2; o > 0; o >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            finite &= __shfl_xor_sync(0xffffffffu, finite ? 1 : 0, o) != 0;
        }
        uint16_t sb = 0x3f80;                       // 1
        if (!finite) {
            sb = 0x7fff;                            // NaN
        } else if (top > 0.0f) {
            const __nv_bfloat16 s = __float2bfloat16_rn(__fmul_rn(top, 1.0f / 7.0f));
            sb = __bfloat16_as_ushort(s);
            if (sb == 0) sb = 1;
        }
        const float s = __uint_as_float((uint32_t)sb << 16);
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            int q = 0;
            if (finite) q = (int)fminf(fmaxf(roundf(__fdiv_rn(v[j], s)), -7.0f), 7.0f);
            bits |= (uint32_t)(q + 8) << (4 * j);
        }
        const int word = lane >> 3, t = (lane & 7) >> 1;
        *reinterpret_cast<uint16_t*>(codes + i * 64 + 16 * t + 4 * word + 2 * (lane & 1)) =
            (uint16_t)bits;
        if (lane % lanes == 0) scales[i * (128 / group) + lane / lanes] = sb;
    }
}

__global__ void __launch_bounds__(256) wq_unpack_kernel(const uint8_t* codes,
                                                        const uint16_t* scales, int64_t rows,
                                                        int cols, int group, int blocks, void* out,
                                                        int64_t ldo, int dtype) {
    const int lane = threadIdx.x & 31;
    const int64_t total = rows * blocks;
    const int64_t step = (int64_t)gridDim.x * 8;
    for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < total; i += step) {
        const int64_t row = i / blocks;
        const int blk = (int)(i - row * blocks);
        const int word = lane >> 3, t = (lane & 7) >> 1;
        const uint32_t bits = *reinterpret_cast<const uint16_t*>(codes + i * 64 + 16 * t +
                                                                 4 * word + 2 * (lane & 1));
        const float s = __uint_as_float(
            (uint32_t)scales[i * (128 / group) + lane * 4 / group] << 16);
        const int k = blk * 128 + lane * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (k + j < cols)
                store_y(out, dtype, row * ldo + k + j, s * (float)((int)((bits >> (4 * j)) & 15u) - 8));
    }
}

bool shape_ok(int64_t rows, int32_t cols, int32_t group, int32_t dtype) {
    return rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= kMaxDim &&
           (group == 32 || group == 64 || group == 128) && dtype >= PVS_BF16 && dtype <= PVS_F32;
}

pvs_status queued(cudaError_t e) {
    if (e == cudaSuccess) return PVS_OK;
    cudaGetLastError();
    return PVS_ERR_CUDA;
}

bool codes_aligned(const void* codes, const void* scales) {
    return ((reinterpret_cast<uintptr_t>(codes) & 15u) | (reinterpret_cast<uintptr_t>(scales) & 7u)) == 0;
}

}  // namespace
}  // namespace head
}  // namespace pvs

using namespace pvs;
using namespace pvs::head;

extern "C" pvs_status pvs_wq_pack(const void* w, int64_t ldw, int64_t rows, int32_t cols,
                                  int32_t dtype, int32_t group, uint8_t* codes, void* scales,
                                  void* cuda_stream) {
    if (!shape_ok(rows, cols, group, dtype) || ldw < cols) return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!w || !codes || !scales || !codes_aligned(codes, scales)) return PVS_ERR_INVALID;
    const int blocks = (cols + 127) / 128;
    count_launches(1);
    wq_pack_kernel<<<(unsigned)std::min<int64_t>((rows * blocks + 7) / 8, 152 * 32), 256, 0,
                     static_cast<cudaStream_t>(cuda_stream)>>>(
        w, ldw, rows, cols, dtype, group, blocks, codes, static_cast<uint16_t*>(scales));
    return queued(cudaGetLastError());
}

extern "C" pvs_status pvs_wq_unpack(const uint8_t* codes, const void* scales, int64_t rows,
                                    int32_t cols, int32_t group, void* out, int64_t ldout,
                                    int32_t dtype, void* cuda_stream) {
    if (!shape_ok(rows, cols, group, dtype) || ldout < cols) return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!out || !codes || !scales || !codes_aligned(codes, scales)) return PVS_ERR_INVALID;
    const int blocks = (cols + 127) / 128;
    count_launches(1);
    wq_unpack_kernel<<<(unsigned)std::min<int64_t>((rows * blocks + 7) / 8, 152 * 32), 256, 0,
                       static_cast<cudaStream_t>(cuda_stream)>>>(
        codes, static_cast<const uint16_t*>(scales), rows, cols, group, blocks, out, ldout, dtype);
    return queued(cudaGetLastError());
}

extern "C" pvs_status pvs_wq_matvec(const void* x, int64_t ldx, int32_t batch,
                                    const uint8_t* codes, const void* scales, int64_t rows,
                                    int32_t cols, int32_t group, int32_t dtype, void* y,
                                    int64_t ldy, void* cuda_stream) {
    if (!shape_ok(rows, cols, group, dtype) || batch < 0 || batch > 64 || ldx < cols || ldy < rows)
        return PVS_ERR_INVALID;
    if (rows == 0 || batch == 0) return PVS_OK;
    if (!x || !y || !codes || !scales || !codes_aligned(codes, scales)) return PVS_ERR_INVALID;
    Device dev;
    cudaError_t e = device(&dev);
    if (e != cudaSuccess) return queued(e);
    const int es = element_bytes(dtype);
    WqArgs a{};
    a.ldx = ldx;
    a.dtype = dtype;
    a.parts = dtype == PVS_BF16 ? 1 : dtype == PVS_F16 ? 2 : 3;
    a.codes = codes;
    a.scales = static_cast<const uint16_t*>(scales);
    a.rows = rows;
    a.cols = cols;
    a.blocks = (cols + 127) / 128;
    a.ldy = ldy;
    // a pass takes what 16 columns hold; one tile of 8 where that is enough
    const int most = 16 / a.parts;
    const int64_t tiles = (rows + 15) / 16;
    // warps share k until there are about 8 warps for every SM
    a.kw = 1;
    while (a.kw < 8 && a.kw * 2 <= a.blocks && tiles * a.kw < 8ll * dev.sms) a.kw *= 2;
    const int64_t groups = (tiles * a.kw + kWqWarps - 1) / kWqWarps;
    for (int b = 0; b < batch && e == cudaSuccess; b += most) {
        a.batch = std::min(most, batch - b);
        a.x = static_cast<const uint8_t*>(x) + (int64_t)b * ldx * es;
        a.y = static_cast<uint8_t*>(y) + (int64_t)b * ldy * es;
        const int nt = a.batch * a.parts > 8 ? 2 : 1;
        a.chunk = std::min(a.blocks, kWqSmem / (nt * kWqBlockBytes));
        const int grid = (int)std::min<int64_t>(groups, 2ll * dev.sms);
        e = nt == 1 ? launch_matvec<1>(a, group, grid, static_cast<cudaStream_t>(cuda_stream))
                    : launch_matvec<2>(a, group, grid, static_cast<cudaStream_t>(cuda_stream));
    }
    return queued(e);
}

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

// 32 codes of each of two rows, and their scales, as they come from memory.
template <int GROUP>
struct RowPair {
    uint4 w0, w1;
    uint2 s0, s1;            // 128 / GROUP bf16 scales each

    __device__ __forceinline__ void load(const uint8_t* c0, const uint8_t* c1, const uint16_t* f0,
                                         const uint16_t* f1, int blk) {
        w0 = __ldg(reinterpret_cast<const uint4*>(c0 + (int64_t)blk * 64));
        w1 = __ldg(reinterpret_cast<const uint4*>(c1 + (int64_t)blk * 64));
        if constexpr (GROUP == 32) {
            s0 = __ldg(reinterpret_cast<const uint2*>(f0) + blk);
            s1 = __ldg(reinterpret_cast<const uint2*>(f1) + blk);
        } else if constexpr (GROUP == 64) {
            s0.x = __ldg(reinterpret_cast<const uint32_t*>(f0) + blk);
            s1.x = __ldg(reinterpret_cast<const uint32_t*>(f1) + blk);
        } else {
            s0.x = __ldg(f0 + blk);
            s1.x = __ldg(f1 + blk);
        }
    }
    static __device__ __forceinline__ float scale(uint2 s, int group) {
        const uint32_t w = group < 2 ? s.x : s.y;
        return __uint_as_float(group & 1 ? w & 0xffff0000u : w << 16);
    }
};

// NT: 8 columns (parts of rows of x) each; GROUP: weights per scale; RT: tiles of 16
// rows a warp takes at once, which share the x fragments it reads.
// A warp's next block is loaded before it works on the present one.
template <int NT, int GROUP, int RT>
__global__ void __launch_bounds__(kWqThreads) wq_matvec_kernel(const WqArgs a) {
    extern __shared__ uint4 xf[];                     // [block][word][NT][lane]
    __shared__ float out[kWqWarps][16][NT * 8 + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int team = warp / a.kw, share = warp % a.kw;
    const int teams = kWqWarps / a.kw;
    const int64_t code_row = (int64_t)a.blocks * 64;
    const int64_t scale_row = (int64_t)a.blocks * (128 / GROUP);
    const int64_t tiles = (a.rows + 16 * RT - 1) / (16 * RT);
    const bool reload = a.chunk < a.blocks;
    bool loaded = false;
    for (int64_t t0 = (int64_t)blockIdx.x * teams; t0 < tiles; t0 += (int64_t)gridDim.x * teams) {
        const int64_t tile = t0 + team;
        const uint8_t* code[RT][2];
        const uint16_t* scale[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t row = min((tile * RT + r) * 16 + g + 8 * h, a.rows - 1);
                code[r][h] = a.codes + row * code_row + t * 16;
                scale[r][h] = a.scales + row * scale_row;
            }
        float acc[RT][NT][4] = {};
        for (int c0 = 0; c0 < a.blocks; c0 += a.chunk) {
            const int c1 = min(c0 + a.chunk, a.blocks);
            RowPair<GROUP> next[RT];
            const bool mine = tile < tiles && c0 + share < c1;
            if (mine) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    next[r].load(code[r][0], code[r][1], scale[r][0], scale[r][1], c0 + share);
            }
            if (reload || !loaded) {
                if (reload) __syncthreads();
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
            if (!mine) continue;
            for (int blk = c0 + share; blk < c1; blk += a.kw) {
                RowPair<GROUP> now[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) now[r] = next[r];
                const int after = min(blk + a.kw, c1 - 1);   // (past the end: read again, unused)
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    next[r].load(code[r][0], code[r][1], scale[r][0], scale[r][1], after);
                const uint4* xb = xf + (blk - c0) * 4 * NT * 32 + lane;
                float part[RT][NT][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint4 x[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) x[n] = xb[(i * NT + n) * 32];
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const uint32_t w0 = i == 0   ? now[r].w0.x
                                            : i == 1 ? now[r].w0.y
                                            : i == 2 ? now[r].w0.z
                                                     : now[r].w0.w;
                        const uint32_t w1 = i == 0   ? now[r].w1.x
                                            : i == 1 ? now[r].w1.y
                                            : i == 2 ? now[r].w1.z
                                                     : now[r].w1.w;
                        if (i % (GROUP / 32) == 0) {
#pragma unroll
                            for (int n = 0; n < NT; ++n)
                                part[r][n][0] = part[r][n][1] = part[r][n][2] = part[r][n][3] = 0.0f;
                        }
                        uint32_t p0[4], p1[4];
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            p0[m] = code_pair(w0, m);
                            p1[m] = code_pair(w1, m);
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma_16816(part[r][n], p0[0], p1[0], p0[1], p1[1], x[n].x, x[n].y);
                            mma_16816(part[r][n], p0[2], p1[2], p0[3], p1[3], x[n].z, x[n].w);
                        }
                        if (i % (GROUP / 32) == GROUP / 32 - 1) {
                            const float f0 = RowPair<GROUP>::scale(now[r].s0, i / (GROUP / 32));
                            const float f1 = RowPair<GROUP>::scale(now[r].s1, i / (GROUP / 32));
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                acc[r][n][0] = fmaf(f0, part[r][n][0], acc[r][n][0]);
                                acc[r][n][1] = fmaf(f0, part[r][n][1], acc[r][n][1]);
                                acc[r][n][2] = fmaf(f1, part[r][n][2], acc[r][n][2]);
                                acc[r][n][3] = fmaf(f1, part[r][n][3], acc[r][n][3]);
                            }
                        }
                    }
                }
            }
        }
        // a row of y takes the sums of a team's warps, smallest parts first
#pragma unroll
        for (int r = 0; r < RT; ++r) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                out[warp][g][n * 8 + 2 * t] = acc[r][n][0];
                out[warp][g][n * 8 + 2 * t + 1] = acc[r][n][1];
                out[warp][g + 8][n * 8 + 2 * t] = acc[r][n][2];
                out[warp][g + 8][n * 8 + 2 * t + 1] = acc[r][n][3];
            }
            const bool alone = a.kw == 1;     // the warp's own sums: no other warp to wait for
            if (alone) __syncwarp(); else __syncthreads();
            const int first = alone ? lane : threadIdx.x, step = alone ? 32 : kWqThreads;
            const int width = alone ? 16 : teams * 16;
            for (int i = first; i < width * a.batch; i += step) {
                const int q = i % width, b = i / width, tm = alone ? warp : q >> 4;
                const int64_t row = ((t0 + tm) * RT + r) * 16 + (q & 15);
                if (t0 + tm >= tiles || row >= a.rows) continue;
                float v = 0.0f;
                for (int p = a.parts - 1; p >= 0; --p)
                    for (int s = 0; s < a.kw; ++s) v += out[tm * a.kw + s][q & 15][b * a.parts + p];
                store_y(a.y, a.dtype, b * a.ldy + row, 8.0f * v);
            }
            if (alone) __syncwarp(); else __syncthreads();
        }
    }
}

template <int NT, int RT>
cudaError_t launch_matvec(const WqArgs& a, int group, int grid, cudaStream_t st) {
    const size_t smem = (size_t)a.chunk * NT * kWqBlockBytes;
    const void* fn = group == 32   ? (const void*)wq_matvec_kernel<NT, 32, RT>
                     : group == 64 ? (const void*)wq_matvec_kernel<NT, 64, RT>
                                   : (const void*)wq_matvec_kernel<NT, 128, RT>;
    cudaError_t e = raise_smem_limit(fn, smem);
    if (e != cudaSuccess) return e;
    count_launches(1);
    if (group == 32)
        wq_matvec_kernel<NT, 32, RT><<<grid, kWqThreads, smem, st>>>(a);
    else if (group == 64)
        wq_matvec_kernel<NT, 64, RT><<<grid, kWqThreads, smem, st>>>(a);
    else
        wq_matvec_kernel<NT, 128, RT><<<grid, kWqThreads, smem, st>>>(a);
    return cudaGetLastError();
}

// Eight weights from column k, zeros past the row: 16-byte loads where WIDE.
template <bool WIDE>
__device__ __forceinline__ void load_eight(const void* w, int dtype, int64_t at, int k, int cols,
                                           float (&v)[8]) {
    if (WIDE && k + 8 <= cols) {
        if (dtype == PVS_F32) {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(w) + at + k);
            const float4 a = __ldg(p), b = __ldg(p + 1);
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
            v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else {
            const uint4 a =
                __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w) + at + k));
            const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t h = (u[j >> 1] >> (16 * (j & 1))) & 0xffffu;
                v[j] = dtype == PVS_BF16 ? __uint_as_float(h << 16)
                                         : __half2float(__ushort_as_half((uint16_t)h));
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < cols ? load_x(w, dtype, at + k + j) : 0.0f;
}

// A word (8 weights) per lane, two blocks of 128 a warp and step; a warp runs
// along a row.  Word l of a block holds k = 8 l ..: group l / 4, byte 16 (l % 4) + 4 (l / 4).
template <bool WIDE>
__global__ void __launch_bounds__(256) wq_pack_kernel(const void* w, int64_t ldw, int64_t rows,
                                                      int cols, int dtype, int group, int blocks,
                                                      uint8_t* codes, uint16_t* scales) {
    const int lane = threadIdx.x & 31, l = lane & 15;
    const int lanes = group / 8;
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < rows;
         row += (int64_t)gridDim.x * 8) {
        const int64_t at = row * ldw;
#pragma unroll 2
        for (int b0 = 0; b0 < blocks; b0 += 2) {
            const int blk = b0 + (lane >> 4);
            float v[8];
            load_eight<WIDE>(w, dtype, at, blk * 128 + l * 8, cols, v);
            // the largest magnitude by its bits: infinities and NaN are above every number
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
            for (int o = lanes / 2; o > 0; o >>= 1)
                top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (blk >= blocks) continue;            // (the shuffles are done: half a warp stops)
            uint32_t sb = 0x3f80;                   // 1
            if (top >= 0x7f800000u) {
                sb = 0x7fff;                        // NaN
            } else if (top != 0u) {
                sb = __bfloat16_as_ushort(
                    __float2bfloat16_rn(__fmul_rn(__uint_as_float(top), 1.0f / 7.0f)));
                if (sb == 0) sb = 1;
            }
            const float s = __uint_as_float(sb << 16);
            uint32_t bits = 0x88888888u;
            if (top < 0x7f800000u) {
                // as in the 8-bit quantizer: w / s by a product, rounded by a sum that
                // leaves q + 8 in the low bits, unless that is near a tie
                const float r = __fdiv_rn(1.0f, s), k = 12582912.0f + 8.0f;
                float far = 0.0f;
                bits = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float t = __fmul_rn(v[j], r), f = __fadd_rn(t, k);
                    far = fmaxf(far, fabsf(__fsub_rn(t, __fsub_rn(f, k))));
                    bits |= (__float_as_uint(f) & 15u) << (4 * j);
                }
                if (!(far < 0.5f - 0x1p-14f) || s < kFastScaleMin) {
                    bits = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int q = (int)fminf(fmaxf(roundf(__fdiv_rn(v[j], s)), -7.0f), 7.0f);
                        bits |= (uint32_t)(q + 8) << (4 * j);
                    }
                }
            }
            const int64_t i = row * blocks + blk;
            *reinterpret_cast<uint32_t*>(codes + i * 64 + 16 * (l & 3) + 4 * (l >> 2)) = bits;
            if (l % lanes == 0) scales[i * (128 / group) + l / lanes] = (uint16_t)sb;
        }
        __syncwarp();
    }
}

template <bool WIDE>
__global__ void __launch_bounds__(256) wq_unpack_kernel(const uint8_t* codes,
                                                        const uint16_t* scales, int64_t rows,
                                                        int cols, int group, int blocks, void* out,
                                                        int64_t ldo, int dtype) {
    const int lane = threadIdx.x & 31, l = lane & 15;
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < rows;
         row += (int64_t)gridDim.x * 8) {
#pragma unroll 4
        for (int blk = lane >> 4; blk < blocks; blk += 2) {
            const int64_t i = row * blocks + blk;
            const uint32_t bits =
                __ldg(reinterpret_cast<const uint32_t*>(codes + i * 64 + 16 * (l & 3) + 4 * (l >> 2)));
            const float s =
                __uint_as_float((uint32_t)__ldg(scales + i * (128 / group) + l * 8 / group) << 16);
            const int k = blk * 128 + l * 8;
            const int64_t at = row * ldo + k;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = s * (float)((int)((bits >> (4 * j)) & 15u) - 8);
            if (WIDE && k + 8 <= cols) {
                if (dtype == PVS_F32) {
                    float4* p = reinterpret_cast<float4*>(static_cast<float*>(out) + at);
                    p[0] = make_float4(v[0], v[1], v[2], v[3]);
                    p[1] = make_float4(v[4], v[5], v[6], v[7]);
                } else {
                    uint32_t h[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (dtype == PVS_BF16) {
                            const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
                            h[j] = *reinterpret_cast<const uint32_t*>(&p);
                        } else {
                            const __half2 p = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
                            h[j] = *reinterpret_cast<const uint32_t*>(&p);
                        }
                    }
                    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at) =
                        make_uint4(h[0], h[1], h[2], h[3]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (k + j < cols) store_y(out, dtype, at + j, v[j]);
            }
        }
    }
}

// Whether every eight elements of a row from a multiple of eight are aligned.
bool wide(const void* p, int64_t ld) {
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % 8 == 0;
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
    const unsigned grid = (unsigned)std::min<int64_t>((rows + 7) / 8, 1 << 20);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    uint16_t* s = static_cast<uint16_t*>(scales);
    count_launches(1);
    if (wide(w, ldw))
        wq_pack_kernel<true><<<grid, 256, 0, st>>>(w, ldw, rows, cols, dtype, group, blocks, codes, s);
    else
        wq_pack_kernel<false><<<grid, 256, 0, st>>>(w, ldw, rows, cols, dtype, group, blocks, codes, s);
    return queued(cudaGetLastError());
}

extern "C" pvs_status pvs_wq_unpack(const uint8_t* codes, const void* scales, int64_t rows,
                                    int32_t cols, int32_t group, void* out, int64_t ldout,
                                    int32_t dtype, void* cuda_stream) {
    if (!shape_ok(rows, cols, group, dtype) || ldout < cols) return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!out || !codes || !scales || !codes_aligned(codes, scales)) return PVS_ERR_INVALID;
    const int blocks = (cols + 127) / 128;
    const unsigned grid = (unsigned)std::min<int64_t>((rows + 7) / 8, 1 << 20);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const uint16_t* s = static_cast<const uint16_t*>(scales);
    count_launches(1);
    if (wide(out, ldout))
        wq_unpack_kernel<true><<<grid, 256, 0, st>>>(codes, s, rows, cols, group, blocks, out, ldout,
                                                     dtype);
    else
        wq_unpack_kernel<false><<<grid, 256, 0, st>>>(codes, s, rows, cols, group, blocks, out, ldout,
                                                      dtype);
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
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    // 32 rows a warp where that still gives every SM 16 warps or more; else 16 rows, and
    // warps share k until there are about 8 for every SM
    const int rt = rows >= 16ll * 32 * dev.sms ? 2 : 1;
    const int64_t tiles = (rows + 16 * rt - 1) / (16 * rt);
    a.kw = 1;
    while (a.kw < 8 && a.kw * 2 <= a.blocks && tiles * a.kw < 8ll * dev.sms) a.kw *= 2;
    const int64_t groups = (tiles * a.kw + kWqWarps - 1) / kWqWarps;
    for (int b = 0; b < batch && e == cudaSuccess; b += most) {
        a.batch = std::min(most, batch - b);
        a.x = static_cast<const uint8_t*>(x) + (int64_t)b * ldx * es;
        a.y = static_cast<uint8_t*>(y) + (int64_t)b * ldy * es;
        const int nt = a.batch * a.parts > 8 ? 2 : 1;
        a.chunk = std::min(a.blocks, kWqSmem / (nt * kWqBlockBytes));
        const int grid = (int)std::min<int64_t>(groups, 4ll * dev.sms);
        e = nt == 1 ? (rt == 1 ? launch_matvec<1, 1>(a, group, grid, st)
                               : launch_matvec<1, 2>(a, group, grid, st))
                    : (rt == 1 ? launch_matvec<2, 1>(a, group, grid, st)
                               : launch_matvec<2, 2>(a, group, grid, st));
    }
    return queued(e);
}

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
//
// 1,000,000 x 768 in groups of 128: one bf16 row 97 us (4.1 TB/s), four float32 rows
// (12 columns) 113 us; issue 56%, tensor pipe 38%, DRAM 45%: none of them full, latency bounds
// it.  Fully memory-bound it would be 58: prefetch deeper in registers, which are at their cap
// (112 us for the one row), and tiles run on into one another (110) were slower.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "../../include/head.h"
#include "f32x2.cuh"
#include "head_gemm.h"
#include "kernels.h"
#include "pvs_common.cuh"

namespace pvs {
namespace head {
namespace {

constexpr int kWqThreads = 256;
constexpr int kWqWarps = kWqThreads / 32;
constexpr int kWqBlockBytes = 2048;      // x fragments of 128 of k and 8 columns
// Of x fragments, at most: two blocks an SM with one or two tiles of columns.  With four (36 KB
// of sums beside) a second block fits up to 1,152 columns of weights; past 1,408 the fragments
// are made again for every 128 rows: 8 float32 rows over 200,000 x 1,024 weights take 55 us, over
// as many weights in rows of 1,280 76, of 2,048 104.
constexpr int kWqSmem = 88 * 1024;

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

// The leading 8 bits of x as a bf16's bits, and what is left of it: cut, not rounded,
// so that the parts add up to x.  Nothing is left of an infinity or a NaN.
__device__ __forceinline__ uint32_t cut_part(float& x) {
    uint32_t h = __float_as_uint(x) & 0xffff0000u;
    const bool finite = h < 0x7f800000u || (h >= 0x80000000u && h < 0xff800000u);
    if (x != x) h |= 0x00400000u;   // a NaN whose payload is in the low bits stays one
    x = finite ? x - __uint_as_float(h) : 0.0f;
    return h;
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

// The same from zero sums.
__device__ __forceinline__ void mma_16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                                uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                          uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight elements of a row from column k, zeros past the row: 16-byte loads where WIDE.
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
    if (k >= cols) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < cols ? load_x(w, dtype, at + k + j) : 0.0f;
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

// acc += the products of 16 rows by a block's 128 columns; x: the block's fragments.
template <int NT, int GROUP, int RT>
__device__ __forceinline__ void multiply(const RowPair<GROUP> (&w)[RT], const uint4* x,
                                         float (&acc)[RT][NT][4]) {
    constexpr int kWords = GROUP / 32;                // words of a group
    float part[RT][NT][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint4 f[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) f[n] = x[(i * NT + n) * 32];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const uint32_t w0 = i == 0 ? w[r].w0.x : i == 1 ? w[r].w0.y : i == 2 ? w[r].w0.z : w[r].w0.w;
            const uint32_t w1 = i == 0 ? w[r].w1.x : i == 1 ? w[r].w1.y : i == 2 ? w[r].w1.z : w[r].w1.w;
            uint32_t p0[4], p1[4];
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                p0[m] = code_pair(w0, m);
                p1[m] = code_pair(w1, m);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (i % kWords == 0)
                    mma_16816_first(part[r][n], p0[0], p1[0], p0[1], p1[1], f[n].x, f[n].y);
                else
                    mma_16816(part[r][n], p0[0], p1[0], p0[1], p1[1], f[n].x, f[n].y);
                mma_16816(part[r][n], p0[2], p1[2], p0[3], p1[3], f[n].z, f[n].w);
            }
            if (i % kWords == kWords - 1) {
                const float f0 = RowPair<GROUP>::scale(w[r].s0, i / kWords);
                const float f1 = RowPair<GROUP>::scale(w[r].s1, i / kWords);
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

// NT: 8 columns (parts of rows of x) each; GROUP: weights per scale; RT: tiles of 16
// rows a warp takes at once, which share the x fragments it reads.
// A warp's next block is loaded before it works on the present one.
template <int NT, int GROUP, int RT>
__global__ void __launch_bounds__(kWqThreads, 2) wq_matvec_kernel(const WqArgs a) {
    constexpr int kRowsAhead = 36;                    // a column's rows, apart in the banks
    extern __shared__ uint4 xf[];                     // [block][word][NT][lane]
    __shared__ float out[kWqWarps][NT * 8][kRowsAhead];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int kw = RT == 2 ? 1 : a.kw;                // (two tiles a warp: rows abound)
    const int team = warp / kw, share = warp % kw;
    const int teams = kWqWarps / kw;
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
                const int64_t row = min(tile * (16 * RT) + r * 16 + g + 8 * h, a.rows - 1);
                code[r][h] = a.codes + row * code_row + t * 16;
                scale[r][h] = a.scales + row * scale_row;
            }
        float acc[RT][NT][4] = {};
        for (int c0 = 0; c0 < a.blocks; c0 += a.chunk) {
            const int c1 = min(c0 + a.chunk, a.blocks);
            RowPair<GROUP> even[RT], odd[RT];
            auto load = [&](RowPair<GROUP>(&w)[RT], int blk) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
                    w[r].load(code[r][0], code[r][1], scale[r][0], scale[r][1], blk);
            };
            const bool mine = tile < tiles && c0 + share < c1;
            if (mine) load(even, c0 + share);
            if (reload || !loaded) {
                if (reload) __syncthreads();
                // eight elements of a row of x make an entry in each of its columns; the
                // columns past the last hold anything, and so do their sums
                const int eights = (c1 - c0) * 16;
                for (int i = threadIdx.x; i < eights * a.batch; i += kWqThreads) {
                    const int b = i / eights, k8 = i - b * eights;
                    float v[8];
                    load_eight<false>(a.x, a.dtype, b * a.ldx, (c0 * 16 + k8) * 8, a.cols, v);
                    const int at = (k8 >> 2) * NT * 32 + (k8 & 3);   // [block, word][0][lane]
                    for (int part = 0; part < a.parts; ++part) {
                        uint32_t h[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) h[j] = cut_part(v[j]);
                        const int col = b * a.parts + part;
                        xf[at + (col >> 3) * 32 + (col & 7) * 4] =
                            make_uint4(__byte_perm(h[0], h[4], 0x7632), __byte_perm(h[1], h[5], 0x7632),
                                       __byte_perm(h[2], h[6], 0x7632), __byte_perm(h[3], h[7], 0x7632));
                    }
                }
                __syncthreads();
                loaded = true;
            }
            if (!mine) continue;
            const uint4* x = xf + share * (4 * NT * 32) + lane;
            const int step = kw * (4 * NT * 32);
            int blk = c0 + share;
            while (true) {
                // two blocks a turn, so that no registers are copied
                int after = blk + kw;
                if (after < c1) load(odd, after);
                multiply<NT, GROUP, RT>(even, x, acc);
                if (after >= c1) break;
                x += step;
                blk = after + kw;
                if (blk < c1) load(even, blk);
                multiply<NT, GROUP, RT>(odd, x, acc);
                if (blk >= c1) break;
                x += step;
            }
        }
        // a row of y takes the sums of a team's warps, each with its smallest part first; a
        // lone warp waits for no other
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    out[warp][n * 8 + 2 * t + (j & 1)][r * 16 + g + 8 * (j >> 1)] = acc[r][n][j];
        if (kw == 1) __syncwarp(); else __syncthreads();
        const int64_t row = tile * (16 * RT) + lane;
        if (share == 0 && lane < 16 * RT && tile < tiles && row < a.rows) {
            const float* o = &out[warp][0][lane];
            for (int b = 0; b < a.batch; ++b) {
                float v = 0.0f;
                for (int s = 0; s < kw; ++s) {
                    const float* q = o + s * (NT * 8 * kRowsAhead);
                    if (a.parts == 3) v += q[2 * kRowsAhead];
                    if (a.parts >= 2) v += q[kRowsAhead];
                    v += q[0];
                }
                o += a.parts * kRowsAhead;
                store_y(a.y, a.dtype, b * a.ldy + row, 8.0f * v);
            }
        }
        if (kw == 1) __syncwarp(); else __syncthreads();
    }
}

using MatvecKernel = void (*)(const WqArgs);

template <int NT, int RT>
cudaError_t launch_matvec(const WqArgs& a, int group, int grid, cudaStream_t st) {
    const size_t smem = (size_t)a.chunk * NT * kWqBlockBytes;
    const MatvecKernel fn = group == 32   ? wq_matvec_kernel<NT, 32, RT>
                            : group == 64 ? wq_matvec_kernel<NT, 64, RT>
                                          : wq_matvec_kernel<NT, 128, RT>;
    const cudaError_t e = raise_smem_limit((const void*)fn, smem);
    if (e != cudaSuccess) return e;
    count_launches(1);
    // (not early: blocks that came before their turn share SMs unevenly, and 100,000 x 4096
    // took 63 us behind another product, 55 on its own)
    fn<<<grid, kWqThreads, smem, st>>>(a);
    return cudaGetLastError();
}

constexpr int kPackAhead = 4;    // steps whose loads are in flight together

// Eight weights as they lie in memory: 16-bit ones two to a word, float32 ones a word each.
template <int TYPE, bool WIDE>
struct Eight {
    static constexpr int kWords = TYPE == PVS_F32 ? 8 : 4;
    uint32_t w[kWords];

    __device__ __forceinline__ void load(const void* p, int64_t at, int k, int cols) {
        if (WIDE && k + 8 <= cols) {
            const uint4* q = TYPE == PVS_F32
                                 ? reinterpret_cast<const uint4*>(static_cast<const float*>(p) + at + k)
                                 : reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at + k);
            const uint4 a = __ldg(q);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
            if constexpr (TYPE == PVS_F32) {
                const uint4 c = __ldg(q + 1);
                w[4] = c.x, w[5] = c.y, w[6] = c.z, w[7] = c.w;
            }
            return;
        }
        if constexpr (TYPE != PVS_F32) {
            if (k + 8 <= cols) {
                load_eight_halves(static_cast<const uint16_t*>(p) + at + k, w);
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
        if (k >= cols) return;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (k + j >= cols) continue;
            if constexpr (TYPE == PVS_F32)
                w[j] = __ldg(static_cast<const uint32_t*>(p) + at + k + j);
            else
                w[j >> 1] |= (uint32_t)__ldg(static_cast<const uint16_t*>(p) + at + k + j)
                             << (16 * (j & 1));
        }
    }
    // the largest magnitude by its bits, in the type's own
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
        if constexpr (TYPE == PVS_F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
            m = max(m & 0xffffu, m >> 16);
        }
        return m;
    }
    // infinities and NaN are above every number
    static __device__ __forceinline__ bool finite(uint32_t top) {
        return top < (TYPE == PVS_F32 ? 0x7f800000u : TYPE == PVS_BF16 ? 0x7f80u : 0x7c00u);
    }
    static __device__ __forceinline__ float value(uint32_t bits) {
        if constexpr (TYPE == PVS_F32) return __uint_as_float(bits);
        if constexpr (TYPE == PVS_BF16) return __uint_as_float(bits << 16);
        return __half2float(__ushort_as_half((uint16_t)bits));
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if constexpr (TYPE == PVS_F32) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
        } else if constexpr (TYPE == PVS_BF16) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                v[j] = __uint_as_float(w[j >> 1] << 16);
                v[j + 1] = __uint_as_float(w[j >> 1] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j >> 1]));
                v[j] = f.x;
                v[j + 1] = f.y;
            }
        }
    }
};

// A word (8 weights) per lane, two blocks of 128 a warp and step; a warp runs
// along a row.  Word l of a block holds k = 8 l ..: group l / 4 of 32, byte 16 (l % 4) +
// 4 (l / 4).  GS: log2 of the group.  200,000 x 1,000 in f16 take 137 us (3.7 TB/s), bound
// by issue (81%, about 20 instructions a weight); with the loads of rows that are not
// aligned, and the same stores, packing and unpacking take 251 us, else 213.
template <int TYPE, bool WIDE, int GS>
__global__ void __launch_bounds__(256) wq_pack_kernel(const void* __restrict__ w, int64_t ldw,
                                                      int64_t rows, int cols, int blocks,
                                                      uint8_t* __restrict__ codes,
                                                      uint16_t* __restrict__ scales) {
    next_early();
    wait_before();
    const int lane = threadIdx.x & 31, l = lane & 15, side = lane >> 4;
    constexpr int kLanes = 1 << (GS - 3);           // of a group
    const int at_code = 16 * (l & 3) + 4 * (l >> 2);
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < rows;
         row += (int64_t)gridDim.x * 8) {
        for (int first = 0; first < blocks; first += 2 * kPackAhead) {
            Eight<TYPE, WIDE> ahead[kPackAhead];
#pragma unroll
            for (int i = 0; i < kPackAhead; ++i)
                ahead[i].load(w, row * ldw, (first + 2 * i + side) * 128 + l * 8, cols);
#pragma unroll
            for (int i = 0; i < kPackAhead; ++i) {
                if (first + 2 * i >= blocks) break;
                const int blk = first + 2 * i + side;
                uint32_t top = ahead[i].top();
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1)
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                const bool finite = Eight<TYPE, WIDE>::finite(top);
                uint32_t sb = __bfloat16_as_ushort(__float2bfloat16_rn(
                    __fmul_rn(Eight<TYPE, WIDE>::value(top), 1.0f / 7.0f)));
                if (sb == 0) sb = 1;
                if (top == 0u) sb = 0x3f80;         // 1
                if (!finite) sb = 0x7fff;           // NaN
                const float s = __uint_as_float(sb << 16);
                uint32_t bits = 0x88888888u;
                if (finite) {
                    // as in the 8-bit quantizer: w / s by a product, rounded by a sum that
                    // leaves q + 8 in the low bits, unless that is near a tie; the sums'
                    // bits times powers of 16 add up to the word and a constant (modulo 2^32)
                    float v[8], r;
                    ahead[i].values(v);
                    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
                    const float k = 12582912.0f + 8.0f;
                    const uint64_t r2 = f2_pack(r, r), k2 = f2_pack(k, k), m2 = f2_pack(-k, -k);
                    const uint64_t minus = f2_pack(-1.0f, -1.0f);
                    float far = 0.0f;
                    bits = 0u - 0x4b400000u * 0x11111111u;
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const uint64_t t = f2_mul(f2_pack(v[j], v[j + 1]), r2), f = f2_add(t, k2);
                        float d0, d1, f0, f1;
                        f2_unpack(f2_fma(f2_add(f, m2), minus, t), d0, d1);
                        f2_unpack(f, f0, f1);
                        far = fmaxf(far, fmaxf(fabsf(d0), fabsf(d1)));
                        bits += (__float_as_uint(f0) << (4 * j)) + (__float_as_uint(f1) << (4 * j + 4));
                    }
                    if (!(far < 0.5f - 0x1p-14f) || s < kFastScaleMin) {
                        bits = 0;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int q =
                                (int)fminf(fmaxf(roundf(__fdiv_rn(v[j], s)), -7.0f), 7.0f);
                            bits |= (uint32_t)(q + 8) << (4 * j);
                        }
                    }
                }
                if (blk < blocks) {
                    const int64_t n = row * blocks + blk;
                    *reinterpret_cast<uint32_t*>(codes + n * 64 + at_code) = bits;
                    if ((l & (kLanes - 1)) == 0)
                        scales[(n << (7 - GS)) + (l >> (GS - 3))] = (uint16_t)sb;
                }
                __syncwarp();
            }
        }
    }
}

using PackKernel = void (*)(const void*, int64_t, int64_t, int, int, uint8_t*, uint16_t*);
template <int TYPE, bool WIDE>
PackKernel pack_kernel(int group) {
    return group == 32   ? wq_pack_kernel<TYPE, WIDE, 5>
           : group == 64 ? wq_pack_kernel<TYPE, WIDE, 6>
                         : wq_pack_kernel<TYPE, WIDE, 7>;
}
template <bool WIDE>
PackKernel pack_kernel(int dtype, int group) {
    return dtype == PVS_BF16  ? pack_kernel<PVS_BF16, WIDE>(group)
           : dtype == PVS_F16 ? pack_kernel<PVS_F16, WIDE>(group)
                              : pack_kernel<PVS_F32, WIDE>(group);
}

// What the codes stand for, in the same turns.  200,000 x 1,000 to f16: 78 us (DRAM 73% busy,
// issue 72%).
template <bool WIDE>
__global__ void __launch_bounds__(256) wq_unpack_kernel(const uint8_t* __restrict__ codes,
                                                        const uint16_t* __restrict__ scales,
                                                        int64_t rows, int cols, int gs, int blocks,
                                                        void* __restrict__ out, int64_t ldo,
                                                        int dtype) {
    next_early();
    wait_before();
    const int lane = threadIdx.x & 31, l = lane & 15, side = lane >> 4;
    const int at_code = 16 * (l & 3) + 4 * (l >> 2), at_scale = l >> (gs - 3);
    // where rows are not aligned, a warp's 256 values go through shared memory, so that
    // neighbours write neighbours
    __shared__ float stage[WIDE ? 1 : 8][WIDE ? 1 : 256 + 8];
    float* mine = stage[WIDE ? 0 : threadIdx.x >> 5];
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < rows;
         row += (int64_t)gridDim.x * 8) {
        for (int first = 0; first < blocks; first += 2 * kPackAhead) {
            uint32_t word[kPackAhead], unit[kPackAhead];
#pragma unroll
            for (int i = 0; i < kPackAhead; ++i) {
                const int64_t n = row * blocks + min(first + 2 * i + side, blocks - 1);
                word[i] = __ldg(reinterpret_cast<const uint32_t*>(codes + n * 64 + at_code));
                unit[i] = __ldg(scales + (n << (7 - gs)) + at_scale);
            }
#pragma unroll
            for (int i = 0; i < kPackAhead; ++i) {
                const int k = (first + 2 * i + side) * 128 + l * 8;
                if (WIDE && k >= cols) continue;
                if (!WIDE && (first + 2 * i) * 128 >= cols) break;
                const float s = __uint_as_float(unit[i] << 16);
                // u under the exponent of 2^23 reads as 2^23 + u
                float v[8];
                const uint64_t s2 = f2_pack(s, s), k2 = f2_pack(-8388616.0f, -8388616.0f);
#pragma unroll
                for (int j = 0; j < 8; j += 2)
                    f2_unpack(f2_mul(f2_add(f2_pack(__uint_as_float(((word[i] >> (4 * j)) & 15u) |
                                                                    0x4b000000u),
                                                    __uint_as_float(((word[i] >> (4 * j + 4)) & 15u) |
                                                                    0x4b000000u)),
                                            k2),
                                     s2),
                              v[j], v[j + 1]);
                if constexpr (!WIDE) {
                    // (every 32 values a word further: the eights of the lanes meet fewer conflicts)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int at = side * 128 + l * 8 + j;
                        mine[at + (at >> 5)] = v[j];
                    }
                    __syncwarp();
                    const int k0 = (first + 2 * i) * 128;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int at = j * 32 + lane;
                        if (k0 + at < cols)
                            store_y(out, dtype, row * ldo + k0 + at, mine[at + (at >> 5)]);
                    }
                    __syncwarp();
                    continue;
                }
                const int64_t at = row * ldo + k;
                if (k + 8 <= cols) {
                    if (dtype == PVS_F32) {
                        float4* p = reinterpret_cast<float4*>(static_cast<float*>(out) + at);
                        p[0] = make_float4(v[0], v[1], v[2], v[3]);
                        p[1] = make_float4(v[4], v[5], v[6], v[7]);
                    } else {
                        uint32_t h[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (dtype == PVS_BF16) {
                                const __nv_bfloat162 p =
                                    __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
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
}

// log2 of a group of 32, 64 or 128.
int group_shift(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }

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
    if (!w || !codes || !scales || !codes_aligned(codes, scales) || !on_elements(w, element_bytes(dtype)))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    const int blocks = (cols + 127) / 128;
    const unsigned grid = (unsigned)std::min<int64_t>((rows + 7) / 8, 1 << 20);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    uint16_t* s = static_cast<uint16_t*>(scales);
    count_launches(1);
    return queued(launch_early(wide(w, ldw) ? pack_kernel<true>(dtype, group)
                                            : pack_kernel<false>(dtype, group),
                               grid, 256, 0, st, w, ldw, rows, cols, blocks, codes, s));
}

extern "C" pvs_status pvs_wq_unpack(const uint8_t* codes, const void* scales, int64_t rows,
                                    int32_t cols, int32_t group, void* out, int64_t ldout,
                                    int32_t dtype, void* cuda_stream) {
    if (!shape_ok(rows, cols, group, dtype) || ldout < cols) return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!out || !codes || !scales || !codes_aligned(codes, scales) ||
        !on_elements(out, element_bytes(dtype)))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    const int blocks = (cols + 127) / 128;
    const unsigned grid = (unsigned)std::min<int64_t>((rows + 7) / 8, 1 << 20);
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const uint16_t* s = static_cast<const uint16_t*>(scales);
    count_launches(1);
    return queued(launch_early(wide(out, ldout) ? wq_unpack_kernel<true> : wq_unpack_kernel<false>,
                               grid, 256, 0, st, codes, s, rows, cols, group_shift(group), blocks,
                               out, ldout, dtype));
}

extern "C" pvs_status pvs_wq_matvec(const void* x, int64_t ldx, int32_t batch,
                                    const uint8_t* codes, const void* scales, int64_t rows,
                                    int32_t cols, int32_t group, int32_t dtype, void* y,
                                    int64_t ldy, void* cuda_stream) {
    if (!shape_ok(rows, cols, group, dtype) || batch < 0 || batch > 64 || ldx < cols || ldy < rows)
        return PVS_ERR_INVALID;
    if (rows == 0 || batch == 0) return PVS_OK;
    if (!x || !y || !codes || !scales || !codes_aligned(codes, scales) ||
        !on_elements(x, element_bytes(dtype)) || !on_elements(y, element_bytes(dtype)))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    const int es = element_bytes(dtype);
    cudaError_t e = cudaSuccess;
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
    // a pass takes what 32 columns hold, in one, two or four tiles of 8
    const int most = 32 / a.parts;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    for (int b = 0; b < batch && e == cudaSuccess; b += most) {
        a.batch = std::min(most, batch - b);
        a.x = static_cast<const uint8_t*>(x) + (int64_t)b * ldx * es;
        a.y = static_cast<uint8_t*>(y) + (int64_t)b * ldy * es;
        const int columns = a.batch * a.parts;
        const int nt = columns > 16 ? 4 : columns > 8 ? 2 : 1;
        // 32 rows a warp where that still gives every SM 16 warps or more (and the sums fit
        // the registers); else 16 rows, and warps share k until there are about 8 for every SM.
        // 1,000,000 x 768: 98 us with 32 rows, 111 with 16; 4,096 x 4,096: 17 with 16, 22 with
        // 32; 16,384 x 4,096: 19 with k shared, 28 without
        const int rt = nt < 4 && rows >= 16ll * 32 * dev.sms ? 2 : 1;
        const int64_t tiles = (rows + 16 * rt - 1) / (16 * rt);
        a.kw = 1;
        while (a.kw < 8 && a.kw * 2 <= a.blocks && tiles * a.kw < 8ll * dev.sms) a.kw *= 2;
        const int64_t groups = (tiles * a.kw + kWqWarps - 1) / kWqWarps;
        a.chunk = std::min(a.blocks, kWqSmem / (nt * kWqBlockBytes));
        // (as many blocks as run at once: each makes the fragments of x for itself)
        const int grid = (int)std::min<int64_t>(groups, 2ll * dev.sms);
        e = nt == 4   ? launch_matvec<4, 1>(a, group, grid, st)
            : nt == 2 ? (rt == 1 ? launch_matvec<2, 1>(a, group, grid, st)
                                 : launch_matvec<2, 2>(a, group, grid, st))
                      : (rt == 1 ? launch_matvec<1, 1>(a, group, grid, st)
                                 : launch_matvec<1, 2>(a, group, grid, st));
    }
    return queued(e);
}

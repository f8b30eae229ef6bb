// Rows kept in 8 bits between a forward and a backward pass (head.h): the
// per-vector quantizer of Sec. 2.3.1 without the norms, with an activation on
// the way, and the backward steps that read the codes.
//
// store, load and act_backward move a few bytes an element and are bound by
// memory; grad_weight is the product of head_gemm.cu over the rows.
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

template <int TYPE> struct Element;
template <> struct Element<PVS_BF16> {
    using T = __nv_bfloat16;
    static __device__ float to(T x) { return __bfloat162float(x); }
    static __device__ T from(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Element<PVS_F16> {
    using T = __half;
    static __device__ float to(T x) { return __half2float(x); }
    static __device__ T from(float x) { return __float2half_rn(x); }
};
template <> struct Element<PVS_F32> {
    using T = float;
    static __device__ float to(T x) { return x; }
    static __device__ T from(float x) { return x; }
};

__device__ __forceinline__ float gelu(float x) {
    return 0.5f * x * (1.0f + erff(x * 0.70710678118654752f));
}
__device__ __forceinline__ float gelu_slope(float x) {
    return 0.5f * (1.0f + erff(x * 0.70710678118654752f)) +
           x * __expf(-0.5f * x * x) * 0.39894228040143268f;
}

// A warp per row, which it reads twice (the second time from L1 or L2).
template <int TYPE>
__global__ void __launch_bounds__(256) ckpt_store_kernel(const void* x, int64_t ldx, int64_t rows,
                                                         int cols, int act, int8_t* codes,
                                                         int64_t ldc, float* scales, void* y,
                                                         int64_t ldy) {
    using E = Element<TYPE>;
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= rows) return;
    const typename E::T* v = static_cast<const typename E::T*>(x) + row * ldx;
    float top = 0.0f;
    bool finite = true;
    for (int j = lane; j < cols; j += 32) {
        const float f = E::to(v[j]);
        finite &= isfinite(f);
        top = fmaxf(top, fabsf(f));
    }
    top = warp_max(top);
    finite = __all_sync(0xffffffffu, finite);
    float s = top == 0.0f ? 1.0f : __fmul_rn(top, 1.0f / 127.0f);
    if (s == 0.0f) s = __uint_as_float(1u);
    const float r = __fdiv_rn(1.0f, s);
    if (lane == 0) scales[row] = finite ? s : __int_as_float(0x7fffffff);
    for (int j = lane; j < cols; j += 32) {
        const float f = E::to(v[j]);
        uint32_t c = 0;
        if (finite) {
            if (s >= kFastScaleMin)
                code_of(f, s, r, c);
            else
                c = (uint32_t)(int)fminf(fmaxf(roundf(__fdiv_rn(f, s)), -127.0f), 127.0f);
        }
        codes[row * ldc + j] = (int8_t)c;
        if (act == PVS_ACT_GELU) static_cast<typename E::T*>(y)[row * ldy + j] = E::from(gelu(f));
    }
}

template <int TYPE>
__global__ void __launch_bounds__(256) ckpt_load_kernel(const int8_t* codes, int64_t ldc,
                                                        const float* scales, int64_t rows,
                                                        int cols, void* out, int64_t ldo) {
    using E = Element<TYPE>;
    const int64_t total = rows * cols, stride = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += stride) {
        const int64_t row = i / cols, j = i - row * cols;
        static_cast<typename E::T*>(out)[row * ldo + j] =
            E::from(scales[row] * (float)codes[row * ldc + j]);
    }
}

template <int TYPE>
__global__ void __launch_bounds__(256) ckpt_act_kernel(const void* dy, int64_t lddy,
                                                       const int8_t* codes, int64_t ldc,
                                                       const float* scales, int64_t rows, int cols,
                                                       void* dx, int64_t lddx) {
    using E = Element<TYPE>;
    const int64_t total = rows * cols, stride = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += stride) {
        const int64_t row = i / cols, j = i - row * cols;
        const float g = E::to(static_cast<const typename E::T*>(dy)[row * lddy + j]);
        static_cast<typename E::T*>(dx)[row * lddx + j] =
            E::from(g * gelu_slope(scales[row] * (float)codes[row * ldc + j]));
    }
}

bool rows_ok(int64_t rows, int32_t cols, int32_t dtype) {
    return rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= kMaxDim && dtype >= PVS_BF16 &&
           dtype <= PVS_F32;
}

pvs_status queued(cudaError_t e = cudaSuccess) {
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e == cudaSuccess) return PVS_OK;
    cudaGetLastError();
    return PVS_ERR_CUDA;
}

unsigned grid_for(int64_t total) {
    return (unsigned)std::min<int64_t>((total + 255) / 256, 152 * 32);
}

struct GradPlan {
    int parts;
    int64_t lda, ldb;
    int splits;
    uint16_t *a, *b;
    float* slots;
    int64_t ldslot;
    size_t bytes;
};
GradPlan grad_plan(int64_t rows, int out_cols, int cols, int dtype, const Device& dev,
                   void* workspace) {
    GradPlan p{};
    p.parts = dtype == PVS_BF16 ? 1 : dtype == PVS_F16 ? 2 : 3;
    p.lda = round_up(out_cols, 8);
    p.ldb = round_up(cols, 8);
    p.ldslot = round_up(cols, 8);
    const int bn = tile_columns(cols);
    const int64_t units = (int64_t)((out_cols + kTileM - 1) / kTileM) * ((cols + bn - 1) / bn);
    const int64_t kc = (rows + kTileK - 1) / kTileK;
    // enough splits for every SM, none under 8 chunks
    int64_t s = std::max<int64_t>(1, std::min<int64_t>(dev.sms / std::min<int64_t>(units, dev.sms), kc / 8));
    // float32 sums: 128 steps at most before the splits are added with rounding
    if (dtype == PVS_F32) s = std::max<int64_t>(s, (kc + 31) / 32);
    p.splits = (int)s;
    Carver c{static_cast<uint8_t*>(workspace)};
    p.a = c.take<uint16_t>((int64_t)p.parts * rows * p.lda);
    p.b = c.take<uint16_t>(rows * p.ldb);
    if (p.splits > 1) p.slots = c.take<float>((int64_t)p.splits * out_cols * p.ldslot);
    p.bytes = c.used;
    return p;
}

}  // namespace
}  // namespace head
}  // namespace pvs

using namespace pvs;
using namespace pvs::head;

#define PVS_BY_TYPE(dtype, CALL)             \
    do {                                     \
        if ((dtype) == PVS_BF16) {           \
            constexpr int TYPE = PVS_BF16;   \
            CALL;                            \
        } else if ((dtype) == PVS_F16) {     \
            constexpr int TYPE = PVS_F16;    \
            CALL;                            \
        } else {                             \
            constexpr int TYPE = PVS_F32;    \
            CALL;                            \
        }                                    \
    } while (0)

extern "C" pvs_status pvs_ckpt_store(const void* x, int64_t ldx, int64_t rows, int32_t cols,
                                     int32_t dtype, int32_t act, int8_t* codes, int64_t ldcodes,
                                     float* scales, void* y, int64_t ldy, void* cuda_stream) {
    if (!rows_ok(rows, cols, dtype) || ldx < cols || ldcodes < cols ||
        (act != PVS_ACT_NONE && act != PVS_ACT_GELU) || (act != PVS_ACT_NONE && ldy < cols))
        return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!x || !codes || !scales || (act != PVS_ACT_NONE && !y)) return PVS_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    count_launches(1);
    PVS_BY_TYPE(dtype, (ckpt_store_kernel<TYPE><<<(unsigned)((rows + 7) / 8), 256, 0, st>>>(
                           x, ldx, rows, cols, act, codes, ldcodes, scales, y, ldy)));
    return queued();
}

extern "C" pvs_status pvs_ckpt_load(const int8_t* codes, int64_t ldcodes, const float* scales,
                                    int64_t rows, int32_t cols, void* out, int64_t ldout,
                                    int32_t dtype, void* cuda_stream) {
    if (!rows_ok(rows, cols, dtype) || ldcodes < cols || ldout < cols) return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!codes || !scales || !out) return PVS_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    count_launches(1);
    PVS_BY_TYPE(dtype, (ckpt_load_kernel<TYPE><<<grid_for(rows * cols), 256, 0, st>>>(
                           codes, ldcodes, scales, rows, cols, out, ldout)));
    return queued();
}

extern "C" pvs_status pvs_ckpt_act_backward(const void* dy, int64_t lddy, const int8_t* codes,
                                            int64_t ldcodes, const float* scales, int64_t rows,
                                            int32_t cols, int32_t dtype, int32_t act, void* dx,
                                            int64_t lddx, void* cuda_stream) {
    if (!rows_ok(rows, cols, dtype) || lddy < cols || ldcodes < cols || lddx < cols ||
        act != PVS_ACT_GELU)
        return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!dy || !codes || !scales || !dx) return PVS_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    count_launches(1);
    PVS_BY_TYPE(dtype, (ckpt_act_kernel<TYPE><<<grid_for(rows * cols), 256, 0, st>>>(
                           dy, lddy, codes, ldcodes, scales, rows, cols, dx, lddx)));
    return queued();
}

extern "C" pvs_status pvs_ckpt_grad_workspace(int64_t rows, int32_t out_cols, int32_t cols,
                                              int32_t dtype, size_t* bytes) {
    if (!bytes || !rows_ok(rows, cols, dtype) || out_cols < 1 || out_cols > kMaxDim)
        return PVS_ERR_INVALID;
    *bytes = 0;
    if (rows == 0) return PVS_OK;
    Device dev;
    const cudaError_t e = device(&dev);
    if (e != cudaSuccess) return queued(e);
    *bytes = grad_plan(rows, out_cols, cols, dtype, dev, nullptr).bytes;
    return PVS_OK;
}

extern "C" pvs_status pvs_ckpt_grad_weight(const void* dy, int64_t lddy, const int8_t* codes,
                                           int64_t ldcodes, const float* scales, int64_t rows,
                                           int32_t out_cols, int32_t cols, int32_t dtype, void* dw,
                                           int64_t lddw, void* workspace, size_t workspace_bytes,
                                           void* cuda_stream) {
    if (!rows_ok(rows, cols, dtype) || out_cols < 1 || out_cols > kMaxDim || lddy < out_cols ||
        ldcodes < cols || lddw < cols || !dw)
        return PVS_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t es = (size_t)element_bytes(dtype);
    if (rows == 0)
        return queued(cudaMemset2DAsync(dw, (size_t)lddw * es, 0, (size_t)cols * es,
                                        (size_t)out_cols, st));
    if (!dy || !codes || !scales) return PVS_ERR_INVALID;
    Device dev;
    cudaError_t e = device(&dev);
    if (e != cudaSuccess) return queued(e);
    const GradPlan p = grad_plan(rows, out_cols, cols, dtype, dev, workspace);
    if (workspace_bytes < p.bytes || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return PVS_ERR_INVALID;
    const pvs_status before = (pvs_status)take_status(dev);
    if (before != PVS_OK) return before;
    SplitArgs s{};
    s.src = dy;
    s.ld = lddy;
    s.rows = rows;
    s.cols = out_cols;
    s.dtype = dtype;
    s.row_scale = scales;
    s.dst = p.a;
    s.ldd = p.lda;
    s.part_stride = rows * p.lda;
    s.parts = p.parts;
    e = launch_split(s, st);
    if (e == cudaSuccess) e = launch_split_codes(codes, ldcodes, rows, cols, p.b, p.ldb, st);
    if (e != cudaSuccess) return queued(e);
    Args g{};
    g.status = dev.status;
    g.nprob = 1;
    Problem& q = g.p[0];
    set_tiles(q, out_cols, cols, tile_columns(cols), rows);
    q.splits = p.splits;
    if (!operand_map(&q.a, Matrix{p.a, rows, out_cols, p.lda, p.parts, rows * p.lda}, true, 0) ||
        !operand_map(&q.b, Matrix{p.b, rows, cols, p.ldb, 1, 0}, true, 0))
        return PVS_ERR_CUDA;
    q.a_mn = q.b_mn = 1;
    q.to_slots = p.splits > 1;
    q.slots = p.slots;
    q.slot_stride = (int64_t)out_cols * p.ldslot;
    q.ldslot = p.ldslot;
    q.out = dw;
    q.ldout = lddw;
    q.out_type = dtype;
    q.alpha0 = 1.0f;
    part_pairs(g, p.parts, 1);
    e = launch_gemm(kOut, g, dev.sms, st);
    if (e == cudaSuccess && q.to_slots)
        e = launch_sum_slots(p.slots, p.splits, q.slot_stride, p.ldslot, out_cols, cols, nullptr,
                             1.0f, dw, lddw, dtype, st);
    return queued(e);
}

// Softmax cross entropy of a few float32 rows and its gradients, without copies of the
// items.
//
//   l_tj = a <x_t, w_j> + b_j,   G_tj = coef_t 2^(l_tj - m_t), or hit_t at the target,
//   dx_t = a sum_j G_tj w_j,     dw_j = a sum_t G_tj x_t
//
// in float32 on the CUDA cores: 2 operations a row and element of w forward, 6 backward.
// The tensor cores want w in 16-bit parts, whose copies move 12 bytes an element forward
// and 40 in a step, where this reads 4 forward, and reads 8 and writes 4 backward.
//
// Logits: x lies in shared memory.  A warp takes I items at a time, its lanes the elements;
// the I R partial sums of R rows are turned round among the lanes as they are added, so
// that a lane ends with whole logits.  Gradients: a thread owns columns, and the items go
// by.  (Both in one kernel, tile by tile with a barrier between them and the second read
// of w from L1 and L2, took 1,640 us for 8 rows over 700,000 items of 768.)
//
// 700,000 items of 768, in us: the loss of 8 rows 411 (5.2 TB/s of w; on the tensor cores,
// with the copies, 1,178), of 16 rows 544 (1,174); a step of 8 rows 1,683 (4,870), of 16
// rows 2,271 (4,801).  Up to 8 rows the memory bounds it, at 16 the products' reads of x
// from shared memory and the FMAs.  More rows go to the tensor cores: 32 in two turns took
// 1,131 where those take 1,173.
#include "xent_few.h"

#include <algorithm>

#include "f32x2.cuh"
#include "kernels.h"
#include "pvs_common.cuh"

namespace pvs {
namespace head {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// A lane's four of 128 elements of a row from column k: in one load, or (rows that are not
// aligned) in four, neighbours at neighbours.  Past the row nothing is read.
template <bool WIDE>
__device__ __forceinline__ void load_four(const float* p, int k, int dim, float (&v)[4]) {
    const int lane = threadIdx.x & 31;
    if constexpr (WIDE) {
        k += 4 * lane;
        const float4 f = k < dim ? __ldg(reinterpret_cast<const float4*>(p + k))
                                 : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int at = k + lane + 32 * e;
            v[e] = at < dim ? __ldg(p + at) : 0.0f;
        }
    }
}

// The elements of a row of x in shared memory, zeros past the row.
__host__ __device__ __forceinline__ int padded(int dim) { return (dim + 127) / 128 * 128; }

__device__ __forceinline__ void fill_rows(const FewArgs& a, float* xs, int r, bool zero_ignored) {
    const int dp = padded(a.dim);
    for (int i = threadIdx.x; i < r * dp; i += blockDim.x) {
        const int t = i / dp, k = i - t * dp;
        float v = 0.0f;
        if (t < a.rows && k < a.dim && !(zero_ignored && a.targets[t] == a.ignore_index))
            v = a.x[t * a.ldx + k];
        xs[i] = v;
    }
}

// 32 values a lane to their sums over the lanes: lane l gets that of value l.
__device__ __forceinline__ float sum_across(float (&v)[32]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int bit = 16; bit > 0; bit >>= 1) {
        const bool upper = (lane & bit) != 0;
#pragma unroll
        for (int i = 0; i < bit; ++i) {
            const float got = __shfl_xor_sync(0xffffffffu, upper ? v[i] : v[i + bit], bit);
            v[i] = (upper ? v[i + bit] : v[i]) + got;
        }
    }
    return v[0];
}

// <x_t, w_j> of R rows and the I items from `item`, R I = 32 n: lane l of sums[q] has row
// l % R of the item (32 q + l) / R.
template <int R, int I, bool WIDE>
__device__ __forceinline__ void products(const FewArgs& a, const float* xs, int64_t item,
                                         float (&sums)[R * I / 32]) {
    const int lane = threadIdx.x & 31, dp = padded(a.dim);
    const float* w[I];
#pragma unroll
    for (int i = 0; i < I; ++i) w[i] = a.w + min(item + i, a.items - 1) * a.ldw;
    float acc[R * I / 32][32];
#pragma unroll
    for (int q = 0; q < R * I / 32; ++q)
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[q][i] = 0.0f;
    float next[I][4];
#pragma unroll
    for (int i = 0; i < I; ++i) load_four<WIDE>(w[i], 0, a.dim, next[i]);
    for (int k = 0; k < a.dim; k += 128) {
        float v[I][4];
#pragma unroll
        for (int i = 0; i < I; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][e] = next[i][e];
            load_four<WIDE>(w[i], k + 128, a.dim, next[i]);
        }
#pragma unroll
        for (int t = 0; t < R; ++t) {
            float x[4];
            if constexpr (WIDE) {
                const float4 f = *reinterpret_cast<const float4*>(xs + t * dp + k + 4 * lane);
                x[0] = f.x, x[1] = f.y, x[2] = f.z, x[3] = f.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = xs[t * dp + k + lane + 32 * e];
            }
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[(i * R + t) / 32][(i * R + t) % 32] =
                        fmaf(v[i][e], x[e], acc[(i * R + t) / 32][(i * R + t) % 32]);
        }
    }
#pragma unroll
    for (int q = 0; q < R * I / 32; ++q) sums[q] = sum_across(acc[q]);
}

// An item's bias in powers of two (a finite one stays one); -inf: not in the softmax.
__device__ __forceinline__ float bias_of(const FewArgs& a, int64_t item) {
    if (item >= a.items) return -INFINITY;
    const float b = a.bias ? __ldg(a.bias + item) : 0.0f;
    return isfinite(b) ? fminf(fmaxf(b * kLog2e, -3.402823466e38f), 3.402823466e38f) : b;
}

__device__ __forceinline__ void join(float& m, float& s, float pm, float ps) {
    const float nm = fmaxf(m, pm), ref = nm == -INFINITY ? 0.0f : nm;
    s = s * exp2f(m - ref) + ps * exp2f(pm - ref);
    m = nm;
}

constexpr int kStatThreads = 512;

// The statistics of the rows over a block's items, each row's target left out.
template <int R, int I, bool WIDE>
__global__ void __launch_bounds__(kStatThreads) few_stats_kernel(const FewArgs a) {
    constexpr int kWarps = kStatThreads / 32;
    extern __shared__ float4 few_smem[];
    __shared__ float2 sh[kWarps][R];
    float* xs = reinterpret_cast<float*>(few_smem);
    next_early();
    wait_before();
    fill_rows(a, xs, R, false);
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane % R;
    const int64_t y = t < a.rows ? a.targets[t] : -1;
    float m = -INFINITY, s = 0.0f;
    for (int64_t item = ((int64_t)blockIdx.x * kWarps + warp) * I; item < a.items;
         item += (int64_t)gridDim.x * kWarps * I) {
        float dots[R * I / 32];
        products<R, I, WIDE>(a, xs, item, dots);
#pragma unroll
        for (int q = 0; q < R * I / 32; ++q) {
            const int64_t j = item + (32 * q + lane) / R;
            const float b = bias_of(a, j);
            if (b != -INFINITY && j != y) join(m, s, fmaf(dots[q], a.k2, b), 1.0f);
        }
    }
#pragma unroll
    for (int bit = R; bit < 32; bit <<= 1) {
        const float pm = __shfl_xor_sync(0xffffffffu, m, bit);
        const float ps = __shfl_xor_sync(0xffffffffu, s, bit);
        // (both lanes add the same two in the same order)
        float lm = lane & bit ? pm : m, ls = lane & bit ? ps : s;
        join(lm, ls, lane & bit ? m : pm, lane & bit ? s : ps);
        m = lm, s = ls;
    }
    if (lane < R) sh[warp][lane] = make_float2(m, s);
    __syncthreads();
    if (threadIdx.x < a.rows) {
        for (int i = 1; i < kWarps; ++i) join(m, s, sh[i][threadIdx.x].x, sh[i][threadIdx.x].y);
        a.part[blockIdx.x * a.part_rows + threadIdx.x] = make_float2(m, s);
    }
}

// G of the items [item][R], as the columns' kernel reads it; zeros for masked items.
template <int R, int I, bool WIDE>
__global__ void __launch_bounds__(kStatThreads) few_softmax_kernel(const FewArgs a) {
    constexpr int kWarps = kStatThreads / 32;
    extern __shared__ float4 few_smem[];
    float* xs = reinterpret_cast<float*>(few_smem);
    next_early();
    wait_before();
    fill_rows(a, xs, R, true);
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    GradRow gr{0.0f, 0.0f, 0.0f, -1};
    if (lane % R < a.rows) gr = a.row[lane % R];
    for (int64_t item = ((int64_t)blockIdx.x * kWarps + warp) * I; item < a.items;
         item += (int64_t)gridDim.x * kWarps * I) {
        float dots[R * I / 32];
        products<R, I, WIDE>(a, xs, item, dots);
#pragma unroll
        for (int q = 0; q < R * I / 32; ++q) {
            const int64_t j = item + (32 * q + lane) / R;
            const float bias = bias_of(a, j);
            float v = 0.0f;
            if (bias != -INFINITY && (gr.coef != 0.0f || gr.hit != 0.0f))
                v = j + a.item0 == gr.y ? gr.hit : gr.coef * exp2f(fmaf(dots[q], a.k2, bias) - gr.m);
            if (j < a.items) a.g[j * R + lane % R] = v;
        }
    }
}

constexpr int kMostThreads = 512;

// dx and dw from G: a thread owns columns, of dx over all of its group's items, which go
// by in runs of U; the next run's loads are under way while one is worked on.  A block
// has as many groups of threads as fit.  Two columns an instruction, G twice in shared
// memory for them: a thread's 128 FMAs of a run are 64.
template <int R, int U>
__global__ void __launch_bounds__(kMostThreads, 1) few_columns_kernel(const FewArgs a, int width) {
    extern __shared__ float4 few_smem[];
    __shared__ ulonglong2 gs[kMostThreads / 32][32];
    static_assert(R * U == 64, "a run's G is two entries a lane");
    next_early();
    wait_before();
    const int group = threadIdx.x / width, groups = blockDim.x / width;
    const int k0 = threadIdx.x - group * width, k1 = k0 + width, lane = threadIdx.x & 31;
    const bool in0 = k0 < a.dim, in1 = k1 < a.dim;
    ulonglong2* g = gs[threadIdx.x >> 5];
    uint64_t x[R], dx[R];
#pragma unroll
    for (int t = 0; t < R; ++t) {
        const bool row = t < a.rows && a.targets[t] != a.ignore_index;
        const float* p = a.x + t * a.ldx;
        x[t] = f2_pack(row && in0 ? p[k0] : 0.0f, row && in1 ? p[k1] : 0.0f);
        dx[t] = f2_pack(0.0f, 0.0f);
    }
    float next[U][2], bias = 0.0f;
    float2 next_g;
    auto fetch = [&](int64_t first) {
        const float* p = a.w + first * a.ldw + k0;
        const int here = (int)min((int64_t)U, a.items - first);
        if (here == U) {
#pragma unroll
            for (int i = 0; i < U; ++i, p += a.ldw) {
                next[i][0] = in0 ? __ldg(p) : 0.0f;
                next[i][1] = in1 ? __ldg(p + width) : 0.0f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i, p += a.ldw) {
                next[i][0] = in0 && i < here ? __ldg(p) : 0.0f;
                next[i][1] = in1 && i < here ? __ldg(p + width) : 0.0f;
            }
        }
        next_g = 2 * lane / R < here ? __ldg(reinterpret_cast<const float2*>(a.g + first * R) + lane)
                                     : make_float2(0.0f, 0.0f);
        if (a.bias && lane < U && lane < here) bias = __ldg(a.bias + first + lane);
    };
    const int64_t step = (int64_t)gridDim.x * groups * U;
    int64_t item = ((int64_t)blockIdx.x * groups + group) * U;
    fetch(item);
    for (; item < a.items; item += step) {
        uint64_t w[U];
#pragma unroll
        for (int i = 0; i < U; ++i) w[i] = f2_pack(next[i][0], next[i][1]);
        if (a.bias) {
            // (a masked item's vector may hold anything)
            const uint32_t masked = __ballot_sync(0xffffffffu, bias == -INFINITY);
#pragma unroll
            for (int i = 0; i < U; ++i) w[i] = masked >> i & 1 ? 0ull : w[i];
        }
        __syncwarp();
        g[lane] = make_ulonglong2(f2_pack(next_g.x, next_g.x), f2_pack(next_g.y, next_g.y));
        __syncwarp();
        fetch(item + step);
        float* o = a.dw + item * a.lddw + k0;
        const int here = (int)min((int64_t)U, a.items - item);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            uint64_t d = f2_pack(0.0f, 0.0f);
#pragma unroll
            for (int t = 0; t < R; t += 2) {
                const ulonglong2 f = g[(i * R + t) / 2];
                dx[t] = f2_fma(f.x, w[i], dx[t]);
                dx[t + 1] = f2_fma(f.y, w[i], dx[t + 1]);
                d = f2_fma(f.x, x[t], d);
                d = f2_fma(f.y, x[t + 1], d);
            }
            if (a.dw && i < here) {
                float d0, d1;
                f2_unpack(d, d0, d1);
                if (in0) o[0] = a.scale * d0;
                if (in1) o[width] = a.scale * d1;
            }
            o += a.lddw;
        }
    }
    if (!a.slots) return;
    // the block's sums, group after group
    float* sum = reinterpret_cast<float*>(few_smem);
    for (int n = 0; n < groups; ++n) {
        if (group == n) {
#pragma unroll
            for (int t = 0; t < R; ++t) {
                if (t >= a.rows) break;
                float v[2];
                f2_unpack(dx[t], v[0], v[1]);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int k = c ? k1 : k0;
                    if (c ? !in1 : !in0) continue;
                    if (n > 0) v[c] += sum[t * a.dim + k];
                    if (n + 1 < groups)
                        sum[t * a.dim + k] = v[c];
                    else {
                        float* to = a.slots + blockIdx.x * a.slot_stride + t * a.ldslot + k;
                        *to = a.accumulate ? *to + v[c] : v[c];
                    }
                }
            }
        }
        __syncthreads();
    }
}

bool by_fours(const FewArgs& a) {
    return (reinterpret_cast<uintptr_t>(a.w) & 15u) == 0 && a.ldw % 4 == 0 && a.dim % 4 == 0;
}

template <typename... More>
cudaError_t few_launch(void (*kernel)(const FewArgs, More...), const FewArgs& a, int r, int blocks,
                       int threads, cudaStream_t st, More... more) {
    const size_t smem = (size_t)r * padded(a.dim) * 4;
    const cudaError_t e =
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             kFewRows * kFewDim * 4);
    if (e != cudaSuccess) return e;
    count_launches(1);
    return launch_early(kernel, blocks, threads, smem, st, a, more...);
}

}  // namespace

int few_rows_padded(int64_t rows) { return rows <= 8 ? 8 : 16; }

int few_blocks(int64_t items, const Device& dev) {
    return (int)std::min<int64_t>((items + 31) / 32, dev.sms);
}

cudaError_t launch_few_stats(const FewArgs& a, int blocks, cudaStream_t st) {
    const bool v = by_fours(a);
    return a.rows <= 8 ? few_launch(v ? few_stats_kernel<8, 4, true> : few_stats_kernel<8, 4, false>, a, 8,
                                    blocks, kStatThreads, st)
                       : few_launch(v ? few_stats_kernel<16, 4, true> : few_stats_kernel<16, 4, false>, a,
                                    16, blocks, kStatThreads, st);
}

cudaError_t launch_few_grads(const FewArgs& a, int blocks, cudaStream_t st) {
    const bool v = by_fours(a);
    const cudaError_t e =
        a.rows <= 8 ? few_launch(v ? few_softmax_kernel<8, 4, true> : few_softmax_kernel<8, 4, false>, a, 8,
                                 blocks, kStatThreads, st)
                    : few_launch(v ? few_softmax_kernel<16, 4, true> : few_softmax_kernel<16, 4, false>, a,
                                 16, blocks, kStatThreads, st);
    if (e != cudaSuccess) return e;
    const int width = (a.dim + 63) / 64 * 32;
    const int threads = kMostThreads / width * width;
    return a.rows <= 8 ? few_launch(few_columns_kernel<8, 8>, a, 8, blocks, threads, st, width)
                       : few_launch(few_columns_kernel<16, 4>, a, 16, blocks, threads, st, width);
}

}  // namespace head
}  // namespace pvs

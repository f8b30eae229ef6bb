// Distillation from a teacher's best logits (head.h): what it adds to the products of xent.cu.
//
//   p_k  = exp(c z_k) / sum_i exp(c z_i)           over the slots of a row's list
//   loss = sum_k p_k (ln p_k - l_k + lse),  G_j = g (q_j - sum_{k: id_k = j} p_k)
//
//   forward    lists, each row's ids in ascending order; their logits (of few rows in the
//              same launch), float32 products of
//              their own (the tensor cores cut each step's sum, and the teacher's items have
//              the largest logits); the product over all items, whose epilogue leaves the
//              listed ones out of the tiles' statistics; and the join, which adds them
//   backward   the product writes G = g q; the listed entries, of which there are few, are
//              written over it with what the forward pass kept, so that q_j - p_j is taken
//              once and from one pair of numbers
//
// Beside the products this costs `top` scattered rows of w a row forward, and `top` sectors of
// each part of G backward.  4,096 rows over 8,192 items of 768 in bf16, lists of 64, in us: lists 13,
// their logits 47 (403 MB of rows, out of the L2: 8.5 TB/s), the product 38 (as without lists), join 12;
// rows and copy 8, G 54, listed entries 11, both gradients 137.  2,048 over 200,000 of 1,024
// in f16, lists of 128: 24, 64 (537 MB), 490, 20; backward 2,700.  (Logits within the joining launch,
// 32 rows of w in flight an SM, took it to 100 and 294.)  It grows with the lists, whatever the
// product takes: the first with lists of 1,024 171, 598 (6.4 GB, 10.8 TB/s; issue at 68%, the
// L2 at 42%), 120 and 187.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <climits>

#include "distill.h"
#include "kernels.h"
#include "pvs_common.cuh"

namespace pvs {
namespace head {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float element(const void* p, int dtype, int64_t i) {
    if (dtype == PVS_F32) return static_cast<const float*>(p)[i];
    if (dtype == PVS_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

// A slot's scaled teacher logit; -inf: not in the list.  An id that is none of the items is in
// it (and makes the row NaN).
__device__ __forceinline__ float teacher_logit(const TopRows& r, int64_t at, int64_t id) {
    if (id == r.a.ignore_index) return -INFINITY;
    if (r.a.bias && id >= 0 && id < r.a.items && r.a.bias[id] == -INFINITY) return -INFINITY;
    return element(r.logits, r.dtype, at) * r.teacher_scale;
}

// ---- logits of the listed items ----------------------------------------------------------
constexpr int kDots = 4;                 // of a warp at once, their loads in flight together

__device__ __forceinline__ void add_pairs(int dtype, uint32_t u, uint32_t v, float& lo, float& hi) {
    if (dtype == PVS_BF16) {
        lo = fmaf(__uint_as_float(u << 16), __uint_as_float(v << 16), lo);
        hi = fmaf(__uint_as_float(u & 0xffff0000u), __uint_as_float(v & 0xffff0000u), hi);
    } else {
        const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&u));
        const float2 q = __half22float2(*reinterpret_cast<const __half2*>(&v));
        lo = fmaf(p.x, q.x, lo);
        hi = fmaf(p.y, q.y, hi);
    }
}

// Elements as they lie, so that no load waits for another's type.
template <int KIND>
__device__ __forceinline__ uint32_t raw_element(const void* p, int64_t i) {
    if constexpr (KIND == 2) return __float_as_uint(__ldg(static_cast<const float*>(p) + i));
    return __ldg(static_cast<const uint16_t*>(p) + i);
}
template <int KIND>
__device__ __forceinline__ float raw_value(uint32_t u, int dtype) {
    if constexpr (KIND == 2) return __uint_as_float(u);
    return dtype == PVS_BF16 ? __uint_as_float(u << 16) : __half2float(__ushort_as_half((uint16_t)u));
}

// A warp's: the logits of entries k0 .. k0 + 3 of a row's list.  KIND 0: 16-bit rows of whole, aligned
// eights; 1: other 16-bit rows; 2: float32.
template <int KIND>
__device__ __forceinline__ void top_dots(const TopDots& j, int64_t row, int k0, const int (&id)[kDots]) {
    const pvs_xent_args& a = j.r.a;
    const int lane = threadIdx.x & 31, top = j.r.top;
    if (id[0] == INT_MAX) return;        // (and so are those behind it)
    float lo[kDots] = {}, hi[kDots] = {};
    if constexpr (KIND == 0) {
        const uint4* x = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.x) + row * a.ldx);
        const uint4* w[kDots];
#pragma unroll
        for (int i = 0; i < kDots; ++i)
            w[i] = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.w) +
                                                  (int64_t)(id[i] == INT_MAX ? id[0] : id[i]) * a.ldw);
#pragma unroll 2
        for (int k = lane; k < a.dim / 8; k += 32) {
            uint4 v[kDots];
#pragma unroll
            for (int i = 0; i < kDots; ++i) v[i] = __ldg(w[i] + k);
            const uint4 p = __ldg(x + k);
#pragma unroll
            for (int i = 0; i < kDots; ++i) {
                add_pairs(a.dtype, p.x, v[i].x, lo[i], hi[i]);
                add_pairs(a.dtype, p.y, v[i].y, lo[i], hi[i]);
                add_pairs(a.dtype, p.z, v[i].z, lo[i], hi[i]);
                add_pairs(a.dtype, p.w, v[i].w, lo[i], hi[i]);
            }
        }
    } else {
        int64_t w[kDots];
#pragma unroll
        for (int i = 0; i < kDots; ++i) w[i] = (int64_t)(id[i] == INT_MAX ? id[0] : id[i]) * a.ldw;
#pragma unroll 4
        for (int k = lane; k < a.dim; k += 32) {
            const uint32_t x = raw_element<KIND>(a.x, row * a.ldx + k);
            uint32_t v[kDots];
#pragma unroll
            for (int i = 0; i < kDots; ++i) v[i] = raw_element<KIND>(a.w, w[i] + k);
#pragma unroll
            for (int i = 0; i < kDots; ++i)
                lo[i] = fmaf(raw_value<KIND>(x, a.dtype), raw_value<KIND>(v[i], a.dtype), lo[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kDots; ++i) {
        const float dot = warp_sum(lo[i] + hi[i]);
        if (lane != i || id[i] == INT_MAX) continue;
        float b = a.bias ? a.bias[id[i]] : 0.0f;
        if (isfinite(b)) b = fminf(fmaxf(b * kLog2e, -3.402823466e38f), 3.402823466e38f);
        j.dots[row * top + k0 + i] = fmaf(dot, j.k2, b);
    }
}

// Bound by the rows of w, `top` for each row of x.
template <int KIND>
__global__ void __launch_bounds__(256) top_dots_kernel(const TopDots j) {
    next_early();
    wait_before();
    const int top = j.r.top, quads = (top + kDots - 1) / kDots;
    const int64_t u = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t row = quotient_of(u, quads);
    if (row >= j.r.a.rows) return;
    const int k0 = (int)(u - row * quads) * kDots;
    int id[kDots];
#pragma unroll
    for (int i = 0; i < kDots; ++i) id[i] = k0 + i < top ? __ldg(j.list + row * top + k0 + i) : INT_MAX;
    top_dots<KIND>(j, row, k0, id);
}

// ---- lists ---------------------------------------------------------------------------
// A bitonic network of (id, slot) over the next power of two, 2^bits; a block takes whole rows, and
// with a KIND (one row a block then) its logits too.
template <int KIND>
__global__ void __launch_bounds__(512) top_lists_kernel(const TopLists a, int bits, int rows_bits,
                                                        const TopDots dots) {
    __shared__ unsigned long long keys[kMaxTop];
    next_early();
    wait_before();
    const TopRows& r = a.r;
    const int padded = 1 << bits, rows_here = 1 << rows_bits;
    const int64_t row0 = (int64_t)blockIdx.x << rows_bits;
    const int total = 1 << (bits + rows_bits);
    for (int i = threadIdx.x; i < total; i += blockDim.x) {
        const int64_t row = row0 + (i >> bits);
        const int k = i & (padded - 1);
        unsigned long long key = (unsigned long long)INT_MAX << 32 | 0xffffffffu;
        if (row < r.a.rows && k < r.top) {
            const int64_t id = r.ids[row * r.top + k];
            key = (unsigned long long)INT_MAX << 32 | (uint32_t)k;
            if (id >= 0 && id < r.a.items && teacher_logit(r, row * r.top + k, id) != -INFINITY)
                key = (unsigned long long)id << 32 | (uint32_t)k;
        }
        keys[i] = key;
    }
    for (int k = 1; k <= bits; ++k) {
        for (int j = k - 1; j >= 0; --j) {
            __syncthreads();
            for (int t = threadIdx.x; t < total / 2; t += blockDim.x) {
                const int i = (t >> j << (j + 1)) | (t & ((1 << j) - 1)), l = i + (1 << j);
                const unsigned long long x = keys[i], y = keys[l];
                if ((x > y) == ((i & (padded - 1) & (1 << k)) == 0)) {
                    keys[i] = y;
                    keys[l] = x;
                }
            }
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < total; i += blockDim.x) {
        const int64_t row = row0 + (i >> bits);
        const int k = i & (padded - 1);
        if (row < r.a.rows && k < r.top) {
            a.list[row * r.top + k] = (int)(keys[i] >> 32);
            a.slot[row * r.top + k] = (uint16_t)keys[i];
        }
    }
    if constexpr (KIND >= 0) {
        for (int k0 = (threadIdx.x >> 5) * kDots; k0 < r.top; k0 += (blockDim.x >> 5) * kDots) {
            int id[kDots];
#pragma unroll
            for (int i = 0; i < kDots; ++i) id[i] = k0 + i < r.top ? (int)(keys[k0 + i] >> 32) : INT_MAX;
            top_dots<KIND>(dots, row0, k0, id);
        }
    }
    // where each tile of items begins in each row's list: the row first, so that neighbours write
    // neighbours
    const int in = threadIdx.x & (rows_here - 1);
    const int64_t row = row0 + in;
    if (row >= r.a.rows) return;
    const unsigned long long* mine = keys + (in << bits);
    uint16_t* out = a.first + row;
    for (int q = threadIdx.x >> rows_bits; q < a.tiles; q += blockDim.x >> rows_bits) {
        const int piece = q / a.piece_tiles;
        const int64_t start = piece * a.piece + (int64_t)(q - piece * a.piece_tiles) * a.tile;
        const unsigned long long from = (unsigned long long)start << 32;
        int lo = 0;
        for (int n = r.top; n > 0;) {
            const int half = n >> 1;
            const bool right = mine[lo + half] < from;
            lo = right ? lo + half + 1 : lo;
            n = right ? n - half - 1 : half;
        }
        out[q * r.a.rows] = (uint16_t)lo;
    }
}

// ---- join ----------------------------------------------------------------------------
__device__ __forceinline__ void join(float& m, float& s, float2 p) {
    const float nm = fmaxf(m, p.x), ref = nm == -INFINITY ? 0.0f : nm;
    s = s * exp2f(m - ref) + p.y * exp2f(p.x - ref);
    m = nm;
}

// R rows a block of eight warps: their tiles' statistics together, then a warp to a row.
template <int R>
__global__ void __launch_bounds__(256) top_join_kernel(const TopJoin j) {
    constexpr int kLanes = 256 / R;
    extern __shared__ float top_smem[];
    __shared__ float2 sh[kLanes][R];
    next_early();
    wait_before();
    const TopRows& r = j.r;
    const pvs_xent_args& a = r.a;
    const int top = r.top;
    const int64_t row0 = (int64_t)blockIdx.x * R;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    {
        const int c = threadIdx.x % R, l = threadIdx.x / R;
        float m = -INFINITY, s = 0.0f;
        if (row0 + c < a.rows) {
#pragma unroll 4
            for (int64_t i = l; i < j.n; i += kLanes) join(m, s, j.part[i * a.rows + row0 + c]);
        }
        sh[l][c] = make_float2(m, s);
        // joined in a fixed order
        for (int w = kLanes / 2; w > 0; w >>= 1) {
            __syncthreads();
            if (l < w) {
                join(m, s, sh[l + w][c]);
                sh[l][c] = make_float2(m, s);
            }
        }
        __syncthreads();
    }
    for (int c = warp; c < R; c += 8) {
        const int64_t row = row0 + c;
        if (row >= a.rows) continue;
        float* t = top_smem + 3 * c * top;           // logits of the listed items, in powers of two
        float* p = t + top;                          // the teacher's, then their shares
        int* id = reinterpret_cast<int*>(p + top);
        float m = sh[0][c].x, s = sh[0][c].y;
        float* hits = j.hits + row * top;
        // ids that are no items, and slots that are not in the list
        float zmax = -INFINITY, zsum = 0.0f;
        bool bad = false;
        int n = 0;
        for (int k = lane; k < top; k += 32) {
            const int slot = j.slot[row * top + k];
            const int64_t raw = r.ids[row * top + slot];
            const float z = teacher_logit(r, row * top + slot, raw);
            p[k] = z;
            id[k] = j.list[row * top + k];
            if (z == -INFINITY) {
                hits[slot] = kNoHit;
                continue;
            }
            if (id[k] == INT_MAX) {
                bad = true;
            } else {
                t[k] = j.dots[row * top + k];
            }
            zmax = fmaxf(zmax, z);
            ++n;
        }
        n = __reduce_add_sync(0xffffffffu, n);
        bad = __any_sync(0xffffffffu, bad);
        zmax = warp_max(zmax);
        __syncwarp();
        const float nan = __int_as_float(0x7fffffff);
        if (n == 0 || bad) {
            if (lane == 0) {
                j.loss[row] = n == 0 ? 0.0f : nan;
                j.stats[row] = n == 0 ? make_float4(-INFINITY, 0.0f, 0.0f, -INFINITY)
                                      : make_float4(m, nan, 0.0f, -INFINITY);
            }
            for (int k = lane; k < top && n > 0; k += 32)
                if (p[k] != -INFINITY) hits[j.slot[row * top + k]] = nan;
            continue;
        }
        // (the listed items come first: n of them)
        float tm = m;
        for (int k = lane; k < n; k += 32) {
            const float e = expf(p[k] - zmax);
            zsum += e;
            if (k == 0 || id[k - 1] != id[k]) tm = fmaxf(tm, t[k]);
        }
        zsum = warp_sum(zsum);
        const float log_sum = logf(zsum);
        if (j.apart) {
            tm = warp_max(tm);
            const float ref = tm == -INFINITY ? 0.0f : tm;
            float ssum = 0.0f;
            for (int k = lane; k < n; k += 32)
                if (k == 0 || id[k - 1] != id[k]) ssum += exp2f(t[k] - ref);
            ssum = warp_sum(ssum);
            s = s * exp2f(m - ref) + ssum;
            m = tm;
        }
        // (every logit is -inf: no softmax, and not the mark of a row without a list)
        if (m == -INFINITY) s = nan;
        const float log_s = logf(s);
        float loss = 0.0f;
        for (int k = lane; k < n; k += 32) {
            // the run of slots that name the same item (each slot walks all of it: 4,096 lists that
            // name one item 64 times take 129 us for 96, 1,024 times 8.2 ms for 1.0)
            int first = k, last = k;
            while (first > 0 && id[first - 1] == id[k]) --first;
            while (last + 1 < n && id[last + 1] == id[k]) ++last;
            const float pk = expf(p[k] - zmax) / zsum;
            float share = pk;
            if (first < last) {
                share = 0.0f;
                for (int i = first; i <= last; ++i) share += expf(p[i] - zmax) / zsum;
            }
            const float d = t[first] - m;
            if (pk > 0.0f || pk != pk)
                loss += pk * ((p[k] - zmax) - log_sum - fmaf(d, kLn2, -log_s));
            hits[j.slot[row * top + k]] = exp2f(d) / s - share;
        }
        loss = warp_sum(loss);
        if (lane == 0) {
            j.loss[row] = loss;
            j.stats[row] = make_float4(m, s, 0.0f, -INFINITY);
        }
    }
}

// ---- backward --------------------------------------------------------------------------
__global__ void __launch_bounds__(256) top_scatter_kernel(const TopScatter a) {
    next_early();
    wait_before();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.rows * a.top) return;
    const int64_t id = a.ids[i] - a.v0;
    const float hit = a.hits[i];
    if (id < 0 || id >= a.n || hit == kNoHit) return;
    const int64_t row = quotient_of(i, a.top);
    float v = a.grad[row] * (a.up ? *a.up : 1.0f) * hit;
    if (a.few) {
        a.few[id * a.few_rows + row] = v;
        return;
    }
    // in parts as the product writes them: cut (f16: rounded) but for the last, which is rounded
    uint16_t* o = a.g + row * a.ldg + id;
    for (int part = 0; part < a.parts; ++part, o += a.g_part) {
        if (a.f16) {
            const __half h = __float2half_rn(v);
            const float f = __half2float(h);
            v = isfinite(f) ? v - f : 0.0f;
            *o = __half_as_ushort(h);
        } else if (part + 1 < a.parts) {
            uint32_t u = __float_as_uint(v) & 0xffff0000u;
            if (v != v) u |= 0x00400000u;   // a NaN stays one
            v = isfinite(v) ? v - __uint_as_float(u) : 0.0f;
            *o = (uint16_t)(u >> 16);
        } else {
            *o = __bfloat16_as_ushort(__float2bfloat16_rn(v));
        }
    }
}

template <int R>
cudaError_t join_launch(const TopJoin& a, cudaStream_t st) {
    const size_t smem = (size_t)R * a.r.top * 12;
    const cudaError_t e = raise_smem_limit((const void*)top_join_kernel<R>, R * kMaxTop * 12);
    if (e != cudaSuccess) return e;
    count_launches(1);
    return launch_early(top_join_kernel<R>, (a.r.a.rows + R - 1) / R, 256, smem, st, a);
}

}  // namespace

cudaError_t launch_top_lists(const TopLists& a, const TopDots& dots, cudaStream_t st) {
    int bits = 1;
    while (1 << bits < a.r.top) ++bits;
    // as many rows a block as 256 threads sort, but a block for every SM first
    int rows_bits = 0;
    while (rows_bits < 5 && bits + rows_bits < 9 && a.r.a.rows >> (rows_bits + 1) >= 256) ++rows_bits;
    const int64_t blocks = ((a.r.a.rows - 1) >> rows_bits) + 1;
    const int threads = bits == 10 ? 512 : 256;
    const int kind = a.r.a.dtype == PVS_F32 ? 2 : dots.wide ? 0 : 1;
    // a short list's logits in the same launch, where that has a block for each row anyway (four
    // entries a warp at once, and four times at most)
    const bool together = rows_bits == 0 && a.r.top <= 16 * kDots * 2;
    count_launches(1);
    cudaError_t e = launch_early(!together   ? top_lists_kernel<-1>
                                 : kind == 0 ? top_lists_kernel<0>
                                 : kind == 1 ? top_lists_kernel<1>
                                             : top_lists_kernel<2>,
                                 blocks, threads, 0, st, a, bits, rows_bits, dots);
    if (e != cudaSuccess || together) return e;
    const int64_t warps = a.r.a.rows * ((a.r.top + kDots - 1) / kDots);
    if (warps > (int64_t)8 * 0x7fffffff) return cudaErrorInvalidValue;
    count_launches(1);
    return launch_early(kind == 0 ? top_dots_kernel<0> : kind == 1 ? top_dots_kernel<1> : top_dots_kernel<2>,
                        (warps + 7) / 8, 256, 0, st, dots);
}

cudaError_t launch_top_join(const TopJoin& a, const Device& dev, cudaStream_t st) {
    // eight rows' statistics share their sectors, where that leaves every SM some blocks
    if (a.r.a.rows >= 4 * dev.sms) return join_launch<8>(a, st);
    return join_launch<1>(a, st);
}

cudaError_t launch_top_scatter(const TopScatter& a, cudaStream_t st) {
    const int64_t blocks = (a.rows * a.top + 255) / 256;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    count_launches(1);
    return launch_early(top_scatter_kernel, blocks, 256, 0, st, a);
}

}  // namespace head
}  // namespace pvs

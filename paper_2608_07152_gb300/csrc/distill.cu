// Distillation from a teacher's best logits (head.h): what it adds to the products of xent.cu.
//
//   p_k  = exp(c z_k) / sum_i exp(c z_i)           over the slots of a row's list
//   loss = sum_k p_k (ln p_k - l_k + lse),  G_j = g (q_j - sum_{k: id_k = j} p_k)
//
//   forward    lists, each row's ids in ascending order; the product, whose epilogue leaves
//              the listed items out of the tiles' statistics; and the join, which adds them
//              with logits that are float32 products of their own (the tensor cores cut each
//              step's sum, and the teacher's items have the largest logits)
//   backward   the product writes G = g q; the listed entries, of which there are few, are
//              written over it with what the forward pass kept, so that q_j - p_j is taken
//              once and from one pair of numbers
//
// Beside the products this costs `top` scattered rows of w a row forward, and `top` sectors of
// each part of G backward.
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

// ---- lists ---------------------------------------------------------------------------
// A bitonic network of (id, slot) over the next power of two, padded / 2 threads to a row.
__global__ void __launch_bounds__(512) top_lists_kernel(const TopLists a, int padded, int rows_here) {
    __shared__ unsigned long long keys[kMaxTop];
    next_early();
    wait_before();
    const TopRows& r = a.r;
    const int64_t row0 = (int64_t)blockIdx.x * rows_here;
    const int total = rows_here * padded;
    for (int i = threadIdx.x; i < total; i += blockDim.x) {
        const int64_t row = row0 + i / padded;
        const int k = i % padded;
        unsigned long long key = (unsigned long long)INT_MAX << 32 | 0xffffffffu;
        if (row < r.a.rows && k < r.top) {
            const int64_t id = r.ids[row * r.top + k];
            key = (unsigned long long)INT_MAX << 32 | (uint32_t)k;
            if (id >= 0 && id < r.a.items && teacher_logit(r, row * r.top + k, id) != -INFINITY)
                key = (unsigned long long)id << 32 | (uint32_t)k;
        }
        keys[i] = key;
    }
    for (int k = 2; k <= padded; k <<= 1) {
        for (int j = k >> 1; j > 0; j >>= 1) {
            __syncthreads();
            for (int t = threadIdx.x; t < total / 2; t += blockDim.x) {
                const int i = (t / j) * 2 * j + t % j, l = i + j;
                const unsigned long long x = keys[i], y = keys[l];
                if ((x > y) == ((i % padded & k) == 0)) {
                    keys[i] = y;
                    keys[l] = x;
                }
            }
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < total; i += blockDim.x) {
        const int64_t row = row0 + i / padded;
        const int k = i % padded;
        if (row < r.a.rows && k < r.top) {
            a.list[row * r.top + k] = (int)(keys[i] >> 32);
            a.slot[row * r.top + k] = (uint16_t)keys[i];
        }
    }
    for (int64_t i = threadIdx.x; i < a.tiles * rows_here; i += blockDim.x) {
        const int in = (int)(i % rows_here);
        const int64_t q = i / rows_here, row = row0 + in;
        if (row >= r.a.rows) continue;
        const int64_t start = q / a.piece_tiles * a.piece + q % a.piece_tiles * a.tile;
        int lo = 0;
        for (int n = r.top; n > 0;) {
            const int half = n >> 1;
            if ((int64_t)(keys[in * padded + lo + half] >> 32) < start) {
                lo += half + 1;
                n -= half + 1;
            } else {
                n = half;
            }
        }
        a.first[q * r.a.rows + row] = (uint16_t)lo;
    }
}

// ---- join ----------------------------------------------------------------------------
__device__ __forceinline__ void join(float& m, float& s, float2 p) {
    const float nm = fmaxf(m, p.x), ref = nm == -INFINITY ? 0.0f : nm;
    s = s * exp2f(m - ref) + p.y * exp2f(p.x - ref);
    m = nm;
}

// A lane's part of <x_row, w_y>.
__device__ __forceinline__ float dot_part(const TopJoin& j, int64_t row, int64_t y) {
    const pvs_xent_args& a = j.r.a;
    float lo = 0.0f, hi = 0.0f;
    if (!j.wide) {
#pragma unroll 4
        for (int k = threadIdx.x & 31; k < a.dim; k += 32)
            lo = fmaf(element(a.x, a.dtype, row * a.ldx + k), element(a.w, a.dtype, y * a.ldw + k), lo);
        return lo;
    }
    const uint4* x = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.x) + row * a.ldx);
    const uint4* w = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.w) + y * a.ldw);
    auto add = [&](uint32_t u, uint32_t v) {
        if (a.dtype == PVS_BF16) {
            lo = fmaf(__uint_as_float(u << 16), __uint_as_float(v << 16), lo);
            hi = fmaf(__uint_as_float(u & 0xffff0000u), __uint_as_float(v & 0xffff0000u), hi);
        } else {
            const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&u));
            const float2 q = __half22float2(*reinterpret_cast<const __half2*>(&v));
            lo = fmaf(p.x, q.x, lo);
            hi = fmaf(p.y, q.y, hi);
        }
    };
#pragma unroll 4
    for (int k = threadIdx.x & 31; k < a.dim / 8; k += 32) {
        const uint4 u = __ldg(x + k), v = __ldg(w + k);
        add(u.x, v.x), add(u.y, v.y), add(u.z, v.z), add(u.w, v.w);
    }
    return lo + hi;
}

// R rows a block of eight warps, which share the products; then a warp to a row.
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
    float* ts = top_smem;                        // logits of the listed items, in powers of two
    float* ps = top_smem + R * top;              // their shares of the teacher's distribution
    int* ids = reinterpret_cast<int*>(ps + R * top);
    const int64_t row0 = (int64_t)blockIdx.x * R;
    {
        const int c = threadIdx.x % R, lane = threadIdx.x / R;
        float m = -INFINITY, s = 0.0f;
        if (row0 + c < a.rows) {
#pragma unroll 4
            for (int64_t i = lane; i < j.n; i += kLanes) join(m, s, j.part[i * a.rows + row0 + c]);
        }
        sh[lane][c] = make_float2(m, s);
    }
    for (int i = threadIdx.x; i < R * top; i += 256)
        ids[i] = row0 + i / top < a.rows ? j.list[row0 * top + i] : INT_MAX;
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = warp; i < R * top; i += 8) {
        if (ids[i] == INT_MAX) continue;         // (the same for the warp)
        float dot = 0.0f;
        if (i % top == 0 || ids[i - 1] != ids[i]) {
            dot = warp_sum(dot_part(j, row0 + i / top, ids[i]));
            if (lane == 0) {
                float b = a.bias ? a.bias[ids[i]] : 0.0f;
                if (isfinite(b)) b = fminf(fmaxf(b * kLog2e, -3.402823466e38f), 3.402823466e38f);
                ts[i] = fmaf(dot, j.k2, b);
            }
        }
    }
    // the tiles' statistics of a row, joined in a fixed order
    for (int w = kLanes / 2; w > 0; w >>= 1) {
        const int c = threadIdx.x % R, l = threadIdx.x / R;
        float2 v{};
        if (l < w) {
            v = sh[l][c];
            join(v.x, v.y, sh[l + w][c]);
        }
        __syncthreads();
        if (l < w) sh[l][c] = v;
        __syncthreads();
    }
    __syncthreads();
    for (int c = warp; c < R; c += 8) {
        const int64_t row = row0 + c;
        if (row >= a.rows) continue;
        const int* id = ids + c * top;
        float* t = ts + c * top;
        float* p = ps + c * top;
        float m = sh[0][c].x, s = sh[0][c].y;
        float* hits = j.hits + row * top;
        // the teacher's distribution; ids that are no items, and slots that are not in the list
        float zmax = -INFINITY, zsum = 0.0f;
        bool bad = false;
        int n = 0;
        for (int k = lane; k < top; k += 32) {
            const int slot = j.slot[row * top + k];
            const int64_t raw = r.ids[row * top + slot];
            const float z = teacher_logit(r, row * top + slot, raw);
            p[k] = z;
            if (z == -INFINITY) {
                hits[slot] = kNoHit;
                continue;
            }
            if (raw < 0 || raw >= a.items) bad = true;
            zmax = fmaxf(zmax, z);
            ++n;
        }
        n = __reduce_add_sync(0xffffffffu, n);
        bad = __any_sync(0xffffffffu, bad);
        zmax = warp_max(zmax);
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
        for (int k = lane; k < n; k += 32) zsum += expf(p[k] - zmax);
        zsum = warp_sum(zsum);
        const float log_sum = logf(zsum);
        if (j.apart) {
            float tm = m;
            for (int k = lane; k < n; k += 32)
                if (k == 0 || id[k - 1] != id[k]) tm = fmaxf(tm, t[k]);
            tm = warp_max(tm);
            const float ref = tm == -INFINITY ? 0.0f : tm;
            float ssum = 0.0f;
            for (int k = lane; k < n; k += 32)
                if (k == 0 || id[k - 1] != id[k]) ssum += exp2f(t[k] - ref);
            ssum = warp_sum(ssum);
            s = s * exp2f(m - ref) + ssum;
            m = tm;
        }
        __syncwarp();
        const float log_s = logf(s);
        float loss = 0.0f;
        for (int k = lane; k < n; k += 32) {
            // the run of slots that name the same item
            int first = k, last = k;
            while (first > 0 && id[first - 1] == id[k]) --first;
            while (last + 1 < n && id[last + 1] == id[k]) ++last;
            float share = 0.0f;
            for (int i = first; i <= last; ++i) share += expf(p[i] - zmax) / zsum;
            const float d = t[first] - m;
            const float pk = expf(p[k] - zmax) / zsum;
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
__global__ void __launch_bounds__(256) top_flags_kernel(const float4* __restrict__ stats, int64_t rows,
                                                        int64_t* __restrict__ flags) {
    next_early();
    wait_before();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows) return;
    const float4 s = stats[i];
    flags[i] = s.x == -INFINITY && s.y == 0.0f ? -1 : 0;
}

__global__ void __launch_bounds__(256) top_scatter_kernel(const TopScatter a) {
    next_early();
    wait_before();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.rows * a.top) return;
    const int64_t id = a.ids[i] - a.v0;
    const float hit = a.hits[i];
    if (id < 0 || id >= a.n || hit == kNoHit) return;
    const int64_t row = i / a.top;
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

cudaError_t launch_top_lists(const TopLists& a, cudaStream_t st) {
    int padded = 2;
    while (padded < a.r.top) padded *= 2;
    const int rows_here = std::max(1, 512 / padded);
    count_launches(1);
    return launch_early(top_lists_kernel, (a.r.a.rows + rows_here - 1) / rows_here,
                        std::max(256, padded / 2), 0, st, a, padded, rows_here);
}

cudaError_t launch_top_join(const TopJoin& a, const Device& dev, cudaStream_t st) {
    // eight rows' statistics share their sectors, where that leaves every SM some blocks
    if (a.r.a.rows >= 4 * dev.sms) return join_launch<8>(a, st);
    return join_launch<1>(a, st);
}

cudaError_t launch_top_flags(const float4* stats, int64_t rows, int64_t* flags, cudaStream_t st) {
    count_launches(1);
    return launch_early(top_flags_kernel, (rows + 255) / 256, 256, 0, st, stats, rows, flags);
}

cudaError_t launch_top_scatter(const TopScatter& a, cudaStream_t st) {
    const int64_t blocks = (a.rows * a.top + 255) / 256;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    count_launches(1);
    return launch_early(top_scatter_kernel, blocks, 256, 0, st, a);
}

}  // namespace head
}  // namespace pvs

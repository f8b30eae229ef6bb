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
#include "f32x2.cuh"
#include "head_gemm.h"
#include "kernels.h"
#include "pvs_common.cuh"

namespace pvs {
namespace head {
namespace {

template <int TYPE> struct Element;
template <> struct Element<PVS_BF16> {
    using T = uint16_t;
    static __device__ __forceinline__ float to(uint32_t x) { return __uint_as_float(x << 16); }
    static __device__ __forceinline__ uint32_t from(float x) {
        return __bfloat16_as_ushort(__float2bfloat16_rn(x));
    }
    static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
};
template <> struct Element<PVS_F16> {
    using T = uint16_t;
    static __device__ __forceinline__ float to(uint32_t x) {
        return __half2float(__ushort_as_half((uint16_t)x));
    }
    static __device__ __forceinline__ uint32_t from(float x) {
        return __half_as_ushort(__float2half_rn(x));
    }
    static __device__ __forceinline__ uint32_t pair(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
};
template <> struct Element<PVS_F32> {
    using T = uint32_t;
    static __device__ __forceinline__ float to(uint32_t x) { return __uint_as_float(x); }
    static __device__ __forceinline__ uint32_t from(float x) { return __float_as_uint(x); }
};

// N consecutive elements (8, aligned to their size, or 1).
template <int TYPE, int N>
__device__ __forceinline__ void load_elements(const void* p, int64_t at, float (&v)[N]) {
    using E = Element<TYPE>;
    if constexpr (N == 1) {
        v[0] = E::to(__ldg(static_cast<const typename E::T*>(p) + at));
    } else if constexpr (TYPE == PVS_F32) {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
        const float4 a = __ldg(q), b = __ldg(q + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
        v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = E::to((w[i >> 1] >> (16 * (i & 1))) & 0xffffu);
    }
}
template <int TYPE, int N>
__device__ __forceinline__ void store_elements(void* p, int64_t at, const float (&v)[N]) {
    using E = Element<TYPE>;
    if constexpr (N == 1) {
        static_cast<typename E::T*>(p)[at] = (typename E::T)E::from(v[0]);
    } else if constexpr (TYPE == PVS_F32) {
        float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
        q[0] = make_float4(v[0], v[1], v[2], v[3]);
        q[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = E::pair(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <int N>
__device__ __forceinline__ void load_codes(const int8_t* p, int64_t at, float (&v)[N]) {
    if constexpr (N == 1) {
        v[0] = (float)__ldg(p + at);
    } else {
        const uint2 a = __ldg(reinterpret_cast<const uint2*>(p + at));
        const uint32_t w[2] = {a.x ^ 0x80808080u, a.y ^ 0x80808080u};
        // the byte code + 128 under the exponent of 2^23 reads as 2^23 + 128 + code
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = __uint_as_float(__byte_perm(w[i >> 2], 0x4b000000u, 0x7440 | (i & 3))) - 8388736.0f;
    }
}

__device__ __forceinline__ float ex2_ftz(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rcp_ftz(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// 1 - Phi(|x|) of two values, and e = exp(-x^2 / 2): half of 1 - erf(z), z = |x| /
// sqrt(2), as a polynomial in t = 1 / (1 + p z) times exp(-z^2) (Abramowitz and
// Stegun 7.1.26, Hastings 1955: 1 - erf off by at most 1.5e-7).  For 16-bit results: with
// erff the activation took three quarters of the store's instructions; this is 8 an
// element, two elements an instruction where the operation has such a form.
__device__ __forceinline__ uint64_t upper_tail(float x0, float x1, float& a0, float& a1, float& e0,
                                               float& e1) {
    a0 = fabsf(x0);
    a1 = fabsf(x1);
    const uint64_t a = f2_pack(a0, a1);
    const float pz = 0.3275911f * 0.70710678118654752f;
    float d0, d1, q0, q1;
    f2_unpack(f2_fma(a, f2_pack(pz, pz), f2_pack(1.0f, 1.0f)), d0, d1);
    const float el = -0.5f * 1.4426950408889634f;
    f2_unpack(f2_mul(f2_mul(a, a), f2_pack(el, el)), q0, q1);
    e0 = ex2_ftz(q0);
    e1 = ex2_ftz(q1);
    const uint64_t t = f2_pack(rcp_ftz(d0), rcp_ftz(d1));
    auto two = [](float c) { return f2_pack(c, c); };
    uint64_t p = f2_fma(two(0.5f * 1.061405429f), t, two(0.5f * -1.453152027f));
    p = f2_fma(p, t, two(0.5f * 1.421413741f));
    p = f2_fma(p, t, two(0.5f * -0.284496736f));
    p = f2_fma(p, t, two(0.5f * 0.254829592f));
    return f2_mul(f2_mul(p, t), f2_pack(e0, e1));
}
// x Phi(x) = max(x, 0) - |x| (1 - Phi(|x|)): the negative side is the tail itself,
// without a difference from 1.
__device__ __forceinline__ void gelu2(float& x0, float& x1) {
    float a0, a1, e0, e1, y0, y1;
    const uint64_t h = upper_tail(x0, x1, a0, a1, e0, e1);
    f2_unpack(f2_fma(f2_pack(-a0, -a1), h, f2_pack(fmaxf(x0, 0.0f), fmaxf(x1, 0.0f))), y0, y1);
    // The tail is 0 at an infinity: -inf gives NaN as x Phi(x) does, and +inf has to stay
    // what it is; a NaN stays one through h.
    x0 = x0 == INFINITY ? x0 : y0;
    x1 = x1 == INFINITY ? x1 : y1;
}
__device__ __forceinline__ void slope2(float x0, float x1, float& s0, float& s1) {
    float a0, a1, e0, e1, h0, h1;
    f2_unpack(upper_tail(x0, x1, a0, a1, e0, e1), h0, h1);
    const float c = 0.39894228040143268f;
    s0 = (x0 < 0.0f ? h0 : 1.0f - h0) + (e0 == 0.0f ? 0.0f : x0 * (e0 * c));
    s1 = (x1 < 0.0f ? h1 : 1.0f - h1) + (e1 == 0.0f ? 0.0f : x1 * (e1 * c));
}
// float32 results take the functions in full: the polynomial's error is 3e-6 of the tail at
// x = -2 and 1.6e-3 at -5, which 16 bits do not show and 24 do.  32,768 x 1,536: the store
// takes 100 us, 67 with the polynomial; the gradient 118 and 82.
__device__ __forceinline__ float gelu_full(float x) {
    return 0.5f * x * erfcf(x * -0.70710678118654752f);
}
__device__ __forceinline__ float slope_full(float x) {
    return fmaf(x, expf(-0.5f * x * x) * 0.39894228040143268f, 0.5f * erfcf(x * -0.70710678118654752f));
}
template <int TYPE, int N>
__device__ __forceinline__ void gelu_all(float (&v)[N]) {
    if constexpr (TYPE == PVS_F32) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = gelu_full(v[k]);
    } else if constexpr (N == 1) {
        float other = 0.0f;
        gelu2(v[0], other);
    } else {
#pragma unroll
        for (int k = 0; k < N; k += 2) gelu2(v[k], v[k + 1]);
    }
}
template <int TYPE, int N>
__device__ __forceinline__ void times_slope(float (&z)[N], const float (&g)[N]) {
    if constexpr (TYPE == PVS_F32) {
#pragma unroll
        for (int k = 0; k < N; ++k) z[k] = g[k] * slope_full(z[k]);
    } else {
        float s[N + 1];
#pragma unroll
        for (int k = 0; k < N; k += 2) slope2(z[k], N == 1 ? 0.0f : z[k + 1], s[k], s[k + 1]);
#pragma unroll
        for (int k = 0; k < N; ++k) z[k] = g[k] * s[k];
    }
}

// Codes of N values against scale s (r = RN(1 / s)), a byte each in the low bits
// of c.  v r is within 2^-15 of v / s, so a product further than 2^-14 from every
// half-integer rounds as the quotient does; a piece with a nearer one (one warp in
// thirty) divides.  The sum with 1.5 2^23 leaves the code in its low byte.
template <int N>
__device__ __forceinline__ void codes_of(const float (&v)[N], float s, float r, bool fast,
                                         uint32_t (&c)[N]) {
    const float k = 12582912.0f;
    float far = 0.0f;
    if constexpr (N == 1) {
        const float t = v[0] * r, f = t + k;
        far = fabsf(t - (f - k));
        c[0] = __float_as_uint(f);
    } else {
        const uint64_t r2 = f2_pack(r, r), k2 = f2_pack(k, k), m2 = f2_pack(-k, -k);
        const uint64_t minus = f2_pack(-1.0f, -1.0f);
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const uint64_t t = f2_mul(f2_pack(v[i], v[i + 1]), r2), f = f2_add(t, k2);
            float d0, d1, f0, f1;
            f2_unpack(f2_fma(f2_add(f, m2), minus, t), d0, d1);
            f2_unpack(f, f0, f1);
            far = fmaxf(far, fmaxf(fabsf(d0), fabsf(d1)));
            c[i] = __float_as_uint(f0);
            c[i + 1] = __float_as_uint(f1);
        }
    }
    if (!fast || !(far < 0.5f - 0x1p-14f)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            c[i] = (uint32_t)(int)fminf(fmaxf(roundf(__fdiv_rn(v[i], s)), -127.0f), 127.0f);
    }
}

// TPR threads per row hold it in registers: read once, the maximum, the codes, the
// activation.  N elements (8, or 1 where nothing is aligned) make a piece; a thread
// holds NV pieces of 8 elements' worth.  FLAT: rows without gaps of any width are cut
// into the aligned eights of the whole matrix: a row's first and last piece may hold
// elements of its neighbours, which are left out (aligned rows took 107 us that way
// where they take 74 without its checks; element by element, 40,000 rows of 1,001 took
// 271 us with the load, in eights 92).
// 32,768 rows of 1,536 in bf16 with GELU: 45 us, 5.6 TB/s (issue 67%).
template <int TYPE, int N, int NV, int TPR, bool FLAT>
__global__ void __launch_bounds__(256) ckpt_store_kernel(const void* __restrict__ x, int64_t ldx,
                                                         int64_t rows, int cols, int act,
                                                         int8_t* __restrict__ codes, int64_t ldc,
                                                         float* __restrict__ scales,
                                                         void* __restrict__ y, int64_t ldy) {
    next_early();
    wait_before();
    constexpr int kPieces = NV * 8 / N;
    constexpr int kRows = 256 / TPR;
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    const bool live = row < rows;
    // (the three leading dimensions are the width then)
    const int before = FLAT ? (int)(row * ldx & 7) : 0;
    const int pieces = (before + cols + N - 1) / N;
    float v[kPieces][N];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int j = i * TPR + lane, e = j * N - before;    // the piece's first element
        if (live && j < pieces && (!FLAT || (e >= 0 && e + N <= cols))) {
            load_elements<TYPE, N>(x, row * ldx + e, v[i]);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float one[1] = {0.0f};
                if (FLAT && live && e + k >= 0 && e + k < cols)
                    load_elements<TYPE, 1>(x, row * ldx + e + k, one);
                v[i][k] = one[0];
            }
        }
    }
    // the largest magnitude by its bits: infinities and NaN are above every number
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) bits = max(bits, __float_as_uint(v[i][k]) & 0x7fffffffu);
    bits = __reduce_max_sync(0xffffffffu, bits);
    if constexpr (TPR > 32) {
        __shared__ uint32_t tops[TPR / 32];
        if (lane % 32 == 0) tops[lane / 32] = bits;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TPR / 32; ++i) bits = max(bits, tops[i]);
    }
    if (!live) return;
    const bool finite = bits < 0x7f800000u;
    float s = bits == 0u ? 1.0f : __fmul_rn(__uint_as_float(bits), 1.0f / 127.0f);
    if (s == 0.0f) s = __uint_as_float(1u);
    const float r = __fdiv_rn(1.0f, s);
    const bool fast = s >= kFastScaleMin;
    if (lane == 0) scales[row] = finite ? s : __int_as_float(0x7fffffff);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int j = i * TPR + lane, e = j * N - before;
        if (j >= pieces) break;
        const bool whole = !FLAT || (e >= 0 && e + N <= cols);
        uint32_t c[N];
        if (finite) {
            codes_of<N>(v[i], s, r, fast, c);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) c[k] = 0;
        }
        int8_t* out = codes + row * ldc + e;
        if constexpr (N == 1) {
            *out = (int8_t)c[0];
        } else if (!whole) {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (e + k >= 0 && e + k < cols) out[k] = (int8_t)c[k];
        } else {
            uint32_t w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                w[h] = __byte_perm(__byte_perm(c[4 * h], c[4 * h + 1], 0x0040),
                                   __byte_perm(c[4 * h + 2], c[4 * h + 3], 0x0040), 0x5410);
            *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
        }
        if (act == PVS_ACT_GELU) {
            gelu_all<TYPE, N>(v[i]);
            if (whole) {
                store_elements<TYPE, N>(y, row * ldy + e, v[i]);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float one[1] = {v[i][k]};
                    if (e + k >= 0 && e + k < cols) store_elements<TYPE, 1>(y, row * ldy + e + k, one);
                }
            }
        }
    }
}

// What the codes stand for (DY: times dy act').  A block takes `per_block` rows;
// a thread's pieces of N elements run over them.  n / pieces by a product:
// m = floor(2^40 / pieces) + 1 is exact for n < 2^23 and pieces < 2^16.
// 32,768 x 1,536 in bf16: 29 us (5.2 TB/s), with dy act' 55 us (4.6 TB/s; issue 70%: the
// error function and the exponential).
template <int TYPE, int N, bool DY>
__global__ void __launch_bounds__(256) ckpt_load_kernel(const void* __restrict__ dy, int64_t lddy,
                                                        const int8_t* __restrict__ codes,
                                                        int64_t ldc,
                                                        const float* __restrict__ scales,
                                                        int64_t rows, int cols, int per_block,
                                                        uint64_t m, void* __restrict__ out,
                                                        int64_t ldo) {
    next_early();
    wait_before();
    const int pieces = cols / N;
    const int64_t row0 = (int64_t)blockIdx.x * per_block;
    const int here = (int)min((int64_t)per_block, rows - row0);
    const uint32_t total = (uint32_t)(here * pieces);
    constexpr int kAhead = N == 1 ? 8 : 2;
    for (uint32_t i0 = threadIdx.x; i0 < total; i0 += 256 * kAhead) {
        float z[kAhead][N], g[kAhead][N], s[kAhead];
        int64_t row[kAhead];
        int col[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            // (past the end: the first piece again, not stored)
            const uint32_t i = i0 + a * 256 < total ? i0 + a * 256 : i0;
            const uint32_t r = (uint32_t)((i * m) >> 40);
            row[a] = row0 + r;
            col[a] = (int)(i - r * (uint32_t)pieces) * N;
            load_codes<N>(codes, row[a] * ldc + col[a], z[a]);
            if constexpr (DY) load_elements<TYPE, N>(dy, row[a] * lddy + col[a], g[a]);
            s[a] = __ldg(scales + row[a]);
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (i0 + a * 256 >= total) break;
#pragma unroll
            for (int k = 0; k < N; ++k) z[a][k] *= s[a];
            if constexpr (DY) times_slope<TYPE, N>(z[a], g[a]);
            store_elements<TYPE, N>(out, row[a] * ldo + col[a], z[a]);
        }
    }
}

// The same for matrices without gaps of any width: the aligned eights of the whole
// matrix, which may hold the end of one row and the start of the next (rows are 8
// elements long at least).  With dy, and the weight's product (of one part) after it, 32,768 rows
// of 1,001 took 138 us this way and 367 element by element.
template <int TYPE, bool DY>
__global__ void __launch_bounds__(256) ckpt_load_flat_kernel(const void* __restrict__ dy,
                                                             const int8_t* __restrict__ codes,
                                                             const float* __restrict__ scales,
                                                             int64_t total, int cols, uint64_t m,
                                                             void* __restrict__ out) {
    next_early();
    wait_before();
    constexpr int kAhead = 2;
    const int64_t e0 = (int64_t)blockIdx.x * (256 * 8 * kAhead);
    const int64_t row0 = e0 / cols;
    const uint32_t in_row = (uint32_t)(e0 - row0 * cols);
    float z[kAhead][8], g[kAhead][8], s[kAhead], next[kAhead];
    uint32_t left[kAhead];                       // elements up to the end of the row
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
        const uint32_t i = (a * 256 + threadIdx.x) * 8;
        const int64_t e = e0 + i;
        if (e >= total) continue;
        const uint32_t r = (uint32_t)(((in_row + i) * m) >> 40);
        left[a] = (r + 1) * (uint32_t)cols - (in_row + i);
        s[a] = __ldg(scales + row0 + r);
        next[a] = left[a] < 8 && e + left[a] < total ? __ldg(scales + row0 + r + 1) : 0.0f;
        if (e + 8 <= total) {
            load_codes<8>(codes, e, z[a]);
            if constexpr (DY) load_elements<TYPE, 8>(dy, e, g[a]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float one[1] = {0.0f}, two[1] = {0.0f};
                if (e + k < total) {
                    load_codes<1>(codes, e + k, one);
                    if constexpr (DY) load_elements<TYPE, 1>(dy, e + k, two);
                }
                z[a][k] = one[0];
                g[a][k] = two[0];
            }
        }
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
        const int64_t e = e0 + (a * 256 + threadIdx.x) * 8;
        if (e >= total) break;
#pragma unroll
        for (int k = 0; k < 8; ++k) z[a][k] *= (uint32_t)k < left[a] ? s[a] : next[a];
        if constexpr (DY) times_slope<TYPE, 8>(z[a], g[a]);
        if (e + 8 <= total) {
            store_elements<TYPE, 8>(out, e, z[a]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float one[1] = {z[a][k]};
                if (e + k < total) store_elements<TYPE, 1>(out, e + k, one);
            }
        }
    }
}

// Whether rows of `elem`-byte elements can be read and written eight at a time.
bool by_eight(const void* p, int64_t ld, int elem) {
    return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(std::min(8 * elem, 16) - 1)) == 0 && ld % 8 == 0;
}

template <int TYPE, int N, int NV, int TPR, bool FLAT>
cudaError_t store_launch(const void* x, int64_t ldx, int64_t rows, int cols, int act, int8_t* codes,
                  int64_t ldc, float* scales, void* y, int64_t ldy, cudaStream_t st) {
    constexpr int kRows = 256 / TPR;
    return launch_early(ckpt_store_kernel<TYPE, N, NV, TPR, FLAT>, (rows + kRows - 1) / kRows, 256, 0, st, x,
                        ldx, rows, cols, act, codes, ldc, scales, y, ldy);
}

// The narrowest layout that holds a row: a warp up to 2048 elements, else a block.
template <int TYPE, int N, bool FLAT, typename... A>
cudaError_t store_rows(int cols, A... a) {
    // (a row may reach into one piece more than its width makes)
    const int nv = (cols + (FLAT ? 14 : 0) + 255) / 256;
    if (nv <= 1) return store_launch<TYPE, N, 1, 32, FLAT>(a...);
    if (nv <= 2) return store_launch<TYPE, N, 2, 32, FLAT>(a...);
    if (nv <= 3) return store_launch<TYPE, N, 3, 32, FLAT>(a...);
    if (nv <= 4) return store_launch<TYPE, N, 4, 32, FLAT>(a...);
    if (nv <= 6) return store_launch<TYPE, N, 6, 32, FLAT>(a...);
    if (nv <= 8) return store_launch<TYPE, N, 8, 32, FLAT>(a...);
    if (nv <= 16) return store_launch<TYPE, N, 2, 256, FLAT>(a...);
    if (nv <= 32) return store_launch<TYPE, N, 4, 256, FLAT>(a...);
    return store_launch<TYPE, N, 16, 256, FLAT>(a...);
}

// Matrices without gaps that start aligned.
bool flat_ok(const void* dy, int64_t lddy, const int8_t* codes, int64_t ldc, int cols, const void* out,
             int64_t ldo, int elem) {
    return cols >= 8 && ldc == cols && ldo == cols && (!dy || lddy == cols) && by_eight(codes, 8, 1) &&
           by_eight(out, 8, elem) && (!dy || by_eight(dy, 8, elem));
}

template <int TYPE, bool DY>
cudaError_t flat_launch(const void* dy, const int8_t* codes, const float* scales, int64_t rows, int cols,
                        void* out, cudaStream_t st) {
    const int64_t total = rows * cols, per_block = 256 * 8 * 2;
    return launch_early(ckpt_load_flat_kernel<TYPE, DY>, (total + per_block - 1) / per_block, 256, 0, st,
                        dy, codes, scales, total, cols, (1ull << 40) / cols + 1, out);
}

template <int TYPE, int N, bool DY>
cudaError_t load_launch(const void* dy, int64_t lddy, const int8_t* codes, int64_t ldc,
                 const float* scales, int64_t rows, int cols, void* out, int64_t ldo,
                 cudaStream_t st) {
    const int pieces = cols / N;
    // about 4096 elements a block; under 2^23 pieces in any case
    const int per_block = std::max(1, 4096 / cols);
    return launch_early(ckpt_load_kernel<TYPE, N, DY>, (rows + per_block - 1) / per_block, 256, 0, st, dy,
                        lddy, codes, ldc, scales, rows, cols, per_block, (1ull << 40) / pieces + 1,
                        out, ldo);
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

// bf16: dy is an operand as it lies, and the kept rows s z the other, in two bf16 parts:
// what they lose is 2^-15 of an entry.  In one part they lost about half of what rounding dw
// does (2.8e-3 against 2.3e-3 in all); dw of 768 -> 1,536 over 32,768 rows takes 128 us, 72 so
// (f16 166, float32 274).  f16 and float32: dy s in two or three bf16 parts, and
// the codes as they are (exact).
// Rows go by in pieces whose copies take 1 GB (4,096 rows at least), each added to the sums of
// the one before.
constexpr int64_t kCopyBytes = (int64_t)1 << 30;
struct GradPlan {
    int parts, kept_parts;   // of dy and of the kept rows
    bool scaled;             // the kept rows are the operand, dy has no scale
    bool copy;               // dy is copied
    int64_t piece;           // rows at a time, a multiple of kTileK (or all)
    int64_t lda, ldb;
    int splits;
    uint16_t *a, *b;
    float* slots;
    int64_t ldslot;
    size_t bytes;
};
GradPlan grad_plan(int64_t rows, int out_cols, int cols, int dtype, bool in_place,
                   const Device& dev, void* workspace) {
    GradPlan p{};
    p.scaled = dtype == PVS_BF16;
    p.copy = !p.scaled || !in_place;
    p.parts = dtype == PVS_BF16 ? 1 : dtype == PVS_F16 ? 2 : 3;
    p.kept_parts = p.scaled ? 2 : 1;
    p.lda = copied_ld(out_cols);
    p.ldb = copied_ld(cols);
    p.ldslot = round_up(cols, 8);
    // (the same pieces whether dy is copied or not: the workspace serves both)
    const int64_t row_bytes = 2 * (p.parts * p.lda + p.kept_parts * p.ldb);
    p.piece = std::min(rows, std::max<int64_t>(kCopyBytes / row_bytes, 4096) / kTileK * kTileK);
    const int bn = tile_columns(cols);
    const int tile_m = kTileM * ctas_for(out_cols, dev);
    const int64_t slots = tile_m > kTileM ? dev.pairs : dev.sms;
    const int64_t units = (int64_t)((out_cols + tile_m - 1) / tile_m) * ((cols + bn - 1) / bn);
    const int64_t kc = (p.piece + kTileK - 1) / kTileK;
    // float32 sums: 64 steps in the tensor cores, which cut the sum to 24 bits each, at
    // most before the splits are added with rounding (as far as 2 GB of them go).  With 128 dw of
    // 25,000 rows was off by 1.5e-6, 2.7 times the plain form; so by 8e-7
    const int64_t room = std::max<int64_t>(1, ((int64_t)2 << 30) / (out_cols * p.ldslot * 4));
    p.splits = best_splits(units, kc, (int)slots, p.parts * p.kept_parts,
                           dtype == PVS_F32 ? std::min((kc + 15) / 16, room) : 1);
    Carver c{static_cast<uint8_t*>(workspace)};
    if (p.copy) p.a = c.take<uint16_t>(p.parts * p.piece * p.lda);
    p.b = c.take<uint16_t>(p.kept_parts * p.piece * p.ldb);
    if (p.splits > 1 || p.piece < rows) p.slots = c.take<float>((int64_t)p.splits * out_cols * p.ldslot);
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
    const int es = element_bytes(dtype);
    if (!x || !codes || !scales || (act != PVS_ACT_NONE && (!y || !on_elements(y, es))) ||
        !on_elements(x, es) || !on_elements(scales, 4))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    count_launches(1);
    cudaError_t e = cudaSuccess;
    // eights: aligned rows, or matrices without gaps that start aligned
    const bool dense = ldx == cols && ldcodes == cols && (act == PVS_ACT_NONE || ldy == cols);
    const bool eight = (cols % 8 == 0 || dense) && by_eight(x, dense ? 8 : ldx, es) &&
                       by_eight(codes, dense ? 8 : ldcodes, 1) &&
                       (act == PVS_ACT_NONE || by_eight(y, dense ? 8 : ldy, es)) &&
                       cols <= 32767 - 8;
    if (eight && cols % 8 != 0)
        PVS_BY_TYPE(dtype, e = (store_rows<TYPE, 8, true>(cols, x, ldx, rows, cols, act, codes,
                                                          ldcodes, scales, y, ldy, st)));
    else if (eight)
        PVS_BY_TYPE(dtype, e = (store_rows<TYPE, 8, false>(cols, x, ldx, rows, cols, act, codes,
                                                           ldcodes, scales, y, ldy, st)));
    else
        PVS_BY_TYPE(dtype, e = (store_rows<TYPE, 1, false>(cols, x, ldx, rows, cols, act, codes,
                                                           ldcodes, scales, y, ldy, st)));
    return queued(e);
}

extern "C" pvs_status pvs_ckpt_load(const int8_t* codes, int64_t ldcodes, const float* scales,
                                    int64_t rows, int32_t cols, void* out, int64_t ldout,
                                    int32_t dtype, void* cuda_stream) {
    if (!rows_ok(rows, cols, dtype) || ldcodes < cols || ldout < cols) return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    if (!codes || !scales || !out || !on_elements(scales, 4) || !on_elements(out, element_bytes(dtype)))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    count_launches(1);
    cudaError_t e = cudaSuccess;
    if (cols % 8 != 0 && flat_ok(nullptr, 0, codes, ldcodes, cols, out, ldout, element_bytes(dtype)) &&
        rows * cols < (int64_t)1 << 42)
        PVS_BY_TYPE(dtype, e = (flat_launch<TYPE, false>(nullptr, codes, scales, rows, cols, out, st)));
    else if (cols % 8 == 0 && by_eight(codes, ldcodes, 1) && by_eight(out, ldout, element_bytes(dtype)))
        PVS_BY_TYPE(dtype, e = (load_launch<TYPE, 8, false>(nullptr, 0, codes, ldcodes, scales, rows,
                                                        cols, out, ldout, st)));
    else
        PVS_BY_TYPE(dtype, e = (load_launch<TYPE, 1, false>(nullptr, 0, codes, ldcodes, scales, rows,
                                                        cols, out, ldout, st)));
    return queued(e);
}

extern "C" pvs_status pvs_ckpt_act_backward(const void* dy, int64_t lddy, const int8_t* codes,
                                            int64_t ldcodes, const float* scales, int64_t rows,
                                            int32_t cols, int32_t dtype, int32_t act, void* dx,
                                            int64_t lddx, void* cuda_stream) {
    if (!rows_ok(rows, cols, dtype) || lddy < cols || ldcodes < cols || lddx < cols ||
        act != PVS_ACT_GELU)
        return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    const int es = element_bytes(dtype);
    if (!dy || !codes || !scales || !dx || !on_elements(dy, es) || !on_elements(scales, 4) ||
        !on_elements(dx, es))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    count_launches(1);
    cudaError_t e = cudaSuccess;
    if (cols % 8 != 0 && flat_ok(dy, lddy, codes, ldcodes, cols, dx, lddx, es) &&
        rows * cols < (int64_t)1 << 42)
        PVS_BY_TYPE(dtype, e = (flat_launch<TYPE, true>(dy, codes, scales, rows, cols, dx, st)));
    else if (cols % 8 == 0 && by_eight(codes, ldcodes, 1) && by_eight(dy, lddy, es) &&
        by_eight(dx, lddx, es))
        PVS_BY_TYPE(dtype, e = (load_launch<TYPE, 8, true>(dy, lddy, codes, ldcodes, scales, rows, cols,
                                                       dx, lddx, st)));
    else
        PVS_BY_TYPE(dtype, e = (load_launch<TYPE, 1, true>(dy, lddy, codes, ldcodes, scales, rows, cols,
                                                       dx, lddx, st)));
    return queued(e);
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
    *bytes = grad_plan(rows, out_cols, cols, dtype, false, dev, nullptr).bytes;
    return PVS_OK;
}

extern "C" pvs_status pvs_ckpt_grad_weight(const void* dy, int64_t lddy, const int8_t* codes,
                                           int64_t ldcodes, const float* scales, int64_t rows,
                                           int32_t out_cols, int32_t cols, int32_t dtype, void* dw,
                                           int64_t lddw, void* workspace, size_t workspace_bytes,
                                           void* cuda_stream) {
    if (!rows_ok(rows, cols, dtype) || out_cols < 1 || out_cols > kMaxDim || lddy < out_cols ||
        ldcodes < cols || lddw < cols || !dw || !on_elements(dw, element_bytes(dtype)))
        return PVS_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t es = (size_t)element_bytes(dtype);
    if (rows == 0)
        return queued(cudaMemset2DAsync(dw, (size_t)lddw * es, 0, (size_t)cols * es,
                                        (size_t)out_cols, st));
    if (!dy || !codes || !scales || !on_elements(dy, (int)es) || !on_elements(scales, 4))
        return PVS_ERR_INVALID;
    Device dev;
    cudaError_t e = device(&dev);
    if (e != cudaSuccess) return queued(e);
    const bool in_place = (reinterpret_cast<uintptr_t>(dy) & 15u) == 0 && lddy % 8 == 0;
    const GradPlan p = grad_plan(rows, out_cols, cols, dtype, in_place, dev, workspace);
    if (workspace_bytes < p.bytes || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return PVS_ERR_INVALID;
    const pvs_status before = (pvs_status)take_status(dev);
    if (before != PVS_OK) return before;
    for (int64_t r0 = 0; r0 < rows && e == cudaSuccess; r0 += p.piece) {
        const int64_t n = std::min(p.piece, rows - r0);
        const void* dy0 = static_cast<const uint8_t*>(dy) + r0 * lddy * (int64_t)es;
        SplitArgs s{};
        if (p.copy) {
            s.src = dy0;
            s.ld = lddy;
            s.rows = n;
            s.cols = out_cols;
            s.dtype = dtype;
            s.row_scale = p.scaled ? nullptr : scales + r0;
            s.dst = p.a;
            s.ldd = p.lda;
            s.part_stride = n * p.lda;
            s.parts = p.parts;
        }
        CodesArgs c{};
        c.codes = codes + r0 * ldcodes;
        c.ldc = ldcodes;
        c.rows = n;
        c.cols = cols;
        c.scales = p.scaled ? scales + r0 : nullptr;
        c.dst = p.b;
        c.ldd = p.ldb;
        c.part_stride = n * p.ldb;
        c.parts = p.kept_parts;
        e = launch_codes(c, s, st);
        if (e != cudaSuccess) break;
        Args g{};
        g.status = dev.status;
        g.nprob = 1;
        Problem& q = g.p[0];
        g.cta = ctas_for(out_cols, dev);
        set_tiles(q, out_cols, cols, tile_columns(cols), n, g.cta);
        q.splits = even_splits(q.kchunks, p.splits);
        const Matrix a = p.copy ? Matrix{p.a, n, out_cols, p.lda, p.parts, n * p.lda}
                                : Matrix{dy0, n, out_cols, lddy, 1, 0};
        if (!operand_map(&q.a, a, true, 0) ||
            !operand_map(&q.b, Matrix{p.b, n, cols, p.ldb, p.kept_parts, n * p.ldb}, true, 0))
            return PVS_ERR_CUDA;
        q.a_mn = q.b_mn = 1;
        q.to_slots = p.slots != nullptr;
        q.accumulate = r0 > 0;
        q.slots = p.slots;
        q.slot_stride = (int64_t)out_cols * p.ldslot;
        q.ldslot = p.ldslot;
        q.out = dw;
        q.ldout = lddw;
        q.out_type = dtype;
        q.alpha0 = 1.0f;
        part_pairs(g, p.parts, p.kept_parts);
        e = launch_gemm(kOut, g, dev, st);
    }
    if (e == cudaSuccess && p.slots)
        e = launch_sum_slots(p.slots, p.splits, (int64_t)out_cols * p.ldslot, p.ldslot, out_cols, cols,
                             nullptr, 1.0f, dw, lddw, dtype, st);
    return queued(e);
}

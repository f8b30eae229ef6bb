// Softmax cross entropy over a large vocabulary and its gradients (head.h), by
// the product of head_gemm.cu.
//
//   forward    l = a x w^T + b, tile by tile; each tile's rows leave a maximum and
//              a sum of 2^(l - max), which a second launch joins; no logit is kept (of
//              many rows and items, a block of the rows at a time)
//   backward   for each piece of the vocabulary: the logits again, and from them
//              G = g (2^(l - m) / s - [j = y]) in 16-bit parts; then, in one launch,
//              dx += G w and dw = G^T x
//
// Every logit costs 2 d operations in the forward pass and 10 d in the backward
// pass: bound by the tensor cores unless there are few rows, when w (and dw) bound
// it.  G of a piece is written once and read twice, in two parts, each a product of its
// own.  With both gradients, bf16: 8,192 rows over 8,192 items of 768 0.49 ms, 256 rows over
// 1,000,000 items 2.2 ms; f16: 4,096 rows over 200,000 items of 1,024 7.2 ms.
#include <algorithm>
#include <cmath>
#include <limits>

#include <cuda_fp16.h>

#include "../../include/head.h"
#include "head_gemm.h"
#include "kernels.h"
#include "pvs_common.cuh"
#include "xent_few.h"

namespace pvs {
namespace head {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;
// G of a piece, and copies of a piece of w, at most about: a piece costs two launches and
// their uneven ends, and the sums of dx one pass over its splits.  With G in one part a step of
// 256 rows over a million items took 2.5 ms in pieces of 32 K items, 1.6 ms in 256 K ones.
constexpr size_t kGradBytes = (size_t)1 << 30;
constexpr size_t kPartsBytes = (size_t)1 << 30;
// The tiles' statistics of the forward pass, 8 bytes for each row and tile of items: the rows
// go by in blocks whose statistics take this much, or of 1,024 (32 bytes an item then).
constexpr int64_t kStatBytes = (int64_t)1 << 30;
constexpr int64_t kStatRows = 1024;

__device__ __forceinline__ float element(const void* p, int dtype, int64_t i) {
    if (dtype == PVS_F32) return static_cast<const float*>(p)[i];
    const uint16_t u = static_cast<const uint16_t*>(p)[i];
    return dtype == PVS_BF16 ? __uint_as_float((uint32_t)u << 16) : __half2float(__ushort_as_half(u));
}

// A lane's part of <x_row, w_y>, element by element or eight 16-bit ones at a time.
__device__ float dot_any(const pvs_xent_args& a, int64_t row, int64_t y) {
    float dot = 0.0f;
#pragma unroll 4
    for (int k = threadIdx.x & 31; k < a.dim; k += 32)
        dot = fmaf(element(a.x, a.dtype, row * a.ldx + k), element(a.w, a.dtype, y * a.ldw + k), dot);
    return dot;
}
__device__ float dot_wide(const pvs_xent_args& a, int64_t row, int64_t y) {
    const uint4* x = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.x) + row * a.ldx);
    const uint4* w = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.w) + y * a.ldw);
    float lo = 0.0f, hi = 0.0f;
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

// ---- rows of the forward pass ------------------------------------------------------
struct JoinArgs {
    const float2* part;          // [n][rows]: the tiles' (m, s), the target left out
    int64_t n;
    pvs_xent_args a;
    float k2;
    bool wide;                   // 16-bit rows of whole, aligned eights
    float* loss;
    float4* stats;
};

__device__ __forceinline__ void join(float& m, float& s, float2 p) {
    const float nm = fmaxf(m, p.x), ref = nm == -INFINITY ? 0.0f : nm;
    s = s * exp2f(m - ref) + p.y * exp2f(p.x - ref);
    m = nm;
}

// A row's statistics from its tiles', joined in a fixed order, and its loss.
// The target's logit is a float32 product of its own: the tensor cores cut each
// step's sum, which takes about d / 16 times 2^-25 of a logit, and the target's is
// the largest and the one that the loss subtracts.  Left out of the tiles' sums, it
// also leaves 1 - p exact where p is near 1.
// R rows a block; a warp's lanes run over the rows first (the tiles' statistics
// are stored by rows).  Eight where that still gives every SM four blocks' rows, else one:
// 8,192 rows over as many items of 768 take a loss of 73 us with eight, 89 with one; 500 rows
// over 100,000 of 256 take 35 and 38, 64 over 500,000 63 and 53.
template <int R>
__global__ void __launch_bounds__(256) xent_join_kernel(const JoinArgs j) {
    constexpr int kLanes = 256 / R;
    __shared__ float2 sh[kLanes][R];
    __shared__ float dots[R];
    next_early();
    wait_before();
    const pvs_xent_args& a = j.a;
    const int r = threadIdx.x % R, lane = threadIdx.x / R;
    const int64_t row = (int64_t)blockIdx.x * R + r;
    float m = -INFINITY, s = 0.0f;
    if (row < a.rows) {
#pragma unroll 4
        for (int64_t i = lane; i < j.n; i += kLanes) join(m, s, j.part[i * a.rows + row]);
    }
    sh[lane][r] = make_float2(m, s);
    for (int i = threadIdx.x >> 5; i < R; i += 8) {
        const int64_t at = (int64_t)blockIdx.x * R + i;
        const int64_t y = at < a.rows ? a.targets[at] : -1;
        float dot = 0.0f;
        if (y >= 0 && y < a.items) dot = j.wide ? dot_wide(a, at, y) : dot_any(a, at, y);
        dot = warp_sum(dot);
        if ((threadIdx.x & 31) == 0) dots[i] = dot;
    }
    __syncthreads();
    for (int w = kLanes / 2; w > 0; w >>= 1) {
        if (lane < w) {
            join(m, s, sh[lane + w][r]);
            sh[lane][r] = make_float2(m, s);
        }
        __syncthreads();
    }
    if (lane != 0 || row >= a.rows) return;
    const int64_t y = a.targets[row];
    const float nan = __int_as_float(0x7fffffff);
    float loss = 0.0f, hit = 0.0f, t = -INFINITY;
    const bool target = y >= 0 && y < a.items;
    if (target) {
        float b = a.bias ? a.bias[y] : 0.0f;
        if (b != -INFINITY) {
            const float b2 = isfinite(b) ? fminf(fmaxf(b * kLog2e, -3.402823466e38f), 3.402823466e38f) : b;
            t = fmaf(dots[r], j.k2, b2);
        }
    }
    if (y == a.ignore_index) {
    } else if (!target) {
        loss = hit = nan;
    } else if (t == -INFINITY) {
        // the target is not in the softmax; nothing else is either: no loss
        loss = m == -INFINITY && s == 0.0f ? 0.0f : INFINITY;
    } else if (m == -INFINITY && s == 0.0f) {
        m = t;                                  // the target alone
        s = 1.0f;
        if (t != t) loss = hit = nan;
    } else {
        const float d = m - t;                  // others against the target
        if (d < 64.0f) {
            const float rest = s * exp2f(d);
            loss = log1pf(rest);
            hit = -rest / (1.0f + rest);
            if (isinf(rest)) hit = -1.0f;
        } else if (t < -1e38f && a.bias) {
            // a bias near the type's lowest value was cut to stay finite here
            loss = (float)((double)m * kLn2 - (double)a.bias[y]) + logf(s);
            hit = -1.0f;
        } else {
            loss = fmaf(d, (float)kLn2, logf(s));
            hit = d != d ? nan : -1.0f;
        }
        join(m, s, make_float2(t, 1.0f));
    }
    j.loss[row] = loss;
    j.stats[row] = make_float4(m, s, hit, t);
}

// ---- rows of the backward pass -----------------------------------------------------
// f16 gradients keep G times a power of two that puts the largest finite
// |grad_loss| at 2^13 .. 2^14: entries down to 2^-38 of it stay above f16's last
// bit, which is below what an f16 gradient can hold.  up[0] is that power, up[1] its
// inverse.  One block: a row's weight is 12 bytes of the thousands that it costs.
__global__ void __launch_bounds__(1024) xent_grad_scale_kernel(const float* __restrict__ grad,
                                                               const int64_t* __restrict__ targets,
                                                               int64_t ignore_index, int64_t rows,
                                                               float* up) {
    next_early();
    wait_before();
    __shared__ float tops[32];
    float v = 0.0f;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) {
        const float g = fabsf(grad[i]);
        if (targets[i] != ignore_index && isfinite(g)) v = fmaxf(v, g);
    }
    v = warp_max(v);
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    v = warp_max(tops[threadIdx.x]);
    if (threadIdx.x != 0) return;
    const int e = v > 0.0f ? min(max(14 - (ilogbf(v) + 1), -126), 126) : 0;
    up[0] = exp2f((float)e);
    up[1] = exp2f((float)-e);
}

// ---- the plan of a call --------------------------------------------------------------
// float32 operands: the logits' product takes them in two f16 parts with a power of two
// for each row and item, which its epilogue undoes (three products, the fourth is below
// 2^-22 of an element); the gradients' products, whose sums run over those rows and
// items, in three bf16 parts (six products).
// 16-bit operands: G has two parts, so that a gradient's error is the rounding of its
// output (bf16 1.7e-3, f16 2.1e-4).  One part would lose as much again (bf16 2.3e-3 to 2.7e-3)
// and take two thirds of the time: a step of 8,192 rows over 8,192 items of 768 485 us, 302 with
// one part; of 256 over a million 2,230 and 1,520.
struct Plan {
    int parts = 1, f16 = 0;     // of the gradients' operands
    int gparts = 1;             // of G
    bool two = false;           // the logits' operands are f16 pairs
    uint16_t *x16 = nullptr, *w16 = nullptr;
    float *xunit = nullptr, *wunit = nullptr;
    int64_t ldp = 0;            // leading dimension of copied operands
    int64_t lds = 0;            // and of float32 sums
    bool copy_x = false, copy_w = false;
    int64_t piece = 0;          // items per piece, a multiple of kTileN (or all)
    int64_t pieces = 0, piece_tiles = 0;
    int64_t ldg = 0;
    int bnl = 0;                // columns per tile of the logits
    int bnd = 0;                // columns per tile of the gradients
    int xsplits = 1, wsplits = 1, slots0 = 0;
    int few = 0;                // few float32 rows: those kernels' blocks
    float* few_g = nullptr;
    // workspace
    uint16_t *x = nullptr, *w = nullptr, *g = nullptr;
    float2* part = nullptr;
    GradRow* row = nullptr;
    unsigned int* words = nullptr;   // [0] up, [1] its inverse, [2] bad masked
    float *xslots = nullptr, *wslots = nullptr;
    size_t bytes = 0;
};

bool aligned(const void* p, int64_t ld, int dtype) {
    return dtype != PVS_F32 && (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % 8 == 0;
}

bool valid(const pvs_xent_args* a) {
    if (!a || a->rows < 0 || a->rows > kMaxRows || a->items < 1 || a->items > kMaxRows ||
        a->dim < 1 || a->dim > kMaxDim || a->dtype < PVS_BF16 || a->dtype > PVS_F32 ||
        a->reserved != 0 || !(a->scale >= 0x1p-126f) || !std::isfinite(a->scale) || a->ldx < a->dim ||
        a->ldw < a->dim)
        return false;
    const int es = element_bytes(a->dtype);
    return a->w && (a->rows == 0 || (a->x && a->targets)) && on_elements(a->x, es) &&
           on_elements(a->w, es) && on_elements(a->targets, 8) && on_elements(a->bias, 4);
}

// How dx (u0 tiles, k0 chunks of k) and dw (u1, k1) share the `slots` CTAs or pairs
// of one launch: each gets slots of its own, and its k is cut where that evens the
// ends.  The cost of a choice, in the time of a chunk's MMAs (npairs of them a
// chunk), is the longer side's rounds of units (unit_cost), and what the splits' sums
// move.
struct Division {
    int xsplits = 1, wsplits = 1, slots0 = 1;
};
// xleast, wleast: the fewest splits that float32 sums take (else 1).
Division divide(int64_t u0, int64_t k0, int64_t u1, int64_t k1, int slots, int npairs,
                int64_t xleast, int64_t wleast, bool accumulate) {
    Division best;
    double least = 1e300;
    for (int64_t wsplits = wleast; wsplits <= k1; wsplits *= 2) {
        if (wsplits > wleast && u1 * wsplits > 8 * slots) break;
        const double w1 = unit_cost((k1 + wsplits - 1) / wsplits * npairs, wsplits > 1);
        const int64_t n1 = u1 * wsplits;
        // (every split up to 8, then in steps of an eighth)
        for (int64_t xsplits = xleast;
             xsplits <= k0 && (xsplits == xleast || u0 * xsplits <= 8 * slots);
             xsplits += std::max<int64_t>(1, xsplits / 8)) {
            const int64_t len = (k0 + xsplits - 1) / xsplits;
            const double w0 = unit_cost(len * npairs, xsplits > 1 || accumulate);
            const int64_t n0 = u0 * xsplits;
            const int p = (int)(slots * (n0 * w0) / (n0 * w0 + n1 * w1) + 0.5);
            for (int s0 = std::min(std::max(1, p - 1), slots - 1); s0 <= std::min(slots - 1, p + 1);
                 ++s0) {
                const double t0 = (double)((n0 + s0 - 1) / s0) * w0;
                const double t1 = (double)((n1 + slots - s0 - 1) / (slots - s0)) * w1;
                // (dx alone, which a head trained against fixed items wants, takes the same
                // splits over every slot: a quarter of its time counts too)
                const double x_alone = (double)((n0 + slots - 1) / slots) * w0;
                const double cost = std::max(t0, t1) + 0.25 * x_alone +
                                    sums_cost((xsplits > 1 ? n0 : 0) + (wsplits > 1 ? n1 : 0), slots) +
                                    kSumsLaunch * ((xsplits > 1 || accumulate) + (wsplits > 1));
                if (cost < least) {
                    least = cost;
                    best.xsplits = (int)xsplits;
                    best.wsplits = (int)wsplits;
                    best.slots0 = s0;
                }
            }
        }
    }
    return best;
}

// Whether a call's rows are few enough for the kernels that take w as it is.
bool few_rows(const pvs_xent_args& a) {
    return a.dtype == PVS_F32 && a.dim <= kFewDim && a.rows <= kFewRows;
}

Plan plan_of(const pvs_xent_args& a, bool backward, const Device& dev, void* workspace) {
    Plan p;
    const int64_t T = a.rows, V = a.items;
    p.parts = parts_of(a.dtype);
    p.f16 = a.dtype == PVS_F16;
    p.gparts = std::max(2, p.parts);
    p.two = a.dtype == PVS_F32;
    p.ldp = copied_ld(a.dim);
    p.lds = round_up(a.dim, 8);
    if (few_rows(a)) {
        Carver c{static_cast<uint8_t*>(workspace)};
        p.few = few_blocks(V, dev);
        if (!backward) {
            p.part = c.take<float2>(p.few * T);
        } else {
            p.row = c.take<GradRow>(T);
            p.words = c.take<unsigned int>(64);
            p.piece = std::min(V, (int64_t)(kGradBytes / (4 * few_rows_padded(T))));
            p.few_g = c.take<float>(p.piece * few_rows_padded(T));
            p.xslots = c.take<float>(p.few * T * p.lds);
        }
        p.bytes = c.used;
        return p;
    }
    p.copy_x = !aligned(a.x, a.ldx, a.dtype);
    p.copy_w = !aligned(a.w, a.ldw, a.dtype);
    int64_t piece = round_up(V, kTileN);
    const bool w_buffer = p.copy_w || (backward && a.bias);
    if (w_buffer) {
        const int64_t most = (int64_t)(kPartsBytes / ((size_t)p.parts * p.ldp * 2)) / kTileN * kTileN;
        piece = std::min(piece, std::max<int64_t>(most, 4 * kTileN));
    }
    if (backward) {
        const int64_t most = (int64_t)(kGradBytes / ((size_t)p.gparts * T * 2)) / kTileN * kTileN;
        piece = std::min(piece, std::max<int64_t>(most, 4 * kTileN));
    }
    p.piece = piece;
    p.pieces = (V + piece - 1) / piece;
    p.bnl = std::min(piece, V) >= kTileN ? kTileN : tile_columns(V);
    // (a piece's tiles of logits: their statistics are numbered on from piece to piece)
    p.piece_tiles = (piece + p.bnl - 1) / p.bnl;
    Carver c{static_cast<uint8_t*>(workspace)};
    if (backward || (p.copy_x && !p.two)) p.x = c.take<uint16_t>((int64_t)p.parts * T * p.ldp);
    if (w_buffer && (backward || !p.two)) p.w = c.take<uint16_t>((int64_t)p.parts * piece * p.ldp);
    if (p.two) {
        p.x16 = c.take<uint16_t>(2 * T * p.ldp);
        p.w16 = c.take<uint16_t>(2 * piece * p.ldp);
        p.xunit = c.take<float>(T);
        p.wunit = c.take<float>(piece);
    }
    if (!backward) {
        p.part = c.take<float2>(p.pieces * p.piece_tiles * T);
    } else {
        p.row = c.take<GradRow>(T);
        p.words = c.take<unsigned int>(64);
        p.ldg = piece;
        p.g = c.take<uint16_t>((int64_t)p.gparts * T * p.ldg);
        p.bnd = tile_columns(a.dim);
        const int64_t first = std::min(piece, V);
        const int64_t nt = (a.dim + p.bnd - 1) / p.bnd;
        const int cta = ctas_for(std::max(T, first), dev);
        const int tile = kTileM * cta;
        const int slots = cta == 2 ? dev.pairs : dev.sms, npairs = a.dtype == PVS_F32 ? 6 : p.gparts;
        const int64_t ux = (T + tile - 1) / tile * nt, kx = (first + kTileK - 1) / kTileK;
        const int64_t uw = (first + tile - 1) / tile * nt, kw = (T + kTileK - 1) / kTileK;
        // float32 sums: each step in the tensor cores cuts the sum to 24 bits, 32 steps
        // at most before the splits are added with rounding (as far as 2 GB of them go).  With 64
        // dw of 6,320 rows over 3,384 items of 128 was off by 1.4e-6, 2.8 times the plain form; so
        // by 8.4e-7.  A step of 8,192 over 20,000 of 384 takes 2.1 ms, 2.0 with 64.
        auto fewest = [&](int64_t chunks, int64_t rows) {
            const int64_t room = ((int64_t)2 << 30) / std::max<int64_t>(1, rows * p.lds * 4);
            return a.dtype == PVS_F32 ? std::max<int64_t>(1, std::min((chunks + 7) / 8, room)) : 1;
        };
        const Division s = divide(ux, kx, uw, kw, slots, npairs, fewest(kx, T), fewest(kw, first),
                                  p.pieces > 1);
        p.xsplits = even_splits((first + kTileK - 1) / kTileK, s.xsplits);
        p.wsplits = even_splits((T + kTileK - 1) / kTileK, s.wsplits);
        p.slots0 = s.slots0;
        if (p.xsplits > 1 || p.pieces > 1)
            p.xslots = c.take<float>((int64_t)p.xsplits * T * p.lds);
        if (p.wsplits > 1) p.wslots = c.take<float>((int64_t)p.wsplits * first * p.lds);
    }
    p.bytes = c.used;
    return p;
}

// Rows of a block of the forward pass.
int64_t block_rows(const pvs_xent_args& a) {
    const int64_t most = kStatBytes / (8 * ((a.items + kTileN - 1) / kTileN));
    return std::min(a.rows, std::max(most / (2 * kTileM) * (2 * kTileM), kStatRows));
}

// The call for the rows [t0, t0 + n).
pvs_xent_args rows_of(const pvs_xent_args& a, int64_t t0, int64_t n) {
    pvs_xent_args b = a;
    b.x = static_cast<const uint8_t*>(a.x) + t0 * a.ldx * element_bytes(a.dtype);
    b.targets = a.targets + t0;
    b.rows = n;
    return b;
}

// What the forward pass wants: that of a whole block, or of the last.
size_t forward_bytes(const pvs_xent_args& a, const Device& dev) {
    const int64_t block = block_rows(a), last = a.rows - (a.rows - 1) / block * block;
    if (block == a.rows) return plan_of(a, false, dev, nullptr).bytes;
    return std::max(plan_of(rows_of(a, 0, block), false, dev, nullptr).bytes,
                    plan_of(rows_of(a, a.rows - last, last), false, dev, nullptr).bytes);
}

// Logits of the piece [v0, v0 + n).
cudaError_t logits(int epilogue, Args& g, const Plan& p, const pvs_xent_args& a, int64_t v0,
                   int64_t n, const Device& dev, cudaStream_t st) {
    const int64_t T = a.rows;
    const Matrix x = p.two      ? Matrix{p.x16, T, a.dim, p.ldp, 2, T * p.ldp}
                     : p.copy_x ? Matrix{p.x, T, a.dim, p.ldp, 1, 0}
                                : Matrix{a.x, T, a.dim, a.ldx, 1, 0};
    const Matrix w = p.two      ? Matrix{p.w16, n, a.dim, p.ldp, 2, p.piece * p.ldp}
                     : p.copy_w ? Matrix{p.w, n, a.dim, p.ldp, 1, 0}
                                : Matrix{a.w, a.items, a.dim, a.ldw, 1, 0};
    g.f16 = a.dtype != PVS_BF16;
    g.sm.row_unit = p.xunit;
    g.sm.col_unit = p.wunit;
    Problem& q = g.p[0];
    q = Problem{};
    g.nprob = 1;
    g.cta = ctas_for(a.rows, dev);
    set_tiles(q, a.rows, n, p.bnl, a.dim, g.cta);
    if (!operand_map(&q.a, x, false, kTileM) || !operand_map(&q.b, w, false, q.bn / g.cta))
        return cudaErrorInvalidValue;
    q.b_no = p.copy_w ? 0 : (int)v0;
    q.m_fast = 1;
    g.sm.item0 = (int)v0;
    part_pairs(g, x.parts, w.parts, 1);
    return launch_gemm(epilogue, g, dev, st);
}

SplitArgs split_of(const pvs_xent_args& a, const Plan& p) {
    SplitArgs s{};
    s.cols = a.dim;
    s.dtype = a.dtype;
    s.ldd = p.ldp;
    s.parts = p.parts;
    s.to_f16 = p.f16;
    s.ignore_index = a.ignore_index;
    return s;
}

// The copy of x (backward: without the rows that have no gradient, whatever they hold:
// it must not meet G's zeros), and that of the items [v0, v0 + n) without masked ones.
Split16Args rows_copy(const pvs_xent_args& a, const Plan& p, bool zero_ignored) {
    SplitArgs s = split_of(a, p);
    s.src = a.x;
    s.ld = a.ldx;
    s.rows = a.rows;
    s.dst = p.x;
    s.part_stride = a.rows * p.ldp;
    if (zero_ignored) s.zero_target = a.targets;
    return Split16Args{s, p.x16, a.rows * p.ldp, p.xunit};
}
Split16Args items_copy(const pvs_xent_args& a, const Plan& p, int64_t v0, int64_t n) {
    SplitArgs s = split_of(a, p);
    s.src = static_cast<const uint8_t*>(a.w) + v0 * a.ldw * element_bytes(a.dtype);
    s.ld = a.ldw;
    s.rows = n;
    s.dst = p.w;
    s.part_stride = p.piece * p.ldp;
    if (a.bias) s.zero_bias = a.bias + v0;
    return Split16Args{s, p.w16, p.piece * p.ldp, p.wunit};
}

Softmax softmax_of(const pvs_xent_args& a) {
    Softmax s{};
    s.k2 = a.scale * kLog2e;
    s.bias = a.bias;
    s.rows = (int)a.rows;
    return s;
}

FewArgs few_args(const pvs_xent_args& a) {
    FewArgs f{};
    f.x = static_cast<const float*>(a.x);
    f.ldx = a.ldx;
    f.rows = (int)a.rows;
    f.w = static_cast<const float*>(a.w);
    f.ldw = a.ldw;
    f.items = a.items;
    f.dim = a.dim;
    f.k2 = a.scale * kLog2e;
    f.bias = a.bias;
    f.targets = a.targets;
    f.ignore_index = a.ignore_index;
    f.scale = a.scale;
    return f;
}

cudaError_t forward(const pvs_xent_args& a, const Plan& p, const Device& dev, float* loss,
                    float* stats, cudaStream_t st) {
    cudaError_t e = cudaSuccess;
    const int64_t T = a.rows, V = a.items;
    if (p.few) {
        FewArgs f = few_args(a);
        f.part = p.part;
        f.part_rows = T;
        e = launch_few_stats(f, p.few, st);
    }
    Args g{};
    g.status = dev.status;
    g.sm = softmax_of(a);
    g.sm.part = p.part;
    g.sm.targets = a.targets;
    for (int64_t v0 = 0; !p.few && v0 < V && e == cudaSuccess; v0 += p.piece) {
        const int64_t n = std::min(p.piece, V - v0);
        PrepareArgs c{};
        if (p.copy_x && v0 == 0) c.copy[0] = rows_copy(a, p, false);
        if (p.copy_w) c.copy[1] = items_copy(a, p, v0, n);
        e = launch_prepare(c, st);
        if (e != cudaSuccess) break;
        g.sm.part0 = (int)(v0 / p.piece * p.piece_tiles);
        e = logits(kStats, g, p, a, v0, n, dev, st);
    }
    if (e != cudaSuccess) return e;
    const int64_t last = V - (p.pieces - 1) * p.piece;
    const int64_t tiles = p.few ? p.few : (p.pieces - 1) * p.piece_tiles + (last + p.bnl - 1) / p.bnl;
    const JoinArgs j{p.part, tiles, a, a.scale * kLog2e,
                     a.dtype != PVS_F32 && !p.copy_x && !p.copy_w && a.dim % 8 == 0, loss,
                     reinterpret_cast<float4*>(stats)};
    count_launches(1);
    if (T >= 4 * dev.sms) return launch_early(xent_join_kernel<8>, (T + 7) / 8, 256, 0, st, j);
    return launch_early(xent_join_kernel<1>, T, 256, 0, st, j);
}

cudaError_t backward(const pvs_xent_args& a, const Plan& p, const Device& dev, const float* stats,
                     const float* grad_loss, void* dx, int64_t lddx, void* dw, int64_t lddw,
                     cudaStream_t st) {
    const int64_t T = a.rows, V = a.items;
    float* up = reinterpret_cast<float*>(p.words);
    const float* undo = up + 1;
    int* bad_masked = reinterpret_cast<int*>(p.words + 2);
    cudaError_t e = cudaSuccess;
    if (p.f16) {
        count_launches(1);
        e = launch_early(xent_grad_scale_kernel, 1, 1024, 0, st, grad_loss, a.targets, a.ignore_index,
                         T, up);
    }
    if (p.few) {
        PrepareArgs c{};
        c.rows = RowArgs{reinterpret_cast<const float4*>(stats), grad_loss, a.targets, T, V,
                         a.ignore_index, nullptr, p.row, bad_masked};
        e = launch_prepare(c, st);
        for (int64_t v0 = 0; v0 < V && e == cudaSuccess; v0 += p.piece) {
            FewArgs f = few_args(a);
            f.w += v0 * a.ldw;
            f.items = std::min(p.piece, V - v0);
            f.item0 = v0;
            if (a.bias) f.bias += v0;
            f.row = p.row;
            f.g = p.few_g;
            f.slots = dx ? p.xslots : nullptr;
            f.slot_stride = T * p.lds;
            f.ldslot = p.lds;
            f.accumulate = v0 > 0;
            if (dw) f.dw = static_cast<float*>(dw) + v0 * lddw;
            f.lddw = lddw;
            e = launch_few_grads(f, p.few, st);
        }
        if (e == cudaSuccess && dx)
            e = launch_sum_slots(p.xslots, p.few, T * p.lds, p.lds, T, a.dim, nullptr, a.scale, dx,
                                 lddx, a.dtype, st);
        return e;
    }
    const Matrix x{p.x, T, a.dim, p.ldp, p.parts, T * p.ldp};
    const float* alpha = p.f16 ? undo : nullptr;
    for (int64_t v0 = 0, i = 0; v0 < V && e == cudaSuccess; v0 += p.piece, ++i) {
        const int64_t n = std::min(p.piece, V - v0);
        const Matrix direct{a.w, V, a.dim, a.ldw, 1, 0};
        const Matrix copied{p.w, n, a.dim, p.ldp, p.parts, p.piece * p.ldp};
        PrepareArgs c{};
        if (i == 0) {
            c.copy[0] = rows_copy(a, p, true);
            c.rows = RowArgs{reinterpret_cast<const float4*>(stats), grad_loss, a.targets, T, V,
                             a.ignore_index, p.f16 ? up : nullptr, p.row, bad_masked};
        }
        if (p.copy_w) c.copy[1] = items_copy(a, p, v0, n);
        e = launch_prepare(c, st);
        if (e != cudaSuccess) break;
        Args g{};
        g.status = dev.status;
        g.f16 = p.f16;
        g.sm = softmax_of(a);
        g.sm.row = p.row;
        g.sm.grad = p.g;
        g.sm.ldg = p.ldg;
        g.sm.grad_part = T * p.ldg;
        g.sm.grad_parts = p.gparts;
        g.sm.grad_f16 = p.f16;
        const bool alt = !p.copy_w && a.bias;
        if (alt) g.sm.bad_masked = bad_masked;
        e = logits(kGrad, g, p, a, v0, n, dev, st);
        // a masked item that holds NaN or infinities: dx takes w from a copy with zeros there
        if (e == cudaSuccess && alt && dx) {
            SplitArgs s = items_copy(a, p, v0, n).s;
            s.only_if = bad_masked;
            e = launch_split(s, st);
        }
        if (e != cudaSuccess) break;
        const Matrix gm{p.g, T, n, p.ldg, p.gparts, T * p.ldg};
        g.nprob = 0;
        g.f16 = p.f16;
        // dw's tiles have items for rows: pairs unless all of it is one CTA's tile
        g.cta = ctas_for(dw ? std::max(T, n) : T, dev);
        if (dx) {
            Problem& q = g.p[g.nprob++];
            q = Problem{};
            set_tiles(q, T, a.dim, p.bnd, n, g.cta);
            q.splits = even_splits(q.kchunks, p.xsplits);
            if (!operand_map(&q.a, gm, false, kTileM) ||
                !operand_map(&q.b, p.copy_w ? copied : direct, true, 0))
                return cudaErrorInvalidValue;
            q.b_mn = 1;
            q.b_ko = p.copy_w ? 0 : (int)v0;
            if (alt) {
                if (!operand_map(&q.b_alt, copied, true, 0)) return cudaErrorInvalidValue;
                q.alt_flag = bad_masked;
            }
            q.to_slots = p.xslots != nullptr;
            q.accumulate = i > 0;
            q.slots = p.xslots;
            q.slot_stride = T * p.lds;
            q.ldslot = p.lds;
            q.out = dx;
            q.ldout = lddx;
            q.out_type = a.dtype;
            q.alpha = alpha;
            q.alpha0 = a.scale;
        }
        Problem* qw = nullptr;
        if (dw) {
            Problem& q = g.p[g.nprob++];
            q = Problem{};
            set_tiles(q, n, a.dim, p.bnd, T, g.cta);
            q.splits = even_splits(q.kchunks, p.wsplits);
            if (!operand_map(&q.a, gm, true, 0) || !operand_map(&q.b, x, true, 0))
                return cudaErrorInvalidValue;
            q.a_mn = q.b_mn = 1;
            q.to_slots = q.splits > 1;
            q.slots = p.wslots;
            q.slot_stride = std::min(p.piece, V) * p.lds;
            q.ldslot = p.lds;
            q.out = static_cast<uint8_t*>(dw) + v0 * lddw * element_bytes(a.dtype);
            q.ldout = lddw;
            q.out_type = a.dtype;
            q.alpha = alpha;
            q.alpha0 = a.scale;
            qw = &q;
        }
        if (g.nprob == 0) break;
        if (n == std::min(p.piece, V)) g.slots0 = p.slots0;   // (the last piece: by its work)
        part_pairs(g, p.gparts, p.parts);
        e = launch_gemm(kOut, g, dev, st);
        if (e == cudaSuccess && qw && qw->to_slots)
            e = launch_sum_slots(p.wslots, qw->splits, qw->slot_stride, p.lds, n, a.dim, alpha,
                                 a.scale, qw->out, lddw, a.dtype, st);
    }
    if (e == cudaSuccess && dx && p.xslots)
        e = launch_sum_slots(p.xslots, p.xsplits, T * p.lds, p.lds, T, a.dim, alpha, a.scale, dx,
                             lddx, a.dtype, st);
    return e;
}

}  // namespace
}  // namespace head
}  // namespace pvs

using namespace pvs::head;

extern "C" pvs_status pvs_xent_workspace(const pvs_xent_args* a, int32_t backward, size_t* bytes) {
    if (!bytes || !valid(a)) return PVS_ERR_INVALID;
    *bytes = 0;
    if (a->rows == 0) return PVS_OK;
    Device dev;
    if (device(&dev) != cudaSuccess) {
        cudaGetLastError();
        return PVS_ERR_CUDA;
    }
    *bytes = backward ? plan_of(*a, true, dev, nullptr).bytes : forward_bytes(*a, dev);
    return PVS_OK;
}

// The device, an earlier timeout, and the workspace of a call.
static pvs_status begin(const void* workspace, size_t have, size_t want, const Device& dev) {
    if (have < want || (want > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))))
        return PVS_ERR_INVALID;
    return (pvs_status)take_status(dev);
}

static pvs_status ended(cudaError_t e) {
    if (e == cudaSuccess) return PVS_OK;
    cudaGetLastError();
    return PVS_ERR_CUDA;
}

extern "C" pvs_status pvs_xent_forward(const pvs_xent_args* a, float* loss, float* stats,
                                       void* workspace, size_t workspace_bytes,
                                       void* cuda_stream) {
    if (!valid(a)) return PVS_ERR_INVALID;
    if (a->rows == 0) return PVS_OK;
    if (!loss || !stats || !on_elements(loss, 4) || !on_elements(stats, 16)) return PVS_ERR_INVALID;
    Device dev;
    if (device(&dev) != cudaSuccess) return ended(cudaErrorUnknown);
    const pvs_status s = begin(workspace, workspace_bytes, forward_bytes(*a, dev), dev);
    if (s != PVS_OK) return s;
    cudaError_t e = cudaSuccess;
    const int64_t block = block_rows(*a);
    for (int64_t t0 = 0; t0 < a->rows && e == cudaSuccess; t0 += block) {
        const pvs_xent_args b = rows_of(*a, t0, std::min(block, a->rows - t0));
        e = forward(b, plan_of(b, false, dev, workspace), dev, loss + t0, stats + 4 * t0,
                    static_cast<cudaStream_t>(cuda_stream));
    }
    return ended(e);
}

extern "C" pvs_status pvs_xent_backward(const pvs_xent_args* a, const float* stats,
                                        const float* grad_loss, void* dx, int64_t lddx, void* dw,
                                        int64_t lddw, void* workspace, size_t workspace_bytes,
                                        void* cuda_stream) {
    if (!valid(a) || (dx && lddx < a->dim) || (dw && lddw < a->dim) ||
        !on_elements(dx, element_bytes(a->dtype)) || !on_elements(dw, element_bytes(a->dtype)))
        return PVS_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (a->rows == 0) {
        if (!dw) return PVS_OK;
        const size_t es = (size_t)element_bytes(a->dtype);
        return ended(cudaMemset2DAsync(dw, (size_t)lddw * es, 0, (size_t)a->dim * es,
                                       (size_t)a->items, st));
    }
    if (!stats || !grad_loss || !on_elements(stats, 16) || !on_elements(grad_loss, 4))
        return PVS_ERR_INVALID;
    Device dev;
    if (device(&dev) != cudaSuccess) return ended(cudaErrorUnknown);
    const Plan p = plan_of(*a, true, dev, workspace);
    const pvs_status s = begin(workspace, workspace_bytes, p.bytes, dev);
    if (s != PVS_OK) return s;
    if (!dx && !dw) return PVS_OK;
    return ended(backward(*a, p, dev, stats, grad_loss, dx, lddx, dw, lddw, st));
}

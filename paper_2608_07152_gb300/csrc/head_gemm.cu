// Persistent tcgen05 product of the projection head's operators (head_gemm.h).
//
// CTA pairs (the two SMs of a TPC, cta_group::2), one CTA per SM, 10 warps.  A unit
// of work is a tile of D (256 x bn) over a range of k; each CTA holds its own 128
// rows of A and half of B's rows, 32 KB a chunk.  A lone CTA needs 48 KB for 128 x
// 256, and its shared memory (fills and the MMAs' reads, 192 bytes a cycle at
// full rate where 128 are there) kept the tensor cores 62% busy; lone CTAs (kCta = 1)
// serve the products of 128 rows or fewer, which memory bounds (a loss of 100 rows over
// 500,000 items of 768: 125 us, in pairs 132; of 256 rows 140 in pairs, 155 in lone CTAs).
//
// 8,192 rows over 8,192 items of 768 in bf16: statistics 56 us (1.84 PFLOP/s, tensor
// pipe 87% busy), G 98 us (49%: two parts of 134 MB are stored), dx and dw 241 us (two
// products each, 1.71 PFLOP/s, 96%).  What is lost beside is the last, half empty, of 14 rounds of
// tiles.  (With lone lanes that issued, and moved each operand to where the instructions
// take it: 69, 117 and 287 us, 70%, 43% and 78%.)
//   warp 0     TMA producer (both CTAs): chunks of A (128 x 64) and B into a ring,
//              128-byte swizzle, the pair's bytes counted on the even CTA's barrier;
//   warp 1     (of the even CTA) issues the MMAs (M = 128 or 256, N = bn,
//              K = 16, four to a chunk) into one of two TMEM accumulators;
//   warps 2-9  epilogue (both CTAs): a TMEM lane (a row of D) per thread; the two
//              warps that share a lane quarter take every other chunk of 32 columns.
// Two accumulators let the epilogue of a unit run under the MMAs of the next.
// Of two problems in one launch each gets CTAs of its own, in proportion to its
// work, so that units of unlike lengths do not wait for one another.
//
// Operands.  K contiguous: a box is 64 elements of k (128 bytes) by the tile's
// rows.  M or N contiguous (gradients contract over rows): a box is 64 of m by
// 64 of k, so that the operand is never transposed in memory; the matrix
// descriptor's major bit and its strides say so.
//
// Softmax arithmetic is in powers of two: l = acc (a log2 e) + b log2 e, one FMA
// and one ex2 an entry; sums are float32 of at most 2^7 terms a thread and
// tile, joined in a fixed order, so a call's results do not depend on timing.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <climits>
#include <mutex>

#include "../../include/head.h"
#include "alloc.h"
#include "f32x2.cuh"
#include "head_gemm.h"
#include "kernels.h"
#include "pvs_common.cuh"
#include "tc.cuh"
#include "tensor_map.h"

namespace pvs {
namespace head {

constexpr int kStageA = kTileM * kTileK * 2;     // 16 KB
template <int kCta> struct Ring {
    static constexpr int kStageB = kTileN / kCta * kTileK * 2;   // this CTA's share of B
    static constexpr int kStageBytes = kStageA + kStageB;
    static constexpr int kStages = kCta == 2 ? 6 : 4;
};
constexpr int kMaxStages = 6;
constexpr int kEpiWarps = 8;     // two to a TMEM lane quarter (four were no faster)
constexpr int kEpiThreads = kEpiWarps * 32;
constexpr int kThreads = (2 + kEpiWarps) * 32;
constexpr uint32_t kTmemCols = 512;
constexpr float kLog2e = 1.4426950408889634f;

constexpr int kEpiGroups = kEpiWarps / 4;
static_assert(kEpiThreads >= kTileN, "an epilogue thread stages one column's bias");

struct Shared {
    uint64_t full[kMaxStages];
    uint64_t empty[kMaxStages];
    uint64_t tfull[2];
    uint64_t tempty[2];
    uint32_t tmem_base;
    int abort;                           // of the pair: set in both its CTAs
    uint32_t fills;                      // stages that this CTA has filled
    uint32_t chunks, tiles;              // even CTA: chunks and tiles committed
    uint32_t masked[2][kTileN / 32];     // items of the tile outside the softmax
    alignas(16) float b2[2][kTileN];     // their biases, in powers of two
    alignas(16) float unit[2][kTileN];   // what their logits are in units of
    float2 rowstat[2][kEpiGroups][kTileM];   // a tile's statistics, by the warps' shares of it
};

template <int kCta>
constexpr size_t smem_bytes() {
    return 1024 + (size_t)Ring<kCta>::kStages * Ring<kCta>::kStageBytes + sizeof(Shared);
}
static_assert(smem_bytes<1>() <= 227 * 1024 && smem_bytes<2>() <= 227 * 1024, "smem");

__device__ __forceinline__ bool abort_set(Shared& sh) {
    return *reinterpret_cast<volatile int*>(&sh.abort) != 0;
}
template <int kCta>
__device__ __forceinline__ void raise_abort(Shared& sh, int* status, int crank) {
    *reinterpret_cast<volatile int*>(&sh.abort) = 1;
    if (kCta == 2)
        asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(
                         cluster_map(&sh.abort, crank ^ 1)),
                     "r"(1)
                     : "memory");
    *reinterpret_cast<volatile int*>(status) = PVS_ERR_TIMEOUT;
}
// A wait of the ring: most have nothing to wait for, and do not look at the limit.
__device__ __forceinline__ bool ring_wait(uint64_t* bar, uint32_t parity, unsigned long long limit_ns) {
    return mbar_test_wait(bar, parity) || (limit_ns != 0 && mbar_wait(bar, parity, limit_ns));
}
// The same by a whole warp, so that what follows is uniform.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, unsigned long long limit_ns) {
    return __all_sync(0xffffffffu, ring_wait(bar, parity, limit_ns));
}
// A wait at a role's end, with the 2 s limit, given up in a millisecond where another role has
// given up (what it waits for may then never come).
template <int kCta>
__device__ __forceinline__ void last_wait(uint64_t* bar, uint32_t parity, Shared& sh, int* status,
                                          int crank) {
    constexpr unsigned long long kTurn = 1000000;
    for (unsigned long long t = 0; t < kWaitLimitNs; t += kTurn) {
        if (abort_set(sh) || mbar_wait(bar, parity, kTurn)) return;
    }
    raise_abort<kCta>(sh, status, crank);
}
// A word of a pair's CTA.
__device__ __forceinline__ uint32_t word_of(const uint32_t* p, int crank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_map(p, crank)) : "memory");
    return v;
}

// M or N contiguous with 128-byte swizzle: 64 elements of m (128 bytes) by 8 of
// k are an atom of 1024 bytes; SBO is the step to the next 8 of k, LBO to the
// next 64 of m (the boxes of 64 of k, 8 KB each, lie one after another).
__device__ __forceinline__ uint64_t smem_desc_sw128_mn(uint32_t smem_addr) {
    return tc::smem_desc_sw128_kmajor(smem_addr) | ((uint64_t)((kTileK * 128) >> 4) << 16);
}

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// A box into this CTA's shared memory, its bytes counted on the mbarrier at
// shared::cluster address `bar` (this CTA's or, of a pair, its peer's).
template <int kCta>
__device__ __forceinline__ void tma_load_3d(void* dst, const void* tmap, int x, int y, int z,
                                            uint32_t bar) {
    if constexpr (kCta == 2)
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
            "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
            "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
}

// 32 bytes to global memory, a whole sector.
__device__ __forceinline__ void store_32b(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]),
                 "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ void load_32b(const void* p, uint32_t* v) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]),
                   "=r"(v[6]), "=r"(v[7])
                 : "l"(p)
                 : "memory");
}

// A lane's 64 bytes of its row, rows `ld` elements apart: neighbouring lanes turn two rows' sectors
// round, so that a store writes 64 bytes of 16 rows, not 32 of 32 (G of 8,192 rows over 8,192
// items took 117 us that way; without any store 73).  `rows` of the warp's 32 exist.
__device__ __forceinline__ void store_two_rows(uint16_t* o, int64_t ld, const uint32_t (&h)[16], int rows) {
    const int lane = threadIdx.x & 31;
    const bool odd = lane & 1;
    uint32_t even_row[8], odd_row[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? h[i] : h[8 + i], 1);
        even_row[i] = odd ? got : h[i];
        odd_row[i] = odd ? h[8 + i] : got;
    }
    uint16_t* p = o - (odd ? ld : 0) + (odd ? 16 : 0);
    if ((lane & ~1) < rows) store_32b(p, even_row);
    if ((lane | 1) < rows) store_32b(p + ld, odd_row);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// The leading 8 bits of two values as bf16, and what is left of them.  Cutting
// (not rounding) makes the parts exact: three hold a float32's 24 bits, and no
// finite value becomes an infinity.
__device__ __forceinline__ uint32_t cut_bf16(float& lo, float& hi) {
    uint32_t l = __float_as_uint(lo) & 0xffff0000u, h = __float_as_uint(hi) & 0xffff0000u;
    if (lo != lo) l |= 0x00400000u;   // a NaN stays one
    if (hi != hi) h |= 0x00400000u;
    lo = isfinite(lo) ? lo - __uint_as_float(l) : 0.0f;
    hi = isfinite(hi) ? hi - __uint_as_float(h) : 0.0f;
    return (l >> 16) | h;
}

template <int kCta>
__device__ __forceinline__ void mma(uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc,
                                    uint32_t acc) {
    if constexpr (kCta == 2)
        tc::mma_f16_pair(d, ad, bd, idesc, acc);
    else
        tc::mma_bf16(d, ad, bd, idesc, acc);
}

// Two values rounded to f16, and what is left of them (nothing of what is not finite).
__device__ __forceinline__ uint32_t cut_f16(float& x, float& y) {
    const uint32_t h = pack_f16(x, y);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    x = isfinite(f.x) ? x - f.x : 0.0f;
    y = isfinite(f.y) ? y - f.y : 0.0f;
    return h;
}

// The units of one slot (a CTA, or a pair): those of one problem, `step` apart.  A unit
// is a tile and a range of k; the next one is found by additions with carries (its
// division by the tiles, in each of the three roles, cost a short unit as much as its
// MMAs).
struct Units {
    int prob, left;              // units still to come, this one included
    int mt, nt, split, k0, k1;   // this unit
    int a, b;                    // the faster and the slower tile index
    int na, nb, sa, sb, ss;      // their extents, and the step in them and in the splits
    int length, chunks;
    bool m_fast;

    __device__ __forceinline__ Units(const Args& args, int slot, int nslots) {
        prob = 0;
        int step = nslots;
        if (args.nprob > 1) {
            if (slot < args.slots0) {
                step = args.slots0;
            } else {
                prob = 1;
                slot -= args.slots0;
                step = nslots - args.slots0;
            }
        }
        const Problem& p = args.p[prob];
        left = slot < p.units ? (p.units - slot + step - 1) / step : 0;
        m_fast = p.m_fast;
        na = m_fast ? p.mtiles : p.ntiles;
        nb = m_fast ? p.ntiles : p.mtiles;
        a = slot % na;
        b = slot / na % nb;
        split = slot / na / nb;
        sa = step % na;
        sb = step / na % nb;
        ss = step / na / nb;
        length = p.klength;
        chunks = p.kchunks;
        place();
    }
    __device__ __forceinline__ void place() {
        mt = m_fast ? a : b;
        nt = m_fast ? b : a;
        k0 = split * length;
        k1 = min(k0 + length, chunks);
    }
    __device__ __forceinline__ void next() {
        --left;
        a += sa;
        b += sb;
        split += ss;
        if (a >= na) {
            a -= na;
            ++b;
        }
        if (b >= nb) {
            b -= nb;
            ++split;
        }
        place();
    }
};

// 32 float32 values of one row to `out` of any type: whole sectors where the
// row is aligned, 16 bytes at a time where it is to those (a step of 9 rows over 300,000
// items of 1,000 in bf16: 600 us, 1,077 by store_block), else one by one.  `valid` of them exist.
__device__ __forceinline__ void store_row(void* out, int type, int64_t at, const float (&v)[32],
                                          int valid) {
    if (type == PVS_F32) {
        float* o = static_cast<float*>(out) + at;
        if (valid == 32 && (reinterpret_cast<uintptr_t>(o) & 31u) == 0) {
#pragma unroll
            for (int i = 0; i < 32; i += 8)
                store_32b(o + i, reinterpret_cast<const uint32_t*>(&v[i]));
        } else if (valid == 32 && (reinterpret_cast<uintptr_t>(o) & 15u) == 0) {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
                *reinterpret_cast<float4*>(o + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < valid) o[i] = v[i];
        }
        return;
    }
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i)
        w[i] = type == PVS_BF16 ? pack_bf16(v[2 * i], v[2 * i + 1])
                                : pack_f16(v[2 * i], v[2 * i + 1]);
    uint16_t* o = static_cast<uint16_t*>(out) + at;
    if (valid == 32 && (reinterpret_cast<uintptr_t>(o) & 31u) == 0) {
        store_32b(o, w);
        store_32b(o + 16, w + 8);
    } else if (valid == 32 && (reinterpret_cast<uintptr_t>(o) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<uint4*>(o + 2 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i < valid) o[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}

// A block of 32 rows of `out` (a row per lane, `rows` and `valid` columns of which exist)
// that is not whole and aligned to 16 bytes: turned round among the warp's lanes, so that
// neighbours write neighbours.  Element by element from a row's lane, dw of 900,000 items
// of 385 (16 rows, bf16) made a step of 5,845 us; this way it takes 2,047.
__device__ __forceinline__ void store_block(void* out, int type, int64_t at, int64_t ld,
                                            float (&v)[32], int rows, int valid) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int bit = 16; bit > 0; bit >>= 1) {
        const bool upper = (lane & bit) != 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (i & bit) continue;
            const float got = __shfl_xor_sync(0xffffffffu, upper ? v[i] : v[i | bit], bit);
            v[i] = upper ? got : v[i];
            v[i | bit] = upper ? v[i | bit] : got;
        }
    }
    if (lane >= valid) return;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        if (i >= rows) break;
        const int64_t to = at + i * ld + lane;
        if (type == PVS_F32)
            static_cast<float*>(out)[to] = v[i];
        else
            static_cast<uint16_t*>(out)[to] =
                (uint16_t)(type == PVS_BF16 ? pack_bf16(v[i], 0.0f) : pack_f16(v[i], 0.0f));
    }
}

// A tile's statistics of one row, from its shares, in their order.
__device__ __forceinline__ void write_stats(const float2 (&share)[kEpiGroups][kTileM],
                                            const Softmax& sm, int at, int row, int row_in_tile) {
    if (row >= sm.rows) return;
    float m = -INFINITY, s = 0.0f;
#pragma unroll
    for (int g = 0; g < kEpiGroups; ++g) m = fmaxf(m, share[g][row_in_tile].x);
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int g = 0; g < kEpiGroups; ++g) {
        const float2 p = share[g][row_in_tile];
        s += p.y * ex2(p.x - ref);
    }
    sm.part[(int64_t)at * sm.rows + row] = make_float2(m, s);
}

// The copies of one fill of a stage, this CTA's share.
struct Producer {
    const Problem& p;
    const CUtensorMap* b;
    int nbox;                    // boxes of B, where N is its contiguous index
    uint32_t bytes;              // of a stage, of both CTAs

    __device__ __forceinline__ Producer(const Problem& p, bool alt, int kcta) : p(p) {
        const int bhalf = p.bn / kcta;                  // rows of B that this CTA supplies
        b = alt ? &p.b_alt : &p.b;
        nbox = (bhalf + 63) / 64;
        bytes = kcta * (kStageA + (uint32_t)(p.b_mn ? nbox * 64 : bhalf) * kTileK * 2u);
    }
    template <int kCta>
    __device__ __forceinline__ void fill(uint8_t* stage, uint64_t* full, bool leader, int am, int ka,
                                         int pa, int bn, int kb, int pb) const {
        uint8_t* sb = stage + kStageA;
        if (leader) mbar_arrive_expect_tx(full, bytes);
        const uint32_t bar = kCta == 2 ? cluster_map(full, 0) : smem_u32(full);
        if (p.a_mn) {
            tma_load_3d<kCta>(stage, &p.a, am, ka, pa, bar);
            tma_load_3d<kCta>(stage + kTileK * 128, &p.a, am + 64, ka, pa, bar);
        } else {
            tma_load_3d<kCta>(stage, &p.a, ka, am, pa, bar);
        }
        if (p.b_mn) {
            for (int i = 0; i < nbox; ++i)
                tma_load_3d<kCta>(sb + i * kTileK * 128, b, bn + 64 * i, kb, pb, bar);
        } else {
            tma_load_3d<kCta>(sb, b, kb, bn, pb, bar);
        }
    }
};

// After a wait that ran out: one thread of each CTA waits for what is still on its way to its
// CTA, which must not end before.  Fills first: those that the other CTA of the pair has issued
// and this one has not are issued here (the stage is free, or the other would not have filled
// it; what is read does not matter), so that every `full` barrier completes.  Then the MMAs and
// their commits.  With the 2 s limit; after one that runs out nothing more is waited for.
template <int kCta>
__device__ __noinline__ void settle(Shared& sh, uint8_t* stages, const Problem& p, int crank) {
    using R = Ring<kCta>;
    const Producer make(p, false, kCta);
    const uint32_t mine = sh.fills;
    const uint32_t fills = kCta == 2 ? max(mine, word_of(&sh.fills, crank ^ 1)) : mine;
    for (uint32_t g = mine; g < fills; ++g) {
        const int s = g % R::kStages;
        make.fill<kCta>(stages + s * R::kStageBytes, &sh.full[s], crank == 0, p.a_mo, p.a_ko, 0, p.b_no,
                        p.b_ko, 0);
    }
    const uint32_t chunks = kCta == 2 ? word_of(&sh.chunks, 0) : sh.chunks;
    const uint32_t tiles = kCta == 2 ? word_of(&sh.tiles, 0) : sh.tiles;
    bool in_time = true;
    for (uint32_t s = 0; s < (uint32_t)R::kStages; ++s) {
        if (in_time && crank == 0 && s < fills)
            in_time = mbar_wait(&sh.full[s], ((fills - 1 - s) / R::kStages) & 1u);
        if (in_time && s < chunks) in_time = mbar_wait(&sh.empty[s], ((chunks - 1 - s) / R::kStages) & 1u);
    }
    for (uint32_t b = 0; b < 2; ++b)
        if (in_time && b < tiles) in_time = mbar_wait(&sh.tfull[b], ((tiles - 1 - b) / 2) & 1u);
}

template <int EPI, int kCta>
__global__ void __launch_bounds__(kThreads, 1) head_gemm_kernel(const __grid_constant__ Args a) {
    using R = Ring<kCta>;
    extern __shared__ uint8_t smem_raw[];
    // the layout is the same in both CTAs of a pair: barriers and the pair's MMAs are
    // addressed by offset
    const uint32_t raw_addr = smem_u32(smem_raw);
    uint8_t* stages = smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
    Shared& sh = *reinterpret_cast<Shared*>(stages + R::kStages * R::kStageBytes);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int crank = kCta == 2 ? (int)cluster_ctarank() : 0;
    const bool leader = crank == 0;
    Units w(a, blockIdx.x / kCta, gridDim.x / kCta);
    const Problem& p = a.p[w.prob];

    if (threadIdx.x == 0) {
        for (int s = 0; s < R::kStages; ++s) {
            mbar_init(&sh.full[s], 1);
            mbar_init(&sh.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sh.tfull[b], 1);
            mbar_init(&sh.tempty[b], kCta * kEpiWarps);   // both CTAs' epilogue warps
        }
        sh.abort = 0;
        sh.fills = sh.chunks = sh.tiles = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        if (kCta == 2)
            tc::tmem_alloc_pair(&sh.tmem_base, kTmemCols);
        else
            tc::tmem_alloc(&sh.tmem_base, kTmemCols);
        tc::fence_before_sync();
    }
    __syncthreads();
    if (kCta == 2) cluster_barrier();   // both CTAs' barriers and TMEM are ready
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem_base, 0);
    next_early();
    wait_before();

    // The producer's and the issuer's loops are run by whole warps, one lane of which issues: their
    // addresses and descriptors then stay in uniform registers, where the instructions want them.
    if (warp == 0) {
        // ---------------- TMA producer ----------------
        const bool one = tc::elect_one();
        uint32_t g = 0;
        Turn at;
        bool go = true;
        const bool alt = p.alt_flag && *p.alt_flag;
        const int bhalf = p.bn / kCta;
        const Producer make(p, alt, kCta);
        for (; go && w.left > 0; w.next()) {
            if (__any_sync(0xffffffffu, abort_set(sh))) break;
            const int am = p.a_mo + (w.mt * kCta + crank) * kTileM;
            const int bnc = (alt ? p.alt_no : p.b_no) + w.nt * p.bn + crank * bhalf;
            const int bk = alt ? p.alt_ko : p.b_ko;
            for (int q = 0; go && q < a.npairs; ++q) {
                const int pa = a.pa[q], pb = a.pb[q];
                for (int kc = w.k0; kc < w.k1; ++kc, ++g, at.next(R::kStages)) {
                    go = warp_wait(&sh.empty[at.stage], at.parity ^ 1u, a.wait_ns);
                    if (!go) break;
                    if (one)
                        make.fill<kCta>(stages + at.stage * R::kStageBytes, &sh.full[at.stage], leader, am,
                                        p.a_ko + kc * kTileK, pa, bnc, bk + kc * kTileK, pb);
                }
            }
        }
        if (one) {
            if (!go) raise_abort<kCta>(sh, a.status, crank);
            sh.fills = g;
            // the MMAs have consumed the last fill of every stage used: no copy into
            // this CTA and no commit to its barriers is still in flight when it ends
            for (int s = 0; s < R::kStages && (uint32_t)s < g; ++s) {
                const uint32_t last = g - 1 - ((g - 1 - s) % R::kStages);
                last_wait<kCta>(&sh.empty[s], (last / R::kStages) & 1u, sh, a.status, crank);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------- MMA issuer (the even CTA of a pair) ----------------
        if (leader) {
            const bool one = tc::elect_one();
            const uint32_t idesc = (a.f16 ? tc::idesc_f16_f32(kTileM * kCta, p.bn)
                                          : tc::idesc_bf16_f32(kTileM * kCta, p.bn)) |
                                   ((uint32_t)p.a_mn << 15) | ((uint32_t)p.b_mn << 16);
            // the first stage's descriptors, and their steps of 16 of k (32 bytes, or two
            // atoms): the upper halves do not change, the address is in the lower ones
            const uint32_t s0 = smem_u32(stages);
            const uint64_t a0 = p.a_mn ? smem_desc_sw128_mn(s0) : tc::smem_desc_sw128_kmajor(s0);
            const uint64_t b0 = p.b_mn ? smem_desc_sw128_mn(s0 + kStageA)
                                       : tc::smem_desc_sw128_kmajor(s0 + kStageA);
            const uint32_t a_hi = (uint32_t)(a0 >> 32), b_hi = (uint32_t)(b0 >> 32);
            auto desc = [](uint32_t hi, uint32_t lo) { return (uint64_t)hi << 32 | lo; };
            const uint32_t astep = p.a_mn ? 128 : 2, bstep = p.b_mn ? 128 : 2;
            uint32_t g = 0;
            int it = 0;
            Turn at;
            bool go = true;
            for (; w.left > 0; w.next(), ++it) {
                const int b = it & 1;
                if (__any_sync(0xffffffffu, abort_set(sh))) break;
                go = warp_wait(&sh.tempty[b], ((uint32_t)(it >> 1) & 1u) ^ 1u, a.wait_ns);
                if (!go) break;
                tc::fence_after_sync();
                const uint32_t d = tmem + (uint32_t)(b * kTileN);
                const int chunks = a.npairs * (w.k1 - w.k0);
                int in_k = w.k0;
                const bool tail = w.k1 == p.kchunks && p.ktail < kTileK / 16;
                for (int kc = 0; kc < chunks; ++kc, ++g, at.next(R::kStages)) {
                    go = warp_wait(&sh.full[at.stage], at.parity, a.wait_ns);
                    if (!go) break;
                    tc::fence_after_sync();
                    const uint32_t off = at.stage * (uint32_t)(R::kStageBytes >> 4);
                    const uint32_t al = (uint32_t)a0 + off, bl = (uint32_t)b0 + off;
                    if (++in_k == w.k1) in_k = w.k0;
                    // the last chunk's steps past k multiply zeros: left out
                    const int steps = tail && in_k == w.k0 ? p.ktail : kTileK / 16;
                    if (one) {
#pragma unroll
                        for (int k = 0; k < kTileK / 16; ++k) {
                            if (k >= steps) break;
                            mma<kCta>(d, desc(a_hi, al + k * astep), desc(b_hi, bl + k * bstep), idesc,
                                      k > 0 || kc > 0 ? 1u : 0u);
                        }
                        if (kCta == 2)
                            tc::commit_pair(&sh.empty[at.stage]);   // the stage is free in both CTAs
                        else
                            tc::commit(&sh.empty[at.stage]);
                    }
                    __syncwarp();
                }
                if (!go) break;
                if (one) {
                    if (kCta == 2)
                        tc::commit_pair(&sh.tfull[b]);
                    else
                        tc::commit(&sh.tfull[b]);
                }
                __syncwarp();
            }
            if (one) {
                if (!go) raise_abort<kCta>(sh, a.status, crank);
                sh.chunks = g;
                sh.tiles = it;
                // TMEM is released after the last unit's MMAs
                if (it > 0) {
                    const int lb = (it - 1) & 1;
                    last_wait<kCta>(&sh.tfull[lb], (uint32_t)((it - 1) >> 1) & 1u, sh, a.status, crank);
                }
            }
            __syncwarp();
        }
    } else {
        // ---------------- epilogue ----------------
        const int quarter = warp & 3;            // TMEM lanes 32 * quarter ..
        const int group = (warp - 2) >> 2;       // this warp's chunks of 32 columns
        const int et = threadIdx.x - 64;
        const int row_in_tile = quarter * 32 + lane;
        const Softmax& sm = a.sm;
        const uint32_t tempty_at[2] = {kCta == 2 ? cluster_map(&sh.tempty[0], 0) : 0u,
                                       kCta == 2 ? cluster_map(&sh.tempty[1], 0) : 0u};
        constexpr bool kAnyStats = EPI == kStats || EPI == kTopStats;
        int it = 0;
        [[maybe_unused]] int part_at = 0, row_before = 0;
        bool dead = false;
        for (; w.left > 0; w.next(), ++it) {
            const int b = it & 1;
            const int row = (w.mt * kCta + crank) * kTileM + row_in_tile;
            const int n0 = w.nt * p.bn;
            const int ncols = min(p.bn, p.n - n0);      // columns of D in the tile
            [[maybe_unused]] int64_t y = -1;
            [[maybe_unused]] float row_k2 = 0.0f;
            [[maybe_unused]] uint32_t yt = ~0u, targets_in = 0;   // the target's column, chunks with one
            [[maybe_unused]] GradRow gr;
            [[maybe_unused]] int listed = INT_MAX, list_left = 0;   // the row's next listed item
            [[maybe_unused]] const int* list = nullptr;
            if constexpr (EPI != kOut) {
                // the tile's biases, and which of its columns are in the softmax
                const int item = sm.item0 + n0 + et;
                float bv = 0.0f;
                if (sm.bias && et < ncols) {
                    bv = __ldg(sm.bias + item);
                    // a finite bias stays one in powers of two
                    if (isfinite(bv)) bv = fminf(fmaxf(bv * kLog2e, -3.402823466e38f), 3.402823466e38f);
                }
                if (et >= ncols) bv = -INFINITY;
                const uint32_t mask = __ballot_sync(0xffffffffu, bv == -INFINITY);
                if (et < kTileN) {
                    sh.b2[b][et] = bv;
                    if (sm.col_unit) sh.unit[b][et] = et < ncols ? __ldg(sm.col_unit + n0 + et) : 0.0f;
                    if (lane == 0) sh.masked[b][et >> 5] = mask;
                }
                if constexpr (EPI == kTopStats) {
                    if (row < sm.rows) {
                        const int at = __ldg(sm.list_first + (int64_t)(sm.part0 + w.nt) * sm.rows + row);
                        list = sm.list + (int64_t)row * sm.top + at;
                        list_left = sm.top - at;
                        if (list_left > 0) listed = __ldg(list);
                    }
                } else if constexpr (EPI == kStats) {
                    if (row < sm.rows) y = __ldg(sm.targets + row) - (sm.item0 + n0);
                } else {
                    gr = GradRow{0.0f, 0.0f, 0.0f, -1};
                    if (row < sm.rows) {
                        const float4 r4 = __ldg(reinterpret_cast<const float4*>(sm.row + row));
                        gr = GradRow{r4.x, r4.y, r4.z, __float_as_int(r4.w)};
                    }
                    y = gr.y < 0 ? -1 : (int64_t)gr.y - (sm.item0 + n0);
                }
                row_k2 = sm.row_unit && row < sm.rows ? sm.k2 * __ldg(sm.row_unit + row) : sm.k2;
                yt = y >= 0 && y < kTileN ? (uint32_t)y : ~0u;
                targets_in = __reduce_or_sync(0xffffffffu, yt < kTileN ? 1u << (yt >> 5) : 0u);
                asm volatile("bar.sync 1, %0;" ::"n"(kEpiThreads) : "memory");
                if constexpr (kAnyStats) {
                    // the tile before this one: all its shares are in shared memory
                    if (it > 0 && group == 0)
                        write_stats(sh.rowstat[b ^ 1], sm, part_at, row_before, row_in_tile);
                    part_at = sm.part0 + w.nt;
                    row_before = row;
                }
            }
            // after a wait that ran out, the warps still meet at every barrier
            if (!dead) {
                bool late = abort_set(sh);
                if (!late && !ring_wait(&sh.tfull[b], (uint32_t)(it >> 1) & 1u, a.wait_ns)) {
                    raise_abort<kCta>(sh, a.status, crank);
                    late = true;
                }
                dead = __any_sync(0xffffffffu, late);
            }
            if (dead) continue;
            tc::fence_after_sync();
            const uint32_t tcol =
                tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(b * kTileN);
            [[maybe_unused]] float mx = -INFINITY, sum = 0.0f;
            // (rows of D in `out` start on 16 bytes, and so do their chunks)
            [[maybe_unused]] const bool out_whole =
                ((reinterpret_cast<uintptr_t>(p.out) |
                  (uintptr_t)p.ldout * (p.out_type == PVS_F32 ? 4 : 2)) & 15u) == 0;
            for (int cc = group; cc * 32 < p.bn; cc += kEpiGroups) {
                uint32_t r[32];
                __syncwarp();
                tc::ld_32x32b_x32(tcol + (uint32_t)(cc * 32), r);
                tc::wait_ld();
                if constexpr (EPI == kOut) {
                    const int valid = min(32, ncols - cc * 32);
                    float v[32];
                    if (p.to_slots) {
                        if (row >= p.m || valid <= 0) continue;   // nothing of D here
                        float* o = p.slots + w.split * p.slot_stride + (int64_t)row * p.ldslot +
                                   n0 + cc * 32;
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
                        if (p.accumulate) {
                            if (valid == 32 && (reinterpret_cast<uintptr_t>(o) & 31u) == 0) {
#pragma unroll
                                for (int i = 0; i < 32; i += 8) {
                                    uint32_t old[8];
                                    load_32b(o + i, old);
#pragma unroll
                                    for (int j = 0; j < 8; ++j) v[i + j] += __uint_as_float(old[j]);
                                }
                            } else {
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (i < valid) v[i] += o[i];
                            }
                        }
                        store_row(o, PVS_F32, 0, v, valid);
                    } else if (row - lane < p.m && valid > 0) {
                        const float alpha = p.alpha ? p.alpha0 * __ldg(p.alpha) : p.alpha0;
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]) * alpha;
                        const int64_t at = (int64_t)row * p.ldout + n0 + cc * 32;
                        if (valid == 32 && out_whole) {
                            if (row < p.m) store_row(p.out, p.out_type, at, v, 32);
                        } else {
                            store_block(p.out, p.out_type, at - lane * p.ldout, p.ldout, v,
                                        p.m - (row - lane), valid);
                        }
                    }
                } else {
                    const uint32_t mask = sh.masked[b][cc];
                    float v[32];
                    [[maybe_unused]] bool bad = false;
                    if (sm.col_unit) {
                        // (the powers of two first: neither may leave the range alone)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            r[i] = __float_as_uint(__uint_as_float(r[i]) *
                                                   (row_k2 * sh.unit[b][cc * 32 + i]));
                    }
                    // the logits are v f: where nothing but the scale is to be done, one FMA takes
                    // it and the reference off together
                    float f = sm.col_unit ? 1.0f : sm.k2;
                    if (sm.bias || mask) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float l = fmaf(__uint_as_float(r[i]), f, sh.b2[b][cc * 32 + i]);
                            const bool out = (mask >> i) & 1u;
                            v[i] = out ? -INFINITY : l;
                            // a masked item that holds an infinity or a NaN has no finite
                            // product with any row (its l does not tell: -inf for one of -inf)
                            if (EPI == kGrad)
                                bad |= out && !(fabsf(__uint_as_float(r[i])) <= 3.402823466e38f);
                        }
                        f = 1.0f;
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
                    }
                    // the column of the row's target, as a bit, where a row has one here
                    bool any_here = (targets_in >> cc) & 1u;
                    uint32_t here = (yt >> 5) == (uint32_t)cc ? 1u << (yt & 31u) : 0u;
                    if constexpr (EPI == kTopStats) {
                        // those of the listed items (past the other warps' chunks)
                        const int first = sm.item0 + n0 + cc * 32;
                        auto advance = [&] { listed = --list_left > 0 ? __ldg(++list) : INT_MAX; };
                        while (listed < first) advance();
                        while (listed - first < 32) {
                            here |= 1u << (listed - first);
                            advance();
                        }
                        any_here = __any_sync(0xffffffffu, here != 0);
                    }
                    const uint64_t ff = f2_pack(f, f);
                    if constexpr (kAnyStats) {
                        if (any_here) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                v[i] = here & (1u << i) ? -INFINITY : v[i];
                        }
                        float c0 = v[0], c1 = v[1];
#pragma unroll
                        for (int i = 2; i < 32; i += 2) {
                            c0 = fmaxf(c0, v[i]);
                            c1 = fmaxf(c1, v[i + 1]);
                        }
                        const float nm = fmaxf(mx, fmaxf(c0, c1) * f);
                        const float ref = nm == -INFINITY ? 0.0f : nm;
                        const uint64_t off = f2_pack(-ref, -ref);
                        uint64_t s0 = 0, s1 = 0;                 // pairs of zeros
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            float e0, e1, e2, e3;
                            f2_unpack(f2_fma(f2_pack(v[i], v[i + 1]), ff, off), e0, e1);
                            f2_unpack(f2_fma(f2_pack(v[i + 2], v[i + 3]), ff, off), e2, e3);
                            s0 = f2_add(s0, f2_pack(ex2(e0), ex2(e1)));
                            s1 = f2_add(s1, f2_pack(ex2(e2), ex2(e3)));
                        }
                        float p0, p1;
                        f2_unpack(f2_add(s0, s1), p0, p1);
                        sum = sum * ex2(mx - ref) + (p0 + p1);
                        mx = nm;
                    } else {
                        if (bad && row < sm.rows && sm.bad_masked)
                            *reinterpret_cast<volatile int*>(sm.bad_masked) = 1;
                        if (gr.coef == 0.0f && gr.hit == 0.0f) {
                            // (whatever the row holds)
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = 0.0f;
                        } else {
                            const uint64_t off = f2_pack(-gr.m, -gr.m), by = f2_pack(gr.coef, gr.coef);
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                float e0, e1;
                                f2_unpack(f2_fma(f2_pack(v[i], v[i + 1]), ff, off), e0, e1);
                                f2_unpack(f2_mul(f2_pack(ex2(e0), ex2(e1)), by), v[i], v[i + 1]);
                            }
                        }
                        __syncwarp();
                        if (any_here) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                v[i] = here & (1u << i) ? gr.hit : v[i];
                        }
                        // (a row of grad has room for the chunk that its last column is in)
                        if (row - lane < sm.rows && cc * 32 < ncols) {
                            uint16_t* o = sm.grad + (int64_t)row * sm.ldg + n0 + cc * 32;
                            for (int part = 0; part < sm.grad_parts; ++part) {
                                uint32_t h[16];
#pragma unroll
                                for (int i = 0; i < 16; ++i)
                                    h[i] = part + 1 < sm.grad_parts
                                               ? (sm.grad_f16 ? cut_f16(v[2 * i], v[2 * i + 1])
                                                              : cut_bf16(v[2 * i], v[2 * i + 1]))
                                           : sm.grad_f16 ? pack_f16(v[2 * i], v[2 * i + 1])
                                                         : pack_bf16(v[2 * i], v[2 * i + 1]);
                                store_two_rows(o, sm.ldg, h, sm.rows - (row - lane));
                                o += sm.grad_part;
                            }
                        }
                    }
                }
            }
            if constexpr (kAnyStats)
                sh.rowstat[b][group][row_in_tile] = make_float2(mx, sum);
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (kCta == 2)
                    mbar_arrive_remote(tempty_at[b]);   // the even CTA's barrier (or its own)
                else
                    mbar_arrive(&sh.tempty[b]);
            }
        }
        if constexpr (kAnyStats) {
            __syncwarp();
            asm volatile("bar.sync 1, %0;" ::"n"(kEpiThreads) : "memory");
            if (it > 0 && group == 0)
                write_stats(sh.rowstat[(it - 1) & 1], sm, part_at, row_before, row_in_tile);
        }
    }
    __syncthreads();
    if (kCta == 2) cluster_barrier();   // no CTA leaves while its peer may still address it
    if (abort_set(sh)) {
        if (threadIdx.x == 0) settle<kCta>(sh, stages, p, crank);
        __syncthreads();
        if (kCta == 2) cluster_barrier();
    }
    if (warp == 1) {
        tc::fence_after_sync();
        if (kCta == 2)
            tc::tmem_dealloc_pair(tmem, kTmemCols);
        else
            tc::tmem_dealloc(tmem, kTmemCols);
    }
}

// ---- sums over the splits ------------------------------------------------------
// Four columns a thread, all of them added in the splits' order.  Small blocks of one
// round each: what a sum waits for is its chain of loads (8 rows of 768
// from 152 splits took 66 us with two rounds a block, 38 in one).
constexpr int kSumThreads = 128;
__global__ void __launch_bounds__(kSumThreads) sum_slots_kernel(
    const float* __restrict__ slots, int splits, int64_t slot_stride, int64_t ldslot, int64_t rows,
    int n, int blocks_per_row, int rows_per_block, const float* __restrict__ alpha, float alpha0,
    void* __restrict__ out, int64_t ldout, int out_type, const float* __restrict__ row_scales,
    const float* __restrict__ col_scales) {
    next_early();
    wait_before();
    const int pieces = (n + 3) / 4;
    const float f = alpha ? alpha0 * __ldg(alpha) : alpha0;
    int64_t row = (int64_t)blockIdx.x * rows_per_block;
    int piece = threadIdx.x;
    if (blocks_per_row > 1) {
        row = blockIdx.x / blocks_per_row;
        piece += (int)(blockIdx.x % blocks_per_row) * kSumThreads;
    } else {
        row += threadIdx.x / pieces;
        piece = threadIdx.x % pieces;
        if (threadIdx.x >= rows_per_block * pieces) return;
    }
    if (row < rows && piece < pieces) {
        const int col = piece * 4;
        // (a slot's rows are padded to eight columns)
        const float* p = slots + row * ldslot + col;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        // (sixteen loads in flight; added in the splits' order)
        int k = 0;
        for (; k + 16 <= splits; k += 16) {
            float4 v[16];
#pragma unroll
            for (int u = 0; u < 16; ++u)
                v[u] = __ldg(reinterpret_cast<const float4*>(p + (k + u) * slot_stride));
#pragma unroll
            for (int u = 0; u < 16; ++u)
                s.x += v[u].x, s.y += v[u].y, s.z += v[u].z, s.w += v[u].w;
        }
#pragma unroll 4
        for (; k < splits; ++k) {
            const float4 v = __ldg(reinterpret_cast<const float4*>(p + k * slot_stride));
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        s.x *= f, s.y *= f, s.z *= f, s.w *= f;
        if (col_scales) {
            const float r = __ldg(row_scales + row);
            const float* c = col_scales + col;
            s.x = times_scales(s.x, r, __ldg(c));
            if (col + 1 < n) s.y = times_scales(s.y, r, __ldg(c + 1));
            if (col + 2 < n) s.z = times_scales(s.z, r, __ldg(c + 2));
            if (col + 3 < n) s.w = times_scales(s.w, r, __ldg(c + 3));
        }
        const int64_t at = row * ldout + col;
        if (out_type == PVS_F32) {
            float* o = static_cast<float*>(out) + at;
            if (col + 4 <= n && (reinterpret_cast<uintptr_t>(o) & 15u) == 0) {
                *reinterpret_cast<float4*>(o) = s;
            } else {
                o[0] = s.x;
                if (col + 1 < n) o[1] = s.y;
                if (col + 2 < n) o[2] = s.z;
                if (col + 3 < n) o[3] = s.w;
            }
        } else {
            uint16_t* o = static_cast<uint16_t*>(out) + at;
            const uint32_t lo = out_type == PVS_BF16 ? pack_bf16(s.x, s.y) : pack_f16(s.x, s.y);
            const uint32_t hi = out_type == PVS_BF16 ? pack_bf16(s.z, s.w) : pack_f16(s.z, s.w);
            if (col + 4 <= n && (reinterpret_cast<uintptr_t>(o) & 7u) == 0) {
                *reinterpret_cast<uint2*>(o) = make_uint2(lo, hi);
            } else {
                o[0] = (uint16_t)lo;
                if (col + 1 < n) o[1] = (uint16_t)(lo >> 16);
                if (col + 2 < n) o[2] = (uint16_t)hi;
                if (col + 3 < n) o[3] = (uint16_t)(hi >> 16);
            }
        }
    }
}

// The same, one column a thread and 32 loads in flight: where four columns a thread leave the SMs
// few threads (200 rows of 385 from 196 splits took 52 us with four columns).
constexpr int kSumFlight = 32;
__global__ void __launch_bounds__(kSumThreads) sum_columns_kernel(
    const float* __restrict__ slots, int splits, int64_t slot_stride, int64_t ldslot, int n, int blocks_per_row,
    const float* __restrict__ alpha, float alpha0, void* __restrict__ out, int64_t ldout, int out_type,
    const float* __restrict__ row_scales, const float* __restrict__ col_scales) {
    next_early();
    wait_before();
    const float f = alpha ? alpha0 * __ldg(alpha) : alpha0;
    const int64_t row = quotient_of(blockIdx.x, blocks_per_row);
    const int col = (int)(blockIdx.x - row * blocks_per_row) * kSumThreads + threadIdx.x;
    if (col >= n) return;
    const float* p = slots + row * ldslot + col;
    float s = 0.0f;
    int k = 0;
    for (; k + kSumFlight <= splits; k += kSumFlight) {
        float v[kSumFlight];
#pragma unroll
        for (int u = 0; u < kSumFlight; ++u) v[u] = __ldg(p + (k + u) * slot_stride);
#pragma unroll
        for (int u = 0; u < kSumFlight; ++u) s += v[u];
    }
#pragma unroll 8
    for (; k < splits; ++k) s += __ldg(p + k * slot_stride);
    s *= f;
    if (col_scales) s = times_scales(s, __ldg(row_scales + row), __ldg(col_scales + col));
    if (out_type == PVS_F32)
        static_cast<float*>(out)[row * ldout + col] = s;
    else
        static_cast<uint16_t*>(out)[row * ldout + col] =
            (uint16_t)(out_type == PVS_BF16 ? pack_bf16(s, 0.0f) : pack_f16(s, 0.0f));
}

cudaError_t launch_sum_slots(const float* slots, int splits, int64_t slot_stride, int64_t ldslot,
                             int64_t m, int n, const float* alpha, float alpha0, void* out,
                             int64_t ldout, int out_type, const Device& dev, cudaStream_t st,
                             const float* row_scales, const float* col_scales) {
    const int pieces = (n + 3) / 4;
    count_launches(1);
    // (less than eight such blocks an SM)
    if (splits >= 16 && m * pieces < (int64_t)dev.sms * 8 * kSumThreads) {
        const int per_row = (n + kSumThreads - 1) / kSumThreads;
        return launch_early(sum_columns_kernel, m * per_row, kSumThreads, 0, st, slots, splits, slot_stride, ldslot,
                            n, per_row, alpha, alpha0, out, ldout, out_type, row_scales, col_scales);
    }
    const int blocks_per_row = (pieces + kSumThreads - 1) / kSumThreads;
    const int rows_per_block = std::max(1, kSumThreads / pieces);
    const int64_t blocks = blocks_per_row > 1 ? m * blocks_per_row : (m + rows_per_block - 1) / rows_per_block;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_early(sum_slots_kernel, blocks, kSumThreads, 0, st, slots, splits, slot_stride, ldslot,
                        m, n, blocks_per_row, rows_per_block, alpha, alpha0, out, ldout, out_type, row_scales,
                        col_scales);
}

// ---- operands in 16-bit parts ----------------------------------------------------
__device__ __forceinline__ float load_as_float(const void* p, int dtype, int64_t i) {
    if (dtype == PVS_F32) return static_cast<const float*>(p)[i];
    if (dtype == PVS_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

// Eight consecutive elements a thread, in one load (two of float32) where rows are
// aligned; n / pieces by a product: m = floor(2^40 / pieces) + 1 is exact for what a block has.
__device__ __forceinline__ void split_rows(const SplitArgs& a, int64_t block, int64_t blocks) {
    const int pieces = (a.cols + 7) / 8, per_block = a.per_block, wide = a.wide;
    const uint64_t m = a.magic;
    const int64_t step = blocks * per_block;
    for (int64_t row0 = block * per_block; row0 < a.rows; row0 += step) {
        const uint32_t total = (uint32_t)(min((int64_t)per_block, a.rows - row0) * pieces);
        for (uint32_t i = threadIdx.x; i < total; i += 256) {
            const uint32_t r = (uint32_t)((i * m) >> 40);
            const int64_t row = row0 + r;
            const int col = (int)(i - r * (uint32_t)pieces) * 8;
            const bool zero = ignored_row(a.zero_target, a.ignore_index, a.zero_stats, row) ||
                              (a.zero_bias && a.zero_bias[row] == -INFINITY);
            const int64_t at = row * a.ld + col;
            float v[8];
            if (wide && col + 8 <= a.cols) {
                if (a.dtype == PVS_F32) {
                    const float4* p =
                        reinterpret_cast<const float4*>(static_cast<const float*>(a.src) + at);
                    const float4 x = __ldg(p), y = __ldg(p + 1);
                    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
                    v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
                } else {
                    const uint4 x = __ldg(
                        reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.src) + at));
                    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const uint32_t h = (u[k >> 1] >> (16 * (k & 1))) & 0xffffu;
                        v[k] = a.dtype == PVS_BF16 ? __uint_as_float(h << 16)
                                                   : __half2float(__ushort_as_half((uint16_t)h));
                    }
                }
            } else if (a.dtype != PVS_F32 && col + 8 <= a.cols) {
                uint32_t u[4];
                load_eight_halves(static_cast<const uint16_t*>(a.src) + at, u);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t h = (u[k >> 1] >> (16 * (k & 1))) & 0xffffu;
                    v[k] = a.dtype == PVS_BF16 ? __uint_as_float(h << 16)
                                               : __half2float(__ushort_as_half((uint16_t)h));
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    v[k] = col + k < a.cols ? load_as_float(a.src, a.dtype, at + k) : 0.0f;
            }
            if (zero) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = 0.0f;
            }
            if (a.row_scale) {
                const float s = a.row_scale[row];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = col + k < a.cols ? v[k] * s : 0.0f;
            }
            for (int part = 0; part < a.parts; ++part) {
                uint32_t h[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    h[k] = part + 1 < a.parts ? cut_bf16(v[2 * k], v[2 * k + 1])
                           : a.to_f16         ? pack_f16(v[2 * k], v[2 * k + 1])
                                              : pack_bf16(v[2 * k], v[2 * k + 1]);
                *reinterpret_cast<uint4*>(a.dst + part * a.part_stride + row * a.ldd + col) =
                    make_uint4(h[0], h[1], h[2], h[3]);
            }
        }
    }
}

__global__ void __launch_bounds__(256) split_kernel(const SplitArgs a) {
    next_early();
    wait_before();
    if (a.only_if && *a.only_if == 0) return;
    split_rows(a, blockIdx.x, gridDim.x);
}

// How a split's blocks share its rows: set before its launch.
int64_t plan_split(SplitArgs& a) {
    const int pieces = (a.cols + 7) / 8;
    a.per_block = std::max(1, 512 / pieces);
    a.magic = (1ull << 40) / pieces + 1;
    a.wide = (reinterpret_cast<uintptr_t>(a.src) & 15u) == 0 && a.ld % (a.dtype == PVS_F32 ? 4 : 8) == 0;
    // (a conditional copy mostly does nothing: few blocks)
    const int64_t most = a.only_if ? 152 * 4 : 1 << 20;
    return std::min((a.rows + a.per_block - 1) / a.per_block, most);
}

cudaError_t launch_split(const SplitArgs& s, cudaStream_t st) {
    if (s.rows <= 0) return cudaSuccess;
    SplitArgs a = s;
    const int64_t blocks = plan_split(a);
    count_launches(1);
    return launch_early(split_kernel, blocks, 256, 0, st, a);
}

// Eight float32 elements of a row from column k, zeros past it.
__device__ __forceinline__ void load_eight_floats(const float* x, int k, int cols, bool wide,
                                                  float (&v)[8]) {
    if (wide && k + 8 <= cols) {
        const float4 p = __ldg(reinterpret_cast<const float4*>(x + k));
        const float4 q = __ldg(reinterpret_cast<const float4*>(x + k) + 1);
        v[0] = p.x, v[1] = p.y, v[2] = p.z, v[3] = p.w;
        v[4] = q.x, v[5] = q.y, v[6] = q.z, v[7] = q.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = k + j < cols ? __ldg(x + k + j) : 0.0f;
    }
}
__device__ __forceinline__ float finite_top(const float (&v)[8], float top) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float f = fabsf(v[j]);
        if (f <= 3.402823466e38f) top = fmaxf(top, f);
    }
    return top;
}
__device__ __forceinline__ void store_parts(const Split16Args& a, int64_t at, float (&v)[8], float up) {
    const SplitArgs& s = a.s;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float f0 = v[2 * j] * up, f1 = v[2 * j + 1] * up;
        hi[j] = pack_f16(f0, f1);
        const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&hi[j]));
        // (nothing is left of an infinity or a NaN)
        lo[j] = pack_f16(isfinite(f0) ? f0 - h.x : 0.0f, isfinite(f1) ? f1 - h.y : 0.0f);
    }
    *reinterpret_cast<uint4*>(a.dst16 + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(a.dst16 + a.part16_stride + at) =
        make_uint4(lo[0], lo[1], lo[2], lo[3]);
    if (!s.dst) return;
    for (int part = 0; part < s.parts; ++part) {
        uint32_t h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            h[j] = part + 1 < s.parts ? cut_bf16(v[2 * j], v[2 * j + 1])
                                      : pack_bf16(v[2 * j], v[2 * j + 1]);
        *reinterpret_cast<uint4*>(s.dst + part * s.part_stride + at) =
            make_uint4(h[0], h[1], h[2], h[3]);
    }
}

// Rows to a warp at a time: four of up to 256 elements, two of up to 512, else one.
__host__ __device__ __forceinline__ int rows_of_warp(int cols) {
    return cols <= 256 ? 4 : cols <= 512 ? 2 : 1;
}

// A warp holds up to 1024 elements of its ROWS rows in registers, all loads in flight at
// once (read twice, 200 rows over 100,003 items of 385 took 189 us in all; with a row to
// a warp, 401,423 items of 128 took 181 us, with four 108); longer rows are read twice,
// the second time from L1.
template <int ROWS>
__device__ __forceinline__ void split16_rows(const Split16Args& a, int64_t block, int64_t blocks) {
    constexpr int kHeld = 4 / ROWS;
    const SplitArgs& s = a.s;
    const int lane = threadIdx.x & 31;
    for (int64_t first = (block * 8 + (threadIdx.x >> 5)) * ROWS; first < s.rows;
         first += blocks * 8 * ROWS) {
        float v[ROWS][kHeld][8];
        int cols[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t row = min(first + r, s.rows - 1);
            const bool zero = ignored_row(s.zero_target, s.ignore_index, s.zero_stats, row) ||
                              (s.zero_bias && s.zero_bias[row] == -INFINITY);
            cols[r] = zero ? 0 : s.cols;          // (a zero row: nothing is read)
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float* x = static_cast<const float*>(s.src) + min(first + r, s.rows - 1) * s.ld;
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                load_eight_floats(x, lane * 8 + 256 * i, cols[r], s.wide, v[r][i]);
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t row = first + r;
            if (row >= s.rows) break;
            const float* x = static_cast<const float*>(s.src) + row * s.ld;
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < kHeld; ++i) top = finite_top(v[r][i], top);
            if (ROWS == 1) {
                for (int k = lane * 8 + 256 * kHeld; k < cols[r]; k += 256) {
                    float w[8];
                    load_eight_floats(x, k, cols[r], s.wide, w);
                    top = finite_top(w, top);
                }
            }
            top = warp_max(top);
            const int e = top > 0.0f ? min(13 - ilogbf(top), 126) : 0;
            const float up = exp2f((float)e);
            if (lane == 0) a.units[row] = exp2f((float)-e);
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                const int k = lane * 8 + 256 * i;
                if (k < s.cols) store_parts(a, row * s.ldd + k, v[r][i], up);
            }
            if (ROWS == 1) {
                for (int k = lane * 8 + 256 * kHeld; k < s.cols; k += 256) {
                    float w[8];
                    load_eight_floats(x, k, cols[r], s.wide, w);
                    store_parts(a, row * s.ldd + k, w, up);
                }
            }
        }
    }
}
__device__ __forceinline__ void split16_any(const Split16Args& a, int64_t block, int64_t blocks) {
    const int n = rows_of_warp(a.s.cols);
    if (n == 4)
        split16_rows<4>(a, block, blocks);
    else if (n == 2)
        split16_rows<2>(a, block, blocks);
    else
        split16_rows<1>(a, block, blocks);
}

// The rows of the backward pass.
__device__ __forceinline__ void prepare_row(const RowArgs& r, int64_t i) {
    if (i == 0) *r.bad_masked = 0;
    if (i >= r.rows) return;
    const float4 st = r.stats[i];
    // (a row that has a list: its logits' entries are not the product's to write)
    const int64_t y = r.targets ? r.targets[i] : 0;
    GradRow o{0.0f, 0.0f, 0.0f, -1};
    if (!(r.targets && y == r.ignore_index) && !(st.x == -INFINITY && st.y == 0.0f)) {
        const float g = r.grad[i] * (r.up ? *r.up : 1.0f);
        o.m = st.x;
        if (y < 0 || y >= r.items) {
            o.coef = o.hit = __int_as_float(0x7fffffff);
        } else {
            o.coef = g / st.y;
            o.hit = g * st.z;
            // (a masked target has no logit, and no gradient of its own)
            if (st.w != -INFINITY) o.y = (int)y;
        }
    }
    r.out[i] = o;
}

// What a pass does before its first product, in one launch: its copies, and the
// backward pass's rows, each on blocks of its own.  Memory bounds it: 400,000 rows of 385 in
// 16 bits 124 us (5.0 TB/s), 401,423 float32 rows of 128 in two parts 108 us (3.8 TB/s).
template <bool TWO>
__global__ void __launch_bounds__(256) prepare_kernel(const PrepareArgs a) {
    next_early();
    wait_before();
    int64_t b = blockIdx.x;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (b < a.blocks[i]) {
            if (TWO)
                split16_any(a.copy[i], b, a.blocks[i]);
            else
                split_rows(a.copy[i].s, b, a.blocks[i]);
            return;
        }
        b -= a.blocks[i];
    }
    prepare_row(a.rows, b * 256 + threadIdx.x);
}

cudaError_t launch_prepare(PrepareArgs& a, cudaStream_t st) {
    int64_t total = 0;
    bool two = false;
    for (int i = 0; i < 2; ++i) {
        Split16Args& c = a.copy[i];
        if (c.s.rows <= 0) {
            a.blocks[i] = 0;
            continue;
        }
        two = c.dst16 != nullptr;
        a.blocks[i] = plan_split(c.s);
        if (two) {
            const int n = 8 * rows_of_warp(c.s.cols);
            a.blocks[i] = std::min<int64_t>((c.s.rows + n - 1) / n, 1 << 20);
        }
        total += a.blocks[i];
    }
    if (a.rows.out) total += (a.rows.rows + 255) / 256;
    if (total == 0) return cudaSuccess;
    if (total > 0x7fffffff) return cudaErrorInvalidValue;
    count_launches(1);
    return launch_early(two ? prepare_kernel<true> : prepare_kernel<false>, total, 256, 0, st, a);
}

// Eight codes a thread, in one load where rows are aligned.
__device__ __forceinline__ void split_codes_rows(const CodesArgs& a, int64_t block) {
    const int8_t* codes = a.codes;
    const float* scales = a.scales;
    uint16_t* dst = a.dst;
    const int64_t ldc = a.ldc, ldd = a.ldd, rows = a.rows;
    const int cols = a.cols, per_block = a.per_block, wide = a.wide, pieces = (cols + 7) / 8;
    const uint64_t m = a.magic;
    const int64_t row0 = block * per_block;
    const uint32_t total = (uint32_t)(min((int64_t)per_block, rows - row0) * pieces);
#pragma unroll 2
    for (uint32_t i = threadIdx.x; i < total; i += 256) {
        const uint32_t r = (uint32_t)((i * m) >> 40);
        const int64_t row = row0 + r;
        const int col = (int)(i - r * (uint32_t)pieces) * 8;
        const int8_t* p = codes + row * ldc + col;
        const float s = scales ? __ldg(scales + row) : 1.0f;
        float v[8];
        if (wide && col + 8 <= cols) {
            const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
            const uint32_t w[2] = {u.x ^ 0x80808080u, u.y ^ 0x80808080u};
            // the byte code + 128 under the exponent of 2^23 reads as 2^23 + 128 + code
#pragma unroll
            for (int k = 0; k < 8; ++k)
                v[k] = __uint_as_float(__byte_perm(w[k >> 2], 0x4b000000u, 0x7440 | (k & 3))) -
                       8388736.0f;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = col + k < cols ? (float)p[k] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = col + k < cols ? v[k] * s : 0.0f;
        for (int part = 0; part < a.parts; ++part) {
            uint32_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                h[k] = part + 1 < a.parts ? cut_bf16(v[2 * k], v[2 * k + 1])
                                          : pack_bf16(v[2 * k], v[2 * k + 1]);
            *reinterpret_cast<uint4*>(dst + part * a.part_stride + row * ldd + col) =
                make_uint4(h[0], h[1], h[2], h[3]);
        }
    }
}

// The operands of a weight gradient from kept rows: codes, and dy where it is copied.
// 32,768 x 768 codes times their scales to two bf16 parts in 26 us (4.9 TB/s; issue 75%).
__global__ void __launch_bounds__(256) codes_kernel(const CodesArgs c, const SplitArgs s,
                                                    int64_t blocks) {
    next_early();
    wait_before();
    if (blockIdx.x < blocks)
        split_rows(s, blockIdx.x, blocks);
    else
        split_codes_rows(c, blockIdx.x - blocks);
}

cudaError_t launch_codes(CodesArgs c, SplitArgs s, cudaStream_t st) {
    const int pieces = (c.cols + 7) / 8;
    c.per_block = std::max(1, 512 / pieces);
    c.magic = (1ull << 40) / pieces + 1;
    c.wide = (reinterpret_cast<uintptr_t>(c.codes) & 7u) == 0 && c.ldc % 8 == 0;
    const int64_t first = s.dst ? plan_split(s) : 0;
    const int64_t total = first + (c.rows + c.per_block - 1) / c.per_block;
    if (total > 0x7fffffff) return cudaErrorInvalidValue;
    count_launches(1);
    return launch_early(codes_kernel, total, 256, 0, st, c, s, first);
}

// ---- host side ---------------------------------------------------------------------
bool operand_map(CUtensorMap* m, const Matrix& x, bool mn, int box_rows) {
    return tensor_map_3d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, x.p, (uint64_t)x.parts,
                         (uint64_t)x.rows, (uint64_t)x.cols, (uint64_t)x.ld,
                         (uint64_t)(x.parts > 1 ? x.part_stride : x.ld * x.rows), 64,
                         (uint32_t)(mn ? kTileK : box_rows));
}

void part_pairs(Args& a, int pa, int pb, int levels) {
    a.npairs = 0;
    // parts are 2^-8 (bf16) or 2^-11 (f16) of one another; what is below the last bits of
    // a float32 is left out.  Smallest first: the tensor cores cut each step's sum to 24
    // bits, so only the leading pair's steps may cost the sum its last bits
    for (int level = levels; level >= 0; --level)
        for (int i = 0; i <= level; ++i)
            if (i < pa && level - i < pb) {
                a.pa[a.npairs] = (uint8_t)i;
                a.pb[a.npairs++] = (uint8_t)(level - i);
            }
}

namespace {

template <int kCta>
const void* kernel_of(int epilogue) {
    return epilogue == kStats      ? (const void*)head_gemm_kernel<kStats, kCta>
           : epilogue == kTopStats ? (const void*)head_gemm_kernel<kTopStats, kCta>
           : epilogue == kGrad     ? (const void*)head_gemm_kernel<kGrad, kCta>
                                   : (const void*)head_gemm_kernel<kOut, kCta>;
}

cudaLaunchConfig_t config(int cta, int grid, cudaStream_t st, cudaLaunchAttribute (&attr)[2]) {
    cudaLaunchConfig_t cfg{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cta;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = cta == 2 ? smem_bytes<2>() : smem_bytes<1>();
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cta == 2 ? 2 : 1;
    return cfg;
}

}  // namespace

cudaError_t launch_gemm(int epilogue, Args& a, const Device& dev, cudaStream_t st) {
    const int cta = a.cta;
    const int slots = cta == 2 ? dev.pairs : dev.sms;
    int64_t total = 0;
    for (int i = 0; i < a.nprob; ++i) {
        Problem& p = a.p[i];
        const int64_t u = (int64_t)p.mtiles * p.ntiles * p.splits;
        if (p.kchunks < 1 || p.splits < 1 || p.splits > p.kchunks || u < 1 || u > (1 << 30))
            return cudaErrorInvalidValue;
        // equal lengths but for the last: every split has a chunk
        p.klength = (p.kchunks + p.splits - 1) / p.splits;
        if ((int64_t)p.klength * (p.splits - 1) >= p.kchunks) return cudaErrorInvalidValue;
        p.units = (int)u;
        total += u;
    }
    int used = (int)std::min<int64_t>(total, slots);
    if (a.nprob == 2) {
        // slots in proportion to the problems' work
        used = std::max(used, 2);
        if (a.slots0 < 1 || a.slots0 >= used) {
            const double w0 = (double)a.p[0].units * a.p[0].kchunks / a.p[0].splits;
            const double w1 = (double)a.p[1].units * a.p[1].kchunks / a.p[1].splits;
            a.slots0 = std::min(std::max((int)(used * w0 / (w0 + w1) + 0.5), 1), used - 1);
        }
    }
    const void* fn = cta == 2 ? kernel_of<2>(epilogue) : kernel_of<1>(epilogue);
    a.wait_ns = dev.wait_ns;
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = config(cta, used * cta, st, attr);
    cudaError_t e = raise_smem_limit(fn, cfg.dynamicSmemBytes);
    if (e != cudaSuccess) return e;
    count_launches(1);
    void* args[1] = {&a};
    return cudaLaunchKernelExC(&cfg, fn, args);
}

namespace {
constexpr int kMaxDevices = 64;
std::mutex g_device_mutex;
Device g_devices[kMaxDevices];
}  // namespace

cudaError_t device(Device* d) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(g_device_mutex);
    Device& g = g_devices[dev];
    if (!g.status) {
        int sms = 0;
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return e;
        // CTA pairs that run at once (0 where none can: lone CTAs serve then)
        int pairs = 0;
        cudaLaunchAttribute attr[2];
        const cudaLaunchConfig_t cfg = config(2, 2 * sms, nullptr, attr);
        if (raise_smem_limit(kernel_of<2>(kOut), cfg.dynamicSmemBytes) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&pairs, kernel_of<2>(kOut), &cfg) != cudaSuccess) {
            cudaGetLastError();
            pairs = 0;
        }
        int* p = nullptr;
        e = pinned_alloc(&p, 64);
        if (e != cudaSuccess) return e;
        *static_cast<volatile int*>(p) = 0;
        g.sms = sms;
        g.pairs = pairs;
        g.wait_ns = kWaitLimitNs;
        g.status = p;
    }
    *d = g;
    return cudaSuccess;
}

int take_status(const Device& d) {
    std::lock_guard<std::mutex> lock(g_device_mutex);
    volatile int* p = d.status;
    const int s = *p;
    if (s != 0) *p = 0;
    return s;
}

int ready(Device* d) {
    if (device(d) != cudaSuccess) {
        cudaGetLastError();
        return PVS_ERR_CUDA;
    }
    return take_status(*d);
}

}  // namespace head
}  // namespace pvs

extern "C" pvs_status pvs_head_status(void) {
    pvs::head::Device d;
    return (pvs_status)pvs::head::ready(&d);
}

extern "C" pvs_status pvs_head_set_wait_limit(int64_t ns) {
    using namespace pvs::head;
    if (ns < 0) return PVS_ERR_INVALID;
    Device d;
    int dev = 0;
    if (device(&d) != cudaSuccess || cudaGetDevice(&dev) != cudaSuccess) {
        cudaGetLastError();
        return PVS_ERR_CUDA;
    }
    std::lock_guard<std::mutex> lock(g_device_mutex);
    g_devices[dev].wait_ns = std::min<unsigned long long>((unsigned long long)ns, pvs::kWaitLimitNs);
    return PVS_OK;
}

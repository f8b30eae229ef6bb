// Product of microscaled 4-bit rows on the tensor cores (head.h).
//
//   y[b, n] = sum_k x[b, k] w[n, k],  both as codes e2m1 with scales of 16 or 32 elements
//
// x is put into the weights' format first (mx_pack.cu); the product then is tcgen05's
// block-scaled one, K = 64 an instruction, with float32 accumulators in TMEM.  Weights are its M
// (128 rows a CTA), rows of x its N, so that a few rows of x make a narrow tile and the
// weights' bytes are read once; a TMEM lane is a row of weights, and neighbouring lanes store
// neighbours of a row of y.
//
// Persistent, 10 warps a CTA:
//   warp 0     TMA producer: chunks of 256 of k, 128 bytes a row (128-byte swizzle), and their
//              blocks of scales;
//   warp 1     one thread copies a chunk's scales from shared memory to TMEM and issues its four
//              MMAs.  Four sets of TMEM columns hold scales, and a set is written again when
//              the MMAs that read it are complete;
//   warps 2-9  epilogue: each takes every other 32 columns of its quarter of the lanes into
//              registers, hands the accumulator back, and stores.
// Many rows of x go to CTA pairs (cta_group::2, 256 x 256 tiles): each CTA holds 128 rows of
// weights and half of the tile's rows of x, and the scales of all of them.  Their accumulator is
// one (two and the scales are more than TMEM): it is handed back when its columns are in
// registers, before they are stored.
//
// 16,384 rows by 4,096 x 4,096 in bf16, groups of 16: 94 us (5.8 PFLOP/s, tensor pipe 67%), of 32 86 (6.3,
// 72%), with 8,192 of k 157 and 146 (7.5, 85%): about 490 cycles a chunk, and beside the mainloop some
// 4,000 a tile for the stores that it does not hide.  32 rows by 1,000,000 x 768, groups of 32: 73 us,
// 6.4 TB/s.  (With lone lanes that issue, a chunk took 1,000 cycles; with a branch at each store
// the first took 440 us.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "../../include/head.h"
#include "f32x2.cuh"
#include "kernels.h"
#include "mx.h"
#include "pvs_common.cuh"
#include "tc.cuh"
#include "tensor_map.h"

namespace pvs {
namespace head {
namespace {

constexpr int kMxK = 256;                // of k a chunk: 128 bytes of codes
constexpr int kMxStages = 8;             // at most
constexpr int kMxEpiWarps = 8;
constexpr int kMxThreads = (2 + kMxEpiWarps) * 32;
constexpr int kMxPart = 128 * 128;       // bytes of 128 rows' codes of a chunk
constexpr uint32_t kMxTmem = 512;
constexpr uint32_t kScaleCol = 256;      // sets of scales behind the accumulators
constexpr uint32_t kScaleSet = 64;       // columns of a set: A's 16, B's 32
constexpr uint32_t kScaleSets = 4;       // (fewer than a ring has stages)

struct MxArgs {
    CUtensorMap a, b, sa, sb;
    int m, n;                            // rows of weights, rows of x
    int bn;                              // rows of x a tile
    int mtiles, ntiles, splits, units, m_fast;
    int steps;                           // of 64 of k
    int kchunks, klength;                // chunks in all, and in a split
    int accs;                            // accumulators
    int stages;
    uint32_t b_bytes, stage_bytes;
    const float *row_a, *row_b;          // row scales, or null
    void* y;
    int64_t ldy;
    int dtype, by_pairs;                 // y in 16 bits, its rows on 4 bytes
    float* slots;                        // splits: float32 sums [split][n][ldslot]
    int64_t slot_stride, ldslot;
    int* status;
    unsigned long long wait_ns;
};

struct MxShared {
    uint64_t full[kMxStages];
    uint64_t empty[kMxStages];
    uint64_t tfull[2];
    uint64_t tempty[2];
    uint32_t tmem_base;
    int abort;                           // of the pair: set in both its CTAs
    uint32_t fills;                      // stages that this CTA has filled
    uint32_t chunks, tiles;              // even CTA: chunks and tiles committed
    alignas(16) float row_b[kMxEpiWarps][4][32];   // a tile's scales of rows of x, by warp
};

constexpr size_t kMxSmem = 227 * 1024;

// A unit: a tile over a range of chunks.
struct MxUnit {
    int mt, nt, split, k0, k1;
    __device__ __forceinline__ MxUnit(const MxArgs& a, int u) {
        const int na = a.m_fast ? a.mtiles : a.ntiles, nb = a.m_fast ? a.ntiles : a.mtiles;
        const int i = u % na, j = u / na % nb;
        split = u / na / nb;
        mt = a.m_fast ? i : j;
        nt = a.m_fast ? j : i;
        k0 = split * a.klength;
        k1 = min(k0 + a.klength, a.kchunks);
    }
};
// Rows of x that a tile's MMAs take: those that are there, in the steps that an MMA takes.
template <int kCta>
__device__ __forceinline__ int columns_of(const MxArgs& a, int nt) {
    const int left = min(a.bn, a.n - nt * a.bn);
    return (left + 16 * kCta - 1) & ~(16 * kCta - 1);
}

__device__ __forceinline__ bool mx_aborted(MxShared& sh) {
    return *reinterpret_cast<volatile int*>(&sh.abort) != 0;
}
template <int kCta>
__device__ __forceinline__ void mx_abort(MxShared& sh, int* status, int crank) {
    *reinterpret_cast<volatile int*>(&sh.abort) = 1;
    if (kCta == 2)
        asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(
                         cluster_map(&sh.abort, crank ^ 1)),
                     "r"(1)
                     : "memory");
    *reinterpret_cast<volatile int*>(status) = PVS_ERR_TIMEOUT;
}
__device__ __forceinline__ bool mx_wait(uint64_t* bar, uint32_t parity, unsigned long long limit_ns) {
    return mbar_test_wait(bar, parity) || (limit_ns != 0 && mbar_wait(bar, parity, limit_ns));
}
// The same by a whole warp, so that what follows is uniform.
__device__ __forceinline__ bool mx_warp_wait(uint64_t* bar, uint32_t parity, unsigned long long limit_ns) {
    return __all_sync(0xffffffffu, mx_wait(bar, parity, limit_ns));
}
// A wait at a role's end, with the 2 s limit, given up in a millisecond where another role has
// given up (what it waits for may then never come).
template <int kCta>
__device__ __forceinline__ void mx_last_wait(uint64_t* bar, uint32_t parity, MxShared& sh, int* status,
                                             int crank) {
    constexpr unsigned long long kTurn = 1000000;
    for (unsigned long long t = 0; t < kWaitLimitNs; t += kTurn) {
        if (mx_aborted(sh) || mbar_wait(bar, parity, kTurn)) return;
    }
    mx_abort<kCta>(sh, status, crank);
}
__device__ __forceinline__ uint32_t mx_word_of(const uint32_t* p, int crank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_map(p, crank)) : "memory");
    return v;
}

template <int kCta>
__device__ __forceinline__ void mx_load(void* dst, const void* tmap, int x, int y, int z, uint32_t bar) {
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

// This CTA's copies of one fill of a stage: 128 rows of A, its share of B's rows, the scales of
// both (of all of B's rows in each CTA of a pair).
template <int kCta, bool kSixteen>
__device__ __forceinline__ void mx_fill(const MxArgs& a, uint8_t* stage, uint64_t* full, int crank, int am,
                                        int bm, int bs, int kc) {
    constexpr int kBlocks = kSixteen ? 4 : 2;
    if (crank == 0) mbar_arrive_expect_tx(full, (uint32_t)kCta * a.stage_bytes);
    const uint32_t bar = kCta == 2 ? cluster_map(full, 0) : smem_u32(full);
    mx_load<kCta>(stage, &a.a, kc * 128, am, 0, bar);
    mx_load<kCta>(stage + kMxPart, &a.b, kc * 128, bm, 0, bar);
    uint8_t* s = stage + kMxPart + a.b_bytes;
    mx_load<kCta>(s, &a.sa, 0, kc * kBlocks, am / 128, bar);
    mx_load<kCta>(s + kBlocks * 512, &a.sb, 0, kc * kBlocks, bs, bar);
    if constexpr (kCta == 2) mx_load<kCta>(s + 2 * kBlocks * 512, &a.sb, 0, kc * kBlocks, bs + 1, bar);
}

// After a wait that ran out: one thread of each CTA waits for what is still on its way to its
// CTA, which must not end before.  Fills first: those that the other CTA of the pair has issued
// and this one has not are issued here (the stage is free, or the other would not have filled
// it; what is read does not matter), so that every `full` barrier completes.  Then the MMAs and
// their commits.  With the 2 s limit; after one that runs out nothing more is waited for.
template <int kCta, bool kSixteen>
__device__ __noinline__ void mx_settle(const MxArgs& a, MxShared& sh, uint8_t* stages, int crank) {
    const uint32_t n = (uint32_t)a.stages;
    const uint32_t mine = sh.fills;
    const uint32_t fills = kCta == 2 ? max(mine, mx_word_of(&sh.fills, crank ^ 1)) : mine;
    for (uint32_t g = mine; g < fills; ++g) {
        const uint32_t s = g % n;
        mx_fill<kCta, kSixteen>(a, stages + s * a.stage_bytes, &sh.full[s], crank, 0, 0, 0, 0);
    }
    const uint32_t chunks = kCta == 2 ? mx_word_of(&sh.chunks, 0) : sh.chunks;
    const uint32_t tiles = kCta == 2 ? mx_word_of(&sh.tiles, 0) : sh.tiles;
    bool in_time = true;
    for (uint32_t s = 0; s < n; ++s) {
        if (in_time && crank == 0 && s < fills) in_time = mbar_wait(&sh.full[s], ((fills - 1 - s) / n) & 1u);
        if (in_time && s < chunks) in_time = mbar_wait(&sh.empty[s], ((chunks - 1 - s) / n) & 1u);
    }
    const uint32_t accs = (uint32_t)a.accs;
    for (uint32_t b = 0; b < accs; ++b)
        if (in_time && b < tiles) in_time = mbar_wait(&sh.tfull[b], ((tiles - 1 - b) / accs) & 1u);
}

// A lane's column of up to 32 rows of y, ld apart (neighbouring lanes: neighbours).
template <typename T>
__device__ __forceinline__ T mx_round(uint32_t u) {
    const float v = __uint_as_float(u);
    if constexpr (sizeof(T) == 4)
        return v;
    else
        return T(v);
}
__device__ __forceinline__ uint32_t mx_two(uint32_t lo, uint32_t hi, __nv_bfloat16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t mx_two(uint32_t lo, uint32_t hi, __half) {
    const __half2 v = __floats2half2_rn(__uint_as_float(lo), __uint_as_float(hi));
    return *reinterpret_cast<const uint32_t*>(&v);
}
// Whether the product of a sum and one of the warp's scales may leave float32's normal range, so that
// the order of its products with both scales matters.  A sum is below 2^38 (32,767 products of
// codes of 6 at most and scales of 448), and no less than 2^-20 where it is not zero (codes are
// whole halves, scales whole 2^-9): 2^-106 to 2^89 keep the product from 2^-126 to 2^128.  Scales
// of rows whose largest element is 2^-95 to 2^98 are in there.  (Scales in either order cost the products
// with them alone: 16,384 rows by 4,096 with 4,096 and 1,024 of k take 139 and 90 us, for 129 and 61.)
__device__ __forceinline__ bool mx_apart(float ra) {
    return __any_sync(0xffffffffu, !(fabsf(ra) >= 0x1p-106f && fabsf(ra) <= 0x1p89f));
}
// 32 whole rows of 32 neighbours of 16 bits, on 4 bytes: even lanes store the pairs of even rows,
// odd ones those of odd rows.
template <typename T>
__device__ __forceinline__ void mx_store_pairs(T* p, int64_t ld, const uint32_t (&r)[32]) {
    const bool odd = threadIdx.x & 1u;
    if (odd) p += ld - 1;
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
        const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? r[j] : r[j + 1], 1);
        *reinterpret_cast<uint32_t*>(p + j * ld) = mx_two(odd ? got : r[j], odd ? r[j + 1] : got, T());
    }
}
template <typename T>
__device__ __forceinline__ void mx_store(T* p, int64_t ld, const uint32_t (&r)[32], int count) {
    if (count >= 32) {
#pragma unroll
        for (int j = 0; j < 32; ++j) p[j * ld] = mx_round<T>(r[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < count) p[j * ld] = mx_round<T>(r[j]);
    }
}

template <int kCta, bool kSixteen>
__global__ void __launch_bounds__(kMxThreads, 1) mx_gemm_kernel(const __grid_constant__ MxArgs a) {
    extern __shared__ uint8_t mx_smem[];
    // the layout is the same in both CTAs of a pair: barriers and the pair's MMAs are
    // addressed by offset
    const uint32_t raw = smem_u32(mx_smem);
    uint8_t* stages = mx_smem + (((raw + 1023u) & ~1023u) - raw);
    MxShared& sh = *reinterpret_cast<MxShared*>(stages + (size_t)a.stages * a.stage_bytes);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int crank = kCta == 2 ? (int)cluster_ctarank() : 0;
    const int slot = blockIdx.x / kCta, nslots = gridDim.x / kCta;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&sh.full[s], 1);
            mbar_init(&sh.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sh.tfull[b], 1);
            mbar_init(&sh.tempty[b], kCta * kMxEpiWarps);
        }
        sh.abort = 0;
        sh.fills = sh.chunks = sh.tiles = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        if (kCta == 2)
            tc::tmem_alloc_pair(&sh.tmem_base, kMxTmem);
        else
            tc::tmem_alloc(&sh.tmem_base, kMxTmem);
        tc::fence_before_sync();
    }
    __syncthreads();
    if (kCta == 2) cluster_barrier();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem_base, 0);
    next_early();
    wait_before();

    // The producer's and the issuer's loops are run by whole warps, one lane of which issues: their
    // addresses and descriptors then stay in uniform registers, where the instructions want them
    // (by lone lanes, which move each operand there, a chunk took 1,000 cycles where its MMAs take
    // 512).
    if (warp == 0) {
        // ---------------- TMA producer ----------------
        const bool one = tc::elect_one();
        uint32_t g = 0;
        Turn at;
        bool go = true;
        for (int u = slot; go && u < a.units; u += nslots) {
            const MxUnit w(a, u);
            const int am = (w.mt * kCta + crank) * 128, bs = w.nt * a.bn / 128;
            const int bm = w.nt * a.bn + crank * (columns_of<kCta>(a, w.nt) / 2);
            if (__any_sync(0xffffffffu, mx_aborted(sh))) break;
            for (int kc = w.k0; kc < w.k1; ++kc, ++g, at.next(a.stages)) {
                go = mx_warp_wait(&sh.empty[at.stage], at.parity ^ 1u, a.wait_ns);
                if (!go) break;
                if (one)
                    mx_fill<kCta, kSixteen>(a, stages + at.stage * a.stage_bytes, &sh.full[at.stage], crank,
                                            am, bm, bs, kc);
            }
        }
        if (one) {
            if (!go) mx_abort<kCta>(sh, a.status, crank);
            sh.fills = g;
            // the MMAs have consumed the last fill of every stage used: no copy into
            // this CTA and no commit to its barriers is still in flight when it ends
            for (uint32_t s = 0; s < (uint32_t)a.stages && s < g; ++s)
                mx_last_wait<kCta>(&sh.empty[s], ((g - 1 - s) / a.stages) & 1u, sh, a.status, crank);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------- MMA issuer (the even CTA of a pair) ----------------
        if (crank == 0) {
            const bool one = tc::elect_one();
            // descriptors: their upper halves do not change, the address is in the lower ones
            const uint32_t s0 = smem_u32(stages);
            const uint64_t codes0 = tc::smem_desc_sw128_kmajor(s0), rows0 = tc::smem_desc_rows16(s0);
            const uint32_t codes_hi = (uint32_t)(codes0 >> 32), rows_hi = (uint32_t)(rows0 >> 32);
            const uint32_t b_off = kMxPart >> 4, s_off = (kMxPart + a.b_bytes) >> 4;
            const uint32_t stage16 = a.stage_bytes >> 4;
            auto codes_at = [&](uint32_t lo) { return (uint64_t)codes_hi << 32 | lo; };
            auto rows_at = [&](uint32_t lo) { return (uint64_t)rows_hi << 32 | lo; };
            constexpr int kBlocks = kSixteen ? 4 : 2;      // of scales for 128 rows
            uint32_t g = 0;
            int it = 0;
            Turn at, before;
            bool go = true;
            for (int u = slot; u < a.units; u += nslots, ++it) {
                const MxUnit w(a, u);
                const int b = a.accs == 2 ? it & 1 : 0;
                const uint32_t turns = (uint32_t)(a.accs == 2 ? it >> 1 : it);
                if (__any_sync(0xffffffffu, mx_aborted(sh))) break;
                go = mx_warp_wait(&sh.tempty[b], (turns & 1u) ^ 1u, a.wait_ns);
                if (!go) break;
                tc::fence_after_sync();
                const uint32_t d = tmem + (uint32_t)(b * 128);
                const int columns = columns_of<kCta>(a, w.nt);
                const uint32_t first = tc::idesc_e2m1_f32(128 * kCta, columns, !kSixteen, 0);
                const uint32_t second = tc::idesc_e2m1_f32(128 * kCta, columns, !kSixteen, 2);
                for (int kc = w.k0; kc < w.k1; ++kc, ++g, at.next(a.stages)) {
                    go = mx_warp_wait(&sh.full[at.stage], at.parity, a.wait_ns);
                    if (!go) break;
                    // the MMAs that read this set of scales before are complete
                    if (g >= kScaleSets) {
                        go = mx_warp_wait(&sh.empty[before.stage], before.parity, a.wait_ns);
                        if (!go) break;
                        before.next(a.stages);
                    }
                    tc::fence_after_sync();
                    const uint32_t al = (uint32_t)codes0 + at.stage * stage16, bl = al + b_off;
                    const uint32_t cl = (uint32_t)rows0 + at.stage * stage16 + s_off;
                    const uint32_t sa = tmem + kScaleCol + g % kScaleSets * kScaleSet, sb = sa + 16;
                    // (the last chunk of k may be half a one)
                    const int steps = min(4, a.steps - 4 * kc);
                    if (one) {
#pragma unroll
                        for (int i = 0; i < kBlocks; ++i) {
                            tc::copy_scales<kCta>(sa + 4 * i, rows_at(cl + 32 * i));
                            tc::copy_scales<kCta>(sb + 8 * i, rows_at(cl + 32 * (kBlocks + i)));
                            if constexpr (kCta == 2)
                                tc::copy_scales<kCta>(sb + 8 * i + 4, rows_at(cl + 32 * (2 * kBlocks + i)));
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (i >= steps) break;
                            const uint32_t c = kSixteen ? i : i / 2;
                            tc::mma_e2m1<kCta, kSixteen>(d, codes_at(al + 2 * i), codes_at(bl + 2 * i),
                                                         !kSixteen && (i & 1) ? second : first, sa + 4 * c,
                                                         sb + 8 * c, i > 0 || kc > w.k0 ? 1u : 0u);
                        }
                        if (kCta == 2)
                            tc::commit_pair(&sh.empty[at.stage]);
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
                if (!go) mx_abort<kCta>(sh, a.status, crank);
                sh.chunks = g;
                sh.tiles = it;
                // TMEM is released after the last unit's MMAs
                if (it > 0)
                    mx_last_wait<kCta>(&sh.tfull[(it - 1) % a.accs], (uint32_t)((it - 1) / a.accs) & 1u, sh,
                                       a.status, crank);
            }
            __syncwarp();
        }
    } else {
        // ---------------- epilogue ----------------
        const int quarter = warp & 3, group = (warp - 2) >> 2;
        const uint32_t tempty_at[2] = {kCta == 2 ? cluster_map(&sh.tempty[0], 0) : 0u,
                                       kCta == 2 ? cluster_map(&sh.tempty[1], 0) : 0u};
        bool dead = false;
        int it = 0;
        for (int u = slot; u < a.units; u += nslots, ++it) {
            const MxUnit w(a, u);
            const int b = it % a.accs;
            const int n0 = w.nt * a.bn, ncols = min(a.bn, a.n - n0);
            const int row = (w.mt * kCta + crank) * 128 + quarter * 32 + lane;
            float ra = 1.0f;
            bool apart = false;
            if (kSixteen && a.splits == 1) {
                // (before the wait, under which the loads are done)
                if (row < a.m) ra = __ldg(a.row_a + row);
                apart = mx_apart(ra);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = (2 * i + group) * 32 + lane;
                    sh.row_b[warp - 2][i][lane] = c < ncols ? __ldg(a.row_b + n0 + c) : 0.0f;
                }
                __syncwarp();
            }
            if (!dead) {
                bool late = mx_aborted(sh);
                if (!late && !mx_wait(&sh.tfull[b], (uint32_t)(it / a.accs) & 1u, a.wait_ns)) {
                    mx_abort<kCta>(sh, a.status, crank);
                    late = true;
                }
                dead = __any_sync(0xffffffffu, late);
            }
            if (dead) continue;
            tc::fence_after_sync();
            const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(b * 128);
            uint32_t r[4][32];
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((2 * i + group) * 32 < ncols)
                    tc::ld_32x32b_x32(at + (uint32_t)(2 * i + group) * 32, r[i]);
            tc::wait_ld();
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                if (kCta == 2)
                    mbar_arrive_remote(tempty_at[b]);
                else
                    mbar_arrive(&sh.tempty[b]);
            }
            const bool pairs = a.by_pairs && row - lane + 32 <= a.m;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c0 = (2 * i + group) * 32, count = ncols - c0;
                if (count <= 0) break;
                if (kSixteen && apart) {
                    const float* rb = sh.row_b[warp - 2][i];
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        r[i][j] = __float_as_uint(times_scales(__uint_as_float(r[i][j]), ra, rb[j]));
                } else if (kSixteen && a.splits == 1) {
                    const float* rb = sh.row_b[warp - 2][i];
                    const uint64_t by = f2_pack(ra, ra);
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(rb + j);
                        auto two = [&](int k) {
                            return f2_mul(f2_pack(__uint_as_float(r[i][k]), __uint_as_float(r[i][k + 1])), by);
                        };
                        float v0, v1, v2, v3;
                        f2_unpack(f2_mul(two(j), f.x), v0, v1);
                        f2_unpack(f2_mul(two(j + 2), f.y), v2, v3);
                        r[i][j] = __float_as_uint(v0), r[i][j + 1] = __float_as_uint(v1);
                        r[i][j + 2] = __float_as_uint(v2), r[i][j + 3] = __float_as_uint(v3);
                    }
                }
                if (pairs && count >= 32) {
                    if (a.dtype == PVS_BF16)
                        mx_store_pairs(static_cast<__nv_bfloat16*>(a.y) + (int64_t)(n0 + c0) * a.ldy + row, a.ldy,
                                       r[i]);
                    else
                        mx_store_pairs(static_cast<__half*>(a.y) + (int64_t)(n0 + c0) * a.ldy + row, a.ldy, r[i]);
                    continue;
                }
                if (row >= a.m) continue;
                if (a.splits > 1)
                    mx_store(a.slots + w.split * a.slot_stride + (int64_t)(n0 + c0) * a.ldslot + row,
                             a.ldslot, r[i], count);
                else if (a.dtype == PVS_F32)
                    mx_store(static_cast<float*>(a.y) + (int64_t)(n0 + c0) * a.ldy + row, a.ldy, r[i], count);
                else if (a.dtype == PVS_BF16)
                    mx_store(static_cast<__nv_bfloat16*>(a.y) + (int64_t)(n0 + c0) * a.ldy + row, a.ldy, r[i],
                             count);
                else
                    mx_store(static_cast<__half*>(a.y) + (int64_t)(n0 + c0) * a.ldy + row, a.ldy, r[i], count);
            }
        }
    }
    __syncthreads();
    if (kCta == 2) cluster_barrier();   // no CTA leaves while its peer may still address it
    if (mx_aborted(sh)) {
        if (threadIdx.x == 0) mx_settle<kCta, kSixteen>(a, sh, stages, crank);
        __syncthreads();
        if (kCta == 2) cluster_barrier();
    }
    if (warp == 1) {
        tc::fence_after_sync();
        if (kCta == 2)
            tc::tmem_dealloc_pair(tmem, kMxTmem);
        else
            tc::tmem_dealloc(tmem, kMxTmem);
    }
}

const void* mx_kernel(int cta, bool sixteen) {
    return cta == 2 ? (sixteen ? (const void*)mx_gemm_kernel<2, true> : (const void*)mx_gemm_kernel<2, false>)
                    : (sixteen ? (const void*)mx_gemm_kernel<1, true> : (const void*)mx_gemm_kernel<1, false>);
}

// ---- the plan of a call --------------------------------------------------------------
struct MxPlan {
    int cta = 1, bn = 0, splits = 1;
    uint8_t *codes = nullptr, *scales = nullptr;
    float *rows = nullptr, *slots = nullptr;
    int64_t ldslot = 0;
    size_t bytes = 0;
};

MxPlan mx_plan(int64_t batch, int64_t rows, int cols, int group, const Device& dev, void* workspace) {
    MxPlan p;
    const int kp = mx_padded(cols);
    p.cta = batch > 128 && dev.pairs > 0 ? 2 : 1;
    p.bn = p.cta == 2 ? 256 : (int)std::min<int64_t>(128, round_up(batch, 16));
    const int64_t units = (rows + 128 * p.cta - 1) / (128 * p.cta) * ((batch + p.bn - 1) / p.bn);
    const int64_t slots = p.cta == 2 ? dev.pairs : dev.sms;
    const int chunks = (kp + kMxK - 1) / kMxK;
    // k is split where that fills the GPU and leaves a split four chunks
    if (2 * units <= slots) p.splits = even_splits(chunks, std::min<int64_t>(slots / units, chunks / 4));
    Carver c{static_cast<uint8_t*>(workspace)};
    p.codes = c.take<uint8_t>(batch * (kp / 2));
    p.scales = c.take<uint8_t>(mx_scale_bytes(batch, kp, group));
    if (group == 16) p.rows = c.take<float>(batch);
    p.ldslot = round_up(rows, 8);
    if (p.splits > 1) p.slots = c.take<float>(p.splits * batch * p.ldslot);
    p.bytes = c.used;
    return p;
}

bool mx_product_shape(int64_t batch, int64_t rows, int32_t cols, int32_t group, int32_t dtype) {
    return batch >= 0 && batch <= kMaxRows && rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= 32767 &&
           (group == 16 || group == 32) && dtype >= PVS_BF16 && dtype <= PVS_F32;
}

cudaError_t mx_product(const MxPlan& p, int64_t batch, const uint8_t* codes, const uint8_t* scales,
                       const float* row_scales, int64_t rows, int cols, int group, int dtype, void* y,
                       int64_t ldy, const Device& dev, cudaStream_t st) {
    const int kp = mx_padded(cols);
    MxArgs a{};
    a.m = (int)rows;
    a.n = (int)batch;
    a.bn = p.bn;
    a.splits = p.splits;
    a.steps = kp / 64;
    a.kchunks = (kp + kMxK - 1) / kMxK;
    a.klength = (a.kchunks + p.splits - 1) / p.splits;
    const int blocks = kMxK / (4 * group);   // of scales in a chunk, for 128 rows
    a.accs = p.bn > 128 ? 1 : 2;
    a.b_bytes = (uint32_t)(p.bn / p.cta * 128);
    a.stage_bytes = kMxPart + a.b_bytes + (uint32_t)((1 + p.cta) * blocks * 512);
    a.stages = std::min<int>(kMxStages, (int)((kMxSmem - 1024 - sizeof(MxShared)) / a.stage_bytes));
    const int64_t mtiles = (rows + 128 * p.cta - 1) / (128 * p.cta), ntiles = (batch + p.bn - 1) / p.bn;
    if (mtiles * ntiles * p.splits > 1 << 30) return cudaErrorInvalidValue;
    a.mtiles = (int)mtiles;
    a.ntiles = (int)ntiles;
    a.units = a.mtiles * a.ntiles * a.splits;
    // the smaller operand goes by for each tile of the larger
    a.m_fast = rows < batch;
    a.row_a = row_scales;
    a.row_b = p.rows;
    a.y = y;
    a.ldy = ldy;
    a.dtype = dtype;
    a.by_pairs = dtype != PVS_F32 && p.splits == 1 && ldy % 2 == 0 && on_elements(y, 4);
    a.slots = p.slots;
    a.slot_stride = batch * p.ldslot;
    a.ldslot = p.ldslot;
    a.status = dev.status;
    a.wait_ns = dev.wait_ns;
    const int64_t ld = kp / 2, sblocks = kp / (4 * group);
    if (!tensor_map_3d(&a.a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, codes, 1, rows, ld, ld, ld * rows, 128, 128) ||
        !tensor_map_3d(&a.b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.codes, 1, batch, ld, ld, ld * batch, 128,
                       (uint32_t)(p.bn / p.cta)) ||
        !tensor_map_blocks(&a.sa, scales, (rows + 127) / 128, sblocks, (uint32_t)blocks) ||
        !tensor_map_blocks(&a.sb, p.scales, (batch + 127) / 128, sblocks, (uint32_t)blocks))
        return cudaErrorInvalidValue;
    const void* fn = mx_kernel(p.cta, group == 16);
    cudaError_t e = raise_smem_limit(fn, kMxSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = p.cta;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    const int slots = p.cta == 2 ? dev.pairs : dev.sms;
    cfg.gridDim = dim3((unsigned)(std::min(a.units, slots) * p.cta));
    cfg.blockDim = dim3(kMxThreads);
    cfg.dynamicSmemBytes = kMxSmem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = p.cta == 2 ? 2 : 1;
    count_launches(1);
    void* args[1] = {&a};
    e = cudaLaunchKernelExC(&cfg, fn, args);
    if (e == cudaSuccess && p.splits > 1)
        e = launch_sum_slots(p.slots, p.splits, a.slot_stride, p.ldslot, batch, (int)rows, nullptr, 1.0f, y, ldy,
                             dtype, dev, st, p.rows, group == 16 ? row_scales : nullptr);
    return e;
}

pvs_status mx_ended(cudaError_t e) {
    if (e == cudaSuccess) return PVS_OK;
    cudaGetLastError();
    return PVS_ERR_CUDA;
}

}  // namespace
}  // namespace head
}  // namespace pvs

using namespace pvs;
using namespace pvs::head;

extern "C" pvs_status pvs_mx_workspace(int64_t batch, int64_t rows, int32_t cols, int32_t group,
                                       size_t* bytes) {
    if (!bytes || !mx_product_shape(batch, rows, cols, group, PVS_F32)) return PVS_ERR_INVALID;
    *bytes = 0;
    if (batch == 0 || rows == 0) return PVS_OK;
    Device dev;
    if (device(&dev) != cudaSuccess) {
        cudaGetLastError();
        return PVS_ERR_CUDA;
    }
    *bytes = mx_plan(batch, rows, cols, group, dev, nullptr).bytes;
    return PVS_OK;
}

extern "C" pvs_status pvs_mx_matmul(const void* x, int64_t ldx, int64_t batch, const uint8_t* codes,
                                    const uint8_t* scales, const float* row_scales, int64_t rows,
                                    int32_t cols, int32_t group, int32_t dtype, void* y, int64_t ldy,
                                    void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!mx_product_shape(batch, rows, cols, group, dtype) || ldx < cols || ldy < rows) return PVS_ERR_INVALID;
    if (batch == 0 || rows == 0) return PVS_OK;
    const int es = element_bytes(dtype);
    if (!x || !y || !on_elements(x, es) || !on_elements(y, es) || !mx_operand(codes, scales, row_scales, group))
        return PVS_ERR_INVALID;
    Device dev;
    if (device(&dev) != cudaSuccess) return mx_ended(cudaErrorUnknown);
    const MxPlan p = mx_plan(batch, rows, cols, group, dev, workspace);
    if (workspace_bytes < p.bytes || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return PVS_ERR_INVALID;
    const pvs_status before = (pvs_status)take_status(dev);
    if (before != PVS_OK) return before;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = launch_mx_pack(x, ldx, batch, cols, dtype, group, p.codes, p.scales, p.rows, st);
    if (e == cudaSuccess)
        e = mx_product(p, batch, codes, scales, row_scales, rows, cols, group, dtype, y, ldy, dev, st);
    return mx_ended(e);
}

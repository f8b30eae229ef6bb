// Rows of a table looked up by their ids, scaled, and the table's gradient (head.h).
//
//   forward    y_t = s w[id_t]
//   backward   dw_v = s sum_{t: id_t = v} dy_t, a float32 sum in the order of t
//
// Both are bound by memory.  The backward pass sorts (id, t) first, so that a row's sum runs
// over neighbours, nothing is added by atomics and the result depends on nothing but the
// call: up to kSmall ids in one block, more in three launches for each 10 bits.  Then a warp takes
// 32 (or 8) sorted entries by 256 columns, eight (or 16) rows' loads in flight, and writes the rows
// whose entries start among them; of rows with more than kLong entries the pieces' sums are
// kept in float32 and joined by a second launch.  Rows without an entry are found by search in
// the sorted ids and filled with zeros by other blocks of the first: no row of dw is written
// twice.
//
// 131,072 ids after Zipf's law in 200,000 rows of 1,024, bf16 (36,000 rows of them named), in us: lookup 66
// (5.1 TB/s of 342 MB; issue 64%), sorting 33 in six launches, sums and zeros 114 (6.0 TB/s of 678
// MB), long runs 15.  (All runs that cross a piece joined by the second launch: it took 300.)
// 5,000 in 10,007 of 385, float32: the gradient 30 in a graph (sorting 10, sums 13, long runs 6), latency.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "../../include/head.h"
#include "head_gemm.h"
#include "kernels.h"
#include "pvs_common.cuh"

namespace pvs {
namespace head {
namespace {

constexpr int kEmbedThreads = 256;
constexpr int kEmbedWarps = kEmbedThreads / 32;
constexpr int kSmall = 8192;         // ids that one block sorts
constexpr int kDigitBits = 10;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kKeysPerThread = 4;
constexpr int kSortTile = kEmbedThreads * kKeysPerThread;
constexpr int kSlab = 256;           // columns to a warp
constexpr int kLong = 32;            // entries of a run that one warp adds, at most

__device__ __forceinline__ uint16_t narrow(float v, int dtype) {
    if (dtype == PVS_BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
    return __half_as_ushort(__float2half_rn(v));
}
__device__ __forceinline__ void put(void* p, int dtype, int64_t i, float v) {
    if (dtype == PVS_F32)
        static_cast<float*>(p)[i] = v;
    else
        static_cast<uint16_t*>(p)[i] = narrow(v, dtype);
}
__device__ __forceinline__ void widen_two(uint32_t u, int dtype, float& lo, float& hi) {
    if (dtype == PVS_BF16) {
        lo = __uint_as_float(u << 16);
        hi = __uint_as_float(u & 0xffff0000u);
    } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
        lo = f.x;
        hi = f.y;
    }
}
__device__ __forceinline__ uint32_t narrow_two(float lo, float hi, int dtype) {
    if (dtype == PVS_BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Eight elements of a row, a lane's share of 256: neighbours (WIDE: the row is aligned to 16
// bytes and holds whole eights; as they lie, four words of 16-bit ones) or 32 apart.  Nothing is
// read past the row.
template <bool WIDE, int DT>
struct Share {
    static constexpr bool F32 = DT == PVS_F32;
    uint32_t u[WIDE && !F32 ? 4 : 8];

    __device__ __forceinline__ void load(const void* p, int64_t row, int col0, int dim) {
        const int lane = threadIdx.x & 31;
        if constexpr (WIDE) {
            const int c = col0 + 8 * lane;
            const uint4 none = make_uint4(0u, 0u, 0u, 0u);
            if constexpr (F32) {
                const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + row + c);
                const uint4 f = c < dim ? __ldg(q) : none, g = c < dim ? __ldg(q + 1) : none;
                u[0] = f.x, u[1] = f.y, u[2] = f.z, u[3] = f.w;
                u[4] = g.x, u[5] = g.y, u[6] = g.z, u[7] = g.w;
            } else {
                const uint4 f =
                    c < dim ? __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + row + c))
                            : none;
                u[0] = f.x, u[1] = f.y, u[2] = f.z, u[3] = f.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = col0 + lane + 32 * i;
                if constexpr (F32)
                    u[i] = c < dim ? __float_as_uint(__ldg(static_cast<const float*>(p) + row + c)) : 0u;
                else
                    u[i] = c < dim ? (uint32_t)__ldg(static_cast<const uint16_t*>(p) + row + c) : 0u;
            }
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if constexpr (WIDE && !F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) widen_two(u[i], DT, v[2 * i], v[2 * i + 1]);
        } else {
            // (a bf16 is the upper half of a float32)
            if (DT == PVS_F16) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __half2float(__ushort_as_half((uint16_t)u[i]));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(F32 ? u[i] : u[i] << 16);
            }
        }
    }
};
template <bool WIDE>
__device__ __forceinline__ void store_share(void* p, int dtype, int64_t row, int col0, int dim,
                                            const float (&v)[8]) {
    const int lane = threadIdx.x & 31;
    if constexpr (WIDE) {
        const int c = col0 + 8 * lane;
        if (c >= dim) return;
        if (dtype == PVS_F32) {
            float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + row + c);
            q[0] = make_float4(v[0], v[1], v[2], v[3]);
            q[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + row + c) =
                make_uint4(narrow_two(v[0], v[1], dtype), narrow_two(v[2], v[3], dtype),
                           narrow_two(v[4], v[5], dtype), narrow_two(v[6], v[7], dtype));
        }
    } else {
        if (dtype == PVS_F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = col0 + lane + 32 * i;
                if (c < dim) static_cast<float*>(p)[row + c] = v[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = col0 + lane + 32 * i;
                if (c < dim) static_cast<uint16_t*>(p)[row + c] = narrow(v[i], dtype);
            }
        }
    }
}

// ---- lookup ------------------------------------------------------------------------
struct LookupArgs {
    const void* w;
    int64_t ldw, items;
    const int64_t* ids;
    int64_t rows, ignore_index;
    int dim;
    float scale;
    void* y;
    int64_t ldy;
    int slabs;
    int lane_bits;                   // 2^this lanes to a row: 5, or fewer where that is all of it
};

// A warp takes neighbouring pieces of 256 columns of y, their loads in flight together: four of
// aligned rows, one of others (whose eight loads a lane are single elements: 200,000 rows of 385 in
// float32 took 110 us with four).
__host__ __device__ constexpr int lookups(bool wide) { return wide ? 4 : 1; }
template <bool WIDE, int DT>
__global__ void __launch_bounds__(kEmbedThreads) embed_forward_kernel(const LookupArgs a) {
    constexpr int kLookups = lookups(WIDE);
    next_early();
    wait_before();
    const int64_t p0 = ((int64_t)blockIdx.x * kEmbedWarps + (threadIdx.x >> 5)) * kLookups;
    int64_t row[kLookups], id[kLookups];
    int col0[kLookups];
    Share<WIDE, DT> in[kLookups];
    if (WIDE && a.lane_bits < 5) {
        // narrow rows: several of them side by side
        const int lane = threadIdx.x & 31, rows = 32 >> a.lane_bits;
        if (p0 * rows >= a.rows) return;
#pragma unroll
        for (int i = 0; i < kLookups; ++i) {
            row[i] = (p0 + i) * rows + (lane >> a.lane_bits);
            col0[i] = -8 * (lane >> a.lane_bits << a.lane_bits);
        }
    } else {
        if (p0 >= a.rows * a.slabs) return;
        row[0] = quotient_of(p0, a.slabs);
        col0[0] = (int)(p0 - row[0] * a.slabs) * kSlab;
#pragma unroll
        for (int i = 1; i < kLookups; ++i) {
            const bool next = col0[i - 1] + kSlab >= a.dim;
            row[i] = row[i - 1] + (next ? 1 : 0);
            col0[i] = next ? 0 : col0[i - 1] + kSlab;
        }
    }
#pragma unroll
    for (int i = 0; i < kLookups; ++i) id[i] = row[i] < a.rows ? __ldg(a.ids + row[i]) : a.ignore_index;
    // (no branches, so that all loads are under way at once: the table's first row for no row)
#pragma unroll
    for (int i = 0; i < kLookups; ++i) {
        const bool there = id[i] != a.ignore_index && id[i] >= 0 && id[i] < a.items;
        in[i].load(a.w, there ? id[i] * a.ldw : 0, col0[i], a.dim);
    }
#pragma unroll
    for (int i = 0; i < kLookups; ++i) {
        if (row[i] >= a.rows) break;
        float v[8];
        if (id[i] == a.ignore_index || id[i] < 0 || id[i] >= a.items) {
            const float f = id[i] == a.ignore_index ? 0.0f : __int_as_float(0x7fffffff);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = f;
        } else {
            in[i].values(v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= a.scale;
        }
        store_share<WIDE>(a.y, DT, row[i] * a.ldy, col0[i], a.dim, v);
    }
}

// ---- sorting -----------------------------------------------------------------------
// An id as a key: `items`, past every row, for what has no row.
__device__ __forceinline__ uint32_t key_of(int64_t id, int64_t ignore_index, int64_t items) {
    return id == ignore_index || id < 0 || id >= items ? (uint32_t)items : (uint32_t)id;
}

__device__ __forceinline__ uint32_t inclusive_sum(uint32_t v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}

// Up to kSmall ids in one block, eight bits a pass.  A warp ranks its neighbours in order, 32 at a
// time: equal digits among them by a match, those before by the warp's own counts.
constexpr int kBlockThreads = 1024;
constexpr int kBlockWarps = kBlockThreads / 32;
constexpr int kBlockKeys = kSmall / kBlockThreads;
constexpr int kBlockDigits = 256;
__global__ void __launch_bounds__(kBlockThreads) embed_sort_block_kernel(const int64_t* __restrict__ ids, int n,
                                                                         int bits, int64_t ignore_index,
                                                                         int64_t items, uint32_t* keys,
                                                                         uint32_t* places, uint32_t* longs) {
    extern __shared__ uint2 sorted[];
    __shared__ uint16_t count[kBlockWarps][kBlockDigits];
    __shared__ uint32_t first[kBlockDigits];
    __shared__ uint32_t sums[kBlockDigits / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    next_early();
    wait_before();
    if (threadIdx.x == 0) *longs = 0;
    const int rounds = (n + kBlockThreads - 1) / kBlockThreads;
    const int base = warp * 32 * rounds + lane;
    uint2 entry[kBlockKeys];
    uint32_t rank[kBlockKeys];
#pragma unroll
    for (int r = 0; r < kBlockKeys; ++r) {
        const int i = base + 32 * r;
        if (r < rounds && i < n) entry[r] = make_uint2(key_of(ids[i], ignore_index, items), (uint32_t)i);
    }
    for (int shift = 0; shift < bits; shift += 8) {
        for (int i = threadIdx.x; i < kBlockWarps * kBlockDigits / 2; i += kBlockThreads)
            reinterpret_cast<uint32_t*>(&count[0][0])[i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kBlockKeys; ++r) {
            if (r >= rounds) break;
            const bool in = base + 32 * r < n;
            const int d = in ? (int)(entry[r].x >> shift & 255u) : kBlockDigits;
            const uint32_t peers = __match_any_sync(0xffffffffu, d);
            const uint32_t before = in ? count[warp][d] : 0u;
            rank[r] = before + __popc(peers & ((1u << lane) - 1u));
            __syncwarp();
            if (in && lane == 31 - __clz(peers)) count[warp][d] = (uint16_t)(before + __popc(peers));
            __syncwarp();
        }
        __syncthreads();
        uint32_t total = 0;
        if (threadIdx.x < kBlockDigits) {
#pragma unroll 8
            for (int w = 0; w < kBlockWarps; ++w) {
                const uint32_t c = count[w][threadIdx.x];
                count[w][threadIdx.x] = (uint16_t)total;
                total += c;
            }
            const uint32_t incl = inclusive_sum(total);
            if (lane == 31) sums[warp] = incl;
            first[threadIdx.x] = incl - total;
        }
        __syncthreads();
        if (threadIdx.x < kBlockDigits) {
            uint32_t start = 0;
            for (int w = 0; w < warp; ++w) start += sums[w];
            first[threadIdx.x] += start;
        }
        __syncthreads();
        const bool last = shift + 8 >= bits;
#pragma unroll
        for (int r = 0; r < kBlockKeys; ++r) {
            if (r >= rounds || base + 32 * r >= n) break;
            const int d = (int)(entry[r].x >> shift & 255u);
            const uint32_t to = first[d] + count[warp][d] + rank[r];
            if (last) {
                keys[to] = entry[r].x;
                places[to] = entry[r].y;
            } else {
                sorted[to] = entry[r];
            }
        }
        if (last) break;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kBlockKeys; ++r)
            if (r < rounds && base + 32 * r < n) entry[r] = sorted[base + 32 * r];
        // (the counts are cleared after this, and a barrier comes before the next entries)
    }
}

struct SortArgs {
    const int64_t* ids;              // of the first pass, else null
    int64_t ignore_index, items;
    const uint32_t *keys, *places;   // of the passes after it
    uint32_t *keys_out, *places_out;
    int64_t n;
    int shift, digits;               // this pass's digit
    int64_t tiles;
    uint32_t* counts;                // [digits][tiles]
    uint32_t* totals;                // [digits]
    uint32_t* longs;                 // of the sums: cleared
};
__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int64_t i) {
    return a.ids ? key_of(a.ids[i], a.ignore_index, a.items) : a.keys[i];
}
__device__ __forceinline__ int digit_of(const SortArgs& a, uint32_t key) {
    return (int)(key >> a.shift) & (a.digits - 1);
}

// How often each digit comes in each tile.
__global__ void __launch_bounds__(kEmbedThreads) embed_count_kernel(const SortArgs a) {
    __shared__ uint32_t count[kDigits];
    for (int d = threadIdx.x; d < a.digits; d += kEmbedThreads) count[d] = 0;
    next_early();
    wait_before();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.longs = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kSortTile;
#pragma unroll
    for (int r = 0; r < kKeysPerThread; ++r) {
        const int64_t i = base + r * kEmbedThreads + threadIdx.x;
        if (i < a.n) atomicAdd(&count[digit_of(a, sort_key(a, i))], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < a.digits; d += kEmbedThreads)
        a.counts[d * a.tiles + blockIdx.x] = count[d];
}

// A digit's counts to what comes before each tile; a warp to a digit.
__global__ void __launch_bounds__(kEmbedThreads) embed_scan_kernel(const SortArgs a) {
    next_early();
    wait_before();
    const int d = blockIdx.x * kEmbedWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (d >= a.digits) return;
    uint32_t before = 0;
    for (int64_t t0 = 0; t0 < a.tiles; t0 += 32) {
        const int64_t t = t0 + lane;
        const uint32_t v = t < a.tiles ? a.counts[d * a.tiles + t] : 0u;
        const uint32_t s = inclusive_sum(v);
        if (t < a.tiles) a.counts[d * a.tiles + t] = before + s - v;
        before += __shfl_sync(0xffffffffu, s, 31);
    }
    if (lane == 0) a.totals[d] = before;
}

// A tile's entries to their places.  A warp ranks its 256 neighbours in order, 32 at a time:
// equal digits among them by a match, those before by the warp's own counts.
__global__ void __launch_bounds__(kEmbedThreads) embed_place_kernel(const SortArgs a) {
    __shared__ uint16_t count[kEmbedWarps][kDigits];
    __shared__ uint32_t first[kDigits];
    __shared__ uint32_t sums[kEmbedWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < kEmbedWarps * a.digits; i += kEmbedThreads)
        count[i / a.digits][i % a.digits] = 0;
    next_early();
    wait_before();
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kSortTile + warp * 32 * kKeysPerThread;
    uint32_t key[kKeysPerThread], place[kKeysPerThread], rank[kKeysPerThread];
#pragma unroll
    for (int r = 0; r < kKeysPerThread; ++r) {
        const int64_t i = base + 32 * r + lane;
        key[r] = i < a.n ? sort_key(a, i) : 0u;
        place[r] = i < a.n ? (a.ids ? (uint32_t)i : a.places[i]) : 0u;
    }
#pragma unroll
    for (int r = 0; r < kKeysPerThread; ++r) {
        const bool in = base + 32 * r + lane < a.n;
        const int d = in ? digit_of(a, key[r]) : kDigits;
        const uint32_t peers = __match_any_sync(0xffffffffu, d);
        const uint32_t before = in ? count[warp][d] : 0u;
        rank[r] = before + __popc(peers & ((1u << lane) - 1u));
        __syncwarp();
        if (in && lane == 31 - __clz(peers)) count[warp][d] = (uint16_t)(before + __popc(peers));
        __syncwarp();
    }
    // where each digit starts among all: a scan of the totals, four to a thread
    const int per = kDigits / kEmbedThreads;
    uint32_t mine[per], sum = 0;
#pragma unroll
    for (int k = 0; k < per; ++k) {
        const int d = threadIdx.x * per + k;
        mine[k] = sum;
        if (d < a.digits) sum += a.totals[d];
    }
    const uint32_t incl = inclusive_sum(sum);
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    uint32_t start = incl - sum;
    for (int w = 0; w < warp; ++w) start += sums[w];
#pragma unroll
    for (int k = 0; k < per; ++k) {
        const int d = threadIdx.x * per + k;
        if (d < a.digits) {
            first[d] = start + mine[k] + a.counts[d * a.tiles + blockIdx.x];
            uint32_t before = 0;
            for (int w = 0; w < kEmbedWarps; ++w) {
                const uint32_t c = count[w][d];
                count[w][d] = (uint16_t)before;
                before += c;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kKeysPerThread; ++r) {
        if (base + 32 * r + lane >= a.n) continue;
        const int d = digit_of(a, key[r]);
        const uint32_t to = first[d] + count[warp][d] + rank[r];
        a.keys_out[to] = key[r];
        a.places_out[to] = place[r];
    }
}

// ---- sums --------------------------------------------------------------------------
struct SumArgs {
    const void* dy;
    int64_t lddy;
    const uint32_t *keys, *places;
    int64_t n, items;
    int dim, dtype, slabs;
    float scale;
    void* dw;
    int64_t lddw;
    float* part;                     // [piece][2][ldp]: of a long run from before, and one that starts
    int64_t ldp;
    int64_t pieces, sum_blocks;
    int zero_rows;                   // table rows to a warp, a multiple of 32
    int zero_bits;                   // 2^this warps share them, 0 to 3
    int lane_bits;                   // lanes to a row of zeros: 2^this
    uint32_t* longs;                 // [0] how many pieces a long run starts in, then which
};

// The first of the sorted keys that is v or more.
__device__ __forceinline__ int64_t lower_bound(const uint32_t* keys, int64_t n, uint32_t v) {
    int64_t lo = 0;
    while (n > 0) {
        const int64_t half = n >> 1;
        if (__ldg(keys + lo + half) < v) {
            lo += half + 1;
            n -= half + 1;
        } else {
            n = half;
        }
    }
    return lo;
}

// Zeros to those of `rows` (a bit each) of the 32 table rows from v0 that are set: as many rows at
// once as the warp's lanes hold.
template <bool WIDE, int DT>
__device__ __forceinline__ void put_zeros(const SumArgs& a, int64_t v0, uint32_t rows) {
    constexpr int kStep = WIDE ? 8 : 1;                    // elements a lane
    const int lane = threadIdx.x & 31, shift = a.lane_bits;
    const int in = lane >> shift, first = (lane & ((1 << shift) - 1)) * kStep, step = kStep << shift;
    for (int r = in; r < 32; r += 32 >> shift) {
        if (!(rows >> r & 1u)) continue;
        const int64_t at = (v0 + r) * a.lddw;
        if constexpr (!WIDE && DT != PVS_F32) {
            // words of two elements, and an element before or after them
            uint16_t* p = static_cast<uint16_t*>(a.dw) + at;
            const int head = (int)(reinterpret_cast<uintptr_t>(p) >> 1 & 1u), words = (a.dim - head) / 2;
            uint32_t* q = reinterpret_cast<uint32_t*>(p + head);
            for (int c = first; c < words; c += step) q[c] = 0;
            if (first == 0 && head) p[0] = 0;
            if (first == 0 && (a.dim - head) % 2) p[a.dim - 1] = 0;
        } else {
            for (int c = first; c < a.dim; c += step) {
                if constexpr (!WIDE) {
                    static_cast<float*>(a.dw)[at + c] = 0.0f;
                } else if constexpr (DT == PVS_F32) {
                    float4* q = reinterpret_cast<float4*>(static_cast<float*>(a.dw) + at + c);
                    q[0] = q[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                } else {
                    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.dw) + at + c) = make_uint4(0u, 0u, 0u, 0u);
                }
            }
        }
    }
}

// The rows without an entry of a.zero_rows table rows, 32 at a time.  The lanes search for the
// groups' first entries at once; a group of few entries shows its rows in one load, one of many is
// searched row by row.
template <bool WIDE, int DT>
__device__ void zero_rows(const SumArgs& a, int64_t first, uint32_t mine) {
    const int lane = threadIdx.x & 31;
    const int64_t end = min(first + a.zero_rows, a.items);
    const int64_t bound = lower_bound(a.keys, a.n, (uint32_t)min(first + 32 * lane, end));
    for (int g = 0; first + 32 * g < end; ++g) {
        const int64_t v0 = first + 32 * g;
        const int64_t lo = __shfl_sync(0xffffffffu, bound, g), hi = __shfl_sync(0xffffffffu, bound, g + 1);
        uint32_t used;
        if (hi - lo <= 32) {
            const bool in = lo + lane < hi;
            used = __reduce_or_sync(0xffffffffu, in ? 1u << (__ldg(a.keys + lo + lane) - (uint32_t)v0) : 0u);
        } else {
            const uint32_t row = (uint32_t)v0 + lane;
            const int64_t at = lo + lower_bound(a.keys + lo, hi - lo, row);
            used = __ballot_sync(0xffffffffu, at < hi && __ldg(a.keys + at) == row);
        }
        const int here = (int)min((int64_t)32, end - v0);
        put_zeros<WIDE, DT>(a, v0, mine & ~used & (here == 32 ? 0xffffffffu : (1u << here) - 1u));
    }
}

// A lane's sums over eight of a warp's 256 columns, and where they go.
template <bool WIDE, int DT>
struct Sum {
    const SumArgs& a;
    int col0;
    float acc[8];

    __device__ __forceinline__ Sum(const SumArgs& a, int col0) : a(a), col0(col0) { clear(); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] = 0.0f;
    }
    __device__ __forceinline__ void row(uint32_t key) {
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] *= a.scale;
        store_share<WIDE>(a.dw, DT, (int64_t)key * a.lddw, col0, a.dim, acc);
        clear();
    }
    __device__ __forceinline__ void piece(int64_t slot) {
        store_share<WIDE>(a.part + slot * a.ldp, PVS_F32, 0, col0, a.dim, acc);
        clear();
    }
};

// kPiece sorted entries to a warp, and 256 columns.  Blocks to an SM: as many as the rows in flight
// leave registers for; small calls (pieces of eight) have few blocks and twice the rows in flight.
constexpr int sum_blocks_of(bool wide, int dtype, int piece) {
    return piece == 8 ? 1 : wide && dtype != PVS_F32 ? 3 : 2;
}
template <bool WIDE, int DT, int kPiece>
__global__ void __launch_bounds__(kEmbedThreads, sum_blocks_of(WIDE, DT, kPiece))
    embed_sum_kernel(const SumArgs a) {
    next_early();
    wait_before();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // blocks that sum and blocks that write zeros take turns, so that reads and writes overlap, as
    // long as there are both
    const int64_t b = blockIdx.x, zero_blocks = gridDim.x - a.sum_blocks;
    const int64_t turns = min(a.sum_blocks, zero_blocks);
    const bool sums = b < 2 * turns ? (b & 1) == 0 : a.sum_blocks > turns;
    const int64_t of_kind = b < 2 * turns ? b >> 1 : b - turns;
    if (!sums) {
        // (2^zero_bits warps share the rows of a group)
        const int64_t w = of_kind * kEmbedWarps + warp;
        const int64_t step = (zero_blocks * kEmbedWarps >> a.zero_bits) * a.zero_rows;
        const uint32_t mine = (a.zero_bits == 0   ? 0xffffffffu
                               : a.zero_bits == 1 ? 0x55555555u
                               : a.zero_bits == 2 ? 0x11111111u
                                                  : 0x01010101u)
                              << (w & ((1 << a.zero_bits) - 1));
        for (int64_t v = (w >> a.zero_bits) * a.zero_rows; v < a.items; v += step) zero_rows<WIDE, DT>(a, v, mine);
        return;
    }
    const int64_t u = of_kind * kEmbedWarps + warp;
    const int64_t piece = quotient_of(u, a.slabs);
    if (piece >= a.pieces) return;
    const int col0 = (int)(u - piece * a.slabs) * kSlab;
    const int64_t base = piece * kPiece;
    const uint32_t none = (uint32_t)a.items;
    // three windows of 32 keys, the middle one from this piece's first: a run of equal keys is long
    // when it has more than kLong = 32 entries, which every piece that it meets sees alike
    uint32_t k[3], place[2];
#pragma unroll
    for (int w = 0; w < 3; ++w) {
        const int64_t i = base + 32 * (w - 1) + lane;
        k[w] = i >= 0 && i < a.n ? __ldg(a.keys + i) : none;
        if (w >= 1) place[w - 1] = i < a.n ? __ldg(a.places + i) : 0u;
    }
    // entries without a row come last
    constexpr int kFlight = kPiece == 8 ? 16 : 8;    // rows whose loads are under way at once
    constexpr uint32_t kHere = kPiece == 32 ? 0xffffffffu : (1u << (kPiece & 31)) - 1u;
    const int count = __popc(__ballot_sync(0xffffffffu, k[1] != none) & kHere);
    if (count == 0) return;
    const uint32_t head = __shfl_sync(0xffffffffu, k[1], 0);
    const uint32_t tail = __shfl_sync(0xffffffffu, k[1], count - 1);
    // how far the first entry's run reaches back, and in; where the last one's starts, and how far
    // it goes past the piece (32 at most)
    const int back = base == 0 ? 0 : __clz(~__ballot_sync(0xffffffffu, k[0] == head));
    const int head_in = min(kPiece, __clz(__brev(~__ballot_sync(0xffffffffu, k[1] == head))));
    const uint32_t same = __ballot_sync(0xffffffffu, k[1] == tail);
    const uint32_t same_next = __ballot_sync(0xffffffffu, k[2] == tail);
    const int tail_at = __ffs(same) - 1;
    int after = 0;
    if (count == kPiece) {
        const uint64_t differ = ~(((uint64_t)same_next << 32 | same) >> kPiece);
        after = min(kLong, __ffsll((long long)differ) - 1);
    }
    const bool one_run = head_in == kPiece;
    int first = 0, last = count;                 // entries that this warp adds
    bool head_part = false, tail_part = false;   // as parts of long runs
    if (back > 0) {
        head_part = back + (one_run ? kPiece + after : head_in) > kLong;
        if (!head_part) first = head_in;         // the piece that it starts in has it
    }
    if (after > 0 && !(one_run && back > 0)) {
        tail_part = kPiece - tail_at + after > kLong;
        if (!tail_part) last = kPiece + after;
        if (tail_part && lane == 0 && col0 == 0) a.longs[1 + atomicAdd(a.longs, 1u)] = (uint32_t)piece;
    }
    Sum<WIDE, DT> sum(a, col0);
    for (int i0 = first; i0 < last; i0 += kFlight) {
        Share<WIDE, DT> in[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int at = i0 + i;
            const uint32_t p0 = __shfl_sync(0xffffffffu, place[0], at & 31);
            const uint32_t p1 = __shfl_sync(0xffffffffu, place[1], at & 31);
            if (at < last) in[i].load(a.dy, (int64_t)(at < 32 ? p0 : p1) * a.lddy, col0, a.dim);
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int at = i0 + i;
            if (at >= last) break;
            float v[8];
            in[i].values(v);
#pragma unroll
            for (int c = 0; c < 8; ++c) sum.acc[c] += v[c];
            if (at + 1 == last) break;
            // (past the piece it is all one run)
            const uint32_t here = __shfl_sync(0xffffffffu, k[1], at & 31);
            const uint32_t next = __shfl_sync(0xffffffffu, k[1], (at + 1) & 31);
            if (at + 1 >= kPiece || here == next) continue;
            if (head_part && at < head_in)
                sum.piece(2 * piece);
            else
                sum.row(here);
        }
    }
    if (first >= last) return;
    if (head_part && last <= head_in)
        sum.piece(2 * piece);
    else if (tail_part)
        sum.piece(2 * piece + 1);
    else
        sum.row(tail);
}

// The long runs: their pieces' sums, by eight groups of threads a stretch of the pieces each, and
// the groups' sums in their order.
constexpr int kJoinThreads = 512;
constexpr int kJoinLanes = 64;       // of four columns
constexpr int kJoinGroups = kJoinThreads / kJoinLanes;
__global__ void __launch_bounds__(kJoinThreads) embed_join_kernel(const SumArgs a, int slabs, int piece_keys) {
    __shared__ float4 sh[kJoinGroups][kJoinLanes];
    next_early();
    wait_before();
    const int64_t total = (int64_t)a.longs[0] * slabs;
    const int group = threadIdx.x / kJoinLanes, lane = threadIdx.x % kJoinLanes;
    for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
        const int64_t piece = a.longs[1 + u / slabs];
        const int col = (int)(u % slabs) * 4 * kJoinLanes + 4 * lane;
        const uint32_t key = __ldg(a.keys + (piece + 1) * piece_keys - 1);
        // the pieces that start with its key follow one another
        int64_t last = piece;
        for (int found = kJoinThreads; found == kJoinThreads; last += found) {
            const int64_t at = (last + 1 + threadIdx.x) * piece_keys;
            found = __syncthreads_count(at < a.n && __ldg(a.keys + min(at, a.n - 1)) == key);
        }
        const int64_t each = (last - piece + kJoinGroups) / kJoinGroups;
        const int64_t q0 = piece + group * each, q1 = min(q0 + each, last + 1);
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (col < a.ldp) {
#pragma unroll 8
            for (int64_t q = q0; q < q1; ++q) {
                const float4 v = __ldg(reinterpret_cast<const float4*>(
                    a.part + (2 * q + (q == piece ? 1 : 0)) * a.ldp + col));
                s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
            }
        }
        sh[group][lane] = s;
        __syncthreads();
        if (group == 0) {
            for (int g = 1; g < kJoinGroups && piece + g * each <= last; ++g) {
                const float4 v = sh[g][lane];
                s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
            }
            const float f[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (col + c < a.dim) put(a.dw, a.dtype, (int64_t)key * a.lddw + col + c, f[c] * a.scale);
        }
        __syncthreads();
    }
}

// ---- the plan of a call --------------------------------------------------------------
struct EmbedPlan {
    int piece = 0;                   // sorted entries to a warp: 32, or 8 where those leave SMs idle
    int passes = 0, bits = 0;
    int64_t tiles = 0, pieces = 0, ldp = 0;
    uint32_t *keys[2] = {}, *places[2] = {}, *counts = nullptr, *totals = nullptr, *longs = nullptr;
    float* part = nullptr;
    size_t bytes = 0;
};

// Pieces of 32 by 256 columns that give each of 152 SMs eight warps (5,000 rows of 385 took a sum of
// 44 us in them).  A constant, not the device's count: the order of a sum and the scratch, which are
// the call's alone, follow from it.
constexpr int64_t kFewUnits = 32 * 8 * 152;

EmbedPlan embed_plan(int64_t n, int64_t items, int dim, void* workspace) {
    EmbedPlan p;
    Carver c{static_cast<uint8_t*>(workspace)};
    p.keys[0] = c.take<uint32_t>(n);
    p.places[0] = c.take<uint32_t>(n);
    int width = 1;
    while (items >> width) ++width;                    // of the largest key, `items`
    p.bits = width;
    if (n > kSmall) {
        p.passes = (width + kDigitBits - 1) / kDigitBits;
        p.bits = (width + p.passes - 1) / p.passes;
        p.tiles = (n + kSortTile - 1) / kSortTile;
        if (p.passes > 1) {
            p.keys[1] = c.take<uint32_t>(n);
            p.places[1] = c.take<uint32_t>(n);
        }
        p.counts = c.take<uint32_t>(p.tiles << p.bits);
        p.totals = c.take<uint32_t>((int64_t)1 << p.bits);
    }
    p.piece = n * ((dim + kSlab - 1) / kSlab) < kFewUnits ? 8 : 32;
    p.pieces = (n + p.piece - 1) / p.piece;
    p.ldp = round_up(dim, 8);
    p.longs = c.take<uint32_t>(1 + p.pieces);
    if (p.pieces > 1) p.part = c.take<float>(p.pieces * 2 * p.ldp);
    p.bytes = c.used;
    return p;
}

bool embed_shape(int64_t rows, int64_t items, int32_t dim, int32_t dtype) {
    return rows >= 0 && rows <= kMaxRows && items >= 1 && items <= kMaxRows && dim >= 1 && dim <= 32767 &&
           dtype >= PVS_BF16 && dtype <= PVS_F32;
}
bool on_16(const void* p, int64_t ld, int dtype) {
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % (dtype == PVS_F32 ? 4 : 8) == 0;
}
pvs_status embed_ended(cudaError_t e) {
    if (e == cudaSuccess) return PVS_OK;
    cudaGetLastError();
    return PVS_ERR_CUDA;
}

using LookupKernel = void (*)(const LookupArgs);
using SumKernel = void (*)(const SumArgs);
template <int DT>
LookupKernel lookup_kernel(bool wide) {
    return wide ? embed_forward_kernel<true, DT> : embed_forward_kernel<false, DT>;
}
template <int DT>
SumKernel sum_kernel(bool wide, int piece) {
    if (piece == 8) return wide ? embed_sum_kernel<true, DT, 8> : embed_sum_kernel<false, DT, 8>;
    return wide ? embed_sum_kernel<true, DT, 32> : embed_sum_kernel<false, DT, 32>;
}

// The sorted entries' place in the plan's buffers.
cudaError_t sort_ids(const int64_t* ids, int64_t n, int64_t items, int64_t ignore_index,
                     const EmbedPlan& p, int* where, cudaStream_t st) {
    *where = 0;
    if (p.passes == 0) {
        const cudaError_t e = raise_smem_limit((const void*)embed_sort_block_kernel, kSmall * 8);
        if (e != cudaSuccess) return e;
        count_launches(1);
        return launch_early(embed_sort_block_kernel, 1, kBlockThreads, (size_t)n * 8, st, ids, (int)n, p.bits,
                            ignore_index, items, p.keys[0], p.places[0], p.longs);
    }
    cudaError_t e = cudaSuccess;
    for (int i = 0; i < p.passes && e == cudaSuccess; ++i) {
        // the last pass ends in the first buffers
        const int to = (p.passes - 1 - i) & 1;
        SortArgs s{};
        s.ids = i == 0 ? ids : nullptr;
        s.ignore_index = ignore_index;
        s.items = items;
        s.keys = p.keys[to ^ 1];
        s.places = p.places[to ^ 1];
        s.keys_out = p.keys[to];
        s.places_out = p.places[to];
        s.n = n;
        s.shift = i * p.bits;
        s.digits = 1 << p.bits;
        s.tiles = p.tiles;
        s.counts = p.counts;
        s.totals = p.totals;
        s.longs = p.longs;
        count_launches(3);
        e = launch_early(embed_count_kernel, p.tiles, kEmbedThreads, 0, st, s);
        if (e == cudaSuccess)
            e = launch_early(embed_scan_kernel, (s.digits + kEmbedWarps - 1) / kEmbedWarps, kEmbedThreads,
                             0, st, s);
        if (e == cudaSuccess) e = launch_early(embed_place_kernel, p.tiles, kEmbedThreads, 0, st, s);
    }
    return e;
}

}  // namespace
}  // namespace head
}  // namespace pvs

using namespace pvs;
using namespace pvs::head;

extern "C" pvs_status pvs_embed_forward(const void* w, int64_t ldw, int64_t items, int32_t dim,
                                        int32_t dtype, const int64_t* ids, int64_t rows, float scale,
                                        int64_t ignore_index, void* y, int64_t ldy, void* cuda_stream) {
    if (!embed_shape(rows, items, dim, dtype) || ldw < dim || ldy < dim || !std::isfinite(scale))
        return PVS_ERR_INVALID;
    if (rows == 0) return PVS_OK;
    const int es = element_bytes(dtype);
    if (!w || !ids || !y || !on_elements(w, es) || !on_elements(y, es) || !on_elements(ids, 8))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    LookupArgs a{};
    a.w = w;
    a.ldw = ldw;
    a.items = items;
    a.ids = ids;
    a.rows = rows;
    a.ignore_index = ignore_index;
    a.dim = dim;
    a.scale = scale;
    a.y = y;
    a.ldy = ldy;
    a.slabs = (dim + kSlab - 1) / kSlab;
    const bool wide = dim % 8 == 0 && on_16(w, ldw, dtype) && on_16(y, ldy, dtype);
    a.lane_bits = 5;
    while (wide && a.lane_bits > 0 && 8 << (a.lane_bits - 1) >= dim) --a.lane_bits;
    const int64_t per_block = (int64_t)kEmbedWarps * lookups(wide) * (32 >> a.lane_bits);
    const int64_t blocks = (rows * a.slabs + per_block - 1) / per_block;
    if (blocks > 0x7fffffff) return PVS_ERR_INVALID;
    count_launches(1);
    return embed_ended(launch_early(dtype == PVS_F32   ? lookup_kernel<PVS_F32>(wide)
                                    : dtype == PVS_F16 ? lookup_kernel<PVS_F16>(wide)
                                                       : lookup_kernel<PVS_BF16>(wide),
                                    blocks, kEmbedThreads, 0,
                                    static_cast<cudaStream_t>(cuda_stream), a));
}

extern "C" pvs_status pvs_embed_workspace(int64_t rows, int64_t items, int32_t dim, size_t* bytes) {
    if (!bytes || !embed_shape(rows, items, dim, PVS_F32)) return PVS_ERR_INVALID;
    *bytes = rows == 0 ? 0 : embed_plan(rows, items, dim, nullptr).bytes;
    return PVS_OK;
}

extern "C" pvs_status pvs_embed_backward(const void* dy, int64_t lddy, const int64_t* ids, int64_t rows,
                                         int64_t items, int32_t dim, int32_t dtype, float scale,
                                         int64_t ignore_index, void* dw, int64_t lddw, void* workspace,
                                         size_t workspace_bytes, void* cuda_stream) {
    if (!embed_shape(rows, items, dim, dtype) || lddy < dim || lddw < dim || !std::isfinite(scale))
        return PVS_ERR_INVALID;
    const int es = element_bytes(dtype);
    if (!dw || !on_elements(dw, es)) return PVS_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (rows > 0 && (!dy || !ids || !on_elements(dy, es) || !on_elements(ids, 8))) return PVS_ERR_INVALID;
    const EmbedPlan p = rows > 0 ? embed_plan(rows, items, dim, workspace) : EmbedPlan{};
    if (workspace_bytes < p.bytes ||
        (p.bytes > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))))
        return PVS_ERR_INVALID;
    Device dev;
    const pvs_status before = (pvs_status)ready(&dev);
    if (before != PVS_OK) return before;
    if (rows == 0)
        return embed_ended(cudaMemset2DAsync(dw, (size_t)lddw * es, 0, (size_t)dim * es, (size_t)items, st));
    int where = 0;
    cudaError_t e = sort_ids(ids, rows, items, ignore_index, p, &where, st);
    if (e != cudaSuccess) return embed_ended(e);
    SumArgs a{};
    a.dy = dy;
    a.lddy = lddy;
    a.keys = p.keys[where];
    a.places = p.places[where];
    a.n = rows;
    a.items = items;
    a.dim = dim;
    a.dtype = dtype;
    a.slabs = (dim + kSlab - 1) / kSlab;
    a.scale = scale;
    a.dw = dw;
    a.lddw = lddw;
    a.part = p.part;
    a.ldp = p.ldp;
    a.pieces = p.pieces;
    a.longs = p.longs;
    a.sum_blocks = (p.pieces * a.slabs + kEmbedWarps - 1) / kEmbedWarps;
    const bool wide = dim % 8 == 0 && on_16(dy, lddy, dtype) && on_16(dw, lddw, dtype);
    // 32 to 256 rows a warp, or up to eight warps to 32 rows, so that there are warps for every SM
    const int64_t groups = (items + 31) / 32, enough = 16ll * dev.sms;
    a.zero_rows = 32 * (int)std::min<int64_t>(8, std::max<int64_t>(1, groups / enough));
    while (a.zero_bits < 3 && groups << (a.zero_bits + 1) <= enough) ++a.zero_bits;
    while (a.lane_bits < 5 && (wide ? 8 : 1) << a.lane_bits < dim) ++a.lane_bits;
    const int64_t units = ((items + a.zero_rows - 1) / a.zero_rows) << a.zero_bits;
    const int64_t zero = std::min<int64_t>((units + kEmbedWarps - 1) / kEmbedWarps, (int64_t)1 << 20);
    count_launches(1);
    e = launch_early(dtype == PVS_F32   ? sum_kernel<PVS_F32>(wide, p.piece)
                     : dtype == PVS_F16 ? sum_kernel<PVS_F16>(wide, p.piece)
                                        : sum_kernel<PVS_BF16>(wide, p.piece),
                     a.sum_blocks + zero, kEmbedThreads, 0, st, a);
    if (e != cudaSuccess || p.pieces < 2) return embed_ended(e);
    if (rows <= kLong) return PVS_OK;            // (no run is long)
    const int slabs = (int)((p.ldp + 4 * kJoinLanes - 1) / (4 * kJoinLanes));
    const int64_t most = std::min<int64_t>(rows / kLong * slabs, 4 * dev.sms);
    count_launches(1);
    return embed_ended(launch_early(embed_join_kernel, most, kJoinThreads, 0, st, a, slabs, p.piece));
}

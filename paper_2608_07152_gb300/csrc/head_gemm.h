// The tensor-core product of the projection head's operators (internal).
//
//   D[m, n] = sum_k A[m, k] B[n, k], float32 accumulators in TMEM,
//
// over operands of 16-bit elements in either order (K contiguous, or M / N
// contiguous), each in up to three parts that add up to it: the product then
// runs over a list of part pairs.  What becomes of D is the kernel's choice:
//   kStats   softmax statistics of D's rows, tile by tile (forward);
//   kTopStats  the same without the items of a list that each row has;
//   kGrad    the softmax gradient of each entry, kept in 16-bit parts (backward);
//   kOut     D itself, split over k where that fills the GPU.
#pragma once

#include <cstdint>

#include <cuda.h>
#include <cuda_runtime.h>

namespace pvs {
namespace head {

constexpr int kTileM = 128;     // a CTA; a pair's tile has 256 rows
constexpr int kTileN = 256;     // at most; a product may use fewer columns (bn, in steps of 32)
constexpr int kTileK = 64;      // 128 bytes: one swizzle row
constexpr int kMaxParts = 3;
constexpr int kMaxPairs = 6;

enum Epilogue { kStats = 0, kGrad = 1, kOut = 2, kTopStats = 3 };

// An operand in memory: `parts` matrices [rows x cols] of 16-bit elements,
// leading dimension ld, part_stride elements apart.  Base 16-byte aligned, ld and
// part_stride multiples of 8.
struct Matrix {
    const void* p;
    int64_t rows, cols, ld;
    int parts;
    int64_t part_stride;
};

struct Problem {
    CUtensorMap a, b, b_alt;     // b_alt in place of b where *alt_flag is set
    const int* alt_flag;
    int a_mn, b_mn;              // 1: M (N) is the contiguous index
    int m, n;                    // extents of D
    int bn;                      // columns per tile: a multiple of 32, <= kTileN
    int mtiles, ntiles, splits;
    int kchunks;                 // chunks of kTileK for one pair of parts
    int ktail;                   // steps of 16 in the last of them
    int klength;                 // launch_gemm: chunks of a split (the last may have fewer)
    int a_mo, a_ko, b_no, b_ko;  // where D's corner lies in the operands
    int alt_no, alt_ko;          // the same in b_alt
    int m_fast;                  // units run over m first (else n first)
    int units;                   // mtiles * ntiles * splits
    // kOut: splits > 1 or accumulate: float32 sums slots[split][m][n];
    // else out = alpha D, rounded once
    float* slots;
    int64_t slot_stride, ldslot;
    int accumulate, to_slots;
    void* out;
    int64_t ldout;
    int out_type;                // pvs_dtype
    const float* alpha;          // device, null: 1
    float alpha0;
};

// A row of the backward pass: G = coef 2^(l - m), and `hit` at item y.
struct alignas(16) GradRow {
    float m, coef, hit;
    int y;                       // -1: none
};

struct Softmax {
    float k2;                    // scale log2(e): logits are powers of two
    const float* row_unit;       // float32 operands: what D's rows and columns (the piece's
    const float* col_unit;       // items) are in units of; else null
    const float* bias;           // of the whole vocabulary, or null
    int item0;                   // the piece's first item
    int rows;
    // kStats
    float2* part;                // [tile of columns][rows]
    int part0;                   // the piece's first tile
    const int64_t* targets;      // a row's own target is left out of its statistics
    // kTopStats: so are the items of its list, ascending, `top` of them ([rows][top], those
    // that are none INT_MAX at the end); a tile's begin at list_first [tile of columns][rows]
    const int* list;
    const uint16_t* list_first;
    int top;
    // kGrad
    const GradRow* row;
    uint16_t* grad;              // [parts][rows][ldg]
    int64_t ldg, grad_part;
    int grad_parts, grad_f16;
    int* bad_masked;             // set where a masked item's logit is not finite
};

struct Args {
    Problem p[2];
    int nprob;
    int npairs;
    uint8_t pa[kMaxPairs], pb[kMaxPairs];
    int f16;
    int cta;                     // CTAs to a tile: 1, or 2 (a pair)
    int slots0;                  // of two problems, the CTAs (pairs) of the first; 0: by work
    Softmax sm;
    int* status;
    unsigned long long wait_ns;  // set by the launch: the limit of a wait
};

// A kernel of a call may be put on the SMs while the one before it ends: its setup then
// costs nothing.  Every kernel launched with launch_early() first lets the next one
// start (next_early) and, before it touches memory, waits for the one before it to be
// complete and visible (wait_before); nothing before the wait depends on memory.
#ifdef __CUDACC__
__device__ __forceinline__ void next_early() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ void wait_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// n / d, n >= 0, d > 0: in 32 bits where n has no more (in 64 a division is some 70 instructions).
__device__ __forceinline__ int64_t quotient_of(int64_t n, int d) {
    return n <= 0xffffffffll ? (int64_t)((uint32_t)n / (uint32_t)d) : n / d;
}

// v a b where one scale alone may take v out of float32's normal range although the product is in it:
// by both scales' product where they are on both sides of 1 (it is between them), else by the larger
// first (on its way to 0 or infinity, v is there by both or still normal).  Powers of two are exact
// to multiply by, so that the product is rounded once.
__device__ __forceinline__ float times_scales(float v, float a, float b) {
    const bool first = fabsf(a) >= fabsf(b);
    const float most = first ? a : b, least = first ? b : a;
    if (fabsf(most) >= 1.0f && fabsf(least) < 1.0f) return v * (most * least);
    return v * most * least;
}

// Whether a row has no gradient, whatever it holds: by its target, or (there are none: rows have
// lists) by its statistics.
__device__ __forceinline__ bool ignored_row(const int64_t* targets, int64_t ignore_index, const float4* stats,
                                            int64_t row) {
    if (targets) return targets[row] == ignore_index;
    if (!stats) return false;
    const float4 s = stats[row];
    return s.x == -INFINITY && s.y == 0.0f;
}

// Eight 16-bit elements from any element's address, in 4-byte loads: the words that hold
// them, shifted by half a word where they start in the middle of one.  Reads up to one
// element before them and one after, within the words of the first and the last.
__device__ __forceinline__ void load_eight_halves(const uint16_t* p, uint32_t (&w)[4]) {
    const bool odd = (reinterpret_cast<uintptr_t>(p) & 2u) != 0;
    const uint32_t* q = reinterpret_cast<const uint32_t*>(p - (odd ? 1 : 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __ldg(q + i);
    if (odd) {
        const uint32_t last = __ldg(q + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], i < 3 ? w[i + 1] : last, 16);
    }
}

template <typename... Params, typename... Given>
cudaError_t launch_early(void (*kernel)(Params...), int64_t grid, int block, size_t smem,
                         cudaStream_t st, Given&&... given) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(given)...);
}
#endif

// The current device: its SMs, the CTA pairs that run at once on them, the status word that
// its kernels set (pinned host memory), and the limit of their waits.
struct Device {
    int sms, pairs;
    int* status;
    unsigned long long wait_ns;
};
cudaError_t device(Device* d);
int take_status(const Device& d);
// What a call that is about to queue work begins with: PVS_OK, or the pvs_status that it
// returns instead.
int ready(Device* d);

// Tensor map of an operand: boxes of kTileK x box_rows (K contiguous) or
// 64 x kTileK (M / N contiguous).
bool operand_map(CUtensorMap* m, const Matrix& x, bool mn, int box_rows);

// Columns per tile for n columns: the fewest tiles, evenly wide, in the steps of 32
// that a pair's MMA takes.
inline int tile_columns(int64_t n) {
    const int64_t t = (n + kTileN - 1) / kTileN;
    const int64_t w = (n + t - 1) / t;
    return (int)((w + 31) / 32 * 32);
}

// The part pairs of a product of operands in `pa` and `pb` parts, i and j of one pair
// adding up to `levels` at most.
void part_pairs(Args& a, int pa, int pb, int levels = 2);

cudaError_t launch_gemm(int epilogue, Args& a, const Device& dev, cudaStream_t st);

// Pairs where there are more rows than one CTA takes.
inline int ctas_for(int64_t m, const Device& dev) { return m > kTileM && dev.pairs > 0 ? 2 : 1; }

// out = alpha sum_s slots[s], rounded once; with scales of its rows and columns, that times both.
cudaError_t launch_sum_slots(const float* slots, int splits, int64_t slot_stride, int64_t ldslot,
                             int64_t m, int n, const float* alpha, float alpha0, void* out,
                             int64_t ldout, int out_type, const Device& dev, cudaStream_t st,
                             const float* row_scales = nullptr, const float* col_scales = nullptr);

// src [rows x cols] of `dtype` to `parts` 16-bit matrices [rows x ldd] (f16 where
// to_f16, else bf16), rows that `zero_target` ignores (or whose zero_bias is
// -inf) as zeros, every row times row_scale where given.  With only_if, nothing
// happens unless *only_if is set.
struct SplitArgs {
    const void* src;
    int64_t ld, rows;
    int cols, dtype;
    const float* row_scale;
    const int64_t* zero_target;
    int64_t ignore_index;
    const float4* zero_stats;    // without zero_target: of the forward pass
    const float* zero_bias;
    const int* only_if;
    uint16_t* dst;
    int64_t ldd, part_stride;
    int parts, to_f16;
    int per_block, wide;         // set by the launch: rows a block, aligned rows, and
    uint64_t magic;              // n / pieces of a row as n magic / 2^40
};
cudaError_t launch_split(const SplitArgs& a, cudaStream_t st);

// float32 rows in two f16 parts for a product whose rows (or columns) undo a scale: each
// row times a power of two that puts its largest finite magnitude at 2^13 .. 2^14,
// rounded twice to 11 bits (what is left is 2^-24 of an element, 2^-39 of the row's
// largest); units gets the powers' inverses.  In the same pass, where given, `parts`
// bf16 parts as launch_split makes them.
struct Split16Args {
    SplitArgs s;                 // s.dst may be null
    uint16_t* dst16;
    int64_t part16_stride;
    float* units;
};

// A row of the backward pass from the forward pass's statistics.
struct RowArgs {
    const float4* stats;
    const float* grad;
    const int64_t* targets;      // null: rows have lists
    int64_t rows, items, ignore_index;
    const float* up;             // f16: the power of two of every gradient, or null
    GradRow* out;                // null: no rows
    int* bad_masked;             // cleared
};

// Up to two copies (of 16-bit operands, or of float32 ones with both kinds of parts) and
// the rows, in one launch.
struct PrepareArgs {
    Split16Args copy[2];         // s.rows 0: none; dst16 null: as launch_split
    int64_t blocks[2];           // set by the launch
    RowArgs rows;
};
cudaError_t launch_prepare(PrepareArgs& a, cudaStream_t st);

// Int8 codes as bf16 (exact), or times their rows' scales in `parts` bf16 parts; in the
// same launch a copy, where s.dst is given.
struct CodesArgs {
    const int8_t* codes;
    int64_t ldc, rows;
    int cols;
    const float* scales;
    uint16_t* dst;
    int64_t ldd, part_stride;
    int parts;
    int per_block, wide;         // set by the launch, as in SplitArgs
    uint64_t magic;
};
cudaError_t launch_codes(CodesArgs c, SplitArgs s, cudaStream_t st);

// A product's tiles; splits and everything else are the caller's.
inline void set_tiles(Problem& p, int64_t m, int64_t n, int bn, int64_t k, int cta) {
    p.m = (int)m;
    p.n = (int)n;
    p.bn = bn;
    p.mtiles = (int)((m + kTileM * cta - 1) / (kTileM * cta));
    p.ntiles = (int)((n + bn - 1) / bn);
    p.kchunks = (int)((k + kTileK - 1) / kTileK);
    p.ktail = (int)((k - (int64_t)(p.kchunks - 1) * kTileK + 15) / 16);
    p.splits = 1;
}

// The splits of k that `want` gives when all but the last are equally long.
inline int even_splits(int64_t kchunks, int64_t want) {
    if (want > kchunks) want = kchunks;
    if (want < 1) want = 1;
    const int64_t len = (kchunks + want - 1) / want;
    return (int)((kchunks + len - 1) / len);
}

// What a unit of `chunks` chunks takes, in the time of a chunk's MMAs: 1.3 times its
// chunks and 7 more (10 where it leaves float32 sums for splits), as dw's tiles of 1, 4 and
// 16 chunks did (64, 256 and 1024 rows over a million items: 8, 10.5 and 27) while lone lanes
// issued the MMAs.  With 1.05 or 1.15 in 1.3's place, nearer to a chunk now, the plans of twelve
// steps of all types took the same times to 2%.
inline double unit_cost(int64_t chunks, bool sums) { return 1.3 * (double)chunks + (sums ? 10 : 7); }
// And for the whole launch: a split tile's store and its later read, and the launch
// that adds the splits.
inline double sums_cost(int64_t tiles, int slots) { return 12.0 * (double)tiles / slots; }
constexpr double kSumsLaunch = 16;

// The splits of k of a product with the launch to itself, u tiles of k chunks, npairs of
// parts, no fewer than `fewest`.
inline int best_splits(int64_t u, int64_t k, int slots, int npairs, int64_t fewest) {
    double least = 1e300;
    int64_t best = 1;
    for (int64_t s = fewest; s <= k && (s == fewest || u * s <= 8 * slots);
         s += s / 8 > 1 ? s / 8 : 1) {
        const double cost = (double)((u * s + slots - 1) / slots) *
                                unit_cost((k + s - 1) / s * npairs, s > 1) +
                            (s > 1 ? sums_cost(u * s, slots) + kSumsLaunch : 0.0);
        if (cost < least) {
            least = cost;
            best = s;
        }
    }
    return even_splits(k, best);
}

// Scratch of one call, carved from the caller's workspace in 256-byte steps.
struct Carver {
    uint8_t* base;
    size_t used = 0;
    template <typename T>
    T* take(int64_t count) {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += ((size_t)count * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Leading dimension of a copied operand: rows start on the 128 bytes that a box reads of
// them (64 for narrow ones).  Rows of 385 elements 784 bytes apart, which start anywhere
// in a sector, took 205 us where these take 177 (200 rows over 100,003 items).
inline int64_t copied_ld(int64_t cols) { return round_up(cols, cols > 256 ? 64 : 32); }
// Rows of any matrix here: coordinates of tiles past the end still fit an int.
constexpr int64_t kMaxRows = 0x7fff0000;
inline int element_bytes(int dtype) { return dtype == 2 ? 4 : 2; }
// Whether a pointer is aligned to its elements (null is).
inline bool on_elements(const void* p, int bytes) {
    return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0;
}
inline int parts_of(int dtype) { return dtype == 2 ? 3 : 1; }

}  // namespace head
}  // namespace pvs

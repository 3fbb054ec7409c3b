// Products of the gated feed-forward block on the tensor cores, 16-bit operands, fp32 sums in tensor memory:
//
//   forward   h = act(x wg^T) * (x wu^T)        a tile of 128 outputs takes both projections, and the epilogue multiplies them
//   input     dx = dg wg + du wu                one sum over both: dg and du lie side by side, the weights' tiles change half way
//   weights   dwg = dg^T x, dwu = du^T x        a tile of either
//
// Pairs of CTAs (cta_group::2) work on tiles of 256 rows x 256 columns: each CTA copies its 128 rows of A and 128 of the 256 rows of B, 32 KB
// per 64 of the summed dimension, for 512 cycles of MMAs.  Forward operands have the summed dimension innermost (K-major); where it is the
// outer one (wg and wu for dx; dg, du and x for dwg, dwu) the MMAs read the tiles as they lie, transposed (MN-major), so nothing is ever
// transposed in memory.  Persistent: warp 0 copies, warp 1 of the pair's first CTA multiplies, warps 4 to 11 drain one accumulator (two, of
// 256 columns each, fill tensor memory) while the other one is summed.
// Forward of up to 128 rows: another kernel streams the weights, which are then the M operand (see there).
// Few tiles: the summed dimension is cut into ranges whose partial sums go to memory, and a second kernel adds them in the ranges' order.
#include <algorithm>

#include "feed_forward.hpp"
#include "linear_device.cuh"

namespace patdnn {
namespace {

constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr int kMostStages = 6;
constexpr int kHalf = 128 * 128;                       // bytes of one CTA's part of an operand in a stage: 128 rows x 64 columns
constexpr int kStage = 2 * kHalf;
constexpr int kPiece = 64;                             // bytes of a row that the epilogue stores at a time
constexpr int kStaging = 32 * kPiece;                  // shared memory of an epilogue warp
constexpr int kSmem = 226 * 1024;                      // all of an SM's: a pair holds all of two SMs' tensor memory (see plan_mx4_linear)

struct GatedParams {
    void *out0, *out1, *gu;                            // h, nullptr | dx, nullptr | dwg, dwu
    int64_t rows, ld;                                  // rows of the output (of either); its stride
    int cols;                                          // columns of the output
    int m_tiles, n_tiles, k_blocks, splits, per_split, stages;
    int f_blocks;                                      // input: blocks of 64 of the gate's part; weights: 256-row tiles of it
    int f_padded;                                      // columns from dg to du
    int box_rows;                                      // rows of A that a CTA copies: fewer than 128 where the product has fewer (K-major A)
    float *partial;
    int *status;
    uint32_t spin_limit;
    int test_skip_load;
};

__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
// An operand part of 128 x 64 elements.  K-major: 128 rows of 128 bytes, groups of 8 rows 1024 bytes apart, K = 16 is 32 bytes further on.
// MN-major: two chunks of 64 columns, 64 rows (the summed dimension) of 128 bytes each, 8192 bytes apart; K = 16 is 16 rows further on.
template <bool KMAJOR> __device__ __forceinline__ uint64_t part_desc(uint32_t addr) {
    constexpr uint64_t leading = KMAJOR ? 1 : 8192 >> 4;
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (leading << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
template <bool KMAJOR> constexpr uint64_t kNextK = KMAJOR ? 2 : 2048 >> 4;

// Partial sums of a unit: a piece per epilogue warp of either CTA, [chunk of 32 columns][column][row].
__device__ __forceinline__ float *part_of(float *partial, int64_t unit, uint32_t rank, int e) {
    return partial + unit * kGatedUnitFloats + (static_cast<int>(rank) * kEpilogueWarps + e) * (kGatedUnitFloats / (2 * kEpilogueWarps));
}

template <int MODE, typename T, int ACT>
__global__ void __launch_bounds__(kThreads, 1)
gated_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b0, const __grid_constant__ CUtensorMap map_b1, const GatedParams p) {
    constexpr bool A_K = MODE != kGatedWeights, B_K = MODE == kGatedForward;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kMostStages + 4];
    __shared__ uint32_t tmem_slot;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cta_rank();
    const WaitCtx ctx{p.status, p.spin_limit ? p.spin_limit : kSpinLimit};
    const uint32_t smem = (smem_u32(smem_raw) + 1023) & ~1023u;
    // full: in the first CTA, which expects the bytes of both (the second one's may come first: a phase ends with the arrival); empty, done: one per CTA, told by the first CTA's MMAs; drained: in the first CTA
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMostStages, done = empty + 8 * kMostStages, drained = done + 16;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(done + 8 * b, 1);
            mbar_init(drained + 8 * b, 2 * kEpilogueWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_allocate_pair(&tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    pair_barrier();                                    // both CTAs' barriers exist, and their tensor memory
    tc_fence_after();
    pdl_trigger();                                     // not before the allocation: see kernels.hpp
    const uint32_t tmem = tmem_slot;
    pdl_wait();

    const int units = p.m_tiles * p.n_tiles * p.splits, first = blockIdx.x >> 1, step = gridDim.x >> 1;
    if (warp == 0) {
        const bool leader = elect_one();
        const uint32_t full0 = in_cta(full, 0);
        // Rows that do not exist are not copied where they are all of a CTA's, or where the product has fewer rows than a tile: the MMAs read whatever is
        // there and give rows that nobody stores.  (Filling 127 of 128 rows with zeros took the copies twice the time of 128 rows: one row,
        // 1536 -> 8192, 17.7 us against 14.4 us for 128 rows.)
        const uint32_t a_bytes = p.box_rows * 128, expected = 2 * kHalf + (A_K && p.rows <= 128 ? 1 : 2) * a_bytes;
        const bool has_rows = !A_K || rank == 0 || p.rows > 128;
        int slot = 0, issued = 0;
        uint32_t phase = 1;                            // (the first pass over the ring does not wait)
        bool ok = true;
        for (int u = first; ok && u < units; u += step) {
            const int tile = u / p.splits, k0 = (u - tile * p.splits) * p.per_split, k1 = min(p.k_blocks, k0 + p.per_split);
            const int nt = tile / p.m_tiles, mt = tile - nt * p.m_tiles;
            for (int k = k0; k < k1; ++k) {
                if (issued >= p.stages && !warp_wait(empty + 8 * slot, phase, ctx, 121)) { ok = false; break; }
                if (leader && issued + 1 != p.test_skip_load) {
                    const uint32_t bar = full0 + 8 * slot, a = smem + slot * kStage, b = a + kHalf;
                    if (rank == 0) mbar_expect_tx(full + 8 * slot, expected);
                    if constexpr (MODE == kGatedForward) {             // this CTA: 128 rows of x, and the gate's or the up projection's weights
                        if (has_rows) tile_load(a, &map_a, bar, k * 64, mt * 256 + rank * 128);
                        tile_load(b, rank == 0 ? &map_b0 : &map_b1, bar, k * 64, nt * 128);
                    } else if constexpr (MODE == kGatedInput) {
                        const bool up = k >= p.f_blocks;
                        const CUtensorMap *map = up ? &map_b1 : &map_b0;
                        const int f = (up ? k - p.f_blocks : k) * 64, n = nt * 256 + rank * 128;
                        if (has_rows) tile_load(a, &map_a, bar, k * 64, mt * 256 + rank * 128);
                        tile_load(b, map, bar, n, f);
                        tile_load(b + kHalf / 2, map, bar, n + 64, f);
                    } else {
                        const int up = mt >= p.f_blocks;
                        const int f = up * p.f_padded + (mt - up * p.f_blocks) * 256 + rank * 128, n = nt * 256 + rank * 128;
                        tile_load(a, &map_a, bar, f, k * 64);
                        tile_load(a + kHalf / 2, &map_a, bar, f + 64, k * 64);
                        tile_load(b, &map_b0, bar, n, k * 64);
                        tile_load(b + kHalf / 2, &map_b0, bar, n + 64, k * 64);
                    }
                }
                ++issued;
                if (++slot == p.stages) { slot = 0; phase ^= 1; }
            }
        }
        // no copy of either CTA may still be in flight when the pair ends, whatever happened to the other roles
        if (rank == 0)
            for (int i = max(0, issued - p.stages); i < issued; ++i) mbar_wait(full + 8 * (i % p.stages), (i / p.stages) & 1, ctx, 122);
    } else if (warp == 1 && rank == 0) {
        const bool leader = elect_one();
        constexpr uint32_t idesc = (1u << 4) | (std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u) | (A_K ? 0u : 1u << 15) |
                                   (B_K ? 0u : 1u << 16) | (uint32_t(256 >> 3) << 17) | (uint32_t(256 >> 4) << 24);
        const uint32_t peer_empty = in_cta(empty, 1), peer_done = in_cta(done, 1), own_empty = in_cta(empty, 0), own_done = in_cta(done, 0);
        const uint64_t da0 = part_desc<A_K>(smem), db0 = part_desc<B_K>(smem + kHalf);
        int slot = 0, t = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int u = first; ok && u < units; u += step, ++t) {
            const int split = u % p.splits, k0 = split * p.per_split, k1 = min(p.k_blocks, k0 + p.per_split);
            const int buf = t & 1;
            if (t > 1 && !warp_wait(drained + 8 * buf, ((t >> 1) - 1) & 1, ctx, 123)) break;
            tc_fence_after();
            uint32_t accumulate = 0;
            for (int k = k0; k < k1; ++k) {
                if (!warp_wait(full + 8 * slot, phase, ctx, 124)) { ok = false; break; }
                tc_fence_after();
                if (leader) {
                    const uint64_t shift = static_cast<uint64_t>(slot) * (kStage >> 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mma_pair(tmem + buf * 256, da0 + shift + j * kNextK<A_K>, db0 + shift + j * kNextK<B_K>, idesc, accumulate | j);
                    commit_pair(own_empty + 8 * slot);
                    commit_pair(peer_empty + 8 * slot);
                }
                __syncwarp();
                accumulate = 1;
                if (++slot == p.stages) { slot = 0; phase ^= 1; }
            }
            if (leader && ok) {
                commit_pair(own_done + 8 * buf);
                commit_pair(peer_done + 8 * buf);
            }
            __syncwarp();
        }
        // no MMA may still run when tensor memory is freed
        const int last = t - 1;
        if (leader && !ok) commit_pair(own_done + 8 * (last & 1));
        __syncwarp();
        if (last >= 0) mbar_wait(done + 8 * (last & 1), (last >> 1) & 1, ctx, 125);
    } else if (warp >= 4) {
        const int e = warp - 4, quadrant = e & 3, half = e >> 2;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quadrant * 32) << 16);
        const uint32_t drained0 = in_cta(drained, 0);
        unsigned char *stage = smem_raw + (smem - smem_u32(smem_raw)) + p.stages * kStage + e * kStaging;
        int t = 0;
        for (int u = first; u < units; u += step, ++t) {
            const int tile = u / p.splits, buf = t & 1;
            const int nt = tile / p.m_tiles;
            int mt = tile - nt * p.m_tiles;
            if (!mbar_wait(done + 8 * buf, (t >> 1) & 1, ctx, 126)) break;
            tc_fence_after();
            T *out = static_cast<T *>(p.out0);
            if constexpr (MODE == kGatedWeights) {
                if (mt >= p.f_blocks) {
                    mt -= p.f_blocks;
                    out = static_cast<T *>(p.out1);
                }
            }
            const int64_t row0 = static_cast<int64_t>(mt) * 256 + rank * 128 + quadrant * 32;
            const int rows_left = static_cast<int>(max(static_cast<int64_t>(-1), min(static_cast<int64_t>(32), p.rows - row0)));
            // chunk j of the warp, 32 columns of the accumulator: forward gate, up, gate, up of its 64 outputs
            auto column = [&](int j) { return MODE == kGatedForward ? (j & 1) * 128 + half * 64 + (j >> 1) * 32 : half * 128 + j * 32; };
            if (p.splits > 1) {
                float *to = part_of(p.partial, u, rank, e) + lane;
                for (int j = 0; j < 4; ++j) {
                    uint32_t v[32];
                    tmem_ld32(lanes + buf * 256 + column(j), v);
                    if (lane < rows_left) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) to[(j * 32 + i) * 32] = __uint_as_float(v[i]);
                    }
                }
            }
            auto fetch = [&](int j, float (&v)[32]) {
                uint32_t w[32];
                tmem_ld32(lanes + buf * 256 + column(j), w);
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(w[i]);
            };
            auto put = [&](const float (&v)[32], T *base, int64_t ld, int col, int left) {
                const uint64_t places = reinterpret_cast<uintptr_t>(base) | static_cast<uint64_t>(ld * sizeof(T));
                const int aligned = places % 16 == 0 ? 16 : places % 4 == 0 ? 4 : 2;
                store_piece<T, kPiece>(v, stage, base + row0 * ld + col, ld, rows_left, left, aligned);
            };
            if (p.splits == 1 && rows_left > 0) {
                if constexpr (MODE == kGatedForward) {
                    for (int c = 0; c < 2; ++c) {
                        const int f = nt * 128 + half * 64 + c * 32;
                        if (f >= p.cols) break;
                        float g[32], up[32];
                        fetch(2 * c, g);
                        fetch(2 * c + 1, up);
                        if (p.gu) {
                            T *gu = static_cast<T *>(p.gu);
                            put(g, gu, 2 * static_cast<int64_t>(p.cols), f, p.cols - f);
                            put(up, gu + p.cols, 2 * static_cast<int64_t>(p.cols), f, p.cols - f);
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) g[i] = activate1<ACT>(g[i]) * up[i];
                        put(g, out, p.ld, f, p.cols - f);
                    }
                } else {
                    for (int j = 0; j < 4; ++j) {
                        const int n = nt * 256 + half * 128 + j * 32;
                        if (n >= p.cols) break;
                        float v[32];
                        fetch(j, v);
                        put(v, out, p.ld, n, p.cols - n);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_pair(drained0 + 8 * buf);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    pair_barrier();                                    // nobody's shared or tensor memory goes away under its peer
    if (warp == 2) tmem_free_pair(tmem, 512);
}

// The sums of a tile's ranges, in their order, and the epilogue.  A warp takes 32 rows and 16 columns (forward: of both projections); the eight
// warps of a CTA are the eight epilogue warps' pieces of one CTA's half of the tile.
template <int MODE, typename T, int ACT>
__global__ void __launch_bounds__(256) gated_join_kernel(const GatedParams p) {
    constexpr int kPieces = MODE == kGatedForward ? 4 : 8, kWide = 16;
    __shared__ __align__(16) unsigned char staging[8][32 * kWide * sizeof(T)];
    pdl_trigger();
    const int e = threadIdx.x >> 5, lane = threadIdx.x & 31, quadrant = e & 3, half = e >> 2;
    const int piece = blockIdx.x % kPieces, rank = blockIdx.x / kPieces & 1, tile = blockIdx.x / (2 * kPieces);
    const int nt = tile / p.m_tiles;
    int mt = tile - nt * p.m_tiles;
    T *out = static_cast<T *>(p.out0);
    if (MODE == kGatedWeights && mt >= p.f_blocks) {
        mt -= p.f_blocks;
        out = static_cast<T *>(p.out1);
    }
    const int64_t row0 = static_cast<int64_t>(mt) * 256 + rank * 128 + quadrant * 32;
    const int rows_left = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(32), p.rows - row0)));
    const int col = MODE == kGatedForward ? nt * 128 + half * 64 + piece * kWide : nt * 256 + half * 128 + piece * kWide, left = p.cols - col;
    if (rows_left == 0 || left <= 0) return;
    pdl_wait();
    auto sum = [&](int chunk, int first, float (&v)[kWide]) {          // columns [first, first + 16) of a chunk
#pragma unroll
        for (int i = 0; i < kWide; ++i) v[i] = 0.f;
        if (lane >= rows_left) return;
        const float *from = part_of(p.partial, static_cast<int64_t>(tile) * p.splits, rank, e) + (chunk * 32 + first) * 32 + lane;
#pragma unroll 4
        for (int s = 0; s < p.splits; ++s, from += kGatedUnitFloats) {
#pragma unroll
            for (int i = 0; i < kWide; ++i) v[i] += from[i * 32];
        }
    };
    auto put = [&](const float (&v)[kWide], T *base, int64_t ld) {
        const uint64_t places = reinterpret_cast<uintptr_t>(base) | static_cast<uint64_t>(ld * sizeof(T));
        const int aligned = places % 16 == 0 ? 16 : places % 4 == 0 ? 4 : 2;
        store_piece<T, kWide * sizeof(T)>(v, staging[e], base + row0 * ld + col, ld, rows_left, left, aligned);
    };
    float v[kWide];
    if constexpr (MODE == kGatedForward) {
        float up[kWide];
        sum(piece >> 1 << 1, (piece & 1) * kWide, v);
        sum((piece >> 1 << 1) + 1, (piece & 1) * kWide, up);
        if (p.gu) {
            T *gu = static_cast<T *>(p.gu);
            put(v, gu, 2 * static_cast<int64_t>(p.cols));
            put(up, gu + p.cols, 2 * static_cast<int64_t>(p.cols));
        }
#pragma unroll
        for (int i = 0; i < kWide; ++i) v[i] = activate1<ACT>(v[i]) * up[i];
    } else {
        sum(piece >> 1, (piece & 1) * kWide, v);
    }
    put(v, out, p.ld);
}

// ---- forward, few rows -----------------------------------------------------------------------------------------------------
// The weights are the M operand, 64 rows of wg and the same 64 of wu in a tile, the rows of x the N operand (16 to 128): a CTA per 64 outputs and
// range of the summed dimension, whose weights it streams.  The CTAs of a cluster share a tile; their partial sums are pushed into the shared
// memory of the one that finishes a row of x, where g and u of an output meet.
constexpr int kRowsThreads = 256;
constexpr int kMostRowsStages = 12;

struct GatedRowsParams {
    void *h, *gu;
    int64_t ldh;
    int rows, F, k_blocks, per_split, splits, stages, tile_n, tensor_columns;
    int *status;
    uint32_t spin_limit;
    int test_skip_load;
};

__device__ __forceinline__ void tile_load_own(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kRowsThreads, 1)
gated_rows_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_g, const __grid_constant__ CUtensorMap map_u, const GatedRowsParams p) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kMostRowsStages + 1];
    __shared__ uint32_t tmem_slot;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = blockIdx.x % p.splits, f0 = blockIdx.x / p.splits * 64;
    const WaitCtx ctx{p.status, p.spin_limit ? p.spin_limit : kSpinLimit};
    const uint32_t smem = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMostRowsStages, done = empty + 8 * kMostRowsStages;
    const uint32_t stage_bytes = kHalf + p.tile_n * 128;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        mbar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_allocate(&tmem_slot, p.tensor_columns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();                                     // not before the allocation: see kernels.hpp
    const uint32_t tmem = tmem_slot;
    pdl_wait();

    const int k0 = rank * p.per_split, k1 = min(p.k_blocks, k0 + p.per_split);
    if (warp == 0) {
        const bool leader = elect_one();
        int slot = 0, issued = 0;
        uint32_t phase = 1;                            // (the first pass over the ring does not wait)
        for (int k = k0; k < k1; ++k) {
            if (issued >= p.stages && !warp_wait(empty + 8 * slot, phase, ctx, 141)) break;
            if (leader && issued + 1 != p.test_skip_load) {
                const uint32_t at = smem + slot * stage_bytes, bar = full + 8 * slot;
                mbar_expect_tx(bar, kHalf + p.rows * 128);             // (rows that do not exist are whatever is there: their sums are not read)
                tile_load_own(at, &map_g, bar, k * 64, f0);
                tile_load_own(at + kHalf / 2, &map_u, bar, k * 64, f0);
                tile_load_own(at + kHalf, &map_x, bar, k * 64, 0);
            }
            ++issued;
            if (++slot == p.stages) { slot = 0; phase ^= 1; }
        }
        // no copy may still be in flight when the CTA ends, whatever happened to the other roles
        for (int i = max(0, issued - p.stages); i < issued; ++i) mbar_wait(full + 8 * (i % p.stages), (i / p.stages) & 1, ctx, 142);
    } else if (warp == 1) {
        const bool leader = elect_one();
        const uint32_t idesc = instr_desc(std::is_same<T, __nv_bfloat16>::value ? 1 : 0, p.tile_n);
        const uint64_t da0 = smem_desc_sw128(smem), db0 = smem_desc_sw128(smem + kHalf);
        int slot = 0;
        uint32_t phase = 0, accumulate = 0;
        for (int k = k0; k < k1; ++k) {
            if (!warp_wait(full + 8 * slot, phase, ctx, 143)) break;
            tc_fence_after();
            if (leader) {
                const uint64_t shift = static_cast<uint64_t>(slot) * (stage_bytes >> 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) umma_f16(tmem, da0 + shift + 2 * j, db0 + shift + 2 * j, idesc, accumulate | j);
                umma_commit(empty + 8 * slot);
            }
            __syncwarp();
            accumulate = 1;
            if (++slot == p.stages) { slot = 0; phase ^= 1; }
        }
        if (leader) umma_commit(done);
    }
    __syncwarp();
    const bool ok = mbar_wait(done, 0, ctx, 144);
    tc_fence_after();
    // CTA r of the cluster finishes the rows j with j % splits == r
    const int shift = 31 - __clz(p.splits), owned = (p.tile_n + p.splits - 1) >> shift;          // splits is a power of two
    const int place = (warp & 3) * 32 + lane;
    pair_barrier();                                    // all pipelines of the cluster are idle: their memory can be reused
    const uint32_t slots = smem + (rank * owned * 128 + place) * 4, lanes = tmem + ((warp & 3) * 32u << 16);
    for (int c = (warp >> 2) * 16; c < p.rows; c += 32) {
        uint32_t v[16];
        tmem_ld16(lanes + c, v);
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (c + j < p.rows)
                asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(in_cta(slots + ((c + j) >> shift) * 512, j & (p.splits - 1))), "r"(k1 > k0 ? v[j] : 0u) : "memory");
    }
    pair_barrier();
    const int f = threadIdx.x & 63;
    if (ok && f0 + f < p.F) {
        const float *from = reinterpret_cast<const float *>(smem_raw + (smem - smem_u32(smem_raw))) + f;
        const int mine = (p.rows - rank + p.splits - 1) >> shift;
#pragma unroll 2
        for (int j = threadIdx.x >> 6; j < mine; j += kRowsThreads / 64) {
            float g = 0.f, up = 0.f;
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < p.splits) {
                    g += from[(r * owned + j) * 128];
                    up += from[(r * owned + j) * 128 + 64];
                }
            const int64_t row = (j << shift) + rank;
            if (p.gu) {
                T *gu = static_cast<T *>(p.gu) + row * 2 * p.F + f0 + f;
                gu[0] = from_float<T>(g);
                gu[p.F] = from_float<T>(up);
            }
            static_cast<T *>(p.h)[row * p.ldh + f0 + f] = from_float<T>(activate1<ACT>(g) * up);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) tmem_free(tmem, p.tensor_columns);
}

// A matrix of `rows` rows and `cols` columns, `row` elements apart (a multiple of 8), read in boxes of 64 columns and `box` rows; zeros outside.
cudaError_t make_map(CUtensorMap *map, int dtype, const void *base, int64_t rows, int64_t cols, int64_t row, int box) {
    return encode_map(map, dtype == PATDNN_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, cols, rows, row * 2, 64, box,
                      CU_TENSOR_MAP_SWIZZLE_128B);
}

// f(product, join): the gradients' products have no activation
template <typename F> cudaError_t by_kernel(int mode, int dtype, int act, F f) {
    auto go = [&](auto t) {
        using T = decltype(t);
        if (mode == kGatedInput) return f(gated_kernel<kGatedInput, T, PATDNN_ACT_NONE>, gated_join_kernel<kGatedInput, T, PATDNN_ACT_NONE>);
        if (mode == kGatedWeights) return f(gated_kernel<kGatedWeights, T, PATDNN_ACT_NONE>, gated_join_kernel<kGatedWeights, T, PATDNN_ACT_NONE>);
        return by_act(act, [&](auto a) { return f(gated_kernel<kGatedForward, T, a.value>, gated_join_kernel<kGatedForward, T, a.value>); });
    };
    return dtype == PATDNN_F16 ? go(__half{}) : go(__nv_bfloat16{});
}

template <typename F> cudaError_t by_rows_kernel(int dtype, int act, F f) {
    return by_act(act, [&](auto a) { return dtype == PATDNN_F16 ? f(gated_rows_kernel<__half, a.value>) : f(gated_rows_kernel<__nv_bfloat16, a.value>); });
}

}  // namespace

int units_most() { return std::max(1, sm_count() / 2); }

GatedPlan plan_gated(int F, int K, int64_t rows, int mode) {
    GatedPlan p{};
    if (mode == kGatedForward && rows <= 128) {
        p.few = true;
        p.tile_n = static_cast<int>(ceil_div(rows, 16) * 16);
        p.m_tiles = 1;
        p.n_tiles = static_cast<int>(ceil_div(F, 64));
        p.k_blocks = static_cast<int>(ceil_div(K, 64));
        p.splits = 1;
        while (p.splits < 8 && p.n_tiles * p.splits * 2 <= sm_count() && p.k_blocks >= p.splits * 8) p.splits *= 2;
        p.per_split = static_cast<int>(ceil_div(p.k_blocks, p.splits));
        p.grid = p.n_tiles * p.splits;
        const int stage = kHalf + p.tile_n * 128;
        // more CTAs than SMs: two to an SM
        p.stages = std::max(1, std::min({kMostRowsStages, p.per_split, (p.grid > sm_count() ? 110 * 1024 : 200 * 1024) / stage}));
        p.tensor_columns = allocation_of(p.tile_n);
        const int owned = static_cast<int>(ceil_div(p.tile_n, p.splits));
        // (shared memory in proportion to tensor memory, see plan_mx4_linear)
        p.smem = std::max({p.stages * stage + 1024, p.splits * owned * 512 + 1024, kSmemPerSm / 512 * p.tensor_columns - 1024});
        return p;
    }
    const int64_t m = mode == kGatedWeights ? 2 * ceil_div(F, 256) : ceil_div(rows, 256);
    p.m_tiles = static_cast<int>(m);
    p.n_tiles = static_cast<int>(mode == kGatedForward ? ceil_div(F, 128) : ceil_div(K, 256));
    p.k_blocks = static_cast<int>(mode == kGatedForward ? ceil_div(K, 64) : mode == kGatedInput ? 2 * ceil_div(F, 64) : ceil_div(rows, 64));
    const int64_t tiles = m * p.n_tiles, most = units_most();
    // Tiles for half the pairs of SMs or fewer: ranges of at least four blocks share a tile.
    p.splits = 1;
    if (tiles * 2 <= most) p.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(most / tiles, p.k_blocks / 4)));
    p.per_split = static_cast<int>(ceil_div(p.k_blocks, p.splits));
    p.splits = static_cast<int>(ceil_div(p.k_blocks, p.per_split));
    p.grid = 2 * static_cast<int>(std::min(tiles * p.splits, most));
    p.stages = kMostStages;
    p.smem = kSmem;
    p.tensor_columns = 512;
    return p;
}

cudaError_t prepare_gated() {
    for (int dtype : {PATDNN_F16, PATDNN_BF16})
        for (int mode : {kGatedForward, kGatedInput, kGatedWeights})
            for (int act : {PATDNN_ACT_NONE, PATDNN_ACT_RELU, PATDNN_ACT_SILU}) {
                const cudaError_t e = by_kernel(mode, dtype, act, [](auto kernel, auto) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); });
                if (e != cudaSuccess) return e;
                const cudaError_t r = by_rows_kernel(dtype, act, [](auto kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); });
                if (r != cudaSuccess) return r;
            }
    return cudaSuccess;
}

cudaError_t launch_gated(const GatedShape &s, const GatedCall &c, const GatedWork &w, int mode, cudaStream_t st, int *launches) {
    const GatedPlan plan = plan_gated(s.F, s.K, c.rows, mode);
    const int padded = gated_padded(s.F);
    CUtensorMap a, b0, b1;
    cudaError_t e;
    *launches = plan.splits > 1 && !plan.few ? 2 : 1;
    if (plan.few) {
        GatedRowsParams p{};
        p.h = c.h; p.gu = c.gu; p.ldh = s.h_row; p.rows = static_cast<int>(c.rows); p.F = s.F;
        p.k_blocks = plan.k_blocks; p.per_split = plan.per_split; p.splits = plan.splits; p.stages = plan.stages; p.tile_n = plan.tile_n;
        p.tensor_columns = plan.tensor_columns; p.status = w.status; p.spin_limit = c.spin_limit; p.test_skip_load = c.test_skip_load;
        e = make_map(&a, s.dtype, c.x, c.rows, s.K, c.x_row, p.rows);
        if (e == cudaSuccess) e = make_map(&b0, s.dtype, c.wg, s.F, s.K, c.w_row, 64);
        if (e == cudaSuccess) e = make_map(&b1, s.dtype, c.wu, s.F, s.K, c.w_row, 64);
        if (e != cudaSuccess) return e;
        return by_rows_kernel(s.dtype, s.act, [&](auto kernel) { return launch_pdl(kernel, dim3(plan.grid), dim3(kRowsThreads), plan.smem, st, plan.splits, a, b0, b1, p); });
    }
    GatedParams p{};
    p.m_tiles = plan.m_tiles; p.n_tiles = plan.n_tiles; p.k_blocks = plan.k_blocks; p.splits = plan.splits; p.per_split = plan.per_split; p.stages = plan.stages;
    p.partial = w.partial; p.status = w.status; p.spin_limit = c.spin_limit; p.test_skip_load = c.test_skip_load;
    p.box_rows = mode == kGatedWeights ? 128 : static_cast<int>(std::min<int64_t>(128, c.rows));
    if (mode == kGatedForward) {
        p.out0 = c.h; p.gu = c.gu; p.rows = c.rows; p.ld = s.h_row; p.cols = s.F;
        e = make_map(&a, s.dtype, c.x, c.rows, s.K, c.x_row, p.box_rows);
        if (e == cudaSuccess) e = make_map(&b0, s.dtype, c.wg, s.F, s.K, c.w_row, 128);
        if (e == cudaSuccess) e = make_map(&b1, s.dtype, c.wu, s.F, s.K, c.w_row, 128);
    } else if (mode == kGatedInput) {
        p.out0 = c.dx; p.rows = c.rows; p.ld = s.x_row; p.cols = s.K; p.f_blocks = padded / 64;
        e = make_map(&a, s.dtype, w.dgu, c.rows, 2 * static_cast<int64_t>(padded), 2 * static_cast<int64_t>(padded), p.box_rows);
        if (e == cudaSuccess) e = make_map(&b0, s.dtype, c.wg, s.F, s.K, c.w_row, 64);
        if (e == cudaSuccess) e = make_map(&b1, s.dtype, c.wu, s.F, s.K, c.w_row, 64);
    } else {
        p.out0 = c.dwg; p.out1 = c.dwu; p.rows = s.F; p.ld = s.w_row; p.cols = s.K; p.f_blocks = plan.m_tiles / 2; p.f_padded = padded;
        e = make_map(&a, s.dtype, w.dgu, c.rows, 2 * static_cast<int64_t>(padded), 2 * static_cast<int64_t>(padded), 64);
        if (e == cudaSuccess) e = make_map(&b0, s.dtype, c.x, c.rows, s.K, c.x_row, 64);
        b1 = b0;
    }
    if (e != cudaSuccess) return e;
    return by_kernel(mode, s.dtype, s.act, [&](auto product, auto join) {
        const cudaError_t r = launch_pdl(product, dim3(plan.grid), dim3(kThreads), plan.smem, st, 2, a, b0, b1, p);
        if (r != cudaSuccess || plan.splits == 1) return r;
        return launch_pdl(join, dim3(plan.m_tiles * plan.n_tiles * (mode == kGatedForward ? 8 : 16)), dim3(256), 0, st, 1, p);
    });
}

}  // namespace patdnn

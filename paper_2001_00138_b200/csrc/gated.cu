// Products of the gated feed-forward block on the tensor cores, 16-bit operands, fp32 sums in tensor memory:
//
//   forward   h = act(x wg^T) * (x wu^T)        a tile of 128 outputs takes both projections, and the epilogue multiplies them
//   input     dx = dg wg + du wu                one sum over both: dg and du lie side by side, the weights' tiles change half way
//   weights   dwg = dg^T x, dwu = du^T x        a tile of either
//
// Pairs of CTAs (cta_group::2) work on tiles of 256 rows x 256 columns: each CTA copies its 128 rows of A and 128 of the 256 rows of B, 32 KB
// per 64 of the summed dimension, for 512 cycles of MMAs.  Forward operands have the summed dimension innermost (K-major); where it is the
// outer one (wg and wu for dx; dg, du and x for dwg, dwu) the MMAs read the tiles as they lie, transposed (MN-major), so nothing is ever
// transposed in memory.  Persistent: warp 0 copies, warp 1 of the pair's first CTA multiplies, warps 4 to 19 drain one accumulator (two, of
// 256 columns each, fill tensor memory) while the other one is summed.
// Forward of few rows: another kernel, whose M operand are the weights (see there).
// Both products of the gradient are one launch, the tiles of the second filling up what the first leaves of the rounds over the SMs.  Few
// tiles: the summed dimension is cut into ranges whose partial sums go to memory, and a second kernel adds them in the ranges' order.
#include <algorithm>

#include "feed_forward.hpp"
#include "linear_device.cuh"

namespace patdnn {
namespace {

constexpr int kThreads = 640;
constexpr int kEpilogueWarps = 16;
constexpr int kMostStages = 6;
constexpr int kMostPairs = 128;
constexpr int kHalf = 128 * 128;                       // bytes of one CTA's part of an operand in a stage: 128 rows x 64 columns
constexpr int kStage = 2 * kHalf;
constexpr int kPiece = 64;                             // bytes of a row that the epilogue stores at a time
constexpr int kStaging = 32 * kPiece;                  // shared memory of an epilogue warp
constexpr int kSmem = 226 * 1024;                      // all of an SM's: a pair holds all of two SMs' tensor memory (see plan_mx4_linear)

struct Product {
    void *out0, *out1;                                 // h, nullptr | dx, nullptr | dwg, dwu
    int64_t rows, ld;                                  // rows of the output (of either); its stride
    int cols;                                          // columns of the output
    int m_tiles, n_tiles, k_blocks, splits, per_split;
    int f_blocks;                                      // input: blocks of 64 of the gate's part; weights: 256-row tiles of it
    int box_rows;                                      // rows of A that a CTA copies: fewer than 128 where a K-major product has fewer
    int units;                                         // tiles times splits
    int slot;                                          // of its first unit among the partial sums
    int band;                                          // tiles of rows to a band
    const float *unscale;                              // half, gradient: of a row of the output; weights: those of the up projection are f_padded further on
};
// Pair q of P takes the units q, q + P, ... of the first product, then of the second those from more[q] to more[q + 1], which even the pairs out, and
// the units more[P] + q, more[P] + q + P, ..., `common` of them: what runs at a time lies together, as the bands of tiles want it.
struct GatedParams {
    Product of[2];
    void *gu;                                          // forward: both projections, or nullptr
    int stages;
    int f_padded;                                      // columns from dg to du
    uint32_t *row_top, *column_top;                    // half, gradient: what is cleared for the next call, a word per row of x and 2 f_padded
    int64_t top_rows;
    float *partial;
    int *status;
    uint32_t spin_limit;
    int test_skip_load;
    int common;
    int more[kMostPairs + 1];
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

// Partial sums of a unit: a piece per epilogue warp of either CTA, [64 columns][32 rows].
__device__ __forceinline__ float *part_of(float *partial, int64_t unit, uint32_t rank, int e) {
    return partial + unit * kGatedUnitFloats + (static_cast<int>(rank) * kEpilogueWarps + e) * (kGatedUnitFloats / (2 * kEpilogueWarps));
}

struct GatedMaps {
    CUtensorMap a, b0, b1;                             // forward x, wg, wu; input dgu, wg, wu
    CUtensorMap wa, wb;                                // weights dgu, x
};

// The i-th unit of pair q: its number, -1 behind the last.
__device__ __forceinline__ int unit_of(const GatedParams &p, int q, int pairs, int i, int &which) {
    const int u = q + i * pairs, units = p.of[0].units;
    which = 0;
    if (u < units) return u;
    which = 1;
    const int later = i - (q < units ? (units - q + pairs - 1) / pairs : 0), v = p.more[q] + later, round = v - p.more[q + 1];
    return round < 0 ? v : round < p.common ? p.more[pairs] + round * pairs + q : -1;
}

// One warp: 64 columns of 32 rows of 16-bit values, 128 bytes each, from registers to rows, 16 rows at a time through `stage`.  Rows that do not begin at a
// multiple of 16 bytes: seven whole 16-byte units of a row, put together from neighbours, and the eight elements around them one by one, a lane each
// (1 x 7371 -> 1577, rows of odd length: 57 us, an element per lane 76; 213 x 5900 -> 4829: 139 us, four bytes per lane 151).
template <typename T, bool ALIGNED>
__device__ __forceinline__ void store_lines(const float (&v)[2][32], unsigned char *stage, T *y, int64_t ldy, int rows_left) {
    const int lane = threadIdx.x & 31;
    uint32_t w[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const float lo = v[j >> 4][(2 * j) & 31], hi = v[j >> 4][(2 * j + 1) & 31];
        if constexpr (std::is_same<T, __half>::value) {
            const __half2 h = __floats2half2_rn(lo, hi);
            w[j] = *reinterpret_cast<const uint32_t *>(&h);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
            w[j] = *reinterpret_cast<const uint32_t *>(&h);
        }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {             // 16-byte unit u of row r sits at unit u ^ (r & 7)
        __syncwarp();
        if ((lane >> 4) == half) {
#pragma unroll
            for (int u = 0; u < 8; ++u)
                *reinterpret_cast<uint4 *>(stage + (lane & 15) * 128 + ((u ^ (lane & 7)) << 4)) = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 4 + (lane >> 3), u = lane & 7;
            const uint4 t = *reinterpret_cast<const uint4 *>(stage + r * 128 + ((u ^ (r & 7)) << 4));
            unsigned char *row = reinterpret_cast<unsigned char *>(y + (half * 16 + r) * ldy);
            if constexpr (ALIGNED) {
                if (half * 16 + r < rows_left) *reinterpret_cast<uint4 *>(row + u * 16) = t;
            } else {
                const int over = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15), begin = 16 - over;         // of the row's bytes in the unit before
                const uint4 b = *reinterpret_cast<const uint4 *>(stage + r * 128 + ((((u + 7) & 7) ^ (r & 7)) << 4));
                uint32_t w[8] = {b.x, b.y, b.z, b.w, t.x, t.y, t.z, t.w};
                if (begin & 16) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] = w[k + 4];
                }
                if (begin & 8) {
#pragma unroll
                    for (int k = 0; k < 6; ++k) w[k] = w[k + 2];
                }
                if (begin & 4) {
#pragma unroll
                    for (int k = 0; k < 5; ++k) w[k] = w[k + 1];
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], (begin & 2) * 8);
                // the element of this lane: one of the last over / 2, or of the first 8 - over / 2
                const int e = u < (over >> 1) ? 64 - (over >> 1) + u : u - (over >> 1);
                const uint16_t edge = *reinterpret_cast<const uint16_t *>(stage + r * 128 + (((e >> 3) ^ (r & 7)) << 4) + (e & 7) * 2);
                if (half * 16 + r < rows_left) {
                    if (u > 0) *reinterpret_cast<uint4 *>(row - over + u * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                    reinterpret_cast<uint16_t *>(row)[e] = edge;
                }
            }
        }
    }
}

// GRAD: the products are dx and dwg, dwu; else the one is h
template <bool GRAD, typename T, int ACT>
__global__ void __launch_bounds__(kThreads, 1) gated_kernel(const __grid_constant__ GatedMaps maps, const __grid_constant__ GatedParams p) {
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

    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    int which, u;
    if (warp == 0) {
        const bool leader = elect_one();
        const uint32_t full0 = in_cta(full, 0);
        int slot = 0, issued = 0;
        uint32_t phase = 1;                            // (the first pass over the ring does not wait)
        bool ok = true;
        for (int i = 0; ok && (u = unit_of(p, pair, pairs, i, which)) >= 0; ++i) {
            const Product &q = p.of[which];
            const int tile = u / q.splits, k0 = (u - tile * q.splits) * q.per_split, k1 = min(q.k_blocks, k0 + q.per_split);
            int mt, nt;
            banded(tile, q.band, q.m_tiles, q.n_tiles, mt, nt);
            // K-major rows that do not exist are not copied where they are all of a CTA's, or where the product has fewer rows than a tile: the MMAs read
            // whatever is there and give rows that nobody stores.  (Filling 127 of 128 rows with zeros took the copies twice the time of 128 rows.)
            const bool one = !(GRAD && which) && q.rows <= 128, has_rows = !one || rank == 0;
            const uint32_t expected = 2 * kHalf + (one ? 1 : 2) * q.box_rows * 128;
            for (int k = k0; k < k1; ++k) {
                if (issued >= p.stages && !warp_wait(empty + 8 * slot, phase, ctx, 121)) { ok = false; break; }
                if (leader && issued + 1 != p.test_skip_load) {
                    const uint32_t bar = full0 + 8 * slot, a = smem + slot * kStage, b = a + kHalf;
                    if (rank == 0) mbar_expect_tx(full + 8 * slot, expected);
                    if constexpr (!GRAD) {             // this CTA: 128 rows of x, and the gate's or the up projection's weights
                        if (has_rows) tile_load(a, &maps.a, bar, k * 64, mt * 256 + rank * 128);
                        tile_load(b, rank == 0 ? &maps.b0 : &maps.b1, bar, k * 64, nt * 128);
                    } else if (which == 0) {
                        const bool up = k >= q.f_blocks;
                        const CUtensorMap *map = up ? &maps.b1 : &maps.b0;
                        const int f = (up ? k - q.f_blocks : k) * 64, n = nt * 256 + rank * 128;
                        if (has_rows) tile_load(a, &maps.a, bar, k * 64, mt * 256 + rank * 128);
                        tile_load(b, map, bar, n, f);
                        tile_load(b + kHalf / 2, map, bar, n + 64, f);
                    } else {
                        const int up = mt >= q.f_blocks;
                        const int f = up * p.f_padded + (mt - up * q.f_blocks) * 256 + rank * 128, n = nt * 256 + rank * 128;
                        tile_load(a, &maps.wa, bar, f, k * 64);
                        tile_load(a + kHalf / 2, &maps.wa, bar, f + 64, k * 64);
                        tile_load(b, &maps.wb, bar, n, k * 64);
                        tile_load(b + kHalf / 2, &maps.wb, bar, n + 64, k * 64);
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
        constexpr uint32_t common = (1u << 4) | (std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u) | (GRAD ? 1u << 16 : 0u) |
                                    (uint32_t(256 >> 3) << 17) | (uint32_t(256 >> 4) << 24);       // GRAD: B is MN-major
        const uint32_t peer_empty = in_cta(empty, 1), peer_done = in_cta(done, 1), own_empty = in_cta(empty, 0), own_done = in_cta(done, 0);
        const uint64_t db0 = part_desc<!GRAD>(smem + kHalf);
        int slot = 0, t = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (; ok && (u = unit_of(p, pair, pairs, t, which)) >= 0; ++t) {
            const Product &q = p.of[which];
            const int split = u % q.splits, k0 = split * q.per_split, k1 = min(q.k_blocks, k0 + q.per_split);
            const int buf = t & 1;
            const bool turned = GRAD && which == 1;                    // A is MN-major too
            const uint32_t idesc = common | (turned ? 1u << 15 : 0u);
            const uint64_t da0 = turned ? part_desc<false>(smem) : part_desc<true>(smem), next = turned ? kNextK<false> : kNextK<true>;
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
                        mma_pair(tmem + buf * 256, da0 + shift + j * next, db0 + shift + j * kNextK<!GRAD>, idesc, accumulate | j);
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
    } else if (GRAD && std::is_same<T, __half>::value && warp == 3) {
        for (int64_t i = blockIdx.x * 32 + lane; i < p.top_rows + 2 * p.f_padded; i += gridDim.x * 32)
            if (i < p.top_rows) p.row_top[i] = 0;
            else p.column_top[i - p.top_rows] = 0;
    } else if (warp >= 4) {
        const int e = warp - 4, quadrant = e & 3, quarter = e >> 2;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(quadrant * 32) << 16);
        const uint32_t drained0 = in_cta(drained, 0);
        unsigned char *stage = smem_raw + (smem - smem_u32(smem_raw)) + p.stages * kStage + e * kStaging;
        for (int t = 0; (u = unit_of(p, pair, pairs, t, which)) >= 0; ++t) {
            const Product &q = p.of[which];
            const int tile = u / q.splits, buf = t & 1;
            int mt, nt;
            banded(tile, q.band, q.m_tiles, q.n_tiles, mt, nt);
            T *out = static_cast<T *>(q.out0);
            int64_t factors = 0;
            if (GRAD && which == 1 && mt >= q.f_blocks) {
                mt -= q.f_blocks;
                out = static_cast<T *>(q.out1);
                factors = p.f_padded;
            }
            const int64_t row0 = static_cast<int64_t>(mt) * 256 + rank * 128 + quadrant * 32;
            const int rows_left = static_cast<int>(max(static_cast<int64_t>(-1), min(static_cast<int64_t>(32), q.rows - row0)));
            if (!warp_wait(done + 8 * buf, (t >> 1) & 1, ctx, 126)) break;
            tc_fence_after();
            // 64 columns of the accumulator; forward: 32 of the gate's and the same 32 of the up projection's
            float v[2][32];
            const uint32_t from = lanes + buf * 256 + quarter * (GRAD ? 64 : 32);
            tmem_ld32_async(from, reinterpret_cast<uint32_t *>(v[0]));
            tmem_ld32_async(from + (GRAD ? 32 : 128), reinterpret_cast<uint32_t *>(v[1]));
            float factor = 1.f;
            if constexpr (GRAD && std::is_same<T, __half>::value)
                if (lane < rows_left) factor = q.unscale[factors + row0 + lane];
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_pair(drained0 + 8 * buf);
            if constexpr (GRAD && std::is_same<T, __half>::value) {
#pragma unroll
                for (int i = 0; i < 64; i += 2) {      // (in pairs: one by one they spill)
                    const float2 two = split(mul_(pair_of(v[i >> 5][i & 31], v[i >> 5][(i & 31) + 1]), pair_of(factor, factor)));
                    v[i >> 5][i & 31] = two.x;
                    v[i >> 5][(i & 31) + 1] = two.y;
                }
            }
            auto put = [&](const float (&w)[32], T *base, int64_t ld, int col, int left) {
                const uint64_t places = reinterpret_cast<uintptr_t>(base) | static_cast<uint64_t>(ld * sizeof(T));
                const int aligned = places % 16 == 0 ? 16 : places % 4 == 0 ? 4 : 2;
                store_piece<T, kPiece>(w, stage, base + row0 * ld + col, ld, rows_left, left, aligned);
            };
            if (rows_left <= 0) continue;
            if (q.splits > 1) {
                float *to = part_of(p.partial, q.slot + u, rank, e) + lane;
                if (lane < rows_left) {
#pragma unroll
                    for (int i = 0; i < 64; ++i) to[i * 32] = v[i >> 5][i & 31];
                }
            } else if constexpr (!GRAD) {
                const int f = nt * 128 + quarter * 32;
                if (f >= q.cols) continue;
                if (p.gu) {
                    T *gu = static_cast<T *>(p.gu);
                    put(v[0], gu, 2 * static_cast<int64_t>(q.cols), f, q.cols - f);
                    put(v[1], gu + q.cols, 2 * static_cast<int64_t>(q.cols), f, q.cols - f);
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) v[0][i] = activate1<ACT>(v[0][i]) * v[1][i];
                put(v[0], out, q.ld, f, q.cols - f);
            } else {
                const int n = nt * 256 + quarter * 64;
                const uint64_t places = reinterpret_cast<uintptr_t>(out) | static_cast<uint64_t>(q.ld * sizeof(T));
                if (q.cols - n >= 64) {
                    if (places % 16 == 0) store_lines<T, true>(v, stage, out + row0 * q.ld + n, q.ld, rows_left);
                    else store_lines<T, false>(v, stage, out + row0 * q.ld + n, q.ld, rows_left);
                } else {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        if (n + 32 * j < q.cols) put(v[j], out, q.ld, n + 32 * j, q.cols - n - 32 * j);
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    pair_barrier();                                    // nobody's shared or tensor memory goes away under its peer
    if (warp == 2) tmem_free_pair(tmem, 512);
}

// The sums of a tile's ranges, and the epilogue.  A CTA takes 32 rows and 16 columns of an epilogue warp's piece (forward: of both projections); its
// warps share the ranges, w, w + 8, ... to warp w, and the first one adds their sums in order.  (A warp alone waits 0.8 us per range.)
constexpr int kJoinWarps = 8;

template <bool GRAD, typename T, int ACT>
__global__ void __launch_bounds__(kJoinWarps * 32) gated_join_kernel(const __grid_constant__ GatedParams p, int first_ctas) {
    constexpr int kPieces = GRAD ? 4 : 2, kWide = 16, kSums = GRAD ? 1 : 2;
    __shared__ float sums[kJoinWarps][kSums][kWide][32];
    __shared__ __align__(16) unsigned char staging[32 * kWide * sizeof(T)];
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const bool second = GRAD && static_cast<int>(blockIdx.x) >= first_ctas;                      // CTAs of the first product come first
    const int block = blockIdx.x - (second ? first_ctas : 0);
    const Product &q = p.of[second];
    const int piece = block % kPieces, e = block / kPieces % kEpilogueWarps, rank = block / (kEpilogueWarps * kPieces) & 1;
    const int tile = block / (2 * kEpilogueWarps * kPieces), quadrant = e & 3, quarter = e >> 2;
    int mt, nt;
    banded(tile, q.band, q.m_tiles, q.n_tiles, mt, nt);
    T *out = static_cast<T *>(q.out0);
    if (second && mt >= q.f_blocks) {
        mt -= q.f_blocks;
        out = static_cast<T *>(q.out1);
    }
    const int64_t row0 = static_cast<int64_t>(mt) * 256 + rank * 128 + quadrant * 32;
    const int rows_left = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(32), q.rows - row0)));
    const int col = (GRAD ? nt * 256 + quarter * 64 : nt * 128 + quarter * 32) + piece * kWide, left = q.cols - col;
    if (rows_left == 0 || left <= 0) return;
    pdl_wait();
    float v[kSums][kWide] = {};
    if (lane < rows_left) {
        const float *from = part_of(p.partial, q.slot + static_cast<int64_t>(tile) * q.splits + warp, rank, e) + piece * kWide * 32 + lane;
        for (int s = warp; s < q.splits; s += warps, from += static_cast<int64_t>(warps) * kGatedUnitFloats) {
            float a[kSums][kWide];
#pragma unroll
            for (int k = 0; k < kSums; ++k)
#pragma unroll
                for (int i = 0; i < kWide; ++i) a[k][i] = from[(k * 32 + i) * 32];
#pragma unroll
            for (int k = 0; k < kSums; ++k)
#pragma unroll
                for (int i = 0; i < kWide; ++i) v[k][i] += a[k][i];
        }
    }
    if (warp > 0) {
#pragma unroll
        for (int k = 0; k < kSums; ++k)
#pragma unroll
            for (int i = 0; i < kWide; ++i) sums[warp][k][i][lane] = v[k][i];
    }
    __syncthreads();
    if (warp > 0) return;
    for (int w = 1; w < warps; ++w)
#pragma unroll
        for (int k = 0; k < kSums; ++k)
#pragma unroll
            for (int i = 0; i < kWide; ++i) v[k][i] += sums[w][k][i][lane];
    auto put = [&](const float (&w)[kWide], T *base, int64_t ld) {
        const uint64_t places = reinterpret_cast<uintptr_t>(base) | static_cast<uint64_t>(ld * sizeof(T));
        const int aligned = places % 16 == 0 ? 16 : places % 4 == 0 ? 4 : 2;
        store_piece<T, kWide * sizeof(T)>(w, staging, base + row0 * ld + col, ld, rows_left, left, aligned);
    };
    if constexpr (!GRAD) {
        if (p.gu) {
            T *gu = static_cast<T *>(p.gu);
            put(v[0], gu, 2 * static_cast<int64_t>(q.cols));
            put(v[1], gu + q.cols, 2 * static_cast<int64_t>(q.cols));
        }
#pragma unroll
        for (int i = 0; i < kWide; ++i) v[0][i] = activate1<ACT>(v[0][i]) * v[1][i];
    }
    put(v[0], out, q.ld);
}

// ---- forward, few rows -----------------------------------------------------------------------------------------------------
// The weights are the M operand, 64 rows of wg and the same 64 of wu in a tile, the rows of x the N operand (16 to 128 of them): a CTA per 64 outputs,
// 128 rows and range of the summed dimension, whose weights it streams.  The CTAs of a cluster share a tile; their partial sums are pushed into the shared
// memory of the one that finishes a row of x, where g and u of an output meet.
// PHASED: rows of the weights are not whole 16-byte units apart, which tensor maps cannot describe; but of 2, 4 or 8 rows every first, every second and so on are.
// A tile takes 64 rows of one such phase, from the 16-byte unit in which each begins: all of them are `shift` columns further right than they should be,
// and so is the copy of x that the phase is multiplied with.  What lies in front of the rows is zeroed where it has arrived.  (8 x 6899 -> 4222: 25 us;
// packing the weights in front 79; rows that are whole units apart 24.)
constexpr int kRowsThreads = 256;
constexpr int kMostRowsStages = 12;

struct GatedRowsParams {
    void *h, *gu;
    int64_t ldh, rows;
    int F, n_tiles, k_blocks, per_split, splits, stages, tile_n, box_rows, tensor_columns;
    int phases, weight_rows;                           // weight_rows: of the weights' boxes
    uint8_t shift[kMostPhases];
    int *status;
    uint32_t spin_limit;
    int test_skip_load;
};

__device__ __forceinline__ void tile_load_own(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}

template <bool PHASED> struct GatedRowsMaps {
    CUtensorMap x, g[PHASED ? kMostPhases : 1], u[PHASED ? kMostPhases : 1];
};

template <typename T, int ACT, bool PHASED>
__global__ void __launch_bounds__(kRowsThreads, 1)
gated_rows_kernel(const __grid_constant__ GatedRowsMaps<PHASED> maps, const __grid_constant__ GatedRowsParams p) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kMostRowsStages + 1];
    __shared__ uint32_t tmem_slot;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = blockIdx.x % p.splits, tile = blockIdx.x / p.splits, mt = tile / p.n_tiles, ft = tile - mt * p.n_tiles;
    const int phase_of = PHASED ? ft % p.phases : 0, f0 = (PHASED ? ft / p.phases : ft) * 64;   // row f0 of the phase's
    const int64_t row0 = static_cast<int64_t>(mt) * 128;
    const int rows = static_cast<int>(min(static_cast<int64_t>(128), p.rows - row0));
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
                // (rows behind the boxes are whatever is there: their sums are not read)
                mbar_expect_tx(bar, (2 * (PHASED ? p.weight_rows : 64) + p.box_rows) * 128);
                tile_load_own(at, &maps.g[phase_of], bar, k * 64, f0);
                tile_load_own(at + kHalf / 2, &maps.u[phase_of], bar, k * 64, f0);
                tile_load_own(at + kHalf, &maps.x, bar, k * 64, static_cast<int>(row0 + (PHASED ? phase_of * p.rows : 0)));
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
            if (PHASED && k == 0 && p.shift[phase_of]) {               // what lies in front of the 128 rows: whatever it is, it is no part of the sums
                unsigned char *at = smem_raw + (smem - smem_u32(smem_raw)) + slot * stage_bytes;
                for (int r = lane; r < 128; r += 32)
                    for (int e = 0; e < p.shift[phase_of]; ++e) *reinterpret_cast<uint16_t *>(at + r * 128 + ((r & 7) << 4) + 2 * e) = 0;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
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
    const bool ok = warp_wait(done, 0, ctx, 144);
    tc_fence_after();
    // CTA r of the cluster finishes the rows j with j % splits == r
    const int shift = 31 - __clz(p.splits), owned = (p.tile_n + p.splits - 1) >> shift;          // splits is a power of two
    const int place = (warp & 3) * 32 + lane;
    pair_barrier();                                    // all pipelines of the cluster are idle: their memory can be reused
    const uint32_t slots = smem + (rank * owned * 128 + place) * 4, lanes = tmem + ((warp & 3) * 32u << 16);
    for (int c = (warp >> 2) * 16; c < rows; c += 32) {
        uint32_t v[16];
        tmem_ld16(lanes + c, v);
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (c + j < rows)
                asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(in_cta(slots + ((c + j) >> shift) * 512, j & (p.splits - 1))), "r"(k1 > k0 ? v[j] : 0u) : "memory");
    }
    pair_barrier();
    const int f = threadIdx.x & 63, column = PHASED ? (f0 + f) * p.phases + phase_of : f0 + f;
    if (ok && column < p.F) {
        const float *from = reinterpret_cast<const float *>(smem_raw + (smem - smem_u32(smem_raw))) + f;
        const int mine = (rows - rank + p.splits - 1) >> shift;
#pragma unroll 2
        for (int j = threadIdx.x >> 6; j < mine; j += kRowsThreads / 64) {
            float g = 0.f, up = 0.f;
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r < p.splits) {
                    g += from[(r * owned + j) * 128];
                    up += from[(r * owned + j) * 128 + 64];
                }
            const int64_t row = row0 + (j << shift) + rank;
            if (p.gu) {
                T *gu = static_cast<T *>(p.gu) + row * 2 * p.F + column;
                gu[0] = from_float<T>(g);
                gu[p.F] = from_float<T>(up);
            }
            static_cast<T *>(p.h)[row * p.ldh + column] = from_float<T>(activate1<ACT>(g) * up);
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
template <typename F> cudaError_t by_kernel(bool grad, int dtype, int act, F f) {
    auto go = [&](auto t) {
        using T = decltype(t);
        if (grad) return f(gated_kernel<true, T, PATDNN_ACT_NONE>, gated_join_kernel<true, T, PATDNN_ACT_NONE>);
        return by_act(act, [&](auto a) { return f(gated_kernel<false, T, a.value>, gated_join_kernel<false, T, a.value>); });
    };
    return dtype == PATDNN_F16 ? go(__half{}) : go(__nv_bfloat16{});
}
template <bool PHASED, typename F> cudaError_t by_rows_kernel(int dtype, int act, F f) {
    return by_act(act, [&](auto a) {
        return dtype == PATDNN_F16 ? f(gated_rows_kernel<__half, a.value, PHASED>) : f(gated_rows_kernel<__nv_bfloat16, a.value, PHASED>);
    });
}

}  // namespace

int pairs_most() { return std::min(kMostPairs, std::max(1, sm_count() / 2)); }

constexpr int64_t kEpilogueBlocks = 6;
// Cuts the summed dimension into `splits` ranges or a few less, none of them empty.
static void cut(GatedPlan &p, int64_t splits) {
    p.per_split = static_cast<int>(ceil_div(p.k_blocks, std::max<int64_t>(1, splits)));
    p.splits = static_cast<int>(ceil_div(p.k_blocks, p.per_split));
}
// A unit's time in blocks: short ones wait for the epilogue of the one before.
static int64_t time_of(const GatedPlan &p) { return std::max<int64_t>(p.per_split, kEpilogueBlocks); }
static int64_t units_of(const GatedPlan &p) { return static_cast<int64_t>(p.m_tiles) * p.n_tiles * p.splits; }
constexpr int64_t kJoinBlocks = 20;                    // what partial sums cost, their stores and the join, in blocks of a tile (6 us, measured)

static GatedPlan plan_few(int f_tiles, int k_blocks, int64_t rows) {
    GatedPlan p{};
    p.few = true;
    p.k_blocks = k_blocks;
    p.tile_n = rows < 128 ? static_cast<int>(ceil_div(rows, 16) * 16) : 128;
    p.m_tiles = static_cast<int>(ceil_div(rows, 128));
    p.n_tiles = f_tiles;
    const int64_t ctas = static_cast<int64_t>(p.m_tiles) * f_tiles;
    p.splits = 1;
    while (p.splits < 8 && ctas * p.splits * 2 <= cluster_room(sm_count(), p.splits * 2) && k_blocks >= p.splits * 8) p.splits *= 2;
    p.per_split = static_cast<int>(ceil_div(k_blocks, p.splits));
    p.grid = static_cast<int>(ctas * p.splits);
    const int stage = kHalf + p.tile_n * 128;
    // more CTAs than SMs: two to an SM
    p.stages = std::max(1, std::min({kMostRowsStages, p.per_split, (p.grid > sm_count() ? 110 * 1024 : 200 * 1024) / stage}));
    p.tensor_columns = allocation_of(p.tile_n);
    const int owned = static_cast<int>(ceil_div(p.tile_n, p.splits));
    // (shared memory in proportion to tensor memory, see plan_mx4_linear)
    p.smem = std::max({p.stages * stage + 1024, p.splits * owned * 512 + 1024, kSmemPerSm / 512 * p.tensor_columns - 1024});
    return p;
}

GatedPlan plan_gated_phased(int F, int K, int64_t rows, int phases) {
    return plan_few(static_cast<int>(phases * ceil_div(ceil_div(F, phases), 64)), static_cast<int>(ceil_div(K + kMostPhases - 1, 64)), rows);
}

GatedPlan plan_gated_forward(int F, int K, int64_t rows) {
    GatedPlan p{};
    p.k_blocks = static_cast<int>(ceil_div(K, 64));
    p.m_tiles = static_cast<int>(ceil_div(rows, 256));
    p.n_tiles = static_cast<int>(ceil_div(F, 128));
    const int64_t tiles = static_cast<int64_t>(p.m_tiles) * p.n_tiles, pairs = pairs_most();
    // as many ranges as give the shortest longest walk, with no more partial sums than fit
    int64_t best = 1, shortest = ceil_div(tiles, pairs) * p.k_blocks;
    for (int64_t n = 2; n <= p.k_blocks / 4 && tiles * n <= kGatedUnits * pairs; ++n) {
        const int64_t walk = ceil_div(tiles * n, pairs) * ceil_div(p.k_blocks, n) + kJoinBlocks;
        if (walk < shortest) best = n, shortest = walk;
    }
    // Few rows: a block of its tile takes about as long as one of a pair's, which is four times as large.  Launch and fill take about six blocks' time
    // in each round, 14 once for the pairs; the exchange in a cluster four.
    const GatedPlan few = plan_few(static_cast<int>(ceil_div(F, 64)), p.k_blocks, rows);
    if (rows <= 128 || ceil_div(few.grid, sm_count()) * (few.per_split + 6) + (few.splits > 1 ? 4 : 0) < shortest + 14) return few;
    cut(p, best);
    p.grid = 2 * static_cast<int>(std::min(units_of(p), pairs));
    p.stages = kMostStages;
    p.smem = kSmem;
    p.tensor_columns = 512;
    return p;
}

void plan_gated_gradient(int F, int K, int64_t rows, bool dx, bool dw, GatedPlan (&plan)[2]) {
    plan[0] = plan[1] = GatedPlan{};
    const int64_t pairs = pairs_most();
    plan[0].m_tiles = static_cast<int>(ceil_div(rows, 256));
    plan[0].k_blocks = gated_padded(F) / 64 * 2;
    plan[1].m_tiles = static_cast<int>(2 * ceil_div(F, 256));
    plan[1].k_blocks = static_cast<int>(ceil_div(rows, 64));
    int64_t blocks = 0;
    for (int i = 0; i < 2; ++i) {
        plan[i].n_tiles = (i ? dw : dx) ? static_cast<int>(ceil_div(K, 256)) : 0;
        blocks += static_cast<int64_t>(plan[i].m_tiles) * plan[i].n_tiles * plan[i].k_blocks;
    }
    // Ranges of about a pair's share of all blocks, of two shares, or none: the first product's units go round the pairs, the second's fill up.
    const int64_t share = std::max<int64_t>(4, ceil_div(blocks, pairs));
    int64_t shortest = INT64_MAX;
    GatedPlan best[2] = {plan[0], plan[1]};
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) {
            const int64_t longest[4] = {INT32_MAX, share, share + share / 4, 2 * share};
            cut(plan[0], ceil_div(plan[0].k_blocks, longest[a]));
            cut(plan[1], ceil_div(plan[1].k_blocks, longest[b]));
            const int64_t u0 = units_of(plan[0]), u1 = units_of(plan[1]);
            if ((plan[0].splits > 1 ? u0 : 0) + (plan[1].splits > 1 ? u1 : 0) > kGatedUnits * pairs) continue;
            const int64_t even = ceil_div(u0 * time_of(plan[0]) + u1 * time_of(plan[1]), pairs) + (u1 ? time_of(plan[1]) / 2 : 0);
            const int64_t walk = std::max({ceil_div(u0, pairs) * time_of(plan[0]), u1 ? time_of(plan[1]) : 0, even}) +
                                 (plan[0].splits + plan[1].splits > 2 ? kJoinBlocks : 0);
            if (walk < shortest) {
                shortest = walk;
                best[0] = plan[0];
                best[1] = plan[1];
            }
        }
    int64_t units = 0;
    for (int i = 0; i < 2; ++i) {
        plan[i] = best[i];
        units += units_of(plan[i]);
        plan[i].stages = kMostStages;
        plan[i].smem = kSmem;
        plan[i].tensor_columns = 512;
    }
    plan[0].grid = plan[1].grid = 2 * static_cast<int>(std::min(units, pairs));
}

cudaError_t prepare_gated() {
    auto allow = [](auto kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); };
    for (int dtype : {PATDNN_F16, PATDNN_BF16})
        for (int act : {PATDNN_ACT_NONE, PATDNN_ACT_RELU, PATDNN_ACT_SILU}) {
            cudaError_t e = by_kernel(false, dtype, act, [&](auto product, auto) { return allow(product); });
            if (e == cudaSuccess) e = by_kernel(true, dtype, act, [&](auto product, auto) { return allow(product); });
            if (e == cudaSuccess) e = by_rows_kernel<false>(dtype, act, allow);
            if (e == cudaSuccess) e = by_rows_kernel<true>(dtype, act, allow);
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

static Product product_of(const GatedPlan &plan, int slot) {
    Product q{};
    q.m_tiles = plan.m_tiles; q.n_tiles = plan.n_tiles; q.k_blocks = plan.k_blocks; q.splits = plan.splits; q.per_split = plan.per_split;
    q.units = static_cast<int>(units_of(plan));
    q.box_rows = 128;
    q.slot = slot;
    q.band = band_of(plan.m_tiles, plan.n_tiles, static_cast<int64_t>(256) * 64 * 2 * plan.k_blocks);
    return q;
}

static cudaError_t launch_products(const GatedMaps &maps, GatedParams &p, const GatedShape &s, const GatedCall &c, const GatedWork &w, int grid, bool grad,
                                   cudaStream_t st, int *launches) {
    p.stages = kMostStages; p.partial = w.partial; p.status = w.status; p.spin_limit = c.spin_limit; p.test_skip_load = c.test_skip_load;
    int joins[2];
    for (int i = 0; i < 2; ++i) joins[i] = p.of[i].splits > 1 ? p.of[i].m_tiles * p.of[i].n_tiles * 2 * kEpilogueWarps * (grad ? 4 : 2) : 0;
    const int join_warps = std::min(kJoinWarps, std::max(p.of[0].splits, p.of[1].splits));
    *launches = joins[0] + joins[1] > 0 ? 2 : 1;
    return by_kernel(grad, s.dtype, s.act, [&](auto product, auto join) {
        const cudaError_t r = launch_pdl(product, dim3(grid), dim3(kThreads), kSmem, st, 2, maps, p);
        if (r != cudaSuccess || *launches == 1) return r;
        return launch_pdl(join, dim3(joins[0] + joins[1]), dim3(join_warps * 32), 0, st, 1, p, joins[0]);
    });
}

template <bool PHASED>
static cudaError_t launch_rows(const GatedRowsMaps<PHASED> &maps, GatedRowsParams &p, const GatedPlan &plan, const GatedShape &s, const GatedCall &c, const GatedWork &w,
                               cudaStream_t st, int *launches) {
    p.h = c.h; p.gu = c.gu; p.ldh = s.h_row; p.rows = c.rows; p.F = s.F; p.n_tiles = plan.n_tiles; p.box_rows = static_cast<int>(std::min<int64_t>(128, c.rows));
    p.k_blocks = plan.k_blocks; p.per_split = plan.per_split; p.splits = plan.splits; p.stages = plan.stages; p.tile_n = plan.tile_n;
    p.tensor_columns = plan.tensor_columns; p.status = w.status; p.spin_limit = c.spin_limit; p.test_skip_load = c.test_skip_load;
    *launches = 1;
    return by_rows_kernel<PHASED>(s.dtype, s.act, [&](auto kernel) {
        return launch_pdl(kernel, dim3(plan.grid), dim3(kRowsThreads), plan.smem, st, plan.splits, maps, p);
    });
}

static cudaError_t launch_phased(const GatedShape &s, const GatedCall &c, const GatedWork &w, cudaStream_t st, int *launches) {
    const GatedPlan plan = plan_gated_phased(s.F, s.K, c.rows, c.phases);
    GatedRowsMaps<true> maps{};
    GatedRowsParams p{};
    p.phases = c.phases;
    p.weight_rows = static_cast<int>(std::min<int64_t>(64, ceil_div(s.F, c.phases)));
    cudaError_t e = make_map(&maps.x, s.dtype, c.x, c.phases * c.rows, c.x_row, c.x_row, static_cast<int>(std::min<int64_t>(128, c.rows)));
    for (int j = 0; j < c.phases && e == cudaSuccess; ++j) {
        p.shift[j] = static_cast<uint8_t>(gated_shift(c.wg, c.w_row, j));
        const int64_t rows = ceil_div(s.F - j, c.phases), first = j * c.w_row - p.shift[j];      // first: at a multiple of 16 bytes
        e = make_map(&maps.g[j], s.dtype, static_cast<const uint16_t *>(c.wg) + first, rows, s.K + p.shift[j], c.phases * c.w_row, p.weight_rows);
        if (e == cudaSuccess) e = make_map(&maps.u[j], s.dtype, static_cast<const uint16_t *>(c.wu) + first, rows, s.K + p.shift[j], c.phases * c.w_row, p.weight_rows);
    }
    return e != cudaSuccess ? e : launch_rows<true>(maps, p, plan, s, c, w, st, launches);
}

cudaError_t launch_gated_forward(const GatedShape &s, const GatedCall &c, const GatedWork &w, cudaStream_t st, int *launches) {
    if (c.phases) return launch_phased(s, c, w, st, launches);
    const GatedPlan plan = plan_gated_forward(s.F, s.K, c.rows);
    GatedMaps maps{};
    const int box = static_cast<int>(std::min<int64_t>(128, c.rows)), weights = plan.few ? 64 : 128;
    cudaError_t e = make_map(&maps.a, s.dtype, c.x, c.rows, s.K, c.x_row, box);
    if (e == cudaSuccess) e = make_map(&maps.b0, s.dtype, c.wg, s.F, s.K, c.w_row, weights);
    if (e == cudaSuccess) e = make_map(&maps.b1, s.dtype, c.wu, s.F, s.K, c.w_row, weights);
    if (e != cudaSuccess) return e;
    if (plan.few) {
        GatedRowsParams p{};
        return launch_rows<false>({maps.a, {maps.b0}, {maps.b1}}, p, plan, s, c, w, st, launches);
    }
    GatedParams p{};
    p.gu = c.gu;
    Product &q = p.of[0] = product_of(plan, 0);
    q.out0 = c.h; q.rows = c.rows; q.ld = s.h_row; q.cols = s.F;
    return launch_products(maps, p, s, c, w, plan.grid, false, st, launches);
}

cudaError_t launch_gated_gradient(const GatedShape &s, const GatedCall &c, const GatedWork &w, cudaStream_t st, int *launches) {
    GatedPlan plan[2];
    plan_gated_gradient(s.F, s.K, c.rows, c.dx != nullptr, c.dwg != nullptr, plan);
    const int padded = gated_padded(s.F);
    const int64_t dgu_row = 2 * static_cast<int64_t>(padded);
    GatedMaps maps{};
    GatedParams p{};
    p.f_padded = padded; p.row_top = w.row_top; p.column_top = w.column_top; p.top_rows = c.rows;
    Product &x = p.of[0] = product_of(plan[0], 0), &dw = p.of[1] = product_of(plan[1], plan[0].splits > 1 ? x.units : 0);
    cudaError_t e = cudaSuccess;
    if (c.dx) {
        x.unscale = w.row_unscale;
        x.out0 = c.dx; x.rows = c.rows; x.ld = s.x_row; x.cols = s.K; x.f_blocks = padded / 64;
        x.box_rows = static_cast<int>(std::min<int64_t>(128, c.rows));
        e = make_map(&maps.a, s.dtype, w.dgu, c.rows, dgu_row, dgu_row, x.box_rows);
        if (e == cudaSuccess) e = make_map(&maps.b0, s.dtype, c.wg, s.F, s.K, c.w_row, 64);
        if (e == cudaSuccess) e = make_map(&maps.b1, s.dtype, c.wu, s.F, s.K, c.w_row, 64);
    }
    if (c.dwg && e == cudaSuccess) {
        dw.unscale = w.column_unscale;
        dw.out0 = c.dwg; dw.out1 = c.dwu; dw.rows = s.F; dw.ld = s.w_row; dw.cols = s.K; dw.f_blocks = dw.m_tiles / 2;
        e = make_map(&maps.wa, s.dtype, w.by_column ? w.by_column : w.dgu, c.rows, dgu_row, dgu_row, 64);
        if (e == cudaSuccess) e = make_map(&maps.wb, s.dtype, c.x, c.rows, s.K, c.x_row, 64);
    }
    if (e != cudaSuccess) return e;
    // The second product's units go to the pairs that the first one left with the fewest blocks: up to a common level, what remains one by one.
    const int pairs = plan[0].grid / 2;
    const int64_t x_time = time_of(plan[0]), dw_time = time_of(plan[1]);
    const int64_t level = (x.units * x_time + dw.units * dw_time) / pairs;
    int64_t given = 0, load[kMostPairs];
    int order[kMostPairs], count[kMostPairs];
    for (int q = 0; q < pairs; ++q) {
        const int64_t before = (x.units / pairs + (q < x.units % pairs)) * x_time;
        count[q] = static_cast<int>(std::max<int64_t>(0, std::min((level - before) / dw_time, dw.units - given)));
        given += count[q];
        load[q] = before + count[q] * dw_time;
        order[q] = q;
    }
    std::sort(order, order + pairs, [&](int a, int b) { return load[a] != load[b] ? load[a] < load[b] : a < b; });
    for (int i = 0; given < dw.units; ++given, i = i + 1 < pairs ? i + 1 : 0) ++count[order[i]];
    p.common = *std::min_element(count, count + pairs);
    for (int q = 0; q < pairs; ++q) p.more[q + 1] = p.more[q] + count[q] - p.common;
    return launch_products(maps, p, s, c, w, plan[0].grid, true, st, launches);
}

}  // namespace patdnn

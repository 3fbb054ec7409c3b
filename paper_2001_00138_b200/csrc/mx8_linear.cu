// Product of two 8-bit matrices on the block-scaled tensor cores: y = act(x w^T + bias), fp32 accumulation in tensor memory.
//
// Both operands lie in the order the tensor cores read (mx8 layout): a tile of 128 rows and 128 columns is one contiguous bulk copy.  A scale
// belongs to 128 columns and the tensor cores take one per 32, so the four MMAs of a column tile (K = 32 each) are given the same scale byte:
// of the four bytes that a row has in tensor memory (a group of four column tiles) the instruction picks the tile's.  No rescaling of
// accumulators, and scales cost a 128th of the elements.
// Two kernels: for few rows the weights are the M operand and are streamed, their column tiles split over the CTAs of a cluster (1 x 4096 -> 4096:
// 5 us for 17 MB); for many rows pairs of CTAs walk over tiles of 256 rows x 256 outputs (8192 x 4096 -> 4096: 95 us, 2.9 PFLOP/s, tensor pipe 79 %;
// 115 us call after call, at the power cap).
#include "feed_forward.hpp"

#include <algorithm>

#include "linear_device.cuh"
#include "mx8_device.cuh"

namespace patdnn {

namespace {

constexpr int kTileCodes = kMx8Tile;                   // bytes of a tile of 128 rows
constexpr int kLinThreads = 256;
constexpr int kMaxStages = 8;

// fp32 += e4m3 * e4m3 with power-of-two scales; M = 128, K = 32.  `byte`: which of a row's four scale bytes.
__device__ __forceinline__ uint32_t mx8_instr_desc(int n, int byte) {
    return (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) | (1u << 27) | (static_cast<uint32_t>(byte) << 4) | (static_cast<uint32_t>(byte) << 29);
}
__device__ __forceinline__ void umma_mx8(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// One tile of 128 weights rows x tile_n rows of x per CTA; the column tiles cut into `splits` ranges, one CTA of a cluster each.
// kFused: the rows of x are elements of T, at most kFusedRows of them, and warps 2 to 7 quantise them into the ring themselves, a column tile at
// a time each: one launch less.  Otherwise they are 8-bit.
template <typename T, int ACT, bool kFused>
__global__ void __launch_bounds__(kLinThreads, 1) mx8_linear_kernel(Mx8Params p) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 1];
    __shared__ uint32_t tmem_slot;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = blockIdx.x % p.splits, tile = blockIdx.x / p.splits;
    const int ft = tile % p.f_tiles, nt = tile / p.f_tiles;
    const WaitCtx ctx{p.status, p.spin_limit ? p.spin_limit : kSpinLimit};
    const uint32_t smem = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages, done = empty + 8 * kMaxStages;

    const uint32_t b_codes = p.tile_n * 128, stage_bytes = kTileCodes + b_codes + 2 * kMx8Scales;
    const int tmem_cols = p.tensor_columns, sf_base = p.tile_n, sf_cols = 8;     // behind the accumulator: scales per stage

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, kFused ? 2 : 1);                     // the copies, and the warp that wrote the rows of x
            mbar_init(empty + 8 * s, 1);
        }
        mbar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_allocate(&tmem_slot, tmem_cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();                                                       // not before the allocation: see kernels.hpp
    const uint32_t tmem = tmem_slot;

    const int t0 = rank * p.tiles_per_split, t1 = min(p.col_tiles, t0 + p.tiles_per_split);
    const int iters = max(0, t1 - t0);
    const int64_t x_tile0 = static_cast<int64_t>(nt) * p.tile_n / 128;

    if (warp == 0) {
        const bool leader = elect_one();
        const uint32_t bytes = kFused ? kTileCodes + kMx8Scales : kTileCodes + b_codes + 2 * kMx8Scales;
        // (ring slots and phases advance without divisions: the instructions of this warp bound short column tiles)
        const uint8_t *wc = p.w + (static_cast<int64_t>(ft) * p.col_tiles + t0) * kTileCodes;
        const uint8_t *ws = p.w + p.w_scales + static_cast<int64_t>(ft) * p.groups * kMx8Scales;
        const uint8_t *xc = p.x + (x_tile0 * p.col_tiles + t0) * kTileCodes;
        const uint8_t *xs = p.x + p.x_scales + x_tile0 * p.groups * kMx8Scales;
        auto load_w = [&](int i, uint32_t at, uint32_t bar) {
            if (leader && i + 1 != p.test_skip_load) {
                mbar_expect_tx(bar, bytes);
                bulk_load(at, wc, kTileCodes, bar);
                bulk_load(at + kTileCodes + b_codes, ws + ((t0 + i) >> 2) * kMx8Scales, kMx8Scales, bar);
            }
            wc += kTileCodes;
        };
        auto load_x = [&](int i, uint32_t at, uint32_t bar) {
            if (leader && !kFused && i + 1 != p.test_skip_load) {
                bulk_load(at + kTileCodes, xc, b_codes, bar);
                bulk_load(at + kTileCodes + b_codes + kMx8Scales, xs + ((t0 + i) >> 2) * kMx8Scales, kMx8Scales, bar);
            }
            xc += kTileCodes;
        };
        // the weights do not depend on the previous kernel: fill the ring with them before waiting for it
        const int ahead = min(iters, p.stages);
        for (int i = 0; i < ahead; ++i) load_w(i, smem + i * stage_bytes, full + 8 * i);
        pdl_wait();
        for (int i = 0; i < ahead; ++i) load_x(i, smem + i * stage_bytes, full + 8 * i);
        int issued = ahead, slot = 0;
        uint32_t phase = 0;
        for (int i = ahead; i < iters; ++i) {
            if (!warp_wait(empty + 8 * slot, phase, ctx, 101)) break;
            load_w(i, smem + slot * stage_bytes, full + 8 * slot);
            load_x(i, smem + slot * stage_bytes, full + 8 * slot);
            ++issued;
            if (++slot == p.stages) { slot = 0; phase ^= 1; }
        }
        // no copy may still be in flight when the CTA ends, whatever happened to the other roles
        for (int i = max(0, issued - p.stages); i < issued; ++i) mbar_wait(full + 8 * (i % p.stages), (i / p.stages) & 1, ctx, 102);
    } else if (warp == 1) {
        const bool leader = elect_one();
        int slot = 0;
        uint32_t phase = 0, accumulate = 0;
        const uint32_t idesc = mx8_instr_desc(p.tile_n, 0), next_byte = (1u << 4) | (1u << 29);
        const uint64_t da0 = smem_desc_sw128(smem), db0 = smem_desc_sw128(smem + kTileCodes);
        const uint64_t sa0 = scale_desc(smem + kTileCodes + b_codes), sb0 = scale_desc(smem + kTileCodes + b_codes + kMx8Scales);
        pdl_wait();                                                      // the bound of the waits below is for this kernel's copies alone
        for (int i = 0; i < iters; ++i) {
            if (!warp_wait(full + 8 * slot, phase, ctx, 103)) break;
            tc_fence_after();
            const uint64_t shift = static_cast<uint64_t>(slot) * (stage_bytes >> 4);
            const uint32_t sfa = tmem + sf_base + slot * sf_cols, sfb = sfa + 4;
            const uint32_t which = idesc + ((t0 + i) & 3) * next_byte;
            const int steps = p.ksteps - (t0 + i) * 4;                   // K-steps that hold data
            if (leader) {
                copy_scales(sfa, sa0 + shift);
                copy_scales(sfb, sb0 + shift);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k < steps) umma_mx8(tmem, da0 + shift + 2 * k, db0 + shift + 2 * k, which, sfa, sfb, accumulate | k);
                umma_commit(empty + 8 * slot);
            }
            __syncwarp();
            accumulate = 1;
            if (++slot == p.stages) { slot = 0; phase ^= 1; }
        }
        if (leader) umma_commit(done);
    } else if constexpr (kFused) {
        constexpr int kProducers = kLinThreads / 32 - 2;
        const T *x = static_cast<const T *>(p.x_raw);
        const bool vector = (reinterpret_cast<uintptr_t>(x) | static_cast<uint64_t>(p.ldx * sizeof(T))) % (4 * sizeof(T)) == 0;
        const int rows = static_cast<int>(p.rows);
        pdl_wait();
        for (int i = warp - 2; i < iters; i += kProducers) {
            const int slot = i % p.stages, turn = i / p.stages;
            const int64_t c = static_cast<int64_t>(t0 + i) * 128 + lane * 4;
            const int count = static_cast<int>(max(int64_t(0), min(int64_t(4), p.K - c)));
            Pack<T, 4> raw[kFusedRows];
#pragma unroll
            for (int r = 0; r < kFusedRows; ++r) {
                const T *src = x + r * p.ldx + c;
                if (vector && count == 4 && r < rows) {
                    raw[r].load(src);
                } else {
                    T v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = r < rows && e < count ? src[e] : from_float<T>(0.f);
                    raw[r] = narrow<T, 4>(Fv<4>::make([&](int e) { return to_float(v[e]); }));
                }
            }
            if (turn > 0 && !warp_wait(empty + 8 * slot, (turn - 1) & 1, ctx, 105)) break;
            unsigned char *at = smem_raw + (smem - smem_u32(smem_raw)) + slot * stage_bytes + kTileCodes;
#pragma unroll
            for (int r = 0; r < kFusedRows; ++r) {
                if (r >= rows) break;
                const Fv<4> f = widen<T, 4>(raw[r]);
                const float v[4] = {f.get(0), f.get(1), f.get(2), f.get(3)};
                const uint32_t top = __reduce_max_sync(0xffffffffu, magnitude_bits(max_abs(max_abs(v[0], v[1]), max_abs(v[2], v[3]))));
                float inverse;
                const uint32_t byte = scale8_of(top, inverse);
                store_codes<4>(at + mx8_place(r, lane * 4), v, inverse);
                if (lane == 0) at[b_codes + kMx8Scales + mx8_scale_place(r, t0 + i)] = static_cast<uint8_t>(byte);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the tensor cores read them through the asynchronous proxy
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(full + 8 * slot) : "memory");
        }
    }
    __syncwarp();
    pdl_wait();
    const bool ok = warp_wait(done, 0, ctx, 104);
    tc_fence_after();
    const int place = (warp & 3) * 32 + lane, f = ft * 128 + place;      // lanes are outputs: a warp stores 32 consecutive ones of a row
    const float bias = p.bias && f < p.F ? p.bias[f] : 0.f;
    const int64_t row0 = static_cast<int64_t>(nt) * p.tile_n;
    const int rows = static_cast<int>(min(static_cast<int64_t>(p.tile_n), p.rows - row0));
    const uint32_t lanes = tmem + ((warp & 3) * 32u << 16);
    T *const y = static_cast<T *>(p.y) + row0 * p.ldy + f;
    if (p.splits == 1) {
        for (int c = (warp >> 2) * 16; c < rows; c += 32) {
            uint32_t v[16];
            tmem_ld16(lanes + c, v);
            if (ok && f < p.F) {
                T *to = y + c * p.ldy;
#pragma unroll
                for (int j = 0; j < 16; ++j, to += p.ldy)
                    if (c + j < rows) *to = from_float<T>(activate1<ACT>(__uint_as_float(v[j]) + bias));
            }
        }
    } else {
        // every CTA of the cluster finishes the columns j with j % splits == its rank: partial sums are pushed into its shared memory
        // and added in rank order
        const int shift = 31 - __clz(p.splits), owned = (p.tile_n + p.splits - 1) >> shift;      // splits is a power of two
        pair_barrier();                                                  // all pipelines are idle: their memory can be reused
        const uint32_t slots = smem + (rank * owned * 128 + place) * 4;
        for (int c = (warp >> 2) * 16; c < rows; c += 32) {
            uint32_t v[16];
            tmem_ld16(lanes + c, v);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < rows)
                    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(in_cta(slots + ((c + j) >> shift) * 512, j & (p.splits - 1))), "r"(iters ? v[j] : 0u) : "memory");
        }
        pair_barrier();
        if (ok && f < p.F) {
            const float *from = reinterpret_cast<const float *>(smem_raw + (smem - smem_u32(smem_raw))) + place;
            const int mine = (rows - rank + p.splits - 1) >> shift;      // of the owned columns, those that are rows of x
#pragma unroll 4
            for (int j = warp >> 2; j < mine; j += 2) {
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < p.splits) sum += from[(r * owned + j) * 128];
                y[((j << shift) + rank) * p.ldy] = from_float<T>(activate1<ACT>(sum + bias));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) tmem_free(tmem, tmem_cols);
}

// ---- many rows ------------------------------------------------------------------------------------------------------------
// Tiles of 256 rows of x (M) by 256 rows of w (N) for pairs of CTAs (cta_group::2), which walk over them: each copies its 128 rows of x and 128 of
// the 256 rows of w, and all the scales that its MMAs need (its own rows', both halves' of w).  Warp 0 fills a ring of column tiles, warp 1
// of the first CTA issues the MMAs, warps 4 to 19 are the epilogue: they move the finished accumulator to registers, hand tensor memory back,
// and convert and store while the next tile is multiplied.  A lane owns a row of y; pieces of 32 rows pass through shared memory so that they
// are stored as whole sectors.
// The scales of four column tiles come and go to tensor memory with the first of them (for each of them: 9 us of 100 for 8192 x 4096 -> 4096).
// Per column tile a CTA writes 33 KB into shared memory and the MMAs read 32 KB from it in the 512 cycles that they take (tiles of 128 x 256 for
// a single CTA: 51 and 48 KB, more than its 128 bytes per cycle).  The tiles come as tensor-map copies of rows that are swizzled already,
// since only such copies may count on the other CTA's barrier.
constexpr int kRowsThreads = 640;
constexpr int kEpilogueWarps = 16;
constexpr int kPiece = 32;                                               // bytes of a row of y that are stored at a time
constexpr int kPairStages = 6;
constexpr int kPairStage = 2 * kTileCodes + 2048;                        // codes, and three chunks of scales
__device__ __forceinline__ void copy_scales_pair(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void umma_mx8_pair(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
struct Mx8Maps {
    CUtensorMap x, w, x_scales, w_scales;
};

template <typename T, int ACT>
__global__ void __launch_bounds__(kRowsThreads, 1) mx8_pair_kernel(const __grid_constant__ Mx8Maps maps, const Mx8Params p) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kPairStages + 2];
    __shared__ uint32_t tmem_slot;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cta_rank();
    const WaitCtx ctx{p.status, p.spin_limit ? p.spin_limit : kSpinLimit};
    const uint32_t smem = (smem_u32(smem_raw) + 1023) & ~1023u;
    // full: in the first CTA; empty, done: one per CTA, told by the first CTA's MMAs; drained: in the first CTA, by the epilogue warps of both
    const uint32_t full = smem_u32(bars), empty = full + 8 * kPairStages, done = empty + 8 * kPairStages, drained = done + 8;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        mbar_init(done, 1);
        mbar_init(drained, 2 * kEpilogueWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_allocate_pair(&tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    pair_barrier();                                                      // both CTAs' barriers exist, and their tensor memory
    tc_fence_after();
    pdl_trigger();                                                       // not before the allocation: see kernels.hpp
    const uint32_t tmem = tmem_slot;
    const int tiles = p.f_tiles * p.n_tiles, first = blockIdx.x >> 1, step = gridDim.x >> 1;     // of 256 outputs and of 256 rows

    if (warp == 0) {
        const bool leader = elect_one();
        const uint32_t full0 = in_cta(full, 0);
        int issued = 0, slot = 0;
        uint32_t phase = 1;                                              // (the first pass over the ring does not wait)
        bool ok = true;
        pdl_wait();
        for (int t = first; ok && t < tiles; t += step) {
            int ft, nt;
            banded(t, p.band, p.f_tiles, p.n_tiles, ft, nt);
            const int xr = nt * 2 + static_cast<int>(rank), wr = ft * 2 + static_cast<int>(rank);      // row tiles of 128
            for (int i = 0; i < p.col_tiles; ++i) {
                if (issued >= kPairStages && !warp_wait(empty + 8 * slot, phase, ctx, 131)) { ok = false; break; }
                if (leader && issued + 1 != p.test_skip_load) {
                    const uint32_t at = smem + slot * kPairStage, bar = full0 + 8 * slot;
                    const bool scales = (i & 3) == 0;                    // of this column tile and the next three
                    if (rank == 0) mbar_expect_tx(full + 8 * slot, 2 * (2 * kTileCodes + (scales ? 3 * kMx8Scales : 0)));
                    // (row tiles that do not exist are outside the maps: zeros; what fits the GPU has fewer than 2^31 rows of 128 bytes)
                    tile_load(at, &maps.x, bar, 0, (xr * p.col_tiles + i) * 128);
                    tile_load(at + kTileCodes, &maps.w, bar, 0, (wr * p.col_tiles + i) * 128);
                    if (scales) {
                        const uint32_t sf = at + 2 * kTileCodes;
                        tile_load(sf, &maps.x_scales, bar, 0, (xr * p.groups + (i >> 2)) * 4);
                        tile_load(sf + kMx8Scales, &maps.w_scales, bar, 0, (ft * 2 * p.groups + (i >> 2)) * 4);
                        tile_load(sf + 2 * kMx8Scales, &maps.w_scales, bar, 0, ((ft * 2 + 1) * p.groups + (i >> 2)) * 4);
                    }
                }
                ++issued;
                if (++slot == kPairStages) { slot = 0; phase ^= 1; }
            }
        }
        // no copy of either CTA may still be in flight when the pair ends, whatever happened to the other roles
        if (rank == 0)
            for (int i = max(0, issued - kPairStages); i < issued; ++i) mbar_wait(full + 8 * (i % kPairStages), (i / kPairStages) & 1, ctx, 132);
    } else if (warp == 1 && rank == 0) {
        const bool leader = elect_one();
        int slot = 0, done_tiles = 0;
        uint32_t phase = 0, group = kPairStages - 1;                     // the scales' place in tensor memory: one of as many as there are stages,
                                                                         // so that the MMAs that used it last are done when it is written again
        const uint32_t idesc = (uint32_t(256 >> 3) << 17) | (1u << 23) | (uint32_t(256 >> 4) << 24), next_byte = (1u << 4) | (1u << 29);
        const uint64_t da0 = smem_desc_sw128(smem), db0 = smem_desc_sw128(smem + kTileCodes), s0 = scale_desc(smem + 2 * kTileCodes);
        const uint32_t own_empty = in_cta(empty, 0), peer_empty = in_cta(empty, 1), own_done = in_cta(done, 0), peer_done = in_cta(done, 1);
        bool ok = true;
        pdl_wait();                                                      // the bound of the waits below is for this kernel's copies alone
        for (int t = first; ok && t < tiles; t += step, ++done_tiles) {
            if (done_tiles > 0 && !warp_wait(drained, (done_tiles - 1) & 1, ctx, 133)) break;
            tc_fence_after();
            int steps = p.ksteps;
            uint32_t accumulate = 0;
            for (int i = 0; i < p.col_tiles; ++i, steps -= 4) {
                if (!warp_wait(full + 8 * slot, phase, ctx, 134)) { ok = false; break; }
                tc_fence_after();
                const uint64_t shift = static_cast<uint64_t>(slot) * (kPairStage >> 4);
                if ((i & 3) == 0) group = group == kPairStages - 1 ? 0 : group + 1;
                const uint32_t sfa = tmem + 256 + group * 12, sfb = sfa + 4;
                const uint32_t which = idesc + (i & 3) * next_byte;
                if (leader) {
                    if ((i & 3) == 0) {
                        copy_scales_pair(sfa, s0 + shift);
                        copy_scales_pair(sfb, s0 + shift + (kMx8Scales >> 4));
                        copy_scales_pair(sfb + 4, s0 + shift + 2 * (kMx8Scales >> 4));
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < steps) umma_mx8_pair(tmem, da0 + shift + 2 * k, db0 + shift + 2 * k, which, sfa, sfb, accumulate | k);
                    commit_pair(own_empty + 8 * slot);
                    commit_pair(peer_empty + 8 * slot);
                }
                __syncwarp();
                accumulate = 1;
                if (++slot == kPairStages) { slot = 0; phase ^= 1; }
            }
            if (leader && ok) {
                commit_pair(own_done);
                commit_pair(peer_done);
            }
            __syncwarp();
        }
        // no MMA may still run when tensor memory is freed
        if (leader && !ok) commit_pair(own_done);
        __syncwarp();
        if (done_tiles > 0) mbar_wait(done, (done_tiles - 1) & 1, ctx, 136);
    } else if (warp >= 4) {
        pdl_wait();
        const int e = warp - 4, quadrant = e & 3, quarter = e >> 2;      // lanes and columns of the accumulator this warp moves
        unsigned char *stage = smem_raw + (smem - smem_u32(smem_raw)) + kPairStages * kPairStage + e * stage_out(kPiece);
        float *bias = reinterpret_cast<float *>(stage + 32 * kPiece);
        const uint32_t from = tmem + (static_cast<uint32_t>(quadrant * 32) << 16) + quarter * 64, drained0 = in_cta(drained, 0);
        T *const y = static_cast<T *>(p.y);
        const uint64_t places = reinterpret_cast<uintptr_t>(p.y) | static_cast<uint64_t>(p.ldy * sizeof(T));
        const int aligned = places % 16 == 0 ? 16 : places % 4 == 0 ? 4 : 2;
        uint32_t phase = 0;
        for (int t = first; t < tiles; t += step) {
            int ft, nt;
            banded(t, p.band, p.f_tiles, p.n_tiles, ft, nt);
            const int f0 = ft * 256 + quarter * 64;
            const int64_t row0 = static_cast<int64_t>(nt) * 256 + rank * 128 + quadrant * 32;
            __syncwarp();
#pragma unroll
            for (int c = lane; c < 64; c += 32) bias[c] = p.bias && f0 + c < p.F ? p.bias[f0 + c] : 0.f;
            __syncwarp();
            if (!warp_wait(done, phase, ctx, 135)) break;
            phase ^= 1;
            tc_fence_after();
            uint32_t v[64];
            tmem_ld32_async(from, v);
            tmem_ld32_async(from + 32, v + 32);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_pair(drained0);
            constexpr int kCols = kPiece / sizeof(T);
            const int rows_left = static_cast<int>(max(static_cast<int64_t>(0), min(static_cast<int64_t>(32), p.rows - row0)));
            T *out = y + row0 * p.ldy + f0;
#pragma unroll
            for (int c = 0; c < 64; c += kCols) {
                if (f0 + c >= p.F || rows_left == 0) continue;
                float o[kCols];
#pragma unroll
                for (int j = 0; j < kCols; j += 4) {
                    const float4 b = *reinterpret_cast<const float4 *>(bias + c + j);
                    o[j] = activate1<ACT>(__uint_as_float(v[c + j]) + b.x);
                    o[j + 1] = activate1<ACT>(__uint_as_float(v[c + j + 1]) + b.y);
                    o[j + 2] = activate1<ACT>(__uint_as_float(v[c + j + 2]) + b.z);
                    o[j + 3] = activate1<ACT>(__uint_as_float(v[c + j + 3]) + b.w);
                }
                store_piece<T, kPiece>(o, stage, out + c, p.ldy, rows_left, p.F - f0 - c, aligned);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    pair_barrier();                                                      // nobody's shared or tensor memory goes away under its peer
    if (warp == 2) tmem_free_pair(tmem, 512);
}

// The codes of a matrix as rows of 128 bytes, its scales as four rows of 128 bytes per chunk.
cudaError_t codes_map(CUtensorMap *map, const uint8_t *base, int64_t row_tiles, int64_t col_tiles) {
    return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, base, 128, row_tiles * col_tiles * 128, 128, 128, 128, CU_TENSOR_MAP_SWIZZLE_NONE);
}
cudaError_t scales_map(CUtensorMap *map, const uint8_t *base, int64_t row_tiles, int64_t groups) {
    return encode_map(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, base, 128, row_tiles * groups * 4, 128, 128, 4, CU_TENSOR_MAP_SWIZZLE_NONE);
}

}  // namespace

cudaError_t prepare_mx8_linear() {
    const cudaFuncAttribute what = cudaFuncAttributeMaxDynamicSharedMemorySize;
    cudaError_t e = cudaSuccess;
    for (int dtype = 0; dtype < 3 && e == cudaSuccess; ++dtype)
        for (int act = PATDNN_ACT_NONE; act <= PATDNN_ACT_SILU && e == cudaSuccess; ++act)
            e = by_output(dtype, act, [&](auto t, auto a) {
                cudaError_t r = cudaFuncSetAttribute(mx8_pair_kernel<decltype(t), a.value>, what, kLinearSmem);
                if (r == cudaSuccess) r = cudaFuncSetAttribute(mx8_linear_kernel<decltype(t), a.value, false>, what, kLinearSmem);
                return r == cudaSuccess ? cudaFuncSetAttribute(mx8_linear_kernel<decltype(t), a.value, true>, what, kLinearSmem) : r;
            });
    return e;
}

Mx8Launch plan_mx8_linear(Mx8Params &p) {
    const Mx8Shape shape = mx8_shape(p.F, p.K);
    p.col_tiles = static_cast<int>(shape.col_tiles);
    p.groups = static_cast<int>(shape.groups);
    p.ksteps = static_cast<int>(ceil_div(p.K, 32));
    Mx8Launch l{};
    p.f_tiles = static_cast<int>(ceil_div(p.F, 128));
    // (row tiles start at multiples of 128: the scales of a tile start at a column of tensor memory that is a multiple of four)
    p.tile_n = p.rows <= 128 ? static_cast<int>(ceil_div(p.rows, 16) * 16) : 128;
    p.n_tiles = static_cast<int>(ceil_div(p.rows, p.tile_n));
    const int64_t tiles = static_cast<int64_t>(p.f_tiles) * p.n_tiles;
    // Exchanging partial sums takes time in proportion to the rows, 3 us for 128: with up to 64 two column tiles per CTA are enough, with more it takes
    // sixteen column tiles, four to a CTA (333 x 2048 -> 1000: 8.6 us in four splits, 10.1 in two; 256 x 1024 -> 1024: 6.2 in none, 7.6 in four).
    // (Lanes push consecutive words to a finisher; 16 bytes per lane, further apart, took 2 us more.)
    const int least = p.tile_n <= 64 ? 2 : p.col_tiles < 16 ? p.col_tiles : 4;
    p.splits = 1;
    while (p.splits < 8 && tiles * p.splits * 2 <= cluster_room(sm_count(), p.splits * 2) && p.col_tiles >= p.splits * 2 * least) p.splits *= 2;
    p.tiles_per_split = static_cast<int>(ceil_div(p.col_tiles, p.splits));
    // Pairs of CTAs where an estimate in cycles says so: a column tile takes about as long in both kernels (512 cycles of MMAs for 256 x 256
    // on two SMs; the traffic of 128 x 128 through one SM's shared memory), so rounds over the SMs decide.
    const int64_t pairs = std::max(1, sm_count() / 2), pair_tiles = ceil_div(p.rows, 256) * ceil_div(p.F, 256);
    const int64_t alone = ceil_div(tiles * p.splits, cluster_room(sm_count(), p.splits)) * (p.tiles_per_split * 600 + 2500);
    const int64_t paired = ceil_div(pair_tiles, pairs) * p.col_tiles * 560 + 3500;
    if (!p.x_raw && paired < alone) {
        l.persistent = true;
        p.tile_n = 256;
        p.f_tiles = static_cast<int>(ceil_div(p.F, 256));
        p.n_tiles = static_cast<int>(ceil_div(p.rows, 256));
        p.band = band_of(p.f_tiles, p.n_tiles, static_cast<int64_t>(256) * 128 * p.col_tiles);
        p.splits = 1;
        p.stages = kPairStages;
        l.piece = kPiece;
        p.tensor_columns = 512;
        l.grid = 2 * static_cast<unsigned>(std::min(pair_tiles, pairs));
        l.smem = kLinearSmem;                          // all of an SM's: a pair holds all of two SMs' tensor memory (see plan_mx4_linear)
        return l;
    }
    const int stage = kTileCodes + p.tile_n * 128 + 2 * kMx8Scales;
    p.stages = std::max(1, std::min({kMaxStages, p.tiles_per_split, 200 * 1024 / stage}));
    const int slots = p.splits > 1 ? static_cast<int>(ceil_div(p.tile_n, p.splits)) * p.splits * 512 : 0;
    p.tensor_columns = allocation_of(p.tile_n + 8 * p.stages);
    // Shared memory in proportion to tensor memory, as for the 4-bit product: where shared memory fits, tensor memory does.
    const int share = kSmemPerSm / 512 * p.tensor_columns - 1024;
    l.smem = std::max({p.stages * stage + 1024, slots + 1024, share});
    l.grid = static_cast<unsigned>(tiles * p.splits);
    return l;
}

cudaError_t launch_mx8_linear(Mx8Params p, cudaStream_t st, int *launches) {
    const Mx8Launch l = plan_mx8_linear(p);
    *launches = 1;
    if (l.persistent) {
        Mx8Maps maps;
        const int64_t x_tiles = ceil_div(p.rows, 128), w_tiles = ceil_div(p.F, 128);
        cudaError_t e = codes_map(&maps.x, p.x, x_tiles, p.col_tiles);
        if (e == cudaSuccess) e = codes_map(&maps.w, p.w, w_tiles, p.col_tiles);
        if (e == cudaSuccess) e = scales_map(&maps.x_scales, p.x + p.x_scales, x_tiles, p.groups);
        if (e == cudaSuccess) e = scales_map(&maps.w_scales, p.w + p.w_scales, w_tiles, p.groups);
        if (e != cudaSuccess) return e;
        return by_output(p.dtype, p.act, [&](auto t, auto a) {
            return launch_pdl(mx8_pair_kernel<decltype(t), a.value>, dim3(l.grid), dim3(kRowsThreads), l.smem, st, 2, maps, p);
        });
    }
    return by_output(p.dtype, p.act, [&](auto t, auto a) {
        const auto kernel = p.x_raw ? mx8_linear_kernel<decltype(t), a.value, true> : mx8_linear_kernel<decltype(t), a.value, false>;
        return launch_pdl(kernel, dim3(l.grid), dim3(kLinThreads), l.smem, st, p.splits, p);
    });
}

}  // namespace patdnn

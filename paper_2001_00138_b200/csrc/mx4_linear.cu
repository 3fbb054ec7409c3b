// Product of two 4-bit matrices on the block-scaled tensor cores: y = act(x w^T + bias), fp32 accumulation in tensor memory.
//
// The weights are the MMA's M operand (128 rows per tile), the rows of x its N operand (16 .. 256), so that one row of x wastes
// little and a warp's lanes write consecutive outputs.  Both operands are stored in the order the tensor cores read (mx4 layout): a
// tile is one contiguous bulk copy, scales included.  The scales travel from shared to tensor memory with tcgen05.cp, one slot per
// pipeline stage, and every MMA covers 64 columns: two blocks of 32, two scale bytes per row.
// (That is the kernel for few rows, where it streams the weights; the one for many rows, further down, has the roles the other way round.)
// Measured, weights in L2: 1 row 4096 -> 4096 4.2 us, 32 rows 25088 -> 4096 10.7 us (55 MB of weights).
#include "ops.hpp"

#include <cooperative_groups.h>

#include <algorithm>

#include "linear_device.cuh"

namespace patdnn {

namespace cg = cooperative_groups;

namespace {

constexpr int kLinThreads = 256;
constexpr int kMaxStages = 8;

// fp32 += e2m1 * e2m1 with power-of-two scales per 32 columns; M = 128, K = 64.  `half`: which two of the four scale bytes.
__device__ __forceinline__ uint32_t mx4_instr_desc(int n, int half) {
    return (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) | (1u << 27) |
           (static_cast<uint32_t>(2 * half) << 4) | (static_cast<uint32_t>(2 * half) << 29);
}
__device__ __forceinline__ void umma_mx4(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// One tile of 128 weights rows x tile_n rows of x per CTA; the column tiles cut into `splits` ranges, one CTA of a cluster each.
// X = void: the rows of x are 4-bit.  Otherwise they are elements of X, at most kFusedRows of them, and warps 2 to 7 quantise them
// into the ring themselves, a column tile at a time each: one launch less.  Measured, half, 4096 -> 4096: 1 row 5.0 us against 6.4 us as
// two launches, 8 rows 5.9 / 6.8; 25088 -> 4096: 10.0 / 12.1, 8 rows 12.0 / 12.5 (fp32 12.2 / 11.9, where it ends).
template <typename X>
__global__ void __launch_bounds__(kLinThreads, 1) mx4_linear_kernel(Mx4Params p) {
    constexpr bool kFused = !std::is_same<X, void>::value;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 1];
    __shared__ uint32_t tmem_slot;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int rank = blockIdx.x % p.splits, tile = blockIdx.x / p.splits;
    const int ft = tile % p.f_tiles, nt = tile / p.f_tiles;
    const WaitCtx ctx{p.status, p.spin_limit ? p.spin_limit : kSpinLimit};
    const uint32_t smem = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages, done = empty + 8 * kMaxStages;

    const int row_bytes = p.width / 2;
    const int atoms = p.width > 128 ? 2 : 1;                             // scale atoms (128 columns each) per column tile
    const uint32_t a_codes = 128 * row_bytes, b_codes = p.tile_n * row_bytes, sf_bytes = 512 * atoms;
    const uint32_t stage_bytes = (a_codes + b_codes + 2 * sf_bytes + 1023) & ~1023u;
    const int tmem_cols = p.tensor_columns, sf_base = p.tile_n, sf_cols = 16;    // behind the accumulator: scales per stage

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, kFused ? 2 : 1);                     // the copies, and the warp that wrote the rows of x
            mbar_init(empty + 8 * s, 1);
        }
        mbar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
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
        const uint32_t bytes = kFused ? a_codes + sf_bytes : a_codes + b_codes + 2 * sf_bytes;
        // (ring slots and phases advance without divisions: the instructions of this warp bound short column tiles)
        const uint8_t *wc = p.w + (static_cast<int64_t>(ft) * p.col_tiles + t0) * a_codes;
        const uint8_t *ws = p.w + p.w_scales + (static_cast<int64_t>(ft) * p.col_tiles + t0) * sf_bytes;
        const uint8_t *xc = p.x + (x_tile0 * p.col_tiles + t0) * a_codes;
        const uint8_t *xs = p.x + p.x_scales + (x_tile0 * p.col_tiles + t0) * sf_bytes;
        auto load_w = [&](int i, uint32_t at, uint32_t bar) {
            if (leader && i + 1 != p.test_skip_load) {
                mbar_expect_tx(bar, bytes);
                bulk_load(at, wc, a_codes, bar);
                bulk_load(at + a_codes + b_codes, ws, sf_bytes, bar);
            }
            wc += a_codes;
            ws += sf_bytes;
        };
        auto load_x = [&](int i, uint32_t at, uint32_t bar) {
            if (leader && !kFused && i + 1 != p.test_skip_load) {
                bulk_load(at + a_codes, xc, b_codes, bar);
                bulk_load(at + a_codes + b_codes + sf_bytes, xs, sf_bytes, bar);
            }
            xc += a_codes;
            xs += sf_bytes;
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
        int slot = 0, steps = min(p.ksteps - t0 * (p.width / 64), iters * (p.width / 64));
        uint32_t phase = 0, accumulate = 0;
        const uint32_t lower = mx4_instr_desc(p.tile_n, 0), upper = mx4_instr_desc(p.tile_n, 1);
        const uint64_t da0 = operand_desc(smem, row_bytes), db0 = operand_desc(smem + a_codes, row_bytes);
        const uint64_t sa0 = scale_desc(smem + a_codes + b_codes), sb0 = scale_desc(smem + a_codes + b_codes + sf_bytes);
        pdl_wait();                                                      // the bound of the waits below is for this kernel's copies alone
        for (int i = 0; i < iters; ++i, steps -= p.width / 64) {
            if (!warp_wait(full + 8 * slot, phase, ctx, 103)) break;
            tc_fence_after();
            const uint64_t shift = static_cast<uint64_t>(slot) * (stage_bytes >> 4);
            const uint32_t sfa = tmem + sf_base + slot * sf_cols, sfb = sfa + 8;
            if (leader) {
                copy_scales(sfa, sa0 + shift);
                copy_scales(sfb, sb0 + shift);
                if (atoms == 2) {
                    copy_scales(sfa + 4, sa0 + shift + 32);
                    copy_scales(sfb + 4, sb0 + shift + 32);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k * 64 < p.width && k < steps)
                        umma_mx4(tmem, da0 + shift + 2 * k, db0 + shift + 2 * k, k & 1 ? upper : lower, sfa + 4 * (k >> 1), sfb + 4 * (k >> 1), accumulate | k);
                }
                umma_commit(empty + 8 * slot);
            }
            __syncwarp();
            accumulate = 1;
            if (++slot == p.stages) { slot = 0; phase ^= 1; }
        }
        if (leader) umma_commit(done);
    } else if constexpr (kFused) {
        constexpr int kProducers = kLinThreads / 32 - 2, A = 16 / sizeof(X);
        const X *x = static_cast<const X *>(p.x_raw);
        const bool vector = (reinterpret_cast<uintptr_t>(x) | static_cast<uint64_t>(p.ldx * sizeof(X))) % 16 == 0;
        const int rows = static_cast<int>(p.rows);
        pdl_wait();
        for (int i = warp - 2; i < iters; i += kProducers) {
            const int slot = i % p.stages, turn = i / p.stages;
            const int64_t c = static_cast<int64_t>(t0 + i) * p.width + lane * 8;
            const int count = lane * 8 < p.width ? static_cast<int>(max(int64_t(0), min(int64_t(8), p.K - c))) : 0;
            Row8<X, A> raw[kFusedRows];
#pragma unroll
            for (int r = 0; r < kFusedRows; ++r) {
                const X *src = x + r * p.ldx + c;
                if (vector && count == 8 && r < rows) raw[r].load(src);
                else raw[r].load(src, r < rows ? count : 0);
            }
            if (turn > 0 && !warp_wait(empty + 8 * slot, (turn - 1) & 1, ctx, 105)) break;
            unsigned char *at = smem_raw + (smem - smem_u32(smem_raw)) + slot * stage_bytes + a_codes;
#pragma unroll
            for (int r = 0; r < kFusedRows; ++r) {
                if (r >= rows) break;
                uint32_t codes, scales = quantise8(raw[r].values(), raw[r].top(), codes);
                int place = r * row_bytes + lane * 4;
                place ^= ((place >> 7) & (p.width / 32 - 1)) << 4;
                if (lane * 8 < p.width) *reinterpret_cast<uint32_t *>(at + place) = codes;
                scales |= __shfl_down_sync(0xffffffffu, scales, 4) << 8;
                scales |= __shfl_down_sync(0xffffffffu, scales, 8) << 16;
                if ((lane & 15) == 0 && lane * 8 < p.width) *reinterpret_cast<uint32_t *>(at + b_codes + sf_bytes + (lane >> 4) * 512 + r * 16) = scales;
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
    const int f = ft * 128 + (warp & 3) * 32 + lane;
    const float bias = p.bias && f < p.F ? p.bias[f] : 0.f;
    const int64_t row0 = static_cast<int64_t>(nt) * p.tile_n;
    const uint32_t lanes = tmem + ((warp & 3) * 32u << 16);
    if (p.splits == 1) {
        for (int c = (warp >> 2) * 16; c < p.tile_n; c += 32) {
            uint32_t v[16];
            tmem_ld16(lanes + c, v);
            if (ok && f < p.F) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (row0 + c + j < p.rows)
                        store_out(p.y, (row0 + c + j) * p.ldy + f, activate(__uint_as_float(v[j]) + bias, p.act), p.dtype);
            }
        }
    } else {
        // every CTA of the cluster finishes the columns j with j % splits == its rank: partial sums are pushed into its shared memory
        // and added in rank order
        float *slots = reinterpret_cast<float *>(smem_raw + (smem - smem_u32(smem_raw)));
        const int shift = 31 - __clz(p.splits), owned = (p.tile_n + p.splits - 1) >> shift;      // splits is a power of two
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();                                                  // all pipelines are idle: their memory can be reused
        for (int c = (warp >> 2) * 16; c < p.tile_n; c += 32) {
            uint32_t v[16];
            tmem_ld16(lanes + c, v);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (row0 + c + j < p.rows) {
                    float *to = cluster.map_shared_rank(slots, (c + j) & (p.splits - 1));
                    to[(rank * owned + ((c + j) >> shift)) * 128 + (warp & 3) * 32 + lane] = iters ? __uint_as_float(v[j]) : 0.f;
                }
        }
        cluster.sync();
        if (ok && f < p.F)
            for (int j = (warp >> 2); j < owned; j += 2) {
                const int64_t row = row0 + (j << shift) + rank;
                if ((j << shift) + rank >= p.tile_n || row >= p.rows) break;
                float s = 0.f;
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < p.splits) s += slots[(r * owned + j) * 128 + (warp & 3) * 32 + lane];
                store_out(p.y, row * p.ldy + f, activate(s + bias, p.act), p.dtype);
            }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols));
}

// ---- many rows ----------------------------------------------------------------------------------------------------------
// Tiles of 128 rows of x (M) by up to 256 rows of w (N), one persistent CTA per SM walking over them.  Warp 0 fills a ring of column
// tiles, warp 1 issues the MMAs, warps 4 to 19 are the epilogue: they move the finished accumulator to registers, hand tensor memory back,
// and convert and store while the next tile is multiplied.  A lane owns a row of y; pieces of 32 rows pass through shared memory so
// that they are stored as whole sectors: 64 bytes of a row at a time where a tile has at most three column tiles and is bound by these
// stores (100352 rows, 64 -> 256 columns, bf16: 15.9 us; 32-byte pieces 17.9, eight warps 16.8), else 32 bytes, whose smaller buffers
// leave room for a fourth column tile in the ring (8192 rows, 4096 -> 4096: 56 us; 64-byte pieces and three column tiles 62).
// A column tile of 256 writes 51 KB into shared memory and the MMAs read 48 KB from it in the 512 cycles that they take: the 128 bytes per
// cycle of shared memory, not the tensor pipe (58 %), bound the large product at 5 PFLOP/s.
constexpr int kRowsThreads = 640;
constexpr int kEpilogueWarps = 16;
template <typename T, int ACT, int PIECE>
__global__ void __launch_bounds__(kRowsThreads, 1) mx4_rows_kernel(Mx4Params p) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 2];
    __shared__ uint32_t tmem_slot;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const WaitCtx ctx{p.status, p.spin_limit ? p.spin_limit : kSpinLimit};
    const uint32_t smem = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages, done = empty + 8 * kMaxStages, drained = done + 8;

    const int row_bytes = p.width / 2;
    const int atoms = p.width > 128 ? 2 : 1;                             // scale atoms (128 columns each) per column tile
    const int wide = p.tile_n / 128;                                     // row tiles of w per tile: 1 or 2
    const uint32_t codes = 128 * row_bytes, sf_bytes = 512 * atoms;      // of one row tile
    const uint32_t stage_bytes = ((1 + wide) * (codes + sf_bytes) + 1023) & ~1023u;
    const int tmem_cols = p.tensor_columns, sf_base = p.tile_n, sf_cols = 8 + 8 * wide;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        mbar_init(done, 1);
        mbar_init(drained, kEpilogueWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();                                                       // not before the allocation: see kernels.hpp
    const uint32_t tmem = tmem_slot;
    const int64_t tiles = static_cast<int64_t>(p.f_tiles) * p.n_tiles;   // f_tiles of tile_n outputs, n_tiles of 128 rows
    const int w_tiles = (p.F + 127) / 128;

    if (warp == 0) {
        const bool leader = elect_one();
        int issued = 0, slot = 0;
        uint32_t phase = 1;                                              // (the first pass over the ring does not wait)
        bool ok = true, waited = false;
        const uint32_t next_codes = p.col_tiles * codes, next_scales = p.col_tiles * sf_bytes;    // from one row tile to the next
        int ft = static_cast<int>(blockIdx.x % static_cast<unsigned>(p.f_tiles));
        int nt = static_cast<int>(blockIdx.x / static_cast<unsigned>(p.f_tiles));
        for (int64_t t = blockIdx.x; ok && t < tiles; t += gridDim.x) {
            const bool two = wide == 2 && ft * 2 + 1 < w_tiles;
            const uint32_t bytes = (two ? 3 : 2) * (codes + sf_bytes);
            const uint8_t *wc = p.w + static_cast<int64_t>(ft) * wide * next_codes;
            const uint8_t *ws = p.w + p.w_scales + static_cast<int64_t>(ft) * wide * next_scales;
            const uint8_t *xc = p.x + static_cast<int64_t>(nt) * next_codes, *xs = p.x + p.x_scales + static_cast<int64_t>(nt) * next_scales;
            for (int i = 0; i < p.col_tiles; ++i) {
                if (issued >= p.stages && !warp_wait(empty + 8 * slot, phase, ctx, 111)) { ok = false; break; }
                const uint32_t at = smem + slot * stage_bytes, bar = full + 8 * slot;
                const uint32_t sf = at + (1 + wide) * codes;
                const bool copies = leader && issued + 1 != p.test_skip_load;
                if (copies) {
                    mbar_expect_tx(bar, bytes);
                    bulk_load(at + codes, wc, codes, bar);
                    bulk_load(sf + sf_bytes, ws, sf_bytes, bar);
                    if (two) {
                        bulk_load(at + 2 * codes, wc + next_codes, codes, bar);
                        bulk_load(sf + 2 * sf_bytes, ws + next_scales, sf_bytes, bar);
                    }
                }
                if (!waited) {                                           // weights do not depend on the previous kernel, x does
                    pdl_wait();
                    waited = true;
                }
                if (copies) {
                    bulk_load(at, xc, codes, bar);
                    bulk_load(sf, xs, sf_bytes, bar);
                }
                wc += codes; ws += sf_bytes; xc += codes; xs += sf_bytes;
                ++issued;
                if (++slot == p.stages) { slot = 0; phase ^= 1; }
            }
            nt += p.step_n;                                              // the tile gridDim.x further on
            ft += p.step_f;
            if (ft >= p.f_tiles) { ft -= p.f_tiles; ++nt; }
        }
        // no copy may still be in flight when the CTA ends, whatever happened to the other roles
        for (int i = max(0, issued - p.stages); i < issued; ++i) mbar_wait(full + 8 * (i % p.stages), (i / p.stages) & 1, ctx, 112);
    } else if (warp == 1) {
        const bool leader = elect_one();
        int slot = 0, done_tiles = 0;
        uint32_t phase = 0;
        const uint32_t lower = mx4_instr_desc(p.tile_n, 0), upper = mx4_instr_desc(p.tile_n, 1);
        const uint64_t da0 = operand_desc(smem, row_bytes), db0 = operand_desc(smem + codes, row_bytes);
        const uint64_t s0 = scale_desc(smem + (1 + wide) * codes);
        const uint32_t row_scales = sf_bytes >> 4;                       // descriptor distance between the scales of two row tiles
        bool ok = true;
        pdl_wait();                                                      // the bound of the waits below is for this kernel's copies alone
        for (int64_t t = blockIdx.x; ok && t < tiles; t += gridDim.x, ++done_tiles) {
            if (done_tiles > 0 && !warp_wait(drained, (done_tiles - 1) & 1, ctx, 113)) break;
            tc_fence_after();
            int steps = p.ksteps;
            uint32_t accumulate = 0;
            for (int i = 0; i < p.col_tiles; ++i, steps -= p.width / 64) {
                if (!warp_wait(full + 8 * slot, phase, ctx, 114)) { ok = false; break; }
                tc_fence_after();
                const uint64_t shift = static_cast<uint64_t>(slot) * (stage_bytes >> 4);
                const uint64_t da = da0 + shift, db = db0 + shift, sd = s0 + shift;
                const uint32_t sfa = tmem + sf_base + slot * sf_cols, sfb = sfa + 8;
                if (leader) {
                    copy_scales(sfa, sd);
                    copy_scales(sfb, sd + row_scales);
                    if (wide == 2) copy_scales(sfb + 4, sd + 2 * row_scales);
                    if (atoms == 2) {
                        copy_scales(sfa + 4, sd + 32);
                        copy_scales(sfb + 4 * wide, sd + row_scales + 32);
                        if (wide == 2) copy_scales(sfb + 12, sd + 2 * row_scales + 32);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k * 64 < p.width && k < steps)
                            umma_mx4(tmem, da + 2 * k, db + 2 * k, k & 1 ? upper : lower, sfa + 4 * (k >> 1), sfb + 4 * wide * (k >> 1), accumulate | k);
                    }
                    umma_commit(empty + 8 * slot);
                }
                __syncwarp();
                accumulate = 1;
                if (++slot == p.stages) { slot = 0; phase ^= 1; }
            }
            if (leader && ok) umma_commit(done);
            __syncwarp();
        }
        // no MMA may still run when tensor memory is freed
        if (leader && !ok) umma_commit(done);
        __syncwarp();
        if (done_tiles > 0) mbar_wait(done, (done_tiles - 1) & 1, ctx, 116);
    } else if (warp >= 4) {
        pdl_wait();
        const int e = warp - 4, quadrant = e & 3, quarter = e >> 2;      // lanes and columns of the accumulator this warp moves
        const int cols = p.tile_n / 4;                                   // 32 or 64
        unsigned char *stage = smem_raw + (smem - smem_u32(smem_raw)) + p.stages * stage_bytes + e * stage_out(PIECE);
        float *bias = reinterpret_cast<float *>(stage + 32 * PIECE);
        const uint32_t from = tmem + (static_cast<uint32_t>(quadrant * 32) << 16) + quarter * cols;
        T *const y = static_cast<T *>(p.y);
        const uint64_t places = reinterpret_cast<uintptr_t>(p.y) | static_cast<uint64_t>(p.ldy * sizeof(T));
        const int aligned = places % 16 == 0 ? 16 : places % 4 == 0 ? 4 : 2;
        int ft = static_cast<int>(blockIdx.x % static_cast<unsigned>(p.f_tiles));
        int nt = static_cast<int>(blockIdx.x / static_cast<unsigned>(p.f_tiles));
        uint32_t phase = 0;
        auto bias_of = [&](int f) { return p.bias && f < p.F ? p.bias[f] : 0.f; };
        float ahead0 = bias_of(ft * p.tile_n + quarter * cols + lane), ahead1 = bias_of(ft * p.tile_n + quarter * cols + 32 + lane);
        for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
            const int f0 = ft * p.tile_n + quarter * cols;
            const int64_t row0 = static_cast<int64_t>(nt) * 128 + quadrant * 32;
            nt += p.step_n;                                              // the tile gridDim.x further on, whose bias is fetched meanwhile
            ft += p.step_f;
            if (ft >= p.f_tiles) { ft -= p.f_tiles; ++nt; }
            __syncwarp();
            bias[lane] = ahead0;
            if (cols == 64) bias[32 + lane] = ahead1;
            ahead0 = bias_of(ft * p.tile_n + quarter * cols + lane);
            ahead1 = bias_of(ft * p.tile_n + quarter * cols + 32 + lane);
            if (!warp_wait(done, phase, ctx, 115)) break;
            phase ^= 1;
            tc_fence_after();
            uint32_t v[64];
            tmem_ld32_async(from, v);
            if (cols == 64) tmem_ld32_async(from + 32, v + 32);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            tc_fence_before();
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(drained) : "memory");
            constexpr int kCols = PIECE / sizeof(T);
            const int rows_left = static_cast<int>(min(static_cast<int64_t>(32), p.rows - row0));
            T *out = y + row0 * p.ldy + f0;
#pragma unroll
            for (int c = 0; c < 64; c += kCols) {
                if (c >= cols || f0 + c >= p.F || rows_left <= 0) continue;
                float o[kCols];
#pragma unroll
                for (int j = 0; j < kCols; j += 4) {
                    const float4 b = *reinterpret_cast<const float4 *>(bias + c + j);
                    o[j] = activate1<ACT>(__uint_as_float(v[c + j]) + b.x);
                    o[j + 1] = activate1<ACT>(__uint_as_float(v[c + j + 1]) + b.y);
                    o[j + 2] = activate1<ACT>(__uint_as_float(v[c + j + 2]) + b.z);
                    o[j + 3] = activate1<ACT>(__uint_as_float(v[c + j + 3]) + b.w);
                }
                store_piece<T, PIECE>(o, stage, out + c, p.ldy, rows_left, p.F - f0 - c, aligned);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols));
}


}  // namespace

cudaError_t prepare_mx4_linear() {
    const cudaFuncAttribute what = cudaFuncAttributeMaxDynamicSharedMemorySize;
    cudaError_t e = cudaFuncSetAttribute(mx4_linear_kernel<void>, what, kLinearSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(mx4_linear_kernel<float>, what, kLinearSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(mx4_linear_kernel<__half>, what, kLinearSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(mx4_linear_kernel<__nv_bfloat16>, what, kLinearSmem);
    for (int dtype = 0; dtype < 3 && e == cudaSuccess; ++dtype)
        for (int act = PATDNN_ACT_NONE; act <= PATDNN_ACT_SILU && e == cudaSuccess; ++act)
            e = by_output(dtype, act, [&](auto t, auto a) {
                const cudaError_t r = cudaFuncSetAttribute(mx4_rows_kernel<decltype(t), a.value, 32>, what, kLinearSmem);
                return r == cudaSuccess ? cudaFuncSetAttribute(mx4_rows_kernel<decltype(t), a.value, 64>, what, kLinearSmem) : r;
            });
    return e;
}

Mx4Launch plan_mx4_linear(Mx4Params &p) {
    const Mx4Shape shape = mx4_shape(p.F, p.K);
    p.width = shape.width;
    p.col_tiles = static_cast<int>(shape.col_tiles);
    p.ksteps = static_cast<int>(ceil_div(p.K, 64));
    const int row_bytes = p.width / 2, atoms = p.width > 128 ? 2 : 1;
    Mx4Launch l{};
    // Many rows: as soon as tiles of 128 x 256 (or 128 x 128) fill the SMs, the persistent kernel.
    const int64_t row_tiles = ceil_div(p.rows, 128);
    const int tile_f = p.F > 128 && row_tiles * ceil_div(p.F, 256) >= sm_count() ? 256 : 128;
    if (!p.x_raw && p.rows > 64 && row_tiles * ceil_div(p.F, tile_f) >= sm_count()) {
        l.persistent = true;
        p.tile_n = tile_f;
        p.f_tiles = static_cast<int>(ceil_div(p.F, tile_f));
        p.n_tiles = static_cast<int>(row_tiles);
        p.splits = 1;
        const int wide = tile_f / 128;
        const int stage = ((1 + wide) * (128 * row_bytes + 512 * atoms) + 1023) / 1024 * 1024;
        l.piece = p.col_tiles <= 3 ? 64 : 32;
        const int out = kEpilogueWarps * stage_out(l.piece) + 1024;
        p.stages = std::min(kMaxStages, (kLinearSmem - out) / stage);
        p.tensor_columns = 512;                        // (one CTA per SM: its threads take most of the registers)
        const int64_t tiles = static_cast<int64_t>(p.f_tiles) * p.n_tiles;
        l.grid = static_cast<unsigned>(std::min<int64_t>(tiles, sm_count()));
        p.step_n = static_cast<int>(l.grid / p.f_tiles);
        p.step_f = static_cast<int>(l.grid % p.f_tiles);
        l.smem = p.stages * stage + out;
        return l;
    }
    p.f_tiles = static_cast<int>(ceil_div(p.F, 128));
    // (row tiles start at multiples of 128: the scales of a tile start at a column of tensor memory that is a multiple of four)
    p.tile_n = p.rows <= 128 ? static_cast<int>(ceil_div(p.rows, 16) * 16) : 128;
    p.n_tiles = static_cast<int>(ceil_div(p.rows, p.tile_n));
    const int64_t tiles = static_cast<int64_t>(p.f_tiles) * p.n_tiles;
    // Exchanging partial sums takes time in proportion to the rows: with up to 64 a column tile per CTA is enough (64 x 2048 -> 1000: 4.7 us
    // in eight splits, 6.9 in none), with more it takes sixteen column tiles, four to a CTA (300 x 4096 -> 1000: 8.4 us, 11.5 in none;
    // but 1000 x 2048 -> 256 with its eight: 8.2 us in none, 10.4 in two splits).
    const int least = p.tile_n <= 64 ? 1 : p.col_tiles < 16 ? p.col_tiles : 4;
    p.splits = 1;
    while (p.splits < 8 && tiles * p.splits * 2 <= sm_count() && p.col_tiles >= p.splits * 2 * least) p.splits *= 2;
    p.tiles_per_split = static_cast<int>(ceil_div(p.col_tiles, p.splits));
    const int stage = (128 * row_bytes + p.tile_n * row_bytes + 512 * atoms * 2 + 1023) / 1024 * 1024;
    p.stages = std::max(1, std::min({kMaxStages, p.tiles_per_split, 200 * 1024 / stage}));
    const int slots = p.splits > 1 ? static_cast<int>(ceil_div(p.tile_n, p.splits)) * p.splits * 512 : 0;
    p.tensor_columns = allocation_of(p.tile_n + 16 * p.stages);
    // The CTAs of a cluster wait for one another while they hold their columns, so none may find an SM's tensor memory full of CTAs that
    // wait likewise.  Every CTA takes shared memory in proportion to its columns (of 228 KB, 1 KB of which the system keeps per CTA, and of
    // 512 columns): where shared memory fits, tensor memory does.  The clusters of the convolutions take more than that share.
    const int share = kSmemPerSm / 512 * p.tensor_columns - 1024;
    l.smem = std::max({p.stages * stage + 1024, slots + 1024, share});
    l.grid = static_cast<unsigned>(tiles * p.splits);
    return l;
}

cudaError_t launch_mx4_linear(Mx4Params p, cudaStream_t st, int *launches) {
    const Mx4Launch l = plan_mx4_linear(p);
    *launches = 1;
    if (l.persistent)
        return by_output(p.dtype, p.act, [&](auto t, auto a) {
            const auto kernel = l.piece == 64 ? mx4_rows_kernel<decltype(t), a.value, 64> : mx4_rows_kernel<decltype(t), a.value, 32>;
            return launch_pdl(kernel, dim3(l.grid), dim3(kRowsThreads), l.smem, st, 1, p);
        });
    const auto kernel = !p.x_raw ? mx4_linear_kernel<void> : p.dtype == PATDNN_F32 ? mx4_linear_kernel<float>
                        : p.dtype == PATDNN_F16 ? mx4_linear_kernel<__half> : mx4_linear_kernel<__nv_bfloat16>;
    return launch_pdl(kernel, dim3(l.grid), dim3(kLinThreads), l.smem, st, p.splits, p);
}

}  // namespace patdnn

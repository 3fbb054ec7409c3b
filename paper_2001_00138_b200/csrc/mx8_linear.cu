// Product of two 8-bit matrices on the block-scaled tensor cores: y = act(x w^T + bias), fp32 accumulation in tensor memory.
//
// Both operands lie in the order the tensor cores read (mx8 layout): a tile of 128 rows and 128 columns is one contiguous bulk copy.  A scale
// belongs to 128 columns and the tensor cores take one per 32, so the four MMAs of a column tile (K = 32 each) are given the same scale byte:
// of the four bytes that a row has in tensor memory (a group of four column tiles) the instruction picks the tile's.  No rescaling of
// accumulators, and scales cost a 128th of the elements.
// Two kernels: for few rows the weights are the M operand and are streamed, their column tiles split over the CTAs of a cluster; for many
// rows persistent CTAs walk over tiles of 128 rows x 256 outputs.
#include "feed_forward.hpp"

#include <cooperative_groups.h>

#include <algorithm>

#include "linear_device.cuh"
#include "mx8_device.cuh"

namespace patdnn {

namespace cg = cooperative_groups;

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
// X = void: the rows of x are 8-bit.  Otherwise they are elements of X, at most kFusedRows of them, and warps 2 to 7 quantise them
// into the ring themselves, a column tile at a time each: one launch less.
template <typename X>
__global__ void __launch_bounds__(kLinThreads, 1) mx8_linear_kernel(Mx8Params p) {
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
        const X *x = static_cast<const X *>(p.x_raw);
        const bool vector = (reinterpret_cast<uintptr_t>(x) | static_cast<uint64_t>(p.ldx * sizeof(X))) % (4 * sizeof(X)) == 0;
        const int rows = static_cast<int>(p.rows);
        pdl_wait();
        for (int i = warp - 2; i < iters; i += kProducers) {
            const int slot = i % p.stages, turn = i / p.stages;
            const int64_t c = static_cast<int64_t>(t0 + i) * 128 + lane * 4;
            const int count = static_cast<int>(max(int64_t(0), min(int64_t(4), p.K - c)));
            Pack<X, 4> raw[kFusedRows];
#pragma unroll
            for (int r = 0; r < kFusedRows; ++r) {
                const X *src = x + r * p.ldx + c;
                if (vector && count == 4 && r < rows) {
                    raw[r].load(src);
                } else {
                    X v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = r < rows && e < count ? src[e] : from_float<X>(0.f);
                    raw[r] = narrow<X, 4>(Fv<4>::make([&](int e) { return to_float(v[e]); }));
                }
            }
            if (turn > 0 && !warp_wait(empty + 8 * slot, (turn - 1) & 1, ctx, 105)) break;
            unsigned char *at = smem_raw + (smem - smem_u32(smem_raw)) + slot * stage_bytes + kTileCodes;
#pragma unroll
            for (int r = 0; r < kFusedRows; ++r) {
                if (r >= rows) break;
                const Fv<4> f = widen<X, 4>(raw[r]);
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
    const bool ok = mbar_wait(done, 0, ctx, 104);
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
    if (warp == 2) tmem_free(tmem, tmem_cols);
}

// ---- many rows ----------------------------------------------------------------------------------------------------------
// Tiles of 128 rows of x (M) by up to 256 rows of w (N), one persistent CTA per SM walking over them.  Warp 0 fills a ring of column
// tiles, warp 1 issues the MMAs, warps 4 to 19 are the epilogue: they move the finished accumulator to registers, hand tensor memory back,
// and convert and store while the next tile is multiplied.  A lane owns a row of y; pieces of 32 rows pass through shared memory so
// that they are stored as whole sectors.
constexpr int kRowsThreads = 640;
constexpr int kEpilogueWarps = 16;
template <typename T, int ACT, int PIECE>
__global__ void __launch_bounds__(kRowsThreads, 1) mx8_rows_kernel(Mx8Params p) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 2];
    __shared__ uint32_t tmem_slot;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const WaitCtx ctx{p.status, p.spin_limit ? p.spin_limit : kSpinLimit};
    const uint32_t smem = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages, done = empty + 8 * kMaxStages, drained = done + 8;

    const int wide = p.tile_n / 128;                                     // row tiles of w per tile: 1 or 2
    constexpr uint32_t codes = kTileCodes, sf_bytes = kMx8Scales;        // of one row tile
    const uint32_t stage_bytes = ((1 + wide) * (codes + sf_bytes) + 1023) & ~1023u;
    const int tmem_cols = p.tensor_columns, sf_base = p.tile_n, sf_cols = 4 + 4 * wide;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        mbar_init(done, 1);
        mbar_init(drained, kEpilogueWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_allocate(&tmem_slot, tmem_cols);
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
        const uint32_t next_codes = p.col_tiles * codes, next_scales = p.groups * sf_bytes;    // from one row tile to the next
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
                wc += codes; xc += codes;
                if ((i & 3) == 3) { ws += sf_bytes; xs += sf_bytes; }
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
        const uint32_t idesc = mx8_instr_desc(p.tile_n, 0), next_byte = (1u << 4) | (1u << 29);
        const uint64_t da0 = smem_desc_sw128(smem), db0 = smem_desc_sw128(smem + codes);
        const uint64_t s0 = scale_desc(smem + (1 + wide) * codes);
        constexpr uint32_t row_scales = sf_bytes >> 4;                   // descriptor distance between the scales of two row tiles
        bool ok = true;
        pdl_wait();                                                      // the bound of the waits below is for this kernel's copies alone
        for (int64_t t = blockIdx.x; ok && t < tiles; t += gridDim.x, ++done_tiles) {
            if (done_tiles > 0 && !warp_wait(drained, (done_tiles - 1) & 1, ctx, 113)) break;
            tc_fence_after();
            int steps = p.ksteps;
            uint32_t accumulate = 0;
            for (int i = 0; i < p.col_tiles; ++i, steps -= 4) {
                if (!warp_wait(full + 8 * slot, phase, ctx, 114)) { ok = false; break; }
                tc_fence_after();
                const uint64_t shift = static_cast<uint64_t>(slot) * (stage_bytes >> 4);
                const uint64_t da = da0 + shift, db = db0 + shift, sd = s0 + shift;
                const uint32_t sfa = tmem + sf_base + slot * sf_cols, sfb = sfa + 4;
                const uint32_t which = idesc + (i & 3) * next_byte;
                if (leader) {
                    copy_scales(sfa, sd);
                    copy_scales(sfb, sd + row_scales);
                    if (wide == 2) copy_scales(sfb + 4, sd + 2 * row_scales);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < steps) umma_mx8(tmem, da + 2 * k, db + 2 * k, which, sfa, sfb, accumulate | k);
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
            if (!mbar_wait(done, phase, ctx, 115)) break;
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
    if (warp == 2) tmem_free(tmem, tmem_cols);
}


}  // namespace

cudaError_t prepare_mx8_linear() {
    const cudaFuncAttribute what = cudaFuncAttributeMaxDynamicSharedMemorySize;
    cudaError_t e = cudaFuncSetAttribute(mx8_linear_kernel<void>, what, kLinearSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(mx8_linear_kernel<float>, what, kLinearSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(mx8_linear_kernel<__half>, what, kLinearSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(mx8_linear_kernel<__nv_bfloat16>, what, kLinearSmem);
    for (int dtype = 0; dtype < 3 && e == cudaSuccess; ++dtype)
        for (int act = PATDNN_ACT_NONE; act <= PATDNN_ACT_SILU && e == cudaSuccess; ++act)
            e = by_output(dtype, act, [&](auto t, auto a) {
                const cudaError_t r = cudaFuncSetAttribute(mx8_rows_kernel<decltype(t), a.value, 32>, what, kLinearSmem);
                return r == cudaSuccess ? cudaFuncSetAttribute(mx8_rows_kernel<decltype(t), a.value, 64>, what, kLinearSmem) : r;
            });
    return e;
}

Mx8Launch plan_mx8_linear(Mx8Params &p) {
    const Mx8Shape shape = mx8_shape(p.F, p.K);
    p.col_tiles = static_cast<int>(shape.col_tiles);
    p.groups = static_cast<int>(shape.groups);
    p.ksteps = static_cast<int>(ceil_div(p.K, 32));
    Mx8Launch l{};
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
        const int stage = ((1 + wide) * (kTileCodes + kMx8Scales) + 1023) / 1024 * 1024;
        l.piece = p.col_tiles <= 6 ? 64 : 32;
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
    // Exchanging partial sums takes time in proportion to the rows: with up to 64 two column tiles per CTA are enough, with more it takes eight.
    const int least = p.tile_n <= 64 ? 2 : 8;
    p.splits = 1;
    while (p.splits < 8 && tiles * p.splits * 2 <= sm_count() && p.col_tiles >= p.splits * 2 * least) p.splits *= 2;
    p.tiles_per_split = static_cast<int>(ceil_div(p.col_tiles, p.splits));
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
    if (l.persistent)
        return by_output(p.dtype, p.act, [&](auto t, auto a) {
            const auto kernel = l.piece == 64 ? mx8_rows_kernel<decltype(t), a.value, 64> : mx8_rows_kernel<decltype(t), a.value, 32>;
            return launch_pdl(kernel, dim3(l.grid), dim3(kRowsThreads), l.smem, st, 1, p);
        });
    const auto kernel = !p.x_raw ? mx8_linear_kernel<void> : p.dtype == PATDNN_F32 ? mx8_linear_kernel<float>
                        : p.dtype == PATDNN_F16 ? mx8_linear_kernel<__half> : mx8_linear_kernel<__nv_bfloat16>;
    return launch_pdl(kernel, dim3(l.grid), dim3(kLinThreads), l.smem, st, p.splits, p);
}

}  // namespace patdnn

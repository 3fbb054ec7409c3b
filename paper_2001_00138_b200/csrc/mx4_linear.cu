// Product of two 4-bit matrices on the block-scaled tensor cores: y = act(x w^T + bias), fp32 accumulation in tensor memory.
//
// The weights are the MMA's M operand (128 rows per tile), the rows of x its N operand (16 .. 256), so that one row of x wastes
// little and a warp's lanes write consecutive outputs.  Both operands are stored in the order the tensor cores read (mx4 layout): a
// tile is one contiguous bulk copy, scales included.  The scales travel from shared to tensor memory with tcgen05.cp, one slot per
// pipeline stage, and every MMA covers 64 columns: two blocks of 32, two scale bytes per row.
#include "ops.hpp"

#include <cooperative_groups.h>

#include <algorithm>

#include "kernels.hpp"
#include "ops_device.cuh"
#include "umma_ptx.cuh"

namespace patdnn {

namespace cg = cooperative_groups;

namespace {

constexpr int kLinThreads = 256;
constexpr int kMaxStages = 8;

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// K-major operand rows of width/2 bytes (32, 64 or 128) in the swizzle of that width; 8-row groups are contiguous.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, int row_bytes) {
    const uint64_t layout = row_bytes == 128 ? 2 : row_bytes == 64 ? 4 : 6;
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (uint64_t(1) << 16) | (static_cast<uint64_t>(row_bytes * 8 >> 4) << 32) |
           (uint64_t(1) << 46) | (layout << 61);
}
// 32 rows of 16 bytes, not swizzled: 8-row groups 128 bytes apart.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (uint64_t(1) << 16) | (uint64_t(128 >> 4) << 32) | (uint64_t(1) << 46);
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
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
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void store_out(void *y, int64_t at, float v, int dtype) {
    if (dtype == PATDNN_F32) static_cast<float *>(y)[at] = v;
    else if (dtype == PATDNN_F16) static_cast<__half *>(y)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(y)[at] = __float2bfloat16_rn(v);
}

// One tile of 128 weights rows x tile_n rows of x per CTA; the column tiles cut into `splits` ranges, one CTA of a cluster each.
__global__ void __launch_bounds__(kLinThreads, 1) mx4_linear_kernel(Mx4Params p) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 1];
    __shared__ uint32_t tmem_slot;
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % p.splits, tile = blockIdx.x / p.splits;
    const int ft = tile % p.f_tiles, nt = tile / p.f_tiles;
    const WaitCtx ctx{p.status, p.spin_limit ? p.spin_limit : kSpinLimit};
    const uint32_t smem = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMaxStages, done = empty + 8 * kMaxStages;

    const int row_bytes = p.width / 2;
    const int atoms = p.width > 128 ? 2 : 1;                             // scale atoms (128 columns each) per column tile
    const int wide = p.tile_n > 128 ? 2 : 1;                             // row tiles of x that the tile spans
    const uint32_t a_codes = 128 * row_bytes, b_codes = p.tile_n * row_bytes, sf_bytes = 512 * atoms;
    const uint32_t stage_bytes = (a_codes + b_codes + sf_bytes * (1 + wide) + 1023) & ~1023u;
    const int tmem_cols = wide == 2 ? 512 : 256, sf_base = wide == 2 ? 256 : 128, sf_cols = 8 + 8 * wide;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full + 8 * s, 1);
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
    const uint32_t tmem = tmem_slot;

    const int t0 = rank * p.tiles_per_split, t1 = min(p.col_tiles, t0 + p.tiles_per_split);
    const int iters = max(0, t1 - t0);
    const int64_t x_tiles = (p.rows + 127) / 128;
    const int64_t x_tile0 = static_cast<int64_t>(nt) * p.tile_n / 128;
    const int x_row0 = static_cast<int>(static_cast<int64_t>(nt) * p.tile_n % 128);

    if (warp == 0 && lane == 0) {
        const uint8_t *wc = p.w + static_cast<int64_t>(ft) * p.col_tiles * a_codes;
        const uint8_t *ws = p.w + p.w_scales + static_cast<int64_t>(ft) * p.col_tiles * sf_bytes;
        const int b_tiles = static_cast<int>(min(static_cast<int64_t>(wide), x_tiles - x_tile0));
        const uint32_t b_part = wide == 2 ? a_codes : b_codes;           // bytes of one row tile's part
        const uint32_t bytes = a_codes + sf_bytes + b_tiles * (b_part + sf_bytes);
        auto load_w = [&](int i) {
            const int s = i % p.stages;
            const uint32_t at = smem + s * stage_bytes, bar = full + 8 * s;
            mbar_expect_tx(bar, bytes);
            bulk_load(at, wc + static_cast<int64_t>(t0 + i) * a_codes, a_codes, bar);
            bulk_load(at + a_codes + b_codes, ws + static_cast<int64_t>(t0 + i) * sf_bytes, sf_bytes, bar);
        };
        auto load_x = [&](int i) {
            const int s = i % p.stages;
            const uint32_t at = smem + s * stage_bytes, bar = full + 8 * s;
            for (int b = 0; b < b_tiles; ++b) {
                const int64_t t = (x_tile0 + b) * p.col_tiles + t0 + i;
                bulk_load(at + a_codes + b * a_codes, p.x + t * a_codes + x_row0 * row_bytes, b_part, bar);
                bulk_load(at + a_codes + b_codes + sf_bytes * (1 + b), p.x + p.x_scales + t * sf_bytes, sf_bytes, bar);
            }
        };
        // the weights do not depend on the previous kernel: fill the ring with them before waiting for it
        const int ahead = min(iters, p.stages);
        for (int i = 0; i < ahead; ++i) load_w(i);
        pdl_wait();
        for (int i = 0; i < ahead; ++i) load_x(i);
        int issued = ahead;
        for (int i = ahead; i < iters; ++i) {
            if (!mbar_wait(empty + 8 * (i % p.stages), (i / p.stages - 1) & 1, ctx, 101)) break;
            load_w(i);
            load_x(i);
            ++issued;
        }
        // no copy may still be in flight when the CTA ends, whatever happened to the other roles
        for (int i = max(0, issued - p.stages); i < issued; ++i) mbar_wait(full + 8 * (i % p.stages), (i / p.stages) & 1, ctx, 102);
    } else if (warp == 1 && lane == 0) {
        for (int i = 0; i < iters; ++i) {
            const int s = i % p.stages;
            if (!mbar_wait(full + 8 * s, (i / p.stages) & 1, ctx, 103)) break;
            tc_fence_after();
            const uint32_t at = smem + s * stage_bytes;
            const uint32_t sfa = tmem + sf_base + s * sf_cols, sfb = sfa + 8;
            for (int k = 0; k < atoms; ++k) {
                copy_scales(sfa + 4 * k, scale_desc(at + a_codes + b_codes + 512 * k));
                for (int b = 0; b < wide; ++b)
                    copy_scales(sfb + 4 * (k * wide + b), scale_desc(at + a_codes + b_codes + sf_bytes * (1 + b) + 512 * k));
            }
            const uint64_t da = operand_desc(at, row_bytes), db = operand_desc(at + a_codes, row_bytes);
            const int steps = min(p.width / 64, p.ksteps - (t0 + i) * (p.width / 64));
            for (int k = 0; k < steps; ++k)
                umma_mx4(tmem, da + 2 * k, db + 2 * k, mx4_instr_desc(p.tile_n, k & 1), sfa + 4 * (k >> 1), sfb + 4 * wide * (k >> 1), i | k);
            umma_commit(empty + 8 * s);
        }
        umma_commit(done);
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
        const int owned = (p.tile_n + p.splits - 1) / p.splits;
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();                                                  // all pipelines are idle: their memory can be reused
        for (int c = (warp >> 2) * 16; c < p.tile_n; c += 32) {
            uint32_t v[16];
            tmem_ld16(lanes + c, v);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (row0 + c + j < p.rows) {
                    float *to = cluster.map_shared_rank(slots, (c + j) % p.splits);
                    to[(rank * owned + (c + j) / p.splits) * 128 + (warp & 3) * 32 + lane] = iters ? __uint_as_float(v[j]) : 0.f;
                }
        }
        cluster.sync();
        if (ok && f < p.F)
            for (int j = (warp >> 2); j < owned; j += 2) {
                const int64_t row = row0 + j * p.splits + rank;
                if (j * p.splits + rank >= p.tile_n || row >= p.rows) break;
                float s = 0.f;
                for (int r = 0; r < p.splits; ++r) s += slots[(r * owned + j) * 128 + (warp & 3) * 32 + lane];
                store_out(p.y, row * p.ldy + f, activate(s + bias, p.act), p.dtype);
            }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols));
}

}  // namespace

cudaError_t prepare_mx4_linear() { return cudaFuncSetAttribute(mx4_linear_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024); }

cudaError_t launch_mx4_linear(Mx4Params p, cudaStream_t st, int *launches) {
    const int row_bytes = p.width / 2, atoms = p.width > 128 ? 2 : 1;
    p.f_tiles = static_cast<int>(ceil_div(p.F, 128));
    p.tile_n = p.rows <= 128 ? static_cast<int>(ceil_div(p.rows, 16) * 16)
                             : (ceil_div(p.rows, 256) * p.f_tiles >= sm_count() ? 256 : 128);
    p.n_tiles = static_cast<int>(ceil_div(p.rows, p.tile_n));
    const int64_t tiles = static_cast<int64_t>(p.f_tiles) * p.n_tiles;
    p.splits = 1;
    while (p.splits < 8 && tiles * p.splits * 2 <= sm_count() && p.splits * 2 <= p.col_tiles) p.splits *= 2;
    p.tiles_per_split = static_cast<int>(ceil_div(p.col_tiles, p.splits));
    const int wide = p.tile_n > 128 ? 2 : 1;
    const int stage = (128 * row_bytes + p.tile_n * row_bytes + 512 * atoms * (1 + wide) + 1023) / 1024 * 1024;
    p.stages = std::max(1, std::min({kMaxStages, p.tiles_per_split, 200 * 1024 / stage}));
    const int slots = p.splits > 1 ? static_cast<int>(ceil_div(p.tile_n, p.splits)) * p.splits * 512 : 0;
    const int smem = std::max(p.stages * stage, slots) + 1024;
    *launches = 1;
    return launch_pdl(mx4_linear_kernel, dim3(static_cast<unsigned>(tiles * p.splits)), dim3(kLinThreads), smem, st, p.splits, p);
}

}  // namespace patdnn

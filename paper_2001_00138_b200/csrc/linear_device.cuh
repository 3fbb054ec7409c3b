// Device and host pieces that the linear layers share: warp-uniform roles, bulk copies, operand and scale descriptors, reads of tensor
// memory, and the epilogue's way from registers to rows of y.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "kernels.hpp"
#include "ops_device.cuh"
#include "umma_ptx.cuh"

namespace patdnn {
namespace {

// The single-thread roles run as whole warps whose values are the same in all lanes (they then live in uniform registers, which the copy
// and MMA instructions take their operands from); one elected lane issues.
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const WaitCtx &ctx, int code) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, ctx, code));
}
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
// Tiles in the order in which the pairs of CTAs take them: bands of tiles of one operand, in a band all tiles of the other one after the other.  A
// band stays in L2 while the other operand passes, which is then read once per band: bands as large as L2 holds besides what passes.  Where that is a
// few tiles, or where the other operand stays in L2 anyway, eight, so that eight by nine tiles at a time share what is read.  (64 x 8 tiles of 256 x 256
// with a summed dimension of 4096 read 1.03 GB from memory without bands, 0.41 in bands of 20, 0.22 in bands of 8; 16 x 64 tiles 0.15 GB in bands of 8,
// 0.08 in one of 16.)
inline int band_of(int m_tiles, int n_tiles, int64_t tile_bytes) {
    if (n_tiles * tile_bytes <= int64_t(32) << 20) return 8;
    const int64_t fit = (int64_t(40) << 20) / tile_bytes;
    return fit < 8 ? 8 : fit < m_tiles ? static_cast<int>(fit) : m_tiles;
}
__device__ __forceinline__ void banded(int tile, int tiles_of_band, int m_tiles, int n_tiles, int &mt, int &nt) {
    const int band = tile / (tiles_of_band * n_tiles), rest = tile - band * tiles_of_band * n_tiles, here = min(tiles_of_band, m_tiles - band * tiles_of_band);
    nt = rest / here;
    mt = band * tiles_of_band + rest - nt * here;
}
// Tensor memory of a CTA: one whole warp takes it and publishes its address behind the next barrier, one whole warp gives it back.
__device__ __forceinline__ void tmem_allocate(uint32_t *slot, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
}
// The same for the two CTAs of a pair, each of which calls it.
__device__ __forceinline__ void tmem_allocate_pair(uint32_t *slot, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free_pair(uint32_t tmem, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
// Pairs of CTAs.  Barriers that both use lie in the first CTA.  The second one's copies count on the first one's barrier; it is the first one
// that expects the bytes of both: an arrival across the pair with release semantics, once per block of copies, takes longer than the block's
// MMAs (measured: 4096 x 4096 x 16384 bf16 677 us, 319 us without).
__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t in_cta(uint32_t local, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(local), "r"(rank));
    return a;
}
__device__ __forceinline__ void pair_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Tells the first CTA that tensor memory has been read (the reads are waited for and fenced before).  Release at the scope of the cluster would also
// wait for the rows that the warp stored before: 100 us of 8192 x 4096 -> 4096, 8 bits, became 95.
__device__ __forceinline__ void arrive_pair(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 rows of 16 bytes, not swizzled: 8-row groups 128 bytes apart.
__device__ __forceinline__ uint64_t scale_desc(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (uint64_t(1) << 16) | (uint64_t(128 >> 4) << 32) | (uint64_t(1) << 46);
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
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

__host__ __device__ constexpr int stage_out(int piece) { return 32 * piece + 64 * 4; }     // shared memory of an epilogue warp: a piece of 32 rows, the bias of its columns

__device__ __forceinline__ void tmem_ld32_async(uint32_t addr, uint32_t *v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
          "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
          "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr) : "memory");
}

// One warp: PIECE bytes of 32 rows, from registers to y.
template <typename T, int PIECE>
__device__ __forceinline__ void store_piece(const float (&v)[PIECE / sizeof(T)], unsigned char *stage, T *y, int64_t ldy, int rows_left, int cols_left, int aligned) {
    const int lane = threadIdx.x & 31;
    constexpr int kCols = PIECE / sizeof(T), kUnits = PIECE / 16, kShift = PIECE == 64 ? 1 : 2;
    uint32_t w[PIECE / 4];
#pragma unroll
    for (int j = 0; j < PIECE / 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            w[j] = __float_as_uint(v[j]);
        } else if constexpr (std::is_same<T, __half>::value) {
            const __half2 h = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t *>(&h);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t *>(&h);
        }
    }
    // 16-byte unit q of row r sits at unit q ^ (r >> kShift): eight lanes of a store, and of a load, touch all banks once
    auto place = [&](int r, int q) { return r * PIECE + ((q ^ ((r >> kShift) & (kUnits - 1))) << 4); };
    __syncwarp();
#pragma unroll
    for (int q = 0; q < kUnits; ++q) *reinterpret_cast<uint4 *>(stage + place(lane, q)) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
    __syncwarp();
    if (aligned == 16 && cols_left >= kCols) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int r = i * (32 / kUnits) + lane / kUnits, q = lane % kUnits;
            const uint4 t = *reinterpret_cast<const uint4 *>(stage + place(r, q));
            if (r < rows_left) *reinterpret_cast<uint4 *>(reinterpret_cast<unsigned char *>(y + r * ldy) + q * 16) = t;
        }
    } else if (sizeof(T) == 2 && aligned >= 4) {       // pairs of columns
        constexpr int kPairs = PIECE / 4;
        const int c = lane % kPairs * 2;
        if (c < cols_left) {
#pragma unroll 8
            for (int r = lane / kPairs; r < 32; r += 32 / kPairs) {
                if (r >= rows_left) continue;
                const uint32_t t = *reinterpret_cast<const uint32_t *>(stage + place(r, c >> 3) + (c * 2 & 15));
                if (c + 1 < cols_left) *reinterpret_cast<uint32_t *>(y + r * ldy + c) = t;
                else *reinterpret_cast<uint16_t *>(y + r * ldy + c) = static_cast<uint16_t>(t);
            }
        }
    } else {
        const int c = lane % kCols, b = c * static_cast<int>(sizeof(T));
        if (c < cols_left) {
#pragma unroll 8
            for (int r = lane / kCols; r < 32; r += 32 / kCols)
                if (r < rows_left) y[r * ldy + c] = *reinterpret_cast<const T *>(stage + place(r, b >> 4) + (b & 15));
        }
    }
}

template <typename F> cudaError_t by_output(int dtype, int act, F f) {
    return by_act(act, [&](auto a) {
        if (dtype == PATDNN_F32) return f(float{}, a);
        if (dtype == PATDNN_F16) return f(__half{}, a);
        return f(__nv_bfloat16{}, a);
    });
}
constexpr int kLinearSmem = 226 * 1024;
constexpr int kSmemPerSm = 228 * 1024;
typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void *sym = nullptr;
        cudaDriverEntryPointQueryResult found;
        const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &found) == cudaSuccess && found == cudaDriverEntryPointSuccess;
        return ok ? reinterpret_cast<EncodeTiled>(sym) : nullptr;
    }();
    return fn;
}
// A matrix of `rows` rows of `cols` elements, `row_bytes` apart (a multiple of 16), read in boxes; zeros outside.
inline cudaError_t encode_map(CUtensorMap *map, CUtensorMapDataType type, const void *base, int64_t cols, int64_t rows, int64_t row_bytes, int box_cols, int box_rows,
                              CUtensorMapSwizzle swizzle) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(row_bytes)};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows)}, ones[2] = {1, 1};
    const CUresult r = encode(map, type, 2, const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// Columns of tensor memory come in powers of two, at least 32.
inline int allocation_of(int columns) {
    int n = 32;
    while (n < columns) n *= 2;
    return n;
}

}  // namespace
}  // namespace patdnn

// Elementwise work of the gated feed-forward block in front of its products, one launch: rows that the tensor-core copies cannot read as they
// lie are packed, and the gradients of both projections are formed from what the forward pass kept:  dg = dh u act'(g), du = dh act(g).
//
// Memory bound (4096 x 8192 bf16: 50 us for 336 MB, 6.7 TB/s with part of it in L2).  A warp takes 256 columns of a row, 8 per lane.  dg and du are
// rounded to the type of the products that read them, which take no wider operands at this rate: at most 2^-8 of each term for bf16 (2^-11 for half),
// independent of one another, so that a product's relative error grows to about sqrt(2) times that of the result's own rounding.
// Half: dg and du may leave its range where the gradients do not (dh = u = 300), or fall below it (dh = 1e-5, act(g) = 1e-3, summed over thousands of
// rows).  They are multiplied by a power of two before they are rounded, which puts the largest finite magnitude of a row (for dx), or of a
// column (for dwg, dwu), between 2^14 and 2^15, and the products' rows are divided by it in fp32: what is below 2^-29 of the largest loses bits, what is
// below 2^-40 is 0.  It takes a pass for the magnitudes in front, and a copy of dg and du for either product (4096 x 8192: 53 and 96 us, where one copy
// as it is takes 57).
#include <algorithm>

#include "feed_forward.hpp"
#include "kernels.hpp"
#include "mx8_device.cuh"

namespace patdnn {
namespace {

constexpr int kWarps = 8, kColumns = 256;
constexpr int kJobs = 4;                               // three matrices to pack, then the slopes

struct AuxJob {
    const void *x, *dh;                                // slopes: gu, dh
    void *to, *by_column;                              // half: to scaled by rows and by_column by columns, or nullptr
    uint32_t *row_top, *column_top;
    float *row_unscale, *column_unscale;
    int64_t row, dh_row, to_row;                       // strides in elements
    int64_t units;                                     // rows, or sets of them, times pieces
    int set;                                           // slopes, half: rows of a unit
    int cols, padded, pieces;                          // padded: columns that are written; pieces of 256 of them
    int aligned;                                       // slopes: rows of gu and dh are, to 16 bytes
    int64_t rows;                                      // of a copy
    int copies;                                        // shifted ones, or 0
    uint8_t shift[kMostPhases];
};
struct AuxArgs {
    AuxJob job[kJobs];
    int64_t units;
};

template <typename T>
__device__ __forceinline__ void pack(const AuxJob &a, int64_t row, int c0) {
    Strip<T, 8, 8> s;
    s.load_any(static_cast<const T *>(a.x) + row * a.row + c0, a.cols - c0);
    s.store(static_cast<T *>(a.to) + row * a.to_row + c0, a.padded - c0);
}

// Copies of few rows, one element at a time.
__device__ __forceinline__ void pack_shifted(const AuxJob &a, int64_t row, int c0) {
    const int copy = static_cast<int>(row / a.rows), c = c0 + (threadIdx.x & 31) * 8 - a.shift[copy];
    if (c + a.shift[copy] >= a.padded) return;
    const uint16_t *from = static_cast<const uint16_t *>(a.x) + (row - copy * a.rows) * a.row + c;
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e >= 0 && c + e < a.cols ? from[e] : 0;
    *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.to) + row * a.to_row + c + a.shift[copy]) =
        make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

template <typename T> __device__ __forceinline__ uint32_t nonzero2(uint32_t pair) {      // all ones where a 16-bit number is not 0 (a NaN is not)
    if constexpr (std::is_same<T, __half>::value) return __hneu2_mask(*reinterpret_cast<const __half2 *>(&pair), __half2half2(__ushort_as_half(0)));
    else return __hneu2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&pair), __bfloat162bfloat162(__ushort_as_bfloat16(0)));
}
// dg and du of 8 columns per lane of a row.
template <typename T, bool ALIGNED, int ACT>
__device__ __forceinline__ void slopes(const AuxJob &a, int64_t row, int c0, float (&dg)[8], float (&du)[8]) {
    const int left = a.cols - c0;
    Strip<T, 8, 8> sg, su, sd;
    const T *g = static_cast<const T *>(a.x) + row * a.row + c0, *dh = static_cast<const T *>(a.dh) + row * a.dh_row + c0;
    if constexpr (ALIGNED) {
        sg.load(g, left);
        su.load(g + a.cols, left);
        sd.load(dh, left);
    } else {
        sg.load_any(g, left);
        su.load_any(g + a.cols, left);
        sd.load_any(dh, left);
    }
    // Nothing passes where dh is 0 or the slope is, whatever gu holds there: an infinity in it is a number too large for the type, and a masked row may hold
    // anything.  (On packed pairs, and with selections: 3 us of 111 for 4096 x 8192; element by element 10.)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t open = nonzero2<T>(sd.v[0].w[k]);
        sg.v[0].w[k] &= open;
        su.v[0].w[k] &= open;
    }
    float fd[8];
    sg.widen_to(dg);
    su.widen_to(du);
    sd.widen_to(fd);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float g = dg[e], through = fd[e] * du[e];
        if constexpr (ACT == PATDNN_ACT_RELU) {        // slope 0 at 0; a NaN passes
            dg[e] = g > 0.f ? through : g <= 0.f ? 0.f : g;
            du[e] = fd[e] * (g < 0.f ? 0.f : g);
        } else if constexpr (ACT == PATDNN_ACT_SILU) {
            const float s = sigmoid(g);                // at infinities (g left the range of the type) the limits: 0 and 0, or g and 1
            const float act = s == 0.f ? 0.f : g * s, slope = s == 1.f ? 1.f : fmaf(act, 1.f - s, s);
            dg[e] = s == 0.f ? 0.f : through * slope;
            du[e] = fd[e] * act;
        } else {
            dg[e] = through;
            du[e] = fd[e] * g;
        }
    }
}

// A row; half: a.set rows
template <typename T, bool ALIGNED, int ACT>
__device__ __forceinline__ void store_slopes(const AuxJob &a, int64_t row, int c0) {
    const int left = a.padded - c0, c = c0 + (threadIdx.x & 31) * 8;
    if constexpr (!std::is_same<T, __half>::value) {
        float dg[8], du[8];
        slopes<T, ALIGNED, ACT>(a, row, c0, dg, du);
        T *to = static_cast<T *>(a.to) + row * a.to_row + c0;
        Strip<T, 8, 8> s;
        s.narrow_from(dg);
        s.store(to, left);
        s.narrow_from(du);
        s.store(to + a.padded, left);
    } else {
        Fv<8> of_column[2];
        const bool columns = a.by_column && c < a.padded;
        if (columns) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint4 *top = reinterpret_cast<const uint4 *>(a.column_top + k * a.padded + c);
                const uint4 lo = top[0], hi = top[1];
                const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                of_column[k] = Fv<8>::make([&](int e) { return gated_scale(w[e]); });
                if (row == 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) a.column_unscale[k * a.padded + c + e] = gated_unscale(w[e]);
                }
            }
        }
        const int64_t last = min(row + a.set, a.rows);
        for (; row < last; ++row) {
            float d[2][8];
            slopes<T, ALIGNED, ACT>(a, row, c0, d[0], d[1]);
            const int64_t at = row * a.to_row + c0;
            const uint32_t row_top = a.row_top[row];
            const Fv<8> of_row = Fv<8>::all(gated_scale(row_top));
            if (c == 0) a.row_unscale[row] = gated_unscale(row_top);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Fv<8> v = Fv<8>::make([&](int e) { return d[k][e]; });
                Strip<T, 8, 8> s;
                if (a.to) {
                    s.v[0] = narrow<T, 8>(v * of_row);
                    s.store(static_cast<T *>(a.to) + at + k * a.padded, left);
                }
                if (columns) {
                    s.v[0] = narrow<T, 8>(v * of_column[k]);
                    s.store(static_cast<T *>(a.by_column) + at + k * a.padded, left);
                }
            }
        }
    }
}

// The largest magnitudes of dg and du, per row and per column of either, as bits (which are in their order; a NaN has none, and where one is an infinity all of
// that row of the product is).  A CTA takes 256 columns; its warps take `rows`
// rows each, four at a time, and join what they have of the columns.  Maxima do not depend on the order; the words are 0 before (the products clear them for
// the next call).
template <bool ALIGNED, int ACT>
__global__ void __launch_bounds__(kWarps * 32, 3) gated_magnitudes_kernel(const __grid_constant__ AuxJob a, int rows) {
    __shared__ __align__(16) uint32_t tops[2][kWarps][kColumns];
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t set = blockIdx.x / a.pieces, first = (set * kWarps + warp) * rows, last = min(first + rows, a.rows) - 1;
    const int c0 = static_cast<int>(blockIdx.x - set * a.pieces) * kColumns;
    pdl_wait();
    float top[2][8] = {};
    for (int64_t row = first; row <= last; row += 4) {
        float of_row[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float dg[8], du[8];
            slopes<__half, ALIGNED, ACT>(a, min(row + k, last), c0, dg, du);           // (the last one again changes nothing)
            of_row[k] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                top[0][e] = fmaxf(top[0][e], fabsf(dg[e]));
                top[1][e] = fmaxf(top[1][e], fabsf(du[e]));
                of_row[k] = fmaxf(of_row[k], fmaxf(fabsf(dg[e]), fabsf(du[e])));
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(of_row[k]));
            if (lane == 0) atomicMax(a.row_top + min(row + k, last), most);
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 8; e += 4) *reinterpret_cast<float4 *>(&tops[k][warp][lane * 8 + e]) = make_float4(top[k][e], top[k][e + 1], top[k][e + 2], top[k][e + 3]);
    __syncthreads();
    const int c = c0 + static_cast<int>(threadIdx.x);
    if (c >= a.padded) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        uint32_t most = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) most = max(most, tops[k][w][threadIdx.x]);
        atomicMax(a.column_top + k * a.padded + c, most);
    }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kWarps * 32, std::is_same<T, __half>::value ? 3 : 4) gated_operands_kernel(const __grid_constant__ AuxArgs args) {
    pdl_trigger();
    pdl_wait();
    const int64_t step = static_cast<int64_t>(gridDim.x) * kWarps;
    for (int64_t unit = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); unit < args.units; unit += step) {
        int64_t u = unit;
        int j = 0;
        while (u >= args.job[j].units) u -= args.job[j++].units;
        const AuxJob &a = args.job[j];
        if (std::is_same<T, __half>::value && j == kJobs - 1) u = a.units - 1 - u;     // backwards through what L2 still holds of the magnitudes' pass
        int64_t row = u / a.pieces;
        const int c0 = static_cast<int>(u - row * a.pieces) * kColumns;
        if (std::is_same<T, __half>::value && j == kJobs - 1) row *= a.set;
        if (j == kJobs - 1) {
            if (a.aligned) store_slopes<T, true, ACT>(a, row, c0);
            else store_slopes<T, false, ACT>(a, row, c0);
        } else if (a.copies) {
            pack_shifted(a, row, c0);
        } else {
            pack<T>(a, row, c0);
        }
    }
}

}  // namespace

cudaError_t launch_gated_operands(const GatedShape &s, const GatedPack (&packs)[3], const GatedSlopes *slopes, int64_t rows, cudaStream_t st, int *launches) {
    AuxArgs args{};
    *launches = 1;
    for (int i = 0; i < 3; ++i) {
        if (packs[i].rows == 0) continue;
        AuxJob &a = args.job[i];
        a.x = packs[i].from; a.to = packs[i].to; a.row = packs[i].row; a.to_row = packs[i].to_row; a.cols = s.K; a.padded = static_cast<int>(packs[i].to_row);
        a.pieces = static_cast<int>(ceil_div(a.padded, kColumns));
        a.rows = packs[i].rows; a.copies = packs[i].copies;
        std::copy(packs[i].shift, packs[i].shift + kMostPhases, a.shift);
        a.units = packs[i].rows * std::max(1, a.copies) * a.pieces;
    }
    if (slopes) {
        AuxJob &a = args.job[kJobs - 1];
        a.x = slopes->gu; a.dh = slopes->dh; a.to = slopes->dgu; a.by_column = slopes->by_column; a.row = 2 * static_cast<int64_t>(s.F); a.dh_row = s.h_row;
        a.row_top = slopes->row_top; a.column_top = slopes->column_top;
        a.row_unscale = slopes->row_unscale; a.column_unscale = slopes->column_unscale;
        a.cols = s.F; a.padded = gated_padded(s.F); a.to_row = 2 * static_cast<int64_t>(a.padded);
        a.pieces = static_cast<int>(ceil_div(a.padded, kColumns));
        a.rows = rows;
        a.units = rows * a.pieces;
        a.aligned = strip_width(s.dtype, {slopes->gu, slopes->dh}, {s.F, s.h_row}) == 8;
        if (s.dtype == PATDNN_F16) {
            a.set = a.units <= static_cast<int64_t>(sm_count()) * 64 ? 1 : 8;          // (the columns' scales are read once per set: 4096 x 8192 154 us a row at a time)
            a.units = ceil_div(rows, a.set) * a.pieces;
            // rows of a warp: four where there are few CTAs, else as many as make a column's maxima cheap
            const int of_warp = ceil_div(rows, kWarps * 4) * a.pieces <= static_cast<int64_t>(sm_count()) * 8 ? 4 : 16;
            const dim3 grid(static_cast<unsigned>(ceil_div(rows, kWarps * of_warp) * a.pieces));
            const cudaError_t e = by_act(s.act, [&](auto act) {
                return a.aligned ? launch_pdl(gated_magnitudes_kernel<true, act.value>, grid, dim3(kWarps * 32), 0, st, 1, a, of_warp)
                                 : launch_pdl(gated_magnitudes_kernel<false, act.value>, grid, dim3(kWarps * 32), 0, st, 1, a, of_warp);
            });
            if (e != cudaSuccess) return e;
            *launches = 2;
        }
    }
    for (const AuxJob &a : args.job) args.units += a.units;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(ceil_div(args.units, kWarps), static_cast<int64_t>(sm_count()) * 32)));
    return by_act(s.act, [&](auto act) {
        return s.dtype == PATDNN_F16 ? launch_pdl(gated_operands_kernel<__half, act.value>, grid, dim3(kWarps * 32), 0, st, 1, args)
                                     : launch_pdl(gated_operands_kernel<__nv_bfloat16, act.value>, grid, dim3(kWarps * 32), 0, st, 1, args);
    });
}

}  // namespace patdnn

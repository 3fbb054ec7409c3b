// Elementwise work of the gated feed-forward block in front of its products, one launch: rows that the tensor-core copies cannot read as they
// lie are packed, and the gradients of both projections are formed from what the forward pass kept:  dg = dh u act'(g), du = dh act(g).
//
// Memory bound (4096 x 8192 bf16: 61 us for 336 MB from cold caches, 5.5 TB/s, issue 66 %).  A warp takes 256 columns of a row, 8 per lane.  dg and du are
// rounded to the type of the products that read them, which take no wider operands at this rate: at most 2^-8 of each term for bf16 (2^-11 for half),
// independent of one another, so that a product's relative error grows to about sqrt(2) times that of the result's own rounding.
// Half: dg and du may leave its range where the gradients do not (dh = u = 300), or fall below it (dh = 1e-5, act(g) = 1e-3, summed over thousands of
// rows).  dx is given a copy of them, dwg and dwu another, and the largest magnitudes of every row and column of them are found on the way.  Where that is between
// 2^-3 and 2^15 the copies stay as they are: half's steps below 2^-14 are 2^-22 of it at most.  Any other row is then written once more into the one copy, any other
// column into the other, times the power of two that puts the largest magnitude between 2^14 and 2^15 (what is below 2^-29 of it loses bits, what is below
// 2^-40 is 0), and the products' rows are divided by it in fp32.  (4096 x 8192: 81 us for the first pass and 7 for the second, 91 where all
// needs a scale; with one copy and no magnitudes 58.  Finding the magnitudes first, and scaling all of both copies, 53 and 96.)
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
    void *to, *by_column;                              // half: the copies for dx and for dwg and dwu, or nullptr
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
template <typename T> __device__ __forceinline__ uint32_t top2(uint32_t a, uint32_t b) {  // larger magnitudes of two pairs; a NaN is larger than anything
    uint32_t r;
    if constexpr (std::is_same<T, __half>::value) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a & 0x7fff7fffu), "r"(b & 0x7fff7fffu));
    else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a & 0x7fff7fffu), "r"(b & 0x7fff7fffu));
    return r;
}
// 8 columns per lane of a row of gu and dh.
template <typename T> struct SlopeRow {
    Strip<T, 8, 8> g, u, dh;
    template <bool ALIGNED> __device__ __forceinline__ void load(const AuxJob &a, int64_t row, int c0) {
        const int left = a.cols - c0;
        const T *from = static_cast<const T *>(a.x) + row * a.row + c0, *of_h = static_cast<const T *>(a.dh) + row * a.dh_row + c0;
        if constexpr (ALIGNED) {
            g.load(from, left);
            u.load(from + a.cols, left);
            dh.load(of_h, left);
        } else {
            g.load_any(from, left);
            u.load_any(from + a.cols, left);
            dh.load_any(of_h, left);
        }
    }
    // Nothing passes where dh is 0 or the slope is, whatever gu holds there: an infinity in it is a number too large for the type, and a masked row may hold
    // anything.  Zeros take the places of such u, and of g where it is dh that is 0.  (Looked for first: 4096 x 8192 bf16 61 us, done always 63; neither 58.)
    template <int ACT> __device__ __forceinline__ void shut() {
        float z[8];
        g.widen_to(z);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t open = nonzero2<T>(dh.v[0].w[k]);
            uint32_t slope = 0xffffffffu;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (ACT == PATDNN_ACT_RELU ? z[2 * k + e] <= 0.f : ACT == PATDNN_ACT_SILU && sigmoid(z[2 * k + e]) == 0.f) slope &= e ? 0x0000ffffu : 0xffff0000u;
            g.v[0].w[k] &= open;
            u.v[0].w[k] &= open & slope;
        }
    }
    // d[0]: dg, d[1]: du
    template <int ACT> __device__ __forceinline__ void slopes(float (&d)[2][8]) {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) top = top2<T>(top, top2<T>(g.v[0].w[k], u.v[0].w[k]));
        constexpr uint32_t kInfinity = std::is_same<T, __half>::value ? 0x7c00 : 0x7f80;
        if ((top & 0x7fff) >= kInfinity || (top >> 16 & 0x7fff) >= kInfinity) shut<ACT>();
        float fd[8];
        g.widen_to(d[0]);
        u.widen_to(d[1]);
        dh.widen_to(fd);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float act = d[0][e], slope = 1.f;
            if constexpr (ACT == PATDNN_ACT_RELU) {    // slope 0 at 0; a NaN passes
                act = d[0][e] < 0.f ? 0.f : d[0][e];
                slope = d[0][e] > 0.f ? 1.f : d[0][e] <= 0.f ? 0.f : d[0][e];
            } else if constexpr (ACT == PATDNN_ACT_SILU) {
                const float s = sigmoid(d[0][e]);      // at infinities (g left the range of the type) the limits: 0 and 0, or g and 1
                act = s == 0.f ? 0.f : d[0][e] * s;
                slope = s == 1.f ? 1.f : fmaf(act, 1.f - s, s);
            }
            d[0][e] = fd[e] * d[1][e] * slope;
            d[1][e] = fd[e] * act;
        }
    }
};

template <typename T, bool ALIGNED, int ACT>
__device__ __forceinline__ void store_slopes(const AuxJob &a, int64_t row, int c0) {
    SlopeRow<T> s;
    float d[2][8];
    s.template load<ALIGNED>(a, row, c0);
    s.template slopes<ACT>(d);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        Strip<T, 8, 8> out;
        out.narrow_from(d[k]);
        out.store(static_cast<T *>(a.to) + row * a.to_row + k * a.padded + c0, a.padded - c0);
    }
}

// Half: both copies as they are, and the largest magnitudes as bits (which are in their order; a NaN has none).  A CTA takes 256 columns; its warps take `rows` rows
// each, two at a time, and join what they have of the columns.  Maxima do not depend on the order; the words are 0 before (the products clear them for the
// next call).
template <bool ALIGNED, int ACT>
__global__ void __launch_bounds__(kWarps * 32, 3) gated_slopes_kernel(const __grid_constant__ AuxJob a, int rows) {
    constexpr int kTogether = 2;
    __shared__ __align__(16) uint32_t tops[2][kWarps][kColumns];
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t set = blockIdx.x / a.pieces, first = (set * kWarps + warp) * rows, last = min(first + rows, a.rows);
    const int c0 = static_cast<int>(blockIdx.x - set * a.pieces) * kColumns;
    pdl_wait();
    float top[2][8] = {};
    for (int64_t row = first; row < last; row += kTogether) {
        SlopeRow<__half> s[kTogether];
#pragma unroll
        for (int k = 0; k < kTogether; ++k) s[k].load<ALIGNED>(a, min(row + k, last - 1), c0);
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            if (row + k >= last) break;
            float d[2][8], of_row = 0.f;
            s[k].slopes<ACT>(d);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    top[i][e] = fmaxf(top[i][e], fabsf(d[i][e]));
                    of_row = fmaxf(of_row, fabsf(d[i][e]));
                }
                Strip<__half, 8, 8> out;
                out.narrow_from(d[i]);
                const int64_t at = (row + k) * a.to_row + i * a.padded + c0;
                if (a.to) out.store(static_cast<__half *>(a.to) + at, a.padded - c0);
                if (a.by_column) out.store(static_cast<__half *>(a.by_column) + at, a.padded - c0);
            }
            const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(of_row));
            if (lane == 0) atomicMax(a.row_top + row + k, most);
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

// Half: the rows and columns of `set` rows and 256 columns that need a scale, once more; and what undoes the scales.
template <bool ALIGNED, int ACT>
__device__ __forceinline__ void store_scaled(const AuxJob &a, int64_t row, int c0) {
    const int lane = threadIdx.x & 31, c = c0 + lane * 8, count = static_cast<int>(min(static_cast<int64_t>(a.set), a.rows - row));
    Fv<8> of_column[2];
    bool some = false;
    if (a.by_column && c < a.padded) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint4 *top = reinterpret_cast<const uint4 *>(a.column_top + k * a.padded + c);
            const uint4 lo = top[0], hi = top[1];
            const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            of_column[k] = Fv<8>::make([&](int e) { return gated_scale(w[e]); });
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                some = some || gated_scaled(w[e]);
                if (row == 0) a.column_unscale[k * a.padded + c + e] = gated_unscale(w[e]);
            }
        }
    }
    const bool columns = __any_sync(0xffffffffu, some);
    const uint32_t row_top = a.to && lane < count ? a.row_top[row + lane] : 0;
    const uint32_t of_rows = __ballot_sync(0xffffffffu, gated_scaled(row_top));
    if (c0 == 0 && lane < count) a.row_unscale[row + lane] = gated_unscale(row_top);
    if (!columns && !of_rows) return;
    for (int i = 0; i < count; ++i) {
        const bool this_row = of_rows >> i & 1;
        if (!columns && !this_row) continue;
        const Fv<8> of_row = Fv<8>::all(gated_scale(__shfl_sync(0xffffffffu, row_top, i)));
        SlopeRow<__half> s;
        float d[2][8];
        s.load<ALIGNED>(a, row + i, c0);
        s.slopes<ACT>(d);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Fv<8> v = Fv<8>::make([&](int e) { return d[k][e]; });
            const int64_t at = (row + i) * a.to_row + k * a.padded + c0;
            Strip<__half, 8, 8> out;
            if (this_row) {
                out.v[0] = narrow<__half, 8>(v * of_row);
                out.store(static_cast<__half *>(a.to) + at, a.padded - c0);
            }
            if (some) {
                out.v[0] = narrow<__half, 8>(v * of_column[k]);
                out.store(static_cast<__half *>(a.by_column) + at, a.padded - c0);
            }
        }
    }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kWarps * 32, std::is_same<T, __half>::value ? 4 : 5) gated_operands_kernel(const __grid_constant__ AuxArgs args) {
    pdl_trigger();
    pdl_wait();
    const int64_t step = static_cast<int64_t>(gridDim.x) * kWarps;
    for (int64_t unit = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); unit < args.units; unit += step) {
        int64_t u = unit;
        int j = 0;
        while (u >= args.job[j].units) u -= args.job[j++].units;
        const AuxJob &a = args.job[j];
        const int64_t row = u / a.pieces;
        const int c0 = static_cast<int>(u - row * a.pieces) * kColumns;
        if (j == kJobs - 1) {
            if constexpr (std::is_same<T, __half>::value) {
                if (a.aligned) store_scaled<true, ACT>(a, row * a.set, c0);
                else store_scaled<false, ACT>(a, row * a.set, c0);
            } else {
                if (a.aligned) store_slopes<T, true, ACT>(a, row, c0);
                else store_slopes<T, false, ACT>(a, row, c0);
            }
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
            const bool small = a.units <= static_cast<int64_t>(sm_count()) * 64;
            a.set = small ? 2 : 32;                    // (that all of them need a scale: 777 x 1333, products included, 36 us, with sets of 8 54; that none does: 30 either way)
            a.units = ceil_div(rows, a.set) * a.pieces;
            // rows of a warp: two where there are few (four: 3 us more), else as many as make a column's maxima cheap
            const int of_warp = small ? 2 : 16;
            const dim3 grid(static_cast<unsigned>(ceil_div(rows, kWarps * of_warp) * a.pieces));
            const cudaError_t e = by_act(s.act, [&](auto act) {
                return a.aligned ? launch_pdl(gated_slopes_kernel<true, act.value>, grid, dim3(kWarps * 32), 0, st, 1, a, of_warp)
                                 : launch_pdl(gated_slopes_kernel<false, act.value>, grid, dim3(kWarps * 32), 0, st, 1, a, of_warp);
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

// Elementwise passes of the gated feed-forward block: rows that the tensor-core copies cannot read as they lie are packed, and the gradients
// of both projections are formed from what the forward pass kept:  dg = dh u act'(g), du = dh act(g).
//
// Memory bound.  A warp takes 256 columns of a row, 8 per lane.  dg and du are rounded to the type of the products that read them: their
// errors are independent and average out in the products' sums (2^-9 per term for bf16, against the 2^-9 that the result is rounded by).
#include <algorithm>

#include "feed_forward.hpp"
#include "kernels.hpp"
#include "mx8_device.cuh"

namespace patdnn {
namespace {

constexpr int kWarps = 8, kColumns = 256;

struct AuxArgs {
    const void *x, *dh;
    void *to;
    int64_t rows, row, dh_row, to_row;                 // strides in elements
    int cols, padded, pieces;                          // padded: columns that are written; pieces of 256 of them
};

template <typename T, int A>
__global__ void __launch_bounds__(kWarps * 32) gated_pack_kernel(AuxArgs a) {
    pdl_trigger();
    pdl_wait();
    const int64_t step = static_cast<int64_t>(gridDim.x) * kWarps, units = a.rows * a.pieces;
    for (int64_t u = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); u < units; u += step) {
        const int64_t row = u / a.pieces;
        const int c0 = static_cast<int>(u - row * a.pieces) * kColumns;
        Strip<T, A, 8> s;
        s.load(static_cast<const T *>(a.x) + row * a.row + c0, a.cols - c0);
        s.store(static_cast<T *>(a.to) + row * a.to_row + c0, a.padded - c0);
    }
}

template <typename T, int A, int ACT>
__global__ void __launch_bounds__(kWarps * 32) gated_slopes_kernel(AuxArgs a) {
    pdl_trigger();
    pdl_wait();
    const int64_t step = static_cast<int64_t>(gridDim.x) * kWarps, units = a.rows * a.pieces;
    for (int64_t unit = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5); unit < units; unit += step) {
        const int64_t row = unit / a.pieces;
        const int c0 = static_cast<int>(unit - row * a.pieces) * kColumns, left = a.cols - c0;
        Strip<T, A, 8> sg, su, sd;
        const T *g = static_cast<const T *>(a.x) + row * a.row + c0;
        sg.load(g, left);
        su.load(g + a.cols, left);
        sd.load(static_cast<const T *>(a.dh) + row * a.dh_row + c0, left);
        float fg[8], fu[8], fd[8];
        sg.widen_to(fg);
        su.widen_to(fu);
        sd.widen_to(fd);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float act = fg[e], slope = 1.f;
            if constexpr (ACT == PATDNN_ACT_RELU) {    // slope 0 at 0; a NaN passes
                act = fg[e] < 0.f ? 0.f : fg[e];
                slope = fg[e] > 0.f ? 1.f : fg[e] <= 0.f ? 0.f : fg[e];
            } else if constexpr (ACT == PATDNN_ACT_SILU) {
                const float s = sigmoid(fg[e]);
                act = fg[e] * s;
                slope = fmaf(act, 1.f - s, s);
            }
            fg[e] = fd[e] * fu[e] * slope;
            fu[e] = fd[e] * act;
        }
        sg.narrow_from(fg);
        su.narrow_from(fu);
        T *to = static_cast<T *>(a.to) + row * a.to_row + c0;
        sg.store(to, a.padded - c0);
        su.store(to + a.padded, a.padded - c0);
    }
}

template <typename F> cudaError_t by_half_strip(int dtype, int width, F f) {
    auto go = [&](auto t) {
        if (width == 8) return f(t, std::integral_constant<int, 8>{});
        if (width == 2) return f(t, std::integral_constant<int, 2>{});
        return f(t, std::integral_constant<int, 1>{});
    };
    return dtype == PATDNN_F16 ? go(__half{}) : go(__nv_bfloat16{});
}
dim3 aux_grid(const AuxArgs &a) {
    return dim3(static_cast<unsigned>(std::min<int64_t>(ceil_div(a.rows * a.pieces, kWarps), static_cast<int64_t>(sm_count()) * 32)));
}

}  // namespace

cudaError_t launch_gated_pack(const void *x, int64_t rows, int cols, int64_t row, void *to, int64_t to_row, int dtype, cudaStream_t st) {
    AuxArgs a{};
    a.x = x; a.to = to; a.rows = rows; a.row = row; a.to_row = to_row; a.cols = cols; a.padded = static_cast<int>(to_row);
    a.pieces = static_cast<int>(ceil_div(a.padded, kColumns));
    return by_half_strip(dtype, strip_width(dtype, {x}, {row}), [&](auto t, auto v) {
        return launch_pdl(gated_pack_kernel<decltype(t), v.value>, aux_grid(a), dim3(kWarps * 32), 0, st, 1, a);
    });
}

cudaError_t launch_gated_slopes(const GatedShape &s, const void *gu, const void *dh, void *dgu, int64_t rows, cudaStream_t st) {
    AuxArgs a{};
    a.x = gu; a.dh = dh; a.to = dgu; a.rows = rows; a.row = 2 * static_cast<int64_t>(s.F); a.dh_row = s.h_row;
    a.cols = s.F; a.padded = gated_padded(s.F); a.to_row = 2 * static_cast<int64_t>(a.padded);
    a.pieces = static_cast<int>(ceil_div(a.padded, kColumns));
    return by_half_strip(s.dtype, strip_width(s.dtype, {gu, dh}, {s.F, s.h_row}), [&](auto t, auto v) {
        return by_act(s.act, [&](auto act) {
            return launch_pdl(gated_slopes_kernel<decltype(t), v.value, act.value>, aux_grid(a), dim3(kWarps * 32), 0, st, 1, a);
        });
    });
}

}  // namespace patdnn

// Elementwise work of the gated feed-forward block in front of its products, one launch: rows that the tensor-core copies cannot read as they
// lie are packed, and the gradients of both projections are formed from what the forward pass kept:  dg = dh u act'(g), du = dh act(g).
//
// Memory bound (4096 x 8192 bf16: 46 us for 336 MB, 7.2 TB/s with part of it in L2).  A warp takes 256 columns of a row, 8 per lane.  dg and du are
// rounded to the type of the products that read them: their errors are independent and average out in the products' sums (2^-9 per term for
// bf16, against the 2^-9 that the result is rounded by).
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
    void *to;
    int64_t row, dh_row, to_row;                       // strides in elements
    int64_t units;                                     // rows times pieces
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

template <typename T, bool ALIGNED, int ACT>
__device__ __forceinline__ void slopes(const AuxJob &a, int64_t row, int c0) {
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
    float fg[8], fu[8], fd[8];
    sg.widen_to(fg);
    su.widen_to(fu);
    sd.widen_to(fd);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float act = fg[e], slope = 1.f;
        if constexpr (ACT == PATDNN_ACT_RELU) {        // slope 0 at 0; a NaN passes
            act = fg[e] < 0.f ? 0.f : fg[e];
            slope = fg[e] > 0.f ? 1.f : fg[e] <= 0.f ? 0.f : fg[e];
        } else if constexpr (ACT == PATDNN_ACT_SILU) {
            const float s = sigmoid(fg[e]);            // at infinities (g left the range of the type) the limits: 0 and 0, or g and 1
            act = s == 0.f ? 0.f : fg[e] * s;
            slope = s == 1.f ? 1.f : fmaf(act, 1.f - s, s);
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

template <typename T, int ACT>
__global__ void __launch_bounds__(kWarps * 32) gated_operands_kernel(const __grid_constant__ AuxArgs args) {
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
            if (a.aligned) slopes<T, true, ACT>(a, row, c0);
            else slopes<T, false, ACT>(a, row, c0);
        } else if (a.copies) {
            pack_shifted(a, row, c0);
        } else {
            pack<T>(a, row, c0);
        }
    }
}

}  // namespace

cudaError_t launch_gated_operands(const GatedShape &s, const GatedPack (&packs)[3], const void *gu, const void *dh, void *dgu, int64_t rows, cudaStream_t st) {
    AuxArgs args{};
    for (int i = 0; i < 3; ++i) {
        if (packs[i].rows == 0) continue;
        AuxJob &a = args.job[i];
        a.x = packs[i].from; a.to = packs[i].to; a.row = packs[i].row; a.to_row = packs[i].to_row; a.cols = s.K; a.padded = static_cast<int>(packs[i].to_row);
        a.pieces = static_cast<int>(ceil_div(a.padded, kColumns));
        a.rows = packs[i].rows; a.copies = packs[i].copies;
        std::copy(packs[i].shift, packs[i].shift + kMostPhases, a.shift);
        a.units = packs[i].rows * std::max(1, a.copies) * a.pieces;
    }
    if (dgu) {
        AuxJob &a = args.job[kJobs - 1];
        a.x = gu; a.dh = dh; a.to = dgu; a.row = 2 * static_cast<int64_t>(s.F); a.dh_row = s.h_row;
        a.cols = s.F; a.padded = gated_padded(s.F); a.to_row = 2 * static_cast<int64_t>(a.padded);
        a.pieces = static_cast<int>(ceil_div(a.padded, kColumns));
        a.units = rows * a.pieces;
        a.aligned = strip_width(s.dtype, {gu, dh}, {s.F, s.h_row}) == 8;
    }
    for (const AuxJob &a : args.job) args.units += a.units;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(ceil_div(args.units, kWarps), static_cast<int64_t>(sm_count()) * 32)));
    return by_act(s.act, [&](auto act) {
        return s.dtype == PATDNN_F16 ? launch_pdl(gated_operands_kernel<__half, act.value>, grid, dim3(kWarps * 32), 0, st, 1, args)
                                     : launch_pdl(gated_operands_kernel<__nv_bfloat16, act.value>, grid, dim3(kWarps * 32), 0, st, 1, args);
    });
}

}  // namespace patdnn

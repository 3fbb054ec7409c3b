// Internal interfaces of the feed-forward operators: RMS norm with the residual's addition, 8-bit matrices, the linear layer with 8-bit
// weights, and the gated block.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "ops.hpp"

namespace patdnn {

// ---- 8-bit blocks (mx8.cu) ---------------------------------------------------------------------------------------------
// A matrix of R rows and K columns is cut into tiles of 128 rows by 128 columns.  All code tiles come first ([row tile][column tile]),
// 128 rows of 128 bytes each; inside a tile the 16-byte unit u of row r sits at unit u ^ (r & 7), the order in which the tensor cores
// read it from shared memory, so that a tile is ONE contiguous copy.  Then the scales: per row tile and FOUR column tiles 512 bytes,
// the scale byte of (row r, column tile t) at (r % 32) * 16 + (r / 32) * 4 + t % 4, the order in which they are copied to tensor memory.
struct Mx8Shape {
    int64_t rows, cols;
    int64_t row_tiles, col_tiles, groups;   // groups: of four column tiles
    int64_t scales_at, bytes;               // offset of the scales; size of the whole buffer
};
constexpr int kMx8Tile = 128 * 128, kMx8Scales = 512;
inline Mx8Shape mx8_shape(int64_t rows, int64_t cols) {
    Mx8Shape m{};
    m.rows = rows; m.cols = cols;
    m.row_tiles = ceil_div(rows, 128);
    m.col_tiles = ceil_div(cols, 128);
    m.groups = ceil_div(m.col_tiles, 4);
    m.scales_at = m.row_tiles * m.col_tiles * kMx8Tile;
    m.bytes = m.scales_at + m.row_tiles * m.groups * kMx8Scales;
    return m;
}
cudaError_t launch_mx8_quantize(const Mx8Shape &m, const void *x, int dtype, int64_t ld, void *mx, cudaStream_t st);
cudaError_t launch_mx8_dequantize(const Mx8Shape &m, const void *mx, void *out, int dtype, int64_t ld, cudaStream_t st);

// CTAs in clusters of `size` that run at a time, one to an SM: a cluster lies inside one group of SMs, and the groups are no multiples of four or
// eight (148 SMs: 132 and 120 CTAs).  More would wait for a second wave.
inline int cluster_room(int sms, int size) { return size <= 2 ? sms : size == 4 ? sms - sms / 9 : sms * 13 / 16; }

// ---- 8-bit product (mx8_linear.cu) --------------------------------------------------------------------------------------
struct Mx8Params {
    const uint8_t *w, *x;                   // 8-bit matrices [F][K], [rows][K] in the layout above
    const void *x_raw;                      // or (x == nullptr) at most kFusedRows rows of x as they are, ldx elements apart
    int64_t ldx, K;
    const float *bias;                      // [F] or nullptr
    void *y;
    int *status;
    int64_t ldy, rows;
    int64_t w_scales, x_scales;             // offsets of the scales
    int F, col_tiles, groups, ksteps;       // groups of four column tiles; ksteps: K-steps of 32 columns that hold data
    int act, dtype;
    int f_tiles, n_tiles;                   // tiles of rows of w; of rows of x
    int tile_n;                             // rows of the N operand in a tile
    int splits, tiles_per_split;            // cluster split of the column tiles
    int stages;
    int band;                               // pairs of CTAs: tiles of rows of w to a band
    int tensor_columns;                     // of tensor memory that a CTA allocates
    uint32_t spin_limit;                    // polls of a bounded wait (0 = the default)
    int test_skip_load;                     // test hook: every CTA leaves out the copies of this (1-based) column tile of its walk (0 = off)
};
using Mx8Launch = Mx4Launch;               // persistent: pairs of CTAs
cudaError_t prepare_mx8_linear();                       // opt in to the dynamic shared memory
Mx8Launch plan_mx8_linear(Mx8Params &p);                // shapes of p (F, K, rows, x_raw) -> its tiling and the launch; no device is touched
cudaError_t launch_mx8_linear(Mx8Params p, cudaStream_t st, int *launches);

// ---- RMS norm (rms_norm.cu) --------------------------------------------------------------------------------------------
constexpr int kRmsMostColumns = 1 << 16;    // a row is held in the registers of at most eight CTAs
struct RmsShape {
    int C, dtype;
    float eps;
    int64_t x_row, r_row, y_row;            // strides in elements
};
struct RmsWait {                            // of the clusters that share a row
    int *status;
    uint32_t spin_limit;                    // polls of a bounded wait (0 = the default)
    int test_skip;                          // test hook: the first CTA of every cluster waits for a value too many at this (1-based) sum over a row of its walk (0 = off)
};
struct RmsCall {
    const void *x, *residual;               // residual may be nullptr
    const float *gamma;
    void *sum, *y, *mx;                     // sum, and one of y and mx, may be nullptr
    float *rstd;                            // may be nullptr
    int64_t rows;
    RmsWait wait;
};
cudaError_t launch_rms_norm(const RmsShape &s, const RmsCall &c, cudaStream_t st);
struct RmsGradCall {
    const void *s, *dy, *dsum;              // dsum may be nullptr
    const float *gamma, *rstd;
    void *dx;
    float *dgamma, *ws;
    int64_t rows;
    RmsWait wait;
};
cudaError_t prepare_rms();                  // opt in to the dynamic shared memory
size_t rms_workspace_floats(const RmsShape &s);
cudaError_t launch_rms_grad(const RmsShape &s, const RmsGradCall &c, cudaStream_t st, int *launches);

// ---- gated feed-forward block (gated.cu, gated_aux.cu) ---------------------------------------------------------------------
struct GatedShape {
    int F, K, act, dtype;                   // dtype: F16 or BF16
    int64_t x_row, w_row, h_row;            // strides in elements
};
struct GatedPlan {
    int m_tiles, n_tiles;                   // tiles of 256 rows, and of 256 columns of the product (forward: 128 outputs, gate and up)
    int k_blocks, splits, per_split;        // blocks of 64 along the summed dimension; ranges of them that share a tile; blocks of a range
    int grid, stages, smem;                 // CTAs; blocks in the ring of copies; dynamic shared memory
    int tensor_columns;                     // of tensor memory that a CTA allocates
    bool few;                               // forward, few rows: n_tiles of 64 outputs, tiles of tile_n rows, splits in a cluster
    int tile_n;
};
GatedPlan plan_gated_forward(int F, int K, int64_t rows);
// Few rows, weights whose rows are not whole 16-byte units apart, read as they lie (see gated_rows_kernel): every `phases`-th row begins at the same place
// of a unit.
constexpr int kMostPhases = 8, kPhasedRows = 128;
inline int gated_phases(int64_t w_row) { return w_row % 8 == 0 ? 1 : w_row % 4 == 0 ? 2 : w_row % 2 == 0 ? 4 : 8; }
inline int gated_phased_row(int K) { return (K + kMostPhases - 1 + 7) / 8 * 8; }       // of a shifted copy of x
GatedPlan plan_gated_phased(int F, int K, int64_t rows, int phases);
// [0] dx, [1] dwg and dwu; one launch, whose grid both have
void plan_gated_gradient(int F, int K, int64_t rows, bool dx, bool dw, GatedPlan (&plan)[2]);
constexpr int kGatedUnitFloats = 256 * 256; // partial sums of a (tile, split) unit
constexpr int kGatedUnits = 2;              // such units that a call may need, per pair of SMs (see plan_gated_gradient)
struct GatedWork {                          // a handle's buffers
    void *dgu;                              // [max_rows][2 Fp]: dg, du in the handle's type, Fp = F rounded up to 64; nullptr without gradients
    void *by_column;                        // half: a copy for dwg and dwu (see gated_aux.cu); else nullptr
    uint32_t *row_top, *column_top;         // half: bits of the largest magnitudes, [max_rows] and [2 Fp], in one buffer, zeros between calls
    float *row_unscale, *column_unscale;    // half: what undoes the scales, likewise
    float *partial;
    int *status;
};
inline int gated_padded(int F) { return (F + 63) / 64 * 64; }
struct GatedCall {
    const void *x, *wg, *wu;                // rows 16-byte aligned, x_row / w_row apart
    int64_t x_row, w_row;                   // of these (not of the outputs)
    void *h, *gu;                           // forward; gu may be nullptr
    void *dx, *dwg, *dwu;
    int64_t rows;
    int phases;                             // 0, or forward: wg and wu as the caller's, x a copy per phase, shifted as its rows of the weights are
    uint32_t spin_limit;
    int test_skip_load;
};
int pairs_most();                           // pairs of CTAs that run at a time
cudaError_t prepare_gated();
cudaError_t launch_gated_forward(const GatedShape &s, const GatedCall &c, const GatedWork &w, cudaStream_t st, int *launches);
cudaError_t launch_gated_gradient(const GatedShape &s, const GatedCall &c, const GatedWork &w, cudaStream_t st, int *launches);   // from dgu
// In front of them: K columns of 16-bit rows to rows `to_row` apart, zeros behind them (rows = 0: nothing to pack), and, where there are slopes, dg and du from
// gu [rows][2 F] and dh
// copies > 0: as many copies of all rows, copy i shifted by shift[i] columns, zeros in front
struct GatedPack {
    const void *from;
    void *to;
    int64_t rows, row, to_row;
    int copies;
    uint8_t shift[kMostPhases];
};
inline int gated_shift(const void *base, int64_t w_row, int phase) {                   // elements between a row and the 16-byte unit in which it begins
    return static_cast<int>((reinterpret_cast<uintptr_t>(base) + static_cast<uintptr_t>(phase) * w_row * 2) % 16 / 2);
}
struct GatedSlopes {
    const void *gu, *dh;
    void *dgu, *by_column;                  // half: either may be nullptr
    uint32_t *row_top, *column_top;         // half
    float *row_unscale, *column_unscale;
};
cudaError_t launch_gated_operands(const GatedShape &s, const GatedPack (&packs)[3], const GatedSlopes *slopes, int64_t rows, cudaStream_t st, int *launches);
// Half: whether magnitudes whose largest has these bits are scaled, the power of two that brings it between 2^14 and 2^15, and what undoes it.  (Magnitudes below
// 2^-100, whose gradients are below half's range whatever they are multiplied with, are taken as 2^-100, so that both factors are normal.)
__device__ __forceinline__ bool gated_scaled(uint32_t top) {
    constexpr uint32_t kLeast = (127 - 3) << 23, kMost = (127 + 15) << 23, kInfinity = 0x7f800000u;
    return (top - 1 < kLeast - 1) || (top >= kMost && top < kInfinity);
}
__device__ __forceinline__ uint32_t gated_top_field(uint32_t top) { return max(top >> 23, 27u); }
__device__ __forceinline__ float gated_scale(uint32_t top) { return gated_scaled(top) ? __uint_as_float((254 + 14 - gated_top_field(top)) << 23) : 1.f; }
__device__ __forceinline__ float gated_unscale(uint32_t top) { return gated_scaled(top) ? __uint_as_float((gated_top_field(top) - 14) << 23) : 1.f; }

}  // namespace patdnn

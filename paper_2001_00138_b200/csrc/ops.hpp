// Internal interfaces of the operators around the convolutions: group norm (channels last) and the 4-bit linear layer.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace patdnn {

// defined in api.cu, shared by every file with C entry points
int cuda_fail(cudaError_t e, const char *what);      // records the text for patdnn_last_cuda_error, returns PATDNN_E_CUDA
void count_launches(int n);                          // patdnn_launch_count

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int elem_bytes(int dtype) { return dtype == 0 ? 4 : 2; }   // PATDNN_F32 = 0; F16 and BF16 have two bytes

// ---- group norm (group_norm.cu) ---------------------------------------------------------------------------------------
struct NormShape {
    int N, C, G, act, dtype;
    int64_t P;                              // pixels per image
    int64_t x_pixel, x_image, y_pixel, y_image;   // strides in elements; a pixel's channels are consecutive
    float eps;
};
struct NormPlan {
    bool resident = false;                  // one launch: the slab of an image stays in the shared memory of a cluster
    int slab = 0, slabs = 0;                // channels per slab (whole groups when resident), slabs = ceil(C / slab)
    int cluster = 1;                        // resident: CTAs that share one (image, slab)
    int chunks = 1;                         // two passes: pixel chunks per image
    int parts = 1;                          // two passes: slabs that share a group wider than a CTA
    int run = 1;                            // two passes: images taken together
    int64_t chunk = 0;                      // pixels per CTA
    int smem = 0;                           // resident: dynamic shared memory
};
constexpr int kNormWidths = 3;              // a handle is planned for accesses of 16 bytes, 2 elements and 1 element
struct NormHandle {
    NormShape s{};
    NormPlan fwd[kNormWidths], mx4[kNormWidths], bwd[kNormWidths];
    float *ws = nullptr;                    // partial sums of the two-pass forms and of the gradient
    unsigned *counters = nullptr;           // [G] arrivals of images per channel slab (there are at most G); zero between calls
    float *stats = nullptr;                 // [N][G][2] where the caller keeps none
};
int norm_width(int dtype, int index);       // elements per access for width index 0 .. 2
void plan_norm(NormHandle &h);
size_t norm_workspace_floats(const NormHandle &h);
cudaError_t prepare_norm();                 // opt in to the dynamic shared memory
// stats may be nullptr
cudaError_t launch_group_norm(const NormHandle &h, const void *x, const float *gamma, const float *beta, void *y, float *stats,
                              cudaStream_t st, int *launches);
// the same as rows of a 4-bit matrix (image * P + pixel)
cudaError_t launch_group_norm_mx4(const NormHandle &h, const void *x, const float *gamma, const float *beta, void *mx, float *stats,
                                  cudaStream_t st, int *launches);
cudaError_t launch_group_norm_grad(const NormHandle &h, const void *x, const float *gamma, const float *beta, const float *stats,
                                   const void *dy, void *dx, float *dgamma, float *dbeta, cudaStream_t st, int *launches);

// ---- 4-bit blocks (mx4.cu) --------------------------------------------------------------------------------------------
// A matrix of R rows and K columns is cut into tiles of 128 rows by `width` columns.  All code tiles come first
// ([row tile][column tile]), 128 rows of width/2 bytes each, two codes per byte, the lower column in the lower half; inside a tile
// the 16-byte unit at offset o sits at o ^ (((o >> 7) & (width/32 - 1)) << 4), the order in which the tensor cores read it from
// shared memory, so that a tile is ONE contiguous copy.  Then all scale tiles: per 128 columns 512 bytes, the scale byte of
// (row r, block b) at (r % 32) * 16 + (r / 32) * 4 + b % 4, the order in which they are copied to tensor memory.
struct Mx4Shape {
    int64_t rows, cols;
    int width;                              // columns of a tile: 64, 128 or 256
    int64_t row_tiles, col_tiles;
    int code_bytes, scale_bytes;            // of one tile
    int64_t scales_at, bytes;               // offset of the scale tiles; size of the whole buffer
};
inline Mx4Shape mx4_shape(int64_t rows, int64_t cols) {
    Mx4Shape m{};
    m.rows = rows; m.cols = cols;
    m.width = cols <= 64 ? 64 : cols <= 128 ? 128 : 256;   // a narrow matrix is not padded to the full width
    m.row_tiles = ceil_div(rows, 128);
    m.col_tiles = ceil_div(cols, m.width);
    m.code_bytes = 64 * m.width;
    m.scale_bytes = m.width > 128 ? 1024 : 512;
    m.scales_at = m.row_tiles * m.col_tiles * m.code_bytes;
    m.bytes = m.scales_at + m.row_tiles * m.col_tiles * m.scale_bytes;
    return m;
}
cudaError_t launch_mx4_quantize(const Mx4Shape &m, const void *x, int dtype, int64_t ld, void *mx, cudaStream_t st);
cudaError_t launch_mx4_dequantize(const Mx4Shape &m, const void *mx, void *out, int dtype, int64_t ld, cudaStream_t st);
// act((x - mean) * rstd * gamma + beta) of the pixels of rows [row0, row0 + rows), row = image * P + pixel; m: the whole matrix
cudaError_t launch_norm_quantize(const NormShape &s, const Mx4Shape &m, const void *x, const float *gamma, const float *beta,
                                 const float *stats, int64_t row0, int64_t rows, void *mx, cudaStream_t st);

// ---- 4-bit product (mx4_linear.cu) ------------------------------------------------------------------------------------
struct Mx4Params {
    const uint8_t *w, *x;                   // 4-bit matrices [F][K], [rows][K] in the layout above
    const void *x_raw;                      // or (x == nullptr) at most kFusedRows rows of x as they are, ldx elements apart
    int64_t ldx, K;
    const float *bias;                      // [F] or nullptr
    void *y;
    int *status;
    int64_t ldy, rows;
    int64_t w_scales, x_scales;             // offsets of the scale tiles
    int F, width, col_tiles, ksteps;        // ksteps: K-steps of 64 columns that hold data, over all column tiles
    int act, dtype;
    int f_tiles, n_tiles;                   // tiles of 128 rows of w; of `tile_n` rows of x
    int tile_n;
    int splits, tiles_per_split;            // cluster split of the column tiles
    int stages;
    int tensor_columns;                     // of tensor memory that a CTA allocates
    int step_n, step_f;                     // persistent kernel: from a CTA's tile to its next one
    uint32_t spin_limit;                    // polls of a bounded wait (0 = the default)
    int test_skip_load;                     // test hook: every CTA leaves out the copies of this (1-based) column tile of its walk (0 = off)
};
struct Mx4Launch {                          // how a product is launched
    bool persistent;                        // the kernel for many rows
    int piece;                              // persistent: bytes of a row of y that are stored at a time
    int smem;                               // dynamic shared memory
    unsigned grid;
};
constexpr int kFusedRows = 8;               // rows that the product's kernel quantises itself
cudaError_t prepare_mx4_linear();                       // opt in to the dynamic shared memory
// Shapes of p (F, K, rows, x_raw) -> its tiling and the launch; no device is touched.
Mx4Launch plan_mx4_linear(Mx4Params &p);
cudaError_t launch_mx4_linear(Mx4Params p, cudaStream_t st, int *launches);

}  // namespace patdnn

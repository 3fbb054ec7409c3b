// C entry points of the RMS norm, the 8-bit matrices, the linear layer with 8-bit weights and the gated block (declared in include/patdnn.h).
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>

#include "../../include/patdnn.h"
#include "feed_forward.hpp"

using namespace patdnn;

#define CU(call)                                             \
    do {                                                     \
        cudaError_t e_ = (call);                             \
        if (e_ != cudaSuccess) return cuda_fail(e_, #call);  \
    } while (0)

struct patdnn_rms_s {
    RmsShape s{};
    int device = -1;
    float *ws = nullptr;                    // the gradient's partial sums, and behind them
    int *status = nullptr;
    uint32_t spin_limit = 0;                // patdnn_rms_debug_wait
    int test_skip = 0;
    RmsWait wait() const { return {status, spin_limit, test_skip}; }
    ~patdnn_rms_s() { cudaFree(ws); }
};

struct patdnn_linear8_s {
    patdnn_linear_desc d{};
    Mx8Shape shape{};                       // of the weights
    int device = -1;
    uint8_t *w = nullptr, *x = nullptr;     // 8-bit weights; buffer for the rows of patdnn_linear8_run where max_rows is above kFusedRows
    float *bias = nullptr;
    int *status = nullptr;
    uint32_t spin_limit = 0;                // patdnn_linear8_debug_wait
    int test_skip_load = 0;
    ~patdnn_linear8_s() {
        cudaFree(w);
        cudaFree(x);
        cudaFree(bias);
        cudaFree(status);
    }
};

struct patdnn_gated_s {
    GatedShape s{};
    GatedWork w{};
    int64_t max_rows = 0;
    int device = -1;
    void *x = nullptr, *weights = nullptr;  // packed rows, where theirs cannot be copied as they lie
    void *shifted = nullptr;                // copies of few rows of x, beside `weights`
    uint32_t spin_limit = 0;                // patdnn_gated_debug_wait
    int test_skip_load = 0;
    ~patdnn_gated_s() {
        cudaFree(w.dgu);
        cudaFree(w.row_top);
        cudaFree(w.partial);
        cudaFree(w.status);
        cudaFree(x);
        cudaFree(weights);
        cudaFree(shifted);
    }
};

namespace {

constexpr int64_t kMostColumns = int64_t(1) << 20;
constexpr int64_t kMostElements = int64_t(1) << 40;

bool known_type(int dtype) { return dtype == PATDNN_F32 || dtype == PATDNN_F16 || dtype == PATDNN_BF16; }
bool known_act(int act) { return act == PATDNN_ACT_NONE || act == PATDNN_ACT_RELU || act == PATDNN_ACT_SILU; }
bool size_ok(int64_t rows, int64_t cols) {
    return rows >= 0 && cols >= 1 && cols <= kMostColumns && rows <= kMostElements / cols && rows <= INT32_MAX;
}
bool aligned(const void *p, unsigned bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
bool elements_aligned(const void *p, int dtype) { return aligned(p, static_cast<unsigned>(elem_bytes(dtype))); }

// A handle's buffers belong to the device that was current when it was made.
int on_device(int device) {
    int now = -1;
    CU(cudaGetDevice(&now));
    return now == device ? PATDNN_OK : PATDNN_E_NO_DEVICE;
}

int launched(cudaError_t e, int n, const char *what) {
    if (e != cudaSuccess) return cuda_fail(e, what);
    count_launches(n);
    return PATDNN_OK;
}

template <typename T> cudaError_t allocate(T **p, size_t count) {
    void *v = nullptr;
    const cudaError_t e = cudaMalloc(&v, std::max<size_t>(16, count * sizeof(T)));
    *p = static_cast<T *>(v);
    return e;
}

template <typename H> int failed(H *h, cudaError_t e, const char *what) {
    const int rc = cuda_fail(e, what);
    delete h;
    return rc;
}

bool too_many_tiles(int64_t rows, int64_t F) { return ceil_div(rows, 128) * ceil_div(F, 128) > INT32_MAX / 8; }   // CTAs of one launch

// Waits for the device, reports a bounded wait that ran out and clears the word.
int check_status(int device, int *status) {
    if (const int rc = on_device(device)) return rc;
    CU(cudaDeviceSynchronize());
    int word = 0;
    CU(cudaMemcpy(&word, status, sizeof(int), cudaMemcpyDeviceToHost));
    if (!word) return PATDNN_OK;
    CU(cudaMemset(status, 0, sizeof(int)));
    return PATDNN_E_DEVICE_TIMEOUT;
}

// mx: 8-bit rows, or nullptr with the rows themselves at x
int product(patdnn_linear8 h, const void *mx, const void *x, int64_t ldx, int64_t rows, void *y, int64_t ldy, cudaStream_t st) {
    if (too_many_tiles(rows, h->d.F)) return PATDNN_E_SHAPE;
    Mx8Params p{};
    p.w = h->w; p.x = static_cast<const uint8_t *>(mx); p.x_raw = x; p.ldx = ldx; p.K = h->d.K; p.bias = h->bias; p.y = y; p.status = h->status;
    p.ldy = ldy; p.rows = rows; p.w_scales = h->shape.scales_at; p.x_scales = mx8_shape(rows, h->d.K).scales_at;
    p.spin_limit = h->spin_limit; p.test_skip_load = h->test_skip_load;
    p.F = h->d.F; p.act = h->d.act; p.dtype = h->d.dtype;
    int n = 0;
    const cudaError_t e = launch_mx8_linear(p, st, &n);
    return launched(e, n, "8-bit product launch");
}

// What patdnn_rms_run and patdnn_rms_run_mx8 refuse; 0 where there is something to do, -1 where there are no rows.
int rms_forward(patdnn_rms h, const void *x, const void *residual, const float *gamma, void *sum, void *out, bool mx, float *rstd, int64_t rows,
                cudaStream_t st) {
    if (!h) return PATDNN_E_NULL;
    const RmsShape &s = h->s;
    if (!size_ok(rows, s.C) || !elements_aligned(x, s.dtype) || !elements_aligned(residual, s.dtype) || !elements_aligned(sum, s.dtype) ||
        !(mx ? aligned(out, 16) : elements_aligned(out, s.dtype)) || !aligned(gamma, 4) || !aligned(rstd, 4))
        return PATDNN_E_SHAPE;
    if (rows == 0) return PATDNN_OK;
    if (!x || !gamma || !out) return PATDNN_E_NULL;
    if (const int rc = on_device(h->device)) return rc;
    RmsCall c{};
    c.x = x; c.residual = residual; c.gamma = gamma; c.sum = sum; c.rstd = rstd; c.rows = rows; c.wait = h->wait();
    (mx ? c.mx : c.y) = out;
    return launched(launch_rms_norm(s, c, st), 1, "RMS norm launch");
}

// The gated block's tiles: 256 rows by 128 outputs, or 256 columns.
bool gated_too_large(int64_t rows, int64_t F, int64_t K) {
    return ceil_div(rows, 256) * ceil_div(std::max(F, K), 128) > INT32_MAX / 8 || 2 * ceil_div(F, 256) * ceil_div(K, 256) > INT32_MAX / 8;
}
bool copies_as_it_lies(int64_t row) { return row % 8 == 0; }           // rows of whole 16-byte units
bool operand_aligned(const void *p, int64_t row) { return aligned(p, copies_as_it_lies(row) ? 16 : 2); }
int64_t packed_row(int64_t K) { return (K + 7) / 8 * 8; }

// Few rows, weights whose rows are not whole 16-byte units apart: a copy of x per phase instead of packed weights, as long as those are fewer rows (8 x 6899 ->
// 4222: 25 us, 79 packed; 128 x 1001 -> 1001: 9.9 and 10.2; 128 x 6899 -> 700: 25.5 and 20.2).  0: not this way; else the phases.
int phases_of(int F, int K, int64_t w_row, int64_t rows) {
    const int phases = gated_phases(w_row);
    return phases > 1 && rows <= kPhasedRows && phases <= F && K + kMostPhases <= phases * w_row && phases * rows <= F ? phases : 0;
}

// x and the weights of a call as the products read them (those that read_x and read_w name): packed first, where they cannot be copied as they lie.
// slopes: the gradient's; or nullptr
int gated_operands(patdnn_gated h, const void *x, const void *wg, const void *wu, const GatedSlopes *slopes, int64_t rows, bool read_x, bool read_w, GatedCall &c, cudaStream_t st) {
    const GatedShape &s = h->s;
    c.x = x; c.wg = wg; c.wu = wu; c.x_row = s.x_row; c.w_row = s.w_row; c.rows = rows;
    c.spin_limit = h->spin_limit; c.test_skip_load = h->test_skip_load;
    const int64_t row = packed_row(s.K);
    GatedPack packs[3] = {};
    int n = 0;
    cudaError_t e;
    const int phases = slopes ? 0 : phases_of(s.F, s.K, s.w_row, rows);
    if (phases && gated_shift(wg, s.w_row, 0) == gated_shift(wu, s.w_row, 0)) {
        packs[0] = {x, h->shifted, rows, s.x_row, gated_phased_row(s.K), phases, {}};
        for (int j = 0; j < phases; ++j) packs[0].shift[j] = static_cast<uint8_t>(gated_shift(wg, s.w_row, j));
        c.x = h->shifted;
        c.x_row = gated_phased_row(s.K);
        c.phases = phases;
        e = launch_gated_operands(s, packs, nullptr, rows, st, &n);
        return launched(e, n, "gated block operands launch");
    }
    if (h->x && read_x) {
        packs[0] = {x, h->x, rows, s.x_row, row, 0, {}};
        c.x = h->x;
        c.x_row = row;
    }
    if (h->weights && read_w) {
        void *second = static_cast<uint16_t *>(h->weights) + s.F * row;
        packs[1] = {wg, h->weights, s.F, s.w_row, row, 0, {}};
        packs[2] = {wu, second, s.F, s.w_row, row, 0, {}};
        c.wg = h->weights;
        c.wu = second;
        c.w_row = row;
    }
    if (!h->x && !h->weights && !slopes) return PATDNN_OK;
    e = launch_gated_operands(s, packs, slopes, rows, st, &n);
    return launched(e, n, "gated block operands launch");
}

}  // namespace

extern "C" {

int patdnn_rms_create(const patdnn_rms_desc *desc, patdnn_rms *out) {
    if (!desc || !out) return PATDNN_E_NULL;
    if (!known_type(desc->dtype)) return PATDNN_E_DTYPE;
    if (desc->C < 1 || desc->C > kRmsMostColumns || !std::isfinite(desc->eps) || desc->eps < 0.f) return PATDNN_E_SHAPE;
    RmsShape s{};
    s.C = desc->C; s.dtype = desc->dtype; s.eps = desc->eps;
    const int64_t rows[3] = {desc->x_row, desc->r_row, desc->y_row};
    int64_t *to[3] = {&s.x_row, &s.r_row, &s.y_row};
    for (int i = 0; i < 3; ++i) {
        *to[i] = rows[i] == 0 ? s.C : rows[i];
        if (*to[i] < s.C || *to[i] > (int64_t(1) << 31)) return PATDNN_E_SHAPE;
    }
    patdnn_rms h = new (std::nothrow) patdnn_rms_s();
    if (!h) return PATDNN_E_ALLOC;
    h->s = s;
    cudaError_t e = cudaGetDevice(&h->device);
    const size_t floats = rms_workspace_floats(s);
    if (e == cudaSuccess) e = allocate(&h->ws, floats + 4);
    h->status = reinterpret_cast<int *>(h->ws + floats);
    if (e == cudaSuccess) e = cudaMemset(h->status, 0, 16);             // (kernels write the word only after seconds of waiting, nothing reads it but patdnn_rms_check)
    if (e == cudaSuccess) e = prepare_rms();
    if (e != cudaSuccess) return failed(h, e, "patdnn_rms_create");
    *out = h;
    return PATDNN_OK;
}

int patdnn_rms_run(patdnn_rms h, const void *x, const void *residual, const float *gamma, void *sum, void *y, float *rstd, int64_t rows, void *stream) {
    return rms_forward(h, x, residual, gamma, sum, y, false, rstd, rows, static_cast<cudaStream_t>(stream));
}

int patdnn_rms_run_mx8(patdnn_rms h, const void *x, const void *residual, const float *gamma, void *sum, void *mx, float *rstd, int64_t rows,
                       void *stream) {
    return rms_forward(h, x, residual, gamma, sum, mx, true, rstd, rows, static_cast<cudaStream_t>(stream));
}

int patdnn_rms_grad(patdnn_rms h, const void *s, const float *gamma, const float *rstd, const void *dy, const void *dsum, void *dx, float *dgamma,
                    int64_t rows, void *stream) {
    if (!h || !dgamma) return PATDNN_E_NULL;
    const int dtype = h->s.dtype;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!size_ok(rows, h->s.C) || !elements_aligned(s, dtype) || !elements_aligned(dy, dtype) || !elements_aligned(dsum, dtype) ||
        !elements_aligned(dx, dtype) || !aligned(gamma, 4) || !aligned(rstd, 4) || !aligned(dgamma, 4))
        return PATDNN_E_SHAPE;
    if (rows > 0 && (!s || !gamma || !rstd || !dy || !dx)) return PATDNN_E_NULL;
    if (const int rc = on_device(h->device)) return rc;
    if (rows == 0) {
        CU(cudaMemsetAsync(dgamma, 0, sizeof(float) * h->s.C, st));
        return PATDNN_OK;
    }
    RmsGradCall c{};
    c.s = s; c.dy = dy; c.dsum = dsum; c.gamma = gamma; c.rstd = rstd; c.dx = dx; c.dgamma = dgamma; c.ws = h->ws; c.rows = rows;
    c.wait = h->wait();
    int n = 0;
    const cudaError_t e = launch_rms_grad(h->s, c, st, &n);
    return launched(e, n, "RMS norm gradient launch");
}

int patdnn_rms_check(patdnn_rms h) {
    return h ? check_status(h->device, h->status) : PATDNN_E_NULL;
}

int patdnn_rms_debug_wait(patdnn_rms h, uint32_t polls, int32_t skip_sum) {
    if (!h) return PATDNN_E_NULL;
    if (skip_sum < 0) return PATDNN_E_SHAPE;
    h->spin_limit = polls;
    h->test_skip = skip_sum;
    return PATDNN_OK;
}

int patdnn_rms_free(patdnn_rms h) {
    delete h;
    return PATDNN_OK;
}

int patdnn_mx8_bytes(int64_t rows, int64_t cols, int64_t *bytes) {
    if (!bytes) return PATDNN_E_NULL;
    if (!size_ok(rows, cols)) return PATDNN_E_SHAPE;
    *bytes = mx8_shape(rows, cols).bytes;
    return PATDNN_OK;
}

int patdnn_mx8_quantize(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, void *mx, void *stream) {
    if (!known_type(dtype)) return PATDNN_E_DTYPE;
    if (!size_ok(rows, cols)) return PATDNN_E_SHAPE;
    if (ld == 0) ld = cols;
    if (ld < cols || !aligned(mx, 16) || !elements_aligned(x, dtype)) return PATDNN_E_SHAPE;
    if (rows == 0) return PATDNN_OK;
    if (!x || !mx) return PATDNN_E_NULL;
    return launched(launch_mx8_quantize(mx8_shape(rows, cols), x, dtype, ld, mx, static_cast<cudaStream_t>(stream)), 1, "8-bit quantisation launch");
}

int patdnn_mx8_dequantize(const void *mx, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, void *out, void *stream) {
    if (!known_type(dtype)) return PATDNN_E_DTYPE;
    if (!size_ok(rows, cols)) return PATDNN_E_SHAPE;
    if (ld == 0) ld = cols;
    if (ld < cols || !aligned(mx, 16) || !elements_aligned(out, dtype)) return PATDNN_E_SHAPE;
    if (rows == 0) return PATDNN_OK;
    if (!out || !mx) return PATDNN_E_NULL;
    return launched(launch_mx8_dequantize(mx8_shape(rows, cols), mx, out, dtype, ld, static_cast<cudaStream_t>(stream)), 1, "8-bit read-back launch");
}

int patdnn_linear8_encode(const void *weights, int64_t ldw, const patdnn_linear_desc *desc, void *stream, patdnn_linear8 *out) {
    if (!weights || !desc || !out) return PATDNN_E_NULL;
    if (!known_type(desc->dtype) || !known_act(desc->act)) return PATDNN_E_DTYPE;
    if (desc->F < 1 || !size_ok(desc->F, desc->K) || desc->F > kMostColumns || !size_ok(desc->max_rows, desc->K)) return PATDNN_E_SHAPE;
    if (ldw == 0) ldw = desc->K;
    if (ldw < desc->K || !elements_aligned(weights, desc->dtype) || !aligned(desc->bias, 4)) return PATDNN_E_SHAPE;
    patdnn_linear8 h = new (std::nothrow) patdnn_linear8_s();
    if (!h) return PATDNN_E_ALLOC;
    h->d = *desc;
    h->d.bias = nullptr;
    h->shape = mx8_shape(desc->F, desc->K);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = allocate(&h->w, static_cast<size_t>(h->shape.bytes));
    if (e == cudaSuccess && desc->max_rows > kFusedRows) e = allocate(&h->x, static_cast<size_t>(mx8_shape(desc->max_rows, desc->K).bytes));
    if (e == cudaSuccess) e = allocate(&h->status, 4);
    if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, 16, st);
    if (e == cudaSuccess && desc->bias) {
        e = allocate(&h->bias, static_cast<size_t>(desc->F));
        if (e == cudaSuccess) e = cudaMemcpyAsync(h->bias, desc->bias, sizeof(float) * desc->F, cudaMemcpyDeviceToDevice, st);
    }
    if (e == cudaSuccess) e = prepare_mx8_linear();
    if (e == cudaSuccess) e = launch_mx8_quantize(h->shape, weights, desc->dtype, ldw, h->w, st);
    if (e == cudaSuccess) {
        count_launches(1);
        e = cudaStreamSynchronize(st);
    }
    if (e != cudaSuccess) return failed(h, e, "patdnn_linear8_encode");
    *out = h;
    return PATDNN_OK;
}

int patdnn_linear8_run(patdnn_linear8 h, const void *x, int64_t rows, int64_t ldx, void *y, int64_t ldy, void *stream) {
    if (!h) return PATDNN_E_NULL;
    if (ldx == 0) ldx = h->d.K;
    if (ldy == 0) ldy = h->d.F;
    if (rows < 0 || rows > h->d.max_rows || ldx < h->d.K || ldy < h->d.F || !elements_aligned(x, h->d.dtype) || !elements_aligned(y, h->d.dtype))
        return PATDNN_E_SHAPE;
    if (rows == 0) return PATDNN_OK;
    if (!x || !y) return PATDNN_E_NULL;
    if (const int rc = on_device(h->device)) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows <= kFusedRows) return product(h, nullptr, x, ldx, rows, y, ldy, st);
    const int rc = launched(launch_mx8_quantize(mx8_shape(rows, h->d.K), x, h->d.dtype, ldx, h->x, st), 1, "8-bit quantisation launch");
    return rc ? rc : product(h, h->x, nullptr, 0, rows, y, ldy, st);
}

int patdnn_linear8_run_mx8(patdnn_linear8 h, const void *mx, int64_t rows, void *y, int64_t ldy, void *stream) {
    if (!h) return PATDNN_E_NULL;
    if (ldy == 0) ldy = h->d.F;
    if (!size_ok(rows, h->d.K) || ldy < h->d.F || !aligned(mx, 16) || !elements_aligned(y, h->d.dtype)) return PATDNN_E_SHAPE;
    if (rows == 0) return PATDNN_OK;
    if (!mx || !y) return PATDNN_E_NULL;
    if (const int rc = on_device(h->device)) return rc;
    return product(h, mx, nullptr, 0, rows, y, ldy, static_cast<cudaStream_t>(stream));
}

int patdnn_linear8_plan(int32_t F, int32_t K, int64_t rows, int32_t from_8_bit_rows, patdnn_linear_plan_info *info) {
    if (!info) return PATDNN_E_NULL;
    if (F < 1 || F > kMostColumns || !size_ok(F, K) || !size_ok(rows, K) || rows < 1 || too_many_tiles(rows, F)) return PATDNN_E_SHAPE;
    Mx8Params p{};
    p.F = F; p.K = K; p.rows = rows;
    const bool fused = !from_8_bit_rows && rows <= kFusedRows;
    p.x_raw = fused ? info : nullptr;                  // (not read)
    const Mx8Launch l = plan_mx8_linear(p);
    *info = patdnn_linear_plan_info{};
    info->persistent = l.persistent; info->quantises = fused;
    info->tile_rows = l.persistent ? 256 : p.tile_n; info->tile_outputs = l.persistent ? p.tile_n : 128;
    info->column_tiles = p.col_tiles; info->splits = p.splits; info->stages = p.stages;
    info->piece_bytes = l.piece; info->grid = static_cast<int32_t>(l.grid); info->smem_bytes = l.smem; info->tensor_columns = p.tensor_columns;
    return PATDNN_OK;
}

int patdnn_linear8_check(patdnn_linear8 h) {
    return h ? check_status(h->device, h->status) : PATDNN_E_NULL;
}

int patdnn_linear8_debug_wait(patdnn_linear8 h, uint32_t polls, int32_t skip_load_iteration) {
    if (!h) return PATDNN_E_NULL;
    if (skip_load_iteration < 0) return PATDNN_E_SHAPE;
    h->spin_limit = polls;
    h->test_skip_load = skip_load_iteration;
    return PATDNN_OK;
}

int patdnn_linear8_free(patdnn_linear8 h) {
    delete h;
    return PATDNN_OK;
}

int patdnn_gated_create(const patdnn_gated_desc *desc, patdnn_gated *out) {
    if (!desc || !out) return PATDNN_E_NULL;
    if ((desc->dtype != PATDNN_F16 && desc->dtype != PATDNN_BF16) || !known_act(desc->act)) return PATDNN_E_DTYPE;
    if (!size_ok(desc->F, desc->K) || desc->F < 1 || desc->F > kMostColumns || !size_ok(desc->max_rows, desc->K) || !size_ok(desc->max_rows, desc->F) ||
        gated_too_large(desc->max_rows, desc->F, desc->K))
        return PATDNN_E_SHAPE;
    GatedShape s{};
    s.F = desc->F; s.K = desc->K; s.act = desc->act; s.dtype = desc->dtype;
    s.x_row = desc->x_row ? desc->x_row : s.K;
    s.w_row = desc->w_row ? desc->w_row : s.K;
    s.h_row = desc->h_row ? desc->h_row : s.F;
    for (int64_t row : {s.x_row, s.w_row, s.h_row})
        if (row > (int64_t(1) << 31)) return PATDNN_E_SHAPE;
    if (s.x_row < s.K || s.w_row < s.K || s.h_row < s.F) return PATDNN_E_SHAPE;
    patdnn_gated h = new (std::nothrow) patdnn_gated_s();
    if (!h) return PATDNN_E_ALLOC;
    h->s = s;
    h->max_rows = desc->max_rows;
    const size_t row = static_cast<size_t>(packed_row(s.K));
    uint16_t *dgu = nullptr, *x = nullptr, *weights = nullptr, *shifted = nullptr;
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = allocate(&h->w.partial, static_cast<size_t>(pairs_most()) * kGatedUnits * kGatedUnitFloats);
    if (e == cudaSuccess) e = allocate(&h->w.status, 4);
    if (e == cudaSuccess) e = cudaMemset(h->w.status, 0, 16);
    const size_t copy = static_cast<size_t>(desc->max_rows) * 2 * gated_padded(s.F);    // dg and du
    const bool scaled = desc->grad && s.dtype == PATDNN_F16;
    if (e == cudaSuccess && desc->grad) e = allocate(&dgu, scaled ? 2 * copy : copy);
    h->w.dgu = dgu;
    if (e == cudaSuccess && scaled) {
        h->w.by_column = dgu + copy;
        const size_t rows = (static_cast<size_t>(desc->max_rows) + 3) / 4 * 4, words = rows + 2 * static_cast<size_t>(gated_padded(s.F));   // (columns are read 16 bytes at a time)
        e = allocate(&h->w.row_top, 2 * words);
        if (e == cudaSuccess) e = cudaMemset(h->w.row_top, 0, words * sizeof(uint32_t));
        h->w.row_unscale = reinterpret_cast<float *>(h->w.row_top + words);
        h->w.column_top = h->w.row_top + rows;
        h->w.column_unscale = h->w.row_unscale + rows;
    }
    if (e == cudaSuccess && !copies_as_it_lies(s.x_row)) e = allocate(&x, static_cast<size_t>(desc->max_rows) * row);
    h->x = x;
    if (e == cudaSuccess && !copies_as_it_lies(s.w_row)) e = allocate(&weights, 2 * static_cast<size_t>(s.F) * row);
    h->weights = weights;
    if (e == cudaSuccess && weights)
        e = allocate(&shifted, static_cast<size_t>(std::min<int64_t>(kPhasedRows, desc->max_rows)) * gated_phases(s.w_row) * gated_phased_row(s.K));
    h->shifted = shifted;
    if (e == cudaSuccess) e = prepare_gated();
    if (e == cudaSuccess) e = cudaDeviceSynchronize();                  // the status word is zero on every stream from here on
    if (e != cudaSuccess) return failed(h, e, "patdnn_gated_create");
    *out = h;
    return PATDNN_OK;
}

int patdnn_gated_run(patdnn_gated h, const void *x, const void *wg, const void *wu, void *hidden, void *gu, int64_t rows, void *stream) {
    if (!h) return PATDNN_E_NULL;
    const GatedShape &s = h->s;
    if (rows < 0 || rows > h->max_rows || !operand_aligned(x, s.x_row) || !operand_aligned(wg, s.w_row) || !operand_aligned(wu, s.w_row) ||
        !aligned(hidden, 2) || !aligned(gu, 2))
        return PATDNN_E_SHAPE;
    if (rows == 0) return PATDNN_OK;
    if (!x || !wg || !wu || !hidden) return PATDNN_E_NULL;
    if (const int rc = on_device(h->device)) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    GatedCall c{};
    if (const int rc = gated_operands(h, x, wg, wu, nullptr, rows, true, true, c, st)) return rc;
    c.h = hidden; c.gu = gu;
    int n = 0;
    const cudaError_t e = launch_gated_forward(s, c, h->w, st, &n);
    return launched(e, n, "gated block launch");
}

int patdnn_gated_grad(patdnn_gated h, const void *x, const void *wg, const void *wu, const void *gu, const void *dh, void *dx, void *dwg, void *dwu,
                      int64_t rows, void *stream) {
    if (!h) return PATDNN_E_NULL;
    if (!h->w.dgu) return PATDNN_E_SCRATCH;
    const GatedShape &s = h->s;
    if (rows < 0 || rows > h->max_rows || !operand_aligned(x, s.x_row) || !operand_aligned(wg, s.w_row) || !operand_aligned(wu, s.w_row) ||
        !aligned(gu, 2) || !aligned(dh, 2) || !aligned(dx, 2) || !aligned(dwg, 2) || !aligned(dwu, 2))
        return PATDNN_E_SHAPE;
    if (!dwg != !dwu) return PATDNN_E_NULL;
    if (rows > 0 && (!x || !wg || !wu || !gu || !dh)) return PATDNN_E_NULL;
    if (const int rc = on_device(h->device)) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {
        for (void *w : {dwg, dwu})
            if (w) CU(cudaMemset2DAsync(w, static_cast<size_t>(s.w_row) * 2, 0, static_cast<size_t>(s.K) * 2, s.F, st));
        return PATDNN_OK;
    }
    if (!dx && !dwg) return PATDNN_OK;
    GatedCall c{};
    GatedSlopes slopes{gu, dh, h->w.dgu, nullptr, h->w.row_top, h->w.column_top, h->w.row_unscale, h->w.column_unscale};
    if (s.dtype == PATDNN_F16) {
        if (!dx) slopes.dgu = nullptr;
        if (dwg) slopes.by_column = h->w.by_column;
    }
    if (const int rc = gated_operands(h, x, wg, wu, &slopes, rows, dwg != nullptr, dx != nullptr, c, st)) return rc;
    c.dx = dx; c.dwg = dwg; c.dwu = dwu;
    int n = 0;
    const cudaError_t e = launch_gated_gradient(s, c, h->w, st, &n);
    return launched(e, n, "gated block gradient launch");
}

int patdnn_gated_plan(int32_t F, int32_t K, int64_t rows, int32_t product, patdnn_gated_plan_info *info) {
    return patdnn_gated_plan_strided(F, K, rows, product, 0, info);
}

int patdnn_gated_plan_strided(int32_t F, int32_t K, int64_t rows, int32_t product, int64_t w_row, patdnn_gated_plan_info *info) {
    if (!info) return PATDNN_E_NULL;
    if (w_row && (w_row < K || w_row > (int64_t(1) << 31))) return PATDNN_E_SHAPE;
    if (!size_ok(F, K) || F < 1 || F > kMostColumns || !size_ok(rows, K) || !size_ok(rows, F) || rows < 1 || gated_too_large(rows, F, K) || product < 0 ||
        product > 2)
        return PATDNN_E_SHAPE;
    GatedPlan gradient[2];
    plan_gated_gradient(F, K, rows, true, true, gradient);
    const int phases = product || !w_row ? 0 : phases_of(F, K, w_row, rows);
    const GatedPlan p = product ? gradient[product - 1] : phases ? plan_gated_phased(F, K, rows, phases) : plan_gated_forward(F, K, rows);
    *info = patdnn_gated_plan_info{};
    info->row_tiles = p.m_tiles; info->column_tiles = p.n_tiles; info->blocks = p.k_blocks; info->splits = p.splits; info->blocks_per_split = p.per_split;
    info->grid = p.grid; info->stages = p.stages; info->smem_bytes = p.smem;
    info->few_rows = p.few; info->tensor_columns = p.tensor_columns;
    return PATDNN_OK;
}

int patdnn_gated_check(patdnn_gated h) {
    return h ? check_status(h->device, h->w.status) : PATDNN_E_NULL;
}

int patdnn_gated_debug_wait(patdnn_gated h, uint32_t polls, int32_t skip_load_iteration) {
    if (!h) return PATDNN_E_NULL;
    if (skip_load_iteration < 0) return PATDNN_E_SHAPE;
    h->spin_limit = polls;
    h->test_skip_load = skip_load_iteration;
    return PATDNN_OK;
}

int patdnn_gated_free(patdnn_gated h) {
    delete h;
    return PATDNN_OK;
}

}  // extern "C"

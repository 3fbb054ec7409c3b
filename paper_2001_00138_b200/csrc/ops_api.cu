// C entry points of the group norm, the 4-bit matrices and the 4-bit linear layer (declared in include/patdnn.h).
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <new>

#include "../../include/patdnn.h"
#include "ops.hpp"

using namespace patdnn;

#define CU(call)                                             \
    do {                                                     \
        cudaError_t e_ = (call);                             \
        if (e_ != cudaSuccess) return cuda_fail(e_, #call);  \
    } while (0)

struct patdnn_norm_s {
    NormHandle h;
    int device = -1;
    ~patdnn_norm_s() {
        cudaFree(h.ws);
        cudaFree(h.counters);
        cudaFree(h.stats);
    }
};

struct patdnn_linear_s {
    patdnn_linear_desc d{};
    Mx4Shape shape{};                       // of the weights
    int device = -1;
    uint8_t *w = nullptr, *x = nullptr;     // 4-bit weights; buffer for the rows of patdnn_linear_run where max_rows is above kFusedRows
    float *bias = nullptr;
    int *status = nullptr;
    uint32_t spin_limit = 0;                // patdnn_linear_debug_wait
    int test_skip_load = 0;
    ~patdnn_linear_s() {
        cudaFree(w);
        cudaFree(x);
        cudaFree(bias);
        cudaFree(status);
    }
};

namespace {

constexpr int64_t kMostColumns = int64_t(1) << 20;
constexpr int64_t kMostElements = int64_t(1) << 40;

bool known_type(int dtype) { return dtype == PATDNN_F32 || dtype == PATDNN_F16 || dtype == PATDNN_BF16; }
bool known_act(int act) { return act == PATDNN_ACT_NONE || act == PATDNN_ACT_RELU || act == PATDNN_ACT_SILU; }
bool mx_size_ok(int64_t rows, int64_t cols) {
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
    const cudaError_t e = cudaMalloc(&v, count * sizeof(T) < 16 ? 16 : count * sizeof(T));
    *p = static_cast<T *>(v);
    return e;
}

bool too_many_tiles(int64_t rows, int64_t F) { return ceil_div(rows, 128) * ceil_div(F, 128) > INT32_MAX / 8; }   // CTAs of one launch

// mx: 4-bit rows, or nullptr with the rows themselves at x
int product(patdnn_linear h, const void *mx, const void *x, int64_t ldx, int64_t rows, void *y, int64_t ldy, cudaStream_t st) {
    if (too_many_tiles(rows, h->d.F)) return PATDNN_E_SHAPE;
    Mx4Params p{};
    p.w = h->w; p.x = static_cast<const uint8_t *>(mx); p.x_raw = x; p.ldx = ldx; p.K = h->d.K; p.bias = h->bias; p.y = y; p.status = h->status;
    p.ldy = ldy; p.rows = rows; p.w_scales = h->shape.scales_at; p.x_scales = mx4_shape(rows, h->d.K).scales_at;
    p.spin_limit = h->spin_limit; p.test_skip_load = h->test_skip_load;
    p.F = h->d.F; p.act = h->d.act; p.dtype = h->d.dtype;
    int n = 0;
    const cudaError_t e = launch_mx4_linear(p, st, &n);
    return launched(e, n, "4-bit product launch");
}

}  // namespace

extern "C" {

int patdnn_norm_create(const patdnn_norm_desc *desc, patdnn_norm *out) {
    if (!desc || !out) return PATDNN_E_NULL;
    if (!known_type(desc->dtype) || !known_act(desc->act)) return PATDNN_E_DTYPE;
    if (desc->N < 0 || desc->N > 65535 || desc->P < 1 || desc->P > INT32_MAX || desc->C < 1 || desc->C > kMostColumns || desc->G < 1 ||
        desc->C % desc->G || !std::isfinite(desc->eps) || desc->eps < 0.f)
        return PATDNN_E_SHAPE;
    if (desc->P > kMostElements / desc->C || (desc->N && desc->P * desc->C > kMostElements / desc->N)) return PATDNN_E_SHAPE;
    NormShape s{};
    s.N = desc->N; s.C = desc->C; s.G = desc->G; s.act = desc->act; s.dtype = desc->dtype; s.P = desc->P; s.eps = desc->eps;
    for (int i = 0; i < 2; ++i) {
        int64_t pixel = i ? desc->y_pixel : desc->x_pixel, image = i ? desc->y_image : desc->x_image;
        if (pixel == 0) pixel = s.C;
        if (pixel < s.C || pixel > kMostElements / s.P) return PATDNN_E_SHAPE;
        if (image == 0) image = s.P * pixel;
        if (image < (s.P - 1) * pixel + s.C || (s.N && image > (int64_t(1) << 60) / s.N)) return PATDNN_E_SHAPE;
        (i ? s.y_pixel : s.x_pixel) = pixel;
        (i ? s.y_image : s.x_image) = image;
    }
    patdnn_norm h = new (std::nothrow) patdnn_norm_s();
    if (!h) return PATDNN_E_ALLOC;
    h->h.s = s;
    if (s.N > 0) {
        const cudaError_t de = cudaGetDevice(&h->device);
        if (de != cudaSuccess) {
            const int rc = cuda_fail(de, "cudaGetDevice");
            delete h;
            return rc;
        }
        plan_norm(h->h);
        const size_t counters = static_cast<size_t>(s.G);
        cudaError_t e = allocate(&h->h.ws, norm_workspace_floats(h->h));
        if (e == cudaSuccess) e = allocate(&h->h.counters, counters);
        if (e == cudaSuccess) e = cudaMemset(h->h.counters, 0, sizeof(unsigned) * counters);
        if (e == cudaSuccess) e = allocate(&h->h.stats, static_cast<size_t>(s.N) * s.G * 2);
        if (e == cudaSuccess) e = prepare_norm();
        if (e == cudaSuccess) e = cudaDeviceSynchronize();              // the counters are zero on every stream from here on
        if (e != cudaSuccess) {
            const int rc = cuda_fail(e, "patdnn_norm_create");
            delete h;
            return rc;
        }
    }
    *out = h;
    return PATDNN_OK;
}

int patdnn_norm_run(patdnn_norm h, const void *x, const float *gamma, const float *beta, void *y, float *stats, void *stream) {
    if (!h) return PATDNN_E_NULL;
    if (h->h.s.N == 0) return PATDNN_OK;
    if (!x || !gamma || !beta || !y) return PATDNN_E_NULL;
    const int dtype = h->h.s.dtype;
    if (!elements_aligned(x, dtype) || !elements_aligned(y, dtype) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(stats, 8)) return PATDNN_E_SHAPE;
    if (const int rc = on_device(h->device)) return rc;
    int n = 0;
    const cudaError_t e = launch_group_norm(h->h, x, gamma, beta, y, stats, static_cast<cudaStream_t>(stream), &n);
    return launched(e, n, "group norm launch");
}

int patdnn_norm_run_mx4(patdnn_norm h, const void *x, const float *gamma, const float *beta, void *mx, float *stats, void *stream) {
    if (!h) return PATDNN_E_NULL;
    const NormShape &s = h->h.s;
    if (s.N == 0) return PATDNN_OK;
    if (!x || !gamma || !beta || !mx) return PATDNN_E_NULL;
    if (!aligned(mx, 16) || !mx_size_ok(s.N * s.P, s.C) || !elements_aligned(x, s.dtype) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(stats, 8))
        return PATDNN_E_SHAPE;
    if (const int rc = on_device(h->device)) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    int n = 0;
    const cudaError_t e = launch_group_norm_mx4(h->h, x, gamma, beta, mx, stats, st, &n);
    return launched(e, n, "group norm launch");
}

int patdnn_norm_grad(patdnn_norm h, const void *x, const float *gamma, const float *beta, const float *stats, const void *dy, void *dx,
                     float *dgamma, float *dbeta, void *stream) {
    if (!h || !dgamma || !dbeta) return PATDNN_E_NULL;
    const NormShape &s = h->h.s;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (s.N == 0) {
        CU(cudaMemsetAsync(dgamma, 0, sizeof(float) * s.C, st));
        CU(cudaMemsetAsync(dbeta, 0, sizeof(float) * s.C, st));
        return PATDNN_OK;
    }
    if (!x || !gamma || !beta || !stats || !dy || !dx) return PATDNN_E_NULL;
    if (!elements_aligned(x, s.dtype) || !elements_aligned(dy, s.dtype) || !elements_aligned(dx, s.dtype) || !aligned(gamma, 4) || !aligned(beta, 4) ||
        !aligned(stats, 8) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
        return PATDNN_E_SHAPE;
    if (const int rc = on_device(h->device)) return rc;
    int n = 0;
    const cudaError_t e = launch_group_norm_grad(h->h, x, gamma, beta, stats, dy, dx, dgamma, dbeta, st, &n);
    return launched(e, n, "group norm gradient launch");
}

int patdnn_norm_free(patdnn_norm h) {
    delete h;
    return PATDNN_OK;
}

int patdnn_mx4_bytes(int64_t rows, int64_t cols, int64_t *bytes) {
    if (!bytes) return PATDNN_E_NULL;
    if (!mx_size_ok(rows, cols)) return PATDNN_E_SHAPE;
    *bytes = mx4_shape(rows, cols).bytes;
    return PATDNN_OK;
}

int patdnn_mx4_quantize(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, void *mx, void *stream) {
    if (!known_type(dtype)) return PATDNN_E_DTYPE;
    if (!mx_size_ok(rows, cols)) return PATDNN_E_SHAPE;
    if (ld == 0) ld = cols;
    if (ld < cols || !aligned(mx, 16) || !elements_aligned(x, dtype)) return PATDNN_E_SHAPE;
    if (rows == 0) return PATDNN_OK;
    if (!x || !mx) return PATDNN_E_NULL;
    return launched(launch_mx4_quantize(mx4_shape(rows, cols), x, dtype, ld, mx, static_cast<cudaStream_t>(stream)), 1, "4-bit quantisation launch");
}

int patdnn_mx4_dequantize(const void *mx, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, void *out, void *stream) {
    if (!known_type(dtype)) return PATDNN_E_DTYPE;
    if (!mx_size_ok(rows, cols)) return PATDNN_E_SHAPE;
    if (ld == 0) ld = cols;
    if (ld < cols || !aligned(mx, 16) || !elements_aligned(out, dtype)) return PATDNN_E_SHAPE;
    if (rows == 0) return PATDNN_OK;
    if (!out || !mx) return PATDNN_E_NULL;
    return launched(launch_mx4_dequantize(mx4_shape(rows, cols), mx, out, dtype, ld, static_cast<cudaStream_t>(stream)), 1, "4-bit read-back launch");
}

int patdnn_linear_encode(const void *weights, int64_t ldw, const patdnn_linear_desc *desc, void *stream, patdnn_linear *out) {
    if (!weights || !desc || !out) return PATDNN_E_NULL;
    if (!known_type(desc->dtype) || !known_act(desc->act)) return PATDNN_E_DTYPE;
    if (desc->F < 1 || desc->K < 1 || !mx_size_ok(desc->F, desc->K) || desc->F > kMostColumns || !mx_size_ok(desc->max_rows, desc->K))
        return PATDNN_E_SHAPE;
    if (ldw == 0) ldw = desc->K;
    if (ldw < desc->K || !elements_aligned(weights, desc->dtype) || !aligned(desc->bias, 4)) return PATDNN_E_SHAPE;
    patdnn_linear h = new (std::nothrow) patdnn_linear_s();
    if (!h) return PATDNN_E_ALLOC;
    h->d = *desc;
    h->d.bias = nullptr;
    h->shape = mx4_shape(desc->F, desc->K);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = allocate(&h->w, static_cast<size_t>(h->shape.bytes));
    if (e == cudaSuccess && desc->max_rows > kFusedRows) e = allocate(&h->x, static_cast<size_t>(mx4_shape(desc->max_rows, desc->K).bytes));
    if (e == cudaSuccess) e = allocate(&h->status, 4);
    if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, 16, st);
    if (e == cudaSuccess && desc->bias) {
        e = allocate(&h->bias, static_cast<size_t>(desc->F));
        if (e == cudaSuccess) e = cudaMemcpyAsync(h->bias, desc->bias, sizeof(float) * desc->F, cudaMemcpyDeviceToDevice, st);
    }
    if (e == cudaSuccess) e = prepare_mx4_linear();
    if (e == cudaSuccess) e = launch_mx4_quantize(h->shape, weights, desc->dtype, ldw, h->w, st);
    if (e == cudaSuccess) {
        count_launches(1);
        e = cudaStreamSynchronize(st);
    }
    if (e != cudaSuccess) {
        const int rc = cuda_fail(e, "patdnn_linear_encode");
        delete h;
        return rc;
    }
    *out = h;
    return PATDNN_OK;
}

int patdnn_linear_run(patdnn_linear h, const void *x, int64_t rows, int64_t ldx, void *y, int64_t ldy, void *stream) {
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
    const int rc = launched(launch_mx4_quantize(mx4_shape(rows, h->d.K), x, h->d.dtype, ldx, h->x, st), 1, "4-bit quantisation launch");
    return rc ? rc : product(h, h->x, nullptr, 0, rows, y, ldy, st);
}

int patdnn_linear_run_mx4(patdnn_linear h, const void *mx, int64_t rows, void *y, int64_t ldy, void *stream) {
    if (!h) return PATDNN_E_NULL;
    if (ldy == 0) ldy = h->d.F;
    if (!mx_size_ok(rows, h->d.K) || ldy < h->d.F || !aligned(mx, 16) || !elements_aligned(y, h->d.dtype)) return PATDNN_E_SHAPE;
    if (rows == 0) return PATDNN_OK;
    if (!mx || !y) return PATDNN_E_NULL;
    if (const int rc = on_device(h->device)) return rc;
    return product(h, mx, nullptr, 0, rows, y, ldy, static_cast<cudaStream_t>(stream));
}

int patdnn_linear_plan(int32_t F, int32_t K, int64_t rows, int32_t from_4_bit_rows, patdnn_linear_plan_info *info) {
    if (!info) return PATDNN_E_NULL;
    if (F < 1 || F > kMostColumns || !mx_size_ok(F, K) || !mx_size_ok(rows, K) || rows < 1 || too_many_tiles(rows, F)) return PATDNN_E_SHAPE;
    Mx4Params p{};
    p.F = F; p.K = K; p.rows = rows;
    const bool fused = !from_4_bit_rows && rows <= kFusedRows;
    p.x_raw = fused ? info : nullptr;                  // (not read)
    const Mx4Launch l = plan_mx4_linear(p);
    *info = patdnn_linear_plan_info{};
    info->persistent = l.persistent; info->quantises = fused;
    info->tile_rows = l.persistent ? 128 : p.tile_n; info->tile_outputs = l.persistent ? p.tile_n : 128;
    info->column_tiles = p.col_tiles; info->splits = p.splits; info->stages = p.stages;
    info->piece_bytes = l.piece; info->grid = static_cast<int32_t>(l.grid); info->smem_bytes = l.smem; info->tensor_columns = p.tensor_columns;
    return PATDNN_OK;
}

int patdnn_linear_check(patdnn_linear h) {
    if (!h) return PATDNN_E_NULL;
    if (const int rc = on_device(h->device)) return rc;
    CU(cudaDeviceSynchronize());
    int word = 0;
    CU(cudaMemcpy(&word, h->status, sizeof(int), cudaMemcpyDeviceToHost));
    if (!word) return PATDNN_OK;
    CU(cudaMemset(h->status, 0, sizeof(int)));
    return PATDNN_E_DEVICE_TIMEOUT;
}

int patdnn_linear_debug_wait(patdnn_linear h, uint32_t polls, int32_t skip_load_iteration) {
    if (!h) return PATDNN_E_NULL;
    if (skip_load_iteration < 0) return PATDNN_E_SHAPE;
    h->spin_limit = polls;
    h->test_skip_load = skip_load_iteration;
    return PATDNN_OK;
}

int patdnn_linear_free(patdnn_linear h) {
    delete h;
    return PATDNN_OK;
}

}  // extern "C"

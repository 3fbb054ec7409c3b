// Microscaled 4-bit floating point: quantisation of a matrix's rows, alone or behind a group norm, and the way back.
//
//   A block is 32 consecutive columns of a row (the last block of a row may be shorter).  With amax its largest magnitude:
//   scale = 2^max(floor(log2(amax)) - 2, -127), held as its 8-bit exponent; element = x / scale rounded to the nearest of
//   {0, 0.5, 1, 1.5, 2, 3, 4, 6} with ties to the even code, sign kept; magnitudes above 6 become 6.  A block with an infinity or a
//   NaN gets the scale NaN (255): all 32 values read back as NaN.  A block of zeros has scale 2^-127.
//
// Memory bound: sizeof(T) bytes read and 17/32 bytes written per element.  A warp takes one row of a column tile at a time: lane l
// holds 8 consecutive columns, four lanes share a block (two shuffles give amax), every lane writes 4 bytes of codes and the warp
// together one row of the tile, 128 consecutive bytes.  It takes four rows 32 apart, since the scales of rows r, r + 32, r + 64 and
// r + 96 are neighbours in memory (16 bytes): 4 loads in flight per lane, and full 32-byte sectors for the scales.
#include "ops.hpp"

#include "kernels.hpp"
#include "ops_device.cuh"

namespace patdnn {
namespace {

constexpr int kWarps = 8;

// The two codes of (lo, hi) in one byte, lo in the lower half; nearest even, magnitudes above 6 become 6.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    asm("{\n\t.reg .b8 b;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %2, %1;\n\t"
        "cvt.u32.u8 %0, b;\n\t}" : "=r"(r) : "f"(lo), "f"(hi));
    return r;
}

// Scale byte of a block from the bits of its largest magnitude (sign bit clear), and the factor 1 / scale.
__device__ __forceinline__ uint32_t scale_of(uint32_t amax_bits, float &inverse) {
    const uint32_t field = amax_bits >> 23;            // biased exponent; 0 for zero and subnormals
    if (field == 255) {
        inverse = 0.f;
        return 255;
    }
    const uint32_t byte = field > 2 ? field - 2 : 0;   // biased by 127: 2^(field - 127 - 2), at least 2^-127
    // 1 / scale = 2^(127 - byte), byte <= 252: exponent field 254 - byte, always normal
    inverse = __uint_as_float((254 - byte) << 23);
    return byte;
}

// Eight values of one lane -> its 4 bytes of codes; returns the block's scale byte (the same in the four lanes of a block).
__device__ __forceinline__ uint32_t quantise8(const float (&v)[8], uint32_t &codes) {
    uint32_t top = 0;                                  // magnitudes compare like their bits; a NaN is above infinity
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    float inverse;
    const uint32_t scale = scale_of(top, inverse);
    codes = 0;
    if (scale != 255) {
#pragma unroll
        for (int j = 0; j < 4; ++j) codes |= pack2(v[2 * j] * inverse, v[2 * j + 1] * inverse) << (8 * j);
    }
    return scale;
}

struct QuantArgs {
    const void *x;
    uint8_t *mx;
    int64_t rows, cols, ld;
    int64_t scales_at;
    int width, col_tiles, code_bytes, scale_bytes;
    // group norm in front (norm kernels only): row = image * P + pixel
    const float *gamma, *beta, *stats;
    int64_t P, x_image;
    int G, per, act;
};

// Columns [c, c + 8) of a row; 0 beyond the last column.  A = elements per access.
template <typename T, int A>
__device__ __forceinline__ void load8(const T *row, int64_t c, int64_t cols, float (&v)[8]) {
    if (c + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < 8 / A; ++i) {
            const Vec<T, A> t = *reinterpret_cast<const Vec<T, A> *>(row + c + i * A);
#pragma unroll
            for (int j = 0; j < A; ++j) v[i * A + j] = to_float(t.v[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? to_float(row[c + j]) : 0.f;
    }
}

// grid: x = column tiles, y.. = groups of 32 "row sets"; a warp's row set is rows r, r+32, r+64, r+96 of a row tile.
// blockIdx.x = (row tile * 4 + quarter) * col_tiles + column tile; quarter: row sets 8 * quarter + warp.
template <typename T, int A, bool NORM>
__global__ void __launch_bounds__(kWarps * 32) mx4_quantize_kernel(QuantArgs a) {
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t tile = blockIdx.x;
    const int ct = static_cast<int>(tile % a.col_tiles);
    const int64_t rest = tile / a.col_tiles;
    const int64_t rt = rest >> 2;
    const int r0 = static_cast<int>(rest & 3) * kWarps + warp;         // first row of the set, 0 .. 31
    const int64_t c = static_cast<int64_t>(ct) * a.width + lane * 8;
    const int tile_row = a.width / 2;                                  // bytes of a row of the code tile
    uint8_t *codes_out = a.mx + (rt * a.col_tiles + ct) * a.code_bytes;
    uint8_t *scales_out = a.mx + a.scales_at + (rt * a.col_tiles + ct) * a.scale_bytes;
    pdl_wait();
    if (rt * 128 + r0 >= a.rows) return;                               // warp-uniform; higher rows of the set do not exist either
    const bool mine = lane * 8 < a.width;                              // narrow tiles leave lanes idle
    float v[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t row = rt * 128 + r0 + 32 * k;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[k][j] = 0.f;
        if (row < a.rows && mine) {
            const T *src = static_cast<const T *>(a.x);
            if constexpr (NORM) src += (row / a.P) * a.x_image + (row % a.P) * a.ld;
            else src += row * a.ld;
            load8<T, A>(src, c, a.cols, v[k]);
        }
    }
    if constexpr (NORM) {
        float gm[8], bt[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = mine && c + j < a.cols;
            gm[j] = in ? a.gamma[c + j] : 0.f;
            bt[j] = in ? a.beta[c + j] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t row = rt * 128 + r0 + 32 * k;
            if (row >= a.rows) continue;
            const float2 *st = reinterpret_cast<const float2 *>(a.stats) + (row / a.P) * a.G;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (!mine || c + j >= a.cols) continue;
                const float2 f = st[(c + j) / a.per];
                v[k][j] = activate(fmaf(v[k][j] - f.x, f.y * gm[j], bt[j]), a.act);
            }
        }
    }
    uint32_t sets[4];                                                  // lane of block b: byte of (row r0 + 32 k, b) in bits 0..7 of sets[k]
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t codes;
        sets[k] = quantise8(v[k], codes);
        if (rt * 128 + r0 + 32 * k < a.rows && mine) {
            int at = (r0 + 32 * k) * tile_row + lane * 4;
            at ^= ((at >> 7) & (a.width / 32 - 1)) << 4;
            *reinterpret_cast<uint32_t *>(codes_out + at) = codes;
        }
    }
    // lanes 0 and 16 gather the scale bytes of blocks 0..3 and 4..7: 16 bytes each
    uint32_t word[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t w = sets[k];
        w |= __shfl_down_sync(0xffffffffu, w, 4) << 8;
        w |= __shfl_down_sync(0xffffffffu, w, 8) << 16;
        word[k] = w;
    }
    if ((lane & 15) == 0 && lane * 8 < a.width)
        *reinterpret_cast<uint4 *>(scales_out + (lane >> 4) * 512 + r0 * 16) = make_uint4(word[0], word[1], word[2], word[3]);
}

__device__ __forceinline__ float value_of(uint32_t code, float scale) {
    // magnitudes of the codes 0..7 as 2 * value: 0 1 2 3 4 6 8 12
    const uint32_t e = (code >> 1) & 3, m = code & 1;
    const float mag = e == 0 ? 0.5f * static_cast<float>(m) : static_cast<float>((2 + m) << (e - 1)) * 0.5f;
    return (code & 8 ? -mag : mag) * scale;
}

template <typename T, int A>
__global__ void __launch_bounds__(kWarps * 32) mx4_dequantize_kernel(QuantArgs a, T *out) {
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t tile = blockIdx.x;
    const int ct = static_cast<int>(tile % a.col_tiles);
    const int64_t rest = tile / a.col_tiles;
    const int64_t rt = rest >> 2;
    const int r0 = static_cast<int>(rest & 3) * kWarps + warp;
    const int64_t c = static_cast<int64_t>(ct) * a.width + lane * 8;
    const int tile_row = a.width / 2;
    const uint8_t *codes_in = a.mx + (rt * a.col_tiles + ct) * a.code_bytes;
    const uint8_t *scales_in = a.mx + a.scales_at + (rt * a.col_tiles + ct) * a.scale_bytes;
    pdl_wait();
    if (lane * 8 >= a.width || c >= a.cols) return;
    uint32_t codes[4], scale[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (rt * 128 + r0 + 32 * k >= a.rows) continue;
        int at = (r0 + 32 * k) * tile_row + lane * 4;
        at ^= ((at >> 7) & (a.width / 32 - 1)) << 4;
        codes[k] = *reinterpret_cast<const uint32_t *>(codes_in + at);
        scale[k] = scales_in[(lane >> 4) * 512 + r0 * 16 + k * 4 + ((lane >> 2) & 3)];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t row = rt * 128 + r0 + 32 * k;
        if (row >= a.rows) continue;
        // 2^(byte - 127): byte 0 is the subnormal 2^-127, 255 is NaN
        const float s = scale[k] == 255 ? __uint_as_float(0x7fffffffu) : scale[k] ? __uint_as_float(scale[k] << 23) : __uint_as_float(0x00400000u);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = value_of((codes[k] >> (4 * j)) & 15, s);
        T *dst = out + row * a.ld;
        if (c + 8 <= a.cols) {
#pragma unroll
            for (int i = 0; i < 8 / A; ++i) {
                Vec<T, A> t;
#pragma unroll
                for (int j = 0; j < A; ++j) t.v[j] = from_float<T>(v[i * A + j]);
                *reinterpret_cast<Vec<T, A> *>(dst + c + i * A) = t;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < a.cols) dst[c + j] = from_float<T>(v[j]);
        }
    }
}

QuantArgs quant_args(const Mx4Shape &m, const void *x, int64_t ld, void *mx) {
    QuantArgs a{};
    a.x = x; a.mx = static_cast<uint8_t *>(mx);
    a.rows = m.rows; a.cols = m.cols; a.ld = ld;
    a.scales_at = m.scales_at; a.width = m.width; a.col_tiles = static_cast<int>(m.col_tiles);
    a.code_bytes = m.code_bytes; a.scale_bytes = m.scale_bytes;
    a.P = 1; a.G = 1; a.per = 1;
    return a;
}

unsigned quant_grid(const Mx4Shape &m) {               // no CTA for quarters without rows in the last row tile
    const int64_t last = m.rows - (m.row_tiles - 1) * 128;
    const int64_t quarters = (m.row_tiles - 1) * 4 + (last >= 32 ? 4 : ceil_div(last, kWarps));
    return static_cast<unsigned>(quarters * m.col_tiles);
}

// elements per access: 16 bytes where addresses and strides allow, else two, else one
int access_index(int dtype, const void *p, int64_t ld, int64_t stride2 = 0) {
    const int e = elem_bytes(dtype);
    for (int i = 0; i < 3; ++i) {
        const int v = i == 0 ? 16 / e : i == 1 ? 2 : 1;
        if (ld % v == 0 && stride2 % v == 0 && reinterpret_cast<uintptr_t>(p) % (static_cast<unsigned>(v) * e) == 0) return i;
    }
    return 2;
}

template <typename F> cudaError_t by_access(int dtype, int i, F f) {
    if (dtype == PATDNN_F32) return i == 0 ? f(float{}, std::integral_constant<int, 4>{}) : i == 1 ? f(float{}, std::integral_constant<int, 2>{}) : f(float{}, std::integral_constant<int, 1>{});
    if (dtype == PATDNN_F16) return i == 0 ? f(__half{}, std::integral_constant<int, 8>{}) : i == 1 ? f(__half{}, std::integral_constant<int, 2>{}) : f(__half{}, std::integral_constant<int, 1>{});
    return i == 0 ? f(__nv_bfloat16{}, std::integral_constant<int, 8>{}) : i == 1 ? f(__nv_bfloat16{}, std::integral_constant<int, 2>{}) : f(__nv_bfloat16{}, std::integral_constant<int, 1>{});
}

}  // namespace

cudaError_t launch_mx4_quantize(const Mx4Shape &m, const void *x, int dtype, int64_t ld, void *mx, cudaStream_t st) {
    const QuantArgs a = quant_args(m, x, ld, mx);
    return by_access(dtype, access_index(dtype, x, ld), [&](auto t, auto v) {
        return launch_pdl(mx4_quantize_kernel<decltype(t), v.value, false>, dim3(quant_grid(m)), dim3(kWarps * 32), 0, st, 1, a);
    });
}

cudaError_t launch_norm_quantize(const NormShape &s, const Mx4Shape &m, const void *x, const float *gamma, const float *beta,
                                 const float *stats, void *mx, cudaStream_t st) {
    QuantArgs a = quant_args(m, x, s.x_pixel, mx);
    a.gamma = gamma; a.beta = beta; a.stats = stats;
    a.P = s.P; a.x_image = s.x_image; a.G = s.G; a.per = s.C / s.G; a.act = s.act;
    return by_access(s.dtype, access_index(s.dtype, x, s.x_pixel, s.x_image), [&](auto t, auto v) {
        return launch_pdl(mx4_quantize_kernel<decltype(t), v.value, true>, dim3(quant_grid(m)), dim3(kWarps * 32), 0, st, 1, a);
    });
}

cudaError_t launch_mx4_dequantize(const Mx4Shape &m, const void *mx, void *out, int dtype, int64_t ld, cudaStream_t st) {
    const QuantArgs a = quant_args(m, nullptr, ld, const_cast<void *>(mx));
    return by_access(dtype, access_index(dtype, out, ld), [&](auto t, auto v) {
        using T = decltype(t);
        return launch_pdl(mx4_dequantize_kernel<T, v.value>, dim3(quant_grid(m)), dim3(kWarps * 32), 0, st, 1, a, static_cast<T *>(out));
    });
}

}  // namespace patdnn

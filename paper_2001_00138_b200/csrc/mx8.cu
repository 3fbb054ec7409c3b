// 8-bit floating point with a scale for each block of 128 columns: quantisation of a matrix's rows, and the way back.
//
//   With amax the largest magnitude of a block: scale = 2^max(ceil(log2(amax / 448)), -127), held as its 8-bit exponent; element = x / scale
//   rounded to the nearest E4M3 value, ties to even.  Nothing saturates: 448 is the largest magnitude of the type.  A block with an infinity
//   or a NaN gets the scale NaN (255): all its values read back as NaN.  A block of zeros has scale 2^-127.
//
// Memory bound: sizeof(T) bytes read and 129/128 written per element.  A warp takes 512 columns of four rows 32 apart, whose 16 scale bytes are
// neighbours in memory: 8 loads of 16 bytes in flight per lane (16-bit types), and scales stored 16 bytes at a time.  Small matrices are spread
// over four times the warps, one row each.
#include "feed_forward.hpp"

#include <algorithm>

#include "kernels.hpp"
#include "mx8_device.cuh"

namespace patdnn {
namespace {

constexpr int kWarps = 8, kColumns = 512;              // columns of a row that a warp takes: 16 per lane

struct Mx8Args {
    const void *x;
    uint8_t *mx;
    int64_t rows, cols, ld, scales_at;
    int col_tiles, groups;
};

// ROWS: of a row set that a warp takes, 4 or 1
template <typename T, int A, int ROWS>
__global__ void __launch_bounds__(kWarps * 32) mx8_quantize_kernel(Mx8Args a, unsigned units) {
    pdl_trigger();
    const unsigned unit = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);   // (row or row set, group of columns)
    if (unit >= units) return;
    const int lane = threadIdx.x & 31;
    const int group = static_cast<int>(unit % static_cast<unsigned>(a.groups));
    const int64_t set = unit / static_cast<unsigned>(a.groups), rt = ROWS == 4 ? set >> 5 : set >> 7;
    const int r0 = static_cast<int>(ROWS == 4 ? set & 31 : set & 127); // its first row in the row tile
    const int64_t c0 = static_cast<int64_t>(group) * kColumns;
    const int left = static_cast<int>(min(static_cast<int64_t>(kColumns), a.cols - c0));
    const int padded = (left + 127) & ~127;
    pdl_wait();
    Strip<T, A, 16> raw[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int64_t row = rt * 128 + r0 + 32 * k;
        if (row < a.rows) raw[k].load(static_cast<const T *>(a.x) + row * a.ld + c0, left);
    }
    constexpr int PER = A == 8 ? 1 : 4 / A, BLOCKS = 16 / A / PER;     // accesses to a block; blocks that a lane knows (A = 8: every other one)
    uint8_t *codes = a.mx + (rt * a.col_tiles + static_cast<int64_t>(group) * 4) * kMx8Tile;
    uint32_t words[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        words[k] = 0;
        if (rt * 128 + r0 + 32 * k >= a.rows) continue;                // (the same for the warp)
        float v[16];
        raw[k].widen_to(v);
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            constexpr int N = A * PER;
            float m = max_abs(v[b * N], v[b * N + N - 1]);
#pragma unroll
            for (int e = 1; e < N - 1; ++e) m = max_abs(m, v[b * N + e]);
            uint32_t top = magnitude_bits(m);
#pragma unroll
            for (int s = 1; s < (A == 8 ? 16 : 32); s *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
            float inverse;
            const uint32_t byte = scale8_of(top, inverse);
            if constexpr (A == 8) words[k] |= (byte << (16 * b)) | (__shfl_down_sync(0xffffffffu, byte, 16) << (16 * b + 8));
            else words[k] |= byte << (8 * b);
#pragma unroll
            for (int j = b * PER; j < (b + 1) * PER; ++j) {
                const int c = (32 * j + lane) * A;
                if (c < padded) store_codes<A>(codes + (c >> 7) * kMx8Tile + mx8_place(r0 + 32 * k, c & 127), v + j * A, inverse);
            }
        }
    }
    if (lane == 0) {                                   // (the words of rows that do not exist belong to nothing)
        uint8_t *scales = a.mx + a.scales_at + (rt * a.groups + group) * kMx8Scales + mx8_scale_place(r0, 0);
        if constexpr (ROWS == 4) *reinterpret_cast<uint4 *>(scales) = make_uint4(words[0], words[1], words[2], words[3]);
        else *reinterpret_cast<uint32_t *>(scales) = words[0];
    }
}

template <typename T, int A, int ROWS>
__global__ void __launch_bounds__(kWarps * 32) mx8_dequantize_kernel(Mx8Args a, T *out, unsigned units) {
    pdl_trigger();
    const unsigned unit = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (unit >= units) return;
    const int lane = threadIdx.x & 31;
    const int group = static_cast<int>(unit % static_cast<unsigned>(a.groups));
    const int64_t set = unit / static_cast<unsigned>(a.groups), rt = ROWS == 4 ? set >> 5 : set >> 7;
    const int r0 = static_cast<int>(ROWS == 4 ? set & 31 : set & 127); // its first row in the row tile
    const int64_t c0 = static_cast<int64_t>(group) * kColumns;
    const int left = static_cast<int>(min(static_cast<int64_t>(kColumns), a.cols - c0));
    const uint8_t *codes = a.mx + (rt * a.col_tiles + static_cast<int64_t>(group) * 4) * kMx8Tile;
    pdl_wait();
    const uint8_t *scales = a.mx + a.scales_at + (rt * a.groups + group) * kMx8Scales + mx8_scale_place(r0, 0);
    uint32_t words[ROWS];
    if constexpr (ROWS == 4) {
        const uint4 four = *reinterpret_cast<const uint4 *>(scales);
        words[0] = four.x;
        words[1] = four.y;
        words[2] = four.z;
        words[3] = four.w;
    } else {
        words[0] = *reinterpret_cast<const uint32_t *>(scales);
    }
    constexpr int NA = 16 / A;
    uint32_t raw[ROWS][NA][A == 8 ? 2 : 1];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        if (rt * 128 + r0 + 32 * k >= a.rows) continue;
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            const int c = (32 * j + lane) * A;
            if (c >= left) continue;
            const uint8_t *from = codes + (c >> 7) * kMx8Tile + mx8_place(r0 + 32 * k, c & 127);
            if constexpr (A == 8) {
                const uint2 t = *reinterpret_cast<const uint2 *>(from);
                raw[k][j][0] = t.x;
                raw[k][j][1] = t.y;
            } else if constexpr (A == 4) raw[k][j][0] = *reinterpret_cast<const uint32_t *>(from);
            else if constexpr (A == 2) raw[k][j][0] = *reinterpret_cast<const uint16_t *>(from);
            else raw[k][j][0] = *from;
        }
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int64_t row = rt * 128 + r0 + 32 * k;
        if (row >= a.rows) continue;
        Strip<T, A, 16> s;
        float v[16];
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            const int block = (32 * j + lane) * A >> 7;
            const float scale = scale8_value((words[k] >> (8 * block)) & 255);
#pragma unroll
            for (int e = 0; e < (A > 1 ? A : 2); e += 2) {
                const float2 f = values2(raw[k][j][e / 4] >> (8 * (e & 3)));
                v[j * A + e] = f.x * scale;
                if constexpr (A > 1) v[j * A + e + 1] = f.y * scale;
            }
        }
        s.narrow_from(v);
        s.store(out + row * a.ld + c0, left);
    }
}

Mx8Args args_of(const Mx8Shape &m, const void *x, int64_t ld, void *mx) {
    Mx8Args a{};
    a.x = x; a.mx = static_cast<uint8_t *>(mx);
    a.rows = m.rows; a.cols = m.cols; a.ld = ld; a.scales_at = m.scales_at;
    a.col_tiles = static_cast<int>(m.col_tiles); a.groups = static_cast<int>(m.groups);
    return a;
}
// f(rows of a warp, units, CTAs, warps of a CTA).  Units are row sets (rows r, r + 32, r + 64, r + 96 of a row tile), or rows where sets would be
// fewer than two warps per scheduler; times groups of columns.  (2^40 elements in rows of one column are 2^29 sets.)
template <typename F> cudaError_t by_units(const Mx8Shape &m, F f) {
    const int64_t last = m.rows - (m.row_tiles - 1) * 128, sets = ((m.row_tiles - 1) * 32 + std::min<int64_t>(32, last)) * m.groups;
    if (sets >= static_cast<int64_t>(sm_count()) * 8) return f(std::integral_constant<int, 4>{}, static_cast<unsigned>(sets), dim3(static_cast<unsigned>(ceil_div(sets, kWarps))), dim3(kWarps * 32));
    const int64_t rows = m.rows * m.groups;
    const int warps = rows >= static_cast<int64_t>(sm_count()) * 8 ? 8 : rows >= static_cast<int64_t>(sm_count()) * 4 ? 4 : 2;
    return f(std::integral_constant<int, 1>{}, static_cast<unsigned>(rows), dim3(static_cast<unsigned>(ceil_div(rows, warps))), dim3(warps * 32));
}

}  // namespace

cudaError_t launch_mx8_quantize(const Mx8Shape &m, const void *x, int dtype, int64_t ld, void *mx, cudaStream_t st) {
    const Mx8Args a = args_of(m, x, ld, mx);
    return by_strip(dtype, strip_width(dtype, {x}, {ld}), [&](auto t, auto v) {
        return by_units(m, [&](auto rows, unsigned units, dim3 grid, dim3 block) {
            return launch_pdl(mx8_quantize_kernel<decltype(t), v.value, rows.value>, grid, block, 0, st, 1, a, units);
        });
    });
}

cudaError_t launch_mx8_dequantize(const Mx8Shape &m, const void *mx, void *out, int dtype, int64_t ld, cudaStream_t st) {
    const Mx8Args a = args_of(m, nullptr, ld, const_cast<void *>(mx));
    return by_strip(dtype, strip_width(dtype, {out}, {ld}), [&](auto t, auto v) {
        using T = decltype(t);
        return by_units(m, [&](auto rows, unsigned units, dim3 grid, dim3 block) {
            return launch_pdl(mx8_dequantize_kernel<T, v.value, rows.value>, grid, block, 0, st, 1, a, static_cast<T *>(out), units);
        });
    });
}

}  // namespace patdnn

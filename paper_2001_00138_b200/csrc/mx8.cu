// 8-bit floating point with a scale for each block of 128 columns: quantisation of a matrix's rows, and the way back.
//
//   With amax the largest magnitude of a block: scale = 2^max(ceil(log2(amax / 448)), -127), held as its 8-bit exponent; element = x / scale
//   rounded to the nearest E4M3 value, ties to even.  Nothing saturates: 448 is the largest magnitude of the type.  A block with an infinity
//   or a NaN gets the scale NaN (255): all its values read back as NaN.  A block of zeros has scale 2^-127.
//
// Memory bound: sizeof(T) bytes read and 129/128 written per element.  A warp takes 512 columns of four rows 32 apart, whose 16 scale bytes are
// neighbours in memory: 8 loads of 16 bytes in flight per lane (16-bit types), and scales stored 16 bytes at a time.  Small matrices are spread
// over four times the warps, one row each; of matrices with up to 256 columns a warp, or a half or a quarter of it, takes whole rows.  Rows that are
// not aligned to 16 bytes are read in aligned units and shifted into place.
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

// ROWS: of a row set that a warp takes, 4 or 1.  ALIGNED: rows are, to 16 bytes
template <typename T, bool ALIGNED, int ROWS>
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
    constexpr int A = 16 / sizeof(T);
    pdl_wait();
    Strip<T, A, 16> raw[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int64_t row = rt * 128 + r0 + 32 * k;
        if (row >= a.rows) continue;                   // (the same for the warp)
        const T *from = static_cast<const T *>(a.x) + row * a.ld + c0;
        if constexpr (ALIGNED) raw[k].load(from, left);
        else raw[k].load_any(from, left);
    }
    constexpr int PER = A == 8 ? 1 : 4 / A, BLOCKS = 16 / A / PER;     // accesses to a block; blocks that a lane knows (A = 8: every other one)
    uint8_t *codes = a.mx + (rt * a.col_tiles + static_cast<int64_t>(group) * 4) * kMx8Tile;
    uint32_t words[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        words[k] = 0;
        if (rt * 128 + r0 + 32 * k >= a.rows) continue;
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

// Up to 8 L columns (64, 128 or 256): a row per L lanes.  Columns up to the next multiple of 64 at least are written: the products read 32 at a time.
template <typename T, bool ALIGNED, int L>
__global__ void __launch_bounds__(kWarps * 32) mx8_quantize_narrow_kernel(Mx8Args a) {
    constexpr int A = 16 / sizeof(T), kTogether = 32 / L;
    pdl_trigger();
    const int64_t step = static_cast<int64_t>(gridDim.x) * kWarps * kTogether;
    const int cols = static_cast<int>(a.cols);
    pdl_wait();
    Strip<T, A, 8, L> raw;
    auto load = [&](int64_t first) {                   // rows from `first` on, one per L lanes
        const int64_t row = first + (threadIdx.x & 31) / L;
        const T *from = static_cast<const T *>(a.x) + (row < a.rows ? row * a.ld : 0);
        if constexpr (ALIGNED) raw.load(from, row < a.rows ? cols : 0);
        else raw.load_any(from, row < a.rows ? cols : 0);
    };
    int64_t first = (static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * kTogether;
    if (first < a.rows) load(first);
    for (; first < a.rows; first += step) {
        const int64_t row = first + (threadIdx.x & 31) / L, rt = row >> 7;
        float v[8];
        raw.widen_to(v);
        if (first + step < a.rows) load(first + step);
        store_blocks<A, 8, L>(a.mx + rt * a.col_tiles * kMx8Tile, a.mx + a.scales_at + rt * kMx8Scales, static_cast<int>(row & 127), 0,
                              row < a.rows ? a.col_tiles * 128 : 0, v);
    }
}

template <typename T, int A, int L>
__global__ void __launch_bounds__(kWarps * 32) mx8_dequantize_narrow_kernel(Mx8Args a, T *out) {
    constexpr int NA = 8 / A;
    pdl_trigger();
    const int lane = threadIdx.x & (L - 1), cols = static_cast<int>(a.cols);
    const int64_t step = static_cast<int64_t>(gridDim.x) * blockDim.x / L;
    pdl_wait();
    for (int64_t row = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) / L; row < a.rows; row += step) {
        const int64_t rt = row >> 7;
        const int r = static_cast<int>(row & 127);
        const uint8_t *codes = a.mx + rt * a.col_tiles * kMx8Tile;
        const uint32_t scales = *reinterpret_cast<const uint32_t *>(a.mx + a.scales_at + rt * kMx8Scales + mx8_scale_place(r, 0));
        Strip<T, A, 8, L> s;
        float v[8];
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            const int c = (L * j + lane) * A;
            if (c >= cols) continue;
            const uint8_t *from = codes + (c >> 7) * kMx8Tile + mx8_place(r, c & 127);
            uint32_t raw[2];
            if constexpr (A == 8) {
                const uint2 t = *reinterpret_cast<const uint2 *>(from);
                raw[0] = t.x;
                raw[1] = t.y;
            } else if constexpr (A == 4) raw[0] = *reinterpret_cast<const uint32_t *>(from);
            else if constexpr (A == 2) raw[0] = *reinterpret_cast<const uint16_t *>(from);
            else raw[0] = *from;
            const float scale = scale8_value((scales >> (8 * (c >> 7))) & 255);
#pragma unroll
            for (int e = 0; e < (A > 1 ? A : 2); e += 2) {
                const float2 f = values2(raw[e / 4] >> (8 * (e & 3)));
                v[j * A + e] = f.x * scale;
                if constexpr (A > 1) v[j * A + e + 1] = f.y * scale;
            }
        }
        s.narrow_from(v);
        s.store(out + row * a.ld, cols);
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

// f(lanes to a row) for matrices of up to 256 columns
template <typename F> cudaError_t by_lanes(int64_t cols, F f) {
    if (cols <= 64) return f(std::integral_constant<int, 8>{});
    if (cols <= 128) return f(std::integral_constant<int, 16>{});
    return f(std::integral_constant<int, 32>{});
}
dim3 narrow_grid(int64_t rows, int lanes) {
    return dim3(static_cast<unsigned>(std::min<int64_t>(ceil_div(rows, kWarps * 32 / lanes), static_cast<int64_t>(sm_count()) * 8)));
}

}  // namespace

cudaError_t launch_mx8_quantize(const Mx8Shape &m, const void *x, int dtype, int64_t ld, void *mx, cudaStream_t st) {
    const Mx8Args a = args_of(m, x, ld, mx);
    const int whole = 16 / elem_bytes(dtype);
    return by_strip(dtype, whole, [&](auto t, auto) {
        using T = decltype(t);
        const bool aligned = strip_width(dtype, {x}, {ld}) == whole;
        if (m.cols <= 256)
            return by_lanes(m.cols, [&](auto l) {
                const auto kernel = aligned ? mx8_quantize_narrow_kernel<T, true, l.value> : mx8_quantize_narrow_kernel<T, false, l.value>;
                return launch_pdl(kernel, narrow_grid(m.rows, l.value), dim3(kWarps * 32), 0, st, 1, a);
            });
        return by_units(m, [&](auto rows, unsigned units, dim3 grid, dim3 block) {
            const auto kernel = aligned ? mx8_quantize_kernel<T, true, rows.value> : mx8_quantize_kernel<T, false, rows.value>;
            return launch_pdl(kernel, grid, block, 0, st, 1, a, units);
        });
    });
}

cudaError_t launch_mx8_dequantize(const Mx8Shape &m, const void *mx, void *out, int dtype, int64_t ld, cudaStream_t st) {
    const Mx8Args a = args_of(m, nullptr, ld, const_cast<void *>(mx));
    return by_strip(dtype, strip_width(dtype, {out}, {ld}), [&](auto t, auto v) {
        using T = decltype(t);
        if (m.cols <= 256)
            return by_lanes(m.cols, [&](auto l) {
                return launch_pdl(mx8_dequantize_narrow_kernel<T, v.value, l.value>, narrow_grid(m.rows, l.value), dim3(kWarps * 32), 0, st, 1, a, static_cast<T *>(out));
            });
        return by_units(m, [&](auto rows, unsigned units, dim3 grid, dim3 block) {
            return launch_pdl(mx8_dequantize_kernel<T, v.value, rows.value>, grid, block, 0, st, 1, a, static_cast<T *>(out), units);
        });
    });
}

}  // namespace patdnn

// Microscaled 4-bit floating point: quantisation of a matrix's rows, alone or behind a group norm, and the way back.
//
//   A block is 32 consecutive columns of a row (the last block of a row may be shorter).  With amax its largest magnitude:
//   scale = 2^max(floor(log2(amax)) - 2, -127), held as its 8-bit exponent; element = x / scale rounded to the nearest of
//   {0, 0.5, 1, 1.5, 2, 3, 4, 6} with ties to the even code, sign kept; magnitudes above 6 become 6.  A block with an infinity or a
//   NaN gets the scale NaN (255): all 32 values read back as NaN.  A block of zeros has scale 2^-127.
//
// Memory bound: sizeof(T) bytes read and 17/32 bytes written per element.  A warp takes one row of a column tile at a time: lane l
// holds 8 consecutive columns, four lanes share a block (two shuffles give amax), every lane writes 4 bytes of codes and the warp
// together one row of the tile, 128 consecutive bytes (two or four rows of a narrow tile).  It takes four rows 32 apart, since the scales of rows r, r + 32, r + 64 and
// r + 96 are neighbours in memory (16 bytes): 4 loads in flight per lane, and full 32-byte sectors for the scales.
// Measured, 16384 x 4096 bf16: 36 us for 134 MB read and 36 MB written (67 % of the issue slots), 27 to 33 us back; an 8192 x 4096
// matrix that is in L2 15.6 us.
#include "ops.hpp"

#include <algorithm>

#include "kernels.hpp"
#include "ops_device.cuh"

namespace patdnn {
namespace {

constexpr int kWarps = 8;

struct QuantArgs {
    const void *x;
    uint8_t *mx;
    int64_t row0, rows, cols, ld;           // rows [row0, rows) of the matrix
    int64_t scales_at;
    int width, col_tiles, code_bytes, scale_bytes;
    int step_ct, step_rest;                 // from a CTA's unit to its next one: column tiles, parts of row tiles
    int lanes, part_shift;                  // lanes to a row of a tile; log2 of the parts (CTAs) of a row tile
    // group norm in front (NORM kernels only): row = image * P + pixel
    const float *gamma, *beta, *stats;
    int64_t P, x_image;
    int G, per;
};

// Eight columns of a row as they lie in memory, in 8 / A accesses.
template <typename T, int A>
struct Raw {
    Vec<T, A> v[8 / A];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < 8 / A; ++i) v[i] = *reinterpret_cast<const Vec<T, A> *>(p + i * A);
    }
    __device__ __forceinline__ void load(const T *p, int count) {      // the first `count`, zeros after them
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i / A].v[i % A] = i < count ? p[i] : from_float<T>(0.f);
    }
    __device__ __forceinline__ float get(int i) const { return to_float(v[i / A].v[i % A]); }
};

// CTAs per SM that the registers of two row sets allow
template <typename T, int A> __host__ __device__ constexpr int quant_ctas() { return sizeof(T) == 4 || A == 1 ? 3 : 4; }

// A row set r0 is the rows r0, r0 + 32, r0 + 64, r0 + 96 of a row tile; a warp takes one, or two or four of narrow tiles, `lanes` lanes
// each.  A unit is a part of a tile, 8 warps' row sets: (row tile * parts + part) * col_tiles + column tile.  CTAs walk over the units and load the next one before they quantise the present
// one, so that loads are always in flight.
template <typename T, int A>
__global__ void __launch_bounds__(kWarps * 32, quant_ctas<T, A>()) mx4_quantize_kernel(QuantArgs a, unsigned parts) {
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int row_bytes = a.width / 2;
    const int in_row = lane & (a.lanes - 1);           // this lane's place in its row
    const int set = warp * (32 / a.lanes) + lane / a.lanes, sets_per_part = kWarps * (32 / a.lanes);
    int ct = static_cast<int>(blockIdx.x % static_cast<unsigned>(a.col_tiles));
    unsigned rest = blockIdx.x / static_cast<unsigned>(a.col_tiles);
    const int64_t down = 32 * a.ld;
    auto load = [&](int at_ct, unsigned at_rest, Row8<T, A> (&raw)[4]) {
        const int64_t row = static_cast<int64_t>(at_rest >> a.part_shift) * 128 + (at_rest & ((1 << a.part_shift) - 1)) * sets_per_part + set;
        const int64_t c = static_cast<int64_t>(at_ct) * a.width + in_row * 8;
        const T *src = static_cast<const T *>(a.x) + row * a.ld + c;
        if (c + 8 <= a.cols && row + 96 < a.rows) {
#pragma unroll
            for (int k = 0; k < 4; ++k, src += down) raw[k].load(src);
        } else if (c + 8 <= a.cols) {
#pragma unroll
            for (int k = 0; k < 4; ++k, src += down) {
                if (row + 32 * k < a.rows) raw[k].load(src);
                else raw[k].clear();
            }
        } else {
            const int count = static_cast<int>(max(int64_t(0), min(int64_t(8), a.cols - c)));
#pragma unroll
            for (int k = 0; k < 4; ++k, src += down) raw[k].load(src, row + 32 * k < a.rows ? count : 0);
        }
    };
    auto store = [&](const Row8<T, A> (&raw)[4]) {
        const int64_t rt = rest >> a.part_shift;
        const int r0 = static_cast<int>(rest & ((1 << a.part_shift) - 1)) * sets_per_part + set;
        const int64_t left = a.rows - rt * 128 - r0;   // rows of the set exist where 32 k < left
        const int64_t tile = rt * a.col_tiles + ct;
        // 32 rows further down the tile, a 16-byte unit keeps its place in the row
        int at = r0 * row_bytes + in_row * 4;
        at ^= ((at >> 7) & (a.width / 32 - 1)) << 4;
        uint8_t *codes_out = a.mx + tile * a.code_bytes + at;
        uint32_t sets[4];                              // lane of block b: scale byte of (row r0 + 32 k, b)
#pragma unroll
        for (int k = 0; k < 4; ++k, codes_out += 32 * row_bytes) {
            uint32_t codes;
            sets[k] = quantise8(raw[k].values(), raw[k].top(), codes);
            if (32 * k < left) *reinterpret_cast<uint32_t *>(codes_out) = codes;
        }
        // the first lane of every 16 of a row gathers the scale bytes of four blocks (two in the narrowest tiles): 16 bytes for four rows
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sets[k] |= __shfl_down_sync(0xffffffffu, sets[k], 4) << 8;
            const uint32_t upper = __shfl_down_sync(0xffffffffu, sets[k], 8) << 16;
            if (a.lanes > 8) sets[k] |= upper;
        }
        if ((in_row & 15) == 0 && left > 0)
            *reinterpret_cast<uint4 *>(a.mx + a.scales_at + tile * a.scale_bytes + (in_row >> 4) * 512 + r0 * 16) = make_uint4(sets[0], sets[1], sets[2], sets[3]);
    };
    pdl_wait();
    Row8<T, A> now[4], next[4];
    if (rest < parts) load(ct, rest, now);
    while (rest < parts) {                          // (the same for all threads of the CTA)
        int next_ct = ct + a.step_ct;
        unsigned next_rest = rest + a.step_rest;
        if (next_ct >= a.col_tiles) { next_ct -= a.col_tiles; ++next_rest; }
        if (next_rest < parts) load(next_ct, next_rest, next);
        store(now);
        ct = next_ct;
        rest = next_rest;
#pragma unroll
        for (int k = 0; k < 4; ++k) now[k] = next[k];
    }
}

// A group norm in front: blockIdx.x = (row tile * parts + part) * col_tiles + column tile.  The warps of a tile's `parts` CTAs (more than
// one where there are too few tiles for the SMs) walk over its 32 row sets; the constants of a lane's columns are loaded once per image.
template <typename T, int A, int ACT>
__global__ void __launch_bounds__(kWarps * 32) norm_quantize_kernel(QuantArgs a) {
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int ct = static_cast<int>(blockIdx.x % static_cast<unsigned>(a.col_tiles));
    const unsigned rest = blockIdx.x / static_cast<unsigned>(a.col_tiles);
    const int parts = 1 << a.part_shift, part = static_cast<int>(rest) & (parts - 1);
    const int64_t rt = a.row0 / 128 + (rest >> a.part_shift);
    const int in_row = lane & (a.lanes - 1), together = 32 / a.lanes;  // this lane's place in its row; row sets a warp takes at a time
    const int64_t c = static_cast<int64_t>(ct) * a.width + in_row * 8;
    const int row_bytes = a.width / 2;
    uint8_t *codes_out = a.mx + (rt * a.col_tiles + ct) * a.code_bytes;
    uint8_t *scales_out = a.mx + a.scales_at + (rt * a.col_tiles + ct) * a.scale_bytes;
    const int count = static_cast<int>(max(int64_t(0), min(int64_t(8), a.cols - c)));
    pdl_wait();
    float mean[8], rstd[8], gamma[8], beta[8];                         // of image `image`
    int image = -1;
    for (int first = (part * kWarps + warp) * together; first < 32; first += parts * kWarps * together) {
        if (rt * 128 + first >= a.rows) return;                        // (the same for the warp; higher rows of its sets do not exist either)
        const int r0 = first + lane / a.lanes;
        Raw<T, A> raw[4];
        bool on[4];
        int at_image[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t row = rt * 128 + r0 + 32 * k;
            on[k] = row >= a.row0 && row < a.rows;
            const T *src = static_cast<const T *>(a.x) + c;
            at_image[k] = static_cast<int>(static_cast<uint32_t>(row) / static_cast<uint32_t>(a.P));
            src += at_image[k] * a.x_image + (row - at_image[k] * a.P) * a.ld;
            if (on[k] && count == 8) raw[k].load(src);
            else raw[k].load(src, on[k] ? count : 0);
        }
        uint32_t sets[4];                                              // lane of block b: scale byte of (row r0 + 32 k, b)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = raw[k].get(j);
            if (on[k] && at_image[k] != image) {
                image = at_image[k];
                const float2 *st = reinterpret_cast<const float2 *>(a.stats) + static_cast<int64_t>(image) * a.G;
                int g = static_cast<int>(c) / a.per, left = a.per - static_cast<int>(c) % a.per;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool in = j < count;
                    const float2 f = in ? st[g] : make_float2(0.f, 0.f);
                    mean[j] = f.x;
                    rstd[j] = f.y;
                    gamma[j] = in ? a.gamma[c + j] : 0.f;
                    beta[j] = in ? a.beta[c + j] : 0.f;
                    if (--left == 0) { ++g; left = a.per; }
                }
            }
            if (on[k]) {
#pragma unroll
                for (int j = 0; j < 8; ++j)                            // as written: see activate_plain
                    v[j] = j < count ? activate_plain<ACT>(__fadd_rn(__fmul_rn(__fmul_rn(v[j] - mean[j], rstd[j]), gamma[j]), beta[j])) : 0.f;
            }
            uint32_t codes;
            sets[k] = quantise8(v, codes);
            if (on[k]) {
                int at = (r0 + 32 * k) * row_bytes + in_row * 4;
                at ^= ((at >> 7) & (a.width / 32 - 1)) << 4;
                *reinterpret_cast<uint32_t *>(codes_out + at) = codes;
            }
        }
        // as in the kernel above
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sets[k] |= __shfl_down_sync(0xffffffffu, sets[k], 4) << 8;
            const uint32_t upper = __shfl_down_sync(0xffffffffu, sets[k], 8) << 16;
            if (a.lanes > 8) sets[k] |= upper;
        }
        if ((in_row & 15) == 0) {
            uint32_t *to = reinterpret_cast<uint32_t *>(scales_out + (in_row >> 4) * 512 + r0 * 16);
            if (on[0] && on[1] && on[2] && on[3]) {
                *reinterpret_cast<uint4 *>(to) = make_uint4(sets[0], sets[1], sets[2], sets[3]);
            } else {                                                   // other rows of the set belong to another launch
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (on[k]) to[k] = sets[k];
            }
        }
    }
}

// The values of eight codes with the scale 2^(byte - 127): byte 0 is the subnormal 2^-127, 255 is NaN.
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return byte == 255 ? __uint_as_float(0x7fffffffu) : byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
}
// The value of one code: sign, two exponent bits, one mantissa bit; exponent 0 has the magnitudes 0 and 1/2.
__device__ __forceinline__ float value_of(uint32_t code, float scale) {
    const uint32_t e = (code >> 1) & 3, m = code & 1;
    const float magnitude = e ? __uint_as_float(((e + 126) << 23) | (m << 22)) : 0.5f * static_cast<float>(m);
    return (code & 8 ? -magnitude : magnitude) * scale;
}
__device__ __forceinline__ Fv<8> values_of(uint32_t codes, uint32_t byte) {
    const float scale = scale_value(byte);
    __half2 h[4];
    unpack8(codes, h);
    Fv<8> v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(h[j]);
        v.p[j] = mul_(pair_of(f.x, f.y), pair_of(scale, scale));
    }
    return v;
}

template <typename T, int A>
__global__ void __launch_bounds__(kWarps * 32) mx4_dequantize_kernel(QuantArgs a, T *out) {
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int ct = static_cast<int>(blockIdx.x % static_cast<unsigned>(a.col_tiles));
    const unsigned rest = blockIdx.x / static_cast<unsigned>(a.col_tiles);
    const int in_row = lane & (a.lanes - 1), sets_per_part = kWarps * (32 / a.lanes);
    const int64_t rt = rest >> a.part_shift;
    const int r0 = static_cast<int>(rest & ((1 << a.part_shift) - 1)) * sets_per_part + warp * (32 / a.lanes) + lane / a.lanes;
    const int64_t c = static_cast<int64_t>(ct) * a.width + in_row * 8;
    const int tile_row = a.width / 2;
    const uint8_t *codes_in = a.mx + (rt * a.col_tiles + ct) * a.code_bytes;
    const uint8_t *scales_in = a.mx + a.scales_at + (rt * a.col_tiles + ct) * a.scale_bytes;
    pdl_wait();
    if (c >= a.cols) return;
    uint32_t codes[4], scale[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (rt * 128 + r0 + 32 * k >= a.rows) continue;
        int at = (r0 + 32 * k) * tile_row + in_row * 4;
        at ^= ((at >> 7) & (a.width / 32 - 1)) << 4;
        codes[k] = *reinterpret_cast<const uint32_t *>(codes_in + at);
        scale[k] = scales_in[(in_row >> 4) * 512 + r0 * 16 + k * 4 + ((in_row >> 2) & 3)];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t row = rt * 128 + r0 + 32 * k;
        if (row >= a.rows) continue;
        const Fv<8> v = values_of(codes[k], scale[k]);
        T *dst = out + row * a.ld;
        if (c + 8 <= a.cols) {
            const Pack<T, 8> t = narrow<T, 8>(v);
            constexpr int kPer = sizeof(T) * A / 4;
#pragma unroll
            for (int i = 0; i < 8 / A; ++i) {
                Pack<T, A> part;
#pragma unroll
                for (int q = 0; q < kPer; ++q) part.w[q] = t.w[i * kPer + q];
                part.store(dst + c + i * A);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < a.cols) dst[c + j] = from_float<T>(v.get(j));
        }
    }
}

// The same for outputs that allow accesses of one element only: a lane takes every 32nd column, so that a warp still stores
// consecutive elements; eight lanes read the same word of codes.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) mx4_dequantize_single_kernel(QuantArgs a, T *out) {
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int ct = static_cast<int>(blockIdx.x % static_cast<unsigned>(a.col_tiles));
    const unsigned rest = blockIdx.x / static_cast<unsigned>(a.col_tiles);
    const int64_t row = static_cast<int64_t>(rest) * kWarps + warp, rt = row >> 7;        // a warp takes one row of a column tile
    const int r = static_cast<int>(row & 127), row_bytes = a.width / 2;
    const uint8_t *codes_in = a.mx + (rt * a.col_tiles + ct) * a.code_bytes;
    const uint8_t *scales_in = a.mx + a.scales_at + (rt * a.col_tiles + ct) * a.scale_bytes + (r & 31) * 16 + (r >> 5) * 4;
    const int cols = static_cast<int>(min(static_cast<int64_t>(a.width), a.cols - static_cast<int64_t>(ct) * a.width));
    pdl_wait();
    if (row >= a.rows) return;
    uint32_t word[8], scale[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = 32 * j + lane;
        if (32 * j >= a.width) continue;               // (the whole tile is there to read, whatever columns it holds)
        int at = r * row_bytes + (c >> 3) * 4;
        at ^= ((at >> 7) & (a.width / 32 - 1)) << 4;
        word[j] = *reinterpret_cast<const uint32_t *>(codes_in + at);
        scale[j] = scales_in[(c >> 7) * 512 + (j & 3)];
    }
    T *dst = out + row * a.ld + static_cast<int64_t>(ct) * a.width;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = 32 * j + lane;
        if (c < cols) dst[c] = from_float<T>(value_of((word[j] >> (4 * (c & 7))) & 15, scale_value(scale[j])));
    }
}

QuantArgs quant_args(const Mx4Shape &m, const void *x, int64_t ld, void *mx) {
    QuantArgs a{};
    a.x = x; a.mx = static_cast<uint8_t *>(mx);
    a.row0 = 0; a.rows = m.rows; a.cols = m.cols; a.ld = ld;
    a.scales_at = m.scales_at; a.width = m.width; a.col_tiles = static_cast<int>(m.col_tiles);
    a.code_bytes = m.code_bytes; a.scale_bytes = m.scale_bytes;
    a.P = 1; a.G = 1; a.per = 1;
    a.lanes = m.width / 8;
    a.part_shift = m.width == 256 ? 2 : m.width == 128 ? 1 : 0;
    return a;
}

// Units of a matrix whose CTAs take `sets` of the 32 row sets of a row tile; none for parts of the last row tile that have no rows.
unsigned quant_grid(const Mx4Shape &m, int sets) {
    const int64_t last = m.rows - (m.row_tiles - 1) * 128;
    const int64_t parts = (m.row_tiles - 1) * (32 / sets) + (last >= 32 ? 32 / sets : ceil_div(last, sets));
    return static_cast<unsigned>(parts * m.col_tiles);
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
    QuantArgs a = quant_args(m, x, ld, mx);
    const unsigned units = quant_grid(m, kWarps * (32 / a.lanes));
    return by_access(dtype, access_index(dtype, x, ld), [&](auto t, auto v) {
        const unsigned grid = std::min(units, static_cast<unsigned>(sm_count() * quant_ctas<decltype(t), v.value>()));
        a.step_ct = static_cast<int>(grid % m.col_tiles);
        a.step_rest = static_cast<int>(grid / m.col_tiles);
        return launch_pdl(mx4_quantize_kernel<decltype(t), v.value>, dim3(grid), dim3(kWarps * 32), 0, st, 1, a, static_cast<unsigned>(units / m.col_tiles));
    });
}

cudaError_t launch_norm_quantize(const NormShape &s, const Mx4Shape &m, const void *x, const float *gamma, const float *beta,
                                 const float *stats, int64_t row0, int64_t rows, void *mx, cudaStream_t st) {
    QuantArgs a = quant_args(m, x, s.x_pixel, mx);
    a.row0 = row0; a.rows = row0 + rows;
    a.gamma = gamma; a.beta = beta; a.stats = stats;
    a.P = s.P; a.x_image = s.x_image; a.G = s.G; a.per = s.C / s.G;
    const int64_t tiles = ceil_div(a.rows, 128) - row0 / 128;
    // (part_shift as quant_args left it: as many parts as there are warps' row sets in a tile)
    while (a.part_shift > 0 && (tiles * m.col_tiles << a.part_shift) > 4 * sm_count()) --a.part_shift;
    return by_access(s.dtype, access_index(s.dtype, x, s.x_pixel, s.x_image), [&](auto t, auto v) {
        return by_act(s.act, [&](auto c) {
            return launch_pdl(norm_quantize_kernel<decltype(t), v.value, c.value>, dim3(static_cast<unsigned>(tiles * m.col_tiles << a.part_shift)), dim3(kWarps * 32), 0, st, 1, a);
        });
    });
}

cudaError_t launch_mx4_dequantize(const Mx4Shape &m, const void *mx, void *out, int dtype, int64_t ld, cudaStream_t st) {
    const QuantArgs a = quant_args(m, nullptr, ld, const_cast<void *>(mx));
    return by_access(dtype, access_index(dtype, out, ld), [&](auto t, auto v) {
        using T = decltype(t);
        if constexpr (sizeof(T) * v.value < 4 || v.value == 1)
            return launch_pdl(mx4_dequantize_single_kernel<T>, dim3(static_cast<unsigned>(ceil_div(m.rows, kWarps) * m.col_tiles)), dim3(kWarps * 32), 0, st, 1, a, static_cast<T *>(out));
        else
            return launch_pdl(mx4_dequantize_kernel<T, v.value>, dim3(quant_grid(m, kWarps * (32 / a.lanes))), dim3(kWarps * 32), 0, st, 1, a, static_cast<T *>(out));
    });
}

}  // namespace patdnn

// Device helpers of the 8-bit blocks, and the way a row's columns are spread over lanes.
#pragma once
#include "ops_device.cuh"

namespace patdnn {
namespace {

// Scale byte of a block from the bits of its largest magnitude (sign clear), and the factor 1 / scale: the smallest power of two, at least
// 2^-127, at which the block's magnitudes are at most 448 (1.75 * 2^8).
__device__ __forceinline__ uint32_t scale8_of(uint32_t amax_bits, float &inverse) {
    const uint32_t field = amax_bits >> 23;            // biased exponent; 0 for zero and subnormals
    if (field == 255) {
        inverse = 0.f;
        return 255;
    }
    const int e = static_cast<int>(field) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u);
    const uint32_t byte = e > 0 ? e : 0;               // at most 247
    inverse = __uint_as_float((254 - byte) << 23);     // 2^(127 - byte), always normal
    return byte;
}
// The value of a scale byte: 0 is the subnormal 2^-127, 255 is NaN.
__device__ __forceinline__ float scale8_value(uint32_t byte) {
    return byte == 255 ? __uint_as_float(0x7fffffffu) : byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
}
// Codes of two values, the first in the lower byte; nearest even (magnitudes are at most 448).
__device__ __forceinline__ uint32_t codes2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// The two values of two codes before scaling, exact in half.
__device__ __forceinline__ float2 values2(uint32_t codes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(codes)));
    return __half22float2(*reinterpret_cast<__half2 *>(&r));
}
__device__ __forceinline__ float max_abs(float a, float b) {           // a NaN stays one
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Byte of column c, row r (of its row tile) inside a tile.
__device__ __forceinline__ int mx8_place(int r, int c) { return r * 128 + ((((c >> 4) ^ r) & 7) << 4) + (c & 15); }
// Byte of the scale of (row r of its row tile, column tile t) inside the group's 512 bytes.
__device__ __forceinline__ int mx8_scale_place(int r, int t) { return (r & 31) * 16 + (r >> 5) * 4 + (t & 3); }

template <int A> __device__ __forceinline__ void store_codes(uint8_t *to, const float *v, float inverse) {
    if constexpr (A == 8) {
        *reinterpret_cast<uint2 *>(to) = make_uint2(codes2(v[0] * inverse, v[1] * inverse) | codes2(v[2] * inverse, v[3] * inverse) << 16,
                                                    codes2(v[4] * inverse, v[5] * inverse) | codes2(v[6] * inverse, v[7] * inverse) << 16);
    } else if constexpr (A == 4) {
        *reinterpret_cast<uint32_t *>(to) = codes2(v[0] * inverse, v[1] * inverse) | codes2(v[2] * inverse, v[3] * inverse) << 16;
    } else if constexpr (A == 2) {
        *reinterpret_cast<uint16_t *>(to) = static_cast<uint16_t>(codes2(v[0] * inverse, v[1] * inverse));
    } else {
        *to = static_cast<uint8_t>(codes2(v[0] * inverse, 0.f));
    }
}

// L lanes (all of a warp, or a half or a quarter of it) take consecutive columns of a row in accesses of A elements per lane: access j, lane l,
// element e is column (L j + l) A + e, so that every access is one contiguous piece whatever A is.
// E elements per lane, from `p` (the first column); `left` of the row's columns are there, zeros behind them.
template <typename T, int A, int E, int L = 32>
struct Strip {
    static constexpr int NA = E / A;
    Pack<T, A> v[NA];
    __device__ __forceinline__ void load(const T *p, int left) {
        const int lane = threadIdx.x & (L - 1);
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            const int c = (L * j + lane) * A;
            if (c + A <= left) {
                v[j].load(p + c);
            } else {
#pragma unroll
                for (int k = 0; k < static_cast<int>(sizeof(v[j].w) / 4); ++k) v[j].w[k] = 0;
                if constexpr (A > 1) {
                    if (c >= left) continue;           // (2072 x 12000 bf16, norm: 43 us; 65 where warps without a lane that is in part there went through what follows)
#pragma unroll
                    for (int e = 0; e < A; ++e)
                        if (c + e < left) {
                            if constexpr (sizeof(T) == 4) v[j].w[e] = reinterpret_cast<const uint32_t *>(p)[c + e];
                            else v[j].w[e / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[c + e]) << (16 * (e & 1));
                        }
                }
            }
        }
    }
    // The same for A = 16 bytes from rows that are aligned to their elements only: a lane reads the aligned 16 bytes in which its own begin, takes the
    // next ones from the next lane and shifts.  Only 16-byte units that hold an element of the row are read.  All lanes of the warp call it.
    __device__ __forceinline__ void load_any(const T *p, int left) {
        static_assert(sizeof(T) * A == 16, "whole units");
        const int lane = threadIdx.x & (L - 1);
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            const T *from = p + j * L * A;
            const int here = left - j * L * A, over = static_cast<int>(reinterpret_cast<uintptr_t>(from) & 15);          // bytes in front of the row's
            const int bytes = here * static_cast<int>(sizeof(T)), first = lane * 16 - over;
            const uint4 *unit = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(from) + first);
            uint4 a = make_uint4(0, 0, 0, 0), b = a;
            if (first < bytes) a = *unit;
            if (lane == L - 1 && over && first + 16 < bytes) b = unit[1];
            uint32_t w[8] = {a.x, a.y, a.z, a.w, 0, 0, 0, 0};
            const uint32_t tail[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t t = __shfl_down_sync(0xffffffffu, w[i], 1, L);
                w[4 + i] = lane == L - 1 ? tail[i] : t;
            }
            if (over & 8) {
#pragma unroll
                for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
            }
            if (over & 4) {
#pragma unroll
                for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[j].w[i] = __funnelshift_r(w[i], w[i + 1], (over & 2) * 8);
            const int there = here - lane * A;         // of the lane's elements
            if (there < A) {
#pragma unroll
                for (int e = 0; e < A; ++e)
                    if (e >= there) {
                        if constexpr (sizeof(T) == 4) v[j].w[e] = 0;
                        else v[j].w[e / 2] &= e & 1 ? 0xffffu : 0xffff0000u;
                    }
            }
        }
    }
    __device__ __forceinline__ void store(T *p, int left) const {
        const int lane = threadIdx.x & (L - 1);
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            const int c = (L * j + lane) * A;
            if (c + A <= left) {
                v[j].store(p + c);
            } else if constexpr (A > 1) {
                if (c >= left) continue;
#pragma unroll
                for (int e = 0; e < A; ++e)
                    if (c + e < left) {
                        if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t *>(p)[c + e] = v[j].w[e];
                        else reinterpret_cast<uint16_t *>(p)[c + e] = static_cast<uint16_t>(v[j].w[e / 2] >> (16 * (e & 1)));
                    }
            }
        }
    }
    __device__ __forceinline__ void widen_to(float (&f)[E]) const {
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            const Fv<A> t = widen<T, A>(v[j]);
#pragma unroll
            for (int e = 0; e < A; ++e) f[j * A + e] = t.get(e);
        }
    }
    __device__ __forceinline__ void narrow_from(const float (&f)[E]) {
#pragma unroll
        for (int j = 0; j < NA; ++j) v[j] = narrow<T, A>(Fv<A>::make([&](int e) { return f[j * A + e]; }));
    }
};

// The strip of a row as 8-bit blocks.  `codes`: the row's place in its first column tile (tile base, row 0 of the tile), `scales`:
// the row tile's scales; `r`: row of the row tile; c0: the strip's first column (a multiple of 128); `padded`: columns up to the end of the
// last column tile, which are written as far as the strip goes.
template <int A, int E, int L>
__device__ __forceinline__ void store_blocks(uint8_t *codes, uint8_t *scales, int r, int64_t c0, int64_t padded, const float (&v)[E]) {
    constexpr int NA = E / A, ONE = L * A >= 128 ? 1 : 128 / (L * A), PER = ONE < NA ? ONE : NA;   // accesses to a block (256 columns: two blocks to an access)
    constexpr int LANES = L * A > 128 ? 128 / A : L;   // lanes that share a block
    const int lane = threadIdx.x & (L - 1);
#pragma unroll
    for (int q = 0; q < NA; q += PER) {
        float m = max_abs(v[q * A], v[q * A + A * PER - 1]);
#pragma unroll
        for (int e = 1; e < A * PER - 1; ++e) m = max_abs(m, v[q * A + e]);
        uint32_t top = magnitude_bits(m);
#pragma unroll
        for (int s = 1; s < LANES; s *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
        float inverse;
        const uint32_t byte = scale8_of(top, inverse);
#pragma unroll
        for (int j = q; j < q + PER; ++j) {
            const int64_t c = c0 + (L * j + lane) * A;
            if (c >= padded) continue;
            const int64_t t = c >> 7;
            store_codes<A>(codes + t * (128 * 128) + mx8_place(r, static_cast<int>(c & 127)), v + j * A, inverse);
            if (j == q && (lane & (LANES - 1)) == 0) scales[(t >> 2) * 512 + mx8_scale_place(r, static_cast<int>(t))] = static_cast<uint8_t>(byte);
        }
    }
}

}  // namespace

// elements per access: 16 bytes where addresses and strides allow, else two, else one
inline int strip_width(int dtype, std::initializer_list<const void *> pointers, std::initializer_list<int64_t> strides) {
    const int e = elem_bytes(dtype);
    for (int v : {16 / e, 2}) {
        bool ok = true;
        for (const void *p : pointers) ok = ok && reinterpret_cast<uintptr_t>(p) % (static_cast<unsigned>(v) * e) == 0;
        for (int64_t s : strides) ok = ok && s % v == 0;
        if (ok) return v;
    }
    return 1;
}
// f(T{}, std::integral_constant<int, A>)
template <typename F> cudaError_t by_strip(int dtype, int width, F f) {
    if (dtype == PATDNN_F32) return width == 4 ? f(float{}, std::integral_constant<int, 4>{}) : width == 2 ? f(float{}, std::integral_constant<int, 2>{}) : f(float{}, std::integral_constant<int, 1>{});
    if (dtype == PATDNN_F16) return width == 8 ? f(__half{}, std::integral_constant<int, 8>{}) : width == 2 ? f(__half{}, std::integral_constant<int, 2>{}) : f(__half{}, std::integral_constant<int, 1>{});
    return width == 8 ? f(__nv_bfloat16{}, std::integral_constant<int, 8>{}) : width == 2 ? f(__nv_bfloat16{}, std::integral_constant<int, 2>{}) : f(__nv_bfloat16{}, std::integral_constant<int, 1>{});
}

}  // namespace patdnn

// Device helpers of the operators: vector access for the three storage types, and the activations.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "../../include/patdnn.h"

namespace patdnn {
namespace {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// V consecutive elements, loaded and stored as one access of V * sizeof(T) bytes (a power of two, at most 16).
template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T v[V];
};

// The same as 32-bit words (a single 16-bit element sits in the lower half), for code that takes the elements out by shifts.
template <typename T, int V>
struct Pack {
    static constexpr int kBytes = sizeof(T) * V;
    uint32_t w[kBytes < 4 ? 1 : kBytes / 4];
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (kBytes == 16) { const uint4 t = *reinterpret_cast<const uint4 *>(p); w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w; }
        else if constexpr (kBytes == 8) { const uint2 t = *reinterpret_cast<const uint2 *>(p); w[0] = t.x; w[1] = t.y; }
        else if constexpr (kBytes == 4) w[0] = *reinterpret_cast<const uint32_t *>(p);
        else w[0] = *reinterpret_cast<const uint16_t *>(p);
    }
    __device__ __forceinline__ void load_shared(uint32_t addr) {       // address as in PTX
        if constexpr (kBytes == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
        else if constexpr (kBytes == 8) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(addr) : "memory");
        else if constexpr (kBytes == 4) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(addr) : "memory");
        else {
            uint16_t t;
            asm volatile("ld.shared.b16 %0, [%1];" : "=h"(t) : "r"(addr) : "memory");
            w[0] = t;
        }
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (kBytes == 16) *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (kBytes == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t *>(p) = w[0];
        else *reinterpret_cast<uint16_t *>(p) = static_cast<uint16_t>(w[0]);
    }
};

// V fp32 values.  Pairs are held in 64-bit registers and go through the packed instructions (one issue slot for two results, each
// rounded as alone).
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 split(uint64_t p) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
    return r;
}
template <int V>
struct Fv {
    uint64_t p[V / 2];
    __device__ __forceinline__ static Fv all(float x) {
        Fv r;
#pragma unroll
        for (int j = 0; j < V / 2; ++j) r.p[j] = pair_of(x, x);
        return r;
    }
    template <typename F> __device__ __forceinline__ static Fv make(F f) {      // f(j) for j = 0 .. V-1
        Fv r;
#pragma unroll
        for (int j = 0; j < V / 2; ++j) r.p[j] = pair_of(f(2 * j), f(2 * j + 1));
        return r;
    }
    __device__ __forceinline__ float get(int j) const { return j & 1 ? split(p[j / 2]).y : split(p[j / 2]).x; }
    template <typename F> __device__ __forceinline__ Fv map(F f) const {
        Fv r;
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            const float2 t = split(p[j]);
            r.p[j] = pair_of(f(t.x), f(t.y));
        }
        return r;
    }
};
template <>
struct Fv<1> {
    float p[1];
    __device__ __forceinline__ static Fv all(float x) { return Fv{{x}}; }
    template <typename F> __device__ __forceinline__ static Fv make(F f) { return Fv{{f(0)}}; }
    __device__ __forceinline__ float get(int) const { return p[0]; }
    template <typename F> __device__ __forceinline__ Fv map(F f) const { return Fv{{f(p[0])}}; }
};
__device__ __forceinline__ float fma_(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float add_(float a, float b) { return a + b; }
__device__ __forceinline__ float mul_(float a, float b) { return a * b; }
__device__ __forceinline__ uint64_t fma_(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul_(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
template <int V> __device__ __forceinline__ Fv<V> fma(const Fv<V> &a, const Fv<V> &b, const Fv<V> &c) {
    Fv<V> r;
#pragma unroll
    for (int j = 0; j < (V + 1) / 2; ++j) r.p[j] = fma_(a.p[j], b.p[j], c.p[j]);
    return r;
}
template <int V> __device__ __forceinline__ Fv<V> operator+(const Fv<V> &a, const Fv<V> &b) {
    Fv<V> r;
#pragma unroll
    for (int j = 0; j < (V + 1) / 2; ++j) r.p[j] = add_(a.p[j], b.p[j]);
    return r;
}
template <int V> __device__ __forceinline__ Fv<V> operator*(const Fv<V> &a, const Fv<V> &b) {
    Fv<V> r;
#pragma unroll
    for (int j = 0; j < (V + 1) / 2; ++j) r.p[j] = mul_(a.p[j], b.p[j]);
    return r;
}
template <typename T, int V> __device__ __forceinline__ Fv<V> widen(const Pack<T, V> &x) {
    Fv<V> r;
    if constexpr (sizeof(T) == 4) {
        if constexpr (V == 1) r.p[0] = __uint_as_float(x.w[0]);
        else
#pragma unroll
            for (int j = 0; j < V / 2; ++j) r.p[j] = pair_of(__uint_as_float(x.w[2 * j]), __uint_as_float(x.w[2 * j + 1]));
    } else {
#pragma unroll
        for (int j = 0; j < (V + 1) / 2; ++j) {
            float lo, hi;
            if constexpr (std::is_same<T, __half>::value) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&x.w[j]));
                lo = f.x; hi = f.y;
            } else {                                   // bfloat16 is the upper half of a float
                lo = __uint_as_float(x.w[j] << 16);
                hi = __uint_as_float(x.w[j] & 0xffff0000u);
            }
            if constexpr (V == 1) r.p[0] = lo;
            else r.p[j] = pair_of(lo, hi);
        }
    }
    return r;
}
template <typename T, int V> __device__ __forceinline__ Pack<T, V> narrow(const Fv<V> &x) {
    Pack<T, V> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < V; ++j) r.w[j] = __float_as_uint(x.get(j));
    } else {
#pragma unroll
        for (int j = 0; j < (V + 1) / 2; ++j) {
            const float2 f = make_float2(x.get(2 * j), V == 1 ? 0.f : x.get(2 * j + 1));
            if constexpr (std::is_same<T, __half>::value) {
                const __half2 h = __floats2half2_rn(f.x, f.y);
                r.w[j] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
                r.w[j] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
    return r;
}

// 1 / (1 + exp(-z)).  2^x and the reciprocal are the hardware's approximations (2 ulp, tiny results flushed to zero): 2^x overflows to
// infinity for z < -88, whose reciprocal is 0, the limit.
__device__ __forceinline__ float sigmoid(float z) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
}
// The same for pairs with one reciprocal for two: 1/a = b / (a b).  It takes a quarter off the work of the special-function unit (the
// elementwise pass over 2 x 512 x 512 x 128 16-bit values: 39 us with 1.5 of its operations per element, 41 with 2; at 6.9 TB/s memory is
// what bounds it then, the unit is at 63 %).  Arguments below -43 are
// taken as -43, so that the product of two denominators stays in range, and a NaN as -43 too, so that it does not reach its neighbour:
// it comes back with z itself.
__device__ __forceinline__ float at_least(float z) {   // max(z, -43); NaN stays NaN
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(z), "f"(-43.f));
    return r;
}
template <int V> __device__ __forceinline__ Fv<V> sigmoid(const Fv<V> &z) {
    Fv<V> s;
    if constexpr (V == 1) {
        s.p[0] = sigmoid(z.p[0]);
    } else {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            const float2 c = split(z.p[j]);
            const float2 t = split(mul_(pair_of(fmaxf(c.x, -43.f), fmaxf(c.y, -43.f)), pair_of(-1.4426950408889634f, -1.4426950408889634f)));
            float e0, e1, r;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(t.x));
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(t.y));
            const float2 d = split(add_(pair_of(e0, e1), pair_of(1.f, 1.f)));
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d.x * d.y));
            s.p[j] = mul_(pair_of(r, r), pair_of(d.y, d.x));
        }
    }
    return s;
}
// z sigmoid(z) below -43 is taken as its value there, -9e-18
template <int ACT, int V> __device__ __forceinline__ Fv<V> activate(const Fv<V> &z) {
    if constexpr (ACT == PATDNN_ACT_RELU) return z.map([](float v) { return v < 0.f ? 0.f : v; });      // NaN stays NaN
    else if constexpr (ACT == PATDNN_ACT_SILU) return z.map([](float v) { return at_least(v); }) * sigmoid<V>(z);
    else return z;
}
// g * act'(z); ReLU has slope 0 at z = 0 and passes a NaN of z on
template <int ACT, int V> __device__ __forceinline__ Fv<V> through(const Fv<V> &g, const Fv<V> &z) {
    if constexpr (ACT == PATDNN_ACT_RELU) {
        return Fv<V>::make([&](int j) { return z.get(j) > 0.f ? g.get(j) : (z.get(j) <= 0.f ? 0.f : z.get(j)); });
    } else if constexpr (ACT == PATDNN_ACT_SILU) {     // s (1 + z (1 - s)) = s + (z s) (1 - s)
        // (the gradient is bound by its instructions: a reciprocal each takes fewer of them, 56 us against 57)
        const Fv<V> s = z.map([](float v) { return sigmoid(v); });
        return g * fma(z * s, fma(s, Fv<V>::all(-1.f), Fv<V>::all(1.f)), s);
    } else {
        return g;
    }
}
template <int ACT> __device__ __forceinline__ float activate1(float z) {
    if constexpr (ACT == PATDNN_ACT_RELU) return z < 0.f ? 0.f : z;
    else if constexpr (ACT == PATDNN_ACT_SILU) return z * sigmoid(z);
    else return z;
}
// The activation as it is written, in correctly rounded or near-exact steps: values that are held in 4 bits afterwards jump at the middles
// between two codes, so they are formed as a plain evaluation in fp32 forms them.
template <int ACT> __device__ __forceinline__ float activate_plain(float z) {
    if constexpr (ACT == PATDNN_ACT_RELU) return z < 0.f ? 0.f : z;
    else if constexpr (ACT == PATDNN_ACT_SILU) return __fdiv_rn(z, 1.f + expf(-z));
    else return z;
}
__device__ __forceinline__ float activate(float z, int act) {
    if (act == PATDNN_ACT_RELU) return z < 0.f ? 0.f : z;
    if (act == PATDNN_ACT_SILU) return z * sigmoid(z);
    return z;
}
// f(std::integral_constant<int, ACT>)
template <typename F> cudaError_t by_act(int act, F f) {
    if (act == PATDNN_ACT_RELU) return f(std::integral_constant<int, PATDNN_ACT_RELU>{});
    if (act == PATDNN_ACT_SILU) return f(std::integral_constant<int, PATDNN_ACT_SILU>{});
    return f(std::integral_constant<int, PATDNN_ACT_NONE>{});
}

// The codes of eight values, the first in the lowest four bits; nearest even, magnitudes above 6 become 6.
__device__ __forceinline__ uint32_t pack8(const Fv<8> &x, float factor) {
    uint32_t r;
    const Fv<8> v = x * Fv<8>::all(factor);
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(v.get(0)), "f"(v.get(1)), "f"(v.get(2)), "f"(v.get(3)), "f"(v.get(4)), "f"(v.get(5)),
          "f"(v.get(6)), "f"(v.get(7)));
    return r;
}
// The eight values that such a word stands for, before scaling (exact in half).
__device__ __forceinline__ void unpack8(uint32_t codes, __half2 (&h)[4]) {
    uint32_t r[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = *reinterpret_cast<__half2 *>(&r[i]);
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

// Bits of the largest magnitude of eight values; a NaN among them gives a NaN.
__device__ __forceinline__ uint32_t top8(const float (&v)[8]) {
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(v[0]), "f"(v[1]), "f"(v[2]));
    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(v[3]), "f"(v[4]));
    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(v[5]), "f"(v[6]));
    asm("max.NaN.abs.f32 %0, %0, %1, %1;" : "+f"(m) : "f"(v[7]));
    return __float_as_uint(m) & 0x7fffffffu;
}
// Eight values of one lane -> its 4 bytes of codes; returns the block's scale byte (the same in the four lanes of a block).
// `top`: bits of the lane's largest magnitude, sign clear (magnitudes compare like their bits, a NaN is above infinity).
__device__ __forceinline__ uint32_t quantise8(const Fv<8> &v, uint32_t top, uint32_t &codes) {
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    float inverse;
    const uint32_t scale = scale_of(top, inverse);
    codes = pack8(v, inverse);                         // a block that is not finite: any codes, its scale is NaN
    return scale;
}
__device__ __forceinline__ uint32_t quantise8(const float (&v)[8], uint32_t &codes) {
    return quantise8(Fv<8>::make([&](int j) { return v[j]; }), top8(v), codes);
}

// Eight columns of a row as 32-bit words, in accesses of A elements.
template <typename T, int A>
struct Row8 {
    static constexpr int kWords = 8 * sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (sizeof(T) * A >= 4) {
            constexpr int kPer = sizeof(T) * A / 4;    // words per access
#pragma unroll
            for (int i = 0; i < 8 / A; ++i) {
                Pack<T, A> t;
                t.load(p + i * A);
#pragma unroll
                for (int k = 0; k < kPer; ++k) w[i * kPer + k] = t.w[k];
            }
        } else {
            load(p, 8);
        }
    }
    __device__ __forceinline__ void load(const T *p, int count) {      // the first `count`, zeros after them
        clear();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) {
                if constexpr (sizeof(T) == 4) w[i] = reinterpret_cast<const uint32_t *>(p)[i];
                else w[i / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[i]) << (16 * (i & 1));
            }
    }
    __device__ __forceinline__ Fv<8> values() const {
        Pack<T, 8> t;
#pragma unroll
        for (int i = 0; i < kWords; ++i) t.w[i] = w[i];
        return widen<T, 8>(t);
    }
    // bits of the largest magnitude; two 16-bit values are compared at a time
    __device__ __forceinline__ uint32_t top() const {
        if constexpr (sizeof(T) == 4) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
            return top8(v);
        } else {
            uint32_t t = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
            t = max(t & 0xffffu, t >> 16);
            if constexpr (std::is_same<T, __nv_bfloat16>::value) return t << 16;
            const uint16_t one = static_cast<uint16_t>(t);
            return __float_as_uint(__half2float(*reinterpret_cast<const __half *>(&one)));
        }
    }
};

}  // namespace
}  // namespace patdnn

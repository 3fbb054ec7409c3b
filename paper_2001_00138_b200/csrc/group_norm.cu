// Group norm with an activation over channels-last tensors, and its gradient.
//
//   x [N][P][C], group g of channel c = c / (C / G); mean, var over the P * C/G values of (n, g), rstd = 1/sqrt(var + eps)
//   d = x - mean, z = d * (rstd * gamma_c) + beta_c, y = act(z)
//   gradient: dz = dy * act'(z); A_nc = sum_p dz, B_nc = rstd * sum_p dz * d; dbeta = sum_n A, dgamma = sum_n B;
//   with m = P * C/G, s1 = sum_{c in g} gamma_c A_nc / m, s2 = sum_{c in g} gamma_c B_nc / m:
//   dx = rstd * gamma_c * dz - rstd * s1 - d * rstd^2 * s2
//
// Both are bound by HBM: the forward's floor is one read of x and one write of y, the gradient's one read of x and dy and one
// write of dx.  Two forms:
//   resident  a thread-block cluster (up to 8 CTAs) owns a slab of whole groups of one image, keeps it in shared memory
//             while the statistics are formed and joined over distributed shared memory, and writes the result from there: one
//             launch, every value read once.
//   two-pass  images whose slabs do not fit, or for which one launch would keep too few SMs busy: partial statistics per (chunk of
//             pixels, group), a small kernel that joins them, and an elementwise pass that reads x again.  Images are taken in runs of
//             at most kRunBytes, and the second pass walks backwards, so that part of that read comes from L2.
// Measured: forward 2 x 512 x 512 x 128 bf16 SiLU 75 us (statistics 29.5 us, 4.6 TB/s; join 3; elementwise 39, 6.9 TB/s: memory), floor 41
// us, of two passes 61; gradient 32 x 56 x 56 x 256 bf16 SiLU 56 us (26 + 4.6 + 27), floor 24 us: half of the issue slots at 31 % of the
// warps (80 registers, some spilled), latency more than anything; resident forward 32 x 56 x 56 x 64 fp16 ReLU 10.8 us, floor 3.9, and into
// 4-bit rows 16 us, with eight warps per SM and 39 % of the issue slots: latency.
// All sums are fp32 per thread, joined in fp64 and in a fixed order, so that mean and variance are rounded to fp32 about once: values that
// are held in 4 bits afterwards jump, and every rounding less is a jump less (100352 x 64: 0.36 values per call differ from
// a plain fp32 evaluation's, 0.57 with joins in fp32).  Variances are never formed as a difference of two large sums: a thread sums (x - m)
// and (x - m)^2 around its own running mean m, a few pixels at a time, and partial results are joined by their means.
#include "ops.hpp"

#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "kernels.hpp"
#include "ops_device.cuh"

namespace patdnn {

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 256;

struct NormArgs {
    const void *x, *dy;
    void *y;                                // dx in the gradient; nullptr: statistics only
    const float *gamma, *beta, *stats_in;
    float *stats_out, *dgamma, *dbeta;
    float *ws;
    unsigned *counters;
    int64_t x_pixel, x_image, y_pixel, y_image, P, chunk;
    int N, C, G, per;                       // per = C / G
    int slab, slabs, cluster, chunks;
    int parts;                              // two-pass: slabs that share a group (1: slabs hold whole groups)
    int n0;                                 // two-pass: first image of the run
    float eps, inv_count;
    double inv_values;                      // the same in fp64
    uint8_t *mx;                            // 4-bit output (resident form)
    int64_t mx_scales;
    int mx_width, mx_col_tiles;
};

template <typename F> __device__ __forceinline__ F warp_sum(F v) {     // float or double
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Running mean and sum of squared deviations of V channels over the pixels a thread visits, up to kMerge at a time:
// the sums are taken around the running mean (around the first pixel in the first run), so a run of b values loses
// at most about b rounding errors of the largest deviation.  16 rather than 32: the rstd of 1024 groups of 6272 values then differ from the
// once-rounded ones in 5 % instead of 13 % (squares of 16-bit values often tie, so their errors do not average out), for 0.1 us of 33.
constexpr int kMerge = 16;
template <int V>
struct Moments {
    Fv<V> mean, m2, s1, s2;
    int n;
    __device__ __forceinline__ void clear() {
        n = 0;
        mean = m2 = Fv<V>::all(0.f);
    }
    template <typename T>
    __device__ __forceinline__ void begin(const Pack<T, V> &first) {
        s1 = s2 = Fv<V>::all(0.f);
        if (n == 0) mean = widen<T, V>(first);         // (NaN and infinities included: they end in every result)
    }
    template <typename T>
    __device__ __forceinline__ void take(const Pack<T, V> &x) {
        const Fv<V> d = fma(mean, Fv<V>::all(-1.f), widen<T, V>(x));
        s1 = s1 + d;
        s2 = fma(d, d, s2);
    }
    __device__ __forceinline__ void end(int count) {
        n += count;
        const Fv<V> inv = Fv<V>::all(__fdividef(1.f, static_cast<float>(n)));
        const Fv<V> shift = s1 * inv;
        mean = mean + shift;
        m2 = (m2 + fma(s1 * Fv<V>::all(-1.f), shift, s2)).map([](float m) { return m < 0.f ? 0.f : m; });   // NaN stays NaN
    }
};

// Groups of V neighbouring channels, the first of which is c.
template <int V>
struct Groups {
    int g[V];
    __device__ __forceinline__ Groups(int c, int per) {
        int at = c / per, in = c - at * per;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            g[j] = at;
            if (++in == per) { in = 0; ++at; }
        }
    }
};

// Position of this thread in its CTA's slab: vector column `col` (V channels), pixel row `row` of `rows`.
struct Place {
    int col, row, rows;
    bool on;
};
template <int V>
__device__ __forceinline__ Place place_of(int channels) {
    Place q;
    const int cols = channels / V;
    q.rows = kThreads / cols;
    q.col = threadIdx.x % cols;
    q.row = threadIdx.x / cols;
    q.on = q.row < q.rows;
    return q;
}
// A thread's own pixels q.row, q.row + q.rows, ... of a slab, brought to shared memory by asynchronous copies kDepth batches ahead of
// their use, so that the bytes in flight cost no registers.  Every thread reads back only what it copied itself: no barrier.
// KEEP: they stay in `tile` [pixels][channels]; otherwise they pass through a ring of kDepth batches, [batch][pixel of it][thread].
// TENSORS (one or two) share at most 256 bytes per thread, so that three CTAs fit an SM.
template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t to, const void *from) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ uint32_t shared_address(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LATER> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LATER) : "memory"); }

template <typename T, int V, bool KEEP, int TENSORS>
struct Stream {
    static constexpr int kBytes = sizeof(T) * V;
    static constexpr int kBatch = KEEP ? 8 : 4 / TENSORS;      // pixels a thread takes at a time
    static constexpr int kDepth = 4;
    const T *src;
    int64_t src_step;                                  // elements between this thread's pixels
    uint32_t to, from, step, ring, end;                // shared memory: next pixel to copy, next to read, distance; the ring's bounds
    int left;                                          // pixels still to copy
    // BACK: from the thread's last pixel to its first
    template <bool BACK = false>
    __device__ __forceinline__ void begin(const T *first, int64_t stride, int pixels, const Place &q, T *space, int channels, int col) {
        src = first + q.row * stride;
        src_step = q.rows * stride;
        step = (KEEP ? q.rows * channels : kThreads * V) * sizeof(T);
        ring = shared_address(KEEP ? space + q.row * channels + col : space + threadIdx.x * V);
        end = ring + kDepth * kBatch * step;
        to = from = ring;
        left = (pixels - q.row + q.rows - 1) / q.rows;
        if constexpr (BACK) {
            src += (left - 1) * src_step;
            src_step = -src_step;
        }
    }
    __device__ __forceinline__ void copy() {           // one batch
        if (left >= kBatch) {
            if constexpr (kBytes >= 4) {
#pragma unroll
                for (int u = 0; u < kBatch; ++u, src += src_step, to += step) copy_async<kBytes>(to, src);
            } else {                                   // two bytes are too few for an asynchronous copy: all loads before the first store
                uint16_t t[kBatch];
#pragma unroll
                for (int u = 0; u < kBatch; ++u, src += src_step) t[u] = *reinterpret_cast<const uint16_t *>(src);
#pragma unroll
                for (int u = 0; u < kBatch; ++u, to += step) asm volatile("st.shared.b16 [%0], %1;" ::"r"(to), "h"(t[u]) : "memory");
            }
        } else {
            for (int u = 0; u < left; ++u, src += src_step, to += step) {
                if constexpr (kBytes >= 4) copy_async<kBytes>(to, src);
                else asm volatile("st.shared.b16 [%0], %1;" ::"r"(to), "h"(*reinterpret_cast<const uint16_t *>(src)) : "memory");
            }
        }
        left -= kBatch;
        if (!KEEP && to == end) to = ring;
    }
    __device__ __forceinline__ Pack<T, V> peek() const {
        Pack<T, V> v;
        v.load_shared(from);
        return v;
    }
    __device__ __forceinline__ Pack<T, V> get() {
        const Pack<T, V> v = peek();
        from += step;
        return v;
    }
    __device__ __forceinline__ void wrap() {           // after each batch read
        if (!KEEP && from == end) from = ring;
    }
};

// Moments of a thread's pixels.
template <typename T, int V, bool KEEP>
__device__ __forceinline__ void moments_of(Stream<T, V, KEEP, 1> &x, Moments<V> &m) {
    constexpr int kBatch = Stream<T, V, KEEP, 1>::kBatch, kDepth = Stream<T, V, KEEP, 1>::kDepth;
    m.clear();
    int count = x.left;                                // pixels still to read
#pragma unroll
    for (int b = 0; b < kDepth; ++b) { x.copy(); copies_commit(); }
    while (count > 0) {
        const int run = min(count, kMerge);
        copies_wait<kDepth - 1>();
        m.begin(x.peek());
        for (int left = run; left > 0; left -= kBatch) {
            if (left < run) copies_wait<kDepth - 1>();
            if (left >= kBatch) {
#pragma unroll
                for (int u = 0; u < kBatch; ++u) m.take(x.get());
                x.wrap();
            } else {
                for (int u = 0; u < left; ++u) m.take(x.get());
            }
            x.copy();
            copies_commit();
        }
        m.end(run);
        count -= run;
    }
}

// How many of a thread's V channels are joined in its registers: all of them or whole groups where sizes allow, else one.
template <int V> __device__ __forceinline__ int joined_channels(int per) { return per % V == 0 ? V : V % per == 0 ? per : 1; }

// Puts a thread's moments into red [rows][channels / joined], joined_channels at a time: the mean of their means, and the squared
// deviations around it.
template <int V>
__device__ __forceinline__ void put_moments(const Moments<V> &m, const Place &q, int channels, int per, float2 *red) {
    const int joined = joined_channels<V>(per);
    float2 *to = red + q.row * (channels / joined) + q.col * V / joined;
    if (joined == 1) {
#pragma unroll
        for (int j = 0; j < V; ++j) to[j] = make_float2(m.mean.get(j), m.m2.get(j));
        return;
    }
    const float n = static_cast<float>(m.n);
    auto put = [&](int first, int count) {             // (unrolled: registers stay registers)
        float s = 0.f, sq = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j >= first && j < first + count) s += m.mean.get(j);
        const float mean = s / static_cast<float>(count);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j >= first && j < first + count) {
                const float d = m.mean.get(j) - mean;
                sq += fmaf(n * d, d, m.m2.get(j));
            }
        to[first / count] = make_float2(mean, sq);
    };
    if (joined == V) put(0, V);
    if constexpr (V >= 4)
        if (joined == 2) {
#pragma unroll
            for (int f = 0; f < V; f += 2) put(f, 2);
        }
    if constexpr (V >= 8)
        if (joined == 4) {
#pragma unroll
            for (int f = 0; f < V; f += 4) put(f, 4);
        }
}

// Joins the entries of red, `width` per group and row, per group: n, mean and squared deviations of each around the first one's mean, in one
// pass; what the entries bring of their own is summed in fp64, and so is the correction to the joint mean, which cancels.  Teams of 1 to 32
// neighbouring lanes share a group, as many as there are threads for.  out(group, mean, m2).
template <int V, typename F>
__device__ __forceinline__ void join_groups(const float2 *red, int rows, int channels, int per, int pixels, F out) {
    const int joined = joined_channels<V>(per), width = per / joined, pitch = channels / joined;
    const int groups = channels / per;
    int team = 32;
    while (team > 1 && groups * team > kThreads) team >>= 1;
    const int member = threadIdx.x & (team - 1);
    const int base = pixels / rows, extra = pixels - base * rows;      // row r visited base pixels, or one more
    const int used = min(rows, pixels);
    const float many = static_cast<float>(joined), total = static_cast<float>(pixels) * static_cast<float>(per);
    for (int g0 = 0; g0 < groups; g0 += kThreads / team) {             // (the same for all threads)
        const int g = g0 + threadIdx.x / team;
        const float2 *from = red + g * width;
        float s = 0.f, around = 0.f;
        double q = 0.;
        if (g < groups) {
            around = from[0].x;
            for (int r = member; r < used; r += team) {
                const float n = static_cast<float>(base + (r < extra)) * many;
                for (int c = 0; c < width; ++c) {
                    const float2 e = from[r * pitch + c];
                    const float d = e.x - around;
                    s = fmaf(n, d, s);
                    q += fmaf(n * d, d, e.y);
                }
            }
        }
        for (int o = team >> 1; o > 0; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            q += __shfl_xor_sync(0xffffffffu, q, o);
        }
        const float shift = s / total;
        if (member == 0 && g < groups) out(g, static_cast<double>(around) + shift, ::fma(-static_cast<double>(s), static_cast<double>(shift), q));
    }
}

// act(norm) of a CTA's pixels from shared memory, as rows of a 4-bit matrix.  A thread keeps eight columns and walks over the
// pixels; four neighbouring lanes share a block of 32.  The product's steps cover 64 columns: where the last one holds a single block,
// the other is written as zeros.
template <typename T, int ACT>
__device__ __forceinline__ void write_mx4(const NormArgs &a, const T *tile, const float2 *fin, const float *gamma, const float *beta_of, int n, int64_t p0, int pixels, int c0, int channels) {
    const int row0 = static_cast<int>(n * a.P + p0);   // (a 4-bit matrix has fewer than 2^31 rows)
    const int row_bytes = a.mx_width / 2, code_bytes = 128 * row_bytes, scale_bytes = a.mx_width > 128 ? 1024 : 512;
    const int units = (channels + 31) / 32 * 4, rows = kThreads / units;
    if (c0 + channels == a.C && (a.C - 1) / 32 % 2 == 0) {             // an odd number of blocks: the one beside the last is zero
        const int c = (a.C + 31) / 32 * 32, ct = c / a.mx_width, in_tile = c - ct * a.mx_width;
        for (int p = threadIdx.x; p < pixels; p += kThreads) {
            const int row = row0 + p, r = row & 127;
            const int64_t t = static_cast<int64_t>(row >> 7) * a.mx_col_tiles + ct;
            int at = r * row_bytes + in_tile / 2;
            at ^= ((at >> 7) & (a.mx_width / 32 - 1)) << 4;
            *reinterpret_cast<uint4 *>(a.mx + t * code_bytes + at) = make_uint4(0, 0, 0, 0);
            a.mx[a.mx_scales + t * scale_bytes + (in_tile >> 7) * 512 + ((in_tile >> 5) & 3) + (r & 31) * 16 + (r >> 5) * 4] = 0;
        }
    }
    const int unit = threadIdx.x % units, first = threadIdx.x / units;
    const int c = unit * 8;
    const Groups<8> at(c, a.per);
    const Fv<8> shift = Fv<8>::make([&](int j) { return c + j < channels ? -fin[at.g[j]].x : 0.f; });
    const Fv<8> rstd = Fv<8>::make([&](int j) { return c + j < channels ? fin[at.g[j]].y : 0.f; });
    const Fv<8> scale = Fv<8>::make([&](int j) { return c + j < channels ? gamma[c + j] : 0.f; });
    const Fv<8> beta = Fv<8>::make([&](int j) { return c + j < channels ? beta_of[c + j] : 0.f; });
    const bool whole = c + 8 <= channels && channels % (16 / sizeof(T)) == 0;
    const int ct = (c0 + c) / a.mx_width, in_tile = (c0 + c) - ct * a.mx_width;
    const int scale_col = (in_tile >> 7) * 512 + ((in_tile >> 5) & 3);
    for (int base = 0; base < pixels; base += rows) {
        const int p = base + first;
        const bool on = first < rows && p < pixels;
        Fv<8> z = Fv<8>::all(0.f);
        if (on) {
            const T *src = tile + p * channels + c;
            if (whole) {
                constexpr int A = 16 / sizeof(T);
                Pack<T, 8> t;
#pragma unroll
                for (int i = 0; i < 8 / A; ++i) {
                    Pack<T, A> part;
                    part.load_shared(shared_address(src + i * A));
#pragma unroll
                    for (int k = 0; k < 4; ++k) t.w[4 * i + k] = part.w[k];
                }
                z = widen<T, 8>(t);
            } else {
                z = Fv<8>::make([&](int j) { return c + j < channels ? to_float(src[j]) : 0.f; });
            }
            // as written: see activate_plain.  The last product and sum are scalar: a packed product and the packed sum behind it
            // become one fused operation with one rounding, whatever roundings they state.
            const Fv<8> xh = (z + shift) * rstd;
            z = Fv<8>::make([&](int j) { return activate_plain<ACT>(__fadd_rn(__fmul_rn(xh.get(j), scale.get(j)), beta.get(j))); });
        }
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = whole || c + j < channels ? z.get(j) : 0.f;
        uint32_t codes;
        const uint32_t byte = quantise8(v, codes);
        if (on) {
            const int row = row0 + p, r = row & 127;
            const int64_t t = static_cast<int64_t>(row >> 7) * a.mx_col_tiles + ct;
            int at = r * row_bytes + in_tile / 2;
            at ^= ((at >> 7) & (a.mx_width / 32 - 1)) << 4;
            *reinterpret_cast<uint32_t *>(a.mx + t * code_bytes + at) = codes;
            if ((unit & 3) == 0) a.mx[a.mx_scales + t * scale_bytes + scale_col + (r & 31) * 16 + (r >> 5) * 4] = static_cast<uint8_t>(byte);
        }
    }
}

// act(norm) of a thread's pixels from shared memory.
template <typename T, int V, int ACT>
__device__ __forceinline__ void write_norm(const NormArgs &a, const T *tile, const float2 *fin, const float *gamma, const float *beta_of, int n, int64_t p0, int pixels,
                                           int c0, int channels, const Place &q) {
    const int col = q.col * V;
    const Groups<V> at(col, a.per);
    const Fv<V> shift = Fv<V>::make([&](int j) { return -fin[at.g[j]].x; });
    const Fv<V> scale = Fv<V>::make([&](int j) { return fin[at.g[j]].y * gamma[col + j]; });
    const Fv<V> beta = Fv<V>::make([&](int j) { return beta_of[col + j]; });
    T *dst = static_cast<T *>(a.y) + n * a.y_image + (p0 + q.row) * a.y_pixel + c0 + q.col * V;
    uint32_t src = shared_address(tile + q.row * channels + col);
    const int64_t dst_step = q.rows * a.y_pixel;
    const uint32_t src_step = q.rows * channels * sizeof(T);
#pragma unroll 4
    for (int p = q.row; p < pixels; p += q.rows, dst += dst_step, src += src_step) {
        Pack<T, V> v;
        v.load_shared(src);
        narrow<T, V>(activate<ACT, V>(fma(widen<T, V>(v) + shift, scale, beta))).store(dst);
    }
}

// A cluster's barrier in halves: nobody leaves before every CTA has read what it wants of the others' shared memory.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// (mean, rstd) from the mean and the sum of squared deviations
__device__ __forceinline__ float2 statistics(const NormArgs &a, double mean, double m2) {
    return make_float2(static_cast<float>(mean), rsqrtf(static_cast<float>(m2 * a.inv_values) + a.eps));
}

// ---- resident form ----------------------------------------------------------------------------------------------------
// Shared memory: [chunk][slab] elements of x, then [rows][slab] float2, then [groups of the slab] double2 and float2, then gamma and beta.
template <typename T, int V, int ACT, bool MX>
__global__ void __launch_bounds__(kThreads, 3) norm_resident_kernel(NormArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    pdl_trigger();
    const int rank = blockIdx.x % a.cluster;
    const int slab = (blockIdx.x / a.cluster) % a.slabs;
    const int n = blockIdx.x / (a.cluster * a.slabs);
    const int c0 = slab * a.slab, channels = min(a.slab, a.C - c0);
    const int64_t p0 = min(a.P, rank * a.chunk), p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(channels);
    T *tile = reinterpret_cast<T *>(smem);
    float2 *red = reinterpret_cast<float2 *>(smem + (a.chunk * a.slab * sizeof(T) + 15) / 16 * 16);
    double2 *grp = reinterpret_cast<double2 *>(red + kThreads * V);    // this CTA's (mean, squared deviations) per group
    float2 *fin = reinterpret_cast<float2 *>(grp + a.slab / a.per);    // the image's (mean, rstd)
    float *gamma = reinterpret_cast<float *>(fin + a.slab / a.per), *beta_of = gamma + a.slab;
    const int groups = channels / a.per;
    pdl_wait();
    for (int c = threadIdx.x; c < channels; c += kThreads) {           // in flight together with x
        copy_async<4>(shared_address(gamma + c), a.gamma + c0 + c);
        copy_async<4>(shared_address(beta_of + c), a.beta + c0 + c);
    }
    if (q.on) {
        Moments<V> m;
        Stream<T, V, true, 1> x;
        x.begin(static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V, a.x_pixel, pixels, q, tile, channels, q.col * V);
        moments_of<T, V, true>(x, m);
        put_moments<V>(m, q, channels, a.per, red);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    if (pixels > 0) join_groups<V>(red, q.rows, channels, a.per, pixels, [&](int g, double mean, double m2) { grp[g] = make_double2(mean, m2); });
    cg::cluster_group cluster = cg::this_cluster();
    if (a.cluster > 1) cluster.sync(); else __syncthreads();
    for (int g = threadIdx.x; g < groups; g += kThreads) {
        double2 e = grp[g];
        if (a.cluster > 1) {
            // around the first CTA's mean; in fp64 the square of the sum takes nothing from the sum of squares that matters
            double around = 0., s = 0., sq = 0., m2 = 0.;
            for (int first = 0; first < a.cluster; first += 4) {
                double2 o[4];                          // in flight together
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (first + k < a.cluster) o[k] = cluster.map_shared_rank(grp, first + k)[g];
                if (first == 0) around = o[0].x;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int64_t count = min(a.P - (first + k) * a.chunk, a.chunk);
                    if (first + k >= a.cluster || count <= 0) continue;                    // (a CTA without pixels has written none)
                    const double n = static_cast<double>(a.per) * static_cast<int>(count), d = o[k].x - around;
                    s = ::fma(n, d, s);
                    sq = ::fma(n * d, d, sq);
                    m2 += o[k].y;
                }
            }
            const double shift = s * a.inv_values;
            e = make_double2(around + shift, m2 + ::fma(-s, shift, sq));
        }
        fin[g] = statistics(a, e.x, e.y);
        if (a.stats_out && rank == 0) reinterpret_cast<float2 *>(a.stats_out)[static_cast<int64_t>(n) * a.G + c0 / a.per + g] = fin[g];
    }
    if (a.cluster > 1) cluster_arrive();               // the other CTAs' grp have been read
    __syncthreads();
    if constexpr (MX) write_mx4<T, ACT>(a, tile, fin, gamma, beta_of, n, p0, pixels, c0, channels);
    else if (q.on) write_norm<T, V, ACT>(a, tile, fin, gamma, beta_of, n, p0, pixels, c0, channels, q);
    if (a.cluster > 1) cluster_wait();
}

// Sums of red [rows][channels] over the rows, with all threads: part [kThreads]; out(channel, sum).
template <typename F>
__device__ __forceinline__ void sum_rows(const float2 *red, int rows, int channels, float2 *part, F out) {
    const int parts = kThreads / channels;             // threads per channel
    if (parts < 2) {
        for (int c = threadIdx.x; c < channels; c += kThreads) {
            float2 s = make_float2(0.f, 0.f);
            for (int r = 0; r < rows; ++r) { s.x += red[r * channels + c].x; s.y += red[r * channels + c].y; }
            out(c, s);
        }
        return;
    }
    const int c = threadIdx.x % channels, p = threadIdx.x / channels;
    float2 s = make_float2(0.f, 0.f);
    if (p < parts) {
#pragma unroll 4
        for (int r = p; r < rows; r += parts) { s.x += red[r * channels + c].x; s.y += red[r * channels + c].y; }
        part[threadIdx.x] = s;
    }
    __syncthreads();
    if (p == 0) {
        for (int k = 1; k < parts; ++k) { s.x += part[k * channels + c].x; s.y += part[k * channels + c].y; }
        out(c, s);
    }
}

// What a thread keeps of its V channels: d = x - mean, z = d * scale + beta with scale = rstd * gamma.
template <int V>
struct Channels {
    Fv<V> shift, scale, beta;                          // shift = -mean
    __device__ __forceinline__ void load(const NormArgs &a, int n, int c) {
        const float2 *st = reinterpret_cast<const float2 *>(a.stats_in) + static_cast<int64_t>(n) * a.G;
        const Groups<V> at(c, a.per);
        shift = Fv<V>::make([&](int j) { return -st[at.g[j]].x; });
        scale = Fv<V>::make([&](int j) { return st[at.g[j]].y * a.gamma[c + j]; });
        beta = Fv<V>::make([&](int j) { return a.beta[c + j]; });
    }
    __device__ __forceinline__ void from_shared(const float2 *stats, const float *gamma, const float *beta_of, int c, int per) {
        const Groups<V> at(c, per);
        shift = Fv<V>::make([&](int j) { return -stats[at.g[j]].x; });
        scale = Fv<V>::make([&](int j) { return stats[at.g[j]].y * gamma[c + j]; });
        beta = Fv<V>::make([&](int j) { return beta_of[c + j]; });
    }
    template <int ACT, typename T>
    __device__ __forceinline__ void slope(const Pack<T, V> &x, const Pack<T, V> &dy, Fv<V> &d, Fv<V> &dz) const {
        d = widen<T, V>(x) + shift;
        dz = through<ACT, V>(widen<T, V>(dy), fma(d, scale, beta));
    }
    // dx = scale * dz - k1 - d * k2; nk = -k
    template <int ACT, typename T>
    __device__ __forceinline__ Pack<T, V> dx(const Pack<T, V> &x, const Pack<T, V> &dy, const Fv<V> &nk1, const Fv<V> &nk2) const {
        Fv<V> d, dz;
        slope<ACT, T>(x, dy, d, dz);
        return narrow<T, V>(fma(d, nk2, fma(scale, dz, nk1)));
    }
};

// Begins the copies of two tensors; returns the number of a thread's pixels.
template <typename S> __device__ __forceinline__ int start_copies(S &x, S &dy) {
    const int count = x.left;
#pragma unroll
    for (int b = 0; b < S::kDepth; ++b) { x.copy(); dy.copy(); copies_commit(); }
    return count;
}

// Sums of dz and dz * d over a thread's pixels, whose copies have begun.
template <typename T, int V, int ACT, bool KEEP>
__device__ __forceinline__ void sums_of(Stream<T, V, KEEP, 2> &x, Stream<T, V, KEEP, 2> &dy, int count, const Channels<V> &f, Fv<V> &sa, Fv<V> &sb) {
    constexpr int kBatch = Stream<T, V, KEEP, 2>::kBatch, kDepth = Stream<T, V, KEEP, 2>::kDepth;
    sa = sb = Fv<V>::all(0.f);
    auto take = [&]() {
        Fv<V> d, dz;
        f.template slope<ACT, T>(x.get(), dy.get(), d, dz);
        sa = sa + dz;
        sb = fma(dz, d, sb);
    };
    for (; count > 0; count -= kBatch) {
        copies_wait<kDepth - 1>();
        if (count >= kBatch) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u) take();
            x.wrap();
            dy.wrap();
        } else {
            for (int u = 0; u < count; ++u) take();
        }
        x.copy();
        dy.copy();
        copies_commit();
    }
}

// Shared memory: [chunk][slab] elements of x, the same of dy, [rows][slab] float2, [slab] float2, [max(slab, kThreads)] float2,
// [groups] float2 twice, gamma and beta.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kThreads, 3) norm_grad_resident_kernel(NormArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ bool last;
    pdl_trigger();
    const int rank = blockIdx.x % a.cluster;
    const int slab = (blockIdx.x / a.cluster) % a.slabs;
    const int n = blockIdx.x / (a.cluster * a.slabs);
    const int c0 = slab * a.slab, channels = min(a.slab, a.C - c0);
    const int64_t p0 = min(a.P, rank * a.chunk), p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(channels);
    const int64_t tile_bytes = (a.chunk * a.slab * sizeof(T) + 15) / 16 * 16;
    T *xt = reinterpret_cast<T *>(smem);
    T *dt = reinterpret_cast<T *>(smem + tile_bytes);
    float2 *red = reinterpret_cast<float2 *>(smem + 2 * tile_bytes);
    float2 *sums = red + kThreads * V;                 // this CTA's (A, B) per channel
    float2 *whole = sums + a.slab;                     // the image's (A, B) per channel; before that, parts of this CTA's
    float2 *fin = whole + max(a.slab, kThreads);       // (rstd * s1, rstd^2 * s2) per group
    float2 *stats = fin + a.slab / a.per;              // (mean, rstd) per group
    float *gamma = reinterpret_cast<float *>(stats + a.slab / a.per), *beta = gamma + a.slab;
    const int groups = channels / a.per;
    pdl_wait();

    for (int g = threadIdx.x; g < groups; g += kThreads)               // in flight together with x and dy
        copy_async<8>(shared_address(stats + g), reinterpret_cast<const float2 *>(a.stats_in) + static_cast<int64_t>(n) * a.G + c0 / a.per + g);
    for (int c = threadIdx.x; c < channels; c += kThreads) {
        copy_async<4>(shared_address(gamma + c), a.gamma + c0 + c);
        copy_async<4>(shared_address(beta + c), a.beta + c0 + c);
    }
    copies_commit();
    using S = Stream<T, V, true, 2>;
    S x, dy;
    int count = 0;
    if (q.on) {
        x.begin(static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V, a.x_pixel, pixels, q, xt, channels, q.col * V);
        dy.begin(static_cast<const T *>(a.dy) + n * a.y_image + p0 * a.y_pixel + c0 + q.col * V, a.y_pixel, pixels, q, dt, channels, q.col * V);
        count = start_copies(x, dy);
        copies_wait<S::kDepth>();                      // the constants: committed before kDepth batches
    } else {
        copies_wait<0>();
    }
    __syncthreads();
    Channels<V> f;
    if (q.on) {
        Fv<V> sa, sb;
        f.from_shared(stats, gamma, beta, q.col * V, a.per);
        sums_of<T, V, ACT, true>(x, dy, count, f, sa, sb);
#pragma unroll
        for (int j = 0; j < V; ++j) red[q.row * channels + q.col * V + j] = make_float2(sa.get(j), sb.get(j));
    }
    __syncthreads();
    sum_rows(red, q.rows, channels, whole, [&](int c, float2 s) { sums[c] = make_float2(s.x, s.y * stats[c / a.per].y); });
    cg::cluster_group cluster = cg::this_cluster();
    if (a.cluster > 1) cluster.sync(); else __syncthreads();
    for (int c = threadIdx.x; c < channels; c += kThreads) {
        float2 s = sums[c];
        if (a.cluster > 1) {
            float2 all[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) all[r] = r < a.cluster ? cluster.map_shared_rank(sums, r)[c] : make_float2(0.f, 0.f);
            s = all[0];
#pragma unroll
            for (int r = 1; r < 8; ++r) { s.x += all[r].x; s.y += all[r].y; }
        }
        whole[c] = s;
        if (rank == 0) reinterpret_cast<float2 *>(a.ws)[static_cast<int64_t>(n) * a.C + c0 + c] = s;
    }
    if (a.cluster > 1) cluster_arrive();               // the other CTAs' sums have been read
    __syncthreads();
    if (rank == 0 && threadIdx.x == kThreads - 1) {    // (its latency lies beside the rest of the work)
        __threadfence();
        last = atomicAdd(a.counters + slab, 1u) == static_cast<unsigned>(a.N) - 1;
        if (last) a.counters[slab] = 0;
        __threadfence();
    }
    for (int g = threadIdx.x; g < groups; g += kThreads) {
        float s1 = 0.f, s2 = 0.f;
        for (int c = 0; c < a.per; ++c) {
            const float gm = gamma[g * a.per + c];
            const float2 e = whole[g * a.per + c];
            s1 = fmaf(gm, e.x, s1);
            s2 = fmaf(gm, e.y, s2);
        }
        const float rstd = stats[g].y;
        fin[g] = make_float2(rstd * (s1 * a.inv_count), rstd * rstd * (s2 * a.inv_count));
    }
    __syncthreads();
    if (q.on) {
        const Groups<V> at(q.col * V, a.per);
        const Fv<V> nk1 = Fv<V>::make([&](int j) { return -fin[at.g[j]].x; });
        const Fv<V> nk2 = Fv<V>::make([&](int j) { return -fin[at.g[j]].y; });
        T *dst = static_cast<T *>(a.y) + n * a.x_image + (p0 + q.row) * a.x_pixel + c0 + q.col * V;
        uint32_t xs = shared_address(xt + q.row * channels + q.col * V), ds = shared_address(dt + q.row * channels + q.col * V);
        const int64_t dst_step = q.rows * a.x_pixel;
        const uint32_t step = q.rows * channels * sizeof(T);
#pragma unroll 2
        for (int p = q.row; p < pixels; p += q.rows, dst += dst_step, xs += step, ds += step) {
            Pack<T, V> xv, dv;
            xv.load_shared(xs);
            dv.load_shared(ds);
            f.template dx<ACT, T>(xv, dv, nk1, nk2).store(dst);
        }
    }
    // The last cluster of this slab to get here adds the images up, in ascending order: the result does not depend on which is last.
    if (rank == 0 && last)                             // (`last` was written before the barrier above)
        for (int c = c0 + threadIdx.x; c < c0 + channels; c += kThreads) {
            float sa = 0.f, sb = 0.f;
#pragma unroll 8
            for (int i = 0; i < a.N; ++i) {
                const float2 e = __ldcg(reinterpret_cast<const float2 *>(a.ws) + static_cast<int64_t>(i) * a.C + c);
                sa += e.x; sb += e.y;
            }
            a.dbeta[c] = sa;
            a.dgamma[c] = sb;
        }
    if (a.cluster > 1) cluster_wait();
}

// ---- two-pass form ----------------------------------------------------------------------------------------------------
// Channels of a slab: whole groups, or (parts > 1) one of the `parts` slabs of a group wider than a CTA.
struct Span {
    int c0, channels;
};
__device__ __forceinline__ Span span_of(const NormArgs &a, int slab) {
    Span s;
    if (a.parts > 1) {
        const int part = slab % a.parts;
        s.c0 = slab / a.parts * a.per + part * a.slab;
        s.channels = min(a.slab, a.per - part * a.slab);
    } else {
        s.c0 = slab * a.slab;
        s.channels = min(a.slab, a.C - s.c0);
    }
    return s;
}

// Sums of two values over the CTA.
template <typename F> __device__ __forceinline__ void block_sums(F &a, F &b, F (*scratch)[2]) {
    a = warp_sum(a);
    b = warp_sum(b);
    if ((threadIdx.x & 31) == 0) {
        scratch[threadIdx.x >> 5][0] = a;
        scratch[threadIdx.x >> 5][1] = b;
    }
    __syncthreads();
    a = b = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        a += scratch[w][0];
        b += scratch[w][1];
    }
}

// blockIdx = (chunk, slab, image of the run); ws [image of the run][cell][chunk] (mean, m2), a cell being a group or a part of one.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 3) norm_moments_kernel(NormArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    float2 *red = reinterpret_cast<float2 *>(smem);
    pdl_trigger();
    const int n = blockIdx.z;
    const Span s = span_of(a, blockIdx.y);
    const int64_t p0 = blockIdx.x * a.chunk, p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(s.channels);
    const int cells = a.parts > 1 ? a.slabs : a.G;
    pdl_wait();
    Moments<V> m;
    if (q.on) {
        Stream<T, V, false, 1> x;
        x.begin(static_cast<const T *>(a.x) + (a.n0 + n) * a.x_image + p0 * a.x_pixel + s.c0 + q.col * V, a.x_pixel, pixels, q,
                reinterpret_cast<T *>(smem), s.channels, 0);
        moments_of<T, V, false>(x, m);
    }
    __syncthreads();                                   // red lies over the rings
    if (q.on) put_moments<V>(m, q, s.channels, a.parts > 1 ? s.channels : a.per, red);
    __syncthreads();
    const int cell = a.parts > 1 ? blockIdx.y : s.c0 / a.per;
    float2 *to = reinterpret_cast<float2 *>(a.ws) + (static_cast<int64_t>(n) * cells + cell) * a.chunks + blockIdx.x;
    join_groups<V>(red, q.rows, s.channels, a.parts > 1 ? s.channels : a.per, pixels, [&](int g, double mean, double m2) {
        to[static_cast<int64_t>(g) * a.chunks] = make_float2(static_cast<float>(mean), static_cast<float>(m2));
    });
}

// One CTA per (group, image of the run): joins the chunks' moments around the first one's mean, in fp64.
__global__ void __launch_bounds__(kThreads) norm_join_kernel(NormArgs a) {
    __shared__ double scratch[kThreads / 32][2];
    pdl_trigger();
    pdl_wait();
    const int g = blockIdx.x, n = blockIdx.y, items = a.chunks * a.parts;
    const float2 *w = reinterpret_cast<const float2 *>(a.ws) + (static_cast<int64_t>(n) * a.G + g) * items;
    const float around = w[0].x;
    double s = 0., q = 0.;
    for (int i = threadIdx.x; i < items; i += kThreads) {
        const int part = i / a.chunks, k = i - part * a.chunks;
        const double values = static_cast<double>(min(a.chunk, a.P - k * a.chunk)) * (a.parts > 1 ? min(a.slab, a.per - part * a.slab) : a.per);
        const float2 e = w[i];
        const double d = e.x - around;
        s = ::fma(values, d, s);
        q += ::fma(values * d, d, static_cast<double>(e.y));
    }
    block_sums(s, q, scratch);
    const double shift = s * a.inv_values;
    if (threadIdx.x == 0) reinterpret_cast<float2 *>(a.stats_out)[static_cast<int64_t>(a.n0 + n) * a.G + g] = statistics(a, around + shift, ::fma(-s, shift, q));
}

// Each CTA takes its pixels in the opposite order of the pass before: what that one read last is still in L2.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kThreads, 3) norm_apply_kernel(NormArgs a) {
    pdl_trigger();
    const int n = a.n0 + blockIdx.z;
    const Span s = span_of(a, blockIdx.y);
    const int64_t p0 = blockIdx.x * a.chunk, p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(s.channels);
    pdl_wait();
    if (!q.on) return;
    extern __shared__ __align__(16) unsigned char smem[];
    using S = Stream<T, V, false, 1>;
    S x;
    x.template begin<true>(static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + s.c0 + q.col * V, a.x_pixel, pixels, q, reinterpret_cast<T *>(smem), s.channels, 0);
    int count = x.left;
#pragma unroll
    for (int b = 0; b < S::kDepth; ++b) { x.copy(); copies_commit(); }
    Channels<V> f;
    f.load(a, n, s.c0 + q.col * V);
    const int64_t dst_step = -q.rows * a.y_pixel;
    T *dst = static_cast<T *>(a.y) + n * a.y_image + (p0 + q.row) * a.y_pixel - (count - 1) * dst_step + s.c0 + q.col * V;
    auto put = [&]() {
        narrow<T, V>(activate<ACT, V>(fma(widen<T, V>(x.get()) + f.shift, f.scale, f.beta))).store(dst);
        dst += dst_step;
    };
    for (; count > 0; count -= S::kBatch) {
        copies_wait<S::kDepth - 1>();
        if (count >= S::kBatch) {
#pragma unroll
            for (int u = 0; u < S::kBatch; ++u) put();
            x.wrap();
        } else {
            for (int u = 0; u < count; ++u) put();
        }
        x.copy();
        copies_commit();
    }
}

// ws [N][chunks][C] (A, B) of the chunk's pixels.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kThreads, 3) norm_grad_sums_kernel(NormArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    float2 *red = reinterpret_cast<float2 *>(smem);
    pdl_trigger();
    const int n = a.n0 + blockIdx.z;
    const Span s = span_of(a, blockIdx.y);
    const int64_t p0 = blockIdx.x * a.chunk, p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(s.channels);
    pdl_wait();
    Fv<V> sa, sb;
    if (q.on) {
        T *ring = reinterpret_cast<T *>(smem);
        Stream<T, V, false, 2> x, dy;
        x.begin(static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + s.c0 + q.col * V, a.x_pixel, pixels, q, ring, s.channels, 0);
        dy.begin(static_cast<const T *>(a.dy) + n * a.y_image + p0 * a.y_pixel + s.c0 + q.col * V, a.y_pixel, pixels, q,
                 ring + Stream<T, V, false, 2>::kDepth * Stream<T, V, false, 2>::kBatch * kThreads * V, s.channels, 0);
        const int count = start_copies(x, dy);
        Channels<V> f;
        f.load(a, n, s.c0 + q.col * V);                // (arrives with the first copies)
        sums_of<T, V, ACT, false>(x, dy, count, f, sa, sb);
    }
    __syncthreads();                                   // red lies over the rings
    if (q.on) {
#pragma unroll
        for (int j = 0; j < V; ++j) red[q.row * s.channels + q.col * V + j] = make_float2(sa.get(j), sb.get(j));
    }
    __syncthreads();
    float2 *out = reinterpret_cast<float2 *>(a.ws) + (static_cast<int64_t>(n) * a.chunks + blockIdx.x) * a.C + s.c0;
    const float2 *st = reinterpret_cast<const float2 *>(a.stats_in) + static_cast<int64_t>(n) * a.G;
    sum_rows(red, q.rows, s.channels, red + kThreads * V, [&](int c, float2 t) { out[c] = make_float2(t.x, t.y * st[(s.c0 + c) / a.per].y); });
}

// One CTA per (group, image of the run): sums the chunks, writes (rstd s1, rstd^2 s2) of the group behind the partial sums and the
// image's (A, B) per channel into chunk 0's place.
__global__ void __launch_bounds__(kThreads) norm_grad_join_kernel(NormArgs a) {
    __shared__ float scratch[kThreads / 32][2];
    pdl_trigger();
    pdl_wait();
    const int g = blockIdx.x, n = a.n0 + blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float2 *part = reinterpret_cast<float2 *>(a.ws) + static_cast<int64_t>(n) * a.chunks * a.C + g * a.per;
    float s1 = 0.f, s2 = 0.f;
    for (int c = warp; c < a.per; c += kThreads / 32) {                // a warp takes a channel at a time
        float sa = 0.f, sb = 0.f;
#pragma unroll 4
        for (int k = lane; k < a.chunks; k += 32) {
            const float2 e = part[static_cast<int64_t>(k) * a.C + c];
            sa += e.x; sb += e.y;
        }
        sa = warp_sum(sa);
        sb = warp_sum(sb);
        if (lane == 0) part[c] = make_float2(sa, sb);                  // (this lane alone has read chunk 0's entry)
        const float gm = a.gamma[g * a.per + c];
        s1 = fmaf(gm, sa, s1);
        s2 = fmaf(gm, sb, s2);
    }
    if (lane) s1 = s2 = 0.f;
    block_sums(s1, s2, scratch);
    if (threadIdx.x == 0) {
        const int64_t at = static_cast<int64_t>(n) * a.G + g;
        const float rstd = reinterpret_cast<const float2 *>(a.stats_in)[at].y;
        reinterpret_cast<float2 *>(a.ws)[static_cast<int64_t>(a.N) * a.chunks * a.C + at] = make_float2(rstd * (s1 * a.inv_count), rstd * rstd * (s2 * a.inv_count));
    }
}

template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kThreads, 3) norm_grad_apply_kernel(NormArgs a) {
    pdl_trigger();
    const int n = a.n0 + blockIdx.z;
    const Span s = span_of(a, blockIdx.y);
    const int64_t p0 = blockIdx.x * a.chunk, p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(s.channels);
    pdl_wait();
    const float2 *ws = reinterpret_cast<const float2 *>(a.ws);
    if (a.n0 + static_cast<int>(gridDim.z) == a.N && threadIdx.x < 32) {
        // in the last run, the first warps of a slab's CTAs add the images up, a channel at a time: a lane takes every 32nd image
        for (int c = blockIdx.z * gridDim.x + blockIdx.x; c < s.channels; c += gridDim.x * gridDim.z) {
            float sa = 0.f, sb = 0.f;
            for (int i = threadIdx.x; i < a.N; i += 32) {
                const float2 e = ws[static_cast<int64_t>(i) * a.chunks * a.C + s.c0 + c];
                sa += e.x; sb += e.y;
            }
            sa = warp_sum(sa);
            sb = warp_sum(sb);
            if (threadIdx.x == 0) {
                a.dbeta[s.c0 + c] = sa;
                a.dgamma[s.c0 + c] = sb;
            }
        }
        __syncwarp();
    }
    if (!q.on) return;
    Channels<V> f;
    f.load(a, n, s.c0 + q.col * V);
    const float2 *k = ws + static_cast<int64_t>(a.N) * a.chunks * a.C + static_cast<int64_t>(n) * a.G;
    const Groups<V> at(s.c0 + q.col * V, a.per);
    const Fv<V> nk1 = Fv<V>::make([&](int j) { return -k[at.g[j]].x; });
    const Fv<V> nk2 = Fv<V>::make([&](int j) { return -k[at.g[j]].y; });
    extern __shared__ __align__(16) unsigned char smem[];
    using S = Stream<T, V, false, 2>;
    S x, dy;
    T *ring = reinterpret_cast<T *>(smem);
    x.template begin<true>(static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + s.c0 + q.col * V, a.x_pixel, pixels, q, ring, s.channels, 0);
    dy.template begin<true>(static_cast<const T *>(a.dy) + n * a.y_image + p0 * a.y_pixel + s.c0 + q.col * V, a.y_pixel, pixels, q,
             ring + S::kDepth * S::kBatch * kThreads * V, s.channels, 0);
    int count = x.left;
#pragma unroll
    for (int b = 0; b < S::kDepth; ++b) { x.copy(); dy.copy(); copies_commit(); }
    const int64_t dst_step = -q.rows * a.x_pixel;
    T *dst = static_cast<T *>(a.y) + n * a.x_image + (p0 + q.row) * a.x_pixel - (count - 1) * dst_step + s.c0 + q.col * V;
    auto put = [&]() {
        f.template dx<ACT, T>(x.get(), dy.get(), nk1, nk2).store(dst);
        dst += dst_step;
    };
    for (; count > 0; count -= S::kBatch) {
        copies_wait<S::kDepth - 1>();
        if (count >= S::kBatch) {
#pragma unroll
            for (int u = 0; u < S::kBatch; ++u) put();
            x.wrap();
            dy.wrap();
        } else {
            for (int u = 0; u < count; ++u) put();
        }
        x.copy();
        dy.copy();
        copies_commit();
    }
}

// ---- planning -----------------------------------------------------------------------------------------------------------
int resident_smem(const NormShape &s, int width, int tensors, int slab, int64_t chunk) {
    const int64_t tile = (chunk * slab * elem_bytes(s.dtype) + 15) / 16 * 16;
    const int64_t groups = slab / (s.C / s.G);
    const int64_t small = (tensors == 1 ? 3 * groups : 2 * groups + slab + std::max(slab, kThreads)) + slab;   // float2 (gamma and beta: one per channel)
    const int64_t total = tensors * tile + (static_cast<int64_t>(kThreads) * width + small) * 8;
    return total > (int64_t(1) << 30) ? (1 << 30) : static_cast<int>(total);
}

constexpr int kSmemMost = 220 * 1024;       // dynamic shared memory of one CTA
constexpr int64_t kRunBytes = int64_t(160) << 20;   // two-pass: bytes of x (and dy) of the images that are taken together

// Picks the slab and the cluster of the resident form by a time estimate, fitted to measurements of ten shapes with every slab and
// cluster that fits (7x7 to 56x56 pixels, 64 to 512 channels, the three types, both directions): the CTAs of an SM share its HBM rate of
// 44 bytes per ns; a wave costs half a microsecond, a cluster one more and 0.3 per doubling; slabs narrower than 128 bytes cost 10 %; the
// gradient, bound by its arithmetic, wants three CTAs per SM.
// Besides, an SM takes at most kRate elements per us through its arithmetic, one half of that time for the statistics and the other for
// writing: few CTAs on a large image lose against the two passes.  The half of the statistics counts three times at single-element accesses
// (1.5 times at two elements), that of writing twice for 4-bit rows, padded to 32 columns, and six times where their SiLU is formed as
// written; in the gradient both count four times.
// In that sweep its choice of slab and cluster was the fastest or within 3 % of it, for 16- and 32-bit outputs.  As a time it is rough: it gives 10 us for
// 32 x 56 x 56 x 64 bf16 into 4-bit rows, which take 16, latency of eight warps per SM.
// `unit`: slabs are a multiple of so many channels (or all of them).
NormPlan plan_one(const NormShape &s, int width, int tensors, int unit) {
    NormPlan best;
    const int per = s.C / s.G, e = elem_bytes(s.dtype);
    const double slow = width == 1 ? 3 : width == 2 ? 1.5 : 1, kRate = 9000, sms = sm_count();
    // two passes: three launches per run and the bytes once more, or the arithmetic of both passes on all SMs
    const double elements = static_cast<double>(s.N) * s.P * s.C;
    double best_us = 8.0 * ceil_div(static_cast<int64_t>(elements) * e * tensors, kRunBytes) +
                     std::max(elements * e * (2 * tensors + 1) / 5.2e6, elements * slow * (tensors == 2 ? 2.8 : 1.2) / (sms * kRate));
    for (int k = 1; k <= s.G; ++k) {
        if (s.G % k) continue;
        const int64_t slab = static_cast<int64_t>(k) * per;
        if (slab % width || slab / width > kThreads) continue;
        if (k < s.G && (slab * e < 64 || slab % unit)) continue;
        for (int cl = 1; cl <= 8; cl *= 2) {
            if (cl > s.P) break;
            const int64_t chunk = ceil_div(s.P, cl);
            const int smem = resident_smem(s, width, tensors, static_cast<int>(slab), chunk);
            if (smem > kSmemMost || static_cast<int64_t>(s.N) * (s.G / k) * cl > INT32_MAX) continue;
            const int per_sm = std::min(3, (224 * 1024) / (smem + 1024));
            const double ctas = static_cast<double>(s.N) * (s.G / k) * cl;
            const double here = std::min<double>(per_sm, std::ceil(ctas / sms));           // CTAs of an SM at a time
            const double waves = std::ceil(ctas / (sms * here));
            const double bytes = static_cast<double>(chunk) * slab * e * (tensors + 1);
            const double wide = unit > 1 ? (slab + 31) / 32 * 32.0 * (s.act == PATDNN_ACT_SILU ? 6 : 2) : static_cast<double>(slab);
            const double work = chunk * (slab * slow + wide) * (tensors == 2 ? 2.0 : 0.5) / kRate;
            const double memory = here * bytes / 44e3 * (slab * e < 128 && k < s.G ? 1.1 : 1.0) * (tensors == 2 ? 1 + 0.4 * (3 - here) : 1.0);
            const double us = waves * (std::max(memory, here * work) +
                                       0.5 + (cl > 1 ? 1.0 + 0.3 * std::log2(cl) : 0.0));
            if (us < best_us) {
                best_us = us;
                best.resident = true; best.slab = static_cast<int>(slab); best.slabs = s.G / k; best.cluster = cl;
                best.chunk = chunk; best.smem = smem; best.chunks = 1;
            }
        }
    }
    if (best.resident) return best;
    const int most = kThreads * width;                 // channels a CTA covers
    if (per > most) {                                  // a group is cut into parts (width divides per: see plan_norm)
        best.parts = static_cast<int>(ceil_div(per, most));
        best.slab = static_cast<int>(ceil_div(ceil_div(per, best.parts), width) * width);
        best.parts = static_cast<int>(ceil_div(per, best.slab));
        best.slabs = s.G * best.parts;
    } else {
        int k = most / per;
        while (k > 1 && (k * per) % width) --k;
        k = std::min(k, s.G);
        best.slab = k * per;
        best.slabs = static_cast<int>(ceil_div(s.G, k));
    }
    const int64_t image = s.P * s.C * e * tensors;     // bytes
    const int64_t runs = ceil_div(s.N, std::max<int64_t>(1, std::min<int64_t>(s.N, kRunBytes / image)));
    best.run = static_cast<int>(ceil_div(s.N, runs));  // runs of about the same number of images
    // one wave of three CTAs per SM over a run: a last, partly filled wave would cost as much as a full one
    const int64_t share = static_cast<int64_t>(sm_count()) * 3 / (static_cast<int64_t>(best.run) * best.slabs);         // CTAs per (image, slab)
    const int64_t each = std::max<int64_t>(1, share);
    const int rows = kThreads / (best.slab / width);
    const int64_t chunk = std::max<int64_t>(ceil_div(s.P, each), rows);
    best.chunk = std::min(std::max<int64_t>(chunk, ceil_div(s.P, 2048)), s.P);
    best.chunks = static_cast<int>(ceil_div(s.P, best.chunk));
    return best;
}

// Dynamic shared memory of the two-pass kernels: the rings, and over them the per-thread results.
template <typename T, int V, int TENSORS> constexpr size_t ring_smem() {
    using S = Stream<T, V, false, TENSORS>;
    return static_cast<size_t>(kThreads) * std::max(8 * (V + 1), TENSORS * S::kDepth * S::kBatch * S::kBytes);   // (and a float2 each for sum_rows)
}

// A plan needs the vector width to divide the channels, and each group's where a group is wider than a CTA.
bool width_fits(const NormShape &s, int v) {
    const int per = s.C / s.G;
    if (s.C % v) return false;
    if (per % v == 0) return true;
    const int64_t together = static_cast<int64_t>(per) * v;    // v groups hold a multiple of v channels
    return together <= static_cast<int64_t>(kThreads) * v && s.G % v == 0;
}

// Widest access that the sizes, the strides and the addresses allow.
int width_index(const NormShape &s, std::initializer_list<const void *> pointers, bool y_too) {
    const int e = elem_bytes(s.dtype);
    for (int i = 0; i < kNormWidths; ++i) {
        const int v = norm_width(s.dtype, i);
        bool ok = width_fits(s, v) && s.x_pixel % v == 0 && s.x_image % v == 0;
        if (y_too) ok = ok && s.y_pixel % v == 0 && s.y_image % v == 0;
        for (const void *p : pointers) ok = ok && reinterpret_cast<uintptr_t>(p) % (static_cast<unsigned>(v) * e) == 0;
        if (ok) return i;
    }
    return kNormWidths - 1;
}

NormArgs args_of(const NormHandle &h, const NormPlan &p) {
    const NormShape &s = h.s;
    NormArgs a{};
    a.ws = h.ws; a.counters = h.counters;
    a.x_pixel = s.x_pixel; a.x_image = s.x_image; a.y_pixel = s.y_pixel; a.y_image = s.y_image;
    a.P = s.P; a.chunk = p.chunk; a.N = s.N; a.C = s.C; a.G = s.G; a.per = s.C / s.G;
    a.slab = p.slab; a.slabs = p.slabs; a.cluster = p.cluster; a.chunks = p.chunks; a.parts = p.parts;
    a.eps = s.eps;
    a.inv_values = 1.0 / (static_cast<double>(s.P) * a.per);
    a.inv_count = static_cast<float>(a.inv_values);
    return a;
}

template <typename T, typename F> cudaError_t by_width(int index, F f) {
    if (index == 0) return f(T{}, std::integral_constant<int, 16 / sizeof(T)>{});
    if (index == 1) return f(T{}, std::integral_constant<int, 2>{});
    return f(T{}, std::integral_constant<int, 1>{});
}
// f(type, std::integral_constant<int, V>)
template <typename F> cudaError_t by_type(int dtype, int index, F f) {
    if (dtype == PATDNN_F32) return by_width<float>(index, f);
    if (dtype == PATDNN_F16) return by_width<__half>(index, f);
    return by_width<__nv_bfloat16>(index, f);
}

dim3 resident_grid(const NormShape &s, const NormPlan &p) {
    return dim3(static_cast<unsigned>(static_cast<int64_t>(s.N) * p.slabs * p.cluster));
}

}  // namespace

int norm_width(int dtype, int index) { return index == 0 ? 16 / elem_bytes(dtype) : index == 1 ? 2 : 1; }

void plan_norm(NormHandle &h) {
    for (int i = 0; i < kNormWidths; ++i) {
        const int v = norm_width(h.s.dtype, i);
        if (!width_fits(h.s, v)) continue;
        h.fwd[i] = plan_one(h.s, v, 1, 1);
        h.mx4[i] = plan_one(h.s, v, 1, 32);
        h.bwd[i] = plan_one(h.s, v, 2, 1);
    }
}

size_t norm_workspace_floats(const NormHandle &h) {
    size_t most = 0;
    for (int i = 0; i < kNormWidths; ++i)
        for (const NormPlan *p : {&h.fwd[i], &h.mx4[i], &h.bwd[i]}) {
            const size_t cells = std::max<size_t>(p->slabs, std::max(h.s.C, h.s.G));
            most = std::max(most, static_cast<size_t>(h.s.N) * p->chunks * cells * 2 + static_cast<size_t>(h.s.N) * h.s.G * 2);
        }
    return most;
}

cudaError_t prepare_norm() {
    for (int dtype = 0; dtype < 3; ++dtype)
        for (int i = 0; i < kNormWidths; ++i) {
            const cudaError_t e = by_type(dtype, i, [](auto t, auto v) {
                using T = decltype(t);
                const cudaFuncAttribute what = cudaFuncAttributeMaxDynamicSharedMemorySize;
                cudaError_t r = cudaFuncSetAttribute(norm_moments_kernel<T, v.value>, what, kSmemMost);
                for (int act = PATDNN_ACT_NONE; act <= PATDNN_ACT_SILU && r == cudaSuccess; ++act)
                    r = by_act(act, [&](auto c) {
                        cudaError_t q = cudaFuncSetAttribute(norm_resident_kernel<T, v.value, c.value, false>, what, kSmemMost);
                        if (q == cudaSuccess) q = cudaFuncSetAttribute(norm_resident_kernel<T, v.value, c.value, true>, what, kSmemMost);
                        if (q == cudaSuccess) q = cudaFuncSetAttribute(norm_grad_resident_kernel<T, v.value, c.value>, what, kSmemMost);
                        if (q == cudaSuccess) q = cudaFuncSetAttribute(norm_apply_kernel<T, v.value, c.value>, what, kSmemMost);
                        if (q == cudaSuccess) q = cudaFuncSetAttribute(norm_grad_sums_kernel<T, v.value, c.value>, what, kSmemMost);
                        if (q == cudaSuccess) q = cudaFuncSetAttribute(norm_grad_apply_kernel<T, v.value, c.value>, what, kSmemMost);
                        return q;
                    });
                return r;
            });
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

namespace {

// Two passes over runs of images; after_run(first image, images) launches what reads the statistics.
template <typename F>
cudaError_t two_pass(const NormHandle &h, const NormPlan &p, int i, NormArgs a, cudaStream_t st, int *launches, F after_run) {
    const NormShape &s = h.s;
    *launches = 0;
    for (int n0 = 0; n0 < s.N; n0 += p.run) {
        const int images = std::min(p.run, s.N - n0);
        a.n0 = n0;
        const dim3 grid(p.chunks, p.slabs, images);
        cudaError_t e = by_type(s.dtype, i, [&](auto t, auto v) {
            return launch_pdl(norm_moments_kernel<decltype(t), v.value>, grid, dim3(kThreads), ring_smem<decltype(t), v.value, 1>(), st, 1, a);
        });
        if (e == cudaSuccess) e = launch_pdl(norm_join_kernel, dim3(s.G, images), dim3(kThreads), 0, st, 1, a);
        if (e == cudaSuccess) e = after_run(a, grid);
        if (e != cudaSuccess) return e;
        *launches += 3;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_group_norm(const NormHandle &h, const void *x, const float *gamma, const float *beta, void *y, float *stats,
                              cudaStream_t st, int *launches) {
    const NormShape &s = h.s;
    const int i = width_index(s, {x, y}, true);
    const NormPlan &p = h.fwd[i];
    NormArgs a = args_of(h, p);
    a.x = x; a.y = y; a.gamma = gamma; a.beta = beta; a.stats_out = stats;
    if (p.resident) {
        *launches = 1;
        return by_type(s.dtype, i, [&](auto t, auto v) {
            return by_act(s.act, [&](auto c) {
                return launch_pdl(norm_resident_kernel<decltype(t), v.value, c.value, false>, resident_grid(s, p), dim3(kThreads), p.smem, st, p.cluster, a);
            });
        });
    }
    if (!stats) stats = h.stats;
    a.stats_out = stats; a.stats_in = stats;
    return two_pass(h, p, i, a, st, launches, [&](const NormArgs &b, dim3 grid) {
        return by_type(s.dtype, i, [&](auto t, auto v) {
            return by_act(s.act, [&](auto c) {
                return launch_pdl(norm_apply_kernel<decltype(t), v.value, c.value>, grid, dim3(kThreads), ring_smem<decltype(t), v.value, 1>(), st, 1, b);
            });
        });
    });
}

cudaError_t launch_group_norm_mx4(const NormHandle &h, const void *x, const float *gamma, const float *beta, void *mx, float *stats,
                                  cudaStream_t st, int *launches) {
    const NormShape &s = h.s;
    const int i = width_index(s, {x}, false);
    const NormPlan &p = h.mx4[i];
    const Mx4Shape m = mx4_shape(s.N * s.P, s.C);
    NormArgs a = args_of(h, p);
    a.x = x; a.gamma = gamma; a.beta = beta; a.stats_out = stats;
    a.mx = static_cast<uint8_t *>(mx); a.mx_scales = m.scales_at; a.mx_width = m.width; a.mx_col_tiles = static_cast<int>(m.col_tiles);
    if (p.resident) {
        *launches = 1;
        return by_type(s.dtype, i, [&](auto t, auto v) {
            return by_act(s.act, [&](auto c) {
                return launch_pdl(norm_resident_kernel<decltype(t), v.value, c.value, true>, resident_grid(s, p), dim3(kThreads), p.smem, st, p.cluster, a);
            });
        });
    }
    if (!stats) stats = h.stats;
    a.stats_out = stats;
    return two_pass(h, p, i, a, st, launches, [&](const NormArgs &b, dim3 grid) {
        return launch_norm_quantize(s, m, x, gamma, beta, stats, b.n0 * s.P, static_cast<int64_t>(grid.z) * s.P, mx, st);
    });
}

cudaError_t launch_group_norm_grad(const NormHandle &h, const void *x, const float *gamma, const float *beta, const float *stats,
                                   const void *dy, void *dx, float *dgamma, float *dbeta, cudaStream_t st, int *launches) {
    const NormShape &s = h.s;
    const int i = width_index(s, {x, dy, dx}, true);
    const NormPlan &p = h.bwd[i];
    NormArgs a = args_of(h, p);
    a.x = x; a.dy = dy; a.y = dx; a.gamma = gamma; a.beta = beta; a.stats_in = stats; a.dgamma = dgamma; a.dbeta = dbeta;
    if (p.resident) {
        *launches = 1;
        return by_type(s.dtype, i, [&](auto t, auto v) {
            return by_act(s.act, [&](auto c) {
                return launch_pdl(norm_grad_resident_kernel<decltype(t), v.value, c.value>, resident_grid(s, p), dim3(kThreads), p.smem, st, p.cluster, a);
            });
        });
    }
    *launches = 0;
    for (int n0 = 0; n0 < s.N; n0 += p.run) {
        const int images = std::min(p.run, s.N - n0);
        a.n0 = n0;
        const dim3 grid(p.chunks, p.slabs, images);
        const cudaError_t e = by_type(s.dtype, i, [&](auto t, auto v) {
            return by_act(s.act, [&](auto c) {
                using T = decltype(t);
                cudaError_t r = launch_pdl(norm_grad_sums_kernel<T, v.value, c.value>, grid, dim3(kThreads), ring_smem<T, v.value, 2>(), st, 1, a);
                if (r == cudaSuccess) r = launch_pdl(norm_grad_join_kernel, dim3(s.G, images), dim3(kThreads), 0, st, 1, a);
                if (r == cudaSuccess) r = launch_pdl(norm_grad_apply_kernel<T, v.value, c.value>, grid, dim3(kThreads), ring_smem<T, v.value, 2>(), st, 1, a);
                return r;
            });
        });
        if (e != cudaSuccess) return e;
        *launches += 3;
    }
    return cudaSuccess;
}

}  // namespace patdnn

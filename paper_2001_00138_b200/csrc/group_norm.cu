// Group norm with an activation over channels-last tensors, and its gradient.
//
//   x [N][P][C], group g of channel c = c / (C / G); mean, var over the P * C/G values of (n, g), rstd = 1/sqrt(var + eps)
//   xh = (x - mean) * rstd, z = xh * gamma_c + beta_c, y = act(z)
//   gradient: dz = dy * act'(z); A_nc = sum_p dz, B_nc = sum_p dz * xh; dbeta = sum_n A, dgamma = sum_n B;
//   with m = P * C/G, s1 = sum_{c in g} gamma_c A_nc / m, s2 = sum_{c in g} gamma_c B_nc / m:
//   dx = rstd * (gamma_c * dz - s1 - xh * s2)
//
// Both are bound by HBM: the forward's floor is one read of x and one write of y, the gradient's one read of x and dy and one
// write of dx.  Two forms:
//   resident  a thread-block cluster (up to 8 CTAs) owns a slab of whole groups of one image, keeps it in shared memory
//             while the statistics are formed and joined over distributed shared memory, and writes the result from there: one
//             launch, every value read once.
//   two-pass  images whose slabs do not fit: partial statistics per (chunk of pixels, channel), a small kernel that joins
//             them, and an elementwise pass that reads x again (from L2 where it still is there).
// All sums are fp32 and joined in a fixed order.  Variances are never formed as a difference of two large sums: a thread sums (x - m)
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
constexpr int kBatch = 8;                   // pixels a thread loads at a time

struct NormArgs {
    const void *x, *dy;
    void *y;                                // dx in the gradient
    const float *gamma, *beta, *stats_in;
    float *stats_out, *dgamma, *dbeta;
    float *ws;
    unsigned *counters;
    int64_t x_pixel, x_image, y_pixel, y_image, P, chunk;
    int N, C, G, per;                       // per = C / G
    int slab, slabs, cluster, chunks, act;
    float eps, inv_count;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Running mean and sum of squared deviations of V channels over the pixels a thread visits.  `add` takes a batch of up to kBatch pixels:
// the sums are taken around the running mean (around the first pixel in the first batch), so a batch of b values loses
// at most about b rounding errors of the largest deviation.
template <int V>
struct Moments {
    float mean[V], m2[V], s1[V], s2[V];
    int n;
    __device__ __forceinline__ void clear() {
        n = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) mean[j] = m2[j] = 0.f;
    }
    template <typename T>
    __device__ __forceinline__ void begin(const Vec<T, V> &first) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            s1[j] = s2[j] = 0.f;
            if (n == 0) mean[j] = to_float(first.v[j]);
        }
    }
    template <typename T>
    __device__ __forceinline__ void take(const Vec<T, V> &x) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = to_float(x.v[j]) - mean[j];
            s1[j] += d;
            s2[j] = fmaf(d, d, s2[j]);
        }
    }
    __device__ __forceinline__ void end(int count) {
        n += count;
        const float inv = __fdividef(1.f, static_cast<float>(n));
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float shift = s1[j] * inv;
            mean[j] += shift;
            m2[j] = fmaxf(m2[j] + s2[j] - s1[j] * shift, 0.f) + 0.f * s2[j];   // the last term keeps NaN and infinity
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

// Joins the per-thread moments of a CTA per group of its slab.  red: [rows][channels] (mean, m2); a warp takes a group at a time:
// first the mean over all its entries, then the squared deviations around it.  grp[g] = (mean, m2) over n0 * per values.
__device__ __forceinline__ void join_groups(const float2 *red, int rows, int channels, int per, int64_t pixels, float2 *grp) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int groups = channels / per;
    const float total = static_cast<float>(pixels) * per;
    for (int g = warp; g < groups; g += kThreads / 32) {
        float s = 0.f;
        for (int r = lane; r < rows; r += 32) {
            const float n = static_cast<float>((pixels - r + rows - 1) / rows);     // pixels that row r visited
            float t = 0.f;
            if (n > 0.f) for (int c = 0; c < per; ++c) t += red[r * channels + g * per + c].x;
            s += n * t;
        }
        const float mean = warp_sum(s) / total;
        float q = 0.f;
        for (int r = lane; r < rows; r += 32) {
            const float n = static_cast<float>((pixels - r + rows - 1) / rows);
            if (n > 0.f)
                for (int c = 0; c < per; ++c) {
                    const float2 e = red[r * channels + g * per + c];
                    const float d = e.x - mean;
                    q += e.y + n * d * d;
                }
        }
        q = warp_sum(q);
        if (lane == 0) grp[g] = make_float2(mean, q);
    }
}

// ---- resident form ----------------------------------------------------------------------------------------------------
// Shared memory: [chunk][slab] elements of x, then [rows][slab] float2, then [groups of the slab] float2 twice.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 2) norm_resident_kernel(NormArgs a) {
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
    float2 *grp = red + kThreads * V;
    float2 *fin = grp + a.slab / a.per;
    const int groups = channels / a.per;
    pdl_wait();

    Moments<V> m;
    m.clear();
    if (q.on) {
        const T *src = static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V;
        for (int p = q.row; p < pixels; p += q.rows * kBatch) {
            Vec<T, V> v[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (p + u * q.rows < pixels) v[u] = *reinterpret_cast<const Vec<T, V> *>(src + (p + u * q.rows) * a.x_pixel);
            m.begin(v[0]);
            int count = 0;
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (p + u * q.rows < pixels) {
                    m.take(v[u]);
                    ++count;
                    *reinterpret_cast<Vec<T, V> *>(tile + (p + u * q.rows) * channels + q.col * V) = v[u];
                }
            m.end(count);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) red[q.row * channels + q.col * V + j] = make_float2(m.mean[j], m.m2[j]);
    }
    __syncthreads();
    join_groups(red, q.rows, channels, a.per, pixels, grp);
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    for (int g = threadIdx.x; g < groups; g += kThreads) {
        float s = 0.f, sq = 0.f;
        for (int r = 0; r < a.cluster; ++r) {
            const float cnt = static_cast<float>(max(int64_t(0), min(a.P - r * a.chunk, a.chunk)));
            if (cnt > 0.f) s += cnt * cluster.map_shared_rank(grp, r)[g].x;
        }
        const float mean = s / static_cast<float>(a.P);
        for (int r = 0; r < a.cluster; ++r) {
            const float cnt = static_cast<float>(max(int64_t(0), min(a.P - r * a.chunk, a.chunk))) * a.per;
            if (cnt > 0.f) {
                const float2 e = cluster.map_shared_rank(grp, r)[g];
                sq += e.y + cnt * (e.x - mean) * (e.x - mean);
            }
        }
        const float rstd = 1.f / sqrtf(sq * a.inv_count + a.eps);
        fin[g] = make_float2(mean, rstd);
        if (a.stats_out && rank == 0) {
            float *o = a.stats_out + (static_cast<int64_t>(n) * a.G + c0 / a.per + g) * 2;
            o[0] = mean; o[1] = rstd;
        }
    }
    cluster.sync();                                    // fin is ready; nobody reads this CTA's grp after this point
    if (!q.on || !a.y) return;
    float mean[V], scale[V], beta[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = q.col * V + j;
        const float2 f = fin[c / a.per];
        mean[j] = f.x; scale[j] = f.y * a.gamma[c0 + c]; beta[j] = a.beta[c0 + c];
    }
    T *dst = static_cast<T *>(a.y) + n * a.y_image + p0 * a.y_pixel + c0 + q.col * V;
#pragma unroll 4
    for (int p = q.row; p < pixels; p += q.rows) {
        const Vec<T, V> v = *reinterpret_cast<const Vec<T, V> *>(tile + p * channels + q.col * V);
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(activate(fmaf(to_float(v.v[j]) - mean[j], scale[j], beta[j]), a.act));
        *reinterpret_cast<Vec<T, V> *>(dst + p * a.y_pixel) = o;
    }
}

// Sums A and B of the gradient over the pixels a thread visits, and dx; x, dy in registers.
template <int V>
struct Affine {
    float mean[V], rstd[V], gamma[V], beta[V];
    template <typename T>
    __device__ __forceinline__ void slope(const Vec<T, V> &x, const Vec<T, V> &dy, int act, float (&xh)[V], float (&dz)[V]) const {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            xh[j] = (to_float(x.v[j]) - mean[j]) * rstd[j];
            dz[j] = to_float(dy.v[j]) * activate_slope(fmaf(xh[j], gamma[j], beta[j]), act);
        }
    }
};

// dgamma and dbeta of the channels [c0, c0 + channels) from the per-image sums ws [N][C] (A, B), images in ascending order.
__device__ __forceinline__ void sum_images(const NormArgs &a, int c0, int channels) {
    for (int c = c0 + threadIdx.x; c < c0 + channels; c += kThreads) {
        float sa = 0.f, sb = 0.f;
        for (int n = 0; n < a.N; ++n) {
            const float2 e = __ldcg(reinterpret_cast<const float2 *>(a.ws) + static_cast<int64_t>(n) * a.C + c);
            sa += e.x; sb += e.y;
        }
        a.dbeta[c] = sa;
        a.dgamma[c] = sb;
    }
}

// Shared memory: [chunk][slab] elements of x, the same of dy, [rows][slab] float2, [slab] float2 twice, [groups] float2.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 2) norm_grad_resident_kernel(NormArgs a) {
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
    float2 *whole = sums + a.slab;                     // the image's (A, B) per channel
    float2 *fin = whole + a.slab;                      // (s1, s2) per group
    pdl_wait();

    Affine<V> f;
    if (q.on) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = c0 + q.col * V + j;
            const float2 st = reinterpret_cast<const float2 *>(a.stats_in)[static_cast<int64_t>(n) * a.G + c / a.per];
            f.mean[j] = st.x; f.rstd[j] = st.y; f.gamma[j] = a.gamma[c]; f.beta[j] = a.beta[c];
        }
        float sa[V], sb[V];
#pragma unroll
        for (int j = 0; j < V; ++j) sa[j] = sb[j] = 0.f;
        const T *xs = static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V;
        const T *ds = static_cast<const T *>(a.dy) + n * a.y_image + p0 * a.y_pixel + c0 + q.col * V;
        constexpr int kHalf = kBatch / 2;              // two tensors: the same bytes in flight
        for (int p = q.row; p < pixels; p += q.rows * kHalf) {
            Vec<T, V> xv[kHalf], dv[kHalf];
#pragma unroll
            for (int u = 0; u < kHalf; ++u)
                if (p + u * q.rows < pixels) {
                    xv[u] = *reinterpret_cast<const Vec<T, V> *>(xs + (p + u * q.rows) * a.x_pixel);
                    dv[u] = *reinterpret_cast<const Vec<T, V> *>(ds + (p + u * q.rows) * a.y_pixel);
                }
#pragma unroll
            for (int u = 0; u < kHalf; ++u)
                if (p + u * q.rows < pixels) {
                    float xh[V], dz[V];
                    f.slope(xv[u], dv[u], a.act, xh, dz);
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        sa[j] += dz[j];
                        sb[j] = fmaf(dz[j], xh[j], sb[j]);
                    }
                    const int at = (p + u * q.rows) * channels + q.col * V;
                    *reinterpret_cast<Vec<T, V> *>(xt + at) = xv[u];
                    *reinterpret_cast<Vec<T, V> *>(dt + at) = dv[u];
                }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) red[q.row * channels + q.col * V + j] = make_float2(sa[j], sb[j]);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < channels; c += kThreads) {
        float2 s = make_float2(0.f, 0.f);
        for (int r = 0; r < q.rows; ++r) {
            const float2 e = red[r * channels + c];
            s.x += e.x; s.y += e.y;
        }
        sums[c] = s;
    }
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    for (int c = threadIdx.x; c < channels; c += kThreads) {
        float2 s = make_float2(0.f, 0.f);
        for (int r = 0; r < a.cluster; ++r) {
            const float2 e = cluster.map_shared_rank(sums, r)[c];
            s.x += e.x; s.y += e.y;
        }
        whole[c] = s;
        if (rank == 0) reinterpret_cast<float2 *>(a.ws)[static_cast<int64_t>(n) * a.C + c0 + c] = s;
    }
    __syncthreads();
    for (int g = threadIdx.x; g < channels / a.per; g += kThreads) {
        float s1 = 0.f, s2 = 0.f;
        for (int c = 0; c < a.per; ++c) {
            const float gm = a.gamma[c0 + g * a.per + c];
            const float2 e = whole[g * a.per + c];
            s1 = fmaf(gm, e.x, s1);
            s2 = fmaf(gm, e.y, s2);
        }
        fin[g] = make_float2(s1 * a.inv_count, s2 * a.inv_count);
    }
    cluster.sync();                                    // fin is ready; nobody reads this CTA's sums after this point
    if (q.on && a.y) {
        float s1[V], s2[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float2 e = fin[(q.col * V + j) / a.per];
            s1[j] = e.x; s2[j] = e.y;
        }
        T *dst = static_cast<T *>(a.y) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V;
#pragma unroll 2
        for (int p = q.row; p < pixels; p += q.rows) {
            const Vec<T, V> xv = *reinterpret_cast<const Vec<T, V> *>(xt + p * channels + q.col * V);
            const Vec<T, V> dv = *reinterpret_cast<const Vec<T, V> *>(dt + p * channels + q.col * V);
            float xh[V], dz[V];
            f.slope(xv, dv, a.act, xh, dz);
            Vec<T, V> o;
#pragma unroll
            for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(f.rstd[j] * (fmaf(f.gamma[j], dz[j], -s1[j]) - xh[j] * s2[j]));
            *reinterpret_cast<Vec<T, V> *>(dst + p * a.x_pixel) = o;
        }
    }
    // the last cluster of this slab to get here adds the images up; what it adds, and in which order, does not depend on who is last
    if (rank != 0) return;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(a.counters + slab, 1u) == static_cast<unsigned>(a.N) - 1;
        if (last) a.counters[slab] = 0;
        __threadfence();
    }
    __syncthreads();
    if (last) sum_images(a, c0, channels);
}

// ---- two-pass form ----------------------------------------------------------------------------------------------------
// blockIdx = (chunk, slab, image); ws [N][chunks][C] (mean, m2) of the chunk's pixels.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) norm_moments_kernel(NormArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    float2 *red = reinterpret_cast<float2 *>(smem);
    pdl_trigger();
    const int n = blockIdx.z, c0 = blockIdx.y * a.slab, channels = min(a.slab, a.C - c0);
    const int64_t p0 = blockIdx.x * a.chunk, p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(channels);
    pdl_wait();
    if (q.on) {
        Moments<V> m;
        m.clear();
        const T *src = static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V;
        for (int p = q.row; p < pixels; p += q.rows * kBatch) {
            Vec<T, V> v[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (p + u * q.rows < pixels) v[u] = *reinterpret_cast<const Vec<T, V> *>(src + (p + u * q.rows) * a.x_pixel);
            m.begin(v[0]);
            int count = 0;
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (p + u * q.rows < pixels) {
                    m.take(v[u]);
                    ++count;
                }
            m.end(count);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) red[q.row * channels + q.col * V + j] = make_float2(m.mean[j], m.m2[j]);
    }
    __syncthreads();
    float2 *out = reinterpret_cast<float2 *>(a.ws) + (static_cast<int64_t>(n) * a.chunks + blockIdx.x) * a.C + c0;
    for (int c = threadIdx.x; c < channels; c += kThreads) {
        float s = 0.f, sq = 0.f;
        const int rows = min(q.rows, pixels);
        for (int r = 0; r < rows; ++r) s += static_cast<float>((pixels - r + q.rows - 1) / q.rows) * red[r * channels + c].x;
        const float mean = s / static_cast<float>(pixels);
        for (int r = 0; r < rows; ++r) {
            const float2 e = red[r * channels + c];
            const float d = e.x - mean;
            sq += e.y + static_cast<float>((pixels - r + q.rows - 1) / q.rows) * d * d;
        }
        out[c] = make_float2(mean, sq);
    }
}

__device__ __forceinline__ float block_sum(float v, float *scratch) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) s += scratch[w];
    return s;
}

// One CTA per (group, image): joins the chunks' moments of the group's channels.
__global__ void __launch_bounds__(kThreads) norm_join_kernel(NormArgs a) {
    __shared__ float scratch[kThreads / 32];
    pdl_trigger();
    pdl_wait();
    const int g = blockIdx.x, n = blockIdx.y;
    const float2 *part = reinterpret_cast<const float2 *>(a.ws) + static_cast<int64_t>(n) * a.chunks * a.C + g * a.per;
    const int items = a.chunks * a.per;
    float s = 0.f, sq = 0.f;
    for (int i = threadIdx.x; i < items; i += kThreads) {
        const int k = i / a.per, c = i % a.per;
        const float cnt = static_cast<float>(min(a.chunk, a.P - k * a.chunk));
        s += cnt * part[static_cast<int64_t>(k) * a.C + c].x;
    }
    const float mean = block_sum(s, scratch) * a.inv_count;
    for (int i = threadIdx.x; i < items; i += kThreads) {
        const int k = i / a.per, c = i % a.per;
        const float cnt = static_cast<float>(min(a.chunk, a.P - k * a.chunk));
        const float2 e = part[static_cast<int64_t>(k) * a.C + c];
        sq += e.y + cnt * (e.x - mean) * (e.x - mean);
    }
    sq = block_sum(sq, scratch);
    if (threadIdx.x == 0) {
        float *o = a.stats_out + (static_cast<int64_t>(n) * a.G + g) * 2;
        o[0] = mean;
        o[1] = 1.f / sqrtf(sq * a.inv_count + a.eps);
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(kThreads) norm_apply_kernel(NormArgs a) {
    pdl_trigger();
    const int n = blockIdx.z, c0 = blockIdx.y * a.slab, channels = min(a.slab, a.C - c0);
    const int64_t p0 = blockIdx.x * a.chunk, p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(channels);
    pdl_wait();
    if (!q.on) return;
    float mean[V], scale[V], beta[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = c0 + q.col * V + j;
        const float2 f = reinterpret_cast<const float2 *>(a.stats_in)[static_cast<int64_t>(n) * a.G + c / a.per];
        mean[j] = f.x; scale[j] = f.y * a.gamma[c]; beta[j] = a.beta[c];
    }
    const T *src = static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V;
    T *dst = static_cast<T *>(a.y) + n * a.y_image + p0 * a.y_pixel + c0 + q.col * V;
#pragma unroll 4
    for (int p = q.row; p < pixels; p += q.rows) {
        const Vec<T, V> v = *reinterpret_cast<const Vec<T, V> *>(src + p * a.x_pixel);
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(activate(fmaf(to_float(v.v[j]) - mean[j], scale[j], beta[j]), a.act));
        *reinterpret_cast<Vec<T, V> *>(dst + p * a.y_pixel) = o;
    }
}

// ws [N][chunks][C] (A, B) of the chunk's pixels.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) norm_grad_sums_kernel(NormArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    float2 *red = reinterpret_cast<float2 *>(smem);
    pdl_trigger();
    const int n = blockIdx.z, c0 = blockIdx.y * a.slab, channels = min(a.slab, a.C - c0);
    const int64_t p0 = blockIdx.x * a.chunk, p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(channels);
    pdl_wait();
    if (q.on) {
        Affine<V> f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = c0 + q.col * V + j;
            const float2 st = reinterpret_cast<const float2 *>(a.stats_in)[static_cast<int64_t>(n) * a.G + c / a.per];
            f.mean[j] = st.x; f.rstd[j] = st.y; f.gamma[j] = a.gamma[c]; f.beta[j] = a.beta[c];
        }
        float sa[V], sb[V];
#pragma unroll
        for (int j = 0; j < V; ++j) sa[j] = sb[j] = 0.f;
        const T *xs = static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V;
        const T *ds = static_cast<const T *>(a.dy) + n * a.y_image + p0 * a.y_pixel + c0 + q.col * V;
#pragma unroll 4
        for (int p = q.row; p < pixels; p += q.rows) {
            float xh[V], dz[V];
            f.slope(*reinterpret_cast<const Vec<T, V> *>(xs + p * a.x_pixel), *reinterpret_cast<const Vec<T, V> *>(ds + p * a.y_pixel),
                    a.act, xh, dz);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sa[j] += dz[j];
                sb[j] = fmaf(dz[j], xh[j], sb[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) red[q.row * channels + q.col * V + j] = make_float2(sa[j], sb[j]);
    }
    __syncthreads();
    float2 *out = reinterpret_cast<float2 *>(a.ws) + (static_cast<int64_t>(n) * a.chunks + blockIdx.x) * a.C + c0;
    for (int c = threadIdx.x; c < channels; c += kThreads) {
        float2 s = make_float2(0.f, 0.f);
        for (int r = 0; r < q.rows; ++r) {
            const float2 e = red[r * channels + c];
            s.x += e.x; s.y += e.y;
        }
        out[c] = s;
    }
}

// One CTA per (group, image): sums the chunks, writes (s1, s2) of the group behind the partial sums and the image's (A, B) per channel
// into chunk 0's place.
__global__ void __launch_bounds__(kThreads) norm_grad_join_kernel(NormArgs a) {
    __shared__ float scratch[kThreads / 32];
    pdl_trigger();
    pdl_wait();
    const int g = blockIdx.x, n = blockIdx.y;
    float2 *part = reinterpret_cast<float2 *>(a.ws) + static_cast<int64_t>(n) * a.chunks * a.C + g * a.per;
    float s1 = 0.f, s2 = 0.f;
    for (int c = 0; c < a.per; ++c) {
        float sa = 0.f, sb = 0.f;
        for (int k = threadIdx.x; k < a.chunks; k += kThreads) {
            const float2 e = part[static_cast<int64_t>(k) * a.C + c];
            sa += e.x; sb += e.y;
        }
        sa = block_sum(sa, scratch);
        sb = block_sum(sb, scratch);                   // (its barriers also order the reads above before the write below)
        if (threadIdx.x == 0) part[c] = make_float2(sa, sb);
        const float gm = a.gamma[g * a.per + c];
        s1 = fmaf(gm, sa, s1);
        s2 = fmaf(gm, sb, s2);
    }
    if (threadIdx.x == 0)
        reinterpret_cast<float2 *>(a.ws)[static_cast<int64_t>(a.N) * a.chunks * a.C + static_cast<int64_t>(n) * a.G + g] =
            make_float2(s1 * a.inv_count, s2 * a.inv_count);
}

template <typename T, int V>
__global__ void __launch_bounds__(kThreads) norm_grad_apply_kernel(NormArgs a) {
    pdl_trigger();
    const int n = blockIdx.z, c0 = blockIdx.y * a.slab, channels = min(a.slab, a.C - c0);
    const int64_t p0 = blockIdx.x * a.chunk, p1 = min(a.P, p0 + a.chunk);
    const int pixels = static_cast<int>(p1 - p0);
    const Place q = place_of<V>(channels);
    pdl_wait();
    const float2 *ws = reinterpret_cast<const float2 *>(a.ws);
    if (n == 0 && blockIdx.x == 0)                     // one CTA per slab also adds the images up
        for (int c = c0 + threadIdx.x; c < c0 + channels; c += kThreads) {
            float sa = 0.f, sb = 0.f;
            for (int i = 0; i < a.N; ++i) {
                const float2 e = ws[static_cast<int64_t>(i) * a.chunks * a.C + c];
                sa += e.x; sb += e.y;
            }
            a.dbeta[c] = sa;
            a.dgamma[c] = sb;
        }
    if (!q.on || !a.y) return;
    Affine<V> f;
    float s1[V], s2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = c0 + q.col * V + j;
        const int64_t g = static_cast<int64_t>(n) * a.G + c / a.per;
        const float2 st = reinterpret_cast<const float2 *>(a.stats_in)[g];
        f.mean[j] = st.x; f.rstd[j] = st.y; f.gamma[j] = a.gamma[c]; f.beta[j] = a.beta[c];
        const float2 e = ws[static_cast<int64_t>(a.N) * a.chunks * a.C + g];
        s1[j] = e.x; s2[j] = e.y;
    }
    const T *xs = static_cast<const T *>(a.x) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V;
    const T *ds = static_cast<const T *>(a.dy) + n * a.y_image + p0 * a.y_pixel + c0 + q.col * V;
    T *dst = static_cast<T *>(a.y) + n * a.x_image + p0 * a.x_pixel + c0 + q.col * V;
#pragma unroll 4
    for (int p = q.row; p < pixels; p += q.rows) {
        float xh[V], dz[V];
        f.slope(*reinterpret_cast<const Vec<T, V> *>(xs + p * a.x_pixel), *reinterpret_cast<const Vec<T, V> *>(ds + p * a.y_pixel),
                a.act, xh, dz);
        Vec<T, V> o;
#pragma unroll
        for (int j = 0; j < V; ++j) o.v[j] = from_float<T>(f.rstd[j] * (fmaf(f.gamma[j], dz[j], -s1[j]) - xh[j] * s2[j]));
        *reinterpret_cast<Vec<T, V> *>(dst + p * a.x_pixel) = o;
    }
}

// ---- planning -----------------------------------------------------------------------------------------------------------
int resident_smem(const NormShape &s, int width, int tensors, int slab, int64_t chunk) {
    const int64_t tile = (chunk * slab * elem_bytes(s.dtype) + 15) / 16 * 16;
    const int64_t groups = slab / (s.C / s.G);
    const int64_t small = tensors == 1 ? 2 * groups : 2 * slab + groups;
    const int64_t total = tensors * tile + (static_cast<int64_t>(kThreads) * width + small) * 8;
    return total > (int64_t(1) << 30) ? (1 << 30) : static_cast<int>(total);
}

constexpr int kSmemMost = 220 * 1024;       // dynamic shared memory of one CTA

// Picks the slab and the cluster of the resident form by a time estimate: a CTA loads its share at its part of an SM's HBM rate
// (44 bytes per ns), then stores it; `per_sm` CTAs overlap; every wave pays a fixed latency.  Slabs narrower than 128
// bytes cost more per byte.
NormPlan plan_one(const NormShape &s, int width, int tensors) {
    NormPlan best;
    const int per = s.C / s.G, e = elem_bytes(s.dtype);
    double best_us = 1e30;
    for (int k = 1; k <= s.G; ++k) {
        if (s.G % k) continue;
        const int64_t slab = static_cast<int64_t>(k) * per;
        if (slab % width || slab / width > kThreads) continue;
        if (slab * e < 64 && k < s.G) continue;
        for (int cl = 1; cl <= 8; cl *= 2) {
            if (cl > s.P) break;
            const int64_t chunk = ceil_div(s.P, cl);
            const int smem = resident_smem(s, width, tensors, static_cast<int>(slab), chunk);
            if (smem > kSmemMost || static_cast<int64_t>(s.N) * (s.G / k) * cl > INT32_MAX) continue;
            const int per_sm = std::min(2, (224 * 1024) / (smem + 2048));
            const double ctas = static_cast<double>(s.N) * (s.G / k) * cl;
            const double waves = std::ceil(ctas / (148.0 * per_sm));
            const double bytes = static_cast<double>(chunk) * slab * e * (tensors + 1);
            const double narrow = slab * e < 128 && k < s.G ? 1.2 : 1.0;
            const double us = waves * ((per_sm * bytes / 44e3) * narrow * (per_sm == 1 ? 1.3 : 1.0) + 2.5 + (cl > 1 ? 0.5 : 0.0));
            if (us < best_us) {
                best_us = us;
                best.resident = true; best.slab = static_cast<int>(slab); best.slabs = s.G / k; best.cluster = cl;
                best.chunk = chunk; best.smem = smem; best.chunks = 1;
            }
        }
    }
    if (best.resident) return best;
    const int cols = std::min(s.C / width, kThreads);
    best.slab = cols * width;
    best.slabs = static_cast<int>(ceil_div(s.C, best.slab));
    // about 64 KB per CTA, at least a few CTAs per SM over the whole tensor
    const int64_t total = static_cast<int64_t>(s.N) * s.P;
    int64_t chunk = std::max<int64_t>(1, 65536 / (static_cast<int64_t>(best.slab) * e));
    chunk = std::min(chunk, std::max<int64_t>(kThreads / cols, ceil_div(total * best.slabs, 148 * 8)));
    chunk = std::max(chunk, ceil_div(s.P, 4096));      // bounds the partial sums
    best.chunk = std::min(chunk, s.P);
    best.chunks = static_cast<int>(ceil_div(s.P, best.chunk));
    return best;
}

// Widest access that the sizes, the strides and the addresses allow.
int width_index(const NormShape &s, std::initializer_list<const void *> pointers, bool y_too) {
    const int e = elem_bytes(s.dtype);
    for (int i = 0; i < kNormWidths; ++i) {
        const int v = norm_width(s.dtype, i);
        bool ok = s.C % v == 0 && s.x_pixel % v == 0 && s.x_image % v == 0;
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
    a.slab = p.slab; a.slabs = p.slabs; a.cluster = p.cluster; a.chunks = p.chunks; a.act = s.act;
    a.eps = s.eps;
    a.inv_count = static_cast<float>(1.0 / (static_cast<double>(s.P) * a.per));
    return a;
}

template <typename F> cudaError_t by_type(int dtype, int index, F f) {
    if (dtype == PATDNN_F32) {
        if (index == 0) return f(float{}, std::integral_constant<int, 4>{});
        if (index == 1) return f(float{}, std::integral_constant<int, 2>{});
        return f(float{}, std::integral_constant<int, 1>{});
    }
    if (dtype == PATDNN_F16) {
        if (index == 0) return f(__half{}, std::integral_constant<int, 8>{});
        if (index == 1) return f(__half{}, std::integral_constant<int, 2>{});
        return f(__half{}, std::integral_constant<int, 1>{});
    }
    if (index == 0) return f(__nv_bfloat16{}, std::integral_constant<int, 8>{});
    if (index == 1) return f(__nv_bfloat16{}, std::integral_constant<int, 2>{});
    return f(__nv_bfloat16{}, std::integral_constant<int, 1>{});
}

}  // namespace

int norm_width(int dtype, int index) { return index == 0 ? 16 / elem_bytes(dtype) : index == 1 ? 2 : 1; }

void plan_norm(NormHandle &h) {
    for (int i = 0; i < kNormWidths; ++i) {
        const int v = norm_width(h.s.dtype, i);
        if (h.s.C % v) continue;
        h.fwd[i] = plan_one(h.s, v, 1);
        h.bwd[i] = plan_one(h.s, v, 2);
    }
}

size_t norm_workspace_floats(const NormHandle &h) {
    size_t most = 0;
    for (int i = 0; i < kNormWidths; ++i)
        for (const NormPlan *p : {&h.fwd[i], &h.bwd[i]})
            most = std::max(most, static_cast<size_t>(h.s.N) * p->chunks * h.s.C * 2 + static_cast<size_t>(h.s.N) * h.s.G * 2);
    return most;
}

cudaError_t prepare_norm() {
    for (int dtype = 0; dtype < 3; ++dtype)
        for (int i = 0; i < kNormWidths; ++i) {
            const cudaError_t e = by_type(dtype, i, [](auto t, auto v) {
                using T = decltype(t);
                cudaError_t r = cudaFuncSetAttribute(norm_resident_kernel<T, v.value>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost);
                if (r == cudaSuccess)
                    r = cudaFuncSetAttribute(norm_grad_resident_kernel<T, v.value>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost);
                return r;
            });
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

cudaError_t launch_group_norm(const NormHandle &h, const void *x, const float *gamma, const float *beta, void *y, float *stats,
                              cudaStream_t st, int *launches) {
    const NormShape &s = h.s;
    const int i = y ? width_index(s, {x, y}, true) : width_index(s, {x}, false);
    const NormPlan &p = h.fwd[i];
    NormArgs a = args_of(h, p);
    a.x = x; a.y = y; a.gamma = gamma; a.beta = beta; a.stats_out = stats;
    if (p.resident) {
        *launches = 1;
        const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(s.N) * p.slabs * p.cluster));
        return by_type(s.dtype, i, [&](auto t, auto v) {
            return launch_pdl(norm_resident_kernel<decltype(t), v.value>, grid, dim3(kThreads), p.smem, st, p.cluster, a);
        });
    }
    if (!stats) stats = h.stats;
    a.stats_out = stats; a.stats_in = stats;
    *launches = y ? 3 : 2;
    const dim3 grid(p.chunks, p.slabs, s.N);
    return by_type(s.dtype, i, [&](auto t, auto v) {
        using T = decltype(t);
        cudaError_t e = launch_pdl(norm_moments_kernel<T, v.value>, grid, dim3(kThreads), static_cast<size_t>(kThreads) * v.value * 8, st, 1, a);
        if (e == cudaSuccess) e = launch_pdl(norm_join_kernel, dim3(s.G, s.N), dim3(kThreads), 0, st, 1, a);
        if (e == cudaSuccess && y) e = launch_pdl(norm_apply_kernel<T, v.value>, grid, dim3(kThreads), 0, st, 1, a);
        return e;
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
        const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(s.N) * p.slabs * p.cluster));
        return by_type(s.dtype, i, [&](auto t, auto v) {
            return launch_pdl(norm_grad_resident_kernel<decltype(t), v.value>, grid, dim3(kThreads), p.smem, st, p.cluster, a);
        });
    }
    *launches = 3;
    const dim3 grid(p.chunks, p.slabs, s.N);
    return by_type(s.dtype, i, [&](auto t, auto v) {
        using T = decltype(t);
        cudaError_t e = launch_pdl(norm_grad_sums_kernel<T, v.value>, grid, dim3(kThreads), static_cast<size_t>(kThreads) * v.value * 8, st, 1, a);
        if (e == cudaSuccess) e = launch_pdl(norm_grad_join_kernel, dim3(s.G, s.N), dim3(kThreads), 0, st, 1, a);
        if (e == cudaSuccess) e = launch_pdl(norm_grad_apply_kernel<T, v.value>, grid, dim3(kThreads), 0, st, 1, a);
        return e;
    });
}

}  // namespace patdnn

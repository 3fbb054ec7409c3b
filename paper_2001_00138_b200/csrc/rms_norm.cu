// RMS norm of rows with the residual's addition in front, written in the rows' type or as 8-bit blocks, and its gradient.
//
//   s = x + residual, rstd = 1 / sqrt(mean(s^2) + eps), y = (s rstd) gamma
//   gradient, with xh = s rstd and u = dy gamma: dx = rstd (u - xh mean(u xh)) + dsum, dgamma = sum over rows of dy xh
//
// s is formed in fp32 and stays there for the statistics and for y; only the stored sum is rounded.  Memory bound: one pass, a row lives in
// the registers of 1 to 16 warps (32 E columns each), of up to eight CTAs of a cluster for very long rows.  The warps of a row walk over
// rows: gamma (and the gradient's dgamma) stay in registers, and the next row's loads are issued before the present row's sums are joined.
#include "feed_forward.hpp"

#include <algorithm>

#include "kernels.hpp"
#include "mx8_device.cuh"

namespace patdnn {
namespace {

constexpr int kMostWarps = 16;

struct RmsArgs {
    const void *x, *residual, *dsum;
    const float *gamma;
    void *sum, *y;
    uint8_t *mx;
    float *rstd, *ws;
    int64_t rows, x_row, r_row, y_row, scales_at;
    int C, warps, cluster, col_tiles, groups;          // warps: of a row, per CTA
    float eps;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    return v;
}
__device__ __forceinline__ uint32_t rank_in_cluster() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The sum over a row of every warp's value, the same bits in all of its threads.  Two sets of slots in turn: a set is written again only
// behind the barrier of the call between.
struct RowSum {
    float (*slots)[8][kMostWarps];                     // [2][CTA of the cluster][warp of the CTA]
    int warps, cluster, row_group, first_warp;
    uint32_t rank;
    int turn;
    __device__ __forceinline__ float operator()(float v) {
        v = warp_sum(v);
        if (warps == 1) return v;
        const int warp = threadIdx.x >> 5;
        float(&set)[8][kMostWarps] = slots[turn];
        turn ^= 1;
        float total = 0.f;
        if (cluster == 1) {
            if ((threadIdx.x & 31) == 0) set[0][warp] = v;
            asm volatile("bar.sync %0, %1;" ::"r"(row_group + 1), "r"(warps * 32) : "memory");
            for (int w = 0; w < warps; ++w) total += set[0][first_warp + w];
            return total;
        }
        if ((threadIdx.x & 31) < cluster) {            // lane l tells CTA l
            const uint32_t local = static_cast<uint32_t>(__cvta_generic_to_shared(&set[rank][warp]));
            uint32_t remote;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(threadIdx.x & 31));
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote), "f"(v) : "memory");
        }
        cluster_barrier();
        for (int c = 0; c < cluster; ++c)
            for (int w = 0; w < warps; ++w) total += set[c][w];
        return total;
    }
};

__device__ __forceinline__ void load_gamma(float *g, const float *gamma, int c, int count, int C) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < count) g[e] = c + e < C ? gamma[c + e] : 0.f;
}
template <int A, int E> __device__ __forceinline__ void load_gamma(float (&g)[E], const float *gamma, int c0, int C) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < E / A; ++j) load_gamma(g + j * A, gamma, c0 + (32 * j + lane) * A, A, C);
}

// MX: the output is 8-bit blocks.
template <typename T, int A, int E, bool MX>
__global__ void __launch_bounds__(kMostWarps * 32) rms_norm_kernel(RmsArgs a) {
    __shared__ float slots[2][8][kMostWarps];
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int groups = static_cast<int>(blockDim.x >> 5) / a.warps, group = warp / a.warps;      // rows at a time
    const uint32_t rank = a.cluster > 1 ? rank_in_cluster() : 0;
    const int c0 = (static_cast<int>(rank) * a.warps + warp % a.warps) * 32 * E, left = a.C - c0;
    RowSum row_sum{slots, a.warps, a.cluster, group, group * a.warps, rank, 0};
    const int64_t step = static_cast<int64_t>(gridDim.x / a.cluster) * groups;
    int64_t row = static_cast<int64_t>(blockIdx.x / a.cluster) * groups + group;
    if (a.cluster > 1) cluster_barrier();              // the peers run: their slots can be written
    pdl_wait();
    const T *x = static_cast<const T *>(a.x) + c0, *res = static_cast<const T *>(a.residual) + c0;
    Strip<T, A, E> in, add;
    if (row < a.rows) {
        in.load(x + row * a.x_row, left);
        if (a.residual) add.load(res + row * a.r_row, left);
    }
    float gamma[E];
    load_gamma<A, E>(gamma, a.gamma, c0, a.C);
    const float columns = static_cast<float>(a.C);
    for (; row < a.rows; row += step) {                // (the same for the warps of a row, and for a cluster)
        float v[E];
        in.widen_to(v);
        if (a.residual) {
            float r[E];
            add.widen_to(r);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += r[e];
        }
        if (a.sum) {
            Strip<T, A, E> out;
            out.narrow_from(v);
            out.store(static_cast<T *>(a.sum) + row * a.r_row + c0, left);
        }
        if (row + step < a.rows) {
            in.load(x + (row + step) * a.x_row, left);
            if (a.residual) add.load(res + (row + step) * a.r_row, left);
        }
        float squares = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) squares = fmaf(v[e], v[e], squares);
        float total = row_sum(squares), eps = a.eps, scale = 1.f;
        if (!(total <= 1e38f) || (total < 1e-27f && a.eps < 1e-18f)) { // squares beyond fp32's range: the row times a power of two, and eps its square
            scale = total < 1.f ? 0x1p80f : 0x1p-80f;
            eps = eps * scale * scale;
            squares = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[e] *= scale;
                squares = fmaf(v[e], v[e], squares);
            }
            total = row_sum(squares);
        }
        const float rstd = __frcp_rn(__fsqrt_rn(__fdiv_rn(total, columns) + eps));
        if (a.rstd && c0 == 0 && lane == 0) a.rstd[row] = rstd * scale;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = __fmul_rn(__fmul_rn(v[e], rstd), gamma[e]);
        if constexpr (MX) {
            const int64_t rt = row >> 7;
            store_blocks<A, E>(a.mx + rt * a.col_tiles * kMx8Tile, a.mx + a.scales_at + rt * a.groups * kMx8Scales, static_cast<int>(row & 127), c0,
                               static_cast<int64_t>(a.col_tiles) * 128, v);
        } else {
            Strip<T, A, E> out;
            out.narrow_from(v);
            out.store(static_cast<T *>(a.y) + row * a.y_row + c0, left);
        }
    }
    // a CTA's slots are written by its peers: it may not end before they have
    if (a.cluster > 1) cluster_barrier();
}

// x: s; y: dx (strides x_row); residual: dy (y_row); dsum (r_row); ws: partial sums of dgamma, [CTA][C], clusters counting as one CTA
template <typename T, int A, int E>
__global__ void __launch_bounds__(kMostWarps * 32) rms_grad_kernel(RmsArgs a) {
    __shared__ float slots[2][8][kMostWarps];
    extern __shared__ float columns_of[];              // sums of dgamma of the CTA's columns, where it takes several rows at a time
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int groups = static_cast<int>(blockDim.x >> 5) / a.warps, group = warp / a.warps;
    const uint32_t rank = a.cluster > 1 ? rank_in_cluster() : 0;
    const int c0 = (static_cast<int>(rank) * a.warps + warp % a.warps) * 32 * E, left = a.C - c0;
    RowSum row_sum{slots, a.warps, a.cluster, group, group * a.warps, rank, 0};
    const int64_t step = static_cast<int64_t>(gridDim.x / a.cluster) * groups;
    int64_t row = static_cast<int64_t>(blockIdx.x / a.cluster) * groups + group;
    if (a.cluster > 1) cluster_barrier();              // the peers run: their slots can be written
    pdl_wait();
    const T *s = static_cast<const T *>(a.x) + c0, *dy = static_cast<const T *>(a.residual) + c0, *ds = static_cast<const T *>(a.dsum) + c0;
    Strip<T, A, E> in, grad, add;
    float rstd = 0.f;
    auto load = [&](int64_t at) {
        in.load(s + at * a.r_row, left);
        grad.load(dy + at * a.y_row, left);
        if (a.dsum) add.load(ds + at * a.r_row, left);
        rstd = a.rstd[at];
    };
    if (row < a.rows) load(row);
    float gamma[E], dgamma[E];
    load_gamma<A, E>(gamma, a.gamma, c0, a.C);
#pragma unroll
    for (int e = 0; e < E; ++e) dgamma[e] = 0.f;
    const float columns = static_cast<float>(a.C);
    for (; row < a.rows; row += step) {
        float xh[E], u[E], r[E];
        const float scale = rstd;
        in.widen_to(xh);
        grad.widen_to(u);
        if (a.dsum) add.widen_to(r);
        if (row + step < a.rows) load(row + step);
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            xh[e] *= scale;
            dgamma[e] = fmaf(u[e], xh[e], dgamma[e]);
            u[e] *= gamma[e];
            dot = fmaf(u[e], xh[e], dot);
        }
        const float mean = __fdiv_rn(row_sum(dot), columns);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float t = fmaf(-xh[e], mean, u[e]);
            u[e] = a.dsum ? fmaf(scale, t, r[e]) : scale * t;
        }
        Strip<T, A, E> out;
        out.narrow_from(u);
        out.store(static_cast<T *>(a.y) + row * a.x_row + c0, left);
    }
    // the CTA's part of dgamma, groups added in order
    float *part = a.ws + static_cast<int64_t>(blockIdx.x / a.cluster) * a.C;
    const int first = c0 - static_cast<int>(rank) * a.warps * 32 * E;  // column of the CTA
    for (int g = 0; g < groups; ++g) {
        if (g == group) {
#pragma unroll
            for (int j = 0; j < E / A; ++j)
#pragma unroll
                for (int e = 0; e < A; ++e) {
                    const int at = (32 * j + lane) * A + e;
                    float v = dgamma[j * A + e];
                    if (g > 0) v += columns_of[first + at];
                    if (g + 1 < groups) columns_of[first + at] = v;
                    else if (at < left) part[c0 + at] = v;
                }
        }
        if (groups > 1) __syncthreads();
    }
    if (a.cluster > 1) cluster_barrier();
}

// dgamma = the partial sums of 32 columns per CTA, added in a fixed order: warp w takes parts w, w + 16, ...
__global__ void __launch_bounds__(512) rms_join_kernel(const float *ws, int parts, int C, float *dgamma) {
    __shared__ float of_warp[16][32];
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane;
    pdl_wait();
    float v = 0.f;
    if (c < C) {
#pragma unroll 8
        for (int p = warp; p < parts; p += 16) v += ws[static_cast<int64_t>(p) * C + c];
    }
    of_warp[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < C) {
        v = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) v += of_warp[w][lane];
        dgamma[c] = v;
    }
}

struct RmsPlan {
    int E, warps, cluster, threads, grid;              // grid: CTAs
};
// Warps of a row: a power of two that covers it with E columns per lane.
RmsPlan plan_of(int C, int64_t rows, int E, int per_sm) {
    RmsPlan p{};
    p.E = E;
    p.cluster = 1;
    p.warps = 1;
    while (p.warps < kMostWarps && p.warps * 32 * E < C) p.warps *= 2;
    while (p.cluster * p.warps * 32 * E < C) p.cluster *= 2;
    p.threads = std::max(p.warps, 8) * 32;
    const int groups = p.threads / 32 / p.warps;
    const int64_t ctas = ceil_div(rows, groups), most = static_cast<int64_t>(sm_count()) * per_sm * 256 / p.threads / p.cluster;
    p.grid = static_cast<int>(std::min(ctas, std::max<int64_t>(1, most))) * p.cluster;
    return p;
}
// Few rows are spread over as many warps as can be; many take more columns per lane, so that more bytes are in flight.
RmsPlan plan_forward(int C, int64_t rows) {
    if (C <= 256 || (C <= kMostWarps * 256 && rows <= sm_count())) return plan_of(C, rows, 8, 4);
    return plan_of(C, rows, 16, 4);
}
RmsPlan plan_backward(int C, int64_t rows) {
    if (C <= kMostWarps * 256) return plan_of(C, rows, 8, 4);
    return plan_of(C, rows, 16, 2);
}

template <typename F> cudaError_t by_columns(int E, F f) {
    if (E == 8) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

}  // namespace

cudaError_t launch_rms_norm(const RmsShape &s, const RmsCall &c, cudaStream_t st) {
    RmsArgs a{};
    a.x = c.x; a.residual = c.residual; a.gamma = c.gamma; a.sum = c.sum; a.y = c.y; a.mx = static_cast<uint8_t *>(c.mx); a.rstd = c.rstd;
    a.rows = c.rows; a.x_row = s.x_row; a.r_row = s.r_row; a.y_row = s.y_row; a.C = s.C; a.eps = s.eps;
    const Mx8Shape m = mx8_shape(c.rows, s.C);
    a.scales_at = m.scales_at; a.col_tiles = static_cast<int>(m.col_tiles); a.groups = static_cast<int>(m.groups);
    const RmsPlan p = plan_forward(s.C, c.rows);
    a.warps = p.warps; a.cluster = p.cluster;
    const int width = strip_width(s.dtype, {c.x, c.residual, c.sum, c.y}, {s.x_row, c.residual || c.sum ? s.r_row : 0, c.y ? s.y_row : 0});
    return by_strip(s.dtype, width, [&](auto t, auto v) {
        return by_columns(p.E, [&](auto e) {
            const auto kernel = c.mx ? rms_norm_kernel<decltype(t), v.value, e.value, true> : rms_norm_kernel<decltype(t), v.value, e.value, false>;
            return launch_pdl(kernel, dim3(p.grid), dim3(p.threads), 0, st, p.cluster, a);
        });
    });
}

size_t rms_workspace_floats(const RmsShape &s) {
    const RmsPlan p = plan_backward(s.C, INT32_MAX);
    return static_cast<size_t>(p.grid / p.cluster) * s.C;
}

cudaError_t launch_rms_grad(const RmsShape &s, const RmsGradCall &c, cudaStream_t st, int *launches) {
    RmsArgs a{};
    a.x = c.s; a.residual = c.dy; a.dsum = c.dsum; a.gamma = c.gamma; a.y = c.dx; a.rstd = const_cast<float *>(c.rstd); a.ws = c.ws;
    a.rows = c.rows; a.x_row = s.x_row; a.r_row = s.r_row; a.y_row = s.y_row; a.C = s.C;
    const RmsPlan p = plan_backward(s.C, c.rows);
    a.warps = p.warps; a.cluster = p.cluster;
    const int groups = p.threads / 32 / p.warps, smem = groups > 1 ? p.warps * 32 * p.E * 4 : 0;
    const int width = strip_width(s.dtype, {c.s, c.dy, c.dsum, c.dx}, {s.x_row, s.r_row, s.y_row});
    *launches = 2;
    const cudaError_t e = by_strip(s.dtype, width, [&](auto t, auto v) {
        return by_columns(p.E, [&](auto n) {
            return launch_pdl(rms_grad_kernel<decltype(t), v.value, n.value>, dim3(p.grid), dim3(p.threads), smem, st, p.cluster, a);
        });
    });
    if (e != cudaSuccess) return e;
    return launch_pdl(rms_join_kernel, dim3(static_cast<unsigned>(ceil_div(s.C, 32))), dim3(512), 0, st, 1, c.ws, p.grid / p.cluster, s.C, c.dgamma);
}

}  // namespace patdnn

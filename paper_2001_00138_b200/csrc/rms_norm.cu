// RMS norm of rows with the residual's addition in front, written in the rows' type or as 8-bit blocks, and its gradient.
//
//   s = x + residual, rstd = 1 / sqrt(mean(s^2) + eps), y = (s rstd) gamma
//   gradient, with xh = s rstd and u = dy gamma: dx = rstd (u - xh mean(u xh)) + dsum, dgamma = sum over rows of dy xh
//
// s is formed in fp32 and stays there for the statistics and for y; only the stored sum is rounded.  Memory bound: one pass, a row lives in
// the registers of 1 to 16 warps (32 E columns each), of up to eight CTAs of a cluster for very long rows, of a part of a warp for very
// short ones.  The warps of a row walk over rows: gamma (and the gradient's dgamma) stay in registers, and the next row's loads are issued before the present row's sums are joined.
#include "feed_forward.hpp"

#include <algorithm>

#include "kernels.hpp"
#include "mx8_device.cuh"
#include "umma_ptx.cuh"

namespace patdnn {
namespace {

constexpr int kMostWarps = 16;
constexpr int kGradSmem = 225 * 1024;                  // dynamic shared memory of a CTA of the gradient, at most

struct RmsArgs {
    const void *x, *residual, *dsum;
    const float *gamma;
    void *sum, *y;
    uint8_t *mx;
    float *rstd, *ws;
    int64_t rows, x_row, r_row, y_row, scales_at;
    int C, warps, cluster, col_tiles, groups;          // warps: of a row, per CTA
    float eps;
    int *status;                                       // clusters: of a wait that ran out
    uint32_t spin_limit;
    int test_skip;
};

template <int L> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int s = L / 2; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
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
// behind the barrier of the call between.  A lane reads one slot (of a cluster four), and five shuffles add them: reading them one by one takes
// as long as a row's loads.
// In a cluster the values are sent with stores that count their bytes on a barrier of the CTA that gets them: a cluster barrier would wait for the rows
// that were stored before it as well (3000 x 16384 bf16: 103 us, so 71; its gradient 103 and 76).  A peer sends its next but one value only behind this CTA's next ones, which
// its warps send when they have read the present ones.
struct alignas(128) RowSlots {                         // what lies behind begins at a multiple of 128 too, as copies of whole lines want it
    float set[2][8][kMostWarps];                       // [2][row group, or CTA of the cluster][warp of the row]; zeros where there is none
    unsigned long long sent[2];                        // barriers
};
// A lane whose wait runs out gives up, and reports it at the end: it waits for nothing and sends nothing any more, so that sums that lack its values are never complete,
// and adds a NaN, so that this row and all later ones of its warp are NaN, never a wrong number.
constexpr int kRowSumCode = 151;                       // status word
template <int L> struct RowSum {
    RowSlots &slots;
    const RmsArgs &a;
    int warps, cluster, row_group;
    uint32_t rank;
    int calls;
    uint32_t there;                                    // 0: this lane has given up
    __device__ __forceinline__ void clear() {
        if (L < 32 || (warps == 1 && cluster == 1)) return;
        float *all = &slots.set[0][0][0];
        for (int i = threadIdx.x; i < 2 * 8 * kMostWarps; i += blockDim.x) all[i] = 0.f;
        if (cluster > 1 && threadIdx.x == 0) {
            for (unsigned long long &b : slots.sent)
                asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(&b))) : "memory");
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
        if (cluster > 1) cluster_barrier();            // the peers run, and their slots can be written
    }
    __device__ __forceinline__ float operator()(float v) {
        v = lanes_sum<L>(v);
        if (L < 32 || (warps == 1 && cluster == 1)) return v;
        const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) % warps;
        float(&set)[8][kMostWarps] = slots.set[calls & 1];
        const uint32_t bar = static_cast<uint32_t>(__cvta_generic_to_shared(&slots.sent[calls & 1])), parity = calls >> 1 & 1;
        ++calls;
        if (cluster == 1) {
            if (lane == 0) set[row_group][warp] = v;
            asm volatile("bar.sync %0, %1;" ::"r"(row_group + 1), "r"(warps * 32) : "memory");
            v = set[row_group][lane & (kMostWarps - 1)];
            return lanes_sum<kMostWarps>(v);
        }
        if (threadIdx.x == 0 && there)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((cluster * warps + (calls == a.test_skip && rank == 0)) * 4) : "memory");
        if (lane < cluster && there) {                 // lane l tells CTA l
            const uint32_t local = static_cast<uint32_t>(__cvta_generic_to_shared(&set[rank][warp]));
            uint32_t remote, remote_bar;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(lane));
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote_bar) : "r"(bar), "r"(lane));
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.u32 [%0], %1, [%2];" ::"r"(remote), "r"(__float_as_uint(v)), "r"(remote_bar) : "memory");
        }
        uint32_t polls = there ? a.spin_limit : 0;
        for (there = 0; polls > 0 && !there; --polls)
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                         : "=r"(there) : "r"(bar), "r"(parity) : "memory");
        __syncwarp();
        v = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) v += set[2 * k + (lane >> 4)][lane & (kMostWarps - 1)];
        return lanes_sum<32>(there ? v : __uint_as_float(0x7fffffffu));
    }
    // In front of a sum that only some rows take: a warp with a lane that has given up sends nothing at all, since its turns are not the others' any more.
    __device__ __forceinline__ void agree() {
        if (cluster > 1) there = __all_sync(0xffffffffu, there);
    }
    // A CTA's slots are written by its peers: it may not end before they have.  Where a wait ran out, what was sent may still be on its way when
    // everybody has stopped sending: a few hundred microseconds for it.
    __device__ __forceinline__ void finish() {
        if (cluster == 1) return;
        cluster_barrier();
        if (!there) {
            atomicCAS(a.status, 0, kRowSumCode);
            for (int i = 0; i < 200; ++i) __nanosleep(1000);
        }
    }
};

__device__ __forceinline__ void load_gamma(float *g, const float *gamma, int c, int count, int C) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < count) g[e] = c + e < C ? gamma[c + e] : 0.f;
}
template <int A, int E, int L> __device__ __forceinline__ void load_gamma(float (&g)[E], const float *gamma, int c0, int C) {
    const int lane = threadIdx.x & (L - 1);
#pragma unroll
    for (int j = 0; j < E / A; ++j) load_gamma(g + j * A, gamma, c0 + (L * j + lane) * A, A, C);
}

// MX: the output is 8-bit blocks.  L: lanes of a row; 32, or 16 or 8 where they take all of it.
template <typename T, int A, int E, int L, bool MX>
__global__ void __launch_bounds__(kMostWarps * 32) rms_norm_kernel(RmsArgs a) {
    __shared__ RowSlots slots;
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & (L - 1);
    const int groups = L < 32 ? blockDim.x / L : (blockDim.x >> 5) / a.warps, group = L < 32 ? threadIdx.x / L : warp / a.warps;   // rows at a time
    const uint32_t rank = a.cluster > 1 ? rank_in_cluster() : 0;
    const int c0 = L < 32 ? 0 : (static_cast<int>(rank) * a.warps + warp % a.warps) * 32 * E, left = a.C - c0;
    RowSum<L> row_sum{slots, a, a.warps, a.cluster, group, rank, 0, 1};
    row_sum.clear();
    const int64_t step = static_cast<int64_t>(gridDim.x / a.cluster) * groups;
    int64_t row = static_cast<int64_t>(blockIdx.x / a.cluster) * groups + group;
    pdl_wait();
    const T *x = static_cast<const T *>(a.x) + c0, *res = static_cast<const T *>(a.residual) + c0;
    Strip<T, A, E, L> in, add;
    if (row < a.rows) {
        in.load(x + row * a.x_row, left);
        if (a.residual) add.load(res + row * a.r_row, left);
    }
    float gamma[E];
    load_gamma<A, E, L>(gamma, a.gamma, c0, a.C);
    const float columns = static_cast<float>(a.C);
    // (the same turns for the warps of a row, and for a cluster; the rows that share a warp end together, the last ones without a row)
    const int64_t past = L < 32 ? group % (32 / L) : 0;
    for (; row - past < a.rows; row += step) {
        const bool on = L == 32 || row < a.rows;
        float v[E];
        in.widen_to(v);
        if (a.residual) {
            float r[E];
            add.widen_to(r);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] += r[e];
        }
        if (row + step < a.rows) {
            in.load(x + (row + step) * a.x_row, left);
            if (a.residual) add.load(res + (row + step) * a.r_row, left);
        }
        float squares = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) squares = fmaf(v[e], v[e], squares);
        float total = row_sum(squares), eps = a.eps, scale = 1.f;
        if (a.sum && on) {                             // (behind the sum: a cluster's barrier waits for stores before it)
            Strip<T, A, E, L> out;
            out.narrow_from(v);
            out.store(static_cast<T *>(a.sum) + row * a.r_row + c0, left);
        }
        const bool tiny = total < 1e-27f && a.eps < 1e-18f, beyond = tiny || !(total <= 1e38f) || a.eps > 1e38f;
        if (L < 32 ? __any_sync(0xffffffffu, beyond) : beyond) {       // squares beyond fp32's range: the row times a power of two, and eps its square
            row_sum.agree();
            if (beyond) scale = tiny ? 0x1p80f : total <= 1e38f ? 0.25f : 0x1p-80f;            // (0.25: it is eps that is large)
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
        if (a.rstd && on && c0 == 0 && lane == 0) a.rstd[row] = rstd * scale;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = __fmul_rn(__fmul_rn(v[e], rstd), gamma[e]);
        if constexpr (MX) {
            const int64_t rt = row >> 7;
            store_blocks<A, E, L>(a.mx + rt * a.col_tiles * kMx8Tile, a.mx + a.scales_at + rt * a.groups * kMx8Scales, static_cast<int>(row & 127), c0,
                                  on ? static_cast<int64_t>(a.col_tiles) * 128 : 0, v);
        } else {
            Strip<T, A, E, L> out;
            out.narrow_from(v);
            out.store(static_cast<T *>(a.y) + row * a.y_row + c0, on ? left : 0);
        }
    }
    row_sum.finish();
}

// x: s; y: dx (strides x_row); residual: dy (y_row); dsum (r_row); ws: partial sums of dgamma, [CTA][C], clusters counting as one CTA
// ASYNC, for many rows: every thread copies what it will read itself into its own slots of shared memory, kStages - 1 rows ahead (cp.async; rows of
// single 16-bit elements, which it cannot copy, come through registers).  Nothing may spill: with that much shared memory the L1 is too small
// for local memory.  A row's instructions count too: 16 columns to a lane where registers allow.
template <typename T, int A, int E, bool ASYNC>
struct RmsCopies {
    static constexpr int kUnit = A * sizeof(T), kStages = E == 16 ? (sizeof(T) == 4 ? 2 : 3) : (sizeof(T) == 4 ? 3 : 4);
    static constexpr bool kAsync = ASYNC && kUnit >= 4, kGammaShared = !(E == 16 && sizeof(T) == 4);
    static constexpr int kThreadBytes = kAsync ? 3 * E * static_cast<int>(sizeof(T)) * kStages : 0;
};
__host__ __device__ constexpr int grad_warps(int E) { return E == 8 ? 24 : 16; }       // of a CTA, at most
template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t dst, const void *src, int there) {    // `there` bytes, zeros behind them
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(there) : "memory");
}

template <typename T, int A, int E, int L, bool ASYNC>
__global__ void __launch_bounds__((ASYNC ? grad_warps(E) : kMostWarps) * 32) rms_grad_kernel(RmsArgs a) {
    using Copies = RmsCopies<T, A, E, ASYNC>;
    constexpr int S = Copies::kStages, NA = E / A, UNIT = Copies::kUnit;
    __shared__ RowSlots slots;
    extern __shared__ __align__(16) unsigned char smem[];              // gamma and the copies; at the end dgamma of every set of warps
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & (L - 1);
    const int groups = L < 32 ? blockDim.x / L : (blockDim.x >> 5) / a.warps, group = L < 32 ? threadIdx.x / L : warp / a.warps;
    const uint32_t rank = a.cluster > 1 ? rank_in_cluster() : 0;
    const int first = L < 32 ? 0 : static_cast<int>(rank) * a.warps * 32 * E;          // column of the CTA
    const int c0 = first + (L < 32 ? 0 : warp % a.warps * 32 * E), left = a.C - c0;
    const int covered = L < 32 ? L * E : a.warps * 32 * E;
    RowSum<L> row_sum{slots, a, a.warps, a.cluster, group, rank, 0, 1};
    row_sum.clear();
    const int64_t step = static_cast<int64_t>(gridDim.x / a.cluster) * groups;
    int64_t row = static_cast<int64_t>(blockIdx.x / a.cluster) * groups + group;
    pdl_wait();
    // rows of this thread, and where the next one to be fetched lies; a row's instructions bound narrow strips, so addresses are added up
    const int64_t behind = a.rows - row;
    int turns = behind > 0 ? static_cast<int>((behind + step - 1) / step) : 0, ahead = turns;
    const int64_t r_step = step * a.r_row, y_step = step * a.y_row, x_step = step * a.x_row;
    const T *s = static_cast<const T *>(a.x) + row * a.r_row + c0, *dy = static_cast<const T *>(a.residual) + row * a.y_row + c0;
    const T *ds = static_cast<const T *>(a.dsum) + row * a.r_row + c0;
    T *dx = static_cast<T *>(a.y) + row * a.x_row + c0;
    const float *rstds = a.rstd + row;
    const bool extra = a.dsum != nullptr, whole = left >= L * E;       // whole: every access of the strip is there
    float *gamma_shared = reinterpret_cast<float *>(smem);
    // the thread's slots: [stage][tensor][access][thread], so that a warp's lie side by side
    const uint32_t next = blockDim.x * UNIT, one = 3 * NA * next;
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(smem)) + (Copies::kGammaShared ? covered * 4 : 0) + threadIdx.x * UNIT;
    uint32_t to = mine;                                // the stage to be filled
    Strip<T, A, E, L> in, grad, add;
    auto copies = [&](const T *from, uint32_t at) {
        if (whole) {
#pragma unroll
            for (int j = 0; j < NA; ++j) copy_async<UNIT>(at + j * next, from + (L * j + lane) * A, UNIT);
        } else {
#pragma unroll
            for (int j = 0; j < NA; ++j) {
                const int c = (L * j + lane) * A, there = max(0, min(A, left - c)) * static_cast<int>(sizeof(T));
                copy_async<UNIT>(at + j * next, there ? from + c : from, there);
            }
        }
    };
    auto fetch = [&]() {                               // the next row into the next stage, or nothing
        if constexpr (Copies::kAsync) {
            if (ahead > 0) {
                copies(s, to);
                copies(dy, to + NA * next);
                if (extra) copies(ds, to + 2 * NA * next);
                to = to == mine + (S - 1) * one ? mine : to + one;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        } else if (ahead > 0) {
            in.load(s, left);
            grad.load(dy, left);
            if (extra) add.load(ds, left);
        }
        --ahead;
        s += r_step;
        dy += y_step;
        ds += r_step;
    };
    float gamma[Copies::kGammaShared ? 1 : E], dgamma[E];
#pragma unroll
    for (int k = 0; k < (Copies::kAsync ? S - 1 : 1); ++k) fetch();
    float rstd = turns > 0 ? *rstds : 0.f;
    if constexpr (Copies::kGammaShared) {
        for (int c = threadIdx.x; c < covered; c += blockDim.x) gamma_shared[c] = first + c < a.C ? a.gamma[first + c] : 0.f;
        __syncthreads();
    } else {
        load_gamma<A, E, L>(gamma, a.gamma, c0, a.C);
    }
    const float *gamma_mine = gamma_shared + (c0 - first) + lane * A;
#pragma unroll
    for (int e = 0; e < E; ++e) dgamma[e] = 0.f;
    const float columns = 1.f / static_cast<float>(a.C);
    uint32_t from = mine;                              // the stage to be read
    int common = turns;                                // turns of the warp: rows that share it end together, the last ones without a row
    if constexpr (L < 32) common = __reduce_max_sync(0xffffffffu, turns);
    for (int turn = 0; turn < common; ++turn) {
        const bool on = L == 32 || turn < turns;
        float xh[E], u[E], r[E];
        const float scale = rstd;
        if constexpr (Copies::kAsync) {
            asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
#pragma unroll
            for (int j = 0; j < NA; ++j) in.v[j].load_shared(from + j * next);
#pragma unroll
            for (int j = 0; j < NA; ++j) grad.v[j].load_shared(from + (NA + j) * next);
            if (extra) {
#pragma unroll
                for (int j = 0; j < NA; ++j) add.v[j].load_shared(from + (2 * NA + j) * next);
            }
            from = from == mine + (S - 1) * one ? mine : from + one;
        }
        in.widen_to(xh);
        grad.widen_to(u);
        if (extra) add.widen_to(r);
        if (turn + 1 < turns) rstd = *(rstds += step);
        fetch();                                       // into the stage that was read a row ago
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < NA; ++j) {
            float g[A];
            if constexpr (!Copies::kGammaShared) {
#pragma unroll
                for (int e = 0; e < A; ++e) g[e] = gamma[j * A + e];
            } else {
                Pack<float, (A > 4 ? 4 : A)> t;
#pragma unroll
                for (int q = 0; q < A; q += 4) {
                    t.load(gamma_mine + j * L * A + q);
#pragma unroll
                    for (int e = 0; e < (A > 4 ? 4 : A); ++e) g[q + e] = __uint_as_float(t.w[e]);
                }
            }
#pragma unroll
            for (int e = 0; e < A; ++e) {
                const int k = j * A + e;
                xh[k] *= scale;
                if (on) dgamma[k] = fmaf(u[k], xh[k], dgamma[k]);
                u[k] *= g[e];
                dot = fmaf(u[k], xh[k], dot);
            }
        }
        const float mean = row_sum(dot) * columns;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float t = fmaf(-xh[e], mean, u[e]);
            u[e] = extra ? fmaf(scale, t, r[e]) : scale * t;
        }
        Strip<T, A, E, L> out;
        out.narrow_from(u);
        if (whole && on) {
#pragma unroll
            for (int j = 0; j < NA; ++j) out.v[j].store(dx + (L * j + lane) * A);
        } else {
            out.store(dx, on ? left : 0);
        }
        dx += x_step;
    }
    // the CTA's part of dgamma: rows that share a warp, then the sets of warps in order
    if constexpr (L < 32) {
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int k = L; k < 32; k *= 2) dgamma[e] += __shfl_xor_sync(0xffffffffu, dgamma[e], k);
    }
    if constexpr (Copies::kAsync) asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();                                   // nobody reads gamma or copies any more
    float *sums = reinterpret_cast<float *>(smem);
    const int sets = L < 32 ? blockDim.x >> 5 : groups, set = L < 32 ? warp : group;
#pragma unroll
    for (int j = 0; j < NA; ++j)
#pragma unroll
        for (int e = 0; e < A; ++e)
            if (L == 32 || (threadIdx.x & 31) < L) sums[set * covered + c0 - first + (L * j + lane) * A + e] = dgamma[j * A + e];
    __syncthreads();
    float *part = a.ws + static_cast<int64_t>(blockIdx.x / a.cluster) * a.C + first;
    for (int c = threadIdx.x; c < min(covered, a.C - first); c += blockDim.x) {
        float v = 0.f;
        for (int k = 0; k < sets; ++k) v += sums[k * covered + c];
        part[c] = v;
    }
    row_sum.finish();
}

// dgamma = the partial sums of 32 columns per CTA, added in a fixed order: warp w takes parts w, w + 32, ..., whose loads are all in flight
__global__ void __launch_bounds__(1024) rms_join_kernel(const float *ws, int parts, int C, float *dgamma) {
    __shared__ float of_warp[32][33];
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane;
    pdl_wait();
    float v = 0.f;
    if (c < C) {
        for (int p = warp; p < parts; p += 320) {
            float t[10];
#pragma unroll
            for (int k = 0; k < 10; ++k) t[k] = p + 32 * k < parts ? ws[static_cast<int64_t>(p + 32 * k) * C + c] : 0.f;
#pragma unroll
            for (int k = 0; k < 10; ++k) v += t[k];
        }
    }
    of_warp[warp][lane] = v;
    __syncthreads();
    v = lanes_sum<32>(of_warp[lane][warp]);            // warp w: column w
    const int column = blockIdx.x * 32 + warp;
    if (lane == 0 && column < C) dgamma[column] = v;
}

struct RmsPlan {
    int E, L, warps, cluster, threads, grid;           // grid: CTAs
    bool async;
};
// As many warps to a row as cover it with E columns per lane (as many as there are in clusters), as many rows to a CTA as make `warps` warps, and no
// more CTAs than are resident together, `ctas_per_sm` of such size.
RmsPlan plan_of(int C, int64_t rows, int E, int warps, int ctas_per_sm) {
    RmsPlan p{};
    p.E = E;
    p.L = E > 8 || C > 128 ? 32 : C > 64 ? 16 : 8;
    p.cluster = 1;
    p.warps = std::min<int>(kMostWarps, static_cast<int>(ceil_div(C, 32 * E)));
    while (p.cluster * p.warps * 32 * E < C) p.cluster *= 2;
    if (p.cluster > 1) p.warps = static_cast<int>(ceil_div(C, p.cluster * 32 * E));        // its CTAs take about as much of a row each
    p.threads = (p.cluster > 1 ? 1 : std::min(8, std::max(1, warps / p.warps))) * p.warps * 32;
    const int groups = p.L < 32 ? p.threads / p.L : p.threads / 32 / p.warps;
    const int64_t ctas = ceil_div(rows, groups), most = cluster_room(sm_count(), p.cluster) * std::max(1, ctas_per_sm * warps * 32 / p.threads) / p.cluster;
    p.grid = static_cast<int>(std::min(ctas, std::max<int64_t>(1, most))) * p.cluster;
    return p;
}
// Eight columns to a lane leave clearly fewer lanes without any than sixteen.
bool narrow(int C) { return 10 * ceil_div(C, 512) * 512 > 13 * ceil_div(C, 256) * 256; }
// Few rows are spread over as many warps as can be; many take more columns per lane, so that more bytes are in flight.
RmsPlan plan_forward(int C, int64_t rows) {
    if (C <= 256 || (C <= kMostWarps * 256 && (rows <= sm_count() || narrow(C)))) return plan_of(C, rows, 8, 8, 4);
    return plan_of(C, rows, 16, 8, 2);
}
RmsPlan plan_backward(int C, int64_t rows, int dtype) {
    const bool few = rows <= 2 * sm_count();           // a row or two per CTA: nothing to copy ahead
    const bool eight = C <= 256 || (C <= kMostWarps * 256 && (few || narrow(C) || dtype == PATDNN_F32)) || (dtype == PATDNN_F32 && C <= 8 * kMostWarps * 256);
    RmsPlan p = plan_of(C, rows, eight ? 8 : 16, few ? 8 : grad_warps(eight ? 8 : 16), 1);
    // Two rows of twelve warps, fp32: their copies and gamma do not fit (5000 x 2900: 16 columns to a lane 43 us, one row at a time 53).
    if (!few && eight && dtype == PATDNN_F32 && p.threads * RmsCopies<float, 4, 8, true>::kThreadBytes + p.warps * 256 * 4 > kGradSmem)
        p = plan_of(C, rows, 16, grad_warps(16), 1);
    p.async = !few;
    return p;
}

// f(E, L)
template <typename F> cudaError_t by_columns(const RmsPlan &p, F f) {
    using Eight = std::integral_constant<int, 8>;
    if (p.E == 16) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 32>{});
    if (p.L == 8) return f(Eight{}, Eight{});
    if (p.L == 16) return f(Eight{}, std::integral_constant<int, 16>{});
    return f(Eight{}, std::integral_constant<int, 32>{});
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
    a.status = c.wait.status; a.spin_limit = c.wait.spin_limit ? c.wait.spin_limit : kSpinLimit; a.test_skip = c.wait.test_skip;
    const int width = strip_width(s.dtype, {c.x, c.residual, c.sum, c.y}, {s.x_row, c.residual || c.sum ? s.r_row : 0, c.y ? s.y_row : 0});
    return by_strip(s.dtype, width, [&](auto t, auto v) {
        return by_columns(p, [&](auto e, auto l) {
            const auto kernel = c.mx ? rms_norm_kernel<decltype(t), v.value, e.value, l.value, true> : rms_norm_kernel<decltype(t), v.value, e.value, l.value, false>;
            return launch_pdl(kernel, dim3(p.grid), dim3(p.threads), 0, st, p.cluster, a);
        });
    });
}

cudaError_t prepare_rms() {
    for (int dtype : {PATDNN_F32, PATDNN_F16, PATDNN_BF16})
        for (int width : {dtype == PATDNN_F32 ? 4 : 8, 2, 1})
            for (int k = 0; k < 4; ++k) {
                RmsPlan p{};
                p.E = k == 3 ? 16 : 8;
                p.L = k == 0 ? 8 : k == 1 ? 16 : 32;
                const cudaError_t e = by_strip(dtype, width, [&](auto t, auto v) {
                    return by_columns(p, [&](auto n, auto l) {
                        const cudaError_t r = cudaFuncSetAttribute(rms_grad_kernel<decltype(t), v.value, n.value, l.value, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGradSmem);
                        return r == cudaSuccess ? cudaFuncSetAttribute(rms_grad_kernel<decltype(t), v.value, n.value, l.value, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, 100 * 1024) : r;
                    });
                });
                if (e != cudaSuccess) return e;
            }
    return cudaSuccess;
}

size_t rms_workspace_floats(const RmsShape &s) {
    size_t most = 0;                                   // parts of either form
    for (int64_t rows : {static_cast<int64_t>(2) * sm_count(), static_cast<int64_t>(INT32_MAX)}) {
        const RmsPlan p = plan_backward(s.C, rows, s.dtype);
        most = std::max(most, static_cast<size_t>(p.grid / p.cluster) * s.C);
    }
    return most;
}

cudaError_t launch_rms_grad(const RmsShape &s, const RmsGradCall &c, cudaStream_t st, int *launches) {
    RmsArgs a{};
    a.x = c.s; a.residual = c.dy; a.dsum = c.dsum; a.gamma = c.gamma; a.y = c.dx; a.rstd = const_cast<float *>(c.rstd); a.ws = c.ws;
    a.rows = c.rows; a.x_row = s.x_row; a.r_row = s.r_row; a.y_row = s.y_row; a.C = s.C;
    const RmsPlan p = plan_backward(s.C, c.rows, s.dtype);
    a.warps = p.warps; a.cluster = p.cluster;
    a.status = c.wait.status; a.spin_limit = c.wait.spin_limit ? c.wait.spin_limit : kSpinLimit; a.test_skip = c.wait.test_skip;
    const int width = strip_width(s.dtype, {c.s, c.dy, c.dsum, c.dx}, {s.x_row, s.r_row, s.y_row});
    const int parts = p.grid / p.cluster;              // (a part alone is dgamma itself)
    if (parts == 1) a.ws = c.dgamma;
    *launches = parts == 1 ? 1 : 2;
    const cudaError_t e = by_strip(s.dtype, width, [&](auto t, auto v) {
        return by_columns(p, [&](auto n, auto l) {
            using Copies = RmsCopies<decltype(t), v.value, n.value, true>;
            const int covered = l.value < 32 ? l.value * n.value : p.warps * 32 * n.value;
            const int sums = (l.value < 32 ? p.threads / 32 : p.threads / 32 / p.warps) * covered * 4;
            const int smem = std::max(sums, (Copies::kGammaShared ? covered * 4 : 0) + (p.async ? p.threads * Copies::kThreadBytes : 0));
            const auto kernel = p.async ? rms_grad_kernel<decltype(t), v.value, n.value, l.value, true> : rms_grad_kernel<decltype(t), v.value, n.value, l.value, false>;
            return launch_pdl(kernel, dim3(p.grid), dim3(p.threads), smem, st, p.cluster, a);
        });
    });
    if (e != cudaSuccess || parts == 1) return e;
    return launch_pdl(rms_join_kernel, dim3(static_cast<unsigned>(ceil_div(s.C, 32))), dim3(1024), 0, st, 1, c.ws, parts, s.C, c.dgamma);
}

}  // namespace patdnn

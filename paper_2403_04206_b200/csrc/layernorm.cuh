// Layer norm over the rows of all M workers' activations, forward and backward.
//
//   forward   mu = mean x, s = (mean (x - mu)^2 + eps)^-1/2, y = gamma (x - mu) s + beta
//   backward  h = (x - mu) s, g = dy gamma
//             dx = s (g - mean g - h mean(g h)),  dgamma = sum over rows dy h,  dbeta = sum over rows dy
//
// Both directions are bound by memory: 2 (forward) and 3 (backward) elements of traffic per element.  A
// row is read once and stays in registers, so the variance is the mean of the squared deviations from
// the finished mean (two passes over registers), not a difference of two large sums.
//
// Rows are handled by 8 lanes, a warp or a CTA, whichever holds the row in its registers; a warp alone holds
// up to 4096 16-bit elements (no barriers, and every lane has up to 256 bytes of loads in flight).  Longer
// rows are read again from L2 instead.
#pragma once
#include "replica_common.cuh"

namespace grawa {
namespace replica {

struct NormForwardArgs {
    In x, gamma, beta;
    Out y, mean, rstd;
    long long rows, x_stride, y_stride;
    int cols;
    float eps, inv_cols;
    int has_gamma, has_beta, has_stats;
};

struct NormBackwardArgs {
    In dy, x, gamma, mean, rstd;
    Out dx, dgamma, dbeta;
    float* partial;                        // [M][parts][2][cols] when parts > 1
    long long rows, x_stride, y_stride;
    int cols, parts;
    float inv_cols;
    int has_gamma, has_dx, has_dgamma, has_dbeta, accumulate;
};

constexpr int kNormThreads = 128;          // CTA of the kernels that give a row to some lanes of a warp
constexpr int kNormMaxBlock = 512;         // largest CTA of the kernels that give a row to a CTA
constexpr int kNormLongThreads = 512;      // CTA of the kernels for rows that do not fit in registers

// Sum over the LPR lanes of a row, or (LPR = 0) over the CTA.  `buf` alternates between calls: a CTA needs
// one barrier per call, because a slot is written again only two calls later.
template <int LPR>
__device__ __forceinline__ float row_sum(float v, int buf)
{
    if constexpr (LPR > 0) {
        return lanes_sum<LPR>(v);
    } else {
        __shared__ float part[2][kNormMaxBlock / 32];
        v = lanes_sum<32>(v);
        if ((threadIdx.x & 31) == 0) part[buf][threadIdx.x >> 5] = v;
        __syncthreads();
        float t = 0.0f;
        for (unsigned w = 0; w < blockDim.x / 32; ++w) t += part[buf][w];
        return t;
    }
}
template <int LPR>
__device__ __forceinline__ float2 row_sum(float2 v, int buf)
{
    if constexpr (LPR > 0) {
        return make_float2(lanes_sum<LPR>(v.x), lanes_sum<LPR>(v.y));
    } else {
        __shared__ float2 part[2][kNormMaxBlock / 32];
        v = make_float2(lanes_sum<32>(v.x), lanes_sum<32>(v.y));
        if ((threadIdx.x & 31) == 0) part[buf][threadIdx.x >> 5] = v;
        __syncthreads();
        float2 t = make_float2(0.0f, 0.0f);
        for (unsigned w = 0; w < blockDim.x / 32; ++w) { t.x += part[buf][w].x; t.y += part[buf][w].y; }
        return t;
    }
}

// 1 / sqrt(v): the fast estimate and one step of Newton's iteration.  (v = 0, a constant row with eps = 0, gives
// infinity like the plain expression.)
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = rsqrtf(v);
    return v > 0.0f && v < 1e30f ? r * fmaf(-0.5f * v * r, r, 1.5f) : r;
}

// LPR = 8 or 32: that many lanes hold a row, kNormThreads / LPR rows a CTA; LPR = 0: the CTA holds it.
// A thread holds NV words of VE elements.
template <typename T, int VE, int NV, int LPR>
__global__ void __launch_bounds__(LPR ? kNormThreads : kNormMaxBlock)
layernorm_forward_kernel(const __grid_constant__ NormForwardArgs a)
{
    using W = WordOf<T, VE>;
    const int m = blockIdx.y;
    const int lanes = LPR ? LPR : blockDim.x, lane = LPR ? threadIdx.x % (LPR ? LPR : 1) : threadIdx.x;
    const long long row = LPR ? static_cast<long long>(blockIdx.x) * (kNormThreads / (LPR ? LPR : 1)) + threadIdx.x / (LPR ? LPR : 1) : blockIdx.x;
    const bool live = row < a.rows;
    if (LPR == 32 && !live) return;                           // a whole warp
    const int words = live ? a.cols / VE : 0;                 // a group of 8 without a row keeps its warp company
    const W* x = reinterpret_cast<const W*>(static_cast<const T*>(a.x.p[m]) + (live ? row : 0) * a.x_stride);

    W xw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (lane + i * lanes < words) xw[i] = x[lane + i * lanes];
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (lane + i * lanes < words) add_elements<T, VE>(xw[i], sum);
    const float mean = row_sum<LPR>(sum[0] + sum[1], 0) * a.inv_cols;
    float square[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (lane + i * lanes >= words) continue;
        float f[VE];
        shifted<T, VE>(xw[i], -mean, f);
#pragma unroll
        for (int e = 0; e < VE; ++e) square[e % 2] = fmaf(f[e], f[e], square[e % 2]);
    }
    const float rstd = inverse_root(fmaf(row_sum<LPR>(square[0] + square[1], 1), a.inv_cols, a.eps));
    if (!live) return;
    if (a.has_stats && lane == 0) {
        static_cast<float*>(a.mean.p[m])[row] = mean;
        static_cast<float*>(a.rstd.p[m])[row] = rstd;
    }
    const W* gamma = static_cast<const W*>(a.gamma.p[m]);
    const W* beta = static_cast<const W*>(a.beta.p[m]);
    const T* gamma1 = static_cast<const T*>(a.gamma.p[m]);
    const T* beta1 = static_cast<const T*>(a.beta.p[m]);
    const bool words_ok = a.has_gamma && a.has_beta && ((reinterpret_cast<uintptr_t>(gamma) | reinterpret_cast<uintptr_t>(beta)) % sizeof(W)) == 0;
    W* y = reinterpret_cast<W*>(static_cast<T*>(a.y.p[m]) + row * a.y_stride);
    if (words_ok) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = lane + i * lanes;
            if (at >= words) continue;
            float f[VE], g[VE], b[VE];
            unpack<T, VE>(gamma[at], g);
            unpack<T, VE>(beta[at], b);
            shifted<T, VE>(xw[i], -mean, f);
#pragma unroll
            for (int e = 0; e < VE; ++e) f[e] = fmaf(f[e] * rstd, g[e], b[e]);
            y[at] = pack<T, VE>(f);
        }
    } else {                                                  // parameters inside a flat vector stand anywhere, or there are none
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = lane + i * lanes;
            if (at >= words) continue;
            float f[VE];
            shifted<T, VE>(xw[i], -mean, f);
#pragma unroll
            for (int e = 0; e < VE; ++e)
                f[e] = fmaf(f[e] * rstd, a.has_gamma ? widen(gamma1[at * VE + e]) : 1.0f, a.has_beta ? widen(beta1[at * VE + e]) : 0.0f);
            y[at] = pack<T, VE>(f);
        }
    }
}

// Rows longer than a CTA's registers: a CTA per row, three reads of it (the second and third from L2).
template <typename T, int VE>
__global__ void __launch_bounds__(kNormLongThreads)
layernorm_forward_long_kernel(const __grid_constant__ NormForwardArgs a)
{
    using W = WordOf<T, VE>;
    const int m = blockIdx.y, words = a.cols / VE;
    const long long row = blockIdx.x;
    const W* x = reinterpret_cast<const W*>(static_cast<const T*>(a.x.p[m]) + row * a.x_stride);
    const T* gamma = static_cast<const T*>(a.gamma.p[m]);
    const T* beta = static_cast<const T*>(a.beta.p[m]);
    W* y = reinterpret_cast<W*>(static_cast<T*>(a.y.p[m]) + row * a.y_stride);
    float sum = 0.0f, f[VE];
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        unpack<T, VE>(x[at], f);
#pragma unroll
        for (int e = 0; e < VE; ++e) sum += f[e];
    }
    const float mean = row_sum<0>(sum, 0) * a.inv_cols;
    float squares = 0.0f;
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        unpack<T, VE>(x[at], f);
#pragma unroll
        for (int e = 0; e < VE; ++e) squares = fmaf(f[e] - mean, f[e] - mean, squares);
    }
    const float rstd = inverse_root(fmaf(row_sum<0>(squares, 1), a.inv_cols, a.eps));
    if (a.has_stats && threadIdx.x == 0) {
        static_cast<float*>(a.mean.p[m])[row] = mean;
        static_cast<float*>(a.rstd.p[m])[row] = rstd;
    }
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        unpack<T, VE>(x[at], f);
#pragma unroll
        for (int e = 0; e < VE; ++e)
            f[e] = fmaf((f[e] - mean) * rstd, a.has_gamma ? widen(gamma[at * VE + e]) : 1.0f, a.has_beta ? widen(beta[at * VE + e]) : 0.0f);
        y[at] = pack<T, VE>(f);
    }
}

// One column's finished gradients: added to what the worker's gradient vector holds, or put in its place.
template <typename T>
__device__ __forceinline__ void store_gradients(const NormBackwardArgs& a, int m, int col, float dg, float db)
{
    if (a.has_dgamma) {
        T* d = static_cast<T*>(a.dgamma.p[m]) + col;
        *d = narrow<T>(a.accumulate ? widen(*d) + dg : dg);
    }
    if (a.has_dbeta) {
        T* d = static_cast<T*>(a.dbeta.p[m]) + col;
        *d = narrow<T>(a.accumulate ? widen(*d) + db : db);
    }
}

// A worker's column sums over the rows of one CTA: to the CTA's place in `partial`, or, when it is the
// worker's only CTA, to the gradients themselves.
template <typename T>
__device__ __forceinline__ void store_column(const NormBackwardArgs& a, int m, int part, int col, float dg, float db)
{
    if (a.parts == 1) {
        store_gradients<T>(a, m, col, dg, db);
    } else {
        float* p = a.partial + (static_cast<size_t>(m) * a.parts + part) * 2 * a.cols + col;
        p[0] = dg;
        p[a.cols] = db;
    }
}

// Rows under way: 16-byte words are staged through shared memory by asynchronous copies, kNormDepth rows ahead of
// the one that is computed (registers are full of column sums; one row ahead in registers left the SM waiting
// for memory), each thread its own words, so that no barrier is needed.
template <typename T, int VE, int EPT> struct NormStage {
    static constexpr bool staged = VE * sizeof(T) == 16;
    static constexpr int words = EPT / VE;
    static constexpr int depth = words <= 3 ? 4 : words <= 4 ? 3 : 2;
    static constexpr size_t bytes_a_thread = staged ? depth * 2 * words * 16 : 0;
};

// gridDim.x CTAs a worker go through its rows in turn; a thread keeps the sums of its own columns in
// registers over all of them, so the weights' gradients cost one small table at the end and no atomics
// (the split depends on the sizes alone: the same bits every time).
template <typename T, int VE, int EPT, int LPR>
__global__ void __launch_bounds__(LPR ? kNormThreads : kNormMaxBlock)
layernorm_backward_kernel(const __grid_constant__ NormBackwardArgs a)
{
    using Stage = NormStage<T, VE, EPT>;
    constexpr int NV = EPT / VE;
    constexpr int GROUPS = LPR ? kNormThreads / (LPR ? LPR : 1) : 1;
    using W = WordOf<T, VE>;
    extern __shared__ uint4 ring[];                           // [depth][x, dy][NV][threads]
    const int m = blockIdx.y;
    const int lanes = LPR ? LPR : blockDim.x, lane = LPR ? threadIdx.x % (LPR ? LPR : 1) : threadIdx.x;
    const int group = LPR ? threadIdx.x / (LPR ? LPR : 1) : 0;
    const int words = a.cols / VE;
    const T* gamma = static_cast<const T*>(a.gamma.p[m]);
    const T* xs = static_cast<const T*>(a.x.p[m]);
    const T* dys = static_cast<const T*>(a.dy.p[m]);
    const float* means = static_cast<const float*>(a.mean.p[m]);
    const float* rstds = static_cast<const float*>(a.rstd.p[m]);

    float gm[EPT], dg[EPT], db[EPT];
#pragma unroll
    for (int k = 0; k < EPT; ++k) {
        const int at = lane + k / VE * lanes;
        gm[k] = a.has_gamma && at < words ? widen(gamma[at * VE + k % VE]) : 1.0f;
        dg[k] = db[k] = 0.0f;
    }
    const long long stride = static_cast<long long>(gridDim.x) * GROUPS;
    long long row = static_cast<long long>(blockIdx.x) * GROUPS + group;
    const auto fetch = [&](int slot, long long r) {
        if (r < a.rows) {
            const W* x = reinterpret_cast<const W*>(xs + r * a.x_stride) + lane;
            const W* dy = reinterpret_cast<const W*>(dys + r * a.y_stride) + lane;
            uint4* to = ring + static_cast<size_t>(slot) * 2 * NV * blockDim.x + threadIdx.x;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (lane + i * lanes < words) {
                    copy_async16(to + i * blockDim.x, x + i * lanes);
                    copy_async16(to + (NV + i) * blockDim.x, dy + i * lanes);
                }
        }
        copy_async_commit();                                  // a group a row, also where there is none
    };
    if constexpr (Stage::staged) {
#pragma unroll
        for (int d = 0; d < Stage::depth - 1; ++d) fetch(d, row + d * stride);
    }
    int buf = 0, slot = 0;
    float mean = row < a.rows ? means[row] : 0.0f, rstd = row < a.rows ? rstds[row] : 0.0f;
    for (; row - group < a.rows; row += stride) {             // the same turns for all groups of the CTA
        const int w_end = row < a.rows ? words : 0;
        W xw[NV], dw[NV];
        if constexpr (Stage::staged) {
            fetch(slot == 0 ? Stage::depth - 1 : slot - 1, row + (Stage::depth - 1) * stride);
            copy_async_wait<Stage::depth - 1>();
            const uint4* from = ring + static_cast<size_t>(slot) * 2 * NV * blockDim.x + threadIdx.x;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (lane + i * lanes < w_end) { xw[i] = from[i * blockDim.x]; dw[i] = from[(NV + i) * blockDim.x]; }
            slot = slot + 1 == Stage::depth ? 0 : slot + 1;
        } else {
            const W* x = reinterpret_cast<const W*>(xs + row * a.x_stride) + lane;
            const W* dy = reinterpret_cast<const W*>(dys + row * a.y_stride) + lane;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (lane + i * lanes < w_end) { xw[i] = x[i * lanes]; dw[i] = dy[i * lanes]; }
        }
        const bool more = row + stride < a.rows;
        const float next_mean = more ? means[row + stride] : 0.0f, next_rstd = more ? rstds[row + stride] : 0.0f;
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (lane + i * lanes >= w_end) continue;
            float f[VE], d[VE];
            shifted<T, VE>(xw[i], -mean, f);
            unpack<T, VE>(dw[i], d);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float h = f[e] * rstd, g = d[e] * gm[i * VE + e];
                s.x += g;
                s.y = fmaf(g, h, s.y);
                dg[i * VE + e] = fmaf(d[e], h, dg[i * VE + e]);
                db[i * VE + e] += d[e];
            }
        }
        if (a.has_dx) {
            s = row_sum<LPR>(s, buf);
            buf ^= 1;
            const float mg = -s.x * a.inv_cols * rstd, mgh = -s.y * a.inv_cols * rstd * rstd;
            W* dx = reinterpret_cast<W*>(static_cast<T*>(a.dx.p[m]) + row * a.x_stride) + lane;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (lane + i * lanes >= w_end) continue;
                float f[VE], d[VE];
                shifted<T, VE>(xw[i], -mean, f);
                unpack<T, VE>(dw[i], d);
#pragma unroll
                for (int e = 0; e < VE; ++e) f[e] = fmaf(d[e] * gm[i * VE + e], rstd, fmaf(f[e], mgh, mg));
                dx[i * lanes] = pack<T, VE>(f);
            }
        }
        mean = next_mean;
        rstd = next_rstd;
    }
    if constexpr (Stage::staged) copy_async_wait<0>();
    if (!a.has_dgamma && !a.has_dbeta) return;
    if constexpr (LPR == 0) {
#pragma unroll
        for (int k = 0; k < EPT; ++k) {
            const int at = lane + k / VE * lanes;
            if (at < words) store_column<T>(a, m, blockIdx.x, at * VE + k % VE, dg[k], db[k]);
        }
    } else {
        // groups of rows: first the groups of a warp, then the warps in order, through shared memory
        __shared__ float2 acc[LPR * EPT];
#pragma unroll
        for (int k = 0; k < EPT; ++k)
#pragma unroll
            for (int d = LPR; d < 32; d <<= 1) {
                dg[k] += __shfl_xor_sync(0xffffffffu, dg[k], d);
                db[k] += __shfl_xor_sync(0xffffffffu, db[k], d);
            }
        const int warp = threadIdx.x >> 5;
        for (int turn = 0; turn < kNormThreads / 32; ++turn) {
            if (warp == turn && (threadIdx.x & 31) < LPR) {
#pragma unroll
                for (int k = 0; k < EPT; ++k) {
                    float2 v = make_float2(dg[k], db[k]);
                    if (turn) { v.x += acc[k * LPR + lane].x; v.y += acc[k * LPR + lane].y; }
                    acc[k * LPR + lane] = v;
                }
            }
            __syncthreads();
        }
        for (int j = threadIdx.x; j < LPR * EPT; j += kNormThreads) {
            const int at = j % LPR + j / LPR / VE * LPR, col = at * VE + j / LPR % VE;
            if (at < words) store_column<T>(a, m, blockIdx.x, col, acc[j].x, acc[j].y);
        }
    }
}

// Rows that do not fit in a CTA's registers: dx by a CTA per row (dy and x are read again from L2) ...
template <typename T, int VE>
__global__ void __launch_bounds__(kNormLongThreads)
layernorm_backward_long_kernel(const __grid_constant__ NormBackwardArgs a)
{
    using W = WordOf<T, VE>;
    const int m = blockIdx.y, words = a.cols / VE;
    const long long row = blockIdx.x;
    const W* x = reinterpret_cast<const W*>(static_cast<const T*>(a.x.p[m]) + row * a.x_stride);
    const W* dy = reinterpret_cast<const W*>(static_cast<const T*>(a.dy.p[m]) + row * a.y_stride);
    const T* gamma = static_cast<const T*>(a.gamma.p[m]);
    W* dx = reinterpret_cast<W*>(static_cast<T*>(a.dx.p[m]) + row * a.x_stride);
    const float mean = static_cast<const float*>(a.mean.p[m])[row], rstd = static_cast<const float*>(a.rstd.p[m])[row];
    float f[VE], d[VE];
    float2 s = make_float2(0.0f, 0.0f);
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        unpack<T, VE>(x[at], f);
        unpack<T, VE>(dy[at], d);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float g = d[e] * (a.has_gamma ? widen(gamma[at * VE + e]) : 1.0f);
            s.x += g;
            s.y = fmaf(g, (f[e] - mean) * rstd, s.y);
        }
    }
    s = row_sum<0>(s, 0);
    const float mg = s.x * a.inv_cols, mgh = s.y * a.inv_cols;
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        unpack<T, VE>(x[at], f);
        unpack<T, VE>(dy[at], d);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float g = d[e] * (a.has_gamma ? widen(gamma[at * VE + e]) : 1.0f);
            f[e] = (g - mg - (f[e] - mean) * rstd * mgh) * rstd;
        }
        dx[at] = pack<T, VE>(f);
    }
}

// ... and the weights' gradients by a thread per column, gridDim.z parts of the rows.
template <typename T>
__global__ void __launch_bounds__(kNormThreads)
layernorm_columns_kernel(const __grid_constant__ NormBackwardArgs a)
{
    const int m = blockIdx.y, col = blockIdx.x * kNormThreads + threadIdx.x, part = blockIdx.z;
    if (col >= a.cols) return;
    const T* x = static_cast<const T*>(a.x.p[m]) + col;
    const T* dy = static_cast<const T*>(a.dy.p[m]) + col;
    const float* means = static_cast<const float*>(a.mean.p[m]);
    const float* rstds = static_cast<const float*>(a.rstd.p[m]);
    float dg = 0.0f, db = 0.0f;
#pragma unroll 4
    for (long long row = part; row < a.rows; row += a.parts) {
        const float d = widen(dy[row * a.y_stride]);
        dg = fmaf(d, (widen(x[row * a.x_stride]) - means[row]) * rstds[row], dg);
        db += d;
    }
    store_column<T>(a, m, part, col, dg, db);
}

// The parts' column sums, added in a fixed order: 32 columns a CTA, kFinishGroups threads a column.
constexpr int kFinishGroups = 16;
template <typename T>
__global__ void __launch_bounds__(32 * kFinishGroups)
layernorm_finish_kernel(const __grid_constant__ NormBackwardArgs a)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    __shared__ float2 acc[kFinishGroups][32];
    const int m = blockIdx.y, lane = threadIdx.x & 31, group = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float2 s = make_float2(0.0f, 0.0f);
    if (col < a.cols) {
        const float* p = a.partial + static_cast<size_t>(m) * a.parts * 2 * a.cols + col;
#pragma unroll 4
        for (int i = group; i < a.parts; i += kFinishGroups) {
            s.x += p[static_cast<size_t>(i) * 2 * a.cols];
            s.y += p[static_cast<size_t>(i) * 2 * a.cols + a.cols];
        }
    }
    acc[group][lane] = s;
    __syncthreads();
    if (group != 0 || col >= a.cols) return;
#pragma unroll
    for (int g = 1; g < kFinishGroups; ++g) { s.x += acc[g][lane].x; s.y += acc[g][lane].y; }
    store_gradients<T>(a, m, col, s.x, s.y);
}

}  // namespace replica
}  // namespace grawa

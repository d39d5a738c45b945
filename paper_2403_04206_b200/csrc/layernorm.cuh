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
// rows are read again, from L2 as far as it still holds them (in the backward pass by two kernels, the second of which finds
// nothing left there).
//
// Measured (B200, 6.54 TB/s copy), in shares of the copy rate: forward of 4 x 8192 x 4096 bf16 98 us (84 %), 16-bit rows of
// 1024 to 12000 elements 75 to 87 %, of 256 69 %, of 768 67 to 85 % (27 to 35 us for 8 x 6184 rows from run to run), fp32 86 to
// 90 %; backward of 8 x 6304 x 768 bf16 47 us (75 %; 26 instructions an element when counted, one more since, held
// to 128 registers by the column sums, 23 % of the warps active, issue slots 68 % busy: no unit is full), 256 to 4096 columns 70 to 76 %,
// fp32 88 %.  Far from it: backward rows of 8192 (57 us, 61 %: a barrier a row, one CTA an SM) and, above what a CTA's registers
// hold, of 12000 (104 us for 34.9, x and dy read twice); 16-bit rows that do not start on 16 bytes, forward 64 us for 23.3 and
// backward 119 for 34.9 (8 x 4745 x 1001: two words read and shifted for every one, and no staging in the backward pass).
#pragma once
#include <cooperative_groups.h>

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
    float* partial;                        // [M][parts][2][slots] when parts > 1
    long long rows, x_stride, y_stride;
    int cols, parts;
    int slots, lanes, word;                // slot j of a part holds the column that slot_column(j) names
    int cluster;                           // the parts are the CTAs of one cluster, which adds them up itself
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

// How rows are read and written, by the alignment that all rows of a call share:
//   kWhole   whole 16-byte words at 16-byte boundaries.  With the streaming hint, as rows are used once (forward of
//            4 x 8192 x 4096 bf16: 95 us, 103 to 113 us without).
//   kUnits   units of 4 bytes (fp32 rows anywhere; 16-bit rows of even length at even addresses): a lane's four
//            units of a word are `lanes` units apart, so that a warp's accesses are contiguous.
//   kFull    kWhole where the row fills every word of every lane: no lane asks whether its word exists.
//   kHalves  16-bit rows anywhere: 16-byte words put together from aligned ones.  (Single 2-byte accesses took
//            1.8 to 2 times as long: 8 x 4745 rows of 1001 bf16, forward 117 us, here 65 us.)
enum RowMode { kWhole = 0, kUnits = 1, kHalves = 2, kFull = 3 };

template <typename T, int MODE>
struct Rows {
    static constexpr int VE = kWordElems<T>, EU = 4 / static_cast<int>(sizeof(T)), HALVES = sizeof(T) / 2;
    static constexpr bool whole = MODE == kWhole || MODE == kFull;

    // The column of element e of a lane's word i.
    static __device__ __forceinline__ int column(int i, int e, int lane, int lanes)
    {
        if constexpr (MODE == kUnits) return ((i * 4 + e / EU) * lanes + lane) * EU + e % EU;
        else return (i * lanes + lane) * VE + e;
    }
    static __device__ __forceinline__ bool any(int i, int lane, int lanes, int cols) { return MODE == kFull || column(i, 0, lane, lanes) < cols; }

    // Word i of a lane that has any() of it; behind the end of the row it holds zeros.
    static __device__ __forceinline__ uint4 load(const T* row, int i, int lane, int lanes, int cols)
    {
        if constexpr (whole) {
            return __ldcs(reinterpret_cast<const uint4*>(row) + i * lanes + lane);
        } else if constexpr (MODE == kUnits) {
            const unsigned* u = reinterpret_cast<const unsigned*>(row) + i * 4 * lanes + lane;
            const int units = cols / EU - i * 4 * lanes - lane;
            return make_uint4(u[0], lanes < units ? u[lanes] : 0u, 2 * lanes < units ? u[2 * lanes] : 0u, 3 * lanes < units ? u[3 * lanes] : 0u);
        } else {
            const int at = (i * lanes + lane) * VE;
            return load_halves(reinterpret_cast<const unsigned short*>(row + at), min(cols - at, VE) * HALVES);
        }
    }
    // Its counterpart; with kHalves all lanes of a warp call it, and `segment` neighbouring lanes hold neighbouring words.
    static __device__ __forceinline__ void store(T* row, int i, int lane, int lanes, int cols, const uint4& v, int segment)
    {
        if constexpr (whole) {
            if (any(i, lane, lanes, cols)) __stcs(reinterpret_cast<uint4*>(row) + i * lanes + lane, v);
        } else if constexpr (MODE == kUnits) {
            unsigned* u = reinterpret_cast<unsigned*>(row) + i * 4 * lanes + lane;
            const int units = cols / EU - i * 4 * lanes - lane;
            if (0 < units) u[0] = v.x;
            if (lanes < units) u[lanes] = v.y;
            if (2 * lanes < units) u[2 * lanes] = v.z;
            if (3 * lanes < units) u[3 * lanes] = v.w;
        } else {
            store_halves(reinterpret_cast<unsigned short*>(row), i * lanes + lane, lane % segment, segment, cols * HALVES, v, skip_of(row));
        }
    }
};

// Whole words, or single elements.
template <typename T, bool WHOLE>
__device__ __forceinline__ void read_elements(const T* row, int at, float* f)
{
    if constexpr (WHOLE) unpack<T>(reinterpret_cast<const uint4*>(row)[at], f);
    else f[0] = widen(row[at]);
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void write_elements(T* row, int at, const float* f)
{
    if constexpr (WHOLE) reinterpret_cast<uint4*>(row)[at] = pack<T>(f);
    else row[at] = narrow<T>(f[0]);
}

// LPR = 8 or 32: that many lanes hold a row, kNormThreads / LPR rows a CTA; LPR = 0: the CTA holds it.
// A thread holds NV words.
template <typename T, int NV, int LPR, int MODE>
__global__ void __launch_bounds__(LPR ? kNormThreads : kNormMaxBlock)
layernorm_forward_kernel(const __grid_constant__ NormForwardArgs a)
{
    stream_order();
    using R = Rows<T, MODE>;
    constexpr int VE = R::VE, LANES = LPR ? LPR : 32;
    const int m = blockIdx.y;
    const int lanes = LPR ? LPR : blockDim.x, lane = LPR ? threadIdx.x % LANES : threadIdx.x;
    const long long row = LPR ? static_cast<long long>(blockIdx.x) * (kNormThreads / LANES) + threadIdx.x / LANES : blockIdx.x;
    const bool live = row < a.rows;
    if (LPR == 32 && !live) return;                           // a whole warp
    const int cols = live ? a.cols : 0;                       // a group of 8 without a row keeps its warp company
    const T* x = static_cast<const T*>(a.x.p[m]) + (live ? row : 0) * a.x_stride;

    uint4 xw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (R::any(i, lane, lanes, cols)) xw[i] = R::load(x, i, lane, lanes, cols);
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (R::any(i, lane, lanes, cols)) add_elements<T>(xw[i], sum);
    const float mean = row_sum<LPR>(sum[0] + sum[1], 0) * a.inv_cols;
    float square[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (!R::any(i, lane, lanes, cols)) continue;
        float f[VE];
        shifted<T>(xw[i], -mean, f);
        if (!R::whole && R::column(i, VE - 1, lane, lanes) >= cols) {          // the row ends inside this word
#pragma unroll
            for (int e = 0; e < VE; ++e)
                if (R::column(i, e, lane, lanes) >= cols) f[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < VE; ++e) square[e % 2] = fmaf(f[e], f[e], square[e % 2]);
    }
    const float rstd = inverse_root(fmaf(row_sum<LPR>(square[0] + square[1], 1), a.inv_cols, a.eps));
    if (a.has_stats && lane == 0 && live) {
        static_cast<float*>(a.mean.p[m])[row] = mean;
        static_cast<float*>(a.rstd.p[m])[row] = rstd;
    }
    const T* gamma = static_cast<const T*>(a.gamma.p[m]);
    const T* beta = static_cast<const T*>(a.beta.p[m]);
    T* y = static_cast<T*>(a.y.p[m]) + (live ? row : 0) * a.y_stride;
    // parameters inside a flat vector stand anywhere, or there are none
    const bool by_words = R::whole && a.has_gamma && a.has_beta && skip_of(gamma) == 0 && skip_of(beta) == 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const bool here = R::any(i, lane, lanes, cols);
        if (MODE != kHalves && !here) continue;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (here) {
            float f[VE], g[VE], b[VE];
            if (by_words) {
                unpack<T>(reinterpret_cast<const uint4*>(gamma)[i * lanes + lane], g);
                unpack<T>(reinterpret_cast<const uint4*>(beta)[i * lanes + lane], b);
            } else if (MODE == kHalves && a.has_gamma && a.has_beta) {
                unpack<T>(R::load(gamma, i, lane, lanes, cols), g);
                unpack<T>(R::load(beta, i, lane, lanes, cols), b);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const int col = R::column(i, e, lane, lanes);
                    const bool in = R::whole || col < cols;
                    g[e] = a.has_gamma && in ? widen(gamma[col]) : 1.0f;
                    b[e] = a.has_beta && in ? widen(beta[col]) : 0.0f;
                }
            }
            shifted<T>(xw[i], -mean, f);
#pragma unroll
            for (int e = 0; e < VE; ++e) f[e] = fmaf(f[e] * rstd, g[e], b[e]);
            v = pack<T>(f);
        }
        R::store(y, i, lane, lanes, cols, v, LANES);
    }
}

// Short rows by the thousand, 16-byte aligned, a warp a row: a warp goes through rows with the next ones on their way
// to shared memory, each lane its own words (no barriers).  For rows of one or two words a lane, whose loads
// alone do not keep memory busy (8 x 18554 rows of 256 bf16: 48 us with a warp for every row, 32 us so); longer
// rows have loads enough in flight, and lose with the fewer warps that the stages leave room for.
constexpr int kAheadDepth = 4, kAheadCtas = 6;                // rows ahead, and CTAs an SM takes
template <typename T, int NV>
__global__ void __launch_bounds__(kNormThreads)
layernorm_forward_short_kernel(const __grid_constant__ NormForwardArgs a)
{
    stream_order();
    constexpr int VE = kWordElems<T>, kWarps = kNormThreads / 32;
    __shared__ uint4 ring[kAheadDepth][NV][kNormThreads];
    const int m = blockIdx.y, lane = threadIdx.x % 32, words = a.cols / VE;
    const T* xs = static_cast<const T*>(a.x.p[m]);
    const uint4* gamma = static_cast<const uint4*>(a.gamma.p[m]) + lane;            // aligned, and whole words, as the host has checked
    const uint4* beta = static_cast<const uint4*>(a.beta.p[m]) + lane;
    const int stride = gridDim.x * kWarps;
    const auto fetch = [&](int slot, long long row) {
        if (row < a.rows) {
            const uint4* x = reinterpret_cast<const uint4*>(xs + row * a.x_stride) + lane;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (lane + i * 32 < words) copy_async16(&ring[slot][i][threadIdx.x], x + i * 32);
        }
        copy_async_commit();                                  // a group a row, also where there is none
    };
    long long row = static_cast<long long>(blockIdx.x) * kWarps + threadIdx.x / 32;
#pragma unroll
    for (int d = 0; d < kAheadDepth - 1; ++d) fetch(d, row + static_cast<long long>(d) * stride);
    uint4 gw[NV], bw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (lane + i * 32 < words) { gw[i] = gamma[i * 32]; bw[i] = beta[i * 32]; }
    for (int slot = 0; row < a.rows; row += stride, slot = (slot + 1) % kAheadDepth) {
        fetch((slot + kAheadDepth - 1) % kAheadDepth, row + static_cast<long long>(kAheadDepth - 1) * stride);
        copy_async_wait<kAheadDepth - 1>();
        uint4 xw[NV];
        float sum[2] = {0.0f, 0.0f}, square[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (lane + i * 32 >= words) continue;
            xw[i] = ring[slot][i][threadIdx.x];
            add_elements<T>(xw[i], sum);
        }
        const float mean = lanes_sum<32>(sum[0] + sum[1]) * a.inv_cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (lane + i * 32 >= words) continue;
            float f[VE];
            shifted<T>(xw[i], -mean, f);
#pragma unroll
            for (int e = 0; e < VE; ++e) square[e % 2] = fmaf(f[e], f[e], square[e % 2]);
        }
        const float rstd = inverse_root(fmaf(lanes_sum<32>(square[0] + square[1]), a.inv_cols, a.eps));
        if (a.has_stats && lane == 0) {
            static_cast<float*>(a.mean.p[m])[row] = mean;
            static_cast<float*>(a.rstd.p[m])[row] = rstd;
        }
        uint4* y = reinterpret_cast<uint4*>(static_cast<T*>(a.y.p[m]) + row * a.y_stride) + lane;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (lane + i * 32 >= words) continue;
            float f[VE], g[VE], b[VE];
            unpack<T>(gw[i], g);
            unpack<T>(bw[i], b);
            shifted<T>(xw[i], -mean, f);
#pragma unroll
            for (int e = 0; e < VE; ++e) f[e] = fmaf(f[e] * rstd, g[e], b[e]);
            __stcs(y + i * 32, pack<T>(f));
        }
    }
    copy_async_wait<0>();
}

// Rows longer than a CTA's registers: a CTA per row, three reads of it (the second and third from L2), by words, or
// element by element (neighbouring threads at neighbouring elements).
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kNormLongThreads)
layernorm_forward_long_kernel(const __grid_constant__ NormForwardArgs a)
{
    stream_order();
    constexpr int VE = WHOLE ? kWordElems<T> : 1;
    const int m = blockIdx.y, words = a.cols / VE;
    const long long row = blockIdx.x;
    const T* x = static_cast<const T*>(a.x.p[m]) + row * a.x_stride;
    const T* gamma = static_cast<const T*>(a.gamma.p[m]);
    const T* beta = static_cast<const T*>(a.beta.p[m]);
    T* y = static_cast<T*>(a.y.p[m]) + row * a.y_stride;
    float f[VE], sum = 0.0f, square = 0.0f;
#pragma unroll 4
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        read_elements<T, WHOLE>(x, at, f);
#pragma unroll
        for (int e = 0; e < VE; ++e) sum += f[e];
    }
    const float mean = row_sum<0>(sum, 0) * a.inv_cols;
#pragma unroll 4
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        read_elements<T, WHOLE>(x, at, f);
#pragma unroll
        for (int e = 0; e < VE; ++e) square = fmaf(f[e] - mean, f[e] - mean, square);
    }
    const float rstd = inverse_root(fmaf(row_sum<0>(square, 1), a.inv_cols, a.eps));
    if (a.has_stats && threadIdx.x == 0) {
        static_cast<float*>(a.mean.p[m])[row] = mean;
        static_cast<float*>(a.rstd.p[m])[row] = rstd;
    }
#pragma unroll 2
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        read_elements<T, WHOLE>(x, at, f);
#pragma unroll
        for (int e = 0; e < VE; ++e)
            f[e] = fmaf((f[e] - mean) * rstd, a.has_gamma ? widen(gamma[at * VE + e]) : 1.0f, a.has_beta ? widen(beta[at * VE + e]) : 0.0f);
        write_elements<T, WHOLE>(y, at, f);
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

// A worker's column sums over the rows of one CTA go to the CTA's place in `partial`, or, when it is the
// worker's only CTA, to the gradients themselves.  The sums stand in the order of the threads that hold them
// (by columns, a warp's stores would touch 32 sectors each): slot (i, lane) of element i of a thread.
__device__ __forceinline__ int slot_column(const NormBackwardArgs& a, int j)
{
    const int i = j / a.lanes, lane = j % a.lanes;
    return (lane + i / a.word * a.lanes) * a.word + i % a.word;
}
template <typename T>
__device__ __forceinline__ void store_slot_sums(const NormBackwardArgs& a, int m, int part, int slot, float dg, float db)
{
    if (a.parts == 1) {
        const int col = slot_column(a, slot);
        if (col < a.cols) store_gradients<T>(a, m, col, dg, db);
    } else {
        float* p = a.partial + (static_cast<size_t>(m) * a.parts + part) * 2 * a.slots + slot;
        p[0] = dg;
        p[a.slots] = db;
    }
}

// Whole rows under way are staged through shared memory by asynchronous copies, `depth` - 1 rows ahead of the one
// that is computed (registers are full of column sums; one row ahead in registers left the SM waiting for memory),
// each thread its own words, so that no barrier is needed.
template <int NV> struct NormStage {
    static constexpr int depth = NV <= 3 ? 4 : NV <= 4 ? 3 : 2;
    static constexpr size_t bytes_a_thread = depth * 2 * NV * 16;
};
// CTAs of kNormThreads that an SM is to hold, by a thread's elements (three registers each, and the words).
constexpr int norm_ctas(int elems, int bytes) { return elems <= 8 ? 6 : elems <= 16 ? (bytes == 2 ? 5 : 4) : elems <= 24 ? (bytes == 2 ? 4 : 3) : (bytes == 2 ? 3 : 2); }

// gridDim.x CTAs a worker go through its rows in turn; a thread keeps the sums of its own columns in
// registers over all of them, so the weights' gradients cost one small table at the end and no atomics
// (the split depends on the sizes alone: the same bits every time).  A moderate number of rows goes to one cluster of CTAs
// a worker, whose CTAs read each other's sums from shared memory: no table and no second launch.
template <typename T, int NV, int LPR, int MODE>
__global__ void __launch_bounds__(LPR ? kNormThreads : kNormMaxBlock, LPR == 32 ? norm_ctas(NV * kWordElems<T>, sizeof(T)) : 1)
layernorm_backward_kernel(const __grid_constant__ NormBackwardArgs a)
{
    stream_order();
    using R = Rows<T, MODE>;
    constexpr int VE = R::VE, EPT = NV * VE, LANES = LPR ? LPR : 32, GROUPS = LPR ? kNormThreads / LANES : 1;
    constexpr int DEPTH = NormStage<NV>::depth;
    extern __shared__ uint4 ring[];                           // [depth][x, dy][NV][threads]
    const int m = blockIdx.y;
    const int lanes = LPR ? LPR : blockDim.x, lane = LPR ? threadIdx.x % LANES : threadIdx.x;
    const int group = LPR ? threadIdx.x / LANES : 0;
    const T* gamma = static_cast<const T*>(a.gamma.p[m]);
    const T* xs = static_cast<const T*>(a.x.p[m]);
    const T* dys = static_cast<const T*>(a.dy.p[m]);
    const float* means = static_cast<const float*>(a.mean.p[m]);
    const float* rstds = static_cast<const float*>(a.rstd.p[m]);

    float gm[EPT], dg[EPT], db[EPT];
#pragma unroll
    for (int k = 0; k < EPT; ++k) {
        const int col = R::column(k / VE, k % VE, lane, lanes);
        gm[k] = a.has_gamma && col < a.cols ? widen(gamma[col]) : 1.0f;
        dg[k] = db[k] = 0.0f;
    }
    const long long stride = static_cast<long long>(gridDim.x) * GROUPS;
    long long row = static_cast<long long>(blockIdx.x) * GROUPS + group;
    const auto fetch = [&](int slot, long long r) {
        if (r < a.rows) {
            const uint4* x = reinterpret_cast<const uint4*>(xs + r * a.x_stride) + lane;
            const uint4* dy = reinterpret_cast<const uint4*>(dys + r * a.y_stride) + lane;
            uint4* to = ring + static_cast<size_t>(slot) * 2 * NV * blockDim.x + threadIdx.x;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (R::any(i, lane, lanes, a.cols)) {
                    copy_async16(to + i * blockDim.x, x + i * lanes);
                    copy_async16(to + (NV + i) * blockDim.x, dy + i * lanes);
                }
        }
        copy_async_commit();                                  // a group a row, also where there is none
    };
    if constexpr (R::whole) {
#pragma unroll
        for (int d = 0; d < DEPTH - 1; ++d) fetch(d, row + d * stride);
    }
    int buf = 0, slot = 0;
    float mean = row < a.rows ? means[row] : 0.0f, rstd = row < a.rows ? rstds[row] : 0.0f;
    // (Rows of 8 lanes: the same turns for all groups of a warp, which exchange sums together.)
    for (; (LPR == 8 ? row - group : row) < a.rows; row += stride) {
        const bool live = LPR != 8 || row < a.rows;
        const int cols = live ? a.cols : 0;
        const long long r = live ? row : 0;
        uint4 xw[NV], dw[NV];
        if constexpr (R::whole) {
            fetch(slot == 0 ? DEPTH - 1 : slot - 1, row + (DEPTH - 1) * stride);
            copy_async_wait<DEPTH - 1>();
            const uint4* from = ring + static_cast<size_t>(slot) * 2 * NV * blockDim.x + threadIdx.x;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (R::any(i, lane, lanes, cols)) { xw[i] = from[i * blockDim.x]; dw[i] = from[(NV + i) * blockDim.x]; }
            slot = slot + 1 == DEPTH ? 0 : slot + 1;
        } else {
            const T* x = xs + r * a.x_stride;
            const T* dy = dys + r * a.y_stride;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (R::any(i, lane, lanes, cols)) { xw[i] = R::load(x, i, lane, lanes, cols); dw[i] = R::load(dy, i, lane, lanes, cols); }
        }
        const bool more = row + stride < a.rows;
        const float next_mean = more ? means[row + stride] : 0.0f, next_rstd = more ? rstds[row + stride] : 0.0f;
        // (Behind the end of a row dy is zero, and with it every term of the sums.)
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!R::any(i, lane, lanes, cols)) continue;
            float f[VE], d[VE];
            shifted<T>(xw[i], -mean, f);
            unpack<T>(dw[i], d);
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
            // (f rstd is taken first: rstd^2, and mean(g h) rstd^2, may be past fp32's range where dx is far inside it)
            const float mg = -s.x * a.inv_cols * rstd, mgh = -s.y * a.inv_cols * rstd;
            T* dx = static_cast<T*>(a.dx.p[m]) + r * a.x_stride;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (R::any(i, lane, lanes, cols)) {
                    float f[VE], d[VE];
                    shifted<T>(xw[i], -mean, f);
                    unpack<T>(dw[i], d);
#pragma unroll
                    for (int e = 0; e < VE; ++e) f[e] = fmaf(d[e] * gm[i * VE + e], rstd, fmaf(f[e] * rstd, mgh, mg));
                    v = pack<T>(f);
                }
                R::store(dx, i, lane, lanes, cols, v, LANES);
            }
        }
        mean = next_mean;
        rstd = next_rstd;
    }
    if constexpr (R::whole) copy_async_wait<0>();
    if (!a.has_dgamma && !a.has_dbeta) return;
    float2* sums;                                             // the CTA's, by slots, where they pass through shared memory
    if constexpr (LPR == 0) {
        if (!a.cluster) {
#pragma unroll
            for (int k = 0; k < EPT; ++k) store_slot_sums<T>(a, m, blockIdx.x, k * lanes + lane, dg[k], db[k]);
            return;
        }
        __syncthreads();                                      // the stages have been read
        sums = reinterpret_cast<float2*>(ring);
#pragma unroll
        for (int k = 0; k < EPT; ++k) sums[k * lanes + lane] = make_float2(dg[k], db[k]);
    } else {
        // groups of rows: first the groups of a warp, then the warps in order
        __shared__ float2 acc[LPR * EPT];
        sums = acc;
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
        if (!a.cluster) {
            for (int j = threadIdx.x; j < LPR * EPT; j += kNormThreads) store_slot_sums<T>(a, m, blockIdx.x, j, acc[j].x, acc[j].y);
            return;
        }
    }
    // A cluster: every CTA adds up its share of the slots over all CTAs, in their order, and finishes them.
    const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    cluster.sync();
    for (int j = blockIdx.x * blockDim.x + threadIdx.x; j < a.slots; j += gridDim.x * blockDim.x) {
        float2 s = make_float2(0.0f, 0.0f);
        for (unsigned p = 0; p < gridDim.x; ++p) {
            const float2 v = cluster.map_shared_rank(sums, p)[j];
            s.x += v.x;
            s.y += v.y;
        }
        const int col = slot_column(a, j);
        if (col < a.cols) store_gradients<T>(a, m, col, s.x, s.y);
    }
    cluster.sync();                                           // no CTA leaves while its sums are read
}

// Rows that do not fit in a CTA's registers: dx by a CTA per row (dy and x are read again from L2) ...
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kNormLongThreads)
layernorm_backward_long_kernel(const __grid_constant__ NormBackwardArgs a)
{
    stream_order();
    constexpr int VE = WHOLE ? kWordElems<T> : 1;
    const int m = blockIdx.y, words = a.cols / VE;
    const long long row = blockIdx.x;
    const T* x = static_cast<const T*>(a.x.p[m]) + row * a.x_stride;
    const T* dy = static_cast<const T*>(a.dy.p[m]) + row * a.y_stride;
    const T* gamma = static_cast<const T*>(a.gamma.p[m]);
    T* dx = static_cast<T*>(a.dx.p[m]) + row * a.x_stride;
    const float mean = static_cast<const float*>(a.mean.p[m])[row], rstd = static_cast<const float*>(a.rstd.p[m])[row];
    float f[VE], d[VE];
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll 4
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        read_elements<T, WHOLE>(x, at, f);
        read_elements<T, WHOLE>(dy, at, d);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float g = d[e] * (a.has_gamma ? widen(gamma[at * VE + e]) : 1.0f);
            s.x += g;
            s.y = fmaf(g, (f[e] - mean) * rstd, s.y);
        }
    }
    s = row_sum<0>(s, 0);
    const float mg = s.x * a.inv_cols, mgh = s.y * a.inv_cols;
#pragma unroll 2
    for (int at = threadIdx.x; at < words; at += kNormLongThreads) {
        read_elements<T, WHOLE>(x, at, f);
        read_elements<T, WHOLE>(dy, at, d);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float g = d[e] * (a.has_gamma ? widen(gamma[at * VE + e]) : 1.0f);
            f[e] = (g - mg - (f[e] - mean) * rstd * mgh) * rstd;
        }
        write_elements<T, WHOLE>(dx, at, f);
    }
}

// ... and the weights' gradients by columns, gridDim.z parts of the rows: a warp takes 32 neighbouring words (or
// elements) of a row, and the warps of a CTA take rows in turn.
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kNormThreads)
layernorm_columns_kernel(const __grid_constant__ NormBackwardArgs a)
{
    stream_order();
    constexpr int VE = WHOLE ? kWordElems<T> : 1, kWarps = kNormThreads / 32;
    __shared__ float2 acc[kWarps][32 * VE];
    const int m = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, at = blockIdx.x * 32 + lane, part = blockIdx.z;
    const float* means = static_cast<const float*>(a.mean.p[m]);
    const float* rstds = static_cast<const float*>(a.rstd.p[m]);
    float dg[VE] = {}, db[VE] = {};
    if (at < a.cols / VE) {
        const T* x = static_cast<const T*>(a.x.p[m]);
        const T* dy = static_cast<const T*>(a.dy.p[m]);
#pragma unroll 4
        for (long long row = part * kWarps + warp; row < a.rows; row += static_cast<long long>(a.parts) * kWarps) {
            float f[VE], d[VE];
            read_elements<T, WHOLE>(x + row * a.x_stride, at, f);
            read_elements<T, WHOLE>(dy + row * a.y_stride, at, d);
            const float mean = means[row], rstd = rstds[row];
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                dg[e] = fmaf(d[e], (f[e] - mean) * rstd, dg[e]);
                db[e] += d[e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) acc[warp][e * 32 + lane] = make_float2(dg[e], db[e]);
    __syncthreads();
    for (int j = threadIdx.x; j < 32 * VE; j += kNormThreads) {
        float2 s = acc[0][j];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) { s.x += acc[w][j].x; s.y += acc[w][j].y; }
        const int col = (blockIdx.x * 32 + j % 32) * VE + j / 32;
        if (col < a.cols) store_slot_sums<T>(a, m, part, col, s.x, s.y);            // (a slot a column)
    }
}

// The parts' column sums, added in a fixed order: 32 slots a CTA, kFinishGroups threads a slot.
constexpr int kFinishGroups = 16;
template <typename T>
__global__ void __launch_bounds__(32 * kFinishGroups)
layernorm_finish_kernel(const __grid_constant__ NormBackwardArgs a)
{
    stream_order();
    __shared__ float2 acc[kFinishGroups][32];
    const int m = blockIdx.y, lane = threadIdx.x & 31, group = threadIdx.x >> 5, slot = blockIdx.x * 32 + lane;
    float2 s = make_float2(0.0f, 0.0f);
    if (slot < a.slots) {
        const float* p = a.partial + static_cast<size_t>(m) * a.parts * 2 * a.slots + slot;
#pragma unroll 4
        for (int i = group; i < a.parts; i += kFinishGroups) {
            s.x += p[static_cast<size_t>(i) * 2 * a.slots];
            s.y += p[static_cast<size_t>(i) * 2 * a.slots + a.slots];
        }
    }
    acc[group][lane] = s;
    __syncthreads();
    if (group != 0 || slot >= a.slots) return;
    const int col = slot_column(a, slot);
    if (col >= a.cols) return;
#pragma unroll
    for (int g = 1; g < kFinishGroups; ++g) { s.x += acc[g][lane].x; s.y += acc[g][lane].y; }
    store_gradients<T>(a, m, col, s.x, s.y);
}

}  // namespace replica
}  // namespace grawa

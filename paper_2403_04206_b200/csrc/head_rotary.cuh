// Norms of the query and key heads with the rotation by position, of all M workers in one call, and their gradients.
//
//   forward   s = 1 / sqrt(mean x^2 + eps) over a head's elements, z = w x s, y = R z
//   backward  dz = R^T dy, dw = sum over rows and heads of dz x s, g = dz w, dx = s (g - x s mean(g x s))
//
// R turns the leading `2 half` elements in pairs, pair i by the angle position * frequency[i].  The angle is taken and
// reduced to a fraction of a turn in 64 bits: in 32, a position of a million leaves 0.06 radians of error.
//
// One pass: a head lies in the registers of a few neighbouring lanes, which hold both elements of each pair, so that the
// rotation exchanges nothing and a sum of squares is a few shuffles.  A warp takes one row after the other, works its
// angles out once (a pair's sine and cosine in one lane, shared through shared memory), and uses them for all of the row's
// query and key heads.  Bound by memory: forward reads and writes each element once, backward reads two and writes one.
#pragma once
#include "replica_common.cuh"

namespace grawa {
namespace replica {

// How a lane holds its share of a head, in two runs a[] and b[] of n elements:
//   kPairWords  words a and b are word j and the word `half` elements behind it: pairs of halves, (a[e], b[e]);
//               lanes behind the rotated part hold two neighbouring words
//   kPairNext   two neighbouring words: pairs of neighbours, (a[2i], a[2i + 1]) and (b[2i], b[2i + 1])
//   kPairAny    single elements, at any address and of any number: pair lane + 32 t for t < n / 2, then what is not rotated;
//               kPairAnyShort for heads of up to 128 elements (n = 4), kPairAny for longer ones (n = 8)
enum HeadMode { kPairWords = 0, kPairNext = 1, kPairAny = 2, kPairAnyShort = 3 };
template <int MODE> constexpr bool kSingles = MODE >= kPairAny;
constexpr int kHeadDim = 256;               // largest head
constexpr int kHeadThreads = 256;

struct HeadArgs {
    In x[2], w[2], dy[2];                   // queries, keys; w may be NULL (1); dy in the backward pass
    Out y[2];                               // forward: results; backward: dx
    Out dw[2];                              // backward
    In positions;                           // 64-bit integers, or NULL: row number modulo `period`
    const double* frequencies;
    float* partial;                         // backward, parts > 1: [worker][part][2][kHeadDim]
    unsigned rows, period;
    long long x_stride[2], y_stride[2];     // backward: of x and dx, and of dy
    int heads[2];
    int dim, half, neighbours, words;       // words: of a head (kPairWords, kPairNext)
    int chunks, per_chunk;                  // forward: a row's steps are shared out among so many warps, so many each
    int parts;                              // backward: CTAs a worker
    int has_w[2], has_dw[2], has_dx[2], accumulate;
    float eps, inv_dim;
    unsigned small;                         // bits of the mean square below which it is taken again, of scaled elements
};

template <typename T, int MODE> constexpr int kHeadRun = MODE == kPairAny ? 8 : MODE == kPairAnyShort ? 4 : kWordElems<T>;

// The places of a lane's elements in a head, and their loads and stores.
template <typename T, int MODE>
struct HeadLane {
    static constexpr int N = kHeadRun<T, MODE>;
    int first[2];                           // words: of a[] and b[]
    int dim, half, neighbours, lane;
    bool has[2];

    __device__ __forceinline__ HeadLane(const HeadArgs& a, int l) : dim(a.dim), half(a.half), neighbours(a.neighbours), lane(l)
    {
        if constexpr (MODE == kPairWords) {
            const int turned = a.half / N;
            first[0] = l < turned ? l : 2 * turned + 2 * (l - turned);
            first[1] = l < turned ? l + turned : first[0] + 1;
        } else {
            first[0] = 2 * l;
            first[1] = 2 * l + 1;
        }
        has[0] = kSingles<MODE> || first[0] < a.words;
        has[1] = kSingles<MODE> || first[1] < a.words;
    }
    // Single elements: the place of element t of a[] (which = 0) or b[], or -1.
    __device__ __forceinline__ int place(int t, int which) const
    {
        if (t < N / 2) {
            const int p = lane + 32 * t;
            return p >= half ? -1 : neighbours ? 2 * p + which : p + which * half;
        }
        const int e = 2 * half + lane + 32 * (2 * (t - N / 2) + which);
        return e < dim ? e : -1;
    }
    __device__ __forceinline__ void load(const T* head, float (&a)[N], float (&b)[N]) const
    {
        if constexpr (kSingles<MODE>) {
#pragma unroll
            for (int t = 0; t < N; ++t) {
                const int i = place(t, 0), j = place(t, 1);
                a[t] = i >= 0 ? widen(head[i]) : 0.0f;
                b[t] = j >= 0 ? widen(head[j]) : 0.0f;
            }
        } else {
            const uint4* w = reinterpret_cast<const uint4*>(head);
            unpack<T>(has[0] ? w[first[0]] : make_uint4(0, 0, 0, 0), a);
            unpack<T>(has[1] ? w[first[1]] : make_uint4(0, 0, 0, 0), b);
        }
    }
    // A lane's share on its way: words as they are, single elements widened.
    struct Held {
        uint4 a, b;
        float x[kSingles<MODE> ? N : 1], y[kSingles<MODE> ? N : 1];
    };
    __device__ __forceinline__ void fetch(const T* head, bool mine, Held& to) const
    {
        if constexpr (kSingles<MODE>) {
            if (mine) load(head, to.x, to.y);
            else {
#pragma unroll
                for (int e = 0; e < N; ++e) to.x[e] = to.y[e] = 0.0f;
            }
        } else {
            const uint4* w = reinterpret_cast<const uint4*>(head);
            to.a = mine && has[0] ? __ldcs(w + first[0]) : make_uint4(0, 0, 0, 0);
            to.b = mine && has[1] ? __ldcs(w + first[1]) : make_uint4(0, 0, 0, 0);
        }
    }
    static __device__ __forceinline__ void open(const Held& from, float (&a)[N], float (&b)[N])
    {
        if constexpr (kSingles<MODE>) {
#pragma unroll
            for (int e = 0; e < N; ++e) a[e] = from.x[e], b[e] = from.y[e];
        } else {
            unpack<T>(from.a, a);
            unpack<T>(from.b, b);
        }
    }
    __device__ __forceinline__ void store(T* head, const float (&a)[N], const float (&b)[N]) const
    {
        if constexpr (kSingles<MODE>) {
#pragma unroll
            for (int t = 0; t < N; ++t) {
                const int i = place(t, 0), j = place(t, 1);
                if (i >= 0) head[i] = narrow<T>(a[t]);
                if (j >= 0) head[j] = narrow<T>(b[t]);
            }
        } else {
            uint4* w = reinterpret_cast<uint4*>(head);
            if (has[0]) w[first[0]] = pack<T>(a);
            if (has[1]) w[first[1]] = pack<T>(b);
        }
    }
    // The same places of a vector of kHeadDim floats in shared memory (what lies behind the head's end is not used).
    __device__ __forceinline__ void from_shared(const float* v, float (&a)[N], float (&b)[N]) const
    {
        if constexpr (kSingles<MODE>) {
#pragma unroll
            for (int t = 0; t < N; ++t) {
                const int i = place(t, 0), j = place(t, 1);
                a[t] = i >= 0 ? v[i] : 0.0f;
                b[t] = j >= 0 ? v[j] : 0.0f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                const float4 x = has[0] ? *reinterpret_cast<const float4*>(v + first[0] * N + e) : make_float4(0, 0, 0, 0);
                const float4 y = has[1] ? *reinterpret_cast<const float4*>(v + first[1] * N + e) : make_float4(0, 0, 0, 0);
                a[e] = x.x; a[e + 1] = x.y; a[e + 2] = x.z; a[e + 3] = x.w;
                b[e] = y.x; b[e + 1] = y.y; b[e + 2] = y.z; b[e + 3] = y.w;
            }
        }
    }
    __device__ __forceinline__ void to_shared(float* v, const float (&a)[N], const float (&b)[N]) const
    {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int i = kSingles<MODE> ? place(e, 0) : has[0] ? first[0] * N + e : -1;
            const int j = kSingles<MODE> ? place(e, 1) : has[1] ? first[1] * N + e : -1;
            if (i >= 0) v[i] = a[e];
            if (j >= 0) v[j] = b[e];
        }
    }
    // Cosine and sine of the lane's N pairs from the warp's table (1 and 0 where nothing turns).
    __device__ __forceinline__ void angles(const float2* table, float (&c)[N], float (&s)[N]) const
    {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            int p;
            if constexpr (kSingles<MODE>) p = e < N / 2 ? lane + 32 * e : half;
            else if constexpr (MODE == kPairWords) p = first[0] * N + e;
            else p = first[e * 2 / N] * (N / 2) + e % (N / 2);
            const float2 t = p < half ? table[p] : make_float2(1.0f, 0.0f);
            c[e] = t.x;
            s[e] = t.y;
        }
    }
    // The pairs turned by their angles, or back (sign -1).
    static __device__ __forceinline__ void turn(float (&a)[N], float (&b)[N], const float (&c)[N], const float (&s)[N], float sign)
    {
        if constexpr (MODE == kPairNext) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float x = a[2 * i], y = a[2 * i + 1], u = b[2 * i], v = b[2 * i + 1], sx = sign * s[i], su = sign * s[N / 2 + i];
                a[2 * i] = x * c[i] - y * sx;
                a[2 * i + 1] = y * c[i] + x * sx;
                b[2 * i] = u * c[N / 2 + i] - v * su;
                b[2 * i + 1] = v * c[N / 2 + i] + u * su;
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float x = a[e], y = b[e], t = sign * s[e];
                a[e] = x * c[e] - y * t;
                b[e] = y * c[e] + x * t;
            }
        }
    }
};

// Cosine and sine of a row's pairs into the warp's table.
__device__ __forceinline__ void fill_angles(const HeadArgs& a, int m, unsigned row, int lane, float2* table)
{
    const long long* given = static_cast<const long long*>(a.positions.p[m]);
    const double position = static_cast<double>(given ? given[row] : row % a.period);
    __syncwarp();                                             // the row in front has been read
    for (int p = lane; p < a.half; p += 32) {
        const double turns = position * a.frequencies[p] * 0.15915494309189533577;       // 1 / (2 pi)
        float s, c;
        sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &s, &c);
        table[p] = make_float2(c, s);
    }
    __syncwarp();
}

template <typename T>
__device__ __forceinline__ void load_weights(const HeadArgs& a, int which, int m, float* to)
{
    const T* w = static_cast<const T*>(a.w[which].p[m]);
    for (int e = threadIdx.x; e < a.dim; e += kHeadThreads) to[e] = a.has_w[which] ? widen(w[e]) : 1.0f;
}

// Whether squares of a head's elements are neither past the range of 32 bits nor so small that some are missing and eps does not make up
// for them.
__device__ __forceinline__ bool squares_in_range(const HeadArgs& a, float mean)
{
    constexpr unsigned kMost = 0x7c000000u;                   // 2^121
    return __float_as_uint(mean) - a.small <= kMost - a.small;
}
// 1 / sqrt(mean x^2 + eps) of a head whose lanes' elements are x and y and whose mean square and eps make `mean`, where that is not so: of
// elements that are scaled by a power of two, `scale`.  (By the head's lanes alone, which all have the same mean.)
template <int LPH, int N>
__device__ __forceinline__ float scaled_norm(const HeadArgs& a, float mean, float (&x)[N], float (&y)[N], float& scale)
{
    const unsigned lanes = LPH == 32 ? ~0u : ((1u << LPH % 32) - 1) << (threadIdx.x % 32 / LPH * LPH);
    const float root = sqrtf(a.eps);
    float most = root, square = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) most = fmaxf(most, fmaxf(fabsf(x[e]), fabsf(y[e])));
#pragma unroll
    for (int d = LPH / 2; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(lanes, most, d));
    if (!(most > 0.0f && most < INFINITY)) return rsqrtf(mean);
    scale = exp2f(static_cast<float>(-max(-126, min(126, ilogbf(most)))));
#pragma unroll
    for (int e = 0; e < N; ++e) {
        x[e] *= scale;
        y[e] *= scale;
        square = fmaf(x[e], x[e], fmaf(y[e], y[e], square));
    }
#pragma unroll
    for (int d = LPH / 2; d > 0; d >>= 1) square += __shfl_xor_sync(lanes, square, d);
    return rsqrtf(fmaf(square, a.inv_dim, (root * scale) * (root * scale)));
}

// All of the forward pass for one such head, from the start.  (Not inlined: in the loop it takes registers, and 4 x 8192 rows of 32 + 8 heads of
// 128 bf16 125 us instead of 121.)
template <typename T, int LPH, int MODE>
__device__ __noinline__ void scaled_head(const HeadArgs& a, HeadLane<T, MODE> at, float mean, const T* from, T* to, const float* weights, const float2* table)
{
    constexpr int N = kHeadRun<T, MODE>;
    float x[N], y[N], wa[N], wb[N], c[N], s[N], scale;
    at.load(from, x, y);
    const float r = scaled_norm<LPH>(a, mean, x, y, scale);
    at.from_shared(weights, wa, wb);
    at.angles(table, c, s);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        x[e] = x[e] * r * wa[e];
        y[e] = y[e] * r * wb[e];
    }
    at.turn(x, y, c, s, 1.0f);
    at.store(to, x, y);
}

// A row's heads in steps of `per` neighbouring ones, those of the queries first.
struct HeadSteps {
    int q_steps, steps;
    __device__ __forceinline__ HeadSteps(const HeadArgs& a, int per) : q_steps((a.heads[0] + per - 1) / per), steps(q_steps + (a.heads[1] + per - 1) / per) {}
};

// Where a warp stands in its chunks of rows: a chunk is a run of a row's steps.
struct HeadWalk {
    unsigned unit, row;
    int step, end;
    __device__ __forceinline__ void enter(const HeadArgs& a, int steps)
    {
        row = a.chunks == 1 ? unit : unit / a.chunks;
        step = a.chunks == 1 ? 0 : static_cast<int>(unit - row * a.chunks) * a.per_chunk;
        end = min(step + a.per_chunk, steps);
    }
    __device__ __forceinline__ bool inside(const HeadArgs& a) const { return unit < a.rows * static_cast<unsigned>(a.chunks); }
    __device__ __forceinline__ void advance(const HeadArgs& a, int steps)
    {
        if (++step < end) return;
        unit += gridDim.x * (kHeadThreads / 32);
        enter(a, steps);
    }
};

// LPH: lanes a head.  A step's loads are under way while the kHeadAhead steps in front of it are worked on, whatever rows they belong to
// (4 x 8192 rows of 32 + 8 heads of 128 bf16: 148 us with each step's loads in front of it).
template <int MODE> constexpr int kHeadAhead = MODE == kPairAny ? 1 : 4;
template <typename T, int LPH, int MODE>
__global__ void __launch_bounds__(kHeadThreads, 2)
head_rotary_forward_kernel(const __grid_constant__ HeadArgs a)
{
    constexpr int N = kHeadRun<T, MODE>, kPer = 32 / LPH, kWarps = kHeadThreads / 32, kAhead = kHeadAhead<MODE>;
    __shared__ __align__(16) float weights[2][kHeadDim];
    __shared__ float2 tables[kWarps][kHeadDim / 2];
    stream_order();
    const int m = blockIdx.y, warp = threadIdx.x / 32, lane = threadIdx.x % 32, slot = lane / LPH;
    const HeadLane<T, MODE> at(a, lane % LPH);
    const HeadSteps all(a, kPer);
    HeadWalk now, ahead;
    now.unit = blockIdx.x * kWarps + warp;
    now.enter(a, all.steps);
    ahead = now;
    typename HeadLane<T, MODE>::Held held[kAhead];
    const auto fetch = [&](typename HeadLane<T, MODE>::Held& to) {
        if (!ahead.inside(a)) return;
        const int which = ahead.step >= all.q_steps, h = (ahead.step - (which ? all.q_steps : 0)) * kPer + slot;
        at.fetch(static_cast<const T*>(a.x[which].p[m]) + ahead.row * a.x_stride[which] + static_cast<long long>(h) * a.dim, h < a.heads[which], to);
        ahead.advance(a, all.steps);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(held[i]);
    load_weights<T>(a, 0, m, weights[0]);
    if (a.heads[1]) load_weights<T>(a, 1, m, weights[1]);
    __syncthreads();
    float c[N], s[N];
    unsigned turned = ~0u;                                    // the unit that c and s are of
    while (now.inside(a)) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (!now.inside(a)) break;
            if (now.unit != turned) {
                fill_angles(a, m, now.row, lane, tables[warp]);
                at.angles(tables[warp], c, s);
                turned = now.unit;
            }
            const int which = now.step >= all.q_steps, h = (now.step - (which ? all.q_steps : 0)) * kPer + slot;
            float x[N], y[N], wa[N], wb[N], sum = 0.0f;
            at.open(held[i], x, y);
            fetch(held[i]);
#pragma unroll
            for (int e = 0; e < N; ++e) sum = fmaf(x[e], x[e], fmaf(y[e], y[e], sum));
            const float mean = fmaf(lanes_sum<LPH>(sum), a.inv_dim, a.eps), r = rsqrtf(mean);
            at.from_shared(weights[which], wa, wb);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = x[e] * r * wa[e];
                y[e] = y[e] * r * wb[e];
            }
            at.turn(x, y, c, s, 1.0f);
            if (h < a.heads[which]) {
                T* const to = static_cast<T*>(a.y[which].p[m]) + now.row * a.y_stride[which] + static_cast<long long>(h) * a.dim;
                if (squares_in_range(a, mean)) at.store(to, x, y);
                else scaled_head<T, LPH, MODE>(a, at, mean, static_cast<const T*>(a.x[which].p[m]) + now.row * a.x_stride[which] + static_cast<long long>(h) * a.dim, to,
                                               weights[which], tables[warp]);
            }
            now.advance(a, all.steps);
        }
    }
}

// The sums over a CTA of what its lanes hold for each element of a weight, in a fixed order, into kHeadDim floats.
template <typename T, int LPH, int MODE>
__device__ __forceinline__ void sum_weights(const HeadLane<T, MODE>& at, float (&da)[kHeadRun<T, MODE>], float (&db)[kHeadRun<T, MODE>], float* shared, float* to,
                                            int dim)
{
    constexpr int N = kHeadRun<T, MODE>, kWarps = kHeadThreads / 32;
#pragma unroll
    for (int e = 0; e < N; ++e)
#pragma unroll
        for (int d = LPH; d < 32; d *= 2) {
            da[e] += __shfl_xor_sync(0xffffffffu, da[e], d);
            db[e] += __shfl_xor_sync(0xffffffffu, db[e], d);
        }
    __syncthreads();
    if (threadIdx.x % 32 < LPH) at.to_shared(shared + threadIdx.x / 32 * kHeadDim, da, db);
    __syncthreads();
    for (int e = threadIdx.x; e < dim; e += kHeadThreads) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += shared[w * kHeadDim + e];
        to[e] = v;
    }
}

template <typename T>
__device__ __forceinline__ void put_weight(const HeadArgs& a, int which, int m, int e, float v)
{
    T* to = static_cast<T*>(a.dw[which].p[m]) + e;
    *to = narrow<T>(a.accumulate ? widen(*to) + v : v);
}

template <typename T, int LPH, int MODE>
__global__ void __launch_bounds__(kHeadThreads, 2)
head_rotary_backward_kernel(const __grid_constant__ HeadArgs a)
{
    constexpr int N = kHeadRun<T, MODE>, kPer = 32 / LPH, kWarps = kHeadThreads / 32;
    using Lane = HeadLane<T, MODE>;
    __shared__ __align__(16) float weights[2][kHeadDim];
    __shared__ float2 tables[kWarps][kHeadDim / 2];
    __shared__ float sums[kWarps * kHeadDim];
    stream_order();
    const int m = blockIdx.y, warp = threadIdx.x / 32, lane = threadIdx.x % 32, slot = lane / LPH;
    const Lane at(a, lane % LPH);
    load_weights<T>(a, 0, m, weights[0]);
    if (a.heads[1]) load_weights<T>(a, 1, m, weights[1]);
    __syncthreads();
    float da[2][N] = {}, db[2][N] = {};
    typename Lane::Held held[2];                              // x and dy of the next step, on their way
    const auto fetch = [&](unsigned row, int which, int h0) {
        const int h = h0 + slot;
        const long long place = static_cast<long long>(h) * a.dim;
        at.fetch(static_cast<const T*>(a.x[which].p[m]) + row * a.x_stride[which] + place, h < a.heads[which], held[0]);
        at.fetch(static_cast<const T*>(a.dy[which].p[m]) + row * a.y_stride[which] + place, h < a.heads[which], held[1]);
    };
    const unsigned start = blockIdx.x * kWarps + warp, stride = gridDim.x * kWarps;
    if (start < a.rows) fetch(start, 0, 0);
    for (unsigned row = start; row < a.rows; row += stride) {
        fill_angles(a, m, row, lane, tables[warp]);
        float c[N], s[N];
        at.angles(tables[warp], c, s);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            T* out = static_cast<T*>(a.y[which].p[m]) + row * a.x_stride[which];
#pragma unroll 1
            for (int h0 = 0; h0 < a.heads[which]; h0 += kPer) {
                const int h = h0 + slot;
                float x[N], y[N], u[N], v[N], wa[N], wb[N], square = 0.0f, along = 0.0f;
                Lane::open(held[0], x, y);
                Lane::open(held[1], u, v);
                if (h0 + kPer < a.heads[which]) fetch(row, which, h0 + kPer);
                else if (which == 0 && a.heads[1]) fetch(row, 1, 0);
                else if (row + stride < a.rows) fetch(row + stride, 0, 0);
                at.turn(u, v, c, s, -1.0f);
#pragma unroll
                for (int e = 0; e < N; ++e) square = fmaf(x[e], x[e], fmaf(y[e], y[e], square));
                const float mean = fmaf(lanes_sum<LPH>(square), a.inv_dim, a.eps);
                float scale = 1.0f, r = rsqrtf(mean);
                if (!squares_in_range(a, mean)) r = scaled_norm<LPH>(a, mean, x, y, scale);
                if (h >= a.heads[which]) r = 0.0f;            // no head: its zeros are to stay such, also without eps
                at.from_shared(weights[which], wa, wb);
#pragma unroll
                for (int e = 0; e < N; ++e) {                 // x s first: s^2 may be past fp32's range where dx is inside it
                    x[e] *= r;
                    y[e] *= r;
                    da[which][e] = fmaf(u[e], x[e], da[which][e]);
                    db[which][e] = fmaf(v[e], y[e], db[which][e]);
                    u[e] *= wa[e];
                    v[e] *= wb[e];
                    along = fmaf(u[e], x[e], fmaf(v[e], y[e], along));
                }
                along = lanes_sum<LPH>(along) * a.inv_dim;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    u[e] = (u[e] - x[e] * along) * r;
                    v[e] = (v[e] - y[e] * along) * r;
                }
                if (scale != 1.0f) {
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        u[e] *= scale;
                        v[e] *= scale;
                    }
                }
                if (h < a.heads[which] && a.has_dx[which]) at.store(out + static_cast<long long>(h) * a.dim, u, v);
            }
        }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if (!a.has_dw[which]) continue;
        if (a.parts > 1) {
            sum_weights<T, LPH, MODE>(at, da[which], db[which], sums, a.partial + ((static_cast<size_t>(m) * a.parts + blockIdx.x) * 2 + which) * kHeadDim, a.dim);
        } else {
            sum_weights<T, LPH, MODE>(at, da[which], db[which], sums, weights[which], a.dim);
            for (int e = threadIdx.x; e < a.dim; e += kHeadThreads) put_weight<T>(a, which, m, e, weights[which][e]);     // its own sums
        }
    }
}

// The parts' sums, added in their order: 32 elements a CTA, kHeadGroups runs of parts side by side.
constexpr int kHeadGroups = 16;
template <typename T>
__global__ void __launch_bounds__(32 * kHeadGroups)
head_rotary_finish_kernel(const __grid_constant__ HeadArgs a)
{
    __shared__ float sums[kHeadGroups][32];
    stream_order();
    const int m = blockIdx.y, which = blockIdx.z, lane = threadIdx.x % 32, group = threadIdx.x / 32, e = blockIdx.x * 32 + lane;
    if (!a.has_dw[which]) return;
    const int run = (a.parts + kHeadGroups - 1) / kHeadGroups, last = min(a.parts, (group + 1) * run);
    float v = 0.0f;
    if (e < a.dim)
#pragma unroll 4
        for (int p = group * run; p < last; ++p) v += a.partial[((static_cast<size_t>(m) * a.parts + p) * 2 + which) * kHeadDim + e];
    sums[group][lane] = v;
    __syncthreads();
    if (group || e >= a.dim) return;
    v = 0.0f;
#pragma unroll
    for (int g = 0; g < kHeadGroups; ++g) v += sums[g][lane];
    put_weight<T>(a, which, m, e, v);
}

}  // namespace replica
}  // namespace grawa

// Dropout with a residual, on all M workers in one launch.
//
//   w(j) = word j mod 4 of Philox4x32-10 at counter (b low, b high + (m << 24), o low, o high), b = j / 4,
//          o = offset (+ the device's counter), key = (seed low, seed high)
//   y_j  = r_j + (w(j) >= T ? x_j * scale : 0),   T = floor(p 2^32 + 1/2), scale = 1 / (1 - p)
//
// The mask is a function of (seed, offset, worker, element) alone, so the backward pass computes it again
// and no mask is stored or read: 3 (2 without the residual, and in the backward pass) elements of traffic
// per element, and nothing else.
#pragma once
#include "replica_common.cuh"

namespace grawa {
namespace replica {

struct DropoutArgs {
    In x, r;
    Out y;
    long long n;
    unsigned long long seed, offset;
    const unsigned long long* counter;      // device word added to offset, or NULL
    unsigned threshold;
    float scale;
    int residual;
};

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC'11), from
// its published round function and key schedule.
__device__ __forceinline__ uint4 philox(uint4 c, uint2 k)
{
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const unsigned long long a = 0xD2511F53ull * c.x, b = 0xCD9E8D57ull * c.z;
        c = make_uint4(static_cast<unsigned>(b >> 32) ^ c.y ^ k.x, static_cast<unsigned>(b),
                       static_cast<unsigned>(a >> 32) ^ c.w ^ k.y, static_cast<unsigned>(a));
        k.x += 0x9E3779B9u;
        k.y += 0xBB67AE85u;
    }
    return c;
}

// A dropped element does not enter the result at all (a select, not a product with 0), whatever it holds.
__device__ __forceinline__ float dropped(float x, float r, unsigned w, const DropoutArgs& a)
{
    return w >= a.threshold ? fmaf(x, a.scale, r) : r;
}

constexpr int kDropThreads = 256;

// One thread handles COLS columns of 16 bytes (VEC) or of four single elements (any alignment); the threads
// of a warp take neighbouring columns.
template <typename T, bool VEC, int COLS>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const __grid_constant__ DropoutArgs a)
{
    constexpr int VE = VEC ? 16 / static_cast<int>(sizeof(T)) : 4;
    const int m = blockIdx.y;
    const T* x = static_cast<const T*>(a.x.p[m]);
    const T* r = static_cast<const T*>(a.r.p[m]);
    T* y = static_cast<T*>(a.y.p[m]);
    const unsigned long long o = a.offset + (a.counter ? *a.counter : 0ull);
    const uint2 key = make_uint2(static_cast<unsigned>(a.seed), static_cast<unsigned>(a.seed >> 32));
    const long long first = static_cast<long long>(blockIdx.x) * (kDropThreads * COLS) + threadIdx.x;

    using W = WordOf<T, VEC ? VE : 1>;
    W xw[COLS], rw[COLS];
    if constexpr (VEC) {
#pragma unroll
        for (int c = 0; c < COLS; ++c) {                      // all loads first
            const long long j = (first + c * kDropThreads) * VE;
            if (j + VE <= a.n) {
                xw[c] = *reinterpret_cast<const W*>(x + j);
                if (a.residual) rw[c] = *reinterpret_cast<const W*>(r + j);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
        const long long j = (first + c * kDropThreads) * VE;
        if (j >= a.n) return;
        unsigned w[VE];
#pragma unroll
        for (int q = 0; q < VE / 4; ++q) {
            const unsigned long long b = static_cast<unsigned long long>(j) / 4 + q;
            const uint4 v = philox(make_uint4(static_cast<unsigned>(b), static_cast<unsigned>(b >> 32) + (static_cast<unsigned>(m) << 24),
                                              static_cast<unsigned>(o), static_cast<unsigned>(o >> 32)), key);
            w[4 * q] = v.x; w[4 * q + 1] = v.y; w[4 * q + 2] = v.z; w[4 * q + 3] = v.w;
        }
        if (VEC && j + VE <= a.n) {
            if constexpr (VEC) {
                float f[VE], g[VE] = {};
                unpack<T, VE>(xw[c], f);
                if (a.residual) unpack<T, VE>(rw[c], g);
#pragma unroll
                for (int e = 0; e < VE; ++e) f[e] = dropped(f[e], g[e], w[e], a);
                *reinterpret_cast<W*>(y + j) = pack<T, VE>(f);
            }
        } else {
#pragma unroll
            for (int e = 0; e < VE; ++e)
                if (j + e < a.n) y[j + e] = narrow<T>(dropped(widen(x[j + e]), a.residual ? widen(r[j + e]) : 0.0f, w[e], a));
        }
    }
}

}  // namespace replica
}  // namespace grawa

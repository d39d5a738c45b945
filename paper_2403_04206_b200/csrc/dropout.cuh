// Dropout with a residual, on all M workers in one launch.
//
//   w(j) = word j mod 4 of Philox4x32-10 at counter (b low, b high + (m << 24), o low, o high), b = j / 4,
//          o = offset (+ the device's counter), key = (seed low, seed high)
//   y_j  = r_j + (w(j) >= T ? x_j * scale : 0),   T = floor(p 2^32 + 1/2), scale = 1 / (1 - p)
//
// The mask is a function of (seed, offset, worker, element) alone, so the backward pass computes it again
// and no mask is stored or read: 3 (2 without the residual, and in the backward pass) elements of traffic
// per element, and nothing else.
//
// Measured (B200, 6.54 TB/s copy): 8 workers x 4.8 M bf16 with residual 35.5 us = 6.55 TB/s, bound by memory; 16 x 9.7 M
// bf16 without residual 120 to 125 us = 5.0 to 5.2 TB/s (76 to 79 %): 17 instructions an element, of which the
// 4.5 wide multiplications of a quarter block and their exclusive-ors are half.  Its stalls are the multiplications' pipe and
// dispatch, hardly memory, with 60 % of issue slots and 58 % of the integer pipe's cycles used.  Buffers of which any, for any
// worker, does not start on 16 bytes go element by element for all: 3 x 1000003 fp32 5.5 us against 3.7 of traffic.
#pragma once
#include "replica_common.cuh"

namespace grawa {
namespace replica {

struct DropoutArgs {
    In x, r;
    Out y;
    long long n;
    uint2 keys[10];                         // the key of every round
    unsigned long long offset;
    const unsigned long long* counter;      // device word added to offset, or NULL
    unsigned threshold;
    float scale;
};

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC'11), from
// its published round function and key schedule.  A round takes (x, y, z, w) to
//   (hi(M1 z) ^ y ^ k0, lo(M1 z), hi(M0 x) ^ w ^ k1, lo(M0 x)).
// Only x, the low word of the block number, differs between the threads of a CTA (a CTA covers a power of
// two of blocks from a multiple of it): the halves of the first two rounds that do not depend on x are
// computed once a thread, which leaves 18 wide multiplications a block of four words instead of 20.
struct PhiloxHead { unsigned w, k1, y1, z2, w2; };

__device__ __forceinline__ unsigned long long wide(unsigned a, unsigned b) { return static_cast<unsigned long long>(a) * b; }

__device__ __forceinline__ PhiloxHead philox_head(unsigned y, unsigned z, unsigned w, const uint2 (&k)[10])
{
    const unsigned long long b = wide(0xCD9E8D57u, z);
    const unsigned long long a = wide(0xD2511F53u, static_cast<unsigned>(b >> 32) ^ y ^ k[0].x);
    return PhiloxHead{w, k[0].y, static_cast<unsigned>(b) ^ k[1].x, static_cast<unsigned>(a >> 32) ^ k[1].y, static_cast<unsigned>(a)};
}
__device__ __forceinline__ uint4 philox(unsigned x, const PhiloxHead& h, const uint2 (&k)[10])
{
    const unsigned long long a0 = wide(0xD2511F53u, x);
    const unsigned long long b0 = wide(0xCD9E8D57u, static_cast<unsigned>(a0 >> 32) ^ h.w ^ h.k1);
    uint4 c = make_uint4(static_cast<unsigned>(b0 >> 32) ^ h.y1, static_cast<unsigned>(b0), h.z2 ^ static_cast<unsigned>(a0), h.w2);
#pragma unroll
    for (int round = 2; round < 10; ++round) {
        const unsigned long long a = wide(0xD2511F53u, c.x), b = wide(0xCD9E8D57u, c.z);
        c = make_uint4(static_cast<unsigned>(b >> 32) ^ c.y ^ k[round].x, static_cast<unsigned>(b),
                       static_cast<unsigned>(a >> 32) ^ c.w ^ k[round].y, static_cast<unsigned>(a));
    }
    return c;
}

// A dropped element does not enter the result at all (a select, not a product with 0), whatever it holds.
__device__ __forceinline__ float dropped(float x, float r, unsigned w, const DropoutArgs& a)
{
    return w >= a.threshold ? fmaf(x, a.scale, r) : r;
}

constexpr int kDropThreads = 256;

// A CTA handles a chunk of kDropThreads * kDropCols columns of 16 bytes, a thread kDropCols of them (4, which
// shares the head of the rounds and the addresses, where that leaves many chunks for every SM; else 1); the
// threads of a warp take neighbouring columns.  Whole chunks of 16-byte aligned buffers (VEC) go by vector
// accesses without bounds checks, the last chunk and unaligned buffers element by element; the counters
// are the same.
template <typename T, int kDropCols, bool VEC, bool RESIDUAL>
__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const __grid_constant__ DropoutArgs a)
{
    stream_order();
    constexpr int VE = 16 / static_cast<int>(sizeof(T));
    constexpr int kChunk = kDropThreads * kDropCols * VE;
    const int m = blockIdx.y;
    const long long begin = static_cast<long long>(blockIdx.x) * kChunk;
    const T* x = static_cast<const T*>(a.x.p[m]) + begin;
    const T* r = RESIDUAL ? static_cast<const T*>(a.r.p[m]) + begin : nullptr;
    T* y = static_cast<T*>(a.y.p[m]) + begin;
    const unsigned long long o = a.offset + (a.counter ? *a.counter : 0ull), block = static_cast<unsigned long long>(begin) / 4;
    const PhiloxHead head = philox_head(static_cast<unsigned>(block >> 32) + (static_cast<unsigned>(m) << 24), static_cast<unsigned>(o),
                                        static_cast<unsigned>(o >> 32), a.keys);
    const unsigned low = static_cast<unsigned>(block);

    if (VEC && begin + kChunk <= a.n) {
        uint4 xw[kDropCols], rw[kDropCols];
#pragma unroll
        for (int c = 0; c < kDropCols; ++c) {                 // all loads first
            const unsigned at = threadIdx.x + c * kDropThreads;
            xw[c] = reinterpret_cast<const uint4*>(x)[at];
            if (RESIDUAL) rw[c] = reinterpret_cast<const uint4*>(r)[at];
        }
#pragma unroll
        for (int c = 0; c < kDropCols; ++c) {
            const unsigned at = threadIdx.x + c * kDropThreads;
            float f[VE], g[VE] = {};
            unpack<T>(xw[c], f);
            if (RESIDUAL) unpack<T>(rw[c], g);
#pragma unroll
            for (int q = 0; q < VE / 4; ++q) {
                const uint4 w = philox(low + at * (VE / 4) + q, head, a.keys);
                f[4 * q] = dropped(f[4 * q], g[4 * q], w.x, a);
                f[4 * q + 1] = dropped(f[4 * q + 1], g[4 * q + 1], w.y, a);
                f[4 * q + 2] = dropped(f[4 * q + 2], g[4 * q + 2], w.z, a);
                f[4 * q + 3] = dropped(f[4 * q + 3], g[4 * q + 3], w.w, a);
            }
            reinterpret_cast<uint4*>(y)[at] = pack<T>(f);
        }
    } else {
        // A thread computes the words of a block of four elements; through shared memory they reach the lanes that
        // hold the elements, which are neighbours of their neighbours'.
        __shared__ uint4 words[kDropThreads / 32][32];
        const int n = static_cast<int>(min(a.n - begin, static_cast<long long>(kChunk)));
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        constexpr int kGroups = kChunk / (kDropThreads * 4), kBatch = kGroups < 4 ? kGroups : 4;   // of 128 elements, a warp's
        for (int g = 0; g < kGroups; g += kBatch) {
            const int first = (warp * kGroups + g) * 128;
            if (first >= n) break;
            T xe[kBatch * 4], re[kBatch * 4];
#pragma unroll
            for (int e = 0; e < kBatch * 4; ++e) {            // all loads of the batch first
                const int j = first + e * 32 + lane;
                if (j < n) {
                    xe[e] = x[j];
                    if (RESIDUAL) re[e] = r[j];
                }
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                __syncwarp();
                words[warp][lane] = philox(low + (first + b * 128) / 4 + lane, head, a.keys);
                __syncwarp();
                const unsigned* w = reinterpret_cast<const unsigned*>(words[warp]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = first + b * 128 + e * 32 + lane;
                    if (j < n) y[j] = narrow<T>(dropped(widen(xe[b * 4 + e]), RESIDUAL ? widen(re[b * 4 + e]) : 0.0f, w[e * 32 + lane], a));
                }
            }
        }
    }
}

}  // namespace replica
}  // namespace grawa

// The gated feed-forward product of all M workers on the tensor cores, and its gradients.
//
//   forward   a = x Wg^T, u = x Wu^T, h = act(a) u                      (one kernel)
//   backward  da = dh u act'(a), du = dh act(a)                          (one elementwise kernel)
//             dx = da Wg + du Wu                                         (one product over both halves)
//             dWg = da^T x, dWu = du^T x                                 (one launch)
//
// All three products run in gemm_kernel: a persistent CTA per SM walks over 128 x 256 tiles; one thread
// fetches operand tiles by TMA into a ring of shared-memory stages, one thread issues tcgen05.mma, four
// warps bring finished accumulators from tensor memory to global memory while the next tile is computed
// (two accumulators of 256 columns take turns).  The forward tile holds 128 columns of a beside the same
// 128 columns of u, so the activation and the product are taken in the epilogue.
//
// Operands are read in the order in which they stand: rows whose products run along the contiguous index
// are "K-major" tiles, the others (weights in dx, both operands in dW) "MN-major" tiles of 64 contiguous
// elements by 64 rows; nothing is transposed in memory.  Elements outside a matrix are filled with zeros
// by TMA.  Accumulation is fp32; da and du are rounded to the storage type once, because the tensor cores
// take 16-bit operands (their rounding errors are independent and average out over the sums).
//
// Every wait is bounded: a CTA whose wait runs out records it in g_ffn_status, waits (bounded) for its own
// copies and products in flight, frees its tensor memory and returns.
#pragma once
#include <cuda.h>

#include "replica_common.cuh"

namespace grawa {
namespace replica {

enum Activation { kSilu = 0, kGelu = 1, kRelu = 2 };
enum GemmMode { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };

constexpr int kGemmWorkers = 16;            // workers a launch (their tensor maps travel as kernel parameters)
constexpr int kTileM = 128, kTileN = 256, kTileK = 64;
constexpr int kStages = 4;
constexpr int kABytes = kTileM * kTileK * 2, kBBytes = kTileN * kTileK * 2;
constexpr int kStageBytes = kABytes + kBBytes;
constexpr int kGemmSmem = kStages * kStageBytes + 1024;     // 1024: the swizzle pattern wants aligned stages
constexpr int kGemmThreads = 192;           // warp 0: copies, warp 1: products, warps 2..5: results
constexpr int kTileGroup = 16;              // tiles along M that are walked through together, for L2

struct GemmArgs {
    // kForward: per = x, Wg, Wu.  kInputGrad: common = da, du of all workers, per = Wg, Wu.
    // kWeightGrad: common = da, du, per = x.
    CUtensorMap common[2];
    CUtensorMap per[3][kGemmWorkers];
    void* out[3][kGemmWorkers];             // kForward: h, a, u (a and u may be NULL).  kInputGrad: dx.  kWeightGrad: dWg, dWu.
    int workers, first_worker;
    int m_tiles, n_tiles, k_blocks;         // k_blocks: of one half
    int rows, cols;                         // of an output
    int activation, accumulate, words;      // words: outputs take 16-byte stores
};

__device__ int g_ffn_status = 0;            // 1: a wait ran out since the word was read
constexpr unsigned long long kGemmWaitLimitNs = 2000000000ull;

// ------------------------------------------------------------------ barriers, copies, tensor memory

__device__ __forceinline__ unsigned smem_address(const void* p) { return static_cast<unsigned>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ unsigned long long nanoseconds()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void barrier_init(unsigned bar, unsigned count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(unsigned bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void barrier_expect(unsigned bar, unsigned bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(unsigned bar, unsigned parity)
{
    unsigned ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// False when the limit passed, or another wait of the CTA gave up (`gave_up`, which may be NULL).
__device__ __forceinline__ bool barrier_wait(unsigned bar, unsigned parity, volatile int* gave_up)
{
    if (barrier_try(bar, parity)) return true;
    const unsigned long long t0 = nanoseconds();
    for (;;) {
        if (barrier_try(bar, parity)) return true;
        if (gave_up && *gave_up) return false;
        if (nanoseconds() - t0 > kGemmWaitLimitNs) {
            if (gave_up) *gave_up = 1;
            atomicOr(&g_ffn_status, 1);
            return false;
        }
    }
}
__device__ __forceinline__ void copy_2d(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
                 "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void copy_3d(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map),
                 "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
// A 16 x 16-bit step of the product: D (+)= A B^T, both operands in shared memory, D in tensor memory.
__device__ __forceinline__ void mma_step(unsigned d, unsigned long long a, unsigned long long b, unsigned shape, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(shape), "r"(add ? 1u : 0u)
        : "memory");
}
// The barrier completes when every product this thread has issued so far is done.
__device__ __forceinline__ void mma_commit(unsigned bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 columns of this warp's 32 lanes: a thread gets one row's 32 neighbouring values, which may be used after
// accumulator_wait (the values pass through it, so that no use can move in front of it).
__device__ __forceinline__ void accumulator_load(unsigned address, unsigned (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
          "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
          "=r"(r[30]), "=r"(r[31])
        : "r"(address));
}
__device__ __forceinline__ void accumulator_wait(unsigned (&r)[32], float (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]),
                   "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                   "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void order_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void order_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory matrix descriptor, 128-byte swizzle.  K-major: groups of 8 rows 1024 bytes apart.
// MN-major: blocks of 64 elements `lead` bytes apart, groups of 8 k 1024 bytes apart.
__device__ __forceinline__ unsigned long long matrix_descriptor(unsigned address, unsigned lead)
{
    return static_cast<unsigned long long>((address & 0x3ffff) >> 4) | static_cast<unsigned long long>(lead >> 4) << 16 |
           static_cast<unsigned long long>(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
template <typename T> struct TypeCode;      // of both operands, in the instruction descriptor
template <> struct TypeCode<__half> { static constexpr unsigned value = 0; };
template <> struct TypeCode<__nv_bfloat16> { static constexpr unsigned value = 1; };

// ------------------------------------------------------------------ activation

__device__ __forceinline__ float activation(int kind, float a)
{
    if (kind == kSilu) return __fdividef(a, 1.0f + __expf(-a));
    if (kind == kGelu) return 0.5f * a * (1.0f + erff(a * 0.70710678118654752f));
    return a <= 0.0f ? 0.0f : a;
}
// Value and slope.
__device__ __forceinline__ float2 activation_slope(int kind, float a)
{
    if (kind == kSilu) {
        const float s = __fdividef(1.0f, 1.0f + __expf(-a));
        return make_float2(a * s, s * (1.0f + a * (1.0f - s)));
    }
    if (kind == kGelu) {
        const float c = 0.5f * (1.0f + erff(a * 0.70710678118654752f));
        return make_float2(a * c, fmaf(a * 0.39894228040143268f, __expf(-0.5f * a * a), c));
    }
    return make_float2(a <= 0.0f ? 0.0f : a, a > 0.0f ? 1.0f : 0.0f);
}

// ------------------------------------------------------------------ the product

struct Tile { int worker, half, m, n; };

// Tiles of one worker and half stand together; inside, kTileGroup tiles along M are walked through before
// the next one along N, so that the operands of the tiles in flight stay in L2.
template <int MODE>
__device__ __forceinline__ Tile tile_of(const GemmArgs& a, int t)
{
    const int per = a.m_tiles * a.n_tiles, whole = t / per, in = t % per;
    Tile r;
    r.worker = MODE == kWeightGrad ? whole / 2 : whole;
    r.half = MODE == kWeightGrad ? whole % 2 : 0;
    const int group = in / (kTileGroup * a.n_tiles), first = group * kTileGroup, high = min(kTileGroup, a.m_tiles - first);
    const int at = in - group * kTileGroup * a.n_tiles;
    r.m = first + at % high;
    r.n = at / high;
    return r;
}

// 32 neighbouring results of one row, columns [col, col + 32).
template <typename T>
__device__ __forceinline__ void store_results(const GemmArgs& a, void* base, int row, int col, float (&v)[32], bool add)
{
    T* out = static_cast<T*>(base) + static_cast<size_t>(row) * a.cols + col;
    if (a.words) {                                            // a.cols is a multiple of 8
        uint4* o = reinterpret_cast<uint4*>(out);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (col + 8 * q >= a.cols) break;
            if (add) {
                float held[8];
                unpack<T, 8>(o[q], held);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[8 * q + e] += held[e];
            }
            o[q] = pack<T, 8>(v + 8 * q);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 32; ++e)
            if (col + e < a.cols) out[e] = narrow<T>(add ? widen(out[e]) + v[e] : v[e]);
    }
}

template <typename T, int MODE>
__global__ void __launch_bounds__(kGemmThreads, 1)
gemm_kernel(const __grid_constant__ GemmArgs a)
{
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kStages + 5];
    __shared__ unsigned tmem_slot;
    __shared__ int gave_up;

    const unsigned ring = (smem_address(raw) + 1023u) & ~1023u;
    const unsigned full = smem_address(bars), empty = full + 8 * kStages, done = empty + 8 * kStages, ready = done + 16, drain = ready + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int halves = MODE == kInputGrad ? 2 : 1;            // products that add up in one accumulator
    const int blocks = a.k_blocks * halves;
    const int tiles = a.workers * (MODE == kWeightGrad ? 2 : 1) * a.m_tiles * a.n_tiles;

    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int s = 0; s < kStages; ++s) { barrier_init(full + 8 * s, 1); barrier_init(empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { barrier_init(done + 8 * s, 1); barrier_init(ready + 8 * s, 4); }   // ready: one arrival a warp
        barrier_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {                                          // all 512 columns: two accumulators of 256
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_address(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    order_before();
    __syncthreads();
    order_after();
    const unsigned tmem = tmem_slot;

    if (warp == 0 && lane == 0) {
        int fills = 0;
        bool ok = true;
        for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
            const Tile tile = tile_of<MODE>(a, t);
            const int m0 = tile.m * kTileM, n0 = tile.n * (MODE == kForward ? kTileN / 2 : kTileN);
            for (int kb = 0; kb < blocks; ++kb, ++fills) {
                const int s = fills % kStages;
                if (fills >= kStages && !barrier_wait(empty + 8 * s, (fills / kStages - 1) & 1, &gave_up)) { ok = false; break; }
                const unsigned bar = full + 8 * s, sa = ring + s * kStageBytes, sb = sa + kABytes;
                const int half = MODE == kInputGrad ? kb / a.k_blocks : tile.half;
                const int k0 = (MODE == kInputGrad ? kb % a.k_blocks : kb) * kTileK;
                barrier_expect(bar, kStageBytes);
                if (MODE == kForward) {
                    copy_2d(sa, &a.per[0][tile.worker], k0, m0, bar);
                    copy_2d(sb, &a.per[1][tile.worker], k0, n0, bar);
                    copy_2d(sb + kBBytes / 2, &a.per[2][tile.worker], k0, n0, bar);
                } else if (MODE == kInputGrad) {
                    copy_3d(sa, &a.common[half], k0, m0, a.first_worker + tile.worker, bar);
#pragma unroll
                    for (int i = 0; i < kTileN / 64; ++i) copy_2d(sb + i * 8192, &a.per[half][tile.worker], n0 + 64 * i, k0, bar);
                } else {
#pragma unroll
                    for (int i = 0; i < kTileM / 64; ++i) copy_3d(sa + i * 8192, &a.common[half], m0 + 64 * i, k0, a.first_worker + tile.worker, bar);
#pragma unroll
                    for (int i = 0; i < kTileN / 64; ++i) copy_2d(sb + i * 8192, &a.per[0][tile.worker], n0 + 64 * i, k0, bar);
                }
            }
        }
        if (!ok)                                              // copies in flight still write shared memory
            for (int f = max(0, fills - kStages); f < fills; ++f) barrier_wait(full + 8 * (f % kStages), (f / kStages) & 1, nullptr);
    } else if (warp == 1 && lane == 0) {
        constexpr bool kAMn = MODE == kWeightGrad, kBMn = MODE != kForward;
        constexpr unsigned shape = 1u << 4 | TypeCode<T>::value << 7 | TypeCode<T>::value << 10 | (kAMn ? 1u : 0u) << 15 | (kBMn ? 1u : 0u) << 16 |
                                   (kTileN >> 3) << 17 | (kTileM >> 4) << 24;
        constexpr unsigned a_step = (kAMn ? 2048 : 32) >> 4, b_step = (kBMn ? 2048 : 32) >> 4;   // 16 k further
        int used = 0, turn = 0;
        bool ok = true;
        for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x, ++turn) {
            const unsigned d = tmem + (turn & 1) * kTileN;
            if (turn >= 2 && !barrier_wait(ready + 8 * (turn & 1), (turn / 2 - 1) & 1, &gave_up)) { ok = false; break; }
            order_after();
            for (int kb = 0; kb < blocks; ++kb, ++used) {
                const int s = used % kStages;
                if (!barrier_wait(full + 8 * s, (used / kStages) & 1, &gave_up)) { ok = false; break; }
                order_after();
                const unsigned sa = ring + s * kStageBytes, sb = sa + kABytes;
                const unsigned long long da = matrix_descriptor(sa, kAMn ? 8192 : 16), db = matrix_descriptor(sb, kBMn ? 8192 : 16);
#pragma unroll
                for (int k = 0; k < kTileK / 16; ++k) mma_step(d, da + k * a_step, db + k * b_step, shape, kb > 0 || k > 0);
                mma_commit(empty + 8 * s);
            }
            if (ok) mma_commit(done + 8 * (turn & 1));
        }
        if (!ok) {
            mma_commit(drain);
            barrier_wait(drain, 0, nullptr);
        }
    } else if (warp >= 2) {
        const int quarter = warp & 3;                         // the lanes of tensor memory that this warp may read
        int turn = 0;
        for (int t = blockIdx.x; t < tiles; t += gridDim.x, ++turn) {
            const Tile tile = tile_of<MODE>(a, t);
            if (!barrier_wait(done + 8 * (turn & 1), (turn / 2) & 1, &gave_up)) break;
            __syncwarp();
            order_after();
            const unsigned d = tmem + (turn & 1) * kTileN + (static_cast<unsigned>(quarter * 32) << 16);
            const int row = tile.m * kTileM + quarter * 32 + lane;
            if (MODE == kForward) {
                const int n0 = tile.n * (kTileN / 2);
#pragma unroll 1
                for (int c = 0; c < kTileN / 2 && n0 + c < a.cols; c += 32) {
                    unsigned gr[32], ur[32];
                    float g[32], u[32];
                    accumulator_load(d + c, gr);
                    accumulator_load(d + kTileN / 2 + c, ur);
                    accumulator_wait(gr, g);
                    accumulator_wait(ur, u);
                    if (row < a.rows) {
                        if (a.out[1][tile.worker]) {
                            store_results<T>(a, a.out[1][tile.worker], row, n0 + c, g, false);
                            store_results<T>(a, a.out[2][tile.worker], row, n0 + c, u, false);
                        }
#pragma unroll
                        for (int e = 0; e < 32; ++e) g[e] = activation(a.activation, g[e]) * u[e];
                        store_results<T>(a, a.out[0][tile.worker], row, n0 + c, g, false);
                    }
                    __syncwarp();
                }
            } else {
                const int n0 = tile.n * kTileN;
#pragma unroll 1
                for (int c = 0; c < kTileN && n0 + c < a.cols; c += 32) {
                    unsigned r[32];
                    float v[32];
                    accumulator_load(d + c, r);
                    accumulator_wait(r, v);
                    if (row < a.rows) store_results<T>(a, a.out[tile.half][tile.worker], row, n0 + c, v, a.accumulate != 0);
                    __syncwarp();
                }
            }
            order_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(ready + 8 * (turn & 1));
        }
    }
    __syncwarp();
    order_before();
    __syncthreads();
    order_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// ------------------------------------------------------------------ elementwise parts

struct GatedGradArgs {
    In dh, gate, up;
    void *da, *du;                         // [M][rows][pitch]
    long long rows;
    int cols, pitch, activation, words;
};

constexpr int kGatedThreads = 256;

// da = dh u act'(a), du = dh act(a): bound by memory, 5 elements of traffic an element.  A thread handles 8
// neighbouring elements of a row.
template <typename T>
__global__ void __launch_bounds__(kGatedThreads)
gated_grad_kernel(const __grid_constant__ GatedGradArgs a)
{
    const int m = blockIdx.y, per_row = a.pitch / 8;
    const long long at = static_cast<long long>(blockIdx.x) * kGatedThreads + threadIdx.x;
    if (at >= a.rows * per_row) return;
    const long long row = at / per_row;
    const int col = static_cast<int>(at % per_row) * 8;
    const long long in = row * a.cols + col;
    const T* dh = static_cast<const T*>(a.dh.p[m]) + in;
    const T* gate = static_cast<const T*>(a.gate.p[m]) + in;
    const T* up = static_cast<const T*>(a.up.p[m]) + in;
    float d[8] = {}, g[8] = {}, u[8] = {};
    if (a.words) {
        unpack<T, 8>(*reinterpret_cast<const uint4*>(dh), d);
        unpack<T, 8>(*reinterpret_cast<const uint4*>(gate), g);
        unpack<T, 8>(*reinterpret_cast<const uint4*>(up), u);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + e < a.cols) { d[e] = widen(dh[e]); g[e] = widen(gate[e]); u[e] = widen(up[e]); }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 f = activation_slope(a.activation, g[e]);
        u[e] = d[e] * u[e] * f.y;
        g[e] = d[e] * f.x;
    }
    const size_t out = (static_cast<size_t>(m) * a.rows + row) * a.pitch + col;
    *reinterpret_cast<uint4*>(static_cast<T*>(a.da) + out) = pack<T, 8>(u);
    *reinterpret_cast<uint4*>(static_cast<T*>(a.du) + out) = pack<T, 8>(g);
}

struct PackArgs {
    In from;
    unsigned short* to;                    // [M][rows][pitch]
    long long rows;
    int cols, pitch;
};

// Rows of 16-bit elements at any address, laid out again with 16-byte aligned rows, as TMA wants them.
static __global__ void __launch_bounds__(kGatedThreads)
pack_rows_kernel(const __grid_constant__ PackArgs a)
{
    const int m = blockIdx.y, per_row = a.pitch / 8;
    const long long at = static_cast<long long>(blockIdx.x) * kGatedThreads + threadIdx.x;
    if (at >= a.rows * per_row) return;
    const long long row = at / per_row;
    const int col = static_cast<int>(at % per_row) * 8;
    const unsigned short* from = static_cast<const unsigned short*>(a.from.p[m]) + row * a.cols + col;
    unsigned short v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = col + e < a.cols ? from[e] : static_cast<unsigned short>(0);
    *reinterpret_cast<uint4*>(a.to + (static_cast<size_t>(m) * a.rows + row) * a.pitch + col) =
        make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

}  // namespace replica
}  // namespace grawa

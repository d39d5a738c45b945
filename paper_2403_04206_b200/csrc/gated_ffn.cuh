// The gated feed-forward product of all M workers on the tensor cores, and its gradients.
//
//   forward   a = x Wg^T, u = x Wu^T, h = act(a) u                      (one kernel; two where the sum is split)
//   backward  da = dh u act'(a), du = dh act(a)                          (one elementwise kernel)
//             dx = da Wg + du Wu, dWg = da^T x, dWu = du^T x             (one kernel where their operands fit in L2
//                                                                         together, else two)
//
// All three products run in gemm_kernel: a persistent pair of CTAs (a cluster) per two SMs walks over 256 x 256
// tiles; each CTA holds 128 rows of A and 128 of the 256 columns of B, so a byte in shared memory feeds twice
// the products that it feeds in a single CTA (whose 128 x 256 tiles were bound by shared memory: tensor pipe 65
// to 76 % busy).  In each CTA one thread fetches operand tiles by TMA into a ring of shared-memory stages; one
// thread of the pair issues tcgen05.mma for both; eight warps of each bring finished accumulators from tensor
// memory to global memory while the next tile is computed (two accumulators of 256 columns take turns).  The
// forward tile holds 128 columns of a beside the same 128 columns of u, so the activation and the product are
// taken in the epilogue.
//
// Operands are read in the order in which they stand: rows whose products run along the contiguous index
// are "K-major" tiles, the others (weights in dx, both operands in dW) "MN-major" tiles of 64 contiguous
// elements by 64 rows; nothing is transposed in memory.  Elements outside a matrix are filled with zeros
// by TMA.  Accumulation is fp32; da and du are rounded to the storage type once, because the tensor cores
// take 16-bit operands (their rounding errors are independent and average out over the sums).
//
// Where a product has fewer tiles than there are pairs of SMs, its sum is split among them and the parts, in fp32,
// are added by a second kernel in a fixed order.
//
// Measured (B200), 4 workers x 4096 tokens, 2048 -> 5632, bf16: forward 590 to 635 us with a, u and h stored (1190 to 1280
// TFLOP/s; cuBLAS takes 570 to 605 for the two projections alone, under the same power limit); backward 1250 to 1400 us,
// of which 130 are the elementwise kernel at 7.1 TB/s and the products run at 1440 TFLOP/s until the power limit
// lowers the clock (cuBLAS 1170 to 1230 us for the products alone).
//
// Every wait for a barrier in shared memory is bounded: a CTA whose wait runs out counts it in g_ffn_timeouts, waits
// (bounded) for its own copies and products in flight, frees its tensor memory and returns.  A warp decides as one: its
// lanes leave together or go on together, as the instructions that take a whole warp need.  (Not bounded by the kernel: the
// two waits of the pair for each other, which both CTAs reach for that reason, and the allocation of tensor
// memory, which waits for whoever holds it on the SM to end.)
#pragma once
#include <cuda.h>

#include <type_traits>

#include "replica_common.cuh"

namespace grawa {
namespace replica {

enum Activation { kSilu = 0, kGelu = 1, kRelu = 2 };
enum GemmPartName { kInputGrad = 0, kWeightGrad = 1 };     // the two products of the backward pass

constexpr int kGemmWorkers = 16;            // workers a launch (their tensor maps travel as kernel parameters)
constexpr int kTileM = 256, kTileN = 256, kTileK = 64;      // of a pair
constexpr int kHalf = 128;                  // rows of A, and columns of B, that a CTA of the pair holds
constexpr int kStages = 6;
constexpr int kABytes = kHalf * kTileK * 2, kBBytes = kHalf * kTileK * 2;
constexpr int kStageBytes = kABytes + kBBytes;
constexpr int kGemmSmem = kStages * kStageBytes + 8 * 4096 + 1024;     // + results on their way out; the swizzle wants aligned stages
constexpr int kGemmThreads = 320;           // warp 0: copies, warp 1: products, warps 2..9: results
constexpr int kTileGroup = 8;               // tiles along M that are walked through together, for L2

// A product: its grid of tiles, and the split of its sum.  A unit of work is one part of one tile's sum.
struct GemmPart {
    float* partial;                         // splits > 1: [split][tile][256 columns][256 rows]
    int m_tiles, n_tiles, tiles, units;     // units = tiles * splits
    int half_blocks, blocks;                // steps of kTileK along the sum: of one half (dx adds two products), and of all
    int splits, split_blocks;               // parts of the sum, and steps of each
    int rows, cols, words;                  // of an output; words: outputs take 16-byte stores
};

struct GemmArgs {
    // forward: per = x, Wg, Wu.  Backward: common = da, du as dx takes them, then as the weights' gradients do, of
    // all workers; per = Wg, Wu, x.
    CUtensorMap common[4];
    CUtensorMap per[3][kGemmWorkers];
    void* out[3][kGemmWorkers];             // forward: h, a, u (a and u may be NULL).  Backward: dx, dWg, dWu.
    GemmPart part[2];                       // forward: one.  Backward: kInputGrad, kWeightGrad; without units where not wanted
    // Pair p of CTAs takes units p, p + pairs, ... of part `lead`, then the other part's units [share[p], share[p + 1]).
    int lead, share[kSms / 2 + 1];
    int workers, first_worker;
    int activation, accumulate;
};

__device__ unsigned g_ffn_timeouts = 0;     // waits that ran out, never set back: no report can be lost between two readers
constexpr unsigned long long kGemmWaitLimitNs = 2000000000ull, kStarvedLimitNs = 2000000ull;

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
// The same place of shared memory in the first CTA of the pair.
__device__ __forceinline__ unsigned in_leader(unsigned address)
{
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(address));
    return r;
}
// Arrival at a barrier of either CTA of the pair.
__device__ __forceinline__ void barrier_arrive(unsigned cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
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
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// False when the limit passed, or another wait of the CTA gave up (`gave_up`, which may be NULL).  Lanes of a warp may get
// different answers.
template <unsigned long long LIMIT>
__device__ __forceinline__ bool barrier_wait(unsigned bar, unsigned parity, volatile int* gave_up)
{
    if (barrier_try(bar, parity)) return true;
    const unsigned long long t0 = nanoseconds();
    for (;;) {
        if (barrier_try(bar, parity)) return true;
        if (gave_up && *gave_up) return false;
        if (nanoseconds() - t0 > LIMIT) {
            if (gave_up) *gave_up = 1;
            atomicAdd(&g_ffn_timeouts, 1u);
            return false;
        }
    }
}
// Copies into this CTA's shared memory that complete on a barrier of the pair's first CTA.
__device__ __forceinline__ void copy_2d(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
                 "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void copy_3d(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map),
                 "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
// A step of 16 along the sum: D (+)= A B^T, each CTA's halves of both operands in its shared memory, its rows
// of D in its tensor memory.
__device__ __forceinline__ void mma_step(unsigned d, unsigned long long a, unsigned long long b, unsigned shape, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(shape), "r"(add ? 1u : 0u)
        : "memory");
}
// Arrives at this barrier in both CTAs when every product this thread has issued so far is done.
__device__ __forceinline__ void mma_commit(unsigned bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"(static_cast<unsigned short>(3))
                 : "memory");
}
// The same in this CTA alone, for a thread that gives up: its pair's other CTA waits for nothing more.
__device__ __forceinline__ void mma_commit_here(unsigned bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 16 columns of this warp's 32 lanes: a thread gets one row's 16 neighbouring values, which may be used after
// accumulator_wait (the values pass through it, so that no use can move in front of it).
__device__ __forceinline__ void accumulator_load(unsigned address, unsigned (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(address));
}
__device__ __forceinline__ void accumulator_wait(unsigned (&r)[16], float (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                   "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :
                 : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
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

// The normal distribution's cdf and density at a.  The tail behind |a| is exp(-a^2 / 2) times a function that falls slowly
// (half the scaled complementary error function at |a| / sqrt 2), here t (c0 + ... + c7 t^7) with t = 1 / (1 + 0.234 |a|):
// coefficients fitted for this file, by weighted least squares with the weights moved to the largest RELATIVE errors
// until those were level, 9.3e-8 for |a| up to 14.5 (behind that the tail is below the smallest normal float), 4.6e-7 with the
// roundings.  So the tail keeps its digits, and small values at large negative a come without cancellation; what remains is the
// exponential's error, which grows with its argument (2e-5 at a = -12).  It shares the exponential with the
// density.  (With the library's erf the elementwise kernel was bound by instructions: 3.2 million elements in
// each of 2 workers, 18.6 us.)
__device__ __forceinline__ float2 normal_distribution(float a)
{
    const float t = __fdividef(1.0f, fmaf(0.234f, fabsf(a), 1.0f)), e = __expf(-0.5f * a * a);
    float q = fmaf(t, -0.06640374660491943f, 0.222660094499588f);
    q = fmaf(t, q, -0.16444748640060425f);
    q = fmaf(t, q, 0.19517424702644348f);
    q = fmaf(t, q, 0.028018606826663017f);
    q = fmaf(t, q, 0.09965468943119049f);
    q = fmaf(t, q, 0.09191432595252991f);
    q = fmaf(t, q, 0.09342921525239944f);
    const float tail = t * q * e;
    return make_float2(a >= 0.0f ? 1.0f - tail : tail, 0.39894228040143268f * e);
}
// The logistic function at a, and at -a (1 minus it, without cancellation).  From exp(-|a|), so that the divisor stays
// between 1 and 2: with exp(-a) in it the quotient is 0 from a = -87.3 on, where it is still a normal number.
__device__ __forceinline__ float2 logistic(float a)
{
    const float e = __expf(-fabsf(a)), r = __fdividef(1.0f, 1.0f + e);
    return a >= 0.0f ? make_float2(r, e * r) : make_float2(e * r, r);
}
__device__ __forceinline__ float activation(int kind, float a)
{
    if (kind == kSilu) return a * logistic(a).x;
    if (kind == kGelu) return a * normal_distribution(a).x;
    return a <= 0.0f ? 0.0f : a;
}
// v <- act(v) u, the kind decided once for 16 values.
__device__ __forceinline__ void gated_product(int kind, float (&v)[16], const float (&u)[16])
{
    if (kind == kSilu) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = activation(kSilu, v[e]) * u[e];
    } else if (kind == kGelu) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = activation(kGelu, v[e]) * u[e];
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = activation(kRelu, v[e]) * u[e];
    }
}
// Value and slope.
__device__ __forceinline__ float2 activation_slope(int kind, float a)
{
    if (kind == kSilu) {
        const float2 s = logistic(a);
        return make_float2(a * s.x, s.x * fmaf(a, s.y, 1.0f));
    }
    if (kind == kGelu) {
        const float2 d = normal_distribution(a);
        return make_float2(a * d.x, fmaf(a, d.y, d.x));
    }
    return make_float2(a <= 0.0f ? 0.0f : a, a > 0.0f ? 1.0f : 0.0f);
}

// ------------------------------------------------------------------ the product

struct Unit { int part, slot, worker, half, m, n, begin, end; };   // slot: the unit's place in its part; [begin, end): steps of the sum

// Tiles of one worker and half stand together; inside, kTileGroup tiles along M are walked through before
// the next one along N, so that the operands of the tiles in flight stay in L2.
template <bool FORWARD>
__device__ __forceinline__ Unit unit_of(const GemmArgs& a, int part, int slot)
{
    const GemmPart& p = a.part[part];
    const int t = slot % p.tiles, per = p.m_tiles * p.n_tiles, whole = t / per, in = t % per, halves = !FORWARD && part == kWeightGrad ? 2 : 1;
    Unit u;
    u.part = part;
    u.slot = slot;
    u.worker = whole / halves;
    u.half = whole % halves;
    const int group = in / (kTileGroup * p.n_tiles), first = group * kTileGroup, high = min(kTileGroup, p.m_tiles - first);
    const int at = in - group * kTileGroup * p.n_tiles;
    u.m = first + at % high;
    u.n = at / high;
    u.begin = slot / p.tiles * p.split_blocks;
    u.end = min(p.blocks, u.begin + p.split_blocks);
    return u;
}
// The pair's unit number `turn`; false when it has no more.
template <bool FORWARD>
__device__ __forceinline__ bool next_unit(const GemmArgs& a, int turn, Unit& u)
{
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2, units = a.part[a.lead].units, own = units > pair ? (units - pair + pairs - 1) / pairs : 0;
    if (turn < own) {
        u = unit_of<FORWARD>(a, a.lead, pair + turn * pairs);
        return true;
    }
    if (FORWARD) return false;
    const int slot = a.share[pair] + turn - own;
    if (slot >= a.share[pair + 1]) return false;
    u = unit_of<FORWARD>(a, 1 - a.lead, slot);
    return true;
}

// Results go to memory by way of a warp's own 4 KB of shared memory, 32 rows by 64 columns of 16 bits: a thread
// has a row of the accumulator, but whole 128-byte rows are what global memory takes well.  The 16-byte pieces
// of a row are permuted so that neither direction meets bank conflicts.  The loops over an accumulator's columns
// stay rolled, 16 columns a turn: two warps an SM quarter cannot hide the instruction fetches of code that runs
// once (unrolled over 64 columns, a forward tile's results took 22 thousand cycles, longer than its products).
constexpr int kStoreCols = 64;
constexpr int kStoreBytes = 32 * kStoreCols * 2;

__device__ __forceinline__ uint4* store_slot(unsigned char* stage, int row, int piece)
{
    return reinterpret_cast<uint4*>(stage + row * 128 + ((piece ^ (row & 7)) * 16));
}

// Outputs that do not take 16-byte accesses: pairs of elements where they stand on 4-byte boundaries, else single ones,
// neighbouring lanes at neighbouring columns, 8 rows under way at a time.  STEP: 16-bit elements of an access.
template <typename W, int STEP, bool TO_MEMORY>
__device__ __noinline__ void move_elements(unsigned char* stage, unsigned short* out, int rows, int cols, int pitch)
{
    const int lane = threadIdx.x & 31;
    for (int c = lane * STEP; c < cols; c += 32 * STEP)
        for (int r0 = 0; r0 < rows; r0 += 8) {
            W v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = r0 + i;
                if (r >= rows) continue;
                if (TO_MEMORY) v[i] = *reinterpret_cast<const W*>(reinterpret_cast<const unsigned short*>(store_slot(stage, r, c / 8)) + c % 8);
                else v[i] = *reinterpret_cast<const W*>(out + static_cast<size_t>(r) * pitch + c);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = r0 + i;
                if (r >= rows) continue;
                if (TO_MEMORY) *reinterpret_cast<W*>(out + static_cast<size_t>(r) * pitch + c) = v[i];
                else *reinterpret_cast<W*>(reinterpret_cast<unsigned short*>(store_slot(stage, r, c / 8)) + c % 8) = v[i];
            }
        }
}

// Between the stage and rows [row, row + 32), columns [col, col + 64) of an output, inside its edges.
template <typename T, bool TO_MEMORY>
__device__ __forceinline__ void move_stage(const GemmPart& a, unsigned char* stage, void* base, int row, int col)
{
    const int lane = threadIdx.x & 31;
    T* out = static_cast<T*>(base) + static_cast<size_t>(row) * a.cols + col;
    __syncwarp();
    if (a.words) {                                            // a.cols is a multiple of 8
        const int piece = lane % 8, first = lane / 8;
        if (col + piece * 8 < a.cols) {
            uint4* at = reinterpret_cast<uint4*>(out + static_cast<size_t>(first) * a.cols + piece * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i, at += a.cols / 2) {   // 4 rows further
                if (row + first + 4 * i >= a.rows) break;
                if (TO_MEMORY) *at = *store_slot(stage, first + 4 * i, piece);
                else *store_slot(stage, first + 4 * i, piece) = *at;
            }
        }
    } else {
        unsigned short* at = reinterpret_cast<unsigned short*>(out);
        const int rows = min(32, a.rows - row), cols = min(kStoreCols, a.cols - col);
        if (a.cols % 2 == 0 && reinterpret_cast<uintptr_t>(at) % 4 == 0) move_elements<unsigned, 2, TO_MEMORY>(stage, at, rows, cols, a.cols);
        else move_elements<unsigned short, 1, TO_MEMORY>(stage, at, rows, cols, a.cols);
    }
    __syncwarp();
}

// STARVED: for the self-test of the bounded waits only; nothing is copied, so that the first wait for operands runs out.
template <typename T, bool FORWARD, bool STARVED = false>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kGemmThreads, 1)
gemm_kernel(const __grid_constant__ GemmArgs a)
{
    constexpr unsigned long long kLimit = STARVED ? kStarvedLimitNs : kGemmWaitLimitNs;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kStages + 5];
    __shared__ unsigned tmem_slot;
    __shared__ int gave_up;

    // full and ready are used in the pair's first CTA only, empty, done and drain in each
    const unsigned ring = (smem_address(raw) + 1023u) & ~1023u;
    const unsigned full = smem_address(bars), empty = full + 8 * kStages, done = empty + 8 * kStages, ready = done + 16, drain = ready + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = blockIdx.x & 1;

    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int s = 0; s < kStages; ++s) { barrier_init(full + 8 * s, 1); barrier_init(empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { barrier_init(done + 8 * s, 1); barrier_init(ready + 8 * s, 16); }  // ready: one arrival a warp of the pair
        barrier_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {                                          // all 512 columns of both: two accumulators of 256
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_address(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    order_before();
    __syncthreads();
    pair_sync();                                              // both CTAs' barriers are ready before either is used
    order_after();
    stream_order();                                           // (what is above touches no operand)
    const unsigned tmem = tmem_slot;

    Unit u;
    if (!STARVED && warp == 0 && lane == 0) {
        const unsigned leader_full = in_leader(full);
        int fills = 0;
        bool ok = true;
        for (int turn = 0; ok && next_unit<FORWARD>(a, turn, u); ++turn) {
            const int m0 = u.m * kTileM + rank * kHalf;
            const int n0 = FORWARD ? u.n * kHalf : u.n * kTileN + rank * kHalf;
            const int half_blocks = a.part[u.part].half_blocks;
            for (int kb = u.begin; kb < u.end; ++kb, ++fills) {
                const int s = fills % kStages;
                if (fills >= kStages && !barrier_wait<kLimit>(empty + 8 * s, (fills / kStages - 1) & 1, &gave_up)) { ok = false; break; }
                const unsigned bar = leader_full + 8 * s, sa = ring + s * kStageBytes, sb = sa + kABytes;
                if (rank == 0) barrier_expect(full + 8 * s, 2 * kStageBytes);           // the bytes of both CTAs
                if (FORWARD) {
                    copy_2d(sa, &a.per[0][u.worker], kb * kTileK, m0, bar);
                    copy_2d(sb, &a.per[1 + rank][u.worker], kb * kTileK, n0, bar);      // a's columns in one CTA, u's in the other
                } else if (u.part == kInputGrad) {
                    const int half = kb >= half_blocks, k0 = (kb - half * half_blocks) * kTileK;
                    copy_3d(sa, &a.common[half], k0, m0, a.first_worker + u.worker, bar);
#pragma unroll
                    for (int i = 0; i < kHalf / 64; ++i) copy_2d(sb + i * 8192, &a.per[half][u.worker], n0 + 64 * i, k0, bar);
                } else {
#pragma unroll
                    for (int i = 0; i < kHalf / 64; ++i) copy_3d(sa + i * 8192, &a.common[2 + u.half], m0 + 64 * i, kb * kTileK, a.first_worker + u.worker, bar);
#pragma unroll
                    for (int i = 0; i < kHalf / 64; ++i) copy_2d(sb + i * 8192, &a.per[2][u.worker], n0 + 64 * i, kb * kTileK, bar);
                }
            }
        }
        // The last arrivals at this CTA's barriers come before it leaves.
        if (ok)
            for (int f = max(0, fills - kStages); f < fills && ok; ++f) ok = barrier_wait<kLimit>(empty + 8 * (f % kStages), (f / kStages) & 1, &gave_up);
        // After a wait ran out, copies in flight still write shared memory: the first CTA sees those of both.
        if (!ok && rank == 0)
            for (int f = max(0, fills - kStages); f < fills; ++f) barrier_wait<kLimit>(full + 8 * (f % kStages), (f / kStages) & 1, nullptr);
    } else if (warp == 1 && lane == 0 && rank == 0) {
        constexpr unsigned kShape = 1u << 4 | TypeCode<T>::value << 7 | TypeCode<T>::value << 10 | (kTileN >> 3) << 17 | (kTileM >> 4) << 24;
        constexpr unsigned kAMn = 1u << 15, kBMn = 1u << 16, kAlongK = 32 >> 4, kAlongMn = 2048 >> 4;   // 16 k further in a K- or an MN-major tile
        int used = 0;
        bool ok = true;
        for (int turn = 0; ok && next_unit<FORWARD>(a, turn, u); ++turn) {
            const bool a_mn = !FORWARD && u.part == kWeightGrad, b_mn = !FORWARD;
            const unsigned shape = kShape | (a_mn ? kAMn : 0u) | (b_mn ? kBMn : 0u), a_step = a_mn ? kAlongMn : kAlongK, b_step = b_mn ? kAlongMn : kAlongK;
            const unsigned d = tmem + (turn & 1) * kTileN;
            if (turn >= 2 && !barrier_wait<kLimit>(ready + 8 * (turn & 1), (turn / 2 - 1) & 1, &gave_up)) { ok = false; break; }
            order_after();
            for (int kb = u.begin; kb < u.end; ++kb, ++used) {
                const int s = used % kStages;
                if (!barrier_wait<kLimit>(full + 8 * s, (used / kStages) & 1, &gave_up)) { ok = false; break; }
                order_after();
                const unsigned sa = ring + s * kStageBytes, sb = sa + kABytes;
                const unsigned long long da = matrix_descriptor(sa, a_mn ? 8192 : 16), db = matrix_descriptor(sb, b_mn ? 8192 : 16);
#pragma unroll
                for (int k = 0; k < kTileK / 16; ++k) mma_step(d, da + k * a_step, db + k * b_step, shape, kb > u.begin || k > 0);
                mma_commit(empty + 8 * s);
            }
            if (ok) mma_commit(done + 8 * (turn & 1));
        }
        if (!ok) {
            mma_commit_here(drain);
            barrier_wait<kLimit>(drain, 0, nullptr);
        }
    } else if (warp >= 2) {
        const int quarter = warp & 3;                         // the lanes of tensor memory that this warp may read
        const int half = (warp - 2) / 4;                      // its half of the columns
        const unsigned leader_ready = in_leader(ready);
        unsigned char* stage = raw + (ring - smem_address(raw)) + kStages * kStageBytes + (warp - 2) * kStoreBytes;
        for (int turn = 0; next_unit<FORWARD>(a, turn, u); ++turn) {
            const GemmPart& p = a.part[u.part];
            if (!__all_sync(0xffffffffu, barrier_wait<kLimit>(done + 8 * (turn & 1), (turn / 2) & 1, &gave_up))) break;
            __syncwarp();
            order_after();
            const unsigned d = tmem + (turn & 1) * kTileN + (static_cast<unsigned>(quarter * 32) << 16);
            const int row = u.m * kTileM + rank * kHalf + quarter * 32;
            if (p.splits > 1) {                               // a part of the sum, as it stands: a warp's 32 rows side by side
                float* to = p.partial + static_cast<size_t>(u.slot) * kTileM * kTileN + rank * kHalf + quarter * 32 + lane;
#pragma unroll 1
                for (int c = half * kHalf; c < (half + 1) * kHalf && row < p.rows; c += 16) {
                    if ((FORWARD ? u.n * kHalf + c % kHalf : u.n * kTileN + c) >= p.cols) break;
                    unsigned r[16];
                    float v[16];
                    accumulator_load(d + c, r);
                    accumulator_wait(r, v);
#pragma unroll
                    for (int e = 0; e < 16; ++e) to[(c + e) * kTileM] = v[e];
                }
            } else if (FORWARD) {
                const int c = half * kStoreCols, col = u.n * kHalf + c;
#pragma unroll 1
                for (int out = 2; out >= 0; --out) {          // u, a, h
                    if (a.out[out][u.worker] == nullptr || row >= p.rows || col >= p.cols) continue;
#pragma unroll 1
                    for (int q = 0; q < kStoreCols / 8; q += 2) {
                        unsigned first[16], second[16];
                        float v[16], up[16];
                        accumulator_load(d + c + q * 8 + (out == 2 ? kHalf : 0), first);
                        if (out == 0) accumulator_load(d + c + q * 8 + kHalf, second);
                        accumulator_wait(first, v);
                        if (out == 0) {
                            accumulator_wait(second, up);
                            gated_product(a.activation, v, up);
                        }
                        *store_slot(stage, lane, q) = pack<T>(v);
                        *store_slot(stage, lane, q + 1) = pack<T>(v + 8);
                    }
                    move_stage<T, true>(p, stage, a.out[out][u.worker], row, col);
                }
            } else {
                void* out = a.out[u.part == kInputGrad ? 0 : 1 + u.half][u.worker];
                const bool add = u.part == kWeightGrad && a.accumulate;
#pragma unroll 1
                for (int c = half * kHalf; c < (half + 1) * kHalf; c += kStoreCols) {
                    const int col = u.n * kTileN + c;
                    if (row >= p.rows || col >= p.cols) break;
                    if (add) move_stage<T, false>(p, stage, out, row, col);
#pragma unroll 1
                    for (int q = 0; q < kStoreCols / 8; q += 2) {
                        unsigned r[16];
                        float v[16];
                        accumulator_load(d + c + q * 8, r);
                        accumulator_wait(r, v);
                        if (add) {
                            float held[16];
                            unpack<T>(*store_slot(stage, lane, q), held);
                            unpack<T>(*store_slot(stage, lane, q + 1), held + 8);
#pragma unroll
                            for (int e = 0; e < 16; ++e) v[e] += held[e];
                        }
                        *store_slot(stage, lane, q) = pack<T>(v);
                        *store_slot(stage, lane, q + 1) = pack<T>(v + 8);
                    }
                    move_stage<T, true>(p, stage, out, row, col);
                }
            }
            order_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(leader_ready + 8 * (turn & 1));
        }
    }
    __syncwarp();
    order_before();
    __syncthreads();
    pair_sync();                                              // neither CTA leaves while the other may reach into it
    order_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// The parts of split sums, added in their order, and what the epilogue would have done with the sum.  A CTA takes 32 rows
// by 32 columns of a tile (of a and of u in the forward pass), through shared memory to rows.
constexpr int kJoinThreads = 256;
template <typename T, bool FORWARD>
__global__ void __launch_bounds__(kJoinThreads)
gemm_join_kernel(const __grid_constant__ GemmArgs a, int part)
{
    stream_order();
    constexpr int kSums = FORWARD ? 8 : 4;                    // of a thread: 4 columns, of a and of u
    __shared__ float sums[FORWARD ? 2 : 1][32][33];
    const GemmPart& p = a.part[part];
    const Unit t = unit_of<FORWARD>(a, part, blockIdx.x);
    const int r0 = blockIdx.y * 32, c0 = blockIdx.z * 32, row0 = t.m * kTileM + r0, col0 = t.n * (FORWARD ? kHalf : kTileN) + c0;
    if (row0 >= p.rows || col0 >= p.cols) return;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const float* from = p.partial + static_cast<size_t>(blockIdx.x) * kTileM * kTileN + r0 + lane;
    const size_t step = static_cast<size_t>(p.tiles) * kTileM * kTileN;
    float s[kSums] = {};
    if (row0 + lane < p.rows) {
#pragma unroll 4
        for (int i = 0; i < p.splits; ++i)
#pragma unroll
            for (int j = 0; j < kSums; ++j) {
                const int c = warp * 4 + j % 4;
                if (col0 + c < p.cols) s[j] += __ldcs(from + i * step + static_cast<size_t>(j / 4 * kHalf + c0 + c) * kTileM);
            }
    }
#pragma unroll
    for (int j = 0; j < kSums; ++j) sums[j / 4][lane][warp * 4 + j % 4] = s[j];
    __syncthreads();
    for (int j = threadIdx.x; j < 32 * 32; j += kJoinThreads) {
        const int r = j / 32, c = j % 32;
        if (row0 + r >= p.rows || col0 + c >= p.cols) continue;
        const size_t at = static_cast<size_t>(row0 + r) * p.cols + col0 + c;
        if (FORWARD) {
            const float g = sums[0][r][c], u = sums[FORWARD ? 1 : 0][r][c];
            if (a.out[1][t.worker]) {
                static_cast<T*>(a.out[1][t.worker])[at] = narrow<T>(g);
                static_cast<T*>(a.out[2][t.worker])[at] = narrow<T>(u);
            }
            static_cast<T*>(a.out[0][t.worker])[at] = narrow<T>(activation(a.activation, g) * u);
        } else {
            T* out = static_cast<T*>(a.out[part == kInputGrad ? 0 : 1 + t.half][t.worker]) + at;
            *out = narrow<T>(part == kWeightGrad && a.accumulate ? widen(*out) + sums[0][r][c] : sums[0][r][c]);
        }
    }
}

// ------------------------------------------------------------------ a few rows

// For a few rows the product is a pass over the weights, which no 256-row tile makes faster: a CTA takes 16 neighbouring
// columns of a and u, its warps steps of 32 along the sum in turn, and the products are 16 x 8 x 16 ones of the warp-wide
// matrix instruction (multiply-adds of the plain cores, two products an instruction, were the bound from 2 rows on:
// 4 x 5 tokens, 768 -> 2048, 11.3 us).  As the order along the sum is free, a lane's operands are 16 neighbouring bytes of
// a row, in the weights and in x alike: four lanes read 64 bytes of a row, where they stand, at any alignment (the
// tcgen05 path would lay unaligned weights out again first).  x comes from the L1 cache.  Four CTAs an SM hold the kernel of up
// to 8 rows to 64 registers, where weights that start anywhere spill 48 bytes: 4 x 5 tokens, 768 -> 2048, 8.2 us for 3.9 of bytes.
struct FewArgs {
    In x, w_gate, w_up;
    Out h, gate, up;                       // gate and up may be NULL
    int rows, d_in, d_hidden, activation;
};
constexpr int kFewThreads = 256, kFewCols = 16, kFewRows = 16;

// d (16 x 8) += a (16 x 16) b (16 x 8)
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1, __nv_bfloat16)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1, __half)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// How the operands are read:
//   kFewWhole    x and the weights in whole 16-byte words at 16-byte boundaries;
//   kFewShifted  weight rows of whole words that start anywhere (a layer inside a flat vector): all rows of a matrix start
//                `skip` halves behind a boundary, so their aligned words are read as they are, against words of x that
//                start `skip` halves early (8 x 1 token, 4096 -> 8192: 342 us with every word put together from two);
//   kFewAny      rows of any length: every word put together.
enum FewMode { kFewAny = 0, kFewWhole = 1, kFewShifted = 2 };

// Word j of a row of n halves (a multiple of 8) that is cut `skip` halves in front of its start and every 8 from there;
// the row is taken as a ring, so that word 0 begins with the `skip` halves that are left at its end.
__device__ __forceinline__ uint4 cut_word(const unsigned short* row, int j, int n, unsigned skip)
{
    if (j > 0 || skip == 0) return load_halves(row + 8 * j - static_cast<int>(skip), 8);
    return shift_halves(load_halves(row + n - 8, 8), load_halves(row, 8), 8 - skip);
}

// NT: groups of 8 rows of x.
template <typename T, int NT, int MODE>
__global__ void __launch_bounds__(kFewThreads, NT == 1 ? 4 : MODE == kFewShifted ? 2 : 3)
gated_few_kernel(const __grid_constant__ FewArgs a)
{
    stream_order();
    constexpr int kWarps = kFewThreads / 32;
    __shared__ float sums[kWarps][2][NT * 8][kFewCols + 1];
    const int m = blockIdx.y, col0 = blockIdx.x * kFewCols;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, line = lane / 4, piece = lane % 4;
    const unsigned short* w[4];                               // of this lane: gate and up rows of columns `line` and line + 8
#pragma unroll
    for (int i = 0; i < 4; ++i)                               // (at the edge the last column again)
        w[i] = static_cast<const unsigned short*>(i & 1 ? a.w_up.p[m] : a.w_gate.p[m]) +
               static_cast<size_t>(min(col0 + line + i / 2 * 8, a.d_hidden - 1)) * a.d_in;
    const unsigned short* x = static_cast<const unsigned short*>(a.x.p[m]) + static_cast<size_t>(line) * a.d_in;
    const unsigned skip[2] = {MODE == kFewShifted ? skip_of(w[0]) : 0u, MODE == kFewShifted ? skip_of(w[1]) : 0u};
    const int words = (a.d_in + 7) / 8;
    float acc[2][NT][4] = {};
    const auto step = [&](int k0, auto first) {               // first: the step with word 0
        const int k = k0 + piece, count = min(8, a.d_in - 8 * k);
        const bool cut = MODE == kFewShifted && decltype(first)::value && k == 0;
        uint4 v[4], in[2][NT];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = make_uint4(0, 0, 0, 0);
            if (k < words) {
                if constexpr (MODE == kFewAny) v[i] = load_halves(w[i] + 8 * k, count);
                else if (cut) v[i] = cut_word(w[i], 0, a.d_in, skip[i & 1]);
                else v[i] = __ldcs(reinterpret_cast<const uint4*>(w[i] - skip[i & 1]) + k);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            in[0][t] = in[1][t] = make_uint4(0, 0, 0, 0);
            if (k < words && t * 8 + line < a.rows) {
                const unsigned short* row = x + static_cast<size_t>(t) * 8 * a.d_in;
                if constexpr (MODE == kFewAny) in[0][t] = load_halves(row + 8 * k, count);
                else if constexpr (MODE == kFewWhole) in[0][t] = reinterpret_cast<const uint4*>(row)[k];
                else if (cut) in[0][t] = cut_word(row, 0, a.d_in, skip[0]);
                else in[0][t] = load_halves(row + 8 * k - static_cast<int>(skip[0]), 8);
                in[1][t] = in[0][t];
                if (MODE == kFewShifted && skip[1] != skip[0]) in[1][t] = cut_word(row, k, a.d_in, skip[1]);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {                     // gate, up
                mma_16x8x16(acc[i][t], v[i].x, v[i + 2].x, v[i].y, v[i + 2].y, in[i][t].x, in[i][t].y, T{});
                mma_16x8x16(acc[i][t], v[i].z, v[i + 2].z, v[i].w, v[i + 2].w, in[i][t].z, in[i][t].w, T{});
            }
    };
    int k0 = warp * 4;
    if (MODE == kFewShifted && warp == 0) {
        step(0, std::true_type{});
        k0 = kWarps * 4;
    }
#pragma unroll 2
    for (; k0 < words; k0 += kWarps * 4) step(k0, std::false_type{});
    // the warps' parts of the sums, added in their order
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[warp][i][t * 8 + piece * 2 + e % 2][line + e / 2 * 8] = acc[i][t][e];
    __syncthreads();
    for (int j = threadIdx.x; j < a.rows * kFewCols; j += kFewThreads) {
        const int r = j / kFewCols, c = j % kFewCols;
        if (col0 + c >= a.d_hidden) continue;
        float g = 0.0f, u = 0.0f;
#pragma unroll
        for (int p = 0; p < kWarps; ++p) { g += sums[p][0][r][c]; u += sums[p][1][r][c]; }
        const size_t at = static_cast<size_t>(r) * a.d_hidden + col0 + c;
        if (a.gate.p[m]) {
            static_cast<T*>(a.gate.p[m])[at] = narrow<T>(g);
            static_cast<T*>(a.up.p[m])[at] = narrow<T>(u);
        }
        static_cast<T*>(a.h.p[m])[at] = narrow<T>(activation(a.activation, g) * u);
    }
}

// ------------------------------------------------------------------ elementwise parts

struct GatedGradArgs {
    In dh, gate, up;
    void *da, *du;                         // [M][rows][pitch]
    long long rows;
    int cols, pitch, activation;
};

constexpr int kGatedThreads = 256;

// da = dh u act'(a), du = dh act(a): bound by memory, 5 elements of traffic an element.  A thread handles 8 elements:
// STEP = 8 neighbouring ones of a row (16-byte accesses), or pairs (4 bytes) or single ones, 32 pairs or elements apart, so
// that a warp's accesses are contiguous.
template <typename T, int STEP>
__global__ void __launch_bounds__(kGatedThreads)
gated_grad_kernel(const __grid_constant__ GatedGradArgs a)
{
    stream_order();
    const int m = blockIdx.y, lane = threadIdx.x & 31, per_row = STEP == 8 ? a.pitch / 8 : (a.pitch + 255) / 256 * 32;
    const long long at = static_cast<long long>(blockIdx.x) * kGatedThreads + threadIdx.x;
    const long long row = at / per_row;
    if (row >= a.rows) return;
    const int col = STEP == 8 ? static_cast<int>(at % per_row) * 8 : static_cast<int>(at % per_row) / 32 * 256 + lane * STEP;
    const long long in = row * a.cols + col;
    const T* dh = static_cast<const T*>(a.dh.p[m]) + in;
    const T* gate = static_cast<const T*>(a.gate.p[m]) + in;
    const T* up = static_cast<const T*>(a.up.p[m]) + in;
    float d[8] = {}, g[8] = {}, u[8] = {};
    if constexpr (STEP == 8) {
        unpack<T>(*reinterpret_cast<const uint4*>(dh), d);
        unpack<T>(*reinterpret_cast<const uint4*>(gate), g);
        unpack<T>(*reinterpret_cast<const uint4*>(up), u);
    } else if constexpr (STEP == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + 64 * e < a.cols) {
                unpack_pair(*reinterpret_cast<const unsigned*>(dh + 64 * e), d + 2 * e, T{});
                unpack_pair(*reinterpret_cast<const unsigned*>(gate + 64 * e), g + 2 * e, T{});
                unpack_pair(*reinterpret_cast<const unsigned*>(up + 64 * e), u + 2 * e, T{});
            }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + 32 * e < a.cols) { d[e] = widen(dh[32 * e]); g[e] = widen(gate[32 * e]); u[e] = widen(up[32 * e]); }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 f = activation_slope(a.activation, g[e]);
        u[e] = d[e] * u[e] * f.y;
        g[e] = d[e] * f.x;
    }
    const size_t out = (static_cast<size_t>(m) * a.rows + row) * a.pitch + col;
    T* da = static_cast<T*>(a.da) + out;
    T* du = static_cast<T*>(a.du) + out;
    if constexpr (STEP == 8) {
        *reinterpret_cast<uint4*>(da) = pack<T>(u);
        *reinterpret_cast<uint4*>(du) = pack<T>(g);
    } else if constexpr (STEP == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + 64 * e < a.cols) {
                *reinterpret_cast<unsigned*>(da + 64 * e) = pack_pair(u[2 * e], u[2 * e + 1], T{});
                *reinterpret_cast<unsigned*>(du + 64 * e) = pack_pair(g[2 * e], g[2 * e + 1], T{});
            }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + 32 * e < a.cols) { da[32 * e] = narrow<T>(u[e]); du[32 * e] = narrow<T>(g[e]); }
    }
}

struct PackArgs {
    In from[2];
    unsigned short* to[2];                 // [M][rows][pitch]
    long long rows;
    int cols, pitch;
};

// Rows of 16-bit elements at any address, laid out again with 16-byte aligned rows, as TMA wants them: gridDim.z
// operands of one shape.  A thread makes one 16-byte word of the result from the two aligned words that hold its
// elements (each of which holds at least one of them, so nothing outside the operand's own words is read).
static __global__ void __launch_bounds__(kGatedThreads)
pack_rows_kernel(const __grid_constant__ PackArgs a)
{
    stream_order();
    const int m = blockIdx.y, per_row = a.pitch / 8;
    const long long at = static_cast<long long>(blockIdx.x) * kGatedThreads + threadIdx.x;
    if (at >= a.rows * per_row) return;
    const long long row = at / per_row;
    const int col = static_cast<int>(at % per_row) * 8, count = min(8, a.cols - col);
    const uint4 v = load_halves(static_cast<const unsigned short*>(a.from[blockIdx.z].p[m]) + row * a.cols + col, count);
    *reinterpret_cast<uint4*>(a.to[blockIdx.z] + (static_cast<size_t>(m) * a.rows + row) * a.pitch + col) = v;
}

}  // namespace replica
}  // namespace grawa

// Attention within a window on the tensor cores (the masks and formulas stand in attention_rows.cuh).
//
// Every kernel here gives a CTA 128 rows of one head, a tile, and lets it walk over the rows that the tile's rows see or
// are seen by, some at a time: the first keys of the sequence that the tile's first row belongs to, then one run of rows (of
// the tile's other sequences, which begin inside it, all rows lie in that run).  Rows are packed, so a tile may hold the ends of
// some sequences and the starts of others; the mask of a row is two intervals, which a thread turns into bits where a
// step is not visible throughout.  One thread fetches operands by TMA, one warp issues tcgen05.mma, and the threads of eight others have
// half of a row of the tile each: its scores come from tensor memory, and what they make of them goes back there as the next
// product's operand, so nothing but tiles of q, k, v and dout passes through shared memory.  A step is 128 rows wide, because products
// of two operands in shared memory take the tensor cores as long for 64 columns as for 128.
//
//   forward    S = Q K^T, P = exp2(S c - m), O += P V.  m is a row's largest score so far (6 less in half precision), but is only moved when
//              that grows by more than 2^8 (P stays below 2^8, or 2^14), so that O, which lies in tensor memory, is rarely scaled.
//   dq         S = Q K^T, dP = dO V^T, dS = P (dP - delta), dQ += dS K
//   dk, dv     S^T = K Q^T, dP^T = V dO^T, dV += P^T dO, dK += dS^T Q, over all query heads of the key head
//
// dq and dk, dv are two kernels that both compute the scores: seven products instead of five, but no sum is made by atomics,
// whose order would change the results.  lse and delta = dout out come from a small kernel in front (two floats a row).
//
// A masked element of P and dS is an exact zero.  Where the value it multiplies is not finite the product is NaN all the same, and spoils
// rows that do not see it.  Tiles with such a result are walked a second time, with care: see "what is not finite" below.
//
// Measured (B200, back to back, where the power limit holds the clock at 1.6 GHz): 2 x 8192 tokens, 16 query heads on 8 of 128, causal, bf16:
// forward 590 us (930 TFLOP/s), backward 1820 us (755); what bounds a CTA is the way of a step from its scores to their exponentials to
// the next product, three waits of some hundred cycles each beside the arithmetic's, and what bounds the SM is power.
//
// Every wait for a barrier in shared memory is bounded, as in the gated feed-forward product: a wait that runs out is counted
// in g_attention_timeouts, and the CTA waits (bounded) for its copies and products in flight, frees its tensor memory
// and returns without storing.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "attention_rows.cuh"
#include "tensor_core.cuh"

namespace grawa {
namespace replica {

constexpr int kTile = 128;                  // rows of a CTA
constexpr int kBox = 64;                    // rows, and elements of a row, of one TMA box
constexpr int kBoxBytes = kBox * kBox * 2;
constexpr int kAttentionWorkers = 16;       // workers a launch (their tensor maps travel as kernel parameters)

struct TileArgs {
    AttentionArgs a;
    CUtensorMap map[4][kAttentionWorkers];  // q, k, v, dout
    const float *lse, *delta;               // backward: [worker][head][pitch], -lse in units of log 2, and -delta
    const float* longest;                   // backward, half precision: [worker][2], the squared length of the longest row of dout, of v
    long long pitch;
    float* partial;                         // backward, where chunks of queries are set apart (or NULL): [worker][key head][chunk][dv, dk][first key][dim]
    int chunks, far;                        // far: this launch is of the chunks
    int beside;                             // backward: this launch needs nothing of the one in front, only of those before that
    int first_worker, workers;
    Divisor per, per_worker;                // tiles of one place in the rows: of all heads and workers of the launch, of one worker
};

__device__ unsigned g_attention_timeouts = 0;   // waits that ran out, never set back
constexpr unsigned long long kAttentionWaitNs = 2000000000ull, kAttentionStarvedNs = 2000000ull;

// ------------------------------------------------------------------ copies, products, tensor memory

template <unsigned long long LIMIT>
__device__ __forceinline__ bool tile_wait(unsigned bar, unsigned parity, volatile int* gave_up)
{
    return bounded_wait<LIMIT, false>(bar, parity, gave_up, &g_attention_timeouts);
}
__device__ __forceinline__ void arrive_here(unsigned bar) { asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void copy_box(unsigned dst, const CUtensorMap* map, int element, int head, int row, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map),
                 "r"(element), "r"(head), "r"(row), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void copy_floats(unsigned dst, const float* from, unsigned bytes, unsigned bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// D (+)= A B^T for 16 steps along the sum, A in shared or in tensor memory.
__device__ __forceinline__ void mma_shared(unsigned d, unsigned long long a, unsigned long long b, unsigned shape, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(shape), "r"(add ? 1u : 0u)
        : "memory");
}
__device__ __forceinline__ void mma_tensor(unsigned d, unsigned a, unsigned long long b, unsigned shape, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(shape), "r"(add ? 1u : 0u)
        : "memory");
}
// One lane of a whole warp, the same every time.  Products are issued by warps that stay together up to here: what they are given is
// then the same in all lanes to the compiler too, and goes to the tensor cores without a detour for each.
__device__ __forceinline__ bool one_lane()
{
    unsigned one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
// Arrives when every product this thread has issued so far is done.
__device__ __forceinline__ void mma_done(unsigned bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <int COLS>
__device__ __forceinline__ void tensor_alloc(unsigned slot)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "n"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int COLS>
__device__ __forceinline__ void tensor_free(unsigned tmem)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(COLS));
}
#define GRAWA_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define GRAWA_RW8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define GRAWA_W8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of this warp's 32 lanes: a thread gets 32 neighbouring values of its row, for use after tensor_wait on them.
__device__ __forceinline__ void tensor_load(unsigned at, unsigned (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : GRAWA_R8(r, 0), GRAWA_R8(r, 8), GRAWA_R8(r, 16), GRAWA_R8(r, 24)
        : "r"(at));
}
__device__ __forceinline__ void tensor_wait(unsigned (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : GRAWA_RW8(r, 0), GRAWA_RW8(r, 8), GRAWA_RW8(r, 16), GRAWA_RW8(r, 24) : : "memory");
}
__device__ __forceinline__ void tensor_load(unsigned at, unsigned (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : GRAWA_R8(r, 0), GRAWA_R8(r, 8)
                 : "r"(at));
}
__device__ __forceinline__ void tensor_wait(unsigned (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : GRAWA_RW8(r, 0), GRAWA_RW8(r, 8) : : "memory");
}
__device__ __forceinline__ void tensor_store(unsigned at, const unsigned (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::GRAWA_W8(r, 0), GRAWA_W8(r, 8),
                 "r"(at)
                 : "memory");
}
__device__ __forceinline__ void tensor_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two floats side by side, for instructions that take two at once.
struct Two { unsigned long long v; };
__device__ __forceinline__ Two two(float a, float b)
{
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ Two two(const unsigned* bits) { return two(__uint_as_float(bits[0]), __uint_as_float(bits[1])); }
__device__ __forceinline__ void apart(Two x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ Two fma_two(Two a, Two b, Two c)
{
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Two add_two(Two a, Two b)
{
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two mul_two(Two a, Two b)
{
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ float max_three(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Powers of two by the special function unit, which makes 16 a cycle and SM; zero below 2^-126.  (A share of them by a polynomial of degree 5 in
// its shadow was tried: 2 x 8192 tokens, 16 heads of 64, causal, forward 407 us with none, 433 with one pair in 8, 473 in 4; backward
// 1153 with none, 1112 with one in 4, but 312 and 328 for 4 x 32 images of 197 tokens, and 1820 and 1885 with heads of 128 on 8.)
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void exp2_fast(Two x, float& a, float& b)
{
    apart(x, a, b);
    a = exp2_fast(a);
    b = exp2_fast(b);
}

// Bits [lo, hi] of a word, either end of which may lie outside it.
__device__ __forceinline__ unsigned bits_between(int lo, int hi)
{
    const unsigned up = lo <= 0 ? ~0u : lo > 31 ? 0u : ~0u << lo;
    const unsigned down = hi >= 31 ? ~0u : hi < 0 ? 0u : ~0u >> (31 - hi);
    return up & down;
}

// ------------------------------------------------------------------ a tile's way

// What the rows of a tile see, or are seen by, in all.
struct Reach { int min_lo, max_lo, min_hi, max_hi, min_start; };

// Of the tile's rows [r0, r0 + 128), by a whole warp.  As sequences and windows only move forward, the ends come from few rows: the
// first and the last that belong to a sequence, the first sequence's first row that is no first key, and the last sequence's
// first row in the tile.  `rows` says of a row and its sequence what it sees.
template <typename F>
__device__ __forceinline__ Reach reach_of(const AttentionArgs& a, int m, int r0, int lane, const F& rows)
{
    const long long* offsets = static_cast<const long long*>(a.offsets.p[m]);
    int begin = r0, end = min(r0 + kTile, a.rows);            // the rows that belong to a sequence
    if (offsets) {
        begin = static_cast<int>(max(static_cast<long long>(begin), min(static_cast<long long>(end), offsets[0])));
        end = static_cast<int>(min(static_cast<long long>(end), max(static_cast<long long>(begin), offsets[a.sequences])));
    }
    const Sequence s = begin < end ? sequence_of(a, m, lane == 0 ? begin : end - 1) : Sequence{0, 0};
    const Sequence first{__shfl_sync(0xffffffffu, s.start, 0), __shfl_sync(0xffffffffu, s.end, 0)}, last{__shfl_sync(0xffffffffu, s.start, 1), __shfl_sync(0xffffffffu, s.end, 1)};
    const int inner = max(begin, a.sinks >= end - first.start ? end : first.start + a.sinks);
    const int row = lane == 0 ? begin : lane == 1 ? end - 1 : lane == 2 ? (inner < min(end, first.end) ? inner : begin) : max(begin, last.start);
    Keys k{};
    const bool in = begin < end && rows(lane == 0 || lane == 2 ? first : last, row, k);
    Reach r;
    r.min_lo = __reduce_min_sync(0xffffffffu, in ? k.lo : 0x7fffffff), r.max_lo = __reduce_max_sync(0xffffffffu, in ? k.lo : -1);
    r.min_hi = __reduce_min_sync(0xffffffffu, in ? k.hi : 0x7fffffff), r.max_hi = __reduce_max_sync(0xffffffffu, in ? k.hi : -1);
    r.min_start = __reduce_min_sync(0xffffffffu, in ? k.start : 0x7fffffff);
    return r;
}
// What queries see.
struct QueryRows {
    const AttentionArgs& a;
    __device__ __forceinline__ bool operator()(const Sequence& s, int row, Keys& k) const
    {
        if (s.start >= s.end) return false;
        k = keys_of(a, s, row);
        return true;
    }
};
template <typename F>
__device__ __forceinline__ bool own_keys(const AttentionArgs& a, int m, int row, const F& rows, Keys& k)
{
    return rows(row < a.rows ? sequence_of(a, m, row) : Sequence{0, 0}, row, k);
}

// The tiles of all heads and workers, those of one place in the rows side by side; each CTA takes one in `gridDim.x`, in an order that
// turns round every time, so that walks that get shorter from place to place come to about the same for all CTAs.
__device__ __forceinline__ int tile_of_round(int round)
{
    return round * static_cast<int>(gridDim.x) + static_cast<int>(round % 2 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
}

// The key rows that a tile of queries walks over, `step` rows at a time.
struct KeyWalk {
    int first, main, sink_steps, steps;     // rows of the first step among the first keys, and of the first other one
    __device__ __forceinline__ KeyWalk(const Reach& r, int sinks, int step)
    {
        first = r.min_start;
        main = r.min_lo;
        const int end = sinks >= main - first ? main : first + sinks;
        sink_steps = 0;
        if (end > first) {
            if (main - first <= step) main = first;           // one run of rows costs no more
            else sink_steps = (end - first + step - 1) / step;
        }
        steps = r.max_hi >= main ? sink_steps + (r.max_hi - main) / step + 1 : 0;
    }
    __device__ __forceinline__ int row(int i, int step) const { return i < sink_steps ? first + i * step : main + (i - sink_steps) * step; }
};
// Which of 32 keys from row j on a query sees, in a step that ends in front of row `limit`.
__device__ __forceinline__ unsigned seen_keys(const Keys& k, int j, int limit)
{
    const int hi = min(k.hi, limit - 1);
    return bits_between(k.lo - j, hi - j) | bits_between(k.start - j, min(k.sinks_end - 1, hi) - j);
}

// The tiles of a CTA on their way from the copying warp, which works them out ahead of the others, to these.
constexpr int kPlaces = 4;
template <typename P>
struct PlaceRing {
    P* slots;                               // in shared memory
    unsigned there, free;                   // barriers of the slots
    __device__ __forceinline__ const P& operator[](int tile) const { return slots[tile % kPlaces]; }
};

// 32 rows of results on their way from tensor memory to memory, a warp's own: columns [from_col, from_col + cols) of the row's
// `elements`, at `tensor` on, with what `add` adds to the 32 values from a column on, times f.  A thread has a row, but whole
// sectors of neighbouring rows are what memory takes well: CHUNK columns at a time pass through 64 CHUNK bytes of shared memory, in
// 16-byte pieces that are permuted against bank conflicts.  Rows without their bit in `valid` are not stored.  Returns whether
// all of this thread's values were finite.
template <typename T, int CHUNK, typename F>
__device__ __forceinline__ bool store_rows(unsigned tensor, int from_col, int cols, float f, unsigned char* stage, T* to, long long stride, int elements, unsigned valid,
                                           const F& add)
{
    constexpr int kPieces = CHUNK / 8, kRows = 32 / kPieces, kTurn = 8 / kPieces;        // rows a store; rows in 128 bytes
    const int lane = threadIdx.x % 32, piece = lane % kPieces, first = lane / kPieces;
    bool fine = true;
#pragma unroll 1
    for (int c = 0; c < cols; c += 32) {
        unsigned r[32];
        tensor_load(tensor + c, r);
        tensor_wait(r);
        float v[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(r[e]);
        add(v, from_col + c);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            v[e] *= f;
            fine = fine && fabsf(v[e]) <= 3.0e38f;
        }
#pragma unroll
        for (int k = 0; k < 32; k += CHUNK) {
#pragma unroll
            for (int e = 0; e < kPieces; ++e)
                *reinterpret_cast<uint4*>(stage + lane * CHUNK * 2 + ((e ^ lane / kTurn % kPieces) * 16)) = pack<T>(v + k + 8 * e);
            __syncwarp();
            const int col = from_col + c + k + piece * 8;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int row = first + kRows * i;
                const uint4 word = *reinterpret_cast<const uint4*>(stage + row * CHUNK * 2 + ((piece ^ row / kTurn % kPieces) * 16));
                if (valid >> row & 1 && col < elements) *reinterpret_cast<uint4*>(to + row * stride + col) = word;
            }
            __syncwarp();
        }
    }
    return fine;
}

// ------------------------------------------------------------------ what is not finite
//
// The products P V, dS K, P^T dO and dS^T Q sum over a step's rows, and take a masked row's zero times infinity for NaN.  (The others make
// a score of one row and one column, which is masked as such.)  So a CTA notes the tiles with a result that is not finite, and when it is
// through walks those once more.  This time the threads of the rows look each step's operand of such a product over, set elements that
// are not finite to zero where they stand in shared memory, and keep for each row they see such elements from in which columns infinity
// of either sign (both: NaN) is to be added to the sum.  An element of P counts as positive even where it is too small for 32 bits; dS, which
// then is zero or not finite itself, as making NaN.  Rows that belong to no sequence, which may hold anything, are zeroed on the first walk
// already, where a step holds some.
//
// Measured (2 x 8192 tokens, 16 query heads on 8 of 128, causal, bf16; 520 us forward, 1610 backward with finite operands): one infinity in
// the first row of v 1390 us forward; in the last one of dout 3540 us backward; v NaN throughout 3570 us forward, dout 7900 us
// backward; one infinity in each row of v 15.9 ms, of dout 19 ms.  Each row done again by one warp in turn, which needs no second
// walk, took 0.4 us for each row that it saw: 255 s for the first 128 of 300000 tokens with 64 query heads on one key head.
constexpr int kMarks = 1024;                // tiles that a CTA tells apart; beyond, those of the same remainder share a mark

// Bits of the 16-bit elements of a word that are not finite.
template <typename T>
__device__ __forceinline__ unsigned not_finite(unsigned w)
{
    constexpr unsigned kField = TypeCode<T>::value ? 0x7f80u : 0x7c00u;
    return ((w & kField) == kField ? 0xffffu : 0u) | ((w & kField << 16) == kField << 16 ? 0xffff0000u : 0u);
}
// Where 8 elements of a row of a step lie in shared memory; piece: which 8 of 64, half: which 64 of the head's elements.
__device__ __forceinline__ uint4* piece_of(unsigned char* slot, int row, int half, int piece)
{
    return reinterpret_cast<uint4*>(slot + (half * 2 + row / 64) * kBoxBytes + row % 64 * 128 + piece * 16);
}
// What generic stores left in shared memory, in the sight of the products that are issued behind the next barrier.
__device__ __forceinline__ void to_products() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// The rows that belong to sequences (up to the largest number, where all from the first on do).
__device__ __forceinline__ void rows_of_sequences(const AttentionArgs& a, int m, int& from, int& to)
{
    const long long* offsets = static_cast<const long long*>(a.offsets.p[m]);
    from = 0, to = 0x7fffffff;
    if (offsets == nullptr) return;
    const long long first = offsets[0], end = offsets[a.sequences];
    from = static_cast<int>(max(0ll, min(first, static_cast<long long>(a.rows))));
    if (end < a.rows) to = static_cast<int>(max(0ll, end));
}

// Sets those among a warp's 16 rows of a step that lie outside [from, to) to zero, when two barriers have been passed; false when that gave up.
template <int DP>
__device__ __noinline__ bool zero_loose_rows(int from, int to, unsigned char* slot, unsigned bar, unsigned parity, unsigned other, unsigned other_parity,
                                             volatile int* gave_up)
{
    const int first = threadIdx.x / 32 * 16;
    if (first >= from && first + 16 <= to) return true;
    if (!__all_sync(0xffffffffu, tile_wait<kAttentionWaitNs>(bar, parity & 1, gave_up) && tile_wait<kAttentionWaitNs>(other, other_parity & 1, gave_up))) return false;
#pragma unroll 1
    for (int i = 0; i < DP / 64 * 4; ++i) {                   // 4 rows of 64 elements each
        const int row = first + i % 4 * 4 + threadIdx.x % 32 / 8;
        if (row < from || row >= to) *piece_of(slot, row, i / 4, threadIdx.x % 8) = make_uint4(0, 0, 0, 0);
    }
    to_products();
    return true;
}
// Sets the elements of a warp's 16 rows of a step that are not finite to zero, and returns bits of their rows.
template <typename T, int DP>
__device__ __noinline__ unsigned zero_not_finite(unsigned char* slot)
{
    unsigned rows = 0;
#pragma unroll 1
    for (int i = 0; i < DP / 64 * 4; ++i) {
        uint4* const at = piece_of(slot, threadIdx.x / 32 * 16 + i % 4 * 4 + threadIdx.x % 32 / 8, i / 4, threadIdx.x % 8);
        uint4 w = *at;
        const uint4 bad = make_uint4(not_finite<T>(w.x), not_finite<T>(w.y), not_finite<T>(w.z), not_finite<T>(w.w));
        const bool any = (bad.x | bad.y | bad.z | bad.w) != 0;
        if (any) {
            w.x &= ~bad.x; w.y &= ~bad.y; w.z &= ~bad.z; w.w &= ~bad.w;
            *at = w;
        }
        const unsigned lanes = __ballot_sync(0xffffffffu, any);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (lanes >> 8 * k & 0xff) rows |= 1u << (i % 4 * 4 + k);
    }
    to_products();
    return rows;
}
// What the warps of a CTA tell each other of a step's rows: their 16 bits each, for two steps in turn.
using BadRows = unsigned short[2][8];
// The columns in which a thread's row gets infinities: bit l of word e stands for column 4 l + e, words 0 to 3 are +, 4 to 7 -.
struct Infinities {
    unsigned bits[8];
    __device__ __forceinline__ void load(const unsigned* mine)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) bits[e] = mine[e];
    }
    // To 32 sums from column `col` on.
    __device__ __forceinline__ void add(float (&v)[32], int col) const
    {
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            if (bits[e % 4] >> (col / 4 + e / 4) & 1) v[e] += INFINITY;
            if (bits[4 + e % 4] >> (col / 4 + e / 4) & 1) v[e] -= INFINITY;
        }
    }
};
// Adds to this thread's words what its row, whose keys (or queries) are `keys`, sees of the marked rows among those from row r on, which
// stand in memory from `rows` on, one head of `dim` elements of each; as NaN with `nan`.
template <typename T>
__device__ __noinline__ void add_infinities(unsigned* mine, const unsigned short* bad, const T* rows, long long stride, int dim, Keys keys, int r, int limit, bool nan)
{
    constexpr int kAtOnce = 4;
    constexpr unsigned kField = TypeCode<T>::value ? 0x7f80u : 0x7c00u, kRest = 0x7fffu & ~kField;
    const int at = threadIdx.x % 32 * 4;
    const unsigned all = dim >= 128 ? ~0u : (1u << dim / 4) - 1;
    Infinities own;
    own.load(mine);
#pragma unroll 1
    for (int warp = 0; warp < 8; ++warp) {
        unsigned left = bad[warp];
#pragma unroll 1
        while (left) {
            int j[kAtOnce];
            uint2 w[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                j[k] = left ? warp * 16 + __ffs(left) - 1 : -1;
                left &= left - 1;
                w[k] = j[k] >= 0 && at < dim ? *reinterpret_cast<const uint2*>(rows + j[k] * stride + at) : make_uint2(0, 0);
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (j[k] < 0) break;
                const bool sees = seen_keys(keys, r + j[k], limit) & 1;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned x = (e < 2 ? w[k].x : w[k].y) >> e % 2 * 16;
                    const bool bad_one = (x & kField) == kField, both = nan || (x & kRest);
                    const unsigned plus = __ballot_sync(0xffffffffu, bad_one && (both || !(x & 0x8000u)));
                    const unsigned minus = __ballot_sync(0xffffffffu, bad_one && (both || (x & 0x8000u)));
                    if (sees) own.bits[e] |= plus, own.bits[4 + e] |= minus;
                }
            }
        }
        unsigned full = all;
#pragma unroll
        for (int e = 0; e < 8; ++e) full &= own.bits[e];
        if (__all_sync(0xffffffffu, full == all)) break;      // NaN throughout, and nothing changes that
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) mine[e] = own.bits[e];
}
// Notes a tile for the second walk, and whether it is noted.
__device__ __forceinline__ void mark_tile(unsigned* marks, int* more, int tile)
{
    atomicOr(marks + tile % kMarks / 32, 1u << tile % 32);
    *more = 1;
}
__device__ __forceinline__ bool marked(const unsigned* marks, int tile) { return marks[tile % kMarks / 32] >> tile % 32 & 1; }

// 8 results to memory.
__device__ __forceinline__ void store_eight(float* to, const float* v)
{
    reinterpret_cast<uint4*>(to)[0] = pack<float>(v);
    reinterpret_cast<uint4*>(to)[1] = pack<float>(v + 4);
}

// ------------------------------------------------------------------ forward

// DP: elements of a head as the products take them, 64 or 128 (what lies behind the head's end is zero).  Two CTAs an SM, so
// that the products of one run beside the exponentials of the other; each takes one tile after the other, and fetches the next one's
// queries while it works.  Two threads share a row, one half of a step's scores each: what they wait for one after the other (scores,
// their exponentials, the sum) bounds a CTA.
constexpr int kForwardThreads = 320;        // warps 0 to 7: rows, 64 columns of a step each; 8: copies, 9: products
template <int DP> constexpr int kForwardStages = DP == 128 ? 2 : 4;
constexpr int kForwardChunk = 16;           // columns of results on their way
template <int DP> constexpr int kForwardSmem = (1 + kForwardStages<DP>) * kTile * DP * 2 + 8 * 64 * kForwardChunk + 1024;

// STARVED: for the self-test of the bounded waits only; nothing is copied, so that the first wait for operands runs out.
struct ForwardPlace {                       // steps = -1: there are no more tiles
    int w, m, h, r0, steps, from, to;       // from, to: the rows that belong to sequences
    Reach all;
    KeyWalk walk;
};
template <typename T, int DP, bool STARVED = false>
__global__ void __launch_bounds__(kForwardThreads, 2)
attention_forward_kernel(const __grid_constant__ TileArgs t)
{
    constexpr unsigned long long kLimit = STARVED ? kAttentionStarvedNs : kAttentionWaitNs;
    constexpr int kStages = kForwardStages<DP>, kBytes = kTile * DP * 2, kHalves = DP / 64;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kStages + 15 + 2 * kPlaces];
    __shared__ __align__(8) unsigned char place_bytes[kPlaces * sizeof(ForwardPlace)];
    __shared__ unsigned tmem_slot, marks[kMarks / 32];
    __shared__ BadRows bad;
    __shared__ int gave_up, more, careful_from;               // more: there are marks; careful_from: steps before the second walk
    __shared__ float most_of[2][2][kTile], total_of[2][kTile];             // a row's largest score in each half, of two steps in turn; its sums

    const unsigned own = (smem_address(raw) + 1023u) & ~1023u, ring = own + kBytes, out = ring + kStages * kBytes;
    const unsigned full = smem_address(bars), empty = full + 8 * kStages, loaded = empty + 8 * kStages, used = loaded + 8, scored = used + 8,
                   weighted = scored + 8, summed = weighted + 8, drain = summed + 8, maxed = drain + 8, totaled = maxed + 32, scanned = totaled + 32;
    const PlaceRing<ForwardPlace> places{reinterpret_cast<ForwardPlace*>(place_bytes), scanned + 8, scanned + 8 + 8 * kPlaces};
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x) >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x < kMarks / 32) marks[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        gave_up = more = 0;
        for (int s = 0; s < kStages; ++s) { barrier_init(full + 8 * s, 1); barrier_init(empty + 8 * s, 1); }
        barrier_init(loaded, 1);                              // q is there
        barrier_init(used, 1);                                // q has done its part
        barrier_init(scored, 1);                              // S of a step is there
        barrier_init(weighted, 8);                            // P is there
        barrier_init(summed, 1);                              // O of a tile is there
        barrier_init(drain, 1);
        for (int s = 0; s < 4; ++s) { barrier_init(maxed + 8 * s, 2); barrier_init(totaled + 8 * s, 2); }        // between the two warps of 32 rows
        barrier_init(scanned, 8);                             // a step has been looked over
        for (int s = 0; s < kPlaces; ++s) { barrier_init(places.there + 8 * s, 1); barrier_init(places.free + 8 * s, 9); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8 && lane < 3 * t.workers) prefetch_map(&t.map[lane % 3][lane / 3]);
    if (warp == 9) tensor_alloc<256>(smem_address(&tmem_slot));
    order_before();
    __syncthreads();
    order_after();
    stream_order();
    const unsigned tmem = tmem_slot, tmem_s = tmem, tmem_o = tmem + 128;

    const AttentionArgs& a = t.a;
    const int tiles = (a.rows + kTile - 1) / kTile, units = tiles * static_cast<int>(t.per.by);
    int fills = 0, loads = 0;                                 // of the copying thread
    int placed = 0, tile = 0, n = 0;                          // tiles handed on and taken, steps, in both walks
    bool ok = true;
    const auto await = [&](unsigned bar, int phase) {         // by a whole warp
        ok = ok && __all_sync(0xffffffffu, tile_wait<kLimit>(bar, phase & 1, &gave_up));
        return ok;
    };
    const auto place_there = [&](int tile) { return await(places.there + 8 * (tile % kPlaces), tile / kPlaces) && places[tile].steps >= 0; };
    const auto place_done = [&](int tile) {
        __syncwarp();
        if (lane == 0) arrive_here(places.free + 8 * (tile % kPlaces));
    };

    // All of a CTA's tiles, or with `second` the marked ones; whether there are marked ones.
    const auto walk_tiles = [&](auto second) __attribute__((always_inline)) {
        constexpr bool careful = decltype(second)::value;
        // (The place without steps that ends a walk counts among the tiles, but not among those of the barriers.)
        if (warp == 8) {
            int round = 0, met = 0;
            const auto place_next = [&] {                         // works the next tile out and hands it on; without steps it is none
                ForwardPlace p{0, 0, 0, 0, -1, 0, 0, Reach{}, KeyWalk(Reach{}, 0, kTile)};
                for (; p.steps <= 0 && round * static_cast<int>(gridDim.x) < units; ++round) {
                    const int unit = tile_of_round(round);
                    if (unit >= units) continue;
                    const int turn = t.per.quotient(unit), in = unit - turn * static_cast<int>(t.per.by), w = t.per_worker.quotient(in), m = t.first_worker + w;
                    const int r0 = (tiles - 1 - turn) * kTile;    // the last rows, which see most, first
                    const Reach all = reach_of(a, m, r0, lane, QueryRows{a});
                    const KeyWalk walk(all, a.sinks, kTile);
                    int from, to;
                    rows_of_sequences(a, m, from, to);
                    p = ForwardPlace{w, m, in - w * a.heads, r0, STARVED ? 1 : walk.steps, from, to, all, walk};
                    if (careful && p.steps > 0 && !marked(marks, met++)) p.steps = 0;
                }
                if (p.steps == 0) p.steps = -1;
                if (placed >= kPlaces && !await(places.free + 8 * (placed % kPlaces), placed / kPlaces - 1)) return p;
                if (lane == 0) {
                    places.slots[placed % kPlaces] = p;
                    arrive_here(places.there + 8 * (placed % kPlaces));
                }
                ++placed;
                return p;
            };
            ForwardPlace at = place_next();
            while (ok && at.steps > 0) {
                const ForwardPlace next = place_next();
                const int kv = a.group_size.quotient(at.h);
                if (!STARVED && ok && lane == 0) {
                    ok = loads == 0 || tile_wait<kLimit>(used, (loads - 1) & 1, &gave_up);
                    if (ok) {
                        barrier_expect(loaded, kBytes);
#pragma unroll
                        for (int i = 0; i < 2 * kHalves; ++i) copy_box(own + i * kBoxBytes, &t.map[0][at.w], i / 2 * 64, at.h, at.r0 + i % 2 * kBox, loaded);
                        ++loads;
                    }
                    for (int i = 0; i < 2 * at.steps && ok; ++i) {               // k, v, k, v, ...
                        const int s = fills % kStages, j = at.walk.row(i / 2, kTile);
                        ok = fills < kStages || tile_wait<kLimit>(empty + 8 * s, (fills / kStages - 1) & 1, &gave_up);
                        if (!ok) break;
                        barrier_expect(full + 8 * s, kBytes);
#pragma unroll
                        for (int b = 0; b < 2 * kHalves; ++b)
                            copy_box(ring + s * kBytes + b * kBoxBytes, &t.map[1 + i % 2][at.w], b / 2 * 64, kv, j + b % 2 * kBox, full + 8 * s);
                        ++fills;
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                at = next;
            }
        } else if (warp == 9) {
            constexpr unsigned kTypes = 1u << 4 | TypeCode<T>::value << 7 | TypeCode<T>::value << 10 | (kTile >> 4) << 24;
            constexpr unsigned kScores = kTypes | (kTile >> 3) << 17, kValues = kTypes | 1u << 16 | (DP >> 3) << 17;
            for (; place_there(tile); ++tile) {
                const int steps = places[tile].steps;
                place_done(tile);
                const auto scores = [&](int i) {
                    const int f = 2 * (n + i), s = f % kStages;
                    if (i >= steps || !await(full + 8 * s, f / kStages)) return;
                    order_after();
                    const unsigned long long dq = matrix_descriptor(own, 16), dk = matrix_descriptor(ring + s * kBytes, 16);
                    if (one_lane()) {
#pragma unroll
                        for (int k = 0; k < DP / 16; ++k) {
                            const unsigned along = (k / 4 * 2 * kBoxBytes + k % 4 * 32) >> 4;
                            mma_shared(tmem_s, dq + along, dk + along, kScores, k > 0);
                        }
                        mma_done(empty + 8 * s);
                        mma_done(scored);
                        if (i + 1 == steps) mma_done(used);
                    }
                    __syncwarp();
                };
                await(loaded, tile - careful);
                scores(0);
                for (int i = 0; i < steps && ok; ++i) {
                    const int f = 2 * (n + i) + 1, s = f % kStages;
                    if (!await(full + 8 * s, f / kStages) || !await(weighted, n + i)) break;
                    order_after();
                    const unsigned long long dv = matrix_descriptor(ring + s * kBytes, 2 * kBoxBytes);
                    if (one_lane()) {
#pragma unroll
                        for (int k = 0; k < kTile / 16; ++k) mma_tensor(tmem_o, tmem_s + k / 4 * 64 + k % 4 * 8, dv + k * (2048 >> 4), kValues, i > 0 || k > 0);
                        mma_done(empty + 8 * s);
                        if (i + 1 == steps) mma_done(summed);
                    }
                    __syncwarp();
                    scores(i + 1);
                }
                if (!ok) break;
                n += steps;
            }
            if (!ok) {
                if (one_lane()) mma_done(drain);
                __syncwarp();
                tile_wait<kLimit>(drain, 0, nullptr);
            }
        } else if (warp < 8) {
            const int quarter = warp % 4, half = warp / 4, line = quarter * 32 + lane;
            const unsigned lanes = static_cast<unsigned>(quarter * 32) << 16, s_at = tmem_s + lanes + half * 64, o_at = tmem_o + lanes + half * (DP / 2);
            unsigned char* const stage = raw + (out - smem_address(raw)) + warp * 64 * kForwardChunk;
            const float c = a.scale * kLog2e;
            unsigned* const mine = reinterpret_cast<unsigned*>(stage) + lane * 8;          // of Infinities
            for (; place_there(tile); ++tile) {
                const ForwardPlace& at = places[tile];
                const KeyWalk walk = at.walk;
                const int steps = at.steps;
                const bool loose = walk.row(steps - 1, kTile) + kTile > at.to;           // some of the rows that are walked over belong to no sequence
                // bfloat16 reaches as far as 32 bits do: on the second walk the weights of a row are 1 at most together, so that no sum of
                // finite values leaves them
                const float unit = careful && TypeCode<T>::value ? exp2f(static_cast<float>(__clz(a.rows) - 40)) : 1.0f;
                Keys keys{};
                const bool valid = own_keys(a, at.m, at.r0 + line, QueryRows{a}, keys);
                float top = -INFINITY, total = 0.0f;
                // Scores past 2^23: the rounding of the largest one's product is more than a factor of the weights should be.  Such tiles are walked
                // a second time too, with products that are rounded before top is taken from them.
                bool far = false, rough = false;              // of top, of any top so far
                if (careful)
                    for (int e = 0; e < 8; ++e) mine[e] = 0;
                for (int i = 0; i < steps; ++i, ++n) {
                    if (!await(scored, n)) break;
                    const int j = walk.row(i, kTile), limit = i < walk.sink_steps ? at.all.min_lo : 0x7fffffff;
                    if (!careful && loose) {
                        const int fill = 2 * n + 1, slot = fill % kStages;
                        ok = zero_loose_rows<DP>(at.from - j, at.to - j, raw + (ring - smem_address(raw)) + slot * kBytes, full + 8 * slot, fill / kStages, full + 8 * slot,
                                                 fill / kStages, &gave_up);
                        if (!ok) break;
                    }
                    if (careful) {
                        const int fill = 2 * n + 1, slot = fill % kStages;
                        if (!await(full + 8 * slot, fill / kStages)) break;
                        const unsigned rows = zero_not_finite<T, DP>(raw + (ring - smem_address(raw)) + slot * kBytes);
                        if (lane == 0) {
                            bad[n % 2][warp] = static_cast<unsigned short>(rows);
                            arrive_here(scanned);
                        }
                        if (!await(scanned, n - careful_from)) break;
                        add_infinities(mine, bad[n % 2], static_cast<const T*>(a.v.p[at.m]) + j * a.v_stride + a.group_size.quotient(at.h) * a.dim, a.v_stride, a.dim, keys, j,
                                       limit, false);
                    }
                    order_after();
                    unsigned s[2][32];
                    tensor_load(s_at, s[0]);
                    tensor_load(s_at + 32, s[1]);
                    tensor_wait(s[0]);
                    tensor_wait(s[1]);
                    if (i < walk.sink_steps || j < at.all.max_lo || j + kTile - 1 > at.all.min_hi) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const unsigned seen = seen_keys(keys, j + half * 64 + q * 32, limit);
                            if (__all_sync(0xffffffffu, seen == ~0u)) continue;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!(seen & 1u << e)) s[q][e] = 0xff800000u;  // -infinity
                        }
                    }
                    float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) most[e / 2 % 4] = max_three(most[e / 2 % 4], __uint_as_float(s[q][e]), __uint_as_float(s[q][e + 1]));
                    }
                    most[0] = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
                    most_of[n % 2][half][line] = most[0];
                    __syncwarp();
                    if (lane == 0) arrive_here(maxed + 8 * quarter);
                    if (!await(maxed + 8 * quarter, n)) break;
                    const float largest = fmaxf(most[0], most_of[n % 2][1 - half][line]), product = largest * c;
                    float here = product;
                    // Half precision's smallest numbers are 2^-24: the largest weight is 2^6, and none is above 2^14 before m moves.  (Not where the
                    // rounding of larger scores could take them past its largest number.)
                    if (TypeCode<T>::value == 0 && fabsf(product) < 1048576.0f) here -= 6.0f;
                    const bool grows = here > top + 8.0f;         // (from -infinity: always)
                    if (__any_sync(0xffffffffu, grows)) {
                        const float f = grows ? exp2_fast(top - here) : 1.0f;
                        if (grows) {
                            far = fabsf(fmaf(largest, c, -product)) > 0.5f;
                            rough = rough || far;
                            top = here;
                        }
                        total *= f;
                        if (i > 0) {
#pragma unroll 1
                            for (int d = 0; d < DP / 2; d += 16) {
                                unsigned o[16];
                                tensor_load(o_at + d, o);
                                tensor_wait(o);
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tensor_store(o_at + d, o);
                            }
                        }
                    }
                    const float ref = top == -INFINITY ? 0.0f : top;             // nothing seen yet: exp2 of -infinity is to be zero, not NaN
                    Two sum[2] = {two(0.0f, 0.0f), two(0.0f, 0.0f)};
                    const auto weigh = [&](const auto& weight) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                float x, y;
                                weight(two(s[q] + 2 * e), x, y);
                                sum[e % 2] = add_two(sum[e % 2], two(x, y));
                                s[q][e] = pack_pair(x, y, T{});
                            }
                            tensor_store(s_at + q * 16, reinterpret_cast<const unsigned(&)[16]>(s[q]));
                        }
                    };
                    if (!careful) {
                        weigh([&](Two score, float& x, float& y) { exp2_fast(fma_two(score, two(c, c), two(-ref, -ref)), x, y); });
                    } else {
                        weigh([&](Two score, float& x, float& y) {
                            Two from_top = fma_two(score, two(c, c), two(-ref, -ref));
                            if (far) {
                                apart(score, x, y);
                                from_top = two(__fadd_rn(__fmul_rn(x, c), -ref), __fadd_rn(__fmul_rn(y, c), -ref));
                            }
                            exp2_fast(from_top, x, y);
                            x *= unit;
                            y *= unit;
                        });
                    }
                    tensor_stored();
                    order_before();
                    __syncwarp();
                    if (lane == 0) arrive_here(weighted);
                    float parts[4];
                    apart(sum[0], parts[0], parts[1]);
                    apart(sum[1], parts[2], parts[3]);
                    total += (parts[0] + parts[1]) + (parts[2] + parts[3]);
                }
                if (!ok) break;
                total_of[half][line] = total;
                __syncwarp();
                if (lane == 0) arrive_here(totaled + 8 * quarter);
                if (!await(totaled + 8 * quarter, tile - careful) || !await(summed, tile - careful)) break;
                order_after();
                total = total_of[0][line] + total_of[1][line];
                T* to = static_cast<T*>(a.to[0].p[at.m]) + static_cast<long long>(at.r0 + quarter * 32) * a.out_stride + static_cast<long long>(at.h) * a.dim;
                Infinities more_of{};
                if (careful) more_of.load(mine);
                __syncwarp();
                const bool fine = store_rows<T, kForwardChunk>(o_at, half * (DP / 2), DP / 2, 1.0f / total, stage, to, a.out_stride, a.dim,
                                                               __ballot_sync(0xffffffffu, valid), [&](float (&v)[32], int col) {
                                                                   if (careful) more_of.add(v, col);
                                                               });
                order_before();
                if (half == 0 && valid && a.to[1].p[at.m])
                    static_cast<float*>(a.to[1].p[at.m])[static_cast<long long>(at.h) * a.rows + at.r0 + line] =
                        (TypeCode<T>::value ? top + log2f(total / unit) : (top + 6.0f) + log2f(total / 64.0f)) * kLn2;
                // (a sum of weights that is NaN comes of a score that the row sees: the row is NaN)
                if (!careful && __any_sync(0xffffffffu, valid && (rough || (!fine && !isnan(total)))) && lane == 0) mark_tile(marks, &more, tile);
                place_done(tile);
            }
            if (threadIdx.x == 0) careful_from = n;
        }
        if (warp != 8 && ok) place_done(tile++);
        __syncwarp();
        order_before();
        const bool again = __syncthreads_or(more && !gave_up);
        order_after();
        return again;
    };
    if (walk_tiles(std::false_type{})) walk_tiles(std::true_type{});
    if (gave_up && loads > 0) {                               // copies in flight write shared memory: none is left behind
        tile_wait<kLimit>(loaded, (loads - 1) & 1, nullptr);
        for (int f = max(0, fills - kStages); f < fills; ++f) tile_wait<kLimit>(full + 8 * (f % kStages), (f / kStages) & 1, nullptr);
    }
    if (warp == 9) tensor_free<256>(tmem);
}

// ------------------------------------------------------------------ backward

// -lse (in units of log 2) and -delta = -dout out of every row, in rows of `pitch`, a multiple of 64: rows that belong to no sequence,
// or to no row at all, get -infinity (P = 0) and 0.  For half precision also the longest rows of dout and v, from the last kv_heads
// CTAs along y.  A CTA takes 64 rows of one head.
struct StatsArgs {
    AttentionArgs a;
    float *lse, *delta;
    unsigned* longest;                      // NULL unless half precision; set to 0 before
    long long pitch;
};
constexpr int kStatsThreads = 256;

// LANES a row (8 or 16), each 8 elements of it.
template <typename T, int LANES>
__global__ void __launch_bounds__(kStatsThreads)
attention_stats_kernel(const __grid_constant__ StatsArgs t)
{
    constexpr int kAtOnce = kStatsThreads / LANES, kTurns = 64 / kAtOnce;
    __shared__ float deltas[64];
    __shared__ unsigned most;
    stream_order();
    const AttentionArgs& a = t.a;
    const int r0 = blockIdx.x * 64, m = blockIdx.z, group = threadIdx.x / LANES, word = threadIdx.x % LANES;
    const bool values = static_cast<int>(blockIdx.y) >= a.heads;
    const int h = values ? blockIdx.y - a.heads : blockIdx.y;
    if (threadIdx.x == 0) most = 0;
    if (t.longest) __syncthreads();
    const long long stride = values ? a.v_stride : a.out_stride;
    const T* x = static_cast<const T*>(values ? a.v.p[m] : a.dout.p[m]) + static_cast<long long>(h) * a.dim + word * 8;
    const T* y = static_cast<const T*>(a.out.p[m]) + static_cast<long long>(h) * a.dim + word * 8;
    const long long* offsets = static_cast<const long long*>(a.offsets.p[m]);
    const int begin = offsets ? static_cast<int>(max(0ll, min(static_cast<long long>(a.rows), offsets[0]))) : 0;
    const int end = offsets ? static_cast<int>(max(0ll, min(static_cast<long long>(a.rows), offsets[a.sequences]))) : a.rows;
    uint4 u[kTurns] = {}, v[kTurns] = {};
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int row = r0 + group + kAtOnce * i;
        if (row >= begin && row < end && word * 8 < a.dim) {
            u[i] = *reinterpret_cast<const uint4*>(x + row * stride);
            if (!values) v[i] = *reinterpret_cast<const uint4*>(y + row * stride);
        }
    }
    float longest = 0.0f;
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        float p[8], q[8], dot = 0.0f, square = 0.0f;
        unpack<T>(u[i], p);
        unpack<T>(v[i], q);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dot = fmaf(p[e], q[e], dot);
            square = fmaf(p[e], p[e], square);
        }
        if (!values) dot = lanes_sum<LANES>(dot);
        if (t.longest) {                                      // rows that are not finite do not count: dS of theirs is not either
            square = lanes_sum<LANES>(square);
            if (square < INFINITY) longest = fmaxf(longest, square);
        }
        if (!values && word == 0) deltas[group + kAtOnce * i] = -dot;
    }
    if (t.longest) {
        const unsigned bits = __reduce_max_sync(0xffffffffu, __float_as_uint(longest));
        if (threadIdx.x % 32 == 0) atomicMax(&most, bits);
    }
    __syncthreads();
    if (!values && threadIdx.x < 64) {
        const int row = r0 + threadIdx.x;
        const long long at = (static_cast<long long>(m) * a.heads + h) * t.pitch + row;
        const bool in = row >= begin && row < end;
        t.delta[at] = in ? deltas[threadIdx.x] : 0.0f;
        t.lse[at] = in ? -lse_of(a, m, h, row) : -INFINITY;
    }
    if (t.longest && threadIdx.x == 0) atomicMax(t.longest + 2 * m + (values ? 1 : 0), most);
}

// The power of two that half precision's dS carries: with it the bound of |dS|, twice the product of the longest finite rows
// of dout and v, lies in [2^14, 2^15).
__device__ __forceinline__ int grad_exponent(const TileArgs& t, int m)
{
    if (t.longest == nullptr) return 0;
    const float most = 2.0f * sqrtf(__ldcg(t.longest + 2 * m)) * sqrtf(__ldcg(t.longest + 2 * m + 1));
    if (!(most > 0.0f && most < INFINITY)) return 0;
    return max(-100, min(100, 14 - ilogbf(most)));
}

// The gradient of a sequence's first keys runs over all of its queries.  So that no tile walks much longer than the others, the
// queries are cut into chunks at multiples of kChunk rows, and those from row far_from() on are left to CTAs that take one chunk
// each, with the sequence's first keys as their tile, and write sums in fp32; the tiles that hold those keys add them.  (2 x 16384
// tokens, 16 query heads on 4 of 128, a window of 1024, 4 first keys: 1370 us without, when a window without first keys took 724.)
constexpr int kChunk = 1024;
__device__ __forceinline__ int far_from(const AttentionArgs& a, const Sequence& s)
{
    const long long reach = static_cast<long long>(s.start) + a.sinks + a.left;
    return static_cast<int>(min((reach + kChunk - 1) / kChunk * kChunk, 0x7fffffffll));
}

constexpr int kBackwardThreads = 320;       // warps 0 to 7: rows, 64 columns of a step each; 8: copies, 9: products
constexpr int kStep = 128;                  // rows of a step: products of 64 columns take the tensor cores as long as of 128
constexpr int kBackwardChunk = 32;          // columns of results on their way
template <int DP, bool KEYS> constexpr int kSlotsU = KEYS && DP == 128 ? 2 : 3;   // of the operand that the scores take
template <int DP, bool KEYS> constexpr int kSlotsW = KEYS || DP == 64 ? 2 : 1;    // of the one that dP takes
template <int DP, bool KEYS>
constexpr int kBackwardSmem = (2 + kSlotsU<DP, KEYS> + kSlotsW<DP, KEYS>) * kTile * DP * 2 + (KEYS ? kSlotsU<DP, KEYS> * 2 * kStep * 4 : 0) +
                              8 * 64 * kBackwardChunk + 1024;

// What keys are seen by; where first keys' far queries are set apart (`chunked`), sinks_end is the end of the sequence that has some.
struct KeyRows {
    const AttentionArgs& a;
    bool chunked;
    __device__ __forceinline__ bool operator()(const Sequence& s, int row, Keys& k) const
    {
        if (s.start >= s.end) return false;
        const Queries q = queries_of(a, s, row);
        k = Keys{q.lo, q.hi, s.start, 0};
        if (chunked && row - s.start < a.sinks && far_from(a, s) < s.end) {
            k.hi = far_from(a, s) - 1;
            k.sinks_end = s.end;
        }
        return true;
    }
};

// KEYS: dk and dv of a tile of keys, walking over queries; else dq of a tile of queries, walking over keys.  The scores of a
// step are S = X U^T and dP = Y W^T with the tile's own X and Y; its sums take P W (dv) and dS U (dk, or dq).  While the
// tensor cores work on one of them, the warps turn the other into an operand.
//
// Tensor memory, in columns: KEYS: dv 0, dk 128 (64 with heads of 64), S (then P) 256 (and 128 in turn, with heads of 64), dP (then dS)
// 384.  Else dq 0, S (then dS) 128 and 256 in turn, dP 384.  A warp's half of an operand stands where its half of the scores stood.
// Where there are two places for S, a step's scores are there before the step in front is done: a warp may be through with a step's P while
// another is still at that of the step in front, so each place has a barrier of its own for P.
struct BackwardPlace {                      // steps = -1: there are no more tiles
    int w, m, h, turn, r0, steps, first, turns, from, to, loose;  // KEYS: `turns` steps from row `first` on, for each query head
    Reach all;
    KeyWalk walk;
};
template <typename T, int DP, bool KEYS>
__global__ void __launch_bounds__(kBackwardThreads, 1)
attention_backward_kernel(const __grid_constant__ TileArgs t)
{
    constexpr unsigned long long kLimit = kAttentionWaitNs;
    constexpr bool kHalf = TypeCode<T>::value == 0;
    constexpr float kWeightExponent = kHalf ? 14.0f : 0.0f;               // of two, on P in half precision
    constexpr int kU = kSlotsU<DP, KEYS>, kW = kSlotsW<DP, KEYS>, kBytes = kTile * DP * 2, kHalves = DP / 64, kScoreSets = KEYS && DP == 128 ? 1 : 2;
    constexpr unsigned kTmemSum = KEYS ? DP : 0, kTmemScores = kScoreSets == 1 ? 256 : 128, kTmemGrads = 384;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) unsigned long long bars[2 * kU + 2 * kW + 11 + 2 * kPlaces];
    __shared__ __align__(8) unsigned char place_bytes[kPlaces * sizeof(BackwardPlace)];
    __shared__ unsigned tmem_slot, marks[kMarks / 32];
    __shared__ BadRows bad_u, bad_w;
    __shared__ int gave_up, more, careful_from;               // as in the forward kernel

    const unsigned own = (smem_address(raw) + 1023u) & ~1023u, ring_u = own + 2 * kBytes, ring_w = ring_u + kU * kBytes, out = ring_w + kW * kBytes,
                   stats = out + 8 * 64 * kBackwardChunk;
    const float* stats_at = reinterpret_cast<const float*>(raw + (stats - smem_address(raw)));
    const unsigned full_u = smem_address(bars), empty_u = full_u + 8 * kU, full_w = empty_u + 8 * kU, empty_w = full_w + 8 * kW, loaded = empty_w + 8 * kW,
                   used = loaded + 8, scored = used + 8, graded = scored + 16, weighted = graded + 8, differed = weighted + 16, summed = differed + 8,
                   drain = summed + 8, scanned = drain + 8;
    const PlaceRing<BackwardPlace> places{reinterpret_cast<BackwardPlace*>(place_bytes), scanned + 8, scanned + 8 + 8 * kPlaces};
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x) >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x < kMarks / 32) marks[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        gave_up = more = 0;
        for (int s = 0; s < kU; ++s) { barrier_init(full_u + 8 * s, 1); barrier_init(empty_u + 8 * s, 1); }
        for (int s = 0; s < kW; ++s) { barrier_init(full_w + 8 * s, 1); barrier_init(empty_w + 8 * s, 1); }
        barrier_init(loaded, 1);                              // X and Y are there
        barrier_init(used, 1);                                // they have done their part
        barrier_init(scored, 1);                              // S of a step (in each of its places) is there
        barrier_init(scored + 8, 1);
        barrier_init(graded, 1);                              // dP is there
        barrier_init(weighted, 8);                            // P of a step (in each of the places of S) is there (KEYS)
        barrier_init(weighted + 8, 8);
        barrier_init(differed, 8);                            // dS is there
        barrier_init(summed, 1);                              // a tile's sums are there
        barrier_init(drain, 1);
        barrier_init(scanned, 8);                             // a step has been looked over
        for (int s = 0; s < kPlaces; ++s) { barrier_init(places.there + 8 * s, 1); barrier_init(places.free + 8 * s, 9); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8 && lane < 4 * t.workers) prefetch_map(&t.map[lane % 4][lane / 4]);
    if (warp == 9) tensor_alloc<512>(smem_address(&tmem_slot));
    order_before();
    __syncthreads();
    order_after();
    // The launch in front has waited for all before it, so that a launch that needs nothing of it may run beside it, and waits at its
    // end, before it lets the next one start.  (The fence keeps reads from what the SM may hold of older results.)
    if (t.beside) __threadfence();
    else stream_order();
    const unsigned tmem = tmem_slot;

    const AttentionArgs& a = t.a;
    const bool far = KEYS && t.far;                           // chunks of queries against the first keys of the sequences that they begin in
    const int heads = KEYS ? a.kv_heads : a.heads, tiles = far ? t.chunks : (a.rows + kTile - 1) / kTile, units = tiles * static_cast<int>(t.per.by);
    const auto own_row = [&](const BackwardPlace& at, int row, Keys& keys) {
        if (far) {
            const Sequence s = sequence_of(a, at.m, at.turn * kChunk);
            keys = Keys{at.all.min_lo, at.all.max_hi, s.start, 0};
            return row < s.end && row - s.start < a.sinks;
        }
        return KEYS ? own_keys(a, at.m, row, KeyRows{a, t.partial != nullptr}, keys) : own_keys(a, at.m, row, QueryRows{a}, keys);
    };
    int fills_u = 0, fills_w = 0, loads = 0;                  // of the copying thread
    int placed = 0, tile = 0, n = 0;                          // tiles handed on and taken, steps, in both walks
    bool ok = true;
    const auto await = [&](unsigned bar, int phase) {         // by a whole warp
        ok = ok && __all_sync(0xffffffffu, tile_wait<kLimit>(bar, phase & 1, &gave_up));
        return ok;
    };
    const auto place_there = [&](int tile) { return await(places.there + 8 * (tile % kPlaces), tile / kPlaces) && places[tile].steps >= 0; };
    const auto place_done = [&](int tile) {
        __syncwarp();
        if (lane == 0) arrive_here(places.free + 8 * (tile % kPlaces));
    };

    // All of a CTA's tiles, or with `second` the marked ones; whether there are marked ones.
    const auto walk_tiles = [&](auto second) __attribute__((always_inline)) {
        constexpr bool careful = decltype(second)::value;
        if (warp == 8) {
            const auto copy_tile = [&](unsigned to, const CUtensorMap* map, int head, int r, unsigned bar) {
#pragma unroll
                for (int i = 0; i < 2 * kHalves; ++i) copy_box(to + i * kBoxBytes, map, i / 2 * 64, head, r + i % 2 * kBox, bar);
            };
            int round = 0, met = 0;
            // Works the next tile out and hands it on; without steps it is none.  (The longest walks come first, where there is no window.)
            const auto place_next = [&] {
                BackwardPlace p{0, 0, 0, 0, 0, -1, 0, 0, 0, 0, 0, Reach{}, KeyWalk(Reach{}, 0, kStep)};
                for (; p.steps <= 0 && round * static_cast<int>(gridDim.x) < units; ++round) {
                    const int unit = tile_of_round(round);
                    if (unit >= units) continue;
                    const int turn = t.per.quotient(unit), in = unit - turn * static_cast<int>(t.per.by), w = t.per_worker.quotient(in), m = t.first_worker + w;
                    int r0 = (KEYS ? turn : tiles - 1 - turn) * kTile;
                    Reach all;
                    if (far) {                                    // all first keys see the whole chunk, where it is far from them
                        const Sequence s = sequence_of(a, m, turn * kChunk);
                        r0 = s.start;
                        all = Reach{turn * kChunk, turn * kChunk, min(turn * kChunk + kChunk, s.end) - 1, 0, s.start};
                        all.max_hi = s.start < s.end && turn * kChunk >= far_from(a, s) ? all.min_hi : -1;
                    } else if (KEYS) {
                        all = reach_of(a, m, r0, lane, KeyRows{a, t.partial != nullptr});
                    } else {
                        all = reach_of(a, m, r0, lane, QueryRows{a});
                    }
                    const KeyWalk walk(all, a.sinks, kStep);
                    // queries are walked from a multiple of 64 rows on, where the rows of lse and delta start on 256 bytes
                    const int first = all.min_lo / 64 * 64, turns = all.max_hi >= all.min_lo ? (all.max_hi - first) / kStep + 1 : 0;
                    int from, to;
                    rows_of_sequences(a, m, from, to);
                    p = BackwardPlace{w, m, in - w * heads, turn, r0, KEYS ? turns * a.group : walk.steps, first, turns, from, to, (KEYS && first < from) || (KEYS ? first + turns * kStep : walk.row(walk.steps - 1, kStep) + kStep) > to, all, walk};
                    if (careful && p.steps > 0 && !marked(marks, met++)) p.steps = 0;
                }
                if (p.steps == 0) p.steps = -1;
                if (placed >= kPlaces && !await(places.free + 8 * (placed % kPlaces), placed / kPlaces - 1)) return p;
                if (lane == 0) {
                    places.slots[placed % kPlaces] = p;
                    arrive_here(places.there + 8 * (placed % kPlaces));
                }
                ++placed;
                return p;
            };
            BackwardPlace at = place_next();
            while (ok && at.steps > 0) {
                const BackwardPlace next = place_next();
                const int kv = KEYS ? at.h : a.group_size.quotient(at.h);
                if (ok && lane == 0) {
                    ok = loads == 0 || tile_wait<kLimit>(used, (loads - 1) & 1, &gave_up);
                    if (ok) {
                        barrier_expect(loaded, 2 * kBytes);
                        copy_tile(own, &t.map[KEYS ? 1 : 0][at.w], at.h, at.r0, loaded);             // X: k or q
                        copy_tile(own + kBytes, &t.map[KEYS ? 2 : 3][at.w], at.h, at.r0, loaded);    // Y: v or dout
                        ++loads;
                    }
                    for (int i = 0, turn = 0, hs = KEYS ? kv * a.group : kv; i < at.steps && ok; ++i, ++turn) {
                        if (KEYS && turn == at.turns) turn = 0, ++hs;            // the next query head
                        const int u = fills_u % kU, v = fills_w % kW, r = KEYS ? at.first + turn * kStep : at.walk.row(i, kStep);
                        ok = fills_u < kU || tile_wait<kLimit>(empty_u + 8 * u, (fills_u / kU - 1) & 1, &gave_up);
                        if (!ok) break;
                        barrier_expect(full_u + 8 * u, kBytes + (KEYS ? 2 * kStep * 4 : 0));
                        copy_tile(ring_u + u * kBytes, &t.map[KEYS ? 0 : 1][at.w], hs, r, full_u + 8 * u);
                        if (KEYS) {
                            const long long from = (static_cast<long long>(at.m) * a.heads + hs) * t.pitch + r;
                            copy_floats(stats + u * 2 * kStep * 4, t.lse + from, kStep * 4, full_u + 8 * u);
                            copy_floats(stats + u * 2 * kStep * 4 + kStep * 4, t.delta + from, kStep * 4, full_u + 8 * u);
                        }
                        ++fills_u;
                        ok = fills_w < kW || tile_wait<kLimit>(empty_w + 8 * v, (fills_w / kW - 1) & 1, &gave_up);
                        if (!ok) break;
                        barrier_expect(full_w + 8 * v, kBytes);
                        copy_tile(ring_w + v * kBytes, &t.map[KEYS ? 3 : 2][at.w], hs, r, full_w + 8 * v);
                        ++fills_w;
                    }
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                at = next;
            }
        } else if (warp == 9) {
            constexpr unsigned kTypes = 1u << 4 | TypeCode<T>::value << 7 | TypeCode<T>::value << 10 | (kTile >> 4) << 24;
            constexpr unsigned kScores = kTypes | (kStep >> 3) << 17, kSums = kTypes | 1u << 16 | (DP >> 3) << 17;
            const auto await_product = [&](unsigned bar, int phase) {
                const bool there = await(bar, phase);
                order_after();
                return there;
            };
            // The scores of a step: both operands in shared memory, the sum along the head's elements.
            const auto scores = [&](unsigned to, unsigned tile_at, unsigned slot) {
                const unsigned long long x = matrix_descriptor(tile_at, 16), y = matrix_descriptor(slot, 16);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    const unsigned along = (k / 4 * 2 * kBoxBytes + k % 4 * 32) >> 4;
                    mma_shared(to, x + along, y + along, kScores, k > 0);
                }
            };
            // What a step adds to a sum: 128 columns of scores as 16-bit operands in two halves, the sum along the step's rows.
            const auto add = [&](unsigned to, unsigned from, unsigned slot, bool more) {
                const unsigned long long y = matrix_descriptor(slot, 2 * kBoxBytes);
#pragma unroll
                for (int k = 0; k < kStep / 16; ++k) mma_tensor(to, from + k / 4 * 64 + k % 4 * 8, y + k * (2048 >> 4), kSums, more || k > 0);
            };
            for (; place_there(tile); ++tile) {
                const int steps = places[tile].steps, end = n + steps;
                place_done(tile);
                // Steps are numbered through all tiles here.  The waits for operands come in front of those for the warps, while earlier
                // products run.
                const auto wait_u = [&](int i) { if (i < end) await_product(full_u + 8 * (i % kU), i / kU); };
                const auto wait_w = [&](int i) { if (i < end) await_product(full_w + 8 * (i % kW), i / kW); };
                const auto step_s = [&](int i) {
                    if (i >= end || !ok) return;
                    if (one_lane()) {
                        scores(tmem + kTmemScores + i % kScoreSets * 128, own, ring_u + i % kU * kBytes);
                        mma_done(scored + 8 * (i % kScoreSets));
                    }
                    __syncwarp();
                };
                const auto step_p = [&](int i) {
                    if (i >= end || !ok) return;
                    if (one_lane()) {
                        scores(tmem + kTmemGrads, own + kBytes, ring_w + i % kW * kBytes);
                        mma_done(graded);
                        if (!KEYS) mma_done(empty_w + 8 * (i % kW));
                        if (i + 1 == end) mma_done(used);         // (the last scores have gone before)
                    }
                    __syncwarp();
                };
                await_product(loaded, tile - careful);
                wait_u(n);
                step_s(n);
                if (kScoreSets == 2) {
                    wait_u(n + 1);
                    step_s(n + 1);
                }
                wait_w(n);
                step_p(n);
                for (int i = n; i < end && ok; ++i) {
                    if (KEYS) {
                        if (kScoreSets == 1) wait_u(i + 1);
                        if (!await_product(weighted + 8 * (i % kScoreSets), i / kScoreSets)) break;
                        if (one_lane()) {
                            add(tmem, tmem + kTmemScores + i % kScoreSets * 128, ring_w + i % kW * kBytes, i > n);
                            mma_done(empty_w + 8 * (i % kW));
                        }
                        __syncwarp();
                        if (kScoreSets == 2) wait_u(i + 2);
                        step_s(i + kScoreSets);
                        wait_w(i + 1);
                        if (!await_product(differed, i)) break;
                        if (one_lane()) {
                            add(tmem + kTmemSum, tmem + kTmemGrads, ring_u + i % kU * kBytes, i > n);
                            mma_done(empty_u + 8 * (i % kU));
                            if (i + 1 == end) mma_done(summed);
                        }
                        __syncwarp();
                        step_p(i + 1);
                    } else {
                        wait_w(i + 1);
                        if (!await_product(differed, i)) break;
                        if (one_lane()) {
                            add(tmem + kTmemSum, tmem + kTmemScores + i % 2 * 128, ring_u + i % kU * kBytes, i > n);
                            mma_done(empty_u + 8 * (i % kU));
                            if (i + 1 == end) mma_done(summed);
                        }
                        __syncwarp();
                        step_p(i + 1);
                        wait_u(i + 2);                            // (its slot has only been free since the step before's sum)
                        step_s(i + 2);
                    }
                }
                if (!ok) break;
                n = end;
            }
            if (!ok) {
                if (one_lane()) mma_done(drain);
                __syncwarp();
                tile_wait<kLimit>(drain, 0, nullptr);
            }
        } else if (warp < 8) {
            const int quarter = warp % 4, half = warp / 4;
            const unsigned lanes = static_cast<unsigned>(quarter * 32) << 16;
            unsigned char* const stage = raw + (out - smem_address(raw)) + warp * 64 * kBackwardChunk;
            const float c = a.scale * kLog2e;
            unsigned* const mine = reinterpret_cast<unsigned*>(stage) + lane * 8;          // of Infinities
            for (; place_there(tile); ++tile) {
                const BackwardPlace& at = places[tile];
                const KeyWalk walk = at.walk;
                const int first = at.first, turns = at.turns, steps = at.steps;
                // some of the rows that are walked over belong to no sequence
                const bool loose = at.loose;
                const int row = at.r0 + quarter * 32 + lane;
                Keys keys{};
                const bool valid = own_row(at, row, keys);
                const int exponent = kHalf ? grad_exponent(t, at.m) : 0;
                const float to_grad = kHalf ? exp2f(static_cast<float>(exponent) - kWeightExponent) : 1.0f;
                if (careful)
                    for (int e = 0; e < 8; ++e) mine[e] = 0;
                float lse = 0.0f, delta = 0.0f;
                if (!KEYS && valid) {
                    const long long from = (static_cast<long long>(at.m) * a.heads + at.h) * t.pitch + row;
                    lse = __ldcg(t.lse + from) + static_cast<float>(exponent);  // P with dS's power of two
                    delta = __ldcg(t.delta + from);
                }
                for (int i = 0, turn = 0; i < steps; ++i, ++n, ++turn) {
                    if (KEYS && turn == turns) turn = 0;
                    const unsigned s_at = tmem + kTmemScores + n % kScoreSets * 128 + half * 64 + lanes, g_at = tmem + kTmemGrads + half * 64 + lanes;
                    const int r = KEYS ? first + turn * kStep : walk.row(i, kStep), limit = !KEYS && i < walk.sink_steps ? at.all.min_lo : 0x7fffffff;
                    const bool masked = (!KEYS && i < walk.sink_steps) || r < at.all.max_lo || r + kStep - 1 > at.all.min_hi;
                    const float* column = stats_at + n % kU * 2 * kStep + half * 64;
                    if (!await(scored + 8 * (n % kScoreSets), n / kScoreSets)) break;
                    if (KEYS && !await(full_u + 8 * (n % kU), n / kU)) break;      // (long past: for the sight of lse and delta)
                    // (The products that made S, and dP of the operand that dv takes, are through with what is set to zero here.)
                    if (!careful && loose) {
                        const int from = at.from - r, to = at.to - r;
                        const unsigned bar_u = full_u + 8 * (n % kU), bar_w = full_w + 8 * (n % kW);
                        ok = zero_loose_rows<DP>(from, to, raw + (ring_u - smem_address(raw)) + n % kU * kBytes, bar_u, n / kU, bar_u, n / kU, &gave_up) &&
                             (!KEYS || zero_loose_rows<DP>(from, to, raw + (ring_w - smem_address(raw)) + n % kW * kBytes, bar_w, n / kW, graded, n, &gave_up));
                        if (!ok) break;
                    }
                    if (careful) {
                        if (KEYS ? !await(full_w + 8 * (n % kW), n / kW) || !await(graded, n) : !await(full_u + 8 * (n % kU), n / kU)) break;
                        const unsigned rows_u = zero_not_finite<T, DP>(raw + (ring_u - smem_address(raw)) + n % kU * kBytes);
                        const unsigned rows_w = KEYS ? zero_not_finite<T, DP>(raw + (ring_w - smem_address(raw)) + n % kW * kBytes) : 0;
                        if (lane == 0) {
                            bad_u[n % 2][warp] = static_cast<unsigned short>(rows_u);
                            bad_w[n % 2][warp] = static_cast<unsigned short>(rows_w);
                            arrive_here(scanned);
                        }
                        if (!await(scanned, n - careful_from)) break;
                        const long long head = KEYS ? at.h * a.group + i / turns : a.group_size.quotient(at.h);
                        if (KEYS && half == 0)
                            add_infinities(mine, bad_w[n % 2], static_cast<const T*>(a.dout.p[at.m]) + r * a.out_stride + head * a.dim, a.out_stride, a.dim,
                                           Keys{keys.lo, keys.hi, 0, 0}, r, limit, false);
                        else if (KEYS)
                            add_infinities(mine, bad_u[n % 2], static_cast<const T*>(a.q.p[at.m]) + r * a.q_stride + head * a.dim, a.q_stride, a.dim,
                                           Keys{keys.lo, keys.hi, 0, 0}, r, limit, true);
                        else
                            add_infinities(mine, bad_u[n % 2], static_cast<const T*>(a.k.p[at.m]) + r * a.k_stride + head * a.dim, a.k_stride, a.dim, keys, r, limit, true);
                    }
                    order_after();
                    Two p[2][16];
                    unsigned seen[2] = {~0u, ~0u};
                    ulonglong2 columns = {0, 0};                  // what four neighbouring columns' queries share
                    {
                        unsigned s[2][32];
                        tensor_load(s_at, s[0]);
                        tensor_load(s_at + 32, s[1]);
                        tensor_wait(s[0]);
                        tensor_wait(s[1]);
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            if (masked) {
                                const int from = r + half * 64 + q * 32;
                                seen[q] = KEYS ? bits_between(keys.lo - from, keys.hi - from) : seen_keys(keys, from, limit);
                            }
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                Two shift = two(lse, lse);
                                if (KEYS) {
                                    if (e % 2 == 0) columns = *reinterpret_cast<const ulonglong2*>(column + q * 32 + 2 * e);
                                    shift.v = e % 2 ? columns.y : columns.x;
                                    if (kHalf) shift = add_two(shift, two(kWeightExponent, kWeightExponent));
                                }
                                float x, y;
                                exp2_fast(fma_two(two(s[q] + 2 * e), two(c, c), shift), x, y);
                                if (masked) {
                                    x = seen[q] & 1u << (2 * e) ? x : 0.0f;
                                    y = seen[q] & 2u << (2 * e) ? y : 0.0f;
                                }
                                p[q][e] = two(x, y);
                                s[q][e] = pack_pair(x, y, T{});
                            }
                            if (KEYS) tensor_store(s_at + q * 16, reinterpret_cast<const unsigned(&)[16]>(s[q]));
                        }
                    }
                    if (KEYS) {
                        tensor_stored();
                        order_before();
                        __syncwarp();
                        if (lane == 0) arrive_here(weighted + 8 * (n % kScoreSets));
                    }
                    if (!await(graded, n)) break;
                    order_after();
                    {
                        unsigned g[2][32];
                        tensor_load(g_at, g[0]);
                        tensor_load(g_at + 32, g[1]);
                        tensor_wait(g[0]);
                        tensor_wait(g[1]);
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                Two shift = two(delta, delta);
                                if (KEYS) {
                                    if (e % 2 == 0) columns = *reinterpret_cast<const ulonglong2*>(column + kStep + q * 32 + 2 * e);
                                    shift.v = e % 2 ? columns.y : columns.x;
                                }
                                Two d = mul_two(p[q][e], add_two(two(g[q] + 2 * e), shift));
                                if (KEYS && kHalf) d = mul_two(d, two(to_grad, to_grad));
                                float x, y;
                                apart(d, x, y);
                                if (masked) {                     // (0 times what is not finite)
                                    x = seen[q] & 1u << (2 * e) ? x : 0.0f;
                                    y = seen[q] & 2u << (2 * e) ? y : 0.0f;
                                }
                                g[q][e] = pack_pair(x, y, T{});
                            }
                            tensor_store((KEYS ? g_at : s_at) + q * 16, reinterpret_cast<const unsigned(&)[16]>(g[q]));
                        }
                    }
                    tensor_stored();
                    order_before();
                    __syncwarp();
                    if (lane == 0) arrive_here(differed);
                }
                if (!await(summed, tile - careful)) break;
                order_after();
                const float of_grad = a.scale * (kHalf ? exp2f(static_cast<float>(-exponent)) : 1.0f);
                const unsigned rows_valid = __ballot_sync(0xffffffffu, valid);
                Infinities more_of{};
                if (careful) more_of.load(mine);
                __syncwarp();
                const auto infinities = [&](float (&v)[32], int col) {
                    if (careful) more_of.add(v, col);
                };
                bool fine = true;
                if (KEYS) {                                       // half of the warps dv, the others dk
                    const long long partial_row = static_cast<long long>(a.sinks) * a.dim, partial_chunk = 2 * partial_row;
                    const long long partial_head = (static_cast<long long>(at.m) * a.kv_heads + at.h) * t.chunks * partial_chunk + half * partial_row;
                    if (far) {
                        float* to = t.partial + partial_head + at.turn * partial_chunk + static_cast<long long>(row - keys.start) * a.dim;
#pragma unroll 1
                        for (int d = 0; d < DP; d += 32) {
                            unsigned bits[32];
                            tensor_load(tmem + half * kTmemSum + lanes + d, bits);
                            tensor_wait(bits);
                            float v[32];
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(bits[e]);
                            infinities(v, d);
#pragma unroll
                            for (int e = 0; e < 32; ++e) fine = fine && fabsf(v[e]) <= 3.0e38f;
#pragma unroll
                            for (int e = 0; e < 32; e += 8)
                                if (valid && d + e < a.dim) store_eight(to + d + e, v + e);
                        }
                    } else {
                        const int from_chunk = (keys.hi + 1) / kChunk, to_chunk = valid && keys.sinks_end > 0 ? (keys.sinks_end - 1) / kChunk + 1 : 0;
                        const auto add = [&](float (&v)[32], int col) {
                            for (int k = from_chunk; k < to_chunk; ++k) {
                                const float* more = t.partial + partial_head + k * partial_chunk + static_cast<long long>(row - keys.start) * a.dim + col;
#pragma unroll
                                for (int e = 0; e < 32; e += 4)
                                    if (col + e < a.dim) {
                                        const float4 x = *reinterpret_cast<const float4*>(more + e);
                                        v[e] += x.x; v[e + 1] += x.y; v[e + 2] += x.z; v[e + 3] += x.w;
                                    }
                            }
                            infinities(v, col);
                        };
                        const long long stride = half ? a.k_stride : a.v_stride;
                        T* to = static_cast<T*>(a.to[half ? 1 : 2].p[at.m]) + (at.r0 + quarter * 32) * stride + static_cast<long long>(at.h) * a.dim;
                        fine = store_rows<T, kBackwardChunk>(tmem + half * kTmemSum + lanes, 0, DP, half ? of_grad : exp2f(-kWeightExponent), stage, to, stride, a.dim,
                                                             rows_valid, add);
                    }
                } else {                                          // half of the columns each
                    const int d = half * (DP / 2);
                    T* to = static_cast<T*>(a.to[0].p[at.m]) + (at.r0 + quarter * 32) * a.q_stride + static_cast<long long>(at.h) * a.dim;
                    fine = store_rows<T, kBackwardChunk>(tmem + d + lanes, d, DP / 2, of_grad, stage, to, a.q_stride, a.dim, rows_valid, infinities);
                }
                if (!careful && __any_sync(0xffffffffu, valid && !fine) && lane == 0) mark_tile(marks, &more, tile);
                order_before();
                place_done(tile);
            }
            if (threadIdx.x == 0) careful_from = n;
        }
        if (warp != 8 && ok) place_done(tile++);
        __syncwarp();
        order_before();
        const bool again = __syncthreads_or(more && !gave_up);
        order_after();
        return again;
    };
    if (walk_tiles(std::false_type{})) walk_tiles(std::true_type{});
    if (gave_up && loads > 0) {                               // copies in flight write shared memory: none is left behind
        tile_wait<kLimit>(loaded, (loads - 1) & 1, nullptr);
        for (int f = max(0, fills_u - kU); f < fills_u; ++f) tile_wait<kLimit>(full_u + 8 * (f % kU), (f / kU) & 1, nullptr);
        for (int f = max(0, fills_w - kW); f < fills_w; ++f) tile_wait<kLimit>(full_w + 8 * (f % kW), (f / kW) & 1, nullptr);
    }
    if (warp == 9) tensor_free<512>(tmem);
    if (t.beside) stream_order();
}

}  // namespace replica
}  // namespace grawa

// Attention within a window: its formulas, and what a query sees.
//
// Sequences lie behind each other in a worker's rows.  Query i of the sequence [start, end) sees key j of the same sequence
// when  j <= i + right  and  (j >= i - left  or  j < start + sinks).  So a query's keys are one run of rows and some of the
// sequence's first ones, and a key's queries are one run of rows:
//   keys of i     [lo, hi] and [start, sinks_end),  lo = max(start, i - left), hi = min(end - 1, i + right), sinks_end <= lo
//   queries of j  [lo, hi],  lo = max(start, j - right), hi = end - 1 for a first key, else min(end - 1, j + left)
//
//   forward   S_ij = scale q_i k_j,  lse_i = log sum_j exp S_ij,  P_ij = exp(S_ij - lse_i),  out_i = sum_j P_ij v_j
//   backward  delta_i = dout_i out_i,  dS_ij = P_ij (dout_i v_j - delta_i),
//             dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij dout_i
// (k_j and v_j of a head are those of key head  head / (heads / kv_heads); a key's sums run over all of its query heads).
#pragma once
#include "replica_common.cuh"

namespace grawa {
namespace replica {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Division by a number that the host knows, of numbers below 2^31 (round-up multiplier of 33 bits, whose highest is the number itself).
struct Divisor {
    unsigned by, multiplier, shift;
    __device__ __forceinline__ int quotient(int n) const { return static_cast<int>((__umulhi(static_cast<unsigned>(n), multiplier) + static_cast<unsigned>(n)) >> shift); }
    __device__ __forceinline__ int remainder(int n) const { return n - quotient(n) * static_cast<int>(by); }
};
inline Divisor divisor(unsigned by)
{
    unsigned shift = 0;
    while ((1ull << shift) < by) ++shift;
    return {by, static_cast<unsigned>(((1ull << 32) * ((1ull << shift) - by)) / by + 1), shift};
}

struct AttentionArgs {
    In q, k, v, dout, out, lse;             // dout, out (as stored by the forward call) and lse in the backward pass
    Out to[3];                              // forward: out, lse (may be NULL); backward: dq, dk, dv
    In offsets;                             // 64-bit integers, or NULL: sequences of `period` rows
    long long q_stride, k_stride, v_stride, out_stride;      // elements from row to row; dq has q's, dk k's, dv v's, dout out's
    int rows, heads, kv_heads, group, dim;  // group: query heads of a key head
    int sequences;
    Divisor period, group_size;
    int left, right, sinks;                 // each at most `rows`
    float scale;
};

struct Sequence { int start, end; };        // start > end - 1: the row belongs to none

// The sequence of a row.  Offsets that decrease or leave the rows give some run of rows that holds this one.
__device__ __forceinline__ Sequence sequence_of(const AttentionArgs& a, int m, int row)
{
    const long long* offsets = static_cast<const long long*>(a.offsets.p[m]);
    if (offsets == nullptr) {
        const int start = row - a.period.remainder(row), length = static_cast<int>(a.period.by);
        return {start, length > a.rows - start ? a.rows : start + length};
    }
    if (row >= a.rows || offsets[0] > row || offsets[a.sequences] <= row) return {0, 0};
    int lo = 0, hi = a.sequences;           // offsets[lo] <= row < offsets[hi]
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (offsets[mid] <= row) lo = mid;
        else hi = mid;
    }
    const long long start = offsets[lo], end = offsets[hi];
    return {start < 0 ? 0 : static_cast<int>(start), end > a.rows ? a.rows : static_cast<int>(end)};
}

struct Keys { int lo, hi, start, sinks_end; };
__device__ __forceinline__ Keys keys_of(const AttentionArgs& a, const Sequence& s, int i)
{
    Keys k;
    k.start = s.start;
    k.lo = a.left >= i - s.start ? s.start : i - a.left;
    k.hi = a.right >= s.end - 1 - i ? s.end - 1 : i + a.right;
    k.sinks_end = a.sinks >= k.lo - s.start ? k.lo : s.start + a.sinks;
    return k;
}
struct Queries { int lo, hi; };
__device__ __forceinline__ Queries queries_of(const AttentionArgs& a, const Sequence& s, int j)
{
    const bool first = j - s.start < a.sinks;
    return {a.right >= j - s.start ? s.start : j - a.right, first || a.left >= s.end - 1 - j ? s.end - 1 : j + a.left};
}

// lse of a row, in units of log 2.
__device__ __forceinline__ float lse_of(const AttentionArgs& a, int m, int h, int i)
{
    return static_cast<const float*>(a.lse.p[m])[static_cast<long long>(h) * a.rows + i] * kLog2e;
}

}  // namespace replica
}  // namespace grawa

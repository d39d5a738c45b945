// Attention within a window, row by row: what a query sees, and a warp's way from one row of the operands to one row of the
// results, in fp32 throughout, for the rows that the tensor cores cannot have right (attention.cuh).
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

// ------------------------------------------------------------------ a warp's rows

// Lane l holds elements 4 l to 4 l + 3 of a row of up to 128 (a multiple of 8).
template <typename T>
__device__ __forceinline__ void load_row(const void* base, long long stride, int row, int head, int dim, float (&x)[4])
{
    const int at = threadIdx.x % 32 * 4;
    if (at < dim) {
        const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const T*>(base) + row * stride + static_cast<long long>(head) * dim + at);
        unpack_pair(w.x, x, T{});
        unpack_pair(w.y, x + 2, T{});
    } else {
        x[0] = x[1] = x[2] = x[3] = 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store_row(void* base, long long stride, int row, int head, int dim, const float (&x)[4], int from, int to)
{
    const int at = threadIdx.x % 32 * 4;
    if (at < dim && at >= from && at < to)
        *reinterpret_cast<uint2*>(static_cast<T*>(base) + row * stride + static_cast<long long>(head) * dim + at) =
            make_uint2(pack_pair(x[0], x[1], T{}), pack_pair(x[2], x[3], T{}));
}
__device__ __forceinline__ float dot_row(const float (&x)[4], const float (&y)[4])
{
    return lanes_sum<32>(fmaf(x[0], y[0], fmaf(x[1], y[1], fmaf(x[2], y[2], x[3] * y[3]))));
}
__device__ __forceinline__ void add_row(float (&x)[4], float f, const float (&y)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = fmaf(f, y[e], x[e]);
}

__device__ __forceinline__ bool any_nan(const float (&x)[4])
{
    return __any_sync(0xffffffffu, isnan(x[0]) || isnan(x[1]) || isnan(x[2]) || isnan(x[3]));
}
__device__ __forceinline__ void fill_row(float (&x)[4], float v) { x[0] = x[1] = x[2] = x[3] = v; }

// Calls f for the rows [begin, end), kRowsAtOnce at a time (the last ones may lie behind the end), so that what they wait for overlaps; until
// all of the sums that it makes are NaN, which they stay.
constexpr int kRowsAtOnce = 4;
template <typename F>
__device__ __forceinline__ void for_rows(int begin, int end, int dim, const float (&sum)[4], const F& f)
{
    const bool none = threadIdx.x % 32 * 4 >= static_cast<unsigned>(dim);
    for (int j = begin; j < end; j += kRowsAtOnce) {
        f(j);
        if (__all_sync(0xffffffffu, none || (isnan(sum[0]) && isnan(sum[1]) && isnan(sum[2]) && isnan(sum[3])))) return;
    }
}

// Elements [from, to) of out_i, and with the first of them lse_i.  (Where q_i holds NaN, all of it is.)
template <typename T>
__device__ __noinline__ void attention_row(const AttentionArgs& a, int m, int h, int i, int from, int to)
{
    const Keys keys = keys_of(a, sequence_of(a, m, i), i);
    const float c = a.scale * kLog2e;
    float q[4], o[4] = {}, top = -INFINITY, total = 0.0f;
    load_row<T>(a.q.p[m], a.q_stride, i, h, a.dim, q);
    if (any_nan(q)) {
        total = NAN;
    } else {
        for (int part = 0; part < 2; ++part) {
            const int end = part ? keys.hi + 1 : keys.sinks_end;
            for_rows(part ? keys.lo : keys.start, end, a.dim, o, [&](int j) {
                float k[kRowsAtOnce][4], v[kRowsAtOnce][4], s[kRowsAtOnce], next = top;
#pragma unroll
                for (int r = 0; r < kRowsAtOnce; ++r) {
                    load_row<T>(a.k.p[m], a.k_stride, min(j + r, end - 1), h / a.group, a.dim, k[r]);
                    load_row<T>(a.v.p[m], a.v_stride, min(j + r, end - 1), h / a.group, a.dim, v[r]);
                }
#pragma unroll
                for (int r = 0; r < kRowsAtOnce; ++r) {
                    s[r] = dot_row(q, k[r]) * c;
                    if (j + r < end) next = fmaxf(next, s[r]);
                }
                const float ref = next == -INFINITY ? 0.0f : next, f = exp2f(top - ref);
                total *= f;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] *= f;
#pragma unroll
                for (int r = 0; r < kRowsAtOnce; ++r)
                    if (j + r < end) {
                        const float p = exp2f(s[r] - ref);
                        total += p;
                        add_row(o, p, v[r]);
                    }
                top = next;
            });
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] /= total;
    store_row<T>(a.to[0].p[m], a.out_stride, i, h, a.dim, o, from, to);
    if (a.to[1].p[m] && from == 0 && threadIdx.x % 32 == 0) static_cast<float*>(a.to[1].p[m])[static_cast<long long>(h) * a.rows + i] = (top + log2f(total)) * kLn2;
}

template <typename T>
__device__ __forceinline__ float delta_of(const AttentionArgs& a, int m, int h, int i, const float (&dout)[4])
{
    float out[4];
    load_row<T>(a.out.p[m], a.out_stride, i, h, a.dim, out);
    return dot_row(dout, out);
}
__device__ __forceinline__ float lse_of(const AttentionArgs& a, int m, int h, int i)
{
    return static_cast<const float*>(a.lse.p[m])[static_cast<long long>(h) * a.rows + i] * kLog2e;
}

// Elements [from, to) of dq_i.  (Where q_i or dout_i holds NaN, all of it is.)
template <typename T>
__device__ __noinline__ void attention_query_grad_row(const AttentionArgs& a, int m, int h, int i, int from, int to)
{
    const Keys keys = keys_of(a, sequence_of(a, m, i), i);
    const float c = a.scale * kLog2e, lse = lse_of(a, m, h, i);
    float q[4], dout[4], dq[4] = {};
    load_row<T>(a.q.p[m], a.q_stride, i, h, a.dim, q);
    load_row<T>(a.dout.p[m], a.out_stride, i, h, a.dim, dout);
    const float delta = delta_of<T>(a, m, h, i, dout);
    if (any_nan(q) || isnan(delta) || isnan(lse)) {
        fill_row(dq, NAN);
    } else {
        for (int part = 0; part < 2; ++part) {
            const int end = part ? keys.hi + 1 : keys.sinks_end;
            for_rows(part ? keys.lo : keys.start, end, a.dim, dq, [&](int j) {
                float k[kRowsAtOnce][4], v[kRowsAtOnce][4];
#pragma unroll
                for (int r = 0; r < kRowsAtOnce; ++r) {
                    load_row<T>(a.k.p[m], a.k_stride, min(j + r, end - 1), h / a.group, a.dim, k[r]);
                    load_row<T>(a.v.p[m], a.v_stride, min(j + r, end - 1), h / a.group, a.dim, v[r]);
                }
#pragma unroll
                for (int r = 0; r < kRowsAtOnce; ++r) {
                    const float ds = exp2f(dot_row(q, k[r]) * c - lse) * (dot_row(dout, v[r]) - delta);
                    if (j + r < end) add_row(dq, ds, k[r]);
                }
            });
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) dq[e] *= a.scale;
    store_row<T>(a.to[0].p[m], a.q_stride, i, h, a.dim, dq, from, to);
}

// dk_j, or dv_j.  (Where k_j holds NaN, or v_j for dk_j, all of it is.)
template <typename T>
__device__ __noinline__ void attention_key_grad_row(const AttentionArgs& a, int m, int kv, int j, bool want_k)
{
    const Queries queries = queries_of(a, sequence_of(a, m, j), j);
    const float c = a.scale * kLog2e;
    float k[4], v[4], sum[4] = {};
    load_row<T>(a.k.p[m], a.k_stride, j, kv, a.dim, k);
    load_row<T>(a.v.p[m], a.v_stride, j, kv, a.dim, v);
    if (any_nan(k) || (want_k && any_nan(v))) {
        fill_row(sum, NAN);
    } else {
        for (int h = kv * a.group; h < (kv + 1) * a.group; ++h)
            for_rows(queries.lo, queries.hi + 1, a.dim, sum, [&](int i) {
                float q[kRowsAtOnce][4], dout[kRowsAtOnce][4];
#pragma unroll
                for (int r = 0; r < kRowsAtOnce; ++r) {
                    load_row<T>(a.q.p[m], a.q_stride, min(i + r, queries.hi), h, a.dim, q[r]);
                    load_row<T>(a.dout.p[m], a.out_stride, min(i + r, queries.hi), h, a.dim, dout[r]);
                }
#pragma unroll
                for (int r = 0; r < kRowsAtOnce; ++r) {
                    const int at = min(i + r, queries.hi);
                    const float p = exp2f(dot_row(q[r], k) * c - lse_of(a, m, h, at));
                    const float ds = want_k ? p * (dot_row(dout[r], v) - delta_of<T>(a, m, h, at, dout[r])) : 0.0f;
                    if (i + r <= queries.hi) add_row(sum, want_k ? ds : p, want_k ? q[r] : dout[r]);
                }
            });
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] *= want_k ? a.scale : 1.0f;
    store_row<T>(a.to[want_k ? 1 : 2].p[m], want_k ? a.k_stride : a.v_stride, j, kv, a.dim, sum, 0, a.dim);
}

}  // namespace replica
}  // namespace grawa

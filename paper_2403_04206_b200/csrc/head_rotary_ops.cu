// Host side of the head norms with rotation: argument checks, the choice of a kernel, launches, and their part of the C ABI in
// include/grawa.h.  No call allocates device memory or keeps anything from one call to the next.
#include <cmath>
#include <type_traits>

#include "head_rotary.cuh"
#include "replica_host.h"

namespace grawa {
namespace replica {

// What both directions are told about the heads.
struct HeadShape {
    grawa_dtype dtype;
    grawa_pairing pairing;
    int64_t rows, q_heads, k_heads, head_dim, rotary;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
    const int64_t* const* positions;
    const double* frequencies;
    int64_t period;
    int M;
    float eps;
};

static bool head_shape_ok(const HeadShape& s)
{
    constexpr int64_t kMostHeads = 1 << 16;
    if (!dtype_known(s.dtype) || (s.pairing != GRAWA_PAIR_HALVES && s.pairing != GRAWA_PAIR_NEIGHBOURS) || s.M < 1 || s.M > GRAWA_MAX_WORKERS) return false;
    if (s.rows < 0 || s.rows > 0x7fffffff || s.q_heads < 1 || s.q_heads > kMostHeads || s.k_heads < 0 || s.k_heads > kMostHeads) return false;
    if (s.head_dim < 1 || s.head_dim > kHeadDim || s.rotary < 0 || s.rotary > s.head_dim || s.rotary % 2 != 0) return false;
    if (!stride_ok(s.rows, s.q_heads * s.head_dim, s.q_stride) || !stride_ok(s.rows, s.q_heads * s.head_dim, s.q_out_stride)) return false;
    if (s.k_heads && (!stride_ok(s.rows, s.k_heads * s.head_dim, s.k_stride) || !stride_ok(s.rows, s.k_heads * s.head_dim, s.k_out_stride))) return false;
    if (!(s.eps >= 0.0f) || std::isinf(s.eps)) return false;
    if (s.rotary && (!s.frequencies || !aligned(s.frequencies, 8) || (!s.positions && s.period < 1))) return false;
    return true;
}

// The buffers that both directions read beside their heads.
static bool add_head_inputs(Buffers& b, const HeadShape& s, const void* const* q_weight, const void* const* k_weight)
{
    const int64_t elem = type_bytes(s.dtype);
    if (q_weight && !b.add(q_weight, s.M, 1, s.head_dim, s.head_dim, elem, false)) return false;
    if (s.k_heads && k_weight && !b.add(k_weight, s.M, 1, s.head_dim, s.head_dim, elem, false)) return false;
    if (s.rotary == 0) return true;
    const void* f = s.frequencies;
    if (!b.add(&f, 1, 1, s.rotary / 2, s.rotary / 2, 8, false)) return false;
    return !s.positions || b.add(reinterpret_cast<const void* const*>(s.positions), s.M, 1, s.rows, s.rows, 8, false);
}

// Heads that are read, and written in place or elsewhere: `in` may be the same buffer as `out` where their strides are equal.
static bool add_in_and_out(Buffers& b, const void* const* in, int64_t in_stride, void* const* out, int64_t out_stride, const HeadShape& s, int64_t heads)
{
    const int64_t elem = type_bytes(s.dtype), cols = heads * s.head_dim;
    const void* apart[GRAWA_MAX_WORKERS];
    int others = 0;
    for (int m = 0; m < s.M; ++m)
        if (!out || in[m] != out[m] || (s.rows > 1 && in_stride != out_stride)) apart[others++] = in[m];
    return b.add(apart, others, s.rows, cols, in_stride, elem, false) && (!out || b.add(out, s.M, s.rows, cols, out_stride, elem, true));
}

static HeadArgs head_args(const HeadShape& s, const void* const* q, const void* const* k, const void* const* q_weight, const void* const* k_weight)
{
    HeadArgs a{};
    copy_table(a.x[0], q, s.M);
    copy_table(a.w[0], q_weight, s.M);
    if (s.k_heads) {
        copy_table(a.x[1], k, s.M);
        copy_table(a.w[1], k_weight, s.M);
    }
    if (s.rotary) copy_table(a.positions, s.positions, s.M);
    a.frequencies = s.frequencies;
    a.rows = static_cast<unsigned>(s.rows); a.period = static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(s.period, 0x7fffffff)));
    a.x_stride[0] = s.q_stride; a.x_stride[1] = s.k_stride;
    a.y_stride[0] = s.q_out_stride; a.y_stride[1] = s.k_out_stride;
    a.heads[0] = static_cast<int>(s.q_heads); a.heads[1] = static_cast<int>(s.k_heads);
    a.dim = static_cast<int>(s.head_dim); a.half = static_cast<int>(s.rotary / 2);
    a.neighbours = s.pairing == GRAWA_PAIR_NEIGHBOURS;
    a.words = static_cast<int>(s.head_dim * type_bytes(s.dtype) / 16);
    a.has_w[0] = q_weight != nullptr; a.has_w[1] = k_weight != nullptr;
    a.eps = s.eps; a.inv_dim = 1.0f / static_cast<float>(s.head_dim);
    a.small = s.eps < 0x1p-80f ? 0x12800000u : 0u;            // 2^-90: squares that are missing are below 2^-149 each
    return a;
}

// How the heads are held by the lanes: in whole 16-byte words where all rows, heads and rotated halves are made of them.
static HeadMode head_mode(const HeadArgs& a, grawa_dtype dtype, int M, bool backward)
{
    const int64_t elem = type_bytes(dtype), word = 16 / elem;
    bool whole = a.dim % word == 0;
    for (int i = 0; i < 2 && whole; ++i) {
        if (a.heads[i] == 0) continue;
        whole = all_aligned(a.x[i].p, M, 16) && all_aligned(a.y[i].p, M, 16) && (!backward || all_aligned(a.dy[i].p, M, 16));
        if (a.rows > 1) whole = whole && a.x_stride[i] % word == 0 && a.y_stride[i] % word == 0;
    }
    if (whole && a.neighbours) return kPairNext;
    if (whole && a.half % word == 0) return kPairWords;
    return a.dim <= 128 ? kPairAnyShort : kPairAny;
}

// Calls f with the number of lanes a head takes, each of which holds two of its words.
template <typename T, typename F>
static grawa_status with_lanes(int words, const F& f)
{
    if (words <= 4) return f(std::integral_constant<int, 2>{});
    if (words <= 8) return f(std::integral_constant<int, 4>{});
    if (words <= 16) return f(std::integral_constant<int, 8>{});
    if (words <= 32) return f(std::integral_constant<int, 16>{});
    return f(std::integral_constant<int, sizeof(T) == 4 ? 32 : 16>{});     // (16-bit heads have up to 32 words)
}

constexpr int kHeadCtas = 4;                                  // an SM's, at most: some turns of each
template <typename T>
static grawa_status head_forward(HeadArgs& a, int M, HeadMode mode, cudaStream_t stream)
{
    const auto run = [&](auto kernel, int per) {
        constexpr int kWarps = kHeadThreads / 32;
        const int64_t steps = ceil_div(a.heads[0], per) + ceil_div(a.heads[1], per);
        // rows whose warps would not fill the SMs are shared out among several each, down to one step of `per` heads
        const int64_t want = std::max<int64_t>(1, std::min<int64_t>(steps, int64_t{kSms} * 32 / (int64_t{a.rows} * M)));
        a.per_chunk = static_cast<int>(ceil_div(steps, want));
        a.chunks = static_cast<int>(ceil_div(steps, a.per_chunk));
        const int64_t ctas = std::max<int64_t>(1, std::min(ceil_div(int64_t{a.rows} * a.chunks, kWarps), static_cast<int64_t>(kSms) * kHeadCtas / M));
        return launch(kernel, dim3(static_cast<unsigned>(ctas), M), kHeadThreads, 0, stream, a);
    };
    if (mode == kPairAny) return run(head_rotary_forward_kernel<T, 32, kPairAny>, 1);
    if (mode == kPairAnyShort) return run(head_rotary_forward_kernel<T, 32, kPairAnyShort>, 1);
    return with_lanes<T>(a.words, [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        return mode == kPairWords ? run(head_rotary_forward_kernel<T, L, kPairWords>, 32 / L) : run(head_rotary_forward_kernel<T, L, kPairNext>, 32 / L);
    });
}

// CTAs a worker's rows are split over in the backward pass (a rule on the sizes alone, so that the order of the additions
// does not change from call to call): two an SM, which is what their registers allow.
static int head_parts(int64_t rows, int M)
{
    return static_cast<int>(std::max<int64_t>(1, std::min(ceil_div(rows, kHeadThreads / 32), static_cast<int64_t>(2 * kSms / M))));
}

template <typename T>
static grawa_status head_backward(const HeadArgs& a, int M, HeadMode mode, cudaStream_t stream)
{
    const auto run = [&](auto kernel) {
        return launch_clusters(kernel, dim3(static_cast<unsigned>(a.parts), M), kHeadThreads, 0, stream, false, 1u, a);
    };
    grawa_status st;
    if (mode == kPairAny) st = run(head_rotary_backward_kernel<T, 32, kPairAny>);
    else if (mode == kPairAnyShort) st = run(head_rotary_backward_kernel<T, 32, kPairAnyShort>);
    else
        st = with_lanes<T>(a.words, [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            return mode == kPairWords ? run(head_rotary_backward_kernel<T, L, kPairWords>) : run(head_rotary_backward_kernel<T, L, kPairNext>);
        });
    if (st != GRAWA_OK || a.parts == 1 || (!a.has_dw[0] && !a.has_dw[1])) return st;
    return launch(head_rotary_finish_kernel<T>, dim3(static_cast<unsigned>(ceil_div(a.dim, 32)), M, 2), 32 * kHeadGroups, 0, stream, a);
}

}  // namespace replica
}  // namespace grawa

using namespace grawa;
using namespace grawa::replica;

extern "C" {

grawa_status grawa_head_rotary_forward(grawa_dtype dtype, grawa_pairing pairing, const void* const* q, const void* const* k, const void* const* q_weight,
                                       const void* const* k_weight, void* const* q_out, void* const* k_out, const int64_t* const* positions,
                                       const double* frequencies, int64_t rows, int64_t q_heads, int64_t k_heads, int64_t head_dim, int64_t rotary,
                                       int64_t q_stride, int64_t k_stride, int64_t q_out_stride, int64_t k_out_stride, int64_t period, int M, float eps,
                                       grawa_stream_t stream)
{
    const HeadShape s{dtype, pairing, rows, q_heads, k_heads, head_dim, rotary, q_stride, k_stride, q_out_stride, k_out_stride, positions, frequencies, period, M, eps};
    if (!head_shape_ok(s) || !q || !q_out || (k_heads && (!k || !k_out))) return GRAWA_ERR_INVALID_ARG;
    if (rows == 0) return GRAWA_OK;
    Buffers b;
    if (!add_head_inputs(b, s, q_weight, k_weight) || !add_in_and_out(b, q, q_stride, q_out, q_out_stride, s, q_heads)) return GRAWA_ERR_INVALID_ARG;
    if (k_heads && !add_in_and_out(b, k, k_stride, k_out, k_out_stride, s, k_heads)) return GRAWA_ERR_INVALID_ARG;
    if (b.clash()) return GRAWA_ERR_INVALID_ARG;
    HeadArgs a = head_args(s, q, k, q_weight, k_weight);
    copy_table(a.y[0], q_out, M);
    if (k_heads) copy_table(a.y[1], k_out, M);
    const HeadMode mode = head_mode(a, dtype, M, false);
    if (dtype == GRAWA_BF16) return head_forward<__nv_bfloat16>(a, M, mode, stream);
    if (dtype == GRAWA_F16) return head_forward<__half>(a, M, mode, stream);
    return head_forward<float>(a, M, mode, stream);
}

size_t grawa_head_rotary_backward_workspace_bytes(int64_t rows, int M)
{
    if (M < 1 || M > GRAWA_MAX_WORKERS || rows < 0 || rows > 0x7fffffff) return 0;
    const int parts = head_parts(rows, M);
    return parts > 1 ? static_cast<size_t>(M) * parts * 2 * kHeadDim * sizeof(float) : 0;
}

grawa_status grawa_head_rotary_backward(grawa_dtype dtype, grawa_pairing pairing, const void* const* dq_out, const void* const* dk_out, const void* const* q,
                                        const void* const* k, const void* const* q_weight, const void* const* k_weight, void* const* dq, void* const* dk,
                                        void* const* dq_weight, void* const* dk_weight, const int64_t* const* positions, const double* frequencies,
                                        int64_t rows, int64_t q_heads, int64_t k_heads, int64_t head_dim, int64_t rotary, int64_t q_stride,
                                        int64_t k_stride, int64_t q_out_stride, int64_t k_out_stride, int64_t period, int M, float eps, int accumulate,
                                        void* workspace, size_t workspace_bytes, grawa_stream_t stream)
{
    const HeadShape s{dtype, pairing, rows, q_heads, k_heads, head_dim, rotary, q_stride, k_stride, q_out_stride, k_out_stride, positions, frequencies, period, M, eps};
    if (!head_shape_ok(s) || !q || !dq_out || (k_heads && (!k || !dk_out)) || (!k_heads && (dk || dk_weight))) return GRAWA_ERR_INVALID_ARG;
    if (!dq && !dk && !dq_weight && !dk_weight) return GRAWA_ERR_INVALID_ARG;
    if (rows == 0 && (accumulate || (!dq_weight && !dk_weight))) return GRAWA_OK;
    const int64_t elem = type_bytes(dtype);
    Buffers b;
    if (!add_head_inputs(b, s, q_weight, k_weight) || !b.add(q, M, rows, q_heads * head_dim, q_stride, elem, false) ||
        !add_in_and_out(b, dq_out, q_out_stride, dq, q_stride, s, q_heads)) return GRAWA_ERR_INVALID_ARG;
    if (k_heads && (!b.add(k, M, rows, k_heads * head_dim, k_stride, elem, false) || !add_in_and_out(b, dk_out, k_out_stride, dk, k_stride, s, k_heads)))
        return GRAWA_ERR_INVALID_ARG;
    if (dq_weight && !b.add(dq_weight, M, 1, head_dim, head_dim, elem, true)) return GRAWA_ERR_INVALID_ARG;
    if (dk_weight && !b.add(dk_weight, M, 1, head_dim, head_dim, elem, true)) return GRAWA_ERR_INVALID_ARG;
    const size_t need = dq_weight || dk_weight ? grawa_head_rotary_backward_workspace_bytes(rows, M) : 0;
    if (need) {
        if (!workspace || !aligned(workspace, 16) || workspace_bytes < need) return GRAWA_ERR_WORKSPACE;
        const void* ws = workspace;
        if (!b.add(&ws, 1, 1, static_cast<int64_t>(need), static_cast<int64_t>(need), 1, true)) return GRAWA_ERR_INVALID_ARG;
    }
    if (b.clash()) return GRAWA_ERR_INVALID_ARG;
    HeadArgs a = head_args(s, q, k, q_weight, k_weight);
    copy_table(a.dy[0], dq_out, M);
    if (k_heads) copy_table(a.dy[1], dk_out, M);
    copy_table(a.y[0], dq, M);
    copy_table(a.y[1], dk, M);
    copy_table(a.dw[0], dq_weight, M);
    copy_table(a.dw[1], dk_weight, M);
    a.has_dx[0] = dq != nullptr; a.has_dx[1] = dk != nullptr;
    a.has_dw[0] = dq_weight != nullptr; a.has_dw[1] = dk_weight != nullptr;
    a.accumulate = accumulate != 0;
    a.parts = head_parts(rows, M);
    a.partial = static_cast<float*>(workspace);
    const HeadMode mode = head_mode(a, dtype, M, true);
    if (dtype == GRAWA_BF16) return head_backward<__nv_bfloat16>(a, M, mode, stream);
    if (dtype == GRAWA_F16) return head_backward<__half>(a, M, mode, stream);
    return head_backward<float>(a, M, mode, stream);
}

}  // extern "C"

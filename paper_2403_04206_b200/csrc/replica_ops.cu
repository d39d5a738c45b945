// Host side of the replica operators: argument checks, the choice of a kernel, launches, and their part of
// the C ABI in include/grawa.h.  No call allocates device memory or keeps anything from one call to the next.
#include <cmath>
#include <cstring>

#include "dropout.cuh"
#include "layernorm.cuh"
#include "replica_host.h"

namespace grawa {
namespace replica {

template <typename P, typename S>
static void copy_table(P& to, S* const* from, int M)
{
    for (int m = 0; m < M; ++m) to.p[m] = const_cast<void*>(static_cast<const void*>(from ? from[m] : nullptr));
}

static bool all_aligned(const void* const* table, int M, size_t bytes)
{
    bool ok = true;
    for (int m = 0; m < M && table; ++m) ok = ok && aligned(table[m], bytes);
    return ok;
}

// ------------------------------------------------------------------ dropout

template <typename T>
static grawa_status launch_dropout(const DropoutArgs& a, int M, bool vec, cudaStream_t stream)
{
    constexpr int kCols = 2;
    const int64_t per_cta = static_cast<int64_t>(kDropThreads) * kCols * (vec ? 16 / static_cast<int>(sizeof(T)) : 4);
    const int64_t ctas = ceil_div(a.n, per_cta);
    if (ctas > 0x7fffffff) return GRAWA_ERR_INVALID_ARG;
    return launch(vec ? dropout_kernel<T, true, kCols> : dropout_kernel<T, false, kCols>, dim3(static_cast<unsigned>(ctas), M), kDropThreads, 0,
                  stream, false, a);
}

// `in` and `r` may each be the same buffer as `out` (every element is read before it is written, by one thread).
static grawa_status dropout(grawa_dtype dtype, const void* const* in, const void* const* r, void* const* out, int64_t n, int M, float p,
                            uint64_t seed, uint64_t offset, const uint64_t* counter, cudaStream_t stream)
{
    if (!dtype_known(dtype) || !in || !out || M < 1 || M > GRAWA_MAX_WORKERS || n < 0 || n > (int64_t{1} << 56)) return GRAWA_ERR_INVALID_ARG;
    if (!(p >= 0.0f && p < 1.0f) || !aligned(counter, 8)) return GRAWA_ERR_INVALID_ARG;
    if (n == 0) return GRAWA_OK;
    const int64_t elem = type_bytes(dtype);
    for (int m = 0; m < M; ++m)
        if (!in[m] || !out[m] || (r && !r[m])) return GRAWA_ERR_INVALID_ARG;
    Buffers b;
    const void* apart[GRAWA_MAX_WORKERS];
    const int64_t counter_words = counter ? 1 : 0;
    if (!b.add(out, M, 1, n, n, elem, true)) return GRAWA_ERR_INVALID_ARG;
    for (const void* const* t : {in, r}) {
        if (!t) continue;
        int others = 0;
        for (int m = 0; m < M; ++m)
            if (t[m] != out[m]) apart[others++] = t[m];
        if (!b.add(apart, others, 1, n, n, elem, false)) return GRAWA_ERR_INVALID_ARG;
    }
    apart[0] = counter;
    if (!b.add(apart, static_cast<int>(counter_words), 1, 1, 1, 8, false) || b.clash()) return GRAWA_ERR_INVALID_ARG;

    DropoutArgs a{};
    copy_table(a.x, in, M);
    copy_table(a.r, r, M);
    copy_table(a.y, out, M);
    a.n = n;
    a.seed = seed;
    a.offset = offset;
    a.counter = reinterpret_cast<const unsigned long long*>(counter);
    a.threshold = static_cast<unsigned>(std::floor(static_cast<double>(p) * 4294967296.0 + 0.5));
    a.scale = static_cast<float>(1.0 / (1.0 - static_cast<double>(p)));
    a.residual = r != nullptr;
    const bool vec = all_aligned(in, M, 16) && all_aligned(r, M, 16) && all_aligned(out, M, 16);
    if (dtype == GRAWA_BF16) return launch_dropout<__nv_bfloat16>(a, M, vec, stream);
    if (dtype == GRAWA_F16) return launch_dropout<__half>(a, M, vec, stream);
    return launch_dropout<float>(a, M, vec, stream);
}

// ------------------------------------------------------------------ layer norm

// Elements per word: 16 bytes, else 4, else one element, whatever the rows' bases, strides and length allow.
static int word_elems(int64_t elem, int64_t cols, int64_t stride_a, int64_t stride_b, const void* const* a, const void* const* b, const void* const* c, int M)
{
    for (int64_t bytes : {int64_t{16}, int64_t{4}}) {
        if (bytes <= elem) break;
        const int64_t ve = bytes / elem;
        if (cols % ve || stride_a % ve || stride_b % ve) continue;
        if (all_aligned(a, M, bytes) && all_aligned(b, M, bytes) && all_aligned(c, M, bytes)) return static_cast<int>(ve);
    }
    return 1;
}

static bool shape_ok(int64_t rows, int64_t cols, int64_t x_stride, int64_t y_stride, int M, int64_t elem)
{
    if (M < 1 || M > GRAWA_MAX_WORKERS || rows < 0 || rows > 0x7fffffff || cols < 1 || cols > (int64_t{1} << 30)) return false;
    const int64_t most = (int64_t{1} << 60) / elem;
    return x_stride >= cols && y_stride >= cols && x_stride <= most / std::max<int64_t>(1, rows) && y_stride <= most / std::max<int64_t>(1, rows);
}

constexpr int kLongForward = kNormMaxBlock * 32, kLongBackward = kNormMaxBlock * 16;   // longest rows held in registers

template <typename T, int VE>
static grawa_status launch_norm_forward(const NormForwardArgs& a, int M, cudaStream_t stream)
{
    const auto lanes = [&](auto kernel, int lpr) {
        return launch(kernel, dim3(static_cast<unsigned>(ceil_div(a.rows, kNormThreads / lpr)), M), kNormThreads, 0, stream, false, a);
    };
    const auto block = [&](auto kernel, int ept) {
        return launch(kernel, dim3(static_cast<unsigned>(a.rows), M), static_cast<int>(ceil_div(a.cols, 32 * ept)) * 32, 0, stream, false, a);
    };
    if (a.cols <= 64) return lanes(layernorm_forward_kernel<T, VE, 8, 8>, 8);
    if (a.cols <= 256) return lanes(layernorm_forward_kernel<T, VE, 8, 32>, 32);
    if (a.cols <= 512) return lanes(layernorm_forward_kernel<T, VE, 16, 32>, 32);
    if (a.cols <= 768) return lanes(layernorm_forward_kernel<T, VE, 24, 32>, 32);
    if (a.cols <= 1024) return lanes(layernorm_forward_kernel<T, VE, 32, 32>, 32);
    if (a.cols <= kLongForward / 2) return block(layernorm_forward_kernel<T, VE, 16, 0>, 16);
    if (a.cols <= kLongForward) return block(layernorm_forward_kernel<T, VE, 32, 0>, 32);
    return launch(layernorm_forward_long_kernel<T, VE>, dim3(static_cast<unsigned>(a.rows), M), kNormLongThreads, 0, stream, false, a);
}

// Rows that a CTA of the register kernels handles at a time.
static int norm_groups(int64_t cols) { return cols <= 64 ? kNormThreads / 8 : cols <= 1024 ? kNormThreads / 32 : 1; }

// CTAs a worker's rows are split over in the backward pass (a rule on the sizes alone, so that the order of
// the additions does not change from call to call).  Few rows go to one CTA, which then writes the
// gradients itself: the second launch costs more than a few rows one after the other.
static int norm_parts(int64_t rows, int64_t cols, int M)
{
    if (cols > kLongBackward) {
        const int64_t want = std::max<int64_t>(1, 8 * kSms / std::max<int64_t>(1, M * ceil_div(cols, kNormThreads)));
        return static_cast<int>(std::max<int64_t>(1, std::min(want, ceil_div(rows, 32))));
    }
    const int64_t steps = ceil_div(rows, norm_groups(cols));
    if (steps <= 4) return 1;
    const int64_t threads = cols <= 1024 ? kNormThreads : ceil_div(cols, 32 * 16) * 32;
    const int64_t resident = kSms * std::max<int64_t>(1, 512 / threads);
    return static_cast<int>(std::max<int64_t>(1, std::min(steps, resident / M)));
}

template <typename T, int VE>
static grawa_status launch_norm_backward(const NormBackwardArgs& a, int M, cudaStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(a.parts), M);
    const int block = static_cast<int>(ceil_div(a.cols, 32 * 16)) * 32;
    if (a.cols <= 64) return launch(layernorm_backward_kernel<T, VE, 8, 8>, grid, kNormThreads, 0, stream, false, a);
    if (a.cols <= 256) return launch(layernorm_backward_kernel<T, VE, 8, 32>, grid, kNormThreads, 0, stream, false, a);
    if (a.cols <= 512) return launch(layernorm_backward_kernel<T, VE, 16, 32>, grid, kNormThreads, 0, stream, false, a);
    if (a.cols <= 768) return launch(layernorm_backward_kernel<T, VE, 24, 32>, grid, kNormThreads, 0, stream, false, a);
    if (a.cols <= 1024) return launch(layernorm_backward_kernel<T, VE, 32, 32>, grid, kNormThreads, 0, stream, false, a);
    if (a.cols <= kLongBackward) return launch(layernorm_backward_kernel<T, VE, 16, 0>, grid, block, 0, stream, false, a);
    if (a.has_dx) {
        const grawa_status st = launch(layernorm_backward_long_kernel<T, VE>, dim3(static_cast<unsigned>(a.rows), M), kNormLongThreads, 0, stream, false, a);
        if (st != GRAWA_OK) return st;
    }
    if (!a.has_dgamma && !a.has_dbeta) return GRAWA_OK;
    return launch(layernorm_columns_kernel<T>, dim3(static_cast<unsigned>(ceil_div(a.cols, kNormThreads)), M, a.parts), kNormThreads, 0, stream, false, a);
}

template <typename T>
static grawa_status norm_backward(const NormBackwardArgs& a, int M, int ve, cudaStream_t stream)
{
    if (a.rows > 0) {
        grawa_status st;
        if (ve == 16 / static_cast<int>(sizeof(T))) st = launch_norm_backward<T, 16 / static_cast<int>(sizeof(T))>(a, M, stream);
        else if (sizeof(T) == 2 && ve == 2) st = launch_norm_backward<T, sizeof(T) == 2 ? 2 : 1>(a, M, stream);
        else st = launch_norm_backward<T, 1>(a, M, stream);
        if (st != GRAWA_OK || a.parts == 1) return st;
    }
    if (!a.has_dgamma && !a.has_dbeta) return GRAWA_OK;
    return launch(layernorm_finish_kernel<T>, dim3(static_cast<unsigned>(ceil_div(a.cols, 32)), M), 32 * kFinishGroups, 0, stream, true, a);
}

template <typename T>
static grawa_status norm_forward(const NormForwardArgs& a, int M, int ve, cudaStream_t stream)
{
    if (ve == 16 / static_cast<int>(sizeof(T))) return launch_norm_forward<T, 16 / static_cast<int>(sizeof(T))>(a, M, stream);
    if (sizeof(T) == 2 && ve == 2) return launch_norm_forward<T, sizeof(T) == 2 ? 2 : 1>(a, M, stream);
    return launch_norm_forward<T, 1>(a, M, stream);
}

}  // namespace replica
}  // namespace grawa

using namespace grawa;
using namespace grawa::replica;

extern "C" {

grawa_status grawa_dropout_forward(grawa_dtype dtype, const void* const* x, const void* const* residual, void* const* y, int64_t n, int M,
                                   float p, uint64_t seed, uint64_t offset, const uint64_t* offset_counter, grawa_stream_t stream)
{
    return dropout(dtype, x, residual, y, n, M, p, seed, offset, offset_counter, stream);
}

grawa_status grawa_dropout_backward(grawa_dtype dtype, const void* const* dy, void* const* dx, int64_t n, int M, float p, uint64_t seed,
                                    uint64_t offset, const uint64_t* offset_counter, grawa_stream_t stream)
{
    return dropout(dtype, dy, nullptr, dx, n, M, p, seed, offset, offset_counter, stream);
}

grawa_status grawa_layernorm_forward(grawa_dtype dtype, const void* const* x, const void* const* gamma, const void* const* beta, void* const* y,
                                     float* const* mean, float* const* rstd, int64_t rows, int64_t cols, int64_t x_stride, int64_t y_stride,
                                     int M, float eps, grawa_stream_t stream)
{
    if (!dtype_known(dtype) || !x || !y || (mean == nullptr) != (rstd == nullptr)) return GRAWA_ERR_INVALID_ARG;
    const int64_t elem = type_bytes(dtype);
    if (!shape_ok(rows, cols, x_stride, y_stride, M, elem) || !(eps >= 0.0f) || std::isinf(eps)) return GRAWA_ERR_INVALID_ARG;
    if (rows == 0) return GRAWA_OK;
    Buffers b;
    if (!b.add(x, M, rows, cols, x_stride, elem, false) || !b.add(y, M, rows, cols, y_stride, elem, true)) return GRAWA_ERR_INVALID_ARG;
    if (gamma && !b.add(gamma, M, 1, cols, cols, elem, false)) return GRAWA_ERR_INVALID_ARG;
    if (beta && !b.add(beta, M, 1, cols, cols, elem, false)) return GRAWA_ERR_INVALID_ARG;
    if (mean && (!b.add(reinterpret_cast<const void* const*>(mean), M, 1, rows, rows, 4, true) ||
                 !b.add(reinterpret_cast<const void* const*>(rstd), M, 1, rows, rows, 4, true))) return GRAWA_ERR_INVALID_ARG;
    if (b.clash()) return GRAWA_ERR_INVALID_ARG;
    NormForwardArgs a{};
    copy_table(a.x, x, M);
    copy_table(a.gamma, gamma, M);
    copy_table(a.beta, beta, M);
    copy_table(a.y, y, M);
    copy_table(a.mean, mean, M);
    copy_table(a.rstd, rstd, M);
    a.rows = rows; a.cols = static_cast<int>(cols);
    a.x_stride = x_stride; a.y_stride = y_stride;
    a.eps = eps;
    a.has_gamma = gamma != nullptr; a.has_beta = beta != nullptr; a.has_stats = mean != nullptr;
    const int ve = word_elems(elem, cols, x_stride, y_stride, x, y, nullptr, M);
    if (dtype == GRAWA_BF16) return norm_forward<__nv_bfloat16>(a, M, ve, stream);
    if (dtype == GRAWA_F16) return norm_forward<__half>(a, M, ve, stream);
    return norm_forward<float>(a, M, ve, stream);
}

size_t grawa_layernorm_backward_workspace_bytes(int64_t rows, int64_t cols, int M)
{
    if (!shape_ok(rows, cols, cols, cols, M, 4)) return 0;
    const int parts = norm_parts(rows, cols, M);
    return parts == 1 ? 0 : static_cast<size_t>(M) * parts * 2 * cols * sizeof(float);
}

grawa_status grawa_layernorm_backward(grawa_dtype dtype, const void* const* dy, const void* const* x, const void* const* gamma,
                                      const float* const* mean, const float* const* rstd, void* const* dx, void* const* dgamma,
                                      void* const* dbeta, int64_t rows, int64_t cols, int64_t x_stride, int64_t y_stride, int M, int accumulate,
                                      void* workspace, size_t workspace_bytes, grawa_stream_t stream)
{
    if (!dtype_known(dtype) || !dy || !x || !mean || !rstd || (!dx && !dgamma && !dbeta)) return GRAWA_ERR_INVALID_ARG;
    const int64_t elem = type_bytes(dtype);
    if (!shape_ok(rows, cols, x_stride, y_stride, M, elem)) return GRAWA_ERR_INVALID_ARG;
    if (rows == 0 && (accumulate || (!dgamma && !dbeta))) return GRAWA_OK;
    Buffers b;
    if (!b.add(dy, M, rows, cols, y_stride, elem, false) || !b.add(x, M, rows, cols, x_stride, elem, false)) return GRAWA_ERR_INVALID_ARG;
    if (!b.add(reinterpret_cast<const void* const*>(mean), M, 1, rows, rows, 4, false) ||
        !b.add(reinterpret_cast<const void* const*>(rstd), M, 1, rows, rows, 4, false)) return GRAWA_ERR_INVALID_ARG;
    if (gamma && !b.add(gamma, M, 1, cols, cols, elem, false)) return GRAWA_ERR_INVALID_ARG;
    if (dx && !b.add(dx, M, rows, cols, x_stride, elem, true)) return GRAWA_ERR_INVALID_ARG;
    if (dgamma && !b.add(dgamma, M, 1, cols, cols, elem, true)) return GRAWA_ERR_INVALID_ARG;
    if (dbeta && !b.add(dbeta, M, 1, cols, cols, elem, true)) return GRAWA_ERR_INVALID_ARG;
    const bool weights = dgamma || dbeta;
    const size_t need = weights ? grawa_layernorm_backward_workspace_bytes(rows, cols, M) : 0;
    if (need) {
        if (!workspace || !aligned(workspace, 16) || workspace_bytes < need) return GRAWA_ERR_WORKSPACE;
        const void* ws = workspace;
        if (!b.add(&ws, 1, 1, static_cast<int64_t>(need), static_cast<int64_t>(need), 1, true)) return GRAWA_ERR_INVALID_ARG;
    }
    if (b.clash()) return GRAWA_ERR_INVALID_ARG;
    NormBackwardArgs a{};
    copy_table(a.dy, dy, M);
    copy_table(a.x, x, M);
    copy_table(a.gamma, gamma, M);
    copy_table(a.mean, mean, M);
    copy_table(a.rstd, rstd, M);
    copy_table(a.dx, dx, M);
    copy_table(a.dgamma, dgamma, M);
    copy_table(a.dbeta, dbeta, M);
    a.partial = static_cast<float*>(workspace);
    a.rows = rows; a.cols = static_cast<int>(cols);
    a.x_stride = x_stride; a.y_stride = y_stride;
    a.parts = rows == 0 ? 0 : norm_parts(rows, cols, M);
    a.has_gamma = gamma != nullptr; a.has_dx = dx != nullptr; a.has_dgamma = dgamma != nullptr; a.has_dbeta = dbeta != nullptr;
    a.accumulate = accumulate != 0;
    const int ve = word_elems(elem, cols, x_stride, y_stride, x, dy, dx, M);
    if (dtype == GRAWA_BF16) return norm_backward<__nv_bfloat16>(a, M, ve, stream);
    if (dtype == GRAWA_F16) return norm_backward<__half>(a, M, ve, stream);
    return norm_backward<float>(a, M, ve, stream);
}

}  // extern "C"

// Host side of the replica operators: argument checks, the choice of a kernel, launches, and their part of
// the C ABI in include/grawa.h.  No call allocates device memory or keeps anything from one call to the next.
#include <cudaTypedefs.h>

#include <cmath>
#include <cstring>
#include <utility>

#include "dropout.cuh"
#include "gated_ffn.cuh"
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

template <typename T, int COLS>
static grawa_status launch_dropout(const DropoutArgs& a, int M, bool vec, bool residual, cudaStream_t stream)
{
    const int64_t ctas = ceil_div(a.n, kDropThreads * COLS * (16 / static_cast<int>(sizeof(T))));
    if (ctas > 0x7fffffff) return GRAWA_ERR_INVALID_ARG;
    auto* const kernel = vec ? (residual ? dropout_kernel<T, COLS, true, true> : dropout_kernel<T, COLS, true, false>)
                             : (residual ? dropout_kernel<T, COLS, false, true> : dropout_kernel<T, COLS, false, false>);
    return launch(kernel, dim3(static_cast<unsigned>(ctas), M), kDropThreads, 0, stream, false, a);
}

template <typename T>
static grawa_status launch_dropout(const DropoutArgs& a, int M, bool vec, bool residual, cudaStream_t stream)
{
    const int64_t columns = ceil_div(a.n, kDropThreads * (16 / static_cast<int>(sizeof(T)))) * M;
    return columns >= 4 * 16 * kSms ? launch_dropout<T, 4>(a, M, vec, residual, stream) : launch_dropout<T, 1>(a, M, vec, residual, stream);
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
    for (unsigned round = 0; round < 10; ++round)
        a.keys[round] = make_uint2(static_cast<unsigned>(seed) + round * 0x9E3779B9u, static_cast<unsigned>(seed >> 32) + round * 0xBB67AE85u);
    a.offset = offset;
    a.counter = reinterpret_cast<const unsigned long long*>(counter);
    a.threshold = static_cast<unsigned>(std::floor(static_cast<double>(p) * 4294967296.0 + 0.5));
    a.scale = static_cast<float>(1.0 / (1.0 - static_cast<double>(p)));
    const bool vec = all_aligned(in, M, 16) && all_aligned(r, M, 16) && all_aligned(out, M, 16);
    if (dtype == GRAWA_BF16) return launch_dropout<__nv_bfloat16>(a, M, vec, r != nullptr, stream);
    if (dtype == GRAWA_F16) return launch_dropout<__half>(a, M, vec, r != nullptr, stream);
    return launch_dropout<float>(a, M, vec, r != nullptr, stream);
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
    if (a.cols <= 64) return lanes(layernorm_forward_kernel<T, VE, 8 / VE, 8>, 8);
    // A warp a row, as long as a lane's words fit in its registers.
    const int64_t per_lane = ceil_div(a.cols / VE, 32);
    if constexpr (VE >= 4) {
        if (per_lane <= 1) return lanes(layernorm_forward_kernel<T, VE, 1, 32>, 32);
        if (per_lane <= 2) return lanes(layernorm_forward_kernel<T, VE, 2, 32>, 32);
        if (per_lane <= 3) return lanes(layernorm_forward_kernel<T, VE, 3, 32>, 32);
        if (per_lane <= 4) return lanes(layernorm_forward_kernel<T, VE, 4, 32>, 32);
        if (per_lane <= 6) return lanes(layernorm_forward_kernel<T, VE, 6, 32>, 32);
        if (per_lane <= 8) return lanes(layernorm_forward_kernel<T, VE, 8, 32>, 32);
        if (per_lane <= 12) return lanes(layernorm_forward_kernel<T, VE, 12, 32>, 32);
        if (per_lane <= 16) return lanes(layernorm_forward_kernel<T, VE, 16, 32>, 32);
    } else {
        if (per_lane <= 8) return lanes(layernorm_forward_kernel<T, VE, 8, 32>, 32);
        if (per_lane <= 16) return lanes(layernorm_forward_kernel<T, VE, 16, 32>, 32);
        if (per_lane <= 32) return lanes(layernorm_forward_kernel<T, VE, 32, 32>, 32);
    }
    if (a.cols <= kLongForward)
        return launch(layernorm_forward_kernel<T, VE, 32 / VE, 0>, dim3(static_cast<unsigned>(a.rows), M), static_cast<int>(ceil_div(a.cols, 32 * 32)) * 32, 0, stream, false, a);
    return launch(layernorm_forward_long_kernel<T, VE>, dim3(static_cast<unsigned>(a.rows), M), kNormLongThreads, 0, stream, false, a);
}

// Rows that a CTA of the register kernels handles at a time.
static int norm_groups(int64_t cols) { return cols <= 64 ? kNormThreads / 8 : cols <= 1024 ? kNormThreads / 32 : 1; }

// CTAs a worker's rows are split over in the backward pass (a rule on the sizes alone, so that the order of
// the additions does not change from call to call).  Few rows go to one CTA, which then writes the
// gradients itself: the second launch costs more than a few rows one after the other.
static int norm_parts(int64_t rows, int64_t cols, int M, int64_t elem)
{
    if (cols > kLongBackward) {
        const int64_t want = std::max<int64_t>(1, 8 * kSms / std::max<int64_t>(1, M * ceil_div(cols, kNormThreads)));
        return static_cast<int>(std::max<int64_t>(1, std::min(want, ceil_div(rows, 32))));
    }
    const int64_t steps = ceil_div(rows, norm_groups(cols));
    if (steps <= 4) return 1;
    // as many CTAs as their registers and stages let an SM hold at once
    const bool narrow = elem == 2;
    const int64_t per_sm = cols <= 256 ? 6 : cols <= 512 ? (narrow ? 5 : 4) : cols <= 768 ? (narrow ? 4 : 3) : cols <= 1024 ? (narrow ? 3 : 2)
                           : 512 / (ceil_div(cols, 32 * 16) * 32);
    return static_cast<int>(std::max<int64_t>(1, std::min(steps, kSms * per_sm / M)));
}

template <typename T, int VE, int EPT, int LPR>
static grawa_status launch_norm_rows(const NormBackwardArgs& a, int M, int block, cudaStream_t stream)
{
    const size_t smem = NormStage<T, VE, EPT>::bytes_a_thread * block;
    if (smem > 0) GRAWA_CUDA_TRY(cudaFuncSetAttribute(layernorm_backward_kernel<T, VE, EPT, LPR>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    return launch(layernorm_backward_kernel<T, VE, EPT, LPR>, dim3(static_cast<unsigned>(a.parts), M), block, smem, stream, false, a);
}

template <typename T, int VE>
static grawa_status launch_norm_backward(const NormBackwardArgs& a, int M, cudaStream_t stream)
{
    if (a.cols <= 64) return launch_norm_rows<T, VE, 8, 8>(a, M, kNormThreads, stream);
    if (a.cols <= 256) return launch_norm_rows<T, VE, 8, 32>(a, M, kNormThreads, stream);
    if (a.cols <= 512) return launch_norm_rows<T, VE, 16, 32>(a, M, kNormThreads, stream);
    if (a.cols <= 768) return launch_norm_rows<T, VE, 24, 32>(a, M, kNormThreads, stream);
    if (a.cols <= 1024) return launch_norm_rows<T, VE, 32, 32>(a, M, kNormThreads, stream);
    if (a.cols <= kLongBackward) return launch_norm_rows<T, VE, 16, 0>(a, M, static_cast<int>(ceil_div(a.cols, 32 * 16)) * 32, stream);
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

// ------------------------------------------------------------------ gated feed-forward product

// The driver's encoder of tensor maps, looked up once through the runtime (the library does not link the driver).
static grawa_status map_encoder(PFN_cuTensorMapEncodeTiled_v12000* out)
{
    static const auto found = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q = cudaDriverEntryPointSymbolNotFound;
        cudaError_t err = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
        if (err == cudaSuccess && (q != cudaDriverEntryPointSuccess || fn == nullptr)) err = cudaErrorNotSupported;
        return std::make_pair(err, reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn));
    }();
    GRAWA_CUDA_TRY(found.first);
    *out = found.second;
    return GRAWA_OK;
}

// Map of a matrix [depth][rows][cols] of 16-bit elements with rows `pitch` elements apart, for boxes of 64
// columns (128 bytes, the swizzle's width) by box_rows rows.  The base is 16-byte aligned, the pitch a
// multiple of 8 elements, and every box starts at a multiple of 64 columns.
static grawa_status encode_map(CUtensorMap* map, grawa_dtype dtype, const void* base, int64_t depth, int64_t rows, int64_t cols, int64_t pitch,
                               int box_rows)
{
    PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
    const grawa_status st = map_encoder(&encode);
    if (st != GRAWA_OK) return st;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(depth)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(pitch) * 2, static_cast<cuuint64_t>(pitch) * 2 * rows};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_rows), 1}, step[3] = {1, 1, 1};
    const CUresult res = encode(map, dtype == GRAWA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, depth ? 3 : 2,
                                const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return res == CUDA_SUCCESS ? GRAWA_OK : cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
}

// One operand of all workers as TMA can read it: in place, or laid out again in the workspace.
struct Operand {
    const void* base[GRAWA_MAX_WORKERS];
    int64_t rows, cols, pitch;
};

// A bump allocator over the caller's workspace; with a NULL base it only counts.
struct Scratch {
    char* base;
    size_t used = 0;
    void* take(size_t bytes)
    {
        void* p = base ? base + used : nullptr;
        used += (bytes + 255) / 256 * 256;
        return p;
    }
};

static int64_t pitch_of(int64_t cols) { return ceil_div(cols, 8) * 8; }
static bool in_place(int64_t cols, bool is_aligned) { return cols % 8 == 0 && is_aligned; }

// Scratch of one operand: nothing when it is read in place.
static void* operand_scratch(Scratch& s, int64_t rows, int64_t cols, int M, bool is_aligned)
{
    return in_place(cols, is_aligned) ? nullptr : s.take(static_cast<size_t>(M) * rows * pitch_of(cols) * 2);
}

static grawa_status make_operand(Operand* op, const void* const* table, int64_t rows, int64_t cols, int M, void* scratch, cudaStream_t stream)
{
    op->rows = rows; op->cols = cols; op->pitch = pitch_of(cols);
    if (in_place(cols, all_aligned(table, M, 16))) {
        for (int m = 0; m < M; ++m) op->base[m] = table[m];
        return GRAWA_OK;
    }
    PackArgs a{};
    copy_table(a.from, table, M);
    a.to = static_cast<unsigned short*>(scratch);
    a.rows = rows; a.cols = static_cast<int>(cols); a.pitch = static_cast<int>(op->pitch);
    for (int m = 0; m < M; ++m) op->base[m] = a.to + static_cast<size_t>(m) * rows * op->pitch;
    return launch(pack_rows_kernel, dim3(static_cast<unsigned>(ceil_div(rows * (op->pitch / 8), kGatedThreads)), M), kGatedThreads, 0, stream, false, a);
}

template <typename T, int MODE>
static grawa_status launch_gemm(const GemmArgs& a, cudaStream_t stream)
{
    const int64_t tiles = static_cast<int64_t>(a.workers) * (MODE == kWeightGrad ? 2 : 1) * a.m_tiles * a.n_tiles;
    if (tiles > 0x7fffffff - kSms) return GRAWA_ERR_TOO_LARGE;
    GRAWA_CUDA_TRY(cudaFuncSetAttribute(gemm_kernel<T, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem));
    return launch(gemm_kernel<T, MODE>, dim3(2 * static_cast<unsigned>(std::min<int64_t>(tiles, kSms / 2))), kGemmThreads, kGemmSmem, stream, false, a);
}

template <int MODE>
static grawa_status launch_gemm(grawa_dtype dtype, const GemmArgs& a, cudaStream_t stream)
{
    return dtype == GRAWA_BF16 ? launch_gemm<__nv_bfloat16, MODE>(a, stream) : launch_gemm<__half, MODE>(a, stream);
}

// Outputs of [rows][cols] for the workers [first, first + count); whether they take 16-byte stores.
static void set_outputs(GemmArgs& a, int slot, void* const* table, int first, int count)
{
    for (int w = 0; w < count; ++w) {
        a.out[slot][w] = table ? table[first + w] : nullptr;
        a.words = a.words && aligned(a.out[slot][w], 16);
    }
}

static bool ffn_shape_ok(int64_t rows, int64_t d_in, int64_t d_hidden, int M)
{
    constexpr int64_t kMost = int64_t{1} << 24;
    return M >= 1 && M <= GRAWA_MAX_WORKERS && rows >= 0 && rows <= kMost && d_in >= 1 && d_in <= kMost && d_hidden >= 1 && d_hidden <= kMost &&
           d_in * d_hidden <= (int64_t{1} << 40) && rows * std::max(d_in, d_hidden) <= (int64_t{1} << 38);
}

static bool ffn_kinds_ok(grawa_dtype dtype, grawa_activation act)
{
    return (dtype == GRAWA_BF16 || dtype == GRAWA_F16) && (act == GRAWA_SILU || act == GRAWA_GELU || act == GRAWA_RELU);
}

// The places of a call's scratch, in the order in which they are taken.
struct FfnScratch {
    void *x, *w_gate, *w_up, *da, *du;
    size_t bytes;
};
static FfnScratch ffn_scratch(void* base, int64_t rows, int64_t d_in, int64_t d_hidden, int M, bool x_ok, bool w_ok, bool backward)
{
    Scratch s{static_cast<char*>(base)};
    FfnScratch f{};
    f.x = operand_scratch(s, rows, d_in, M, x_ok);
    f.w_gate = operand_scratch(s, d_hidden, d_in, M, w_ok);
    f.w_up = operand_scratch(s, d_hidden, d_in, M, w_ok);
    if (backward) {
        f.da = s.take(static_cast<size_t>(M) * rows * pitch_of(d_hidden) * 2);
        f.du = s.take(static_cast<size_t>(M) * rows * pitch_of(d_hidden) * 2);
    }
    f.bytes = s.used;
    return f;
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
    a.eps = eps; a.inv_cols = 1.0f / static_cast<float>(cols);
    a.has_gamma = gamma != nullptr; a.has_beta = beta != nullptr; a.has_stats = mean != nullptr;
    const int ve = word_elems(elem, cols, x_stride, y_stride, x, y, nullptr, M);
    if (dtype == GRAWA_BF16) return norm_forward<__nv_bfloat16>(a, M, ve, stream);
    if (dtype == GRAWA_F16) return norm_forward<__half>(a, M, ve, stream);
    return norm_forward<float>(a, M, ve, stream);
}

size_t grawa_layernorm_backward_workspace_bytes(int64_t rows, int64_t cols, int M)
{
    if (!shape_ok(rows, cols, cols, cols, M, 4)) return 0;
    const int parts = norm_parts(rows, cols, M, 2);            // 16-bit storage takes the most
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
    a.rows = rows; a.cols = static_cast<int>(cols); a.inv_cols = 1.0f / static_cast<float>(cols);
    a.x_stride = x_stride; a.y_stride = y_stride;
    a.parts = rows == 0 ? 0 : norm_parts(rows, cols, M, elem);
    a.has_gamma = gamma != nullptr; a.has_dx = dx != nullptr; a.has_dgamma = dgamma != nullptr; a.has_dbeta = dbeta != nullptr;
    a.accumulate = accumulate != 0;
    const int ve = word_elems(elem, cols, x_stride, y_stride, x, dy, dx, M);
    if (dtype == GRAWA_BF16) return norm_backward<__nv_bfloat16>(a, M, ve, stream);
    if (dtype == GRAWA_F16) return norm_backward<__half>(a, M, ve, stream);
    return norm_backward<float>(a, M, ve, stream);
}

size_t grawa_gated_ffn_workspace_bytes(int64_t rows, int64_t d_in, int64_t d_hidden, int M, int backward, int aligned)
{
    if (!ffn_shape_ok(rows, d_in, d_hidden, M) || rows == 0) return 0;
    return ffn_scratch(nullptr, rows, d_in, d_hidden, M, aligned != 0, aligned != 0, backward != 0).bytes;
}

grawa_status grawa_gated_ffn_forward(grawa_dtype dtype, grawa_activation act, const void* const* x, const void* const* w_gate,
                                     const void* const* w_up, void* const* h, void* const* gate_out, void* const* up_out, int64_t rows,
                                     int64_t d_in, int64_t d_hidden, int M, void* workspace, size_t workspace_bytes, grawa_stream_t stream)
{
    if (!ffn_kinds_ok(dtype, act) || !x || !w_gate || !w_up || !h || (gate_out == nullptr) != (up_out == nullptr)) return GRAWA_ERR_INVALID_ARG;
    if (!ffn_shape_ok(rows, d_in, d_hidden, M)) return GRAWA_ERR_INVALID_ARG;
    if (rows == 0) return GRAWA_OK;
    Buffers b;
    if (!b.add(x, M, 1, rows * d_in, rows * d_in, 2, false) || !b.add(w_gate, M, 1, d_in * d_hidden, d_in * d_hidden, 2, false) ||
        !b.add(w_up, M, 1, d_in * d_hidden, d_in * d_hidden, 2, false) || !b.add(h, M, 1, rows * d_hidden, rows * d_hidden, 2, true))
        return GRAWA_ERR_INVALID_ARG;
    if (gate_out && (!b.add(gate_out, M, 1, rows * d_hidden, rows * d_hidden, 2, true) ||
                     !b.add(up_out, M, 1, rows * d_hidden, rows * d_hidden, 2, true))) return GRAWA_ERR_INVALID_ARG;
    const FfnScratch f = ffn_scratch(workspace, rows, d_in, d_hidden, M, all_aligned(x, M, 16), all_aligned(w_gate, M, 16) && all_aligned(w_up, M, 16), false);
    if (f.bytes) {
        if (!workspace || !aligned(workspace, 256) || workspace_bytes < f.bytes) return GRAWA_ERR_WORKSPACE;
        const void* ws = workspace;
        if (!b.add(&ws, 1, 1, static_cast<int64_t>(f.bytes), static_cast<int64_t>(f.bytes), 1, true)) return GRAWA_ERR_INVALID_ARG;
    }
    if (b.clash()) return GRAWA_ERR_INVALID_ARG;

    Operand xo, go, uo;
    grawa_status st = make_operand(&xo, x, rows, d_in, M, f.x, stream);
    if (st == GRAWA_OK) st = make_operand(&go, w_gate, d_hidden, d_in, M, f.w_gate, stream);
    if (st == GRAWA_OK) st = make_operand(&uo, w_up, d_hidden, d_in, M, f.w_up, stream);
    for (int first = 0; first < M && st == GRAWA_OK; first += kGemmWorkers) {
        GemmArgs a{};
        a.workers = std::min(kGemmWorkers, M - first);
        a.first_worker = first;
        a.m_tiles = static_cast<int>(ceil_div(rows, kTileM)); a.n_tiles = static_cast<int>(ceil_div(d_hidden, kHalf));
        a.k_blocks = static_cast<int>(ceil_div(d_in, kTileK));
        a.rows = static_cast<int>(rows); a.cols = static_cast<int>(d_hidden);
        a.activation = act;
        a.words = d_hidden % 8 == 0;
        set_outputs(a, 0, h, first, a.workers);
        set_outputs(a, 1, gate_out, first, a.workers);
        set_outputs(a, 2, up_out, first, a.workers);
        for (int w = 0; w < a.workers && st == GRAWA_OK; ++w) {
            st = encode_map(&a.per[0][w], dtype, xo.base[first + w], 0, rows, d_in, xo.pitch, kHalf);
            if (st == GRAWA_OK) st = encode_map(&a.per[1][w], dtype, go.base[first + w], 0, d_hidden, d_in, go.pitch, kHalf);
            if (st == GRAWA_OK) st = encode_map(&a.per[2][w], dtype, uo.base[first + w], 0, d_hidden, d_in, uo.pitch, kHalf);
        }
        if (st == GRAWA_OK) st = launch_gemm<kForward>(dtype, a, stream);
    }
    return st;
}

grawa_status grawa_gated_ffn_backward(grawa_dtype dtype, grawa_activation act, const void* const* dh, const void* const* x,
                                      const void* const* w_gate, const void* const* w_up, const void* const* gate, const void* const* up,
                                      void* const* dx, void* const* dw_gate, void* const* dw_up, int64_t rows, int64_t d_in, int64_t d_hidden,
                                      int M, int accumulate, void* workspace, size_t workspace_bytes, grawa_stream_t stream)
{
    if (!ffn_kinds_ok(dtype, act) || !dh || !x || !w_gate || !w_up || !gate || !up) return GRAWA_ERR_INVALID_ARG;
    if ((dw_gate == nullptr) != (dw_up == nullptr) || (!dx && !dw_gate) || !ffn_shape_ok(rows, d_in, d_hidden, M)) return GRAWA_ERR_INVALID_ARG;
    const int64_t weights = d_in * d_hidden;
    Buffers b;
    for (const void* const* t : {dh, gate, up})
        if (!b.add(t, M, rows, d_hidden, d_hidden, 2, false)) return GRAWA_ERR_INVALID_ARG;
    if (!b.add(x, M, rows, d_in, d_in, 2, false)) return GRAWA_ERR_INVALID_ARG;
    if (!b.add(w_gate, M, 1, weights, weights, 2, false) || !b.add(w_up, M, 1, weights, weights, 2, false)) return GRAWA_ERR_INVALID_ARG;
    if (dx && !b.add(dx, M, rows, d_in, d_in, 2, true)) return GRAWA_ERR_INVALID_ARG;
    if (dw_gate && (!b.add(dw_gate, M, 1, weights, weights, 2, true) || !b.add(dw_up, M, 1, weights, weights, 2, true))) return GRAWA_ERR_INVALID_ARG;
    const FfnScratch f = ffn_scratch(workspace, rows, d_in, d_hidden, M, all_aligned(x, M, 16), all_aligned(w_gate, M, 16) && all_aligned(w_up, M, 16), true);
    if (rows > 0) {
        if (!workspace || !aligned(workspace, 256) || workspace_bytes < f.bytes) return GRAWA_ERR_WORKSPACE;
        const void* ws = workspace;
        if (!b.add(&ws, 1, 1, static_cast<int64_t>(f.bytes), static_cast<int64_t>(f.bytes), 1, true)) return GRAWA_ERR_INVALID_ARG;
    }
    if (b.clash()) return GRAWA_ERR_INVALID_ARG;
    if (rows == 0) {                                          // sums over no rows
        for (int m = 0; m < M && dw_gate && !accumulate; ++m) {
            GRAWA_CUDA_TRY(cudaMemsetAsync(dw_gate[m], 0, static_cast<size_t>(weights) * 2, stream));
            GRAWA_CUDA_TRY(cudaMemsetAsync(dw_up[m], 0, static_cast<size_t>(weights) * 2, stream));
        }
        return GRAWA_OK;
    }

    const int64_t pitch = pitch_of(d_hidden);
    GatedGradArgs e{};
    copy_table(e.dh, dh, M);
    copy_table(e.gate, gate, M);
    copy_table(e.up, up, M);
    e.da = f.da; e.du = f.du;
    e.rows = rows; e.cols = static_cast<int>(d_hidden); e.pitch = static_cast<int>(pitch);
    e.activation = act;
    e.words = d_hidden % 8 == 0 && all_aligned(dh, M, 16) && all_aligned(gate, M, 16) && all_aligned(up, M, 16);
    const dim3 grid(static_cast<unsigned>(ceil_div(rows * (pitch / 8), kGatedThreads)), M);
    grawa_status st = dtype == GRAWA_BF16 ? launch(gated_grad_kernel<__nv_bfloat16>, grid, kGatedThreads, 0, stream, false, e)
                                          : launch(gated_grad_kernel<__half>, grid, kGatedThreads, 0, stream, false, e);
    Operand xo, go, uo;
    if (dx) {
        if (st == GRAWA_OK) st = make_operand(&go, w_gate, d_hidden, d_in, M, f.w_gate, stream);
        if (st == GRAWA_OK) st = make_operand(&uo, w_up, d_hidden, d_in, M, f.w_up, stream);
        for (int first = 0; first < M && st == GRAWA_OK; first += kGemmWorkers) {
            GemmArgs a{};
            a.workers = std::min(kGemmWorkers, M - first);
            a.first_worker = first;
            a.m_tiles = static_cast<int>(ceil_div(rows, kTileM)); a.n_tiles = static_cast<int>(ceil_div(d_in, kTileN));
            a.k_blocks = static_cast<int>(ceil_div(d_hidden, kTileK));
            a.rows = static_cast<int>(rows); a.cols = static_cast<int>(d_in);
            a.words = d_in % 8 == 0;
            set_outputs(a, 0, dx, first, a.workers);
            st = encode_map(&a.common[0], dtype, f.da, M, rows, d_hidden, pitch, kHalf);
            if (st == GRAWA_OK) st = encode_map(&a.common[1], dtype, f.du, M, rows, d_hidden, pitch, kHalf);
            for (int w = 0; w < a.workers && st == GRAWA_OK; ++w) {
                st = encode_map(&a.per[0][w], dtype, go.base[first + w], 0, d_hidden, d_in, go.pitch, kTileK);
                if (st == GRAWA_OK) st = encode_map(&a.per[1][w], dtype, uo.base[first + w], 0, d_hidden, d_in, uo.pitch, kTileK);
            }
            if (st == GRAWA_OK) st = launch_gemm<kInputGrad>(dtype, a, stream);
        }
    }
    if (dw_gate) {
        if (st == GRAWA_OK) st = make_operand(&xo, x, rows, d_in, M, f.x, stream);
        for (int first = 0; first < M && st == GRAWA_OK; first += kGemmWorkers) {
            GemmArgs a{};
            a.workers = std::min(kGemmWorkers, M - first);
            a.first_worker = first;
            a.m_tiles = static_cast<int>(ceil_div(d_hidden, kTileM)); a.n_tiles = static_cast<int>(ceil_div(d_in, kTileN));
            a.k_blocks = static_cast<int>(ceil_div(rows, kTileK));
            a.rows = static_cast<int>(d_hidden); a.cols = static_cast<int>(d_in);
            a.words = d_in % 8 == 0;
            a.accumulate = accumulate != 0;
            set_outputs(a, 0, dw_gate, first, a.workers);
            set_outputs(a, 1, dw_up, first, a.workers);
            st = encode_map(&a.common[0], dtype, f.da, M, rows, d_hidden, pitch, kTileK);
            if (st == GRAWA_OK) st = encode_map(&a.common[1], dtype, f.du, M, rows, d_hidden, pitch, kTileK);
            for (int w = 0; w < a.workers && st == GRAWA_OK; ++w) st = encode_map(&a.per[0][w], dtype, xo.base[first + w], 0, rows, d_in, xo.pitch, kTileK);
            if (st == GRAWA_OK) st = launch_gemm<kWeightGrad>(dtype, a, stream);
        }
    }
    return st;
}

grawa_status grawa_gated_ffn_status(grawa_stream_t stream)
{
    int word = 0, zero = 0;
    GRAWA_CUDA_TRY(cudaMemcpyFromSymbolAsync(&word, g_ffn_status, sizeof word, 0, cudaMemcpyDeviceToHost, stream));
    GRAWA_CUDA_TRY(cudaStreamSynchronize(stream));
    if (word == 0) return GRAWA_OK;
    GRAWA_CUDA_TRY(cudaMemcpyToSymbolAsync(g_ffn_status, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, stream));
    GRAWA_CUDA_TRY(cudaStreamSynchronize(stream));
    return GRAWA_ERR_TIMEOUT;
}

}  // extern "C"

// Host side of the replica operators: argument checks, the choice of a kernel, launches, and their part of
// the C ABI in include/grawa.h.  No call allocates device memory or keeps anything from one call to the next.
#include <cudaTypedefs.h>

#include <cmath>
#include <cstring>
#include <map>
#include <mutex>
#include <new>
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
    return launch(kernel, dim3(static_cast<unsigned>(ctas), M), kDropThreads, 0, stream, a);
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

// Do all rows of a row-strided operand start on, and last for, multiples of `bytes`?
static bool rows_by(const void* const* table, int M, int64_t rows, int64_t cols, int64_t stride, int64_t elem, int64_t bytes)
{
    return cols * elem % bytes == 0 && (rows <= 1 || stride * elem % bytes == 0) && all_aligned(table, M, static_cast<size_t>(bytes));
}

static bool shape_ok(int64_t rows, int64_t cols, int64_t x_stride, int64_t y_stride, int M, int64_t elem)
{
    if (M < 1 || M > GRAWA_MAX_WORKERS || rows < 0 || rows > 0x7fffffff || cols < 1 || cols > (int64_t{1} << 30)) return false;
    const int64_t most = (int64_t{1} << 60) / elem;
    return x_stride >= cols && y_stride >= cols && x_stride <= most / std::max<int64_t>(1, rows) && y_stride <= most / std::max<int64_t>(1, rows);
}

template <typename T, int NV>
static grawa_status launch_norm_short(const NormForwardArgs& a, int M, cudaStream_t stream)
{
    const int64_t ctas = std::max<int64_t>(1, std::min(ceil_div(a.rows, kNormThreads / 32), static_cast<int64_t>(kSms) * kAheadCtas / M));
    return launch_clusters(layernorm_forward_short_kernel<T, NV>, dim3(static_cast<unsigned>(ctas), M), kNormThreads, 0, stream, false, 1u, a);
}

template <typename T, int MODE>
static grawa_status launch_norm_forward(const NormForwardArgs& a, int M, cudaStream_t stream)
{
    constexpr int VE = kWordElems<T>;
    constexpr int kFilled = MODE == kWhole ? kFull : MODE;    // where a row fills every word of a warp's lanes
    const int64_t words = ceil_div(a.cols, VE), per_lane = ceil_div(words, 32);
    const bool full = a.cols == per_lane * 32 * VE;
    const auto lanes = [&](auto kernel, int lpr) {
        return launch(kernel, dim3(static_cast<unsigned>(ceil_div(a.rows, kNormThreads / lpr)), M), kNormThreads, 0, stream, a);
    };
    if (words <= 8) return lanes(layernorm_forward_kernel<T, 1, 8, MODE>, 8);
    if (MODE == kWhole && per_lane <= 2 && a.has_gamma && a.has_beta && a.rows * M >= 32 * kSms * kAheadCtas &&
        all_aligned(a.gamma.p, M, 16) && all_aligned(a.beta.p, M, 16))
        return per_lane == 1 ? launch_norm_short<T, 1>(a, M, stream) : launch_norm_short<T, 2>(a, M, stream);
    if (per_lane <= 1) return lanes(full && per_lane == 1 ? layernorm_forward_kernel<T, 1, 32, kFilled> : layernorm_forward_kernel<T, 1, 32, MODE>, 32);
    if (per_lane <= 2) return lanes(full && per_lane == 2 ? layernorm_forward_kernel<T, 2, 32, kFilled> : layernorm_forward_kernel<T, 2, 32, MODE>, 32);
    if (per_lane <= 3) return lanes(full && per_lane == 3 ? layernorm_forward_kernel<T, 3, 32, kFilled> : layernorm_forward_kernel<T, 3, 32, MODE>, 32);
    if (per_lane <= 4) return lanes(full && per_lane == 4 ? layernorm_forward_kernel<T, 4, 32, kFilled> : layernorm_forward_kernel<T, 4, 32, MODE>, 32);
    if (per_lane <= 6) return lanes(full && per_lane == 6 ? layernorm_forward_kernel<T, 6, 32, kFilled> : layernorm_forward_kernel<T, 6, 32, MODE>, 32);
    if (per_lane <= 8) return lanes(full && per_lane == 8 ? layernorm_forward_kernel<T, 8, 32, kFilled> : layernorm_forward_kernel<T, 8, 32, MODE>, 32);
    if (per_lane <= 12) return lanes(full && per_lane == 12 ? layernorm_forward_kernel<T, 12, 32, kFilled> : layernorm_forward_kernel<T, 12, 32, MODE>, 32);
    if (per_lane <= 16) return lanes(full && per_lane == 16 ? layernorm_forward_kernel<T, 16, 32, kFilled> : layernorm_forward_kernel<T, 16, 32, MODE>, 32);
    constexpr int kBlockWords = 4;                            // a thread's, where a CTA holds the row
    if (words <= kNormMaxBlock * kBlockWords)
        return launch(layernorm_forward_kernel<T, kBlockWords, 0, MODE>, dim3(static_cast<unsigned>(a.rows), M),
                      static_cast<int>(ceil_div(words, 32 * kBlockWords)) * 32, 0, stream, a);
    return launch(layernorm_forward_long_kernel<T, MODE == kWhole>, dim3(static_cast<unsigned>(a.rows), M), kNormLongThreads, 0, stream, a);
}

// How the backward pass lays a row out: NV words in each of `lanes` lanes (8, 32, or a CTA's threads), rows too long for
// that apart.
struct NormLayout {
    int words, lanes;                                         // words of a lane; 0: the row is too long
};
static NormLayout norm_layout(int64_t cols, int64_t elem)
{
    const int64_t words = ceil_div(cols * elem, 16);
    const int step = elem == 4 ? 2 : 1;                       // words of 8 elements
    const int block_words = 2 * step, warp_words = 4 * step;
    if (words <= 8) return {1, 8};
    if (words <= 32 * warp_words) return {static_cast<int>(ceil_div(words, 32 * step)) * step, 32};
    if (words <= kNormMaxBlock * block_words) return {block_words, static_cast<int>(ceil_div(words, 32 * block_words)) * 32};
    return {0, 0};
}
// Slots of a part's column sums: one for every element of every thread, whether there is a column for it or not.
static int64_t norm_slots(int64_t cols, int64_t elem)
{
    const NormLayout l = norm_layout(cols, elem);
    return l.words ? static_cast<int64_t>(l.words) * l.lanes * (16 / elem) : cols;
}

// CTAs a worker's rows are split over in the backward pass (a rule on the sizes alone, so that the order of
// the additions does not change from call to call).  Few rows go to one CTA, and a moderate number to one
// cluster, which then write the gradients themselves: the second launch costs more than a few rows one after
// the other (called from Python, the second launch and its scratch take 6 us of the host's time).
constexpr int kMostCluster = 8;                               // CTAs
// Turns of each at most: some 0.8 us a turn with the rows staged ahead, and twice that without.
static int cluster_turns(RowMode mode) { return mode == kWhole ? 6 : 2; }
struct NormSplit { int parts; bool cluster; };
static NormSplit norm_split(int64_t rows, int64_t cols, int M, int64_t elem, RowMode mode)
{
    const NormLayout l = norm_layout(cols, elem);
    if (l.words == 0) {
        const int64_t want = 16 * kSms / (M * ceil_div(cols, 256));                 // CTAs of the column kernel
        return {static_cast<int>(std::max<int64_t>(1, std::min(want, ceil_div(rows, 32)))), false};
    }
    const int64_t steps = l.lanes > 32 ? rows : ceil_div(rows, kNormThreads / l.lanes);
    if (steps <= 4) return {1, false};
    if (steps <= kMostCluster * cluster_turns(mode)) return {static_cast<int>(std::min<int64_t>(kMostCluster, ceil_div(steps, 2))), true};
    // as many CTAs as their registers and stages let an SM hold at once
    const int elems = l.words * (16 / static_cast<int>(elem));
    const int64_t per_sm = l.lanes > 32 ? std::max(1, 512 / l.lanes) : norm_ctas(elems, static_cast<int>(elem));
    return {static_cast<int>(std::max<int64_t>(1, std::min(steps, kSms * per_sm / M))), false};
}

template <typename T, int NV, int LPR, int MODE>
static grawa_status launch_norm_rows(const NormBackwardArgs& a, int M, int block, cudaStream_t stream)
{
    auto* const kernel = layernorm_backward_kernel<T, NV, LPR, MODE>;
    constexpr size_t kThread = MODE == kWhole || MODE == kFull ? NormStage<NV>::bytes_a_thread : 0;
    constexpr size_t kSums = LPR == 0 ? sizeof(float2) * NV * kWordElems<T> : 0;      // a thread's column sums, where a cluster reads them
    const size_t smem = std::max(kThread, a.cluster ? kSums : 0) * block;
    // The limit belongs to the kernel, not to the call: the largest that any call needs, so that no host thread lowers it
    // between another one's setting and its launch.
    constexpr size_t kLimit = std::max(kThread, kSums) * (LPR ? kNormThreads : kNormMaxBlock);
    if (kLimit > 0) GRAWA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kLimit)));
    return launch_clusters(kernel, dim3(static_cast<unsigned>(a.parts), M), block, smem, stream, false, a.cluster ? a.parts : 1u, a);
}

template <typename T, int MODE>
static grawa_status launch_norm_backward(const NormBackwardArgs& a, int M, cudaStream_t stream)
{
    const NormLayout l = norm_layout(a.cols, sizeof(T));      // its words are one of the kernels below
    constexpr int kStep = sizeof(T) == 4 ? 2 : 1;
    // Where a row fills every word of every lane.  (16-bit rows lose by it: without the branches the compiler has more
    // values live than there are registers for; 8 x 6304 x 768 bf16: 53 us, 47 with them.)
    constexpr int kFilled = MODE == kWhole && sizeof(T) == 4 ? kFull : MODE;
    const bool full = kFilled == kFull && a.cols == static_cast<int64_t>(l.words) * l.lanes * kWordElems<T>;
    if (l.lanes == 8) return launch_norm_rows<T, 1, 8, MODE>(a, M, kNormThreads, stream);
    if (full && l.lanes == 32) {
        if (l.words == kStep) return launch_norm_rows<T, kStep, 32, kFilled>(a, M, kNormThreads, stream);
        if (l.words == 2 * kStep) return launch_norm_rows<T, 2 * kStep, 32, kFilled>(a, M, kNormThreads, stream);
        if (l.words == 3 * kStep) return launch_norm_rows<T, 3 * kStep, 32, kFilled>(a, M, kNormThreads, stream);
        return launch_norm_rows<T, 4 * kStep, 32, kFilled>(a, M, kNormThreads, stream);
    }
    if (full && l.lanes > 32) return launch_norm_rows<T, 2 * kStep, 0, kFilled>(a, M, l.lanes, stream);
    if (l.lanes == 32) {
        if (l.words == kStep) return launch_norm_rows<T, kStep, 32, MODE>(a, M, kNormThreads, stream);
        if (l.words == 2 * kStep) return launch_norm_rows<T, 2 * kStep, 32, MODE>(a, M, kNormThreads, stream);
        if (l.words == 3 * kStep) return launch_norm_rows<T, 3 * kStep, 32, MODE>(a, M, kNormThreads, stream);
        return launch_norm_rows<T, 4 * kStep, 32, MODE>(a, M, kNormThreads, stream);
    }
    if (l.lanes > 32) return launch_norm_rows<T, 2 * kStep, 0, MODE>(a, M, l.lanes, stream);
    if (a.has_dx) {
        const grawa_status st = launch(layernorm_backward_long_kernel<T, MODE == kWhole>, dim3(static_cast<unsigned>(a.rows), M), kNormLongThreads, 0, stream, a);
        if (st != GRAWA_OK) return st;
    }
    if (!a.has_dgamma && !a.has_dbeta) return GRAWA_OK;
    return launch(layernorm_columns_kernel<T, MODE == kWhole>, dim3(static_cast<unsigned>(ceil_div(a.cols, 32 * (MODE == kWhole ? kWordElems<T> : 1))), M, a.parts), kNormThreads, 0, stream, a);
}

template <typename T>
static grawa_status norm_backward(const NormBackwardArgs& a, int M, RowMode mode, cudaStream_t stream)
{
    if (a.rows > 0) {
        grawa_status st;
        if (mode == kWhole) st = launch_norm_backward<T, kWhole>(a, M, stream);
        else if (sizeof(T) == 4 || mode == kUnits) st = launch_norm_backward<T, kUnits>(a, M, stream);
        else st = launch_norm_backward<T, sizeof(T) == 4 ? kUnits : kHalves>(a, M, stream);
        if (st != GRAWA_OK || a.parts == 1 || a.cluster) return st;
    }
    if (!a.has_dgamma && !a.has_dbeta) return GRAWA_OK;
    return launch(layernorm_finish_kernel<T>, dim3(static_cast<unsigned>(ceil_div(a.slots, 32)), M), 32 * kFinishGroups, 0, stream, a);
}

template <typename T>
static grawa_status norm_forward(const NormForwardArgs& a, int M, RowMode mode, cudaStream_t stream)
{
    if (mode == kWhole) return launch_norm_forward<T, kWhole>(a, M, stream);
    if (sizeof(T) == 4 || mode == kUnits) return launch_norm_forward<T, kUnits>(a, M, stream);
    return launch_norm_forward<T, sizeof(T) == 4 ? kUnits : kHalves>(a, M, stream);
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

// Operands of one shape: those that cannot be read in place are laid out again, all in one launch.
static grawa_status make_operands(Operand* const* ops, const void* const* const* tables, void* const* scratch, int count, int64_t rows, int64_t cols, int M,
                                  cudaStream_t stream)
{
    PackArgs a{};
    int packed = 0;
    for (int i = 0; i < count; ++i) {
        Operand& op = *ops[i];
        op.rows = rows; op.cols = cols; op.pitch = pitch_of(cols);
        const bool stays = in_place(cols, all_aligned(tables[i], M, 16));
        unsigned short* to = static_cast<unsigned short*>(scratch[i]);
        for (int m = 0; m < M; ++m) op.base[m] = stays ? tables[i][m] : to + static_cast<size_t>(m) * rows * op.pitch;
        if (stays) continue;
        copy_table(a.from[packed], tables[i], M);
        a.to[packed++] = to;
    }
    if (packed == 0) return GRAWA_OK;
    a.rows = rows; a.cols = static_cast<int>(cols); a.pitch = static_cast<int>(pitch_of(cols));
    return launch(pack_rows_kernel, dim3(static_cast<unsigned>(ceil_div(rows * (a.pitch / 8), kGatedThreads)), M, packed), kGatedThreads, 0, stream, a);
}
static grawa_status make_operand(Operand* op, const void* const* table, int64_t rows, int64_t cols, int M, void* scratch, cudaStream_t stream)
{
    return make_operands(&op, &table, &scratch, 1, rows, cols, M, stream);
}
static grawa_status make_weights(Operand* gate, Operand* up, const void* const* w_gate, const void* const* w_up, int64_t d_hidden, int64_t d_in, int M,
                                 void* gate_scratch, void* up_scratch, cudaStream_t stream)
{
    Operand* const ops[2] = {gate, up};
    const void* const* const tables[2] = {w_gate, w_up};
    void* const scratch[2] = {gate_scratch, up_scratch};
    return make_operands(ops, tables, scratch, 2, d_hidden, d_in, M, stream);
}

// The number of parts that the sum of a product of `tiles` tiles, of `blocks` steps each, is split into: by an estimate of
// the time in microseconds (a step 0.4, a tile's start and results 3; a second kernel 3, and the parts written and
// read at 5 TB/s).
static int64_t gemm_splits(int64_t tiles, int64_t blocks, double tile_bytes)
{
    const int64_t pairs = kSms / 2;
    if (tiles >= pairs) return 1;
    const auto time = [&](int64_t s) {
        const double steps = static_cast<double>(ceil_div(tiles * s, pairs) * ceil_div(blocks, s));
        return steps * 0.4 + 3.0 + (s > 1 ? 3.0 + static_cast<double>(tiles * s) * 2.0 * tile_bytes / 5e6 : 0.0);
    };
    int64_t best = 1;
    for (int64_t s = 2; s <= std::min<int64_t>(blocks, 16); ++s)
        if (time(s) < time(best)) best = s;
    return best;
}

// A product of [out_rows][out_cols] results for each of `copies` matrices: its tiles, with `halves` sums of `sum` elements
// that add up in one result.  Splits are set apart (set_splits).
static GemmPart gemm_part(int64_t copies, int64_t out_rows, int64_t out_cols, int tile_cols, int64_t sum, int halves)
{
    GemmPart p{};
    p.m_tiles = static_cast<int>(ceil_div(out_rows, kTileM));
    p.n_tiles = static_cast<int>(ceil_div(out_cols, tile_cols));
    p.tiles = p.units = static_cast<int>(copies * p.m_tiles * p.n_tiles);
    p.half_blocks = static_cast<int>(ceil_div(sum, kTileK));
    p.blocks = p.split_blocks = p.half_blocks * halves;
    p.splits = 1;
    p.rows = static_cast<int>(out_rows);
    p.cols = static_cast<int>(out_cols);
    return p;
}
static void set_splits(GemmPart& p, int64_t splits)
{
    p.split_blocks = static_cast<int>(ceil_div(p.blocks, splits));
    p.splits = static_cast<int>(ceil_div(p.blocks, p.split_blocks));
    p.units = p.tiles * p.splits;
}
static size_t partial_bytes(const GemmPart& p) { return p.splits > 1 ? static_cast<size_t>(p.units) * kTileM * kTileN * sizeof(float) : 0; }
// What the results of a tile come to in fp32 (rows behind the edge are not written).
static double tile_bytes(const GemmPart& p) { return std::min(kTileM, (p.rows + 31) / 32 * 32) * static_cast<double>(kTileN) * 4.0; }

static GemmPart forward_part(int workers, int64_t rows, int64_t d_in, int64_t d_hidden)
{
    GemmPart p = gemm_part(workers, rows, d_hidden, kHalf, d_in, 1);
    set_splits(p, gemm_splits(p.tiles, p.blocks, tile_bytes(p)));
    return p;
}

// The two products of a backward pass.  Where all their operands and results fit in L2 together, one launch takes both:
// the pairs of SMs then share out the steps of both evenly, where two launches leave many idle at the end of each
// (2 x 1576 tokens, 768 -> 2050: 66 steps for 42 pairs, then 25 steps for 108 tiles on 74 pairs).
struct BackwardPlan {
    GemmPart part[2];
    bool together;
};
static BackwardPlan backward_plan(int workers, int64_t rows, int64_t d_in, int64_t d_hidden, bool want_dx, bool want_dw)
{
    BackwardPlan b{};
    if (want_dx) b.part[kInputGrad] = gemm_part(workers, rows, d_in, kTileN, d_hidden, 2);
    if (want_dw) b.part[kWeightGrad] = gemm_part(2 * workers, d_hidden, d_in, kTileN, rows, 1);
    constexpr double kFitsL2 = 96e6;
    const double bytes = 2.0 * workers * (2.0 * rows * d_hidden + 4.0 * d_hidden * d_in + 2.0 * rows * d_in);
    b.together = want_dx && want_dw && bytes <= kFitsL2;
    if (b.together) {
        // no unit much longer than an even share of all the steps: a sum is split where that saves more than joining its
        // parts costs (and not into units of less than 8 steps)
        const int64_t all = static_cast<int64_t>(b.part[0].tiles) * b.part[0].blocks + static_cast<int64_t>(b.part[1].tiles) * b.part[1].blocks;
        const int64_t share = std::max<int64_t>(8, ceil_div(all, kSms / 2)) * 5 / 4;
        for (GemmPart& p : b.part) set_splits(p, ceil_div(p.blocks, share));
    } else {
        for (GemmPart& p : b.part)
            if (p.tiles) set_splits(p, gemm_splits(p.tiles, p.blocks, tile_bytes(p)));
    }
    return b;
}

// Scratch for the parts of split sums (the launches of a call use it one after the other), with whatever gradients the
// call wants.
static size_t forward_partial_bytes(int M, int64_t rows, int64_t d_in, int64_t d_hidden)
{
    size_t most = 0;
    for (int first = 0; first < M; first += kGemmWorkers) most = std::max(most, partial_bytes(forward_part(std::min(kGemmWorkers, M - first), rows, d_in, d_hidden)));
    return most;
}
static size_t backward_partial_bytes(int M, int64_t rows, int64_t d_in, int64_t d_hidden)
{
    size_t most = 0;
    for (int first = 0; first < M; first += kGemmWorkers)
        for (int want = 1; want < 4; ++want) {
            const BackwardPlan b = backward_plan(std::min(kGemmWorkers, M - first), rows, d_in, d_hidden, want & 1, want & 2);
            most = std::max(most, partial_bytes(b.part[0]) + partial_bytes(b.part[1]));
        }
    return most;
}

// Shares the units of both parts out among the pairs: the longer ones in turn, then the shorter ones so that all pairs
// come to about the same number of steps (a unit counts for 2 more, and for at least the 7 that its results take).
static void set_shares(GemmArgs& a, int pairs)
{
    const auto length = [](const GemmPart& p) { return std::max(7, p.split_blocks) + 2; };
    a.lead = a.part[1].units == 0 || (a.part[0].units > 0 && length(a.part[0]) >= length(a.part[1])) ? 0 : 1;
    const GemmPart &lead = a.part[a.lead], &rest = a.part[1 - a.lead];
    if (rest.units == 0) return;                              // all shares are empty
    const int64_t len = length(rest);
    const auto load = [&](int p) { return static_cast<int64_t>(lead.units > p ? (lead.units - p + pairs - 1) / pairs : 0) * length(lead); };
    const auto takes = [&](int p, int64_t level) { return std::max<int64_t>(0, (level - load(p)) / len); };
    int64_t low = 0, high = load(0) + len * (rest.units + 1);  // the lowest level at which the pairs take all units
    while (low < high) {
        const int64_t level = (low + high) / 2;
        int64_t taken = 0;
        for (int p = 0; p < pairs; ++p) taken += takes(p, level);
        if (taken >= rest.units) high = level;
        else low = level + 1;
    }
    int64_t at = 0;
    for (int p = 0; p < pairs; ++p) {
        a.share[p] = static_cast<int>(at);
        at = std::min<int64_t>(rest.units, at + takes(p, low));
    }
    a.share[pairs] = rest.units;
}

template <typename T, bool FORWARD>
static grawa_status launch_gemm(GemmArgs& a, cudaStream_t stream)
{
    const int64_t units = static_cast<int64_t>(a.part[0].units) + a.part[1].units;
    if (units == 0) return GRAWA_OK;
    const int pairs = static_cast<int>(std::min<int64_t>(units, kSms / 2));
    set_shares(a, pairs);
    GRAWA_CUDA_TRY(cudaFuncSetAttribute(gemm_kernel<T, FORWARD>, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem));
    grawa_status st = launch(gemm_kernel<T, FORWARD>, dim3(static_cast<unsigned>(2 * pairs)), kGemmThreads, kGemmSmem, stream, a);
    for (int part = 0; part < 2 && st == GRAWA_OK; ++part)
        if (a.part[part].splits > 1)
            st = launch(gemm_join_kernel<T, FORWARD>, dim3(static_cast<unsigned>(a.part[part].tiles), kTileM / 32, (FORWARD ? kHalf : kTileN) / 32), kJoinThreads,
                        0, stream, a, part);
    return st;
}
template <bool FORWARD>
static grawa_status launch_gemm(grawa_dtype dtype, GemmArgs& a, cudaStream_t stream)
{
    return dtype == GRAWA_BF16 ? launch_gemm<__nv_bfloat16, FORWARD>(a, stream) : launch_gemm<__half, FORWARD>(a, stream);
}

// Up to kFewRows rows go by the kernel for a few rows.  (4 workers, 2048 -> 5632, bf16: 31 us for 1 row and 39 for 16,
// against 55 and 50 by the tensor cores' tiles; 24 rows 67 against 49.  Narrow weights leave most SMs idle, and it still
// wins: 1 worker, 4096 -> 64, 5.5 to 13 us against 16 to 18; only a very long sum loses, 12288 -> 17 at odd places 21 to 32
// against 16.)
static bool takes_few(int64_t rows) { return rows <= kFewRows; }

template <typename T, int NT>
static grawa_status launch_few(const FewArgs& a, int M, FewMode mode, cudaStream_t stream)
{
    auto* const kernel = mode == kFewWhole ? gated_few_kernel<T, NT, kFewWhole> : mode == kFewShifted ? gated_few_kernel<T, NT, kFewShifted> : gated_few_kernel<T, NT, kFewAny>;
    return launch(kernel, dim3(static_cast<unsigned>(ceil_div(a.d_hidden, kFewCols)), M), kFewThreads, 0, stream, a);
}
template <typename T>
static grawa_status launch_few(const FewArgs& a, int M, FewMode mode, cudaStream_t stream)
{
    return a.rows <= 8 ? launch_few<T, 1>(a, M, mode, stream) : launch_few<T, 2>(a, M, mode, stream);
}

// Outputs of the workers [first, first + count); whether they take 16-byte stores.
static bool set_outputs(GemmArgs& a, int slot, void* const* table, int first, int count)
{
    bool words = true;
    for (int w = 0; w < count; ++w) {
        a.out[slot][w] = table ? table[first + w] : nullptr;
        words = words && aligned(a.out[slot][w], 16);
    }
    return words;
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
    void *x, *w_gate, *w_up, *da, *du, *partial;
    size_t bytes;
};
static FfnScratch ffn_scratch(void* base, int64_t rows, int64_t d_in, int64_t d_hidden, int M, bool x_ok, bool w_ok, bool backward)
{
    Scratch s{static_cast<char*>(base)};
    FfnScratch f{};
    if (rows == 0 || (!backward && takes_few(rows))) return f;
    f.x = operand_scratch(s, rows, d_in, M, x_ok);
    f.w_gate = operand_scratch(s, d_hidden, d_in, M, w_ok);
    f.w_up = operand_scratch(s, d_hidden, d_in, M, w_ok);
    if (backward) {
        f.da = s.take(static_cast<size_t>(M) * rows * pitch_of(d_hidden) * 2);
        f.du = s.take(static_cast<size_t>(M) * rows * pitch_of(d_hidden) * 2);
        f.partial = s.take(backward_partial_bytes(M, rows, d_in, d_hidden));
    } else {
        f.partial = s.take(forward_partial_bytes(M, rows, d_in, d_hidden));
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
    const auto by = [&](int64_t bytes) { return rows_by(x, M, rows, cols, x_stride, elem, bytes) && rows_by(y, M, rows, cols, y_stride, elem, bytes); };
    const RowMode mode = by(16) ? kWhole : by(4) ? kUnits : kHalves;
    if (dtype == GRAWA_BF16) return norm_forward<__nv_bfloat16>(a, M, mode, stream);
    if (dtype == GRAWA_F16) return norm_forward<__half>(a, M, mode, stream);
    return norm_forward<float>(a, M, mode, stream);
}

size_t grawa_layernorm_backward_workspace_bytes(int64_t rows, int64_t cols, int M, int aligned)
{
    if (!shape_ok(rows, cols, cols, cols, M, 4)) return 0;
    size_t most = 0;                                          // of the storage types
    for (const int64_t elem : {int64_t{2}, int64_t{4}}) {
        const NormSplit s = norm_split(rows, cols, M, elem, aligned ? kWhole : kUnits);
        if (s.parts > 1 && !s.cluster) most = std::max(most, static_cast<size_t>(M) * s.parts * 2 * norm_slots(cols, elem) * sizeof(float));
    }
    return most;
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
    const auto by = [&](int64_t bytes) {
        return rows_by(x, M, rows, cols, x_stride, elem, bytes) && rows_by(dy, M, rows, cols, y_stride, elem, bytes) &&
               (!dx || rows_by(dx, M, rows, cols, x_stride, elem, bytes));
    };
    const RowMode mode = by(16) ? kWhole : by(4) ? kUnits : kHalves;
    const NormSplit split = norm_split(rows, cols, M, elem, mode);
    const size_t need = weights && rows > 0 && split.parts > 1 && !split.cluster ? grawa_layernorm_backward_workspace_bytes(rows, cols, M, mode == kWhole) : 0;
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
    a.parts = rows == 0 ? 0 : split.parts;
    a.cluster = split.cluster;
    a.has_gamma = gamma != nullptr; a.has_dx = dx != nullptr; a.has_dgamma = dgamma != nullptr; a.has_dbeta = dbeta != nullptr;
    a.accumulate = accumulate != 0;
    const NormLayout l = norm_layout(cols, elem);
    a.slots = static_cast<int>(norm_slots(cols, elem));
    a.lanes = l.words ? l.lanes : a.slots;
    a.word = l.words == 0 ? 1 : static_cast<int>((mode == kUnits ? 4 : 16) / elem);
    if (dtype == GRAWA_BF16) return norm_backward<__nv_bfloat16>(a, M, mode, stream);
    if (dtype == GRAWA_F16) return norm_backward<__half>(a, M, mode, stream);
    return norm_backward<float>(a, M, mode, stream);
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

    if (takes_few(rows)) {
        FewArgs a{};
        copy_table(a.x, x, M);
        copy_table(a.w_gate, w_gate, M);
        copy_table(a.w_up, w_up, M);
        copy_table(a.h, h, M);
        copy_table(a.gate, gate_out, M);
        copy_table(a.up, up_out, M);
        a.rows = static_cast<int>(rows); a.d_in = static_cast<int>(d_in); a.d_hidden = static_cast<int>(d_hidden);
        a.activation = act;
        const bool all = all_aligned(x, M, 16) && all_aligned(w_gate, M, 16) && all_aligned(w_up, M, 16);
        const FewMode mode = d_in % 8 ? kFewAny : all ? kFewWhole : kFewShifted;
        return dtype == GRAWA_BF16 ? launch_few<__nv_bfloat16>(a, M, mode, stream) : launch_few<__half>(a, M, mode, stream);
    }
    Operand xo, go, uo;
    grawa_status st = make_operand(&xo, x, rows, d_in, M, f.x, stream);
    if (st == GRAWA_OK) st = make_weights(&go, &uo, w_gate, w_up, d_hidden, d_in, M, f.w_gate, f.w_up, stream);
    for (int first = 0; first < M && st == GRAWA_OK; first += kGemmWorkers) {
        GemmArgs a{};
        a.workers = std::min(kGemmWorkers, M - first);
        a.first_worker = first;
        a.activation = act;
        GemmPart& p = a.part[0];
        p = forward_part(a.workers, rows, d_in, d_hidden);
        p.partial = static_cast<float*>(f.partial);
        p.words = d_hidden % 8 == 0;
        p.words = set_outputs(a, 0, h, first, a.workers) && p.words;
        p.words = set_outputs(a, 1, gate_out, first, a.workers) && p.words;
        p.words = set_outputs(a, 2, up_out, first, a.workers) && p.words;
        for (int w = 0; w < a.workers && st == GRAWA_OK; ++w) {
            st = encode_map(&a.per[0][w], dtype, xo.base[first + w], 0, rows, d_in, xo.pitch, kHalf);
            if (st == GRAWA_OK) st = encode_map(&a.per[1][w], dtype, go.base[first + w], 0, d_hidden, d_in, go.pitch, kHalf);
            if (st == GRAWA_OK) st = encode_map(&a.per[2][w], dtype, uo.base[first + w], 0, d_hidden, d_in, uo.pitch, kHalf);
        }
        if (st == GRAWA_OK) st = launch_gemm<true>(dtype, a, stream);
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
    const auto by = [&](size_t bytes) {
        return d_hidden * 2 % static_cast<int64_t>(bytes) == 0 && all_aligned(dh, M, bytes) && all_aligned(gate, M, bytes) && all_aligned(up, M, bytes);
    };
    const int step = by(16) ? 8 : by(4) ? 2 : 1;
    const int64_t threads = rows * (step == 8 ? pitch / 8 : ceil_div(pitch, 256) * 32);
    const auto elementwise = [&](auto kernel) {
        return launch(kernel, dim3(static_cast<unsigned>(ceil_div(threads, kGatedThreads)), M), kGatedThreads, 0, stream, e);
    };
    const auto of_type = [&](auto type) {
        using T = decltype(type);
        return step == 8 ? elementwise(gated_grad_kernel<T, 8>) : step == 2 ? elementwise(gated_grad_kernel<T, 2>) : elementwise(gated_grad_kernel<T, 1>);
    };
    grawa_status st = dtype == GRAWA_BF16 ? of_type(__nv_bfloat16{}) : of_type(__half{});
    Operand xo, go, uo;
    if (st == GRAWA_OK && dx) st = make_weights(&go, &uo, w_gate, w_up, d_hidden, d_in, M, f.w_gate, f.w_up, stream);
    if (st == GRAWA_OK && dw_gate) st = make_operand(&xo, x, rows, d_in, M, f.x, stream);
    for (int first = 0; first < M && st == GRAWA_OK; first += kGemmWorkers) {
        GemmArgs a{};
        a.workers = std::min(kGemmWorkers, M - first);
        a.first_worker = first;
        a.accumulate = accumulate != 0;
        const BackwardPlan plan = backward_plan(a.workers, rows, d_in, d_hidden, dx != nullptr, dw_gate != nullptr);
        GemmPart parts[2] = {plan.part[0], plan.part[1]};
        parts[0].partial = static_cast<float*>(f.partial);
        parts[1].partial = parts[0].partial + partial_bytes(parts[0]) / sizeof(float);
        const bool whole = d_in % 8 == 0;
        parts[0].words = set_outputs(a, 0, dx, first, a.workers) && whole;
        parts[1].words = set_outputs(a, 1, dw_gate, first, a.workers) && whole;
        parts[1].words = set_outputs(a, 2, dw_up, first, a.workers) && parts[1].words;
        const void* const halves[2] = {f.da, f.du};
        for (int i = 0; i < 2 && st == GRAWA_OK; ++i) {
            st = encode_map(&a.common[i], dtype, halves[i], M, rows, d_hidden, pitch, kHalf);
            if (st == GRAWA_OK) st = encode_map(&a.common[2 + i], dtype, halves[i], M, rows, d_hidden, pitch, kTileK);
        }
        for (int w = 0; w < a.workers && st == GRAWA_OK; ++w) {
            if (dx) {
                st = encode_map(&a.per[0][w], dtype, go.base[first + w], 0, d_hidden, d_in, go.pitch, kTileK);
                if (st == GRAWA_OK) st = encode_map(&a.per[1][w], dtype, uo.base[first + w], 0, d_hidden, d_in, uo.pitch, kTileK);
            }
            if (st == GRAWA_OK && dw_gate) st = encode_map(&a.per[2][w], dtype, xo.base[first + w], 0, rows, d_in, xo.pitch, kTileK);
        }
        if (plan.together) {
            a.part[0] = parts[0];
            a.part[1] = parts[1];
            if (st == GRAWA_OK) st = launch_gemm<false>(dtype, a, stream);
        } else {
            for (int i = 0; i < 2 && st == GRAWA_OK; ++i) {
                a.part[i] = parts[i];
                a.part[1 - i] = GemmPart{};
                st = launch_gemm<false>(dtype, a, stream);
            }
        }
    }
    return st;
}

grawa_status grawa_selftest_gated_ffn_wait(grawa_stream_t stream)
{
    auto* const kernel = gemm_kernel<__nv_bfloat16, true, true>;
    GemmArgs a{};                                             // two tiles of one worker, of four steps; no operands, no outputs
    a.workers = 1;
    a.part[0] = gemm_part(1, 2 * kTileM, kHalf, kHalf, 4 * kTileK, 1);
    GRAWA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem));
    return launch(kernel, dim3(2), kGemmThreads, kGemmSmem, stream, a);
}

grawa_status grawa_gated_ffn_status(grawa_stream_t stream)
{
    // What each stream's reports have seen of its device's count.  A call's own stream is not known to the count (a captured
    // call may run on any), so every stream is told of every wait that ran out, once.
    int device = 0;
    unsigned count = 0;
    GRAWA_CUDA_TRY(cudaGetDevice(&device));
    GRAWA_CUDA_TRY(cudaMemcpyFromSymbolAsync(&count, g_ffn_timeouts, sizeof count, 0, cudaMemcpyDeviceToHost, stream));
    GRAWA_CUDA_TRY(cudaStreamSynchronize(stream));
    try {
        static std::mutex mutex;
        static auto& seen = *new std::map<std::pair<int, cudaStream_t>, unsigned>;
        const std::lock_guard<std::mutex> lock(mutex);
        unsigned& last = seen[{device, stream}];
        if (static_cast<int>(count - last) <= 0) return GRAWA_OK;      // (another thread's report may have seen more)
        last = count;
        return GRAWA_ERR_TIMEOUT;
    } catch (const std::bad_alloc&) {
        return cuda_fail(cudaErrorMemoryAllocation, "grawa_gated_ffn_status");
    }
}

}  // extern "C"

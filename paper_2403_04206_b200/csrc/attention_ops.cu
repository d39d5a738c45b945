// Host side of attention within a window: argument checks, the choice of a kernel, launches, and its part of the C ABI in
// include/grawa.h.  No call allocates device memory or keeps anything from one call to the next.
#include <cmath>
#include <utility>

#include "attention.cuh"
#include "replica_host.h"

namespace grawa {
namespace replica {

// ------------------------------------------------------------------ attention within a window

struct AttentionShape {
    grawa_dtype dtype;
    const int64_t* const* offsets;
    int64_t sequences, period, left, right, sinks, rows, q_heads, kv_heads, head_dim;
    int64_t q_stride, k_stride, v_stride, out_stride;
    int M;
    float scale;
};

static bool attention_shape_ok(const AttentionShape& s)
{
    constexpr int64_t kMostStride = int64_t{1} << 38;          // of a tensor map, in elements
    if ((s.dtype != GRAWA_BF16 && s.dtype != GRAWA_F16) || s.M < 1 || s.M > GRAWA_MAX_WORKERS) return false;
    if (s.rows < 0 || s.rows > 0x7fffffff - 1024 || s.q_heads < 1 || s.q_heads > 0x7fff || s.kv_heads < 1 || s.q_heads % s.kv_heads != 0) return false;
    if (ceil_div(s.rows, kTile) * s.q_heads * std::min(s.M, kAttentionWorkers) > 0x7fffffff - 4096) return false;          // tiles of a launch
    if (s.head_dim < 8 || s.head_dim > 128 || s.head_dim % 8 != 0) return false;
    if (s.left < 0 || s.right < 0 || s.sinks < 0 || !(s.scale > 0.0f) || std::isinf(s.scale)) return false;
    if (s.offsets ? s.sequences < 0 || s.sequences > 0x7fffffff - 1 : s.period < 1) return false;
    for (const int64_t stride : {s.q_stride, s.out_stride})
        if (stride % 8 != 0 || stride > kMostStride || !stride_ok(s.rows, s.q_heads * s.head_dim, stride)) return false;
    for (const int64_t stride : {s.k_stride, s.v_stride})
        if (stride % 8 != 0 || stride > kMostStride || !stride_ok(s.rows, s.kv_heads * s.head_dim, stride)) return false;
    return true;
}

// 16-byte aligned rows of heads.
static bool add_heads(Buffers& b, const void* const* table, const AttentionShape& s, int64_t heads, int64_t stride, bool output)
{
    return all_aligned(table, s.M, 16) && b.add(table, s.M, s.rows, heads * s.head_dim, stride, 2, output);
}
static bool add_offsets(Buffers& b, const AttentionShape& s)
{
    return !s.offsets || b.add(reinterpret_cast<const void* const*>(s.offsets), s.M, 1, s.sequences + 1, s.sequences + 1, 8, false);
}

static AttentionArgs attention_args(const AttentionShape& s, const void* const* q, const void* const* k, const void* const* v)
{
    AttentionArgs a{};
    copy_table(a.q, q, s.M);
    copy_table(a.k, k, s.M);
    copy_table(a.v, v, s.M);
    copy_table(a.offsets, s.offsets, s.M);
    a.q_stride = s.q_stride; a.k_stride = s.k_stride; a.v_stride = s.v_stride; a.out_stride = s.out_stride;
    a.rows = static_cast<int>(s.rows); a.heads = static_cast<int>(s.q_heads); a.kv_heads = static_cast<int>(s.kv_heads);
    a.group = a.heads / a.kv_heads; a.dim = static_cast<int>(s.head_dim);
    a.sequences = static_cast<int>(s.offsets ? s.sequences : 0);
    a.period = divisor(static_cast<unsigned>(std::min(s.offsets ? s.rows : s.period, s.rows)));
    a.group_size = divisor(static_cast<unsigned>(a.group));
    a.left = static_cast<int>(std::min(s.left, s.rows)); a.right = static_cast<int>(std::min(s.right, s.rows));
    a.sinks = static_cast<int>(std::min(s.sinks, s.rows));
    a.scale = s.scale;
    return a;
}

// Map of a worker's heads as [row][head][element], for boxes of 64 elements of one head by 64 rows.
static grawa_status encode_heads(CUtensorMap* map, grawa_dtype dtype, const void* base, const AttentionShape& s, int64_t heads, int64_t stride)
{
    PFN_cuTensorMapEncodeTiled_v12000 encode = nullptr;
    const grawa_status st = map_encoder(&encode);
    if (st != GRAWA_OK) return st;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(s.head_dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(s.rows)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(s.head_dim) * 2, static_cast<cuuint64_t>(stride) * 2};
    const cuuint32_t box[3] = {kBox, 1, kBox}, step[3] = {1, 1, 1};
    const CUresult res = encode(map, dtype == GRAWA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims,
                                strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return res == CUDA_SUCCESS ? GRAWA_OK : cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
}

// The workers [first, first + count) of a launch, with the maps of q, k, v and (backward) dout.
static grawa_status set_workers(TileArgs& t, const AttentionShape& s, int first, int count)
{
    t.first_worker = first;
    t.workers = count;
    grawa_status st = GRAWA_OK;
    for (int w = 0; w < count && st == GRAWA_OK; ++w) {
        const int m = first + w;
        st = encode_heads(&t.map[0][w], s.dtype, t.a.q.p[m], s, s.q_heads, s.q_stride);
        if (st == GRAWA_OK) st = encode_heads(&t.map[1][w], s.dtype, t.a.k.p[m], s, s.kv_heads, s.k_stride);
        if (st == GRAWA_OK) st = encode_heads(&t.map[2][w], s.dtype, t.a.v.p[m], s, s.kv_heads, s.v_stride);
        if (st == GRAWA_OK && t.a.dout.p[m]) st = encode_heads(&t.map[3][w], s.dtype, t.a.dout.p[m], s, s.q_heads, s.out_stride);
    }
    return st;
}

// As many CTAs as the SMs hold, `per_sm` each, or one a tile.
template <typename Kernel>
static grawa_status launch_tiles(Kernel kernel, const TileArgs& t, int heads, int per_sm, int threads, int smem, cudaStream_t stream)
{
    GRAWA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    const int64_t units = (t.far ? t.chunks : ceil_div(t.a.rows, kTile)) * heads * t.workers;
    TileArgs args = t;
    args.per = divisor(static_cast<unsigned>(heads * t.workers));
    args.per_worker = divisor(static_cast<unsigned>(heads));
    return launch(kernel, dim3(static_cast<unsigned>(std::min<int64_t>(units, kSms * per_sm))), threads, smem, stream, args);
}
template <typename T>
static grawa_status launch_forward(const TileArgs& t, cudaStream_t stream)
{
    return t.a.dim <= 64 ? launch_tiles(attention_forward_kernel<T, 64>, t, t.a.heads, 2, kForwardThreads, kForwardSmem<64>, stream)
                         : launch_tiles(attention_forward_kernel<T, 128>, t, t.a.heads, 2, kForwardThreads, kForwardSmem<128>, stream);
}
template <typename T, bool KEYS>
static grawa_status launch_backward(const TileArgs& t, cudaStream_t stream)
{
    const int heads = KEYS ? t.a.kv_heads : t.a.heads;
    return t.a.dim <= 64 ? launch_tiles(attention_backward_kernel<T, 64, KEYS>, t, heads, 1, kBackwardThreads, kBackwardSmem<64, KEYS>, stream)
                         : launch_tiles(attention_backward_kernel<T, 128, KEYS>, t, heads, 1, kBackwardThreads, kBackwardSmem<128, KEYS>, stream);
}

// The places of a backward call's scratch: lse and delta of every row, the longest rows, and the sums of chunks of queries for the
// first keys.
struct AttentionScratch {
    int64_t pitch, chunks;                                    // chunks: 0 where none are set apart
    size_t delta, longest, partial, bytes;                    // offsets (lse stands first), and the whole
};
// Chunks are set apart for up to a tile of first keys.  (Where the window leaves no query beyond the first chunk, none has work.)
static AttentionScratch attention_scratch(int64_t rows, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t sinks, int M)
{
    AttentionScratch s{};
    s.pitch = ceil_div(rows, 64) * 64 + 64;                   // a step of queries starts at a multiple of 64 rows
    s.chunks = sinks > 0 && sinks <= kTile && rows > kChunk ? ceil_div(rows, kChunk) : 0;
    const size_t table = static_cast<size_t>(M) * q_heads * s.pitch * sizeof(float);        // a multiple of 256 bytes
    s.delta = table;
    s.longest = 2 * table;
    s.partial = 2 * table + (static_cast<size_t>(M) * 2 * sizeof(float) + 255) / 256 * 256;
    s.bytes = s.partial + static_cast<size_t>(M) * kv_heads * s.chunks * 2 * std::min<int64_t>(sinks, kTile) * head_dim * sizeof(float);
    return s;
}

template <typename T>
static grawa_status attention_stats(const StatsArgs& t, int M, cudaStream_t stream)
{
    const int heads = t.a.heads + (t.longest ? t.a.kv_heads : 0);
    auto* const kernel = t.a.dim <= 64 ? attention_stats_kernel<T, 8> : attention_stats_kernel<T, 16>;
    return launch(kernel, dim3(static_cast<unsigned>(t.pitch / 64), heads, M), kStatsThreads, 0, stream, t);
}

}  // namespace replica
}  // namespace grawa

using namespace grawa;
using namespace grawa::replica;

extern "C" {

grawa_status grawa_window_attention_forward(grawa_dtype dtype, const void* const* q, const void* const* k, const void* const* v, void* const* out,
                                            float* const* lse, const int64_t* const* offsets, int64_t sequences, int64_t period, int64_t left,
                                            int64_t right, int64_t sinks, int64_t rows, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                                            int64_t q_stride, int64_t k_stride, int64_t v_stride, int64_t out_stride, int M, float scale,
                                            grawa_stream_t stream)
{
    const AttentionShape s{dtype, offsets, sequences, period, left, right, sinks, rows, q_heads, kv_heads, head_dim, q_stride, k_stride, v_stride, out_stride, M, scale};
    if (!attention_shape_ok(s) || !q || !k || !v || !out) return GRAWA_ERR_INVALID_ARG;
    if (rows == 0) return GRAWA_OK;
    Buffers b;
    if (!add_heads(b, q, s, q_heads, q_stride, false) || !add_heads(b, k, s, kv_heads, k_stride, false) || !add_heads(b, v, s, kv_heads, v_stride, false) ||
        !add_heads(b, out, s, q_heads, out_stride, true) || !add_offsets(b, s)) return GRAWA_ERR_INVALID_ARG;
    if (lse && !b.add(reinterpret_cast<const void* const*>(lse), M, 1, q_heads * rows, q_heads * rows, 4, true)) return GRAWA_ERR_INVALID_ARG;
    if (b.clash()) return GRAWA_ERR_INVALID_ARG;
    TileArgs t{};
    t.a = attention_args(s, q, k, v);
    copy_table(t.a.to[0], out, M);
    copy_table(t.a.to[1], lse, M);
    grawa_status st = GRAWA_OK;
    for (int first = 0; first < M && st == GRAWA_OK; first += kAttentionWorkers) {
        st = set_workers(t, s, first, std::min(kAttentionWorkers, M - first));
        if (st == GRAWA_OK) st = dtype == GRAWA_BF16 ? launch_forward<__nv_bfloat16>(t, stream) : launch_forward<__half>(t, stream);
    }
    return st;
}

size_t grawa_window_attention_backward_workspace_bytes(int64_t rows, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t sinks, int M)
{
    if (q_heads < 1 || q_heads > 0x7fff || kv_heads < 1 || kv_heads > q_heads || head_dim < 8 || head_dim > 128) return 0;
    const int64_t wide = q_heads * head_dim, narrow = kv_heads * head_dim;
    if (!attention_shape_ok({GRAWA_BF16, nullptr, 0, 1, 0, 0, sinks, rows, q_heads, kv_heads, head_dim, wide, narrow, narrow, wide, M, 1.0f})) return 0;
    return attention_scratch(rows, q_heads, kv_heads, head_dim, sinks, M).bytes;
}

grawa_status grawa_window_attention_backward(grawa_dtype dtype, const void* const* dout, const void* const* q, const void* const* k, const void* const* v,
                                             const void* const* out, const float* const* lse, void* const* dq, void* const* dk, void* const* dv,
                                             const int64_t* const* offsets, int64_t sequences, int64_t period, int64_t left, int64_t right, int64_t sinks,
                                             int64_t rows, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t q_stride, int64_t k_stride,
                                             int64_t v_stride, int64_t out_stride, int M, float scale, void* workspace, size_t workspace_bytes,
                                             grawa_stream_t stream)
{
    const AttentionShape s{dtype, offsets, sequences, period, left, right, sinks, rows, q_heads, kv_heads, head_dim, q_stride, k_stride, v_stride, out_stride, M, scale};
    if (!attention_shape_ok(s) || !dout || !q || !k || !v || !out || !lse || (dk == nullptr) != (dv == nullptr) || (!dq && !dk)) return GRAWA_ERR_INVALID_ARG;
    if (rows == 0) return GRAWA_OK;
    Buffers b;
    if (!add_heads(b, dout, s, q_heads, out_stride, false) || !add_heads(b, q, s, q_heads, q_stride, false) || !add_heads(b, k, s, kv_heads, k_stride, false) ||
        !add_heads(b, v, s, kv_heads, v_stride, false) || !add_heads(b, out, s, q_heads, out_stride, false) || !add_offsets(b, s) ||
        !b.add(reinterpret_cast<const void* const*>(lse), M, 1, q_heads * rows, q_heads * rows, 4, false)) return GRAWA_ERR_INVALID_ARG;
    if (dq && !add_heads(b, dq, s, q_heads, q_stride, true)) return GRAWA_ERR_INVALID_ARG;
    if (dk && (!add_heads(b, dk, s, kv_heads, k_stride, true) || !add_heads(b, dv, s, kv_heads, v_stride, true))) return GRAWA_ERR_INVALID_ARG;
    const AttentionScratch scratch = attention_scratch(rows, q_heads, kv_heads, head_dim, sinks, M);
    const size_t need = scratch.bytes;
    if (need) {
        if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return GRAWA_ERR_WORKSPACE;
        const void* ws = workspace;
        if (!b.add(&ws, 1, 1, static_cast<int64_t>(need), static_cast<int64_t>(need), 1, true)) return GRAWA_ERR_INVALID_ARG;
    }
    if (b.clash()) return GRAWA_ERR_INVALID_ARG;
    char* const base = static_cast<char*>(workspace);
    TileArgs t{};
    t.a = attention_args(s, q, k, v);
    copy_table(t.a.dout, dout, M);
    copy_table(t.a.out, out, M);
    copy_table(t.a.lse, lse, M);
    copy_table(t.a.to[0], dq, M);
    copy_table(t.a.to[1], dk, M);
    copy_table(t.a.to[2], dv, M);
    t.lse = reinterpret_cast<float*>(base);
    t.delta = reinterpret_cast<float*>(base + scratch.delta);
    t.longest = dtype == GRAWA_F16 ? reinterpret_cast<float*>(base + scratch.longest) : nullptr;
    t.pitch = scratch.pitch;
    t.chunks = static_cast<int>(scratch.chunks);
    t.partial = t.chunks > 0 && int64_t{t.a.left} + t.a.sinks < rows - kChunk ? reinterpret_cast<float*>(base + scratch.partial) : nullptr;
    StatsArgs stats{t.a, reinterpret_cast<float*>(base), reinterpret_cast<float*>(base + scratch.delta),
                    dtype == GRAWA_F16 ? reinterpret_cast<unsigned*>(base + scratch.longest) : nullptr, scratch.pitch};
    if (stats.longest) GRAWA_CUDA_TRY(cudaMemsetAsync(stats.longest, 0, static_cast<size_t>(M) * 2 * sizeof(float), stream));
    grawa_status st = dtype == GRAWA_BF16 ? attention_stats<__nv_bfloat16>(stats, M, stream) : attention_stats<__half>(stats, M, stream);
    for (int first = 0; first < M && st == GRAWA_OK; first += kAttentionWorkers) {
        st = set_workers(t, s, first, std::min(kAttentionWorkers, M - first));
        // dq needs nothing of dk and dv: its kernel runs beside the one in front, wherever that leaves SMs free.  (3 x 1001 tokens, 6 heads on 2 of
        // 80: 59 us one after the other.)  The chunks' sums come before the tiles that add them.
        const auto keys = [&](int far) {
            t.far = far;
            t.beside = 0;
            return dtype == GRAWA_BF16 ? launch_backward<__nv_bfloat16, true>(t, stream) : launch_backward<__half, true>(t, stream);
        };
        const auto queries = [&] {
            t.far = 0;
            t.beside = dk != nullptr;
            return dtype == GRAWA_BF16 ? launch_backward<__nv_bfloat16, false>(t, stream) : launch_backward<__half, false>(t, stream);
        };
        if (st == GRAWA_OK && dk) st = keys(t.partial ? 1 : 0);
        if (st == GRAWA_OK && dq) st = queries();
        if (st == GRAWA_OK && dk && t.partial) st = keys(0);
    }
    return st;
}

grawa_status grawa_selftest_window_attention_wait(grawa_stream_t stream)
{
    TileArgs t{};                                             // one row of one head; nothing is read or written
    t.a.rows = t.a.heads = t.a.kv_heads = t.a.group = 1;
    t.a.period = t.a.group_size = divisor(1);
    t.a.dim = 64;
    t.a.scale = 1.0f;
    t.workers = 1;
    return launch_tiles(attention_forward_kernel<__nv_bfloat16, 64, true>, t, 1, 1, kForwardThreads, kForwardSmem<64>, stream);
}

grawa_status grawa_window_attention_status(grawa_stream_t stream)
{
    return timeout_status(stream, g_attention_timeouts, "grawa_window_attention_status");
}

}  // extern "C"

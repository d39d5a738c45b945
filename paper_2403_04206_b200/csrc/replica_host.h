// Host-side checks of the replica operators: worker counts, pointers, and overlap of row-strided buffers.
#pragma once
#include "host_common.h"

#include <algorithm>
#include <cstdint>

namespace grawa {
namespace replica {

inline bool dtype_known(grawa_dtype d) { return d == GRAWA_F32 || d == GRAWA_BF16 || d == GRAWA_F16; }
inline int64_t type_bytes(grawa_dtype d) { return d == GRAWA_F32 ? 4 : 2; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// The buffers of a call.  add() takes one buffer a worker, `rows` rows of `cols` elements `stride` elements
// apart; clash() says whether an output shares a byte with any other buffer of the call.  A buffer of one row, or of rows
// of the same stride, that lies between the rows of another is no overlap.  (Rows of two strides that lie
// between each other are taken for one.)
class Buffers {
public:
    static constexpr int kMost = 10 * GRAWA_MAX_WORKERS;

    // false: a NULL entry, or one that is not aligned to its element size
    bool add(const void* const* table, int M, int64_t rows, int64_t cols, int64_t stride, int64_t elem, bool output)
    {
        for (int m = 0; m < M; ++m) {
            if (rows == 0 || cols == 0) continue;                   // nothing is read or written: any address will do
            if (table[m] == nullptr || !aligned(table[m], static_cast<size_t>(elem))) return false;
            const uintptr_t lo = reinterpret_cast<uintptr_t>(table[m]);
            const uintptr_t stride_bytes = static_cast<uintptr_t>(stride * elem), row_bytes = static_cast<uintptr_t>(cols * elem);
            item_[count_++] = Item{lo, lo + static_cast<uintptr_t>(rows - 1) * stride_bytes + row_bytes, rows > 1 ? stride_bytes : 0, row_bytes, output};
        }
        return true;
    }
    bool clash()
    {
        std::sort(item_, item_ + count_, [](const Item& a, const Item& b) { return a.lo < b.lo; });
        for (int i = 0; i < count_; ++i)
            for (int j = i + 1; j < count_ && item_[j].lo < item_[i].hi; ++j) {
                if (!item_[i].output && !item_[j].output) continue;
                const uintptr_t stride = item_[i].stride;
                if (stride && (item_[j].stride == stride || item_[j].stride == 0)) {
                    const uintptr_t d = (item_[j].lo - item_[i].lo) % stride;
                    if (d >= item_[i].row && d + item_[j].row <= stride) continue;
                }
                return true;
            }
        return false;
    }

private:
    struct Item { uintptr_t lo, hi, stride, row; bool output; };
    Item item_[kMost];
    int count_ = 0;
};

// One launch over grid (gx, gy, gz), in clusters of `cluster` CTAs along x.  `overlap`, with the "dependent_launch" option:
// its launch may overlap the end of the kernel in front of it on the stream, whose results it waits for by itself
// (stream_order).  Not for kernels whose CTAs share the work out evenly beforehand, several to an SM: those that come
// early crowd onto the SMs that are free first (8 x 18554 rows of 256 bf16: 33 us, 43 with it).
template <typename... KArgs, typename... Args>
grawa_status launch_clusters(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, cudaStream_t stream, bool overlap, unsigned cluster,
                             const Args&... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(block));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    if (overlap && dependent_launch()) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = cluster;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    cfg.attrs = attr;
    GRAWA_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    ++g_launches;
    return GRAWA_OK;
}
template <typename... KArgs, typename... Args>
grawa_status launch(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, cudaStream_t stream, const Args&... args)
{
    return launch_clusters(kernel, grid, block, smem, stream, true, 1u, args...);
}

}  // namespace replica
}  // namespace grawa

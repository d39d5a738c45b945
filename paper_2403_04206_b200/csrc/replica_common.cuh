// Shared by the replica operators (dropout, layer norm, gated feed-forward product): storage types,
// tables of one pointer per worker, small reductions.  Every operator reads its operands once, widens
// them exactly to fp32, computes there, and rounds each stored value once, to nearest even.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace grawa {
namespace replica {

constexpr int kWorkers = 64;           // GRAWA_MAX_WORKERS
constexpr int kSms = 148;              // a B200; the shapes of the persistent grids follow it

// The first thing in every kernel: waits until the kernel in front on the stream is done and its results are visible, then
// lets the kernel behind start launching, which waits in the same way.  So a kernel's launch and ramp-up overlap the end of
// the one in front, and nothing else does.  (Without the launch attribute both do nothing.)
__device__ __forceinline__ void stream_order()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

struct In { const void* p[kWorkers]; };
struct Out { void* p[kWorkers]; };

// Elements travel in words of 16 bytes: 8 of 16 bits, 4 of 32.
template <typename T> constexpr int kWordElems = 16 / static_cast<int>(sizeof(T));

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }

// Two 16-bit elements of a 32-bit word.
__device__ __forceinline__ void unpack_pair(unsigned w, float* o, __nv_bfloat16)
{
    o[0] = __uint_as_float(w << 16);                // a bfloat16 is the upper half of a float
    o[1] = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack_pair(unsigned w, float* o, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    o[0] = f.x; o[1] = f.y;
}
__device__ __forceinline__ unsigned pack_pair(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
}
__device__ __forceinline__ unsigned pack_pair(float lo, float hi, __half)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
}

template <typename T>
__device__ __forceinline__ void unpack(const uint4& w, float* o)
{
    if constexpr (sizeof(T) == 4) {
        o[0] = __uint_as_float(w.x); o[1] = __uint_as_float(w.y); o[2] = __uint_as_float(w.z); o[3] = __uint_as_float(w.w);
    } else {
        unpack_pair(w.x, o, T{}); unpack_pair(w.y, o + 2, T{}); unpack_pair(w.z, o + 4, T{}); unpack_pair(w.w, o + 6, T{});
    }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float* o)
{
    if constexpr (sizeof(T) == 4)
        return make_uint4(__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3]));
    else
        return make_uint4(pack_pair(o[0], o[1], T{}), pack_pair(o[2], o[3], T{}), pack_pair(o[4], o[5], T{}), pack_pair(o[6], o[7], T{}));
}

// o[e] = element e + c, and acc[e % 2] += element e.  For 16-bit elements these are single instructions that
// take the 16-bit source as it is (widened exactly, one rounding), so nothing is unpacked first.
__device__ __forceinline__ void pair_add(unsigned w, float c, float* o, __nv_bfloat16)
{
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.bf16 %0, l, %3;\n\tadd.rn.f32.bf16 %1, h, %3;\n\t}"
        : "=f"(o[0]), "=f"(o[1]) : "r"(w), "f"(c));
}
__device__ __forceinline__ void pair_add(unsigned w, float c, float* o, __half)
{
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.f16 %0, l, %3;\n\tadd.rn.f32.f16 %1, h, %3;\n\t}"
        : "=f"(o[0]), "=f"(o[1]) : "r"(w), "f"(c));
}
__device__ __forceinline__ void pair_sum(unsigned w, float* acc, __nv_bfloat16)
{
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.bf16 %0, l, %0;\n\tadd.rn.f32.bf16 %1, h, %1;\n\t}"
        : "+f"(acc[0]), "+f"(acc[1]) : "r"(w));
}
__device__ __forceinline__ void pair_sum(unsigned w, float* acc, __half)
{
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.f16 %0, l, %0;\n\tadd.rn.f32.f16 %1, h, %1;\n\t}"
        : "+f"(acc[0]), "+f"(acc[1]) : "r"(w));
}
template <typename T>
__device__ __forceinline__ void shifted(const uint4& w, float c, float* o)
{
    if constexpr (sizeof(T) == 2) {
        pair_add(w.x, c, o, T{}); pair_add(w.y, c, o + 2, T{}); pair_add(w.z, c, o + 4, T{}); pair_add(w.w, c, o + 6, T{});
    } else {
        unpack<T>(w, o);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += c;
    }
}
template <typename T>
__device__ __forceinline__ void add_elements(const uint4& w, float (&acc)[2])
{
    if constexpr (sizeof(T) == 2) {
        pair_sum(w.x, acc, T{}); pair_sum(w.y, acc, T{}); pair_sum(w.z, acc, T{}); pair_sum(w.w, acc, T{});
    } else {
        float o[4];
        unpack<T>(w, o);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e % 2] += o[e];
    }
}

// Words at addresses of any alignment, in halves (16 bits): a word of 8 halves lies in one or two aligned words.
// The 8 halves from half `skip` (0..7) on of the 16 halves (lo, hi).
__device__ __forceinline__ uint4 shift_halves(const uint4& lo, const uint4& hi, unsigned skip)
{
    const unsigned w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    unsigned t[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) {                             // by whole 32-bit words, two steps of a binary shift
        const unsigned a = skip & 4 ? w[i + 2] : w[i], b = skip & 4 ? w[i + 3 < 8 ? i + 3 : 7] : w[i + 1];
        t[i] = skip & 2 ? b : a;
    }
    const unsigned bits = (skip & 1) * 16;
    return make_uint4(__funnelshift_r(t[0], t[1], bits), __funnelshift_r(t[1], t[2], bits), __funnelshift_r(t[2], t[3], bits),
                      __funnelshift_r(t[3], t[4], bits));
}
// The first `count` (1 to 8) halves of v, zeros behind them.
__device__ __forceinline__ uint4 keep_halves(uint4 v, int count)
{
    if (count < 8) {
        unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (2 * i + 1 >= count) w[i] = 2 * i >= count ? 0u : w[i] & 0xffffu;
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}
__device__ __forceinline__ unsigned skip_of(const void* p) { return static_cast<unsigned>(reinterpret_cast<uintptr_t>(p) & 15) / 2; }

// `count` (1 to 8) halves from p on, zeros behind them, from the aligned words that hold them (each of which holds
// at least one of them).
__device__ __forceinline__ uint4 load_halves(const unsigned short* p, int count)
{
    const unsigned skip = skip_of(p);
    const uint4* word = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) & ~static_cast<uintptr_t>(15));
    const uint4 lo = word[0];
    const uint4 hi = static_cast<int>(skip) + count > 8 ? word[1] : make_uint4(0, 0, 0, 0);
    return keep_halves(shift_halves(lo, hi, skip), count);
}

// Stores of a row of `halves` halves whose words stand in order in neighbouring lanes: lane l of a segment of `lanes`
// neighbouring lanes holds word `at` = (the segment's first) + l, v; lanes behind the row's last word hold none.  All
// 32 lanes of the warp call it.  Where the row does not start on a 16-byte boundary, a lane stores the aligned word
// that its halves share with the lane in front; what is left at the ends of a segment goes half by half.
// (Rows of one warp may start at different offsets, so every lane takes part in the exchange whether it needs it or not.)
__device__ __forceinline__ void store_halves(unsigned short* row, int at, int lane, int lanes, int halves, const uint4& v, unsigned skip)
{
    const int count = min(8, halves - 8 * at);
    const uint4 before = make_uint4(__shfl_up_sync(0xffffffffu, v.x, 1), __shfl_up_sync(0xffffffffu, v.y, 1),
                                    __shfl_up_sync(0xffffffffu, v.z, 1), __shfl_up_sync(0xffffffffu, v.w, 1));
    if (skip == 0) {
        if (count == 8) {
            *reinterpret_cast<uint4*>(row + 8 * at) = v;
        } else if (count > 0) {
            const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < count) row[8 * at + e] = static_cast<unsigned short>(w[e / 2] >> (e % 2 * 16));
        }
        return;
    }
    if (count <= 0) return;
    const int own = 8 - static_cast<int>(skip);               // halves of v in the aligned word that v begins in
    const bool joined = lane > 0 && count >= own;
    const bool passed = lane + 1 < lanes && halves - 8 * (at + 1) >= own;          // the rest of v goes with the next lane's word
    if (joined) *reinterpret_cast<uint4*>(row + 8 * at - static_cast<int>(skip)) = shift_halves(before, v, own);
    if (!joined || !passed) {
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
        const int from = joined ? own : 0, to = passed ? min(count, own) : count;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= from && e < to) row[8 * at + e] = static_cast<unsigned short>(w[e / 2] >> (e % 2 * 16));
    }
}

// 16 bytes from global to shared memory behind this thread's back; a thread waits for its own copies.
__device__ __forceinline__ void copy_async16(void* shared, const void* global)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<unsigned>(__cvta_generic_to_shared(shared))), "l"(global) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING> __device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

// Sum over groups of LPR neighbouring lanes (a power of two up to 32); every lane gets it.  All 32 lanes take part.
template <int LPR>
__device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int d = LPR / 2; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

}  // namespace replica
}  // namespace grawa

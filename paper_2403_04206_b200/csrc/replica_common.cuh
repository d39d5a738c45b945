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

struct In { const void* p[kWorkers]; };
struct Out { void* p[kWorkers]; };

// The word that carries VE elements of T: 16, 4 or 2 bytes.
template <int BYTES> struct Word;
template <> struct Word<16> { using type = uint4; };
template <> struct Word<4> { using type = unsigned; };
template <> struct Word<2> { using type = unsigned short; };
template <typename T, int VE> using WordOf = typename Word<VE * static_cast<int>(sizeof(T))>::type;

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

template <typename T, int VE>
__device__ __forceinline__ void unpack(const WordOf<T, VE>& w, float* o)
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (VE == 4) {
            o[0] = __uint_as_float(w.x); o[1] = __uint_as_float(w.y); o[2] = __uint_as_float(w.z); o[3] = __uint_as_float(w.w);
        } else {
            o[0] = __uint_as_float(w);
        }
    } else if constexpr (VE == 8) {
        unpack_pair(w.x, o, T{}); unpack_pair(w.y, o + 2, T{}); unpack_pair(w.z, o + 4, T{}); unpack_pair(w.w, o + 6, T{});
    } else if constexpr (VE == 2) {
        unpack_pair(w, o, T{});
    } else {
        o[0] = widen(*reinterpret_cast<const T*>(&w));
    }
}

template <typename T, int VE>
__device__ __forceinline__ WordOf<T, VE> pack(const float* o)
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (VE == 4)
            return make_uint4(__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3]));
        else
            return __float_as_uint(o[0]);
    } else if constexpr (VE == 8) {
        return make_uint4(pack_pair(o[0], o[1], T{}), pack_pair(o[2], o[3], T{}), pack_pair(o[4], o[5], T{}), pack_pair(o[6], o[7], T{}));
    } else if constexpr (VE == 2) {
        return pack_pair(o[0], o[1], T{});
    } else {
        const T v = narrow<T>(o[0]);
        return *reinterpret_cast<const unsigned short*>(&v);
    }
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
template <typename T, int VE>
__device__ __forceinline__ void shifted(const WordOf<T, VE>& w, float c, float* o)
{
    if constexpr (sizeof(T) == 2 && VE == 8) {
        pair_add(w.x, c, o, T{}); pair_add(w.y, c, o + 2, T{}); pair_add(w.z, c, o + 4, T{}); pair_add(w.w, c, o + 6, T{});
    } else if constexpr (sizeof(T) == 2 && VE == 2) {
        pair_add(w, c, o, T{});
    } else {
        unpack<T, VE>(w, o);
#pragma unroll
        for (int e = 0; e < VE; ++e) o[e] += c;
    }
}
template <typename T, int VE>
__device__ __forceinline__ void add_elements(const WordOf<T, VE>& w, float (&acc)[2])
{
    if constexpr (sizeof(T) == 2 && VE == 8) {
        pair_sum(w.x, acc, T{}); pair_sum(w.y, acc, T{}); pair_sum(w.z, acc, T{}); pair_sum(w.w, acc, T{});
    } else if constexpr (sizeof(T) == 2 && VE == 2) {
        pair_sum(w, acc, T{});
    } else {
        float o[VE];
        unpack<T, VE>(w, o);
#pragma unroll
        for (int e = 0; e < VE; ++e) acc[e % 2] += o[e];
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

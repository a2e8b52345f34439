// ccq_ops.cuh -- what the operators of ccq_ops.h share: argument errors, and loads and stores of
// a few elements as one access of 2 to 16 bytes, converted to and from fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include <atomic>
#include <type_traits>

#include "../../include/ccq_ops.h"
#include "ccq_internal.h"
#include "sm100_ptx.cuh"

namespace ccq {

inline ccq_status op_fail(ccq_status st, const char *fmt, ...) {
    char msg[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    return static_cast<ccq_status>(record_error_code(st, msg));
}

inline ccq_status op_cuda(cudaError_t e, const char *what) {
    return e == cudaSuccess ? CCQ_OK : op_fail(CCQ_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

inline bool valid_dtype(int d) { return d == CCQ_BF16 || d == CCQ_FP32; }
inline int dtype_bytes(ccq_dtype d) { return d == CCQ_BF16 ? 2 : 4; }

// A required device pointer, aligned to its element type (and to `least`).
inline ccq_status op_pointer(const char *name, const void *p, uintptr_t least) {
    if (!p) return op_fail(CCQ_ERR_INVALID_ARG, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) % least)
        return op_fail(CCQ_ERR_INVALID_ARG, "%s is not aligned to %d bytes", name, static_cast<int>(least));
    return CCQ_OK;
}

// The device status word that a call's kernels write.
inline ccq_status op_status_word(int **word) {
    *word = device_status_word();
    return *word ? CCQ_OK : op_fail(CCQ_ERR_CUDA, "cannot resolve the device status word");
}

// The largest of 16, 8, 4, 2 bytes that divides a base address or row stride, `bytes`.
inline int access_bytes(uintptr_t bytes, int most = 16) {
    while (most > 2 && bytes % most) most >>= 1;
    return most;
}

// A 2-D operand's common access width: its base and, with more than one row, its row stride.
inline int row_access(const void *p, int64_t stride, int elem, int64_t rows, int most) {
    most = access_bytes(reinterpret_cast<uintptr_t>(p), most);
    return rows > 1 ? access_bytes(static_cast<uintptr_t>(stride) * elem, most) : most;
}

inline int sm_count_now() {
    static std::atomic<int> counts[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 152;
    int n = counts[dev].load(std::memory_order_relaxed);
    if (!n) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = 152;
        counts[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

// Opts a kernel into `bytes` of dynamic shared memory, once for a kernel and device.
template <auto Kernel> cudaError_t allow_shared(int bytes) {
    static std::atomic<int> allowed[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64 && allowed[dev].load(std::memory_order_relaxed) >= bytes) return cudaSuccess;
    e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev >= 0 && dev < 64) allowed[dev].store(bytes, std::memory_order_relaxed);
    return e;
}

// ---------------------------------------------------------------- elements and accesses

template <int B> struct RawOf;
template <> struct RawOf<16> { using type = uint4; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<2> { using type = uint16_t; };

// N elements of T as one access.  A single bf16 is held in a 32-bit register: with 16-bit ones the compiler packs two
// loads' results into one register, and each load is then waited for as it is made.
template <typename T, int N> struct Pack {
    using Mem = typename RawOf<N * static_cast<int>(sizeof(T))>::type;
    using Raw = typename std::conditional<sizeof(Mem) == 2, uint32_t, Mem>::type;
    Raw raw;
};

// Read once, not kept in L1 (the data streams through).
template <typename T, int N> __device__ __forceinline__ Pack<T, N> load_stream(const T *p) {
    Pack<T, N> r;
    if constexpr (N * sizeof(T) == 2)
        asm volatile("ld.global.cs.u16 %0, [%1];" : "=r"(r.raw) : "l"(p));
    else
        r.raw = __ldcs(reinterpret_cast<const typename Pack<T, N>::Mem *>(p));
    return r;
}
template <typename T, int N> __device__ __forceinline__ Pack<T, N> load_plain(const T *p) {
    Pack<T, N> r;
    if constexpr (N * sizeof(T) == 2)
        asm volatile("ld.global.u16 %0, [%1];" : "=r"(r.raw) : "l"(p));
    else
        r.raw = *reinterpret_cast<const typename Pack<T, N>::Mem *>(p);
    return r;
}
template <typename T, int N> __device__ __forceinline__ void store_stream(T *p, const Pack<T, N> &v) {
    __stcs(reinterpret_cast<typename Pack<T, N>::Mem *>(p), static_cast<typename Pack<T, N>::Mem>(v.raw));
}

template <int W> __device__ __forceinline__ uint32_t word_of(const uint4 &r) {
    return W == 0 ? r.x : W == 1 ? r.y : W == 2 ? r.z : r.w;
}

template <int W> __device__ __forceinline__ uint32_t word_of(const uint2 &r) { return W == 0 ? r.x : r.y; }

template <int W> __device__ __forceinline__ uint32_t word_of(uint32_t r) { return r; }
template <int W> __device__ __forceinline__ void set_word(uint4 &r, uint32_t w) {
    (W == 0 ? r.x : W == 1 ? r.y : W == 2 ? r.z : r.w) = w;
}
template <int W> __device__ __forceinline__ void set_word(uint2 &r, uint32_t w) { (W == 0 ? r.x : r.y) = w; }
template <int W> __device__ __forceinline__ void set_word(uint32_t &r, uint32_t w) { r = w; }

template <typename T> struct IsBf16 { static constexpr bool value = false; };
template <> struct IsBf16<__nv_bfloat16> { static constexpr bool value = true; };

template <int W = 0, typename T, int N> __device__ __forceinline__ void unpack(const Pack<T, N> &p, float (&f)[N]) {
    const uint32_t w = word_of<W>(p.raw);
    if constexpr (IsBf16<T>::value) {
        f[2 * W] = __uint_as_float(w << 16);
        if constexpr (2 * W + 1 < N) f[2 * W + 1] = __uint_as_float(w & 0xffff0000u);
        if constexpr (2 * W + 2 < N) unpack<W + 1>(p, f);
    } else {
        f[W] = __uint_as_float(w);
        if constexpr (W + 1 < N) unpack<W + 1>(p, f);
    }
}

template <int W = 0, typename T, int N> __device__ __forceinline__ void pack(const float (&f)[N], Pack<T, N> &p) {
    if constexpr (IsBf16<T>::value && N == 1) {
        p.raw = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
    } else if constexpr (IsBf16<T>::value) {
        set_word<W>(p.raw, pack_bf16(f[2 * W], f[2 * W + 1]));
        if constexpr (2 * W + 2 < N) pack<W + 1>(f, p);
    } else {
        set_word<W>(p.raw, __float_as_uint(f[W]));
        if constexpr (W + 1 < N) pack<W + 1>(f, p);
    }
}

// A thread's own asynchronous copy of one access to shared memory (4, 8 or 16 bytes), not kept in L1 where it is 16.
template <int B> __device__ __forceinline__ void copy_async(void *dst, const void *src) {
    if constexpr (B == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(dst)), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_addr(dst)), "l"(src), "n"(B) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

// 1 / x within a unit in the last place; subnormal numbers, and results, are 0.
__device__ __forceinline__ float fast_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
    return __float2bfloat16_rn(x);
}

// An index of 4 or 8 bytes.
__device__ __forceinline__ int64_t load_index(const void *p, int bytes, int64_t i) {
    return bytes == 8 ? static_cast<const int64_t *>(p)[i] : static_cast<const int32_t *>(p)[i];
}

// Wait until the shared-memory sources of all but the N most recently committed bulk-store groups have been read.
template <int N> __device__ __forceinline__ void tma_store_wait_read_but() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}

// Status code of an index outside its range (CCQ_ERR_INDEX), for the device status word.  It concerns a row, the other codes
// say that outputs are not valid, so it is left in a clear word alone (and the others replace it).
constexpr int kStatusIndex = 6;
__device__ __forceinline__ void note_index(int *status) { atomicCAS(status, 0, kStatusIndex); }

}  // namespace ccq

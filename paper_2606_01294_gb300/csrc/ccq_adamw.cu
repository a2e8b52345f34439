// ccq_adamw.cu -- one AdamW update of many tensors in one launch, states in 32 or 8 bits (ccq_ops.h).
//
//   g = c grad, m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
//   p = (1 - lr wd) p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// Every element is read and written once: 28 bytes an element with everything in fp32, 16 with bf16 weights and
// gradients, an fp32 master and 8-bit states.  The tensors' addresses are the launch's own arguments (constant
// memory), and a CTA finds its tensor among them by the tensors' first chunks.  A warp updates kBlock
// consecutive elements, 8 a lane, which is also what shares a scale in the 8-bit state: the block's largest moment is
// a warp's maximum, and the state never leaves registers between its decoding and its rounding.
// The 8-bit state's arithmetic up to the rounding is done without fused multiply-adds, so that its e4m3
// codes are those of the formula's fp32 operations taken one by one.
// Measured: 84 M elements in fp32 340 us (6.9 TB/s, the copy rate; HBM bounds it); 253 M with masters and 8-bit states 720 us
// (5.6 TB/s, 83 %; about 69 instructions an element, half of them integer, bound it beside HBM).
// (Tried and taken back: the next block's operands by asynchronous copies while one is computed, 748 us.)
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <float.h>
#include <math.h>

#include <algorithm>

#include "ccq_ops.cuh"

namespace ccq {
namespace {

constexpr int kBlock = CCQ_ADAMW_BLOCK;
static_assert(kBlock == 32 * 8, "8 elements a lane");
constexpr int kAdamThreads = 256;
constexpr int kChunk = kBlock * (kAdamThreads / 32);  // elements of a CTA
constexpr int kMaxTensors = 482;                      // of a launch: its arguments hold 32764 bytes

struct AdamTensor {
    void *param;
    const void *grad;
    void *m, *v;
    float *scale;
    float *master;
    int64_t n;
    uint32_t first;  // chunk of the launch
    uint32_t vec;    // every address allows 8 elements at a time
};

struct AdamConst {
    float beta1, rest1, beta2, rest2;  // rest = 1 - beta
    float keep;                        // 1 - lr weight_decay
    float rate;                        // lr / (1 - beta1^step)
    float root;                        // 1 / sqrt(1 - beta2^step)
    float eps;
    uint32_t turn;                     // step 0x9E3779B1
    const float *grad_scale;
};

template <int CAP> struct AdamArgs {
    AdamConst c;
    int count;
    AdamTensor t[CAP];
};
static_assert(sizeof(AdamArgs<kMaxTensors>) <= 32764, "a launch's arguments");

// The exponent field of the smallest power of two 2^e >= 2^-100 with top <= 448 * 2^e (448 = 1.75 * 2^8).
__device__ __forceinline__ uint32_t scale_exponent(float top) {
    const int e = static_cast<int>((__float_as_uint(top) + 0x1FFFFFu) >> 23) - 8;
    return static_cast<uint32_t>(max(e, 27));
}

// y = |x| / scale as a number whose upper bits are its e4m3 code: below 2^-6 the neighbours are 2^-9 apart, and
// 2^-7 + y / 2 (cut, not rounded) has them in its upper three mantissa bits.  Not a number, and infinity: the code 127.
__device__ __forceinline__ uint32_t code_bits(float y) {
    return __float_as_uint(y < 0.015625f ? __fmaf_rz(y, 0.5f, 0.0078125f) : fminf(y, 480.f));
}
// The code, rounded up where the fraction between neighbours reaches 2^20 - turn.
__device__ __forceinline__ uint32_t encode(float y, uint32_t turn) { return ((code_bits(y) + turn) >> 20) - (120u << 3); }

// Within two units in the last place, as fast_rcp is: of an update's step, which is a small part of the parameter, in both
// forms of the state (the stored 8-bit roots are corrected below; the 32-bit moments take neither).
__device__ __forceinline__ float approx_sqrt(float x) {
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void decode4(uint32_t codes, float *f) {
    const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes & 0xffffu), __NV_E4M3);
    const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes >> 16), __NV_E4M3);
    const float2 x = __half22float2(__half2(a)), y = __half22float2(__half2(b));
    f[0] = x.x; f[1] = x.y; f[2] = y.x; f[3] = y.y;
}

// Eight consecutive elements in the wide form; in the narrow one (unaligned tensors, a tensor's last block) lane l
// holds elements l, l + 32, ... of the block, one access each.
template <typename T> __device__ __forceinline__ void load8(const T *p, float (&f)[8]) {
    if constexpr (sizeof(T) == 2) {
        unpack(load_stream<T, 8>(p), f);
    } else {
        float h[4];
        const Pack<T, 4> a = load_stream<T, 4>(p), b = load_stream<T, 4>(p + 4);
        unpack(a, h);
        for (int i = 0; i < 4; ++i) f[i] = h[i];
        unpack(b, h);
        for (int i = 0; i < 4; ++i) f[4 + i] = h[i];
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&f)[8]) {
    if constexpr (sizeof(T) == 2) {
        Pack<T, 8> a;
        pack(f, a);
        store_stream<T, 8>(p, a);
    } else {
        Pack<T, 4> a;
        const float lo[4] = {f[0], f[1], f[2], f[3]}, hi[4] = {f[4], f[5], f[6], f[7]};
        pack(lo, a);
        store_stream<T, 4>(p, a);
        pack(hi, a);
        store_stream<T, 4>(p + 4, a);
    }
}

template <typename P, typename G, int BITS, int MASTER, int CAP>
__global__ void __launch_bounds__(kAdamThreads, 4) adamw_kernel(const __grid_constant__ AdamArgs<CAP> a) {
    // the last tensor whose first chunk is not past this one
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.t[mid].first <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const AdamTensor &t = a.t[lo];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t start = static_cast<int64_t>(blockIdx.x - t.first) * kChunk + warp * kBlock;
    if (start >= t.n) return;
    const int left = t.n - start < kBlock ? static_cast<int>(t.n - start) : kBlock;
    const bool wide = t.vec && left == kBlock;
    const float clip = a.c.grad_scale ? *a.c.grad_scale : 1.f;
    P *param = static_cast<P *>(t.param) + start;
    const G *grad = static_cast<const G *>(t.grad) + start;
    float *master = MASTER ? t.master + start : nullptr;
    float g[8], m[8], v[8], p[8];
    float sm = 1.f, sv = 1.f;
    float *scale = nullptr;
    if constexpr (BITS == 8) {
        scale = t.scale + start / kBlock * 2;
        sm = scale[0];
        sv = scale[1];
    }
    if (wide) {
        load8(grad + lane * 8, g);
        if constexpr (MASTER) load8(master + lane * 8, p);
        else load8(param + lane * 8, p);
        if constexpr (BITS == 8) {
            const Pack<float, 2> cm = load_stream<float, 2>(reinterpret_cast<const float *>(static_cast<uint8_t *>(t.m) + start + lane * 8));
            const Pack<float, 2> cv = load_stream<float, 2>(reinterpret_cast<const float *>(static_cast<uint8_t *>(t.v) + start + lane * 8));
            decode4(cm.raw.x, m);
            decode4(cm.raw.y, m + 4);
            decode4(cv.raw.x, v);
            decode4(cv.raw.y, v + 4);
        } else {
            load8(static_cast<const float *>(t.m) + start + lane * 8, m);
            load8(static_cast<const float *>(t.v) + start + lane * 8, v);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = e * 32 + lane;
            g[e] = p[e] = m[e] = v[e] = 0.f;
            if (i >= left) continue;
            g[e] = to_f32(grad[i]);
            p[e] = MASTER ? master[i] : to_f32(param[i]);
            if constexpr (BITS == 8) {
                float f[4];
                decode4(static_cast<const uint8_t *>(t.m)[start + i], f);
                m[e] = f[0];
                decode4(static_cast<const uint8_t *>(t.v)[start + i], f);
                v[e] = f[0];
            } else {
                m[e] = static_cast<const float *>(t.m)[start + i];
                v[e] = static_cast<const float *>(t.v)[start + i];
            }
        }
    }
    // two elements an operation; every product and sum of the moments is rounded by itself
    float top_m = 0.f, top_v = 0.f, root[8];
    auto two = [](float x) { return f2_make(x, x); };
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const uint64_t ge = f2_mul(f2_make(g[e], g[e + 1]), two(clip));
        uint64_t me = f2_make(m[e], m[e + 1]), ve = f2_make(v[e], v[e + 1]);
        if constexpr (BITS == 8) {
            me = f2_mul(me, two(sm));
            ve = f2_mul(ve, two(sv));
            ve = f2_mul(ve, ve);
        }
        // (the sums one by one: a packed sum of packed products is contracted, whatever their rounding says)
        const float2 ma = f2_split(f2_mul(me, two(a.c.beta1))), mb = f2_split(f2_mul(ge, two(a.c.rest1)));
        const float2 va = f2_split(f2_mul(ve, two(a.c.beta2))), vb = f2_split(f2_mul(f2_mul(ge, ge), two(a.c.rest2)));
        const float2 m2 = make_float2(__fadd_rn(ma.x, mb.x), __fadd_rn(ma.y, mb.y));
        const float2 v2 = make_float2(__fadd_rn(va.x, vb.x), __fadd_rn(va.y, vb.y));
        me = f2_make(m2.x, m2.y);
        const float r0 = approx_sqrt(v2.x), r1 = approx_sqrt(v2.y);
        const float2 d = f2_split(f2_fma(f2_make(r0, r1), two(a.c.root), two(a.c.eps)));
        const uint64_t step = f2_mul(f2_mul(me, two(-a.c.rate)), f2_make(fast_rcp(d.x), fast_rcp(d.y)));
        const float2 q = f2_split(f2_fma(f2_make(p[e], p[e + 1]), two(a.c.keep), step));
        p[e] = q.x;
        p[e + 1] = q.y;
        m[e] = m2.x;
        m[e + 1] = m2.y;
        v[e] = v2.x;
        v[e + 1] = v2.y;
        if constexpr (BITS == 8) {
            root[e] = r0;
            root[e + 1] = r1;
            // (the larger number of a number and a NaN)
            top_m = fmaxf(fmaxf(top_m, fabsf(m2.x)), fabsf(m2.y));
            top_v = fmaxf(fmaxf(top_v, v2.x), v2.y);
        }
    }
    uint32_t code_m[8], code_v[8];
    if constexpr (BITS == 8) {
        // non-negative floats order as their bits do
        top_m = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(top_m)));
        top_v = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(top_v)));
        if (!(top_m < INFINITY) || !(top_v < INFINITY)) {  // an infinite moment is its own element's alone
            top_m = top_v = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (fabsf(m[e]) < INFINITY) top_m = fmaxf(top_m, fabsf(m[e]));
                if (v[e] < INFINITY) top_v = fmaxf(top_v, v[e]);
            }
            top_m = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(top_m)));
            top_v = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(top_v)));
        }
        const uint32_t em = scale_exponent(top_m), ev = scale_exponent(__fsqrt_rn(top_v));
        const float inv_m = __uint_as_float((254 - em) << 23), inv_v = __uint_as_float((254 - ev) << 23);
        if (lane == 0) *reinterpret_cast<float2 *>(scale) = make_float2(__uint_as_float(em << 23), __uint_as_float(ev << 23));
        const uint32_t hop = wide ? 1u : 32u;
        const uint32_t word0 = (static_cast<uint32_t>(start) + (wide ? lane * 8 : lane)) * 0x6A09E667u + a.c.turn;
        uint32_t word = word0, near = ~0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t turn = word >> 12;
            word += hop * 0x6A09E667u;
            code_m[e] = encode(fabsf(m[e]) * inv_m, turn ^ 0xFFFFFu) | ((__float_as_uint(m[e]) >> 24) & 128u);
            const uint32_t at = code_bits(root[e] * inv_v) + turn;
            code_v[e] = max((at >> 20) - (120u << 3), min(__float_as_uint(v[e]), 1u));
            near = min(near, (at + 8u) & 0xFFFFFu);
        }
        // The approximate root is within two units in the last place; where that could pass a threshold (a few elements of a
        // million), the rounded root decides.
        if (near < 16u) {
            word = word0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                code_v[e] = max(encode(__fsqrt_rn(v[e]) * inv_v, word >> 12), min(__float_as_uint(v[e]), 1u));
                word += hop * 0x6A09E667u;
            }
        }
    }
    if (wide) {
        store8(param + lane * 8, p);
        if constexpr (MASTER) store8(master + lane * 8, p);
        if constexpr (BITS == 8) {
            auto word = [](const uint32_t *c) { return c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24; };
            __stcs(reinterpret_cast<uint2 *>(static_cast<uint8_t *>(t.m) + start + lane * 8), make_uint2(word(code_m), word(code_m + 4)));
            __stcs(reinterpret_cast<uint2 *>(static_cast<uint8_t *>(t.v) + start + lane * 8), make_uint2(word(code_v), word(code_v + 4)));
        } else {
            store8(static_cast<float *>(t.m) + start + lane * 8, m);
            store8(static_cast<float *>(t.v) + start + lane * 8, v);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = e * 32 + lane;
        if (i >= left) continue;
        param[i] = from_f32<P>(p[e]);
        if constexpr (MASTER) master[i] = p[e];
        if constexpr (BITS == 8) {
            static_cast<uint8_t *>(t.m)[start + i] = static_cast<uint8_t>(code_m[e]);
            static_cast<uint8_t *>(t.v)[start + i] = static_cast<uint8_t>(code_v[e]);
        } else {
            static_cast<float *>(t.m)[start + i] = m[e];
            static_cast<float *>(t.v)[start + i] = v[e];
        }
    }
}

template <typename P, typename G, int BITS, int MASTER>
cudaError_t launch_adamw(const AdamArgs<kMaxTensors> &a, unsigned chunks, cudaStream_t s) {
    // a short list is passed as a short argument block
    constexpr int kFew = 48;
    if (a.count <= kFew) {
        AdamArgs<kFew> few;
        few.c = a.c;
        few.count = a.count;
        std::copy(a.t, a.t + a.count, few.t);
        adamw_kernel<P, G, BITS, MASTER, kFew><<<chunks, kAdamThreads, 0, s>>>(few);
    } else {
        adamw_kernel<P, G, BITS, MASTER, kMaxTensors><<<chunks, kAdamThreads, 0, s>>>(a);
    }
    return cudaGetLastError();
}

ccq_status check_tensor(const ccq_adamw_tensor &t, int i, int pe, int ge, int bits, bool master) {
    struct { const char *name; const void *p; int least; } need[] = {
        {"param", t.param, pe}, {"grad", t.grad, ge}, {"m", t.m, bits / 8}, {"v", t.v, bits / 8},
        {"scale", t.scale, bits == 8 ? 8 : 0}, {"master", t.master, master ? 4 : 0}};
    for (const auto &q : need) {
        if (!q.least) {
            if (q.p) return op_fail(CCQ_ERR_INVALID_ARG, "tensor %d: %s is given but not used", i, q.name);
        } else if (!q.p) {
            return op_fail(CCQ_ERR_INVALID_ARG, "tensor %d: %s is NULL", i, q.name);
        } else if (reinterpret_cast<uintptr_t>(q.p) % q.least) {
            return op_fail(CCQ_ERR_INVALID_ARG, "tensor %d: %s is not aligned to %d bytes", i, q.name, q.least);
        }
    }
    return CCQ_OK;
}

}  // namespace
}  // namespace ccq

using namespace ccq;

extern "C" ccq_status ccq_adamw_step(const ccq_adamw_tensor *tensors, int count, ccq_dtype param_dtype, ccq_dtype grad_dtype,
                                     int state_bits, const ccq_adamw_params *p, const float *grad_scale, void *stream) {
    if (count < 0) return op_fail(CCQ_ERR_INVALID_ARG, "count=%d", count);
    if (!p) return op_fail(CCQ_ERR_INVALID_ARG, "params is NULL");
    if (count && !tensors) return op_fail(CCQ_ERR_INVALID_ARG, "tensors is NULL");
    if (!valid_dtype(param_dtype) || !valid_dtype(grad_dtype))
        return op_fail(CCQ_ERR_INVALID_ARG, "unknown dtype %d or grad dtype %d", param_dtype, grad_dtype);
    if (state_bits != 8 && state_bits != 32) return op_fail(CCQ_ERR_INVALID_ARG, "state_bits=%d: 8 or 32", state_bits);
    if (p->step < 1) return op_fail(CCQ_ERR_INVALID_ARG, "step=%lld must be >= 1", static_cast<long long>(p->step));
    if (!(p->beta1 >= 0 && p->beta1 < 1) || !(p->beta2 >= 0 && p->beta2 < 1))
        return op_fail(CCQ_ERR_INVALID_ARG, "betas must be in [0, 1)");
    if (!(p->eps >= 0)) return op_fail(CCQ_ERR_INVALID_ARG, "eps must be >= 0");
    // (a smaller one is 0 to the approximate reciprocal, and 0 / eps not a number)
    if (p->eps > 0 && p->eps < FLT_MIN)
        return op_fail(CCQ_ERR_INVALID_ARG, "eps=%g: 0, or at least fp32's smallest normal number %g", p->eps, static_cast<double>(FLT_MIN));
    if (grad_scale && reinterpret_cast<uintptr_t>(grad_scale) % 4)
        return op_fail(CCQ_ERR_INVALID_ARG, "grad_scale is not aligned to 4 bytes");
    const int pe = dtype_bytes(param_dtype), ge = dtype_bytes(grad_dtype);
    bool master = false;
    for (int i = 0; i < count; ++i)
        if (tensors[i].n > 0) {
            master = tensors[i].master != nullptr;
            break;
        }
    if (master && param_dtype != CCQ_BF16)
        return op_fail(CCQ_ERR_INVALID_ARG, "a master copy needs bf16 parameters");
    for (int i = 0; i < count; ++i) {
        if (tensors[i].n < 0) return op_fail(CCQ_ERR_INVALID_ARG, "tensor %d: n=%lld", i, static_cast<long long>(tensors[i].n));
        if (tensors[i].n > (static_cast<int64_t>(1) << 40)) return op_fail(CCQ_ERR_UNSUPPORTED, "tensor %d: n above 2^40", i);
        if (tensors[i].n == 0) continue;
        ccq_status st = check_tensor(tensors[i], i, pe, ge, state_bits, master);
        if (st != CCQ_OK) return st;
    }
    static thread_local AdamArgs<kMaxTensors> a;
    const double b1 = p->beta1, b2 = p->beta2, c1 = 1 - pow(b1, static_cast<double>(p->step)),
                 c2 = 1 - pow(b2, static_cast<double>(p->step));
    a.c.beta1 = static_cast<float>(b1);
    a.c.rest1 = static_cast<float>(1 - b1);
    a.c.beta2 = static_cast<float>(b2);
    a.c.rest2 = static_cast<float>(1 - b2);
    a.c.keep = static_cast<float>(1 - p->lr * p->weight_decay);
    a.c.rate = static_cast<float>(p->lr / c1);
    a.c.root = static_cast<float>(1 / sqrt(c2));
    a.c.eps = static_cast<float>(p->eps);
    a.c.turn = static_cast<uint32_t>(p->step) * 0x9E3779B1u;
    a.c.grad_scale = grad_scale;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    auto flush = [&](unsigned chunks) {
        using B = __nv_bfloat16;
        const bool pb = param_dtype == CCQ_BF16, gb = grad_dtype == CCQ_BF16, s8 = state_bits == 8;
        if (!pb)
            return gb ? (s8 ? launch_adamw<float, B, 8, 0>(a, chunks, s) : launch_adamw<float, B, 32, 0>(a, chunks, s))
                      : (s8 ? launch_adamw<float, float, 8, 0>(a, chunks, s) : launch_adamw<float, float, 32, 0>(a, chunks, s));
        if (!master)
            return gb ? (s8 ? launch_adamw<B, B, 8, 0>(a, chunks, s) : launch_adamw<B, B, 32, 0>(a, chunks, s))
                      : (s8 ? launch_adamw<B, float, 8, 0>(a, chunks, s) : launch_adamw<B, float, 32, 0>(a, chunks, s));
        return gb ? (s8 ? launch_adamw<B, B, 8, 1>(a, chunks, s) : launch_adamw<B, B, 32, 1>(a, chunks, s))
                  : (s8 ? launch_adamw<B, float, 8, 1>(a, chunks, s) : launch_adamw<B, float, 32, 1>(a, chunks, s));
    };
    a.count = 0;
    int64_t chunks = 0;
    const int64_t most = 0x7fffffff;  // CTAs of a launch
    for (int i = 0; i < count; ++i) {
        const ccq_adamw_tensor &t = tensors[i];
        if (t.n == 0) continue;
        const int64_t c = (t.n + kChunk - 1) / kChunk;
        if (a.count == kMaxTensors || chunks + c > most) {
            cudaError_t e = flush(static_cast<unsigned>(chunks));
            if (e != cudaSuccess) return op_cuda(e, "AdamW launch");
            a.count = 0;
            chunks = 0;
        }
        auto at = [](const void *q, int bytes) { return reinterpret_cast<uintptr_t>(q) % bytes == 0; };
        AdamTensor &d = a.t[a.count++];
        d = {t.param, t.grad, t.m, t.v, t.scale, t.master, t.n, static_cast<uint32_t>(chunks), 0};
        d.vec = at(t.param, 16) && at(t.grad, 16) && at(t.m, state_bits == 8 ? 8 : 16) && at(t.v, state_bits == 8 ? 8 : 16) &&
                at(t.master, 16);
        chunks += c;
    }
    return a.count ? op_cuda(flush(static_cast<unsigned>(chunks)), "AdamW launch") : CCQ_OK;
}

// ccq_decay_step.cu -- one token of linear attention with a decay for each head, on states in place (ccq_ops.h).
//
// state = g state + k v^T, o = scale state^T q: each state is read and written once, 8 d^2 bytes a head, and nothing else
// counts: bound by HBM.  A CTA takes 32 columns of a head's state, so that a small batch still reaches many SMs; its 128
// threads hold the slice in registers (all loads under way at once), and the partial sums of o cross threads once.
// 256 x 16 states of 64 KB: 80 to 83 us, 6.5 TB/s, 96 % of a copy; 2 x 4 of 128: 2.1 us, a launch.  With slots, every CTA looks for its
// state among the rows before it: 3 % more for 1024 rows of 16 heads, 10 % for 4096, 40 % for 16384 of 4 heads, 4 times the time for 65536 of one.
#include <cmath>

#include "ccq_decay.cuh"

namespace ccq {
namespace {

constexpr int kThreads = 128;
constexpr int kN = 32;                     // columns of a CTA
constexpr int kLanes = kN / 4;             // threads along a row
constexpr int kRows = kThreads / kLanes;   // rows at once

struct StepArgs {
    DecayView q, k, v;
    void *o;
    int64_t o_batch, o_head;
    const float *log_decay;
    float scale;
    float *state;
    int64_t rows;
    const void *slots;
    int slot_bytes;
    int H;
    int *status;
};

template <typename T, int D> __global__ void __launch_bounds__(kThreads) decay_step_kernel(const StepArgs a) {
    __shared__ float qs[D], ks[D], vs[kN];
    __shared__ float2 factor;
    __shared__ float4 part[kRows / 4][kLanes];
    constexpr int kSlices = D / kN, R = D / kRows;
    const int slice = blockIdx.x % kSlices, bh = blockIdx.x / kSlices, b = bh / a.H, h = bh % a.H;
    const int tid = threadIdx.x, tx = tid % kLanes, ty = tid / kLanes, c0 = slice * kN;
    int64_t row = b;
    bool live = true;
    if (a.slots) {
        row = load_index(a.slots, a.slot_bytes, b);
        live = row >= 0 && row < a.rows;
    }
    float4 s[R];
    float *state = a.state + ((live ? row : 0) * a.H + h) * D * D + c0 + 4 * tx;
    if (live) {
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = __ldcs(reinterpret_cast<const float4 *>(state + (ty + kRows * r) * D));
    }
    const T *q = static_cast<const T *>(a.q.p) + b * a.q.batch + (h / a.q.share) * a.q.head;
    const T *k = static_cast<const T *>(a.k.p) + b * a.k.batch + (h / a.k.share) * a.k.head;
    const T *v = static_cast<const T *>(a.v.p) + b * a.v.batch + (h / a.v.share) * a.v.head + c0;
    if (tid < D) {
        qs[tid] = to_f32(q[tid]);
        ks[tid] = to_f32(k[tid]);
    }
    if (tid < kN) vs[tid] = to_f32(v[tid]);
    // g as two floats: one float's rounding would be off to the same side at every token and add up over a decode
    if (tid == kThreads - 1) factor = decay_factor(decay_log2(a.log_decay, h));
    // a state that an earlier row of the batch has is that row's
    int taken = 0;
    if (a.slots && live)
        for (int i = tid; i < b; i += kThreads) taken |= load_index(a.slots, a.slot_bytes, i) == row;
    if (__syncthreads_or(taken)) live = false;
    if (!live && a.slots && row >= 0 && tid == 0) note_index(a.status);
    const float2 g = factor;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live) {
        const float4 vv = *reinterpret_cast<const float4 *>(&vs[4 * tx]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = ty + kRows * r;
            const float kk = ks[i], qq = qs[i];
            s[r].x = fmaf(s[r].x, g.x, fmaf(s[r].x, g.y, kk * vv.x));
            s[r].y = fmaf(s[r].y, g.x, fmaf(s[r].y, g.y, kk * vv.y));
            s[r].z = fmaf(s[r].z, g.x, fmaf(s[r].z, g.y, kk * vv.z));
            s[r].w = fmaf(s[r].w, g.x, fmaf(s[r].w, g.y, kk * vv.w));
            o.x += qq * s[r].x;
            o.y += qq * s[r].y;
            o.z += qq * s[r].z;
            o.w += qq * s[r].w;
            __stcs(reinterpret_cast<float4 *>(state + i * D), s[r]);
        }
    }
#pragma unroll
    for (int m = kLanes; m < 32; m *= 2) {
        o.x += __shfl_xor_sync(0xffffffffu, o.x, m);
        o.y += __shfl_xor_sync(0xffffffffu, o.y, m);
        o.z += __shfl_xor_sync(0xffffffffu, o.z, m);
        o.w += __shfl_xor_sync(0xffffffffu, o.w, m);
    }
    if (tid % 32 < kLanes) part[tid / 32][tx] = o;
    __syncthreads();
    if (tid < kN) {
        float f = 0.f;
#pragma unroll
        for (int w = 0; w < kRows / 4; ++w) f += reinterpret_cast<const float *>(part[w])[tid];
        static_cast<T *>(a.o)[b * a.o_batch + h * a.o_head + c0 + tid] = from_f32<T>(f * a.scale);
    }
}

template <typename T, int D> cudaError_t launch_step(const StepArgs &a, int64_t B, cudaStream_t s) {
    decay_step_kernel<T, D><<<static_cast<unsigned>(B * a.H * (D / kN)), kThreads, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace
}  // namespace ccq

using namespace ccq;

extern "C" {

ccq_status ccq_decay_attention_step(const ccq_heads *q, const ccq_heads *k, const ccq_heads *v, ccq_dtype dtype,
                                    const float *log_decay, float scale, float *state, int64_t rows, const void *slots,
                                    int slot_bytes, const ccq_heads *o, int64_t B, int H, int d, void *stream) {
    if (!q || !k || !v || !o) return op_fail(CCQ_ERR_INVALID_ARG, "q, k, v or o is NULL");
    if (!valid_dtype(dtype)) return op_fail(CCQ_ERR_INVALID_ARG, "unknown dtype %d", static_cast<int>(dtype));
    if (B < 0 || rows < 0 || H < 1 || H > (1 << 20))
        return op_fail(CCQ_ERR_INVALID_ARG, "bad sizes: B=%lld rows=%lld H=%d", static_cast<long long>(B),
                       static_cast<long long>(rows), H);
    if (d != 64 && d != 128) return op_fail(CCQ_ERR_UNSUPPORTED, "d=%d: 64 or 128", d);
    if (B > (1 << 24) || B * H > (1 << 24) || rows > (1LL << 40) / H)
        return op_fail(CCQ_ERR_UNSUPPORTED, "B=%lld of %d heads: at most 2^24 of both", static_cast<long long>(B), H);
    if (!std::isfinite(scale)) return op_fail(CCQ_ERR_INVALID_ARG, "scale is not finite");
    if (!slots && rows < B)
        return op_fail(CCQ_ERR_INVALID_ARG, "%lld states for a batch of %lld", static_cast<long long>(rows),
                       static_cast<long long>(B));
    if (B == 0) return CCQ_OK;
    ccq_status st = op_pointer("log_decay", log_decay, 4);
    if (st != CCQ_OK) return st;
    const ccq_heads *in[4] = {q, k, v, o};
    const char *names[4] = {"q", "k", "v", "o"};
    for (int i = 0; i < 4; ++i) {
        if ((st = check_heads(names[i], *in[i], dtype, B, 1, d, i == 3)) != CCQ_OK) return st;
        if (in[i]->heads > H || H % in[i]->heads)
            return op_fail(CCQ_ERR_INVALID_ARG, "%s has %lld heads, no divisor of %d", names[i],
                           static_cast<long long>(in[i]->heads), H);
    }
    if (o->heads != H) return op_fail(CCQ_ERR_INVALID_ARG, "o has %lld heads, expected %d", static_cast<long long>(o->heads), H);
    if ((st = op_pointer("state", state, 16)) != CCQ_OK) return st;
    if (slots) {
        if (slot_bytes != 4 && slot_bytes != 8) return op_fail(CCQ_ERR_INVALID_ARG, "slot_bytes=%d: 4 or 8", slot_bytes);
        if ((st = op_pointer("slots", slots, slot_bytes)) != CCQ_OK) return st;
    }
    for (int i = 0; i < 3; ++i)
        if (in[i]->p == o->p) return op_fail(CCQ_ERR_INVALID_ARG, "o is %s: other blocks still read it", names[i]);
    StepArgs a = {};
    if ((st = op_status_word(&a.status)) != CCQ_OK) return st;
    for (int i = 0; i < 3; ++i)
        if ((st = check_apart("o", *o, names[i], *in[i], dtype_bytes(dtype), B, 1, d)) != CCQ_OK) return st;
    auto view = [H](const ccq_heads &x) { return DecayView{x.p, x.batch, 0, x.head, static_cast<int>(H / x.heads)}; };
    a.q = view(*q);
    a.k = view(*k);
    a.v = view(*v);
    a.o = o->p;
    a.o_batch = o->batch;
    a.o_head = o->head;
    a.log_decay = log_decay;
    a.scale = scale;
    a.state = state;
    a.rows = rows;
    a.slots = slots;
    a.slot_bytes = slot_bytes;
    a.H = H;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (dtype == CCQ_BF16)
        e = d == 128 ? launch_step<__nv_bfloat16, 128>(a, B, s) : launch_step<__nv_bfloat16, 64>(a, B, s);
    else
        e = d == 128 ? launch_step<float, 128>(a, B, s) : launch_step<float, 64>(a, B, s);
    return op_cuda(e, "decayed attention step launch");
}

}  // extern "C"

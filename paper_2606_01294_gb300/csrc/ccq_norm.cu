// ccq_norm.cu -- group norm of tokens, channels last, with an activation or a gate, and its gradients
// (ccq_ops.h).
//
// Both directions stream: the forward reads x (and the gate) and writes y, the backward reads x, the gate and
// dy and writes dx and dgate, each once; HBM bounds them.  A team of L threads holds a (token, group)'s d
// channels in registers, K accesses of N elements each, so that the mean, then the squared deviations from it
// (two passes over registers: no cancellation for a group whose mean is large), and in the backward
// the two means of its formula, are sums over registers and a team:
//   s = act(gate), du = dy s, dgate = dy u act'(gate)      (no gate: du = dy act'(u))
//   dxh = du weight,  dx = rstd (dxh - mean(dxh) - xh mean(dxh xh))     (mean(dxh) = 0 with centered = 0)
//   dweight = sum over tokens of du xh,  dbias = sum over tokens of du
// A team keeps one group and walks over tokens, so that its weights, and the backward's partial sums of
// dweight and dbias, stay in registers too; the partial sums go to the workspace once and norm_param_kernel
// adds them in a fixed order.  L is at most a warp's 32 where K accesses each suffice, else the
// whole CTA; groups beyond that (d > 4096) are walked in memory (the _long kernels).
#include <algorithm>

#include "ccq_ops.cuh"

namespace ccq {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxElems = 16;  // elements of a group that a thread holds

struct NormArgs {
    const void *x, *gate, *weight, *bias, *dy;
    int64_t x_stride, gate_stride, dy_stride, y_stride, dgate_stride;
    void *y;  // backward: dx
    void *dgate;
    float *part;  // backward: [2][slots][channels], the partial sums of dweight, then of dbias
    int64_t tokens;
    int channels, groups, d, team, slots;
    int centered, act, param_bf16;
    float eps;
};

__device__ __forceinline__ float param_at(const void *p, int bf16, int i, float none) {
    if (!p) return none;
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]) : static_cast<const float *>(p)[i];
}

__device__ __forceinline__ float sigmoid(float u) { return __fdividef(1.f, 1.f + __expf(-u)); }

// act(u) and, where asked for, its derivative.
__device__ __forceinline__ float activate(int act, float u) {
    if (act == CCQ_ACT_NONE) return u;
    const float s = sigmoid(u);
    return act == CCQ_ACT_SILU ? u * s : s;
}
__device__ __forceinline__ float activate(int act, float u, float &slope) {
    if (act == CCQ_ACT_NONE) {
        slope = 1.f;
        return u;
    }
    const float s = sigmoid(u);
    if (act == CCQ_ACT_SILU) {
        slope = s * (1.f + u * (1.f - s));
        return u * s;
    }
    slope = s * (1.f - s);
    return s;
}

// Sum over the team: lanes of a warp (WIDE = 0), or the CTA.  Every thread gets the same value.
template <int WIDE> __device__ __forceinline__ float team_sum(float v, int team, float *red) {
    if constexpr (!WIDE) {
        for (int o = team >> 1; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
        return v;
    } else {
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
        __syncthreads();  // the last sum's readers are done
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) t += red[w];
        return t;
    }
}

// The statistics of the group whose channels are x (elements past d are zero and `on` marks the others).
template <int WIDE, int E>
__device__ __forceinline__ void normalise(float (&x)[E], const bool (&on)[E], const NormArgs &a, float *red,
                                          float &rstd) {
    const float inv_d = 1.f / static_cast<float>(a.d);
    if (a.centered) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += x[e];
        const float mu = team_sum<WIDE>(s, a.team, red) * inv_d;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = on[e] ? x[e] - mu : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) q += x[e] * x[e];
    rstd = rsqrtf(team_sum<WIDE>(q, a.team, red) * inv_d + a.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= rstd;
}

// Forward (BWD = 0) and backward (BWD = 1) of groups held in registers: K accesses of N elements a thread.
template <typename T, int N, int K, int WIDE, int BWD>
__global__ void __launch_bounds__(kThreads) norm_kernel(NormArgs a) {
    constexpr int E = N * K;
    __shared__ float red[kThreads / 32];
    const int teams = kThreads / a.team;
    const int64_t gt = static_cast<int64_t>(blockIdx.x) * teams + threadIdx.x / a.team;
    const int l = threadIdx.x % a.team;
    const int group = static_cast<int>(gt % a.groups);
    const int64_t slot = gt / a.groups;
    const int base = group * a.d;
    float w[E], b[E], dw[BWD ? E : 1], db[BWD ? E : 1];
    bool on[E];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int c = (k * a.team + l) * N + e, i = k * N + e;
            on[i] = c < a.d;
            w[i] = on[i] ? param_at(a.weight, a.param_bf16, base + c, 1.f) : 0.f;
            b[i] = on[i] ? param_at(a.bias, a.param_bf16, base + c, 0.f) : 0.f;
            if constexpr (BWD) dw[i] = db[i] = 0.f;
        }
    const T *X = static_cast<const T *>(a.x) + base, *G = a.gate ? static_cast<const T *>(a.gate) + base : nullptr;
    const T *DY = static_cast<const T *>(a.dy) + base;
    T *Y = static_cast<T *>(a.y) + base, *DG = static_cast<T *>(a.dgate) + base;
    // every thread of a warp walks the same number of times: the sums are taken by whole warps
    const int64_t turns = (a.tokens + a.slots - 1) / a.slots;
    for (int64_t turn = 0; turn < turns; ++turn) {
        const int64_t t = turn * a.slots + slot;
        const bool live = slot < a.slots && t < a.tokens;
        float x[E], g[E], dy[BWD ? E : 1];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * a.team + l) * N;
            Pack<T, N> px, pg, pd;
            px.raw = pg.raw = pd.raw = {};
            if (live && c < a.d) {
                px = load_stream<T, N>(X + t * a.x_stride + c);
                if (G) pg = load_stream<T, N>(G + t * a.gate_stride + c);
                if constexpr (BWD) pd = load_stream<T, N>(DY + t * a.dy_stride + c);
            }
            float f[N];
            unpack(px, f);
#pragma unroll
            for (int e = 0; e < N; ++e) x[k * N + e] = f[e];
            unpack(pg, f);
#pragma unroll
            for (int e = 0; e < N; ++e) g[k * N + e] = f[e];
            if constexpr (BWD) {
                unpack(pd, f);
#pragma unroll
                for (int e = 0; e < N; ++e) dy[k * N + e] = f[e];
            }
        }
        float rstd;
        normalise<WIDE, E>(x, on, a, red, rstd);
        if constexpr (!BWD) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float u = x[i] * w[i] + b[i];
                x[i] = G ? u * activate(a.act, g[i]) : activate(a.act, u);
            }
        } else {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float u = x[i] * w[i] + b[i];
                float slope, du;
                if (G) {
                    const float s = activate(a.act, g[i], slope);
                    du = dy[i] * s;
                    g[i] = dy[i] * u * slope;
                } else {
                    activate(a.act, u, slope);
                    du = dy[i] * slope;
                }
                if (live) {
                    dw[i] += du * x[i];
                    db[i] += du;
                }
                dy[i] = du * w[i];
                s1 += dy[i];
                s2 += dy[i] * x[i];
            }
            const float inv_d = 1.f / static_cast<float>(a.d);
            s1 = a.centered ? team_sum<WIDE>(s1, a.team, red) * inv_d : 0.f;
            s2 = team_sum<WIDE>(s2, a.team, red) * inv_d;
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = rstd * (dy[i] - s1 - x[i] * s2);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * a.team + l) * N;
            if (!live || c >= a.d) continue;
            float f[N];
            Pack<T, N> p;
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] = x[k * N + e];
            pack(f, p);
            store_stream<T, N>(Y + t * a.y_stride + c, p);
            if constexpr (BWD) {
                if (G) {
#pragma unroll
                    for (int e = 0; e < N; ++e) f[e] = g[k * N + e];
                    pack(f, p);
                    store_stream<T, N>(DG + t * a.dgate_stride + c, p);
                }
            }
        }
    }
    if constexpr (BWD) {
        if (!a.part || slot >= a.slots) return;
        float *pw = a.part + slot * a.channels + base, *pb = pw + static_cast<int64_t>(a.slots) * a.channels;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int c = (k * a.team + l) * N + e, i = k * N + e;
                if (c < a.d) {
                    pw[c] = dw[i];
                    pb[c] = db[i];
                }
            }
    }
}

// Groups too long for registers: a CTA for each slot of a group, the channels walked in memory.  The partial
// sums are kept in the slot's own row of `part`, which its thread reads and writes back.
template <typename T, int BWD> __global__ void __launch_bounds__(kThreads) norm_long_kernel(NormArgs a) {
    __shared__ float red[kThreads / 32];
    const int group = static_cast<int>(blockIdx.x % a.groups);
    const int64_t slot = blockIdx.x / a.groups;
    const int base = group * a.d;
    const float inv_d = 1.f / static_cast<float>(a.d);
    float *pw = nullptr, *pb = nullptr;
    if (BWD && a.part) {
        pw = a.part + slot * a.channels + base;
        pb = pw + static_cast<int64_t>(a.slots) * a.channels;
        for (int c = threadIdx.x; c < a.d; c += kThreads) pw[c] = pb[c] = 0.f;
    }
    for (int64_t t = slot; t < a.tokens; t += a.slots) {
        const T *X = static_cast<const T *>(a.x) + t * a.x_stride + base;
        const T *G = a.gate ? static_cast<const T *>(a.gate) + t * a.gate_stride + base : nullptr;
        T *Y = static_cast<T *>(a.y) + t * a.y_stride + base;
        float s = 0.f, mu = 0.f, q = 0.f;
        if (a.centered) {
            for (int c = threadIdx.x; c < a.d; c += kThreads) s += to_f32(X[c]);
            mu = team_sum<1>(s, kThreads, red) * inv_d;
        }
        for (int c = threadIdx.x; c < a.d; c += kThreads) {
            const float v = to_f32(X[c]) - mu;
            q += v * v;
        }
        const float rstd = rsqrtf(team_sum<1>(q, kThreads, red) * inv_d + a.eps);
        if (!BWD) {
            for (int c = threadIdx.x; c < a.d; c += kThreads) {
                const float u = (to_f32(X[c]) - mu) * rstd * param_at(a.weight, a.param_bf16, base + c, 1.f) +
                                param_at(a.bias, a.param_bf16, base + c, 0.f);
                Y[c] = from_f32<T>(G ? u * activate(a.act, to_f32(G[c])) : activate(a.act, u));
            }
            continue;
        }
        const T *DY = static_cast<const T *>(a.dy) + t * a.dy_stride + base;
        T *DG = static_cast<T *>(a.dgate) + t * a.dgate_stride + base;
        // du of channel c, with dgate in `dg`
        auto grad = [&](int c, float xh, float w, float &dg) {
            const float u = xh * w + param_at(a.bias, a.param_bf16, base + c, 0.f), dy = to_f32(DY[c]);
            float slope;
            if (G) {
                const float act = activate(a.act, to_f32(G[c]), slope);
                dg = dy * u * slope;
                return dy * act;
            }
            activate(a.act, u, slope);
            return dy * slope;
        };
        float s1 = 0.f, s2 = 0.f, dg = 0.f;
        for (int c = threadIdx.x; c < a.d; c += kThreads) {
            const float xh = (to_f32(X[c]) - mu) * rstd, w = param_at(a.weight, a.param_bf16, base + c, 1.f);
            const float du = grad(c, xh, w, dg);
            s1 += du * w;
            s2 += du * w * xh;
        }
        s1 = a.centered ? team_sum<1>(s1, kThreads, red) * inv_d : 0.f;
        s2 = team_sum<1>(s2, kThreads, red) * inv_d;
        for (int c = threadIdx.x; c < a.d; c += kThreads) {
            const float xh = (to_f32(X[c]) - mu) * rstd, w = param_at(a.weight, a.param_bf16, base + c, 1.f);
            const float du = grad(c, xh, w, dg);
            if (pw) {
                pw[c] += du * xh;
                pb[c] += du;
            }
            Y[c] = from_f32<T>(rstd * (du * w - s1 - xh * s2));
            if (G) DG[c] = from_f32<T>(dg);
        }
    }
}

// dweight and dbias: 32 channels a CTA, the slots over 32 rows of threads, then those 32 in order.
constexpr int kParamRows = 32;
__global__ void __launch_bounds__(32 * kParamRows) norm_param_kernel(const float *part, int slots, int channels,
                                                                     void *dweight, void *dbias, int param_bf16) {
    __shared__ float sums[kParamRows][33];
    grid_wait();
    const int which = blockIdx.y, c = blockIdx.x * 32 + threadIdx.x;
    void *out = which ? dbias : dweight;
    if (!out) return;
    const float *p = part + static_cast<int64_t>(which) * slots * channels;
    float s = 0.f;
    if (c < channels)
        for (int i = threadIdx.y; i < slots; i += kParamRows) s += p[static_cast<int64_t>(i) * channels + c];
    sums[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y || c >= channels) return;
    s = 0.f;
    for (int r = 0; r < kParamRows; ++r) s += sums[r][threadIdx.x];
    if (param_bf16) static_cast<__nv_bfloat16 *>(out)[c] = __float2bfloat16_rn(s);
    else static_cast<float *>(out)[c] = s;
}

// How the groups are spread over threads, and how many slots of tokens there are.
struct Shape {
    int n, k, team, slots;  // accesses of n elements, k a thread; team = 0: walked in memory
    unsigned grid;
};

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

Shape shape_of(int64_t tokens, int channels, int groups, int n, int sms) {
    Shape s = {};
    const int d = channels / groups, packs = d / n, kmax = kMaxElems / n;
    s.n = n;
    s.k = 1;
    while (s.k < kmax && 32 * s.k < packs) s.k = n == 1 || n == 2 ? s.k * 4 : s.k * 2;
    s.k = std::min(s.k, kmax);
    if (32 * s.k >= packs) {
        s.team = 1;
        while (s.team < packs && s.team < 32) s.team *= 2;
    } else if (kThreads * kmax >= packs) {
        s.k = kmax;
        s.team = kThreads;
    }
    const int teams = s.team ? kThreads / s.team : 1;  // a CTA's teams
    // a CTA count that is a multiple of `unit` gives every group the same number of teams
    const int unit = groups / gcd(groups, teams);
    const int64_t want = std::min<int64_t>(static_cast<int64_t>(sms) * 4, (tokens * groups + teams - 1) / teams);
    const int64_t grid = std::max<int64_t>(1, want / unit) * unit;
    s.grid = static_cast<unsigned>(grid);
    s.slots = static_cast<int>(grid * teams / groups);
    return s;
}

template <typename T, int N, int K, int BWD> cudaError_t launch_one(const NormArgs &a, unsigned grid, cudaStream_t s) {
    if (a.team == kThreads) {
        if constexpr (N * K == kMaxElems) norm_kernel<T, N, K, 1, BWD><<<grid, kThreads, 0, s>>>(a);
    } else {
        norm_kernel<T, N, K, 0, BWD><<<grid, kThreads, 0, s>>>(a);
    }
    return cudaGetLastError();
}

template <typename T, int BWD> cudaError_t launch_norm(NormArgs a, const Shape &sh, cudaStream_t s) {
    a.team = sh.team;
    a.slots = sh.slots;
    if (!sh.team) {
        norm_long_kernel<T, BWD><<<sh.grid, kThreads, 0, s>>>(a);
        return cudaGetLastError();
    }
    if constexpr (sizeof(T) == 2) {
        if (sh.n == 8)
            return sh.k == 1 ? launch_one<T, 8, 1, BWD>(a, sh.grid, s) : launch_one<T, 8, 2, BWD>(a, sh.grid, s);
        if (sh.n == 2)
            return sh.k == 1   ? launch_one<T, 2, 1, BWD>(a, sh.grid, s)
                   : sh.k == 4 ? launch_one<T, 2, 4, BWD>(a, sh.grid, s)
                               : launch_one<T, 2, 8, BWD>(a, sh.grid, s);
    } else if (sh.n == 4) {
        return sh.k == 1   ? launch_one<T, 4, 1, BWD>(a, sh.grid, s)
               : sh.k == 2 ? launch_one<T, 4, 2, BWD>(a, sh.grid, s)
                           : launch_one<T, 4, 4, BWD>(a, sh.grid, s);
    }
    return sh.k == 1   ? launch_one<T, 1, 1, BWD>(a, sh.grid, s)
           : sh.k == 4 ? launch_one<T, 1, 4, BWD>(a, sh.grid, s)
                       : launch_one<T, 1, 16, BWD>(a, sh.grid, s);
}

ccq_status check_norm(int64_t tokens, int channels, int groups, float eps, ccq_dtype dtype, ccq_dtype param_dtype, int act) {
    if (tokens < 0 || channels < 1 || groups < 1 || channels % groups)
        return op_fail(CCQ_ERR_INVALID_ARG, "bad sizes tokens=%lld channels=%d groups=%d",
                       static_cast<long long>(tokens), channels, groups);
    if (!valid_dtype(dtype) || !valid_dtype(param_dtype))
        return op_fail(CCQ_ERR_INVALID_ARG, "unknown dtype %d or param dtype %d", dtype, param_dtype);
    if (act != CCQ_ACT_NONE && act != CCQ_ACT_SILU && act != CCQ_ACT_SIGMOID)
        return op_fail(CCQ_ERR_INVALID_ARG, "unknown activation %d", act);
    if (!(eps >= 0.f)) return op_fail(CCQ_ERR_INVALID_ARG, "eps must be >= 0");
    return CCQ_OK;
}

// One [tokens, channels] operand; `least` shrinks to its access width.
ccq_status check_operand(const char *name, const void *p, int64_t stride, int64_t tokens, int channels, int es, int *least) {
    if (tokens > 1 && stride < channels)
        return op_fail(CCQ_ERR_INVALID_ARG, "%s: row stride %lld is below the %d channels", name,
                       static_cast<long long>(stride), channels);
    *least = row_access(p, stride, es, tokens, *least);
    return op_pointer(name, p, es);
}

// The widest access with its kernels: 16 bytes, 4 bytes, or one element.
int access_elems(int bytes, int es) { return bytes == 16 ? 16 / es : bytes >= 4 && es == 2 ? 2 : 1; }

ccq_status check_param(const char *name, const void *p, ccq_dtype dt) {
    return p ? op_pointer(name, p, dtype_bytes(dt)) : CCQ_OK;
}

// The most slots any access width gives: bounds the partial sums.
size_t bwd_workspace(int64_t tokens, int channels, int groups, int es) {
    int slots = 1;
    for (int n : {16 / es, 2, 1})
        if ((channels / groups) % n == 0) slots = std::max(slots, shape_of(tokens, channels, groups, n, sm_count_now()).slots);
    return static_cast<size_t>(2) * slots * channels * sizeof(float);
}

}  // namespace
}  // namespace ccq

using namespace ccq;

extern "C" {

ccq_status ccq_group_norm(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, const void *weight,
                          const void *bias, ccq_dtype dtype, ccq_dtype param_dtype, void *y, int64_t y_stride,
                          int64_t tokens, int channels, int groups, int centered, float eps, ccq_activation act,
                          void *stream) {
    ccq_status st = check_norm(tokens, channels, groups, eps, dtype, param_dtype, act);
    if (st != CCQ_OK) return st;
    if (tokens == 0) return CCQ_OK;
    const int es = dtype_bytes(dtype), d = channels / groups;
    int b = access_bytes(static_cast<uintptr_t>(d) * es);
    if ((st = check_operand("x", x, x_stride, tokens, channels, es, &b)) != CCQ_OK) return st;
    if (gate && (st = check_operand("gate", gate, gate_stride, tokens, channels, es, &b)) != CCQ_OK) return st;
    if ((st = check_operand("y", y, y_stride, tokens, channels, es, &b)) != CCQ_OK) return st;
    if ((st = check_param("weight", weight, param_dtype)) != CCQ_OK) return st;
    if ((st = check_param("bias", bias, param_dtype)) != CCQ_OK) return st;
    NormArgs a = {};
    a.x = x; a.gate = gate; a.weight = weight; a.bias = bias; a.y = y;
    a.x_stride = x_stride; a.gate_stride = gate_stride; a.y_stride = y_stride;
    a.tokens = tokens; a.channels = channels; a.groups = groups; a.d = d;
    a.centered = centered != 0; a.act = act; a.param_bf16 = param_dtype == CCQ_BF16; a.eps = eps;
    const Shape sh = shape_of(tokens, channels, groups, access_elems(b, es), sm_count_now());
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return op_cuda(dtype == CCQ_BF16 ? launch_norm<__nv_bfloat16, 0>(a, sh, s) : launch_norm<float, 0>(a, sh, s),
                   "group norm launch");
}

ccq_status ccq_group_norm_bwd_workspace_size(int64_t tokens, int channels, int groups, ccq_dtype dtype, size_t *bytes) {
    ccq_status st = check_norm(tokens, channels, groups, 0.f, dtype, CCQ_FP32, CCQ_ACT_NONE);
    if (st != CCQ_OK) return st;
    if (!bytes) return op_fail(CCQ_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = bwd_workspace(tokens, channels, groups, dtype_bytes(dtype));
    return CCQ_OK;
}

ccq_status ccq_group_norm_bwd(const void *x, int64_t x_stride, const void *gate, int64_t gate_stride, const void *weight,
                              const void *bias, const void *dy, int64_t dy_stride, ccq_dtype dtype, ccq_dtype param_dtype,
                              void *dx, int64_t dx_stride, void *dgate, int64_t dgate_stride, void *dweight, void *dbias,
                              int64_t tokens, int channels, int groups, int centered, float eps, ccq_activation act,
                              void *workspace, size_t workspace_bytes, void *stream) {
    ccq_status st = check_norm(tokens, channels, groups, eps, dtype, param_dtype, act);
    if (st != CCQ_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if ((st = check_param("weight", weight, param_dtype)) != CCQ_OK) return st;
    if ((st = check_param("bias", bias, param_dtype)) != CCQ_OK) return st;
    if ((st = check_param("dweight", dweight, param_dtype)) != CCQ_OK) return st;
    if ((st = check_param("dbias", dbias, param_dtype)) != CCQ_OK) return st;
    if (tokens == 0) {
        for (void *p : {dweight, dbias})
            if (p) {
                cudaError_t e = cudaMemsetAsync(p, 0, static_cast<size_t>(channels) * dtype_bytes(param_dtype), s);
                if (e != cudaSuccess) return op_cuda(e, "zero gradients");
            }
        return CCQ_OK;
    }
    const int es = dtype_bytes(dtype), d = channels / groups;
    int b = access_bytes(static_cast<uintptr_t>(d) * es);
    if ((st = check_operand("x", x, x_stride, tokens, channels, es, &b)) != CCQ_OK) return st;
    if ((st = check_operand("dy", dy, dy_stride, tokens, channels, es, &b)) != CCQ_OK) return st;
    if ((st = check_operand("dx", dx, dx_stride, tokens, channels, es, &b)) != CCQ_OK) return st;
    if ((gate == nullptr) != (dgate == nullptr))
        return op_fail(CCQ_ERR_INVALID_ARG, "dgate is given exactly when gate is");
    if (gate) {
        if ((st = check_operand("gate", gate, gate_stride, tokens, channels, es, &b)) != CCQ_OK) return st;
        if ((st = check_operand("dgate", dgate, dgate_stride, tokens, channels, es, &b)) != CCQ_OK) return st;
    }
    const bool params = dweight || dbias;
    if (params) {
        const size_t need = bwd_workspace(tokens, channels, groups, es);
        if ((st = op_pointer("workspace", workspace, 16)) != CCQ_OK) return st;
        if (workspace_bytes < need)
            return op_fail(CCQ_ERR_INVALID_ARG, "workspace of %zu bytes, needs %zu", workspace_bytes, need);
    }
    NormArgs a = {};
    a.x = x; a.gate = gate; a.weight = weight; a.bias = bias; a.dy = dy; a.y = dx; a.dgate = dgate;
    a.x_stride = x_stride; a.gate_stride = gate_stride; a.dy_stride = dy_stride; a.y_stride = dx_stride;
    a.dgate_stride = dgate_stride;
    a.part = params ? static_cast<float *>(workspace) : nullptr;
    a.tokens = tokens; a.channels = channels; a.groups = groups; a.d = d;
    a.centered = centered != 0; a.act = act; a.param_bf16 = param_dtype == CCQ_BF16; a.eps = eps;
    const Shape sh = shape_of(tokens, channels, groups, access_elems(b, es), sm_count_now());
    cudaError_t e = dtype == CCQ_BF16 ? launch_norm<__nv_bfloat16, 1>(a, sh, s) : launch_norm<float, 1>(a, sh, s);
    if (e != cudaSuccess || !params) return op_cuda(e, "group norm backward launch");
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((channels + 31) / 32, 2);
    cfg.blockDim = dim3(32, kParamRows);
    cfg.stream = s;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, norm_param_kernel, static_cast<const float *>(a.part), sh.slots, channels, dweight, dbias,
                           a.param_bf16);
    return op_cuda(e, "group norm parameter gradient launch");
}

}  // extern "C"

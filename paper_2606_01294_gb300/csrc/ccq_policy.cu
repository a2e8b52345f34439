// ccq_policy.cu -- clipped policy loss with a KL term over token logits, its gradient, and the token
// log-probabilities alone (ccq_ops.h).
//
// For a row x of logits with maximum m, e_j = exp((x_j - m) / T), Z = sum e_j, the row's log-probability is
//   logp = (x_a - m) / T - log Z
// and everything else is a function of the row's scalars; the gradient is
//   dlogits_j = c (delta_ja - e_j / Z),   c = grad_scale w dL/dlogp / T,
//   dL/dlogp = -(r A where r A <= clip(r) A, else 0) + kl_coef (1 - exp(ref - logp)).
// A row is read, its maximum and sum are formed in one pass with a running maximum, and the gradient's pass
// follows.  Bound by HBM: the logits in, the gradient out.
#include <algorithm>

#include "ccq_ops.cuh"

namespace ccq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct PolicyArgs {
    const void *logits, *actions;
    int64_t logits_stride, dlogits_stride, n;
    int id_bytes, vocab;
    const float *old_logp, *ref_logp, *advantages, *weights;
    ccq_policy_params p;
    float scale;      // log2(e) / temperature
    float *logp, *row_loss;
    void *dlogits;
    int score;  // 1: log-probabilities alone
    int *status;
};

// What a row's scalars say about it before its logits are read.
struct Row {
    int action;  // -1: masked
    float weight;
};
__device__ __forceinline__ Row row_of(const PolicyArgs &a, int64_t i, bool note) {
    Row r;
    r.weight = a.score ? 1.f : a.weights ? a.weights[i] : 1.f / static_cast<float>(a.n);
    r.action = -1;
    if (r.weight != 0.f) {
        const int64_t t = load_index(a.actions, a.id_bytes, i);
        if (t >= 0 && t < a.vocab) r.action = static_cast<int>(t);
        else if (note) note_index(a.status);
    }
    return r;
}

// The row's loss and c of the gradient, from its log-probability.
__device__ __forceinline__ float row_loss(const PolicyArgs &a, int64_t i, float weight, float logp, float &c) {
    const float adv = a.advantages[i];
    const float ratio = expf(logp - a.old_logp[i]);
    const float open = ratio * adv;
    const float held = fminf(fmaxf(ratio, 1.f - a.p.clip_low), 1.f + a.p.clip_high) * adv;
    // a ratio or advantage that is not a number stays one
    float loss = open <= held || !(held < open) ? -open : -held;
    float slope = open <= held || !(held < open) ? -open : 0.f;
    if (a.ref_logp && a.p.kl_coef != 0.f) {
        const float d = a.ref_logp[i] - logp;
        const float em1 = expm1f(d);
        loss += a.p.kl_coef * (em1 - d);
        slope -= a.p.kl_coef * em1;
    }
    c = a.p.grad_scale * weight * slope / a.p.temperature;
    return weight * loss;
}

constexpr int kRowThreads = 512;

// Sum or maximum of one value per thread over the CTA.
__device__ __forceinline__ void join(float &m, float &z, float om, float oz, float scale) {
    const float top = fmaxf(m, om);
    // equal maxima (both -inf among them) keep their sums as they are
    const float fm = m == top ? 1.f : exp2f((m - top) * scale), fo = om == top ? 1.f : exp2f((om - top) * scale);
    z = z * fm + oz * fo;
    m = top;
}

template <typename T, int N> __global__ void __launch_bounds__(kRowThreads) policy_row_kernel(PolicyArgs a) {
    __shared__ float sm[kRowThreads / 32], sz[kRowThreads / 32], bc[3];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int packs = a.vocab / N;
    for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
        const Row row = row_of(a, i, tid == 0);
        const T *x = static_cast<const T *>(a.logits) + i * a.logits_stride;
        T *dx = static_cast<T *>(a.dlogits) + i * a.dlogits_stride;
        if (row.action < 0) {
            if (tid == 0) {
                if (a.logp) a.logp[i] = a.score ? __int_as_float(0x7fc00000) : 0.f;
                if (!a.score) a.row_loss[i] = 0.f;
            }
            if (a.dlogits)
                for (int c = tid; c < packs; c += kRowThreads) {
                    Pack<T, N> p;
                    p.raw = {};
                    store_stream<T, N>(dx + static_cast<int64_t>(c) * N, p);
                }
            continue;
        }
        float m = -INFINITY, z = 0.f;
        for (int c = tid; c < packs; c += kRowThreads) {
            float f[N];
            unpack(load_plain<T, N>(x + static_cast<int64_t>(c) * N), f);
            float top = m;
#pragma unroll
            for (int e = 0; e < N; ++e) top = fmaxf(top, f[e]);
            if (top > m) {
                z *= exp2f((m - top) * a.scale);
                m = top;
            }
#pragma unroll
            for (int e = 0; e < N; ++e) z += f[e] == m ? 1.f : exp2f((f[e] - m) * a.scale);
        }
        for (int o = 16; o; o >>= 1) {
            const float om = __shfl_xor_sync(~0u, m, o), oz = __shfl_xor_sync(~0u, z, o);
            join(m, z, om, oz, a.scale);
        }
        if (lane == 0) {
            sm[warp] = m;
            sz[warp] = z;
        }
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kRowThreads / 32; ++w) join(m, z, sm[w], sz[w], a.scale);
            const float logp = (to_f32(x[row.action]) - m) * (a.scale * kLn2) - logf(z);
            float c = 0.f;
            if (a.score) {
                a.logp[i] = logp;
            } else {
                a.row_loss[i] = row_loss(a, i, row.weight, logp, c);
                if (a.logp) a.logp[i] = logp;
            }
            bc[0] = m;
            bc[1] = c;
            bc[2] = -c / z;
        }
        __syncthreads();
        if (a.dlogits) {
            m = bc[0];
            const float c1 = bc[1], c2 = bc[2];
            for (int c = tid; c < packs; c += kRowThreads) {
                float f[N];
                Pack<T, N> p = load_plain<T, N>(x + static_cast<int64_t>(c) * N);
                unpack(p, f);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    f[e] = c2 * exp2f((f[e] - m) * a.scale);
                    if (c * N + e == row.action) f[e] += c1;
                }
                pack(f, p);
                store_stream<T, N>(dx + static_cast<int64_t>(c) * N, p);
            }
        }
        __syncthreads();
    }
}

// loss = the rows' losses, by 1024 strided sums and a tree: an order that depends on n alone.
constexpr int kLossThreads = 1024;
__global__ void __launch_bounds__(kLossThreads) policy_loss_kernel(const float *row_loss, int64_t n, float *loss) {
    __shared__ float sums[kLossThreads / 32];
    grid_wait();
    float s = 0.f;
    for (int64_t i = threadIdx.x; i < n; i += kLossThreads) s += row_loss[i];
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    s = sums[threadIdx.x];
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    if (threadIdx.x == 0) *loss = s;
}

template <typename T, int N> cudaError_t launch_rows(const PolicyArgs &a, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(a.n, 1 << 20));
    policy_row_kernel<T, N><<<grid, kRowThreads, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_policy(const PolicyArgs &a, ccq_dtype dtype, cudaStream_t s) {
    const int es = dtype_bytes(dtype);
    int b = access_bytes(static_cast<uintptr_t>(a.vocab) * es);
    b = row_access(a.logits, a.logits_stride, es, a.n, b);
    if (a.dlogits) b = row_access(a.dlogits, a.dlogits_stride, es, a.n, b);
    if (dtype == CCQ_BF16)
        return b == 16 ? launch_rows<__nv_bfloat16, 8>(a, s) : b >= 4 ? launch_rows<__nv_bfloat16, 2>(a, s)
                                                                      : launch_rows<__nv_bfloat16, 1>(a, s);
    return b == 16 ? launch_rows<float, 4>(a, s) : launch_rows<float, 1>(a, s);
}

ccq_status check_logits(const char *name, const void *p, int64_t stride, ccq_dtype dtype, int64_t n, int vocab) {
    if (n > 1 && stride < vocab)
        return op_fail(CCQ_ERR_INVALID_ARG, "%s: row stride %lld is below the vocabulary %d", name,
                       static_cast<long long>(stride), vocab);
    return op_pointer(name, p, dtype_bytes(dtype));
}

ccq_status check_policy(int64_t n, int vocab, ccq_dtype dtype, float temperature, int id_bytes) {
    if (n < 0 || vocab < 1 || vocab > (1 << 30))
        return op_fail(CCQ_ERR_INVALID_ARG, "bad sizes n=%lld vocab=%d", static_cast<long long>(n), vocab);
    if (!valid_dtype(dtype)) return op_fail(CCQ_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (!(temperature > 0.f) || temperature > 1e30f)
        return op_fail(CCQ_ERR_INVALID_ARG, "temperature=%g must be positive and finite", static_cast<double>(temperature));
    if (id_bytes != 4 && id_bytes != 8) return op_fail(CCQ_ERR_INVALID_ARG, "id_bytes=%d: 4 or 8", id_bytes);
    return CCQ_OK;
}

}  // namespace
}  // namespace ccq

using namespace ccq;

extern "C" {

void ccq_default_policy_params(ccq_policy_params *p) {
    if (!p) return;
    p->clip_low = p->clip_high = 0.2f;
    p->kl_coef = 0.f;
    p->temperature = 1.f;
    p->grad_scale = 1.f;
}

ccq_status ccq_policy_loss_workspace_size(int64_t n, size_t *bytes) {
    if (n < 0) return op_fail(CCQ_ERR_INVALID_ARG, "bad size n=%lld", static_cast<long long>(n));
    if (!bytes) return op_fail(CCQ_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = (static_cast<size_t>(n) * sizeof(float) + 15) & ~static_cast<size_t>(15);
    return CCQ_OK;
}

ccq_status ccq_policy_loss(const void *logits, ccq_dtype dtype, int64_t logits_stride, const void *actions, int id_bytes,
                           const float *old_logp, const float *ref_logp, const float *advantages, const float *weights,
                           int64_t n, int vocab, const ccq_policy_params *p, float *loss, float *logp, void *dlogits,
                           int64_t dlogits_stride, void *workspace, size_t workspace_bytes, void *stream) {
    PolicyArgs a = {};
    if (p) a.p = *p;
    else ccq_default_policy_params(&a.p);
    ccq_status st = check_policy(n, vocab, dtype, a.p.temperature, id_bytes);
    if (st != CCQ_OK) return st;
    if (!(a.p.clip_low >= 0.f) || !(a.p.clip_high >= 0.f))
        return op_fail(CCQ_ERR_INVALID_ARG, "clip_low and clip_high must be >= 0");
    if ((st = op_pointer("loss", loss, 4)) != CCQ_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (n == 0) return op_cuda(cudaMemsetAsync(loss, 0, sizeof(float), s), "zero loss");
    if ((st = check_logits("logits", logits, logits_stride, dtype, n, vocab)) != CCQ_OK) return st;
    if (dlogits && (st = check_logits("dlogits", dlogits, dlogits_stride, dtype, n, vocab)) != CCQ_OK) return st;
    if (dlogits == logits && dlogits_stride != logits_stride && n > 1)
        return op_fail(CCQ_ERR_INVALID_ARG, "dlogits over the logits needs their row stride");
    if ((st = op_pointer("actions", actions, id_bytes)) != CCQ_OK) return st;
    if ((st = op_pointer("old_logp", old_logp, 4)) != CCQ_OK) return st;
    if ((st = op_pointer("advantages", advantages, 4)) != CCQ_OK) return st;
    if (ref_logp && (st = op_pointer("ref_logp", ref_logp, 4)) != CCQ_OK) return st;
    if (weights && (st = op_pointer("weights", weights, 4)) != CCQ_OK) return st;
    if (logp && (st = op_pointer("logp", logp, 4)) != CCQ_OK) return st;
    size_t need = 0;
    ccq_policy_loss_workspace_size(n, &need);
    if ((st = op_pointer("workspace", workspace, 16)) != CCQ_OK) return st;
    if (workspace_bytes < need)
        return op_fail(CCQ_ERR_INVALID_ARG, "workspace of %zu bytes, needs %zu", workspace_bytes, need);
    a.logits = logits; a.logits_stride = logits_stride; a.actions = actions; a.id_bytes = id_bytes;
    a.n = n; a.vocab = vocab;
    a.old_logp = old_logp; a.ref_logp = ref_logp; a.advantages = advantages; a.weights = weights;
    a.scale = kLog2e / a.p.temperature;
    a.logp = logp; a.row_loss = static_cast<float *>(workspace);
    a.dlogits = dlogits; a.dlogits_stride = dlogits_stride;
    a.status = device_status_word();
    cudaError_t e = launch_policy(a, dtype, s);
    if (e != cudaSuccess) return op_cuda(e, "policy loss launch");
    e = launch_after(policy_loss_kernel, 1, kLossThreads, 0, s, static_cast<const float *>(a.row_loss), n, loss);
    return op_cuda(e, "policy loss sum launch");
}

ccq_status ccq_token_logp(const void *logits, ccq_dtype dtype, int64_t logits_stride, const void *actions, int id_bytes,
                          int64_t n, int vocab, float temperature, float *logp, void *stream) {
    ccq_status st = check_policy(n, vocab, dtype, temperature, id_bytes);
    if (st != CCQ_OK) return st;
    if (n == 0) return CCQ_OK;
    if ((st = check_logits("logits", logits, logits_stride, dtype, n, vocab)) != CCQ_OK) return st;
    if ((st = op_pointer("actions", actions, id_bytes)) != CCQ_OK) return st;
    if ((st = op_pointer("logp", logp, 4)) != CCQ_OK) return st;
    PolicyArgs a = {};
    a.logits = logits; a.logits_stride = logits_stride; a.actions = actions; a.id_bytes = id_bytes;
    a.n = n; a.vocab = vocab;
    a.p.temperature = temperature;
    a.scale = kLog2e / temperature;
    a.logp = logp;
    a.score = 1;
    a.status = device_status_word();
    return op_cuda(launch_policy(a, dtype, static_cast<cudaStream_t>(stream)), "token log-probability launch");
}

}  // extern "C"
